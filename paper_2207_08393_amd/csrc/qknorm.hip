// Norm (root mean square) of every head of the queries and keys and rotation of its first values by the token's position, in one pass,
// and its gradients (gfx950).
//
// A row is one head of one token: a team of 2^k lanes holds it in registers, in pairs that turn together, so that the rotation needs no
// exchange between lanes and the norm one sum over the team.  A wave works on the rows of one token, or of several where one has few: the
// angles are formed once, a lane an angle, and handed round in LDS.  An angle is pos * freq in 64 bits, taken to turns and to its
// fraction there, which float32 would lose from a few thousand positions on; the float32 rest goes to sincospi.
// Backward: the row's x and g in registers, nothing stored by the forward pass; gradients of gamma are summed by lane over all rows of a
// wave, a workgroup writes one partial sum per column and a second launch adds them up in a fixed order.
//
// What bounds it: HBM, two passes over the arrays forward and three backward.  20 x 192 x 160 pixels, 4 + 4 heads of 16, bfloat16: 73 us for 157 MB
// each way, 4.3 TB/s, half of the vector instructions' time (16 lanes that turn one token hold four rows; an angle in 64 bits is worked out
// once for them).  Gradients of 16384 tokens, 16 + 4 heads of 128: 63 us for 252 MB, 4.0 TB/s, and 4.8 us for the sums;
// of 3 x 1001 tokens, 6 + 6 heads of 40, float32: 12 us, latency of the angles and then of the first row, and 3.8.  One token of 64
// sequences: 4.9 us, latency of a launch, of the angle and of one row.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "layer_common.h"
#include "layer_ops.h"

namespace gleam {
namespace {

constexpr int kQkThreads = 256, kQkWaves = kQkThreads / 64;
constexpr long long kQkGroupsFwd = 8192, kQkGroupsBwd = 1024;

struct QkTensor {
    const void *x, *g;        // rows in, and the gradients of their results
    void* out;
    gleam_seq_strides sx, so; // of x, and of the results; out has those of so forward, of sx backward
    const float* gamma;
    unsigned heads, rows;     // rows of a token: P heads
    unsigned magic, shift;    // r / heads = r * magic >> (32 + shift) of r < 2^31; magic 0: one head
    int steps;                // of a wave through a token's rows
};
struct QkArgs {
    QkTensor t[2];            // queries, keys
    const float* freq;
    const int *positions, *lengths;
    float* part;              // backward: [workgroup][2][d] partial sums, or null
    long long T, tokens, units;   // units of work: `per` steps through the rows of 2^tokens_log tokens
    int per, parts;           // units of these tokens
    int few;                  // units and tokens are numbers of 32 bits
    int d, rot, each, lanes_log, tokens_log;
    float eps;
};

// The sum over a team of 2^log lanes, in all of them.
__device__ __forceinline__ float team_sum(float v, int log) {
    if (log > 0) v += dpp<0xB1>(v);    // lane i and i ^ 1
    if (log > 1) v += dpp<0x4E>(v);    // i ^ 2
    if (log > 2) v += dpp<0x141>(v);   // 7 - i of eight lanes, which are equal in fours
    if (log > 3) v += dpp<0x140>(v);   // 15 - i of sixteen
    if (log > 4) v = sum_of_pair(__builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false));
    if (log > 5) v = sum_of_pair(__builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false));
    return v;
}

// W pairs of a row: two vectors of W values.  Halves: the pairs' first values and their second ones; neighbours: 2 W values in a row.
// Behind the rotated part both are 2 W values in a row.  W = 1 takes any width: the last pair of an odd one has no second value.
template <class T, int W>
struct Place {
    int e0, e1;
    bool on, two;     // there are pairs; the second vector is there
    __device__ __forceinline__ void set(int pair, bool halves, int d, int rot) {
        on = 2 * pair < d;
        const bool turned = 2 * pair < rot;
        e0 = halves ? (turned ? pair : 2 * pair) : 2 * pair;
        e1 = halves && turned ? pair + rot / 2 : e0 + W;
        two = on && e1 < d;
        if (!on) e0 = 0;
        if (!two) e1 = e0;
    }
    __device__ __forceinline__ void store(T* row, const float* v) const {
        if (on) store_vec<T, W>(row + e0, v);
        if (two) store_vec<T, W>(row + e1, v + W);
    }
    __device__ __forceinline__ void load_gamma(const float* p, float* v) const {
#pragma unroll
        for (int i = 0; i < W; ++i) {
            v[i] = p ? p[e0 + i] : 1.f;
            v[W + i] = p ? p[e1 + i] : 1.f;
        }
    }
};

template <int W, bool HALVES>
__device__ __forceinline__ void turn(float* v, const float* c, const float* s, float sign) {
#pragma unroll
    for (int i = 0; i < W; ++i) {
        float &a = v[HALVES ? i : 2 * i], &b = v[HALVES ? W + i : 2 * i + 1];
        const float x = a, y = b, si = sign * s[i];
        a = x * c[i] - y * si;
        b = y * c[i] + x * si;
    }
}

// A lane's part of a row on its way.
template <class T, int W, int NV>
struct Row {
    Raw<T, W> v[NV][2];
    __device__ __forceinline__ void load(const T* row, const Place<T, W> (&at)[NV]) {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            v[j][0].load(row + at[j].e0);
            v[j][1].load(row + at[j].e1);
        }
    }
    __device__ __forceinline__ void get(const Place<T, W> (&at)[NV], float (&to)[NV][2 * W]) const {
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < W; ++i) {
                to[j][i] = at[j].on ? v[j][0].get(i) : 0.f;
                to[j][W + i] = at[j].two ? v[j][1].get(i) : 0.f;
            }
    }
};

template <class T, int W, bool HALVES, bool BWD>
__global__ __launch_bounds__(kQkThreads) void qknorm_kernel(QkArgs a) {
    constexpr int NV = W == 1 ? 2 : 1, E = 2 * W;   // vectors of pairs of a lane, values of one
    constexpr int kAngles = 64 * W * NV;            // of a wave, at most
    __shared__ __attribute__((aligned(16))) float turns[kQkWaves][2][kAngles];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), L = 1 << a.lanes_log, half = a.rot / 2;
    const int sub = lane & (L - 1), team = lane >> a.lanes_log;
    const int rows_log = 6 - a.lanes_log - a.tokens_log;        // of the teams of a token
    const int my_token = team >> rows_log, my_row = team & ((1 << rows_log) - 1);
    Place<T, W> at[NV];
    float sums[2][NV][E];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        at[j].set((sub + j * L) * W, HALVES, a.d, a.rot);
#pragma unroll
        for (int i = 0; i < E; ++i) sums[0][j][i] = sums[1][j][i] = 0.f;
    }
    const float inv_d = 1.f / (float)a.d;
    for (long long unit = (long long)blockIdx.x * kQkWaves + wave; unit < a.units; unit += (long long)gridDim.x * kQkWaves) {
        long long group = a.few ? (long long)((unsigned)unit / (unsigned)a.parts) : unit / a.parts;
        const int step0 = (int)(unit - group * a.parts) * a.per;
        const long long first = group << a.tokens_log, b0 = a.few ? (long long)((unsigned)first / (unsigned)a.T) : first / a.T;
        const unsigned t_first = (unsigned)(first - b0 * a.T);
        // sequence and place of the token that is `ahead` of the first
        auto find = [&](unsigned ahead, long long& b, unsigned& t) {
            const unsigned over = a.tokens_log ? (t_first + ahead) / (unsigned)a.T : 0;
            b = b0 + over;
            t = t_first + ahead - over * (unsigned)a.T;
        };
        const int n_angles = half << a.tokens_log;
        for (int i = lane; i < n_angles; i += 64) {
            const unsigned ahead = a.tokens_log ? (unsigned)i / (unsigned)half : 0, pair = i - ahead * half;
            float sn = 0.f, cs = 1.f;
            if (first + ahead < a.tokens) {
                long long b;
                unsigned t;
                find(ahead, b, t);
                const double pos = !a.positions ? (double)t : a.each ? (double)a.positions[first + ahead] : (double)a.positions[b] + (double)t;
                double part = pos * (double)a.freq[pair] * 0.15915494309189533577;   // 1 / (2 pi)
                part -= rint(part);
                sincospif((float)(2.0 * part), &sn, &cs);
            }
            turns[wave][0][i] = cs;
            turns[wave][1][i] = sn;
        }
        wave_sync();
        float c[NV][W], s[NV][W];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int pair = (sub + j * L) * W, from = my_token * half + pair;
            const bool turned = 2 * pair < a.rot;
#pragma unroll
            for (int i = 0; i < W; ++i) {
                c[j][i] = turned ? turns[wave][0][from + i] : 1.f;
                s[j][i] = turned ? turns[wave][1][from + i] : 0.f;
            }
        }
        wave_sync();
        long long b;
        unsigned t;
        find((unsigned)my_token, b, t);
        const bool exists = first + my_token < a.tokens, there = exists && (!a.lengths || (int)t < a.lengths[b]);
        const bool any = __ballot(there) != 0;
        if (!exists) b = b0, t = t_first;   // work on the first token, and nothing is written
        auto tensor = [&](auto which) {
            constexpr int k = decltype(which)::value;
            const QkTensor& q = a.t[k];
            const int from = step0 - (k ? a.t[0].steps : 0), lo = from < 0 ? 0 : from, hi = from + a.per < q.steps ? from + a.per : q.steps;
            if (lo >= hi) return;
            float gamma[NV][E];
#pragma unroll
            for (int j = 0; j < NV; ++j) at[j].load_gamma(q.gamma, gamma[j]);
            const long long base_x = b * q.sx.b + t * q.sx.t, base_o = b * q.so.b + t * q.so.t;
            // offsets of the row of a step; a lane without one works on the token's last row and writes nothing
            auto place = [&](int step, long long& off_x, long long& off_o) {
                const unsigned row = ((unsigned)step << rows_log) + my_row, r = row < q.rows ? row : q.rows - 1;
                const unsigned p = q.magic ? __umulhi(r, q.magic) >> q.shift : r;
                const long long h = r - p * q.heads;
                off_x = base_x + p * q.sx.p + h * q.sx.h;
                off_o = base_o + p * q.so.p + h * q.so.h;
                return row < q.rows && exists;
            };
            if (!any) {   // tokens behind their sequences' ends
                for (int step = lo; step < hi; ++step) {
                    long long off_x, off_o;
                    const bool mine = place(step, off_x, off_o);
                    const float none[E] = {};
#pragma unroll
                    for (int j = 0; j < NV; ++j)
                        if (mine) at[j].store((T*)q.out + (BWD ? off_x : off_o), none);
                }
                return;
            }
            Row<T, W, NV> next_x, next_g;
            long long next_at_x, next_at_o;
            bool next_mine = place(lo, next_at_x, next_at_o);
            next_x.load((const T*)q.x + next_at_x, at);
            if (BWD) next_g.load((const T*)q.g + next_at_o, at);
            for (int step = lo; step < hi; ++step) {
                float v[NV][E], g[NV][E];
                next_x.get(at, v);
                if (BWD) next_g.get(at, g);
                const bool mine = next_mine;
                T* out = (T*)q.out + (BWD ? next_at_x : next_at_o);
                if (step + 1 < hi) {
                    next_mine = place(step + 1, next_at_x, next_at_o);
                    next_x.load((const T*)q.x + next_at_x, at);
                    if (BWD) next_g.load((const T*)q.g + next_at_o, at);
                }
                float ss = 0.f, dot = 0.f;
#pragma unroll
                for (int j = 0; j < NV; ++j) {
                    if (BWD) turn<W, HALVES>(g[j], c[j], s[j], -1.f);
#pragma unroll
                    for (int i = 0; i < E; ++i) {
                        ss += v[j][i] * v[j][i];
                        if (BWD) dot += g[j][i] * gamma[j][i] * v[j][i];
                    }
                }
                const float r = __builtin_amdgcn_rsqf(team_sum(ss, a.lanes_log) * inv_d + a.eps);
                if (!BWD) {
#pragma unroll
                    for (int j = 0; j < NV; ++j) {
#pragma unroll
                        for (int i = 0; i < E; ++i) v[j][i] *= r * gamma[j][i];
                        turn<W, HALVES>(v[j], c[j], s[j], 1.f);
#pragma unroll
                        for (int i = 0; i < E; ++i) v[j][i] = there ? v[j][i] : 0.f;
                        if (mine) at[j].store(out, v[j]);
                    }
                } else {
                    const float along = r * r * (team_sum(dot, a.lanes_log) * inv_d);
#pragma unroll
                    for (int j = 0; j < NV; ++j) {
#pragma unroll
                        for (int i = 0; i < E; ++i) {
                            sums[k][j][i] += mine && there ? g[j][i] * (v[j][i] * r) : 0.f;
                            g[j][i] = there ? r * (g[j][i] * gamma[j][i] - v[j][i] * along) : 0.f;
                        }
                        if (mine) at[j].store(out, g[j]);
                    }
                }
            }
        };
        tensor(std::integral_constant<int, 0>{});
        tensor(std::integral_constant<int, 1>{});
    }
    if constexpr (BWD) {
        if (!a.part) return;
        float (*red)[2][256] = (float (*)[2][256])turns;   // [wave][tensor][column]
        static_assert(sizeof(turns) >= kQkWaves * 2 * 256 * sizeof(float) || W < 4, "the sums meet in the same memory");
        __shared__ float more[W < 4 ? kQkWaves : 1][2][256];
        if (W < 4) red = more;
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    float v = sums[k][j][i];
                    for (int o = L; o < 64; o *= 2) v += __shfl_xor(v, o);
                    if (team == 0 && at[j].on && (i < W || at[j].two)) red[wave][k][i < W ? at[j].e0 + i : at[j].e1 + i - W] = v;
                }
        __syncthreads();
        for (int e = threadIdx.x; e < 2 * a.d; e += kQkThreads) {
            const int k = e >= a.d, col = e - k * a.d;
            float v = red[0][k][col];
#pragma unroll
            for (int w = 1; w < kQkWaves; ++w) v += red[w][k][col];
            a.part[(long long)blockIdx.x * 2 * a.d + e] = v;
        }
    }
}

// Sums of the partial sums: 16 columns a workgroup, 64 lanes of each.
__global__ __launch_bounds__(1024) void qknorm_sums_kernel(const float* part, int groups, int d, float* g_q, float* g_k) {
    __shared__ float red[64][17];
    const int col = threadIdx.x & 15, slice = threadIdx.x >> 4, e = blockIdx.x * 16 + col;
    float v = 0.f;
    if (e < 2 * d)
#pragma unroll 4
        for (int g = slice; g < groups; g += 64) v += part[(long long)g * 2 * d + e];
    red[slice][col] = v;
    __syncthreads();
    if (slice >= 4) return;
    for (int i = slice + 4; i < 64; i += 4) v += red[i][col];
    red[slice][col] = v;
    wave_sync();
    if (slice || e >= 2 * d) return;
    v = (red[0][col] + red[1][col]) + (red[2][col] + red[3][col]);
    float* out = e < d ? g_q : g_k;
    if (out) out[e < d ? e : e - d] = v;
}

// Pairs of a lane's vector: up to four, as many as divide both the rotated part and the rest.  (Eight, 16 bytes of bfloat16, took 74 us backward at
// 16384 tokens where four take 66, with twice the registers, and as long forward.)
int vector_of(const gleam_qknorm_desc& d) {
    int w = 4;
    while (w > 1 && (d.rot / 2 % w || (d.d - d.rot) % (2 * w))) w /= 2;
    return w;
}

struct QkPlan {
    int w, lanes_log, tokens_log, steps[2], per, parts;
    long long units, groups;
};
QkPlan plan_of(const gleam_qknorm_desc& d, bool backward) {
    QkPlan p;
    p.w = vector_of(d);
    const int nv = p.w == 1 ? 2 : 1, lanes = ((d.d + 1) / 2 + nv * p.w - 1) / (nv * p.w);
    for (p.lanes_log = 0; 1 << p.lanes_log < lanes;) ++p.lanes_log;
    const long long tokens = d.B * d.T, rows[2] = {d.P * d.q_heads, d.P * d.k_heads};
    // Teams of a token: as many as leave the fewest without a row, the most of these; with fewer, a wave takes several tokens.
    long long best = -1;
    for (int log = 0; log <= 6 - p.lanes_log; ++log) {
        const long long teams = 1LL << log, taken = ((rows[0] + teams - 1) / teams + (rows[1] + teams - 1) / teams) * teams;
        if (best < 0 || taken <= best) {
            best = taken;
            p.tokens_log = 6 - p.lanes_log - log;
            p.steps[0] = (int)((rows[0] + teams - 1) / teams);
            p.steps[1] = (int)((rows[1] + teams - 1) / teams);
        }
    }
    while (p.tokens_log > 0 && tokens < 1LL << p.tokens_log) {   // no more tokens than there are
        --p.tokens_log;
        const long long teams = 1LL << (6 - p.lanes_log - p.tokens_log);
        for (int k = 0; k < 2; ++k) p.steps[k] = (int)((rows[k] + teams - 1) / teams);
    }
    const long long steps = (long long)p.steps[0] + p.steps[1], groups = (tokens + (1LL << p.tokens_log) - 1) >> p.tokens_log;
    // up to 16 steps of a wave share the angles, fewer where waves would be missing (backward, those of the largest launch are there at once)
    const long long waves = backward ? kQkGroupsBwd * kQkWaves : 8192;
    long long per = (steps * groups + waves - 1) / waves;
    per = per > 16 ? 16 : per < steps ? per : steps;
    p.parts = (int)((steps + per - 1) / per);
    p.per = (int)((steps + p.parts - 1) / p.parts);
    p.units = groups * p.parts;
    const long long most = backward ? kQkGroupsBwd : kQkGroupsFwd, all = (p.units + kQkWaves - 1) / kQkWaves;
    p.groups = all < most ? all : most;
    return p;
}

template <class T, int W, bool BWD>
void launch_pairs(const QkArgs& a, const QkPlan& p, bool halves, hipStream_t st) {
    const dim3 grid((unsigned)p.groups), block(kQkThreads);
    if (halves) hipLaunchKernelGGL((qknorm_kernel<T, W, true, BWD>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((qknorm_kernel<T, W, false, BWD>), grid, block, 0, st, a);
}
template <class T, bool BWD>
void launch(const QkArgs& a, const QkPlan& p, bool halves, hipStream_t st) {
    if (p.w == 1) launch_pairs<T, 1, BWD>(a, p, halves, st);
    else if (p.w == 2) launch_pairs<T, 2, BWD>(a, p, halves, st);
    else launch_pairs<T, 4, BWD>(a, p, halves, st);
}

QkArgs args_of(const gleam_qknorm_desc& d, const QkPlan& p, const void* q, const void* k, const float* gamma_q, const float* gamma_k,
               const float* freq, const int* positions, const int* lengths) {
    QkArgs a{};
    a.t[0].x = q;
    a.t[1].x = k;
    a.t[0].sx = d.q;
    a.t[1].sx = d.k;
    a.t[0].so = d.q_out;
    a.t[1].so = d.k_out;
    a.t[0].gamma = gamma_q;
    a.t[1].gamma = d.k_heads ? gamma_k : nullptr;
    a.freq = freq;
    a.positions = positions;
    a.lengths = lengths;
    for (int k = 0; k < 2; ++k) {
        QkTensor& t = a.t[k];
        t.heads = (unsigned)(k ? d.k_heads : d.q_heads);
        t.rows = (unsigned)(d.P * t.heads);
        t.steps = p.steps[k];
        if (t.heads > 1) {   // n / h = n ceil(2^(31 + l) / h) >> (31 + l) of n < 2^31, 2^(l - 1) < h <= 2^l
            unsigned l = 1;
            while (1ull << l < t.heads) ++l;
            t.magic = (unsigned)(((1ull << (31 + l)) + t.heads - 1) / t.heads);
            t.shift = l - 1;
        }
    }
    a.T = d.T;
    a.tokens = d.B * d.T;
    a.units = p.units;
    a.per = p.per;
    a.parts = p.parts;
    a.few = p.units < 0x7fffffff && a.tokens < 0x7fffffff;
    a.d = d.d;
    a.rot = d.rot;
    a.each = d.each;
    a.lanes_log = p.lanes_log;
    a.tokens_log = p.tokens_log;
    a.eps = d.eps;
    return a;
}

}  // namespace

hipError_t qknorm_forward(const gleam_qknorm_desc& d, const void* q, const void* k, const float* gamma_q, const float* gamma_k,
                          const float* freq, const int* positions, const int* lengths, void* q_out, void* k_out, hipStream_t st) {
    const QkPlan p = plan_of(d, false);
    QkArgs a = args_of(d, p, q, k, gamma_q, gamma_k, freq, positions, lengths);
    a.t[0].out = q_out;
    a.t[1].out = k_out;
    const double size = (double)d.B * d.T * d.P * (d.q_heads + d.k_heads) * d.d;
    KernelScope ks("qknorm_fwd", 8.0 * size, 2.0 * (d.dtype ? 2 : 4) * size, st);
    if (d.dtype) launch<unsigned short, false>(a, p, !d.pairs, st);
    else launch<float, false>(a, p, !d.pairs, st);
    return hipGetLastError();
}

size_t qknorm_ws_bytes(const gleam_qknorm_desc& d) { return ((size_t)plan_of(d, true).groups * 2 * d.d * sizeof(float) + 255) / 256 * 256; }

hipError_t qknorm_backward(const gleam_qknorm_desc& d, const void* q, const void* k, const float* gamma_q, const float* gamma_k,
                           const float* freq, const int* positions, const int* lengths, const void* g_q_out, const void* g_k_out, void* g_q,
                           void* g_k, float* g_gamma_q, float* g_gamma_k, void* ws, hipStream_t st) {
    const QkPlan p = plan_of(d, true);
    QkArgs a = args_of(d, p, q, k, gamma_q, gamma_k, freq, positions, lengths);
    a.t[0].g = g_q_out;
    a.t[1].g = g_k_out;
    a.t[0].out = g_q;
    a.t[1].out = g_k;
    a.part = g_gamma_q || g_gamma_k ? (float*)ws : nullptr;
    {
        const double size = (double)d.B * d.T * d.P * (d.q_heads + d.k_heads) * d.d;
        KernelScope ks("qknorm_bwd", 16.0 * size, 3.0 * (d.dtype ? 2 : 4) * size, st);
        if (d.dtype) launch<unsigned short, true>(a, p, !d.pairs, st);
        else launch<float, true>(a, p, !d.pairs, st);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || !a.part) return e;
    KernelScope ks("qknorm_sums", 0.0, 8.0 * p.groups * d.d, st);
    hipLaunchKernelGGL(qknorm_sums_kernel, dim3((unsigned)((2 * d.d + 15) / 16)), dim3(1024), 0, st, a.part, (int)p.groups, d.d, g_gamma_q, g_gamma_k);
    return hipGetLastError();
}

}  // namespace gleam
