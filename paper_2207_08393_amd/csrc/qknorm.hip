// Norm (root mean square) of every head of the queries and keys and rotation of its first values by the token's position, in one pass,
// and its gradients (gfx950).
//
// A row is one head of one token: a team of 2^k lanes holds it in registers, in pairs that turn together, so that the rotation needs no
// exchange between lanes and the norm one sum over the team.  A wave works on one token's rows at a time (all heads of q and k, all
// pixels, or a part of them): the angles are formed once and serve every row.  An angle is pos * freq in 64 bits, taken to turns and
// to its fraction there, which float32 would lose from a few thousand positions on; the float32 rest goes to sincospi.
// Backward: the row's x and g in registers, nothing stored by the forward pass; gradients of gamma are summed by lane over all rows of a
// wave, a workgroup writes one partial sum per column and a second launch adds them up in a fixed order.
#include <hip/hip_runtime.h>

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
};
struct QkArgs {
    QkTensor t[2];            // queries, keys
    const float* freq;
    const int *positions, *lengths;
    float* part;              // backward: [workgroup][2][d] partial sums, or null
    long long T, units;       // units of work: rows_unit rows of a token
    unsigned rows, rows_unit, parts;   // rows of a token, of a unit, units of a token
    int d, rot, H, Hq, each, lanes_log;
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
    __device__ __forceinline__ void load(const T* row, float* v) const {
        load_vec<T, W>(row + e0, v);
        load_vec<T, W>(row + e1, v + W);
#pragma unroll
        for (int i = 0; i < W; ++i) {
            v[i] = on ? v[i] : 0.f;
            v[W + i] = two ? v[W + i] : 0.f;
        }
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

template <class T, int W, bool HALVES, bool BWD>
__global__ __launch_bounds__(kQkThreads) void qknorm_kernel(QkArgs a) {
    constexpr int NV = W == 1 ? 2 : 1, E = 2 * W;   // vectors of pairs of a lane, values of one
    __shared__ float red[BWD ? kQkWaves : 1][2][256];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, L = 1 << a.lanes_log;
    const int sub = lane & (L - 1), first_row = lane >> a.lanes_log, rows_step = 64 >> a.lanes_log;
    Place<T, W> at[NV];
    float gamma[2][NV][E], sums[2][NV][E];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        at[j].set((sub + j * L) * W, HALVES, a.d, a.rot);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            at[j].load_gamma(a.t[k].gamma, gamma[k][j]);
#pragma unroll
            for (int i = 0; i < E; ++i) sums[k][j][i] = 0.f;
        }
    }
    const float inv_d = 1.f / (float)a.d;
    for (long long unit = (long long)blockIdx.x * kQkWaves + wave; unit < a.units; unit += (long long)gridDim.x * kQkWaves) {
        const long long token = unit / a.parts, b = token / a.T, t = token - b * a.T;
        const unsigned row0 = (unsigned)(unit - token * a.parts) * a.rows_unit;
        const unsigned row1 = row0 + a.rows_unit < a.rows ? row0 + a.rows_unit : a.rows;
        const bool there = !a.lengths || t < a.lengths[b];
        float c[NV][W], s[NV][W];
        if (there && a.rot) {
            const double pos = !a.positions ? (double)t : a.each ? (double)a.positions[token] : (double)a.positions[b] + (double)t;
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int i = 0; i < W; ++i) {
                    const int pair = (sub + j * L) * W + i;
                    c[j][i] = 1.f, s[j][i] = 0.f;
                    if (2 * pair < a.rot) {
                        double turns = pos * (double)a.freq[pair] * 0.15915494309189533577;   // 1 / (2 pi)
                        turns -= rint(turns);
                        sincospif((float)(2.0 * turns), &s[j][i], &c[j][i]);
                    }
                }
        } else {
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int i = 0; i < W; ++i) c[j][i] = 1.f, s[j][i] = 0.f;
        }
        for (unsigned first = row0; first < row1; first += rows_step) {
            const bool mine = first + first_row < row1;
            const unsigned row = mine ? first + first_row : row1 - 1;   // lanes without a row work on the last one and write nothing
            const unsigned p = row / (unsigned)a.H, hh = row - p * (unsigned)a.H;
            const int k = hh < (unsigned)a.Hq ? 0 : 1;
            const QkTensor& q = a.t[0];
            const QkTensor& w = a.t[1];
            const long long h = k ? hh - (unsigned)a.Hq : hh;
            const gleam_seq_strides sx = k ? w.sx : q.sx, so = k ? w.so : q.so;
            const long long off_x = b * sx.b + t * sx.t + p * sx.p + h * sx.h, off_o = b * so.b + t * so.t + p * so.p + h * so.h;
            T* out = (T*)(k ? w.out : q.out) + (BWD ? off_x : off_o);
            float v[NV][E], g[NV][E];
            if (!there) {
#pragma unroll
                for (int j = 0; j < NV; ++j) {
#pragma unroll
                    for (int i = 0; i < E; ++i) v[j][i] = 0.f;
                    if (mine) at[j].store(out, v[j]);
                }
                continue;
            }
            const T* x = (const T*)(k ? w.x : q.x) + off_x;
            const T* gr = BWD ? (const T*)(k ? w.g : q.g) + off_o : nullptr;
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                at[j].load(x, v[j]);
                if (BWD) at[j].load(gr, g[j]);
            }
            float ss = 0.f, dot = 0.f;
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                if (BWD) turn<W, HALVES>(g[j], c[j], s[j], -1.f);
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    ss += v[j][i] * v[j][i];
                    if (BWD) dot += g[j][i] * (k ? gamma[1][j][i] : gamma[0][j][i]) * v[j][i];
                }
            }
            const float r = 1.f / sqrtf(team_sum(ss, a.lanes_log) * inv_d + a.eps);
            if (!BWD) {
#pragma unroll
                for (int j = 0; j < NV; ++j) {
#pragma unroll
                    for (int i = 0; i < E; ++i) v[j][i] *= r * (k ? gamma[1][j][i] : gamma[0][j][i]);
                    turn<W, HALVES>(v[j], c[j], s[j], 1.f);
                    if (mine) at[j].store(out, v[j]);
                }
            } else {
                const float along = r * r * (team_sum(dot, a.lanes_log) * inv_d);
#pragma unroll
                for (int j = 0; j < NV; ++j) {
#pragma unroll
                    for (int i = 0; i < E; ++i) {
                        const float own = mine ? g[j][i] * (v[j][i] * r) : 0.f;
                        sums[0][j][i] += k ? 0.f : own;
                        sums[1][j][i] += k ? own : 0.f;
                        g[j][i] = r * (g[j][i] * (k ? gamma[1][j][i] : gamma[0][j][i]) - v[j][i] * along);
                    }
                    if (mine) at[j].store(out, g[j]);
                }
            }
        }
    }
    if constexpr (BWD) {
        if (!a.part) return;
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    float v = sums[k][j][i];
                    for (int o = L; o < 64; o *= 2) v += __shfl_xor(v, o);
                    if (first_row == 0 && at[j].on && (i < W || at[j].two)) red[wave][k][i < W ? at[j].e0 + i : at[j].e1 + i - W] = v;
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

// Sums of the partial sums: 16 columns a workgroup, 16 lanes of each.
__global__ __launch_bounds__(256) void qknorm_sums_kernel(const float* part, int groups, int d, float* g_q, float* g_k) {
    __shared__ float red[16][17];
    const int col = threadIdx.x & 15, slice = threadIdx.x >> 4, e = blockIdx.x * 16 + col;
    float v = 0.f;
    if (e < 2 * d)
        for (int g = slice; g < groups; g += 16) v += part[(long long)g * 2 * d + e];
    red[slice][col] = v;
    __syncthreads();
    if (slice || e >= 2 * d) return;
    for (int i = 1; i < 16; ++i) v += red[i][col];
    float* out = e < d ? g_q : g_k;
    if (out) out[e < d ? e : e - d] = v;
}

// Pairs of a lane's vector: as many as 16 bytes take and divide both the rotated part and the rest.
int vector_of(const gleam_qknorm_desc& d) {
    int w = d.dtype ? 8 : 4;
    while (w > 1 && (d.rot / 2 % w || (d.d - d.rot) % (2 * w))) w /= 2;
    return w;
}

struct QkPlan {
    int w, lanes_log;
    unsigned rows, rows_unit, parts;
    long long units, groups;
};
QkPlan plan_of(const gleam_qknorm_desc& d, bool backward) {
    QkPlan p;
    p.w = vector_of(d);
    const int nv = p.w == 1 ? 2 : 1, lanes = ((d.d + 1) / 2 + nv * p.w - 1) / (nv * p.w);
    for (p.lanes_log = 0; 1 << p.lanes_log < lanes;) ++p.lanes_log;
    p.rows = (unsigned)(d.P * (d.q_heads + d.k_heads));
    const long long step = 64 >> p.lanes_log, steps = (p.rows + step - 1) / step, tokens = d.B * d.T;
    // up to 16 steps of a wave share the angles, fewer where waves would be missing
    long long per = steps * tokens / 16384;
    per = per < 1 ? 1 : per > 16 ? 16 : per;
    per = per < steps ? per : steps;
    p.rows_unit = (unsigned)(per * step);
    p.parts = (unsigned)((steps + per - 1) / per);
    p.units = tokens * p.parts;
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
    else if (p.w == 4) launch_pairs<T, 4, BWD>(a, p, halves, st);
    else if constexpr (sizeof(T) == 2) launch_pairs<T, 8, BWD>(a, p, halves, st);
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
    a.T = d.T;
    a.units = p.units;
    a.rows = p.rows;
    a.rows_unit = p.rows_unit;
    a.parts = p.parts;
    a.d = d.d;
    a.rot = d.rot;
    a.H = d.q_heads + d.k_heads;
    a.Hq = d.q_heads;
    a.each = d.each;
    a.lanes_log = p.lanes_log;
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
    const double size = (double)d.B * d.T * p.rows * d.d;
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
        const double size = (double)d.B * d.T * p.rows * d.d;
        KernelScope ks("qknorm_bwd", 16.0 * size, 3.0 * (d.dtype ? 2 : 4) * size, st);
        if (d.dtype) launch<unsigned short, true>(a, p, !d.pairs, st);
        else launch<float, true>(a, p, !d.pairs, st);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || !a.part) return e;
    KernelScope ks("qknorm_sums", 0.0, 8.0 * p.groups * d.d, st);
    hipLaunchKernelGGL(qknorm_sums_kernel, dim3((unsigned)((2 * d.d + 15) / 16)), dim3(256), 0, st, a.part, (int)p.groups, d.d, g_gamma_q, g_gamma_k);
    return hipGetLastError();
}

}  // namespace gleam
