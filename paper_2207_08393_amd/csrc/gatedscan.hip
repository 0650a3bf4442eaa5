// Gated scan along the tokens and its gradients (gfx950):
//     s = sigmoid(r),  a = exp(-c s),  h <- a h + sqrt(1 - a^2) sigmoid(i) x      c = kappa softplus(lambda), channel by channel
//
// Numbers.  Where a > 2^-0.36, what is kept of it is -d, d = 1 - a = -expm1(-c s), good to float32 however near to 1 a is: h <- h - (d h - b)
// forgets at the right rate over thousands of tokens, where a rounded to float32 would be off by 2^-25 / d of it.  Smaller ones are kept as they
// are, so that little is left of a state to its last bits too; the sign tells which.  sqrt(1 - a^2) = sqrt(d (2 - d)).  Over a
// stretch of tokens, a state passes as exp(-sum c s) h + (what the stretch adds), with the sum in the exponent.
//
// Gradients.  With E_t = a_t G_t what token t hands back to the one before it and G_t = g_t + E_(t+1):
//     dL/d log a = G (a h_(t-1) - (a^2 / m) u),   m = sqrt(1 - a^2), u = sigmoid(i) x
// and log a = -c s, so W = (dL/d log a) log a = G a (a u (c s / m) - h_(t-1) c s) has no pole where the gate closes (m -> 0 as sqrt(2 c s)):
// g_r = W (1 - s), and g_lambda = sigmoid(lambda) / softplus(lambda) sum W.  h_(t-1) is formed again from x, r and i in float32.
//
// Layout.  A lane owns V neighbouring channels of a pixel, a wave 64 such columns.  Forward, a wave walks along the tokens with its state in
// registers, four tokens ahead of itself with its loads: all of a sequence where there are columns enough, or in pieces of 16 tokens and more,
// which takes two more launches: what every piece does to a state, and the carries at the pieces' starts from that, in order.  Backward, a
// wave holds up to 8 tokens in registers and the waves of a workgroup stand one behind the other along them, with their carries in LDS,
// since gates and states are needed again on the way back; sequences longer than a workgroup's tokens take the same two launches.
//
// What bounds it: vector instructions, some 60 issue slots a token and channel forward (three exponentials, two quotients and a root count four
// each).  20 x 192 x 160 pixels, 64 channels, bfloat16: 67 us (float32 121, its bytes' time), 4.7 TB/s and 96 % of the vector
// instructions' time, 2.4 ms as separate products; 16384 tokens x 1024 channels: 28 + 8 + 29 us, 76 and 85 % in the two passes (26 us are its bytes, so that a scan that reads
// them once would still take some 40).  Gradients of 4 x 2048 x 1024: 19 + 6 + 38 + 5 us, 3.1 TB/s in the long pass (23 us of bytes in all);
// 3 x 1001 x 301 in float32: 7 + 6 + 10 + 4, latency of four launches; 20 x 192 x 160 x 64 in bfloat16 162 us (106 of bytes), in float32 236 (212).
// One token of 64 sequences, 1024 channels: 4.2 us, a launch.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "layer_common.h"
#include "layer_ops.h"

namespace gleam {
namespace {

constexpr int kTokens = 8;         // of a wave that keeps them in registers, at most
constexpr int kScanWaves = 8;      // of a workgroup, at most

struct ScanArgs {
    const void *x, *r, *i, *g;
    void *out, *out_r, *out_i;            // h; or the gradients of x, r and i
    gleam_scan_strides sx, sr, si, sh;
    const float *lambda, *state_in, *state_end;   // state_end: gradient of the last state
    const int* lengths;
    float *state_out, *g_state_in;
    float *log_a, *add_h, *add_e;         // [b][chunk][p][c]: sum of log2 a, what a chunk adds to h and to E; then h and E that enter it
    float* part;                          // [b][chunk][p][c]: sums of W
    long long B, T, P, C, chunks, groups; // groups of 64 columns
    float kappa;
    int tokens;                           // of a wave
    int odd;                              // C is odd
    int few;                              // groups of workgroups and columns of a sequence are numbers of 32 bits
};

constexpr float kLog2e = 1.44269504f;

// The gates are worked out for every token and channel, and the kernels are bound by vector instructions: decays are kept as their logarithms to
// base 2, which the exponential instruction takes, and a product with log2 e is rounded once, which puts 2^-24 |v| of its value on e^-v.
__device__ __forceinline__ float exp2_of(float v) { return __builtin_amdgcn_exp2f(v); }
__device__ __forceinline__ float sigmoid(float v) { return __builtin_amdgcn_rcpf(1.f + exp2_of(-kLog2e * v)); }
__device__ __forceinline__ void sigmoids(float v, float& s, float& rest) {   // and 1 - sigmoid(v), to its last bits too
    float x = -kLog2e * v;
    x = x > 126.f ? 126.f : x;   // (a NaN stays)
    const float e = exp2_of(x);
    s = __builtin_amdgcn_rcpf(1.f + e);
    rest = e * s;
}
__device__ __forceinline__ float softplus(float v) { return fmaxf(v, 0.f) + log1pf(expf(-fabsf(v))); }

__device__ __forceinline__ bool near_one(float w) { return __float_as_int(w) < 0; }
__device__ __forceinline__ float a_of(float w) { return near_one(w) ? 1.f + w : w; }
// a h + b: where a is near 1, w is a - 1 and h itself is added
__device__ __forceinline__ float step_h(float h, float w, float b, bool near) { return __builtin_fmaf(w, h, b) + (near ? h : 0.f); }
__device__ __forceinline__ float step_h(float h, float w, float b) { return step_h(h, w, b, near_one(w)); }

// The token's gates of one channel from z = log2 a <= 0: a as it is kept, w (2^z - 1 above z = -0.36, by the series to z^6, whose rest is 5e-8 of it;
// 2^z below), m = sqrt(1 - a^2) = sqrt(d (2 - d)).  The coefficients, (ln 2)^k / k!, stand in scalar registers: as literals each would be moved
// into a vector register first.
struct Gate {
    float w, m;
    bool near;
};
struct Series {
    float c[6];
    __device__ __forceinline__ Series() : c{0.693147181f, 0.240226507f, 0.0555041087f, 0.00961812911f, 0.00133335581f, 0.000154035304f} {
#pragma unroll
        for (int i = 0; i < 6; ++i) asm("" : "+s"(c[i]));
    }
};
__device__ __forceinline__ Gate gate_of(float z, const Series& k) {
    float p = __builtin_fmaf(k.c[5], z, k.c[4]);
    p = __builtin_fmaf(p, z, k.c[3]);
    p = __builtin_fmaf(p, z, k.c[2]);
    p = __builtin_fmaf(p, z, k.c[1]);
    p = __builtin_fmaf(p, z, k.c[0]);
    const float less = p * z, a = exp2_of(z);   // a - 1, and a
    Gate g;
    g.near = z > -0.36f;
    g.w = g.near ? less : a;
    const float d = g.near ? -less : 1.f - a;
    g.m = __builtin_amdgcn_sqrtf(d * (2.f - d));
    return g;
}

// Where a wave and a lane are.
template <int V>
struct Spot {
    long long b, k, col;       // sequence, chunk, p * C + first channel
    long long p;
    int c, back;               // first channel; 1: the vector's second channel does not exist, and it is read from the one before on
    bool live;                 // lanes past the last column do the last one's work too, and write nothing
    int t0, t1, t2;            // tokens of the wave: from t0, those before t1 are there, those before t2 in the array
    // group: of 64 columns of a chunk of a sequence; first, count: the wave's tokens
    __device__ __forceinline__ bool set(const ScanArgs& a, long long group) {
        if (a.few) {   // numbers of 32 bits
            const unsigned rest = (unsigned)group / (unsigned)a.groups, sb = rest / (unsigned)a.chunks;
            b = sb;
            k = rest - sb * (unsigned)a.chunks;
            group = (unsigned)group - rest * (unsigned)a.groups;
        } else {
            const long long rest = group / a.groups;
            b = rest / a.chunks;
            k = rest - b * a.chunks;
            group -= rest * a.groups;
        }
        if (b >= a.B) return false;
        const long long vecs = (a.C + V - 1) / V, all = vecs * a.P, mine = group * 64 + (threadIdx.x & 63);
        live = mine < all;
        const long long n = live ? mine : all - 1;
        p = a.P == 1 ? 0 : a.few ? (long long)((unsigned)n / (unsigned)vecs) : n / vecs;
        c = (int)((n - p * vecs) * V);
        back = V > 1 && (long long)c + V > a.C;
        col = p * a.C + c;
        return true;
    }
    __device__ __forceinline__ void tokens(const ScanArgs& a, long long first, int count) {
        int len = (int)a.T;
        if (a.lengths) {
            len = a.lengths[b];
            len = len < 0 ? 0 : len > a.T ? (int)a.T : len;
        }
        const long long end = first + count;
        t0 = (int)(first < a.T ? first : a.T);
        t2 = (int)(end < a.T ? end : a.T);
        t1 = t2 < len ? t2 : len > t0 ? len : t0;
    }
    // of a workgroup whose waves stand one behind the other along a chunk
    __device__ __forceinline__ bool set_chunk(const ScanArgs& a) {
        if (!set(a, group_of_grid())) return false;
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
        tokens(a, (k * waves + wave) * a.tokens, a.tokens);
        return true;
    }
    __device__ __forceinline__ long long at(const gleam_scan_strides& s) const { return b * s.b + p * s.p + c; }
    template <class T>
    __device__ __forceinline__ void store(T* p, const float* v) const {
        if (!live) return;
        if (back) put_f32(p, v[0]);
        else store_vec<T, V>(p, v);
    }
    __device__ __forceinline__ void load_state(const float* p, float* v) const {   // null: zeros
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = p ? p[e && back ? 0 : e] : 0.f;
    }
    __device__ __forceinline__ void store_state(float* p, const float* v) const {
#pragma unroll
        for (int e = 0; e < V; ++e)
            if (live && !(e && back)) p[e] = v[e];
    }
    __device__ __forceinline__ long long slot(const ScanArgs& a) const { return (b * a.chunks + k) * a.P * a.C + col; }
    __device__ __forceinline__ long long state(const ScanArgs& a) const { return b * a.P * a.C + col; }
};

// A wave's tokens as it reads them.  Where there are fewer than L, the last one is read again: requests without branches between them can be
// waited for one by one.
template <class T, int V, int L, bool WITH_G>
struct Tokens {
    Raw<T, V> x[L], r[L], i[L], g[WITH_G ? L : 1];
    __device__ __forceinline__ void load(const ScanArgs& a, const Spot<V>& s) {
        const T *px = (const T*)a.x + s.at(a.sx) + s.t0 * a.sx.t - s.back, *pr = (const T*)a.r + s.at(a.sr) + s.t0 * a.sr.t - s.back;
        const T *pi = (const T*)a.i + s.at(a.si) + s.t0 * a.si.t - s.back, *pg = WITH_G ? (const T*)a.g + s.at(a.sh) + s.t0 * a.sh.t - s.back : nullptr;
        if (s.t0 >= s.t1) return;
#pragma unroll
        for (int j = 0; j < L; ++j) {
            const long long t = s.t0 + j < s.t1 ? j : s.t1 - 1 - s.t0;
            r[j].load(pr + t * a.sr.t);
            i[j].load(pi + t * a.si.t);
            x[j].load(px + t * a.sx.t);
            if (WITH_G) g[j].load(pg + t * a.sh.t);
        }
    }
    // Where C is odd, a vector that was read from `back` before its first channel has that channel behind.
    __device__ __forceinline__ void settle(const ScanArgs& a, const Spot<V>& s) {
        if constexpr (V == 2 && sizeof(T) == 2) {
            if (!a.odd) return;
#pragma unroll
            for (int j = 0; j < L; ++j) {
                x[j].v.w[0] >>= 16 * s.back;
                r[j].v.w[0] >>= 16 * s.back;
                i[j].v.w[0] >>= 16 * s.back;
                if (WITH_G) g[j].v.w[0] >>= 16 * s.back;
            }
        }
    }
};

// -log2 e times c of a workgroup's columns, worked out by its first wave; a barrier stands behind it.
template <int V>
__device__ __forceinline__ void put_rates(const ScanArgs& a, const Spot<V>& s, float (&shared)[V][64]) {
    if (threadIdx.x < 64)
#pragma unroll
        for (int e = 0; e < V; ++e) shared[e][threadIdx.x] = -kLog2e * a.kappa * softplus(a.lambda[s.c + (e && s.back ? 0 : e)]);
}

// What a chunk does to a state, h' = 2^log_a h + add_h, and backwards, E' = 2^log_a E + add_e.
template <class T, int V, int L>
__global__ __launch_bounds__(64 * kScanWaves) void scan_chunk_kernel(ScanArgs a) {
    __shared__ float ends[kScanWaves][3][V][64], shared[V][64];
    Spot<V> s;
    if (!s.set_chunk(a)) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    Tokens<T, V, L, true> tok;
    tok.load(a, s);
    put_rates(a, s, shared);
    __syncthreads();
    tok.settle(a, s);
    const Series series;
    float c[V], sum[V], h[V], e_add[V], w[L][V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
        c[e] = shared[e][lane];
        sum[e] = h[e] = e_add[e] = 0.f;
    }
#pragma unroll
    for (int j = 0; j < L; ++j)
        if (s.t0 + j < s.t1)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float z = c[e] * sigmoid(tok.r[j].get(e));
                const Gate g = gate_of(z, series);
                w[j][e] = g.w;
                sum[e] += z;
                h[e] = step_h(h[e], g.w, g.m * (sigmoid(tok.i[j].get(e)) * tok.x[j].get(e)), g.near);
            }
#pragma unroll
    for (int j = L - 1; j >= 0; --j)
        if (s.t0 + j < s.t1)
#pragma unroll
            for (int e = 0; e < V; ++e) e_add[e] = step_h(tok.g[j].get(e) + e_add[e], w[j][e], 0.f);
#pragma unroll
    for (int e = 0; e < V; ++e) {
        ends[wave][0][e][lane] = sum[e];
        ends[wave][1][e][lane] = h[e];
        ends[wave][2][e][lane] = e_add[e];
    }
    __syncthreads();
    if (wave) return;
    for (int v = 1; v < waves; ++v)
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const float more = ends[v][0][e][lane];
            e_add[e] += exp2_of(sum[e]) * ends[v][2][e][lane];
            h[e] = __builtin_fmaf(exp2_of(more), h[e], ends[v][1][e][lane]);
            sum[e] += more;
        }
    const long long at = s.slot(a);
    s.store_state(a.log_a + at, sum);
    s.store_state(a.add_h + at, h);
    s.store_state(a.add_e + at, e_add);
}

// Carries at the chunks' starts (and ends, backwards), in the place of what the chunks add: 32 states a workgroup, 32 lanes of each one behind
// the other along the chunks.
template <bool BWD>
__global__ __launch_bounds__(1024) void scan_carry_kernel(ScanArgs a) {
    __shared__ float ends[32][BWD ? 3 : 2][32];
    const int lane = threadIdx.x & 31, wave = threadIdx.x >> 5;   // a state, and the stretch of chunks
    const long long pc = a.P * a.C, all = a.B * pc, mine = group_of_grid() * 32 + lane, n = mine < all ? mine : all - 1;
    const long long b = a.B == 1 ? 0 : n / pc, base = b * a.chunks * pc + (n - b * pc);
    const int k0 = (int)(a.chunks * wave / 32), k1 = (int)(a.chunks * (wave + 1) / 32);
    float sum = 0.f, h = 0.f, e = 0.f;
#pragma unroll 8
    for (int k = k0; k < k1; ++k) {
        const float la = a.log_a[base + k * pc];
        h = __builtin_fmaf(exp2_of(la), h, a.add_h[base + k * pc]);
        if (BWD) e += exp2_of(sum) * a.add_e[base + k * pc];
        sum += la;
    }
    ends[wave][0][lane] = sum;
    ends[wave][1][lane] = h;
    if (BWD) ends[wave][2][lane] = e;
    __syncthreads();
    h = a.state_in ? a.state_in[n] : 0.f;
    for (int v = 0; v < wave; ++v) h = __builtin_fmaf(exp2_of(ends[v][0][lane]), h, ends[v][1][lane]);
    if (BWD) {
        e = a.state_end ? a.state_end[n] : 0.f;
        for (int v = 31; v > wave; --v) e = __builtin_fmaf(exp2_of(ends[v][0][lane]), e, ends[v][2][lane]);
    }
    if (mine >= all) return;
    // four chunks' numbers are read before the first of them is written over
    for (int k = k0; k < k1; k += 4) {
        float la[4], add[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const long long at = base + (k + i < k1 ? k + i : k) * pc;
            la[i] = a.log_a[at], add[i] = a.add_h[at];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (k + i < k1) {
                a.add_h[base + (k + i) * pc] = h;
                h = __builtin_fmaf(exp2_of(la[i]), h, add[i]);
            }
    }
    if (!BWD) return;
    for (int k = k1 - 1; k >= k0; k -= 4) {
        float la[4], add[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const long long at = base + (k - i >= k0 ? k - i : k) * pc;
            la[i] = a.log_a[at], add[i] = a.add_e[at];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (k - i >= k0) {
                a.add_e[base + (k - i) * pc] = e;
                e = __builtin_fmaf(exp2_of(la[i]), e, add[i]);
            }
    }
}

// Forward, one wave, one chunk of 64 columns from its first token to its last: all of a sequence where there are columns enough, or few tokens.
// Four tokens are on their way while four are worked on.  SUM: what the chunk does to a state, instead of h.
template <class T, int V, bool SUM>
__global__ __launch_bounds__(256) void scan_walk_kernel(ScanArgs a) {
    constexpr int L = 4;
    Spot<V> s;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (!s.set(a, group_of_grid() * 4 + wave)) return;
    s.tokens(a, s.k * a.tokens, a.tokens);
    const int first = s.t0, len = s.t1, end = s.t2;
    Tokens<T, V, L, false> tok;
    tok.load(a, s);
    float c[V], h[V], sum[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
        c[e] = -kLog2e * a.kappa * softplus(a.lambda[s.c + (e && s.back ? 0 : e)]);
        sum[e] = 0.f;
    }
    s.load_state(SUM ? nullptr : a.chunks > 1 ? a.add_h + s.slot(a) : a.state_in ? a.state_in + s.state(a) : nullptr, h);
    T* out = (T*)a.out + s.at(a.sh);
    const Series series;
    for (int t = first; t < len; t += L) {
        Tokens<T, V, L, false> now = tok;
        now.settle(a, s);
        s.t0 = t + L < len ? t + L : len;
        tok.load(a, s);
#pragma unroll
        for (int j = 0; j < L; ++j)
            if (t + j < len) {
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float z = c[e] * sigmoid(now.r[j].get(e));
                    const Gate g = gate_of(z, series);
                    h[e] = step_h(h[e], g.w, g.m * (sigmoid(now.i[j].get(e)) * now.x[j].get(e)), g.near);
                    if (SUM) sum[e] += z;
                }
                if (!SUM) s.store(out + (t + j) * a.sh.t, h);
            }
    }
    if (SUM) {
        s.store_state(a.log_a + s.slot(a), sum);
        s.store_state(a.add_h + s.slot(a), h);
        return;
    }
    const float none[V] = {};
    for (int t = len; t < end; ++t) s.store(out + t * a.sh.t, none);
    if (a.state_out && s.k == a.chunks - 1) s.store_state(a.state_out + s.state(a), h);
}

// Forward, few tokens and few columns: one workgroup's waves one behind the other.
template <class T, int V, int L>
__global__ __launch_bounds__(64 * kScanWaves) void scan_fwd_kernel(ScanArgs a) {
    __shared__ float ends[kScanWaves][2][V][64], shared[V][64];
    Spot<V> s;
    if (!s.set_chunk(a)) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    Tokens<T, V, L, false> tok;
    tok.load(a, s);
    float c[V], sum[V], h[V], carry[V], w[L][V], b[L][V];
    s.load_state(a.state_in ? a.state_in + s.state(a) : nullptr, carry);
    put_rates(a, s, shared);
    __syncthreads();
    tok.settle(a, s);
    const Series series;
#pragma unroll
    for (int e = 0; e < V; ++e) {
        c[e] = shared[e][lane];
        sum[e] = h[e] = 0.f;
    }
#pragma unroll
    for (int j = 0; j < L; ++j)
        if (s.t0 + j < s.t1)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float z = c[e] * sigmoid(tok.r[j].get(e));
                const Gate g = gate_of(z, series);
                w[j][e] = g.w;
                b[j][e] = g.m * (sigmoid(tok.i[j].get(e)) * tok.x[j].get(e));
                sum[e] += z;
                h[e] = step_h(h[e], g.w, b[j][e], g.near);
            }
#pragma unroll
    for (int e = 0; e < V; ++e) {
        ends[wave][0][e][lane] = sum[e];
        ends[wave][1][e][lane] = h[e];
    }
    __syncthreads();
    for (int v = 0; v < wave; ++v)
#pragma unroll
        for (int e = 0; e < V; ++e) carry[e] = __builtin_fmaf(exp2_of(ends[v][0][e][lane]), carry[e], ends[v][1][e][lane]);
    T* out = (T*)a.out + s.at(a.sh) + s.t0 * a.sh.t;
#pragma unroll
    for (int j = 0; j < L; ++j) {
        if (s.t0 + j < s.t1) {
#pragma unroll
            for (int e = 0; e < V; ++e) carry[e] = step_h(carry[e], w[j][e], b[j][e]);
            s.store(out + j * a.sh.t, carry);
        } else if (s.t0 + j < s.t2) {
            const float none[V] = {};
            s.store(out + j * a.sh.t, none);
        }
    }
    if (a.state_out && wave == waves - 1) s.store_state(a.state_out + s.state(a), carry);
}

template <class T, int V, int L>
__global__ __launch_bounds__(64 * kScanWaves) void scan_bwd_kernel(ScanArgs a) {
    __shared__ float ends[kScanWaves][3][V][64], shared[V][64];
    Spot<V> s;
    if (!s.set_chunk(a)) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    Tokens<T, V, L, true> tok;
    tok.load(a, s);
    const bool split = a.chunks > 1;
    float c[V], sum[V], h[V], e_add[V], carry[V], ahead[V], w_sum[V], w[L][V], b[L][V];
    s.load_state(split ? a.add_h + s.slot(a) : a.state_in ? a.state_in + s.state(a) : nullptr, carry);
    s.load_state(split ? a.add_e + s.slot(a) : a.state_end ? a.state_end + s.state(a) : nullptr, ahead);
    put_rates(a, s, shared);
    __syncthreads();
    tok.settle(a, s);
    const Series series;
#pragma unroll
    for (int e = 0; e < V; ++e) {
        c[e] = shared[e][lane];
        sum[e] = h[e] = e_add[e] = w_sum[e] = 0.f;
    }
#pragma unroll
    for (int j = 0; j < L; ++j)
        if (s.t0 + j < s.t1)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float z = c[e] * sigmoid(tok.r[j].get(e));
                const Gate g = gate_of(z, series);
                w[j][e] = g.w;
                b[j][e] = g.m * (sigmoid(tok.i[j].get(e)) * tok.x[j].get(e));
                sum[e] += z;
                h[e] = step_h(h[e], g.w, b[j][e], g.near);
            }
    if (waves > 1) {
#pragma unroll
        for (int j = L - 1; j >= 0; --j)
            if (s.t0 + j < s.t1)
#pragma unroll
                for (int e = 0; e < V; ++e) e_add[e] = step_h(tok.g[j].get(e) + e_add[e], w[j][e], 0.f);
#pragma unroll
        for (int e = 0; e < V; ++e) {
            ends[wave][0][e][lane] = sum[e];
            ends[wave][1][e][lane] = h[e];
            ends[wave][2][e][lane] = e_add[e];
        }
        __syncthreads();
        for (int v = 0; v < wave; ++v)
#pragma unroll
            for (int e = 0; e < V; ++e) carry[e] = __builtin_fmaf(exp2_of(ends[v][0][e][lane]), carry[e], ends[v][1][e][lane]);
        for (int v = waves - 1; v > wave; --v)
#pragma unroll
            for (int e = 0; e < V; ++e) ahead[e] = __builtin_fmaf(exp2_of(ends[v][0][e][lane]), ahead[e], ends[v][2][e][lane]);
    }
    // h before each token, in the place of b
#pragma unroll
    for (int j = 0; j < L; ++j)
        if (s.t0 + j < s.t1)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float next = step_h(carry[e], w[j][e], b[j][e]);
                b[j][e] = carry[e];
                carry[e] = next;
            }
    T *gx = (T*)a.out + s.at(a.sx) + s.t0 * a.sx.t, *gr = (T*)a.out_r + s.at(a.sr) + s.t0 * a.sr.t, *gi = (T*)a.out_i + s.at(a.si) + s.t0 * a.si.t;
#pragma unroll
    for (int j = L - 1; j >= 0; --j) {
        float ox[V] = {}, orr[V] = {}, oi[V] = {};
        if (s.t0 + j < s.t1) {
#pragma unroll
            for (int e = 0; e < V; ++e) {
                float sr, rest, si, rest_i;
                sigmoids(tok.r[j].get(e), sr, rest);
                sigmoids(tok.i[j].get(e), si, rest_i);
                const float G = tok.g[j].get(e) + ahead[e], wj = w[j][e], y = (-0.693147181f * c[e]) * sr, al = a_of(wj), d = near_one(wj) ? -wj : 1.f - wj;
                const float m2 = d * (2.f - d), one_m = m2 < 0x1p-126f ? 0.f : __builtin_amdgcn_rsqf(m2), q = y * one_m, m = m2 * one_m;   // (a NaN stays)
                const float u = si * tok.x[j].get(e), gu = G * m;
                const float W = G * al * (al * u * q - b[j][e] * y);
                ox[e] = gu * si;
                oi[e] = gu * (u * rest_i);
                orr[e] = W * rest;
                w_sum[e] += W;
                ahead[e] = step_h(G, wj, 0.f);
            }
        }
        if (s.t0 + j < s.t2) {
            s.store(gx + j * a.sx.t, ox);
            s.store(gr + j * a.sr.t, orr);
            s.store(gi + j * a.si.t, oi);
        }
    }
    if (a.g_state_in && s.k == 0 && wave == 0) s.store_state(a.g_state_in + s.state(a), ahead);
    if (waves > 1) {
        __syncthreads();
#pragma unroll
        for (int e = 0; e < V; ++e) ends[wave][0][e][lane] = w_sum[e];
        __syncthreads();
        if (wave) return;
        for (int v = 1; v < waves; ++v)
#pragma unroll
            for (int e = 0; e < V; ++e) w_sum[e] += ends[v][0][e][lane];
    }
    s.store_state(a.part + s.slot(a), w_sum);
}

// Sums over rows of C columns: 64 columns and a slab of rows a workgroup.  lambda not null: the last sum, out = g_lambda.
__global__ __launch_bounds__(1024) void scan_sums_kernel(const float* part, long long rows, long long C, long long slab, const float* lambda, float* out) {
    __shared__ float red[16][64];
    const long long col_groups = (C + 63) / 64, id = group_of_grid(), s = id / col_groups;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const long long c = (id - s * col_groups) * 64 + lane, end = (s + 1) * slab < rows ? (s + 1) * slab : rows;
    float v = 0.f;
    if (c < C)
        for (long long r = s * slab + wave; r < end; r += 16) v += part[r * C + c];
    red[wave][lane] = v;
    __syncthreads();
    if (wave || c >= C || s * slab >= rows) return;
    for (int i = 1; i < 16; ++i) v += red[i][lane];
    if (lambda) {
        // d softplus / softplus: goes to 1 where both vanish
        const float l = lambda[c];
        v *= l < -20.f ? 1.f : 1.f / ((1.f + expf(-l)) * softplus(l));
    }
    out[s * C + c] = v;
}

struct ScanPlan {
    bool walk;
    int waves, tokens, vec;
    long long chunks, groups, slots;     // slots: states of all chunks
    long long rows, slabs, slab;         // of the sums of W
};
ScanPlan plan_of(const gleam_gatedscan_desc& d, bool backward) {
    ScanPlan p;
    p.vec = d.dtype && d.C > 1 ? 2 : 1;
    p.groups = ((d.C + p.vec - 1) / p.vec * d.P + 63) / 64;
    const long long columns = d.B * p.groups;   // waves
    // Forward, waves that walk: all tokens where there are waves for every SIMD twice, or few tokens; sequences of more than a workgroup of
    // the other kind takes in pieces of 16 tokens, or more as long as 4096 waves remain (a wave works out c first, 110 instructions a channel).
    p.walk = !backward && (d.T <= 4 || d.T > kTokens * kScanWaves || columns >= 2048);
    if (p.walk) {
        long long per = columns >= 2048 || d.T <= 4 ? d.T : d.T * columns / 4096;
        per = (per < 16 ? 16 : per + 3) / 4 * 4;
        p.waves = 1;
        p.chunks = (d.T + per - 1) / per;
        p.tokens = (int)(p.chunks == 1 ? d.T : per);
    } else {
        p.waves = 1;
        while (p.waves < kScanWaves && p.waves * kTokens < d.T) p.waves *= 2;
        p.chunks = (d.T + p.waves * kTokens - 1) / (p.waves * kTokens);
        const long long per = (d.T + p.chunks - 1) / p.chunks;
        p.tokens = (int)((per + p.waves - 1) / p.waves);
    }
    p.slots = d.B * p.chunks * d.P * d.C;
    p.rows = d.B * p.chunks * d.P;
    const long long col_groups = (d.C + 63) / 64;
    p.slabs = p.rows <= 512 ? 1 : p.rows / 128;
    const long long most_slabs = col_groups < 1024 ? 1024 / col_groups : 1;
    if (p.slabs > most_slabs) p.slabs = most_slabs;
    p.slab = (p.rows + p.slabs - 1) / p.slabs;
    p.slabs = (p.rows + p.slab - 1) / p.slab;   // rounded up, fewer slabs may hold all rows: none is without one, every sum is written that is read
    return p;
}
size_t up256(size_t n) { return (n + 255) / 256 * 256; }

ScanArgs args_of(const gleam_gatedscan_desc& d, const ScanPlan& p, const void* x, const void* r, const void* i, const float* lambda,
                 const int* lengths, const float* state_in) {
    ScanArgs a{};
    a.x = x;
    a.r = r;
    a.i = i;
    a.sx = d.x;
    a.sr = d.r;
    a.si = d.i;
    a.sh = d.h;
    a.lambda = lambda;
    a.lengths = lengths;
    a.state_in = state_in;
    a.B = d.B;
    a.T = d.T;
    a.P = d.P;
    a.C = d.C;
    a.chunks = p.chunks;
    a.groups = p.groups;
    a.kappa = d.kappa;
    a.tokens = p.tokens;
    a.odd = d.C & 1;
    a.few = d.B * p.chunks * p.groups < 0x7fffffff && p.groups < 0x1ffffff;
    return a;
}

template <bool SUM>
void launch_walk(const ScanArgs& a, const ScanPlan& p, int dtype, hipStream_t st) {
    const dim3 grid = grid_of((a.B * p.chunks * p.groups + 3) / 4), block(256);
    if (!dtype) hipLaunchKernelGGL((scan_walk_kernel<float, 1, SUM>), grid, block, 0, st, a);
    else if (p.vec == 2) hipLaunchKernelGGL((scan_walk_kernel<unsigned short, 2, SUM>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((scan_walk_kernel<unsigned short, 1, SUM>), grid, block, 0, st, a);
}

// What chunks do to a state, one way or both, and the carries of a split sequence from that.
template <bool BWD>
hipError_t find_carries(const ScanArgs& a, const ScanPlan& p, int dtype, hipStream_t st) {
    if (p.chunks == 1) return hipSuccess;
    {
        const double size = (double)a.B * a.T * a.P * a.C;
        KernelScope ks(BWD ? "scan_chunk_bwd" : "scan_chunk", (BWD ? 30.0 : 25.0) * size, (BWD ? 4.0 : 3.0) * (dtype ? 2 : 4) * size, st);
        const long long groups = a.B * p.chunks * p.groups;
        if constexpr (BWD) {
            const dim3 grid = grid_of(groups), block(64 * p.waves);
            if (!dtype) hipLaunchKernelGGL((scan_chunk_kernel<float, 1, kTokens>), grid, block, 0, st, a);
            else if (p.vec == 2) hipLaunchKernelGGL((scan_chunk_kernel<unsigned short, 2, kTokens>), grid, block, 0, st, a);
            else hipLaunchKernelGGL((scan_chunk_kernel<unsigned short, 1, kTokens>), grid, block, 0, st, a);
        } else {
            launch_walk<true>(a, p, dtype, st);
        }
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    KernelScope ks("scan_carry", 0.0, (BWD ? 20.0 : 12.0) * p.slots, st);
    hipLaunchKernelGGL(scan_carry_kernel<BWD>, grid_of((a.B * a.P * a.C + 31) / 32), dim3(1024), 0, st, a);
    return hipGetLastError();
}

}  // namespace

size_t gatedscan_fwd_ws_bytes(const gleam_gatedscan_desc& d) {
    const ScanPlan p = plan_of(d, false);
    return p.chunks > 1 ? 2 * up256(p.slots * sizeof(float)) : 0;
}

hipError_t gatedscan_forward(const gleam_gatedscan_desc& d, const void* x, const void* r, const void* i, const float* lambda,
                             const int* lengths, const float* state_in, void* h, float* state_out, void* ws, hipStream_t st) {
    const ScanPlan p = plan_of(d, false);
    ScanArgs a = args_of(d, p, x, r, i, lambda, lengths, state_in);
    a.out = h;
    a.state_out = state_out;
    const size_t each = up256(p.slots * sizeof(float));
    if (p.chunks > 1) {
        a.log_a = (float*)ws;
        a.add_h = (float*)((char*)ws + each);
    }
    const hipError_t e = find_carries<false>(a, p, d.dtype, st);
    if (e != hipSuccess) return e;
    const double size = (double)d.B * d.T * d.P * d.C;
    KernelScope ks("scan_fwd", 25.0 * size, 4.0 * (d.dtype ? 2 : 4) * size, st);
    if (p.walk) {
        launch_walk<false>(a, p, d.dtype, st);
        return hipGetLastError();
    }
    const dim3 grid = grid_of(d.B * p.chunks * p.groups), block(64 * p.waves);
    if (!d.dtype) hipLaunchKernelGGL((scan_fwd_kernel<float, 1, kTokens>), grid, block, 0, st, a);
    else if (p.vec == 2) hipLaunchKernelGGL((scan_fwd_kernel<unsigned short, 2, kTokens>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((scan_fwd_kernel<unsigned short, 1, kTokens>), grid, block, 0, st, a);
    return hipGetLastError();
}

size_t gatedscan_bwd_ws_bytes(const gleam_gatedscan_desc& d) {
    const ScanPlan p = plan_of(d, true);
    return (p.chunks > 1 ? 4 : 1) * up256(p.slots * sizeof(float)) + up256(p.slabs * d.C * sizeof(float));
}

hipError_t gatedscan_backward(const gleam_gatedscan_desc& d, const void* x, const void* r, const void* i, const float* lambda,
                              const int* lengths, const float* state_in, const void* g_h, const float* g_state_out, void* g_x, void* g_r,
                              void* g_i, float* g_lambda, float* g_state_in, void* ws, hipStream_t st) {
    const ScanPlan p = plan_of(d, true);
    ScanArgs a = args_of(d, p, x, r, i, lambda, lengths, state_in);
    a.g = g_h;
    a.state_end = g_state_out;
    a.out = g_x;
    a.out_r = g_r;
    a.out_i = g_i;
    a.g_state_in = g_state_in;
    const size_t each = up256(p.slots * sizeof(float));
    char* at = (char*)ws;
    a.part = (float*)at;
    float* sums = (float*)(at + each);
    at += each + up256(p.slabs * d.C * sizeof(float));
    if (p.chunks > 1) {
        a.log_a = (float*)at;
        a.add_h = (float*)(at + each);
        a.add_e = (float*)(at + 2 * each);
    }
    hipError_t e = find_carries<true>(a, p, d.dtype, st);
    if (e != hipSuccess) return e;
    {
        const double size = (double)d.B * d.T * d.P * d.C;
        KernelScope ks("scan_bwd", 50.0 * size, 7.0 * (d.dtype ? 2 : 4) * size, st);
        const dim3 grid = grid_of(d.B * p.chunks * p.groups), block(64 * p.waves);
        if (!d.dtype) hipLaunchKernelGGL((scan_bwd_kernel<float, 1, kTokens>), grid, block, 0, st, a);
        else if (p.vec == 2) hipLaunchKernelGGL((scan_bwd_kernel<unsigned short, 2, kTokens>), grid, block, 0, st, a);
        else hipLaunchKernelGGL((scan_bwd_kernel<unsigned short, 1, kTokens>), grid, block, 0, st, a);
    }
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    const long long col_groups = (d.C + 63) / 64;
    KernelScope ks("scan_sums", 0.0, 4.0 * p.slots, st);
    if (p.slabs > 1) {
        hipLaunchKernelGGL(scan_sums_kernel, grid_of(p.slabs * col_groups), dim3(1024), 0, st, a.part, p.rows, (long long)d.C, p.slab, (const float*)nullptr, sums);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(scan_sums_kernel, grid_of(col_groups), dim3(1024), 0, st, p.slabs > 1 ? sums : a.part, p.slabs > 1 ? p.slabs : p.rows, (long long)d.C,
                       p.slabs > 1 ? p.slabs : p.rows, lambda, g_lambda);
    return hipGetLastError();
}

}  // namespace gleam
