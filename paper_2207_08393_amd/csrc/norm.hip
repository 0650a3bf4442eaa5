// Layer norm over rows of n elements, forward and backward (gfx950).
//
// Forward: one read and one write of the row.  A team of lanes holds a whole row in registers, so the variance is the mean of the
// squared distances from the mean (no cancellation where the mean is large) without a second read.  The mean is a sum of x / n (which stays
// in range) and then the mean of what the elements are away from that, which takes out what the first sum was rounded by: it is
// good to its last bits whatever the row's order and size, and a row of equal numbers has exactly that mean and becomes zeros.  Where the
// variance passes the range of a float32, r = 0 and outputs are beta.  Backward: one read of x and g_y,
// one write of g_x; every lane keeps its columns from row to row and sums g_gamma and g_beta in registers, a workgroup writes one
// partial sum per column and a second launch adds them up in a fixed order.  Both are bound by HBM.
// Measured: forward 4 x 320 x 256 pixels of 100 channels, float32, 60 us (4.4 TB/s); backward 4 x 640 x 320 of 128 channels, bfloat16, 121 us
// (5.2 TB/s, the rate of a copy), 2000 rows of 5001 float32 34 us (3.5 TB/s; some 6 us of it the sum of the partial sums).
//
// Rows too long for the registers of a workgroup are read three times (forward) or twice (backward), see the streaming kernels.
#include <hip/hip_runtime.h>

#include <cfloat>

#include "layer_common.h"
#include "layer_ops.h"

namespace gleam {
namespace {

constexpr int kNormThreads = 256;

template <class T>
constexpr int vec_of() { return 16 / (int)sizeof(T); }

template <int LANES>
constexpr int threads_of() { return LANES > 64 ? LANES : kNormThreads; }

// Sums over a team of LANES lanes, the same values in all of them.  A team wider than a wave is the workgroup; `red` is then LDS for
// N floats a wave, and the barrier in front makes its last use over.
template <int LANES, int N>
__device__ __forceinline__ void team_sum(float (&v)[N], float* red) {
#pragma unroll
    for (int k = 0; k < N; ++k) {
        v[k] += dpp<0xB1>(v[k]);                      // lane i and i ^ 1
        v[k] += dpp<0x4E>(v[k]);                      // i ^ 2
        if (LANES >= 8) v[k] += dpp<0x141>(v[k]);     // 7 - i of eight lanes, which are equal in fours
        if (LANES >= 16) v[k] += dpp<0x140>(v[k]);    // 15 - i of sixteen
        if (LANES >= 32) v[k] = sum_of_pair(__builtin_amdgcn_permlane16_swap(__float_as_uint(v[k]), __float_as_uint(v[k]), false, false));
        if (LANES >= 64) v[k] = sum_of_pair(__builtin_amdgcn_permlane32_swap(__float_as_uint(v[k]), __float_as_uint(v[k]), false, false));
    }
    if constexpr (LANES > 64) {
        constexpr int W = LANES / 64;
        __syncthreads();
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int k = 0; k < N; ++k) red[k * W + (threadIdx.x >> 6)] = v[k];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < N; ++k) {
            v[k] = red[k * W];
#pragma unroll
            for (int w = 1; w < W; ++w) v[k] += red[k * W + w];
        }
    }
}

// The columns of one of a lane's vectors, the same in every row.  The row's last vector is moved back to end with the row; its first
// elements are then those of the vector before it and stay out of sums (their results are written twice, the same bits).  What stays out
// is masked and not multiplied by zero, which would make NaN of an infinity or a square that overflows.
// Rows shorter than a vector: hi < VE, element by element.
template <int VE>
struct Columns {
    int col, hi;
    unsigned counts[VE];      // all bits where the element is one of the vector's own
    __device__ __forceinline__ float own(int i, float v) const { return __uint_as_float(__float_as_uint(v) & counts[i]); }
    __device__ __forceinline__ void set(int unit, int n) {
        col = unit * VE;
        hi = col < n ? VE : 0;
        int lo = 0;
        if (hi && col + VE > n) {
            if (n >= VE) {
                lo = col + VE - n;
                col = n - VE;
            } else {
                hi = n;
            }
        }
        if (!hi) col = 0;
#pragma unroll
        for (int i = 0; i < VE; ++i) {
            counts[i] = i >= lo && i < hi ? ~0u : 0u;
            asm("" : "+v"(counts[i]));   // stays a number: as conditions they would be pairs of scalar registers, more than there are
        }
    }
};
// A team is as small as the row allows, so that the first half of every lane's vectors (rounded up, of more than one) is whole: no mask.
template <int NV, int VE>
__device__ __forceinline__ float own(const Columns<VE>& c, int j, int i, float v) { return NV > 1 && j < (NV + 1) / 2 ? v : c.own(i, v); }
// Lanes without columns read the row's first elements, or nothing where a row is shorter than a vector; they count for nothing.
template <class T, int VE>
__device__ __forceinline__ void load_cols(const T* row, const Columns<VE>& c, bool narrow, Pack<T, VE>& p) {
    if (!narrow) {
        p.load(row + c.col);
    } else {
        float v[VE];
#pragma unroll
        for (int i = 0; i < VE; ++i) v[i] = i < c.hi ? to_f32(row[i]) : 0.f;
        p.set(v);
    }
}
template <class T, int VE>
__device__ __forceinline__ void store_cols(T* row, const Columns<VE>& c, const float* v) {
    if (c.hi == VE) {
        Pack<T, VE> p;
        p.set(v);
        p.store(row + c.col);
    } else {
#pragma unroll
        for (int i = 0; i < VE; ++i)
            if (i < c.hi) put_f32(row + c.col + i, v[i]);
    }
}
template <int VE>
__device__ __forceinline__ void load_param(const float* p, const Columns<VE>& c, float fallback, float* v) {
#pragma unroll
    for (int i = 0; i < VE; ++i) v[i] = fallback;
    if (!p) return;
    if (c.hi == VE) {
#pragma unroll
        for (int i = 0; i < VE; i += 4) __builtin_memcpy(v + i, p + c.col + i, 16);
    } else {
#pragma unroll
        for (int i = 0; i < VE; ++i)
            if (i < c.hi) v[i] = p[c.col + i];
    }
}

// The first mean and the mean of the distances from it.  The latter is out of range only where the row holds infinities or NaN (then the
// first mean is one of them), or numbers of both signs near the end of the range.
__device__ __forceinline__ float mean_of(float first, float rest) { return fabsf(rest) <= FLT_MAX ? first + rest : first; }
// The variance from the mean distance d[0] and the sum d[1] of squared distances from the first mean.  False where it would be lost in the
// difference (the spread is of the size of the first mean's rounding, as in a row of equal numbers) or is out of range: then the squared
// distances from the mean itself are summed.
__device__ __forceinline__ bool variance_of(const float (&d)[2], float inv_n, float& var) {
    const float about = d[1] * inv_n, off = d[0] * d[0];
    var = about - off;
    return d[1] <= FLT_MAX && off <= 0.0625f * about;
}

struct NormArgs {
    const void *x, *g;
    const float *gamma, *beta, *mean_in, *rstd_in;
    void* out;
    float *mean, *rstd;
    float* part;              // backward: [workgroup][2][n] partial sums, or null
    long long rows, n, ld_x, ld_y;
    float eps;
};

// A workgroup walks rows.  The next row is on its way while one is computed on, where registers allow it, and the parameters
// stay in registers up to kKept of them a lane (more are read again from the cache for every row).
constexpr int kKept = 16;

template <class T, int LANES, int NV>
__global__ __launch_bounds__(threads_of<LANES>()) void norm_fwd_kernel(NormArgs a) {
    constexpr int VE = vec_of<T>(), TEAMS = threads_of<LANES>() / LANES;
    constexpr bool kKeep = NV * VE <= kKept;
    __shared__ float red[LANES > 64 ? 2 * LANES / 64 : 1];
    const int lane = threadIdx.x % LANES, team = threadIdx.x / LANES, n = (int)a.n;
    const bool narrow = n < VE;
    const float inv_n = 1.f / (float)n;
    const T* x = (const T*)a.x;
    T* y = (T*)a.out;
    Columns<VE> cols[NV];
    float gm[NV][VE], bt[NV][VE];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        cols[j].set(lane + j * LANES, n);
        if (kKeep) {
            load_param(a.gamma, cols[j], 1.f, gm[j]);
            load_param(a.beta, cols[j], 0.f, bt[j]);
        }
    }
    const long long step = (long long)gridDim.x * TEAMS;
    // a row beyond the last is read as the last and not written, so that every lane of a wave takes part in the sums
    auto there = [&](long long row) { return row < a.rows ? row : a.rows - 1; };
    long long row = (long long)blockIdx.x * TEAMS + team;
    Pack<T, VE> next[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) load_cols(x + there(row) * a.ld_x, cols[j], narrow, next[j]);
    for (long long first = (long long)blockIdx.x * TEAMS; first < a.rows; first += step, row += step) {
        float v[NV][VE], s[1] = {0.f};
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < VE; ++i) v[j][i] = next[j].get(i);
        if (first + step < a.rows) {
            const T* p = x + there(row + step) * a.ld_x;
#pragma unroll
            for (int j = 0; j < NV; ++j) load_cols(p, cols[j], narrow, next[j]);
        }
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < VE; ++i) s[0] += own<NV>(cols[j], j, i, v[j][i]) * inv_n;
        team_sum<LANES>(s, red);
        const float first_mean = s[0];
        float t[2] = {0.f, 0.f};
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < VE; ++i) {
                const float d = own<NV>(cols[j], j, i, v[j][i] - first_mean);
                t[0] += d * inv_n;
                t[1] += d * d;
            }
        team_sum<LANES>(t, red);
        const float mean = mean_of(first_mean, t[0]);
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < VE; ++i) v[j][i] -= mean;
        float var;
        if (!variance_of(t, inv_n, var)) {
            s[0] = 0.f;
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int i = 0; i < VE; ++i) {
                    const float d = own<NV>(cols[j], j, i, v[j][i]);
                    s[0] += d * d;
                }
            team_sum<LANES>(s, red);
            var = s[0] * inv_n;
        }
        const float rstd = 1.f / sqrtf(var + a.eps);
        if (row >= a.rows) continue;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if (!cols[j].hi) continue;
            if (!kKeep) {
                load_param(a.gamma, cols[j], 1.f, gm[j]);
                load_param(a.beta, cols[j], 0.f, bt[j]);
            }
            float o[VE];
#pragma unroll
            for (int i = 0; i < VE; ++i) o[i] = v[j][i] * rstd * gm[j][i] + bt[j][i];
            store_cols(y + row * a.ld_y, cols[j], o);
        }
        if (lane == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
    }
}

template <class T, int LANES, int NV>
__global__ __launch_bounds__(threads_of<LANES>(), (NV * vec_of<T>() <= 8 && LANES <= 64 ? 4 : 1)) void norm_bwd_kernel(NormArgs a) {
    constexpr int VE = vec_of<T>(), TEAMS = threads_of<LANES>() / LANES;
    // 1024 lanes leave 128 registers each: gamma is read for every row, and the next row when it is needed (500 rows of 16384: float32 55 -> 45 us,
    // bfloat16 47 -> 38)
    constexpr int kHeld = LANES == 1024 ? 8 : kKept;
    constexpr bool kKeep = NV * VE <= kHeld, kAhead = NV * VE <= kHeld;
    __shared__ float red[LANES > 64 ? 2 * LANES / 64 : 1];
    __shared__ float fold[TEAMS > 1 ? kNormThreads / 64 : 1][TEAMS > 1 ? LANES * VE : 1];
    const int lane = TEAMS == 1 ? threadIdx.x : threadIdx.x % LANES, n = (int)a.n;
    const int team = TEAMS == 1 ? 0 : LANES == 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : threadIdx.x / LANES;
    const bool narrow = n < VE;
    const float inv_n = 1.f / (float)n;
    const T *x = (const T*)a.x, *g = (const T*)a.g;
    T* gx = (T*)a.out;
    Columns<VE> cols[NV];
    float gm[NV][VE], dg[NV][VE] = {}, db[NV][VE] = {};
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        cols[j].set(lane + j * LANES, n);
        if (kKeep) load_param(a.gamma, cols[j], 1.f, gm[j]);
    }
    const long long step = (long long)gridDim.x * TEAMS;
    long long row = (long long)blockIdx.x * TEAMS + team;
    Pack<T, VE> nx[NV], ng[NV];
    float next_mean, next_rstd;
    auto fetch = [&](long long at) {
        next_mean = a.mean_in[at];
        next_rstd = a.rstd_in[at];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            load_cols(x + at * a.ld_x, cols[j], narrow, nx[j]);
            load_cols(g + at * a.ld_y, cols[j], narrow, ng[j]);
        }
    };
    if (kAhead) fetch(row < a.rows ? row : a.rows - 1);
    // teams end at different rows: their sums need no other lanes, or (a team that is the workgroup) all end alike
    for (; row < a.rows; row += step) {
        if constexpr (LANES >= 64) asm("" : "+s"(row));   // addresses from the row's number every time: kept from row to row they are spilled
        if (!kAhead) fetch(row);
        const float mean = next_mean, rstd = next_rstd;
        float xh[NV][VE], gg[NV][VE], s[2] = {0.f, 0.f};
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < VE; ++i) {
                xh[j][i] = nx[j].get(i);
                gg[j][i] = ng[j].get(i);
            }
        if (kAhead && row + step < a.rows) fetch(row + step);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if (!kKeep) load_param(a.gamma, cols[j], 1.f, gm[j]);
#pragma unroll
            for (int i = 0; i < VE; ++i) {
                xh[j][i] = (xh[j][i] - mean) * rstd;
                const float gy = own<NV>(cols[j], j, i, gg[j][i]);
                dg[j][i] += gy * xh[j][i];
                db[j][i] += gy;
                gg[j][i] *= gm[j][i];
                const float kept = own<NV>(cols[j], j, i, gg[j][i]);
                s[0] += kept;
                s[1] += kept * xh[j][i];
            }
        }
        team_sum<LANES>(s, red);
        const float s0 = s[0] * inv_n, s1 = s[1] * inv_n;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if (!cols[j].hi) continue;
            float o[VE];
#pragma unroll
            for (int i = 0; i < VE; ++i) o[i] = rstd * (gg[j][i] - s0 - xh[j][i] * s1);
            store_cols(gx + row * a.ld_x, cols[j], o);
        }
    }
    if (!a.part) return;
    float* part = a.part + (long long)blockIdx.x * 2 * a.n;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            float v[VE];
#pragma unroll
            for (int i = 0; i < VE; ++i) v[i] = k ? db[j][i] : dg[j][i];
            if constexpr (TEAMS > 1) {                // the teams of a wave, then the waves
#pragma unroll
                for (int o = LANES; o < 64; o *= 2)
#pragma unroll
                    for (int i = 0; i < VE; ++i) v[i] += __shfl_xor(v[i], o);
                __syncthreads();
                if ((threadIdx.x & 63) < LANES)
#pragma unroll
                    for (int i = 0; i < VE; ++i) fold[threadIdx.x >> 6][lane * VE + i] = v[i];
                __syncthreads();
                if (team == 0) {
#pragma unroll
                    for (int i = 0; i < VE; ++i)
#pragma unroll
                        for (int w = 1; w < kNormThreads / 64; ++w) v[i] += fold[w][lane * VE + i];
                }
            }
            if (team == 0) {
#pragma unroll
                for (int i = 0; i < VE; ++i)
                    if (cols[j].counts[i]) part[k * a.n + cols[j].col + i] = v[i];
            }
        }
    }
}

// Column sums of n_part partial sums [n_part][2][n]; 32 columns and 32 groups of partials a workgroup.
__global__ __launch_bounds__(1024) void norm_reduce_kernel(const float* __restrict__ part, int n_part, long long n, float* g_gamma,
                                                           float* g_beta) {
    __shared__ float red[32][33];
    const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5;
    const long long col = group_of_grid() * 32 + tx;
    float s = 0.f;
    if (col < 2 * n)
#pragma unroll 8
        for (int w = ty; w < n_part; w += 32) s += part[(long long)w * 2 * n + col];
    red[ty][tx] = s;
    __syncthreads();
    if (ty == 0 && col < 2 * n) {
        for (int k = 1; k < 32; ++k) s += red[k][tx];
        if (col < n) {
            if (g_gamma) g_gamma[col] = s;
        } else {
            if (g_beta) g_beta[col - n] = s;
        }
    }
}

// ------------------------------------------------------------------ rows longer than the registers of a workgroup
constexpr int kLongThreads = 1024;

// f(first column, columns) of the vectors of a row that are this thread's.
template <class T, class F>
__device__ __forceinline__ void each_vector(long long n, F&& f) {
    constexpr int VE = vec_of<T>();
    for (long long c = (long long)threadIdx.x * VE; c < n; c += (long long)kLongThreads * VE) f(c, n - c < VE ? (int)(n - c) : VE);
}
template <class T>
__device__ __forceinline__ void load_some(const T* p, int left, float* v) {
    constexpr int VE = vec_of<T>();
    if (left == VE) {
        Pack<T, VE> x;
        x.load(p);
#pragma unroll
        for (int i = 0; i < VE; ++i) v[i] = x.get(i);
    } else {
#pragma unroll
        for (int i = 0; i < VE; ++i) v[i] = i < left ? to_f32(p[i]) : 0.f;
    }
}
template <class T>
__device__ __forceinline__ void store_some(T* p, int left, const float* v) {
    constexpr int VE = vec_of<T>();
    if (left == VE) {
        Pack<T, VE> x;
        x.set(v);
        x.store(p);
    } else {
#pragma unroll
        for (int i = 0; i < VE; ++i)
            if (i < left) put_f32(p + i, v[i]);
    }
}

// One workgroup a row, the row read three times (from the cache after the first, up to its size).
template <class T>
__global__ __launch_bounds__(kLongThreads) void norm_fwd_long_kernel(NormArgs a) {
    constexpr int VE = vec_of<T>();
    __shared__ float red[2 * kLongThreads / 64];
    const long long row = group_of_grid();
    if (row >= a.rows) return;
    const T* x = (const T*)a.x + row * a.ld_x;
    T* y = (T*)a.out + row * a.ld_y;
    const float inv_n = 1.f / (float)a.n;
    float s[1] = {0.f}, v[VE];
    each_vector<T>(a.n, [&](long long c, int left) {
        load_some(x + c, left, v);
#pragma unroll
        for (int i = 0; i < VE; ++i) s[0] += i < left ? v[i] * inv_n : 0.f;
    });
    team_sum<kLongThreads>(s, red);
    const float first_mean = s[0];
    float t[2] = {0.f, 0.f};
    each_vector<T>(a.n, [&](long long c, int left) {
        load_some(x + c, left, v);
#pragma unroll
        for (int i = 0; i < VE; ++i) {
            const float d = i < left ? v[i] - first_mean : 0.f;
            t[0] += d * inv_n;
            t[1] += d * d;
        }
    });
    team_sum<kLongThreads>(t, red);
    const float mean = mean_of(first_mean, t[0]);
    float var;
    if (!variance_of(t, inv_n, var)) {
        s[0] = 0.f;
        each_vector<T>(a.n, [&](long long c, int left) {
            load_some(x + c, left, v);
#pragma unroll
            for (int i = 0; i < VE; ++i) s[0] += i < left ? (v[i] - mean) * (v[i] - mean) : 0.f;
        });
        team_sum<kLongThreads>(s, red);
        var = s[0] * inv_n;
    }
    const float rstd = 1.f / sqrtf(var + a.eps);
    each_vector<T>(a.n, [&](long long c, int left) {
        load_some(x + c, left, v);
#pragma unroll
        for (int i = 0; i < VE; ++i)
            if (i < left) v[i] = (v[i] - mean) * rstd * (a.gamma ? a.gamma[c + i] : 1.f) + (a.beta ? a.beta[c + i] : 0.f);
        store_some(y + c, left, v);
    });
    if (threadIdx.x == 0) {
        if (a.mean) a.mean[row] = mean;
        if (a.rstd) a.rstd[row] = rstd;
    }
}

template <class T>
__global__ __launch_bounds__(kLongThreads) void norm_bwd_long_kernel(NormArgs a) {
    constexpr int VE = vec_of<T>();
    __shared__ float red[2 * kLongThreads / 64];
    const long long row = group_of_grid();
    if (row >= a.rows) return;
    const T *x = (const T*)a.x + row * a.ld_x, *g = (const T*)a.g + row * a.ld_y;
    T* gx = (T*)a.out + row * a.ld_x;
    const float inv_n = 1.f / (float)a.n, mean = a.mean_in[row], rstd = a.rstd_in[row];
    float s[2] = {0.f, 0.f}, v[VE], w[VE];
    auto load = [&](long long c, int left) {          // normalised values and g gamma
        load_some(x + c, left, v);
        load_some(g + c, left, w);
#pragma unroll
        for (int i = 0; i < VE; ++i) {
            v[i] = (v[i] - mean) * rstd;
            if (i < left && a.gamma) w[i] *= a.gamma[c + i];
        }
    };
    each_vector<T>(a.n, [&](long long c, int left) {
        load(c, left);
#pragma unroll
        for (int i = 0; i < VE; ++i) {
            s[0] += i < left ? w[i] : 0.f;
            s[1] += i < left ? w[i] * v[i] : 0.f;
        }
    });
    team_sum<kLongThreads>(s, red);
    each_vector<T>(a.n, [&](long long c, int left) {
        load(c, left);
#pragma unroll
        for (int i = 0; i < VE; ++i) w[i] = rstd * (w[i] - s[0] * inv_n - v[i] * (s[1] * inv_n));
        store_some(gx + c, left, w);
    });
}

// Partial sums over rows blockIdx.y, + gridDim.y, ...: one column a thread.  Runs before norm_bwd_long_kernel, whose output may
// take the place of g.
template <class T>
__global__ __launch_bounds__(kNormThreads) void norm_cols_kernel(NormArgs a) {
    const long long c = (long long)blockIdx.x * kNormThreads + threadIdx.x;
    if (c >= a.n) return;
    float dg = 0.f, db = 0.f;
    for (long long row = blockIdx.y; row < a.rows; row += gridDim.y) {
        const float g = to_f32(((const T*)a.g)[row * a.ld_y + c]);
        dg += g * ((to_f32(((const T*)a.x)[row * a.ld_x + c]) - a.mean_in[row]) * a.rstd_in[row]);
        db += g;
    }
    float* part = a.part + (long long)blockIdx.y * 2 * a.n;
    part[c] = dg;
    part[a.n + c] = db;
}

// ------------------------------------------------------------------ choice of the team
// The smallest team whose lanes hold the row in one vector each, up to a wave; then more vectors a lane, then the workgroup.
struct Team {
    int lanes, nv;
};
Team team_for(const gleam_layer_norm_desc& d) {
    const long long units = (d.n * (d.dtype ? 2 : 4) + 15) / 16;
    for (Team t : {Team{4, 1}, Team{8, 1}, Team{16, 1}, Team{32, 1}, Team{64, 1}, Team{64, 2}, Team{64, 4}, Team{256, 2}, Team{256, 4},
                   Team{512, 3}, Team{1024, 2}, Team{1024, d.dtype ? 0 : 4}})
        if (units <= (long long)t.lanes * t.nv) return t;
    return Team{0, 0};
}
// Workgroups that walk the rows.  Backward: every one leaves 2 n partial sums, so there are no more than keep the chip busy (from 512 lanes on
// 256 against 512 of them: float32 500 x 5001 17 and 25 us, 2000 x 5001 30 and 39, 20000 x 5001 226 and 238, 2000 x 8000 49 and 59, bfloat16
// 500 x 16384 47 and 80, 6000 x 16384 180 and 210).  Forward: 327680 rows of 100 float32 65 us with 2048 workgroups, 62
// with 8192, 69 with one for every eight rows; 60000 of 512 bfloat16 21.8, 21.5, 23.5.
int grid_for(const gleam_layer_norm_desc& d, Team t, bool backward) {
    const long long teams = t.lanes > 64 ? 1 : kNormThreads / t.lanes, wgs = (d.rows + teams - 1) / teams;
    const int most = backward ? (t.lanes >= 512 ? 256 : 1024) : 8192;
    return (int)(wgs < most ? wgs : most);
}
int long_parts(const gleam_layer_norm_desc& d) { return (int)(d.rows < 64 ? d.rows : 64); }

template <class T, class F>
void with_team(Team t, F&& f) {
#define GLEAM_TEAM(L, N) \
    if (t.lanes == L && t.nv == N) return f(std::integral_constant<int, L>{}, std::integral_constant<int, N>{})
    GLEAM_TEAM(4, 1);
    GLEAM_TEAM(8, 1);
    GLEAM_TEAM(16, 1);
    GLEAM_TEAM(32, 1);
    GLEAM_TEAM(64, 1);
    GLEAM_TEAM(64, 2);
    GLEAM_TEAM(64, 4);
    GLEAM_TEAM(256, 2);
    GLEAM_TEAM(256, 4);
    GLEAM_TEAM(512, 3);
    GLEAM_TEAM(1024, 2);
    if constexpr (sizeof(T) == 4) GLEAM_TEAM(1024, 4);
#undef GLEAM_TEAM
}

template <class T>
hipError_t forward(const gleam_layer_norm_desc& d, const NormArgs& a, hipStream_t st) {
    const Team t = team_for(d);
    KernelScope ks("layer_norm_fwd", 7.0 * d.rows * d.n, 2.0 * sizeof(T) * d.rows * d.n, st);
    if (!t.lanes) {
        hipLaunchKernelGGL(norm_fwd_long_kernel<T>, grid_of(d.rows), dim3(kLongThreads), 0, st, a);
        return hipGetLastError();
    }
    with_team<T>(t, [&](auto L, auto N) {
        hipLaunchKernelGGL((norm_fwd_kernel<T, L(), N()>), dim3(grid_for(d, t, false)), dim3(threads_of<L()>()), 0, st, a);
    });
    return hipGetLastError();
}

template <class T>
hipError_t backward(const gleam_layer_norm_desc& d, const NormArgs& a, float* g_gamma, float* g_beta, hipStream_t st) {
    const Team t = team_for(d);
    int parts;
    if (!t.lanes) {
        parts = long_parts(d);
        if (a.part) {
            KernelScope ks("layer_norm_cols", 4.0 * d.rows * d.n, 2.0 * sizeof(T) * d.rows * d.n, st);
            hipLaunchKernelGGL(norm_cols_kernel<T>, dim3((unsigned)((d.n + kNormThreads - 1) / kNormThreads), parts), dim3(kNormThreads), 0, st, a);
        }
        KernelScope ks("layer_norm_bwd", 8.0 * d.rows * d.n, 3.0 * sizeof(T) * d.rows * d.n, st);
        hipLaunchKernelGGL(norm_bwd_long_kernel<T>, grid_of(d.rows), dim3(kLongThreads), 0, st, a);
    } else {
        parts = grid_for(d, t, true);
        KernelScope ks("layer_norm_bwd", 12.0 * d.rows * d.n, 3.0 * sizeof(T) * d.rows * d.n, st);
        with_team<T>(t, [&](auto L, auto N) {
            hipLaunchKernelGGL((norm_bwd_kernel<T, L(), N()>), dim3(parts), dim3(threads_of<L()>()), 0, st, a);
        });
    }
    if (a.part) {
        KernelScope ks("layer_norm_reduce", 2.0 * parts * d.n, 8.0 * parts * d.n, st);
        hipLaunchKernelGGL(norm_reduce_kernel, grid_of((2 * d.n + 31) / 32), dim3(1024), 0, st, (const float*)a.part, parts,
                           (long long)d.n, g_gamma, g_beta);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t layer_norm_forward(const gleam_layer_norm_desc& d, const void* x, const float* gamma, const float* beta, void* y, float* mean,
                              float* rstd, hipStream_t st) {
    NormArgs a{};
    a.x = x;
    a.gamma = gamma;
    a.beta = beta;
    a.out = y;
    a.mean = mean;
    a.rstd = rstd;
    a.rows = d.rows;
    a.n = d.n;
    a.ld_x = d.ld_in;
    a.ld_y = d.ld_out;
    a.eps = d.eps;
    return d.dtype ? forward<unsigned short>(d, a, st) : forward<float>(d, a, st);
}

size_t layer_norm_ws_bytes(const gleam_layer_norm_desc& d) {
    const Team t = team_for(d);
    return (size_t)(t.lanes ? grid_for(d, t, true) : long_parts(d)) * 2 * (size_t)d.n * sizeof(float);
}

hipError_t layer_norm_backward(const gleam_layer_norm_desc& d, const void* x, const float* gamma, const float* mean, const float* rstd,
                               const void* g_y, void* g_x, float* g_gamma, float* g_beta, void* ws, hipStream_t st) {
    NormArgs a{};
    a.x = x;
    a.g = g_y;
    a.gamma = gamma;
    a.mean_in = mean;
    a.rstd_in = rstd;
    a.out = g_x;
    a.part = g_gamma || g_beta ? (float*)ws : nullptr;
    a.rows = d.rows;
    a.n = d.n;
    a.ld_x = d.ld_in;
    a.ld_y = d.ld_out;
    return d.dtype ? backward<unsigned short>(d, a, g_gamma, g_beta, st) : backward<float>(d, a, g_gamma, g_beta, st);
}

}  // namespace gleam
