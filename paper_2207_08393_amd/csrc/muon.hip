// Orthogonalised update of weight matrices (gfx950): momentum, X = u / |u|, Newton-Schulz steps X <- (a I + b A + c A^2) X with A = X X^T of
// the smaller side, and the update of the weights.
//
// A step amplifies small singular values by a = 3.4 and with them what X was rounded by, so products are as good as float32 ones: every
// matrix is kept as three bfloat16 parts (split.h), and a product is six of the bfloat16 matrix cores' (2.7 times as fast as the
// float32 ones at equal work).  Matrices are split once, by the kernel that writes them, and kept as the matrix instruction reads its operands:
// blocks of 32 rows x 16 columns, each 1 KB of a part (half of the columns, row, 8 columns), so that a wave's operand is one access of 16
// bytes a lane, without conflicts in LDS.  X is kept in that form both ways round, since X X^T sums over its columns and (..) X over its rows.
// A and the polynomial B = a I + b A + c A^2 are symmetric: only blocks on and above the diagonal are computed, and written twice.
#include <hip/hip_runtime.h>

#include <cmath>

#include "layer_common.h"
#include "layer_ops.h"
#include "split.h"

namespace gleam {
namespace {

constexpr int kBlockBytes = 1024;          // a part of 32 x 16
constexpr int kMuonNorms = 128;            // partial sums of |u|^2 of a matrix, at most

struct MuonArgs {
    float *theta, *m;
    const float* grad;
    double* norms;                         // [matrix][kMuonNorms]
    char *x, *xt, *xt_out, *a, *b;         // parts of X [short][long], of its transpose, of A and B
    long long stride, count;
    int rows, cols, tall;                  // tall: X is the transpose of u
    int mb, nb;                            // blocks of 32 of the short and of the long side
    int parts;                             // partial sums of |u|^2
    int nesterov, last;
    float lr_scale, decay, momentum, eps, ca, cb, cc;
};

// A matrix of R x K blocks of 32 x 32: part p of the 16 columns k16 of rows 32 r ..
__device__ __forceinline__ char* block_at(char* base, long long matrix, int R, int K, int r, int k16, int p) {
    return base + (((matrix * R + r) * (2 * K) + k16) * 3 + p) * kBlockBytes;
}

// m <- momentum m + g and the partial sums of |u|^2, in 64 bits: squares of float32 numbers stay in range
__global__ __launch_bounds__(256) void muon_momentum_kernel(MuonArgs a) {
    __shared__ double red[4];
    const long long id = group_of_grid(), matrix = id / a.parts;
    const int part = (int)(id - matrix * a.parts);
    if (matrix >= a.count) return;
    const long long size = (long long)a.rows * a.cols;
    const float* g = a.grad + matrix * a.stride;
    float* m = a.m + matrix * a.stride;
    double sum = 0.0;
    for (long long e = part * 256 + threadIdx.x; e < size; e += a.parts * 256) {
        const float gv = g[e], mv = __builtin_fmaf(a.momentum, m[e], gv);
        m[e] = mv;
        const double u = a.nesterov ? __builtin_fmaf(a.momentum, mv, gv) : mv;
        sum += u * u;
    }
    for (int o = 1; o < 64; o *= 2) sum += __shfl_xor(sum, o);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) a.norms[matrix * kMuonNorms + part] = (red[0] + red[1]) + (red[2] + red[3]);
}

// The parts of 8 values in a row, to block + offset of each part.
__device__ __forceinline__ void store_parts8(char* block, const float* v) {
    SplitWords s;
#pragma unroll
    for (int i = 0; i < 4; ++i) split_pair(v[2 * i], v[2 * i + 1], i, s);
#pragma unroll
    for (int p = 0; p < 3; ++p) *(uint4*)(block + p * kBlockBytes) = make_uint4(s.w[p][0], s.w[p][1], s.w[p][2], s.w[p][3]);
}

// X = u / (|u| + eps), both ways round; a workgroup takes blocks of 32 x 32.
__global__ __launch_bounds__(128) void muon_split_kernel(MuonArgs a) {
    __shared__ float tile[32][33];
    const long long id = group_of_grid(), per = (long long)a.mb * a.nb, matrix = id / per;
    if (matrix >= a.count) return;
    const int at = (int)(id - matrix * per), bi = at / a.nb, bj = at - bi * a.nb;   // of X
    double norm = 0.0;
    for (int i = 0; i < a.parts; ++i) norm += a.norms[matrix * kMuonNorms + i];
    const float scale = (float)(1.0 / (sqrt(norm) + (double)a.eps));
    const float *g = a.grad + matrix * a.stride, *m = a.m + matrix * a.stride;
    const int r0 = 32 * (a.tall ? bj : bi), c0 = 32 * (a.tall ? bi : bj);           // of u
    for (int e = threadIdx.x; e < 1024; e += 128) {
        const int r = e >> 5, c = e & 31;
        float u = 0.f;
        if (r0 + r < a.rows && c0 + c < a.cols) {
            const long long o = (long long)(r0 + r) * a.cols + c0 + c;
            u = m[o];
            if (a.nesterov) u = __builtin_fmaf(a.momentum, u, g[o]);
            u *= scale;
        }
        tile[a.tall ? c : r][a.tall ? r : c] = u;
    }
    __syncthreads();
    const int line = threadIdx.x & 31, k8 = threadIdx.x >> 5;   // a row, or column, and which 8 of its values
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = tile[line][8 * k8 + i];
    store_parts8(block_at(a.x, matrix, a.mb, a.nb, bi, 2 * bj + (k8 >> 1), 0) + (k8 & 1) * 512 + line * 16, v);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = tile[8 * k8 + i][line];
    store_parts8(block_at(a.xt, matrix, a.nb, a.mb, bj, 2 * bi + (k8 >> 1), 0) + (k8 & 1) * 512 + line * 16, v);
}

enum MuonProduct { kGram, kSquare, kApply };

// One of the three products of a step, rows of the left operand against rows of the right one:
//   kGram  A = X X^T;   kSquare  B = a I + b A + c A A;   kApply  X <- B X, or at the last step the weights' update.
// A workgroup computes 2 WT x 2 WT blocks of 32 x 32, its four waves WT x WT each.
template <int MODE, int WT>
__global__ __launch_bounds__(256) void muon_product_kernel(MuonArgs a) {
    const int R = a.mb, Cb = MODE == kApply ? a.nb : a.mb, K = MODE == kGram ? a.nb : a.mb;   // blocks of the result's sides and of the sum
    const int tr = (R + 2 * WT - 1) / (2 * WT), tc = (Cb + 2 * WT - 1) / (2 * WT);
    const long long id = group_of_grid(), matrix = id / ((long long)tr * tc);
    if (matrix >= a.count) return;
    const int tile = (int)(id - matrix * tr * tc), ti = tile / tc, tj = tile - ti * tc;
    if (MODE != kApply && ti > tj) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int bi0 = ti * 2 * WT + (wave >> 1) * WT, bj0 = tj * 2 * WT + (wave & 1) * WT;
    char* left = MODE == kGram ? a.x : MODE == kSquare ? a.a : a.b;
    char* right = MODE == kGram ? a.x : MODE == kSquare ? a.a : a.xt;
    const char *pl[WT], *pr[WT];
#pragma unroll
    for (int w = 0; w < WT; ++w) {   // blocks past the end: the last one's, computed and not written
        pl[w] = block_at(left, matrix, R, K, min(bi0 + w, R - 1), 0, 0) + lane * 16;
        pr[w] = block_at(right, matrix, Cb, K, min(bj0 + w, Cb - 1), 0, 0) + lane * 16;
    }
    floatx16 acc[WT][WT];
#pragma unroll
    for (int i = 0; i < WT; ++i)
#pragma unroll
        for (int j = 0; j < WT; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
    for (int k = 0; k < 2 * K; ++k) {
        bf16x8 l[WT][3], r[WT][3];
#pragma unroll
        for (int w = 0; w < WT; ++w)
#pragma unroll
            for (int p = 0; p < 3; ++p) {
                l[w][p] = *(const bf16x8*)(pl[w] + (k * 3 + p) * kBlockBytes);
                r[w][p] = *(const bf16x8*)(pr[w] + (k * 3 + p) * kBlockBytes);
            }
#pragma unroll
        for (int q = 0; q < kProducts; ++q)
#pragma unroll
            for (int i = 0; i < WT; ++i)
#pragma unroll
                for (int j = 0; j < WT; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(l[i][kPartA[q]], r[j][kPartB[q]], acc[i][j], 0, 0, 0);
    }
    // lane: column lane % 32 of the result's block, rows 8 q + 4 (lane / 32) + 0..3 in registers 4 q + 0..3
    const int col = lane & 31, up = lane >> 5;
#pragma unroll
    for (int i = 0; i < WT; ++i)
#pragma unroll
        for (int j = 0; j < WT; ++j) {
            const int bi = bi0 + i, bj = bj0 + j;
            if (bi >= R || bj >= Cb || (MODE != kApply && bi > bj)) continue;
            char* across = MODE == kGram ? a.a : MODE == kSquare ? a.b : a.xt_out;   // [column][row] parts
            char* along = MODE == kGram ? a.a : MODE == kSquare ? a.b : a.x;         // [row][column] parts
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                float v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = acc[i][j][4 * q + e];
                const int row0 = 8 * q + 4 * up;
                const long long to = (q & 1) * 512 + col * 16 + up * 8;
                if (MODE == kSquare) {
                    const char* from = block_at(a.a, matrix, R, R, bj, 2 * bi + (q >> 1), 0) + to;   // A is symmetric
                    uint2 w[3];
#pragma unroll
                    for (int p = 0; p < 3; ++p) w[p] = *(const uint2*)(from + p * kBlockBytes);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        float av = 0.f;
#pragma unroll
                        for (int p = 2; p >= 0; --p) {
                            const unsigned u = e < 2 ? w[p].x : w[p].y;
                            av += __uint_as_float(e & 1 ? u & 0xffff0000u : u << 16);
                        }
                        v[e] = a.cb * av + a.cc * v[e] + (bi == bj && row0 + e == col ? a.ca : 0.f);
                    }
                }
                if (MODE == kApply && a.last) {
                    const int r = 32 * bi + row0, c = 32 * bj + col;
                    float* th = a.theta + matrix * a.stride;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int ur = a.tall ? c : r + e, uc = a.tall ? r + e : c;
                        if (ur < a.rows && uc < a.cols) {
                            float* p = th + (long long)ur * a.cols + uc;
                            *p = a.decay * *p - a.lr_scale * v[e];
                        }
                    }
                    continue;
                }
                SplitWords s;
                split_pair(v[0], v[1], 0, s);
                split_pair(v[2], v[3], 1, s);
                char* t = block_at(across, matrix, Cb, R, bj, 2 * bi + (q >> 1), 0) + to;
#pragma unroll
                for (int p = 0; p < 3; ++p) *(uint2*)(t + p * kBlockBytes) = make_uint2(s.w[p][0], s.w[p][1]);
                if (MODE != kApply && bi == bj) continue;
                char* d = block_at(along, matrix, R, Cb, bi, 2 * bj + (col >> 4), 0) + ((col >> 3) & 1) * 512 + row0 * 16 + (col & 7) * 2;
#pragma unroll
                for (int p = 0; p < 3; ++p)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        *(unsigned short*)(d + p * kBlockBytes + e * 16) = (unsigned short)(s.w[p][e >> 1] >> (e & 1 ? 16 : 0));
            }
        }
}

struct MuonPlan {
    int mb, nb, parts;
    size_t x_bytes, a_bytes, norm_bytes;
};
MuonPlan plan_of(long long count, long long rows, long long cols) {
    MuonPlan p;
    const long long m = rows < cols ? rows : cols, n = rows < cols ? cols : rows;
    p.mb = (int)((m + 31) / 32);
    p.nb = (int)((n + 31) / 32);
    const long long parts = (rows * cols + 2047) / 2048;
    p.parts = (int)(parts < kMuonNorms ? parts : kMuonNorms);
    p.x_bytes = (size_t)count * p.mb * p.nb * 6 * kBlockBytes;
    p.a_bytes = (size_t)count * p.mb * p.mb * 6 * kBlockBytes;
    p.norm_bytes = (size_t)count * kMuonNorms * sizeof(double);
    return p;
}

template <int MODE>
void launch_product(const MuonArgs& a, hipStream_t st) {
    const long long R = a.mb, C = MODE == kApply ? a.nb : a.mb, K = MODE == kGram ? a.nb : a.mb;
    const double work = 2.0 * 32768.0 * R * C * K * a.count;
    KernelScope ks(MODE == kGram ? "muon_gram" : MODE == kSquare ? "muon_square" : "muon_apply", work, 0.0, st, 6.0 * work);
    hipLaunchKernelGGL((muon_product_kernel<MODE, 1>), grid_of(a.count * ((R + 1) / 2) * ((C + 1) / 2)), dim3(256), 0, st, a);
}

}  // namespace

size_t muon_ws_bytes(long long count, long long rows, long long cols) {
    const MuonPlan p = plan_of(count, rows, cols);
    return 3 * p.x_bytes + 2 * p.a_bytes + p.norm_bytes;
}

hipError_t muon_update(const gleam_muon& h, long long count, long long rows, long long cols, long long stride, float* theta,
                       const float* grad, float* m, void* ws, hipStream_t st) {
    const MuonPlan p = plan_of(count, rows, cols);
    MuonArgs a{};
    a.theta = theta;
    a.grad = grad;
    a.m = m;
    char* at = (char*)ws;
    a.x = at;
    a.xt = at + p.x_bytes;
    a.xt_out = at + 2 * p.x_bytes;
    a.a = at + 3 * p.x_bytes;
    a.b = a.a + p.a_bytes;
    a.norms = (double*)(a.b + p.a_bytes);
    a.stride = stride;
    a.count = count;
    a.rows = (int)rows;
    a.cols = (int)cols;
    a.tall = rows > cols;
    a.mb = p.mb;
    a.nb = p.nb;
    a.parts = p.parts;
    a.nesterov = h.nesterov;
    a.lr_scale = (float)((double)h.lr * std::sqrt(a.tall ? (double)rows / (double)cols : 1.0));
    a.decay = (float)(1.0 - (double)h.lr * h.weight_decay);
    a.momentum = h.momentum;
    a.eps = h.eps;
    a.ca = h.a;
    a.cb = h.b;
    a.cc = h.c;
    {
        KernelScope ks("muon_momentum", 4.0 * count * rows * cols, 12.0 * count * rows * cols, st);
        hipLaunchKernelGGL(muon_momentum_kernel, grid_of(count * p.parts), dim3(256), 0, st, a);
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    {
        KernelScope ks("muon_split", 0.0, 20.0 * count * rows * cols, st);
        hipLaunchKernelGGL(muon_split_kernel, grid_of(count * p.mb * p.nb), dim3(128), 0, st, a);
    }
    e = hipGetLastError();
    for (int k = 0; k < h.steps && e == hipSuccess; ++k) {
        a.last = k == h.steps - 1;
        launch_product<kGram>(a, st);
        launch_product<kSquare>(a, st);
        launch_product<kApply>(a, st);
        char* t = a.xt;
        a.xt = a.xt_out;
        a.xt_out = t;
        e = hipGetLastError();
    }
    return e;
}

}  // namespace gleam
