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
    float* part;                           // of products split along their sum
    int splits;
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

// What becomes of a 32 x 32 block (bi, bj) of a product, R x Cb blocks in all; `tile`: 32 x 33 floats of LDS of this wave alone.  Lane:
// column lane % 32, rows 8 q + 4 (lane / 32) + 0..3 in registers 4 q + 0..3.
template <int MODE>
__device__ __forceinline__ void put_block(const MuonArgs& a, long long matrix, int bi, int bj, const floatx16& acc, float* tile) {
    const int lane = threadIdx.x & 63, col = lane & 31, up = lane >> 5, R = a.mb, Cb = MODE == kApply ? a.nb : a.mb;
    char* across = MODE == kGram ? a.a : MODE == kSquare ? a.b : a.xt_out;   // [column][row] parts
    char* along = MODE == kGram ? a.a : MODE == kSquare ? a.b : a.x;         // [row][column] parts
    const bool both = MODE == kApply || bi != bj;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = acc[4 * q + e];
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
        if (both)
#pragma unroll
            for (int e = 0; e < 4; ++e) tile[(row0 + e) * 33 + col] = v[e];
    }
    if (!both || (MODE == kApply && a.last)) return;
    // the other way round: a row and eight of its columns a lane
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int g = 0; g < 2; ++g) {
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = tile[col * 33 + 8 * (up + 2 * g) + e];
        store_parts8(block_at(along, matrix, R, Cb, bi, 2 * bj + g, 0) + up * 512 + col * 16, v);
    }
    __builtin_amdgcn_wave_barrier();
}

// One of the three products of a step, rows of the left operand against rows of the right one:
//   kGram  A = X X^T;   kSquare  B = a I + b A + c A A;   kApply  X <- B X, or at the last step the weights' update.
// A workgroup computes 2 WT x 2 WT blocks of 32 x 32, its four waves WT x WT each, over one of `splits` parts of the sum.  16 columns of both
// operands are in LDS (24 KB for WT = 2) while the next 16 are written and the ones after those are on their way in registers.
constexpr int kTileFloats = 32 * 33;

template <int MODE, int WT>
__global__ __launch_bounds__(256, 2) void muon_product_kernel(MuonArgs a) {
    constexpr int kRows = 2 * WT, kStage = 2 * kRows * 3 * kBlockBytes, kLoads = kStage / (256 * 16);   // row blocks of an operand in a tile
    constexpr int kLds = 2 * kStage > 4 * kTileFloats * 4 ? 2 * kStage : 4 * kTileFloats * 4;
    __shared__ __attribute__((aligned(16))) char lds[kLds];
    const int R = a.mb, Cb = MODE == kApply ? a.nb : a.mb, K = MODE == kGram ? a.nb : a.mb;   // blocks of the result's sides and of the sum
    const int tr = (R + kRows - 1) / kRows, tc = (Cb + kRows - 1) / kRows;
    const long long id = group_of_grid(), all = (long long)tr * tc * a.splits, matrix = id / all;
    if (matrix >= a.count) return;
    const int rest = (int)(id - matrix * all), split = rest % a.splits, tile = rest / a.splits, ti = tile / tc, tj = tile - ti * tc;
    if (MODE != kApply && ti > tj) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wi = wave >> 1, wj = wave & 1;
    const char* left = MODE == kGram ? a.x : MODE == kSquare ? a.a : a.b;
    const char* right = MODE == kGram ? a.x : MODE == kSquare ? a.a : a.xt;
    // loads: wave w takes the 1 KB pieces w, w + 4, ... of a stage: operand, row block, part
    const char* src[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        const int piece = wave + 4 * i, op = piece / (kRows * 3), rb = piece / 3 % kRows, p = piece % 3;
        const int r = op ? min(tj * kRows + rb, Cb - 1) : min(ti * kRows + rb, R - 1);   // blocks past the end: the last one's, not written
        src[i] = block_at((char*)(op ? right : left), matrix, op ? Cb : R, K, r, 0, p) + lane * 16;
    }
    const int steps = 2 * K, k0 = (int)((long long)steps * split / a.splits), k1 = (int)((long long)steps * (split + 1) / a.splits);
    uint4v in[2][kLoads];
    auto load = [&](int k, uint4v (&to)[kLoads]) {
        const long long off = (long long)min(k, k1 - 1) * 3 * kBlockBytes;   // past the end: the last again, not used
#pragma unroll
        for (int i = 0; i < kLoads; ++i) to[i] = *(const uint4v*)(src[i] + off);
    };
    auto store = [&](int buf, const uint4v (&from)[kLoads]) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) *(uint4v*)(lds + buf * kStage + (wave + 4 * i) * kBlockBytes + lane * 16) = from[i];
    };
    floatx16 acc[WT][WT];
#pragma unroll
    for (int i = 0; i < WT; ++i)
#pragma unroll
        for (int j = 0; j < WT; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
    auto compute = [&](int buf) {
        bf16x8 l[WT][3], r[WT][3];
        const char* base = lds + buf * kStage + lane * 16;
#pragma unroll
        for (int w = 0; w < WT; ++w)
#pragma unroll
            for (int p = 0; p < 3; ++p) {
                l[w][p] = *(const bf16x8*)(base + ((wi * WT + w) * 3 + p) * kBlockBytes);
                r[w][p] = *(const bf16x8*)(base + ((kRows + wj * WT + w) * 3 + p) * kBlockBytes);
            }
#pragma unroll
        for (int q = 0; q < kProducts; ++q)
#pragma unroll
            for (int i = 0; i < WT; ++i)
#pragma unroll
                for (int j = 0; j < WT; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(l[i][kPartA[q]], r[j][kPartB[q]], acc[i][j], 0, 0, 0);
    };
    load(k0, in[0]);
    load(k0 + 1, in[1]);
    store(0, in[0]);
    load(k0 + 2, in[0]);
    __syncthreads();
    for (int k = k0; k < k1; k += 2) {   // stage k is in buffer 0, k + 1 in registers 1, k + 2 in registers 0
        store(1, in[1]);
        load(k + 3, in[1]);
        compute(0);
        __syncthreads();
        if (k + 1 == k1) break;
        store(0, in[0]);
        load(k + 4, in[0]);
        compute(1);
        __syncthreads();
    }
    if (a.splits > 1) {   // as the registers have it: [matrix][tile][split][wave][block][register][lane]
        float* part = a.part + (((matrix * tr * tc + tile) * a.splits + split) * 4 + wave) * (WT * WT * 1024) + lane;
#pragma unroll
        for (int i = 0; i < WT; ++i)
#pragma unroll
            for (int j = 0; j < WT; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r) part[((i * WT + j) * 16 + r) * 64] = acc[i][j][r];
        return;
    }
    // every wave is past its last reads of the operands (the loop ends with a barrier)
#pragma unroll
    for (int i = 0; i < WT; ++i)
#pragma unroll
        for (int j = 0; j < WT; ++j) {
            const int bi = (ti * 2 + wi) * WT + i, bj = (tj * 2 + wj) * WT + j;
            if (bi < R && bj < Cb && (MODE == kApply || bi <= bj)) put_block<MODE>(a, matrix, bi, bj, acc[i][j], (float*)lds + wave * kTileFloats);
        }
}

// Sums the parts of a split product, a wave a block, in order.
template <int MODE, int WT>
__global__ __launch_bounds__(64) void muon_join_kernel(MuonArgs a) {
    __shared__ float lds[kTileFloats];
    constexpr int kBlocks = 4 * WT * WT;
    const int R = a.mb, Cb = MODE == kApply ? a.nb : a.mb, tr = (R + 2 * WT - 1) / (2 * WT), tc = (Cb + 2 * WT - 1) / (2 * WT);
    const long long id = group_of_grid(), tile_id = id / kBlocks, matrix = tile_id / ((long long)tr * tc);
    if (matrix >= a.count) return;
    const int block = (int)(id - tile_id * kBlocks), tile = (int)(tile_id - matrix * tr * tc), ti = tile / tc, tj = tile - ti * tc;
    const int wave = block / (WT * WT), i = block / WT % WT, j = block % WT;
    const int bi = (ti * 2 + (wave >> 1)) * WT + i, bj = (tj * 2 + (wave & 1)) * WT + j;
    if (bi >= R || bj >= Cb || (MODE != kApply && bi > bj)) return;
    const float* part = a.part + tile_id * a.splits * (kBlocks * 1024) + block * 1024 + (threadIdx.x & 63);
    floatx16 acc;
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[r] = part[r * 64];
    for (int s = 1; s < a.splits; ++s) {
        part += kBlocks * 1024;
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[r] += part[r * 64];
    }
    put_block<MODE>(a, matrix, bi, bj, acc, lds);
}

// Blocks of a wave's side, and parts of the sum: a product of few tiles is split so that the chip has two workgroups for each CU, no part
// under four steps.
struct ProductPlan {
    int wt, splits;
    long long tiles;          // of a matrix
};
ProductPlan product_plan(long long count, int mb, int nb, MuonProduct mode) {
    const long long R = mb, C = mode == kApply ? nb : mb, steps = 2LL * (mode == kGram ? nb : mb);
    ProductPlan p;
    p.wt = mb <= 2 ? 1 : 2;
    const long long tr = (R + 2 * p.wt - 1) / (2 * p.wt), tc = (C + 2 * p.wt - 1) / (2 * p.wt);
    p.tiles = tr * tc;
    const long long work = count * (mode == kApply ? tr * tc : tr * (tr + 1) / 2);
    long long s = 512 / work;
    if (s > steps / 4) s = steps / 4;
    p.splits = (int)(s < 1 ? 1 : s > 32 ? 32 : s);
    return p;
}
size_t part_bytes(long long count, const ProductPlan& p) { return p.splits > 1 ? (size_t)count * p.tiles * p.splits * p.wt * p.wt * 4 * 4096 : 0; }

struct MuonPlan {
    int mb, nb, parts;
    size_t x_bytes, a_bytes, norm_bytes, part_bytes;
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
    p.part_bytes = 0;
    for (MuonProduct mode : {kGram, kSquare, kApply}) {
        const size_t n = part_bytes(count, product_plan(count, p.mb, p.nb, mode));
        if (n > p.part_bytes) p.part_bytes = n;
    }
    return p;
}

template <int MODE, int WT>
void launch_tiles(const MuonArgs& a, const ProductPlan& p, double work, hipStream_t st) {
    {
        KernelScope ks(MODE == kGram ? "muon_gram" : MODE == kSquare ? "muon_square" : "muon_apply", work, 0.0, st, 6.0 * work);
        hipLaunchKernelGGL((muon_product_kernel<MODE, WT>), grid_of(a.count * p.tiles * p.splits), dim3(256), 0, st, a);
    }
    if (p.splits == 1) return;
    KernelScope ks("muon_join", 0.0, (double)part_bytes(a.count, p), st);
    hipLaunchKernelGGL((muon_join_kernel<MODE, WT>), grid_of(a.count * p.tiles * 4 * WT * WT), dim3(64), 0, st, a);
}
template <int MODE>
void launch_product(MuonArgs& a, hipStream_t st) {
    const ProductPlan p = product_plan(a.count, a.mb, a.nb, (MuonProduct)MODE);
    const double R = a.mb, C = MODE == kApply ? a.nb : (a.mb + 1) * 0.5, K = MODE == kGram ? a.nb : a.mb, work = 65536.0 * R * C * K * a.count;
    a.splits = p.splits;
    if (p.wt == 1) launch_tiles<MODE, 1>(a, p, work, st);
    else launch_tiles<MODE, 2>(a, p, work, st);
}

}  // namespace

size_t muon_ws_bytes(long long count, long long rows, long long cols) {
    const MuonPlan p = plan_of(count, rows, cols);
    return 3 * p.x_bytes + 2 * p.a_bytes + p.norm_bytes + p.part_bytes;
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
    a.part = (float*)(a.b + p.a_bytes + p.norm_bytes);
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
