// Orthogonalised update of weight matrices (gfx950): momentum, X = u / |u|, Newton-Schulz steps X <- (a I + b A + c A^2) X with A = X X^T of
// the smaller side, and the update of the weights.
//
// A step amplifies small singular values by a = 3.4 and with them what X was rounded by, so products are made nearly as good as float32 ones: every
// matrix is kept as the sum of two float16 numbers, 11 bits each, and a product is three of the float16 matrix cores' (the product of the two
// second parts, 2^-22 of the whole at most, is left out): 2^-21 where float32 operands bring 2^-23, and the same sums.  After five steps X is 0.4 to 1.7
// times as far from exact as float32 products leave it (30 x 800 to 512 x 2048, noise, strong directions over noise, singular values spread from 1
// to 1e-4).  That is 5 times as fast as the float32 matrix cores, and twice as fast as three
// bfloat16 parts and six products.  Float16 has a range to mind: every matrix is scaled by a power of two that keeps it under 2^15, from the
// largest singular value that the polynomial can make of [0, 1], which the host works out; small second parts may be subnormal.
// Matrices are split once, by the kernel that writes them, and kept as the matrix instruction reads its operands:
// blocks of 32 rows x 16 columns, each 1 KB of a part (half of the columns, row, 8 columns), so that a wave's operand is one access of 16
// bytes a lane, without conflicts in LDS.  X is kept in that form both ways round, since X X^T sums over its columns and (..) X over its rows.
// A and the polynomial B = a I + b A + c A^2 are symmetric: only blocks on and above the diagonal are computed, and written twice.
//
// What bounds it.  Matrices of up to 16 blocks: the latency of six phases a step, one workgroup (192 x 64: 35 us, of which a launch is 6).
// Larger ones: launches and the latency of one wave's share while the chip is not full (24 x 100 x 900: 104 to 109 us, 12 of it bytes and
// matrix instructions), then operands on their way through the L1 caches, 50 bytes a clock and CU (1024 x 4096: X X^T 27 us, 480 TFLOP/s of
// float16 products, B X 36 us, 720 TFLOP/s; a library product of that type reaches 1211),
// and in a product of the short side, 10 us, the 120 CUs that 136 tiles leave without one.  Momentum and split move 12 and 16 bytes an element
// at 4.4 and 5.2 TB/s.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "layer_common.h"
#include "layer_ops.h"

namespace gleam {
namespace {

typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef unsigned uint4v __attribute__((ext_vector_type(4)));
typedef _Float16 halfx8 __attribute__((ext_vector_type(8)));
typedef _Float16 halfx4 __attribute__((ext_vector_type(4)));

constexpr int kBlockBytes = 1024;          // a part of 32 x 16
constexpr int kParts = 2;
constexpr int kMuonNorms = 512;            // partial sums of |u|^2 of a matrix, at most

struct MuonArgs {
    float *theta, *m;
    const float* grad;
    double* norms;                         // [matrix][kMuonNorms]
    char *x, *xt, *xt_out, *a, *b;         // parts of X [short][long], of its transpose, of A and B
    const char *left, *right;              // of a symmetric product, and of kApply the left one
    char* sym;                             // where a symmetric product goes
    int sum;                               // blocks of its sum
    long long stride, count;
    int rows, cols, tall;                  // tall: X is the transpose of u
    int mb, nb;                            // blocks of 32 of the short and of the long side
    int parts;                             // partial sums of |u|^2
    float* part;                           // of products split along their sum
    int splits;
    int nesterov, last, no_square;
    float lr_scale, decay, momentum, eps;
    float turn_scale, q_scale;             // of B A and (B A) B, and of Q
    float x_scale, sym_scale, apply_scale, ca, cb, cc;   // of the sums, so that results have their scale; B = ca I + cc (cb A + A A)
};

// A matrix of R x K blocks of 32 x 32: part p of the 16 columns k16 of rows 32 r ..
__device__ __forceinline__ char* block_at(char* base, long long matrix, int R, int K, int r, int k16, int p) {
    return base + (((matrix * R + r) * (2 * K) + k16) * kParts + p) * kBlockBytes;
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
    // four elements a lane at a time, all requested before the first is used; the end one by one
    const long long quads = size / 4, step = a.parts * 256LL;
    auto one = [&](float gv, float& mv) {
        mv = __builtin_fmaf(a.momentum, mv, gv);
        const double u = a.nesterov ? __builtin_fmaf(a.momentum, mv, gv) : mv;
        sum += u * u;
    };
    for (long long q = part * 256 + threadIdx.x; q < quads; q += 2 * step) {
        const bool more = q + step < quads;
        const long long q2 = more ? q + step : q;
        Pack<float, 4> g0, g1, m0, m1;
        g0.load(g + 4 * q), m0.load(m + 4 * q), g1.load(g + 4 * q2), m1.load(m + 4 * q2);
        float v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) one(g0.get(i), v[i] = m0.get(i));
        m0.set(v);
        m0.store(m + 4 * q);
        if (more) {
#pragma unroll
            for (int i = 0; i < 4; ++i) one(g1.get(i), v[i] = m1.get(i));
            m1.set(v);
            m1.store(m + 4 * q2);
        }
    }
    if (part == 0 && threadIdx.x < size - 4 * quads) {
        const long long e = 4 * quads + threadIdx.x;
        float v = m[e];
        one(g[e], v);
        m[e] = v;
    }
    for (int o = 1; o < 64; o *= 2) sum += __shfl_xor(sum, o);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) a.norms[matrix * kMuonNorms + part] = (red[0] + red[1]) + (red[2] + red[3]);
}

// The parts of 8 values in a row, to block + offset of each part.
__device__ __forceinline__ void store_parts8(char* block, const float* v) {
    halfx8 hi, lo;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        hi[i] = (_Float16)v[i];
        lo[i] = (_Float16)(v[i] - (float)hi[i]);
    }
    *(halfx8*)block = hi;
    *(halfx8*)(block + kBlockBytes) = lo;
}

// X = u / (|u| + eps), both ways round; a workgroup takes blocks of 32 x 32.
__global__ __launch_bounds__(128) void muon_split_kernel(MuonArgs a) {
    __shared__ float tile[32][33];
    const long long id = group_of_grid(), per = (long long)a.mb * a.nb, matrix = id / per;
    if (matrix >= a.count) return;
    const int at = (int)(id - matrix * per), bi = at / a.nb, bj = at - bi * a.nb;   // of X
    const int lane = threadIdx.x & 63;
    double norm = 0.0;
#pragma unroll
    for (int i = 0; i < kMuonNorms; i += 64) norm += lane + i < a.parts ? a.norms[matrix * kMuonNorms + lane + i] : 0.0;
    for (int o = 1; o < 64; o *= 2) norm += __shfl_xor(norm, o);
    const double scale = (double)a.x_scale / (sqrt(norm) + (double)a.eps);   // may lie outside the range of a float32 where u is small
    const float *g = a.grad + matrix * a.stride, *m = a.m + matrix * a.stride;
    const int r0 = 32 * (a.tall ? bj : bi), c0 = 32 * (a.tall ? bi : bj);           // of u
    float mv[8], gv[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int e = threadIdx.x + 128 * i, r = e >> 5, c = e & 31;
        const bool in = r0 + r < a.rows && c0 + c < a.cols;
        const long long o = in ? (long long)(r0 + r) * a.cols + c0 + c : 0;
        mv[i] = in ? m[o] : 0.f;
        gv[i] = in && a.nesterov ? g[o] : 0.f;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int e = threadIdx.x + 128 * i, r = e >> 5, c = e & 31;
        tile[a.tall ? c : r][a.tall ? r : c] = (float)((double)(a.nesterov ? __builtin_fmaf(a.momentum, mv[i], gv[i]) : mv[i]) * scale);
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

enum MuonProduct { kSym, kSquare, kApply };

// Blocks of 32 x 32 on their way out, in LDS: 32 rows of 33 floats.
constexpr int kTileFloats = 32 * 33;

// Lane: column lane % 32, rows 8 q + 4 (lane / 32) + 0..3 in registers 4 q + 0..3.
__device__ __forceinline__ void stage_block(const floatx16& acc, float* tile) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int i = 0; i < 16; ++i) tile[(8 * (i >> 2) + 4 * (lane >> 5) + (i & 3)) * 33 + (lane & 31)] = acc[i];
}

// A block (bi, bj) of a product, R x Cb blocks in all, out of LDS by one wave: the parts of its rows and of its columns, eight values a lane, or
// the weights' update.
template <int MODE>
__device__ __forceinline__ void put_block(const MuonArgs& a, long long matrix, int bi, int bj, const float* tile) {
    const int lane = threadIdx.x & 63, line = lane & 31, up = lane >> 5, R = a.mb, Cb = MODE == kApply ? a.nb : a.mb;
    if (MODE == kApply && a.last) {   // rows of the weights: of X, or its columns; two of them at a time
        const int row0 = 32 * (a.tall ? bj : bi) + up, col = 32 * (a.tall ? bi : bj) + line;
        float* th = a.theta + matrix * a.stride + (long long)row0 * a.cols + col;
        if (col >= a.cols) return;
        float v[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = row0 + 2 * i < a.rows ? th[(long long)2 * i * a.cols] : 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int k = 2 * i + up;
            if (row0 + 2 * i < a.rows) th[(long long)2 * i * a.cols] = a.decay * v[i] - a.lr_scale * tile[a.tall ? line * 33 + k : k * 33 + line];
        }
        return;
    }
    const int sides = MODE == kApply || bi != bj ? 2 : 1;   // a block on the diagonal is its own transpose
#pragma unroll 1
    for (int side = 0; side < sides; ++side) {
        const int sl = side ? 1 : 33, sk = side ? 33 : 1;
        char* out = MODE == kSym ? block_at(a.sym, matrix, R, R, side ? bj : bi, 2 * (side ? bi : bj), 0)
                    : MODE == kSquare ? block_at(a.b, matrix, R, R, side ? bj : bi, 2 * (side ? bi : bj), 0)
                    : side ? block_at(a.xt_out, matrix, Cb, R, bj, 2 * bi, 0) : block_at(a.x, matrix, R, Cb, bi, 2 * bj, 0);
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int k = 8 * (up + 2 * g) + e;
                v[e] = (MODE == kSym ? a.sym_scale : MODE == kSquare ? a.cc : a.apply_scale) * tile[line * sl + k * sk];
                if (MODE == kSquare) v[e] += bi == bj && k == line ? a.ca : 0.f;
            }
            store_parts8(out + g * kParts * kBlockBytes + up * 512 + line * 16, v);
        }
    }
}

// (b / c) A, which A A is added to: c times the sum and a on the diagonal are B.  Registers as the matrix instruction has them; A is symmetric.
__device__ __forceinline__ floatx16 start_of_square(const MuonArgs& a, long long matrix, int bi, int bj) {
    const int lane = threadIdx.x & 63;
    floatx16 acc;
    halfx4 w[4][kParts];
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int p = 0; p < kParts; ++p)
            w[q][p] = *(const halfx4*)(block_at(a.a, matrix, a.mb, a.mb, bj, 2 * bi + (q >> 1), p) + (q & 1) * 512 + (lane & 31) * 16 + (lane >> 5) * 8);
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[i] = a.cb * ((float)w[i >> 2][1][i & 3] + (float)w[i >> 2][0][i & 3]);
    return acc;
}

// The tile of a result that a workgroup computes, and its part of the sum.  Workgroups go round the eight XCDs, each with an L2 of its own:
// an XCD gets neighbours in [matrix][part of the sum][column of tiles][row of tiles], so that its workgroups read the same rows of both
// operands at about the same time.
struct Tile {
    long long matrix, tile;   // tile: of all matrices' stored ones
    int split, ti, tj;
};
template <int MODE>
__device__ __forceinline__ void place_tile(int at, int tr, Tile& t) {
    if (MODE == kApply) {
        t.tj = at / tr;
        t.ti = at - t.tj * tr;
    } else {   // on and above the diagonal, column by column
        t.tj = (int)((sqrtf(8.f * at + 1.f) - 1.f) * 0.5f);
        if (t.tj * (t.tj + 1) / 2 > at) --t.tj;
        if ((t.tj + 1) * (t.tj + 2) / 2 <= at) ++t.tj;
        t.ti = at - t.tj * (t.tj + 1) / 2;
    }
}
template <int MODE>
__device__ __forceinline__ bool find_tile(const MuonArgs& a, int tr, int tc, Tile& t) {
    const unsigned per_split = MODE == kApply ? tr * tc : tr * (tr + 1) / 2, per = per_split * a.splits, all = per * (unsigned)a.count;   // below 2^31
    const unsigned id = (unsigned)group_of_grid(), each = (all + 7) / 8, item = (id & 7) * each + (id >> 3);
    if ((id >> 3) >= each || item >= all) return false;
    const unsigned matrix = item / per, rest = item - matrix * per, split = rest / per_split, at = rest - split * per_split;
    t.matrix = matrix;
    t.split = (int)split;
    place_tile<MODE>((int)at, tr, t);
    t.tile = (long long)matrix * per_split + at;
    return true;
}

// One of the products of a step, rows of the left operand against rows of the right one:
//   kSym  A = X X^T, or a product of two symmetric matrices that commute;   kSquare  B = a I + b A + c A A;   kApply  X <- B X, or at the end
//   the weights' update.
// A workgroup computes 2 x 2 blocks of 32 x 32 over one of `splits` parts of the sum, and each of its four waves all of them over every fourth step of that: no
// operand is needed by two waves, so they go from memory into registers as they lie there, kAhead steps of 16 columns before their use, with
// no barrier until the four sums meet in LDS.  Short sums (SHORT) are not shared out: a wave computes one block, and the waves do not meet.
constexpr int kProducts = 3;
__device__ constexpr int kPartA[kProducts] = {1, 0, 0}, kPartB[kProducts] = {0, 1, 0};   // small ones first

template <int MODE, bool SHORT>
__global__ __launch_bounds__(256, 2) void muon_product_kernel(MuonArgs a) {
    constexpr int kAhead = 3, W = SHORT ? 1 : 2;   // blocks of a wave's sides
    __shared__ __attribute__((aligned(16))) float lds[4][SHORT ? 1 : 4][kTileFloats];
    const int R = a.mb, Cb = MODE == kApply ? a.nb : a.mb, K = MODE == kSym ? a.sum : a.mb;   // blocks of the result's sides and of the sum
    Tile t;
    if (!find_tile<MODE>(a, (R + 1) / 2, (Cb + 1) / 2, t)) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const char* left = MODE == kSquare ? a.a : a.left;
    const char* right = MODE == kSym ? a.right : MODE == kSquare ? a.a : a.xt;
    // steps k0, k0 + kEvery ..: the waves go through the sum side by side, so that workgroups that share rows read them at about the same time
    constexpr int kEvery = SHORT ? 1 : 4;
    const int s0 = (int)((long long)2 * K * t.split / a.splits), s1 = (int)((long long)2 * K * (t.split + 1) / a.splits);
    const int k0 = SHORT ? s0 : s0 + wave;
    const int bi = 2 * t.ti + (wave >> 1), bj = 2 * t.tj + (wave & 1);   // the block that this wave writes
    const bool mine = bi < R && bj < Cb && (MODE == kApply || bi <= bj);
    if (SHORT && !mine) return;
    const char *pl[W], *pr[W];   // blocks past the end: the last one's, computed and not written
#pragma unroll
    for (int w = 0; w < W; ++w) pl[w] = block_at((char*)left, t.matrix, R, K, SHORT ? bi : min(2 * t.ti + w, R - 1), k0, 0) + lane * 16;
#pragma unroll
    for (int w = 0; w < W; ++w) pr[w] = block_at((char*)right, t.matrix, Cb, K, SHORT ? bj : min(2 * t.tj + w, Cb - 1), k0, 0) + lane * 16;
    floatx16 acc[W][W];
#pragma unroll
    for (int i = 0; i < W; ++i)
#pragma unroll
        for (int j = 0; j < W; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
    const int steps = MODE == kSquare && a.no_square ? 0 : (s1 - k0 + kEvery - 1) / kEvery;
    halfx8 l[kAhead][W][kParts], r[kAhead][W][kParts];
    auto load = [&](int k, int at) {
        const int off = min(k, steps - 1) * (kEvery * kParts * kBlockBytes);   // past the end: the last again, not used
#pragma unroll
        for (int p = 0; p < kParts; ++p) {
#pragma unroll
            for (int w = 0; w < W; ++w) l[at][w][p] = *(const halfx8*)(pl[w] + off + p * kBlockBytes);
#pragma unroll
            for (int w = 0; w < W; ++w) r[at][w][p] = *(const halfx8*)(pr[w] + off + p * kBlockBytes);
        }
    };
    auto multiply = [&](int at) {
#pragma unroll
        for (int q = 0; q < kProducts; ++q)
#pragma unroll
            for (int i = 0; i < W; ++i)
#pragma unroll
                for (int j = 0; j < W; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(l[at][i][kPartA[q]], r[at][j][kPartB[q]], acc[i][j], 0, 0, 0);
    };
    if (steps > 0) {
#pragma unroll
        for (int i = 0; i < kAhead - 1; ++i) load(i, i);
        int k = 0;
        for (; k + kAhead <= steps; k += kAhead)
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {   // requests, into the operands of the step before, among the matrix instructions
                load(k + i + kAhead - 1, (i + kAhead - 1) % kAhead);
                multiply(i);
#pragma unroll
                for (int j = 0; j < kProducts * W * W; ++j) {
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                    if (j < kParts * 2 * W) __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
        for (int i = 0; i < kAhead - 1; ++i)
            if (k + i < steps) multiply(i);
    }
    if constexpr (!SHORT)
#pragma unroll
        for (int i = 0; i < W; ++i)
#pragma unroll
            for (int j = 0; j < W; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    *(floatx4*)(lds[wave][i * W + j] + (q * 64 + lane) * 4) = floatx4{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
    floatx16 sum;
    if (MODE == kSquare && mine) sum = start_of_square(a, t.matrix, bi, bj);
    else
#pragma unroll
        for (int i = 0; i < 16; ++i) sum[i] = 0.f;
    if constexpr (SHORT) {
#pragma unroll
        for (int i = 0; i < 16; ++i) sum[i] += acc[0][0][i];
    } else {
        __syncthreads();
        if (!mine) return;
#pragma unroll
        for (int w = 0; w < 4; ++w)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const floatx4 v = *(const floatx4*)(lds[w][wave] + (q * 64 + lane) * 4);
#pragma unroll
                for (int e = 0; e < 4; ++e) sum[4 * q + e] += v[e];
            }
    }
    if constexpr (MODE == kSym && !SHORT)
        if (a.splits > 1) {   // as the registers have it: [tile][split][block][four registers][lane]
            float* to = a.part + ((t.tile * a.splits + t.split) * 4 + wave) * 1024 + lane * 4;
#pragma unroll
            for (int q = 0; q < 4; ++q) *(floatx4*)(to + q * 256) = floatx4{sum[4 * q], sum[4 * q + 1], sum[4 * q + 2], sum[4 * q + 3]};
            return;
        }
    float* tile = lds[wave][SHORT ? 0 : wave];   // read by this wave alone
    wave_sync();
    stage_block(sum, tile);
    wave_sync();
    put_block<MODE>(a, t.matrix, bi, bj, tile);
}

// Sums the parts of a split X X^T, a wave a block, in order.
__global__ __launch_bounds__(64) void muon_join_kernel(MuonArgs a) {
    __shared__ float lds[kTileFloats];
    constexpr int kBlocks = 4;
    const int R = a.mb, tr = (R + 1) / 2;
    const unsigned id = (unsigned)group_of_grid(), tile_id = id / kBlocks, per = tr * (tr + 1) / 2;
    const unsigned matrix = tile_id / per;
    if (matrix >= (unsigned)a.count) return;
    const int block = (int)(id - tile_id * kBlocks), at = (int)(tile_id - matrix * per);
    Tile t;
    place_tile<kSym>(at, tr, t);
    const int bi = 2 * t.ti + (block >> 1), bj = 2 * t.tj + (block & 1);
    if (bi > bj || bj >= R) return;
    const float* part = a.part + (long long)tile_id * a.splits * (kBlocks * 1024) + block * 1024 + (threadIdx.x & 63) * 4;
    floatx16 acc;
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[r] = 0.f;
#pragma unroll 4
    for (int s = 0; s < a.splits; ++s) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const floatx4 v = *(const floatx4*)(part + s * (kBlocks * 1024) + q * 256);
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[4 * q + e] += v[e];
        }
    }
    stage_block(acc, lds);
    wave_sync();
    put_block<kSym>(a, matrix, bi, bj, lds);
}

// Small matrices, of up to 16 blocks: all of a step in one workgroup.  A wave keeps one block of X in registers, as the matrix instruction returns
// it; parts of X by rows, then of its transpose, and of A, then of B, stand in LDS.
constexpr int kSmallBlocks = 16, kSmallLds = 32 * 2 * kParts * kBlockBytes;
bool is_small(int mb, int nb) { return mb * nb <= kSmallBlocks && mb * nb + mb * mb <= 32; }

// The lane, as a number that is not known to stay the same: addresses made of it are worked out where they are used, and not kept through the loop
// over the steps (they were more than there are registers).
__device__ __forceinline__ int lane_now() {
    int lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));
    return lane;
}
// Rows r of `left` against rows c of `right`, both of K blocks.
__device__ __forceinline__ floatx16 small_product(const char* left, int r, const char* right, int c, int K, floatx16 acc) {
    const int lane = lane_now();
    const char *pl = left + r * 2 * K * kParts * kBlockBytes + lane * 16, *pr = right + c * 2 * K * kParts * kBlockBytes + lane * 16;
#pragma unroll 4
    for (int k = 0; k < 2 * K; ++k) {
        halfx8 l[kParts], rt[kParts];
#pragma unroll
        for (int p = 0; p < kParts; ++p) {
            l[p] = *(const halfx8*)(pl + (k * kParts + p) * kBlockBytes);
            rt[p] = *(const halfx8*)(pr + (k * kParts + p) * kBlockBytes);
        }
#pragma unroll
        for (int q = 0; q < kProducts; ++q) acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(l[kPartA[q]], rt[kPartB[q]], acc, 0, 0, 0);
    }
    return acc;
}
// The parts of a block (bi, bj) of registers: by columns (rows of the transpose, K blocks each), and by rows.
__device__ __forceinline__ void small_across(char* base, int K, int bi, int bj, const floatx16& v) {
    const int lane = lane_now(), col = lane & 31, up = lane >> 5;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        halfx4 hi, lo;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            hi[e] = (_Float16)v[4 * q + e];
            lo[e] = (_Float16)(v[4 * q + e] - (float)hi[e]);
        }
        char* to = base + ((bj * 2 * K + 2 * bi + (q >> 1)) * kParts) * kBlockBytes + (q & 1) * 512 + col * 16 + up * 8;
        *(halfx4*)to = hi;
        *(halfx4*)(to + kBlockBytes) = lo;
    }
}
// The transpose of a block, in the same registers, through 4 KB where column c of row r stands at c ^ r, so that neither a row nor a column is on
// one bank.
__device__ __forceinline__ floatx16 turned_block(float* tile, const floatx16& v) {
    const int lane = lane_now(), line = lane & 31, up = lane >> 5;
    floatx16 to;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int row = 8 * (i >> 2) + 4 * up + (i & 3);
        tile[row * 32 + (line ^ row)] = v[i];
    }
    wave_sync();
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int row = 8 * (i >> 2) + 4 * up + (i & 3);
        to[i] = tile[line * 32 + (row ^ line)];
    }
    wave_sync();
    return to;
}
// By rows: through the block's own 4 KB (its two times 16 columns and parts lie in a row), as above.
__device__ __forceinline__ void small_along(char* base, int K, int bi, int bj, const floatx16& v) {
    const int lane = lane_now(), line = lane & 31, up = lane >> 5;
    char* block = base + ((bi * 2 * K + 2 * bj) * kParts) * kBlockBytes;
    float* tile = (float*)block;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int row = 8 * (i >> 2) + 4 * up + (i & 3);
        tile[row * 32 + (line ^ row)] = v[i];
    }
    wave_sync();
    float w[2][8];
#pragma unroll
    for (int g = 0; g < 2; ++g)
#pragma unroll
        for (int e = 0; e < 8; ++e) w[g][e] = tile[line * 32 + ((8 * (up + 2 * g) + e) ^ line)];
    wave_sync();
#pragma unroll
    for (int g = 0; g < 2; ++g) store_parts8(block + g * kParts * kBlockBytes + up * 512 + line * 16, w[g]);
}

__global__ __launch_bounds__(64 * kSmallBlocks) void muon_small_kernel(MuonArgs a, int steps) {
    __shared__ __attribute__((aligned(16))) char lds[kSmallLds];
    __shared__ double norms[kSmallBlocks];
    const long long matrix = group_of_grid();
    if (matrix >= a.count) return;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, waves = blockDim.x >> 6;
    const int mb = a.mb, nb = a.nb, bi = wave / nb, bj = wave - bi * nb;
    const bool mine = wave < mb * nb;                       // of X; the others may have a block of A
    Tile t;
    place_tile<kSym>(wave, mb, t);
    const bool of_a = wave < mb * (mb + 1) / 2;
    char *xs = lds, *as = lds + mb * nb * 2 * kParts * kBlockBytes;
    // this lane's elements of u as they lie in memory: column lane % 32, rows 8 q + 4 (lane / 32) + e of a block that is X's or its transpose
    const int r0 = 32 * (a.tall ? bj : bi) + 4 * (lane >> 5), c = 32 * (a.tall ? bi : bj) + (lane & 31);
    auto row_of = [&](int i) { return r0 + 8 * (i >> 2) + (i & 3); };
    auto in = [&](int i) { return mine && c < a.cols && row_of(i) < a.rows; };
    auto at = [&](int i) { return in(i) ? row_of(i) * a.cols + c : 0; };
    const float* g = a.grad + matrix * a.stride;
    float *m = a.m + matrix * a.stride, *theta = a.theta + matrix * a.stride;
    char* own = xs + (mine ? wave : 0) * 2 * kParts * kBlockBytes;   // 4 KB
    floatx16 x;
    {
        float gv[16], mv[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) gv[i] = g[at(i)], mv[i] = m[at(i)];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float now = __builtin_fmaf(a.momentum, mv[i], gv[i]);
            if (in(i)) m[at(i)] = now;
            x[i] = in(i) ? (a.nesterov ? __builtin_fmaf(a.momentum, now, gv[i]) : now) : 0.f;
        }
    }
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < 16; ++i) sum += (double)x[i] * (double)x[i];
    for (int o = 1; o < 64; o *= 2) sum += __shfl_xor(sum, o);
    if (lane == 0) norms[wave] = sum;
    __syncthreads();
    sum = 0.0;
    for (int w = 0; w < waves; ++w) sum += norms[w];
    const double scale = (double)a.x_scale / (sqrt(sum) + (double)a.eps);
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = (float)((double)x[i] * scale);
    if (a.tall && mine) x = turned_block((float*)own, x);
    const floatx16 zero = {};
    for (int s = 0;; ++s) {
        if (mine) small_along(xs, nb, bi, bj, x);
        __syncthreads();
        floatx16 av = zero;
        if (of_a) {
            av = small_product(xs, t.ti, xs, t.tj, nb, zero);
#pragma unroll
            for (int i = 0; i < 16; ++i) av[i] *= a.sym_scale;
            if (t.ti != t.tj) small_along(as, mb, t.ti, t.tj, av);
            small_across(as, mb, t.ti, t.tj, av);
        }
        __syncthreads();   // A is there, and X has been read
        if (mine) small_across(xs, mb, bi, bj, x);
        if (of_a) {
#pragma unroll
            for (int i = 0; i < 16; ++i) av[i] *= a.cb;
            if (!a.no_square) av = small_product(as, t.ti, as, t.tj, mb, av);
        }
        __syncthreads();   // A has been read
        if (of_a) {
#pragma unroll
            for (int i = 0; i < 16; ++i) av[i] = a.cc * av[i] + (t.ti == t.tj && 8 * (i >> 2) + 4 * (lane >> 5) + (i & 3) == (lane & 31) ? a.ca : 0.f);
            if (t.ti != t.tj) small_along(as, mb, t.ti, t.tj, av);
            small_across(as, mb, t.ti, t.tj, av);
        }
        __syncthreads();
        if (mine) x = small_product(as, bi, xs, bj, mb, zero);
        if (s + 1 == steps) break;
        __syncthreads();   // B and the transpose of X have been read
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] *= a.apply_scale;
    }
    __syncthreads();
    if (a.tall && mine) x = turned_block((float*)own, x);
    float old[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) old[i] = theta[at(i)];
#pragma unroll
    for (int i = 0; i < 16; ++i)
        if (in(i)) theta[at(i)] = a.decay * old[i] - a.lr_scale * x[i];
}

// One step or two (below) of a short side of up to four blocks, in one workgroup a matrix: from A to Q, the product of the steps' B.  A wave computes one
// block of mb x mb of each product; the two operands stand in LDS as parts.  All these matrices are symmetric, so a block may be written as its transpose.
// Latency bounds it: 24 of 100 x 900, 15.8 us for the five products of two steps and 7 for the one of a single step, where a launch takes 4.6 to 5 us.
constexpr int kCoreSide = 4;
__global__ __launch_bounds__(64 * kCoreSide * kCoreSide) void muon_core_kernel(MuonArgs a, int steps) {
    constexpr int kMost = kCoreSide * kCoreSide * 2 * kParts * kBlockBytes;
    __shared__ __attribute__((aligned(16))) char first[kMost], second[kMost];   // A, then B A, the next A and its B; and B
    const long long matrix = group_of_grid();
    if (matrix >= a.count) return;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, mb = a.mb, bi = wave / mb, bj = wave - bi * mb;
    const char* from = block_at(a.a, matrix, mb, mb, 0, 0, 0) + threadIdx.x * 16;
#pragma unroll
    for (int i = 0; i < 4; ++i)   // 4 KB a wave
        *(uint4v*)(first + (i * blockDim.x + threadIdx.x) * 16) = *(const uint4v*)(from + i * blockDim.x * 16);
    __syncthreads();
    const floatx16 zero = {};
    floatx16 v;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const char* at = first + ((bj * 2 * mb + 2 * bi + (k >> 1)) * kParts) * kBlockBytes + (k & 1) * 512 + (lane & 31) * 16 + (lane >> 5) * 8;
        const halfx4 hi = *(const halfx4*)at, lo = *(const halfx4*)(at + kBlockBytes);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[4 * k + e] = (float)lo[e] + (float)hi[e];
    }
    auto times = [&](float by) {
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] *= by;
    };
    // B of A, which is there.  A A is summed from zero: added to one by one, (b / c) A would be rounded with every 16 columns (96 x 200: 2.6 times as far
    // from exact as float32 products, 1.2 this way).
    auto polynomial = [&]() {
        floatx16 square = zero;
        if (!a.no_square) square = small_product(first, bi, first, bj, mb, zero);
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = a.cc * (a.cb * v[i] + square[i]) + (bi == bj && 8 * (i >> 2) + 4 * (lane >> 5) + (i & 3) == (lane & 31) ? a.ca : 0.f);
    };
    auto put = [&](char* to) {
        small_across(to, mb, bi, bj, v);
        __syncthreads();
    };
    polynomial();
    if (steps > 1) {
        put(second);
        v = small_product(second, bi, first, bj, mb, zero);
        times(a.turn_scale);
        __syncthreads();   // A has been read
        put(first);
        v = small_product(first, bi, second, bj, mb, zero);
        times(a.turn_scale);
        __syncthreads();   // B A has been read
        put(first);        // the next A
        polynomial();
        __syncthreads();   // it has been read
        put(first);
        v = small_product(second, bi, first, bj, mb, zero);
        times(a.q_scale);
    }
    small_across(block_at(a.b, matrix, mb, mb, 0, 0, 0), mb, bi, bj, v);
}

// Tiles of 64 x 64, and parts of the sum: an X X^T of few tiles is split so that every CU has a workgroup, where the sum has 32 steps of 32 columns and more,
// no part under eight.  us of the update, whole and split: 24 x 100 x 900 (29 steps) 109, 115; one 100 x 900 89, 87; 64 x 576 (18) 57, 61; 300 x 900 (29) 118, 116; 512 x 960 (30) 141, 168;
// from 32 steps on 300 x 1000 121, 115; 100 x 1024 89, 85; 64 x 2048 73, 64; 512 x 2048 161, 151; 300 x 4000 181, 143.
// The other products sum over the short side, and have 136 tiles where that is 32 steps.
struct ProductPlan {
    bool is_short;            // sums of up to eight steps of 32 columns
    int splits;
    long long tiles;          // of a matrix
};
ProductPlan product_plan(long long count, int mb, int nb, MuonProduct mode, int sum) {
    const long long R = mb, C = mode == kApply ? nb : mb, steps = sum, tr = (R + 1) / 2, tc = (C + 1) / 2;
    ProductPlan p;
    p.tiles = mode == kApply ? tr * tc : tr * (tr + 1) / 2;
    long long s = 256 / (count * p.tiles);
    if (s > steps / 8) s = steps / 8;
    if (mode != kSym || steps < 32) s = 1;
    p.splits = (int)(s < 1 ? 1 : s > 32 ? 32 : s);
    p.is_short = p.splits == 1 && steps <= 8;
    return p;
}
size_t part_bytes(long long count, const ProductPlan& p) { return p.splits > 1 ? (size_t)count * p.tiles * p.splits * 4 * 4096 : 0; }

// Two steps at a time (below) leave out two products over the long side, 1.5 mb^2 nb blocks, and take three over the short one, 1.5 mb^3, and a launch more: worth it
// from 8192 blocks on.  us of five steps, one at a time against two, one and two: 160x2000 (1400 blocks) 107, 107; 300x1000 (2200) 114, 121; 512x1024 (4096) 138, 144;
// 8 of 160x2000 (11600) 143, 130; 512x2048 (12288) 153, 151; 1024x1536 (16384, but one and a half as wide as high) 214, 215; 512x4096 (28672) 177, 168; 12 of 200x2000
// (32928) 213, 185; 1024x4096 (98304) 372, 313; 4 of it 1225, 979.  A short side of up to kCoreSide blocks goes by the kernel above in any case.
bool is_wide(long long count, int mb, int nb) { return mb > kCoreSide && nb >= 2 * mb && count * (nb - mb) * mb * mb > 8192; }

struct MuonPlan {
    int mb, nb, parts;
    int squares;              // matrices of mb x mb: A and B, and where two steps are taken at a time another B and what is multiplied
    size_t x_bytes, a_bytes, norm_bytes, part_bytes;
};
MuonPlan plan_of(long long count, long long rows, long long cols) {
    MuonPlan p;
    const long long m = rows < cols ? rows : cols, n = rows < cols ? cols : rows;
    p.mb = (int)((m + 31) / 32);
    p.nb = (int)((n + 31) / 32);
    const long long parts = (rows * cols + 2047) / 2048;
    p.parts = (int)(parts < kMuonNorms ? parts : kMuonNorms);
    p.x_bytes = (size_t)count * p.mb * p.nb * 2 * kParts * kBlockBytes;
    p.a_bytes = (size_t)count * p.mb * p.mb * 2 * kParts * kBlockBytes;
    p.squares = is_wide(count, p.mb, p.nb) ? 4 : 2;
    p.norm_bytes = (size_t)count * kMuonNorms * sizeof(double);
    p.part_bytes = part_bytes(count, product_plan(count, p.mb, p.nb, kSym, p.nb));
    return p;
}

template <int MODE>
void launch_product(MuonArgs& a, hipStream_t st) {
    const int sum = MODE == kSym ? a.sum : a.mb;
    const ProductPlan p = product_plan(a.count, a.mb, a.nb, (MuonProduct)MODE, sum);
    const double R = a.mb, C = MODE == kApply ? a.nb : (a.mb + 1) * 0.5, K = sum, work = 65536.0 * R * C * K * a.count;
    a.splits = p.splits;
    {
        KernelScope ks(MODE == kSym ? "muon_sym" : MODE == kSquare ? "muon_square" : "muon_apply", work, 0.0, st, kProducts * work);
        const dim3 grid = grid_of((a.count * p.tiles * p.splits + 7) / 8 * 8), block(256);
        if (p.is_short) hipLaunchKernelGGL((muon_product_kernel<MODE, true>), grid, block, 0, st, a);
        else hipLaunchKernelGGL((muon_product_kernel<MODE, false>), grid, block, 0, st, a);
    }
    if (MODE != kSym || p.splits == 1) return;
    KernelScope ks("muon_join", 0.0, (double)part_bytes(a.count, p), st);
    hipLaunchKernelGGL(muon_join_kernel, grid_of(a.count * p.tiles * 4), dim3(64), 0, st, a);
}

// The power of two that takes v to (2^13, 2^14].
double scale_of(double v) { return std::ldexp(1.0, 14 - (int)std::ceil(std::log2(v))); }

// Scales of X, A and B, and the largest value of the polynomial; false where numbers would leave their range.
bool bounds_of(const gleam_muon& p, double& sx, double& sa, double& sb, double& most_b) {
    const double a = p.a, b = p.b, c = p.c;
    double most = 1.0, top = 1.0;   // singular values of any X, and of this one: |u|_F bounds the largest
    for (int k = 0; k + 1 < p.steps; ++k) {   // the last X goes to the weights in float32
        // largest |s (a + b s^2 + c s^4)| of 0 <= s <= top: there, or where the slope a + 3 b z + 5 c z^2 is 0, z = s^2
        auto value = [&](double z) { return z > 0.0 && z < top * top ? std::sqrt(z) * std::fabs(a + z * (b + z * c)) : 0.0; };
        double next = top * std::fabs(a + top * top * (b + top * top * c));
        const double disc = 9.0 * b * b - 20.0 * a * c;
        if (c != 0.0 && disc >= 0.0)
            for (double sign : {-1.0, 1.0}) next = std::max(next, value((-3.0 * b + sign * std::sqrt(disc)) / (10.0 * c)));
        if (c == 0.0 && b != 0.0) next = std::max(next, value(-a / (3.0 * b)));
        top = 1.001 * next;         // and what products are rounded by
        if (!(top < 128.0)) return false;
        most = std::max(most, top);
    }
    const double z1 = most * most, vertex = c != 0.0 ? -b / (2.0 * c) : 0.0;
    auto poly = [&](double z) { return std::fabs(a + z * (b + z * c)); };
    most_b = std::max(poly(0.0), poly(z1));
    if (vertex > 0.0 && vertex < z1) most_b = std::max(most_b, poly(vertex));
    most_b = std::max(most_b, 1e-3);
    if (!(most_b < 16384.0)) return false;
    sx = scale_of(most);
    sa = scale_of(z1);
    sb = scale_of(most_b);
    return true;
}

// Two steps at a time, of wide matrices and of short sides: B is a polynomial of A and commutes with it, so the next step's A is (B A) B, and the two B
// multiply to one Q that X is multiplied by: instead of X X^T and B X, sums over the long side, three products of the short one.  What A is rounded by,
// 2^-24 of its largest eigenvalue, is then not found again in the next X X^T: an eigenvalue near 0 grows by a^2 a step and Q changes by 2 b / a of that,
// 2^-23 |b / a| (1 + a^2) of itself after two steps, 2.1e-6 with the default polynomial.  A third step would bring 2.5e-5, however many parts A has,
// where float32 products leave X to 1e-6 (a strong direction over noise, 64 x 576: three steps together are 28 times as far from exact as float32 products,
// two 1.1 times).  For the same reason the single step of an odd number is the second and not the last, by when the eigenvalues near 0 have grown
// to what most of X is (96 x 200, an eighth of the directions strong, products emulated on the host: 1.0 times as far as float32 products, and 2.0).
// And Q has to be in reach of its scale, which is made for the largest value that the steps' B could have, most_b^2, where what is there is about a^2, and 1
// beside it: above 2^12 of that its second parts would begin to go below the smallest float16 (at 2^16 of it; (1, -3, 6) has 2^21: 2500 x 700 X off by
// 1.2e-4 of itself together, 2.4e-7 one by one).
bool may_go_together(const gleam_muon& h, double most_b) {
    const double a = std::fabs((double)h.a), loss = 0x1p-23 * std::fabs((double)h.b) / std::max(a, 1e-3) * (1.0 + a * a);
    const double over = most_b / std::min(std::max(a, 1e-6), 1.0);
    return loss < 3e-5 && over * over <= 0x1p12;
}

}  // namespace

bool muon_scales(const gleam_muon& p) {
    double sx, sa, sb, most_b;
    return bounds_of(p, sx, sa, sb, most_b);
}

size_t muon_ws_bytes(long long count, long long rows, long long cols) {
    const MuonPlan p = plan_of(count, rows, cols);
    if (is_small(p.mb, p.nb)) return 0;
    return 3 * p.x_bytes + p.squares * p.a_bytes + p.norm_bytes + p.part_bytes;
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
    char *b[2] = {a.a + p.a_bytes, p.squares > 2 ? a.a + 2 * p.a_bytes : nullptr}, *t = p.squares > 2 ? a.a + 3 * p.a_bytes : nullptr;
    a.norms = (double*)(a.a + p.squares * p.a_bytes);
    a.part = (float*)(a.a + p.squares * p.a_bytes + p.norm_bytes);
    a.stride = stride;
    a.count = count;
    a.rows = (int)rows;
    a.cols = (int)cols;
    a.tall = rows > cols;
    a.mb = p.mb;
    a.nb = p.nb;
    a.parts = p.parts;
    a.nesterov = h.nesterov;
    a.decay = (float)(1.0 - (double)h.lr * h.weight_decay);
    a.momentum = h.momentum;
    a.eps = h.eps;
    // b A + c A A = c ((b / c) A + A A); where c A A is below 2^-60 of b A, or c is 0, it is b A alone
    a.no_square = std::fabs((double)h.c) <= std::fabs((double)h.b) * 0x1p-60;
    double sx = 1.0, sa = 1.0, sb = 1.0, most_b = 1.0;
    bounds_of(h, sx, sa, sb, most_b);
    const double lr = (double)h.lr * std::sqrt(a.tall ? (double)rows / (double)cols : 1.0);
    a.x_scale = (float)sx;
    a.sym_scale = (float)(sa / (sx * sx));
    a.apply_scale = (float)(1.0 / sb);
    a.lr_scale = (float)(lr / (sb * sx));
    a.ca = (float)(h.a * sb);
    a.cb = (float)(a.no_square ? sa : sa * (double)h.b / (double)h.c);
    a.cc = (float)((a.no_square ? h.b : h.c) * (sb / (sa * sa)));
    if (is_small(p.mb, p.nb)) {
        KernelScope ks("muon_small", (double)count * h.steps * 65536.0 * p.mb * (p.mb * p.nb + (p.mb + 1) * 0.5 * (p.nb + p.mb)), 20.0 * count * rows * cols, st);
        hipLaunchKernelGGL(muon_small_kernel, grid_of(count), dim3(64 * std::max(p.mb * p.nb, p.mb * (p.mb + 1) / 2)), 0, st, a, (int)h.steps);
        return hipGetLastError();
    }
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
    // symmetric products of `left` and `right`, whose numbers have these scales, to `to`
    auto sym = [&](const char* left, double sl, const char* right, double sr, int sum, char* to, double s_to) {
        a.left = left;
        a.right = right;
        a.sum = sum;
        a.sym = to;
        a.sym_scale = (float)(s_to / (sl * sr));
        launch_product<kSym>(a, st);
    };
    const bool core = p.mb <= kCoreSide, two = (core || p.squares > 2) && may_go_together(h, most_b);
    for (int k = 0, turn = 0; k < h.steps && e == hipSuccess; ++turn) {
        const int now = two && h.steps - k > 1 && !(turn == 1 && h.steps % 2) ? 2 : 1;   // steps taken together
        sym(a.x, sx, a.x, sx, a.nb, a.a, sa);
        const char* q = a.b = b[0];
        const double sq = now == 1 ? sb : scale_of(most_b * most_b);
        if (core) {
            a.turn_scale = (float)(1.0 / sb);
            a.q_scale = (float)(sq / (sb * sb));
            const double work = 65536.0 * p.mb * p.mb * p.mb * count * (now == 1 ? 1 : 5);
            KernelScope ks("muon_core", work, 0.0, st, kProducts * work);
            hipLaunchKernelGGL(muon_core_kernel, grid_of(count), dim3(64 * p.mb * p.mb), 0, st, a, now);
        } else {
            launch_product<kSquare>(a, st);
            if (now == 2) {
                sym(b[0], sb, a.a, sa, a.mb, t, sa);      // B A, under the largest singular values of two X
                sym(t, sa, b[0], sb, a.mb, a.a, sa);      // A of the next step
                a.b = b[1];
                launch_product<kSquare>(a, st);
                sym(b[1], sb, b[0], sb, a.mb, t, sq);     // Q; B A is not needed any more
                q = t;
            }
        }
        k += now;
        a.last = k == h.steps;
        a.left = q;
        a.apply_scale = (float)(1.0 / sq);
        a.lr_scale = (float)(lr / (sq * sx));
        launch_product<kApply>(a, st);
        std::swap(a.xt, a.xt_out);
        e = hipGetLastError();
    }
    return e;
}

}  // namespace gleam
