// Dropout from a counter-based generator, residual added in the same pass (gfx950).
//
// The mask is a function of (seed, counter, element index): Philox 4x32-10 gives 128 bits for a counter, that is eight draws of 16 bits
// for eight consecutive elements, so that a thread's 16 bytes of bfloat16 (32 of float32) need one evaluation.  Nothing is stored for
// the backward pass, which draws the same mask again.  Bound by HBM: 20 x 192 x 160 pixels of 64 channels with a residual, bfloat16, 42 us
// (5.7 TB/s, part of it from the 256 MB cache), 4 x 320 x 256 pixels of 100 channels, float32, 50 us (5.3 TB/s).
#include <hip/hip_runtime.h>

#include "layer_ops.h"
#include "layer_common.h"

namespace gleam {
namespace {

constexpr int kDropThreads = 256;

// Ten rounds on the counter c with the key k (Salmon et al. 2011, section 3): two 32 x 32 -> 64 bit products a round.
__device__ __forceinline__ uint4 philox(uint4 c, uint2 k) {
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        const unsigned long long a = (unsigned long long)c.x * 0xD2511F53u, b = (unsigned long long)c.z * 0xCD9E8D57u;
        c = make_uint4((unsigned)(b >> 32) ^ c.y ^ k.x, (unsigned)b, (unsigned)(a >> 32) ^ c.w ^ k.y, (unsigned)a);
        k.x += 0x9E3779B9u;
        k.y += 0xBB67AE85u;
    }
    return c;
}

// Draw i of a block: low half of word i/2 first.
__device__ __forceinline__ unsigned draw16(const uint4& r, int i) {
    const unsigned w[4] = {r.x, r.y, r.z, r.w};
    return i & 1 ? w[i >> 1] >> 16 : w[i >> 1] & 0xffffu;
}
__device__ __forceinline__ uint4 draws_of(const DropoutArgs& a, unsigned long long block) {
    unsigned long long c = a.offset + (a.step ? *a.step : 0ull);
    return philox(make_uint4((unsigned)block, (unsigned)(block >> 32), (unsigned)c, (unsigned)(c >> 32)),
                  make_uint2((unsigned)a.seed, (unsigned)(a.seed >> 32)));
}

// One thread, one block of eight elements; a block that crosses rows, or the end, goes element by element.
template <class T>
__global__ __launch_bounds__(kDropThreads) void dropout_kernel(DropoutArgs a) {
    const long long blk = group_of_grid() * kDropThreads + threadIdx.x;
    const long long first = blk * 8, size = a.rows * a.n;
    if (first >= size) return;
    const T *x = (const T*)a.x, *res = (const T*)a.res;
    T* out = (T*)a.out;
    const bool few = size <= 0x7fffffff;   // a division of 32 bits does
    const long long row = a.rows == 1 ? 0 : few ? (long long)((unsigned)first / (unsigned)a.n) : first / a.n, col = first - row * a.n;
    if (col + 8 <= a.n) {
        Pack<T, 8> px, pr;
        px.load(x + row * a.ld_x + col);
        if (res) pr.load(res + row * a.ld_res + col);
        const uint4 r = draws_of(a, (unsigned long long)blk);
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            v[i] = draw16(r, i) < a.kept ? px.get(i) * a.scale : 0.f;
            if (res) v[i] += pr.get(i);
        }
        px.set(v);
        px.store(out + row * a.ld_out + col);
        return;
    }
    // places of the eight elements, then all loads, then the rest
    const int there = size - first < 8 ? (int)(size - first) : 8;
    const T *px = x + row * a.ld_x + col, *pr = res ? res + row * a.ld_res + col : nullptr;
    T* po = out + row * a.ld_out + col;
    T vx[8], vr[8];
    T* to[8];
    long long cc = col;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        to[i] = po;
        vx[i] = vr[i] = (T)0;
        if (i < there) {
            vx[i] = *px;
            if (res) vr[i] = *pr;
        }
        const bool end = ++cc == a.n;
        px += end ? a.ld_x - a.n + 1 : 1;
        pr += end ? a.ld_res - a.n + 1 : 1;
        po += end ? a.ld_out - a.n + 1 : 1;
        cc = end ? 0 : cc;
    }
    const uint4 r = draws_of(a, (unsigned long long)blk);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        float v = draw16(r, i) < a.kept ? to_f32(vx[i]) * a.scale : 0.f;
        if (res) v += to_f32(vr[i]);
        if (i < there) put_f32(to[i], v);
    }
}

template <class T>
hipError_t launch(const DropoutArgs& a, hipStream_t st) {
    const long long blocks = (a.rows * a.n + 7) / 8;
    KernelScope ks("dropout", 2.0 * a.rows * a.n, (a.res ? 3.0 : 2.0) * sizeof(T) * a.rows * a.n, st);
    hipLaunchKernelGGL(dropout_kernel<T>, grid_of((blocks + kDropThreads - 1) / kDropThreads), dim3(kDropThreads), 0, st, a);
    return hipGetLastError();
}

}  // namespace

hipError_t dropout(const DropoutArgs& args, hipStream_t st) {
    DropoutArgs a = args;
    if (a.ld_x == a.n && a.ld_out == a.n && (!a.res || a.ld_res == a.n)) {   // no gaps: one long row
        a.n *= a.rows;
        a.rows = 1;
    }
    return a.dtype ? launch<unsigned short>(a, st) : launch<float>(a, st);
}

}  // namespace gleam
