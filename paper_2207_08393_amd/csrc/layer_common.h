// What the kernels of the sequence-layer operators share (gfx950 device code): 16 bytes of float32 or bfloat16 elements in registers.
#pragma once
#include "prox_common.h"

namespace gleam {
namespace {

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(unsigned short v) { return bf16_to_f32(v); }
__device__ __forceinline__ void put_f32(float* p, float v) { *p = v; }
__device__ __forceinline__ void put_f32(unsigned short* p, float v) { *p = (unsigned short)pack_bf16x2(v, v); }

// Workgroups of a launch.  A grid's dimension holds fewer than 2^32 work-items (2^22 workgroups of 1024), so workgroups past the first
// kGridX go on in the second dimension; there may be up to 2^37 of them, and some more than asked for, which have nothing to do.
constexpr unsigned kGridX = 1u << 21;
inline dim3 grid_of(long long groups) {
    return dim3((unsigned)(groups < kGridX ? groups : kGridX), (unsigned)((groups + kGridX - 1) / kGridX));
}
__device__ __forceinline__ long long group_of_grid() { return (long long)blockIdx.y * kGridX + blockIdx.x; }

// N elements of type T; 16 bytes, or two times 16 for eight float32.  Global addresses need the alignment of an element only: the
// memory unit takes 16 bytes from any address (an access that crosses a cache line costs two).
template <class T, int N>
struct Pack {
    static constexpr int kWords = N * (int)sizeof(T) / 4;
    static_assert(kWords * 4 == N * (int)sizeof(T), "whole words");
    unsigned w[kWords];
    __device__ __forceinline__ void load(const T* p) { __builtin_memcpy(w, p, sizeof(w)); }
    __device__ __forceinline__ void store(T* p) const { __builtin_memcpy(p, w, sizeof(w)); }
    __device__ __forceinline__ void store_lds(T* p) const {   // p aligned to 16 bytes
        static_assert(kWords == 4, "one access");
        *(uint4*)p = make_uint4(w[0], w[1], w[2], w[3]);
    }
    __device__ __forceinline__ float get(int i) const {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
        else return __uint_as_float(i & 1 ? w[i >> 1] & 0xffff0000u : w[i >> 1] << 16);
    }
    __device__ __forceinline__ void set(const float* v) {
#pragma unroll
        for (int i = 0; i < kWords; ++i) {
            if constexpr (sizeof(T) == 4) w[i] = __float_as_uint(v[i]);
            else w[i] = pack_bf16x2(v[2 * i], v[2 * i + 1]);
        }
    }
};

}  // namespace
}  // namespace gleam
