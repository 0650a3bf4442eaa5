// Linear attention with a decay for each head (gfx950): chunked form, recurrent form for one token, gradients.
//
//   S_t = e^a S_{t-1} + k_t v_t^T,   o_t = scale S_t^T q_t
//
// Chunked form.  Within a chunk of L tokens i, j = 0..L-1 that begins with state X:
//   o_i = out_scale (e^{a(i+1)} q_i X + in_scale sum_{j<=i} e^{a(i-j)} (q_i . k_j) v_j)
//   X'  = e^{aL} X + in_scale sum_j e^{a(L-1-j)} k_j v_j^T
// that is four matrix products per chunk, 4 dk dv + 2 L (dk + dv) flops a token instead of 4 dk dv, on the matrix cores.
//
// Gradients are the same sums with the roles exchanged.  With X transposed, g_q = mix(q: g_o, k: v, v: k); from a sequence's
// end to its start, g_k = mix(q: v, k: g_o, v: q) and g_v = mix(q: k, k: q, v: g_o), where the state that comes in is dL/d state_out.
// Backwards the decay of the state is applied after a token has read it (dL/dv_s = .. + e^{a(T-1-s)} k_s . dS_T): the
// exponents i+1 and L-1-j above become i and L-j ("shift" in the code).
//
// One problem is one sequence, pixel and head.  D is dk and dv rounded up to 32, 64 or 128; a problem is worked on by D/32 waves, and
// a wave owns 32 columns (dv) of the state, in registers in the layout of a 16x16 product's result: the lane holds
// column l % 16 and four rows.  That is also an operand's layout, so the state enters the next product without a trip through LDS.
// Scores are formed by all waves, each for its rows of the chunk, and exchanged through LDS.
#include <hip/hip_runtime.h>

#include "layer_common.h"
#include "layer_ops.h"

namespace gleam {
namespace {

typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef short short4v __attribute__((ext_vector_type(4)));
constexpr float kLog2e = 1.44269504088896340736f;

// Within each group of 16 lanes, lane s passes the address of 4 consecutive 16-bit values of row s/4; lane j gets column j of the
// 4 x 16 block, rows 0..3.
__device__ __forceinline__ uint2 read_tr16(const unsigned short* p) {
    const short4v v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((short4v __attribute__((address_space(3)))*)(p));
    return __builtin_bit_cast(uint2, v);
}

// Operands of a product over a block of kBlock values of the contracted index.  Lane l = 16 g + m holds row (column) m and the
// kBlock/4 values from g kBlock/4 on, 16 bytes.  Results: column m, rows 4 g .. 4 g + 3 of a 16 x 16 tile.
//   row_frag : from an LDS array whose rows are the operand's rows
//   col_frag : from an LDS array whose rows are the contracted index (a transposing read)
//   tile     : which row (column) of a 32-wide block is number m of tile t.  For bfloat16 the rows of tiles 2u and 2u+1 alternate in
//              fours, so that the two results of a lane are eight consecutive values: what an operand holds, and 16 bytes of output.
template <class T>
struct Mma;
template <>
struct Mma<unsigned short> {
    static constexpr int kBlock = 32, kVec = 8;
    typedef bf16x8 Frag;
    static __device__ __forceinline__ int tile(int t, int m) { return 32 * (t >> 1) + 8 * (m >> 2) + 4 * (t & 1) + (m & 3); }
    static __device__ __forceinline__ floatx4 mma(Frag a, Frag b, floatx4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ Frag row_frag(const unsigned short* p) { return *(const Frag*)p; }
    // rows 8 g .. 8 g + 7 of the block that begins at p, column tile(t, m)
    static __device__ __forceinline__ Frag col_frag(const unsigned short* p, int stride, int t, int lane) {
        const int g = lane >> 4, s = lane & 15;
        const unsigned short* q = p + (8 * g + (s >> 2)) * stride + 32 * (t >> 1) + 8 * (s & 3) + 4 * (t & 1);
        const uint2 lo = read_tr16(q), hi = read_tr16(q + 4 * stride);
        return __builtin_bit_cast(Frag, make_uint4(lo.x, lo.y, hi.x, hi.y));
    }
    // Parts whose sum is f times w: bfloat16 numbers w[i] f[i] rounded, what that left over rounded, and so on; 8 bits each.
    static constexpr int kParts = 3, kStateParts = 2;
    static __device__ __forceinline__ void scaled(Frag f, const float* w, Frag* parts, int n) {
        const uint4 u = __builtin_bit_cast(uint4, f);
        const unsigned x[4] = {u.x, u.y, u.z, u.w};
        float v[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(x[i] << 16) * w[2 * i];
            v[2 * i + 1] = __uint_as_float(x[i] & 0xffff0000u) * w[2 * i + 1];
        }
        split(v, parts, n);
    }
    static __device__ __forceinline__ void split(float* v, Frag* parts, int n) {
#pragma unroll
        for (int k = 0; k < n; ++k) {
            unsigned y[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                y[i] = pack_bf16x2(v[2 * i], v[2 * i + 1]);
                if (k + 1 < n) {
                    v[2 * i] -= __uint_as_float(y[i] << 16);
                    v[2 * i + 1] -= __uint_as_float(y[i] & 0xffff0000u);
                }
            }
            parts[k] = __builtin_bit_cast(Frag, make_uint4(y[0], y[1], y[2], y[3]));
        }
    }
    // the results of two tiles as an operand, in kStateParts parts
    static __device__ __forceinline__ void pack(const floatx4* x, Frag* parts) {
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = x[i >> 2][i & 3];
        split(v, parts, kStateParts);
    }
    static __device__ __forceinline__ void put4(unsigned short* p, floatx4 v) {
        *(uint2*)p = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
    }
};
template <>
struct Mma<float> {
    static constexpr int kBlock = 16, kVec = 4;
    typedef floatx4 Frag;
    static __device__ __forceinline__ int tile(int t, int m) { return 16 * t + m; }
    static __device__ __forceinline__ floatx4 mma(Frag a, Frag b, floatx4 c) {
#pragma unroll
        for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], c, 0, 0, 0);
        return c;
    }
    static __device__ __forceinline__ Frag row_frag(const float* p) { return *(const Frag*)p; }
    static __device__ __forceinline__ Frag col_frag(const float* p, int stride, int t, int lane) {
        const float* q = p + 4 * (lane >> 4) * stride + 16 * t + (lane & 15);
        return Frag{q[0], q[stride], q[2 * stride], q[3 * stride]};
    }
    static constexpr int kParts = 1, kStateParts = 1;
    static __device__ __forceinline__ void scaled(Frag f, const float* w, Frag* parts, int) { parts[0] = Frag{f[0] * w[0], f[1] * w[1], f[2] * w[2], f[3] * w[3]}; }
    static __device__ __forceinline__ void pack(const floatx4* x, Frag* parts) { parts[0] = x[0]; }
    static __device__ __forceinline__ void put4(float* p, floatx4 v) { *(floatx4*)p = v; }
};

// e^{a n}; 1 for n = 0 whatever a is.
__device__ __forceinline__ float decay_of(float a, int n) { return n == 0 ? 1.f : exp2f(a * kLog2e * (float)n); }

// Tokens a chunk has, and waves and problems of a workgroup.
template <class T, int D>
struct Shape {
    static constexpr int kWaves = D / 32, kProblems = kWaves == 1 ? 4 : 1, kThreads = 64 * kWaves * kProblems;
    static constexpr int kL = sizeof(T) == 2 && D > 32 ? 64 : 32;
    static constexpr int kRow = D + (sizeof(T) == 2 ? 8 : 4);       // elements between rows in LDS
    static constexpr int kScoreRow = kL + (sizeof(T) == 2 ? 8 : 4);
    static constexpr int kTiles = D / 16;                            // rows of tiles of the state
    static constexpr int kStateFloats = D * D;
};

// Waves of a problem wait for each other's LDS writes: a barrier, or for a single wave the order of its own accesses.
template <int WAVES>
__device__ __forceinline__ void exchange() {
    if constexpr (WAVES > 1) {
        __syncthreads();
    } else {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
}

struct Problem {
    long long index;    // (b P + p) H + h
    long long b, p;
    int h, len;         // head, tokens
};
__device__ __forceinline__ Problem problem_of(const MixArgs& a, long long index) {
    Problem r;
    r.index = index;
    r.h = (int)(index % a.H);
    const long long rest = index / a.H;
    r.p = rest % a.P;
    r.b = rest / a.P;
    r.len = (int)a.T;
    if (a.lengths) {
        const int l = a.lengths[r.b];
        r.len = l < 0 ? 0 : l < r.len ? l : r.len;
    }
    return r;
}
template <class T>
__device__ __forceinline__ const T* base_of(const MixTensor& x, const Problem& r) {
    return (const T*)x.p + r.b * x.s.b + r.p * x.s.p + (long long)(r.h / x.share) * x.s.h;
}

// State element (row of dk, column of dv in this pass's roles) in the natural layout of the layer.
__device__ __forceinline__ long long state_at(const MixArgs& a, int row, int col) {
    return a.state_t ? (long long)col * a.k.d + row : (long long)row * a.v.d + col;
}

// STATES: only the sum of k (x) v over segment blockIdx.y, for the scan over segments; seg_state slot blockIdx.y + 1.
template <class T, int D, bool STATES>
__global__ __launch_bounds__((Shape<T, D>::kThreads)) void mix_kernel(MixArgs a) {
    typedef Shape<T, D> S;
    typedef Mma<T> M;
    typedef typename M::Frag Frag;
    constexpr int L = S::kL, VE = M::kVec, KB = M::kBlock, W = S::kWaves, NT = 64 * W;
    constexpr int NV = L * D / VE / NT;               // 16-byte vectors of an array a lane stages
    constexpr int kPair = KB / 16;                    // result tiles that make an operand
    __shared__ __attribute__((aligned(16))) T lds_q[STATES ? 1 : S::kProblems][STATES ? 8 : L * S::kRow];
    __shared__ __attribute__((aligned(16))) T lds_k[S::kProblems][L * S::kRow];
    __shared__ __attribute__((aligned(16))) T lds_v[S::kProblems][L * S::kRow];
    __shared__ __attribute__((aligned(16))) T lds_p[STATES ? 1 : S::kProblems][STATES ? 8 : L * S::kScoreRow];
    __shared__ float lds_w[S::kProblems][L + 2];
    const int slot = S::kProblems == 1 ? 0 : threadIdx.x >> 6;
    const int tid = S::kProblems == 1 ? threadIdx.x : threadIdx.x & 63;
    const int lane = tid & 63, m = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const long long index = (long long)blockIdx.x * S::kProblems + slot;
    if (index >= a.B * a.P * a.H) return;             // several problems a workgroup: a wave each, and no barriers
    const Problem r = problem_of(a, index);
    const int seg = blockIdx.y;
    const long long r_begin = (long long)seg * a.seg_chunks * L;
    const int c_begin = seg * a.seg_chunks;
    int c_end = (r.len + L - 1) / L;
    if (c_end > c_begin + a.seg_chunks) c_end = c_begin + a.seg_chunks;
    const int shift = a.reverse;
    const float decay = a.log_decay[r.h];
    T *sq = lds_q[STATES ? 0 : slot], *sk = lds_k[slot], *sv = lds_v[slot], *sp = lds_p[STATES ? 0 : slot];
    float* sw = lds_w[slot];
    const T *gq = base_of<T>(a.q, r), *gk = base_of<T>(a.k, r), *gv = base_of<T>(a.v, r);
    for (int i = tid; i < L + 2; i += NT) sw[i] = decay_of(decay, i);

    // staging: vectors tid + i NT of the chunk's rows
    const int col = tid % (D / VE) * VE, row0 = tid / (D / VE);
    constexpr int kRowStep = NT / (D / VE);
    Pack<T, VE> nq[NV], nk[NV], nv[NV];
    auto fetch_one = [&](const T* base, const MixTensor& x, long long token, bool ok, Pack<T, VE>& p) {
        if (ok && col + VE <= x.d) {
            p.load(base + token * x.s.t + col);
        } else {
            float f[VE];
#pragma unroll
            for (int e = 0; e < VE; ++e) f[e] = ok && col + e < x.d ? to_f32(base[token * x.s.t + col + e]) : 0.f;
            p.set(f);
        }
    };
    auto fetch = [&](int c) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int at = c * L + row0 + i * kRowStep;
            const bool ok = at < r.len;
            const long long token = a.reverse ? r.len - 1 - at : at;
            if constexpr (!STATES) fetch_one(gq, a.q, token, ok, nq[i]);
            fetch_one(gk, a.k, token, ok, nk[i]);
            fetch_one(gv, a.v, token, ok, nv[i]);
        }
    };
    auto stage = [&] {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int at = (row0 + i * kRowStep) * S::kRow + col;
            if constexpr (!STATES) nq[i].store_lds(sq + at);
            nk[i].store_lds(sk + at);
            nv[i].store_lds(sv + at);
        }
    };

    floatx4 x[S::kTiles][2];                          // the state: rows of tile t, columns 32 wave + tile(u, m)
    bool have = false;                                // it is not zero
#pragma unroll
    for (int t = 0; t < S::kTiles; ++t) x[t][0] = x[t][1] = floatx4{0.f, 0.f, 0.f, 0.f};
    auto seg_slot = [&](int s) {
        return (floatx4*)a.seg_state + (((r.index * a.n_seg + s) * W + wave) * S::kTiles * 2) * 64 + lane;
    };
    auto for_state = [&](auto&& f) {                  // f(t, u, i, natural offset) for this lane's elements that exist
#pragma unroll
        for (int t = 0; t < S::kTiles; ++t)
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int row = M::tile(t, 4 * g + i), c = 32 * wave + M::tile(u, m);
                    if (row < a.k.d && c < a.v.d) f(t, u, i, r.index * a.k.d * a.v.d + state_at(a, row, c));
                }
    };
    if constexpr (!STATES) {
        if (a.seg_state) {
            const floatx4* s = seg_slot(seg);
#pragma unroll
            for (int t = 0; t < S::kTiles; ++t)
#pragma unroll
                for (int u = 0; u < 2; ++u) x[t][u] = s[(t * 2 + u) * 64];
            have = true;
        } else if (a.state_in) {
            for_state([&](int t, int u, int i, long long at) { x[t][u][i] = a.state_in[at]; });
            have = true;
        }
    }
    if (c_begin < c_end) fetch(c_begin);
    for (int c = c_begin; c < c_end; ++c) {
        const int left = r.len - c * L, count = left < L ? left : L;
        exchange<W>();                                // everyone is done with the chunk before
        stage();
        exchange<W>();
        if (c + 1 < c_end) fetch(c + 1);
        Frag vf[L / KB][2];
#pragma unroll
        for (int s = 0; s < L / KB; ++s)
#pragma unroll
            for (int u = 0; u < 2; ++u) vf[s][u] = M::col_frag(sv + s * KB * S::kRow, S::kRow, 2 * wave + u, lane);
        if constexpr (!STATES) {
            // scores of rows it (mod waves): the lane has four consecutive columns j of row i
            for (int it = wave; it < L / 16; it += W) {
                if (it * 16 >= count) break;
                Frag qf[D / KB];
#pragma unroll
                for (int s = 0; s < D / KB; ++s) qf[s] = M::row_frag(sq + (16 * it + m) * S::kRow + s * KB + g * VE);
                const int last = (it * 16 / KB + 1) * (KB / 16);    // tiles up to the end of the diagonal's block
                for (int jt = 0; jt < last; ++jt) {
                    floatx4 p{0.f, 0.f, 0.f, 0.f};
                    if (jt <= it) {
#pragma unroll
                        for (int s = 0; s < D / KB; ++s) p = M::mma(M::row_frag(sk + (16 * jt + m) * S::kRow + s * KB + g * VE), qf[s], p);
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int n = 16 * (it - jt) + m - 4 * g - i;
                        p[i] = n >= 0 ? p[i] * (a.in_scale * a.out_scale * sw[n < 0 ? 0 : n]) : 0.f;
                    }
                    M::put4(sp + (16 * it + m) * S::kScoreRow + 16 * jt + 4 * g, p);
                }
            }
            exchange<W>();
            for (int it = 0; it * 16 < count; ++it) {
                floatx4 o[2] = {};
                if (have) {
#pragma unroll
                    for (int s = 0; s < D / KB; ++s) {
                        const Frag qf = M::row_frag(sq + (16 * it + m) * S::kRow + s * KB + g * VE);
#pragma unroll
                        for (int u = 0; u < 2; ++u) {
                            const floatx4 both[2] = {x[kPair * s][u], x[kPair * s + kPair - 1][u]};
                            Frag part[M::kStateParts];
                            M::pack(both, part);
#pragma unroll
                            for (int n = 0; n < M::kStateParts; ++n) o[u] = M::mma(part[n], qf, o[u]);
                        }
                    }
                    const float f = a.out_scale * sw[16 * it + m + 1 - shift];
                    o[0] *= f;
                    o[1] *= f;
                }
                const int last = it * 16 / KB;
#pragma unroll
                for (int s = 0; s < L / KB; ++s) {
                    if (s > last) break;
                    const Frag pf = M::row_frag(sp + (16 * it + m) * S::kScoreRow + s * KB + g * VE);
#pragma unroll
                    for (int u = 0; u < 2; ++u) o[u] = M::mma(vf[s][u], pf, o[u]);
                }
                const int i = 16 * it + m;
                if (i < count) {
                    const long long token = a.reverse ? r.len - 1 - (c * L + i) : c * L + i;
                    const long long at = r.b * a.o.s.b + token * a.o.s.t + r.p * a.o.s.p + (long long)(r.h / a.o.share) * a.o.s.h;
#pragma unroll
                    for (int u = 0; u < 2; ++u)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const int cc = 32 * wave + M::tile(u, 4 * g + e);
                            if (cc < a.o.d) {
                                if (a.out_f32) ((float*)a.out)[at + cc] = o[u][e];
                                else put_f32((T*)a.out + at + cc, o[u][e]);
                            }
                        }
                }
            }
        }
        // the state: decay over the chunk, then k (x) v with each token's decay to its end
        const float whole = sw[count];
#pragma unroll
        for (int t = 0; t < S::kTiles; ++t) {
            x[t][0] *= whole;
            x[t][1] *= whole;
        }
#pragma unroll
        for (int s = 0; s < L / KB; ++s) {
            if (s * KB >= count) break;
            float w[VE];
#pragma unroll
            for (int e = 0; e < VE; ++e) {
                const int j = s * KB + g * VE + e;
                w[e] = j < count ? a.in_scale * sw[count - 1 - j + shift] : 0.f;
            }
            Frag part[2][M::kParts];
#pragma unroll
            for (int u = 0; u < 2; ++u) M::scaled(vf[s][u], w, part[u], M::kParts);
#pragma unroll
            for (int t = 0; t < S::kTiles; ++t) {
                const Frag kf = M::col_frag(sk + s * KB * S::kRow, S::kRow, t, lane);
#pragma unroll
                for (int n = 0; n < M::kParts; ++n)
#pragma unroll
                    for (int u = 0; u < 2; ++u) x[t][u] = M::mma(kf, part[u][n], x[t][u]);
            }
        }
        have = true;
    }
    if constexpr (STATES) {
        floatx4* s = seg_slot(seg + 1);
#pragma unroll
        for (int t = 0; t < S::kTiles; ++t)
#pragma unroll
            for (int u = 0; u < 2; ++u) s[(t * 2 + u) * 64] = x[t][u];
        return;
    }
    // zeros behind the end of the sequence, in this segment's range of tokens
    long long r_end = r_begin + (long long)a.seg_chunks * L;
    if (r_end > a.T) r_end = a.T;
    static_assert(NT % D == 0, "a thread keeps its column");
    for (long long t = (r_begin > r.len ? r_begin : r.len) + tid / D; t < r_end && tid % D < a.o.d; t += NT / D) {
        const long long at = r.b * a.o.s.b + t * a.o.s.t + r.p * a.o.s.p + (long long)(r.h / a.o.share) * a.o.s.h + tid % D;
        if (a.out_f32) ((float*)a.out)[at] = 0.f;
        else put_f32((T*)a.out + at, 0.f);
    }
    if (a.state_out && ((r.len > r_begin && c_end * (long long)L >= r.len) || (r.len == 0 && seg == 0)))
        for_state([&](int t, int u, int i, long long at) { a.state_out[at] = x[t][u][i]; });
}

// States at the start of every segment from the sums of the segments: X_{s+1} = e^{a n} X_s + sum_s, n tokens a segment.  A thread
// has four elements; slot 0 is the state that comes in.
template <class T, int D>
__global__ __launch_bounds__(256) void mix_scan_kernel(MixArgs a) {
    typedef Shape<T, D> S;
    typedef Mma<T> M;
    const long long at = (long long)blockIdx.x * 256 + threadIdx.x;
    const long long index = at / (S::kStateFloats / 4);
    if (index >= a.B * a.P * a.H) return;
    const int e = (int)(at % (S::kStateFloats / 4));
    const int lane = e & 63, u = (e >> 6) & 1, t = (e >> 7) % S::kTiles, wave = (e >> 7) / S::kTiles;
    floatx4 x{0.f, 0.f, 0.f, 0.f};
    if (a.state_in) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = M::tile(t, 4 * (lane >> 4) + i), c = 32 * wave + M::tile(u, lane & 15);
            if (row < a.k.d && c < a.v.d) x[i] = a.state_in[index * a.k.d * a.v.d + state_at(a, row, c)];
        }
    }
    const float whole = decay_of(a.log_decay[index % a.H], a.seg_chunks * S::kL);
    floatx4* s = (floatx4*)a.seg_state + index * a.n_seg * (S::kStateFloats / 4) + e;
    s[0] = x;
    for (int k = 1; k < a.n_seg; ++k) {
        x = x * whole + s[(long long)k * (S::kStateFloats / 4)];
        s[(long long)k * (S::kStateFloats / 4)] = x;
    }
}

// Sum over the output heads that share a head: float32 [B][T][P][H][d] to x.  One thread an element.
template <class T>
__global__ __launch_bounds__(256) void mix_share_kernel(const float* __restrict__ part, MixTensor x, void* out, long long T_, long long P, int H,
                                                        long long n) {
    const long long at = (long long)blockIdx.x * 256 + threadIdx.x;
    if (at >= n) return;
    const int c = (int)(at % x.d);
    long long rest = at / x.d;
    const int heads = H / x.share, h = (int)(rest % heads);
    rest /= heads;
    const long long p = rest % P, bt = rest / P, t = bt % T_, b = bt / T_;
    const float* src = part + ((bt * P + p) * H + (long long)h * x.share) * x.d + c;
    float s = src[0];
    for (int k = 1; k < x.share; ++k) s += src[(long long)k * x.d];
    put_f32((T*)out + b * x.s.b + t * x.s.t + p * x.s.p + h * x.s.h + c, s);
}

// One token: S' = e^a S + k v^T, o = scale q S'.  A workgroup has a problem; a thread has column c of dv and every R-th row.
constexpr int kStepThreads = 256;
template <class T>
__global__ __launch_bounds__(kStepThreads) void mix_step_kernel(MixArgs a) {
    __shared__ float sq[128], sk[128], red[kStepThreads];
    const Problem r = problem_of(a, blockIdx.x);
    const T *gq = base_of<T>(a.q, r), *gk = base_of<T>(a.k, r), *gv = base_of<T>(a.v, r);
    const int tid = threadIdx.x, dk = a.k.d, dv = a.v.d;
    const bool live = r.len > 0;
    if (tid < dk) {
        sq[tid] = live ? to_f32(gq[tid]) : 0.f;
        sk[tid] = live ? to_f32(gk[tid]) : 0.f;
    }
    __syncthreads();
    const int width = dv <= 32 ? 32 : dv <= 64 ? 64 : 128, c = tid % width, rows = kStepThreads / width;
    const float whole = live ? decay_of(a.log_decay[r.h], 1) : 1.f, v = c < dv && live ? to_f32(gv[c]) : 0.f;
    const long long base = r.index * dk * dv;
    float o = 0.f;
    if (c < dv)
        for (int row = tid / width; row < dk; row += rows) {
            const float s = (a.state_in ? a.state_in[base + (long long)row * dv + c] : 0.f) * whole + sk[row] * v;
            o += sq[row] * s;
            if (a.state_out) a.state_out[base + (long long)row * dv + c] = s;
        }
    red[tid] = o;
    __syncthreads();
    if (tid < dv) {
        for (int k = 1; k < rows; ++k) o += red[k * width + tid];
        put_f32((T*)a.out + r.b * a.o.s.b + r.p * a.o.s.p + r.h * a.o.s.h + tid, live ? o * a.out_scale : 0.f);
    }
}

// ------------------------------------------------------------------ host
inline size_t align_up(size_t v) { return (v + 255) / 256 * 256; }
int width_of(int dk, int dv) {
    const int d = dk > dv ? dk : dv;
    return d <= 32 ? 32 : d <= 64 ? 64 : 128;
}
// Segments of a pass: enough workgroups to fill the chip where there are few problems.
struct Split {
    int n_seg, chunks;
};
Split split_of(const gleam_linattn_desc& d) {
    const int D = width_of(d.dk, d.dv), L = d.dtype && D > 32 ? 64 : 32;
    const long long problems = d.B * d.P * d.heads, groups = D == 32 ? (problems + 3) / 4 : problems, chunks = (d.T + L - 1) / L;
    long long n = 1024 / groups;
    if (n > chunks / 4) n = chunks / 4;
    if (n < 2) return {1, (int)chunks};
    const long long per = (chunks + n - 1) / n;
    return {(int)((chunks + per - 1) / per), (int)per};
}
size_t seg_bytes(const gleam_linattn_desc& d) {
    const Split s = split_of(d);
    const size_t D = width_of(d.dk, d.dv);
    return s.n_seg < 2 ? 0 : align_up((size_t)(d.B * d.P * d.heads) * s.n_seg * D * D * sizeof(float));
}
size_t share_bytes(const gleam_linattn_desc& d) {   // float32 gradients of the widest array whose heads are shared
    size_t w = 0;
    if (d.q_heads < d.heads || d.k_heads < d.heads) w = d.dk;
    if (d.v_heads < d.heads && (size_t)d.dv > w) w = d.dv;
    return align_up((size_t)(d.B * d.T * d.P * d.heads) * w * sizeof(float));
}

template <class T, int D>
hipError_t mix_pass(MixArgs& a, const char* name, hipStream_t st) {
    typedef Shape<T, D> S;
    const long long problems = a.B * a.P * a.H;
    const unsigned groups = (unsigned)((problems + S::kProblems - 1) / S::kProblems);
    const double tokens = (double)problems * a.T;
    const double state_flops = 2.0 * a.k.d * a.v.d, bytes = sizeof(T);
    if (a.n_seg > 1) {
        {
            KernelScope ks("linattn_segments", tokens * state_flops, tokens * bytes * (a.k.d + a.v.d), st);
            hipLaunchKernelGGL((mix_kernel<T, D, true>), dim3(groups, a.n_seg - 1), dim3(S::kThreads), 0, st, a);
        }
        const double floats = (double)problems * a.n_seg * S::kStateFloats;
        KernelScope ks("linattn_scan", 2.0 * floats, 8.0 * floats, st);
        hipLaunchKernelGGL((mix_scan_kernel<T, D>), dim3((unsigned)((problems * (S::kStateFloats / 4) + 255) / 256)), dim3(256), 0, st, a);
    } else {
        a.seg_state = nullptr;
    }
    KernelScope ks(name, tokens * 2.0 * state_flops, tokens * bytes * (a.q.d + a.k.d + a.v.d + a.o.d), st);
    hipLaunchKernelGGL((mix_kernel<T, D, false>), dim3(groups, a.n_seg), dim3(S::kThreads), 0, st, a);
    return hipGetLastError();
}
template <class T>
hipError_t mix_any(MixArgs& a, const char* name, hipStream_t st) {
    switch (width_of(a.k.d, a.v.d)) {
        case 32: return mix_pass<T, 32>(a, name, st);
        case 64: return mix_pass<T, 64>(a, name, st);
        default: return mix_pass<T, 128>(a, name, st);
    }
}
hipError_t mix(const gleam_linattn_desc& d, MixArgs& a, const char* name, hipStream_t st) {
    return d.dtype ? mix_any<unsigned short>(a, name, st) : mix_any<float>(a, name, st);
}

gleam_seq_strides row_major(const gleam_linattn_desc& d, int heads, int width) {
    return {d.T * d.P * heads * width, d.P * heads * width, (int64_t)heads * width, width};
}
MixArgs common(const gleam_linattn_desc& d, const float* log_decay, const int* lengths, void* ws) {
    MixArgs a{};
    a.B = d.B;
    a.P = d.P;
    a.T = d.T;
    a.H = d.heads;
    a.log_decay = log_decay;
    a.lengths = lengths;
    a.seg_state = (float*)ws;
    const Split s = split_of(d);
    a.n_seg = s.n_seg;
    a.seg_chunks = s.chunks;
    return a;
}

}  // namespace

size_t linattn_fwd_ws_bytes(const gleam_linattn_desc& d) { return d.T == 1 ? 0 : seg_bytes(d); }
size_t linattn_bwd_ws_bytes(const gleam_linattn_desc& d) { return seg_bytes(d) + share_bytes(d); }

hipError_t linattn_forward(const gleam_linattn_desc& d, const void* q, const void* k, const void* v, const float* log_decay,
                           const int* lengths, const float* state_in, void* o, float* state_out, void* ws, hipStream_t st) {
    MixArgs a = common(d, log_decay, lengths, ws);
    a.q = {q, d.q, d.heads / d.q_heads, d.dk};
    a.k = {k, d.k, d.heads / d.k_heads, d.dk};
    a.v = {v, d.v, d.heads / d.v_heads, d.dv};
    a.o = {nullptr, d.o, 1, d.dv};
    a.out = o;
    a.state_in = state_in;
    a.state_out = state_out;
    a.in_scale = 1.f;
    a.out_scale = d.scale;
    if (d.T == 1) {
        const double states = (double)d.B * d.P * d.heads * d.dk * d.dv;
        KernelScope ks("linattn_step", 4.0 * states, 8.0 * states, st);
        const dim3 grid((unsigned)(d.B * d.P * d.heads));
        if (d.dtype) hipLaunchKernelGGL(mix_step_kernel<unsigned short>, grid, dim3(kStepThreads), 0, st, a);
        else hipLaunchKernelGGL(mix_step_kernel<float>, grid, dim3(kStepThreads), 0, st, a);
        return hipGetLastError();
    }
    return mix(d, a, "linattn_fwd", st);
}

hipError_t linattn_backward(const gleam_linattn_desc& d, const void* q, const void* k, const void* v, const float* log_decay,
                            const int* lengths, const float* state_in, const void* g_o, const float* g_state_out, void* g_q, void* g_k,
                            void* g_v, float* g_state_in, void* ws, hipStream_t st) {
    const MixTensor tq = {q, d.q, d.heads / d.q_heads, d.dk};
    const MixTensor tk = {k, d.k, d.heads / d.k_heads, d.dk};
    const MixTensor tv = {v, d.v, d.heads / d.v_heads, d.dv};
    const MixTensor tg = {g_o, d.o, 1, d.dv};
    float* part = (float*)((unsigned char*)ws + seg_bytes(d));
    // one pass into `out` of the layout of x, by way of a float32 array of all output heads where heads are shared
    auto pass = [&](MixArgs& a, const MixTensor& x, void* out, const char* name) {
        a.o = x;
        a.out = out;
        if (x.share > 1) {
            a.o.s = row_major(d, d.heads, x.d);
            a.o.share = 1;
            a.out = part;
            a.out_f32 = 1;
        }
        hipError_t e = mix(d, a, name, st);
        if (e != hipSuccess || x.share == 1) return e;
        const long long n = d.B * d.T * d.P * (d.heads / x.share) * x.d;
        KernelScope ks("linattn_share", (double)n * x.share, 4.0 * n * x.share + (d.dtype ? 2.0 : 4.0) * n, st);
        const dim3 grid((unsigned)((n + 255) / 256));
        if (d.dtype) hipLaunchKernelGGL(mix_share_kernel<unsigned short>, grid, dim3(256), 0, st, (const float*)part, x, out, d.T, d.P, d.heads, n);
        else hipLaunchKernelGGL(mix_share_kernel<float>, grid, dim3(256), 0, st, (const float*)part, x, out, d.T, d.P, d.heads, n);
        return hipGetLastError();
    };
    MixArgs a = common(d, log_decay, lengths, ws);
    a.q = tg;
    a.k = tv;
    a.v = tk;
    a.state_in = state_in;
    a.state_t = 1;
    a.in_scale = 1.f;
    a.out_scale = d.scale;
    hipError_t e = pass(a, tq, g_q, "linattn_bwd_q");
    if (e != hipSuccess) return e;
    a = common(d, log_decay, lengths, ws);
    a.reverse = 1;
    a.q = tv;
    a.k = tg;
    a.v = tq;
    a.state_in = g_state_out;
    a.state_t = 1;
    a.in_scale = d.scale;
    a.out_scale = 1.f;
    e = pass(a, tk, g_k, "linattn_bwd_k");
    if (e != hipSuccess) return e;
    a = common(d, log_decay, lengths, ws);
    a.reverse = 1;
    a.q = tk;
    a.k = tq;
    a.v = tg;
    a.state_in = g_state_out;
    a.state_out = g_state_in;
    a.in_scale = d.scale;
    a.out_scale = 1.f;
    return pass(a, tv, g_v, "linattn_bwd_v");
}

}  // namespace gleam
