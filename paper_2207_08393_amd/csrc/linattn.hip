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
// Few problems of many chunks are split along the tokens into segments: one launch forms every segment's k (x) v, a second carries the
// states from segment to segment, the third has all segments side by side; the three passes of a backward call share each of the launches.
//
// Measured (listed calls; copy rate of the card 5.2 TB/s, bfloat16 matrix products 1212 TFLOP/s):
//   4 x 2048 tokens, 16 heads of 64, bfloat16                 40 us (all read once and written once: 13)
//   16384 tokens, 16 heads of 128, 4 of k and v, gradients    320   (52)
//   3 x 1001 tokens, 6 heads of 40 and 72, float32, gradients 65    (5)
// Under a profiler, which makes them a tenth longer, segments, states and outputs take 13 + 8 + 23, 79 + 8 + 214 and 16 + 6 + 46 us, and the
// sums over the heads that share keys and values 2 x 27 in the second.
// What bounds the chunk loop at a width of 128 is no single unit: vector instructions 40 %, matrix instructions 33 %, LDS 47 % of the
// time busy, at the two workgroups of 256 registers a lane that a compute unit holds.  Tried without gain: other paddings of the LDS rows
// (0 to +3 % time), chunks without branches where they are whole.
//
// One problem is one sequence, pixel and head.  D is dk and dv rounded up to 32, 64, 96 or 128; a problem is worked on by D/32 waves, and
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
constexpr long long kFarBytes = 0x7fffffff / 64 - 128;   // between tokens: 64 of them and a row fit 31 bits

// Within each group of 16 lanes, lane s passes the address of 4 consecutive 16-bit values of row s/4; lane j gets column j of the
// 4 x 16 block, rows 0..3.
__device__ __forceinline__ uint2 read_tr16(const unsigned short* p) {
    const short4v v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((short4v __attribute__((address_space(3)))*)(p));
    return __builtin_bit_cast(uint2, v);
}

// The first `left` of N values.
template <class O, int N>
__device__ __forceinline__ void store_part(O* p, int left, const float* v) {
    if (left >= N) {
        Pack<O, N> x;
        x.set(v);
        x.store(p);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < left) put_f32(p + i, v[i]);
    }
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
    static __device__ __forceinline__ int tile4(int t, int g) { return 32 * (t >> 1) + 8 * g + 4 * (t & 1); }   // of results 4 g .. 4 g + 3
    static __device__ __forceinline__ floatx4 mma(Frag a, Frag b, floatx4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ Frag row_frag(const unsigned short* p) { return *(const Frag*)p; }
    // rows 8 g .. 8 g + 7 of the block that begins at p, column tile(t, m), or 16 t + m (PLAIN)
    template <bool PLAIN = false>
    static __device__ __forceinline__ Frag col_frag(const unsigned short* p, int stride, int t, int lane) {
        const int g = lane >> 4, s = lane & 15;
        const unsigned short* q = p + (8 * g + (s >> 2)) * stride + (PLAIN ? 16 * t + 4 * (s & 3) : 32 * (t >> 1) + 8 * (s & 3) + 4 * (t & 1));
        const uint2 lo = read_tr16(q), hi = read_tr16(q + 4 * stride);
        return __builtin_bit_cast(Frag, make_uint4(lo.x, lo.y, hi.x, hi.y));
    }
    // the same with the block's rows in the order in which score_parts has them
    static __device__ __forceinline__ Frag col_frag_of_scores(const unsigned short* p, int stride, int col, int lane) {
        const int g = lane >> 4, s = lane & 15;
        const unsigned short* q = p + (4 * g + (s >> 2)) * stride + col;
        const uint2 lo = read_tr16(q), hi = read_tr16(q + 16 * stride);
        return __builtin_bit_cast(Frag, make_uint4(lo.x, lo.y, hi.x, hi.y));
    }
    static __device__ __forceinline__ int col_of(int t, int lane) { return 32 * (t >> 1) + 8 * (lane & 3) + 4 * (t & 1); }
    static __device__ __forceinline__ int narrow_col_of(int lane) { return 4 * (lane & 3); }
    // results of two tiles (rows 4 g .. 4 g + 3 of either) as an operand.  Scores are two bfloat16 numbers each, here and in put_score: with one an
    // output is sqrt 2 times as far from exact as its own rounding, with two that alone, for 2 to 6 % more time (20 x 192 x 160 pixels, 4 heads
    // of 16: 75 -> 78 us; 4 x 2048 tokens, 16 heads of 64: 39.3 -> 40.5; 16384 tokens, 16 heads of 128, gradients: 310 -> 319).
    static constexpr int kScoreParts = 2;
    static __device__ __forceinline__ void score_parts(floatx4 a, floatx4 b, Frag* parts) {
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < 4 ? a[i] : b[i & 3];
        split(v, parts, kScoreParts);
    }
    // Parts whose sum is f times w: bfloat16 numbers w[i] f[i] rounded, what that left over rounded, and so on; 8 bits each.
    static constexpr int kStateParts = 2;
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
    // a lane's results of tiles 0 and 1 of a 32-wide block, which are its elements 8 g .. 8 g + 7
    template <class O>
    static __device__ __forceinline__ void store(O* p, int left, int g, const floatx4* o) {
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = o[i >> 2][i & 3];
        store_part<O, 8>(p + 8 * g, left - 8 * g, v);
    }
    // the same into LDS, where width and address are multiples of 16 bytes
    static __device__ __forceinline__ void keep(unsigned short* p, int width, int g, const floatx4* o) {
        if (8 * g < width) {
            put4(p + 8 * g, o[0]);
            put4(p + 8 * g + 4, o[1]);
        }
    }
    static __device__ __forceinline__ void put4(unsigned short* p, floatx4 v) {
        *(uint2*)p = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
    }
    // the same as two parts, each into an array of its own
    static __device__ __forceinline__ void put_score(unsigned short* p, unsigned short* rest, floatx4 v) {
        const unsigned a = pack_bf16x2(v[0], v[1]), b = pack_bf16x2(v[2], v[3]);
        *(uint2*)p = make_uint2(a, b);
        *(uint2*)rest = make_uint2(pack_bf16x2(v[0] - __uint_as_float(a << 16), v[1] - __uint_as_float(a & 0xffff0000u)),
                                   pack_bf16x2(v[2] - __uint_as_float(b << 16), v[3] - __uint_as_float(b & 0xffff0000u)));
    }
};
template <>
struct Mma<float> {
    static constexpr int kBlock = 16, kVec = 4;
    typedef floatx4 Frag;
    static __device__ __forceinline__ int tile(int t, int m) { return 16 * t + m; }
    static __device__ __forceinline__ int tile4(int t, int g) { return 16 * t + 4 * g; }
    static __device__ __forceinline__ floatx4 mma(Frag a, Frag b, floatx4 c) {
#pragma unroll
        for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], c, 0, 0, 0);
        return c;
    }
    static __device__ __forceinline__ Frag row_frag(const float* p) { return *(const Frag*)p; }
    template <bool PLAIN = false>
    static __device__ __forceinline__ Frag col_frag(const float* p, int stride, int t, int lane) {
        const float* q = p + 4 * (lane >> 4) * stride + 16 * t + (lane & 15);
        return Frag{q[0], q[stride], q[2 * stride], q[3 * stride]};
    }
    static __device__ __forceinline__ Frag col_frag_of_scores(const float* p, int stride, int col, int lane) {
        const float* q = p + 4 * (lane >> 4) * stride + col;
        return Frag{q[0], q[stride], q[2 * stride], q[3 * stride]};
    }
    static __device__ __forceinline__ int col_of(int t, int lane) { return 16 * t + (lane & 15); }
    static __device__ __forceinline__ int narrow_col_of(int lane) { return lane & 15; }
    static constexpr int kScoreParts = 1;
    static __device__ __forceinline__ void score_parts(floatx4 a, floatx4, Frag* parts) { parts[0] = a; }
    static constexpr int kStateParts = 1;
    static __device__ __forceinline__ void scaled(Frag f, const float* w, Frag* parts, int) { parts[0] = Frag{f[0] * w[0], f[1] * w[1], f[2] * w[2], f[3] * w[3]}; }
    static __device__ __forceinline__ void pack(const floatx4* x, Frag* parts) { parts[0] = x[0]; }
    template <class O>
    static __device__ __forceinline__ void store(O* p, int left, int g, const floatx4* o) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const float v[4] = {o[u][0], o[u][1], o[u][2], o[u][3]};
            store_part<O, 4>(p + 16 * u + 4 * g, left - 16 * u - 4 * g, v);
        }
    }
    static __device__ __forceinline__ void keep(float* p, int width, int g, const floatx4* o) {
#pragma unroll
        for (int u = 0; u < 2; ++u)
            if (16 * u + 4 * g < width) put4(p + 16 * u + 4 * g, o[u]);
    }
    static __device__ __forceinline__ void put4(float* p, floatx4 v) { *(floatx4*)p = v; }
    static __device__ __forceinline__ void put_score(float* p, float*, floatx4 v) { put4(p, v); }
};

// 16 bytes from byte `at` of a buffer; zeros beyond its end (also for a negative `at`).  A plain function: the host pass drops the
// stub of a kernel template whose own body makes this call.
__device__ __forceinline__ void load_buffer(__amdgpu_buffer_rsrc_t rs, int at, unsigned* w) {
    typedef unsigned uint4v __attribute__((ext_vector_type(4)));
    const uint4v v = __builtin_amdgcn_raw_buffer_load_b128(rs, at, 0, 0);
    w[0] = v[0];
    w[1] = v[1];
    w[2] = v[2];
    w[3] = v[3];
}

// e^{a n}; 1 for n = 0 whatever a is.
__device__ __forceinline__ float decay_of(float a, int n) { return n == 0 ? 1.f : __builtin_amdgcn_exp2f(a * kLog2e * (float)n); }

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

// The elements [col, col + VE) of rows of d elements that exist.
template <class T>
struct Edge {
    static constexpr int VE = 16 / (int)sizeof(T);
    int at, back, d;     // where the vector is read, elements in front of those that are wanted, width
    bool live, narrow;   // whether any exists; whether a row is shorter than a vector (then none of this is used)
    __device__ __forceinline__ Edge(int col, int width) {
        d = width;
        narrow = d < VE;
        live = col < d;
        back = live && col + VE > d && !narrow ? col + VE - d : 0;
        at = live ? col - back : 0;
    }
    __device__ __forceinline__ Pack<T, VE> in_place(Pack<T, VE> x) const {
        if (d % VE) {
            unsigned long long lo = x.w[0] | (unsigned long long)x.w[1] << 32, hi = x.w[2] | (unsigned long long)x.w[3] << 32;
            const int bits = 8 * (int)sizeof(T) * back, b = bits & 63;
            const unsigned long long from_hi = b ? hi << (64 - b) : 0;
            lo = bits >= 64 ? hi >> b : lo >> b | from_hi;
            hi = bits >= 64 ? 0 : hi >> b;
            x.w[0] = (unsigned)lo;
            x.w[1] = (unsigned)(lo >> 32);
            x.w[2] = (unsigned)hi;
            x.w[3] = (unsigned)(hi >> 32);
        }
        return x;
    }
    // zeros where nothing exists, the rest in its place
    __device__ __forceinline__ Pack<T, VE> settle(Pack<T, VE> x, bool there) const {
        x = in_place(x);
#pragma unroll
        for (int i = 0; i < 4; ++i) x.w[i] = there && live ? x.w[i] : 0;
        return x;
    }
};

struct Problem {
    long long index;    // (b P + p) H + h
    long long b, p;
    int h, len;         // head, tokens
};
__device__ __forceinline__ Problem problem_of(const MixArgs& a, long long index) {   // there are fewer than 2^31
    Problem r;
    r.index = index;
    const unsigned i = (unsigned)index, rest = i / (unsigned)a.H, b = rest / (unsigned)a.P;
    r.h = (int)(i - rest * (unsigned)a.H);
    r.p = rest - b * (unsigned)a.P;
    r.b = b;
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

// What a workgroup works on.  Workgroups are dealt to the 8 XCDs by their number, and each XCD has its own L2, so an XCD gets a
// contiguous range of the work: heads that share keys, and the passes of a backward call over the same tokens, run next to each other on
// one XCD and read from its L2 what the first of them fetched.
struct Work {
    long long group;    // of S::kProblems problems
    int seg, role;
    bool none;
};
__device__ __forceinline__ Work work_of(const MixArgs& a, unsigned groups, unsigned segs, unsigned roles) {
    const unsigned total = groups * segs * roles, per = (total + 7) / 8, n = (unsigned)group_of_grid(), i = (n & 7) * per + (n >> 3);
    Work w;
    w.none = n >> 3 >= per || i >= total;
    const unsigned inner = a.near_groups, outer = i / (inner * segs * roles), in = i - outer * (inner * segs * roles);
    const unsigned in_seg = in / (inner * roles), rest = in - in_seg * (inner * roles);
    w.role = rest / inner;
    w.group = (long long)outer * inner + (rest - w.role * inner);
    w.seg = in_seg;
    return w;
}

// STATES: only the sum of k (x) v over a segment, for the scan over segments; slot seg + 1 of seg_state.
// PARTS: numbers a decayed value is the sum of on its way into the state (bfloat16: 3 give 24 bits, for a state that is handed out; 2
// where the state only feeds outputs, which are rounded to 8 bits).
// NARROW: rows shorter than a vector, and tokens so far apart that a chunk's offsets pass 31 bits, go element by element, nothing
// ahead of time.  (A kernel of its own: where one kernel has both ways the compiler waits for loads in flight when it reuses their
// registers, since it cannot see that they have arrived.)
template <class T, int D, bool STATES, int PARTS, bool NARROW>
__global__ __launch_bounds__((Shape<T, D>::kThreads), (STATES && PARTS < 3 ? 3 : 2)) void mix_kernel(MixArgs args) {
    typedef Shape<T, D> S;
    typedef Mma<T> M;
    typedef typename M::Frag Frag;
    constexpr int L = S::kL, VE = M::kVec, KB = M::kBlock, W = S::kWaves, NT = 64 * W;
    constexpr int NV = L * D / VE / NT;               // 16-byte vectors of an array a lane stages
    constexpr int kPair = KB / 16;                    // result tiles that make an operand
    constexpr int kRows = L / 16;                     // row tiles of a chunk
    __shared__ __attribute__((aligned(16))) T lds_q[STATES ? 1 : S::kProblems][STATES ? 8 : L * S::kRow];
    __shared__ __attribute__((aligned(16))) T lds_k[S::kProblems][L * S::kRow];
    __shared__ __attribute__((aligned(16))) T lds_v[S::kProblems][L * S::kRow];
    __shared__ __attribute__((aligned(16))) T lds_p[STATES ? 1 : S::kProblems][STATES ? 8 : L * S::kScoreRow];
    __shared__ __attribute__((aligned(16))) float lds_w[S::kProblems][L + 4];   // decay over n tokens
    __shared__ __attribute__((aligned(16))) float lds_e[S::kProblems][L];       // from token j to the end of a whole chunk, with scale
    const int slot = S::kProblems == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int tid = S::kProblems == 1 ? threadIdx.x : threadIdx.x & 63;
    const int lane = tid & 63, m = lane & 15, g = lane >> 4;
    const int wave = W == 1 ? 0 : __builtin_amdgcn_readfirstlane(tid >> 6);
    const Work work = work_of(args, args.groups, STATES ? args.n_seg - 1 : args.n_seg, args.roles);
    if (work.none) return;
    const MixRole& a = args.role[work.role];
    const long long index = work.group * S::kProblems + slot;
    if (index >= args.B * args.P * args.H) return;    // several problems a workgroup: a wave each, and no barriers
    const Problem r = problem_of(args, index);
    // passes in reverse count segments from the end: those over the same tokens stand next to each other
    const int seg = a.reverse ? (STATES ? args.n_seg - 2 : args.n_seg - 1) - work.seg : work.seg;
    const int c_begin = seg * args.seg_chunks;
    int c_end = (r.len + L - 1) / L;
    if (c_end > c_begin + args.seg_chunks) c_end = c_begin + args.seg_chunks;
    const bool last_seg = (r.len > c_begin * L && c_end * L >= r.len) || (r.len == 0 && seg == 0);
    const int shift = a.reverse;
    const float decay = args.log_decay[r.h];
    T *sq = lds_q[STATES ? 0 : slot], *sk = lds_k[slot], *sv = lds_v[slot], *sp = lds_p[STATES ? 0 : slot];
    float *sw = lds_w[slot], *se = lds_e[slot];
    for (int i = tid; i < L + 2; i += NT) sw[i] = decay_of(decay, i);
    for (int i = tid; i < L; i += NT) se[i] = a.in_scale * decay_of(decay, L - 1 - i + shift);

    // tokens of the chunk from the first one on (or, in reverse, from the last one down)
    const long long way = a.reverse ? -1 : 1, start = a.reverse ? r.len - 1 : 0;
    // Staging: vectors tid + i NT of the chunk's rows, read a chunk ahead from a buffer that holds the chunk's tokens and ends with the
    // last of them: rows behind the sequence's end are out of its range, so they need no branch and touch no memory, and become zero on the
    // way into LDS.  A row's last vector ends with the row and is moved into place there.
    const int col = tid % (D / VE) * VE, row0 = tid / (D / VE);
    constexpr int kRowStep = NT / (D / VE);
    const Edge<T> ek(col, a.k.d), ev(col, a.v.d);
    const T *gq = base_of<T>(a.q, r), *gk = base_of<T>(a.k, r), *gv = base_of<T>(a.v, r);
    Pack<T, VE> nq[NV], nk[NV], nv[NV];
    auto fetch_array = [&](int c, int count, const T* base, long long t, const Edge<T>& e, Pack<T, VE>(&n)[NV]) {
        const T* low = base + (start + way * (c * L + (a.reverse ? count - 1 : 0))) * t;
        const int token = (int)(t * (long long)sizeof(T));
        const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc((void*)low, 0, (count - 1) * token + e.d * (int)sizeof(T), 0x00027000);
        const int first = (a.reverse ? count - 1 - row0 : row0) * token + e.at * (int)sizeof(T), step = (a.reverse ? -kRowStep : kRowStep) * token;
#pragma unroll
        for (int i = 0; i < NV; ++i) load_buffer(rs, first + i * step, n[i].w);
    };
    auto fetch = [&](int c) {
        if (NARROW) return;
        const int left = r.len - c * L, count = left < L ? left : L;
        if constexpr (!STATES) fetch_array(c, count, gq, a.q.s.t, ek, nq);
        fetch_array(c, count, gk, a.k.s.t, ek, nk);
        fetch_array(c, count, gv, a.v.s.t, ev, nv);
    };
    auto stage = [&](int c, int count) {
        if (NARROW) {
            for (int e = tid; e < L * S::kRow; e += NT) {
                const int row = e / S::kRow, cc = e % S::kRow, at = c * L + row;
                const long long token = a.reverse ? r.len - 1 - at : at;
                if constexpr (!STATES) sq[e] = row < count && cc < a.q.d ? gq[token * a.q.s.t + cc] : (T)0;
                sk[e] = row < count && cc < a.k.d ? gk[token * a.k.s.t + cc] : (T)0;
                sv[e] = row < count && cc < a.v.d ? gv[token * a.v.s.t + cc] : (T)0;
            }
            return;
        }
        const bool as_is = count == L && a.k.d == D && a.v.d == D;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int row = row0 + i * kRowStep, at = row * S::kRow + col;
            if (as_is) {
                if constexpr (!STATES) nq[i].store_lds(sq + at);
                nk[i].store_lds(sk + at);
                nv[i].store_lds(sv + at);
            } else {
                if constexpr (!STATES) ek.settle(nq[i], row < count).store_lds(sq + at);
                ek.settle(nk[i], row < count).store_lds(sk + at);
                ev.settle(nv[i], row < count).store_lds(sv + at);
            }
        }
    };

    floatx4 x[S::kTiles][2];                          // the state: rows of tile t, columns 32 wave + tile(u, m)
    bool have = false;                                // it is not zero
#pragma unroll
    for (int t = 0; t < S::kTiles; ++t) x[t][0] = x[t][1] = floatx4{0.f, 0.f, 0.f, 0.f};
    // f(tile t, u, values there are, offset of the first and between them in the layer's [dk][dv]) of every four elements of the lane
    auto for_state = [&](auto&& f) {
#pragma unroll
        for (int t = 0; t < S::kTiles; ++t)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int row = M::tile4(t, g), c = 32 * wave + M::tile(u, m), pitch = args.dv;
                f(t, u, c < a.v.d ? a.k.d - row : 0, a.state_t ? c * pitch + row : row * pitch + c, a.state_t ? 1 : pitch);
            }
    };
    const long long state_base = r.index * args.dk * args.dv;
    auto segment = [&](int s) { return a.seg_state + (r.index * args.n_seg + s) * S::kStateFloats; };
    if (c_begin < c_end) fetch(c_begin);
    if constexpr (!STATES) {
        if (a.seg_state) {
            const float* s = segment(seg);
            // [column][row] of the pass over segments, whose roles are this pass's or (seg_t) exchanged
#pragma unroll
            for (int t = 0; t < S::kTiles; ++t)
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const int row = M::tile4(t, g), c = 32 * wave + M::tile(u, m);
                    if (!a.seg_t) x[t][u] = *(const floatx4*)(s + c * D + row);
                    else x[t][u] = floatx4{s[row * D + c], s[(row + 1) * D + c], s[(row + 2) * D + c], s[(row + 3) * D + c]};
                }
            have = seg > 0 || a.state_in;
        } else if (a.state_in) {
            for_state([&](int t, int u, int left, int at, int step) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (i < left) x[t][u][i] = a.state_in[state_base + at + i * step];
            });
            have = true;
        }
    }
    // decays between a row and a column of scores whose tiles are n apart (0 where the column is the later one), and with scale
    floatx4 wt[STATES ? 1 : kRows];
    if constexpr (!STATES) {
#pragma unroll
        for (int n = 0; n < kRows; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int apart = 16 * n + m - 4 * g - i;
                wt[n][i] = apart < 0 ? 0.f : a.in_scale * a.out_scale * decay_of(decay, apart);
            }
    }
    long long out_at = r.b * a.o.s.b + r.p * a.o.s.p + (long long)(r.h / a.o.share) * a.o.s.h + (start + way * ((long long)c_begin * L + m)) * a.o.s.t + 32 * wave;
    const long long out_step = way * 16 * a.o.s.t;
    // Scores into LDS, rows `it`: the lane has four consecutive columns of row m of the tile.  Their second parts take the place of the
    // values, which are in registers by then.
    auto scores = [&](int count) {
#pragma unroll
        for (int rr = 0; rr < (kRows + W - 1) / W; ++rr) {
            const int it = wave + rr * W;
            if (it < kRows && it * 16 < count) {
                Frag qf[D / KB];
#pragma unroll
                for (int s = 0; s < D / KB; ++s) qf[s] = M::row_frag(sq + (16 * it + m) * S::kRow + s * KB + g * VE);
#pragma unroll
                for (int n = 0; n < kRows; ++n) {
                    if (n >= rr * W + W) continue;            // n <= it, whatever the wave
                    // a tile beyond the first column: zeros into tile n, right of the diagonal
                    const int jt = it >= n ? it - n : n;
                    floatx4 p{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int s = 0; s < D / KB; ++s) p = M::mma(M::row_frag(sk + (16 * jt + m) * S::kRow + s * KB + g * VE), qf[s], p);
#pragma unroll
                    for (int i = 0; i < 4; ++i) p[i] = (n > 0 || m >= 4 * g + i) && it >= n ? p[i] * wt[n][i] : 0.f;
                    const int at = (16 * it + m) * S::kScoreRow + 16 * jt + 4 * g;
                    M::put_score(sp + at, sv + at, p);
                }
                // the tile right of the diagonal, where it shares an operand with it and is not among those
                if (kPair == 2 && W % 2 && !(it & 1)) {
                    const int at = (16 * it + m) * S::kScoreRow + 16 * (it + 1) + 4 * g;
                    M::put_score(sp + at, sv + at, floatx4{0.f, 0.f, 0.f, 0.f});
                }
            }
        }
    };
    // What the queries read of the state.
    auto from_state = [&](floatx4(&o)[kRows][2]) {
#pragma unroll
        for (int s = 0; s < D / KB; ++s) {
            Frag xf[2][M::kStateParts];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const floatx4 both[2] = {x[kPair * s][u], x[kPair * s + kPair - 1][u]};
                M::pack(both, xf[u]);
            }
#pragma unroll
            for (int it = 0; it < kRows; ++it) {
                const Frag qf = M::row_frag(sq + (16 * it + m) * S::kRow + s * KB + g * VE);
#pragma unroll
                for (int n = 0; n < M::kStateParts; ++n)
#pragma unroll
                    for (int u = 0; u < 2; ++u) o[it][u] = M::mma(xf[u][n], qf, o[it][u]);
            }
        }
#pragma unroll
        for (int it = 0; it < kRows; ++it) {
            const float f = a.out_scale * sw[16 * it + m + 1 - shift];
            o[it][0] *= f;
            o[it][1] *= f;
        }
    };
    auto from_chunk = [&](int count, const Frag(&vf)[L / KB][2], floatx4(&o)[kRows][2]) {
#pragma unroll
        for (int it = 0; it < kRows; ++it) {
            if (it * 16 >= count) break;
#pragma unroll
            for (int s = 0; s <= it * 16 / KB; ++s) {
#pragma unroll
                for (int n = 0; n < M::kScoreParts; ++n) {
                    const Frag pf = M::row_frag((n ? sv : sp) + (16 * it + m) * S::kScoreRow + s * KB + g * VE);
#pragma unroll
                    for (int u = 0; u < 2; ++u) o[it][u] = M::mma(vf[s][u], pf, o[it][u]);
                }
            }
        }
        auto put = [&](auto* out) {
#pragma unroll
            for (int it = 0; it < kRows; ++it)
                if (16 * it + m < count) M::store(out + out_at + it * out_step, a.o.d - 32 * wave, g, o[it]);
        };
        if (a.out_f32) put((float*)a.out);
        else put((T*)a.out);
        out_at += kRows * out_step;
    };
    for (int c = c_begin; c < c_end; ++c) {
        const int left = r.len - c * L, count = left < L ? left : L;
        exchange<W>();                                // everyone is done with the chunk before
        stage(c, count);
        exchange<W>();
        if (c + 1 < c_end) fetch(c + 1);
        Frag vf[L / KB][2];
#pragma unroll
        for (int s = 0; s < L / KB; ++s)
#pragma unroll
            for (int u = 0; u < 2; ++u) vf[s][u] = M::template col_frag<STATES>(sv + s * KB * S::kRow, S::kRow, 2 * wave + u, lane);
        if constexpr (!STATES) {
            floatx4 o[kRows][2] = {};
            if constexpr (M::kScoreParts > 1) exchange<W>();          // everyone has its values
            scores(count);
            if (have) from_state(o);                  // needs no scores, so it stands in front of their exchange
            exchange<W>();
            from_chunk(count, vf, o);
        }
        // the state: decay over the chunk, then k (x) v with each token's decay to its end; not where nothing reads it
        if (!STATES && c + 1 == c_end && !(a.state_out && last_seg)) break;
        const float whole = sw[count];
#pragma unroll
        for (int t = 0; t < S::kTiles; ++t) {
            x[t][0] *= whole;
            x[t][1] *= whole;
        }
#pragma unroll
        for (int s = 0; s < L / KB; ++s) {            // tokens behind the end are zeros: their weights only have to be finite
            float w[VE];
            if (count == L) {
#pragma unroll
                for (int e = 0; e < VE; e += 4) *(floatx4*)(w + e) = *(const floatx4*)(se + s * KB + g * VE + e);
            } else {
#pragma unroll
                for (int e = 0; e < VE; ++e) {
                    const int j = s * KB + g * VE + e;
                    w[e] = j < count ? se[j + L - count] : 0.f;
                }
            }
            Frag part[2][PARTS];
#pragma unroll
            for (int u = 0; u < 2; ++u) M::scaled(vf[s][u], w, part[u], PARTS);
#pragma unroll
            for (int t = 0; t < S::kTiles; ++t) {
                const Frag kf = M::template col_frag<STATES>(sk + s * KB * S::kRow, S::kRow, t, lane);
#pragma unroll
                for (int n = 0; n < PARTS; ++n)
#pragma unroll
                    for (int u = 0; u < 2; ++u) x[t][u] = M::mma(kf, part[u][n], x[t][u]);
            }
        }
        have = true;
    }
    if constexpr (STATES) {
        float* s = segment(seg + 1);
#pragma unroll
        for (int t = 0; t < S::kTiles; ++t)           // tiles in their own order here: whole 64 bytes of a column
#pragma unroll
            for (int u = 0; u < 2; ++u) *(floatx4*)(s + (32 * wave + 16 * u + m) * D + 16 * t + 4 * g) = x[t][u];
        return;
    }
    // zeros behind the end of the sequence, in this segment's range of tokens
    const long long r_begin = (long long)c_begin * L;
    long long r_end = r_begin + (long long)args.seg_chunks * L;
    if (r_end > args.T) r_end = args.T;
    static_assert(NT % D == 0, "a thread keeps its column");
    for (long long t = (r_begin > r.len ? r_begin : r.len) + tid / D; t < r_end && tid % D < a.o.d; t += NT / D) {
        const long long at = r.b * a.o.s.b + t * a.o.s.t + r.p * a.o.s.p + (long long)(r.h / a.o.share) * a.o.s.h + tid % D;
        if (a.out_f32) ((float*)a.out)[at] = 0.f;
        else put_f32((T*)a.out + at, 0.f);
    }
    if (a.state_out && last_seg)
        for_state([&](int t, int u, int left, int at, int step) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (i < left) a.state_out[state_base + at + i * step] = x[t][u][i];
        });
}

// ------------------------------------------------------------------ short sequences of narrow heads
// At most 64 tokens of at most 32 values without a state, as the frames of a series at one pixel: a wave has a whole problem, all
// three gradients of it in the backward pass.  Scores go from the result of one product to the operand of the next in registers: the
// contracted tokens may come in any order that both operands have.
// 20 x 192 x 160 pixels, 4 heads of 16, bfloat16: 78 us, 4.0 TB/s, bound by vector instructions (85 % of the time busy) and memory (275 us by
// the kernel above); gradients 210 us, 2.6 TB/s.
// TT: tiles of 16 tokens.  U: tiles of 16 columns.
// ROWS: the four problems of a workgroup are neighbouring heads of a pixel, whose values lie side by side; the workgroup moves whole
// rows of the four through LDS.  Otherwise an operand whose rows are tokens is loaded straight from memory in the layout of the product,
// and LDS only turns over those whose contracted index is the token; there are no barriers then.
constexpr int kShortTokens = 64, kShortWidth = 32, kShortWaves = 4;

template <class T, int TT, int U, bool BWD, bool ROWS>
__global__ __launch_bounds__(64 * kShortWaves) void mix_short_kernel(MixArgs args) {
    typedef Mma<T> M;
    typedef typename M::Frag Frag;
    constexpr int VE = M::kVec, KB = M::kBlock, KS = (16 * U + KB - 1) / KB, kPair = KB / 16, TS = (TT + kPair - 1) / kPair;
    constexpr int kArrays = ROWS ? (BWD ? 4 : 3) : (BWD ? 3 : 1), kTokens = TS * KB;
    // between tokens in LDS: a wave's own columns, or those of four heads
    constexpr int kRow = ROWS ? 4 * 16 * U + VE : 32 + VE;
    __shared__ __attribute__((aligned(16))) T lds[ROWS ? 1 : kShortWaves][kArrays][kTokens * kRow];
    __shared__ float weights[kShortWaves][16 + kShortTokens];
    const int lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4, slot = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const long long index = group_of_grid() * kShortWaves + slot;
    if (index >= args.B * args.P * args.H) return;   // not where ROWS: a multiple of four heads
    const Problem r = problem_of(args, index);
    const float decay = args.log_decay[r.h];
    auto own = [&](int which, int width) { return lds[ROWS ? 0 : slot][which] + (ROWS ? slot * width : 0); };

    // ROWS: tokens of the four heads to LDS and back, 16 bytes a lane, zeros behind the sequence's end.  f(token, first value)
    // of the vectors of this lane; the products fit 24 bits by the rule that chooses ROWS.
    auto vectors = [&](int width, int tokens, auto&& f) {
        const int per = 4 * width / VE, n = tokens * per;
        const float share = 1.f / (float)per;
        for (int v = threadIdx.x; v < n; v += 64 * kShortWaves) {
            const int t = (int)(((float)v + 0.5f) * share);
            f(t, (v - t * per) * VE);
        }
    };
    auto take = [&](const MixTensor& x, int which) {
        const T* base = (const T*)x.p + r.b * x.s.b + r.p * x.s.p + (long long)(r.h - slot) * x.s.h;
        vectors(x.d, kTokens, [&](int t, int c) {
            Pack<T, VE> n{};
            if (t < r.len) n.load(base + (unsigned)(__umul24(t, (unsigned)x.s.t) + c));
            n.store_lds(lds[0][which] + t * kRow + c);
        });
    };
    auto give = [&](const MixRole& ro, int which) {
        T* base = (T*)ro.out + r.b * ro.o.s.b + r.p * ro.o.s.p + (long long)(r.h - slot) * ro.o.s.h;
        vectors(ro.o.d, (int)args.T, [&](int t, int c) {
            uint4 n = *(const uint4*)(lds[0][which] + t * kRow + c);
            if (t >= r.len) n = make_uint4(0, 0, 0, 0);           // behind the end, also where a token before it is not finite
            __builtin_memcpy(base + (unsigned)(__umul24(t, (unsigned)ro.o.s.t) + c), &n, 16);
        });
    };
    // rows of tokens in the layout of an operand: token 16 t + m, values s KB + g VE on
    auto rows = [&](const MixTensor& x, int which, Frag(&f)[TT][KS]) {
        if constexpr (ROWS) {
#pragma unroll
            for (int t = 0; t < TT; ++t)
#pragma unroll
                for (int s = 0; s < KS; ++s) {
                    const int c = s * KB + g * VE;
                    f[t][s] = c < x.d ? M::row_frag(own(which, x.d) + (16 * t + m) * kRow + c) : Frag{};
                }
            return;
        }
        // lanes without values load nothing: addresses are what bounds this, one a lane (20 x 192 x 160 pixels, 4 heads of 16:
        // 124 us where all lanes load, 110 so)
        const T* base = base_of<T>(x, r);
        Pack<T, VE> n[TT][KS];
#pragma unroll
        for (int t = 0; t < TT; ++t)
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                const Edge<T> e(s * KB + g * VE, x.d);
#pragma unroll
                for (int i = 0; i < 4; ++i) n[t][s].w[i] = 0;
                if (16 * t + m < r.len && e.live && !e.narrow) n[t][s].load(base + (16 * t + m) * x.s.t + e.at);
            }
#pragma unroll
        for (int t = 0; t < TT; ++t)
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                if (x.d < VE) {                       // rows shorter than a vector
                    float v[VE];
#pragma unroll
                    for (int i = 0; i < VE; ++i) v[i] = 16 * t + m < r.len && s * KB + g * VE + i < x.d ? to_f32(base[(16 * t + m) * x.s.t + g * VE + i]) : 0.f;
                    n[t][s].set(v);
                } else {
                    n[t][s] = Edge<T>(s * KB + g * VE, x.d).in_place(n[t][s]);
                }
                f[t][s] = __builtin_bit_cast(Frag, n[t][s]);
            }
    };
    auto turn = [&](const Frag(&f)[TT][KS], int which) {
        if constexpr (!ROWS) {
#pragma unroll
            for (int t = 0; t < TS * kPair; ++t)
#pragma unroll
                for (int s = 0; s < KS; ++s) *(Frag*)(lds[slot][which] + (16 * t + m) * kRow + s * KB + g * VE) = t < TT ? f[t < TT ? t : 0][s] : Frag{};
        }
    };
    // tokens of block s of the columns of tile u; columns that do not exist only reach results that are not stored
    auto turned = [&](int which, int width, int s, int u) {
        return M::col_frag_of_scores(own(which, width) + s * KB * kRow, kRow, U == 1 ? M::narrow_col_of(lane) : M::col_of(u, lane), lane);
    };
    auto store = [&](const MixRole& ro, int which, int t, const floatx4(&o)[U]) {
        T* keep = own(which, ro.o.d) + (16 * t + m) * kRow;       // ROWS: in the place of the wave's own columns of an input
        if (!ROWS && 16 * t + m >= r.len) return;
        const long long at = r.b * ro.o.s.b + (16 * t + m) * ro.o.s.t + r.p * ro.o.s.p + (long long)(r.h / ro.o.share) * ro.o.s.h;
        if constexpr (U == 1) {
            const float v[4] = {o[0][0], o[0][1], o[0][2], o[0][3]};
            if constexpr (ROWS) {
                if (4 * g < ro.o.d) M::put4(keep + 4 * g, o[0]);
            } else if (ro.out_f32) {
                store_part<float, 4>((float*)ro.out + at + 4 * g, ro.o.d - 4 * g, v);
            } else {
                store_part<T, 4>((T*)ro.out + at + 4 * g, ro.o.d - 4 * g, v);
            }
        } else {
            if constexpr (ROWS) M::keep(keep, ro.o.d, g, o);
            else if (ro.out_f32) M::store((float*)ro.out + at, ro.o.d, g, o);
            else M::store((T*)ro.out + at, ro.o.d, g, o);
        }
    };
    if constexpr (!ROWS) {                           // zeros behind the end, whatever the tokens before it hold
        if (r.len < args.T) {
#pragma unroll
            for (int i = 0; i < (BWD ? 3 : 1); ++i) {
                const MixRole& ro = args.role[i];
                const int c = lane & 31;
                for (int t = r.len + (lane >> 5); t < args.T && c < ro.o.d; t += 2) {
                    const long long at = r.b * ro.o.s.b + t * ro.o.s.t + r.p * ro.o.s.p + (long long)(r.h / ro.o.share) * ro.o.s.h + c;
                    if (ro.out_f32) ((float*)ro.out)[at] = 0.f;
                    else put_f32((T*)ro.out + at, 0.f);
                }
            }
        }
        if (r.len == 0) return;
    }
    // decays of scores whose tiles are n apart, with scale: the later token's row m, or (up) the earlier one's
    const float scale = args.role[0].in_scale * args.role[0].out_scale;
    float* table = weights[slot];
    if (lane < 16) table[lane] = 0.f;
    table[16 + lane] = scale * decay_of(decay, lane);
    exchange<1>();
    floatx4 down[TT], up[BWD ? TT : 1];
#pragma unroll
    for (int n = 0; n < TT; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            down[n][i] = table[16 + m - 4 * g + 16 * n - i];
            if constexpr (BWD) up[n][i] = table[16 + 4 * g - m + 16 * n + i];
        }
    // scores of the tiles of one output row tile as operands: columns of the product are the output's tokens, which are the later
    // (UP: the earlier) ones of the two; tiles that the mask leaves out are zero
    auto scores = [&](const Frag(&contracted)[TT][KS], const Frag(&output)[TT][KS], int t, const floatx4* w, bool is_up, Frag(&p)[TS][M::kScoreParts]) {
        floatx4 tile[2 * TS];
#pragma unroll
        for (int j = 0; j < 2 * TS; ++j) {
            tile[j] = floatx4{0.f, 0.f, 0.f, 0.f};
            const int n = is_up ? j - t : t - j;     // tiles apart
            if (j >= TT || n < 0) continue;
#pragma unroll
            for (int s = 0; s < KS; ++s) tile[j] = M::mma(contracted[j][s], output[t][s], tile[j]);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const bool masked = n == 0 && (is_up ? 4 * g + i < m : m < 4 * g + i);
                tile[j][i] = masked ? 0.f : tile[j][i] * w[n][i];
            }
        }
#pragma unroll
        for (int s = 0; s < TS; ++s) M::score_parts(tile[kPair * s], tile[kPair * s + kPair - 1], p[s]);
    };
    auto product = [&](int which, int width, const Frag(&p)[TS][M::kScoreParts], int t, bool is_up, floatx4(&o)[U]) {
#pragma unroll
        for (int u = 0; u < U; ++u) o[u] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < TS; ++s) {
            if (is_up ? (s + 1) * kPair <= t : s * kPair > t) continue;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const Frag f = turned(which, width, s, u);
#pragma unroll
                for (int n = 0; n < M::kScoreParts; ++n) o[u] = M::mma(f, p[s][n], o[u]);
            }
        }
    };
    if constexpr (!BWD) {
        const MixRole& ro = args.role[0];
        Frag q[TT][KS], k[TT][KS], v[TT][KS];
        if constexpr (ROWS) {
            take(ro.v, 0);
            take(ro.q, 1);
            take(ro.k, 2);
            __syncthreads();
        }
        rows(ro.q, 1, q);
        rows(ro.k, 2, k);
        if constexpr (!ROWS) rows(ro.v, 0, v);
        turn(v, 0);
        if constexpr (!ROWS) exchange<1>();
        floatx4 o[TT][U];
#pragma unroll
        for (int t = 0; t < TT; ++t) {
            Frag p[TS][M::kScoreParts];
            scores(k, q, t, down, false, p);
            product(0, ro.v.d, p, t, false, o[t]);
            if constexpr (!ROWS) store(ro, 0, t, o[t]);
        }
        if constexpr (ROWS) {
            exchange<1>();                           // the wave is done with its own columns of v
#pragma unroll
            for (int t = 0; t < TT; ++t) store(ro, 0, t, o[t]);
            __syncthreads();
            give(ro, 0);
        }
    } else {
        const MixRole &rq = args.role[0], &rk = args.role[1], &rv = args.role[2];
        Frag q[TT][KS], k[TT][KS], v[TT][KS], go[TT][KS];
        if constexpr (ROWS) {
            take(rv.q, 0);
            take(rv.k, 1);
            take(rq.q, 2);
            take(rq.k, 3);
            __syncthreads();
        }
        rows(rv.k, 1, q);
        rows(rv.q, 0, k);
        rows(rq.k, 3, v);
        rows(rq.q, 2, go);
        turn(k, 0);
        turn(q, 1);
        turn(go, 2);
        if constexpr (!ROWS) exchange<1>();
        floatx4 oq[TT][U], ok[TT][U], ov[TT][U];
#pragma unroll
        for (int t = 0; t < TT; ++t) {
            Frag p[TS][M::kScoreParts];
            scores(v, go, t, down, false, p);        // g_q of token t: earlier tokens' keys
            product(0, rv.q.d, p, t, false, oq[t]);
            if constexpr (!ROWS) store(rq, 0, t, oq[t]);
            scores(go, v, t, up, true, p);           // g_k: later tokens' queries
            product(1, rv.k.d, p, t, true, ok[t]);
            if constexpr (!ROWS) store(rk, 0, t, ok[t]);
            scores(q, k, t, up, true, p);            // g_v: later tokens' gradients
            product(2, rq.q.d, p, t, true, ov[t]);
            if constexpr (!ROWS) store(rv, 0, t, ov[t]);
        }
        if constexpr (ROWS) {
            exchange<1>();
#pragma unroll
            for (int t = 0; t < TT; ++t) {
                store(rq, 1, t, oq[t]);
                store(rk, 0, t, ok[t]);
                store(rv, 3, t, ov[t]);
            }
            __syncthreads();
            give(rq, 1);
            give(rk, 0);
            give(rv, 3);
        }
    }
}

// States at the start of every segment from the sums of the segments: X_{s+1} = e^{a n} X_s + sum_s, n tokens a segment.  A thread
// has four elements; slot 0 is the state that comes in.
template <int D>
__global__ __launch_bounds__(256) void mix_scan_kernel(MixArgs args, int chunk) {
    const MixRole& a = args.role[blockIdx.z];
    constexpr int kQuads = D * D / 4;
    const long long at = (long long)blockIdx.x * 256 + threadIdx.x, index = at / kQuads;
    if (index >= args.B * args.P * args.H) return;
    const int e = (int)(at % kQuads), row = 4 * e / D, col = 4 * e % D;
    floatx4 x{0.f, 0.f, 0.f, 0.f};
    if (a.state_in) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {                 // row: of the pass's columns; col: of its rows
            const int at_k = a.state_t ? row : col + i, at_v = a.state_t ? col + i : row;
            if (at_k < args.dk && at_v < args.dv) x[i] = a.state_in[(index * args.dk + at_k) * args.dv + at_v];
        }
    }
    const float whole = decay_of(args.log_decay[index % args.H], args.seg_chunks * chunk);
    floatx4* s = (floatx4*)a.seg_state + index * args.n_seg * kQuads + e;
    s[0] = x;
#pragma unroll 8
    for (int k = 1; k < args.n_seg; ++k) {
        x = x * whole + s[(long long)k * kQuads];
        s[(long long)k * kQuads] = x;
    }
}

// Sum over the output heads that share a head: float32 [B][T][P][H][d] to x.  A thread has N neighbouring elements.
template <class T, int N>
__global__ __launch_bounds__(256) void mix_share_kernel(const float* __restrict__ part, MixTensor x, void* out, unsigned T_, unsigned P, unsigned H,
                                                        long long n) {
    const long long at = group_of_grid() * 256 + threadIdx.x;
    if (at >= n) return;
    const unsigned per = x.d / N, heads = H / x.share;
    const long long row = at / (per * heads);         // (b T + t) P + p
    const unsigned in = (unsigned)(at - row * (per * heads)), h = in / per, c = (in - h * per) * N;
    const long long bt = P == 1 ? row : row / P, b = bt / T_;
    const float* src = part + (row * H + (long long)h * x.share) * x.d + c;
    float s[N], v[N];
    __builtin_memcpy(s, src, sizeof(s));
    for (int k = 1; k < x.share; ++k) {
        __builtin_memcpy(v, src + (long long)k * x.d, sizeof(v));
#pragma unroll
        for (int i = 0; i < N; ++i) s[i] += v[i];
    }
    T* dst = (T*)out + b * x.s.b + (bt - b * T_) * x.s.t + (row - bt * P) * x.s.p + h * x.s.h + c;
    if constexpr (N == 1) put_f32(dst, s[0]);
    else store_part<T, N>(dst, N, s);
}

// One token: S' = e^a S + k v^T, o = scale q S'.  Bound by the state, read once and written once.  TP threads have a problem, a workgroup
// or (states of up to 8 KB) a wave; a thread has four columns of dv and every R-th row of dk, kStepRows of them on their way at a time, the
// first before it waits for q, k and v.  64 sequences x 16 heads of 128 x 128: 33 us, 4.1 TB/s.  40000 pixels x 4 heads of 16 x 16: 413 us
// with a workgroup each, 137 with a wave each.
constexpr int kStepThreads = 256, kStepRows = 8;
template <class T, int TP>
__global__ __launch_bounds__(kStepThreads) void mix_step_kernel(MixArgs args) {
    constexpr int kSlots = kStepThreads / TP, kWaves = TP / 64;
    const MixRole& a = args.role[0];
    __shared__ float lds_q[kSlots][128], lds_k[kSlots][128];
    __shared__ floatx4 red[kWaves][64];
    const int slot = kSlots == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / TP), tid = threadIdx.x % TP;
    const long long index = group_of_grid() * kSlots + slot;
    if (index >= args.B * args.P * args.H) return;    // a wave each: no barriers
    const Problem r = problem_of(args, index);
    const T *gq = base_of<T>(a.q, r), *gk = base_of<T>(a.k, r), *gv = base_of<T>(a.v, r);
    const int dk = a.k.d, dv = a.v.d;
    float *sq = lds_q[slot], *sk = lds_k[slot];
    const bool live = r.len > 0;
    const int quads = (dv + 3) / 4, log_w = quads <= 1 ? 0 : 32 - __clz(quads - 1), row0 = tid >> log_w, rows = TP >> log_w;
    const int c = 4 * (tid & ((1 << log_w) - 1)), width = dv - c < 4 ? dv - c : 4;   // columns that exist, none or fewer: <= 0
    const long long base = r.index * dk * dv + c;
    const float* in = a.state_in ? a.state_in + base : nullptr;
    floatx4 s[kStepRows];
    auto fetch = [&](int first) {
#pragma unroll
        for (int k = 0; k < kStepRows; ++k) {
            const int row = first + k * rows;
            s[k] = floatx4{0.f, 0.f, 0.f, 0.f};
            if (!in || row >= dk) continue;
            if (width == 4) {
                __builtin_memcpy(&s[k], in + row * dv, 16);
            } else {
#pragma unroll
                for (int i = 0; i < 3; ++i)
                    if (i < width) s[k][i] = in[row * dv + i];
            }
        }
    };
    fetch(row0);
    for (int i = tid; i < dk; i += TP) {
        sq[i] = live ? to_f32(gq[i]) : 0.f;
        sk[i] = live ? to_f32(gk[i]) : 0.f;
    }
    floatx4 v{0.f, 0.f, 0.f, 0.f}, o{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < width && live) v[i] = to_f32(gv[c + i]);
    const float whole = live ? decay_of(args.log_decay[r.h], 1) : 1.f;
    exchange<kWaves>();
    for (int first = row0; first < dk; first += kStepRows * rows) {
        if (first != row0) fetch(first);
#pragma unroll
        for (int k = 0; k < kStepRows; ++k) {
            const int row = first + k * rows;
            if (row >= dk) break;
            s[k] = s[k] * whole + v * sk[row];
            o += s[k] * sq[row];
            if (!a.state_out) continue;
            float* out = a.state_out + base + row * dv;
            if (width == 4) {
                __builtin_memcpy(out, &s[k], 16);
            } else {
#pragma unroll
                for (int i = 0; i < 3; ++i)
                    if (i < width) out[i] = s[k][i];
            }
        }
    }
    // the sum over the rows: across the lanes of a column quad, then the waves
    for (int off = 1 << log_w; off < 64; off *= 2)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] += __shfl_xor(o[i], off);
    if constexpr (kWaves > 1) {
        red[tid >> 6][tid & 63] = o;
        __syncthreads();
#pragma unroll
        for (int w = 1; w < kWaves; ++w) o += red[w][tid & 63];
    }
    if (tid < 1 << log_w) {                           // wave 0 has its own sums and those of the others
        T* out = (T*)a.out + r.b * a.o.s.b + r.p * a.o.s.p + r.h * a.o.s.h + c;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < width) put_f32(out + i, live ? o[i] * a.out_scale : 0.f);
    }
}

// ------------------------------------------------------------------ host
inline size_t align_up(size_t v) { return (v + 255) / 256 * 256; }
int width_of(int dk, int dv) {
    const int d = dk > dv ? dk : dv;
    return d <= 32 ? 32 : d <= 64 ? 64 : d <= 96 ? 96 : 128;
}
// Segments of a call of `roles` passes, where there are few problems: as many workgroups as run at once (256 compute units hold two of
// them each, four at a width of 64), of two chunks at least.  Against twice as many where they have eight chunks each all the same:
// 16384 tokens, 16 heads of 128, bfloat16 gradients 259 and 274 us (322 and 326 with 4 heads of keys and values), 50000 of them forward 305 and
// 337, 100000 tokens, 4 heads of 32, gradients 90 and 105, 8192 x 4, 8 heads of 96, gradients 255 and 264; float32 the same within 1 %.
// Against half as many: 431 us for the 322, 459 for the 255, and 3 x 1001 tokens, 6 heads of 40 and 72, float32, gradients 82 for 65.
struct Split {
    int n_seg, chunks;
};
Split split_of(const gleam_linattn_desc& d, int roles) {
    const int D = width_of(d.dk, d.dv), L = d.dtype && D > 32 ? 64 : 32;
    const long long problems = d.B * d.P * d.heads, groups = D == 32 ? (problems + 3) / 4 : problems, chunks = (d.T + L - 1) / L;
    long long n = (D == 64 ? 1024 : 512) / (groups * roles);
    if (n > chunks / 2) n = chunks / 2;
    if (n < 2) return {1, (int)chunks};
    const long long per = (chunks + n - 1) / n;
    return {(int)((chunks + per - 1) / per), (int)per};
}
size_t seg_bytes(const gleam_linattn_desc& d, int roles) {
    const Split s = split_of(d, roles);
    const size_t D = width_of(d.dk, d.dv);
    return s.n_seg < 2 ? 0 : align_up((size_t)(d.B * d.P * d.heads) * s.n_seg * D * D * sizeof(float));
}
// float32 gradients of all output heads of an array whose heads are shared
size_t share_bytes(const gleam_linattn_desc& d, int heads, int width) {
    return heads == d.heads ? 0 : align_up((size_t)(d.B * d.T * d.P * d.heads) * width * sizeof(float));
}

// Workgroups of a launch: the ranges of the 8 XCDs are of one length.
dim3 blocks_of(unsigned groups, unsigned segs, unsigned roles) { return grid_of((groups * segs * roles + 7) / 8 * 8); }

// `roles` passes side by side; `states` of them first, over segments, where there are several.
template <class T, int D, int PARTS, bool NARROW>
hipError_t mix_passes(MixArgs a, int roles, MixArgs states, int n_states, const char* name, hipStream_t st) {
    typedef Shape<T, D> S;
    const long long problems = a.B * a.P * a.H;
    const unsigned groups = (unsigned)((problems + S::kProblems - 1) / S::kProblems);
    a.groups = states.groups = groups;
    a.roles = roles;
    states.roles = n_states;
    // workgroups that share keys or values stand next to each other
    int share = 1;
    for (int i = 0; i < roles; ++i) share = share > a.role[i].k.share ? share : a.role[i].k.share;
    a.near_groups = states.near_groups = S::kProblems == 1 && groups % share == 0 ? share : 1;
    const double tokens = (double)problems * a.T, flops = 2.0 * tokens * a.dk * a.dv, bytes = tokens * sizeof(T) * (a.dk + a.dv);
    if (a.n_seg > 1) {
        {
            KernelScope ks("linattn_segments", n_states * flops, n_states * bytes, st);
            hipLaunchKernelGGL((mix_kernel<T, D, true, PARTS, NARROW>), blocks_of(groups, a.n_seg - 1, n_states), dim3(S::kThreads), 0, st, states);
        }
        const double floats = (double)n_states * problems * a.n_seg * S::kStateFloats;
        KernelScope ks("linattn_scan", 2.0 * floats, 8.0 * floats, st);
        const unsigned blocks = (unsigned)((problems * (S::kStateFloats / 4) + 255) / 256);
        hipLaunchKernelGGL(mix_scan_kernel<D>, dim3(blocks, 1, n_states), dim3(256), 0, st, states, S::kL);
    }
    KernelScope ks(name, roles * 2.0 * flops, roles * 2.0 * bytes, st);
    hipLaunchKernelGGL((mix_kernel<T, D, false, PARTS, NARROW>), blocks_of(groups, a.n_seg, roles), dim3(S::kThreads), 0, st, a);
    return hipGetLastError();
}
template <class T, int D>
hipError_t mix_parts(const MixArgs& a, int roles, const MixArgs& states, int n_states, bool state_out, const char* name, hipStream_t st) {
    constexpr int kMost = sizeof(T) == 4 ? 1 : 3;
    const int vec = 16 / (int)sizeof(T);
    bool narrow = a.dk < vec || a.dv < vec;
    for (int i = 0; i < roles; ++i)
        for (const MixTensor* x : {&a.role[i].q, &a.role[i].k, &a.role[i].v}) narrow = narrow || x->s.t > kFarBytes / (long long)sizeof(T);
    if (narrow) return mix_passes<T, D, kMost, true>(a, roles, states, n_states, name, st);
    if (state_out) return mix_passes<T, D, kMost, false>(a, roles, states, n_states, name, st);
    return mix_passes<T, D, (kMost < 2 ? kMost : 2), false>(a, roles, states, n_states, name, st);
}
template <class T>
hipError_t mix_any(const MixArgs& a, int roles, const MixArgs& states, int n_states, bool state_out, const char* name, hipStream_t st) {
    switch (width_of(a.dk, a.dv)) {
        case 32: return mix_parts<T, 32>(a, roles, states, n_states, state_out, name, st);
        case 64: return mix_parts<T, 64>(a, roles, states, n_states, state_out, name, st);
        case 96: return mix_parts<T, 96>(a, roles, states, n_states, state_out, name, st);
        default: return mix_parts<T, 128>(a, roles, states, n_states, state_out, name, st);
    }
}

// Rule for the kernel of short sequences.  It reads and writes every array once, in the backward pass as well, and a problem is one wave;
// it has no state, and beyond these sizes the operands do not fit its registers.
bool is_short(const gleam_linattn_desc& d, bool state) { return !state && d.T <= kShortTokens && d.dk <= kShortWidth && d.dv <= kShortWidth; }
// Whether four neighbouring heads lie side by side in an array, in whole 16 bytes (so that they are aligned in LDS), and tokens no further
// apart than the kernel's 24-bit products allow.
bool side_by_side(const MixTensor& x, int elements16) { return x.share == 1 && x.s.h == x.d && x.d % elements16 == 0 && x.s.t < 1 << 24; }
template <class T, int TT, int U, bool BWD>
void launch_short(const MixArgs& a, unsigned groups, hipStream_t st) {
    const int e = 16 / (int)sizeof(T);
    const MixRole& r = a.role[BWD ? 2 : 0];           // q and k in any case
    bool whole = a.H % kShortWaves == 0 && side_by_side(r.q, e) && side_by_side(r.k, e) && side_by_side(a.role[0].k, e) && side_by_side(r.v, e);
    for (int i = 0; i < (BWD ? 3 : 1); ++i) whole = whole && !a.role[i].out_f32 && side_by_side(a.role[i].o, e);
    if (whole) hipLaunchKernelGGL((mix_short_kernel<T, TT, U, BWD, true>), grid_of(groups), dim3(64 * kShortWaves), 0, st, a);
    else hipLaunchKernelGGL((mix_short_kernel<T, TT, U, BWD, false>), grid_of(groups), dim3(64 * kShortWaves), 0, st, a);
}
template <class T, int TT, bool BWD>
void launch_short(const MixArgs& a, unsigned groups, hipStream_t st) {
    if (a.dk <= 16 && a.dv <= 16) launch_short<T, TT, 1, BWD>(a, groups, st);
    else launch_short<T, TT, 2, BWD>(a, groups, st);
}
template <class T, bool BWD>
hipError_t mix_short(const MixArgs& a, const char* name, hipStream_t st) {
    const long long problems = a.B * a.P * a.H;
    const unsigned groups = (unsigned)((problems + kShortWaves - 1) / kShortWaves);
    const double tokens = (double)problems * a.T;
    KernelScope ks(name, (BWD ? 10.0 : 4.0) * tokens * a.dk * a.dv, (BWD ? 3.5 : 2.0) * tokens * sizeof(T) * (a.dk + a.dv), st);
    if (a.T <= 16) launch_short<T, 1, BWD>(a, groups, st);
    else if (a.T <= 32) launch_short<T, 2, BWD>(a, groups, st);
    else launch_short<T, 4, BWD>(a, groups, st);
    return hipGetLastError();
}

template <class T, int N>
hipError_t share_sum(const gleam_linattn_desc& d, const float* part, const MixTensor& x, void* out, long long n, hipStream_t st) {
    hipLaunchKernelGGL((mix_share_kernel<T, N>), grid_of((n / N + 255) / 256), dim3(256), 0, st, part, x, out, (unsigned)d.T, (unsigned)d.P,
                       (unsigned)d.heads, n / N);
    return hipGetLastError();
}

template <class T>
hipError_t mix_step(const MixArgs& a, hipStream_t st) {
    const long long problems = a.B * a.P * a.H;
    // the whole state is on its way to a wave at once, or in two turns where the columns' fours are not a power of two
    if (a.dk * ((a.dv + 3) / 4) <= 64 * kStepRows)
        hipLaunchKernelGGL((mix_step_kernel<T, 64>), grid_of((problems + 3) / 4), dim3(kStepThreads), 0, st, a);
    else
        hipLaunchKernelGGL((mix_step_kernel<T, kStepThreads>), grid_of(problems), dim3(kStepThreads), 0, st, a);
    return hipGetLastError();
}

gleam_seq_strides row_major(const gleam_linattn_desc& d, int heads, int width) {
    return {d.T * d.P * heads * width, d.P * heads * width, (int64_t)heads * width, width};
}
MixArgs common(const gleam_linattn_desc& d, int roles, const float* log_decay, const int* lengths) {
    MixArgs a{};
    a.B = d.B;
    a.P = d.P;
    a.T = d.T;
    a.H = d.heads;
    a.dk = d.dk;
    a.dv = d.dv;
    a.log_decay = log_decay;
    a.lengths = lengths;
    const Split s = split_of(d, roles);
    a.n_seg = s.n_seg;
    a.seg_chunks = s.chunks;
    return a;
}
MixRole role_of(const MixTensor& q, const MixTensor& k, const MixTensor& v, int state_t, int reverse, float in_scale, float out_scale,
                const float* state_in, float* seg_state) {
    MixRole r{};
    r.q = q;
    r.k = k;
    r.v = v;
    r.state_t = state_t;
    r.reverse = reverse;
    r.in_scale = in_scale;
    r.out_scale = out_scale;
    r.state_in = state_in;
    r.seg_state = seg_state;
    return r;
}

}  // namespace

size_t linattn_fwd_ws_bytes(const gleam_linattn_desc& d) { return d.T == 1 ? 0 : seg_bytes(d, 1); }
size_t linattn_bwd_ws_bytes(const gleam_linattn_desc& d) {
    return 2 * seg_bytes(d, 3) + share_bytes(d, d.q_heads, d.dk) + share_bytes(d, d.k_heads, d.dk) + share_bytes(d, d.v_heads, d.dv);
}

hipError_t linattn_forward(const gleam_linattn_desc& d, const void* q, const void* k, const void* v, const float* log_decay,
                           const int* lengths, const float* state_in, void* o, float* state_out, void* ws, hipStream_t st) {
    const MixTensor tq = {q, d.q, d.heads / d.q_heads, d.dk}, tk = {k, d.k, d.heads / d.k_heads, d.dk}, tv = {v, d.v, d.heads / d.v_heads, d.dv};
    MixArgs a = common(d, 1, log_decay, lengths), states = a;
    float* seg = a.n_seg > 1 ? (float*)ws : nullptr;
    a.role[0] = role_of(tq, tk, tv, 0, 0, 1.f, d.scale, state_in, seg);
    a.role[0].o = {nullptr, d.o, 1, d.dv};
    a.role[0].out = o;
    a.role[0].state_out = state_out;
    if (d.T == 1) {
        const double floats = (double)d.B * d.P * d.heads * d.dk * d.dv;
        KernelScope ks("linattn_step", 4.0 * floats, 8.0 * floats, st);
        return d.dtype ? mix_step<unsigned short>(a, st) : mix_step<float>(a, st);
    }
    if (is_short(d, state_in || state_out))
        return d.dtype ? mix_short<unsigned short, false>(a, "linattn_fwd_short", st) : mix_short<float, false>(a, "linattn_fwd_short", st);
    states.role[0] = role_of(tq, tk, tv, 0, 0, 1.f, 1.f, state_in, seg);
    return d.dtype ? mix_any<unsigned short>(a, 1, states, 1, state_out, "linattn_fwd", st)
                   : mix_any<float>(a, 1, states, 1, state_out, "linattn_fwd", st);
}

hipError_t linattn_backward(const gleam_linattn_desc& d, const void* q, const void* k, const void* v, const float* log_decay,
                            const int* lengths, const float* state_in, const void* g_o, const float* g_state_out, void* g_q, void* g_k,
                            void* g_v, float* g_state_in, void* ws, hipStream_t st) {
    const MixTensor tq = {q, d.q, d.heads / d.q_heads, d.dk}, tk = {k, d.k, d.heads / d.k_heads, d.dk}, tv = {v, d.v, d.heads / d.v_heads, d.dv};
    const MixTensor tg = {g_o, d.o, 1, d.dv};
    MixArgs a = common(d, 3, log_decay, lengths), states = a;
    unsigned char* at = (unsigned char*)ws;
    float* seg_s = a.n_seg > 1 ? (float*)at : nullptr;               // states of the forward pass
    at += seg_bytes(d, 3);
    float* seg_g = a.n_seg > 1 ? (float*)at : nullptr;               // their gradients
    at += seg_bytes(d, 3);
    a.role[0] = role_of(tg, tv, tk, 1, 0, 1.f, d.scale, state_in, seg_s);
    a.role[1] = role_of(tv, tg, tq, 1, 1, d.scale, 1.f, g_state_out, seg_g);
    a.role[2] = role_of(tk, tq, tg, 0, 1, d.scale, 1.f, g_state_out, seg_g);
    a.role[2].state_out = g_state_in;
    a.role[2].seg_t = 1;
    states.role[0] = role_of(tg, tv, tk, 1, 0, 1.f, 1.f, state_in, seg_s);
    states.role[1] = role_of(tv, tg, tq, 1, 1, d.scale, 1.f, g_state_out, seg_g);
    const MixTensor* of[3] = {&tq, &tk, &tv};
    void* out[3] = {g_q, g_k, g_v};
    float* part[3] = {};
    for (int i = 0; i < 3; ++i) {
        const MixTensor& x = *of[i];
        a.role[i].o = x;
        a.role[i].out = out[i];
        if (x.share > 1) {                                           // by way of a float32 array of all output heads
            part[i] = (float*)at;
            at += share_bytes(d, d.heads / x.share, x.d);
            a.role[i].o = {nullptr, row_major(d, d.heads, x.d), 1, x.d};
            a.role[i].out = part[i];
            a.role[i].out_f32 = 1;
        }
    }
    hipError_t e;
    if (is_short(d, state_in || g_state_out || g_state_in))
        e = d.dtype ? mix_short<unsigned short, true>(a, "linattn_bwd_short", st) : mix_short<float, true>(a, "linattn_bwd_short", st);
    else
        e = d.dtype ? mix_any<unsigned short>(a, 3, states, 2, g_state_in, "linattn_bwd", st)
                    : mix_any<float>(a, 3, states, 2, g_state_in, "linattn_bwd", st);
    for (int i = 0; i < 3 && e == hipSuccess; ++i) {
        if (!part[i]) continue;
        const MixTensor& x = *of[i];
        const long long n = d.B * d.T * d.P * (d.heads / x.share) * x.d;
        KernelScope ks("linattn_share", (double)n * x.share, 4.0 * n * x.share + (d.dtype ? 2.0 : 4.0) * n, st);
        e = x.d % 4 ? (d.dtype ? share_sum<unsigned short, 1>(d, part[i], x, out[i], n, st) : share_sum<float, 1>(d, part[i], x, out[i], n, st))
                    : (d.dtype ? share_sum<unsigned short, 4>(d, part[i], x, out[i], n, st) : share_sum<float, 4>(d, part[i], x, out[i], n, st));
    }
    return e;
}

}  // namespace gleam
