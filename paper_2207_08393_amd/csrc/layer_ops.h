// Internal declarations of the sequence-layer operators: layer norm, dropout, linear attention with a decay for each head, norm and
// rotation of queries and keys, the gated scan, and the orthogonalised update of weight matrices.
#pragma once
#include "internal.h"

namespace gleam {

// ------------------------------------------------------------------ layer norm (norm.hip)
hipError_t layer_norm_forward(const gleam_layer_norm_desc& d, const void* x, const float* gamma, const float* beta, void* y, float* mean,
                              float* rstd, hipStream_t st);
size_t layer_norm_ws_bytes(const gleam_layer_norm_desc& d);
hipError_t layer_norm_backward(const gleam_layer_norm_desc& d, const void* x, const float* gamma, const float* mean, const float* rstd,
                               const void* g_y, void* g_x, float* g_gamma, float* g_beta, void* ws, hipStream_t st);

// ------------------------------------------------------------------ dropout (dropout.hip)
// out = residual + dropout(x); residual may be null.  Row strides of the three arrays in elements.
struct DropoutArgs {
    const void *x, *res;
    void* out;
    long long rows, n, ld_x, ld_res, ld_out;
    unsigned long long seed, offset;
    const unsigned long long* step;
    unsigned kept;      // of 65536 draws
    float scale;
    int dtype;
};
hipError_t dropout(const DropoutArgs& a, hipStream_t st);

// ------------------------------------------------------------------ linear attention (linattn.hip)
// Elements of an activation: base + b*s.b + t*s.t + p*s.p + (h / share)*s.h + c, in elements.
struct MixTensor {
    const void* p;
    gleam_seq_strides s;
    int share;          // output heads that use one head of this tensor
    int d;              // width of a head
};
// One pass over all problems, see linattn.hip; a launch runs up to three of them side by side.
struct MixRole {
    MixTensor q, k, v, o;
    void* out;
    int out_f32;                        // the output is float32 whatever the type of q, k, v
    int state_t;                        // this pass has the roles of dk and dv exchanged
    int reverse;                        // tokens from a sequence's end to its start
    float in_scale, out_scale;          // on k (x) v, and on what a query reads
    const float* state_in;              // natural layout [B][P][H][dk][dv] of the layer, or null: zero
    float* state_out;                   // or null
    float* seg_state;                   // [problem][segment][D][D]: states at the segments' starts, or null for one segment
    int seg_t;                          // they come from a pass with the roles of dk and dv exchanged against this one's
};
struct MixArgs {
    MixRole role[3];
    long long B, P, T;
    int H, dk, dv;
    const float* log_decay;             // [H]
    const int* lengths;                 // [B] or null
    int n_seg, seg_chunks;
    unsigned groups, roles, near_groups;   // of a launch: workgroups of problems, passes, groups that stand next to each other
};
size_t linattn_fwd_ws_bytes(const gleam_linattn_desc& d);
size_t linattn_bwd_ws_bytes(const gleam_linattn_desc& d);
hipError_t linattn_forward(const gleam_linattn_desc& d, const void* q, const void* k, const void* v, const float* log_decay,
                           const int* lengths, const float* state_in, void* o, float* state_out, void* ws, hipStream_t st);
hipError_t linattn_backward(const gleam_linattn_desc& d, const void* q, const void* k, const void* v, const float* log_decay,
                            const int* lengths, const float* state_in, const void* g_o, const float* g_state_out, void* g_q, void* g_k,
                            void* g_v, float* g_state_in, void* ws, hipStream_t st);

// ------------------------------------------------------------------ norm and rotation of queries and keys (qknorm.hip)
hipError_t qknorm_forward(const gleam_qknorm_desc& d, const void* q, const void* k, const float* gamma_q, const float* gamma_k,
                          const float* freq, const int* positions, const int* lengths, void* q_out, void* k_out, hipStream_t st);
size_t qknorm_ws_bytes(const gleam_qknorm_desc& d);
hipError_t qknorm_backward(const gleam_qknorm_desc& d, const void* q, const void* k, const float* gamma_q, const float* gamma_k,
                           const float* freq, const int* positions, const int* lengths, const void* g_q_out, const void* g_k_out, void* g_q,
                           void* g_k, float* g_gamma_q, float* g_gamma_k, void* ws, hipStream_t st);

// ------------------------------------------------------------------ gated scan (gatedscan.hip)
size_t gatedscan_fwd_ws_bytes(const gleam_gatedscan_desc& d);
size_t gatedscan_bwd_ws_bytes(const gleam_gatedscan_desc& d);
hipError_t gatedscan_forward(const gleam_gatedscan_desc& d, const void* x, const void* r, const void* i, const float* lambda,
                             const int* lengths, const float* state_in, void* h, float* state_out, void* ws, hipStream_t st);
hipError_t gatedscan_backward(const gleam_gatedscan_desc& d, const void* x, const void* r, const void* i, const float* lambda,
                              const int* lengths, const float* state_in, const void* g_h, const float* g_state_out, void* g_x, void* g_r,
                              void* g_i, float* g_lambda, float* g_state_in, void* ws, hipStream_t st);

// ------------------------------------------------------------------ orthogonalised update (muon.hip)
// Whether X, A = X X^T and the polynomial B of it stay in the range that they may reach.
bool muon_scales(const gleam_muon& p);
size_t muon_ws_bytes(long long count, long long rows, long long cols);
hipError_t muon_update(const gleam_muon& p, long long count, long long rows, long long cols, long long stride, float* theta,
                       const float* grad, float* m, void* ws, hipStream_t st);

}  // namespace gleam
