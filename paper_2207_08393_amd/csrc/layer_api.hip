// C ABI of the sequence-layer operators: host-side validation, then the kernels of norm.hip, dropout.hip, linattn.hip, qknorm.hip,
// gatedscan.hip and muon.hip on the caller's stream.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "layer_ops.h"

using namespace gleam;

namespace {

constexpr long long kMostElements = 1LL << 40;   // keeps every byte offset far inside int64

constexpr long long kMostProblems = 1LL << 29;   // sequences x pixels x heads: the numbers of three workgroups for each fit 32 bits

inline bool aligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) % 256) == 0; }

// a * b, or -1 beyond kMostElements; both at least 1
long long product(long long a, long long b) { return a > 0 && b > 0 && a <= kMostElements / b ? a * b : -1; }

int check_rows(int dtype, long long rows, long long n, std::initializer_list<int64_t> strides) {
    if (dtype != 0 && dtype != 1) return GLEAM_E_DESC;
    if (rows < 1 || n < 1 || rows > 0x7fffffffLL || product(rows, n) < 0) return GLEAM_E_DIMS;
    for (int64_t ld : strides)
        if (ld < n || product(rows, ld) < 0) return GLEAM_E_DIMS;
    return GLEAM_OK;
}

int check_norm(const gleam_layer_norm_desc* d) {
    if (!d) return GLEAM_E_NULL;
    const int rc = check_rows(d->dtype, d->rows, d->n, {d->ld_in, d->ld_out});
    if (rc) return rc;
    if (d->n > 0x7fffffffLL) return GLEAM_E_DIMS;
    return d->eps > 0.f && std::isfinite(d->eps) ? GLEAM_OK : GLEAM_E_DESC;
}

int check_dropout(const gleam_dropout_desc* d, bool residual) {
    if (!d) return GLEAM_E_NULL;
    const int rc = check_rows(d->dtype, d->rows, d->n, {d->ld_in, d->ld_out, residual ? d->ld_res : d->ld_in});
    if (rc) return rc;
    return d->p >= 0.f && d->p <= 1.f ? GLEAM_OK : GLEAM_E_DESC;
}

DropoutArgs dropout_args(const gleam_dropout_desc& d, const uint64_t* step) {
    DropoutArgs a{};
    a.rows = d.rows;
    a.n = d.n;
    a.ld_x = d.ld_in;
    a.ld_res = d.ld_res;
    a.ld_out = d.ld_out;
    a.seed = d.seed;
    a.offset = d.offset;
    a.step = (const unsigned long long*)step;
    a.kept = (unsigned)std::floor(65536.0 * (1.0 - (double)d.p) + 0.5);
    a.scale = a.kept ? (float)(65536.0 / a.kept) : 0.f;
    a.dtype = d.dtype;
    return a;
}

// An array [B][T][P][heads][width]: strides that reach no further than they may, and that keep elements apart where it is written.
int check_strides(long long B, long long T, long long P, const gleam_seq_strides& s, long long heads, long long width, bool written) {
    struct Axis {
        long long n, stride;
    } axis[4] = {{B, s.b}, {T, s.t}, {P, s.p}, {heads, s.h}};
    long long reach = width;
    for (const Axis& x : axis) {
        if (x.stride < 0 || x.stride > kMostElements) return GLEAM_E_DIMS;
        if (x.n > 1 && x.stride > 0 && product(x.n - 1, x.stride) < 0) return GLEAM_E_DIMS;
        if (x.n > 1) reach += (x.n - 1) * x.stride;
    }
    if (reach > kMostElements) return GLEAM_E_DIMS;
    if (!written) return GLEAM_OK;
    std::sort(axis, axis + 4, [](const Axis& x, const Axis& y) { return x.stride < y.stride; });
    long long covered = width;   // elements from the first to the last of the axes so far
    for (const Axis& x : axis) {
        if (x.n == 1) continue;
        if (x.stride < covered) return GLEAM_E_DIMS;
        covered += (x.n - 1) * x.stride;
    }
    return GLEAM_OK;
}

int check_linattn(const gleam_linattn_desc* d, bool gradients) {
    if (!d) return GLEAM_E_NULL;
    if (d->dtype != 0 && d->dtype != 1) return GLEAM_E_DESC;
    if (!std::isfinite(d->scale)) return GLEAM_E_DESC;
    if (d->dk < 1 || d->dk > 128 || d->dv < 1 || d->dv > 128) return GLEAM_E_DIMS;
    for (int h : {d->q_heads, d->k_heads, d->v_heads})
        if (h < 1 || d->heads < h || d->heads % h) return GLEAM_E_DIMS;
    if (d->B < 1 || d->T < 1 || d->P < 1 || d->T > (1 << 30)) return GLEAM_E_DIMS;
    const long long problems = product(product(d->B, d->P), d->heads);
    if (problems < 0 || problems > kMostProblems || product(problems, d->T) < 0) return GLEAM_E_DIMS;
    if (product(problems * d->T, std::max(d->dk, d->dv)) < 0 || product(problems, d->dk * d->dv) < 0) return GLEAM_E_DIMS;
    int rc = check_strides(d->B, d->T, d->P, d->q, d->q_heads, d->dk, gradients);
    if (!rc) rc = check_strides(d->B, d->T, d->P, d->k, d->k_heads, d->dk, gradients);
    if (!rc) rc = check_strides(d->B, d->T, d->P, d->v, d->v_heads, d->dv, gradients);
    if (!rc) rc = check_strides(d->B, d->T, d->P, d->o, d->heads, d->dv, !gradients);
    return rc;
}

bool same(const gleam_seq_strides& a, const gleam_seq_strides& b) { return a.b == b.b && a.t == b.t && a.p == b.p && a.h == b.h; }

int check_qknorm(const gleam_qknorm_desc* d, bool gradients) {
    if (!d) return GLEAM_E_NULL;
    if (d->dtype != 0 && d->dtype != 1) return GLEAM_E_DESC;
    if ((d->pairs != 0 && d->pairs != 1) || (d->each != 0 && d->each != 1)) return GLEAM_E_DESC;
    if (!(d->eps > 0.f) || !std::isnormal(d->eps)) return GLEAM_E_DESC;
    if (d->d < 1 || d->d > 256 || d->rot < 0 || d->rot > d->d || d->rot % 2) return GLEAM_E_DIMS;
    if (d->q_heads < 1 || d->k_heads < 0 || d->B < 1 || d->T < 1 || d->P < 1 || d->T > (1 << 30)) return GLEAM_E_DIMS;
    const long long heads = (long long)d->q_heads + d->k_heads, tokens = product(d->B, d->T);
    if (product(d->P, heads) < 0 || d->P * heads > 0x7fffffffLL) return GLEAM_E_DIMS;
    if (tokens < 0 || product(tokens, d->P * heads) < 0 || product(tokens * d->P * heads, d->d) < 0) return GLEAM_E_DIMS;
    int rc = check_strides(d->B, d->T, d->P, d->q, d->q_heads, d->d, gradients);
    if (!rc) rc = check_strides(d->B, d->T, d->P, d->q_out, d->q_heads, d->d, !gradients);
    if (!rc && d->k_heads) rc = check_strides(d->B, d->T, d->P, d->k, d->k_heads, d->d, gradients);
    if (!rc && d->k_heads) rc = check_strides(d->B, d->T, d->P, d->k_out, d->k_heads, d->d, !gradients);
    return rc;
}

int check_gatedscan(const gleam_gatedscan_desc* d, bool gradients) {
    if (!d) return GLEAM_E_NULL;
    if (d->dtype != 0 && d->dtype != 1) return GLEAM_E_DESC;
    if (!(d->kappa >= 0.f) || !std::isfinite(d->kappa)) return GLEAM_E_DESC;
    if (d->B < 1 || d->T < 1 || d->P < 1 || d->C < 1 || d->T > (1 << 30) || d->C > 0x7fffffffLL) return GLEAM_E_DIMS;
    const long long states = product(product(d->B, d->P), d->C);
    if (states < 0 || product(states, d->T) < 0) return GLEAM_E_DIMS;
    auto check = [&](const gleam_scan_strides& s, bool written) {
        return check_strides(d->B, d->T, d->P, gleam_seq_strides{s.b, s.t, s.p, d->C}, 1, d->C, written);
    };
    int rc = check(d->x, gradients);
    if (!rc) rc = check(d->r, gradients);
    if (!rc) rc = check(d->i, gradients);
    if (!rc) rc = check(d->h, !gradients);
    return rc;
}

int check_muon_sizes(long long count, long long rows, long long cols) {
    if (count < 1 || rows < 1 || cols < 1 || count > (1 << 20) || rows > 65536 || cols > 65536) return GLEAM_E_DIMS;
    return product(product(rows, cols), count) < 0 ? GLEAM_E_DIMS : GLEAM_OK;
}

int check_muon(const gleam_muon* p) {
    if (!p) return GLEAM_E_NULL;
    for (float v : {p->lr, p->momentum, p->weight_decay, p->eps, p->a, p->b, p->c})
        if (!std::isfinite(v)) return GLEAM_E_DESC;
    if (!(p->eps > 0.f) || p->momentum < 0.f || p->momentum >= 1.f) return GLEAM_E_DESC;
    if (p->steps < 1 || p->steps > 100 || (p->nesterov != 0 && p->nesterov != 1)) return GLEAM_E_DESC;
    return muon_scales(*p) ? GLEAM_OK : GLEAM_E_DESC;
}

int check_ws(const void* ws, size_t ws_bytes, size_t need) {
    if (!need) return GLEAM_OK;
    if (!ws) return GLEAM_E_NULL;
    return aligned(ws) && ws_bytes >= need ? GLEAM_OK : GLEAM_E_WORKSPACE;
}

int status_of(hipError_t e) { return e == hipSuccess ? GLEAM_OK : GLEAM_E_LAUNCH; }

}  // namespace

extern "C" {

int gleam_layer_norm_fwd(const gleam_layer_norm_desc* desc, const void* x, const float* gamma, const float* beta, void* y, float* mean,
                         float* rstd, void* stream) {
    const int rc = check_norm(desc);
    if (rc) return rc;
    if (!x || !y) return GLEAM_E_NULL;
    if (x == y && desc->ld_in != desc->ld_out) return GLEAM_E_DIMS;
    return status_of(layer_norm_forward(*desc, x, gamma, beta, y, mean, rstd, (hipStream_t)stream));
}

int gleam_layer_norm_workspace_bytes(const gleam_layer_norm_desc* desc, size_t* ws_bytes) {
    const int rc = check_norm(desc);
    if (rc) return rc;
    if (!ws_bytes) return GLEAM_E_NULL;
    *ws_bytes = layer_norm_ws_bytes(*desc);
    return GLEAM_OK;
}

int gleam_layer_norm_bwd(const gleam_layer_norm_desc* desc, const void* x, const float* gamma, const float* mean, const float* rstd,
                         const void* g_y, void* g_x, float* g_gamma, float* g_beta, void* ws, size_t ws_bytes, void* stream) {
    int rc = check_norm(desc);
    if (rc) return rc;
    if (!x || !mean || !rstd || !g_y || !g_x) return GLEAM_E_NULL;
    if (g_x == x || (g_x == g_y && desc->ld_in != desc->ld_out)) return GLEAM_E_DIMS;
    rc = check_ws(ws, ws_bytes, g_gamma || g_beta ? layer_norm_ws_bytes(*desc) : 0);
    if (rc) return rc;
    return status_of(layer_norm_backward(*desc, x, gamma, mean, rstd, g_y, g_x, g_gamma, g_beta, ws, (hipStream_t)stream));
}

int gleam_dropout_fwd(const gleam_dropout_desc* desc, const void* x, const void* residual, void* out, const uint64_t* step, void* stream) {
    const int rc = check_dropout(desc, residual != nullptr);
    if (rc) return rc;
    if (!x || !out) return GLEAM_E_NULL;
    if ((out == x && desc->ld_out != desc->ld_in) || (out == residual && desc->ld_out != desc->ld_res)) return GLEAM_E_DIMS;
    DropoutArgs a = dropout_args(*desc, step);
    a.x = x;
    a.res = residual;
    a.out = out;
    return status_of(dropout(a, (hipStream_t)stream));
}

int gleam_dropout_bwd(const gleam_dropout_desc* desc, const void* g_out, void* g_x, const uint64_t* step, void* stream) {
    const int rc = check_dropout(desc, false);
    if (rc) return rc;
    if (!g_out || !g_x) return GLEAM_E_NULL;
    if (g_x == g_out && desc->ld_out != desc->ld_in) return GLEAM_E_DIMS;
    DropoutArgs a = dropout_args(*desc, step);
    a.x = g_out;
    a.ld_x = desc->ld_out;
    a.out = g_x;
    a.ld_out = desc->ld_in;
    return status_of(dropout(a, (hipStream_t)stream));
}

int gleam_linattn_workspace_bytes(const gleam_linattn_desc* desc, size_t* fwd_bytes, size_t* bwd_bytes) {
    if (!fwd_bytes || !bwd_bytes) return GLEAM_E_NULL;
    const int rc = check_linattn(desc, false);
    if (rc) return rc;
    *fwd_bytes = linattn_fwd_ws_bytes(*desc);
    *bwd_bytes = linattn_bwd_ws_bytes(*desc);
    return GLEAM_OK;
}

int gleam_linattn_fwd(const gleam_linattn_desc* desc, const void* q, const void* k, const void* v, const float* log_decay,
                      const int32_t* lengths, const float* state_in, void* o, float* state_out, void* ws, size_t ws_bytes, void* stream) {
    int rc = check_linattn(desc, false);
    if (rc) return rc;
    if (!q || !k || !v || !log_decay || !o) return GLEAM_E_NULL;
    if (o == q || o == k || o == v) return GLEAM_E_DIMS;
    rc = check_ws(ws, ws_bytes, linattn_fwd_ws_bytes(*desc));
    if (rc) return rc;
    return status_of(linattn_forward(*desc, q, k, v, log_decay, lengths, state_in, o, state_out, ws, (hipStream_t)stream));
}

int gleam_linattn_bwd(const gleam_linattn_desc* desc, const void* q, const void* k, const void* v, const float* log_decay,
                      const int32_t* lengths, const float* state_in, const void* g_o, const float* g_state_out, void* g_q, void* g_k,
                      void* g_v, float* g_state_in, void* ws, size_t ws_bytes, void* stream) {
    int rc = check_linattn(desc, true);
    if (rc) return rc;
    if (!q || !k || !v || !log_decay || !g_o || !g_q || !g_k || !g_v) return GLEAM_E_NULL;
    for (const void* g : {g_q, g_k, g_v})
        for (const void* x : {q, k, v, g_o})
            if (g == x) return GLEAM_E_DIMS;
    if (g_q == g_k || g_q == g_v || g_k == g_v) return GLEAM_E_DIMS;
    if (g_state_in && (g_state_in == g_state_out || g_state_in == state_in)) return GLEAM_E_DIMS;   // read and written side by side
    rc = check_ws(ws, ws_bytes, linattn_bwd_ws_bytes(*desc));
    if (rc) return rc;
    return status_of(linattn_backward(*desc, q, k, v, log_decay, lengths, state_in, g_o, g_state_out, g_q, g_k, g_v, g_state_in, ws,
                                      (hipStream_t)stream));
}

int gleam_qknorm_fwd(const gleam_qknorm_desc* desc, const void* q, const void* k, const float* gamma_q, const float* gamma_k,
                     const float* freq, const int32_t* positions, const int32_t* lengths, void* q_out, void* k_out, void* stream) {
    const int rc = check_qknorm(desc, false);
    if (rc) return rc;
    const bool with_k = desc->k_heads > 0;
    if (!q || !q_out || (with_k && (!k || !k_out)) || (desc->rot && !freq)) return GLEAM_E_NULL;
    if (q_out == q && !same(desc->q, desc->q_out)) return GLEAM_E_DIMS;
    if (with_k && ((k_out == k && !same(desc->k, desc->k_out)) || q_out == k || k_out == q || q_out == k_out)) return GLEAM_E_DIMS;
    return status_of(qknorm_forward(*desc, q, k, gamma_q, gamma_k, freq, positions, lengths, q_out, k_out, (hipStream_t)stream));
}

int gleam_qknorm_workspace_bytes(const gleam_qknorm_desc* desc, size_t* ws_bytes) {
    if (!ws_bytes) return GLEAM_E_NULL;
    const int rc = check_qknorm(desc, true);
    if (rc) return rc;
    *ws_bytes = qknorm_ws_bytes(*desc);
    return GLEAM_OK;
}

int gleam_qknorm_bwd(const gleam_qknorm_desc* desc, const void* q, const void* k, const float* gamma_q, const float* gamma_k,
                     const float* freq, const int32_t* positions, const int32_t* lengths, const void* g_q_out, const void* g_k_out,
                     void* g_q, void* g_k, float* g_gamma_q, float* g_gamma_k, void* ws, size_t ws_bytes, void* stream) {
    int rc = check_qknorm(desc, true);
    if (rc) return rc;
    const bool with_k = desc->k_heads > 0;
    if (!q || !g_q_out || !g_q || (with_k && (!k || !g_k_out || !g_k)) || (desc->rot && !freq)) return GLEAM_E_NULL;
    if (g_q == q || (g_q == g_q_out && !same(desc->q, desc->q_out))) return GLEAM_E_DIMS;
    if (with_k && (g_k == k || g_k == q || g_q == k || g_q == g_k || g_q == g_k_out || g_k == g_q_out || (g_k == g_k_out && !same(desc->k, desc->k_out))))
        return GLEAM_E_DIMS;
    if (!with_k) g_gamma_k = nullptr;
    if (g_gamma_q && g_gamma_q == g_gamma_k) return GLEAM_E_DIMS;
    rc = check_ws(ws, ws_bytes, g_gamma_q || g_gamma_k ? qknorm_ws_bytes(*desc) : 0);
    if (rc) return rc;
    return status_of(qknorm_backward(*desc, q, k, gamma_q, gamma_k, freq, positions, lengths, g_q_out, g_k_out, g_q, g_k, g_gamma_q,
                                     g_gamma_k, ws, (hipStream_t)stream));
}

int gleam_gatedscan_workspace_bytes(const gleam_gatedscan_desc* desc, size_t* fwd_bytes, size_t* bwd_bytes) {
    if (!fwd_bytes || !bwd_bytes) return GLEAM_E_NULL;
    int rc = check_gatedscan(desc, false);
    if (rc == GLEAM_E_DIMS) rc = check_gatedscan(desc, true);   // g_h may repeat, where h may not
    if (rc) return rc;
    *fwd_bytes = gatedscan_fwd_ws_bytes(*desc);
    *bwd_bytes = gatedscan_bwd_ws_bytes(*desc);
    return GLEAM_OK;
}

int gleam_gatedscan_fwd(const gleam_gatedscan_desc* desc, const void* x, const void* r, const void* i, const float* lambda,
                        const int32_t* lengths, const float* state_in, void* h, float* state_out, void* ws, size_t ws_bytes, void* stream) {
    int rc = check_gatedscan(desc, false);
    if (rc) return rc;
    if (!x || !r || !i || !lambda || !h) return GLEAM_E_NULL;
    if (h == x || h == r || h == i) return GLEAM_E_DIMS;
    rc = check_ws(ws, ws_bytes, gatedscan_fwd_ws_bytes(*desc));
    if (rc) return rc;
    return status_of(gatedscan_forward(*desc, x, r, i, lambda, lengths, state_in, h, state_out, ws, (hipStream_t)stream));
}

int gleam_gatedscan_bwd(const gleam_gatedscan_desc* desc, const void* x, const void* r, const void* i, const float* lambda,
                        const int32_t* lengths, const float* state_in, const void* g_h, const float* g_state_out, void* g_x, void* g_r,
                        void* g_i, float* g_lambda, float* g_state_in, void* ws, size_t ws_bytes, void* stream) {
    int rc = check_gatedscan(desc, true);
    if (rc) return rc;
    if (!x || !r || !i || !lambda || !g_h || !g_x || !g_r || !g_i || !g_lambda) return GLEAM_E_NULL;
    for (const void* g : {g_x, g_r, g_i})
        for (const void* a : {x, r, i, g_h})
            if (g == a) return GLEAM_E_DIMS;
    if (g_x == g_r || g_x == g_i || g_r == g_i || g_lambda == lambda) return GLEAM_E_DIMS;
    if (g_state_in && (g_state_in == g_state_out || g_state_in == state_in)) return GLEAM_E_DIMS;
    rc = check_ws(ws, ws_bytes, gatedscan_bwd_ws_bytes(*desc));
    if (rc) return rc;
    return status_of(gatedscan_backward(*desc, x, r, i, lambda, lengths, state_in, g_h, g_state_out, g_x, g_r, g_i, g_lambda, g_state_in,
                                        ws, (hipStream_t)stream));
}

int gleam_muon_workspace_bytes(int64_t count, int64_t rows, int64_t cols, size_t* ws_bytes) {
    if (!ws_bytes) return GLEAM_E_NULL;
    const int rc = check_muon_sizes(count, rows, cols);
    if (rc) return rc;
    *ws_bytes = muon_ws_bytes(count, rows, cols);
    return GLEAM_OK;
}

int gleam_muon_step(const gleam_muon* hyper, int64_t count, int64_t rows, int64_t cols, int64_t stride, float* theta, const float* grad,
                    float* m, void* ws, size_t ws_bytes, void* stream) {
    int rc = check_muon(hyper);
    if (!rc) rc = check_muon_sizes(count, rows, cols);
    if (rc) return rc;
    if (stride < 0 || (count > 1 && (stride < rows * cols || product(count, stride) < 0))) return GLEAM_E_DIMS;
    if (!theta || !grad || !m) return GLEAM_E_NULL;
    if (theta == grad || theta == m || grad == m) return GLEAM_E_DIMS;
    rc = check_ws(ws, ws_bytes, muon_ws_bytes(count, rows, cols));
    if (rc) return rc;
    return status_of(muon_update(*hyper, count, rows, cols, stride, theta, grad, m, ws, (hipStream_t)stream));
}

}  // extern "C"
