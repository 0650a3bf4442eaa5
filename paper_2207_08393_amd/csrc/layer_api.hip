// C ABI of the sequence-layer operators: host-side validation, then the kernels of norm.hip, dropout.hip and linattn.hip on the
// caller's stream.
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

// An array of a linear attention call: strides that reach no further than they may, and that keep elements apart where it is written.
int check_strides(const gleam_linattn_desc& d, const gleam_seq_strides& s, int heads, int width, bool written) {
    struct Axis {
        long long n, stride;
    } axis[4] = {{d.B, s.b}, {d.T, s.t}, {d.P, s.p}, {heads, s.h}};
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
    int rc = check_strides(*d, d->q, d->q_heads, d->dk, gradients);
    if (!rc) rc = check_strides(*d, d->k, d->k_heads, d->dk, gradients);
    if (!rc) rc = check_strides(*d, d->v, d->v_heads, d->dv, gradients);
    if (!rc) rc = check_strides(*d, d->o, d->heads, d->dv, !gradients);
    return rc;
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

}  // extern "C"
