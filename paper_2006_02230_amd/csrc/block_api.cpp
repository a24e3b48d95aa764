// The C entry points of what stands around a layer of experts: argument checks and launches.  No data is touched on the host.
#include <hip/hip_runtime.h>
#include <math.h>
#include <algorithm>
#include <new>
#include "block.hpp"
#include "experts.hpp"
#include "internal.hpp"

using namespace polydl;

namespace {

bool aligned(const void *p, uintptr_t bytes) { return ((uintptr_t)p & (bytes - 1)) == 0; }
bool any_act(int act) { return act == POLYDL_ACT_NONE || act == POLYDL_ACT_RELU || act == POLYDL_ACT_RELU6; }
bool any_type(int type) { return type == POLYDL_F32 || type == POLYDL_BF16; }
int type_bytes(int type) { return type == POLYDL_F32 ? 4 : 2; }
bool aligned_type(const void *p, int type) { return aligned(p, type_bytes(type)); }
// lengths whose last tile stays within the kernels' 32-bit arithmetic; strides and counts whose byte offsets 64 bits hold with room to spare
constexpr int kMaxLength = 0x7fff0000, kMaxRow = 1 << 24;
constexpr int64_t kMaxRowStride = 1ll << 40, kMaxElements = 1ll << 60, kMaxValues = 1ll << 42;
bool too_many(int64_t a, int64_t b, int64_t c) { return (__int128)a * b * c >= kMaxElements; }

// hipErrorInvalidValue from a launcher here: no kernel holds the problem
int launched_or_refused(hipError_t e) { return e == hipErrorInvalidValue ? POLYDL_ERR_UNSUPPORTED : launched(e); }

int clip_check(int n, const void *const *grads, const int64_t *counts, const int *types, const float *norm)
{
    if (n < 0) return POLYDL_ERR_BAD_DIMENSION;
    if (!norm || (n > 0 && (!grads || !counts || !types))) return POLYDL_ERR_NULL_POINTER;
    for (int i = 0; i < n; ++i) {
        if (counts[i] < 0) return POLYDL_ERR_BAD_DIMENSION;
        if (counts[i] > 0 && !grads[i]) return POLYDL_ERR_NULL_POINTER;
        if (!any_type(types[i]) || counts[i] > kMaxValues) return POLYDL_ERR_UNSUPPORTED;
        if (!aligned_type(grads[i], types[i])) return POLYDL_ERR_UNSUPPORTED;
    }
    return aligned(norm, 4) ? POLYDL_OK : POLYDL_ERR_UNSUPPORTED;
}

int clip_workspace(int n, const int64_t *counts, const void *workspace, size_t bytes)
{
    if (!workspace) return POLYDL_ERR_NULL_POINTER;
    if (bytes < clip_workspace_bytes(n, counts)) return POLYDL_ERR_BAD_DIMENSION;
    return aligned(workspace, 8) ? POLYDL_OK : POLYDL_ERR_UNSUPPORTED;
}

struct Span { uintptr_t begin, end; bool written; };

// Whether a tensor that is written overlaps another one: the launches would read or scale its values twice.
int clip_overlap(int n, const void *const *grads, const int64_t *counts, const int *types, void *const *out)
{
    Span *spans = new (std::nothrow) Span[2 * (size_t)n + 1];
    if (!spans) return POLYDL_ERR_LAUNCH;
    size_t count = 0;
    for (int i = 0; i < n; ++i) {
        if (counts[i] == 0) continue;
        const uintptr_t bytes = (uintptr_t)counts[i] * type_bytes(types[i]), from = (uintptr_t)grads[i], to = (uintptr_t)out[i];
        spans[count++] = {to, to + bytes, true};
        if (from != to) spans[count++] = {from, from + bytes, false};
    }
    std::sort(spans, spans + count, [](const Span &a, const Span &b) { return a.begin < b.begin; });
    uintptr_t read = 0, written = 0;        // how far what came before goes
    bool bad = false;
    for (size_t i = 0; i < count; ++i) {
        bad |= spans[i].begin < written || (spans[i].written && spans[i].begin < read);
        (spans[i].written ? written : read) = std::max(spans[i].written ? written : read, spans[i].end);
    }
    delete[] spans;
    return bad ? POLYDL_ERR_UNSUPPORTED : POLYDL_OK;
}

}  // namespace

extern "C" {

int polydl_layernorm_fwd(int T, int D, const void *x, int64_t ldx, int x_type, const float *gamma, const float *beta, float eps, void *y,
                         int64_t ldy, int y_type, float *mean, float *rstd, void *stream)
{
    if (T < 0 || D <= 0 || ldx < D || ldy < D) return POLYDL_ERR_BAD_DIMENSION;
    if (T > 0 && (!x || !y)) return POLYDL_ERR_NULL_POINTER;
    if (!any_type(x_type) || !any_type(y_type) || D > kMaxRow || ldx > kMaxRowStride || ldy > kMaxRowStride || !(eps >= 0.f) || eps == INFINITY)
        return POLYDL_ERR_UNSUPPORTED;
    if (!aligned_type(x, x_type) || !aligned_type(y, y_type) || !aligned(gamma, 4) || !aligned(beta, 4) || !aligned(mean, 4) || !aligned(rstd, 4))
        return POLYDL_ERR_UNSUPPORTED;
    if (!on_gfx950()) return POLYDL_ERR_NO_DEVICE;
    if (T == 0) return POLYDL_OK;
    const NormProblem p{T, D, x, ldx, x_type == POLYDL_F32, gamma, beta, eps, y, ldy, y_type == POLYDL_F32, mean, rstd};
    return launched(norm_launch(p, (hipStream_t)stream));
}

size_t polydl_layernorm_bwd_workspace_bytes(int T, int D)
{
    return T <= 0 || D <= 0 || D > kMaxRow ? 0 : norm_bwd_workspace_bytes(T, D);
}

int polydl_layernorm_bwd(int T, int D, const void *dy, int64_t lddy, int dy_type, const void *x, int64_t ldx, int x_type, const float *mean,
                         const float *rstd, const float *gamma, void *dx, int64_t lddx, float *dgamma, float *dbeta, int accumulate,
                         void *workspace, size_t workspace_bytes, void *stream)
{
    if (T < 0 || D <= 0 || lddy < D || ldx < D || (dx && lddx < D)) return POLYDL_ERR_BAD_DIMENSION;
    if (T > 0 && (!dy || !x || !mean || !rstd)) return POLYDL_ERR_NULL_POINTER;
    if (!any_type(dy_type) || !any_type(x_type) || D > kMaxRow || lddy > kMaxRowStride || ldx > kMaxRowStride || (dx && lddx > kMaxRowStride))
        return POLYDL_ERR_UNSUPPORTED;
    if (!aligned_type(dy, dy_type) || !aligned_type(x, x_type) || !aligned_type(dx, x_type) || !aligned(mean, 4) || !aligned(rstd, 4) ||
        !aligned(gamma, 4) || !aligned(dgamma, 4) || !aligned(dbeta, 4))
        return POLYDL_ERR_UNSUPPORTED;
    const size_t need = dgamma || dbeta ? polydl_layernorm_bwd_workspace_bytes(T, D) : 0;
    if (need > 0) {
        if (!workspace) return POLYDL_ERR_NULL_POINTER;
        if (workspace_bytes < need) return POLYDL_ERR_BAD_DIMENSION;
        if (!aligned(workspace, 4)) return POLYDL_ERR_UNSUPPORTED;
    }
    if (!on_gfx950()) return POLYDL_ERR_NO_DEVICE;
    if (T == 0 && (accumulate || (!dgamma && !dbeta))) return POLYDL_OK;
    const NormGradProblem p{T,    D,     dy, x,    lddy,   ldx,   dy_type == POLYDL_F32, x_type == POLYDL_F32, mean,
                            rstd, gamma, dx, lddx, dgamma, dbeta, accumulate != 0};
    return launched(norm_bwd_launch(p, workspace, (hipStream_t)stream));
}

size_t polydl_balance_workspace_bytes(int T, int E)
{
    return T <= 0 || E <= 0 || E > kRouteMaxExperts ? 0 : balance_workspace_bytes(T, E);
}

int polydl_balance(int T, int E, int k, const float *logits, const int32_t *ids, float *loss, int32_t *counts, float *shares, int32_t *rows,
                   void *workspace, size_t workspace_bytes, void *stream)
{
    if (T < 0 || E <= 0 || k <= 0) return POLYDL_ERR_BAD_DIMENSION;
    if (!loss || !counts || !shares || !rows || (T > 0 && (!logits || !ids))) return POLYDL_ERR_NULL_POINTER;
    if (E > kRouteMaxExperts || k > kRouteMaxChoices || (int64_t)T * k > 0x7fffffffll) return POLYDL_ERR_UNSUPPORTED;
    if (!aligned(logits, 4) || !aligned(ids, 4) || !aligned(loss, 4) || !aligned(counts, 4) || !aligned(shares, 4) || !aligned(rows, 4))
        return POLYDL_ERR_UNSUPPORTED;
    const size_t need = polydl_balance_workspace_bytes(T, E);
    if (need > 0) {
        if (!workspace) return POLYDL_ERR_NULL_POINTER;
        if (workspace_bytes < need) return POLYDL_ERR_BAD_DIMENSION;
        if (!aligned(workspace, 4)) return POLYDL_ERR_UNSUPPORTED;
    }
    if (!on_gfx950()) return POLYDL_ERR_NO_DEVICE;
    const BalanceProblem p{T, E, k, logits, ids, loss, counts, shares, rows};
    return launched(balance_launch(p, workspace, (hipStream_t)stream));
}

int polydl_balance_bwd(int T, int E, const float *logits, const int32_t *counts, const int32_t *rows, float coefficient, const float *dloss,
                       float *dlogits, int accumulate, void *stream)
{
    if (T < 0 || E <= 0) return POLYDL_ERR_BAD_DIMENSION;
    if (T > 0 && (!logits || !counts || !rows || !dlogits)) return POLYDL_ERR_NULL_POINTER;
    if (E > kRouteMaxExperts) return POLYDL_ERR_UNSUPPORTED;
    if (!aligned(logits, 4) || !aligned(counts, 4) || !aligned(rows, 4) || !aligned(dloss, 4) || !aligned(dlogits, 4)) return POLYDL_ERR_UNSUPPORTED;
    if (!on_gfx950()) return POLYDL_ERR_NO_DEVICE;
    if (T == 0) return POLYDL_OK;
    return launched(balance_bwd_launch(T, E, logits, counts, rows, coefficient, dloss, dlogits, accumulate != 0, (hipStream_t)stream));
}

size_t polydl_clip_workspace_bytes(int n, const int64_t *counts)
{
    if (n < 0 || (n > 0 && !counts)) return 0;
    for (int i = 0; i < n; ++i)
        if (counts[i] < 0 || counts[i] > kMaxValues) return 0;
    return clip_workspace_bytes(n, counts);
}

int polydl_grad_norm(int n, const void *const *grads, const int64_t *counts, const int *types, float *norm, void *workspace,
                     size_t workspace_bytes, void *stream)
{
    int s = clip_check(n, grads, counts, types, norm);
    if (s == POLYDL_OK) s = clip_workspace(n, counts, workspace, workspace_bytes);
    if (s != POLYDL_OK) return s;
    if (!on_gfx950()) return POLYDL_ERR_NO_DEVICE;
    return launched(clip_launch(n, grads, counts, types, 0.0, nullptr, norm, workspace, (hipStream_t)stream));
}

int polydl_clip_grads(int n, const void *const *grads, const int64_t *counts, const int *types, double max_norm, void *const *out,
                      float *norm, void *workspace, size_t workspace_bytes, void *stream)
{
    int s = clip_check(n, grads, counts, types, norm);
    if (s != POLYDL_OK) return s;
    if (!(max_norm >= 0.0)) return POLYDL_ERR_UNSUPPORTED;
    void *const *to = out ? out : const_cast<void *const *>(grads);
    for (int i = 0; i < n; ++i) {
        if (counts[i] > 0 && !to[i]) return POLYDL_ERR_NULL_POINTER;
        if (!aligned_type(to[i], types[i])) return POLYDL_ERR_UNSUPPORTED;
    }
    s = clip_workspace(n, counts, workspace, workspace_bytes);
    if (s == POLYDL_OK) s = clip_overlap(n, grads, counts, types, to);
    if (s != POLYDL_OK) return s;
    if (!on_gfx950()) return POLYDL_ERR_NO_DEVICE;
    return launched(clip_launch(n, grads, counts, types, max_norm, to, norm, workspace, (hipStream_t)stream));
}

int polydl_mx4_quantise(int64_t rows, int K, const void *x, int64_t ldx, int x_type, uint8_t *q, uint8_t *scales, void *stream)
{
    if (rows < 0 || K <= 0 || ldx < K) return POLYDL_ERR_BAD_DIMENSION;
    if (rows > 0 && (!x || !q || !scales)) return POLYDL_ERR_NULL_POINTER;
    if (!any_type(x_type) || K > kMaxLength || ldx > kMaxRowStride || too_many(rows, 1, (int64_t)K + 127)) return POLYDL_ERR_UNSUPPORTED;
    if (!aligned_type(x, x_type) || !aligned(q, 16) || !aligned(scales, 4)) return POLYDL_ERR_UNSUPPORTED;
    if (!on_gfx950()) return POLYDL_ERR_NO_DEVICE;
    if (rows == 0) return POLYDL_OK;
    return launched_or_refused(mx4_quantise_launch(rows, K, x, ldx, x_type == POLYDL_F32, q, scales, (hipStream_t)stream));
}

int polydl_mx4_dequantise(int64_t rows, int K, const uint8_t *q, const uint8_t *scales, void *y, int64_t ldy, int y_type, void *stream)
{
    if (rows < 0 || K <= 0 || ldy < K) return POLYDL_ERR_BAD_DIMENSION;
    if (rows > 0 && (!y || !q || !scales)) return POLYDL_ERR_NULL_POINTER;
    if (!any_type(y_type) || K > kMaxLength || ldy > kMaxRowStride || too_many(rows, 1, (int64_t)K + 127)) return POLYDL_ERR_UNSUPPORTED;
    if (!aligned_type(y, y_type) || !aligned(q, 16) || !aligned(scales, 4)) return POLYDL_ERR_UNSUPPORTED;
    if (!on_gfx950()) return POLYDL_ERR_NO_DEVICE;
    if (rows == 0) return POLYDL_OK;
    return launched_or_refused(mx4_dequantise_launch(rows, K, q, scales, y, ldy, y_type == POLYDL_F32, (hipStream_t)stream));
}

int polydl_mx4_gemm(int E, int M, int N, int K, const int32_t *offsets, const int32_t *rows, int x_rows, const uint8_t *xq,
                    const uint8_t *x_scales, const uint8_t *wq, const uint8_t *w_scales, void *y, int64_t ldy, int out_type, int act, void *stream)
{
    if (E <= 0 || M < 0 || N <= 0 || K <= 0 || ldy < N || x_rows < 0 || (!rows && x_rows != M)) return POLYDL_ERR_BAD_DIMENSION;
    if ((E > 1 && !offsets) || !wq || !w_scales || (M > 0 && ((x_rows > 0 && (!xq || !x_scales)) || !y))) return POLYDL_ERR_NULL_POINTER;
    if (!any_act(act) || !any_type(out_type) || ldy > kMaxRowStride || E > kMaxLength || M > kMaxLength || N > kMaxLength || K > kMaxLength ||
        too_many(E, (int64_t)N + 255, (int64_t)K + 127))
        return POLYDL_ERR_UNSUPPORTED;
    if (!aligned(offsets, 4) || !aligned(rows, 4) || !aligned(xq, 16) || !aligned(x_scales, 4) || !aligned(wq, 16) || !aligned(w_scales, 4) ||
        !aligned_type(y, out_type))
        return POLYDL_ERR_UNSUPPORTED;
    if (!on_gfx950()) return POLYDL_ERR_NO_DEVICE;
    if (M == 0) return POLYDL_OK;
    const Mx4Problem p{E, M, N, mx4_blocks(K), offsets, rows, x_rows, xq, x_scales, wq, w_scales, y, ldy, out_type == POLYDL_F32, act};
    return launched_or_refused(mx4_gemm_launch(p, (hipStream_t)stream));
}

}  // extern "C"
