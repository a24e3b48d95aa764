// The C entry points of the layer of experts: argument checks and launches.  No data is touched on the host.
#include <hip/hip_runtime.h>
#include "experts.hpp"
#include "internal.hpp"

using namespace polydl;

namespace {

bool aligned(const void *p, uintptr_t bytes) { return ((uintptr_t)p & (bytes - 1)) == 0; }
bool any_act(int act) { return act == POLYDL_ACT_NONE || act == POLYDL_ACT_RELU || act == POLYDL_ACT_RELU6; }
bool any_type(int type) { return type == POLYDL_F32 || type == POLYDL_BF16; }
bool aligned_type(const void *p, int type) { return aligned(p, type == POLYDL_F32 ? 4 : 2); }
// Lengths (groups, slots, columns, reductions) whose last tile, the stages asked for past their end and the row indices kept in LDS
// stay within the kernels' 32-bit arithmetic.
constexpr int kMaxLength = 0x7fff0000;
bool too_long(int E, int M, int N, int K) { return E > kMaxLength || M > kMaxLength || N > kMaxLength || K > kMaxLength; }
// element counts whose byte offsets a 64-bit product holds with room to spare
constexpr int64_t kMaxElements = 1ll << 60, kMaxRowStride = 1ll << 40;
bool too_many(int64_t a, int64_t b, int64_t c) { return (__int128)a * b * c >= kMaxElements; }

// hipErrorInvalidValue from a launcher here: no kernel holds the problem (2^31 - 2^20 workgroups)
int launched_or_refused(hipError_t e) { return e == hipErrorInvalidValue ? POLYDL_ERR_UNSUPPORTED : launched(e); }

}  // namespace

extern "C" {

size_t polydl_route_workspace_bytes(int T, int E)
{
    return T <= 0 || E <= 0 || E > kRouteMaxExperts ? 0 : route_workspace_bytes(T, E);
}

int polydl_route(int T, int E, int k, const float *logits, int renorm, int32_t *ids, float *weights, int32_t *offsets, int32_t *tokens,
                 int32_t *slots, void *workspace, size_t workspace_bytes, void *stream)
{
    if (T < 0 || E <= 0 || k <= 0 || k > E) return POLYDL_ERR_BAD_DIMENSION;
    if (!offsets || (T > 0 && (!logits || !ids || !weights || !tokens || !slots))) return POLYDL_ERR_NULL_POINTER;
    if (E > kRouteMaxExperts || k > kRouteMaxChoices || (int64_t)T * k > 0x7fffffffll) return POLYDL_ERR_UNSUPPORTED;
    if (!aligned(logits, 4) || !aligned(ids, 4) || !aligned(weights, 4) || !aligned(offsets, 4) || !aligned(tokens, 4) || !aligned(slots, 4))
        return POLYDL_ERR_UNSUPPORTED;
    const size_t need = polydl_route_workspace_bytes(T, E);
    if (need > 0) {
        if (!workspace) return POLYDL_ERR_NULL_POINTER;
        if (workspace_bytes < need) return POLYDL_ERR_BAD_DIMENSION;
        if (!aligned(workspace, 4)) return POLYDL_ERR_UNSUPPORTED;
    }
    if (!on_gfx950()) return POLYDL_ERR_NO_DEVICE;
    const RouteProblem p{T, E, k, logits, renorm != 0, ids, weights, offsets, tokens, slots};
    return launched(route_launch(p, workspace, (hipStream_t)stream));
}

int polydl_route_bwd(int T, int E, int k, const float *logits, const int32_t *ids, const float *weights, const float *dweights, int renorm,
                     float *dlogits, void *stream)
{
    if (T < 0 || E <= 0 || k <= 0 || k > E) return POLYDL_ERR_BAD_DIMENSION;
    if (T > 0 && (!ids || !dweights || !dlogits || (renorm ? !weights : !logits))) return POLYDL_ERR_NULL_POINTER;
    if (E > kRouteMaxExperts || k > kRouteMaxChoices || (int64_t)T * k > 0x7fffffffll) return POLYDL_ERR_UNSUPPORTED;
    if (!aligned(logits, 4) || !aligned(ids, 4) || !aligned(weights, 4) || !aligned(dweights, 4) || !aligned(dlogits, 4))
        return POLYDL_ERR_UNSUPPORTED;
    if (!on_gfx950()) return POLYDL_ERR_NO_DEVICE;
    if (T == 0) return POLYDL_OK;
    return launched(route_bwd_launch(T, E, k, logits, ids, weights, dweights, renorm != 0, dlogits, (hipStream_t)stream));
}

int polydl_combine_bf16(int T, int k, int M, int D, const uint16_t *y, const int32_t *slots, const float *weights, void *out, int out_type,
                        void *stream)
{
    if (T < 0 || k <= 0 || M < 0 || D <= 0) return POLYDL_ERR_BAD_DIMENSION;
    if (T > 0 && ((M > 0 && !y) || !slots || !out)) return POLYDL_ERR_NULL_POINTER;
    if (!any_type(out_type) || D > (1 << 24) || (int64_t)T * k > 0x7fffffffll) return POLYDL_ERR_UNSUPPORTED;
    if (!aligned(y, 2) || !aligned(slots, 4) || !aligned(weights, 4) || !aligned_type(out, out_type)) return POLYDL_ERR_UNSUPPORTED;
    if (!on_gfx950()) return POLYDL_ERR_NO_DEVICE;
    if (T == 0) return POLYDL_OK;
    return launched(combine_launch(T, k, M, D, y, slots, weights, out, out_type == POLYDL_F32, (hipStream_t)stream));
}

int polydl_combine_bwd_bf16(int T, int k, int M, int D, const uint16_t *dout, const uint16_t *y, const int32_t *slots, const float *weights,
                            uint16_t *dy, float *dweights, void *stream)
{
    if (T < 0 || k <= 0 || M < 0 || D <= 0) return POLYDL_ERR_BAD_DIMENSION;
    if (T > 0 && (!dout || !slots || (M > 0 && (!dy || (dweights && !y))))) return POLYDL_ERR_NULL_POINTER;
    if (D > (1 << 24) || (int64_t)T * k > 0x7fffffffll) return POLYDL_ERR_UNSUPPORTED;
    if (!aligned(dout, 2) || !aligned(y, 2) || !aligned(slots, 4) || !aligned(weights, 4) || !aligned(dy, 2) || !aligned(dweights, 4))
        return POLYDL_ERR_UNSUPPORTED;
    if (!on_gfx950()) return POLYDL_ERR_NO_DEVICE;
    if (T == 0) return POLYDL_OK;
    return launched(combine_bwd_launch(T, k, M, D, dout, y, slots, weights, dy, dweights, (hipStream_t)stream));
}

int polydl_grouped_gemm_bf16(int E, int M, int N, int K, const int32_t *offsets, const int32_t *rows, int x_rows, const uint16_t *x, int64_t ldx,
                             const uint16_t *w, void *y, int64_t ldy, int out_type, int act, void *stream)
{
    if (E <= 0 || M < 0 || N <= 0 || K <= 0 || ldx < K || ldy < N || x_rows < 0 || (!rows && x_rows != M)) return POLYDL_ERR_BAD_DIMENSION;
    if (!offsets || !w || (M > 0 && ((x_rows > 0 && !x) || !y))) return POLYDL_ERR_NULL_POINTER;
    if (!any_act(act) || !any_type(out_type) || ldx > kMaxRowStride || ldy > kMaxRowStride || too_long(E, M, N, K) || too_many(E, N, K))
        return POLYDL_ERR_UNSUPPORTED;
    if (!aligned(offsets, 4) || !aligned(rows, 4) || !aligned(x, 2) || !aligned(w, 2) || !aligned_type(y, out_type)) return POLYDL_ERR_UNSUPPORTED;
    if (!on_gfx950()) return POLYDL_ERR_NO_DEVICE;
    if (M == 0) return POLYDL_OK;
    GroupedProblem q{};
    q.form = GROUPED_FWD;
    q.E = E; q.M = M; q.cols = N; q.red = K;
    q.offsets = offsets; q.rows = rows; q.src_rows = x_rows;
    q.a = x; q.lda = ldx; q.b = w; q.ldb = K;
    q.c = y; q.ldc = ldy; q.out_f32 = out_type == POLYDL_F32; q.act = act;
    return launched_or_refused(grouped_gemm_launch(q, (hipStream_t)stream));
}

int polydl_grouped_gemm_dx_bf16(int E, int M, int N, int K, const int32_t *offsets, const uint16_t *dy, int64_t lddy, const uint16_t *w,
                                const uint16_t *h, int64_t ldh, int act, void *dx, int64_t lddx, int out_type, void *stream)
{
    if (E <= 0 || M < 0 || N <= 0 || K <= 0 || lddy < N || lddx < K || (act != POLYDL_ACT_NONE && ldh < K)) return POLYDL_ERR_BAD_DIMENSION;
    if (!offsets || !w || (M > 0 && (!dy || !dx || (act != POLYDL_ACT_NONE && !h)))) return POLYDL_ERR_NULL_POINTER;
    if (!any_act(act) || !any_type(out_type) || lddy > kMaxRowStride || lddx > kMaxRowStride || ldh > kMaxRowStride ||
        too_long(E, M, N, K) || too_many(E, N, K))
        return POLYDL_ERR_UNSUPPORTED;
    if (!aligned(offsets, 4) || !aligned(dy, 2) || !aligned(w, 2) || !aligned(h, 2) || !aligned_type(dx, out_type)) return POLYDL_ERR_UNSUPPORTED;
    if (!on_gfx950()) return POLYDL_ERR_NO_DEVICE;
    if (M == 0) return POLYDL_OK;
    GroupedProblem q{};
    q.form = GROUPED_DX;
    q.E = E; q.M = M; q.cols = K; q.red = N;
    q.offsets = offsets; q.src_rows = M;
    q.a = dy; q.lda = lddy; q.b = w; q.ldb = K;
    q.c = dx; q.ldc = lddx; q.out_f32 = out_type == POLYDL_F32;
    q.act = act; q.h = h; q.ldh = act == POLYDL_ACT_NONE ? 0 : ldh;
    return launched_or_refused(grouped_gemm_launch(q, (hipStream_t)stream));
}

int polydl_grouped_gemm_dw_bf16(int E, int M, int N, int K, const int32_t *offsets, const uint16_t *dy, int64_t lddy, const int32_t *rows,
                                int x_rows, const uint16_t *x, int64_t ldx, void *dw, int out_type, int accumulate, void *stream)
{
    if (E <= 0 || M < 0 || N <= 0 || K <= 0 || lddy < N || ldx < K || x_rows < 0 || (!rows && x_rows != M)) return POLYDL_ERR_BAD_DIMENSION;
    if (!offsets || !dw || (M > 0 && (!dy || (x_rows > 0 && !x)))) return POLYDL_ERR_NULL_POINTER;
    if (!any_type(out_type) || (accumulate && out_type != POLYDL_F32) || lddy > kMaxRowStride || ldx > kMaxRowStride ||
        too_long(E, M, N, K) || too_many(E, N, K))
        return POLYDL_ERR_UNSUPPORTED;
    if (!aligned(offsets, 4) || !aligned(rows, 4) || !aligned(dy, 2) || !aligned(x, 2) || !aligned_type(dw, out_type)) return POLYDL_ERR_UNSUPPORTED;
    if (!on_gfx950()) return POLYDL_ERR_NO_DEVICE;
    if (M == 0 && accumulate) return POLYDL_OK;
    GroupedProblem q{};
    q.form = GROUPED_DW;
    q.E = E; q.M = M; q.out_rows = N; q.cols = K;
    q.offsets = offsets; q.rows = rows; q.src_rows = x_rows;
    q.a = dy; q.lda = lddy; q.b = x; q.ldb = ldx;
    q.c = dw; q.ldc = K; q.out_f32 = out_type == POLYDL_F32; q.accumulate = accumulate != 0;
    return launched_or_refused(grouped_gemm_launch(q, (hipStream_t)stream));
}

static bool w4_group(int group) { return group == 32 || group == 64 || group == 128; }

int polydl_w4_pack_bf16(int E, int N, int K, int group, const uint16_t *w, uint8_t *q, uint16_t *scales, uint8_t *zeros, void *stream)
{
    if (E <= 0 || N <= 0 || K <= 0) return POLYDL_ERR_BAD_DIMENSION;
    if (!w || !q || !scales) return POLYDL_ERR_NULL_POINTER;
    if (!w4_group(group) || too_long(E, 0, N, K) || too_many(E, (int64_t)N + 15, (int64_t)K + 127)) return POLYDL_ERR_UNSUPPORTED;
    if (!aligned(w, 2) || !aligned(q, 16) || !aligned(scales, 8)) return POLYDL_ERR_UNSUPPORTED;
    if (!on_gfx950()) return POLYDL_ERR_NO_DEVICE;
    return launched_or_refused(w4_pack_launch(E, N, K, group, w, q, scales, zeros, (hipStream_t)stream));
}

int polydl_w4_gemm_bf16(int E, int M, int N, int K, int group, const int32_t *offsets, const int32_t *rows, int x_rows, const uint16_t *x,
                        int64_t ldx, const uint8_t *q, const uint16_t *scales, const uint8_t *zeros, void *y, int64_t ldy, int out_type, int act,
                        void *stream)
{
    if (E <= 0 || M < 0 || N <= 0 || K <= 0 || ldx < K || ldy < N || x_rows < 0 || (!rows && x_rows != M)) return POLYDL_ERR_BAD_DIMENSION;
    if ((E > 1 && !offsets) || !q || !scales || (M > 0 && ((x_rows > 0 && !x) || !y))) return POLYDL_ERR_NULL_POINTER;
    if (!w4_group(group) || !any_act(act) || !any_type(out_type) || ldx > kMaxRowStride || ldy > kMaxRowStride || too_long(E, M, N, K) ||
        too_many(E, (int64_t)N + 15, (int64_t)K + 127))
        return POLYDL_ERR_UNSUPPORTED;
    if (!aligned(offsets, 4) || !aligned(rows, 4) || !aligned(x, 2) || !aligned(q, 16) || !aligned(scales, 8) ||
        !aligned_type(y, out_type))
        return POLYDL_ERR_UNSUPPORTED;
    if (!on_gfx950()) return POLYDL_ERR_NO_DEVICE;
    if (M == 0) return POLYDL_OK;
    const FewRowsProblem p{E, M, N, K, group, offsets, rows, x_rows, x, ldx, nullptr, q, scales, zeros, y, ldy, out_type == POLYDL_F32, act};
    return launched_or_refused(few_rows_launch(p, (hipStream_t)stream));
}

}  // extern "C"
