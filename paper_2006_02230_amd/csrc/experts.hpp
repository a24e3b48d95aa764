// Host-side declarations of the layer of experts: the router, the products grouped by expert, the weighted sum, the products
// with 4-bit weights (not part of the C ABI).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace polydl {

// route_kernels.hip
constexpr int kRouteMaxExperts = 1024, kRouteMaxChoices = 32;
constexpr int kRouteTokens = 64;                       // tokens of a workgroup: a bit each in two words
struct RouteProblem {
    int T, E, k;
    const float *logits;
    bool renorm;
    int32_t *ids;
    float *weights;
    int32_t *offsets, *tokens, *slots;
};
size_t route_workspace_bytes(int T, int E);
hipError_t route_launch(const RouteProblem &p, void *workspace, hipStream_t st);
hipError_t route_bwd_launch(int T, int E, int k, const float *logits, const int32_t *ids, const float *weights, const float *dweights,
                            bool renorm, float *dlogits, hipStream_t st);
hipError_t combine_launch(int T, int k, int M, int D, const uint16_t *y, const int32_t *slots, const float *weights, void *out,
                          bool out_f32, hipStream_t st);
hipError_t combine_bwd_launch(int T, int k, int M, int D, const uint16_t *dout, const uint16_t *y, const int32_t *slots,
                              const float *weights, uint16_t *dy, float *dweights, hipStream_t st);

// grouped_gemm.hip: products of bfloat16 matrices, a weight matrix a group of rows.  `form` names what is asked for:
//   GROUPED_FWD  c[s] = act(a[row(s)] B_e^T)    a [a_rows][red], B_e [cols][red]
//   GROUPED_DX   c[s] = (a[s] B_e) * act'(h[s]) a [M][red],      B_e [red][cols]
//   GROUPED_DW   C_e  = sum_{s in e} a[s]^T b[row(s)]   a [M][rows of C_e], b [b_rows][cols]
enum { GROUPED_FWD = 0, GROUPED_DX = 1, GROUPED_DW = 2 };
struct GroupedProblem {
    int form;
    int E, M;                      // groups, slots
    int out_rows, cols, red;       // of the result: rows (GROUPED_DW), columns; the reduction (not GROUPED_DW)
    const int32_t *offsets, *rows; // [E+1]; [M] or NULL
    int src_rows;                  // rows of the tensor that `rows` indexes
    const uint16_t *a, *b;
    int64_t lda, ldb;              // elements from row to row; ldb inside one B_e (not GROUPED_DW: dense)
    void *c;
    int64_t ldc;
    bool out_f32, accumulate;
    int act;                       // polydl_act
    const uint16_t *h;             // GROUPED_DX: what the activation gave, [M][cols], rows ldh apart; NULL: no activation
    int64_t ldh;
};
hipError_t grouped_gemm_launch(const GroupedProblem &p, hipStream_t st);   // hipErrorInvalidValue: no kernel holds it

// few_rows.hip: products of few rows, with weights in bfloat16 (w) or in 4 bits, a scale (and a zero point) for `group` inputs of
// an output.
struct FewRowsProblem {
    int E, M, N, K, group;
    const int32_t *offsets, *rows;  // offsets NULL: one group of all rows
    int src_rows;
    const uint16_t *x;
    int64_t ldx;
    const uint16_t *w;              // NULL: in 4 bits
    const uint8_t *q;
    const uint16_t *scales;
    const uint8_t *zeros;           // NULL: 8
    void *y;
    int64_t ldy;
    bool out_f32;
    int act;
};
hipError_t few_rows_launch(const FewRowsProblem &p, hipStream_t st);
// w4_kernels.hip
hipError_t w4_pack_launch(int E, int N, int K, int group, const uint16_t *w, uint8_t *q, uint16_t *scales, uint8_t *zeros, hipStream_t st);

}  // namespace polydl
