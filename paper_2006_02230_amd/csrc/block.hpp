// Host-side declarations of what stands around a layer of experts: layer norm, balance loss, gradient norm and clipping, products in
// microscaled 4 bits (not part of the C ABI).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace polydl {

// norm_kernels.hip
struct NormProblem {
    int T, D;
    const void *x;
    int64_t ldx;
    bool x_f32;
    const float *gamma, *beta;      // NULL: ones, zeros
    float eps;
    void *y;
    int64_t ldy;
    bool y_f32;
    float *mean, *rstd;
};
struct NormGradProblem {
    int T, D;
    const void *dy, *x;
    int64_t lddy, ldx;
    bool dy_f32, x_f32;
    const float *mean, *rstd, *gamma;
    void *dx;                       // NULL: not asked for; so dgamma, dbeta
    int64_t lddx;
    float *dgamma, *dbeta;
    bool accumulate;
};
hipError_t norm_launch(const NormProblem &p, hipStream_t st);
size_t norm_bwd_workspace_bytes(int T, int D);
hipError_t norm_bwd_launch(const NormGradProblem &p, void *workspace, hipStream_t st);

// balance_kernels.hip (E <= kRouteMaxExperts)
struct BalanceProblem {
    int T, E, k;
    const float *logits;
    const int32_t *ids;
    float *loss;
    int32_t *counts;
    float *shares;
    int32_t *rows;
};
size_t balance_workspace_bytes(int T, int E);
hipError_t balance_launch(const BalanceProblem &p, void *workspace, hipStream_t st);
hipError_t balance_bwd_launch(int T, int E, const float *logits, const int32_t *counts, const int32_t *rows, float coefficient, const float *dloss,
                              float *dlogits, bool accumulate, hipStream_t st);

// clip_kernels.hip
size_t clip_workspace_bytes(int n, const int64_t *counts);
// out NULL: the norm alone
hipError_t clip_launch(int n, const void *const *grads, const int64_t *counts, const int *types, double max_norm, void *const *out, float *norm,
                       void *workspace, hipStream_t st);

// mx4_kernels.hip, mx4_gemm.hip
inline int mx4_blocks(int K) { return (int)(((int64_t)K + 127) / 128) * 4; }
hipError_t mx4_quantise_launch(int64_t rows, int K, const void *x, int64_t ldx, bool x_f32, uint8_t *q, uint8_t *scales, hipStream_t st);
hipError_t mx4_dequantise_launch(int64_t rows, int K, const uint8_t *q, const uint8_t *scales, void *y, int64_t ldy, bool y_f32, hipStream_t st);
struct Mx4Problem {
    int E, M, N, KB;                // KB: blocks of 32 inputs a row, a multiple of 4
    const int32_t *offsets, *rows;  // offsets NULL: one group of all rows
    int x_rows;
    const uint8_t *xq, *xs, *wq, *ws;
    void *y;
    int64_t ldy;
    bool out_f32;
    int act;                        // polydl_act
};
hipError_t mx4_gemm_launch(const Mx4Problem &p, hipStream_t st);           // hipErrorInvalidValue: no kernel holds it

}  // namespace polydl
