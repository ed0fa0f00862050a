// operators.hpp -- host-side launch interface of the operators around the
// recurrent layers: embedding, residual norm, linear attention.  Arguments
// have been validated (operators.cpp); strides are resolved, in elements.
#pragma once
#include "kernels.hpp"

namespace lstm355 {

// --- embed.hip ---------------------------------------------------------------
hipError_t embed_forward(DType t, long N, long V, int D, const int64_t *ids, const void *table, float scale, void *out,
                         long ldo, hipStream_t s);
size_t embed_workspace_bytes(long N, long V, int D);
hipError_t embed_backward(DType t, long N, long V, int D, const int64_t *ids, const void *dout, long ldo, float scale,
                          float *dtable, int accumulate, void *ws, hipStream_t s);

// --- norm.hip ----------------------------------------------------------------
constexpr int NORM_MAX_D = 16384;
struct NormArgs {
    long rows;
    int D;
    const void *x, *res, *g;
    long ldx, ldr, ldy;
    float eps;
    void *sum, *y;            // y: storage type, or e4m3 when scale is given
    float *scale;
};
hipError_t add_norm(DType t, const NormArgs &a, hipStream_t s);
struct NormBwdArgs {
    long rows;
    int D;
    const void *dy, *dsum, *sum, *g;
    long ldx, ldr, ldy;
    float eps;
    void *dx;
    float *dg;
    int accumulate;
    float *partial;           // norm_partial_floats(rows, D) floats
};
size_t norm_partial_floats(long rows, int D);
hipError_t add_norm_backward(DType t, const NormBwdArgs &a, hipStream_t s);

// --- linattn.hip -------------------------------------------------------------
constexpr int LINATTN_MAX_WIDTH = 256;
struct LinAttnShape {
    int T, B, N, K, M;
    float scale;
    long ldq, ldk, ldv, ldo;
};
size_t linattn_workspace_bytes(DType t, const LinAttnShape &sh);
hipError_t linattn_forward(DType t, const LinAttnShape &sh, const void *q, const void *k, const void *v,
                           const float *decay, const int32_t *lengths, const float *S0, void *o, float *ST, void *ws,
                           hipStream_t s);
hipError_t linattn_backward(DType t, const LinAttnShape &sh, const void *d_o, const void *q, const void *k,
                            const void *v, const float *decay, const int32_t *lengths, const float *S0,
                            const float *dST, void *dq, void *dk, void *dv, float *dS0, void *ws, hipStream_t s);
hipError_t linattn_step(DType t, const LinAttnShape &sh, const void *q, const void *k, const void *v,
                        const float *decay, const int32_t *lengths, const float *S, float *S_out, void *o,
                        hipStream_t s);

}  // namespace lstm355
