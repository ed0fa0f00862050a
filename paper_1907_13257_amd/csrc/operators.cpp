// operators.cpp -- entry points of the operators around the recurrent layers:
// argument validation, resolved strides, launches.
#include <initializer_list>

#include "operators.hpp"
#include "status.hpp"

using namespace lstm355;

namespace {

// The status of a launch; nothing is thrown across the C boundary.
template <typename F>
lstm_status_t launched(const char *what, F launch)
{
    try {
        return hip_status(what, launch());
    } catch (...) {
        return invalid("exception");
    }
}

constexpr long MAX_INDEX = (1L << 31) - (1L << 20);   // rows of a table, tokens of a call: 32-bit positions

bool known(lstm_dtype_t t) { return t == LSTM_F32 || t == LSTM_BF16; }
DType dtype_of(lstm_dtype_t t) { return t == LSTM_BF16 ? DType::BF16 : DType::F32; }

// A row stride, 0 meaning dense; false when it is too short or no multiple of 8.
bool stride_ok(long given, long width, long *out)
{
    *out = given ? given : width;
    return *out >= width && *out % 8 == 0 && *out <= (1L << 40);
}

lstm_status_t check_embed(lstm_dtype_t dtype, long N, long V, int D, long ldo, long *ld)
{
    if (!known(dtype)) return invalid("unknown dtype");
    if (N < 0 || N > MAX_INDEX || V < 1 || V > MAX_INDEX) return invalid("N must be 0 .. 2^31 - 2^20 and V 1 .. 2^31 - 2^20");
    if (D < 8 || D % 8 || D > (1 << 20)) return invalid("D must be a multiple of 8, at most 2^20");
    if (!stride_ok(ldo, D, ld)) return invalid("ldo must be >= D and a multiple of 8");
    return LSTM_OK;
}

lstm_status_t check_norm(lstm_dtype_t dtype, long rows, int D, float eps, long *ldx, long *ldr, long *ldy)
{
    if (!known(dtype)) return invalid("unknown dtype");
    if (rows < 0 || rows > (1L << 40)) return invalid("rows must be 0 .. 2^40");
    if (D < 8 || D % 8) return invalid("D must be a multiple of 8");
    if (!(eps >= 0.0f)) return invalid("eps must not be negative");
    if (!stride_ok(*ldx, D, ldx) || !stride_ok(*ldr, D, ldr) || !stride_ok(*ldy, D, ldy))
        return invalid("row strides must be >= D and multiples of 8");
    if (D > NORM_MAX_D) {
        invalid("rows wider than 16384");
        return LSTM_ERR_UNSUPPORTED;
    }
    return LSTM_OK;
}

lstm_status_t add_norm_any(lstm_dtype_t dtype, long rows, int D, const void *x, long ldx, const void *res, long ldr,
                           const void *g, float eps, void *sum, void *y, long ldy, float *scale, bool q8, void *stream)
{
    const lstm_status_t st = check_norm(dtype, rows, D, eps, &ldx, &ldr, &ldy);
    if (st != LSTM_OK) return st;
    if (rows == 0) return LSTM_OK;
    if (!x || !g || !y || (q8 && !scale)) return invalid("required pointer is NULL");
    if (res && !sum) return invalid("sum is required with res");
    for (const void *p : {x, res, g, (const void *)sum, (const void *)y})
        if (p && !aligned16(p)) return invalid("device tensors must be 16-byte aligned");
    if (scale && !aligned4(scale)) return invalid("fp32 tensors must be 4-byte aligned");
    if (sum && sum == x && ldx != ldr) return invalid("sum may be x only when ldx = ldr");
    const NormArgs a{rows, D, x, res, g, ldx, ldr, ldy, eps, sum, y, scale};
    return launched("add_norm", [&] {
        return add_norm(dtype_of(dtype), a, static_cast<hipStream_t>(stream));
    });
}

lstm_status_t check_linattn(const lstm_linattn_desc_t *d, LinAttnShape *sh)
{
    if (!d) return invalid("desc is NULL");
    if (!known(d->dtype)) return invalid("unknown dtype");
    if (d->T < 1 || d->B < 1 || d->N < 1) return invalid("T, B and N must be positive");
    if (d->K < 8 || d->K > LINATTN_MAX_WIDTH || d->K % 8 || d->M < 8 || d->M > LINATTN_MAX_WIDTH || d->M % 8)
        return invalid("K and M must be multiples of 8 in 8 .. 256");
    if ((long)d->B * d->N > (1L << 22) || (long)d->T * d->B > (1L << 31) - 1 || d->T > (1 << 30))
        return invalid("sizes too large");
    if (!(d->scale == d->scale)) return invalid("scale is NaN");
    *sh = LinAttnShape{d->T, d->B, d->N, d->K, d->M, d->scale, 0, 0, 0, 0};
    if (!stride_ok(d->ldq, (long)d->N * d->K, &sh->ldq) || !stride_ok(d->ldk, (long)d->N * d->K, &sh->ldk) ||
        !stride_ok(d->ldv, (long)d->N * d->M, &sh->ldv) || !stride_ok(d->ldo, (long)d->N * d->M, &sh->ldo))
        return invalid("row strides must be >= the heads' columns and multiples of 8");
    return LSTM_OK;
}

lstm_status_t check_linattn_pointers(std::initializer_list<const void *> required,
                                     std::initializer_list<const void *> optional, const float *decay,
                                     const int32_t *lengths)
{
    for (const void *p : required)
        if (!p) return invalid("required pointer is NULL");
    if (!decay) return invalid("required pointer is NULL");
    for (const auto &list : {required, optional})
        for (const void *p : list)
            if (p && !aligned16(p)) return invalid("device tensors must be 16-byte aligned");
    if (!aligned4(decay) || !aligned4(lengths)) return invalid("decay and lengths must be 4-byte aligned");
    return LSTM_OK;
}

lstm_status_t check_workspace(const void *ws, size_t given, size_t need)
{
    if (given < need) return short_buffer("workspace", given, need);
    if (need && !ws) return invalid("required pointer is NULL");
    if (need && !aligned16(ws)) return invalid("device tensors must be 16-byte aligned");
    return LSTM_OK;
}

}  // namespace

extern "C" lstm_status_t lstm_embed_forward(lstm_dtype_t dtype, long N, long V, int D, const int64_t *ids,
                                            const void *table, float scale, void *out, long ldo, void *stream)
{
    long ld;
    const lstm_status_t st = check_embed(dtype, N, V, D, ldo, &ld);
    if (st != LSTM_OK) return st;
    if (N == 0) return LSTM_OK;
    if (!ids || !table || !out) return invalid("required pointer is NULL");
    for (const void *p : {table, (const void *)out})
        if (!aligned16(p)) return invalid("device tensors must be 16-byte aligned");
    if (!aligned8(ids)) return invalid("ids must be 8-byte aligned");
    return launched("embed_forward", [&] {
        return embed_forward(dtype_of(dtype), N, V, D, ids, table, scale, out, ld, static_cast<hipStream_t>(stream));
    });
}

extern "C" size_t lstm_embed_workspace_size(long N, long V, int D)
{
    long ld;
    return check_embed(LSTM_F32, N, V, D, 0, &ld) == LSTM_OK ? embed_workspace_bytes(N, V, D) : 0;
}

extern "C" lstm_status_t lstm_embed_backward(lstm_dtype_t dtype, long N, long V, int D, const int64_t *ids,
                                             const void *dout, long ldo, float scale, float *dtable, int accumulate,
                                             void *workspace, size_t workspace_bytes, void *stream)
{
    long ld;
    lstm_status_t st = check_embed(dtype, N, V, D, ldo, &ld);
    if (st != LSTM_OK) return st;
    if (accumulate != 0 && accumulate != 1) return invalid("accumulate must be 0 or 1");
    if (N == 0 && accumulate) return LSTM_OK;
    if (!dtable || (N > 0 && (!ids || !dout))) return invalid("required pointer is NULL");
    for (const void *p : {dout, (const void *)dtable})
        if (!aligned16(p)) return invalid("device tensors must be 16-byte aligned");
    if (!aligned8(ids)) return invalid("ids must be 8-byte aligned");
    st = check_workspace(workspace, workspace_bytes, embed_workspace_bytes(N, V, D));
    if (st != LSTM_OK) return st;
    return launched("embed_backward", [&] {
        return embed_backward(dtype_of(dtype), N, V, D, ids, dout, ld, scale, dtable, accumulate, workspace,
                              static_cast<hipStream_t>(stream));
    });
}

extern "C" lstm_status_t lstm_add_norm(lstm_dtype_t dtype, long rows, int D, const void *x, long ldx, const void *res,
                                       long ldr, const void *g, float eps, void *sum, void *y, long ldy, void *stream)
{
    return add_norm_any(dtype, rows, D, x, ldx, res, ldr, g, eps, sum, y, ldy, nullptr, false, stream);
}

extern "C" lstm_status_t lstm_add_norm_q8(lstm_dtype_t dtype, long rows, int D, const void *x, long ldx,
                                          const void *res, long ldr, const void *g, float eps, void *sum, uint8_t *y8,
                                          float *scale, void *stream)
{
    return add_norm_any(dtype, rows, D, x, ldx, res, ldr, g, eps, sum, y8, 0, scale, true, stream);
}

extern "C" size_t lstm_add_norm_workspace_size(long rows, int D)
{
    long a = 0, b = 0, c = 0;
    return check_norm(LSTM_F32, rows, D, 0.0f, &a, &b, &c) == LSTM_OK ? norm_partial_floats(rows, D) * 4 : 0;
}

extern "C" lstm_status_t lstm_add_norm_backward(lstm_dtype_t dtype, long rows, int D, const void *dy, long ldy,
                                                const void *dsum, const void *sum, long ldr, const void *g, float eps,
                                                void *dx, long ldx, float *dg, int accumulate, void *workspace,
                                                size_t workspace_bytes, void *stream)
{
    lstm_status_t st = check_norm(dtype, rows, D, eps, &ldx, &ldr, &ldy);
    if (st != LSTM_OK) return st;
    if (accumulate != 0 && accumulate != 1) return invalid("accumulate must be 0 or 1");
    if (rows == 0 && accumulate) return LSTM_OK;
    if (!dg || (rows > 0 && (!dy || !sum || !g || !dx))) return invalid("required pointer is NULL");
    for (const void *p : {dy, dsum, sum, g, (const void *)dx, (const void *)dg})
        if (p && !aligned16(p)) return invalid("device tensors must be 16-byte aligned");
    if ((dx == dsum || dx == sum) && ldx != ldr) return invalid("dx may be dsum or sum only when ldx = ldr");
    if (dx == dy && ldx != ldy) return invalid("dx may be dy only when ldx = ldy");
    st = check_workspace(workspace, workspace_bytes, norm_partial_floats(rows, D) * 4);
    if (st != LSTM_OK) return st;
    const NormBwdArgs a{rows, D, dy, dsum, sum, g, ldx, ldr, ldy, eps, dx, dg, accumulate, static_cast<float *>(workspace)};
    return launched("add_norm_backward", [&] {
        return add_norm_backward(dtype_of(dtype), a, static_cast<hipStream_t>(stream));
    });
}

extern "C" size_t lstm_linattn_workspace_size(const lstm_linattn_desc_t *d)
{
    LinAttnShape sh;
    return check_linattn(d, &sh) == LSTM_OK ? linattn_workspace_bytes(dtype_of(d->dtype), sh) : 0;
}

extern "C" lstm_status_t lstm_linattn_forward(const lstm_linattn_desc_t *d, const void *q, const void *k, const void *v,
                                              const float *decay, const int32_t *lengths, const float *S0, void *o,
                                              float *ST, void *workspace, size_t workspace_bytes, void *stream)
{
    LinAttnShape sh;
    lstm_status_t st = check_linattn(d, &sh);
    if (st == LSTM_OK) st = check_linattn_pointers({q, k, v, o}, {S0, ST}, decay, lengths);
    if (st == LSTM_OK) st = check_workspace(workspace, workspace_bytes, linattn_workspace_bytes(dtype_of(d->dtype), sh));
    if (st != LSTM_OK) return st;
    return launched("linattn_forward", [&] {
        return linattn_forward(dtype_of(d->dtype), sh, q, k, v, decay, lengths, S0, o, ST, workspace,
                               static_cast<hipStream_t>(stream));
    });
}

extern "C" lstm_status_t lstm_linattn_backward(const lstm_linattn_desc_t *d, const void *d_o, const void *q,
                                               const void *k, const void *v, const float *decay, const int32_t *lengths,
                                               const float *S0, const float *dST, void *dq, void *dk, void *dv,
                                               float *dS0, void *workspace, size_t workspace_bytes, void *stream)
{
    LinAttnShape sh;
    lstm_status_t st = check_linattn(d, &sh);
    if (st == LSTM_OK) st = check_linattn_pointers({d_o, q, k, v}, {S0, dST, dq, dk, dv, dS0}, decay, lengths);
    if (st == LSTM_OK) st = check_workspace(workspace, workspace_bytes, linattn_workspace_bytes(dtype_of(d->dtype), sh));
    if (st != LSTM_OK) return st;
    return launched("linattn_backward", [&] {
        return linattn_backward(dtype_of(d->dtype), sh, d_o, q, k, v, decay, lengths, S0, dST, dq, dk, dv, dS0,
                                workspace, static_cast<hipStream_t>(stream));
    });
}

extern "C" lstm_status_t lstm_linattn_step(const lstm_linattn_desc_t *d, const void *q, const void *k, const void *v,
                                           const float *decay, const int32_t *lengths, const float *S, float *S_out,
                                           void *o, void *stream)
{
    LinAttnShape sh;
    lstm_status_t st = check_linattn(d, &sh);
    if (st == LSTM_OK && sh.T != 1) st = invalid("a step takes one token: T must be 1");
    if (st == LSTM_OK) st = check_linattn_pointers({q, k, v, o, S, S_out}, {}, decay, lengths);
    if (st != LSTM_OK) return st;
    return launched("linattn_step", [&] {
        return linattn_step(dtype_of(d->dtype), sh, q, k, v, decay, lengths, S, S_out, o,
                            static_cast<hipStream_t>(stream));
    });
}
