// linattn.hip -- linear attention with one decay per head: whole sequences,
// their gradients, and single tokens.
//
// Every direction is the same recurrence over rows A_t, B_t, C_t of a
// sequence, with a state X of (width of A and B) x (width of C):
//   X_t = decay X_{t-1} + B_t^T C_t ,   out_t = A_t X_t
//   outputs             A = q,  B = k,  C = v
//   gradient of q       A = do, B = v,  C = k          (states transposed)
//   gradient of k       A = v,  B = do, C = q, from the last token backwards (transposed)
//   gradient of v       A = k,  B = q,  C = do, from the last token backwards
// The gradient of the states runs backwards with the last two: G_t = scale
// q_t^T do_t + decay G_{t+1}, and the gradient of S0 is decay G_0.
#include "device_common.hpp"
#include "operators.hpp"

namespace lstm355 {

namespace {

template <typename T>
struct Role {
    const T *a, *b, *c;
    T *out;                  // NULL: only the final state is wanted
    long lda, ldb, ldc, ldo;
    int da, dc;              // width of a and b rows, of c and out rows
    bool reverse;
    float intra, inter, update;   // factors of the sum over tokens, of what is left of X0, of the tokens in the final state
    const float *X0;         // state before the first token; element (i, j) at i * si + j * sj of a head's K*M values
    float *XT;
    int si, sj;
};

// decay^n; 0^0 = 1.  `lg` is log2(decay) rounded from 64 bits: log2 of a decay
// near 1 in 32 bits would lose the digits that far distances multiply.
__device__ __forceinline__ float decay_log2(float decay) { return (float)log2((double)decay); }
__device__ __forceinline__ float decay_pow(float lg, int n) { return n == 0 ? 1.0f : exp2f(lg * (float)n); }

__device__ __forceinline__ int sequence_length(const int32_t *lengths, int b, int T)
{
    if (!lengths) return T;
    const int n = lengths[b];
    return n < 0 ? 0 : (n > T ? T : n);
}

// One output row per block, as the sum over its earlier tokens.
template <typename T>
__global__ __launch_bounds__(256) void linattn_rows_kernel(Role<T> r, int Tn, int B, int N, const float *decay,
                                                           const int32_t *lengths)
{
    __shared__ float arow[LINATTN_MAX_WIDTH], score[256];
    const int t = blockIdx.x, b = blockIdx.y / N, h = blockIdx.y % N, tid = threadIdx.x;
    const int n = sequence_length(lengths, b, Tn);
    auto at = [&](int i) { return (long)(r.reverse ? n - 1 - i : i) * B + b; };
    if (t >= n) {
        if (tid < r.dc) r.out[((long)t * B + b) * r.ldo + (long)h * r.dc + tid] = from_f32<T>(0.0f);
        return;
    }
    const float lg = decay_log2(decay[h]);
    if (tid < r.da) arow[tid] = to_f32(r.a[at(t) * r.lda + (long)h * r.da + tid]);
    __syncthreads();
    float acc = 0.0f;
    for (int s0 = 0; s0 <= t; s0 += 256) {
        const int s = s0 + tid;
        if (s <= t) {
            const T *br = r.b + at(s) * r.ldb + (long)h * r.da;
            float d = 0.0f;
            for (int i = 0; i < r.da; ++i) d += arow[i] * to_f32(br[i]);
            score[tid] = d * decay_pow(lg, t - s);
        }
        __syncthreads();
        if (tid < r.dc)
            for (int s = s0; s < s0 + 256 && s <= t; ++s)
                acc += score[s - s0] * to_f32(r.c[at(s) * r.ldc + (long)h * r.dc + tid]);
        __syncthreads();
    }
    if (tid < r.dc) {
        acc *= r.intra;
        if (r.X0) {
            const float *X = r.X0 + (long)blockIdx.y * r.da * r.dc;
            float d = 0.0f;
            for (int i = 0; i < r.da; ++i) d += arow[i] * X[i * r.si + tid * r.sj];
            acc += d * r.inter * decay_pow(lg, t + (r.reverse ? 0 : 1));
        }
        r.out[at(t) * r.ldo + (long)h * r.dc + tid] = from_f32<T>(acc);
    }
}

template <typename T>
__global__ __launch_bounds__(256) void linattn_state_kernel(Role<T> r, int Tn, int B, int N, const float *decay,
                                                            const int32_t *lengths)
{
    const int b = blockIdx.y / N, h = blockIdx.y % N, e = blockIdx.x * 256 + threadIdx.x;
    if (e >= r.da * r.dc) return;
    const int i = e / r.dc, j = e % r.dc;
    const int n = sequence_length(lengths, b, Tn);
    const float lg = decay_log2(decay[h]);
    float acc = 0.0f;
    for (int s = 0; s < n; ++s) {
        const long row = (long)(r.reverse ? n - 1 - s : s) * B + b;
        acc += decay_pow(lg, n - 1 - s + (r.reverse ? 1 : 0)) * to_f32(r.b[row * r.ldb + (long)h * r.da + i]) *
               to_f32(r.c[row * r.ldc + (long)h * r.dc + j]);
    }
    acc *= r.update;
    const long o = (long)blockIdx.y * r.da * r.dc + i * r.si + j * r.sj;
    if (r.X0) acc += decay_pow(lg, n) * r.X0[o];
    r.XT[o] = acc;
}

template <typename T>
hipError_t launch_role(const Role<T> &r, const LinAttnShape &sh, const float *decay, const int32_t *lengths, hipStream_t s)
{
    if (r.out)
        hipLaunchKernelGGL(linattn_rows_kernel<T>, dim3(sh.T, sh.B * sh.N), dim3(256), 0, s, r, sh.T, sh.B, sh.N, decay,
                           lengths);
    if (r.XT)
        hipLaunchKernelGGL(linattn_state_kernel<T>, dim3((r.da * r.dc + 255) / 256, sh.B * sh.N), dim3(256), 0, s, r,
                           sh.T, sh.B, sh.N, decay, lengths);
    return hipGetLastError();
}

// One token of one head per block: the state's rows are read four values per
// thread, M/4 threads to a row, and written back with the token's product.
template <typename T>
__global__ __launch_bounds__(256) void linattn_step_kernel(int B, int N, int K, int M, float scale, const T *q, long ldq,
                                                           const T *k, long ldk, const T *v, long ldv,
                                                           const float *decay, const int32_t *lengths, const float *S,
                                                           float *S_out, T *o, long ldo)
{
    __shared__ float qs[LINATTN_MAX_WIDTH], ks[LINATTN_MAX_WIDTH];
    __shared__ f32x4 part[256];
    const int b = blockIdx.x / N, h = blockIdx.x % N, tid = threadIdx.x;
    const bool on = sequence_length(lengths, b, 1) > 0;
    const float lam = on ? decay[h] : 1.0f;
    if (tid < K) {
        qs[tid] = to_f32(q[(long)b * ldq + (long)h * K + tid]) * scale;
        ks[tid] = to_f32(k[(long)b * ldk + (long)h * K + tid]);
    }
    __syncthreads();
    const int cpr = M / 4, rpp = 256 / cpr;   // threads to a row, rows at a time
    const int c = tid % cpr, r0 = tid / cpr;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    if (r0 < rpp) {
        f32x4 vv = {0.f, 0.f, 0.f, 0.f};
        if (on)
#pragma unroll
            for (int e = 0; e < 4; ++e) vv[e] = to_f32(v[(long)b * ldv + (long)h * M + c * 4 + e]);
        const long base = (long)blockIdx.x * K * M + c * 4;
        for (int r = r0; r < K; r += rpp) {
            f32x4 x = *reinterpret_cast<const f32x4 *>(S + base + (long)r * M);
            if (on) x = lam * x + ks[r] * vv;
            *reinterpret_cast<f32x4 *>(S_out + base + (long)r * M) = x;
            acc += qs[r] * x;
        }
    }
    part[tid] = acc;
    __syncthreads();
    if (tid < cpr) {
        for (int r = 1; r < rpp; ++r) acc += part[r * cpr + tid];
#pragma unroll
        for (int e = 0; e < 4; ++e)
            o[(long)b * ldo + (long)h * M + c * 4 + e] = from_f32<T>(on ? acc[e] : 0.0f);
    }
}

template <typename T>
hipError_t forward_t(const LinAttnShape &sh, const T *q, const T *k, const T *v, const float *decay,
                     const int32_t *lengths, const float *S0, T *o, float *ST, hipStream_t s)
{
    const Role<T> r{q, k, v, o, sh.ldq, sh.ldk, sh.ldv, sh.ldo, sh.K, sh.M, false, sh.scale, sh.scale, 1.0f, S0, ST, sh.M, 1};
    return launch_role(r, sh, decay, lengths, s);
}

template <typename T>
hipError_t backward_t(const LinAttnShape &sh, const T *d_o, const T *q, const T *k, const T *v, const float *decay,
                      const int32_t *lengths, const float *S0, const float *dST, T *dq, T *dk, T *dv, float *dS0,
                      hipStream_t s)
{
    const int K = sh.K, M = sh.M;
    hipError_t e = hipSuccess;
    if (dq) {
        const Role<T> r{d_o, v, k, dq, sh.ldo, sh.ldv, sh.ldk, sh.ldq, M, K, false, sh.scale, sh.scale, 1.0f, S0, nullptr, 1, M};
        e = launch_role(r, sh, decay, lengths, s);
        if (e != hipSuccess) return e;
    }
    if (dk) {
        const Role<T> r{v, d_o, q, dk, sh.ldv, sh.ldo, sh.ldq, sh.ldk, M, K, true, sh.scale, 1.0f, sh.scale, dST, nullptr, 1, M};
        e = launch_role(r, sh, decay, lengths, s);
        if (e != hipSuccess) return e;
    }
    if (dv || dS0) {
        const Role<T> r{k, q, d_o, dv, sh.ldk, sh.ldq, sh.ldo, sh.ldv, K, M, true, sh.scale, 1.0f, sh.scale, dST, dS0, M, 1};
        e = launch_role(r, sh, decay, lengths, s);
    }
    return e;
}

}  // namespace

size_t linattn_workspace_bytes(DType, const LinAttnShape &) { return 0; }

hipError_t linattn_forward(DType t, const LinAttnShape &sh, const void *q, const void *k, const void *v,
                           const float *decay, const int32_t *lengths, const float *S0, void *o, float *ST, void *ws,
                           hipStream_t s)
{
    (void)ws;
    const double n = (double)sh.T * sh.B * sh.N;
    ProfScope ps(K_LINATTN, s, 4.0 * n * sh.K * sh.M, n * 2.0 * (sh.K + sh.M) * dsize(t));
    if (t == DType::BF16)
        return forward_t(sh, static_cast<const bf16_t *>(q), static_cast<const bf16_t *>(k),
                         static_cast<const bf16_t *>(v), decay, lengths, S0, static_cast<bf16_t *>(o), ST, s);
    return forward_t(sh, static_cast<const float *>(q), static_cast<const float *>(k), static_cast<const float *>(v),
                     decay, lengths, S0, static_cast<float *>(o), ST, s);
}

hipError_t linattn_backward(DType t, const LinAttnShape &sh, const void *d_o, const void *q, const void *k,
                            const void *v, const float *decay, const int32_t *lengths, const float *S0,
                            const float *dST, void *dq, void *dk, void *dv, float *dS0, void *ws, hipStream_t s)
{
    (void)ws;
    const double n = (double)sh.T * sh.B * sh.N;
    ProfScope ps(K_LINATTN, s, 10.0 * n * sh.K * sh.M, n * (4.0 * sh.K + 3.0 * sh.M) * dsize(t));
    if (t == DType::BF16)
        return backward_t(sh, static_cast<const bf16_t *>(d_o), static_cast<const bf16_t *>(q),
                          static_cast<const bf16_t *>(k), static_cast<const bf16_t *>(v), decay, lengths, S0, dST,
                          static_cast<bf16_t *>(dq), static_cast<bf16_t *>(dk), static_cast<bf16_t *>(dv), dS0, s);
    return backward_t(sh, static_cast<const float *>(d_o), static_cast<const float *>(q), static_cast<const float *>(k),
                      static_cast<const float *>(v), decay, lengths, S0, dST, static_cast<float *>(dq),
                      static_cast<float *>(dk), static_cast<float *>(dv), dS0, s);
}

hipError_t linattn_step(DType t, const LinAttnShape &sh, const void *q, const void *k, const void *v,
                        const float *decay, const int32_t *lengths, const float *S, float *S_out, void *o,
                        hipStream_t s)
{
    const double n = (double)sh.B * sh.N;
    ProfScope ps(K_LINATTN, s, 4.0 * n * sh.K * sh.M, n * 8.0 * sh.K * sh.M);
    const dim3 grid(sh.B * sh.N);
    if (t == DType::BF16)
        hipLaunchKernelGGL(linattn_step_kernel<bf16_t>, grid, dim3(256), 0, s, sh.B, sh.N, sh.K, sh.M, sh.scale,
                           static_cast<const bf16_t *>(q), sh.ldq, static_cast<const bf16_t *>(k), sh.ldk,
                           static_cast<const bf16_t *>(v), sh.ldv, decay, lengths, S, S_out, static_cast<bf16_t *>(o),
                           sh.ldo);
    else
        hipLaunchKernelGGL(linattn_step_kernel<float>, grid, dim3(256), 0, s, sh.B, sh.N, sh.K, sh.M, sh.scale,
                           static_cast<const float *>(q), sh.ldq, static_cast<const float *>(k), sh.ldk,
                           static_cast<const float *>(v), sh.ldv, decay, lengths, S, S_out, static_cast<float *>(o),
                           sh.ldo);
    return hipGetLastError();
}

}  // namespace lstm355
