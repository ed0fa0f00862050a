// norm.hip -- residual addition and root-mean-square norm of rows, its 8-bit
// output, and its gradient.
#include "device_common.hpp"
#include "operators.hpp"

namespace lstm355 {

namespace {

template <typename T>
__device__ __forceinline__ void load_vec(const T *p, float (&f)[VEC<T>]) { unpack<T>(ldg16(p), f); }
template <typename T>
__device__ __forceinline__ void store_vec(T *p, const float (&f)[VEC<T>]) { *reinterpret_cast<u32x4 *>(p) = pack<T>(f); }

// 8 (bf16 storage) or 4 (fp32) values as e4m3 bytes, round to nearest even.
__device__ __forceinline__ unsigned e4m3x4(float a, float b, float c, float d)
{
    int v = 0;
    v = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, v, false);
    v = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, v, true);
    return (unsigned)v;
}

struct Sum2 { float a, b; };

// Sums (a) and sums or maxima (b) over the W waves of a block, in a fixed
// order; every thread gets both.  `red` holds 2 W floats.
template <int W, bool MAXB>
__device__ __forceinline__ Sum2 reduce_row(Sum2 v, float *red)
{
#pragma unroll
    for (int d = 32; d > 0; d /= 2) {
        v.a += __shfl_xor(v.a, d);
        const float o = __shfl_xor(v.b, d);
        v.b = MAXB ? fmaxf(v.b, o) : v.b + o;
    }
    if constexpr (W > 1) {
        const int wave = threadIdx.x >> 6;
        __syncthreads();   // the previous row's values have been read
        if ((threadIdx.x & 63) == 0) {
            red[2 * wave] = v.a;
            red[2 * wave + 1] = v.b;
        }
        __syncthreads();
        v = Sum2{red[0], red[1]};
#pragma unroll
        for (int w = 1; w < W; ++w) {
            v.a += red[2 * w];
            v.b = MAXB ? fmaxf(v.b, red[2 * w + 1]) : v.b + red[2 * w + 1];
        }
    }
    return v;
}

// A thread's squares (32 at most) are summed as they are, a row's as a 64th: 16384
// squares of 1e18 are beyond fp32.  A power of two changes no digit.
constexpr float SQUARES = 0x1p-6f;
__device__ __forceinline__ float inverse_root(float squares, int D, float eps)   // 1 / sqrt(mean + eps)
{
    return rsqrtf(squares / ((float)D * SQUARES) + eps);
}

// A row is held in registers by W waves, P vectors per thread (thread t has
// vectors t, t + 64 W, ...), so it is read once and both sums over it need no
// second pass.  A block has four rows where a row is one wave's, else one.
// Bound by memory: 6400 rows of 1024 bf16 in 10.2 us (52 MB, 5.1 TB/s), 20001 of
// 8192 with the 8-bit output in 213 us (1.15 GB, 5.4 TB/s); 16 rows in 3.6 us.
template <int W> constexpr int ROWS = W == 1 ? 4 : 1;
template <int W> constexpr int THREADS = W == 1 ? 256 : W * 64;

template <typename T, int W, int P, bool Q8>
__global__ __launch_bounds__(THREADS<W>) void add_norm_kernel(NormArgs a, int nv)
{
    __shared__ float red[2 * W];
    constexpr int E = VEC<T>;
    const int tid = W == 1 ? threadIdx.x & 63 : threadIdx.x;
    for (long row = (long)blockIdx.x * ROWS<W> + (W == 1 ? threadIdx.x >> 6 : 0); row < a.rows;
         row += (long)gridDim.x * ROWS<W>) {
        const T *x = static_cast<const T *>(a.x) + row * a.ldx;
        const T *res = a.res ? static_cast<const T *>(a.res) + row * a.ldr : nullptr;
        T *sum = a.sum ? static_cast<T *>(a.sum) + row * a.ldr : nullptr;
        const T *g = static_cast<const T *>(a.g);
        float s[P][E];
        Sum2 r{0.0f, 0.0f};
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const int c = tid + p * 64 * W;
            if (c < nv) {
                load_vec<T>(x + (long)c * E, s[p]);
                if (res) {
                    float o[E];
                    load_vec<T>(res + (long)c * E, o);
#pragma unroll
                    for (int e = 0; e < E; ++e) s[p][e] = to_f32(from_f32<T>(s[p][e] + o[e]));
                }
                if (sum) store_vec<T>(sum + (long)c * E, s[p]);
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e) s[p][e] = 0.0f;
            }
#pragma unroll
            for (int e = 0; e < E; ++e) r.a += s[p][e] * s[p][e];
            if (c < nv) {
                float gv[E];
                load_vec<T>(g + (long)c * E, gv);
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    s[p][e] *= gv[e];
                    if (Q8) r.b = fmaxf(r.b, fabsf(s[p][e]));
                }
            }
        }
        r.a *= SQUARES;
        r = reduce_row<W, true>(r, red);
        const float rho = inverse_root(r.a, nv * E, a.eps);
        if constexpr (Q8) {
            // y / scale = (sum g) 448 / max|sum g|: the norm's factor cancels.
            // Where the maximum is so small that the quotient could overflow or
            // the products have lost digits, the row is taken again from what is
            // stored, 2^112 times as large; what is below 2^-119 then has a scale
            // of 0 in fp32.
            float down = 1.0f;
            if (r.b < 0x1p-64f) {
                const T *from = sum ? sum : x;
                Sum2 m{0.0f, 0.0f};
#pragma unroll
                for (int p = 0; p < P; ++p) {
                    const int c = tid + p * 64 * W;
                    if (c >= nv) continue;
                    float gv[E];
                    load_vec<T>(from + (long)c * E, s[p]);
                    load_vec<T>(g + (long)c * E, gv);
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        s[p][e] = s[p][e] * 0x1p64f * gv[e] * 0x1p48f;
                        m.b = fmaxf(m.b, fabsf(s[p][e]));
                    }
                }
                r.b = reduce_row<W, true>(m, red).b;
                down = 0x1p-112f;
            }
            const bool some = !(r.b < 0x1p-119f);
            const float inv = some ? 448.0f / r.b : 0.0f;
            uint8_t *y = static_cast<uint8_t *>(a.y) + row * (long)nv * E;
#pragma unroll
            for (int p = 0; p < P; ++p) {
                const int c = tid + p * 64 * W;
                if (c >= nv) continue;
                unsigned w[E / 4];
#pragma unroll
                for (int q = 0; q < E / 4; ++q)
                    w[q] = e4m3x4(s[p][4 * q] * inv, s[p][4 * q + 1] * inv, s[p][4 * q + 2] * inv, s[p][4 * q + 3] * inv);
                __builtin_memcpy(y + (long)c * E, w, E);
            }
            if (tid == 0) a.scale[row] = some ? r.b * rho / 448.0f * down : r.a * 0.0f;   // NaN if the sum is
        } else {
            T *y = static_cast<T *>(a.y) + row * a.ldy;
#pragma unroll
            for (int p = 0; p < P; ++p) {
                const int c = tid + p * 64 * W;
                if (c >= nv) continue;
#pragma unroll
                for (int e = 0; e < E; ++e) s[p][e] *= rho;
                store_vec<T>(y + (long)c * E, s[p]);
            }
        }
    }
}

// dx = dsum + rho (g dy - s rho rho mean(g dy s)), the root's factors apart: their
// cube leaves fp32 for rows beyond 1e13 or (eps = 0) below 1e-13.  A block adds
// dy s rho of its rows (a fixed set) in registers and leaves its sums in `partial`.
// Bound by memory: 6400 rows of 1024 bf16 in 12.8 us (52 MB needed, 4.1 TB/s).
template <typename T, int W, int P>
__global__ __launch_bounds__(THREADS<W>) void add_norm_backward_kernel(NormBwdArgs a, int nv)
{
    __shared__ float red[2 * W];
    constexpr int E = VEC<T>;
    const int tid = W == 1 ? threadIdx.x & 63 : threadIdx.x;
    float dg[P][E], gv[P][E];
#pragma unroll
    for (int p = 0; p < P; ++p) {
        const int c = tid + p * 64 * W;
#pragma unroll
        for (int e = 0; e < E; ++e) dg[p][e] = gv[p][e] = 0.0f;
        if (c < nv) load_vec<T>(static_cast<const T *>(a.g) + (long)c * E, gv[p]);
    }
    for (long row = (long)blockIdx.x * ROWS<W> + (W == 1 ? threadIdx.x >> 6 : 0); row < a.rows;
         row += (long)gridDim.x * ROWS<W>) {
        const T *dy = static_cast<const T *>(a.dy) + row * a.ldy;
        const T *sum = static_cast<const T *>(a.sum) + row * a.ldr;
        const T *ds = a.dsum ? static_cast<const T *>(a.dsum) + row * a.ldr : nullptr;
        float s[P][E], d[P][E], u[P][E];
        Sum2 r{0.0f, 0.0f};
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const int c = tid + p * 64 * W;
#pragma unroll
            for (int e = 0; e < E; ++e) s[p][e] = d[p][e] = u[p][e] = 0.0f;
            if (c >= nv) continue;
            load_vec<T>(sum + (long)c * E, s[p]);
            load_vec<T>(dy + (long)c * E, d[p]);
            if (ds) load_vec<T>(ds + (long)c * E, u[p]);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                r.a += s[p][e] * s[p][e];
                r.b += gv[p][e] * d[p][e] * s[p][e];
            }
        }
        r.a *= SQUARES;
        r = reduce_row<W, false>(r, red);
        const float rho = inverse_root(r.a, nv * E, a.eps);
        const float k = rho * (rho * (r.b / (float)(nv * E)));
        T *dx = static_cast<T *>(a.dx) + row * a.ldx;
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const int c = tid + p * 64 * W;
            if (c >= nv) continue;
            float o[E];
#pragma unroll
            for (int e = 0; e < E; ++e) {
                o[e] = u[p][e] + rho * (gv[p][e] * d[p][e] - s[p][e] * k);
                dg[p][e] += d[p][e] * s[p][e] * rho;
            }
            store_vec<T>(dx + (long)c * E, o);
        }
    }
    // one row of sums per block: its waves' rows in order
    const long D = (long)nv * E;
    if constexpr (W == 1) {
        __shared__ float sums[ROWS<W>][64 * P * E];
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int e = 0; e < E; ++e) sums[threadIdx.x >> 6][(tid + p * 64) * E + e] = dg[p][e];
        __syncthreads();
        for (int c = threadIdx.x; c < D; c += THREADS<W>)
            a.partial[blockIdx.x * D + c] = (sums[0][c] + sums[1][c]) + (sums[2][c] + sums[3][c]);
    } else {
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const int c = tid + p * 64 * W;
            if (c >= nv) continue;
#pragma unroll
            for (int e = 0; e < E; e += 4)
                *reinterpret_cast<f32x4 *>(a.partial + blockIdx.x * D + (long)c * E + e) =
                    f32x4{dg[p][e], dg[p][e + 1], dg[p][e + 2], dg[p][e + 3]};
        }
    }
}

// dg (+)= the sum of the blocks' rows: 32 groups of 16 lanes take every 32nd
// row of 64 columns, and their sums are added in order.  3.9 us for 1024
// columns, the latency of a launch and 16 loads; one thread per column took 234.
__global__ __launch_bounds__(512) void norm_gain_kernel(const float *__restrict__ partial, int rows, int D,
                                                        float *__restrict__ dg, int accumulate)
{
    __shared__ f32x4 part[32][16];
    const int lane = threadIdx.x & 15, grp = threadIdx.x >> 4, c = (blockIdx.x * 16 + lane) * 4;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    if (c < D)
#pragma unroll 8
        for (int r = grp; r < rows; r += 32) acc += *reinterpret_cast<const f32x4 *>(partial + (long)r * D + c);
    part[grp][lane] = acc;
    __syncthreads();
    if (grp == 0 && c < D) {
        f32x4 *p = reinterpret_cast<f32x4 *>(dg + c);
        acc = accumulate ? *p : f32x4{0.f, 0.f, 0.f, 0.f};
        f32x4 sum = part[0][lane];
        for (int k = 1; k < 32; ++k) sum += part[k][lane];
        *p = accumulate ? acc + sum : sum;
    }
}

// Blocks of the backward pass, each of which leaves one row of partial sums.
// Forward and backward with 256, 512, 1024 blocks: 6400 rows of 1024 33.5, 28.4,
// 28.9 us, of 4096 110, 86, 86, 40000 rows of 1024 150, 126, 129.
constexpr int BWD_BLOCKS = 512;

int bwd_blocks(long rows, int rows_per_block)
{
    const long need = (rows + rows_per_block - 1) / rows_per_block;
    return (int)(need < BWD_BLOCKS ? need : BWD_BLOCKS);
}

template <typename T, int W, int P>
hipError_t launch_norm(const NormArgs &a, hipStream_t s)
{
    const int nv = a.D / VEC<T>;
    const long need = (a.rows + ROWS<W> - 1) / ROWS<W>;
    const dim3 grid((unsigned)(need < 65536 ? need : 65536)), block(THREADS<W>);
    if (a.scale)
        hipLaunchKernelGGL((add_norm_kernel<T, W, P, true>), grid, block, 0, s, a, nv);
    else
        hipLaunchKernelGGL((add_norm_kernel<T, W, P, false>), grid, block, 0, s, a, nv);
    return hipGetLastError();
}

template <typename T, int W, int P>
hipError_t launch_norm_bwd(const NormBwdArgs &a, hipStream_t s)
{
    const int blocks = bwd_blocks(a.rows, ROWS<W>);
    hipLaunchKernelGGL((add_norm_backward_kernel<T, W, P>), dim3(blocks), dim3(THREADS<W>), 0, s, a, a.D / VEC<T>);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(norm_gain_kernel, dim3((a.D + 63) / 64), dim3(512), 0, s, a.partial, blocks, a.D, a.dg,
                       a.accumulate);
    return hipGetLastError();
}

// Waves and vectors per thread of a row of nv vectors: one wave as long as it
// has the row in two vectors per lane, since four waves meet at barriers and a
// quarter of a wave's rows are in flight.  6400 rows forward and backward with
// one wave and with four: 1024 bf16 (128 vectors) 28 and 39 us, 2048 56 and 51,
// 4096 147 and 86.
#define NORM_BY_WIDTH(CALL)                    \
    if (nv <= 64) return CALL(1, 1);           \
    if (nv <= 128) return CALL(1, 2);          \
    if (nv <= 256) return CALL(4, 1);          \
    if (nv <= 512) return CALL(4, 2);          \
    if (nv <= 1024) return CALL(4, 4);         \
    if constexpr (NORM_MAX_D / VEC<T> > 2048)  \
        if (nv > 2048) return CALL(16, 4);     \
    return CALL(8, 4);

template <typename T>
hipError_t add_norm_t(const NormArgs &a, hipStream_t s)
{
    const int nv = a.D / VEC<T>;
#define CALL(W, P) launch_norm<T, W, P>(a, s)
    NORM_BY_WIDTH(CALL)
#undef CALL
}

template <typename T>
hipError_t add_norm_backward_t(const NormBwdArgs &a, hipStream_t s)
{
    const int nv = a.D / VEC<T>;
#define CALL(W, P) launch_norm_bwd<T, W, P>(a, s)
    NORM_BY_WIDTH(CALL)
#undef CALL
}

}  // namespace

hipError_t add_norm(DType t, const NormArgs &a, hipStream_t s)
{
    if (a.rows == 0) return hipSuccess;
    const double n = (double)a.rows * a.D;
    ProfScope ps(K_NORM, s, 0.0, n * (dsize(t) * (1.0 + (a.res ? 1 : 0) + (a.sum ? 1 : 0)) + (a.scale ? 1 : dsize(t))));
    return t == DType::BF16 ? add_norm_t<bf16_t>(a, s) : add_norm_t<float>(a, s);
}

size_t norm_partial_floats(long rows, int D) { return (size_t)(rows < BWD_BLOCKS ? rows : BWD_BLOCKS) * D; }

hipError_t add_norm_backward(DType t, const NormBwdArgs &a, hipStream_t s)
{
    const double n = (double)a.rows * a.D;
    if (a.rows == 0) return a.accumulate ? hipSuccess : fill_u32(a.dg, a.D, 0u, s);
    ProfScope ps(K_NORM, s, 0.0, n * dsize(t) * (a.dsum ? 4.0 : 3.0));
    return t == DType::BF16 ? add_norm_backward_t<bf16_t>(a, s) : add_norm_backward_t<float>(a, s);
}

}  // namespace lstm355
