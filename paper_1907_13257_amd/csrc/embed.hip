// embed.hip -- rows of an embedding picked by tokens, and the gradient of the
// table as sums over the tokens sorted by row.
#include "device_common.hpp"
#include "operators.hpp"

namespace lstm355 {

namespace {

template <typename T> constexpr int VEC = 16 / (int)sizeof(T);   // elements of a 16-byte access

template <typename T>
__device__ __forceinline__ void unpack(u32x4 v, float (&f)[VEC<T>])
{
    T e[VEC<T>];
    __builtin_memcpy(e, &v, 16);
#pragma unroll
    for (int i = 0; i < VEC<T>; ++i) f[i] = to_f32(e[i]);
}

template <typename T>
__device__ __forceinline__ u32x4 pack(const float (&f)[VEC<T>])
{
    T e[VEC<T>];
#pragma unroll
    for (int i = 0; i < VEC<T>; ++i) e[i] = from_f32<T>(f[i]);
    u32x4 v;
    __builtin_memcpy(&v, e, 16);
    return v;
}

// Lanes that share a row: the power of two that covers its vectors, 64 at most.
int lanes_per_row(int nv)
{
    int l = 1;
    while (l < 64 && l < nv) l *= 2;
    return l;
}

// out[n] = scale * table[ids[n]]; `lpr` lanes per row, one row after another.
template <typename T>
__global__ __launch_bounds__(256) void embed_forward_kernel(long N, long V, int nv, const int64_t *__restrict__ ids,
                                                            const T *__restrict__ table, float scale,
                                                            T *__restrict__ out, long ldo, int lpr)
{
    const int rpb = 256 / lpr, col = threadIdx.x % lpr;
    for (long n = (long)blockIdx.x * rpb + threadIdx.x / lpr; n < N; n += (long)gridDim.x * rpb) {
        const int64_t id = ids[n];
        const bool in = id >= 0 && id < V;
        const T *src = table + (in ? id : 0) * (long)nv * VEC<T>;
        T *dst = out + n * ldo;
        for (int c = col; c < nv; c += lpr) {
            float f[VEC<T>];
            unpack<T>(in ? ldg16(src + (long)c * VEC<T>) : zero16(), f);
#pragma unroll
            for (int e = 0; e < VEC<T>; ++e) f[e] *= scale;
            *reinterpret_cast<u32x4 *>(dst + (long)c * VEC<T>) = in ? pack<T>(f) : zero16();
        }
    }
}

// ---------------------------------------------------------------------------
// The tokens sorted by table row, position by position within a row: a stable
// radix sort of (row, position), least significant digit first.  The key of a
// token outside the table is V, behind every row.  A pass is a count of each
// block's digits and a scatter; a block owns `span` consecutive tokens.
// ---------------------------------------------------------------------------
constexpr int SORT_TILE = 1024;        // tokens sorted at a time by a block, one per thread
constexpr int SORT_MAX_BLOCKS = 256;
constexpr int SORT_MAX_BITS = 11;      // of a digit: 2048 counters per wave of the block, 64 KiB of LDS

struct SortPlan {
    int bits, passes, blocks;
    long span;
};

SortPlan sort_plan(long N, long V)
{
    SortPlan p;
    int keybits = 0;
    while (keybits < 32 && (V >> keybits)) ++keybits;   // keys are 0 .. V
    p.passes = (keybits + SORT_MAX_BITS - 1) / SORT_MAX_BITS;
    if (p.passes < 1) p.passes = 1;
    p.bits = (keybits + p.passes - 1) / p.passes;
    const long tiles = (N + SORT_TILE - 1) / SORT_TILE;
    const long per = (tiles + SORT_MAX_BLOCKS - 1) / SORT_MAX_BLOCKS;
    p.span = (per < 1 ? 1 : per) * SORT_TILE;
    p.blocks = (int)((N + p.span - 1) / p.span);
    return p;
}

__device__ __forceinline__ unsigned token_key(const int64_t *ids, const unsigned *keys, long i, long V)
{
    if (keys) return keys[i];
    const int64_t id = ids[i];
    return id >= 0 && id < V ? (unsigned)id : (unsigned)V;
}

__global__ __launch_bounds__(SORT_TILE) void sort_count_kernel(long N, long V, const int64_t *__restrict__ ids,
                                                               const unsigned *__restrict__ keys, int shift, int bits,
                                                               long span, int *__restrict__ hist)
{
    __shared__ int cnt[1 << SORT_MAX_BITS];
    const int bins = 1 << bits;
    for (int b = threadIdx.x; b < bins; b += SORT_TILE) cnt[b] = 0;
    __syncthreads();
    const long i0 = blockIdx.x * span, i1 = min(N, i0 + span);
    for (long i = i0 + threadIdx.x; i < i1; i += SORT_TILE)
        atomicAdd(&cnt[(token_key(ids, keys, i, V) >> shift) & (bins - 1)], 1);
    __syncthreads();
    for (int b = threadIdx.x; b < bins; b += SORT_TILE) hist[(long)b * gridDim.x + blockIdx.x] = cnt[b];
}

__global__ __launch_bounds__(SORT_TILE) void sort_scatter_kernel(long N, long V, const int64_t *__restrict__ ids,
                                                                 const unsigned *__restrict__ keys,
                                                                 const int *__restrict__ pos, int shift, int bits,
                                                                 long span, const int *__restrict__ hist,
                                                                 unsigned *__restrict__ keys_out,
                                                                 int *__restrict__ pos_out)
{
    constexpr int WAVES = SORT_TILE / 64;
    __shared__ unsigned short in_wave[WAVES][1 << SORT_MAX_BITS];   // per wave: counts, then counts of earlier waves
    __shared__ int base[1 << SORT_MAX_BITS];                         // next place of each digit
    __shared__ int sums[WAVES];
    const int bins = 1 << bits, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int nb = gridDim.x;

    // this block's first place of each digit: all smaller digits, and the
    // digit's tokens in earlier blocks.  Thread t takes digits 2t and 2t + 1.
    int total[2] = {0, 0}, before[2] = {0, 0};
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int b = 2 * tid + j;
        if (b < bins)
            for (int k = 0; k < nb; ++k) {
                const int c = hist[(long)b * nb + k];
                total[j] += c;
                if (k < (int)blockIdx.x) before[j] += c;
            }
    }
    int run = total[0] + total[1];
    for (int d = 1; d < 64; d *= 2) {
        const int o = __shfl_up(run, d);
        if (lane >= d) run += o;
    }
    if (lane == 63) sums[wave] = run;
    __syncthreads();
    for (int w = 0; w < wave; ++w) run += sums[w];
    const int first = run - total[0] - total[1];
    if (2 * tid < bins) base[2 * tid] = first + before[0];
    if (2 * tid + 1 < bins) base[2 * tid + 1] = first + total[0] + before[1];

    const long i0 = blockIdx.x * span, i1 = min(N, i0 + span);
    for (long t0 = i0; t0 < i1; t0 += SORT_TILE) {
        for (int e = tid; e < WAVES * bins; e += SORT_TILE) in_wave[e >> bits][e & (bins - 1)] = 0;
        __syncthreads();
        const long i = t0 + tid;
        const bool on = i < i1;
        const unsigned key = on ? token_key(ids, keys, i, V) : 0u;
        const int digit = (key >> shift) & (bins - 1);
        // lanes of this wave with the same digit
        unsigned long long same = __ballot(on);
        for (int b = 0; b < bits; ++b) {
            const bool set = (digit >> b) & 1;
            const unsigned long long m = __ballot(set);
            same &= set ? m : ~m;
        }
        const int rank = __popcll(same & ((1ull << lane) - 1));
        if (on && rank == 0) in_wave[wave][digit] = (unsigned short)__popcll(same);
        __syncthreads();
        int add[2] = {0, 0};
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int b = 2 * tid + j;
            if (b < bins)
                for (int w = 0; w < WAVES; ++w) {
                    const int c = in_wave[w][b];
                    in_wave[w][b] = (unsigned short)add[j];
                    add[j] += c;
                }
        }
        __syncthreads();
        if (on) {
            const int at = base[digit] + in_wave[wave][digit] + rank;
            keys_out[at] = key;
            pos_out[at] = pos ? pos[i] : (int)i;
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 2; ++j)
            if (2 * tid + j < bins) base[2 * tid + j] += add[j];
    }
}

// ---------------------------------------------------------------------------
// Sums over the sorted tokens.  Equal rows are neighbours, so each run of RUN
// sorted tokens is summed by one group of threads, whatever the frequencies:
// a row whose tokens lie within one run is final, a row that reaches over runs
// leaves a partial sum per run (the first of a run's two slots if it came from
// the run before, else the second), which embed_combine_kernel adds in order.
// ---------------------------------------------------------------------------
constexpr int RUN = 16;

template <typename T>
__global__ __launch_bounds__(256) void embed_runs_kernel(long N, long V, int nv, const unsigned *__restrict__ keys,
                                                         const int *__restrict__ pos, const T *__restrict__ dout,
                                                         long ldo, float scale, float *__restrict__ dtable,
                                                         int accumulate, float *__restrict__ partial, int tpr)
{
    const long D = (long)nv * VEC<T>, nruns = (N + RUN - 1) / RUN;
    const long r = (long)blockIdx.x * (256 / tpr) + threadIdx.x / tpr;
    if (r >= nruns) return;
    const long i0 = r * RUN, i1 = min(N, i0 + RUN);
    const unsigned none = (unsigned)V;
    const unsigned prev = i0 > 0 ? keys[i0 - 1] : none, next = i1 < N ? keys[i1] : none;
    for (int c = blockIdx.y * tpr + threadIdx.x % tpr; c < nv; c += gridDim.y * tpr) {
        float acc[VEC<T>];
#pragma unroll
        for (int e = 0; e < VEC<T>; ++e) acc[e] = 0.0f;
        unsigned cur = keys[i0];
        bool head = cur == prev;
        auto flush = [&](bool more) {
            if (cur >= none) return;
            if (head || more) {
                float *p = partial + (2 * r + (head ? 0 : 1)) * D + (long)c * VEC<T>;
#pragma unroll
                for (int e = 0; e < VEC<T>; ++e) p[e] = acc[e];
                return;
            }
            float *p = dtable + (long)cur * D + (long)c * VEC<T>;
#pragma unroll
            for (int e = 0; e < VEC<T>; ++e) p[e] = accumulate ? p[e] + scale * acc[e] : scale * acc[e];
        };
        for (long i = i0; i < i1; ++i) {
            const unsigned k = keys[i];
            if (k != cur) {
                flush(false);
                cur = k;
                head = false;
#pragma unroll
                for (int e = 0; e < VEC<T>; ++e) acc[e] = 0.0f;
            }
            if (k >= none) break;   // the tokens outside the table are the last
            float f[VEC<T>];
            unpack<T>(ldg16(dout + (long)pos[i] * ldo + (long)c * VEC<T>), f);
#pragma unroll
            for (int e = 0; e < VEC<T>; ++e) acc[e] += f[e];
        }
        flush(cur == next);
    }
}

// Rows that reach over several runs: the block of the run a row starts in adds
// its partial sums, a quarter of them per group of 64 lanes.
__global__ __launch_bounds__(256) void embed_combine_kernel(long N, long V, int D, const unsigned *__restrict__ keys,
                                                            const float *__restrict__ partial, float scale,
                                                            float *__restrict__ dtable, int accumulate)
{
    __shared__ f32x4 part[4][64];
    const long r = blockIdx.x, i0 = r * RUN, i1 = i0 + RUN;
    if (i1 >= N) return;
    const unsigned key = keys[i1 - 1];
    if (key >= (unsigned)V || keys[i1] != key) return;             // the last row of the run ends with it
    if (i0 > 0 && keys[i0] == key && keys[i0 - 1] == key) return;  // it started in an earlier run
    const long nruns = (N + RUN - 1) / RUN;
    long lo = r + 1, hi = nruns;   // the last run that starts with the row: in [lo, hi)
    while (hi - lo > 1) {
        const long mid = (lo + hi) / 2;
        if (keys[mid * RUN] == key) lo = mid; else hi = mid;
    }
    const long n = lo - r + 1, per = (n + 3) / 4;   // partial sums in all, and of a group
    const int lane = threadIdx.x & 63, grp = threadIdx.x >> 6;
    const int c = (blockIdx.y * 64 + lane) * 4;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    if (c < D)
        for (long j = grp * per; j < min(n, (grp + 1) * per); ++j)
            acc += *reinterpret_cast<const f32x4 *>(partial + (j == 0 ? 2 * r + 1 : 2 * (r + j)) * D + c);
    part[grp][lane] = acc;
    __syncthreads();
    if (grp == 0 && c < D) {
        acc = (part[0][lane] + part[1][lane]) + (part[2][lane] + part[3][lane]);
        f32x4 *p = reinterpret_cast<f32x4 *>(dtable + (long)key * D + c);
        *p = accumulate ? *p + scale * acc : scale * acc;
    }
}

struct EmbedWs {
    size_t keys[2], pos[2], hist, partial, total;
};

EmbedWs embed_ws(long N, long V, int D)
{
    const SortPlan p = sort_plan(N, V);
    EmbedWs w;
    size_t o = 0;
    auto take = [&](size_t bytes) {
        const size_t at = o;
        o = (o + bytes + 255) & ~(size_t)255;
        return at;
    };
    for (int i = 0; i < 2; ++i) {
        w.keys[i] = take((size_t)N * 4);
        w.pos[i] = take((size_t)N * 4);
    }
    w.hist = take(((size_t)1 << p.bits) * p.blocks * 4);
    w.partial = take((size_t)((N + RUN - 1) / RUN) * 2 * D * 4);
    w.total = o;
    return w;
}

template <typename T>
hipError_t embed_backward_t(long N, long V, int D, const int64_t *ids, const T *dout, long ldo, float scale,
                            float *dtable, int accumulate, char *ws, hipStream_t s)
{
    if (!accumulate) {
        const hipError_t e = fill_u32(dtable, (size_t)V * D, 0u, s);
        if (e != hipSuccess) return e;
    }
    if (N == 0) return hipSuccess;
    const EmbedWs w = embed_ws(N, V, D);
    const SortPlan p = sort_plan(N, V);
    unsigned *keys[2] = {reinterpret_cast<unsigned *>(ws + w.keys[0]), reinterpret_cast<unsigned *>(ws + w.keys[1])};
    int *pos[2] = {reinterpret_cast<int *>(ws + w.pos[0]), reinterpret_cast<int *>(ws + w.pos[1])};
    int *hist = reinterpret_cast<int *>(ws + w.hist);
    float *partial = reinterpret_cast<float *>(ws + w.partial);
    const unsigned *ksrc = nullptr;
    const int *psrc = nullptr;
    int to = 0;
    for (int k = 0; k < p.passes; ++k, to ^= 1) {
        hipLaunchKernelGGL(sort_count_kernel, dim3(p.blocks), dim3(SORT_TILE), 0, s, N, V, ids, ksrc, k * p.bits,
                           p.bits, p.span, hist);
        hipLaunchKernelGGL(sort_scatter_kernel, dim3(p.blocks), dim3(SORT_TILE), 0, s, N, V, ids, ksrc, psrc,
                           k * p.bits, p.bits, p.span, hist, keys[to], pos[to]);
        ksrc = keys[to];
        psrc = pos[to];
    }
    const int nv = D / VEC<T>;
    int tpr = lanes_per_row(nv);
    while (tpr < 256 && tpr < nv) tpr *= 2;
    const long nruns = (N + RUN - 1) / RUN;
    const int rpb = 256 / tpr;
    hipLaunchKernelGGL(embed_runs_kernel<T>, dim3((unsigned)((nruns + rpb - 1) / rpb), (nv + tpr - 1) / tpr), dim3(256), 0,
                       s, N, V, nv, ksrc, psrc, dout, ldo, scale, dtable, accumulate, partial, tpr);
    hipLaunchKernelGGL(embed_combine_kernel, dim3((unsigned)nruns, (D + 255) / 256), dim3(256), 0, s, N, V, D, ksrc,
                       partial, scale, dtable, accumulate);
    return hipGetLastError();
}

}  // namespace

hipError_t embed_forward(DType t, long N, long V, int D, const int64_t *ids, const void *table, float scale, void *out,
                         long ldo, hipStream_t s)
{
    if (N == 0) return hipSuccess;
    ProfScope ps(K_EMBED, s, 0.0, (double)N * (2.0 * D * dsize(t) + 8));
    const int nv = D * (int)dsize(t) / 16, lpr = lanes_per_row(nv), rpb = 256 / lpr;
    const long need = (N + rpb - 1) / rpb;
    const dim3 grid((unsigned)(need < 65536 ? need : 65536));
    if (t == DType::BF16)
        hipLaunchKernelGGL(embed_forward_kernel<bf16_t>, grid, dim3(256), 0, s, N, V, nv, ids,
                           static_cast<const bf16_t *>(table), scale, static_cast<bf16_t *>(out), ldo, lpr);
    else
        hipLaunchKernelGGL(embed_forward_kernel<float>, grid, dim3(256), 0, s, N, V, nv, ids,
                           static_cast<const float *>(table), scale, static_cast<float *>(out), ldo, lpr);
    return hipGetLastError();
}

size_t embed_workspace_bytes(long N, long V, int D) { return N > 0 ? embed_ws(N, V, D).total : 0; }

hipError_t embed_backward(DType t, long N, long V, int D, const int64_t *ids, const void *dout, long ldo, float scale,
                          float *dtable, int accumulate, void *ws, hipStream_t s)
{
    ProfScope ps(K_EMBED, s, (double)N * D, (double)N * D * dsize(t) + (accumulate ? 0.0 : 4.0 * V * D));
    if (t == DType::BF16)
        return embed_backward_t(N, V, D, ids, static_cast<const bf16_t *>(dout), ldo, scale, dtable, accumulate,
                                static_cast<char *>(ws), s);
    return embed_backward_t(N, V, D, ids, static_cast<const float *>(dout), ldo, scale, dtable, accumulate,
                            static_cast<char *>(ws), s);
}

}  // namespace lstm355
