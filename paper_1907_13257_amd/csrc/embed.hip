// embed.hip -- rows of an embedding picked by tokens, and the gradient of the
// table as sums over the tokens sorted by row.
#include "device_common.hpp"
#include "operators.hpp"

namespace lstm355 {

namespace {

// Lanes that share a row: the power of two that covers its vectors, 64 at most.
int lanes_per_row(int nv)
{
    int l = 1;
    while (l < 64 && l < nv) l *= 2;
    return l;
}

// out[n] = scale * table[ids[n]]; `lpr` lanes per row, one row after another, 16
// bytes a lane.  Bound by memory: 40000 rows of 1024 bf16 in 28 to 32 us (164 MB, of
// which 127 reach memory, at 4.0 TB/s), 6400 in 4.4 to 5.7; 16 rows in 2.1 us, a
// launch's latency.
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
// The tokens sorted by table row, position by position within a row.  The key
// of a token outside the table is V, behind every row.  Every launch of the
// sort takes a share of the work beside it that needs no order: the zeros of an
// overwritten gradient, written by blocks behind the sorting ones, so that the
// sort's few blocks and their latency hide behind those stores (6400 tokens and
// 32000 rows of 1024: 22 us, the 131 MB of zeros at 6.0 TB/s; zeros and a radix
// sort one after the other took 18 and 17 us).
// ---------------------------------------------------------------------------
constexpr int SORT_TILE = 1024;        // threads of a sorting block, tokens sorted at a time

struct Fill {
    f32x4 *p;
    long n;      // zeros p[0 .. n)
    int first;   // number of sorting blocks
};

// Whether this block writes zeros (and has).
__device__ __forceinline__ bool fill_block(const Fill &f)
{
    if ((int)blockIdx.x < f.first) return false;
    const long step = (long)(gridDim.x - f.first) * SORT_TILE;
    for (long i = (long)(blockIdx.x - f.first) * SORT_TILE + threadIdx.x; i < f.n; i += step)
        f.p[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    return true;
}

__device__ __forceinline__ unsigned token_key(const int64_t *ids, const unsigned *keys, long i, long V)
{
    if (keys) return keys[i];
    const int64_t id = ids[i];
    return id >= 0 && id < V ? (unsigned)id : (unsigned)V;
}

// Few tokens: a token's place is the number of keys before its own, counted
// outright.  A block places 64 tokens, one per lane; each of its 16 waves
// compares them with a sixteenth of all keys.  One launch instead of four, but
// the square of the tokens: a gradient of 6400 tokens (1024 columns) in 50 us
// and with the radix sort in 62, of 8192 (64 columns) in 37.0 and 38.3; the keys
// of more would not fit the 32 KiB either.
constexpr int RANK_MAX = 8192;
__global__ __launch_bounds__(SORT_TILE) void rank_kernel(int N, long V, const int64_t *__restrict__ ids,
                                                         unsigned *__restrict__ keys_out, int *__restrict__ pos_out,
                                                         Fill fill)
{
    __shared__ __align__(16) unsigned keys[RANK_MAX];
    __shared__ int counts[16][64];
    if (fill_block(fill)) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    for (int i = tid; i < N; i += SORT_TILE) keys[i] = token_key(ids, nullptr, i, V);
    __syncthreads();
    const int i = blockIdx.x * 64 + lane, i0 = blockIdx.x * 64;
    const unsigned mine = i < N ? keys[i] : 0u;
    const int per = ((N + 63) / 64 + 15) / 16 * 64;   // keys of a wave, whole groups of 64
    const int j0 = wave * per, j1 = min(N, j0 + per);
    int c = 0;
    // equal keys count if they come first: those of earlier groups do, and in
    // the token's own group those of lower lanes
    for (int j = j0; j < min(j1, i0); j += 4) {
        const u32x4 k = *reinterpret_cast<const u32x4 *>(keys + j);
        c += (k[0] <= mine) + (k[1] <= mine) + (k[2] <= mine) + (k[3] <= mine);
    }
    if (i0 >= j0 && i0 < j1)
        for (int j = i0; j < min(j1, i0 + 64); ++j) c += keys[j] < mine || (keys[j] == mine && j < i);
    int j = max(j0, i0 + 64);
    for (; j + 4 <= j1; j += 4) {
        const u32x4 k = *reinterpret_cast<const u32x4 *>(keys + j);
        c += (k[0] < mine) + (k[1] < mine) + (k[2] < mine) + (k[3] < mine);
    }
    for (; j < j1; ++j) c += keys[j] < mine;
    counts[wave][lane] = c;
    __syncthreads();
    if (wave == 0 && i < N) {
        int at = 0;
#pragma unroll
        for (int w = 0; w < 16; ++w) at += counts[w][lane];
        keys_out[at] = mine;
        pos_out[at] = i;
    }
}

// Many tokens: a stable radix sort of (key, position), least significant digit
// first.  A pass is a count of each block's digits and a scatter; a block owns
// `span` consecutive tokens.
constexpr int SORT_MAX_BLOCKS = 256;
constexpr int SORT_MAX_BITS = 11;      // of a digit: 2048 counters per wave of the block, with the digits' places 72 KiB of LDS

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
    p.bits = (keybits + p.passes - 1) / p.passes;
    const long tiles = (N + SORT_TILE - 1) / SORT_TILE;
    const long per = (tiles + SORT_MAX_BLOCKS - 1) / SORT_MAX_BLOCKS;
    p.span = (per < 1 ? 1 : per) * SORT_TILE;
    p.blocks = (int)((N + p.span - 1) / p.span);
    return p;
}

__global__ __launch_bounds__(SORT_TILE) void sort_count_kernel(long N, long V, const int64_t *__restrict__ ids,
                                                               const unsigned *__restrict__ keys, int shift, int bits,
                                                               long span, int *__restrict__ hist, Fill fill)
{
    __shared__ int cnt[1 << SORT_MAX_BITS];
    if (fill_block(fill)) return;
    const int bins = 1 << bits;
    for (int b = threadIdx.x; b < bins; b += SORT_TILE) cnt[b] = 0;
    __syncthreads();
    const long i0 = blockIdx.x * span, i1 = min(N, i0 + span);
    for (long i = i0 + threadIdx.x; i < i1; i += SORT_TILE)
        atomicAdd(&cnt[(token_key(ids, keys, i, V) >> shift) & (bins - 1)], 1);
    __syncthreads();
    for (int b = threadIdx.x; b < bins; b += SORT_TILE) hist[(long)blockIdx.x * bins + b] = cnt[b];
}

__global__ __launch_bounds__(SORT_TILE) void sort_scatter_kernel(long N, long V, const int64_t *__restrict__ ids,
                                                                 const unsigned *__restrict__ keys,
                                                                 const int *__restrict__ pos, int shift, int bits,
                                                                 long span, const int *__restrict__ hist,
                                                                 unsigned *__restrict__ keys_out,
                                                                 int *__restrict__ pos_out, Fill fill)
{
    constexpr int WAVES = SORT_TILE / 64;
    __shared__ unsigned short in_wave[WAVES][1 << SORT_MAX_BITS];   // per wave: counts, then counts of earlier waves
    __shared__ int base[1 << SORT_MAX_BITS];                         // next place of each digit
    __shared__ int sums[WAVES];
    if (fill_block(fill)) return;
    const int bins = 1 << bits, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int nb = fill.first;

    // this block's first place of each digit: all smaller digits, and the
    // digit's tokens in earlier blocks.  Thread t takes digits 2t and 2t + 1.
    int total[2] = {0, 0}, before[2] = {0, 0};
    if (2 * tid < bins) {
        int k = 0;
#pragma unroll 8
        for (; k < (int)blockIdx.x; ++k) {
            const int2 c = *reinterpret_cast<const int2 *>(hist + (long)k * bins + 2 * tid);
            before[0] += c.x;
            before[1] += c.y;
        }
        total[0] = before[0];
        total[1] = before[1];
#pragma unroll 8
        for (; k < nb; ++k) {
            const int2 c = *reinterpret_cast<const int2 *>(hist + (long)k * bins + 2 * tid);
            total[0] += c.x;
            total[1] += c.y;
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
    if (2 * tid < bins) {
        base[2 * tid] = first + before[0];
        base[2 * tid + 1] = first + total[0] + before[1];
    }

    const long i0 = blockIdx.x * span, i1 = min(N, i0 + span);
    for (long t0 = i0; t0 < i1; t0 += SORT_TILE) {
        for (int e = tid; e < WAVES * bins / 2; e += SORT_TILE)
            reinterpret_cast<unsigned *>(&in_wave[2 * e >> bits][0])[e & (bins / 2 - 1)] = 0;
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
// Sums over the sorted tokens.  Equal rows are neighbours, so the work is cut
// by tokens, whatever the frequencies: a wave has RUN sorted tokens and 64
// vectors of the columns.  A row of at most RUN tokens is summed whole by the
// run its first token lies in; of a longer row every run sums its own tokens
// and leaves a partial sum (in the first of a run's two slots if the row came
// from the run before, else in the second), which embed_combine_kernel adds in
// order.  Whether a row is longer shows in the RUN keys before and behind the
// run, a lane each, as the bits at which the key changes (so RUN is at most 21).
// Bound by memory: 40000 tokens of 1024 bf16 columns in 45 us, for 82 MB read
// and the rows met written (and read, where they accumulate); 6400 in 9, mostly
// latency.  The whole gradient with RUN = 8, 16, 20: 6400 tokens 49, 50, 51 us,
// 2 x 40000 309, 281, 278.
// ---------------------------------------------------------------------------
constexpr int RUN = 16;

struct Window {
    unsigned key;                // lane l: that of sorted token RUN * (r - 1) + l, l < 3 RUN
    int pos;
    unsigned long long change;   // bit l: the key of lane l differs from lane l - 1's
};

__device__ __forceinline__ Window run_window(const unsigned *keys, const int *pos, long N, long r, int lane)
{
    const long i = RUN * (r - 1) + lane;
    const bool in = i >= 0 && i < N && lane < 3 * RUN;
    Window w;
    w.key = in ? keys[i] : (i < 0 ? 0xffffffffu : 0xfffffffeu);
    w.pos = in && pos ? pos[i] : 0;
    w.change = __ballot(w.key != __shfl_up(w.key, 1));
    return w;
}

__device__ __forceinline__ int next_change(const Window &w, int from)   // the first at or behind `from`, 64 if none
{
    const unsigned long long m = w.change >> from;
    return from < 64 && m ? from + __builtin_ctzll(m) : 64;
}

template <typename T>
__global__ __launch_bounds__(256) void embed_runs_kernel(long N, long V, int nv, const unsigned *__restrict__ keys,
                                                         const int *__restrict__ pos, const T *__restrict__ dout,
                                                         long ldo, float scale, float *__restrict__ dtable,
                                                         int accumulate, float *__restrict__ partial)
{
    constexpr int BATCH = 8;     // rows in flight
    const int lane = threadIdx.x & 63, blocks = (nv + 63) / 64;
    const long D = (long)nv * VEC<T>, tasks = (N + RUN - 1) / RUN * blocks;
    for (long task = (long)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); task < tasks;
         task += (long)gridDim.x * 4) {
        const long r = task / blocks;
        const int c = (int)(task % blocks) * 64 + lane;
        const Window w = run_window(keys, pos, N, r, lane);
        // tokens p0 .. p1 - 1 of the window
        int p0 = RUN, p1 = 2 * RUN;
        if (!(w.change >> RUN & 1)) {   // a row from the run before: this run's if it is longer than RUN
            const unsigned long long before = w.change & ((1ull << RUN) - 2);
            const int end = next_change(w, RUN + 1);
            if (before && end - (63 - __builtin_clzll(before)) <= RUN) p0 = end;
        }
        if (p0 >= p1) continue;
        const int last = 63 - __builtin_clzll((w.change | 1ull << p0) & ((1ull << p1) - 1));   // where the last row starts
        if (!(w.change >> p1 & 1) && (w.change >> last & 1)) {
            const int end = next_change(w, p1);
            if (end - last <= RUN) p1 = end;
        }
        // tokens outside the table are behind all others
        const unsigned long long outside = __ballot(w.key >= (unsigned)V) >> p0;
        if (outside) p1 = min(p1, p0 + __builtin_ctzll(outside));

        float acc[VEC<T>];
#pragma unroll
        for (int e = 0; e < VEC<T>; ++e) acc[e] = 0.0f;
        int start = p0;
        auto flush = [&](int end) {   // the row of tokens start .. end - 1
            const bool head = !(w.change >> start & 1), more = !(w.change >> end & 1);
            if (c < nv) {
                const bool part = head || more;
                float *p = part ? partial + (2 * r + (head ? 0 : 1)) * D + (long)c * VEC<T>
                                : dtable + (long)(unsigned)__builtin_amdgcn_readlane(w.key, start) * D + (long)c * VEC<T>;
#pragma unroll
                for (int e = 0; e < VEC<T>; e += 4) {
                    f32x4 v = {acc[e], acc[e + 1], acc[e + 2], acc[e + 3]};
                    f32x4 *to = reinterpret_cast<f32x4 *>(p + e);
                    if (!part) v = accumulate ? *to + scale * v : scale * v;
                    *to = v;
                }
            }
#pragma unroll
            for (int e = 0; e < VEC<T>; ++e) acc[e] = 0.0f;
            start = end;
        };
        for (int b = p0; b < p1; b += BATCH) {
            u32x4 v[BATCH];
#pragma unroll
            for (int k = 0; k < BATCH; ++k) {
                const long row = __builtin_amdgcn_readlane(w.pos, min(b + k, p1 - 1));
                v[k] = c < nv ? ldg16(dout + row * ldo + (long)c * VEC<T>) : zero16();
            }
#pragma unroll
            for (int k = 0; k < BATCH; ++k) {
                if (b + k >= p1) break;
                if (b + k > start && (w.change >> (b + k) & 1)) flush(b + k);
                float f[VEC<T>];
                unpack<T>(v[k], f);
#pragma unroll
                for (int e = 0; e < VEC<T>; ++e) acc[e] += f[e];
            }
        }
        if (p1 > start) flush(p1);
    }
}

// Rows of more than RUN tokens: a block looks at 16 runs, one per wave, for a
// long row that starts in the run and reaches over its end.  The wave adds up
// to ALONE partial sums by itself; of a longer row all the block's waves add a
// sixteenth each, so that a word that makes up a tenth of 40000 tokens is no
// tail.  Latency: three or four loads that wait for each other, 7 us at 6400
// tokens, 16 at 40000 (with ALONE = 1 the whole gradient is 4 and 15 us slower).
constexpr int ALONE = 32;
__global__ __launch_bounds__(1024) void embed_combine_kernel(long N, long V, int D, const unsigned *__restrict__ keys,
                                                             const float *__restrict__ partial, float scale,
                                                             float *__restrict__ dtable, int accumulate)
{
    __shared__ long owner_runs[16];
    __shared__ f32x4 part[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const long nruns = (N + RUN - 1) / RUN;
    const int c = (blockIdx.y * 64 + lane) * 4;
    for (long r0 = (long)blockIdx.x * 16; r0 < nruns; r0 += (long)gridDim.x * 16) {
        long runs = 0;   // that the long row of run `mine` reaches over
        const long mine = r0 + wave;
        if (mine < nruns) {
            const Window w = run_window(keys, nullptr, N, mine, lane);
            const int last = 63 - __builtin_clzll((w.change | 1) & ((1ull << 2 * RUN) - 1));
            const unsigned key = __builtin_amdgcn_readlane(w.key, 2 * RUN - 1);
            if (key < (unsigned)V && last >= RUN && !(w.change >> 2 * RUN & 1) && next_change(w, 2 * RUN) - last > RUN) {
                long lo = mine + 1;
                // the last run that starts with the row: among the next 64, or
                // by 64 probes at a time
                auto starting = [&](long step, long below) {   // of runs lo, lo + step, ...
                    const long at = lo + lane * step;
                    return __popcll(__ballot(at < below && keys[min(at, nruns - 1) * RUN] == key));
                };
                const int hits = starting(1, nruns);
                lo += hits - 1;
                long left = hits < 64 ? 1 : nruns - lo;   // run lo starts with it, run lo + left does not
                while (left > 1) {
                    const long step = (left + 63) / 64;
                    lo += (starting(step, lo + left) - 1) * step;
                    left = min(step, nruns - lo);
                }
                runs = lo - mine + 1;
                if (runs <= ALONE) {
                    if (c < D) {
                        f32x4 acc = *reinterpret_cast<const f32x4 *>(partial + (2 * mine + 1) * D + c);
#pragma unroll 8
                        for (long j = 1; j < runs; ++j)
                            acc += *reinterpret_cast<const f32x4 *>(partial + 2 * (mine + j) * D + c);
                        f32x4 *p = reinterpret_cast<f32x4 *>(dtable + (long)key * D + c);
                        *p = accumulate ? *p + scale * acc : scale * acc;
                    }
                    runs = 0;
                }
            }
        }
        if (lane == 0) owner_runs[wave] = runs;
        __syncthreads();
        for (int o = 0; o < 16; ++o) {
            const long n = owner_runs[o];
            if (!n) continue;
            const long r = r0 + o, per = (n + 15) / 16;
            f32x4 acc = {0.f, 0.f, 0.f, 0.f};
            if (c < D) {
                const long end = min(n, (wave + 1) * per);
#pragma unroll 8
                for (long j = wave * per; j < end; ++j)
                    acc += *reinterpret_cast<const f32x4 *>(partial + (j == 0 ? 2 * r + 1 : 2 * (r + j)) * D + c);
            }
            part[wave][lane] = acc;
            __syncthreads();
            if (wave == 0 && c < D) {
                acc = part[0][lane];
#pragma unroll
                for (int k = 1; k < 16; ++k) acc += part[k][lane];
                f32x4 *p = reinterpret_cast<f32x4 *>(dtable + (long)keys[r * RUN + RUN - 1] * D + c);
                *p = accumulate ? *p + scale * acc : scale * acc;
            }
            __syncthreads();
        }
        __syncthreads();   // owner_runs has been read
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
    const EmbedWs w = embed_ws(N, V, D);
    const SortPlan p = sort_plan(N, V);
    const bool few = N <= RANK_MAX;
    // the zeros, in equal shares of the sort's launches
    const long zeros = accumulate ? 0 : V * (D / 4);
    const int launches = few ? 1 : 2 * p.passes;
    long zeroed = 0;
    int fill_blocks = 0;
    auto share = [&](int sort_blocks, int k) {
        const long upto = zeros * (k + 1) / launches, n = upto - zeroed;
        const long need = (n + SORT_TILE - 1) / SORT_TILE;
        fill_blocks = (int)(need < 1024 ? need : 1024);
        const Fill f{reinterpret_cast<f32x4 *>(dtable) + zeroed, n, sort_blocks};
        zeroed = upto;
        return f;
    };
    unsigned *keys[2] = {reinterpret_cast<unsigned *>(ws + w.keys[0]), reinterpret_cast<unsigned *>(ws + w.keys[1])};
    int *pos[2] = {reinterpret_cast<int *>(ws + w.pos[0]), reinterpret_cast<int *>(ws + w.pos[1])};
    int *hist = reinterpret_cast<int *>(ws + w.hist);
    const unsigned *ksrc = nullptr;
    const int *psrc = nullptr;
    if (few) {
        const int blocks = (int)((N + 63) / 64);
        const Fill f = share(blocks, 0);
        if (blocks + fill_blocks)
            hipLaunchKernelGGL(rank_kernel, dim3(blocks + fill_blocks), dim3(SORT_TILE), 0, s, (int)N, V, ids, keys[0],
                               pos[0], f);
        ksrc = keys[0];
        psrc = pos[0];
    }
    for (int k = 0, to = 0; !few && k < p.passes; ++k, to ^= 1) {
        Fill f = share(p.blocks, 2 * k);
        hipLaunchKernelGGL(sort_count_kernel, dim3(p.blocks + fill_blocks), dim3(SORT_TILE), 0, s, N, V, ids, ksrc,
                           k * p.bits, p.bits, p.span, hist, f);
        f = share(p.blocks, 2 * k + 1);
        hipLaunchKernelGGL(sort_scatter_kernel, dim3(p.blocks + fill_blocks), dim3(SORT_TILE), 0, s, N, V, ids, ksrc,
                           psrc, k * p.bits, p.bits, p.span, hist, keys[to], pos[to], f);
        ksrc = keys[to];
        psrc = pos[to];
    }
    if (N > 0) {
        float *partial = reinterpret_cast<float *>(ws + w.partial);
        const int nv = D / VEC<T>;
        const long nruns = (N + RUN - 1) / RUN, tasks = nruns * ((nv + 63) / 64);
        hipLaunchKernelGGL(embed_runs_kernel<T>, dim3((unsigned)(tasks < 4 * 65536 ? (tasks + 3) / 4 : 65536)), dim3(256), 0,
                           s, N, V, nv, ksrc, psrc, dout, ldo, scale, dtable, accumulate, partial);
        if (N > RUN)
            hipLaunchKernelGGL(embed_combine_kernel, dim3((unsigned)(nruns < 16 * 16384 ? (nruns + 15) / 16 : 16384), (D + 255) / 256),
                               dim3(1024), 0, s, N, V, D, ksrc, partial, scale, dtable, accumulate);
    }
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
