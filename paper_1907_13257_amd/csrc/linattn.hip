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
    float *slots;            // where the sequences are split: states [B*N][parts], laid out as X0 (see below)
};
constexpr int MAX_ROLES = 3;
template <typename T>
struct Roles {
    Role<T> r[MAX_ROLES];
    const float *decay;
    const int32_t *lengths;
    int T_, B, N;
    int parts, part_len;     // parts of a sequence, their tokens (a multiple of the chunk)
    int tiles;               // result tiles of 16 columns per wave, 1 or 2
    int roles, each;         // grouped launches: its roles; its blocks for each head and part
    unsigned inv_each;       // 2^32 / each, rounded up
    bool joined;             // the slots hold the states at the parts' starts
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

// ---------------------------------------------------------------------------
// Sequences, one chunk of C tokens after another.  A block has one head of one
// batch row (or a part of its tokens); each of its waves owns 32 or 16 columns
// of the state, which stay in its registers, and takes the chunk's rows of A and
// B (shared) and C (its own columns) from LDS:
//   out^T = decay^t X^T A^T + C^T P ,  P = (B A^T) * decay^(t-s) for s <= t
//   X     = decay^C X + B^T (C decay^(C-1-s))
// C is the depth of one matrix instruction, so the sums over a chunk's tokens
// are one instruction each.  The layouts chain without leaving the registers:
// a 16x16 result has its rows 4q .. 4q+3 (q = lane / 16) in a lane, which is
// what the next product's operand wants of the dimension it sums over, if
// both its operands take that dimension in the order {4q.., 16 + 4q..} (bf16:
// two result tiles make one operand) or {4q..} (fp32).  So X goes from the
// accumulators into A X and P from its product into C^T P; only the rows A, B
// (in that order: two 8-byte reads) and the transposes B^T, C^T (transposing
// reads) come from LDS.  Every wave forms P for itself.
//
// bf16 storage: X, P and the decayed C are fp32 values that the matrix cores
// take in three bf16 parts of eight bits each, so nothing of a value is left out
// and results are those of fp32 factors, whichever states a call gives or wants.
// (Two parts, which leave out 2^-17 of a factor, take 395 us instead of 460 for 4 x
// 4096 tokens of 16 heads of 128, forward and backward, 51 instead of 57 for 128 x
// 50 of 16 heads of 64, 31 and 31 for 2 x 1999; but where terms cancel, the
// result's own rounding is below what they lose.)
//
// What bounds it: with the chip full (two waves per SIMD at heads of 128), the
// chain of a wave's instructions: per chunk and wave 120 matrix instructions and
// some 700 others, the split of X and P the most of them (46 to 49 % of a wave's
// time in the main launch it issues, 32 to 34 % it waits its turn to, 17 to 22 % for
// data and barriers), and the registers of a 128-wide state allow no third wave to
// fill the gaps.  A forward of 4 x 4096 tokens of 16 heads of 128 takes 121 us for
// 268 MB, 2.2 TB/s against 4.9 of a copy, in three launches: the parts' states (35),
// their join (11) and the outputs (83, each by itself under a profiler).  The three
// gradients read 9 and write 3 widths of rows where 4 and 3 would do: 342 us for 805
// MB, 61 of them for the parts' states; one launch that formed all three would have
// to run the tokens in both directions.  Short or few sequences are bound by
// latency: about 2 us per chunk and 5 before the first.
// ---------------------------------------------------------------------------
template <typename T> struct Mat;
template <> struct Mat<bf16_t> {
    static constexpr int C = 32;   // tokens of a chunk, depth of a matrix instruction
    static constexpr int TT = 2;   // result tiles of 16 that make an operand of that depth
};
template <> struct Mat<float> {
    static constexpr int C = 16;
    static constexpr int TT = 1;
};
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) char lds_char;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4_t;
typedef __attribute__((address_space(3))) const u32x4 lds_u32x4_t;
typedef __attribute__((address_space(3))) const u32x2 lds_u32x2_t;
typedef __attribute__((address_space(3))) const unsigned lds_u32_t;

__device__ __align__(16) const unsigned zero_chunk[4] = {0, 0, 0, 0};

// 16 bytes per lane from a lane's own address to LDS byte lds_byte + 16 * lane.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void dma16_from(const void *p, unsigned lds_byte)
{
    asm volatile("s_mov_b32 m0, %0\n\tglobal_load_lds_dwordx4 %1, off" : : "s"(lds_byte), "v"(p) : "memory", "m0");
}
#pragma clang diagnostic pop

// A tile of rows of CH chunks of 16 bytes in LDS.  One load instruction fills
// 64 chunks, 64 / CH rows; instructions are some bytes more than that apart, and
// chunk c of a row stands at c ^ flip(row).  Which rows an instruction takes and
// their order in it (bits b0 .. b3 of the row), the gaps and the flips are such
// that, of the 256 bytes LDS serves at a time,
//   - the 16 rows one operand read touches at one chunk get 16 different places,
//   - the rows 0-7 (8-15) of half a transposing read get 8 different 32 bytes,
// while the address stays a lane's own offset plus a constant, with one other
// offset for odd column blocks, and the two halves of an operand lie 32 bytes
// apart (one read instruction, no copies to bring them together).
template <int CH>
struct Tile {
    __host__ __device__ static constexpr int b(int row, int bit) { return (row >> bit) & 1; }
    __device__ static constexpr int flip(int row)
    {
        return CH == 2 ? 0 : CH == 4 ? 2 * b(row, 2) + b(row, 3) : 4 * b(row, 2) + b(row, 3);
    }
    // instruction of a row, and its place there
    __device__ static constexpr int instr(int row)
    {
        const int hi = row >> 4;
        return CH == 64 ? row : CH == 32 ? (row & 7) + 8 * hi : CH == 16 ? (row & 3) + 4 * hi
                                                              : CH == 8 ? (row & 1) + 2 * hi : CH == 4 ? hi : 0;
    }
    __device__ static constexpr int place(int row)
    {
        const int f = 2 * b(row, 2) + b(row, 3);
        return CH == 64 ? 0 : CH == 32 ? b(row, 3) : CH == 16 ? f : CH == 8 ? b(row, 1) + 2 * f
                                                                : CH == 4 ? (row & 3) + 4 * f : row;
    }
    // the row of place j of instruction k: row_k(k) + row_j(j)
    __device__ static constexpr int row_k(int k)
    {
        return CH == 64 ? k : CH == 32 ? (k & 7) + 16 * (k >> 3) : CH == 16 ? (k & 3) + 16 * (k >> 2)
                                       : CH == 8 ? (k & 1) + 16 * (k >> 1) : CH == 4 ? 16 * k : 32 * k;
    }
    __device__ static constexpr int row_j(int j)
    {
        return CH == 64 ? 0 : CH == 32 ? 8 * j : CH == 16 ? 4 * b(j, 1) + 8 * b(j, 0)
                                       : CH == 8 ? 2 * b(j, 0) + 8 * b(j, 1) + 4 * b(j, 2)
                                                 : CH == 4 ? (j & 3) + 8 * b(j, 2) + 4 * b(j, 3) : j;
    }
    __host__ __device__ static constexpr int start(int k)   // byte of instruction k
    {
        return k * 1024 + (CH >= 16 ? 32 * b(k, 0) + 128 * b(k, 1) + (k >> 2) * 256 : CH == 8 ? 32 * b(k, 0) + (k >> 1) * 256 : 0);
    }
    __host__ __device__ static constexpr int bytes(int instrs) { return start(instrs - 1) + 1024; }
    __device__ static constexpr int offset(int row) { return start(instr(row)) + place(row) * CH * 16; }
};

// Where a lane's share of a tile's rows comes from: rows of `width` elements,
// `step` apart.
template <typename T, int CH>
struct Loader {
    static constexpr int E = 16 / (int)sizeof(T);
    const T *own;   // the lane's row and chunk of instruction 0
    long step;
    int row, chunk, chunks;
    __device__ __forceinline__ void init(const T *base, long step_, int width, int lane)
    {
        step = step_;
        row = Tile<CH>::row_j(lane / CH);
        chunk = (lane % CH) ^ Tile<CH>::flip(row);
        chunks = width / E;
        own = base + row * step + chunk * E;
    }
    // instruction k of the tile whose first row is token t0, `rows` of them; zeros
    // elsewhere (`whole`: nowhere)
    __device__ __forceinline__ void issue(int t0, int rows, int k, unsigned tile, bool whole) const
    {
        const int rk = Tile<CH>::row_k(k);
        int c = chunk;
        const T *p = own + (t0 + rk) * step;
        if constexpr (CH >= 32) {   // such rows' bit 2 (and 3) is the instruction's
            c ^= Tile<CH>::flip(rk);
            p += (c - chunk) * E;
        }
        if (!whole && !(row + rk < rows && c < chunks)) p = reinterpret_cast<const T *>(zero_chunk);
        dma16_from(p, __builtin_amdgcn_readfirstlane(tile + (unsigned)Tile<CH>::start(k)));
    }
};

// Where a lane finds the operands of a tile.
template <int CH, typename T> struct Reader;
template <int CH>
struct Reader<CH, bf16_t> {
    unsigned rows, cols;
    __device__ __forceinline__ void init(int c16, int q)
    {
        // rows c16: 8 bytes at columns 4q and 16 + 4q of 32
        rows = Tile<CH>::offset(c16) + ((q >> 1) ^ Tile<CH>::flip(c16)) * 16 + (q & 1) * 8;
        // columns: in each group of 16 lanes, lane s addresses the 8 bytes of
        // row 4q + s/4 and columns 4 (s%4); lane i receives four rows of column i
        const int r = 4 * q + (c16 >> 2);
        cols = Tile<CH>::offset(r) + (((c16 & 3) >> 1) ^ Tile<CH>::flip(r)) * 16 + (c16 & 1) * 8;
    }
    // row 16 s + c16 at column block kb
    __device__ __forceinline__ u32x4 row(lds_char *tile, int s, int kb) const
    {
        u32x2 lo, hi;
        if constexpr (CH == 4) {   // one column block; the flip swaps its halves
            lo = *(lds_u32x2_t *)(tile + rows + Tile<CH>::offset(16 * s));
            hi = *(lds_u32x2_t *)(tile + (rows ^ 32) + Tile<CH>::offset(16 * s));
        } else {
            lds_char *p = tile + (rows ^ (kb & 1) * 64) + (kb >> 1) * 128 + Tile<CH>::offset(16 * s);
            lo = *(lds_u32x2_t *)p;
            hi = *(lds_u32x2_t *)(p + 32);
        }
        return u32x4{lo[0], lo[1], hi[0], hi[1]};
    }
    // columns 16 ct .. 16 ct + 15 over the tile's rows
    __device__ __forceinline__ u32x4 col(lds_char *tile, int ct) const
    {
        lds_char *p = CH == 4 ? tile + (cols ^ ct * 32) : tile + (cols ^ ((ct >> 1) & 1) * 64) + (ct >> 2) * 128 + (ct & 1) * 32;
        const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t *)p));
        const u32x2 hi = __builtin_bit_cast(
            u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t *)(p + Tile<CH>::offset(16))));
        return u32x4{lo[0], lo[1], hi[0], hi[1]};
    }
};
template <int CH>
struct Reader<CH, float> {
    unsigned rows, odd, cols;   // rows at even and odd column blocks
    __device__ __forceinline__ void init(int c16, int q)
    {
        rows = Tile<CH>::offset(c16) + (q ^ Tile<CH>::flip(c16)) * 16;
        odd = Tile<CH>::offset(c16) + (q ^ 4 ^ Tile<CH>::flip(c16)) * 16;
        cols = Tile<CH>::offset(4 * q) + ((c16 >> 2) ^ Tile<CH>::flip(4 * q)) * 16 + (c16 & 3) * 4;
    }
    __device__ __forceinline__ u32x4 row(lds_char *tile, int, int kb) const
    {
        return *(lds_u32x4_t *)(tile + (kb & 1 ? odd : rows) + (kb >> 1) * 128);
    }
    __device__ __forceinline__ u32x4 col(lds_char *tile, int ct) const
    {
        u32x4 f;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            f[e] = *(lds_u32_t *)(tile + (cols ^ (ct & 1) * 64) + (ct >> 1) * 128 + Tile<CH>::offset(e));
        return f;
    }
};

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ unsigned pack_bf16(float a, float b)   // one conversion instruction for both
{
    return __builtin_bit_cast(unsigned, __builtin_convertvector((f32x2{a, b}), bf16x2));
}

// fp32 values of an operand as the parts the matrix cores take.  A part is the
// upper half of what the parts before it left over: eight bits of the value, cut
// off and not rounded, so the three of them are the value and the largest values
// stay finite.
template <int NP>
__device__ __forceinline__ void split(const float (&x)[8], u32x4 (&f)[NP], bf16_t)
{
    unsigned r[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = __float_as_uint(x[e]);
#pragma unroll
    for (int p = 0; p < NP; ++p) {
#pragma unroll
        for (int e = 0; e < 8; e += 2) f[p][e / 2] = __builtin_amdgcn_perm(r[e + 1], r[e], 0x07060302u);
        if (p + 1 < NP)   // what is left over, exactly
#pragma unroll
            for (int e = 0; e < 8; ++e)
                r[e] = __float_as_uint(__uint_as_float(r[e]) - __uint_as_float(r[e] & 0xffff0000u));
    }
}
template <int NP>
__device__ __forceinline__ void split(const float (&x)[4], u32x4 (&f)[NP], float)
{
    f[0] = __builtin_bit_cast(u32x4, f32x4{x[0], x[1], x[2], x[3]});
}

// Four consecutive values of an output row.
template <typename T> struct Out4;
template <> struct Out4<bf16_t> { typedef u32x2 type; };
template <> struct Out4<float> { typedef f32x4 type; };
__device__ __forceinline__ u32x2 out4(f32x4 a, bf16_t) { return u32x2{pack_bf16(a[0], a[1]), pack_bf16(a[2], a[3])}; }
__device__ __forceinline__ f32x4 out4(f32x4 a, float) { return a; }

// Chunks of 16 bytes a tile's row has in LDS: a power of two.
template <typename T, int DA>
constexpr int row_chunks()
{
    int c = 4;
    while (c * 16 < DA * (int)sizeof(T)) c *= 2;
    return c;
}

// A long sequence of few heads is split into parts: a first launch (not OUT)
// leaves in slot p + 1 the state that the tokens of part p add, and in slot 0
// the first state (which the final one may replace while other blocks run); the
// second (OUT) starts a part from slots 0 .. p, joined with the decays between
// them, by itself or, where they are many, from what linattn_join_kernel made of
// them.  The last part of a sequence adds to no other and has no slot.
//
// OUT: rows of the output, and the final state; else the slots.
// DA: the width of A and B, padded with zeros to a multiple of 32.  MT: result
// tiles of 16 columns per wave.  GROUP: the order of the blocks (see
// launch_chunks).
template <typename T, int DA, bool OUT, int MT, bool GROUP>
__global__ __launch_bounds__(512, DA <= 64 ? 3 : 2) void linattn_chunks_kernel(Roles<T> g)
{
    constexpr int C = Mat<T>::C, TT = Mat<T>::TT, E = C / 4;   // E: values of an operand per lane
    constexpr int WCOLS = 16 * MT;                             // columns of a wave
    constexpr int CHA = row_chunks<T, DA>(), CHC = WCOLS * (int)sizeof(T) / 16;
    constexpr int KB = DA / C, KT = DA / 16, KEEP = KB < 4 ? KB : 4;
    constexpr int NA = C * CHA / 64, NC = C * CHC / 64;        // load instructions of a tile
    constexpr int ABYTES = Tile<CHA>::bytes(NA), CBYTES = Tile<CHC>::bytes(NC);
    constexpr int NP = sizeof(T) == 2 ? 3 : 1;                 // parts of an fp32 factor
    extern __shared__ __align__(16) char lds[];
    unsigned bx = blockIdx.x, by = blockIdx.y, bz = blockIdx.z;
    if constexpr (GROUP) {   // a head's blocks eight apart
        const unsigned grp = __umulhi(bx / 8, g.inv_each), sub = bx / 8 - grp * g.each;   // bx / 8 / each, and what is left
        bx = grp * 8 + bx % 8;
        bz = sub >= (unsigned)g.roles ? 1 : 0;
        by = sub - bz * g.roles;
        if (bx >= (unsigned)(g.B * g.N * g.parts)) return;
    }
    const Role<T> &r = g.r[by];
    const int waves = blockDim.x >> 6, lane = threadIdx.x & 63, q = lane >> 4, c16 = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int h = bx % g.N, b = (int)((bx / g.N) % g.B), part = (int)(bx / g.N / g.B);
    const long bh = (long)b * g.N + h;
    // (a value read from memory that is the same for all lanes stays in a scalar
    // register only if it is said to be)
    const int n = __builtin_amdgcn_readfirstlane(sequence_length(g.lengths, b, g.T_));
    const int begin = part * g.part_len, stop = min(g.T_, begin + g.part_len), end = min(n, stop);
    const int da = r.da, dc = r.dc, col0 = ((int)bz * waves + wave) * WCOLS;
    T *const out = r.out;
    const long size = (long)da * dc, slots = bh * g.parts * size;
    const bool last = end >= n;   // of this sequence
    float *const XT = OUT && last && (n > 0 || part == 0) ? r.XT : nullptr;

    if (!OUT && part == 0 && bz == 0 && r.X0)   // the first state
        for (int i = threadIdx.x; i < size / 4; i += blockDim.x)
            reinterpret_cast<f32x4 *>(r.slots + slots)[i] = reinterpret_cast<const f32x4 *>(r.X0 + bh * size)[i];
    if (!OUT && last) return;
    if (OUT && !out && !XT) return;
    if (OUT && out && n < stop && bz == 0) {   // behind the sequence's end
        const int per = dc * (int)sizeof(T) / 16, t0 = max(n, begin);
        const long all = (long)(stop - t0) * per;
        for (long i = threadIdx.x; i < all; i += blockDim.x) {
            T *row = out + ((t0 + i / per) * g.B + b) * r.ldo + (long)h * dc;
            reinterpret_cast<u32x4 *>(row)[i % per] = zero16();
        }
    }
    if (begin >= end && (part > 0 || !OUT)) return;

    // rows of token i of the sequence: first + i * dir
    const long first = r.reverse ? (long)(n - 1) * g.B + b : b, dir = r.reverse ? -g.B : g.B;

    // LDS: two buffers of a chunk's rows of A and B and every wave's columns of C
    const int chunk_bytes = (OUT ? 2 : 1) * ABYTES + waves * CBYTES;
    const unsigned lds0 = lds_addr(lds);
    Loader<T, CHA> la, lb;
    Loader<T, CHC> lc;
    if (OUT) la.init(r.a + first * r.lda + (long)h * da, dir * r.lda, da, lane);
    lb.init(r.b + first * r.ldb + (long)h * da, dir * r.ldb, da, lane);
    lc.init(r.c + first * r.ldc + (long)h * dc + col0, dir * r.ldc, dc - col0, lane);
    auto issue = [&](int t0, int buf) {
        const int rows = min(C, end - t0);
        const unsigned base = lds0 + (unsigned)(buf * chunk_bytes);
        if (rows == C && da * (int)sizeof(T) == CHA * 16) {
#pragma unroll 1
            for (int k = wave; k < NA; k += waves) {
                lb.issue(t0, C, k, base, true);
                if (OUT) la.issue(t0, C, k, base + ABYTES, true);
            }
        } else {
#pragma unroll 1
            for (int k = wave; k < NA; k += waves) {
                lb.issue(t0, rows, k, base, false);
                if (OUT) la.issue(t0, rows, k, base + ABYTES, false);
            }
        }
#pragma unroll
        for (int k = 0; k < NC; ++k) lc.issue(t0, rows, k, base + (OUT ? 2 : 1) * ABYTES + wave * CBYTES, false);
    };
    if (begin < end) issue(begin, 0);

    const float lg = decay_log2(g.decay[h]);
    // the state: element (16 kt + 4 q + v, col0 + 16 mt + c16) in X[kt][mt][v]
    f32x4 X[KT][MT];
    const int si = r.si, sj = r.sj;
    const int own = 4 * q * si + (col0 + c16) * sj;   // the lane's element (0, 0, 0)
    bool zero = true;   // X is zero
    auto join = [&](const float *from, float keep) {   // X = keep X + from
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) {
            if (kt % 4 == 0) __builtin_amdgcn_sched_barrier(0);   // loads of four tiles in flight, not of all
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
                if (16 * kt + 4 * q < da && col0 + 16 * mt + c16 < dc)
#pragma unroll
                    for (int v = 0; v < 4; ++v)
                        X[kt][mt][v] = from[own + (16 * kt + v) * si + 16 * mt * sj] + keep * X[kt][mt][v];
        }
        zero = false;
    };
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) X[kt][mt] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (OUT) {
        if (r.X0) join(g.parts > 1 ? r.slots + slots : r.X0 + bh * size, 0.0f);
        const float keep = part > 0 && !g.joined ? decay_pow(lg, g.part_len) : 0.0f;
        for (int k = g.joined ? max(part, 1) : 1; k <= part; ++k) join(r.slots + slots + k * size, keep);
    }

    // decays between the state and the row of the first token: one forwards; the
    // state of the backward directions stands at that token, one decay further
    const int pre = r.reverse ? 0 : 1;
    // P's factors within a tile (zero above the diagonal) and one tile below;
    // the rows' factors of what is left of the state
    float w0[4], w1[4], rowf[TT];
#pragma unroll
    for (int v = 0; v < 4; ++v) {
        const int d = c16 - 4 * q - v;
        w0[v] = d < 0 ? 0.0f : r.intra * decay_pow(lg, d);
        w1[v] = r.intra * decay_pow(lg, 16 + d);
    }
#pragma unroll
    for (int ti = 0; ti < TT; ++ti) rowf[ti] = r.inter * decay_pow(lg, 16 * ti + c16 + pre);
    float wc[E];          // the tokens' factors in the chunk's final state
    int wc_rows = -1;     // for a chunk of so many tokens
    // The state is gain * X: a chunk's decay goes into gain, its tokens are
    // added divided by gain, and X is multiplied only when gain gets small
    // (one chunk in many for the usual decays; so X is at most 2^10 times the
    // state).  gain is the power of the decay over all tokens since then: a
    // product of the chunks' powers would have each one's rounding, the same one
    // every time, which adds up to 1e-4 of the state of a head that remembers
    // 65536 tokens.
    float gain = 1.0f;
    int since = 0;

    Reader<CHA, T> ra;
    Reader<CHC, T> rc;
    ra.init(c16, q);
    rc.init(c16, q);
    const long ldo = r.ldo, sto = dir * ldo;
    T *orow = OUT && out ? out + (first + (begin + c16) * dir) * ldo + (long)h * dc + col0 + 4 * q : nullptr;

    int buf = 0;
    for (int t0 = begin; t0 < end; t0 += C, buf ^= 1) {
        waitcnt_vm<0>();   // this chunk's rows
        __syncthreads();   // everyone's; and the other buffer has been read
        if (t0 + C < end) issue(t0 + C, buf ^ 1);
        if (col0 >= dc) continue;   // a wave beyond this role's columns only loads
        lds_char *tb = (lds_char *)lds + buf * chunk_bytes, *ta = tb + ABYTES;
        lds_char *tc = tb + (OUT ? 2 : 1) * ABYTES + wave * CBYTES;
        const int rows = min(C, end - t0);

        u32x4 ct[MT];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) ct[mt] = rc.col(tc, mt);

        if constexpr (OUT) {
            // P^T: tile of tokens s (rows) by tile of tokens ti (columns)
            f32x4 P[TT][TT];
#pragma unroll
            for (int ti = 0; ti < TT; ++ti)
#pragma unroll
                for (int s = 0; s <= ti; ++s) P[s][ti] = f32x4{0.f, 0.f, 0.f, 0.f};
            // the operands of all column blocks are read before the first product
            // waits for one (up to KEEP blocks: registers), and A's stay
            u32x4 a[TT][KEEP], bf[TT][KEEP];
            auto read = [&](int kb) {
#pragma unroll
                for (int ti = 0; ti < TT; ++ti) {
                    a[ti][kb % KEEP] = ra.row(ta, ti, kb);
                    bf[ti][kb % KEEP] = ra.row(tb, ti, kb);
                }
            };
#pragma unroll
            for (int k0 = 0; k0 < KB; k0 += KEEP) {
#pragma unroll
                for (int kb = k0; kb < k0 + KEEP && kb < KB; ++kb) read(kb);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int kb = k0; kb < k0 + KEEP && kb < KB; ++kb)
#pragma unroll
                    for (int s = 0; s < TT; ++s)
#pragma unroll
                        for (int ti = s; ti < TT; ++ti) mfma16(P[s][ti], bf[s][kb % KEEP], a[ti][kb % KEEP], T());
            }
            u32x4 pf[TT][NP];
#pragma unroll
            for (int ti = 0; ti < TT; ++ti) {
                float x[E];
#pragma unroll
                for (int e = 0; e < E; ++e)
                    x[e] = e / 4 > ti ? 0.0f : P[e / 4][ti][e % 4] * (e / 4 == ti ? w0[e % 4] : w1[e % 4]);
                split<NP>(x, pf[ti], T());
            }
            // X^T A^T, scaled by row, and C^T P onto it
            f32x4 o[TT][MT];
#pragma unroll
            for (int ti = 0; ti < TT; ++ti)
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) o[ti][mt] = f32x4{0.f, 0.f, 0.f, 0.f};
            if (!zero) {
#pragma unroll
                for (int kb = 0; kb < KB; ++kb) {
                    if constexpr (KB > KEEP)
#pragma unroll
                        for (int ti = 0; ti < TT; ++ti) a[ti][kb % KEEP] = ra.row(ta, ti, kb);
                    u32x4 f[MT][NP];
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt) {
                        float x[E];
#pragma unroll
                        for (int e = 0; e < E; ++e) x[e] = X[TT * kb + e / 4][mt][e % 4];
                        split<NP>(x, f[mt], T());
                    }
#pragma unroll
                    for (int p = 0; p < NP; ++p)   // neighbours add to different tiles
#pragma unroll
                        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                            for (int ti = 0; ti < TT; ++ti) mfma16(o[ti][mt], f[mt][p], a[ti][kb % KEEP], T());
                }
#pragma unroll
                for (int ti = 0; ti < TT; ++ti) {
                    const float f = rowf[ti] * gain;
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt) o[ti][mt] *= f;
                }
            }
#pragma unroll
            for (int p = 0; p < NP; ++p)
#pragma unroll
                for (int ti = 0; ti < TT; ++ti)
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt) mfma16(o[ti][mt], ct[mt], pf[ti][p], T());
#pragma unroll
            for (int ti = 0; ti < TT; ++ti)
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    if (orow && 16 * ti + c16 < rows && col0 + 16 * mt + 4 * q < dc)
                        *reinterpret_cast<typename Out4<T>::type *>(orow + 16 * ti * sto + 16 * mt) = out4(o[ti][mt], T());
                }
            if (orow) orow += C * sto;
        }

        // the state behind the chunk
        if (!OUT || t0 + C < end || XT) {
            if (rows != wc_rows) {
                wc_rows = rows;
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const int left = rows - 1 - (16 * (e / 4) + 4 * q + e % 4);
                    wc[e] = left < 0 ? 0.0f : r.update * decay_pow(lg, left + 1 - pre);
                }
            }
            since += rows;
            gain = decay_pow(lg, since);
            if (__builtin_amdgcn_readfirstlane(gain < 0x1p-10f)) {
#pragma unroll
                for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt) X[kt][mt] *= gain;
                gain = 1.0f;
                since = 0;
            }
            const float inv = 1.0f / gain;
            float w[E];
#pragma unroll
            for (int e = 0; e < E; ++e) w[e] = wc[e] * inv;
            u32x4 f[MT][NP];
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                float x[E];
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    if constexpr (sizeof(T) == 2)
                        x[e] = __uint_as_float(e % 2 ? ct[mt][e / 2] & 0xffff0000u : ct[mt][e / 2] << 16) * w[e];
                    else
                        x[e] = __uint_as_float(ct[mt][e]) * w[e];
                }
                split<NP>(x, f[mt], T());
            }
            constexpr int AHEAD = KT < 4 ? KT : 4;
#pragma unroll
            for (int k0 = 0; k0 < KT; k0 += AHEAD) {
                u32x4 bt[AHEAD];
#pragma unroll
                for (int k = 0; k < AHEAD && k0 + k < KT; ++k) bt[k] = ra.col(tb, k0 + k);
#pragma unroll
                for (int p = 0; p < NP; ++p)
#pragma unroll
                    for (int k = 0; k < AHEAD && k0 + k < KT; ++k)
#pragma unroll
                        for (int mt = 0; mt < MT; ++mt) mfma16(X[k0 + k][mt], bt[k], f[mt][p], T());
            }
            zero = false;
        }
    }

    // what the part adds, or the sequence's final state
    float *fin = !OUT ? r.slots + slots + (part + 1) * size : (XT ? XT + bh * size : nullptr);
    if (!fin) return;
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
            if (16 * kt + 4 * q < da && col0 + 16 * mt + c16 < dc)
#pragma unroll
                for (int v = 0; v < 4; ++v) fin[own + (16 * kt + v) * si + 16 * mt * sj] = gain * X[kt][mt][v];
}

// Turns the slots into the states at the parts' starts.  A batch of them is read
// before the first is written.  The parts' decay multiplies in 64 bits, lest its
// rounding add up over many parts (as a chunk's would, above).
template <typename T>
__global__ __launch_bounds__(256) void linattn_join_kernel(Roles<T> g)
{
    constexpr int BATCH = 8;
    const Role<T> &r = g.r[blockIdx.y];
    const int size = r.da * r.dc, per = (size / 4 + 255) / 256;
    const long bh = blockIdx.x / per;
    const int e = ((int)(blockIdx.x % per) * 256 + threadIdx.x) * 4;
    if (e >= size) return;
    const int n = sequence_length(g.lengths, (int)(bh / g.N), g.T_);
    const int live = (n + g.part_len - 1) / g.part_len;   // slots 1 .. live - 1 are filled
    f32x4 *p = reinterpret_cast<f32x4 *>(r.slots + bh * g.parts * (long)size + e);
    f32x4 x = r.X0 ? *p : f32x4{0.f, 0.f, 0.f, 0.f};
    const double keep = exp2(log2((double)g.decay[bh % g.N]) * g.part_len);
    for (int k0 = 1; k0 < live; k0 += BATCH) {
        f32x4 add[BATCH];
#pragma unroll
        for (int k = 0; k < BATCH; ++k)
            if (k0 + k < live) add[k] = p[(long)(k0 + k) * (size / 4)];
#pragma unroll
        for (int k = 0; k < BATCH; ++k)
            if (k0 + k < live) {
#pragma unroll
                for (int v = 0; v < 4; ++v) x[v] = (float)(keep * x[v] + add[k][v]);
                p[(long)(k0 + k) * (size / 4)] = x;
            }
    }
}

struct SplitPlan {
    int parts, len, tiles;
};

// How a call is spread over the chip's 1024 SIMDs.  Sequences are split into as
// many parts as it takes to give the chip TARGET_WAVES waves of 32 columns, but
// none shorter than MIN_CHUNKS chunks.  A wave has 32 columns: P and the shared
// rows cost a wave the same for 16.  Where that leaves the SIMDs with less than
// one wave each unsplit and few chunks in all (FEW_CHUNKS of a wave per SIMD),
// time is the latency of a wave's chunks, and 16 columns shorten it, up to heads
// of 64 (bf16) or 80 (fp32); wider ones would make more waves than a block's
// SIMDs take at a time.  Forward or backward in us with 32 and with 16 columns:
//   2 x 1999 tokens, 16 heads of 64                   forward 35, 31   backward 50, 54
//   8, 24 x 200, 16 heads of 64                       forward 18, 15 and 26, 22
//   32, 64 x 200 (too many waves)                     forward 29, 28 and 26, 30
//   4, 8 x 1000, 16 heads of 64                       forward 34, 28 and 40, 40
//   4, 16 x 1000 (the second has too many)            backward 51, 53 and 98, 105
//   4 x 700, 8 heads of 72, 96                        forward 30, 29 and 32, 32   backward 47, 56 and 51, 65
//   4 x 1000, 8 heads of 128                          forward 38, 37   backward 77, 96
//   12 x 333, 5 heads of 40 and 72, fp32              forward 30, 31   backward 76, 69
//   4 x 333, 8 heads of 80, 88, 128, fp32             backward 57, 57 and 59, 63 and 73, 92
// Heads wider than 128 always take 16: twice the state does not fit the registers.
constexpr int MAX_WAVES = 8;   // of a block
constexpr int TARGET_WAVES = 2048, MIN_CHUNKS = 3, FEW_CHUNKS = 16, SIMDS = 1024;
SplitPlan split_plan(const LinAttnShape &sh, int chunk, int roles)
{
    const int width = sh.K > sh.M ? sh.K : sh.M;
    const long waves = (long)sh.B * sh.N * roles * ((width + 31) / 32);
    const int chunks = (sh.T + chunk - 1) / chunk;
    long parts = (TARGET_WAVES + waves - 1) / waves;
    const long most = chunks / MIN_CHUNKS;
    if (parts > most) parts = most;
    if (parts < 1) parts = 1;
    const int per = (int)((chunks + parts - 1) / parts);
    const bool few = waves < SIMDS && waves * chunks < (long)FEW_CHUNKS * SIMDS;
    const bool narrow = width <= (chunk == Mat<bf16_t>::C ? 64 : 80);
    return SplitPlan{(chunks + per - 1) / per, per * chunk, (few && narrow) || width > 128 ? 1 : 2};
}

// The blocks of a head (its roles; the columns of a wide one), which read the
// same rows, are launched eight apart where they have many chunks: on one XCD at
// about one time, so that its L2 serves what another of them has read.  Backward in
// us so and role after role, by a block's chunks: 8 (64 x 256 tokens of 16 heads of
// 64) 69 and 72, 13 (64 x 400) 138 and 138, 16 (16 x 1000 of 8 heads of 128) 142 and
// 161, 43 (4 x 4096 of 16 of 128) 341 and 349; of 4 heads of 256, 8 chunks, forward
// 142 and 151, backward 315 and 325.  Short blocks stay one role after another: 2
// chunks (128 x 50 of 16 heads of 64) 39 and 39, 4 (64 x 100) 36 and 35, 7 (64 x 200)
// 63 and 63, 7 (32 x 200 of 8 of 128) 50 and 48; for heads of 256 the order pays from
// 4 chunks on (16 x 300, forward 61 and 65).
constexpr int GROUP_CHUNKS = 8;
template <typename T, int DA, bool OUT, int MT>
hipError_t launch_chunks(Roles<T> g, int roles, int width, hipStream_t s)
{
    constexpr int WCOLS = 16 * MT;
    constexpr int C = Mat<T>::C, CHA = row_chunks<T, DA>(), CHC = WCOLS * (int)sizeof(T) / 16;
    const int columns = (width + WCOLS - 1) / WCOLS, blocks = (columns + MAX_WAVES - 1) / MAX_WAVES;
    const int waves = (columns + blocks - 1) / blocks;   // of a block; the columns of a head may take two
    const int lds = 2 * ((OUT ? 2 : 1) * Tile<CHA>::bytes(C * CHA / 64) + waves * Tile<CHC>::bytes(C * CHC / 64));
    const long n = (long)g.B * g.N * g.parts;
    auto launch = [&](auto kernel, dim3 grid) {
        if (lds > 64 * 1024) {
            const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel),
                                                     hipFuncAttributeMaxDynamicSharedMemorySize, lds);
            if (e != hipSuccess) return e;
        }
        hipLaunchKernelGGL(kernel, grid, dim3(64 * waves), lds, s, g);
        return hipGetLastError();
    };
    if constexpr (MT == 2 || DA > 128)   // (with waves of 16 columns else, blocks have few chunks)
        if (roles * blocks > 1 && g.part_len >= GROUP_CHUNKS * C) {
            g.roles = roles;
            g.each = roles * blocks;   // at most 6
            g.inv_each = 0xffffffffu / g.each + 1;
            return launch(linattn_chunks_kernel<T, DA, OUT, MT, true>, dim3((unsigned)((n + 7) / 8 * 8 * g.each)));
        }
    return launch(linattn_chunks_kernel<T, DA, OUT, MT, false>, dim3((unsigned)n, roles, blocks));
}

// Roles of one launch: padded to the widest of them.
template <typename T, bool OUT>
hipError_t launch_roles(const Roles<T> &g, int roles, hipStream_t s)
{
    int da = 0, dc = 0;
    for (int k = 0; k < roles; ++k) {
        da = g.r[k].da > da ? g.r[k].da : da;
        dc = g.r[k].dc > dc ? g.r[k].dc : dc;
    }
    const bool one = g.tiles == 1;
    switch ((da + 31) / 32) {
    case 1: return one ? launch_chunks<T, 32, OUT, 1>(g, roles, dc, s) : launch_chunks<T, 32, OUT, 2>(g, roles, dc, s);
    case 2: return one ? launch_chunks<T, 64, OUT, 1>(g, roles, dc, s) : launch_chunks<T, 64, OUT, 2>(g, roles, dc, s);
    case 3: return one ? launch_chunks<T, 96, OUT, 1>(g, roles, dc, s) : launch_chunks<T, 96, OUT, 2>(g, roles, dc, s);
    case 4: return one ? launch_chunks<T, 128, OUT, 1>(g, roles, dc, s) : launch_chunks<T, 128, OUT, 2>(g, roles, dc, s);
    case 5: return launch_chunks<T, 160, OUT, 1>(g, roles, dc, s);
    case 6: return launch_chunks<T, 192, OUT, 1>(g, roles, dc, s);
    case 7: return launch_chunks<T, 224, OUT, 1>(g, roles, dc, s);
    default: return launch_chunks<T, 256, OUT, 1>(g, roles, dc, s);
    }
}

// Parts from which on their states are joined by a launch of its own.  A block's
// own joins cost it up to 1 us each, one after another; the launch takes 5 to
// 11 us.  Us joined by the blocks and by the launch:
//   heads of 64    forward   7 parts 22, 28 and 33, 33   10 29, 31   13 39, 36   21 36, 31
//                  backward  3 parts 55, 57   5 42, 45   6 56, 58 and 65, 61   11 66, 54
//   heads of 128   forward   4 parts 30, 35   7 39, 39   10 52, 45   16 74, 54
//                  backward  4 parts 60, 54   5 76, 67   6 96, 84 and 132, 114
//   40 x 72, fp32  forward   4 parts 22, 24   7 23, 22   8 28, 26   13 37, 35
//                  backward  4 parts 33, 35   7 45, 44   8 64, 55
// The larger a state and the more roles, the sooner the launch pays.
constexpr int JOIN_PARTS = 6;
template <typename T>
hipError_t launch_join(const Roles<T> &g, int roles, hipStream_t s)
{
    const int per = (g.r[0].da * g.r[0].dc / 4 + 255) / 256;
    hipLaunchKernelGGL(linattn_join_kernel<T>, dim3((unsigned)((long)g.B * g.N * per), roles), dim3(256), 0, s, g);
    return hipGetLastError();
}

// One token of one head per block: the state's rows are read four values per
// thread, M/4 threads to a row, and written back with the token's product.
// Bound by memory: 256 rows of 16 heads of 128 x 128 in 104 us (537 MB, 5.2
// TB/s); one row of 16 heads of 64 x 64 in 4 us, latency.
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
Roles<T> call_of(const LinAttnShape &sh, const float *decay, const int32_t *lengths, int roles)
{
    Roles<T> g{};
    const SplitPlan p = split_plan(sh, Mat<T>::C, roles);
    g.decay = decay;
    g.lengths = lengths;
    g.T_ = sh.T; g.B = sh.B; g.N = sh.N;
    g.parts = p.parts;
    g.part_len = p.len;
    g.tiles = p.tiles;
    g.joined = p.parts >= JOIN_PARTS;
    return g;
}

template <typename T>
hipError_t forward_t(const LinAttnShape &sh, const T *q, const T *k, const T *v, const float *decay,
                     const int32_t *lengths, const float *S0, T *o, float *ST, float *ws, hipStream_t s)
{
    Roles<T> g = call_of<T>(sh, decay, lengths, 1);
    g.r[0] = Role<T>{q, k, v, o, sh.ldq, sh.ldk, sh.ldv, sh.ldo, sh.K, sh.M, false, sh.scale, sh.scale, 1.0f, S0, ST,
                     sh.M, 1, ws};
    if (g.parts > 1) {
        hipError_t e = launch_roles<T, false>(g, 1, s);
        if (e == hipSuccess && g.joined) e = launch_join(g, 1, s);
        if (e != hipSuccess) return e;
    }
    return launch_roles<T, true>(g, 1, s);
}

template <typename T>
hipError_t backward_t(const LinAttnShape &sh, const T *d_o, const T *q, const T *k, const T *v, const float *decay,
                      const int32_t *lengths, const float *S0, const float *dST, T *dq, T *dk, T *dv, float *dS0,
                      float *ws, hipStream_t s)
{
    const int K = sh.K, M = sh.M;
    const float sc = sh.scale;
    Roles<T> g = call_of<T>(sh, decay, lengths, MAX_ROLES);
    // the states of dk and dv are each other's transposes: dv's slots serve both
    float *const ws2 = ws + (g.parts > 1 ? (size_t)sh.B * sh.N * g.parts * K * M : 0);
    const Role<T> rq{d_o, v, k, dq, sh.ldo, sh.ldv, sh.ldk, sh.ldq, M, K, false, sc, sc, 1.0f, S0, nullptr, 1, M, ws};
    const Role<T> rk{v, d_o, q, dk, sh.ldv, sh.ldo, sh.ldq, sh.ldk, M, K, true, sc, 1.0f, sc, dST, nullptr, 1, M, ws2};
    const Role<T> rv{k, q, d_o, dv, sh.ldk, sh.ldq, sh.ldo, sh.ldv, K, M, true, sc, 1.0f, sc, dST, dS0, M, 1, ws2};
    const bool back = dk || dv || dS0;
    if (g.parts > 1) {
        int n = 0;
        if (dq) g.r[n++] = rq;
        if (back) g.r[n++] = rv;
        hipError_t e = n ? launch_roles<T, false>(g, n, s) : hipSuccess;
        if (e == hipSuccess && n && g.joined) e = launch_join(g, n, s);
        if (e != hipSuccess) return e;
    }
    int n = 0;
    if (dq) g.r[n++] = rq;
    if (dk) g.r[n++] = rk;
    if (n && dS0 && dS0 == dST && g.parts == 1) {   // dk's blocks read dST before dv's replace it
        const hipError_t e = launch_roles<T, true>(g, n, s);
        if (e != hipSuccess) return e;
        n = 0;
    }
    if (dv || dS0) g.r[n++] = rv;
    return n ? launch_roles<T, true>(g, n, s) : hipSuccess;
}

}  // namespace

size_t linattn_workspace_bytes(DType t, const LinAttnShape &sh)
{
    const int chunk = t == DType::BF16 ? Mat<bf16_t>::C : Mat<float>::C;
    const size_t state = (size_t)sh.B * sh.N * sh.K * sh.M * 4;
    const int fwd = split_plan(sh, chunk, 1).parts, bwd = split_plan(sh, chunk, MAX_ROLES).parts;
    const size_t f = fwd > 1 ? fwd * state : 0, b = bwd > 1 ? 2 * bwd * state : 0;
    return f > b ? f : b;
}

hipError_t linattn_forward(DType t, const LinAttnShape &sh, const void *q, const void *k, const void *v,
                           const float *decay, const int32_t *lengths, const float *S0, void *o, float *ST, void *ws,
                           hipStream_t s)
{
    const double n = (double)sh.T * sh.B * sh.N;
    ProfScope ps(K_LINATTN, s, 4.0 * n * sh.K * sh.M, n * 2.0 * (sh.K + sh.M) * dsize(t));
    if (t == DType::BF16)
        return forward_t(sh, static_cast<const bf16_t *>(q), static_cast<const bf16_t *>(k),
                         static_cast<const bf16_t *>(v), decay, lengths, S0, static_cast<bf16_t *>(o), ST,
                         static_cast<float *>(ws), s);
    return forward_t(sh, static_cast<const float *>(q), static_cast<const float *>(k), static_cast<const float *>(v),
                     decay, lengths, S0, static_cast<float *>(o), ST, static_cast<float *>(ws), s);
}

hipError_t linattn_backward(DType t, const LinAttnShape &sh, const void *d_o, const void *q, const void *k,
                            const void *v, const float *decay, const int32_t *lengths, const float *S0,
                            const float *dST, void *dq, void *dk, void *dv, float *dS0, void *ws, hipStream_t s)
{
    const double n = (double)sh.T * sh.B * sh.N;
    ProfScope ps(K_LINATTN, s, 10.0 * n * sh.K * sh.M, n * (4.0 * sh.K + 3.0 * sh.M) * dsize(t));
    if (t == DType::BF16)
        return backward_t(sh, static_cast<const bf16_t *>(d_o), static_cast<const bf16_t *>(q),
                          static_cast<const bf16_t *>(k), static_cast<const bf16_t *>(v), decay, lengths, S0, dST,
                          static_cast<bf16_t *>(dq), static_cast<bf16_t *>(dk), static_cast<bf16_t *>(dv), dS0,
                          static_cast<float *>(ws), s);
    return backward_t(sh, static_cast<const float *>(d_o), static_cast<const float *>(q), static_cast<const float *>(k),
                      static_cast<const float *>(v), decay, lengths, S0, dST, static_cast<float *>(dq),
                      static_cast<float *>(dk), static_cast<float *>(dv), dS0, static_cast<float *>(ws), s);
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
