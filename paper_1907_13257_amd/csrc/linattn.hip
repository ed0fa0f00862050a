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
    float *parts;            // states of the parts [B*N][parts][da][dc], where the sequences are split
};
constexpr int MAX_ROLES = 3;
template <typename T>
struct Roles {
    Role<T> r[MAX_ROLES];
    const float *decay;
    const int32_t *lengths;
    int T_, B, N;
    int parts, part_len;     // parts of a sequence, their tokens (a multiple of the chunk)
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
// batch row (or a part of its tokens); each of its waves owns 32 columns of
// the state, which stay in its registers, and takes the chunk's rows of A and
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
// take in bf16 parts: two parts, hi = bf16(x) and lo = bf16(x - hi), leave out
// 2^-16 of a value, well below the rounding of the result; a state that is an
// output is updated with three parts (2^-24).
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
constexpr int MT = 2;              // result tiles of 16 columns per wave
constexpr int WCOLS = 16 * MT;

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
// 64 chunks, 64 / CH rows; instructions are 64 bytes more than that apart, and
// chunk c of a row stands at c ^ flip(row), flip being bits 2 and 3 of the row.
// Which rows an instruction takes and their order in it (bits b0 .. b3 of the
// row below) are such that, of the 256 bytes LDS serves at a time,
//   - the 16 rows one operand read touches at one chunk get 16 different places,
//   - the rows 0-7 (8-15) of half a transposing read get 8 different 32 bytes,
// while the address stays a lane's own offset plus a constant.
template <int CH>
struct Tile {
    static constexpr int PITCH = 1024 + 64;
    static constexpr int RPI = 64 / CH;    // rows of an instruction
    __device__ static constexpr int flip(int row) { return ((row >> 2) & 1) * 2 + ((row >> 3) & 1); }
    // instruction of a row, and its place there
    __device__ static constexpr int instr(int row)
    {
        const int hi = row >> 4;
        return CH == 64 ? row : CH == 32 ? (row & 7) + 8 * hi : CH == 16 ? (row & 3) + 4 * hi : CH == 8 ? (row & 1) + 2 * hi : hi;
    }
    __device__ static constexpr int place(int row)
    {
        const int b1 = (row >> 1) & 1, b3 = (row >> 3) & 1;
        return CH == 64 ? 0 : CH == 32 ? b3 : CH == 16 ? flip(row) : CH == 8 ? b1 + 2 * b3 + 4 * ((row >> 2) & 1)
                                                                             : (row & 3) + 4 * flip(row);
    }
    __device__ static constexpr int offset(int row) { return instr(row) * PITCH + place(row) * CH * 16; }
    // the row of place j of instruction k: row_k(k) + row_j(j)
    __device__ static constexpr int row_k(int k)
    {
        return CH == 64 ? k : CH == 32 ? (k & 7) + 16 * (k >> 3) : CH == 16 ? (k & 3) + 16 * (k >> 2)
                                                                   : CH == 8 ? (k & 1) + 16 * (k >> 1) : 16 * k;
    }
    __device__ static constexpr int row_j(int j)
    {
        return CH == 64 ? 0 : CH == 32 ? 8 * j : CH == 16 ? 4 * (j >> 1) + 8 * (j & 1)
                                       : CH == 8 ? 2 * (j & 1) + 8 * ((j >> 1) & 1) + 4 * (j >> 2)
                                                 : (j & 3) + 4 * ((j >> 3) & 1) + 8 * ((j >> 2) & 1);
    }
};

// Instruction k of a tile: rows of `width` elements, `step` apart, `rows` of
// them; zeros elsewhere.
template <typename T, int CH>
__device__ __forceinline__ void load_rows(const T *base, long step, int rows, int width, int k, unsigned tile, int lane)
{
    constexpr int E = 16 / (int)sizeof(T);
    const int row = Tile<CH>::row_k(k) + Tile<CH>::row_j(lane / CH), c = (lane % CH) ^ Tile<CH>::flip(row);
    const bool in = row < rows && c * E < width;
    const void *p = in ? static_cast<const void *>(base + row * step + c * E) : static_cast<const void *>(zero_chunk);
    dma16_from(p, __builtin_amdgcn_readfirstlane(tile + (unsigned)(k * Tile<CH>::PITCH)));
}

// Where a lane finds the operands of a tile.
template <int CH, typename T> struct Reader;
template <int CH>
struct Reader<CH, bf16_t> {
    unsigned row0, row1, col0, col1;
    __device__ __forceinline__ void init(int c16, int q)
    {
        // rows c16: 8 bytes at columns 4q and 16 + 4q of 32
        const int f = Tile<CH>::flip(c16);
        row0 = Tile<CH>::offset(c16) + ((q >> 1) ^ f) * 16 + (q & 1) * 8;
        row1 = row0 ^ 32;
        // columns: in each group of 16 lanes, lane s addresses the 8 bytes of
        // row 4q + s/4 and columns 4 (s%4); lane i receives four rows of column i
        const int r = 4 * q + (c16 >> 2);
        col0 = Tile<CH>::offset(r) + (((c16 & 3) >> 1) ^ Tile<CH>::flip(r)) * 16 + (c16 & 1) * 8;
        col1 = col0 ^ 32;
    }
    // row 16 s + c16 at column block kb
    __device__ __forceinline__ u32x4 row(lds_char *tile, int s, int kb) const
    {
        const int at = Tile<CH>::offset(16 * s) + kb * 64;
        const u32x2 lo = *(lds_u32x2_t *)(tile + row0 + at), hi = *(lds_u32x2_t *)(tile + row1 + at);
        return u32x4{lo[0], lo[1], hi[0], hi[1]};
    }
    // columns 16 ct .. 16 ct + 15 over the tile's rows
    __device__ __forceinline__ u32x4 col(lds_char *tile, int ct) const
    {
        lds_char *p = tile + (ct & 1 ? col1 : col0) + (ct >> 1) * 64;
        const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t *)p));
        const u32x2 hi = __builtin_bit_cast(
            u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t *)(p + Tile<CH>::offset(16))));
        return u32x4{lo[0], lo[1], hi[0], hi[1]};
    }
};
template <int CH>
struct Reader<CH, float> {
    unsigned row0, col0;
    __device__ __forceinline__ void init(int c16, int q)
    {
        row0 = Tile<CH>::offset(c16) + (q ^ Tile<CH>::flip(c16)) * 16;
        col0 = Tile<CH>::offset(4 * q) + ((c16 >> 2) ^ Tile<CH>::flip(4 * q)) * 16 + (c16 & 3) * 4;
    }
    __device__ __forceinline__ u32x4 row(lds_char *tile, int, int kb) const
    {
        return *(lds_u32x4_t *)(tile + row0 + kb * 64);
    }
    __device__ __forceinline__ u32x4 col(lds_char *tile, int ct) const
    {
        u32x4 f;
#pragma unroll
        for (int e = 0; e < 4; ++e) f[e] = *(lds_u32_t *)(tile + col0 + Tile<CH>::offset(e) + ct * 64);
        return f;
    }
};

__device__ __forceinline__ unsigned pack_bf16(float a, float b)
{
    return (unsigned)f32_to_bf16(a) | ((unsigned)f32_to_bf16(b) << 16);
}

// fp32 values of an operand as the parts the matrix cores take.
template <int NP>
__device__ __forceinline__ void split(const float (&x)[8], u32x4 (&f)[NP], bf16_t)
{
    float r[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = x[e];
#pragma unroll
    for (int p = 0; p < NP; ++p)
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
            const unsigned w = pack_bf16(r[e], r[e + 1]);
            f[p][e / 2] = w;
            if (p + 1 < NP) {
                r[e] -= __uint_as_float(w << 16);
                r[e + 1] -= __uint_as_float(w & 0xffff0000u);
            }
        }
}
template <int NP>
__device__ __forceinline__ void split(const float (&x)[4], u32x4 (&f)[NP], float)
{
    f[0] = __builtin_bit_cast(u32x4, f32x4{x[0], x[1], x[2], x[3]});
}

// Four consecutive values of an output row.
template <typename T> struct Out4;
template <> struct Out4<bf16_t> { u32x2 v; };
template <> struct Out4<float> { f32x4 v; };
__device__ __forceinline__ Out4<bf16_t> out4(f32x4 a, bf16_t) { return {u32x2{pack_bf16(a[0], a[1]), pack_bf16(a[2], a[3])}}; }
__device__ __forceinline__ Out4<float> out4(f32x4 a, float) { return {a}; }

// OUT: rows of the output, from the state at the start of the part (and the
// final state where nothing is split); else the state a part adds, from zero.
// NP: parts of the state's update (bf16).
template <typename T, int DA, bool OUT, int NP>
__global__ __launch_bounds__(512) void linattn_chunks_kernel(Roles<T> g)
{
    constexpr int C = Mat<T>::C, TT = Mat<T>::TT, E = C / 4;   // E: values of an operand per lane
    constexpr int CHA = DA * (int)sizeof(T) / 16, CHC = WCOLS * (int)sizeof(T) / 16;
    constexpr int KB = DA / C, KT = DA / 16;
    constexpr int NA = C * CHA / 64, NC = C * CHC / 64;        // load instructions of a tile
    constexpr int ABYTES = NA * Tile<CHA>::PITCH, CBYTES = NC * Tile<CHC>::PITCH;
    constexpr int SP = sizeof(T) == 2 ? 2 : 1;                 // parts of X and P
    extern __shared__ __align__(16) char lds[];
    const Role<T> &r = g.r[blockIdx.y];
    const int waves = blockDim.x >> 6, lane = threadIdx.x & 63, q = lane >> 4, c16 = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int h = blockIdx.x % g.N, b = (int)((blockIdx.x / g.N) % g.B), part = (int)(blockIdx.x / g.N / g.B);
    const long bh = (long)b * g.N + h;
    const int n = sequence_length(g.lengths, b, g.T_);
    const int begin = part * g.part_len, stop = min(g.T_, begin + g.part_len), end = min(n, stop);
    const int da = r.da, dc = r.dc, col0 = wave * WCOLS;

    if (OUT && !r.out && g.parts > 1) return;   // the final state is known
    if (OUT && r.out)   // behind the sequence's end
        for (int t = max(n, begin); t < stop; ++t)
            for (int c = threadIdx.x; c < dc; c += blockDim.x)
                r.out[((long)t * g.B + b) * r.ldo + (long)h * dc + c] = from_f32<T>(0.0f);
    if (begin >= end && (part > 0 || !OUT)) return;

    // rows of token i of the sequence: at + i * step
    const long first = r.reverse ? (long)(n - 1) * g.B + b : b, dir = r.reverse ? -g.B : g.B;
    const T *A = r.a + first * r.lda + (long)h * da, *Bp = r.b + first * r.ldb + (long)h * da;
    const T *Cp = r.c + first * r.ldc + (long)h * dc + col0;
    const long sa = dir * r.lda, sb = dir * r.ldb, sc = dir * r.ldc;

    // LDS: two buffers of A, B and every wave's columns of C
    const int buf_bytes = (OUT ? 2 : 1) * ABYTES + waves * CBYTES;
    const unsigned lds0 = lds_addr(lds);
    auto issue = [&](int t0, int buf) {
        const unsigned base = lds0 + (unsigned)(buf * buf_bytes);
        const int rows = min(C, end - t0);
        for (int k = wave; k < NA; k += waves) {
            load_rows<T, CHA>(Bp + t0 * sb, sb, rows, da, k, base, lane);
            if (OUT) load_rows<T, CHA>(A + t0 * sa, sa, rows, da, k, base + ABYTES, lane);
        }
#pragma unroll
        for (int k = 0; k < NC; ++k)
            load_rows<T, CHC>(Cp + t0 * sc, sc, rows, dc - col0, k, base + (OUT ? 2 : 1) * ABYTES + wave * CBYTES, lane);
    };
    if (begin < end) issue(begin, 0);

    // the state: element (16 kt + 4 q + v, col0 + 16 mt + c16) in X[kt][mt][v]
    f32x4 X[KT][MT];
    const float *start = !OUT ? nullptr : g.parts > 1 ? r.parts + (bh * g.parts + part) * da * dc
                                                      : (r.X0 ? r.X0 + bh * da * dc : nullptr);
    const int si = g.parts > 1 ? dc : r.si, sj = g.parts > 1 ? 1 : r.sj;
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const int i = 16 * kt + 4 * q + v, j = col0 + 16 * mt + c16;
                X[kt][mt][v] = start && i < da && j < dc ? start[i * si + j * sj] : 0.0f;
            }
    bool zero = !start;   // X is zero

    const float lg = decay_log2(g.decay[h]);
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
    float whole = 1.0f;   // the state's factor over that chunk

    Reader<CHA, T> ra;
    Reader<CHC, T> rc;
    ra.init(c16, q);
    rc.init(c16, q);
    Out4<T> held[TT][MT];   // the last chunk's output, stored while the next one is computed
    auto store = [&](int t0) {
        if (!r.out) return;
#pragma unroll
        for (int ti = 0; ti < TT; ++ti) {
            const int t = t0 + 16 * ti + c16;
            if (t >= end) continue;
            T *row = r.out + (first + t * dir) * r.ldo + (long)h * dc + col0 + 4 * q;
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
                if (col0 + 16 * mt + 4 * q < dc) *reinterpret_cast<Out4<T> *>(row + 16 * mt) = held[ti][mt];
        }
    };

    int buf = 0;
    for (int t0 = begin; t0 < end; t0 += C, buf ^= 1) {
        waitcnt_vm<0>();   // this chunk's rows
        __syncthreads();   // everyone's; and the other buffer has been read
        if (t0 + C < end) issue(t0 + C, buf ^ 1);
        if (OUT && t0 > begin) store(t0 - C);
        lds_char *tb = (lds_char *)lds + buf * buf_bytes, *ta = tb + ABYTES;
        lds_char *tc = tb + (OUT ? 2 : 1) * ABYTES + wave * CBYTES;
        const int rows = min(C, end - t0);

        u32x4 ct[MT];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) ct[mt] = rc.col(tc, mt);

        if constexpr (OUT) {
            // X^T A^T, and P^T: tile of tokens s (rows) by tile of tokens ti (columns)
            f32x4 o[TT][MT], P[TT][TT];
#pragma unroll
            for (int ti = 0; ti < TT; ++ti) {
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) o[ti][mt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int s = 0; s <= ti; ++s) P[s][ti] = f32x4{0.f, 0.f, 0.f, 0.f};
            }
#pragma unroll
            for (int kb = 0; kb < KB; ++kb) {
                u32x4 a[TT];
#pragma unroll
                for (int ti = 0; ti < TT; ++ti) a[ti] = ra.row(ta, ti, kb);
#pragma unroll
                for (int s = 0; s < TT; ++s) {
                    const u32x4 bf = ra.row(tb, s, kb);
#pragma unroll
                    for (int ti = s; ti < TT; ++ti) mfma16(P[s][ti], bf, a[ti], T());
                }
                if (!zero)
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt) {
                        float x[E];
#pragma unroll
                        for (int e = 0; e < E; ++e) x[e] = X[TT * kb + e / 4][mt][e % 4];
                        u32x4 f[SP];
                        split<SP>(x, f, T());
#pragma unroll
                        for (int p = 0; p < SP; ++p)
#pragma unroll
                            for (int ti = 0; ti < TT; ++ti) mfma16(o[ti][mt], f[p], a[ti], T());
                    }
            }
#pragma unroll
            for (int ti = 0; ti < TT; ++ti)
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) o[ti][mt] *= rowf[ti];
#pragma unroll
            for (int ti = 0; ti < TT; ++ti) {
                float x[E];
#pragma unroll
                for (int e = 0; e < E; ++e)
                    x[e] = e / 4 > ti ? 0.0f : P[e / 4][ti][e % 4] * (e / 4 == ti ? w0[e % 4] : w1[e % 4]);
                u32x4 f[SP];
                split<SP>(x, f, T());
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
                    for (int p = 0; p < SP; ++p) mfma16(o[ti][mt], ct[mt], f[p], T());
                    held[ti][mt] = out4(o[ti][mt], T());
                }
            }
        }

        // the state behind the chunk
        if (!OUT || t0 + C < end || (g.parts == 1 && r.XT)) {
            if (rows != wc_rows) {
                wc_rows = rows;
                whole = decay_pow(lg, rows);
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const int left = rows - 1 - (16 * (e / 4) + 4 * q + e % 4);
                    wc[e] = left < 0 ? 0.0f : r.update * decay_pow(lg, left + 1 - pre);
                }
            }
            u32x4 f[MT][NP];
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                float x[E];
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    if constexpr (sizeof(T) == 2)
                        x[e] = __uint_as_float(e % 2 ? ct[mt][e / 2] & 0xffff0000u : ct[mt][e / 2] << 16) * wc[e];
                    else
                        x[e] = __uint_as_float(ct[mt][e]) * wc[e];
                }
                split<NP>(x, f[mt], T());
            }
#pragma unroll
            for (int kt = 0; kt < KT; ++kt) {
                const u32x4 bt = ra.col(tb, kt);
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    X[kt][mt] *= whole;
#pragma unroll
                    for (int p = 0; p < NP; ++p) mfma16(X[kt][mt], bt, f[mt][p], T());
                }
            }
            zero = false;
        }
    }
    if (OUT && begin < end) store(begin + (end - 1 - begin) / C * C);

    // the part's state, or the sequence's final one
    float *fin = !OUT ? r.parts + (bh * g.parts + part) * da * dc : (g.parts == 1 && r.XT ? r.XT + bh * da * dc : nullptr);
    if (!fin) return;
    const int fi = OUT ? r.si : dc, fj = OUT ? r.sj : 1;
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const int i = 16 * kt + 4 * q + v, j = col0 + 16 * mt + c16;
                if (i < da && j < dc) fin[i * fi + j * fj] = X[kt][mt][v];
            }
}

// The parts' states, in order: on entry what each part adds, on exit the state
// at its start; and the final state.
template <typename T>
__global__ __launch_bounds__(256) void linattn_scan_kernel(Roles<T> g)
{
    const Role<T> &r = g.r[blockIdx.y];
    const int per = (r.da * r.dc + 255) / 256;
    const long bh = blockIdx.x / per;
    const int e = (int)(blockIdx.x % per) * 256 + threadIdx.x;
    if (e >= r.da * r.dc) return;
    const int n = sequence_length(g.lengths, (int)(bh / g.N), g.T_);
    const float lg = decay_log2(g.decay[bh % g.N]);
    const long at = bh * r.da * r.dc + (e / r.dc) * r.si + (e % r.dc) * r.sj;
    float x = r.X0 ? r.X0[at] : 0.0f;
    float *p = r.parts + bh * g.parts * (long)(r.da * r.dc) + e;
    for (int k = 0; k < g.parts && k * g.part_len < n; ++k, p += r.da * r.dc) {
        const float add = *p;
        *p = x;
        x = decay_pow(lg, min(g.part_len, n - k * g.part_len)) * x + add;
    }
    if (r.XT) r.XT[at] = x;
}

struct SplitPlan {
    int parts, len;
};

// Parts a sequence is split into: as many as it takes to give the chip
// TARGET_WAVES waves, but none shorter than MIN_CHUNKS chunks.
constexpr int TARGET_WAVES = 2048, MIN_CHUNKS = 4;
SplitPlan split_plan(const LinAttnShape &sh, int chunk, int roles, int dc)
{
    const long waves = (long)sh.B * sh.N * roles * ((dc + WCOLS - 1) / WCOLS);
    const int chunks = (sh.T + chunk - 1) / chunk;
    long parts = (TARGET_WAVES + waves - 1) / waves;
    const long most = chunks / MIN_CHUNKS;
    if (parts > most) parts = most;
    if (parts < 1) parts = 1;
    const int per = (int)((chunks + parts - 1) / parts);
    return SplitPlan{(chunks + per - 1) / per, per * chunk};
}

template <typename T, int DA, bool OUT, int NP>
hipError_t launch_chunks(const Roles<T> &g, int roles, hipStream_t s)
{
    constexpr int C = Mat<T>::C;
    const int waves = (g.r[0].dc + WCOLS - 1) / WCOLS;
    constexpr int CHA = DA * (int)sizeof(T) / 16, CHC = WCOLS * (int)sizeof(T) / 16;
    const int lds = 2 * (C * CHA / 64 * (OUT ? 2 : 1) * Tile<CHA>::PITCH + C * CHC / 64 * waves * Tile<CHC>::PITCH);
    if (lds > 64 * 1024) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(linattn_chunks_kernel<T, DA, OUT, NP>),
                                                 hipFuncAttributeMaxDynamicSharedMemorySize, lds);
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL((linattn_chunks_kernel<T, DA, OUT, NP>), dim3((unsigned)((long)g.B * g.N * g.parts), roles),
                       dim3(64 * waves), lds, s, g);
    return hipGetLastError();
}

template <typename T, bool OUT, int NP>
hipError_t launch_width(const Roles<T> &g, int roles, hipStream_t s)
{
    const int da = g.r[0].da;
    if (da <= 32) return launch_chunks<T, 32, OUT, NP>(g, roles, s);
    if (da <= 64) return launch_chunks<T, 64, OUT, NP>(g, roles, s);
    if (da <= 128) return launch_chunks<T, 128, OUT, NP>(g, roles, s);
    return launch_chunks<T, 256, OUT, NP>(g, roles, s);
}

// Roles of equal widths, at once; `planned` of them if all were wanted (results
// do not depend on which are).  `states`: the call carries states, so that one
// may be an output.  `parts`: workspace of all roles.
template <typename T>
hipError_t launch_roles(Roles<T> &g, int roles, int planned, bool states, const LinAttnShape &sh, float *parts, hipStream_t s)
{
    const SplitPlan p = split_plan(sh, Mat<T>::C, planned, g.r[0].dc);
    g.T_ = sh.T; g.B = sh.B; g.N = sh.N;
    g.parts = p.parts;
    g.part_len = p.len;
    for (int k = 0; k < roles; ++k)
        g.r[k].parts = parts + (size_t)k * sh.B * sh.N * p.parts * sh.K * sh.M;
    constexpr int MORE = sizeof(T) == 2 ? 3 : 1, FEWER = sizeof(T) == 2 ? 2 : 1;
    hipError_t e;
    if (p.parts > 1) {
        e = states ? launch_width<T, false, MORE>(g, roles, s) : launch_width<T, false, FEWER>(g, roles, s);
        if (e != hipSuccess) return e;
        const int per = (sh.K * sh.M + 255) / 256;
        hipLaunchKernelGGL(linattn_scan_kernel<T>, dim3((unsigned)((long)sh.B * sh.N * per), roles), dim3(256), 0, s, g);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
        states = false;
    }
    return states ? launch_width<T, true, MORE>(g, roles, s) : launch_width<T, true, FEWER>(g, roles, s);
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
                     const int32_t *lengths, const float *S0, T *o, float *ST, float *ws, hipStream_t s)
{
    Roles<T> g{};
    g.decay = decay;
    g.lengths = lengths;
    g.r[0] = Role<T>{q, k, v, o, sh.ldq, sh.ldk, sh.ldv, sh.ldo, sh.K, sh.M, false, sh.scale, sh.scale, 1.0f, S0, ST,
                     sh.M, 1, nullptr};
    return launch_roles(g, 1, 1, S0 || ST, sh, ws, s);
}

template <typename T>
hipError_t backward_t(const LinAttnShape &sh, const T *d_o, const T *q, const T *k, const T *v, const float *decay,
                      const int32_t *lengths, const float *S0, const float *dST, T *dq, T *dk, T *dv, float *dS0,
                      float *ws, hipStream_t s)
{
    const int K = sh.K, M = sh.M;
    const float sc = sh.scale;
    const bool states = S0 || dST || dS0;
    const Role<T> rq{d_o, v, k, dq, sh.ldo, sh.ldv, sh.ldk, sh.ldq, M, K, false, sc, sc, 1.0f, S0, nullptr, 1, M, nullptr};
    const Role<T> rk{v, d_o, q, dk, sh.ldv, sh.ldo, sh.ldq, sh.ldk, M, K, true, sc, 1.0f, sc, dST, nullptr, 1, M, nullptr};
    const Role<T> rv{k, q, d_o, dv, sh.ldk, sh.ldq, sh.ldo, sh.ldv, K, M, true, sc, 1.0f, sc, dST, dS0, M, 1, nullptr};
    Roles<T> g{};
    g.decay = decay;
    g.lengths = lengths;
    int n = 0;
    if (dq) g.r[n++] = rq;
    if (dk) g.r[n++] = rk;
    if (K == M && (dv || dS0)) g.r[n++] = rv;   // equal widths: all in one launch
    if (n) {
        const hipError_t e = launch_roles(g, n, K == M ? 3 : 2, states, sh, ws, s);
        if (e != hipSuccess) return e;
    }
    if (K != M && (dv || dS0)) {
        g.r[0] = rv;
        return launch_roles(g, 1, 1, states, sh, ws, s);
    }
    return hipSuccess;
}

}  // namespace

size_t linattn_workspace_bytes(DType t, const LinAttnShape &sh)
{
    const int chunk = t == DType::BF16 ? Mat<bf16_t>::C : Mat<float>::C;
    const size_t state = (size_t)sh.B * sh.N * sh.K * sh.M * 4;
    size_t most = 0;
    for (int roles = 1; roles <= MAX_ROLES; ++roles)
        for (const int dc : {sh.K, sh.M}) {
            const SplitPlan p = split_plan(sh, chunk, roles, dc);
            if (p.parts > 1 && p.parts * roles * state > most) most = p.parts * roles * state;
        }
    return most;
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
