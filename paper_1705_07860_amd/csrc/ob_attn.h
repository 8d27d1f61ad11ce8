// Decay attention on packed sequences: the kernels, for one element type a translation unit (ob_attn_*.hip instantiates them).
//
// One kernel serves the forward pass and all three gradients, which are scans of one launch where their widths take the same tiles.  For rows a_i, b_j, c_j of one head in the order of the scan it makes
//     y_i = sp * sum_{j <= i} lambda^(i-j) (a_i . b_j) c_j  +  sy * lambda^(i+once) a_i S
// chunk by chunk, S being the DA x DC state at the chunk's start, and carries S' = lambda^n S + ss * sum_j lambda^(n-once'-j) b_j c_j^T on:
//     o  : a, b, c = q, k, v                        S the state behind the token before the chunk
//     dq : a, b, c = do, v, k                       the same state, transposed
//     dv : a, b, c = k, q, do, tokens reversed      S the gradient of the state behind the chunk's first row
//     dk : a, b, c = v, do, q, tokens reversed      the same, transposed
// (backward: dS_t = lambda dS_(t+1) + scale q_t do_t^T, dk_t = dS_t v_t, dv_t = dS_t^T k_t, dq_t = scale S_t do_t.)
#pragma once

#include "ob_dev.h"

constexpr int ATT_SEQS = 512;      // sequences of one launch: its tables travel in the 4 KiB of kernel arguments, so nothing is copied or kept
constexpr int ATT_SPLIT = 96;      // of these, the ones that are cut into segments
constexpr int CH = 32;             // rows of a chunk

struct Rows {
    const void *p;
    i64 token, head;               // strides in elements
    int div;                       // query heads that share one of these heads
    int pad;
};

struct Scan {
    Rows a, b, c;
    void *y;
    i64 y_token, y_head;
    const float *s_in;             // [sequence][head] planes, element (row, column) at row * s_row + column * s_col; null: zeros
    float *s_out;
    float sp, ss, sy;
    int da, dc, s_row, s_col;
    int reverse, y_float, exact_state;
};
constexpr int ATT_SCANS = 3;       // of one launch, over the same sequences and tiles

struct ScanArgs {
    const float *log_decay;
    float *slots;                  // states of segments, in the layout of the registers, scan by scan
    int n_scans, heads;
    int segment;                   // tokens of a segment
    int n_units, n_split, n_cut, first_seq;    // n_cut: units of the first n_split sequences of the order
    int ordered;                   // the sequences are in order as they are
    Scan scan[ATT_SCANS];
    u32 off[ATT_SEQS + 1];         // first token of each sequence
    uint16_t order[ATT_SEQS];      // sequences, the longest first
    u32 cum[ATT_SPLIT + 1];        // units before each of the first n_split sequences of the order
};
static_assert(sizeof(ScanArgs) <= 4096 - 16, "kernel arguments");

// ---- matrix tiles ----------------------------------------------------------------------------------------------------
// Operands go by 16 x 16 blocks.  A lane holds, of a block, index (lane & 15) of the outer dimension and the four elements
// 4 (lane >> 4) .. + 3 of the summed one; a result block has its column at lane & 15 and its rows at the same four places.  So a result is,
// as it stands, an operand of the next product whose summed index is its row: the state goes from accumulator to operand without leaving the
// registers.  The order of the summed index inside one instruction is free, hence one instruction of depth 32 takes two blocks.

template <typename T> struct Tile;

template <> struct Tile<bf16> {
    typedef s4 Frag;
    static constexpr int PAD = 16;         // elements behind a row
    static constexpr int ODD = 8;          // elements that rows 8 .. 15 of 16 are moved by
    static constexpr int SPLIT = 3;        // terms of 8 bits that hold 24
    static constexpr int BUFFERS = 2;
    static constexpr bool SCALED = false;
    static __device__ __forceinline__ f4 mma(Frag a0, Frag a1, Frag b0, Frag b1, f4 acc)
    {
        typedef bf16 V __attribute__((ext_vector_type(8)));
        const s8 a = __builtin_shufflevector(a0, a1, 0, 1, 2, 3, 4, 5, 6, 7), b = __builtin_shufflevector(b0, b1, 0, 1, 2, 3, 4, 5, 6, 7);
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(V, a), __builtin_bit_cast(V, b), acc, 0, 0, 0);
    }
};
template <> struct Tile<f16> {
    typedef s4 Frag;
    static constexpr int PAD = 16;
    static constexpr int ODD = 8;
    static constexpr int SPLIT = 2;        // terms of 11 bits
    static constexpr int BUFFERS = 2;
    static constexpr bool SCALED = true;   // sums and states pass the range of fp16: they enter products with a common power of two taken out
    static __device__ __forceinline__ f4 mma(Frag a0, Frag a1, Frag b0, Frag b1, f4 acc)
    {
        typedef f16 V __attribute__((ext_vector_type(8)));
        const s8 a = __builtin_shufflevector(a0, a1, 0, 1, 2, 3, 4, 5, 6, 7), b = __builtin_shufflevector(b0, b1, 0, 1, 2, 3, 4, 5, 6, 7);
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(V, a), __builtin_bit_cast(V, b), acc, 0, 0, 0);
    }
};
template <> struct Tile<float> {
    typedef f4 Frag;
    static constexpr int PAD = 4;
    static constexpr int ODD = 0;
    static constexpr int SPLIT = 1;
    static constexpr int BUFFERS = 1;
    static constexpr bool SCALED = false;
    static __device__ __forceinline__ f4 mma(Frag a0, Frag a1, Frag b0, Frag b1, f4 acc)
    {
#pragma unroll
        for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(a0[e], b0[e], acc, 0, 0, 0);
#pragma unroll
        for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(a1[e], b1[e], acc, 0, 0, 0);
        return acc;
    }
};

// four fp32 numbers as operand elements, rounded to nearest
template <typename T> __device__ __forceinline__ typename Tile<T>::Frag to_frag(f4 x)
{
    if constexpr (std::is_same<T, float>::value) return x;
    else {
        typedef T V __attribute__((ext_vector_type(4)));
        return __builtin_bit_cast(s4, __builtin_convertvector(x, V));
    }
}
template <typename T> __device__ __forceinline__ f4 from_frag(typename Tile<T>::Frag x)
{
    if constexpr (std::is_same<T, float>::value) return x;
    else {
        typedef T V __attribute__((ext_vector_type(4)));
        return __builtin_convertvector(__builtin_bit_cast(V, x), f4);
    }
}

// Place of a row in LDS.  Rows start 8 of the 64 banks apart (times an odd number), so that a transposing read, 8 rows of 32 bytes for half a
// wave, meets no bank twice; rows 8 .. 15 another 4 further, so that a read of 16 bytes from each of 16 rows doesn't either (without
// that step these cost twice as much and LDS was what a chunk waited for: 281 of 508 us on 43 628 tokens of 32 heads).  fp32 reads 16
// bytes of 16 rows, or 16 neighbours of 4 rows that are 4 apart: rows 4 banks apart serve both.
template <typename T> __device__ __forceinline__ int row_place(int row, int ld) { return row * ld + (Tile<T>::ODD ? (row & 8) * (Tile<T>::ODD / 8) : 0); }

// operand from rows: outer index = row r0 + (lane & 15), summed index = column k0 + 4 (lane >> 4) + e
template <typename T> __device__ __forceinline__ typename Tile<T>::Frag rows_frag(const T *x, int ld, int r0, int k0, int lane)
{
    return *(const typename Tile<T>::Frag *)(x + r0 * ld + row_place<T>(lane & 15, ld) + k0 + 4 * (lane >> 4));
}

// operand from columns: outer index = column c0 + (lane & 15), summed index = row r0 + 4 (lane >> 4) + e.  16 lanes read a 4 x 16 block of
// 16-bit elements, four of a row each, and get its columns (the transposing read of LDS).
template <typename T> __device__ __forceinline__ typename Tile<T>::Frag cols_frag(const T *x, int ld, int r0, int c0, int lane)
{
    if constexpr (std::is_same<T, float>::value) {
        f4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = x[(r0 + 4 * (lane >> 4) + e) * ld + c0 + (lane & 15)];
        return v;
    } else {
        typedef __attribute__((address_space(3))) s4 *Local;
        const T *p = x + r0 * ld + row_place<T>(4 * (lane >> 4) + ((lane & 15) >> 2), ld) + c0 + 4 * (lane & 3);
        return __builtin_amdgcn_ds_read_tr16_b64_v4i16((Local)(s4 *)p);
    }
}

// the largest of the lanes' non-negative 32-bit numbers, in every lane
__device__ __forceinline__ int wave_max(int x)
{
    x = max(x, __builtin_amdgcn_mov_dpp(x, 0xB1, 0xf, 0xf, true));    // quad: 1 0 3 2
    x = max(x, __builtin_amdgcn_mov_dpp(x, 0x4E, 0xf, 0xf, true));    // quad: 2 3 0 1
    x = max(x, __builtin_amdgcn_mov_dpp(x, 0x141, 0xf, 0xf, true));   // halves of a row mirrored
    x = max(x, __builtin_amdgcn_mov_dpp(x, 0x140, 0xf, 0xf, true));   // rows mirrored
    const int a = max(__builtin_amdgcn_readlane(x, 0), __builtin_amdgcn_readlane(x, 16));
    const int b = max(__builtin_amdgcn_readlane(x, 32), __builtin_amdgcn_readlane(x, 48));
    return max(a, b);
}
__device__ __forceinline__ int bits_of(float x) { return __builtin_bit_cast(int, __builtin_fabsf(x)); }
constexpr int BITS_INF = 0x7f800000;
// the same, 0 of what is no finite number: a range is that of the finite ones, which an infinity beside them may not push out of fp16
__device__ __forceinline__ int finite_bits(float x)
{
    const int b = bits_of(x);
    return b < BITS_INF ? b : 0;
}
// the power of two that brings a finite magnitude (its bits) to 2^11 .. 2^12, as an exponent: products keep 26 binary places below the largest.
// -116 .. 126: itself and its inverse are normal numbers; what is below 2^-115 stays smaller.
__device__ __forceinline__ int fit_exponent(int bits) { return 11 - max((bits >> 23) - 127, -115); }
__device__ __forceinline__ float two_to(int e) { return __builtin_amdgcn_ldexpf(1.0f, e); }

// ---- rows of a chunk -------------------------------------------------------------------------------------------------
// From memory to LDS through registers: 16 bytes a thread and step where a row has them; the elements behind a row's last 16 bytes one by one.
// Columns at and beyond the width, and rows behind the last, are zeros.
template <typename T, int D, int THREADS, bool FULL> struct ChunkRows {
    static constexpr int VEC = 16 / (int)sizeof(T);
    static constexpr int PER_ROW = D / VEC, ROWS = THREADS / PER_ROW;
    static constexpr int N = ROWS > CH ? 1 : CH / ROWS;             // more rows than there are: the threads of the others rest
    static constexpr int TAIL = CH * VEC > THREADS ? CH * VEC / THREADS : 1;
    static_assert((ROWS > CH || CH % ROWS == 0) && THREADS % PER_ROW == 0 && THREADS % VEC == 0, "tiles of whole steps");
    typedef typename Pack<T, VEC>::V V;
    V r[N];
    T e[TAIL];
    const char *base;               // the same for all threads: the row of the next chunk that lies first in memory
    i64 next;                       // bytes from chunk to chunk
    int step;                       // bytes from row to row in the order of the scan
    u32 off, tail;                  // bytes to the thread's first 16 bytes, and to its element behind the last 16 of a row
    int cols, rest, at;             // columns from the thread's first on; elements behind the last 16 bytes; their first column

    __device__ __forceinline__ void begin(const Rows &x, i64 token, int head, int width, bool reverse, int tid)
    {
        const int bytes = (int)x.token * (int)sizeof(T);            // the entry holds it below 2^26
        base = (const char *)x.p + (token * x.token + head / x.div * x.head) * (i64)sizeof(T);
        step = reverse ? -bytes : bytes, next = (i64)CH * step;
        const u32 first = reverse ? (CH - 1) * bytes : 0;
        base -= first;
        cols = width - tid % PER_ROW * VEC;
        rest = width % VEC, at = width - rest;
        off = first + tid / PER_ROW * step + tid % PER_ROW * 16;
        tail = first + tid / VEC * step + (at + tid % VEC) * (int)sizeof(T);
    }
    // the next chunk, `left` rows from its first on
    __device__ __forceinline__ void load(int left, int tid)
    {
        const int row = tid / PER_ROW, rows = min(left, CH);
#pragma unroll
        for (int k = 0; k < N; ++k) {
            if constexpr (FULL && ROWS <= CH) {         // rows behind the last: the last one, put as zeros
                const int behind = row + k * ROWS - (rows - 1);
                r[k] = load_n<T, VEC>((const T *)(base + (u32)(off + k * ROWS * step - max(behind, 0) * step)));
            } else {
                r[k] = V{};
                if (row + k * ROWS < rows && cols >= VEC) r[k] = load_n<T, VEC>((const T *)(base + (u32)(off + k * ROWS * step)));
            }
        }
        if (!FULL && rest)
#pragma unroll
            for (int k = 0; k < TAIL; ++k) {
                e[k] = (T)0.0f;
                if (tid / VEC + k * (THREADS / VEC) < rows && tid % VEC < rest) e[k] = *(const T *)(base + (u32)(tail + k * (THREADS / VEC) * step));
            }
        base += next;
    }
    // `left`: rows from the chunk's first on
    __device__ __forceinline__ void put(T *lds, int ld, int tid, int left)
    {
        if constexpr (FULL && ROWS <= CH)
            if (left < CH)
#pragma unroll
                for (int k = 0; k < N; ++k)
                    if (tid / PER_ROW + k * ROWS >= left) r[k] = V{};
        if ((FULL || cols >= VEC || cols <= 0) && (ROWS <= CH || tid / PER_ROW < CH))
#pragma unroll
            for (int k = 0; k < N; ++k) *(V *)(lds + row_place<T>(k * ROWS + tid / PER_ROW, ld) + tid % PER_ROW * VEC) = r[k];
        if (!FULL && rest && tid < CH * VEC)
#pragma unroll
            for (int k = 0; k < TAIL; ++k) lds[row_place<T>(tid / VEC + k * (THREADS / VEC), ld) + at + tid % VEC] = e[k];
    }
};

// Rows of whole tiles of 16 bits may go from memory to LDS directly, 16 bytes a lane: no registers hold them on the way.  Such a load writes 64 lanes'
// bytes side by side, so rows lie in LDS without a gap, and their 16-byte pieces are permuted instead: piece c of row r at c ^ turn(r), by the
// lane's choice of what it reads.  Half a wave's transposing read (two pieces of 8 rows that follow each other) and its read of one piece
// of each of 16 rows both meet every bank once.
template <int D> __device__ __forceinline__ int turn(int row)
{
    constexpr int G = D / 8, BITS = G == 16 ? 4 : G == 8 ? 3 : 2;          // pieces of a row; 16 pieces are all banks
    const int t = (row & 15) / (16 / G);
    return (t << 1 & (G - 1)) | t >> (BITS - 1);
}
typedef __attribute__((address_space(3))) char *Local;
typedef __attribute__((address_space(1))) char *Global;
template <typename T, int D, int THREADS> struct DirectRows {
    static constexpr int PER_ROW = D / 8, ROWS = THREADS / PER_ROW, N = ROWS > CH ? 1 : CH / ROWS, TURNS = ROWS < 16 ? 16 / ROWS : 1;
    const char *base;
    i64 next;
    int step;
    u32 off[TURNS];

    __device__ __forceinline__ void begin(const Rows &x, i64 token, int head, int, bool reverse, int tid)
    {
        const int bytes = (int)x.token * (int)sizeof(T), row = tid / PER_ROW;
        base = (const char *)x.p + (token * x.token + head / x.div * x.head) * (i64)sizeof(T);
        step = reverse ? -bytes : bytes, next = (i64)CH * step;
        const u32 first = reverse ? (ROWS - 1) * bytes : 0;
        base -= first;
#pragma unroll
        for (int k = 0; k < TURNS; ++k) off[k] = first + row * step + ((tid % PER_ROW) ^ turn<D>(row + k * ROWS)) * 16;
    }
    // The next chunk to `lds`, whole or `left` rows of it.  Rows behind the last are zeros.
    template <bool WHOLE> __device__ __forceinline__ void load(u32 lds, int left, int lane, int wave)
    {
        const int row = wave * (64 / PER_ROW) + lane / PER_ROW;
        lds += wave * 1024;
        if (ROWS <= CH || wave * 64 < CH * PER_ROW)
#pragma unroll
            for (int k = 0; k < N; ++k) {
                u32 o = off[k % TURNS];
                asm("" : "+v"(o));              // stays an offset of 32 bits to a base in scalar registers
                const u32 to = lds + k * ROWS * D * 2;
                if (WHOLE || row + k * ROWS < left)
                    __builtin_amdgcn_global_load_lds((Global)(base + (i64)(k * ROWS) * step + o), (Local)(uintptr_t)to, 16, 0, 0);
                else
                    *(__attribute__((address_space(3))) s8 *)(uintptr_t)(to + lane * 16) = s8{};
            }
        base += next;
    }
};
// operands from such rows: `at` is the tile's place plus the lane's, below
__device__ __forceinline__ s4 direct_rows(u32 at, int r0_bytes, int k0)
{
    return *(__attribute__((address_space(3))) s4 *)(uintptr_t)((at ^ (u32)(k0 * 2)) + r0_bytes);
}
// The transposing read through a pointer that says of itself what it may alias: of one that doesn't the compiler thinks that it might read what a
// direct load is about to write, and waits for all of these before it.
__device__ __forceinline__ s4 read_cols(__attribute__((address_space(3))) s4 *__restrict p) { return __builtin_amdgcn_ds_read_tr16_b64_v4i16(p); }
__device__ __forceinline__ s4 direct_cols(u32 at, int r0_bytes, int c0)
{
    return read_cols((__attribute__((address_space(3))) s4 *)(uintptr_t)((at ^ (u32)(c0 * 2)) + r0_bytes));
}
// a lane's place for operands from rows, and for those from columns
template <int D> __device__ __forceinline__ u32 direct_row_lane(int lane)
{
    const int row = lane & 15, g = lane >> 4;
    return (row * D + ((g >> 1) ^ turn<D>(row)) * 8 + 4 * (g & 1)) * 2;
}
template <int D> __device__ __forceinline__ u32 direct_col_lane(int lane)
{
    const int row = 4 * (lane >> 4) + ((lane & 15) >> 2);
    return (row * D + ((lane >> 1 & 1) ^ turn<D>(row)) * 8 + 4 * (lane & 1)) * 2;
}

// Which sequence, segment and head a workgroup has.  Heads that share keys and values get workgroups that are 8 apart: dealt out in turn to the
// 8 XCDs they share an L2.
struct Unit {
    int scan, seq, head, part, parts;
    i64 slot;                       // -1: the sequence is one unit
    i64 token;                      // its first row
    int n;
};
// Its scan, head and number, from the arguments' first line alone; then where it lies.  Each step further into the tables is a miss of the scalar
// cache, some 700 clocks, which short sequences feel: what does not depend on the tables is asked for in between.
__device__ __forceinline__ bool find_unit(const ScanArgs &A, int group, Unit &u, int &unit)
{
    const int kv_heads = A.heads / group, each = A.n_scans * kv_heads;
    const int octet = (int)(blockIdx.x >> 3), place = group == 1 ? 0 : octet % group;
    const int pair = (group == 1 ? octet : octet / group) * 8 + (int)(blockIdx.x & 7);
    if (pair >= A.n_units * each) return false;
    unit = pair / each;
    const int rest = pair - unit * each;
    u.scan = A.n_scans == 1 ? 0 : rest / kv_heads;
    u.head = (rest - u.scan * kv_heads) * group + place;
    return true;
}
__device__ __forceinline__ void place_unit(const ScanArgs &A, int unit, bool reverse, Unit &u)
{
    int rank = unit;
    u.slot = -1, u.part = 0, u.parts = 1;
    if (unit < A.n_cut) {
        int lo = 0, hi = A.n_split;                     // cum[lo] <= unit < cum[hi]
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if ((int)A.cum[mid] <= unit) lo = mid; else hi = mid;
        }
        rank = lo;
        u.part = unit - (int)A.cum[lo], u.parts = (int)(A.cum[lo + 1] - A.cum[lo]);
        u.slot = ((i64)u.scan * A.n_cut + unit) * A.heads + u.head;
    } else
        rank = A.n_split + unit - A.n_cut;
    u.seq = A.ordered ? rank : A.order[rank];
    const int t0 = (int)A.off[u.seq], t1 = (int)A.off[u.seq + 1], at = u.part * A.segment;
    u.n = u.parts == 1 ? t1 - t0 : min(A.segment, t1 - t0 - at);
    u.token = reverse ? (i64)t1 - 1 - at : (i64)t0 + at;
}

template <int DC> constexpr int scan_waves() { return DC >= 64 ? 4 : 2; }
// Direct loads, for whole tiles of 16 bits: no registers on the way, and LDS without gaps, so that fp16 of 128 x 128 has three workgroups a compute
// unit for two.  43 628 tokens of 32 heads, direct for through registers, us: fp16 128 x 128 322 for 347, 128 x 64 207 for 224, 64 x 64 183 for
// 191, 32 x 32 135 for 142; bf16 64 x 128 241 for 254, 64 x 64 180 for 183, 32 x 32 116 for 123.  But bf16 of 128 x 128: 351 for 339,
// and 65 536 tokens of 16 heads 388 for 377: loads through registers are a chunk further ahead, and what three workgroups would gain there
// the finer cuts lose (397).
template <typename T, int DA, int DC, bool FULL> constexpr bool scan_direct()
{
    return FULL && sizeof(T) == 2 && (Tile<T>::SCALED || DA < 128 || DC < 128);
}
// waves of a SIMD: what LDS leaves room for
template <typename T, int DA, int DC, bool FULL> constexpr int scan_occupancy()
{
    return sizeof(T) == 4 ? (DA == 128 || DC == 128 || DC < DA ? 2 : DA < 64 && DC < 64 ? 3 : 4) : DC == 32 ? (DA == 32 ? 3 : 2) : DA == 128 || DC == 128 ? (FULL && Tile<T>::SCALED ? 3 : 2) : 4;
}

// One workgroup walks the chunks of one unit for one head.  A wave has NC blocks of 16 columns of S and y and holds its part of S in fp32 in the
// accumulators throughout; the scores inside a chunk are made once, a block a wave, and pass through LDS.  What is rounded to 16 bits: scores
// (after decay) and the state where it is multiplied with a_i, one rounding each like that of y itself, which over a chunk's rows and columns
// average out to 1.4 times y's own error; not in a unit's last chunk, where both are two terms (0.8% of 48 ragged prompts in fp16; in every chunk
// second terms of scores would cost fp16 of 128 x 128 its third workgroup).  What is added to the state is not:
// decayed rows of c enter as SPLIT terms whose sum holds 22 (fp16) or 24 bits (bf16; two terms, 16 bits, where the state itself is not
// returned and only feeds 16-bit outputs).
// Chunks of 32 rows: a state of 128 x 128 takes 64 registers a lane of four waves, and a chunk's rows twice in LDS leave room for two or three
// workgroups a compute unit; with 64 rows registers spill (1050 us for the 241 below).  128 x 128: bf16, 65 536 tokens of 16 heads 242 us,
// 4.5 TB/s (a copy reaches 4.7), and 123 for the states of the segments; fp16, 43 628 tokens of 32 heads over 8 of keys 317 us, 3.45 TB/s.  Two
// chunks take a compute unit 6400 clocks in bf16: the vector units are busy 2800 of them, the matrix units 1760, LDS 1450; what is left are
// memory and their latencies.  Loads a chunk further ahead, reads of LDS ahead of their products, eight waves of 16 columns, rows of y put
// together in LDS, one decay for several chunks: within 2%.  y stored past the caches: 608 us for the 366 of both passes, since a wave has
// half of a line of 128 bytes.
// STATE_ONLY: no y; the segment's own contribution to the state goes to its slot.
template <typename T, int DA, int DC, bool STATE_ONLY, bool FULL>
__global__ void __launch_bounds__(64 * scan_waves<DC>(), (scan_occupancy<T, DA, DC, FULL>())) k_scan(const ScanArgs args, int group)
{
    typedef Tile<T> Q;
    typedef typename Q::Frag Frag;
    constexpr int NW = scan_waves<DC>(), THREADS = 64 * NW, ND = DA / 16, NC = DC / 16 / NW;
    constexpr bool DIRECT = scan_direct<T, DA, DC, FULL>();
    constexpr int LA = DIRECT ? DA : DA + Q::PAD, LC = DIRECT ? DC : DC + Q::PAD;
    constexpr int BUF = Q::BUFFERS;
    constexpr int TB = 0, TC = CH * LA, TA = TC + CH * LC, HALF = TA + (STATE_ONLY ? 0 : CH * LA);       // places of the tiles, elements
    __shared__ __align__(256) T s_x[BUF * HALF];
    __shared__ Frag s_p[2][STATE_ONLY ? 1 : 3][64];          // blocks of scores, as the lanes have them
    __shared__ int s_exp[2][4];
    __shared__ float s_power[64], s_weight[2 * CH];

    Unit u;
    int unit;
    if (!find_unit(args, group, u, unit)) return;
    const Scan &A = args.scan[u.scan];
    const float decay = args.log_decay[u.head];
    // what the loops need of the arguments, held in registers (they would be loaded anew at each use)
    float sp_scale = A.sp, sy = A.sy, ss = A.ss;
    int da = A.da, dc = A.dc, y_float = A.y_float, s_row = A.s_row, s_col = A.s_col;
    const float *s_in = A.s_in;
    float *s_out = A.s_out;
    asm volatile("" : "+s"(sp_scale), "+s"(sy), "+s"(dc), "+s"(y_float), "+s"(s_in), "+s"(s_out));
    place_unit(args, unit, A.reverse, u);
    if (STATE_ONLY) {
        if (u.slot < 0 || u.part == u.parts - 1) return;
        // From the segment's last chunk to its first, all of them whole: what the scan reads first is then in the last-level cache still.
        // Rows whose weight behind the segment is 0 in fp32 are not read: decay_power is 0 from 104 / -log_decay rows on.
        u.token += (A.reverse ? -1 : 1) * (u.n - CH);
        const float far = -104.0f / decay + 2.0f;
        if (decay < 0.0f && far < (float)u.n) u.n = min(u.n, (max((int)far, 1) + CH - 1) / CH * CH);
    }
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 4, l = lane & 15;
    const int dir = A.reverse ? -1 : 1, once = A.reverse ? 0 : 1;
    const int col0 = wave * 16 * NC;
    const i64 plane = ((i64)(args.first_seq + u.seq) * args.heads + u.head) * A.da * A.dc;
    const int n_all = u.n;

    typename std::conditional<DIRECT, DirectRows<T, DA, THREADS>, ChunkRows<T, DA, THREADS, FULL>>::type ra, rb;
    typename std::conditional<DIRECT, DirectRows<T, DC, THREADS>, ChunkRows<T, DC, THREADS, FULL>>::type rc;
    if constexpr (!STATE_ONLY) ra.begin(A.a, u.token, u.head, da, A.reverse, tid);
    rb.begin(A.b, u.token, u.head, da, A.reverse, tid);
    rc.begin(A.c, u.token, u.head, dc, A.reverse, tid);
    if constexpr (STATE_ONLY) rb.next = -rb.next, rc.next = -rc.next;
    const u32 lds = (u32)(uintptr_t)(Local)(char *)s_x;
    auto load = [&](int to, int left) {
        if constexpr (DIRECT) {
            const u32 half = lds + to * (HALF * 2);
            if (left >= CH) {
                if constexpr (!STATE_ONLY) ra.template load<true>(half + TA * 2, left, lane, wave);
                rb.template load<true>(half + TB * 2, left, lane, wave);
                rc.template load<true>(half + TC * 2, left, lane, wave);
            } else {
                if constexpr (!STATE_ONLY) ra.template load<false>(half + TA * 2, left, lane, wave);
                rb.template load<false>(half + TB * 2, left, lane, wave);
                rc.template load<false>(half + TC * 2, left, lane, wave);
            }
        } else {
            if constexpr (!STATE_ONLY) ra.load(left, tid);
            rb.load(left, tid);
            rc.load(left, tid);
        }
    };
    auto put = [&](int to, int left) {
        if constexpr (!DIRECT) {
            if constexpr (!STATE_ONLY) ra.put(s_x + to * HALF + TA, LA, tid, left);
            rb.put(s_x + to * HALF + TB, LA, tid, left);
            rc.put(s_x + to * HALF + TC, LC, tid, left);
        }
    };
    // direct loads write LDS by themselves: a wave's own have come before it passes the barrier
    auto landed = [&]() {
        if constexpr (DIRECT) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    };
    if (n_all > 0) load(0, n_all);

    f4 S[NC][ND];
    float *slot = u.slot < 0 ? nullptr : args.slots + u.slot * (DA * DC);
    const bool from_slot = !STATE_ONLY && slot, from_user = !STATE_ONLY && !slot && s_in;
#pragma unroll
    for (int ct = 0; ct < NC; ++ct)
#pragma unroll
        for (int dt = 0; dt < ND; ++dt) S[ct][dt] = f4{};
    if (from_slot) {
#pragma unroll
        for (int ct = 0; ct < NC; ++ct)
#pragma unroll
            for (int dt = 0; dt < ND; ++dt) S[ct][dt] = *(const f4 *)(slot + ((((wave * NC + ct) * ND + dt) * 64 + lane) << 2));
    } else if (from_user) {
#pragma unroll
        for (int ct = 0; ct < NC; ++ct)
#pragma unroll
            for (int dt = 0; dt < ND; ++dt)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int row = dt * 16 + 4 * g + r, col = col0 + ct * 16 + l;
                    if (FULL || (row < da && col < dc)) S[ct][dt][r] = s_in[plane + row * s_row + col * s_col];
                }
    }
    const bool give = !STATE_ONLY && s_out && u.part == u.parts - 1;
    const bool exact = STATE_ONLY ? A.exact_state : give;
    bool have = from_slot || from_user;         // the state may hold something
    int s_scale = 0;                            // fp16: S (STATE_ONLY: what is added to it) is held times held = 2^s_scale
    float held = 1.0f, loose = 1.0f;            // loose: STATE_ONLY, 2^-s_scale

    // powers of the decay, and what a whole chunk's rows weigh in the state behind it: those of a chunk of n rows lie CH - n further on
    if (tid < 64) {
        s_power[tid] = decay_power(decay, tid);
        s_weight[tid] = tid < CH ? ss * decay_power(decay, CH - once - tid) : 0.0f;
    }
    // y by rows: as for the chunks, a base that is the same for all threads and an offset
    const int y_size = y_float ? 4 : (int)sizeof(T), y_bytes = (int)A.y_token * y_size, y_first = A.reverse ? (CH - 1) * y_bytes : 0;
    char *py = (char *)A.y + (u.token * A.y_token + u.head * A.y_head) * y_size - y_first;
    const i64 y_next = (i64)CH * dir * y_bytes;
    const u32 y_off = y_first + l * dir * y_bytes + (col0 + 4 * g) * y_size, y_step = 16 * dir * y_bytes;

    if (n_all > 0) put(0, n_all);
    landed();
    __syncthreads();
    if (n_all > CH) load(1, n_all - CH);
    const u32 row_lane = lds + direct_row_lane<DA>(lane), col_lane_b = lds + direct_col_lane<DA>(lane), col_lane_c = lds + direct_col_lane<DC>(lane);

    // One barrier a chunk: the next rows go to the other half of the buffers, which everybody has left at the barrier before, and the
    // rows after them are on their way from memory in the meantime.  With one buffer (fp32, which leaves room for twice the workgroups
    // so) the next rows follow that barrier and another one them.
    int half = 0;
    const Frag none = {};
#pragma clang loop unroll(disable)
    for (int at = 0; at < n_all; at += CH, half ^= 1) {
        const int n = min(CH, n_all - at), left = n_all - at - CH;
        const int from = BUF == 2 ? half : 0;
        const T *sa = s_x + from * HALF + TA, *sb = s_x + from * HALF + TB, *sc = s_x + from * HALF + TC;
        const u32 at_half = from * (HALF * 2);
        // In the last chunk of a unit, the only one of a short sequence, scores and the state enter products as two terms: a score is one rounding for all
        // columns of a row, and the roundings of few rows do not average out (errors of up to twice the output's own).  Second
        // terms of scores lie in the half of the buffers that is free then.
        Frag *s_low = (Frag *)(s_x + (BUF == 2 ? half ^ 1 : 0) * HALF);
        auto a_rows = [&](int r0, int k0) -> Frag {
            if constexpr (DIRECT) return direct_rows(row_lane + at_half, (TA + r0 * DA) * 2, k0);
            else return rows_frag(sa, LA, r0, k0, lane);
        };
        auto b_rows = [&](int r0, int k0) -> Frag {
            if constexpr (DIRECT) return direct_rows(row_lane + at_half, (TB + r0 * DA) * 2, k0);
            else return rows_frag(sb, LA, r0, k0, lane);
        };
        auto b_cols = [&](int r0, int c0) -> Frag {
            if constexpr (DIRECT) return direct_cols(col_lane_b + at_half, (TB + r0 * DA) * 2, c0);
            else return cols_frag(sb, LA, r0, c0, lane);
        };
        auto c_cols = [&](int r0, int c0) -> Frag {
            if constexpr (DIRECT) return direct_cols(col_lane_c + at_half, (TC + r0 * DC) * 2, c0);
            else return cols_frag(sc, LC, r0, c0, lane);
        };
        f4 acc[NC][2] = {};
        float by_state = 1.0f;
        if constexpr (!STATE_ONLY) {
            // Blocks of scores: (0, 0), (1, 0) and (1, 1), a wave each; decay between their rows as lambda^(i - j), or lambda^(16 + i - j) for the
            // one off the diagonal (i, j places in the block); 0 above the diagonal.  The lane gets one i and four j.
#pragma unroll 1
            for (int t = wave; t < 3; t += NW) {
                const int ib = t > 0, jb = t > 1;
                f4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int k = 0; k < DA; k += 32)
                    x = Q::mma(b_rows(jb * 16, k), b_rows(jb * 16, k + 16),
                               a_rows(ib * 16, k), a_rows(ib * 16, k + 16), x);
                // by selection above the diagonal: what lies there may be infinite
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int far = (t == 1 ? 16 : 0) + l - 4 * g - r;
                    const float y = x[r] * (sp_scale * s_power[max(far, 0)]);
                    x[r] = far >= 0 ? y : 0.0f;
                }
                if constexpr (Q::SCALED) {
                    const float most = fmaxf(fmaxf(fabsf(x[0]), fabsf(x[1])), fmaxf(fabsf(x[2]), fabsf(x[3])));
                    int e = 0;
                    if (__builtin_amdgcn_ballot_w64(most > 32768.0f) || !__builtin_amdgcn_ballot_w64(most >= 0.125f)) {
                        e = fit_exponent(wave_max(max(max(finite_bits(x[0]), finite_bits(x[1])), max(finite_bits(x[2]), finite_bits(x[3])))));
                        x *= two_to(e);
                    }
                    if (lane == 0) s_exp[half][t] = e;
                }
                const Frag p = to_frag<T>(x);
                s_p[half][t][lane] = p;
                if (Q::SPLIT > 1 && left <= 0) s_low[t * 64 + lane] = to_frag<T>(x - from_frag<T>(p));
            }
            // what the state before the chunk gives
            if (have) {
                auto from_state = [&](auto scaled, auto low, float by) {
#pragma unroll
                    for (int dt = 0; dt < ND; dt += 2) {
                        const Frag a0 = a_rows(0, dt * 16), a1 = a_rows(0, dt * 16 + 16);
                        const Frag b0 = a_rows(16, dt * 16), b1 = a_rows(16, dt * 16 + 16);
#pragma unroll
                        for (int ct = 0; ct < NC; ++ct) {
                            const f4 x0 = scaled ? S[ct][dt] * by : S[ct][dt], x1 = scaled ? S[ct][dt + 1] * by : S[ct][dt + 1];
                            Frag s0 = to_frag<T>(x0), s1 = to_frag<T>(x1);
                            if (low) s0 = to_frag<T>(x0 - from_frag<T>(s0)), s1 = to_frag<T>(x1 - from_frag<T>(s1));
                            acc[ct][0] = Q::mma(s0, s1, a0, a1, acc[ct][0]);
                            acc[ct][1] = Q::mma(s0, s1, b0, b1, acc[ct][1]);
                        }
                    }
                };
                float by = 1.0f;
                if constexpr (Q::SCALED) {
                    by_state = two_to(-s_scale);
                    // As it is where the largest element is one that leaves 13 binary places below it, else times a power of two.  The largest
                    // sum of two magnitudes, at most twice the largest, stands for it: a maximum of a matrix product's results would
                    // first make each of them canonical.
                    float most = 0.0f;
#pragma unroll
                    for (int ct = 0; ct < NC; ++ct)
#pragma unroll
                        for (int dt = 0; dt < ND; ++dt)
#pragma unroll
                            for (int r = 0; r < 4; r += 2) most = fmaxf(most, fabsf(S[ct][dt][r]) + fabsf(S[ct][dt][r + 1]));
                    if (__builtin_amdgcn_ballot_w64(most > 32768.0f) || !__builtin_amdgcn_ballot_w64(most >= 1.0f)) {
                        int bits = wave_max(bits_of(most));
                        if (bits >= BITS_INF) {
                            bits = 0;
#pragma unroll
                            for (int ct = 0; ct < NC; ++ct)
#pragma unroll
                                for (int dt = 0; dt < ND; ++dt)
#pragma unroll
                                    for (int r = 0; r < 4; ++r) bits = max(bits, finite_bits(S[ct][dt][r]));
                            bits = wave_max(bits);
                        }
                        const int e = fit_exponent(bits);
                        by_state = two_to(-e - s_scale), by = two_to(e);
                        from_state(std::true_type(), std::false_type(), by);
                    } else
                        from_state(std::false_type(), std::false_type(), by);
                } else
                    from_state(std::false_type(), std::false_type(), by);
                if (Q::SPLIT > 1 && left <= 0) from_state(std::bool_constant<Q::SCALED>(), std::true_type(), by);
            }
        }
        // the state behind the chunk
        Frag v0[NC], v1[NC];
#pragma unroll
        for (int ct = 0; ct < NC; ++ct) v0[ct] = c_cols(0, col0 + ct * 16), v1[ct] = c_cols(16, col0 + ct * 16);
        if (STATE_ONLY || left > 0 || give) {
            f4 x0[NC], x1[NC];
            float keep = STATE_ONLY ? 1.0f : s_power[n];
            const float *w = s_weight + (CH - n) + 4 * g;          // one by one: with typed reads the compiler doesn't wait for direct loads
            const f4 w0 = {w[0], w[1], w[2], w[3]}, w1 = {w[16], w[17], w[18], w[19]};
#pragma unroll
            for (int ct = 0; ct < NC; ++ct) x0[ct] = from_frag<T>(v0[ct]) * w0, x1[ct] = from_frag<T>(v1[ct]) * w1;
            if constexpr (Q::SCALED) {
                float most_x = 0.0f;
#pragma unroll
                for (int ct = 0; ct < NC; ++ct)
#pragma unroll
                    for (int r = 0; r < 4; ++r) most_x = fmaxf(most_x, fmaxf(fabsf(x0[ct][r]), fabsf(x1[ct][r])));
                // held times 2^s_scale, the largest between 2^11 and 2^14: the second term has its bits then down to 2^-24 of the largest
                most_x *= held;
                if (__builtin_amdgcn_ballot_w64(most_x > 16384.0f) || !__builtin_amdgcn_ballot_w64(most_x >= 2048.0f)) {
                    // of the rows as they are: held, they may have left fp32's range where the power changes much, as it does when rows of zeros
                    // follow a fast decay
                    int bits = 0;
#pragma unroll
                    for (int ct = 0; ct < NC; ++ct)
#pragma unroll
                        for (int r = 0; r < 4; ++r) bits = max(bits, max(finite_bits(x0[ct][r]), finite_bits(x1[ct][r])));
                    bits = wave_max(bits);
                    if (bits) {
                        const int to = min(max(fit_exponent(bits), -100), min(100, s_scale + 120));
                        keep *= two_to(to - s_scale), held = two_to(to), loose = two_to(-to), s_scale = to;
                    }
                }
#pragma unroll
                for (int ct = 0; ct < NC; ++ct) x0[ct] *= held, x1[ct] *= held;
            }
            // The rows behind the chunk.  A type of fp32's range takes their decay before it is split into terms; fp16 would lose what has decayed
            // below its own range, so its products are made of rows as they are and decayed as they are added, in fp32.
            float behind = 1.0f;
            if constexpr (STATE_ONLY) {
                behind = decay_power(decay, at);
                if constexpr (Q::SCALED) behind *= loose;
                else
#pragma unroll
                    for (int ct = 0; ct < NC; ++ct) x0[ct] *= behind, x1[ct] *= behind;
            }
            if constexpr (!STATE_ONLY)
#pragma unroll
                for (int ct = 0; ct < NC; ++ct)
#pragma unroll
                    for (int dt = 0; dt < ND; ++dt) S[ct][dt] *= keep;
            constexpr int M = Q::SPLIT < 2 ? 1 : 2;
            Frag t0[NC][M], t1[NC][M];
#pragma unroll
            for (int ct = 0; ct < NC; ++ct)
#pragma unroll
                for (int m = 0; m < M; ++m) {
                    t0[ct][m] = to_frag<T>(x0[ct]), t1[ct][m] = to_frag<T>(x1[ct]);
                    if (Q::SPLIT > 1) x0[ct] -= from_frag<T>(t0[ct][m]), x1[ct] -= from_frag<T>(t1[ct][m]);
                }
            // several blocks at a time, so that no product waits for the one before it
#pragma unroll
            for (int dt = 0; dt < ND; dt += 2) {
                const Frag u0 = b_cols(0, dt * 16), u1 = b_cols(16, dt * 16);
                const Frag z0 = b_cols(0, dt * 16 + 16), z1 = b_cols(16, dt * 16 + 16);
                if constexpr (STATE_ONLY && Q::SCALED) {
                    f4 y[NC][2] = {};
#pragma unroll
                    for (int m = 0; m < M; ++m)
#pragma unroll
                        for (int ct = 0; ct < NC; ++ct) {
                            y[ct][0] = Q::mma(u0, u1, t0[ct][m], t1[ct][m], y[ct][0]);
                            y[ct][1] = Q::mma(z0, z1, t0[ct][m], t1[ct][m], y[ct][1]);
                        }
#pragma unroll
                    for (int ct = 0; ct < NC; ++ct) S[ct][dt] += y[ct][0] * behind, S[ct][dt + 1] += y[ct][1] * behind;
                } else
#pragma unroll
                    for (int m = 0; m < M; ++m)
#pragma unroll
                        for (int ct = 0; ct < NC; ++ct) {
                            S[ct][dt] = Q::mma(u0, u1, t0[ct][m], t1[ct][m], S[ct][dt]);
                            S[ct][dt + 1] = Q::mma(z0, z1, t0[ct][m], t1[ct][m], S[ct][dt + 1]);
                        }
            }
            // the sums stay on this side of the loop's branches, behind which the compiler may place them too near to the products that they add
            if constexpr (STATE_ONLY && Q::SCALED)
#pragma unroll
                for (int ct = 0; ct < NC; ++ct)
#pragma unroll
                    for (int dt = 0; dt < ND; ++dt) asm volatile("" : "+v"(S[ct][dt]));
            if constexpr (Q::SPLIT > 2) {
                if (exact) {
#pragma unroll
                    for (int ct = 0; ct < NC; ++ct) t0[ct][0] = to_frag<T>(x0[ct]), t1[ct][0] = to_frag<T>(x1[ct]);
#pragma unroll
                    for (int dt = 0; dt < ND; ++dt) {
                        const Frag u0 = b_cols(0, dt * 16), u1 = b_cols(16, dt * 16);
#pragma unroll
                        for (int ct = 0; ct < NC; ++ct) S[ct][dt] = Q::mma(u0, u1, t0[ct][0], t1[ct][0], S[ct][dt]);
                    }
                }
            }
        }
        if constexpr (BUF == 2)
            if (left > 0) {
                put(half ^ 1, left);
                if (!DIRECT && left > CH) load(0, left - CH);
            }
        landed();
        __syncthreads();                        // the scores and the next rows are there
        if constexpr (DIRECT)
            if (left > CH) load(half, left - CH);
        if constexpr (BUF == 1)
            if (left > 0) {
                put(0, left);
                if (left > CH) load(0, left - CH);
            }
        if constexpr (!STATE_ONLY) {
            const float into0 = sy * s_power[l + once] * by_state, into1 = sy * s_power[16 + l + once] * by_state;
            const bool p_scaled = Q::SCALED && __builtin_amdgcn_readfirstlane(s_exp[half][0] | s_exp[half][1] | s_exp[half][2]);
            const Frag p00 = s_p[half][0][lane], p10 = s_p[half][1][lane], p11 = s_p[half][2][lane];
            Frag r00 = none, r10 = none, r11 = none;
            if (Q::SPLIT > 1 && left <= 0) r00 = s_low[lane], r10 = s_low[64 + lane], r11 = s_low[128 + lane];
#pragma unroll
            for (int ct = 0; ct < NC; ++ct) {
                acc[ct][0] *= into0, acc[ct][1] *= into1;
                if (Q::SCALED && p_scaled) {
                    const f4 zero = {0.f, 0.f, 0.f, 0.f};
                    acc[ct][0] += Q::mma(v0[ct], v0[ct], p00, r00, zero) * two_to(-s_exp[half][0]);
                    acc[ct][1] += Q::mma(v0[ct], v0[ct], p10, r10, zero) * two_to(-s_exp[half][1]) + Q::mma(v1[ct], v1[ct], p11, r11, zero) * two_to(-s_exp[half][2]);
                } else if constexpr (Q::SPLIT > 1) {
                    acc[ct][0] = Q::mma(v0[ct], v0[ct], p00, r00, acc[ct][0]);
                    acc[ct][1] = Q::mma(v0[ct], v1[ct], p10, p11, acc[ct][1]);
                    if (left <= 0) acc[ct][1] = Q::mma(v0[ct], v1[ct], r10, r11, acc[ct][1]);
                } else {
                    acc[ct][0] = Q::mma(v0[ct], none, p00, none, acc[ct][0]);
                    acc[ct][1] = Q::mma(v0[ct], v1[ct], p10, p11, acc[ct][1]);
                }
            }
            auto give_row = [&](u32 to, f4 y, int col) {
                asm("" : "+v"(to));
                typedef typename Pack<T, 4>::V V;
                if (FULL || col + 16 <= dc) {
                    if (y_float) store_n<float, 4>((float *)(py + to), y);
                    else store_n<T, 4>((T *)(py + to), __builtin_convertvector(y, V));
                } else
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (col + 4 * g + r < dc) {
                            if (y_float) ((float *)(py + to))[r] = y[r];
                            else ((T *)(py + to))[r] = (T)y[r];
                        }
            };
#pragma unroll
            for (int ct = 0; ct < NC; ++ct) {
                if (l < n) give_row(y_off + ct * 16 * y_size, acc[ct][0], col0 + ct * 16);
                if (16 + l < n) give_row(y_off + y_step + ct * 16 * y_size, acc[ct][1], col0 + ct * 16);
            }
            py += y_next;
        }
        have = true;
        if constexpr (BUF == 1) __syncthreads();
    }
    if (STATE_ONLY || give) {
        const float by = !STATE_ONLY && Q::SCALED ? two_to(-s_scale) : 1.0f;
#pragma unroll
        for (int ct = 0; ct < NC; ++ct)
#pragma unroll
            for (int dt = 0; dt < ND; ++dt) {
                if constexpr (STATE_ONLY) *(f4 *)(slot + ((((wave * NC + ct) * ND + dt) * 64 + lane) << 2)) = S[ct][dt] * by;
                else
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int row = dt * 16 + 4 * g + r, col = col0 + ct * 16 + l;
                        if (FULL || (row < da && col < dc)) s_out[plane + row * s_row + col * s_col] = S[ct][dt][r] * by;
                    }
            }
    }
}

// The states at the starts of segments from what each segment adds: slot s of a sequence becomes lambda^(s L) s_in + the slots before it, decayed.
// A thread has one element of the state; eight loads are under way at a time (32 segments of 16 heads, 128 x 128: 13 us).
template <int DA, int DC> __global__ void __launch_bounds__(256) k_join(const ScanArgs args)
{
    constexpr int ND = DA / 16;
    const int rank = blockIdx.z % args.n_split, scan = blockIdx.z / args.n_split, head = blockIdx.y, i = blockIdx.x * 256 + threadIdx.x;
    const Scan &A = args.scan[scan];
    const int first = (int)args.cum[rank], parts = (int)(args.cum[rank + 1] - args.cum[rank]);
    const int r = i & 3, lane = (i >> 2) & 63, tile = i >> 8, dt = tile % ND, wave = tile / ND;
    const int row = dt * 16 + 4 * (lane >> 4) + r, col = wave * 16 + (lane & 15);
    float run = 0.0f;
    if (A.s_in && row < A.da && col < A.dc)
        run = A.s_in[((i64)(args.first_seq + args.order[rank]) * args.heads + head) * A.da * A.dc + row * A.s_row + col * A.s_col];
    const float keep = decay_power(args.log_decay[head], args.segment);
    float *at = args.slots + (((i64)scan * args.n_cut + first) * args.heads + head) * (DA * DC) + i;
    const i64 step = (i64)args.heads * (DA * DC);
    for (int s = 0; s < parts; s += 8) {
        float x[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = s + k < parts - 1 ? at[(s + k) * step] : 0.0f;
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (s + k < parts) {
                at[(s + k) * step] = run;
                run = run * keep + x[k];
            }
    }
}

// One launch of the scan over the tables in A (the states of segments first, where sequences are cut).
typedef int (*ScanLaunch)(hipStream_t, const ScanArgs &, int group);
int scan_f32(hipStream_t, const ScanArgs &, int group);
int scan_bf16(hipStream_t, const ScanArgs &, int group);
int scan_f16(hipStream_t, const ScanArgs &, int group);

template <typename T, int DA, int DC, bool FULL> static int scan_launch(hipStream_t s, const ScanArgs &A, int group)
{
    const int each = A.n_scans * (A.heads / group);
    const i64 blocks = ((i64)A.n_units * each + 7) / 8 * 8 * group;
    if (!launch_fits(blocks, 64 * scan_waves<DC>())) return ops_fail(OB_E_RANGE, "decay attention: %d units of %d heads in one launch", A.n_units, A.heads);
    const dim3 grid((unsigned)blocks), block(64 * scan_waves<DC>());
    if (A.n_split) {
        const int cut = A.n_cut * each;                                 // the units of cut sequences come first
        k_scan<T, DA, DC, true, FULL><<<dim3((unsigned)((cut + 7) / 8 * 8 * group)), block, 0, s>>>(A, group);
        k_join<DA, DC><<<dim3(DA * DC / 256, (unsigned)A.heads, (unsigned)(A.n_split * A.n_scans)), 256, 0, s>>>(A);
    }
    k_scan<T, DA, DC, false, FULL><<<grid, block, 0, s>>>(A, group);
    return ops_launched("decay attention");
}
// direct loads take pieces of 16 bytes at such places
static inline bool pieces_aligned(const Rows &x) { return ((uintptr_t)x.p | (uintptr_t)(x.token * 2) | (uintptr_t)(x.head * 2)) % 16 == 0; }
template <typename T, int DA, int DC> static int scan_width(hipStream_t s, const ScanArgs &A, int group)
{
    // widths of whole tiles need no questions about columns: a tenth of the operations of a chunk
    bool full = true;
    for (int i = 0; i < A.n_scans; ++i) {
        full = full && A.scan[i].da == DA && A.scan[i].dc == DC;
        if (scan_direct<T, DA, DC, true>()) full = full && pieces_aligned(A.scan[i].a) && pieces_aligned(A.scan[i].b) && pieces_aligned(A.scan[i].c);
    }
    return full ? scan_launch<T, DA, DC, true>(s, A, group) : scan_launch<T, DA, DC, false>(s, A, group);
}
template <typename T> static int scan_any(hipStream_t s, const ScanArgs &A, int group)
{
    const int da = A.scan[0].da, dc = A.scan[0].dc;                     // the other scans' widths take the same tiles
    const int a = da <= 32 ? 0 : da <= 64 ? 1 : 2, c = dc <= 32 ? 0 : dc <= 64 ? 1 : 2;
    switch (3 * a + c) {
    case 0: return scan_width<T, 32, 32>(s, A, group);
    case 1: return scan_width<T, 32, 64>(s, A, group);
    case 2: return scan_width<T, 32, 128>(s, A, group);
    case 3: return scan_width<T, 64, 32>(s, A, group);
    case 4: return scan_width<T, 64, 64>(s, A, group);
    case 5: return scan_width<T, 64, 128>(s, A, group);
    case 6: return scan_width<T, 128, 32>(s, A, group);
    case 7: return scan_width<T, 128, 64>(s, A, group);
    default: return scan_width<T, 128, 128>(s, A, group);
    }
}
