// Log probabilities of labels with the entropy of each row and its most likely classes, and the gradient of the first two.
#include "ob_dev.h"
#include "ob_ctx.h"

namespace {

struct ScoreArgs {
    const void *x;
    i64 x_row;                      // elements between rows
    const void *labels;
    int labels_wide;                // 64 bits
    int first, rows, classes, top;  // rows of one launch, from `first` on
    float *logprob, *entropy, *row_max, *row_sum, *top_logprob;
    int *top_id;
};

// order-preserving bits of a score; -0 is 0
__device__ __forceinline__ u32 order_of(float x)
{
    const u32 b = __builtin_bit_cast(u32, x + 0.0f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
constexpr u32 LOWEST = 0x007fffffu;  // order_of(-inf)
__device__ __forceinline__ float score_of(u32 o) { return __builtin_bit_cast(float, o & 0x80000000u ? o & 0x7fffffffu : ~o); }

__device__ __forceinline__ float wave_maxf(float x)
{
#pragma unroll
    for (int d = 32; d; d >>= 1) x = fmaxf(x, __shfl_xor(x, d));
    return x;
}
__device__ __forceinline__ float wave_sumf(float x)
{
#pragma unroll
    for (int d = 32; d; d >>= 1) x += __shfl_xor(x, d);
    return x;
}

__device__ __forceinline__ i64 label_of(const void *p, int wide, int row) { return wide ? ((const i64 *)p)[row] : (i64)((const int *)p)[row]; }

constexpr int KEPT = 512;            // candidates for the most likely classes

// One workgroup has one row and reads it once: 4 vectors of 16 bytes a thread and step, the running maximum of the thread, sum e and sum e d
// for d = x - maximum, rescaled when it grows.
// Ten operations and an exponential (which counts four) an element take 2/3 of the time of reading two bytes of it.
// For the most likely classes each lane of the first wave has the largest elements of two groups of threads; the top-th largest of these 128,
// found bit by bit from how many reach each prefix, is a bound that at least `top` elements reach and, unless many are equal, few more do: some 8
// for 8, 37 for 32, 89 for 64.  The few threads that have any read theirs again, out of the caches, and put them to a list, where they are
// ranked by (score, lower class first).  If too many reach the bound, as in rows of equal scores, they are picked one by one, the row read again for
// each (8192 rows of 32 000 equal bf16 scores: 8 classes 785 us, 64 classes 5.1 ms).
// 8192 rows of 32 000 bf16: without classes 89 us, 5.9 TB/s; 8 classes 115, 64 138 (with one group a lane 740: too many reach the least of 64).
// Slower for 8: ranks of the groups by comparing each with each 123, all threads reading again 147, the row kept in LDS 174 (room for two
// workgroups a compute unit), in registers 561.  Comparing differences to the maximum so far in place of the elements saves a third
// of the operations, but needs 96 registers for 48 and a branch that some lane nearly always takes: 113 for the 89.
template <typename T, int THREADS> __global__ void __launch_bounds__(THREADS) k_logprobs(const ScoreArgs A)
{
    constexpr int VEC = 16 / (int)sizeof(T), WAVES = THREADS / 64, U = 4;
    typedef u32 Raw __attribute__((ext_vector_type(4)));
    struct __attribute__((packed, aligned(sizeof(T)))) RawAt { Raw v; };
    __shared__ float s_red[3][WAVES];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, row = A.first + (int)blockIdx.x;
    const T *first = (const T *)A.x + row * A.x_row;
    // vectors from the first place of 16 bytes on (4096 rows of 50 257 bf16 by
    // themselves, inputs that take turns: 83 us for 93); what lies before it goes one by one
    const int head = min((int)(-(uintptr_t)first & 15) / (int)sizeof(T), A.classes), classes = A.classes - head;
    const T *x = first + head;
    const int full = classes / VEC, vecs = (classes + VEC - 1) / VEC;
    const float low = -__builtin_inff();

    constexpr u32 fill = sizeof(T) == 4 ? 0xff800000u : std::is_same<T, bf16>::value ? 0xff80ff80u : 0xfc00fc00u;   // -inf
    auto whole = [&](int i) { return ((const RawAt *)(x + i * VEC))->v; };
    auto partial = [&]() {                              // the last vector, -inf behind the row's end
        Raw r = {fill, fill, fill, fill};
#pragma unroll
        for (int e = 0; e < VEC - 1; ++e)
            if (full * VEC + e < classes) {
                if constexpr (sizeof(T) == 4) r[e] = ((const u32 *)x)[full * VEC + e];
                else {
                    const u32 h = ((const uint16_t *)x)[full * VEC + e];
                    r[e / 2] = e & 1 ? (r[e / 2] & 0xffffu) | h << 16 : (r[e / 2] & 0xffff0000u) | h;
                }
            }
        return r;
    };
    // element e of a vector as it lies in four registers
    auto wide = [](const Raw &r, int e) {
        if constexpr (sizeof(T) == 4) return __builtin_bit_cast(float, (u32)r[e]);
        else if constexpr (std::is_same<T, bf16>::value) return __builtin_bit_cast(float, e & 1 ? r[e / 2] & 0xffff0000u : r[e / 2] << 16);
        else {
            typedef f16 H __attribute__((ext_vector_type(2)));
            return (float)__builtin_bit_cast(H, (u32)r[e / 2])[e & 1];
        }
    };
    const i64 y = label_of(A.labels, A.labels_wide, row);
    const float xy = y >= 0 && y < A.classes ? (float)first[y] : 0.0f;
    float own = low, s = 0.0f, w = 0.0f;
    auto add = [&](const Raw *r, int n) {
        float most = own;
#pragma unroll
        for (int k = 0; k < U; ++k)
            if (k < n)
#pragma unroll
                for (int e = 0; e < VEC; ++e) most = fmaxf(most, wide(r[k], e));
        if (most > own) {
            // sums of e^(x - own) and of (x - own) e^(x - own) seen from the new maximum
            const float by = __expf(own - most), d = fmaxf(own - most, -1e30f);
            w = by * (w + d * s);
            s *= by;
            own = most;
        }
        const float from = own == low ? 0.0f : own;
#pragma unroll
        for (int k = 0; k < U; ++k)
            if (k < n)
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const float d = wide(r[k], e) - from, p = __expf(d);
                    s += p;
                    w += p * fmaxf(d, -1e30f);       // nothing where p is 0; a NaN goes on through p
                }
    };
    int i0 = 0;
    for (; i0 + U * THREADS <= full; i0 += U * THREADS) {
        Raw r[U];
#pragma unroll
        for (int k = 0; k < U; ++k) r[k] = whole(i0 + k * THREADS + tid);
        add(r, U);
    }
    {
        // what is left: fewer than U vectors a thread, the last of which may not be full
        const int n = (vecs - i0 + THREADS - 1) / THREADS;
        Raw r[U];
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const int i = i0 + k * THREADS + tid;
            r[k] = Raw{fill, fill, fill, fill};
            if (i < full) r[k] = whole(i);
        }
        if (full < vecs && (full - i0) % THREADS == tid) {
            const Raw last = partial();
#pragma unroll
            for (int k = 0; k < U; ++k)
                if (k == (full - i0) / THREADS) r[k] = last;
        }
        add(r, n);
    }
    if (tid < head) {
        const float v = (float)first[tid], most = fmaxf(own, v);
        if (most > own) {
            const float by = __expf(own - most), d = fmaxf(own - most, -1e30f);
            w = by * (w + d * s);
            s *= by;
            own = most;
        }
        const float d = v - (own == low ? 0.0f : own), p = __expf(d);
        s += p;
        w += p * fmaxf(d, -1e30f);
    }
    float m = wave_maxf(own);
    if (WAVES > 1) {
        if (lane == 0) s_red[0][wave] = m;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < WAVES; ++i) m = fmaxf(m, s_red[0][i]);
    }
    if (own == low) s = s == s ? 0.0f : s, w = 0.0f;       // nothing seen, or only NaN
    else {
        // bounded as above: with all of a thread's scores at the type's lowest value d * s passes fp32's range where by is 0
        const float by = __expf(own - m), d = fmaxf(own - m, -1e30f);
        w = by * (w + d * s);
        s *= by;
    }
    s = wave_sumf(s), w = wave_sumf(w);
    if (WAVES > 1) {
        if (lane == 0) s_red[1][wave] = s, s_red[2][wave] = w;
        __syncthreads();
        s = 0.0f, w = 0.0f;
#pragma unroll
        for (int i = 0; i < WAVES; ++i) s += s_red[1][i], w += s_red[2][i];
    }
    // a NaN or +inf anywhere makes the sum NaN; a row of nothing but -inf sums to 0
    const bool bad = !(s >= 0.0f) || m == __builtin_inff(), empty = !bad && m == low;
    const float nan = __builtin_nanf(""), log_sum = logf(s);
    if (tid == 0) {
        const float lp = (xy - m) - log_sum;
        A.logprob[row] = y < 0 ? 0.0f : bad || y >= A.classes ? nan : empty ? low : lp;
        A.entropy[row] = bad ? nan : empty ? 0.0f : log_sum - w / s;
        A.row_max[row] = empty ? 0.0f : m;
        A.row_sum[row] = bad ? nan : empty ? 0.0f : s;
    }
    if (A.top <= 0) return;
    float *top_lp = A.top_logprob + (i64)row * A.top;
    int *top_id = A.top_id + (i64)row * A.top;
    if (bad || empty) {
        for (int i = tid; i < A.top; i += THREADS) top_lp[i] = bad ? nan : low, top_id[i] = -1;
        return;
    }
    __shared__ u32 s_order[THREADS];
    __shared__ u64 s_key[KEPT];
    __shared__ u32 s_bound, s_count;
    __shared__ u64 s_pick[WAVES];
    auto each = [&](auto &&f) {                         // all elements of the thread, classes in ascending order
        if (tid < head) f((float)first[tid], tid);
        for (int i = tid; i < vecs; i += THREADS) {
            const Raw r = i < full ? whole(i) : partial();
#pragma unroll
            for (int e = 0; e < VEC; ++e) f(wide(r, e), head + i * VEC + e);
        }
    };
    s_order[tid] = order_of(own);
    if (tid == 0) s_count = 0;
    __syncthreads();
    if (wave == 0) {
        u32 mine = s_order[lane], other = 0;
#pragma unroll
        for (int i = 1; i < WAVES; ++i) (i & 1 ? other : mine) = max(i & 1 ? other : mine, s_order[i * 64 + lane]);
        // the top-th largest of these, or a little less: its upper 20 bits, which hold all that bf16 and fp16 have
        u32 bound = 0;
#pragma unroll
        for (int bit = 31; bit >= 12; --bit) {
            const u32 c = bound | 1u << bit;
            int n = __builtin_popcountll(__builtin_amdgcn_ballot_w64(mine >= c));
            if (WAVES > 1) n += __builtin_popcountll(__builtin_amdgcn_ballot_w64(other >= c));
            bound = n >= A.top ? c : bound;
        }
        if (lane == 0) s_bound = bound;
    }
    __syncthreads();
    const u32 bound = max(s_bound, LOWEST + 1);         // -inf is no alternative
    const float least = score_of(bound);
    if (own >= least) {                                 // the thread has the same elements as before: few threads have any
        auto keep = [&](float v, int c) {
            if (v >= least) {
                const u32 at = atomicAdd(&s_count, 1u);
                if (at < KEPT) s_key[at] = (u64)order_of(v) << 32 | (u32)~c;
            }
        };
        if (tid < head) keep((float)first[tid], tid);
        for (int i0 = tid; i0 < vecs; i0 += U * THREADS) {
            Raw r[U];
#pragma unroll
            for (int k = 0; k < U; ++k) {
                const int i = i0 + k * THREADS;
                r[k] = Raw{fill, fill, fill, fill};
                if (i < full) r[k] = whole(i);
                else if (i < vecs) r[k] = partial();
            }
#pragma unroll
            for (int k = 0; k < U; ++k)
#pragma unroll
                for (int e = 0; e < VEC; ++e) keep(wide(r[k], e), head + (i0 + k * THREADS) * VEC + e);
        }
    }
    __syncthreads();
    const int count = (int)s_count;
    auto give = [&](int rank, u64 key) {
        const u32 o = (u32)(key >> 32);
        const float v = score_of(o);
        top_lp[rank] = (v - m) - log_sum;
        top_id[rank] = (int)~(u32)key;
    };
    if (count <= KEPT) {
        for (int i = tid; i < count; i += THREADS) {
            const u64 key = s_key[i];
            int rank = 0;
            for (int j = 0; j < count; ++j) rank += s_key[j] > key;
            if (rank < A.top) give(rank, key);
        }
        for (int i = count + tid; i < A.top; i += THREADS) top_lp[i] = low, top_id[i] = -1;
    } else {
        u64 last = ~0ull;
        for (int r = 0; r < A.top; ++r) {               // more candidates than KEPT >= top: every round finds one
            u64 best = 0;
            each([&](float v, int c) {
                const u32 o = order_of(v);
                const u64 key = (u64)o << 32 | (u32)~c;
                if (o >= bound && key < last && key > best) best = key;
            });
#pragma unroll
            for (int d = 32; d; d >>= 1) {
                const u64 other = __shfl_xor(best, d);
                best = other > best ? other : best;
            }
            if (lane == 0) s_pick[wave] = best;
            __syncthreads();
#pragma unroll
            for (int i = 0; i < WAVES; ++i) best = s_pick[i] > best ? s_pick[i] : best;
            __syncthreads();
            if (tid == 0) give(r, best);
            last = best;
        }
    }
}

constexpr int ROWS = 1 << 21;        // of one launch: 1024 threads each stay below 2^32

template <typename T> int logprobs_launch(hipStream_t s, ScoreArgs &A, int rows)
{
    constexpr int VEC = 16 / (int)sizeof(T);
    const int vecs = (A.classes + VEC - 1) / VEC;
    // eight vectors a thread; where there are fewer rows than compute units a row's latency is all that counts: two
    const int want = rows <= 256 ? vecs / 2 : vecs / 8;
    for (A.first = 0; A.first < rows; A.first += A.rows) {
        A.rows = rows - A.first < ROWS ? rows - A.first : ROWS;
        const dim3 grid((unsigned)A.rows);
        if (want <= 64) k_logprobs<T, 64><<<grid, 64, 0, s>>>(A);
        else if (want <= 256) k_logprobs<T, 256><<<grid, 256, 0, s>>>(A);
        else if (want <= 512) k_logprobs<T, 512><<<grid, 512, 0, s>>>(A);
        else k_logprobs<T, 1024><<<grid, 1024, 0, s>>>(A);
    }
    return ops_launched("ob_token_logprobs");
}

struct ScoreGradArgs {
    const void *x;
    i64 x_row;
    const void *labels;
    int labels_wide, first, rows, classes, piece;      // rows of one launch, from `first` on; piece: vectors of a row for one workgroup
    const float *row_max, *row_sum, *entropy, *dlogprob, *dentropy;
    void *dx;
    i64 dx_row;
};

// dx_c = a (1[c = y] - p_c) - b p_c (log p_c + H).  Elementwise: a reading and a writing, rows from the last on, since the last ones that the
// forward pass read are still in the last-level cache.  4096 rows of 50 257 bf16: 156 us, 5.3 TB/s (and 104 us for the
// forward pass before it, which finds the caches full of the last gradient; by itself that takes 83 to 88).
template <typename T> __global__ void __launch_bounds__(256) k_logprobs_grad(const ScoreGradArgs A)
{
    constexpr int VEC = 16 / (int)sizeof(T), U = 4;
    typedef typename Pack<T, VEC>::V V;
    const int row = A.first + A.rows - 1 - (int)blockIdx.x;
    const T *x = (const T *)A.x + row * A.x_row;
    T *dx = (T *)A.dx + row * A.dx_row;
    const i64 label = label_of(A.labels, A.labels_wide, row);
    const int y = label >= 0 && label < A.classes ? (int)label : -1;
    const float m = A.row_max[row], sum = A.row_sum[row], h = A.entropy[row];
    float a = A.dlogprob && label >= 0 ? A.dlogprob[row] : 0.0f;
    const float b = A.dentropy ? A.dentropy[row] : 0.0f;
    if (label >= A.classes) a = __builtin_nanf("");
    const bool empty = sum == 0.0f;
    // without a gradient of the entropy, the entropy has no part (a row that is not finite has a sum of NaN)
    const float inv = 1.0f / sum, log_sum = logf(sum), ab = b == 0.0f ? a : a + b * (h - log_sum);
    const int full = A.classes / VEC, vecs = (A.classes + VEC - 1) / VEC;
    const int v0 = (int)blockIdx.y * A.piece, v1 = min(vecs, v0 + A.piece);
    auto grad = [&](float v, int c) {
        const float d = fmaxf(v - m, -1e4f), p = __expf(v - m) * inv;      // a NaN goes on through p
        const float r = (c == y ? a : 0.0f) - p * (ab + b * d);
        return empty ? 0.0f : r;
    };
    for (int i0 = v0 + (int)threadIdx.x; i0 < v1; i0 += U * 256) {
        V v[U];
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const int i = i0 + k * 256;
            if (i < min(v1, full)) v[k] = load_n<T, VEC>(x + i * VEC);
        }
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const int i = i0 + k * 256;
            if (i >= v1) break;
            if (i < full) {
                V r;
#pragma unroll
                for (int e = 0; e < VEC; ++e) r[e] = (T)grad((float)v[k][e], i * VEC + e);
                store_n<T, VEC>(dx + i * VEC, r);
            } else
                for (int c = i * VEC; c < A.classes; ++c) dx[c] = (T)grad((float)x[c], c);
        }
    }
}

template <typename T> int grad_launch(hipStream_t s, ScoreGradArgs &A, int rows)
{
    constexpr int VEC = 16 / (int)sizeof(T);
    const int vecs = (A.classes + VEC - 1) / VEC;
    // a workgroup has a whole row where there are rows enough for the chip, else a piece of one
    int pieces = 1;
    while (pieces < 64 && (i64)rows * pieces < 1024 && vecs > 256 * pieces) pieces *= 2;
    A.piece = (vecs + pieces - 1) / pieces;
    for (int end = rows; end; end = A.first) {                  // the last rows first, here too
        A.first = end > ROWS ? end - ROWS : 0, A.rows = end - A.first;
        k_logprobs_grad<T><<<dim3((unsigned)A.rows, (unsigned)pieces), 256, 0, s>>>(A);
    }
    return ops_launched("ob_token_logprobs_grad");
}

int check_scores(const ob_logprobs *p, const char *who)
{
    if (!p) return ops_fail(OB_E_ARG, "%s: null argument", who);
    if (p->type < OB_TYPE_FP32 || p->type > OB_TYPE_FP16) return ops_fail(OB_E_ARG, "%s: element type %d", who, p->type);
    if (p->rows < 0 || p->classes < 1 || p->classes > (1 << 30)) return ops_fail(OB_E_DIM, "%s: %d rows of %d classes", who, p->rows, p->classes);
    if (p->top < 0 || p->top > OB_TOP_MAX || p->top > p->classes) return ops_fail(OB_E_RANGE, "%s: %d alternatives of %d classes (at most %d)", who, p->top, p->classes, OB_TOP_MAX);
    if (p->rows && (!p->scores || !p->labels || !p->logprob || !p->entropy || !p->row_max || !p->row_sum)) return ops_fail(OB_E_ARG, "%s: null array", who);
    return OB_OK;
}

}  // namespace

extern "C" {

int ob_token_logprobs(void *hip_stream, const ob_logprobs *p)
{
    if (int rc = check_scores(p, "ob_token_logprobs")) return rc;
    if (p->rows && p->top && (!p->top_logprobs || !p->top_ids)) return ops_fail(OB_E_ARG, "ob_token_logprobs: null array");
    if (!p->rows) return OB_OK;
    ScoreArgs A;
    A.x = p->scores, A.x_row = p->score_stride, A.labels = p->labels, A.labels_wide = p->labels_wide;
    A.first = 0, A.rows = 0, A.classes = p->classes, A.top = p->top;
    A.logprob = p->logprob, A.entropy = p->entropy, A.row_max = p->row_max, A.row_sum = p->row_sum;
    A.top_logprob = p->top_logprobs, A.top_id = p->top_ids;
    hipStream_t s = (hipStream_t)hip_stream;
    return p->type == OB_TYPE_FP32 ? logprobs_launch<float>(s, A, p->rows) : p->type == OB_TYPE_BF16 ? logprobs_launch<bf16>(s, A, p->rows) : logprobs_launch<f16>(s, A, p->rows);
}

int ob_token_logprobs_grad(void *hip_stream, const ob_logprobs *p)
{
    if (int rc = check_scores(p, "ob_token_logprobs_grad")) return rc;
    if (p->rows && !p->dscores) return ops_fail(OB_E_ARG, "ob_token_logprobs_grad: null array");
    if (!p->rows) return OB_OK;
    ScoreGradArgs A;
    A.x = p->scores, A.x_row = p->score_stride, A.labels = p->labels, A.labels_wide = p->labels_wide;
    A.first = 0, A.rows = 0, A.classes = p->classes, A.piece = 0;
    A.row_max = p->row_max, A.row_sum = p->row_sum, A.entropy = p->entropy, A.dlogprob = p->dlogprob, A.dentropy = p->dentropy;
    A.dx = p->dscores, A.dx_row = p->dscore_stride;
    hipStream_t s = (hipStream_t)hip_stream;
    return p->type == OB_TYPE_FP32 ? grad_launch<float>(s, A, p->rows) : p->type == OB_TYPE_BF16 ? grad_launch<bf16>(s, A, p->rows) : grad_launch<f16>(s, A, p->rows);
}

}  // extern "C"
