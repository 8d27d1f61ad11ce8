// Operators on device arrays: decay attention (forward, gradients, one token at a time).  The scan's kernels are in ob_attn.h.
#include "ob_attn.h"
#include "ob_ctx.h"

#include <algorithm>
#include <cstdarg>
#include <cstdio>

int ops_fail(int code, const char *fmt, ...)
{
    char buf[480];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    return ctx_fail(nullptr, code, "%s", buf);
}

// ---- one token -------------------------------------------------------------------------------------------------------
// S = lambda S + k v^T, o = scale q S, the state in place: 8 bytes of state an element against 5 operations, so the state's bytes are all that
// counts.  A workgroup has the state of one sequence and head; a thread has 4 of its columns and every TY-th row, 8 rows of loads under way at a
// time, and the sums over rows meet in LDS in a fixed order.  256 sequences of 16 heads, 128 x 128: 105 us, 5.1 TB/s (a copy: 4.7).
struct StepArgs {
    Rows q, k, v;
    void *o;
    i64 o_token, o_head;
    const float *log_decay;
    float *state;
    float scale;
    int heads, dk, dv;
};

template <typename T, int TX> __global__ void __launch_bounds__(256) k_step(const StepArgs A)
{
    __shared__ float s_q[128], s_k[128];
    __shared__ f4 s_o[256];
    const int tx = threadIdx.x % TX, ty = threadIdx.x / TX, TY = blockDim.x / TX;
    const int seq = blockIdx.x / A.heads, head = blockIdx.x % A.heads, col = 4 * tx;
    const int cols = min(4, A.dv - col);                // <= 0: no column of this thread
    float *S = A.state + (i64)blockIdx.x * A.dk * A.dv + col;
    const T *pv = (const T *)A.v.p + seq * A.v.token + head / A.v.div * A.v.head + col;
    f4 v = {0.f, 0.f, 0.f, 0.f}, o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (e < cols) v[e] = (float)pv[e];
    for (int i = threadIdx.x; i < A.dk; i += blockDim.x) {
        s_q[i] = (float)((const T *)A.q.p)[seq * A.q.token + head / A.q.div * A.q.head + i] * A.scale;
        s_k[i] = (float)((const T *)A.k.p)[seq * A.k.token + head / A.k.div * A.k.head + i];
    }
    const float keep = decay_power(A.log_decay[head], 1);
    __syncthreads();
    for (int r0 = ty; r0 < A.dk; r0 += 8 * TY) {
        f4 x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int row = r0 + j * TY;
            x[j] = f4{0.f, 0.f, 0.f, 0.f};
            if (row < A.dk) {
                const float *p = S + row * A.dv;
                if (cols == 4) x[j] = load_n<float, 4>(p);
                else
#pragma unroll
                    for (int e = 0; e < 3; ++e)
                        if (e < cols) x[j][e] = p[e];
            }
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int row = r0 + j * TY;
            if (row < A.dk) {
                const f4 y = x[j] * keep + v * s_k[row];
                o += y * s_q[row];
                float *p = S + row * A.dv;
                if (cols == 4) store_n<float, 4>(p, y);
                else
#pragma unroll
                    for (int e = 0; e < 3; ++e)
                        if (e < cols) p[e] = y[e];
            }
        }
    }
    s_o[threadIdx.x] = o;
    __syncthreads();
    if ((int)threadIdx.x < A.dv) {
        const float *p = (const float *)s_o + threadIdx.x;
        float sum = 0.0f;
        for (int y = 0; y < TY; ++y) sum += p[y * (4 * TX)];
        ((T *)A.o)[seq * A.o_token + head * A.o_head + threadIdx.x] = (T)sum;
    }
}

template <typename T> static int step_launch(hipStream_t s, const StepArgs &A, int n)
{
    // threads: as many columns as the width needs, rows for 256 threads or 8 rows each, whichever is less, but a thread for each column of o
    const int tx = A.dv <= 32 ? 8 : A.dv <= 64 ? 16 : 32;
    int threads = 64;
    while (threads < 256 && (threads < 4 * tx || 8 * (threads / tx) < A.dk)) threads *= 2;
    if (!launch_fits((i64)n * A.heads, threads)) return ops_fail(OB_E_RANGE, "ob_decay_attention_step: %d sequences of %d heads", n, A.heads);
    const dim3 grid((unsigned)n * (unsigned)A.heads);
    if (tx == 8) k_step<T, 8><<<grid, threads, 0, s>>>(A);
    else if (tx == 16) k_step<T, 16><<<grid, threads, 0, s>>>(A);
    else k_step<T, 32><<<grid, threads, 0, s>>>(A);
    return ops_launched("ob_decay_attention_step");
}

// ---- gradients of shared heads ---------------------------------------------------------------------------------------
// The fp32 gradients of each query head, summed over the heads that share keys and values: two arrays a launch, four elements a thread
// (24 915 tokens, 16 heads over 4, 128 + 128: 90 us, 5.1 TB/s; element by element 135).
struct SumArgs {
    const float *part[2];
    void *out[2];
    i64 out_token[2], out_head[2];
    int width[2];
    i64 rows;                       // tokens * heads of keys and values
    int kv_heads, group;
};
template <typename T> __global__ void __launch_bounds__(256) k_sum_heads(const SumArgs A)
{
    const int which = blockIdx.y, d = A.width[which], quads = (d + 3) / 4, per = 256 / quads;
    const int c = (int)threadIdx.x % quads * 4;
    const i64 row = (i64)blockIdx.x * per + (int)threadIdx.x / quads;
    if ((int)threadIdx.x >= per * quads || row >= A.rows) return;
    const float *p = A.part[which] + row * A.group * d + c;
    T *o = (T *)A.out[which] + row / A.kv_heads * A.out_token[which] + row % A.kv_heads * A.out_head[which] + c;
    if (c + 4 <= d) {
        f4 sum = load_n<float, 4>(p);
        for (int g = 1; g < A.group; ++g) sum += load_n<float, 4>(p + g * d);
        typename Pack<T, 4>::V z;
#pragma unroll
        for (int e = 0; e < 4; ++e) z[e] = (T)sum[e];
        store_n<T, 4>(o, z);
    } else
        for (int e = 0; c + e < d; ++e) {
            float sum = 0.0f;
            for (int g = 0; g < A.group; ++g) sum += p[g * d + e];
            o[e] = (T)sum;
        }
}

// ---- the entries' host side ------------------------------------------------------------------------------------------
static int check_decay(const ob_decay *p, const char *who, bool packed)
{
    if (!p) return ops_fail(OB_E_ARG, "%s: null argument", who);
    if (p->type < OB_TYPE_FP32 || p->type > OB_TYPE_FP16) return ops_fail(OB_E_ARG, "%s: element type %d", who, p->type);
    if (p->heads < 1 || p->kv_heads < 1 || p->heads % p->kv_heads || p->heads > 65535)
        return ops_fail(OB_E_DIM, "%s: %d heads over %d of keys and values", who, p->heads, p->kv_heads);
    if (p->dk < 1 || p->dk > 128 || p->dv < 1 || p->dv > 128) return ops_fail(OB_E_DIM, "%s: widths %d and %d (1 .. 128)", who, p->dk, p->dv);
    if (p->n_seqs < 0 || p->tokens < 0 || p->tokens > 0x7fffffff) return ops_fail(OB_E_RANGE, "%s: %d sequences, %lld tokens", who, p->n_seqs, (long long)p->tokens);
    if (p->n_seqs && !p->log_decay) return ops_fail(OB_E_ARG, "%s: no decay", who);
    if (p->tokens && (!p->q.data || !p->k.data || !p->v.data || !p->o.data)) return ops_fail(OB_E_ARG, "%s: null array", who);
    // a scan's places in a chunk are 32-bit offsets; single tokens' are 64 bits, and of one row the stride is not looked at
    const bool walked = packed && p->tokens > 1;
    for (const ob_rows *r : {&p->q, &p->k, &p->v, &p->o, &p->dq, &p->dk_rows, &p->dv_rows})
        if (r->token_stride < 0 || (walked && r->token_stride >= 1 << 24) || r->head_stride < 0)
            return ops_fail(OB_E_RANGE, "%s: strides of %lld and %lld elements", who, (long long)r->token_stride, (long long)r->head_stride);
    if (!packed) {
        if (p->tokens != p->n_seqs) return ops_fail(OB_E_DIM, "%s: %lld tokens of %d sequences", who, (long long)p->tokens, p->n_seqs);
        return OB_OK;
    }
    if (!p->offsets) return ops_fail(OB_E_ARG, "%s: no offsets", who);
    if (p->offsets[0] != 0 || p->offsets[p->n_seqs] != p->tokens)
        return ops_fail(OB_E_RANGE, "%s: offsets go from %lld to %lld, tokens from 0 to %lld", who, (long long)p->offsets[0], (long long)p->offsets[p->n_seqs],
                        (long long)p->tokens);
    for (int i = 0; i < p->n_seqs; ++i)
        if (p->offsets[i + 1] < p->offsets[i]) return ops_fail(OB_E_RANGE, "%s: offsets fall at sequence %d", who, i);
    return OB_OK;
}

// A few long sequences are cut into segments, so that they fill the chip: their segments' states are made first (one more reading of two of the
// three inputs).  A segment is what 512 workgroups, two a compute unit, have each if they share all tokens of all scans evenly.
// Where the longest sequence has at most two segments nothing is cut, else what is longer than five quarters of one (us, cut then for left whole):
// 24 sequences of up to 4096, gradients, 451 for 427; 24 and 20 of 4096 each, 16 heads, 720 for 405 and 602 for 372; 28 prompts of up to 2900,
// 32 heads, 264 for 233.  With sequences of up to three segments left whole: 24 prompts of up to 4096 309 for 266, 14 sequences' gradients
// 353 for 335 (but 15 of 4096 each 325 for 389).  Cut from 3/2, 2 and 3 segments on in place of 5/4: 8 prompts of up to 16 384, 393, 456 and
// 505 for 378.  One sequence of 65 536, 16 heads: 368, and 411 for segments of 768 workgroups, 423 of 1024.
static bool is_cut(i64 n, i64 segment) { return 4 * n > 5 * segment; }
static int segment_of(const ob_decay *p, int scans)
{
    i64 seg = (p->tokens * p->heads * scans + 511) / 512;
    seg = std::max<i64>(256, (seg + CH - 1) / CH * CH);
    i64 longest = 0;
    for (int i = 0; i < p->n_seqs; ++i) longest = std::max<i64>(longest, p->offsets[i + 1] - p->offsets[i]);
    if (longest <= 2 * seg) seg = std::max(seg, (longest + CH - 1) / CH * CH);
    for (;;) {
        int most = 0;
        for (int first = 0; first < p->n_seqs; first += ATT_SEQS) {
            int cut = 0;
            for (int i = first; i < std::min(p->n_seqs, first + ATT_SEQS); ++i) cut += is_cut(p->offsets[i + 1] - p->offsets[i], seg);
            most = std::max(most, cut);
        }
        if (most <= ATT_SPLIT) return (int)std::min<i64>(seg, 0x7fffffff);
        seg *= 2;
    }
}

// the tables of the launch that has the sequences from first_seq on
static void fill_units(ScanArgs &A, const ob_decay *p, int first_seq, int segment)
{
    A.first_seq = first_seq;
    const int n_seqs = std::min(ATT_SEQS, p->n_seqs - first_seq);
    A.segment = segment;
    A.n_split = 0;
    bool ordered = true;
    i64 longest = 0;
    for (int i = 0; i < n_seqs; ++i) {
        A.off[i] = (u32)p->offsets[first_seq + i];
        A.order[i] = (uint16_t)i;
        const i64 n = p->offsets[first_seq + i + 1] - p->offsets[first_seq + i];
        longest = std::max(longest, n);
        A.n_split += is_cut(n, segment);
        if (i && n > (i64)(A.off[i] - A.off[i - 1])) ordered = false;
    }
    A.off[n_seqs] = (u32)p->offsets[first_seq + n_seqs];
    // the longest first: they end last (512 sequences of up to 60 tokens in the order they came: 48 us for 43).  Sequences of one chunk take the
    // same time whatever their lengths are, and are spared the look into the order.
    A.ordered = ordered || longest <= CH;
    if (!A.ordered)
        std::sort(A.order, A.order + n_seqs, [&](uint16_t x, uint16_t y) {
            const u32 a = A.off[x + 1] - A.off[x], b = A.off[y + 1] - A.off[y];
            return a != b ? a > b : x < y;
        });
    A.cum[0] = 0;
    for (int r = 0; r < A.n_split; ++r) {
        const u32 n = A.off[A.order[r] + 1] - A.off[A.order[r]];
        A.cum[r + 1] = A.cum[r] + (n + segment - 1) / segment;
    }
    A.n_cut = (int)A.cum[A.n_split];
    A.n_units = A.n_cut + n_seqs - A.n_split;
}

// workgroups read the states that enter while others write those that leave
static bool share_memory(const ob_decay *p, const float *x, const float *y)
{
    const uintptr_t a = (uintptr_t)x, b = (uintptr_t)y, bytes = (uintptr_t)p->n_seqs * p->heads * p->dk * p->dv * sizeof(float);
    return a && b && a < b + bytes && b < a + bytes;
}

static int pad_width(int d) { return d <= 32 ? 32 : d <= 64 ? 64 : 128; }

// bytes of the states of segments, at most over the launches
static size_t slot_bytes(const ob_decay *p, int segment, int scans)
{
    size_t most = 0;
    for (int first = 0; first < p->n_seqs; first += ATT_SEQS) {
        size_t units = 0;
        for (int i = first; i < std::min(p->n_seqs, first + ATT_SEQS); ++i) {
            const i64 n = p->offsets[i + 1] - p->offsets[i];
            if (is_cut(n, segment)) units += (size_t)((n + segment - 1) / segment);
        }
        most = std::max(most, units);
    }
    return (most * p->heads * pad_width(p->dk) * pad_width(p->dv) * 4 * scans + 255) & ~(size_t)255;
}
static size_t part_bytes(const ob_decay *p)
{
    return p->heads == p->kv_heads ? 0 : (size_t)p->tokens * p->heads * (p->dk + p->dv) * 4;
}
// the gradients' scans go together where keys and values take the same tiles, else that of dv goes by itself
static int grad_scans(const ob_decay *p) { return pad_width(p->dk) == pad_width(p->dv) ? 3 : 2; }

static Rows rows_of(const ob_rows &r, int div) { return Rows{r.data, r.token_stride, r.head_stride, div, 0}; }
static i64 token_step(const ob_decay *p, const ob_rows &r) { return p->tokens > 1 ? r.token_stride : 0; }
static Rows scan_rows(const ob_decay *p, const ob_rows &r, int div) { return Rows{r.data, token_step(p, r), r.head_stride, div, 0}; }

static int scan_all(hipStream_t s, ScanArgs &A, const ob_decay *p, int segment)
{
    const ScanLaunch f = p->type == OB_TYPE_FP32 ? scan_f32 : p->type == OB_TYPE_BF16 ? scan_bf16 : scan_f16;
    for (int first = 0; first < p->n_seqs; first += ATT_SEQS) {
        fill_units(A, p, first, segment);
        if (int rc = f(s, A, p->heads / p->kv_heads)) return rc;
    }
    return OB_OK;
}

static int sum_heads(hipStream_t s, const ob_decay *p, const float *dk, const float *dv)
{
    SumArgs A;
    const ob_rows *out[2] = {&p->dk_rows, &p->dv_rows};
    A.part[0] = dk, A.part[1] = dv, A.width[0] = p->dk, A.width[1] = p->dv;
    for (int i = 0; i < 2; ++i) A.out[i] = out[i]->data, A.out_token[i] = out[i]->token_stride, A.out_head[i] = out[i]->head_stride;
    A.rows = p->tokens * p->kv_heads, A.kv_heads = p->kv_heads, A.group = p->heads / p->kv_heads;
    if (!A.rows) return OB_OK;
    const int per = 256 / ((std::max(p->dk, p->dv) + 3) / 4);       // rows of a workgroup, at least
    const i64 blocks = (A.rows + per - 1) / per;
    if (!launch_fits(blocks, 256)) return ops_fail(OB_E_RANGE, "ob_decay_attention_grad: %lld rows", (long long)A.rows);
    const dim3 grid((unsigned)blocks, 2);
    if (p->type == OB_TYPE_FP32) k_sum_heads<float><<<grid, 256, 0, s>>>(A);
    else if (p->type == OB_TYPE_BF16) k_sum_heads<bf16><<<grid, 256, 0, s>>>(A);
    else k_sum_heads<f16><<<grid, 256, 0, s>>>(A);
    return ops_launched("ob_decay_attention_grad");
}

extern "C" {

int ob_decay_workspace(const ob_decay *p, int grad, uint64_t *bytes)
{
    if (!bytes) return ops_fail(OB_E_ARG, "ob_decay_workspace: null argument");
    *bytes = 0;
    if (int rc = check_decay(p, "ob_decay_workspace", true)) return rc;
    const int scans = grad ? grad_scans(p) : 1;
    *bytes = slot_bytes(p, segment_of(p, scans), scans) + (grad ? part_bytes(p) : 0);
    return OB_OK;
}

int ob_decay_attention(void *hip_stream, const ob_decay *p)
{
    if (int rc = check_decay(p, "ob_decay_attention", true)) return rc;
    if (!p->n_seqs) return OB_OK;
    if (share_memory(p, p->state_in, p->state_out)) return ops_fail(OB_E_ARG, "ob_decay_attention: state_in and state_out share memory");
    const int segment = segment_of(p, 1), group = p->heads / p->kv_heads;
    const size_t need = slot_bytes(p, segment, 1);
    if (need > p->workspace_bytes || (need && !p->workspace))
        return ops_fail(OB_E_OOM, "ob_decay_attention: workspace of %llu bytes, %zu are needed", (unsigned long long)p->workspace_bytes, need);
    ScanArgs A;
    A.n_scans = 1, A.heads = p->heads, A.log_decay = p->log_decay, A.slots = (float *)p->workspace;
    Scan &x = A.scan[0];
    x.a = scan_rows(p, p->q, 1), x.b = scan_rows(p, p->k, group), x.c = scan_rows(p, p->v, group);
    x.y = p->o.data, x.y_token = token_step(p, p->o), x.y_head = p->o.head_stride;
    x.s_in = p->state_in, x.s_out = p->state_out;
    x.sp = x.sy = (float)p->scale, x.ss = 1.0f;
    x.da = p->dk, x.dc = p->dv, x.s_row = p->dv, x.s_col = 1;
    x.reverse = 0, x.y_float = p->type == OB_TYPE_FP32, x.exact_state = p->state_out != nullptr;
    return scan_all((hipStream_t)hip_stream, A, p, segment);
}

int ob_decay_attention_grad(void *hip_stream, const ob_decay *p)
{
    if (int rc = check_decay(p, "ob_decay_attention_grad", true)) return rc;
    if (!p->n_seqs) return OB_OK;
    if (p->tokens && (!p->dq.data || !p->dk_rows.data || !p->dv_rows.data)) return ops_fail(OB_E_ARG, "ob_decay_attention_grad: null array");
    if (share_memory(p, p->state_in, p->dstate_in) || share_memory(p, p->dstate_out, p->dstate_in))
        return ops_fail(OB_E_ARG, "ob_decay_attention_grad: dstate_in shares memory with a state that is read");
    hipStream_t s = (hipStream_t)hip_stream;
    const int scans = grad_scans(p), segment = segment_of(p, scans), group = p->heads / p->kv_heads;
    const size_t slots = slot_bytes(p, segment, scans), need = slots + part_bytes(p);
    if (need > p->workspace_bytes || (need && !p->workspace))
        return ops_fail(OB_E_OOM, "ob_decay_attention_grad: workspace of %llu bytes, %zu are needed", (unsigned long long)p->workspace_bytes, need);
    float *part_k = (float *)((char *)p->workspace + slots), *part_v = part_k + p->tokens * p->heads * p->dk;
    ScanArgs A;
    A.n_scans = scans, A.heads = p->heads, A.log_decay = p->log_decay, A.slots = (float *)p->workspace;
    // dq: the scan of do against v and k, on the transposed state
    Scan &q = A.scan[0], &k = A.scan[1];
    q.a = scan_rows(p, p->o, 1), q.b = scan_rows(p, p->v, group), q.c = scan_rows(p, p->k, group);
    q.y = p->dq.data, q.y_token = token_step(p, p->dq), q.y_head = p->dq.head_stride;
    q.s_in = p->state_in, q.s_out = nullptr;
    q.sp = q.sy = (float)p->scale, q.ss = 1.0f;
    q.da = p->dv, q.dc = p->dk, q.s_row = 1, q.s_col = p->dv;
    q.reverse = 0, q.y_float = p->type == OB_TYPE_FP32, q.exact_state = 0;
    // dk and dv: from the last token to the first, on the gradient of the state; the heads of a group are summed in fp32
    k = q;
    k.reverse = 1, k.y_float = group > 1 || p->type == OB_TYPE_FP32;
    k.sp = k.ss = (float)p->scale, k.sy = 1.0f;
    k.s_in = p->dstate_out;
    Scan v = k;
    k.a = scan_rows(p, p->v, group), k.b = scan_rows(p, p->o, 1), k.c = scan_rows(p, p->q, 1);
    k.y = p->dk_rows.data, k.y_token = token_step(p, p->dk_rows), k.y_head = p->dk_rows.head_stride;
    if (group > 1) k.y = part_k, k.y_token = (i64)p->heads * p->dk, k.y_head = p->dk;
    v.a = scan_rows(p, p->k, group), v.b = scan_rows(p, p->q, 1), v.c = scan_rows(p, p->o, 1);
    v.y = p->dv_rows.data, v.y_token = token_step(p, p->dv_rows), v.y_head = p->dv_rows.head_stride;
    if (group > 1) v.y = part_v, v.y_token = (i64)p->heads * p->dv, v.y_head = p->dv;
    v.da = p->dk, v.dc = p->dv, v.s_row = p->dv, v.s_col = 1;
    v.s_out = p->dstate_in, v.exact_state = p->dstate_in != nullptr;
    if (scans == 3) A.scan[2] = v;
    if (int rc = scan_all(s, A, p, segment)) return rc;
    if (scans == 2) {
        A.n_scans = 1, A.scan[0] = v;
        if (int rc = scan_all(s, A, p, segment)) return rc;
    }
    return group > 1 ? sum_heads(s, p, part_k, part_v) : OB_OK;
}

int ob_decay_attention_step(void *hip_stream, const ob_decay *p)
{
    if (int rc = check_decay(p, "ob_decay_attention_step", false)) return rc;
    if (!p->n_seqs) return OB_OK;
    if (!p->state_out) return ops_fail(OB_E_ARG, "ob_decay_attention_step: no state");
    const int group = p->heads / p->kv_heads;
    StepArgs A;
    A.q = rows_of(p->q, 1), A.k = rows_of(p->k, group), A.v = rows_of(p->v, group);
    A.o = p->o.data, A.o_token = p->o.token_stride, A.o_head = p->o.head_stride;
    A.log_decay = p->log_decay, A.state = p->state_out, A.scale = (float)p->scale;
    A.heads = p->heads, A.dk = p->dk, A.dv = p->dv;
    hipStream_t s = (hipStream_t)hip_stream;
    return p->type == OB_TYPE_FP32 ? step_launch<float>(s, A, p->n_seqs) : p->type == OB_TYPE_BF16 ? step_launch<bf16>(s, A, p->n_seqs)
                                                                                                    : step_launch<f16>(s, A, p->n_seqs);
}

}  // extern "C"
