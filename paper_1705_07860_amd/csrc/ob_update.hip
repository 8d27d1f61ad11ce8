// The norm of all gradients together, and the gradient step (or the gradients themselves) clipped to it.
#include "ob_dev.h"
#include "ob_ctx.h"

#include <algorithm>
#include <memory>
#include <new>

namespace {

constexpr int TENSORS = 128;         // of one launch: the table travels in the kernel's arguments
constexpr int CHUNK = 8192;          // elements that a workgroup takes at a time
constexpr int NORM_BLOCKS = 1024;    // partial sums of one launch

struct Entry {
    void *g, *p;
    i64 n_types;                     // elements * 16 + type of p * 4 + type of g
};
struct UpdateArgs {
    double *part;                    // partial sums of all launches
    int part_first, part_count, n, clip_grads;
    float *norm;
    double max_norm, lr;
    u32 cum[TENSORS + 1];            // chunks before each tensor
    Entry t[TENSORS];
};
static_assert(sizeof(UpdateArgs) <= 4096, "kernel arguments");

__device__ __forceinline__ int tensor_of(const UpdateArgs &A, u32 chunk)
{
    int lo = 0, hi = A.n;            // cum[lo] <= chunk < cum[hi]; tensors of no chunk are passed over
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (A.cum[mid] <= chunk) lo = mid; else hi = mid;
    }
    return lo;
}

// the sum of 256 threads' numbers, in every thread, added in a fixed order
__device__ __forceinline__ double block_sum(double x, double *s_part)
{
#pragma unroll
    for (int d = 32; d; d >>= 1) x += __shfl_xor(x, d);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) s_part[threadIdx.x >> 6] = x;
    __syncthreads();
    return (s_part[0] + s_part[1]) + (s_part[2] + s_part[3]);
}

template <typename T> __device__ __forceinline__ double squares(const T *g, i64 n)
{
    constexpr int VEC = 16 / (int)sizeof(T), U = CHUNK / VEC / 256;
    typedef typename Pack<T, VEC>::V V;
    double sum[2] = {0.0, 0.0};
    const int at = (int)threadIdx.x * VEC;
    if (n == CHUNK) {
        V v[U];
#pragma unroll
        for (int k = 0; k < U; ++k) v[k] = load_n<T, VEC>(g + at + k * 256 * VEC);
#pragma unroll
        for (int k = 0; k < U; ++k)
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                const double x = (double)(float)v[k][e];
                sum[e & 1] += x * x;
            }
    } else
        for (int i = (int)threadIdx.x; i < n; i += 256) {
            const double x = (double)(float)g[i];
            sum[0] += x * x;
        }
    return sum[0] + sum[1];
}

// Squares are added in 64 bits (their range and the long sum both need it; the reading of the gradients takes longer), each workgroup's in
// the same order whatever the timing, so that the norm is the same bits every time.  400 million bf16: 160 us, 5.0 TB/s.
__global__ void __launch_bounds__(256) k_norm(const UpdateArgs A)
{
    __shared__ double s_part[4];
    double sum = 0.0;
    for (u32 c = blockIdx.x; c < A.cum[A.n]; c += gridDim.x) {
        const int t = tensor_of(A, c);
        const i64 at = (i64)(c - A.cum[t]) * CHUNK, left = (A.t[t].n_types >> 4) - at, n = left < CHUNK ? left : CHUNK;
        const int type = (int)A.t[t].n_types & 3;
        if (type == OB_TYPE_FP32) sum += squares((const float *)A.t[t].g + at, n);
        else if (type == OB_TYPE_BF16) sum += squares((const bf16 *)A.t[t].g + at, n);
        else sum += squares((const f16 *)A.t[t].g + at, n);
    }
    sum = block_sum(sum, s_part);
    if (threadIdx.x == 0) A.part[A.part_first + blockIdx.x] = sum;
}

template <typename P, typename G> __device__ __forceinline__ void step(P *p, const G *g, i64 n, float rate)
{
    constexpr int VEC = 4, U = CHUNK / VEC / 256;
    const int at = (int)threadIdx.x * VEC;
    if (n == CHUNK) {
        typename Pack<G, VEC>::V gv[U];
        typename Pack<P, VEC>::V pv[U];
#pragma unroll
        for (int k = 0; k < U; ++k) gv[k] = load_n<G, VEC>(g + at + k * 256 * VEC), pv[k] = load_n<P, VEC>(p + at + k * 256 * VEC);
#pragma unroll
        for (int k = 0; k < U; ++k) {
            typename Pack<P, VEC>::V r;
#pragma unroll
            for (int e = 0; e < VEC; ++e) r[e] = (P)((float)pv[k][e] - rate * (float)gv[k][e]);
            store_n<P, VEC>(p + at + k * 256 * VEC, r);
        }
    } else
        for (int i = (int)threadIdx.x; i < n; i += 256) p[i] = (P)((float)p[i] - rate * (float)g[i]);
}
template <typename G> __device__ __forceinline__ void clip(G *g, i64 n, float rate)
{
    constexpr int VEC = 16 / (int)sizeof(G);
    i64 i = (i64)threadIdx.x * VEC;
    for (; i + VEC <= n; i += 256 * VEC) {
        typename Pack<G, VEC>::V v = load_n<G, VEC>(g + i);
#pragma unroll
        for (int e = 0; e < VEC; ++e) v[e] = (G)((float)v[e] * rate);
        store_n<G, VEC>(g + i, v);
    }
    for (; i < n; ++i) g[i] = (G)((float)g[i] * rate);
}
template <typename G> __device__ __forceinline__ void step_any(const Entry &t, i64 at, i64 n, float rate, bool clip_grads)
{
    G *g = (G *)t.g + at;
    const int type = (int)t.n_types >> 2 & 3;
    if (clip_grads) clip(g, n, rate);
    else if (type == OB_TYPE_FP32) step((float *)t.p + at, g, n, rate);
    else if (type == OB_TYPE_BF16) step((bf16 *)t.p + at, g, n, rate);
    else step((f16 *)t.p + at, g, n, rate);
}

// Every workgroup adds up the partial sums by itself (some KiB from the L2: less than a launch of their own), then walks its chunks from the
// last on: the gradients that were read last are still in the last-level cache.  400 million parameters of fp32, gradients of bf16: 750 us, 5.3 TB/s.
// Clipping 400 million bf16 gradients in place takes 434 us with the norm, whose reading leaves part of them in the caches.
__global__ void __launch_bounds__(256) k_update(const UpdateArgs A)
{
    __shared__ double s_part[4];
    double sum = 0.0;
    for (int i = (int)threadIdx.x; i < A.part_count; i += 256) sum += A.part[i];
    const double norm = sqrt(block_sum(sum, s_part));
    if (A.norm && blockIdx.x == 0 && threadIdx.x == 0) *A.norm = (float)norm;
    // no limit and an infinite norm clip nothing, nor do zeros; a norm of NaN makes NaN of everything, whatever the limit is
    double by = A.max_norm / norm;
    if (norm != norm) by = norm;
    else if (by > 1.0 || A.max_norm == __builtin_inf() || norm == 0.0) by = 1.0;
    const float rate = (float)(by * A.lr);
    const u32 chunks = A.cum[A.n];
    if (A.clip_grads && rate == 1.0f) return;
    for (u32 i = blockIdx.x; i < chunks; i += gridDim.x) {
        const u32 c = chunks - 1 - i;
        const int t = tensor_of(A, c);
        const i64 at = (i64)(c - A.cum[t]) * CHUNK, left = (A.t[t].n_types >> 4) - at, n = left < CHUNK ? left : CHUNK;
        const int type = (int)A.t[t].n_types & 3;
        if (type == OB_TYPE_FP32) step_any<float>(A.t[t], at, n, rate, A.clip_grads);
        else if (type == OB_TYPE_BF16) step_any<bf16>(A.t[t], at, n, rate, A.clip_grads);
        else step_any<f16>(A.t[t], at, n, rate, A.clip_grads);
    }
}

constexpr int SIZE[3] = {4, 2, 2};   // bytes of an element

// Whether two of the arrays that a call writes share memory: 0 no, 1 yes, -1 no room to find out.  Lists mostly rise in memory already.
int share_memory(const ob_tensor *t, int n)
{
    struct Range { uintptr_t lo, hi; };
    auto range = [](const ob_tensor &x) {
        const uintptr_t lo = (uintptr_t)(x.param ? x.param : x.grad);
        return Range{lo, lo + (uintptr_t)x.n * SIZE[x.param ? x.param_type : x.grad_type]};
    };
    uintptr_t end = 0;
    int i = 0, count = 0;
    for (; i < n; ++i) {
        if (!t[i].n) continue;
        const Range r = range(t[i]);
        if (r.lo < end) break;
        end = r.hi;
    }
    if (i == n) return 0;
    std::unique_ptr<Range[]> all(new (std::nothrow) Range[n]);
    if (!all) return -1;
    for (i = 0; i < n; ++i)
        if (t[i].n) all[count++] = range(t[i]);
    std::sort(all.get(), all.get() + count, [](const Range &a, const Range &b) { return a.lo < b.lo; });
    for (i = 1; i < count; ++i)
        if (all[i].lo < all[i - 1].hi) return 1;
    return 0;
}

// The table of the tensors from `i` on; arrays that adjoin in memory (views of one buffer) become one entry.  Returns the first tensor that
// found no place.
int fill(UpdateArgs &A, const ob_tensor *t, int i, int count)
{
    A.n = 0, A.cum[0] = 0;
    u64 chunks = 0;
    for (; i < count; ++i) {
        if (!t[i].n) continue;
        const i64 types = t[i].param_type * 4 + t[i].grad_type;
        if (A.n) {
            Entry &e = A.t[A.n - 1];
            const i64 n = e.n_types >> 4;
            if ((e.n_types & 15) == types && (char *)e.g + n * SIZE[t[i].grad_type] == (char *)t[i].grad &&
                (t[i].param == nullptr ? e.p == nullptr : (char *)e.p + n * SIZE[t[i].param_type] == (char *)t[i].param)) {
                const i64 all = n + t[i].n;
                chunks = A.cum[A.n - 1] + (u64)((all + CHUNK - 1) / CHUNK);
                e.n_types = all << 4 | types;
                A.cum[A.n] = (u32)chunks;
                continue;
            }
        }
        if (A.n == TENSORS) break;
        A.t[A.n] = Entry{t[i].grad, t[i].param, t[i].n << 4 | types};
        chunks += (u64)((t[i].n + CHUNK - 1) / CHUNK);         // the entry refuses what would pass 32 bits
        A.cum[++A.n] = (u32)chunks;
    }
    return i;
}

}  // namespace

extern "C" {

int ob_clip_workspace(const ob_tensor *tensors, int n, uint64_t *bytes)
{
    if (!bytes || n < 0 || (n && !tensors)) return ops_fail(OB_E_ARG, "ob_clip_workspace: null argument");
    *bytes = (uint64_t)((n + TENSORS - 1) / TENSORS + 1) * NORM_BLOCKS * sizeof(double);
    return OB_OK;
}

int ob_clip_step(void *hip_stream, const ob_tensor *tensors, int n, double max_norm, double lr, float *norm, void *workspace, uint64_t workspace_bytes)
{
    if (n < 0 || (n && !tensors) || !norm) return ops_fail(OB_E_ARG, "ob_clip_step: null argument");
    if (!(max_norm >= 0.0)) return ops_fail(OB_E_ARG, "ob_clip_step: norm %g to clip to", max_norm);
    const uint64_t need = (uint64_t)((n + TENSORS - 1) / TENSORS + 1) * NORM_BLOCKS * sizeof(double);
    if (!workspace || workspace_bytes < need)
        return ops_fail(OB_E_OOM, "ob_clip_step: workspace of %llu bytes, %llu are needed", (unsigned long long)workspace_bytes, (unsigned long long)need);
    bool params = false, none = false;
    int64_t all = 0;
    for (int i = 0; i < n; ++i) {
        const ob_tensor &t = tensors[i];
        if (t.n < 0 || t.n >= (1ll << 40)) return ops_fail(OB_E_RANGE, "ob_clip_step: tensor %d has %lld elements", i, (long long)t.n);
        if (t.grad_type < OB_TYPE_FP32 || t.grad_type > OB_TYPE_FP16 || t.param_type < OB_TYPE_FP32 || t.param_type > OB_TYPE_FP16)
            return ops_fail(OB_E_ARG, "ob_clip_step: tensor %d has element types %d and %d", i, t.grad_type, t.param_type);
        if ((all += t.n) >= (1ll << 43)) return ops_fail(OB_E_RANGE, "ob_clip_step: more than 2^43 elements");
        if (!t.n) continue;
        if (!t.grad) return ops_fail(OB_E_ARG, "ob_clip_step: tensor %d has no gradient", i);
        (t.param ? params : none) = true;
    }
    if (params && none) return ops_fail(OB_E_ARG, "ob_clip_step: parameters for some of the gradients only");
    if (const int shared = share_memory(tensors, n))
        return shared < 0 ? ops_fail(OB_E_OOM, "ob_clip_step: no host memory for %d tensors", n)
                          : ops_fail(OB_E_ARG, "ob_clip_step: two %s share memory", params ? "parameters" : "gradients");
    hipStream_t s = (hipStream_t)hip_stream;
    UpdateArgs A;
    A.part = (double *)workspace, A.part_first = 0, A.part_count = 0;
    A.clip_grads = !params, A.norm = nullptr, A.max_norm = max_norm, A.lr = params ? lr : 1.0;
    for (int i = 0; i < n;) {
        i = fill(A, tensors, i, n);
        if (!A.n) break;
        const u32 blocks = A.cum[A.n] < NORM_BLOCKS ? A.cum[A.n] : NORM_BLOCKS;
        k_norm<<<blocks, 256, 0, s>>>(A);
        A.part_first += (int)blocks;
    }
    A.part_count = A.part_first, A.norm = norm;
    bool done = false;
    for (int i = 0; i < n || !done;) {
        i = fill(A, tensors, i, n);
        const u32 chunks = A.cum[A.n];
        if (!A.n && done) break;
        k_update<<<chunks < 1 ? 1 : chunks < 2048 ? chunks : 2048, 256, 0, s>>>(A);
        A.norm = nullptr, done = true;
    }
    return ops_launched("ob_clip_step");
}

}  // extern "C"
