// grads.hip -- norms of a list of gradient tensors (sf_grad_norm) and their
// scaling to a largest norm (sf_grad_clip).
//
// A list may hold hundreds of tensors from one entry to billions.  It is cut
// into chunks of one size, none of which spans two tensors; a workgroup takes
// a chunk and finds its tensor among the first chunks of all.  Pointers,
// counts and types travel in the kernel's arguments, a batch of tensors a
// launch, so nothing is copied to the device first.

#include <algorithm>
#include <new>

#include "sf_device.h"
#include "sf_host.h"
#include "sf_train.h"

namespace sfk {

constexpr int kGradWG = 256;
constexpr int kNormBatch = 192;  // tensors per launch: 20 bytes each of 4 KB of arguments
constexpr int kClipBatch = 128;  // 28 bytes each
constexpr uint64_t kListMagic = 0x7366677261643031ull;
constexpr int64_t kGradMax = (int64_t)1 << 40;

struct GradItem {
    uintptr_t ptr;
    int64_t numel;
    int32_t dtype;
    int32_t pad;
    int64_t first;  // index of its first chunk in the list
};
struct GradSpan {
    uintptr_t lo, hi;
};
// The caller's host memory: this, then n items, then n address ranges in order.
struct GradList {
    uint64_t magic;
    int32_t n;
    int32_t overlaps;  // some two of its tensors overlap
    int64_t chunk;     // elements
    int64_t chunks;
    const GradItem* items() const { return reinterpret_cast<const GradItem*>(this + 1); }
    const GradSpan* spans() const { return reinterpret_cast<const GradSpan*>(items() + n); }
};

struct NormArgs {
    uintptr_t ptr[kNormBatch];
    int64_t numel[kNormBatch];  // count << 2 | type
    uint32_t first[kNormBatch + 1];
};
struct ClipArgs {
    uintptr_t ptr[kClipBatch];
    uintptr_t out[kClipBatch];
    int64_t numel[kClipBatch];
    uint32_t first[kClipBatch + 1];
};
struct Partial {
    double sum;
    int64_t wrong;
};

// Index of the tensor whose chunks hold chunk b: first[] ascends, and unused
// entries hold the batch's chunk count.
template <int BATCH>
__device__ __forceinline__ int find_item(const uint32_t* first, uint32_t b)
{
    const int lane = threadIdx.x & 63;
    int n = 0;
#pragma unroll
    for (int k = 0; k < BATCH; k += 64) n += __popcll(__ballot(first[k + lane] <= b));
    return __builtin_amdgcn_readfirstlane(n) - 1;
}

__device__ __forceinline__ bool not_finite(float x) { return (__float_as_uint(x) & 0x7F800000u) == 0x7F800000u; }

// Sum of squares of a chunk in 64 bits; a thread whose own sum is not finite
// (no finite input makes it so) reads its elements again and counts.
template <int DT>
__device__ __forceinline__ void chunk_norm(const typename Elem<DT>::T* p, int64_t n, double* sum, int64_t* wrong)
{
    constexpr int E = kVec<DT>;
    const int tid = threadIdx.x;
    const int64_t head = head_elems<DT>(p, n);
    const int64_t nv = (n - head) / E, tail0 = head + nv * E;
    const typename Elem<DT>::T* body = p + head;
    double s = 0.0;
    for (int64_t v = tid; v < nv; v += kGradWG) {
        const VecU<DT> x = *(const VecU<DT>*)(body + v * E);
#pragma unroll
        for (int j = 0; j < E; ++j) {
            const double y = (double)(float)x[j];
            s = fma(y, y, s);
        }
    }
    const int64_t j = tid < head ? tid : tail0 + (tid - head);
    const bool edge = tid < head + (n - tail0);
    if (edge) {
        const double y = (double)(float)p[j];
        s = fma(y, y, s);
    }
    int64_t w = 0;
    if (!(s < (double)INFINITY)) {
        for (int64_t v = tid; v < nv; v += kGradWG) {
            const VecU<DT> x = *(const VecU<DT>*)(body + v * E);
            for (int i = 0; i < E; ++i) w += not_finite((float)x[i]);
        }
        if (edge) w += not_finite((float)p[j]);
    }
    *sum = s;
    *wrong = w;
}

__global__ __launch_bounds__(kGradWG) void k_grad_norm(NormArgs a, int n, int64_t chunk, int64_t base,
                                                       int64_t item0, Partial* __restrict__ partial,
                                                       uint32_t* __restrict__ table, uint32_t* __restrict__ done)
{
    __shared__ double sums[kGradWG / 64];
    __shared__ int64_t wrongs[kGradWG / 64];
    const int tid = threadIdx.x;
    const uint32_t b = blockIdx.x;
    if (b == 0) {
        // where each tensor's chunks begin, and the join's counter
        for (int i = tid; i <= n; i += kGradWG) table[item0 + i] = (uint32_t)(base + a.first[i]);
        if (item0 == 0 && tid == 0) *done = 0;
    }
    if (b >= a.first[n]) return;
    const int i = find_item<kNormBatch>(a.first, b);
    const int64_t count = a.numel[i] >> 2;
    const int dtype = (int)(a.numel[i] & 3);
    const int64_t e0 = (int64_t)(b - a.first[i]) * chunk;
    const int64_t len = count - e0 < chunk ? count - e0 : chunk;
    double s;
    int64_t w;
    if (dtype == SF_F32)
        chunk_norm<SF_F32>((const float*)a.ptr[i] + e0, len, &s, &w);
    else if (dtype == SF_BF16)
        chunk_norm<SF_BF16>((const __bf16*)a.ptr[i] + e0, len, &s, &w);
    else
        chunk_norm<SF_F16>((const _Float16*)a.ptr[i] + e0, len, &s, &w);
    s = wave_sum_f64(s);
    w = wave_sum64(w);
    if ((tid & 63) == 0) {
        sums[tid >> 6] = s;
        wrongs[tid >> 6] = w;
    }
    __syncthreads();
    if (tid == 0) {
        for (int k = 1; k < kGradWG / 64; ++k) {
            s += sums[k];
            w += wrongs[k];
        }
        partial[base + b] = {s, w};
    }
}

// One wave per tensor adds its chunks' sums in order; the workgroup that
// finishes last adds the tensors'.
__global__ __launch_bounds__(kGradWG) void k_grad_norm_join(int64_t n, const Partial* __restrict__ partial,
                                                            const uint32_t* __restrict__ table, double* squares,
                                                            uint32_t* done, float* __restrict__ norms,
                                                            float* __restrict__ total,
                                                            int64_t* __restrict__ nonfinite)
{
    __shared__ double sums[kGradWG / 64];
    __shared__ bool last;
    const int tid = threadIdx.x, lane = tid & 63;
    const int64_t i = (int64_t)blockIdx.x * (kGradWG / 64) + (tid >> 6);
    if (i < n) {
        double s = 0.0;
        int64_t w = 0;
        for (uint32_t k = table[i] + lane; k < table[i + 1]; k += 64) {
            s += partial[k].sum;
            w += partial[k].wrong;
        }
        s = wave_sum_f64(s);
        w = wave_sum64(w);
        if (lane == 0) {
            norms[i] = (float)sqrt(s);
            nonfinite[i] = w;
            squares[i] = s;
        }
    }
    __threadfence();
    __syncthreads();
    if (tid == 0) last = atomicAdd(done, 1u) == gridDim.x - 1;
    __syncthreads();
    if (!last) return;
    __threadfence();
    double s = 0.0;
    for (int64_t k = tid; k < n; k += kGradWG) s += squares[k];
    s = wave_sum_f64(s);
    if (lane == 0) sums[tid >> 6] = s;
    __syncthreads();
    if (tid == 0) {
        for (int k = 1; k < kGradWG / 64; ++k) s += sums[k];
        *total = (float)sqrt(s);
    }
}

__global__ void k_grad_norm_empty(float* total) { *total = 0.0f; }

template <int DT>
__device__ __forceinline__ void chunk_scale(const typename Elem<DT>::T* p, typename Elem<DT>::T* o, int64_t n,
                                            float c)
{
    typedef typename Elem<DT>::T T;
    constexpr int E = kVec<DT>;
    const int tid = threadIdx.x;
    const int64_t head = head_elems<DT>(o, n);
    const int64_t nv = (n - head) / E, tail0 = head + nv * E;
    for (int64_t v = tid; v < nv; v += kGradWG) {
        VecU<DT> x = *(const VecU<DT>*)(p + head + v * E);
#pragma unroll
        for (int j = 0; j < E; ++j) x[j] = (T)((float)x[j] * c);
        *(VecU<DT>*)(o + head + v * E) = x;
    }
    if (tid < head + (n - tail0)) {
        const int64_t j = tid < head ? tid : tail0 + (tid - head);
        o[j] = (T)((float)p[j] * c);
    }
}

__global__ __launch_bounds__(kGradWG) void k_grad_clip(ClipArgs a, int n, int64_t chunk, int in_place,
                                                       const float* __restrict__ norms, int64_t m, float max_norm,
                                                       float eps, uint32_t* status)
{
    __shared__ double sums[kGradWG / 64];
    const int tid = threadIdx.x;
    const uint32_t b = blockIdx.x;
    // the norm of all parts, every workgroup for itself
    double s = 0.0;
    for (int64_t k = tid; k < m; k += kGradWG) s = fma((double)norms[k], (double)norms[k], s);
    s = wave_sum_f64(s);
    if ((tid & 63) == 0) sums[tid >> 6] = s;
    __syncthreads();
    s = 0.0;
    for (int k = 0; k < kGradWG / 64; ++k) s += sums[k];
    const bool wrong = !(s < (double)INFINITY);
    const double c = (double)max_norm / (sqrt(s) + (double)eps);
    const float coef = wrong || !(c < 1.0) ? 1.0f : (float)c;
    if (wrong && status && b == 0 && tid == 0) atomicOr(status, (uint32_t)SF_ERANGE);
    if (coef == 1.0f && in_place) return;
    if (b >= a.first[n]) return;
    const int i = find_item<kClipBatch>(a.first, b);
    const int64_t count = a.numel[i] >> 2;
    const int dtype = (int)(a.numel[i] & 3);
    const int64_t e0 = (int64_t)(b - a.first[i]) * chunk;
    const int64_t len = count - e0 < chunk ? count - e0 : chunk;
    if (dtype == SF_F32)
        chunk_scale<SF_F32>((const float*)a.ptr[i] + e0, (float*)a.out[i] + e0, len, coef);
    else if (dtype == SF_BF16)
        chunk_scale<SF_BF16>((const __bf16*)a.ptr[i] + e0, (__bf16*)a.out[i] + e0, len, coef);
    else
        chunk_scale<SF_F16>((const _Float16*)a.ptr[i] + e0, (_Float16*)a.out[i] + e0, len, coef);
}

static inline const GradList* as_list(const void* p)
{
    const GradList* l = static_cast<const GradList*>(p);
    return l && aligned(l, 8) && l->magic == kListMagic ? l : nullptr;
}

// true if [p, p + bytes) meets none of the list's tensors
static bool clear_of(const GradList* l, const void* p, int64_t bytes)
{
    for (int32_t i = 0; i < l->n; ++i)
        if (l->spans()[i].hi > l->spans()[i].lo &&
            !disjoint(p, bytes, (const void*)l->spans()[i].lo, (int64_t)(l->spans()[i].hi - l->spans()[i].lo)))
            return false;
    return true;
}

struct NormLayout {
    int64_t squares, table, done, bytes;  // offsets; the chunks' sums come first
};

static NormLayout norm_layout(const GradList* l)
{
    NormLayout w;
    w.squares = l->chunks * (int64_t)sizeof(Partial);
    w.table = w.squares + (int64_t)l->n * 8;
    w.done = w.table + ((int64_t)l->n + 1) * 4;
    w.bytes = (w.done + 4 + 15) & ~(int64_t)15;
    return w;
}

}  // namespace sfk

using namespace sfk;

SF_API int64_t sf_grad_list_bytes(int32_t n)
{
    if (n < 0 || n > (1 << 20)) return -1;
    return (int64_t)sizeof(GradList) + (int64_t)n * (int64_t)(sizeof(GradItem) + sizeof(GradSpan));
}

SF_API int sf_grad_list_init(void* list, int64_t list_bytes, const void* const* grads, const int64_t* numel,
                             const int32_t* dtype, int32_t n)
{
    const int64_t need = sf_grad_list_bytes(n);
    if (!list || !aligned(list, 8) || need < 0 || list_bytes < need || (n > 0 && (!grads || !numel || !dtype)))
        return SF_EINVAL;
    int64_t total = 0;
    for (int32_t i = 0; i < n; ++i) {
        if (dtype[i] < SF_F32 || dtype[i] > SF_F16 || numel[i] < 0 || numel[i] >= kGradMax) return SF_EINVAL;
        if (numel[i] > 0 && (!grads[i] || !aligned(grads[i], elem_size(dtype[i])))) return SF_EINVAL;
        total += numel[i];
    }
    // Chunks of 2 K to 1 M elements, about 4096 of them: enough to fill the
    // chip, and few enough that their sums cost little to add up.
    int64_t chunk = 2048;
    while (chunk < (1 << 20) && chunk * 4096 < total) chunk *= 2;
    int64_t chunks = 0;
    for (int32_t i = 0; i < n; ++i) chunks += (numel[i] + chunk - 1) / chunk;
    if (chunks > INT32_MAX) return SF_EINVAL;
    GradList* l = new (list) GradList;
    l->magic = 0;
    l->n = n;
    l->chunk = chunk;
    l->chunks = chunks;
    GradItem* items = reinterpret_cast<GradItem*>(l + 1);
    GradSpan* spans = reinterpret_cast<GradSpan*>(items + n);
    int64_t at = 0;
    for (int32_t i = 0; i < n; ++i) {
        items[i] = {(uintptr_t)grads[i], numel[i], dtype[i], 0, at};
        spans[i] = {(uintptr_t)grads[i], (uintptr_t)grads[i] + (uintptr_t)(numel[i] * elem_size(dtype[i]))};
        at += (numel[i] + chunk - 1) / chunk;
    }
    std::sort(spans, spans + n, [](const GradSpan& x, const GradSpan& y) { return x.lo != y.lo ? x.lo < y.lo : x.hi < y.hi; });
    l->overlaps = 0;
    uintptr_t end = 0;
    for (int32_t i = 0; i < n; ++i) {
        if (spans[i].hi == spans[i].lo) continue;
        if (spans[i].lo < end) l->overlaps = 1;
        end = spans[i].hi > end ? spans[i].hi : end;
    }
    l->magic = kListMagic;
    return SF_OK;
}

SF_API int64_t sf_grad_norm_workspace(const void* list)
{
    const GradList* l = as_list(list);
    return l ? norm_layout(l).bytes : -1;
}

SF_API int sf_grad_norm(const void* list, float* out_norms, float* out_total, int64_t* out_nonfinite,
                        void* workspace, int64_t workspace_bytes, sf_stream_t stream)
{
    const GradList* l = as_list(list);
    if (!l || !out_total || !aligned(out_total, 4)) return SF_EINVAL;
    const NormLayout w = norm_layout(l);
    const int64_t n = l->n;
    if (n > 0 && (!out_norms || !out_nonfinite || !workspace || workspace_bytes < w.bytes)) return SF_EINVAL;
    if (!aligned(out_norms, 4) || !aligned(out_nonfinite, 8) || !aligned(workspace, 16)) return SF_EINVAL;
    if (n == 0) {
        void* args[] = {(void*)&out_total};
        return launch((const void*)&k_grad_norm_empty, dim3(1), dim3(1), args, 0, stream);
    }
    const void* outs[4] = {out_norms, out_total, out_nonfinite, workspace};
    const int64_t sizes[4] = {n * 4, 4, n * 8, w.bytes};
    for (int x = 0; x < 4; ++x) {
        if (!clear_of(l, outs[x], sizes[x])) return SF_EINVAL;
        for (int y = x + 1; y < 4; ++y)
            if (!disjoint(outs[x], sizes[x], outs[y], sizes[y])) return SF_EINVAL;
    }
    Partial* partial = (Partial*)workspace;
    double* squares = (double*)((char*)workspace + w.squares);
    uint32_t* table = (uint32_t*)((char*)workspace + w.table);
    uint32_t* done = (uint32_t*)((char*)workspace + w.done);
    int64_t chunk = l->chunk;
    const GradItem* items = l->items();
    for (int64_t i0 = 0; i0 < n; i0 += kNormBatch) {
        NormArgs a;
        int m = (int)(n - i0 < kNormBatch ? n - i0 : kNormBatch);
        int64_t base = items[i0].first;
        const int64_t stop = i0 + m < n ? items[i0 + m].first : l->chunks;
        for (int k = 0; k < kNormBatch; ++k) {
            a.ptr[k] = k < m ? items[i0 + k].ptr : 0;
            a.numel[k] = k < m ? items[i0 + k].numel << 2 | items[i0 + k].dtype : 0;
            a.first[k] = (uint32_t)((k < m ? items[i0 + k].first : stop) - base);
        }
        a.first[kNormBatch] = (uint32_t)(stop - base);
        const unsigned grid = stop > base ? (unsigned)(stop - base) : 1;
        void* args[] = {(void*)&a,  (void*)&m,       (void*)&chunk, (void*)&base,
                        (void*)&i0, (void*)&partial, (void*)&table, (void*)&done};
        const int rc = launch((const void*)&k_grad_norm, dim3(grid), dim3(kGradWG), args, 0, stream);
        if (rc != SF_OK) return rc;
    }
    int64_t nn = n;
    void* args[] = {(void*)&nn,   (void*)&partial,   (void*)&table,     (void*)&squares,
                    (void*)&done, (void*)&out_norms, (void*)&out_total, (void*)&out_nonfinite};
    return launch((const void*)&k_grad_norm_join, dim3((unsigned)((n + kGradWG / 64 - 1) / (kGradWG / 64))),
                  dim3(kGradWG), args, 0, stream);
}

SF_API int sf_grad_clip(const void* list, const void* out_list, const float* norms, int64_t m, float max_norm,
                        float eps, uint32_t* status, sf_stream_t stream)
{
    const GradList* l = as_list(list);
    const GradList* o = as_list(out_list);
    if (!l || !o || l->n != o->n || !norms || !aligned(norms, 4) || !aligned(status, 4)) return SF_EINVAL;
    if (m < 1 || m > SF_MAX_R || !(max_norm > 0.0f && max_norm <= kF32Max) || !(eps >= 0.0f && eps <= kF32Max))
        return SF_EINVAL;
    if (o->overlaps || !clear_of(o, norms, m * 4) || (status && (!clear_of(o, status, 4) || !clear_of(l, status, 4))))
        return SF_EINVAL;
    if (status && !disjoint(status, 4, norms, m * 4)) return SF_EINVAL;
    const int64_t n = l->n;
    const GradItem* in = l->items();
    const GradItem* out = o->items();
    int same = 1;
    for (int64_t i = 0; i < n; ++i) {
        if (in[i].numel != out[i].numel || in[i].dtype != out[i].dtype) return SF_EINVAL;
        if (in[i].ptr != out[i].ptr && in[i].numel > 0) same = 0;
    }
    if (!same) {
        // an output may meet a gradient only where it is that gradient itself
        for (int64_t i = 0; i < n; ++i) {
            if (out[i].numel == 0) continue;
            const uintptr_t lo = out[i].ptr, hi = lo + (uintptr_t)(out[i].numel * elem_size(out[i].dtype));
            const GradSpan* sp = l->spans();
            // the last gradient that begins before hi; with no overlaps among
            // the gradients it is the only one that can reach past lo
            const GradSpan* q = std::lower_bound(sp, sp + n, hi, [](const GradSpan& x, uintptr_t v) { return x.lo < v; });
            int met = 0;
            for (; q != sp; --q) {
                const GradSpan& g = q[-1];
                if (g.hi > lo && g.hi > g.lo) {
                    if (in[i].ptr != lo || g.lo != lo || g.hi != hi || ++met > 1) return SF_EINVAL;
                }
                if (!l->overlaps && g.hi > g.lo) break;
            }
        }
    }
    int64_t chunk = l->chunk;
    for (int64_t i0 = 0; i0 < n; i0 += kClipBatch) {
        ClipArgs a;
        int k1 = (int)(n - i0 < kClipBatch ? n - i0 : kClipBatch);
        const int64_t base = in[i0].first;
        const int64_t stop = i0 + k1 < n ? in[i0 + k1].first : l->chunks;
        for (int k = 0; k < kClipBatch; ++k) {
            a.ptr[k] = k < k1 ? in[i0 + k].ptr : 0;
            a.out[k] = k < k1 ? out[i0 + k].ptr : 0;
            a.numel[k] = k < k1 ? in[i0 + k].numel << 2 | in[i0 + k].dtype : 0;
            a.first[k] = (uint32_t)((k < k1 ? in[i0 + k].first : stop) - base);
        }
        a.first[kClipBatch] = (uint32_t)(stop - base);
        const unsigned grid = stop > base ? (unsigned)(stop - base) : 1;
        void* args[] = {(void*)&a,     (void*)&k1, (void*)&chunk,    (void*)&same, (void*)&norms,
                        (void*)&m,     (void*)&max_norm, (void*)&eps, (void*)&status};
        const int rc = launch((const void*)&k_grad_clip, dim3(grid), dim3(kGradWG), args, 0, stream);
        if (rc != SF_OK) return rc;
    }
    return SF_OK;
}
