// grads.hip -- norms of a list of gradient tensors (sf_grad_norm) and their
// scaling to a largest norm (sf_grad_clip).
//
// A list may hold hundreds of tensors from one entry to billions.  It is cut
// into chunks of one size, none of which spans two tensors; a workgroup takes
// a chunk and finds its tensor among the first chunks of all.  Pointers,
// counts and types travel in the kernel's arguments, a batch of tensors a
// launch, so nothing is copied to the device first.
//
// Both are bound by HBM where they are large.  Norm: 1.34e9 bf16 entries in 193
// tensors 398 us, 6.7 TB/s (the plain read reaches 7.13); squares are taken in 64
// bits, a conversion and a multiply-add an entry, a quarter of the VALU's time.
// Clip: 4.7e8 f32 entries 631 us, 6.0 TB/s read and written.  Loads and stores go
// past the caches (clip: 712 us with cached stores, 706 with cached loads, 692
// with neither, at chunks of 64 K entries), in chunks of 8 K entries for the clip
// (16 K: 682, 8 K: 637, 4 K: 635 us) and of up to 64 K for the norm, whose sums
// have to be added up (32 K to 128 K: the same within 1%).

#include <algorithm>
#include <new>

#include "sf_device.h"
#include "sf_host.h"
#include "sf_train.h"

namespace sfk {

constexpr int kGradWG = 256;
// Tensors per launch: 20 bytes each of 4 KB of arguments.  Batches of a list hold
// equal numbers (193 tensors as 192 + 1 left the last one alone on the chip: 126
// us for 1.7e7 entries).
constexpr int kNormBatch = 192;
constexpr int kClipBatch = 128;  // 28 bytes each
constexpr uint64_t kListMagic = 0x7366677261643031ull;
constexpr int64_t kGradMax = (int64_t)1 << 40;
// Entries of a chunk: the norm's from 4 K up to 64 K, about 4096 chunks where
// that is enough; the clip's.
constexpr int64_t kChunkMax = 1 << 16, kChunkWant = 4096;
constexpr int64_t kChunkMost = 1 << 23;  // and n more, of 256 threads each
constexpr int64_t kClipChunk = 8192;

struct GradItem {
    uintptr_t ptr;
    int64_t numel;
    int64_t dtype;
    int64_t first, clip_first;  // index of its first chunk in the list, for the norm and the clip
};
struct GradSpan {
    uintptr_t lo, hi;
};
// The caller's host memory: this, then n items, then n address ranges in order.
struct GradList {
    uint64_t magic;
    int32_t n;
    int32_t overlaps;  // some two of its tensors overlap
    int64_t chunk;     // elements, for the norm
    int64_t chunks;
    int64_t most;      // chunks of a tensor, at most
    int64_t clip_chunks;
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
constexpr int kNormU = 4;  // vectors per lane in flight

template <int DT>
__device__ __forceinline__ void chunk_norm(uintptr_t at, int n, double* sum, int64_t* wrong)
{
    constexpr int E = kVec<DT>;
    constexpr int U = kNormU;
    const int tid = threadIdx.x;
    const GlobalElem<DT>* p = (const GlobalElem<DT>*)at;
    const int head = (int)head_elems<DT, 128>((const void*)at, n);
    const int nv = (n - head) / E, tail0 = head + nv * E;
    const GlobalVec<DT>* body = (const GlobalVec<DT>*)(p + head);
    double s = 0.0;
    auto add = [&](const VecU<DT>& x) {
#pragma unroll
        for (int j = 0; j < E; ++j) {
            const double y = (double)(float)x[j];
            s = fma(y, y, s);
        }
    };
    int v = tid;
    for (; v + (U - 1) * kGradWG < nv; v += U * kGradWG) {
        VecU<DT> x[U];
#pragma unroll
        for (int k = 0; k < U; ++k) x[k] = __builtin_nontemporal_load(body + v + k * kGradWG);
#pragma unroll
        for (int k = 0; k < U; ++k) add(x[k]);
    }
    for (; v < nv; v += kGradWG) add(__builtin_nontemporal_load(body + v));
    const bool edge = tid < head + (n - tail0);
    const int j = tid < head ? tid : tail0 + (tid - head);
    if (edge) {
        const double y = (double)(float)p[j];
        s = fma(y, y, s);
    }
    int64_t w = 0;
    if (!(s < (double)INFINITY)) {
        for (v = tid; v < nv; v += kGradWG) {
            const VecU<DT> x = body[v];
            for (int i = 0; i < E; ++i) w += not_finite((float)x[i]);
        }
        if (edge) w += not_finite((float)p[j]);
    }
    *sum = s;
    *wrong = w;
}

__global__ __launch_bounds__(kGradWG) void k_grad_norm(NormArgs a, int n, int64_t chunk, int64_t base,
                                                       int64_t item0, Partial* __restrict__ partial,
                                                       uint32_t* __restrict__ table)
{
    __shared__ double sums[kGradWG / 64];
    __shared__ int64_t wrongs[kGradWG / 64];
    const int tid = threadIdx.x;
    const uint32_t b = blockIdx.x;
    if (b == 0) {
        // where each tensor's chunks begin, for the join
        for (int i = tid; i <= n; i += kGradWG) table[item0 + i] = (uint32_t)(base + a.first[i]);
    }
    if (b >= a.first[n]) return;
    const int i = find_item<kNormBatch>(a.first, b);
    const int64_t count = a.numel[i] >> 2;
    const int dtype = (int)(a.numel[i] & 3);
    const int64_t e0 = (int64_t)(b - a.first[i]) * chunk;
    const int len = (int)(count - e0 < chunk ? count - e0 : chunk);
    double s;
    int64_t w;
    if (dtype == SF_F32)
        chunk_norm<SF_F32>(a.ptr[i] + e0 * 4, len, &s, &w);
    else if (dtype == SF_BF16)
        chunk_norm<SF_BF16>(a.ptr[i] + e0 * 2, len, &s, &w);
    else
        chunk_norm<SF_F16>(a.ptr[i] + e0 * 2, len, &s, &w);
    s = wave_sum_f64(s);
    w = wave_sum_i64(w);
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

// Joins, in a fixed order, by launches of their own: with a counter of finished
// workgroups the memory fence of each writes back an L2, and the join of 33
// tensors took 4.8 us instead of 3.0.  Few tensors of few chunks: one workgroup
// for all, 16 lanes a tensor.
constexpr int kJoinWG = 1024;
constexpr int kJoinLanes = 16;
constexpr int kJoinItems = kJoinWG;  // at most
constexpr int kJoinChunks = 16 * kJoinLanes;  // of a tensor, at most

__global__ __launch_bounds__(kJoinWG) void k_grad_norm_join(int n, const Partial* __restrict__ partial,
                                                            const uint32_t* __restrict__ table,
                                                            float* __restrict__ norms, float* __restrict__ total,
                                                            int64_t* __restrict__ nonfinite)
{
    __shared__ double squares[kJoinItems];
    __shared__ double sums[kJoinWG / 64];
    const int tid = threadIdx.x, lane = tid & (kJoinLanes - 1);
    for (int i = tid / kJoinLanes; i < n; i += kJoinWG / kJoinLanes) {
        double s = 0.0;
        int64_t w = 0;
        const uint32_t end = table[i + 1];
        for (uint32_t k = table[i] + lane; k < end; k += kJoinLanes) {
            s += partial[k].sum;
            w += partial[k].wrong;
        }
        for (int off = kJoinLanes / 2; off > 0; off >>= 1) {
            s += __shfl_xor(s, off, kJoinLanes);
            w += __shfl_xor(w, off, kJoinLanes);
        }
        if (lane == 0) {
            norms[i] = (float)sqrt(s);
            nonfinite[i] = w;
            squares[i] = s;
        }
    }
    __syncthreads();
    double s = tid < n ? squares[tid] : 0.0;
    s = wave_sum_f64(s);
    if ((tid & 63) == 0) sums[tid >> 6] = s;
    __syncthreads();
    if (tid == 0) {
        for (int k = 1; k < kJoinWG / 64; ++k) s += sums[k];
        *total = (float)sqrt(s);
    }
}

// Else a workgroup per tensor, and one for all of them.
__global__ __launch_bounds__(kGradWG) void k_grad_norm_item(const Partial* __restrict__ partial,
                                                            const uint32_t* __restrict__ table,
                                                            double* __restrict__ squares, float* __restrict__ norms,
                                                            int64_t* __restrict__ nonfinite)
{
    __shared__ double sums[kGradWG / 64];
    __shared__ int64_t wrongs[kGradWG / 64];
    const int tid = threadIdx.x, i = blockIdx.x;
    double s = 0.0;
    int64_t w = 0;
    const uint32_t end = table[i + 1];
    for (uint32_t k = table[i] + tid; k < end; k += kGradWG) {
        s += partial[k].sum;
        w += partial[k].wrong;
    }
    s = wave_sum_f64(s);
    w = wave_sum_i64(w);
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
        norms[i] = (float)sqrt(s);
        nonfinite[i] = w;
        squares[i] = s;
    }
}

__global__ __launch_bounds__(kJoinWG) void k_grad_norm_total(int n, const double* __restrict__ squares,
                                                             float* __restrict__ total)
{
    __shared__ double sums[kJoinWG / 64];
    const int tid = threadIdx.x;
    double s = 0.0;
    for (int k = tid; k < n; k += kJoinWG) s += squares[k];
    s = wave_sum_f64(s);
    if ((tid & 63) == 0) sums[tid >> 6] = s;
    __syncthreads();
    if (tid == 0) {
        for (int k = 1; k < kJoinWG / 64; ++k) s += sums[k];
        *total = (float)sqrt(s);
    }
}

__global__ void k_grad_norm_empty(float* total) { *total = 0.0f; }

constexpr int kClipU = 4;
template <int DT>
__device__ __forceinline__ void chunk_scale(uintptr_t from, uintptr_t to, int n, float c)
{
    typedef typename Elem<DT>::T T;
    constexpr int E = kVec<DT>;
    constexpr int U = kClipU;
    const int tid = threadIdx.x;
    const GlobalElem<DT>* p = (const GlobalElem<DT>*)from;
    GlobalElem<DT>* o = (GlobalElem<DT>*)to;
    const int head = (int)head_elems<DT, 128>((const void*)to, n);
    const int nv = (n - head) / E, tail0 = head + nv * E;
    const GlobalVec<DT>* pv = (const GlobalVec<DT>*)(p + head);
    GlobalVec<DT>* ov = (GlobalVec<DT>*)(o + head);
    auto scale = [&](VecU<DT> x) {
#pragma unroll
        for (int j = 0; j < E; ++j) x[j] = (T)((float)x[j] * c);
        return x;
    };
    int v = tid;
    for (; v + (U - 1) * kGradWG < nv; v += U * kGradWG) {
        VecU<DT> x[U];
#pragma unroll
        for (int k = 0; k < U; ++k) x[k] = __builtin_nontemporal_load(pv + v + k * kGradWG);
#pragma unroll
        for (int k = 0; k < U; ++k) __builtin_nontemporal_store(scale(x[k]), ov + v + k * kGradWG);
    }
    for (; v < nv; v += kGradWG) ov[v] = scale(pv[v]);
    if (tid < head + (n - tail0)) {
        const int j = tid < head ? tid : tail0 + (tid - head);
        o[j] = (T)((float)p[j] * c);
    }
}

__global__ __launch_bounds__(kGradWG) void k_grad_clip(ClipArgs a, int n, int in_place,
                                                       const float* __restrict__ norms, int64_t m, float max_norm,
                                                       float eps, uint32_t* status)
{
    __shared__ double sums[kGradWG / 64];
    const int tid = threadIdx.x;
    // the norm of all parts, every workgroup for itself
    double s = 0.0;
    if (m == 1) {
        s = fabs((double)norms[0]);
    } else {
        for (int64_t k = tid; k < m; k += kGradWG) s = fma((double)norms[k], (double)norms[k], s);
        s = wave_sum_f64(s);
        if ((tid & 63) == 0) sums[tid >> 6] = s;
        __syncthreads();
        s = 0.0;
        for (int k = 0; k < kGradWG / 64; ++k) s += sums[k];
        s = sqrt(s);
    }
    const bool wrong = !(s < (double)INFINITY);
    const double c = (double)max_norm / (s + (double)eps);
    const float coef = wrong || !(c < 1.0) ? 1.0f : (float)c;
    if (wrong && status && blockIdx.x == 0 && tid == 0) atomicOr(status, (uint32_t)SF_ERANGE);
    if (coef == 1.0f && in_place) return;
    for (uint32_t b = blockIdx.x; b < a.first[n]; b += gridDim.x) {
        const int i = find_item<kClipBatch>(a.first, b);
        const int64_t count = a.numel[i] >> 2;
        const int dtype = (int)(a.numel[i] & 3);
        const int64_t e0 = (int64_t)(b - a.first[i]) * kClipChunk;
        const int len = (int)(count - e0 < kClipChunk ? count - e0 : kClipChunk);
        if (dtype == SF_F32)
            chunk_scale<SF_F32>(a.ptr[i] + e0 * 4, a.out[i] + e0 * 4, len, coef);
        else if (dtype == SF_BF16)
            chunk_scale<SF_BF16>(a.ptr[i] + e0 * 2, a.out[i] + e0 * 2, len, coef);
        else
            chunk_scale<SF_F16>(a.ptr[i] + e0 * 2, a.out[i] + e0 * 2, len, coef);
    }
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
    int64_t squares, table, bytes;  // offsets; the chunks' sums come first
};

static NormLayout norm_layout(const GradList* l)
{
    NormLayout w;
    w.squares = l->chunks * (int64_t)sizeof(Partial);
    w.table = w.squares + (int64_t)l->n * 8;
    w.bytes = (w.table + ((int64_t)l->n + 1) * 4 + 15) & ~(int64_t)15;
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
    if (total >= kGradMax) return SF_EINVAL;
    // (past 2^39 entries longer ones: a launch has fewer than 2^32 threads)
    int64_t chunk = 4096;
    while ((chunk < kChunkMax && chunk * kChunkWant < total) || total / chunk >= kChunkMost) chunk *= 2;
    int64_t chunks = 0, most = 0;
    for (int32_t i = 0; i < n; ++i) {
        const int64_t c = (numel[i] + chunk - 1) / chunk;
        chunks += c;
        most = c > most ? c : most;
    }
    GradList* l = new (list) GradList;
    l->magic = 0;
    l->n = n;
    l->chunk = chunk;
    l->chunks = chunks;
    l->most = most;
    GradItem* items = reinterpret_cast<GradItem*>(l + 1);
    GradSpan* spans = reinterpret_cast<GradSpan*>(items + n);
    int64_t at = 0, clip_at = 0;
    for (int32_t i = 0; i < n; ++i) {
        items[i] = {(uintptr_t)grads[i], numel[i], dtype[i], at, clip_at};
        spans[i] = {(uintptr_t)grads[i], (uintptr_t)grads[i] + (uintptr_t)(numel[i] * elem_size(dtype[i]))};
        at += (numel[i] + chunk - 1) / chunk;
        clip_at += (numel[i] + kClipChunk - 1) / kClipChunk;
    }
    if (clip_at > INT32_MAX) return SF_EINVAL;
    l->clip_chunks = clip_at;
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
    int64_t chunk = l->chunk;
    const GradItem* items = l->items();
    const int64_t batches = (n + kNormBatch - 1) / kNormBatch, each = (n + batches - 1) / batches;
    for (int64_t i0 = 0; i0 < n; i0 += each) {
        NormArgs a;
        int m = (int)(n - i0 < each ? n - i0 : each);
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
                        (void*)&i0, (void*)&partial, (void*)&table};
        const int rc = launch((const void*)&k_grad_norm, dim3(grid), dim3(kGradWG), args, 0, stream);
        if (rc != SF_OK) return rc;
    }
    int nn = l->n;
    if (nn <= kJoinItems && l->most <= kJoinChunks) {
        void* args[] = {(void*)&nn,        (void*)&partial,   (void*)&table,
                        (void*)&out_norms, (void*)&out_total, (void*)&out_nonfinite};
        return launch((const void*)&k_grad_norm_join, dim3(1), dim3(kJoinWG), args, 0, stream);
    }
    void* args[] = {(void*)&partial, (void*)&table, (void*)&squares, (void*)&out_norms, (void*)&out_nonfinite};
    const int rc = launch((const void*)&k_grad_norm_item, dim3((unsigned)n), dim3(kGradWG), args, 0, stream);
    if (rc != SF_OK) return rc;
    void* targs[] = {(void*)&nn, (void*)&squares, (void*)&out_total};
    return launch((const void*)&k_grad_norm_total, dim3(1), dim3(kJoinWG), targs, 0, stream);
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
    const int64_t batches = (n + kClipBatch - 1) / kClipBatch, each = n > 0 ? (n + batches - 1) / batches : 1;
    for (int64_t i0 = 0; i0 < n; i0 += each) {
        ClipArgs a;
        int k1 = (int)(n - i0 < each ? n - i0 : each);
        const int64_t base = in[i0].clip_first;
        const int64_t stop = i0 + k1 < n ? in[i0 + k1].clip_first : l->clip_chunks;
        for (int k = 0; k < kClipBatch; ++k) {
            a.ptr[k] = k < k1 ? in[i0 + k].ptr : 0;
            a.out[k] = k < k1 ? out[i0 + k].ptr : 0;
            a.numel[k] = k < k1 ? in[i0 + k].numel << 2 | in[i0 + k].dtype : 0;
            a.first[k] = (uint32_t)((k < k1 ? in[i0 + k].clip_first : stop) - base);
        }
        a.first[kClipBatch] = (uint32_t)(stop - base);
        // a workgroup a chunk, but fewer than 2^32 threads
        const int64_t want = stop - base < 1 ? 1 : stop - base;
        const unsigned grid = (unsigned)(want < (1 << 23) ? want : (1 << 23));
        void* args[] = {(void*)&a,     (void*)&k1, (void*)&same, (void*)&norms,
                        (void*)&m,     (void*)&max_norm, (void*)&eps, (void*)&status};
        const int rc = launch((const void*)&k_grad_clip, dim3(grid), dim3(kGradWG), args, 0, stream);
        if (rc != SF_OK) return rc;
    }
    return SF_OK;
}
