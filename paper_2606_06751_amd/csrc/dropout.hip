// dropout.hip -- uniform numbers by counter (sf_uniform), and dropout with a mask
// that is made where it is used and never stored (sf_dropout).

#include "sf_draw.h"
#include "sf_host.h"

namespace sfk {

constexpr int kDrawWG = 256;
constexpr int64_t kLastCache = 256 << 20;  // bytes that the chip's last cache holds

// One block of four numbers a lane and turn.  Bound by the writes and, close behind,
// the generator's 60 instructions a block: 20480007 numbers 14.8 us, 5.5 TB/s; without
// its rounds 13 us.
__global__ __launch_bounds__(kDrawWG) void k_uniform(const int64_t* __restrict__ key, uint32_t site, int64_t first,
                                                     int64_t n, float* __restrict__ out)
{
    typedef float F4 __attribute__((ext_vector_type(4), aligned(4)));
    const int64_t b0 = first >> 2, b1 = (first + n + 3) >> 2;
    for (int64_t b = b0 + (int64_t)blockIdx.x * kDrawWG + threadIdx.x; b < b1; b += (int64_t)gridDim.x * kDrawWG) {
        const Words r = draw_words(key, b, 1, site);
        const int64_t at = b * 4 - first;
        F4 v;
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = (float)(r.w[j] >> 8) * 0x1p-24f;
        if (at >= 0 && at + 4 <= n) {
            *(F4*)(out + at) = v;
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (at + j >= 0 && at + j < n) out[at + j] = v[j];
        }
    }
}

struct DropShape {
    int64_t N, C, x_stride, residual_stride, out_stride, first, index_stride;
    uint32_t site, threshold;
    float scale;
    int lanes;  // a row's, a power of two up to kDrawWG
};

template <int DT>
using Eight = typename Elem<DT>::T __attribute__((ext_vector_type(8), aligned(sizeof(typename Elem<DT>::T))));

template <bool FAR, class V>
__device__ __forceinline__ V load_eight(const V* p)
{
    if (FAR) return __builtin_nontemporal_load(p);
    return *p;
}

// A lane takes the eight entries of one block of the generator, whose place in
// the row depends on the row's first index, so that equal indexes keep equal
// entries at any alignment.  Bound by HBM: 16384 x 8192 bf16 onto a residual 130 us,
// 6.2 TB/s read + write, the same without the generator (16 bits an entry: a block
// of 10 rounds for eight).  Loads go past the caches where the call moves more than
// the last of them holds (130 against 135 us; stores, too: 134), else not (4099 x 2048
// f32 to bf16, 50 MB: 9.6 against 11.8 us).
template <int XT, int OT, bool FAR>
__global__ __launch_bounds__(kDrawWG) void k_dropout(const typename Elem<XT>::T* x, const int64_t* __restrict__ key,
                                                     const typename Elem<OT>::T* residual, typename Elem<OT>::T* out,
                                                     DropShape p)
{
    typedef typename Elem<OT>::T O;
    const int rows = kDrawWG / p.lanes, t = threadIdx.x & (p.lanes - 1), sub = threadIdx.x / p.lanes;
    for (int64_t r = (int64_t)blockIdx.y * rows + sub; r < p.N; r += (int64_t)gridDim.y * rows) {
        const int64_t e0 = p.first + r * p.index_stride;
        const int64_t b1 = (e0 + p.C + 7) >> 3;
        const typename Elem<XT>::T* xr = x + r * p.x_stride;
        const O* rr = residual + r * p.residual_stride;
        O* o = out + r * p.out_stride;
        for (int64_t b = (e0 >> 3) + (int64_t)blockIdx.x * p.lanes + t; b < b1; b += (int64_t)gridDim.x * p.lanes) {
            const int64_t at = b * 8 - e0;
            const bool whole = at >= 0 && at + 8 <= p.C;
            Eight<XT> v;
            Eight<OT> w;
            if (whole) {
                v = load_eight<FAR>((const Eight<XT>*)(xr + at));
                if (residual) w = load_eight<FAR>((const Eight<OT>*)(rr + at));
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (at + j >= 0 && at + j < p.C) {
                        v[j] = xr[at + j];
                        if (residual) w[j] = rr[at + j];
                    }
            }
            const Words m = draw_words(key, b, 0, p.site);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint32_t bits = j & 1 ? m.w[j / 2] >> 16 : m.w[j / 2] & 0xFFFFu;
                const bool keep = bits >= p.threshold;
                const float s = keep ? p.scale : 0.0f, xv = keep ? (float)v[j] : 0.0f;
                w[j] = (O)(residual ? fmaf(xv, s, (float)w[j]) : xv * s);
            }
            if (whole) {
                *(Eight<OT>*)(o + at) = w;
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (at + j >= 0 && at + j < p.C) o[at + j] = w[j];
            }
        }
    }
}

}  // namespace sfk

using namespace sfk;

SF_API int sf_uniform(const int64_t* key, uint32_t site, int64_t first, int64_t n, float* out, sf_stream_t stream)
{
    constexpr int64_t most = (int64_t)1 << 60;
    if (first < 0 || n < 0 || first > most || n > most - first) return SF_EINVAL;
    if (n == 0) return SF_OK;
    if (!key || !out || !aligned(key, 8) || !aligned(out, 4) || !disjoint(key, 16, out, n * 4)) return SF_EINVAL;
    const int64_t groups = ((n + 3) / 4 + 1 + kDrawWG - 1) / kDrawWG;
    void* args[] = {(void*)&key, (void*)&site, (void*)&first, (void*)&n, (void*)&out};
    return launch((const void*)k_uniform, dim3((unsigned)(groups < 4096 ? groups : 4096)), dim3(kDrawWG), args, 0, stream);
}

static inline bool dtype_ok(int32_t d) { return d == SF_F32 || d == SF_BF16 || d == SF_F16; }

// Whether rows of `stride` may be written while those of another array are read:
// the very same rows, or none of their bytes.
static inline bool apart_or_same(const void* out, int64_t out_bytes, int64_t out_stride, int32_t out_dtype, const void* in,
                                 int64_t in_bytes, int64_t in_stride, int32_t in_dtype, int64_t N)
{
    return (out == in && out_dtype == in_dtype && (N == 1 || out_stride == in_stride)) ||
           disjoint(out, out_bytes, in, in_bytes);
}

SF_API int sf_dropout(const void* x, int32_t dtype, int64_t N, int64_t C, int64_t x_stride, float p,
                      const int64_t* key, uint32_t site, int64_t first, int64_t index_stride, const void* residual,
                      int64_t residual_stride, void* out, int32_t out_dtype, int64_t out_stride, sf_stream_t stream)
{
    constexpr int64_t most = (int64_t)1 << 40, indexes = (int64_t)1 << 60;
    if (!dtype_ok(dtype) || !dtype_ok(out_dtype) || !(p >= 0.0f && p <= 1.0f)) return SF_EINVAL;
    if (N < 0 || N > most || C < 0 || C > most || x_stride < C || x_stride > most || out_stride < C || out_stride > most)
        return SF_EINVAL;
    if (residual && (residual_stride < C || residual_stride > most)) return SF_EINVAL;
    if (first < 0 || first > indexes || index_stride < C || index_stride > indexes) return SF_EINVAL;
    if (N == 0 || C == 0) return SF_OK;
    if (N > 1 && index_stride > (indexes - first) / (N - 1)) return SF_EINVAL;
    if (first + (N - 1) * index_stride > indexes - C) return SF_EINVAL;
    const int64_t longest = x_stride > out_stride ? x_stride : out_stride;
    if ((residual && residual_stride > longest ? residual_stride : longest) > ((int64_t)1 << 56) / N) return SF_EINVAL;
    const int xb = elem_size(dtype), ob = elem_size(out_dtype);
    if (!x || !key || !out || !aligned(x, xb) || !aligned(key, 8) || !aligned(out, ob) || !aligned(residual, ob))
        return SF_EINVAL;
    const int64_t x_bytes = ((N - 1) * x_stride + C) * xb, out_bytes = ((N - 1) * out_stride + C) * ob;
    if (!apart_or_same(out, out_bytes, out_stride, out_dtype, x, x_bytes, x_stride, dtype, N) ||
        !disjoint(out, out_bytes, key, 16))
        return SF_EINVAL;
    if (residual && !apart_or_same(out, out_bytes, out_stride, out_dtype, residual, ((N - 1) * residual_stride + C) * ob,
                                   residual_stride, out_dtype, N))
        return SF_EINVAL;
    DropShape a = {N, C, x_stride, residual ? residual_stride : 0, out_stride, first, index_stride, site, 0, 0.0f, kDrawWG};
    // rows that follow each other in memory and in index are one
    if (x_stride == C && out_stride == C && index_stride == C && (!residual || residual_stride == C)) {
        a.C = N * C;
        a.N = 1;
    }
    a.threshold = (uint32_t)(p * 65536.0 + 0.5);
    a.scale = a.threshold < 65536 ? (float)(65536.0 / (65536 - (int)a.threshold)) : 0.0f;
    const bool far = a.N * a.C * (xb + (residual ? 2 : 1) * ob) > kLastCache;
    const int64_t blocks = a.C / 8 + 2;  // a row's, at most
    if (a.N > 1)
        while (a.lanes > 1 && a.lanes / 2 >= blocks) a.lanes /= 2;
    const int64_t across = (blocks + a.lanes - 1) / a.lanes, down = (a.N * a.lanes + kDrawWG - 1) / kDrawWG;
    void* args[] = {(void*)&x, (void*)&key, (void*)&residual, (void*)&out, (void*)&a};
#define SF_DROPOUT(X, O) {(const void*)&k_dropout<X, O, false>, (const void*)&k_dropout<X, O, true>}
    const void* fn[3][3][2] = {{SF_DROPOUT(SF_F32, SF_F32), SF_DROPOUT(SF_F32, SF_BF16), SF_DROPOUT(SF_F32, SF_F16)},
                               {SF_DROPOUT(SF_BF16, SF_F32), SF_DROPOUT(SF_BF16, SF_BF16), SF_DROPOUT(SF_BF16, SF_F16)},
                               {SF_DROPOUT(SF_F16, SF_F32), SF_DROPOUT(SF_F16, SF_BF16), SF_DROPOUT(SF_F16, SF_F16)}};
#undef SF_DROPOUT
    return launch(fn[dtype][out_dtype][far], dim3((unsigned)(across < (1 << 20) ? across : 1 << 20), (unsigned)(down < 65535 ? down : 65535)),
                  dim3(kDrawWG), args, 0, stream);
}
