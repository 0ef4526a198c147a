// sf_draw.h -- what the kernels of stagefrontier_draw.h share: the generator,
// powers of two in 64 bits, sums of rows of logits by segments, and the choice
// of an entry by its place in the cumulative sums.
#pragma once

#include "sf_train.h"

namespace sfk {

// -- random numbers by counter -----------------------------------------------

struct Words {
    uint32_t w[4];
};

// Philox4x32-10 (Salmon, Moraes, Dror, Shaw, SC 2011): ten rounds of two
// 32 x 32 -> 64 bit products and exclusive ors, the key raised by Weyl constants
// in between.
__device__ __forceinline__ Words philox(uint32_t c0, uint32_t c1, uint32_t c2, uint32_t c3, uint32_t k0, uint32_t k1)
{
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
        c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
        c1 = (uint32_t)b;
        c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
        c3 = (uint32_t)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return {{c0, c1, c2, c3}};
}

// The words of a block of a kind (sf_uniform 1, sf_dropout 0) at a site.
__device__ __forceinline__ Words draw_words(const int64_t* key, int64_t block, uint32_t kind, uint32_t site)
{
    return philox((uint32_t)block, (uint32_t)(block >> 32) | kind << 31, site, (uint32_t)key[1], (uint32_t)key[0],
                  (uint32_t)(key[0] >> 32));
}

// -- powers of two in 64 bits ------------------------------------------------

// 2^(d c) for |d c| < 2^31, within 2^-45: the whole part by the addition of
// 1.5 * 2^52, whose sum holds it in its low word, the rest f in [-1/2, 1/2] by the
// interpolation of 2^f of degree 9 at Chebyshev's points (error 1.9e-14; degree
// 8 gives 1.1e-12, one multiply-add less of 18).  A product that rounds once, in
// either multiply-add, so d need not be rounded to a whole number of anything.
__device__ __forceinline__ double pow2(double d, double c)
{
    const double big = 6755399441055744.0;
    const double whole = fma(d, c, big);
    const double f = fma(d, c, big - whole);
    double p = 1.0205905413765595e-07;
    p = fma(p, f, 1.325964524488711e-06);
    p = fma(p, f, 1.5252672924850737e-05);
    p = fma(p, f, 0.0001540343375125101);
    p = fma(p, f, 0.0013333558200794592);
    p = fma(p, f, 0.009618129193934313);
    p = fma(p, f, 0.05550410866465167);
    p = fma(p, f, 0.2402265069564034);
    p = fma(p, f, 0.6931471805599462);
    p = fma(p, f, 1.0000000000000135);
    return ldexp(p, (int)(uint32_t)(uint64_t)__double_as_longlong(whole));
}

// The same for any d c up to 0 and any c > 0: nothing is left below 2^-1000.
__device__ __forceinline__ double pow2_any(double d, double c) { return d * c < -1000.0 ? 0.0 : pow2(d, c); }

// -- rows of logits by segments ----------------------------------------------

// A segment is 64 lanes times kSegU vectors of consecutive entries of a row; a
// wave sums it.  Its place depends on the row's first entry alone, so sums do
// not depend on addresses or on the split of the work.
constexpr int kSegU = 4;
template <int DT>
constexpr int kSeg = 64 * kSegU * kVec<DT>;

static inline int64_t seg_count(int dtype, int64_t V)
{
    const int64_t seg = dtype == SF_F32 ? kSeg<SF_F32> : kSeg<SF_BF16>;
    return (V + seg - 1) / seg;
}

// s = sum 2^((x - m) c) over a segment or row, m its largest x.  m = -inf: nothing
// but -inf, s = 0.  s is NaN where there is +inf or NaN.
struct RowSum {
    double s;
    float m, pad;
};

template <int DT>
struct SegData {
    VecU<DT> y[kSegU];
    float edge;  // an entry behind the last whole vector, -inf: none
};

template <int DT>
__device__ __forceinline__ SegData<DT> seg_load(const typename Elem<DT>::T* row, int seg, int V, int lane)
{
    typedef typename Elem<DT>::T T;
    constexpr int E = kVec<DT>;
    const int at = seg * kSeg<DT> + lane * E;
    SegData<DT> a;
    a.edge = -INFINITY;
    if (seg * kSeg<DT> + kSeg<DT> <= V) {
#pragma unroll
        for (int k = 0; k < kSegU; ++k) a.y[k] = __builtin_nontemporal_load((const VecU<DT>*)(row + at + k * 64 * E));
    } else {
#pragma unroll
        for (int k = 0; k < kSegU; ++k) {
            a.y[k] = (VecU<DT>)(T)-INFINITY;
            if (at + k * 64 * E + E <= V) a.y[k] = __builtin_nontemporal_load((const VecU<DT>*)(row + at + k * 64 * E));
        }
        const int tail = V - V % E + lane;
        if (tail < V) a.edge = (float)row[tail];
    }
    return a;
}

// The segment's sum, in every lane.  Where no entry lies so far below the
// largest that its power leaves 64 bits' range, none is asked about.
template <int DT>
__device__ __forceinline__ RowSum seg_sum(const SegData<DT>& a, double c)
{
    constexpr int E = kVec<DT>;
    float top = a.edge, low = INFINITY;
#pragma unroll
    for (int k = 0; k < kSegU; ++k)
#pragma unroll
        for (int j = 0; j < E; ++j) {
            top = fmaxf(top, (float)a.y[k][j]);
            low = fminf(low, (float)a.y[k][j]);
        }
    const float m = wave_max_f32(top);
    double s = 0.0;
    if (m == -INFINITY || m == INFINITY) {
        bool nan = m == INFINITY || a.edge != a.edge;
#pragma unroll
        for (int k = 0; k < kSegU; ++k)
#pragma unroll
            for (int j = 0; j < E; ++j) nan |= (float)a.y[k][j] != (float)a.y[k][j];
        return {__any(nan) ? (double)NAN : 0.0, m, 0.0f};
    }
    const double md = m;
    if (__any(!(((double)low - md) * c >= -1000.0))) {
        s = pow2_any((double)a.edge - md, c);
#pragma unroll
        for (int k = 0; k < kSegU; ++k)
#pragma unroll
            for (int j = 0; j < E; ++j) s += pow2_any((double)(float)a.y[k][j] - md, c);
    } else {
        // (a segment with an edge lacks a vector, so it holds -inf and is not summed here)
#pragma unroll
        for (int k = 0; k < kSegU; ++k)
#pragma unroll
            for (int j = 0; j < E; ++j) s += pow2((double)(float)a.y[k][j] - md, c);
    }
    return {wave_sum_f64(s), m, 0.0f};
}

// A segment's weight relative to the row's largest entry.
__device__ __forceinline__ double seg_weight(const RowSum& a, float top, double c)
{
    return a.m == -INFINITY ? a.s : a.s * pow2_any((double)a.m - (double)top, c);
}

// Joins a row's segments by one wave, in every lane.
__device__ __forceinline__ RowSum row_sum(const RowSum* seg, int n, double c, int lane)
{
    float top = -INFINITY;
    for (int i = lane; i < n; i += 64) top = fmaxf(top, seg[i].m);
    top = wave_max_f32(top);
    double s = 0.0;
    for (int i = lane; i < n; i += 64) s += seg_weight(seg[i], top, c);
    return {wave_sum_f64(s), top, 0.0f};
}

// log p of an entry, rounded once.
__device__ __forceinline__ float row_logp(float x, const RowSum& r, float inv_t)
{
    return (float)(((double)x - (double)r.m) * (double)inv_t - log(r.s));
}

// -- the choice of an entry --------------------------------------------------

// Inclusive sums over the lanes of a wave, in a fixed order.
__device__ __forceinline__ double wave_scan_f64(double v)
{
    v += dpp_f64<0x111, 0xF>(v);  // row_shr:1, 2, 4, 8
    v += dpp_f64<0x112, 0xF>(v);
    v += dpp_f64<0x114, 0xF>(v);
    v += dpp_f64<0x118, 0xF>(v);
    v += dpp_f64<0x142, 0xA>(v);  // row_bcast:15 -> rows 1, 3
    v += dpp_f64<0x143, 0xC>(v);  // row_bcast:31 -> rows 2, 3
    return v;
}
__device__ __forceinline__ double lane_f64(double v, int lane)
{
    const uint64_t u = (uint64_t)__double_as_longlong(v);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)u, lane);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(u >> 32), lane);
    return __longlong_as_double((long long)((uint64_t)hi << 32 | lo));
}

struct Place {
    int i;        // -1: nothing has weight
    double base;  // the sum before it
};

// The first of n weights whose inclusive sum passes `target`, or the last that
// is not 0 where rounding leaves none; by one wave.  (Inclusive sums of lanes
// come from different orders, so a weight of 0 may pass by a rounding: it is
// never chosen.)
template <class F>
__device__ __forceinline__ Place pick_weight(F weight, int n, double target, int lane)
{
    double run = 0.0;
    Place last = {-1, 0.0};
    for (int i0 = 0; i0 < n; i0 += 64) {
        const double v = i0 + lane < n ? weight(i0 + lane) : 0.0;
        const double sum = wave_scan_f64(v);
        const uint64_t some = __ballot(v > 0.0), past = __ballot(v > 0.0 && run + sum > target);
        if (past) {
            const int l = __builtin_ctzll(past);
            return {i0 + l, run + lane_f64(sum - v, l)};
        }
        if (some) {
            const int l = 63 - __builtin_clzll(some);
            last = {i0 + l, run + lane_f64(sum - v, l)};
        }
        run += lane_f64(sum, 63);
    }
    return last;
}

// The same over the entries of a segment: value(j) of entry j, asked for below V
// only.  Entries are taken vector by vector, so that their order is the row's.
// -1 where none has weight, or there is no segment.
template <int DT, class F>
__device__ __forceinline__ int pick_entry(F value, int seg, int V, double base, double target, int lane)
{
    constexpr int E = kVec<DT>;
    double run = base;
    int last = -1;
#pragma unroll 1
    for (int k = seg < 0 ? kSegU : 0; k < kSegU; ++k) {
        const int at = seg * kSeg<DT> + (k * 64 + lane) * E;
        double v[E], own = 0.0;
#pragma unroll
        for (int j = 0; j < E; ++j) {
            v[j] = at + j < V ? value(at + j) : 0.0;
            own += v[j];
        }
        const double sum = wave_scan_f64(own);
        double r = run + (sum - own);
        int first = -1;
#pragma unroll
        for (int j = 0; j < E; ++j) {
            r += v[j];
            if (v[j] > 0.0) {
                last = at + j;
                if (first < 0 && r > target) first = at + j;
            }
        }
        if (own > 0.0 && first < 0 && run + sum > target) first = last;
        const uint64_t past = __ballot(first >= 0);
        if (past) return __builtin_amdgcn_readlane(first, __builtin_ctzll(past));
        run += lane_f64(sum, 63);
    }
    for (int off = 32; off > 0; off >>= 1) last = max(last, __shfl_xor(last, off, 64));
    return last;
}

}  // namespace sfk
