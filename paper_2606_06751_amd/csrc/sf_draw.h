// sf_draw.h -- what the kernels of stagefrontier_draw.h share: the generator,
// powers of two in 64 bits, sums of rows of logits by segments, and the choice
// of an entry by its place in the cumulative sums.
#pragma once

#include <type_traits>

#include "sf_train.h"

namespace sfk {

// -- random numbers by counter -----------------------------------------------

struct Words {
    uint32_t w[4];
};

// One instruction, which the compiler does not take by itself here (20480007 numbers:
// 14.8 us, with two 15.5).
__device__ __forceinline__ uint32_t xor3(uint32_t a, uint32_t b, uint32_t c)
{
    return (uint32_t)__builtin_amdgcn_bitop3_b32((int)a, (int)b, (int)c, 0x96);
}

// Philox4x32-10 (Salmon, Moraes, Dror, Shaw, SC 2011): ten rounds of two
// 32 x 32 -> 64 bit products and exclusive ors, the key raised by Weyl constants
// in between.  (A product of 64 bits is one instruction at the full rate here.)
__device__ __forceinline__ Words philox(uint32_t c0, uint32_t c1, uint32_t c2, uint32_t c3, uint32_t k0, uint32_t k1)
{
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
        c0 = xor3((uint32_t)(b >> 32), c1, k0);
        c1 = (uint32_t)b;
        c2 = xor3((uint32_t)(a >> 32), c3, k1);
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

// 2^f for f in [-1/2, 1/2] within 2^-39.7: the interpolation of degree 8 at
// Chebyshev's points.  (Each degree is one of 16 instructions an entry, and a
// factor of 58 in the error.)
__device__ __forceinline__ double pow2_rest(double f)
{
    double p = 1.3255224878668817e-06;
    p = fma(p, f, 1.5310079402249296e-05);
    p = fma(p, f, 0.00015403455852453838);
    p = fma(p, f, 0.0013333450568000645);
    p = fma(p, f, 0.009618129159402558);
    p = fma(p, f, 0.05550410941205933);
    p = fma(p, f, 0.2402265069581299);
    p = fma(p, f, 0.6931471805459335);
    return fma(p, f, 1.0);
}

// The sum of kWhole and a number below 2^31 is a whole number plus kWhole, and holds
// it in its low word.
constexpr double kWhole = 6755399441055744.0;  // 1.5 * 2^52

// s 2^(x c) for |x c| < 2^31: x c = whole + f by two multiply-adds, each rounded once.
__device__ __forceinline__ double pow2_times(double s, double x, double c)
{
    const double whole = fma(x, c, kWhole);
    const double p = pow2_rest(fma(x, c, kWhole - whole));
    return ldexp(s * p, (int)(uint32_t)(uint64_t)__double_as_longlong(whole));
}
__device__ __forceinline__ double pow2(double x, double c) { return pow2_times(1.0, x, c); }

// 2^(d c) for any d c up to 0 (or somewhat above): 0 below 2^-1000, NaN for NaN.
// (Chosen, not branched for: the power of 0 in its place.)
__device__ __forceinline__ double pow2_any(double d, double c)
{
    const bool far = d * c < -1000.0;
    const double p = pow2(far ? 0.0 : d, c);
    return far ? 0.0 : p;
}

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

// What a call knows of its rows.
struct RowArg {
    int64_t stride;
    int V, nseg;
    double c;  // log2(e) / T
    float inv_t;
    float floor, top;  // x c = -1000 and 1000
};

// s = sum 2^((x - m) c) over a segment or row.  m is 0 for a segment of ordinary
// logits, else its largest x; a row's is the largest of its segments'.  m = -inf:
// nothing but -inf, s = 0.  s is NaN where there is +inf or NaN.
struct RowSum {
    double s;
    float m, pad;
};

// What a lane holds of a segment: its vectors, and one of the entries behind the
// row's last whole vector; -inf where there is none.
template <int DT>
struct SegData {
    VecU<DT> y[kSegU];
    float edge;
};

// How many of a segment's vectors have entries.
template <int DT>
__device__ __forceinline__ int seg_live(int seg, int V)
{
    const int n = V - seg * kSeg<DT>, step = 64 * kVec<DT>;
    return n >= kSeg<DT> ? kSegU : (n - n % kVec<DT> + step - 1) / step;
}

template <int DT, int LIVE = kSegU>
__device__ __forceinline__ SegData<DT> seg_load(const typename Elem<DT>::T* row, int seg, int V, int lane)
{
    typedef typename Elem<DT>::T T;
    constexpr int E = kVec<DT>;
    const int at = seg * kSeg<DT> + lane * E;
    SegData<DT> a;
    a.edge = -INFINITY;
    if (LIVE == kSegU && seg * kSeg<DT> + kSeg<DT> <= V) {
#pragma unroll
        for (int k = 0; k < kSegU; ++k) a.y[k] = __builtin_nontemporal_load((const VecU<DT>*)(row + at + k * 64 * E));
    } else {
#pragma unroll
        for (int k = 0; k < kSegU; ++k) {
            a.y[k] = (VecU<DT>)(T)-INFINITY;
            if (k < LIVE && at + k * 64 * E + E <= V) a.y[k] = __builtin_nontemporal_load((const VecU<DT>*)(row + at + k * 64 * E));
        }
        const int tail = V - V % E + lane;
        if (tail < V) a.edge = (float)row[tail];
    }
    return a;
}

// The larger, NaN where one of them is, unlike fmaxf.
__device__ __forceinline__ float max_or_nan(float a, float b) { return __builtin_elementwise_maximum(a, b); }

// The segment's sum, in every lane, for any logits: relative to the largest, each
// entry asked about.
template <int DT>
__device__ __forceinline__ RowSum seg_sum_any(const SegData<DT>& a, double c)
{
    constexpr int E = kVec<DT>;
    float top = a.edge;
#pragma unroll
    for (int k = 0; k < kSegU; ++k)
#pragma unroll
        for (int j = 0; j < E; ++j) top = max_or_nan(top, (float)a.y[k][j]);
    const float m = wave_max_f32(top);
    if (__any(!(top < INFINITY))) return {(double)NAN, m, 0.0f};
    if (m == -INFINITY) return {0.0, m, 0.0f};
    double s = pow2_any((double)a.edge - (double)m, c);
#pragma unroll
    for (int k = 0; k < kSegU; ++k)
#pragma unroll
        for (int j = 0; j < E; ++j) s += pow2_any((double)(float)a.y[k][j] - (double)m, c);
    return {wave_sum_f64(s), m, 0.0f};
}

// A power as a segment of ordinary logits takes it: held at 2^-1000 below, NaN for NaN.
__device__ __forceinline__ double pow2_held(float x, const RowArg& z) { return pow2((double)max_or_nan(x, z.floor), z.c); }

template <int DT>
__device__ __forceinline__ double vector_sum(const VecU<DT>& y, const RowArg& z)
{
    double s = 0.0;
#pragma unroll
    for (int j = 0; j < kVec<DT>; ++j) s += pow2_held((float)y[j], z);
    return s;
}

// A vector's bits as whole numbers, whose order is that of positive entries, NaN
// above all: packed comparisons take half an instruction an entry.
template <int DT>
using VecBits = typename std::conditional<DT == SF_F32, int32_t, int16_t>::type __attribute__((ext_vector_type(kVec<DT>)));
template <int DT>
__device__ __forceinline__ bool bits_above(const VecBits<DT>& top, float limit)
{
    const auto bits = __builtin_bit_cast(typename std::conditional<DT == SF_F32, int32_t, int16_t>::type,
                                         (typename Elem<DT>::T)limit);
    bool above = false;
#pragma unroll
    for (int j = 0; j < kVec<DT>; ++j) above |= top[j] >= bits;
    return above;
}
// Whether an entry of the lane lies at or above a positive limit.
template <int DT>
__device__ __forceinline__ bool seg_above(const SegData<DT>& a, float limit)
{
    VecBits<DT> top = __builtin_bit_cast(VecBits<DT>, (VecU<DT>)a.y[0]);
#pragma unroll
    for (int k = 1; k < kSegU; ++k) top = __builtin_elementwise_max(top, __builtin_bit_cast(VecBits<DT>, (VecU<DT>)a.y[k]));
    return bits_above<DT>(top, limit) || !(a.edge < limit);
}

// Whether sums of powers taken as they are keep what counts: at least 2^800 over
// what is held, and far from the largest number.
__device__ __forceinline__ bool sum_is_ordinary(double s) { return s > 0x1p-200 && s < 0x1p900; }

// The segment's sum, in every lane.  64 bits have room for powers of ordinary
// logits as they are, so no maximum is looked for: only whether one lies above
// that room.  Where the sum shows that the segment is another, it is done again.
// (Without the maximum 84 in place of 95 us at 900 rows of 131072.)
template <int DT>
__device__ __forceinline__ RowSum seg_sum(const SegData<DT>& a, int live, const RowArg& z)
{
    constexpr int E = kVec<DT>;
    const bool above = __any(seg_above<DT>(a, z.top));
    double s = 0.0;
#pragma unroll
    for (int k = 0; k < kSegU; ++k)
        if (k < live) s += vector_sum<DT>(a.y[k], z);
    if (__any(a.edge != -INFINITY)) s += pow2_held(a.edge, z);
    s = wave_sum_f64(s);
    if (!above && sum_is_ordinary(s)) return {s, 0.0f, 0.0f};
    return seg_sum_any<DT>(a, z.c);
}

// -- the same of many bfloat16 rows: powers from a table ----------------------

// A bfloat16 is one of few numbers, and of those between 2^-55 / c and 2^10 / c,
// whose powers are neither 1 nor held, there are 65 binades of 128 of each sign:
// 130 KB of a compute unit's 160 KB of LDS.  A power then takes half of five packed
// instructions, two for an address and a read of 8 bytes, in place of 15 of 64 bits,
// and it is the same number, bit for bit.  (float16 has eight times the numbers a
// binade: its table would not fit.)  2304 rows of 131072: 115 us in place of 192; HBM
// alone takes 85, and what is left is neither the banks of LDS (reads without
// conflicts: 112) nor reads in flight (all 32 of a segment before the first is added:
// the same).  (Binades below 2^-42 / c, whose powers are within 2^-41 of 1, are 0.6 us
// of it.)
constexpr int kTableBinades = 65;
constexpr int kTableSize = 2 * kTableBinades * 128;  // sign in the lowest bit of the place
constexpr int kTableWG = 1024;

// The bits of the magnitude that the table begins at, or -1 where c is so far from 1
// that a float's range does not hold it.  At 2^-55 / c or up to twice that, so that
// what lies below has a power within 2^-54.5 of 1, which rounds to 1.
static inline int table_begin(double c)
{
    const int e = (int)ceil(log2(0x1p-55 / c)) + 127;
    return e >= 1 && e + kTableBinades <= 254 ? e * 128 : -1;
}

// By every thread of a workgroup, before its first use.
__device__ __forceinline__ void table_fill(double* table, int begin, const RowArg& z)
{
    for (int i = threadIdx.x; i < kTableSize; i += kTableWG) {
        const int r = i >> 1;
        table[i] = pow2_held(__uint_as_float((r == 0 ? 0u : (uint32_t)(begin + r) << 16) | (uint32_t)i << 31), z);
    }
    __syncthreads();
}

typedef uint16_t Two __attribute__((ext_vector_type(2)));

// The places of two entries.
__device__ __forceinline__ Two table_places(uint32_t two, uint32_t begin)
{
    const Two size = __builtin_bit_cast(Two, two & 0x7FFF7FFFu);
    Two r = __builtin_elementwise_sub_sat(size, (Two)(uint16_t)begin);
    r = __builtin_elementwise_min(r, (Two)(uint16_t)(kTableSize / 2 - 1));
    return r * (Two)(uint16_t)2 + (__builtin_bit_cast(Two, two) >> 15);
}

typedef uint32_t Words4 __attribute__((ext_vector_type(4)));

// seg_sum, where entries that the table does not hold (NaN of either sign, ones
// above) send the segment the other way.
__device__ __forceinline__ RowSum seg_sum_table(const SegData<SF_BF16>& a, int live, const RowArg& z, const double* table, uint32_t begin)
{
    typedef uint16_t V8 __attribute__((ext_vector_type(8)));
    V8 top = __builtin_bit_cast(V8, (VecU<SF_BF16>)a.y[0]);
#pragma unroll
    for (int k = 1; k < kSegU; ++k) top = __builtin_elementwise_max(top, __builtin_bit_cast(V8, (VecU<SF_BF16>)a.y[k]));
    bool other = seg_above<SF_BF16>(a, z.top) || a.edge != a.edge;
#pragma unroll
    for (int j = 0; j < 8; ++j) other |= top[j] > 0xFF80u;
    double s = 0.0;
#pragma unroll
    for (int k = 0; k < kSegU; ++k)
        if (k < live) {
            const Words4 w = __builtin_bit_cast(Words4, (VecU<SF_BF16>)a.y[k]);
            double own = 0.0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const Two at = table_places(w[j], begin);
                own += table[at[0]];
                own += table[at[1]];
            }
            s += own;
        }
    if (__any(a.edge != -INFINITY)) s += pow2_held(a.edge, z);
    s = wave_sum_f64(s);
    if (!__any(other) && sum_is_ordinary(s)) return {s, 0.0f, 0.0f};
    return seg_sum_any<SF_BF16>(a, z.c);
}

// A segment's weight relative to the row's reference, whose own entry weighs 1 (the
// sums of ordinary rows, relative to 0, 2^-200 at least).  The power is scaled with
// the sum, which may be up to 2^900, and what is left below 2^-900 counts as 0: a
// segment that weighs something has an entry within 2^-1000, which weighs something by
// itself (pow2_any), so the choice that a segment is given finds one.
__device__ __forceinline__ double seg_weight(const RowSum& a, float top, double c)
{
    if (a.m == top || a.m == -INFINITY) return a.s;
    const double d = (double)a.m - (double)top;
    const bool far = d * c < -2000.0;
    const double s = pow2_times(far ? a.s * 0.0 : a.s, far ? 0.0 : d, c);
    return s < 0x1p-900 ? 0.0 : s;  // (NaN stays)
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

// log2 s for s > 0, within 2^-39: that of the fraction in 32 bits, and the logarithm
// of the little by which its power misses the fraction.  (A fourth of the
// instructions of log().)
__device__ __forceinline__ double log2_of(double s)
{
    int whole;
    const double x = frexp(s, &whole);  // in [1/2, 1)
    const double l = (double)__builtin_amdgcn_logf((float)x);
    const double d = fma(x, pow2(-l, 1.0), -1.0);  // below 2^-20
    return (double)whole + fma(fma(d, -0.5, 1.0) * d, kLog2eD, l);
}

// log p of an entry x of the row, rounded once, at most 0.  Near 0 the logarithms of the
// sum and of the power cancel, and 2^-38.5 of error would be left: there the power e is
// taken out of the sum s that holds it bit for bit (what has more than half of a row has
// the row's reference), and log(e / s) = -2 artanh((s - e) / (s + e)) is as exact as what
// is left.  The series' first term left out, v^11 / 11, is 2^-43 of it at v = 1/16.
__device__ __forceinline__ float row_logp(float x, const RowSum& r, const RowArg& z)
{
    constexpr double ln2 = 0.69314718055994530942;
    const double d = (double)x - (double)r.m, far = fma(-ln2, log2_of(r.s), d * (double)z.inv_t);
    if (far < -0.125) return (float)far;
    const double e = pow2_any(d, z.c), v = fmax(r.s - e, 0.0) / (r.s + e), q = v * v;
    return (float)(0.0 - 2.0 * v * fma(fma(fma(fma(q, 1.0 / 9, 1.0 / 7), q, 1.0 / 5), q, 1.0 / 3), q, 1.0));
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

// Of E neighbouring entries a lane, whose sums are `own` and whose inclusive sums
// over the lanes are `sum`: the number of the first whose inclusive sum from `run`
// on passes `target`, wave-uniform, -1: none.  `last` becomes the number of the last
// that has weight, if there is one.  Weights up to `none` count as 0.
template <int E>
__device__ __forceinline__ int pick_scanned(const double (&v)[E], double own, double sum, double run, double target, int lane,
                                            int& last, double none = 0.0)
{
    double r = run + (sum - own);
    int first = -1, mine = -1;
#pragma unroll
    for (int j = 0; j < E; ++j) {
        r += v[j];
        if (v[j] > none) {
            mine = lane * E + j;
            if (first < 0 && r > target) first = mine;
        }
    }
    if (first < 0 && run + sum > target) first = mine;  // (between the two orders of summation)
    const uint64_t past = __ballot(first >= 0), some = __ballot(mine >= 0);
    if (some) last = __builtin_amdgcn_readlane(mine, 63 - __builtin_clzll(some));
    return past ? __builtin_amdgcn_readlane(first, __builtin_ctzll(past)) : -1;
}

// A lane's entries of vector k of a segment as `value(x, at)` weighs them, 0 behind the row.
template <int DT, class F>
__device__ __forceinline__ void entry_values(const typename Elem<DT>::T* row, int at, int V, F value, double (&v)[kVec<DT>])
{
    constexpr int E = kVec<DT>;
    if (at + E <= V) {
        const VecU<DT> x = *(const VecU<DT>*)(row + at);
#pragma unroll
        for (int j = 0; j < E; ++j) v[j] = value((float)x[j], at + j);
    } else {
#pragma unroll
        for (int j = 0; j < E; ++j) v[j] = at + j < V ? value((float)row[at + j], at + j) : 0.0;
    }
}

// The entry of a segment whose inclusive sum, from `base` on, passes `target`, or
// the last with weight where rounding leaves none; -1 where none has weight, or
// there is no segment.  By one wave, vector by vector, in the row's order.
template <int DT, class F>
__device__ __forceinline__ int pick_entry(const typename Elem<DT>::T* row, F value, Place p, int V, double target, int lane)
{
    constexpr int E = kVec<DT>;
    int last = -1;
#pragma unroll 1
    for (int k = p.i < 0 ? kSegU : 0; k < kSegU; ++k) {
        const int first = p.i * kSeg<DT> + k * 64 * E;
        double v[E];
        entry_values<DT>(row, first + lane * E, V, value, v);
        double own = 0.0;
#pragma unroll
        for (int j = 0; j < E; ++j) own += v[j];
        const double sum = wave_scan_f64(own);
        int some = -1;
        const int hit = pick_scanned<E>(v, own, sum, p.base, target, lane, some);
        p.base += lane_f64(sum, 63);
        if (hit >= 0) return first + hit;
        if (some >= 0) last = first + some;
    }
    return last;
}

// The same by the first kSegU waves of a workgroup, a vector each, in every lane;
// every wave of it takes part.
struct PickShared {
    double sum[kSegU];
    int hit[kSegU], last[kSegU];
};
// The sum of a segment's values by the first kSegU waves, in every lane.
template <int DT, class F>
__device__ __forceinline__ double entry_sum_group(const typename Elem<DT>::T* row, F value, int seg, int V, PickShared& shared)
{
    constexpr int E = kVec<DT>;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    double v[E], own = 0.0;
    if (wave < kSegU) {
        entry_values<DT>(row, seg * kSeg<DT> + (wave * 64 + lane) * E, V, value, v);
#pragma unroll
        for (int j = 0; j < E; ++j) own += v[j];
    }
    own = wave_sum_f64(own);
    __syncthreads();  // former sums are read
    if (lane == 0 && wave < kSegU) shared.sum[wave] = own;
    __syncthreads();
    own = 0.0;
    for (int w = 0; w < kSegU; ++w) own += shared.sum[w];
    return own;
}

template <int DT, class F>
__device__ __forceinline__ int pick_entry_group(const typename Elem<DT>::T* row, F value, Place p, int V, double target,
                                                PickShared& shared)
{
    constexpr int E = kVec<DT>;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const bool works = wave < kSegU && p.i >= 0;
    const int first = p.i * kSeg<DT> + wave * 64 * E;
    double v[E];
#pragma unroll
    for (int j = 0; j < E; ++j) v[j] = 0.0;
    if (works) entry_values<DT>(row, first + lane * E, V, value, v);
    double own = 0.0;
#pragma unroll
    for (int j = 0; j < E; ++j) own += v[j];
    const double sum = wave_scan_f64(own);
    __syncthreads();  // a former choice is read
    if (lane == 63 && wave < kSegU) shared.sum[wave] = sum;
    __syncthreads();
    double run = p.base;
    for (int w = 0; w < wave && w < kSegU; ++w) run += shared.sum[w];
    int last = -1;
    const int hit = pick_scanned<E>(v, own, sum, run, target, lane, last);
    if (lane == 0 && wave < kSegU) {
        shared.hit[wave] = hit < 0 ? -1 : first + hit;
        shared.last[wave] = last < 0 ? -1 : first + last;
    }
    __syncthreads();
    int t = -1;
    for (int w = 0; w < kSegU; ++w) t = shared.last[w] >= 0 ? shared.last[w] : t;
    for (int w = kSegU - 1; w >= 0; --w) t = shared.hit[w] >= 0 ? shared.hit[w] : t;
    return t;
}

}  // namespace sfk
