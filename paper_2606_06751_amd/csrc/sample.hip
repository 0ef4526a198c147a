// sample.hip -- a token of each row of logits by given uniform numbers
// (sf_token_sample), and the verification of drafted tokens (sf_draft_verify).
//
// Tokens are whole numbers, so they are either the definition's or wrong: every
// sum and comparison that decides one is in 64 bits.  (In 32 bits a cumulative sum
// over 131072 entries is off by up to 2^-20 of the whole, more than most entries of
// a flat distribution have.)  A row is summed by segments (sf_draw.h), whose sums
// give the normaliser and, in order, the cumulative sums at the segments' ends;
// the segment that the uniform number falls into is read again for its entry.
//
// What bounds it: 18 instructions an entry, 14 of them of 64 bits, which issue at
// the rate of 32-bit ones but draw power enough to lower the clock (2.1 GHz).  302
// million bfloat16 entries take 192 us at 81% of the issue slots, 115 us by a table
// of powers in LDS, and HBM alone 85 us.

#include "sf_draw.h"
#include "sf_host.h"

namespace sfk {

constexpr int kRowsWG = 256;
constexpr int kRowsWaves = kRowsWG / 64;
static_assert(kRowsWaves == kSegU, "a wave for each vector of a segment");
constexpr int64_t kFewSegments = 1024;     // of residuals that are decided where they are summed
constexpr int64_t kManySegments = 65536;   // of rows that are summed in two rounds
constexpr int64_t kTableSegments = 8192;   // of rows whose powers come from a table
constexpr int kLdsSegs = 1024;             // of a row that one workgroup takes

__device__ __forceinline__ bool in_unit(float u) { return u >= 0.0f && u < 1.0f; }

// What is written of a row without a token: there is nothing to draw from, or it
// is not a number.
__device__ __forceinline__ float no_token(const RowSum& r) { return r.s == 0.0 ? -INFINITY : NAN; }

// Draws a row's token from its segments' sums: by one wave, or by every wave of a
// workgroup.
template <int DT, bool GROUP>
__device__ __forceinline__ void draw_token(const typename Elem<DT>::T* row, const RowSum* seg, const RowSum& r, double u,
                                           const RowArg& z, PickShared* shared, int64_t* token, float* logp)
{
    const int lane = threadIdx.x & 63;
    int t = -1;
    if (r.s > 0.0) {
        const double target = u * r.s;
        const Place at = pick_weight([&](int i) { return seg_weight(seg[i], r.m, z.c); }, z.nseg, target, lane);
        auto value = [&](float x, int) { return pow2_any((double)x - (double)r.m, z.c); };
        t = GROUP ? pick_entry_group<DT>(row, value, at, z.V, target, *shared) : pick_entry<DT>(row, value, at, z.V, target, lane);
    }
    if (GROUP ? threadIdx.x == 0 : lane == 0) {
        *token = t;
        *logp = t >= 0 ? row_logp((float)row[t], r, z) : no_token(r);
    }
}

// Rows of one segment, LIVE vectors a lane: a wave each, which keeps the powers
// from the sum to the choice, with the next row on its way.  (16000 x 515 f16: 14.5
// us, in place of 48 by segments of 2048 places and a second read; 370 instructions a
// row are 10 us of it, 144 of them the powers of 512 entries.)
template <int DT, int LIVE>
__global__ __launch_bounds__(kRowsWG) void k_token_short(const typename Elem<DT>::T* __restrict__ logits, int64_t N,
                                                         const float* __restrict__ uniform, RowArg z,
                                                         int64_t* __restrict__ token, float* __restrict__ logp)
{
    constexpr int E = kVec<DT>;
    const int lane = threadIdx.x & 63;
    const int64_t step = (int64_t)gridDim.x * kRowsWaves;
    int64_t i = (int64_t)blockIdx.x * kRowsWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (i >= N) return;
    float u = uniform[i];
    SegData<DT> a;
    if (in_unit(u)) a = seg_load<DT, LIVE>(logits + i * z.stride, 0, z.V, lane);
    for (;;) {
        const int64_t next = i + step;
        const float u_next = next < N ? uniform[next] : -1.0f;
        SegData<DT> b;
        if (in_unit(u_next)) b = seg_load<DT, LIVE>(logits + next * z.stride, 0, z.V, lane);
        int t = -1;
        float lp = 0.0f;
        if (in_unit(u)) {
            const bool above = __any(seg_above<DT>(a, z.top)), edge = __any(a.edge != -INFINITY);
            double v[LIVE][E], ve[1] = {0.0}, own[LIVE], sum[LIVE], s = 0.0, edges = 0.0;
#pragma unroll
            for (int k = 0; k < LIVE; ++k) {
                own[k] = 0.0;
#pragma unroll
                for (int j = 0; j < E; ++j) own[k] += v[k][j] = pow2_held((float)a.y[k][j], z);
                sum[k] = wave_scan_f64(own[k]);
                s += lane_f64(sum[k], 63);
            }
            if (edge) {
                ve[0] = pow2_held(a.edge, z);
                edges = wave_scan_f64(ve[0]);
                s += lane_f64(edges, 63);
            }
            const typename Elem<DT>::T* row = logits + i * z.stride;
            if (!above && sum_is_ordinary(s)) {
                const double target = (double)u * s, none = 0x1p-999;
                double run = 0.0;
                bool found = false;
#pragma unroll
                for (int k = 0; k < LIVE; ++k) {
                    const double behind = run + lane_f64(sum[k], 63);
                    if (!found && (behind > target || k == LIVE - 1)) {
                        int last = -1;
                        const int hit = pick_scanned<E>(v[k], own[k], sum[k], run, target, lane, last, none);
                        t = hit >= 0 ? hit + k * 64 * E : last >= 0 ? last + k * 64 * E : t;
                        found = hit >= 0;
                    }
                    run = behind;
                }
                if (!found && edge) {
                    int last = -1;
                    const int hit = pick_scanned<1>(ve, ve[0], edges, run, target, lane, last, none);
                    t = hit >= 0 ? hit + z.V - z.V % E : last >= 0 ? last + z.V - z.V % E : t;
                }
                lp = t >= 0 ? row_logp((float)row[t], {s, 0.0f, 0.0f}, z) : 0.0f;
            } else {
                const RowSum r = seg_sum_any<DT>(a, z.c);
                if (r.s > 0.0) {
                    const double target = (double)u * r.s;
                    t = pick_entry<DT>(row, [&](float x, int) { return pow2_any((double)x - (double)r.m, z.c); }, {0, 0.0}, z.V,
                                       target, lane);
                }
                lp = t >= 0 ? row_logp((float)row[t], r, z) : no_token(r);
            }
        }
        if (lane == 0) {
            token[i] = t;
            logp[i] = lp;
        }
        if (next >= N) break;
        i = next;
        u = u_next;
        a = b;
    }
}

// Rows of a wave each (WAVES = 1) or a workgroup of WG threads each.
template <int DT, int WG, int WAVES>
__global__ __launch_bounds__(WG) void k_token_sample(const typename Elem<DT>::T* __restrict__ logits, int64_t N,
                                                     const float* __restrict__ uniform, RowArg z,
                                                     int64_t* __restrict__ token, float* __restrict__ logp)
{
    typedef typename Elem<DT>::T T;
    constexpr int ROWS = WG / 64 / WAVES;
    __shared__ RowSum seg[ROWS][kLdsSegs / ROWS];
    __shared__ PickShared shared;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int sub = WAVES == 1 ? wave : 0, w0 = WAVES == 1 ? 0 : wave;
    for (int64_t i = (int64_t)blockIdx.x * ROWS + sub; i < N; i += (int64_t)gridDim.x * ROWS) {
        const float u = uniform[i];
        if (!in_unit(u)) {
            if (lane == 0 && w0 == 0) {
                token[i] = -1;
                logp[i] = 0.0f;
            }
            continue;
        }
        const T* row = logits + i * z.stride;
        for (int s = w0; s < z.nseg; s += WAVES) {
            const RowSum a = seg_sum<DT>(seg_load<DT>(row, s, z.V, lane), seg_live<DT>(s, z.V), z);
            if (lane == 0) seg[sub][s] = a;
        }
        if (WAVES > 1)
            __syncthreads();
        else
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        draw_token<DT, (WAVES > 1)>(row, seg[sub], row_sum(seg[sub], z.nseg, z.c, lane), u, z, &shared, token + i, logp + i);
        if (WAVES > 1) __syncthreads();
    }
}

// A segment's sum by one wave, to its place.
template <int DT>
__device__ __forceinline__ void sum_segment(const typename Elem<DT>::T* row, int g, const RowArg& z, int lane, RowSum* out)
{
    const RowSum r = seg_sum<DT>(seg_load<DT>(row, g, z.V, lane), seg_live<DT>(g, z.V), z);
    if (lane == 0) out[g] = r;
}

// Sums of the segments of two groups of rows (those of b behind those of a), a wave
// each; rows of a whose uniform number says that they take no part are left out.
template <int DT>
__global__ __launch_bounds__(kRowsWG) void k_row_segments(const typename Elem<DT>::T* __restrict__ a, int64_t rows_a, RowArg za,
                                                          const typename Elem<DT>::T* __restrict__ b, int64_t rows_b, RowArg zb,
                                                          const float* __restrict__ uniform, RowSum* __restrict__ out)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int g = (int)blockIdx.x * kRowsWaves + wave;
    if (g >= za.nseg) return;
    for (int64_t i = blockIdx.y; i < rows_a + rows_b; i += gridDim.y) {
        const bool first = i < rows_a;
        if (first && uniform && !in_unit(uniform[i])) continue;
        const typename Elem<DT>::T* row = first ? a + i * za.stride : b + (i - rows_a) * zb.stride;
        // (member by member: a choice between the two as they are puts them into memory)
        RowArg z = za;
        z.c = first ? za.c : zb.c;
        z.floor = first ? za.floor : zb.floor;
        z.top = first ? za.top : zb.top;
        sum_segment<DT>(row, g, z, lane, out + i * za.nseg);
    }
}

// The sums of the segments of many bfloat16 rows, by powers from a table that each of
// the workgroups, one a compute unit, makes once; rows as for k_row_segments, of one
// temperature.
__global__ __launch_bounds__(kTableWG) void k_row_table(const __bf16* __restrict__ a, uint32_t rows_a, RowArg za,
                                                        const __bf16* __restrict__ b, uint32_t rows_b, RowArg zb, uint32_t begin,
                                                        const float* __restrict__ uniform, RowSum* __restrict__ out)
{
    __shared__ double table[kTableSize];
    table_fill(table, begin, za);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t step = gridDim.x * (kTableWG / 64), nseg = (uint32_t)za.nseg, segments = (rows_a + rows_b) * nseg;
    for (uint32_t k = blockIdx.x * (kTableWG / 64) + wave; k < segments; k += step) {
        const uint32_t i = k / nseg;
        const int g = (int)(k - i * nseg);
        if (uniform && !in_unit(uniform[i])) continue;
        const __bf16* row = i < rows_a ? a + i * za.stride : b + (i - rows_a) * zb.stride;
        const RowSum r = seg_sum_table(seg_load<SF_BF16>(row, g, za.V, lane), seg_live<SF_BF16>(g, za.V), za, table, begin);
        if (lane == 0) out[k] = r;
    }
}

// Whether rows' sums go by a table: many of bfloat16, at a temperature not too far
// from 1.  (us of the sums without / with it: 128 rows of 131072, 8192 segments, 14.0 /
// 12.0; 1000 rows 82 / 52; 64 x 4 drafts of 65536, 576 rows, 27.4 / 20.4; 128 x 4 of
// 65536 50 / 32; 256 x 4 of 131072 192 / 115.)
static inline bool by_table(int32_t dtype, int64_t rows, const RowArg& z)
{
    return dtype == SF_BF16 && rows * z.nseg >= kTableSegments && rows * z.nseg < (int64_t)1 << 30 && table_begin(z.c) >= 0;
}

static int sum_by_table(const void* a, int64_t rows_a, RowArg za, const void* b, int64_t rows_b, RowArg zb, const float* uniform,
                        RowSum* out, sf_stream_t stream)
{
    if (rows_b > 0 && za.c != zb.c) {  // a table each
        const int rc = sum_by_table(a, rows_a, za, nullptr, 0, za, uniform, out, stream);
        return rc != SF_OK ? rc : sum_by_table(b, rows_b, zb, nullptr, 0, zb, nullptr, out + rows_a * za.nseg, stream);
    }
    uint32_t first = (uint32_t)rows_a, others = (uint32_t)rows_b, begin = (uint32_t)table_begin(za.c);
    int cus;
    if (device_cus(stream, &cus) != SF_OK) return SF_EHIP;
    void* args[] = {(void*)&a, (void*)&first, (void*)&za, (void*)&b, (void*)&others, (void*)&zb, (void*)&begin, (void*)&uniform, (void*)&out};
    return launch((const void*)&k_row_table, dim3(cus), dim3(kTableWG), args, 0, stream);
}

// Workgroups that a row's segments make, a wave each.
static inline unsigned segment_groups(const RowArg& z) { return (unsigned)((z.nseg + kRowsWaves - 1) / kRowsWaves); }

template <int DT>
static int sum_segments(const void* a, int64_t rows_a, RowArg za, const void* b, int64_t rows_b, RowArg zb,
                        const float* uniform, RowSum* out, sf_stream_t stream)
{
    const int64_t rows = rows_a + rows_b;
    if (by_table(DT, rows_a, za) && (rows_b == 0 || by_table(DT, rows_b, zb)))
        return sum_by_table(a, rows_a, za, b, rows_b, zb, uniform, out, stream);
    void* args[] = {(void*)&a, (void*)&rows_a, (void*)&za, (void*)&b, (void*)&rows_b, (void*)&zb, (void*)&uniform, (void*)&out};
    return launch((const void*)&k_row_segments<DT>,
                  dim3(segment_groups(za), (unsigned)(rows < 65535 ? rows : 65535)), dim3(kRowsWG), args, 0,
                  stream);
}

// Draws from rows whose segments are summed: a workgroup each.
template <int DT>
__global__ __launch_bounds__(kRowsWG) void k_token_draw(const typename Elem<DT>::T* __restrict__ logits, int64_t N,
                                                        const float* __restrict__ uniform, RowArg z,
                                                        const RowSum* __restrict__ sums, int64_t* __restrict__ token,
                                                        float* __restrict__ logp)
{
    __shared__ PickShared shared;
    for (int64_t i = blockIdx.x; i < N; i += gridDim.x) {
        const float u = uniform[i];
        if (!in_unit(u)) {
            if (threadIdx.x == 0) {
                token[i] = -1;
                logp[i] = 0.0f;
            }
            continue;
        }
        const RowSum* seg = sums + i * z.nseg;
        draw_token<DT, true>(logits + i * z.stride, seg, row_sum(seg, z.nseg, z.c, threadIdx.x & 63), u, z, &shared, token + i,
                             logp + i);
    }
}

// -- verification ------------------------------------------------------------

// What becomes of a row of a sequence.
enum {
    ROW_ACCEPT,    // the draft is taken, the next row is looked at
    ROW_RESIDUAL,  // a token is drawn from max(p - q, 0)
    ROW_OTHER,     // from p without the draft
    ROW_PLAIN,     // from p
    ROW_END        // none
};

// Sums of max(p - q, 0) below this are rounding's.
constexpr double kLeastResidual = 0x1p-30;

struct Fate {
    RowSum p, q;
    int what;
    float logp;  // of the draft, or what stands in place of one
};

template <int DT>
struct VerifyArg {
    const typename Elem<DT>::T* target;
    const typename Elem<DT>::T* drafts;  // NULL: every draft is certain
    const int64_t* draft;
    const int64_t* start;
    const float* uniform;
    int64_t D, B;
    RowArg z, zq;
    const RowSum* sums;  // [D + B][nseg], then [D][nseg] of the drafts' rows
    double* residual;    // [B][nseg]
    int64_t* accepted;
    int64_t* token;
    float* logp;
};

// A sequence's first draft and its number of drafts, held within the arrays.
__device__ __forceinline__ int64_t held(int64_t v, int64_t lo, int64_t hi) { return v < lo ? lo : v > hi ? hi : v; }

// What becomes of row k of a sequence with n drafts, by one wave.  What it reads
// is asked for before it is known to be needed: a wave waits for two answers of
// memory, not five.
template <int DT>
__device__ __forceinline__ Fate row_fate(const VerifyArg<DT>& a, int64_t b, int64_t s, int64_t n, int64_t k, int lane)
{
    const int64_t i = s + b + k;
    const int64_t d = k < n ? a.draft[s + k] : -1;
    const float u = a.uniform[i];
    const bool some = d >= 0 && d < a.z.V, has_q = some && a.drafts;
    const float x = some ? (float)a.target[i * a.z.stride + d] : 0.0f;
    const float y = has_q ? (float)a.drafts[(s + k) * a.zq.stride + d] : 0.0f;
    Fate v = {};
    v.p = row_sum(a.sums + i * a.z.nseg, a.z.nseg, a.z.c, lane);
    if (has_q) v.q = row_sum(a.sums + (a.D + a.B + s + k) * a.z.nseg, a.z.nseg, a.zq.c, lane);
    v.what = ROW_END;
    if (!in_unit(u)) return v;
    if (!(v.p.s > 0.0)) {
        v.logp = no_token(v.p);
        return v;
    }
    v.what = ROW_PLAIN;
    if (!some) return v;
    const double pd = pow2_any((double)x - (double)v.p.m, a.z.c) / v.p.s;
    double qd = 1.0;
    if (has_q) {
        if (v.q.s != v.q.s) {
            v.what = ROW_END;
            v.logp = NAN;
            return v;
        }
        qd = v.q.s > 0.0 ? pow2_any((double)y - (double)v.q.m, a.zq.c) / v.q.s : 0.0;
    }
    if ((double)u * qd < pd) {
        v.what = ROW_ACCEPT;
        v.logp = row_logp(x, v.p, a.z);
    } else if (!has_q) {
        v.what = ROW_OTHER;
    } else if (v.q.s > 0.0) {
        v.what = ROW_RESIDUAL;
    }
    return v;
}

// What the entries of a segment of residuals that hold nothing may add up to is below
// this: powers held at 2^-1000, over the sum of an ordinary row, 2^-200 at least.  A
// segment above it has an entry whose own difference is not 0.
constexpr double kNoResidual = 0x1p-700;

// max(p - q, 0) of entries.  Of two rows of ordinary logits powers are taken as they
// are; what is held at 2^-1000 counts in no sum.  (Not at temperatures so high that no
// float but -inf is that far: it would be held as itself, whose power is NaN.)
struct Residual {
    RowArg z, zq;
    double mp, mq, p_of, q_of;
    bool plain;
    __device__ Residual(const Fate& v, const RowArg& z, const RowArg& zq)
        : z(z), zq(zq), mp(v.p.m), mq(v.q.m), p_of(1.0 / v.p.s), q_of(1.0 / v.q.s),
          plain(v.p.m == 0.0f && v.q.m == 0.0f && z.floor > -INFINITY && zq.floor > -INFINITY)
    {
    }
    __device__ __forceinline__ double left(double p, double q) const { return fmax(fma(p, p_of, -(q * q_of)), 0.0); }
    __device__ __forceinline__ double operator()(float xp, float xq) const
    {
        return left(pow2_any((double)xp - mp, z.c), pow2_any((double)xq - mq, zq.c));
    }
    template <int DT>
    __device__ __forceinline__ double sum(const VecU<DT>& x, const VecU<DT>& y) const
    {
        double s = 0.0;
        if (plain) {
#pragma unroll
            for (int j = 0; j < kVec<DT>; ++j) s += left(pow2_held((float)x[j], z), pow2_held((float)y[j], zq));
        } else {
#pragma unroll 1
            for (int j = 0; j < kVec<DT>; ++j) s += (*this)((float)x[j], (float)y[j]);
        }
        return s;
    }
    // of a segment, from its lanes' sums
    __device__ __forceinline__ double segment(double s) const
    {
        s = wave_sum_f64(s);
        return s > kNoResidual ? s : 0.0;
    }
};

// Where a sequence ends, for the launch that draws its token.
struct Outcome {
    Fate v;
    int64_t at, last;  // the row of the target, and its last, with the sequence's uniform number
    int64_t draft;     // the draft refused
};

// Draws a sequence's last token by every wave of a workgroup.
template <int DT>
__device__ __forceinline__ void draw_last(const VerifyArg<DT>& a, int64_t b, const Outcome& o, PickShared& shared)
{
    typedef typename Elem<DT>::T T;
    const int lane = threadIdx.x & 63;
    const Fate& v = o.v;
    const float u = a.uniform[o.last];
    if (v.what == ROW_END || !in_unit(u)) {
        if (threadIdx.x == 0) {
            a.token[o.at] = -1;
            a.logp[o.at] = v.what == ROW_END ? v.logp : 0.0f;
        }
        return;
    }
    const T* xp = a.target + o.at * a.z.stride;
    const RowSum* seg = a.sums + o.at * a.z.nseg;
    int t = -1;
    if (v.what == ROW_RESIDUAL) {
        const double* part = a.residual + b * a.z.nseg;
        double total = 0.0;
        for (int g = lane; g < a.z.nseg; g += 64) total += part[g];
        total = wave_sum_f64(total);
        if (total >= kLeastResidual) {
            const T* xq = a.drafts + (o.at - b) * a.zq.stride;
            const Residual residual(v, a.z, a.zq);
            const double target = (double)u * total;
            const Place at = pick_weight([&](int g) { return part[g]; }, a.z.nseg, target, lane);
            t = pick_entry_group<DT>(xp, [&](float x, int j) { return residual(x, (float)xq[j]); }, at, a.z.V, target, shared);
        }
    } else if (v.what == ROW_OTHER) {
        const int d = (int)o.draft, gd = d / kSeg<DT>;
        auto value = [&](float x, int j) { return j == d ? 0.0 : pow2_any((double)x - (double)v.p.m, a.z.c); };
        const double own = entry_sum_group<DT>(xp, value, gd, a.z.V, shared);
        auto weight = [&](int g) { return g == gd ? own : seg_weight(seg[g], v.p.m, a.z.c); };
        double total = 0.0;
        for (int g = lane; g < a.z.nseg; g += 64) total += weight(g);
        total = wave_sum_f64(total);
        // (2^-24 of the row at least: what refused the draft is below 1, and no less than its share)
        const double target = (double)u * total;
        t = pick_entry_group<DT>(xp, value, pick_weight(weight, a.z.nseg, target, lane), a.z.V, target, shared);
    }
    if (t < 0) {  // from p, also where next to nothing of it is left
        draw_token<DT, true>(xp, seg, v.p, u, a.z, &shared, a.token + o.at, a.logp + o.at);
    } else if (threadIdx.x == 0) {
        a.token[o.at] = t;
        a.logp[o.at] = row_logp((float)xp[t], v.p, a.z);
    }
}

constexpr int kVerifyWG = 512;
constexpr int kVerifyWaves = kVerifyWG / 64;

// Where sequence b ends, found by a workgroup: its rows eight at a time.  One of the
// workgroups that do the same (`writes`) writes what is accepted.
template <int DT>
__device__ __forceinline__ Outcome decide(const VerifyArg<DT>& a, int64_t b, Fate (&row)[kVerifyWaves], bool writes)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t s = held(a.start[b], 0, a.D), n = held(a.start[b + 1], s, a.D) - s;
    int64_t end;
    for (int64_t k0 = 0;; k0 += kVerifyWaves) {
        const int64_t k = k0 + wave;
        Fate v = {};
        v.what = ROW_PLAIN;
        if (k <= n) v = row_fate<DT>(a, b, s, n, k, lane);
        __syncthreads();  // former ones are read
        if (lane == 0) row[wave] = v;
        __syncthreads();
        int w = 0;
        while (w < kVerifyWaves && row[w].what == ROW_ACCEPT) ++w;
        if (writes && wave < w && lane == 0) {
            a.token[s + b + k] = a.draft[s + k];
            a.logp[s + b + k] = v.logp;
        }
        end = k0 + w;
        if (w < kVerifyWaves) break;  // row n at the latest
    }
    Outcome o;
    o.v = row[end % kVerifyWaves];
    o.at = s + b + end;
    o.last = s + b + n;
    o.draft = end < n ? a.draft[s + end] : -1;
    if (writes) {
        if (threadIdx.x == 0) a.accepted[b] = end;
        for (int64_t k = end + 1 + threadIdx.x; k <= n; k += kVerifyWG) {
            a.token[s + b + k] = -1;
            a.logp[s + b + k] = 0.0f;
        }
    }
    return o;
}

// Whether the first k1 drafts of sequences are accepted, a workgroup each.
template <int DT>
__global__ __launch_bounds__(kRowsWG) void k_draft_alive(VerifyArg<DT> a, int64_t k1, Outcome* __restrict__ outcomes)
{
    __shared__ int what[kRowsWaves];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    for (int64_t b = blockIdx.x; b < a.B; b += gridDim.x) {
        const int64_t s = held(a.start[b], 0, a.D), n = held(a.start[b + 1], s, a.D) - s;
        bool alive = n >= k1;
        for (int64_t k = wave; alive && k - wave < k1; k += kRowsWaves) {
            const int is = k < k1 ? row_fate<DT>(a, b, s, n, k, lane).what : ROW_ACCEPT;
            __syncthreads();  // former ones are read
            if (lane == 0) what[wave] = is;
            __syncthreads();
            for (int w = 0; w < kRowsWaves; ++w) alive &= what[w] == ROW_ACCEPT;
        }
        if (threadIdx.x == 0) outcomes[b].v.what = alive ? ROW_ACCEPT : ROW_END;
        __syncthreads();
    }
}

// Sums of segments of the rows k0 .. k1 - 1 of every sequence, a wave the same
// segments of every gridDim.z-th of them.  With k0 > 0 only of sequences that are alive: rows
// behind a refused draft are not read.
template <int DT>
__global__ __launch_bounds__(kRowsWG) void k_draft_segments(VerifyArg<DT> a, int64_t k0, int64_t k1,
                                                            const Outcome* __restrict__ outcomes, RowSum* __restrict__ sums)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int g = (int)blockIdx.x * kRowsWaves + wave;
    if (g >= a.z.nseg) return;
    for (int64_t b = blockIdx.y; b < a.B; b += gridDim.y) {
        if (k0 > 0 && outcomes[b].v.what != ROW_ACCEPT) continue;
        const int64_t s = held(a.start[b], 0, a.D), n = held(a.start[b + 1], s, a.D) - s;
        const int64_t end = n + 1 < k1 ? n + 1 : k1;
        // rows of the target and the drafts in turn, by one piece of code
        const int kinds = a.drafts ? 2 : 1;
        for (int64_t j = kinds * k0 + blockIdx.z; j < kinds * end; j += gridDim.z) {
            const int64_t k = kinds == 2 ? j / 2 : j;
            const bool drafts = kinds == 2 && (j & 1);
            if (drafts && k == n) continue;
            const int64_t i = drafts ? s + k : s + b + k;
            const RowArg& z = drafts ? a.zq : a.z;
            sum_segment<DT>((drafts ? a.drafts : a.target) + i * z.stride, g, z, lane,
                            sums + (i + (drafts ? a.D + a.B : 0)) * z.nseg);
        }
    }
}

// Decides sequences, and (DRAW) draws their last tokens where no residual's sums
// are needed for it.  Bound by waiting: the starts, then drafts and uniform numbers,
// then the logits that these name, each an answer of memory (256 sequences: 5.2 us).
template <int DT, bool DRAW>
__global__ __launch_bounds__(kVerifyWG) void k_draft_decide(VerifyArg<DT> a, Outcome* __restrict__ outcomes)
{
    __shared__ Fate row[kVerifyWaves];
    __shared__ PickShared shared;
    for (int64_t b = blockIdx.x; b < a.B; b += gridDim.x) {
        const Outcome o = decide<DT>(a, b, row, true);
        if (DRAW)
            draw_last<DT>(a, b, o, shared);
        else if (threadIdx.x == 0)
            outcomes[b] = o;
    }
}

// Where there are few segments: decides a sequence in every workgroup of it, which
// then takes two segments of its residual, four waves each: a launch less.  (us under
// replay in three launches / in four: 4 x 4 drafts of 131072, 256 segments, 15.7 / 18.5;
// 64 x 4 of 32003, 1024 segments, 25.7 / 27.1; 61 x 8 of 32003 f32, 1952 segments, 40.9 /
// 36.2; 64 x 4 of 131072, 4096 segments, 56 / 50.)
template <int DT>
__global__ __launch_bounds__(kVerifyWG) void k_draft_few(VerifyArg<DT> a, Outcome* __restrict__ outcomes)
{
    constexpr int E = kVec<DT>;
    __shared__ Fate row[kVerifyWaves];
    __shared__ double part[kVerifyWaves][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int g = (int)blockIdx.x * (kVerifyWaves / kSegU) + wave / kSegU, k = wave % kSegU;
    const int at = g * kSeg<DT> + (k * 64 + lane) * E, tail = a.z.V - a.z.V % E + lane;
    for (int64_t b = blockIdx.y; b < a.B; b += gridDim.y) {
        const Outcome o = decide<DT>(a, b, row, blockIdx.x == 0);
        if (blockIdx.x == 0 && threadIdx.x == 0) outcomes[b] = o;
        if (o.v.what != ROW_RESIDUAL) continue;
        const typename Elem<DT>::T* xp = a.target + o.at * a.z.stride;
        const typename Elem<DT>::T* xq = a.drafts + (o.at - b) * a.zq.stride;
        const Residual residual(o.v, a.z, a.zq);
        double sum = 0.0;
        if (at + E <= a.z.V) sum = residual.template sum<DT>(*(const VecU<DT>*)(xp + at), *(const VecU<DT>*)(xq + at));
        part[wave][lane] = sum;  // (a former sequence's are read: decide waits)
        __syncthreads();
        if (k == 0 && g < a.z.nseg) {
            sum = g == a.z.nseg - 1 && tail < a.z.V ? residual((float)xp[tail], (float)xq[tail]) : 0.0;
            for (int i = 0; i < kSegU; ++i) sum += part[wave + i][lane];
            sum = residual.segment(sum);
            if (lane == 0) a.residual[b * a.z.nseg + g] = sum;
        }
    }
}

// The sums of the residuals' segments of sequences that are decided, a wave each.
// (146 of 256 sequences refused, 131072 entries: 33 us, two powers an entry.)
template <int DT>
__global__ __launch_bounds__(kRowsWG) void k_draft_residual(VerifyArg<DT> a, const Outcome* __restrict__ outcomes)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int g = (int)blockIdx.x * kRowsWaves + wave;
    if (g >= a.z.nseg) return;
    for (int64_t b = blockIdx.y; b < a.B; b += gridDim.y) {
        const Outcome& o = outcomes[b];
        if (o.v.what != ROW_RESIDUAL) continue;
        const SegData<DT> x = seg_load<DT>(a.target + o.at * a.z.stride, g, a.z.V, lane);
        const SegData<DT> y = seg_load<DT>(a.drafts + (o.at - b) * a.zq.stride, g, a.z.V, lane);
        const Residual residual(o.v, a.z, a.zq);
        double sum = __any(x.edge != -INFINITY) ? residual(x.edge, y.edge) : 0.0;
        const int live = seg_live<DT>(g, a.z.V);
#pragma unroll
        for (int k = 0; k < kSegU; ++k)
            if (k < live) sum += residual.template sum<DT>(x.y[k], y.y[k]);
        sum = residual.segment(sum);
        if (lane == 0) a.residual[b * a.z.nseg + g] = sum;
    }
}

// The same by a table, where both temperatures are the same.  (26 us in place of 33.)
__global__ __launch_bounds__(kTableWG) void k_residual_table(VerifyArg<SF_BF16> a, uint32_t begin, const Outcome* __restrict__ outcomes)
{
    constexpr int E = kVec<SF_BF16>;
    __shared__ double table[kTableSize];
    table_fill(table, begin, a.z);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t step = gridDim.x * (kTableWG / 64), nseg = (uint32_t)a.z.nseg, all = (uint32_t)a.B * nseg;
    for (uint32_t u = blockIdx.x * (kTableWG / 64) + wave; u < all; u += step) {
        const int64_t b = u / nseg;
        const Outcome& o = outcomes[b];
        if (o.v.what != ROW_RESIDUAL) continue;
        const int g = (int)(u - (uint32_t)b * nseg), live = seg_live<SF_BF16>(g, a.z.V);
        const SegData<SF_BF16> x = seg_load<SF_BF16>(a.target + o.at * a.z.stride, g, a.z.V, lane);
        const SegData<SF_BF16> y = seg_load<SF_BF16>(a.drafts + (o.at - b) * a.zq.stride, g, a.z.V, lane);
        const Residual residual(o.v, a.z, a.zq);
        double sum = __any(x.edge != -INFINITY) ? residual(x.edge, y.edge) : 0.0;
#pragma unroll
        for (int k = 0; k < kSegU; ++k) {
            if (k >= live) break;
            if (!residual.plain) {
                sum += residual.template sum<SF_BF16>(x.y[k], y.y[k]);
                continue;
            }
            const Words4 p = __builtin_bit_cast(Words4, (VecU<SF_BF16>)x.y[k]), q = __builtin_bit_cast(Words4, (VecU<SF_BF16>)y.y[k]);
            double own = 0.0;
#pragma unroll
            for (int j = 0; j < E / 2; ++j) {
                const Two at = table_places(p[j], begin), to = table_places(q[j], begin);
                own += residual.left(table[at[0]], table[to[0]]);
                own += residual.left(table[at[1]], table[to[1]]);
            }
            sum += own;
        }
        sum = residual.segment(sum);
        if (lane == 0) a.residual[b * a.z.nseg + g] = sum;
    }
}

// Draws the last tokens of sequences whose residuals were summed by parts: a
// workgroup each.
template <int DT>
__global__ __launch_bounds__(kRowsWG) void k_draft_draw(VerifyArg<DT> a, const Outcome* __restrict__ outcomes)
{
    __shared__ PickShared shared;
    for (int64_t b = blockIdx.x; b < a.B; b += gridDim.x) draw_last<DT>(a, b, outcomes[b], shared);
}

static inline bool rows_ok(int32_t dtype, int64_t N, int64_t V, int64_t stride, float inv_t)
{
    return (dtype == SF_F32 || dtype == SF_BF16 || dtype == SF_F16) && N >= 0 && V >= 1 &&
           V <= ((int64_t)1 << 30) && stride >= V && inv_t > 0.0f && inv_t <= 0x1p100f &&
           (N == 0 || stride <= (((int64_t)1 << 56) / N));
}

static inline RowArg row_arg(int32_t dtype, int64_t V, int64_t stride, float inv_t)
{
    const double c = (double)inv_t * kLog2eD, far = 1000.0 / c;
    const float limit = far < 3.4e38 ? (float)far : INFINITY;
    return {stride, (int)V, (int)seg_count(dtype, V), c, inv_t, -limit, limit};
}

// Vectors a lane of a row of one segment.
static inline int seg_live(int dtype, int64_t V)
{
    const int step = dtype == SF_F32 ? 64 * kVec<SF_F32> : 64 * kVec<SF_BF16>;
    return (int)((V - V % (step / 64) + step - 1) / step);
}

static inline unsigned up_to(int64_t n, int64_t most) { return (unsigned)(n < most ? n : most); }

// Threads that a row has to itself: 64, kRowsWG or 1024, or 0 where rows are split
// over workgroups, which costs a second launch.  Measured (f16, us under replay, 64 /
// 256 / 1024 / split):
//   1 x 20000: 17.5 / 8.7 / 8.1 / 7.7;  1 x 50001: 36 / 13.9 / 11.5 / 7.8, but in a
//   queue of calls, where a launch and a workspace cost the host 3 us, - / - / 10.8 /
//   13.3;  200 x 32768: 28 / 10.8 / 10.0 / 12.8;  64 x 131072: 97 / 30 / 23 / 13.6;
//   400 x 65536: 56 / 28 / 29 / 27;  512 x 131072: 111 / 52 / 53 / 53;
//   600 x 8000: 13.6 / 10.1 / 17.5 / 13.0;  1024 x 32768: 35 / 27 / 38 / 33;
//   2048 x 32768: 58 / 52 / 75 / 63;  4096 x 8000: 34 / 36 / 90 / 44;
//   4096 x 16384: 54 / 58 / 98 / 67;  8000 x 32768: 181 / 186 / 288 / 203.
// Many bfloat16 rows are split for the table's sake (by_table); short ones have more
// to draw than to sum.
static inline int sample_threads(int32_t dtype, int64_t N, int64_t nseg)
{
    if (dtype == SF_BF16 && nseg >= 16 && N * nseg >= kTableSegments) return 0;
    if (nseg == 1 || (N >= 4096 && nseg <= kLdsSegs / kRowsWaves)) return 64;
    if (N >= 512) return nseg <= kLdsSegs ? kRowsWG : 0;
    return nseg <= 32 ? 1024 : 0;
}

}  // namespace sfk

using namespace sfk;

SF_API int64_t sf_token_sample_workspace(int32_t dtype, int64_t N, int64_t V)
{
    if (!rows_ok(dtype, N, V, V, 1.0f)) return -1;
    const int64_t nseg = seg_count(dtype, V);
    return N == 0 || sample_threads(dtype, N, nseg) ? 0 : N * nseg * (int64_t)sizeof(RowSum);
}

SF_API int sf_token_sample(const void* logits, int32_t dtype, int64_t N, int64_t V, int64_t row_stride,
                           const float* uniform, float inv_temperature, int64_t* out_token, float* out_logp,
                           void* workspace, int64_t workspace_bytes, sf_stream_t stream)
{
    if (!rows_ok(dtype, N, V, row_stride, inv_temperature)) return SF_EINVAL;
    if (N == 0) return SF_OK;
    const int64_t need = sf_token_sample_workspace(dtype, N, V);
    if (!logits || !uniform || !out_token || !out_logp || (need > 0 && !workspace) || workspace_bytes < need)
        return SF_EINVAL;
    if (!aligned(logits, elem_size(dtype)) || !aligned(uniform, 4) || !aligned(out_token, 8) || !aligned(out_logp, 4) ||
        (need > 0 && !aligned(workspace, 16)))
        return SF_EINVAL;
    const int64_t in_bytes = ((N - 1) * row_stride + V) * elem_size(dtype);
    const void* outs[3] = {out_token, out_logp, workspace};
    const int64_t sizes[3] = {N * 8, N * 4, need};
    for (int i = 0; i < 3; ++i) {
        if (sizes[i] == 0) continue;
        if (!disjoint(outs[i], sizes[i], logits, in_bytes) || !disjoint(outs[i], sizes[i], uniform, N * 4)) return SF_EINVAL;
        for (int j = i + 1; j < 3; ++j)
            if (sizes[j] > 0 && !disjoint(outs[i], sizes[i], outs[j], sizes[j])) return SF_EINVAL;
    }
    RowArg z = row_arg(dtype, V, row_stride, inv_temperature);
    const int threads = sample_threads(dtype, N, z.nseg);
    void* args[] = {(void*)&logits, (void*)&N, (void*)&uniform, (void*)&z, (void*)&out_token, (void*)&out_logp};
    if (z.nseg == 1) {
        const int live = seg_live(dtype, V);
        const void* fn[3][3] = {
            {(const void*)&k_token_short<SF_F32, 1>, (const void*)&k_token_short<SF_BF16, 1>, (const void*)&k_token_short<SF_F16, 1>},
            {(const void*)&k_token_short<SF_F32, 2>, (const void*)&k_token_short<SF_BF16, 2>, (const void*)&k_token_short<SF_F16, 2>},
            {(const void*)&k_token_short<SF_F32, 4>, (const void*)&k_token_short<SF_BF16, 4>, (const void*)&k_token_short<SF_F16, 4>}};
        return launch(fn[live <= 1 ? 0 : live == 2 ? 1 : 2][dtype], dim3(up_to((N + kRowsWaves - 1) / kRowsWaves, 2048)),
                      dim3(kRowsWG), args, 0, stream);
    }
    if (threads) {
        const void* fn[3][3] = {{(const void*)&k_token_sample<SF_F32, kRowsWG, 1>, (const void*)&k_token_sample<SF_BF16, kRowsWG, 1>,
                                 (const void*)&k_token_sample<SF_F16, kRowsWG, 1>},
                                {(const void*)&k_token_sample<SF_F32, kRowsWG, 4>, (const void*)&k_token_sample<SF_BF16, kRowsWG, 4>,
                                 (const void*)&k_token_sample<SF_F16, kRowsWG, 4>},
                                {(const void*)&k_token_sample<SF_F32, 1024, 16>, (const void*)&k_token_sample<SF_BF16, 1024, 16>,
                                 (const void*)&k_token_sample<SF_F16, 1024, 16>}};
        const int wg = threads == 64 ? kRowsWG : threads, rows = wg / threads;
        return launch(fn[threads == 64 ? 0 : threads == kRowsWG ? 1 : 2][dtype], dim3(up_to((N + rows - 1) / rows, 1 << 21)),
                      dim3(wg), args, 0, stream);
    }
    auto sums = dtype == SF_F32 ? sum_segments<SF_F32> : dtype == SF_BF16 ? sum_segments<SF_BF16> : sum_segments<SF_F16>;
    const int rc = sums(logits, N, z, nullptr, 0, z, uniform, (RowSum*)workspace, stream);
    if (rc != SF_OK) return rc;
    void* draw_args[] = {(void*)&logits, (void*)&N, (void*)&uniform, (void*)&z, (void*)&workspace, (void*)&out_token,
                         (void*)&out_logp};
    const void* draw[3] = {(const void*)&k_token_draw<SF_F32>, (const void*)&k_token_draw<SF_BF16>,
                           (const void*)&k_token_draw<SF_F16>};
    return launch(draw[dtype], dim3(up_to(N, 1 << 21)), dim3(kRowsWG), draw_args, 0, stream);
}

// The workspace: the segments' sums of the target's rows and of the drafts', the
// residuals' sums, and the outcomes.
static inline int64_t verify_sums(int64_t D, int64_t B, int64_t nseg) { return (2 * D + B) * nseg * (int64_t)sizeof(RowSum); }
static inline int64_t verify_residuals(int64_t B, int64_t nseg) { return (B * nseg * 8 + 15) / 16 * 16; }

SF_API int64_t sf_draft_verify_workspace(int32_t dtype, int64_t D, int64_t B, int64_t V)
{
    constexpr int64_t most = (int64_t)1 << 31;
    if (D < 0 || D >= most || B < 0 || B >= most || !rows_ok(dtype, D, V, V, 1.0f)) return -1;
    if (B == 0) return 0;
    const int64_t nseg = seg_count(dtype, V);
    return verify_sums(D, B, nseg) + verify_residuals(B, nseg) + B * (int64_t)sizeof(Outcome);
}

namespace sfk {

template <int DT>
static int verify(const void* target, const void* drafts, int64_t D, int64_t B, RowArg z, RowArg zq, const int64_t* draft,
                  const int64_t* start, const float* uniform, int64_t* accepted, int64_t* token, float* logp,
                  void* workspace, sf_stream_t stream)
{
    typedef typename Elem<DT>::T T;
    char* ws = (char*)workspace;
    RowSum* sums = (RowSum*)ws;
    double* residual = (double*)(ws + verify_sums(D, B, z.nseg));
    Outcome* outcomes = (Outcome*)(ws + verify_sums(D, B, z.nseg) + verify_residuals(B, z.nseg));
    const int64_t rows = D + B, more = drafts ? D : 0;
    VerifyArg<DT> a = {(const T*)target, (const T*)drafts, draft, start, uniform, D, B, z, zq, sums, residual, accepted, token, logp};
    int rc;
    if (D >= 2 * B && !(drafts && by_table(DT, D, zq)) && (rows + more) * z.nseg > (drafts ? kManySegments : kManySegments / 4)) {
        // The first rows, then those behind accepted drafts, which costs two launches of
        // 5 us.  (f16, us with the first 1 / 2 / 3 rows / all at once: 256 x 4 drafts of
        // 131072, 79% accepted, 230 / 224 / 233 / 245; 128 x 4 125 / 125 / 130 / 133; 64 x 4
        // 78 / 76 / 76 / 77; 200 x 9 without logits of 50001, 12% accepted, 36 / 40 / 38 / 56.
        // By a table, all at once, 256 x 4 bf16 take 140, and 156 in two rounds.)  How many
        // will be accepted is not known to the host, and rounds pay where it is few: us in
        // rounds / all at once under replay, f16, 256 x 4 drafts of 131072, 15% accepted 191 /
        // 259, 38% 200 / 246, 58% 208 / 239, 86% 222 / 221, all 221 / 203; 200 x 0 to 9 without
        // logits of 50001, 2% 34 / 49, 14% 44 / 54, 38% 51 / 47, 68% 58 / 48, all 56 / 45.
        int64_t k0 = 0, k1 = drafts ? 1 + D / B / 3 : 1, all = (int64_t)1 << 31;
        const int64_t kinds = drafts ? 2 : 1, rest = kinds * (D / B - k1 + 1);
        void* first[] = {(void*)&a, (void*)&k0, (void*)&k1, (void*)&outcomes, (void*)&sums};
        void* alive[] = {(void*)&a, (void*)&k1, (void*)&outcomes};
        void* others[] = {(void*)&a, (void*)&k1, (void*)&all, (void*)&outcomes, (void*)&sums};
        const unsigned gx = segment_groups(z), gy = up_to(B, 65535);
        rc = launch((const void*)&k_draft_segments<DT>, dim3(gx, gy, up_to(kinds * k1, 64)), dim3(kRowsWG), first, 0, stream);
        if (rc != SF_OK) return rc;
        rc = launch((const void*)&k_draft_alive<DT>, dim3(up_to(B, 1 << 21)), dim3(kRowsWG), alive, 0, stream);
        if (rc != SF_OK) return rc;
        rc = launch((const void*)&k_draft_segments<DT>, dim3(gx, gy, up_to(rest, 6)), dim3(kRowsWG), others, 0, stream);
    } else {
        rc = sum_segments<DT>(target, rows, z, drafts, more, zq, nullptr, sums, stream);
    }
    if (rc != SF_OK) return rc;
    void* args[] = {(void*)&a, (void*)&outcomes};
    const dim3 draws(up_to(B, 1 << 21));
    if (!drafts)
        return launch((const void*)&k_draft_decide<DT, true>, draws, dim3(kVerifyWG), args, 0, stream);
    if (B * z.nseg <= kFewSegments) {
        constexpr int each = kVerifyWaves / kSegU;
        rc = launch((const void*)&k_draft_few<DT>, dim3((z.nseg + each - 1) / each, up_to(B, 65535)), dim3(kVerifyWG), args, 0,
                    stream);
    } else {
        rc = launch((const void*)&k_draft_decide<DT, false>, draws, dim3(kVerifyWG), args, 0, stream);
        if (rc != SF_OK) return rc;
        if (z.c == zq.c && by_table(DT, B, z)) {
            uint32_t begin = (uint32_t)table_begin(z.c);
            int cus;
            if (device_cus(stream, &cus) != SF_OK) return SF_EHIP;
            void* by_args[] = {(void*)&a, (void*)&begin, (void*)&outcomes};
            rc = launch((const void*)&k_residual_table, dim3(cus), dim3(kTableWG), by_args, 0, stream);
        } else {
            rc = launch((const void*)&k_draft_residual<DT>, dim3(segment_groups(z), up_to(B, 65535)), dim3(kRowsWG), args, 0, stream);
        }
    }
    if (rc != SF_OK) return rc;
    return launch((const void*)&k_draft_draw<DT>, draws, dim3(kRowsWG), args, 0, stream);
}

}  // namespace sfk

SF_API int sf_draft_verify(const void* target_logits, const void* draft_logits, int32_t dtype, int64_t D, int64_t B,
                           int64_t V, int64_t target_stride, int64_t draft_stride, const int64_t* draft,
                           const int64_t* seq_start, const float* uniform, float inv_temperature,
                           float draft_inv_temperature, int64_t* out_accepted, int64_t* out_token, float* out_logp,
                           void* workspace, int64_t workspace_bytes, sf_stream_t stream)
{
    const int64_t need = sf_draft_verify_workspace(dtype, D, B, V);
    if (need < 0 || !rows_ok(dtype, D + B, V, target_stride, inv_temperature)) return SF_EINVAL;
    if (!draft_logits) {
        draft_stride = V;
        draft_inv_temperature = 1.0f;
    }
    if (!rows_ok(dtype, D, V, draft_stride, draft_inv_temperature)) return SF_EINVAL;
    if (B == 0) return SF_OK;
    if (!target_logits || !seq_start || !uniform || !out_accepted || !out_token || !out_logp || !workspace ||
        workspace_bytes < need || (D > 0 && !draft))
        return SF_EINVAL;
    const int e = elem_size(dtype);
    if (!aligned(target_logits, e) || !aligned(draft_logits, e) || !aligned(draft, 8) || !aligned(seq_start, 8) ||
        !aligned(uniform, 4) || !aligned(out_accepted, 8) || !aligned(out_token, 8) || !aligned(out_logp, 4) ||
        !aligned(workspace, 16))
        return SF_EINVAL;
    const int64_t rows = D + B;
    const void* ins[5] = {target_logits, draft_logits, draft, seq_start, uniform};
    const int64_t in_sizes[5] = {((rows - 1) * target_stride + V) * e,
                                 draft_logits && D > 0 ? ((D - 1) * draft_stride + V) * e : 0, D * 8, (B + 1) * 8, rows * 4};
    const void* outs[4] = {out_accepted, out_token, out_logp, workspace};
    const int64_t out_sizes[4] = {B * 8, rows * 8, rows * 4, need};
    for (int i = 0; i < 4; ++i) {
        for (int j = 0; j < 5; ++j)
            if (in_sizes[j] > 0 && !disjoint(outs[i], out_sizes[i], ins[j], in_sizes[j])) return SF_EINVAL;
        for (int j = i + 1; j < 4; ++j)
            if (!disjoint(outs[i], out_sizes[i], outs[j], out_sizes[j])) return SF_EINVAL;
    }
    RowArg z = row_arg(dtype, V, target_stride, inv_temperature), zq = row_arg(dtype, V, draft_stride, draft_inv_temperature);
    auto fn = dtype == SF_F32 ? verify<SF_F32> : dtype == SF_BF16 ? verify<SF_BF16> : verify<SF_F16>;
    return fn(target_logits, draft_logits, D, B, z, zq, draft, seq_start, uniform, out_accepted, out_token, out_logp,
              workspace, stream);
}
