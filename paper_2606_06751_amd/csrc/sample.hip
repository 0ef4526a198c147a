// sample.hip -- a token of each row of logits by given uniform numbers
// (sf_token_sample), and the verification of drafted tokens (sf_draft_verify).
//
// Tokens are whole numbers, so they are either the definition's or wrong: every
// sum and comparison that decides one is in 64 bits, whose vector rate on this
// chip is that of 32 bits.  A row is summed by segments (sf_draw.h), whose sums
// give the normaliser and, in order, the cumulative sums at the segments' ends;
// the segment that the uniform number falls into is read again for its entry.

#include "sf_draw.h"
#include "sf_host.h"

namespace sfk {

constexpr int kRowsWG = 256;
constexpr int kRowsWaves = kRowsWG / 64;
constexpr int kLdsSegs = 1024;  // of a row that one workgroup takes

struct RowArg {
    int64_t stride;
    int V, nseg;
    double c;
    float inv_t;
};

__device__ __forceinline__ bool in_unit(float u) { return u >= 0.0f && u < 1.0f; }

// Draws a row's token by one wave from its segments' sums.
template <int DT>
__device__ __forceinline__ void draw_token(const typename Elem<DT>::T* row, const RowSum* seg, const RowSum& r, double u,
                                           RowArg z, int lane, int64_t* token, float* logp)
{
    int t = -1;
    if (r.s > 0.0) {
        const double target = u * r.s;
        const Place at = pick_weight([&](int i) { return seg_weight(seg[i], r.m, z.c); }, z.nseg, target, lane);
        const double m = r.m;
        t = pick_entry<DT>([&](int j) { return pow2_any((double)(float)row[j] - m, z.c); }, at.i, z.V, at.base, target, lane);
    }
    if (lane == 0) {
        *token = t;
        *logp = t >= 0 ? row_logp((float)row[t], r, z.inv_t) : r.s == 0.0 ? -INFINITY : NAN;
    }
}

// Rows of a wave each (WAVES = 1) or a workgroup each.
template <int DT, int WAVES>
__global__ __launch_bounds__(kRowsWG) void k_token_sample(const typename Elem<DT>::T* __restrict__ logits, int64_t N,
                                                          const float* __restrict__ uniform, RowArg z,
                                                          int64_t* __restrict__ token, float* __restrict__ logp)
{
    typedef typename Elem<DT>::T T;
    constexpr int ROWS = kRowsWaves / WAVES;
    __shared__ RowSum seg[ROWS][kLdsSegs / ROWS];
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
            const RowSum a = seg_sum<DT>(seg_load<DT>(row, s, z.V, lane), z.c);
            if (lane == 0) seg[sub][s] = a;
        }
        if (WAVES > 1)
            __syncthreads();
        else
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (w0 == 0)
            draw_token<DT>(row, seg[sub], row_sum(seg[sub], z.nseg, z.c, lane), u, z, lane, token + i, logp + i);
        if (WAVES > 1) __syncthreads();
    }
}

// Sums of the segments of two groups of rows (those of b behind those of a), each
// wave `per` neighbouring segments; rows of a whose uniform number says that they
// take no part are left out.
template <int DT>
__global__ __launch_bounds__(kRowsWG) void k_row_segments(const typename Elem<DT>::T* __restrict__ a, int64_t rows_a, RowArg za,
                                                          const typename Elem<DT>::T* __restrict__ b, int64_t rows_b, RowArg zb,
                                                          const float* __restrict__ uniform, int per, RowSum* __restrict__ out)
{
    typedef typename Elem<DT>::T T;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int s0 = ((int)blockIdx.x * kRowsWaves + wave) * per;
    const int s1 = min(s0 + per, za.nseg);
    for (int64_t i = blockIdx.y; i < rows_a + rows_b; i += gridDim.y) {
        const bool first = i < rows_a;
        if (first && uniform && !in_unit(uniform[i])) continue;
        const T* row = first ? a + i * za.stride : b + (i - rows_a) * zb.stride;
        const double c = first ? za.c : zb.c;
        for (int s = s0; s < s1; ++s) {
            const RowSum r = seg_sum<DT>(seg_load<DT>(row, s, za.V, lane), c);
            if (lane == 0) out[i * za.nseg + s] = r;
        }
    }
}

// Draws from rows whose segments are summed: a wave each.
template <int DT>
__global__ __launch_bounds__(kRowsWG) void k_token_draw(const typename Elem<DT>::T* __restrict__ logits, int64_t N,
                                                        const float* __restrict__ uniform, RowArg z,
                                                        const RowSum* __restrict__ sums, int64_t* __restrict__ token,
                                                        float* __restrict__ logp)
{
    const int lane = threadIdx.x & 63;
    for (int64_t i = (int64_t)blockIdx.x * kRowsWaves + (threadIdx.x >> 6); i < N; i += (int64_t)gridDim.x * kRowsWaves) {
        const float u = uniform[i];
        if (!in_unit(u)) {
            if (lane == 0) {
                token[i] = -1;
                logp[i] = 0.0f;
            }
            continue;
        }
        const RowSum* seg = sums + i * z.nseg;
        draw_token<DT>(logits + i * z.stride, seg, row_sum(seg, z.nseg, z.c, lane), u, z, lane, token + i, logp + i);
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

struct Verdict {
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

// What becomes of row k of a sequence with n drafts, by one wave.
template <int DT>
__device__ __forceinline__ Verdict row_verdict(const VerifyArg<DT>& a, int64_t b, int64_t s, int64_t n, int64_t k, int lane)
{
    const int64_t i = s + b + k;
    const float u = a.uniform[i];
    Verdict v = {};
    v.what = ROW_END;
    if (!in_unit(u)) return v;
    v.p = row_sum(a.sums + i * a.z.nseg, a.z.nseg, a.z.c, lane);
    if (!(v.p.s > 0.0)) {
        v.logp = v.p.s == 0.0 ? -INFINITY : NAN;
        return v;
    }
    v.what = ROW_PLAIN;
    if (k == n) return v;
    const int64_t d = a.draft[s + k];
    if (d < 0 || d >= a.z.V) return v;
    const float x = (float)a.target[i * a.z.stride + d];
    const double pd = pow2_any((double)x - (double)v.p.m, a.z.c) / v.p.s;
    double qd = 1.0;
    if (a.drafts) {
        v.q = row_sum(a.sums + (a.D + a.B + s + k) * a.z.nseg, a.z.nseg, a.zq.c, lane);
        if (v.q.s != v.q.s) {
            v.what = ROW_END;
            v.logp = NAN;
            return v;
        }
        if (v.q.s == 0.0)
            qd = 0.0;
        else
            qd = pow2_any((double)(float)a.drafts[(s + k) * a.zq.stride + d] - (double)v.q.m, a.zq.c) / v.q.s;
    }
    if ((double)u * qd < pd) {
        v.what = ROW_ACCEPT;
        v.logp = row_logp(x, v.p, a.z.inv_t);
    } else if (!a.drafts) {
        v.what = ROW_OTHER;
    } else if (v.q.s > 0.0) {
        v.what = ROW_RESIDUAL;
    }
    return v;
}

template <int DT>
__device__ __forceinline__ double entry_residual(float xp, float xq, const Verdict& v, double p_of, double q_of, RowArg z,
                                                 RowArg zq)
{
#pragma clang fp contract(off)  // equal rows leave nothing
    const double p = pow2_any((double)xp - (double)v.p.m, z.c) * p_of;
    const double q = pow2_any((double)xq - (double)v.q.m, zq.c) * q_of;
    return p > q ? p - q : 0.0;
}

// Where a sequence ends, for the launch that draws its token.
struct Outcome {
    Verdict v;
    int64_t at, last;  // the row of the target, and its last, with the sequence's uniform number
    int64_t draft;     // the draft refused
};

// Draws a sequence's last token by one wave.
template <int DT>
__device__ __forceinline__ void draw_last(const VerifyArg<DT>& a, int64_t b, const Outcome& o, int lane)
{
    typedef typename Elem<DT>::T T;
    const Verdict& v = o.v;
    const double u = a.uniform[o.last];
    const bool drawn = v.what != ROW_END && in_unit((float)u);
    if (!drawn) {
        if (lane == 0) {
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
            const double p_of = 1.0 / v.p.s, q_of = 1.0 / v.q.s, target = u * total;
            const Place at = pick_weight([&](int g) { return part[g]; }, a.z.nseg, target, lane);
            t = pick_entry<DT>(
                [&](int j) { return entry_residual<DT>((float)xp[j], (float)xq[j], v, p_of, q_of, a.z, a.zq); }, at.i,
                a.z.V, at.base, target, lane);
        }
    } else if (v.what == ROW_OTHER) {
        const int d = (int)o.draft, gd = d / kSeg<DT>;
        const double m = v.p.m;
        auto value = [&](int j) { return j == d ? 0.0 : pow2_any((double)(float)xp[j] - m, a.z.c); };
        double own = 0.0;
        for (int j = gd * kSeg<DT> + lane; j < a.z.V && j < (gd + 1) * kSeg<DT>; j += 64) own += value(j);
        own = wave_sum_f64(own);
        auto weight = [&](int g) { return g == gd ? own : seg_weight(seg[g], v.p.m, a.z.c); };
        double total = 0.0;
        for (int g = lane; g < a.z.nseg; g += 64) total += weight(g);
        total = wave_sum_f64(total);
        if (total >= kLeastResidual * v.p.s) {
            const double target = u * total;
            const Place at = pick_weight(weight, a.z.nseg, target, lane);
            t = pick_entry<DT>(value, at.i, a.z.V, at.base, target, lane);
        }
    }
    if (t < 0) {  // from p, also where rounding leaves nothing else
        draw_token<DT>(xp, seg, v.p, u, a.z, lane, a.token + o.at, a.logp + o.at);
    } else if (lane == 0) {
        a.token[o.at] = t;
        a.logp[o.at] = row_logp((float)xp[t], v.p, a.z.inv_t);
    }
}

// A workgroup takes a sequence, or part blockIdx.x of its residual's sums: the
// drafts four at a time (every part the same), then segments of the residual.
// With one part it draws the token, too.
template <int DT>
__global__ __launch_bounds__(kRowsWG) void k_draft_verify(VerifyArg<DT> a, Outcome* __restrict__ outcomes)
{
    typedef typename Elem<DT>::T T;
    __shared__ Verdict row[kRowsWaves];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    for (int64_t b = blockIdx.y; b < a.B; b += gridDim.y) {
        const int64_t s = held(a.start[b], 0, a.D), n = held(a.start[b + 1], s, a.D) - s;
        int64_t end;
        for (int64_t k0 = 0;; k0 += kRowsWaves) {
            const int64_t k = k0 + wave;
            Verdict v = {};
            v.what = ROW_PLAIN;
            if (k <= n) v = row_verdict<DT>(a, b, s, n, k, lane);
            if (lane == 0) row[wave] = v;
            __syncthreads();
            int w = 0;
            while (w < kRowsWaves && row[w].what == ROW_ACCEPT) ++w;
            if (blockIdx.x == 0 && wave < w && lane == 0) {
                a.token[s + b + k] = a.draft[s + k];
                a.logp[s + b + k] = v.logp;
            }
            end = k0 + w;
            if (w < kRowsWaves) break;  // row n at the latest
            __syncthreads();
        }
        Outcome o;
        o.v = row[end % kRowsWaves];
        o.at = s + b + end;
        o.last = s + b + n;
        o.draft = end < n ? a.draft[s + end] : -1;
        if (blockIdx.x == 0) {
            if (threadIdx.x == 0) a.accepted[b] = end;
            for (int64_t k = end + 1 + threadIdx.x; k <= n; k += kRowsWG) {
                a.token[s + b + k] = -1;
                a.logp[s + b + k] = 0.0f;
            }
            if (gridDim.x > 1 && threadIdx.x == 0) outcomes[b] = o;
        }
        if (o.v.what == ROW_RESIDUAL) {
            const T* xp = a.target + o.at * a.z.stride;
            const T* xq = a.drafts + (s + end) * a.zq.stride;
            const double p_of = 1.0 / o.v.p.s, q_of = 1.0 / o.v.q.s;
            for (int g = (int)blockIdx.x * kRowsWaves + wave; g < a.z.nseg; g += (int)gridDim.x * kRowsWaves) {
                const SegData<DT> x = seg_load<DT>(xp, g, a.z.V, lane), y = seg_load<DT>(xq, g, a.z.V, lane);
                double sum = entry_residual<DT>(x.edge, y.edge, o.v, p_of, q_of, a.z, a.zq);
#pragma unroll
                for (int k = 0; k < kSegU; ++k)
#pragma unroll
                    for (int j = 0; j < kVec<DT>; ++j)
                        sum += entry_residual<DT>((float)x.y[k][j], (float)y.y[k][j], o.v, p_of, q_of, a.z, a.zq);
                sum = wave_sum_f64(sum);
                if (lane == 0) a.residual[b * a.z.nseg + g] = sum;
            }
        }
        __syncthreads();
        if (gridDim.x == 1 && wave == 0) draw_last<DT>(a, b, o, lane);
        __syncthreads();
    }
}

// Draws the last tokens of sequences whose residuals were summed by parts.
template <int DT>
__global__ __launch_bounds__(kRowsWG) void k_draft_draw(VerifyArg<DT> a, const Outcome* __restrict__ outcomes)
{
    const int lane = threadIdx.x & 63;
    for (int64_t b = (int64_t)blockIdx.x * kRowsWaves + (threadIdx.x >> 6); b < a.B; b += (int64_t)gridDim.x * kRowsWaves)
        draw_last<DT>(a, b, outcomes[b], lane);
}

static inline bool rows_ok(int32_t dtype, int64_t N, int64_t V, int64_t stride, float inv_t)
{
    return (dtype == SF_F32 || dtype == SF_BF16 || dtype == SF_F16) && N >= 0 && V >= 1 &&
           V <= ((int64_t)1 << 30) && stride >= V && inv_t > 0.0f && inv_t <= 0x1p100f &&
           (N == 0 || stride <= (((int64_t)1 << 56) / N));
}

static inline RowArg row_arg(int32_t dtype, int64_t V, int64_t stride, float inv_t)
{
    return {stride, (int)V, (int)seg_count(dtype, V), (double)inv_t * kLog2eD, inv_t};
}

// Segments a wave takes where rows are split over workgroups.
static inline int segs_per_wave(int64_t rows, int64_t nseg)
{
    const int64_t per = rows * nseg / 16384;
    return (int)(per < 1 ? 1 : per > 16 ? 16 : per);
}

static inline unsigned up_to(int64_t n, int64_t most) { return (unsigned)(n < most ? n : most); }

// Waves of a row: 1, kRowsWaves, or 0 where rows are split over workgroups.
static inline int sample_waves(int64_t N, int64_t nseg)
{
    if (nseg <= 2 || (N >= 4096 && nseg <= kLdsSegs / kRowsWaves)) return 1;
    return N >= 512 && nseg <= kLdsSegs ? kRowsWaves : 0;
}

}  // namespace sfk

using namespace sfk;

SF_API int64_t sf_token_sample_workspace(int32_t dtype, int64_t N, int64_t V)
{
    if (!rows_ok(dtype, N, V, V, 1.0f)) return -1;
    const int64_t nseg = seg_count(dtype, V);
    return N == 0 || sample_waves(N, nseg) ? 0 : N * nseg * (int64_t)sizeof(RowSum);
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
    const int waves = sample_waves(N, z.nseg);
    void* args[] = {(void*)&logits, (void*)&N, (void*)&uniform, (void*)&z, (void*)&out_token, (void*)&out_logp};
    if (waves) {
        const void* fn[2][3] = {{(const void*)&k_token_sample<SF_F32, 1>, (const void*)&k_token_sample<SF_BF16, 1>,
                                 (const void*)&k_token_sample<SF_F16, 1>},
                                {(const void*)&k_token_sample<SF_F32, kRowsWaves>, (const void*)&k_token_sample<SF_BF16, kRowsWaves>,
                                 (const void*)&k_token_sample<SF_F16, kRowsWaves>}};
        const int rows = kRowsWaves / waves;
        return launch(fn[waves > 1][dtype], dim3(up_to((N + rows - 1) / rows, 1 << 21)), dim3(kRowsWG), args, 0, stream);
    }
    const void* none = nullptr;
    int64_t zero = 0;
    int per = segs_per_wave(N, z.nseg);
    const int64_t each = (int64_t)kRowsWaves * per;
    void* sum_args[] = {(void*)&logits, (void*)&N, (void*)&z, (void*)&none, (void*)&zero, (void*)&z, (void*)&uniform,
                        (void*)&per, (void*)&workspace};
    const void* sums[3] = {(const void*)&k_row_segments<SF_F32>, (const void*)&k_row_segments<SF_BF16>,
                           (const void*)&k_row_segments<SF_F16>};
    const int rc = launch(sums[dtype], dim3((unsigned)((z.nseg + each - 1) / each), up_to(N, 65535)), dim3(kRowsWG), sum_args,
                          0, stream);
    if (rc != SF_OK) return rc;
    void* draw_args[] = {(void*)&logits, (void*)&N, (void*)&uniform, (void*)&z, (void*)&workspace, (void*)&out_token,
                         (void*)&out_logp};
    const void* draw[3] = {(const void*)&k_token_draw<SF_F32>, (const void*)&k_token_draw<SF_BF16>,
                           (const void*)&k_token_draw<SF_F16>};
    return launch(draw[dtype], dim3(up_to((N + kRowsWaves - 1) / kRowsWaves, 1 << 21)), dim3(kRowsWG), draw_args, 0, stream);
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
    int64_t rows = D + B, more = drafts ? D : 0;
    const void* none = nullptr;
    int per = segs_per_wave(rows + more, z.nseg);
    const int64_t each = (int64_t)kRowsWaves * per;
    void* sum_args[] = {(void*)&target, (void*)&rows, (void*)&z,    (void*)&drafts, (void*)&more,
                        (void*)&zq,     (void*)&none, (void*)&per, (void*)&sums};
    int rc = launch((const void*)&k_row_segments<DT>, dim3((unsigned)((z.nseg + each - 1) / each), up_to(rows + more, 65535)),
                    dim3(kRowsWG), sum_args, 0, stream);
    if (rc != SF_OK) return rc;
    VerifyArg<DT> a = {(const T*)target, (const T*)drafts, draft, start, uniform, D, B, z, zq, sums, residual, accepted, token, logp};
    // parts of a residual: about 1024 workgroups in all
    const int64_t most = (z.nseg + kRowsWaves - 1) / kRowsWaves, want = 1024 / B;
    const int64_t parts = !drafts || want < 2 ? 1 : most < want ? most : want;
    void* args[] = {(void*)&a, (void*)&outcomes};
    rc = launch((const void*)&k_draft_verify<DT>, dim3((unsigned)parts, up_to(B, 65535)), dim3(kRowsWG), args, 0, stream);
    if (rc != SF_OK || parts == 1) return rc;
    return launch((const void*)&k_draft_draw<DT>, dim3(up_to((B + kRowsWaves - 1) / kRowsWaves, 1 << 21)), dim3(kRowsWG), args,
                  0, stream);
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
