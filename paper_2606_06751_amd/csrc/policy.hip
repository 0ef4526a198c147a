// policy.hip -- clipped policy loss with a KL term over ragged sequences, and
// its gradient (sf_policy_loss).
//
// A token's terms depend on its own inputs, its sequence's advantage and the
// reduction's weight, which needs to know how many tokens take part (in all or
// per sequence) before the first gradient is written.  So the mask is counted
// first, with one byte a token; then one pass over the tokens writes the
// gradient and a workgroup's sums, which one workgroup adds up in their order.
// Small inputs take one workgroup and one launch.
//
// What bounds it is the number of instructions as much as the bytes: some 75
// a token, and two exponentials at a quarter of the VALU's rate.  So a lane takes
// 4 consecutive tokens (16-byte loads) and a wave 256 a round, which are mostly
// of one sequence: it is found once, in LDS, and followed; only in a round that
// meets another does each lane look for its own (64 tokens a round: 31.7 us for
// 2e6 tokens of 1024 sequences, 256: 14.4; the kernel alone).  Terms are weighed
// and summed in 64 bits and weights are 64-bit quotients, which costs 0.5 us there
// (14.9).  The sums go to a launch of their own: a counter of finished workgroups
// with the memory fences that it needs cost 25 us more, since each fence writes
// back an L2.

#include "sf_device.h"
#include "sf_host.h"
#include "sf_train.h"

namespace sfk {

constexpr int kPolicyWG = 512;
constexpr int kTok = 4;                 // consecutive tokens of a lane: 16-byte loads
constexpr int kRoundTok = 64 * kTok;    // of a wave's round
constexpr int kPolicyChunk = kPolicyWG / 64 * kRoundTok;  // of a workgroup: a round a wave
// Tokens at most: a launch has fewer than 2^32 threads.
constexpr int64_t kPolicyMax = ((((int64_t)1 << 32) / kPolicyWG) - 1) * kPolicyChunk;
static_assert(kPolicyMax == ((int64_t)1 << 34) - (1 << 11), "as the header says");
constexpr int kSliceMax = 2048;  // sequences that a workgroup keeps in LDS
// Sequences of which every workgroup keeps all; with more, a chunk's are looked
// up first (2e6 tokens of 1024: 14.0 us, all of them kept 15.9).
constexpr int kFewSeqs = 256;
constexpr int kCountMax = 2048;  // counts that every workgroup adds up by itself
constexpr int kCountBlocks = 512;
constexpr int kSmallWG = 1024;
constexpr int kSmallRounds = 2;
constexpr int kSmallN = kSmallWG * kTok * kSmallRounds;  // tokens of the one-launch path
constexpr int kSmallSeqs = kSmallWG;                     // and its sequences
constexpr int kJoinWG = 512;
constexpr int kFar = INT32_MAX;

typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v4f_a4 __attribute__((ext_vector_type(4), aligned(4)));

struct Policy {
    const float* logp;
    const float* old_logp;
    const float* ref;
    const float* adv;
    const uint8_t* mask;
    const int64_t* start;
    int64_t N, B;
    float hi, lo;          // the clip's bounds of r
    float log_hi, log_lo;  // and of log r
    float kl_coef, scale;
    int32_t adv_per_token, reduction;
};

__device__ __forceinline__ int64_t clamp_tok(int64_t x, int64_t N) { return x < 0 ? 0 : x > N ? N : x; }

// Index of the first of n ascending starts that lies past t: by a lane for
// itself, or by a wave in looks at 64 starts.
__device__ __forceinline__ int64_t find_start(const int64_t* start, int64_t n, int64_t t)
{
    int64_t lo = 0, hi = n;
    while (lo < hi) {
        const int64_t mid = (lo + hi) >> 1;
        if (start[mid] <= t)
            lo = mid + 1;
        else
            hi = mid;
    }
    return lo;
}
__device__ __forceinline__ int64_t find_start_wave(const int64_t* start, int64_t n, int64_t t)
{
    int64_t lo = 0;
    while (n > 0) {
        const int64_t stride = (n + 63) >> 6, at = (int64_t)(threadIdx.x & 63) * stride;
        const int c = __popcll(__ballot(at < n && start[lo + (at < n ? at : 0)] <= t));
        if (c == 0) break;
        const int64_t from = (c - 1) * stride + 1, to = from - 1 + stride < n ? from - 1 + stride : n;
        lo += from;
        n = to - from;
    }
    return lo;
}

// Tokens of [t0, t1) that take part, by one wave: 16 mask bytes a lane at a time.
__device__ __forceinline__ int64_t count_mask(const uint8_t* mask, int64_t t0, int64_t t1)
{
    const int lane = threadIdx.x & 63;
    int64_t n = 0;
    int64_t body = t0 + (int64_t)((0 - (uintptr_t)(mask + t0)) & 15);
    if (body > t1) body = t1;
    const int64_t nv = (t1 - body) >> 4, tail = body + (nv << 4);
    const uint4* v = (const uint4*)(mask + body);
    // one bit a byte that is not 0
    auto bits = [](uint32_t w) { return __popc((((w & 0x7F7F7F7Fu) + 0x7F7F7F7Fu) | w) & 0x80808080u); };
    for (int64_t k = lane; k < nv; k += 64) {
        const uint4 w = v[k];
        n += bits(w.x) + bits(w.y) + bits(w.z) + bits(w.w);
    }
    const int edges = (int)(body - t0 + t1 - tail);
    if (lane < edges) n += mask[lane < body - t0 ? t0 + lane : tail + (lane - (body - t0))] != 0;
    return wave_sum_i64(n);
}

__device__ __forceinline__ void seq_range(const Policy& a, int64_t b, int64_t* s0, int64_t* s1)
{
    *s0 = clamp_tok(a.start[b], a.N);
    *s1 = clamp_tok(a.start[b + 1], a.N);
    if (*s1 < *s0) *s1 = *s0;
}

// Counts of tokens that take part.  SHARES: equal shares of all tokens, one a
// workgroup.  PARTS (up to kCountMax): part blockIdx.y of gridDim.y of sequence
// blockIdx.x, by a workgroup.  SEQS (more): whole sequences by one wave each, and
// behind them a workgroup's number of those that are not empty.
enum { COUNT_SHARES, COUNT_PARTS, COUNT_SEQS };

template <int KIND>
__global__ __launch_bounds__(kPolicyWG) void k_policy_count(Policy a, int64_t* __restrict__ counts)
{
    constexpr int NW = kPolicyWG / 64;
    __shared__ int64_t part[NW];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int64_t sum = 0;
    if (KIND == COUNT_SEQS) {
        for (int64_t b = (int64_t)blockIdx.x * NW + wave; b < a.B; b += (int64_t)gridDim.x * NW) {
            int64_t t0, t1;
            seq_range(a, b, &t0, &t1);
            const int64_t n = a.mask ? count_mask(a.mask, t0, t1) : t1 - t0;
            if (lane == 0) counts[b] = n;
            sum += n > 0;
        }
    } else {
        int64_t t0, t1, pieces = NW, piece = wave;
        if (KIND == COUNT_SHARES) {
            t0 = clamp_tok(a.start[0], a.N);
            t1 = clamp_tok(a.start[a.B], a.N);
            pieces *= gridDim.x;
            piece += (int64_t)blockIdx.x * NW;
        } else {
            seq_range(a, blockIdx.x, &t0, &t1);
            pieces *= gridDim.y;
            piece += (int64_t)blockIdx.y * NW;
        }
        // at least a round of 1 KB of mask each
        int64_t share = t1 > t0 ? ((t1 - t0 + pieces - 1) / pieces + 1023) & ~(int64_t)1023 : 0;
        t0 += piece * share;
        if (t0 + share < t1) t1 = t0 + share;
        if (t0 < t1) sum = a.mask ? count_mask(a.mask, t0, t1) : t1 - t0;
    }
    if (lane == 0) part[wave] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < NW; ++w) sum += part[w];
        const int64_t at = KIND == COUNT_SEQS    ? a.B + blockIdx.x
                           : KIND == COUNT_PARTS ? (int64_t)blockIdx.x * gridDim.y + blockIdx.y
                                                 : blockIdx.x;
        counts[at] = sum;
    }
}

struct TokenTerms {
    float surr, kl, grad;
    bool clipped;
};

// e^x, within 2 units in the last place wherever it is a float: 2^(x log2 e)
// with the product's rounding put right.  The instruction gives 0 where its
// result is below the normal range, so there it runs 2^64 higher.
__device__ __forceinline__ float exp_f32(float x)
{
#pragma clang fp contract(off)  // h + 64 is the rounded h's, exactly
    const float h = x * kLog2e;
    const float l = fmaf(x, kLog2eLow, fmaf(x, kLog2e, -h));
    const bool low = h < -126.0f;
    const float e = fast_exp2(low ? h + 64.0f : h);
    const float r = fabsf(h) < 128.0f + 64.0f && e != INFINITY ? fmaf(e, l * kLn2, e) : e;
    return low ? r * 0x1p-64f : r;
}

// e^x - x - 1 and e^x - 1.  Near 0 both differences cancel, so a series takes
// over: x^2 (1/2 + x/6 + ... + x^8/10!), within 2^-28 of it for |x| <= 1/2.
__device__ __forceinline__ void kl_terms(float x, float* kl, float* em1)
{
    float q = 1.0f / 3628800.0f;
    q = fmaf(q, x, 1.0f / 362880.0f);
    q = fmaf(q, x, 1.0f / 40320.0f);
    q = fmaf(q, x, 1.0f / 5040.0f);
    q = fmaf(q, x, 1.0f / 720.0f);
    q = fmaf(q, x, 1.0f / 120.0f);
    q = fmaf(q, x, 1.0f / 24.0f);
    q = fmaf(q, x, 1.0f / 6.0f);
    q = fmaf(q, x, 0.5f);
    const float near = x * x * q;
    const float e = exp_f32(x);
    const bool is_near = fabsf(x) <= 0.5f;
    *em1 = is_near ? near + x : e == INFINITY ? kF32Max : e - 1.0f;
    *kl = is_near ? near : e == INFINITY ? kF32Max : *em1 - x;
}

__device__ __forceinline__ TokenTerms token_terms(const Policy& a, float logp, float old, float ref, float adv)
{
    TokenTerms r;
    const float d = logp - old;
    const bool up = adv > 0.0f;
    const bool clipped = up ? d > a.log_hi : adv < 0.0f && d < a.log_lo;
    float ratio = exp_f32(d);
    ratio = ratio == INFINITY ? kF32Max : ratio;
    r.clipped = clipped;
    r.surr = -adv * (clipped ? (up ? a.hi : a.lo) : ratio);
    r.grad = clipped ? 0.0f : r.surr;
    r.kl = 0.0f;
    if (a.ref) {
        float em1;
        kl_terms(ref - logp, &r.kl, &em1);
        r.grad = fmaf(-a.kl_coef, em1, r.grad);
    }
    return r;
}

// scale / n for a count n, and 0 where nothing takes part; one rounding.
__device__ __forceinline__ float share_of(float scale, double n) { return n > 0.0 ? (float)((double)scale / n) : 0.0f; }

// Sum over a workgroup of WG threads, in every thread.
template <int WG>
__device__ __forceinline__ int64_t group_sum(int64_t v, int64_t* part)
{
    v = wave_sum_i64(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0;
#pragma unroll 1
    for (int w = 0; w < WG / 64; ++w) v += part[w];
    return v;
}

// A lane's kTok consecutive tokens, as loaded.
struct Tokens {
    v4f lp, old, ref, adv;
    uint32_t on;  // bit j: token j is there and its mask is not 0
};

__device__ __forceinline__ v4f load4(const float* p, int n)
{
    if (n >= kTok) return *(const v4f_a4*)p;
    v4f x = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int j = 0; j < kTok - 1; ++j)
        if (j < n) x[j] = p[j];
    return x;
}

__device__ __forceinline__ uint32_t load_mask(const uint8_t* p, int n)
{
    if (n <= 0) return 0;
    uint32_t on = n >= kTok ? 0xFu : (1u << n) - 1;
    if (p) {
        uint32_t m = 0;
        if (n >= kTok)
            __builtin_memcpy(&m, p, 4);
        else
            for (int j = 0; j < n; ++j) m |= (uint32_t)p[j] << (8 * j);
        // a bit a byte that is not 0, gathered
        m = (((m & 0x7F7F7F7Fu) + 0x7F7F7F7Fu) | m) & 0x80808080u;
        on &= (m >> 7 | m >> 14 | m >> 21 | m >> 28) & 0xFu;
    }
    return on;
}

// The tokens from t0 + off on, of the wave's [t0, t0 + len).
__device__ __forceinline__ Tokens load_tokens(const Policy& a, int64_t t0, int off, int len)
{
    Tokens x = {};
    const int n = len - off;
    if (n <= 0) return x;
    x.lp = load4(a.logp + t0 + off, n);
    x.old = load4(a.old_logp + t0 + off, n);
    if (a.ref) x.ref = load4(a.ref + t0 + off, n);
    if (a.adv_per_token) x.adv = load4(a.adv + t0 + off, n);
    x.on = load_mask(a.mask ? a.mask + t0 + off : nullptr, n);
    return x;
}

// Index of the last of `n` ascending starts at or before t, -1: none.
__device__ __forceinline__ int last_start(const int* start, int n, int t)
{
    int lo = 0, hi = n;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (start[mid] <= t)
            lo = mid + 1;
        else
            hi = mid;
    }
    return lo - 1;
}

// The sequences of a wave's tokens, a round at a time, in the slice of n
// sequences whose n + 1 starts lie in LDS: mostly all of one, which is followed.
struct Walk {
    const int* start;
    int n, k;  // k: the sequence, or gap, of the round's first token

    __device__ __forceinline__ int next() const
    {
        return k < n ? __builtin_amdgcn_readfirstlane(start[k + 1]) : kFar;
    }
    // to the round of tokens [t, t + kRoundTok); true where all are of one
    __device__ __forceinline__ bool round(int t)
    {
        while (next() <= t) ++k;
        return next() > t + kRoundTok - 1;
    }
    __device__ __forceinline__ bool inside(int q) const { return q >= 0 && q < n; }
};

// From token t on: the last start at or before it, found by the wave in two
// looks (every stride-th start, then those between).
__device__ __forceinline__ Walk walk_from(const int* start, int n, int t)
{
    const int lane = threadIdx.x & 63;
    const int stride = (n + 64) >> 6;  // 64 strides hold n + 1 starts
    int at = lane * stride;
    int k = __popcll(__ballot(at <= n && start[at <= n ? at : 0] <= t)) - 1;
    if (k >= 0 && stride > 1) {
        at = k * stride + lane;
        const bool in = lane < stride && at <= n;
        k = k * stride + __popcll(__ballot(in && start[in ? at : 0] <= t)) - 1;
    }
    return {start, n, k};
}

__device__ __forceinline__ void write_terms(const double (&s)[3], float kl_coef, float* terms)
{
    terms[0] = (float)(kl_coef == 0.0f ? s[0] : s[0] + (double)kl_coef * s[1]);
    terms[1] = (float)s[0];
    terms[2] = (float)s[1];
    terms[3] = (float)s[2];
}

// Sums over a workgroup; valid in thread 0.
template <int WG>
__device__ __forceinline__ void group_terms(double (&sum)[3], double (*part)[WG / 64])
{
#pragma unroll
    for (int q = 0; q < 3; ++q) {
        sum[q] = wave_sum_f64(sum[q]);
        if ((threadIdx.x & 63) == 0) part[q][threadIdx.x >> 6] = sum[q];
    }
    __syncthreads();
    if (threadIdx.x == 0)
#pragma unroll
        for (int q = 0; q < 3; ++q) {
            sum[q] = part[q][0];
#pragma unroll 1
            for (int w = 1; w < WG / 64; ++w) sum[q] += part[q][w];
        }
}

// Adds a token with its weight to the sums, in 64 bits, where no product of two
// floats overflows or rounds.
__device__ __forceinline__ void add_terms(const TokenTerms& r, float w, bool on, double (&sum)[3])
{
    const double d = on ? (double)w : 0.0;
    sum[0] = fma(d, on ? (double)r.surr : 0.0, sum[0]);
    sum[1] = fma(d, on ? (double)r.kl : 0.0, sum[1]);
    sum[2] += r.clipped ? d : 0.0;
}

// Adds a lane's tokens with their weights and advantages to its sums; their
// gradients.
__device__ __forceinline__ v4f add_tokens(const Policy& a, const Tokens& x, uint32_t on, v4f w, v4f adv, double (&sum)[3])
{
    v4f g;
#pragma unroll
    for (int j = 0; j < kTok; ++j) {
        const TokenTerms r = token_terms(a, x.lp[j], x.old[j], x.ref[j], adv[j]);
        const bool is_on = on >> j & 1;
        g[j] = is_on ? w[j] * r.grad : 0.0f;
        add_terms(r, w[j], is_on, sum);
    }
    return g;
}

// One round: the tokens' weights and advantages by their sequences (the slice's,
// in LDS), their terms and gradients.
__device__ __forceinline__ void add_round(const Policy& a, const Tokens& x, Walk& walk, int t, int off, int len,
                                          const float* seq_adv, const float* weight, double (&sum)[3], float* out)
{
    v4f w = {0.0f, 0.0f, 0.0f, 0.0f}, adv = x.adv;
    uint32_t on = x.on;
    if (walk.round(t)) {
        if (walk.inside(walk.k)) {
            const float w1 = weight[walk.k];
            w = v4f{w1, w1, w1, w1};
            if (!a.adv_per_token) {
                const float a1 = seq_adv[walk.k];
                adv = v4f{a1, a1, a1, a1};
            }
        } else {
            on = 0;
        }
    } else {
        const int mine = t + (int)(threadIdx.x & 63) * kTok;
        int k = last_start(walk.start, walk.n + 1, mine);
#pragma unroll
        for (int j = 0; j < kTok; ++j) {
            while (k < walk.n && walk.start[k + 1] <= mine + j) ++k;
            if (walk.inside(k)) {
                w[j] = weight[k];
                if (!a.adv_per_token) adv[j] = seq_adv[k];
            } else {
                on &= ~(1u << j);
            }
        }
    }
    const v4f g = add_tokens(a, x, on, w, adv, sum);
    if (len - off >= kTok)
        *(v4f_a4*)(out + off) = g;
    else
#pragma unroll
        for (int j = 0; j < kTok - 1; ++j)
            if (j < len - off) out[off + j] = g[j];
}

// What the count left: n counts, of shares of all tokens, or of parts of
// sequences (1 << shift a sequence); or (numbers) a count per sequence and,
// behind all of them, n workgroups' numbers of sequences that are not empty; or
// nothing (n = 0).
struct Weights {
    const int64_t* counts;
    int32_t n, shift, numbers;
};

// One workgroup, one chunk of tokens.  The sequences that the chunk meets (all
// of them where they are few) lie in LDS; where even these are too many, each
// token looks its own up in memory.
__global__ __launch_bounds__(kPolicyWG) void k_policy_loss(Policy a, Weights wt, float* __restrict__ out_grad,
                                                           double* __restrict__ partial)
{
    __shared__ int start[kSliceMax + 1];  // relative to the chunk
    __shared__ unsigned long long count[kFewSeqs];
    __shared__ float weight[kSliceMax], seq_adv[kSliceMax];
    __shared__ int64_t ints[kPolicyWG / 64];
    __shared__ double part[3][kPolicyWG / 64];
    const int tid = threadIdx.x, lane = tid & 63;
    const int64_t t0 = (int64_t)blockIdx.x * kPolicyChunk;
    const int64_t t1 = t0 + kPolicyChunk < a.N ? t0 + kPolicyChunk : a.N;
    const int first = __builtin_amdgcn_readfirstlane(tid >> 6) * kRoundTok;  // of the wave, in the chunk
    const int64_t wave0 = t0 + first;
    const int len = wave0 >= t1 ? 0 : t1 - wave0 < kRoundTok ? (int)(t1 - wave0) : kRoundTok;
    const Tokens x = load_tokens(a, wave0, lane * kTok, len);

    // the slice of sequences [b0, b0 + slice)
    int64_t b0 = 0, slice = a.B;
    if (a.B > kFewSeqs) {
        const int wave = tid >> 6;
        if (wave < 2) {
            const int64_t k = find_start_wave(a.start, a.B + 1, wave == 0 ? t0 : t1 - 1);
            if (lane == 0) ints[wave] = k;
        }
        __syncthreads();
        b0 = ints[0] > 0 ? ints[0] - 1 : 0;
        const int64_t b1 = ints[1] < a.B ? ints[1] : a.B;
        slice = b1 > b0 ? b1 - b0 : 0;
    }
    const bool few = a.B <= kFewSeqs, fits = slice <= kSliceMax;
    // every load of the prologue before the first wait for one
    constexpr int RS = kFewSeqs / kPolicyWG + 1, RC = kCountMax / kPolicyWG;
    int64_t starts[RS], counts[RC];
    const int64_t* from = wt.counts + (wt.numbers ? a.B : 0);
#pragma unroll
    for (int r = 0; r < RS; ++r) starts[r] = fits && tid + r * kPolicyWG <= slice ? a.start[b0 + tid + r * kPolicyWG] : 0;
#pragma unroll
    for (int r = 0; r < RC; ++r) counts[r] = tid + r * kPolicyWG < wt.n ? from[tid + r * kPolicyWG] : 0;
    auto keep = [&](int k, int64_t v) {
        const int64_t d = v - t0;
        start[k] = d < -1 ? -1 : d > kPolicyChunk ? kPolicyChunk : (int)d;
    };
    if (fits) {
#pragma unroll
        for (int r = 0; r < RS; ++r)
            if (tid + r * kPolicyWG <= slice) keep(tid + r * kPolicyWG, starts[r]);
        for (int k = tid + RS * kPolicyWG; k <= slice; k += kPolicyWG) keep(k, a.start[b0 + k]);
    }

    // one weight for all tokens, or one per sequence
    float scale = a.scale;
    double some = 0.0;  // sequences that are not empty
    if (a.reduction == SF_MEAN_TOKENS) {
        int64_t all = 0;
#pragma unroll
        for (int r = 0; r < RC; ++r) all += counts[r];
        if (wt.n == 0 && tid == 0) all = clamp_tok(a.start[a.B], a.N) - clamp_tok(a.start[0], a.N);
        all = group_sum<kPolicyWG>(all, ints);
        scale = share_of(scale, (double)all);
    } else if (a.reduction == SF_MEAN_SEQUENCES) {
        int64_t mine = 0;
        if (!few) {
#pragma unroll
            for (int r = 0; r < RC; ++r) mine += wt.numbers ? counts[r] : counts[r] > 0;
        } else {
            if (wt.n == 0) {  // no mask: their lengths
                for (int k = tid; k < slice; k += kPolicyWG) {
                    int64_t s0, s1;
                    seq_range(a, k, &s0, &s1);
                    count[k] = (unsigned long long)(s1 - s0);
                }
            } else if (wt.shift == 0) {
#pragma unroll
                for (int r = 0; r < RC; ++r)
                    if (tid + r * kPolicyWG < wt.n) count[tid + r * kPolicyWG] = (unsigned long long)counts[r];
            } else {
                for (int k = tid; k < slice; k += kPolicyWG) count[k] = 0;
                __syncthreads();
#pragma unroll
                for (int r = 0; r < RC; ++r)
                    if (tid + r * kPolicyWG < wt.n)
                        atomicAdd(&count[(tid + r * kPolicyWG) >> wt.shift], (unsigned long long)counts[r]);
                __syncthreads();
            }
            for (int k = tid; k < slice; k += kPolicyWG) mine += count[k] > 0;
        }
        some = (double)group_sum<kPolicyWG>(mine, ints);
    }
    __syncthreads();
    auto weight_of = [&](int64_t k) {
        if (a.reduction != SF_MEAN_SEQUENCES) return scale;
        return share_of(scale, some * (few ? (double)count[k] : (double)wt.counts[b0 + k]));
    };
    if (fits) {
        for (int k = tid; k < slice; k += kPolicyWG) {
            weight[k] = weight_of(k);
            if (!a.adv_per_token) seq_adv[k] = a.adv[b0 + k];
        }
        __syncthreads();
    }
    double sum[3] = {0.0, 0.0, 0.0};
    float* grad = out_grad + wave0;
    if (fits) {
        Walk walk = walk_from(start, (int)slice, first);
        if (len > 0) add_round(a, x, walk, first, lane * kTok, len, seq_adv, weight, sum, grad);
    } else {
#pragma unroll 1
        for (int off = lane; off < len; off += 64) {
            const int64_t k = find_start(a.start, a.B + 1, wave0 + off);
            const bool on = k >= 1 && k <= a.B && (!a.mask || a.mask[wave0 + off] != 0);
            float g = 0.0f;
            if (on) {
                const TokenTerms r = token_terms(a, a.logp[wave0 + off], a.old_logp[wave0 + off],
                                                 a.ref ? a.ref[wave0 + off] : 0.0f,
                                                 a.adv_per_token ? a.adv[wave0 + off] : a.adv[k - 1]);
                const float w = weight_of(k - 1 - b0);
                g = w * r.grad;
                add_terms(r, w, true, sum);
            }
            grad[off] = g;
        }
    }
    group_terms<kPolicyWG>(sum, part);
    if (tid == 0)
        for (int q = 0; q < 3; ++q) partial[(int64_t)blockIdx.x * 3 + q] = sum[q];
}

// The whole loss by one workgroup: up to kSmallN tokens in kSmallSeqs sequences.
__global__ __launch_bounds__(kSmallWG) void k_policy_small(Policy a, float* __restrict__ out_grad,
                                                           float* __restrict__ out_terms)
{
    __shared__ int start[kSmallSeqs + 1];
    __shared__ int count[kSmallSeqs];
    __shared__ float weight[kSmallSeqs], seq_adv[kSmallSeqs];
    __shared__ int64_t ints[kSmallWG / 64];
    __shared__ double part[3][kSmallWG / 64];
    const int tid = threadIdx.x, lane = tid & 63;
    const int B = (int)a.B;
    const int N = (int)a.N, rounds = N <= kSmallWG * kTok ? 1 : kSmallRounds;
    const int each = rounds * kRoundTok;  // consecutive tokens of a wave
    const int first = __builtin_amdgcn_readfirstlane(tid >> 6) * each;
    const int len = first >= N ? 0 : N - first < each ? N - first : each;
    Tokens next = load_tokens(a, first, lane * kTok, len);
    uint32_t ons = next.on;  // kTok bits a round
#pragma unroll
    for (int q = 1; q < kSmallRounds; ++q) {
        const int off = q * kRoundTok + lane * kTok;
        ons |= load_mask(a.mask ? a.mask + first + off : nullptr, len - off) << (q * kTok);
    }
    const float adv = !a.adv_per_token && tid < B ? a.adv[tid] : 0.0f;
    for (int k = tid; k <= B; k += kSmallWG) {
        start[k] = (int)clamp_tok(a.start[k], a.N);
        if (k < B) count[k] = 0;
    }
    __syncthreads();
    float scale = a.scale;
    double some = 0.0;  // sequences that are not empty
    if (a.reduction == SF_MEAN_TOKENS) {
        int64_t n = 0;
#pragma unroll
        for (int q = 0; q < kSmallRounds * kTok; ++q) {
            const int t = first + (q / kTok) * kRoundTok + lane * kTok + q % kTok;
            n += (ons >> q & 1) && t >= start[0] && t < start[B];
        }
        n = group_sum<kSmallWG>(n, ints);
        scale = share_of(scale, (double)n);
    } else if (a.reduction == SF_MEAN_SEQUENCES) {
        Walk walk = walk_from(start, B, first);
        uint32_t left = ons;
#pragma unroll 1
        for (int q = 0; q < len; q += kRoundTok, left >>= kTok) {
            // a wave whose tokens are all of one sequence adds once
            if (walk.round(first + q)) {
                const int n = (int)wave_sum_i64(__popc(left & ((1u << kTok) - 1)));
                if (lane == 0 && walk.inside(walk.k) && n > 0) atomicAdd(&count[walk.k], n);
            } else {
                for (int j = 0; j < kTok; ++j) {
                    const int k = last_start(start, B + 1, first + q + lane * kTok + j);
                    if ((left >> j & 1) && walk.inside(k)) atomicAdd(&count[k], 1);
                }
            }
        }
        __syncthreads();
        some = (double)group_sum<kSmallWG>(tid < B && count[tid] > 0, ints);
    }
    if (tid < B) {
        weight[tid] = a.reduction != SF_MEAN_SEQUENCES ? scale : share_of(scale, some * count[tid]);
        if (!a.adv_per_token) seq_adv[tid] = adv;
    }
    __syncthreads();
    double sum[3] = {0.0, 0.0, 0.0};
    Walk walk = walk_from(start, B, first);
#pragma unroll 1
    for (int q = 0; q < len; q += kRoundTok) {
        const Tokens x = next;
        next = load_tokens(a, first, q + kRoundTok + lane * kTok, len);
        add_round(a, x, walk, first + q, q + lane * kTok, len, seq_adv, weight, sum, out_grad + first);
    }
    group_terms<kSmallWG>(sum, part);
    if (tid == 0) write_terms(sum, a.kl_coef, out_terms);
}

// The workgroups' sums in their order.
__global__ __launch_bounds__(kJoinWG) void k_policy_join(int64_t chunks, float kl_coef,
                                                           const double* __restrict__ partial,
                                                           float* __restrict__ terms)
{
    __shared__ double part[3][kJoinWG / 64];
    double sum[3] = {0.0, 0.0, 0.0};
    for (int64_t k = threadIdx.x; k < chunks; k += kJoinWG)
        for (int q = 0; q < 3; ++q) sum[q] += partial[k * 3 + q];
    group_terms<kJoinWG>(sum, part);
    if (threadIdx.x == 0) write_terms(sum, kl_coef, terms);
}

// One workgroup for all of it takes 11.2 us for 5003 tokens, where two or three
// launches take the host 6 to 10 us more than one.
static inline bool small_policy(int64_t N, int64_t B) { return N <= kSmallN && B <= kSmallSeqs; }

// log2 of the workgroups that count a sequence, where there are few: each has
// about four rounds of 4 KB of mask.
static inline int count_shift(int64_t N, int64_t B)
{
    int shift = 0;
    while ((B << (shift + 1)) <= kCountMax && (N >> shift) > 16384 * B) ++shift;
    return shift;
}

struct PolicyLayout {
    int64_t partial, bytes;  // offsets; the counts come first
};

static inline int64_t up16(int64_t n) { return (n + 15) & ~(int64_t)15; }

static inline PolicyLayout policy_layout(int64_t N, int64_t B)
{
    PolicyLayout l;
    l.partial = up16((B > kCountMax ? B + kCountBlocks : kCountMax) * 8);
    l.bytes = l.partial + up16((N + kPolicyChunk - 1) / kPolicyChunk * 3 * 8);
    return l;
}

static inline bool policy_sizes_ok(int64_t N, int64_t B)
{
    return N >= 0 && N <= kPolicyMax && B >= 0 && B < ((int64_t)1 << 31);
}

}  // namespace sfk

using namespace sfk;

SF_API int64_t sf_policy_loss_workspace(int64_t N, int64_t B)
{
    if (!policy_sizes_ok(N, B)) return -1;
    return small_policy(N, B) ? 0 : policy_layout(N, B).bytes;
}

SF_API int sf_policy_loss(const float* logp, const float* old_logp, const float* ref_logp, const float* advantage,
                          int32_t advantage_per_token, const uint8_t* mask, const int64_t* seq_start, int64_t N,
                          int64_t B, int32_t reduction, float scale, float clip_low, float clip_high,
                          float kl_coef, float* out_terms, float* out_grad, void* workspace,
                          int64_t workspace_bytes, sf_stream_t stream)
{
    if (!policy_sizes_ok(N, B) || reduction < SF_MEAN_TOKENS || reduction > SF_SUM_TOKENS) return SF_EINVAL;
    if (!(fabsf(scale) <= kF32Max) || !(clip_low >= 0.0f && clip_low < 1.0f) ||
        !(clip_high >= 0.0f && clip_high <= kF32Max) || !(fabsf(kl_coef) <= kF32Max))
        return SF_EINVAL;
    const PolicyLayout l = policy_layout(N, B);
    const int64_t need = small_policy(N, B) ? 0 : l.bytes;
    if (!out_terms || !seq_start) return SF_EINVAL;
    if (need > 0 && (!workspace || workspace_bytes < need || !aligned(workspace, 16))) return SF_EINVAL;
    const int64_t n_adv = advantage_per_token ? N : B;
    if (N > 0 && (!logp || !old_logp || !out_grad)) return SF_EINVAL;
    if (n_adv > 0 && !advantage) return SF_EINVAL;
    if (!aligned(logp, 4) || !aligned(old_logp, 4) || !aligned(ref_logp, 4) || !aligned(advantage, 4) ||
        !aligned(seq_start, 8) || !aligned(out_terms, 4) || !aligned(out_grad, 4))
        return SF_EINVAL;
    const void* ins[6] = {logp, old_logp, ref_logp, advantage, mask, seq_start};
    const int64_t in_bytes[6] = {N * 4, N * 4, N * 4, n_adv * 4, N, (B + 1) * 8};
    const void* outs[3] = {out_terms, out_grad, workspace};
    const int64_t out_bytes[3] = {16, N * 4, need};
    for (int o = 0; o < 3; ++o) {
        if (!outs[o] || out_bytes[o] == 0) continue;
        for (int i = 0; i < 6; ++i)
            if (ins[i] && in_bytes[i] > 0 && !disjoint(ins[i], in_bytes[i], outs[o], out_bytes[o])) return SF_EINVAL;
        for (int q = o + 1; q < 3; ++q)
            if (outs[q] && out_bytes[q] > 0 && !disjoint(outs[q], out_bytes[q], outs[o], out_bytes[o]))
                return SF_EINVAL;
    }
    Policy a;
    a.logp = logp;
    a.old_logp = old_logp;
    a.ref = ref_logp;
    a.adv = advantage;
    a.mask = mask;
    a.start = seq_start;
    a.N = N;
    a.B = B;
    a.hi = 1.0f + clip_high;
    a.lo = 1.0f - clip_low;
    a.log_hi = (float)log1p((double)clip_high);
    a.log_lo = (float)log1p(-(double)clip_low);
    a.kl_coef = kl_coef;
    a.scale = scale;
    a.adv_per_token = advantage_per_token != 0;
    a.reduction = reduction;
    if (small_policy(N, B)) {
        void* args[] = {(void*)&a, (void*)&out_grad, (void*)&out_terms};
        return launch((const void*)&k_policy_small, dim3(1), dim3(kSmallWG), args, 0, stream);
    }
    int64_t* counts = (int64_t*)workspace;
    double* partial = (double*)((char*)workspace + l.partial);
    int64_t chunks = (N + kPolicyChunk - 1) / kPolicyChunk;
    Weights wt = {counts, 0, 0, 0};
    if (N > 0 && B > 0 && reduction != SF_SUM_TOKENS && (mask || (reduction == SF_MEAN_SEQUENCES && B > kFewSeqs))) {
        const void* fn;
        dim3 grid;
        if (reduction == SF_MEAN_TOKENS) {
            // shares of at least four rounds
            const int64_t want = N / 16384 + 1;
            wt.n = (int)(want < kCountBlocks ? want : kCountBlocks);
            fn = (const void*)&k_policy_count<COUNT_SHARES>;
            grid = dim3((unsigned)wt.n);
        } else if (B <= kCountMax) {
            wt.shift = B <= kFewSeqs ? count_shift(N, B) : 0;
            wt.n = (int)B << wt.shift;
            fn = (const void*)&k_policy_count<COUNT_PARTS>;
            grid = dim3((unsigned)B, 1u << wt.shift);
        } else {
            const int64_t want = (B + kPolicyWG / 64 - 1) / (kPolicyWG / 64);
            wt.n = (int)(want < kCountBlocks ? want : kCountBlocks);
            wt.numbers = 1;
            fn = (const void*)&k_policy_count<COUNT_SEQS>;
            grid = dim3((unsigned)wt.n);
        }
        void* args[] = {(void*)&a, (void*)&counts};
        const int rc = launch(fn, grid, dim3(kPolicyWG), args, 0, stream);
        if (rc != SF_OK) return rc;
    }
    if (chunks > 0) {
        void* args[] = {(void*)&a, (void*)&wt, (void*)&out_grad, (void*)&partial};
        const int rc = launch((const void*)&k_policy_loss, dim3((unsigned)chunks), dim3(kPolicyWG), args, 0, stream);
        if (rc != SF_OK) return rc;
    }
    void* jargs[] = {(void*)&chunks, (void*)&kl_coef, (void*)&partial, (void*)&out_terms};
    return launch((const void*)&k_policy_join, dim3(1), dim3(kJoinWG), jargs, 0, stream);
}
