// policy.hip -- clipped policy loss with a KL term over ragged sequences, and
// its gradient (sf_policy_loss).
//
// A token's terms depend on its own inputs, its sequence's advantage and the
// reduction's weight.  The weights come first (how many tokens take part, in
// all or per sequence), then one pass over the tokens writes the gradient and
// a workgroup's sums, which a last workgroup adds up in their order.

#include "sf_device.h"
#include "sf_host.h"
#include "sf_train.h"

namespace sfk {

constexpr int kPolicyWG = 256;
constexpr int kPolicyTok = 4;                          // tokens per thread
constexpr int64_t kPolicyChunk = kPolicyWG * kPolicyTok;  // tokens per workgroup
constexpr int kJoinWG = 1024;

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

// Sequence that holds token t, or -1: the last one that starts at or before t,
// where it also ends after t.
__device__ __forceinline__ int64_t find_seq(const int64_t* start, int64_t B, int64_t t)
{
    int64_t lo = 0, hi = B + 1;  // first index whose start lies past t
    while (lo < hi) {
        const int64_t mid = (lo + hi) >> 1;
        if (start[mid] <= t)
            lo = mid + 1;
        else
            hi = mid;
    }
    return lo >= 1 && lo <= B ? lo - 1 : -1;
}

// Tokens that take part: part p of P of sequence b, by one wave.
__global__ __launch_bounds__(kPolicyWG) void k_policy_count(Policy a, int P, int64_t* __restrict__ counts)
{
    const int lane = threadIdx.x & 63;
    const int64_t waves = (int64_t)gridDim.x * (kPolicyWG / 64);
    for (int64_t w = (int64_t)blockIdx.x * (kPolicyWG / 64) + (threadIdx.x >> 6); w < a.B * P; w += waves) {
        const int64_t b = w / P, p = w - b * P;
        const int64_t s0 = clamp_tok(a.start[b], a.N), s1 = clamp_tok(a.start[b + 1], a.N);
        const int64_t len = s1 > s0 ? s1 - s0 : 0;
        const int64_t t0 = s0 + len * p / P, t1 = s0 + len * (p + 1) / P;
        int64_t n = 0;
        if (a.mask)
            for (int64_t t = t0 + lane; t < t1; t += 64) n += a.mask[t] != 0;
        else
            n = lane == 0 ? t1 - t0 : 0;
        n = wave_sum64(n);
        if (lane == 0) counts[w] = n;
    }
}

// The weight of a token: one for all (weights[0]) or one per sequence.
__global__ __launch_bounds__(kJoinWG) void k_policy_weight(Policy a, int P, const int64_t* __restrict__ counts,
                                                           float* __restrict__ weights)
{
    __shared__ int64_t part[2][kJoinWG / 64];
    const int tid = threadIdx.x;
    int64_t all = 0, some = 0;
    for (int64_t b = tid; b < a.B; b += kJoinWG) {
        int64_t n = 0;
        for (int p = 0; p < P; ++p) n += counts[b * P + p];
        all += n;
        some += n > 0;
    }
    all = wave_sum64(all);
    some = wave_sum64(some);
    if ((tid & 63) == 0) {
        part[0][tid >> 6] = all;
        part[1][tid >> 6] = some;
    }
    __syncthreads();
    all = some = 0;
    for (int w = 0; w < kJoinWG / 64; ++w) {
        all += part[0][w];
        some += part[1][w];
    }
    if (a.reduction == SF_MEAN_TOKENS) {
        if (tid == 0) weights[0] = all > 0 ? (float)((double)a.scale / (double)all) : 0.0f;
        return;
    }
    for (int64_t b = tid; b < a.B; b += kJoinWG) {
        int64_t n = 0;
        for (int p = 0; p < P; ++p) n += counts[b * P + p];
        weights[b] = n > 0 ? (float)((double)a.scale / ((double)some * (double)n)) : 0.0f;
    }
}

struct TokenTerms {
    float surr, kl, clipped, grad;
};

// e^x - x - 1 and e^x - 1.  Near 0 both differences cancel, so a series takes
// over: x^2 (1/2 + x/6 + ... + x^8/10!), within 2^-28 of it for |x| <= 1/2.
__device__ __forceinline__ void kl_terms(float x, float* kl, float* em1)
{
    if (fabsf(x) <= 0.5f) {
        float q = 1.0f / 3628800.0f;
        q = fmaf(q, x, 1.0f / 362880.0f);
        q = fmaf(q, x, 1.0f / 40320.0f);
        q = fmaf(q, x, 1.0f / 5040.0f);
        q = fmaf(q, x, 1.0f / 720.0f);
        q = fmaf(q, x, 1.0f / 120.0f);
        q = fmaf(q, x, 1.0f / 24.0f);
        q = fmaf(q, x, 1.0f / 6.0f);
        q = fmaf(q, x, 0.5f);
        *kl = x * x * q;
        *em1 = *kl + x;
        return;
    }
    const float e = expf(x);
    if (e == INFINITY) {
        *kl = *em1 = kF32Max;
        return;
    }
    *em1 = e - 1.0f;
    *kl = *em1 - x;
}

__device__ __forceinline__ TokenTerms token_terms(const Policy& a, float logp, float old, float ref, float adv)
{
    TokenTerms r;
    const float d = logp - old;
    const bool over = adv > 0.0f && d > a.log_hi, under = adv < 0.0f && d < a.log_lo;
    float ratio = expf(d);
    if (ratio == INFINITY) ratio = kF32Max;
    r.clipped = over || under ? 1.0f : 0.0f;
    r.surr = -adv * (over ? a.hi : under ? a.lo : ratio);
    r.grad = over || under ? 0.0f : r.surr;
    r.kl = 0.0f;
    if (a.ref) {
        float em1;
        kl_terms(ref - logp, &r.kl, &em1);
        r.grad = fmaf(-a.kl_coef, em1, r.grad);
    }
    return r;
}

__global__ __launch_bounds__(kPolicyWG) void k_policy_loss(Policy a, const float* __restrict__ weights,
                                                           float* __restrict__ out_grad,
                                                           double* __restrict__ partial)
{
    __shared__ double part[3][kPolicyWG / 64];
    const int tid = threadIdx.x;
    const int64_t chunks = (a.N + kPolicyChunk - 1) / kPolicyChunk;
    for (int64_t ch = blockIdx.x; ch < chunks; ch += gridDim.x) {
        const int64_t t0 = ch * kPolicyChunk + (int64_t)tid * kPolicyTok;
        double sum[3] = {0.0, 0.0, 0.0};
        if (t0 < a.N) {
            const int n = (int)(a.N - t0 < kPolicyTok ? a.N - t0 : kPolicyTok);
            float lp[kPolicyTok], old[kPolicyTok], ref[kPolicyTok], adv[kPolicyTok], g[kPolicyTok];
            bool on[kPolicyTok];
            int64_t b = find_seq(a.start, a.B, t0);
            int64_t end = b >= 0 ? a.start[b + 1] : 0;
            float w = 0.0f, seq_adv = 0.0f;
            for (int k = 0; k < kPolicyTok; ++k) {
                const int64_t t = t0 + (k < n ? k : 0);
                lp[k] = a.logp[t];
                old[k] = a.old_logp[t];
                ref[k] = a.ref ? a.ref[t] : 0.0f;
                adv[k] = a.adv_per_token ? a.adv[t] : 0.0f;
                on[k] = k < n && (!a.mask || a.mask[t] != 0);
            }
            bool fresh = true;
            for (int k = 0; k < kPolicyTok; ++k) {
                const int64_t t = t0 + k;
                if (k > 0 && t >= end) {
                    b = find_seq(a.start, a.B, t);
                    end = b >= 0 ? a.start[b + 1] : 0;
                    fresh = true;
                }
                if (fresh && b >= 0) {
                    w = a.reduction == SF_MEAN_SEQUENCES ? weights[b]
                        : a.reduction == SF_MEAN_TOKENS  ? weights[0]
                                                         : a.scale;
                    if (!a.adv_per_token) seq_adv = a.adv[b];
                    fresh = false;
                }
                g[k] = 0.0f;
                if (!on[k] || b < 0) continue;
                const TokenTerms r = token_terms(a, lp[k], old[k], ref[k], a.adv_per_token ? adv[k] : seq_adv);
                g[k] = w * r.grad;
                sum[0] += (double)(w * r.surr);
                sum[1] += (double)(w * r.kl);
                sum[2] += (double)(w * r.clipped);
            }
            if (n == kPolicyTok)
                *(v4f_a4*)(out_grad + t0) = v4f_a4{g[0], g[1], g[2], g[3]};
            else
                for (int k = 0; k < kPolicyTok; ++k)
                    if (k < n) out_grad[t0 + k] = g[k];
        }
        for (int q = 0; q < 3; ++q) {
            sum[q] = wave_sum_f64(sum[q]);
            if ((tid & 63) == 0) part[q][tid >> 6] = sum[q];
        }
        __syncthreads();
        if (tid < 3) {
            double s = 0.0;
            for (int w = 0; w < kPolicyWG / 64; ++w) s += part[tid][w];
            partial[ch * 3 + tid] = s;
        }
        __syncthreads();
    }
}

// The workgroups' sums in their order, and the loss from them.
__global__ __launch_bounds__(kJoinWG) void k_policy_join(int64_t chunks, float kl_coef,
                                                         const double* __restrict__ partial,
                                                         float* __restrict__ terms)
{
    __shared__ double part[3][kJoinWG / 64];
    const int tid = threadIdx.x;
    double sum[3] = {0.0, 0.0, 0.0};
    for (int64_t ch = tid; ch < chunks; ch += kJoinWG)
        for (int q = 0; q < 3; ++q) sum[q] += partial[ch * 3 + q];
    for (int q = 0; q < 3; ++q) {
        sum[q] = wave_sum_f64(sum[q]);
        if ((tid & 63) == 0) part[q][tid >> 6] = sum[q];
    }
    __syncthreads();
    if (tid == 0) {
        double s[3] = {0.0, 0.0, 0.0};
        for (int q = 0; q < 3; ++q)
            for (int w = 0; w < kJoinWG / 64; ++w) s[q] += part[q][w];
        terms[0] = (float)(kl_coef == 0.0f ? s[0] : s[0] + (double)kl_coef * s[1]);
        terms[1] = (float)s[0];
        terms[2] = (float)s[1];
        terms[3] = (float)s[2];
    }
}

// Parts that a sequence's count is split into: one wave each, enough for the
// chip where there are few sequences.
static inline int count_parts(int64_t N, int64_t B)
{
    const int64_t want = (2048 + B - 1) / B;
    const int64_t most = N / 4096 + 1;
    const int64_t p = want < most ? want : most;
    return p < 1 ? 1 : (int)p;
}

struct PolicyLayout {
    int P;
    int64_t counts, weights, partial, bytes;  // offsets
};

static inline int64_t up16(int64_t n) { return (n + 15) & ~(int64_t)15; }

static inline PolicyLayout policy_layout(int64_t N, int64_t B)
{
    PolicyLayout l;
    l.P = B > 0 ? count_parts(N, B) : 1;
    l.counts = 0;
    l.weights = up16(B * l.P * 8);
    l.partial = l.weights + up16((B > 0 ? B : 1) * 4);
    l.bytes = l.partial + up16((N + kPolicyChunk - 1) / kPolicyChunk * 3 * 8) + 16;
    return l;
}

static inline bool policy_sizes_ok(int64_t N, int64_t B)
{
    return N >= 0 && N < ((int64_t)1 << 40) && B >= 0 && B < ((int64_t)1 << 31);
}

}  // namespace sfk

using namespace sfk;

SF_API int64_t sf_policy_loss_workspace(int64_t N, int64_t B)
{
    return policy_sizes_ok(N, B) ? policy_layout(N, B).bytes : -1;
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
    if (!out_terms || !workspace || workspace_bytes < l.bytes || !aligned(workspace, 16) || !seq_start)
        return SF_EINVAL;
    const int64_t n_adv = advantage_per_token ? N : B;
    if (N > 0 && (!logp || !old_logp || !out_grad)) return SF_EINVAL;
    if (n_adv > 0 && !advantage) return SF_EINVAL;
    if (!aligned(logp, 4) || !aligned(old_logp, 4) || !aligned(ref_logp, 4) || !aligned(advantage, 4) ||
        !aligned(seq_start, 8) || !aligned(out_terms, 4) || !aligned(out_grad, 4))
        return SF_EINVAL;
    const void* ins[6] = {logp, old_logp, ref_logp, advantage, mask, seq_start};
    const int64_t in_bytes[6] = {N * 4, N * 4, N * 4, n_adv * 4, N, (B + 1) * 8};
    const void* outs[3] = {out_terms, out_grad, workspace};
    const int64_t out_bytes[3] = {16, N * 4, l.bytes};
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
    int64_t* counts = (int64_t*)((char*)workspace + l.counts);
    float* weights = (float*)((char*)workspace + l.weights);
    double* partial = (double*)((char*)workspace + l.partial);
    int64_t chunks = (N + kPolicyChunk - 1) / kPolicyChunk;
    int P = l.P;
    if (N > 0 && B > 0 && reduction != SF_SUM_TOKENS) {
        const int64_t nw = (B * P + kPolicyWG / 64 - 1) / (kPolicyWG / 64);
        void* cargs[] = {(void*)&a, (void*)&P, (void*)&counts};
        int rc = launch((const void*)&k_policy_count, dim3((unsigned)(nw < (1 << 20) ? nw : (1 << 20))),
                        dim3(kPolicyWG), cargs, 0, stream);
        if (rc != SF_OK) return rc;
        void* wargs[] = {(void*)&a, (void*)&P, (void*)&counts, (void*)&weights};
        rc = launch((const void*)&k_policy_weight, dim3(1), dim3(kJoinWG), wargs, 0, stream);
        if (rc != SF_OK) return rc;
    }
    if (N > 0) {
        void* args[] = {(void*)&a, (void*)&weights, (void*)&out_grad, (void*)&partial};
        const int rc = launch((const void*)&k_policy_loss, dim3((unsigned)(chunks < (1 << 20) ? chunks : (1 << 20))),
                              dim3(kPolicyWG), args, 0, stream);
        if (rc != SF_OK) return rc;
    }
    void* jargs[] = {(void*)&chunks, (void*)&kl_coef, (void*)&partial, (void*)&out_terms};
    return launch((const void*)&k_policy_join, dim3(1), dim3(kJoinWG), jargs, 0, stream);
}
