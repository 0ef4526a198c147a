// tokens.hip -- log-probability of the taken token, normaliser and entropy of
// rows of logits (sf_token_logp), and their gradient (sf_token_logp_grad).
//
// Forward: one pass over a row with the running maximum m and, relative to it,
//     s = sum e^((x - m) / T),   u = sum e^((x - m) / T) (x - m) / T
// (the exponent in base 2, c = log2(e) / T): log p, lse and the entropy
// H = log s - u / s come from m, s, u and the taken token's logit.  The
// difference is taken before it is scaled, so the largest term is exactly 1
// and a row of very low logits, all masked alike, still has its distribution.

#include "sf_device.h"
#include "sf_host.h"
#include "sf_train.h"

namespace sfk {

constexpr int kRowWG = 256;

struct RowState {
    float m, s, u;
};

// e^((x - m) / T) and its share of u.  A logit of -inf has e = 0; the bound
// keeps 0 * -inf out of u.  NaN passes through e.
__device__ __forceinline__ void row_add(RowState& a, float x, float ref, float c)
{
    const float t = (x - ref) * c;
    const float e = fast_exp2(t);
    a.s += e;
    a.u = fmaf(e, fmaxf(t, -1000.0f), a.u);
}

// The state's terms relative to a larger maximum.
__device__ __forceinline__ void row_rebase(RowState& a, float m, float ref, float c)
{
    const float t = (a.m - ref) * c;
    const float e = fast_exp2(t);
    a.u = e * fmaf(fmaxf(t, -1000.0f), a.s, a.u);
    a.s *= e;
    a.m = m;
}

// What the terms are taken relative to: 0 while every logit was -inf.
__device__ __forceinline__ float row_ref(float m) { return m == -INFINITY ? 0.0f : m; }

__device__ __forceinline__ RowState row_merge(RowState a, RowState b, float c)
{
    const float m = fmaxf(a.m, b.m), ref = row_ref(m);
    row_rebase(a, m, ref, c);
    row_rebase(b, m, ref, c);
    return {m, a.s + b.s, a.u + b.u};
}

__device__ __forceinline__ RowState row_wave(RowState a, float c)
{
    for (int off = 32; off > 0; off >>= 1) {
        const RowState b = {__shfl_xor(a.m, off, 64), __shfl_xor(a.s, off, 64), __shfl_xor(a.u, off, 64)};
        a = row_merge(a, b, c);
    }
    return a;
}

__device__ __forceinline__ void row_write(RowState a, float xt, float inv_t, int64_t i, float* logp,
                                          float* lse, float* entropy)
{
    if (a.m == -INFINITY && a.s == 0.0f) {
        logp[i] = lse[i] = -INFINITY;
        if (entropy) entropy[i] = 0.0f;
        return;
    }
    const float ls = logf(a.s);
    logp[i] = (xt - a.m) * inv_t - ls;
    lse[i] = fmaf(a.m, inv_t, ls);
    if (entropy) entropy[i] = fmaxf(ls - kLn2 * (a.u / a.s), 0.0f) + 0.0f * a.s;
}

// One workgroup per (row, part): part p of P takes the p-th share of the row's
// 16-byte vectors; with P > 1 its state goes to the workspace.
template <int DT>
__global__ __launch_bounds__(kRowWG) void k_token_logp(const typename Elem<DT>::T* __restrict__ logits,
                                                       int64_t N, int64_t V, int64_t stride,
                                                       const int64_t* __restrict__ targets, float inv_t,
                                                       int P, float* __restrict__ logp,
                                                       float* __restrict__ lse, float* __restrict__ entropy,
                                                       RowState* __restrict__ parts)
{
    typedef typename Elem<DT>::T T;
    constexpr int E = kVec<DT>;
    constexpr int U = 4;
    __shared__ RowState wave_state[kRowWG / 64];
    const float c = inv_t * kLog2e;
    const int tid = threadIdx.x;
    for (int64_t blk = blockIdx.x; blk < N * P; blk += gridDim.x) {
        const int64_t i = blk / P;
        const int p = (int)(blk - i * P);
        const int64_t t = targets[i];
        if (t < 0 || t >= V) {
            if (tid == 0 && p == 0) {
                logp[i] = lse[i] = 0.0f;
                if (entropy) entropy[i] = 0.0f;
            }
            continue;
        }
        const T* row = logits + i * stride;
        const int64_t head = head_elems<DT>(row, V);
        const int64_t nv = (V - head) / E;
        const int64_t v0 = nv * p / P, v1 = nv * (p + 1) / P;
        RowState a = {-INFINITY, 0.0f, 0.0f};
        const T* body = row + head;
        for (int64_t v = v0 + tid; v < v1; v += U * kRowWG) {
            VecU<DT> x[U];
            int n = 0;
#pragma unroll
            for (int k = 0; k < U; ++k) {
                const int64_t w = v + k * kRowWG;
                x[k] = *(const VecU<DT>*)(body + (w < v1 ? w : v) * E);
                n += w < v1;
            }
            float m = a.m;
#pragma unroll
            for (int k = 0; k < U; ++k)
#pragma unroll
                for (int j = 0; j < E; ++j) m = fmaxf(m, (float)x[k][j]);
            const float ref = row_ref(m);
            row_rebase(a, m, ref, c);
#pragma unroll
            for (int k = 0; k < U; ++k)
                if (k < n)
#pragma unroll
                    for (int j = 0; j < E; ++j) row_add(a, (float)x[k][j], ref, c);
        }
        // the elements before the first and after the last whole vector
        const int64_t tail0 = head + nv * E;
        const int nh = p == 0 ? (int)head : 0;
        const int nt = p == P - 1 ? (int)(V - tail0) : 0;
        if (tid < nh + nt) {
            const float x = (float)row[tid < nh ? tid : tail0 + (tid - nh)];
            const float m = fmaxf(a.m, x), ref = row_ref(m);
            row_rebase(a, m, ref, c);
            row_add(a, x, ref, c);
        }
        a = row_wave(a, c);
        if ((tid & 63) == 0) wave_state[tid >> 6] = a;
        __syncthreads();
        if (tid == 0) {
#pragma unroll
            for (int w = 1; w < kRowWG / 64; ++w) a = row_merge(a, wave_state[w], c);
            if (P == 1)
                row_write(a, (float)row[t], inv_t, i, logp, lse, entropy);
            else
                parts[blk] = a;
        }
        __syncthreads();
    }
}

// Joins a row's parts: one wave per row.
template <int DT>
__global__ __launch_bounds__(kRowWG) void k_token_logp_join(const typename Elem<DT>::T* __restrict__ logits,
                                                            int64_t N, int64_t V, int64_t stride,
                                                            const int64_t* __restrict__ targets, float inv_t,
                                                            int P, float* __restrict__ logp,
                                                            float* __restrict__ lse, float* __restrict__ entropy,
                                                            const RowState* __restrict__ parts)
{
    const float c = inv_t * kLog2e;
    const int lane = threadIdx.x & 63;
    const int64_t waves = (int64_t)gridDim.x * (kRowWG / 64);
    for (int64_t i = (int64_t)blockIdx.x * (kRowWG / 64) + (threadIdx.x >> 6); i < N; i += waves) {
        const int64_t t = targets[i];
        if (t < 0 || t >= V) continue;
        RowState a = {-INFINITY, 0.0f, 0.0f};
        for (int p = lane; p < P; p += 64) a = row_merge(a, parts[i * P + p], c);
        a = row_wave(a, c);
        if (lane == 0) row_write(a, (float)logits[i * stride + t], inv_t, i, logp, lse, entropy);
    }
}

// out = inv_t (g ([j = t] - p) - h p (log p + H)): element by element from the
// row's lse; one workgroup per (row, kGradVecs vectors).
constexpr int kGradU = 4;
constexpr int kGradVecs = kRowWG * kGradU;

template <int DT>
__global__ __launch_bounds__(kRowWG) void k_token_logp_grad(const typename Elem<DT>::T* logits, int64_t N,
                                                            int64_t V, int64_t stride,
                                                            const int64_t* __restrict__ targets, float inv_t,
                                                            const float* __restrict__ lse,
                                                            const float* __restrict__ grad_logp,
                                                            const float* __restrict__ entropy,
                                                            const float* __restrict__ grad_entropy,
                                                            typename Elem<DT>::T* out, int64_t out_stride,
                                                            int64_t chunks)
{
    typedef typename Elem<DT>::T T;
    constexpr int E = kVec<DT>;
    const int tid = threadIdx.x;
    for (int64_t blk = blockIdx.x; blk < N * chunks; blk += gridDim.x) {
        const int64_t i = blk / chunks;
        const int64_t ch = blk - i * chunks;
        const int64_t t = targets[i];
        T* o = out + i * out_stride;
        const T* row = logits + i * stride;
        const int64_t head = head_elems<DT>(o, V);
        const int64_t nv = (V - head) / E, tail0 = head + nv * E;
        const float l = lse[i];
        const bool none = t < 0 || t >= V || l == -INFINITY;
        const float g = none ? 0.0f : grad_logp[i] * inv_t;
        const float h = none || !grad_entropy ? 0.0f : grad_entropy[i] * inv_t;
        // -(g + h (log p + H)) = -(k0 + h log p)
        const float k0 = h != 0.0f ? fmaf(h, entropy[i], g) : g;
        auto value = [&](float x, int64_t j) {
            const float q = fmaf(x, inv_t, -l);  // log p
            const float p = fast_exp2(q * kLog2e);
            const float y = -p * fmaf(h, fmaxf(q, -1000.0f), k0);
            return j == t ? y + g : y;
        };
        const int64_t v0 = ch * kGradVecs;
#pragma unroll
        for (int k = 0; k < kGradU; ++k) {
            const int64_t v = v0 + k * kRowWG + tid;
            if (v >= nv) break;
            const int64_t j0 = head + v * E;
            VecU<DT> y;
            if (none) {
#pragma unroll
                for (int j = 0; j < E; ++j) y[j] = (T)0.0f;
            } else {
                const VecU<DT> x = *(const VecU<DT>*)(row + j0);
#pragma unroll
                for (int j = 0; j < E; ++j) y[j] = (T)value((float)x[j], j0 + j);
            }
            *(VecU<DT>*)(o + j0) = y;
        }
        if (ch == 0 && tid < (int)(head + V - tail0)) {
            const int64_t j = tid < head ? tid : tail0 + (tid - head);
            o[j] = none ? (T)0.0f : (T)value((float)row[j], j);
        }
    }
}

// Parts of a row: enough workgroups for the chip, at least 16 KB each.
static inline int row_parts(int64_t N, int64_t V)
{
    const int64_t want = (1024 + N - 1) / N;
    const int64_t most = V / 8192;
    const int64_t p = want < most ? want : most;
    return p < 1 ? 1 : p > 64 ? 64 : (int)p;
}

static inline bool rows_ok(int32_t dtype, int64_t N, int64_t V, int64_t stride, float inv_t)
{
    return (dtype == SF_F32 || dtype == SF_BF16 || dtype == SF_F16) && N >= 0 && V >= 1 &&
           V <= ((int64_t)1 << 30) && stride >= V && inv_t > 0.0f && inv_t <= kF32Max &&
           (N == 0 || stride <= (((int64_t)1 << 56) / N));
}

static inline unsigned grid_of(int64_t n) { return (unsigned)(n < (1 << 30) ? n : (1 << 30)); }

}  // namespace sfk

using namespace sfk;

SF_API int64_t sf_token_logp_workspace(int64_t N, int64_t V)
{
    if (N < 0 || V < 1 || V > ((int64_t)1 << 30) || N > ((int64_t)1 << 56)) return -1;
    if (N == 0) return 0;
    const int P = row_parts(N, V);
    return P == 1 ? 0 : N * P * (int64_t)sizeof(RowState);
}

SF_API int sf_token_logp(const void* logits, int32_t dtype, int64_t N, int64_t V, int64_t row_stride,
                         const int64_t* targets, float inv_temperature, float* out_logp, float* out_lse,
                         float* out_entropy, void* workspace, int64_t workspace_bytes, sf_stream_t stream)
{
    if (!rows_ok(dtype, N, V, row_stride, inv_temperature)) return SF_EINVAL;
    if (N == 0) return SF_OK;
    const int64_t need = sf_token_logp_workspace(N, V);
    if (!logits || !targets || !out_logp || !out_lse || (need > 0 && !workspace) || workspace_bytes < need)
        return SF_EINVAL;
    const int64_t in_bytes = ((N - 1) * row_stride + V) * elem_size(dtype);
    if (!aligned(logits, elem_size(dtype)) || !aligned(targets, 8) || !aligned(out_logp, 4) ||
        !aligned(out_lse, 4) || !aligned(out_entropy, 4) || (need > 0 && !aligned(workspace, 16)))
        return SF_EINVAL;
    const void* outs[4] = {out_logp, out_lse, out_entropy, workspace};
    const int64_t sizes[4] = {N * 4, N * 4, out_entropy ? N * 4 : 0, need};
    for (int a = 0; a < 4; ++a) {
        if (sizes[a] == 0) continue;
        if (!disjoint(outs[a], sizes[a], logits, in_bytes) || !disjoint(outs[a], sizes[a], targets, N * 8))
            return SF_EINVAL;
        for (int b = a + 1; b < 4; ++b)
            if (sizes[b] > 0 && !disjoint(outs[a], sizes[a], outs[b], sizes[b])) return SF_EINVAL;
    }
    int P = row_parts(N, V);
    void* args[] = {(void*)&logits,   (void*)&N,       (void*)&V,           (void*)&row_stride,
                    (void*)&targets,  (void*)&inv_temperature, (void*)&P,   (void*)&out_logp,
                    (void*)&out_lse,  (void*)&out_entropy,     (void*)&workspace};
    const void* fn[3] = {(const void*)&k_token_logp<SF_F32>, (const void*)&k_token_logp<SF_BF16>,
                         (const void*)&k_token_logp<SF_F16>};
    const void* join[3] = {(const void*)&k_token_logp_join<SF_F32>, (const void*)&k_token_logp_join<SF_BF16>,
                           (const void*)&k_token_logp_join<SF_F16>};
    const int rc = launch(fn[dtype], dim3(grid_of(N * P)), dim3(kRowWG), args, 0, stream);
    if (rc != SF_OK || P == 1) return rc;
    return launch(join[dtype], dim3(grid_of((N + kRowWG / 64 - 1) / (kRowWG / 64))), dim3(kRowWG), args, 0, stream);
}

SF_API int sf_token_logp_grad(const void* logits, int32_t dtype, int64_t N, int64_t V, int64_t row_stride,
                              const int64_t* targets, float inv_temperature, const float* lse,
                              const float* grad_logp, const float* entropy, const float* grad_entropy,
                              void* out_grad, int64_t out_row_stride, sf_stream_t stream)
{
    if (!rows_ok(dtype, N, V, row_stride, inv_temperature) || !rows_ok(dtype, N, V, out_row_stride, 1.0f))
        return SF_EINVAL;
    if (N == 0) return SF_OK;
    if (!logits || !targets || !lse || !grad_logp || !out_grad || (grad_entropy && !entropy)) return SF_EINVAL;
    const int b = elem_size(dtype);
    if (!aligned(logits, b) || !aligned(out_grad, b) || !aligned(targets, 8) || !aligned(lse, 4) ||
        !aligned(grad_logp, 4) || !aligned(entropy, 4) || !aligned(grad_entropy, 4))
        return SF_EINVAL;
    const int64_t in_bytes = ((N - 1) * row_stride + V) * b, out_bytes = ((N - 1) * out_row_stride + V) * b;
    const bool in_place = out_grad == logits && out_row_stride == row_stride;
    if (!in_place && !disjoint(logits, in_bytes, out_grad, out_bytes)) return SF_EINVAL;
    const void* ins[5] = {targets, lse, grad_logp, entropy, grad_entropy};
    for (int a = 0; a < 5; ++a)
        if (ins[a] && !disjoint(ins[a], N * (a == 0 ? 8 : 4), out_grad, out_bytes)) return SF_EINVAL;
    const int64_t e = 16 / b;
    int64_t chunks = (V / e + kGradVecs - 1) / kGradVecs;
    if (chunks < 1) chunks = 1;
    void* args[] = {(void*)&logits,  (void*)&N,         (void*)&V,       (void*)&row_stride,   (void*)&targets,
                    (void*)&inv_temperature, (void*)&lse, (void*)&grad_logp, (void*)&entropy,
                    (void*)&grad_entropy, (void*)&out_grad, (void*)&out_row_stride, (void*)&chunks};
    const void* fn[3] = {(const void*)&k_token_logp_grad<SF_F32>, (const void*)&k_token_logp_grad<SF_BF16>,
                         (const void*)&k_token_logp_grad<SF_F16>};
    return launch(fn[dtype], dim3(grid_of(N * chunks)), dim3(kRowWG), args, 0, stream);
}
