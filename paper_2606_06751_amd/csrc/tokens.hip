// tokens.hip -- log-probability of the taken token, normaliser and entropy of
// rows of logits (sf_token_logp), and their gradient (sf_token_logp_grad).
//
// Forward: one pass over a row.  With c = log2(e) / T, each wave keeps a
// reference (b, R), R a whole number, and its lanes
//     s = sum 2^t,   u = sum 2^t t,   t = (x - b) c - R,
// from which log p, lse and the entropy H = log s - ln 2 u / s follow.  b is 0
// but for rows of huge logits, so t is one multiply-add whose only error is its
// own rounding, and a change of R scales by a power of two, without any.
//
// What bounds it is HBM and, close behind, the VALU: one exponential (a quarter
// of the VALU's rate), a conversion, two multiply-adds, an add and a bound per
// logit.  So the running maximum is not taken per logit: a chunk is added
// relative to the wave's reference as it stands, and only where its sum shows
// that a logit lies far above is the chunk done again with its maximum.  The
// reference is a wave's, not a lane's, so that this is rare.  (Without the bound,
// -inf logits sent every chunk the second way: 144 against 94 us at 4096 x 65536
// bf16 with a hundredth of them masked, 89 against 92 without masks.)
// 4096 x 131072 bf16: 174 us, 6.2 TB/s, 87% of the 7.13 TB/s plain read; loads
// that do not go past the caches gave 103 instead of 92 us at 4096 x 65536.

#include "sf_device.h"
#include "sf_host.h"
#include "sf_train.h"

namespace sfk {

constexpr int kRowWG = 256;

// Terms relative to (b, R): s = sum 2^t, u = sum 2^t t with t = (x - b) c - R.
// Either b is 0 and R a whole number near the largest x c, so that t is one
// multiply-add of x whose only error is its own rounding, or, for huge logits, R
// is 0 and b the largest x.
struct RowState {
    float b, R, s, u;  // R = -inf: nothing but -inf so far
};

struct RowScale {
    float inv_t, c, eps;  // c (1 + eps) = inv_t log2(e) more exactly than c is
};

// A reference's place on the exponents' scale, -inf where there is none yet.
__device__ __forceinline__ double row_height(float b, float R, float c) { return fma((double)b, (double)c, (double)R); }

// The state's sums relative to another reference.  In 64 bits, where nothing
// of the type's range overflows; a state without terms weighs 0.
__device__ __forceinline__ void row_rebase(RowState& a, float b, float R, float c)
{
    const float t = (float)fma((double)a.b - (double)b, (double)c, (double)a.R - (double)R);
    const float e = fast_exp2(t);
    a.u = e * fmaf(fmaxf(t, -1000.0f), a.s, a.u);
    a.s *= e;
    a.b = b;
    a.R = R;
}


// Vectors of a chunk per lane (2, 4, 8: 98, 92, 95 us at 4096 x 65536, 34, 28, 27
// at 2048 x 32000; 8 spills with 1024 threads).
constexpr int kRowU = 4;

// Adds `live` vectors a lane and an edge logit (-inf: none) after taking their
// maximum.  Lanes without a logit hold -inf, whose e is 0; the bound keeps
// 0 * -inf out of u; NaN passes through e.  Where |m c| reaches 2^22, and
// its rounding is no longer small beside 1, the reference is the maximum
// itself, taken off before the product: a row of very low logits, all masked
// alike, keeps its distribution.
template <int DT>
__device__ __forceinline__ void row_add(RowState& a, const VecU<DT> (&y)[kRowU], int live, float edge, float c)
{
    constexpr int E = kVec<DT>, U = kRowU;
    float m = edge;
#pragma unroll
    for (int k = 0; k < U; ++k)
        if (k < live)
#pragma unroll
            for (int j = 0; j < E; ++j) m = fmaxf(m, (float)y[k][j]);
    m = wave_max_f32(m);
    if (m != -INFINITY) {
        const float top = m * c;
        const bool huge = !(fabsf(top) < 4194304.0f);
        const float b = huge ? m : 0.0f, R = huge ? 0.0f : rintf(top);
        if (a.R == -INFINITY) {  // the first: nothing to scale
            a.b = b;
            a.R = R;
        } else if (row_height(b, R, c) > row_height(a.b, a.R, c)) {
            row_rebase(a, b, R, c);
        }
    }
    const float R = a.R == -INFINITY ? 0.0f : a.R;
    auto add = [&](float v) {
        const float t = fmaf(v - a.b, c, -R);
        const float e = fast_exp2(t);
        a.s += e;
        a.u = fmaf(e, fmaxf(t, -1000.0f), a.u);
    };
    add(edge);
#pragma unroll
    for (int k = 0; k < U; ++k)
        if (k < live)
#pragma unroll
            for (int j = 0; j < E; ++j) add((float)y[k][j]);
}

// Adds a full chunk relative to the reference as it is; false where that would
// lose digits (a term far above 1).
template <int DT>
__device__ __forceinline__ bool row_try(RowState& a, const VecU<DT> (&y)[kRowU], float c)
{
    constexpr int E = kVec<DT>, U = kRowU, K = U * E;
    float s = 0.0f, u = 0.0f;
#pragma unroll
    for (int k = 0; k < U; ++k)
#pragma unroll
        for (int j = 0; j < E; ++j) {
            const float t = fmaf((float)y[k][j], c, -a.R);
            const float e = fast_exp2(t);
            s += e;
            u = fmaf(e, fmaxf(t, -1000.0f), u);
        }
    // no term above 2^(1/2) gives K * 1.42 at most.  (u is not a number only
    // where s is not; asked for here, it is summed beside s.  Else the compiler
    // sums it after the branch, from values that take 105 registers, not 66.)
    if (__any(!(s < 2.0f * K) || u != u)) return false;
    a.s += s;
    a.u += u;
    return true;
}

// The wave's sums in every lane.
__device__ __forceinline__ RowState row_wave(RowState a)
{
    a.s = wave_sum_f32(a.s);
    a.u = wave_sum_f32(a.u);
    return a;
}

// Two states as one, relative to the higher reference.
__device__ __forceinline__ RowState row_merge(RowState a, RowState o, float c)
{
    if (row_height(o.b, o.R, c) > row_height(a.b, a.R, c))
        row_rebase(a, o.b, o.R, c);
    else if (a.R != -INFINITY)
        row_rebase(o, a.b, a.R, c);
    a.s += o.s;
    a.u += o.u;
    return a;
}

// Joins the states that a wave's lanes hold, in every lane.  Without references
// of huge logits that is a maximum and powers of two.
__device__ __forceinline__ RowState row_join(RowState a, float c)
{
    if (__all(a.b == 0.0f)) {
        const float top = wave_max_f32(a.R);
        if (top != -INFINITY) {
            const float t = a.R - top, e = fast_exp2(t);
            a.u = e * fmaf(fmaxf(t, -1000.0f), a.s, a.u);
            a.s *= e;
            a.R = top;
        }
        return row_wave(a);
    }
#pragma unroll 1
    for (int off = 32; off > 0; off >>= 1)
        a = row_merge(a, {__shfl_xor(a.b, off, 64), __shfl_xor(a.R, off, 64), __shfl_xor(a.s, off, 64),
                          __shfl_xor(a.u, off, 64)}, c);
    return a;
}

__device__ __forceinline__ void row_write(RowState a, float xt, RowScale z, int64_t i, float* logp, float* lse,
                                          float* entropy)
{
    if (a.s == 0.0f) {
        logp[i] = lse[i] = -INFINITY;
        if (entropy) entropy[i] = 0.0f;
        return;
    }
    const float ls = logf(a.s), mean = a.u / a.s;  // mean exponent
    const float t = fmaf(xt - a.b, z.c, -a.R);
    const float turn = z.eps * kLn2;
    // the exponents are off by c's own rounding, which turns log p by their
    // distance from the mean and lse by the mean
    logp[i] = fmaf(t, kLn2, -ls) + (t > -1000.0f ? turn * (t - mean) : 0.0f);
    // held within the floats: -inf is for rows that have no distribution
    const float l = a.b == 0.0f ? fmaf(a.R, kLn2, fmaf(a.R, kLn2Low, ls)) + turn * (a.R + mean) : fmaf(a.b, z.inv_t, ls);
    lse[i] = fabsf(l) == INFINITY ? copysignf(kF32Max, l) : l;
    if (entropy) {
        const float h = ls - kLn2 * mean;
        entropy[i] = h < 0.0f ? 0.0f : h;
    }
}

// WAVES waves per row; a workgroup of WG threads takes WG / 64 / WAVES rows,
// or, with gridDim.y > 1, part blockIdx.y of one row (`share` 16-byte vectors
// each), whose state goes to the workspace.  The elements before the first and
// after the last whole vector join the last chunk, one a lane.  Every chunk
// that needs its maximum goes through one piece of code: where few rows give a
// compute unit little work, fetching the code is a good part of the time.
template <int DT, int WG, int WAVES>
__global__ __launch_bounds__(WG) void k_token_logp(const typename Elem<DT>::T* __restrict__ logits, int64_t N, int V,
                                                   int64_t stride, const int64_t* __restrict__ targets, RowScale z,
                                                   int share, float* __restrict__ logp, float* __restrict__ lse,
                                                   float* __restrict__ entropy, RowState* __restrict__ parts)
{
    typedef typename Elem<DT>::T T;
    constexpr int E = kVec<DT>;
    constexpr int U = kRowU;
    constexpr int LANES = WAVES * 64;
    constexpr int ROWS = WG / LANES;
    static_assert(ROWS == 1 || WAVES == 1, "rows of one wave, or one row");
    __shared__ RowState wave_state[WAVES];
    const int tid = ROWS == 1 ? threadIdx.x : threadIdx.x & 63;  // within the row
    const int wave0 = __builtin_amdgcn_readfirstlane(tid & ~63);
    const int p = ROWS == 1 ? blockIdx.y : 0, P = ROWS == 1 ? gridDim.y : 1;
    const int64_t step = (int64_t)gridDim.x * ROWS;
    for (int64_t i = (int64_t)blockIdx.x * ROWS + (ROWS == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6));
         i < N; i += step) {
        const int64_t t = targets[i];
        if (t < 0 || t >= V) {
            if (tid == 0 && p == 0) {
                logp[i] = lse[i] = 0.0f;
                if (entropy) entropy[i] = 0.0f;
            }
            continue;
        }
        const T* row = logits + i * stride;
        const int head = (int)head_elems<DT, WAVES == 1 ? 64 : 128>(row, V);
        const int nv = (V - head) / E, tail0 = head + nv * E;
        const T* body = row + head;
        const int v0 = min(nv, p * share), v1 = min(nv, v0 + share);
        const int nh = p == 0 ? head : 0, nt = p == P - 1 ? V - tail0 : 0;
        const T xt = row[t];
        const bool has_edge = tid < nh + nt;
        const T edge = row[has_edge ? (tid < nh ? tid : tail0 + (tid - nh)) : 0];
        RowState a = {0.0f, -INFINITY, 0.0f, 0.0f};
        for (int w = v0 + wave0;; w += U * LANES) {
            const int v = w + (tid & 63);
            const bool last = w + U * LANES >= v1;
            VecU<DT> y[U];
            if (!last) {
#pragma unroll
                for (int k = 0; k < U; ++k) y[k] = __builtin_nontemporal_load((const VecU<DT>*)(body + (int64_t)(v + k * LANES) * E));
                if (a.b == 0.0f && a.R != -INFINITY && row_try<DT>(a, y, z.c)) continue;
            } else {
#pragma unroll
                for (int k = 0; k < U; ++k) {
                    y[k] = (VecU<DT>)(T)-INFINITY;
                    if (v + k * LANES < v1) y[k] = __builtin_nontemporal_load((const VecU<DT>*)(body + (int64_t)(v + k * LANES) * E));
                }
            }
            const int live = last ? (v1 - w + LANES - 1) / LANES : U;
            row_add<DT>(a, y, live, last && has_edge ? (float)edge : -INFINITY, z.c);
            if (last) break;
        }
        a = row_wave(a);
        if (ROWS > 1) {
            if (tid == 0) row_write(a, (float)xt, z, i, logp, lse, entropy);
            continue;
        }
        if ((tid & 63) == 0) wave_state[tid >> 6] = a;
        __syncthreads();
        if (tid < 64) {
            a = tid < WAVES ? wave_state[tid] : RowState{0.0f, -INFINITY, 0.0f, 0.0f};
            a = row_join(a, z.c);
            if (tid == 0) {
                if (P == 1)
                    row_write(a, (float)xt, z, i, logp, lse, entropy);
                else
                    parts[i * P + p] = a;
            }
        }
        __syncthreads();
    }
}

// Joins a row's parts: one wave per row.
template <int DT>
__global__ __launch_bounds__(kRowWG) void k_token_logp_join(const typename Elem<DT>::T* __restrict__ logits, int64_t N,
                                                            int V, int64_t stride, const int64_t* __restrict__ targets,
                                                            RowScale z, int P, float* __restrict__ logp,
                                                            float* __restrict__ lse, float* __restrict__ entropy,
                                                            const RowState* __restrict__ parts)
{
    const float c = z.c;
    const int lane = threadIdx.x & 63;
    const int64_t waves = (int64_t)gridDim.x * (kRowWG / 64);
    for (int64_t i = (int64_t)blockIdx.x * (kRowWG / 64) + (threadIdx.x >> 6); i < N; i += waves) {
        const int64_t t = targets[i];
        if (t < 0 || t >= V) continue;
        const float xt = (float)logits[i * stride + t];
        RowState a = {0.0f, -INFINITY, 0.0f, 0.0f};
        for (int p = lane; p < P; p += 64) a = row_merge(a, parts[i * P + p], c);
        a = row_join(a, c);
        if (lane == 0) row_write(a, xt, z, i, logp, lse, entropy);
    }
}

// out = inv_t (g ([j = t] - p) - h p (log p + H)): element by element from the
// row's lse, bound by HBM.  LANES lanes take chunk blockIdx.x of a row, kGradU
// vectors each, aligned by the output: a workgroup of 256 one chunk, or a wave
// each of 4 short rows (16000 x 515 f16: 8.4 us, by workgroups 14).  Measured at
// 16411 x 131072 bf16, vectors a lane / loads and stores past the caches or not:
// 1 / both 1212, 2 / loads 1210, 2 / both 1298, 2 / none 1237, 4 / both 1362 us;
// at 512 x 100003 41.5, 37.1, 37.8, 41.3, 39.1.  (8 waves a SIMD are asked for:
// the code of far rows would take registers that leave 6.)
constexpr int kGradU = 2;
// From this |lse| on (2^16) its own rounding, up to 2^-24 of it and with that
// an error of log p, passes that of a bfloat16, 2^-9 of p, and from 2^24 on
// nothing is left of p.  Such a row takes its normaliser from its logits again.
constexpr float kFarLse = 65536.0f;

// -p (g + h (log p + H)) = -p (k0 + h q), q = log p; the bound keeps 0 * -inf out.
// exp2f keeps probabilities below 2^-126, which h and T may raise again.
__device__ __forceinline__ float grad_term(float q, float h, float k0)
{
    return -exp2f(q * kLog2e) * fmaf(h, fmaxf(q, -1000.0f), k0);
}

// Such a row by LANES lanes, each of which reads the elements that it writes:
// log p = (x - m) / T - log s with the row's maximum m, s = sum e^((x - m) / T).
// The row is its `nv` vectors from `head` on and the elements around them.  (All
// rows of 1024 x 65536 bf16 far: 120 us, none 44; two vectors a lane in flight
// take more registers than leave 8 waves.)
template <int DT, int LANES>
__device__ __forceinline__ void far_row(const typename Elem<DT>::T* row, int V, int head, int nv, float inv_t, int tid,
                                        float* part, int at, float g, float h, float entropy, typename Elem<DT>::T* o)
{
    typedef typename Elem<DT>::T T;
    constexpr int E = kVec<DT>, NW = LANES / 64;
    const VecU<DT>* xv = (const VecU<DT>*)(row + head);
    VecU<DT>* ov = (VecU<DT>*)(o + head);
    const int tail0 = head + nv * E;
    const bool edge = tid < head + V - tail0;
    const int je = edge ? (tid < head ? tid : tail0 + (tid - head)) : 0;
    const float xe = edge ? (float)row[je] : -INFINITY;
    auto vectors = [&](auto f) {
#pragma unroll 1
        for (int v = tid; v < nv; v += LANES) f(xv[v], v);
    };
    float m = xe, s = 0.0f;
    vectors([&](const VecU<DT>& x, int) {
#pragma unroll
        for (int j = 0; j < E; ++j) m = fmaxf(m, (float)x[j]);
    });
    m = wave_max_f32(m);
    if (NW > 1) {
        __syncthreads();  // a former row's sums are read
        if ((tid & 63) == 0) part[tid >> 6] = m;
        __syncthreads();
        for (int w = 0; w < NW; ++w) m = fmaxf(m, part[w]);
    }
    auto add = [&](float x) { s += fast_exp2((x - m) * inv_t * kLog2e); };
    vectors([&](const VecU<DT>& x, int) {
#pragma unroll
        for (int j = 0; j < E; ++j) add((float)x[j]);
    });
    add(xe);
    s = wave_sum_f32(s);
    if (NW > 1) {
        if ((tid & 63) == 0) part[NW + (tid >> 6)] = s;
        __syncthreads();
        s = 0.0f;
        for (int w = 0; w < NW; ++w) s += part[NW + w];
    }
    const float ls = logf(s), k0 = fmaf(h, entropy, g);
    auto value = [&](float x, int j) { return (T)(grad_term(fmaf(x - m, inv_t, -ls), h, k0) + (j == at ? g : 0.0f)); };
    vectors([&](const VecU<DT>& x, int v) {
        VecU<DT> r;
#pragma unroll
        for (int j = 0; j < E; ++j) r[j] = value((float)x[j], head + v * E + j);
        ov[v] = r;
    });
    if (edge) o[je] = value(xe, je);
}

template <int DT, int LANES>
__global__ __launch_bounds__(kRowWG, 8) void k_token_logp_grad(const typename Elem<DT>::T* logits, int64_t N, int V,
                                                               int64_t stride, const int64_t* __restrict__ targets,
                                                               float inv_t, const float* __restrict__ lse,
                                                               const float* __restrict__ grad_logp,
                                                               const float* __restrict__ entropy,
                                                               const float* __restrict__ grad_entropy,
                                                               typename Elem<DT>::T* out, int64_t out_stride)
{
    typedef typename Elem<DT>::T T;
    constexpr int E = kVec<DT>;
    constexpr int ROWS = kRowWG / LANES;
    __shared__ float part[2 * LANES / 64];
    const int tid = threadIdx.x & (LANES - 1);
    const int sub = ROWS == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / LANES);
    for (int64_t i = (int64_t)blockIdx.y * ROWS + sub; i < N; i += (int64_t)gridDim.y * ROWS) {
        const int64_t t = targets[i];
        const float l = lse[i];
        T* o = out + i * out_stride;
        const T* row = logits + i * stride;
        const int head = (int)head_elems<DT, LANES == 64 ? 64 : 128>(o, V);
        const int nv = (V - head) / E, tail0 = head + nv * E;
        const int v0 = (int)blockIdx.x * (kGradU * LANES) + tid;
        VecU<DT>* ov = (VecU<DT>*)(o + head);
        const VecU<DT>* xv = (const VecU<DT>*)(row + head);
        const bool edge = blockIdx.x == 0 && tid < head + V - tail0;
        const int je = tid < head ? tid : tail0 + (tid - head);
        if (t < 0 || t >= V || l == -INFINITY) {
#pragma unroll
            for (int k = 0; k < kGradU; ++k)
                if (v0 + k * LANES < nv) ov[v0 + k * LANES] = (VecU<DT>)(T)0.0f;
            if (edge) o[je] = (T)0.0f;
            continue;
        }
        if (fabsf(l) >= kFarLse) {
            // the whole row by the lanes of one chunk, so that none reads what another wrote in
            // place; of another chunk row by row, as workgroups go to the XCDs in turn (the
            // first of each: 599 us in place of 120)
            if (blockIdx.x == (unsigned)i % gridDim.x)
                far_row<DT, LANES>(row, V, head, nv, inv_t, tid, part, (int)t, grad_logp[i] * inv_t,
                                   grad_entropy ? grad_entropy[i] * inv_t : 0.0f, grad_entropy ? entropy[i] : 0.0f, o);
            continue;
        }
        VecU<DT> x[kGradU];
#pragma unroll
        for (int k = 0; k < kGradU; ++k)
            if (v0 + k * LANES < nv) x[k] = __builtin_nontemporal_load(xv + v0 + k * LANES);
        const T xe = row[edge ? je : 0];
        const float g = grad_logp[i] * inv_t;
        const float h = grad_entropy ? grad_entropy[i] * inv_t : 0.0f;
        const float k0 = grad_entropy ? fmaf(h, entropy[i], g) : g;
        const int at = (int)t;
        auto value = [&](float z) { return grad_term(fmaf(z, inv_t, -l), h, k0); };
#pragma unroll
        for (int k = 0; k < kGradU; ++k) {
            const int v = v0 + k * LANES;
            if (v < nv) {
                float y[E];
#pragma unroll
                for (int j = 0; j < E; ++j) y[j] = value((float)x[k][j]);
                const int hit = at - (head + v * E);  // the taken token's place, if here
                if ((unsigned)hit < (unsigned)E)
#pragma unroll
                    for (int j = 0; j < E; ++j) y[j] += j == hit ? g : 0.0f;
                VecU<DT> r;
#pragma unroll
                for (int j = 0; j < E; ++j) r[j] = (T)y[j];
                ov[v] = r;
            }
        }
        if (edge) o[je] = (T)(value((float)xe) + (je == at ? g : 0.0f));
    }
}

// How rows are shared out: a wave each (wg = 64), a workgroup of wg threads
// each, or P such workgroups each.
struct RowShape {
    int wg, P;
};

// Measured (bf16, us, a wave / 256 / 1024 threads a row / 256 threads in parts):
//   300 x 1000: 3.4 / 4.0 / 6.4;  4096 x 16000: 27 / 30 / 64;  2048 x 32000:
//   26.5 / 28.3 / 46;  8192 x 8000: 27.5 / 28.5;  8192 x 32003: 96 / 89;
//   4096 x 65536: 100 / 94 / 137;  1024 x 16000: 13.0 / 11.7 / 18;
//   512 x 16000: 11.5 / 7.8 / 9.5;  256 x 32000: 17.8 / 8.7 / 7.5;  128 x 65536:
//   32 / 11.8 / 9.1 / 9.9;  64 x 131072: 59 / 19 / 12.5 / 9.9;  1 x 65536: 25 / 10 /
//   7.8 / 5.2;  1 x 262144: 105 / 31 / 18 / 6.3.
// Parts cost a second launch, so a row of up to 128 KB stays with one workgroup.
static inline RowShape row_shape(int64_t N, int64_t V, int bytes)
{
    const int64_t row = V * bytes;
    if (row <= 4096 || (N >= 2048 && row <= (N < 8192 ? 65536 : 20480))) return {64, 1};
    if (row > 131072 && N <= 64) {
        const int64_t want = 1024 / N, most = row / 8192;
        return {256, (int)(want < most ? want : most)};
    }
    return {N <= 256 ? 1024 : 256, 1};
}

static inline bool rows_ok(int32_t dtype, int64_t N, int64_t V, int64_t stride, float inv_t)
{
    return (dtype == SF_F32 || dtype == SF_BF16 || dtype == SF_F16) && N >= 0 && V >= 1 &&
           V <= ((int64_t)1 << 30) && stride >= V && inv_t > 0.0f && inv_t <= 0x1p100f &&
           (N == 0 || stride <= (((int64_t)1 << 56) / N));
}

// Workgroups for n units; the kernels take the rest in turns.  (A launch has
// fewer than 2^32 threads a dimension.)
static inline unsigned grid_of(int64_t n) { return (unsigned)(n < (1 << 21) ? n : (1 << 21)); }

}  // namespace sfk

using namespace sfk;

SF_API int64_t sf_token_logp_workspace(int32_t dtype, int64_t N, int64_t V)
{
    if (!rows_ok(dtype, N, V, V, 1.0f)) return -1;
    if (N == 0) return 0;
    const int P = row_shape(N, V, elem_size(dtype)).P;
    return P == 1 ? 0 : N * P * (int64_t)sizeof(RowState);
}

SF_API int sf_token_logp(const void* logits, int32_t dtype, int64_t N, int64_t V, int64_t row_stride,
                         const int64_t* targets, float inv_temperature, float* out_logp, float* out_lse,
                         float* out_entropy, void* workspace, int64_t workspace_bytes, sf_stream_t stream)
{
    if (!rows_ok(dtype, N, V, row_stride, inv_temperature)) return SF_EINVAL;
    if (N == 0) return SF_OK;
    const int64_t need = sf_token_logp_workspace(dtype, N, V);
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
    const RowShape shape = row_shape(N, V, elem_size(dtype));
    int P = shape.P, Vi = (int)V;
    int share = (Vi / (16 / elem_size(dtype)) + P - 1) / P;
    RowScale z;
    z.inv_t = inv_temperature;
    z.c = (float)((double)inv_temperature * kLog2eD);
    z.eps = (float)(((double)inv_temperature * kLog2eD - (double)z.c) / (double)z.c);
    void* args[] = {(void*)&logits, (void*)&N,     (void*)&Vi,       (void*)&row_stride, (void*)&targets,    (void*)&z,
                    (void*)&share,  (void*)&out_logp, (void*)&out_lse, (void*)&out_entropy, (void*)&workspace};
    const void* fn[3][3] = {{(const void*)&k_token_logp<SF_F32, 256, 1>, (const void*)&k_token_logp<SF_BF16, 256, 1>,
                             (const void*)&k_token_logp<SF_F16, 256, 1>},
                            {(const void*)&k_token_logp<SF_F32, 256, 4>, (const void*)&k_token_logp<SF_BF16, 256, 4>,
                             (const void*)&k_token_logp<SF_F16, 256, 4>},
                            {(const void*)&k_token_logp<SF_F32, 1024, 16>, (const void*)&k_token_logp<SF_BF16, 1024, 16>,
                             (const void*)&k_token_logp<SF_F16, 1024, 16>}};
    const int rows = shape.wg == 64 ? 4 : 1;
    const int rc = launch(fn[shape.wg == 64 ? 0 : shape.wg == 256 ? 1 : 2][dtype], dim3(grid_of((N + rows - 1) / rows), P),
                          dim3(shape.wg == 64 ? 256 : shape.wg), args, 0, stream);
    if (rc != SF_OK || P == 1) return rc;
    const void* join[3] = {(const void*)&k_token_logp_join<SF_F32>, (const void*)&k_token_logp_join<SF_BF16>,
                           (const void*)&k_token_logp_join<SF_F16>};
    args[6] = (void*)&P;
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
    int Vi = (int)V;
    const int64_t vecs = V / (16 / b);
    const int lanes = vecs <= 64 * kGradU ? 64 : 256;
    const int64_t chunks = (vecs + kGradU * lanes - 1) / (kGradU * lanes);
    const int64_t groups = (N + kRowWG / lanes - 1) / (kRowWG / lanes);
    void* args[] = {(void*)&logits,  (void*)&N,         (void*)&Vi,      (void*)&row_stride,   (void*)&targets,
                    (void*)&inv_temperature, (void*)&lse, (void*)&grad_logp, (void*)&entropy,
                    (void*)&grad_entropy, (void*)&out_grad, (void*)&out_row_stride};
    const void* fn[2][3] = {{(const void*)&k_token_logp_grad<SF_F32, 256>, (const void*)&k_token_logp_grad<SF_BF16, 256>,
                             (const void*)&k_token_logp_grad<SF_F16, 256>},
                            {(const void*)&k_token_logp_grad<SF_F32, 64>, (const void*)&k_token_logp_grad<SF_BF16, 64>,
                             (const void*)&k_token_logp_grad<SF_F16, 64>}};
    return launch(fn[lanes == 64][dtype], dim3((unsigned)(chunks < 1 ? 1 : chunks), (unsigned)(groups < 65535 ? groups : 65535)),
                  dim3(kRowWG), args, 0, stream);
}
