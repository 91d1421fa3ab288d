// Clipped policy loss with a KL term and an entropy bonus, from the logits of N rows, and its gradient (gfx950).
//
// With m the largest logit of a row, d_k = x_k - m and e_k = exp(d_k):  s = sum e_k, t = sum e_k d_k give lse = m + log s and
// entropy = log s - t / s, in which nothing large cancels.  Log-probabilities are (x_k - m) - log s, or (x_k - x_a) + logp in the gradient pass on its own,
// never x_k - lse, whose rounding at logits of 10^4 would put every probability off by 10^-3.  The gradient of a row is  a_k = p_k (c + w eta log p_k) + [k = a] w g  with
// c = w (eta entropy - g): one exponential and two products per logit.
#include "elem.h"
#include "ssm_internal.h"

namespace ssm {
namespace {

constexpr size_t ALIGN = 256;
inline bool misaligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }

constexpr float LOG2E = 1.44269504f, LN2 = 0.69314718f;

struct PolicyArgs {
    const void *logits; int64_t pitch;
    const int64_t *action;
    const float *logp_old, *advantage, *weight, *logp_ref;
    ssm_policy_terms terms;
    int64_t N; int K;
    float *logp, *entropy, *lse;             // written by the forward pass, read by the gradient pass on its own
    const float *dloss;
    void *dlogits; int64_t dpitch;
    float *row_loss;                         // [N] weighted
};

// What the loss of a row is and its slope with respect to logp.
struct RowTerms { float loss, slope; };
__device__ __forceinline__ RowTerms row_terms(const PolicyArgs &a, int64_t n, float logp, float entropy)
{
    const float A = a.advantage[n], rho = expf(logp - a.logp_old[n]);
    // (an advantage of zero makes the term zero, also where the ratio overflows)
    const float raw = A == 0.f ? 0.f : rho * A, clipped = (rho < 1.f - a.terms.clip_low ? 1.f - a.terms.clip_low : rho > 1.f + a.terms.clip_high ? 1.f + a.terms.clip_high : rho) * A;
    const bool held = clipped < raw;         // (a NaN is not held: it reaches the results)
    RowTerms r = {-(held ? clipped : raw) - a.terms.entropy_coef * entropy, held ? 0.f : -raw};
    if (a.logp_ref) {
        const float d = a.logp_ref[n] - logp, e = expm1f(d);
        r.loss += a.terms.kl_coef * (e - d);
        r.slope -= a.terms.kl_coef * e;
    }
    return r;
}

__device__ __forceinline__ float wave_sum(float v)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    return v;
}
__device__ __forceinline__ float wave_max(float v)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
    return v;
}

// One workgroup per row, three sweeps over it.
template <class T, bool STATS, bool GRAD>
__global__ void __launch_bounds__(256) policy_row_kernel(PolicyArgs a)
{
    __shared__ float red[2][4];
    const int64_t n = blockIdx.x;
    const int tid = threadIdx.x, K = a.K, w = tid >> 6;
    const T *x = static_cast<const T *>(a.logits) + n * a.pitch;
    T *dx = GRAD ? static_cast<T *>(a.dlogits) + n * a.dpitch : nullptr;
    const int64_t act = a.action[n];
    const float weight = a.weight ? a.weight[n] : 1.f / (float)a.N;
    bool idle = weight == 0.f || act < 0;
    float lse = 0.f, entropy = 0.f, logp = 0.f, loss = 0.f, slope = 0.f;
    float base = 0.f, off = 0.f;             // log p_k = (x_k - base) + off
    if (!idle) {
        if constexpr (STATS) {
            const float xa = act < K ? (float)x[act] : NAN;      // (before the barriers: the gradient may be stored over the logits)
            float m = -INFINITY;
            for (int k = tid; k < K; k += 256) m = fmaxf(m, (float)x[k]);
            m = wave_max(m);
            if ((tid & 63) == 0) red[0][w] = m;
            __syncthreads();
            m = fmaxf(fmaxf(red[0][0], red[0][1]), fmaxf(red[0][2], red[0][3]));
            __syncthreads();
            float s = 0.f, t = 0.f;
            for (int k = tid; k < K; k += 256) {
                const float d = (float)x[k] - m, e = __builtin_amdgcn_exp2f(d * LOG2E);
                s += e;
                t += e == 0.f ? 0.f : e * d;
            }
            s = wave_sum(s); t = wave_sum(t);
            if ((tid & 63) == 0) { red[0][w] = s; red[1][w] = t; }
            __syncthreads();
            s = red[0][0] + red[0][1] + red[0][2] + red[0][3];
            t = red[1][0] + red[1][1] + red[1][2] + red[1][3];
            if (m == -INFINITY) {            // (uniform; a maximum passes over NaN)
                bool nan = false;
                for (int k = 0; k < K; ++k) nan |= x[k] != x[k];
                idle = !nan;
            }
            const float ls = logf(s);
            lse = m + ls; entropy = ls - t / s; logp = (xa - m) - ls;
            base = m; off = -ls;
        } else {
            lse = a.lse[n]; entropy = a.entropy[n]; logp = a.logp[n];
            idle = lse == -INFINITY;
            const float xa = act < K ? (float)x[act] : NAN;
            __syncthreads();
            const bool taken = xa != -INFINITY;          // (else the action cannot be taken, and lse has to do)
            base = taken ? xa : lse; off = taken ? logp : 0.f;
        }
    }
    if (!idle) {
        const RowTerms r = row_terms(a, n, logp, entropy);
        loss = weight * r.loss; slope = weight * r.slope;
    }
    if (STATS && tid == 0) {
        a.row_loss[n] = idle ? 0.f : loss;
        a.logp[n] = idle ? 0.f : logp; a.entropy[n] = idle ? 0.f : entropy; a.lse[n] = idle ? -INFINITY : lse;
    }
    if constexpr (GRAD) {
        if (a.dloss) slope *= a.dloss[0];
        const float eta = weight * a.terms.entropy_coef * (a.dloss ? a.dloss[0] : 1.f), c = eta * entropy - slope;
        for (int k = tid; k < K; k += 256) {
            float g = 0.f;
            if (!idle) {
                const float lp = ((float)x[k] - base) + off, p = __builtin_amdgcn_exp2f(lp * LOG2E);
                g = p == 0.f ? 0.f : p * fmaf(eta, lp, c);
                if (k == act) g += slope;
            }
            dx[k] = rounded<T>(g);
        }
    }
}

// loss = sum of the rows', in one fixed order
__global__ void __launch_bounds__(1024) policy_sum_kernel(const float *__restrict__ row_loss, int64_t n, float *__restrict__ loss)
{
    __shared__ double red[16];
    double s = 0.0;
    for (int64_t i = threadIdx.x; i < n; i += 1024) s += (double)row_loss[i];
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < 16; ++i) s += red[i];
        loss[0] = (float)s;
    }
}

ssm_status check_policy(const PolicyArgs &a, int dtype, int64_t N, int64_t K)
{
    if (!a.logits || !a.action || !a.logp_old || !a.advantage || !a.logp || !a.entropy || !a.lse) return SSM_ERR_INVALID_ARG;
    if (N <= 0 || K <= 0 || !dtype_known(dtype) || a.pitch < 0) return SSM_ERR_INVALID_ARG;
    if (N > SSM_MAX_TOKENS || K > (1LL << 30) || a.pitch > SSM_MAX_ELEMS / N || K > SSM_MAX_ELEMS / N) return SSM_ERR_UNSUPPORTED;
    if (misaligned(a.logits, dtype_bytes(dtype)) || misaligned(a.action, 8) || misaligned(a.logp_old, 4) || misaligned(a.advantage, 4) ||
        misaligned(a.weight, 4) || misaligned(a.logp_ref, 4) || misaligned(a.logp, 4) || misaligned(a.entropy, 4) || misaligned(a.lse, 4) || misaligned(a.dloss, 4))
        return SSM_ERR_INVALID_ARG;
    const ssm_policy_terms &t = a.terms;
    if (!(t.clip_low >= 0.f) || !(t.clip_high >= 0.f) || t.kl_coef != t.kl_coef || t.entropy_coef != t.entropy_coef) return SSM_ERR_INVALID_ARG;
    return SSM_OK;
}
ssm_status check_gradient(const PolicyArgs &a, int dtype, int64_t N, int64_t K)
{
    if (!a.dlogits || misaligned(a.dlogits, dtype_bytes(dtype))) return SSM_ERR_INVALID_ARG;
    if (N > 1 && (a.dpitch < K || (a.dlogits == a.logits && a.dpitch != a.pitch))) return SSM_ERR_INVALID_ARG;
    return N > 1 && a.dpitch > SSM_MAX_ELEMS / N ? SSM_ERR_UNSUPPORTED : SSM_OK;
}

ssm_status launch_sum(const PolicyArgs &a, float *loss, hipStream_t s)
{
    hipLaunchKernelGGL(policy_sum_kernel, dim3(1), dim3(1024), 0, s, a.row_loss, a.N, loss);
    return hipGetLastError() == hipSuccess ? SSM_OK : SSM_ERR_HIP;
}
template <bool STATS, bool GRAD> ssm_status launch_rows(const PolicyArgs &a, int dtype, hipStream_t s)
{
    with_dtype(dtype, [&](auto t) { hipLaunchKernelGGL((policy_row_kernel<decltype(t), STATS, GRAD>), dim3((unsigned)a.N), dim3(256), 0, s, a); });
    return hipGetLastError() == hipSuccess ? SSM_OK : SSM_ERR_HIP;
}

}  // namespace
}  // namespace ssm

using namespace ssm;

extern "C" {

size_t ssm_policy_loss_workspace_bytes(int64_t N, int64_t K)
{
    if (N <= 0 || K <= 0 || N > SSM_MAX_TOKENS || K > (1LL << 30) || K > SSM_MAX_ELEMS / N) return 0;
    return ((size_t)N * 4 + ALIGN - 1) / ALIGN * ALIGN;
}

ssm_status ssm_policy_loss_fwd(const void *logits, int64_t pitch, const int64_t *action, const float *logp_old,
                               const float *advantage, const float *weight, const float *logp_ref, ssm_policy_terms terms,
                               int dtype, int64_t N, int64_t K, float *loss, float *logp, float *entropy, float *lse,
                               void *workspace, size_t ws_bytes, void *stream)
{
    PolicyArgs a{logits, pitch, action, logp_old, advantage, weight, logp_ref, terms, N, (int)K, logp, entropy, lse, nullptr, nullptr, 0,
                 static_cast<float *>(workspace)};
    if (const ssm_status rc = check_policy(a, dtype, N, K)) return rc;
    if (!loss || misaligned(loss, 4)) return SSM_ERR_INVALID_ARG;
    if (!workspace || misaligned(workspace, ALIGN) || ws_bytes < ssm_policy_loss_workspace_bytes(N, K)) return SSM_ERR_WORKSPACE;
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (const ssm_status rc = launch_rows<true, false>(a, dtype, s)) return rc;
    return launch_sum(a, loss, s);
}

ssm_status ssm_policy_loss_bwd(const void *logits, int64_t pitch, const int64_t *action, const float *logp_old,
                               const float *advantage, const float *weight, const float *logp_ref, ssm_policy_terms terms,
                               int dtype, int64_t N, int64_t K, const float *logp, const float *entropy, const float *lse,
                               const float *dloss, void *dlogits, int64_t dpitch, void *stream)
{
    PolicyArgs a{logits, pitch, action, logp_old, advantage, weight, logp_ref, terms, N, (int)K, const_cast<float *>(logp),
                 const_cast<float *>(entropy), const_cast<float *>(lse), dloss, dlogits, dpitch, nullptr};
    if (const ssm_status rc = check_policy(a, dtype, N, K)) return rc;
    if (const ssm_status rc = check_gradient(a, dtype, N, K)) return rc;
    return launch_rows<false, true>(a, dtype, static_cast<hipStream_t>(stream));
}

ssm_status ssm_policy_loss_grad(const void *logits, int64_t pitch, const int64_t *action, const float *logp_old,
                                const float *advantage, const float *weight, const float *logp_ref, ssm_policy_terms terms,
                                int dtype, int64_t N, int64_t K, const float *dloss, float *loss, float *logp, float *entropy,
                                float *lse, void *dlogits, int64_t dpitch, void *workspace, size_t ws_bytes, void *stream)
{
    PolicyArgs a{logits, pitch, action, logp_old, advantage, weight, logp_ref, terms, N, (int)K, logp, entropy, lse, dloss, dlogits, dpitch,
                 static_cast<float *>(workspace)};
    if (const ssm_status rc = check_policy(a, dtype, N, K)) return rc;
    if (const ssm_status rc = check_gradient(a, dtype, N, K)) return rc;
    if (!loss || misaligned(loss, 4)) return SSM_ERR_INVALID_ARG;
    if (!workspace || misaligned(workspace, ALIGN) || ws_bytes < ssm_policy_loss_workspace_bytes(N, K)) return SSM_ERR_WORKSPACE;
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (const ssm_status rc = launch_rows<true, true>(a, dtype, s)) return rc;
    return launch_sum(a, loss, s);
}

}  // extern "C"
