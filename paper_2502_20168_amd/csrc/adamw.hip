// AdamW over many tensors at once (gfx950), states in 32 or in 8 bits.
//
// One pass over parameters, gradients and states.  The tensors of a launch are described in its arguments (no table in memory that would have to be
// copied and kept); a workgroup finds its tensor among them by counting the first workgroups that are not behind its own.
//
// 8 bits: a wavefront holds a block of 256 elements, four to a lane, so the block's largest magnitudes are maxima over its lanes.  Codes of sqrt(v) are the
// upper bits of the value as a float whose exponent was moved to the bottom of the range by one exact product: rounding to nearest even is an
// integer addition there, and small codes become that format's denormal numbers by themselves.  What is rounded to a code is computed in single operations
// (no contraction), so that a state depends on the formula alone.
//
// 32 bits: 28 bytes an element with f32 parameters, bound by memory: 2^21 x 48 elements in 522 us, 5.4 TB/s, where a large copy reaches 5.0.  8 bits: 14 bytes (f32, gradients bf16)
// 306 us, 4.6 TB/s; 10 (all bf16) 238 us, 4.3 TB/s: some 75 instructions an element, the exact root and quotient 25 of them, leave little time beside the memory's.
// (With codes put together by integers and maxima through LDS 337 and 306 us.)
#include "elem.h"
#include "ssm_internal.h"
#include "wave.h"

#include <cmath>

namespace ssm {
namespace {

inline bool misaligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }

constexpr int ADAMW_TENSORS = 48;            // tensors of a launch
// Elements of a workgroup, a whole number of blocks of 256 per wavefront.  48 tensors of 2^21 elements, us, with 1024, 2048, 4096 of them: states in 32 bits, f32 523, 547, 548,
// bf16 400, 430, 445 (bound by memory: short workgroups keep loads and stores mixed); in 8 bits, parameters f32 and gradients bf16 410, 326, 319, both bf16 383, 302, 286 (a workgroup's
// start counts, finding its tensor in particular).
constexpr int adamw_chunk(int bits) { return bits == 8 ? 4096 : 1024; }
constexpr int VALUES_CHUNK = 2048;

struct AdamwLaunch {
    ssm_adamw_tensor t[ADAMW_TENSORS];
    unsigned first[ADAMW_TENSORS];           // first workgroup of every tensor
    int count;
    const float *grad_scale, *skip;
    float decay, beta1, beta2, one_minus_beta1, one_minus_beta2, rate, inv_root2, eps;
};
struct ValuesLaunch {
    ssm_adamw_stored t[ADAMW_TENSORS];
    unsigned first[ADAMW_TENSORS];
    int count;
};

__device__ __forceinline__ int find_tensor(const unsigned *first, int count)
{
    int k = 0;
    for (int i = 1; i < count; ++i) k += blockIdx.x >= first[i];
    return k;
}

// Codes of sqrt(v): 4 mantissa bits below a bias of 15, largest 1.9375.  Those of m (3 below a bias of 7, largest 448) come from the hardware's conversion, two at a time, which
// rounds to nearest even and knows the denormal ones.
constexpr float R_DOWN = 0x1p-112f, R_UP = 0x1p112f;
__device__ __forceinline__ unsigned root_code(float magnitude)
{
    const unsigned b = __float_as_uint(magnitude * R_DOWN), drop = 19;
    return (b + ((1u << (drop - 1)) - 1u) + ((b >> drop) & 1u)) >> drop;
}
__device__ __forceinline__ float root_value(unsigned code) { return __uint_as_float(code << 19) * R_UP; }
// (by hand: the conversion takes the code above the largest for NaN, here it is 480 like any other)
__device__ __forceinline__ f32x4 m_values(unsigned codes)
{
    f32x4 m;
#pragma unroll
    for (int e = 0; e < 4; ++e) m[e] = __uint_as_float((unsigned)((int)(codes << (24 - 8 * e)) >> 4) & 0x87f00000u) * 0x1p120f;
    return m;
}
__device__ __forceinline__ unsigned m_codes(f32x4 m)
{
    return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(m[2], m[3], __builtin_amdgcn_cvt_pk_fp8_f32(m[0], m[1], 0, false), true);
}
__device__ __forceinline__ unsigned wave_max(unsigned v) { return over_group(v, 6, [](unsigned a, unsigned b) { return max(a, b); }); }
constexpr float M_TOP = 448.f, R_TOP = 1.9375f, SCALE_FLOOR = 0x1p-100f;

template <bool FULL, class T> __device__ __forceinline__ f32x4 load_upto4(const T *p, int n)
{
    if (FULL || n >= 4) return widened4<T>(load_pack<T, 4>(p));
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < 3; ++k) if (k < n) v[k] = (float)p[k];
    return v;
}
template <bool FULL, class T> __device__ __forceinline__ void store_upto4(T *p, int n, f32x4 v)
{
    if (FULL || n >= 4) { store_pack<T, 4>(p, rounded4<T>(v)); return; }
#pragma unroll
    for (int k = 0; k < 3; ++k) if (k < n) p[k] = rounded<T>(v[k]);
}
template <bool FULL> __device__ __forceinline__ unsigned load_bytes(const uint8_t *p, int n)
{
    typedef unsigned loose __attribute__((aligned(1)));
    if (FULL || n >= 4) return *reinterpret_cast<const loose *>(p);
    unsigned v = 0;
#pragma unroll
    for (int k = 0; k < 3; ++k) if (k < n) v |= (unsigned)p[k] << (8 * k);
    return v;
}
template <bool FULL> __device__ __forceinline__ void store_bytes(uint8_t *p, int n, unsigned v)
{
    typedef unsigned loose __attribute__((aligned(1)));
    if (FULL || n >= 4) { *reinterpret_cast<loose *>(p) = v; return; }
#pragma unroll
    for (int k = 0; k < 3; ++k) if (k < n) p[k] = (uint8_t)(v >> (8 * k));
}

// The chunk from element `start` on.  FULL: none of it is past the end.
template <class P, class G, int BITS, bool FULL>
__device__ __forceinline__ void step_chunk(const AdamwLaunch &a, const ssm_adamw_tensor &t, int64_t start, float gs)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    P *param = static_cast<P *>(t.param);
    const G *grad = static_cast<const G *>(t.grad);
#pragma unroll
    for (int j = 0; j < adamw_chunk(BITS) / (4 * SSM_ADAMW_BLOCK); ++j) {
        const int64_t at = start + (j * 4 + wave) * SSM_ADAMW_BLOCK + lane * 4;
        const int64_t left = t.n - at;
        const int n = FULL || left >= 4 ? 4 : left > 0 ? (int)left : 0;
        const int64_t block = at / SSM_ADAMW_BLOCK;
        if (!FULL && block * SSM_ADAMW_BLOCK >= t.n) break;      // (uniform over the wavefront)
        f32x4 p = load_upto4<FULL, P>(param + at, n), g = load_upto4<FULL, G>(grad + at, n), m, v;
        if constexpr (BITS == 32) {
            m = load_upto4<FULL, float>(static_cast<float *>(t.m) + at, n);
            v = load_upto4<FULL, float>(static_cast<float *>(t.v) + at, n);
        } else {
            const unsigned mc = load_bytes<FULL>(static_cast<uint8_t *>(t.m) + at, n), vc = load_bytes<FULL>(static_cast<uint8_t *>(t.v) + at, n);
            const float ms = t.m_scale[block], vs = t.v_scale[block];
            m = m_values(mc);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                m[e] *= ms;
                const float r = root_value((vc >> (8 * e)) & 255u) * vs;
                v[e] = r * r;
            }
        }
        f32x4 root;
        {
#pragma clang fp contract(off)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float ge = g[e] * gs;
                m[e] = m[e] * a.beta1 + ge * a.one_minus_beta1;
                v[e] = v[e] * a.beta2 + (ge * ge) * a.one_minus_beta2;
                root[e] = sqrtf(v[e]);
                p[e] = p[e] * a.decay - a.rate * (m[e] / (root[e] * a.inv_root2 + a.eps));
            }
        }
        store_upto4<FULL, P>(param + at, n, p);
        if constexpr (BITS == 32) {
            store_upto4<FULL, float>(static_cast<float *>(t.m) + at, n, m);
            store_upto4<FULL, float>(static_cast<float *>(t.v) + at, n, v);
        } else {
            if (!FULL && (block + 1) * SSM_ADAMW_BLOCK > t.n) {           // (uniform: the last block of a tensor)
#pragma unroll
                for (int e = 0; e < 4; ++e) { m[e] = e < n ? m[e] : 0.f; root[e] = e < n ? root[e] : 0.f; }
            }
            // (as bit patterns: NaN is above infinity is above every number, so either reaches the scale)
            unsigned mb = 0, rb = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                mb = max(mb, __float_as_uint(m[e]) & 0x7fffffffu);
                rb = max(rb, __float_as_uint(root[e]) & 0x7fffffffu);
            }
            const float mbig = __uint_as_float(wave_max(mb)), rbig = __uint_as_float(wave_max(rb));
            const float mk = mbig < SCALE_FLOOR ? 0.f : mbig, rk = rbig < SCALE_FLOOR ? 0.f : rbig;
            // (both quotients in one division, in the even lanes and in the odd)
            const bool odd = lane & 1;
            const int over = __float_as_int((odd ? R_TOP : M_TOP) / (odd ? rk : mk));
            const float mi = mk == 0.f ? 0.f : __int_as_float(__builtin_amdgcn_readlane(over, 0)), ri = rk == 0.f ? 0.f : __int_as_float(__builtin_amdgcn_readlane(over, 1));
            unsigned vc = 0;
            f32x4 scaled;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                scaled[e] = m[e] * mi;
                const float y = root[e] * ri;
                vc |= (y > 0.f ? max(root_code(y), 1u) & 255u : 0u) << (8 * e);
            }
            const unsigned mc = m_codes(scaled);
            store_bytes<FULL>(static_cast<uint8_t *>(t.m) + at, n, mc);
            store_bytes<FULL>(static_cast<uint8_t *>(t.v) + at, n, vc);
            if (lane == 0) { t.m_scale[block] = mk * (1.f / M_TOP); t.v_scale[block] = rk * (1.f / R_TOP); }
        }
    }
}

template <class P, class G, int BITS>
__global__ void __launch_bounds__(256) adamw_kernel(AdamwLaunch a)
{
    if (a.skip && a.skip[0] != 0.f) return;
    const int k = find_tensor(a.first, a.count);
    const ssm_adamw_tensor t = a.t[k];
    const float gs = a.grad_scale ? a.grad_scale[0] : 1.f;
    const int64_t start = (int64_t)(blockIdx.x - a.first[k]) * adamw_chunk(BITS);
    // (in 32 bits there is little arithmetic to spare, and the smaller kernel is faster: parameters bf16 403 us, with both 416)
    if (BITS == 8 && t.n - start >= adamw_chunk(BITS)) step_chunk<P, G, BITS, true>(a, t, start, gs);
    else step_chunk<P, G, BITS, false>(a, t, start, gs);
}

__global__ void __launch_bounds__(256) adamw_values_kernel(ValuesLaunch a)
{
    const int k = find_tensor(a.first, a.count);
    const ssm_adamw_stored t = a.t[k];
#pragma unroll
    for (int j = 0; j < VALUES_CHUNK / 1024; ++j) {
        const int64_t at = (int64_t)(blockIdx.x - a.first[k]) * VALUES_CHUNK + j * 1024 + threadIdx.x * 4;
        const int64_t left = t.n - at, block = at / SSM_ADAMW_BLOCK;
        if (left <= 0) break;
        const int n = left >= 4 ? 4 : (int)left;
        const unsigned mc = load_bytes<false>(static_cast<const uint8_t *>(t.m) + at, n), vc = load_bytes<false>(static_cast<const uint8_t *>(t.v) + at, n);
        const float ms = t.m_scale[block], vs = t.v_scale[block];
        f32x4 m = m_values(mc), v;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            m[e] *= ms;
            const float r = root_value((vc >> (8 * e)) & 255u) * vs;
            v[e] = r * r;
        }
        if (t.m_out) store_upto4<false, float>(t.m_out + at, n, m);
        if (t.v_out) store_upto4<false, float>(t.v_out + at, n, v);
    }
}

// Launches `kernel(launch)` over all tensors, ADAMW_TENSORS at a time; empty ones take no place.
template <class L, class D, class K> ssm_status launch_all(L &a, const D *tensors, int64_t count, int chunk, hipStream_t s, K kernel)
{
    int64_t blocks = 0;
    a.count = 0;
    const auto flush = [&]() {
        if (a.count == 0) return hipSuccess;
        kernel(dim3((unsigned)blocks), a, s);
        a.count = 0; blocks = 0;
        return hipGetLastError();
    };
    for (int64_t i = 0; i < count; ++i) {
        if (tensors[i].n == 0) continue;
        const int64_t mine = (tensors[i].n + chunk - 1) / chunk;
        if (a.count == ADAMW_TENSORS || !fits_a_grid(blocks + mine, 256)) { if (flush() != hipSuccess) return SSM_ERR_HIP; }
        a.t[a.count] = tensors[i];
        a.first[a.count++] = (unsigned)blocks;
        blocks += mine;
    }
    return flush() == hipSuccess ? SSM_OK : SSM_ERR_HIP;
}

template <class P, class G, int BITS> ssm_status run_step(AdamwLaunch &a, const ssm_adamw_tensor *tensors, int64_t count, hipStream_t s)
{
    return launch_all(a, tensors, count, adamw_chunk(BITS), s, [](dim3 grid, const AdamwLaunch &l, hipStream_t st) {
        hipLaunchKernelGGL((adamw_kernel<P, G, BITS>), grid, dim3(256), 0, st, l);
    });
}

}  // namespace
}  // namespace ssm

using namespace ssm;

extern "C" {

ssm_status ssm_adamw_step(const ssm_adamw_tensor *tensors, int64_t count, ssm_adamw_rates r, int param_dtype, int grad_dtype,
                          int state_bits, const float *grad_scale, const float *skip, void *stream)
{
    if (!tensors || count <= 0 || !dtype_known(param_dtype) || !dtype_known(grad_dtype) || (state_bits != 8 && state_bits != 32)) return SSM_ERR_INVALID_ARG;
    if (param_dtype != SSM_F32 && param_dtype != grad_dtype) return SSM_ERR_INVALID_ARG;
    if (!(r.beta1 >= 0. && r.beta1 < 1.) || !(r.beta2 >= 0. && r.beta2 < 1.) || !(r.eps >= 0.) || r.step < 1 || r.lr != r.lr || r.weight_decay != r.weight_decay)
        return SSM_ERR_INVALID_ARG;
    if (misaligned(grad_scale, 4) || misaligned(skip, 4)) return SSM_ERR_INVALID_ARG;
    const size_t pb = dtype_bytes(param_dtype), gb = dtype_bytes(grad_dtype);
    for (int64_t i = 0; i < count; ++i) {
        const ssm_adamw_tensor &t = tensors[i];
        if (t.n < 0) return SSM_ERR_INVALID_ARG;
        if (t.n == 0) continue;
        if (t.n > SSM_MAX_ELEMS || !fits_a_grid((t.n + adamw_chunk(state_bits) - 1) / adamw_chunk(state_bits), 256)) return SSM_ERR_UNSUPPORTED;
        if (!t.param || !t.grad || !t.m || !t.v || misaligned(t.param, pb) || misaligned(t.grad, gb)) return SSM_ERR_INVALID_ARG;
        if (state_bits == 32 ? misaligned(t.m, 4) || misaligned(t.v, 4)
                             : !t.m_scale || !t.v_scale || misaligned(t.m_scale, 4) || misaligned(t.v_scale, 4))
            return SSM_ERR_INVALID_ARG;
    }
    AdamwLaunch a{};
    a.grad_scale = grad_scale; a.skip = skip;
    a.decay = (float)(1. - r.lr * r.weight_decay);
    a.beta1 = (float)r.beta1; a.beta2 = (float)r.beta2;
    a.one_minus_beta1 = (float)(1. - r.beta1); a.one_minus_beta2 = (float)(1. - r.beta2);
    a.rate = (float)(r.lr / (1. - std::pow(r.beta1, (double)r.step)));
    a.inv_root2 = 1.f / (float)std::sqrt(1. - std::pow(r.beta2, (double)r.step));
    a.eps = (float)r.eps;
    hipStream_t s = static_cast<hipStream_t>(stream);
    return with_dtype(grad_dtype, [&](auto g) {
        using G = decltype(g);
        if (param_dtype == SSM_F32) return state_bits == 8 ? run_step<float, G, 8>(a, tensors, count, s) : run_step<float, G, 32>(a, tensors, count, s);
        return state_bits == 8 ? run_step<G, G, 8>(a, tensors, count, s) : run_step<G, G, 32>(a, tensors, count, s);
    });
}

ssm_status ssm_adamw_values(const ssm_adamw_stored *tensors, int64_t count, void *stream)
{
    if (!tensors || count <= 0) return SSM_ERR_INVALID_ARG;
    for (int64_t i = 0; i < count; ++i) {
        const ssm_adamw_stored &t = tensors[i];
        if (t.n < 0) return SSM_ERR_INVALID_ARG;
        if (t.n == 0) continue;
        if (t.n > SSM_MAX_ELEMS || !fits_a_grid((t.n + VALUES_CHUNK - 1) / VALUES_CHUNK, 256)) return SSM_ERR_UNSUPPORTED;
        if (!t.m || !t.v || !t.m_scale || !t.v_scale || misaligned(t.m_scale, 4) || misaligned(t.v_scale, 4) || misaligned(t.m_out, 4) || misaligned(t.v_out, 4))
            return SSM_ERR_INVALID_ARG;
    }
    ValuesLaunch a{};
    return launch_all(a, tensors, count, VALUES_CHUNK, static_cast<hipStream_t>(stream), [](dim3 grid, const ValuesLaunch &l, hipStream_t st) {
        hipLaunchKernelGGL(adamw_values_kernel, grid, dim3(256), 0, st, l);
    });
}

}  // extern "C"
