// Clipped policy loss with a KL term and an entropy bonus, from the logits of N rows, and its gradient (gfx950).
//
// With m the largest logit of a row, d_k = x_k - m and e_k = exp(d_k):  s = sum e_k, t = sum e_k d_k give lse = m + log s and
// entropy = log s - t / s, in which nothing large cancels.  Log-probabilities are (x_k - m) - log s; in the gradient pass on its own, which has lse and logp in 32 bits,
// (x_k - x_a) + logp or x_k - lse, whichever of logp and lse is the smaller and so rounded less.  The gradient of a row is  a_k = p_k (c + w eta log p_k) + [k = a] w g  with
// c = w (eta entropy - g): one exponential and two products per logit.
//
// Large calls are bound by memory where a row's registers hold it between its sums and its gradient, so that it is read once: 4096 x 65536 bf16 forward 98 us (5.5 TB/s), loss and gradient
// 203 us (5.3 TB/s), where a copy reaches 5.0; the vector units are busy two thirds of that.  Who holds a row goes by its length (below).  Small calls are bound by two launches: 16384 x 32
// f32 4.4 us for loss and gradient and 2.0 for the sum of their parts.
#include "elem.h"
#include "ssm_internal.h"
#include "wave.h"

#include <type_traits>

namespace ssm {
namespace {

constexpr size_t ALIGN = 256;
inline bool misaligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }

constexpr float LOG2E = 1.44269504f;

struct PolicyArgs {
    const void *logits; int64_t pitch;
    const int64_t *action;
    const float *logp_old, *advantage, *weight, *logp_ref;
    ssm_policy_terms terms;
    int64_t N; int K;
    float *logp, *entropy, *lse;             // written by the forward pass, read by the gradient pass on its own
    const float *dloss;
    void *dlogits; int64_t dpitch;
    float *part_loss;                        // weighted, of every workgroup's rows
    float mean_weight;                       // of a row where none are given
};

__device__ __forceinline__ float group_sum(float v, int lanes) { return over_group(v, lanes, [](float a, float b) { return a + b; }); }
__device__ __forceinline__ float group_max(float v, int lanes) { return over_group(v, lanes, [](float a, float b) { return fmaxf(a, b); }); }
__device__ __forceinline__ float wave_sum(float v) { return group_sum(v, 6); }
__device__ __forceinline__ float wave_max(float v) { return group_max(v, 6); }

// What is given per row, and what comes of it.  Sums and differences of a row's few numbers are formed in 64 bits (in 32, the logarithm of a large sum alone would put a
// ratio off by 5e-7), functions of them in 32 where their argument is small or its rounded part is put back.  (With the 64-bit functions a row cost its wavefront
// some 2500 cycles, more than the logits of a short one: 65536 x 200 bf16 forward 28.6 us, with these 22.5.)
struct Row {
    int64_t action;
    float old, advantage, ref, weight;
    bool idle;
};
__device__ __forceinline__ Row load_row(const PolicyArgs &a, int64_t n)
{
    Row r;
    r.action = a.action[n];
    r.weight = a.weight ? a.weight[n] : a.mean_weight;
    r.old = a.logp_old[n]; r.advantage = a.advantage[n];
    r.ref = a.logp_ref ? a.logp_ref[n] : 0.f;
    r.idle = r.weight == 0.f || r.action < 0;
    return r;
}
struct Terms { float loss, slope; };         // of the row's loss, and of it with respect to logp
__device__ __forceinline__ Terms row_terms(const PolicyArgs &a, const Row &r, double logp, float entropy)
{
    const double gap = logp - (double)r.old;
    const float g = (float)gap, A = r.advantage, rho0 = expf(g);
    const float low = 1.f - a.terms.clip_low, high = 1.f + a.terms.clip_high;
    // (0: also of an action whose logit is -infinity, whose gap is -infinity and has no rounded part)
    const float ratio = rho0 == 0.f || rho0 == INFINITY ? rho0 : fmaf(rho0, (float)(gap - (double)g), rho0);
    // (an advantage of zero makes the term zero also where the ratio overflows, but not where it is NaN)
    const float raw = A == 0.f && ratio == INFINITY ? 0.f : ratio * A, clipped = (ratio < low ? low : ratio > high ? high : ratio) * A;
    const bool held = clipped < raw;         // (a NaN is not held: it reaches the results)
    Terms t = {-(held ? clipped : raw) - a.terms.entropy_coef * entropy, held ? 0.f : -raw};
    if (a.logp_ref && a.terms.kl_coef != 0.f) {              // (0 times a distance that overflows is 0)
        // e^d - 1 - d cancels to d^2 / 2: its series up to a half, whose first term left out is 1e-9 of it
        const float d = (float)((double)r.ref - logp);
        float p = 1.f / 3628800.f;
        p = fmaf(p, d, 1.f / 362880.f); p = fmaf(p, d, 1.f / 40320.f); p = fmaf(p, d, 1.f / 5040.f); p = fmaf(p, d, 1.f / 720.f);
        p = fmaf(p, d, 1.f / 120.f); p = fmaf(p, d, 1.f / 24.f); p = fmaf(p, d, 1.f / 6.f); p = fmaf(p, d, 0.5f);
        const bool near = fabsf(d) < 0.5f;
        const float far = expf(d) - 1.f, k = near ? p * d * d : far - d, e = near ? d + k : far;
        t.loss += a.terms.kl_coef * k;
        t.slope -= a.terms.kl_coef * e;
    }
    return t;
}
// log s for s > 0: the exponent's part in 64 bits, the rest between log 0.75 and log 1.5
__device__ __forceinline__ double log_of_sum(float s)
{
    int e;
    float f = frexpf(s, &e);                 // [0.5, 1)
    if (f < 0.75f) { f *= 2.f; --e; }
    return (double)e * 0.6931471805599453 + (double)logf(f);
}

// Sums of a row (of a part of one): largest logit m, s = sum 2^d, t = sum 2^d d with d = (x - m) log2 e.  m starts at the lowest number, not at -infinity: a row with
// no logit above -infinity ends with s = 0, and no difference of infinities is formed.  (A maximum passes over NaN; s does not.)
constexpr float LOWEST = -3.402823466e38f, FAR = -1e4f;
struct Sums { float m, s, t; };

template <class T> struct Unit {             // 16 bytes of a row
    static constexpr int V = 16 / sizeof(T);
    typedef typename Pack<T, V>::type raw;
    typedef float wide __attribute__((ext_vector_type(V)));
};
// unit from element k0 on; what lies past the end of the row is an action that cannot be taken.  (As words on both sides: put together element by element, the compiler gives
// a 16-bit element a register of its own, four units more than 100 of them.)
template <class T> __device__ __forceinline__ typename Unit<T>::raw load_unit(const T *x, int k0, int K)
{
    typedef unsigned words __attribute__((ext_vector_type(4)));
    typedef typename std::conditional<sizeof(T) == 2, uint16_t, uint32_t>::type bits;
    constexpr int V = Unit<T>::V;
    words w;
    if (K - k0 >= V) {
        w = __builtin_bit_cast(words, load_pack<T, V>(x + k0));
    } else {
        const unsigned none = __builtin_bit_cast(bits, (T)-INFINITY);
        const bits *q = reinterpret_cast<const bits *>(x);
        unsigned e[V];
#pragma unroll
        for (int i = 0; i < V; ++i) e[i] = k0 + i < K ? (unsigned)q[k0 + i] : none;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (V == 8) w[i] = e[2 * i] | e[2 * i + 1] << 16;
            else w[i] = e[i];
        }
    }
    return __builtin_bit_cast(typename Unit<T>::raw, w);
}
template <class T> __device__ __forceinline__ void store_unit(T *x, int k0, int K, typename Unit<T>::wide g)
{
    constexpr int V = Unit<T>::V;
    const typename Unit<T>::raw v = __builtin_convertvector(g, typename Unit<T>::raw);
    if (K - k0 >= V) { store_pack<T, V>(x + k0, v); return; }
#pragma unroll
    for (int i = 0; i < V; ++i) if (k0 + i < K) x[k0 + i] = v[i];
}
template <class T> __device__ __forceinline__ typename Unit<T>::wide widen(typename Unit<T>::raw v) { return __builtin_convertvector(v, typename Unit<T>::wide); }

// (16-bit units stay packed from one sweep over them to the next, and until `known` is: widened ones, or such that are widened ahead of what they wait for, would not
// fit the registers)
template <class T, int U> __device__ __forceinline__ void stay_packed(typename Unit<T>::raw (&v)[U], float &known)
{
    typedef unsigned words __attribute__((ext_vector_type(4)));
    if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int j = 0; j < U; ++j) {
            words w = __builtin_bit_cast(words, v[j]);
            asm volatile("" : "+v"(w), "+v"(known));
            v[j] = __builtin_bit_cast(typename Unit<T>::raw, w);
        }
    }
}

template <class T> __device__ __forceinline__ float max_of(typename Unit<T>::raw v, float m)
{
    const typename Unit<T>::wide x = widen<T>(v);
#pragma unroll
    for (int i = 0; i < Unit<T>::V; ++i) m = fmaxf(m, x[i]);
    return m;
}
template <class T> __device__ __forceinline__ void add_unit(typename Unit<T>::raw v, float m, float &s, float &t)
{
    const typename Unit<T>::wide x = widen<T>(v);
#pragma unroll
    for (int i = 0; i < Unit<T>::V; ++i) {
        const float d = (x[i] - m) * LOG2E, e = __builtin_amdgcn_exp2f(d);
        s += e;
        t = fmaf(e, fmaxf(d, FAR), t);       // (0 times -infinity is 0 here)
    }
}

// What the gradient of a row needs: log2 p_k = (x_k - base) log2 e + off,  a_k = p_k (c + eta log2 p_k) + [k = action] slope.
struct Slope { float base, off, c, eta, slope; int action; bool idle; };
template <class T> __device__ __forceinline__ typename Unit<T>::wide gradient(typename Unit<T>::raw v, int k0, const Slope &g)
{
    const typename Unit<T>::wide x = widen<T>(v);
    typename Unit<T>::wide r;
#pragma unroll
    for (int i = 0; i < Unit<T>::V; ++i) {
        const float lp = fmaf(x[i] - g.base, LOG2E, g.off), p = __builtin_amdgcn_exp2f(lp);
        r[i] = p * fmaf(g.eta, fmaxf(lp, FAR), g.c);
    }
    if ((unsigned)(g.action - k0) < (unsigned)Unit<T>::V) {
#pragma unroll
        for (int i = 0; i < Unit<T>::V; ++i) r[i] += k0 + i == g.action ? g.slope : 0.f;
    }
    if (g.idle) {
#pragma unroll
        for (int i = 0; i < Unit<T>::V; ++i) r[i] = 0.f;
    }
    return r;
}

// The end of a row's statistics: its results (stored by one lane), its weighted loss and what its gradient needs.
__device__ __forceinline__ Slope finish_row(const PolicyArgs &a, int64_t n, const Row &r, const Sums &q, float xa, bool store, float &loss)
{
    const bool idle = r.idle || q.s == 0.f;
    const double ls = log_of_sum(q.s), logp = ((double)xa - (double)q.m) - ls;
    const float entropy = (float)(ls - (double)(q.t * 0.69314718f / q.s));
    const Terms t = row_terms(a, r, logp, entropy);
    loss = idle ? 0.f : r.weight * t.loss;
    if (store) {
        a.logp[n] = idle ? 0.f : (float)logp;
        a.entropy[n] = idle ? 0.f : entropy;
        a.lse[n] = idle ? -INFINITY : (float)((double)q.m + ls);
    }
    const float w = r.weight * (a.dloss ? a.dloss[0] : 1.f), eta = w * a.terms.entropy_coef, slope = w * t.slope;
    return {q.m, (float)(-ls * 1.4426950408889634), fmaf(eta, entropy, -slope), eta * 0.69314718f, slope, (int)r.action, idle};
}
// The same from what the forward pass stored.  lse and logp are both rounded at their own size: the row's other logits are taken relative to lse where that is the smaller one (an own
// action far below them, or one that cannot be taken), else relative to the logit of the action (lse is rounded by 10^-3 at logits of 10^4).  logp itself likewise.
__device__ __forceinline__ Slope stored_row(const PolicyArgs &a, int64_t n, const Row &r, float xa)
{
    const float lse = a.lse[n], logp = a.logp[n], entropy = a.entropy[n];
    const bool by_action = fabsf(logp) <= fabsf(lse);
    const Terms t = row_terms(a, r, by_action ? (double)logp : (double)xa - (double)lse, entropy);
    const float w = r.weight * (a.dloss ? a.dloss[0] : 1.f), eta = w * a.terms.entropy_coef, slope = w * t.slope;
    return {by_action ? xa : lse, by_action ? logp * LOG2E : 0.f, fmaf(eta, entropy, -slope), eta * 0.69314718f, slope, (int)r.action,
            r.idle || lse == -INFINITY};
}
template <class T> __device__ __forceinline__ float logit_of_action(const T *x, const Row &r, int K)
{
    return r.idle ? 0.f : r.action < K ? (float)x[r.action] : NAN;
}

// Short rows: 2^lanes neighbouring lanes hold a row, one unit of 16 bytes each, so a wavefront holds R = 64 >> lanes of them at a time and B such batches. What is
// computed once per row would cost as much as its logits do; lane j does it for row j of the R B <= 64.  (65536 x 200 bf16, one batch and eight (forward) or four: forward
// 20.9 -> 16.4 us, loss and gradient 28.0 -> 23.6; 65536 x 512: 34.4 -> 26.2, 47.5 -> 38.0.)
template <class T, int B, bool STATS, bool GRAD>
__global__ void __launch_bounds__(256) policy_wave_kernel(PolicyArgs a, int lanes)
{
    constexpr int V = Unit<T>::V;
    __shared__ float red[4];
    const int lane = threadIdx.x & 63, width = 1 << lanes, k0 = (lane & (width - 1)) * V, group = lane >> lanes, R = 64 >> lanes, K = a.K;
    const int64_t first = ((int64_t)blockIdx.x * 4 + (threadIdx.x >> 6)) * (R * B);
    const auto row_of = [&](int j) { const int64_t n = first + j; return n < a.N ? n : a.N - 1; };
    typename Unit<T>::raw v[B];
#pragma unroll
    for (int b = 0; b < B; ++b) v[b] = load_unit<T>(static_cast<const T *>(a.logits) + row_of(b * R + group) * a.pitch, k0, K);
    const int64_t mine = row_of(lane);
    const bool own = lane < R * B && first + lane < a.N;
    Row r{-1, 0.f, 0.f, 0.f, 0.f, true};
    float xa = 0.f;
    if (own) {
        r = load_row(a, mine);
        xa = logit_of_action(static_cast<const T *>(a.logits) + mine * a.pitch, r, K);
    }
    Slope g{};
    if constexpr (STATS) {
        Sums q = {LOWEST, 0.f, 0.f};
        const int from = (lane & (R - 1)) << lanes, batch = lane >> (6 - lanes);     // who holds row `lane`: that group, of that batch
#pragma unroll
        for (int b = 0; b < B; ++b) {
            Sums p = {group_max(max_of<T>(v[b], LOWEST), lanes), 0.f, 0.f};
            add_unit<T>(v[b], p.m, p.s, p.t);
            p = {__shfl(p.m, from), __shfl(group_sum(p.s, lanes), from), __shfl(group_sum(p.t, lanes), from)};
            q = {batch == b ? p.m : q.m, batch == b ? p.s : q.s, batch == b ? p.t : q.t};
        }
        float loss;
        g = finish_row(a, mine, r, q, xa, own, loss);
        loss = wave_sum(own ? loss : 0.f);
        if (lane == 0) red[threadIdx.x >> 6] = loss;
        __syncthreads();
        if (threadIdx.x == 0) a.part_loss[blockIdx.x] = (red[0] + red[1]) + (red[2] + red[3]);
    } else if (own) {
        g = stored_row(a, mine, r, xa);
    }
    if constexpr (GRAD) {
        if (g.idle) g.action = -2;
#pragma unroll
        for (int b = 0; b < B; ++b) {
            const int j = b * R + group, action = __shfl(g.action, j);
            const Slope h = {__shfl(g.base, j), __shfl(g.off, j), __shfl(g.c, j), __shfl(g.eta, j), __shfl(g.slope, j), action, action == -2};
            if (first + j < a.N && k0 < K) store_unit<T>(static_cast<T *>(a.dlogits) + row_of(j) * a.dpitch, k0, K, gradient<T>(v[b], k0, h));
        }
    }
}

struct RowLds { float m[16], s[16], t[16]; };
// over all wavefronts of a workgroup; every thread gets the result
__device__ __forceinline__ float row_max(RowLds &lds, float m, int waves)
{
    m = wave_max(m);
    if ((threadIdx.x & 63) == 0) lds.m[threadIdx.x >> 6] = m;
    __syncthreads();
    m = lds.m[0];
    for (int w = 1; w < waves; ++w) m = fmaxf(m, lds.m[w]);
    return m;
}
__device__ __forceinline__ void row_sums(RowLds &lds, Sums &q, int waves)
{
    q.s = wave_sum(q.s); q.t = wave_sum(q.t);
    if ((threadIdx.x & 63) == 0) { lds.s[threadIdx.x >> 6] = q.s; lds.t[threadIdx.x >> 6] = q.t; }
    __syncthreads();
    q.s = lds.s[0]; q.t = lds.t[0];
    for (int w = 1; w < waves; ++w) { q.s += lds.s[w]; q.t += lds.t[w]; }
}

// Longer rows: a workgroup (of one wavefront up to sixteen) holds one in registers, U units of 16 bytes per thread, and reads it once.
template <class T, int U, bool GRAD>
__global__ void __launch_bounds__(1024) policy_row_kernel(PolicyArgs a)
{
    constexpr int V = Unit<T>::V;
    __shared__ RowLds lds;
    const int64_t n = blockIdx.x;
    const int tid = threadIdx.x, threads = blockDim.x, waves = threads >> 6, K = a.K;
    const Row r = load_row(a, n);
    const T *x = static_cast<const T *>(a.logits) + n * a.pitch;
    T *dx = GRAD ? static_cast<T *>(a.dlogits) + n * a.dpitch : nullptr;
    typename Unit<T>::raw v[U];
    Slope g;
    float loss;
    if (r.idle) {                            // (uniform)
        g = finish_row(a, n, r, Sums{0.f, 0.f, 0.f}, 0.f, tid == 0, loss);
#pragma unroll
        for (int j = 0; j < U; ++j) {
#pragma unroll
            for (int i = 0; i < V; ++i) v[j][i] = (T)0.f;
        }
    } else {
        const float xa = logit_of_action(x, r, K);
#pragma unroll
        for (int j = 0; j < U; ++j) v[j] = load_unit<T>(x, (tid + j * threads) * V, K);
        Sums q = {LOWEST, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < U; ++j) q.m = max_of<T>(v[j], q.m);
        q.m = row_max(lds, q.m, waves);
        stay_packed<T>(v, q.m);
#pragma unroll
        for (int j = 0; j < U; ++j) add_unit<T>(v[j], q.m, q.s, q.t);
        stay_packed<T>(v, q.s);
        row_sums(lds, q, waves);             // (behind its barrier the gradient may be stored over the logits)
        g = finish_row(a, n, r, q, xa, tid == 0, loss);
    }
    if (tid == 0) a.part_loss[n] = loss;
    if constexpr (GRAD) {
#pragma unroll
        for (int j = 0; j < U; ++j) {
            const int k0 = (tid + j * threads) * V;
            if (k0 < K) store_unit<T>(dx, k0, K, gradient<T>(v[j], k0, g));
        }
    }
}

// Sums over units first .. last - 1 of a row, four of them in flight per thread, over the workgroup (every thread gets the result).  The maximum is the one so far: what
// was added up under a smaller one is scaled.
template <class T> __device__ __forceinline__ Sums running_sums(RowLds &lds, const T *x, int first, int last, int K)
{
    constexpr int V = Unit<T>::V, U = 4;
    const int threads = blockDim.x, waves = threads >> 6;
    const auto under = [](Sums &q, float m) {
        const float d = fmaxf((q.m - m) * LOG2E, FAR), scale = __builtin_amdgcn_exp2f(d);
        q = {m, q.s * scale, scale * fmaf(q.s, d, q.t)};
    };
    Sums q = {LOWEST, 0.f, 0.f};
    for (int u = first + (int)threadIdx.x; u < last; u += U * threads) {
        typename Unit<T>::raw v[U];
        float m = q.m;
#pragma unroll
        for (int j = 0; j < U; ++j) v[j] = load_unit<T>(x, u + j * threads < last ? (u + j * threads) * V : K, K);
#pragma unroll
        for (int j = 0; j < U; ++j) m = max_of<T>(v[j], m);
        stay_packed<T>(v, m);
        under(q, m);
#pragma unroll
        for (int j = 0; j < U; ++j) add_unit<T>(v[j], m, q.s, q.t);
    }
    under(q, row_max(lds, q.m, waves));
    row_sums(lds, q, waves);
    return q;
}

// Rows that no workgroup's registers hold, and the gradient from stored statistics, which needs nothing held: the row is read for either part.
template <class T, bool STATS, bool GRAD>
__global__ void __launch_bounds__(1024) policy_stream_kernel(PolicyArgs a)
{
    constexpr int V = Unit<T>::V;
    __shared__ RowLds lds;
    const int64_t n = blockIdx.x;
    const int tid = threadIdx.x, threads = blockDim.x, K = a.K, stride = threads * V;
    const Row r = load_row(a, n);
    const T *x = static_cast<const T *>(a.logits) + n * a.pitch;
    const float xa = logit_of_action(x, r, K);
    Slope g;
    if constexpr (STATS) {
        Sums q = {LOWEST, 0.f, 0.f};
        if (!r.idle) q = running_sums<T>(lds, x, 0, (K + V - 1) / V, K);         // (uniform)
        float loss;
        g = finish_row(a, n, r, q, xa, tid == 0, loss);
        if (tid == 0) a.part_loss[n] = loss;
    } else {
        __syncthreads();                     // every thread has read the action's logit before the first one stores over it
        g = stored_row(a, n, r, xa);
    }
    if constexpr (GRAD) {
        T *dx = static_cast<T *>(a.dlogits) + n * a.dpitch;
        for (int k0 = tid * V; k0 < K; k0 += stride) {
            typename Unit<T>::raw v;
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] = (T)0.f;
            if (!g.idle) v = load_unit<T>(x, k0, K);
            store_unit<T>(dx, k0, K, gradient<T>(v, k0, g));
        }
    }
}

// Few long rows: a row in pieces, a workgroup each, joined in the launch behind.  Partial sums lie as [N][pieces] m, s, t; then [N] the logits of the actions, which
// another piece's gradient may be stored over.
struct Pieces { int units, count; float *sums, *xa; };
constexpr int MAX_PIECES = 64;
template <class T>
__global__ void __launch_bounds__(256) policy_piece_kernel(PolicyArgs a, Pieces c)
{
    constexpr int V = Unit<T>::V;
    __shared__ RowLds lds;
    const int64_t n = blockIdx.x / (unsigned)c.count;
    const int piece = (int)(blockIdx.x - n * c.count), units = (a.K + V - 1) / V;
    const Row r = load_row(a, n);
    if (r.idle) return;                      // (uniform)
    const T *x = static_cast<const T *>(a.logits) + n * a.pitch;
    const Sums q = running_sums<T>(lds, x, piece * c.units, min((piece + 1) * c.units, units), a.K);
    if (threadIdx.x == 0) {
        float *o = c.sums + 3 * (n * c.count + piece);
        o[0] = q.m; o[1] = q.s; o[2] = q.t;
        if (piece == 0) c.xa[n] = logit_of_action(x, r, a.K);
    }
}
__device__ __forceinline__ Sums joined(const Pieces &c, int64_t n)
{
    const float *p = c.sums + 3 * n * c.count;
    float m = LOWEST;
    for (int i = 0; i < c.count; ++i) m = fmaxf(m, p[3 * i]);
    Sums q = {m, 0.f, 0.f};
    for (int i = 0; i < c.count; ++i) {
        const float d = fmaxf((p[3 * i] - m) * LOG2E, FAR), scale = __builtin_amdgcn_exp2f(d), s = p[3 * i + 1];
        q.s += s * scale;
        q.t += scale * fmaf(s, d, p[3 * i + 2]);
    }
    return q;
}
// the rows' results, a thread each, and the loss
__global__ void __launch_bounds__(256) policy_join_kernel(PolicyArgs a, Pieces c, float *__restrict__ loss_out)
{
    __shared__ double red[4];
    const int n = threadIdx.x;
    float loss = 0.f;
    if (n < a.N) {
        const Row r = load_row(a, n);
        const Sums q = r.idle ? Sums{LOWEST, 0.f, 0.f} : joined(c, n);
        finish_row(a, n, r, q, r.idle ? 0.f : c.xa[n], true, loss);
    }
    double s = loss;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o);
    if ((n & 63) == 0) red[n >> 6] = s;
    __syncthreads();
    if (n == 0) {
        for (int k = 1; k < (int)blockDim.x >> 6; ++k) s += red[k];
        loss_out[0] = (float)s;
    }
}
// a piece's gradient; every workgroup of a row joins its pieces for itself, or takes what a forward pass stored (not over the logits: one workgroup would read the
// action's logit where another had stored the gradient)
template <class T, bool STORED>
__global__ void __launch_bounds__(256) policy_piece_gradient_kernel(PolicyArgs a, Pieces c)
{
    constexpr int V = Unit<T>::V;
    const int64_t n = blockIdx.x / (unsigned)c.count;
    const int piece = (int)(blockIdx.x - n * c.count), units = (a.K + V - 1) / V, last = min((piece + 1) * c.units, units);
    const Row r = load_row(a, n);
    const T *x = static_cast<const T *>(a.logits) + n * a.pitch;
    T *dx = static_cast<T *>(a.dlogits) + n * a.dpitch;
    Slope g;
    if constexpr (STORED) {
        g = stored_row(a, n, r, logit_of_action(x, r, a.K));
    } else {
        const bool first = piece == 0 && threadIdx.x == 0;
        float loss;
        g = finish_row(a, n, r, r.idle ? Sums{LOWEST, 0.f, 0.f} : joined(c, n), r.idle ? 0.f : c.xa[n], first, loss);
        if (first) a.part_loss[n] = loss;
    }
    for (int u = piece * c.units + (int)threadIdx.x; u < last; u += 4 * 256) {
        typename Unit<T>::raw v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
#pragma unroll
            for (int i = 0; i < V; ++i) v[j][i] = (T)0.f;
            if (!g.idle && u + j * 256 < last) v[j] = load_unit<T>(x, (u + j * 256) * V, a.K);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int k0 = (u + j * 256) * V;
            if (u + j * 256 < last) store_unit<T>(dx, k0, a.K, gradient<T>(v[j], k0, g));
        }
    }
}

// loss = sum of the parts, in one fixed order
__global__ void __launch_bounds__(1024) policy_sum_kernel(const float *__restrict__ part, int64_t n, float *__restrict__ loss)
{
    __shared__ double red[16];
    double s = 0.0;
    int64_t i = threadIdx.x;
    const int64_t step = blockDim.x;
    for (; i + 7 * step < n; i += 8 * step) {
        float v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = part[i + k * step];
#pragma unroll
        for (int k = 0; k < 8; ++k) s += (double)v[k];
    }
    for (; i < n; i += step) s += (double)part[i];
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int k = 1; k < (int)blockDim.x >> 6; ++k) s += red[k];
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

// Few long rows go in pieces: a workgroup works through 65536 logits in about 6 us, whatever the other CUs do.  us, a workgroup per row and in pieces (forward; loss
// and gradient), bf16:  1 x 65536: 10.0, 7.2; 15.8, 9.9    16 x 65536: 10.4, 7.5; 16.3, 10.3    64 x 65536: 10.5, 8.3; 17.1, 12.5    4 x 300000: 28.7, 13.3; 52.6, 14.4
// and not:  16 x 16384: 6.3, 6.9; 8.2, 9.7    64 x 16384: 6.4, 6.6; 8.4, 9.8    128 x 32768: 8.2, 7.7; 12.1, 12.7    256 x 65536: 11.9, 13.7; 23.1, 26.4
constexpr int64_t PIECES_MAX_ROWS = 64, PIECES_MIN_UNITS = 4096, PIECE_UNITS = 256 * 4;
int pieces_of(int64_t N, int64_t units)
{
    if (N > PIECES_MAX_ROWS || units <= PIECES_MIN_UNITS) return 0;
    return units <= PIECE_UNITS * MAX_PIECES ? (int)((units + PIECE_UNITS - 1) / PIECE_UNITS) : MAX_PIECES;
}

// Who holds a row: part of a wavefront, a wavefront, a workgroup, or nobody.
// Workgroups, and so parts of the loss; none where a grid does not hold them.  With one, its part is the loss: `a.part_loss` is where that goes then (set here), and nothing is left to add up.
template <class T, bool STATS, bool GRAD> int64_t launch_rows_of(PolicyArgs &a, float *loss, hipStream_t s)
{
    constexpr int V = Unit<T>::V;
    const int64_t units = ((int64_t)a.K + V - 1) / V;
    if (units <= 64) {
        int lanes = 0;
        while ((1 << lanes) < units) ++lanes;
        const auto wave = [&](auto batches) {
            constexpr int B = decltype(batches)::value;
            const int64_t rows = 4 * (64 >> lanes) * B, blocks = (a.N + rows - 1) / rows;
            if (!fits_a_grid(blocks, 256)) return (int64_t)0;
            if (blocks == 1) a.part_loss = loss;
            hipLaunchKernelGGL((policy_wave_kernel<T, B, STATS, GRAD>), dim3((unsigned)blocks), dim3(256), 0, s, a, lanes);
            return blocks;
        };
        // (as many batches as leave two wavefronts to a SIMD; eight with a gradient would take half the wavefronts of a SIMD for their registers)
        const int64_t waves = a.N >> (6 - lanes);
        if constexpr (!GRAD) { if (lanes >= 3 && waves >= 8 * 2048) return wave(std::integral_constant<int, 8>{}); }
        if (lanes >= 2 && waves >= 4 * 2048) return wave(std::integral_constant<int, 4>{});
        if (lanes >= 1 && waves >= 2 * 2048) return wave(std::integral_constant<int, 2>{});
        return wave(std::integral_constant<int, 1>{});
    }
    if (a.N == 1) a.part_loss = loss;
    if constexpr (STATS) {
        const auto row = [&](auto u, int threads) {
            if (!fits_a_grid(a.N, threads)) return (int64_t)0;
            hipLaunchKernelGGL((policy_row_kernel<T, decltype(u)::value, GRAD>), dim3((unsigned)a.N), dim3(threads), 0, s, a);
            return a.N;
        };
        if (units <= 64 * 2) return row(std::integral_constant<int, 2>{}, 64);
        if (units <= 64 * 4) return row(std::integral_constant<int, 4>{}, 64);
        if (units <= 64 * 8) return row(std::integral_constant<int, 8>{}, 64);
        if (units <= 256 * 4) return row(std::integral_constant<int, 4>{}, 256);
        if (units <= 256 * 8) return row(std::integral_constant<int, 8>{}, 256);
        if (units <= 512 * 8) return row(std::integral_constant<int, 8>{}, 512);
        if (units <= 512 * 16) return row(std::integral_constant<int, 16>{}, 512);
        if constexpr (GRAD && sizeof(T) == 4) { if (units <= 1024 * 16) return row(std::integral_constant<int, 16>{}, 1024); }
    }
    // Beyond, held rows leave a CU one workgroup, which loads, computes and stores in turn; two that read the row again for the gradient are faster, but for
    // 32-bit logits. us, held and read: forward 2048 x 65536 f32 131, 95; 2048 x 131072 bf16 154, 100; 1024 x 70000 bf16 71, 36.  Loss and gradient 2048 x 131072 bf16 276, 259;
    // 1024 x 70000 bf16 104, 69; 300 x 100000 bf16 51, 41; 2048 x 65536 f32 228, 265; 2048 x 50000 f32 185, 196.  (Forward with 512 threads and 1024: 4096 x 65536 bf16 103, 111;
    // 1024 x 81920 f16 37, 43; 130 x 100000 bf16 14.9, 14.0; 100 x 131072 f32 18.8, 17.1.)
    const int threads = units <= 256 ? 64 : units <= 2048 ? 256 : STATS && !GRAD && a.N >= 512 ? 512 : 1024;
    if (!fits_a_grid(a.N, threads)) return 0;
    hipLaunchKernelGGL((policy_stream_kernel<T, STATS, GRAD>), dim3((unsigned)a.N), dim3(threads), 0, s, a);
    return a.N;
}
template <bool STATS, bool GRAD> ssm_status launch_rows(PolicyArgs &a, int dtype, float *loss, hipStream_t s)
{
    const int64_t units = ((int64_t)a.K * (int64_t)dtype_bytes(dtype) + 15) / 16;
    const int count = pieces_of(a.N, units);
    if (count && (STATS || a.dlogits != a.logits)) {
        Pieces c{(int)((units + count - 1) / count), count, STATS ? a.part_loss + PIECES_MAX_ROWS : nullptr, nullptr};
        if (STATS) c.xa = c.sums + 3 * a.N * count;
        if (STATS && a.N == 1) a.part_loss = loss;
        const dim3 grid((unsigned)(a.N * count));
        with_dtype(dtype, [&](auto t) {
            using T = decltype(t);
            if constexpr (STATS) hipLaunchKernelGGL(policy_piece_kernel<T>, grid, dim3(256), 0, s, a, c);
            if constexpr (GRAD) hipLaunchKernelGGL((policy_piece_gradient_kernel<T, !STATS>), grid, dim3(256), 0, s, a, c);
        });
        if constexpr (STATS && GRAD) { if (a.N > 1) hipLaunchKernelGGL(policy_sum_kernel, dim3(1), dim3(64), 0, s, a.part_loss, a.N, loss); }
        else if constexpr (STATS) hipLaunchKernelGGL(policy_join_kernel, dim3(1), dim3(64), 0, s, a, c, loss);
        return hipGetLastError() == hipSuccess ? SSM_OK : SSM_ERR_HIP;
    }
    const int64_t parts = with_dtype(dtype, [&](auto t) { return launch_rows_of<decltype(t), STATS, GRAD>(a, loss, s); });
    if (parts == 0) return SSM_ERR_UNSUPPORTED;
    if (hipGetLastError() != hipSuccess) return SSM_ERR_HIP;
    if (STATS && parts > 1) {
        hipLaunchKernelGGL(policy_sum_kernel, dim3(1), dim3(parts <= 256 ? 256 : 1024), 0, s, a.part_loss, parts, loss);
        if (hipGetLastError() != hipSuccess) return SSM_ERR_HIP;
    }
    return SSM_OK;
}

}  // namespace
}  // namespace ssm

using namespace ssm;

extern "C" {

size_t ssm_policy_loss_workspace_bytes(int64_t N, int64_t K)
{
    if (N <= 0 || K <= 0 || N > SSM_MAX_TOKENS || K > (1LL << 30) || K > SSM_MAX_ELEMS / N) return 0;
    // parts of the loss; few rows, which may go in pieces: the pieces' sums and the actions' logits
    const size_t floats = N <= PIECES_MAX_ROWS ? PIECES_MAX_ROWS + (3 * MAX_PIECES + 1) * (size_t)N : (size_t)N;
    return (floats * 4 + ALIGN - 1) / ALIGN * ALIGN;
}

ssm_status ssm_policy_loss_fwd(const void *logits, int64_t pitch, const int64_t *action, const float *logp_old,
                               const float *advantage, const float *weight, const float *logp_ref, ssm_policy_terms terms,
                               int dtype, int64_t N, int64_t K, float *loss, float *logp, float *entropy, float *lse,
                               void *workspace, size_t ws_bytes, void *stream)
{
    PolicyArgs a{logits, pitch, action, logp_old, advantage, weight, logp_ref, terms, N, (int)K, logp, entropy, lse, nullptr, nullptr, 0,
                 static_cast<float *>(workspace), N > 0 ? 1.f / (float)N : 0.f};
    if (const ssm_status rc = check_policy(a, dtype, N, K)) return rc;
    if (!loss || misaligned(loss, 4)) return SSM_ERR_INVALID_ARG;
    if (!workspace || misaligned(workspace, ALIGN) || ws_bytes < ssm_policy_loss_workspace_bytes(N, K)) return SSM_ERR_WORKSPACE;
    hipStream_t s = static_cast<hipStream_t>(stream);
    return launch_rows<true, false>(a, dtype, loss, s);
}

ssm_status ssm_policy_loss_bwd(const void *logits, int64_t pitch, const int64_t *action, const float *logp_old,
                               const float *advantage, const float *weight, const float *logp_ref, ssm_policy_terms terms,
                               int dtype, int64_t N, int64_t K, const float *logp, const float *entropy, const float *lse,
                               const float *dloss, void *dlogits, int64_t dpitch, void *stream)
{
    PolicyArgs a{logits, pitch, action, logp_old, advantage, weight, logp_ref, terms, N, (int)K, const_cast<float *>(logp),
                 const_cast<float *>(entropy), const_cast<float *>(lse), dloss, dlogits, dpitch, nullptr, N > 0 ? 1.f / (float)N : 0.f};
    if (const ssm_status rc = check_policy(a, dtype, N, K)) return rc;
    if (const ssm_status rc = check_gradient(a, dtype, N, K)) return rc;
    return launch_rows<false, true>(a, dtype, nullptr, static_cast<hipStream_t>(stream));
}

ssm_status ssm_policy_loss_grad(const void *logits, int64_t pitch, const int64_t *action, const float *logp_old,
                                const float *advantage, const float *weight, const float *logp_ref, ssm_policy_terms terms,
                                int dtype, int64_t N, int64_t K, const float *dloss, float *loss, float *logp, float *entropy,
                                float *lse, void *dlogits, int64_t dpitch, void *workspace, size_t ws_bytes, void *stream)
{
    PolicyArgs a{logits, pitch, action, logp_old, advantage, weight, logp_ref, terms, N, (int)K, logp, entropy, lse, dloss, dlogits, dpitch,
                 static_cast<float *>(workspace), N > 0 ? 1.f / (float)N : 0.f};
    if (const ssm_status rc = check_policy(a, dtype, N, K)) return rc;
    if (const ssm_status rc = check_gradient(a, dtype, N, K)) return rc;
    if (!loss || misaligned(loss, 4)) return SSM_ERR_INVALID_ARG;
    if (!workspace || misaligned(workspace, ALIGN) || ws_bytes < ssm_policy_loss_workspace_bytes(N, K)) return SSM_ERR_WORKSPACE;
    hipStream_t s = static_cast<hipStream_t>(stream);
    return launch_rows<true, true>(a, dtype, loss, s);
}

}  // extern "C"
