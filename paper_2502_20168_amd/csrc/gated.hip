// Gated linear recurrence with episode resets (gfx950): h_t = [not first_t] f_t h_{t-1} + (1 - f_t) u_t with f = sigmoid(gate), or
// with given coefficients, over sequences; its gradient pass; one step.
//
// Every (sequence, channel) is a lane of its own.  The recurrence over consecutive steps is the map h -> A h + S with A the product of
// the decays, and a reset among the steps makes it the constant S: maps compose as (A, S, r) after (A', S', r') = (A A', r ? S : A S' + S,
// r or r').  The flag stands beside A because a product of zero would let an infinite or NaN state through a reset.
// The gradient runs the same maps backwards: what flows from step t to t-1 is b_t = c_t (dh_t + b_{t+1}) with c_t = [not first_t] f_t, so steps t0..t1 map b
// to A b + G with the same A and r.
#include "elem.h"
#include "lookback.h"
#include "ssm_internal.h"

#include <type_traits>

namespace ssm {
namespace {

inline bool misaligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }

constexpr int GE = 4;                        // consecutive steps of a thread
constexpr int GV = 4;                        // neighbouring channels of a thread
constexpr int GATED_MAX_THREADS = 512;

struct GatedArgs {
    const void *gate, *u, *dh;
    ssm_strides gs, us, dhs;
    const uint8_t *is_first;
    const float *h0, *dh_last;
    const float *carry_in;
    void *h, *dgate, *du;
    ssm_strides hs, dgs, dus;
    float *h_last, *carry, *dh0;
    int Bt, L, D;
    int lgcx, lgspan;                        // log2 of a workgroup's vectors of channels and of the lanes of a wavefront that hold one sequence
    int rows, seqs;                          // threads along time of a sequence, sequences of a workgroup (several: each within a wavefront)
    int nCX, nTB, carry_rows;                // channel blocks, chunks along time
    // chunks in workgroups of their own
    unsigned long long *desc;                // [nTB][nCX * Bt][3][64] tagged words, zero on entry: A, S and the state behind the chunk
    uint32_t *ticket, *err;
    uint32_t spin_limit;
    FastDiv by_chains;                       // nCX * Bt
};
constexpr int GATED_DESC_WORDS = 3 * 64;

// sigmoid(z) and 1 - sigmoid(z), both to the relative precision of the exponential: the difference where it is at least a half, exp(-z) sigmoid(z) else.
struct Gate { float f, i; };
__device__ __forceinline__ Gate gate_of(float z)
{
    const float e = __builtin_amdgcn_exp2f(z * -1.44269504f), f = __builtin_amdgcn_rcpf(1.f + e);
    return {f, e > 1.f ? 1.f - f : e * f};
}

__device__ __forceinline__ f32x4 fma4(f32x4 a, f32x4 b, f32x4 c)
{
    f32x4 r;
#pragma unroll
    for (int k = 0; k < 4; ++k) r[k] = fmaf(a[k], b[k], c[k]);
    return r;
}
__device__ __forceinline__ f32x4 pick4(bool c, f32x4 a, f32x4 b)
{
    f32x4 r;
#pragma unroll
    for (int k = 0; k < 4; ++k) r[k] = c ? a[k] : b[k];
    return r;
}
__device__ __forceinline__ f32x4 up4(f32x4 v, int d)
{
    f32x4 r;
#pragma unroll
    for (int k = 0; k < 4; ++k) r[k] = __shfl_up(v[k], d);
    return r;
}
__device__ __forceinline__ f32x4 down4(f32x4 v, int d)
{
    f32x4 r;
#pragma unroll
    for (int k = 0; k < 4; ++k) r[k] = __shfl_down(v[k], d);
    return r;
}

// a map over consecutive steps: v -> A v + S, or the constant S where r
struct Map { f32x4 A, S; int r; };
__device__ __forceinline__ Map identity() { return {f32x4{1.f, 1.f, 1.f, 1.f}, f32x4{0.f, 0.f, 0.f, 0.f}, 0}; }
__device__ __forceinline__ Map after(const Map &y, const Map &x)      // x first, then y
{
    return {y.A * x.A, pick4(y.r, y.S, fma4(y.A, x.S, y.S)), y.r | x.r};
}
__device__ __forceinline__ f32x4 apply(const Map &m, f32x4 v) { return pick4(m.r, m.S, fma4(m.A, v, m.S)); }
__device__ __forceinline__ Map pick(bool c, const Map &a, const Map &b) { return {pick4(c, a.A, b.A), pick4(c, a.S, b.S), c ? a.r : b.r}; }

// Exclusive composition over the threads along time of a chunk: of the earlier ones (UP) or the later ones.  `lds`: a map per wavefront and vector of channels.
struct MapLds { f32x4 A[GATED_MAX_THREADS / 64][16], S[GATED_MAX_THREADS / 64][16]; int r[GATED_MAX_THREADS / 64][16]; };
template <bool UP> __device__ __forceinline__ Map inclusive_in_wave(Map m, int lane, int cx, int span)
{
    const int l = lane & (span - 1);
    for (int d = cx; d < span; d <<= 1) {
        Map o;
        if constexpr (UP) o = {up4(m.A, d), up4(m.S, d), __shfl_up(m.r, d)};
        else o = {down4(m.A, d), down4(m.S, d), __shfl_down(m.r, d)};
        m = pick(UP ? l >= d : l + d < span, after(m, o), m);
    }
    return m;
}
template <bool UP> __device__ __forceinline__ Map exclusive_in_wave(const Map &incl, int lane, int cx, int span)
{
    const int l = lane & (span - 1);
    Map o;
    if constexpr (UP) o = {up4(incl.A, cx), up4(incl.S, cx), __shfl_up(incl.r, cx)};
    else o = {down4(incl.A, cx), down4(incl.S, cx), __shfl_down(incl.r, cx)};
    return pick(UP ? l >= cx : l + cx < span, o, identity());
}
__device__ __forceinline__ void put(MapLds &s, int w, int c, const Map &m) { s.A[w][c] = m.A; s.S[w][c] = m.S; s.r[w][c] = m.r; }
__device__ __forceinline__ Map get(const MapLds &s, int w, int c) { return {s.A[w][c], s.S[w][c], s.r[w][c]}; }

// What a thread owns: GE steps of GV channels of one sequence.  Threads past the end of an axis take the last valid place and store nothing.
// The last vector of a row is moved back so that it ends with the row: its channels are computed twice, with the same operations, and the same values stored twice.
struct Place {
    int vec, row, seq, ch, lane, span, wave, waves;      // waves: of a sequence, where there is one per workgroup
    bool stored;
    __device__ __forceinline__ Place(const GatedArgs &a, int chain)
    {
        const int tid = threadIdx.x, cx = 1 << a.lgcx;
        const bool several = a.seqs > 1;
        lane = tid & 63;
        wave = tid >> 6;
        span = 1 << a.lgspan;
        vec = tid & (cx - 1);
        row = (several ? tid & (span - 1) : tid) >> a.lgcx;
        waves = several ? 1 : (int)blockDim.x >> 6;
        const int s = several ? tid >> a.lgspan : 0, sb = chain / a.nCX, cb = chain - sb * a.nCX;
        const int b = sb * a.seqs + s, v = cb * cx + vec;
        stored = b < a.Bt && v * GV < a.D;
        seq = min(b, a.Bt - 1);
        ch = max(0, min(v * GV, a.D - GV));
    }
};

// What a chunk's neighbours hand over where every chunk has a workgroup of its own.  A workgroup publishes the map of its chunk before it waits for anything; then
// each of its rows fetches the map of one earlier chunk of its group of `rows` chunks, all at once, and one row the state behind the last chunk of
// the group before.  The order of the compositions is fixed, whatever the timing: results are repeatable.  Chunks are numbered by a ticket per chain (the chunks of one
// sequence and channel block), so that a workgroup waits for such as have started; a wait that gives up hands on NaN and says so in the workspace.
__device__ __forceinline__ bool wait_words(const unsigned long long *w, unsigned limit, f32x4 &v, unsigned &tag)
{
    for (unsigned spins = 0;; ++spins) {
        unsigned long long q[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) q[k] = poll_word(w + k);
        bool all = true;
#pragma unroll
        for (int k = 0; k < 4; ++k) { all = all && word_tag(q[k]) != 0; v[k] = word_value(q[k]); }
        tag = word_tag(q[0]);
        if (all) return true;
        if (spins >= limit) return false;
        __builtin_amdgcn_s_sleep(2);
    }
}
__device__ __forceinline__ void publish4(unsigned long long *w, f32x4 v, unsigned tag)
{
#pragma unroll
    for (int k = 0; k < 4; ++k) publish_word(w + k, v[k], tag);
}
// UP: rows in the order of time.  `chunk`: number along the direction of the scan; `total`: the chunk's map, valid where `ends`; v0: what flows into the first chunk.
template <bool UP> __device__ __forceinline__ f32x4 look_back(const GatedArgs &a, const Place &p, MapLds &lds, f32x4 *s_base, int chunk, int chain, const Map &total, bool ends, f32x4 v0)
{
    const int cx = 1 << a.lgcx, chains = a.nCX * a.Bt, group = chunk / a.rows * a.rows, row = UP ? p.row : a.rows - 1 - p.row;
    unsigned long long *mine = a.desc + ((int64_t)chunk * chains + chain) * GATED_DESC_WORDS + p.vec * GV;
    const int64_t back = (int64_t)chains * GATED_DESC_WORDS;
    if (ends && chunk + 1 < a.nTB) {
        publish4(mine, total.A, 1);
        publish4(mine + 64, total.S, total.r ? 2 : 1);
    }
    f32x4 v = v0;
    if (chunk > 0) {                         // (uniform)
        const f32x4 nan = {__builtin_nanf(""), __builtin_nanf(""), __builtin_nanf(""), __builtin_nanf("")};
        Map m = identity();
        if (group + row < chunk) {
            const unsigned long long *w = mine - (chunk - group - row) * back;
            unsigned tag;
            const bool got = wait_words(w, a.spin_limit, m.A, tag) && wait_words(w + 64, a.spin_limit, m.S, tag);
            m.r = tag == 2;
            if (!got) { atomicOr(a.err, 1u); m.S = nan; m.r = 1; }
        }
        if (group > 0 && row == 0) {
            unsigned tag;
            f32x4 base;
            if (!wait_words(mine - (chunk - group + 1) * back + 128, a.spin_limit, base, tag)) { atomicOr(a.err, 1u); base = nan; }
            s_base[p.vec] = base;
        }
        m = inclusive_in_wave<UP>(m, p.lane, cx, p.span);
        __syncthreads();                     // (the maps of the chunk itself have been read)
        if (UP ? p.lane >= 64 - cx : p.lane < cx) put(lds, p.wave, p.vec, m);
        __syncthreads();
        Map w = identity();
        for (int k = 0; k < p.waves; ++k) w = after(get(lds, UP ? k : p.waves - 1 - k, p.vec), w);
        v = apply(w, group > 0 ? s_base[p.vec] : v0);
    }
    if (ends && chunk + 1 < a.nTB && (chunk + 1) % a.rows == 0) publish4(mine + 128, apply(total, v), 3);
    return v;
}
// the chunk and the chain of this workgroup
__device__ __forceinline__ int take_ticket(const GatedArgs &a, int &chain)
{
    __shared__ int s_chunk;
    const int chains = a.nCX * a.Bt;
    chain = (int)blockIdx.x - (int)a.by_chains(blockIdx.x) * chains;
    if (threadIdx.x == 0) s_chunk = (int)atomicAdd(a.ticket + (int64_t)chain * SCAN_TICKET_STRIDE, 1u);
    __syncthreads();
    return __builtin_amdgcn_readfirstlane(s_chunk);
}

// NARROW: rows of fewer than GV channels, whose one vector repeats the last of them.
template <class T, bool NARROW> __device__ __forceinline__ typename Pack<T, 4>::type load_channels(const T *p, int D)
{
    if constexpr (!NARROW) return load_pack<T, 4>(p);
    typename Pack<T, 4>::type v;
#pragma unroll
    for (int k = 0; k < GV; ++k) v[k] = p[min(k, D - 1)];
    return v;
}
template <class T, bool NARROW> __device__ __forceinline__ void store_channels(T *p, int D, typename Pack<T, 4>::type v)
{
    if constexpr (!NARROW) { store_pack<T, 4>(p, v); return; }
#pragma unroll
    for (int k = 0; k < GV; ++k) if (k < D) p[k] = v[k];
}

// (steps past the end repeat the last one)
template <class T, bool NARROW> __device__ __forceinline__ void load_steps(typename Pack<T, 4>::type (&v)[GE], const void *base, const ssm_strides &st, const Place &p, int t0, int L, int D)
{
    const T *q = static_cast<const T *>(base) + (int64_t)p.seq * st.seq + p.ch + (int64_t)min(t0, L - 1) * st.step;
#pragma unroll
    for (int e = 0; e < GE; ++e) {
        v[e] = load_channels<T, NARROW>(q, D);
        q += t0 + e + 1 < L ? st.step : 0;
    }
}

// (values of 16 bits that are needed again stay packed meanwhile)
template <class T> __device__ __forceinline__ void stay_packed(typename Pack<T, 4>::type (&v)[GE])
{
    typedef unsigned words __attribute__((ext_vector_type(2)));
    if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int e = 0; e < GE; ++e) {
            words w = __builtin_bit_cast(words, v[e]);
            asm volatile("" : "+v"(w));
            v[e] = __builtin_bit_cast(typename Pack<T, 4>::type, w);
        }
    }
}

// flags of a thread's steps, bit e = the state that flows into step t0 + e is dropped
__device__ __forceinline__ unsigned reset_mask(const GatedArgs &a, const Place &p, int t0)
{
    unsigned m = 0;
    if (a.is_first) {
        const uint8_t *q = a.is_first + (int64_t)p.seq * a.L;
#pragma unroll
        for (int e = 0; e < GE; ++e) m |= (unsigned)(q[min(t0 + e, a.L - 1)] != 0) << e;
        const int left = a.L - t0;
        if (left < GE) m &= (1u << max(left, 0)) - 1u;
    }
    return m;
}

template <class T, bool LINEAR, bool NARROW, bool LOOK>
__global__ void __launch_bounds__(GATED_MAX_THREADS) gated_fwd_kernel(GatedArgs a)
{
    __shared__ MapLds lds;
    __shared__ f32x4 s_end[16];              // state at the end of the chunk before
    int chain = blockIdx.x, first = 0;
    if constexpr (LOOK) first = take_ticket(a, chain);
    const Place p(a, chain);
    const int cx = 1 << a.lgcx, steps = GE * a.rows;
    f32x4 in = {0.f, 0.f, 0.f, 0.f};         // state that flows into the chunk
    if (a.h0) in = load_channels<float, NARROW>(a.h0 + (int64_t)p.seq * a.D + p.ch, a.D);
    for (int tb = first; tb < (LOOK ? first + 1 : a.nTB); ++tb) {
        const int t0 = tb * steps + p.row * GE;
        typename Pack<T, 4>::type z[GE], u[GE];
        load_steps<T, NARROW>(z, a.gate, a.gs, p, t0, a.L, a.D);
        load_steps<T, NARROW>(u, a.u, a.us, p, t0, a.L, a.D);
        const unsigned cut = reset_mask(a, p, t0);
        f32x4 f[GE], b[GE];
        Map m = identity();
#pragma unroll
        for (int e = 0; e < GE; ++e) {
            const f32x4 ze = widened4<T>(z[e]), ue = widened4<T>(u[e]);
            if constexpr (LINEAR) {
                f[e] = ze; b[e] = ue;
            } else {
#pragma unroll
                for (int k = 0; k < GV; ++k) { const Gate g = gate_of(ze[k]); f[e][k] = g.f; b[e][k] = g.i * ue[k]; }
            }
            m = after(Map{f[e], b[e], (int)((cut >> e) & 1u)}, m);
        }
        m = inclusive_in_wave<true>(m, p.lane, cx, p.span);
        Map before = exclusive_in_wave<true>(m, p.lane, cx, p.span);
        if (p.waves > 1) {                   // (uniform)
            if (p.lane >= 64 - cx) put(lds, p.wave, p.vec, m);
            __syncthreads();
            Map w = identity();
            for (int k = 0; k < p.wave; ++k) w = after(get(lds, k, p.vec), w);
            if constexpr (LOOK) m = after(m, w);
            before = after(before, w);
        }
        if constexpr (LOOK) in = look_back<true>(a, p, lds, s_end, tb, chain, m, p.row == a.rows - 1, in);
        f32x4 h = apply(before, in);
        if (a.carry && p.stored && t0 > 0 && t0 < a.L && t0 % SSM_GATED_CARRY_STEPS == 0)
            store_channels<float, NARROW>(a.carry + ((int64_t)p.seq * a.carry_rows + t0 / SSM_GATED_CARRY_STEPS - 1) * a.D + p.ch, a.D, h);
        T *out = static_cast<T *>(a.h) + (int64_t)p.seq * a.hs.seq + p.ch;
#pragma unroll
        for (int e = 0; e < GE; ++e) {
            h = pick4((cut >> e) & 1u, b[e], fma4(f[e], h, b[e]));
            const int t = t0 + e;
            if (p.stored && t < a.L) {
                store_channels<T, NARROW>(out + (int64_t)t * a.hs.step, a.D, rounded4<T>(h));
                if (t == a.L - 1 && a.h_last) store_channels<float, NARROW>(a.h_last + (int64_t)p.seq * a.D + p.ch, a.D, h);
            }
        }
        if (!LOOK && tb + 1 < a.nTB) {
            if (p.row == a.rows - 1) s_end[p.vec] = h;
            __syncthreads();
            in = s_end[p.vec];
        }
    }
}

template <class T, bool LINEAR, bool NARROW, bool LOOK>
__global__ void __launch_bounds__(GATED_MAX_THREADS) gated_bwd_kernel(GatedArgs a)
{
    __shared__ MapLds lds_up, lds_down;
    __shared__ f32x4 s_end[16];
    int chain = blockIdx.x, first = a.nTB - 1;
    if constexpr (LOOK) first = a.nTB - 1 - take_ticket(a, chain);
    const Place p(a, chain);
    const int cx = 1 << a.lgcx, steps = GE * a.rows;
    const int64_t state = (int64_t)p.seq * a.D + p.ch;
    f32x4 from_right = {0.f, 0.f, 0.f, 0.f};
    if (a.dh_last) from_right = load_channels<float, NARROW>(a.dh_last + state, a.D);
    for (int tb = first; tb >= (LOOK ? first : 0); --tb) {
        const int t0 = tb * steps + p.row * GE;
        typename Pack<T, 4>::type z[GE], u[GE], d[GE];
        load_steps<T, NARROW>(d, a.dh, a.dhs, p, t0, a.L, a.D);
        load_steps<T, NARROW>(z, a.gate, a.gs, p, t0, a.L, a.D);
        load_steps<T, NARROW>(u, a.u, a.us, p, t0, a.L, a.D);
        const unsigned cut = reset_mask(a, p, t0);
        f32x4 in = {0.f, 0.f, 0.f, 0.f};
        if (tb > 0) in = load_channels<float, NARROW>(a.carry_in + ((int64_t)p.seq * a.carry_rows + tb * steps / SSM_GATED_CARRY_STEPS - 1) * a.D + p.ch, a.D);
        else if (a.h0) in = load_channels<float, NARROW>(a.h0 + state, a.D);
        // steps past the end let what flows backwards through: decay 1, no term of their own
        f32x4 f[GE], i[LINEAR ? 1 : GE];
        Map up = identity();
#pragma unroll
        for (int e = 0; e < GE; ++e) {
            const f32x4 ze = widened4<T>(z[e]), ue = widened4<T>(u[e]);
            const bool past = t0 + e >= a.L;
            f32x4 b;
            if constexpr (LINEAR) {
                f[e] = ze; b = ue;
            } else {
#pragma unroll
                for (int k = 0; k < GV; ++k) { const Gate g = gate_of(ze[k]); f[e][k] = g.f; i[e][k] = g.i; }
                b = i[e] * ue;
            }
            f[e] = pick4(past, f32x4{1.f, 1.f, 1.f, 1.f}, f[e]);
            up = after(Map{f[e], b, (int)((cut >> e) & 1u)}, up);
        }
        Map down = {up.A, f32x4{0.f, 0.f, 0.f, 0.f}, up.r};
#pragma unroll
        for (int e = GE - 1; e >= 0; --e) {
            const f32x4 de = pick4(t0 + e >= a.L, f32x4{0.f, 0.f, 0.f, 0.f}, widened4<T>(d[e]));
            down.S = pick4((cut >> e) & 1u, f32x4{0.f, 0.f, 0.f, 0.f}, f[e] * (de + down.S));
        }
        stay_packed<T>(u);
        stay_packed<T>(d);
        __builtin_amdgcn_sched_barrier(0);
        up = inclusive_in_wave<true>(up, p.lane, cx, p.span);
        Map before = exclusive_in_wave<true>(up, p.lane, cx, p.span);
        __builtin_amdgcn_sched_barrier(0);
        down = inclusive_in_wave<false>(down, p.lane, cx, p.span);
        Map behind = exclusive_in_wave<false>(down, p.lane, cx, p.span);
        __builtin_amdgcn_sched_barrier(0);
        if (p.waves > 1) {
            if (p.lane >= 64 - cx) put(lds_up, p.wave, p.vec, up);
            if (p.lane < cx) put(lds_down, p.wave, p.vec, down);
            __syncthreads();
            Map w = identity();
            for (int k = 0; k < p.wave; ++k) w = after(get(lds_up, k, p.vec), w);
            before = after(before, w);
            w = identity();
            for (int k = p.waves - 1; k > p.wave; --k) w = after(get(lds_down, k, p.vec), w);
            if constexpr (LOOK) down = after(down, w);
            behind = after(behind, w);
        }
        if constexpr (LOOK) from_right = look_back<false>(a, p, lds_down, s_end, a.nTB - 1 - tb, chain, down, p.row == 0, from_right);
        // chi, last step first
        f32x4 back = apply(behind, from_right), chi[GE];
#pragma unroll
        for (int e = GE - 1; e >= 0; --e) {
            const bool past = t0 + e >= a.L;
            chi[e] = widened4<T>(d[e]) + back;
            back = pick4((cut >> e) & 1u, f32x4{0.f, 0.f, 0.f, 0.f}, pick4(past, back, f[e] * chi[e]));
        }
        // the states again, first step first, and the gradients
        f32x4 h = apply(before, in);
        T *dgate = static_cast<T *>(a.dgate) + (int64_t)p.seq * a.dgs.seq + p.ch, *du = static_cast<T *>(a.du) + (int64_t)p.seq * a.dus.seq + p.ch;
#pragma unroll
        for (int e = 0; e < GE; ++e) {
            const int t = t0 + e;
            const f32x4 ue = widened4<T>(u[e]), prev = pick4((cut >> e) & 1u, f32x4{0.f, 0.f, 0.f, 0.f}, h);
            f32x4 gu, gz;
            if constexpr (LINEAR) {
                gu = chi[e]; gz = prev * chi[e];
                h = fma4(f[e], prev, ue);
            } else {
                gu = i[e] * chi[e]; gz = f[e] * (prev - ue) * gu;
                h = fma4(f[e], prev, i[e] * ue);
            }
            if (p.stored && t < a.L) {
                store_channels<T, NARROW>(du + (int64_t)t * a.dus.step, a.D, rounded4<T>(gu));
                store_channels<T, NARROW>(dgate + (int64_t)t * a.dgs.step, a.D, rounded4<T>(gz));
            }
        }
        if (t0 == 0 && a.dh0 && p.stored) store_channels<float, NARROW>(a.dh0 + state, a.D, back);
        if (!LOOK && tb > 0) {
            if (p.row == 0) s_end[p.vec] = back;
            __syncthreads();
            from_right = s_end[p.vec];
        }
    }
}

template <class T, bool LINEAR>
__global__ void __launch_bounds__(256) gated_step_kernel(const T *__restrict__ gate, int64_t gate_pitch, const T *__restrict__ u, int64_t u_pitch,
                                                         const float *h_prev, const uint8_t *__restrict__ is_first, int64_t n, int D, float *h, T *__restrict__ y)
{
    const int64_t j = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (j >= n) return;
    const int64_t b = j / D, c = j - b * D;
    const float z = (float)gate[b * gate_pitch + c], x = (float)u[b * u_pitch + c];
    const bool cut = (is_first && is_first[b]) || !h_prev;
    float f = z, v = x;
    if constexpr (!LINEAR) { const Gate g = gate_of(z); f = g.f; v = g.i * x; }
    const float r = cut ? v : fmaf(f, h_prev[j], v);
    h[j] = r;
    if (y) y[j] = rounded<T>(r);
}

// Vectors of channels and threads along time of a workgroup, sequences per workgroup, chunks of a sequence; look: a workgroup per chunk.
struct GatedPlan { int lgcx, lgspan, rows, seqs, threads, nCX, nTB; bool look; int64_t blocks; size_t ticket_bytes, desc_bytes; };
GatedPlan plan_gated(int64_t Bt, int64_t L, int64_t D)
{
    GatedPlan pl{};
    const int64_t vecs = (D + GV - 1) / GV, rows = (L + GE - 1) / GE;
    const auto blocks_at = [&](int lg) { return Bt * ((vecs + (1 << lg) - 1) >> lg); };
    pl.lgcx = 0;
    while (pl.lgcx < 4 && (1 << pl.lgcx) < vecs) ++pl.lgcx;
    const int widest = pl.lgcx;
    while (pl.lgcx > 2 && rows > (GATED_MAX_THREADS >> pl.lgcx) && blocks_at(pl.lgcx) < 512) --pl.lgcx;
    if (rows > (GATED_MAX_THREADS >> pl.lgcx)) pl.lgcx = widest;
    const int cx = 1 << pl.lgcx;
    if (rows * cx <= 64) {                   // a sequence within a wavefront
        pl.lgspan = pl.lgcx;
        while ((1 << pl.lgspan) < rows * cx) ++pl.lgspan;
        pl.rows = 1 << (pl.lgspan - pl.lgcx);
        pl.threads = 256;
        while (pl.threads > 64 && (Bt * vecs * pl.rows) / pl.threads < 512) pl.threads /= 2;
        pl.seqs = pl.threads >> pl.lgspan;
        pl.nTB = 1;
    } else {                                 // a sequence, or a chunk of one, per workgroup: whole wavefronts
        const int per_wave = 64 >> pl.lgcx, most = GATED_MAX_THREADS >> pl.lgcx;
        pl.lgspan = 6;
        pl.rows = (int)(rows <= most ? (rows + per_wave - 1) / per_wave * per_wave : most);
        pl.threads = pl.rows * cx;
        pl.seqs = 1;
        pl.nTB = (int)((rows + pl.rows - 1) / pl.rows);
    }
    pl.nCX = (int)((vecs + cx - 1) >> pl.lgcx);
    const int64_t chains = (int64_t)pl.nCX * ((Bt + pl.seqs - 1) / pl.seqs);
    pl.look = pl.nTB > 1 && chains < 512 && chains * pl.nTB <= 0x7fffffffLL;
    pl.blocks = pl.look ? chains * pl.nTB : chains;
    if (pl.look) {
        pl.ticket_bytes = (size_t)chains * SCAN_TICKET_STRIDE * sizeof(uint32_t);
        pl.desc_bytes = (size_t)pl.blocks * GATED_DESC_WORDS * sizeof(unsigned long long);
    }
    return pl;
}
constexpr size_t GATED_HEADER = 256;

bool input_strides_ok(const ssm_strides &s) { return s.seq >= 0 && s.step >= 0; }
// no two elements in one place: steps within sequences, or sequences within steps
bool output_strides_ok(const ssm_strides &s, int64_t Bt, int64_t L, int64_t D)
{
    const bool steps_apart = L == 1 || s.step >= D, seqs_apart = Bt == 1 || s.seq >= D;
    if (s.seq < 0 || s.step < 0 || !steps_apart || !seqs_apart) return false;
    return L == 1 || Bt == 1 || s.seq / L >= s.step || s.step / Bt >= s.seq || s.seq >= (L - 1) * s.step + D || s.step >= (Bt - 1) * s.seq + D;
}
constexpr int64_t MAX_STRIDE = 1LL << 40;
bool strides_in_range(const ssm_strides &s, int64_t Bt, int64_t L)
{
    return s.seq <= MAX_STRIDE && s.step <= MAX_STRIDE && (Bt == 1 || s.seq <= (1LL << 60) / Bt) && (L == 1 || s.step <= (1LL << 60) / L);
}
ssm_status check_shape(int dtype, int64_t Bt, int64_t L, int64_t D)
{
    if (Bt <= 0 || L <= 0 || D <= 0 || !dtype_known(dtype)) return SSM_ERR_INVALID_ARG;
    if (D > SSM_MAX_WIDTH || Bt > SSM_MAX_TOKENS || L > SSM_MAX_TOKENS / Bt || Bt * L > SSM_MAX_ELEMS / D) return SSM_ERR_UNSUPPORTED;
    return SSM_OK;
}

ssm_status launch_gated(GatedArgs &a, bool reverse, int dtype, int linear, void *workspace, size_t ws_bytes, hipStream_t s)
{
    const GatedPlan pl = plan_gated(a.Bt, a.L, a.D);
    if (pl.blocks > 0x7fffffffLL) return SSM_ERR_UNSUPPORTED;
    a.lgcx = pl.lgcx; a.lgspan = pl.lgspan; a.rows = pl.rows; a.seqs = pl.seqs; a.nCX = pl.nCX; a.nTB = pl.nTB;
    a.carry_rows = (int)ssm_gated_carry_rows(a.L);
    if (pl.look) {
        const size_t scratch = pl.ticket_bytes + pl.desc_bytes;
        if (!workspace || misaligned(workspace, 256) || ws_bytes < GATED_HEADER + scratch) return SSM_ERR_WORKSPACE;
        char *ws = static_cast<char *>(workspace);
        a.err = reinterpret_cast<uint32_t *>(ws);
        a.ticket = reinterpret_cast<uint32_t *>(ws + GATED_HEADER);
        a.desc = reinterpret_cast<unsigned long long *>(ws + GATED_HEADER + pl.ticket_bytes);
        a.spin_limit = scan_spin_limit();
        a.by_chains = FastDiv::by((unsigned)((int64_t)pl.nCX * a.Bt));
        if (launch_clear(reinterpret_cast<WsHeader *>(ws), ws + GATED_HEADER, scratch, s) != hipSuccess) return SSM_ERR_HIP;
    }
    const dim3 grid((unsigned)pl.blocks), block((unsigned)pl.threads);
    with_dtype(dtype, [&](auto t) {
        using T = decltype(t);
        const auto go = [&](auto lin, auto nar, auto look) {
            constexpr bool LIN = decltype(lin)::value, NAR = decltype(nar)::value, LOOK = decltype(look)::value;
            if (reverse) hipLaunchKernelGGL((gated_bwd_kernel<T, LIN, NAR, LOOK>), grid, block, 0, s, a);
            else hipLaunchKernelGGL((gated_fwd_kernel<T, LIN, NAR, LOOK>), grid, block, 0, s, a);
        };
        const std::true_type yes; const std::false_type no;
        const auto chunks = [&](auto lin, auto nar) { if (pl.look) go(lin, nar, yes); else go(lin, nar, no); };
        const auto width = [&](auto lin) { if (a.D < GV) chunks(lin, yes); else chunks(lin, no); };
        if (linear) width(yes); else width(no);
    });
    return hipGetLastError() == hipSuccess ? SSM_OK : SSM_ERR_HIP;
}

}  // namespace
}  // namespace ssm

using namespace ssm;

extern "C" {

int64_t ssm_gated_carry_rows(int64_t L) { return L > 0 ? (L - 1) / SSM_GATED_CARRY_STEPS : 0; }

size_t ssm_gated_workspace_bytes(int64_t Bt, int64_t L, int64_t D, int dtype, int)
{
    if (check_shape(dtype, Bt, L, D) != SSM_OK) return 0;
    const GatedPlan pl = plan_gated(Bt, L, D);
    return pl.look ? GATED_HEADER + pl.ticket_bytes + pl.desc_bytes : 0;
}

ssm_status ssm_gated_scan_fwd(const void *gate, ssm_strides gate_strides, const void *u, ssm_strides u_strides,
                              const uint8_t *is_first, const float *h0, int dtype, int linear,
                              int64_t Bt, int64_t L, int64_t D, void *h, ssm_strides h_strides, float *h_last, float *carry,
                              void *workspace, size_t ws_bytes, void *stream)
{
    if (!gate || !u || !h) return SSM_ERR_INVALID_ARG;
    if (const ssm_status rc = check_shape(dtype, Bt, L, D)) return rc;
    const size_t e = dtype_bytes(dtype);
    if (misaligned(gate, e) || misaligned(u, e) || misaligned(h, e) || misaligned(h0, 4) || misaligned(h_last, 4) || misaligned(carry, 4))
        return SSM_ERR_INVALID_ARG;
    if (!input_strides_ok(gate_strides) || !input_strides_ok(u_strides) || !output_strides_ok(h_strides, Bt, L, D)) return SSM_ERR_INVALID_ARG;
    if (!strides_in_range(gate_strides, Bt, L) || !strides_in_range(u_strides, Bt, L) || !strides_in_range(h_strides, Bt, L)) return SSM_ERR_UNSUPPORTED;
    GatedArgs a{};
    a.gate = gate; a.gs = gate_strides; a.u = u; a.us = u_strides; a.is_first = is_first; a.h0 = h0;
    a.h = h; a.hs = h_strides; a.h_last = h_last; a.carry = carry;
    a.Bt = (int)Bt; a.L = (int)L; a.D = (int)D;
    return launch_gated(a, false, dtype, linear, workspace, ws_bytes, static_cast<hipStream_t>(stream));
}

ssm_status ssm_gated_scan_bwd(const void *gate, ssm_strides gate_strides, const void *u, ssm_strides u_strides,
                              const uint8_t *is_first, const float *h0, const float *carry,
                              const void *dh, ssm_strides dh_strides, const float *dh_last, int dtype, int linear,
                              int64_t Bt, int64_t L, int64_t D, void *dgate, ssm_strides dgate_strides,
                              void *du, ssm_strides du_strides, float *dh0,
                              void *workspace, size_t ws_bytes, void *stream)
{
    if (!gate || !u || !dh || !dgate || !du) return SSM_ERR_INVALID_ARG;
    if (const ssm_status rc = check_shape(dtype, Bt, L, D)) return rc;
    if (!carry && ssm_gated_carry_rows(L) > 0) return SSM_ERR_INVALID_ARG;
    const size_t e = dtype_bytes(dtype);
    if (misaligned(gate, e) || misaligned(u, e) || misaligned(dh, e) || misaligned(dgate, e) || misaligned(du, e) || misaligned(h0, 4) ||
        misaligned(carry, 4) || misaligned(dh_last, 4) || misaligned(dh0, 4))
        return SSM_ERR_INVALID_ARG;
    if (!input_strides_ok(gate_strides) || !input_strides_ok(u_strides) || !input_strides_ok(dh_strides) ||
        !output_strides_ok(dgate_strides, Bt, L, D) || !output_strides_ok(du_strides, Bt, L, D))
        return SSM_ERR_INVALID_ARG;
    if (!strides_in_range(gate_strides, Bt, L) || !strides_in_range(u_strides, Bt, L) || !strides_in_range(dh_strides, Bt, L) ||
        !strides_in_range(dgate_strides, Bt, L) || !strides_in_range(du_strides, Bt, L))
        return SSM_ERR_UNSUPPORTED;
    GatedArgs a{};
    a.gate = gate; a.gs = gate_strides; a.u = u; a.us = u_strides; a.is_first = is_first; a.h0 = h0; a.carry_in = carry;
    a.dh = dh; a.dhs = dh_strides; a.dh_last = dh_last;
    a.dgate = dgate; a.dgs = dgate_strides; a.du = du; a.dus = du_strides; a.dh0 = dh0;
    a.Bt = (int)Bt; a.L = (int)L; a.D = (int)D;
    return launch_gated(a, true, dtype, linear, workspace, ws_bytes, static_cast<hipStream_t>(stream));
}

ssm_status ssm_gated_step(const void *gate, int64_t gate_pitch, const void *u, int64_t u_pitch, const float *h_prev,
                          const uint8_t *is_first, int dtype, int linear, int64_t Bt, int64_t D, float *h, void *y, void *stream)
{
    if (!gate || !u || !h) return SSM_ERR_INVALID_ARG;
    if (const ssm_status rc = check_shape(dtype, Bt, 1, D)) return rc;
    const size_t e = dtype_bytes(dtype);
    if (misaligned(gate, e) || misaligned(u, e) || misaligned(y, e) || misaligned(h_prev, 4) || misaligned(h, 4) || gate_pitch < 0 || u_pitch < 0)
        return SSM_ERR_INVALID_ARG;
    if (!strides_in_range({gate_pitch, 0}, Bt, 1) || !strides_in_range({u_pitch, 0}, Bt, 1)) return SSM_ERR_UNSUPPORTED;
    const int64_t n = Bt * D;
    if (n > 0x7fffffffLL * 256) return SSM_ERR_UNSUPPORTED;
    const dim3 grid((unsigned)((n + 255) / 256)), block(256);
    hipStream_t s = static_cast<hipStream_t>(stream);
    with_dtype(dtype, [&](auto t) {
        using T = decltype(t);
        const T *g = static_cast<const T *>(gate), *x = static_cast<const T *>(u);
        if (linear) hipLaunchKernelGGL((gated_step_kernel<T, true>), grid, block, 0, s, g, gate_pitch, x, u_pitch, h_prev, is_first, n, (int)D, h, static_cast<T *>(y));
        else hipLaunchKernelGGL((gated_step_kernel<T, false>), grid, block, 0, s, g, gate_pitch, x, u_pitch, h_prev, is_first, n, (int)D, h, static_cast<T *>(y));
    });
    return hipGetLastError() == hipSuccess ? SSM_OK : SSM_ERR_HIP;
}

}  // extern "C"
