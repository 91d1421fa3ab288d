// Gated linear recurrence with episode resets (gfx950): h_t = [not first_t] f_t h_{t-1} + (1 - f_t) u_t with f = sigmoid(gate), or
// with given coefficients, over sequences; its gradient pass; one step.
//
// A thread owns eight consecutive steps of two neighbouring channels.  The recurrence over consecutive steps is the map h -> A h + S with A the product of
// the decays, and a reset among the steps makes it the constant S: maps compose as (A, S, r) after (A', S', r') = (A A', r ? S : A S' + S,
// r or r').  The flag stands beside A because a product of zero would let an infinite or NaN state through a reset.
// The gradient runs the same maps backwards: what flows from step t to t-1 is b_t = c_t (dh_t + b_{t+1}) with c_t = [not first_t] f_t, so steps t0..t1 map b
// to A b + G with the same A and r.
//
// A large call is bound by memory: three arrays forward, five back (gate and u again: the states are formed anew from fp32 ones kept every 128 steps, which costs less than reading
// rounded ones and 1/64 of an array of them).  128 x 256 x 1024 bf16 38.6 and 76.5 us, 5.2 and 4.4 TB/s, where a copy reaches 5.0.  A small one is bound by the chain of one workgroup: loads,
// the maps of its threads through lanes and LDS, stores (16 x 256 x 512 f32 6.0 and 10.5 us).  So a sequence is spread over as many threads as it fills, and all
// its loads are in flight before the first is used.
#include "elem.h"
#include "lookback.h"
#include "ssm_internal.h"

#include <type_traits>

namespace ssm {
namespace {

inline bool misaligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }

constexpr int GE = 8;                        // consecutive steps of a thread
constexpr int GV = 2;                        // neighbouring channels of a thread
constexpr int GATED_MAX_THREADS = 1024, GATED_MAX_VECS = 32, GATED_CUS = 256;
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
    unsigned long long *desc;                // [nTB][chains][5][64] tagged words, zero on entry
    uint32_t *ticket, *err;
    int groups;                              // of a block
    uint32_t spin_limit;
    int chains, per_xcd;                     // chains: channel blocks of sequences (of groups of sequences); of them in an XCD, 0: in turn
    int round; FastDiv by_round;             // workgroups per chunk of all chains
};
constexpr int GATED_DESC_WORDS = 5 * 64;

// sigmoid(z) and 1 - sigmoid(z), both to the relative precision of the exponential: the difference where it is at least a half, exp(-z) sigmoid(z) else.
struct Gate { float f, i; };
__device__ __forceinline__ Gate gate_of(float z)
{
    const float e = __builtin_amdgcn_exp2f(z * -1.44269504f), f = __builtin_amdgcn_rcpf(1.f + e);
    return {f, e > 1.f ? 1.f - f : e * f};
}

__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) { return f32x2{fmaf(a[0], b[0], c[0]), fmaf(a[1], b[1], c[1])}; }
__device__ __forceinline__ f32x2 pick2(bool c, f32x2 a, f32x2 b) { return f32x2{c ? a[0] : b[0], c ? a[1] : b[1]}; }

// a map over consecutive steps: v -> A v + S, or the constant S where r.  R: whether a reset can be among the steps at all.  LIN: whether A is a product of given coefficients, which may
// be infinite where every state is finite: what is zero passes such a product as zero (a sequence that starts with padding).  A step's own coefficient is no product, and
// is multiplied as it is.
struct Map { f32x2 A, S; int r; };
template <bool LIN> __device__ __forceinline__ f32x2 through(f32x2 A, f32x2 v, f32x2 S)
{
    const f32x2 w = fma2(A, v, S);
    return LIN ? f32x2{v[0] == 0.f ? S[0] : w[0], v[1] == 0.f ? S[1] : w[1]} : w;
}
__device__ __forceinline__ Map identity() { return {f32x2{1.f, 1.f}, f32x2{0.f, 0.f}, 0}; }
template <bool R, bool LIN> __device__ __forceinline__ Map after(const Map &y, const Map &x)      // x first, then y
{
    const f32x2 s = through<LIN>(y.A, x.S, y.S);
    return {y.A * x.A, R ? pick2(y.r, y.S, s) : s, R ? y.r | x.r : 0};
}
template <bool LIN> __device__ __forceinline__ f32x2 apply(const Map &m, f32x2 v) { return pick2(m.r, m.S, through<LIN>(m.A, v, m.S)); }
template <bool R> __device__ __forceinline__ Map pick(bool c, const Map &a, const Map &b) { return {pick2(c, a.A, b.A), pick2(c, a.S, b.S), R ? (c ? a.r : b.r) : 0}; }
template <bool UP, bool R> __device__ __forceinline__ Map neighbour(const Map &m, int d)
{
    const auto of = [&](float v) { return UP ? __shfl_up(v, d) : __shfl_down(v, d); };
    return {f32x2{of(m.A[0]), of(m.A[1])}, f32x2{of(m.S[0]), of(m.S[1])}, R ? (UP ? __shfl_up(m.r, d) : __shfl_down(m.r, d)) : 0};
}

// Composition over the threads along time of a chunk: within a wavefront between lanes, over wavefronts in LDS (a map per wavefront and vector of channels; the
// flag is the same for all channels of a sequence).  `lost`: a wait of the workgroup gave up.
struct MapLds { f32x4 m[GATED_MAX_THREADS / 64][GATED_MAX_VECS]; int r[GATED_MAX_THREADS / 64]; int lost; };
template <bool UP, bool R, bool LIN> __device__ __forceinline__ Map inclusive_in_wave(Map m, int lane, int cx, int span)
{
    const int l = lane & (span - 1);
    for (int d = cx; d < span; d <<= 1) m = pick<R>(UP ? l >= d : l + d < span, after<R, LIN>(m, neighbour<UP, R>(m, d)), m);
    return m;
}
template <bool UP, bool R> __device__ __forceinline__ Map exclusive_in_wave(const Map &incl, int lane, int cx, int span)
{
    const int l = lane & (span - 1);
    return pick<R>(UP ? l >= cx : l + cx < span, neighbour<UP, R>(incl, cx), identity());
}
__device__ __forceinline__ void put(MapLds &s, int w, int c, const Map &m)
{
    s.m[w][c] = f32x4{m.A[0], m.A[1], m.S[0], m.S[1]};
    if (c == 0) s.r[w] = m.r;
}
__device__ __forceinline__ Map get(const MapLds &s, int w, int c)
{
    const f32x4 q = s.m[w][c];
    return {f32x2{q[0], q[1]}, f32x2{q[2], q[3]}, s.r[w]};
}
// the maps of wavefronts 0 .. n-1 (UP) or waves-1 .. waves-n, the first one first.  (Four are read at a time: one by one, every step would wait for LDS.)
template <bool UP, bool LIN> __device__ __forceinline__ Map fold(const MapLds &s, int c, int n, int waves)
{
    Map w = identity();
    for (int k0 = 0; k0 < n; k0 += 4) {
        Map q[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) { const int i = min(k0 + k, n - 1); q[k] = get(s, UP ? i : waves - 1 - i, c); }
#pragma unroll
        for (int k = 0; k < 4; ++k) if (k0 + k < n) w = after<true, LIN>(q[k], w);
    }
    return w;
}

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
        wave = __builtin_amdgcn_readfirstlane(tid >> 6);
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

// What a chunk's neighbours hand over where every chunk has a workgroup of its own.  With R threads along time to a workgroup, R chunks are a group and `groups` groups a
// block.  A workgroup publishes the map of its chunk before it waits for anything; then each of its rows fetches the map of one earlier chunk of
// its group, all at once.  With several groups to a block the last workgroup of a group publishes the map of the group, and each row fetches that of one earlier group of the
// block; one row fetches the state behind the block before.  R groups to a block, and the state reaches every chunk in two trips up to R^2 chunks (256: 32768
// steps); one, and it goes from group to group.  That costs less for two groups, and where the grid takes several rounds and the groups before have long ended:
// forward and gradient of 8 x 8192 x 512 f32 101 and 144 us, with R groups 105 and 149; of 1 x 16384 x 1024 bf16 42.7 and 48.7, 45.0 and 51.5; of 1 x 16384 x 256 f32 22.9 and 25.8,
// 20.0 and 24.5; of 1 x 60000 x 64 41.5 and 42.4, 25.0 and 27.4.
// The order of the compositions is fixed, whatever the timing: results are repeatable.  Chunks are numbered by a ticket per chain (the chunks of one
// sequence and channel block), so that a workgroup waits for such as have started; a wait that gives up hands on NaN and says so in the workspace.
__device__ __forceinline__ bool wait_words(const unsigned long long *w, unsigned limit, f32x2 &v, unsigned &tag)
{
    for (unsigned spins = 0;; ++spins) {
        const unsigned long long a = poll_word(w), b = poll_word(w + 1);
        v = f32x2{word_value(a), word_value(b)};
        tag = word_tag(a);
        if (tag != 0 && word_tag(b) != 0) return true;
        if (spins >= limit) return false;
        __builtin_amdgcn_s_sleep(2);
    }
}
__device__ __forceinline__ void publish2(unsigned long long *w, f32x2 v, unsigned tag)
{
    publish_word(w, v[0], tag);
    publish_word(w + 1, v[1], tag);
}
__device__ __forceinline__ void give_up(const GatedArgs &a, MapLds &lds)
{
    atomicOr(a.err, 1u);
    lds.lost = 1;
}
// the map at w
__device__ __forceinline__ Map wait_map(const GatedArgs &a, MapLds &lds, const unsigned long long *w)
{
    Map m;
    unsigned tag;
    if (!(wait_words(w, a.spin_limit, m.A, tag) && wait_words(w + 64, a.spin_limit, m.S, tag))) give_up(a, lds);
    m.r = tag == 2;
    return m;
}
__device__ __forceinline__ void publish_map(unsigned long long *w, const Map &m)
{
    publish2(w, m.A, 1);
    publish2(w + 64, m.S, m.r ? 2 : 1);
}
// one map per row and vector of channels -> their composition, the first row's first
template <bool UP, bool LIN> __device__ __forceinline__ Map compose_rows(const Place &p, MapLds &lds, Map m, int cx)
{
    m = inclusive_in_wave<UP, true, LIN>(m, p.lane, cx, p.span);
    __syncthreads();                         // (what was in lds has been read)
    if (UP ? p.lane >= 64 - cx : p.lane < cx) put(lds, p.wave, p.vec, m);
    __syncthreads();
    return fold<UP, LIN>(lds, p.vec, p.waves, p.waves);
}
// m, or the map to NaN where a wait of the workgroup gave up: what it got may be anything, its flag among it, and threads of one row may differ
__device__ __forceinline__ Map or_nan(const MapLds &lds, const Map &m)
{
    const f32x2 nan = {__builtin_nanf(""), __builtin_nanf("")};
    return lds.lost ? Map{nan, nan, 1} : m;
}
// UP: rows in the order of time.  `chunk`: number along the direction of the scan; `total`: the chunk's map, valid where `ends`; v0: what flows into the first chunk.
// Words of a chunk: its map [0, 128), the state behind the block that it ends [128, 192), the map of the group that it ends [192, 320).
template <bool UP, bool LIN> __device__ __forceinline__ f32x2 look_back(const GatedArgs &a, const Place &p, MapLds &lds, f32x2 *s_base, int chunk, int chain, const Map &total, bool ends, f32x2 v0)
{
    const int cx = 1 << a.lgcx, R = a.rows, RB = R * a.groups, group = chunk / R * R, block = chunk / RB * RB, row = UP ? p.row : R - 1 - p.row;
    unsigned long long *mine = a.desc + ((int64_t)chunk * a.chains + chain) * GATED_DESC_WORDS + p.vec * GV;
    const int64_t back = (int64_t)a.chains * GATED_DESC_WORDS;
    const bool more = chunk + 1 < a.nTB;
    if (ends && more) publish_map(mine, total);
    Map chunks = identity(), groups = identity();
    if (chunk > group) chunks = compose_rows<UP, LIN>(p, lds, group + row < chunk ? wait_map(a, lds, mine - (chunk - group - row) * back) : identity(), cx);
    if (ends && more && a.groups > 1 && (chunk + 1) % R == 0) publish_map(mine + 192, after<true, LIN>(total, or_nan(lds, chunks)));
    if (block > 0 && row == 0) {
        unsigned tag;
        f32x2 base;
        if (!wait_words(mine - (chunk - block + 1) * back + 128, a.spin_limit, base, tag)) give_up(a, lds);
        s_base[p.vec] = base;
    }
    if (group > block) groups = compose_rows<UP, LIN>(p, lds, block + row * R < group ? wait_map(a, lds, mine - (chunk - block - row * R - R + 1) * back + 192) : identity(), cx);
    else if (block > 0) __syncthreads();
    const f32x2 v = apply<LIN>(or_nan(lds, chunks), apply<LIN>(groups, block > 0 ? s_base[p.vec] : v0));
    if (ends && more && (chunk + 1) % RB == 0) publish2(mine + 128, apply<LIN>(total, v), 3);
    return v;
}
// Workgroups go to the eight XCDs in turn.  Neighbouring channel blocks share cache lines where rows are not whole lines (or a block is not), so
// neighbouring chains go to one XCD, whose L2 puts the pieces of a line together (64 x 1000 x 300 f32 forward 58 -> 47 us, bf16 gradient 68 -> 55; where rows are whole
// lines no difference).  Not with fewer than 64 chains, which would leave XCDs idle.  The chain of workgroup n of a round, or one past the last.
__device__ __forceinline__ int chain_of(const GatedArgs &a, int n) { return a.per_xcd ? (n & 7) * a.per_xcd + (n >> 3) : n; }
// the chunk of this workgroup, of those of its chain in the order in which they start
__device__ __forceinline__ int take_ticket(const GatedArgs &a, MapLds &lds, int chain)
{
    __shared__ int s_chunk;
    if (threadIdx.x == 0) {
        s_chunk = (int)atomicAdd(a.ticket + (int64_t)chain * SCAN_TICKET_STRIDE, 1u);
        lds.lost = 0;
    }
    __syncthreads();
    return __builtin_amdgcn_readfirstlane(s_chunk);
}

// NARROW: a single channel, held twice.
template <class T, bool NARROW> __device__ __forceinline__ typename Pack<T, 2>::type load_channels(const T *p)
{
    if constexpr (!NARROW) return load_pack<T, 2>(p);
    else return typename Pack<T, 2>::type{p[0], p[0]};
}
template <class T, bool NARROW> __device__ __forceinline__ void store_channels(T *p, f32x2 v)
{
    const typename Pack<T, 2>::type q = __builtin_convertvector(v, typename Pack<T, 2>::type);
    if constexpr (!NARROW) store_pack<T, 2>(p, q);
    else p[0] = q[0];
}
template <class T> __device__ __forceinline__ const T *first_step(const void *base, const ssm_strides &st, const Place &p, int t)
{
    return static_cast<const T *>(base) + (int64_t)p.seq * st.seq + (int64_t)t * st.step + p.ch;
}
// (steps past the end repeat the last one)
template <class T, bool NARROW> __device__ __forceinline__ void load_steps(typename Pack<T, 2>::type (&v)[GE], const void *base, const ssm_strides &st, const Place &p, int t0, int L, bool full)
{
    const T *q = first_step<T>(base, st, p, min(t0, L - 1));
    if (full) {                              // (uniform)
#pragma unroll
        for (int e = 0; e < GE; ++e) v[e] = load_channels<T, NARROW>(q + e * st.step);
    } else {
#pragma unroll
        for (int e = 0; e < GE; ++e) {
            v[e] = load_channels<T, NARROW>(q);
            q += t0 + e + 1 < L ? st.step : 0;
        }
    }
}
template <class T, bool NARROW> __device__ __forceinline__ void store_steps(const f32x2 (&v)[GE], void *base, const ssm_strides &st, const Place &p, int t0, int L, bool full)
{
    T *q = const_cast<T *>(first_step<T>(base, st, p, t0));
    if (!p.stored) return;
    if (full) {
#pragma unroll
        for (int e = 0; e < GE; ++e) store_channels<T, NARROW>(q + e * st.step, v[e]);
    } else {
#pragma unroll
        for (int e = 0; e < GE; ++e) if (t0 + e < L) store_channels<T, NARROW>(q + e * st.step, v[e]);
    }
}

// flags of a thread's steps, bit e = the state that flows into step t0 + e is dropped
__device__ __forceinline__ unsigned reset_mask(const GatedArgs &a, const Place &p, int t0, bool full)
{
    if (!a.is_first) return 0;
    const uint8_t *q = a.is_first + (int64_t)p.seq * a.L;
    unsigned m = 0;
    if (full) {
        typedef unsigned long long loose __attribute__((aligned(1)));
        const unsigned long long w = *reinterpret_cast<const loose *>(q + t0);
        if (w == 0) return 0;
#pragma unroll
        for (int e = 0; e < GE; ++e) m |= (unsigned)(((w >> (8 * e)) & 255u) != 0) << e;
        return m;
    }
#pragma unroll
    for (int e = 0; e < GE; ++e) m |= (unsigned)(q[min(t0 + e, a.L - 1)] != 0) << e;
    const int left = a.L - t0;
    return left < GE ? m & ((1u << max(left, 0)) - 1u) : m;
}

template <class T, bool LINEAR> __device__ __forceinline__ void gates(const typename Pack<T, 2>::type (&z)[GE], f32x2 (&f)[GE], f32x2 (&i)[GE])
{
#pragma unroll
    for (int e = 0; e < GE; ++e) {
        const f32x2 ze = __builtin_convertvector(z[e], f32x2);
        if constexpr (LINEAR) {
            f[e] = ze;
        } else {
            const Gate a = gate_of(ze[0]), b = gate_of(ze[1]);
            f[e] = f32x2{a.f, b.f};
            i[e] = f32x2{a.i, b.i};
        }
    }
}
template <class F> __device__ __forceinline__ void if_resets(bool plain, F f)
{
    if (plain) f(std::false_type{}); else f(std::true_type{});
}

template <class T, bool LINEAR, bool NARROW, bool LOOK>
__global__ void __launch_bounds__(GATED_MAX_THREADS) gated_fwd_kernel(GatedArgs a)
{
    __shared__ MapLds lds;
    __shared__ f32x2 s_end[GATED_MAX_VECS];  // state at the end of the chunk before
    const int chain = chain_of(a, LOOK ? (int)(blockIdx.x - a.by_round(blockIdx.x) * (unsigned)a.round) : (int)blockIdx.x);
    if (chain >= a.chains) return;
    int first = 0;
    if constexpr (LOOK) first = take_ticket(a, lds, chain);
    const Place p(a, chain);
    const int cx = 1 << a.lgcx, steps = GE * a.rows;
    const int64_t state = (int64_t)p.seq * a.D + p.ch;
    f32x2 in = {0.f, 0.f};                   // state that flows into the chunk
    if (a.h0) in = load_channels<float, NARROW>(a.h0 + state);
    for (int tb = first; tb < (LOOK ? first + 1 : a.nTB); ++tb) {
        const int t0 = tb * steps + p.row * GE;
        const bool full = (tb + 1) * steps <= a.L;
        typename Pack<T, 2>::type z[GE], u[GE];
        load_steps<T, NARROW>(z, a.gate, a.gs, p, t0, a.L, full);
        load_steps<T, NARROW>(u, a.u, a.us, p, t0, a.L, full);
        const unsigned cut = reset_mask(a, p, t0, full);
        const bool plain = __builtin_amdgcn_ballot_w64(cut != 0) == 0;
        f32x2 f[GE], b[GE];
        gates<T, LINEAR>(z, f, b);
#pragma unroll
        for (int e = 0; e < GE; ++e) {
            const f32x2 ue = __builtin_convertvector(u[e], f32x2);
            b[e] = LINEAR ? ue : b[e] * ue;
        }
        Map m, before;
        if_resets(plain, [&](auto r) {
            constexpr bool R = decltype(r)::value;
            m = identity();
#pragma unroll
            for (int e = 0; e < GE; ++e) m = after<R, false>(Map{f[e], b[e], (int)((cut >> e) & 1u)}, m);
            m = inclusive_in_wave<true, R, LINEAR>(m, p.lane, cx, p.span);
            before = exclusive_in_wave<true, R>(m, p.lane, cx, p.span);
        });
        if (p.waves > 1) {                   // (uniform)
            if (p.lane >= 64 - cx) put(lds, p.wave, p.vec, m);
            __syncthreads();
            const Map w = fold<true, LINEAR>(lds, p.vec, p.wave, p.waves);
            if constexpr (LOOK) m = after<true, LINEAR>(m, w);
            before = after<true, LINEAR>(before, w);
        }
        if constexpr (LOOK) in = look_back<true, LINEAR>(a, p, lds, s_end, tb, chain, m, p.row == a.rows - 1, in);
        f32x2 h = apply<LINEAR>(before, in);
        if (a.carry && p.stored && t0 > 0 && t0 < a.L && t0 % SSM_GATED_CARRY_STEPS == 0)
            store_channels<float, NARROW>(a.carry + ((int64_t)p.seq * a.carry_rows + t0 / SSM_GATED_CARRY_STEPS - 1) * a.D + p.ch, h);
        if_resets(plain, [&](auto r) {
            constexpr bool R = decltype(r)::value;
#pragma unroll
            for (int e = 0; e < GE; ++e) {
                h = R ? pick2((cut >> e) & 1u, b[e], fma2(f[e], h, b[e])) : fma2(f[e], h, b[e]);
                b[e] = h;
            }
        });
        store_steps<T, NARROW>(b, a.h, a.hs, p, t0, a.L, full);
        if (a.h_last && p.stored && t0 < a.L && a.L - t0 <= GE) {
            f32x2 last = b[0];
#pragma unroll
            for (int e = 1; e < GE; ++e) last = pick2(t0 + e < a.L, b[e], last);
            store_channels<float, NARROW>(a.h_last + state, last);
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
    __shared__ f32x2 s_end[GATED_MAX_VECS];
    const int chain = chain_of(a, LOOK ? (int)(blockIdx.x - a.by_round(blockIdx.x) * (unsigned)a.round) : (int)blockIdx.x);
    if (chain >= a.chains) return;
    int first = a.nTB - 1;
    if constexpr (LOOK) first = a.nTB - 1 - take_ticket(a, lds_down, chain);
    Place p(a, chain);
    const int cx = 1 << a.lgcx, steps = GE * a.rows;
    const f32x2 zero = {0.f, 0.f};
    f32x2 from_right = zero;
    if (a.dh_last) from_right = load_channels<float, NARROW>(a.dh_last + (int64_t)p.seq * a.D + p.ch);
    for (int tb = first; tb >= (LOOK ? first : 0); --tb) {
        asm volatile("" : "+v"(p.seq), "+v"(p.ch));          // (addresses are formed where they are used, not kept from one chunk to the next)
        const int64_t state = (int64_t)p.seq * a.D + p.ch;
        const int t0 = tb * steps + p.row * GE;
        const bool full = (tb + 1) * steps <= a.L;
        f32x2 f[GE], i[GE], u[GE], d[GE];
        {
            typename Pack<T, 2>::type rz[GE], ru[GE], rd[GE];
            load_steps<T, NARROW>(rz, a.gate, a.gs, p, t0, a.L, full);
            load_steps<T, NARROW>(ru, a.u, a.us, p, t0, a.L, full);
            load_steps<T, NARROW>(rd, a.dh, a.dhs, p, t0, a.L, full);
            gates<T, LINEAR>(rz, f, i);
#pragma unroll
            for (int e = 0; e < GE; ++e) { u[e] = __builtin_convertvector(ru[e], f32x2); d[e] = __builtin_convertvector(rd[e], f32x2); }
        }
        const unsigned cut = reset_mask(a, p, t0, full);
        const bool plain = __builtin_amdgcn_ballot_w64(cut != 0) == 0;
        f32x2 in = zero;
        if (tb > 0) in = load_channels<float, NARROW>(a.carry_in + ((int64_t)p.seq * a.carry_rows + tb * steps / SSM_GATED_CARRY_STEPS - 1) * a.D + p.ch);
        else if (a.h0) in = load_channels<float, NARROW>(a.h0 + state);
        if (!full) {                         // steps past the end let what flows backwards through: decay 1, no term of their own
#pragma unroll
            for (int e = 0; e < GE; ++e) {
                const bool past = t0 + e >= a.L;
                f[e] = pick2(past, f32x2{1.f, 1.f}, f[e]);
                d[e] = pick2(past, zero, d[e]);
            }
        }
        // (pinned: the compiler otherwise keeps products of these beside them, 20 registers more, one wavefront of a SIMD fewer)
#pragma unroll
        for (int e = 0; e < GE; ++e) {
            asm volatile("" : "+v"(f[e]), "+v"(u[e]), "+v"(d[e]));
            if constexpr (!LINEAR) asm volatile("" : "+v"(i[e]));
        }
        Map up, down, before, behind;
        if_resets(plain, [&](auto r) {
            constexpr bool R = decltype(r)::value;
            up = identity();
#pragma unroll
            for (int e = 0; e < GE; ++e) up = after<R, false>(Map{f[e], LINEAR ? u[e] : i[e] * u[e], (int)((cut >> e) & 1u)}, up);
            down = {up.A, zero, up.r};
#pragma unroll
            for (int e = GE - 1; e >= 0; --e) {
                const f32x2 back = f[e] * (d[e] + down.S);
                down.S = R ? pick2((cut >> e) & 1u, zero, back) : back;
            }
            up = inclusive_in_wave<true, R, LINEAR>(up, p.lane, cx, p.span);
            before = exclusive_in_wave<true, R>(up, p.lane, cx, p.span);
            down = inclusive_in_wave<false, R, LINEAR>(down, p.lane, cx, p.span);
            behind = exclusive_in_wave<false, R>(down, p.lane, cx, p.span);
        });
        if (p.waves > 1) {
            if (p.lane >= 64 - cx) put(lds_up, p.wave, p.vec, up);
            if (p.lane < cx) put(lds_down, p.wave, p.vec, down);
            __syncthreads();
            before = after<true, LINEAR>(before, fold<true, LINEAR>(lds_up, p.vec, p.wave, p.waves));
            const Map w = fold<false, LINEAR>(lds_down, p.vec, p.waves - 1 - p.wave, p.waves);
            if constexpr (LOOK) down = after<true, LINEAR>(down, w);
            behind = after<true, LINEAR>(behind, w);
        }
        if constexpr (LOOK) from_right = look_back<false, LINEAR>(a, p, lds_down, s_end, a.nTB - 1 - tb, chain, down, p.row == 0, from_right);
        f32x2 back = apply<LINEAR>(behind, from_right), h = apply<LINEAR>(before, in);
        if_resets(plain, [&](auto r) {
            constexpr bool R = decltype(r)::value;
            // chi, last step first (in place of dh)
#pragma unroll
            for (int e = GE - 1; e >= 0; --e) {
                d[e] += back;
                back = R ? pick2((cut >> e) & 1u, zero, f[e] * d[e]) : f[e] * d[e];
            }
            // the states again, first step first, and the gradients (du in place of chi, dgate in place of u)
#pragma unroll
            for (int e = 0; e < GE; ++e) {
                const f32x2 prev = R ? pick2((cut >> e) & 1u, zero, h) : h;
                if constexpr (LINEAR) {
                    h = fma2(f[e], prev, u[e]);
                    u[e] = prev * d[e];
                } else {
                    // (with the complement of f as it is, like the forward pass: u + f (prev - u) would round the state by u's last place, and a gate near one
                    // hands on little of a large u.  u is pinned: its product would be kept from the maps above, in registers that are not there)
                    asm volatile("" : "+v"(u[e]));
                    const f32x2 w = prev - u[e];
                    h = fma2(f[e], prev, i[e] * u[e]);
                    d[e] *= i[e];
                    u[e] = f[e] * w * d[e];
                }
            }
        });
        store_steps<T, NARROW>(d, a.du, a.dus, p, t0, a.L, full);
        store_steps<T, NARROW>(u, a.dgate, a.dgs, p, t0, a.L, full);
        if (t0 == 0 && a.dh0 && p.stored) store_channels<float, NARROW>(a.dh0 + state, back);
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
//   A sequence whose channels fit a wavefront with all its steps shares it with others.
//   More than 256 chains of 64 channels: workgroups of 512 threads that walk the chunks of a chain.  Nothing is handed over, and whole cache lines are read at once.  (A workgroup
//   per chunk: 64 x 2048 x 512 bf16 forward and gradient pass 94 and 167 us, 122 and 171; 1024 threads: 106 and 165; 100 x 300 x 300 f32 22 and 38, 29 and 41, 31 and 46.)
//   256 and fewer: a workgroup of up to 1024 threads for each, the chains narrower (32, 16, 8 channels) where that gives a CU fewer threads' work; of equal ones the widest.
//   With 64 channels (32 from 256 steps on) and narrower, us: 4 x 512 x 256 f32 6.6 and 9.8, 4.9 and 7.1 (8); 12 x 400 x 192 bf16 6.5 and 9.6, 5.5 and 7.6 (16); 1 x 100 x 64 f32
//   4.9 and 6.5, 3.9 and 5.3 (8).  Of 4 channels: 5.5 and 8.1, 7.3 and 10.8, 4.0 and 5.4.
//   That beats a workgroup per chunk, which costs a second launch and the hand-over, as long as a CU's share is short, or all CUs have one of whole cache lines.  Per chunk and
//   so (channels, share in workgroups of 1024): 16 x 1024 x 256 f32 15.2 and 21.2, 11.7 and 18.7 (16, 1); 10 x 900 x 400 bf16 15.7 and 19.9, 8.6 and 14.4 (16, 0.9);
//   16 x 1500 x 400 f16 26.2 and 32.8, 19.2 and 30.8 (32, 2.9); 64 x 3000 x 64 bf16 29.3 and 36.7, 23.1 and 36.6 (16, 2.9); 30 x 1024 x 512 bf16 32 and 41, 24 and 39 (64, 4, 240 chains);
//   28 x 4096 x 512 bf16 113 and 161, 98 and 158 (64, 16, 224 chains); 16 x 4096 x 512 bf16 59 and 95, 48 and 103 (32, 8); 32 x 4096 x 512 bf16 127 and 173, 101 and 164 (64, 16; 512 threads: 120 and 183).
//   The other way round: 4 x 4096 x 256 bf16 14.3 and 17.4, 15.7 and 27.6 (8, 2, 128 chains); 16 x 3000 x 300 f32 41 and 68, 42 and 89 (32, 5.9, 160 chains);
//   20 x 4096 x 512 bf16 73 and 125, 72 and 151 (64, 16, 160 chains); 8 x 8192 x 512 f32 95 and 146, 110 and 182 (16, 8).
struct GatedPlan { int lgcx, lgspan, rows, seqs, threads, nCX, nTB; bool look; int per_xcd; int64_t chains, round, blocks; size_t ticket_bytes, desc_bytes; };
GatedPlan plan_gated(int64_t Bt, int64_t L, int64_t D)
{
    GatedPlan pl{};
    const int64_t vecs = (D + GV - 1) / GV, rows = (L + GE - 1) / GE;
    while (pl.lgcx < 5 && (1 << pl.lgcx) < vecs) ++pl.lgcx;
    int most = 512 >> pl.lgcx;               // threads along time
    const auto chains_at = [&](int lg) { return Bt * ((vecs + (1 << lg) - 1) >> lg); };
    bool few = chains_at(pl.lgcx) < GATED_CUS;
    if (chains_at(pl.lgcx) <= GATED_CUS && rows << pl.lgcx > 64) {
        const int widest = pl.lgcx, narrowest = pl.lgcx < 2 ? pl.lgcx : 2;
        const auto share = [&](int lg) { return (chains_at(lg) + GATED_CUS - 1) / GATED_CUS * (rows << lg); };     // threads' work of a CU
        int best = widest;
        for (int lg = widest - 1; lg >= narrowest && chains_at(lg + 1) < GATED_CUS; --lg) if (share(lg) < share(best)) best = lg;
        if (share(best) <= GATED_MAX_THREADS || (share(best) <= 3 * GATED_MAX_THREADS && chains_at(best) >= GATED_CUS * 5 / 8) ||
            (best >= 4 && chains_at(best) >= GATED_CUS * 7 / 8)) {
            pl.lgcx = best;
            most = GATED_MAX_THREADS >> best;
            few = false;
        }
    }
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
        const int per_wave = 64 >> pl.lgcx;
        pl.lgspan = 6;
        pl.rows = (int)(rows <= most ? (rows + per_wave - 1) / per_wave * per_wave : most);
        pl.threads = pl.rows * cx;
        pl.seqs = 1;
        pl.nTB = (int)((rows + pl.rows - 1) / pl.rows);
    }
    pl.nCX = (int)((vecs + cx - 1) >> pl.lgcx);
    pl.chains = (int64_t)pl.nCX * ((Bt + pl.seqs - 1) / pl.seqs);
    pl.look = pl.nTB > 1 && few;
    pl.per_xcd = pl.chains >= 64 ? (int)((pl.chains + 7) / 8) : 0;
    pl.round = pl.per_xcd ? 8 * (int64_t)pl.per_xcd : pl.chains;
    pl.blocks = pl.round * (pl.look ? pl.nTB : 1);
    if (pl.look) {
        pl.ticket_bytes = (size_t)pl.chains * SCAN_TICKET_STRIDE * sizeof(uint32_t);
        pl.desc_bytes = (size_t)pl.chains * pl.nTB * GATED_DESC_WORDS * sizeof(unsigned long long);
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
    if (L > SSM_MAX_TOKENS - GE * GATED_MAX_THREADS) return SSM_ERR_UNSUPPORTED;          // (the last chunk's end is an int too)
    return SSM_OK;
}

ssm_status launch_gated(GatedArgs &a, bool reverse, int dtype, int linear, void *workspace, size_t ws_bytes, hipStream_t s)
{
    const GatedPlan pl = plan_gated(a.Bt, a.L, a.D);
    if (!fits_a_grid(pl.blocks, pl.threads)) return SSM_ERR_UNSUPPORTED;
    a.lgcx = pl.lgcx; a.lgspan = pl.lgspan; a.rows = pl.rows; a.seqs = pl.seqs; a.nCX = pl.nCX; a.nTB = pl.nTB;
    a.carry_rows = (int)ssm_gated_carry_rows(a.L);
    a.chains = (int)pl.chains; a.per_xcd = pl.per_xcd; a.round = (int)pl.round;
    a.by_round = FastDiv::by((unsigned)a.round);
    if (pl.look) {
        const size_t scratch = pl.ticket_bytes + pl.desc_bytes;
        if (!workspace || misaligned(workspace, 256) || ws_bytes < GATED_HEADER + scratch) return SSM_ERR_WORKSPACE;
        char *ws = static_cast<char *>(workspace);
        a.err = reinterpret_cast<uint32_t *>(ws);
        a.ticket = reinterpret_cast<uint32_t *>(ws + GATED_HEADER);
        a.desc = reinterpret_cast<unsigned long long *>(ws + GATED_HEADER + pl.ticket_bytes);
        a.spin_limit = scan_spin_limit();
        a.groups = pl.blocks <= 1024 && pl.nTB > 2 * pl.rows ? pl.rows : 1;          // (up to about two rounds, three groups and more)
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
    const int64_t n = Bt * D, blocks = (n + 255) / 256;
    if (!fits_a_grid(blocks, 256)) return SSM_ERR_UNSUPPORTED;
    const dim3 grid((unsigned)blocks), block(256);
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
