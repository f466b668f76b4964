// The chains of the gated delta rule: the states from the first chunk to the last, and their gradients from the last to the first
// (delta_chunk.hip and delta_grad.hip have the formulas).  The value channels are independent: a workgroup takes 16 of one (sample,
// head).  Its first 4 waves carry the chain, each with D / 4 key channels of the state in accumulators; a chunk is
//   1. K S: every wave its own channels' share for all 64 tokens, straight from the accumulators, which are an operand as they stand
//      (the order of a contraction is free, so K's operand takes the channels in theirs); the shares meet in LDS
//   2. T R: 16 tokens a wave, R from LDS
//   3. S <- gamma S + K^T (tail u): u from LDS, K^T by transposing reads
// Its other 4 waves, one on each SIMD beside a wave of the chain, do what the chain does not wait for: they bring the next chunk's K,
// and forward compute O = scale gamma Q S + P u, backward Q^T (scale gamma dO), dv and the sums of dR v.
// Three exchanges through LDS and 36 products deep, the chain is bound by their latency, not by memory.  Operands of the next chunk are loaded a
// chunk ahead into a second set of registers, the barriers wait for LDS alone, and stores are never skipped by a branch, so that no
// wait for a load waits for a store.
#include <algorithm>

#include "causal.h"
#include "delta_planes.h"

namespace salad {

namespace {

constexpr int UP = 72;      // pitch of the exchanges' tiles: 64 tokens, 16 bytes aside

template <typename T, int D> struct ChainLds {
    static constexpr int P = planes_of<T>(), OP = D / 4 + (P == 1 ? 8 : 4), OWN = P * 64 * OP;     // a wave's channels of K or Q: [64 tokens][D / 4]
    static constexpr int KBUFS = P == 1 ? 2 : 1, QP = D + 8, QT = P * 16 * QP;                    // a wave's tokens of Q: [16 tokens][D]
    union {
        f32x4 ks[4][4][64];             // by wave: its share of K S, by row tile and lane
        f32x4 y[4][4][64];              // backward: Q^T (scale gamma dO) for the wave's channels, once the shares are read
    };
    union {
        struct { u16 q[4][QT]; u32x4 so[4][P][64]; } f;         // forward: Q, and the state as an operand
        struct { u16 q[4][OWN]; f32x4 dr[4][64]; } b;           // backward: Q, and dR
    };
    u16 k[KBUFS][4][OWN];
    u16 r[3 * 16 * UP], u[3 * 16 * UP], g[3 * 16 * UP];
};

// ROWS rows of W channels of a tensor (a wave's part) on their way to an LDS tile: a wave loads them, 16 bytes a lane, and puts them down later
template <typename T, int D, int ROWS, int W, int PITCH> struct Part {
    static constexpr int P = planes_of<T>(), PER = 16 / sizeof(T), LPR = W / PER, RPI = 64 / LPR, NL = ROWS / RPI;
    u32x4 r[NL];
    __device__ inline void load(const T *base, int r0, int last, int lane)      // rows r0.., none behind `last`
    {
#pragma unroll
        for (int i = 0; i < NL; ++i)
            r[i] = *reinterpret_cast<const u32x4 *>(base + (unsigned)(min(r0 + i * RPI + lane / LPR, last) * D + lane % LPR * PER));
    }
    __device__ inline void put(u16 *tile, int lane) const
    {
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            u16 *at = tile + (i * RPI + lane / LPR) * PITCH + lane % LPR * PER;
            if constexpr (P == 1) *reinterpret_cast<u32x4 *>(at) = r[i];
            else put4<3>(at, ROWS * PITCH, __builtin_bit_cast(f32x4, r[i]));
        }
    }
};

// operand from a tile's row, the channels in the order of the accumulators: lane group l4 has 4 l4.. of the first 16 channels from c0 on and
// 4 l4.. of the second (NT = 1: there is none; zeros)
template <int P, int NT>
__device__ inline Op<P> frag_own(const u16 *tile, int plane, int pitch, int row, int c0, int l4)
{
    Op<P> f;
#pragma unroll
    for (int p = 0; p < P; ++p) {
        const u16 *at = tile + p * plane + row * pitch + c0 + 4 * l4;
        const u32x2 x = *reinterpret_cast<const u32x2 *>(at), y = NT > 1 ? *reinterpret_cast<const u32x2 *>(at + 16) : u32x2{0, 0};
        f.p[p] = __builtin_bit_cast(bf16x8, u32x4{x.x, x.y, y.x, y.y});
    }
    return f;
}

// 4 tokens of a value channel, loaded as they are and converted later
template <typename T> struct Four {
    T r[4];
    __device__ inline void load(const T *base, int stride, int t0, int last, int c)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) r[i] = base[(unsigned)(min(t0 + i, last) * stride + c)];
    }
    __device__ inline f32x4 get(int t0, int valid) const    // zeros behind the last token
    {
        f32x4 x;
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = t0 + i < valid ? load1(&r[i]) : 0.f;
        return x;
    }
};

template <int P>
__device__ inline Op<P> first_planes(const Op<3> &f)
{
    Op<P> o;
#pragma unroll
    for (int i = 0; i < P; ++i) o.p[i] = f.p[i];
    return o;
}

// the accumulators of the wave's channels as an operand
template <int NT>
__device__ inline Op<3> state_op(const f32x4 (&s)[NT])
{
    const f32x4 z = {0.f, 0.f, 0.f, 0.f};
    return op_of<3>(s[0], NT > 1 ? s[NT - 1] : z);
}

template <int P>
__device__ inline Op<P> packed_op(const u16 *from, int w, int kt, int lane)
{
    Op<P> f;
#pragma unroll
    for (int p = 0; p < P; ++p) f.p[p] = *reinterpret_cast<const bf16x8 *>(from + (((p * 4 + w) * 2 + kt) * 64 + lane) * 8);
    return f;
}

// where a workgroup and a lane of it work
template <typename T, int D> struct Place {
    int bh, slice, c0, len, chunks, lane, w, l16, l4, arow, i0;     // arow, i0: first of an accumulator's 4 key channels, 4 tokens
    const T *k, *q;                                                 // of the head
    __device__ Place(const DeltaArgs &a, int bh_, int slice_, int w_) : bh(bh_), slice(slice_), c0(slice_ * 16), w(w_)
    {
        const int b = bh / a.H, h = bh - b * a.H, hk = h / (a.H / a.Hk);
        len = delta_len(a, b);
        chunks = (len + 63) / 64;
        lane = threadIdx.x & 63;
        l16 = lane & 15;
        l4 = lane >> 4;
        arow = w * (D / 4) + 4 * l4;
        i0 = 16 * w + 4 * l4;
        k = reinterpret_cast<const T *>(a.k) + ((size_t)b * a.Hk + hk) * a.N * D;
        q = reinterpret_cast<const T *>(a.q) + ((size_t)b * a.Hk + hk) * a.N * D;
    }
    __device__ int last(int ch) const { return min(len - ch * 64, 64) - 1; }
    __device__ size_t at(const DeltaArgs &a, int ch) const { return (size_t)bh * a.chunks + ch; }
    __device__ size_t rows(const DeltaArgs &a, int ch) const { return ((size_t)bh * a.N + (size_t)ch * 64) * D; }
};

template <typename T, int D>
__device__ inline void load_state(const float *from, const Place<T, D> &p, f32x4 (&s)[D / 64])
{
#pragma unroll
    for (int x = 0; x < D / 64; ++x)
#pragma unroll
        for (int r = 0; r < 4; ++r) s[x][r] = from ? from[((size_t)p.bh * D + p.arow + 16 * x + r) * D + p.c0 + p.l16] : 0.f;
}
template <typename T, int D>
__device__ inline void store_state(float *to, const Place<T, D> &p, const f32x4 (&s)[D / 64])
{
    if (!to) return;
#pragma unroll
    for (int x = 0; x < D / 64; ++x)
#pragma unroll
        for (int r = 0; r < 4; ++r) to[((size_t)p.bh * D + p.arow + 16 * x + r) * D + p.c0 + p.l16] = s[x][r];
}

// Barriers of both roles: one before the first chunk (K of it is there), three in a chunk, and a fourth where K has one buffer only.

// ---- forward.  OUT: the layer's output; else what the gradients need (the states and u) ----------------------------
template <typename T, int D, bool OUT>
__device__ inline void forward_chain(const DeltaArgs &a, const Place<T, D> p, ChainLds<T, D> &lds)
{
    using L = ChainLds<T, D>;
    constexpr int P = L::P, NT = D / 64, UO = P == 1 ? 2 : 3;               // planes of u as a factor of O
    f32x4 s[NT];
    load_state(a.state_in, p, s);
    struct In {
        Op<3> t[2];
        Four<T> v;
        f32x4 gamma, tail, beta;
        float end;
    } in0, in1;
    auto fetch = [&](In &n, int ch) __attribute__((always_inline)) {
        const size_t at = p.at(a, ch);
        const DeltaGate &gate = a.gate[at];
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) n.t[kt] = packed_op<3>(a.tf + at * DELTA_T_ELEMS, p.w, kt, p.lane);
        n.v.load(reinterpret_cast<const T *>(a.v) + p.rows(a, ch), D, p.i0, p.last(ch), p.c0 + p.l16);
        n.gamma = load4(gate.gamma + p.i0);
        n.tail = load4(gate.tail + p.i0);
        n.beta = load4(gate.beta + p.i0);
        n.end = gate.gamma[63];
    };
    if (!p.chunks) { store_state(a.state_out, p, s); return; }
    Op<P> k[4];
    auto take_k = [&](int ch) __attribute__((always_inline)) {
#pragma unroll
        for (int rt = 0; rt < 4; ++rt) k[rt] = frag_own<P, NT>(lds.k[ch & (L::KBUFS - 1)][p.w], 64 * L::OP, L::OP, 16 * rt + p.l16, 0, p.l4);
    };
    fetch(in0, 0);
    lds_barrier();
    take_k(0);
    auto step = [&](const In &in, In &next, int ch) __attribute__((always_inline)) {
        const size_t at = p.at(a, ch);
        const u16 *K = lds.k[ch & (L::KBUFS - 1)][p.w];
        const Op<3> so = state_op(s);
#pragma unroll
        for (int rt = 0; rt < 4; ++rt) {
            f32x4 c = {0.f, 0.f, 0.f, 0.f};
            mma(c, k[rt], so);
            lds.ks[p.w][rt][p.lane] = c;
        }
        if (OUT)
#pragma unroll
            for (int i = 0; i < P; ++i) lds.f.so[p.w][i][p.lane] = __builtin_bit_cast(u32x4, so.p[i]);
        lds_barrier();
        f32x4 ks = lds.ks[0][p.w][p.lane], rr;
#pragma unroll
        for (int w = 1; w < 4; ++w) ks += lds.ks[w][p.w][p.lane];
        if (!OUT)
#pragma unroll
            for (int x = 0; x < NT; ++x) store4(a.s0 + (at * D + p.c0 + p.l16) * D + p.arow + 16 * x, s[x]);
        const f32x4 v = in.v.get(p.i0, p.last(ch) + 1);
#pragma unroll
        for (int r = 0; r < 4; ++r) rr[r] = in.beta[r] * (v[r] - in.gamma[r] * ks[r]);
        put4<3>(lds.r + p.l16 * UP + p.i0, 16 * UP, rr);
        lds_barrier();
        const Op<3> r0 = frag_n<3>(lds.r, 16 * UP, UP, 0, 0, p.lane), r1 = frag_n<3>(lds.r, 16 * UP, UP, 0, 32, p.lane);
        Op<P> kt[NT][2];
#pragma unroll
        for (int x = 0; x < NT; ++x) {
            kt[x][0] = frag_t<P>(K, 64 * L::OP, L::OP, 16 * x, 0, p.lane);
            kt[x][1] = frag_t<P>(K, 64 * L::OP, L::OP, 16 * x, 32, p.lane);
        }
        fetch(next, min(ch + 1, p.chunks - 1));
        f32x4 u = {0.f, 0.f, 0.f, 0.f};
        mma(u, in.t[0], r0);
        if (p.w >= 2) mma(u, in.t[1], r1);                              // T is lower triangular
        f32x4 ut;
#pragma unroll
        for (int r = 0; r < 4; ++r) ut[r] = u[r] * in.tail[r];
        put4<3>(lds.u + p.l16 * UP + p.i0, 16 * UP, ut);
        if (OUT) put4<UO>(lds.g + p.l16 * UP + p.i0, 16 * UP, u);
        else store4(a.u + (at * D + p.c0 + p.l16) * 64 + p.i0, u);
        lds_barrier();
        const Op<3> u0 = frag_n<3>(lds.u, 16 * UP, UP, 0, 0, p.lane), u1 = frag_n<3>(lds.u, 16 * UP, UP, 0, 32, p.lane);
        if (L::KBUFS > 1) take_k(ch + 1);
#pragma unroll
        for (int x = 0; x < NT; ++x) {
            s[x] *= in.end;
            mma(s[x], kt[x][0], u0);
            mma(s[x], kt[x][1], u1);
        }
        if (L::KBUFS == 1) { lds_barrier(); take_k(ch + 1); }
    };
    for (int ch = 0; ch < p.chunks; ch += 2) {
        step(in0, in1, ch);
        if (ch + 1 < p.chunks) step(in1, in0, ch + 1);
    }
    store_state(a.state_out, p, s);
}

template <typename T, int D, bool OUT>
__device__ inline void forward_helper(const DeltaArgs &a, const Place<T, D> p, ChainLds<T, D> &lds)
{
    using L = ChainLds<T, D>;
    constexpr int P = L::P, NT = D / 64, UO = P == 1 ? 2 : 3;
    if (!p.chunks) return;
    Part<T, D, 64, D / 4, L::OP> kn;
    Part<T, D, 16, D, L::QP> qn;
    struct In {
        Op<P> pf[2];
        f32x4 gamma;
    } in0, in1;
    u16 *Q = lds.f.q[p.w];
    auto fetch_rows = [&](int ch) __attribute__((always_inline)) {
        kn.load(p.k + (size_t)ch * 64 * D + p.w * (D / 4), 0, p.last(ch), p.lane);
        if (OUT) qn.load(p.q + (size_t)ch * 64 * D, 16 * p.w, p.last(ch), p.lane);
    };
    auto fetch = [&](In &n, int ch) __attribute__((always_inline)) {
        if (!OUT) return;
        const size_t at = p.at(a, ch);
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) n.pf[kt] = packed_op<P>(a.pf + at * (P * 4096), p.w, kt, p.lane);
        n.gamma = load4(a.gate[at].gamma + p.i0);
    };
    fetch_rows(0);
    fetch(in0, 0);
    kn.put(lds.k[0][p.w], p.lane);
    if (OUT) qn.put(Q, p.lane);
    lds_barrier();
    auto step = [&](const In &in, In &next, int ch) __attribute__((always_inline)) {
        fetch_rows(min(ch + 1, p.chunks - 1));
        fetch(next, min(ch + 1, p.chunks - 1));
        Op<P> q[4];
        if (OUT)
#pragma unroll
            for (int g = 0; g < 4; ++g) q[g] = frag_own<P, NT>(Q, 16 * L::QP, L::QP, p.l16, g * (D / 4), p.l4);
        lds_barrier();
        f32x4 o = {0.f, 0.f, 0.f, 0.f};
        if (OUT)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                Op<P> so;
#pragma unroll
                for (int i = 0; i < P; ++i) so.p[i] = __builtin_bit_cast(bf16x8, lds.f.so[g][i][p.lane]);
                mma(o, q[g], so);
            }
        lds_barrier();
        if (L::KBUFS > 1) kn.put(lds.k[(ch + 1) & 1][p.w], p.lane);
        lds_barrier();
        if (L::KBUFS == 1) { kn.put(lds.k[0][p.w], p.lane); lds_barrier(); }
        if (OUT) {
#pragma unroll
            for (int r = 0; r < 4; ++r) o[r] *= a.scale * in.gamma[r];
            mma(o, in.pf[0], frag_n<UO>(lds.g, 16 * UP, UP, 0, 0, p.lane));
            if (p.w >= 2) mma(o, in.pf[1], frag_n<UO>(lds.g, 16 * UP, UP, 0, 32, p.lane));       // P is lower triangular
            const auto rows = bounded(reinterpret_cast<T *>(a.out) + p.rows(a, ch), (p.last(ch) + 1) * D);
#pragma unroll
            for (int r = 0; r < 4; ++r) store_bounded(rows, T(), (p.i0 + r) * D + p.c0 + p.l16, o[r]);
            qn.put(Q, p.lane);
        }
    };
    for (int ch = 0; ch < p.chunks; ch += 2) {
        step(in0, in1, ch);
        if (ch + 1 < p.chunks) step(in1, in0, ch + 1);
    }
}

// ---- backward: the states' gradients; also dR, dv, and the sums of dR v that dbeta takes ---------------------------
template <typename T, int D>
__device__ inline void backward_chain(const DeltaArgs &a, const Place<T, D> p, ChainLds<T, D> &lds)
{
    using L = ChainLds<T, D>;
    constexpr int P = L::P, NT = D / 64;
    f32x4 s[NT];
    load_state(a.dstate_out, p, s);
    struct In {
        Op<3> t[2];
        f32x4 gamma, tail, beta, x;
        float end;
    } in0, in1;
    auto fetch = [&](In &n, int ch) __attribute__((always_inline)) {
        const size_t at = p.at(a, ch);
        const DeltaGate &gate = a.gate[at];
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) n.t[kt] = packed_op<3>(a.ttf + at * DELTA_T_ELEMS, p.w, kt, p.lane);
        n.x = load4(a.dr + (at * D + p.c0 + p.l16) * 64 + p.i0);
        n.gamma = load4(gate.gamma + p.i0);
        n.tail = load4(gate.tail + p.i0);
        n.beta = load4(gate.beta + p.i0);
        n.end = gate.gamma[63];
    };
    if (!p.chunks) { store_state(a.dstate_in, p, s); return; }
    Op<P> k[4];
    auto take_k = [&](int i) __attribute__((always_inline)) {
#pragma unroll
        for (int rt = 0; rt < 4; ++rt) k[rt] = frag_own<P, NT>(lds.k[i & (L::KBUFS - 1)][p.w], 64 * L::OP, L::OP, 16 * rt + p.l16, 0, p.l4);
    };
    fetch(in0, p.chunks - 1);
    lds_barrier();
    take_k(0);
    auto step = [&](const In &in, In &next, int i) __attribute__((always_inline)) {
        const int ch = p.chunks - 1 - i;
        const size_t at = p.at(a, ch);
        const u16 *K = lds.k[i & (L::KBUFS - 1)][p.w];
        const Op<3> so = state_op(s);
#pragma unroll
        for (int rt = 0; rt < 4; ++rt) {
            f32x4 c = {0.f, 0.f, 0.f, 0.f};
            mma(c, k[rt], so);
            lds.ks[p.w][rt][p.lane] = c;
        }
        lds_barrier();
        f32x4 du = lds.ks[0][p.w][p.lane];
#pragma unroll
        for (int w = 1; w < 4; ++w) du += lds.ks[w][p.w][p.lane];
#pragma unroll
        for (int x = 0; x < NT; ++x) store4(a.ds1 + (at * D + p.c0 + p.l16) * D + p.arow + 16 * x, s[x]);
#pragma unroll
        for (int r = 0; r < 4; ++r) du[r] = in.x[r] + in.tail[r] * du[r];
        put4<3>(lds.r + p.l16 * UP + p.i0, 16 * UP, du);
        lds_barrier();
        const Op<3> r0 = frag_n<3>(lds.r, 16 * UP, UP, 0, 0, p.lane), r1 = frag_n<3>(lds.r, 16 * UP, UP, 0, 32, p.lane);
        Op<P> kt[NT][2];
#pragma unroll
        for (int x = 0; x < NT; ++x) {
            kt[x][0] = frag_t<P>(K, 64 * L::OP, L::OP, 16 * x, 0, p.lane);
            kt[x][1] = frag_t<P>(K, 64 * L::OP, L::OP, 16 * x, 32, p.lane);
        }
        fetch(next, max(ch - 1, 0));
        f32x4 dr = {0.f, 0.f, 0.f, 0.f}, w;
        if (p.w < 2) mma(dr, in.t[0], r0);                              // T^T is upper triangular
        mma(dr, in.t[1], r1);
#pragma unroll
        for (int r = 0; r < 4; ++r) w[r] = -in.gamma[r] * in.beta[r] * dr[r];
        put4<3>(lds.u + p.l16 * UP + p.i0, 16 * UP, w);
        lds.b.dr[p.w][p.lane] = dr;
        lds_barrier();
        const Op<3> w0 = frag_n<3>(lds.u, 16 * UP, UP, 0, 0, p.lane), w1 = frag_n<3>(lds.u, 16 * UP, UP, 0, 32, p.lane);
        f32x4 y[NT];
#pragma unroll
        for (int x = 0; x < NT; ++x) y[x] = lds.y[p.w][x][p.lane];
        if (L::KBUFS > 1) take_k(i + 1);
#pragma unroll
        for (int x = 0; x < NT; ++x) {
            s[x] = s[x] * in.end + y[x];
            mma(s[x], kt[x][0], w0);
            mma(s[x], kt[x][1], w1);
        }
        if (L::KBUFS == 1) { lds_barrier(); take_k(i + 1); }
    };
    for (int i = 0; i < p.chunks; i += 2) {
        step(in0, in1, i);
        if (i + 1 < p.chunks) step(in1, in0, i + 1);
    }
    store_state(a.dstate_in, p, s);
}

template <typename T, int D>
__device__ inline void backward_helper(const DeltaArgs &a, const Place<T, D> p, ChainLds<T, D> &lds)
{
    using L = ChainLds<T, D>;
    constexpr int P = L::P, NT = D / 64;
    if (!p.chunks) return;
    Part<T, D, 64, D / 4, L::OP> kn, qn;
    struct In {
        Four<T> v, o;
        f32x4 gamma, beta;
    } in0, in1;
    u16 *Q = lds.b.q[p.w];
    auto fetch_rows = [&](int ch) __attribute__((always_inline)) {
        kn.load(p.k + (size_t)ch * 64 * D + p.w * (D / 4), 0, p.last(ch), p.lane);
        qn.load(p.q + (size_t)ch * 64 * D + p.w * (D / 4), 0, p.last(ch), p.lane);
    };
    auto fetch = [&](In &n, int ch) __attribute__((always_inline)) {
        n.v.load(reinterpret_cast<const T *>(a.v) + p.rows(a, ch), D, p.i0, p.last(ch), p.c0 + p.l16);
        n.o.load(reinterpret_cast<const T *>(a.dout) + p.rows(a, ch), D, p.i0, p.last(ch), p.c0 + p.l16);
        n.gamma = load4(a.gate[p.at(a, ch)].gamma + p.i0);
        n.beta = load4(a.gate[p.at(a, ch)].beta + p.i0);
    };
    fetch_rows(p.chunks - 1);
    fetch(in0, p.chunks - 1);
    kn.put(lds.k[0][p.w], p.lane);
    qn.put(Q, p.lane);
    lds_barrier();
    auto step = [&](const In &in, In &next, int i) __attribute__((always_inline)) {
        const int ch = p.chunks - 1 - i, valid = p.last(ch) + 1;
        const size_t at = p.at(a, ch);
        fetch_rows(max(ch - 1, 0));
        fetch(next, max(ch - 1, 0));
        f32x4 go = in.o.get(p.i0, valid);
        const f32x4 v = in.v.get(p.i0, valid);
#pragma unroll
        for (int r = 0; r < 4; ++r) go[r] *= a.scale * in.gamma[r];
        put4<3>(lds.g + p.l16 * UP + p.i0, 16 * UP, go);
        lds_barrier();
        const Op<3> g0 = frag_n<3>(lds.g, 16 * UP, UP, 0, 0, p.lane), g1 = frag_n<3>(lds.g, 16 * UP, UP, 0, 32, p.lane);
        f32x4 y[NT];
#pragma unroll
        for (int x = 0; x < NT; ++x) {
            y[x] = f32x4{0.f, 0.f, 0.f, 0.f};
            mma(y[x], frag_t<P>(Q, 64 * L::OP, L::OP, 16 * x, 0, p.lane), g0);
            mma(y[x], frag_t<P>(Q, 64 * L::OP, L::OP, 16 * x, 32, p.lane), g1);
        }
        lds_barrier();
#pragma unroll
        for (int x = 0; x < NT; ++x) lds.y[p.w][x][p.lane] = y[x];
        if (L::KBUFS > 1) kn.put(lds.k[(i + 1) & 1][p.w], p.lane);
        lds_barrier();
        const f32x4 dr = lds.b.dr[p.w][p.lane];
        if (L::KBUFS == 1) { kn.put(lds.k[0][p.w], p.lane); lds_barrier(); }
        store4(a.dr + (at * D + p.c0 + p.l16) * 64 + p.i0, dr);
        const auto rows = bounded(reinterpret_cast<T *>(a.dv) + p.rows(a, ch), valid * D);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            store_bounded(rows, T(), (p.i0 + r) * D + p.c0 + p.l16, in.beta[r] * dr[r]);
            float d = dr[r] * v[r];                                     // over the 16 channels
#pragma unroll
            for (int m = 1; m < 16; m <<= 1) d += __shfl_xor(d, m);
            a.dbv[(at * (D / 16) + p.slice) * 64 + p.i0 + r] = d;       // the same from all 16 lanes
        }
        qn.put(Q, p.lane);
    };
    for (int i = 0; i < p.chunks; i += 2) {
        step(in0, in1, i);
        if (i + 1 < p.chunks) step(in1, in0, i + 1);
    }
}

// Slices of a head on one XCD, whose L2 then serves K, Q, T and P to all of them.
__device__ inline int chain_of(int block, int total) { return (block & 7) * ((total + 7) / 8) + (block >> 3); }

}  // namespace

template <typename T, int D>
__global__ __launch_bounds__(512, 1) void delta_forward_kernel(DeltaArgs a)
{
    __shared__ __attribute__((aligned(16))) ChainLds<T, D> lds;
    const int total = a.B * a.H * (D / 16), L = chain_of(blockIdx.x, total), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (L >= total) return;
    const Place<T, D> p(a, L / (D / 16), L % (D / 16), wave & 3);
    if (wave < 4) forward_chain<T, D, true>(a, p, lds);
    else forward_helper<T, D, true>(a, p, lds);
}

// Both chains of the backward pass in one launch: the states again, and the states' gradients.  Neither needs the other.
template <typename T, int D>
__global__ __launch_bounds__(512, 1) void delta_backward_kernel(DeltaArgs a)
{
    __shared__ __attribute__((aligned(16))) ChainLds<T, D> lds;
    const int total = a.B * a.H * (D / 16), blocks = (total + 7) / 8 * 8, which = blockIdx.x >= (unsigned)blocks;
    const int L = chain_of(blockIdx.x - which * blocks, total), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (L >= total) return;
    const Place<T, D> p(a, L / (D / 16), L % (D / 16), wave & 3);
    if (which) {
        if (wave < 4) forward_chain<T, D, false>(a, p, lds);
        else forward_helper<T, D, false>(a, p, lds);
    } else {
        if (wave < 4) backward_chain<T, D>(a, p, lds);
        else backward_helper<T, D>(a, p, lds);
    }
}

template <typename T, int D>
static hipError_t chains(const DeltaArgs &a, bool backward, hipStream_t st)
{
    const int blocks = (a.B * a.H * (D / 16) + 7) / 8 * 8;
    if (backward) launch_kernel((delta_backward_kernel<T, D>), dim3(2 * blocks), dim3(512), 0, st, a);
    else launch_kernel((delta_forward_kernel<T, D>), dim3(blocks), dim3(512), 0, st, a);
    return take_launch_status();
}

hipError_t launch_delta_chains(const DeltaArgs &a, bool backward, hipStream_t st)
{
    if (a.bf16) return a.D == 128 ? chains<u16, 128>(a, backward, st) : chains<u16, 64>(a, backward, st);
    return a.D == 128 ? chains<float, 128>(a, backward, st) : chains<float, 64>(a, backward, st);
}

hipError_t launch_delta_fwd(const DeltaArgs &a, hipStream_t st)
{
    if (const hipError_t e = launch_delta_chunk(a, st)) return e;
    return launch_delta_chains(a, false, st);
}

}  // namespace salad
