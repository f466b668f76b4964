// The chains of the gated delta rule: the states from the first chunk to the last, and their gradients from the last to the first
// (delta_chunk.hip and delta_grad.hip have the formulas).  The value channels are independent, and a wave takes 16 of them with the whole
// state, D key channels, in accumulators.  A chunk is
//   K S,   R = beta (V - gamma K S),   U = T R,   S <- gamma_63 S + K^T (tail U)
// (backward: dU = X + tail K dS, dR = T^T dU, dS <- gamma_63 dS + Q^T (scale gamma dO) - K^T (beta gamma dR)), and what one product leaves in the
// accumulators is an operand of the next as it stands (delta_planes.h): the chain never leaves its wave's registers.  What all waves
// read, K, T, V and the decays, lies in LDS, a chunk's while the next one's is on its way: 4 more waves, one on each SIMD, load it, and
// forward compute O = scale gamma Q S + P U from the operands that the chain leaves behind.
// A chunk takes 2.8 us at d = 128 (bf16 tensors; with O 3.1), about 6700 cycles: 132 products of 16 cycles each (backward 180) and about 400 vector
// instructions, most of them splits into planes, one behind the other in one wave, with 490 of the helper on the same SIMD and the latency of
// LDS between them.  Neither memory (406 MB in 590 us at 12 heads, N = 32760) nor the chip's matrix rate is near its bound.
//
// Few heads leave most of the chip idle, so the chunks are cut into groups.  The state behind a group is linear in the one before it,
// S' = M S + B: chains from zeros give B and chains from the unit matrix without values give M, for all groups at once; a short
// kernel goes through the groups, and then every group runs from its own state.  The gradients' map is M transposed.
#include <algorithm>
#include <type_traits>

#include "causal.h"
#include "delta_planes.h"

namespace salad {

namespace {

enum Kind { OUT, KEEP, SUM };       // forward call: the output; backward call: states and u, or dS and dR, are kept; a group's B or M alone

template <typename T, int D, bool BACK> struct Shape {
    static constexpr int P = planes_of<T>();
    static constexpr int SL = P == 1 ? 4 : 2;                               // waves of the chain, 16 value channels each
    static constexpr int KBUFS = P == 1 ? 2 : 1;                            // K (and Q) of two chunks, where LDS has room
    static constexpr int VP = 16 * SL + 8;                                  // pitch
    static constexpr int UO = out_planes<T>();
    static constexpr bool QTILE = BACK || P == 1;                           // Q goes through LDS
    static constexpr int THREADS = 64 * (SL + 4);
};

template <typename T, int D, bool BACK> struct ChainLds {
    using H = Shape<T, D, BACK>;
    u16 k[H::KBUFS][H::P * 64 * D];
    u16 q[BACK ? H::KBUFS : 1][H::QTILE ? H::P * 64 * D : 8];
    u16 t[3 * TRI];
    T v[64][H::VP];                             // values; backward: dO
    float gamma[64], tail[64], beta[64];
    struct Side { u32x4 so[H::SL][D / 32][H::P][64], uo[H::SL][2][H::UO][64]; };
    Side side[BACK ? 0 : 2];                    // the state and u as operands, for O a chunk later
};

// a 64 x 16 SL part of V or dO
template <typename T, int D, int W, int PITCH> struct Vals {
    static constexpr int PER = 16 / sizeof(T), LPR = W / PER, RPI = 256 / LPR, NL = (64 + RPI - 1) / RPI;
    u32x4 r[NL];
    __device__ inline void load(const T *base, int last, int t)
    {
#pragma unroll
        for (int i = 0; i < NL; ++i) r[i] = *reinterpret_cast<const u32x4 *>(base + (unsigned)(min(i * RPI + t / LPR, last) * D + t % LPR * PER));
    }
    __device__ inline void put(T (*tile)[PITCH], int t, int valid) const    // zeros behind the last token
    {
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            const int row = i * RPI + t / LPR;
            if (NL * RPI == 64 || row < 64) *reinterpret_cast<u32x4 *>(&tile[row][t % LPR * PER]) = row < valid ? r[i] : u32x4{0, 0, 0, 0};
        }
    }
};

// where a workgroup works: value channels from c0 on, chunks [first, end) of the sample
struct Job {
    int bh, group, c0, len, first, end;
    bool unit;                                  // SUM: the chain from the unit matrix
};

template <int VP>
__device__ inline f32x4 values(const u16 (*v)[VP], int row, int c, int lane)    // rows row + 4 (lane / 16).., column c + lane % 16
{
    const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        (s16x4 __attribute__((address_space(3))) *)LDS_PTR(&v[row + 4 * (lane >> 4) + ((lane >> 2) & 3)][c + 4 * (lane & 3)]));
    return f32x4{__uint_as_float((uint32_t)(u16)x[0] << 16), __uint_as_float((uint32_t)(u16)x[1] << 16), __uint_as_float((uint32_t)(u16)x[2] << 16),
                 __uint_as_float((uint32_t)(u16)x[3] << 16)};
}
template <int VP>
__device__ inline f32x4 values(const float (*v)[VP], int row, int c, int lane)
{
    f32x4 x;
#pragma unroll
    for (int r = 0; r < 4; ++r) x[r] = v[row + 4 * (lane >> 4) + r][c + (lane & 15)];
    return x;
}

__device__ inline Op<3> tri_op(const u16 *t, int piece, int lane)
{
    Op<3> f;
#pragma unroll
    for (int p = 0; p < 3; ++p) f.p[p] = *reinterpret_cast<const bf16x8 *>(t + p * TRI + (piece * 64 + lane) * 8);
    return f;
}

// Barriers of both roles: before the first chunk; in a chunk behind T R (T, V and the decays are free), where K has one buffer behind
// the products with it, and at its end (the next chunk's operands are there).

template <typename T, int D, bool BACK, Kind KIND>
__device__ inline void chain(const DeltaArgs &a, const Job &j, ChainLds<T, D, BACK> &lds, int w, int lane)
{
    using H = Shape<T, D, BACK>;
    constexpr int P = H::P, NK = D / 32;
    const int l16 = lane & 15, l4 = lane >> 4, c = j.c0 + 16 * w + l16, n = j.end - j.first;
    const bool unit = KIND == SUM && !BACK && j.unit;       // the chain from the unit matrix, without values
    f32x4 s[2 * NK];                            // tile 2 ks + x
    // state: key channel 32 ks + 8 l4 + 4 x + r, value channel c
    const float *from = KIND == SUM ? nullptr : a.groups > 1 ? (BACK ? a.gstart_b : a.gstart) + ((size_t)j.bh * a.groups + j.group) * D * D
                                                             : BACK ? a.dstate_out + (a.dstate_out ? (size_t)j.bh * D * D : 0)
                                                                    : a.state_in + (a.state_in ? (size_t)j.bh * D * D : 0);
    const bool first_group = BACK ? j.group == a.groups - 1 : j.group == 0;
    if (KIND == SUM && first_group) {           // nothing is before it: its B is the state behind it
        const float *in = BACK ? a.dstate_out : a.state_in;
        from = in ? in + (size_t)j.bh * D * D : nullptr;
    }
#pragma unroll
    for (int ks = 0; ks < NK; ++ks)
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int row = 32 * ks + 8 * l4 + 4 * x + r;
                s[2 * ks + x][r] = unit ? (row == c ? 1.f : 0.f) : from ? from[(size_t)row * D + c] : 0.f;
            }
    f32x4 x[4];                                 // backward: X = P^T dO of the next chunk
    auto load_x = [&](int i) __attribute__((always_inline)) {
#pragma unroll
        for (int rt = 0; rt < 4; ++rt) x[rt] = load4(a.dr + (((size_t)j.bh * a.chunks + j.end - 1 - i) * D + c) * 64 + 16 * rt + 4 * l4);
    };
    if (BACK && n > 0) load_x(0);
    // What is an operand next is split while the matrix cores are at the product before: the tokens go in two halves, the first of them (of the
    // last in the backward pass) complete one product earlier.
    constexpr int A = BACK ? 2 : 0, B = BACK ? 0 : 2, KA = BACK ? 1 : 0, KB = BACK ? 0 : 1;      // first tiles of the halves; their contraction halves
    Op<3> so[NK];                               // the state as an operand
#pragma unroll
    for (int ks = 0; ks < NK; ++ks) so[ks] = op_of<3>(s[2 * ks], s[2 * ks + 1]);
    if (n > 0) lds_barrier();
    for (int i = 0; i < n; ++i) {
        const int ch = BACK ? j.end - 1 - i : j.first + i;
        const size_t at = (size_t)j.bh * a.chunks + ch;
        const u16 *K = lds.k[i & (H::KBUFS - 1)], *Q = lds.q[BACK ? i & (H::KBUFS - 1) : 0];
        const float end = lds.gamma[63];
        if (KIND == KEEP)
#pragma unroll
            for (int ks = 0; ks < NK; ++ks)
#pragma unroll
                for (int y = 0; y < 2; ++y) store4((BACK ? a.ds1 : a.s0) + (at * D + c) * D + 32 * ks + 8 * l4 + 4 * y, s[2 * ks + y]);
        f32x4 acc[4], u[4];
#pragma unroll
        for (int rt = 0; rt < 4; ++rt) acc[rt] = u[rt] = f32x4{0.f, 0.f, 0.f, 0.f};
        // K S
        auto k_s = [&](int half) __attribute__((always_inline)) {
#pragma unroll
            for (int ks = 0; ks < NK; ++ks) {
                const Op<P> kf[2] = {frag_k<P, D>(K, 16 * half, ks, lane), frag_k<P, D>(K, 16 * half + 16, ks, lane)};
                mmas<2>(acc + half, kf, so[ks]);
            }
        };
        // R, or dU, of a half, as an operand
        auto r_op = [&](int half) __attribute__((always_inline)) {
#pragma unroll
            for (int rt = half; rt < half + 2; ++rt) {
                if (BACK) {
                    acc[rt] = x[rt] + load4(lds.tail + 16 * rt + 4 * l4) * acc[rt];
                } else {
                    const f32x4 gamma = load4(lds.gamma + 16 * rt + 4 * l4), beta = load4(lds.beta + 16 * rt + 4 * l4);
                    if (unit) acc[rt] = -beta * gamma * acc[rt];
                    else acc[rt] = beta * (values(lds.v, 16 * rt, 16 * w, lane) - gamma * acc[rt]);
                }
            }
            return op_of<3>(acc[half], acc[half + 1]);
        };
        // u of a half on its way into the state, as an operand
        auto u_op = [&](int half) __attribute__((always_inline)) {
            if constexpr (KIND == OUT) {
                const Op<H::UO> o = op_of<H::UO>(u[half], u[half + 1]);
#pragma unroll
                for (int p = 0; p < H::UO; ++p) lds.side[i & 1].uo[w][half / 2][p][lane] = __builtin_bit_cast(u32x4, o.p[p]);
            }
#pragma unroll
            for (int rt = half; rt < half + 2; ++rt) {
                if (KIND == KEEP) store4((BACK ? a.dr : a.u) + (at * D + c) * 64 + 16 * rt + 4 * l4, u[rt]);
                if (BACK) u[rt] *= -load4(lds.gamma + 16 * rt + 4 * l4) * load4(lds.beta + 16 * rt + 4 * l4);
                else u[rt] *= load4(lds.tail + 16 * rt + 4 * l4);
            }
            return op_of<3>(u[half], u[half + 1]);
        };
        // into the state, over half kt of the tokens
        auto into = [&](const u16 *tile, int ks, int kt, const Op<3> &o) __attribute__((always_inline)) {
            const Op<P> f[2] = {frag_c<P, D>(tile, ks, 0, kt, lane), frag_c<P, D>(tile, ks, 1, kt, lane)};
            mmas<2>(s + 2 * ks, f, o);
        };
        if constexpr (KIND == OUT)
#pragma unroll
            for (int ks = 0; ks < NK; ++ks)
#pragma unroll
                for (int p = 0; p < P; ++p) lds.side[i & 1].so[w][ks][p][lane] = __builtin_bit_cast(u32x4, so[ks].p[p]);
        k_s(A);
        Op<3> ta[4], tb[2];                     // T's pieces by the first half and by the second
#pragma unroll
        for (int rt = 0; rt < 4; ++rt) ta[rt] = tri_op(lds.t, BACK ? tri_upper(rt, 1) : tri_lower(rt, 0), lane);
        const Op<3> ra = r_op(A);
        k_s(B);
#pragma unroll
        for (int x2 = 0; x2 < 2 * NK; ++x2) s[x2] *= end;
        mmas<4>(u, ta, ra);
        const Op<3> rb = r_op(B);
        tb[0] = tri_op(lds.t, BACK ? tri_upper(0, 0) : tri_lower(2, 1), lane);
        tb[1] = tri_op(lds.t, BACK ? tri_upper(1, 0) : tri_lower(3, 1), lane);
        if (BACK) {
            load_x(min(i + 1, n - 1));
            f32x4 go[4];
#pragma unroll
            for (int rt = 0; rt < 4; ++rt) go[rt] = a.scale * load4(lds.gamma + 16 * rt + 4 * l4) * values(lds.v, 16 * rt, 16 * w, lane);
            const Op<3> g0 = op_of<3>(go[0], go[1]), g1 = op_of<3>(go[2], go[3]);
#pragma unroll
            for (int ks = 0; ks < NK; ++ks) { into(Q, ks, 0, g0); into(Q, ks, 1, g1); }
        }
        mmas<2>(u + B, tb, rb);
        const Op<3> ua = u_op(A);
#pragma unroll
        for (int ks = 0; ks < NK; ++ks) into(K, ks, KA, ua);
        const Op<3> ub = u_op(B);
        lds_barrier();
#pragma unroll
        for (int ks = 0; ks < NK; ++ks) {
            into(K, ks, KB, ub);
            so[ks] = op_of<3>(s[2 * ks], s[2 * ks + 1]);
        }
        if (H::KBUFS == 1) lds_barrier();
        lds_barrier();
    }
    // the state behind the last chunk
    const bool last_group = BACK ? j.group == 0 : j.group == a.groups - 1;
    float *to = KIND == SUM ? (unit ? a.gmap : BACK ? a.gsum_b : a.gsum) + ((size_t)j.bh * a.groups + j.group) * D * D
                : !last_group ? nullptr : BACK ? (a.dstate_in ? a.dstate_in + (size_t)j.bh * D * D : nullptr) : (a.state_out ? a.state_out + (size_t)j.bh * D * D : nullptr);
    if (to)
#pragma unroll
        for (int ks = 0; ks < NK; ++ks)
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int r = 0; r < 4; ++r) to[(size_t)(32 * ks + 8 * l4 + 4 * x + r) * D + c] = s[2 * ks + x][r];
}

// The next chunk's operands, and O of the chunk before.  Wave w of 4: 16 tokens of O.
template <typename T, int D, bool BACK, Kind KIND>
__device__ inline void helper(const DeltaArgs &a, const Job &j, ChainLds<T, D, BACK> &lds, int w, int lane)
{
    using H = Shape<T, D, BACK>;
    constexpr int P = H::P, NK = D / 32, SL = H::SL;
    const int t = w * 64 + lane, l16 = lane & 15, l4 = lane >> 4, n = j.end - j.first;
    if (n <= 0) return;
    const int b = j.bh / a.H, h = j.bh - b * a.H, hk = h / (a.H / a.Hk);
    const T *k = reinterpret_cast<const T *>(a.k) + ((size_t)b * a.Hk + hk) * a.N * D, *q = reinterpret_cast<const T *>(a.q) + ((size_t)b * a.Hk + hk) * a.N * D;
    const T *v = reinterpret_cast<const T *>(BACK ? a.dout : a.v) + (size_t)j.bh * a.N * D + j.c0;
    const u16 *tri = BACK ? a.ttf : a.tf;
    auto chunk_of = [&](int i) { return BACK ? j.end - 1 - i : j.first + i; };
    auto valid_of = [&](int ch) { return min(j.len - ch * 64, 64); };

    Tile64<T, D> kr, qr;
    Vals<T, D, 16 * SL, H::VP> vr;
    u32x4 tr[(3 * TRI / 8 + 255) / 256];
    float gr = 0.f;
    constexpr int NT = sizeof(tr) / 16;
    auto load = [&](int i) __attribute__((always_inline)) {
        const int ch = chunk_of(i), valid = valid_of(ch);
        const size_t at = (size_t)j.bh * a.chunks + ch;
        kr.load_clamped(k + (size_t)ch * 64 * D, valid - 1, t);
        if (BACK) qr.load_clamped(q + (size_t)ch * 64 * D, valid - 1, t);
        vr.load(v + (size_t)ch * 64 * D, valid - 1, t);
#pragma unroll
        for (int x = 0; x < NT; ++x) tr[x] = *reinterpret_cast<const u32x4 *>(tri + at * (3 * TRI) + (size_t)min(x * 256 + t, 3 * TRI / 8 - 1) * 8);
        gr = reinterpret_cast<const float *>(a.gate + at)[min(t, 191)];
    };
    auto put_small = [&](int i) __attribute__((always_inline)) {
        vr.put(lds.v, t, valid_of(chunk_of(i)));
#pragma unroll
        for (int x = 0; x < NT; ++x)
            if ((x + 1) * 256 <= 3 * TRI / 8 || x * 256 + t < 3 * TRI / 8) *reinterpret_cast<u32x4 *>(lds.t + (x * 256 + t) * 8) = tr[x];
        if (t < 64) lds.gamma[t] = gr;
        else if (t < 128) lds.tail[t - 64] = gr;
        else if (t < 192) lds.beta[t - 128] = gr;
    };
    auto put_rows = [&](int i) __attribute__((always_inline)) {
        kr.store_swizzled(lds.k[i & (H::KBUFS - 1)], t);
        if (BACK) qr.store_swizzled(lds.q[i & (H::KBUFS - 1)], t);
    };
    // O: what it takes besides the chain's operands, loaded in its chunk, used in the next
    Op<H::UO> pf[2];
    Op<P> qn[P == 1 ? 1 : NK];
    float gamma = 0.f;
    auto load_out = [&](int i) __attribute__((always_inline)) {
        const int ch = chunk_of(i), valid = valid_of(ch);
        const size_t at = (size_t)j.bh * a.chunks + ch;
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int p = 0; p < H::UO; ++p)
                pf[kt].p[p] = *reinterpret_cast<const bf16x8 *>(a.pf + at * (H::UO * TRI) + p * TRI + (tri_lower(w, w < 2 ? 0 : kt) * 64 + lane) * 8);
        gamma = a.scale * a.gate[at].gamma[16 * w + l16];
        if constexpr (H::QTILE) qr.load_clamped(q + (size_t)ch * 64 * D, valid - 1, t);
        else
#pragma unroll
            for (int ks = 0; ks < NK; ++ks) qn[ks] = frag_g(q + (size_t)(ch * 64 + min(16 * w + l16, valid - 1)) * D + 32 * ks + 8 * l4, true);
    };
    auto output = [&](int i) __attribute__((always_inline)) {
        if constexpr (KIND == OUT) {
            const int ch = chunk_of(i);
            const auto &side = lds.side[i & 1];
            const auto rows = bounded(reinterpret_cast<T *>(a.out) + ((size_t)j.bh * a.N + (size_t)ch * 64) * D, valid_of(ch) * D);
            Op<P> qo[NK];
#pragma unroll
            for (int ks = 0; ks < NK; ++ks) {
                if constexpr (H::QTILE) qo[ks] = frag_k<P, D>(lds.q[0], 16 * w, ks, lane);
                else qo[ks] = qn[ks];
            }
#pragma unroll
            for (int sl = 0; sl < SL; ++sl) {           // transposed: rows value channels, columns tokens
                f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int ks = 0; ks < NK; ++ks) {
                    Op<P> so;
#pragma unroll
                    for (int p = 0; p < P; ++p) so.p[p] = __builtin_bit_cast(bf16x8, side.so[sl][ks][p][lane]);
                    mma(o, so, qo[ks]);
                }
                o *= gamma;
#pragma unroll
                for (int kt = 0; kt < 2; ++kt) {
                    if (kt && w < 2) continue;          // P is lower triangular
                    Op<H::UO> uo;
#pragma unroll
                    for (int p = 0; p < H::UO; ++p) uo.p[p] = __builtin_bit_cast(bf16x8, side.uo[sl][kt][p][lane]);
                    mma(o, uo, pf[kt]);
                }
                store_bounded(rows, T(), (16 * w + l16) * D + j.c0 + 16 * sl + 4 * l4, o);
            }
        }
    };

    load(0);
    put_rows(0);
    put_small(0);
    lds_barrier();
    for (int i = 0; i < n; ++i) {
        load(min(i + 1, n - 1));
        if (KIND == OUT && i > 0) output(i - 1);
        if (KIND == OUT) load_out(i);
        if (H::KBUFS > 1) put_rows(i + 1);
        lds_barrier();
        put_small(min(i + 1, n - 1));
        if (KIND == OUT && H::QTILE) qr.store_swizzled(lds.q[0], t);
        if (H::KBUFS == 1) { lds_barrier(); put_rows(i + 1); }
        lds_barrier();
    }
    if (KIND == OUT) output(n - 1);
}

template <typename T, int D, bool BACK, Kind KIND>
__device__ inline void run(const DeltaArgs &a, const Job &j, ChainLds<T, D, BACK> &lds)
{
    constexpr int SL = Shape<T, D, BACK>::SL;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (wave < SL) chain<T, D, BACK, KIND>(a, j, lds, wave, lane);
    else helper<T, D, BACK, KIND>(a, j, lds, wave - SL, lane);
}

// Workgroups of a head next to each other, on one XCD: its L2 then serves the operands to all of them
__device__ inline int place_of(int block, int total) { return (block & 7) * ((total + 7) / 8) + (block >> 3); }

__device__ inline Job job_of(const DeltaArgs &a, int bh, int group, int c0, bool unit)
{
    Job j{bh, group, c0, delta_len(a, bh / a.H), 0, 0, unit};
    const int chunks = (j.len + 63) / 64;
    j.first = min(group * a.per_group, chunks);
    j.end = min(j.first + a.per_group, chunks);
    return j;
}

}  // namespace

template <typename T, int D> union BothLds {
    ChainLds<T, D, false> f;
    ChainLds<T, D, true> b;
};
template <typename T, int D> constexpr int PARTS = D / (16 * Shape<T, D, false>::SL);      // workgroups across the value channels

template <typename T, int D>
__global__ __launch_bounds__((Shape<T, D, false>::THREADS), 1) void delta_forward_kernel(DeltaArgs a)
{
    __shared__ __attribute__((aligned(16))) ChainLds<T, D, false> lds;
    constexpr int NP = PARTS<T, D>;
    const int total = a.B * a.H * a.groups * NP, L = place_of(blockIdx.x, total);
    if (L >= total) return;
    run<T, D, false, OUT>(a, job_of(a, L / NP / a.groups, L / NP % a.groups, L % NP * (D / NP), false), lds);
}

// Both chains of the backward pass, the longer one first.  Neither needs the other.
template <typename T, int D>
__global__ __launch_bounds__((Shape<T, D, false>::THREADS), 1) void delta_backward_kernel(DeltaArgs a)
{
    __shared__ __attribute__((aligned(16))) BothLds<T, D> lds;
    constexpr int NP = PARTS<T, D>;
    const int total = a.B * a.H * a.groups * NP, half = (total + 7) / 8 * 8;
    const bool back = (int)blockIdx.x < half;
    const int L = place_of(back ? blockIdx.x : blockIdx.x - half, total);
    if (L >= total) return;
    const Job j = job_of(a, L / NP / a.groups, L / NP % a.groups, L % NP * (D / NP), false);
    if (back) run<T, D, true, KEEP>(a, j, lds.b);
    else run<T, D, false, KEEP>(a, j, lds.f);
}

// B and M of the groups that another one follows, and for the backward pass B of the gradients (their map is M transposed).  The first
// group needs no M.
template <typename T, int D>
__global__ __launch_bounds__((Shape<T, D, false>::THREADS), 1) void delta_sum_kernel(DeltaArgs a, int kinds)
{
    __shared__ __attribute__((aligned(16))) BothLds<T, D> lds;
    constexpr int NP = PARTS<T, D>;
    const int total = a.B * a.H * (a.groups - 1) * kinds * NP, L = place_of(blockIdx.x, total);
    if (L >= total) return;
    const int part = L % NP, kind = L / NP % kinds, g = L / NP / kinds % (a.groups - 1), bh = L / NP / kinds / (a.groups - 1);
    if (kind == 1 && g == 0) return;
    const Job j = job_of(a, bh, kind == 2 ? g + 1 : g, part * (D / NP), kind == 1);
    if (kind == 2) run<T, D, true, SUM>(a, j, lds.b);
    else run<T, D, false, SUM>(a, j, lds.f);
}

// The states that the groups start from: S <- M S + B from group to group (backward: M transposed, from the last).  A workgroup has 16 value
// channels; S is in LDS, the products are fp32.  6 groups of 12 heads, d = 128: 19 us (35 with operands that are no neighbours in memory).
template <int D>
__global__ __launch_bounds__(256) void delta_start_kernel(DeltaArgs a, int blocks)
{
    __shared__ float S[D][17];
    const bool BACK = (int)blockIdx.x >= blocks;
    const int bh = blockIdx.x % blocks / (D / 16), c0 = blockIdx.x % (D / 16) * 16;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l16 = lane & 15, l4 = lane >> 4;
    const float *in = BACK ? a.dstate_out : a.state_in;
    for (int i = 0; i < a.groups; ++i) {
        const int g = BACK ? a.groups - 1 - i : i;
        const size_t at = ((size_t)bh * a.groups + g) * D * D;
        float *start = (BACK ? a.gstart_b : a.gstart) + at;
        if (i == 0) {
            for (int e = tid; e < D * 16; e += 256) start[(size_t)(e / 16) * D + c0 + e % 16] = in ? in[((size_t)bh * D + e / 16) * D + c0 + e % 16] : 0.f;
            continue;
        }
        const size_t before = BACK ? at + (size_t)D * D : at - (size_t)D * D;
        const float *sum = (BACK ? a.gsum_b : a.gsum) + before, *map = a.gmap + before;
        f32x4 c[D / 64];
#pragma unroll
        for (int x = 0; x < D / 64; ++x) {
            const int row = wave * (D / 4) + 16 * x;
#pragma unroll
            for (int r = 0; r < 4; ++r) c[x][r] = sum[(size_t)(row + 4 * l4 + r) * D + c0 + l16];
            if (i > 1) {
                // step 4 kb + y of the contraction takes rows 16 kb + 4 l4 + y of S: a lane's operands are neighbours in M
                f32x4 m[D / 16];
#pragma unroll
                for (int kb = 0; kb < D / 16; ++kb) {
                    if (!BACK) m[kb] = load4(map + (size_t)(row + l16) * D + 16 * kb + 4 * l4);
                    else
#pragma unroll
                        for (int y = 0; y < 4; ++y) m[kb][y] = map[(size_t)(16 * kb + 4 * l4 + y) * D + row + l16];
                }
#pragma unroll
                for (int kb = 0; kb < D / 16; ++kb)
#pragma unroll
                    for (int y = 0; y < 4; ++y) c[x] = __builtin_amdgcn_mfma_f32_16x16x4f32(m[kb][y], S[16 * kb + 4 * l4 + y][l16], c[x], 0, 0, 0);
            }
        }
        __syncthreads();
#pragma unroll
        for (int x = 0; x < D / 64; ++x)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int row = wave * (D / 4) + 16 * x + 4 * l4 + r;
                S[row][l16] = c[x][r];
                start[(size_t)row * D + c0 + l16] = c[x][r];
            }
        __syncthreads();
    }
}

// Groups: as many as shorten the passes.  One pass of all chunks without groups; with G groups one of a G-th for B and M, and one
// of a G-th for the rest, each as often as its workgroups fill the chip's 256 compute units; 4 chunks of time for a step of the start kernel.
// Fewer than 8 chunks a group, or less than a fifth to win, leave one group: the sum and start kernels cost that much.
// Whole calls, us, in one group, as the rule cuts them, and at best (groups):
//   12 heads, d = 128   forward, 512 chunks 1490 591 (6) 564 (10),  64 chunks 189 120 (5) 116 (6);   backward, 195 chunks 1189 825 (4) 812 (10)
//   40 heads, d = 128   forward, 256 chunks 870 870 (1) 834 (3);                                     backward 2862 2862 (1) 2862 (1)
//   64 heads, d = 64    forward, 64 chunks 181 181 (1) 164 (3);                                      backward 613 612 (1) 610 (2)
//   4 heads, d = 128    forward, 32 chunks 96 96 (1) 73 (4);                                         backward 178 178 (1) 129 (8)
//   2 heads, d = 64     forward, 55 chunks 120 66 (5) 56 (8);                                        backward 194 108 (5) 91 (10)
// So it is within 5 % of the best for many chunks; short sequences of few heads would take more groups than it gives them.
int delta_groups(const DeltaArgs &a, bool backward)
{
    const int parts = a.D / (a.bf16 ? 64 : 32);
    const long long one = (long long)a.B * a.H * parts * (backward ? 2 : 1);
    auto rounds = [](long long wgs) { return (wgs + 255) / 256; };
    const double alone = (double)a.chunks * rounds(one);
    int best = 1;
    double least = 0.8 * alone;                 // three short kernels for one long: not for little
    for (int g = 2; g <= 32 && a.chunks / g >= 8; ++g) {
        const double per = (a.chunks + g - 1) / g;
        const double t = per * (rounds((long long)a.B * a.H * (g - 1) * parts * (backward ? 3 : 2)) + rounds(one * g)) + 4.0 * g;
        if (t < least) { best = g; least = t; }
    }
    return best;
}

template <typename T, int D>
static hipError_t chains(const DeltaArgs &a, bool backward, hipStream_t st)
{
    const long long BH = (long long)a.B * a.H, total = (BH * a.groups * PARTS<T, D> + 7) / 8 * 8;
    const dim3 threads(Shape<T, D, false>::THREADS);
    if (a.groups > 1) {
        const int kinds = backward ? 3 : 2, blocks = (int)BH * (D / 16);
        launch_kernel((delta_sum_kernel<T, D>), dim3((unsigned)((BH * (a.groups - 1) * kinds * PARTS<T, D> + 7) / 8 * 8)), threads, 0, st, a, kinds);
        launch_kernel((delta_start_kernel<D>), dim3(backward ? 2 * blocks : blocks), dim3(256), 0, st, a, blocks);
    }
    if (backward) launch_kernel((delta_backward_kernel<T, D>), dim3((unsigned)(2 * total)), threads, 0, st, a);
    else launch_kernel((delta_forward_kernel<T, D>), dim3((unsigned)total), threads, 0, st, a);
    return take_launch_status();
}

hipError_t launch_delta_chains(const DeltaArgs &a, bool backward, hipStream_t st)
{
    if (a.bf16) return a.D == 128 ? chains<u16, 128>(a, backward, st) : chains<u16, 64>(a, backward, st);
    return a.D == 128 ? chains<float, 128>(a, backward, st) : chains<float, 64>(a, backward, st);
}

hipError_t launch_delta_fwd(const DeltaArgs &a, hipStream_t st)
{
    if (const hipError_t e = launch_delta_chunk(a, false, st)) return e;
    return launch_delta_chains(a, false, st);
}

}  // namespace salad
