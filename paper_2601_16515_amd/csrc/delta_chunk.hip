// The gated delta rule over whole sequences, in chunks of 64 tokens.  Within a chunk, with b_i the running sum of g, gamma_i = e^b_i and
// S_0 the state before it,
//   u_i = beta_i (v_i - gamma_i S_0^T k_i - sum_{j<i} e^(b_i - b_j) (k_i.k_j) u_j),
// a triangular system (I + A) U = R, A_ij = beta_i e^(b_i - b_j) k_i.k_j (j < i), R = beta (V - gamma K S_0), and
//   S_64 = gamma_63 S_0 + K^T (e^(b_63 - b_i) u_i),     O = scale gamma Q S_0 + P U,  P_ij = scale e^(b_i - b_j) q_i.k_j  (j <= i).
// T = (I + A)^-1 and P do not depend on the state.  So there are three kernels:
//   delta_chunk_kernel   T of every chunk, all at once
//   delta_scan_kernel    the states, chunk after chunk; the value channels are independent, 16 of them a workgroup
//   delta_out_kernel     O of every chunk, all at once
// All exponents are differences of sums held in 64 bits.  Products in the chain of states keep fp32 (delta_planes.h); O is rounded
// to the tensors' type, and for bf16 so are S_0, U and P as operands of its products (half a step each, 2^-9).
#include <algorithm>

#include "causal.h"
#include "delta_planes.h"

namespace salad {

// ---- T ------------------------------------------------------------------------------------------------
template <typename T, int D>
__global__ __launch_bounds__(256) void delta_chunk_kernel(DeltaArgs a)
{
    constexpr int P = planes_of<T>(), NK = D / 32, AP = 68;
    __shared__ double bd[64];
    __shared__ float bt[64];
    __shared__ __attribute__((aligned(16))) float A[64][AP], X[64][AP], Y[32][AP];     // A, its inverse, a product on the way
    const int ch = blockIdx.x % a.chunks, bh = blockIdx.x / a.chunks, b = bh / a.H, h = bh - b * a.H, hk = h / (a.H / a.Hk);
    const int valid = min(delta_len(a, b) - ch * 64, 64);
    if (valid <= 0) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l16 = lane & 15, l4 = lane >> 4;
    const T *kp = reinterpret_cast<const T *>(a.k) + (((size_t)b * a.Hk + hk) * a.N + (size_t)ch * 64) * D;
    const size_t at = (size_t)bh * a.chunks + ch;
    if (wave == 0) {
        const size_t t = (size_t)bh * a.N + ch * 64 + lane;
        float g = lane < valid ? a.g[t] : 0.f;
        const float beta = lane < valid ? a.beta[t] : 0.f;
        g = g < -100.f ? -100.f : g;                    // e^-100 is 0 in fp32 next to anything; -infinity would leave no differences
        double s = g;
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) {
            const double o = __shfl_up(s, m);
            if (lane >= m) s += o;
        }
        const double last = __shfl(s, 63);
        bd[lane] = s;
        bt[lane] = beta;
        a.gate[at * 64 + lane] = DeltaGate{expf((float)s), expf((float)(last - s)), beta, 0.f};
        const float hi = (float)s;
        a.bsum[at * 64 + lane] = make_float2(hi, (float)(s - hi));
    }
    // A: rows 16 wave.., columns up to the diagonal
    f32x4 kk[4];
    Op<P> own[NK];
#pragma unroll
    for (int x = 0; x < NK; ++x) own[x] = frag_g(kp + (size_t)(16 * wave + l16) * D + x * 32 + 8 * l4, 16 * wave + l16 < valid);
#pragma unroll
    for (int ct = 0; ct < 4; ++ct) {
        kk[ct] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (ct <= wave)
#pragma unroll
            for (int x = 0; x < NK; ++x) mma(kk[ct], own[x], frag_g(kp + (size_t)(16 * ct + l16) * D + x * 32 + 8 * l4, 16 * ct + l16 < valid));
    }
    __syncthreads();
#pragma unroll
    for (int ct = 0; ct < 4; ++ct)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int i = 16 * wave + 4 * l4 + r, j = 16 * ct + l16;
            A[i][j] = j < i ? bt[i] * expf((float)(bd[i] - bd[j])) * kk[ct][r] : 0.f;
            X[i][j] = 0.f;
        }
    __syncthreads();
    // inverses of the four 16 x 16 blocks on the diagonal, a wave each, a column a lane: x_i = [i = c] - sum_{j<i} A_ij x_j
    if (lane < 16) {
        const int o = 16 * wave;
        float x[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            float s = i == lane ? 1.f : 0.f;
#pragma unroll
            for (int j = 0; j < i; ++j) s = fmaf(-A[o + i][o + j], x[j], s);
            x[i] = s;
            X[o + i][o + lane] = s;
        }
    }
    __syncthreads();
    // [X1 0; -X2 A21 X1, X2], for blocks of 16 and then of 32, on the fp32 matrix instruction
    auto block = [&](const float *l, int lp, const float *r, int rp, int n) {
        f32x4 c = {0.f, 0.f, 0.f, 0.f};
        for (int s = 0; s < n; s += 4) c = __builtin_amdgcn_mfma_f32_16x16x4f32(l[l16 * lp + s + l4], r[(s + l4) * rp + l16], c, 0, 0, 0);
        return c;
    };
    if (wave < 2) {
        const int o = 32 * wave;
        const f32x4 c = block(&A[o + 16][o], AP, &X[o][o], AP, 16);
#pragma unroll
        for (int r = 0; r < 4; ++r) Y[16 * wave + 4 * l4 + r][l16] = c[r];
    }
    __syncthreads();
    if (wave < 2) {
        const int o = 32 * wave;
        const f32x4 c = block(&X[o + 16][o + 16], AP, &Y[16 * wave][0], AP, 16);
#pragma unroll
        for (int r = 0; r < 4; ++r) X[o + 16 + 4 * l4 + r][o + l16] = -c[r];
    }
    __syncthreads();
    {
        const int i = wave >> 1, j = wave & 1;
        const f32x4 c = block(&A[32 + 16 * i][0], AP, &X[0][16 * j], AP, 32);
#pragma unroll
        for (int r = 0; r < 4; ++r) Y[16 * i + 4 * l4 + r][16 * j + l16] = c[r];
    }
    __syncthreads();
    {
        const int i = wave >> 1, j = wave & 1;
        const f32x4 c = block(&X[32 + 16 * i][32], AP, &Y[0][16 * j], AP, 32);
#pragma unroll
        for (int r = 0; r < 4; ++r) X[32 + 16 * i + 4 * l4 + r][16 * j + l16] = -c[r];
    }
    __syncthreads();
    // as operands: row tile = wave, halves kt of the contraction
    u16 *tf = a.tf + at * DELTA_T_ELEMS, *ttf = a.ttf ? a.ttf + at * DELTA_T_ELEMS : nullptr;
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
        const int row = 16 * wave + l16, k0 = 32 * kt + 8 * l4;
        f32x4 x = *reinterpret_cast<const f32x4 *>(&X[row][k0]), y = *reinterpret_cast<const f32x4 *>(&X[row][k0 + 4]);
        u32x2 p[3], q[3];
        split4<3>(x, p);
        split4<3>(y, q);
#pragma unroll
        for (int i = 0; i < 3; ++i) *reinterpret_cast<u32x4 *>(tf + (((i * 4 + wave) * 2 + kt) * 64 + lane) * 8) = u32x4{p[i].x, p[i].y, q[i].x, q[i].y};
        if (ttf) {
            x = f32x4{X[k0][row], X[k0 + 1][row], X[k0 + 2][row], X[k0 + 3][row]};
            y = f32x4{X[k0 + 4][row], X[k0 + 5][row], X[k0 + 6][row], X[k0 + 7][row]};
            split4<3>(x, p);
            split4<3>(y, q);
#pragma unroll
            for (int i = 0; i < 3; ++i) *reinterpret_cast<u32x4 *>(ttf + (((i * 4 + wave) * 2 + kt) * 64 + lane) * 8) = u32x4{p[i].x, p[i].y, q[i].x, q[i].y};
        }
    }
}

// ---- states ---------------------------------------------------------------------------------------------
// A workgroup: 16 value channels of one (sample, head).  Each wave keeps D / 4 rows of the state (key channels) in accumulators; a
// chunk is three products, K S_0, T R and K^T (tail u), each behind an exchange through LDS.  The chain is bound by the latency of these
// three exchanges; operands of the next chunk are loaded a chunk ahead.
// S: what is kept of the states and of u (the tensors' type forward, fp32 for the backward pass)
template <typename T, typename S, int D>
__global__ __launch_bounds__(256, 1) void delta_scan_kernel(DeltaArgs a)
{
    constexpr int P = planes_of<T>(), NT = D / 64, NK = D / 32;
    constexpr int SP = D + 8, UP = 72;
    using Tile = Tile64<T, D>;
    extern __shared__ __attribute__((aligned(16))) u16 lds[];
    u16 *Kt = lds, *St = Kt + 2 * P * Tile::PLANE, *Rt = St + 3 * 16 * SP, *Ut = Rt + 3 * 16 * UP;
    const int slices = D / 16;
    const int bh = blockIdx.x / slices, c0 = (blockIdx.x - bh * slices) * 16, b = bh / a.H, h = bh - b * a.H, hk = h / (a.H / a.Hk);
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l16 = lane & 15, l4 = lane >> 4;
    const int len = delta_len(a, b), chunks = (len + 63) / 64;
    const T *kp = reinterpret_cast<const T *>(a.k) + ((size_t)b * a.Hk + hk) * a.N * D;
    const T *vp = reinterpret_cast<const T *>(a.v) + (size_t)bh * a.N * D + c0 + l16;
    const int arow = wave * (D / 4) + 4 * l4;                           // first of the 4 key channels of an accumulator
    f32x4 s[NT];
#pragma unroll
    for (int x = 0; x < NT; ++x)
#pragma unroll
        for (int r = 0; r < 4; ++r) s[x][r] = a.state_in ? a.state_in[((size_t)bh * D + arow + 16 * x + r) * D + c0 + l16] : 0.f;

    const int i0 = 16 * wave + 4 * l4;                                  // first of the 4 tokens of an accumulator
    Tile kr;
    Op<3> tn[2];
    float vn[4];
    f32x4 gn[4];
    float endn = 0.f;
    auto fetch = [&](int ch) {
        const size_t at = (size_t)bh * a.chunks + ch;
        kr.load(kp + (size_t)ch * 64 * D, min(len - ch * 64, 64), tid);
        const u16 *tf = a.tf + at * DELTA_T_ELEMS;
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int p = 0; p < 3; ++p) tn[kt].p[p] = *reinterpret_cast<const bf16x8 *>(tf + (((p * 4 + wave) * 2 + kt) * 64 + lane) * 8);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            vn[r] = ch * 64 + i0 + r < len ? load1(vp + (size_t)(ch * 64 + i0 + r) * D) : 0.f;
            gn[r] = *reinterpret_cast<const f32x4 *>(a.gate + at * 64 + i0 + r);
        }
        endn = a.gate[at * 64 + 63].gamma;
    };
    if (chunks > 0) {
        fetch(0);
        kr.store(Kt, tid);
    }
    for (int ch = 0; ch < chunks; ++ch) {
        const size_t at = (size_t)bh * a.chunks + ch;
        const u16 *K = Kt + (ch & 1) * P * Tile::PLANE;
        Op<3> tc[2] = {tn[0], tn[1]};
        float vc[4];
        f32x4 gc[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) { vc[r] = vn[r]; gc[r] = gn[r]; }
        const float end = endn;
#pragma unroll
        for (int x = 0; x < NT; ++x) {
            put4<3>(St + l16 * SP + arow + 16 * x, 16 * SP, s[x]);
            store4(reinterpret_cast<S *>(a.s0) + (at * D + c0 + l16) * D + arow + 16 * x, s[x]);
        }
        __syncthreads();
        if (ch + 1 < chunks) fetch(ch + 1);
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int x = 0; x < NK; ++x) mma(acc, frag_n<P>(K, Tile::PLANE, Tile::PITCH, 16 * wave, 32 * x, lane), frag_n<3>(St, 16 * SP, SP, 0, 32 * x, lane));
        f32x4 rr;
#pragma unroll
        for (int r = 0; r < 4; ++r) rr[r] = gc[r][2] * (vc[r] - gc[r][0] * acc[r]);
        put4<3>(Rt + l16 * UP + i0, 16 * UP, rr);
        __syncthreads();
        f32x4 u = {0.f, 0.f, 0.f, 0.f};
        mma(u, tc[0], frag_n<3>(Rt, 16 * UP, UP, 0, 0, lane));
        if (wave >= 2) mma(u, tc[1], frag_n<3>(Rt, 16 * UP, UP, 0, 32, lane));      // T is lower triangular
        store4(reinterpret_cast<S *>(a.u) + (at * D + c0 + l16) * 64 + i0, u);
#pragma unroll
        for (int r = 0; r < 4; ++r) u[r] *= gc[r][1];
        put4<3>(Ut + l16 * UP + i0, 16 * UP, u);
        __syncthreads();
        if (ch + 1 < chunks) kr.store(Kt + ((ch + 1) & 1) * P * Tile::PLANE, tid);
#pragma unroll
        for (int x = 0; x < NT; ++x) {
            s[x] *= end;
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
                mma(s[x], frag_t<P>(K, Tile::PLANE, Tile::PITCH, wave * (D / 4) + 16 * x, 32 * kt, lane), frag_n<3>(Ut, 16 * UP, UP, 0, 32 * kt, lane));
        }
    }
    if (a.state_out)
#pragma unroll
        for (int x = 0; x < NT; ++x)
#pragma unroll
            for (int r = 0; r < 4; ++r) a.state_out[((size_t)bh * D + arow + 16 * x + r) * D + c0 + l16] = s[x][r];
}

// ---- O --------------------------------------------------------------------------------------------------
// 64 value channels of a chunk a workgroup.  Computed transposed (value channel, token): a lane's column is its token, whose decay is
// one factor, and P never leaves its wave.
template <typename T, int D>
__global__ __launch_bounds__(256, 1) void delta_out_kernel(DeltaArgs a)
{
    constexpr int P = planes_of<T>(), NK = D / 32, SP = D + 8, UP = 72;
    extern __shared__ __attribute__((aligned(16))) u16 lds[];
    u16 *S0 = lds, *Ut = S0 + P * 64 * SP, *Pt = Ut + P * 64 * UP;      // [64][D], [64][64], [64][64] by planes
    const int item = blockIdx.x / (D / 64), c0 = blockIdx.x % (D / 64) * 64;
    const int ch = item % a.chunks, bh = item / a.chunks, b = bh / a.H, h = bh - b * a.H, hk = h / (a.H / a.Hk);
    const int valid = min(delta_len(a, b) - ch * 64, 64);
    if (valid <= 0) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l16 = lane & 15, l4 = lane >> 4;
    const size_t at = (size_t)bh * a.chunks + ch, row0 = ((size_t)b * a.Hk + hk) * a.N + (size_t)ch * 64;
    const T *qp = reinterpret_cast<const T *>(a.q) + row0 * D, *kp = reinterpret_cast<const T *>(a.k) + row0 * D;
    const T *s0 = reinterpret_cast<const T *>(a.s0) + (at * D + c0) * D, *up = reinterpret_cast<const T *>(a.u) + (at * D + c0) * 64;
    for (int i = tid; i < D * 16; i += 256) {
        u16 *to = S0 + (i * 4 / D) * SP + i * 4 % D;
        if constexpr (P == 1) *reinterpret_cast<u32x2 *>(to) = *reinterpret_cast<const u32x2 *>(s0 + i * 4);
        else put4<P>(to, 64 * SP, load4(s0 + i * 4));
    }
    for (int i = tid; i < 64 * 16; i += 256) {
        u16 *to = Ut + (i / 16) * UP + i % 16 * 4;
        if constexpr (P == 1) *reinterpret_cast<u32x2 *>(to) = *reinterpret_cast<const u32x2 *>(up + i * 4);
        else put4<P>(to, 64 * UP, load4(up + i * 4));
    }
    const int tok = 16 * wave + l16;
    Op<P> q[NK];
#pragma unroll
    for (int x = 0; x < NK; ++x) q[x] = frag_g(qp + (size_t)tok * D + x * 32 + 8 * l4, tok < valid);
    const float2 bi = a.bsum[at * 64 + tok];
    const float gamma = a.gate[at * 64 + tok].gamma * a.scale;
    u16 *Pw = Pt + 16 * wave * UP;                                      // this wave's 16 rows (tokens) of P
#pragma unroll
    for (int jt = 0; jt < 4; ++jt) {
        f32x4 c = {0.f, 0.f, 0.f, 0.f};
        if (jt <= wave) {
#pragma unroll
            for (int x = 0; x < NK; ++x) mma(c, frag_g(kp + (size_t)(16 * jt + l16) * D + x * 32 + 8 * l4, 16 * jt + l16 < valid), q[x]);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int j = 16 * jt + 4 * l4 + r;
                const float2 bj = a.bsum[at * 64 + j];
                c[r] = j <= tok ? a.scale * expf((bi.x - bj.x) + (bi.y - bj.y)) * c[r] : 0.f;
            }
        }
        put4<P>(Pw + l16 * UP + 16 * jt + 4 * l4, 64 * UP, c);
    }
    __syncthreads();
    T *outp = reinterpret_cast<T *>(a.out) + ((size_t)bh * a.N + (size_t)ch * 64 + tok) * D + c0;
    Op<P> pf[2] = {frag_n<P>(Pw, 64 * UP, UP, 0, 0, lane), frag_n<P>(Pw, 64 * UP, UP, 0, 32, lane)};
#pragma unroll
    for (int ct = 0; ct < 4; ++ct) {
        f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int x = 0; x < NK; ++x) mma(o, frag_n<P>(S0, 64 * SP, SP, 16 * ct, 32 * x, lane), q[x]);
        o *= gamma;
        mma(o, frag_n<P>(Ut, 64 * UP, UP, 16 * ct, 0, lane), pf[0]);
        if (wave >= 2) mma(o, frag_n<P>(Ut, 64 * UP, UP, 16 * ct, 32, lane), pf[1]);
        if (tok < valid) store4(outp + 16 * ct + 4 * l4, o);
    }
}

// ---- launches --------------------------------------------------------------------------------------------
namespace {

hipError_t raise_lds(const void *kernel, int bytes, bool (&done)[16]) { return dyn_lds_attr_once(kernel, bytes, done); }

template <typename T, typename S, int D>
hipError_t scan(const DeltaArgs &a, hipStream_t st)
{
    constexpr int bytes = (2 * planes_of<T>() * Tile64<T, D>::PLANE + 3 * 16 * (D + 8) + 2 * 3 * 16 * 72) * sizeof(u16);
    static bool done[16];
    if (const hipError_t e = raise_lds(reinterpret_cast<const void *>(delta_scan_kernel<T, S, D>), bytes, done)) return e;
    launch_kernel((delta_scan_kernel<T, S, D>), dim3(a.B * a.H * (D / 16)), dim3(256), bytes, st, a);
    return take_launch_status();
}

template <typename T, int D>
hipError_t out(const DeltaArgs &a, hipStream_t st)
{
    constexpr int bytes = planes_of<T>() * (64 * (D + 8) + 2 * 64 * 72) * sizeof(u16);
    static bool done[16];
    if (const hipError_t e = raise_lds(reinterpret_cast<const void *>(delta_out_kernel<T, D>), bytes, done)) return e;
    launch_kernel((delta_out_kernel<T, D>), dim3(a.B * a.H * a.chunks * (D / 64)), dim3(256), bytes, st, a);
    return take_launch_status();
}

}  // namespace

hipError_t launch_delta_chunk(const DeltaArgs &a, hipStream_t st)
{
    const dim3 grid(a.B * a.H * a.chunks);
    if (a.bf16) {
        if (a.D == 128) launch_kernel((delta_chunk_kernel<u16, 128>), grid, dim3(256), 0, st, a);
        else launch_kernel((delta_chunk_kernel<u16, 64>), grid, dim3(256), 0, st, a);
    } else {
        if (a.D == 128) launch_kernel((delta_chunk_kernel<float, 128>), grid, dim3(256), 0, st, a);
        else launch_kernel((delta_chunk_kernel<float, 64>), grid, dim3(256), 0, st, a);
    }
    return take_launch_status();
}

hipError_t launch_delta_scan(const DeltaArgs &a, bool backward, hipStream_t st)
{
    if (!a.bf16) return a.D == 128 ? scan<float, float, 128>(a, st) : scan<float, float, 64>(a, st);
    if (backward) return a.D == 128 ? scan<u16, float, 128>(a, st) : scan<u16, float, 64>(a, st);
    return a.D == 128 ? scan<u16, u16, 128>(a, st) : scan<u16, u16, 64>(a, st);
}

hipError_t launch_delta_fwd(const DeltaArgs &a, hipStream_t st)
{
    if (const hipError_t e = launch_delta_chunk(a, st)) return e;
    if (const hipError_t e = launch_delta_scan(a, false, st)) return e;
    if (a.bf16) return a.D == 128 ? out<u16, 128>(a, st) : out<u16, 64>(a, st);
    return a.D == 128 ? out<float, 128>(a, st) : out<float, 64>(a, st);
}

}  // namespace salad
