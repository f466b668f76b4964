// The gated delta rule over whole sequences, in chunks of 64 tokens.  Within a chunk, with b_i the running sum of g, gamma_i = e^b_i and
// S_0 the state before it,
//   u_i = beta_i (v_i - gamma_i S_0^T k_i - sum_{j<i} e^(b_i - b_j) (k_i.k_j) u_j),
// a triangular system (I + A) U = R, A_ij = beta_i e^(b_i - b_j) k_i.k_j (j < i), R = beta (V - gamma K S_0), and
//   S_64 = gamma_63 S_0 + K^T (tail u),  tail_i = e^(b_63 - b_i),     O = scale gamma Q S_0 + P U,  P_ij = scale e^(b_i - b_j) q_i.k_j  (j <= i).
// T = (I + A)^-1 and P do not depend on the state: delta_chunk_kernel here computes them for every chunk at once.  The states go from
// chunk to chunk in delta_chain.hip.  All exponents are differences of sums held in 64 bits; T keeps fp32 (three planes), P for bf16
// tensors two.
// 12 heads, N = 32760, d = 128, bf16: 126 us for 406 MB of inputs and outputs, of which this kernel moves about half: the inverse's 16-token
// blocks wait for each other and for LDS, two workgroups to a compute unit.
#include <algorithm>
#include <type_traits>

#include "causal.h"
#include "delta_planes.h"

namespace salad {

// ---- T and P ------------------------------------------------------------------------------------------------
template <typename T, int D> struct ChunkLds {
    static constexpr int P = planes_of<T>(), AP = 68;
    float A[64][AP], Y[32][AP], X[64][AP];                      // A, a product on the way to its inverse, the inverse
    u16 k[P][64][D + 8];
    double bd[64];
    float beta[64];
};

// BWD: the backward pass's operands
template <typename T, int D, bool BWD>
__global__ __launch_bounds__(256, 2) void delta_chunk_kernel(DeltaArgs a)
{
    using L = ChunkLds<T, D>;
    constexpr int P = L::P, NK = D / 32, AP = L::AP, KP = D + 8;
    extern __shared__ __attribute__((aligned(16))) unsigned char lds_bytes[];
    L &lds = *reinterpret_cast<L *>(lds_bytes);
    auto &A = lds.A; auto &X = lds.X; auto &Y = lds.Y; auto &bd = lds.bd;
    const int ch = blockIdx.x % a.chunks, bh = blockIdx.x / a.chunks, b = bh / a.H, h = bh - b * a.H, hk = h / (a.H / a.Hk);
    const int valid = min(delta_len(a, b) - ch * 64, 64);
    if (valid <= 0) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15, l4 = lane >> 4;
    const size_t row0 = ((size_t)b * a.Hk + hk) * a.N + (size_t)ch * 64;
    const T *kp = reinterpret_cast<const T *>(a.k) + row0 * D, *qp = reinterpret_cast<const T *>(a.q) + row0 * D;
    const size_t at = (size_t)bh * a.chunks + ch;
    Tile64<T, D> kt64;
    kt64.load(kp, valid, tid);
    if (wave == 0) {
        const size_t t = (size_t)bh * a.N + ch * 64 + min(lane, valid - 1);
        float g = a.g[t], beta = a.beta[t];
        g = lane < valid ? g : 0.f;
        beta = lane < valid ? beta : 0.f;
        g = g < -100.f ? -100.f : g;                    // e^-100 is 0 in fp32 next to anything; -infinity would leave no differences
        double s = g;
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) {
            const double o = __shfl_up(s, m);
            if (lane >= m) s += o;
        }
        const double last = __shfl(s, 63);
        const float gamma = expf((float)s), tail = lane < valid ? expf((float)(last - s)) : 0.f, hi = (float)s;
        bd[lane] = s;
        lds.beta[lane] = beta;
        DeltaGate &gate = a.gate[at];
        gate.gamma[lane] = gamma;
        gate.tail[lane] = tail;
        gate.beta[lane] = beta;
        if (BWD) a.bsum[at * 64 + lane] = make_float2(hi, (float)(s - hi));
    }
    const int tok = 16 * wave + l16;
    Op<P> ownq[NK];
    if (!BWD)
#pragma unroll
        for (int x = 0; x < NK; ++x) ownq[x] = frag_g(qp + (size_t)min(tok, valid - 1) * D + x * 32 + 8 * l4, tok < valid);
    kt64.store(&lds.k[0][0][0], tid);
    __syncthreads();
    // A: rows 16 wave.., columns up to the diagonal.  P transposed, so that a lane has 4 neighbours of a row
    f32x4 kk[4], pp[4];
    {
        Op<P> own[NK];
#pragma unroll
        for (int x = 0; x < NK; ++x) own[x] = frag_n<P>(&lds.k[0][0][0], 64 * KP, KP, 16 * wave, 32 * x, lane);
#pragma unroll
        for (int ct = 0; ct < 4; ++ct) {
            kk[ct] = pp[ct] = f32x4{0.f, 0.f, 0.f, 0.f};
            if (ct <= wave)
#pragma unroll
                for (int x = 0; x < NK; ++x) {
                    const Op<P> f = frag_n<P>(&lds.k[0][0][0], 64 * KP, KP, 16 * ct, 32 * x, lane);
                    mma(kk[ct], own[x], f);
                    if (!BWD) mma(pp[ct], f, ownq[x]);
                }
        }
    }
#pragma unroll
    for (int ct = 0; ct < 4; ++ct) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int i = 16 * wave + 4 * l4 + r, j = 16 * ct + l16;
            A[i][j] = j < i ? lds.beta[i] * expf((float)(bd[i] - bd[j])) * kk[ct][r] : 0.f;
            X[i][j] = 0.f;
            if (!BWD) {
                const int l = 16 * ct + 4 * l4 + r;
                pp[ct][r] = l <= tok ? a.scale * expf((float)(bd[tok] - bd[l])) * pp[ct][r] : 0.f;
            }
        }
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
    // as operands: row tile = wave, the tokens of the contraction in the order of accumulators
    auto out = [&](auto planes, u16 *to, int piece, const f32x4 &x, const f32x4 &y) {
        constexpr int N = decltype(planes)::value;
        const Op<N> o = op_of<N>(x, y);
#pragma unroll
        for (int i = 0; i < N; ++i) *reinterpret_cast<bf16x8 *>(to + i * TRI + (piece * 64 + lane) * 8) = o.p[i];
    };
    const std::integral_constant<int, 3> three;
    u16 *tf = a.tf + at * (3 * TRI);
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
        const int j = 32 * kt + 4 * l4;
        if (kt == 0 || wave >= 2) out(three, tf, tri_lower(wave, kt), load4(&X[tok][j]), load4(&X[tok][j + 16]));
        if (BWD && (kt == 1 || wave < 2))
            out(three, a.ttf + at * (3 * TRI), tri_upper(wave, kt), f32x4{X[j][tok], X[j + 1][tok], X[j + 2][tok], X[j + 3][tok]},
                f32x4{X[j + 16][tok], X[j + 17][tok], X[j + 18][tok], X[j + 19][tok]});
        if (!BWD && (kt == 0 || wave >= 2))
            out(std::integral_constant<int, out_planes<T>()>(), a.pf + at * (out_planes<T>() * TRI), tri_lower(wave, kt), pp[2 * kt], pp[2 * kt + 1]);
    }
}

template <typename T, int D, bool BWD>
static hipError_t chunk(const DeltaArgs &a, hipStream_t st)
{
    static bool done[16];
    if (const hipError_t e = dyn_lds_attr_once(reinterpret_cast<const void *>(delta_chunk_kernel<T, D, BWD>), sizeof(ChunkLds<T, D>), done)) return e;
    launch_kernel((delta_chunk_kernel<T, D, BWD>), dim3(a.B * a.H * a.chunks), dim3(256), sizeof(ChunkLds<T, D>), st, a);
    return take_launch_status();
}

hipError_t launch_delta_chunk(const DeltaArgs &a, bool backward, hipStream_t st)
{
    if (a.bf16) {
        if (backward) return a.D == 128 ? chunk<u16, 128, true>(a, st) : chunk<u16, 64, true>(a, st);
        return a.D == 128 ? chunk<u16, 128, false>(a, st) : chunk<u16, 64, false>(a, st);
    }
    if (backward) return a.D == 128 ? chunk<float, 128, true>(a, st) : chunk<float, 64, true>(a, st);
    return a.D == 128 ? chunk<float, 128, false>(a, st) : chunk<float, 64, false>(a, st);
}

}  // namespace salad
