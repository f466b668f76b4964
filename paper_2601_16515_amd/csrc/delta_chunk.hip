// The gated delta rule over whole sequences, in chunks of 64 tokens.  Within a chunk, with b_i the running sum of g, gamma_i = e^b_i and
// S_0 the state before it,
//   u_i = beta_i (v_i - gamma_i S_0^T k_i - sum_{j<i} e^(b_i - b_j) (k_i.k_j) u_j),
// a triangular system (I + A) U = R, A_ij = beta_i e^(b_i - b_j) k_i.k_j (j < i), R = beta (V - gamma K S_0), and
//   S_64 = gamma_63 S_0 + K^T (tail u),  tail_i = e^(b_63 - b_i),     O = scale gamma Q S_0 + P U,  P_ij = scale e^(b_i - b_j) q_i.k_j  (j <= i).
// T = (I + A)^-1 and P do not depend on the state: delta_chunk_kernel here computes them for every chunk at once.  The states go from
// chunk to chunk in delta_chain.hip.  All exponents are differences of sums held in 64 bits; T keeps fp32 (three planes), P for bf16
// tensors is rounded to bf16 (half a step of each term of O).
#include <algorithm>

#include "causal.h"
#include "delta_planes.h"

namespace salad {

// ---- T and P ------------------------------------------------------------------------------------------------
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
    const size_t row0 = ((size_t)b * a.Hk + hk) * a.N + (size_t)ch * 64;
    const T *kp = reinterpret_cast<const T *>(a.k) + row0 * D, *qp = reinterpret_cast<const T *>(a.q) + row0 * D;
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
        DeltaGate &gate = a.gate[at];
        gate.gamma[lane] = expf((float)s);
        gate.tail[lane] = lane < valid ? expf((float)(last - s)) : 0.f;
        gate.beta[lane] = beta;
        const float hi = (float)s;
        a.bsum[at * 64 + lane] = make_float2(hi, (float)(s - hi));
    }
    // A: rows 16 wave.., columns up to the diagonal.  P transposed, so that a lane has 4 neighbours of a row
    f32x4 kk[4], pp[4];
    Op<P> own[NK], ownq[NK];
    const int tok = 16 * wave + l16;
#pragma unroll
    for (int x = 0; x < NK; ++x) {
        own[x] = frag_g(kp + (size_t)min(tok, valid - 1) * D + x * 32 + 8 * l4, tok < valid);
        if (a.pf) ownq[x] = frag_g(qp + (size_t)min(tok, valid - 1) * D + x * 32 + 8 * l4, tok < valid);
    }
#pragma unroll
    for (int ct = 0; ct < 4; ++ct) {
        kk[ct] = pp[ct] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (ct <= wave)
#pragma unroll
            for (int x = 0; x < NK; ++x) {
                const Op<P> f = frag_g(kp + (size_t)min(16 * ct + l16, valid - 1) * D + x * 32 + 8 * l4, 16 * ct + l16 < valid);
                mma(kk[ct], own[x], f);
                if (a.pf) mma(pp[ct], f, ownq[x]);
            }
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
    if (!a.pf) return;
    // P through this wave's 16 rows of A, which nobody reads any more
#pragma unroll
    for (int ct = 0; ct < 4; ++ct) {
        f32x4 c;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int j = 16 * ct + 4 * l4 + r;
            c[r] = j <= tok ? a.scale * expf((float)(bd[tok] - bd[j])) * pp[ct][r] : 0.f;
        }
        *reinterpret_cast<f32x4 *>(&A[tok][16 * ct + 4 * l4]) = c;
    }
    __syncthreads();
    u16 *pf = a.pf + at * (P * 4 * 2 * 64 * 8);
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
        const int k0 = 32 * kt + 8 * l4;
        u32x2 p[P], q[P];
        split4<P>(*reinterpret_cast<const f32x4 *>(&A[tok][k0]), p);
        split4<P>(*reinterpret_cast<const f32x4 *>(&A[tok][k0 + 4]), q);
#pragma unroll
        for (int i = 0; i < P; ++i) *reinterpret_cast<u32x4 *>(pf + (((i * 4 + wave) * 2 + kt) * 64 + lane) * 8) = u32x4{p[i].x, p[i].y, q[i].x, q[i].y};
    }
}

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

}  // namespace salad
