// The gated delta rule token by token, for a few tokens:
//   u_t = beta_t (v_t - e^g_t S^T k_t),   S <- e^g_t S + k_t u_t^T,   out_t = scale S^T q_t.
// The value channels (columns of S) are independent: a workgroup takes CW of them for one (sample, head) and keeps its part of S in
// registers, 4 columns x D / groups rows a thread.  Both sums over the key channels are taken at once, since
//   S_new^T q = e^g S^T q + (q.k) u,
// so that a token costs one pass over the registers and one exchange through LDS.  Bound by reading and writing the state once
// (8 D^2 bytes a head).  Many heads: all columns in one workgroup, rows of 512 bytes, past the caches (128 samples, 40 heads, d = 128:
// 113.8 us = 5.93 TB/s; 118.2 through the caches, 122.4 with 64 columns a workgroup).  Fewer than 512 heads: 16 columns, for more workgroups.
// In a graph, whole rows and 16 columns, us: d = 128, one token 12 heads 3.8 and 3.2, 32 heads 3.9 and 4.0, 128 heads 4.6 and 8.5, 512 heads 8.6 and
// 20.7; 32 tokens 12 heads 38 and 32, 64 heads 39 and 42, 256 heads 41 and 131.  d = 64, one token 12 heads 2.8 and 2.9, 512 heads 3.9 and
// 9.9.  So 16 columns win below some 40 heads of 128 alone, by a sixth, and the bound of 512 is too far out.
#include <algorithm>

#include "causal.h"
#include "delta_planes.h"

namespace salad {

template <typename T, int D, int CW>
__global__ __launch_bounds__(256, 2) void delta_step_kernel(DeltaArgs a)
{
    constexpr int LC = CW / 4, GR = 256 / LC, RPT = D / GR;              // lanes across the columns, row groups, rows a thread
    __shared__ __attribute__((aligned(16))) float red[2][4][2][CW];     // by wave: sums of k and of q; two tokens in turn
    const int slices = D / CW;
    const int bh = blockIdx.x / slices, c0 = (blockIdx.x - bh * slices) * CW;
    const int b = bh / a.H, h = bh - b * a.H, hk = h / (a.H / a.Hk);
    const int tid = threadIdx.x, wave = tid >> 6, lc = tid % LC, gr = tid / LC, len = delta_len(a, b);
    const T *q = reinterpret_cast<const T *>(a.q) + ((size_t)b * a.Hk + hk) * a.N * D + gr * RPT;
    const T *k = reinterpret_cast<const T *>(a.k) + ((size_t)b * a.Hk + hk) * a.N * D + gr * RPT;
    const T *v = reinterpret_cast<const T *>(a.v) + (size_t)bh * a.N * D + c0 + lc * 4;
    T *out = reinterpret_cast<T *>(a.out) + (size_t)bh * a.N * D + c0 + lc * 4;
    const size_t at = ((size_t)bh * D + gr * RPT) * D + c0 + lc * 4;
    f32x4 S[RPT];
#pragma unroll
    for (int r = 0; r < RPT; ++r) {
        S[r] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (a.state_in) {
            const f32x4 *from = reinterpret_cast<const f32x4 *>(a.state_in + at + (size_t)r * D);
            S[r] = CW == D ? __builtin_nontemporal_load(from) : *from;
        }
    }
    for (int t = 0; t < len; ++t) {
        float kr[RPT], qr[RPT];
#pragma unroll
        for (int r = 0; r < RPT; ++r) { kr[r] = load1(k + (size_t)t * D + r); qr[r] = load1(q + (size_t)t * D + r); }
        const f32x4 vt = load4(v + (size_t)t * D);
        const float decay = expf(a.g[(size_t)bh * a.N + t]), beta = a.beta[(size_t)bh * a.N + t];
        f32x4 sk = {0.f, 0.f, 0.f, 0.f}, sq = sk;
        float qk = 0.f;
#pragma unroll
        for (int r = 0; r < RPT; ++r) { sk += kr[r] * S[r]; sq += qr[r] * S[r]; qk += kr[r] * qr[r]; }
        // the row groups of a wave, then the waves
#pragma unroll
        for (int m = LC; m < 64; m <<= 1) {
#pragma unroll
            for (int i = 0; i < 4; ++i) { sk[i] += __shfl_xor(sk[i], m); sq[i] += __shfl_xor(sq[i], m); }
            qk += __shfl_xor(qk, m);
        }
        float (*to)[2][CW] = red[t & 1];
        __shared__ float qks[2][4];
        if ((tid & 63) < LC) {
            *reinterpret_cast<f32x4 *>(&to[wave][0][lc * 4]) = sk;
            *reinterpret_cast<f32x4 *>(&to[wave][1][lc * 4]) = sq;
            if (lc == 0) qks[t & 1][wave] = qk;
        }
        __syncthreads();
        sk = sq = f32x4{0.f, 0.f, 0.f, 0.f};
        qk = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            sk += *reinterpret_cast<const f32x4 *>(&to[w][0][lc * 4]);
            sq += *reinterpret_cast<const f32x4 *>(&to[w][1][lc * 4]);
            qk += qks[t & 1][w];
        }
        const f32x4 u = beta * (vt - decay * sk);
#pragma unroll
        for (int r = 0; r < RPT; ++r) S[r] = decay * S[r] + kr[r] * u;
        if (gr == 0) store4(out + (size_t)t * D, a.scale * (decay * sq + qk * u));
    }
    if (a.state_out)
#pragma unroll
        for (int r = 0; r < RPT; ++r) {
            f32x4 *to = reinterpret_cast<f32x4 *>(a.state_out + at + (size_t)r * D);
            if (CW == D) __builtin_nontemporal_store(S[r], to);
            else *to = S[r];
        }
}

// Up to 32 tokens, as the interface says (what a value that is not finite may reach changes there).  Token by token and in a chunk, us: 12 heads,
// d = 128 8 tokens 10.1 and 16.4, 14 15.1 and 15.4, 32 32.0 and 16.4; 5120 heads 8 tokens 153 and 350, 24 314 and 357, 32 395 and 361;
// 64 heads, d = 64 14 tokens 14.4 and 14.3, 32 30.0 and 15.3.  They cross at 14 tokens for few heads and at 28 for many.
bool delta_takes_step(const DeltaArgs &a) { return a.N <= 32; }

template <typename T, int D>
static void launch_step(const DeltaArgs &a, hipStream_t st)
{
    const int BH = a.B * a.H;
    if (BH >= 512) launch_kernel((delta_step_kernel<T, D, D>), dim3(BH), dim3(256), 0, st, a);
    else launch_kernel((delta_step_kernel<T, D, 16>), dim3(BH * (D / 16)), dim3(256), 0, st, a);
}

hipError_t launch_delta_step(const DeltaArgs &a, hipStream_t st)
{
    if (a.bf16) { if (a.D == 128) launch_step<u16, 128>(a, st); else launch_step<u16, 64>(a, st); }
    else { if (a.D == 128) launch_step<float, 128>(a, st); else launch_step<float, 64>(a, st); }
    return take_launch_status();
}

}  // namespace salad
