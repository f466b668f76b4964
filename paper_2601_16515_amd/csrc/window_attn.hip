// Softmax attention over a sliding window with a few first tokens that stay visible (sinks), forward.  Causal: query n of a sample
// stands at position p = kv_len - q_len + n and sees key j <= p with j > p - window or j < sinks.
//   out = sum_j exp(s_j - m) v_j / sum_j exp(s_j - m),  s_j = scale q.k_j,  m a running reference  (one pass over the keys)
//   lse = m + log sum_j exp(s_j - m)
//
// Three kernels:
//   window_fwd_kernel    bf16, many queries: 128 or 256 queries of one head per workgroup, 64-key tiles through LDS
//   window_step_kernel   bf16, few queries against a long cache: the heads of a group and their tokens are the 32 rows of a
//                        matrix product, the keys are dealt to waves and workgroups and joined afterwards
//   window_f32_kernel    fp32
// Both bf16 kernels compute S^T = K Q^T with the keys' rows permuted (kappa) so that the accumulators of 16 keys are, packed to bf16,
// the B operand of O^T += V^T P^T as they stand: P never leaves the registers.  P is rounded to bf16 for that product (half a step,
// 2^-8 relative at most, as the result itself is rounded to bf16); maxima, sums and accumulators are fp32.
#include <algorithm>

#include "causal.h"

namespace salad {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

#define LDS_PTR(p) ((__attribute__((address_space(3))) void *)(p))
#define GLB_PTR(p) ((const __attribute__((address_space(1))) void *)(p))

namespace {

constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.69314718055994530942f;

__device__ inline uint32_t pack2(float a, float b)
{
    f32x2 x = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, bf16x2));
}

union Frag {
    bf16x8 v;
    uint4 u;
    uint32_t w[4];
    s16x4 h[2];
};

// 16-byte pieces of a row in LDS are swizzled by the row: piece c of row r lies at c ^ sigma(r).  K is read a piece per row (16
// lanes, 16 rows), V by transposing reads (4 rows x 4 pieces); both touch every bank once.
template <int D> __device__ inline int sigma_k(int r) { return D == 128 ? r & 15 : (r >> 1) & 7; }
template <int D> __device__ inline int sigma_v(int r) { return D == 128 ? (r & 3) << 2 : ((r >> 1) & 1) << 2; }
// the matrix row l holds key kappa(l) of 32: accumulator r of lane half hh is then key 16 (r / 8) + 8 hh + r % 8
__device__ inline int kappa_of(int l) { return (l & 0x13) | ((l & 4) << 1) | ((l & 8) >> 1); }

}  // namespace

// ---- many queries -----------------------------------------------------------------------------------
template <int D, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 2) void window_fwd_kernel(WindowArgs a, int ntiles, int total, int per_xcd)
{
    constexpr int NS = D / 16, NDT = D / 32, CH = D / 8, TILE = 64 * D, RPP = 64 * WAVES / CH, NP = 64 / RPP, ROWS = 32 * WAVES;
    __shared__ __attribute__((aligned(1024))) u16 Kb[2 * TILE];
    __shared__ __attribute__((aligned(1024))) u16 Vb[2 * TILE];
    // consecutive workgroups go to the 8 XCDs in turn: each gets a contiguous range, so that neighbouring tiles of a head share an L2
    const int gi = blockIdx.x;
    const int L = (gi & 7) * per_xcd + (gi >> 3);
    if (L >= total) return;
    const int bh = L / ntiles, tile = ntiles - 1 - (L - bh * ntiles);    // the last queries see most
    const int b = bh / a.H, h = bh - b * a.H, hk = h / (a.H / a.Hk);
    const WindowSpan sp = window_span(a, b);
    const int n0 = tile * ROWS;
    if (n0 >= sp.qlen) return;

    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l32 = lane & 31, hh = lane >> 5;
    const u16 *qb = reinterpret_cast<const u16 *>(a.q) + (size_t)bh * a.Nq * D;
    const u16 *kb = reinterpret_cast<const u16 *>(a.k) + ((size_t)b * a.Hk + hk) * a.Nk * D;
    const u16 *vb = reinterpret_cast<const u16 *>(a.v) + ((size_t)b * a.Hk + hk) * a.Nk * D;

    const int n = n0 + wave * 32 + l32;
    const bool live = n < sp.qlen;
    const int qrow = live ? n : sp.qlen - 1;
    const int p = sp.off + qrow;
    const int pw0 = sp.off + min(n0 + wave * 32, sp.qlen - 1), pw1 = sp.off + min(n0 + wave * 32 + 31, sp.qlen - 1);
    const int p1 = sp.off + min(n0 + ROWS - 1, sp.qlen - 1);
    const int first = window_first(a, sp.off + n0);
    const KeyTiles kt_list(a, sp.off + n0, p1, 64);

    Frag qf[NS];
#pragma unroll
    for (int s = 0; s < NS; ++s) qf[s].u = *reinterpret_cast<const uint4 *>(qb + (size_t)qrow * D + s * 16 + hh * 8);

    const int lr = tid / CH, pc = tid % CH;
    auto issue = [&](int t, int buf) {
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int r = i * RPP + lr;
            const size_t row = window_row(a, window_nearest(a, t * 64 + r, first, p1));
            __builtin_amdgcn_global_load_lds(GLB_PTR(kb + row * D + (pc ^ sigma_k<D>(r)) * 8),
                                             LDS_PTR(Kb + buf * TILE + (i * 64 * WAVES + wave * 64) * 8), 16, 0, 0);
            __builtin_amdgcn_global_load_lds(GLB_PTR(vb + row * D + (pc ^ sigma_v<D>(r)) * 8),
                                             LDS_PTR(Vb + buf * TILE + (i * 64 * WAVES + wave * 64) * 8), 16, 0, 0);
        }
    };

    const int kappa = kappa_of(l32);
    int koff[NS];
#pragma unroll
    for (int st = 0; st < NS; ++st) koff[st] = kappa * D + (((2 * st + hh) ^ sigma_k<D>(kappa)) << 3);
    const int vr = 8 * hh + ((l32 >> 2) & 3);
    int voff[NDT];
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt) {
        const int chunk = 4 * dt + 2 * (l32 >> 4) + ((l32 & 3) >> 1);
        voff[dt] = vr * D + ((chunk ^ sigma_v<D>(vr)) << 3) + 4 * (l32 & 1);
    }

    f32x16 o[NDT];
#pragma unroll
    for (int i = 0; i < NDT; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[i][r] = 0.f;
    float m_run = -1e30f, l_run = 0.f;
    const float c2 = a.scale * LOG2E;

    auto step = [&](const int i, const int buf) {
        landed_barrier();  // tile `buf` is there; buf^1 is free
        if (i + 1 < kt_list.n) issue(kt_list.tile(i + 1), buf ^ 1);
        const int j0 = kt_list.tile(i) * 64;
        if (j0 > pw1 || (j0 >= a.sinks && j0 + 63 <= pw0 - a.window)) return;          // nothing for this wave
        const u16 *Kt = Kb + buf * TILE, *Vt = Vb + buf * TILE;
        f32x16 s[2];
        {
            bf16x8 kf[2][NS];
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int st = 0; st < NS; ++st) kf[kt][st] = *reinterpret_cast<const bf16x8 *>(Kt + kt * 32 * D + koff[st]);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int r = 0; r < 16; ++r) s[kt][r] = 0.f;
#pragma unroll
            for (int st = 0; st < NS; ++st) {
                s[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[0][st], qf[st].v, s[0], 0, 0, 0);
                s[1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[1][st], qf[st].v, s[1], 0, 0, 0);
            }
        }
        if (!(j0 + 63 <= pw0 && (j0 > pw1 - a.window || j0 + 63 < a.sinks))) {         // some query of the wave does not see some key
            const int jb = j0 + hh * 8;
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (!window_sees(a, jb + kt * 32 + 16 * (r >> 3) + (r & 7), p)) s[kt][r] = -INFINITY;
        }
        float mx = s[0][0];
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[kt][r]);
        mx = fmaxf(mx, __shfl_xor(mx, 32)) * c2;
        if (__any(mx > m_run + 8.0f)) {      // the reference is raised when some query exceeds it by 2^8; P stays below that
            const float m_new = fmaxf(m_run, mx);
            const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);
            m_run = m_new;
            l_run *= alpha;
#pragma unroll
            for (int i2 = 0; i2 < NDT; ++i2)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[i2][r] *= alpha;
        }
        float psum = 0.f;
        Frag pf[4];
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int r = 0; r < 16; r += 2) {
                const float x0 = __builtin_amdgcn_exp2f(fmaf(s[kt][r], c2, -m_run));
                const float x1 = __builtin_amdgcn_exp2f(fmaf(s[kt][r + 1], c2, -m_run));
                psum += x0 + x1;
                pf[kt * 2 + (r >> 3)].w[(r & 7) >> 1] = pack2(x0, x1);
            }
        l_run += psum;
        Frag vf[2][NDT];
        auto vread = [&](int c16, Frag (&f)[NDT]) {
#pragma unroll
            for (int dt = 0; dt < NDT; ++dt) {
                const u16 *vp = Vt + c16 * 16 * D + voff[dt];
                f[dt].h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3))) *)LDS_PTR(vp));
                f[dt].h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3))) *)LDS_PTR(vp + 4 * D));
            }
        };
        vread(0, vf[0]);
        vread(1, vf[1]);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int c16 = 0; c16 < 4; ++c16) {
#pragma unroll
            for (int dt = 0; dt < NDT; ++dt)
                o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[c16 & 1][dt].v, pf[c16].v, o[dt], 0, 0, 0);
            if (c16 + 2 < 4) vread(c16 + 2, vf[c16 & 1]);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    if (kt_list.n > 0) issue(kt_list.tile(0), 0);
    for (int i = 0; i < kt_list.n; i += 2) {
        step(i, 0);
        if (i + 1 < kt_list.n) step(i + 1, 1);
    }

    const float l_tot = l_run + __shfl_xor(l_run, 32);
    const float inv_l = l_tot > 0.f ? 1.f / l_tot : l_tot == 0.f ? 0.f : l_tot;       // no visible key: zeros; NaN stays
    if (!live) return;
    u16 *outp = reinterpret_cast<u16 *>(a.out) + ((size_t)bh * a.Nq + qrow) * D;
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
        for (int g4 = 0; g4 < 4; ++g4) {
            uint2 pk;
            pk.x = pack2(o[dt][g4 * 4] * inv_l, o[dt][g4 * 4 + 1] * inv_l);
            pk.y = pack2(o[dt][g4 * 4 + 2] * inv_l, o[dt][g4 * 4 + 3] * inv_l);
            *reinterpret_cast<uint2 *>(outp + dt * 32 + 8 * g4 + 4 * hh) = pk;
        }
    if (a.lse && hh == 0) a.lse[(size_t)bh * a.Nq + qrow] = l_tot == 0.f ? -INFINITY : (m_run + __builtin_amdgcn_logf(l_tot)) * LN2;
}

template <int D, int WAVES>
static void launch_fwd(const WindowArgs &a, hipStream_t st)
{
    const int ntiles = (a.Nq + 32 * WAVES - 1) / (32 * WAVES), total = a.B * a.H * ntiles, per_xcd = (total + 7) / 8;
    launch_kernel((window_fwd_kernel<D, WAVES>), dim3(per_xcd * 8), dim3(64 * WAVES), 0, st, a, ntiles, total, per_xcd);
}

hipError_t launch_window_fwd_bf16(const WindowArgs &a, hipStream_t st)
{
    // 8 waves share a tile of K and V where that leaves two workgroups for each compute unit.  d = 128, 4 and 8 waves: 12 heads, window 6240, 1560
    // sinks, N = 32760 1501 and 1411 us, N = 16384 (768 workgroups) 701 and 686, N = 10922 (516) 458 and 469, N = 2048 49 and 59.  Short
    // windows lose by it at any size, which the rule does not ask: 48 heads, N = 8190, window 500 185 and 198, 24 heads, N = 32760, window 300 293 and
    // 330 (every wave waits at the edge tiles of 256 queries).  d = 64: 4 waves leave room for a third workgroup, and 8 are slower (24 heads,
    // N = 4095, window 1000 144 and 183; 12 heads, N = 32760, window 6240 868 and 947).
    if (a.D == 128 && (long long)a.B * a.H * ((a.Nq + 255) / 256) >= 512) launch_fwd<128, 8>(a, st);
    else if (a.D == 128) launch_fwd<128, 4>(a, st);
    else launch_fwd<64, 4>(a, st);
    return take_launch_status();
}

// ---- few queries --------------------------------------------------------------------------------------
// A workgroup takes 32 rows (row = head of the group x token) of one (sample, key head) and one share of the keys; its 4 waves take
// 32-key tiles in turn, each with a running maximum and sum of its own, and meet in LDS.  Bound by reading the cache: a key costs
// 4 D bytes and 128 D multiply-adds on 32 rows, of which the matrix cores do 2^11 per cycle.
template <int D>
__global__ __launch_bounds__(256, 2) void window_step_kernel(WindowArgs a, int row_tiles)
{
    constexpr int NS = D / 16, NDT = D / 32, CH = D / 8, TILE = 32 * D, RPP = 64 / CH, NP = 32 / RPP;
    __shared__ __attribute__((aligned(1024))) u16 stage[4][2 * TILE];   // a wave's K and V tile; afterwards its 32 x D partial result
    __shared__ float ml[4][2][32];
    const int split = blockIdx.x % a.splits, rest = blockIdx.x / a.splits;
    const int rt = rest % row_tiles, bk = rest / row_tiles, b = bk / a.Hk, hk = bk - b * a.Hk, G = a.H / a.Hk;
    const WindowSpan sp = window_span(a, b);
    if (sp.qlen == 0) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l32 = lane & 31, hh = lane >> 5;
    const int R = G * a.Nq, idx = rt * STEP_ROWS + l32, row = idx < R ? idx : R - 1;
    const int tok = row % a.Nq, h = hk * G + row / a.Nq;
    const bool live = idx < R && tok < sp.qlen;
    const int n = min(tok, sp.qlen - 1);        // the rows of a wave share the choice of a new reference: what lies behind the last has no say in it
    const u16 *kb = reinterpret_cast<const u16 *>(a.k) + (size_t)bk * a.Nk * D;
    const u16 *vb = reinterpret_cast<const u16 *>(a.v) + (size_t)bk * a.Nk * D;
    const size_t orow = ((size_t)b * a.H + h) * a.Nq + n;
    const int p = sp.off + n;

    const int first = window_first(a, sp.off);
    const KeyTiles tiles(a, sp.off, sp.kv - 1, 32);
    const int t0 = (int)((long long)tiles.n * split / a.splits), t1 = (int)((long long)tiles.n * (split + 1) / a.splits);

    Frag qf[NS];
#pragma unroll
    for (int s = 0; s < NS; ++s) qf[s].u = *reinterpret_cast<const uint4 *>(reinterpret_cast<const u16 *>(a.q) + orow * D + s * 16 + hh * 8);

    const int lr = lane / CH, pc = lane % CH;
    u32x4 kr[NP], vv[NP];
    auto load = [&](int t) {
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const size_t r = window_row(a, window_nearest(a, t * 32 + i * RPP + lr, first, sp.kv - 1));
            kr[i] = *reinterpret_cast<const u32x4 *>(kb + r * D + pc * 8);
            vv[i] = *reinterpret_cast<const u32x4 *>(vb + r * D + pc * 8);
        }
    };
    u16 *Kt = stage[wave], *Vt = stage[wave] + TILE;
    const int kappa = kappa_of(l32);
    const int vr = 8 * hh + ((l32 >> 2) & 3);
    f32x16 o[NDT];
#pragma unroll
    for (int i = 0; i < NDT; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[i][r] = 0.f;
    float m_run = -1e30f, l_run = 0.f;
    const float c2 = a.scale * LOG2E;

    int t = t0 + wave;
    if (t < t1) load(tiles.tile(t));
    for (; t < t1; t += 4) {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");          // the tile belongs to this wave: its own order is enough
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int r = i * RPP + lr;
            *reinterpret_cast<u32x4 *>(Kt + r * D + ((pc ^ sigma_k<D>(r)) << 3)) = kr[i];
            *reinterpret_cast<u32x4 *>(Vt + r * D + ((pc ^ sigma_v<D>(r)) << 3)) = vv[i];
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        const int j0 = tiles.tile(t) * 32;
        if (t + 4 < t1) load(tiles.tile(t + 4));
        f32x16 s;
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = 0.f;
#pragma unroll
        for (int st = 0; st < NS; ++st)
            s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8 *>(Kt + kappa * D + (((2 * st + hh) ^ sigma_k<D>(kappa)) << 3)),
                                                        qf[st].v, s, 0, 0, 0);
        const int jb = j0 + hh * 8;
        float mx = -INFINITY;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            if (!window_sees(a, jb + 16 * (r >> 3) + (r & 7), p)) s[r] = -INFINITY;
            mx = fmaxf(mx, s[r]);
        }
        mx = fmaxf(mx, __shfl_xor(mx, 32)) * c2;
        if (__any(mx > m_run + 8.0f)) {
            const float m_new = fmaxf(m_run, mx);
            const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);
            m_run = m_new;
            l_run *= alpha;
#pragma unroll
            for (int i = 0; i < NDT; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[i][r] *= alpha;
        }
        Frag pf[2];
#pragma unroll
        for (int r = 0; r < 16; r += 2) {
            const float x0 = __builtin_amdgcn_exp2f(fmaf(s[r], c2, -m_run)), x1 = __builtin_amdgcn_exp2f(fmaf(s[r + 1], c2, -m_run));
            l_run += x0 + x1;
            pf[r >> 3].w[(r & 7) >> 1] = pack2(x0, x1);
        }
#pragma unroll
        for (int c16 = 0; c16 < 2; ++c16)
#pragma unroll
            for (int dt = 0; dt < NDT; ++dt) {
                Frag f;
                const int chunk = 4 * dt + 2 * (l32 >> 4) + ((l32 & 3) >> 1);
                const u16 *vp = Vt + (c16 * 16 + vr) * D + ((chunk ^ sigma_v<D>(vr)) << 3) + 4 * (l32 & 1);
                f.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3))) *)LDS_PTR(vp));
                f.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3))) *)LDS_PTR(vp + 4 * D));
                o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f.v, pf[c16].v, o[dt], 0, 0, 0);
            }
    }
    // ---- the waves' results meet
    const float l_tot = l_run + __shfl_xor(l_run, 32);
    if (hh == 0) { ml[wave][0][l32] = m_run; ml[wave][1][l32] = l_tot; }
    __syncthreads();                                                    // also: every wave is done with its tiles
    float M = ml[0][0][l32], Ls = 0.f;
#pragma unroll
    for (int w = 1; w < 4; ++w) M = fmaxf(M, ml[w][0][l32]);
#pragma unroll
    for (int w = 0; w < 4; ++w) Ls += ml[w][1][l32] * __builtin_amdgcn_exp2f(ml[w][0][l32] - M);
    const float mine = __builtin_amdgcn_exp2f(m_run - M);
    float *po = reinterpret_cast<float *>(stage[wave]);                 // [D][32]
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) po[(dt * 32 + 8 * (r >> 2) + 4 * hh + (r & 3)) * 32 + l32] = o[dt][r] * mine;
    __syncthreads();
    const float *ps = reinterpret_cast<const float *>(&stage[0][0]);
    const size_t part = (size_t)rest * a.splits + split;
    const float inv = Ls > 0.f ? 1.f / Ls : Ls == 0.f ? 0.f : Ls;
    // lane pairs (l32) keep their row; the channels are dealt to the 8 groups of 32 lanes
#pragma unroll
    for (int c = 0; c < D / 8; c += 4) {
        const int ch = (wave * 2 + hh) * (D / 8) + c;
        float x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[i] = 0.f;
#pragma unroll
            for (int w = 0; w < 4; ++w) x[i] += ps[w * TILE + (ch + i) * 32 + l32];
        }
        if (a.splits == 1) {
            if (live) {
                uint2 pk;
                pk.x = pack2(x[0] * inv, x[1] * inv);
                pk.y = pack2(x[2] * inv, x[3] * inv);
                *reinterpret_cast<uint2 *>(reinterpret_cast<u16 *>(a.out) + orow * D + ch) = pk;
            }
        } else if (idx < R) {
            *reinterpret_cast<float4 *>(a.part_o + (part * STEP_ROWS + l32) * D + ch) = make_float4(x[0], x[1], x[2], x[3]);
        }
    }
    if (tid < 32) {
        if (a.splits > 1) { a.part_ml[part * 64 + l32] = M; a.part_ml[part * 64 + 32 + l32] = Ls; }
        else if (live && a.lse) a.lse[orow] = Ls == 0.f ? -INFINITY : (M + __builtin_amdgcn_logf(Ls)) * LN2;
    }
}

// joins the shares of a row: a wave per row
template <int D>
__global__ __launch_bounds__(256) void window_join_kernel(WindowArgs a, int row_tiles)
{
    const int w = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int G = a.H / a.Hk, R = G * a.Nq;
    if (w >= a.B * a.Hk * R) return;
    const int bk = w / R, row = w - bk * R, b = bk / a.Hk, hk = bk - b * a.Hk;
    const int n = row % a.Nq, h = hk * G + row / a.Nq;
    if (n >= window_span(a, b).qlen) return;
    const size_t part0 = ((size_t)bk * row_tiles + row / STEP_ROWS) * a.splits;
    const int r32 = row % STEP_ROWS;
    // a share a lane (there are at most 64): reference and sum of each, and its weight
    const int mine = min(lane, a.splits - 1);
    const float ms = lane < a.splits ? a.part_ml[(part0 + mine) * 64 + r32] : -1e30f, ls = a.part_ml[(part0 + mine) * 64 + 32 + r32];
    float M = ms;
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) M = fmaxf(M, __shfl_xor(M, m));
    const float f = lane < a.splits ? __builtin_amdgcn_exp2f(ms - M) : 0.f;
    float Ls = lane < a.splits ? f * ls : 0.f;
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) Ls += __shfl_xor(Ls, m);
    constexpr int C = D / 64;
    float x[C] = {};
    const float *po = a.part_o + (part0 * STEP_ROWS + r32) * D + lane * C;
#pragma unroll 8
    for (int s = 0; s < a.splits; ++s) {
        const float fs = __shfl(f, s);
#pragma unroll
        for (int c = 0; c < C; ++c) x[c] = fmaf(fs, po[(size_t)s * STEP_ROWS * D + c], x[c]);
    }
    const float inv = Ls > 0.f ? 1.f / Ls : Ls == 0.f ? 0.f : Ls;
    const size_t orow = ((size_t)b * a.H + h) * a.Nq + n;
    u16 *outp = reinterpret_cast<u16 *>(a.out) + orow * D + lane * C;
#pragma unroll
    for (int c = 0; c < C; ++c) outp[c] = f32_to_bf16_rne(x[c] * inv);
    if (a.lse && lane == 0) a.lse[orow] = Ls == 0.f ? -INFINITY : (M + __builtin_amdgcn_logf(Ls)) * LN2;
}

// Shares that the keys are cut into: enough workgroups for the chip, no more than about 1024 keys each (streams of one batch are of very
// different ages: 64 samples, 8 key heads, up to 4100 keys take 89.7 us in one share, 65.7 in two, 61.7 in four, 71.7 in eight), and at
// least 4 tiles, one a wave
int window_step_splits(int B, int Hk, int row_tiles, int max_keys)
{
    const long long base = (long long)B * Hk * row_tiles;
    const long long want = (512 + base - 1) / base, most = std::max(1, max_keys / 128), even = max_keys / 1024;
    return (int)std::max(1ll, std::min({std::max(want, even), most, 64ll}));
}

// Up to 16 queries a sample go with the keys in shares, more by tiles of 128 queries, each over all its keys.  Here and by tiles, us:
//   12 heads, window 6240, 1560 sinks, d = 128:             1 query 32 and 173,   16 33 and 174,    64 34 and 177
//   64 samples, 40 heads on 8, window 4096, 4 sinks:        1 query 195 and 1205, 16 355 and 1235,  64 990 and 1268
//   4 samples, 24 heads on 8, window 1000, 4 sinks, d = 64: 1 query 11 and 21,    16 13 and 23,     64 20 and 24
// So the two cross past 64 queries, and 17 to 64 would be faster here, too.
bool window_takes_step(const WindowArgs &a) { return a.Nq <= 16; }

hipError_t launch_window_step_bf16(const WindowArgs &a, hipStream_t st)
{
    const int R = a.H / a.Hk * a.Nq, row_tiles = (R + STEP_ROWS - 1) / STEP_ROWS;
    const dim3 grid((unsigned)((size_t)a.B * a.Hk * row_tiles * a.splits));
    if (a.D == 128) launch_kernel((window_step_kernel<128>), grid, dim3(256), 0, st, a, row_tiles);
    else launch_kernel((window_step_kernel<64>), grid, dim3(256), 0, st, a, row_tiles);
    if (a.splits > 1) {
        const dim3 jgrid((unsigned)(((size_t)a.B * a.Hk * R + 3) / 4));
        if (a.D == 128) launch_kernel((window_join_kernel<128>), jgrid, dim3(256), 0, st, a, row_tiles);
        else launch_kernel((window_join_kernel<64>), jgrid, dim3(256), 0, st, a, row_tiles);
    }
    return take_launch_status();
}

// ---- fp32 ---------------------------------------------------------------------------------------------
// 16 rows (head of the group x token) per workgroup; its 4 waves take 16-key tiles in turn and meet in LDS.  Products on
// v_mfma_f32_16x16x4_f32, transposed as above: lane i + 16 g belongs to row i, step 4 x + y of S^T = K Q^T takes channels
// 16 x + 4 g + y, and the accumulators of S^T are the B operands of O^T += V^T P^T (step r: key 4 g + r).
template <int D>
__global__ __launch_bounds__(256, 2) void window_f32_kernel(WindowArgs a, int row_tiles)
{
    constexpr int NX = D / 16, PITCH = D + 4, LPR = D / 4, RPI = 64 / LPR, NK = 16 / RPI;
    __shared__ __attribute__((aligned(16))) float stage[4][2][16][PITCH];
    __shared__ float msh[4][16], lsh[4][16];
    const int rt = blockIdx.x % row_tiles, bk = blockIdx.x / row_tiles, b = bk / a.Hk, hk = bk - b * a.Hk, G = a.H / a.Hk;
    const WindowSpan sp = window_span(a, b);
    if (sp.qlen == 0) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), i = lane & 15, g = lane >> 4;
    const int R = G * a.Nq, first = rt * 16, last = min(first + 15, R - 1);
    const int idx = first + i, row = idx < R ? idx : R - 1;
    const int tok = row % a.Nq, n = min(tok, sp.qlen - 1), h = hk * G + row / a.Nq;
    const bool live = idx < R && tok < sp.qlen;
    const size_t orow = ((size_t)b * a.H + h) * a.Nq + n;
    const int p = sp.off + n;
    // positions of the tile's rows: a range, or all of them where it holds rows of two heads
    const bool one = first / a.Nq == last / a.Nq;
    const int nlo = one ? first % a.Nq : 0, nhi = min(one ? last % a.Nq : a.Nq - 1, sp.qlen - 1);
    const int p1 = nhi >= nlo ? sp.off + nhi : -1;
    const int seen = window_first(a, sp.off + nlo);
    const KeyTiles tiles(a, sp.off + nlo, p1, 16);
    const float *kb = reinterpret_cast<const float *>(a.k) + (size_t)bk * a.Nk * D + (lane % LPR) * 4;
    const float *vb = reinterpret_cast<const float *>(a.v) + (size_t)bk * a.Nk * D + (lane % LPR) * 4;
    const float *qp = reinterpret_cast<const float *>(a.q) + orow * D + 4 * g;
    f32x4 qv[NX], o[NX];
#pragma unroll
    for (int x = 0; x < NX; ++x) {
        qv[x] = *reinterpret_cast<const f32x4 *>(qp + 16 * x);
        o[x] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    float m_run = -1e30f, l_run = 0.f;
    const float c2 = a.scale * LOG2E;
    for (int t = wave; t < tiles.n; t += 4) {
        const int j0 = tiles.tile(t) * 16;
        f32x4 kv[NK], vv[NK];
#pragma unroll
        for (int u = 0; u < NK; ++u) {
            const size_t r = window_row(a, window_nearest(a, j0 + u * RPI + lane / LPR, seen, p1));
            kv[u] = *reinterpret_cast<const f32x4 *>(kb + r * D);
            vv[u] = *reinterpret_cast<const f32x4 *>(vb + r * D);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int u = 0; u < NK; ++u) {
            *reinterpret_cast<f32x4 *>(&stage[wave][0][u * RPI + lane / LPR][(lane % LPR) * 4]) = kv[u];
            *reinterpret_cast<f32x4 *>(&stage[wave][1][u * RPI + lane / LPR][(lane % LPR) * 4]) = vv[u];
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int x = 0; x < NX; ++x) {
            const f32x4 kk = *reinterpret_cast<const f32x4 *>(&stage[wave][0][i][16 * x + 4 * g]);
#pragma unroll
            for (int y = 0; y < 4; ++y) s = __builtin_amdgcn_mfma_f32_16x16x4f32(kk[y], qv[x][y], s, 0, 0, 0);
        }
        float mx = -INFINITY;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            s[r] = window_sees(a, j0 + 4 * g + r, p) ? s[r] * c2 : -INFINITY;
            mx = fmaxf(mx, s[r]);
        }
        mx = fmaxf(mx, __shfl_xor(mx, 16));
        mx = fmaxf(mx, __shfl_xor(mx, 32));
        const float m_new = fmaxf(m_run, mx), alpha = exp2f(m_run - m_new);
        m_run = m_new;
        l_run *= alpha;
#pragma unroll
        for (int x = 0; x < NX; ++x) o[x] *= alpha;
#pragma unroll
        for (int r = 0; r < 4; ++r) { s[r] = exp2f(s[r] - m_run); l_run += s[r]; }
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            f32x4 vf[NX / 4];
#pragma unroll
            for (int x = 0; x < NX / 4; ++x) vf[x] = *reinterpret_cast<const f32x4 *>(&stage[wave][1][4 * g + r][i * NX + 4 * x]);
#pragma unroll
            for (int x = 0; x < NX; ++x) o[x] = __builtin_amdgcn_mfma_f32_16x16x4f32(vf[x / 4][x % 4], s[r], o[x], 0, 0, 0);
        }
    }
    l_run += __shfl_xor(l_run, 16);
    l_run += __shfl_xor(l_run, 32);
    if (g == 0) { msh[wave][i] = m_run; lsh[wave][i] = l_run; }
    __syncthreads();
    float M = msh[0][i], Ls = 0.f;
#pragma unroll
    for (int w = 1; w < 4; ++w) M = fmaxf(M, msh[w][i]);
#pragma unroll
    for (int w = 0; w < 4; ++w) Ls += lsh[w][i] * exp2f(msh[w][i] - M);
    const float mine = exp2f(m_run - M);
    float (*po)[PITCH] = stage[wave][0];                                // accumulator r of tile x is channel (4 g + r) D/16 + x
#pragma unroll
    for (int x = 0; x < NX; ++x)
#pragma unroll
        for (int r = 0; r < 4; ++r) po[i][(4 * g + r) * NX + x] = o[x][r] * mine;
    __syncthreads();
    if (!live) return;
    const float inv = Ls > 0.f ? 1.f / Ls : Ls == 0.f ? 0.f : Ls;
    float *outp = reinterpret_cast<float *>(a.out) + orow * D;
#pragma unroll
    for (int x = 0; x < NX / 4; ++x) {
        const int c = ((wave * 4 + g) * (NX / 4) + x) * 4;
        f32x4 y = {0.f, 0.f, 0.f, 0.f};
        if (c < D) {
#pragma unroll
            for (int w = 0; w < 4; ++w) y += *reinterpret_cast<const f32x4 *>(&stage[w][0][i][c]);
            *reinterpret_cast<f32x4 *>(outp + c) = y * inv;
        }
    }
    if (a.lse && tid < 16) a.lse[orow] = Ls == 0.f ? -INFINITY : (M + log2f(Ls)) * LN2;
}

hipError_t launch_window_fwd_f32(const WindowArgs &a, hipStream_t st)
{
    const int R = a.H / a.Hk * a.Nq, row_tiles = (R + 15) / 16;
    const dim3 grid((unsigned)((size_t)a.B * a.Hk * row_tiles));
    if (a.D == 128) launch_kernel((window_f32_kernel<128>), grid, dim3(256), 0, st, a, row_tiles);
    else launch_kernel((window_f32_kernel<64>), grid, dim3(256), 0, st, a, row_tiles);
    return take_launch_status();
}

// ---- new tokens into the cache --------------------------------------------------------------------------
__global__ __launch_bounds__(256) void window_append_kernel(AppendArgs a, long long total)
{
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
    if (i >= total) return;
    const int piece = (int)(i % a.pieces);
    const long long r = i / a.pieces;
    const int n = (int)(r % a.Nq);
    const long long bk = r / a.Nq;
    const int b = (int)(bk / a.Hk);
    int ql = a.q_lens ? a.q_lens[b] : a.Nq;
    ql = ql < 0 ? 0 : ql > a.Nq ? a.Nq : ql;
    const int kv = min(max(a.kv_lens[b], 0), WINDOW_MAX_POSITION), p = kv - ql + n;    // lengths are device data, as in window_span
    if (n >= ql || p < 0) return;
    int row = p;
    if (a.ring && p >= a.sinks) {
        const int R = a.Nk - a.sinks;
        if (p < kv - R) return;                                         // a later token of this call takes the row
        row = a.sinks + (int)((unsigned)(p - a.sinks) % (unsigned)R);
    }
    if (row >= a.Nk) return;
    const size_t to = ((size_t)bk * a.Nk + row) * a.pieces + piece;
    reinterpret_cast<uint4 *>(a.k)[to] = reinterpret_cast<const uint4 *>(a.k_new)[i];
    reinterpret_cast<uint4 *>(a.v)[to] = reinterpret_cast<const uint4 *>(a.v_new)[i];
}

hipError_t launch_window_append(const AppendArgs &a, hipStream_t st)
{
    const long long total = (long long)a.B * a.Hk * a.Nq * a.pieces;
    launch_kernel(window_append_kernel, dim3((unsigned)((total + 255) / 256)), dim3(256), 0, st, a, total);
    return take_launch_status();
}

}  // namespace salad
