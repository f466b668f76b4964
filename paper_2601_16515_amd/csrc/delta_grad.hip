// Gradients of the gated delta rule (delta_chunk.hip has the forward pass and its names).  Nothing of the forward pass is kept: T,
// the states before the chunks and U are computed again.  With dS the gradient of the state behind a chunk,
//   dU = X + tail K dS,   X = P^T dO,          dR = T^T dU,
//   gradient of the state before the chunk = gamma_63 dS + Q^T (scale gamma dO) - K^T (beta gamma dR),
// a chain from the last chunk to the first like the forward one (delta_chain.hip), and then for every chunk at once, with dA = -(dR U^T) below the diagonal
// and dP = dO U^T,
//   dv = beta dR,
//   dq = scale gamma dO S_0^T + (scale e^(b_i - b_j) dP) K,
//   dk = -beta gamma dR S_0^T + tail U dS^T + E K + E^T K + (scale e^(b_i - b_j) dP)^T Q,   E = dA beta e^(b_i - b_j),
//   dbeta_i = dR_i.v_i - gamma_i k_i.(dR S_0^T)_i + sum_j dA_ij e^(b_i - b_j) k_i.k_j,
// and by the decays b_i: each term's product with what it decays, summed over rows (+) and columns (-); dg is the running sum of that
// from the end of the chunk.  dg, dbeta and the state's gradient are fp32 results: their products keep fp32 (three planes).  The four
// 64 x 64 x D products that reach only dq and dk take E and dP in two planes for bf16 tensors: with keys of nearly one direction the terms of dq are
// 30 to 70 times their sum, and one plane left dq off by 1.1e-2, seven times its own rounding (now 1.7e-3, in 0.7 % more time of the call).
#include <algorithm>

#include "causal.h"
#include "delta_planes.h"

namespace salad {

// ---- X = P^T dO of every chunk ----------------------------------------------------------------------------
template <typename T, int D>
__global__ __launch_bounds__(256) void delta_x_kernel(DeltaArgs a)
{
    constexpr int P = planes_of<T>(), NK = D / 32, UP = 72;
    using Tile = Tile64<T, D>;
    extern __shared__ __attribute__((aligned(16))) u16 lds[];
    u16 *DO = lds, *Pt = DO + P * Tile::PLANE;                          // dO [64][D]; P transposed: [token j][later token]
    const int ch = blockIdx.x % a.chunks, bh = blockIdx.x / a.chunks, b = bh / a.H, h = bh - b * a.H, hk = h / (a.H / a.Hk);
    const int valid = min(delta_len(a, b) - ch * 64, 64);
    if (valid <= 0) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l16 = lane & 15, l4 = lane >> 4;
    const size_t at = (size_t)bh * a.chunks + ch, row0 = ((size_t)b * a.Hk + hk) * a.N + (size_t)ch * 64;
    const T *qp = reinterpret_cast<const T *>(a.q) + row0 * D, *kp = reinterpret_cast<const T *>(a.k) + row0 * D;
    Tile t;
    t.load(reinterpret_cast<const T *>(a.dout) + ((size_t)bh * a.N + (size_t)ch * 64) * D, valid, tid);
    t.store(DO, tid);
    const int tok = 16 * wave + l16;
    const float2 bi = a.bsum[at * 64 + tok];
    Op<P> k[NK];
#pragma unroll
    for (int x = 0; x < NK; ++x) k[x] = frag_g(kp + (size_t)min(tok, valid - 1) * D + x * 32 + 8 * l4, tok < valid);
#pragma unroll
    for (int it = 0; it < 4; ++it) {
        f32x4 c = {0.f, 0.f, 0.f, 0.f};
        if (it >= wave) {
#pragma unroll
            for (int x = 0; x < NK; ++x) mma(c, frag_g(qp + (size_t)min(16 * it + l16, valid - 1) * D + x * 32 + 8 * l4, 16 * it + l16 < valid), k[x]);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int i = 16 * it + 4 * l4 + r;
                const float2 bl = a.bsum[at * 64 + i];
                c[r] = i >= tok ? a.scale * expf((bl.x - bi.x) + (bl.y - bi.y)) * c[r] : 0.f;
            }
        }
        put4<3>(Pt + tok * UP + 16 * it + 4 * l4, 64 * UP, c);
    }
    __syncthreads();
    float *x = a.dr + at * D * 64;
#pragma unroll
    for (int ct = 0; ct < D / 16; ++ct) {
        f32x4 c = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
            mma(c, frag_t<P>(DO, Tile::PLANE, Tile::PITCH, 16 * ct, 32 * kt, lane), frag_n<3>(Pt, 64 * UP, UP, 16 * wave, 32 * kt, lane));
#pragma unroll
        for (int r = 0; r < 4; ++r) x[(16 * ct + 4 * l4 + r) * 64 + tok] = c[r];
    }
}

// ---- the rest, every chunk at once ----------------------------------------------------------------------------
// Transposed: a lane's column is token i = 16 wave + l % 16, rows are key channels or the other token.  The contractions over the value
// channels go in blocks of 32 through LDS, the next block on its way meanwhile.  8 waves: 4 of the tokens by 2 of the key channels; of the products
// over pairs of tokens one half takes A's, the other P's.  12 heads, N = 12480, d = 128, bf16: 333 us (321 with E and dP in one plane; 400 with 4 waves and blocks loaded
// when needed), bound by LDS: every plane of every operand is read from there by 8 waves, one workgroup to a compute unit.
template <typename T, int D>
__global__ __launch_bounds__(512, 1) void delta_grad_kernel(DeltaArgs a)
{
    constexpr int P = planes_of<T>(), EP = out_planes<T>(), NK = D / 32, NA = D / 32, SP = D + 8, UP = 72, SPL = 32 * SP, UPL = 32 * UP;
    using Tile = Tile64<T, D>;
    extern __shared__ __attribute__((aligned(16))) u16 lds[];
    u16 *S0 = lds, *S1 = S0 + 3 * SPL, *Ut = S1 + 3 * SPL, *Rt = Ut + 3 * UPL;          // [32][D], [32][D], [32][64], [32][64]
    u16 *X = lds, *Et = X + P * Tile::PLANE, *Pt = Et + EP * 64 * UP;                    // afterwards: K or Q [64][D]; E and dP [token i][token j]
    __shared__ float cols[8][64], red[8], fin[2][64], fdb[2][64];
    const int ch = blockIdx.x % a.chunks, bh = blockIdx.x / a.chunks, b = bh / a.H, h = bh - b * a.H, G = a.H / a.Hk, hk = h / G;
    const int valid = min(delta_len(a, b) - ch * 64, 64);
    if (valid <= 0) return;
    const int tid = threadIdx.x, lane = tid & 63, wave8 = __builtin_amdgcn_readfirstlane(tid >> 6), wave = wave8 & 3, half = wave8 >> 2, l16 = lane & 15, l4 = lane >> 4;
    const size_t at = (size_t)bh * a.chunks + ch, row0 = ((size_t)b * a.Hk + hk) * a.N + (size_t)ch * 64, vrow0 = (size_t)bh * a.N + (size_t)ch * 64;
    const T *qp = reinterpret_cast<const T *>(a.q) + row0 * D, *kp = reinterpret_cast<const T *>(a.k) + row0 * D;
    const T *gp = reinterpret_cast<const T *>(a.dout) + vrow0 * D, *vp = reinterpret_cast<const T *>(a.v) + vrow0 * D;
    T *dvp = reinterpret_cast<T *>(a.dv) + vrow0 * D;
    const int tok = 16 * wave + l16;
    const bool live = tok < valid;
    const int a0 = half * (D / 2);                                      // this half's key channels
    f32x4 qs[NA], ks[NA], ke[NA], pu[4];                                // pu: dR U^T, or dO U^T
#pragma unroll
    for (int x = 0; x < NA; ++x) qs[x] = ks[x] = ke[x] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int x = 0; x < 4; ++x) pu[x] = f32x4{0.f, 0.f, 0.f, 0.f};
    float sds = 0.f, rv = 0.f;                                          // S_0 . dS, dR . v
    const float beta = a.gate[at].beta[tok];
    constexpr int NS = 8 * D / 512;
    f32x4 xs[NS], ys[NS], xu, xr;
    auto load = [&](int cb) __attribute__((always_inline)) {
        const float *s0 = a.s0 + (at * D + cb * 32) * D, *s1 = a.ds1 + (at * D + cb * 32) * D;
#pragma unroll
        for (int i = 0; i < NS; ++i) { xs[i] = load4(s0 + (i * 512 + tid) * 4); ys[i] = load4(s1 + (i * 512 + tid) * 4); }
        xu = load4(a.u + (at * D + cb * 32) * 64 + tid * 4);
        xr = load4(a.dr + (at * D + cb * 32) * 64 + tid * 4);
    };
    load(0);
    for (int cb = 0; cb < D / 32; ++cb) {
        lds_barrier();
#pragma unroll
        for (int i = 0; i < NS; ++i) {
            const int e = (i * 512 + tid) * 4;
            sds += xs[i][0] * ys[i][0] + xs[i][1] * ys[i][1] + xs[i][2] * ys[i][2] + xs[i][3] * ys[i][3];
            put4<3>(S0 + (e / D) * SP + e % D, SPL, xs[i]);
            put4<3>(S1 + (e / D) * SP + e % D, SPL, ys[i]);
        }
        put4<3>(Ut + (tid / 16) * UP + tid % 16 * 4, UPL, xu);
        put4<3>(Rt + (tid / 16) * UP + tid % 16 * 4, UPL, xr);
        lds_barrier();
        load(min(cb + 1, D / 32 - 1));
        const Op<P> go = frag_g(gp + (size_t)min(tok, valid - 1) * D + cb * 32 + 8 * l4, live);
        const Op<3> ui = frag_t<3>(Ut, UPL, UP, 16 * wave, 0, lane), ri = frag_t<3>(Rt, UPL, UP, 16 * wave, 0, lane);
        if (half == 0) {        // dv = beta dR: this lane's token and 8 value channels
            const size_t at8 = (size_t)min(tok, valid - 1) * D + cb * 32 + 8 * l4;
            const f32x4 va = load4(vp + at8), vb = load4(vp + at8 + 4);
            f32x4 x, y;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x[i] = (float)ri.p[0][i] + (float)ri.p[1][i] + (float)ri.p[2][i];
                y[i] = (float)ri.p[0][i + 4] + (float)ri.p[1][i + 4] + (float)ri.p[2][i + 4];
                rv += x[i] * va[i] + y[i] * vb[i];
            }
            if (live) {
                store4(dvp + at8, x * beta);
                store4(dvp + at8 + 4, y * beta);
            }
        }
#pragma unroll
        for (int x = 0; x < NA; ++x) {
            const Op<3> f0 = frag_t<3>(S0, SPL, SP, a0 + 16 * x, 0, lane);
            mma(qs[x], f0, go);
            mma(ks[x], f0, ri);
            mma(ke[x], frag_t<3>(S1, SPL, SP, a0 + 16 * x, 0, lane), ui);
        }
#pragma unroll
        for (int x = 0; x < 4; ++x)
            if (x <= wave) {
                const Op<3> uj = frag_t<3>(Ut, UPL, UP, 16 * x, 0, lane);
                if (half == 0) mma(pu[x], uj, ri);
                else mma(pu[x], uj, go);
            }
    }
    const float gamma = a.gate[at].gamma[tok], tail = a.gate[at].tail[tok];
    const float2 bi = a.bsum[at * 64 + tok];
    Op<P> ti[NK];                                                       // the token's key, or query
#pragma unroll
    for (int x = 0; x < NK; ++x) ti[x] = frag_g((half == 0 ? kp : qp) + (size_t)min(tok, valid - 1) * D + x * 32 + 8 * l4, live);
    __syncthreads();                                                    // the blocks' tiles make room
    // pairs (i = own token, j): what A and P have to say
    float rows = 0.f, db = rv;
#pragma unroll
    for (int x = 0; x < 4; ++x) {
        f32x4 kk = {0.f, 0.f, 0.f, 0.f}, e = kk, cs = kk;
        if (x <= wave) {
#pragma unroll
            for (int y = 0; y < NK; ++y)
                mma(kk, frag_g(kp + (size_t)min(16 * x + l16, valid - 1) * D + y * 32 + 8 * l4, 16 * x + l16 < valid), ti[y]);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int j = 16 * x + 4 * l4 + r;
                const float2 bj = a.bsum[at * 64 + j];
                const float ratio = j <= tok ? expf((bi.x - bj.x) + (bi.y - bj.y)) : 0.f;
                if (half == 0) {
                    const float da = j < tok ? -pu[x][r] * ratio : 0.f;
                    e[r] = da * beta;
                    db += da * kk[r];
                } else {
                    e[r] = a.scale * ratio * pu[x][r];
                }
                cs[r] = j < tok ? e[r] * kk[r] : 0.f;                   // by the decay between j and i; none from a token to itself
                rows += cs[r];
            }
        }
        put4<EP>((half == 0 ? Et : Pt) + tok * UP + 16 * x + 4 * l4, 64 * UP, e);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            float c = cs[r];
#pragma unroll
            for (int m = 1; m < 16; m <<= 1) c += __shfl_xor(c, m);
            if (l16 == 0) cols[wave8][16 * x + 4 * l4 + r] = c;
        }
    }
    // products with the states: scales, and what reaches the decays
    float end = 0.f;
#pragma unroll
    for (int x = 0; x < NA; ++x) {
        f32x4 q4 = {0.f, 0.f, 0.f, 0.f}, k4 = q4;
        if (live) { q4 = load4(qp + (size_t)tok * D + a0 + 16 * x + 4 * l4); k4 = load4(kp + (size_t)tok * D + a0 + 16 * x + 4 * l4); }
        qs[x] *= a.scale * gamma;
        ks[x] *= -gamma;
        ke[x] *= tail;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            db += ks[x][r] * k4[r];
            rows += qs[x][r] * q4[r] + beta * ks[x][r] * k4[r];
            end += ke[x][r] * k4[r];
        }
        ks[x] = ks[x] * beta + ke[x];
    }
    rows -= end;
#pragma unroll
    for (int m = 16; m < 64; m <<= 1) { rows += __shfl_xor(rows, m); db += __shfl_xor(db, m); end += __shfl_xor(end, m); }
#pragma unroll
    for (int m = 1; m < 16; m <<= 1) end += __shfl_xor(end, m);         // over the wave's tokens
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) sds += __shfl_xor(sds, m);
    const float gend = a.gate[at].gamma[63];
    if (lane == 0) red[wave8] = end + gend * sds;
    if (l4 == 0) { fin[half][tok] = rows; fdb[half][tok] = db; }
    Tile t;
    if (tid < 256) {
        t.load(kp, valid, tid);
        t.store(X, tid);
        t.load(qp, valid, tid);
    }
    __syncthreads();
    if (wave8 == 0) {                                                   // dbeta, and dg: the sums from each token to the end of the chunk
        if (lane < valid) a.dbeta[vrow0 + lane] = fdb[0][lane] + fdb[1][lane];
        float d = fin[0][lane] + fin[1][lane];
#pragma unroll
        for (int w = 0; w < 8; ++w) {
            d -= cols[w][lane];
            if (lane == 63) d += red[w];
        }
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) {
            const float o = __shfl_down(d, m);
            if (lane + m < 64) d += o;
        }
        if (lane < valid) a.dg[vrow0 + lane] = d;
    }
    Op<EP> en[2], pn[2], et[2], pt[2];
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
        en[kt] = frag_n<EP>(Et, 64 * UP, UP, 16 * wave, 32 * kt, lane);
        pn[kt] = frag_n<EP>(Pt, 64 * UP, UP, 16 * wave, 32 * kt, lane);
        et[kt] = frag_t<EP>(Et, 64 * UP, UP, 16 * wave, 32 * kt, lane);
        pt[kt] = frag_t<EP>(Pt, 64 * UP, UP, 16 * wave, 32 * kt, lane);
    }
#pragma unroll
    for (int x = 0; x < NA; ++x)
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
            const Op<P> f = frag_t<P>(X, Tile::PLANE, Tile::PITCH, a0 + 16 * x, 32 * kt, lane);
            mma(qs[x], f, pn[kt]);
            mma(ks[x], f, en[kt]);
            mma(ks[x], f, et[kt]);
        }
    __syncthreads();
    if (tid < 256) t.store(X, tid);
    __syncthreads();
#pragma unroll
    for (int x = 0; x < NA; ++x) {
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) mma(ks[x], frag_t<P>(X, Tile::PLANE, Tile::PITCH, a0 + 16 * x, 32 * kt, lane), pt[kt]);
        if (live) {
            const size_t c = a0 + 16 * x + 4 * l4;
            if (a.dq_part) {
                store4(a.dq_part + (vrow0 + tok) * D + c, qs[x]);
                store4(a.dk_part + (vrow0 + tok) * D + c, ks[x]);
            } else {
                store4(reinterpret_cast<T *>(a.dq) + (row0 + tok) * D + c, qs[x]);
                store4(reinterpret_cast<T *>(a.dk) + (row0 + tok) * D + c, ks[x]);
            }
        }
    }
}

// heads that share queries and keys add up, in order
template <typename T>
__global__ __launch_bounds__(256) void delta_share_kernel(DeltaArgs a, long long total)
{
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x;      // four channels
    if (i >= total) return;
    const long long per = (long long)a.N * a.D / 4, bk = i / per, r = i - bk * per;
    const int b = (int)(bk / a.Hk), hk = (int)(bk - (long long)b * a.Hk), G = a.H / a.Hk;
    if ((int)(r / (a.D / 4)) >= delta_len(a, b)) return;
    f32x4 q = {0.f, 0.f, 0.f, 0.f}, k = q;
    for (int g = 0; g < G; ++g) {
        const long long from = (((long long)b * a.H + hk * G + g) * per + r) * 4;
        q += load4(a.dq_part + from);
        k += load4(a.dk_part + from);
    }
    store4(reinterpret_cast<T *>(a.dq) + i * 4, q);
    store4(reinterpret_cast<T *>(a.dk) + i * 4, k);
}

// ---- launches ------------------------------------------------------------------------------------------------
namespace {

template <typename T, int D>
hipError_t run(const DeltaArgs &a, hipStream_t st)
{
    constexpr int P = planes_of<T>(), tile = P * Tile64<T, D>::PLANE;
    constexpr int x_bytes = (tile + 3 * 64 * 72) * 2;
    constexpr int blocks = 2 * 3 * 32 * (D + 8) + 2 * 3 * 32 * 72, pairs = tile + 2 * out_planes<T>() * 64 * 72, grad_bytes = (blocks > pairs ? blocks : pairs) * 2;
    static bool dx[16], dg[16];
    if (const hipError_t e = dyn_lds_attr_once(reinterpret_cast<const void *>(delta_x_kernel<T, D>), x_bytes, dx)) return e;
    if (const hipError_t e = dyn_lds_attr_once(reinterpret_cast<const void *>(delta_grad_kernel<T, D>), grad_bytes, dg)) return e;
    const dim3 all(a.B * a.H * a.chunks);
    launch_kernel((delta_x_kernel<T, D>), all, dim3(256), x_bytes, st, a);
    if (const hipError_t e = launch_delta_chains(a, true, st)) return e;
    launch_kernel((delta_grad_kernel<T, D>), all, dim3(512), grad_bytes, st, a);
    if (a.dq_part) {
        const long long total = (long long)a.B * a.Hk * a.N * D / 4;
        launch_kernel((delta_share_kernel<T>), dim3((unsigned)((total + 255) / 256)), dim3(256), 0, st, a, total);
    }
    return take_launch_status();
}

}  // namespace

hipError_t launch_delta_bwd(const DeltaArgs &a, hipStream_t st)
{
    if (const hipError_t e = launch_delta_chunk(a, true, st)) return e;
    if (a.bf16) return a.D == 128 ? run<u16, 128>(a, st) : run<u16, 64>(a, st);
    return a.D == 128 ? run<float, 128>(a, st) : run<float, 64>(a, st);
}

}  // namespace salad
