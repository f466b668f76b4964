// Gradients of window attention (window_attn.hip has the forward pass and the mask).  With P = exp(s - lse), s = scale q.k,
//   delta_i = dout_i . out_i,   dP = dout V^T,   dS = P (dP - delta),
//   dV = P^T dout,   dQ = scale dS K,   dK = scale dS^T Q;
// dK and dV sum over the query heads of a group.  P is computed again from lse, nothing of the forward pass but out and lse is read.
//
// One kernel serves both directions.  A workgroup owns 128 rows (KEYS: keys, else queries), a wave 32 of them, and streams the other
// side's rows through LDS in tiles of 64.  Both products
//   s = Y1 X1^T,  dP = Y2 X2^T      (queries own: X = (q, dout), Y = (k, v);   keys own: X = (k, v), Y = (q, dout))
// have the own row in the lane, so that P and dS, packed to bf16, are the B operand of
//   acc1^T += Y1^T dS,  acc2^T += Y2^T P      (dq;   dk and dv)
// without leaving the registers.  Each own row's sum runs over the streamed rows in order: no atomics, the same bits every time.
// P and dS are rounded to bf16 for the products (half a step, 2^-8 at most, as the results are); sums and accumulators are fp32.
// 12 heads, N = 12480, d = 128, by the trace: keys 1333 us, queries 720 us (fastest 1246, 679).  The keys' workgroup reads each streamed tile
// from LDS as often as the matrix cores need its products, so both take the same time, and its accumulators leave one wave to a SIMD to
// overlap them.
#include <algorithm>
#include <type_traits>

#include "causal.h"

namespace salad {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

#define LDS_PTR(p) ((__attribute__((address_space(3))) void *)(p))
#define GLB_PTR(p) ((const __attribute__((address_space(1))) void *)(p))

namespace {

constexpr float LOG2E = 1.44269504088896340736f;

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
// Tiles are read both ways, a 16-byte piece of 16 rows at a time and 4 rows x 4 pieces at a time (transposing): this order of a row's
// pieces touches every bank once in either.
template <int D> __device__ inline int sigma(int r) { return D == 128 ? ((r & 3) << 2) | ((r >> 2) & 3) : (((r >> 1) & 1) << 2) | ((r >> 2) & 3); }
__device__ inline int kappa_of(int l) { return (l & 0x13) | ((l & 4) << 1) | ((l & 8) >> 1); }

// The streamed rows of an own tile, in tiles of `size`: keys for queries at p0..p1, or the queries of all heads of the group for
// keys j0..j1, of which this workgroup takes piece `piece` of `pieces`.  Of a tile's rows only those are loaded that some own row sees, or is
// seen by (rows lo..hi, and the sinks): what is not finite in others would outlast their P = 0.
struct Stream {
    KeyTiles keys;
    int lo, hi, first, per_head, t0, n;
    __device__ Stream(const WindowArgs &a, const WindowSpan &sp, int p0, int p1, int size)
        : keys(a, p0, p1, size), lo(window_first(a, p0)), hi(p1), first(0), per_head(0), t0(0), n(keys.n) {}
    __device__ Stream(const WindowArgs &a, const WindowSpan &sp, int j0, int j1, int size, int piece, int pieces) : keys(a, 0, -1, size)
    {
        const long long last_p = j0 < a.sinks ? (long long)sp.kv - 1 : min((long long)sp.kv - 1, (long long)j1 + a.window - 1);
        lo = max(0, j0 - sp.off);
        hi = (int)min((long long)sp.qlen - 1, last_p - sp.off);
        first = lo / size;
        per_head = hi >= lo ? hi / size - first + 1 : 0;
        const long long all = (long long)per_head * (a.H / a.Hk);
        t0 = (int)(all * piece / pieces);
        n = (int)(all * (piece + 1) / pieces) - t0;
    }
};

}  // namespace

// ---- delta = sum of dout * out over a row --------------------------------------------------------------
template <typename T, int D>
__global__ __launch_bounds__(256) void window_delta_kernel(WindowArgs a, long long rows)
{
    constexpr int LPR = 16, PER = D / LPR;
    const long long r = (long long)blockIdx.x * (256 / LPR) + threadIdx.x / LPR;
    const int l = threadIdx.x % LPR;
    float s = 0.f;
    const bool live = r < rows && (int)(r % a.Nq) < window_span(a, (int)(r / a.Nq / a.H)).qlen;     // rows behind a sample's last may hold anything
    if (live) {
        const T *o = reinterpret_cast<const T *>(a.out) + r * D + l * PER, *d = reinterpret_cast<const T *>(a.dout) + r * D + l * PER;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            if constexpr (sizeof(T) == 2) s = fmaf(__uint_as_float((uint32_t)o[i] << 16), __uint_as_float((uint32_t)d[i] << 16), s);
            else s = fmaf(o[i], d[i], s);
        }
    }
#pragma unroll
    for (int m = 1; m < LPR; m <<= 1) s += __shfl_xor(s, m);
    if (r < rows && l == 0) a.delta[r] = s;
}

// ---- bf16 -------------------------------------------------------------------------------------------------
template <int D, bool KEYS>
__global__ __launch_bounds__(256, KEYS ? 1 : 2) void window_grad_kernel(WindowArgs a, int ntiles, int total, int per_xcd)
{
    constexpr int NS = D / 16, NDT = D / 32, CH = D / 8, TILE = 64 * D, RPP = 256 / CH, NP = 64 / RPP;
    __shared__ __attribute__((aligned(1024))) u16 Yb[2][2 * TILE];
    __shared__ float rowv[2][2][64];                                    // KEYS: lse and delta of the streamed queries
    const int gi = blockIdx.x;
    const int L = (gi & 7) * per_xcd + (gi >> 3);
    if (L >= total) return;
    // queries own: [B H][tiles], the last first; keys own: [B Hk][work items], the pieces of the tiles with sinks first
    const int outer = L / ntiles, item = L - outer * ntiles;
    const int heads = KEYS ? a.Hk : a.H, b = outer / heads, hx = outer - b * heads, G = a.H / a.Hk, hk = KEYS ? hx : hx / G;
    const int sink_items = KEYS ? window_sink_tiles_of(a) * a.sink_pieces : 0;
    const int tile = !KEYS ? ntiles - 1 - item : item < sink_items ? item / a.sink_pieces : item - sink_items + window_sink_tiles_of(a);
    const int piece = KEYS && item < sink_items ? item % a.sink_pieces : 0, pieces = KEYS && item < sink_items ? a.sink_pieces : 1;
    const WindowSpan sp = window_span(a, b);
    const int r0 = tile * 128, own_rows = KEYS ? sp.kv : sp.qlen;
    if (r0 >= own_rows) return;

    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l32 = lane & 31, hh = lane >> 5;
    const size_t qhead = (size_t)(b * a.H + (KEYS ? hk * G : hx)), khead = (size_t)b * a.Hk + hk;
    const u16 *Q = reinterpret_cast<const u16 *>(a.q) + qhead * a.Nq * D, *DO = reinterpret_cast<const u16 *>(a.dout) + qhead * a.Nq * D;
    const u16 *K = reinterpret_cast<const u16 *>(a.k) + khead * a.Nk * D, *V = reinterpret_cast<const u16 *>(a.v) + khead * a.Nk * D;
    const float *lse = a.lse + qhead * a.Nq, *delta = a.delta + qhead * a.Nq;
    const u16 *X1 = KEYS ? K : Q, *X2 = KEYS ? V : DO, *Y1 = KEYS ? Q : K, *Y2 = KEYS ? DO : V;

    const int r = r0 + wave * 32 + l32;
    const bool live = r < own_rows;
    const int row = live ? r : own_rows - 1;
    const int base = KEYS ? 0 : sp.off;                                 // own position = base + row
    const int pos = base + row;
    const int w0 = base + min(r0 + wave * 32, own_rows - 1), w1 = base + min(r0 + wave * 32 + 31, own_rows - 1);
    const int t1 = base + min(r0 + 127, own_rows - 1);
    const Stream str = KEYS ? Stream(a, sp, r0, t1, 64, piece, pieces) : Stream(a, sp, base + r0, t1, 64);

    Frag x1[NS], x2[NS];
#pragma unroll
    for (int s = 0; s < NS; ++s) {
        x1[s].u = *reinterpret_cast<const uint4 *>(X1 + (size_t)row * D + s * 16 + hh * 8);
        x2[s].u = *reinterpret_cast<const uint4 *>(X2 + (size_t)row * D + s * 16 + hh * 8);
    }
    float own_lse = 0.f, own_delta = 0.f;
    if (!KEYS) { own_lse = lse[row] * LOG2E; own_delta = delta[row]; }

    const int lr = tid / CH, pc = tid % CH;
    // first row of streamed tile i within Y1, Y2, and its head in the group
    auto where = [&](int i, int &head, int &y0) {
        if (KEYS) { const int t = str.t0 + i; head = t / str.per_head; y0 = (str.first + t - head * str.per_head) * 64; }
        else { head = 0; y0 = str.keys.tile(i) * 64; }
    };
    auto nearest = [&](int y) { return KEYS ? min(max(y, str.lo), str.hi) : window_nearest(a, y, str.lo, str.hi); };
    auto issue = [&](int i, int buf) {
        int head, y0;
        where(i, head, y0);
        const size_t hoff = (size_t)head * a.Nq;
#pragma unroll
        for (int u = 0; u < NP; ++u) {
            const int rr = u * RPP + lr;
            const size_t off = (hoff + nearest(y0 + rr)) * D + (pc ^ sigma<D>(rr)) * 8;
            __builtin_amdgcn_global_load_lds(GLB_PTR(Y1 + off), LDS_PTR(Yb[buf] + (u * 256 + wave * 64) * 8), 16, 0, 0);
            __builtin_amdgcn_global_load_lds(GLB_PTR(Y2 + off), LDS_PTR(Yb[buf] + TILE + (u * 256 + wave * 64) * 8), 16, 0, 0);
        }
        if (KEYS && wave < 2)
            __builtin_amdgcn_global_load_lds(GLB_PTR((wave ? delta : lse) + hoff + nearest(y0 + lane)), LDS_PTR(&rowv[buf][wave][0]), 4, 0, 0);
    };

    const int kappa = kappa_of(l32), vr = 8 * hh + ((l32 >> 2) & 3);
    f32x16 acc1[NDT], acc2[KEYS ? NDT : 1];
#pragma unroll
    for (int i = 0; i < NDT; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) { acc1[i][e] = 0.f; if (KEYS) acc2[i][e] = 0.f; }
    const float c2 = a.scale * LOG2E;

    // The products of one streamed tile; full: every pair is visible.  Where keys own, with registers for it, that is a stretch of code of its
    // own without branches, whose matrix products, exponentials and LDS reads can be put side by side.
    auto products = [&](auto full, const int y0, const int buf) __attribute__((always_inline)) {
        const u16 *T1 = Yb[buf], *T2 = Yb[buf] + TILE;
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
            f32x16 s, dp;
#pragma unroll
            for (int e = 0; e < 16; ++e) { s[e] = 0.f; dp[e] = 0.f; }
            bf16x8 y1[NS], y2[NS];
#pragma unroll
            for (int st = 0; st < NS; ++st) {
                const int off = (kt * 32 + kappa) * D + (((2 * st + hh) ^ sigma<D>(kappa)) << 3);
                y1[st] = *reinterpret_cast<const bf16x8 *>(T1 + off);
                y2[st] = *reinterpret_cast<const bf16x8 *>(T2 + off);
            }
            if (KEYS) __builtin_amdgcn_sched_barrier(0);        // all requested ahead of the first product (1392 -> 1330 us at 12 heads, N = 12480)
#pragma unroll
            for (int st = 0; st < NS; ++st) {
                s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(y1[st], x1[st].v, s, 0, 0, 0);
                dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(y2[st], x2[st].v, dp, 0, 0, 0);
            }
            Frag pf[2], sf[2];
#pragma unroll
            for (int e = 0; e < 16; e += 2) {
                float pp[2], ds[2];
#pragma unroll
                for (int f = 0; f < 2; ++f) {
                    const int yr = kt * 32 + 16 * ((e + f) >> 3) + 8 * hh + ((e + f) & 7);
                    const float ls = KEYS ? rowv[buf][0][yr] * LOG2E : own_lse, dl = KEYS ? rowv[buf][1][yr] : own_delta;
                    float x = __builtin_amdgcn_exp2f(fmaf(s[e + f], c2, -ls));
                    float y = x * (dp[e + f] - dl);
                    if (!full) {
                        const bool see = KEYS ? y0 + yr <= str.hi && window_sees(a, pos, (KEYS ? sp.off : 0) + y0 + yr) : window_sees(a, y0 + yr, pos);
                        x = see ? x : 0.f;
                        y = see ? y : 0.f;
                    }
                    pp[f] = x;
                    ds[f] = y;
                }
                if (KEYS) pf[e >> 3].w[(e & 7) >> 1] = pack2(pp[0], pp[1]);
                sf[e >> 3].w[(e & 7) >> 1] = pack2(ds[0], ds[1]);
            }
#pragma unroll
            for (int c16 = 0; c16 < 2; ++c16)
#pragma unroll
                for (int dt = 0; dt < NDT; ++dt) {
                    const int chunk = 4 * dt + 2 * (l32 >> 4) + ((l32 & 3) >> 1);
                    const int ra = kt * 32 + c16 * 16 + vr, rb = ra + 4;
                    const int oa = ra * D + ((chunk ^ sigma<D>(ra)) << 3) + 4 * (l32 & 1), ob = rb * D + ((chunk ^ sigma<D>(rb)) << 3) + 4 * (l32 & 1);
                    Frag f;
                    f.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3))) *)LDS_PTR(T1 + oa));
                    f.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3))) *)LDS_PTR(T1 + ob));
                    acc1[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f.v, sf[c16].v, acc1[dt], 0, 0, 0);
                    if (KEYS) {
                        Frag f2;
                        f2.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3))) *)LDS_PTR(T2 + oa));
                        f2.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3))) *)LDS_PTR(T2 + ob));
                        acc2[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f2.v, pf[c16].v, acc2[dt], 0, 0, 0);
                    }
                }
        }
    };
    auto step = [&](const int i, const int buf) {
        landed_barrier();
        if (i + 1 < str.n) issue(i + 1, buf ^ 1);
        int head, y0;
        where(i, head, y0);
        // positions of the streamed rows y0..y0+63, and whether all, or none, of the wave's pairs are visible
        const int ybase = KEYS ? sp.off : 0, ya = ybase + y0, yb = KEYS ? ybase + min(y0 + 63, str.hi) : y0 + 63;
        const int pa = KEYS ? ya : w0, pb = KEYS ? yb : w1, ja = KEYS ? w0 : ya, jb = KEYS ? w1 : yb;      // queries pa..pb, keys ja..jb
        if (ja > pb || (ja >= a.sinks && jb <= pa - a.window)) return;
        const bool full = jb <= pa && (ja > pb - a.window || jb < a.sinks) && (!KEYS || y0 + 63 <= str.hi);
        if constexpr (!KEYS) products(full, y0, buf);
        else if (full) products(std::true_type(), y0, buf);
        else products(std::false_type(), y0, buf);
    };
    if (str.n > 0) issue(0, 0);
    if constexpr (KEYS) {
        for (int i = 0; i < str.n; ++i) step(i, i & 1);
    } else {
        for (int i = 0; i < str.n; i += 2) {
            step(i, 0);
            if (i + 1 < str.n) step(i + 1, 1);
        }
    }
    if (KEYS && pieces > 1) {       // a piece's sums: joined afterwards, in order
        float *part = a.sink_part + ((((size_t)outer * window_sink_tiles_of(a) + tile) * pieces + piece) * 2 * 128 + wave * 32 + l32) * D;
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
            for (int g4 = 0; g4 < 4; ++g4) {
                float *to = part + dt * 32 + 8 * g4 + 4 * hh;
                *reinterpret_cast<float4 *>(to) = make_float4(acc1[dt][g4 * 4], acc1[dt][g4 * 4 + 1], acc1[dt][g4 * 4 + 2], acc1[dt][g4 * 4 + 3]);
                *reinterpret_cast<float4 *>(to + 128 * D) = make_float4(acc2[KEYS ? dt : 0][g4 * 4], acc2[KEYS ? dt : 0][g4 * 4 + 1],
                                                                        acc2[KEYS ? dt : 0][g4 * 4 + 2], acc2[KEYS ? dt : 0][g4 * 4 + 3]);
            }
        return;
    }
    if (!live) return;
    u16 *o1 = (KEYS ? reinterpret_cast<u16 *>(a.dk) + khead * a.Nk * D : reinterpret_cast<u16 *>(a.dq) + qhead * a.Nq * D) + (size_t)row * D;
    u16 *o2 = KEYS ? reinterpret_cast<u16 *>(a.dv) + (khead * a.Nk + row) * D : nullptr;
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
        for (int g4 = 0; g4 < 4; ++g4) {
            const int col = dt * 32 + 8 * g4 + 4 * hh;
            uint2 pk;
            pk.x = pack2(acc1[dt][g4 * 4] * a.scale, acc1[dt][g4 * 4 + 1] * a.scale);
            pk.y = pack2(acc1[dt][g4 * 4 + 2] * a.scale, acc1[dt][g4 * 4 + 3] * a.scale);
            *reinterpret_cast<uint2 *>(o1 + col) = pk;
            if (KEYS) {
                pk.x = pack2(acc2[KEYS ? dt : 0][g4 * 4], acc2[KEYS ? dt : 0][g4 * 4 + 1]);
                pk.y = pack2(acc2[KEYS ? dt : 0][g4 * 4 + 2], acc2[KEYS ? dt : 0][g4 * 4 + 3]);
                *reinterpret_cast<uint2 *>(o2 + col) = pk;
            }
        }
}

// ---- pieces of the keys with sinks: summed in order -----------------------------------------------------
template <int D>
__global__ __launch_bounds__(256) void window_sink_join_kernel(WindowArgs a, int sink_tiles)
{
    constexpr int PER = D / 4, RPW = 256 / PER;
    const int row = (blockIdx.x % (128 / RPW)) * RPW + threadIdx.x / PER, c = threadIdx.x % PER * 4;
    const int rest = blockIdx.x / (128 / RPW), which = rest & 1, ot = rest >> 1, tile = ot % sink_tiles, outer = ot / sink_tiles;
    const WindowSpan sp = window_span(a, outer / a.Hk);
    const int j = tile * 128 + row;
    if (j >= sp.kv) return;
    const float *part = a.sink_part + ((size_t)ot * a.sink_pieces * 2 + which) * 128 * D + (size_t)row * D + c;
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
    for (int i = 0; i < a.sink_pieces; ++i) s += *reinterpret_cast<const f32x4 *>(part + (size_t)i * 2 * 128 * D);
    const float f = which ? 1.f : a.scale;
    uint2 pk;
    pk.x = pack2(s[0] * f, s[1] * f);
    pk.y = pack2(s[2] * f, s[3] * f);
    *reinterpret_cast<uint2 *>(reinterpret_cast<u16 *>(which ? a.dv : a.dk) + ((size_t)outer * a.Nk + j) * D + c) = pk;
}

// ---- fp32 --------------------------------------------------------------------------------------------------
// As above with 16 own rows a workgroup; its 4 waves take 16-row tiles of the streamed side in turn and meet in LDS.  Products on
// v_mfma_f32_16x16x4_f32 (lane i + 16 g: own row i; step 4 x + y takes channels 16 x + 4 g + y).
template <int D, bool KEYS>
__global__ __launch_bounds__(256, 2) void window_grad_f32_kernel(WindowArgs a, int ntiles)
{
    constexpr int NX = D / 16, PITCH = D + 4, LPR = D / 4, RPI = 64 / LPR, NK = 16 / RPI;
    __shared__ __attribute__((aligned(16))) float stage[4][2][16][PITCH];
    const int outer = blockIdx.x / ntiles, tile = blockIdx.x - outer * ntiles;
    const int heads = KEYS ? a.Hk : a.H, b = outer / heads, hx = outer - b * heads, G = a.H / a.Hk, hk = KEYS ? hx : hx / G;
    const WindowSpan sp = window_span(a, b);
    const int r0 = tile * 16, own_rows = KEYS ? sp.kv : sp.qlen;
    if (r0 >= own_rows) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), i = lane & 15, g = lane >> 4;
    const size_t qhead = (size_t)(b * a.H + (KEYS ? hk * G : hx)), khead = (size_t)b * a.Hk + hk;
    const float *Q = reinterpret_cast<const float *>(a.q) + qhead * a.Nq * D, *DO = reinterpret_cast<const float *>(a.dout) + qhead * a.Nq * D;
    const float *K = reinterpret_cast<const float *>(a.k) + khead * a.Nk * D, *V = reinterpret_cast<const float *>(a.v) + khead * a.Nk * D;
    const float *lse = a.lse + qhead * a.Nq, *delta = a.delta + qhead * a.Nq;
    const float *X1 = KEYS ? K : Q, *X2 = KEYS ? V : DO, *Y1 = KEYS ? Q : K, *Y2 = KEYS ? DO : V;
    const int r = r0 + i;
    const bool live = r < own_rows;
    const int row = live ? r : own_rows - 1, base = KEYS ? 0 : sp.off, pos = base + row, t1 = base + min(r0 + 15, own_rows - 1);
    const Stream str = KEYS ? Stream(a, sp, r0, t1, 16, 0, 1) : Stream(a, sp, base + r0, t1, 16);
    auto nearest = [&](int y) { return KEYS ? min(max(y, str.lo), str.hi) : window_nearest(a, y, str.lo, str.hi); };
    f32x4 x1[NX], x2[NX], acc1[NX], acc2[NX];
#pragma unroll
    for (int x = 0; x < NX; ++x) {
        x1[x] = *reinterpret_cast<const f32x4 *>(X1 + (size_t)row * D + 16 * x + 4 * g);
        x2[x] = *reinterpret_cast<const f32x4 *>(X2 + (size_t)row * D + 16 * x + 4 * g);
        acc1[x] = acc2[x] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const float own_lse = KEYS ? 0.f : lse[row] * LOG2E, own_delta = KEYS ? 0.f : delta[row], c2 = a.scale * LOG2E;
    for (int t = wave; t < str.n; t += 4) {
        int head = 0, y0;
        if (KEYS) { const int u = str.t0 + t; head = u / str.per_head; y0 = (str.first + u - head * str.per_head) * 16; }
        else y0 = str.keys.tile(t) * 16;
        const size_t hoff = (size_t)head * a.Nq;
        f32x4 v1[NK], v2[NK];
#pragma unroll
        for (int u = 0; u < NK; ++u) {
            const size_t off = (hoff + nearest(y0 + u * RPI + lane / LPR)) * D + (lane % LPR) * 4;
            v1[u] = *reinterpret_cast<const f32x4 *>(Y1 + off);
            v2[u] = *reinterpret_cast<const f32x4 *>(Y2 + off);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int u = 0; u < NK; ++u) {
            *reinterpret_cast<f32x4 *>(&stage[wave][0][u * RPI + lane / LPR][(lane % LPR) * 4]) = v1[u];
            *reinterpret_cast<f32x4 *>(&stage[wave][1][u * RPI + lane / LPR][(lane % LPR) * 4]) = v2[u];
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        f32x4 s = {0.f, 0.f, 0.f, 0.f}, dp = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int x = 0; x < NX; ++x) {
            const f32x4 y1 = *reinterpret_cast<const f32x4 *>(&stage[wave][0][i][16 * x + 4 * g]);
            const f32x4 y2 = *reinterpret_cast<const f32x4 *>(&stage[wave][1][i][16 * x + 4 * g]);
#pragma unroll
            for (int y = 0; y < 4; ++y) {
                s = __builtin_amdgcn_mfma_f32_16x16x4f32(y1[y], x1[x][y], s, 0, 0, 0);
                dp = __builtin_amdgcn_mfma_f32_16x16x4f32(y2[y], x2[x][y], dp, 0, 0, 0);
            }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int yr = y0 + 4 * g + e, yc = nearest(yr);
            const float ls = KEYS ? lse[hoff + yc] * LOG2E : own_lse, dl = KEYS ? delta[hoff + yc] : own_delta;
            const bool see = KEYS ? yr <= str.hi && window_sees(a, pos, sp.off + yr) : window_sees(a, yr, pos);
            const float x = exp2f(fmaf(s[e], c2, -ls));
            s[e] = see ? x : 0.f;
            dp[e] = see ? x * (dp[e] - dl) : 0.f;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
#pragma unroll
            for (int x = 0; x < NX / 4; ++x) {
                const f32x4 y1 = *reinterpret_cast<const f32x4 *>(&stage[wave][0][4 * g + e][i * NX + 4 * x]);
                const f32x4 y2 = *reinterpret_cast<const f32x4 *>(&stage[wave][1][4 * g + e][i * NX + 4 * x]);
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                    acc1[4 * x + y] = __builtin_amdgcn_mfma_f32_16x16x4f32(y1[y], dp[e], acc1[4 * x + y], 0, 0, 0);
                    if (KEYS) acc2[4 * x + y] = __builtin_amdgcn_mfma_f32_16x16x4f32(y2[y], s[e], acc2[4 * x + y], 0, 0, 0);
                }
            }
        }
    }
    __syncthreads();
#pragma unroll
    for (int x = 0; x < NX; ++x)                                        // accumulator e of tile x is channel (4 g + e) D/16 + x
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            stage[wave][0][i][(4 * g + e) * NX + x] = acc1[x][e];
            if (KEYS) stage[wave][1][i][(4 * g + e) * NX + x] = acc2[x][e];
        }
    __syncthreads();
    if (!live) return;
    float *o1 = (KEYS ? reinterpret_cast<float *>(a.dk) + khead * a.Nk * D : reinterpret_cast<float *>(a.dq) + qhead * a.Nq * D) + (size_t)row * D;
    float *o2 = KEYS ? reinterpret_cast<float *>(a.dv) + (khead * a.Nk + row) * D : nullptr;
#pragma unroll
    for (int x = 0; x < NX / 4; ++x) {
        const int c = ((wave * 4 + g) * (NX / 4) + x) * 4;
        f32x4 y1 = {0.f, 0.f, 0.f, 0.f}, y2 = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            y1 += *reinterpret_cast<const f32x4 *>(&stage[w][0][i][c]);
            if (KEYS) y2 += *reinterpret_cast<const f32x4 *>(&stage[w][1][i][c]);
        }
        *reinterpret_cast<f32x4 *>(o1 + c) = y1 * a.scale;
        if (KEYS) *reinterpret_cast<f32x4 *>(o2 + c) = y2;
    }
}

// ---- launches ------------------------------------------------------------------------------------------------
template <typename T>
static void launch_delta_rows(const WindowArgs &a, hipStream_t st)
{
    const long long rows = (long long)a.B * a.H * a.Nq;
    const dim3 grid((unsigned)((rows + 15) / 16));
    if (a.D == 128) launch_kernel((window_delta_kernel<T, 128>), grid, dim3(256), 0, st, a, rows);
    else launch_kernel((window_delta_kernel<T, 64>), grid, dim3(256), 0, st, a, rows);
}

// Keys among the sinks are seen by every later query, the others by `window` of them: their queries are cut into pieces of about as many, as
// long as the pieces of the call are no more than 8 for each of the 256 compute units.  More would balance nothing, and each costs 2 D x 128
// floats of scratch (at most 256 MiB in all).  N = 12480, window 300, 1560 sinks, d = 128, without that end and with it: 12 heads 1044 (30 pieces) and
// 921 us (13), 96 heads 7709 (30) and 6302 (1); 12 heads, all keys sinks, window 16: 6782 (64) and 2856 (1).  The same calls in one
// piece: 12 heads 1039; with 4 sinks 907 (307 in the rule's 30), with window 4680 2197 (1938 in 3).
int window_sink_pieces(const WindowArgs &a)
{
    const long long tiles = (long long)a.B * a.Hk * window_sink_tiles_of(a);
    if (!tiles) return 1;
    const long long one = (long long)a.window + 128;
    return (int)std::max(1ll, std::min({64ll, (a.Nq + one - 1) / one, 2048 / tiles}));
}

hipError_t launch_window_bwd_bf16(const WindowArgs &a, hipStream_t st)
{
    launch_delta_rows<u16>(a, st);
    const int qtiles = (a.Nq + 127) / 128, qtotal = a.B * a.H * qtiles, qper = (qtotal + 7) / 8;
    const int sinks = window_sink_tiles_of(a), ktiles = (a.Nk + 127) / 128 + sinks * (a.sink_pieces - 1), ktotal = a.B * a.Hk * ktiles, kper = (ktotal + 7) / 8;
    if (a.D == 128) {
        launch_kernel((window_grad_kernel<128, true>), dim3(kper * 8), dim3(256), 0, st, a, ktiles, ktotal, kper);
        launch_kernel((window_grad_kernel<128, false>), dim3(qper * 8), dim3(256), 0, st, a, qtiles, qtotal, qper);
    } else {
        launch_kernel((window_grad_kernel<64, true>), dim3(kper * 8), dim3(256), 0, st, a, ktiles, ktotal, kper);
        launch_kernel((window_grad_kernel<64, false>), dim3(qper * 8), dim3(256), 0, st, a, qtiles, qtotal, qper);
    }
    if (a.sink_pieces > 1) {
        const dim3 grid((unsigned)((size_t)a.B * a.Hk * sinks * 2 * 128 / (256 / (a.D / 4))));
        if (a.D == 128) launch_kernel((window_sink_join_kernel<128>), grid, dim3(256), 0, st, a, sinks);
        else launch_kernel((window_sink_join_kernel<64>), grid, dim3(256), 0, st, a, sinks);
    }
    return take_launch_status();
}

hipError_t launch_window_bwd_f32(const WindowArgs &a, hipStream_t st)
{
    launch_delta_rows<float>(a, st);
    const int qtiles = (a.Nq + 15) / 16, ktiles = (a.Nk + 15) / 16;
    const dim3 qgrid((unsigned)((size_t)a.B * a.H * qtiles)), kgrid((unsigned)((size_t)a.B * a.Hk * ktiles));
    if (a.D == 128) {
        launch_kernel((window_grad_f32_kernel<128, true>), kgrid, dim3(256), 0, st, a, ktiles);
        launch_kernel((window_grad_f32_kernel<128, false>), qgrid, dim3(256), 0, st, a, qtiles);
    } else {
        launch_kernel((window_grad_f32_kernel<64, true>), kgrid, dim3(256), 0, st, a, ktiles);
        launch_kernel((window_grad_f32_kernel<64, false>), qgrid, dim3(256), 0, st, a, qtiles);
    }
    return take_launch_status();
}

}  // namespace salad
