// Products of the delta rule's kernels: v_mfma_f32_16x16x32_bf16 on operands kept as one or three bf16 planes.
//
// The state, u and their gradients are fp32 results of long recurrences, and their products have to keep that.  A float x is
// x0 + x1 + x2 with x0 = bf16(x), x1 = bf16(x - x0), x2 = bf16(x - x0 - x1): 24 bits, exact but for values below the range.  The product
// of three planes by three takes the six terms down to 2^-16 of the first (what is left out adds up to 2^-23 of it at most), by a tensor that is bf16
// already three.  The fp32 matrix instruction has a sixteenth of the bf16 rate: six products are 2.7 times faster, three 5.3 times.
//
// Lane l of an operand holds row l % 16 and the 8 contraction indices from 8 (l / 16) on; accumulator r is row 4 (l / 16) + r,
// column l % 16.  An LDS tile is row-major with `pitch` elements a row; it serves as an operand along its rows (frag_n) or, by
// transposing reads, along its columns (frag_t).
#pragma once
#include "causal.h"

namespace salad {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

namespace {

#define LDS_PTR(p) ((__attribute__((address_space(3))) void *)(p))

__device__ inline uint32_t pack2(float a, float b)
{
    f32x2 x = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, bf16x2));
}
__device__ inline float low(uint32_t w) { return __uint_as_float(w << 16); }
__device__ inline float high(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// A workgroup's barrier for what it exchanges through LDS.  __syncthreads() would also wait for every load and store to memory in flight, and
// with that for the operands that are loaded a chunk ahead.
__device__ inline void lds_barrier()
{
    __builtin_amdgcn_sched_barrier(0);      // what uses an operand late does not wait for it early
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
    __builtin_amdgcn_sched_barrier(0);
}

// A store that the hardware drops where `offset` is not below the size that the resource was made with.  Loads and stores are counted
// together, in order: behind a store that may be skipped nobody could wait for an earlier load without waiting for the store, too.
template <typename T>
__device__ inline __amdgpu_buffer_rsrc_t bounded(T *p, int elems)
{
    return __builtin_amdgcn_make_buffer_rsrc(p, 0, elems * (int)sizeof(T), 0x00027000);
}
__device__ inline void store_bounded(__amdgpu_buffer_rsrc_t r, u16, int elem, f32x4 x)
{
    __builtin_amdgcn_raw_buffer_store_b64(u32x2{pack2(x[0], x[1]), pack2(x[2], x[3])}, r, elem * 2, 0, 0);
}
__device__ inline void store_bounded(__amdgpu_buffer_rsrc_t r, float, int elem, f32x4 x)
{
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, x), r, elem * 4, 0, 0);
}

template <int P> struct Op { bf16x8 p[P]; };

// c += A B, the small terms first
template <int PA, int PB>
__device__ inline void mma(f32x4 &c, const Op<PA> &a, const Op<PB> &b)
{
#pragma unroll
    for (int s = 2; s >= 0; --s)
#pragma unroll
        for (int i = 0; i < PA; ++i)
            if (s - i >= 0 && s - i < PB) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.p[i], b.p[s - i], c, 0, 0, 0);
}

// N such products by the same B in turn: a product takes longer than the next one's issue, so neighbours go to different accumulators
template <int N, int PA, int PB>
__device__ inline void mmas(f32x4 *c, const Op<PA> *a, const Op<PB> &b)
{
#pragma unroll
    for (int s = 2; s >= 0; --s)
#pragma unroll
        for (int i = 0; i < PA; ++i)
            if (s - i >= 0 && s - i < PB)
#pragma unroll
                for (int n = 0; n < N; ++n) c[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[n].p[i], b.p[s - i], c[n], 0, 0, 0);
}

// four floats as P planes
template <int P>
__device__ inline void split4(f32x4 x, u32x2 (&o)[P])
{
#pragma unroll
    for (int p = 0; p < P; ++p) {
        o[p].x = pack2(x[0], x[1]);
        o[p].y = pack2(x[2], x[3]);
        if (p + 1 < P) x -= f32x4{low(o[p].x), high(o[p].x), low(o[p].y), high(o[p].y)};
    }
}
// 4 floats into 4 neighbouring elements of a tile's planes
template <int P>
__device__ inline void put4(u16 *tile, int plane, f32x4 x)
{
    u32x2 o[P];
    split4<P>(x, o);
#pragma unroll
    for (int p = 0; p < P; ++p) *reinterpret_cast<u32x2 *>(tile + p * plane) = o[p];
}

// operand whose row is row r0 + l % 16 of the tile, contraction along the row from k0 on
template <int P>
__device__ inline Op<P> frag_n(const u16 *tile, int plane, int pitch, int r0, int k0, int lane)
{
    Op<P> f;
    const u16 *at = tile + (r0 + (lane & 15)) * pitch + k0 + 8 * (lane >> 4);
#pragma unroll
    for (int p = 0; p < P; ++p) f.p[p] = *reinterpret_cast<const bf16x8 *>(at + p * plane);
    return f;
}
// operand whose row is column c0 + l % 16 of the tile, contraction down the column from row k0 on.  Each group of 16 lanes
// transposes 4 rows x 16 columns; the lane supplies the address of row (l / 4) % 4, columns 4 (l % 4) on.
template <int P>
__device__ inline Op<P> frag_t(const u16 *tile, int plane, int pitch, int c0, int k0, int lane)
{
    union { bf16x8 v; s16x4 h[2]; } u;
    Op<P> f;
    const u16 *at = tile + (k0 + 8 * (lane >> 4) + ((lane >> 2) & 3)) * pitch + c0 + 4 * (lane & 3);
#pragma unroll
    for (int p = 0; p < P; ++p) {
        u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3))) *)LDS_PTR(at + p * plane));
        u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3))) *)LDS_PTR(at + p * plane + 4 * pitch));
        f.p[p] = u.v;
    }
    return f;
}

// a tensor's type: planes of its operands, 4 neighbouring values as floats
template <typename T> constexpr int planes_of() { return sizeof(T) == 2 ? 1 : 3; }
// planes of P and u in O = scale gamma Q S + P u: for bf16 tensors S is rounded to bf16 there (one plane: half a step of its terms, as O itself),
// and with u and P rounded, too, O's error against 64 bits is 1.7 times that of its own rounding (480p clip: 2.8e-3; 2.4e-3 with P alone,
// 1.8e-3 with neither, for 3 % more time)
template <typename T> constexpr int out_planes() { return sizeof(T) == 2 ? 2 : 3; }
__device__ inline f32x4 load4(const u16 *p)
{
    const u32x2 w = *reinterpret_cast<const u32x2 *>(p);
    return f32x4{low(w.x), high(w.x), low(w.y), high(w.y)};
}
__device__ inline f32x4 load4(const float *p) { return *reinterpret_cast<const f32x4 *>(p); }
__device__ inline float load1(const u16 *p) { return __uint_as_float((uint32_t)*p << 16); }
__device__ inline float load1(const float *p) { return *p; }
__device__ inline void store4(u16 *p, f32x4 x) { *reinterpret_cast<u32x2 *>(p) = u32x2{pack2(x[0], x[1]), pack2(x[2], x[3])}; }
__device__ inline void store4(float *p, f32x4 x) { *reinterpret_cast<f32x4 *>(p) = x; }

// operand straight from a tensor's row, 8 values from p on (a valid address in any case); zeros where !ok
__device__ inline Op<1> frag_g(const u16 *p, bool ok)
{
    u32x4 w = *reinterpret_cast<const u32x4 *>(p);
    w = ok ? w : u32x4{0, 0, 0, 0};
    return Op<1>{{__builtin_bit_cast(bf16x8, w)}};
}
// Accumulators as an operand.  The order of a contraction is free, so it is chosen such that two tiles of accumulators stand as the operand of
// the next product as they are: lane group l4 of an operand over 32 indices has the four of the first tile and the four of the second.
// Tokens: tile t has token 16 t + 4 l4 + r, so the operand goes 32 kt + 4 l4.., 32 kt + 16 + 4 l4.. .  Key channels: tiles 2 ks and
// 2 ks + 1 are given the channels 32 ks + 8 l4 + r and 32 ks + 8 l4 + 4 + r, so that the operand's order is the channels' own.
//
// A tile [64 tokens][D] that is read both ways, along its rows (row r0 + l % 16, channels 32 ks.. in their order) and down its columns (row l % 16
// of channel tile 2 ks + x, tokens 32 kt.. in the accumulators' order, by transposing reads).  Its rows' 16-byte pieces are
// swizzled, so that 16 rows of one piece and 4 rows of 4 pieces both spread over the banks.
template <int D> __device__ inline int sigma(int r) { return D == 128 ? ((r & 3) << 2) | ((r >> 2) & 3) : (((r >> 1) & 1) << 2) | ((r >> 2) & 3); }
template <int P, int D>
__device__ inline Op<P> frag_k(const u16 *tile, int r0, int ks, int lane)
{
    Op<P> f;
    const int row = r0 + (lane & 15);
    const u16 *at = tile + row * D + (((4 * ks + (lane >> 4)) ^ sigma<D>(row)) << 3);
#pragma unroll
    for (int p = 0; p < P; ++p) f.p[p] = *reinterpret_cast<const bf16x8 *>(at + p * 64 * D);
    return f;
}
template <int P, int D>
__device__ inline Op<P> frag_c(const u16 *tile, int ks, int x, int kt, int lane)
{
    union { bf16x8 v; s16x4 h[2]; } u;
    Op<P> f;
    const int row = 32 * kt + 4 * (lane >> 4) + ((lane >> 2) & 3);          // and 16 rows on, swizzled alike
    const u16 *at = tile + row * D + (((4 * ks + (lane & 3)) ^ sigma<D>(row)) << 3) + 4 * x;
#pragma unroll
    for (int p = 0; p < P; ++p) {
        u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3))) *)LDS_PTR(at + p * 64 * D));
        u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3))) *)LDS_PTR(at + p * 64 * D + 16 * D));
        f.p[p] = u.v;
    }
    return f;
}

template <int P>
__device__ inline Op<P> op_of(f32x4 x, f32x4 y)
{
    u32x2 a[P], b[P];
    split4<P>(x, a);
    split4<P>(y, b);
    Op<P> f;
#pragma unroll
    for (int i = 0; i < P; ++i) f.p[i] = __builtin_bit_cast(bf16x8, u32x4{a[i].x, a[i].y, b[i].x, b[i].y});
    return f;
}
__device__ inline Op<3> frag_g(const float *p, bool ok)
{
    const f32x4 x = *reinterpret_cast<const f32x4 *>(p), y = *reinterpret_cast<const f32x4 *>(p + 4), z = {0.f, 0.f, 0.f, 0.f};
    return op_of<3>(ok ? x : z, ok ? y : z);
}

// 64 rows x D of a tensor on their way to an LDS tile: 256 threads load them into registers, and put them down later
template <typename T, int D> struct Tile64 {
    static constexpr int P = planes_of<T>(), PITCH = D + 8, PLANE = 64 * PITCH, PER = 16 / sizeof(T), LPR = D / PER, RPP = 256 / LPR, NP = 64 / RPP;
    u32x4 r[NP];
    __device__ inline void load(const T *base, int valid, int tid)
    {
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int row = i * RPP + tid / LPR;
            const u32x4 w = *reinterpret_cast<const u32x4 *>(base + (size_t)min(row, valid - 1) * D + tid % LPR * PER);
            r[i] = row < valid ? w : u32x4{0, 0, 0, 0};
        }
    }
    __device__ inline void load_clamped(const T *base, int last, int tid)       // rows behind the last are the last once more
    {
#pragma unroll
        for (int i = 0; i < NP; ++i) r[i] = *reinterpret_cast<const u32x4 *>(base + (unsigned)(min(i * RPP + tid / LPR, last) * D + tid % LPR * PER));
    }
    __device__ inline void store(u16 *tile, int tid) const
    {
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            u16 *at = tile + (i * RPP + tid / LPR) * PITCH + tid % LPR * PER;
            if constexpr (sizeof(T) == 2) *reinterpret_cast<u32x4 *>(at) = r[i];
            else put4<3>(at, PLANE, __builtin_bit_cast(f32x4, r[i]));
        }
    }
    __device__ inline void store_swizzled(u16 *tile, int tid) const
    {
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int row = i * RPP + tid / LPR, col = tid % LPR * PER;
            u16 *at = tile + row * D + (((col >> 3) ^ sigma<D>(row)) << 3) + (col & 7);
            if constexpr (sizeof(T) == 2) *reinterpret_cast<u32x4 *>(at) = r[i];
            else put4<3>(at, 64 * D, __builtin_bit_cast(f32x4, r[i]));
        }
    }
};

}  // namespace

// of a chunk, for the kernels behind delta_chunk_kernel, by token: gamma = exp(b_i), tail = exp(b_63 - b_i), beta_i with b the running sum of g
// (tail and beta are zero for tokens that are not there)
struct DeltaGate { float gamma[64], tail[64], beta[64]; };
constexpr int DELTA_C = 64;
// A chunk's triangular 64 x 64 matrix as operands: planes of six pieces (row tile, half of the contraction), 64 lanes x 8 elements each
constexpr int TRI = 6 * 64 * 8;
__host__ __device__ constexpr int tri_lower(int rt, int kt) { return rt < 2 ? rt : 2 * rt - 2 + kt; }         // (0,0) (1,0) (2,0) (2,1) (3,0) (3,1)
__host__ __device__ constexpr int tri_upper(int rt, int kt) { return rt < 2 ? 2 * rt + kt : 2 + rt; }          // (0,0) (0,1) (1,0) (1,1) (2,1) (3,1)

}  // namespace salad
