// Internal declarations of the causal layer's operators: window attention with sinks (window_attn.hip, window_grad.hip) and the
// gated delta rule (delta_step.hip, delta_chunk.hip, delta_chain.hip, delta_grad.hip).  Host side: causal_api.hip.
#pragma once
#include "salad_internal.h"

namespace salad {

// ---- window attention ------------------------------------------------------------------------------
// Query n of sample b stands at position p = kv_len - q_len + n and sees key j <= p with j > p - window or j < sinks.
struct WindowArgs {
    const void *q, *k, *v;          // [B,H,Nq,D], [B,Hk,Nk,D]
    void *out;                      // [B,H,Nq,D]
    float *lse;                     // [B,H,Nq] natural logarithm; may be null in the forward pass
    const int32_t *q_lens, *kv_lens;// [B] or null: Nq, Nk
    int B, H, Hk, Nq, Nk, D;
    int window, sinks, ring;        // ring: position j >= sinks lies in row sinks + (j - sinks) % (Nk - sinks)
    float scale;
    // step kernel: the keys of a row tile are cut into `splits`; partial results where there are several
    int splits;
    float *part_o, *part_ml;        // [B Hk row tiles][splits][32][D]; [..][splits][2][32]
    // backward
    const void *dout;
    void *dq, *dk, *dv;
    float *delta;                   // [B,H,Nq] sum of dout * out
    int sink_pieces;                // pieces that the queries of a key tile with sinks are cut into
    float *sink_part;               // [B Hk][key tiles with sinks][sink_pieces][2][128][D]; null where sink_pieces is 1
};

constexpr int WINDOW_MAX_POSITION = 1 << 30;    // positions, windows and tile ends stay within 32 bits
struct WindowSpan { int qlen, off, kv; };       // of one sample; off: position of its query 0
__host__ __device__ inline WindowSpan window_span(const WindowArgs &a, int b)
{
    int ql = a.q_lens ? a.q_lens[b] : a.Nq, kv = a.kv_lens ? a.kv_lens[b] : a.Nk;
    ql = ql < 0 ? 0 : ql > a.Nq ? a.Nq : ql;    // lengths are device data: whatever they say, no row outside the tensors is touched
    kv = kv < 0 ? 0 : (!a.ring && kv > a.Nk) ? a.Nk : kv > WINDOW_MAX_POSITION ? WINDOW_MAX_POSITION : kv;
    return {ql, kv - ql, kv};
}
__device__ inline bool window_sees(const WindowArgs &a, int j, int p) { return j <= p && (j > p - a.window || j < a.sinks); }
__device__ inline int window_row(const WindowArgs &a, int j)
{
    return !a.ring || j < a.sinks ? j : a.sinks + (int)((unsigned)(j - a.sinks) % (unsigned)(a.Nk - a.sinks));
}
// Keys that queries at positions p0..p1 see: the sinks and first..p1, with first = p0 - window + 1.  Tiles hold others, too; what is loaded for
// those is the nearest that is seen, since P = 0 times an infinity or NaN (a row that was never written) would not be 0.
__device__ inline int window_first(const WindowArgs &a, int p0) { return p0 - a.window + 1; }
__device__ inline int window_nearest(const WindowArgs &a, int j, int first, int p1) { return min(j < a.sinks ? j : max(j, first), p1); }
// Tiles of `size` keys (aligned at 0) that queries at positions p0..p1 see: those of the sinks, then those of the windows.
struct KeyTiles {
    int ns, w0, n;
    __device__ KeyTiles(const WindowArgs &a, int p0, int p1, int size)
    {
        if (p1 < 0) { ns = w0 = n = 0; return; }
        const int last = p1 / size;
        ns = (int)(((long long)a.sinks + size - 1) / size);
        ns = ns < last + 1 ? ns : last + 1;
        const long long lo = (long long)p0 - a.window + 1;
        w0 = lo > 0 ? (int)(lo / size) : 0;
        w0 = w0 > ns ? w0 : ns;
        n = ns + (last >= w0 ? last - w0 + 1 : 0);
    }
    __device__ int tile(int i) const { return i < ns ? i : w0 + (i - ns); }
};

// Barrier behind loads that go straight into LDS: each wave waits for its own first, which a barrier alone leaves to chance.
__device__ inline void landed_barrier()
{
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
}

constexpr int STEP_ROWS = 32;       // rows (heads of a group x tokens) of a step-kernel workgroup
int window_step_splits(int B, int Hk, int row_tiles, int max_keys);     // 0: the call takes the tile kernel
bool window_takes_step(const WindowArgs &a);
hipError_t launch_window_fwd_bf16(const WindowArgs &a, hipStream_t st);
hipError_t launch_window_step_bf16(const WindowArgs &a, hipStream_t st);
hipError_t launch_window_fwd_f32(const WindowArgs &a, hipStream_t st);
hipError_t launch_window_bwd_bf16(const WindowArgs &a, hipStream_t st);
hipError_t launch_window_bwd_f32(const WindowArgs &a, hipStream_t st);
// 128-key tiles of the backward pass that hold sinks
__host__ __device__ inline int window_sink_tiles_of(const WindowArgs &a)
{
    const int s = a.sinks < a.Nk ? a.sinks : a.Nk;
    return (s + 127) / 128;
}
int window_sink_pieces(const WindowArgs &a);

struct AppendArgs {
    const void *k_new, *v_new; void *k, *v;     // [B,Hk,Nq,row], [B,Hk,Nk,row], rows in 16-byte pieces
    const int32_t *q_lens, *kv_lens;
    int B, Hk, Nq, Nk, pieces, sinks, ring;
};
hipError_t launch_window_append(const AppendArgs &a, hipStream_t st);

// ---- gated delta rule --------------------------------------------------------------------------------
struct DeltaArgs {
    const void *q, *k, *v;          // [B,Hk,N,D], [B,Hk,N,D], [B,H,N,D]
    const float *g, *beta;          // [B,H,N]
    void *out;                      // [B,H,N,D]
    const float *state_in;          // [B,H,D,D] or null (zeros)
    float *state_out;               // [B,H,D,D] or null
    const int32_t *lens;            // [B] or null: N
    int B, H, Hk, N, D, bf16;
    float scale;
    int chunks;                     // of 64 tokens
    // workspace, by (sample, head, chunk of 64 tokens)
    struct DeltaGate *gate;
    float2 *bsum;                   // [64] each: running sum of g as two floats
    u16 *tf, *ttf;                  // T = (I + A)^-1 and (backward) its transpose, operands in three planes
    u16 *pf;                        // forward: P, operand in two planes for bf16 tensors, three for fp32
    int groups, per_group;          // the chunks are cut into groups whose chains run side by side
    float *gsum, *gmap, *gstart;    // [BH][groups][D][D]: a group's chain from zeros, its linear map, and the state it starts from
    float *gsum_b, *gstart_b;       // backward: the same of the gradients' chain (its map is the transpose)
    // backward: what the gradients need of the forward pass
    float *s0;                      // [D][D] the state before the chunk, transposed (value channel, key channel)
    float *u;                       // [D][64] u, transposed
    // backward
    const void *dout;
    const float *dstate_out;
    void *dq, *dk, *dv;
    float *dg, *dbeta, *dstate_in;
    float *ds1;                     // [D][D] gradient of the state behind the chunk, transposed
    float *dr;                      // [D][64] first X = P^T dout, then dR = T^T du, transposed
    float *dq_part, *dk_part;       // [B,H,N,D] where heads share queries and keys, else null
};
__host__ __device__ inline int delta_len(const DeltaArgs &a, int b)
{
    const int n = a.lens ? a.lens[b] : a.N;
    return n < 0 ? 0 : n > a.N ? a.N : n;
}
bool delta_takes_step(const DeltaArgs &a);
hipError_t launch_delta_step(const DeltaArgs &a, hipStream_t st);
// steps shared by both directions
hipError_t launch_delta_chunk(const DeltaArgs &a, bool backward, hipStream_t st);
hipError_t launch_delta_chains(const DeltaArgs &a, bool backward, hipStream_t st);
int delta_groups(const DeltaArgs &a, bool backward);      // how many groups of chunks
hipError_t launch_delta_fwd(const DeltaArgs &a, hipStream_t st);
hipError_t launch_delta_bwd(const DeltaArgs &a, hipStream_t st);

}  // namespace salad
