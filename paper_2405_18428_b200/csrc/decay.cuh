// Linear attention with a decay for each head: S_t = g S_{t-1} + k_t^T v_t, o_t = q_t S_t, g = exp(log_decay[h]).
//
// With g a number, the products of a tile of positions p0 .. p0 + n - 1 need no scaling per channel: with X the state after position
// p0 - 1,
//     O_i = sum_{j <= i} g^(i-j) (q_i . k_j) v_j + g^(i+1) q_i X,     X' = g^n X + sum_j g^(n-1-j) k_j^T v_j,
// every power at most 1.  The gradients have the same form.  For W_ij = g^(i-j) (j <= i) the matrix of a whole sequence,
//     dq = (dO V^T . W) K,   dk = (V dO^T . W^T) Q,   dv = (K Q^T . W^T) dO,
// which are linear attentions with (query, key, value) = (dO, v, k) in the scan order and (v, dO, q), (k, q, dO) in the opposite one,
// started from s_in^T, ds_out^T and ds_out.  The start state counts with g^(p+1) at position p in the first, with g^p in the other two
// (`first`).  So one kind of kernel serves both directions, and a launch takes up to three such passes side by side.
//
// A sequence of tiles is cut into segments, one CTA each, where there are fewer sequences than CTAs: a local pass gives every segment's
// own contribution to the state behind it, a scan over the segments gives the states that enter them.
#pragma once

#include "dig_common.cuh"

namespace dig {
namespace decay {

constexpr int kMaxHeads = 256;
constexpr int kMaxPasses = 3;
constexpr int kSms = 148;                // of a B200: plans do not ask the device, so that a workspace fits wherever it was sized

struct Log2Decay { float v[kMaxHeads]; };

// Rows of one operand: token t of head h is at p + b * batch + t * token + (h / share) * d, in elements.
struct Rows {
    const void *p;
    long long batch, token;
    int share;
};

// One linear attention.  `dir`: its scan order; x0: start state [B][H][dk][dv] (transposed: [dv][dk]) or null, in force with
// g^(p + first) at position p.  out: [B][L][H][dv], of the storage type, or fp32 where out_f32.  local: [B*H][nseg][dk][dv] fp32, written
// by the local pass (where there are several segments) and turned into the entering states by the scan; `from`: the pass whose entering states this one reads
// (transposed where they differ).
struct Pass {
    Rows q, k, v;
    void *out;
    const float *x0;
    float *local;
    float *x_end;                        // where wanted, g^last (state behind the last position); the scan: instead of the entering states
    float *final;                        // local pass on tensor cores: where the final state is wanted, what adds up to it, [B*H][nseg][dk][dv] in fp32 accuracy
    int dk, dv, dir, first, last, x_transposed, local_transposed, out_f32;
};

struct Args {
    Pass pass[kMaxPasses];
    int passes, B, H, L, gh, gw, nseg, G;         // G: tiles of a segment
    // Uncut sequences whose final state is wanted: the local pass, which needs nothing of the passes, runs beside them, on SMs that they leave
    // free (80 sequences of 20 tiles of 128 channels: 88 us, 141 one after the other).  The passes let it start once what precedes them is
    // complete, and it waits for them before it ends.
    int beside;
    const int *lengths;                  // [B] or null
    uint32_t gh_inv;                     // floor(2^32 / gh), 2^32 - 1 for one row: column orders divide by the grid's height
    Log2Decay lam;
};

// Tokens of sequence b; values outside 0 .. L count as the nearest of the two.
__device__ __forceinline__ int length_of(const int *lengths, int L, int b)
{
    return lengths ? min(max(__ldcg(lengths + b), 0), L) : L;
}
__device__ __forceinline__ float exp2_of(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Joins segments: kernel of decay.cu.
dig_status launch_scan(const Args &a, int tile, cudaStream_t stream);

// Rows of a tile, and the two kinds of kernels.
constexpr int kTileFma = 64, kTileTc = 128;
dig_status fma_pass(const Args &a, bool local, cudaStream_t stream);         // fp32 storage
dig_status tc_pass(const Args &a, bool local, cudaStream_t stream);          // bf16 storage

}  // namespace decay
}  // namespace dig
