// Host side of linear attention with a decay for each head: how sequences are cut, and the workspace that takes.  Plain arithmetic
// without CUDA calls.
#pragma once

#include <cmath>

#include "decay.cuh"

namespace dig {

// Arguments of a whole-sequence call, checked by the entry point.
struct DecayCall {
    const void *q, *k, *v;
    const long long *strides;            // batch and token strides of q, k, v, or null: dense
    const float *log_decay;
    const int *lengths;
    const float *s_in, *ds_out;
    const void *d_out;
    void *out, *dq, *dk_out, *dv_out;
    float *s_out, *ds_in;
    int B, H, H_kv, L, gh, gw, dk, dv, dir, dtype;
    void *ws;
    cudaStream_t stream;
};

namespace decay {

struct Plan {
    int tile, nseg, G;
};
// How many segments.  Costs in tiles of the pass: a round of segments on all CTAs that run together takes its tiles and a fill; a cut
// adds the local pass (of the states that enter segments: one pass of them forward, two backward), its launches, and the scan over all segments.
// Fitted to 2283 measured calls of 6 to 480 sequences of 2 to 128 tiles, 1 to 64 segments, heads of 64, 72 and 128 channels: the cut chosen
// is 0.15% off the best on average in bf16 (worst 12%), 1.2% in fp32 (worst 18%); forward passes that return the final state, 3% (worst 37%:
// results are not to depend on whether it is asked for).
struct Cost {
    int slots;                           // CTAs on an SM: of the pass,
    int local_slots;                     // of the local pass
    double fill, tile, local_fill, cut, scan;
};
constexpr Cost kCostTc = {1, 2, 2.0, 0.69, 1.2, 1.6, 0.5}, kCostTcWide = {1, 1, 0.55, 0.32, 0.5, 2.2, 0.1};           // to 80 channels, to 128
constexpr Cost kCostFma = {2, 2, 0.4, 0.94, 0.0, 0.3, 0.0}, kCostFmaWide = {1, 1, 1.0, 0.23, 0.4, 0.0, 0.2};
inline Plan make_plan(int B, int H, int L, bool backward, int d, int dtype)
{
    const Cost &c = dtype == DIG_F32 ? (d <= 80 ? kCostFma : kCostFmaWide) : d <= 80 ? kCostTc : kCostTcWide;
    Plan p;
    p.tile = dtype == DIG_F32 ? kTileFma : kTileTc;
    const long long tiles = (L + p.tile - 1) / p.tile, seqs = (long long)B * H, passes = backward ? 3 : 1, states = backward ? 2 : 1;
    auto ceil_div = [](long long x, long long y) { return (x + y - 1) / y; };
    double least = 0;
    p.nseg = 0;
    for (long long nseg = 1; nseg <= tiles; ++nseg) {
        const long long G = ceil_div(tiles, nseg);
        if (ceil_div(tiles, G) != nseg) continue;
        double t = ceil_div(seqs * passes * nseg, c.slots * kSms) * (G + c.fill);
        if (nseg > 1) t += ceil_div(seqs * states * nseg, c.local_slots * kSms) * (G * c.tile + c.local_fill) + c.cut + c.scan * seqs * states * nseg / kSms;
        if (p.nseg == 0 || t < least) {
            least = t;
            p.nseg = (int)nseg;
            p.G = (int)G;
        }
        if (seqs * passes * nseg >= 3 * c.slots * kSms) break;
    }
    return p;
}

// Workspace, every block 256-byte aligned: where sequences are cut states of the segments, [B*H][nseg][dk][dv] fp32 (backward: of two
// passes), the same once more for the final state of bf16 calls, and where heads share keys and values the gradients of each head before they are summed, fp32 [B][L][H][d].
struct Carved {
    Plan plan;
    float *local[2], *final, *part_k, *part_v;
    size_t bytes;
};
inline Carved carve(char *base, int B, int H, int H_kv, int L, int dk, int dv, int dtype, bool backward)
{
    Carved w{};
    w.plan = make_plan(B, H, L, backward, dk > dv ? dk : dv, dtype);
    size_t o = 0;
    auto take = [&](size_t bytes) { char *p = base + o; o += align256(bytes); return reinterpret_cast<float *>(p); };
    const size_t state = w.plan.nseg > 1 ? (size_t)B * H * w.plan.nseg * dk * dv * 4 : 16;
    w.local[0] = take(state);
    w.final = take(dtype == DIG_F32 ? 0 : state);
    if (backward) {
        w.local[1] = take(state);
        if (H != H_kv) {
            w.part_k = take((size_t)B * L * H * dk * 4);
            w.part_v = take((size_t)B * L * H * dv * 4);
        }
    }
    w.bytes = o;
    return w;
}

// log2 of the decays; false where one is no decay: above 0 or no finite number.
inline bool set_decay(Log2Decay &l, const float *log_decay, int H)
{
    for (int h = 0; h < H; ++h) {
        const float x = log_decay[h];
        if (!(x <= 0.f) || std::isinf(x)) return false;
        l.v[h] = (float)std::fmax(x * 1.4426950408889634, -1e6);          // 2^-1e6 is 0 as well, and its multiples are finite
    }
    return true;
}

inline dig_status pass_kernel(const Args &a, bool local, int dtype, cudaStream_t stream)
{
    return dtype == DIG_F32 ? fma_pass(a, local, stream) : tc_pass(a, local, stream);
}

}  // namespace decay
}  // namespace dig
