// Linear attention with a decay for each head: cuts, workspace, the scan that joins segments, the sum over heads that share
// keys and values, and the single-token form.  Equations in decay.cuh.
#include <algorithm>

#include "decay_plan.cuh"

namespace dig {
namespace decay {
namespace {

// Joins the segments of a sequence: the state entering every one, in place of the segment's own contribution, or (x_end) the state
// behind the last.  A thread has one element of the state; the loads of a group of segments do not depend on one another.
struct ScanArgs {
    Pass pass[kMaxPasses];
    int H, L, nseg, span;                // span: positions of a segment
    const int *lengths;
    Log2Decay lam;
};
constexpr int kGroup = 8;
__global__ void __launch_bounds__(256) decay_scan(const __grid_constant__ ScanArgs a)
{
    const Pass &ps = a.pass[blockIdx.z];
    const int bh = blockIdx.y, b = bh / a.H, dd = ps.dk * ps.dv, e = blockIdx.x * 256 + threadIdx.x;
    const float lam = a.lam.v[bh - b * a.H];
    pdl_wait();
    pdl_launch_dependents();
    if (e >= dd) return;
    const int n = length_of(a.lengths, a.L, b);
    const int r = e / ps.dv, c = e - r * ps.dv;
    float x = ps.x0 ? ps.x0[(size_t)bh * dd + (ps.x_transposed ? c * ps.dk + r : e)] : 0.f;
    float *u = ps.local + (size_t)bh * a.nseg * dd + e;
    const int used = ps.x_end ? a.nseg : a.nseg - 1;             // the last segment's contribution goes into the final state only
    for (int s0 = 0; s0 < a.nseg; s0 += kGroup) {
        float own[kGroup];
#pragma unroll
        for (int i = 0; i < kGroup; ++i) own[i] = s0 + i < used ? u[(size_t)(s0 + i) * dd] : 0.f;
#pragma unroll
        for (int i = 0; i < kGroup; ++i) {
            const int s = s0 + i, rows = min(max(n - s * a.span, 0), a.span);
            if (s >= a.nseg) break;
            if (!ps.x_end) u[(size_t)s * dd] = x;
            if (rows > 0) x = fmaf(exp2_of(lam * (rows - (s == 0 ? 1 - ps.first : 0))), x, own[i]);
        }
    }
    if (ps.x_end) ps.x_end[(size_t)bh * dd + e] = n > 0 && ps.last ? x * exp2_of(lam) : x;         // no token: the start state
}

// out[t][hk] = sum over the heads that share hk, in their order; of dk and dv (blockIdx.y).  Bound by the bytes of the partial gradients.
struct ShareArgs {
    const float *part[2];
    void *out[2];
    int d4[2];
    long long rows;                      // tokens times shared heads
    int share;
};
template <typename S>
__global__ void __launch_bounds__(256) share_sum(const __grid_constant__ ShareArgs a)
{
    pdl_wait();
    pdl_launch_dependents();
    const int d4 = a.d4[blockIdx.y], share = a.share;
    const float *part = a.part[blockIdx.y];
    S *out = (S *)a.out[blockIdx.y];
    const size_t step = (size_t)gridDim.x * 256, n4 = (size_t)a.rows * d4;
    for (size_t i = blockIdx.x * (size_t)256 + threadIdx.x; i < n4; i += step) {
        const size_t row = i / d4;
        const float *p = part + (row * share * d4 + (i - row * d4)) * 4;
        float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int g = 0; g < share; g += 4) {                     // four are asked for together
            float4 x[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = load4(p + (size_t)min(g + e, share - 1) * d4 * 4);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (g + e >= share) break;
                s.x += x[e].x; s.y += x[e].y; s.z += x[e].z; s.w += x[e].w;
            }
        }
        store4(out + i * 4, s);
    }
}

}  // namespace

dig_status launch_scan(const Args &a, int tile, cudaStream_t stream)
{
    ScanArgs s;
    int most = 0;
    for (int i = 0; i < a.passes; ++i) {
        s.pass[i] = a.pass[i];
        const int dd = s.pass[i].dk * s.pass[i].dv;
        most = dd > most ? dd : most;
    }
    s.H = a.H; s.L = a.L; s.nseg = a.nseg; s.span = a.G * tile; s.lengths = a.lengths; s.lam = a.lam;
    KernelTimer t(KID_DECAY_SCAN, stream);
    return cuda_ok(launch_pdl(decay_scan, dim3((most + 255) / 256, a.B * a.H, a.passes), dim3(256), 0, stream, s));
}

dig_status launch_share_sum(const ShareArgs &a, int dtype, cudaStream_t stream)
{
    const size_t blocks = ((size_t)a.rows * std::max(a.d4[0], a.d4[1]) + 255) / 256, most = (size_t)kSms * 8;
    const dim3 grid((unsigned)std::min(blocks, most), 2);
    KernelTimer t(KID_DECAY_SUM, stream);
    return cuda_ok(dtype == DIG_F32 ? launch_pdl(share_sum<float>, grid, dim3(256), 0, stream, a) : launch_pdl(share_sum<__nv_bfloat16>, grid, dim3(256), 0, stream, a));
}

// ---- one token ------------------------------------------------------------------------------------------------------
namespace {

struct StepArgs {
    const void *q, *k, *v;
    const float *s_in;
    void *out;
    float *s_out;
    int H, share, dk, dv;
    Log2Decay lam;
};
// A CTA has one head of one sequence.  S = g S + k^T v, o = q S: a thread has four value channels of every `groups`-th state row.  Bound by
// the state's bytes, in and out.  The rows of a batch are asked for together before the first is written: the state may be updated in
// place, so no load would pass a store (192 sequences of 16 heads of 72 x 72: 27 us, 4.7 TB/s).
constexpr int kBatch = 8;
template <typename S>
__global__ void __launch_bounds__(256) decay_step(const __grid_constant__ StepArgs a)
{
    __shared__ float q[128], k[128];
    __shared__ float4 part[256];
    const int bh = blockIdx.x, b = bh / a.H, h = bh - b * a.H, dk = a.dk, dv = a.dv, hk = b * (a.H / a.share) + h / a.share;
    const int cols = dv / 4, groups = 256 / cols, g = threadIdx.x / cols, c = (threadIdx.x - g * cols) * 4;
    const float gamma = exp2_of(a.lam.v[h]);
    pdl_wait();
    float4 s[kBatch], v = make_float4(0.f, 0.f, 0.f, 0.f);
    const size_t at = (size_t)bh * dk * dv + c;
    auto load = [&](int r0) {
#pragma unroll
        for (int i = 0; i < kBatch; ++i)
            if (r0 + i * groups < dk) s[i] = load4(a.s_in + at + (size_t)(r0 + i * groups) * dv);
    };
    if (g < groups) {
        load(g);
        v = load4((const S *)a.v + (size_t)hk * dv + c);
    }
    if (threadIdx.x < dk) {
        q[threadIdx.x] = (float)((const S *)a.q)[(size_t)bh * dk + threadIdx.x];
        k[threadIdx.x] = (float)((const S *)a.k)[(size_t)hk * dk + threadIdx.x];
    }
    __syncthreads();
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    if (g < groups) {
        for (int r0 = g; r0 < dk; r0 += kBatch * groups) {
            if (r0 > g) load(r0);
#pragma unroll
            for (int i = 0; i < kBatch; ++i) {
                const int r = r0 + i * groups;
                if (r >= dk) break;
                const float x = k[r], y = q[r];
                float4 &z = s[i];
                z.x = fmaf(gamma, z.x, x * v.x); z.y = fmaf(gamma, z.y, x * v.y); z.z = fmaf(gamma, z.z, x * v.z); z.w = fmaf(gamma, z.w, x * v.w);
                store4(a.s_out + at + (size_t)r * dv, z);
                o.x = fmaf(y, z.x, o.x); o.y = fmaf(y, z.y, o.y); o.z = fmaf(y, z.z, o.z); o.w = fmaf(y, z.w, o.w);
            }
        }
    }
    part[threadIdx.x] = o;
    __syncthreads();
    if (threadIdx.x < cols) {
        for (int i = 1; i < groups; ++i) {
            const float4 x = part[i * cols + threadIdx.x];
            o.x += x.x; o.y += x.y; o.z += x.z; o.w += x.w;
        }
        store4((S *)a.out + (size_t)bh * dv + c, o);
    }
    pdl_launch_dependents();
}

}  // namespace
}  // namespace decay

using namespace decay;

dig_status decay_step_launch(const void *q, const void *k, const void *v, const float *log_decay, const float *s_in, void *out, float *s_out,
                             int B, int H, int H_kv, int dk, int dv, int dtype, cudaStream_t stream)
{
    StepArgs a;
    a.q = q; a.k = k; a.v = v; a.s_in = s_in; a.out = out; a.s_out = s_out;
    a.H = H; a.share = H / H_kv; a.dk = dk; a.dv = dv;
    if (!set_decay(a.lam, log_decay, H)) return DIG_ERR_INVALID_ARG;
    KernelTimer t(KID_DECAY_STEP, stream);
    if (dtype == DIG_F32) return cuda_ok(launch_pdl(decay_step<float>, dim3(B * H), dim3(256), 0, stream, a));
    return cuda_ok(launch_pdl(decay_step<__nv_bfloat16>, dim3(B * H), dim3(256), 0, stream, a));
}

// ---- whole sequences -------------------------------------------------------------------------------------------------
size_t decay_workspace_bytes(int B, int H, int H_kv, int L, int dk, int dv, int dtype, bool backward)
{
    return carve(nullptr, B, H, H_kv, L, dk, dv, dtype, backward).bytes;
}

namespace {

Rows rows_of(const void *p, const long long *strides, long long L, int heads, int d, int share)
{
    Rows r{p, (long long)L * heads * d, (long long)heads * d, share};
    if (strides) { r.batch = strides[0]; r.token = strides[1]; }
    return r;
}

// Local pass and scan for the states that enter segments, where the sequences are cut (of the passes that have states of their own, the
// first `n`), then the passes themselves.  The state that the caller wants (of the pass `end`): the fp32 kernels' last segments end with it;
// the tensor-core kernels sum it apart, in the local pass.
dig_status run(Args &a, const Carved &w, int n, int end, int dtype, cudaStream_t stream)
{
    a.nseg = w.plan.nseg; a.G = w.plan.G;
    Pass &last = a.pass[end];
    const bool cut = a.nseg > 1, apart = last.x_end && dtype != DIG_F32;
    if (apart) last.final = w.final;                 // uncut: not written, but says that the state is wanted
    Args l = a;
    if (cut) {
        l.passes = n;
        dig_status st = pass_kernel(l, true, dtype, stream);
        if (st != DIG_OK) return st;
        // the scan: entering states of n passes, and the final one
        for (int i = 0; i < n; ++i) l.pass[i].x_end = nullptr;
        if (apart) {
            l.pass[n] = last;
            l.pass[l.passes++].local = w.final;
        }
        st = launch_scan(l, w.plan.tile, stream);
        return st != DIG_OK ? st : pass_kernel(a, false, dtype, stream);
    }
    a.beside = l.beside = apart;
    const dig_status st = pass_kernel(a, false, dtype, stream);
    if (st != DIG_OK || !apart) return st;
    l.passes = 1;
    l.pass[0] = last;
    return pass_kernel(l, true, dtype, stream);
}

// The tensor-core kernels count results in 16 bytes with 32 bits.
bool too_large(const DecayCall &c) { return c.dtype == DIG_BF16 && (size_t)c.B * c.L * c.H * (c.dk > c.dv ? c.dk : c.dv) / 8 >= 0xffffffffull; }

}  // namespace

dig_status decay_fwd_launch(const DecayCall &c)
{
    if (too_large(c)) return DIG_ERR_UNSUPPORTED;
    const int share = c.H / c.H_kv;
    const Carved w = carve(reinterpret_cast<char *>(c.ws), c.B, c.H, c.H_kv, c.L, c.dk, c.dv, c.dtype, false);
    Args a{};
    if (!set_decay(a.lam, c.log_decay, c.H)) return DIG_ERR_INVALID_ARG;
    a.passes = 1; a.B = c.B; a.H = c.H; a.L = c.L; a.gh = c.gh; a.gw = c.gw; a.lengths = c.lengths;
    a.gh_inv = c.gh == 1 ? 0xffffffffu : (uint32_t)((1ull << 32) / c.gh);
    Pass &p = a.pass[0];
    p.q = rows_of(c.q, c.strides, c.L, c.H, c.dk, 1);
    p.k = rows_of(c.k, c.strides ? c.strides + 2 : nullptr, c.L, c.H_kv, c.dk, share);
    p.v = rows_of(c.v, c.strides ? c.strides + 4 : nullptr, c.L, c.H_kv, c.dv, share);
    p.out = c.out; p.x0 = c.s_in; p.local = w.local[0]; p.x_end = c.s_out;
    p.dk = c.dk; p.dv = c.dv; p.dir = c.dir; p.first = 1; p.last = 0;
    return run(a, w, 1, 0, c.dtype, c.stream);
}

dig_status decay_bwd_launch(const DecayCall &c)
{
    if (too_large(c)) return DIG_ERR_UNSUPPORTED;
    const int share = c.H / c.H_kv;
    const Carved w = carve(reinterpret_cast<char *>(c.ws), c.B, c.H, c.H_kv, c.L, c.dk, c.dv, c.dtype, true);
    Args a{};
    if (!set_decay(a.lam, c.log_decay, c.H)) return DIG_ERR_INVALID_ARG;
    a.passes = 3; a.B = c.B; a.H = c.H; a.L = c.L; a.gh = c.gh; a.gw = c.gw; a.lengths = c.lengths;
    a.gh_inv = c.gh == 1 ? 0xffffffffu : (uint32_t)((1ull << 32) / c.gh);
    const Rows q = rows_of(c.q, c.strides, c.L, c.H, c.dk, 1), k = rows_of(c.k, c.strides ? c.strides + 2 : nullptr, c.L, c.H_kv, c.dk, share),
               v = rows_of(c.v, c.strides ? c.strides + 4 : nullptr, c.L, c.H_kv, c.dv, share), g = rows_of(c.d_out, nullptr, c.L, c.H, c.dv, 1);
    Pass &dq = a.pass[0], &dv = a.pass[1], &dk = a.pass[2];
    dq.q = g; dq.k = v; dq.v = k; dq.out = c.dq; dq.x0 = c.s_in; dq.x_transposed = 1; dq.local = w.local[0];
    dq.dk = c.dv; dq.dv = c.dk; dq.dir = c.dir; dq.first = 1;
    dv.q = k; dv.k = q; dv.v = g; dv.out = share > 1 ? (void *)w.part_v : c.dv_out; dv.x0 = c.ds_out; dv.local = w.local[1]; dv.x_end = c.ds_in;
    dv.dk = c.dk; dv.dv = c.dv; dv.dir = c.dir ^ 1; dv.last = 1; dv.out_f32 = share > 1;
    dk.q = v; dk.k = g; dk.v = q; dk.out = share > 1 ? (void *)w.part_k : c.dk_out; dk.x0 = c.ds_out; dk.x_transposed = 1; dk.local = w.local[1];
    dk.local_transposed = 1; dk.dk = c.dv; dk.dv = c.dk; dk.dir = c.dir ^ 1; dk.out_f32 = share > 1;
    dig_status st = run(a, w, 2, 1, c.dtype, c.stream);
    if (st != DIG_OK || share == 1) return st;
    ShareArgs sum{};
    sum.part[0] = w.part_k; sum.part[1] = w.part_v; sum.out[0] = c.dk_out; sum.out[1] = c.dv_out;
    sum.d4[0] = c.dk / 4; sum.d4[1] = c.dv / 4; sum.rows = (long long)c.B * c.L * c.H_kv; sum.share = share;
    return launch_share_sum(sum, c.dtype, c.stream);
}

}  // namespace dig
