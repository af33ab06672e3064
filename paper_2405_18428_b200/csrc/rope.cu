// Rotary positions with several axes.  Pair i of a head's channels is turned by positions[token][axis[i]] * freq[i]; the inverse
// rotation is the gradient of the rotation.  Angles are formed in 64 bits, in turns, and reduced before they are rounded to fp32: far
// positions (2^31 at frequency 1) keep angles within 2e-7.
// Moved once: q and k in and out.  A token's angles are computed once by its CTA and serve all of its heads.
#include <cmath>

#include "dig_common.cuh"

namespace dig {
namespace {

constexpr int kMaxPairs = 64, kNT = 256, kMaxTokens = 8;

struct RopeArgs {
    const void *x[2];                // q, k (null: none)
    void *y[2];
    long long xb[2], xt[2], yb[2], yt[2];        // batch and token strides in elements
    const int *pos;
    long long pos_batch;
    int heads[2];
    int L, d, n, axes, tokens;       // n: pairs; tokens of a CTA
    long long total;                 // B * L
    double turns[kMaxPairs];         // freq / (2 pi), negative for the inverse
    unsigned char axis[kMaxPairs];
};

template <typename T, int V> struct Vec;
template <> struct Vec<float, 1> { using U = float; };
template <> struct Vec<float, 2> { using U = float2; };
template <> struct Vec<float, 4> { using U = float4; };
template <> struct Vec<__nv_bfloat16, 1> { using U = unsigned short; };
template <> struct Vec<__nv_bfloat16, 2> { using U = uint32_t; };
template <> struct Vec<__nv_bfloat16, 4> { using U = uint2; };
template <> struct Vec<__nv_bfloat16, 8> { using U = uint4; };
template <typename T, int V>
__device__ __forceinline__ void ldv(const T *p, float (&f)[V])
{
    using U = typename Vec<T, V>::U;
    const U u = *reinterpret_cast<const U *>(p);
    const T *e = reinterpret_cast<const T *>(&u);
#pragma unroll
    for (int i = 0; i < V; ++i) f[i] = (float)e[i];
}
template <typename T, int V>
__device__ __forceinline__ void stv(T *p, const float (&f)[V])
{
    using U = typename Vec<T, V>::U;
    U u;
    T *e = reinterpret_cast<T *>(&u);
#pragma unroll
    for (int i = 0; i < V; ++i) e[i] = (T)f[i];
    *reinterpret_cast<U *>(p) = u;
}

// V pairs per thread and turn: neighbours (2 i, 2 i + 1) where INTER, else (i, i + n).
template <typename T, int V, bool INTER>
__global__ void __launch_bounds__(kNT) rope(const __grid_constant__ RopeArgs a)
{
    __shared__ float2 cs[kMaxTokens * kMaxPairs];            // cosine, sine
    __shared__ double turns[kMaxPairs];
    __shared__ int axis[kMaxPairs];
    const long long first = (long long)blockIdx.x * a.tokens;
    const int here = (int)min((long long)a.tokens, a.total - first), n = a.n;
    if (threadIdx.x < n) {
        turns[threadIdx.x] = a.turns[threadIdx.x];
        axis[threadIdx.x] = a.axis[threadIdx.x];
    }
    pdl_wait();
    __syncthreads();
    for (int i = threadIdx.x; i < here * n; i += kNT) {
        const int t = i / n, j = i - t * n;
        const long long tok = first + t, b = tok / a.L;
        const double z = a.pos[b * a.pos_batch + (tok - b * a.L) * a.axes + axis[j]] * turns[j];
        float2 v;
        sincospif((float)(2.0 * (z - rint(z))), &v.y, &v.x);
        cs[i] = v;
    }
    __syncthreads();
    const int units = n / V, rest = (a.d - 2 * n) / 4;         // units of a head, and vectors of its channels that are not turned
    const int per = units + rest, heads = a.heads[0] + a.heads[1];
    for (int i = threadIdx.x; i < here * heads * per; i += kNT) {
        const int t = i / (heads * per), r = i - t * heads * per, hh = r / per, u = r - hh * per;
        const int which = hh >= a.heads[0], h = which ? hh - a.heads[0] : hh;
        const long long tok = first + t, b = tok / a.L, l = tok - b * a.L;
        const T *x = (const T *)a.x[which] + b * a.xb[which] + l * a.xt[which] + (long long)h * a.d;
        T *y = (T *)a.y[which] + b * a.yb[which] + l * a.yt[which] + (long long)h * a.d;
        if (u >= units) {
            const int c = 2 * n + (u - units) * 4;
#pragma unroll
            for (int e = 0; e < 4; ++e) y[c + e] = x[c + e];
            continue;
        }
        const float2 *w = cs + t * n + u * V;
        if constexpr (INTER) {
            float f[2 * V];
            ldv<T, 2 * V>(x + u * 2 * V, f);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float p = f[2 * e], q = f[2 * e + 1];
                f[2 * e] = p * w[e].x - q * w[e].y;
                f[2 * e + 1] = p * w[e].y + q * w[e].x;
            }
            stv<T, 2 * V>(y + u * 2 * V, f);
        } else {
            float p[V], q[V];
            ldv<T, V>(x + u * V, p);
            ldv<T, V>(x + n + u * V, q);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float s = p[e], c = q[e];
                p[e] = s * w[e].x - c * w[e].y;
                q[e] = s * w[e].y + c * w[e].x;
            }
            stv<T, V>(y + u * V, p);
            stv<T, V>(y + n + u * V, q);
        }
    }
    pdl_launch_dependents();
}

template <typename T, int V, bool INTER>
dig_status go(const RopeArgs &a, cudaStream_t stream)
{
    KernelTimer t(KID_ROPE, stream);
    return cuda_ok(launch_pdl(rope<T, V, INTER>, dim3((unsigned)((a.total + a.tokens - 1) / a.tokens)), dim3(kNT), 0, stream, a));
}

}  // namespace

dig_status launch_rope(const void *q, const void *k, const long long *strides, const int *positions, int pos_batches, int n_axes,
                       const double *freqs, const int *axes, int n_pairs, void *q_out, void *k_out, int B, int L, int H, int H_k, int d,
                       bool interleaved, bool inverse, int dtype, cudaStream_t stream)
{
    RopeArgs a{};
    const int heads[2] = {H, k ? H_k : 0};
    const void *x[2] = {q, k};
    void *y[2] = {q_out, k_out};
    for (int i = 0; i < 2; ++i) {
        a.x[i] = x[i]; a.y[i] = y[i]; a.heads[i] = heads[i];
        a.yt[i] = (long long)heads[i] * d; a.yb[i] = a.yt[i] * L;
        a.xb[i] = strides ? strides[2 * i] : a.yb[i];
        a.xt[i] = strides ? strides[2 * i + 1] : a.yt[i];
        if (x[i] == y[i]) { a.yb[i] = a.xb[i]; a.yt[i] = a.xt[i]; }
    }
    a.pos = positions; a.pos_batch = pos_batches > 1 ? (long long)L * n_axes : 0;
    a.L = L; a.d = d; a.n = n_pairs; a.axes = n_axes; a.total = (long long)B * L;
    a.tokens = (int)(a.total / (148 * 8));
    a.tokens = a.tokens < 1 ? 1 : a.tokens > kMaxTokens ? kMaxTokens : a.tokens;
    if (a.total > 0x7fffffffll) return DIG_ERR_UNSUPPORTED;
    for (int i = 0; i < n_pairs; ++i) {
        a.turns[i] = (inverse ? -freqs[i] : freqs[i]) * 0.15915494309189533577;
        a.axis[i] = (unsigned char)axes[i];
    }
    const bool f = dtype == DIG_F32;
    if (interleaved) {
        if (f) return n_pairs % 2 == 0 ? go<float, 2, true>(a, stream) : go<float, 1, true>(a, stream);
        return n_pairs % 4 == 0 ? go<__nv_bfloat16, 4, true>(a, stream) : go<__nv_bfloat16, 1, true>(a, stream);
    }
    if (f) return n_pairs % 4 == 0 ? go<float, 4, false>(a, stream) : go<float, 1, false>(a, stream);
    return n_pairs % 8 == 0 ? go<__nv_bfloat16, 8, false>(a, stream) : n_pairs % 4 == 0 ? go<__nv_bfloat16, 4, false>(a, stream) : go<__nv_bfloat16, 1, false>(a, stream);
}

}  // namespace dig
