// Rotary positions with several axes.  Pair i of a head's channels is turned by positions[token][axis[i]] * freq[i]; the inverse
// rotation is the gradient of the rotation.  Angles are formed in 64 bits, in turns, and reduced before they are rounded to fp32, with what
// the rounded product leaves and 1 / (2 pi) in two parts: far positions (2^31 at frequency 1) keep angles within 1e-7, the rounding to fp32 (one product with one
// part of 1 / (2 pi): 3.2e-7).
// Moved once: q and k in and out.  A token's angles are computed once by its CTA and serve all of its heads.
#include <cmath>

#include "dig_common.cuh"

namespace dig {
namespace {

constexpr int kMaxPairs = 64, kNT = 256, kMaxTokens = 8, kCtas = 4;          // kCtas: on an SM

constexpr double kTurn = 0x1.45f306dc9c883p-3, kTurnLow = -0x1.6b01ec5417056p-57;            // 1 / (2 pi) and what its rounding leaves

// Division of i < 2^31 through the reciprocal rounded up: the estimate is at most one too large.
struct Div {
    uint32_t d, inv;                 // ceil(2^32 / d)
    __device__ __forceinline__ uint32_t operator()(uint32_t i) const
    {
        if (d == 1) return i;
        const uint32_t q = __umulhi(i, inv);
        return q * d > i ? q - 1 : q;
    }
};
struct RopeArgs {
    const void *x[2];                // q, k (null: none)
    void *y[2];
    long long xb[2], xt[2], yb[2], yt[2];        // batch and token strides in elements
    const int *pos;
    long long pos_batch;
    int heads[2];
    int L, d, n, axes, tokens;       // n: pairs; tokens of a CTA
    Div by_token, by_head;           // units of a token, of a head
    long long total;                 // B * L
    double freqs[kMaxPairs];         // negative for the inverse
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
__device__ __forceinline__ void unpack(const typename Vec<T, V>::U &u, float (&f)[V])
{
    if constexpr (sizeof(T) == 2 && V > 1) {
        const uint32_t *w = reinterpret_cast<const uint32_t *>(&u);
#pragma unroll
        for (int i = 0; i < V; i += 2) { f[i] = lo_f(w[i / 2]); f[i + 1] = hi_f(w[i / 2]); }
    } else {
        const T *e = reinterpret_cast<const T *>(&u);
#pragma unroll
        for (int i = 0; i < V; ++i) f[i] = (float)e[i];
    }
}
template <typename T, int V>
__device__ __forceinline__ void stv(T *p, const float (&f)[V])
{
    using U = typename Vec<T, V>::U;
    U u;
    if constexpr (sizeof(T) == 2 && V > 1) {
        uint32_t *w = reinterpret_cast<uint32_t *>(&u);
#pragma unroll
        for (int i = 0; i < V; i += 2) {
            const __nv_bfloat162 t = __floats2bfloat162_rn(f[i], f[i + 1]);
            w[i / 2] = *reinterpret_cast<const uint32_t *>(&t);
        }
    } else {
        T *e = reinterpret_cast<T *>(&u);
#pragma unroll
        for (int i = 0; i < V; ++i) e[i] = (T)f[i];
    }
    *reinterpret_cast<U *>(p) = u;
}

template <int V>
__device__ __forceinline__ void angles(const float *p, float (&f)[V])
{
    if constexpr (V % 4 == 0) {
#pragma unroll
        for (int i = 0; i < V; i += 4) *reinterpret_cast<float4 *>(f + i) = load4(p + i);
    } else if constexpr (V == 2) *reinterpret_cast<float2 *>(f) = *reinterpret_cast<const float2 *>(p);
    else f[0] = p[0];
}

// V pairs per thread and turn: neighbours (2 i, 2 i + 1) where INTER, else (i, i + n).  kTurns turns' loads are on their way together, the first
// ones while the angles are formed (with the angles first: 48 us for 16384 tokens of 32 heads of 72; 34 so, 4.4 TB/s, where a plain copy of as
// many bytes takes 27).  The widest accesses (eight pairs in bf16, four in fp32, by halves) spill 40 bytes at the 64 registers that four CTAs leave.
constexpr int kTurns = 4;
template <typename T, int V, bool INTER>
__global__ void __launch_bounds__(kNT, kCtas) rope(const __grid_constant__ RopeArgs a)
{
    constexpr int E = INTER ? 2 * V : V, HALVES = INTER ? 1 : 2;
    using U = typename Vec<T, E>::U;
    // apart, so that lanes read consecutive vectors of them
    __shared__ __align__(16) float cosines[kMaxTokens * kMaxPairs], sines[kMaxTokens * kMaxPairs];
    __shared__ double freqs[kMaxPairs];
    __shared__ int axis[kMaxPairs];
    __shared__ long long xo[2][kMaxTokens], yo[2][kMaxTokens];               // where a token's q and k stand
    const long long first = (long long)blockIdx.x * a.tokens;
    const int here = (int)min((long long)a.tokens, a.total - first), n = a.n;
    if (threadIdx.x < n) {
        freqs[threadIdx.x] = a.freqs[threadIdx.x];
        axis[threadIdx.x] = a.axis[threadIdx.x];
    }
    if (threadIdx.x < 2 * here) {
        const int t = threadIdx.x >> 1, w = threadIdx.x & 1;
        const uint32_t tok = (uint32_t)(first + t), b = tok / (uint32_t)a.L, l = tok - b * a.L;          // tokens fit 31 bits
        xo[w][t] = b * a.xb[w] + l * a.xt[w];
        yo[w][t] = b * a.yb[w] + l * a.yt[w];
    }
    const uint32_t units = n / V, heads = a.heads[0] + a.heads[1], per = heads * units, count = here * per;
    // unit i: token, tensor, place in a token, pair
    auto place = [&](uint32_t i, uint32_t &t, int &which, uint32_t &h, uint32_t &pair) {
        t = a.by_token(i);
        const uint32_t r = i - t * per, hh = a.by_head(r), u = r - hh * units;
        which = hh >= (uint32_t)a.heads[0];
        h = (which ? hh - a.heads[0] : hh) * a.d + u * E;
        pair = u * V;
    };
    U raw[kTurns][HALVES];
    uint32_t to[kTurns], pair[kTurns];               // place in the token's output, token and tensor; angles
    auto load = [&](uint32_t i0) {
#pragma unroll
        for (int m = 0; m < kTurns; ++m) {
            const uint32_t i = i0 + m * kNT;
            if (i < count) {
                uint32_t t, h, p;
                int which;
                place(i, t, which, h, p);
                to[m] = h << 4 | t << 1 | which;
                pair[m] = t * n + p;
                const T *x = (const T *)a.x[which] + xo[which][t] + h;
                raw[m][0] = *reinterpret_cast<const U *>(x);
                if constexpr (!INTER) raw[m][1] = *reinterpret_cast<const U *>(x + n);
            }
        }
    };
    __syncthreads();
    pdl_wait();
    load(threadIdx.x);
    for (int i = threadIdx.x; i < here * n; i += kNT) {
        const int t = i / n, j = i - t * n;
        const uint32_t tok = (uint32_t)(first + t), b = tok / (uint32_t)a.L;
        const double p = a.pos[b * a.pos_batch + (long long)(tok - b * a.L) * a.axes + axis[j]], f = freqs[j], z = __dmul_rn(p, f), low = fma(p, f, -z);
        const double turn = fma(low, kTurn, fma(z, kTurnLow, fma(z, kTurn, -rint(z * kTurn))));
        sincospif((float)(2.0 * turn), sines + i, cosines + i);
    }
    __syncthreads();
    for (uint32_t i0 = threadIdx.x; i0 < count; i0 += kTurns * kNT) {
        if (i0 > threadIdx.x) load(i0);
#pragma unroll
        for (int m = 0; m < kTurns; ++m) {
            const uint32_t i = i0 + m * kNT;
            if (i >= count) break;
            const int which = to[m] & 1;
            T *y = (T *)a.y[which] + yo[which][to[m] >> 1 & 7] + (to[m] >> 4);
            float f[E];
            __align__(16) float co[V], si[V];
            angles<V>(cosines + pair[m], co);
            angles<V>(sines + pair[m], si);
            unpack<T, E>(raw[m][0], f);
            if constexpr (INTER) {
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float p = f[2 * e], q = f[2 * e + 1];
                    f[2 * e] = p * co[e] - q * si[e];
                    f[2 * e + 1] = p * si[e] + q * co[e];
                }
                stv<T, E>(y, f);
            } else {
                float g[E];
                unpack<T, E>(raw[m][HALVES - 1], g);
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float p = f[e], q = g[e];
                    f[e] = p * co[e] - q * si[e];
                    g[e] = p * si[e] + q * co[e];
                }
                stv<T, E>(y, f);
                stv<T, E>(y + n, g);
            }
        }
    }
    // channels that are not turned, four at a time
    const uint32_t rest = (a.d - 2 * n) / 4;
    for (uint32_t i = threadIdx.x; i < here * heads * rest; i += kNT) {
        const uint32_t t = i / (heads * rest), r = i - t * heads * rest, hh = r / rest;
        const int which = hh >= (uint32_t)a.heads[0];
        const size_t h = (size_t)(which ? hh - a.heads[0] : hh) * a.d + 2 * n + (r - hh * rest) * 4;
        const T *x = (const T *)a.x[which] + xo[which][t] + h;
        T *y = (T *)a.y[which] + yo[which][t] + h;
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = x[e];
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
    for (int i = 0; i < (k ? 2 : 1); ++i) {              // without keys the strides may end with those of q
        a.x[i] = x[i]; a.y[i] = y[i]; a.heads[i] = heads[i];
        a.yt[i] = (long long)heads[i] * d; a.yb[i] = a.yt[i] * L;
        a.xb[i] = strides ? strides[2 * i] : a.yb[i];
        a.xt[i] = strides ? strides[2 * i + 1] : a.yt[i];
        if (x[i] == y[i]) { a.yb[i] = a.xb[i]; a.yt[i] = a.xt[i]; }
    }
    a.pos = positions; a.pos_batch = pos_batches > 1 ? (long long)L * n_axes : 0;
    a.L = L; a.d = d; a.n = n_pairs; a.axes = n_axes; a.total = (long long)B * L;
    if (a.total > 0x7fffffffll) return DIG_ERR_UNSUPPORTED;
    for (int i = 0; i < n_pairs; ++i) {
        a.freqs[i] = inverse ? -freqs[i] : freqs[i];
        a.axis[i] = (unsigned char)axes[i];
    }
    const bool f = dtype == DIG_F32;
    const int v = interleaved ? (f ? (n_pairs % 2 == 0 ? 2 : 1) : n_pairs % 4 == 0 ? 4 : 1) : f ? (n_pairs % 4 == 0 ? 4 : 1) : n_pairs % 8 == 0 ? 8 : n_pairs % 4 == 0 ? 4 : 1;
    const uint32_t units = n_pairs / v, per = units * (heads[0] + heads[1]);
    // The number of tokens with which the rounds of CTAs take the fewest turns, the largest of those, or the smallest where one round holds
    // all (16384 tokens of 32 heads of 72 channels, 7 tokens a CTA: 34 us; 8, the most that there are angles for, 36).
    long long least = 0;
    for (int t = kMaxTokens; t >= 1; --t) {
        const long long ctas = (a.total + t - 1) / t, rounds = (ctas + 148 * kCtas - 1) / (148 * kCtas), turns = rounds * ((t * per + kNT - 1) / kNT);
        if (least == 0 || turns < least || (turns == least && rounds == 1)) {
            least = turns;
            a.tokens = t;
        }
    }
    a.by_head = {units, 0xffffffffu / units + 1};
    a.by_token = {per, 0xffffffffu / per + 1};
    using bf16 = __nv_bfloat16;
    if (interleaved) {
        if (f) return v == 2 ? go<float, 2, true>(a, stream) : go<float, 1, true>(a, stream);
        return v == 4 ? go<bf16, 4, true>(a, stream) : go<bf16, 1, true>(a, stream);
    }
    if (f) return v == 4 ? go<float, 4, false>(a, stream) : go<float, 1, false>(a, stream);
    return v == 8 ? go<bf16, 8, false>(a, stream) : v == 4 ? go<bf16, 4, false>(a, stream) : go<bf16, 1, false>(a, stream);
}

}  // namespace dig
