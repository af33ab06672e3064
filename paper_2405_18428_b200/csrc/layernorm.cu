// Layer norm over rows of D values, forward and backward, with the affine parameters of all rows or of groups of rows.
//   y = xh w + b,  xh = (x - mean) r,  r = 1 / sqrt(var + eps)
//   dx = r (g - mean(g) - xh mean(g xh)),  g = w dy;   dw = sum of dy xh,  db = sum of dy over a group's rows
// The variance is taken about the mean, everything is fp32.  Moved once: forward x in, y out; backward x and dy in, dx out.
// A CTA is as wide as a row and takes R rows at a time: their loads are on their way together, a turn ahead, the affine parameters and the sums of dw
// and db stay in registers (beyond 4096 values one by one, odd rows, most of them do not fit and spill: 0.8 to 1.5 KB a thread), and an exchange of sums between the warps serves all R rows.  Arithmetic on packed pairs: with one
// multiply-add per value (and a row per warp, its parameters read again for every row) 16384 rows of 1152 in bf16 took 30 us forward,
// 53 backward, bound by instructions; 21 and 29 us so (3.5 and 3.9 TB/s), bound by the turns' exchanges of sums and their barriers.
#include <atomic>
#include <type_traits>

#include "dig_common.cuh"

namespace dig {
namespace {

constexpr int kSms = 148;

// W values as they are stored, and as pairs.  All loads of a turn are asked for before the first is unpacked (unpacked one by one under
// their conditions, each row waited for memory by itself), so addresses are always valid and what is not there is cleared after.
template <typename T, int W> struct Raw;
template <> struct Raw<float, 4> {
    float4 v;
    __device__ __forceinline__ void load(const float *p) { v = load4(p); }
    __device__ __forceinline__ void unpack(float2 *f, bool in) const
    {
        f[0] = in ? make_float2(v.x, v.y) : make_float2(0.f, 0.f);
        f[1] = in ? make_float2(v.z, v.w) : make_float2(0.f, 0.f);
    }
};
template <> struct Raw<__nv_bfloat16, 8> {
    uint4 v;
    __device__ __forceinline__ void load(const __nv_bfloat16 *p) { v = *reinterpret_cast<const uint4 *>(p); }
    __device__ __forceinline__ void unpack(float2 *f, bool in) const
    {
        f[0] = bf2(in ? v.x : 0u); f[1] = bf2(in ? v.y : 0u); f[2] = bf2(in ? v.z : 0u); f[3] = bf2(in ? v.w : 0u);
    }
};
template <> struct Raw<float, 2> {
    float2 v;
    __device__ __forceinline__ void load(const float *p) { v = *reinterpret_cast<const float2 *>(p); }
    __device__ __forceinline__ void unpack(float2 *f, bool in) const { f[0] = in ? v : make_float2(0.f, 0.f); }
};
template <> struct Raw<__nv_bfloat16, 2> {
    uint32_t v;
    __device__ __forceinline__ void load(const __nv_bfloat16 *p) { v = *reinterpret_cast<const uint32_t *>(p); }
    __device__ __forceinline__ void unpack(float2 *f, bool in) const { f[0] = bf2(in ? v : 0u); }
};
template <typename T> struct Raw<T, 1> {
    T v;
    __device__ __forceinline__ void load(const T *p) { v = p[0]; }
    __device__ __forceinline__ void unpack(float2 *f, bool in) const { f[0] = make_float2(in ? (float)v : 0.f, 0.f); }
};
template <int W>
__device__ __forceinline__ void put(float *p, const float2 *f)
{
    if constexpr (W == 1) p[0] = f[0].x;
    else if constexpr (W == 2) *reinterpret_cast<float2 *>(p) = f[0];
    else {
#pragma unroll
        for (int i = 0; i < W / 2; i += 2) store4(p + 2 * i, make_float4(f[i].x, f[i].y, f[i + 1].x, f[i + 1].y));
    }
}
template <int W>
__device__ __forceinline__ void put(__nv_bfloat16 *p, const float2 *f)
{
    if constexpr (W == 1) p[0] = (__nv_bfloat16)f[0].x;
    else if constexpr (W == 2) *reinterpret_cast<__nv_bfloat162 *>(p) = __floats2bfloat162_rn(f[0].x, f[0].y);
    else {
        uint4 u;
        uint32_t *o = &u.x;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 t = __floats2bfloat162_rn(f[i].x, f[i].y);
            o[i] = *reinterpret_cast<const uint32_t *>(&t);
        }
        *reinterpret_cast<uint4 *>(p) = u;
    }
}
// W fp32 parameters.
template <int W>
__device__ __forceinline__ void get_affine(const float *p, float2 *f)
{
    if constexpr (W == 1) f[0] = make_float2(p[0], 0.f);
    else if constexpr (W == 2) f[0] = *reinterpret_cast<const float2 *>(p);
    else {
#pragma unroll
        for (int i = 0; i < W / 4; ++i) {
            const float4 x = load4(p + 4 * i);
            f[2 * i] = make_float2(x.x, x.y);
            f[2 * i + 1] = make_float2(x.z, x.w);
        }
    }
}
__device__ __forceinline__ float2 both(float c) { return make_float2(c, c); }
// s / n, exact where n divides s: a row of one value has that value as its mean.
__device__ __forceinline__ float over(float s, float n, float inv)
{
    const float q = s * inv;
    return fmaf(fmaf(-q, n, s), inv, q);
}

// Sums of N values at a time over a CTA.  Within a warp the values change places with the lanes, so that eight take 9 exchanges instead
// of 40: afterwards lane l has the sum of value l / (32 / N).
template <int N>
__device__ __forceinline__ void cta_sums(float (&v)[N], float *slots)          // slots: [warps][N]
{
    const int lane = threadIdx.x & 31, warps = blockDim.x >> 5;
#pragma unroll
    for (int n = N / 2, o = 16; n > 0; n /= 2, o /= 2) {
#pragma unroll
        for (int i = 0; i < n; ++i) {
            const bool up = lane & o;
            const float keep = up ? v[n + i] : v[i], give = up ? v[i] : v[n + i];
            v[i] = keep + __shfl_xor_sync(0xffffffffu, give, o);
        }
    }
    float s = v[0];
#pragma unroll
    for (int o = 16 / N; o > 0; o /= 2) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (lane % (32 / N) == 0) slots[(threadIdx.x >> 5) * N + lane / (32 / N)] = s;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = slots[i];
    for (int w = 1; w < warps; ++w)
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += slots[w * N + i];
}

// NV vectors of W values a thread, R rows a turn; CTA (x, y): rows R x ..., then R gridDim.x further, of group y.
template <typename T, int W, int NV, int R>
__global__ void __launch_bounds__(512) ln_fwd(const T *__restrict__ x, const float *__restrict__ w, const float *__restrict__ b, T *__restrict__ y, long long group_rows, int D,
                                              float eps)
{
    constexpr int P = W > 1 ? W / 2 : 1;             // pairs of a vector
    __shared__ float slots[2][16 * R];
    const int width = blockDim.x;
    const float n = D, inv = 1.f / n;
    const long long row0 = (long long)blockIdx.y * group_rows, affine = (long long)blockIdx.y * D;
    float2 ww[NV][P], bb[NV][P];
    pdl_wait();
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (threadIdx.x + i * width) * W;
#pragma unroll
        for (int e = 0; e < P; ++e) {
            ww[i][e] = both(1.f);
            bb[i][e] = both(0.f);
        }
        if (w && c < D) get_affine<W>(w + affine + c, ww[i]);
        if (b && c < D) get_affine<W>(b + affine + c, bb[i]);
    }
    Raw<T, W> fx[R][NV];
    auto load = [&](long long j) {
#pragma unroll
        for (int q = 0; q < R; ++q) {
            const T *p = x + (row0 + min(j + q, group_rows - 1)) * D;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = (threadIdx.x + i * width) * W;
                fx[q][i].load(p + (c < D ? c : 0));
            }
        }
    };
    const long long step = (long long)gridDim.x * R;
    load((long long)blockIdx.x * R);
    for (long long j = (long long)blockIdx.x * R; j < group_rows; j += step) {
        float2 f[R][NV][P];
        float s[R];
#pragma unroll
        for (int q = 0; q < R; ++q)
#pragma unroll
            for (int i = 0; i < NV; ++i) fx[q][i].unpack(f[q][i], (threadIdx.x + i * width) * W < D);
        if (j + step < group_rows) load(j + step);
#pragma unroll
        for (int q = 0; q < R; ++q) {
            float2 t = both(0.f);
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int e = 0; e < P; ++e) t = add2(t, f[q][i][e]);
            s[q] = t.x + t.y;
        }
        cta_sums<R>(s, slots[0]);
#pragma unroll
        for (int q = 0; q < R; ++q) {
            const float m = over(s[q], n, inv);
            float2 t = both(0.f);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const bool in = (threadIdx.x + i * width) * W < D;               // else zeros stay zeros
                const float2 off = make_float2(in ? -m : 0.f, in && W > 1 ? -m : 0.f);
#pragma unroll
                for (int e = 0; e < P; ++e) {
                    f[q][i][e] = add2(f[q][i][e], off);
                    t = fma2(f[q][i][e], f[q][i][e], t);
                }
            }
            s[q] = t.x + t.y;
        }
        cta_sums<R>(s, slots[1]);
#pragma unroll
        for (int q = 0; q < R; ++q) {
            if (j + q >= group_rows) break;
            const float2 r = both(rsqrtf(over(s[q], n, inv) + eps));
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = (threadIdx.x + i * width) * W;
                if (c >= D) continue;
#pragma unroll
                for (int e = 0; e < P; ++e) f[q][i][e] = fma2(mul2(f[q][i][e], r), ww[i][e], bb[i][e]);
                put<W>(y + (row0 + j + q) * D + c, f[q][i]);
            }
        }
    }
    pdl_launch_dependents();
}

// Sums of dw and db go to part[group][CTA][2][D], or straight to dw and db where the CTA is the group's only one.
template <typename T, int W, int NV, int R>
__global__ void __launch_bounds__(512) ln_bwd(const T *__restrict__ x, const T *__restrict__ dy, const float *__restrict__ w, T *__restrict__ dx, float *__restrict__ dw,
                                              float *__restrict__ db, float *__restrict__ part, long long group_rows, int D, float eps)
{
    constexpr int P = W > 1 ? W / 2 : 1;
    __shared__ float slots[2][16 * 2 * R];
    const int width = blockDim.x;
    const float n = D, inv = 1.f / n;
    const long long row0 = (long long)blockIdx.y * group_rows;
    float2 ww[NV][P], aw[NV][P], ab[NV][P];
    pdl_wait();
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (threadIdx.x + i * width) * W;
#pragma unroll
        for (int e = 0; e < P; ++e) {
            ww[i][e] = both(1.f);
            aw[i][e] = ab[i][e] = both(0.f);
        }
        if (w && c < D) get_affine<W>(w + (long long)blockIdx.y * D + c, ww[i]);
    }
    Raw<T, W> fx[R][NV], fg[R][NV];
    auto load = [&](long long j) {
#pragma unroll
        for (int q = 0; q < R; ++q) {
            const long long at = (row0 + min(j + q, group_rows - 1)) * D;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = (threadIdx.x + i * width) * W, to = c < D ? c : 0;
                fx[q][i].load(x + at + to);
                fg[q][i].load(dy + at + to);
            }
        }
    };
    const long long step = (long long)gridDim.x * R;
    load((long long)blockIdx.x * R);
    for (long long j = (long long)blockIdx.x * R; j < group_rows; j += step) {
        float2 f[R][NV][P], g[R][NV][P];
        float s[2 * R];
#pragma unroll
        for (int q = 0; q < R; ++q)
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const bool in = (threadIdx.x + i * width) * W < D;
                fx[q][i].unpack(f[q][i], in);
                fg[q][i].unpack(g[q][i], in);
            }
        if (j + step < group_rows) load(j + step);
#pragma unroll
        for (int q = 0; q < R; ++q) {
            float2 t = both(0.f), u = both(0.f);
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int e = 0; e < P; ++e) {
                    t = add2(t, f[q][i][e]);
                    u = fma2(g[q][i][e], ww[i][e], u);
                }
            s[q] = t.x + t.y;
            s[R + q] = u.x + u.y;
        }
        cta_sums<2 * R>(s, slots[0]);
        float mg[R];
#pragma unroll
        for (int q = 0; q < R; ++q) {
            const float m = over(s[q], n, inv);
            mg[q] = s[R + q] * inv;
            float2 t = both(0.f), u = both(0.f);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const bool in = (threadIdx.x + i * width) * W < D;               // else zeros stay zeros
                const float2 off = make_float2(in ? -m : 0.f, in && W > 1 ? -m : 0.f);
#pragma unroll
                for (int e = 0; e < P; ++e) {
                    f[q][i][e] = add2(f[q][i][e], off);
                    t = fma2(f[q][i][e], f[q][i][e], t);
                    u = fma2(mul2(g[q][i][e], ww[i][e]), f[q][i][e], u);
                }
            }
            s[q] = t.x + t.y;
            s[R + q] = u.x + u.y;
        }
        cta_sums<2 * R>(s, slots[1]);
#pragma unroll
        for (int q = 0; q < R; ++q) {
            if (j + q >= group_rows) break;
            // dx = r (w dy) - r mean(g) - (x - mean) r^3 mean(g (x - mean)); r^3 by itself overflows where eps is 1e-26 or less
            const float r = rsqrtf(over(s[q], n, inv) + eps);
            const float2 r2 = both(r), shift = both(-r * mg[q]), slope = both(-r * (r * (r * (s[R + q] * inv))));
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = (threadIdx.x + i * width) * W;
                if (c >= D) continue;
                float2 o[P];
#pragma unroll
                for (int e = 0; e < P; ++e) {
                    o[e] = fma2(f[q][i][e], slope, fma2(mul2(g[q][i][e], ww[i][e]), r2, shift));
                    aw[i][e] = fma2(g[q][i][e], mul2(f[q][i][e], r2), aw[i][e]);
                    ab[i][e] = add2(ab[i][e], g[q][i][e]);
                }
                put<W>(dx + (row0 + j + q) * D + c, o);
            }
        }
    }
    pdl_launch_dependents();
    if (!dw && !db) return;
    float *pw = gridDim.x > 1 ? part + ((long long)blockIdx.y * gridDim.x + blockIdx.x) * 2 * D : dw ? dw + (long long)blockIdx.y * D : nullptr;
    float *pb = gridDim.x > 1 ? pw + D : db ? db + (long long)blockIdx.y * D : nullptr;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (threadIdx.x + i * width) * W;
        if (c >= D) continue;
        if (pw) put<W>(pw + c, aw[i]);
        if (pb) put<W>(pb + c, ab[i]);
    }
}

// Sums part[group][CTA][2][D] over the CTAs, in a fixed order.  FEW: a thread a column (128 groups of 768 values, five CTAs each: 30 us with
// 32 threads a column); else 32 threads share a column's CTAs.
template <bool FEW>
__global__ void __launch_bounds__(1024) ln_sum(const float *__restrict__ part, float *__restrict__ dw, float *__restrict__ db, int ctas, int D)
{
    const int n = 2 * D;
    const float *p = part + (long long)blockIdx.y * ctas * n;
    pdl_wait();
    pdl_launch_dependents();
    int col;
    float t = 0.f;
    if constexpr (FEW) {
        col = blockIdx.x * blockDim.x + threadIdx.x;
        if (col >= n) return;
#pragma unroll 8
        for (int i = 0; i < ctas; ++i) t += p[(long long)i * n + col];
    } else {
        __shared__ float s[32][33];
        const int c = blockIdx.x * 32 + (threadIdx.x & 31), sub = threadIdx.x >> 5;
        if (c < n)
#pragma unroll 8
            for (int i = sub; i < ctas; i += 32) t += p[(long long)i * n + c];
        s[sub][threadIdx.x & 31] = t;
        __syncthreads();
        t = s[threadIdx.x & 31][sub];                // warp `sub` sums the column of the same number
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
        col = blockIdx.x * 32 + sub;
        if ((threadIdx.x & 31) || col >= n) return;
    }
    float *out = col < D ? dw : db;
    if (out) out[(long long)blockIdx.y * D + (col < D ? col : col - D)] = t;
}

// Vectors of a thread (at most 512 threads a CTA), rows of a turn, CTAs of a group.
int vectors(int vecs) { return vecs <= 512 ? 1 : vecs <= 1024 ? 2 : vecs <= 2048 ? 4 : vecs <= 4096 ? 8 : 16; }
constexpr int rows_at_once(int vectors, int pairs, bool backward) { return vectors * pairs <= (backward ? 2 : 4) ? 4 : vectors * pairs <= (backward ? 4 : 8) ? 2 : 1; }
int threads_of(int vecs, int nv) { return ((vecs + nv - 1) / nv + 31) / 32 * 32; }

// CTAs of a group: all that run together, with as equal numbers of turns as can be.
long long even(long long turns, long long room)
{
    if (turns <= room) return turns;
    const long long each = (turns + room - 1) / room;
    return (turns + each - 1) / each;
}
// CTAs of `threads` that share an SM (asked for once per kernel and width: all devices are alike).
template <typename K>
int resident(K kernel, std::atomic<int> (&known)[17], int threads)
{
    int n = known[threads / 32].load();
    if (n == 0) {
        if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kernel, threads, 0) != cudaSuccess || n < 1) n = 1;
        known[threads / 32].store(n);
    }
    return n;
}

template <typename T, int W, int NV>
dig_status go_fwd(const void *x, const float *w, const float *b, void *y, int groups, long long group_rows, int D, float eps, cudaStream_t stream)
{
    constexpr int R = rows_at_once(NV, (W + 1) / 2, false);
    const int threads = threads_of(D / W, NV);
    static std::atomic<int> known[17];
    const long long turns = (group_rows + R - 1) / R, room = ((long long)kSms * resident(ln_fwd<T, W, NV, R>, known, threads) + groups - 1) / groups, n = even(turns, room);
    KernelTimer t(KID_LN_FWD, stream);
    return cuda_ok(launch_pdl(ln_fwd<T, W, NV, R>, dim3((unsigned)n, groups), dim3(threads), 0, stream, (const T *)x, w, b, (T *)y, group_rows, D, eps));
}
template <typename T, int W>
dig_status pick_fwd(const void *x, const float *w, const float *b, void *y, int groups, long long each, int D, float eps, cudaStream_t s)
{
    const int nv = vectors(D / W);
    if (nv == 1) return go_fwd<T, W, 1>(x, w, b, y, groups, each, D, eps, s);
    if (nv == 2) return go_fwd<T, W, 2>(x, w, b, y, groups, each, D, eps, s);
    if constexpr (W < 8) {
        if (nv == 4) return go_fwd<T, W, 4>(x, w, b, y, groups, each, D, eps, s);
        if constexpr (W < 4)
            if (nv == 8) return go_fwd<T, W, 8>(x, w, b, y, groups, each, D, eps, s);
        if constexpr (W < 2) return go_fwd<T, W, 16>(x, w, b, y, groups, each, D, eps, s);
    }
    return DIG_ERR_UNSUPPORTED;
}

// CTAs of a group in the backward pass: as many as run together where rows go by eight values, since each leaves sums of 2 D values.  By D alone,
// not by type: the workspace is asked for without it.  Narrower accesses have more threads to a row and more registers: 128 groups of 768 values in fp32 are
// 768 CTAs where 296 run together, 2.6 rounds.
int bwd_ctas(long long group_rows, int groups, int D)
{
    const int threads = threads_of((D + 7) / 8, vectors((D + 7) / 8));
    const long long turns = (group_rows + 3) / 4, room = ((long long)kSms * (512 / threads) + groups - 1) / groups;
    return (int)even(turns, room);
}
template <typename T, int W, int NV>
dig_status go_bwd(const void *x, const void *dy, const float *w, void *dx, float *dw, float *db, float *part, int ctas, int groups, long long group_rows, int D, float eps,
                  cudaStream_t stream)
{
    KernelTimer t(KID_LN_BWD, stream);
    return cuda_ok(launch_pdl(ln_bwd<T, W, NV, rows_at_once(NV, (W + 1) / 2, true)>, dim3(ctas, groups), dim3(threads_of(D / W, NV)), 0, stream, (const T *)x, (const T *)dy, w, (T *)dx, dw, db,
                              part, group_rows, D, eps));
}
template <typename T, int W>
dig_status pick_bwd(const void *x, const void *dy, const float *w, void *dx, float *dw, float *db, float *part, int ctas, int groups, long long each, int D, float eps, cudaStream_t s)
{
    const int nv = vectors(D / W);
    if (nv == 1) return go_bwd<T, W, 1>(x, dy, w, dx, dw, db, part, ctas, groups, each, D, eps, s);
    if (nv == 2) return go_bwd<T, W, 2>(x, dy, w, dx, dw, db, part, ctas, groups, each, D, eps, s);
    if constexpr (W < 8) {
        if (nv == 4) return go_bwd<T, W, 4>(x, dy, w, dx, dw, db, part, ctas, groups, each, D, eps, s);
        if constexpr (W < 4)
            if (nv == 8) return go_bwd<T, W, 8>(x, dy, w, dx, dw, db, part, ctas, groups, each, D, eps, s);
        if constexpr (W < 2) return go_bwd<T, W, 16>(x, dy, w, dx, dw, db, part, ctas, groups, each, D, eps, s);
    }
    return DIG_ERR_UNSUPPORTED;
}

}  // namespace

// The widest access that rows of D values allow: 16 bytes, two values, or one.  16384 rows in bf16, forward / backward: 1152 values by
// eights 21 / 29 us, 1002 by twos 46 / 66 (one by one 56 / 108), 1001 one by one 56 / 111.
template <typename F>
dig_status with_width(int D, int dtype, F go)
{
    using bf16 = __nv_bfloat16;
    if (dtype == DIG_F32) return D % 4 == 0 ? go(float(), std::integral_constant<int, 4>()) : D % 2 == 0 ? go(float(), std::integral_constant<int, 2>()) : go(float(), std::integral_constant<int, 1>());
    return D % 8 == 0 ? go(bf16(), std::integral_constant<int, 8>()) : D % 2 == 0 ? go(bf16(), std::integral_constant<int, 2>()) : go(bf16(), std::integral_constant<int, 1>());
}

dig_status launch_layernorm_fwd(const void *x, const float *w, const float *b, void *y, long long rows, int groups, int D, float eps, int dtype, cudaStream_t s)
{
    return with_width(D, dtype, [&](auto t, auto width) { return pick_fwd<decltype(t), decltype(width)::value>(x, w, b, y, groups, rows / groups, D, eps, s); });
}

size_t layernorm_bwd_workspace_bytes(long long rows, int groups, int D)
{
    return align256((size_t)bwd_ctas(rows / groups, groups, D) * groups * 2 * D * 4);
}

dig_status launch_layernorm_bwd(const void *x, const void *dy, const float *w, void *dx, float *dw, float *db, long long rows, int groups, int D, float eps, int dtype,
                                float *part, cudaStream_t s)
{
    const long long each = rows / groups;
    const int ctas = bwd_ctas(each, groups, D);
    const dig_status st =
        with_width(D, dtype, [&](auto t, auto width) { return pick_bwd<decltype(t), decltype(width)::value>(x, dy, w, dx, dw, db, part, ctas, groups, each, D, eps, s); });
    if (st != DIG_OK || (!dw && !db) || ctas == 1) return st;
    KernelTimer t(KID_LN_SUM, s);
    if (ctas <= 16) return cuda_ok(launch_pdl(ln_sum<true>, dim3((2 * D + 255) / 256, groups), dim3(256), 0, s, (const float *)part, dw, db, ctas, D));
    return cuda_ok(launch_pdl(ln_sum<false>, dim3((2 * D + 31) / 32, groups), dim3(1024), 0, s, (const float *)part, dw, db, ctas, D));
}

}  // namespace dig
