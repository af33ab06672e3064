// Layer norm over rows of D values, forward and backward, with the affine parameters of all rows or of groups of rows.
//   y = xh w + b,  xh = (x - mean) r,  r = 1 / sqrt(var + eps)
//   dx = r (g - mean(g) - xh mean(g xh)),  g = w dy;   dw = sum of dy xh,  db = sum of dy over a group's rows
// A row stays in registers between its sums, the variance is taken about the mean, and everything is fp32.  Bound by memory: forward
// x in, y out; backward x and dy in, dx out, and the partial sums of dw and db.
#include "dig_common.cuh"

namespace dig {
namespace {

constexpr int kSms = 148;

template <typename T, int W>
__device__ __forceinline__ void load_w(const T *p, float (&f)[W])
{
    if constexpr (W == 1) f[0] = (float)p[0];
    else {
#pragma unroll
        for (int i = 0; i < W; i += 4) {
            const float4 x = load4(p + i);
            f[i] = x.x; f[i + 1] = x.y; f[i + 2] = x.z; f[i + 3] = x.w;
        }
    }
}
template <typename T, int W>
__device__ __forceinline__ void store_w(T *p, const float (&f)[W])
{
    if constexpr (W == 1) p[0] = (T)f[0];
    else {
#pragma unroll
        for (int i = 0; i < W; i += 4) store4(p + i, make_float4(f[i], f[i + 1], f[i + 2], f[i + 3]));
    }
}

// Sum of a pair over the threads of a row: a warp's, or all of the CTA's.  `slot`: 2 * 32 floats of shared memory that the sum before
// last used.
__device__ __forceinline__ float2 row_sum(float2 v, bool warp, float2 *slot)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        v.x += __shfl_xor_sync(0xffffffffu, v.x, o);
        v.y += __shfl_xor_sync(0xffffffffu, v.y, o);
    }
    if (warp) return v;
    if ((threadIdx.x & 31) == 0) slot[threadIdx.x >> 5] = v;
    __syncthreads();
    float2 s = make_float2(0.f, 0.f);
    for (int i = 0; i < (int)(blockDim.x >> 5); ++i) { s.x += slot[i].x; s.y += slot[i].y; }
    return s;
}

// NV vectors of W values per thread; a row per warp (WARP) or per CTA.
template <typename T, int W, int NV, bool WARP>
__global__ void __launch_bounds__(WARP ? 256 : 1024) ln_fwd(const T *__restrict__ x, const float *__restrict__ w, const float *__restrict__ b, T *__restrict__ y,
                                                            long long rows, long long group_rows, int D, float eps)
{
    __shared__ float2 slots[2][32];
    const int lane = WARP ? threadIdx.x & 31 : threadIdx.x, width = WARP ? 32 : blockDim.x;
    const long long step = WARP ? (long long)gridDim.x * (blockDim.x >> 5) : gridDim.x;
    const float n = D;               // divided by, not multiplied by its inverse: a row of one value has that value as its mean
    pdl_wait();
    for (long long row = WARP ? (long long)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5) : blockIdx.x; row < rows; row += step) {
        const T *xr = x + row * D;
        float f[NV][W];
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (lane + i * width) * W;
            if (c < D) load_w<T, W>(xr + c, f[i]);
            else {
#pragma unroll
                for (int e = 0; e < W; ++e) f[i][e] = 0.f;
            }
#pragma unroll
            for (int e = 0; e < W; ++e) s += f[i][e];
        }
        const float m = row_sum(make_float2(s, 0.f), WARP, slots[0]).x / n;
        s = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const bool in = (lane + i * width) * W < D;
#pragma unroll
            for (int e = 0; e < W; ++e) {
                f[i][e] -= m;
                s = in ? fmaf(f[i][e], f[i][e], s) : s;
            }
        }
        const float r = rsqrtf(row_sum(make_float2(s, 0.f), WARP, slots[1]).x / n + eps);
        const long long at = row / group_rows * D;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (lane + i * width) * W;
            if (c >= D) continue;
            float ww[W], bb[W];
            if (w) load_w<float, W>(w + at + c, ww);
            if (b) load_w<float, W>(b + at + c, bb);
#pragma unroll
            for (int e = 0; e < W; ++e) f[i][e] = fmaf(f[i][e] * r, w ? ww[e] : 1.f, b ? bb[e] : 0.f);
            store_w<T, W>(y + row * D + c, f[i]);
        }
    }
    pdl_launch_dependents();
}

// A CTA has every gridDim.x-th row of group blockIdx.y; its sums of dw and db go to part[group][CTA][2][D], or straight to dw and db
// where it is the group's only one.
template <typename T, int W, int NV>
__global__ void __launch_bounds__(1024) ln_bwd(const T *__restrict__ x, const T *__restrict__ dy, const float *__restrict__ w, T *__restrict__ dx, float *__restrict__ dw,
                                               float *__restrict__ db, float *__restrict__ part, long long group_rows, int D, float eps)
{
    __shared__ float2 slots[2][32];
    const int width = blockDim.x;
    const float n = D;               // divided by, not multiplied by its inverse: a row of one value has that value as its mean
    const long long row0 = (long long)blockIdx.y * group_rows;
    float ww[NV][W], aw[NV][W] = {}, ab[NV][W] = {};
    pdl_wait();
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (threadIdx.x + i * width) * W;
#pragma unroll
        for (int e = 0; e < W; ++e) ww[i][e] = 1.f;
        if (w && c < D) load_w<float, W>(w + (long long)blockIdx.y * D + c, ww[i]);
    }
    for (long long j = blockIdx.x; j < group_rows; j += gridDim.x) {
        const long long at = (row0 + j) * D;
        float f[NV][W], g[NV][W];
        float2 s = make_float2(0.f, 0.f);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (threadIdx.x + i * width) * W;
            if (c < D) {
                load_w<T, W>(x + at + c, f[i]);
                load_w<T, W>(dy + at + c, g[i]);
            } else {
#pragma unroll
                for (int e = 0; e < W; ++e) f[i][e] = g[i][e] = 0.f;
            }
#pragma unroll
            for (int e = 0; e < W; ++e) {
                s.x += f[i][e];
                s.y = fmaf(g[i][e], ww[i][e], s.y);
            }
        }
        s = row_sum(s, false, slots[0]);
        const float m = s.x / n, mg = s.y / n;
        s = make_float2(0.f, 0.f);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const bool in = (threadIdx.x + i * width) * W < D;
#pragma unroll
            for (int e = 0; e < W; ++e) {
                f[i][e] = in ? f[i][e] - m : 0.f;
                s.x = fmaf(f[i][e], f[i][e], s.x);
                s.y = fmaf(g[i][e] * ww[i][e], f[i][e], s.y);
            }
        }
        s = row_sum(s, false, slots[1]);
        const float r = rsqrtf(s.x / n + eps), mx = s.y * r / n;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (threadIdx.x + i * width) * W;
            if (c >= D) continue;
            float o[W];
#pragma unroll
            for (int e = 0; e < W; ++e) {
                const float xh = f[i][e] * r;
                o[e] = r * (g[i][e] * ww[i][e] - mg - xh * mx);
                aw[i][e] = fmaf(g[i][e], xh, aw[i][e]);
                ab[i][e] += g[i][e];
            }
            store_w<T, W>(dx + at + c, o);
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
        if (pw) store_w<float, W>(pw + c, aw[i]);
        if (pb) store_w<float, W>(pb + c, ab[i]);
    }
}

// Sums part[group][CTA][2][D] over the CTAs, in a fixed order: eight threads share a value's CTAs.
__global__ void __launch_bounds__(256) ln_sum(const float *__restrict__ part, float *__restrict__ dw, float *__restrict__ db, int ctas, int D)
{
    __shared__ float s[8][33];
    const int c = blockIdx.x * 32 + (threadIdx.x & 31), sub = threadIdx.x >> 5, n = 2 * D;
    pdl_wait();
    pdl_launch_dependents();
    float t = 0.f;
    if (c < n)
        for (int i = sub; i < ctas; i += 8) t += part[((long long)blockIdx.y * ctas + i) * n + c];
    s[sub][threadIdx.x & 31] = t;
    __syncthreads();
    if (sub || c >= n) return;
#pragma unroll
    for (int i = 1; i < 8; ++i) t += s[i][threadIdx.x];
    float *out = c < D ? dw : db;
    if (out) out[(long long)blockIdx.y * D + (c < D ? c : c - D)] = t;
}

template <typename T, int W, int NV, bool WARP>
dig_status go_fwd(const void *x, const float *w, const float *b, void *y, long long rows, long long group_rows, int D, float eps, int threads, cudaStream_t stream)
{
    const long long per = WARP ? 8 : 1, blocks = (rows + per - 1) / per, most = (long long)kSms * (2048 / (WARP ? 256 : threads)) * 4;
    KernelTimer t(KID_LN_FWD, stream);
    return cuda_ok(launch_pdl(ln_fwd<T, W, NV, WARP>, dim3((unsigned)(blocks < most ? blocks : most)), dim3(WARP ? 256 : threads), 0, stream, (const T *)x, w, b, (T *)y, rows,
                              group_rows, D, eps));
}
template <typename T, int W>
dig_status pick_fwd(const void *x, const float *w, const float *b, void *y, long long rows, long long group_rows, int D, float eps, cudaStream_t s)
{
    const int vecs = D / W;
    if (vecs <= 32) return go_fwd<T, W, 1, true>(x, w, b, y, rows, group_rows, D, eps, 32, s);
    if (vecs <= 64) return go_fwd<T, W, 2, true>(x, w, b, y, rows, group_rows, D, eps, 32, s);
    if (vecs <= 96) return go_fwd<T, W, 3, true>(x, w, b, y, rows, group_rows, D, eps, 32, s);
    if (vecs <= 160) return go_fwd<T, W, 5, true>(x, w, b, y, rows, group_rows, D, eps, 32, s);
    if (vecs <= 256) return go_fwd<T, W, 8, true>(x, w, b, y, rows, group_rows, D, eps, 32, s);
    const int nv = vecs <= 4096 ? 4 : 8, threads = ((vecs + nv - 1) / nv + 31) / 32 * 32;
    return nv == 4 ? go_fwd<T, W, 4, false>(x, w, b, y, rows, group_rows, D, eps, threads, s) : go_fwd<T, W, 8, false>(x, w, b, y, rows, group_rows, D, eps, threads, s);
}

// Threads of a backward CTA and CTAs of a group.
template <int W> int bwd_nv(int D) { return D / W <= 1024 ? 1 : D / W <= 2048 ? 2 : D / W <= 4096 ? 4 : 8; }
int bwd_ctas(long long group_rows, int groups, int D)
{
    (void)D;
    long long n = (kSms * 4 + groups - 1) / groups;
    return (int)(n < 1 ? 1 : n > group_rows ? group_rows : n);
}

template <typename T, int W, int NV>
dig_status go_bwd(const void *x, const void *dy, const float *w, void *dx, float *dw, float *db, float *part, int ctas, int groups, long long group_rows, int D, float eps,
                  cudaStream_t stream)
{
    const int threads = ((D / W + NV - 1) / NV + 31) / 32 * 32;
    KernelTimer t(KID_LN_BWD, stream);
    return cuda_ok(launch_pdl(ln_bwd<T, W, NV>, dim3(ctas, groups), dim3(threads), 0, stream, (const T *)x, (const T *)dy, w, (T *)dx, dw, db, part, group_rows, D, eps));
}
template <typename T, int W>
dig_status pick_bwd(const void *x, const void *dy, const float *w, void *dx, float *dw, float *db, float *part, int ctas, int groups, long long group_rows, int D, float eps,
                    cudaStream_t s)
{
    switch (bwd_nv<W>(D)) {
        case 1: return go_bwd<T, W, 1>(x, dy, w, dx, dw, db, part, ctas, groups, group_rows, D, eps, s);
        case 2: if constexpr (W < 8) return go_bwd<T, W, 2>(x, dy, w, dx, dw, db, part, ctas, groups, group_rows, D, eps, s);
        case 4: if constexpr (W < 4) return go_bwd<T, W, 4>(x, dy, w, dx, dw, db, part, ctas, groups, group_rows, D, eps, s);
        default: if constexpr (W < 4) return go_bwd<T, W, 8>(x, dy, w, dx, dw, db, part, ctas, groups, group_rows, D, eps, s);
    }
    return DIG_ERR_UNSUPPORTED;
}

}  // namespace

dig_status launch_layernorm_fwd(const void *x, const float *w, const float *b, void *y, long long rows, int groups, int D, float eps, int dtype, cudaStream_t s)
{
    const long long each = rows / groups;
    if (dtype == DIG_F32) return D % 4 == 0 ? pick_fwd<float, 4>(x, w, b, y, rows, each, D, eps, s) : pick_fwd<float, 1>(x, w, b, y, rows, each, D, eps, s);
    return D % 8 == 0 ? pick_fwd<__nv_bfloat16, 8>(x, w, b, y, rows, each, D, eps, s) : pick_fwd<__nv_bfloat16, 1>(x, w, b, y, rows, each, D, eps, s);
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
    const dig_status st = dtype == DIG_F32 ? (D % 4 == 0 ? pick_bwd<float, 4>(x, dy, w, dx, dw, db, part, ctas, groups, each, D, eps, s)
                                                         : pick_bwd<float, 1>(x, dy, w, dx, dw, db, part, ctas, groups, each, D, eps, s))
                                           : (D % 8 == 0 ? pick_bwd<__nv_bfloat16, 8>(x, dy, w, dx, dw, db, part, ctas, groups, each, D, eps, s)
                                                         : pick_bwd<__nv_bfloat16, 1>(x, dy, w, dx, dw, db, part, ctas, groups, each, D, eps, s));
    if (st != DIG_OK || (!dw && !db) || ctas == 1) return st;
    KernelTimer t(KID_LN_SUM, s);
    return cuda_ok(launch_pdl(ln_sum, dim3((2 * D + 31) / 32, groups), dim3(256), 0, s, (const float *)part, dw, db, ctas, D));
}

}  // namespace dig
