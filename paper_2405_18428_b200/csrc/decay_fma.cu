// Linear attention with a decay for each head in fp32 arithmetic (equations in decay.cuh): one CTA per segment of a sequence walks
// over tiles of 64 positions with the state in shared memory.  Serves fp32 storage, whose products have to be fp32-accurate.  A thread has 4 x 4
// scores, rows of results or state elements at a time; bound by latency: three to five warps on a scheduler issue in every second cycle, the FMA pipes
// are 27 to 38 % busy, and a tile's loads are waited for before its products (12 heads of 4096 tokens, 64 channels: 82 us with the local pass, 17 TFLOP/s).
#include "decay.cuh"

namespace dig {
namespace decay {
namespace {

constexpr int T = kTileFma, NT = 256, LDP = T + 4;

// Rows of a tile to shared memory, stride d + 4 floats (a step of one row is a step of 4 banks); rows behind the end zero.  Asynchronous:
// loaded through registers, 16 bytes at a time, a tile's loads waited for memory four times over.
__device__ __forceinline__ void load_rows(float *dst, const Rows &r, int d, int b, int h, const int (&tok)[4])
{
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    const float *base = (const float *)r.p + (size_t)b * r.batch + (size_t)(h / r.share) * d;
    const uint32_t to = (uint32_t)__cvta_generic_to_shared(dst);
#pragma unroll
    for (int i = 0; i < 4; ++i)
        for (int c = tx * 4; c < d; c += 64)
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;"
                         :: "r"(to + ((ty + 16 * i) * (d + 4) + c) * 4), "l"(base + (size_t)max(tok[i], 0) * r.token + c), "r"(tok[i] >= 0 ? 16 : 0) : "memory");
}
__device__ __forceinline__ void loads_done() { asm volatile("cp.async.wait_all;" ::: "memory"); }

__device__ __forceinline__ float dot4(float4 x, float4 y, float s) { return fmaf(x.x, y.x, fmaf(x.y, y.y, fmaf(x.z, y.z, fmaf(x.w, y.w, s)))); }
__device__ __forceinline__ void axpy4(float4 &s, float w, float4 x)
{
    s.x = fmaf(w, x.x, s.x); s.y = fmaf(w, x.y, s.y); s.z = fmaf(w, x.z, s.z); s.w = fmaf(w, x.w, s.w);
}
__device__ __forceinline__ float4 scaled(float4 x, float w) { return make_float4(x.x * w, x.y * w, x.z * w, x.w * w); }

// o[i] += rows ty + 16 i of A times B[..][c .. c + 3], over n (a multiple of 4) columns of A; LOWER: A is a lower triangle, of which what lies behind
// a row is neither read as a factor nor, where it is NaN or infinite in B, spread.
template <bool LOWER>
__device__ __forceinline__ void rows4(float4 (&o)[4], const float *A, int lda, const float *B, int ldb, int ty, int c, int n)
{
#pragma unroll 1
    for (int j = 0; j < n; j += 4) {
        float4 p[4], x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            p[i] = *reinterpret_cast<const float4 *>(A + (ty + 16 * i) * lda + j);
            x[i] = *reinterpret_cast<const float4 *>(B + (j + i) * ldb + c);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int last = ty + 16 * i;
            if (!LOWER || j + 3 <= last) {
                axpy4(o[i], p[i].x, x[0]); axpy4(o[i], p[i].y, x[1]); axpy4(o[i], p[i].z, x[2]); axpy4(o[i], p[i].w, x[3]);
            } else if (j <= last) {
                axpy4(o[i], p[i].x, x[0]);
                if (j + 1 <= last) axpy4(o[i], p[i].y, x[1]);
                if (j + 2 <= last) axpy4(o[i], p[i].z, x[2]);
            }
        }
    }
}

template <bool LOCAL>
__global__ void __launch_bounds__(NT) decay_fma(const __grid_constant__ Args a)
{
    if (LOCAL && blockIdx.x == a.nseg - 1) {                     // enters no segment
        pdl_wait();
        pdl_launch_dependents();
        return;
    }
    extern __shared__ float4 smem4[];
    float *sm = reinterpret_cast<float *>(smem4);
    const Pass &ps = a.pass[blockIdx.z];
    const int seg = blockIdx.x, bh = blockIdx.y, b = bh / a.H, h = bh - b * a.H, dk = ps.dk, dv = ps.dv, ldk = dk + 4, ldv = dv + 4;
    float *X = sm, *K = X + dk * ldv, *V = K + T * ldk, *pw = V + T * ldv, *Q = pw + T + 4, *P = Q + T * ldk;
    const float lam = a.lam.v[h];
    const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
    if (tid <= T) pw[tid] = exp2_of(lam * tid);
    pdl_wait();
    const int n = length_of(a.lengths, a.L, b);
    const size_t dd = (size_t)dk * dv;
    float *local = ps.local + ((size_t)bh * a.nseg + seg) * dd;
    const float *x0 = LOCAL ? nullptr : seg > 0 ? local : ps.x0 ? ps.x0 + (size_t)bh * dd : nullptr;
    const bool turned = seg > 0 ? ps.local_transposed : ps.x_transposed;
    if (x0 && turned) {
        for (int c = ty; c < dv; c += 16)
            for (int r = tx; r < dk; r += 16) X[r * ldv + c] = x0[c * dk + r];
    } else {
        for (int r = ty; r < dk; r += 16)
            for (int c = tx * 4; c < dv; c += 64) *reinterpret_cast<float4 *>(X + r * ldv + c) = x0 ? load4(x0 + r * dv + c) : make_float4(0.f, 0.f, 0.f, 0.f);
    }
    const int tiles = (a.L + T - 1) / T, t1 = min((seg + 1) * a.G, tiles);
    float *end = !LOCAL && ps.x_end && seg == a.nseg - 1 ? ps.x_end + bh * dd : nullptr;         // the final state is wanted, and this is the last segment
    for (int t = seg * a.G; t < t1; ++t) {
        const int p0 = t * T, rows = min(T, n - p0), lead = p0 == 0 ? ps.first : 1;
        __syncthreads();
        int tok[4];                              // of rows ty + 16 i
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int p = p0 + ty + 16 * i;
            tok[i] = p < n ? scan_token(p, ps.dir, a.gh, a.gw, n) : -1;
        }
        if (rows > 0) {
            load_rows(K, ps.k, dk, b, h, tok);
            load_rows(V, ps.v, dv, b, h, tok);
            if (!LOCAL) load_rows(Q, ps.q, dk, b, h, tok);
            loads_done();
        }
        __syncthreads();
        if (!LOCAL) {
            if (rows > 0) {
                float s[4][4] = {};
                for (int c = 0; c < dk; c += 4) {
                    float4 qv[4], kv[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        qv[i] = *reinterpret_cast<const float4 *>(Q + (ty + 16 * i) * ldk + c);
                        kv[i] = *reinterpret_cast<const float4 *>(K + (tx + 16 * i) * ldk + c);
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int j = 0; j <= i; ++j) s[i][j] = dot4(qv[i], kv[j], s[i][j]);           // blocks of 16 x 16 behind the diagonal are left out
                }
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int r = ty + 16 * i, c = tx + 16 * j;
                        P[r * LDP + c] = r >= c ? s[i][j] * pw[r - c] : 0.f;
                    }
            }
            __syncthreads();
            const size_t out = (size_t)a.H * dv;
            for (int c = tx * 4; c < dv; c += 64) {
                float4 o[4] = {}, e[4] = {};
                if (rows > 0) {
                    rows4<true>(o, P, LDP, V, ldv, ty, c, T);
                    rows4<false>(e, Q, ldk, X, ldv, ty, c, dk);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int r = ty + 16 * i, p = p0 + r;
                    if (p >= a.L) continue;
                    if (p < n) axpy4(o[i], pw[r] * (lead ? pw[1] : 1.f), e[i]);
                    const size_t at = ((size_t)b * a.L + (p < n ? tok[i] : p)) * out + (size_t)h * dv + c;
                    const float4 y = p < n ? o[i] : make_float4(0.f, 0.f, 0.f, 0.f);
                    store4((float *)ps.out + at, y);
                }
            }
            __syncthreads();
        }
        if (rows <= 0 || (!LOCAL && t + 1 == t1 && !end)) continue;
        const float whole = pw[rows - 1] * (lead ? pw[1] : 1.f);
        for (int r0 = ty * 4; r0 < dk; r0 += 64)
            for (int c = tx * 4; c < dv; c += 64) {
                float4 x[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) x[i] = scaled(*reinterpret_cast<const float4 *>(X + (r0 + i) * ldv + c), whole);
#pragma unroll 4
                for (int j = 0; j < rows; ++j) {
                    const float4 kv = scaled(*reinterpret_cast<const float4 *>(K + j * ldk + r0), pw[rows - 1 - j]);
                    const float4 vv = *reinterpret_cast<const float4 *>(V + j * ldv + c);
                    axpy4(x[0], kv.x, vv); axpy4(x[1], kv.y, vv); axpy4(x[2], kv.z, vv); axpy4(x[3], kv.w, vv);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) *reinterpret_cast<float4 *>(X + (r0 + i) * ldv + c) = x[i];
            }
    }
    __syncthreads();
    if (LOCAL || end) {
        const float w = end && ps.last && n > 0 ? pw[1] : 1.f;
        for (int r = ty; r < dk; r += 16)
            for (int c = tx * 4; c < dv; c += 64) store4((LOCAL ? local : end) + r * dv + c, scaled(*reinterpret_cast<const float4 *>(X + r * ldv + c), w));
    }
    pdl_launch_dependents();
}

size_t smem_bytes(int dk, int dv, bool local)
{
    const size_t f = (size_t)dk * (dv + 4) + (size_t)T * (dk + 4 + dv + 4) + T + 4 + (local ? 0 : (size_t)T * (dk + 4) + T * LDP);
    return f * 4;
}

template <bool LOCAL>
dig_status launch(const Args &a, cudaStream_t stream)
{
    int segs = a.nseg;
    size_t smem = 0;
    for (int i = 0; i < a.passes; ++i) smem = smem > smem_bytes(a.pass[i].dk, a.pass[i].dv, LOCAL) ? smem : smem_bytes(a.pass[i].dk, a.pass[i].dv, LOCAL);
    dig_status st = ensure_dynamic_smem((const void *)decay_fma<LOCAL>, smem);
    if (st != DIG_OK) return st;
    KernelTimer t(LOCAL ? KID_DECAY_LOCAL : KID_DECAY, stream);
    return cuda_ok(launch_pdl(decay_fma<LOCAL>, dim3(segs, a.B * a.H, a.passes), dim3(NT), smem, stream, a));
}

}  // namespace

dig_status fma_pass(const Args &a, bool local, cudaStream_t stream) { return local ? launch<true>(a, stream) : launch<false>(a, stream); }

}  // namespace decay
}  // namespace dig
