// Linear attention with a decay for each head on the tcgen05 tensor cores (equations in decay.cuh): bf16 storage, heads of up to
// 128 channels.  A CTA walks over the 128-position tiles of a segment with the state in registers.
//
// The decay is a number per head, so q, k and v are operands as they come: a tile is copied to shared memory (cp.async, 16 bytes a
// thread, any row strides and scan order), S = Q K^T and I = Q X go to tensor memory, threads weigh the scores, P = S . g^(i-j), and
// leave them there as the bf16 A operand of O = P V, and the state takes U = (g^(n-1-j) k_j)^T v_j: X' = g^n X + U.
// Powers are at most 1 everywhere; only within the diagonal blocks of 16 keys they are formed one by one, elsewhere as
// g^(i-j0-15) g^(15-(j-j0)), the second factor the same for all rows.
//
// Roundings to bf16: P, the state where it is an operand, the decayed keys; each 2^-9 of its term on average, as much as the rounding of
// the results.  A state that the caller gets has its decayed keys in two bf16 parts (2^-16).
//
// Tile layout: chunk-major without swizzle, element (row, col) at (col / 8) * (16 R + 16) + 16 row + 2 (col % 8): both operand orientations
// from the same bytes, heads of any multiple of 8, no bank conflicts for rows or columns of 16 bytes.
#include "decay_plan.cuh"
#include "umma.cuh"

namespace dig {
namespace decay {
namespace {

using namespace umma;
using bf16 = __nv_bfloat16;

constexpr int T = kTileTc, NT = 256, CH = T * 16 + 16;

// D: channels that tiles provide for keys and values, the smallest of 64, 80 and 128 that holds both.
template <int D>
struct Cfg {
    static constexpr int NCH = D / 8, KS = D / 16, TILE = NCH * CH, CHX = D * 16 + 16, XT = NCH * CHX;
    static constexpr int HALF = D / 2;                       // columns of a thread
    // tensor memory: scores 0 .. 127, over them the decayed scores of keys 0 .. 63 (0 .. 31) and O; those of keys 64 .. 127 last
    static constexpr int S = 0, P0 = 0, O = 64, I = O + D < 128 ? 128 : O + D, P1 = I + D, COLS = P1 + 32 <= 256 ? 256 : 512;
};

struct Ctl {
    uint64_t bar[2];
    uint32_t tmem;
    int dead;                            // a wait gave up: no more waiting
    int tok[2][T];
};

__host__ __device__ constexpr uint32_t idesc_bf16(int M, int N, bool a_mn, bool b_mn) { return idesc_f16(M, N, a_mn, b_mn) | (1u << 7) | (1u << 10); }
__device__ __forceinline__ uint64_t kmajor(uint32_t a, uint32_t ch) { return make_desc(a, ch, 128, 0); }
__device__ __forceinline__ uint64_t mnmajor(uint32_t a, uint32_t ch) { return make_desc(a, 128, ch, 0); }

// A from tensor memory.  Lanes of the quarters below `skip` keep what they hold.
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, bool accumulate, int skip)
{
    const uint32_t m0 = skip > 0 ? ~0u : 0u, m1 = skip > 1 ? ~0u : 0u, m2 = skip > 2 ? ~0u : 0u, m3 = 0u;
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, {%5, %6, %7, %8}, p;\n\t}"
        :: "r"(d), "r"(a), "l"(b), "r"(idesc), "r"((uint32_t)accumulate), "r"(m0), "r"(m1), "r"(m2), "r"(m3) : "memory");
}
__device__ __forceinline__ void ld16(uint32_t addr, uint32_t (&r)[16])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]),
          "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ld8(uint32_t addr, uint32_t *r)
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ld_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void st8(uint32_t addr, const uint32_t (&r)[8])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
        :: "r"(addr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]) : "memory");
}
__device__ __forceinline__ uint32_t pack(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ float f(uint32_t u) { return __uint_as_float(u); }

// 16 bytes to shared memory, zeros where `bytes` is 0.
__device__ __forceinline__ void copy16(uint32_t dst, const void *src, int bytes)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" :: "r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ __forceinline__ void copy_wait_all() { asm volatile("cp.async.wait_all;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" :: "n"(N) : "memory"); }

__device__ __forceinline__ void zero16(char *p) { *reinterpret_cast<uint4 *>(p) = make_uint4(0, 0, 0, 0); }

// The rows of one operand for this CTA's sequence and head.
struct Src {
    const bf16 *p;
    long long token;
    int nch;                             // chunks of 8 channels
};
__device__ __forceinline__ Src src_of(const Rows &r, int b, int h, int d)
{
    return {(const bf16 *)r.p + (size_t)b * r.batch + (size_t)(h / r.share) * d, r.token, d / 8};
}
// A tile's rows; consecutive threads take the chunks of a row.
__device__ __forceinline__ void load_tile(uint32_t dst, const Src &s, const int *tok)
{
    const uint32_t inv = (0xffffffffu / s.nch) + 1;          // exact for dividends below 2^16, but 2^32 does not fit: one chunk apart
    for (uint32_t i = threadIdx.x; i < (uint32_t)(T * s.nch); i += NT) {
        const uint32_t row = s.nch == 1 ? i : __umulhi(i, inv), c = i - row * s.nch;
        const int t = tok[row];
        copy16(dst + c * CH + row * 16, s.p + (size_t)max(t, 0) * s.token + c * 8, t >= 0 ? 16 : 0);
    }
}
// Token of every row of a tile, -1 behind the end.
__device__ __forceinline__ void tokens(int *tok, const Args &a, int dir, int tile, int n)
{
    if (threadIdx.x < T) {
        const int p = tile * T + threadIdx.x;
        tok[threadIdx.x] = p < n ? scan_token(p, dir, a.gh, a.gw, n) : -1;
    }
}
// Decayed keys, hi + lo: row j times g^(last - j).  Thread: one row, every second chunk.
__device__ __forceinline__ void decay_keys(const char *K, char *hi, char *lo, int nch, float lam, int last, bool exact)
{
    const int j = threadIdx.x & (T - 1);
    const float w = exp2_of(lam * max(last - j, 0));
    for (int c = threadIdx.x / T; c < nch; c += NT / T) {
        const uint4 u = *reinterpret_cast<const uint4 *>(K + c * CH + j * 16);
        uint32_t x[4] = {u.x, u.y, u.z, u.w}, y[4], z[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float p = lo_f(x[i]) * w, q = hi_f(x[i]) * w;
            y[i] = pack(p, q);
            z[i] = pack(p - lo_f(y[i]), q - hi_f(y[i]));
        }
        *reinterpret_cast<uint4 *>(hi + c * CH + j * 16) = make_uint4(y[0], y[1], y[2], y[3]);
        if (exact) *reinterpret_cast<uint4 *>(lo + c * CH + j * 16) = make_uint4(z[0], z[1], z[2], z[3]);
    }
}
__device__ __forceinline__ void wait(Ctl *ctl, int which, uint32_t parity, int *status)
{
    if (*(volatile int *)&ctl->dead) return;
    if (!mbar_wait(&ctl->bar[which], parity, status)) *(volatile int *)&ctl->dead = 1;
}
// U (+)= KT^T V: M = 128, rows beyond the keys' channels are whatever follows in shared memory and are not used.
template <int D>
__device__ __forceinline__ void issue_state(uint32_t d, uint32_t kt, uint32_t v, bool accumulate)
{
    const uint64_t a = mnmajor(kt, CH), b = mnmajor(v, CH);
#pragma unroll
    for (int kk = 0; kk < T / 16; ++kk) mma_f16(d, a + kk * 16, b + kk * 16, idesc_bf16(128, D, true, true), accumulate || kk > 0);
}

// Rows of results: 8 columns of one.
__device__ __forceinline__ void put8(const Pass &ps, size_t at, const float (&o)[8])
{
    if (ps.out_f32) {
        float *p = (float *)ps.out + at;
        store4(p, make_float4(o[0], o[1], o[2], o[3]));
        store4(p + 4, make_float4(o[4], o[5], o[6], o[7]));
    } else {
        *reinterpret_cast<uint4 *>((bf16 *)ps.out + at) = make_uint4(pack(o[0], o[1]), pack(o[2], o[3]), pack(o[4], o[5]), pack(o[6], o[7]));
    }
}

template <int D>
__global__ void __launch_bounds__(NT, D <= 80 ? 2 : 1) decay_pass(const __grid_constant__ Args a, int *status)
{
    using C = Cfg<D>;
    extern __shared__ __align__(128) char sm[];
    __shared__ Ctl ctl;
    const Pass &ps = a.pass[blockIdx.x % a.passes];
    const int seg = blockIdx.x / a.passes, bh = blockIdx.y, b = bh / a.H, h = bh - b * a.H, dk = ps.dk, dv = ps.dv;
    const float lam = a.lam.v[h];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, quarter = warp & 3, half = warp >> 2, row = quarter * 32 + lane;
    const bool exact = true, ends = ps.x_end && a.nseg == 1;
    // decayed keys first: their products read sixteen chunks from their start
    char *KH = sm, *KL = KH + dk / 8 * CH, *Q = KL + (exact ? dk / 8 * CH : 0), *K = Q + C::TILE, *V = K + C::TILE, *X = V + C::TILE;
    const uint32_t kh = smem_u32(KH), kl = smem_u32(KL), q = smem_u32(Q), k = smem_u32(K), v = smem_u32(V), x = smem_u32(X);

    if (warp == 0) tmem_alloc(&ctl.tmem, C::COLS);
    if (tid == 32) {
        mbar_init(&ctl.bar[0], 1);
        mbar_init(&ctl.bar[1], 1);
        ctl.dead = 0;
        fence_barrier_init();
    }
    for (int i = dk / 8 * T + tid; i < C::NCH * T; i += NT) {           // channels that are not there
        zero16(Q + i / T * CH + i % T * 16);
        zero16(K + i / T * CH + i % T * 16);
    }
    for (int i = dv / 8 * T + tid; i < C::NCH * T; i += NT) zero16(V + i / T * CH + i % T * 16);
    float cw[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) cw[i] = exp2_of(lam * (15 - i));

    pdl_wait();
    const int n = length_of(a.lengths, a.L, b), t0 = seg * a.G, t1 = min(t0 + a.G, (a.L + T - 1) / T), t_end = min(t1, (n + T - 1) / T);
    const Src sq = src_of(ps.q, b, h, dk), sk = src_of(ps.k, b, h, dk), sv = src_of(ps.v, b, h, dv);
    const size_t dd = (size_t)dk * dv;

    // state: row `row`, columns half * HALF ...
    float s[C::HALF];
    const float *x0 = seg > 0 ? ps.local + ((size_t)bh * a.nseg + seg) * dd : ps.x0 ? ps.x0 + (size_t)bh * dd : nullptr;
    const bool turned = seg > 0 ? ps.local_transposed : ps.x_transposed;
#pragma unroll
    for (int c = 0; c < C::HALF; ++c) {
        const int col = half * C::HALF + c;
        s[c] = x0 && row < dk && col < dv ? x0[turned ? (size_t)col * dk + row : (size_t)row * dv + col] : 0.f;
    }
    auto put_state = [&] {
        if (row >= D) return;
#pragma unroll
        for (int c = 0; c < C::HALF; c += 8)
            *reinterpret_cast<uint4 *>(X + (half * C::HALF + c) / 8 * C::CHX + row * 16) =
                make_uint4(pack(s[c], s[c + 1]), pack(s[c + 2], s[c + 3]), pack(s[c + 4], s[c + 5]), pack(s[c + 6], s[c + 7]));
    };
    put_state();
    tokens(ctl.tok[t0 & 1], a, ps.dir, t0, n);
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tm = ctl.tmem, mine = tm + ((uint32_t)(quarter * 32) << 16);
    if (t0 < t_end) {
        load_tile(q, sq, ctl.tok[t0 & 1]);
        load_tile(k, sk, ctl.tok[t0 & 1]);
        copy_commit();
        load_tile(v, sv, ctl.tok[t0 & 1]);
        copy_commit();
    }
    for (int t = t0; t < t_end; ++t) {
        const int p0 = t * T, rows = min(T, n - p0), lead = p0 == 0 ? ps.first : 1;
        const uint32_t parity = (t - t0) & 1;
        const bool has_state = t > t0 || x0, next = t + 1 < t_end, keep = next || ends;
        copy_wait<1>();
        fence_async_smem();
        tc_fence_before_sync();
        __syncthreads();
        if (warp == 4 && elect_one()) {
            tc_fence_after_sync();
            const uint64_t qa = kmajor(q, CH), kb = kmajor(k, CH), xb = mnmajor(x, C::CHX);
#pragma unroll
            for (int kk = 0; kk < C::KS; ++kk) mma_f16(tm + C::S, qa + kk * (2 * CH / 16), kb + kk * (2 * CH / 16), idesc_bf16(128, T, false, false), kk > 0);
            if (has_state) {
#pragma unroll
                for (int kk = 0; kk < C::KS; ++kk) mma_f16(tm + C::I, qa + kk * (2 * CH / 16), xb + kk * 16, idesc_bf16(128, D, false, true), kk > 0);
            }
            mma_commit(&ctl.bar[0]);
        }
        __syncwarp();
        if (keep) decay_keys(K, KH, KL, dk / 8, lam, rows - 1, exact);
        if (next) tokens(ctl.tok[(t + 1) & 1], a, ps.dir, t + 1, n);
        wait(&ctl, 0, parity, status);
        __syncthreads();                                     // q and k are free
        tc_fence_after_sync();
        if (next) {
            load_tile(q, sq, ctl.tok[(t + 1) & 1]);
            load_tile(k, sk, ctl.tok[(t + 1) & 1]);
        }
        copy_commit();
        // decayed scores: keys 64 half .. of the row, in pairs of blocks of 16
        for (int j0 = half * 64; j0 < min(half * 64 + 64, quarter * 32 + 32); j0 += 32) {
            uint32_t r[2][16];
            ld16(mine + C::S + j0, r[0]);
            ld16(mine + C::S + j0 + 16, r[1]);
            ld_wait();
            const bool diagonal = j0 == quarter * 32;
#pragma unroll
            for (int g = 0; g < 2; ++g) {
                uint32_t p[8];
                if (diagonal) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const int gap = row - (j0 + g * 16 + i);
                        r[g][i] = __float_as_uint(gap >= 0 ? f(r[g][i]) * exp2_of(lam * gap) : 0.f);
                    }
                } else {
                    const float w = exp2_of(lam * (row - (j0 + g * 16 + 15)));
#pragma unroll
                    for (int i = 0; i < 16; ++i) r[g][i] = __float_as_uint(f(r[g][i]) * (w * cw[i]));
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) p[i] = pack(f(r[g][2 * i]), f(r[g][2 * i + 1]));
                st8(mine + (half ? C::P1 : C::P0) + (j0 - half * 64) / 2 + g * 8, p);
            }
        }
        // what the entering state gives
        float o[C::HALF];
        if (has_state) {
            uint32_t r[C::HALF];
#pragma unroll
            for (int c = 0; c < C::HALF; c += 8) ld8(mine + C::I + half * C::HALF + c, r + c);
            ld_wait();
            const float w = exp2_of(lam * (row + lead));
#pragma unroll
            for (int c = 0; c < C::HALF; ++c) o[c] = f(r[c]) * w;
        } else {
#pragma unroll
            for (int c = 0; c < C::HALF; ++c) o[c] = 0.f;
        }
        tmem_st_wait();
        copy_wait<1>();                                      // v
        fence_async_smem();                                  // v and the decayed keys
        tc_fence_before_sync();
        __syncthreads();
        if (warp == 4 && elect_one()) {
            tc_fence_after_sync();
            const uint64_t vb = mnmajor(v, CH);
            // keys 16 kk .. are behind the rows of the quarters below kk / 2: those stay as they are, so that no zero meets a NaN there
#pragma unroll
            for (int kk = 0; kk < T / 16; ++kk)
                mma_ts(tm + C::O, tm + (kk < 4 ? C::P0 + kk * 8 : C::P1 + (kk - 4) * 8), vb + kk * 16, idesc_bf16(128, D, false, true), kk > 0, kk / 2);
            if (keep) {
                issue_state<D>(tm + C::I, kh, v, false);
                if (exact) issue_state<D>(tm + C::I, kl, v, true);
            }
            mma_commit(&ctl.bar[1]);
        }
        __syncwarp();
        wait(&ctl, 1, parity, status);
        tc_fence_after_sync();
        if (next) load_tile(v, sv, ctl.tok[(t + 1) & 1]);
        copy_commit();
        {
            uint32_t r[C::HALF];
#pragma unroll
            for (int c = 0; c < C::HALF; c += 8) ld8(mine + C::O + half * C::HALF + c, r + c);
            ld_wait();
            const int p = p0 + row, tok = p < a.L ? token_at(a, ps.dir, p, n) : -1;
            if (tok >= 0) {
                const size_t at = (((size_t)b * a.L + tok) * a.H + h) * dv + half * C::HALF;
#pragma unroll
                for (int c = 0; c < C::HALF; c += 8) {
                    float y[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) y[e] = p < n ? o[c + e] + f(r[c + e]) : 0.f;
                    if (half * C::HALF + c < dv) put8(ps, at + c, y);
                }
            }
        }
        if (keep && quarter * 32 < D) {
            uint32_t r[C::HALF];
#pragma unroll
            for (int c = 0; c < C::HALF; c += 8) ld8(mine + C::I + half * C::HALF + c, r + c);
            ld_wait();
            const float w = exp2_of(lam * (rows - 1 + lead));
#pragma unroll
            for (int c = 0; c < C::HALF; ++c) s[c] = row < dk ? fmaf(w, s[c], f(r[c])) : 0.f;
            put_state();
        }
    }
    copy_wait<0>();
    if (ends && row < dk) {
        const float w = n > 0 && ps.last ? exp2_of(lam) : 1.f;            // no token: the start state
#pragma unroll
        for (int c = 0; c < C::HALF; ++c) {
            const int col = half * C::HALF + c;
            if (col < dv) ps.x_end[(size_t)bh * dd + (size_t)row * dv + col] = s[c] * w;
        }
    }
    // whole tiles behind the end
    for (int p = max(t_end, t0) * T + warp; p < min(t1 * T, a.L); p += NT / 32)
        for (int c = lane * 8; c < dv; c += 256) {
            const float y[8] = {};
            put8(ps, (((size_t)b * a.L + p) * a.H + h) * dv + c, y);
        }
    tc_fence_before_sync();
    __syncthreads();
    pdl_launch_dependents();
    if (warp == 0) tmem_dealloc(tm, C::COLS);
}

// What a segment adds to the state behind it.
template <int D>
__global__ void __launch_bounds__(NT, 2) decay_local(const __grid_constant__ Args a, int *status)
{
    using C = Cfg<D>;
    constexpr int COLS = D <= 64 ? 64 : 128;
    extern __shared__ __align__(128) char sm[];
    __shared__ Ctl ctl;
    const Pass &ps = a.pass[blockIdx.x % a.passes];
    const int seg = blockIdx.x / a.passes, bh = blockIdx.y, b = bh / a.H, h = bh - b * a.H, dk = ps.dk, dv = ps.dv;
    const bool exact = true;
    if (seg == a.nseg - 1 && !ps.x_end) {           // goes into the final state only
        pdl_wait();
        pdl_launch_dependents();
        return;
    }
    const float lam = a.lam.v[h];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, quarter = warp & 3, half = warp >> 2, row = quarter * 32 + lane;
    char *KH = sm, *KL = KH + dk / 8 * CH, *K = KL + (exact ? dk / 8 * CH : 0), *V = K + dk / 8 * CH;
    const uint32_t kh = smem_u32(KH), kl = smem_u32(KL), k = smem_u32(K), v = smem_u32(V);
    if (warp == 0) tmem_alloc(&ctl.tmem, COLS);
    if (tid == 32) {
        mbar_init(&ctl.bar[0], 1);
        ctl.dead = 0;
        fence_barrier_init();
    }
    for (int i = dv / 8 * T + tid; i < C::NCH * T; i += NT) {
        zero16(V + i / T * CH + i % T * 16);
        zero16(V + C::TILE + i / T * CH + i % T * 16);
    }
    pdl_wait();
    const int n = length_of(a.lengths, a.L, b), t0 = seg * a.G, t_end = min(t0 + a.G, (n + T - 1) / T), end = min((t0 + a.G) * T, n);
    const Src sk = src_of(ps.k, b, h, dk), sv = src_of(ps.v, b, h, dv);
    tokens(ctl.tok[t0 & 1], a, ps.dir, t0, n);
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tm = ctl.tmem, mine = tm + ((uint32_t)(quarter * 32) << 16);
    if (t0 < t_end) {
        load_tile(k, sk, ctl.tok[t0 & 1]);
        load_tile(v, sv, ctl.tok[t0 & 1]);
    }
    for (int t = t0; t < t_end; ++t) {
        const int i = t - t0;
        copy_wait_all();
        if (t + 1 < t_end) tokens(ctl.tok[(t + 1) & 1], a, ps.dir, t + 1, n);
        if (i > 0) wait(&ctl, 0, (i - 1) & 1, status);       // decayed keys and the other v are free
        __syncthreads();
        decay_keys(K, KH, KL, dk / 8, lam, end - 1 - t * T, exact);
        fence_async_smem();
        __syncthreads();
        if (warp == 4 && elect_one()) {
            tc_fence_after_sync();
            const uint32_t vt = v + (i & 1) * C::TILE;
            issue_state<D>(tm, kh, vt, i > 0);
            if (exact) issue_state<D>(tm, kl, vt, true);
            mma_commit(&ctl.bar[0]);
        }
        __syncwarp();
        if (t + 1 < t_end) {
            load_tile(k, sk, ctl.tok[(t + 1) & 1]);
            load_tile(v + (~i & 1) * C::TILE, sv, ctl.tok[(t + 1) & 1]);
        }
    }
    if (t0 < t_end) {
        wait(&ctl, 0, (t_end - 1 - t0) & 1, status);
        tc_fence_after_sync();
    }
    float *out = ps.local + ((size_t)bh * a.nseg + seg) * dk * dv + (size_t)row * dv;
    uint32_t r[C::HALF] = {};
    if (t0 < t_end) {
#pragma unroll
        for (int c = 0; c < C::HALF; c += 8) ld8(mine + half * C::HALF + c, r + c);
        ld_wait();
    }
    if (row < dk) {
#pragma unroll
        for (int c = 0; c < C::HALF; c += 4)
            if (half * C::HALF + c < dv) store4(out + half * C::HALF + c, make_float4(f(r[c]), f(r[c + 1]), f(r[c + 2]), f(r[c + 3])));
    }
    tc_fence_before_sync();
    __syncthreads();
    pdl_launch_dependents();
    if (warp == 0) tmem_dealloc(tm, COLS);
}

template <int D>
dig_status launch(const Args &a, bool local, cudaStream_t stream)
{
    using C = Cfg<D>;
    int *status = device_status_ptr();
    if (!status) return DIG_ERR_CUDA;
    size_t smem = 0;
    for (int i = 0; i < a.passes; ++i) {
        const Pass &p = a.pass[i];
        const size_t keys = (size_t)p.dk / 8 * CH * 2;
        // sixteen chunks from the start of the last part of the decayed keys are read
        size_t need = local ? keys + (size_t)p.dk / 8 * CH + 2 * C::TILE : keys + 3 * C::TILE + C::XT;
        const size_t read = keys - (size_t)p.dk / 8 * CH + 16 * CH;
        need = need > read ? need : read;
        smem = smem > need ? smem : need;
    }
    const void *fn = local ? (const void *)decay_local<D> : (const void *)decay_pass<D>;
    const dig_status st = ensure_dynamic_smem(fn, smem);
    if (st != DIG_OK) return st;
    KernelTimer t(local ? KID_DECAY_LOCAL : KID_DECAY, stream);
    const dim3 grid(a.nseg * a.passes, a.B * a.H);
    return cuda_ok(local ? launch_pdl(decay_local<D>, grid, dim3(NT), smem, stream, a, status) : launch_pdl(decay_pass<D>, grid, dim3(NT), smem, stream, a, status));
}

}  // namespace

dig_status tc_pass(const Args &a, bool local, cudaStream_t stream)
{
    int d = 0;
    for (int i = 0; i < a.passes; ++i) d = a.pass[i].dk > d ? a.pass[i].dk : d, d = a.pass[i].dv > d ? a.pass[i].dv : d;
    return d <= 64 ? launch<64>(a, local, stream) : d <= 80 ? launch<80>(a, local, stream) : launch<128>(a, local, stream);
}

}  // namespace decay
}  // namespace dig
