// Linear attention with a decay for each head on the tcgen05 tensor cores (equations in decay.cuh): bf16 storage, heads of up to
// 128 channels.
//
// The decay is a number per head, so q, k and v are operands as they come: a tile of 128 positions is copied to shared memory, S = Q K^T
// and I = Q X go to tensor memory, threads weigh the scores, P = S . g^(i-j), and leave them there as the bf16 A operand of O = P V,
// and the state takes U = (g^(n-1-j) k_j)^T v_j: X' = g^n X + U.  Powers are at most 1 everywhere; only within the diagonal blocks of 32
// keys they are formed one by one, elsewhere as g^(i-j0-15) g^(15-(j-j0)), the second factor the same for all rows.
//
// Roundings to bf16: P and the decayed keys, each 2^-9 of its term on average, as much as the rounding of the results; the state
// is an operand in two bf16 parts.  A state that the caller gets is summed apart, with its decayed keys in three bf16 parts (2^-24).
//
// One CTA per SM works through a list of segments; its warps have parts of their own, so that the loads of one tile, the scores of the
// next, the state of this one and the results of the one before overlap:
//   warps 0 .. 7    scores to decayed scores; of heads beyond 64 channels decayed keys
//   warps 8 .. 15   state; of heads up to 64 channels decayed keys
//   warps 16 .. 19  results, through shared memory to global memory
//   warps 20 .. 22  loads of q, k, v;  warp 23  products
// Five parts on every scheduler share its instruction cache: loops are kept short and rolled, and what is rare stands apart.  Unrolled, two
// thirds of the warps' time went by waiting for instructions (4 x 4096 tokens of 12 heads of 64 channels: 60 us, 30 rolled).
// A tile of 64 channels takes 3700 cycles, 17 bytes a cycle and SM in and out: two thirds of the copy bandwidth; issue slots are 60 % busy, warps
// that poll barriers included.  The loads are issued by single warps, a tile of rows in 2600 cycles; with all rows at one address, which spares their time in
// memory but not their instructions, a tile takes 3430.  The widest heads spill (120 bytes a thread stored, at 80 registers).
#include <type_traits>

#include "decay_plan.cuh"
#include "umma.cuh"

namespace dig {
namespace decay {
namespace {

using namespace umma;
using bf16 = __nv_bfloat16;

constexpr int T = kTileTc, CH = T * 16 + 16;
constexpr int kScore = 8, kState = 8, kOut = 4, kLoad = kScore + kState + kOut, kMma = kLoad + 3, kThreads = (kMma + 1) * 32;

// Layouts in shared memory.  q, k, v: panels of 64 channels, rows of 128 bytes under the 128-byte swizzle (a copy of eight lanes then
// writes one line; chunk by chunk of 16 bytes apart it took four times as long), and where 64 or 128 do not hold the head, 16 channels
// more in two chunks.  Decayed keys, state and results: chunk-major without swizzle, element (row, col) of R rows at
// (col / 8) * (16 R + 16) + 16 row + 2 (col % 8).
// D: channels that tiles provide for keys and values, the smallest of 64, 80 and 128 that holds both.
template <int D>
struct Cfg {
    static constexpr int PANELS = D / 64, REST = D % 64 / 16, TILE = PANELS * T * 128 + (REST ? 2 * CH + 992 : 0);
    static constexpr int NCH = D / 8, CHX = D * 16 + 16, XT = NCH * CHX, KEYS = NCH * CH;
    // What shared and tensor memory hold: tiles of q, k, v, and scores.  Wide heads have their keys decayed in place, which makes room for
    // a second tile of them; with one tile of each, and keys apart, loads and decays took turns (80 sequences of 20 tiles: 112 us).
    static constexpr bool IN_PLACE = D == 128;
    static constexpr int Q_TILES = IN_PLACE ? 1 : 2, K_TILES = 2, V_TILES = Q_TILES, S_BUFS = Q_TILES;
    // Who decays keys: the state's warps, or where they have the most to do the scores'.
    static constexpr bool KEYS_BY_SCORE = D > 64;
    static constexpr int HALF = D / 2;                       // columns of a thread
    // tensor memory: scores (over them the decayed ones), outputs, what the entering state gives, the tile's own state
    static constexpr int S = 0, O = S_BUFS * 128, I = O + D, U = I + D;
    // shared memory: tiles, decayed keys, state (two parts), results
    static constexpr int Q = 0, K = Q_TILES * TILE, V = K + K_TILES * TILE, KD = V + V_TILES * TILE, X = KD + (IN_PLACE ? 0 : 2 * KEYS), R = X + 2 * XT;
    static constexpr int BYTES = R + KEYS + 1024;
    // a product reads sixteen chunks of decayed keys from where they start
    static_assert(TILE % 1024 == 0 && U + D <= 512 && (IN_PLACE || KD + KEYS + 16 * CH <= BYTES - 1024) && BYTES + 768 <= 227 * 1024, "fits");
};
// Column of the decayed scores of keys 16 kk ..: the warps of keys 0 .. 31 and 64 .. 95 write over scores they have read themselves, and
// so do those of the others.
__device__ __forceinline__ constexpr int p_col(int kk) { return (kk >> 2) * 16 + (kk >> 1 & 1) * 32 + (kk & 1) * 8; }

// Barriers: two of each, tile i of the CTA's list uses i & 1 in phase i >> 1.  Nobody may be two phases behind on one: each is completed
// again only after all that wait for it have gone on.
constexpr uint32_t kNone = 0xffffffffu;                          // a row that is not written
struct Bars {
    uint64_t q[2], k[2], v[2];           // loaded
    uint64_t s[2], i[2], u[2], o[2];     // products done: scores; scores and what the state gives; the tile's state; outputs
    uint64_t p[2], kd[2], x[2];          // written: decayed scores, decayed keys, state
    uint64_t uf[2], of[2];               // read: the tile's state; outputs and what the state gives
    uint32_t tmem;
    int dead;                            // a wait gave up: no more waiting
};
__host__ __device__ constexpr uint32_t idesc_bf16(int M, int N, bool a_mn, bool b_mn) { return idesc_f16(M, N, a_mn, b_mn) | (1u << 7) | (1u << 10); }
__device__ __forceinline__ uint64_t kmajor(uint32_t a, uint32_t ch) { return make_desc(a, ch, 128, 0); }
__device__ __forceinline__ uint64_t mnmajor(uint32_t a, uint32_t ch) { return make_desc(a, 128, ch, 0); }
// Panels: groups of 8 rows are 1024 bytes apart; along the channels, the next panel.
__device__ __forceinline__ uint64_t kmajor_panel(uint32_t a) { return make_desc(a, 16, 1024, 2); }
__device__ __forceinline__ uint64_t mnmajor_panel(uint32_t a) { return make_desc(a, T * 128, 1024, 2); }

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
// One arrival once this thread's copies are there.  Who waits for it makes them visible to the tensor core.
__device__ __forceinline__ void copies_arrive(uint64_t *bar) { asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" :: "r"(smem_u32(bar)) : "memory"); }
// Until this thread's copies have arrived; then they are there for the tensor core too.
__device__ __forceinline__ void copies_done()
{
    asm volatile("cp.async.wait_all;" ::: "memory");
    fence_async_smem();
}
__device__ __forceinline__ void arrive(uint64_t *bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" :: "r"(smem_u32(bar)) : "memory"); }
// A warp's writes to shared or tensor memory are done.
__device__ __forceinline__ void warp_arrive(uint64_t *bar)
{
    __syncwarp();
    if ((threadIdx.x & 31) == 0) arrive(bar);
}
__device__ __forceinline__ void zero16(char *p) { *reinterpret_cast<uint4 *>(p) = make_uint4(0, 0, 0, 0); }

__device__ __forceinline__ bool passed(uint64_t *bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(ok) : "r"(smem_u32(bar)), "r"(parity) : "memory");
    return ok;
}
__device__ __noinline__ void wait_on(Bars *ctl, uint64_t *bar, uint32_t parity, int *status)
{
    if (*(volatile int *)&ctl->dead) return;
    if (!mbar_wait(bar, parity, status)) *(volatile int *)&ctl->dead = 1;
}
// Waits for tile i's phase of a pair of barriers.
__device__ __forceinline__ void wait(Bars *ctl, uint64_t *pair, int i, int *status)
{
    if (!passed(pair + (i & 1), i >> 1 & 1)) wait_on(ctl, pair + (i & 1), i >> 1 & 1, status);
    __syncwarp();
}
__device__ __forceinline__ bool ready(uint64_t *pair, int i)
{
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(ok) : "r"(smem_u32(pair + (i & 1))), "r"(i >> 1 & 1) : "memory");
    return __all_sync(0xffffffffu, ok);
}

// One segment of one sequence and pass.
struct Item {
    int pass, seg, b, h, n, t0, t1, t_end;       // n: tokens of the sequence; t_end: behind the last tile that has any
};
__device__ __forceinline__ Item item_at(const Args &a, int i)
{
    Item w;
    w.pass = i % a.passes; i /= a.passes;
    w.seg = i % a.nseg; i /= a.nseg;
    w.b = i / a.H; w.h = i - w.b * a.H;
    w.n = length_of(a.lengths, a.L, w.b);
    w.t0 = w.seg * a.G;
    w.t1 = min(w.t0 + a.G, (a.L + T - 1) / T);
    w.t_end = min(w.t1, (w.n + T - 1) / T);
    return w;
}

// ---- the loading warps --------------------------------------------------------------------------------------------------
// Token at a position before the end; behind it, ~position.
__device__ __forceinline__ int token_or_not(const Args &a, int dir, int p, int n)
{
    int q = dir & 1 ? n - 1 - p : p;
    if (dir & 2) {
        // q / gh with a reciprocal rounded down: the estimate is at most one too small for q < 2^24
        int x = (int)__umulhi((uint32_t)q, a.gh_inv), y = q - x * a.gh;
        if (y >= a.gh) { y -= a.gh; ++x; }
        q = y * a.gw + x;
    }
    return p < n ? q : ~p;
}
// Rows of one operand for a sequence and head, 32 at a time: panels, eight lanes to a row's 128 bytes, and the rest.
template <int D>
__device__ __forceinline__ void load_tile(const Args &a, uint32_t dst, const Rows &r, const Item &w, int dir, int tile, int d)
{
    using C = Cfg<D>;
    const bf16 *base = (const bf16 *)r.p + (size_t)w.b * r.batch + (size_t)(w.h / r.share) * d;
    const int stride = (int)r.token, nch = d / 8, lane = threadIdx.x & 31, c0 = lane & 7, r0 = lane >> 3;
    // rows r0, r0 + 4, ...: their low three bits alternate
    const uint32_t even = r0 * 128 + ((c0 ^ r0) << 4), odd = (r0 + 4) * 128 + ((c0 ^ (r0 + 4)) << 4);
#pragma unroll 1
    for (int i = 0; i < T / 32; ++i) {
        const int mine = token_or_not(a, dir, tile * T + i * 32 + lane, w.n);
#pragma unroll 1
        for (int panel = 0; panel < C::PANELS; ++panel) {
            const int c = panel * 8 + c0;
            const bf16 *p = base + c * 8;
            const uint32_t to = dst + panel * T * 128 + i * 32 * 128;
#pragma unroll
            for (int m = 0; m < 8; ++m) {
                const int t = __shfl_sync(0xffffffffu, mine, m * 4 + r0);
                if (c < nch) copy16(to + (m & 1 ? odd : even) + (m & ~1) * 4 * 128, p + (long long)max(t, 0) * stride, t >= 0 ? 16 : 0);
            }
        }
        if constexpr (C::REST > 0)
            for (int c = C::PANELS * 8; c < nch; ++c)
                copy16(dst + C::PANELS * T * 128 + (c - C::PANELS * 8) * CH + (i * 32 + lane) * 16, base + (long long)max(mine, 0) * stride + c * 8, mine >= 0 ? 16 : 0);
    }
}
// Place of chunk c of row r in a tile.
template <int D>
__device__ __forceinline__ int chunk_at(int r, int c)
{
    using C = Cfg<D>;
    return C::REST > 0 && c >= C::PANELS * 8 ? C::PANELS * T * 128 + (c - C::PANELS * 8) * CH + r * 16 : (c >> 3) * T * 128 + r * 128 + (((c & 7) ^ (r & 7)) << 4);
}

// ---- products -----------------------------------------------------------------------------------------------------------
// Over the channels of q, 16 at a time: go(step, descriptor of q, its offset from the tile's start in panels and steps of 32 bytes).
template <int D, class F>
__device__ __forceinline__ void each_channel_step(uint32_t tile, int ks, F go)
{
    using C = Cfg<D>;
#pragma unroll (D == 128 ? 1 : 8)
    for (int kk = 0; kk < C::PANELS * 4; ++kk) {
        const uint32_t off = (kk >> 2) * T * 128 / 16 + (kk & 3) * 2;
        if (kk < ks) go(kk, kmajor_panel(tile) + off, off);
    }
    if constexpr (C::REST > 0)
        if (ks > C::PANELS * 4) go(C::PANELS * 4, kmajor(tile + C::PANELS * T * 128, CH), 0u);
}
// One step of 16 tokens with v as B: N in one go, or the panel and the rest apart.  mma(d, b, idesc)
template <int D, bool A_MN, class F>
__device__ __forceinline__ void value_step(uint32_t d, uint32_t v, int kk, F mma)
{
    using C = Cfg<D>;
    mma(d, mnmajor_panel(v) + kk * 128, idesc_bf16(128, C::PANELS * 64, A_MN, true));
    if constexpr (C::REST > 0) mma(d + C::PANELS * 64, mnmajor(v + C::PANELS * T * 128, CH) + kk * 16, idesc_bf16(128, 16, A_MN, true));
}
// U (+)= KD^T V: M = 128, rows beyond the keys' channels are whatever follows in shared memory and are not used.
template <int D, bool IN_PLACE = false>
__device__ __forceinline__ void issue_state(uint32_t d, uint32_t kd, uint32_t v, bool accumulate)
{
    const uint64_t a = IN_PLACE ? mnmajor_panel(kd) : mnmajor(kd, CH);
    constexpr int step = IN_PLACE ? 128 : 16;
#pragma unroll (D == 128 ? 1 : 8)
    for (int kk = 0; kk < T / 16; ++kk)
        value_step<D, true>(d, v, kk, [&](uint32_t dd, uint64_t b, uint32_t idesc) { mma_f16(dd, a + kk * step, b, idesc, accumulate || kk > 0); });
}

// Decayed keys in PARTS parts of 8 bits: row j times g^(last - j).  Thread i of 256: one row, every second chunk.
template <int D, int PARTS, bool IN_PLACE = false>
__device__ __forceinline__ void decay_keys(int i, const char *K, char *out, int nch, float lam, int last)
{
    const int j = i & (T - 1);
    const float w1 = exp2_of(lam * max(last - j, 0));
    const float2 w = make_float2(w1, w1);
#pragma unroll 1
    for (int c = i / T; c < nch; c += 2) {
        const uint4 u = *reinterpret_cast<const uint4 *>(K + chunk_at<D>(j, c));
        uint32_t x[4] = {u.x, u.y, u.z, u.w}, y[PARTS][4];
#pragma unroll
        for (int m = 0; m < 4; ++m) {
            float2 p = mul2(bf2(x[m]), w);
#pragma unroll
            for (int part = 0; part < PARTS; ++part) {
                y[part][m] = pack(p.x, p.y);
                if (part + 1 < PARTS) p = sub2(p, bf2(y[part][m]));
            }
        }
#pragma unroll
        for (int part = 0; part < PARTS; ++part)
            *reinterpret_cast<uint4 *>(out + (IN_PLACE ? chunk_at<D>(j, c) : (part * nch + c) * CH + j * 16)) = make_uint4(y[part][0], y[part][1], y[part][2], y[part][3]);
    }
}
// 8 columns of a row of results in fp32.
__device__ __forceinline__ void put8(float *p, const float *o)
{
    store4(p, make_float4(o[0], o[1], o[2], o[3]));
    store4(p + 4, make_float4(o[4], o[5], o[6], o[7]));
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1) decay_pass(const __grid_constant__ Args a, int items, int *status)
{
    using C = Cfg<D>;
    extern __shared__ char raw[];
    __shared__ Bars ctl;
    char *sm = raw + (-smem_u32(raw) & 1023);
    const uint32_t base = smem_u32(sm);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

    if (warp == 0) tmem_alloc(&ctl.tmem, 512);
    if (tid == 32) {
        for (int j = 0; j < 2; ++j) {
            mbar_init(&ctl.q[j], 32); mbar_init(&ctl.k[j], 32); mbar_init(&ctl.v[j], 32);
            mbar_init(&ctl.s[j], 1); mbar_init(&ctl.i[j], 1); mbar_init(&ctl.u[j], 1); mbar_init(&ctl.o[j], 1);
            mbar_init(&ctl.p[j], kScore); mbar_init(&ctl.kd[j], kState); mbar_init(&ctl.x[j], kState);
            mbar_init(&ctl.uf[j], kState); mbar_init(&ctl.of[j], kOut);
        }
        ctl.dead = 0;
        fence_barrier_init();
    }
    // q and k are summed over in steps of 16 channels: zeros where the last step has 8.  Where the passes have keys of different sizes,
    // with every tile.
    bool alike = true;
    for (int j = 1; j < a.passes; ++j) alike &= a.pass[j].dk == a.pass[0].dk;
    const int odd = a.pass[0].dk & 8 ? a.pass[0].dk / 8 : 0;
    if (alike && odd) {
        for (int j = tid; j < (C::Q_TILES + C::K_TILES) * T; j += kThreads) zero16(sm + j / T * C::TILE + chunk_at<D>(j % T, odd));
        fence_async_smem();
    }
    pdl_wait();
    if (a.beside) pdl_launch_dependents();
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tm = ctl.tmem;
    int i = 0;                                   // tiles so far

    if (warp >= kLoad && warp < kMma) {
        const int which = warp - kLoad;          // q, k, v
        for (int item = blockIdx.x; item < items; item += gridDim.x) {
            const Item w = item_at(a, item);
            const Pass &ps = a.pass[w.pass];
            const Rows &r = which == 0 ? ps.q : which == 1 ? ps.k : ps.v;
            const int d = which == 2 ? ps.dv : ps.dk;
            for (int t = w.t0; t < w.t_end; ++t, ++i) {
                const int tiles = which == 0 ? C::Q_TILES : which == 1 ? C::K_TILES : C::V_TILES, old = i - tiles;
                if (old >= 0) {                  // its readers are done
                    // keys are free after the scores and their decays; where the scores' warps decay them, loading that early takes 1% longer
                    if (which == 1 && !C::KEYS_BY_SCORE) wait(&ctl, ctl.s, old, status);
                    else if (which < 2) wait(&ctl, ctl.i, old, status);
                    if (which == 1) wait(&ctl, ctl.kd, old, status);
                    if (which == 2 || (which == 1 && C::IN_PLACE)) wait(&ctl, ctl.u, old, status);
                    if (which == 2) wait(&ctl, ctl.o, old, status);
                }
                const uint32_t tile = (which == 0 ? C::Q : which == 1 ? C::K : C::V) + i % tiles * C::TILE;
                uint64_t *bar = which == 0 ? &ctl.q[i & 1] : which == 1 ? &ctl.k[i & 1] : &ctl.v[i & 1];
                load_tile<D>(a, base + tile, r, w, ps.dir, t, d);
                if (alike) {
                    copies_arrive(bar);
                } else {
                    if (which < 2 && (d & 8)) {
#pragma unroll
                        for (int j = 0; j < T / 32; ++j) zero16(sm + tile + chunk_at<D>(j * 32 + lane, d / 8));
                    }
                    copies_done();
                    arrive(bar);
                }
            }
        }
    } else if (warp == kMma) {
        const uint32_t tm = warp_uniform(ctl.tmem), base = warp_uniform(smem_u32(sm));       // operands in uniform registers
        int ahead = 0;                           // tiles whose scores have been issued
        auto scores = [&](int j, int ks) {       // of tile j
            tc_fence_after_sync();
            fence_async_smem();                  // q and k, as they have been waited for
            const uint32_t q = base + C::Q + j % C::Q_TILES * C::TILE, k = base + C::K + j % C::K_TILES * C::TILE, d = tm + C::S + j % C::S_BUFS * 128;
            if (elect_one()) {
                each_channel_step<D>(q, ks, [&](int kk, uint64_t qa, uint32_t off) {
                    mma_f16(d, qa, C::REST > 0 && kk >= C::PANELS * 4 ? kmajor(k + C::PANELS * T * 128, CH) : kmajor_panel(k) + off, idesc_bf16(128, T, false, false), kk > 0);
                });
                mma_commit(&ctl.s[j & 1]);
            }
            __syncwarp();
            ++ahead;
        };
        for (int item = blockIdx.x; item < items; item += gridDim.x) {
            const Item w = item_at(a, item);
            const Pass &ps = a.pass[w.pass];
            const bool start = w.seg > 0 || ps.x0;
            const int ks = (ps.dk + 15) / 16;
            for (int t = w.t0; t < w.t_end; ++t, ++i) {
                const bool next = t + 1 < w.t_end;
                const uint32_t q = base + C::Q + i % C::Q_TILES * C::TILE, v = base + C::V + i % C::V_TILES * C::TILE;
                if (ahead == i) {
                    if (C::S_BUFS == 1 && i > 0) wait(&ctl, ctl.o, i - 1, status);          // the decayed scores before are used up
                    wait(&ctl, ctl.q, i, status);
                    wait(&ctl, ctl.k, i, status);
                    scores(i, ks);
                }
                auto state = [&] {
                    if (next) {
                        wait(&ctl, ctl.kd, i, status);
                        if (i > 0) wait(&ctl, ctl.uf, i - 1, status);
                    }
                    tc_fence_after_sync();
                    if (elect_one()) {
                        if (next) issue_state<D, C::IN_PLACE>(tm + C::U, C::IN_PLACE ? base + C::K + (i & 1) * C::TILE : base + C::KD + (i & 1) * C::KEYS, v, false);
                        mma_commit(&ctl.u[i & 1]);
                    }
                    __syncwarp();
                };
                auto values = [&] {
                    wait(&ctl, ctl.v, i, status);
                    fence_async_smem();
                };
                if (!C::IN_PLACE) {
                    values();
                    state();
                }
                wait(&ctl, ctl.x, i, status);
                if (i > 0) wait(&ctl, ctl.of, i - 1, status);
                tc_fence_after_sync();
                if (elect_one()) {
                    if (t > w.t0 || start) {
                        const uint64_t xh = mnmajor(base + C::X, C::CHX), xl = mnmajor(base + C::X + C::XT, C::CHX);
                        each_channel_step<D>(q, ks, [&](int kk, uint64_t qa, uint32_t) {
                            mma_f16(tm + C::I, qa, xh + kk * 16, idesc_bf16(128, D, false, true), kk > 0);
                            mma_f16(tm + C::I, qa, xl + kk * 16, idesc_bf16(128, D, false, true), true);
                        });
                    }
                    mma_commit(&ctl.i[i & 1]);
                }
                __syncwarp();
                // The next tile's scores, where they need not be waited for.  The decayed scores that they take the place of were used up before
                // the results that the wait above was for.
                if (C::S_BUFS == 2 && next && ready(ctl.q, i + 1) && ready(ctl.k, i + 1)) scores(i + 1, ks);
                if (C::IN_PLACE) values();       // the product before lets go of q
                wait(&ctl, ctl.p, i, status);
                tc_fence_after_sync();
                if (elect_one()) {
                    // keys 16 kk .. are behind the rows of the quarters below kk / 2: those stay as they are, so that no zero meets a NaN there
#pragma unroll (D == 128 ? 1 : 8)
                    for (int kk = 0; kk < T / 16; ++kk)
                        value_step<D, false>(tm + C::O, v, kk, [&](uint32_t d, uint64_t b, uint32_t idesc) {
                            mma_ts(d, tm + C::S + i % C::S_BUFS * 128 + p_col(kk), b, idesc, kk > 0, kk / 2);
                        });
                    mma_commit(&ctl.o[i & 1]);
                }
                __syncwarp();
                if (C::IN_PLACE) state();        // the keys are decayed after the scores
            }
        }
    } else if (warp < kScore) {
        const int quarter = warp & 3, half = warp >> 2, row = quarter * 32 + lane;
        const uint32_t mine = tm + ((uint32_t)(quarter * 32) << 16);
        auto keys = [&](const Item &w, int t, int j) {       // of the item's tile t, the list's tile j
            wait(&ctl, ctl.k, j, status);
            if (t + 1 < w.t_end) {
                char *K = sm + C::K + (j & 1) * C::TILE;
                if (!C::IN_PLACE && j >= 2) wait(&ctl, ctl.u, j - 2, status);        // what stood there has been used
                decay_keys<D, 1, C::IN_PLACE>(tid, K, C::IN_PLACE ? K : sm + C::KD + (j & 1) * C::KEYS, a.pass[w.pass].dk / 8, a.lam.v[w.h], T - 1);
                fence_async_smem();
            }
            warp_arrive(&ctl.kd[j & 1]);
        };
        for (int item = blockIdx.x; item < items; item += gridDim.x) {
            const Item w = item_at(a, item);
            const float lam = a.lam.v[w.h];
            if (C::KEYS_BY_SCORE && !C::IN_PLACE && w.t0 < w.t_end) keys(w, w.t0, i);
            // Factors of a block's 16 keys, g^(row - j0 - 15) and g^15 .. g^0.  Within the diagonal block the first goes up to g^-31, beyond
            // what fp32 holds where a position leaves less than 1/16: there the powers are formed one by one.
            const bool strong = lam < -4.f;
            float2 cw[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) cw[j] = make_float2(exp2_of(lam * (15 - 2 * j)), exp2_of(lam * (14 - 2 * j)));
            for (int t = w.t0; t < w.t_end; ++t, ++i) {
                const uint32_t sp = mine + C::S + i % C::S_BUFS * 128;
                wait(&ctl, ctl.s, i, status);
                tc_fence_after_sync();
                // 16 keys at a time, of the blocks of 32 half and half + 2, where they are not behind the row
#pragma unroll 1
                for (int m = 0; m < 4; ++m) {
                    const int block = half + (m & 2), g = m & 1, gap = row - (block * 32 + g * 16 + 15);
                    if (block > quarter) break;
                    uint32_t r[16], p[8];
                    ld16(sp + block * 32 + g * 16, r);
                    const float w1 = exp2_of(lam * gap);
                    const float2 ww = make_float2(w1, w1);
                    ld_wait();
                    if (block == quarter && strong) {
#pragma unroll
                        for (int j = 0; j < 16; ++j) r[j] = __float_as_uint(f(r[j]) * exp2_of(lam * max(gap + 15 - j, 0)));
                    } else {
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            const float2 y = mul2(make_float2(f(r[2 * j]), f(r[2 * j + 1])), mul2(ww, cw[j]));
                            r[2 * j] = __float_as_uint(y.x);
                            r[2 * j + 1] = __float_as_uint(y.y);
                        }
                    }
                    if (block == quarter) {
#pragma unroll
                        for (int j = 0; j < 16; ++j) r[j] = gap + 15 >= j ? r[j] : 0u;
                    }
#pragma unroll
                    for (int j = 0; j < 8; ++j) p[j] = pack(f(r[2 * j]), f(r[2 * j + 1]));
                    st8(sp + p_col(2 * block + g), p);
                }
                tmem_st_wait();
                tc_fence_before_sync();
                warp_arrive(&ctl.p[i & 1]);
                if (C::IN_PLACE) keys(w, t, i);  // the scores have them
                if (C::KEYS_BY_SCORE && !C::IN_PLACE && t + 1 < w.t_end) keys(w, t + 1, i + 1);
            }
        }
    } else if (warp < kScore + kState) {
        const int quarter = warp & 3, half = (warp >> 2) & 1, row = quarter * 32 + lane, me = tid - kScore * 32;
        const uint32_t mine = tm + ((uint32_t)(quarter * 32) << 16);
        char *X = sm + C::X;
        float s[C::HALF];                        // state: row `row`, columns half * HALF ...; as an operand in two bf16 parts
        auto put_state = [&](int dk) {
            if (row >= dk) {                     // rows that are summed over all the same: up to a multiple of 16
                if (row < (dk + 15) / 16 * 16) {
#pragma unroll
                    for (int c = 0; c < C::HALF; c += 8) {
                        char *at = X + (half * C::HALF + c) / 8 * C::CHX + row * 16;
                        zero16(at);
                        zero16(at + C::XT);
                    }
                    fence_async_smem();
                }
                return;
            }
#pragma unroll
            for (int c = 0; c < C::HALF; c += 8) {
                uint32_t hi[4], lo[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float2 y = make_float2(s[c + 2 * j], s[c + 2 * j + 1]);
                    hi[j] = pack(y.x, y.y);
                    const float2 z = sub2(y, bf2(hi[j]));
                    lo[j] = pack(z.x, z.y);
                }
                char *at = X + (half * C::HALF + c) / 8 * C::CHX + row * 16;
                *reinterpret_cast<uint4 *>(at) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
                *reinterpret_cast<uint4 *>(at + C::XT) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
            }
            fence_async_smem();
        };
        for (int item = blockIdx.x; item < items; item += gridDim.x) {
            const Item w = item_at(a, item);
            if (w.t0 >= w.t_end) continue;
            const Pass &ps = a.pass[w.pass];
            const float lam = a.lam.v[w.h];
            const int dk = ps.dk, dv = ps.dv, bh = w.b * a.H + w.h;
            const float *x0 = w.seg > 0 ? ps.local + ((size_t)bh * a.nseg + w.seg) * dk * dv : ps.x0 ? ps.x0 + (size_t)bh * dk * dv : nullptr;
            auto keys = [&](int t, int j) {      // of tile t, the list's tile j
                wait(&ctl, ctl.k, j, status);
                if (t + 1 < w.t_end) {
                    decay_keys<D, 1>(me, sm + C::K + (j & 1) * C::TILE, sm + C::KD + (j & 1) * C::KEYS, dk / 8, lam, T - 1);
                    fence_async_smem();
                }
                warp_arrive(&ctl.kd[j & 1]);
            };
            const bool turned = w.seg > 0 ? ps.local_transposed : ps.x_transposed;
            if (x0 && turned) {
#pragma unroll
                for (int c = 0; c < C::HALF; ++c) {
                    const int col = half * C::HALF + c;
                    s[c] = row < dk && col < dv ? x0[col * dk + row] : 0.f;
                }
            } else {
#pragma unroll
                for (int c = 0; c < C::HALF; c += 4) {
                    const int col = half * C::HALF + c;
                    float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
                    if (x0 && row < dk && col < dv) y = *reinterpret_cast<const float4 *>(x0 + row * dv + col);
                    s[c] = y.x; s[c + 1] = y.y; s[c + 2] = y.z; s[c + 3] = y.w;
                }
            }
            if (i > 0) wait(&ctl, ctl.i, i - 1, status);             // the state before has been used
            if (x0) put_state(dk);
            warp_arrive(&ctl.x[i & 1]);
            if (!C::KEYS_BY_SCORE) keys(w.t0, i);
            for (int t = w.t0; t < w.t_end; ++t, ++i) {
                const bool next = t + 1 < w.t_end;
                if (!C::KEYS_BY_SCORE && next) keys(t + 1, i + 1);
                const float wn = exp2_of(lam * (T - 1 + (t == 0 ? ps.first : 1)));
                wait(&ctl, ctl.u, i, status);
                if (next && quarter * 32 < D) {
                    tc_fence_after_sync();
                    auto update = [&](int c, auto count) {
                        constexpr int N = decltype(count)::value;
                        uint32_t r[N];
#pragma unroll
                        for (int e = 0; e < N; e += 8) ld8(mine + C::U + half * C::HALF + c + e, r + e);
                        ld_wait();
#pragma unroll
                        for (int e = 0; e < N; ++e) s[c + e] = fmaf(wn, s[c + e], f(r[e]));
                    };
#pragma unroll
                    for (int c = 0; c + 16 <= C::HALF; c += 16) update(c, std::integral_constant<int, 16>());
                    if constexpr (C::HALF % 16 != 0) update(C::HALF - 8, std::integral_constant<int, 8>());
                    tc_fence_before_sync();
                }
                warp_arrive(&ctl.uf[i & 1]);
                if (next) {
                    wait(&ctl, ctl.i, i, status);
                    put_state(dk);
                    warp_arrive(&ctl.x[(i + 1) & 1]);
                }
            }
        }
    } else {
        const int quarter = warp & 3, row = quarter * 32 + lane;
        const uint32_t mine = tm + ((uint32_t)(quarter * 32) << 16);
        char *R = sm + C::R;
        for (int item = blockIdx.x; item < items; item += gridDim.x) {
            const Item w = item_at(a, item);
            const Pass &ps = a.pass[w.pass];
            const float lam = a.lam.v[w.h];
            const int dv = ps.dv, nch = dv / 8;
            const uint32_t nch_inv = 65536 / nch + 1;        // e / nch for e < 512: off by less than 512 / 65536, less than 1 / nch
            const bool start = w.seg > 0 || ps.x0;
            const size_t tok_out = (size_t)a.H * dv, head_out = (size_t)w.b * a.L * tok_out + (size_t)w.h * dv;
            for (int t = w.t0; t < w.t_end; ++t, ++i) {
                const int p0 = t * T, rows = min(T, w.n - p0);
                const bool has_state = t > w.t0 || start;
                const float wr = exp2_of(lam * (row + (t == 0 ? ps.first : 1)));
                const float2 w2 = make_float2(wr, wr);
                const int mt = token_or_not(a, ps.dir, p0 + row, w.n), token = mt >= 0 ? mt : ~mt;
                const size_t at = head_out + (size_t)token * tok_out;
                const uint32_t here = token < a.L ? (uint32_t)(at / 8) : kNone;
                wait(&ctl, ctl.o, i, status);
                tc_fence_after_sync();
#pragma unroll 1
                for (int c = 0; c < D; c += 16) {
                    uint32_t r[16], y[16];
                    ld16(mine + C::O + c, r);
                    if (has_state) ld16(mine + C::I + c, y);
                    ld_wait();
                    if (c + 16 >= D) {
                        tc_fence_before_sync();
                        warp_arrive(&ctl.of[i & 1]);
                    }
                    if (has_state) {
#pragma unroll
                        for (int e = 0; e < 16; e += 2) {
                            const float2 z = fma2(w2, make_float2(f(y[e]), f(y[e + 1])), make_float2(f(r[e]), f(r[e + 1])));
                            r[e] = __float_as_uint(z.x);
                            r[e + 1] = __float_as_uint(z.y);
                        }
                    }
                    if (rows < T) {
#pragma unroll
                        for (int e = 0; e < 16; ++e) r[e] = row < rows ? r[e] : 0u;
                    }
                    if (ps.out_f32) {
#pragma unroll
                        for (int e = 0; e < 16; e += 8)
                            if (token < a.L && c + e < dv) put8((float *)ps.out + at + c + e, reinterpret_cast<const float *>(r + e));
                        continue;
                    }
#pragma unroll
                    for (int e = 0; e < 16; e += 8)
                        *reinterpret_cast<uint4 *>(R + (c + e) / 8 * CH + row * 16) = make_uint4(pack(f(r[e]), f(r[e + 1])), pack(f(r[e + 2]), f(r[e + 3])), pack(f(r[e + 4]), f(r[e + 5])),
                                                                                                pack(f(r[e + 6]), f(r[e + 7])));
                }
                // The warp's 32 rows from shared to global memory, consecutive lanes the chunks of a row.  (A bulk copy a row took 5700 cycles a
                // tile; by the scores' warps, a tile later, 2% longer.)
                __syncwarp();
                if (!ps.out_f32) {
#pragma unroll 1
                    for (int e0 = lane; e0 < 32 * nch; e0 += 64) {
                        uint32_t to[2];
                        uint4 y[2];
                        int c[2];
#pragma unroll
                        for (int m = 0; m < 2; ++m) {
                            const int e = min(e0 + m * 32, 32 * nch - 1), r = (int)(e * nch_inv >> 16);
                            c[m] = e - r * nch;
                            to[m] = __shfl_sync(0xffffffffu, here, r);
                            if (e0 + m * 32 != e) to[m] = kNone;
                            y[m] = *reinterpret_cast<const uint4 *>(R + c[m] * CH + (quarter * 32 + r) * 16);
                        }
#pragma unroll
                        for (int m = 0; m < 2; ++m)
                            if (to[m] != kNone) *reinterpret_cast<uint4 *>((char *)ps.out + (size_t)(to[m] + c[m]) * 16) = y[m];
                    }
                }
                __syncwarp();
            }
            // whole tiles behind the end
            for (int p = max(w.t_end, w.t0) * T + (warp - kScore - kState); p < min(w.t1 * T, a.L); p += kOut)
                for (int c = lane * 8; c < dv; c += 256) {
                    const float zero[8] = {};
                    const size_t at = head_out + p * tok_out + c;
                    if (ps.out_f32) put8((float *)ps.out + at, zero);
                    else zero16((char *)((bf16 *)ps.out + at));
                }
        }
    }
    tc_fence_before_sync();
    __syncthreads();
    pdl_launch_dependents();
    if (warp == 0) tmem_dealloc(tm, 512);
}

// What a segment adds to the state behind it: for the states that enter segments with the decayed keys in bf16, and where the final state
// is wanted besides with two more parts of them, 24 bits, in accumulators of their own.
// Warps: 0 .. 7 decayed keys, sums to global memory; 8 and 9 loads of k and v; 10 products.
template <int D>
struct LocalCfg {
    // decayed keys first: their products read sixteen chunks from where a part starts, whatever stands there
    static constexpr int THREADS = 11 * 32;
    __host__ __device__ static constexpr int keys(int parts, int nch) { return (parts * nch * CH + 1023) / 1024 * 1024; }
    // two buffers of decayed keys where they have three parts and there is room
    __host__ __device__ static constexpr int bufs(int parts) { return parts > 1 && D <= 80 ? 2 : 1; }
    static constexpr int bytes(int parts, int nch) { return bufs(parts) * keys(parts, nch) + 4 * Cfg<D>::TILE + 1024; }
    // tensor memory: two items' accumulators, of one part or of both
    __host__ __device__ static constexpr int cols(bool exact) { return exact ? (D <= 64 ? 256 : 512) : D <= 64 ? 128 : 256; }
    static_assert(bufs(3) * keys(3, Cfg<D>::NCH) + 4 * Cfg<D>::TILE + 1024 + sizeof(Bars) <= 227 * 1024, "fits");
};
template <int D>
__global__ void __launch_bounds__(LocalCfg<D>::THREADS, 2) decay_local(const __grid_constant__ Args a, int items, int *status)
{
    using C = Cfg<D>;
    using LC = LocalCfg<D>;
    extern __shared__ char raw[];
    __shared__ Bars ctl;
    char *sm = raw + (-smem_u32(raw) & 1023);
    const uint32_t base = smem_u32(sm);
    bool any_final = false;
    int most = 0;
    for (int j = 0; j < a.passes; ++j) {
        any_final |= a.pass[j].final != nullptr;
        most = max(most, a.pass[j].dk);
    }
    const int parts = any_final ? 3 : 1, KB = LC::keys(parts, most / 8), bufs = LC::bufs(parts), K0 = bufs * KB, V0 = K0 + 2 * C::TILE, cols = LC::cols(any_final);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (warp == 0) tmem_alloc(&ctl.tmem, cols);
    if (tid == 32) {
        for (int j = 0; j < 2; ++j) {
            mbar_init(&ctl.k[j], 32); mbar_init(&ctl.v[j], 32);
            mbar_init(&ctl.o[j], 1); mbar_init(&ctl.kd[j], 8); mbar_init(&ctl.of[j], 8);
        }
        ctl.dead = 0;
        fence_barrier_init();
    }
    if (!a.beside) pdl_wait();
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tm = ctl.tmem;
    // Tokens whose power of the decay is 0 in fp32 count too: 0 times a NaN or an infinity is a NaN, as in the passes.  (Without their tiles 5 x 2500
    // tokens of 16 heads of 128 channels, slopes, took 98.3 us instead of 99.9.)
    auto next_item = [&](int item, Item &w, int &end) {
        w = item_at(a, item);
        end = min((w.t0 + a.G) * T, w.n);
        if (w.seg == a.nseg - 1 && !a.pass[w.pass].final) w.t_end = w.t0 = w.t1;           // goes into the final state only
    };
    int i = 0, done = 0;                         // tiles and items with any so far
    if (warp == 8 || warp == 9) {
        const bool value = warp == 9;
        for (int item = blockIdx.x; item < items; item += gridDim.x) {
            Item w;
            int end;
            next_item(item, w, end);
            const Pass &ps = a.pass[w.pass];
            for (int t = w.t0; t < w.t_end; ++t, ++i) {
                if (i >= 2) wait(&ctl, value ? ctl.o : ctl.kd, i - 2, status);
                load_tile<D>(a, base + (value ? V0 : K0) + (i & 1) * C::TILE, value ? ps.v : ps.k, w, ps.dir, t, value ? ps.dv : ps.dk);
                copies_arrive(value ? &ctl.v[i & 1] : &ctl.k[i & 1]);
            }
        }
    } else if (warp == 10) {
        const uint32_t tm = warp_uniform(ctl.tmem), kd = warp_uniform(smem_u32(sm));
        for (int item = blockIdx.x; item < items; item += gridDim.x) {
            Item w;
            int end;
            next_item(item, w, end);
            if (w.t0 >= w.t_end) continue;
            const Pass &ps = a.pass[w.pass];
            const uint32_t acc = tm + (done & 1) * (cols / 2), part = ps.dk / 8 * CH;
            if (done >= 2) wait(&ctl, ctl.of, done - 2, status);
            ++done;
            for (int t = w.t0; t < w.t_end; ++t, ++i) {
                wait(&ctl, ctl.kd, i, status);
                wait(&ctl, ctl.v, i, status);
                fence_async_smem();
                tc_fence_after_sync();
                if (elect_one()) {
                    const uint32_t v = kd + V0 + (i & 1) * C::TILE, keys = kd + (bufs == 2 ? (i & 1) * KB : 0);
                    issue_state<D>(acc, keys, v, t > w.t0);
                    if (ps.final)
#pragma unroll 1
                        for (int j = 1; j < 3; ++j) issue_state<D>(acc + D, keys + j * part, v, t > w.t0 || j > 1);
                    mma_commit(&ctl.o[i & 1]);
                }
                __syncwarp();
            }
        }
    } else {
        const int quarter = warp & 3, half = warp >> 2, row = quarter * 32 + lane;
        for (int item = blockIdx.x; item < items; item += gridDim.x) {
            Item w;
            int end;
            next_item(item, w, end);
            const Pass &ps = a.pass[w.pass];
            if (w.seg == a.nseg - 1 && !ps.final) continue;
            const float lam = a.lam.v[w.h];
            const int dk = ps.dk, dv = ps.dv;
            for (int t = w.t0; t < w.t_end; ++t, ++i) {
                wait(&ctl, ctl.k, i, status);
                if (i >= bufs) wait(&ctl, ctl.o, i - bufs, status);  // decayed keys are free
                const char *K = sm + K0 + (i & 1) * C::TILE;
                char *to = sm + (bufs == 2 ? (i & 1) * KB : 0);
                if (ps.final) decay_keys<D, 3>(tid, K, to, dk / 8, lam, end - 1 - t * T);
                else decay_keys<D, 1>(tid, K, to, dk / 8, lam, end - 1 - t * T);
                fence_async_smem();
                warp_arrive(&ctl.kd[i & 1]);
            }
            const bool some = w.t0 < w.t_end;
            const uint32_t acc = tm + ((uint32_t)(quarter * 32) << 16) + (done & 1) * (cols / 2) + half * C::HALF;
            if (some) {
                wait(&ctl, ctl.o, i - 1, status);
                tc_fence_after_sync();
            }
            const size_t at = ((size_t)(w.b * a.H + w.h) * a.nseg + w.seg) * dk * dv + (size_t)row * dv + half * C::HALF;
            // an uncut sequence: the final state itself
            const float *x0 = a.nseg == 1 ? ps.x0 : nullptr;
            float *final = a.nseg == 1 ? ps.x_end : ps.final;
            const float w0 = w.n > 0 ? exp2_of(lam * (w.n - 1 + ps.first + ps.last)) : 1.f, w1 = a.nseg == 1 && ps.last ? exp2_of(lam) : 1.f;
#pragma unroll 1
            for (int c = 0; c < C::HALF; c += 8) {
                uint32_t r[8] = {}, y[8] = {};
                if (some) {
                    ld8(acc + c, r);
                    if (ps.final) ld8(acc + D + c, y);
                    ld_wait();
                }
                if (row < dk && half * C::HALF + c < dv) {
                    if (a.nseg > 1) put8(ps.local + at + c, reinterpret_cast<const float *>(r));
                    if (ps.final) {
                        float z[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            z[e] = (f(r[e]) + f(y[e])) * w1;
                            if (x0) z[e] = fmaf(w0, __ldcg(x0 + at + c + e), z[e]);           // passes with a final state have theirs not transposed
                        }
                        put8(final + at + c, z);
                    }
                }
            }
            if (some) {
                tc_fence_before_sync();
                warp_arrive(&ctl.of[done & 1]);
                ++done;
            }
        }
    }
    tc_fence_before_sync();
    __syncthreads();
    pdl_launch_dependents();
    if (warp == 0) tmem_dealloc(tm, cols);
    if (a.beside && blockIdx.x == 0) pdl_wait();             // complete only after the passes; the other CTAs make room
}

template <int D>
dig_status launch(const Args &a, bool local, cudaStream_t stream)
{
    int *status = device_status_ptr();
    if (!status) return DIG_ERR_CUDA;
    const long long items = (long long)a.nseg * a.passes * a.B * a.H;
    KernelTimer t(local ? KID_DECAY_LOCAL : KID_DECAY, stream);
    if (!local) {
        const dig_status st = ensure_dynamic_smem((const void *)decay_pass<D>, Cfg<D>::BYTES);
        if (st != DIG_OK) return st;
        return cuda_ok(launch_pdl(decay_pass<D>, dim3((unsigned)(items < kSms ? items : kSms)), dim3(kThreads), Cfg<D>::BYTES, stream, a, (int)items, status));
    }
    int parts = 1, most = 0;
    for (int i = 0; i < a.passes; ++i) {
        if (a.pass[i].final) parts = 3;
        most = a.pass[i].dk > most ? a.pass[i].dk : most;
    }
    const size_t smem = LocalCfg<D>::bytes(parts, most / 8);
    const dig_status st = ensure_dynamic_smem((const void *)decay_local<D>, smem);
    if (st != DIG_OK) return st;
    const long long room = (2 * (smem + 1024 + sizeof(Bars)) <= 228 * 1024 && 2 * LocalCfg<D>::cols(parts > 1) <= 512 ? 2ll : 1ll) * kSms;
    return cuda_ok(launch_pdl(decay_local<D>, dim3((unsigned)(items < room ? items : room)), dim3(LocalCfg<D>::THREADS), smem, stream, a, (int)items, status));
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
