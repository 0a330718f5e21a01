// Latent attention over packed prompts in the expanded form on the tensor cores (bf16,
// P up to 64): keys of a head's own part and of a rotary part that all heads share.
//
// One CTA holds two tiles of 128 tokens of one head, which read the same keys. Per tile
// of 128 keys and for each query tile t:
//   S_t = Q_t K^T      three chunks of 64 elements, the shared part as the last one, in
//                      shared memory; S in TMEM
//   P_t = exp2(scale S_t - m)   one thread per row: S from TMEM to registers,
//                      running maximum and sum, P as bf16 over S in TMEM
//   O_t += P_t V       P from TMEM, V in shared memory (its rows are keys, so V is the
//                      MN-major operand)
// While one tile's softmax runs, the tensor cores work for the other. The row
// maximum m is raised, and O in TMEM rescaled, only when a row's maximum has
// grown by more than 2^8 since the last time: P then stays below 2^8 and the
// final division by the same row's sum makes up for it.
// K and V come through one ring of 16 KB chunks: 64 elements of 128 keys, or 128 of 64 keys
// (a chunk of V is whole in its place, so the ring may end inside a tile). Two query
// tiles of 192 elements leave room for eight: V of one tile, K of the next and three more.
// kDeal, where there is too little work for every SM: the two tiles are one tile
// of 128 rows twice, with every other tile of keys each, and their results are
// joined at the end.
// Warps 0-3 and 4-7: softmax of tile 0 and 1 and their results; warp 8: TMA; warps 9
// and 11: MMA of tile 0 and 1; warp 10: scheduler. A CTA goes on with the work of CTAs that have not
// started (cluster launch control), so the loads, the first products and the search
// for the next work run while the softmax warps still write the last results.
// TMEM columns: S_0, S_1 (128 each), O_0, O_1 (128 each).
//
// What bounds it: of 128 keys of two tiles the products take 2560 cycles, their operands in shared memory and the
// copies into it 2660 (340 KB), the copies from L2 2880 (27.8 bytes a cycle and SM at most): all three are near each
// other. 16384 tokens of 32 heads, causal: 1.80 ms, 1.53 PFLOP/s; 7 prompts of 8192 in all 130 us (ends, masks,
// results and the first products of eight items a CTA). One MMA warp for both tiles, which stood still in its waits and
// commits, took 2.02 ms.
//
// P is rounded to bf16, an error of up to 2^-8 of each weight beside the result's
// own rounding: the MMA takes both operands in one 16-bit type, and V is bf16.
//
// A masked score gives P = 0, but 0 times a NaN value is a NaN: a row whose sums are finite
// and whose result is not is looked after as in attn_prompt.cu (repair_rows).
//
// Waits are bounded as in the GEMM kernels (tc_ptx.cuh).
#include "attn_prompt.cuh"
#include "latent.h"

namespace gbmoe {
namespace {

using namespace tc;

constexpr int kTile = kPromptTile;
constexpr int kThreads = 384;
constexpr int kHalf = kTile * 128;     // bytes of a chunk: 128 rows of 64 elements
constexpr int kQTile = 3 * kHalf;
constexpr int kSlots = 8;              // chunks of K and V in flight
constexpr int kAhead = 4;              // tiles of K and V of an item still to be loaded when the CTA asks for its next item
constexpr float kGrow = 8.0f;          // log2 of how far a row's maximum may run ahead of m
constexpr int kSmem = 1024 + 2 * kQTile + kSlots * kHalf + 512;
static_assert((2 * kSlots + 26) * 8 <= 512 && kSmem + 1024 <= 227 * 1024, "shared memory");

// bytes that are to come, without an arrival
__device__ __forceinline__ void mbar_expect_only(uint64_t* bar, uint32_t bytes) {
    asm volatile("mbarrier.expect_tx.relaxed.cta.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(bar)), "r"(bytes) : "memory");
}

// 32 bytes to a 32-byte aligned address
__device__ __forceinline__ void store32(__nv_bfloat16* dst, const uint32_t (&a)[4], const uint32_t (&b)[4]) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(dst), "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]),
                 "r"(b[0]), "r"(b[1]), "r"(b[2]), "r"(b[3])
                 : "memory");
}

struct Params {
    LatentProblem l;
    uint64_t wait_limit_ns;
};

// Descriptor of a chunk of V: 64 keys' rows of 64 values (128-byte swizzled; the MMA's N runs along a row), the next
// 64 columns behind them (leading offset), groups of 8 keys 1024 bytes apart (stride offset).
__device__ __forceinline__ uint64_t half_desc(uint32_t saddr) {
    return (uint64_t)((saddr & 0x3FFFFu) >> 4) | (uint64_t)(kHalf / 2 >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 |
           (uint64_t)1 << 46 | (uint64_t)2 << 61;
}

// A query's product with its key, which has two parts (repair_rows).
struct TwoPartKeys {
    __device__ __forceinline__ static float dot(const LatentProblem& l, int64_t t, int h, int64_t key) {
        const AttnProblem& p = l.a;
        const __nv_bfloat16* q = static_cast<const __nv_bfloat16*>(p.q.p) + t * p.q.ts + h * p.q.hs;
        const __nv_bfloat16* k = static_cast<const __nv_bfloat16*>(p.k.p) + h * p.k.hs + key * p.k.ts;
        const __nv_bfloat16* r = static_cast<const __nv_bfloat16*>(l.k_rope.p) + key * l.k_rope.ts;
        float s = 0.0f;
        for (int c = 0; c < l.K; c += 8) {
            float a[8], b[8];
            Vec8<__nv_bfloat16>::load(q + c, a);
            Vec8<__nv_bfloat16>::load(c < l.own ? k + c : r + (c - l.own), b);
#pragma unroll
            for (int i = 0; i < 8; ++i) s = fmaf(a[i], b[i], s);
        }
        return s;
    }
};

// One work item as the scheduler warp hands it out.
struct Work {
    Seq s;
    int tok0[2], rows[2];   // query tile t: first token of the sequence, rows (<= 0: none)
    int n[2];               // its key tiles, from k_first on
    int k_first, head0;
    int end;                // 1: no more work
};

template <bool kDeal>
__global__ void __launch_bounds__(kThreads, 1)
latent_prompt_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                     const __grid_constant__ CUtensorMap tm_r, const __grid_constant__ CUtensorMap tm_v,
                     const __grid_constant__ Params pp) {
    pdl_enter();
    const AttnProblem& p = pp.l.a;
    const int own = pp.l.own, rope = pp.l.K - own;        // elements of a key's two parts
    const int own_chunks = (own + 63) / 64, k_chunks = own_chunks + (rope > 0);
    __shared__ Work work_slots[2];
    __shared__ __align__(16) uint4 answer;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    uint8_t* sQ = smem;  // two query tiles
    uint8_t* sKV = smem + 2 * kQTile;
    // kDeal, which has one query tile: maximum, sum and results' check of the softmax warps' rows
    float(*stats)[8][32] = reinterpret_cast<float(*)[8][32]>(sQ + kQTile);
    uint64_t* bars = reinterpret_cast<uint64_t*>(sKV + kSlots * kHalf);
    // tiles of K and V in the order in which they are loaded, tile i on the barriers i % kSlots (a tile has a slot at least)
    uint64_t* full = bars;            // it landed
    uint64_t* done = full + kSlots;   // the MMAs of both query tiles that read it finished
    uint64_t* q_full = done + kSlots;
    uint64_t* q_empty = q_full + 2;   // the last product with a query tile finished
    uint64_t* s_full = q_empty + 2;   // S of a query tile is complete (and so is every MMA before it)
    uint64_t* p_full = s_full + 2;    // its P is written and O rescaled
    uint64_t* o_full = p_full + 2;    // its O is complete
    uint64_t* w_full = o_full + 2;    // a work item is in its slot
    uint64_t* w_empty = w_full + 2;   // every role has read it
    uint64_t* ans = w_empty + 2;      // the answer to try_cancel
    uint64_t* ask = ans + 1;          // the loads of a work item are nearly all on their way
    uint64_t* drain = ask + 1;
    uint64_t* pair = drain + 2;       // kDeal: the two warps of the same rows
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(pair + 4);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int i = 0; i < kSlots; ++i) {
            mbar_init(&full[i], 1);
            mbar_init(&done[i], 2);
        }
        for (int t = 0; t < 2; ++t) {
            mbar_init(&q_full[t], 1);
            mbar_init(&q_empty[t], kDeal ? 2 : 1);
            mbar_init(&s_full[t], 1);
            mbar_init(&p_full[t], 4);
            mbar_init(&o_full[t], 1);
            mbar_init(&w_full[t], 1);
            mbar_init(&w_empty[t], 11);  // softmax warps, TMA, MMA warps
        }
        mbar_init(ans, 1);
        mbar_init(ask, 1);
        mbar_init(&drain[0], 1);
        mbar_init(&drain[1], 1);
        for (int i = 0; i < 4; ++i) mbar_init(&pair[i], 2);
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 9) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(tmem_slot)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    auto wait = [&](uint64_t* bar, uint32_t parity) { return mbar_wait(bar, parity, abort_flag, p.err, pp.wait_limit_ns); };
    auto wait_warp = [&](uint64_t* bar, uint32_t parity) { return warp_wait(bar, parity, abort_flag, p.err, pp.wait_limit_ns); };

    // Registers: 384 threads start with 168 each; the softmax rows take 216, the others keep 72.
    if (warp < 8) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
        // ------------------------------------------------- softmax, one row each
        const int t = warp >> 2, r = (warp & 3) * 32 + lane;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t tS = tmem + lanes + t * kTile, tO = tmem + lanes + 2 * kTile + t * kTile;
        const uint32_t tO2 = tmem + lanes + 2 * kTile + (t ^ 1) * kTile;
        const float scale = p.scale_log2;
        uint32_t sn = 0, items = 0, items2 = 0;  // key tiles and items of this query tile so far; items of the other
        uint32_t meets = 0;
        auto meet = [&] {  // with the other warp of the same rows
            __syncwarp();
            if (lane == 0) mbar_arrive(&pair[warp & 3]);
            return wait_warp(&pair[warp & 3], meets++ & 1u);
        };
        // whole sectors of 32 bytes for a thread's stores, where the results lie so
        const bool wide = ((reinterpret_cast<uintptr_t>(p.out.p) | (uintptr_t)(2 * p.out.ts) | (uintptr_t)(2 * p.out.hs) | (uintptr_t)(2 * p.D)) & 31) == 0;
        bool ok = true;
        for (int k = 0; ok; ++k) {
            if (!wait_warp(&w_full[k & 1], (uint32_t)(k >> 1) & 1u)) break;
            const Work& slot = work_slots[k & 1];
            const Seq s = slot.s;
            const int n = slot.n[t], n2 = slot.n[t ^ 1], rows = slot.rows[t], row = slot.tok0[t] + r, k_first = slot.k_first, end = slot.end;
            const int head = slot.head0;
            const bool have = r < rows;
            __syncwarp();
            if (lane == 0) mbar_arrive(&w_empty[k & 1]);
            if (end) break;
            int lo = 0, hi = INT_MAX;  // (rows past the tile's end and empty ones are never stored: no mask for them)
            if (have) seen_keys(p, s, row, lo, hi);
            float m = neg_inf(), l = 0.0f;
            for (int j = 0; j < n; ++j) {
                ok = wait_warp(&s_full[t], sn++ & 1u);
                if (!ok) break;
                tc_fence_after();
                uint32_t u[4][32];
#pragma unroll
                for (int c = 0; c < 4; ++c) tmem_ld32_async(tS + 32 * c, u[c]);
                ld_wait();
#pragma unroll
                for (int c = 0; c < 4; ++c) pin32(u[c]);
                const int key0 = k_first + (kDeal ? 2 * j + t : j) * kTile;
                const int first = lo - key0, last = hi - key0;  // columns first .. last are seen
                if (__any_sync(0xffffffffu, first > 0 || last < kTile - 1)) {
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        // the columns of this chunk that the row sees, as bits
                        const int f = first - 32 * c, e = last - 32 * c;
                        const uint32_t seen = (f <= 0 ? ~0u : f > 31 ? 0u : ~0u << f) & (e >= 31 ? ~0u : e < 0 ? 0u : (2u << e) - 1u);
                        if (!__any_sync(0xffffffffu, seen != ~0u)) continue;
#pragma unroll
                        for (int i = 0; i < 32; ++i) u[c][i] = seen & (1u << i) ? u[c][i] : 0xff800000u;
                    }
                }
                float mx[4];
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    mx[c] = fmaxf(__uint_as_float(u[c][0]), __uint_as_float(u[c][1]));
#pragma unroll
                    for (int i = 2; i < 32; i += 2) mx[c] = max3(mx[c], __uint_as_float(u[c][i]), __uint_as_float(u[c][i + 1]));
                }
                const float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * scale;
                if (__any_sync(0xffffffffu, top > m + kGrow || (j == 0 && top > m))) {
                    const float m_new = fmaxf(m, top);
                    const float f = m_new == neg_inf() ? 1.0f : ex2(m - m_new);  // (m = -inf: 0)
                    l *= f;
                    m = m_new;
                    if (j > 0) {  // (this tile's S is complete, so its last O += P V is too)
#pragma unroll 1
                        for (int c = 0; c < p.D; c += 32) {
                            uint32_t o[32];
                            tmem_ld32_async(tO + c, o);
                            ld_wait();
                            pin32(o);
#pragma unroll
                            for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
                            tmem_st32(tO + c, o);
                        }
                    }
                }
                const float base = m == neg_inf() ? 0.0f : -m;
                const uint64_t sc2 = pack2(scale, scale), nb2 = pack2(base, base);
                uint64_t sum[2] = {pack2(0.0f, 0.0f), pack2(0.0f, 0.0f)};
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    uint32_t w[32];
#pragma unroll
                    for (int i = 0; i < 32; ++i) {
                        const int e = 64 * half + 2 * i;
                        const float2 x = unpack2(fma2(pack2(__uint_as_float(u[e >> 5][e & 31]), __uint_as_float(u[e >> 5][(e & 31) + 1])), sc2, nb2));
                        const float a = ex2(x.x), b = ex2(x.y);
                        sum[i & 1] = add2(sum[i & 1], pack2(a, b));
                        w[i] = pack_bf16x2(a, b);
                    }
                    tmem_st32(tS + 32 * half, w);
                }
                const float2 s01 = unpack2(add2(sum[0], sum[1]));
                l += s01.x + s01.y;
                st_wait();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&p_full[t]);
            }
            // -------------------------------------------------------- result
            if (ok && n > 0) ok = wait_warp(&o_full[t], items++ & 1u);
            if (kDeal && ok && n2 > 0) ok = wait_warp(&o_full[t ^ 1], items2++ & 1u);
            if (!ok) break;
            tc_fence_after();
            if (rows <= (warp & 3) * 32) {  // no row of this warp
                // kDeal: the two warps of these rows meet all the same. Each has waited for both halves' sums then, so neither
                // barrier can complete a phase of the next item before the other warp has seen this item's.
                if (kDeal) ok = meet();
                continue;
            }
            const bool empty = hi < lo;
            float inv = empty ? 0.0f : 1.0f / l, inv2 = 0.0f;  // (kDeal: factors of this tile's and the other's sums)
            if constexpr (kDeal) {
                stats[0][warp][lane] = m, stats[1][warp][lane] = l;
                ok = meet();
                if (!ok) break;
                const float m2 = stats[0][warp ^ 4][lane], l2 = stats[1][warp ^ 4][lane];
                const float top = fmaxf(m, m2), base = top == neg_inf() ? 0.0f : top;
                const float f = ex2(m - base), f2 = ex2(m2 - base);
                l = t == 0 ? fmaf(l, f, l2 * f2) : fmaf(l2, f2, l * f);  // the same in both warps
                inv = empty ? 0.0f : f / l, inv2 = empty ? 0.0f : f2 / l;
                m = top;
            }
            const int64_t tok = s.q0 + row;
            __nv_bfloat16* out = const_cast<__nv_bfloat16*>(static_cast<const __nv_bfloat16*>(p.out.p)) + tok * p.out.ts + head * p.out.hs;
            float check = 0.0f;  // NaN once a value is not finite
#pragma unroll 1
            for (int c = kDeal ? 32 * t : 0; c < p.D; c += kDeal ? 64 : 32) {
                uint32_t o[32];
                if constexpr (kDeal) {
                    uint32_t o2[32];
                    tmem_ld32_async(tO + c, o);
                    tmem_ld32_async(tO2 + c, o2);
                    ld_wait();
                    pin32(o), pin32(o2);
                    // (a tile without keys for this row has a factor of 0; what it holds may be anything. Loads
                    // that depend on n made the compiler spill 540 bytes)
#pragma unroll
                    for (int i = 0; i < 32; ++i) {
                        const float a = inv != 0.0f ? __uint_as_float(o[i]) * inv : 0.0f;
                        o[i] = __float_as_uint(inv2 != 0.0f ? fmaf(__uint_as_float(o2[i]), inv2, a) : a);
                    }
                } else if (n > 0) {
                    tmem_ld32_async(tO + c, o);
                    ld_wait();
                    pin32(o);
                }
                uint32_t before[4];
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    uint32_t w[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float a = empty ? 0.0f : __uint_as_float(o[8 * q + 2 * i]) * (kDeal ? 1.0f : inv);
                        const float b = empty ? 0.0f : __uint_as_float(o[8 * q + 2 * i + 1]) * (kDeal ? 1.0f : inv);
                        if (c + 8 * q < p.D) check = fmaf(a, 0.0f, fmaf(b, 0.0f, check));
                        w[i] = pack_bf16x2(a, b);
                    }
                    if (q & 1) {
                        if (wide) {
                            if (have && c + 8 * q < p.D) store32(out + c + 8 * (q - 1), before, w);
                            continue;
                        }
                        if (have && c + 8 * (q - 1) < p.D) *reinterpret_cast<uint4*>(out + c + 8 * (q - 1)) = make_uint4(before[0], before[1], before[2], before[3]);
                        if (have && c + 8 * q < p.D) *reinterpret_cast<uint4*>(out + c + 8 * q) = make_uint4(w[0], w[1], w[2], w[3]);
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) before[i] = w[i];
                }
            }
            if constexpr (kDeal) {
                stats[2][warp][lane] = check;
                tc_fence_before();
                ok = meet();  // the other warp has read this tile's sums
                if (!ok) break;
                check += stats[2][warp ^ 4][lane];
            }
            if (have && p.lse && (!kDeal || t == 0)) p.lse[tok * p.Hq + head] = empty ? neg_inf() : (m + log2f(l)) * kLn2;
            // rows that may hold a masked key's NaN
            uint32_t again = __ballot_sync(0xffffffffu, have && !empty && check != check && finite(m) && finite(l) && l > 0.0f);
            if (kDeal && again) {  // (the same in both warps; one repairs, when both have stored)
                __threadfence();
                ok = meet();
                if (t != 0 || !ok) again = 0;
            }
            if (again) repair_rows<TwoPartKeys>(p, pp.l, again, s.k0, k_first, kDeal ? n + n2 : n, tok, head, lo, hi, m, l);
        }
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
        if (warp == 10) {
            // --------------------------------------------------------- scheduler
            constexpr int toks = kDeal ? kTile : 2 * kTile;
            uint32_t block = blockIdx.x;
            TileFinder tiles;
            bool more = true, asked = false;
            uint32_t turn = 0;
            int k = 0;
            for (; more; ++turn) {
                const Place at = tiles.find(p, block / p.Hq, toks);
                if (at.b >= 0) {
                    if (!wait_warp(&w_empty[k & 1], ((uint32_t)(k >> 1) & 1u) ^ 1u)) break;
                    Work w;
                    w.s = load_seq(p, at.b);
                    // The last tiles, which see the most keys, first. Of an odd number the sequence's first is alone, as the
                    // second of its CTA: a tile alone takes nearly as long as two (3000 and 3500 cycles for 128 keys).
                    const int n_tiles = (w.s.nq + kTile - 1) / kTile, last = (w.s.nq + toks - 1) / toks - 1 - (int)at.at;
                    const int first = kDeal ? last : 2 * last - (n_tiles & 1);
                    w.head0 = (int)(block % p.Hq);
                    w.end = 0;
                    int lo, hi;
                    seen_keys(p, w.s, max(first, 0) * kTile, lo, hi);
                    w.k_first = hi < 0 ? 0 : lo & ~(kTile - 1);
#pragma unroll
                    for (int t = 0; t < 2; ++t) {
                        w.tok0[t] = (kDeal ? first : first + t) * kTile;
                        w.rows[t] = w.tok0[t] < 0 ? 0 : min(kTile, w.s.nq - w.tok0[t]);
                        w.n[t] = 0;
                        if (w.rows[t] > 0) {
                            seen_keys(p, w.s, w.tok0[t] + w.rows[t] - 1, lo, hi);  // its last token sees the furthest
                            if (hi >= w.k_first) w.n[t] = (hi - w.k_first) / kTile + 1;
                        }
                    }
                    if (kDeal) w.n[0] = (w.n[0] + 1) / 2, w.n[1] /= 2;
                    if (lane == 0) {
                        work_slots[k & 1] = w;
                        mbar_arrive(&w_full[k & 1]);
                    }
                    __syncwarp();
                    ++k;
                    // (not before: a CTA that has work for long is not to hold more of it. Packed prompts of 8192 tokens, 32 heads:
                    // 131 us; asked for when the item begins 143, an item earlier 152, with CTAs done after 82 to 156)
                    if (!wait_warp(ask, (uint32_t)(k - 1) & 1u)) break;
                }
                if (lane == 0) try_cancel(&answer, ans);
                asked = true;
                if (!wait_warp(ans, turn & 1u)) break;
                asked = false;
                more = cancelled(&answer, block);
                __syncwarp();
                // the answer is read before the next one is asked for (another proxy writes it)
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            }
            if (!more && wait_warp(&w_empty[k & 1], ((uint32_t)(k >> 1) & 1u) ^ 1u) && lane == 0) {
                work_slots[k & 1].end = 1;
                mbar_arrive(&w_full[k & 1]);
            }
            if (asked && lane == 0) drain_wait(ans, turn & 1u);  // (a wait gave up: the answer lands before the CTA leaves)
        } else if (warp == 8 && lane == 0) {
            // ------------------------------------------------------ TMA producer
            uint32_t qn[2] = {0, 0};
            int slot = 0, used = 0;       // next slot, slots that are not free
            uint32_t seq = 0, oldest = 0;  // tiles begun, and of those the first whose slots are not free
            uint64_t sizes = 0;           // slots of the latest tiles, four bits each
            bool open = false;            // the last tile's chunks are not all asked for
            bool ok = true;
            const int v_boxes = (p.D + 63) / 64;
            for (int k = 0; ok; ++k) {
                if (!wait(&w_full[k & 1], (uint32_t)(k >> 1) & 1u)) break;
                const Work w = work_slots[k & 1];
                mbar_arrive(&w_empty[k & 1]);
                if (w.end) break;
                const int n_max = max(w.n[0], w.n[1]);
                // K_0, V_0, K_1, V_1, ..; kDeal: K_0, K_1, V_0, K_2, V_1, .., K_n-1, V_n-2, V_n-1
                const int n_all = kDeal ? w.n[0] + w.n[1] : n_max;
                if (n_all == 0) mbar_arrive(ask);
                auto tile = [&](int i) {
                    if (i == max(0, 2 * n_all - kAhead)) mbar_arrive(ask);
                    bool value = i & 1;
                    int at = i >> 1;
                    if constexpr (kDeal) {
                        value = i == 2 * n_all - 1 || (i > 0 && !(i & 1));
                        at = i == 0 ? 0 : i == 2 * n_all - 1 ? n_all - 1 : value ? at - 1 : at + 1;
                    }
                    const int key = (int)(w.s.k0 + w.k_first + at * kTile);
                    const int chunks = value ? 2 : k_chunks, bits = 4 * (int)(seq % kSlots);
                    uint64_t* bar = &full[seq % kSlots];
                    sizes = (sizes & ~((uint64_t)15 << bits)) | (uint64_t)chunks << bits;
                    for (int c = 0; c < chunks; ++c) {
                        while (ok && used == kSlots) {
                            ok = wait(&done[oldest % kSlots], (oldest / kSlots) & 1u);
                            used -= (int)(sizes >> 4 * (oldest % kSlots) & 15);
                            ++oldest;
                        }
                        if (!ok) break;
                        if (c == 0) ++seq;
                        mbar_expect_only(bar, value ? v_boxes * kHalf / 2 : kHalf);
                        uint8_t* dst = sKV + slot * kHalf;
                        if (value)
                            for (int x = 0; x < v_boxes; ++x) tma_load_3d(dst + x * kHalf / 2, &tm_v, 64 * x, w.head0, key + 64 * c, bar);
                        else if (c < own_chunks)
                            tma_load_3d(dst, &tm_k, 64 * c, w.head0, key, bar);
                        else
                            tma_load_3d(dst, &tm_r, 0, 0, key, bar);
                        ++used;
                        if (++slot == kSlots) slot = 0;
                        open = c + 1 < chunks;
                        if (!open) mbar_arrive(bar);
                    }
                };
                // (the first keys between the tiles' queries: the last product with the second tile's of the item before comes
                // later than the ring has room for them)
                for (int t = 0; t < (kDeal ? 1 : 2) && ok; ++t) {
                    if (t == 1 && n_all > 0) tile(0);
                    if (w.n[t] == 0) continue;
                    ok = ok && wait(&q_empty[t], (qn[t] & 1u) ^ 1u);
                    if (!ok) break;
                    mbar_expect_tx(&q_full[t], k_chunks * kHalf);
                    for (int c = 0; c < k_chunks; ++c)
                        tma_load_3d(sQ + t * kQTile + c * kHalf, &tm_q, c < own_chunks ? 64 * c : own, w.head0, w.s.q0 + w.tok0[t], &q_full[t]);
                    ++qn[t];
                }
                for (int i = kDeal ? 0 : 1; i < 2 * n_all && ok; ++i) tile(i);
            }
            // every copy has landed before the CTA leaves (a wait that gave up inside a tile: those that were asked for)
            if (open) mbar_arrive(&full[(seq - 1) % kSlots]);
            const uint64_t t0 = global_ns();
            for (int t = 0; t < 2; ++t)
                if (qn[t] > 0) drain_wait(&q_full[t], (qn[t] - 1) & 1u, t0);
            for (uint32_t i = seq > kSlots ? seq - kSlots : 0; i < seq; ++i) drain_wait(&full[i % kSlots], (i / kSlots) & 1u, t0);
        } else if (warp == 9 || warp == 11) {
            // ------------------------- MMA issuers, one for each query tile (a whole warp, one lane issues)
            // What a warp's wait or commit takes between two of its MMAs its own MMAs stand still (some 100 and 50
            // cycles); two warps fill each other's gaps. Every value that an MMA takes comes from constants, kernel
            // parameters and warp-wide reductions, so that it stays in uniform registers.
            const int t = __reduce_max_sync(0xffffffffu, warp == 11);
            constexpr uint32_t kIdS = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(kTile >> 3) << 17) | ((uint32_t)(kTile >> 4) << 24);
            const uint32_t id_o = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 16) | ((uint32_t)((p.D + 15) / 16 * 2) << 17) |
                                  ((uint32_t)(kTile >> 4) << 24);
            const uint64_t dq = sw128_desc(smem_u32(sQ + (kDeal ? 0 : t * kQTile))), dk = sw128_desc(smem_u32(sKV));
            const uint64_t dv = half_desc(smem_u32(sKV));
            const uint32_t tm = __reduce_max_sync(0xffffffffu, tmem), tS = tm + t * kTile, tO = tm + 2 * kTile + t * kTile;
            bool issued = false, ok = true;
            uint32_t qn = 0, pn = 0;  // phases of q_full and p_full
            int slot = 0;             // ring slot of the next tile's first chunk
            uint32_t seq = 0;         // tiles before it
            auto place = [&](int at) { return at >= kSlots ? at - kSlots : at; };
            auto landed = [&] {
                ok = wait_warp(&full[seq % kSlots], (seq / kSlots) & 1u);
                tc_fence_after();
                return ok;
            };
            auto advance = [&](int chunks) {
                slot = place(slot + chunks);
                ++seq;
            };
            // A tile that this query tile does not read. (It has landed: so its barriers' next phase has not begun.)
            auto skip = [&](int chunks) {
                if (!landed()) return;
                if (lane == 0) mbar_arrive(&done[seq % kSlots]);
                __syncwarp();
                advance(chunks);
            };
            // S = Q K^T with the next tile; last: the item's last use of Q
            auto scores = [&](bool last) {
                if (!landed()) return;
                if (elect_one()) {
#pragma unroll
                    for (int c = 0; c < 3; ++c) {
                        if (c >= k_chunks) break;
                        const int part = c < own_chunks ? own - 64 * c : rope;  // elements of the chunk, or more
                        const uint64_t b = dk + (uint64_t)((uint32_t)(place(slot + c) * kHalf) >> 4);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            if (16 * i >= part) break;
                            mma_ss(tS, dq + (uint64_t)((c * kHalf + i * 32) >> 4), b + (uint64_t)(i * 32 >> 4), kIdS, c + i != 0);
                        }
                    }
                    mma_commit(&s_full[t]);
                    mma_commit(&done[seq % kSlots]);
                    if (last) mma_commit(&q_empty[kDeal ? 0 : t]);
                }
                __syncwarp();
                issued = true;
                advance(k_chunks);
            };
            // O += P V with the next tile
            auto values = [&](bool first, bool last) {
                if (!landed()) return;
                ok = wait_warp(&p_full[t], pn++ & 1u);
                if (!ok) return;
                tc_fence_after();
                if (elect_one()) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const uint64_t b = dv + (uint64_t)((uint32_t)(place(slot + h) * kHalf) >> 4);
#pragma unroll
                        for (int c = 0; c < 4; ++c)  // 16 keys: 8 columns of P, 2 KB of V
                            mma_ts(tO, tS + 8 * (4 * h + c), b + (uint64_t)(c * 2048 >> 4), id_o, h + c != 0 || !first);
                    }
                    mma_commit(&done[seq % kSlots]);
                    if (last) mma_commit(&o_full[t]);
                }
                __syncwarp();
                advance(2);
            };
            for (int k = 0; ok; ++k) {
                ok = wait_warp(&w_full[k & 1], (uint32_t)(k >> 1) & 1u);
                if (!ok) break;
                const int n0 = __reduce_max_sync(0xffffffffu, work_slots[k & 1].n[0]);
                const int n1 = __reduce_max_sync(0xffffffffu, work_slots[k & 1].n[1]);
                const int end = __reduce_max_sync(0xffffffffu, work_slots[k & 1].end);
                if (lane == 0) mbar_arrive(&w_empty[k & 1]);
                if (end) break;
                const int mine = t ? n1 : n0, n = kDeal ? n0 + n1 : max(n0, n1);
                if (n == 0) continue;
                if (kDeal || mine > 0) ok = wait_warp(&q_full[kDeal ? 0 : t], qn++ & 1u);
                if (kDeal) {
                    if (mine == 0) {
                        if (lane == 0) mbar_arrive(&q_empty[0]);
                        __syncwarp();
                    }
                    auto key = [&](int i) {
                        if ((i & 1) == t) scores(i + 2 >= n);
                        else skip(k_chunks);
                    };
                    for (int i = 0; i < min(n, 2) && ok; ++i) key(i);
                    for (int i = 0; i < n && ok; ++i) {
                        if ((i & 1) == t) values(i < 2, i + 2 >= n);
                        else skip(2);
                        if (ok && i + 2 < n) key(i + 2);
                    }
                    continue;
                }
                for (int j = 0; j < n && ok; ++j) {
                    if (j == 0) {
                        if (mine > 0) scores(mine == 1);
                        else skip(k_chunks);
                        if (!ok) break;
                    }
                    if (j < mine) values(j == 0, j + 1 == mine);
                    else skip(2);
                    if (!ok || j + 1 == n) break;
                    if (j + 1 < mine) scores(j + 2 == mine);
                    else skip(k_chunks);
                }
            }
            if (issued) {  // no MMA is in flight when TMEM is released
                if (elect_one()) mma_commit(&drain[t]);
                __syncwarp();
                drain_wait(&drain[t], 0);
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 9) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
}

// [T, heads, D] bf16 rows as a 3-D tensor in boxes of 64 columns (128-byte
// swizzled; elements past D and rows past T read as 0) of `rows` tokens of one head
bool rows_map(CUtensorMap* map, const Rows& r, int64_t T, int heads, int D, int rows) {
    EncodeTiled fn = encode_fn();
    if (!fn) return false;
    const cuuint64_t least = (cuuint64_t)(2 * D);
    cuuint64_t dims[3] = {(cuuint64_t)D, (cuuint64_t)heads, (cuuint64_t)T};
    cuuint64_t strides[2] = {heads > 1 ? (cuuint64_t)(2 * r.hs) : least, T > 1 ? (cuuint64_t)(2 * r.ts) : least};
    cuuint32_t box[3] = {64, 1, (cuuint32_t)rows}, estr[3] = {1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(r.p), dims, strides, box, estr,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// strides that a tensor map holds: below 2^40 bytes, and not 0 (broadcast rows
// take the CUDA-core kernel)
bool tma_strides(const Rows& r, int64_t T, int heads) {
    const int64_t most = int64_t(1) << 39;
    return (T <= 1 || (r.ts > 0 && r.ts < most)) && (heads <= 1 || (r.hs > 0 && r.hs < most));
}

// the most items of `rows` rows that the lengths can make
int64_t items_of(const AttnProblem& p, int rows) { return (p.T / rows + p.B) * (int64_t)p.Hq; }

template <bool kDeal>
cudaError_t prompt_as(const LatentProblem& p, cudaStream_t stream) {
    constexpr auto kernel = latent_prompt_kernel<kDeal>;
    static DeviceOnce once;
    if (cudaError_t e = once.run([] { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem); });
        e != cudaSuccess)
        return e;
    const AttnProblem& a = p.a;
    CUtensorMap q, k, r, v;
    if (!rows_map(&q, a.q, a.T, a.Hq, p.K, kTile) || !rows_map(&k, a.k, a.Tk, a.Hkv, p.own, kTile) ||
        !rows_map(&v, a.v, a.Tk, a.Hkv, a.D, kTile / 2))
        return cudaErrorInvalidValue;
    if (p.K > p.own) {
        if (!rows_map(&r, p.k_rope, a.Tk, 1, p.K - p.own, kTile)) return cudaErrorInvalidValue;
    } else {
        r = k;  // (not read)
    }
    const int64_t grid = items_of(a, kDeal ? kTile : 2 * kTile);
    if (grid > INT32_MAX) return cudaErrorInvalidConfiguration;
    return launch_k(kernel, dim3((unsigned)grid), dim3(kThreads), kSmem, stream, q, k, r, v, Params{p, tc_wait_limit_ns()});
}

}  // namespace

// (a negative scale would make a row's smallest product its largest score)
bool latent_prompt_tc_supported(const LatentProblem& p) {
    const AttnProblem& a = p.a;
    return a.act_dtype == GBMOE_BF16 && p.K - p.own <= 64 && a.Tk > 0 && a.scale_log2 > 0.0f && tma_strides(a.q, a.T, a.Hq) &&
           tma_strides(a.k, a.Tk, a.Hkv) && tma_strides(a.v, a.Tk, a.Hkv) && (p.K == p.own || tma_strides(p.k_rope, a.Tk, 1));
}

cudaError_t launch_latent_prompt_tc(const LatentProblem& p, cudaStream_t stream) {
    // Too few items for every SM. Us without and with: 1000 tokens of 4 heads 25.7 and 18.5; 4096 of 8 (136 items) 73.8 and
    // 68.5; four prompts of 4000 in all, 8 heads (152 items) 38.3 and 40.1; 4096 of 16 92 and 112 (dealt keys are
    // loaded for half as many rows).
    const bool deal = items_of(p.a, 2 * kTile) < sm_count();
    return deal ? prompt_as<true>(p, stream) : prompt_as<false>(p, stream);
}

}  // namespace gbmoe
