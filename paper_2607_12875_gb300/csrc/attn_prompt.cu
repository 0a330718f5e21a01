// Attention over packed prompts on the tensor cores (bf16, D up to 128).
//
// One CTA holds two tiles of 128 query rows that read the same keys: the same
// 128 tokens of two heads of a group where the group has an even number of
// heads (equal work under a causal mask), else 256 tokens of one head. Per tile
// of 128 keys and for each query tile t:
//   S_t = Q_t K^T      tcgen05.mma, both operands in shared memory, S in TMEM
//   P_t = exp2(scale S_t - m)   one thread per row: S from TMEM to registers,
//                      running maximum and sum, P as bf16 over S in TMEM
//   O_t += P_t V       tcgen05.mma, P from TMEM, V in shared memory (its rows
//                      are keys, so V is the MN-major operand)
// While one tile's softmax runs, the tensor cores work for the other. The row
// maximum m is raised, and O in TMEM rescaled, only when a row's maximum has
// grown by more than 2^8 since the last time: P then stays below 2^8 and the
// final division by the same row's sum makes up for it.
// Warps 0-3 and 4-7: softmax of tile 0 and 1; warp 8: TMA; warp 9: MMA.
// TMEM columns: S_0, S_1 (128 each), O_0, O_1 (128 each).
//
// A masked score gives P = 0, but 0 times a NaN value is a NaN: a row whose
// sums are finite and whose result is not is checked for non-finite values at
// keys that it does not see and computed again without them (repair_row).
//
// Waits are bounded as in the GEMM kernels (tc_ptx.cuh).
#include <climits>

#include "attn_plan.cuh"
#include "tc_ptx.cuh"

namespace gbmoe {
namespace {

using namespace tc;

constexpr int kTile = 128;             // query rows of a tile, keys of a tile
constexpr int kThreads = 320;
constexpr int kHalf = kTile * 128;     // bytes of 128 rows x 64 bf16
constexpr float kGrow = 8.0f;          // log2 of how far a row's maximum may run ahead of m

template <int DK>
struct Smem {
    static constexpr int TILE = DK / 64 * kHalf;          // one Q, K or V tile
    static constexpr int STAGES = DK == 128 ? 5 : 8;      // K and V tiles in flight, in turn
    static constexpr int BYTES = 1024 + (2 + STAGES) * TILE + 256;
};

struct Params {
    AttnProblem a;
    int pair_heads;  // the two query tiles are two heads (else 256 tokens)
    uint64_t wait_limit_ns;
};

__device__ __forceinline__ void tma_load_3d(void* dst, const CUtensorMap* map, int x, int y, int z, uint64_t* bar) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
        ::"r"(smem_u32(dst)), "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(smem_u32(bar))
        : "memory");
}

// S = A B^T: both K-major
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
        : "memory");
}
// A from TMEM
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
        "r"(a), "l"(b), "r"(idesc), "r"(accumulate)
        : "memory");
}

// Descriptor of a V tile (rows of 64 values of one key, 128-byte swizzled; the
// MMA's N runs along a row): 64-column groups kHalf apart (leading offset),
// groups of 8 keys 1024 bytes apart (stride offset).
__device__ __forceinline__ uint64_t v_desc(uint32_t saddr) {
    return (uint64_t)((saddr & 0x3FFFFu) >> 4) | (uint64_t)(kHalf >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 |
           (uint64_t)1 << 46 | (uint64_t)2 << 61;
}

#define GB_R32(r)                                                                                                     \
    "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]),       \
        "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]), "+r"(r[16]),        \
        "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]), "+r"(r[24]),       \
        "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31])

// 32 columns of this thread's TMEM lane, without the wait: several in flight,
// then ld_wait(), then pin32 of each (so that no use moves above the wait)
__device__ __forceinline__ void tmem_ld32_async(uint32_t taddr, uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, "
        "%15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
          "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
          "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(taddr));
}
__device__ __forceinline__ void ld_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void pin32(uint32_t (&r)[32]) { asm volatile("" : GB_R32(r)); }

__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, "
        "%14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};" ::"r"(r[0]),
        "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
        "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]),
        "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]),
        "r"(r[29]), "r"(r[30]), "r"(r[31]), "r"(taddr)
        : "memory");
}
__device__ __forceinline__ void st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

__device__ __forceinline__ bool finite(float x) { return fabsf(x) <= 3.402823466e38f; }

// The row of token t, head h once more, by a whole warp and without the values
// it does not see: m and l are its softmax's maximum (base 2) and sum, lo .. hi
// the keys it sees. Stops when every column is NaN.
__device__ __noinline__ void repair_row(const AttnProblem& p, int64_t k0, int64_t t, int h, int lo, int hi, float m, float l) {
    const int lane = threadIdx.x & 31, hk = h / (p.Hq / p.Hkv), d = 4 * lane;
    const __nv_bfloat16* q = static_cast<const __nv_bfloat16*>(p.q.p) + t * p.q.ts + h * p.q.hs;
    const __nv_bfloat16* k = static_cast<const __nv_bfloat16*>(p.k.p) + hk * p.k.hs;
    const __nv_bfloat16* v = static_cast<const __nv_bfloat16*>(p.v.p) + hk * p.v.hs;
    float o[4] = {0.f, 0.f, 0.f, 0.f};
    for (int j0 = lo; j0 <= hi; j0 += 32) {
        float w = 0.0f;
        if (j0 + lane <= hi) {
            float s = 0.0f;
            for (int c = 0; c < p.D; c += 8) {
                float a[8], b[8];
                Vec8<__nv_bfloat16>::load(q + c, a);
                Vec8<__nv_bfloat16>::load(k + (k0 + j0 + lane) * p.k.ts + c, b);
#pragma unroll
                for (int i = 0; i < 8; ++i) s = fmaf(a[i], b[i], s);
            }
            w = exp2f(fmaf(s, p.scale_log2, -m));
        }
        for (int i = 0; i < 32 && j0 + i <= hi; ++i) {
            const float wi = __shfl_sync(0xffffffffu, w, i);
            if (d < p.D) {
                const uint2 u = *reinterpret_cast<const uint2*>(v + (k0 + j0 + i) * p.v.ts + d);
                o[0] = fmaf(wi, bf16lo(u.x), o[0]), o[1] = fmaf(wi, bf16hi(u.x), o[1]);
                o[2] = fmaf(wi, bf16lo(u.y), o[2]), o[3] = fmaf(wi, bf16hi(u.y), o[3]);
            }
        }
        const bool dead = d >= p.D || (isnan(o[0]) && isnan(o[1]) && isnan(o[2]) && isnan(o[3]));
        if (__all_sync(0xffffffffu, dead)) break;
    }
    __nv_bfloat16* out = const_cast<__nv_bfloat16*>(static_cast<const __nv_bfloat16*>(p.out.p)) + t * p.out.ts + h * p.out.hs;
    const float inv = 1.0f / l;
    if (d < p.D)
        *reinterpret_cast<uint2*>(out + d) = make_uint2(pack_bf16x2(o[0] * inv, o[1] * inv), pack_bf16x2(o[2] * inv, o[3] * inv));
}

template <int DK>
__global__ void __launch_bounds__(kThreads, 1)
attn_prompt_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                   const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ Params pp) {
    pdl_enter();
    using L = Smem<DK>;
    constexpr int STAGES = L::STAGES;
    constexpr int TILE = L::TILE;
    const AttnProblem& p = pp.a;
    __shared__ int64_t plan[plan_words(kThreads)];
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    uint8_t* sQ = smem;               // two query tiles; at the end the output rows
    uint8_t* sKV = smem + 2 * TILE;
    uint64_t* bars = reinterpret_cast<uint64_t*>(sKV + STAGES * TILE);
    uint64_t* full = bars;            // a K or V tile landed
    uint64_t* empty = full + STAGES;  // the MMAs that read it finished
    uint64_t* q_full = empty + STAGES;
    uint64_t* s_full = q_full + 2;    // S of a query tile is complete (and so is every MMA before it)
    uint64_t* p_full = s_full + 2;    // its P is written, O rescaled
    uint64_t* o_full = p_full + 2;    // its O is complete
    uint64_t* drain = o_full + 2;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(drain + 1);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int groups = pp.pair_heads ? p.Hq / 2 : p.Hq;
    const int rows_per = pp.pair_heads ? kTile : 2 * kTile;
    const Place at = find_tile(p, blockIdx.x / groups, rows_per, plan);
    if (at.b < 0) return;
    const Seq s = load_seq(p, at.b);
    // the last tiles, which see the most keys, first
    const int tile = (s.nq + rows_per - 1) / rows_per - 1 - (int)at.at;
    const int head0 = pp.pair_heads ? 2 * (blockIdx.x % groups) : blockIdx.x % groups;
    const int head_kv = head0 / (p.Hq / p.Hkv);
    // query tile t: rows row0(t) .. of the sequence, n_rows(t) of them, and the key tiles 0 .. n_tiles(t) - 1 from k_first on
    auto row0 = [&](int t) { return tile * rows_per + (pp.pair_heads ? 0 : t * kTile); };
    auto n_rows = [&](int t) { return min(kTile, s.nq - row0(t)); };
    int lo0, hi0;
    seen_keys(p, s, row0(0), lo0, hi0);
    const int k_first = hi0 < 0 ? 0 : lo0 & ~(kTile - 1);
    auto n_tiles = [&](int t) {
        if (n_rows(t) <= 0) return 0;
        int lo, hi;
        seen_keys(p, s, row0(t) + n_rows(t) - 1, lo, hi);  // its last row sees the furthest
        return hi < k_first ? 0 : (hi - k_first) / kTile + 1;
    };
    const int n0 = n_tiles(0), n1 = n_tiles(1), n_max = max(n0, n1);

    if (threadIdx.x == 0) {
        for (int i = 0; i < STAGES; ++i) {
            mbar_init(&full[i], 1);
            mbar_init(&empty[i], 1);
        }
        for (int t = 0; t < 2; ++t) {
            mbar_init(&q_full[t], 1);
            mbar_init(&s_full[t], 1);
            mbar_init(&p_full[t], 4);  // one arrival per softmax warp
            mbar_init(&o_full[t], 1);
        }
        mbar_init(drain, 1);
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

    if (warp == 8 && lane == 0 && n_max > 0) {
        // ------------------------------------------------------ TMA producer
        uint32_t inflight = 0, par = 0;
        for (int t = 0; t < 2; ++t) {
            if ((t ? n1 : n0) == 0) continue;
            mbar_expect_tx(&q_full[t], TILE);
            for (int c = 0; c < DK / 64; ++c)
                tma_load_3d(sQ + t * TILE + c * kHalf, &tm_q, 64 * c, head0 + (pp.pair_heads ? t : 0), s.q0 + row0(t), &q_full[t]);
        }
        int stage = 0;
        uint32_t phase = 0;
        for (int i = 0; i < 2 * n_max; ++i) {  // K_0, V_0, K_1, V_1, ...
            if (!mbar_wait(&empty[stage], phase ^ 1, abort_flag, p.err, pp.wait_limit_ns)) break;
            const CUtensorMap* map = i & 1 ? &tm_v : &tm_k;
            mbar_expect_tx(&full[stage], TILE);
            for (int c = 0; c < DK / 64; ++c)
                tma_load_3d(sKV + stage * TILE + c * kHalf, map, 64 * c, head_kv, (int)(s.k0 + k_first + (i >> 1) * kTile), &full[stage]);
            inflight |= 1u << stage;
            par = (par & ~(1u << stage)) | (phase << stage);
            if (++stage == STAGES) { stage = 0; phase ^= 1; }
        }
        // every copy has landed before the CTA leaves
        const uint64_t t0 = global_ns();
        for (int t = 0; t < 2; ++t)
            if ((t ? n1 : n0) > 0) drain_wait(&q_full[t], 0, t0);
        for (int i = 0; i < STAGES; ++i)
            if ((inflight >> i) & 1u) drain_wait(&full[i], (par >> i) & 1u, t0);
    } else if (warp == 9 && n_max > 0) {
        // ------------------------- MMA issuer (the whole warp, one lane issues)
        const int ksteps = (p.D + 15) / 16;
        constexpr uint32_t kIdS = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(kTile >> 3) << 17) | ((uint32_t)(kTile >> 4) << 24);
        const uint32_t id_o = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 16) | ((uint32_t)(ksteps * 2) << 17) |
                              ((uint32_t)(kTile >> 4) << 24);
        const uint64_t dq = sw128_desc(smem_u32(sQ)), dk = sw128_desc(smem_u32(sKV)), dv = v_desc(smem_u32(sKV));
        bool ok = true, issued = false;
        auto slot_of = [](int i) { return i % STAGES; };
        auto wait_tile = [&](int i) {  // tile i of the K_0, V_0, K_1, .. sequence
            ok = ok && warp_wait(&full[slot_of(i)], (uint32_t)(i / STAGES) & 1u, abort_flag, p.err, pp.wait_limit_ns);
            return ok;
        };
        auto scores = [&](int t, int i) {  // S_t = Q_t K^T with the K tile i
            if (elect_one()) {
                const uint64_t a = dq + (uint64_t)(t * TILE >> 4), b = dk + (uint64_t)(slot_of(i) * TILE >> 4);
                for (int c = 0; c < ksteps; ++c) {
                    const uint64_t off = (uint64_t)((c >> 2) * kHalf + (c & 3) * 32) >> 4;
                    mma_ss(tmem + t * kTile, a + off, b + off, kIdS, c != 0);
                }
                mma_commit(&s_full[t]);
            }
            __syncwarp();
            issued = true;
        };
        for (int t = 0; t < 2 && ok; ++t)
            if ((t ? n1 : n0) > 0) ok = warp_wait(&q_full[t], 0, abort_flag, p.err, pp.wait_limit_ns);
        if (ok && wait_tile(0)) {
            tc_fence_after();
            for (int t = 0; t < 2; ++t)
                if ((t ? n1 : n0) > 0) scores(t, 0);
            if (elect_one()) mma_commit(&empty[slot_of(0)]);
            __syncwarp();
        }
        for (int j = 0; j < n_max && ok; ++j) {
            if (!wait_tile(2 * j + 1)) break;
            if (j + 1 < n_max && !wait_tile(2 * j + 2)) break;
            for (int t = 0; t < 2 && ok; ++t) {
                const int n = t ? n1 : n0;
                if (j >= n) continue;
                ok = warp_wait(&p_full[t], (uint32_t)j & 1u, abort_flag, p.err, pp.wait_limit_ns);
                if (!ok) break;
                tc_fence_after();
                if (elect_one()) {
                    const uint64_t b = dv + (uint64_t)(slot_of(2 * j + 1) * TILE >> 4);
                    const uint32_t d = tmem + 2 * kTile + t * kTile, a = tmem + t * kTile;
#pragma unroll
                    for (int c = 0; c < kTile / 16; ++c)  // 16 keys: 8 columns of P, 2 KB of V
                        mma_ts(d, a + 8 * c, b + (uint64_t)(c * 2048 >> 4), id_o, (j | c) != 0);
                    if (j == n - 1) mma_commit(&o_full[t]);
                }
                __syncwarp();
                if (j + 1 < n) scores(t, 2 * j + 2);
            }
            if (!ok) break;
            if (elect_one()) {
                mma_commit(&empty[slot_of(2 * j + 1)]);
                if (j + 1 < n_max) mma_commit(&empty[slot_of(2 * j + 2)]);
            }
            __syncwarp();
        }
        if (issued) {  // no MMA is in flight when TMEM is released
            if (elect_one()) mma_commit(drain);
            __syncwarp();
            drain_wait(drain, 0);
        }
    } else if (warp < 8) {
        // ------------------------------------------------- softmax, one row each
        const int t = warp >> 2, r = (warp & 3) * 32 + lane;
        const int n = t ? n1 : n0, rows = n_rows(t);
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t tS = tmem + lanes + t * kTile, tO = tmem + lanes + 2 * kTile + t * kTile;
        int lo = 0, hi = -1;
        if (r < rows) seen_keys(p, s, row0(t) + r, lo, hi);
        const float scale = p.scale_log2;
        float m = neg_inf(), l = 0.0f;
        bool ok = true;
        for (int j = 0; j < n; ++j) {
            if (!warp_wait(&s_full[t], (uint32_t)j & 1u, abort_flag, p.err, pp.wait_limit_ns)) { ok = false; break; }
            tc_fence_after();
            uint32_t u[4][32];
#pragma unroll
            for (int c = 0; c < 4; ++c) tmem_ld32_async(tS + 32 * c, u[c]);
            ld_wait();
#pragma unroll
            for (int c = 0; c < 4; ++c) pin32(u[c]);
            const int first = lo - (k_first + j * kTile), last = hi - (k_first + j * kTile);  // columns first .. last are seen
            if (__any_sync(0xffffffffu, first > 0 || last < kTile - 1)) {
#pragma unroll
                for (int c = 0; c < 4; ++c)
#pragma unroll
                    for (int i = 0; i < 32; ++i)
                        if (32 * c + i < first || 32 * c + i > last) u[c][i] = 0xff800000u;
            }
            float mx[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                mx[c] = __uint_as_float(u[c][0]);
#pragma unroll
                for (int i = 1; i < 32; ++i) mx[c] = fmaxf(mx[c], __uint_as_float(u[c][i]));
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
            float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                uint32_t w[32];
#pragma unroll
                for (int i = 0; i < 32; ++i) {
                    const int e = 64 * half + 2 * i;
                    const float2 x = unpack2(fma2(pack2(__uint_as_float(u[e >> 5][e & 31]), __uint_as_float(u[e >> 5][(e & 31) + 1])), sc2, nb2));
                    const float a = ex2(x.x), b = ex2(x.y);
                    sum[2 * (i & 1)] += a;
                    sum[2 * (i & 1) + 1] += b;
                    w[i] = pack_bf16x2(a, b);
                }
                tmem_st32(tS + 32 * half, w);
            }
            l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
            st_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&p_full[t]);
        }
        // ------------------------------------------------------------ result
        if (ok && n > 0) ok = warp_wait(&o_full[t], 0, abort_flag, p.err, pp.wait_limit_ns);
        tc_fence_after();
        if (ok && rows > 0) {
            const bool empty = hi < lo;
            const float inv = empty ? 0.0f : 1.0f / l;
            const int64_t tok = s.q0 + row0(t) + r;
            const int head = head0 + (pp.pair_heads ? t : 0);
            uint8_t* buf = sQ + t * TILE + (warp & 3) * 32 * (2 * DK);  // this warp's 32 rows of 2 DK bytes
            bool good = true;
#pragma unroll 1
            for (int c = 0; c < DK; c += 32) {
                uint32_t o[32];
                if (n > 0) {
                    tmem_ld32_async(tO + c, o);
                    ld_wait();
                    pin32(o);
                }
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    uint32_t w[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float a = empty ? 0.0f : __uint_as_float(o[8 * q + 2 * i]) * inv;
                        const float b = empty ? 0.0f : __uint_as_float(o[8 * q + 2 * i + 1]) * inv;
                        if (c + 8 * q < p.D) good = good && finite(a) && finite(b);
                        w[i] = pack_bf16x2(a, b);
                    }
                    // 16-byte chunk c/8 + q of row `lane`, spread over the banks
                    const int chunk = (c / 8 + q) ^ (lane & 7);
                    *reinterpret_cast<uint4*>(buf + lane * (2 * DK) + chunk * 16) = make_uint4(w[0], w[1], w[2], w[3]);
                }
            }
            __syncwarp();
            // whole rows to memory: 2 DK / 16 lanes per row
            constexpr int kChunks = DK / 8;
            __nv_bfloat16* out = const_cast<__nv_bfloat16*>(static_cast<const __nv_bfloat16*>(p.out.p)) + head * p.out.hs;
            const int64_t tok0 = tok - lane;
            const int left = min(32, rows - (warp & 3) * 32);
#pragma unroll 1
            for (int i = lane; i < 32 * kChunks; i += 32) {
                const int rr = i / kChunks, ch = i % kChunks;
                if (rr < left && 8 * ch < p.D)
                    *reinterpret_cast<uint4*>(out + (tok0 + rr) * p.out.ts + 8 * ch) =
                        *reinterpret_cast<const uint4*>(buf + rr * (2 * DK) + ((ch ^ (rr & 7)) * 16));
            }
            if (r < rows && p.lse) p.lse[tok * p.Hq + head] = empty ? neg_inf() : (m + log2f(l)) * kLn2;
            // rows that may hold a masked key's NaN
            uint32_t again = __ballot_sync(0xffffffffu, r < rows && !empty && !good && finite(m) && finite(l) && l > 0.0f);
            while (again) {
                const int src = __ffs(again) - 1;
                again &= again - 1;
                const int rlo = __shfl_sync(0xffffffffu, lo, src), rhi = __shfl_sync(0xffffffffu, hi, src);
                const float rm = __shfl_sync(0xffffffffu, m, src), rl = __shfl_sync(0xffffffffu, l, src);
                __syncwarp();  // (the row's first version is stored before the second)
                repair_row(p, s.k0, tok0 + src, head, rlo, rhi, rm, rl);
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 9) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
}

// [T, heads, D] bf16 rows as a 3-D tensor in boxes of 64 x 1 x 128 (128-byte
// swizzled); elements past D and rows past T read as 0
bool rows_map(CUtensorMap* map, const Rows& r, int64_t T, int heads, int D) {
    EncodeTiled fn = encode_fn();
    if (!fn) return false;
    const cuuint64_t least = (cuuint64_t)(2 * D);
    cuuint64_t dims[3] = {(cuuint64_t)D, (cuuint64_t)heads, (cuuint64_t)T};
    cuuint64_t strides[2] = {heads > 1 ? (cuuint64_t)(2 * r.hs) : least, T > 1 ? (cuuint64_t)(2 * r.ts) : least};
    cuuint32_t box[3] = {64, 1, kTile}, estr[3] = {1, 1, 1};
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

template <int DK>
cudaError_t prompt_as(const AttnProblem& p, cudaStream_t stream) {
    constexpr auto kernel = attn_prompt_kernel<DK>;
    static DeviceOnce once;
    if (cudaError_t e = once.run([] {
            return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, Smem<DK>::BYTES);
        });
        e != cudaSuccess)
        return e;
    CUtensorMap q, k, v;
    if (!rows_map(&q, p.q, p.T, p.Hq, p.D) || !rows_map(&k, p.k, p.Tk, p.Hkv, p.D) || !rows_map(&v, p.v, p.Tk, p.Hkv, p.D))
        return cudaErrorInvalidValue;
    Params pp{p, (p.Hq / p.Hkv) % 2 == 0, tc_wait_limit_ns()};
    const int64_t grid = (p.T / (pp.pair_heads ? kTile : 2 * kTile) + p.B) * (int64_t)(pp.pair_heads ? p.Hq / 2 : p.Hq);
    if (grid > INT32_MAX) return cudaErrorInvalidConfiguration;
    return launch_k(kernel, dim3((unsigned)grid), dim3(kThreads), Smem<DK>::BYTES, stream, q, k, v, pp);
}

}  // namespace

// (a negative scale would make a row's smallest product its largest score)
bool attn_prompt_tc_supported(const AttnProblem& p) {
    return p.act_dtype == GBMOE_BF16 && p.D <= 128 && !p.paged && p.Tk > 0 && p.scale_log2 > 0.0f &&
           tma_strides(p.q, p.T, p.Hq) && tma_strides(p.k, p.Tk, p.Hkv) && tma_strides(p.v, p.Tk, p.Hkv);
}

cudaError_t launch_attn_prompt_tc(const AttnProblem& p, cudaStream_t stream) {
    return p.D <= 64 ? prompt_as<64>(p, stream) : prompt_as<128>(p, stream);
}

}  // namespace gbmoe
