// Attention over packed prompts on the tensor cores (bf16, D up to 128).
//
// One CTA holds two tiles of 128 query rows that read the same keys. A row is a
// token and one of H heads of a group, H the largest power of two in the group's
// number of heads (up to 32): 256 / H tokens, so that short prompts and the ends
// of long ones fill the tiles. Or, for short prompts, the group's heads and empty
// rows up to the next power of two (kPad). Per tile
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
// kDeal, where there is too little work for every SM: the two tiles are one tile
// of 128 rows twice, with every other tile of keys each, and their results are
// joined at the end.
// Warps 0-3 and 4-7: softmax of tile 0 and 1 and their results; warp 8: TMA; warp
// 9: MMA; warp 10: scheduler. A CTA goes on with the work of CTAs that have not
// started (cluster launch control), so the loads, the first products and the search
// for the next work run while the softmax warps still write the last results.
// TMEM columns: S_0, S_1 (128 each), O_0, O_1 (128 each).
//
// Bound by the exponentials and the hand-overs between the softmax warps and the
// MMA: 2680 cycles for 128 keys of two tiles of D 128, whose products take 2048
// (the softmax alone takes 930 for one tile, a hand-over there and back 360), and
// some 5 us for each pair of tiles that a CTA takes. 16384 tokens of 32 query and 8
// kv heads, causal: 1.41 ms, 1.56 PFLOP/s, call after call (1.30 ms one at a time);
// 7 prompts of 8192 in all: 100 us.
//
// P is rounded to bf16, an error of up to 2^-8 of each weight beside the result's
// own rounding (2.0e-3 against 1.6e-3 of the result on average): the MMA takes both
// operands in one 16-bit type, and V is bf16.
//
// A masked score gives P = 0, but 0 times a NaN value is a NaN: a row whose
// sums are finite and whose result is not is checked for non-finite values at
// keys of its tiles that it does not see, and computed again without them if there
// are any (repair_rows: by one warp, 0.15 us for each key of a row; a function of its
// own, of no more registers than leave the softmax its own). The last tile brings
// along values from behind a sequence's end: to set those to 0 in shared memory
// before the product took 8 to 11 % of batches of prompts of up to 100 tokens (and of
// long ones alone, 1 to 5 % by the code's arrangement), so they are left in.
//
// Waits are bounded as in the GEMM kernels (tc_ptx.cuh).
#include <climits>

#include "attn_plan.cuh"
#include "tc_ptx.cuh"

namespace gbmoe {
namespace {

using namespace tc;

constexpr int kTile = 128;             // query rows of a tile, keys of a tile
constexpr int kThreads = 384;
constexpr int kHalf = kTile * 128;     // bytes of 128 rows x 64 bf16
constexpr float kGrow = 8.0f;          // log2 of how far a row's maximum may run ahead of m

template <int DK>
struct Smem {
    static constexpr int TILE = DK / 64 * kHalf;          // one Q, K or V tile
    static constexpr int STAGES = DK == 128 ? 4 : 8;      // K and V tiles in flight, in turn
    static constexpr int OUT = 8 * 2 * 2048;              // output rows on their way: two buffers of each softmax warp
    static_assert(STAGES * 16 + 256 <= 512, "barriers");
    static constexpr int BYTES = 1024 + (2 + STAGES) * TILE + OUT + 512;
};

struct Params {
    AttnProblem a;
    int hlog, heads;  // log2 of a token's rows in a tile, and how many of them are heads
    uint64_t wait_limit_ns;
};

__device__ __forceinline__ void tma_load_3d(void* dst, const CUtensorMap* map, int x, int y, int z, uint64_t* bar) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
        ::"r"(smem_u32(dst)), "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(smem_u32(bar))
        : "memory");
}

__device__ __forceinline__ void tma_store_3d(const CUtensorMap* map, const void* src, int x, int y, int z) {
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%1, %2, %3}], [%4];" ::"l"(
                     reinterpret_cast<uint64_t>(map)),
                 "r"(x), "r"(y), "r"(z), "r"(smem_u32(src))
                 : "memory");
    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
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

__device__ __forceinline__ float max3(float a, float b, float c) {
    float y;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
    return y;
}

__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {  // two fp32 sums
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

__device__ __forceinline__ bool finite(float x) { return fabsf(x) <= 3.402823466e38f; }

// The first and last of the keys from .. to - 1 of kv head hk, those that every
// row of the warp sees (seen_lo .. seen_hi) left out, at which a value is not
// finite (x > y: none). By a whole warp, a key for each lane.
__device__ __forceinline__ int2 bad_keys(const AttnProblem& p, int64_t k0, int hk, int from, int to, int seen_lo, int seen_hi) {
    const int lane = threadIdx.x & 31;
    const __nv_bfloat16* v = static_cast<const __nv_bfloat16*>(p.v.p) + k0 * p.v.ts + hk * p.v.hs;
    int first = INT_MAX, last = -1;
    for (int j0 = from; j0 < to; j0 += 32) {
        if (j0 >= seen_lo && j0 < seen_hi - 31) {  // (on to the keys that some row does not see)
            j0 += (seen_hi - 31 - j0) / 32 * 32;
            continue;
        }
        const int j = j0 + lane;
        if (j >= to || (j >= seen_lo && j <= seen_hi)) continue;
        bool bad = false;
        for (int c = 0; c < p.D; c += 8) {
            const uint4 u = *reinterpret_cast<const uint4*>(v + j * p.v.ts + c);
            bad = bad || (__vcmpgeu2(u.x & 0x7fff7fffu, 0x7f807f80u) | __vcmpgeu2(u.y & 0x7fff7fffu, 0x7f807f80u) |
                          __vcmpgeu2(u.z & 0x7fff7fffu, 0x7f807f80u) | __vcmpgeu2(u.w & 0x7fff7fffu, 0x7f807f80u)) != 0;
        }
        if (bad) first = min(first, j), last = j;
    }
    return make_int2(__reduce_min_sync(0xffffffffu, first), __reduce_max_sync(0xffffffffu, last));
}

// The row of token t, head h once more, by a whole warp and without the values
// it does not see: m and l are its softmax's maximum (base 2) and sum, lo .. hi
// the keys it sees. Stops when every column is NaN.
__device__ __forceinline__ void repair_row(const AttnProblem& p, int64_t k0, int64_t t, int h, int lo, int hi, float m, float l) {
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
        for (int i0 = 0; i0 < 32 && j0 + i0 <= hi; i0 += 8) {  // loads in flight
            uint2 u[8];
#pragma unroll
            for (int i = 0; i < 8; ++i)
                u[i] = d < p.D && j0 + i0 + i <= hi ? *reinterpret_cast<const uint2*>(v + (k0 + j0 + i0 + i) * p.v.ts + d) : make_uint2(0, 0);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float wi = __shfl_sync(0xffffffffu, w, i0 + i);
                o[0] = fmaf(wi, bf16lo(u[i].x), o[0]), o[1] = fmaf(wi, bf16hi(u[i].x), o[1]);
                o[2] = fmaf(wi, bf16lo(u[i].y), o[2]), o[3] = fmaf(wi, bf16hi(u[i].y), o[3]);
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

// Rows `again` of the warp, which hold values that are not finite (a lane's own: token t, head h and so on):
// those are computed again that have such a value among the keys of their `tiles` tiles that they do not
// see. (A row that sees it is not a number, and computing it again takes as long as all its
// products.) Keys of the tiles: up to the end of the buffer, past which the tiles hold zeros.
__device__ __noinline__ void repair_rows(const AttnProblem& p, uint32_t again, int64_t k0, int k_first, int tiles, int64_t t, int h,
                                         int lo, int hi, float m, float l) {
    const int lane = threadIdx.x & 31;
    const bool mine = again >> lane & 1u;
    const int seen_lo = __reduce_max_sync(0xffffffffu, mine ? lo : 0), seen_hi = __reduce_min_sync(0xffffffffu, mine ? hi : INT_MAX);
    const int hk = __shfl_sync(0xffffffffu, h / (p.Hq / p.Hkv), __ffs(again) - 1);
    const int2 bad = bad_keys(p, k0, hk, k_first, (int)min64(k_first + (int64_t)tiles * kTile, p.Tk - k0), seen_lo, seen_hi);
    again = __ballot_sync(0xffffffffu, mine && (bad.x < lo || bad.y > hi));
    if (again == 0) return;
    if (lane == 0) bulk_wait_all();  // the rows' first versions are stored before the second
    __syncwarp();
    while (again) {
        const int src = __ffs(again) - 1;
        again &= again - 1;
        repair_row(p, k0, __shfl_sync(0xffffffffu, t, src), __shfl_sync(0xffffffffu, h, src), __shfl_sync(0xffffffffu, lo, src),
                   __shfl_sync(0xffffffffu, hi, src), __shfl_sync(0xffffffffu, m, src), __shfl_sync(0xffffffffu, l, src));
    }
}

// One work item as the scheduler warp hands it out.
struct Work {
    Seq s;
    int tok0[2], rows[2];   // query tile t: first token of the sequence, rows (<= 0: none)
    int n[2];               // its key tiles, from k_first on
    int k_first, head0, head_kv;
    int end;                // 1: no more work
};

// Finds row tiles of the list, by a whole warp (every lane gets the answer). The
// indices that a CTA is given mostly rise, so a search goes on where the last one ended.
struct TileFinder {
    int base = 0;        // first of the 32 sequences looked at last
    int64_t before = 0;  // tiles before them

    // b = -1: past the end
    __device__ __forceinline__ Place find(const AttnProblem& p, int64_t index, int rows) {
        const int lane = threadIdx.x & 31;
        if (index < before) base = 0, before = 0;
        for (; base < p.B; base += 32) {
            const int64_t v = base + lane < p.B ? row_tiles(p, load_seq(p, base + lane), rows) : 0;
            const int64_t pre = warp_scan(v) + before;
            const uint32_t hit = __ballot_sync(0xffffffffu, index < pre);
            if (hit) {
                const int l = __ffs(hit) - 1;
                return Place{base + l, index - __shfl_sync(0xffffffffu, pre - v, l)};
            }
            before = __shfl_sync(0xffffffffu, pre, 31);
        }
        return Place{-1, 0};
    }
};

// Asks for a CTA of this grid that has not started (its index comes as 16 bytes at dst, counted on bar).
__device__ __forceinline__ void try_cancel(void* dst, uint64_t* bar) {
    mbar_expect_tx(bar, 16);
    asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];" ::"r"(smem_u32(dst)),
                 "r"(smem_u32(bar))
                 : "memory");
}
// the answer: whether there was one, and its blockIdx.x
__device__ __forceinline__ bool cancelled(const void* src, uint32_t& x) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .b128 h;\n\t.reg .pred q;\n\t.reg .b32 y, z, w;\n\t"
        "ld.shared.b128 h, [%2];\n\t"
        "clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 q, h;\n\t"
        "selp.u32 %0, 1, 0, q;\n\t"
        "mov.b32 %1, 0;\n\t"
        "@q clusterlaunchcontrol.query_cancel.get_first_ctaid.v4.b32.b128 {%1, y, z, w}, h;\n\t}"
        : "=r"(ok), "=r"(x)
        : "r"(smem_u32(src))
        : "memory");
    return ok != 0;
}

template <int DK, bool kDeal, bool kPad>
__global__ void __launch_bounds__(kThreads, 1)
attn_prompt_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                   const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ CUtensorMap tm_o,
                   const __grid_constant__ Params pp) {
    pdl_enter();
    using L = Smem<DK>;
    constexpr int STAGES = L::STAGES;
    constexpr int TILE = L::TILE;
    const AttnProblem& p = pp.a;
    __shared__ Work work_slots[2];
    __shared__ __align__(16) uint4 answer;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    uint8_t* sQ = smem;  // two query tiles
    uint8_t* sKV = smem + 2 * TILE;
    // kDeal, which has one query tile: maximum, sum and results' check of the softmax warps' rows
    float(*stats)[8][32] = reinterpret_cast<float(*)[8][32]>(sQ + TILE);
    uint8_t* sO = sKV + STAGES * TILE;
    uint64_t* bars = reinterpret_cast<uint64_t*>(sO + L::OUT);
    uint64_t* full = bars;            // a K or V tile landed
    uint64_t* empty = full + STAGES;  // the MMAs that read it finished
    uint64_t* q_full = empty + STAGES;
    uint64_t* q_empty = q_full + 2;   // the last product with a query tile finished
    uint64_t* s_full = q_empty + 2;   // S of a query tile is complete (and so is every MMA before it)
    uint64_t* p_full = s_full + 2;    // its P is written, O rescaled, and the V and next K tile are there
    uint64_t* o_full = p_full + 2;    // its O is complete
    uint64_t* w_full = o_full + 2;    // a work item is in its slot
    uint64_t* w_empty = w_full + 2;   // every role has read it
    uint64_t* ans = w_empty + 2;      // the answer to try_cancel
    uint64_t* drain = ans + 1;
    uint64_t* pair = drain + 1;       // kDeal: the two warps of the same rows
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(pair + 4);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int i = 0; i < STAGES; ++i) {
            mbar_init(&full[i], 1);
            mbar_init(&empty[i], 1);
        }
        for (int t = 0; t < 2; ++t) {
            mbar_init(&q_full[t], 1);
            mbar_init(&q_empty[t], 1);
            mbar_init(&s_full[t], 1);
            mbar_init(&p_full[t], 5);    // one arrival per softmax warp, one of the tile watcher
            mbar_init(&o_full[t], 1);
            mbar_init(&w_full[t], 1);
            mbar_init(&w_empty[t], 11);  // softmax warps, TMA, MMA, tile watcher
        }
        mbar_init(ans, 1);
        mbar_init(drain, 1);
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
        bool ok = true;
        for (int k = 0; ok; ++k) {
            if (!wait_warp(&w_full[k & 1], (uint32_t)(k >> 1) & 1u)) break;
            const Work& slot = work_slots[k & 1];
            const Seq s = slot.s;
            const int n = slot.n[t], n2 = slot.n[t ^ 1], rows = slot.rows[t], row = slot.tok0[t] + (r >> pp.hlog), k_first = slot.k_first, end = slot.end;
            const int head0 = slot.head0, place = r & ((1 << pp.hlog) - 1), head = head0 + place;
            const bool have = r < rows && (!kPad || place < pp.heads);
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
            // all 32 rows of this warp belong to the tile: a TMA store of each 32 columns;
            // else plain stores of the valid rows (the others are another sequence's or group's)
            const bool via_tma = !kPad && (warp & 3) * 32 + 32 <= rows;
            uint8_t* stage_buf = sO + warp * 4096;
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
                uint8_t* buf = stage_buf + ((c >> (kDeal ? 6 : 5)) & 1) * 2048;
                if (via_tma) {
                    // The store that last read buf is done reading: within an item the one before the latest. An
                    // item begins with the same buffer whatever the last one ended with (an odd number of chunks: with this
                    // one too, and an item without keys comes here at once), so there every store.
                    if (lane == 0) {
                        if (c < (kDeal ? 64 : 32)) bulk_wait_read<0>();
                        else bulk_wait_read<1>();
                    }
                    __syncwarp();
                }
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
                    const uint4 v = make_uint4(w[0], w[1], w[2], w[3]);
                    // (64-byte rows, 64-byte swizzle; columns past D are not written)
                    if (via_tma) *reinterpret_cast<uint4*>(buf + lane * 64 + ((q ^ ((lane >> 1) & 3)) << 4)) = v;
                    else if (have && c + 8 * q < p.D) *reinterpret_cast<uint4*>(out + c + 8 * q) = v;
                }
                if (via_tma) {
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                    if (lane == 0) tma_store_3d(&tm_o, buf, c, head0, (int)tok);
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
                if (lane == 0) bulk_wait_all();
                __syncwarp();
                __threadfence();
                ok = meet();
                if (t != 0 || !ok) again = 0;
            }
            if (again) repair_rows(p, again, s.k0, k_first, kDeal ? n + n2 : n, tok, head, lo, hi, m, l);
        }
        if (lane == 0) bulk_wait_all();  // stores complete before the CTA leaves
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
        if (warp == 10) {
            // --------------------------------------------------------- scheduler
            const int groups = kPad ? p.Hq / pp.heads : p.Hq >> pp.hlog;
            const int tile_toks = kTile >> pp.hlog, toks = kDeal ? tile_toks : 2 * tile_toks;
            uint32_t block = blockIdx.x;
            TileFinder tiles;
            bool more = true, asked = false;
            uint32_t turn = 0;
            int k = 0;
            for (; more; ++turn) {
                if (lane == 0) try_cancel(&answer, ans);
                asked = true;
                const Place at = tiles.find(p, block / groups, toks);
                if (at.b >= 0) {
                    if (!wait_warp(&w_empty[k & 1], ((uint32_t)(k >> 1) & 1u) ^ 1u)) break;
                    Work w;
                    w.s = load_seq(p, at.b);
                    // the last tiles, which see the most keys, first
                    const int first = ((w.s.nq + toks - 1) / toks - 1 - (int)at.at) * toks;
                    w.head0 = kPad ? (int)(block % groups) * pp.heads : (int)(block % groups) << pp.hlog;
                    w.head_kv = w.head0 / (p.Hq / p.Hkv);
                    w.end = 0;
                    int lo, hi;
                    seen_keys(p, w.s, first, lo, hi);
                    w.k_first = hi < 0 ? 0 : lo & ~(kTile - 1);
#pragma unroll
                    for (int t = 0; t < 2; ++t) {
                        w.tok0[t] = first + (kDeal ? 0 : t * tile_toks);
                        w.rows[t] = min(tile_toks, w.s.nq - w.tok0[t]) << pp.hlog;
                        w.n[t] = 0;
                        if (w.rows[t] > 0) {
                            seen_keys(p, w.s, w.tok0[t] + (w.rows[t] >> pp.hlog) - 1, lo, hi);  // its last token sees the furthest
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
                }
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
            uint32_t inflight = 0, par = 0, qn[2] = {0, 0};
            int stage = 0;
            uint32_t phase = 0;
            bool ok = true;
            for (int k = 0; ok; ++k) {
                if (!wait(&w_full[k & 1], (uint32_t)(k >> 1) & 1u)) break;
                const Work w = work_slots[k & 1];
                mbar_arrive(&w_empty[k & 1]);
                if (w.end) break;
                const int n_max = max(w.n[0], w.n[1]);
                for (int t = 0; t < (kDeal ? 1 : 2) && ok; ++t) {
                    if (w.n[t] == 0) continue;
                    ok = wait(&q_empty[t], (qn[t] & 1u) ^ 1u);
                    if (!ok) break;
                    mbar_expect_tx(&q_full[t], TILE);
                    for (int c = 0; c < DK / 64; ++c)
                        tma_load_3d(sQ + t * TILE + c * kHalf, &tm_q, 64 * c, w.head0, w.s.q0 + w.tok0[t], &q_full[t]);
                    ++qn[t];
                }
                // K_0, V_0, K_1, V_1, ..; kDeal: K_0, K_1, V_0, K_2, V_1, .., K_n-1, V_n-2, V_n-1
                const int n_all = kDeal ? w.n[0] + w.n[1] : n_max;
                for (int i = 0; i < 2 * n_all && ok; ++i) {
                    ok = wait(&empty[stage], phase ^ 1);
                    if (!ok) break;
                    bool value = i & 1;
                    int at = i >> 1;
                    if constexpr (kDeal) {
                        value = i == 2 * n_all - 1 || (i > 0 && !(i & 1));
                        at = i == 0 ? 0 : i == 2 * n_all - 1 ? n_all - 1 : value ? at - 1 : at + 1;
                    }
                    const CUtensorMap* map = value ? &tm_v : &tm_k;
                    mbar_expect_tx(&full[stage], TILE);
                    for (int c = 0; c < DK / 64; ++c)
                        tma_load_3d(sKV + stage * TILE + c * kHalf, map, 64 * c, w.head_kv, (int)(w.s.k0 + w.k_first + at * kTile), &full[stage]);
                    inflight |= 1u << stage;
                    par = (par & ~(1u << stage)) | (phase << stage);
                    if (++stage == STAGES) { stage = 0; phase ^= 1; }
                }
            }
            // every copy has landed before the CTA leaves
            const uint64_t t0 = global_ns();
            for (int t = 0; t < 2; ++t)
                if (qn[t] > 0) drain_wait(&q_full[t], (qn[t] - 1) & 1u, t0);
            for (int i = 0; i < STAGES; ++i)
                if ((inflight >> i) & 1u) drain_wait(&full[i], (par >> i) & 1u, t0);
        } else if (warp == 9) {
            // ------------------------- MMA issuer (the whole warp, one lane issues)
            // Every value that an MMA takes comes from constants, kernel parameters and
            // warp-wide reductions, so that it stays in uniform registers.
            const int ksteps = (p.D + 15) / 16;
            constexpr uint32_t kIdS = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(kTile >> 3) << 17) | ((uint32_t)(kTile >> 4) << 24);
            const uint32_t id_o = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 16) | ((uint32_t)(ksteps * 2) << 17) |
                                  ((uint32_t)(kTile >> 4) << 24);
            const uint64_t dq = sw128_desc(smem_u32(sQ)), dk = sw128_desc(smem_u32(sKV)), dv = v_desc(smem_u32(sKV));
            const uint32_t tm = __reduce_max_sync(0xffffffffu, tmem);
            bool issued = false;
            uint32_t qn0 = 0, qn1 = 0, pn0 = 0, pn1 = 0;  // phases of q_full and p_full
            int stage = 0;  // ring slot of the next tile and its phase
            uint32_t phase = 0;
            auto advance = [&](int& st, uint32_t& ph) {
                if (++st == STAGES) st = 0, ph ^= 1;
            };
            // S_t = Q_t K^T with the K tile in slot st; last: the item's last use of Q_t (kDeal: of the one Q)
            auto scores = [&](int t, int st, bool last) {
                if (elect_one()) {
                    const uint64_t a = dq + (kDeal ? 0 : (uint64_t)(t * TILE >> 4)), b = dk + (uint64_t)((uint32_t)(st * TILE) >> 4);
#pragma unroll
                    for (int c = 0; c < DK / 16; ++c) {
                        if (c >= ksteps) break;
                        const uint64_t off = (uint64_t)((c >> 2) * kHalf + (c & 3) * 32) >> 4;
                        mma_ss(tm + t * kTile, a + off, b + off, kIdS, c != 0);
                    }
                    mma_commit(&s_full[t]);
                    if (last) mma_commit(&q_empty[kDeal ? 0 : t]);
                }
                __syncwarp();
                issued = true;
            };
            // O_t += P_t V with the V tile in slot st
            auto values = [&](int t, int st, bool first, bool last) {
                if (elect_one()) {
                    const uint64_t b = dv + (uint64_t)((uint32_t)(st * TILE) >> 4);
#pragma unroll
                    for (int c = 0; c < kTile / 16; ++c)  // 16 keys: 8 columns of P, 2 KB of V
                        mma_ts(tm + 2 * kTile + t * kTile, tm + t * kTile + 8 * c, b + (uint64_t)(c * 2048 >> 4), id_o, c != 0 || !first);
                    if (last) mma_commit(&o_full[t]);
                }
                __syncwarp();
            };
            auto release = [&](int st) {
                if (elect_one()) mma_commit(&empty[st]);
                __syncwarp();
            };
            for (int k = 0;; ++k) {
                if (!wait_warp(&w_full[k & 1], (uint32_t)(k >> 1) & 1u)) break;
                const int n0 = __reduce_max_sync(0xffffffffu, work_slots[k & 1].n[0]);
                const int n1 = __reduce_max_sync(0xffffffffu, work_slots[k & 1].n[1]);
                const int end = __reduce_max_sync(0xffffffffu, work_slots[k & 1].end);
                if (lane == 0) mbar_arrive(&w_empty[k & 1]);
                if (end) break;
                const int n_max = max(n0, n1);
                if (n_max == 0) continue;
                if constexpr (kDeal) {
                    const int n = n0 + n1;
                    bool ok = wait_warp(&q_full[0], qn0++ & 1u);
                    for (int i = 0; i < min(n, 2) && ok; ++i) {
                        ok = wait_warp(&full[stage], phase);
                        if (!ok) break;
                        tc_fence_after();
                        scores(i, stage, i + 1 == n);
                        release(stage);
                        advance(stage, phase);
                    }
                    for (int i = 0; i < n && ok; ++i) {
                        const int t = i & 1, sv = stage;  // V_i, then K_i+2: there when p_full is complete
                        advance(stage, phase);
                        ok = wait_warp(&p_full[t], (t ? pn1++ : pn0++) & 1u);
                        if (!ok) break;
                        tc_fence_after();
                        values(t, sv, i < 2, i + 2 >= n);
                        release(sv);
                        if (i + 2 < n) {
                            scores(t, stage, i + 3 == n);
                            release(stage);
                            advance(stage, phase);
                        }
                    }
                    if (!ok) break;
                    continue;
                }
                if (n0 > 0 && !wait_warp(&q_full[0], qn0++ & 1u)) break;
                if (n1 > 0 && !wait_warp(&q_full[1], qn1++ & 1u)) break;
                if (!wait_warp(&full[stage], phase)) break;
                tc_fence_after();
                if (n0 > 0) scores(0, stage, n0 == 1);
                if (n1 > 0) scores(1, stage, n1 == 1);
                release(stage);
                advance(stage, phase);
                bool ok = true;
                for (int j = 0; j < n_max; ++j) {
                    // V_j in slot sv, K_j+1 in slot sk: there when p_full is complete
                    const int sv = stage;
                    advance(stage, phase);
                    const int sk = stage;
                    if (j + 1 < n_max) advance(stage, phase);
                    if (j < n0) {
                        ok = wait_warp(&p_full[0], pn0++ & 1u);
                        if (!ok) break;
                        tc_fence_after();
                        values(0, sv, j == 0, j == n0 - 1);
                        if (j + 1 < n0) scores(0, sk, j + 2 == n0);
                    }
                    if (j < n1) {
                        ok = wait_warp(&p_full[1], pn1++ & 1u);
                        if (!ok) break;
                        tc_fence_after();
                        values(1, sv, j == 0, j == n1 - 1);
                        if (j + 1 < n1) scores(1, sk, j + 2 == n1);
                    }
                    release(sv);
                    if (j + 1 < n_max) release(sk);
                }
                if (!ok) break;
            }
            if (issued) {  // no MMA is in flight when TMEM is released
                if (elect_one()) mma_commit(drain);
                __syncwarp();
                drain_wait(drain, 0);
            }
        } else if (warp == 11 && lane == 0) {
            // ------------------------------------------------------- tile watcher
            // Waits for the tiles in the MMA warp's stead, whose issue queue is shallow: each
            // barrier that it waits for itself delays the MMAs behind it.
            int stage = 0;
            uint32_t phase = 0, pn[2] = {0, 0};
            auto next = [&] {
                if (++stage == STAGES) stage = 0, phase ^= 1;
            };
            bool ok = true;
            for (int k = 0; ok; ++k) {
                if (!wait(&w_full[k & 1], (uint32_t)(k >> 1) & 1u)) break;
                const int n0 = work_slots[k & 1].n[0], n1 = work_slots[k & 1].n[1], end = work_slots[k & 1].end;
                mbar_arrive(&w_empty[k & 1]);
                if (end) break;
                const int n_max = max(n0, n1);
                if constexpr (kDeal) {
                    const int n = n0 + n1;
                    for (int i = 0; i < min(n, 2); ++i) next();  // (the first K tiles: the MMA warp's)
                    for (int i = 0; i < n && ok; ++i) {
                        for (int x = 0; x < (i + 2 < n ? 2 : 1) && ok; ++x) {
                            ok = wait(&full[stage], phase);
                            next();
                        }
                        const int t = i & 1;
                        if (ok && pn[t] > 0) ok = wait(&p_full[t], (pn[t] - 1) & 1u);
                        ++pn[t];
                        if (ok) mbar_arrive(&p_full[t]);
                    }
                    continue;
                }
                if (n_max > 0) next();  // (the first K tile: the MMA warp's)
                for (int j = 0; j < n_max && ok; ++j) {
                    ok = wait(&full[stage], phase);
                    next();
                    if (j + 1 < n_max) {
                        ok = ok && wait(&full[stage], phase);
                        next();
                    }
                    for (int t = 0; t < 2 && ok; ++t) {
                        if (j >= (t ? n1 : n0)) continue;
                        if (pn[t] > 0) ok = wait(&p_full[t], (pn[t] - 1) & 1u);  // one arrival in a phase
                        ++pn[t];
                        if (ok) mbar_arrive(&p_full[t]);
                    }
                }
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 9) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
}

// [T, heads, D] bf16 rows as a 3-D tensor in boxes of 64 columns (128-byte
// swizzled; elements past D and rows past T read as 0) of 128 rows, each token's
// 2^hlog heads beside each other, or, for the output, of 32 columns (64-byte
// swizzled) of 32 rows
bool rows_map(CUtensorMap* map, const Rows& r, int64_t T, int heads, int D, int hlog, bool out = false) {
    EncodeTiled fn = encode_fn();
    if (!fn) return false;
    const cuuint64_t least = (cuuint64_t)(2 * D);
    cuuint64_t dims[3] = {(cuuint64_t)D, (cuuint64_t)heads, (cuuint64_t)T};
    cuuint64_t strides[2] = {heads > 1 ? (cuuint64_t)(2 * r.hs) : least, T > 1 ? (cuuint64_t)(2 * r.ts) : least};
    cuuint32_t box[3] = {out ? 32u : 64u, 1u << hlog, (out ? 32u : (cuuint32_t)kTile) >> hlog}, estr[3] = {1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(r.p), dims, strides, box, estr,
              CU_TENSOR_MAP_INTERLEAVE_NONE, out ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B,
              CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// strides that a tensor map holds: below 2^40 bytes, and not 0 (broadcast rows
// take the CUDA-core kernel)
bool tma_strides(const Rows& r, int64_t T, int heads) {
    const int64_t most = int64_t(1) << 39;
    return (T <= 1 || (r.ts > 0 && r.ts < most)) && (heads <= 1 || (r.hs > 0 && r.hs < most));
}

// the most items of `rows` rows that the lengths can make
int64_t items_of(const AttnProblem& p, int rows, int hlog, int heads) { return (p.T / (rows >> hlog) + p.B) * (int64_t)(p.Hq / heads); }

template <int DK, bool kDeal, bool kPad>
cudaError_t prompt_as(const AttnProblem& p, int hlog, int heads, cudaStream_t stream) {
    constexpr auto kernel = attn_prompt_kernel<DK, kDeal, kPad>;
    static DeviceOnce once;
    if (cudaError_t e = once.run([] {
            return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, Smem<DK>::BYTES);
        });
        e != cudaSuccess)
        return e;
    CUtensorMap q, k, v, o;
    Params pp{p, hlog, heads, tc_wait_limit_ns()};
    if (!rows_map(&q, p.q, p.T, p.Hq, p.D, pp.hlog) || !rows_map(&o, p.out, p.T, p.Hq, p.D, pp.hlog, true) ||
        !rows_map(&k, p.k, p.Tk, p.Hkv, p.D, 0) || !rows_map(&v, p.v, p.Tk, p.Hkv, p.D, 0))
        return cudaErrorInvalidValue;
    const int64_t grid = items_of(p, kDeal ? kTile : 2 * kTile, hlog, heads);
    if (grid > INT32_MAX) return cudaErrorInvalidConfiguration;
    return launch_k(kernel, dim3((unsigned)grid), dim3(kThreads), Smem<DK>::BYTES, stream, q, k, v, o, pp);
}

}  // namespace

// (a negative scale would make a row's smallest product its largest score)
bool attn_prompt_tc_supported(const AttnProblem& p) {
    return p.act_dtype == GBMOE_BF16 && p.D <= 128 && !p.paged && p.Tk > 0 && p.scale_log2 > 0.0f &&
           tma_strides(p.q, p.T, p.Hq) && tma_strides(p.out, p.T, p.Hq) && tma_strides(p.k, p.Tk, p.Hkv) && tma_strides(p.v, p.Tk, p.Hkv);
}

cudaError_t launch_attn_prompt_tc(const AttnProblem& p, cudaStream_t stream) {
    const int G = p.Hq / p.Hkv;
    int hlog = 0;
    while (hlog < 5 && G % (2 << hlog) == 0) ++hlog;
    const int heads = 1 << hlog;
    // The whole group with empty rows, where there are more items than SMs and a prompt of the mean
    // length makes fewer so: 16 prompts of 36 tokens in all, 56 and 8 heads 10 us, one head at a time 32.
    int all = 0;
    while (1 << all < G) ++all;
    auto of_mean = [&](int log, int n) { return (((int64_t)p.T << log) / p.B + 2 * kTile) / (2 * kTile) * (G / n); };
    if (all <= 5 && items_of(p, 2 * kTile, hlog, heads) > sm_count() && of_mean(all, G) < of_mean(hlog, heads))
        return p.D <= 64 ? prompt_as<64, false, true>(p, all, G, stream) : prompt_as<128, false, true>(p, all, G, stream);
    // Too few items for every SM (or, of long prompts, to even out over them). Us without and with: 7596
    // tokens, 4 heads 91 and 62; two prompts of 7344 in all, 8 heads 77 and 65; 476 tokens, 4 heads 13.4
    // and 9.8; 16 prompts of 2242 in all, 7 heads, which the second condition leaves out, 10.8 and 12.8.
    const int64_t items = items_of(p, 2 * kTile, hlog, heads);
    const bool deal = items <= sm_count() || (items <= 2 * sm_count() && p.T >= (int64_t)2 * kTile * p.B);
    if (p.D <= 64) return deal ? prompt_as<64, true, false>(p, hlog, heads, stream) : prompt_as<64, false, false>(p, hlog, heads, stream);
    return deal ? prompt_as<128, true, false>(p, hlog, heads, stream) : prompt_as<128, false, false>(p, hlog, heads, stream);
}

}  // namespace gbmoe
