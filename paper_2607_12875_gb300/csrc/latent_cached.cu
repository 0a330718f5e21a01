// Absorbed latent attention of few query tokens over the paged cache on the tensor
// cores (bf16, R a multiple of 128, P up to 64), the work dealt out in equal shares of
// the key axis (Deal).
//
// A cached row serves every head, as key whole and as value in its first R elements, so
// a tile of 64 rows is loaded once and enters both products from the same place in
// shared memory. The products are transposed: the keys, and then the latent's elements,
// are the rows of the MMA and N query rows (token and head; 16, 32 or 64) its
// columns, because the sums of 128 heads would fill all of TMEM (128 lanes x 512 fp32)
// and leave no place for scores. Per tile of 64 keys:
//   S^T = K Q^T      K-major tiles of 64 elements, M 64: 16 keys in 16 lanes of each warp's quarter
//   P^T = exp2(scale S^T - m)   a thread has two keys and every fourth pair of half of the columns
//   O^T += C^T P^T   the same tiles, read MN-major, M 128; P^T in shared memory, in the place of
//                    the rotary keys, which the second product does not need
// The scores of the next tile are multiplied while the softmax of this one runs, and the
// tile after that is on its way: queries of 64 rows and two tiles fill shared memory.
// The columns' maxima m are shared by all keys of a tile. They come from a segment's first
// tile and are raised, and O^T rescaled, only when a score passes its column's by 2^16:
// fp32 and bf16 weights lose nothing by that (their exponents reach 2^127). The four warps
// of half of the columns tell each other of such a score while the weights are computed, which
// is done once more then. A thread sums its own keys' weights; the threads' sums are joined at
// the end of a segment.
// More rows than N: up to kMostSides CTAs beside each other take the same keys with N rows
// each, at about the same time, so that HBM is read once.
// Warps 0-3 and 4-7: softmax of the first and second half of the columns, queries and
// results; warp 8: TMA; warps 9 and 10: MMA of the scores and of the values.
//
// What bounds it (64 rows, R 512, P 64, a tile of 64 keys): HBM allows a tile on every SM each 3190 cycles; L2 hands an
// SM 27.8 bytes a cycle whatever the copies' pattern (8 TB/s in all), which is 2650 for a tile, and is what two CTAs
// beside each other share HBM's bytes through; both products' operands, the copies and P are 335 KB of shared
// memory's 128 bytes a cycle, 2620; the MMAs 1930. A tile takes 3560 to 3900: its copies are asked for when the values of
// the tile before the last are done and take some 2000 cycles, so a third of the ring is in flight on average.
// 4 sequences of up to 131072 keys, 56 heads: 100 us, 4.1 TB/s; 32 of up to 32768 keys, 128 heads: 280 us, 640 TFLOP/s.
// Few keys: latency, 19.1 us for one sequence of 4000 keys and 128 heads: 11 until the last CTA is done (search for the
// share, queries and first rows, the first tile's softmax, whose code is not yet in the instruction cache, results) and
// 8 of the join (1.5 until it runs and knows the parts, 4 for their sums, 1.5 for the results).
// Steps that led here, us for those two long cases: one MMA warp, tiles of 128 keys, one after the other 146 and 369;
// tiles of 64 keys with the next tile's scores ahead 120 and 339; one copy for two chunks instead of one for each, and an
// MMA warp each for scores and values 114 and 296. Prefetching rows to L2 in the order they lie in took more from
// L2's rate than it gave (112 and 304 against 108 and 293 then); TMA multicast to two CTAs runs at 10 bytes a cycle.
//
// P is rounded to bf16, an error of up to 2^-8 of each weight beside the result's own
// rounding: the MMA takes both operands in one 16-bit type, and the cache is bf16. The
// weights' sum is not rounded.
//
// Masked keys: slots behind a sequence's end may hold anything, so a tile that some row
// does not see whole has its unseen rows set to 0 in shared memory (pages outside the
// pool come as zeros). A key that some rows see and others do not, and that holds what is
// no number, is set to 0 too and makes the weights of the rows that see it NaN.
//
// Waits are bounded as in the GEMM kernels (tc_ptx.cuh).
#include "attn_mma.cuh"
#include "attn_plan.cuh"
#include "latent.h"

namespace gbmoe {
namespace {

using namespace tc;

constexpr int kKeys = 64;                 // keys of a tile
constexpr int kThreads = 352;
constexpr int kChunk = kKeys * 128;       // bytes of 64 rows x 64 elements
constexpr unsigned kFull = 0xffffffffu;
constexpr float kGrow = 16.0f;            // log2 of how far a column's maximum may run ahead of m
constexpr float kMost = 3.402823466e38f;  // -kMost: a maximum of nothing
// Least blocks of 64 keys of a share, and how many a segment's set-up counts for. Us at (1, 0), (2, 1), (3, 1) and (4, 2):
// one sequence of 4000 keys 26.2, 23.4, 24.2, 25.4; 32 of up to 32768, 128 heads 305, 283, 283, 303; short contexts (2 MB
// of rows in all) 27, 27, 46, 46.
constexpr int kMinBlocks = 2, kTileCost = 1;
// Us at 0, 3 and 8: 4 sequences of up to 131072 keys, 56 heads 111.5, 102.6, 102.8 (0: parts are longer than the shares).
constexpr int kSetup = 3;
constexpr int kMostSides = 8;

// N: query rows of a CTA. Rings of pairs of chunks (128 latent elements) and of the rotary chunks.
template <int N>
struct Shape {
    static constexpr int COLS = N / 2;                       // columns of a warp
    static constexpr int G = COLS / 8;                       // groups of eight: a thread has two of each, of two keys
    // (two rotary chunks, whatever the room: a tile's scores then wait for the values of the one before the last, so the
    // pairs of barriers for even and odd tiles are never two phases ahead of who waits for them)
    static constexpr int PAIRS = N == 64 ? 8 : N == 32 ? 10 : 11, TAILS = 2;
    static constexpr int Q = 9 * N * 128;
    static constexpr int BODY = Q + PAIRS * 2 * kChunk + TAILS * kChunk;
    static constexpr int BYTES = 1024 + BODY;
    static_assert(BYTES + 4096 <= 227 * 1024 && 6 * N <= 512, "shared and tensor memory");
};

template <int C>
__device__ __forceinline__ void tmem_load(uint32_t taddr, uint32_t (&r)[C]) {
    if constexpr (C == 32) {
        tmem_ld32_async(taddr, r);
        ld_wait();
        pin32(r);
    } else if constexpr (C == 16) {
        float v[16];
        tmem_ld16(taddr, v);
#pragma unroll
        for (int i = 0; i < 16; ++i) r[i] = __float_as_uint(v[i]);
    } else {
        static_assert(C == 8, "columns");
        asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                     : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                     : "r"(taddr));
        asm volatile("tcgen05.wait::ld.sync.aligned;"
                     : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7])
                     :
                     : "memory");
    }
}
// C columns of 16 lanes: this thread's u[4 g ..] are columns 8 g + 2 (lane % 4) + {0, 1} of row lane / 4, then of row
// lane / 4 + 8.
template <int C>
__device__ __forceinline__ void tmem_load16(uint32_t taddr, uint32_t (&r)[C / 2]) {
    if constexpr (C == 32) {
        asm volatile(
            "tcgen05.ld.sync.aligned.16x256b.x4.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
            : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
              "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
            : "r"(taddr));
    } else if constexpr (C == 16) {
        asm volatile("tcgen05.ld.sync.aligned.16x256b.x2.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                     : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                     : "r"(taddr));
    } else {
        static_assert(C == 8, "columns");
        asm volatile("tcgen05.ld.sync.aligned.16x256b.x1.b32 {%0, %1, %2, %3}, [%4];"
                     : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                     : "r"(taddr));
    }
}
template <int n>
__device__ __forceinline__ void pin(uint32_t (&r)[n]) {  // no use moves above the wait before
#pragma unroll
    for (int i = 0; i < n; ++i) asm volatile("" : "+r"(r[i]));
}

template <int C>
__device__ __forceinline__ void tmem_store(uint32_t taddr, const uint32_t (&r)[C]) {
    if constexpr (C == 32) {
        tmem_st32(taddr, r);
    } else if constexpr (C == 16) {
        asm volatile(
            "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, "
            "%15};" ::"r"(r[0]),
            "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
            "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(taddr)
            : "memory");
    } else {
        static_assert(C == 8, "columns");
        asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};" ::"r"(r[0]), "r"(r[1]),
                     "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(taddr)
                     : "memory");
    }
}

// Tiles that lie as [key][64 elements], 128-byte swizzled, read with the MMA's rows or
// columns along the elements: groups of 64 elements kChunk apart (leading offset),
// groups of 8 keys 1024 bytes apart (stride offset).
__device__ __forceinline__ uint64_t mn_desc(uint32_t saddr) {
    return (uint64_t)((saddr & 0x3FFFFu) >> 4) | (uint64_t)(kChunk >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 |
           (uint64_t)2 << 61;
}

// A segment as one CTA sees it: its rows and its tiles of keys. The TMA warp walks the
// share and hands the segments to the other warps.
struct Job {
    int row0, rows;       // first row of the sequence's, how many (<= 0: none)
    int key0, tiles;
    int all_hi, most_hi;  // last key that all rows see, that any row sees
    int q0, pos0;         // the sequence's first token, its position
    int len, key_end;     // the sequence's keys; end of the segment's
    int b;
    int end;              // 1: no more segments
    int64_t slot;
};
template <int N>
__device__ __forceinline__ Job job_of(const AttnProblem& p, const Segment& g, int side) {
    Job x;
    const int64_t row0 = (int64_t)g.tile * p.tile_rows + side * N;
    x.row0 = (int)row0;
    x.rows = (int)min64(N, (int64_t)g.s.nq * p.R - row0);
    x.key0 = g.blk0 * kKeys;
    x.tiles = 0, x.all_hi = x.most_hi = -1;
    x.q0 = g.s.q0, x.pos0 = g.s.len - g.s.nq, x.len = g.s.len, x.b = g.b, x.end = 0, x.slot = g.slot;
    x.key_end = (int)min64((int64_t)g.blk1 * kKeys, g.s.len);
    if (x.rows <= 0) return x;
    int lo;
    seen_keys(p, g.s, x.row0 / p.R, lo, x.all_hi);
    seen_keys(p, g.s, (x.row0 + x.rows - 1) / p.R, lo, x.most_hi);
    const int end = (int)min64((int64_t)g.blk1 * kKeys, (int64_t)x.most_hi + 1);
    x.tiles = end > x.key0 ? (end - x.key0 + kKeys - 1) / kKeys : 0;
    return x;
}

// A share of the key axis that is part of one tile, where every tile can be cut into equal parts that are hardly longer
// than the shares of Walk (kSetup blocks at most): a share with the end of one tile and the beginning of the next sets up
// and finishes twice, which takes as long as several blocks (17 sequences of up to 3000 keys: 23 us for such a CTA, 15
// for the others; with parts 34.3 to 30.3 us, 4 long ones 110 to 100). Else the shares of Walk. Up to 32 sequences, a lane for each.
struct Deal : Walk<0, kKeys> {
    static constexpr int kAlone = 32;  // sequences that a warp looks through by itself
    int per = 0;  // parts of this share's tile (0: a share of Walk)

    // (Out of line: what the loops' code shares the instruction cache with counts. 32 sequences of up to 32768 keys, 128
    // heads: 290 us inline, 280 so.)
    __device__ __noinline__ bool begin_together(const AttnProblem& p, int64_t index, int64_t* sm) { return Walk::begin(p, index, sm); }
    __device__ __forceinline__ bool begin(const AttnProblem& p, int64_t index, int64_t* sm) {
        per = 0;
        if (p.B > kAlone) return begin_together(p, index, sm);
        const int lane = threadIdx.x & 31;
        Seq s{};
        if (lane < p.B) s = load_seq(p, lane);
        const int64_t tiles_here = lane < p.B ? tiles_of(p, s) : 0;
        const int nb = key_blocks<kKeys>(s);
        const int64_t v = tiles_here * (nb + p.tile_cost), pre = warp_scan(v);
        sh.set(p, __shfl_sync(kFull, pre, 31));
        const uint32_t all = __reduce_add_sync(kFull, (uint32_t)tiles_here);  // (T heads is 2^30 at most)
        const int shares = p.shares;
        auto parts_of = [&](int blocks) { return (uint32_t)tiles_here * (uint32_t)max(1, (nb + blocks - 1) / blocks); };
        if (all <= (uint32_t)shares) {
            // (the shares hold all blocks, so the sums of parts are small)
            int lo = p.min_blocks, hi = (int)sh.each + kSetup;
            if (__reduce_add_sync(kFull, parts_of(hi)) <= (uint32_t)shares) {
                lo = max(lo, (int)sh.each - p.tile_cost - 1);
                while (lo < hi) {
                    const int mid = (lo + hi) >> 1;
                    if (__reduce_add_sync(kFull, parts_of(mid)) <= (uint32_t)shares) hi = mid;
                    else lo = mid + 1;
                }
                const uint32_t mine = parts_of(hi);
                const int end = (int)warp_scan(mine), i = (int)index;
                const uint32_t hit = __ballot_sync(kFull, i < end);
                if (!hit) return false;
                const int b = __ffs(hit) - 1, at = i - __shfl_sync(kFull, end - (int)mine, b);
                enter(p, b);
                share = index;
                per = max(1, (g.nb + hi - 1) / hi);
                const int part = at % per, each = (g.nb + per - 1) / per;
                g.head = 0, g.tile = at / per;
                g.blk0 = part * each, g.blk1 = min(g.blk0 + each, g.nb);
                g.slot = per == 1 ? -1 : 2 * share;
                return true;
            }
        }
        const int64_t want = index * sh.each;
        const uint32_t hit = __ballot_sync(kFull, want < pre);
        if (!hit) return false;
        const int b = __ffs(hit) - 1;
        start(p, index, Place{b, want - __shfl_sync(kFull, pre - v, b)});
        return true;
    }
    __device__ __forceinline__ bool next(const AttnProblem& p) { return per == 0 && Walk::next(p); }
    __device__ __forceinline__ void note(const AttnProblem& p) const {
        if (per == 0) Walk::note(p);
        else note_parts(p, per);
    }
};

struct Params {
    LatentProblem l;
    int sides;
    uint64_t wait_limit_ns;
};

template <int N>
__global__ void __launch_bounds__(kThreads, 1)
latent_cached_kernel(const __grid_constant__ CUtensorMap latents, const __grid_constant__ CUtensorMap pool, const __grid_constant__ Params pp) {
    using L = Shape<N>;
    constexpr int COLS = L::COLS, G = L::G, PAIRS = L::PAIRS, TAILS = L::TAILS;
    const AttnProblem& p = pp.l.a;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* sq = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    uint8_t* pairs = sq + L::Q;
    uint8_t* tails = pairs + PAIRS * 2 * kChunk;
    constexpr int kBars = 2 * (PAIRS + TAILS) + 16;
    __shared__ uint64_t bars[kBars];
    __shared__ Job jobs[2], first_job;
    uint64_t* full = bars;              // a pair landed
    uint64_t* empty = full + PAIRS;     // the products that read it finished
    uint64_t* tfull = empty + PAIRS;
    uint64_t* tempty = tfull + TAILS;
    uint64_t* q_full = tempty + TAILS;  // the queries are in shared memory
    uint64_t* s_full = q_full + 1;      // scores of even and odd tiles
    uint64_t* p_full = s_full + 2;      // P is written, O rescaled, unseen rows are 0
    uint64_t* o_full = p_full + 2;      // O holds this tile too (even and odd ones: a parity tells one phase from the one before)
    uint64_t* drain = o_full + 2;
    uint64_t* half = drain + 2;         // the four warps of half of the columns meet
    uint64_t* both = half + 2;          // all eight
    uint64_t* j_full = both + 1;        // a job is in its slot
    uint64_t* j_empty = j_full + 2;     // every role has read it
    __shared__ uint32_t tmem_slot, good[TAILS];  // good: pages of the tile that are in the pool
    __shared__ int abort_word, row_hi[N];
    __shared__ uint32_t raised[2];      // tile number (from 1 on) in which a score far above its maximum was found
    // The same for a key that holds what is no number. The warps of one half of the columns may mark keys of the next tile
    // before those of the other half have read this one's marks, but never the same word: keys that some rows see and others
    // do not lie within N - 1 in a row, and the next segment begins when all warps' weights of this one are written.
    static_assert(N <= kKeys, "no two tiles of a segment mark the same word");
    __shared__ uint32_t poisoned[kKeys];
    __shared__ __align__(8) float sums[8][COLS];
    __shared__ __align__(16) float low[N], factor[N];  // the columns' -m, and what a raise multiplies by
    __shared__ int64_t plan[plan_words(kThreads)];
    volatile int* abort_flag = &abort_word;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int R = p.D, pairs_of_tile = R / 128, W = pp.l.K;
    const int box_log2 = min(p.page_log2, 6), per_tile = kKeys >> box_log2;  // rows of a copy, copies of a chunk
    const int share = blockIdx.x / pp.sides, side = blockIdx.x - share * pp.sides;
    // (each barrier by a thread of its own: one thread for all took over a microsecond)
    if (tid < kBars) {
        uint64_t* bar = bars + tid;
        uint32_t count = 1;
        if (bar == q_full || bar == both || (bar >= p_full && bar < p_full + 2)) count = 8;  // (softmax warps)
        if (bar >= half && bar < half + 2) count = 4;
        if (bar >= j_empty && bar < j_empty + 2) count = 10;  // (softmax warps, MMA warps)
        mbar_init(bar, count);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (tid >= 64 && tid < 64 + kKeys) poisoned[tid - 64] = 0;
    if (tid == 128) abort_word = 0, raised[0] = raised[1] = 0;
    if (warp == 9) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&tmem_slot)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    // (up to here nothing in memory is read: barriers and TMEM are set up while the kernel before still runs)
    pdl_enter();
    tc_fence_before();
    Deal walk;
    if (warp == 8 || p.B > Deal::kAlone) {
        const bool some = __any_sync(kFull, walk.begin(p, share, plan));
        Job x{};
        if (some) x = job_of<N>(p, walk.g, side);
        x.end = !some;
        if (warp == 8 && lane == 0) first_job = x;
    }
    __syncthreads();
    const bool any = !first_job.end;
    tc_fence_after();
    const uint32_t tmem = tmem_slot, tS = tmem, tO = tmem + 2 * N;  // S: even and odd tiles; O: pairs_of_tile times N columns
    auto wait_warp = [&](uint64_t* bar, uint32_t parity) { return warp_wait(bar, parity, abort_flag, p.err, pp.wait_limit_ns); };

    if (!any) {
        if (tid == 0 && side == 0) Deal::note_idle(p, share);
    } else if (warp < 8) {
        // ------------------------------------------------------------ softmax
        const int wg = warp >> 2, r = (warp & 3) * 32 + lane, c0 = wg * COLS, wt = tid & 127;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t mS = tS + lanes + c0, mO = tO + lanes + c0;
        const int key_a = (warp & 3) * 16 + (lane >> 2), col = c0 + 2 * (lane & 3);  // keys key_a, key_a + 8; columns col + 8 g + {0, 1}
        const float scale = p.scale_log2;
        uint32_t n_tiles = 0;  // so far
        int tail = 0, pair = 0;
        uint32_t tphase = 0;
        uint32_t meets = 0, meets_both = 0;
        // (mbarriers, not bar.sync: a warp whose wait gave up does not come)
        auto meet = [&](uint64_t* bar, uint32_t& n) {
            __syncwarp();
            if (lane == 0) mbar_arrive(bar);
            return wait_warp(bar, n++ & 1u);
        };
        auto values_of = [&](uint32_t n) { return wait_warp(&o_full[n & 1u], n >> 1 & 1u); };
        bool ok = true;
        auto take = [&](int j) {
            ok = wait_warp(&j_full[j & 1], (uint32_t)(j >> 1) & 1u);
            const Job x = jobs[j & 1];
            __syncwarp();
            if (lane == 0) mbar_arrive(&j_empty[j & 1]);
            return x;
        };
        // a segment's queries on their way: rows of 64 elements, 128-byte swizzled, zeros where there are none
        auto fetch_queries = [&](const Job& x) {
            if (x.end || x.tiles <= 0) return;
            constexpr int kOf = 256 / N;  // threads of a row
            const int row = tid / kOf, rr = x.row0 + (row < x.rows ? row : 0), tok = rr / p.R;
            const __nv_bfloat16* src = static_cast<const __nv_bfloat16*>(p.q.p) + (int64_t)(x.q0 + tok) * p.q.ts + (rr - tok * p.R) * p.q.hs;
            const uint32_t dst = smem_u32(sq) + row * 128;
#pragma unroll 9
            for (int c = tid % kOf; c < pairs_of_tile * 16 + 8; c += kOf) {
                const bool there = row < x.rows && 8 * c < W;
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst + (c >> 3) * (N * 128) + ((c ^ row) & 7) * 16),
                             "l"(src + (there ? 8 * c : 0)), "r"(there ? 16 : 0)
                             : "memory");
            }
        };
        Job next = first_job;
        fetch_queries(next);
        for (int j = 0; ok; ++j) {
            const Job x = next;
            if (x.end) break;
            if (x.rows > 0) {
                if (x.tiles > 0) {
                    asm volatile("cp.async.wait_all;" ::: "memory");
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                    if (lane == 0) mbar_arrive(q_full);
                }
                if (wt < COLS) {
                    low[c0 + wt] = kMost;
                    int hi = -1;
                    if (c0 + wt < x.rows) hi = p.causal ? min(x.pos0 + (x.row0 + c0 + wt) / p.R, x.len - 1) : x.len - 1;
                    row_hi[c0 + wt] = hi < 0 ? -1 : hi;
                }
                ok = meet(&half[wg], meets);
                if (!ok) break;
            }
            uint64_t l[G];  // sums of the weights of this thread's keys
#pragma unroll
            for (int c = 0; c < G; ++c) l[c] = pack2(0.0f, 0.0f);
            for (int t = 0; t < x.tiles && ok; ++t) {
                ok = wait_warp(&s_full[n_tiles & 1u], (n_tiles >> 1) & 1u) && wait_warp(&tfull[tail], tphase);
                if (!ok) break;
                tc_fence_after();
                uint32_t u[2 * G * 2];
                const uint32_t mine_s = mS + (n_tiles & 1u) * N;
                tmem_load16<COLS>(mine_s, u);
                ld_wait();
                pin(u);
                const int key0 = x.key0 + t * kKeys;
                const uint32_t pages = *const_cast<volatile uint32_t*>(&good[tail]);
                const bool all = key0 + kKeys - 1 <= x.all_hi && pages == (1u << per_tile) - 1u;
                bool there[2] = {true, true}, poison[2] = {false, false};  // of the two keys
                if (!all) {
#pragma unroll
                    for (int z = 0; z < 2; ++z) there[z] = pages >> ((key_a + 8 * z) >> box_log2) & 1u;
                    // four threads for a key: what is no number where some rows see it and others do not, rows that none sees
                    const int k = tid >> 2, key = key0 + k;
                    auto at = [&](int i) {  // piece i of its latent
                        int slot = pair + (i >> 4);
                        if (slot >= PAIRS) slot -= PAIRS;
                        return reinterpret_cast<uint4*>(pairs + slot * 2 * kChunk + (i >> 3 & 1) * kChunk + sw128_off(k, i & 7));
                    };
                    if (key > x.all_hi && key <= x.most_hi) {
                        bool bad = false;
                        for (int i = tid & 3; i < R / 8; i += 4) {
                            const uint4 v = *at(i);
                            bad = bad || (__vcmpgeu2(v.x & 0x7fff7fffu, 0x7f807f80u) | __vcmpgeu2(v.y & 0x7fff7fffu, 0x7f807f80u) |
                                          __vcmpgeu2(v.z & 0x7fff7fffu, 0x7f807f80u) | __vcmpgeu2(v.w & 0x7fff7fffu, 0x7f807f80u)) != 0;
                        }
                        if (bad) *const_cast<volatile uint32_t*>(&poisoned[k]) = n_tiles + 1;
                    }
                    ok = meet(both, meets_both);
                    if (!ok) break;
                    if (key > x.most_hi || *const_cast<volatile uint32_t*>(&poisoned[k]) == n_tiles + 1)
                        for (int i = tid & 3; i < R / 8; i += 4) *at(i) = make_uint4(0, 0, 0, 0);
#pragma unroll
                    for (int z = 0; z < 2; ++z) poison[z] = *const_cast<volatile uint32_t*>(&poisoned[key_a + 8 * z]) == n_tiles + 1;
                }
                auto unseen = [&](int c, int z) { return !there[z] || key0 + key_a + 8 * z > row_hi[c]; };
                uint8_t* dst = tails + tail * kChunk;
                // The maxima are brought up to this tile's scores, the sums so far to the maxima.
                auto raise = [&] {
#pragma unroll
                    for (int g = 0; g < G; ++g)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            float best = -kMost;
#pragma unroll
                            for (int z = 0; z < 2; ++z)
                                if (all || !unseen(col + 8 * g + e, z)) best = fmaxf(best, __uint_as_float(u[4 * g + 2 * z + e]) * scale);
#pragma unroll
                            for (int d = 4; d < 32; d <<= 1) best = fmaxf(best, __shfl_xor_sync(kFull, best, d));
                            if (lane < 4) sums[warp][8 * g + 2 * lane + e] = best;
                        }
                    ok = meet(&half[wg], meets);
                    if (!ok) return;
                    if (wt < COLS) {
                        float m = -low[c0 + wt];
#pragma unroll
                        for (int w = 0; w < 4; ++w) m = fmaxf(m, sums[4 * wg + w][wt]);
                        factor[c0 + wt] = ex2(-low[c0 + wt] - m);  // (nothing yet: 0)
                        low[c0 + wt] = -m;
                    }
                    ok = meet(&half[wg], meets);
                    if (!ok || t == 0) return;
                    ok = values_of(n_tiles - 1);
                    if (!ok) return;
                    tc_fence_after();
#pragma unroll
                    for (int g = 0; g < G; ++g) {
                        const float2 f = *reinterpret_cast<const float2*>(&factor[col + 8 * g]);
                        l[g] = fma2(l[g], pack2(f.x, f.y), pack2(0.0f, 0.0f));
                    }
#pragma unroll 1
                    for (int i = 0; i < pairs_of_tile; ++i) {
                        uint32_t o[COLS];
                        tmem_load<COLS>(mO + i * N, o);
#pragma unroll
                        for (int c = 0; c < COLS; ++c) o[c] = __float_as_uint(__uint_as_float(o[c]) * factor[c0 + c]);
                        tmem_store<COLS>(mO + i * N, o);
                    }
                    st_wait();
                };
                // Scores relative to the maxima, base 2, and the largest of them.
                float r2[4 * G];
                auto relative = [&] {
                    const uint64_t sc2 = pack2(scale, scale);
                    float most = -kMost;
#pragma unroll
                    for (int g = 0; g < G; ++g) {
                        const float2 m = *reinterpret_cast<const float2*>(&low[col + 8 * g]);
#pragma unroll
                        for (int z = 0; z < 2; ++z) {
                            const float2 a = unpack2(fma2(pack2(__uint_as_float(u[4 * g + 2 * z]), __uint_as_float(u[4 * g + 2 * z + 1])), sc2, pack2(m.x, m.y)));
                            r2[4 * g + 2 * z] = a.x, r2[4 * g + 2 * z + 1] = a.y;
                        }
                    }
                    if (!all) {
#pragma unroll
                        for (int i = 0; i < 4 * G; ++i)
                            if (unseen(col + 8 * (i >> 2) + (i & 1), i >> 1 & 1)) r2[i] = neg_inf();
                    }
#pragma unroll
                    for (int i = 0; i < 4 * G; i += 2) most = max3(most, r2[i], r2[i + 1]);
                    return most;
                };
                auto weights = [&](bool count) {
                    if (poison[0] || poison[1]) {  // (a NaN's weight is a NaN)
#pragma unroll
                        for (int i = 0; i < 4 * G; ++i)
                            if (poison[i >> 1 & 1] && !unseen(col + 8 * (i >> 2) + (i & 1), i >> 1 & 1)) r2[i] = __uint_as_float(0x7fc00000u);
                    }
#pragma unroll
                    for (int g = 0; g < G; ++g)
#pragma unroll
                        for (int z = 0; z < 2; ++z) {
                            const float e0 = ex2(r2[4 * g + 2 * z]), e1 = ex2(r2[4 * g + 2 * z + 1]);
                            if (count) l[g] = add2(l[g], pack2(e0, e1));
                            *reinterpret_cast<uint32_t*>(dst + sw128_off(key_a + 8 * z, (c0 >> 3) + g) + 4 * (lane & 3)) = pack_bf16x2(e0, e1);
                        }
                };
                // (a loop of one or two turns: each step's code is there once, the first tile's has not to be fetched for it alone)
                bool up = t == 0, count = true;
                for (;;) {
                    if (up) raise();
                    if (!ok) break;
                    const bool over = __any_sync(kFull, relative() > kGrow) && !up;
                    if (!up && lane == 0) {
                        if (over) *const_cast<volatile uint32_t*>(&raised[wg]) = n_tiles + 1;
                        mbar_arrive(&half[wg]);
                    }
                    if (!over) weights(count);
                    if (up) break;
                    ok = wait_warp(&half[wg], meets++ & 1u);
                    if (!ok || *const_cast<volatile uint32_t*>(&raised[wg]) != n_tiles + 1) break;
                    up = true, count = over;  // (the others have counted theirs, which the raise rescales)
                }
                if (!ok) break;
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&p_full[n_tiles & 1u]);
                ++n_tiles;
                pair += pairs_of_tile;
                while (pair >= PAIRS) pair -= PAIRS;
                if (++tail == TAILS) tail = 0, tphase ^= 1;
            }
            if (!ok) break;
            // the next segment's queries come while this one's results go (every product with these is done)
            next = take(j);
            if (!ok) break;
            fetch_queries(next);
            // ------------------------------------------------------------ result
            if (x.rows > 0) {
                // each column's sum of weights over the keys
#pragma unroll
                for (int g = 0; g < G; ++g) {
                    float2 v = unpack2(l[g]);
#pragma unroll
                    for (int d = 4; d < 32; d <<= 1) v.x += __shfl_xor_sync(kFull, v.x, d), v.y += __shfl_xor_sync(kFull, v.y, d);
                    if (lane < 4) *reinterpret_cast<float2*>(&sums[warp][8 * g + 2 * lane]) = v;
                }
                if (x.tiles > 0) {
                    ok = values_of(n_tiles - 1);
                    if (!ok) break;
                }
                tc_fence_after();
                ok = meet(&half[wg], meets);
                if (!ok) break;
                if (wt < COLS && c0 + wt < x.rows) {
                    const int c = c0 + wt, row = x.row0 + c;
                    float sum = 0.0f;
#pragma unroll
                    for (int w = 0; w < 4; ++w) sum += sums[4 * wg + w][wt];
                    const float mx = low[c] == kMost ? neg_inf() : -low[c];
                    // Without a score above -inf: whether the row sees a key at all (if not it gives 0, else 0 / 0)
                    const bool blank = mx == neg_inf() && sum == 0.0f;
                    const bool sees = !blank || any_page(p, x.b, x.key0, min(row_hi[c], x.key_end - 1));
                    const bool none = row_hi[c] < 0 || !sees;
                    factor[c] = none ? 0.0f : 1.0f / sum;
                    if (x.slot >= 0)
                        reinterpret_cast<float4*>(p.part_s)[x.slot * p.tile_rows + side * N + c] = make_float4(mx, sum, mx, sees ? 1.0f : 0.0f);
                    else if (p.lse)
                        p.lse[(int64_t)x.q0 * p.Hq + row] = none ? neg_inf() : (mx + log2f(sum)) * kLn2;
                }
                ok = meet(&half[wg], meets);
                if (!ok) break;
                for (int i = 0; i < pairs_of_tile; ++i) {
                    const int d = i * 128 + r;
                    uint32_t u[COLS];
                    if (x.tiles > 0) {
                        tmem_load<COLS>(mO + i * N, u);
                    } else {
#pragma unroll
                        for (int c = 0; c < COLS; ++c) u[c] = 0;
                    }
                    if (x.slot >= 0) {
                        float* dst = p.part_o + (x.slot * p.tile_rows + side * N + c0) * R + d;
#pragma unroll
                        for (int c = 0; c < COLS; ++c)
                            if (c0 + c < x.rows) dst[(int64_t)c * R] = __uint_as_float(u[c]);
                    } else {
#pragma unroll
                        for (int c = 0; c < COLS; ++c) {
                            if (c0 + c >= x.rows) break;
                            const int row = x.row0 + c0 + c, tok = row / p.R;
                            __nv_bfloat16* out = const_cast<__nv_bfloat16*>(static_cast<const __nv_bfloat16*>(p.out.p)) +
                                                 (int64_t)(x.q0 + tok) * p.out.ts + (row - tok * p.R) * p.out.hs + d;
                            const float f = factor[c0 + c];
                            *out = __float2bfloat16_rn(f == 0.0f ? 0.0f : __uint_as_float(u[c]) * f);
                        }
                    }
                }
                tc_fence_before();
                // (the next segment's maxima and factors are written after this one's are read)
                ok = meet(&half[wg], meets);
                if (!ok) break;
            }
        }
        asm volatile("cp.async.wait_all;" ::: "memory");  // (a wait gave up: queries may be on their way)
    } else if (warp == 8) {
        // ------------------------------------------------------------ TMA producer
        uint32_t inflight = 0, par = 0, tinflight = 0, tpar = 0;
        int slot = 0, tail = 0;
        uint32_t phase = 0, tphase = 0;
        const int box = 128 << box_log2;
        const int nowhere = p.n_pages << p.page_log2;  // rows past the pool: the copy brings zeros
        bool ok = true, more = true;
        auto on_its_way = [&] {
            inflight |= 1u << slot;
            par = (par & ~(1u << slot)) | (phase << slot);
            if (++slot == PAIRS) slot = 0, phase ^= 1;
        };
        for (int j = 0; ok; ++j) {
            Job x = first_job;
            if (j > 0) {  // (which every thread has)
                ok = wait_warp(&j_empty[(j - 1) & 1], ((uint32_t)((j - 1) >> 1) & 1u) ^ 1u);
                if (!ok) break;
                if (more) x = job_of<N>(p, walk.g, side);
                else x.end = 1;
                if (lane == 0) {
                    jobs[(j - 1) & 1] = x;
                    mbar_arrive(&j_full[(j - 1) & 1]);
                }
            }
            if (lane == 0 && more && side == 0) walk.note(p);
            __syncwarp();
            if (!more) break;
            const int32_t* ids = p.page_table + (int64_t)x.b * p.max_pages;
            auto first_row = [&](int t) {  // of this lane's page of tile t
                const int at = x.key0 + t * kKeys + (lane << box_log2);
                if (lane >= per_tile || t >= x.tiles || at > x.most_hi) return nowhere;
                const int id = ids[at >> p.page_log2];
                return id >= 0 && id < p.n_pages ? (id << p.page_log2) + (at & (p.page - 1)) : nowhere;
            };
            int row = first_row(0);
            for (int t = 0; t < x.tiles && ok; ++t) {
                const int ahead = first_row(t + 1);
                const uint32_t mask = __ballot_sync(kFull, row != nowhere);
                int from[4];
#pragma unroll
                for (int c = 0; c < 4; ++c) from[c] = __shfl_sync(kFull, row, c & (per_tile - 1));
                // (by one lane from here on, and in as few copies as there can be: with a warp's meetings around each of
                // them a pair took 590 cycles, which set the pace)
                if (per_tile == 4) {  // (pages of 16: eight copies of a pair, a lane for each)
                    for (int i = 0; i < pairs_of_tile && ok; ++i) {
                        ok = wait_warp(&empty[slot], phase ^ 1);
                        if (!ok) break;
                        if (lane == 0) mbar_expect_tx(&full[slot], 2 * kChunk);
                        __syncwarp();
                        const int mine = __shfl_sync(kFull, row, lane & 3);
                        if (lane < 8)
                            tma_load_3d(pairs + (2 * slot + (lane >> 2)) * kChunk + (lane & 3) * box, &latents, 0, mine, 2 * i + (lane >> 2), &full[slot]);
                        on_its_way();
                    }
                } else if (lane == 0) {
                    for (int i = 0; i < pairs_of_tile; ++i) {
                        ok = mbar_wait(&empty[slot], phase ^ 1, abort_flag, p.err, pp.wait_limit_ns);
                        if (!ok) break;
                        uint8_t* dst = pairs + slot * 2 * kChunk;
                        mbar_expect_tx(&full[slot], 2 * kChunk);
                        if (per_tile == 1) {
                            tma_load_3d(dst, &latents, 0, from[0], 2 * i, &full[slot]);
                        } else {
#pragma unroll
                            for (int c = 0; c < 2; ++c) {
                                tma_load_3d(dst + c * box, &latents, 0, from[c], 2 * i, &full[slot]);
                                tma_load_3d(dst + kChunk + c * box, &latents, 0, from[c], 2 * i + 1, &full[slot]);
                            }
                        }
                        on_its_way();
                    }
                }
                if (lane == 0) {
                    if (ok) ok = mbar_wait(&tempty[tail], tphase ^ 1, abort_flag, p.err, pp.wait_limit_ns);
                    if (ok) {
                        *const_cast<volatile uint32_t*>(&good[tail]) = mask;
                        mbar_expect_tx(&tfull[tail], W > R ? kChunk : 0);
                        if (W > R) {
#pragma unroll
                            for (int c = 0; c < 4; ++c)
                                if (c < per_tile) tma_load_2d(tails + tail * kChunk + c * box, &pool, R, from[c], &tfull[tail]);
                        }
                        tinflight |= 1u << tail;
                        tpar = (tpar & ~(1u << tail)) | (tphase << tail);
                        if (++tail == TAILS) tail = 0, tphase ^= 1;
                    }
                }
                ok = __shfl_sync(kFull, ok, 0);
                row = ahead;
            }
            more = walk.next(p);
        }
        // every copy has landed before the CTA leaves
        if (lane == 0) {
            const uint64_t t0 = global_ns();
            for (int i = 0; i < PAIRS; ++i)
                if ((inflight >> i) & 1u) drain_wait(&full[i], (par >> i) & 1u, t0);
            for (int i = 0; i < TAILS; ++i)
                if ((tinflight >> i) & 1u) drain_wait(&tfull[i], (tpar >> i) & 1u, t0);
        }
    } else {
        // ------------------------- MMA issuers (two whole warps, one lane of each issues): scores, and values
        // What a warp's wait or commit takes between two of its MMAs its own MMAs stand still (some 100 and 50 cycles); two
        // warps fill each other's gaps, and the values of a tile wait for no loads of the one after the next.
        // (What the loops run to comes from warp-wide reductions, so that the MMA's operands stay in uniform registers.)
        const int values = __reduce_max_sync(kFull, warp == 10);
        constexpr uint32_t kId = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(N >> 3) << 17);
        constexpr uint32_t kIdS = kId | 64u >> 4 << 24, kIdO = kId | 128u >> 4 << 24 | 1u << 15 | 1u << 16;  // O: both operands MN-major
        const uint32_t tm = __reduce_max_sync(kFull, tmem);
        const uint64_t dq = sw128_desc(smem_u32(sq)), dk = sw128_desc(smem_u32(pairs)), dt = sw128_desc(smem_u32(tails));
        const uint64_t dv = mn_desc(smem_u32(pairs)), dp = mn_desc(smem_u32(tails));
        const int tail_steps = (W - R + 15) / 16;
        int slot = 0, tail = 0;
        uint32_t phase = 0, tphase = 0, qn = 0, tile = 0;
        bool ok = true, issued = false;
        auto weights_of = [&](uint32_t n) { return wait_warp(&p_full[n & 1u], n >> 1 & 1u); };
        for (int j = 0; ok; ++j) {
            int tiles = __reduce_max_sync(kFull, first_job.tiles);
            if (j > 0) {
                ok = wait_warp(&j_full[(j - 1) & 1], (uint32_t)((j - 1) >> 1) & 1u);
                if (!ok) break;
                tiles = __reduce_max_sync(kFull, jobs[(j - 1) & 1].tiles);
                const int end = __reduce_max_sync(kFull, jobs[(j - 1) & 1].end);
                __syncwarp();
                if (lane == 0) mbar_arrive(&j_empty[(j - 1) & 1]);
                if (end) break;
            }
            if (tiles <= 0) continue;
            if (!values) ok = wait_warp(q_full, qn++ & 1u);
            for (int t = 0; t < tiles && ok; ++t, ++tile) {
                if (values) {
                    ok = weights_of(tile);
                    if (!ok) break;
                    tc_fence_after();
                    issued = true;
                    for (int i = 0; i < pairs_of_tile; ++i) {
                        if (elect_one()) {
                            const uint64_t a = dv + (uint64_t)((uint32_t)(slot * 2 * kChunk) >> 4), b = dp + (uint64_t)((uint32_t)(tail * kChunk) >> 4);
#pragma unroll
                            for (int k = 0; k < kKeys / 16; ++k)
                                mma_ss(tm + 2 * N + i * N, a + (uint64_t)(k * 2048 >> 4), b + (uint64_t)(k * 2048 >> 4), kIdO, t > 0 || k > 0);
                            mma_commit(&empty[slot]);
                        }
                        __syncwarp();
                        if (++slot == PAIRS) slot = 0;
                    }
                    if (elect_one()) {
                        mma_commit(&tempty[tail]);
                        mma_commit(&o_full[tile & 1u]);
                    }
                } else {
                    if (tile >= 2) ok = weights_of(tile - 2);  // the scores that lay there have been read
                    const uint32_t d = tm + (tile & 1u) * N;
                    for (int i = 0; i < pairs_of_tile && ok; ++i) {
                        ok = wait_warp(&full[slot], phase);
                        if (!ok) break;
                        tc_fence_after();
                        issued = true;
                        if (elect_one()) {
                            const uint64_t a = dk + (uint64_t)((uint32_t)(slot * 2 * kChunk) >> 4), b = dq + (uint64_t)((uint32_t)(i * 2 * N * 128) >> 4);
#pragma unroll
                            for (int k = 0; k < 8; ++k)
                                mma_ss(d, a + (((k >> 2) * kChunk + (k & 3) * 32) >> 4), b + (((k >> 2) * N * 128 + (k & 3) * 32) >> 4), kIdS,
                                       i > 0 || k > 0);
                        }
                        __syncwarp();
                        if (++slot == PAIRS) slot = 0, phase ^= 1;
                    }
                    ok = ok && wait_warp(&tfull[tail], tphase);
                    if (!ok) break;
                    tc_fence_after();
                    if (elect_one()) {
                        const uint64_t a = dt + (uint64_t)((uint32_t)(tail * kChunk) >> 4), b = dq + (uint64_t)((uint32_t)(pairs_of_tile * 2 * N * 128) >> 4);
                        for (int k = 0; k < tail_steps; ++k) mma_ss(d, a + (uint64_t)(k * 2), b + (uint64_t)(k * 2), kIdS, 1);
                        mma_commit(&s_full[tile & 1u]);
                    }
                }
                __syncwarp();
                if (++tail == TAILS) tail = 0, tphase ^= 1;
            }
        }
        if (issued) {  // no MMA is in flight when TMEM is released
            if (elect_one()) mma_commit(&drain[values]);
            __syncwarp();
            drain_wait(&drain[values], 0);
        }
    }
    tc_fence_before();
    __syncthreads();
    if (tid == 0 && side == 0 && *abort_flag) Deal::note_idle(p, share);  // (the join leaves this share's tile alone)
    if (warp == 9) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
}

template <int N>
cudaError_t cached_as(LatentProblem p, int sides, cudaStream_t stream) {
    constexpr auto kernel = latent_cached_kernel<N>;
    static DeviceOnce once;
    if (cudaError_t e = once.run([] { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, Shape<N>::BYTES); });
        e != cudaSuccess)
        return e;
    EncodeTiled fn = encode_fn();
    if (!fn) return cudaErrorInvalidValue;
    AttnProblem& a = p.a;
    // The pool as rows of R + P elements: its latents in boxes of one or two chunks of 64 elements (128-byte swizzled) of
    // a page's rows, up to a tile's, and the rest in boxes of one chunk, with zeros past a row's end.
    CUtensorMap latents, pool;
    const cuuint32_t rows = (cuuint32_t)(a.page < kKeys ? a.page : kKeys);
    cuuint64_t dims[3] = {64, (cuuint64_t)a.n_pages * a.page, (cuuint64_t)(a.D / 64)}, strides[2] = {(cuuint64_t)(2 * p.K), 128};
    cuuint32_t box[3] = {64, rows, rows == kKeys ? 2u : 1u}, estr[3] = {1, 1, 1};
    auto encode = [&](CUtensorMap* m, int rank) {
        return fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, rank, const_cast<void*>(a.k_pool), dims, strides, box, estr,
                  CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
    };
    if (!encode(&latents, 3)) return cudaErrorInvalidValue;
    dims[0] = (cuuint64_t)p.K;
    if (!encode(&pool, 2)) return cudaErrorInvalidValue;
    const int ctas = min(sm_count(), kLatentMaxParts / (2 * kLatentMaxRows));
    set_shares(a, sides * N, 1, ctas / sides, kMinBlocks, kTileCost, kKeys);
    Params pp{p, sides, tc_wait_limit_ns()};
    if (cudaError_t e = launch_k(kernel, dim3(a.shares * sides), dim3(kThreads), Shape<N>::BYTES, stream, latents, pool, pp); e != cudaSuccess) return e;
    return a.shares > 1 ? launch_attn_join(a, stream) : cudaSuccess;
}

}  // namespace

bool latent_cached_tc_supported(const LatentProblem& p) {
    return p.a.act_dtype == GBMOE_BF16 && p.a.D % 128 == 0 && p.K - p.a.D <= 64 && p.a.n_pages > 0;
}

cudaError_t launch_latent_cached_tc(const LatentProblem& p, cudaStream_t stream) {
    // Rows of a sequence, on average. As many of them in a CTA as there are, up to 64; fewer, and more CTAs beside each
    // other, where the key axis has too few blocks for every SM: a CTA's queries and results are then less (one sequence
    // of 4000 keys and 128 heads: 21.8 us with 64 rows, 19.8 with 32).
    const AttnProblem& a = p.a;
    const int64_t rows = ((int64_t)a.T * a.R + a.B - 1) / a.B;
    int n = rows <= 16 ? 16 : rows <= 32 ? 32 : 64;
    auto sides = [&] { return (int)min64(kMostSides, (rows + n - 1) / n); };
    const int64_t blocks = a.B * (((int64_t)a.max_pages * a.page + kKeys - 1) / kKeys + kTileCost);
    while (n > 16 && 2 * sides() <= kMostSides && 2 * sides() * ((blocks + kMinBlocks - 1) / kMinBlocks) <= sm_count()) n /= 2;
    return n == 16 ? cached_as<16>(p, sides(), stream) : n == 32 ? cached_as<32>(p, sides(), stream) : cached_as<64>(p, sides(), stream);
}

}  // namespace gbmoe
