// Absorbed latent attention of few query tokens over the paged cache on the tensor
// cores (bf16, R a multiple of 128, P up to 64), the work dealt out in equal shares of
// the key axis (Walk).
//
// A cached row serves every head, as key whole and as value in its first R elements, so
// a tile of 128 rows is loaded once and enters both products from the same place in
// shared memory. The products are transposed: the keys, and then the latent's elements,
// are the 128 rows of the MMA and N query rows (token and head; 16, 32 or 64) its
// columns, because the sums of 128 heads would fill all of TMEM (128 lanes x 512 fp32)
// and leave no place for scores. Per tile of 128 keys:
//   S^T = K Q^T      K-major tiles of 64 elements; N columns of TMEM, a lane is a key
//   P^T = exp2(scale S^T - m)   a thread has one key and half of the columns
//   O^T += C^T P^T   the same tiles, read MN-major; P^T in shared memory, in the place of
//                    the rotary keys, which the second product does not need
// The columns' maxima m are shared by all keys of a tile. They come from a segment's first
// tile and are raised, and O^T rescaled, only when a score passes its column's by 2^16:
// fp32 and bf16 weights lose nothing by that (their exponents reach 2^127), and tiles
// need no exchange between threads. The thread that finds such a score leaves a note, the
// MMA warp, which meets all of them anyway, sends the tile back once more.
// A thread sums its own key's weights, and the threads' sums are joined at the end of a segment.
// More rows than N: up to kMostSides CTAs beside each other take the same keys with N rows
// each, at about the same time, so that HBM is read once.
// Warps 0-3 and 4-7: softmax of the first and second half of the columns, queries and
// results; warp 8: TMA; warp 9: MMA.
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

constexpr int kKeys = 128;                // keys of a tile
constexpr int kThreads = 320;
constexpr int kChunk = kKeys * 128;       // bytes of 128 rows x 64 elements
constexpr unsigned kFull = 0xffffffffu;
constexpr float kGrow = 16.0f;            // log2 of how far a column's maximum may run ahead of m
constexpr float kMost = 3.402823466e38f;  // -kMost: a maximum of nothing
constexpr int kMinBlocks = 1, kTileCost = 0;
constexpr int kMostSides = 8;

// N: query rows of a CTA. Rings of pairs of chunks (128 latent elements) and of the rotary chunks.
template <int N>
struct Shape {
    static constexpr int COLS = N / 2;                       // columns of a thread
    static constexpr int PAIRS = N == 64 ? 4 : 5, TAILS = N == 16 ? 2 : 1;
    static constexpr int Q = 9 * N * 128;
    static constexpr int BODY = Q + PAIRS * 2 * kChunk + TAILS * kChunk;
    static constexpr int BYTES = 1024 + BODY;
    static_assert(BYTES + 4096 <= 227 * 1024, "shared memory");
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

struct Params {
    LatentProblem l;
    int sides;
    uint64_t wait_limit_ns;
};

template <int N>
__global__ void __launch_bounds__(kThreads, 1)
latent_cached_kernel(const __grid_constant__ CUtensorMap pool, const __grid_constant__ Params pp) {
    pdl_enter();
    using L = Shape<N>;
    constexpr int COLS = L::COLS, PAIRS = L::PAIRS, TAILS = L::TAILS;
    const AttnProblem& p = pp.l.a;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* sq = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    uint8_t* pairs = sq + L::Q;
    uint8_t* tails = pairs + PAIRS * 2 * kChunk;
    __shared__ uint64_t bars[2 * (PAIRS + TAILS) + 12];
    __shared__ Job jobs[2];
    uint64_t* full = bars;              // a pair landed
    uint64_t* empty = full + PAIRS;     // the products that read it finished
    uint64_t* tfull = empty + PAIRS;
    uint64_t* tempty = tfull + TAILS;
    uint64_t* q_full = tempty + TAILS;  // the queries are in shared memory
    uint64_t* s_full = q_full + 1;
    uint64_t* p_full = s_full + 1;      // P is written, O rescaled, unseen rows are 0
    uint64_t* o_full = p_full + 1;      // O holds this tile too
    uint64_t* drain = o_full + 1;
    uint64_t* half = drain + 1;         // the four warps of half of the columns meet
    uint64_t* both = half + 2;          // all eight
    uint64_t* j_full = both + 1;        // a job is in its slot
    uint64_t* j_empty = j_full + 2;     // every role has read it
    __shared__ uint32_t tmem_slot, good[TAILS];  // good: pages of the tile that are in the pool
    __shared__ int abort_word, row_hi[N];
    __shared__ uint32_t raised, again;  // a score far above its maximum was found in tile .. - 1; that tile is to be done once more
    __shared__ float sums[8][COLS];
    __shared__ __align__(16) float low[N], factor[N];  // the columns' -m, and what a raise multiplies by
    __shared__ int64_t plan[plan_words(kThreads)];
    volatile int* abort_flag = &abort_word;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int R = p.D, pairs_of_tile = R / 128, W = pp.l.K;
    const int share = blockIdx.x / pp.sides, side = blockIdx.x - share * pp.sides;
    if (tid == 0) {
        for (int i = 0; i < PAIRS; ++i) mbar_init(&full[i], 1), mbar_init(&empty[i], 1);
        for (int i = 0; i < TAILS; ++i) mbar_init(&tfull[i], 1), mbar_init(&tempty[i], 1);
        mbar_init(q_full, 8);
        mbar_init(s_full, 1);
        mbar_init(p_full, 8);
        mbar_init(o_full, 1);
        mbar_init(drain, 1);
        mbar_init(&half[0], 4);
        mbar_init(&half[1], 4);
        mbar_init(both, 8);
        for (int i = 0; i < 2; ++i) mbar_init(&j_full[i], 1), mbar_init(&j_empty[i], 9);  // (softmax warps, MMA)
        abort_word = 0;
        raised = again = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 9) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&tmem_slot)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    Walk<0, kKeys> walk;
    const bool any = __any_sync(kFull, walk.begin(p, share, plan));
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_slot, tS = tmem, tO = tmem + 128;  // O: pairs_of_tile times N columns
    auto wait_warp = [&](uint64_t* bar, uint32_t parity) { return warp_wait(bar, parity, abort_flag, p.err, pp.wait_limit_ns); };

    if (!any) {
        if (tid == 0 && side == 0) walk.note_idle(p, share);
    } else if (warp < 8) {
        // ------------------------------------------------------------ softmax
        const int wg = warp >> 2, r = (warp & 3) * 32 + lane, c0 = wg * COLS, wt = tid & 127;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t mS = tS + lanes + c0, mO = tO + lanes + c0;
        const float scale = p.scale_log2;
        uint32_t n_tiles = 0;  // so far
        int tail = 0, pair = 0;
        uint32_t tphase = 0, sn = 0;
        uint32_t meets = 0, meets_both = 0;
        // (mbarriers, not bar.sync: a warp whose wait gave up does not come)
        auto meet = [&](uint64_t* bar, uint32_t& n) {
            __syncwarp();
            if (lane == 0) mbar_arrive(bar);
            return wait_warp(bar, n++ & 1u);
        };
        bool ok = true;
        for (int j = 0; ok; ++j) {
            ok = wait_warp(&j_full[j & 1], (uint32_t)(j >> 1) & 1u);
            if (!ok) break;
            const Job x = jobs[j & 1];
            __syncwarp();
            if (lane == 0) mbar_arrive(&j_empty[j & 1]);
            if (x.end) break;
            if (x.rows > 0) {
                // queries: rows of N x 64 elements, 128-byte swizzled, zeros where there are none
                if (x.tiles > 0) {
                    const int pieces = (pairs_of_tile * 2 + 1) * 8;
                    for (int i = tid; i < N * pieces; i += 256) {
                        const int row = i / pieces, c = i - row * pieces;
                        const bool there = row < x.rows && 8 * c < W;
                        const int rr = x.row0 + (there ? row : 0), tok = rr / p.R;
                        const __nv_bfloat16* src = static_cast<const __nv_bfloat16*>(p.q.p) + (int64_t)(x.q0 + tok) * p.q.ts +
                                                   (rr - tok * p.R) * p.q.hs + (there ? 8 * c : 0);
                        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(sq + (c >> 3) * (N * 128) + sw128_off(row, c & 7))),
                                     "l"(src), "r"(there ? 16 : 0)
                                     : "memory");
                    }
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
            uint64_t l[COLS / 2];  // sums of the weights of this thread's keys, two columns each
#pragma unroll
            for (int c = 0; c < COLS / 2; ++c) l[c] = pack2(0.0f, 0.0f);
            if (x.tiles > 0) ok = wait_warp(s_full, sn++ & 1u);
            for (int t = 0; t < x.tiles && ok; ++t) {
                const int key = x.key0 + t * kKeys + r;
                ok = wait_warp(&tfull[tail], tphase);
                if (!ok) break;
                const uint32_t pages = *const_cast<volatile uint32_t*>(&good[tail]);
                const bool all = x.key0 + (t + 1) * kKeys - 1 <= x.all_hi && pages == (1u << (kKeys >> p.page_log2)) - 1u;
                const bool mine = pages >> (r >> p.page_log2) & 1u;
                bool poison = false;
                if (!all) {
                    auto at = [&](int i) {  // piece i of this key's latent
                        int slot = pair + (i >> 4);
                        if (slot >= PAIRS) slot -= PAIRS;
                        return reinterpret_cast<uint4*>(pairs + slot * 2 * kChunk + (i >> 3 & 1) * kChunk + sw128_off(r, i & 7));
                    };
                    if (mine && key > x.all_hi && key <= x.most_hi) {
                        for (int i = 0; i < R / 8; ++i) {
                            const uint4 v = *at(i);
                            poison = poison || (__vcmpgeu2(v.x & 0x7fff7fffu, 0x7f807f80u) | __vcmpgeu2(v.y & 0x7fff7fffu, 0x7f807f80u) |
                                                __vcmpgeu2(v.z & 0x7fff7fffu, 0x7f807f80u) | __vcmpgeu2(v.w & 0x7fff7fffu, 0x7f807f80u)) != 0;
                        }
                    }
                    ok = meet(both, meets_both);  // both threads of the key have looked
                    if (!ok) break;
                    if (poison || key > x.most_hi)
                        for (int i = wg * (R / 16); i < (wg + 1) * (R / 16); ++i) *at(i) = make_uint4(0, 0, 0, 0);
                }
                uint8_t* dst = tails + tail * kChunk;
                // One pass over the tile's scores. raise: the maxima are brought up to them first (the first tile, and
                // where a pass before found one too far above); else, whether one is. count: the weights enter the sums.
                auto pass = [&](bool raise, bool count) {
                    tc_fence_after();
                    uint32_t u[COLS];
                    tmem_load<COLS>(mS, u);
                    auto unseen = [&](int c) { return !all && (!mine || key > row_hi[c0 + c]); };
                    if (raise) {
                        // each column's largest score: over the warp's keys by a transposing maximum (lane: column), then
                        // over the four warps
                        float best[COLS];
#pragma unroll
                        for (int c = 0; c < COLS; ++c) best[c] = unseen(c) ? -kMost : fmaxf(__uint_as_float(u[c]) * scale, -kMost);
#pragma unroll
                        for (int d = 16; d >= COLS; d >>= 1)
#pragma unroll
                            for (int c = 0; c < COLS; ++c) best[c] = fmaxf(best[c], __shfl_xor_sync(kFull, best[c], d));
#pragma unroll
                        for (int d = COLS / 2; d; d >>= 1)
#pragma unroll
                            for (int c = 0; c < d; ++c) {
                                const bool up = lane & d;
                                const float give = up ? best[c] : best[c + d], keep = up ? best[c + d] : best[c];
                                best[c] = fmaxf(keep, __shfl_xor_sync(kFull, give, d));
                            }
                        if (lane < COLS) sums[warp][lane] = best[0];
                        ok = meet(&half[wg], meets);
                        if (!ok) return false;
                        if (wt < COLS) {
                            float m = -low[c0 + wt];
#pragma unroll
                            for (int w = 0; w < 4; ++w) m = fmaxf(m, sums[4 * wg + w][wt]);
                            factor[c0 + wt] = ex2(-low[c0 + wt] - m);  // (nothing yet: 0)
                            low[c0 + wt] = -m;
                        }
                        ok = meet(&half[wg], meets) && (t == 0 || wait_warp(o_full, (n_tiles - 1) & 1u));
                        if (!ok) return false;
                        if (t > 0) {
                            tc_fence_after();
#pragma unroll
                            for (int c = 0; c < COLS / 2; ++c) {
                                const float2 f = *reinterpret_cast<const float2*>(&factor[c0 + 2 * c]);
                                l[c] = fma2(l[c], pack2(f.x, f.y), pack2(0.0f, 0.0f));
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
                        }
                    }
                    const uint64_t sc2 = pack2(scale, scale);
                    float most = -kMost;
#pragma unroll
                    for (int c = 0; c < COLS; c += 4) {
                        const float4 m = *reinterpret_cast<const float4*>(&low[c0 + c]);
                        float2 a = unpack2(fma2(pack2(__uint_as_float(u[c]), __uint_as_float(u[c + 1])), sc2, pack2(m.x, m.y)));
                        float2 b = unpack2(fma2(pack2(__uint_as_float(u[c + 2]), __uint_as_float(u[c + 3])), sc2, pack2(m.z, m.w)));
                        if (!all) {
                            a.x = unseen(c) ? neg_inf() : a.x, a.y = unseen(c + 1) ? neg_inf() : a.y;
                            b.x = unseen(c + 2) ? neg_inf() : b.x, b.y = unseen(c + 3) ? neg_inf() : b.y;
                        }
                        most = max3(most, fmaxf(a.x, a.y), fmaxf(b.x, b.y));
                        u[c] = __float_as_uint(a.x), u[c + 1] = __float_as_uint(a.y);
                        u[c + 2] = __float_as_uint(b.x), u[c + 3] = __float_as_uint(b.y);
                    }
                    const bool over = __any_sync(kFull, most > kGrow) && !raise;
                    if (over) {
                        if (lane == 0) *const_cast<volatile uint32_t*>(&raised) = n_tiles + 1;
                    } else {
#pragma unroll
                        for (int c = 0; c < COLS; c += 8) {
                            uint32_t w[4];
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const int k = c + 2 * i;
                                float e0 = ex2(__uint_as_float(u[k])), e1 = ex2(__uint_as_float(u[k + 1]));
                                if (poison) {
                                    if (key <= row_hi[c0 + k]) e0 = __uint_as_float(0x7fc00000u);
                                    if (key <= row_hi[c0 + k + 1]) e1 = __uint_as_float(0x7fc00000u);
                                }
                                if (count) l[k >> 1] = add2(l[k >> 1], pack2(e0, e1));
                                w[i] = pack_bf16x2(e0, e1);
                            }
                            *reinterpret_cast<uint4*>(dst + sw128_off(r, (c0 + c) >> 3)) = make_uint4(w[0], w[1], w[2], w[3]);
                        }
                        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    }
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(p_full);
                    return over;
                };
                const bool over = pass(t == 0, true);
                // the next tile's scores, or the last tile's results, or this tile once more
                ok = ok && wait_warp(s_full, sn++ & 1u);
                if (ok && *const_cast<volatile uint32_t*>(&again) == n_tiles + 1) {
                    pass(true, over);
                    ok = ok && wait_warp(s_full, sn++ & 1u);
                }
                ++n_tiles;
                pair += pairs_of_tile;
                while (pair >= PAIRS) pair -= PAIRS;
                if (++tail == TAILS) tail = 0, tphase ^= 1;
            }
            if (!ok) break;
            // ------------------------------------------------------------ result
            if (x.rows > 0) {
                // each column's sum of weights over the keys, a transposing sum within the warp first
                float lc[COLS];
#pragma unroll
                for (int c = 0; c < COLS / 2; ++c) lc[2 * c] = unpack2(l[c]).x, lc[2 * c + 1] = unpack2(l[c]).y;
#pragma unroll
                for (int d = 16; d >= COLS; d >>= 1)
#pragma unroll
                    for (int c = 0; c < COLS; ++c) lc[c] += __shfl_xor_sync(kFull, lc[c], d);
#pragma unroll
                for (int d = COLS / 2; d; d >>= 1)
#pragma unroll
                    for (int c = 0; c < d; ++c) {
                        const bool up = lane & d;
                        const float give = up ? lc[c] : lc[c + d], keep = up ? lc[c + d] : lc[c];
                        lc[c] = keep + __shfl_xor_sync(kFull, give, d);
                    }
                if (lane < COLS) sums[warp][lane] = lc[0];
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
    } else if (warp == 8) {
        // ------------------------------------------------------------ TMA producer
        uint32_t inflight = 0, par = 0, tinflight = 0, tpar = 0;
        int slot = 0, tail = 0;
        uint32_t phase = 0, tphase = 0;
        const int per_tile = kKeys >> p.page_log2, box = p.page * 128;
        const int nowhere = p.n_pages << p.page_log2;  // rows past the pool: the copy brings zeros
        bool ok = true, more = true;
        for (int j = 0; ok; ++j) {
            ok = wait_warp(&j_empty[j & 1], ((uint32_t)(j >> 1) & 1u) ^ 1u);
            if (!ok) break;
            Job x = job_of<N>(p, walk.g, side);
            if (!more) x.end = 1;
            if (lane == 0) {
                jobs[j & 1] = x;
                mbar_arrive(&j_full[j & 1]);
                if (more && side == 0) walk.note(p);
            }
            __syncwarp();
            if (!more) break;
            const int32_t* ids = p.page_table + (int64_t)x.b * p.max_pages;
            auto first_row = [&](int t) {  // of this lane's page of tile t
                const int at = x.key0 + t * kKeys + (lane << p.page_log2);
                if (lane >= per_tile || t >= x.tiles || at > x.most_hi) return nowhere;
                const int id = ids[at >> p.page_log2];
                return id >= 0 && id < p.n_pages ? id << p.page_log2 : nowhere;
            };
            int row = first_row(0);
            for (int t = 0; t < x.tiles && ok; ++t) {
                const int ahead = first_row(t + 1);
                const uint32_t mask = __ballot_sync(kFull, row != nowhere);
                // lane: page lane % per_tile of the first or second chunk of a pair
                const int from = __shfl_sync(kFull, row, lane & (per_tile - 1)), chunk = lane / per_tile;
                for (int i = 0; i < pairs_of_tile; ++i) {
                    ok = wait_warp(&empty[slot], phase ^ 1);
                    if (!ok) break;
                    if (lane == 0) mbar_expect_tx(&full[slot], 2 * kChunk);
                    __syncwarp();
                    if (chunk < 2)
                        tma_load_2d(pairs + (2 * slot + chunk) * kChunk + (lane & (per_tile - 1)) * box, &pool, 128 * i + 64 * chunk, from, &full[slot]);
                    inflight |= 1u << slot;
                    par = (par & ~(1u << slot)) | (phase << slot);
                    if (++slot == PAIRS) slot = 0, phase ^= 1;
                }
                if (!ok) break;
                ok = wait_warp(&tempty[tail], tphase ^ 1);
                if (!ok) break;
                if (lane == 0) {
                    *const_cast<volatile uint32_t*>(&good[tail]) = mask;
                    mbar_expect_tx(&tfull[tail], W > R ? kChunk : 0);
                }
                __syncwarp();
                if (chunk < 1 && W > R) tma_load_2d(tails + tail * kChunk + lane * box, &pool, R, from, &tfull[tail]);
                tinflight |= 1u << tail;
                tpar = (tpar & ~(1u << tail)) | (tphase << tail);
                if (++tail == TAILS) tail = 0, tphase ^= 1;
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
        // ------------------------- MMA issuer (the whole warp, one lane issues)
        constexpr uint32_t kId = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(kKeys >> 4) << 24);
        constexpr uint32_t kIdO = kId | (1u << 15) | (1u << 16);  // both operands MN-major
        const uint32_t tm = __reduce_max_sync(kFull, tmem);
        const uint64_t dq = sw128_desc(smem_u32(sq)), dk = sw128_desc(smem_u32(pairs)), dt = sw128_desc(smem_u32(tails));
        const uint64_t dv = mn_desc(smem_u32(pairs)), dp = mn_desc(smem_u32(tails));
        const int tail_steps = (W - R + 15) / 16;
        int slot = 0, tail = 0;
        uint32_t phase = 0, tphase = 0, qn = 0, pn = 0, tile = 0;
        bool ok = true, issued = false;
        for (int j = 0; ok; ++j) {
            ok = wait_warp(&j_full[j & 1], (uint32_t)(j >> 1) & 1u);
            if (!ok) break;
            // (what the loops run to comes from warp-wide reductions, so that the MMA's operands stay in uniform registers)
            const int tiles = __reduce_max_sync(kFull, jobs[j & 1].tiles), end = __reduce_max_sync(kFull, jobs[j & 1].end);
            __syncwarp();
            if (lane == 0) mbar_arrive(&j_empty[j & 1]);
            if (end) break;
            if (tiles <= 0) continue;
            ok = wait_warp(q_full, qn++ & 1u);
            for (int t = 0; t < tiles && ok; ++t) {
                const int slot0 = slot;
                // The issue queue is shallow: what a wait takes after a batch of MMAs the tensor cores stand still. So the
                // next batch's barrier is looked at before the last MMAs of this one.
                auto peek = [&](uint64_t* bar, uint32_t parity) { return __all_sync(kFull, mbar_test_wait(bar, parity)); };
                bool ready = false;
                for (int i = 0; i < pairs_of_tile; ++i) {
                    ok = ready || wait_warp(&full[slot], phase);
                    if (!ok) break;
                    tc_fence_after();
                    const uint64_t a = dk + (uint64_t)((uint32_t)(slot * 2 * kChunk) >> 4), b = dq + (uint64_t)((uint32_t)(i * 2 * N * 128) >> 4);
                    if (++slot == PAIRS) slot = 0, phase ^= 1;
                    if (elect_one()) {
#pragma unroll
                        for (int k = 0; k < 5; ++k)
                            mma_ss(tm, a + (((k >> 2) * kChunk + (k & 3) * 32) >> 4), b + (((k >> 2) * N * 128 + (k & 3) * 32) >> 4), kId, i > 0 || k > 0);
                    }
                    __syncwarp();
                    ready = i + 1 < pairs_of_tile ? peek(&full[slot], phase) : peek(&tfull[tail], tphase);
                    if (elect_one()) {
#pragma unroll
                        for (int k = 5; k < 8; ++k)
                            mma_ss(tm, a + (((k >> 2) * kChunk + (k & 3) * 32) >> 4), b + (((k >> 2) * N * 128 + (k & 3) * 32) >> 4), kId, 1);
                    }
                    __syncwarp();
                    issued = true;
                }
                if (!ok) break;
                ok = ready || wait_warp(&tfull[tail], tphase);
                if (!ok) break;
                tc_fence_after();
                if (elect_one()) {
                    const uint64_t a = dt + (uint64_t)((uint32_t)(tail * kChunk) >> 4), b = dq + (uint64_t)((uint32_t)(pairs_of_tile * 2 * N * 128) >> 4);
                    for (int k = 0; k < tail_steps; ++k) mma_ss(tm, a + (uint64_t)(k * 2), b + (uint64_t)(k * 2), kId, 1);
                    mma_commit(s_full);
                }
                __syncwarp();
                ok = wait_warp(p_full, pn++ & 1u);
                if (!ok) break;
                ++tile;
                if (__any_sync(kFull, *const_cast<volatile uint32_t*>(&raised) == tile)) {
                    if (lane == 0) {
                        *const_cast<volatile uint32_t*>(&again) = tile;
                        mbar_arrive(s_full);
                    }
                    __syncwarp();
                    ok = wait_warp(p_full, pn++ & 1u);
                    if (!ok) break;
                }
                tc_fence_after();
                int sv = slot0;
                for (int i = 0; i < pairs_of_tile; ++i) {
                    if (elect_one()) {
                        const uint64_t a = dv + (uint64_t)((uint32_t)(sv * 2 * kChunk) >> 4), b = dp + (uint64_t)((uint32_t)(tail * kChunk) >> 4);
#pragma unroll
                        for (int k = 0; k < kKeys / 16; ++k)
                            mma_ss(tm + 128 + i * N, a + (uint64_t)(k * 2048 >> 4), b + (uint64_t)(k * 2048 >> 4), kIdO, t > 0 || k > 0);
                        mma_commit(&empty[sv]);
                        if (i == pairs_of_tile - 1) {
                            mma_commit(&tempty[tail]);
                            mma_commit(o_full);
                            if (t == tiles - 1) mma_commit(s_full);
                        }
                    }
                    __syncwarp();
                    if (++sv == PAIRS) sv = 0;
                }
                if (++tail == TAILS) tail = 0, tphase ^= 1;
            }
        }
        if (issued) {  // no MMA is in flight when TMEM is released
            if (elect_one()) mma_commit(drain);
            __syncwarp();
            drain_wait(drain, 0);
        }
    }
    tc_fence_before();
    __syncthreads();
    if (tid == 0 && side == 0 && *abort_flag) Walk<0, kKeys>::note_idle(p, share);  // (the join leaves this share's tile alone)
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
    // the pool as rows of R + P elements, in boxes of 64 elements (128-byte swizzled, zeros past a row's end) of a page
    CUtensorMap map;
    cuuint64_t dims[2] = {(cuuint64_t)p.K, (cuuint64_t)a.n_pages * a.page}, strides[1] = {(cuuint64_t)(2 * p.K)};
    cuuint32_t box[2] = {64, (cuuint32_t)a.page}, estr[2] = {1, 1};
    if (fn(&map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(a.k_pool), dims, strides, box, estr,
           CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
           CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
        return cudaErrorInvalidValue;
    const int ctas = min(sm_count(), kLatentMaxParts / (2 * kLatentMaxRows));
    set_shares(a, sides * N, 1, ctas / sides, kMinBlocks, kTileCost, kKeys);
    Params pp{p, sides, tc_wait_limit_ns()};
    if (cudaError_t e = launch_k(kernel, dim3(a.shares * sides), dim3(kThreads), Shape<N>::BYTES, stream, map, pp); e != cudaSuccess) return e;
    return a.shares > 1 ? launch_attn_join(a, stream) : cudaSuccess;
}

}  // namespace

bool latent_cached_tc_supported(const LatentProblem& p) {
    return p.a.act_dtype == GBMOE_BF16 && p.a.D % 128 == 0 && p.K - p.a.D <= 64 && p.a.n_pages > 0;
}

cudaError_t launch_latent_cached_tc(const LatentProblem& p, cudaStream_t stream) {
    // rows of a sequence, on average
    const int64_t rows = ((int64_t)p.a.T * p.a.R + p.a.B - 1) / p.a.B;
    auto sides = [&](int n) { return (int)min64(kMostSides, (rows + n - 1) / n); };
    if (rows <= 16) return cached_as<16>(p, 1, stream);
    if (rows <= 32) return cached_as<32>(p, 1, stream);
    return cached_as<64>(p, sides(64), stream);
}

}  // namespace gbmoe
