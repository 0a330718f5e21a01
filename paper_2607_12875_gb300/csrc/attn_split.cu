// Attention of few query tokens over the paged cache (bf16; D 64, 96 or 128),
// the work dealt out to CTAs in equal shares of the key axis (Walk).
//
// A segment is a tile of 8 or 16 rows (token and head of the group) of one kv
// head and a run of its keys. The CTA's four warps take 16 keys each of every 64,
// each with its own ring of stages in shared memory that its own lane 0 fills by
// bulk copies (the keys of a page of one head are contiguous), so no warp waits
// for another within a segment and over 100 KB are in flight on an SM. Per stage:
// S^T = K Q^T and O^T += V^T P^T with mma.sync (m16n8k16), the running maximum
// and sum in between; at the end of a segment the warps' results are joined in
// shared memory.
//
// Bound by HBM for long keys (32 sequences, 1.07 GB of e4m3 pages of 8 kv heads of
// 128: 176 us, 6.1 TB/s), by its instructions with tiles of 16 rows (half of that
// rate), by latency for few keys: 4000 in 12 us, of which three blocks' loop is
// 2.5, the search for the share 1.5, page ids and scales 1.3, the queries 0.8, the
// warps' join 1 and the join kernel 3.
//
// The products are transposed, with keys and head columns as the 16 rows of the
// MMA, because query rows are few: eight of them fill the MMA's n. Both
// operands may have their k index permuted alike, and V's columns their order at
// will, so each lane reads whole pieces of a key's row and neighbouring columns
// of a value's row, and no transposing load is needed; P^T is turned by
// movmatrix. tcgen05 is not used: its 64 or 128 rows would be the keys here too,
// with operands in shared memory, and the e4m3 pages would have to be decoded
// into a second copy there.
//
// e4m3: codes become fp16 exactly. The scale of a page of keys multiplies its
// scores in fp32; the power of two of a page of values is added to its scores
// instead (base 2), with a maximum of its own: the weights that enter the second
// product are relative to the largest weight times scale, so pages of tiny
// values keep their accuracy. They are 2^kRoom at that weight, which uses fp16 up
// to its largest power: a weight is off by 2^-11 of itself or 2^-34 of the
// largest, so many keys of little weight beside one of much weight still count.
// The queries enter in fp16, each row divided by a power of two that brings its
// largest value into [1, 2): exact for values down to 2^-14 of it, an error of
// 2^-25 of it below.
//
// The weights are rounded to the 16-bit type of the MMA's other operand: fp16
// (e4m3) does not show beside the result's own rounding to bf16 (1.7e-3 of it on
// average), bf16 does (2.1e-3). Sums and statistics are fp32.

#include "attn_plan.cuh"
#include "tc_ptx.cuh"

namespace gbmoe {
namespace {

using namespace tc;

constexpr int kWarps = 4, kThreads = 32 * kWarps;
constexpr int kKeys = kBlockKeys / kWarps;  // keys of a stage of one warp
constexpr unsigned kFull = 0xffffffffu;
constexpr float kGrow = 6.0f;  // log2 of how far a row's maximum may run ahead
constexpr float kRoom = 9.0f;  // e4m3: log2 of a weight as large as the maximum; kGrow + kRoom is fp16's largest power
// Least blocks of 64 keys of a share, and how many a tile's set-up counts for. Us at (3, 2)
// and (2, 1): one sequence of 4000 e4m3 keys, 8 kv heads 12.3 and 11.6; two of 19000, 1 kv head 16.9
// and 20.1; 19 of up to 322 with 5 tokens, 4 kv heads 17.3 and 19.7. With (3, 0), where a share holds
// up to three tiles of one block in turn, the last takes 25 and three sequences of one key 12.6 instead of 7.0.
constexpr int kMinBlocks = 3, kTileCost = 2;
static_assert(kKeys == 16, "one MMA of keys, and never more than a page");

// kRows: 8 or 16
template <bool kE4m3, int D, int kRows>
struct Shape {
    static constexpr int EB = kE4m3 ? 1 : 2;           // bytes of an element
    static constexpr int ROW = D * EB;                 // bytes of a key's or value's row
    static constexpr int TILE = kKeys * ROW;
    // CTAs on an SM: by registers (kRows 16 holds twice the sums) and by ring size
    static constexpr int PER_SM = kRows == 8 && (kE4m3 || D == 64) ? 4 : 3;
    static constexpr int STAGES = (PER_SM == 4 ? 12288 : 16384) / (2 * TILE);
    static constexpr int RING = STAGES * 2 * TILE;
    static constexpr int LD = D + 4;                   // of a row in the join buffer, its statistics at the end
    static constexpr int JOIN = kWarps * kRows * LD * 4;
    static constexpr int BODY = kWarps * RING > JOIN ? kWarps * RING : JOIN;
    static constexpr int SMEM = BODY + kWarps * STAGES * 8;
    static constexpr int KS = D / 16;                  // MMAs along D of the scores; row tiles of the result
    static constexpr int NQ = kRows / 8;
    static_assert(STAGES >= 2, "stages");
};

__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_u32(dst)),
                 "l"(src), "r"(bytes), "r"(smem_u32(bar))
                 : "memory");
}

template <bool kF16>
__device__ __forceinline__ void mma16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    if constexpr (kF16)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                     : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                     : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// 8 x 8 matrix of 16-bit elements: lane 4 r + c holds row r, columns 2c, 2c + 1, before and after
__device__ __forceinline__ uint32_t transpose8(uint32_t v) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}

// the two e4m3 bytes of each half of w -> f16x2
__device__ __forceinline__ void f16x4_of(uint32_t w, uint32_t& lo, uint32_t& hi) {
    asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}"
        : "=r"(lo), "=r"(hi)
        : "r"(w));
}
template <bool kF16>
__device__ __forceinline__ uint32_t pack(float lo, float hi) {
    if constexpr (kF16) {
        __half2 h = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<uint32_t*>(&h);
    } else {
        return pack_bf16x2(lo, hi);
    }
}

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// N consecutive 32-bit words of shared memory (aligned to the largest power of two in 4 N bytes, up to 16)
template <int N>
__device__ __forceinline__ void lds(const uint8_t* p, uint32_t (&w)[N]) {
    if constexpr (N % 4 == 0) {
#pragma unroll
        for (int i = 0; i < N / 4; ++i) {
            const uint4 u = reinterpret_cast<const uint4*>(p)[i];
            w[4 * i] = u.x, w[4 * i + 1] = u.y, w[4 * i + 2] = u.z, w[4 * i + 3] = u.w;
        }
    } else if constexpr (N % 2 == 0) {
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            const uint2 u = reinterpret_cast<const uint2*>(p)[i];
            w[2 * i] = u.x, w[2 * i + 1] = u.y;
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) w[i] = reinterpret_cast<const uint32_t*>(p)[i];
    }
}

// A key's row in pieces of 16 bytes (8 where it is not 64-byte groups throughout)
// dealt to the four lanes of a quad in turn: lane c's k step i of the scores
// holds four neighbouring elements of D from element(i, c) on.
template <bool kE4m3, int D>
struct Pieces {
    static constexpr int PB = D * (kE4m3 ? 1 : 2) % 64 == 0 ? 16 : 8;     // bytes of a piece
    static constexpr int PE = PB / (kE4m3 ? 1 : 2);                       // its elements
    static constexpr int PER = PE / 4;                                    // k steps of a piece
    static constexpr int N = D / 16 / PER;                                // pieces of a lane
    __device__ static __forceinline__ int element(int i, int c) { return ((i / PER) * 4 + c) * PE + (i % PER) * 4; }
};

template <bool kE4m3, int D, int kRows>
__global__ void __launch_bounds__(kThreads, (Shape<kE4m3, D, kRows>::PER_SM))
attn_split_kernel(const __grid_constant__ AttnProblem p, uint64_t wait_limit_ns) {
    pdl_enter();
    using S = Shape<kE4m3, D, kRows>;
    using P = Pieces<kE4m3, D>;
    constexpr int STAGES = S::STAGES, KS = S::KS, NQ = S::NQ;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ int64_t plan[plan_words(kThreads)];
    __shared__ int abort_word;
    volatile int* abort_flag = &abort_word;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, c = lane & 3;
    const int G = p.R;
    uint8_t* ring = smem + warp * S::RING;
    uint64_t* full = reinterpret_cast<uint64_t*>(smem + S::BODY) + warp * STAGES;
    if (tid == 0) *abort_flag = 0;
    if (lane == 0) {
        for (int i = 0; i < STAGES; ++i) mbar_init(&full[i], 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    Walk<kRows> walk;
    if (!walk.begin(p, blockIdx.x, plan)) {  // (every thread synchronised in there)
        if (tid == 0) walk.note_idle(p, blockIdx.x);
        return;
    }
    int slot = 0;         // of the next stage to be read; fetches run ahead of it
    uint32_t parity = 0;  // of its barrier
    int pending = 0;      // copies in flight when a wait gave up

    do {
        const Segment& it = walk.g;
        const int h = it.head, row0 = it.tile * kRows;
        const int n_rows = (int)min64(kRows, (int64_t)it.s.nq * G - row0);
        // keys that some row of the tile sees; the keys that all of them see are all_lo .. all_hi
        int t_lo, all_hi, all_lo, u_hi;
        seen_keys(p, it.s, row0 / G, t_lo, all_hi);
        seen_keys(p, it.s, (row0 + n_rows - 1) / G, all_lo, u_hi);
        const int t_hi = u_hi + 1;
        // this segment's keys, in blocks of 64 that some row sees
        const int base = it.s.start + it.blk0 * kBlockKeys;
        const int skip = max(0, t_lo - base) / kBlockKeys;
        const int k_lo = base + skip * kBlockKeys + warp * kKeys;
        const int64_t k_end = min64((int64_t)it.s.start + (int64_t)it.blk1 * kBlockKeys, t_hi);
        const int mine = k_lo < k_end ? (int)((k_end - k_lo + kBlockKeys - 1) / kBlockKeys) : 0;  // stages of this warp

        // Page ids and scales of this warp's stages 32 w .. 32 w + 31 (lane: stage), for
        // the current w and the next.
        const int32_t* pages = p.page_table + (int64_t)it.b * p.max_pages;
        int pg[2];
        uint32_t sc[2] = {0, 0};  // scale bytes: keys, values << 8
        auto load_pages = [&](int w, int& id, uint32_t& s) {
            const int i = 32 * w + lane;
            id = -1;
            s = 0;
            if (i >= mine) return;
            const int v = pages[(k_lo + i * kBlockKeys) >> p.page_log2];
            if (v < 0 || v >= p.n_pages) return;
            id = v;
            if (kE4m3) s = p.k_scale[(int64_t)v * p.Hkv + h] | (uint32_t)p.v_scale[(int64_t)v * p.Hkv + h] << 8;
        };
        load_pages(0, pg[0], sc[0]);
        pg[1] = -1;
        auto fetch = [&](int i, int id, int at) {  // stage i, from page id, into ring slot `at`
            uint64_t* bar = &full[at];
            uint8_t* dst = ring + at * 2 * S::TILE;
            if (id < 0) {
                mbar_expect_tx(bar, 0);
                return;
            }
            const int64_t from = (((int64_t)id * p.Hkv + h) * p.page + ((k_lo + i * kBlockKeys) & (p.page - 1))) * S::ROW;
            mbar_expect_tx(bar, 2 * S::TILE);
            bulk_load(dst, static_cast<const uint8_t*>(p.k_pool) + from, S::TILE, bar);
            bulk_load(dst + S::TILE, static_cast<const uint8_t*>(p.v_pool) + from, S::TILE, bar);
        };
        int ahead = 0, ahead_slot = slot;  // the next stage to be fetched
        for (; ahead < STAGES - 1 && ahead < mine; ++ahead) {
            const int id = __shfl_sync(kFull, pg[0], ahead);
            if (lane == 0) fetch(ahead, id, ahead_slot);
            if (++ahead_slot == STAGES) ahead_slot = 0;
        }

        // queries as B fragments (row 8 n + g of this lane), and the rows 8 n + 2 c + z of
        // the lane's scores: the keys they see and what their products are multiplied by
        uint32_t qb[NQ][KS][2];
        int lo[NQ][2], hi[NQ][2];
        float qscale[NQ][2];
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            const int row = row0 + 8 * n + g;
            const bool have = 8 * n + g < n_rows;
            const __nv_bfloat16* src =
                static_cast<const __nv_bfloat16*>(p.q.p) + (it.s.q0 + row / G) * p.q.ts + (h * G + row % G) * p.q.hs;
            float top = 0.0f;
#pragma unroll
            for (int i = 0; i < KS; ++i) {
                const uint2 raw = have ? *reinterpret_cast<const uint2*>(src + P::element(i, c)) : make_uint2(0, 0);
                qb[n][i][0] = raw.x, qb[n][i][1] = raw.y;
                if constexpr (kE4m3)
                    top = fmaxf(fmaxf(fmaxf(top, fabsf(bf16lo(raw.x))), fmaxf(fabsf(bf16hi(raw.x)), fabsf(bf16lo(raw.y)))),
                                fabsf(bf16hi(raw.y)));
            }
            float mine_scale = p.scale_log2;
            if constexpr (kE4m3) {
                top = fmaxf(top, __shfl_xor_sync(kFull, top, 1));
                top = fmaxf(top, __shfl_xor_sync(kFull, top, 2));
                // 2^e of top's binade and 2^-e, kept inside fp32's normal range
                const int e = min(max((int)(__float_as_uint(top) >> 23), 1), 253);
                const float inv = __uint_as_float((uint32_t)(254 - e) << 23);
                mine_scale *= __uint_as_float((uint32_t)e << 23);
#pragma unroll
                for (int i = 0; i < KS; ++i)
#pragma unroll
                    for (int z = 0; z < 2; ++z) qb[n][i][z] = pack<true>(bf16lo(qb[n][i][z]) * inv, bf16hi(qb[n][i][z]) * inv);
            }
#pragma unroll
            for (int z = 0; z < 2; ++z) {
                const int r = 8 * n + 2 * c + z;
                qscale[n][z] = __shfl_sync(kFull, mine_scale, 4 * (2 * c + z));
                lo[n][z] = 0, hi[n][z] = -1;
                if (r < n_rows) seen_keys(p, it.s, (row0 + r) / G, lo[n][z], hi[n][z]);
            }
        }

        float m[NQ][2], mo[NQ][2], l[NQ][2];
        float o[NQ][KS][4];  // (columns g KS 2 + 2 y + {0, 1}; rows 2 c, 2 c + 1)
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            m[n][0] = m[n][1] = mo[n][0] = mo[n][1] = neg_inf();
            l[n][0] = l[n][1] = 0.0f;
#pragma unroll
            for (int y = 0; y < KS; ++y) o[n][y][0] = o[n][y][1] = o[n][y][2] = o[n][y][3] = 0.0f;
        }
        load_pages(1, pg[1], sc[1]);

        for (int i = 0; i < mine; ++i) {
            if ((i & 31) == 0 && i > 0) {
                pg[0] = pg[1], sc[0] = sc[1];
                load_pages((i >> 5) + 1, pg[1], sc[1]);
            }
            __syncwarp();  // every lane has read the stage before, whose slot the next fetch fills
            if (ahead < mine) {
                const int a = __shfl_sync(kFull, pg[0], ahead & 31), b = __shfl_sync(kFull, pg[1], ahead & 31);
                if (lane == 0) fetch(ahead, (ahead ^ i) & ~31 ? b : a, ahead_slot);
                ++ahead;
                if (++ahead_slot == STAGES) ahead_slot = 0;
            }
            const int id = __shfl_sync(kFull, pg[0], i & 31);
            const uint32_t scales = kE4m3 ? __shfl_sync(kFull, sc[0], i & 31) : 0;
            if (!warp_wait(&full[slot], parity, abort_flag, p.err, wait_limit_ns)) {
                pending = ahead - i;
                break;
            }
            uint8_t* sk = ring + slot * 2 * S::TILE;
            uint8_t* sv = sk + S::TILE;
            if (++slot == STAGES) slot = 0, parity ^= 1;
            const int key0 = k_lo + i * kBlockKeys;

            // ---- scores of keys g and g + 8
            float s[NQ][4];
            float s2[NQ][4];  // odd k steps apart: two chains of MMAs
#pragma unroll
            for (int n = 0; n < NQ; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[n][e] = s2[n][e] = 0.0f;
#pragma unroll
            for (int x = 0; x < P::N; ++x) {
                uint32_t ka[P::PB / 4], kb[P::PB / 4];
                lds(sk + g * S::ROW + (4 * x + c) * P::PB, ka);
                lds(sk + (g + 8) * S::ROW + (4 * x + c) * P::PB, kb);
#pragma unroll
                for (int y = 0; y < P::PER; ++y) {
                    const int ks = x * P::PER + y;
                    uint32_t a0, a1, a2, a3;
                    if constexpr (kE4m3) {
                        f16x4_of(ka[y], a0, a2);
                        f16x4_of(kb[y], a1, a3);
                    } else {
                        a0 = ka[2 * y], a2 = ka[2 * y + 1], a1 = kb[2 * y], a3 = kb[2 * y + 1];
                    }
#pragma unroll
                    for (int n = 0; n < NQ; ++n) mma16816<kE4m3>(ks & 1 ? s2[n] : s[n], a0, a1, a2, a3, qb[n][ks][0], qb[n][ks][1]);
                }
            }
            const float kf = kE4m3 ? e8m0_to_f32(scales & 255u) : 1.0f;
            const float ve = kE4m3 ? (float)((int)(scales >> 8) - 127) : 0.0f;
            const bool all = id >= 0 && key0 >= all_lo && key0 + kKeys - 1 <= all_hi;
#pragma unroll
            for (int n = 0; n < NQ; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    s[n][e] = (s[n][e] + s2[n][e]) * (kE4m3 ? qscale[n][e & 1] * kf : qscale[n][e & 1]);
                    const int key = key0 + g + 8 * (e >> 1);
                    if (!all && (id < 0 || key < lo[n][e & 1] || key > hi[n][e & 1])) s[n][e] = neg_inf();
                }

            // ---- running maximum and sum of rows 2 c + z
            // The maxima are raised, and the sums rescaled, only when a score has passed its row's by more
            // than 2^kGrow (a power that the weights have room for): most stages exchange nothing.
            bool raise = false;
#pragma unroll
            for (int n = 0; n < NQ; ++n)
#pragma unroll
                for (int z = 0; z < 2; ++z) {
                    const float top = fmaxf(s[n][z], s[n][2 + z]);
                    raise = raise || top > m[n][z] + kGrow || (kE4m3 && top + ve > mo[n][z] + kGrow);
                }
            if (__any_sync(kFull, raise)) {
#pragma unroll
                for (int n = 0; n < NQ; ++n) {
                    float f_o[2];
#pragma unroll
                    for (int z = 0; z < 2; ++z) {
                        float top = fmaxf(s[n][z], s[n][2 + z]);
                        top = fmaxf(top, __shfl_xor_sync(kFull, top, 4));
                        top = fmaxf(top, __shfl_xor_sync(kFull, top, 8));
                        top = fmaxf(top, __shfl_xor_sync(kFull, top, 16));
                        const float m_new = fmaxf(m[n][z], top);
                        f_o[z] = ex2(m[n][z] - (m_new == neg_inf() ? 0.0f : m_new));
                        l[n][z] *= f_o[z];
                        m[n][z] = m_new;
                        if constexpr (kE4m3) {
                            const float mo_new = fmaxf(mo[n][z], top + ve);
                            f_o[z] = ex2(mo[n][z] - (mo_new == neg_inf() ? 0.0f : mo_new));
                            mo[n][z] = mo_new;
                        }
                    }
#pragma unroll
                    for (int y = 0; y < KS; ++y) o[n][y][0] *= f_o[0], o[n][y][1] *= f_o[1], o[n][y][2] *= f_o[0], o[n][y][3] *= f_o[1];
                }
            }
#pragma unroll
            for (int n = 0; n < NQ; ++n)
#pragma unroll
                for (int z = 0; z < 2; ++z) {
                    const float b = m[n][z] == neg_inf() ? 0.0f : m[n][z];
                    const float p0 = ex2(s[n][z] - b), p1 = ex2(s[n][2 + z] - b);
                    l[n][z] += p0 + p1;
                    if constexpr (kE4m3) {
                        const float v = ve + kRoom - (mo[n][z] == neg_inf() ? 0.0f : mo[n][z]);
                        s[n][z] = ex2(s[n][z] + v), s[n][2 + z] = ex2(s[n][2 + z] + v);
                    } else {
                        s[n][z] = p0, s[n][2 + z] = p1;
                    }
                }
            if (kE4m3 && scales >> 8 == 255u) {  // values that are no numbers, for the rows that see them
#pragma unroll
                for (int n = 0; n < NQ; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int key = key0 + g + 8 * (e >> 1);
                        if (key >= lo[n][e & 1] && key <= hi[n][e & 1]) s[n][e] = __uint_as_float(0x7fc00000u);
                    }
            }
            uint32_t pb[NQ][2];
#pragma unroll
            for (int n = 0; n < NQ; ++n) {
                pb[n][0] = transpose8(pack<kE4m3>(s[n][0], s[n][1]));
                pb[n][1] = transpose8(pack<kE4m3>(s[n][2], s[n][3]));
            }
            if (!all) {
                // Values at masked keys may be NaN or infinite (unwritten slots), and 0 times
                // them is not 0. Keys that no row sees become 0; where another key's value is
                // not finite it is taken out and added for the rows that see it.
                bool bad = false;
                for (int x = lane * 16; x < S::TILE; x += 512) {
                    const int key = key0 + x / S::ROW;
                    uint4* at = reinterpret_cast<uint4*>(sv + x);
                    if (id < 0 || key < t_lo || key >= t_hi) {
                        *at = make_uint4(0, 0, 0, 0);
                        continue;
                    }
                    const uint4 u = *at;
                    const uint32_t q[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
                    for (int y = 0; y < 4; ++y)
                        bad = bad || (kE4m3 ? __vcmpeq4(q[y] & 0x7f7f7f7fu, 0x7f7f7f7fu) != 0
                                            : __vcmpgeu2(q[y] & 0x7fff7fffu, 0x7f807f80u) != 0);
                }
                __syncwarp();
                if (__any_sync(kFull, bad)) {
                    for (int e0 = 0; e0 < kKeys * D; e0 += 32) {
                        const int e = e0 + lane;
                        float val = 0.0f;
                        bool hit;
                        if constexpr (kE4m3) {
                            hit = (sv[e] & 0x7f) == 0x7f;
                            if (hit) val = __uint_as_float(0x7fc00000u), sv[e] = 0;
                        } else {
                            uint16_t* q = reinterpret_cast<uint16_t*>(sv) + e;
                            hit = (*q & 0x7fff) >= 0x7f80;
                            if (hit) val = __uint_as_float((uint32_t)*q << 16), *q = 0;
                        }
                        uint32_t hits = __ballot_sync(kFull, hit);
                        while (hits) {
                            const int src = __ffs(hits) - 1;
                            hits &= hits - 1;
                            const float v = __shfl_sync(kFull, val, src);
                            const int key = (e0 + src) / D, col = (e0 + src) % D;
#pragma unroll
                            for (int n = 0; n < NQ; ++n)
#pragma unroll
                                for (int z = 0; z < 2; ++z) {
                                    // the weight of this key and the lane's row, from the lane that has it
                                    const float w = __shfl_sync(kFull, key < 8 ? s[n][z] : s[n][2 + z], 4 * (key & 7) + c);
                                    const bool sees = key0 + key >= lo[n][z] && key0 + key <= hi[n][z];
#pragma unroll
                                    for (int y = 0; y < KS; ++y)
#pragma unroll
                                        for (int x = 0; x < 2; ++x)
                                            if (sees && col == g * 2 * KS + 2 * y + x) o[n][y][2 * x + z] += w * v;
                                }
                        }
                    }
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // before a later copy into this slot
                __syncwarp();
            }

            // ---- values: lane g takes columns 2 KS g .. 2 KS g + 2 KS - 1 of the keys 2 c, 2 c + 1, 2 c + 8, 2 c + 9
            {
                constexpr int WORDS = 2 * KS * S::EB / 4;
                uint32_t v[4][WORDS];
                const uint8_t* from = sv + 2 * c * S::ROW + g * 2 * KS * S::EB;
                lds(from, v[0]);
                lds(from + S::ROW, v[1]);
                lds(from + 8 * S::ROW, v[2]);
                lds(from + 9 * S::ROW, v[3]);
#pragma unroll
                for (int y = 0; y < WORDS; ++y) {
                    if constexpr (kE4m3) {
#pragma unroll
                        for (int x = 0; x < 2; ++x) {  // bytes 2 x, 2 x + 1 of the word: one row tile of the result
                            const uint32_t sel = x ? 0x7362u : 0x5140u;
                            uint32_t a0, a1, a2, a3;
                            f16x4_of(__byte_perm(v[0][y], v[1][y], sel), a0, a1);
                            f16x4_of(__byte_perm(v[2][y], v[3][y], sel), a2, a3);
#pragma unroll
                            for (int n = 0; n < NQ; ++n) mma16816<true>(o[n][2 * y + x], a0, a1, a2, a3, pb[n][0], pb[n][1]);
                        }
                    } else {
                        const uint32_t a0 = __byte_perm(v[0][y], v[1][y], 0x5410), a1 = __byte_perm(v[0][y], v[1][y], 0x7632);
                        const uint32_t a2 = __byte_perm(v[2][y], v[3][y], 0x5410), a3 = __byte_perm(v[2][y], v[3][y], 0x7632);
#pragma unroll
                        for (int n = 0; n < NQ; ++n) mma16816<false>(o[n][y], a0, a1, a2, a3, pb[n][0], pb[n][1]);
                    }
                }
            }
        }

        // ---- the four warps' results: sums relative to 2^mo, statistics
#pragma unroll
        for (int n = 0; n < NQ; ++n)
#pragma unroll
            for (int z = 0; z < 2; ++z) {
                l[n][z] += __shfl_xor_sync(kFull, l[n][z], 4);
                l[n][z] += __shfl_xor_sync(kFull, l[n][z], 8);
                l[n][z] += __shfl_xor_sync(kFull, l[n][z], 16);
            }
        __syncthreads();  // every warp has left its ring
        if (*abort_flag) break;
        constexpr int LD = S::LD;
        float* jo = reinterpret_cast<float*>(smem) + warp * kRows * LD;
#pragma unroll
        for (int n = 0; n < NQ; ++n)
#pragma unroll
            for (int z = 0; z < 2; ++z) {
                float* row = jo + (8 * n + 2 * c + z) * LD;
#pragma unroll
                for (int y = 0; y < KS; ++y)
                    *reinterpret_cast<float2*>(row + g * 2 * KS + 2 * y) = make_float2(o[n][y][z], o[n][y][2 + z]);
                if (g == 0) *reinterpret_cast<float4*>(row + D) = make_float4(m[n][z], l[n][z], kE4m3 ? mo[n][z] : m[n][z], 0.0f);
            }
        __syncthreads();
        constexpr int LANES = kThreads / kRows;  // threads of a row
        const int r = tid / LANES, x = tid % LANES;
        if (r < n_rows) {
            const float* rows = reinterpret_cast<const float*>(smem) + r * LD;
            float wt[kWarps];
            float M = neg_inf(), MO = neg_inf(), L = 0.0f;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                M = fmaxf(M, rows[w * kRows * LD + D]);
                MO = fmaxf(MO, rows[w * kRows * LD + D + 2]);
            }
            const float b = M == neg_inf() ? 0.0f : M, bo = MO == neg_inf() ? 0.0f : MO;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                L += rows[w * kRows * LD + D + 1] * ex2(rows[w * kRows * LD + D] - b);
                wt[w] = ex2(rows[w * kRows * LD + D + 2] - bo);
                if (kE4m3) wt[w] *= 1.0f / (1 << (int)kRoom);
            }
            int rlo, rhi;
            seen_keys(p, it.s, (row0 + r) / G, rlo, rhi);
            // without a score above -inf: whether the row sees a key at all (if not it gives 0, else 0 / 0)
            const bool sees = !(M == neg_inf() && L == 0.0f) || any_page(p, it.b, max(rlo, base), min(rhi, (int)k_end - 1));
            const bool empty = rhi < rlo || !sees;
            const int64_t t = it.s.q0 + (row0 + r) / G;
            const int hq = h * G + (row0 + r) % G;
            const int64_t at = it.slot * kRows + r;
            const float inv = empty ? 0.0f : ex2(bo - b) / L;
            if (x == 0) {
                if (it.slot >= 0) reinterpret_cast<float4*>(p.part_s)[at] = make_float4(M, L, MO, sees ? 1.0f : 0.0f);
                else if (p.lse) p.lse[t * p.Hq + hq] = empty ? neg_inf() : (b + log2f(L)) * kLn2;
            }
            for (int d = 4 * x; d < D; d += 4 * LANES) {
                float v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int w = 0; w < kWarps; ++w) {
                    const float4 q = *reinterpret_cast<const float4*>(rows + w * kRows * LD + d);
                    v[0] = fmaf(q.x, wt[w], v[0]), v[1] = fmaf(q.y, wt[w], v[1]);
                    v[2] = fmaf(q.z, wt[w], v[2]), v[3] = fmaf(q.w, wt[w], v[3]);
                }
                if (it.slot >= 0) {
                    *reinterpret_cast<float4*>(p.part_o + at * D + d) = make_float4(v[0], v[1], v[2], v[3]);
                } else {
                    __nv_bfloat16* out = const_cast<__nv_bfloat16*>(static_cast<const __nv_bfloat16*>(p.out.p)) + t * p.out.ts +
                                         hq * p.out.hs + d;
                    *reinterpret_cast<uint2*>(out) = empty ? make_uint2(0, 0)
                                                           : make_uint2(pack_bf16x2(v[0] * inv, v[1] * inv),
                                                                        pack_bf16x2(v[2] * inv, v[3] * inv));
                }
            }
        }
        if (tid == 0) walk.note(p);
        // the next segment's copies follow these reads and writes of the ring
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncthreads();
    } while (walk.next(p));
    // (a warp whose wait gave up has copies in flight: they land before the CTA leaves;
    // the join leaves this share's tile alone)
    if (*abort_flag && tid == 0) walk.note_idle(p, blockIdx.x);
    if (lane == 0) {
        const uint64_t t0 = global_ns();
        for (int i = 0; i < pending; ++i) {
            drain_wait(&full[slot], parity, t0);
            if (++slot == STAGES) slot = 0, parity ^= 1;
        }
    }
}

template <bool kE4m3, int D, int kRows>
cudaError_t split_as(AttnProblem p, cudaStream_t stream) {
    using S = Shape<kE4m3, D, kRows>;
    constexpr auto kernel = attn_split_kernel<kE4m3, D, kRows>;
    static DeviceOnce once;
    if (cudaError_t e = once.run([] { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, S::SMEM); });
        e != cudaSuccess)
        return e;
    set_shares(p, kRows, S::PER_SM, sm_count(), kMinBlocks, kTileCost);
    if (cudaError_t e = launch_k(kernel, dim3(p.shares), dim3(kThreads), S::SMEM, stream, p, tc_wait_limit_ns()); e != cudaSuccess)
        return e;
    return p.shares > 1 ? launch_attn_join(p, stream) : cudaSuccess;
}

template <bool kE4m3, int D>
cudaError_t split_rows(const AttnProblem& p, cudaStream_t stream) {
    // rows per sequence, on average: eight of them fit one MMA's n
    return (int64_t)p.T * p.R <= 8 * (int64_t)p.B ? split_as<kE4m3, D, 8>(p, stream) : split_as<kE4m3, D, 16>(p, stream);
}

template <bool kE4m3>
cudaError_t split_width(const AttnProblem& p, cudaStream_t stream) {
    return p.D == 64 ? split_rows<kE4m3, 64>(p, stream) : p.D == 96 ? split_rows<kE4m3, 96>(p, stream) : split_rows<kE4m3, 128>(p, stream);
}

}  // namespace

bool attn_split_supported(const AttnProblem& p) {
    return p.act_dtype == GBMOE_BF16 && p.paged && (p.D == 64 || p.D == 96 || p.D == 128);
}

cudaError_t launch_attn_split(const AttnProblem& p, cudaStream_t stream) {
    return p.e4m3 ? split_width<true>(p, stream) : split_width<false>(p, stream);
}

}  // namespace gbmoe
