// Attention of few query tokens over the paged cache (bf16; D 64, 96 or 128),
// the key axis split over CTAs and, in a CTA, over its warps.
//
// A work item is 16 rows (token and head of the group) of one kv head and a
// chunk of the sequence's keys. Its four warps take turns at stages of 32 (e4m3)
// or 16 (bf16) keys, each with its own ring of stages in shared memory that its
// own lane 0 fills by bulk copies (a page of one head is contiguous), so no warp
// waits for another before the end, and a CTA keeps up to 96 KB in flight: HBM
// is the bound. Per stage: S = Q K^T and O += P V with mma.sync (m16n8k16),
// the running maximum and sum in between; at the end the warps' results are
// joined in shared memory.
//
// Both operands of an MMA may have their k index permuted alike, and the n index
// of V (the columns of the result) at will, so each lane reads whole 16-byte
// pieces of a key's row and neighbouring columns of a value's row, and no
// transposing load is needed. tcgen05 is not used: at 16 rows its 128-row tiles
// would be mostly padding, and the products take a fraction of the load time.
//
// e4m3: codes become fp16 exactly. The scale of a page of keys multiplies its
// scores in fp32; the power of two of a page of values is added to its scores
// instead (base 2), with a maximum of its own: the weights that enter the second
// product are relative to the largest weight times scale, so pages of tiny
// values keep their accuracy. The queries enter in fp16, each row divided by a
// power of two that brings its largest value into [1, 2): exact for values down
// to 2^-14 of it, an error of 2^-25 of it below. The weights are rounded to fp16
// (e4m3) or bf16.
#include <climits>

#include "attn_plan.cuh"
#include "tc_ptx.cuh"

namespace gbmoe {
namespace {

using namespace tc;

constexpr int kWarps = 4, kThreads = 32 * kWarps;
constexpr unsigned kFull = 0xffffffffu;

template <bool kE4m3, int D>
struct Shape {
    static constexpr int EB = kE4m3 ? 1 : 2;              // bytes of an element
    static constexpr int KEYS = kE4m3 ? 32 : 16;          // keys of a stage
    static constexpr int ROW = D * EB;                    // bytes of a key's or value's row
    static constexpr int TILE = KEYS * ROW;
    static constexpr int STAGES = 24576 / (2 * TILE);     // 24 KB of a warp
    static constexpr int RING = STAGES * 2 * TILE;
    static constexpr int SMEM = kWarps * RING + kWarps * STAGES * 8;
    static constexpr int KS = D / 16;                     // MMAs along D of the scores
    static constexpr int NT = D / 8;                      // column tiles of the result
    static_assert(STAGES >= 2, "stages");
    // the join at the end: sums and statistics of each warp
    static_assert(kWarps * 16 * (D + 4) * 4 <= kWarps * RING, "join buffer");
};

__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_u32(dst)),
                 "l"(src), "r"(bytes), "r"(smem_u32(bar))
                 : "memory");
}

template <bool kF16>
__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    if constexpr (kF16)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// two e4m3 bytes (the low half of w) -> f16x2
__device__ __forceinline__ uint32_t f16x2_of(uint32_t w) {
    uint32_t r;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((unsigned short)w));
    return r;
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

// N consecutive 32-bit words of shared memory (N words aligned to the largest power of two in 4 N bytes)
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

// first of the four neighbouring elements of D that lane quarter c (lane % 4)
// holds in k step i of the scores: pieces of 16 bytes (8 where a row is not
// 64-byte pieces throughout) dealt to the four lanes in turn
template <bool kE4m3, int D>
struct Pieces {
    static constexpr int PB = D * (kE4m3 ? 1 : 2) % 64 == 0 ? 16 : 8;     // bytes of a piece
    static constexpr int PE = PB / (kE4m3 ? 1 : 2);                       // its elements
    static constexpr int PER = PE / 4;                                    // k steps of a piece
    static constexpr int N = D / 16 / PER;                                // pieces of a lane
    __device__ static __forceinline__ int element(int i, int c) { return ((i / PER) * 4 + c) * PE + (i % PER) * 4; }
};

template <bool kE4m3, int D>
__global__ void __launch_bounds__(kThreads) attn_split_kernel(const AttnProblem p, uint64_t wait_limit_ns) {
    pdl_enter();
    using S = Shape<kE4m3, D>;
    using P = Pieces<kE4m3, D>;
    constexpr int KEYS = S::KEYS, SN = KEYS / 8, STAGES = S::STAGES;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ int64_t plan[plan_words(kThreads)];
    __shared__ int abort_word;
    volatile int* abort_flag = &abort_word;
    const int h = blockIdx.x % p.Hkv, G = p.R;
    const Item it = find_item<kSplitRows>(p, blockIdx.x / p.Hkv, plan);
    if (it.b < 0) return;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, c = lane & 3;
    const int row0 = it.tile * kSplitRows;
    const int n_rows = (int)min64(kSplitRows, (int64_t)it.s.nq * G - row0);
    uint8_t* ring = smem + warp * S::RING;
    uint64_t* full = reinterpret_cast<uint64_t*>(smem + kWarps * S::RING) + warp * STAGES;
    if (tid == 0) *abort_flag = 0;
    if (lane == 0) {
        for (int i = 0; i < STAGES; ++i) mbar_init(&full[i], 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();

    // this lane's rows g and g + 8: the keys they see, and their queries as A fragments
    int lo[2], hi[2];
    uint32_t qa[S::KS][4];
    float qscale[2];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const int row = row0 + g + 8 * r;
        lo[r] = 0, hi[r] = -1, qscale[r] = p.scale_log2;
        const bool have = g + 8 * r < n_rows;
        if (have) seen_keys(p, it.s, row / G, lo[r], hi[r]);
        const __nv_bfloat16* src = static_cast<const __nv_bfloat16*>(p.q.p) + (it.s.q0 + row / G) * p.q.ts + (h * G + row % G) * p.q.hs;
        uint2 raw[S::KS];
        float top = 0.0f;
#pragma unroll
        for (int i = 0; i < S::KS; ++i) {
            raw[i] = have ? *reinterpret_cast<const uint2*>(src + P::element(i, c)) : make_uint2(0, 0);
            if constexpr (kE4m3)
                top = fmaxf(fmaxf(fmaxf(top, fabsf(bf16lo(raw[i].x))), fmaxf(fabsf(bf16hi(raw[i].x)), fabsf(bf16lo(raw[i].y)))),
                            fabsf(bf16hi(raw[i].y)));
        }
        float inv = 1.0f;
        if constexpr (kE4m3) {
            top = fmaxf(top, __shfl_xor_sync(kFull, top, 1));
            top = fmaxf(top, __shfl_xor_sync(kFull, top, 2));
            // 2^-e and 2^e of top's binade, kept inside fp32's normal range
            const int e = min(max((int)(__float_as_uint(top) >> 23), 1), 253);
            inv = __uint_as_float((uint32_t)(254 - e) << 23);
            qscale[r] = p.scale_log2 * __uint_as_float((uint32_t)e << 23);
        }
#pragma unroll
        for (int i = 0; i < S::KS; ++i) {
            if constexpr (kE4m3) {
                qa[i][r] = pack<true>(bf16lo(raw[i].x) * inv, bf16hi(raw[i].x) * inv);
                qa[i][r + 2] = pack<true>(bf16lo(raw[i].y) * inv, bf16hi(raw[i].y) * inv);
            } else {
                qa[i][r] = raw[i].x;
                qa[i][r + 2] = raw[i].y;
            }
        }
    }
    // keys that some row of the tile sees, in this chunk
    int t_lo, t_hi, u_lo, u_hi;
    seen_keys(p, it.s, row0 / G, t_lo, t_hi);
    seen_keys(p, it.s, (row0 + n_rows - 1) / G, u_lo, u_hi);
    if (t_hi < 0) t_lo = 0;
    const int k_lo = max(it.k_lo, t_lo) & ~(KEYS - 1), k_hi = min(it.k_hi, u_hi + 1);
    const int n_stages = k_hi > k_lo ? (k_hi - k_lo + KEYS - 1) / KEYS : 0;
    const int mine = n_stages > warp ? (n_stages - warp + kWarps - 1) / kWarps : 0;  // stages warp, warp + 4, ..

    const int32_t* pages = p.page_table + (int64_t)it.b * p.max_pages;
    const int copy_keys = min(p.page, KEYS);  // keys of one bulk copy
    const int copies = KEYS / copy_keys;      // 1, or 2 (e4m3, pages of 16)
    // Page ids of this warp's stages 16 w .. 16 w + 15, two per stage: lane 2 i + x
    // holds the page of half x of stage 16 w + i (-1: outside the pool, or past the
    // chunk), and its scales.
    int pg = -1, next_pg = -1;
    uint32_t ksc = 0, vsc = 0;
    auto load_pages = [&](int w) {
        const int i = 16 * w + (lane >> 1);
        const int key = k_lo + (warp + kWarps * i) * KEYS + (lane & 1) * (KEYS / 2);
        if (i >= mine || key >= k_hi) return -1;
        const int id = pages[key / p.page];
        return id >= 0 && id < p.n_pages ? id : -1;
    };
    auto load_scales = [&](int id, uint32_t& a, uint32_t& b) {
        a = b = 0;
        if (kE4m3 && id >= 0) a = p.k_scale[(int64_t)id * p.Hkv + h], b = p.v_scale[(int64_t)id * p.Hkv + h];
    };
    // stage i (of this warp) into its slot; id0, id1: the pages of its halves
    auto fetch = [&](int i, int id0, int id1) {
        uint8_t* dst = ring + (i % STAGES) * 2 * S::TILE;
        uint64_t* bar = &full[i % STAGES];
        const int key = k_lo + (warp + kWarps * i) * KEYS;
        const uint32_t bytes = copy_keys * S::ROW;
        uint32_t total = 0;
        for (int x = 0; x < copies; ++x)
            if ((x ? id1 : id0) >= 0) total += 2 * bytes;
        mbar_expect_tx(bar, total);
        for (int x = 0; x < copies; ++x) {
            const int id = x ? id1 : id0;
            if (id < 0) continue;
            const int64_t at = (((int64_t)id * p.Hkv + h) * p.page + (key + x * copy_keys) % p.page) * S::ROW;
            bulk_load(dst + x * bytes, static_cast<const uint8_t*>(p.k_pool) + at, bytes, bar);
            bulk_load(dst + S::TILE + x * bytes, static_cast<const uint8_t*>(p.v_pool) + at, bytes, bar);
        }
    };

    float m[2] = {neg_inf(), neg_inf()}, mo[2] = {neg_inf(), neg_inf()}, l[2] = {0.f, 0.f};
    float o[S::NT][4];
#pragma unroll
    for (int i = 0; i < S::NT; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.0f;

    // pages of 32 stages ahead: the ids of this window and the next one
    pg = load_pages(0);
    load_scales(pg, ksc, vsc);
    next_pg = load_pages(1);
    uint32_t next_ksc, next_vsc;
    load_scales(next_pg, next_ksc, next_vsc);
    auto page_of = [&](int i, int w, int x) {  // page of half x of stage i, window w current; warp-uniform i
        const int src = 2 * (i & 15) + x;
        const int a = __shfl_sync(kFull, pg, src), b = __shfl_sync(kFull, next_pg, src);
        return (i >> 4) == w ? a : b;
    };
    int ahead = 0;  // stages fetched
    for (; ahead < STAGES - 1 && ahead < mine; ++ahead) {
        const int a = page_of(ahead, 0, 0), b = page_of(ahead, 0, 1);
        if (lane == 0) fetch(ahead, a, b);
    }
    bool ok = true;
    for (int i = 0; i < mine; ++i) {
        const int w = i >> 4;
        if ((i & 15) == 0 && i > 0) {
            pg = next_pg, ksc = next_ksc, vsc = next_vsc;
            next_pg = load_pages(w + 1);
            load_scales(next_pg, next_ksc, next_vsc);
        }
        // the slot that stage i - 1 used is free (every lane has read it)
        __syncwarp();
        if (ahead < mine) {
            const int a = page_of(ahead, w, 0), b = page_of(ahead, w, 1);
            if (lane == 0) fetch(ahead, a, b);
            ++ahead;
        }
        if (!warp_wait(&full[i % STAGES], (uint32_t)(i / STAGES) & 1u, abort_flag, p.err, wait_limit_ns)) { ok = false; break; }
        uint8_t* sk = ring + (i % STAGES) * 2 * S::TILE;
        uint8_t* sv = sk + S::TILE;
        const int key0 = k_lo + (warp + kWarps * i) * KEYS;
        const int id0 = __shfl_sync(kFull, pg, 2 * (i & 15)), id1 = __shfl_sync(kFull, pg, 2 * (i & 15) + 1);

        // ---- scores
        float s[SN][4];
#pragma unroll
        for (int n = 0; n < SN; ++n) {
            s[n][0] = s[n][1] = s[n][2] = s[n][3] = 0.0f;
            const uint8_t* row = sk + (8 * n + g) * S::ROW;
#pragma unroll
            for (int x = 0; x < P::N; ++x) {
                uint32_t b[P::PB / 4];
                lds(row + (4 * x + c) * P::PB, b);
#pragma unroll
                for (int y = 0; y < P::PER; ++y) {
                    if constexpr (kE4m3) mma16816<true>(s[n], qa[x * P::PER + y], f16x2_of(b[y]), f16x2_of(b[y] >> 16));
                    else mma16816<false>(s[n], qa[x * P::PER + y], b[2 * y], b[2 * y + 1]);
                }
            }
        }
        // ---- scale and mask; this stage's scales are per half
        float kf[2] = {1.0f, 1.0f}, ve[2] = {0.0f, 0.0f};
        if constexpr (kE4m3) {
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                kf[x] = e8m0_to_f32(__shfl_sync(kFull, ksc, 2 * (i & 15) + x));
                const uint32_t v = __shfl_sync(kFull, vsc, 2 * (i & 15) + x);
                ve[x] = v == 255u ? __uint_as_float(0x7fc00000u) : (float)((int)v - 127);
            }
        }
        const bool whole = id0 >= 0 && id1 >= 0;
        bool all = whole;
#pragma unroll
        for (int r = 0; r < 2; ++r) all = all && (g + 8 * r >= n_rows || (lo[r] <= key0 && hi[r] >= key0 + KEYS - 1));
        all = __all_sync(kFull, all);
#pragma unroll
        for (int n = 0; n < SN; ++n) {
            const float f = kE4m3 ? kf[n >= SN / 2] : 1.0f;
#pragma unroll
            for (int e = 0; e < 4; ++e) s[n][e] *= qscale[e >> 1] * f;
        }
        if (!all) {
#pragma unroll
            for (int n = 0; n < SN; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int key = key0 + 8 * n + 2 * c + (e & 1);
                    const bool have = (n >= SN / 2 ? id1 : id0) >= 0;
                    if (!have || key < lo[e >> 1] || key > hi[e >> 1]) s[n][e] = neg_inf();
                }
        }
        // ---- running maximum and sum
        uint32_t pa[KEYS / 16][4];
        float f_o[2];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            float top = neg_inf(), topo = neg_inf();
#pragma unroll
            for (int n = 0; n < SN; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    top = fmaxf(top, s[n][2 * r + e]);
                    if (kE4m3) topo = fmaxf(topo, s[n][2 * r + e] + ve[n >= SN / 2]);
                }
            top = fmaxf(top, __shfl_xor_sync(kFull, top, 1));
            top = fmaxf(top, __shfl_xor_sync(kFull, top, 2));
            const float m_new = fmaxf(m[r], top), base = m_new == neg_inf() ? 0.0f : m_new;
            const float f = ex2(m[r] - base);
            float sum = 0.0f;
            if constexpr (kE4m3) {
                topo = fmaxf(topo, __shfl_xor_sync(kFull, topo, 1));
                topo = fmaxf(topo, __shfl_xor_sync(kFull, topo, 2));
                const float mo_new = fmaxf(mo[r], topo), base_o = mo_new == neg_inf() ? 0.0f : mo_new;
                f_o[r] = ex2(mo[r] - base_o);
                mo[r] = mo_new;
#pragma unroll
                for (int n = 0; n < SN; ++n) {
                    const float a = s[n][2 * r], b = s[n][2 * r + 1], v = ve[n >= SN / 2] - base_o;
                    sum += ex2(a - base) + ex2(b - base);
                    s[n][2 * r] = ex2(a + v);
                    s[n][2 * r + 1] = ex2(b + v);
                }
            } else {
                f_o[r] = f;
                mo[r] = m_new;
#pragma unroll
                for (int n = 0; n < SN; ++n) {
                    s[n][2 * r] = ex2(s[n][2 * r] - base);
                    s[n][2 * r + 1] = ex2(s[n][2 * r + 1] - base);
                    sum += s[n][2 * r] + s[n][2 * r + 1];
                }
            }
            m[r] = m_new;
            l[r] = l[r] * f + sum;
        }
#pragma unroll
        for (int n = 0; n < SN; ++n) {
            pa[n >> 1][(n & 1) * 2] = pack<kE4m3>(s[n][0], s[n][1]);
            pa[n >> 1][(n & 1) * 2 + 1] = pack<kE4m3>(s[n][2], s[n][3]);
        }
        if (__any_sync(kFull, f_o[0] != 1.0f || f_o[1] != 1.0f)) {
#pragma unroll
            for (int n = 0; n < S::NT; ++n) o[n][0] *= f_o[0], o[n][1] *= f_o[0], o[n][2] *= f_o[1], o[n][3] *= f_o[1];
        }
        // ---- values: lane g takes columns g * NT .. + NT - 1 of four keys; column tile
        // n of the MMA is column g * NT + n, so a lane ends with columns
        // (2 c) NT + n and (2 c + 1) NT + n
        if (!all) {
            // Values at masked keys may be NaN or infinite (unwritten slots), and 0 times
            // them is not 0. Keys that no row sees become 0; where another key's value is
            // not finite it is taken out and added for the rows that see it.
            bool bad = false;
            for (int x = lane * 16; x < S::TILE; x += 512) {
                const int n = x / S::ROW, key = key0 + n;
                uint4* at = reinterpret_cast<uint4*>(sv + x);
                if (key < t_lo || key >= k_hi || (n >= KEYS / 2 ? id1 : id0) < 0) {
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
            if (__any_sync(kFull, bad)) {
                const int elems = KEYS * D;
                for (int e0 = 0; e0 < elems; e0 += 32) {
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
                        // the weight of (row, key) is held by the lanes of that row with c = key % 8 / 2
#pragma unroll
                        for (int n = 0; n < SN; ++n) {
                            if (n != key / 8) continue;
                            const float w0 = key & 1 ? s[n][1] : s[n][0], w1 = key & 1 ? s[n][3] : s[n][2];
                            const int from = (lane & ~3) | ((key & 7) >> 1);
                            const float a0 = __shfl_sync(kFull, w0, from), a1 = __shfl_sync(kFull, w1, from);
#pragma unroll
                            for (int y = 0; y < S::NT; ++y)
#pragma unroll
                                for (int z = 0; z < 2; ++z)
                                    if (col == (2 * c + z) * S::NT + y) {
                                        if (key0 + key >= lo[0] && key0 + key <= hi[0]) o[y][z] += a0 * v;
                                        if (key0 + key >= lo[1] && key0 + key <= hi[1]) o[y][2 + z] += a1 * v;
                                    }
                        }
                    }
                }
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // before a later copy into this slot
            __syncwarp();
        }
#pragma unroll
        for (int x = 0; x < KEYS / 16; ++x) {
            constexpr int WORDS = S::NT * S::EB / 4;  // of a lane's columns of one key
            uint32_t v[4][WORDS];
            const uint8_t* base = sv + (16 * x + 2 * c) * S::ROW + g * S::NT * S::EB;
            lds(base, v[0]);
            lds(base + S::ROW, v[1]);
            lds(base + 8 * S::ROW, v[2]);
            lds(base + 9 * S::ROW, v[3]);
#pragma unroll
            for (int y = 0; y < WORDS; ++y) {
                if constexpr (kE4m3) {
                    // (a0 b0 a1 b1), (a2 b2 a3 b3) of keys a, b
                    const uint32_t p0 = __byte_perm(v[0][y], v[1][y], 0x5140), p1 = __byte_perm(v[0][y], v[1][y], 0x7362);
                    const uint32_t q0 = __byte_perm(v[2][y], v[3][y], 0x5140), q1 = __byte_perm(v[2][y], v[3][y], 0x7362);
                    mma16816<true>(o[4 * y], pa[x], f16x2_of(p0), f16x2_of(q0));
                    mma16816<true>(o[4 * y + 1], pa[x], f16x2_of(p0 >> 16), f16x2_of(q0 >> 16));
                    mma16816<true>(o[4 * y + 2], pa[x], f16x2_of(p1), f16x2_of(q1));
                    mma16816<true>(o[4 * y + 3], pa[x], f16x2_of(p1 >> 16), f16x2_of(q1 >> 16));
                } else {
                    mma16816<false>(o[2 * y], pa[x], __byte_perm(v[0][y], v[1][y], 0x5410), __byte_perm(v[2][y], v[3][y], 0x5410));
                    mma16816<false>(o[2 * y + 1], pa[x], __byte_perm(v[0][y], v[1][y], 0x7632), __byte_perm(v[2][y], v[3][y], 0x7632));
                }
            }
        }
    }
    // copies still in flight after a wait that gave up
    if (!ok && lane == 0) {
        const uint64_t t0 = global_ns();
        for (int i = max(0, ahead - STAGES); i < ahead; ++i) drain_wait(&full[i % STAGES], (uint32_t)(i / STAGES) & 1u, t0);
    }

    // ---- the four warps' results: sums relative to 2^mo, statistics
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        l[r] += __shfl_xor_sync(kFull, l[r], 1);
        l[r] += __shfl_xor_sync(kFull, l[r], 2);
    }
    __syncthreads();  // every warp has left its ring
    constexpr int LD = D + 4;
    float* jo = reinterpret_cast<float*>(smem) + warp * 16 * LD;
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        float* row = jo + (g + 8 * r) * LD;
#pragma unroll
        for (int z = 0; z < 2; ++z)
#pragma unroll
            for (int y = 0; y < S::NT; ++y) row[(2 * c + z) * S::NT + y] = o[y][2 * r + z];
        if (c == 0) *reinterpret_cast<float4*>(row + D) = make_float4(m[r], l[r], mo[r], 0.0f);
    }
    __syncthreads();
    if (*abort_flag) return;
    // 8 lanes per row: columns 4 x ..
    const int r = tid >> 3, x = tid & 7;
    if (r >= n_rows) return;
    const float* rows = reinterpret_cast<const float*>(smem) + r * LD;
    float4 st[kWarps];
    float M = neg_inf(), MO = neg_inf(), L = 0.0f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
        st[w] = *reinterpret_cast<const float4*>(rows + w * 16 * LD + D);
        M = fmaxf(M, st[w].x), MO = fmaxf(MO, st[w].z);
    }
    const float base = M == neg_inf() ? 0.0f : M, base_o = MO == neg_inf() ? 0.0f : MO;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
        L += st[w].y * ex2(st[w].x - base);
        st[w].w = ex2(st[w].z - base_o);
    }
    int rlo, rhi;
    seen_keys(p, it.s, (row0 + r) / G, rlo, rhi);
    const bool empty = rhi < rlo || (M == neg_inf() && L == 0.0f);  // (or none of its keys has a page)
    const int64_t t = it.s.q0 + (row0 + r) / G;
    const int hq = h * G + (row0 + r) % G;
    const int64_t at = (it.slot * p.Hkv + h) * kSplitRows + r;
    const float inv = empty ? 0.0f : ex2(base_o - base) / L;
    if (x == 0) {
        if (it.chunks > 1) reinterpret_cast<float4*>(p.part_s)[at] = make_float4(M, L, MO, 0.0f);
        else if (p.lse) p.lse[t * p.Hq + hq] = empty ? neg_inf() : (base + log2f(L)) * kLn2;
    }
    for (int d = 4 * x; d < D; d += 32) {
        float v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            const float4 q = *reinterpret_cast<const float4*>(rows + w * 16 * LD + d);
            v[0] = fmaf(q.x, st[w].w, v[0]), v[1] = fmaf(q.y, st[w].w, v[1]);
            v[2] = fmaf(q.z, st[w].w, v[2]), v[3] = fmaf(q.w, st[w].w, v[3]);
        }
        if (it.chunks > 1) {
            *reinterpret_cast<float4*>(p.part_o + at * D + d) = make_float4(v[0], v[1], v[2], v[3]);
        } else {
            __nv_bfloat16* out = const_cast<__nv_bfloat16*>(static_cast<const __nv_bfloat16*>(p.out.p)) + t * p.out.ts + hq * p.out.hs + d;
            *reinterpret_cast<uint2*>(out) = empty ? make_uint2(0, 0) : make_uint2(pack_bf16x2(v[0] * inv, v[1] * inv), pack_bf16x2(v[2] * inv, v[3] * inv));
        }
    }
}

template <bool kE4m3, int D>
cudaError_t split_as(const AttnProblem& p, cudaStream_t stream) {
    using S = Shape<kE4m3, D>;
    constexpr auto kernel = attn_split_kernel<kE4m3, D>;
    static DeviceOnce once;
    if (cudaError_t e = once.run([] { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, S::SMEM); });
        e != cudaSuccess)
        return e;
    const int64_t items = attn_items(p, kSplitRows);
    if (items * p.Hkv > INT32_MAX) return cudaErrorInvalidConfiguration;
    return launch_k(kernel, dim3((unsigned)(items * p.Hkv)), dim3(kThreads), S::SMEM, stream, p, tc_wait_limit_ns());
}

}  // namespace

bool attn_split_supported(const AttnProblem& p) {
    return p.act_dtype == GBMOE_BF16 && p.paged && (p.D == 64 || p.D == 96 || p.D == 128);
}

cudaError_t launch_attn_split(const AttnProblem& p, cudaStream_t stream) {
    if (p.e4m3) return p.D == 64 ? split_as<true, 64>(p, stream) : p.D == 96 ? split_as<true, 96>(p, stream) : split_as<true, 128>(p, stream);
    return p.D == 64 ? split_as<false, 64>(p, stream) : p.D == 96 ? split_as<false, 96>(p, stream) : split_as<false, 128>(p, stream);
}

}  // namespace gbmoe
