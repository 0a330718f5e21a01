// Latent attention on CUDA cores: fp32 activations, and sizes that the tensor-core
// kernels do not take. Both forms.
//
// One pass over the keys with the running maximum and sum of the softmax: a block
// holds 8 or 16 rows, token and head (absorbed), or 16 or 32 tokens of one head (expanded), walks
// its keys in tiles of 32 through two buffers in shared memory (cp.async) and keeps
// the weighted sums in registers. Absorbed: a tile's rows are keys and values at once.
// Bound by the latency of its loads and by shared-memory wavefronts of a few warps: 333 tokens of 8 heads (96 and 64
// elements) 15.4 us, 11 sequences of up to 500 keys, 8 heads of 256 + 32 elements 15.9 us (tiles of 16 rows, half of
// them empty, and shares of 64 keys: 27.5).
#include <type_traits>

#include "attn_plan.cuh"
#include "latent.h"
#include "tc_ptx.cuh"

namespace gbmoe {
namespace {

constexpr int kThreads = 128;
constexpr int kKeys = 32;
static_assert(4 * kKeys == kThreads, "four threads for a key");
constexpr int kBlock = kKeys, kMinBlocks = 1, kTileCost = 0;  // absorbed: shares of one tile at least

// 16 bytes global -> shared, or 16 bytes of zeros
__device__ __forceinline__ void cp_async_or_zero(void* dst, const void* src, bool good) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(tc::smem_u32(dst)), "l"(src), "r"(good ? 16 : 0) : "memory");
}

template <typename TA>
__device__ __forceinline__ float4 load4(const uint8_t* p) {
    if constexpr (sizeof(TA) == 4) return *reinterpret_cast<const float4*>(p);
    const uint2 u = *reinterpret_cast<const uint2*>(p);
    return make_float4(bf16lo(u.x), bf16hi(u.x), bf16lo(u.y), bf16hi(u.y));
}

// Shared memory: query rows, two buffers of key (and value) rows, weights, marks of
// keys whose page is in the pool. Rows lie an odd number of 16-byte pieces apart.
struct Sizes {
    int q_pitch, k_pitch, total;
};
__host__ __device__ constexpr Sizes sizes_of(int key, int value, int eb, int rows, int least = 0) {
    Sizes s{};
    s.q_pitch = ((key * eb / 16) | 1) * 16;
    s.k_pitch = (((key + value) * eb / 16) | 1) * 16;
    s.total = rows * s.q_pitch + 2 * kKeys * s.k_pitch + rows * (kKeys + 1) * 4 + 2 * kKeys * 4;
    if (s.total < least) s.total = least;
    return s;
}

// N: rows of a thread, 2 (expanded) or 1 (absorbed); TX: threads of its rows, 8 or 16
// (all in one warp); NC: its float4 columns. Thread (ty, tx) = (tid / TX, tid % TX)
// holds rows N ty .., of the scores the keys tx + TX j, of the result the columns 4 tx +
// 4 TX j .. KG: groups of 128 threads, with every KG-th tile of the keys and shared memory of their own, whose results
// the first one joins.
template <int N, int TX>
constexpr int kTileRows = kThreads / TX * N;
// bytes of what a group passes on
template <int N, int NC, int KG>
constexpr int kPart = KG > 1 ? N * (NC + 1) * kThreads * 16 : 0;
template <typename TA, int N, int TX, int NC, int KG>
__device__ __forceinline__ void attend(const LatentProblem& lp, const Segment& it) {
    constexpr int kRows = kTileRows<N, TX>, EB = sizeof(TA), JK = kKeys / TX;
    constexpr bool kPaged = N == 1;
    static_assert(KG == 1 || !kPaged, "groups of the expanded form");
    const AttnProblem& p = lp.a;
    extern __shared__ float4 smem4[];
    const Sizes sz = sizes_of(lp.K, kPaged ? 0 : p.D, EB, kRows, kPart<N, NC, KG>);
    const int group = KG == 1 ? 0 : threadIdx.x / kThreads;
    uint8_t* sq = reinterpret_cast<uint8_t*>(smem4) + group * sz.total;
    auto sync = [&] {  // of the group
        if constexpr (KG == 1) __syncthreads();
        else asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "n"(kThreads) : "memory");
    };
    uint8_t* skv = sq + kRows * sz.q_pitch;
    float* sp = reinterpret_cast<float*>(skv + 2 * kKeys * sz.k_pitch);
    int* marks = reinterpret_cast<int*>(sp + kRows * (kKeys + 1));
    const int R = p.R, head0 = kPaged ? 0 : it.head, row0 = it.tile * kRows;
    const int n_rows = (int)min64(kRows, (int64_t)it.s.nq * R - row0);
    const int c_lo = (int)min64((int64_t)it.blk0 * kBlock, it.s.len);
    const int c_hi = (int)min64((int64_t)it.blk1 * kBlock, it.s.len);

    const int tid = threadIdx.x % kThreads, ty = tid / TX, tx = tid % TX;
    const int qp = lp.K * EB / 16;  // pieces of a query
    for (int i = tid; i < kRows * qp; i += kThreads) {
        const int r = i / qp, c = i % qp;
        const bool good = r < n_rows;
        const int rr = row0 + (good ? r : 0);
        const TA* src = static_cast<const TA*>(p.q.p) + (it.s.q0 + rr / R) * p.q.ts + (head0 + rr % R) * p.q.hs;
        cp_async_or_zero(sq + r * sz.q_pitch + 16 * c, reinterpret_cast<const uint8_t*>(src) + 16 * c, good);
    }
    int lo[N], hi[N];
#pragma unroll
    for (int r = 0; r < N; ++r) {
        lo[r] = 0, hi[r] = -1;
        if (N * ty + r < n_rows) seen_keys(p, it.s, (row0 + N * ty + r) / R, lo[r], hi[r]);
    }
    // keys that some row of the tile sees
    int k_lo, last_hi;
    seen_keys(p, it.s, (row0 + n_rows - 1) / R, k_lo, last_hi);
    k_lo = c_lo + group * kKeys;
    const int k_hi = min(c_hi, last_hi + 1);

    // Four threads for a key's row, whose page is looked up a tile ahead.
    const int own = lp.own * EB / 16, key = lp.K * EB / 16, all_pieces = key + (kPaged ? 0 : p.D * EB / 16);
    const int lr = tid >> 2, lc = tid & 3;
    auto page_of = [&](int k0) {
        if (!kPaged || k0 + lr >= k_hi) return -1;
        const int id = p.page_table[(int64_t)it.b * p.max_pages + ((k0 + lr) >> p.page_log2)];
        return id >= 0 && id < p.n_pages ? id : -1;
    };
    int page = page_of(k_lo);
    auto load = [&](int k0, int buf) {
        const bool good = kPaged ? page >= 0 : k0 + lr < k_hi;
        uint8_t* dst = skv + (buf * kKeys + lr) * sz.k_pitch;
        if constexpr (kPaged) {
            const uint8_t* src = static_cast<const uint8_t*>(p.k_pool) +
                                 ((int64_t)max(page, 0) * p.page + ((k0 + lr) & (p.page - 1))) * lp.K * EB;
            for (int c = lc; c < key; c += 4) cp_async_or_zero(dst + 16 * c, good ? src + 16 * c : static_cast<const uint8_t*>(p.k_pool), good);
            if (lc == 0) marks[buf * kKeys + lr] = good;
            page = page_of(k0 + kKeys);
        } else {
            const int64_t at = it.s.k0 + (good ? k0 + lr : 0);
            const uint8_t* k = reinterpret_cast<const uint8_t*>(static_cast<const TA*>(p.k.p) + at * p.k.ts + it.head * p.k.hs);
            const uint8_t* r = reinterpret_cast<const uint8_t*>(static_cast<const TA*>(lp.k_rope.p) + at * lp.k_rope.ts);
            const uint8_t* v = reinterpret_cast<const uint8_t*>(static_cast<const TA*>(p.v.p) + at * p.v.ts + it.head * p.v.hs);
            for (int c = lc; c < all_pieces; c += 4)
                cp_async_or_zero(dst + 16 * c, c < own ? k + 16 * c : c < key ? r + 16 * (c - own) : v + 16 * (c - key), good);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };

    float4 o[N][NC];
    float m[N], l[N];
#pragma unroll
    for (int r = 0; r < N; ++r) {
        m[r] = neg_inf(), l[r] = 0.0f;
#pragma unroll
        for (int c = 0; c < NC; ++c) o[r][c] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
    if (k_lo < k_hi) load(k_lo, 0);
    int buf = 0;
    for (int k0 = k_lo; k0 < k_hi; k0 += KG * kKeys, buf ^= 1) {
        if (k0 + KG * kKeys < k_hi) {
            load(k0 + KG * kKeys, buf ^ 1);
            asm volatile("cp.async.wait_group 1;" ::: "memory");
        } else {
            asm volatile("cp.async.wait_group 0;" ::: "memory");
        }
        sync();
        const uint8_t* tile = skv + buf * kKeys * sz.k_pitch;
        if (N * (32 / TX) * (tid >> 5) < n_rows) {  // (else no row of this warp)
            float s[N][JK] = {};
            for (int d = 0; d < lp.K; d += 4) {
                float4 a[N], b[JK];
#pragma unroll
                for (int r = 0; r < N; ++r) a[r] = load4<TA>(sq + (N * ty + r) * sz.q_pitch + d * EB);
#pragma unroll
                for (int j = 0; j < JK; ++j) b[j] = load4<TA>(tile + (tx + TX * j) * sz.k_pitch + d * EB);
#pragma unroll
                for (int r = 0; r < N; ++r)
#pragma unroll
                    for (int j = 0; j < JK; ++j)
                        s[r][j] = fmaf(a[r].x, b[j].x, fmaf(a[r].y, b[j].y, fmaf(a[r].z, b[j].z, fmaf(a[r].w, b[j].w, s[r][j]))));
            }
            bool all = true;  // this thread's rows see every key of the tile
#pragma unroll
            for (int r = 0; r < N; ++r) {
                float mx = neg_inf();
#pragma unroll
                for (int j = 0; j < JK; ++j) {
                    const int k = k0 + tx + TX * j;
                    const bool see = k >= lo[r] && k <= hi[r] && k < k_hi && (!kPaged || marks[buf * kKeys + tx + TX * j]);
                    all &= see;
                    s[r][j] = see ? s[r][j] * p.scale_log2 : neg_inf();
                    mx = fmaxf(mx, s[r][j]);
                }
#pragma unroll
                for (int d = 1; d < TX; d <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
                const float m_new = fmaxf(m[r], mx);
                const float base = m_new == neg_inf() ? 0.0f : m_new;
                const float f = exp2f(m[r] - base);
                m[r] = m_new;
                float sum = 0.0f;
#pragma unroll
                for (int j = 0; j < JK; ++j) {
                    s[r][j] = exp2f(s[r][j] - base);
                    sum += s[r][j];
                    sp[(N * ty + r) * (kKeys + 1) + tx + TX * j] = s[r][j];
                }
                l[r] = l[r] * f + sum;
#pragma unroll
                for (int c = 0; c < NC; ++c) o[r][c].x *= f, o[r][c].y *= f, o[r][c].z *= f, o[r][c].w *= f;
            }
            all = __all_sync(0xffffffffu, all);
            __syncwarp();
            const uint8_t* values = tile + (kPaged ? 0 : lp.K * EB);
            // weights times values; a value that a row does not see is left out, not multiplied by 0 (it may be NaN)
            auto products = [&](auto masked) {
#pragma unroll 4
                for (int j = 0; j < kKeys; ++j) {
                    float w[N];
                    bool see[N];
#pragma unroll
                    for (int r = 0; r < N; ++r) {
                        w[r] = sp[(N * ty + r) * (kKeys + 1) + j];
                        see[r] = k0 + j >= lo[r] && k0 + j <= hi[r];
                    }
#pragma unroll
                    for (int c = 0; c < NC; ++c) {
                        const int d = 4 * tx + 4 * TX * c;
                        if (d >= p.D) break;
                        const float4 v = load4<TA>(values + j * sz.k_pitch + d * EB);
#pragma unroll
                        for (int r = 0; r < N; ++r) {
                            if (decltype(masked)::value && !see[r]) continue;
                            o[r][c].x = fmaf(w[r], v.x, o[r][c].x), o[r][c].y = fmaf(w[r], v.y, o[r][c].y);
                            o[r][c].z = fmaf(w[r], v.z, o[r][c].z), o[r][c].w = fmaf(w[r], v.w, o[r][c].w);
                        }
                    }
                }
            };
            if (all) products(std::false_type{});
            else products(std::true_type{});
        }
        sync();
    }
    if (k_lo >= k_hi) asm volatile("cp.async.wait_all;" ::: "memory");
#pragma unroll
    for (int r = 0; r < N; ++r)
#pragma unroll
        for (int d = 1; d < TX; d <<= 1) l[r] += __shfl_xor_sync(0xffffffffu, l[r], d);
    if constexpr (KG > 1) {
        // a thread's maxima, sums and results in its group's shared memory, a row of all threads' for each
        auto part = [&](int g, int i) { return reinterpret_cast<float4*>(reinterpret_cast<uint8_t*>(smem4) + g * sz.total) + i * kThreads + tid; };
        if (group > 0) {
            if (k_lo >= k_hi) sync();  // (the queries of all of the group's threads have landed)
#pragma unroll
            for (int r = 0; r < N; ++r) {
                *part(group, r) = make_float4(m[r], l[r], 0.f, 0.f);
#pragma unroll
                for (int c = 0; c < NC; ++c) *part(group, N + r * NC + c) = o[r][c];
            }
        }
        __syncthreads();
        if (group > 0) return;
#pragma unroll
        for (int g = 1; g < KG; ++g)
#pragma unroll
            for (int r = 0; r < N; ++r) {
                const float4 other = *part(g, r);
                const float m_new = fmaxf(m[r], other.x), base = m_new == neg_inf() ? 0.0f : m_new;
                const float a = exp2f(m[r] - base), b = exp2f(other.x - base);
                m[r] = m_new, l[r] = l[r] * a + other.y * b;
#pragma unroll
                for (int c = 0; c < NC; ++c) {
                    const float4 v = *part(g, N + r * NC + c);
                    o[r][c].x = o[r][c].x * a + v.x * b, o[r][c].y = o[r][c].y * a + v.y * b;
                    o[r][c].z = o[r][c].z * a + v.z * b, o[r][c].w = o[r][c].w * a + v.w * b;
                }
            }
    }
#pragma unroll
    for (int r = 0; r < N; ++r) {
        const int rr = N * ty + r;
        if (rr >= n_rows) continue;
        const int64_t t = it.s.q0 + (row0 + rr) / R;
        const int hq = head0 + (row0 + rr) % R;
        // Without a score above -inf: whether the row sees a key at all (if not it gives 0, else 0 / 0)
        const bool blank = m[r] == neg_inf() && l[r] == 0.0f;
        const bool sees = !kPaged || !blank || any_page(p, it.b, max(lo[r], c_lo), min(hi[r], c_hi - 1));
        if (it.slot >= 0) {
            const int64_t at = it.slot * kRows + rr;
            if (tx == 0) reinterpret_cast<float4*>(p.part_s)[at] = make_float4(m[r], l[r], m[r], sees ? 1.0f : 0.0f);
#pragma unroll
            for (int c = 0; c < NC; ++c)
                if (4 * tx + 4 * TX * c < p.D) *reinterpret_cast<float4*>(p.part_o + at * p.D + 4 * tx + 4 * TX * c) = o[r][c];
            continue;
        }
        const bool empty = hi[r] < lo[r] || !sees;
        const float inv = empty ? 0.0f : 1.0f / l[r];
        if (p.lse && tx == 0) p.lse[t * p.Hq + hq] = empty ? neg_inf() : (m[r] + log2f(l[r])) * kLn2;
        TA* out = const_cast<TA*>(static_cast<const TA*>(p.out.p)) + t * p.out.ts + hq * p.out.hs;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int d = 4 * tx + 4 * TX * c;
            if (d >= p.D) continue;
            const float v[4] = {o[r][c].x * inv, o[r][c].y * inv, o[r][c].z * inv, o[r][c].w * inv};
            if constexpr (EB == 4)
                *reinterpret_cast<float4*>(out + d) = make_float4(v[0], v[1], v[2], v[3]);
            else
                *reinterpret_cast<uint2*>(out + d) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
        }
    }
}

template <typename TA, int N, int TX, int NC, int KG>
__global__ void __launch_bounds__(KG* kThreads) latent_simt_kernel(const __grid_constant__ LatentProblem lp) {
    pdl_enter();
    const AttnProblem& p = lp.a;
    __shared__ int64_t plan[plan_words(KG * kThreads)];
    if constexpr (N == 1) {
        Walk<kTileRows<N, TX>, kBlock> w;
        if (!w.begin(p, blockIdx.x, plan)) {
            if (threadIdx.x == 0) w.note_idle(p, blockIdx.x);
            return;
        }
        do {
            attend<TA, N, TX, NC, KG>(lp, w.g);
            if (threadIdx.x == 0) w.note(p);
            __syncthreads();
        } while (w.next(p));
    } else {
        Segment g{};
        g.head = blockIdx.x % p.Hq;
        const Place at = find_tile(p, blockIdx.x / p.Hq, kTileRows<N, TX>, plan);
        if (at.b < 0) return;
        g.b = at.b, g.s = load_seq(p, at.b);
        g.tile = (int)(row_tiles(p, g.s, kTileRows<N, TX>) - 1 - at.at);  // the last tiles, which see the most keys, first
        g.blk1 = key_blocks<kBlock>(g.s), g.slot = -1;
        attend<TA, N, TX, NC, KG>(lp, g);
    }
}

template <typename TA, int N, int TX, int NC, int KG>
cudaError_t simt_as(const LatentProblem& p, cudaStream_t stream) {
    constexpr auto kernel = latent_simt_kernel<TA, N, TX, NC, KG>;
    constexpr int kRows = kTileRows<N, TX>;
    static DeviceOnce once;
    constexpr int kMost = 227 * 1024;
    if (cudaError_t e = once.run([] { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMost - 1024); });
        e != cudaSuccess)
        return e;
    const int smem = sizes_of(p.K, N == 1 ? 0 : p.a.D, (int)sizeof(TA), kRows, kPart<N, NC, KG>).total;
    if constexpr (N == 1) {
        LatentProblem a = p;
        const int fit = kMost / (smem + 2048);
        set_shares(a.a, kRows, fit < 1 ? 1 : fit > 4 ? 4 : fit, sm_count(), kMinBlocks, kTileCost, kBlock);
        if (cudaError_t e = launch_k(kernel, dim3(a.a.shares), dim3(kThreads), smem, stream, a); e != cudaSuccess) return e;
        return a.a.shares > 1 ? launch_attn_join(a.a, stream) : cudaSuccess;
    } else {
        // fewer groups where these do not fit (keys have up to 256 elements, values NC float4 of each thread)
        if constexpr (KG * sizes_of(256, 4 * TX * NC, (int)sizeof(TA), kRows, kPart<N, NC, KG>).total > kMost - 1024)
            if (KG * smem > kMost - 1024) return simt_as<TA, N, TX, NC, KG / 2>(p, stream);
        const int64_t grid = ((int64_t)p.a.T / kRows + p.a.B) * p.a.Hq;
        if (grid > INT32_MAX) return cudaErrorInvalidConfiguration;
        return launch_k(kernel, dim3((unsigned)grid), dim3(KG * kThreads), KG * smem, stream, p);
    }
}

template <typename TA>
cudaError_t simt_type(const LatentProblem& p, cudaStream_t stream) {
    if (p.a.paged) {
        // eight rows where a sequence has no more, so that none of the warps stands idle
        const bool few = (int64_t)p.a.T * p.a.R <= 8 * (int64_t)p.a.B;
        if (p.a.D <= 256) return few ? simt_as<TA, 1, 16, 4, 1>(p, stream) : simt_as<TA, 1, 8, 8, 1>(p, stream);
        return few ? simt_as<TA, 1, 16, 8, 1>(p, stream) : simt_as<TA, 1, 8, 16, 1>(p, stream);
    }
    // Where 32 tokens for a block leave SMs without one: 16, and the keys dealt to four groups of threads. Us for 333 tokens
    // of 8 heads with 32 tokens 23.4; with 16 and one, two and four groups 20.2, 17.3 and 15.4.
    const bool few = ((int64_t)p.a.T / 32 + p.a.B) * p.a.Hq <= sm_count();
    if (p.a.D <= 64) return few ? simt_as<TA, 2, 16, 1, 4>(p, stream) : simt_as<TA, 2, 8, 2, 1>(p, stream);
    return few ? simt_as<TA, 2, 16, 2, 4>(p, stream) : simt_as<TA, 2, 8, 4, 1>(p, stream);
}

}  // namespace

cudaError_t launch_latent_simt(const LatentProblem& p, cudaStream_t stream) {
    return p.a.act_dtype == GBMOE_F32 ? simt_type<float>(p, stream) : simt_type<__nv_bfloat16>(p, stream);
}

}  // namespace gbmoe
