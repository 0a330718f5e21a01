// Attention on CUDA cores: fp32 activations, and head sizes that the
// tensor-core kernels do not take. Also the join of a split key axis.
//
// One pass over the keys with the running maximum and sum of the softmax: a
// block holds 32 tokens of one head (packed queries) or 16 rows, token and head
// of the group (cache), walks its keys in tiles of 32 through shared memory and
// keeps the weighted sum of values in registers. Bound by the
// fp32 pipes for prompts, by the latency of its loads for single tokens.
#include <climits>

#include "attn_plan.cuh"

namespace gbmoe {
namespace {

constexpr int kThreads = 128;
constexpr int kKeys = 32;

// Eight elements of key or value row `key` of sequence s, widened; a key whose
// page is outside the pool gives false.
template <typename TA, bool kE4m3, bool kPaged>
struct Source {
    const AttnProblem& p;
    const void* pool;
    const uint8_t* scales;
    Rows rows;
    int h, b;
    int64_t k0;

    __device__ __forceinline__ bool load(int key, int d, float (&v)[8]) const {
        if (!kPaged) {
            Vec8<TA>::load(static_cast<const TA*>(rows.p) + (k0 + key) * rows.ts + h * rows.hs + d, v);
            return true;
        }
        const int pg = key / p.page, id = p.page_table[(int64_t)b * p.max_pages + pg];
        if (id < 0 || id >= p.n_pages) return false;
        const int64_t head = (int64_t)id * p.Hkv + h;
        const int64_t at = (head * p.page + (key - pg * p.page)) * p.D + d;
        if constexpr (kE4m3) {
            const uint2 c = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(pool) + at);
            const float sc = e8m0_to_f32(scales[head]);
            const float2 a = e4m3x2_to_f32x2(c.x & 0xffffu), e = e4m3x2_to_f32x2(c.x >> 16);
            const float2 f = e4m3x2_to_f32x2(c.y & 0xffffu), g = e4m3x2_to_f32x2(c.y >> 16);
            v[0] = a.x * sc, v[1] = a.y * sc, v[2] = e.x * sc, v[3] = e.y * sc;
            v[4] = f.x * sc, v[5] = f.y * sc, v[6] = g.x * sc, v[7] = g.y * sc;
        } else {
            Vec8<TA>::load(static_cast<const TA*>(pool) + at, v);
        }
        return true;
    }
};

template <int DP>
constexpr int kLd = DP + 4;  // row length in shared memory
template <int DP, int N>
constexpr size_t kSmem = ((size_t)(2 * kKeys + 16 * N) * kLd<DP> + 16 * N * (kKeys + 1) + kKeys) * 4;

// DP: head size rounded up to 64, 128 or 256. N: rows of a thread, 2 (packed) or
// 1. Thread (ty, tx) = (tid / 8, tid % 8) holds rows N ty .., of the scores the
// keys tx + 8 j, of the result the columns 4 tx + 32 j ..; a row's eight threads
// lie in one warp.
template <typename TA, bool kE4m3, int DP, int N>
__device__ __forceinline__ void attend(const AttnProblem& p, const Segment& it) {
    constexpr int kRows = 16 * N;
    constexpr bool kPaged = N == 1;
    extern __shared__ float4 smem4[];
    float* sq = reinterpret_cast<float*>(smem4);
    float* sk = sq + kRows * kLd<DP>;
    float* sv = sk + kKeys * kLd<DP>;
    float* sp = sv + kKeys * kLd<DP>;
    int* ok = reinterpret_cast<int*>(sp + kRows * (kKeys + 1));
    const int G = p.Hq / p.Hkv, R = p.R;
    const int head0 = it.head * R;  // query head of row 0
    const int h = head0 / G;        // kv head
    const int row0 = it.tile * kRows;
    const int n_rows = (int)min64(kRows, (int64_t)it.s.nq * R - row0);
    // keys of the segment
    const int c_lo = (int)min64((int64_t)it.s.start + (int64_t)it.blk0 * kBlockKeys, it.s.len);
    const int c_hi = (int)min64((int64_t)it.s.start + (int64_t)it.blk1 * kBlockKeys, it.s.len);

    const int tid = threadIdx.x, ty = tid >> 3, tx = tid & 7;
    for (int i = tid; i < kRows * (DP / 8); i += kThreads) {
        const int r = i / (DP / 8), d = 8 * (i % (DP / 8));
        float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (r < n_rows && d < p.D)
            Vec8<TA>::load(static_cast<const TA*>(p.q.p) + (it.s.q0 + (row0 + r) / R) * p.q.ts + (head0 + (row0 + r) % R) * p.q.hs + d, v);
        Vec8<float>::store(sq + r * kLd<DP> + d, v);
    }
    int lo[N], hi[N];
#pragma unroll
    for (int r = 0; r < N; ++r) {
        lo[r] = 0, hi[r] = -1;
        if (N * ty + r < n_rows) seen_keys(p, it.s, (row0 + N * ty + r) / R, lo[r], hi[r]);
    }
    // keys that some row of the tile sees
    int k_lo, k_hi, last_lo, last_hi;
    seen_keys(p, it.s, row0 / R, k_lo, k_hi);
    seen_keys(p, it.s, (row0 + n_rows - 1) / R, last_lo, last_hi);
    if (k_hi < 0) k_lo = 0;
    k_lo = max(c_lo, k_lo), k_hi = min(c_hi, last_hi + 1);

    constexpr int NC = DP / 32;  // float4 columns of a thread
    float4 o[N][NC];
    float m[N], l[N];
#pragma unroll
    for (int r = 0; r < N; ++r) {
        m[r] = neg_inf(), l[r] = 0.0f;
#pragma unroll
        for (int c = 0; c < NC; ++c) o[r][c] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
    const Source<TA, kE4m3, kPaged> src_k{p, p.k_pool, p.k_scale, p.k, h, it.b, it.s.k0};
    const Source<TA, kE4m3, kPaged> src_v{p, p.v_pool, p.v_scale, p.v, h, it.b, it.s.k0};
    for (int k0 = k_lo; k0 < k_hi; k0 += kKeys) {
        __syncthreads();
        for (int i = tid; i < kKeys * (DP / 8); i += kThreads) {
            const int r = i / (DP / 8), d = 8 * (i % (DP / 8));
            float a[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, b[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            bool good = k0 + r < k_hi;
            if (good && d < p.D) good = src_k.load(k0 + r, d, a) && src_v.load(k0 + r, d, b);
            Vec8<float>::store(sk + r * kLd<DP> + d, a);
            Vec8<float>::store(sv + r * kLd<DP> + d, b);
            if (d == 0) ok[r] = good;
        }
        __syncthreads();
        float s[N][4] = {};
        for (int d = 0; d < p.D; d += 4) {
            float4 a[N], b[4];
#pragma unroll
            for (int r = 0; r < N; ++r) a[r] = *reinterpret_cast<const float4*>(sq + (N * ty + r) * kLd<DP> + d);
#pragma unroll
            for (int j = 0; j < 4; ++j) b[j] = *reinterpret_cast<const float4*>(sk + (tx + 8 * j) * kLd<DP> + d);
#pragma unroll
            for (int r = 0; r < N; ++r)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    s[r][j] = fmaf(a[r].x, b[j].x, fmaf(a[r].y, b[j].y, fmaf(a[r].z, b[j].z, fmaf(a[r].w, b[j].w, s[r][j]))));
        }
        bool all = true;  // this thread's rows see every key of the tile
#pragma unroll
        for (int r = 0; r < N; ++r) {
            float mx = neg_inf();
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int key = k0 + tx + 8 * j;
                const bool see = key >= lo[r] && key <= hi[r] && ok[tx + 8 * j];
                all &= see;
                s[r][j] = see ? s[r][j] * p.scale_log2 : neg_inf();
                mx = fmaxf(mx, s[r][j]);
            }
#pragma unroll
            for (int d = 1; d < 8; d <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
            const float m_new = fmaxf(m[r], mx);
            const float base = m_new == neg_inf() ? 0.0f : m_new;
            const float f = exp2f(m[r] - base);
            m[r] = m_new;
            float sum = 0.0f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                s[r][j] = exp2f(s[r][j] - base);
                sum += s[r][j];
                sp[(N * ty + r) * (kKeys + 1) + tx + 8 * j] = s[r][j];
            }
            l[r] = l[r] * f + sum;
#pragma unroll
            for (int c = 0; c < NC; ++c) o[r][c].x *= f, o[r][c].y *= f, o[r][c].z *= f, o[r][c].w *= f;
        }
        all = __all_sync(0xffffffffu, all);
        __syncwarp();
        // weights times values; a value that a row does not see is left out, not multiplied by 0 (it may be NaN)
        for (int j = 0; j < kKeys; ++j) {
            float w[N];
            bool see[N];
#pragma unroll
            for (int r = 0; r < N; ++r) {
                w[r] = sp[(N * ty + r) * (kKeys + 1) + j];
                see[r] = all || (k0 + j >= lo[r] && k0 + j <= hi[r]);
            }
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                const float4 v = *reinterpret_cast<const float4*>(sv + j * kLd<DP> + 4 * tx + 32 * c);
#pragma unroll
                for (int r = 0; r < N; ++r)
                    if (see[r]) {
                        o[r][c].x = fmaf(w[r], v.x, o[r][c].x), o[r][c].y = fmaf(w[r], v.y, o[r][c].y);
                        o[r][c].z = fmaf(w[r], v.z, o[r][c].z), o[r][c].w = fmaf(w[r], v.w, o[r][c].w);
                    }
            }
        }
    }
#pragma unroll
    for (int r = 0; r < N; ++r) {
#pragma unroll
        for (int d = 1; d < 8; d <<= 1) l[r] += __shfl_xor_sync(0xffffffffu, l[r], d);
        const int rr = N * ty + r;
        if (rr >= n_rows) continue;
        const int64_t t = it.s.q0 + (row0 + rr) / R;
        const int hq = head0 + (row0 + rr) % R;
        if (it.slot >= 0) {
            const int64_t at = it.slot * kRows + rr;
            if (tx == 0) reinterpret_cast<float4*>(p.part_s)[at] = make_float4(m[r], l[r], m[r], 0.0f);
#pragma unroll
            for (int c = 0; c < NC; ++c)
                if (4 * tx + 32 * c < p.D) *reinterpret_cast<float4*>(p.part_o + at * p.D + 4 * tx + 32 * c) = o[r][c];
            continue;
        }
        const bool empty = hi[r] < lo[r] || (kPaged && m[r] == neg_inf() && l[r] == 0.0f);  // (or none of its keys has a page)
        const float inv = empty ? 0.0f : 1.0f / l[r];
        if (p.lse && tx == 0) p.lse[t * p.Hq + hq] = empty ? neg_inf() : (m[r] + log2f(l[r])) * kLn2;
        TA* out = const_cast<TA*>(static_cast<const TA*>(p.out.p)) + t * p.out.ts + hq * p.out.hs;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int d = 4 * tx + 32 * c;
            if (d >= p.D) continue;
            const float v[4] = {o[r][c].x * inv, o[r][c].y * inv, o[r][c].z * inv, o[r][c].w * inv};
            if constexpr (sizeof(TA) == 4)
                *reinterpret_cast<float4*>(out + d) = make_float4(v[0], v[1], v[2], v[3]);
            else
                *reinterpret_cast<uint2*>(out + d) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
        }
    }
}

template <typename TA, bool kE4m3, int DP, int N>
__global__ void __launch_bounds__(kThreads) attn_simt_kernel(const AttnProblem p) {
    pdl_enter();
    __shared__ int64_t plan[plan_words(kThreads)];
    if constexpr (N == 1) {
        Walk<16> w;
        if (!w.begin(p, blockIdx.x, plan)) return;
        do {
            attend<TA, kE4m3, DP, N>(p, w.g);
            __syncthreads();
        } while (w.next(p));
    } else {
        Segment g{};
        g.head = blockIdx.x % p.Hq;
        const Place at = find_tile(p, blockIdx.x / p.Hq, 16 * N, plan);
        if (at.b < 0) return;
        g.b = at.b, g.s = load_seq(p, at.b), g.tile = (int)at.at;
        g.blk1 = key_blocks(g.s), g.slot = -1;
        attend<TA, kE4m3, DP, N>(p, g);
    }
}

template <typename TA, bool kE4m3, int DP, int N>
cudaError_t simt_as(const AttnProblem& p, cudaStream_t stream) {
    constexpr auto kernel = attn_simt_kernel<TA, kE4m3, DP, N>;
    static DeviceOnce once;
    if (cudaError_t e = once.run([] {
            return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmem<DP, N>);
        });
        e != cudaSuccess)
        return e;
    if constexpr (N == 1) {
        AttnProblem a = p;
        a.tile_rows = 16;
        a.shares = shares_of(p, 16, DP == 256 ? 2 : 4, sm_count());
        if (cudaError_t e = launch_k(kernel, dim3(a.shares), dim3(kThreads), kSmem<DP, N>, stream, a); e != cudaSuccess) return e;
        return a.shares > 1 ? launch_attn_join(a, stream) : cudaSuccess;
    } else {
        const int64_t grid = ((int64_t)p.T / (16 * N) + p.B) * p.Hq;
        if (grid > INT32_MAX) return cudaErrorInvalidConfiguration;
        return launch_k(kernel, dim3((unsigned)grid), dim3(kThreads), kSmem<DP, N>, stream, p);
    }
}

template <typename TA, bool kE4m3, int N>
cudaError_t simt_width(const AttnProblem& p, cudaStream_t stream) {
    if (p.D <= 64) return simt_as<TA, kE4m3, 64, N>(p, stream);
    if (p.D <= 128) return simt_as<TA, kE4m3, 128, N>(p, stream);
    return simt_as<TA, kE4m3, 256, N>(p, stream);
}

template <typename TA>
cudaError_t simt_source(const AttnProblem& p, cudaStream_t stream) {
    if (!p.paged) return simt_width<TA, false, 2>(p, stream);
    return p.e4m3 ? simt_width<TA, true, 1>(p, stream) : simt_width<TA, false, 1>(p, stream);
}

// ------------------------------------------------------------------- join
//
// Block x: where share x ends inside a tile that begins in it, that tile. The
// parts' sums, each relative to 2^(its own third statistic), are brought to the
// largest of those and added, the softmax sums likewise relative to the first
// statistic: out = sum / l. A row has as many of the eight warps as there are to
// spare, each adding every so many parts; the order is fixed by the lengths.
// The search for the tile reads only what the kernel before this launch's
// predecessor has written, so it runs before the wait for that one.
constexpr int kJoinThreads = 256, kJoinWarps = kJoinThreads / 32;

template <typename TA>
__global__ void __launch_bounds__(kJoinThreads) attn_join_kernel(const __grid_constant__ AttnProblem p) {
    __shared__ int64_t plan[plan_words(kJoinThreads)];
    __shared__ float4 acc[kJoinWarps][64];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, rows = p.tile_rows;
    Shares sh;
    const Place at = find_place(
        p.B, [&](int b) { const Seq s = load_seq(p, b); return row_tiles(p, s, rows) * key_blocks(s) * p.Hkv; },
        [&](int64_t total) { sh.set(p, total); return (blockIdx.x + 1) * sh.each; }, plan);
    Seq s{};
    int nb = 1, blk = 0, h = 0, tile = 0;
    if (at.b >= 0) {
        s = load_seq(p, at.b);
        nb = key_blocks(s);
        const int tiles = (int)row_tiles(p, s, rows);
        const int64_t ht = at.at / nb;
        blk = (int)(at.at - ht * nb);
        h = (int)(ht / tiles), tile = (int)(ht - (int64_t)h * tiles);
    }
    pdl_enter();
    if (blk == 0 || blk > sh.each) return;  // no tile, or it begins here, or before this share
    const int G = p.R;
    const int n_rows = (int)min64(rows, (int64_t)s.nq * G - (int64_t)tile * rows);
    const int per = n_rows <= 1 ? 8 : n_rows <= 2 ? 4 : n_rows <= 4 ? 2 : 1;  // warps of a row
    // parts: the end of this share, then the beginnings of the next ones
    const int64_t i0 = blockIdx.x;
    const int n = (int)((nb - blk + sh.each - 1) / sh.each) + 1;
    const int64_t first = blk == sh.each ? 2 * i0 : 2 * i0 + 1;  // (the tile may be all of this share)
    const float4* st = reinterpret_cast<const float4*>(p.part_s);
    for (int r0 = 0; r0 < n_rows; r0 += kJoinWarps / per) {
        const int r = r0 + warp / per, mine = warp % per;
        const bool have = r < n_rows;
        float m = neg_inf(), mo = neg_inf(), l = 0.0f;
        float o[2][4] = {};
        float base = 0.0f, base_o = 0.0f;
        const int d = 4 * lane;
        if (have) {
            auto slot = [&](int c) { return (c > 0 ? 2 * (i0 + c) : first) * rows + r; };
            for (int c = lane; c < n; c += 32) {
                const float4 v = __ldcg(st + slot(c));
                m = fmaxf(m, v.x), mo = fmaxf(mo, v.z);
            }
#pragma unroll
            for (int e = 16; e; e >>= 1) {
                m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, e));
                mo = fmaxf(mo, __shfl_xor_sync(0xffffffffu, mo, e));
            }
            base = m == neg_inf() ? 0.0f : m, base_o = mo == neg_inf() ? 0.0f : mo;
            for (int c0 = 0; c0 < n; c0 += 32) {
                float f = 0.0f;
                if (c0 + lane < n) {
                    const float4 v = __ldcg(st + slot(c0 + lane));
                    l += v.y * exp2f(v.x - base);
                    f = exp2f(v.z - base_o);
                }
                const int k = min(32, n - c0);
                for (int c = mine; c < k; c += 8 * per) {  // eight parts' loads in flight
                    float4 v[8][2];
                    float w[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int cc = c + i * per;
                        w[i] = __shfl_sync(0xffffffffu, f, min(cc, k - 1));
                        const float* src = p.part_o + slot(c0 + min(cc, k - 1)) * p.D + d;
#pragma unroll
                        for (int z = 0; z < 2; ++z)
                            v[i][z] = cc < k && d + 128 * z < p.D ? __ldcg(reinterpret_cast<const float4*>(src + 128 * z))
                                                                  : make_float4(0.f, 0.f, 0.f, 0.f);
                    }
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        if (c + i * per >= k || w[i] == 0.0f) continue;  // (a part that this row does not see: its sums are 0)
#pragma unroll
                        for (int z = 0; z < 2; ++z) {
                            o[z][0] = fmaf(v[i][z].x, w[i], o[z][0]), o[z][1] = fmaf(v[i][z].y, w[i], o[z][1]);
                            o[z][2] = fmaf(v[i][z].z, w[i], o[z][2]), o[z][3] = fmaf(v[i][z].w, w[i], o[z][3]);
                        }
                    }
                }
            }
#pragma unroll
            for (int e = 16; e; e >>= 1) l += __shfl_xor_sync(0xffffffffu, l, e);
        }
        if (per > 1) {
            __syncthreads();
#pragma unroll
            for (int z = 0; z < 2; ++z) acc[warp][lane + 32 * z] = make_float4(o[z][0], o[z][1], o[z][2], o[z][3]);
            __syncthreads();
            if (mine == 0)
                for (int w = 1; w < per; ++w)
#pragma unroll
                    for (int z = 0; z < 2; ++z) {
                        const float4 v = acc[warp + w][lane + 32 * z];
                        o[z][0] += v.x, o[z][1] += v.y, o[z][2] += v.z, o[z][3] += v.w;
                    }
        }
        if (!have || mine != 0) continue;
        const int64_t row = (int64_t)tile * rows + r;
        int lo, hi;
        seen_keys(p, s, (int)(row / G), lo, hi);
        const bool empty = hi < lo || (m == neg_inf() && l == 0.0f);
        const int64_t t = s.q0 + row / G;
        const int hq = h * G + (int)(row % G);
        if (p.lse && lane == 0) p.lse[t * p.Hq + hq] = empty ? neg_inf() : (base + log2f(l)) * kLn2;
        const float inv = empty ? 0.0f : exp2f(base_o - base) / l;
        TA* out = const_cast<TA*>(static_cast<const TA*>(p.out.p)) + t * p.out.ts + hq * p.out.hs + d;
#pragma unroll
        for (int z = 0; z < 2; ++z) {
            if (d + 128 * z >= p.D) break;
            if constexpr (sizeof(TA) == 4)
                *reinterpret_cast<float4*>(out + 128 * z) = make_float4(o[z][0] * inv, o[z][1] * inv, o[z][2] * inv, o[z][3] * inv);
            else
                *reinterpret_cast<uint2*>(out + 128 * z) =
                    make_uint2(pack_bf16x2(o[z][0] * inv, o[z][1] * inv), pack_bf16x2(o[z][2] * inv, o[z][3] * inv));
        }
    }
}

}  // namespace

cudaError_t launch_attn_simt(const AttnProblem& p, cudaStream_t stream) {
    return p.act_dtype == GBMOE_F32 ? simt_source<float>(p, stream) : simt_source<__nv_bfloat16>(p, stream);
}

cudaError_t launch_attn_join(const AttnProblem& p, cudaStream_t stream) {
    const dim3 grid(p.shares - 1);
    return p.act_dtype == GBMOE_F32 ? launch_k(attn_join_kernel<float>, grid, dim3(kJoinThreads), 0, stream, p)
                                    : launch_k(attn_join_kernel<__nv_bfloat16>, grid, dim3(kJoinThreads), 0, stream, p);
}

}  // namespace gbmoe
