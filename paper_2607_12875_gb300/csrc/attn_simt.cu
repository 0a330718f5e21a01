// Attention on CUDA cores: fp32 activations, and head sizes that the
// tensor-core kernels do not take. Also the join of a split key axis.
//
// One pass over the keys with the running maximum and sum of the softmax: a
// block holds 32 tokens of one head (packed queries; tiles of 16 took 25 us
// against 20 for 333 tokens of 16 heads of 64) or 16 rows, token and head of the
// group (cache), walks its keys in tiles of 32 through shared memory and keeps
// the weighted sum of values in registers. Bound by shared-memory wavefronts for
// long prompts (1200 tokens of 16 heads of 64 in 0.2 ms, 15 TFLOP/s: 70 % of their
// rate, ends of the grid included), by too few warps for short ones (333 tokens:
// 208 blocks, 8 % of an SM's warps, 21 % of that rate, 19 us), by the latency of its
// loads for single tokens.
#include <atomic>
#include <type_traits>

#include "attn_plan.cuh"

namespace gbmoe {
namespace {

constexpr int kThreads = 128;
constexpr int kKeys = 32;
// Cached: shares of one block of 64 keys (11 sequences of up to 518 keys, 4 kv heads of 64, e4m3:
// 18 us, with 2: 24), which take so long that a tile's set-up counts for nothing.
constexpr int kMinBlocks = 1, kTileCost = 0;

// Eight elements of a key or value row as loaded (several loads in flight), and
// their scale; good: false where the key's page is outside the pool.
template <typename TA, bool kE4m3>
struct Piece {
    uint4 v[kE4m3 ? 1 : sizeof(TA) / 2];
    float sc;
    bool good;
    __device__ __forceinline__ void widen(float (&x)[8]) const {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = 0.0f;
        if (!good) return;
        if constexpr (kE4m3) {
            const float2 a = e4m3x2_to_f32x2(v[0].x & 0xffffu), b = e4m3x2_to_f32x2(v[0].x >> 16);
            const float2 c = e4m3x2_to_f32x2(v[0].y & 0xffffu), d = e4m3x2_to_f32x2(v[0].y >> 16);
            x[0] = a.x * sc, x[1] = a.y * sc, x[2] = b.x * sc, x[3] = b.y * sc;
            x[4] = c.x * sc, x[5] = c.y * sc, x[6] = d.x * sc, x[7] = d.y * sc;
        } else if constexpr (sizeof(TA) == 4) {
            const uint32_t w[8] = {v[0].x, v[0].y, v[0].z, v[0].w, v[1].x, v[1].y, v[1].z, v[1].w};
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(w[i]);
        } else {
            const uint32_t w[4] = {v[0].x, v[0].y, v[0].z, v[0].w};
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = i & 1 ? bf16hi(w[i >> 1]) : bf16lo(w[i >> 1]);
        }
    }
};

// Key or value rows of sequence b: packed rows, or the pool's.
template <typename TA, bool kE4m3, bool kPaged>
struct Source {
    const AttnProblem& p;
    const void* pool;
    const uint8_t* scales;
    Rows rows;
    int h, b;
    int64_t k0;

    __device__ __forceinline__ void load(int key, int d, Piece<TA, kE4m3>& x) const {
        x.good = true;
        x.sc = 1.0f;
        const void* src;
        if (!kPaged) {
            src = static_cast<const TA*>(rows.p) + (k0 + key) * rows.ts + h * rows.hs + d;
        } else {
            const int id = p.page_table[(int64_t)b * p.max_pages + (key >> p.page_log2)];
            x.good = id >= 0 && id < p.n_pages;
            if (!x.good) return;
            const int64_t head = (int64_t)id * p.Hkv + h;
            const int64_t at = (head * p.page + (key & (p.page - 1))) * p.D + d;
            if constexpr (kE4m3) x.sc = e8m0_to_f32(scales[head]);
            src = static_cast<const char*>(pool) + at * (kE4m3 ? 1 : (int)sizeof(TA));
        }
        if constexpr (kE4m3) {
            const uint2 c = *static_cast<const uint2*>(src);
            x.v[0].x = c.x, x.v[0].y = c.y;
        } else {
#pragma unroll
            for (int i = 0; i < (int)sizeof(TA) / 2; ++i) x.v[i] = static_cast<const uint4*>(src)[i];
        }
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
    // A thread's pieces of a tile: rows (tid + 128 i) / (DP / 8). Up to head sizes of 128
    // the next tile's are in flight while this one is computed (beyond, the registers are short).
    constexpr int PIECES = kKeys * (DP / 8) / kThreads;
    constexpr bool kAhead = DP <= 128;
    Piece<TA, kE4m3> pk[PIECES], pv[PIECES];
    auto load = [&](int k0) {
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int x = tid + kThreads * i, r = x / (DP / 8), d = 8 * (x % (DP / 8));
            pk[i].good = pv[i].good = false;
            if (k0 + r >= k_hi || d >= p.D) continue;
            src_k.load(k0 + r, d, pk[i]);
            src_v.load(k0 + r, d, pv[i]);
        }
    };
    if (kAhead && k_lo < k_hi) load(k_lo);
    for (int k0 = k_lo; k0 < k_hi; k0 += kKeys) {
        __syncthreads();
        if (!kAhead) load(k0);
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int x = tid + kThreads * i, r = x / (DP / 8), d = 8 * (x % (DP / 8));
            float a[8];
            pk[i].widen(a);
            Vec8<float>::store(sk + r * kLd<DP> + d, a);
            pv[i].widen(a);
            Vec8<float>::store(sv + r * kLd<DP> + d, a);
            if (d == 0) ok[r] = pk[i].good;
        }
        __syncthreads();
        if (kAhead && k0 + kKeys < k_hi) load(k0 + kKeys);
        if (N * 4 * (tid >> 5) >= n_rows) continue;  // no row of this warp
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
        auto products = [&](auto masked) {
#pragma unroll 4
            for (int j = 0; j < kKeys; ++j) {
                float w[N];
#pragma unroll
                for (int r = 0; r < N; ++r) w[r] = sp[(N * ty + r) * (kKeys + 1) + j];
#pragma unroll
                for (int c = 0; c < NC; ++c) {
                    const float4 v = *reinterpret_cast<const float4*>(sv + j * kLd<DP> + 4 * tx + 32 * c);
#pragma unroll
                    for (int r = 0; r < N; ++r) {
                        if (decltype(masked)::value && !(k0 + j >= lo[r] && k0 + j <= hi[r])) continue;
                        o[r][c].x = fmaf(w[r], v.x, o[r][c].x), o[r][c].y = fmaf(w[r], v.y, o[r][c].y);
                        o[r][c].z = fmaf(w[r], v.z, o[r][c].z), o[r][c].w = fmaf(w[r], v.w, o[r][c].w);
                    }
                }
            }
        };
        if (all) products(std::false_type{});
        else products(std::true_type{});
    }
#pragma unroll
    for (int r = 0; r < N; ++r) {
#pragma unroll
        for (int d = 1; d < 8; d <<= 1) l[r] += __shfl_xor_sync(0xffffffffu, l[r], d);
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
                if (4 * tx + 32 * c < p.D) *reinterpret_cast<float4*>(p.part_o + at * p.D + 4 * tx + 32 * c) = o[r][c];
            continue;
        }
        const bool empty = hi[r] < lo[r] || !sees;
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
        if (!w.begin(p, blockIdx.x, plan)) {
            if (threadIdx.x == 0) w.note_idle(p, blockIdx.x);
            return;
        }
        do {
            attend<TA, kE4m3, DP, N>(p, w.g);
            if (threadIdx.x == 0) w.note(p);
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
    static std::atomic<int> per_sm;  // CTAs
    if (cudaError_t e = once.run([] {
            if (cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmem<DP, N>); e != cudaSuccess)
                return e;
            int n = 1;
            const cudaError_t e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kernel, kThreads, kSmem<DP, N>);
            per_sm.store(n, std::memory_order_relaxed);
            return e;
        });
        e != cudaSuccess)
        return e;
    if constexpr (N == 1) {
        AttnProblem a = p;
        set_shares(a, 16, per_sm.load(std::memory_order_relaxed), sm_count(), kMinBlocks, kTileCost);
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
// Rows of tiles that were cut. The parts' sums, each relative to 2^(its own third
// statistic), are brought to the largest of those and added, the softmax sums
// likewise relative to the first statistic: out = sum / l. (The fourth: 0 where the
// row sees no key of the part.) Every block counts the
// rows of all cut tiles for itself and takes its share of them, 1 to 8 at a time
// and then with 8 to 1 warps for a row, which take every so many of its parts: the
// order is fixed by the lengths. (A block for each share, most of them with
// nothing to join, cost 2 ns a block.)
constexpr int kJoinThreads = 256, kJoinWarps = kJoinThreads / 32, kJoinChunks = 3;
static_assert(kMaxShares <= kJoinThreads * kJoinChunks && kJoinWarps * kJoinChunks <= 32, "shares that a block counts");

// Z: groups of 128 columns, of which a lane takes four each; kFly: parts whose loads are in flight
template <typename TA, int Z>
__global__ void __launch_bounds__(kJoinThreads) attn_join_kernel(const __grid_constant__ AttnProblem p) {
    pdl_enter();
    constexpr int kFly = Z > 2 ? 4 : 8;
    __shared__ float4 acc[kJoinWarps][32 * Z];
    __shared__ int pre[kJoinThreads * kJoinChunks], sums[kJoinWarps * kJoinChunks];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    // rows of the cut tiles: running sums over 32 shares, sums of those
    int2 rec[kJoinChunks];
#pragma unroll
    for (int c = 0; c < kJoinChunks; ++c) {
        const int i = c * kJoinThreads + threadIdx.x;
        rec[c] = i < p.shares - 1 ? __ldcg(reinterpret_cast<const int2*>(p.cuts + i)) : make_int2(0, 0);
    }
#pragma unroll
    for (int c = 0; c < kJoinChunks; ++c) {
        int v = rec[c].x > 0 ? rec[c].y : 0;
#pragma unroll
        for (int e = 1; e < 32; e <<= 1) {
            const int u = __shfl_up_sync(0xffffffffu, v, e);
            if (lane >= e) v += u;
        }
        pre[c * kJoinThreads + threadIdx.x] = v;
        if (lane == 31) sums[c * kJoinWarps + warp] = v;
    }
    __syncthreads();
    int upto = lane < kJoinWarps * kJoinChunks ? sums[lane] : 0;
    const int own = upto;
#pragma unroll
    for (int e = 1; e < 32; e <<= 1) {
        const int u = __shfl_up_sync(0xffffffffu, upto, e);
        if (lane >= e) upto += u;
    }
    const int total = __shfl_sync(0xffffffffu, upto, 31), grid = gridDim.x;
    const int at_once = total > 4 * grid ? 8 : total > 2 * grid ? 4 : total > grid ? 2 : 1;  // rows
    const int W = kJoinWarps / at_once, in = warp / W, part = warp % W;                     // warps of a row
    for (int q0 = blockIdx.x * at_once; q0 < total; q0 += grid * at_once) {
        const int q = q0 + in;
        const bool have = q < total;
        int d = 4 * lane, n = 0;
        float m = neg_inf(), mo = neg_inf(), l = 0.0f, base = 0.0f, base_o = 0.0f;
        float o[Z][4] = {};
        int4 c0 = make_int4(0, 0, 0, 0), c1 = c0;
        int r = 0;
        bool sees = true;
        if (have) {
            const int chunk = __ffs(__ballot_sync(0xffffffffu, q < upto)) - 1;
            r = q - __shfl_sync(0xffffffffu, upto - own, chunk);
            const int run = pre[32 * chunk + lane];
            const int at = __ffs(__ballot_sync(0xffffffffu, r < run)) - 1;
            const int before = __shfl_sync(0xffffffffu, run, max(at - 1, 0));
            if (at > 0) r -= before;
            const int share = 32 * chunk + at;
            const int4* rec4 = reinterpret_cast<const int4*>(p.cuts + share);
            c0 = __ldcg(rec4), c1 = __ldcg(rec4 + 1);
            n = c0.x;
            const int rows = p.tile_rows, first = c0.z;
            const float4* st = reinterpret_cast<const float4*>(p.part_s);
            auto slot = [&](int c) { return (c > 0 ? 2 * ((int64_t)share + c) : first) * rows + r; };
            float4 mine = make_float4(neg_inf(), 0.0f, neg_inf(), 0.0f);  // of part `lane`
            if (lane < n) mine = __ldcg(st + slot(lane));
            m = mine.x, mo = mine.z;
            for (int c = lane + 32; c < n; c += 32) {
                const float4 v = __ldcg(st + slot(c));
                m = fmaxf(m, v.x), mo = fmaxf(mo, v.z);
            }
#pragma unroll
            for (int e = 16; e; e >>= 1) {
                m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, e));
                mo = fmaxf(mo, __shfl_xor_sync(0xffffffffu, mo, e));
            }
            base = m == neg_inf() ? 0.0f : m, base_o = mo == neg_inf() ? 0.0f : mo;
            for (int g0 = 0; g0 < n; g0 += 32) {
                if (g0 > 0) {
                    mine = make_float4(neg_inf(), 0.0f, neg_inf(), 0.0f);
                    if (g0 + lane < n) mine = __ldcg(st + slot(g0 + lane));
                }
                l += mine.y * exp2f(mine.x - base);
                const float f = exp2f(mine.z - base_o);
                const int k = min(32, n - g0);
                for (int c = part; c < k; c += kFly * W) {
                    float4 v[kFly][Z];
                    float w[kFly];
#pragma unroll
                    for (int i = 0; i < kFly; ++i) {
                        const int cc = c + W * i;
                        w[i] = __shfl_sync(0xffffffffu, f, min(cc, k - 1));
                        const float* src = p.part_o + slot(g0 + min(cc, k - 1)) * p.D + d;
#pragma unroll
                        for (int z = 0; z < Z; ++z)
                            v[i][z] = cc < k && d + 128 * z < p.D ? __ldcg(reinterpret_cast<const float4*>(src + 128 * z))
                                                                  : make_float4(0.f, 0.f, 0.f, 0.f);
                    }
#pragma unroll
                    for (int i = 0; i < kFly; ++i) {
                        if (c + W * i >= k) continue;  // (a part that this row does not see: its sums are 0)
#pragma unroll
                        for (int z = 0; z < Z; ++z) {
                            o[z][0] = fmaf(v[i][z].x, w[i], o[z][0]), o[z][1] = fmaf(v[i][z].y, w[i], o[z][1]);
                            o[z][2] = fmaf(v[i][z].z, w[i], o[z][2]), o[z][3] = fmaf(v[i][z].w, w[i], o[z][3]);
                        }
                    }
                }
            }
#pragma unroll
            for (int e = 16; e; e >>= 1) l += __shfl_xor_sync(0xffffffffu, l, e);
            if (m == neg_inf() && l == 0.0f) {  // no score above -inf: whether a part saw a key
                sees = false;
                for (int c = lane; c < n; c += 32) sees = sees || __ldcg(st + slot(c)).w != 0.0f;
                sees = __any_sync(0xffffffffu, sees);
            }
        }
        if (W > 1) {  // (uniform)
            if (q0 != blockIdx.x * at_once) __syncthreads();  // the rows before are done with acc
#pragma unroll
            for (int z = 0; z < Z; ++z) acc[warp][lane + 32 * z] = make_float4(o[z][0], o[z][1], o[z][2], o[z][3]);
            __syncthreads();
        }
        if (!have || part > 0) continue;
        const int G = p.R, row = c1.x * p.tile_rows + r;
        Seq s{};
        s.q0 = c1.y, s.nq = c1.z, s.len = c1.w;
        int lo, hi;
        seen_keys(p, s, row / G, lo, hi);
        const bool empty = hi < lo || !sees;
        const int64_t t = s.q0 + row / G;
        const int hq = c0.w * G + row % G;
        if (p.lse && lane == 0) p.lse[t * p.Hq + hq] = empty ? neg_inf() : (base + log2f(l)) * kLn2;
        const float inv = empty ? 0.0f : exp2f(base_o - base) / l;
        TA* out = const_cast<TA*>(static_cast<const TA*>(p.out.p)) + t * p.out.ts + hq * p.out.hs + d;
#pragma unroll
        for (int z = 0; z < Z; ++z) {
            if (d + 128 * z >= p.D) break;
            float y[4] = {o[z][0], o[z][1], o[z][2], o[z][3]};
            for (int w = 1; w < W; ++w) {
                const float4 v = acc[warp + w][lane + 32 * z];
                y[0] += v.x, y[1] += v.y, y[2] += v.z, y[3] += v.w;
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) y[i] *= inv;
            if constexpr (sizeof(TA) == 4) *reinterpret_cast<float4*>(out + 128 * z) = make_float4(y[0], y[1], y[2], y[3]);
            else *reinterpret_cast<uint2*>(out + 128 * z) = make_uint2(pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]));
        }
    }
}

template <typename TA>
cudaError_t join_as(const AttnProblem& p, cudaStream_t stream) {
    // as many blocks as there may be rows, up to two on each SM (one or four: up to 2 us slower at 20)
    const int64_t rows = min64((int64_t)p.T * p.Hq, (int64_t)(p.shares - 1) * p.tile_rows);
    const dim3 grid((unsigned)min64(rows, 2 * sm_count()));
    auto as = [&](auto kernel) { return launch_k(kernel, grid, dim3(kJoinThreads), 0, stream, p); };
    return p.D > 256 ? as(attn_join_kernel<TA, 4>) : p.D > 128 ? as(attn_join_kernel<TA, 2>) : as(attn_join_kernel<TA, 1>);
}

}  // namespace

cudaError_t launch_attn_simt(const AttnProblem& p, cudaStream_t stream) {
    return p.act_dtype == GBMOE_F32 ? simt_source<float>(p, stream) : simt_source<__nv_bfloat16>(p, stream);
}

cudaError_t launch_attn_join(const AttnProblem& p, cudaStream_t stream) {
    return p.act_dtype == GBMOE_F32 ? join_as<float>(p, stream) : join_as<__nv_bfloat16>(p, stream);
}

}  // namespace gbmoe
