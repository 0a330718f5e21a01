// Rotary positions, and appending keys and values to the paged cache with the
// rotation on the way.
//
// Pair (a, b) number i of a head turns by position * f_i. The table holds f_i
// in turns as a binary fraction of 2^64, so the 64-bit product with the
// position, wrapped, is the fraction of a turn to 2^-64 * position, whatever
// the position; its top 32 bits go to sincospif (an error of 2^-25 half turns,
// below fp32's own on the rotated values). One block computes the angles of its
// tokens once, in shared memory, for all the heads that it turns.
//
// Both kernels are bound by HBM: each element is read once and written once
// (the append's second walk over its few KB hits the L1 cache).
#include <climits>

#include "attn_plan.cuh"

namespace gbmoe {
namespace {

constexpr int kRopeThreads = 256;

// (cos, sin) of pair i at position pos
__device__ __forceinline__ float2 turn(const RopeParams& r, int64_t pos, int i) {
    const uint64_t f = (uint64_t)pos * r.table[i];
    float s, c;
    sincospif((float)(int32_t)(f >> 32) * 4.656612873077393e-10f, &s, &c);  // 2^-31: half turns
    return make_float2(c * r.mag, s * r.mag * r.sin_sign);
}

// A unit of a head: for u < R / 16 the eight pairs 8u .. 8u+7, else eight
// elements that do not turn. Returns the offset of its second half (-1: none).
__device__ __forceinline__ int unit_offsets(const RopeParams& r, int u, int& first) {
    const int nr = r.R >> 4;
    if (u >= nr) {
        first = r.R + 8 * (u - nr);
        return -1;
    }
    first = r.half ? 8 * u : 16 * u;
    return r.half ? first + (r.R >> 1) : first + 8;
}
__device__ __forceinline__ int head_units(const RopeParams& r, int D) { return (r.R >> 4) + ((D - r.R) >> 3); }

// x (first half), y (second half) turned by the eight angles at cs
__device__ __forceinline__ void turn8(const RopeParams& r, const float2* cs, float (&x)[8], float (&y)[8]) {
    if (r.half) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float2 t = cs[j];
            const float a = x[j], b = y[j];
            x[j] = a * t.x - b * t.y;
            y[j] = a * t.y + b * t.x;
        }
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float2 t = cs[j], w = cs[j + 4];
            float a = x[2 * j], b = x[2 * j + 1];
            x[2 * j] = a * t.x - b * t.y;
            x[2 * j + 1] = a * t.y + b * t.x;
            a = y[2 * j], b = y[2 * j + 1];
            y[2 * j] = a * w.x - b * w.y;
            y[2 * j + 1] = a * w.y + b * w.x;
        }
    }
}

// unit u of a head: src turned to dst
template <typename TA>
__device__ __forceinline__ void turn_unit(const RopeParams& r, const float2* cs, int u, const TA* src, TA* dst) {
    int f;
    const int s = unit_offsets(r, u, f);
    float x[8];
    Vec8<TA>::load(src + f, x);
    if (s >= 0) {
        float y[8];
        Vec8<TA>::load(src + s, y);
        turn8(r, cs + 8 * u, x, y);
        Vec8<TA>::store(dst + s, y);
    }
    Vec8<TA>::store(dst + f, x);
}

template <typename TA>
__device__ __forceinline__ TA* row(const Rows& r, int64_t t, int h) {
    return const_cast<TA*>(static_cast<const TA*>(r.p)) + t * r.ts + h * r.hs;
}

// Block (x, y): tokens x * tokens .., heads y * heads .. of q and k together.
template <typename TA>
__global__ void __launch_bounds__(kRopeThreads) rope_kernel(const RopeProblem p, int tokens, int heads) {
    pdl_enter();
    extern __shared__ float2 cs[];
    const int t0 = blockIdx.x * tokens, nt = min(tokens, p.T - t0);
    const int h0 = blockIdx.y * heads, nh = min(heads, p.Hq + p.Hk - h0);
    const int pairs = p.r.R >> 1;
    for (int i = threadIdx.x; i < nt * pairs; i += kRopeThreads)
        cs[i] = turn(p.r, p.positions[t0 + i / pairs], i % pairs);
    __syncthreads();
    const int nu = head_units(p.r, p.D), per = nh * nu;
    for (int i = threadIdx.x; i < nt * per; i += kRopeThreads) {
        const int t = i / per, w = i - t * per, h = h0 + w / nu, u = w % nu;
        const bool is_q = h < p.Hq;
        const Rows& src = is_q ? p.q : p.k;
        const Rows& dst = is_q ? p.q_out : p.k_out;
        const int hh = is_q ? h : h - p.Hq;
        turn_unit<TA>(p.r, cs + t * pairs, u, row<TA>(src, t0 + t, hh), row<TA>(dst, t0 + t, hh));
    }
}

// ------------------------------------------------------------------ append

// Exponent of the smallest power of two 2^e (e >= -127) with amax <= 448 * 2^e
__device__ __forceinline__ int scale_exponent(float amax) {
    int x;
    const float m = frexpf(amax, &x);  // amax = m * 2^x, m in [0.5, 1); 448 = 0.875 * 2^9
    if (amax == 0.0f) return -127;
    return max(x - 9 + (m > 0.875f ? 1 : 0), -127);
}

// 2^e for e in -127 .. 127 (subnormal at -127)
__device__ __forceinline__ float pow2(int e) { return e > -127 ? __uint_as_float((uint32_t)(e + 127) << 23) : __uint_as_float(0x00400000u); }

// two fp32 -> two e4m3 bytes (low byte: a), nearest, ties to even, +-448 beyond
__device__ __forceinline__ uint32_t e4m3x2(float a, float b) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(b), "f"(a));
    return r;
}
__device__ __forceinline__ uint2 e4m3x8(const float (&v)[8], float s) {
    return make_uint2(e4m3x2(v[0] * s, v[1] * s) | e4m3x2(v[2] * s, v[3] * s) << 16,
                      e4m3x2(v[4] * s, v[5] * s) | e4m3x2(v[6] * s, v[7] * s) << 16);
}

__device__ __forceinline__ float max_finite(float m, const float (&v)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float a = fabsf(v[j]);
        m = a <= 3.402823466e38f ? fmaxf(m, a) : m;  // (false for NaN)
    }
    return m;
}

__device__ __forceinline__ float block_max(float m, float* sm) {
#pragma unroll
    for (int d = 16; d; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
    __syncthreads();
    if ((threadIdx.x & 31) == 0) sm[threadIdx.x >> 5] = m;
    __syncthreads();
    for (int w = 0; w < (int)(blockDim.x >> 5); ++w) m = fmaxf(m, sm[w]);
    return m;
}

// A segment: the new tokens of one sequence that fall into one of its pages.
struct Segment {
    int t0, n;      // its tokens
    int64_t pos;    // position of the first one in the sequence
    int page, off;  // pool page (-1: not stored) and slot of the first one
};

// Segment `index` (sequences in order, a sequence's pages in order), found by
// the whole block; sm holds warps + 4 words. n = 0: none.
__device__ Segment find_segment(const AppendProblem& p, int64_t index, int64_t* sm) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, nthr = blockDim.x;
    int64_t* found = sm + (nthr >> 5);
    if (tid == 0) found[0] = -1;
    auto bounds = [&](int b, int& q0, int& n, int64_t& pos0) {
        q0 = min(max(p.cu_q[b], 0), p.T);
        n = min(max(p.cu_q[b + 1], q0), p.T) - q0;
        pos0 = (int64_t)p.kv_len[b] - n;
    };
    auto page_of = [&](int64_t pos) { return pos >= 0 ? pos / p.page : -1 - (-1 - pos) / p.page; };
    int64_t before = 0;
    for (int base = 0; base < p.B; base += nthr) {
        const int b = base + tid;
        int64_t segs = 0;
        if (b < p.B) {
            int q0, n;
            int64_t pos0;
            bounds(b, q0, n, pos0);
            if (n > 0) segs = page_of(pos0 + n - 1) - page_of(pos0) + 1;
        }
        int64_t pre = segs;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int64_t a = __shfl_up_sync(0xffffffffu, pre, d);
            if (lane >= d) pre += a;
        }
        __syncthreads();
        if (lane == 31) sm[warp] = pre;
        __syncthreads();
        int64_t w0 = before;
        for (int w = 0; w < (nthr >> 5); ++w) {
            if (w < warp) w0 += sm[w];
            before += sm[w];
        }
        if (segs > 0 && index >= w0 + pre - segs && index < w0 + pre) {
            found[0] = b;
            found[1] = w0 + pre - segs;
        }
        __syncthreads();
        if (index < before) break;  // uniform
    }
    __syncthreads();
    Segment s{};
    const int b = (int)found[0];
    if (b < 0) return s;
    int q0, n;
    int64_t pos0;
    bounds(b, q0, n, pos0);
    const int64_t pg = page_of(pos0) + (index - found[1]);
    const int64_t from = max64(pos0, pg * p.page), to = min64(pos0 + n, (pg + 1) * p.page);
    s.t0 = q0 + (int)(from - pos0);
    s.n = (int)(to - from);
    s.pos = from;
    s.off = (int)(from - pg * p.page);
    s.page = -1;
    if (pg >= 0 && pg < p.max_pages) {
        const int id = p.page_table[(int64_t)b * p.max_pages + pg];
        if (id >= 0 && id < p.n_pages) s.page = id;
    }
    return s;
}

// The segment's rows of one head of k (kTurn) or v to the cache in e4m3.
template <typename TA, bool kTurn>
__device__ void append_e4m3(const AppendProblem& p, const RopeParams& r, const Segment& s, const float2* cs, const Rows& src,
                            int h, uint8_t* pool, uint8_t* scale, const Rows* out, float* sm) {
    const int nu = head_units(r, p.D), pairs = r.R >> 1, nthr = blockDim.x;
    const int64_t head = (int64_t)s.page * p.Hkv + h;
    uint8_t* codes = pool + head * p.page * p.D;
    float amax = 0.0f;
    for (int i = threadIdx.x; i < s.n * nu; i += nthr) {
        const int t = i / nu, u = i - t * nu;
        const TA* x = row<TA>(src, s.t0 + t, h);
        int f;
        const int f2 = unit_offsets(r, u, f);
        float a[8];
        Vec8<TA>::load(x + f, a);
        if (kTurn && f2 >= 0) {
            float b[8];
            Vec8<TA>::load(x + f2, b);
            turn8(r, cs + t * pairs + 8 * u, a, b);
            amax = max_finite(amax, b);
        }
        amax = max_finite(amax, a);
    }
    const int need = scale_exponent(block_max(amax, sm));
    int e = need;
    if (s.off > 0) {
        const int old = (int)scale[head] - 127;  // (every thread reads it before the barrier below)
        e = max(old, need);
        if (e > old) {  // the earlier tokens' codes to the new scale
            const float g = old - e >= -126 ? pow2(old - e) : 0.0f;
            for (int i = threadIdx.x; i < s.off * p.D / 8; i += nthr) {
                uint2 c = reinterpret_cast<uint2*>(codes)[i];
                const float2 v0 = e4m3x2_to_f32x2(c.x & 0xffffu), v1 = e4m3x2_to_f32x2(c.x >> 16);
                const float2 v2 = e4m3x2_to_f32x2(c.y & 0xffffu), v3 = e4m3x2_to_f32x2(c.y >> 16);
                const float v[8] = {v0.x, v0.y, v1.x, v1.y, v2.x, v2.y, v3.x, v3.y};
                reinterpret_cast<uint2*>(codes)[i] = e4m3x8(v, g);
            }
        }
        __syncthreads();
    }
    if (threadIdx.x == 0) scale[head] = (uint8_t)(e + 127);
    // 2^-e in two factors: 2^127 at e = -127 is a float, 2^-e never overflows
    const float inv = pow2(-e);
    for (int i = threadIdx.x; i < s.n * nu; i += nthr) {
        const int t = i / nu, u = i - t * nu;
        const TA* x = row<TA>(src, s.t0 + t, h);
        uint8_t* dst = codes + (int64_t)(s.off + t) * p.D;
        int f;
        const int f2 = unit_offsets(r, u, f);
        float a[8];
        Vec8<TA>::load(x + f, a);
        if (kTurn && f2 >= 0) {
            float b[8];
            Vec8<TA>::load(x + f2, b);
            turn8(r, cs + t * pairs + 8 * u, a, b);
            *reinterpret_cast<uint2*>(dst + f2) = e4m3x8(b, inv);
            if (out) Vec8<TA>::store(row<TA>(*out, s.t0 + t, h) + f2, b);
        }
        *reinterpret_cast<uint2*>(dst + f) = e4m3x8(a, inv);
        if (out) Vec8<TA>::store(row<TA>(*out, s.t0 + t, h) + f, a);
    }
}

// The same to a cache of the activations' type, and for rows that are only
// turned (pool null): one walk.
template <typename TA>
__device__ void append_plain(const AppendProblem& p, const RopeParams& r, const Segment& s, const float2* cs, const Rows& src,
                             int h, TA* pool, const Rows* out) {
    const int nu = head_units(r, p.D), pairs = r.R >> 1;
    TA* dst0 = pool ? pool + (((int64_t)s.page * p.Hkv + h) * p.page + s.off) * p.D : nullptr;
    for (int i = threadIdx.x; i < s.n * nu; i += blockDim.x) {
        const int t = i / nu, u = i - t * nu;
        const TA* x = row<TA>(src, s.t0 + t, h);
        int f;
        const int f2 = unit_offsets(r, u, f);
        float a[8], b[8];
        Vec8<TA>::load(x + f, a);
        if (f2 >= 0) {
            Vec8<TA>::load(x + f2, b);
            turn8(r, cs + t * pairs + 8 * u, a, b);
        }
        TA* o = out ? row<TA>(*out, s.t0 + t, h) : nullptr;
        TA* dst = dst0 ? dst0 + (int64_t)t * p.D : nullptr;
        if (dst) Vec8<TA>::store(dst + f, a);
        if (o) Vec8<TA>::store(o + f, a);
        if (f2 >= 0) {
            if (dst) Vec8<TA>::store(dst + f2, b);
            if (o) Vec8<TA>::store(o + f2, b);
        }
    }
}

// Block x: segment x / Hkv, kv head x % Hkv: its keys and values, and the query heads
// of its group. One block owns a page and head, so its scale needs no atomics.
template <typename TA>
__global__ void __launch_bounds__(kRopeThreads) append_kernel(const AppendProblem p) {
    pdl_enter();
    extern __shared__ float2 cs[];
    __shared__ int64_t plan[kRopeThreads / 32 + 4];
    __shared__ float red[kRopeThreads / 32];
    const Segment s = find_segment(p, blockIdx.x / p.Hkv, plan);
    if (s.n == 0) return;
    const int h = blockIdx.x % p.Hkv, pairs = p.r.R >> 1;
    for (int i = threadIdx.x; i < s.n * pairs; i += blockDim.x) {
        const int t = i / pairs;
        cs[i] = turn(p.r, p.positions ? (int64_t)p.positions[s.t0 + t] : s.pos + t, i - t * pairs);
    }
    __syncthreads();
    RopeParams still = p.r;  // values do not turn
    still.R = 0;
    const Rows* k_out = p.k_out.p ? &p.k_out : nullptr;
    if (s.page < 0) {
        if (k_out) append_plain<TA>(p, p.r, s, cs, p.k, h, nullptr, k_out);
    } else if (p.e4m3) {
        append_e4m3<TA, true>(p, p.r, s, cs, p.k, h, static_cast<uint8_t*>(p.k_pool), p.k_scale, k_out, red);
        append_e4m3<TA, false>(p, still, s, cs, p.v, h, static_cast<uint8_t*>(p.v_pool), p.v_scale, nullptr, red);
    } else {
        append_plain<TA>(p, p.r, s, cs, p.k, h, static_cast<TA*>(p.k_pool), k_out);
        append_plain<TA>(p, still, s, cs, p.v, h, static_cast<TA*>(p.v_pool), nullptr);
    }
    if (p.Hq) {
        const int G = p.Hq / p.Hkv;
        for (int g = 0; g < G; ++g) append_plain<TA>(p, p.r, s, cs, p.q, h * G + g, nullptr, &p.q_out);
    }
}

template <typename TA>
cudaError_t rope_as(const RopeProblem& p, cudaStream_t stream) {
    const int H = p.Hq + p.Hk, nu = p.r.R / 16 + (p.D - p.r.R) / 8;
    // about 1024 units of work per block, fewer where that would leave SMs idle
    int tokens = 1024 / (H * nu) > 1 ? 1024 / (H * nu) : 1;
    while (tokens > 1 && (p.T + tokens - 1) / tokens < 2 * sm_count()) tokens /= 2;
    int heads = H;
    while (heads > 1 && (int64_t)((p.T + tokens - 1) / tokens) * ((H + heads - 1) / heads) < 2 * sm_count() &&
           heads * nu * tokens > kRopeThreads)
        heads = (heads + 1) / 2;
    const size_t smem = (size_t)tokens * (p.r.R / 2) * sizeof(float2);
    return launch_k(rope_kernel<TA>, dim3((p.T + tokens - 1) / tokens, (H + heads - 1) / heads), dim3(kRopeThreads), smem,
                    stream, p, tokens, heads);
}

template <typename TA>
cudaError_t append_as(const AppendProblem& p, cudaStream_t stream) {
    const int most = p.page < p.T ? p.page : p.T;  // tokens of a segment
    const size_t smem = (size_t)most * (p.r.R / 2) * sizeof(float2);
    static DeviceOnce once;
    if (cudaError_t e = once.run([] {
            return cudaFuncSetAttribute(append_kernel<TA>, cudaFuncAttributeMaxDynamicSharedMemorySize, 128 * 128 * 8);
        });
        e != cudaSuccess)
        return e;
    const int64_t segs = min64(p.T, (int64_t)p.T / p.page + 2 * (int64_t)p.B);
    // few tokens per sequence: half the threads would have nothing to do
    const int threads = p.T <= 4 * (int64_t)p.B ? 128 : kRopeThreads;
    if (segs * p.Hkv > INT32_MAX) return cudaErrorInvalidConfiguration;
    return launch_k(append_kernel<TA>, dim3((unsigned)(segs * p.Hkv)), dim3(threads), smem, stream, p);
}

}  // namespace

cudaError_t launch_rope(const RopeProblem& p, cudaStream_t stream) {
    return p.act_dtype == GBMOE_F32 ? rope_as<float>(p, stream) : rope_as<__nv_bfloat16>(p, stream);
}

cudaError_t launch_append(const AppendProblem& p, cudaStream_t stream) {
    return p.act_dtype == GBMOE_F32 ? append_as<float>(p, stream) : append_as<__nv_bfloat16>(p, stream);
}

}  // namespace gbmoe
