// New tokens' latents into the paged cache: RMS norm of the latent, rotation of the
// shared key, and of the rotary parts of the queries, in one launch.
//
// A group of threads has one token: its first warp the token's row (a lane has up to
// two pieces of eight latent elements in registers between the sum of squares and the
// product, and one unit of 16 rotary elements), all of its threads one unit each of
// every step-th head of the queries, with the unit's angles in registers. Which
// sequence a token belongs to, every warp finds for itself (find_seq).
//
// Each element is read once and written once, so HBM bounds it for prompts (8192 tokens, 128 heads, rows also in
// place: 58 us, 5.1 TB/s; the next heads' loads in flight while these turn: 64 without) and the launch with three
// dependent loads (offsets, length, page) for single tokens: 128 in 7.1 us.
#include <climits>

#include "attn_plan.cuh"
#include "attn_turn.cuh"
#include "latent.h"

namespace gbmoe {
namespace {

constexpr int kThreads = 256;
constexpr unsigned kFull = 0xffffffffu;

// The sequence whose tokens t is one of (-1: none), by a whole warp: the first b with
// cu_q[b + 1] > t, 32 offsets at a time of the interval that holds it.
__device__ __forceinline__ int find_seq(const LatentAppend& p, int t) {
    const int lane = threadIdx.x & 31;
    if (p.B <= 256) {  // all of them at once: one round trip to memory instead of two
        int upto = 0, ends[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) ends[i] = lane + 32 * i < p.B ? p.cu_q[lane + 32 * i + 1] : INT_MAX;
#pragma unroll
        for (int i = 0; i < 8; ++i) upto += __popc(__ballot_sync(kFull, ends[i] <= t));
        return upto < p.B && p.cu_q[upto] <= t ? upto : -1;
    }
    int lo = 0, hi = p.B;
    while (lo < hi) {
        const int step = (hi - lo + 31) / 32;
        const int at = min((int)min64(lo + (int64_t)(lane + 1) * step, hi) - 1, hi - 1);
        const uint32_t past = __ballot_sync(kFull, p.cu_q[at + 1] > t);
        if (past == 0) return -1;
        const int f = __ffs(past) - 1;
        const int from = (int)min64(lo + (int64_t)f * step, hi - 1);
        if (step == 1) return p.cu_q[from] <= t ? from : -1;
        hi = (int)min64(from + (int64_t)step, hi), lo = from;
    }
    return -1;
}

// Block x: tokens x * (256 / G) .., a group of G threads each. bits: log2 of the threads of a head's units.
template <typename TA, int G>
__global__ void __launch_bounds__(kThreads, 2) latent_append_kernel(const __grid_constant__ LatentAppend p, int bits) {
    pdl_enter();
    constexpr int B = sizeof(TA) == 2 ? 4 : 1;  // heads of a thread whose loads are in flight
    const int lane = threadIdx.x & 31, r = threadIdx.x % G;
    const int t = (int)min64((int64_t)blockIdx.x * (kThreads / G) + threadIdx.x / G, p.T);
    if (t >= p.T) return;  // (whole warps)
    const int u = r & ((1 << bits) - 1), step = G >> bits;
    const bool turns = p.H > 0 && u < p.r.R >> 4;
    const Unit unit = unit_of(p.r, p.r.R, min(u, max((p.r.R >> 4) - 1, 0)));
    Held<TA> held[B];
    auto fetch = [&](int h) {
#pragma unroll
        for (int k = 0; k < B; ++k)
            if (turns && h + k * step < p.H) held[k].load(unit, row<TA>(p.q, t, h + k * step));
    };
    fetch(r >> bits);
    // the token's own row
    const bool own = r < 32;
    const TA* src = row<TA>(p.kv, t, 0);
    const int chunks = p.R >> 3;
    Raw8<TA> c[2];
    Held<TA> key;
    const bool key_unit = own && lane < p.r.R >> 4;
    const Unit ku = unit_of(p.r, p.r.R, key_unit ? lane : 0);
    if (own) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (lane + 32 * i < chunks) c[i].load(src + 8 * (lane + 32 * i));
        if (key_unit) key.load(ku, src + p.R);
    }
    const int b = find_seq(p, t);
    if (b < 0) return;
    const int q0 = clampi(p.cu_q[b], 0, p.T), n = clampi(p.cu_q[b + 1], q0, p.T) - q0;
    const int64_t at = (int64_t)p.kv_len[b] - n + (t - q0);  // its place in the sequence
    const int64_t pos = p.positions ? (int64_t)p.positions[t] : at;
    if (own) {
        int id = -1;
        const int64_t pg = at >> p.page_log2;
        if (at >= 0 && pg < p.max_pages) id = p.page_table[(int64_t)b * p.max_pages + pg];
        if (id >= p.n_pages) id = -1;
        const int W = p.R + p.r.R;
        TA* slot = id >= 0 ? static_cast<TA*>(p.pool) + ((int64_t)id * p.page + (at & (p.page - 1))) * W : nullptr;
        TA* out = p.kv_out.p ? row<TA>(p.kv_out, t, 0) : nullptr;
        float inv = 1.0f;
        if (p.gamma) {
            float ss = 0.0f;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                if (lane + 32 * i >= chunks) continue;
#pragma unroll
                for (int j = 0; j < 8; ++j) ss = fmaf(c[i].at(j), c[i].at(j), ss);
            }
#pragma unroll
            for (int d = 16; d; d >>= 1) ss += __shfl_xor_sync(kFull, ss, d);
            inv = 1.0f / sqrtf(ss / (float)p.R + p.eps);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int at8 = 8 * (lane + 32 * i);
            if (at8 >= p.R) continue;
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = c[i].at(j);
            if (p.gamma) {
                float g[8];
                Vec8<TA>::load(static_cast<const TA*>(p.gamma) + at8, g);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = v[j] * inv * g[j];
            }
            if (slot) Vec8<TA>::store(slot + at8, v);
            if (out) Vec8<TA>::store(out + at8, v);
        }
        if (key_unit) {
            Angles angles;
            angles.set(p.r, ku, pos);
            Values v;
            v.from(key, ku);
            v.turn(p.r, ku, angles);
            if (slot) v.store(ku, slot + p.R);
            if (out) v.store(ku, out + p.R);
        }
    }
    if (!turns) return;
    Angles angles;
    angles.set(p.r, unit, pos);
    for (int h = r >> bits; h < p.H; h += B * step) {
        Held<TA> now[B];
#pragma unroll
        for (int k = 0; k < B; ++k) now[k] = held[k];
        fetch(h + B * step);  // the next heads' loads fly while these turn
#pragma unroll
        for (int k = 0; k < B; ++k) {
            if (h + k * step >= p.H) break;
            Values v;
            v.from(now[k], unit);
            v.turn(p.r, unit, angles);
            v.store(unit, row<TA>(p.q_out, t, h + k * step));
        }
    }
}

template <typename TA, int G>
cudaError_t append_as(const LatentAppend& p, cudaStream_t stream) {
    const int tokens = kThreads / G;
    return launch_k(latent_append_kernel<TA, G>, dim3((unsigned)(((int64_t)p.T + tokens - 1) / tokens)), dim3(kThreads), 0, stream, p,
                    unit_bits(max(p.r.R >> 4, 1)));
}

template <typename TA>
cudaError_t append_type(const LatentAppend& p, cudaStream_t stream) {
    // A token's search and angles cost as much as several of its heads, so it has as few threads as keep its loads in
    // flight. Us with 32, 64 and 128: 8192 tokens of 128 heads 59, 57 and 72, of 16 heads 20, 28 and 48; 128 tokens of
    // 128 heads 9.6, 7.4 and 7.3 (one session's figures).
    return (p.H << unit_bits(max(p.r.R >> 4, 1))) <= 128 ? append_as<TA, 32>(p, stream) : append_as<TA, 64>(p, stream);
}

}  // namespace

cudaError_t launch_latent_append(const LatentAppend& p, cudaStream_t stream) {
    return p.act_dtype == GBMOE_F32 ? append_type<float>(p, stream) : append_type<__nv_bfloat16>(p, stream);
}

}  // namespace gbmoe
