// What the tensor-core kernels for packed prompts share: the search for the next row
// tile, taking over the work of CTAs that have not started, and rows computed again
// where a value that they do not see is no number.
#pragma once

#include <climits>

#include "attn_mma.cuh"
#include "attn_plan.cuh"

namespace gbmoe {

constexpr int kPromptTile = 128;  // query rows of a tile, keys of a tile

namespace tc {

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
// the keys it sees. Stops when every column is NaN. Keys::dot(problem, token, head, key row): the unscaled score.
template <typename Keys, typename Problem>
__device__ __forceinline__ void repair_row(const AttnProblem& p, const Problem& pr, int64_t k0, int64_t t, int h, int lo, int hi, float m, float l) {
    const int lane = threadIdx.x & 31, hk = h / (p.Hq / p.Hkv), d = 4 * lane;
    const __nv_bfloat16* v = static_cast<const __nv_bfloat16*>(p.v.p) + hk * p.v.hs;
    float o[4] = {0.f, 0.f, 0.f, 0.f};
    for (int j0 = lo; j0 <= hi; j0 += 32) {
        float w = 0.0f;
        if (j0 + lane <= hi) w = exp2f(fmaf(Keys::dot(pr, t, h, k0 + j0 + lane), p.scale_log2, -m));
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
template <typename Keys, typename Problem>
__device__ __noinline__ void repair_rows(const AttnProblem& p, const Problem& pr, uint32_t again, int64_t k0, int k_first, int tiles, int64_t t, int h,
                                         int lo, int hi, float m, float l) {
    const int lane = threadIdx.x & 31;
    const bool mine = again >> lane & 1u;
    const int seen_lo = __reduce_max_sync(0xffffffffu, mine ? lo : 0), seen_hi = __reduce_min_sync(0xffffffffu, mine ? hi : INT_MAX);
    const int hk = __shfl_sync(0xffffffffu, h / (p.Hq / p.Hkv), __ffs(again) - 1);
    const int2 bad = bad_keys(p, k0, hk, k_first, (int)min64(k_first + (int64_t)tiles * kPromptTile, p.Tk - k0), seen_lo, seen_hi);
    again = __ballot_sync(0xffffffffu, mine && (bad.x < lo || bad.y > hi));
    if (again == 0) return;
    if (lane == 0) bulk_wait_all();  // the rows' first versions are stored before the second
    __syncwarp();
    while (again) {
        const int src = __ffs(again) - 1;
        again &= again - 1;
        repair_row<Keys>(p, pr, k0, __shfl_sync(0xffffffffu, t, src), __shfl_sync(0xffffffffu, h, src), __shfl_sync(0xffffffffu, lo, src),
                   __shfl_sync(0xffffffffu, hi, src), __shfl_sync(0xffffffffu, m, src), __shfl_sync(0xffffffffu, l, src));
    }
}

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

}  // namespace tc
}  // namespace gbmoe
