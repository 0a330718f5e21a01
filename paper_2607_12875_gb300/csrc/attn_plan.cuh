// What the attention kernels share: a sequence's lengths, which keys a row
// sees, and the list of work items that every CTA derives for itself from the
// lengths on the device (no host read, no planning launch).
#pragma once

#include "attn.h"
#include "common.cuh"

namespace gbmoe {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
__device__ __forceinline__ float neg_inf() { return __uint_as_float(0xff800000u); }

struct Seq {
    int q0, nq;     // its query rows
    int64_t k0;     // first key row (packed keys)
    int len;        // keys
    int start;      // first key that any of its queries sees, rounded down to a multiple of 128
};

__device__ __forceinline__ int clampi(int v, int lo, int hi) { return min(max(v, lo), hi); }

// lengths of sequence b, cut to what the buffers hold
__device__ __forceinline__ Seq load_seq(const AttnProblem& p, int b) {
    Seq s;
    s.q0 = clampi(p.cu_q[b], 0, p.T);
    s.nq = clampi(p.cu_q[b + 1], s.q0, p.T) - s.q0;
    if (p.paged) {
        s.k0 = 0;
        s.len = (int)min64(max(p.kv_len[b], 0), (int64_t)p.max_pages * p.page);
    } else {
        const int k0 = clampi(p.cu_k[b], 0, p.Tk);
        s.k0 = k0;
        s.len = clampi(p.cu_k[b + 1], k0, p.Tk) - k0;
    }
    s.start = 0;
    if (p.window > 0) s.start = (int)max64(0, (int64_t)s.len - s.nq - p.window + 1) & ~127;
    return s;
}

// keys lo .. hi that the row of query i (of sequence s) sees; hi < lo: none
__device__ __forceinline__ void seen_keys(const AttnProblem& p, const Seq& s, int i, int& lo, int& hi) {
    const int64_t pos = (int64_t)s.len - s.nq + i;
    hi = p.causal ? (int)min64(pos, s.len - 1) : s.len - 1;
    lo = p.window > 0 ? (int)max64(0, pos - p.window + 1) : 0;
    if (hi < lo) hi = -1, lo = 0;
}

// rows of queries (token i, head g of R: row i * R + g) in tiles of kRows
template <int kRows>
__device__ __forceinline__ int row_tiles(const AttnProblem& p, const Seq& s) {
    return (int)(((int64_t)s.nq * p.R + kRows - 1) / kRows);
}

// One work item: a row tile of a sequence and a chunk of its keys.
struct Item {
    int b;           // -1: none
    Seq s;
    int tile;
    int k_lo, k_hi;  // keys of the chunk (k_hi exclusive)
    int chunks;      // chunks of this sequence
    int64_t slot;    // its partial results' slot (chunks > 1)
};

__device__ __forceinline__ int64_t block_sum(int64_t v, int64_t* sm) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, n = blockDim.x >> 5;
#pragma unroll
    for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    __syncthreads();
    if (lane == 0) sm[warp] = v;
    __syncthreads();
    int64_t t = 0;
    for (int w = 0; w < n; ++w) t += sm[w];
    return t;
}

// keys per chunk: the items aimed at over all row tiles' keys, in multiples of 128
__device__ __forceinline__ int chunk_keys(const AttnProblem& p, int64_t work) {
    int64_t c = (work + p.target - 1) / p.target;
    c = max64(c, p.min_chunk);
    return (int)min64((c + 127) & ~(int64_t)127, 0x7fffff80);
}

// Item `index` of the list (sequences in order; a sequence's tiles; a tile's
// chunks), found by the whole block: sm holds 2 * warps + 8 words of 64 bits.
// The number of partial slots before a sequence counts only sequences with
// several chunks; their slots are at most 2 * target. kSplit: the list of row
// tiles of such sequences instead (slot: their first chunk's).
template <int kRows, bool kSplit = false>
__device__ Item find_item(const AttnProblem& p, int64_t index, int64_t* sm) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, n = blockDim.x;
    int64_t work = 0;
    for (int b = tid; b < p.B; b += n) {
        const Seq s = load_seq(p, b);
        work += (int64_t)row_tiles<kRows>(p, s) * (s.len - min(s.start, s.len));
    }
    const int C = chunk_keys(p, block_sum(work, sm));
    int64_t* found = sm + 2 * (n >> 5);  // sequence, items before it, slots before it
    __syncthreads();
    if (tid == 0) found[0] = -1;
    int64_t items0 = 0, slots0 = 0;
    for (int base = 0; base < p.B; base += n) {
        const int b = base + tid;
        int64_t it = 0, sl = 0;
        if (b < p.B) {
            const Seq s = load_seq(p, b);
            const int64_t tiles = row_tiles<kRows>(p, s), eff = s.len - min(s.start, s.len);
            const int64_t chunks = max64(1, (eff + C - 1) / C);
            sl = chunks > 1 ? tiles * chunks : 0;
            it = !kSplit ? tiles * chunks : chunks > 1 ? tiles : 0;
        }
        int64_t pi = it, ps = sl;  // inclusive prefix sums in the warp
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int64_t a = __shfl_up_sync(0xffffffffu, pi, d), c = __shfl_up_sync(0xffffffffu, ps, d);
            if (lane >= d) pi += a, ps += c;
        }
        __syncthreads();
        if (lane == 31) sm[2 * warp] = pi, sm[2 * warp + 1] = ps;
        __syncthreads();
        int64_t ti = 0, tsl = 0, wi = items0, wsl = slots0;
        for (int w = 0; w < (n >> 5); ++w) {
            if (w < warp) wi += sm[2 * w], wsl += sm[2 * w + 1];
            ti += sm[2 * w], tsl += sm[2 * w + 1];
        }
        const int64_t before = wi + pi - it;
        if (it > 0 && index >= before && index < before + it) {
            found[0] = b;
            found[1] = before;
            found[2] = wsl + ps - sl;
        }
        items0 += ti, slots0 += tsl;
        __syncthreads();
        if (index < items0) break;  // uniform
    }
    __syncthreads();
    Item r;
    r.b = (int)found[0];
    if (r.b < 0) return r;
    r.s = load_seq(p, r.b);
    const int64_t eff = r.s.len - min(r.s.start, r.s.len);
    r.chunks = (int)max64(1, (eff + C - 1) / C);
    const int64_t local = index - found[1];
    if (kSplit) {
        r.tile = (int)local;
        r.slot = found[2] + local * r.chunks;
        return r;
    }
    r.tile = (int)(local / r.chunks);
    const int chunk = (int)(local - (int64_t)r.tile * r.chunks);
    r.k_lo = (int)min64((int64_t)r.s.start + (int64_t)chunk * C, r.s.len);
    r.k_hi = (int)min64((int64_t)r.k_lo + C, r.s.len);
    r.slot = found[2] + local;
    return r;
}

// sequence of packed row t (rows outside every sequence: -1): the last b with cu_q[b] <= t
__device__ __forceinline__ int seq_of_row(const int32_t* cu, int B, int t) {
    int lo = 0, hi = B;  // cu[lo] <= t < cu[hi] when it lies in one
    if (t < cu[0] || t >= cu[B]) return -1;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (cu[mid] <= t) lo = mid;
        else hi = mid;
    }
    return lo;
}

// what find_item needs in shared memory for a block of n threads
constexpr int plan_words(int n) { return 2 * (n / 32) + 8; }

}  // namespace gbmoe
