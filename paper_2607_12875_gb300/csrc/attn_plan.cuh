// What the attention kernels share: a sequence's lengths, which keys a row
// sees, and the CTA's part of the work, which every CTA derives for itself from
// the lengths on the device (no host read, no planning launch).
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

// whether one of sequence b's cached keys lo .. hi has a page in the pool
__device__ __forceinline__ bool any_page(const AttnProblem& p, int b, int lo, int hi) {
    if (hi < lo) return false;
    const int32_t* pages = p.page_table + (int64_t)b * p.max_pages;
    for (int i = lo >> p.page_log2; i <= hi >> p.page_log2; ++i)
        if (pages[i] >= 0 && pages[i] < p.n_pages) return true;
    return false;
}

// tiles of `rows` rows of queries (token i, head g of R: row i * R + g)
__device__ __forceinline__ int64_t row_tiles(const AttnProblem& p, const Seq& s, int rows) {
    return ((int64_t)s.nq * p.R + rows - 1) / rows;
}

// blocks of kBlock keys of a sequence's tiles (at least one, so that rows
// without keys are written too)
template <int kBlock = kBlockKeys>
__device__ __forceinline__ int key_blocks(const Seq& s) {
    return max(1, (s.len - min(s.start, s.len) + kBlock - 1) / kBlock);
}

__device__ __forceinline__ int64_t warp_scan(int64_t v) {  // inclusive
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int64_t a = __shfl_up_sync(0xffffffffu, v, d);
        if (lane >= d) v += a;
    }
    return v;
}

// Where unit `index` of the list lies whose sequence b holds units(b) units: the
// sequence (-1: past the end) and the unit's place in it. `index` comes from the
// list's total, whose loads and sums a batch of at most blockDim sequences
// shares with the search. For the whole block; sm holds plan_words words.
struct Place {
    int b;
    int64_t at;
};
template <typename Units, typename Index>
__device__ __forceinline__ Place find_place(int B, Units units, Index index_of, int64_t* sm) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, n = blockDim.x, warps = n >> 5;
    int64_t* found = sm + warps;
    if (tid == 0) found[0] = -1;
    int64_t index = -1, before = 0;
    if (B > n) {  // the total first
        int64_t v = 0;
        for (int b = tid; b < B; b += n) v += units(b);
        v = warp_scan(v);
        if (lane == 31) sm[warp] = v;
        __syncthreads();
        int64_t total = 0;
        for (int w = 0; w < warps; ++w) total += sm[w];
        index = index_of(total);
        __syncthreads();
    }
    for (int base = 0; base < B; base += n) {
        const int b = base + tid;
        const int64_t v = b < B ? units(b) : 0;
        const int64_t pre = warp_scan(v);
        if (lane == 31) sm[warp] = pre;
        __syncthreads();
        int64_t here = before, sum = 0;
        for (int w = 0; w < warps; ++w) {
            if (w < warp) here += sm[w];
            sum += sm[w];
        }
        if (B <= n) index = index_of(sum);
        const int64_t first = here + pre - v;
        if (index >= first && index < first + v) {
            found[0] = b;
            found[1] = index - first;
        }
        before += sum;
        __syncthreads();
        if (index < before) break;  // uniform
    }
    return Place{(int)found[0], found[1]};
}
constexpr int plan_words(int threads) { return threads / 32 + 2; }

// Row tile `index` of packed queries (sequences in order, their tiles in order).
__device__ __forceinline__ Place find_tile(const AttnProblem& p, int64_t index, int rows, int64_t* sm) {
    return find_place(p.B, [&](int b) { return row_tiles(p, load_seq(p, b), rows); }, [&](int64_t) { return index; }, sm);
}

// a / b for a >= 0, b > 0: 64-bit division takes over a hundred instructions
__device__ __forceinline__ int64_t div64(int64_t a, int64_t b) {
    return ((a | b) >> 32) == 0 ? (int64_t)((uint32_t)a / (uint32_t)b) : a / b;
}

// Cached attention: the blocks of kBlock keys of all row tiles and kv heads, in the
// order sequence, head, tile, block, are dealt out in equal shares, one per CTA.
// A tile begins with tile_cost empty blocks, about what its set-up and results
// cost, so that a share of many short tiles is not more work than the others.
// A share is a run of segments: blocks blk0 .. blk1 - 1 of one tile and head. A
// tile that lies whole in a share is finished there; the first and the last
// segment of a share may be parts of tiles, whose results go to the share's
// partial slots 2 i and 2 i + 1 for the join.
struct Shares {
    int64_t total, each;  // blocks, blocks of a share (more than tile_cost: its first segment is never empty)

    __device__ __forceinline__ void set(const AttnProblem& p, int64_t blocks) {
        total = blocks;
        each = max64(p.min_blocks, div64(blocks + p.shares - 1, p.shares));
    }
};

struct Segment {
    int b, head, tile, blk0, blk1, nb;
    Seq s;
    int64_t slot;  // -1: whole
};

// kRows: rows of a tile (0: p.tile_rows).
template <int kRows, int kBlock = kBlockKeys>
struct Walk {
    __device__ __forceinline__ static int tile_rows(const AttnProblem& p) { return kRows > 0 ? kRows : p.tile_rows; }
    __device__ __forceinline__ static int64_t tiles_of(const AttnProblem& p, const Seq& s) {
        if constexpr (kRows > 0) return row_tiles(p, s, kRows);
        return div64((int64_t)s.nq * p.R + p.tile_rows - 1, p.tile_rows);
    }
    Shares sh;
    int64_t u, u0, u1;  // where the segment begins; the share's begin and end
    int64_t share;
    int tiles, x0, x1;  // tiles of a head; the segment's place in its tile, the empty blocks counted
    Segment g;

    // whether share `index` holds anything (then g is its first segment)
    __device__ __forceinline__ bool begin(const AttnProblem& p, int64_t index, int64_t* sm) {
        const Place at = find_place(
            p.B,
            [&](int b) { const Seq s = load_seq(p, b); return tiles_of(p, s) * (key_blocks<kBlock>(s) + p.tile_cost) * p.Hkv; },
            [&](int64_t total) { sh.set(p, total); return index * sh.each; }, sm);
        if (at.b < 0) return false;
        start(p, index, at);
        return true;
    }
    // the share that begins at this place
    __device__ __forceinline__ void start(const AttnProblem& p, int64_t index, const Place& at) {
        share = index;
        u = u0 = index * sh.each;
        u1 = min64(u0 + sh.each, sh.total);
        enter(p, at.b);
        const int nx = g.nb + p.tile_cost;
        const int64_t per = (int64_t)tiles * nx;
        g.head = (int)div64(at.at, per);
        const int64_t rest = at.at - g.head * per;
        g.tile = (int)div64(rest, nx);
        x0 = (int)(rest - (int64_t)g.tile * nx);
        cut(p);
    }
    __device__ __forceinline__ bool next(const AttnProblem& p) {
        if (last(p)) return false;
        u += x1 - x0;
        x0 = 0;
        if (++g.tile == tiles) {
            g.tile = 0;
            if (++g.head == p.Hkv) {
                g.head = 0;
                int b = g.b;
                do enter(p, ++b);
                while (tiles == 0);  // (u < u1 <= total: there is one)
            }
        }
        cut(p);
        return true;
    }
    // whether nothing but empty blocks of the next tile follows in the share
    __device__ __forceinline__ bool last(const AttnProblem& p) const { return u + (x1 - x0) + p.tile_cost >= u1; }
    // For one thread, at a segment's end (or, idle, where the share holds nothing): what the join is to know
    __device__ __forceinline__ void note(const AttnProblem& p) const {
        if (last(p)) note_parts(p, (int)div64(g.nb - g.blk1 + sh.each - 1, sh.each) + 1);
    }
    __device__ __forceinline__ void note_parts(const AttnProblem& p, int parts) const {
        CutTile c{};
        if (g.blk0 == 0 && g.blk1 < g.nb) {
            c.parts = parts;
            c.first = (int)g.slot;
            c.rows = (int)min64(tile_rows(p), (int64_t)g.s.nq * p.R - (int64_t)g.tile * tile_rows(p));
            c.head = g.head, c.tile = g.tile;
            c.q0 = g.s.q0, c.nq = g.s.nq, c.len = g.s.len;
        }
        p.cuts[share] = c;
    }
    __device__ __forceinline__ static void note_idle(const AttnProblem& p, int64_t share) { p.cuts[share] = CutTile{}; }
    __device__ __forceinline__ void enter(const AttnProblem& p, int b) {
        g.b = b;
        g.s = load_seq(p, b);
        tiles = (int)tiles_of(p, g.s);
        g.nb = key_blocks<kBlock>(g.s);
    }
    __device__ __forceinline__ void cut(const AttnProblem& p) {
        x1 = (int)min64(g.nb + p.tile_cost, x0 + (u1 - u));
        g.blk0 = max(0, x0 - p.tile_cost), g.blk1 = x1 - p.tile_cost;
        g.slot = g.blk0 == 0 && g.blk1 == g.nb ? -1 : 2 * share + (u != u0);
    }
};

}  // namespace gbmoe
