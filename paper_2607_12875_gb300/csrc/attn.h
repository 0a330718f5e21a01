// Internal launch interface between the attention entry points (attn_api.cu)
// and their kernels.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/gbattn.h"

namespace gbmoe {

// [tokens, heads, D] rows, strides in elements
struct Rows {
    const void* p;
    int64_t ts, hs;
};

struct RopeParams {
    int R;          // rotary_dim (0: nothing turns)
    int half;       // 1: pairs (i, i + R/2), 0: (2i, 2i + 1)
    float mag;      // factor of cos and sin
    float sin_sign; // 1, or -1: turns back
    const uint64_t* table;
};

struct RopeProblem {
    RopeParams r;
    int T, D, Hq, Hk;  // Hq or Hk is 0 when that tensor is left out
    int act_dtype;
    const int32_t* positions;
    Rows q, k, q_out, k_out;
};
cudaError_t launch_rope(const RopeProblem& p, cudaStream_t stream);

struct AppendProblem {
    RopeParams r;
    int T, B, D, Hq, Hkv;  // Hq 0: no queries
    int act_dtype, e4m3;
    int page, page_log2, max_pages, n_pages;
    const int32_t *cu_q, *kv_len, *page_table, *positions;
    Rows q, k, v, q_out, k_out;  // k_out.p may be null
    void *k_pool, *v_pool;
    uint8_t *k_scale, *v_scale;
};
cudaError_t launch_append(const AppendProblem& p, cudaStream_t stream);

// Attention of packed queries over packed keys (paged = 0) or over the cache.
struct AttnProblem {
    int B, T, Tk, Hq, Hkv, D;
    int R;  // rows of a token in a row tile: G where a tile holds the heads of a group, else 1
    int act_dtype, causal, window;
    float scale_log2;  // scale * log2(e)
    const int32_t* cu_q;
    const int32_t* cu_k;  // packed keys
    Rows q, k, v, out;
    float* lse;
    int paged, e4m3, page, max_pages, n_pages;
    const int32_t *kv_len, *page_table;
    const void *k_pool, *v_pool;
    const uint8_t *k_scale, *v_scale;
    int page_log2;
    // cached attention: CTAs (shares of the work), the least blocks of a share, blocks that
    // a tile's set-up is counted as, rows of a tile, and the partial results [2 * shares, rows, D] sums and [2 * shares, rows, 4]
    // statistics of tiles cut by the shares' ends, with a record of the tile that each
    // share's end cuts for the join
    int shares, min_blocks, tile_cost, tile_rows;
    float *part_o, *part_s;
    struct CutTile* cuts;
    int32_t* err;
};

// The tile that begins in a share and goes on in the next ones.
struct CutTile {
    int parts;           // shares that it lies in; 0: the share cuts none
    int rows;            // its rows
    int first;           // slot of its first part (the next ones: 2 (share + 1), 2 (share + 2), ..)
    int head, tile;      // kv head, row tile
    int q0, nq, len;     // its sequence
};
static_assert(sizeof(CutTile) == 32, "two 16-byte loads");

constexpr int kBlockKeys = 64;   // keys of a block of work
constexpr int kMaxTileRows = 16;
constexpr int kMaxShares = 608;  // four CTAs on each of 152 SMs

// Deals out the work of cached attention in tiles of `rows` rows to `per_sm` CTAs on an
// SM, or as many as there can be shares of min_blocks (more than tile_cost).
inline void set_shares(AttnProblem& p, int rows, int per_sm, int sms, int min_blocks, int tile_cost) {
    p.tile_rows = rows, p.min_blocks = min_blocks, p.tile_cost = tile_cost;
    const int64_t tiles = (int64_t)p.T * p.R / rows + p.B;
    const int64_t blocks = tiles * p.Hkv * (((int64_t)p.max_pages * p.page + kBlockKeys - 1) / kBlockKeys + 1 + p.tile_cost);
    const int64_t most = (blocks + p.min_blocks - 1) / p.min_blocks;
    const int64_t cap = (int64_t)per_sm * sms < kMaxShares ? (int64_t)per_sm * sms : kMaxShares;
    p.shares = (int)(most < cap ? most : cap);
}

cudaError_t launch_attn_simt(const AttnProblem& p, cudaStream_t stream);
// cached attention on the tensor cores: bf16, D 64, 96 or 128
bool attn_split_supported(const AttnProblem& p);
cudaError_t launch_attn_split(const AttnProblem& p, cudaStream_t stream);
// joins the partial results of the tiles that the two kernels above cut
cudaError_t launch_attn_join(const AttnProblem& p, cudaStream_t stream);
// packed attention on the tensor cores: bf16, D up to 128
bool attn_prompt_tc_supported(const AttnProblem& p);
cudaError_t launch_attn_prompt_tc(const AttnProblem& p, cudaStream_t stream);

}  // namespace gbmoe
