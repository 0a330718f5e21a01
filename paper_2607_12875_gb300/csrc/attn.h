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
    float mag;      // factor of cos and sin, negative angle for the inverse:
    float sin_sign; // -1 turns back
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
    int page, max_pages, n_pages;
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
    // chunks of a long key axis (cached attention): items aimed at per kv head, the
    // smallest chunk, and their partial results: [slots, Hkv, rows, D] sums and
    // [slots, Hkv, rows, 4] statistics
    int target, min_chunk;
    float *part_o, *part_s;
    int32_t* err;
};

constexpr int kSplitRows = 16;      // (token, head of the group) rows of a work item of the split kernels
constexpr int kMaxSplitItems = 2432; // items aimed at over all kv heads: 16 waves of one CTA on 152 SMs

// work items aimed at per kv head, and the partial slots that can then be needed
inline int split_target(int Hkv) { return kMaxSplitItems / Hkv > 1 ? kMaxSplitItems / Hkv : 1; }
inline int64_t split_slots(int Hkv) { return 2 * (int64_t)split_target(Hkv) + 2; }

// most items (row tiles of `rows` rows times chunks) of a problem
inline int64_t attn_items(const AttnProblem& p, int rows) {
    return (int64_t)p.T * p.R / rows + p.B + (p.paged ? p.target : 0);
}

cudaError_t launch_attn_simt(const AttnProblem& p, cudaStream_t stream);
// cached attention on the tensor cores: bf16, D 64, 96 or 128
bool attn_split_supported(const AttnProblem& p);
cudaError_t launch_attn_split(const AttnProblem& p, cudaStream_t stream);
// joins the chunks' partial results of the two kernels above
cudaError_t launch_attn_join(const AttnProblem& p, cudaStream_t stream);
// packed attention on the tensor cores: bf16, D up to 128
bool attn_prompt_tc_supported(const AttnProblem& p);
cudaError_t launch_attn_prompt_tc(const AttnProblem& p, cudaStream_t stream);

}  // namespace gbmoe
