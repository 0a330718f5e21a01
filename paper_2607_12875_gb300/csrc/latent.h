// Internal launch interface between the latent attention entry points
// (latent_api.cu) and their kernels.
#pragma once

#include "../../include/gblatent.h"
#include "attn.h"

namespace gbmoe {

// Absorbed or expanded attention: AttnProblem with one kv head for all query heads
// (absorbed: D = R, rows of a token R = heads, k_pool the pool of rows) or a kv
// head for each (expanded: D = V, k and v the heads' own rows).
struct LatentProblem {
    AttnProblem a;
    int K;         // elements of a query and a whole key: R + P, or N + P
    int own;       // of them a head's own (expanded: N), before the shared ones
    Rows k_rope;   // expanded: the shared rotary keys (one head)
};

constexpr int kLatentMaxRows = 64;      // rows of a tile of absorbed attention
constexpr int kLatentMaxParts = 19456;  // rows of partial results: 152 SMs, 2 parts of 64 rows each

struct LatentAppend {
    RopeParams r;
    int T, B, R, H;  // H 0: no queries
    int act_dtype;
    float eps;
    int page, page_log2, max_pages, n_pages;
    const int32_t *cu_q, *kv_len, *page_table, *positions;
    const void* gamma;
    Rows kv, kv_out, q, q_out;  // kv_out.p may be null
    void* pool;
};
cudaError_t launch_latent_append(const LatentAppend& p, cudaStream_t stream);

// CUDA cores: any covered sizes and types
cudaError_t launch_latent_simt(const LatentProblem& p, cudaStream_t stream);

// absorbed on the tensor cores: bf16, R a multiple of 128, P up to 64
bool latent_cached_tc_supported(const LatentProblem& p);
cudaError_t launch_latent_cached_tc(const LatentProblem& p, cudaStream_t stream);
// expanded on the tensor cores: bf16, P up to 64
bool latent_prompt_tc_supported(const LatentProblem& p);
cudaError_t launch_latent_prompt_tc(const LatentProblem& p, cudaStream_t stream);

}  // namespace gbmoe
