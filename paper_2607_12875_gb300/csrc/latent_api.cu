// C ABI of latent attention (declared in include/gblatent.h): argument checks on
// the host and the choice of kernels.
#include <cmath>
#include <cstdint>

#include "api_status.h"
#include "latent.h"

using namespace gbmoe;

namespace {

constexpr size_t kAlign = 256;
constexpr int kMaxHeads = 4096;
constexpr int kMaxRows = 1 << 30;  // tokens, query rows of a sequence, keys, slots of the pool: the kernels count them in 32 bits

size_t align_up(size_t v) { return (v + kAlign - 1) & ~(kAlign - 1); }
int64_t act_bytes(int act) { return act == GBMOE_F32 ? 4 : 2; }
bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

int check_cfg(const gblatent_config* c) {
    if (!c) return GBMOE_EINVAL;
    if (c->heads <= 0 || c->latent_dim <= 0 || c->rope_dim < 0 || c->nope_dim <= 0 || c->value_dim <= 0) return GBMOE_EINVAL;
    if (c->act_dtype != GBMOE_F32 && c->act_dtype != GBMOE_BF16) return GBMOE_EINVAL;
    if (c->causal != 0 && c->causal != 1) return GBMOE_EINVAL;
    if (!std::isfinite(c->scale) || !std::isfinite(c->rotary_scale)) return GBMOE_EINVAL;
    if (!(c->norm_eps >= 0.0f) || !std::isfinite(c->norm_eps)) return GBMOE_EINVAL;
    if (c->rotary_layout != GBATTN_HALF && c->rotary_layout != GBATTN_INTERLEAVED) return GBMOE_EINVAL;
    if (c->page <= 0) return GBMOE_EINVAL;
    // what the kernels cover
    if (c->heads > kMaxHeads || c->latent_dim % 8 != 0 || c->latent_dim > 512) return GBMOE_EUNSUPPORTED;
    if (c->rope_dim % 16 != 0 || c->rope_dim > 128) return GBMOE_EUNSUPPORTED;
    if (c->nope_dim % 8 != 0 || c->nope_dim > 128 || c->value_dim % 8 != 0 || c->value_dim > 128) return GBMOE_EUNSUPPORTED;
    if (c->page != 16 && c->page != 32 && c->page != 64 && c->page != 128) return GBMOE_EUNSUPPORTED;
    return GBMOE_OK;
}

// rows [T, heads, D] that the kernels read (or, out = true, write: then no two of
// them may share an element)
bool rows_ok(const gblatent_config* c, const gbattn_rows* r, int64_t T, int64_t heads, int64_t D, bool out) {
    if (!r || !r->data || !aligned(r->data, 16)) return false;
    const int64_t eb = act_bytes(c->act_dtype);
    if (T > 1 && (r->token_stride < 0 || r->token_stride * eb % 16 != 0)) return false;
    if (heads > 1 && (r->head_stride < 0 || r->head_stride * eb % 16 != 0)) return false;
    if (!out) return true;
    if (T > 1 && r->token_stride < D) return false;
    if (heads > 1 && r->head_stride < D) return false;
    return T <= 1 || heads <= 1 || r->token_stride >= (heads - 1) * r->head_stride + D ||
           r->head_stride >= (T - 1) * r->token_stride + D;
}

// strides that no access uses (one token, one head) read as 0
Rows rows_of(const gbattn_rows* r, int64_t T, int64_t heads) {
    return Rows{r->data, T > 1 ? r->token_stride : 0, heads > 1 ? r->head_stride : 0};
}

int check_batch(const gbattn_batch* b, int32_t T) {
    if (!b || b->B < 0 || b->max_pages < 0 || T < 0) return GBMOE_EINVAL;
    if (T > kMaxRows || b->B > kMaxRows) return GBMOE_EUNSUPPORTED;
    if (T == 0 || b->B == 0) return GBMOE_OK;
    if (!b->cu_q || !b->kv_len || (b->max_pages > 0 && !b->page_table)) return GBMOE_EINVAL;
    if (!aligned(b->cu_q, 4) || !aligned(b->kv_len, 4) || !aligned(b->page_table, 4)) return GBMOE_EINVAL;
    return GBMOE_OK;
}

int check_cache(const gblatent_config* c, const gblatent_cache* k) {
    if (!k || !k->rows || k->n_pages < 0 || !aligned(k->rows, 16)) return GBMOE_EINVAL;
    return (int64_t)k->n_pages * c->page > kMaxRows ? GBMOE_EUNSUPPORTED : GBMOE_OK;
}

int log2_of(int v) {
    int b = 0;
    while (1 << b < v) ++b;
    return b;
}

struct Layout {
    size_t err, cuts, part_s, part_o, total;
};

Layout layout(const gblatent_config* c) {
    Layout L{};
    size_t o = 0;
    auto take = [&](size_t bytes) { size_t at = o; o = align_up(o + bytes); return at; };
    L.err = take(4);
    L.cuts = take(kMaxShares * sizeof(CutTile));
    L.part_s = take((size_t)kLatentMaxParts * 16);
    L.part_o = take((size_t)kLatentMaxParts * c->latent_dim * 4);
    L.total = o;
    return L;
}

int check_ws(const gblatent_config* c, void* ws, size_t bytes) {
    if (!ws || !aligned(ws, kAlign)) return GBMOE_EINVAL;
    return bytes < layout(c).total ? GBMOE_EWORKSPACE : GBMOE_OK;
}

LatentProblem problem(const gblatent_config* c, int32_t T, int32_t B, float* lse, void* ws) {
    const Layout L = layout(c);
    char* w = static_cast<char*>(ws);
    LatentProblem p{};
    AttnProblem& a = p.a;
    a.B = B; a.T = T; a.Hq = c->heads;
    a.act_dtype = c->act_dtype; a.causal = c->causal;
    a.scale_log2 = c->scale * 1.4426950408889634f;
    a.lse = lse;
    a.page = 1;
    a.err = reinterpret_cast<int32_t*>(w + L.err);
    a.cuts = reinterpret_cast<CutTile*>(w + L.cuts);
    a.part_s = reinterpret_cast<float*>(w + L.part_s);
    a.part_o = reinterpret_cast<float*>(w + L.part_o);
    return p;
}

}  // namespace

extern "C" {

int latent_check_config(const gblatent_config* cfg) { return check_cfg(cfg); }

size_t latent_workspace_size(const gblatent_config* cfg, int32_t T, int32_t B) {
    if (check_cfg(cfg) != GBMOE_OK || T < 0 || B < 0) return 0;
    return layout(cfg).total;
}

int latent_append(const gblatent_config* cfg, int32_t T, const gbattn_batch* batch, const gbattn_rows* kv, const void* gamma,
                  const gbattn_rows* q, const int32_t* positions, const uint64_t* table, const gblatent_cache* cache,
                  const gbattn_rows* kv_out, const gbattn_rows* q_out, void* stream) {
    if (int s = check_cfg(cfg)) return s;
    if (int s = check_batch(batch, T)) return s;
    if (T == 0 || batch->B == 0) return GBMOE_OK;
    if (int s = check_cache(cfg, cache)) return s;
    const int R = cfg->latent_dim, P = cfg->rope_dim, W = R + P;
    if (P > 0 && (!table || !aligned(table, 16))) return GBMOE_EINVAL;
    if (!aligned(positions, 4) || !aligned(gamma, 16)) return GBMOE_EINVAL;
    if (!rows_ok(cfg, kv, T, 1, W, false)) return GBMOE_EINVAL;
    const bool has_q = q_out && q_out->data, has_kv = kv_out && kv_out->data;
    if (has_q && (P == 0 || !rows_ok(cfg, q, T, cfg->heads, P, false) || !rows_ok(cfg, q_out, T, cfg->heads, P, true)))
        return GBMOE_EINVAL;
    if (has_kv && !rows_ok(cfg, kv_out, T, 1, W, true)) return GBMOE_EINVAL;
    LatentAppend p{};
    p.r = RopeParams{P, cfg->rotary_layout == GBATTN_HALF, cfg->rotary_scale, 1.0f, table};
    p.T = T; p.B = batch->B; p.R = R; p.act_dtype = cfg->act_dtype; p.eps = cfg->norm_eps;
    p.page = cfg->page; p.page_log2 = log2_of(p.page); p.max_pages = batch->max_pages; p.n_pages = cache->n_pages;
    p.cu_q = batch->cu_q; p.kv_len = batch->kv_len; p.page_table = batch->page_table; p.positions = positions;
    p.gamma = gamma; p.pool = cache->rows;
    p.kv = rows_of(kv, T, 1);
    if (has_kv) p.kv_out = rows_of(kv_out, T, 1);
    if (has_q) p.H = cfg->heads, p.q = rows_of(q, T, cfg->heads), p.q_out = rows_of(q_out, T, cfg->heads);
    return cuda_status(launch_latent_append(p, static_cast<cudaStream_t>(stream)));
}

int latent_prompt(const gblatent_config* cfg, int32_t Tq, int32_t Tk, int32_t B, const gbattn_rows* q, const gbattn_rows* k,
                  const gbattn_rows* k_rope, const gbattn_rows* v, const int32_t* cu_q, const int32_t* cu_k,
                  const gbattn_rows* out, float* lse, void* ws, size_t ws_bytes, void* stream) {
    if (int s = check_cfg(cfg)) return s;
    if (Tq < 0 || Tk < 0 || B < 0) return GBMOE_EINVAL;
    if (Tq > kMaxRows || Tk > kMaxRows || B > kMaxRows) return GBMOE_EUNSUPPORTED;
    if (int s = check_ws(cfg, ws, ws_bytes)) return s;
    if (Tq == 0 || B == 0) return GBMOE_OK;
    const int H = cfg->heads, P = cfg->rope_dim, N = cfg->nope_dim, V = cfg->value_dim;
    if (!cu_q || !cu_k || !aligned(cu_q, 4) || !aligned(cu_k, 4) || !aligned(lse, 4)) return GBMOE_EINVAL;
    if (!rows_ok(cfg, q, Tq, H, N + P, false) || !rows_ok(cfg, out, Tq, H, V, true)) return GBMOE_EINVAL;
    if (Tk > 0 && (!rows_ok(cfg, k, Tk, H, N, false) || !rows_ok(cfg, v, Tk, H, V, false) ||
                   (P > 0 && !rows_ok(cfg, k_rope, Tk, 1, P, false))))
        return GBMOE_EINVAL;
    LatentProblem p = problem(cfg, Tq, B, lse, ws);
    AttnProblem& a = p.a;
    a.Tk = Tk; a.Hkv = H; a.D = V; a.R = 1; a.cu_q = cu_q; a.cu_k = cu_k;
    a.q = rows_of(q, Tq, H); a.out = rows_of(out, Tq, H);
    p.K = N + P; p.own = N;
    if (Tk > 0) {
        a.k = rows_of(k, Tk, H), a.v = rows_of(v, Tk, H);
        if (P > 0) p.k_rope = rows_of(k_rope, Tk, 1);
    }
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return cuda_status(latent_prompt_tc_supported(p) ? launch_latent_prompt_tc(p, st) : launch_latent_simt(p, st));
}

int latent_cached(const gblatent_config* cfg, int32_t T, const gbattn_batch* batch, const gbattn_rows* q,
                  const gblatent_cache* cache, const gbattn_rows* out, float* lse, void* ws, size_t ws_bytes, void* stream) {
    if (int s = check_cfg(cfg)) return s;
    if (int s = check_batch(batch, T)) return s;
    if (int s = check_ws(cfg, ws, ws_bytes)) return s;
    if (T == 0 || batch->B == 0) return GBMOE_OK;
    if (int s = check_cache(cfg, cache)) return s;
    const int H = cfg->heads, R = cfg->latent_dim, W = R + cfg->rope_dim;
    if (!aligned(lse, 4)) return GBMOE_EINVAL;
    if (!rows_ok(cfg, q, T, H, W, false) || !rows_ok(cfg, out, T, H, R, true)) return GBMOE_EINVAL;
    if ((int64_t)T * H > kMaxRows || (int64_t)batch->max_pages * cfg->page > kMaxRows) return GBMOE_EUNSUPPORTED;
    LatentProblem p = problem(cfg, T, batch->B, lse, ws);
    AttnProblem& a = p.a;
    a.paged = 1; a.Hkv = 1; a.D = R; a.R = H;
    a.page = cfg->page; a.page_log2 = log2_of(a.page); a.max_pages = batch->max_pages; a.n_pages = cache->n_pages;
    a.cu_q = batch->cu_q; a.kv_len = batch->kv_len; a.page_table = batch->page_table; a.k_pool = cache->rows;
    a.q = rows_of(q, T, H); a.out = rows_of(out, T, H);
    p.K = W; p.own = W;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return cuda_status(latent_cached_tc_supported(p) ? launch_latent_cached_tc(p, st) : launch_latent_simt(p, st));
}

}  // extern "C"
