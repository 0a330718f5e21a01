// C ABI of the attention operators (declared in include/gbattn.h): argument
// checks on the host and the choice of kernels.
#include <cmath>
#include <cstdint>

#include "api_status.h"
#include "attn.h"

using namespace gbmoe;

namespace {

constexpr size_t kAlign = 256;
constexpr int kMaxHeads = 4096;
constexpr int kMaxRows = 1 << 30;  // tokens, query rows of a sequence (tokens times G), keys: the kernels count them in 32 bits

int log2_of(int v) {
    int b = 0;
    while (1 << b < v) ++b;
    return b;
}
size_t align_up(size_t v) { return (v + kAlign - 1) & ~(kAlign - 1); }
size_t act_bytes(int act) { return act == GBMOE_F32 ? 4 : 2; }
bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

int check_cfg(const gbattn_config* c) {
    if (!c) return GBMOE_EINVAL;
    if (c->heads_q <= 0 || c->heads_kv <= 0 || c->heads_q % c->heads_kv != 0 || c->head_dim <= 0) return GBMOE_EINVAL;
    if (c->act_dtype != GBMOE_F32 && c->act_dtype != GBMOE_BF16) return GBMOE_EINVAL;
    if ((c->causal != 0 && c->causal != 1) || c->window < 0) return GBMOE_EINVAL;
    if (!std::isfinite(c->scale) || !std::isfinite(c->rotary_scale)) return GBMOE_EINVAL;
    if (c->rotary_dim < 0 || c->rotary_dim > c->head_dim) return GBMOE_EINVAL;
    if (c->rotary_layout != GBATTN_HALF && c->rotary_layout != GBATTN_INTERLEAVED) return GBMOE_EINVAL;
    if (c->cache_dtype != GBATTN_CACHE_ACT && c->cache_dtype != GBATTN_CACHE_E4M3) return GBMOE_EINVAL;
    if (c->page <= 0) return GBMOE_EINVAL;
    // what the kernels cover
    if (c->head_dim % 8 != 0 || c->head_dim > 256 || c->heads_q > kMaxHeads) return GBMOE_EUNSUPPORTED;
    if (c->rotary_dim % 16 != 0) return GBMOE_EUNSUPPORTED;
    if (c->page != 16 && c->page != 32 && c->page != 64 && c->page != 128) return GBMOE_EUNSUPPORTED;
    return GBMOE_OK;
}

// rows [T, heads, D] that the kernels read (or, out = true, write: then no two
// of them may share an element)
bool rows_ok(const gbattn_config* c, const gbattn_rows* r, int64_t T, int64_t heads, bool out) {
    if (!r || !r->data || !aligned(r->data, 16)) return false;
    const int64_t eb = (int64_t)act_bytes(c->act_dtype), D = c->head_dim;
    if (r->token_stride < 0 || r->head_stride < 0) return false;
    if (T > 1 && r->token_stride * eb % 16 != 0) return false;
    if (heads > 1 && r->head_stride * eb % 16 != 0) return false;
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

int check_cache(const gbattn_config* c, const gbattn_cache* k) {
    if (!k || !k->k || !k->v || k->n_pages < 0 || !aligned(k->k, 16) || !aligned(k->v, 16)) return GBMOE_EINVAL;
    if (c->cache_dtype == GBATTN_CACHE_E4M3 && (!k->k_scale || !k->v_scale)) return GBMOE_EINVAL;
    return GBMOE_OK;
}

struct Layout {
    size_t err, cuts, part_s, part_o, total;
};

Layout layout(const gbattn_config* c) {
    Layout L{};
    size_t o = 0;
    auto take = [&](size_t bytes) { size_t at = o; o = align_up(o + bytes); return at; };
    const size_t rows = (size_t)2 * kMaxShares * kMaxTileRows;
    L.err = take(4);
    L.cuts = take(kMaxShares * sizeof(CutTile));
    L.part_s = take(rows * 16);
    L.part_o = take(rows * c->head_dim * 4);
    L.total = o;
    return L;
}

int check_ws(const gbattn_config* c, void* ws, size_t bytes) {
    if (!ws || !aligned(ws, kAlign)) return GBMOE_EINVAL;
    return bytes < layout(c).total ? GBMOE_EWORKSPACE : GBMOE_OK;
}

RopeParams rope_params(const gbattn_config* c, const uint64_t* table, bool inverse) {
    return RopeParams{c->rotary_dim, c->rotary_layout == GBATTN_HALF, c->rotary_scale, inverse ? -1.0f : 1.0f, table};
}

AttnProblem problem(const gbattn_config* c, int32_t T, int32_t B, const gbattn_rows* q, const gbattn_rows* out, float* lse,
                    void* ws) {
    const Layout L = layout(c);
    char* w = static_cast<char*>(ws);
    AttnProblem p{};
    p.B = B; p.T = T; p.Hq = c->heads_q; p.Hkv = c->heads_kv; p.D = c->head_dim;
    p.act_dtype = c->act_dtype; p.causal = c->causal; p.window = c->window;
    p.scale_log2 = c->scale * 1.4426950408889634f;
    p.q = rows_of(q, T, c->heads_q);
    p.out = rows_of(out, T, c->heads_q);
    p.lse = lse;
    p.page = 1;
    p.err = reinterpret_cast<int32_t*>(w + L.err);
    p.cuts = reinterpret_cast<CutTile*>(w + L.cuts);
    p.part_s = reinterpret_cast<float*>(w + L.part_s);
    p.part_o = reinterpret_cast<float*>(w + L.part_o);
    return p;
}

}  // namespace

extern "C" {

int attn_check_config(const gbattn_config* cfg) { return check_cfg(cfg); }

size_t attn_workspace_size(const gbattn_config* cfg, int32_t T, int32_t B) {
    if (check_cfg(cfg) != GBMOE_OK || T < 0 || B < 0) return 0;
    return layout(cfg).total;
}

int attn_rope_table(int32_t rotary_dim, double base, int32_t scaling, double factor, double original_ctx, double slow,
                    double fast, uint64_t* table) {
    if (rotary_dim <= 0 || rotary_dim % 2 != 0 || !table) return GBMOE_EINVAL;
    if (!(base > 1.0) || !std::isfinite(base) || !(factor > 0.0) || !std::isfinite(factor)) return GBMOE_EINVAL;
    if (scaling < GBATTN_ROPE_PLAIN || scaling > GBATTN_ROPE_RAMP) return GBMOE_EINVAL;
    if (scaling == GBATTN_ROPE_NTK && rotary_dim <= 2) return GBMOE_EINVAL;
    const double R = rotary_dim, two_pi = 6.283185307179586476925;
    double lo = 0.0, hi = 0.0;
    if (scaling == GBATTN_ROPE_RAMP) {
        if (!(original_ctx > 0.0) || !(slow > 0.0) || !(fast > slow) || !std::isfinite(original_ctx) || !std::isfinite(fast))
            return GBMOE_EINVAL;
        // the (fractional) index whose pair turns n times within the original context
        auto index_of = [&](double n) { return R * std::log(original_ctx / (n * two_pi)) / (2.0 * std::log(base)); };
        lo = std::fmax(std::floor(index_of(fast)), 0.0);
        hi = std::fmin(std::ceil(index_of(slow)), R - 1.0);
    }
    if (scaling == GBATTN_ROPE_NTK) base *= std::pow(factor, R / (R - 2.0));
    for (int i = 0; i < rotary_dim / 2; ++i) {
        double f = std::pow(base, -2.0 * i / R);
        if (scaling == GBATTN_ROPE_LINEAR) f /= factor;
        if (scaling == GBATTN_ROPE_RAMP) {
            const double ramp = std::fmin(1.0, std::fmax(0.0, (i - lo) / std::fmax(hi - lo, 1e-3)));
            f = f * (1.0 - ramp) + f / factor * ramp;
        }
        double t = f / two_pi;
        t -= std::floor(t);
        table[i] = (uint64_t)std::ldexp(t, 64);  // t < 1
    }
    return GBMOE_OK;
}

int attn_rope(const gbattn_config* cfg, int32_t T, const gbattn_rows* q, const gbattn_rows* k, const int32_t* positions,
              const uint64_t* table, int32_t inverse, const gbattn_rows* q_out, const gbattn_rows* k_out, void* stream) {
    if (int s = check_cfg(cfg)) return s;
    if (T < 0 || (inverse != 0 && inverse != 1)) return GBMOE_EINVAL;
    if (T > kMaxRows) return GBMOE_EUNSUPPORTED;
    const bool has_q = q && q->data, has_k = k && k->data;
    if (!has_q && !has_k) return GBMOE_EINVAL;
    if (T == 0) return GBMOE_OK;
    if (cfg->rotary_dim > 0 && (!positions || !table || !aligned(positions, 4) || !aligned(table, 16))) return GBMOE_EINVAL;
    if (has_q && (!rows_ok(cfg, q, T, cfg->heads_q, false) || !rows_ok(cfg, q_out, T, cfg->heads_q, true))) return GBMOE_EINVAL;
    if (has_k && (!rows_ok(cfg, k, T, cfg->heads_kv, false) || !rows_ok(cfg, k_out, T, cfg->heads_kv, true)))
        return GBMOE_EINVAL;
    RopeProblem p{};
    p.r = rope_params(cfg, table, inverse == 1);
    p.T = T; p.D = cfg->head_dim; p.act_dtype = cfg->act_dtype; p.positions = positions;
    if (has_q) p.Hq = cfg->heads_q, p.q = rows_of(q, T, cfg->heads_q), p.q_out = rows_of(q_out, T, cfg->heads_q);
    if (has_k) p.Hk = cfg->heads_kv, p.k = rows_of(k, T, cfg->heads_kv), p.k_out = rows_of(k_out, T, cfg->heads_kv);
    return cuda_status(launch_rope(p, static_cast<cudaStream_t>(stream)));
}

int attn_append(const gbattn_config* cfg, int32_t T, const gbattn_batch* batch, const gbattn_rows* q, const gbattn_rows* k,
                const gbattn_rows* v, const int32_t* positions, const uint64_t* table, const gbattn_cache* cache,
                const gbattn_rows* q_out, const gbattn_rows* k_out, void* stream) {
    if (int s = check_cfg(cfg)) return s;
    if (int s = check_batch(batch, T)) return s;
    if (T == 0 || batch->B == 0) return GBMOE_OK;
    if (int s = check_cache(cfg, cache)) return s;
    if (cfg->rotary_dim > 0 && (!table || !aligned(table, 16))) return GBMOE_EINVAL;
    if (positions && !aligned(positions, 4)) return GBMOE_EINVAL;
    if (!rows_ok(cfg, k, T, cfg->heads_kv, false) || !rows_ok(cfg, v, T, cfg->heads_kv, false)) return GBMOE_EINVAL;
    const bool has_q = q_out && q_out->data, has_k = k_out && k_out->data;
    if (has_q && (!rows_ok(cfg, q, T, cfg->heads_q, false) || !rows_ok(cfg, q_out, T, cfg->heads_q, true))) return GBMOE_EINVAL;
    if (has_k && !rows_ok(cfg, k_out, T, cfg->heads_kv, true)) return GBMOE_EINVAL;
    AppendProblem p{};
    p.r = rope_params(cfg, table, false);
    p.T = T; p.B = batch->B; p.D = cfg->head_dim; p.Hkv = cfg->heads_kv;
    p.act_dtype = cfg->act_dtype; p.e4m3 = cfg->cache_dtype == GBATTN_CACHE_E4M3;
    p.page = cfg->page; p.max_pages = batch->max_pages; p.n_pages = cache->n_pages;
    p.page_log2 = log2_of(p.page);
    p.cu_q = batch->cu_q; p.kv_len = batch->kv_len; p.page_table = batch->page_table; p.positions = positions;
    p.k = rows_of(k, T, cfg->heads_kv);
    p.v = rows_of(v, T, cfg->heads_kv);
    if (has_q) p.Hq = cfg->heads_q, p.q = rows_of(q, T, cfg->heads_q), p.q_out = rows_of(q_out, T, cfg->heads_q);
    if (has_k) p.k_out = rows_of(k_out, T, cfg->heads_kv);
    p.k_pool = cache->k; p.v_pool = cache->v; p.k_scale = cache->k_scale; p.v_scale = cache->v_scale;
    return cuda_status(launch_append(p, static_cast<cudaStream_t>(stream)));
}

int attn_prompt(const gbattn_config* cfg, int32_t Tq, int32_t Tk, int32_t B, const gbattn_rows* q, const gbattn_rows* k,
                const gbattn_rows* v, const int32_t* cu_q, const int32_t* cu_k, const gbattn_rows* out, float* lse,
                void* ws, size_t ws_bytes, void* stream) {
    if (int s = check_cfg(cfg)) return s;
    if (Tq < 0 || Tk < 0 || B < 0) return GBMOE_EINVAL;
    if (Tq > kMaxRows || Tk > kMaxRows || B > kMaxRows) return GBMOE_EUNSUPPORTED;
    if (int s = check_ws(cfg, ws, ws_bytes)) return s;
    if (Tq == 0 || B == 0) return GBMOE_OK;
    if (!cu_q || !cu_k || !aligned(cu_q, 4) || !aligned(cu_k, 4) || !aligned(lse, 4)) return GBMOE_EINVAL;
    if (!rows_ok(cfg, q, Tq, cfg->heads_q, false) || !rows_ok(cfg, out, Tq, cfg->heads_q, true)) return GBMOE_EINVAL;
    if (Tk > 0 && (!rows_ok(cfg, k, Tk, cfg->heads_kv, false) || !rows_ok(cfg, v, Tk, cfg->heads_kv, false)))
        return GBMOE_EINVAL;
    AttnProblem p = problem(cfg, Tq, B, q, out, lse, ws);
    p.Tk = Tk; p.cu_q = cu_q; p.cu_k = cu_k; p.R = 1;
    if (Tk > 0) p.k = rows_of(k, Tk, cfg->heads_kv), p.v = rows_of(v, Tk, cfg->heads_kv);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return cuda_status(attn_prompt_tc_supported(p) ? launch_attn_prompt_tc(p, st) : launch_attn_simt(p, st));
}

int attn_cached(const gbattn_config* cfg, int32_t T, const gbattn_batch* batch, const gbattn_rows* q,
                const gbattn_cache* cache, const gbattn_rows* out, float* lse, void* ws, size_t ws_bytes, void* stream) {
    if (int s = check_cfg(cfg)) return s;
    if (int s = check_batch(batch, T)) return s;
    if (int s = check_ws(cfg, ws, ws_bytes)) return s;
    if (T == 0 || batch->B == 0) return GBMOE_OK;
    if (int s = check_cache(cfg, cache)) return s;
    if (!aligned(lse, 4)) return GBMOE_EINVAL;
    if (!rows_ok(cfg, q, T, cfg->heads_q, false) || !rows_ok(cfg, out, T, cfg->heads_q, true)) return GBMOE_EINVAL;
    if ((int64_t)T * (cfg->heads_q / cfg->heads_kv) > kMaxRows || (int64_t)batch->max_pages * cfg->page > kMaxRows)
        return GBMOE_EUNSUPPORTED;
    AttnProblem p = problem(cfg, T, batch->B, q, out, lse, ws);
    p.paged = 1; p.e4m3 = cfg->cache_dtype == GBATTN_CACHE_E4M3; p.R = cfg->heads_q / cfg->heads_kv;
    p.page = cfg->page; p.max_pages = batch->max_pages; p.n_pages = cache->n_pages;
    p.cu_q = batch->cu_q; p.kv_len = batch->kv_len; p.page_table = batch->page_table;
    p.k_pool = cache->k; p.v_pool = cache->v; p.k_scale = cache->k_scale; p.v_scale = cache->v_scale;
    p.page_log2 = log2_of(p.page);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return cuda_status(attn_split_supported(p) ? launch_attn_split(p, st) : launch_attn_simt(p, st));
}

}  // extern "C"
