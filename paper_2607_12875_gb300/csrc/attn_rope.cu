// Rotary positions, and appending keys and values to the paged cache with the
// rotation on the way.
//
// Pair (a, b) number i of a head turns by position * f_i. The table holds f_i
// in turns as a binary fraction of 2^64, so the 64-bit product with the
// position, wrapped, is the fraction of a turn to 2^-64 * position, whatever
// the position; its top 32 bits, less the nearest quarter turn so that fp32 holds the
// rest to 2^-27 half turns, go to sincospif: an error of 2.4e-8 radians, below fp32's
// own on the rotated values (without the quarter: 9.4e-8, above it). A thread keeps the angles of its eight
// pairs of a token in registers and takes them through several heads. The rotation has
// no shared memory and no barrier; an append looks its page up through shared memory first, and
// one to e4m3 exchanges the maxima of a page and head through it between its loads and its rounding.
//
// Each element is read once and written once, but for e4m3 pages of more new tokens than a block takes
// at a time, whose keys and values are read twice. 8192 tokens, 32 query and 8 kv heads of 128, bf16: rotation
// 33 us, 5.1 TB/s, bound by HBM (768 blocks, 1.7 times what is resident); append of e4m3 with the queries 46 us,
// 4.0 TB/s (pages of 128, read twice: 8 % more), held back by one block of 512 threads on an SM between its loads and its rounding.

#include "attn_plan.cuh"
#include "attn_turn.cuh"
#include "e4m3.cuh"

namespace gbmoe {
namespace {

constexpr int kRopeThreads = 256;

// Heads of a thread whose loads are in flight together, on their own and with a
// key and a value row (8192 tokens, 32 + 8 heads of 128, us: rotation 36 with 4 heads,
// 33 with 2; append 50 with 4, 55 with 1).
template <typename TA>
constexpr int kTurnBatch = sizeof(TA) == 2 ? 2 : 1;
template <typename TA>
constexpr int kQueryBatch = sizeof(TA) == 2 ? 4 : 2;

// Block x, y: a thread takes one unit of one token through every `heads`-th head
// of q and k together, starting at its own. bits: log2 of the threads of a head.
template <typename TA>
__global__ void __launch_bounds__(kRopeThreads) rope_kernel(const __grid_constant__ RopeProblem p, int bits, int heads) {
    pdl_enter();
    constexpr int B = kTurnBatch<TA>;
    const int64_t i = (int64_t)blockIdx.x * kRopeThreads + threadIdx.x;
    const int u = (int)i & ((1 << bits) - 1);
    const int64_t rest = i >> bits;
    const int t = (int)(rest / heads), h0 = (int)(rest - (int64_t)t * heads), H = p.Hq + p.Hk;
    if (t >= p.T || u >= head_units(p.r.R, p.D)) return;
    const Unit unit = unit_of(p.r, p.D, u);
    const int64_t pos = p.r.R > 0 ? p.positions[t] : 0;
    Angles angles;
    for (int h = h0; h < H; h += B * heads) {
        Held<TA> held[B];
#pragma unroll
        for (int k = 0; k < B; ++k) {
            const int hh = h + k * heads;
            if (hh < H) held[k].load(unit, hh < p.Hq ? row<TA>(p.q, t, hh) : row<TA>(p.k, t, hh - p.Hq));
        }
        if (h == h0) angles.set(p.r, unit, pos);  // computed while the first loads are in flight
#pragma unroll
        for (int k = 0; k < B; ++k) {
            const int hh = h + k * heads;
            if (hh >= H) break;
            Values v;
            v.from(held[k], unit);
            v.turn(p.r, unit, angles);
            v.store(unit, hh < p.Hq ? row<TA>(p.q_out, t, hh) : row<TA>(p.k_out, t, hh - p.Hq));
        }
    }
}

// ------------------------------------------------------------------ append

// maximum of |v| and m, infinities and NaN left out where `careful` (else NaN alone)
__device__ __forceinline__ float max_abs(float m, const Values& v, bool careful) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float a = fabsf(v.x[j]), b = fabsf(v.y[j]);
        if (!careful) {
            m = fmaxf(m, fmaxf(a, b));
        } else {
            m = a <= 3.402823466e38f ? fmaxf(m, a) : m;  // (false for NaN)
            m = b <= 3.402823466e38f ? fmaxf(m, b) : m;
        }
    }
    return m;
}

// The new tokens of one sequence that fall into one of its pages.
struct PageTokens {
    int t0, n;      // its tokens
    int64_t pos;    // position of the first one in the sequence
    int page, off;  // pool page (-1: not stored) and slot of the first one
};

// PageTokens `index` (sequences in order, a sequence's pages in order). n = 0: none.
__device__ __forceinline__ PageTokens find_segment(const AppendProblem& p, int64_t index, int64_t* sm) {
    auto bounds = [&](int b, int& q0, int& n, int64_t& pos0) {
        q0 = min(max(p.cu_q[b], 0), p.T);
        n = min(max(p.cu_q[b + 1], q0), p.T) - q0;
        pos0 = (int64_t)p.kv_len[b] - n;
    };
    const int bits = p.page_log2;  // (shifts: pages before position 0 are negative)
    PageTokens s{};
    const Place at = find_place(
        p.B,
        [&](int b) {
            int q0, n;
            int64_t pos0;
            bounds(b, q0, n, pos0);
            return n > 0 ? ((pos0 + n - 1) >> bits) - (pos0 >> bits) + 1 : 0;
        },
        [&](int64_t) { return index; }, sm);
    if (at.b < 0) return s;
    int q0, n;
    int64_t pos0;
    bounds(at.b, q0, n, pos0);
    const int64_t pg = (pos0 >> bits) + at.at;
    const int64_t from = max64(pos0, pg << bits), to = min64(pos0 + n, (pg + 1) << bits);
    s.t0 = q0 + (int)(from - pos0);
    s.n = (int)(to - from);
    s.pos = from;
    s.off = (int)(from - (pg << bits));
    s.page = -1;
    if (pg >= 0 && pg < p.max_pages) {
        const int id = p.page_table[(int64_t)at.b * p.max_pages + pg];
        if (id >= 0 && id < p.n_pages) s.page = id;
    }
    return s;
}

// The threads that share a task: a warp, or the whole block.
template <bool kWarpTeam>
struct Team {
    int rank, size;
    float2* sm;  // block: one word per warp and value
    __device__ __forceinline__ Team(float2* s)
        : rank(kWarpTeam ? threadIdx.x & 31 : threadIdx.x), size(kWarpTeam ? 32 : blockDim.x), sm(s) {}
    // maxima of the team's a and b, to every thread
    __device__ __forceinline__ void max(float& a, float& b) const {
#pragma unroll
        for (int d = 16; d; d >>= 1) {
            a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, d));
            b = fmaxf(b, __shfl_xor_sync(0xffffffffu, b, d));
        }
        if (kWarpTeam) return;
        __syncthreads();
        if ((threadIdx.x & 31) == 0) sm[threadIdx.x >> 5] = make_float2(a, b);
        __syncthreads();
        for (int w = 0; w < (int)(blockDim.x >> 5); ++w) a = fmaxf(a, sm[w].x), b = fmaxf(b, sm[w].y);
    }
};

// The scale of one page and head that covers amax too, the page's earlier codes
// brought to it; returns the factor of the new values.
template <bool kWarpTeam>
__device__ __forceinline__ float rescale(const AppendProblem& p, const PageTokens& s, uint8_t* codes, uint8_t* scale, int old,
                                         float amax, const Team<kWarpTeam>& team) {
    const int e = ::max(old, scale_exponent(amax));
    if (s.off > 0 && e > old) {
        const float f = old - e >= -126 ? pow2(old - e) : 0.0f;
        for (int i = team.rank; i < s.off * p.D / 8; i += team.size) {
            const uint2 c = reinterpret_cast<uint2*>(codes)[i];
            const float2 v0 = e4m3x2_to_f32x2(c.x & 0xffffu), v1 = e4m3x2_to_f32x2(c.x >> 16);
            const float2 v2 = e4m3x2_to_f32x2(c.y & 0xffffu), v3 = e4m3x2_to_f32x2(c.y >> 16);
            const float w[8] = {v0.x, v0.y, v1.x, v1.y, v2.x, v2.y, v3.x, v3.y};
            reinterpret_cast<uint2*>(codes)[i] = e4m3x8(w, f);
        }
    }
    if (team.rank == 0) *scale = (uint8_t)(e + 127);
    return pow2(-e);  // (e >= -127: at most 2^127)
}

// A segment's keys and values of kv head h to the cache, its keys to k_out and the
// query heads of the group to q_out. A thread has one unit of every step-th
// token. e4m3: up to kHeld tokens of a thread stay in registers between the
// search for the maximum and the rounding; longer segments are read twice, and
// k_out, which may be k, is written at the last reading.
template <typename TA, bool kE4m3, bool kWarpTeam>
__device__ __forceinline__ void append_head(const AppendProblem& p, const PageTokens& s, int h, const Team<kWarpTeam>& team) {
    constexpr int kHeld = 1, B = kQueryBatch<TA>;
    const int units = head_units(p.r.R, p.D), bits = unit_bits(units);
    const int u = team.rank & ((1 << bits) - 1), step = team.size >> bits, first = team.rank >> bits;
    const int n = u < units ? s.n : 0;  // (threads without a unit have no rows)
    const Unit unit = unit_of(p.r, p.D, u);
    const int G = p.Hq / p.Hkv;
    const bool stored = s.page >= 0;
    const int64_t head = (int64_t)s.page * p.Hkv + h, slot0 = (head * p.page + s.off) * p.D;
    int old_k = -127, old_v = -127;
    if (kE4m3 && stored && s.off > 0) old_k = (int)p.k_scale[head] - 127, old_v = (int)p.v_scale[head] - 127;
    Values kv[kHeld];
    Held<TA> vh[kHeld];
    const bool once = s.n <= kHeld * step || !kE4m3 || !stored;  // k is read once
    float top_k = 0.0f, top_v = 0.0f;
    auto load = [&](int t0, bool queries, bool keys_out) {
        Held<TA> kh[kHeld];
#pragma unroll
        for (int k = 0; k < kHeld; ++k) {
            if (t0 + k * step >= n) break;
            kh[k].load(unit, row<TA>(p.k, s.t0 + t0 + k * step, h));
            vh[k].load(unit, row<TA>(p.v, s.t0 + t0 + k * step, h));
        }
#pragma unroll
        for (int k = 0; k < kHeld; ++k) {
            const int t = t0 + k * step, tok = s.t0 + t;
            if (t >= n) break;
            Angles angles;
            bool ready = false;
            if (queries)
                for (int g0 = 0; g0 < G; g0 += B) {
                    Held<TA> q[B];
#pragma unroll
                    for (int g = 0; g < B; ++g)
                        if (g0 + g < G) q[g].load(unit, row<TA>(p.q, tok, h * G + g0 + g));
                    if (!ready) angles.set(p.r, unit, p.positions ? (int64_t)p.positions[tok] : s.pos + t);
                    ready = true;
#pragma unroll
                    for (int g = 0; g < B; ++g) {
                        if (g0 + g >= G) break;
                        Values w;
                        w.from(q[g], unit);
                        w.turn(p.r, unit, angles);
                        w.store(unit, row<TA>(p.q_out, tok, h * G + g0 + g));
                    }
                }
            if (!ready) angles.set(p.r, unit, p.positions ? (int64_t)p.positions[tok] : s.pos + t);
            kv[k].from(kh[k], unit);
            kv[k].turn(p.r, unit, angles);
            if (keys_out && p.k_out.p) kv[k].store(unit, row<TA>(p.k_out, tok, h));
        }
    };
    auto maxima = [&](int t0, bool careful) {
#pragma unroll
        for (int k = 0; k < kHeld; ++k) {
            if (t0 + k * step >= n) break;
            Values w;
            w.from(vh[k], unit);
            top_k = max_abs(top_k, kv[k], careful);
            top_v = max_abs(top_v, w, careful);
        }
    };
    auto write = [&](int t0, float inv_k, float inv_v) {
#pragma unroll
        for (int k = 0; k < kHeld; ++k) {
            const int t = t0 + k * step;
            if (t >= n) break;
            Values w;
            w.from(vh[k], unit);
            if constexpr (kE4m3) {
                uint8_t* dk = static_cast<uint8_t*>(p.k_pool) + slot0 + t * p.D;
                uint8_t* dv = static_cast<uint8_t*>(p.v_pool) + slot0 + t * p.D;
                *reinterpret_cast<uint2*>(dk + unit.first) = e4m3x8(kv[k].x, inv_k);
                *reinterpret_cast<uint2*>(dv + unit.first) = e4m3x8(w.x, inv_v);
                if (unit.second < 0) continue;
                *reinterpret_cast<uint2*>(dk + unit.second) = e4m3x8(kv[k].y, inv_k);
                *reinterpret_cast<uint2*>(dv + unit.second) = e4m3x8(w.y, inv_v);
            } else {
                kv[k].store(unit, static_cast<TA*>(p.k_pool) + slot0 + t * p.D);
                w.store(unit, static_cast<TA*>(p.v_pool) + slot0 + t * p.D);
            }
        }
    };
    for (int t0 = first; t0 < n; t0 += kHeld * step) {
        load(t0, true, once);
        if (kE4m3) maxima(t0, false);
        else if (stored) write(t0, 1.0f, 1.0f);
    }
    if constexpr (kE4m3) {
        if (!stored) return;  // (uniform)
        team.max(top_k, top_v);
        if (top_k > 3.402823466e38f || top_v > 3.402823466e38f) {  // an infinity: once more without
            top_k = top_v = 0.0f;
            for (int t0 = first; t0 < n; t0 += kHeld * step) {
                if (!once) load(t0, false, false);
                maxima(t0, true);
            }
            team.max(top_k, top_v);
        }
        // (the maxima's exchange has come after every thread's read of the old scales)
        uint8_t* page = static_cast<uint8_t*>(p.k_pool) + head * p.page * p.D;
        const float inv_k = rescale(p, s, page, p.k_scale + head, old_k, top_k, team);
        page = static_cast<uint8_t*>(p.v_pool) + head * p.page * p.D;
        const float inv_v = rescale(p, s, page, p.v_scale + head, old_v, top_v, team);
        for (int t0 = first; t0 < n; t0 += kHeld * step) {
            if (!once) load(t0, false, true);
            write(t0, inv_k, inv_v);
        }
    }
}

// Block x: segment x / Hkv, kv head x % Hkv by the whole block; or (kWarpTeam, few
// tokens per sequence) segment x, its kv heads dealt to the warps. One team owns
// a page and head, so its scale needs no atomics.
template <typename TA, bool kE4m3, bool kWarpTeam, int kThreads>
__global__ void __launch_bounds__(kThreads, kWarpTeam || kThreads == 512 ? 1 : 2) append_kernel(const __grid_constant__ AppendProblem p) {
    pdl_enter();
    __shared__ int64_t plan[plan_words(kThreads)];
    __shared__ float2 red[kThreads / 32];
    const PageTokens s = find_segment(p, kWarpTeam ? blockIdx.x : blockIdx.x / p.Hkv, plan);
    if (s.n == 0) return;
    const Team<kWarpTeam> team(red);
    if constexpr (kWarpTeam) {
        for (int h = threadIdx.x >> 5; h < p.Hkv; h += blockDim.x / 32) append_head<TA, kE4m3, true>(p, s, h, team);
    } else {
        append_head<TA, kE4m3, false>(p, s, blockIdx.x % p.Hkv, team);
    }
}

template <typename TA>
cudaError_t rope_as(const RopeProblem& p, cudaStream_t stream) {
    const int H = p.Hq + p.Hk, bits = unit_bits(head_units(p.r.R, p.D));
    // Threads of a token over its heads: a thread's angles cost about as much as four
    // units of work, so it takes as many heads as leave 1024 threads for each SM.
    int heads = H;
    while (heads > 1 && ((int64_t)p.T * ((heads + 1) / 2) << bits) >= (int64_t)1024 * sm_count()) heads = (heads + 1) / 2;
    const int64_t grid = (((int64_t)p.T * heads << bits) + kRopeThreads - 1) / kRopeThreads;
    if (grid > INT32_MAX) return cudaErrorInvalidConfiguration;
    return launch_k(rope_kernel<TA>, dim3((unsigned)grid), dim3(kRopeThreads), 0, stream, p, bits, heads);
}

template <typename TA, bool kE4m3, bool kWarpTeam, int kThreads>
cudaError_t append_as(const AppendProblem& p, int threads, cudaStream_t stream) {
    const int64_t segs = min64(p.T, (int64_t)p.T / p.page + 2 * (int64_t)p.B);
    const int64_t grid = kWarpTeam ? segs : segs * p.Hkv;
    if (grid > INT32_MAX) return cudaErrorInvalidConfiguration;
    threads = threads < 64 ? 64 : threads < kThreads ? threads : kThreads;
    return launch_k(append_kernel<TA, kE4m3, kWarpTeam, kThreads>, dim3((unsigned)grid), dim3((unsigned)threads), 0, stream, p);
}

template <typename TA, bool kE4m3>
cudaError_t append_type(const AppendProblem& p, cudaStream_t stream) {
    // few tokens per sequence: a head is a warp's work
    if (p.T <= 4 * (int64_t)p.B) return append_as<TA, kE4m3, true, 256>(p, 32 * p.Hkv, stream);
    // else a thread for each unit of a page's tokens. One block of 512 fills an SM's registers, but
    // spares e4m3 a second reading of its values: 8192 tokens of 8 kv heads, D 128, pages of 64 in 47 us,
    // with blocks of 256 58. Other caches take two blocks of 256 on an SM: 1583 tokens, 4 kv heads of 64, pages of 128
    // 9.4 us (blocks of 512: 14.4).
    const int threads = p.page << unit_bits(head_units(p.r.R, p.D));
    return kE4m3 && threads > 256 ? append_as<TA, kE4m3, false, kE4m3 ? 512 : 256>(p, threads, stream)
                                  : append_as<TA, kE4m3, false, 256>(p, threads, stream);
}

}  // namespace

cudaError_t launch_rope(const RopeProblem& p, cudaStream_t stream) {
    return p.act_dtype == GBMOE_F32 ? rope_as<float>(p, stream) : rope_as<__nv_bfloat16>(p, stream);
}

cudaError_t launch_append(const AppendProblem& p, cudaStream_t stream) {
    if (p.act_dtype == GBMOE_F32) return p.e4m3 ? append_type<float, true>(p, stream) : append_type<float, false>(p, stream);
    return p.e4m3 ? append_type<__nv_bfloat16, true>(p, stream) : append_type<__nv_bfloat16, false>(p, stream);
}

}  // namespace gbmoe
