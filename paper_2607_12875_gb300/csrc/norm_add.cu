// The residual's addition, the RMS norm and its rounding to 8 bits in one pass.
//
// A warp has a row and keeps the sum (as rounded to the activations' type, which is
// what is normed) in registers, so x and the residual are read once and nothing is
// read back: up to 32 pieces of eight elements a lane (H up to 8192); wider rows are
// read again for the second half. The sum of squares takes the elements in the order
// of moe_rmsnorm (lane p the pieces p, p + 32, .. one by one, then pairs of lanes),
// so the norm is the same bit for bit, whatever the launch.
//
// 8 bits: 128 columns are 16 lanes' pieces of the same number, so a block's maximum
// is four exchanges.
//
// Bound by HBM (three to four elements moved for one of arithmetic) for many rows,
// by one row's chain of loads and 8 H / 256 dependent additions for few.
#include "common.cuh"
#include "e4m3.cuh"
#include "kernels.h"

namespace gbmoe {
namespace {

constexpr unsigned kFull = 0xffffffffu;

// 2^e of a block of 128 columns with this largest absolute value
__device__ __forceinline__ int block_exponent(float amax) { return max(scale_exponent(amax), -126); }

struct NormAdd {
    const void *x, *residual, *gamma;
    float eps;
    int T, H;
    void *sum, *y;
    uint8_t* codes;
    float* scales;
};

// The sum of one piece, rounded to the activations' type.
template <typename TA>
__device__ __forceinline__ void add_piece(const Raw8<TA>& a, const Raw8<TA>& b, bool both, Raw8<TA>& s) {
    if (!both) {
        s = a;
        return;
    }
    if constexpr (sizeof(TA) == 4) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
            s.v[i] = make_uint4(__float_as_uint(__fadd_rn(a.at(4 * i), b.at(4 * i))), __float_as_uint(__fadd_rn(a.at(4 * i + 1), b.at(4 * i + 1))),
                                __float_as_uint(__fadd_rn(a.at(4 * i + 2), b.at(4 * i + 2))),
                                __float_as_uint(__fadd_rn(a.at(4 * i + 3), b.at(4 * i + 3))));
    } else {
        s.v[0] = make_uint4(pack_bf16x2(a.at(0) + b.at(0), a.at(1) + b.at(1)), pack_bf16x2(a.at(2) + b.at(2), a.at(3) + b.at(3)),
                            pack_bf16x2(a.at(4) + b.at(4), a.at(5) + b.at(5)), pack_bf16x2(a.at(6) + b.at(6), a.at(7) + b.at(7)));
    }
}

// One row by one warp. kHeld: pieces of a lane that stay in registers (0: none, they are read again).
template <typename TA, int kHeld>
__global__ void __launch_bounds__(128) norm_add_kernel(const __grid_constant__ NormAdd p) {
    pdl_enter();
    const int lane = threadIdx.x & 31;
    const int64_t t = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5);
    if (t >= p.T) return;
    const int pieces = p.H / 8;  // a multiple of 32: every lane has as many
    const TA* x = static_cast<const TA*>(p.x) + t * p.H;
    const TA* res = p.residual ? static_cast<const TA*>(p.residual) + t * p.H : nullptr;
    TA* sum = p.sum ? static_cast<TA*>(p.sum) + t * p.H : nullptr;
    const int n = pieces / 32;
    constexpr int kKept = kHeld > 0 ? kHeld : 1;
    Raw8<TA> kept[kKept];
    float ss = 0.0f;
    auto square = [&](const Raw8<TA>& s) {
#pragma unroll
        for (int j = 0; j < 8; ++j) ss = __fmaf_rn(s.at(j), s.at(j), ss);
    };
    auto put = [&](TA* dst, const Raw8<TA>& s) {
#pragma unroll
        for (int j = 0; j < (int)sizeof(TA) / 2; ++j) reinterpret_cast<uint4*>(dst)[j] = s.v[j];
    };
    constexpr int kBatch = sizeof(TA) == 2 ? 8 : 4;  // pieces of both terms in flight
    if constexpr (kHeld > 0) {
#pragma unroll
        for (int i0 = 0; i0 < kHeld; i0 += kBatch) {
            Raw8<TA> b[kBatch];
#pragma unroll
            for (int i = 0; i < kBatch; ++i) {
                if (i0 + i >= kHeld || i0 + i >= n) continue;
                const int at = 8 * (lane + 32 * (i0 + i));
                kept[i0 + i].load(x + at);
                if (res) b[i].load(res + at);
            }
#pragma unroll
            for (int i = 0; i < kBatch; ++i) {
                if (i0 + i >= kHeld || i0 + i >= n) continue;
                add_piece(kept[i0 + i], b[i], res != nullptr, kept[i0 + i]);
                if (sum) put(sum + 8 * (lane + 32 * (i0 + i)), kept[i0 + i]);
                square(kept[i0 + i]);
            }
        }
    } else {
        for (int i = 0; i < n; ++i) {
            const int at = 8 * (lane + 32 * i);
            Raw8<TA> a, b, s;
            a.load(x + at);
            if (res) b.load(res + at);
            add_piece(a, b, res != nullptr, s);
            square(s);
        }
    }
#pragma unroll
    for (int d = 16; d >= 1; d >>= 1) ss = __fadd_rn(ss, __shfl_xor_sync(kFull, ss, d));
    const float ms = __fdiv_rn(ss, (float)p.H);
    const float inv = __fdiv_rn(1.0f, __fsqrt_rn(__fadd_rn(ms, p.eps)));
    auto finish = [&](int i, const Raw8<TA>& s) {
        const int at = 8 * (lane + 32 * i);
        float g[8], o[8];
        Vec8<TA>::load(static_cast<const TA*>(p.gamma) + at, g);
#pragma unroll
        for (int j = 0; j < 8; ++j) o[j] = __fmul_rn(__fmul_rn(s.at(j), inv), g[j]);
        if (p.y) Vec8<TA>::store(static_cast<TA*>(p.y) + t * p.H + at, o);
        if (p.codes) {
            float top = 0.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float a = fabsf(o[j]);
                top = a <= 3.402823466e38f ? fmaxf(top, a) : top;  // (false for infinities and NaN)
            }
#pragma unroll
            for (int d = 8; d >= 1; d >>= 1) top = fmaxf(top, __shfl_xor_sync(kFull, top, d));
            const int e = block_exponent(top);
            *reinterpret_cast<uint2*>(p.codes + t * p.H + at) = e4m3x8(o, pow2(-e));  // (-e <= 126)
            if ((lane & 15) == 0) p.scales[(t * p.H + at) >> 7] = pow2(e);
        }
    };
    if constexpr (kHeld > 0) {
#pragma unroll
        for (int i = 0; i < kHeld; ++i)
            if (i < n) finish(i, kept[i]);
    } else {
        for (int i = 0; i < n; ++i) {
            const int at = 8 * (lane + 32 * i);
            Raw8<TA> a, b, s;
            a.load(x + at);
            if (res) b.load(res + at);
            add_piece(a, b, res != nullptr, s);
            if (sum) put(sum + at, s);  // (after both readings: it may be x or the residual)
            finish(i, s);
        }
    }
}

template <typename TA>
cudaError_t norm_add_as(const NormAdd& p, cudaStream_t stream) {
    const dim3 grid((unsigned)(((int64_t)p.T + 3) / 4));
    auto run = [&](auto kernel) { return launch_k(kernel, grid, dim3(128), 0, stream, p); };
    const int n = p.H / 256;
    if (n <= 8) return run(norm_add_kernel<TA, 8>);
    if (n <= 16) return run(norm_add_kernel<TA, 16>);
    if (sizeof(TA) == 2 && n <= 32) return run(norm_add_kernel<TA, sizeof(TA) == 2 ? 32 : 16>);
    return run(norm_add_kernel<TA, 0>);
}

}  // namespace

cudaError_t launch_rmsnorm_add(const void* x, const void* residual, const void* gamma, float eps, int T, int H, int act_dtype,
                               void* sum, void* y, uint8_t* codes, float* scales, cudaStream_t stream) {
    const NormAdd p{x, residual, gamma, eps, T, H, sum, y, codes, scales};
    return act_dtype == GBMOE_BF16 ? norm_add_as<__nv_bfloat16>(p, stream) : norm_add_as<float>(p, stream);
}

}  // namespace gbmoe
