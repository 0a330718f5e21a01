// The residual's addition, the RMS norm and its rounding to 8 bits in one pass.
//
// A block has a row and keeps the sum (as rounded to the activations' type, which is
// what is normed) in registers, so x and the residual are read once and nothing is
// read back (H up to 8192; wider rows are read again for the second half). The sum of
// squares takes the elements in the order of moe_rmsnorm (lane p the pieces p, p + 32,
// .. one by one, then pairs of lanes), so the norm is the same bit for bit: one warp
// adds, on the rows in shared memory, while other blocks load and store.
//
// 8 bits: 128 columns are 16 lanes' pieces of the same number, so a block's maximum
// is four exchanges.
//
// Bound by HBM (three to four elements moved for one of arithmetic) for many rows: 8192 of 4096 with both outputs
// 47.5 us, 6.4 TB/s (a warp for a row, which holds it all in registers: 67.6); by one row's loads and the 8 H / 256
// dependent additions for few: 32 of 7168 5.5 us (11.9).
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

// 1 / sqrt(mean + eps) = rest * power, a power of two. Taken first, the power brings a row to about 1 without a rounding, so
// that its product with gamma leaves fp32's range only where the norm does too.
struct Inverse {
    float rest, power;
};

// A lane's piece of the result, to the outputs that there are.
template <typename TA>
__device__ __forceinline__ void finish(const NormAdd& p, int64_t t, int at, const Raw8<TA>& s, const Raw8<TA>& g, float inv, const Inverse& close) {
    float o[8];
    if (p.y) {
#pragma unroll
        for (int j = 0; j < 8; ++j) o[j] = __fmul_rn(__fmul_rn(s.at(j), inv), g.at(j));
        Vec8<TA>::store(static_cast<TA*>(p.y) + t * p.H + at, o);
    }
    if (!p.codes) return;
    // (bf16: the first two products are exact, so there is one rounding before the code's)
#pragma unroll
    for (int j = 0; j < 8; ++j) o[j] = __fmul_rn(__fmul_rn(__fmul_rn(s.at(j), close.power), g.at(j)), close.rest);
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
    if ((threadIdx.x & 15) == 0) p.scales[(t * p.H + at) >> 7] = pow2(e);
}

template <typename TA>
__device__ __forceinline__ void put(TA* dst, const Raw8<TA>& s) {
#pragma unroll
    for (int j = 0; j < (int)sizeof(TA) / 2; ++j) reinterpret_cast<uint4*>(dst)[j] = s.v[j];
}
template <typename TA>
__device__ __forceinline__ void add_squares(float& ss, const Raw8<TA>& s) {
#pragma unroll
    for (int j = 0; j < 8; ++j) ss = __fmaf_rn(s.at(j), s.at(j), ss);
}
// The squares once more, for the codes: eight sums and then a tree, whose roundings do not add up as those of the fixed
// order do (of 33.5 million codes 19 to 32 came out one step off the nearest with that order's sum).
template <typename TA>
__device__ __forceinline__ void add_squares8(float (&ss)[8], const Raw8<TA>& s) {
#pragma unroll
    for (int j = 0; j < 8; ++j) ss[j] = fmaf(s.at(j), s.at(j), ss[j]);
}
__device__ __forceinline__ float tree(const float (&ss)[8]) {
    float v = ((ss[0] + ss[1]) + (ss[2] + ss[3])) + ((ss[4] + ss[5]) + (ss[6] + ss[7]));
#pragma unroll
    for (int d = 16; d >= 1; d >>= 1) v += __shfl_xor_sync(kFull, v, d);
    return v;
}
__device__ __forceinline__ Inverse close_inverse(const NormAdd& p, float sum) {
    const float v = __frsqrt_rn(sum / (float)p.H + p.eps);
    const float power = __uint_as_float(__float_as_uint(v) & 0x7f800000u);
    if (!(power > 0.0f && power <= 3.402823466e38f)) return Inverse{v, 1.0f};  // (a row of zeros, of infinities, of NaN)
    return Inverse{__uint_as_float((__float_as_uint(v) & 0x007fffffu) | 0x3f800000u), power};
}
// 1 / sqrt(mean + eps) from the lanes' sums
__device__ __forceinline__ float inverse(const NormAdd& p, float ss) {
#pragma unroll
    for (int d = 16; d >= 1; d >>= 1) ss = __fadd_rn(ss, __shfl_xor_sync(kFull, ss, d));
    return __fdiv_rn(1.0f, __fsqrt_rn(__fadd_rn(__fdiv_rn(ss, (float)p.H), p.eps)));
}

// One row by a block: warp w has the 256 columns w, w + kWarps, .. (kHeld of them at most) in registers, and passes them
// through shared memory to the first warp, which adds their squares up in the fixed order.
constexpr int kWarps = 4;
template <typename TA, int kHeld>
__global__ void __launch_bounds__(32 * kWarps) norm_add_kernel(const __grid_constant__ NormAdd p) {
    pdl_enter();
    extern __shared__ uint4 rows[];
    __shared__ float scale, sums[kWarps];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, n = p.H / 256;
    const int64_t t = blockIdx.x;
    const TA* x = static_cast<const TA*>(p.x) + t * p.H;
    const TA* res = p.residual ? static_cast<const TA*>(p.residual) + t * p.H : nullptr;
    TA* sum = p.sum ? static_cast<TA*>(p.sum) + t * p.H : nullptr;
    TA* shared = reinterpret_cast<TA*>(rows);
    auto column = [&](int i) { return 256 * (warp + kWarps * i) + 8 * lane; };
    Raw8<TA> s[kHeld], r[kHeld], g[kHeld];
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
        if (warp + kWarps * i >= n) continue;
        s[i].load(x + column(i));
        if (res) r[i].load(res + column(i));
    }
#pragma unroll
    for (int i = 0; i < kHeld; ++i)
        if (warp + kWarps * i < n) g[i].load(static_cast<const TA*>(p.gamma) + column(i));
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
        if (warp + kWarps * i >= n) continue;
        add_piece(s[i], r[i], res != nullptr, s[i]);
        put(shared + column(i), s[i]);
        if (sum) put(sum + column(i), s[i]);
    }
    if (p.codes) {
        float ss[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < kHeld; ++i)
            if (warp + kWarps * i < n) add_squares8(ss, s[i]);
        const float v = tree(ss);
        if (lane == 0) sums[warp] = v;
    }
    __syncthreads();
    if (warp == 0 && p.y) {
        float ss = 0.0f;
#pragma unroll 4
        for (int i = 0; i < n; ++i) {
            Raw8<TA> v;
            v.load(shared + 256 * i + 8 * lane);
            add_squares(ss, v);
        }
        const float inv = inverse(p, ss);
        if (lane == 0) scale = inv;
    }
    if (p.y) __syncthreads();
    const float inv = p.y ? scale : 0.0f;
    Inverse close{};
    if (p.codes) close = close_inverse(p, (sums[0] + sums[1]) + (sums[2] + sums[3]));
#pragma unroll
    for (int i = 0; i < kHeld; ++i)
        if (warp + kWarps * i < n) finish(p, t, column(i), s[i], g[i], inv, close);
}

// Rows of any width, one by a warp, read twice.
template <typename TA>
__global__ void __launch_bounds__(128) norm_add_wide_kernel(const __grid_constant__ NormAdd p) {
    pdl_enter();
    const int lane = threadIdx.x & 31, n = p.H / 256;
    const int64_t t = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5);
    if (t >= p.T) return;
    const TA* x = static_cast<const TA*>(p.x) + t * p.H;
    const TA* res = p.residual ? static_cast<const TA*>(p.residual) + t * p.H : nullptr;
    TA* sum = p.sum ? static_cast<TA*>(p.sum) + t * p.H : nullptr;
    auto piece = [&](int i) {
        const int at = 256 * i + 8 * lane;
        Raw8<TA> a, b, s;
        a.load(x + at);
        if (res) b.load(res + at);
        add_piece(a, b, res != nullptr, s);
        return s;
    };
    float ss = 0.0f, ss8[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    for (int i = 0; i < n; ++i) {
        const Raw8<TA> s = piece(i);
        add_squares(ss, s);
        add_squares8(ss8, s);
    }
    const float inv = inverse(p, ss);
    const Inverse close = close_inverse(p, tree(ss8));
    for (int i = 0; i < n; ++i) {
        const int at = 256 * i + 8 * lane;
        const Raw8<TA> s = piece(i);
        Raw8<TA> g;
        g.load(static_cast<const TA*>(p.gamma) + at);
        if (sum) put(sum + at, s);  // (after both readings: it may be x or the residual)
        finish(p, t, at, s, g, inv, close);
    }
}

template <typename TA>
cudaError_t norm_add_as(const NormAdd& p, cudaStream_t stream) {
    const int n = p.H / 256, held = (n + kWarps - 1) / kWarps;
    auto run = [&](auto kernel) {
        return launch_k(kernel, dim3((unsigned)p.T), dim3(32 * kWarps), (size_t)p.H * sizeof(TA), stream, p);
    };
    if (held <= 1) return run(norm_add_kernel<TA, 1>);
    if (held <= 2) return run(norm_add_kernel<TA, 2>);
    if (held <= 4) return run(norm_add_kernel<TA, 4>);
    if (held <= 8) return run(norm_add_kernel<TA, 8>);
    return launch_k(norm_add_wide_kernel<TA>, dim3((unsigned)(((int64_t)p.T + 3) / 4)), dim3(128), 0, stream, p);
}

}  // namespace

cudaError_t launch_rmsnorm_add(const void* x, const void* residual, const void* gamma, float eps, int T, int H, int act_dtype,
                               void* sum, void* y, uint8_t* codes, float* scales, cudaStream_t stream) {
    const NormAdd p{x, residual, gamma, eps, T, H, sum, y, codes, scales};
    return act_dtype == GBMOE_BF16 ? norm_add_as<__nv_bfloat16>(p, stream) : norm_add_as<float>(p, stream);
}

}  // namespace gbmoe
