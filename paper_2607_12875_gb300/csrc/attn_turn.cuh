// Device pieces of the rotations: angles from the 64-bit table (the arithmetic and its
// errors are described in attn_rope.cu), units of 16 elements of a head, and rows.
#pragma once

#include "attn.h"
#include "common.cuh"

namespace gbmoe {

// (cos, sin) at position pos of the pair that turns by `entry` per position
__device__ __forceinline__ float2 turn(const RopeParams& r, int64_t pos, uint64_t entry) {
    const uint32_t f = (uint32_t)((uint64_t)pos * entry >> 32);
    const uint32_t quarter = (f + 0x20000000u) >> 30;  // the nearest quarter turn
    float s, c;
    sincospif((float)(int32_t)(f - (quarter << 30)) * 4.656612873077393e-10f, &s, &c);  // 2^-31: half turns
    float2 cs = quarter & 1u ? make_float2(-s, c) : make_float2(c, s);
    if (quarter & 2u) cs = make_float2(-cs.x, -cs.y);
    return make_float2(cs.x * r.mag, cs.y * r.mag * r.sin_sign);
}

// A head's units of 16 elements: R / 16 of eight pairs that turn, then the
// elements that do not (the last unit may be 8).
struct Unit {
    int first, second;  // offsets of its two halves (second -1: none)
    int index;          // its number; below R / 16: it turns
};
__host__ __device__ __forceinline__ int head_units(int R, int D) { return (R >> 4) + ((D - R + 15) >> 4); }
__device__ __forceinline__ Unit unit_of(const RopeParams& r, int D, int u) {
    if (u < r.R >> 4) {
        const int first = r.half ? 8 * u : 16 * u;
        return Unit{first, r.half ? first + (r.R >> 1) : first + 8, u};
    }
    const int first = 16 * u;
    return Unit{first, first + 8 < D ? first + 8 : -1, u};
}
// log2 of the threads that a head's units are dealt to
__host__ __device__ __forceinline__ int unit_bits(int units) {
    int b = 0;
    while (1 << b < units) ++b;
    return b;
}

// The angles of a unit's eight pairs.
struct Angles {
    float2 cs[8];
    __device__ __forceinline__ void set(const RopeParams& r, const Unit& u, int64_t pos) {
        if (u.index >= r.R >> 4) return;
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
            const ulonglong2 f = *reinterpret_cast<const ulonglong2*>(r.table + 8 * u.index + j);
            cs[j] = turn(r, pos, f.x);
            cs[j + 1] = turn(r, pos, f.y);
        }
    }
};

// A unit of one row as loaded (several rows' loads in flight), and widened.
template <typename TA>
struct Held {
    Raw8<TA> a, b;
    __device__ __forceinline__ void load(const Unit& u, const TA* src) {
        a.load(src + u.first);
        if (u.second >= 0) b.load(src + u.second);
    }
};
struct Values {
    float x[8], y[8];
    template <typename TA>
    __device__ __forceinline__ void from(const Held<TA>& h, const Unit& u) {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = h.a.at(j), y[j] = u.second >= 0 ? h.b.at(j) : 0.0f;
    }
    __device__ __forceinline__ void turn(const RopeParams& r, const Unit& u, const Angles& t) {
        if (u.index >= r.R >> 4) return;
        if (r.half) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float c = t.cs[j].x, s = t.cs[j].y, a = x[j], b = y[j];
                x[j] = a * c - b * s;
                y[j] = a * s + b * c;
            }
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float c = t.cs[j].x, s = t.cs[j].y, a = x[2 * j], b = x[2 * j + 1];
                x[2 * j] = a * c - b * s;
                x[2 * j + 1] = a * s + b * c;
                c = t.cs[j + 4].x, s = t.cs[j + 4].y, a = y[2 * j], b = y[2 * j + 1];
                y[2 * j] = a * c - b * s;
                y[2 * j + 1] = a * s + b * c;
            }
        }
    }
    template <typename TA>
    __device__ __forceinline__ void store(const Unit& u, TA* dst) const {
        Vec8<TA>::store(dst + u.first, x);
        if (u.second >= 0) Vec8<TA>::store(dst + u.second, y);
    }
};

template <typename TA>
__device__ __forceinline__ TA* row(const Rows& r, int64_t t, int h) {
    return const_cast<TA*>(static_cast<const TA*>(r.p)) + t * r.ts + h * r.hs;
}

}  // namespace gbmoe
