// What the norms (norm.hip, layernorm.hip) share: a row held in the registers of its lanes.
#pragma once
#include "seq.h"

namespace gorila {

constexpr int MAX_ROW = 65536;

// A row in the registers of its LANES lanes, QUADS runs of four values each.  W: values
// a load (8: two quads of bf16 side by side; 4; 1: no alignment).
template <int W, int LANES>
__device__ __forceinline__ int column(int l, int i) {
    return W == 8 ? (l + (i >> 1) * LANES) * 8 + (i & 1) * 4 : (l + i * LANES) * 4;
}
template <int W, int LANES, int QUADS, class T>
__device__ __forceinline__ void load_row(f32x4 (&v)[QUADS], const T* p, int width, int l) {
    if constexpr (W == 8) {
#pragma unroll
        for (int i = 0; i < QUADS; i += 2) {
            const int c = column<W, LANES>(l, i);
            uint4 u{0, 0, 0, 0};
            if (c < width) u = *(const uint4*)(p + c);
            v[i] = f32x4{__uint_as_float(u.x << 16), __uint_as_float(u.x & 0xffff0000u), __uint_as_float(u.y << 16), __uint_as_float(u.y & 0xffff0000u)};
            v[i + 1] = f32x4{__uint_as_float(u.z << 16), __uint_as_float(u.z & 0xffff0000u), __uint_as_float(u.w << 16), __uint_as_float(u.w & 0xffff0000u)};
        }
    } else {
#pragma unroll
        for (int i = 0; i < QUADS; ++i) {
            const int c = column<W, LANES>(l, i), n = width - c;
            v[i] = row_load<W == 4>(p + (n > 0 ? c : 0), n);
        }
    }
}
template <int W, int LANES, int QUADS>
__device__ __forceinline__ void load_weight(f32x4 (&v)[QUADS], const float* p, int width, int l) {
#pragma unroll
    for (int i = 0; i < QUADS; ++i) {
        const int c = column<W, LANES>(l, i), n = width - c;
        v[i] = row_load<W != 1>(p + (n > 0 ? c : 0), n);
    }
}
template <int W, int LANES, int QUADS, class T>
__device__ __forceinline__ void store_row(const f32x4 (&v)[QUADS], T* p, int width, int l) {
    if constexpr (W == 8) {
#pragma unroll
        for (int i = 0; i < QUADS; i += 2) {
            const int c = column<W, LANES>(l, i);
            uint32_t u[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const f32x4& q = v[i + (j >> 1)];
                u[j] = row_round<T>(q[2 * (j & 1)]) | (uint32_t)row_round<T>(q[2 * (j & 1) + 1]) << 16;
            }
            if (c < width) *(uint4*)(p + c) = uint4{u[0], u[1], u[2], u[3]};
        }
    } else {
#pragma unroll
        for (int i = 0; i < QUADS; ++i) {
            const int c = column<W, LANES>(l, i);
            if (c < width) row_store<W == 4>(p + c, v[i], width - c);
        }
    }
}

// Workgroups of a backward, a part each: two of eight waves a compute unit.
constexpr int NORM_PARTS = 512;

template <class F>
void by_width(int width, F&& f) {
    auto k = [&](auto lanes, auto quads) { f(lanes, quads); };
    using std::integral_constant;
    if (width <= 512) k(integral_constant<int, 64>{}, integral_constant<int, 2>{});
    else if (width <= 1024) k(integral_constant<int, 64>{}, integral_constant<int, 4>{});
    else if (width <= 2048) k(integral_constant<int, 64>{}, integral_constant<int, 8>{});
    else if (width <= 4096) k(integral_constant<int, 256>{}, integral_constant<int, 4>{});
    else if (width <= 8192) k(integral_constant<int, 256>{}, integral_constant<int, 8>{});
    else if (width <= 16384) k(integral_constant<int, 1024>{}, integral_constant<int, 4>{});
    else k(integral_constant<int, 1024>{}, integral_constant<int, 16>{});
}

// Calls f(row type, values a load) as constants.
template <class F>
void by_load(int dtype, bool vec, bool pairs, F&& f) {
    using std::integral_constant;
    if (dtype == GORILA_F32) vec ? f(float{}, integral_constant<int, 4>{}) : f(float{}, integral_constant<int, 1>{});
    else if (pairs) f(uint16_t{}, integral_constant<int, 8>{});
    else vec ? f(uint16_t{}, integral_constant<int, 4>{}) : f(uint16_t{}, integral_constant<int, 1>{});
}

}  // namespace gorila
