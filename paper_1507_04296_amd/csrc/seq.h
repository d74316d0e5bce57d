// What the sequence operators (norm.hip, layernorm.hip, shortconv.hip, scan.hip, gated.hip,
// qmatvec.hip), adamw.hip and sample.hip share: the context as they see it, rows of fp32
// or bf16 values, and sums over a wave.
#pragma once
#include "common.h"
#include "kernels.h"

namespace gorila {

// The context's stream and device, the workspace behind its fixed head (null
// without one) and its sticky error word (null without one).
struct CtxView {
    hipStream_t stream;
    int cus;
    char* ws;
    unsigned* err;
};
// Checks the context and that `need` workspace bytes are there; a call that
// needs any overwrites what a learner call left.
int ctx_view(gorila_ctx* ctx, size_t need, CtxView& out);
// Bytes in front of the part that CtxView::ws names.
extern const size_t WS_FIXED_BYTES;

__device__ __forceinline__ float row_value(float v) { return v; }
__device__ __forceinline__ float row_value(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }
template <class T> __device__ __forceinline__ T row_round(float v);
template <> __device__ __forceinline__ float row_round<float>(float v) { return v; }
template <> __device__ __forceinline__ uint16_t row_round<uint16_t>(float v) {
    return __builtin_bit_cast(uint16_t, (__bf16)v);  // nearest even
}

// Four consecutive values, aligned to four elements.
__device__ __forceinline__ f32x4 row_load4(const float* p) { return *(const f32x4*)p; }
__device__ __forceinline__ f32x4 row_load4(const uint16_t* p) {
    const uint2 v = *(const uint2*)p;
    return f32x4{__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xffff0000u),
                 __uint_as_float(v.y << 16), __uint_as_float(v.y & 0xffff0000u)};
}
__device__ __forceinline__ void row_store4(float* p, f32x4 v) { *(f32x4*)p = v; }
__device__ __forceinline__ void row_store4(uint16_t* p, f32x4 v) {
    const uint32_t a = row_round<uint16_t>(v[0]), b = row_round<uint16_t>(v[1]);
    const uint32_t c = row_round<uint16_t>(v[2]), d = row_round<uint16_t>(v[3]);
    *(uint2*)p = uint2{a | b << 16, c | d << 16};
}
// The first n (at most 4) of four consecutive values; the others are zeros.
template <bool VEC, class T>
__device__ __forceinline__ f32x4 row_load(const T* p, int n) {
    f32x4 v{0.0f, 0.0f, 0.0f, 0.0f};
    if (VEC) {
        if (n > 0) v = row_load4(p);  // n is a multiple of four
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j < n) v[j] = row_value(p[j]);
    }
    return v;
}
template <bool VEC, class T>
__device__ __forceinline__ void row_store(T* p, f32x4 v, int n) {
    if (VEC) {
        if (n > 0) row_store4(p, v);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j < n) p[j] = row_round<T>(v[j]);
    }
}

// A value at any address of its elements.  Global memory takes wide loads and stores there; those
// that cross a line of the cache are two.
template <class V>
__device__ __forceinline__ V load_any(const void* p) {
    V v;
    __builtin_memcpy(&v, p, sizeof(V));
    return v;
}
template <class V>
__device__ __forceinline__ void store_any(void* p, V v) { __builtin_memcpy(p, &v, sizeof(V)); }
// As row_load() and row_store() of quads, n of which exist: in one piece where all four do.
__device__ __forceinline__ f32x4 quad_load(const float* p, int n) { return n >= 4 ? load_any<f32x4>(p) : row_load<false>(p, n); }
__device__ __forceinline__ f32x4 quad_load(const uint16_t* p, int n) {
    if (n < 4) return row_load<false>(p, n);
    const uint2 v = load_any<uint2>(p);
    return f32x4{__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xffff0000u), __uint_as_float(v.y << 16), __uint_as_float(v.y & 0xffff0000u)};
}
__device__ __forceinline__ void quad_store(float* p, f32x4 v, int n) {
    if (n >= 4) store_any(p, v);
    else row_store<false>(p, v, n);
}
__device__ __forceinline__ void quad_store(uint16_t* p, f32x4 v, int n) {
    if (n >= 4) {
        const uint32_t a = row_round<uint16_t>(v[0]), b = row_round<uint16_t>(v[1]);
        const uint32_t c = row_round<uint16_t>(v[2]), d = row_round<uint16_t>(v[3]);
        store_any(p, uint2{a | b << 16, c | d << 16});
    } else {
        row_store<false>(p, v, n);
    }
}

// v of the lane that DPP's control names, 0 where there is none (or where the row of 16 lanes is
// not in ROWS).
template <int CONTROL, int ROWS>
__device__ __forceinline__ float lane_of(float v) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CONTROL, ROWS, 0xf, false));
}
// f(v, ..) over a wave's lanes, in a scalar register, for an f with the neutral element 0: inside
// rows of 16 lanes (one lane down, two, four, eight), then from row to row.  Shuffles through
// LDS wait 0.3 us for the same six steps.
template <class F>
__device__ __forceinline__ float over_wave(float v, F&& f) {
    v = f(v, lane_of<0x111, 0xf>(v));
    v = f(v, lane_of<0x112, 0xf>(v));
    v = f(v, lane_of<0x114, 0xf>(v));
    v = f(v, lane_of<0x118, 0xf>(v));
    v = f(v, lane_of<0x142, 0xa>(v));  // lane 15 of a row to the next row
    v = f(v, lane_of<0x143, 0xc>(v));  // lane 31 to the upper half
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
}

// A quotient of 127 or 7 by a value below TINY may be past the range of fp32: such values
// are taken TINY_UP times as large before (a power of two, so no bit changes).
constexpr float TINY = 0x1p-100f, TINY_UP = 0x1p64f;

inline int dtype_bytes(int dtype) { return dtype == GORILA_BF16 ? 2 : 4; }
inline bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }
inline bool row_dtype(int dtype) { return dtype == GORILA_F32 || dtype == GORILA_BF16; }
// Whether an address is one of an element of `bytes`, or of four of them.
inline bool at_element(const void* p, int bytes) { return ((uintptr_t)p & (uintptr_t)(bytes - 1)) == 0; }
inline bool at_four(const void* p, int bytes) { return at_element(p, 4 * bytes); }
// Sums of parts[0 .. n_parts-1][i] in a fixed order (norm.hip): column i < first, read
// as [taps][first / taps], to out as [first / taps][taps]; the others to out2 (which may
// be null).
void launch_sum_parts(const float* parts, int n_parts, int64_t n, int64_t first, int taps, float* out, float* out2, hipStream_t st);
// HIP refuses a launch of 2^32 lanes or more in one dimension: such calls are unsupported.
// (In floating point: products of sizes may be past 64 bits.)
inline bool launch_fits(double blocks, int threads) { return blocks * threads < 4294967296.0; }
inline int launched() { return hipGetLastError() == hipSuccess ? GORILA_OK : GORILA_EHIP; }

}  // namespace gorila
