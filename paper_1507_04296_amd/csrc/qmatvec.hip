// Products with 4-bit weights and group scales (gorila_quantize_weights,
// gorila_qmatvec).
//
// With few rows the codes are what has to be read: 16 bytes a lane are 32 codes of
// one output and one group.  Codes are multiplied as 0 .. 15, and the group's
// offset of 8 comes off through the sum of its inputs, so a code costs one
// conversion and one multiply-add a row (8-bit rows: a quarter of an integer dot
// product, exact).
#include "seq.h"

namespace gorila {
namespace {

struct MatvecView {
    const void* x;
    int64_t xs, rows;
    const float* x_scale;
    const uint8_t* codes;
    const float* scales;
    int outputs, inputs, group, chunks, groups;  // chunks of 32 codes a row
    void* y;
};

// A wave's lanes form 64 / lk teams of lk lanes; a team takes OUT outputs, its lanes
// the chunks of the row in turn.
template <class T, int R, int OUT, bool VEC>
__global__ __launch_bounds__(256) void matvec_kernel(MatvecView s, int lk) {
    const int l = threadIdx.x & 63, k = l % lk;
    const int team = ((int)blockIdx.x * 4 + (threadIdx.x >> 6)) * (64 / lk) + l / lk;
    const int o0 = team * OUT;
    const int64_t r0 = (int64_t)blockIdx.y * R;
    float acc[R][OUT];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int o = 0; o < OUT; ++o) acc[r][o] = 0.0f;
    for (int c = k; c < s.chunks; c += lk) {
        uint4 q[OUT];
        float sc[OUT];
#pragma unroll
        for (int o = 0; o < OUT; ++o) {
            const int64_t at = o0 + o < s.outputs ? o0 + o : 0;
            q[o] = *(const uint4*)(s.codes + (at * s.chunks + c) * 16);
            sc[o] = s.scales[at * s.groups + c * 32 / s.group];
        }
        const int n = s.inputs - c * 32;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const bool in = r0 + r < s.rows;
            if constexpr (std::is_same<T, int8_t>::value) {
                const int8_t* x = (const int8_t*)s.x + (in ? (r0 + r) * s.xs : 0) + c * 32;
                int xe[4], xo[4], sum = 0;  // even and odd inputs of eight, as the codes' halves lie
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    uint32_t a, b;
                    if (VEC && n >= 32) {
                        const uint2 v = ((const uint2*)x)[j];
                        a = v.x, b = v.y;
                    } else {
                        a = b = 0;
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            if (8 * j + i < n) a |= (uint32_t)(uint8_t)x[8 * j + i] << (8 * i);
                            if (8 * j + 4 + i < n) b |= (uint32_t)(uint8_t)x[8 * j + 4 + i] << (8 * i);
                        }
                    }
                    xe[j] = (int)__builtin_amdgcn_perm(b, a, 0x06040200u);
                    xo[j] = (int)__builtin_amdgcn_perm(b, a, 0x07050301u);
                    sum = __builtin_amdgcn_sdot4(xe[j], 0x01010101, sum, false);
                    sum = __builtin_amdgcn_sdot4(xo[j], 0x01010101, sum, false);
                }
#pragma unroll
                for (int o = 0; o < OUT; ++o) {
                    const uint32_t qs[4] = {q[o].x, q[o].y, q[o].z, q[o].w};
                    int d = -8 * sum;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        d = __builtin_amdgcn_sdot4(xe[j], (int)(qs[j] & 0x0f0f0f0fu), d, false);
                        d = __builtin_amdgcn_sdot4(xo[j], (int)(qs[j] >> 4 & 0x0f0f0f0fu), d, false);
                    }
                    acc[r][o] = fmaf((float)d, sc[o], acc[r][o]);
                }
            } else {
                const T* x = (const T*)s.x + (in ? (r0 + r) * s.xs : 0) + c * 32;
                float v[32], sum = 0.0f;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const f32x4 a = row_load<VEC>(x + (n > 4 * j ? 4 * j : 0), n - 4 * j);
#pragma unroll
                    for (int i = 0; i < 4; ++i) v[4 * j + i] = a[i];
                    sum += (a[0] + a[1]) + (a[2] + a[3]);
                }
#pragma unroll
                for (int o = 0; o < OUT; ++o) {
                    const uint32_t qs[4] = {q[o].x, q[o].y, q[o].z, q[o].w};
                    float d = -8.0f * sum;
#pragma unroll
                    for (int j = 0; j < 4; ++j)
#pragma unroll
                        for (int i = 0; i < 8; ++i) d = fmaf((float)(qs[j] >> (4 * i) & 15u), v[8 * j + i], d);
                    acc[r][o] = fmaf(d, sc[o], acc[r][o]);
                }
            }
        }
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int o = 0; o < OUT; ++o) {
            float v = acc[r][o];
            for (int m = lk >> 1; m; m >>= 1) v += __shfl_xor(v, m, 64);
            if (k == 0 && o0 + o < s.outputs && r0 + r < s.rows) {
                const int64_t at = (r0 + r) * s.outputs + o0 + o;
                if constexpr (std::is_same<T, int8_t>::value) ((float*)s.y)[at] = v * s.x_scale[r0 + r];
                else ((T*)s.y)[at] = row_round<T>(v);
            }
        }
}

// A lane takes four weights; the lanes of a group find its largest together.
template <class T, bool VEC>
__global__ __launch_bounds__(256) void quantize_kernel(const T* w, int64_t ws, int outputs, int inputs, int group, int chunks,
                                                       int groups, uint8_t* codes, float* scales) {
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int per = groups * (group / 4);  // lanes a row, whole groups
    const int64_t row = id / per;
    const int k = (int)(id % per) * 4, lanes = group / 4;
    const bool on = row < outputs;
    const f32x4 v = row_load<VEC>(w + (on && k < inputs ? row * ws + k : 0), on ? inputs - k : 0);
    float most = 0.0f, bad = 0.0f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        most = fmaxf(most, fabsf(v[j]));
        bad += v[j] * 0.0f;
    }
    if (bad != bad) most = INFINITY;
    for (int m = lanes >> 1; m; m >>= 1) most = fmaxf(most, __shfl_xor(most, m, 64));
    if (!on) return;
    const bool fine = most < INFINITY;
    const float inv = most > 0.0f && fine ? 7.0f / most : 0.0f;
    if (k % group == 0) scales[row * groups + k / group] = fine ? most / 7.0f : NAN;
    if (k >= chunks * 32) return;  // past the row's codes
    uint32_t q = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) q |= (uint32_t)(8 + (fine ? (int)rintf(v[j] * inv) : 0)) << (4 * j);
    *(uint16_t*)(codes + row * chunks * 16 + k / 2) = (uint16_t)q;
}

bool group_size(int g) { return g == 32 || g == 64 || g == 128; }

}  // namespace
}  // namespace gorila

using namespace gorila;

extern "C" {

int gorila_quantize_weights(const void* weights, int64_t weights_stride, int32_t outputs, int32_t inputs, int32_t dtype,
                            int32_t group, uint8_t* codes, float* scales, gorila_ctx* ctx) {
    CtxView c;
    const int rc = ctx_view(ctx, 0, c);
    if (rc) return rc;
    if (!row_dtype(dtype) || outputs < 0 || inputs < 1 || !group_size(group)) return GORILA_EINVAL;
    if (inputs > INT32_MAX - 128) return GORILA_EUNSUPPORTED;
    if (outputs == 0) return GORILA_OK;
    const int e = dtype_bytes(dtype);
    if (!weights || !codes || !scales || !at_element(weights, e) || !aligned16(codes) || !at_element(scales, 4)) return GORILA_EINVAL;
    const int chunks = (inputs + 31) / 32, groups = (inputs + group - 1) / group;
    const int64_t lanes = (int64_t)outputs * groups * (group / 4);
    if ((lanes + 255) / 256 > INT32_MAX) return GORILA_EUNSUPPORTED;
    const bool vec = !((weights_stride | inputs) & 3) && at_four(weights, e);
    const unsigned grid = (unsigned)((lanes + 255) / 256);
    auto go = [&](auto t, auto al) {
        using T = decltype(t);
        quantize_kernel<T, decltype(al)::value><<<grid, 256, 0, c.stream>>>((const T*)weights, weights_stride, outputs, inputs, group,
                                                                          chunks, groups, codes, scales);
    };
    if (dtype == GORILA_F32) vec ? go(float{}, std::true_type{}) : go(float{}, std::false_type{});
    else vec ? go(uint16_t{}, std::true_type{}) : go(uint16_t{}, std::false_type{});
    return launched();
}

int gorila_qmatvec(const void* x, int64_t x_stride, const float* x_scale, int32_t x_dtype, int64_t rows, const uint8_t* codes,
                   const float* scales, int32_t outputs, int32_t inputs, int32_t group, void* y, gorila_ctx* ctx) {
    CtxView c;
    const int rc = ctx_view(ctx, 0, c);
    if (rc) return rc;
    if (!row_dtype(x_dtype) && x_dtype != GORILA_CODES) return GORILA_EINVAL;
    if (rows < 0 || outputs < 0 || inputs < 1 || !group_size(group)) return GORILA_EINVAL;
    if (rows == 0 || outputs == 0) return GORILA_OK;
    const int e = x_dtype == GORILA_CODES ? 1 : dtype_bytes(x_dtype);
    if (!x || !codes || !scales || !y || (x_dtype == GORILA_CODES && !x_scale)) return GORILA_EINVAL;
    if (!at_element(x, e) || !aligned16(codes) || !at_element(scales, 4) || !at_element(x_scale, 4) ||
        !at_element(y, x_dtype == GORILA_BF16 ? 2 : 4))
        return GORILA_EINVAL;
    if (inputs > INT32_MAX - 128 || rows > 65535) return GORILA_EUNSUPPORTED;
    MatvecView v{x, x_stride, rows, x_scale, codes, scales, outputs, inputs, group, (inputs + 31) / 32, (inputs + group - 1) / group, y};
    int lk = 64;
    while (lk > 1 && lk / 2 >= v.chunks) lk >>= 1;
    auto go = [&](auto t, auto r, auto al) {
        constexpr int R = decltype(r)::value, OUT = 4;
        const int64_t teams = (outputs + OUT - 1) / OUT, per = 4 * (64 / lk);
        matvec_kernel<decltype(t), R, OUT, decltype(al)::value>
            <<<dim3((unsigned)((teams + per - 1) / per), (unsigned)((rows + R - 1) / R)), 256, 0, c.stream>>>(v, lk);
    };
    auto al = [&](auto t, auto r, bool vec) { vec ? go(t, r, std::true_type{}) : go(t, r, std::false_type{}); };
    auto by = [&](auto t, bool vec) {
        if (rows == 1) al(t, std::integral_constant<int, 1>{}, vec);
        else al(t, std::integral_constant<int, 4>{}, vec);
    };
    const bool four = !((x_stride | inputs) & 3) && at_four(x, e);
    if (x_dtype == GORILA_F32) by(float{}, four);
    else if (x_dtype == GORILA_BF16) by(uint16_t{}, four);
    else by(int8_t{}, !(x_stride & 7) && ((uintptr_t)x & 7) == 0);
    return launched();
}

}  // extern "C"
