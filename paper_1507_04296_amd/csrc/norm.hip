// Norm with the residual's addition (gorila_add_rmsnorm, _codes, _backward).
//
// Memory bound: every value is read once and written once, a row stays in the
// registers of its lanes between the sum of squares and the output.
#include "seq.h"

namespace gorila {
namespace {

constexpr int MAX_ROW = 65536;

// Sum of v over the LANES lanes of a row (all of them get it); sm: LDS of the
// workgroup, used where a row has more than one wave.
template <int LANES>
__device__ __forceinline__ float row_sum(float v, float* sm) {
#pragma unroll
    for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o, 64);
    if (LANES == 64) return v;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) sm[threadIdx.x >> 6] = v;
    __syncthreads();
    v = sm[0];
#pragma unroll
    for (int i = 1; i < LANES / 64; ++i) v += sm[i];
    return v;
}
template <int LANES>
__device__ __forceinline__ float row_max(float v, float* sm) {
#pragma unroll
    for (int o = 32; o; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
    if (LANES == 64) return v;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) sm[threadIdx.x >> 6] = v;
    __syncthreads();
    v = sm[0];
#pragma unroll
    for (int i = 1; i < LANES / 64; ++i) v = fmaxf(v, sm[i]);
    return v;
}

struct NormArgs {
    const void *x, *residual, *dy, *dtotal, *total_in;
    int64_t xs, rs, dys, dts;
    const float *weight, *rstd_in;
    int64_t rows;
    int width;
    float eps;
    void *y, *total, *dx;
    float *rstd, *scale, *parts;
    int8_t* codes;
};

// A row is taken by LANES lanes, QUADS runs of four values each.
template <class T, int LANES, int QUADS, bool VEC, bool CODES>
__global__ __launch_bounds__(LANES < 256 ? 256 : LANES) void norm_kernel(NormArgs a) {
    __shared__ float sm[LANES / 64];
    constexpr int PER = LANES < 256 ? 256 / LANES : 1;  // rows a workgroup
    const int64_t row = (int64_t)blockIdx.x * PER + threadIdx.x / LANES;
    const int l = threadIdx.x % LANES;
    if (row >= a.rows) return;  // whole waves, and no barrier where a workgroup has several rows
    const T* x = (const T*)a.x + row * a.xs;
    const T* r = (const T*)a.residual + row * a.rs;
    f32x4 v[QUADS];
    float sq = 0.0f;
#pragma unroll
    for (int i = 0; i < QUADS; ++i) {
        const int c = (l + i * LANES) * 4, n = a.width - c;
        v[i] = row_load<VEC>(x + (n > 0 ? c : 0), n);
        if (a.residual) {
            v[i] += row_load<VEC>(r + (n > 0 ? c : 0), n);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[i][j] = row_value(row_round<T>(v[i][j]));
        }
        sq += (v[i][0] * v[i][0] + v[i][1] * v[i][1]) + (v[i][2] * v[i][2] + v[i][3] * v[i][3]);
    }
    sq = row_sum<LANES>(sq, sm);
    const float rho = 1.0f / sqrtf(sq / (float)a.width + a.eps);
    if (a.total) {
        T* t = (T*)a.total + row * a.width;
#pragma unroll
        for (int i = 0; i < QUADS; ++i) {
            const int c = (l + i * LANES) * 4;
            if (c < a.width) row_store<VEC>(t + c, v[i], a.width - c);
        }
    }
    if (!CODES) {
        if (a.rstd && l == 0) a.rstd[row] = rho;
        T* y = (T*)a.y + row * a.width;
#pragma unroll
        for (int i = 0; i < QUADS; ++i) {
            const int c = (l + i * LANES) * 4;
            if (c < a.width) row_store<VEC>(y + c, v[i] * rho * row_load<VEC>(a.weight + c, a.width - c), a.width - c);
        }
        return;
    }
    // codes: the norm's factor is in the scale alone, so they depend on no sum
    float most = 0.0f, bad = 0.0f;
#pragma unroll
    for (int i = 0; i < QUADS; ++i) {
        const int c = (l + i * LANES) * 4;
        v[i] = v[i] * row_load<VEC>(a.weight + (c < a.width ? c : 0), a.width - c);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            most = fmaxf(most, fabsf(v[i][j]));
            bad += v[i][j] * 0.0f;
        }
    }
    most = row_max<LANES>(bad == bad ? most : INFINITY, sm);
    const bool fine = most < INFINITY;
    const float inv = most > 0.0f && fine ? 127.0f / most : 0.0f;
    if (l == 0) a.scale[row] = fine ? rho * (most / 127.0f) : NAN;
    int8_t* q = a.codes + row * a.width;
#pragma unroll
    for (int i = 0; i < QUADS; ++i) {
        const int c = (l + i * LANES) * 4;
        int k[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) k[j] = fine ? (int)rintf(v[i][j] * inv) : 0;
        if (VEC) {
            if (c < a.width)
                *(uint32_t*)(q + c) = (uint32_t)(k[0] & 255) | (uint32_t)(k[1] & 255) << 8 | (uint32_t)(k[2] & 255) << 16 | (uint32_t)k[3] << 24;
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (c + j < a.width) q[c + j] = (int8_t)k[j];
        }
    }
}

// Backward: a workgroup walks rows, its lanes keep the weight gradient's sums of
// their columns and write them as one part.
template <class T, int LANES, int QUADS, bool VEC>
__global__ __launch_bounds__(LANES < 256 ? 256 : LANES) void norm_backward_kernel(NormArgs a) {
    __shared__ float sm[LANES / 64];
    constexpr int PER = LANES < 256 ? 256 / LANES : 1;
    const int l = threadIdx.x % LANES, own = threadIdx.x / LANES;
    f32x4 dw[QUADS], w[QUADS];
#pragma unroll
    for (int i = 0; i < QUADS; ++i) {
        const int c = (l + i * LANES) * 4, n = a.width - c;
        dw[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        w[i] = row_load<VEC>(a.weight + (n > 0 ? c : 0), n);
    }
    for (int64_t row = (int64_t)blockIdx.x * PER + own; row < a.rows; row += (int64_t)gridDim.x * PER) {
        const T* dy = (const T*)a.dy + row * a.dys;
        const T* dt = (const T*)a.dtotal + row * a.dts;
        const T* t = (const T*)a.total_in + row * a.width;
        T* dx = (T*)a.dx + row * a.width;
        const float rho = a.rstd_in[row];
        f32x4 g[QUADS], v[QUADS];
        float dot = 0.0f;
#pragma unroll
        for (int i = 0; i < QUADS; ++i) {
            const int c = (l + i * LANES) * 4, n = a.width - c, at = n > 0 ? c : 0;
            g[i] = row_load<VEC>(dy + at, n);
            v[i] = row_load<VEC>(t + at, n);
            dw[i] += g[i] * (v[i] * rho);
            g[i] = g[i] * w[i];
            dot += (g[i][0] * v[i][0] + g[i][1] * v[i][1]) + (g[i][2] * v[i][2] + g[i][3] * v[i][3]);
        }
        dot = row_sum<LANES>(dot, sm);
        const float k = rho * rho * (dot / (float)a.width);
#pragma unroll
        for (int i = 0; i < QUADS; ++i) {
            const int c = (l + i * LANES) * 4, n = a.width - c;
            if (n <= 0) continue;
            f32x4 d = (g[i] - v[i] * k) * rho;
            if (a.dtotal) d += row_load<VEC>(dt + c, n);
            row_store<VEC>(dx + c, d, n);
        }
    }
    float* part = a.parts + ((int64_t)blockIdx.x * PER + own) * a.width;
#pragma unroll
    for (int i = 0; i < QUADS; ++i) {
        const int c = (l + i * LANES) * 4;
        if (c < a.width) row_store<VEC>(part + c, dw[i], a.width - c);
    }
}

// 64 columns a workgroup, its four waves a quarter of the parts each.
__global__ __launch_bounds__(256) void sum_parts_kernel(const float* __restrict__ parts, int n_parts, int64_t n, int64_t first,
                                                        float* __restrict__ out, float* __restrict__ out2) {
    __shared__ float sm[4][64];
    const int l = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int64_t i = (int64_t)blockIdx.x * 64 + l;
    float v = 0.0f;
    if (i < n)
        for (int p = w; p < n_parts; p += 4) v += parts[p * n + i];
    sm[w][l] = v;
    __syncthreads();
    if (w != 0 || i >= n) return;
    v = (sm[0][l] + sm[1][l]) + (sm[2][l] + sm[3][l]);
    if (i < first) out[i] = v;
    else if (out2) out2[i - first] = v;
}

// Rows of the backward's parts: as many as rows are walked side by side.
int norm_parts(int width) { return width <= 2048 ? 2048 : width <= 8192 ? 512 : 256; }

template <class F>
void by_width(int width, F&& f) {
    auto k = [&](auto lanes, auto quads) { f(lanes, quads); };
    using std::integral_constant;
    if (width <= 256) k(integral_constant<int, 64>{}, integral_constant<int, 1>{});
    else if (width <= 512) k(integral_constant<int, 64>{}, integral_constant<int, 2>{});
    else if (width <= 1024) k(integral_constant<int, 64>{}, integral_constant<int, 4>{});
    else if (width <= 2048) k(integral_constant<int, 64>{}, integral_constant<int, 8>{});
    else if (width <= 4096) k(integral_constant<int, 256>{}, integral_constant<int, 4>{});
    else if (width <= 8192) k(integral_constant<int, 256>{}, integral_constant<int, 8>{});
    else if (width <= 16384) k(integral_constant<int, 1024>{}, integral_constant<int, 4>{});
    else k(integral_constant<int, 1024>{}, integral_constant<int, 16>{});
}

int check_norm(const NormArgs& a, int dtype) {
    if (!row_dtype(dtype) || a.rows < 0 || a.width < 1 || a.width > MAX_ROW || !a.weight || !at_element(a.weight, 4)) return GORILA_EINVAL;
    return a.rows > INT32_MAX ? GORILA_EUNSUPPORTED : GORILA_OK;
}

int norm_forward(NormArgs a, int dtype, gorila_ctx* ctx, bool codes) {
    CtxView c;
    int rc = ctx_view(ctx, 0, c);
    if (rc || (rc = check_norm(a, dtype))) return rc;
    if (!(a.eps >= 0.0f) || !(a.eps < INFINITY)) return GORILA_EINVAL;
    if (a.rows == 0) return GORILA_OK;
    if (!a.x || (codes ? !a.codes || !a.scale : !a.y)) return GORILA_EINVAL;
    const int e = dtype_bytes(dtype);
    for (const void* p : {a.x, a.residual, (const void*)a.y, (const void*)a.total})
        if (!at_element(p, e)) return GORILA_EINVAL;
    if (!at_element(a.rstd, 4) || !at_element(a.scale, 4)) return GORILA_EINVAL;
    const bool vec = !((a.xs | a.rs | a.width) & 3) && at_four(a.x, e) && at_four(a.residual, e) && at_four(a.y, e) &&
                     at_four(a.total, e) && at_four(a.weight, 4) && at_four(a.codes, 1);
    by_width(a.width, [&](auto lanes, auto quads) {
        constexpr int L = decltype(lanes)::value, QD = decltype(quads)::value, PER = L < 256 ? 256 / L : 1;
        auto go = [&](auto t, auto al, auto co) {
            norm_kernel<decltype(t), L, QD, decltype(al)::value, decltype(co)::value>
                <<<(unsigned)((a.rows + PER - 1) / PER), L < 256 ? 256 : L, 0, c.stream>>>(a);
        };
        auto al = [&](auto t, auto co) { vec ? go(t, std::true_type{}, co) : go(t, std::false_type{}, co); };
        auto ty = [&](auto co) { dtype == GORILA_F32 ? al(float{}, co) : al(uint16_t{}, co); };
        codes ? ty(std::true_type{}) : ty(std::false_type{});
    });
    return launched();
}

}  // namespace

void launch_sum_parts(const float* parts, int n_parts, int64_t n, int64_t first, float* out, float* out2, hipStream_t st) {
    sum_parts_kernel<<<(unsigned)((n + 63) / 64), 256, 0, st>>>(parts, n_parts, n, first, out, out2);
}

}  // namespace gorila

using namespace gorila;

extern "C" {

int gorila_add_rmsnorm(const void* x, int64_t x_stride, const void* residual, int64_t residual_stride, const float* weight,
                       int64_t rows, int32_t width, int32_t dtype, float eps, void* y, void* total, float* rstd, gorila_ctx* ctx) {
    NormArgs a{};
    a.x = x, a.xs = x_stride, a.residual = residual, a.rs = residual ? residual_stride : 0, a.weight = weight;
    a.rows = rows, a.width = width, a.eps = eps, a.y = y, a.total = total, a.rstd = rstd;
    return norm_forward(a, dtype, ctx, false);
}

int gorila_add_rmsnorm_codes(const void* x, int64_t x_stride, const void* residual, int64_t residual_stride, const float* weight,
                             int64_t rows, int32_t width, int32_t dtype, float eps, int8_t* codes, float* scale, void* total,
                             gorila_ctx* ctx) {
    NormArgs a{};
    a.x = x, a.xs = x_stride, a.residual = residual, a.rs = residual ? residual_stride : 0, a.weight = weight;
    a.rows = rows, a.width = width, a.eps = eps, a.codes = codes, a.scale = scale, a.total = total;
    return norm_forward(a, dtype, ctx, true);
}

size_t gorila_add_rmsnorm_workspace_bytes(int32_t width) {
    if (width < 1 || width > MAX_ROW) return 0;
    return WS_FIXED_BYTES + (size_t)norm_parts(width) * width * 4;
}

int gorila_add_rmsnorm_backward(const void* dy, int64_t dy_stride, const void* dtotal, int64_t dtotal_stride, const void* total,
                                const float* rstd, const float* weight, int64_t rows, int32_t width, int32_t dtype, void* dx,
                                float* dweight, gorila_ctx* ctx) {
    NormArgs a{};
    a.dy = dy, a.dys = dy_stride, a.dtotal = dtotal, a.dts = dtotal ? dtotal_stride : 0, a.total_in = total, a.rstd_in = rstd;
    a.weight = weight, a.rows = rows, a.width = width, a.dx = dx;
    CtxView c;
    int rc = ctx_view(ctx, 0, c);
    if (rc || (rc = check_norm(a, dtype))) return rc;
    if (!dweight || !at_element(dweight, 4) || (rows > 0 && (!dy || !total || !rstd || !dx))) return GORILA_EINVAL;
    const int e = dtype_bytes(dtype);
    for (const void* p : {dy, dtotal, total, (const void*)dx})
        if (!at_element(p, e)) return GORILA_EINVAL;
    if (!at_element(rstd, 4)) return GORILA_EINVAL;
    const int most = norm_parts(width);
    if ((rc = ctx_view(ctx, (size_t)most * width * 4, c))) return rc;
    a.parts = (float*)c.ws;
    const bool vec = !((a.dys | a.dts | width) & 3) && at_four(dy, e) && at_four(dtotal, e) && at_four(total, e) && at_four(dx, e) &&
                     at_four(weight, 4);
    int parts = 0;
    by_width(width, [&](auto lanes, auto quads) {
        constexpr int L = decltype(lanes)::value, QD = decltype(quads)::value, PER = L < 256 ? 256 / L : 1;
        const int64_t need = (rows + PER - 1) / PER;
        const int blocks = (int)(need < most / PER ? need : most / PER);
        parts = blocks * PER;
        if (blocks == 0) return;
        auto go = [&](auto t, auto al) {
            norm_backward_kernel<decltype(t), L, QD, decltype(al)::value><<<blocks, L < 256 ? 256 : L, 0, c.stream>>>(a);
        };
        auto al = [&](auto t) { vec ? go(t, std::true_type{}) : go(t, std::false_type{}); };
        dtype == GORILA_F32 ? al(float{}) : al(uint16_t{});
    });
    launch_sum_parts(a.parts, parts, width, width, dweight, nullptr, c.stream);
    return launched();
}

}  // extern "C"
