// Layer norm with the residual's addition (gorila_add_layernorm, _backward).
//
// Memory bound, as the root-mean-square norm: every value is read once and written once,
// a row stays in the registers of its lanes between its sums and the output.  (Where it
// fits: widths above 16384, backward 8192, keep part of it in scratch memory.)
#include "norm_rows.h"

namespace gorila {
namespace {

// The sums of N values over the LANES lanes of a row (all of them get them); sm: LDS, N
// for each wave, used where a row has more than one.
template <int LANES, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], float (*sm)[N]) {
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = over_wave(v[k], [](float a, float b) { return a + b; });
    if (LANES == 64) return;
    __syncthreads();
    if ((threadIdx.x & 63) == 0)
#pragma unroll
        for (int k = 0; k < N; ++k) sm[threadIdx.x >> 6][k] = v[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < N; ++k) {
        v[k] = sm[0][k];
#pragma unroll
        for (int i = 1; i < LANES / 64; ++i) v[k] += sm[i][k];
    }
}

// v - mean at the row's columns, zero past them.
template <int W, int LANES, int QUADS>
__device__ __forceinline__ void center(f32x4 (&v)[QUADS], float mean, int width, int l) {
#pragma unroll
    for (int i = 0; i < QUADS; ++i) {
        const int n = width - column<W, LANES>(l, i);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[i][j] = (W == 1 ? j < n : 0 < n) ? v[i][j] - mean : 0.0f;
    }
}
__device__ __forceinline__ float sum4(f32x4 v) { return (v[0] + v[1]) + (v[2] + v[3]); }

struct LayerArgs {
    const void *x, *residual, *dy, *dtotal, *total_in;
    int64_t xs, rs, dys, dts;
    const float *weight, *bias, *mean_in, *rstd_in;
    int64_t rows;
    int width;
    float eps;
    void *y, *total, *dx;
    float *mean, *rstd, *parts;
};

// The mean is rounded, and a row's offset may be many times its deviations: the sum of
// the deviations, which comes with the sum of their squares, is what it is off by.
template <class T, int LANES, int QUADS, int W>
__global__ __launch_bounds__(LANES < 256 ? 256 : LANES) void layernorm_kernel(LayerArgs a) {
    __shared__ float sm1[LANES / 64][1], sm2[LANES / 64][2];
    constexpr int PER = LANES < 256 ? 256 / LANES : 1;  // rows a workgroup
    const int64_t row = (int64_t)blockIdx.x * PER + threadIdx.x / LANES;
    const int l = threadIdx.x % LANES;
    if (row >= a.rows) return;  // whole waves, and no barrier where a workgroup has several rows
    f32x4 v[QUADS], w[QUADS];
    load_row<W, LANES>(v, (const T*)a.x + row * a.xs, a.width, l);
    if (a.residual) {
        f32x4 r[QUADS];
        load_row<W, LANES>(r, (const T*)a.residual + row * a.rs, a.width, l);
#pragma unroll
        for (int i = 0; i < QUADS; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) v[i][j] = row_value(row_round<T>(v[i][j] + r[i][j]));
    }
    load_weight<W, LANES>(w, a.weight, a.width, l);
    float sum[1] = {0.0f};
#pragma unroll
    for (int i = 0; i < QUADS; ++i) sum[0] += sum4(v[i]);
    row_sums<LANES>(sum, sm1);
    if (a.total) store_row<W, LANES>(v, (T*)a.total + row * a.width, a.width, l);
    const float mean = sum[0] / (float)a.width;
    center<W, LANES>(v, mean, a.width, l);
    float two[2] = {0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < QUADS; ++i) two[0] += sum4(v[i]), two[1] += sum4(v[i] * v[i]);
    row_sums<LANES>(two, sm2);
    const float off = two[0] / (float)a.width;
    float var = two[1] / (float)a.width - off * off;
    if (var < 0.0f) var = 0.0f;  // (NaN stays)
    const float rho = 1.0f / sqrtf(var + a.eps);
    if (l == 0) {
        if (a.mean) a.mean[row] = mean + off;
        if (a.rstd) a.rstd[row] = rho;
    }
    f32x4 b[QUADS];
    if (a.bias) load_weight<W, LANES>(b, a.bias, a.width, l);
#pragma unroll
    for (int i = 0; i < QUADS; ++i) {
        v[i] = (v[i] - off) * rho * w[i];
        if (a.bias) v[i] += b[i];
    }
    store_row<W, LANES>(v, (T*)a.y + row * a.width, a.width, l);
}

// Backward: as the root-mean-square norm's, with both parameters' sums, and with the
// saved mean's rounding taken out again: its part comes with the row's other sums.
template <class T, int LANES, int QUADS, int W>
__global__ __launch_bounds__(LANES == 64 ? 512 : LANES) void layernorm_backward_kernel(LayerArgs a) {
    constexpr int PER = LANES == 64 ? 8 : 1, COLS = LANES * QUADS * 4;
    __shared__ __align__(16) float sums[PER > 1 ? PER / 2 * COLS : 4];
    __shared__ float sm[LANES / 64][3];
    const int l = threadIdx.x % LANES, own = threadIdx.x / LANES;
    f32x4 dw[QUADS], db[QUADS], w[QUADS];
    load_weight<W, LANES>(w, a.weight, a.width, l);
#pragma unroll
    for (int i = 0; i < QUADS; ++i) dw[i] = db[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    for (int64_t row = (int64_t)blockIdx.x * PER + own; row < a.rows; row += (int64_t)gridDim.x * PER) {
        const float rho = a.rstd_in[row], mean = a.mean_in[row];
        f32x4 g[QUADS], v[QUADS], d[QUADS];
        load_row<W, LANES>(g, (const T*)a.dy + row * a.dys, a.width, l);
        load_row<W, LANES>(v, (const T*)a.total_in + row * a.width, a.width, l);
        if (a.dtotal) load_row<W, LANES>(d, (const T*)a.dtotal + row * a.dts, a.width, l);
        center<W, LANES>(v, mean, a.width, l);
        float s[3] = {0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < QUADS; ++i) {
            const f32x4 gw = g[i] * w[i];
            s[0] += sum4(v[i]), s[1] += sum4(gw), s[2] += sum4(gw * v[i]);
        }
        row_sums<LANES>(s, sm);
        const float per = 1.0f / (float)a.width, off = s[0] * per, mg = s[1] * per;
        const float k = rho * rho * (s[2] * per - off * mg);  // mean(g xh) rho
#pragma unroll
        for (int i = 0; i < QUADS; ++i) {
            v[i] = v[i] - off;
            dw[i] += g[i] * (v[i] * rho);
            db[i] += g[i];
            g[i] = (g[i] * w[i] - mg - v[i] * k) * rho;
            if (a.dtotal) g[i] += d[i];
        }
        store_row<W, LANES>(g, (T*)a.dx + row * a.width, a.width, l);
    }
    // the workgroup's rows joined: the upper half's sums to the lower half, and again
#pragma unroll
    for (int half = PER / 2; half; half >>= 1)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            f32x4(&v)[QUADS] = k ? db : dw;
            __syncthreads();
            if (own >= half && own < 2 * half) {
#pragma unroll
                for (int i = 0; i < QUADS; ++i) *(f32x4*)(sums + (own - half) * COLS + (l + i * LANES) * 4) = v[i];
            }
            __syncthreads();
            if (own < half) {
#pragma unroll
                for (int i = 0; i < QUADS; ++i) v[i] += *(const f32x4*)(sums + own * COLS + (l + i * LANES) * 4);
            }
        }
    if (own != 0) return;
    float* part = a.parts + (int64_t)blockIdx.x * 2 * a.width;
#pragma unroll
    for (int i = 0; i < QUADS; ++i) {
        const int c = column<W, LANES>(l, i);
        if (c >= a.width) continue;
        row_store<W != 1>(part + c, dw[i], a.width - c);
        row_store<W != 1>(part + a.width + c, db[i], a.width - c);
    }
}

// Lanes and quads of the backward's rows: it holds six values a column, where the
// root-mean-square norm's holds five.
template <class F>
void by_backward_width(int width, F&& f) {
    auto k = [&](auto lanes, auto quads) { f(lanes, quads); };
    using std::integral_constant;
    if (width <= 512) k(integral_constant<int, 64>{}, integral_constant<int, 2>{});
    else if (width <= 1024) k(integral_constant<int, 64>{}, integral_constant<int, 4>{});
    else if (width <= 2048) k(integral_constant<int, 256>{}, integral_constant<int, 2>{});
    else if (width <= 4096) k(integral_constant<int, 256>{}, integral_constant<int, 4>{});
    else if (width <= 8192) k(integral_constant<int, 512>{}, integral_constant<int, 4>{});
    else if (width <= 16384) k(integral_constant<int, 1024>{}, integral_constant<int, 4>{});
    else k(integral_constant<int, 1024>{}, integral_constant<int, 16>{});
}

int check_layer(const LayerArgs& a, int dtype) {
    if (!row_dtype(dtype) || a.rows < 0 || a.width < 1 || a.width > MAX_ROW || !a.weight) return GORILA_EINVAL;
    for (const float* p : {a.weight, a.bias, a.mean_in, a.rstd_in, (const float*)a.mean, (const float*)a.rstd})
        if (!at_element(p, 4)) return GORILA_EINVAL;
    return a.rows > INT32_MAX ? GORILA_EUNSUPPORTED : GORILA_OK;
}

}  // namespace
}  // namespace gorila

using namespace gorila;

extern "C" {

int gorila_add_layernorm(const void* x, int64_t x_stride, const void* residual, int64_t residual_stride, const float* weight,
                         const float* bias, int64_t rows, int32_t width, int32_t dtype, float eps, void* y, void* total, float* mean,
                         float* rstd, gorila_ctx* ctx) {
    LayerArgs a{};
    a.x = x, a.xs = x_stride, a.residual = residual, a.rs = residual ? residual_stride : 0, a.weight = weight, a.bias = bias;
    a.rows = rows, a.width = width, a.eps = eps, a.y = y, a.total = total, a.mean = mean, a.rstd = rstd;
    CtxView c;
    int rc = ctx_view(ctx, 0, c);
    if (rc || (rc = check_layer(a, dtype))) return rc;
    if (!(eps >= 0.0f) || !(eps < INFINITY)) return GORILA_EINVAL;
    if (rows == 0) return GORILA_OK;
    if (!x || !y) return GORILA_EINVAL;
    const int e = dtype_bytes(dtype);
    for (const void* p : {x, residual, (const void*)y, (const void*)total})
        if (!at_element(p, e)) return GORILA_EINVAL;
    const int64_t strides = a.xs | a.rs | width;
    const bool vec = !(strides & 3) && at_four(x, e) && at_four(residual, e) && at_four(y, e) && at_four(total, e) && at_four(weight, 4) &&
                     at_four(bias, 4);
    const bool pairs = vec && !(strides & 7) && aligned16(x) && aligned16(residual) && aligned16(y) && aligned16(total);
    bool fits = true;
    by_width(width, [&](auto lanes, auto quads) {
        constexpr int L = decltype(lanes)::value, QD = decltype(quads)::value, PER = L < 256 ? 256 / L : 1;
        fits = launch_fits((double)((rows + PER - 1) / PER), L < 256 ? 256 : L);
        if (!fits) return;
        by_load(dtype, vec, pairs, [&](auto t, auto wide) {
            layernorm_kernel<decltype(t), L, QD, decltype(wide)::value><<<(unsigned)((rows + PER - 1) / PER), L < 256 ? 256 : L, 0, c.stream>>>(a);
        });
    });
    return fits ? launched() : GORILA_EUNSUPPORTED;
}

size_t gorila_add_layernorm_workspace_bytes(int32_t width) {
    if (width < 1 || width > MAX_ROW) return 0;
    return WS_FIXED_BYTES + (size_t)NORM_PARTS * width * 8;
}

int gorila_add_layernorm_backward(const void* dy, int64_t dy_stride, const void* dtotal, int64_t dtotal_stride, const void* total,
                                  const float* mean, const float* rstd, const float* weight, int64_t rows, int32_t width, int32_t dtype,
                                  void* dx, float* dweight, float* dbias, gorila_ctx* ctx) {
    LayerArgs a{};
    a.dy = dy, a.dys = dy_stride, a.dtotal = dtotal, a.dts = dtotal ? dtotal_stride : 0, a.total_in = total, a.mean_in = mean;
    a.rstd_in = rstd, a.weight = weight, a.rows = rows, a.width = width, a.dx = dx;
    CtxView c;
    int rc = ctx_view(ctx, 0, c);
    if (rc || (rc = check_layer(a, dtype))) return rc;
    if (!dweight || !at_element(dweight, 4) || !at_element(dbias, 4) || (rows > 0 && (!dy || !total || !mean || !rstd || !dx)))
        return GORILA_EINVAL;
    const int e = dtype_bytes(dtype);
    for (const void* p : {dy, dtotal, total, (const void*)dx})
        if (!at_element(p, e)) return GORILA_EINVAL;
    if ((rc = ctx_view(ctx, (size_t)NORM_PARTS * width * 8, c))) return rc;
    a.parts = (float*)c.ws;
    const int64_t strides = a.dys | a.dts | width;
    const bool vec = !(strides & 3) && at_four(dy, e) && at_four(dtotal, e) && at_four(total, e) && at_four(dx, e) && at_four(weight, 4);
    const bool pairs = vec && !(strides & 7) && aligned16(dy) && aligned16(dtotal) && aligned16(total) && aligned16(dx);
    int parts = 0;
    by_backward_width(width, [&](auto lanes, auto quads) {
        constexpr int L = decltype(lanes)::value, QD = decltype(quads)::value, THREADS = L == 64 ? 512 : L, PER = THREADS / L;
        const int64_t need = (rows + PER - 1) / PER;
        parts = (int)(need < NORM_PARTS ? need : NORM_PARTS);
        if (parts == 0) return;
        by_load(dtype, vec, pairs, [&](auto t, auto wide) {
            layernorm_backward_kernel<decltype(t), L, QD, decltype(wide)::value><<<parts, THREADS, 0, c.stream>>>(a);
        });
    });
    launch_sum_parts(a.parts, parts, 2 * (int64_t)width, width, 1, dweight, dbias, c.stream);
    return launched();
}

}  // extern "C"
