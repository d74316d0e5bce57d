// Norm with the residual's addition (gorila_add_rmsnorm, _codes, _backward).
//
// Memory bound: every value is read once and written once, a row stays in the
// registers of its lanes between the sum of squares and the output.  (Where it fits:
// forward up to 16384 values, backward up to 8192 but for unaligned rows of 1025 to 2048.
// Else the compiler keeps part of it in scratch memory: widths to 65536 are taken for
// completeness, and are not fast.)
//
// 16384 x 512 fp32: forward 23.8 us (5.6 TB/s), backward 22.0 us (6.1 TB/s; part of it
// from the cache) and 4 us for the sums of the workgroups' weight gradients.  40007 x
// 1000 bf16: 53 us (6.0 TB/s), 59 us (5.4 TB/s) and 4 us.  A large copy reaches 4.8
// TB/s, one that fits the cache 8.5.
#include "norm_rows.h"

namespace gorila {
namespace {

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

template <class T, int LANES, int QUADS, int W, bool CODES>
__global__ __launch_bounds__(LANES < 256 ? 256 : LANES) void norm_kernel(NormArgs a) {
    __shared__ float sm[LANES / 64];
    constexpr int PER = LANES < 256 ? 256 / LANES : 1;  // rows a workgroup
    const int64_t row = (int64_t)blockIdx.x * PER + threadIdx.x / LANES;
    const int l = threadIdx.x % LANES;
    if (row >= a.rows) return;  // whole waves, and no barrier where a workgroup has several rows
    f32x4 v[QUADS], w[QUADS];
    load_row<W, LANES>(v, (const T*)a.x + row * a.xs, a.width, l);
    load_weight<W, LANES>(w, a.weight, a.width, l);
    if (a.residual) {
        f32x4 r[QUADS];
        load_row<W, LANES>(r, (const T*)a.residual + row * a.rs, a.width, l);
#pragma unroll
        for (int i = 0; i < QUADS; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) v[i][j] = row_value(row_round<T>(v[i][j] + r[i][j]));
    }
    float sq = 0.0f;
#pragma unroll
    for (int i = 0; i < QUADS; ++i) sq += (v[i][0] * v[i][0] + v[i][1] * v[i][1]) + (v[i][2] * v[i][2] + v[i][3] * v[i][3]);
    sq = row_sum<LANES>(sq, sm);
    const float rho = 1.0f / sqrtf(sq / (float)a.width + a.eps);
    if (a.total) store_row<W, LANES>(v, (T*)a.total + row * a.width, a.width, l);
    if (!CODES) {
        if (a.rstd && l == 0) a.rstd[row] = rho;
#pragma unroll
        for (int i = 0; i < QUADS; ++i) v[i] = v[i] * rho * w[i];
        store_row<W, LANES>(v, (T*)a.y + row * a.width, a.width, l);
        return;
    }
    // codes: the norm's factor is in the scale alone, so they depend on no sum
    float most = 0.0f, bad = 0.0f;
#pragma unroll
    for (int i = 0; i < QUADS; ++i) {
        v[i] = v[i] * w[i];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            most = fmaxf(most, fabsf(v[i][j]));
            bad += v[i][j] * 0.0f;
        }
    }
    most = row_max<LANES>(bad == bad ? most : INFINITY, sm);
    const bool fine = most < INFINITY, tiny = most < TINY;
    if (tiny) {
#pragma unroll
        for (int i = 0; i < QUADS; ++i) v[i] *= TINY_UP;
        most *= TINY_UP;
    }
    const float inv = most > 0.0f && fine ? 127.0f / most : 0.0f;
    if (l == 0)  // (rho of a row of zeros is infinite where eps is 0)
        a.scale[row] = !fine ? NAN : most > 0.0f ? rho * (most / 127.0f) * (tiny ? 1.0f / TINY_UP : 1.0f) : 0.0f;
    int8_t* q = a.codes + row * a.width;
#pragma unroll
    for (int i = 0; i < QUADS; ++i) {
        const int c = column<W, LANES>(l, i);
        int k[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) k[j] = fine ? (int)rintf(v[i][j] * inv) : 0;
        if (W != 1) {
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
// their columns and write them as one part.  A row of one wave needs no barrier, so
// eight of them share a workgroup; a row of more has a workgroup of its own.
template <class T, int LANES, int QUADS, int W>
__global__ __launch_bounds__(LANES == 64 ? 512 : LANES) void norm_backward_kernel(NormArgs a) {
    constexpr int PER = LANES == 64 ? 8 : 1, COLS = LANES * QUADS * 4;
    __shared__ __align__(16) float sums[PER > 1 ? PER / 2 * COLS : 4];
    __shared__ float sm[LANES / 64];
    const int l = threadIdx.x % LANES, own = threadIdx.x / LANES;
    f32x4 dw[QUADS], w[QUADS];
    load_weight<W, LANES>(w, a.weight, a.width, l);
#pragma unroll
    for (int i = 0; i < QUADS; ++i) dw[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    for (int64_t row = (int64_t)blockIdx.x * PER + own; row < a.rows; row += (int64_t)gridDim.x * PER) {
        const float rho = a.rstd_in[row];
        f32x4 g[QUADS], v[QUADS], d[QUADS];
        load_row<W, LANES>(g, (const T*)a.dy + row * a.dys, a.width, l);
        load_row<W, LANES>(v, (const T*)a.total_in + row * a.width, a.width, l);
        if (a.dtotal) load_row<W, LANES>(d, (const T*)a.dtotal + row * a.dts, a.width, l);
        float dot = 0.0f;
#pragma unroll
        for (int i = 0; i < QUADS; ++i) {
            dw[i] += g[i] * (v[i] * rho);
            g[i] = g[i] * w[i];
            dot += (g[i][0] * v[i][0] + g[i][1] * v[i][1]) + (g[i][2] * v[i][2] + g[i][3] * v[i][3]);
        }
        dot = row_sum<LANES>(dot, sm);
        const float k = rho * rho * (dot / (float)a.width);
#pragma unroll
        for (int i = 0; i < QUADS; ++i) {
            g[i] = (g[i] - v[i] * k) * rho;
            if (a.dtotal) g[i] += d[i];
        }
        store_row<W, LANES>(g, (T*)a.dx + row * a.width, a.width, l);
    }
    // the workgroup's rows joined: the upper half's sums to the lower half, and again
#pragma unroll
    for (int half = PER / 2; half; half >>= 1) {
        __syncthreads();
        if (own >= half && own < 2 * half) {
#pragma unroll
            for (int i = 0; i < QUADS; ++i) *(f32x4*)(sums + (own - half) * COLS + (l + i * LANES) * 4) = dw[i];
        }
        __syncthreads();
        if (own < half) {
#pragma unroll
            for (int i = 0; i < QUADS; ++i) dw[i] += *(const f32x4*)(sums + own * COLS + (l + i * LANES) * 4);
        }
    }
    if (own != 0) return;
    float* part = a.parts + (int64_t)blockIdx.x * a.width;
#pragma unroll
    for (int i = 0; i < QUADS; ++i) {
        const int c = column<W, LANES>(l, i);
        if (c < a.width) row_store<W != 1>(part + c, dw[i], a.width - c);
    }
}

// 16 columns a workgroup; its 64 teams of 16 lanes take the parts in turn, so that a
// lane has few loads to wait for, and their sums are added in LDS.  2048 parts of 512
// columns, four waves of 64 columns each: 95 us; 512 parts, this way: 3 us.
constexpr int SUM_COLS = 16, SUM_TEAMS = 64;
__global__ __launch_bounds__(SUM_COLS * SUM_TEAMS) void sum_parts_kernel(const float* __restrict__ parts, int n_parts, int64_t n, int64_t first, int taps,
                                                                        float* __restrict__ out, float* __restrict__ out2) {
    __shared__ float sm[SUM_TEAMS][SUM_COLS + 1];
    const int c = threadIdx.x % SUM_COLS, team = threadIdx.x / SUM_COLS;
    const int64_t i = (int64_t)blockIdx.x * SUM_COLS + c;
    float v = 0.0f;
    if (i < n) {
#pragma unroll 8
        for (int p = team; p < n_parts; p += SUM_TEAMS) v += parts[p * n + i];
    }
    sm[team][c] = v;
    __syncthreads();
    if (threadIdx.x >= 64) return;  // one wave: four lanes a column, 16 sums each
    v = 0.0f;
#pragma unroll
    for (int t = 0; t < SUM_TEAMS / 4; ++t) v += sm[4 * t + team][c];
    v += __shfl_xor(v, 16, 64);
    v += __shfl_xor(v, 32, 64);
    if (team != 0 || i >= n) return;
    if (i < first) out[i % (first / taps) * taps + i / (first / taps)] = v;
    else if (out2) out2[i - first] = v;
}

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
    const int64_t strides = a.xs | a.rs | a.width;
    const bool vec = !(strides & 3) && at_four(a.x, e) && at_four(a.residual, e) && at_four(a.y, e) && at_four(a.total, e) &&
                     at_four(a.weight, 4) && at_four(a.codes, 1);
    const bool pairs = vec && !(strides & 7) && aligned16(a.x) && aligned16(a.residual) && aligned16(a.y) && aligned16(a.total);
    bool fits = true;
    by_width(a.width, [&](auto lanes, auto quads) {
        constexpr int L = decltype(lanes)::value, QD = decltype(quads)::value, PER = L < 256 ? 256 / L : 1;
        fits = launch_fits((double)((a.rows + PER - 1) / PER), L < 256 ? 256 : L);
        if (!fits) return;
        by_load(dtype, vec, pairs, [&](auto t, auto wide) {
            auto go = [&](auto co) {
                norm_kernel<decltype(t), L, QD, decltype(wide)::value, decltype(co)::value>
                    <<<(unsigned)((a.rows + PER - 1) / PER), L < 256 ? 256 : L, 0, c.stream>>>(a);
            };
            codes ? go(std::true_type{}) : go(std::false_type{});
        });
    });
    return fits ? launched() : GORILA_EUNSUPPORTED;
}

}  // namespace

void launch_sum_parts(const float* parts, int n_parts, int64_t n, int64_t first, int taps, float* out, float* out2, hipStream_t st) {
    sum_parts_kernel<<<(unsigned)((n + SUM_COLS - 1) / SUM_COLS), SUM_COLS * SUM_TEAMS, 0, st>>>(parts, n_parts, n, first, taps, out, out2);
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
    return WS_FIXED_BYTES + (size_t)NORM_PARTS * width * 4;
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
    if ((rc = ctx_view(ctx, (size_t)NORM_PARTS * width * 4, c))) return rc;
    a.parts = (float*)c.ws;
    const int64_t strides = a.dys | a.dts | width;
    const bool vec = !(strides & 3) && at_four(dy, e) && at_four(dtotal, e) && at_four(total, e) && at_four(dx, e) && at_four(weight, 4);
    const bool pairs = vec && !(strides & 7) && aligned16(dy) && aligned16(dtotal) && aligned16(total) && aligned16(dx);
    int parts = 0;
    by_width(width, [&](auto lanes, auto quads) {
        constexpr int L = decltype(lanes)::value, QD = decltype(quads)::value, THREADS = L == 64 ? 512 : L, PER = THREADS / L;
        const int64_t need = (rows + PER - 1) / PER;
        parts = (int)(need < NORM_PARTS ? need : NORM_PARTS);
        if (parts == 0) return;
        by_load(dtype, vec, pairs, [&](auto t, auto wide) {
            norm_backward_kernel<decltype(t), L, QD, decltype(wide)::value><<<parts, THREADS, 0, c.stream>>>(a);
        });
    });
    launch_sum_parts(a.parts, parts, width, width, 1, dweight, nullptr, c.stream);
    return launched();
}

}  // extern "C"
