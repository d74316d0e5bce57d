// Layer norm with the residual's addition (gorila_add_layernorm, _backward).
//
// Memory bound, as the root-mean-square norm: every value is read once and written once,
// a row stays in the registers of its lanes between its sums and the output.  (Where it
// fits: widths above 16384, backward 8192, keep part of it in scratch memory, up to 680 and
// 2400 bytes a lane, and uneven fp32 rows of 6145 to 8192 keep 12 bytes of it backward.  Such
// widths are taken for completeness: 1281 x 16384 bf16 39 us forward (4.3 TB/s) and 92
// backward (1.8), 320 x 65536 bf16 112 (1.5) and 495 (0.3).)
// 40007 x 1000 bf16: forward 60 us, backward 61 (5.4 and 5.2 TB/s) and 5 for its parts'
// sums; 4096 x 512 fp32: 8.6 and 8.7, all rows in flight at once.
#include "norm_rows.h"

namespace gorila {
namespace {

// The sum over a row's 4, 8, 16 or 32 lanes, inside a wave: lanes beside one another, pairs, then
// from half a row of DPP's 16 lanes to the other, and from row to row.
template <int LANES>
__device__ __forceinline__ float over_lanes(float v) {
    v += lane_of<0xb1, 0xf>(v);
    v += lane_of<0x4e, 0xf>(v);
    if (LANES > 4) v += lane_of<0x141, 0xf>(v);
    if (LANES > 8) v += lane_of<0x140, 0xf>(v);
    if (LANES > 16) v += __shfl_xor(v, 16, 64);
    return v;
}
// The sums of N values over the LANES lanes of a row (all of them get them); sm: LDS, N
// for each wave, used where a row has more than one.
template <int LANES, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], float (*sm)[N]) {
#pragma unroll
    for (int k = 0; k < N; ++k)
        if constexpr (LANES < 64) v[k] = over_lanes<LANES>(v[k]);
        else v[k] = over_wave(v[k], [](float a, float b) { return a + b; });
    if (LANES <= 64) return;
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

// 16 bytes of a row from column c on, zeros past its end.  EVEN: rows are whole loads at
// multiples of 16 bytes.  Others are read where they are, and their end as the last 16 bytes
// of the row, moved: no branch, so that all loads of a row are under way at once
// (34571 x 781 bf16: 51 us forward, 54 backward; with a branch for the end 63 and 153, in
// single values 132 and 225).
template <class T> constexpr int PER = 16 / sizeof(T);  // values
template <bool EVEN, bool PAST, class T>
__device__ __forceinline__ uint4 load_piece(const T* p, int c, int width) {
    constexpr int W = PER<T>;
    uint4 u{0, 0, 0, 0};
    if constexpr (EVEN) {
        if (c < width) u = *(const uint4*)(p + c);
    } else if (width >= W) {
        if (PAST || c < width) u = load_any<uint4>(p + (c < width - W ? c : width - W));
    } else if (c == 0) {
        T t[W] = {};
#pragma unroll
        for (int j = 0; j < W - 1; ++j)
            if (j < width) t[j] = p[j];
        __builtin_memcpy(&u, t, 16);
    }
    return u;
}
template <bool EVEN, bool PAST, class T>
__device__ __forceinline__ uint4 move_piece(uint4 u, int c, int width) {
    constexpr int W = PER<T>;
    if (EVEN || width < W) return u;
    const int by = c - (width - W);  // 1 to W - 1 at the row's end, more past it
    if (W == 8 && __ballot(by > 0) == 0) return u;
    if (by > 0 && (by & (W / 2))) u = uint4{u.z, u.w, 0, 0};
    if (by > 0 && (by & (W / 4))) u = uint4{u.y, u.z, u.w, 0};
    if (W == 8 && by > 0 && (by & 1)) u = uint4{u.x >> 16 | u.y << 16, u.y >> 16 | u.z << 16, u.z >> 16 | u.w << 16, u.w >> 16};
    return PAST && by >= W ? uint4{0, 0, 0, 0} : u;
}
template <bool EVEN, class T>
__device__ __forceinline__ void store_piece(T* p, uint4 u, int c, int width) {
    constexpr int W = PER<T>;
    const int n = width - c;
    p += c;
    if constexpr (EVEN) {
        if (n > 0) *(uint4*)p = u;
    } else if (n >= W) {
        store_any(p, u);
    } else if (n > 0) {
        if (n & (W / 2)) store_any(p, uint2{u.x, u.y}), u.x = u.z, u.y = u.w, p += W / 2;
        if (n & (W / 4)) store_any(p, u.x), u.x = u.y, p += W / 4;
        if (W == 8 && (n & 1)) *p = (T)u.x;
    }
}
__device__ __forceinline__ f32x4 floats(uint4 u) { return f32x4{__uint_as_float(u.x), __uint_as_float(u.y), __uint_as_float(u.z), __uint_as_float(u.w)}; }
__device__ __forceinline__ uint4 bits(f32x4 v) { return uint4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])}; }

// A row as it is read; its values as norm_rows.h holds them.
template <class T, int LANES, int QUADS, bool EVEN, bool PAST = false>
struct Row {
    static constexpr int W = PER<T>, PIECES = QUADS * 4 / W;
    uint4 u[PIECES];
    __device__ __forceinline__ static int column_of(int l, int i) { return (l + i * LANES) * W; }
    __device__ __forceinline__ Row(const T* p, int width, int l) {
#pragma unroll
        for (int i = 0; i < PIECES; ++i) u[i] = load_piece<EVEN, PAST>(p, column_of(l, i), width);
    }
    __device__ __forceinline__ void values(f32x4 (&v)[QUADS], int width, int l) const {
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const uint4 m = move_piece<EVEN, PAST, T>(u[i], column_of(l, i), width);
            if constexpr (W == 8) {
                v[2 * i] = floats(uint4{m.x << 16, m.x & 0xffff0000u, m.y << 16, m.y & 0xffff0000u});
                v[2 * i + 1] = floats(uint4{m.z << 16, m.z & 0xffff0000u, m.w << 16, m.w & 0xffff0000u});
            } else {
                v[i] = floats(m);
            }
        }
    }
    __device__ __forceinline__ static void store(const f32x4 (&v)[QUADS], T* p, int width, int l) {
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            uint4 m;
            if constexpr (W == 8) {
                const f32x4 &a = v[2 * i], &b = v[2 * i + 1];
                m.x = row_round<T>(a[0]) | (uint32_t)row_round<T>(a[1]) << 16, m.y = row_round<T>(a[2]) | (uint32_t)row_round<T>(a[3]) << 16;
                m.z = row_round<T>(b[0]) | (uint32_t)row_round<T>(b[1]) << 16, m.w = row_round<T>(b[2]) | (uint32_t)row_round<T>(b[3]) << 16;
            } else {
                m = bits(v[i]);
            }
            store_piece<EVEN>(p, m, column_of(l, i), width);
        }
    }
    // the same columns of an fp32 vector
    __device__ __forceinline__ static void columns(f32x4 (&v)[QUADS], const float* p, int width, int l) {
        uint4 m[QUADS];
#pragma unroll
        for (int i = 0; i < QUADS; ++i) m[i] = load_piece<EVEN, PAST>(p, column<W, LANES>(l, i), width);
#pragma unroll
        for (int i = 0; i < QUADS; ++i) v[i] = floats(move_piece<EVEN, PAST, float>(m[i], column<W, LANES>(l, i), width));
    }
    __device__ __forceinline__ static void store_columns(const f32x4 (&v)[QUADS], float* p, int width, int l) {
#pragma unroll
        for (int i = 0; i < QUADS; ++i) store_piece<EVEN>(p, bits(v[i]), column<W, LANES>(l, i), width);
    }
    // v - mean at the row's columns, zero past them
    __device__ __forceinline__ static void center(f32x4 (&v)[QUADS], float mean, int width, int l) {
#pragma unroll
        for (int i = 0; i < QUADS; ++i) {
            const int n = width - column<W, LANES>(l, i);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[i][j] = (EVEN ? 0 < n : j < n) ? v[i][j] - mean : 0.0f;
        }
    }
};

__device__ __forceinline__ float sum4(f32x4 v) { return (v[0] + v[1]) + (v[2] + v[3]); }

struct LayerArgs {
    const void *x, *residual, *dy, *dtotal, *total_in;
    int64_t xs, rs, dys, dts;
    const float *weight, *bias, *mean_in, *rstd_in;
    int64_t rows;
    int width;
    float eps;
    void *y, *total, *dx;
    float *mean, *rstd, *parts, *dweight, *dbias;
};

// The mean is rounded, and a row's offset may be many times its deviations: the sum of
// the deviations, which comes with the sum of their squares, is what it is off by.
template <class T, int LANES, int QUADS, bool EVEN>
__global__ __launch_bounds__(LANES < 256 ? 256 : LANES) void layernorm_kernel(LayerArgs a) {
    __shared__ float sm1[(LANES + 63) / 64][1], sm2[(LANES + 63) / 64][2];
    constexpr int ROWS = LANES < 256 ? 256 / LANES : 1;  // of a workgroup
    const int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / LANES;
    const int l = threadIdx.x % LANES;
    if (row >= a.rows) return;  // all lanes of a row, and no barrier where a workgroup has several
    using Row = Row<T, LANES, QUADS, EVEN>;
    f32x4 v[QUADS], w[QUADS];
    const Row x((const T*)a.x + row * a.xs, a.width, l);
    if (a.residual) {
        f32x4 r[QUADS];
        const Row second((const T*)a.residual + row * a.rs, a.width, l);
        x.values(v, a.width, l);
        second.values(r, a.width, l);
#pragma unroll
        for (int i = 0; i < QUADS; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) v[i][j] = row_value(row_round<T>(v[i][j] + r[i][j]));
    } else {
        x.values(v, a.width, l);
    }
    Row::columns(w, a.weight, a.width, l);
    float sum[1] = {0.0f};
#pragma unroll
    for (int i = 0; i < QUADS; ++i) sum[0] += sum4(v[i]);
    row_sums<LANES>(sum, sm1);
    if (a.total) Row::store(v, (T*)a.total + row * a.width, a.width, l);
    const float mean = sum[0] / (float)a.width;
    Row::center(v, mean, a.width, l);
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
    if (a.bias) Row::columns(b, a.bias, a.width, l);
#pragma unroll
    for (int i = 0; i < QUADS; ++i) {
        v[i] = (v[i] - off) * rho * w[i];
        if (a.bias) v[i] += b[i];
    }
    Row::store(v, (T*)a.y + row * a.width, a.width, l);
}

// Backward: as the root-mean-square norm's, with both parameters' sums, and with the
// saved mean's rounding taken out again: its part comes with the row's other sums.
template <class T, int LANES, int QUADS, bool EVEN>
__global__ __launch_bounds__(LANES <= 64 ? 512 : LANES) void layernorm_backward_kernel(LayerArgs a) {
    constexpr int ROWS = LANES <= 64 ? 512 / LANES : 1, COLS = LANES * QUADS * 4;
    __shared__ __align__(16) float sums[ROWS > 1 ? ROWS / 2 * COLS : 4];
    __shared__ float sm[(LANES + 63) / 64][3];
    const int l = threadIdx.x % LANES, own = threadIdx.x / LANES;
    using Row = Row<T, LANES, QUADS, EVEN, sizeof(T) == 4>;
    f32x4 dw[QUADS], db[QUADS], w[QUADS];
    Row::columns(w, a.weight, a.width, l);
#pragma unroll
    for (int i = 0; i < QUADS; ++i) dw[i] = db[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    for (int64_t row = (int64_t)blockIdx.x * ROWS + own; row < a.rows; row += (int64_t)gridDim.x * ROWS) {
        const float rho = a.rstd_in[row], mean = a.mean_in[row];
        f32x4 g[QUADS], v[QUADS], d[QUADS];
        const Row dy((const T*)a.dy + row * a.dys, a.width, l), total((const T*)a.total_in + row * a.width, a.width, l);
        const Row dt((const T*)a.dtotal + row * a.dts, a.dtotal ? a.width : 0, l);
        dy.values(g, a.width, l), total.values(v, a.width, l);
        Row::center(v, mean, a.width, l);
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
        }
        if (a.dtotal) {
            dt.values(d, a.width, l);
#pragma unroll
            for (int i = 0; i < QUADS; ++i) g[i] += d[i];
        }
        Row::store(g, (T*)a.dx + row * a.width, a.width, l);
    }
    // the workgroup's rows joined: the upper half's sums to the lower half, and again
#pragma unroll
    for (int half = ROWS / 2; half; half >>= 1)
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
    if (gridDim.x == 1) {  // no other workgroup's to add
        using Any = gorila::Row<T, LANES, QUADS, false>;
        Any::store_columns(dw, a.dweight, a.width, l);
        if (a.dbias) Any::store_columns(db, a.dbias, a.width, l);
        return;
    }
    float* part = a.parts + (int64_t)blockIdx.x * 2 * a.width;
    Row::store_columns(dw, part, a.width, l);
    Row::store_columns(db, part + a.width, a.width, l);
}

// Turns over the rows up to which one workgroup takes all of them, so that no launch adds sums: a
// turn is 0.7 us (1.4 where rows are wide), the launch 2.2 us in a graph and 3 outside.
constexpr int ALONE = 4, ALONE_WIDE = 3;

// Lanes and quads of a row: narrow rows share a wave, 8 values a lane (421875 x 64 bf16: 37 us
// forward, 43 backward, with 16 lanes a row 51 and 50; a wave each takes three times as
// long), wide ones have 8 or 16 values a lane: with 32, as the root-mean-square norm's
// forward, uneven rows have few waves a unit (10494 x 2001 fp32 72 us, so 64; even ones of
// 1200 bf16 34 and 37).  Backward of 4797 x 4377: 65 us bf16 and 78 fp32, with 16 values 70 and 87.
template <class F>
void by_layer_width(int width, F&& f) {
    auto k = [&](auto lanes, auto quads) { f(lanes, quads); };
    using std::integral_constant;
    if (width <= 32) k(integral_constant<int, 4>{}, integral_constant<int, 2>{});
    else if (width <= 64) k(integral_constant<int, 8>{}, integral_constant<int, 2>{});
    else if (width <= 128) k(integral_constant<int, 16>{}, integral_constant<int, 2>{});
    else if (width <= 256) k(integral_constant<int, 32>{}, integral_constant<int, 2>{});
    else if (width <= 512) k(integral_constant<int, 64>{}, integral_constant<int, 2>{});
    else if (width <= 1024) k(integral_constant<int, 64>{}, integral_constant<int, 4>{});
    else if (width <= 2048) k(integral_constant<int, 256>{}, integral_constant<int, 2>{});
    else if (width <= 4096) k(integral_constant<int, 256>{}, integral_constant<int, 4>{});
    else if (width <= 6144) k(integral_constant<int, 768>{}, integral_constant<int, 2>{});
    else if (width <= 8192) k(integral_constant<int, 1024>{}, integral_constant<int, 2>{});
    else if (width <= 16384) k(integral_constant<int, 1024>{}, integral_constant<int, 4>{});
    else k(integral_constant<int, 1024>{}, integral_constant<int, 16>{});
}

template <class F>
void by_rows(int dtype, bool even, F&& f) {
    if (dtype == GORILA_F32) even ? f(float{}, std::true_type{}) : f(float{}, std::false_type{});
    else even ? f(uint16_t{}, std::true_type{}) : f(uint16_t{}, std::false_type{});
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
    bool even = !(strides & (16 / e - 1)) && aligned16(weight) && aligned16(bias);
    for (const void* p : {x, residual, (const void*)y, (const void*)total}) even = even && aligned16(p);
    bool fits = true;
    by_layer_width(width, [&](auto lanes, auto quads) {
        constexpr int L = decltype(lanes)::value, QD = decltype(quads)::value, ROWS = L < 256 ? 256 / L : 1;
        fits = launch_fits((double)((rows + ROWS - 1) / ROWS), L < 256 ? 256 : L);
        if (!fits) return;
        by_rows(dtype, even, [&](auto t, auto ev) {
            layernorm_kernel<decltype(t), L, QD, decltype(ev)::value><<<(unsigned)((rows + ROWS - 1) / ROWS), L < 256 ? 256 : L, 0, c.stream>>>(a);
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
    a.rstd_in = rstd, a.weight = weight, a.rows = rows, a.width = width, a.dx = dx, a.dweight = dweight, a.dbias = dbias;
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
    bool even = !(strides & (16 / e - 1)) && aligned16(weight);
    for (const void* p : {dy, dtotal, total, (const void*)dx}) even = even && aligned16(p);
    int parts = 0;
    by_layer_width(width, [&](auto lanes, auto quads) {
        constexpr int L = decltype(lanes)::value, QD = decltype(quads)::value, THREADS = L <= 64 ? 512 : L, ROWS = THREADS / L;
        const int64_t need = (rows + ROWS - 1) / ROWS;
        constexpr int MOST = L < 512 ? NORM_PARTS : NORM_PARTS / 2;  // one a compute unit; a part's sums are 8 bytes a column
        parts = need <= (L <= 256 ? ALONE : ALONE_WIDE) ? rows > 0 : (int)(need < MOST ? need : MOST);
        if (parts == 0) return;
        by_rows(dtype, even, [&](auto t, auto ev) {
            layernorm_backward_kernel<decltype(t), L, QD, decltype(ev)::value><<<parts, THREADS, 0, c.stream>>>(a);
        });
    });
    if (parts != 1) launch_sum_parts(a.parts, parts, 2 * (int64_t)width, width, 1, dweight, dbias, c.stream);
    return launched();
}

}  // extern "C"
