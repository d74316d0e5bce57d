// The short causal convolution (gorila_causal_conv, _backward, _step).
//
// Memory bound.  A lane takes four channels (one, where quads are not aligned) of a
// run of steps and keeps the last taps in registers, so a value is read once (and
// once more by the next run's lane, from the cache).  An episode start empties the
// registers: nothing before it is multiplied, whatever it holds.
#include "seq.h"

namespace gorila {
namespace {

constexpr int RUN = 16;         // steps a lane
constexpr int MAX_TAPS = 4;
constexpr int MAX_PARTS = 512;  // of the weight gradient's sums

struct ConvView {
    const void *x, *window, *dy, *dwindow_out;
    int64_t xb, xt, dyb, dyt;
    const float *weight, *bias;
    const uint8_t* reset;
    int B, T, C, silu, runs, quads, parts;
    void *y, *window_out, *dx, *dwindow;
    float* sums;
};

// W channels from p (a quad, or one value in element 0).
template <bool VEC, class T>
__device__ __forceinline__ f32x4 get(const T* p) {
    return VEC ? row_load4(p) : f32x4{row_value(p[0]), 0.0f, 0.0f, 0.0f};
}
template <bool VEC, class T>
__device__ __forceinline__ void put(T* p, f32x4 v) {
    if (VEC) row_store4(p, v);
    else p[0] = row_round<T>(v[0]);
}
constexpr f32x4 ZERO4{0.0f, 0.0f, 0.0f, 0.0f};

template <int K, bool VEC>
__device__ __forceinline__ void load_taps(const ConvView& s, int c, f32x4 (&w)[K], f32x4& bias) {
    constexpr int W = VEC ? 4 : 1;
#pragma unroll
    for (int j = 0; j < K; ++j) {
        w[j] = ZERO4;
#pragma unroll
        for (int i = 0; i < W; ++i) w[j][i] = s.weight[(int64_t)(c + i) * K + j];
    }
    bias = s.bias ? get<VEC>(s.bias + c) : ZERO4;
}

// The K - 1 steps before t0, oldest first; a start at a step empties those before it.
template <class T, int K, bool VEC>
__device__ __forceinline__ void load_past(const ConvView& s, int b, int c, int t0, const T* x, const uint8_t* rs, f32x4 (&e)[K]) {
    bool live = true;
#pragma unroll
    for (int j = 1; j < K; ++j) {  // step t0 - j
        const int t = t0 - j;
        e[K - 1 - j] = ZERO4;
        if (live) {
            if (t >= 0) e[K - 1 - j] = get<VEC>(x + (int64_t)t * s.xt);
            else if (s.window) e[K - 1 - j] = get<VEC>((const T*)s.window + ((int64_t)b * (K - 1) + K - 1 + t) * s.C + c);
        }
        if (t >= 0 && rs && rs[t]) live = false;
    }
}

__device__ __forceinline__ float sigmoid(float v) { return 1.0f / (1.0f + expf(-v)); }

template <class T, int K, bool VEC>
__global__ __launch_bounds__(256) void conv_kernel(ConvView s) {
    constexpr int W = VEC ? 4 : 1;
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int c = (int)(id % s.quads) * W;
    const int64_t unit = id / s.quads;
    const int run = (int)(unit % s.runs);
    const int64_t bl = unit / s.runs;
    if (bl >= s.B) return;
    const int b = (int)bl, t0 = run * RUN, t1 = t0 + RUN < s.T ? t0 + RUN : s.T;
    const T* x = (const T*)s.x + b * s.xb + c;
    const uint8_t* rs = s.reset ? s.reset + (int64_t)b * s.T : nullptr;
    T* y = (T*)s.y + (int64_t)b * s.T * s.C + c;
    f32x4 w[K], bias, e[K];
    load_taps<K, VEC>(s, c, w, bias);
    load_past<T, K, VEC>(s, b, c, t0, x, rs, e);
    for (int t = t0; t < t1; ++t) {
        if (rs && rs[t]) {
#pragma unroll
            for (int j = 0; j < K - 1; ++j) e[j] = ZERO4;
        }
        e[K - 1] = get<VEC>(x + (int64_t)t * s.xt);
        f32x4 v = bias;
#pragma unroll
        for (int j = 0; j < K; ++j) v += w[j] * e[j];
        if (s.silu) {
#pragma unroll
            for (int i = 0; i < W; ++i) v[i] *= sigmoid(v[i]);
        }
        put<VEC>(y + (int64_t)t * s.C, v);
#pragma unroll
        for (int j = 0; j < K - 1; ++j) e[j] = e[j + 1];
    }
    if (s.window_out && run == s.runs - 1) {
#pragma unroll
        for (int j = 0; j < K - 1; ++j) put<VEC>((T*)s.window_out + ((int64_t)b * (K - 1) + j) * s.C + c, e[j]);
    }
}

// A lane walks units (runs of sequences) part, part + parts, ...  In a run it forms
// the gradient of v for its steps and the K - 1 after them, and keeps the sums of
// dx of the last K steps (own, of a step: written when its last tap has passed).
template <class T, int K, bool VEC>
__global__ __launch_bounds__(256) void conv_backward_kernel(ConvView s) {
    constexpr int W = VEC ? 4 : 1;
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int c = (int)(id % s.quads) * W;
    const int64_t part = id / s.quads;
    if (part >= s.parts) return;
    f32x4 w[K], bias, dw[K], db = ZERO4;
    load_taps<K, VEC>(s, c, w, bias);
#pragma unroll
    for (int j = 0; j < K; ++j) dw[j] = ZERO4;
    for (int64_t unit = part; unit < (int64_t)s.B * s.runs; unit += s.parts) {
        const int run = (int)(unit % s.runs), b = (int)(unit / s.runs);
        const int t0 = run * RUN, t1 = t0 + RUN < s.T ? t0 + RUN : s.T;
        const T* x = (const T*)s.x + b * s.xb + c;
        const T* dy = (const T*)s.dy + b * s.dyb + c;
        const uint8_t* rs = s.reset ? s.reset + (int64_t)b * s.T : nullptr;
        T* dx = (T*)s.dx + (int64_t)b * s.T * s.C + c;
        const T* dwo = s.dwindow_out ? (const T*)s.dwindow_out + (int64_t)b * (K - 1) * s.C + c : nullptr;
        T* dwi = s.dwindow ? (T*)s.dwindow + (int64_t)b * (K - 1) * s.C + c : nullptr;
        f32x4 e[K], d[K];  // d[j]: of step t - (K - 1) + j
        load_past<T, K, VEC>(s, b, c, t0, x, rs, e);
#pragma unroll
        for (int j = 0; j < K; ++j) d[j] = ZERO4;
        // steps of the episode before t that a tap at t reaches
        int reach = K - 1;
        if (rs) {
#pragma unroll
            for (int j = K - 1; j >= 1; --j)
                if (t0 - j >= 0 && rs[t0 - j]) reach = j;
        }
        const int last = t1 + K - 1;
        for (int t = t0; t < last; ++t) {
            // past the end nothing is added, but the window behind it has gradients
            const bool in = t < s.T;
            f32x4 dv = ZERO4;
            if (in) {
                if (rs && rs[t]) {
                    reach = 0;
#pragma unroll
                    for (int j = 0; j < K - 1; ++j) e[j] = ZERO4;
                }
                e[K - 1] = get<VEC>(x + (int64_t)t * s.xt);
                dv = get<VEC>(dy + (int64_t)t * s.dyt);
                if (s.silu) {
                    f32x4 v = bias;
#pragma unroll
                    for (int j = 0; j < K; ++j) v += w[j] * e[j];
#pragma unroll
                    for (int i = 0; i < W; ++i) {
                        const float g = sigmoid(v[i]);
                        dv[i] *= g * (1.0f + v[i] * (1.0f - g));
                    }
                }
                if (t < t1) {
                    db += dv;
#pragma unroll
                    for (int j = 0; j < K; ++j) dw[j] += dv * e[j];
                }
#pragma unroll
                for (int j = 0; j < K; ++j)
                    if (K - 1 - j <= reach) d[j] += w[j] * dv;
                if (reach < K - 1) ++reach;
            }
            // step t - (K - 1) is complete
            const int at = t - (K - 1);
            if (at < t0 && at >= 0) {
                // another run's
            } else if (at >= t0 || run == 0) {
                f32x4 v = d[0];
                const int k = at - (s.T - (K - 1));  // its place in the window behind
                if (dwo && k >= 0) {
                    bool live = true;
                    for (int u = at + 1 > 0 ? at + 1 : 0; u < s.T; ++u)
                        if (rs && rs[u]) live = false;
                    if (live) v += get<VEC>(dwo + (int64_t)k * s.C);
                }
                if (at >= 0) put<VEC>(dx + (int64_t)at * s.C, v);
                else if (dwi) put<VEC>(dwi + (int64_t)(at + K - 1) * s.C, v);
            }
#pragma unroll
            for (int j = 0; j < K - 1; ++j) {
                d[j] = d[j + 1];
                e[j] = e[j + 1];
            }
            d[K - 1] = ZERO4;
        }
    }
    float* o = s.sums + part * (int64_t)s.C * (K + 1);
#pragma unroll
    for (int i = 0; i < W; ++i) {
#pragma unroll
        for (int j = 0; j < K; ++j) o[(int64_t)(c + i) * K + j] = dw[j][i];
        o[(int64_t)s.C * K + c + i] = db[i];
    }
}

template <class T, int K, bool VEC>
__global__ __launch_bounds__(256) void conv_step_kernel(ConvView s, T* pool, int64_t slots, const int32_t* slot, unsigned* err) {
    constexpr int W = VEC ? 4 : 1;
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int c = (int)(id % s.quads) * W;
    const int64_t row = id / s.quads;
    if (row >= s.B) return;
    int64_t at = slot ? slot[row] : row;
    const bool out = at < 0 || at >= slots;
    if (out) {
        if (c == 0 && err) atomicOr(err, ERR_IDX_RANGE);
        at = 0;
    }
    const bool empty = out || (s.reset && s.reset[row]);
    T* p = pool + at * (K - 1) * s.C + c;
    f32x4 w[K], bias, e[K];
    load_taps<K, VEC>(s, c, w, bias);
#pragma unroll
    for (int j = 0; j < K - 1; ++j) e[j] = empty ? ZERO4 : get<VEC>(p + (int64_t)j * s.C);
    e[K - 1] = get<VEC>((const T*)s.x + row * s.xb + c);
    f32x4 v = bias;
#pragma unroll
    for (int j = 0; j < K; ++j) v += w[j] * e[j];
    if (s.silu) {
#pragma unroll
        for (int i = 0; i < W; ++i) v[i] *= sigmoid(v[i]);
    }
    put<VEC>((T*)s.y + row * s.C + c, v);
    if (!out) {
#pragma unroll
        for (int j = 0; j < K - 1; ++j) put<VEC>(p + (int64_t)j * s.C, e[j + 1]);
    }
}

int conv_view(const gorila_causal_conv_args* a, bool step, ConvView& v, bool& vec) {
    if (!a || !row_dtype(a->dtype) || a->batch < 0 || a->length < 0 || a->channels < 1) return GORILA_EINVAL;
    if (a->taps < 2 || a->taps > MAX_TAPS || (a->silu != 0 && a->silu != 1) || !a->weight) return GORILA_EINVAL;
    if (a->batch > 0 && a->length > 0 && !a->x) return GORILA_EINVAL;
    const int e = dtype_bytes(a->dtype);
    if (!at_element(a->x, e) || !at_element(a->window, e) || !at_element(a->weight, 4) || !at_element(a->bias, 4)) return GORILA_EINVAL;
    v = ConvView{};
    v.x = a->x, v.xb = a->x_batch_stride, v.xt = a->x_step_stride, v.weight = a->weight, v.bias = a->bias;
    v.reset = a->reset, v.window = step ? nullptr : a->window;
    v.B = a->batch, v.T = a->length, v.C = a->channels, v.silu = a->silu;
    v.runs = v.T > 0 ? (v.T + RUN - 1) / RUN : 1;
    vec = !((v.C | v.xb | (step ? 0 : v.xt)) & 3) && at_four(a->x, e) && at_four(v.window, e) && at_four(a->bias, 4);
    // a lane a quad and run, in workgroups of 256, in a 32-bit grid
    if ((int64_t)v.B * v.runs > INT32_MAX || (int64_t)v.B * v.runs * v.C / 256 > INT32_MAX / 2) return GORILA_EUNSUPPORTED;
    return GORILA_OK;
}

template <class F>
void by_taps(int taps, int dtype, bool vec, F&& f) {
    auto al = [&](auto t, auto k) { vec ? f(t, k, std::true_type{}) : f(t, k, std::false_type{}); };
    auto ty = [&](auto k) { dtype == GORILA_F32 ? al(float{}, k) : al(uint16_t{}, k); };
    if (taps == 2) ty(std::integral_constant<int, 2>{});
    else if (taps == 3) ty(std::integral_constant<int, 3>{});
    else ty(std::integral_constant<int, 4>{});
}

unsigned lanes_grid(int64_t lanes) { return (unsigned)((lanes + 255) / 256); }

}  // namespace
}  // namespace gorila

using namespace gorila;

extern "C" {

int gorila_causal_conv(const gorila_causal_conv_args* args, void* y, void* window_out, gorila_ctx* ctx) {
    ConvView v;
    CtxView c;
    bool vec;
    int rc = ctx_view(ctx, 0, c);
    if (rc || (rc = conv_view(args, false, v, vec))) return rc;
    if (v.B == 0 || (v.T == 0 && !window_out)) return GORILA_OK;
    const int e = dtype_bytes(args->dtype);
    if ((v.T > 0 && !y) || !at_element(y, e) || !at_element(window_out, e)) return GORILA_EINVAL;
    if (window_out && window_out == args->window) return GORILA_EINVAL;
    vec = vec && at_four(y, e) && at_four(window_out, e);
    v.y = y;
    v.window_out = window_out;
    v.quads = vec ? v.C / 4 : v.C;
    by_taps(args->taps, args->dtype, vec, [&](auto t, auto k, auto al) {
        conv_kernel<decltype(t), decltype(k)::value, decltype(al)::value>
            <<<lanes_grid((int64_t)v.B * v.runs * v.quads), 256, 0, c.stream>>>(v);
    });
    return launched();
}

size_t gorila_causal_conv_workspace_bytes(int32_t channels, int32_t taps) {
    if (channels < 1 || taps < 2 || taps > MAX_TAPS) return 0;
    return WS_FIXED_BYTES + (size_t)MAX_PARTS * channels * (taps + 1) * 4;
}

int gorila_causal_conv_backward(const gorila_causal_conv_args* args, const void* dy, int64_t dy_batch_stride,
                                int64_t dy_step_stride, const void* dwindow_out, void* dx, float* dweight, float* dbias,
                                void* dwindow, gorila_ctx* ctx) {
    ConvView v;
    CtxView c;
    bool vec;
    int rc = ctx_view(ctx, 0, c);
    if (rc || (rc = conv_view(args, false, v, vec))) return rc;
    const int e = dtype_bytes(args->dtype);
    if (!dweight || (args->bias && !dbias)) return GORILA_EINVAL;
    if (v.B > 0 && v.T > 0 && (!dy || !dx)) return GORILA_EINVAL;
    for (const void* p : {dy, dwindow_out, (const void*)dx, (const void*)dwindow})
        if (!at_element(p, e)) return GORILA_EINVAL;
    if (!at_element(dweight, 4) || !at_element(dbias, 4)) return GORILA_EINVAL;
    const size_t cols = (size_t)v.C * (args->taps + 1);
    if ((rc = ctx_view(ctx, MAX_PARTS * cols * 4, c))) return rc;
    vec = vec && !((dy_batch_stride | dy_step_stride) & 3) && at_four(dy, e) && at_four(dx, e) && at_four(dwindow_out, e) &&
          at_four(dwindow, e);
    v.dy = dy, v.dyb = dy_batch_stride, v.dyt = dy_step_stride;
    v.dwindow_out = dwindow_out, v.dx = dx, v.dwindow = dwindow;
    v.quads = vec ? v.C / 4 : v.C;
    v.sums = (float*)c.ws;
    const int64_t units = (int64_t)v.B * v.runs;
    v.parts = (int)(units < MAX_PARTS ? units : MAX_PARTS);
    if (v.parts > 0)
        by_taps(args->taps, args->dtype, vec, [&](auto t, auto k, auto al) {
            conv_backward_kernel<decltype(t), decltype(k)::value, decltype(al)::value>
                <<<lanes_grid((int64_t)v.parts * v.quads), 256, 0, c.stream>>>(v);
        });
    launch_sum_parts(v.sums, v.parts, (int64_t)cols, (int64_t)v.C * args->taps, dweight, dbias, c.stream);
    return launched();
}

int gorila_causal_conv_step(const gorila_causal_conv_args* args, void* window_pool, int64_t slots, const int32_t* slot, void* y,
                            gorila_ctx* ctx) {
    ConvView v;
    CtxView c;
    bool vec;
    int rc = ctx_view(ctx, 0, c);
    if (rc || (rc = conv_view(args, true, v, vec))) return rc;
    if (v.T != 1 || slots < 0) return GORILA_EINVAL;
    if (v.B == 0) return GORILA_OK;
    const int e = dtype_bytes(args->dtype);
    if (!window_pool || !y || !at_element(window_pool, e) || !at_element(y, e) || !at_element(slot, 4)) return GORILA_EINVAL;
    if (slot ? !c.err : slots < v.B) return slot ? GORILA_EWORKSPACE : GORILA_EINVAL;
    vec = vec && at_four(window_pool, e) && at_four(y, e);
    v.y = y;
    v.quads = vec ? v.C / 4 : v.C;
    by_taps(args->taps, args->dtype, vec, [&](auto t, auto k, auto al) {
        using T = decltype(t);
        conv_step_kernel<T, decltype(k)::value, decltype(al)::value>
            <<<lanes_grid((int64_t)v.B * v.quads), 256, 0, c.stream>>>(v, (T*)window_pool, slots, slot, c.err);
    });
    return launched();
}

}  // extern "C"
