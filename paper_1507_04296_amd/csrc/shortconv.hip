// The short causal convolution (gorila_causal_conv, _backward, _step).
//
// Memory bound.  A lane takes four channels (backward two; one, where quads are not
// aligned) and walks a run of steps with the last taps in a ring of registers, the
// loads of the next four steps ahead of it, so a value is read once (and once more by
// the next run's lane, from the cache).  A wave has one run, so that its steps, episode starts and
// addresses are scalars: with runs that differ in a wave, the address arithmetic and
// the masks were twice the convolution, and a wait for every step's reset cost 0.5 us a
// step.  An episode start empties the ring: nothing before it is multiplied, whatever
// it holds.
//
// 32 sequences of 128 steps, 1152 channels, fp32: 10.6 us forward (3.6 TB/s), 23.2 us
// backward with the sums of the workgroups' gradients of the taps (2.4 TB/s).  1 x 8192
// steps: 18.3 and 42.7 us.  Backward, 4 x 2000 steps, 2304 channels, bf16: 56.6 us with
// two channels a lane, 70.9 with four (half the waves, 192 registers), 64.3 with one.
#include "seq.h"

namespace gorila {
namespace {

constexpr int RUN = 8;          // steps a lane, forward
constexpr int BACK_RUN = 16;    // and backward, which walks K - 1 more
constexpr int BACK_W = 2;      // channels a lane, backward
constexpr int MAX_TAPS = 4;
constexpr int MAX_PARTS = 512;  // of the weight gradient's sums
constexpr int MAX_SIZE = 1 << 30;  // steps, channels, runs: sums of them and of a workgroup's are 32 bits

struct ConvView {
    const void *x, *window, *dy, *dwindow_out;
    int64_t xb, xt, dyb, dyt;
    const float *weight, *bias;
    const uint8_t* reset;
    int B, T, C, silu, runs, quads, parts;
    int blocks;  // of a run's lanes
    void *y, *window_out, *dx, *dwindow;
    float* sums;
};

// W channels (1, 2 or 4) from p.
template <int W> using Vec = float __attribute__((ext_vector_type(W)));
template <int W, class T>
__device__ __forceinline__ Vec<W> get(const T* p) {
    constexpr bool F = std::is_same<T, float>::value;
    if constexpr (W == 4) return row_load4(p);
    else if constexpr (W == 2 && F) return *(const Vec<2>*)p;
    else if constexpr (W == 2) {
        const uint32_t v = *(const uint32_t*)p;
        return Vec<2>{__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u)};
    } else {
        Vec<1> v;
        v[0] = row_value(p[0]);
        return v;
    }
}
template <int W, class T>
__device__ __forceinline__ void put(T* p, Vec<W> v) {
    constexpr bool F = std::is_same<T, float>::value;
    if constexpr (W == 4) row_store4(p, v);
    else if constexpr (W == 2 && F) *(Vec<2>*)p = v;
    else if constexpr (W == 2) *(uint32_t*)p = (uint32_t)row_round<uint16_t>(v[0]) | (uint32_t)row_round<uint16_t>(v[1]) << 16;
    else p[0] = row_round<T>(v[0]);
}

template <int K, int W>
__device__ __forceinline__ void load_taps(const ConvView& s, int c, Vec<W> (&w)[K], Vec<W>& bias) {
#pragma unroll
    for (int j = 0; j < K; ++j) {
        w[j] = Vec<W>(0.0f);
#pragma unroll
        for (int i = 0; i < W; ++i) w[j][i] = s.weight[(int64_t)(c + i) * K + j];
    }
    bias = s.bias ? get<W>(s.bias + c) : Vec<W>(0.0f);
}

// The steps that a walk loads ahead: whole turns of the ring of K.
template <int K> constexpr int ahead() { return K == 3 ? 3 : 4; }

// Episode starts as bits, bit i for step t + i (64 of them; none outside the sequence).
__device__ __forceinline__ uint64_t starts_from(const uint8_t* rs, int t, int T) {
    if (!rs) return 0;
    const int at = t + (int)(threadIdx.x & 63);
    return __ballot(at >= 0 && at < T && rs[at >= 0 && at < T ? at : 0] != 0);
}

// Ring places of the K - 1 steps before t0 (step t at place (t - t0) mod K): their
// values, or zeros where an episode starts behind them.  starts: from t0 - (K - 1) on.
template <class T, int K, int W>
__device__ __forceinline__ void load_past(const ConvView& s, int b, int c, int t0, const T* x, uint64_t starts, Vec<W> (&e)[K]) {
    e[0] = Vec<W>(0.0f);
#pragma unroll
    for (int j = 1; j < K; ++j) {  // step t0 - j
        const int t = t0 - j;
        Vec<W> v = Vec<W>(0.0f);
        const uint64_t behind = (starts >> (K - j)) & ((1ull << (j - 1)) - 1);  // steps t + 1 .. t0 - 1
        if (!behind) {
            if (t >= 0) v = get<W>(x + (int64_t)t * s.xt);
            else if (s.window) v = get<W>((const T*)s.window + ((int64_t)b * (K - 1) + K - 1 + t) * s.C + c);
        }
        e[K - j] = v;
    }
}

// The exponential's argument is rounded once (2^-24 of |v| log2 e), it and the reciprocal
// are exact to a unit each: the relative error is about (2 + |v|) 2^-23, 1e-6 at v = -8
// and 1e-5 at -80, where the value is 1e-35.  The exact quotient and the library's
// exponential took a third of these kernels' time.
__device__ __forceinline__ float sigmoid(float v) {
    return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(v * -1.44269504088896341f));
}

template <class T, int K, int W>
__global__ __launch_bounds__(256) void conv_kernel(ConvView s) {
    constexpr int A = ahead<K>();
    const int unit = (int)(blockIdx.x / (unsigned)s.blocks), run = unit % s.runs, b = unit / s.runs;
    const int quad = (int)(blockIdx.x % (unsigned)s.blocks) * (int)blockDim.x + (int)threadIdx.x;
    const int t0 = run * RUN, t1 = t0 + RUN < s.T ? t0 + RUN : s.T;
    const uint64_t starts = starts_from(s.reset ? s.reset + (int64_t)b * s.T : nullptr, t0 - (K - 1), s.T);
    if (quad >= s.quads) return;
    const int c = quad * W;
    const T* x = (const T*)s.x + b * s.xb + c;
    T* y = (T*)s.y + (int64_t)b * s.T * s.C + c;
    Vec<W> w[K], bias, e[K], now[A], next[A];
    load_taps<K, W>(s, c, w, bias);
    load_past<T, K, W>(s, b, c, t0, x, starts, e);
    auto load = [&](int t, Vec<W> (&v)[A]) {  // steps past the run's take its last one's place
#pragma unroll
        for (int u = 0; u < A; ++u) v[u] = get<W>(x + (int64_t)(t + u < t1 ? t + u : t1 - 1) * s.xt);
    };
    if (t0 < t1) load(t0, now);
    for (int tb = t0; tb < t1; tb += A) {
        load(tb + A, next);
#pragma unroll
        for (int u = 0; u < A; ++u) {
            const int t = tb + u;
            if (t < t1) {
                if (starts >> (t - t0 + K - 1) & 1u) {
#pragma unroll
                    for (int j = 0; j < K; ++j) e[j] = Vec<W>(0.0f);
                }
                e[u % K] = now[u];
                Vec<W> v = bias;
#pragma unroll
                for (int j = 0; j < K; ++j) v += w[j] * e[(u + 1 + j) % K];
                if (s.silu) {
#pragma unroll
                    for (int i = 0; i < W; ++i) v[i] *= sigmoid(v[i]);
                }
                put<W>(y + (int64_t)t * s.C, v);
            }
            now[u] = next[u];
        }
    }
    if (s.window_out && run == s.runs - 1) {  // step T - (K - 1) + j at its place of the ring
        const int n = t1 - t0;
#pragma unroll
        for (int j = 0; j < K - 1; ++j) {
            Vec<W> v = Vec<W>(0.0f);
#pragma unroll
            for (int i = 0; i < K; ++i)
                if ((n - (K - 1) + j + K) % K == i) v = e[i];
            put<W>((T*)s.window_out + ((int64_t)b * (K - 1) + j) * s.C + c, v);
        }
    }
}

// A workgroup walks units (runs of sequences) part, part + parts, ...  In a run it
// forms the gradient of v for its steps and the K - 1 after them, and keeps the sums of
// dx of the last K steps in a ring.  A step's is written when its last tap has passed,
// or an episode starts.
template <class T, int K, int W>
__global__ __launch_bounds__(256) void conv_backward_kernel(ConvView s) {
    constexpr int A = ahead<K>();
    static_assert(BACK_RUN + 2 * (K - 1) <= 64, "a bit a step");
    const int part = (int)(blockIdx.x / (unsigned)s.blocks);
    const int quad = (int)(blockIdx.x % (unsigned)s.blocks) * (int)blockDim.x + (int)threadIdx.x;
    const int c = (quad < s.quads ? quad : 0) * W;
    Vec<W> w[K], bias, dw[K], db = Vec<W>(0.0f);
    load_taps<K, W>(s, c, w, bias);
#pragma unroll
    for (int j = 0; j < K; ++j) dw[j] = Vec<W>(0.0f);
    for (int unit = part; unit < s.B * s.runs; unit += s.parts) {
        const int run = unit % s.runs, b = unit / s.runs;
        const int t0 = run * BACK_RUN, t1 = t0 + BACK_RUN < s.T ? t0 + BACK_RUN : s.T;
        const uint8_t* rs = s.reset ? s.reset + (int64_t)b * s.T : nullptr;
        const uint64_t starts = starts_from(rs, t0 - (K - 1), s.T), tail = starts_from(rs, s.T - (K - 1), s.T);
        if (quad >= s.quads) continue;
        const T* x = (const T*)s.x + b * s.xb + c;
        const T* dy = (const T*)s.dy + b * s.dyb + c;
        T* dx = (T*)s.dx + (int64_t)b * s.T * s.C + c;
        const T* dwo = s.dwindow_out ? (const T*)s.dwindow_out + (int64_t)b * (K - 1) * s.C + c : nullptr;
        T* dwi = s.dwindow ? (T*)s.dwindow + (int64_t)b * (K - 1) * s.C + c : nullptr;
        Vec<W> e[K], d[K], xs[A], gs[A], nx[A], ng[A];  // rings: step t at place (t - t0) mod K
        load_past<T, K, W>(s, b, c, t0, x, starts, e);
#pragma unroll
        for (int j = 0; j < K; ++j) d[j] = Vec<W>(0.0f);
        const int end = t1 + K - 1, most = (end < s.T ? end : s.T) - 1;
        auto load = [&](int t, Vec<W> (&vx)[A], Vec<W> (&vg)[A]) {
#pragma unroll
            for (int u = 0; u < A; ++u) {
                const int at = t + u < most ? t + u : most;
                vx[u] = get<W>(x + (int64_t)at * s.xt);
                vg[u] = get<W>(dy + (int64_t)at * s.dyt);
            }
        };
        int done = run == 0 ? -(K - 1) : t0;  // the next step to write; of the first run, the window's before
        // Writes step `at` if it is this run's; the window behind the sequence adds its
        // gradient where no episode starts after it.
        auto write = [&](int at, Vec<W> v) {
            if (at < done || at >= t1) return;
            done = at + 1;
            const int k = at - (s.T - (K - 1));  // its place in the window behind
            if (dwo && k >= 0 && !(tail >> (k + 1))) v += get<W>(dwo + (int64_t)k * s.C);
            if (at >= 0) put<W>(dx + (int64_t)at * s.C, v);
            else if (dwi) put<W>(dwi + (int64_t)(at + K - 1) * s.C, v);
        };
        if (s.T > 0) load(t0, xs, gs);
        for (int tb = t0; tb < end; tb += A) {
            if (s.T > 0) load(tb + A, nx, ng);
#pragma unroll
            for (int u = 0; u < A; ++u) {
                const int t = tb + u;
                if (t < end) {
                    if (t < s.T) {  // past the end nothing is added
                        if (starts >> (t - t0 + K - 1) & 1u) {
#pragma unroll
                            for (int j = K - 1; j >= 1; --j) write(t - j, d[(u + K - j) % K]);
#pragma unroll
                            for (int j = 0; j < K; ++j) e[j] = Vec<W>(0.0f);
                        }
                        e[u % K] = xs[u];
                        Vec<W> dv = gs[u];
                        if (s.silu) {
                            Vec<W> v = bias;
#pragma unroll
                            for (int j = 0; j < K; ++j) v += w[j] * e[(u + 1 + j) % K];
#pragma unroll
                            for (int i = 0; i < W; ++i) {
                                const float g = sigmoid(v[i]);
                                dv[i] *= g * (1.0f + v[i] * (1.0f - g));
                            }
                        }
                        if (t < t1) {
                            db += dv;
#pragma unroll
                            for (int j = 0; j < K; ++j) dw[j] += dv * e[(u + 1 + j) % K];
                        }
                        d[u % K] = Vec<W>(0.0f);
#pragma unroll
                        for (int j = 0; j < K; ++j) d[(u + 1 + j) % K] += w[j] * dv;
                    } else {
                        d[u % K] = Vec<W>(0.0f);
                    }
                    write(t - (K - 1), d[(u + 1) % K]);  // its last tap has passed
                }
                xs[u] = nx[u];
                gs[u] = ng[u];
            }
        }
    }
    if (quad >= s.quads) return;
    float* o = s.sums + part * (int64_t)s.C * (K + 1);
#pragma unroll
    for (int j = 0; j < K; ++j) put<W>(o + (int64_t)j * s.C + c, dw[j]);  // [taps][channels]
    put<W>(o + (int64_t)K * s.C + c, db);
}

template <class T, int K, int W>
__global__ __launch_bounds__(256) void conv_step_kernel(ConvView s, T* pool, int64_t slots, const int32_t* slot, unsigned* err) {
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
    Vec<W> w[K], bias, e[K];
    load_taps<K, W>(s, c, w, bias);
#pragma unroll
    for (int j = 0; j < K - 1; ++j) e[j] = empty ? Vec<W>(0.0f) : get<W>(p + (int64_t)j * s.C);
    e[K - 1] = get<W>((const T*)s.x + row * s.xb + c);
    Vec<W> v = bias;
#pragma unroll
    for (int j = 0; j < K; ++j) v += w[j] * e[j];
    if (s.silu) {
#pragma unroll
        for (int i = 0; i < W; ++i) v[i] *= sigmoid(v[i]);
    }
    put<W>((T*)s.y + row * s.C + c, v);
    if (!out) {
#pragma unroll
        for (int j = 0; j < K - 1; ++j) put<W>(p + (int64_t)j * s.C, e[j + 1]);
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
    if (v.T > MAX_SIZE || v.C > MAX_SIZE) return GORILA_EUNSUPPORTED;
    v.runs = v.T > 0 ? (v.T + RUN - 1) / RUN : 1;  // the backward takes fewer
    vec = !((v.C | v.xb | (step ? 0 : v.xt)) & 3) && at_four(a->x, e) && at_four(v.window, e) && at_four(a->bias, 4);
    return (int64_t)v.B * v.runs > MAX_SIZE ? GORILA_EUNSUPPORTED : GORILA_OK;
}

template <class F>
void by_taps(int taps, int dtype, bool vec, F&& f) {
    auto al = [&](auto t, auto k) { vec ? f(t, k, std::true_type{}) : f(t, k, std::false_type{}); };
    auto ty = [&](auto k) { dtype == GORILA_F32 ? al(float{}, k) : al(uint16_t{}, k); };
    if (taps == 2) ty(std::integral_constant<int, 2>{});
    else if (taps == 3) ty(std::integral_constant<int, 3>{});
    else ty(std::integral_constant<int, 4>{});
}

// Threads a workgroup (whole waves) for a run's lanes, and workgroups a run.
int run_threads(ConvView& v) {
    const int threads = v.quads < 256 ? (v.quads + 63) / 64 * 64 : 256;
    v.blocks = (v.quads + threads - 1) / threads;
    // lanes that are left over: as many workgroups of fewer waves
    const int waves = (v.quads + 63) / 64, per = (waves + v.blocks - 1) / v.blocks;
    v.blocks = (waves + per - 1) / per;
    return per * 64;
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
    const int threads = run_threads(v);
    if (!launch_fits((double)v.B * v.runs * v.blocks, threads)) return GORILA_EUNSUPPORTED;
    by_taps(args->taps, args->dtype, vec, [&](auto t, auto k, auto al) {
        conv_kernel<decltype(t), decltype(k)::value, decltype(al)::value ? 4 : 1>
            <<<(unsigned)(v.B * v.runs * v.blocks), threads, 0, c.stream>>>(v);
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
    v.quads = vec ? v.C / BACK_W : v.C;
    const int threads = run_threads(v);
    v.sums = (float*)c.ws;
    v.runs = v.T > 0 ? (v.T + BACK_RUN - 1) / BACK_RUN : 1;
    const int64_t units = (int64_t)v.B * v.runs;
    v.parts = (int)(units < MAX_PARTS ? units : MAX_PARTS);
    // the sums take 64 lanes a column
    if (!launch_fits((double)v.parts * v.blocks, threads) || !launch_fits((double)cols, 64)) return GORILA_EUNSUPPORTED;
    if (v.parts > 0)
        by_taps(args->taps, args->dtype, vec, [&](auto t, auto k, auto al) {
            conv_backward_kernel<decltype(t), decltype(k)::value, decltype(al)::value ? BACK_W : 1>
                <<<(unsigned)(v.parts * v.blocks), threads, 0, c.stream>>>(v);
        });
    launch_sum_parts(v.sums, v.parts, (int64_t)cols, (int64_t)v.C * args->taps, args->taps, dweight, dbias, c.stream);
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
    if (!launch_fits((double)v.B * v.quads + 255, 1)) return GORILA_EUNSUPPORTED;
    by_taps(args->taps, args->dtype, vec, [&](auto t, auto k, auto al) {
        using T = decltype(t);
        conv_step_kernel<T, decltype(k)::value, decltype(al)::value ? 4 : 1>
            <<<lanes_grid((int64_t)v.B * v.quads), 256, 0, c.stream>>>(v, (T*)window_pool, slots, slot, c.err);
    });
    return launched();
}

}  // extern "C"
