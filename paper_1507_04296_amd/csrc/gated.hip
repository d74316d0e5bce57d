// Gated scan (gorila_gated_scan, _backward, _step): h_t = a_t h_{t-1} + b_t i_t x_t in every
// channel, with a = exp(-exp(a_log) sigmoid(gate_a)), b = sqrt(1 - a^2), i = sigmoid(gate_x).
//
// Memory bound where it can be: a step of a channel is 40 operations forward and 100
// backward on 4 and 7 values.  So a value is read once: the steps of a chunk lie in the
// lanes' registers (4 steps of 4 channels a lane, 16 lanes a step, 4 runs of steps a
// wave), each lane runs through its own steps from zero, and what enters a lane's run is
// joined from the products of decays and the ends of the runs before it: over the lanes
// of a wave by shuffles, over the waves in LDS, over the chunks in registers.  An episode
// start is a flag beside the product of decays, not a factor of zero: what is before
// it may be infinite.
#include "seq.h"

namespace gorila {
namespace {

constexpr int STEPS = 4, RUNS = 4, TILE = 64;  // steps a lane, runs a wave, channels a workgroup
constexpr int WAVES = 4, BLOCK = 64 * WAVES, CHUNK = STEPS * RUNS * WAVES;
static_assert(CHUNK == GORILA_GATED_MARK, "a chunk of the backward starts at a mark");
constexpr float LOG2E = 1.44269504088896341f;

struct Rows {
    const void* p;
    int64_t b, t;  // strides
};
struct GatedView {
    int B, T, C, tiles, nseg, seg;  // segments, and steps of one
    Rows x, ga, gx, dy;
    const float *a_log, *state, *dstate_out, *marks_in;
    const uint8_t* reset;
    void *y, *dx, *dga, *dgx;
    float *state_out, *marks, *dstate;
    float* state_copy;     // [B][C] where there are segments: state_out may be state
    float *seg_a, *seg_h;  // [B][nseg][C]: product of decays (negative: an episode starts in the segment), end
    float* parts;          // [items][C] of da_log
    int items;             // workgroups that share a tile's sequences and segments
};

__device__ __forceinline__ float sigmoid(float v) {
    return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(v * -LOG2E));
}
__device__ __forceinline__ float rate_of(float a_log) {
    const float e = expf(a_log);
    return e > 3.40282347e38f ? 3.40282347e38f : e;  // (NaN stays)
}
// a = exp(l) and b = sqrt(1 - a^2) for l <= 0: 1 - exp(u), u = 2 l, is its series where
// u > -1/2 (the next term is 2^-27 of the sum).
struct Decay {
    float a, b;
};
__device__ __forceinline__ Decay decay(float l) {
    const float a = __builtin_amdgcn_exp2f(l * LOG2E);
    const float u = 2.0f * l;
    float s = fmaf(u, 1.0f / 40320.0f, 1.0f / 5040.0f);
    s = fmaf(u, s, 1.0f / 720.0f);
    s = fmaf(u, s, 1.0f / 120.0f);
    s = fmaf(u, s, 1.0f / 24.0f);
    s = fmaf(u, s, 1.0f / 6.0f);
    s = fmaf(u, s, 0.5f);
    s = fmaf(u, s, 1.0f);
    const float q = u > -0.5f ? -u * s : fmaf(-a, a, 1.0f);
    return {a, __builtin_amdgcn_sqrtf(q)};
}

// A run of steps as a map of the state before it: h -> cut ? end : a h + end.
struct Map {
    f32x4 a, h;
    bool cut;
};
__device__ __forceinline__ f32x4 through(const Map& m, f32x4 h) {
    f32x4 o;
#pragma unroll
    for (int j = 0; j < 4; ++j) o[j] = m.cut ? m.h[j] : fmaf(m.a[j], h[j], m.h[j]);
    return o;
}
// `later` after `first`.
__device__ __forceinline__ Map join(const Map& first, const Map& later) {
    Map o;
    o.a = first.a * later.a;
    o.h = through(later, first.h);
    o.cut = first.cut || later.cut;
    return o;
}
__device__ __forceinline__ Map none() { return Map{f32x4{1.0f, 1.0f, 1.0f, 1.0f}, f32x4{0.0f, 0.0f, 0.0f, 0.0f}, false}; }
__device__ __forceinline__ Map moved(const Map& m, int by) {  // of the lane `by` further
    Map o;
#pragma unroll
    for (int j = 0; j < 4; ++j) o.a[j] = __shfl(m.a[j], (threadIdx.x + by) & 63, 64), o.h[j] = __shfl(m.h[j], (threadIdx.x + by) & 63, 64);
    o.cut = __shfl((int)m.cut, (threadIdx.x + by) & 63, 64);
    return o;
}
// The map of the runs before this lane's in its wave (BACK: behind it); `all` that of the wave's last (first)
// run and all others.
template <bool BACK>
__device__ __forceinline__ Map before(const Map& own, Map& all) {
    const int g = BACK ? RUNS - 1 - (threadIdx.x & 63) / 16 : (threadIdx.x & 63) / 16;
    const int dir = BACK ? 1 : -1;
    Map m = own, p = moved(m, dir * 16);
    if (g >= 1) m = join(p, m);
    p = moved(m, dir * 32);
    if (g >= 2) m = join(p, m);
    all = m;  // in the lanes of the last run
    p = moved(m, dir * 16);
    return g >= 1 ? p : none();
}

// One wave's map in LDS.
struct Shared {
    f32x4 a[WAVES][16], h[WAVES][16];
    int cut[WAVES];
};
// What enters this lane's run, and what leaves the chunk, of what enters the chunk
// (`carry`, replaced).  The caller uses two Shared in turn: one barrier a chunk.
template <bool BACK>
__device__ __forceinline__ f32x4 enter(const Map& own, f32x4& carry, Shared& sh) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = lane & 15;
    Map all;
    const Map inside = before<BACK>(own, all);
    if (lane / 16 == (BACK ? 0 : RUNS - 1)) {
        sh.a[wave][c] = all.a;
        sh.h[wave][c] = all.h;
        if (c == 0) sh.cut[wave] = all.cut;
    }
    __syncthreads();
    f32x4 mine = carry;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) {
        const int w = BACK ? WAVES - 1 - i : i;
        if (w == wave) mine = carry;
        carry = through(Map{sh.a[w][c], sh.h[w][c], sh.cut[w] != 0}, carry);
    }
    return through(inside, mine);
}

// The steps of a lane's run: x and the gates as they are read.
struct Steps {
    f32x4 x[STEPS], ga[STEPS], gx[STEPS];
    bool start[STEPS], in[STEPS];
};
template <bool VEC, class T>
__device__ __forceinline__ f32x4 load(const Rows& r, int64_t b, int64_t t, int c, int n) {
    return row_load<VEC>((const T*)r.p + b * r.b + t * r.t + c, n);
}
// Time t0 and on, channels c and on (n of them, 0: none); what is past the end moves nothing.
template <bool VEC, class T, bool X>
__device__ __forceinline__ void load_steps(Steps& s, const GatedView& v, int64_t b, int t0, int end, int c, int n) {
#pragma unroll
    for (int k = 0; k < STEPS; ++k) {
        const int t = t0 + k;
        s.in[k] = t < end;
        const int m = s.in[k] ? n : 0, at = s.in[k] ? t : 0, ch = m > 0 ? c : 0;
        s.ga[k] = load<VEC, T>(v.ga, b, at, ch, m);
        if (X) {
            s.x[k] = load<VEC, T>(v.x, b, at, ch, m);
            s.gx[k] = load<VEC, T>(v.gx, b, at, ch, m);
        }
        s.start[k] = s.in[k] && v.reset && v.reset[b * v.T + t];
    }
}

// Forward.  A workgroup walks the chunks of one segment of 64 channels.
// AGG: the segment's map alone, for the workgroups of the segments behind it.
template <class T, bool VEC, bool AGG>
__global__ __launch_bounds__(BLOCK) void gated_kernel(GatedView v) {
    __shared__ Shared sh[2];
    const int tile = blockIdx.x % v.tiles, item = blockIdx.x / v.tiles, seg = item % v.nseg;
    const int64_t b = item / v.nseg;
    const int lane = threadIdx.x & 63, q = threadIdx.x / 16, c = tile * TILE + (lane & 15) * 4, n = v.C - c > 0 ? v.C - c : 0;
    if (AGG && seg == v.nseg - 1) return;
    const int begin = seg * v.seg, end = begin + v.seg < v.T ? begin + v.seg : v.T;
    f32x4 rate = row_load<VEC>(v.a_log + (n > 0 ? c : 0), n);
#pragma unroll
    for (int j = 0; j < 4; ++j) rate[j] = rate_of(rate[j]);
    f32x4 carry{0.0f, 0.0f, 0.0f, 0.0f}, prod{1.0f, 1.0f, 1.0f, 1.0f};
    bool cut = false;
    if (AGG) {
        if (seg == 0 && q == 0 && n > 0) row_store<VEC>(v.state_copy + b * v.C + c, v.state ? row_load<VEC>(v.state + b * v.C + c, n) : carry, n);
    } else {
        const float* from = v.nseg > 1 ? v.state_copy : v.state;
        if (from) carry = row_load<VEC>(from + b * v.C + (n > 0 ? c : 0), n);
        for (int s = 0; s < seg; ++s) {
            const int64_t at = (b * v.nseg + s) * v.C + (n > 0 ? c : 0);
            const f32x4 a = row_load<VEC>(v.seg_a + at, n), h = row_load<VEC>(v.seg_h + at, n);
#pragma unroll
            for (int j = 0; j < 4; ++j) carry[j] = a[j] < 0.0f ? h[j] : fmaf(a[j], carry[j], h[j]);
        }
    }
    int turn = 0;
    for (int t0 = begin; t0 < end; t0 += CHUNK, turn ^= 1) {
        Steps s;
        load_steps<VEC, T, true>(s, v, b, t0 + q * STEPS, end, c, n);
        if (!AGG && v.marks && q == 0 && n > 0)
            row_store<VEC>(v.marks + (b * ((v.T + CHUNK - 1) / CHUNK) + t0 / CHUNK) * v.C + c, carry, n);
        f32x4 a[STEPS], u[STEPS];
        Map own = none();
#pragma unroll
        for (int k = 0; k < STEPS; ++k) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const Decay d = decay(-rate[j] * sigmoid(s.ga[k][j]));
                a[k][j] = d.a;
                u[k][j] = (s.start[k] ? 1.0f : d.b) * sigmoid(s.gx[k][j]) * s.x[k][j];
                if (!s.in[k]) a[k][j] = 1.0f, u[k][j] = 0.0f;
                own.h[j] = s.start[k] ? u[k][j] : fmaf(a[k][j], own.h[j], u[k][j]);
                own.a[j] *= a[k][j];
            }
            own.cut = own.cut || s.start[k];
        }
        if (AGG) {
            enter<false>(own, carry, sh[turn]);
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                prod *= sh[turn].a[w][lane & 15];
                cut = cut || sh[turn].cut[w] != 0;
            }
            continue;
        }
        f32x4 h = enter<false>(own, carry, sh[turn]);
#pragma unroll
        for (int k = 0; k < STEPS; ++k) {
#pragma unroll
            for (int j = 0; j < 4; ++j) h[j] = s.start[k] ? u[k][j] : fmaf(a[k][j], h[j], u[k][j]);
            if (s.in[k] && n > 0) row_store<VEC>((T*)v.y + (b * v.T + t0 + q * STEPS + k) * v.C + c, h, n);
        }
    }
    if (q != 0 || n <= 0) return;
    if (AGG) {
        const int64_t at = (b * v.nseg + seg) * v.C + c;
        if (cut) prod = f32x4{-1.0f, -1.0f, -1.0f, -1.0f};
        row_store<VEC>(v.seg_a + at, prod, n);
        row_store<VEC>(v.seg_h + at, carry, n);
    } else if (seg == v.nseg - 1 && v.state_out) {
        row_store<VEC>(v.state_out + b * v.C + c, carry, n);
    }
}

// What passes back through a segment, for the segments before it: back -> a back + end.
template <class T, bool VEC>
__global__ __launch_bounds__(BLOCK) void gated_back_kernel(GatedView v) {
    __shared__ Shared sh[2];
    const int tile = blockIdx.x % v.tiles, item = blockIdx.x / v.tiles, seg = item % v.nseg;
    const int64_t b = item / v.nseg;
    const int lane = threadIdx.x & 63, q = threadIdx.x / 16, c = tile * TILE + (lane & 15) * 4, n = v.C - c > 0 ? v.C - c : 0;
    if (seg == 0) return;
    const int begin = seg * v.seg, end = begin + v.seg < v.T ? begin + v.seg : v.T;
    f32x4 rate = row_load<VEC>(v.a_log + (n > 0 ? c : 0), n);
#pragma unroll
    for (int j = 0; j < 4; ++j) rate[j] = rate_of(rate[j]);
    f32x4 carry{0.0f, 0.0f, 0.0f, 0.0f}, prod{1.0f, 1.0f, 1.0f, 1.0f};
    bool cut = false;
    int turn = 0;
    for (int t0 = begin + (end - begin - 1) / CHUNK * CHUNK; t0 >= begin && t0 < end; t0 -= CHUNK, turn ^= 1) {
        Steps s;
        load_steps<VEC, T, false>(s, v, b, t0 + q * STEPS, end, c, n);
        Map own = none();
#pragma unroll
        for (int k = STEPS - 1; k >= 0; --k) {
            const int t = t0 + q * STEPS + k, m = s.in[k] ? n : 0;
            const f32x4 dy = load<VEC, T>(v.dy, b, s.in[k] ? t : 0, m > 0 ? c : 0, m);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float a = s.in[k] ? __builtin_amdgcn_exp2f(-rate[j] * sigmoid(s.ga[k][j]) * LOG2E) : 1.0f;
                own.h[j] = s.start[k] ? 0.0f : a * (own.h[j] + dy[j]);
                own.a[j] *= a;
            }
            own.cut = own.cut || s.start[k];
        }
        enter<true>(own, carry, sh[turn]);
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            prod *= sh[turn].a[w][lane & 15];
            cut = cut || sh[turn].cut[w] != 0;
        }
    }
    if (q != 0 || n <= 0) return;
    const int64_t at = (b * v.nseg + seg) * v.C + c;
    if (cut) prod = f32x4{-1.0f, -1.0f, -1.0f, -1.0f};
    row_store<VEC>(v.seg_a + at, prod, n);
    row_store<VEC>(v.seg_h + at, carry, n);
}

// Backward: with R_t = dy_t + a_{t+1} R_{t+1},
//   dx = R b i,   dgate_x = R b i (1 - i) x,   G = log a (R a h_{t-1} - R i x a^2 / b),
//   dgate_a = G (1 - r),   da_log = sum of G      (at a start G is zero).
// Chunks are walked from the last on; the state before one is its mark, so that both
// directions are in registers at once and every value is read once.
template <class T, bool VEC>
__global__ __launch_bounds__(BLOCK) void gated_backward_kernel(GatedView v) {
    __shared__ Shared sh[2], shf[2];
    __shared__ f32x4 sums[RUNS * WAVES][16];
    const int tile = blockIdx.x % v.tiles;
    const int lane = threadIdx.x & 63, q = threadIdx.x / 16, c = tile * TILE + (lane & 15) * 4, n = v.C - c > 0 ? v.C - c : 0;
    f32x4 rate = row_load<VEC>(v.a_log + (n > 0 ? c : 0), n), dal{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int j = 0; j < 4; ++j) rate[j] = rate_of(rate[j]);
    int turn = 0;
    for (int64_t item = blockIdx.x / v.tiles; item < (int64_t)v.B * v.nseg; item += v.items) {
        const int seg = (int)(item % v.nseg);
        const int64_t b = item / v.nseg;
        const int begin = seg * v.seg, end = begin + v.seg < v.T ? begin + v.seg : v.T;
        f32x4 carry{0.0f, 0.0f, 0.0f, 0.0f};
        if (v.dstate_out) carry = row_load<VEC>(v.dstate_out + b * v.C + (n > 0 ? c : 0), n);
        for (int s = v.nseg - 1; s > seg; --s) {
            const int64_t at = (b * v.nseg + s) * v.C + (n > 0 ? c : 0);
            const f32x4 a = row_load<VEC>(v.seg_a + at, n), h = row_load<VEC>(v.seg_h + at, n);
#pragma unroll
            for (int j = 0; j < 4; ++j) carry[j] = a[j] < 0.0f ? h[j] : fmaf(a[j], carry[j], h[j]);
        }
        for (int t0 = begin + (end - begin - 1) / CHUNK * CHUNK; t0 >= begin && t0 < end; t0 -= CHUNK, turn ^= 1) {
            Steps s;
            f32x4 dy[STEPS];
            load_steps<VEC, T, true>(s, v, b, t0 + q * STEPS, end, c, n);
#pragma unroll
            for (int k = 0; k < STEPS; ++k) {
                const int m = s.in[k] ? n : 0;
                dy[k] = load<VEC, T>(v.dy, b, s.in[k] ? t0 + q * STEPS + k : 0, m > 0 ? c : 0, m);
            }
            f32x4 mark = row_load<VEC>(v.marks_in + (b * ((v.T + CHUNK - 1) / CHUNK) + t0 / CHUNK) * v.C + (n > 0 ? c : 0), n);
            f32x4 a[STEPS], bb[STEPS], h[STEPS];  // h: the state before the step
            Map fwd = none(), own = none();
#pragma unroll
            for (int k = 0; k < STEPS; ++k) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    s.ga[k][j] = sigmoid(s.ga[k][j]);
                    s.gx[k][j] = sigmoid(s.gx[k][j]);
                    const Decay d = decay(-rate[j] * s.ga[k][j]);
                    a[k][j] = d.a, bb[k][j] = d.b;
                    if (!s.in[k]) a[k][j] = 1.0f, bb[k][j] = 0.0f;
                    if (s.start[k]) bb[k][j] = 1.0f;
                    const float u = bb[k][j] * s.gx[k][j] * s.x[k][j];
                    fwd.h[j] = s.start[k] ? u : fmaf(a[k][j], fwd.h[j], u);
                    fwd.a[j] *= a[k][j];
                }
                fwd.cut = fwd.cut || s.start[k];
            }
            own.a = fwd.a;
            own.cut = fwd.cut;
#pragma unroll
            for (int k = STEPS - 1; k >= 0; --k)
#pragma unroll
                for (int j = 0; j < 4; ++j) own.h[j] = s.start[k] ? 0.0f : a[k][j] * (own.h[j] + dy[k][j]);
            f32x4 now = enter<false>(fwd, mark, shf[turn]);
            f32x4 back = enter<true>(own, carry, sh[turn]);
#pragma unroll
            for (int k = 0; k < STEPS; ++k) {
                h[k] = now;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float u = bb[k][j] * s.gx[k][j] * s.x[k][j];
                    now[j] = s.start[k] ? u : fmaf(a[k][j], now[j], u);
                }
            }
#pragma unroll
            for (int k = STEPS - 1; k >= 0; --k) {
                f32x4 dx, dga, dgx;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float r = s.ga[k][j], i = s.gx[k][j], x = s.x[k][j], l = a[k][j] * (-rate[j] * r);
                    const float R = dy[k][j] + back[j], Ri = R * i;
                    dx[j] = Ri * bb[k][j];
                    dgx[j] = dx[j] * x * (1.0f - i);
                    // log a times a, before any other factor: log a may be as large as fp32 goes where a is 0;
                    // with log a, its quotient by b goes to zero as a root
                    const float over = bb[k][j] > 0.0f ? l * a[k][j] * __builtin_amdgcn_rcpf(bb[k][j]) : 0.0f;
                    const float G = s.start[k] ? 0.0f : R * (l * h[k][j]) - Ri * x * over;
                    dga[j] = G * (1.0f - r);
                    if (s.in[k]) dal[j] += G;
                    back[j] = s.start[k] ? 0.0f : a[k][j] * R;
                }
                if (s.in[k] && n > 0) {
                    const int64_t at = (b * v.T + t0 + q * STEPS + k) * v.C + c;
                    row_store<VEC>((T*)v.dx + at, dx, n);
                    row_store<VEC>((T*)v.dga + at, dga, n);
                    row_store<VEC>((T*)v.dgx + at, dgx, n);
                }
            }
        }
        if (seg == 0 && v.dstate && q == 0 && n > 0) row_store<VEC>(v.dstate + b * v.C + c, carry, n);
    }
    sums[q][lane & 15] = dal;
    __syncthreads();
    if (q != 0 || n <= 0) return;
#pragma unroll
    for (int k = 1; k < RUNS * WAVES; ++k) dal += sums[k][lane & 15];
    row_store<VEC>(v.parts + (int64_t)(blockIdx.x / v.tiles) * v.C + c, dal, n);
}

// One step of every row: four channels a lane.
template <class T, bool VEC>
__global__ __launch_bounds__(256) void gated_step_kernel(GatedView v, float* pool, int64_t slots, const int32_t* slot, unsigned* err) {
    const int quads = (v.C + 3) / 4;
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x, row = id / quads;
    if (row >= v.B) return;
    const int c = (int)(id % quads) * 4, n = v.C - c;
    int64_t at = slot ? slot[row] : row;
    const bool out = at < 0 || at >= slots, reset = out || (v.reset && v.reset[row]);
    if (out) {
        if (c == 0 && err) atomicOr(err, ERR_IDX_RANGE);
        at = 0;
    }
    const bool start = v.reset && v.reset[row];
    const f32x4 ga = load<VEC, T>(v.ga, row, 0, c, n), gx = load<VEC, T>(v.gx, row, 0, c, n), x = load<VEC, T>(v.x, row, 0, c, n);
    const f32x4 al = row_load<VEC>(v.a_log + c, n);
    float* st = pool + at * v.C + c;
    f32x4 h{0.0f, 0.0f, 0.0f, 0.0f};
    if (!reset) h = row_load<VEC>(st, n);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const Decay d = decay(-rate_of(al[j]) * sigmoid(ga[j]));
        const float u = (start ? 1.0f : d.b) * sigmoid(gx[j]) * x[j];
        h[j] = reset ? u : fmaf(d.a, h[j], u);
    }
    if (!out) row_store<VEC>(st, h, n);
    row_store<VEC>((T*)v.y + row * v.C + c, h, n);
}

// ---- host ----

constexpr int FULL = 512;       // workgroups that fill the chip
constexpr int LEAST_SEG = 256;  // steps of a segment at least
constexpr int MAX_SEG = 64;     // segments of a sequence at most
constexpr int WALKS = 2048;     // workgroups of the backward at most: each adds a part of da_log

struct Cut {
    int tiles, nseg = 1, seg;
    Cut(int64_t B, int T, int C) {
        tiles = (C + TILE - 1) / TILE;
        const int64_t have = B * tiles, want = have > 0 ? (FULL + have - 1) / have : 1, most = (T + LEAST_SEG - 1) / LEAST_SEG;
        int64_t k = want < most ? want : most;
        k = k < MAX_SEG ? k : MAX_SEG;
        whole(T);
        if (k < 2) return;
        seg = (int)((T + k - 1) / k + CHUNK - 1) / CHUNK * CHUNK;
        nseg = (T + seg - 1) / seg;
    }
    void whole(int T) { nseg = 1, seg = T > 0 ? T : 1; }
};

size_t up256(size_t n) { return (n + 255) / 256 * 256; }
// Bytes of the workspace: the segments' maps and the states before the first (cut
// calls have B * tiles < FULL, so B * nseg < 2 FULL / tiles), then the parts.
struct Plan {
    size_t maps, states, parts, total;
    Plan(int T, int C, bool backward) {
        const int tiles = (C + TILE - 1) / TILE;
        const size_t cut = T > LEAST_SEG ? 4 * (size_t)C : 0;
        maps = up256(cut * (2 * FULL / tiles + 1));
        states = up256(cut * (FULL / tiles + 1));
        parts = up256(backward ? 4 * (size_t)C * walks(tiles) : 0);
        total = 2 * maps + states + parts;
    }
    static int walks(int tiles) { return (WALKS + tiles - 1) / tiles; }
};

int gated_view(const gorila_gated_scan_args* a, bool step, GatedView& v, bool& vec) {
    if (!a || !row_dtype(a->dtype) || a->batch < 0 || a->length < 0 || a->channels < 1) return GORILA_EINVAL;
    if (a->length > 1 << 30 || a->channels > 1 << 30) return GORILA_EUNSUPPORTED;
    if (!a->a_log) return GORILA_EINVAL;
    if (a->batch > 0 && a->length > 0 && (!a->x || !a->gate_a || !a->gate_x)) return GORILA_EINVAL;
    const int e = dtype_bytes(a->dtype);
    for (const void* p : {a->x, a->gate_a, a->gate_x})
        if (!at_element(p, e)) return GORILA_EINVAL;
    for (const float* p : {a->a_log, a->state})
        if (!at_element(p, 4)) return GORILA_EINVAL;
    v = GatedView{};
    v.B = a->batch, v.T = a->length, v.C = a->channels;
    v.x = {a->x, a->x_batch_stride, a->x_step_stride};
    v.ga = {a->gate_a, a->gate_a_batch_stride, a->gate_a_step_stride};
    v.gx = {a->gate_x, a->gate_x_batch_stride, a->gate_x_step_stride};
    v.a_log = a->a_log, v.reset = a->reset, v.state = a->state;
    const int64_t strides = v.x.b | v.ga.b | v.gx.b | (step ? 0 : v.x.t | v.ga.t | v.gx.t);
    vec = !(v.C & 3) && !(strides & 3) && at_four(a->x, e) && at_four(a->gate_a, e) && at_four(a->gate_x, e) && at_four(a->a_log, 4) &&
          at_four(a->state, 4);
    return GORILA_OK;
}

template <class F>
void by_rows(int dtype, bool vec, F&& f) {
    if (dtype == GORILA_F32) vec ? f(float{}, std::true_type{}) : f(float{}, std::false_type{});
    else vec ? f(uint16_t{}, std::true_type{}) : f(uint16_t{}, std::false_type{});
}

}  // namespace
}  // namespace gorila

using namespace gorila;

extern "C" {

size_t gorila_gated_scan_workspace_bytes(int32_t batch, int32_t length, int32_t channels, int32_t backward) {
    if (batch < 0 || length < 0 || channels < 1) return 0;
    const Plan p(length, channels, backward != 0);
    return p.total ? WS_FIXED_BYTES + p.total : 0;
}

int gorila_gated_scan(const gorila_gated_scan_args* args, void* y, float* state_out, float* marks, gorila_ctx* ctx) {
    GatedView v;
    CtxView c;
    bool vec;
    int rc = ctx_view(ctx, 0, c);
    if (rc || (rc = gated_view(args, false, v, vec))) return rc;
    if (v.B == 0 || (v.T == 0 && !state_out)) return GORILA_OK;
    const int e = dtype_bytes(args->dtype);
    if ((v.T > 0 && !y) || !at_element(y, e) || !at_element(state_out, 4) || !at_element(marks, 4)) return GORILA_EINVAL;
    const Cut k(v.B, v.T, v.C);
    const Plan p(v.T, v.C, false);
    const double blocks = (double)v.B * k.nseg * k.tiles;
    if (!launch_fits(blocks, BLOCK)) return GORILA_EUNSUPPORTED;
    if ((rc = ctx_view(ctx, k.nseg > 1 ? p.total : 0, c))) return rc;
    vec = vec && at_four(y, e) && at_four(state_out, 4) && at_four(marks, 4);
    v.tiles = k.tiles, v.nseg = k.nseg, v.seg = k.seg;
    v.y = y, v.state_out = state_out, v.marks = marks;
    if (k.nseg > 1) v.seg_a = (float*)c.ws, v.seg_h = (float*)(c.ws + p.maps), v.state_copy = (float*)(c.ws + 2 * p.maps);
    by_rows(args->dtype, vec, [&](auto t, auto al) {
        using T = decltype(t);
        constexpr bool VEC = decltype(al)::value;
        if (k.nseg > 1) gated_kernel<T, VEC, true><<<(unsigned)blocks, BLOCK, 0, c.stream>>>(v);
        gated_kernel<T, VEC, false><<<(unsigned)blocks, BLOCK, 0, c.stream>>>(v);
    });
    return launched();
}

int gorila_gated_scan_backward(const gorila_gated_scan_args* args, const float* marks, const void* dy, int64_t dy_batch_stride,
                               int64_t dy_step_stride, const float* dstate_out, void* dx, void* dgate_a, void* dgate_x, float* da_log,
                               float* dstate, gorila_ctx* ctx) {
    GatedView v;
    CtxView c;
    bool vec;
    int rc = ctx_view(ctx, 0, c);
    if (rc || (rc = gated_view(args, false, v, vec))) return rc;
    const int e = dtype_bytes(args->dtype);
    if (!da_log) return GORILA_EINVAL;
    if (v.B > 0 && v.T > 0 && (!marks || !dy || !dx || !dgate_a || !dgate_x)) return GORILA_EINVAL;
    for (const void* p : {dy, (const void*)dx, (const void*)dgate_a, (const void*)dgate_x})
        if (!at_element(p, e)) return GORILA_EINVAL;
    for (const float* p : {marks, dstate_out, (const float*)da_log, (const float*)dstate})
        if (!at_element(p, 4)) return GORILA_EINVAL;
    const Cut k(v.B, v.T, v.C);
    const Plan p(v.T, v.C, true);
    const double all = (double)v.B * k.nseg * k.tiles;
    if (!launch_fits(all, BLOCK)) return GORILA_EUNSUPPORTED;
    if ((rc = ctx_view(ctx, p.total, c))) return rc;
    vec = vec && !((dy_batch_stride | dy_step_stride) & 3) && at_four(dy, e) && at_four(dx, e) && at_four(dgate_a, e) && at_four(dgate_x, e) &&
          at_four(marks, 4) && at_four(dstate_out, 4) && at_four(dstate, 4);
    v.tiles = k.tiles, v.nseg = k.nseg, v.seg = k.seg;
    const int64_t items = (int64_t)v.B * k.nseg;
    v.items = (int)(items < Plan::walks(k.tiles) ? items : Plan::walks(k.tiles));
    v.dy = {dy, dy_batch_stride, dy_step_stride};
    v.marks_in = marks, v.dstate_out = dstate_out, v.dx = dx, v.dga = dgate_a, v.dgx = dgate_x, v.dstate = dstate;
    v.seg_a = (float*)c.ws, v.seg_h = (float*)(c.ws + p.maps), v.parts = (float*)(c.ws + 2 * p.maps + p.states);
    if (items > 0)
        by_rows(args->dtype, vec, [&](auto t, auto al) {
            using T = decltype(t);
            constexpr bool VEC = decltype(al)::value;
            if (k.nseg > 1) gated_back_kernel<T, VEC><<<(unsigned)all, BLOCK, 0, c.stream>>>(v);
            gated_backward_kernel<T, VEC><<<(unsigned)(v.items * k.tiles), BLOCK, 0, c.stream>>>(v);
        });
    launch_sum_parts(v.parts, v.items, v.C, v.C, 1, da_log, nullptr, c.stream);
    return launched();
}

int gorila_gated_scan_step(const gorila_gated_scan_args* args, float* state_pool, int64_t slots, const int32_t* slot, void* y,
                           gorila_ctx* ctx) {
    GatedView v;
    CtxView c;
    bool vec;
    int rc = ctx_view(ctx, 0, c);
    if (rc || (rc = gated_view(args, true, v, vec))) return rc;
    if (v.T != 1 || slots < 0) return GORILA_EINVAL;
    if (v.B == 0) return GORILA_OK;
    const int e = dtype_bytes(args->dtype);
    if (!state_pool || !y || !at_element(state_pool, 4) || !at_element(y, e) || !at_element(slot, 4)) return GORILA_EINVAL;
    if (slot ? !c.err : slots < v.B) return slot ? GORILA_EWORKSPACE : GORILA_EINVAL;
    vec = vec && at_four(state_pool, 4) && at_four(y, e);
    v.y = y;
    const int64_t blocks = ((int64_t)v.B * ((v.C + 3) / 4) + 255) / 256;
    if (!launch_fits((double)blocks, 256)) return GORILA_EUNSUPPORTED;
    by_rows(args->dtype, vec, [&](auto t, auto al) {
        gated_step_kernel<decltype(t), decltype(al)::value><<<(unsigned)blocks, 256, 0, c.stream>>>(v, state_pool, slots, slot, c.err);
    });
    return launched();
}

}  // extern "C"
