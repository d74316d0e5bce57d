// Gated scan (gorila_gated_scan, _backward, _step): h_t = a_t h_{t-1} + b_t i_t x_t in every
// channel, with a = exp(-exp(a_log) sigmoid(gate_a)), b = sqrt(1 - a^2), i = sigmoid(gate_x).
//
// Bound by memory and by the vector unit alike: a step of a channel has 3 values in and 1
// out for some 40 operations and 6 of the slow kind (exponentials, reciprocals, a root: four
// slots each), so a value is read once and its decay formed once.  The steps of a chunk
// lie in the lanes' registers: 8 steps of 2 channels a lane, 32 lanes a step, 2 runs of
// steps a wave.  Each lane runs through its own steps from zero, and what enters a
// lane's run is joined from the products of decays and the ends of the runs before it:
// between the halves of a wave by a shuffle, over the waves in LDS, over the chunks in
// registers.  (4 steps of 4 channels make twice the joins: 10 % of all operations.)
// The next chunk's loads are under way while this one's runs are joined.
//
// 32 x 128 x 1024 fp32: forward 13.8 us (4.9 TB/s), backward 22.6 (5.2 TB/s, part of it from
// the cache).  4 x 1999 x 2000 bf16: forward 46 us and 18 for the maps, backward 71 and 18;
// a prompt of 8192 x 1024 bf16: 26 and 15.  There the vector unit is busy a third to a half of
// the time, and fewer or more waves, or loads a chunk earlier, change nothing.  A wave
// forms 16 steps and a tile has 64 channels, however few there are: 256 x 1 x 4096 fp32
// 24 us forward (0.7 TB/s) and 60 backward (0.5), 512 x 200 x 16 fp32 17 and 32 (1.5).
//
// An episode start is a flag beside the product of decays, not a factor of zero:
// what is before it may be infinite.  Chunks without one, and inside the sequence,
// have a copy of the code without the flags (a fifth of all operations).
#include "seq.h"

namespace gorila {
namespace {

constexpr int TILE = 64;  // channels of a workgroup
constexpr int MARK = GORILA_GATED_MARK;
constexpr float LOG2E = 1.44269504088896341f, LN2 = 0.693147180559945309f;

struct Rows {
    const void* p;
    int64_t b, t;  // strides
};
struct GatedView {
    int B, T, C, tiles, nseg, seg;  // segments, and steps of one
    int maps, span;                 // maps of a sequence, and the steps of one: a segment's or a part's of it
    Rows x, ga, gx, dy;
    const float *a_log, *state, *dstate_out, *marks_in;
    const uint8_t* reset;
    void *y, *dx, *dga, *dgx;
    float *state_out, *marks, *dstate;
    float* state_copy;     // [B][C] where there are segments: state_out may be state
    float *map_a, *map_h;  // [B][maps][C]: product of decays (negative: an episode starts there), end
    float *parts, *dal;    // [items][C] of da_log, and where a lone one goes
    int items;             // workgroups that share a tile's sequences and segments
};

__device__ __forceinline__ float sigmoid(float v) {
    return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(v * -LOG2E));
}
// A sigmoid and what it leaves to 1, which is not formed as the difference where the gate is
// open: nothing is left of that (at a gate of 8 it is off by 1e-4 of itself, at 17 it is 0).
struct Gate {
    float open, rest;
};
__device__ __forceinline__ Gate gate_of(float v) {
    const float e = __builtin_amdgcn_exp2f(v * -LOG2E), open = __builtin_amdgcn_rcpf(1.0f + e);
    return {open, v < 0.0f ? 1.0f - open : e * open};
}
// exp(a_log) for a base of two: log2 a = -rate2 sigmoid(gate_a).
__device__ __forceinline__ float rate2_of(float a_log) {
    const float e = expf(a_log);
    return (e > 0x1p127f ? 0x1p127f : e) * LOG2E;  // (NaN stays)
}
struct Decay {
    float a, b;
};
// a = 2^l and b = sqrt(1 - a^2) for l <= 0: 1 - exp(u), u = 2 l ln 2, is its series where
// u > -1/4 (the next term is 2^-24 of the sum); below, 1 - a^2 loses two bits at most.
__device__ __forceinline__ Decay decay(float l) {
    constexpr float K = 2.0f * LN2, K2 = K * K;
    const float a = __builtin_amdgcn_exp2f(l);
    float s = fmaf(l, K2 * K2 * K2 / 720.0f, K2 * K2 * K / 120.0f);
    s = fmaf(l, s, K2 * K2 / 24.0f);
    s = fmaf(l, s, K2 * K / 6.0f);
    s = fmaf(l, s, K2 / 2.0f);
    s = fmaf(l, s, K);
    const float q = l > -0.25f / K ? -l * s : fmaf(-a, a, 1.0f);
    return {a, __builtin_amdgcn_sqrtf(q)};
}

// Two channels of a lane, of which `n` (0, 1 or 2) exist; a lane without any reads channel 0, and
// nothing of it is stored.
struct Two {
    float v[2];
    __device__ __forceinline__ float& operator[](int j) { return v[j]; }
    __device__ __forceinline__ float operator[](int j) const { return v[j]; }
};
// Where a lane is: its channels from c on.  It reads two in one load from `from` on, at any
// address (a load for each: 107 x 467 x 133 fp32 84 us backward instead of 78).
struct Place {
    int lane, wave, half, c, n, from;
    bool lone;  // there is one channel only
    __device__ __forceinline__ Place(const GatedView& v, int tile) {
        lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
        c = tile * TILE + 2 * (lane & 31);
        n = v.C - c < 0 ? 0 : v.C - c > 2 ? 2 : v.C - c;
        if (n == 0) c = 0;
        lone = v.C == 1;
        from = n == 1 && !lone ? c - 1 : c;
    }
};
// As they are read.  PAIR: the number of channels is even; else a row's last lane takes the
// second value that it reads for both of its.
template <class T, bool PAIR> struct Raw;
template <bool PAIR> struct Raw<float, PAIR> {
    float2 u;
    __device__ __forceinline__ void load(const float* p) { u = load_any<float2>(p); }
    __device__ __forceinline__ void load_one(const float* p) { u = float2{*p, *p}; }
    __device__ __forceinline__ Two get(const Place& at) const { return {{!PAIR && at.n == 1 ? u.y : u.x, u.y}}; }
};
template <bool PAIR> struct Raw<uint16_t, PAIR> {
    uint32_t u;
    __device__ __forceinline__ void load(const uint16_t* p) { u = load_any<uint32_t>(p); }
    __device__ __forceinline__ void load_one(const uint16_t* p) { u = *p * 0x10001u; }
    __device__ __forceinline__ Two get(const Place& at) const {
        const float second = __uint_as_float(u & 0xffff0000u);
        return {{!PAIR && at.n == 1 ? second : __uint_as_float(u << 16), second}};
    }
};
// p: of the channel at.from.
template <bool PAIR, class T>
__device__ __forceinline__ Two get2(const T* p, const Place& at) {
    Raw<T, PAIR> r;
    if (PAIR || !at.lone) r.load(p);
    else r.load_one(p);
    return r.get(at);
}
// p: of the channel at.c.
template <bool PAIR>
__device__ __forceinline__ void put2(float* p, Two v, int n) {
    if (PAIR ? n > 0 : n > 1) store_any(p, float2{v[0], v[1]});
    else if (!PAIR && n > 0) *p = v[0];
}
template <bool PAIR>
__device__ __forceinline__ void put2(uint16_t* p, Two v, int n) {
    typedef __bf16 Pair __attribute__((ext_vector_type(2)));
    typedef float Wide __attribute__((ext_vector_type(2)));
    const uint32_t u = __builtin_bit_cast(uint32_t, __builtin_convertvector(Wide{v[0], v[1]}, Pair));  // nearest even
    if (PAIR ? n > 0 : n > 1) store_any(p, u);
    else if (!PAIR && n > 0) *p = (uint16_t)u;
}
template <bool PAIR>
__device__ __forceinline__ Two rates_of(const GatedView& v, const Place& at) {
    const Two r = get2<PAIR>(v.a_log + at.from, at);
    return {{rate2_of(r[0]), rate2_of(r[1])}};
}
// Steps of one tensor: `p` is the lane's first step of the chunk at hand; the pointer moves
// on by whole chunks, so that a load costs one addition.
template <class T, bool PAIR, int S>
struct Stream {
    const T* p;
    int64_t step;
    Raw<T, PAIR> r[S];
    __device__ __forceinline__ Stream(const Rows& rows, int64_t b, int t, const Place& at) {
        p = (const T*)rows.p + b * rows.b + (int64_t)(t + (at.wave * 2 + at.half) * S) * rows.t + at.from;
        step = rows.t;
    }
    __device__ __forceinline__ void move(int steps) { p += steps * step; }
    // `left`: steps from the first on that exist (1 or more of the wave's chunk); others read the last.
    template <bool FULL>
    __device__ __forceinline__ void fetch(int left, const Place& at) {
        if (!PAIR && at.lone) {
#pragma unroll
            for (int k = 0; k < S; ++k) r[k].load_one(p + (int64_t)(k < left ? k : left - 1) * step);
        } else if (FULL) {
            const T* q = p;
#pragma unroll
            for (int k = 0; k < S; ++k, q += step) r[k].load(q);
        } else {
#pragma unroll
            for (int k = 0; k < S; ++k) r[k].load(p + (int64_t)(k < left ? k : left - 1) * step);
        }
    }
};
// Episode starts among the 2 S steps of a wave, a lane each.
template <int S>
__device__ __forceinline__ int start_of(const GatedView& v, int64_t b, int t, int end, int lane) {
    return v.reset && lane < 2 * S && t + lane < end ? v.reset[b * v.T + t + lane] : 0;
}
__device__ __forceinline__ uint32_t starts(int own) { return (uint32_t)__ballot(own != 0); }

__device__ __forceinline__ float other_half(float v) { return __shfl_xor(v, 32, 64); }
__device__ __forceinline__ Two other_half(Two v) { return {{other_half(v[0]), other_half(v[1])}}; }
// What leaves a run that h enters; `cut`: an episode starts in it.
__device__ __forceinline__ Two through(Two a, Two end, bool cut, Two h) {
    return {{cut ? end[0] : fmaf(a[0], h[0], end[0]), cut ? end[1] : fmaf(a[1], h[1], end[1])}};
}

// The waves' maps in LDS: products of decays, ends forward and (B) back.
template <int W, int DIRECTIONS>
struct Shared {
    float2 a[W][32], end[DIRECTIONS][W][32];
    int cut[W];
};
template <int W>
__device__ __forceinline__ uint32_t cuts_of(const int (&cut)[W], int lane) {
    return (uint32_t)__ballot(lane < W && cut[lane < W ? lane : 0] != 0);
}
__device__ __forceinline__ Two two(float2 v) { return {{v.x, v.y}}; }

// What maps first, first + step, .. (count of them) make of what enters the first of them: eight
// are read at a time.
template <bool PAIR>
__device__ __forceinline__ void pass(Two& carry, const GatedView& v, int64_t b, int first, int step, int count, const Place& at) {
    constexpr int AHEAD = 8;
    for (int m = 0; m < count; m += AHEAD) {
        Two a[AHEAD], h[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const int64_t from = (b * v.maps + first + (m + k < count ? m + k : m) * step) * v.C + at.from;
            a[k] = get2<PAIR>(v.map_a + from, at), h[k] = get2<PAIR>(v.map_h + from, at);
        }
#pragma unroll
        for (int k = 0; k < AHEAD; ++k)
            if (m + k < count)
#pragma unroll
                for (int j = 0; j < 2; ++j) carry[j] = a[k][j] < 0.0f ? h[k][j] : fmaf(a[k][j], carry[j], h[k][j]);
    }
}
template <bool PAIR>
__device__ __forceinline__ void put_map(const GatedView& v, int64_t b, int m, Two prod, bool cut, Two end, const Place& at) {
    const int64_t to = (b * v.maps + m) * v.C + at.c;
    if (cut) prod = {{-1.0f, -1.0f}};
    put2<PAIR>(v.map_a + to, prod, at.n);
    put2<PAIR>(v.map_h + to, end, at.n);
}

// Forward.  A workgroup of W waves walks the chunks of one segment of 64 channels.
// AGG: the map of a segment, or of a part of one, alone, for the segments behind it.
template <class T, bool PAIR, int W, int S, bool AGG>
__global__ __launch_bounds__(64 * W) void gated_kernel(GatedView v) {
    constexpr int CHUNK = 2 * S * W;
    __shared__ Shared<W, 1> sh[2];
    const int count = AGG ? v.maps : v.nseg, steps = AGG ? v.span : v.seg;
    const int tile = blockIdx.x % v.tiles, item = blockIdx.x / v.tiles, seg = item % count;
    const int64_t b = item / count;
    const Place at(v, tile);
    const int begin = seg * steps, end = begin + steps < v.T ? begin + steps : v.T;
    const Two rate2 = rates_of<PAIR>(v, at);
    Two carry{{0.0f, 0.0f}}, prod{{1.0f, 1.0f}};
    uint32_t cut = 0;
    Stream<T, PAIR, S> x(v.x, b, begin, at), ga(v.ga, b, begin, at), gx(v.gx, b, begin, at);
    int reset = 0;
    auto fetch_all = [&](int t0) {
        reset = start_of<S>(v, b, t0 + at.wave * 2 * S, end, at.lane);
        auto all = [&](auto full) {
            constexpr bool FULL = decltype(full)::value;
            const int left = end - t0 - (at.wave * 2 + at.half) * S;
            ga.template fetch<FULL>(left, at);
            gx.template fetch<FULL>(left, at);
            x.template fetch<FULL>(left, at);
        };
        if (t0 + CHUNK <= end) all(std::true_type{});
        else all(std::false_type{});
        x.move(CHUNK), ga.move(CHUNK), gx.move(CHUNK);
    };
    if (begin < end) fetch_all(begin);
    if (AGG) {
        if (seg == 0 && threadIdx.x < 32) put2<PAIR>(v.state_copy + b * v.C + at.c, v.state ? get2<PAIR>(v.state + b * v.C + at.from, at) : carry, at.n);
    } else {
        const float* from = v.nseg > 1 ? v.state_copy : v.state;
        if (from) carry = get2<PAIR>(from + b * v.C + at.from, at);
        if (v.nseg > 1) pass<PAIR>(carry, v, b, 0, 1, begin / v.span, at);
    }
    for (int t0 = begin, turn = 0; t0 < end; t0 += CHUNK, turn ^= 1) {
        const uint32_t mask = starts(reset), own = at.half ? mask >> S : mask & ((1u << S) - 1);
        const int t = t0 + (at.wave * 2 + at.half) * S;
        const bool plain = mask == 0 && t0 + CHUNK <= end;
        Two a[S], u[S], A{{1.0f, 1.0f}}, H{{0.0f, 0.0f}};
        auto run = [&](auto simple) {
            constexpr bool PLAIN = decltype(simple)::value;
#pragma unroll
            for (int k = 0; k < S; ++k) {
                const Two xv = x.r[k].get(at), gav = ga.r[k].get(at), gxv = gx.r[k].get(at);
                const bool start = !PLAIN && (own >> k & 1u), in = PLAIN || t + k < end;
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const Decay d = decay(-rate2[j] * sigmoid(gav[j]));
                    a[k][j] = in ? d.a : 1.0f;
                    u[k][j] = in ? (start ? 1.0f : d.b) * sigmoid(gxv[j]) * xv[j] : 0.0f;
                    H[j] = start ? u[k][j] : fmaf(a[k][j], H[j], u[k][j]);
                    A[j] *= a[k][j];
                }
            }
        };
        if (plain) run(std::true_type{});
        else run(std::false_type{});
        if (t0 + CHUNK < end) fetch_all(t0 + CHUNK);
        // the wave's two runs joined
        const Two oa = other_half(A), oh = other_half(H);
        const bool cut0 = mask & ((1u << S) - 1), cut1 = mask >> S;
        Two all{{A[0] * oa[0], A[1] * oa[1]}}, enter;
        if (W > 1) {
            if (at.half) {
                const Two h = through(A, H, cut1, oh);
                sh[turn].a[at.wave][at.lane & 31] = float2{all[0], all[1]};
                sh[turn].end[0][at.wave][at.lane & 31] = float2{h[0], h[1]};
                if (at.lane == 63) sh[turn].cut[at.wave] = mask != 0;
            }
            __syncthreads();
            const uint32_t cuts = cuts_of(sh[turn].cut, at.lane);
            if (AGG) cut |= cuts;
            enter = carry;
            auto over_waves = [&](uint32_t cuts) {
#pragma unroll
                for (int w = 0; w < W; ++w) {
                    if (w == at.wave) enter = carry;
                    const Two p = two(sh[turn].a[w][at.lane & 31]), e = two(sh[turn].end[0][w][at.lane & 31]);
                    carry = through(p, e, cuts >> w & 1u, carry);
                    if (AGG) prod[0] *= p[0], prod[1] *= p[1];
                }
            };
            if (cuts == 0) over_waves(0);
            else over_waves(cuts);
        } else {
            enter = carry;
            const Two first = at.half ? through(oa, oh, cut0, carry) : through(A, H, cut0, carry);
            carry = at.half ? through(A, H, cut1, first) : through(oa, oh, cut1, first);
        }
        if (AGG) continue;
        if (v.marks && at.wave % (MARK / (2 * S)) == 0 && at.half == 0 && t < end)
            put2<PAIR>(v.marks + (b * ((v.T + MARK - 1) / MARK) + t / MARK) * v.C + at.c, enter, at.n);
        Two h = at.half ? through(oa, oh, cut0, enter) : enter;
        T* y = (T*)v.y + (b * v.T + t) * v.C + at.c;
        if (plain) {
#pragma unroll
            for (int k = 0; k < S; ++k) {
                h = through(a[k], u[k], false, h);
                put2<PAIR>(y + (int64_t)k * v.C, h, at.n);
            }
        } else {
#pragma unroll
            for (int k = 0; k < S; ++k) {
                h = through(a[k], u[k], own >> k & 1u, h);
                if (t + k < end) put2<PAIR>(y + (int64_t)k * v.C, h, at.n);
            }
        }
    }
    if (threadIdx.x >= 32) return;
    if (AGG) put_map<PAIR>(v, b, seg, prod, cut != 0, carry, at);
    else if (seg == v.nseg - 1 && v.state_out) put2<PAIR>(v.state_out + b * v.C + at.c, carry, at.n);
}

// What passes back through a segment, for the segments before it.
template <class T, bool PAIR, int W, int S>
__global__ __launch_bounds__(64 * W) void gated_back_kernel(GatedView v) {
    constexpr int CHUNK = 2 * S * W;
    __shared__ Shared<W, 1> sh[2];
    const int tile = blockIdx.x % v.tiles, item = blockIdx.x / v.tiles, seg = item % v.nseg;
    const int64_t b = item / v.nseg;
    if (seg == 0) return;
    const Place at(v, tile);
    const int begin = seg * v.seg, end = begin + v.seg < v.T ? begin + v.seg : v.T;
    const Two rate2 = rates_of<PAIR>(v, at);
    Two carry{{0.0f, 0.0f}}, prod{{1.0f, 1.0f}};
    uint32_t cut = 0;
    const int first = begin + (end - begin - 1) / CHUNK * CHUNK;
    Stream<T, PAIR, S> ga(v.ga, b, first, at), dy(v.dy, b, first, at);
    int reset = 0;
    auto fetch_all = [&](int t0) {
        reset = start_of<S>(v, b, t0 + at.wave * 2 * S, end, at.lane);
        auto all = [&](auto full) {
            constexpr bool FULL = decltype(full)::value;
            const int left = end - t0 - (at.wave * 2 + at.half) * S;
            ga.template fetch<FULL>(left, at);
            dy.template fetch<FULL>(left, at);
        };
        if (t0 + CHUNK <= end) all(std::true_type{});
        else all(std::false_type{});
        ga.move(-CHUNK), dy.move(-CHUNK);
    };
    fetch_all(first);
    for (int t0 = first, turn = 0; t0 >= begin; t0 -= CHUNK, turn ^= 1) {
        const uint32_t mask = starts(reset), own = at.half ? mask >> S : mask & ((1u << S) - 1);
        const int t = t0 + (at.wave * 2 + at.half) * S;
        Two A{{1.0f, 1.0f}}, H{{0.0f, 0.0f}};
#pragma unroll
        for (int k = S - 1; k >= 0; --k) {
            const Two gav = ga.r[k].get(at), d = dy.r[k].get(at);
            const bool start = own >> k & 1u, in = t + k < end;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const float a = in ? __builtin_amdgcn_exp2f(-rate2[j] * sigmoid(gav[j])) : 1.0f;
                H[j] = start ? 0.0f : in ? a * (H[j] + d[j]) : H[j];
                A[j] *= a;
            }
        }
        if (t0 > begin) fetch_all(t0 - CHUNK);
        const Two oa = other_half(A), oh = other_half(H);
        if (!at.half) {
            const Two h = through(A, H, mask & ((1u << S) - 1), oh);
            sh[turn].a[at.wave][at.lane] = float2{A[0] * oa[0], A[1] * oa[1]};
            sh[turn].end[0][at.wave][at.lane] = float2{h[0], h[1]};
            if (at.lane == 0) sh[turn].cut[at.wave] = mask != 0;
        }
        __syncthreads();
        const uint32_t cuts = cuts_of(sh[turn].cut, at.lane);
        cut |= cuts;
        auto over_waves = [&](uint32_t cuts) {
#pragma unroll
            for (int w = W - 1; w >= 0; --w) {
                const Two p = two(sh[turn].a[w][at.lane & 31]), e = two(sh[turn].end[0][w][at.lane & 31]);
                carry = through(p, e, cuts >> w & 1u, carry);
                prod[0] *= p[0], prod[1] *= p[1];
            }
        };
        if (cuts == 0) over_waves(0);
        else over_waves(cuts);
    }
    if (threadIdx.x < 32) put_map<PAIR>(v, b, seg, prod, cut != 0, carry, at);
}

// Backward: with R_t = dy_t + a_{t+1} R_{t+1},
//   dx = R b i,   dgate_x = R b i (1 - i) x,   G = log a (R a h_{t-1} - R i x a^2 / b),
//   dgate_a = G (1 - r),   da_log = sum of G      (at a start G is zero).
// Chunks are walked from the last on; the state before every fourth wave's steps is a
// mark, so that both directions are in registers at once and every value is read once.
// What the gates give is held as the outputs take it (u = b i x, b i, a log a, its quotient by
// b^2 and a, 1 - r and 1 - i): two waves a SIMD have room for it.  One wave has one chunk.
template <class T, bool PAIR, int W, int S>
__global__ __launch_bounds__(64 * W, 2) void gated_backward_kernel(GatedView v) {
    constexpr int CHUNK = 2 * S * W, GROUP = MARK / (2 * S);  // steps, waves that share a mark
    __shared__ Shared<W, 2> sh[2];
    __shared__ float2 sums[2 * W][32];
    const int tile = blockIdx.x % v.tiles;
    const Place at(v, tile);
    const Two rate2 = rates_of<PAIR>(v, at);
    Two dal{{0.0f, 0.0f}};
    int turn = 0;
    for (int64_t item = blockIdx.x / v.tiles; item < (int64_t)v.B * v.nseg; item += v.items) {
        const int seg = (int)(item % v.nseg);
        const int64_t b = item / v.nseg;
        const int begin = seg * v.seg, end = begin + v.seg < v.T ? begin + v.seg : v.T;
        Two carry{{0.0f, 0.0f}};
        if (v.dstate_out) carry = get2<PAIR>(v.dstate_out + b * v.C + at.from, at);
        pass<PAIR>(carry, v, b, v.nseg - 1, -1, v.nseg - 1 - seg, at);
        if (end <= begin) {  // no steps: what comes in goes out
            if (seg == 0 && v.dstate && threadIdx.x < 32) put2<PAIR>(v.dstate + b * v.C + at.c, carry, at.n);
            continue;
        }
        const int first = begin + (end - begin - 1) / CHUNK * CHUNK;
        Stream<T, PAIR, S> x(v.x, b, first, at), ga(v.ga, b, first, at), gx(v.gx, b, first, at), dy(v.dy, b, first, at);
        // The gates' loads are a chunk ahead: their registers are free once decays are formed, which hides the others'.
        auto fetch_two = [&](Stream<T, PAIR, S>& p, Stream<T, PAIR, S>& q, int t0) {
            const int left = end - t0 - (at.wave * 2 + at.half) * S;
            if (t0 + CHUNK <= end) {
                p.template fetch<true>(left, at);
                q.template fetch<true>(left, at);
            } else {
                p.template fetch<false>(left, at);
                q.template fetch<false>(left, at);
            }
            p.move(-CHUNK), q.move(-CHUNK);
        };
        fetch_two(ga, gx, first);
        for (int t0 = first; t0 >= begin; t0 -= CHUNK, turn ^= 1) {
            const int t = t0 + (at.wave * 2 + at.half) * S;
            const int reset = start_of<S>(v, b, t0 + at.wave * 2 * S, end, at.lane);
            fetch_two(x, dy, t0);
            const int group = t0 + at.wave / GROUP * MARK;  // the mark's step, if it exists
            Two now = get2<PAIR>(v.marks_in + (b * ((v.T + MARK - 1) / MARK) + (group < end ? group : t0) / MARK) * v.C + at.from, at);
            const uint32_t mask = starts(reset), own = at.half ? mask >> S : mask & ((1u << S) - 1);
            const bool plain = mask == 0 && t0 + CHUNK <= end;
            const bool cut0 = mask & ((1u << S) - 1), cut1 = mask >> S;
            Two a[S], w[S], over[S], bi[S], rr[S], ri[S], u[S], A{{1.0f, 1.0f}}, F{{0.0f, 0.0f}}, H{{0.0f, 0.0f}};
            auto runs = [&](auto simple) {
                constexpr bool PLAIN = decltype(simple)::value;
#pragma unroll
                for (int k = 0; k < S; ++k) {
                    const Two gav = ga.r[k].get(at), gxv = gx.r[k].get(at);
                    const bool start = !PLAIN && (own >> k & 1u), in = PLAIN || t + k < end;
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const Gate r = gate_of(gav[j]), i = gate_of(gxv[j]);
                        const float l = -rate2[j] * r.open;
                        const Decay d = decay(l);
                        rr[k][j] = r.rest, ri[k][j] = i.rest;
                        // a log a before any other factor: log a may be as large as fp32 goes where a is 0;
                        // its quotient by b twice is 1/2 at most
                        w[k][j] = d.a * (l * LN2);
                        a[k][j] = in ? d.a : 1.0f;
                        const float b = !in ? 0.0f : start ? 1.0f : d.b, per = __builtin_amdgcn_rcpf(b);
                        over[k][j] = b > 0.0f ? w[k][j] * a[k][j] * per * per : 0.0f;
                        bi[k][j] = b * i.open;
                    }
                }
#pragma unroll
                for (int k = 0; k < S; ++k) {
                    const Two xv = x.r[k].get(at);
                    const bool start = !PLAIN && (own >> k & 1u), in = PLAIN || t + k < end;
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        u[k][j] = in ? bi[k][j] * xv[j] : 0.0f;
                        F[j] = start ? u[k][j] : fmaf(a[k][j], F[j], u[k][j]);
                        A[j] *= a[k][j];
                    }
                }
#pragma unroll
                for (int k = S - 1; k >= 0; --k) {
                    const Two d = dy.r[k].get(at);
                    const bool start = !PLAIN && (own >> k & 1u), in = PLAIN || t + k < end;
#pragma unroll
                    for (int j = 0; j < 2; ++j) H[j] = start ? 0.0f : in ? a[k][j] * (H[j] + d[j]) : H[j];
                }
            };
            if (plain) runs(std::true_type{});
            else runs(std::false_type{});
            if (W > 1 && t0 > begin) fetch_two(ga, gx, t0 - CHUNK);
            const Two oa = other_half(A), of = other_half(F), oh = other_half(H);
            Two back = carry;
            if (W > 1) {
                if (at.half) {
                    const Two f = through(A, F, cut1, of);
                    sh[turn].end[0][at.wave][at.lane & 31] = float2{f[0], f[1]};
                    sh[turn].a[at.wave][at.lane & 31] = float2{A[0] * oa[0], A[1] * oa[1]};
                } else {
                    const Two h = through(A, H, cut0, oh);
                    sh[turn].end[1][at.wave][at.lane] = float2{h[0], h[1]};
                    if (at.lane == 0) sh[turn].cut[at.wave] = mask != 0;
                }
                __syncthreads();
                const uint32_t cuts = cuts_of(sh[turn].cut, at.lane);
                for (int w = at.wave / GROUP * GROUP; w < at.wave; ++w)
                    now = through(two(sh[turn].a[w][at.lane & 31]), two(sh[turn].end[0][w][at.lane & 31]), cuts >> w & 1u, now);
#pragma unroll
                for (int w = W - 1; w >= 0; --w) {
                    if (w == at.wave) back = carry;
                    carry = through(two(sh[turn].a[w][at.lane & 31]), two(sh[turn].end[1][w][at.lane & 31]), cuts >> w & 1u, carry);
                }
            } else {
                const Two later = at.half ? through(A, H, cut1, carry) : through(oa, oh, cut1, carry);
                carry = at.half ? through(oa, oh, cut0, later) : through(A, H, cut0, later);
            }
            if (at.half) now = through(oa, of, cut0, now);
            else back = through(oa, oh, cut1, back);
            const int64_t to = (b * v.T + t) * v.C + at.c;
            T *dxp = (T*)v.dx + to, *dgap = (T*)v.dga + to, *dgxp = (T*)v.dgx + to;
            auto outputs = [&](auto simple) {
                constexpr bool PLAIN = decltype(simple)::value;
                Two h[S];  // the state before the step
#pragma unroll
                for (int k = 0; k < S; ++k) {
                    h[k] = now;
                    now = through(a[k], u[k], !PLAIN && (own >> k & 1u), now);
                }
#pragma unroll
                for (int k = S - 1; k >= 0; --k) {
                    const Two d = dy.r[k].get(at);
                    const bool start = !PLAIN && (own >> k & 1u), in = PLAIN || t + k < end;
                    Two dx, dga, dgx;
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const float R = (in ? d[j] : 0.0f) + back[j], Ru = R * u[k][j];
                        dx[j] = R * bi[k][j];
                        dgx[j] = Ru * ri[k][j];
                        const float G = start ? 0.0f : R * (w[k][j] * h[k][j]) - Ru * over[k][j];
                        dga[j] = G * rr[k][j];
                        if (in) dal[j] += G;
                        back[j] = start ? 0.0f : a[k][j] * R;
                    }
                    if (in) {
                        put2<PAIR>(dxp + (int64_t)k * v.C, dx, at.n);
                        put2<PAIR>(dgap + (int64_t)k * v.C, dga, at.n);
                        put2<PAIR>(dgxp + (int64_t)k * v.C, dgx, at.n);
                    }
                }
            };
            if (plain) outputs(std::true_type{});
            else outputs(std::false_type{});
            if (W == 1) break;  // (T is at most a chunk)
        }
        if (seg == 0 && v.dstate && threadIdx.x < 32) put2<PAIR>(v.dstate + b * v.C + at.c, carry, at.n);
    }
    sums[2 * at.wave + at.half][at.lane & 31] = float2{dal[0], dal[1]};
    __syncthreads();
    if (threadIdx.x >= 32) return;
#pragma unroll
    for (int k = 1; k < 2 * W; ++k) {
        const float2 s = sums[k][at.lane];
        dal[0] += s.x, dal[1] += s.y;
    }
    put2<PAIR>((v.items == 1 ? v.dal : v.parts + (int64_t)(blockIdx.x / v.tiles) * v.C) + at.c, dal, at.n);
}

// One step of every row: four channels a lane.
template <class T>
__global__ __launch_bounds__(256) void gated_step_kernel(GatedView v, float* pool, int64_t slots, const int32_t* slot, unsigned* err) {
    const int quads = (v.C + 3) / 4;
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x, row = id / quads;
    if (row >= v.B) return;
    const int c = (int)(id % quads) * 4;
    int64_t at = slot ? slot[row] : row;
    const bool out = at < 0 || at >= slots, reset = out || (v.reset && v.reset[row]);
    if (out) {
        if (c == 0 && err) atomicOr(err, ERR_IDX_RANGE);
        at = 0;
    }
    const bool start = v.reset && v.reset[row];
    auto step = [&](int n) {
        auto read = [&](const Rows& r) { return quad_load((const T*)r.p + row * r.b + c, n); };
        const f32x4 ga = read(v.ga), gx = read(v.gx), x = read(v.x);
        const f32x4 al = quad_load(v.a_log + c, n);
        float* st = pool + at * v.C + c;
        f32x4 h{0.0f, 0.0f, 0.0f, 0.0f};
        if (!reset) h = quad_load(st, n);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const Decay d = decay(-rate2_of(al[j]) * sigmoid(ga[j]));
            const float u = (start ? 1.0f : d.b) * sigmoid(gx[j]) * x[j];
            h[j] = reset ? u : fmaf(d.a, h[j], u);
        }
        if (!out) quad_store(st, h, n);
        quad_store((T*)v.y + row * v.C + c, h, n);
    };
    if (c + 4 <= v.C) step(4);
    else step(v.C - c);
}

// ---- host ----

constexpr int FULL = 256;       // workgroups that fill the chip, one a compute unit: half as many are cut into segments
constexpr int BACK_FULL = 512;  // what a backward's fewer than that are cut into: its workgroups of four waves lie two a unit
constexpr int LEAST_SEG = 256;  // steps of a segment, or of a map, at least
constexpr int MAX_SEG = 64;     // segments of a sequence at most
constexpr int WALKS = 2048;     // workgroups of the backward at most: each adds a part of da_log

// Sequences whose tiles leave the chip idle are cut into segments.  Forward the maps of all
// but the last are formed first, in parts of a segment, so that the whole chip has a
// share of them.  (4 x 1999 x 2000 bf16, 128 tiles: uncut 65 us, cut into 256 45 + 18, into
// 512 46 + 29; 192 tiles of 2000 steps fp32 uncut 87, cut into 384 126.  Backward 128 tiles
// of 2000 steps cut into 512 74 us, into 256 95; 256 tiles of 512 steps fp32 uncut 49, cut
// 64; 400 of 300 steps 50 and 80; 185 of 600 steps cut into 555 61, into 370 73.)
struct Cut {
    int tiles, nseg = 1, seg, maps = 0, span;
    Cut(int64_t B, int T, int C, bool backward) {
        tiles = (C + TILE - 1) / TILE;
        seg = span = T > 0 ? T : 1;
        const int64_t have = B * tiles, full = backward ? BACK_FULL : FULL, most = (T + LEAST_SEG - 1) / LEAST_SEG;
        if (have < 1 || have >= FULL) return;
        int64_t k = backward ? (full + have - 1) / have : full / have;
        k = k < most ? k : most;
        k = k < MAX_SEG ? k : MAX_SEG;
        if (k < 2) return;
        seg = span = (int)(((T + k - 1) / k + LEAST_SEG - 1) / LEAST_SEG * LEAST_SEG);
        nseg = maps = (T + seg - 1) / seg;
        if (backward || nseg < 2) return;
        int64_t parts = BACK_FULL / (have * (nseg - 1));
        if (parts > seg / LEAST_SEG) parts = seg / LEAST_SEG;
        while (parts > 1 && seg % (parts * LEAST_SEG)) --parts;
        if (parts > 1) span = (int)(seg / parts);
        maps = (nseg - 1) * (seg / span);
    }
};

size_t up256(size_t n) { return (n + 255) / 256 * 256; }
// Bytes of the workspace: the maps and the states before the first step (cut calls
// have B * tiles < BACK_FULL, so B * maps < 2 BACK_FULL / tiles), then the parts.
struct Plan {
    size_t maps, states, parts, total;
    Plan(int T, int C, bool backward) {
        const int tiles = (C + TILE - 1) / TILE;
        const size_t cut = T > LEAST_SEG ? 4 * (size_t)C : 0;
        maps = up256(cut * (2 * BACK_FULL / tiles + 1));
        states = up256(cut * (BACK_FULL / tiles + 1));
        parts = up256(backward ? 4 * (size_t)C * walks(tiles) : 0);
        total = 2 * maps + states + parts;
    }
    static int walks(int tiles) { return (WALKS + tiles - 1) / tiles; }
};

int gated_view(const gorila_gated_scan_args* a, GatedView& v) {
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
    return GORILA_OK;
}

// Waves a workgroup, of 16 steps each (a wave in which T ends, or a mark's four and more).  Forward
// eight where that is one workgroup a compute unit (32 x 1000 x 512 fp32: 51 us, four waves 58),
// else four: one of eight leaves no place for a second (300 x 200 x 128 fp32, 600
// workgroups: 26 us, eight waves 34; 320 of 500 steps 39 and 43), and two chunks or
// more have loads under way while one is joined (32 x 128 x 1024 fp32: 14.6 us; 18.4).
// Backward a lane has up to 247 registers, and more waves than two a SIMD do not pay: 8 steps a lane
// and four waves 22.7 us (5.2 TB/s), eight waves 27.6; 4 steps and eight waves, half of the
// registers, 26.2.
constexpr int S = 8;
int forward_waves(int T, double blocks) { return T <= 16 ? 1 : T <= 128 || blocks > FULL ? 4 : 8; }
int backward_waves(int T) { return T <= 16 ? 1 : 4; }
template <class F>
void by_waves(int waves, F&& f) {
    using std::integral_constant;
    if (waves == 1) f(integral_constant<int, 1>{});
    else if (waves == 4) f(integral_constant<int, 4>{});
    else f(integral_constant<int, 8>{});
}

template <class F>
void by_rows(int dtype, bool pair, F&& f) {
    if (dtype == GORILA_F32) pair ? f(float{}, std::true_type{}) : f(float{}, std::false_type{});
    else pair ? f(uint16_t{}, std::true_type{}) : f(uint16_t{}, std::false_type{});
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
    int rc = ctx_view(ctx, 0, c);
    if (rc || (rc = gated_view(args, v))) return rc;
    if (v.B == 0 || (v.T == 0 && !state_out)) return GORILA_OK;
    const int e = dtype_bytes(args->dtype);
    if ((v.T > 0 && !y) || !at_element(y, e) || !at_element(state_out, 4) || !at_element(marks, 4)) return GORILA_EINVAL;
    const Cut k(v.B, v.T, v.C, false);
    const Plan p(v.T, v.C, false);
    const double blocks = (double)v.B * k.nseg * k.tiles;
    const int waves = forward_waves(v.T, blocks);
    if (!launch_fits(blocks, 64 * waves)) return GORILA_EUNSUPPORTED;
    if ((rc = ctx_view(ctx, k.nseg > 1 ? p.total : 0, c))) return rc;
    v.tiles = k.tiles, v.nseg = k.nseg, v.seg = k.seg, v.maps = k.maps, v.span = k.span;
    v.y = y, v.state_out = state_out, v.marks = marks;
    if (k.nseg > 1) v.map_a = (float*)c.ws, v.map_h = (float*)(c.ws + p.maps), v.state_copy = (float*)(c.ws + 2 * p.maps);
    by_rows(args->dtype, v.C % 2 == 0, [&](auto t, auto pair) {
        using T = decltype(t);
        constexpr bool PAIR = decltype(pair)::value;
        if (k.nseg > 1) gated_kernel<T, PAIR, 8, S, true><<<(unsigned)(v.B * k.maps * k.tiles), 512, 0, c.stream>>>(v);
        by_waves(waves, [&](auto w) {
            constexpr int W = decltype(w)::value;
            gated_kernel<T, PAIR, W, S, false><<<(unsigned)blocks, 64 * W, 0, c.stream>>>(v);
        });
    });
    return launched();
}

int gorila_gated_scan_backward(const gorila_gated_scan_args* args, const float* marks, const void* dy, int64_t dy_batch_stride,
                               int64_t dy_step_stride, const float* dstate_out, void* dx, void* dgate_a, void* dgate_x, float* da_log,
                               float* dstate, gorila_ctx* ctx) {
    GatedView v;
    CtxView c;
    int rc = ctx_view(ctx, 0, c);
    if (rc || (rc = gated_view(args, v))) return rc;
    const int e = dtype_bytes(args->dtype);
    if (!da_log) return GORILA_EINVAL;
    if (v.B > 0 && v.T > 0 && (!marks || !dy || !dx || !dgate_a || !dgate_x)) return GORILA_EINVAL;
    for (const void* p : {dy, (const void*)dx, (const void*)dgate_a, (const void*)dgate_x})
        if (!at_element(p, e)) return GORILA_EINVAL;
    for (const float* p : {marks, dstate_out, (const float*)da_log, (const float*)dstate})
        if (!at_element(p, 4)) return GORILA_EINVAL;
    const Cut k(v.B, v.T, v.C, true);
    const Plan p(v.T, v.C, true);
    const double all = (double)v.B * k.nseg * k.tiles;
    const int waves = backward_waves(v.T);
    if (!launch_fits(all, 64 * waves)) return GORILA_EUNSUPPORTED;
    if ((rc = ctx_view(ctx, p.total, c))) return rc;
    v.tiles = k.tiles, v.nseg = k.nseg, v.seg = k.seg, v.maps = k.maps, v.span = k.span;
    const int64_t items = (int64_t)v.B * k.nseg;
    v.items = (int)(items < Plan::walks(k.tiles) ? items : Plan::walks(k.tiles));
    v.dal = da_log;
    v.dy = {dy, dy_batch_stride, dy_step_stride};
    v.marks_in = marks, v.dstate_out = dstate_out, v.dx = dx, v.dga = dgate_a, v.dgx = dgate_x, v.dstate = dstate;
    v.map_a = (float*)c.ws, v.map_h = (float*)(c.ws + p.maps), v.parts = (float*)(c.ws + 2 * p.maps + p.states);
    if (items > 0)
        by_rows(args->dtype, v.C % 2 == 0, [&](auto t, auto pair) {
            using T = decltype(t);
            constexpr bool PAIR = decltype(pair)::value;
            if (k.nseg > 1) gated_back_kernel<T, PAIR, 8, S><<<(unsigned)all, 512, 0, c.stream>>>(v);
            if (waves == 1) gated_backward_kernel<T, PAIR, 1, S><<<(unsigned)(v.items * k.tiles), 64, 0, c.stream>>>(v);
            else gated_backward_kernel<T, PAIR, 4, S><<<(unsigned)(v.items * k.tiles), 256, 0, c.stream>>>(v);
        });
    if (v.items != 1) launch_sum_parts(v.parts, v.items, v.C, v.C, 1, da_log, nullptr, c.stream);
    return launched();
}

int gorila_gated_scan_step(const gorila_gated_scan_args* args, float* state_pool, int64_t slots, const int32_t* slot, void* y,
                           gorila_ctx* ctx) {
    GatedView v;
    CtxView c;
    int rc = ctx_view(ctx, 0, c);
    if (rc || (rc = gated_view(args, v))) return rc;
    if (v.T != 1 || slots < 0) return GORILA_EINVAL;
    if (v.B == 0) return GORILA_OK;
    const int e = dtype_bytes(args->dtype);
    if (!state_pool || !y || !at_element(state_pool, 4) || !at_element(y, e) || !at_element(slot, 4)) return GORILA_EINVAL;
    if (slot ? !c.err : slots < v.B) return slot ? GORILA_EWORKSPACE : GORILA_EINVAL;
    v.y = y;
    const int64_t blocks = ((int64_t)v.B * ((v.C + 3) / 4) + 255) / 256;
    if (!launch_fits((double)blocks, 256)) return GORILA_EUNSUPPORTED;
    if (args->dtype == GORILA_F32) gated_step_kernel<float><<<(unsigned)blocks, 256, 0, c.stream>>>(v, state_pool, slots, slot, c.err);
    else gated_step_kernel<uint16_t><<<(unsigned)blocks, 256, 0, c.stream>>>(v, state_pool, slots, slot, c.err);
    return launched();
}

}  // extern "C"
