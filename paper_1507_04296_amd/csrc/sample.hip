// Actions sampled from values (gorila_sample_actions).
//
// Weights are whole numbers, 2^40 exp((value - most) / temperature) rounded: their sums
// are exact in 64 bits whatever the order (2^20 actions give at most 2^60), so that the
// filters' borders and the drawn action do not depend on how a row is cut.
//
// Rows of up to 64 actions have a wave each, a value a lane: a walk over the lanes
// gives every action's rank and the sum before it.  Longer rows have a workgroup: the
// border of top_k (top_p) is the value at which the count (the sum of weights) from the
// largest on reaches its target, found by its ordered bits, 11, 11 and 10 at a time,
// with histograms in LDS; equal values at the border are taken in the order of
// actions.  min_p is a border of the weights themselves.
#include "seq.h"

namespace gorila {
namespace {

constexpr uint64_t ONE = 1ull << 40;  // the weight of the largest value
constexpr int MAX_SAMPLE = 1 << 20, PIECE = 256, BINS = 2048;

struct SampleArgs {
    const void* values;
    int64_t stride, rows;
    int actions;
    const float *u, *temperature, *top_p, *min_p;
    const int32_t* top_k;
    int32_t* action;
    float* probability;
};

struct Filter {
    float most;
    double per;  // 1 / temperature
    int k;       // actions that top_k leaves
    uint64_t least;  // weight that min_p asks for
    float top_p;
};
__device__ __forceinline__ Filter filter_of(const SampleArgs& a, int64_t row) {
    Filter f;
    const float t = a.temperature ? a.temperature[row] : 1.0f;
    const bool greedy = !(t > 0.0f);
    f.per = greedy ? 1.0 : 1.0 / (double)t;
    f.k = a.top_k ? a.top_k[row] : a.actions;
    if (f.k < 1 || f.k > a.actions) f.k = a.actions;
    if (greedy) f.k = 1;
    f.top_p = a.top_p ? a.top_p[row] : 1.0f;
    const float m = a.min_p ? a.min_p[row] : 0.0f;
    f.least = !(m > 0.0f) ? 0 : m >= 1.0f ? ONE : (uint64_t)ceil((double)m * (double)ONE);
    f.most = -INFINITY;
    return f;
}
__device__ __forceinline__ float value_at(float v) { return v == v ? v + 0.0f : -INFINITY; }  // (-0 is 0)
// Whole number with the order of the values.
__device__ __forceinline__ uint32_t key_of(float v) {
    const uint32_t b = __float_as_uint(v);
    return b ^ (b >> 31 ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float value_of_key(uint32_t k) { return __uint_as_float(k ^ (k >> 31 ? 0x80000000u : 0xffffffffu)); }
__device__ __forceinline__ uint64_t weight(float v, const Filter& f) {
    if (v == f.most) return ONE;
    if (v == -INFINITY || f.most == INFINITY) return 0;
    const double x = exp(((double)v - (double)f.most) * f.per) * (double)ONE;
    // 2^52 + x has x's nearest whole number in its low bits
    return (uint64_t)__double_as_longlong(x + 4503599627370496.0) & 0xfffffffffffffull;
}
__device__ __forceinline__ uint64_t limit_of(float p, uint64_t sum) {
    if (!(p < 1.0f)) return sum;
    const uint64_t l = p > 0.0f ? (uint64_t)ceil((double)p * (double)sum) : 0;
    return l < 1 ? 1 : l;
}
// The place in the running sum that u stands for.
__device__ __forceinline__ uint64_t place_of(float u, uint64_t sum) {
    if (!(u > 0.0f)) return 0;
    if (u >= 1.0f) return sum - 1;
    const uint64_t at = (uint64_t)((double)u * (double)sum);
    return at < sum ? at : sum - 1;
}

__device__ __forceinline__ uint64_t shuffle64(uint64_t v, int lane) { return (uint64_t)__shfl((unsigned long long)v, lane, 64); }
__device__ __forceinline__ uint64_t wave_sum(uint64_t v) {
#pragma unroll
    for (int o = 32; o; o >>= 1) v += (uint64_t)__shfl_xor((unsigned long long)v, o, 64);
    return v;
}
// Sum over the lanes up to this one.
__device__ __forceinline__ uint64_t wave_running(uint64_t v) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const uint64_t p = shuffle64(v, lane >= o ? lane - o : lane);
        if (lane >= o) v += p;
    }
    return v;
}
__device__ __forceinline__ float wave_most(float v) {
#pragma unroll
    for (int o = 32; o; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
    return v;
}

template <class T>
__global__ __launch_bounds__(256) void sample_wave_kernel(SampleArgs a) {
    const int64_t row = (int64_t)blockIdx.x * 4 + threadIdx.x / 64;
    const int lane = threadIdx.x & 63;
    if (row >= a.rows) return;
    const T* p = (const T*)a.values + row * a.stride;
    const bool in = lane < a.actions;
    const float v = in ? value_at(row_value(p[lane])) : -INFINITY;
    Filter f = filter_of(a, row);
    f.most = wave_most(v);
    if (f.most == -INFINITY) {
        if (lane == 0) {
            a.action[row] = -1;
            if (a.probability) a.probability[row] = 0.0f;
        }
        return;
    }
    uint64_t w = in ? weight(v, f) : 0;
    if (f.k < a.actions || f.top_p < 1.0f) {
        int rank = 0;
        uint64_t ahead = 0;
        for (int j = 0; j < a.actions; ++j) {
            const float o = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), j));
            const uint32_t lo = __builtin_amdgcn_readlane((uint32_t)w, j), hi = __builtin_amdgcn_readlane((uint32_t)(w >> 32), j);
            if (o > v || (o == v && j < lane)) {
                ++rank;
                ahead += (uint64_t)hi << 32 | lo;
            }
        }
        if (rank >= f.k) w = 0;
        const uint64_t limit = limit_of(f.top_p, wave_sum(w));
        if (ahead >= limit) w = 0;
    }
    if (w < f.least) w = 0;
    const uint64_t running = wave_running(w), sum = shuffle64(running, 63), at = place_of(a.u[row], sum);
    const int first = __ffsll((unsigned long long)__ballot(running > at)) - 1;
    if (lane == first) {
        a.action[row] = lane;
        if (a.probability) a.probability[row] = (float)((double)w / (double)sum);
    }
}

// Of n whole numbers in LDS, in this order (DOWN: from the last on): the one at which the
// sum passes `at` (less than the sum of all), the sum before it, itself.  By a whole wave.
struct Found {
    int index;
    uint64_t above, level;
};
template <bool DOWN>
__device__ __forceinline__ Found find(const unsigned long long* v, int n, uint64_t at) {
    const int lane = threadIdx.x & 63, per = (n + 63) / 64;
    auto get = [&](int i) -> uint64_t { return i < n ? v[DOWN ? n - 1 - i : i] : 0; };
    uint64_t own = 0;
    for (int i = 0; i < per; ++i) own += get(lane * per + i);
    const uint64_t upto = wave_running(own);
    uint64_t sum = upto - own, level = 0;
    const bool here = sum <= at && at < upto;
    int i = lane * per;
    if (here) {
        while (i < n && sum + get(i) <= at) sum += get(i++);
        level = get(i);
    }
    const int from = __ffsll((unsigned long long)__ballot(here)) - 1;
    Found f;
    i = __shfl(i, from, 64);
    f.index = DOWN ? n - 1 - i : i;
    f.above = shuffle64(sum, from);
    f.level = shuffle64(level, from);
    return f;
}

// A workgroup's row.
struct RowShared {
    unsigned long long bins[BINS];
    unsigned long long pieces[MAX_SAMPLE / PIECE];
    float most[16];
    Found found;  // what the first wave tells the others
};

template <class T, int THREADS>
__global__ __launch_bounds__(THREADS) void sample_row_kernel(SampleArgs a) {
    __shared__ RowShared sh;
    constexpr int NW = THREADS / 64;
    const int64_t row = blockIdx.x;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = a.actions, pieces = (n + PIECE - 1) / PIECE;
    const T* p = (const T*)a.values + row * a.stride;
    // f(value, action) of all of them; a wave takes whole pieces
    auto each = [&](auto&& f) {
        for (int piece = wave; piece < pieces; piece += NW) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int i = piece * PIECE + j * 64 + lane;
                if (i < n) f(value_at(row_value(p[i])), i);
            }
        }
    };
    // pieces[] = sums of f(value, action) over each
    auto sums = [&](auto&& f) {
        __syncthreads();
        for (int piece = wave; piece < pieces; piece += NW) {
            uint64_t s = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int i = piece * PIECE + j * 64 + lane;
                if (i < n) s += f(value_at(row_value(p[i])), i);
            }
            s = wave_sum(s);
            if (lane == 0) sh.pieces[piece] = s;
        }
        __syncthreads();
    };
    auto total = [&]() -> uint64_t {  // of the pieces, for every lane
        uint64_t s = 0;
        for (int i = lane; i < pieces; i += 64) s += sh.pieces[i];
        return wave_sum(s);
    };

    Filter f = filter_of(a, row);
    float most = -INFINITY;
    each([&](float v, int) { most = fmaxf(most, v); });
    most = wave_most(most);
    if (lane == 0) sh.most[wave] = most;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NW; ++i) most = fmaxf(most, sh.most[i]);
    f.most = most;
    if (most == -INFINITY) {
        if (threadIdx.x == 0) {
            a.action[row] = -1;
            if (a.probability) a.probability[row] = 0.0f;
        }
        return;
    }

    // The key at which the sum of `measure` from the largest on reaches `target` (1 or more),
    // the sum above it, and its own.
    struct Border {
        uint32_t key;
        uint64_t above, own;
    };
    auto border = [&](uint64_t target, auto&& measure) {
        Border b{0, 0, 0};
        uint32_t mask = 0;
        constexpr int SHIFT[3] = {21, 10, 0}, BITS[3] = {11, 11, 10};
#pragma unroll
        for (int d = 0; d < 3; ++d) {
            __syncthreads();
            for (int i = threadIdx.x; i < BINS; i += THREADS) sh.bins[i] = 0;
            __syncthreads();
            each([&](float v, int) {
                const uint32_t key = key_of(v);
                if ((key & mask) != b.key) return;
                const uint64_t m = measure(v);
                if (m) atomicAdd(&sh.bins[key >> SHIFT[d] & ((1u << BITS[d]) - 1)], (unsigned long long)m);
            });
            __syncthreads();
            if (wave == 0) {
                const Found got = find<true>(sh.bins, 1 << BITS[d], target - 1 - b.above);
                if (lane == 0) sh.found = got;
            }
            __syncthreads();
            b.key |= (uint32_t)sh.found.index << SHIFT[d];
            b.above += sh.found.above;
            b.own = sh.found.level;
            mask |= ((1u << BITS[d]) - 1) << SHIFT[d];
        }
        return b;
    };

    uint32_t key = 0;                        // larger ones stay,
    uint64_t ties = ~0ull, equal = 0;        // and so many of the `equal` ones that are equal
    if (f.k < n) {
        const Border b = border((uint64_t)f.k, [](float) { return 1; });
        key = b.key, ties = (uint64_t)f.k - b.above, equal = b.own;
    }
    if (f.top_p < 1.0f) {
        sums([&](float v, int) { return key_of(v) > key ? weight(v, f) : 0; });
        uint64_t sum = total();
        if (f.k < n) sum += ties * weight(value_of_key(key), f);
        const uint64_t limit = limit_of(f.top_p, sum);
        const Border b = border(limit, [&](float v) { return weight(v, f); });
        const uint64_t w = weight(value_of_key(b.key), f), t = (limit - b.above + w - 1) / w;
        if (f.k >= n || b.key != key || t < ties) ties = t;
        key = b.key, equal = b.own / w;
    }
    int end = n;  // equal ones of this action and later ones do not stay
    if (ties < equal) {
        sums([&](float v, int) { return key_of(v) == key ? 1 : 0; });
        const Found got = find<false>(sh.pieces, pieces, ties);
        const int piece = got.index;
        uint64_t before = got.above;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int i = piece * PIECE + j * 64 + lane;
            const uint64_t is = __ballot(i < n && key_of(value_at(row_value(p[i < n ? i : 0]))) == key);
            const int here = __popcll(is);
            if (before <= ties && ties < before + here) {
                // the lane with ties - before of them in front of it
                const bool me = (is >> lane & 1) && (uint64_t)__popcll(is & ((1ull << lane) - 1)) == ties - before;
                end = piece * PIECE + j * 64 + __ffsll((unsigned long long)__ballot(me)) - 1;
            }
            before += here;
        }
    }
    auto kept = [&](float v, int i) -> uint64_t {
        const uint32_t k = key_of(v);
        if (k < key || (k == key && i >= end)) return 0;
        const uint64_t w = weight(v, f);
        return w < f.least ? 0 : w;
    };
    sums(kept);
    const uint64_t sum = total(), at = place_of(a.u[row], sum);
    if (wave != 0) return;
    const Found got = find<false>(sh.pieces, pieces, at);
    const int piece = got.index;
    uint64_t before = got.above;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int i = piece * PIECE + j * 64 + lane;
        const uint64_t w = i < n ? kept(value_at(row_value(p[i])), i) : 0;
        const uint64_t upto = wave_running(w) + before;
        if (upto - w <= at && at < upto) {
            a.action[row] = i;
            if (a.probability) a.probability[row] = (float)((double)w / (double)sum);
        }
        before = shuffle64(upto, 63);
    }
}

}  // namespace
}  // namespace gorila

using namespace gorila;

extern "C" {

int gorila_sample_actions(const void* values, int64_t stride, int64_t rows, int32_t actions, int32_t dtype, const float* u,
                          const float* temperature, const int32_t* top_k, const float* top_p, const float* min_p, int32_t* action_out,
                          float* probability_out, gorila_ctx* ctx) {
    CtxView c;
    const int rc = ctx_view(ctx, 0, c);
    if (rc) return rc;
    if (!row_dtype(dtype) || rows < 0 || actions < 1) return GORILA_EINVAL;
    if (actions > MAX_SAMPLE) return GORILA_EUNSUPPORTED;
    if (rows == 0) return GORILA_OK;
    if (!values || !u || !action_out || !at_element(values, dtype_bytes(dtype))) return GORILA_EINVAL;
    for (const void* p : {(const void*)u, (const void*)temperature, (const void*)top_k, (const void*)top_p, (const void*)min_p,
                          (const void*)action_out, (const void*)probability_out})
        if (!at_element(p, 4)) return GORILA_EINVAL;
    const SampleArgs a{values, stride, rows, actions, u, temperature, top_p, min_p, top_k, action_out, probability_out};
    const int threads = actions <= 64 ? 64 : actions <= 2048 ? 256 : 1024;
    if (!(threads == 64 ? launch_fits((double)((rows + 3) / 4), 256) : launch_fits((double)rows, threads))) return GORILA_EUNSUPPORTED;
    auto go = [&](auto t) {
        using T = decltype(t);
        if (threads == 64) sample_wave_kernel<T><<<(unsigned)((rows + 3) / 4), 256, 0, c.stream>>>(a);
        else if (threads == 256) sample_row_kernel<T, 256><<<(unsigned)rows, 256, 0, c.stream>>>(a);
        else sample_row_kernel<T, 1024><<<(unsigned)rows, 1024, 0, c.stream>>>(a);
    };
    dtype == GORILA_F32 ? go(float{}) : go(uint16_t{});
    return launched();
}

}  // extern "C"
