// Actions sampled from values (gorila_sample_actions).
//
// Weights are whole numbers, 2^40 exp((value - most) / temperature) rounded: their sums
// are exact in 64 bits whatever the order (2^20 actions give at most 2^60), so that the
// filters' borders and the drawn action do not depend on how a row is cut.
//
// Rows of up to 64 actions have a wave each, a value a lane: a walk over the lanes
// gives every action's rank and the sum before it (1024 x 18: 5.3 us, most of it the
// launch).  Longer rows have a workgroup.  The border of top_k (top_p) is the value at
// which the count (the sum of weights) from the largest on reaches its target.  A
// histogram over 2048 even bins of (most - value) / temperature, which spreads a row's
// values over many LDS addresses, says in which bin it lies; the bin's values, few as a
// rule, are taken to LDS, where each is held against the others (more than 256: searched
// by their ordered bits, eight at a time; more than 4096: over the whole row).  top_k
// takes all values above its bin with it, if they fit, so that only they need weights.
// Equal values at the border are taken in the order of actions.  min_p is a border
// of the weights themselves.
//
// What bounds a workgroup: a weight is some 25 operations in fp64, of 10 cycles each
// as measured, so 32000 of them take it 13 us.  They are formed once for every value (top_p's
// histogram) and once more for those that stay; under top_k for those alone.
// 256 x 32000 bf16: 21 us without a filter, 27 with top_k, 54 with top_p, 33 with all.
//
// Few rows of many actions would leave the chip idle: each is shared by up to 64
// workgroups, a launch for each step (largest value, histogram, list, sums, action).
// 1 x 100003 fp32, top_p: 28 us, by one workgroup 100.
#include "seq.h"

namespace gorila {
namespace {

constexpr uint64_t ONE = 1ull << 40;  // the weight of the largest value
constexpr int MAX_SAMPLE = 1 << 20, SMALL = 256, SHARED_FROM = 16384;
constexpr double LOG2E = 1.4426950408889634;
constexpr double GONE = -41.0;  // a base-2 exponent from which on a weight is 0

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
    double per;  // log2(e) / temperature
    int k;       // actions that top_k leaves
    uint64_t least;  // weight that min_p asks for
    float top_p;
};
__device__ __forceinline__ Filter filter_of(const SampleArgs& a, int64_t row) {
    Filter f;
    const float t = a.temperature ? a.temperature[row] : 1.0f;
    const bool greedy = !(t > 0.0f);
    f.per = greedy ? LOG2E : LOG2E / (double)t;
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
// 2^40 2^y for y in [-41, 0] in fp64: the series of 2^r, |r| <= 1/2 (the next term is
// 2^-53 of it).  Its coefficients are kept in scalar registers: as literals each takes an
// instruction of its own for every value.
struct Series {
    double c[13];
    __device__ __forceinline__ Series() {
        double t = 1.0;
#pragma unroll
        for (int k = 0; k <= 12; ++k) {
            c[k] = t;
            t *= 0.69314718055994531 / (k + 1);
        }
#pragma unroll
        for (int k = 0; k <= 12; ++k) asm("" : "+s"(c[k]));
    }
    __device__ __forceinline__ double power40(double y) const {
        // 1.5 2^52 + y has y's nearest whole number n in its low bits; s, between 0.7 and 1.5, takes n + 40 into its exponent
        const double big = y + 6755399441055744.0, r = y - (big - 6755399441055744.0);
        double s = c[12];
#pragma unroll
        for (int k = 11; k >= 0; --k) s = fma(r, s, c[k]);
        const int n = (int)(uint32_t)__double_as_longlong(big);
        return __longlong_as_double(__double_as_longlong(s) + ((int64_t)(n + 40) << 52));
    }
};
__device__ __forceinline__ uint64_t weight(float v, const Filter& f, const Series& e) {
    // -infinity (and NaN: what lies beside an infinite most) come out as the exponent -41, a weight of 1/2: 0
    const double y = fmax(((double)v - (double)f.most) * f.per, GONE);
    // 2^52 + x has x's nearest whole number in its low bits
    const uint64_t w = (uint64_t)__double_as_longlong(e.power40(y) + 4503599627370496.0) & 0xfffffffffffffull;
    return v == f.most ? ONE : w;
}
// The bin of a value: the same for equal ones, and not less for a smaller one.
template <int BINS>
__device__ __forceinline__ int bin_of(float v, float most, float per) {
    return v == most ? 0 : (int)(uint32_t)fminf((most - v) * per, (float)(BINS - 1));
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

__device__ __forceinline__ uint64_t lane64(uint64_t v, int lane) {  // of a lane that the wave agrees on
    return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((uint32_t)(v >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((uint32_t)v, lane);
}
template <int CONTROL, int ROWS>
__device__ __forceinline__ uint64_t plus_lane64(uint64_t v) {
    const uint32_t lo = __builtin_amdgcn_update_dpp(0, (uint32_t)v, CONTROL, ROWS, 0xf, false);
    const uint32_t hi = __builtin_amdgcn_update_dpp(0, (uint32_t)(v >> 32), CONTROL, ROWS, 0xf, false);
    return v + ((uint64_t)hi << 32 | lo);
}
// Sum over the lanes up to this one, as over_wave() goes.  (Twelve shuffles through LDS wait 0.6 us.)
__device__ __forceinline__ uint64_t wave_running(uint64_t v) {
    v = plus_lane64<0x111, 0xf>(v);
    v = plus_lane64<0x112, 0xf>(v);
    v = plus_lane64<0x114, 0xf>(v);
    v = plus_lane64<0x118, 0xf>(v);
    v = plus_lane64<0x142, 0xa>(v);
    return plus_lane64<0x143, 0xc>(v);
}
__device__ __forceinline__ uint64_t wave_sum(uint64_t v) { return lane64(wave_running(v), 63); }
template <int CONTROL, int ROWS>
__device__ __forceinline__ float most_lane(float v) {
    const int b = __builtin_bit_cast(int, v);
    return fmaxf(v, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(b, b, CONTROL, ROWS, 0xf, false)));
}
__device__ __forceinline__ float wave_most(float v) {
    v = most_lane<0x111, 0xf>(v);
    v = most_lane<0x112, 0xf>(v);
    v = most_lane<0x114, 0xf>(v);
    v = most_lane<0x118, 0xf>(v);
    v = most_lane<0x142, 0xa>(v);
    v = most_lane<0x143, 0xc>(v);
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
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
    uint64_t w = in ? weight(v, f, Series()) : 0;
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
    const uint64_t running = wave_running(w), sum = lane64(running, 63), at = place_of(a.u[row], sum);
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
template <bool DOWN, class I>
__device__ __forceinline__ Found find(const I* v, int n, uint64_t at) {
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
    i = __builtin_amdgcn_readlane(i, from);
    f.index = DOWN ? n - 1 - i : i;
    f.above = lane64(sum, from);
    f.level = lane64(level, from);
    return f;
}

// A row in parts of 256 places, a load of four values for each lane of a wave.  Loads start where
// the addresses allow them: place i is action i - shift.
template <class T>
struct Row {
    const T* p;
    int n, shift, parts, lane;
    __device__ __forceinline__ Row(const SampleArgs& a, int64_t row) {
        p = (const T*)a.values + row * a.stride;
        n = a.actions, shift = (int)((uintptr_t)p / sizeof(T) & 3), parts = (n + shift + 255) / 256, lane = threadIdx.x & 63;
    }
    __device__ __forceinline__ int action(int part, int j) const { return part * 256 + lane * 4 + j - shift; }
    __device__ __forceinline__ bool inside(int action) const { return action >= 0 && action < n; }
    __device__ __forceinline__ bool whole(int part) const { return part * 256 >= shift && part * 256 + 256 - shift <= n; }
    // As it is read (outside the row: -infinity), and as values.
    __device__ __forceinline__ f32x4 load(int part) const {
        const int first = action(part, 0);
        f32x4 u;
        if (first >= 0 && first + 4 <= n) {
            u = row_load4(p + first);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) u[j] = inside(first + j) ? row_value(p[first + j]) : -INFINITY;
        }
        return u;
    }
};
__device__ __forceinline__ f32x4 values_of(f32x4 u) { return f32x4{value_at(u[0]), value_at(u[1]), value_at(u[2]), value_at(u[3])}; }
// f(values, part) for the parts of a wave, `step` apart, the next load under way.
template <class R, class F>
__device__ __forceinline__ void each_part(const R& r, int first, int step, F&& f) {
    if (first >= r.parts) return;
    f32x4 next = r.load(first);
#pragma unroll 1
    for (int part = first; part < r.parts; part += step) {
        const f32x4 v = values_of(next);
        if (part + step < r.parts) next = r.load(part + step);
        f(v, part);
    }
}

// What the workgroups that share a row tell each other, in the workspace.
constexpr int SHARES = 64, ALL_BINS = 2048, ALL_LIST = 4096;
struct RowSpace {
    unsigned long long bins[ALL_BINS], sums[MAX_SAMPLE / 256 + 1];
    uint32_t count[ALL_BINS], key[ALL_LIST], act[ALL_LIST];
    float most[SHARES];
    uint32_t listed, done, border;  // done: the border and the parts' sums are known
    int end;
};

template <int BINS, int LIST, int PARTS>
struct RowShared {
    unsigned long long bins[BINS], weight[LIST], sums[PARTS], digits[256], part[16];
    unsigned long long small_weight[SMALL];
    uint32_t count[BINS], key[LIST], act[LIST], small_key[SMALL], small_act[SMALL];
    float most[16];
    Found found;
    uint32_t listed, few;
    int end;
};

// The largest of a workgroup's values, for all.
template <int NW>
__device__ __forceinline__ float block_most(float v, float (&sm)[16]) {
    v = wave_most(v);
    if ((threadIdx.x & 63) == 0) sm[threadIdx.x >> 6] = v;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NW; ++i) v = fmaxf(v, sm[i]);
    return v;
}
// As find() by the whole workgroup, N entries, for all; `sum`: of all of them; target(): the sum to pass.
template <int N, int THREADS, class S, class I, class F>
__device__ __forceinline__ Found find_all(S& sh, const I* entries, uint64_t& sum, bool down, F&& target) {
    constexpr int NW = THREADS / 64, PER = N > THREADS ? N / THREADS : 1;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    __syncthreads();
    uint64_t own[PER], mine = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int e = threadIdx.x * PER + i;
        own[i] = e < N ? entries[down ? N - 1 - e : e] : 0;
        mine += own[i];
    }
    uint64_t upto = wave_running(mine);
    if (lane == 63) sh.part[wave] = upto;
    __syncthreads();
    sum = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        if (w == wave) upto += sum;
        sum += sh.part[w];
    }
    const uint64_t at = target();
    uint64_t before = upto - mine;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int e = threadIdx.x * PER + i;
        if (before <= at && at < before + own[i]) sh.found = Found{down ? N - 1 - e : e, before, own[i]};
        before += own[i];
    }
    __syncthreads();
    return sh.found;
}
template <int NW, class S>
__device__ __forceinline__ uint64_t block_sum(S& sh, uint64_t v) {
    __syncthreads();
    v = wave_sum(v);
    if ((threadIdx.x & 63) == 0) sh.part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0;
#pragma unroll
    for (int i = 0; i < NW; ++i) v += sh.part[i];
    return v;
}

// A wave's values into a histogram of numbers (COUNT) or of weights.  Lanes that meet in an
// address wait for each other: a wave in one bin adds once, and numbers in the last bin, where
// all that is far below the largest value lies, are counted over the wave.
template <int BINS, bool COUNT, class R, class W, class I>
__device__ __forceinline__ void add_to_bins(const R& r, f32x4 v, int part, float most, float per, W&& weigh, I* bins) {
    uint64_t w[4];
    const bool whole = r.whole(part);
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = COUNT ? whole || r.inside(r.action(part, j)) : weigh(v[j]);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int b = bin_of<BINS>(v[j], most, per);
        if (COUNT) {
            const uint64_t far = __ballot(w[j] && b == BINS - 1);
            if (far) {
                if (r.lane == 0) atomicAdd(bins + BINS - 1, (I)__popcll(far));
                if (b == BINS - 1) w[j] = 0;
            }
        }
        if (__all(b == __builtin_amdgcn_readfirstlane(b))) {
            const uint64_t s = COUNT ? __popcll(__ballot(w[j] != 0)) : wave_sum(w[j]);
            if (r.lane == 0 && s) atomicAdd(bins + b, (I)s);
        } else if (w[j]) {
            atomicAdd(bins + b, (I)w[j]);
        }
    }
}
// A wave's values of the bins first .. last to a list (of which *listed counts them all, and LIST are kept).
template <int BINS, int LIST, class R>
__device__ __forceinline__ void add_to_list(const R& r, f32x4 v, int part, float most, float per, int first, int last, uint32_t* listed,
                                            uint32_t* key, uint32_t* act) {
    bool is[4], any = false;
#pragma unroll
    for (int j = 0; j < 4; ++j) {  // as bin_of() says; what is no number is in the last bin
        const float d = v[j] == most ? 0.0f : (most - v[j]) * per;
        is[j] = last == BINS - 1 ? !(d < (float)first) : d >= (float)first && d < (float)(last + 1);
    }
    if (!r.whole(part)) {
#pragma unroll
        for (int j = 0; j < 4; ++j) is[j] = is[j] && r.inside(r.action(part, j));
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) any = any || is[j];
    if (!__any(any)) return;
    uint64_t who[4];
    int all = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        who[j] = __ballot(is[j]);
        all += __popcll(who[j]);
    }
    uint32_t base = 0;
    if (r.lane == 0) base = atomicAdd(listed, (uint32_t)all);
    base = __builtin_amdgcn_readfirstlane(base);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t at = base + __builtin_amdgcn_mbcnt_hi((uint32_t)(who[j] >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)who[j], 0));
        if (is[j] && at < (uint32_t)LIST) key[at] = key_of(v[j]), act[at] = r.action(part, j);
        base += __popcll(who[j]);
    }
}

// The rows' shares: a workgroup takes 16 parts in turn with the others of its row.
struct Share {
    int64_t row;
    int g, first, step;  // the workgroup's number, its wave's first part, and the next
    __device__ __forceinline__ Share(int shares)
        : row(blockIdx.x / shares), g(blockIdx.x % shares), first(g * 16 + (threadIdx.x >> 6)), step(shares * 16) {}
};
template <class T>
__global__ __launch_bounds__(1024) void share_most_kernel(SampleArgs a, RowSpace* space, int shares) {
    __shared__ float sm[16];
    const Share s(shares);
    const Row<T> r(a, s.row);
    RowSpace& w = space[s.row];
    for (int i = s.g * 1024 + threadIdx.x; i < ALL_BINS; i += shares * 1024) w.bins[i] = 0, w.count[i] = 0;
    if (s.g == 0 && threadIdx.x == 0) w.listed = w.done = 0;
    float most = -INFINITY;
    each_part(r, s.first, s.step, [&](f32x4 v, int) { most = fmaxf(fmaxf(most, fmaxf(v[0], v[1])), fmaxf(v[2], v[3])); });
    most = block_most<16>(most, sm);
    if (threadIdx.x == 0) w.most[s.g] = most;
}
__device__ __forceinline__ float most_of(const RowSpace& w, int shares) {
    const int lane = threadIdx.x & 63;
    return wave_most(lane < shares ? w.most[lane] : -INFINITY);
}
// A row's histogram.
template <class T>
__global__ __launch_bounds__(1024) void share_bins_kernel(SampleArgs a, RowSpace* space, int shares) {
    __shared__ unsigned long long bins[ALL_BINS];
    const Share s(shares);
    const Row<T> r(a, s.row);
    RowSpace& w = space[s.row];
    const Series series;
    Filter f = filter_of(a, s.row);
    f.most = most_of(w, shares);
    const bool by_count = f.k < r.n;
    if (f.most == -INFINITY || !(by_count || f.top_p < 1.0f)) return;
    const float per = (float)(f.per * (ALL_BINS / -GONE));
    auto weigh = [&](float x) { return weight(x, f, series); };
    uint32_t* count = (uint32_t*)bins;
    for (int i = threadIdx.x; i < ALL_BINS; i += 1024) bins[i] = 0;
    __syncthreads();
    if (by_count) each_part(r, s.first, s.step, [&](f32x4 v, int part) { add_to_bins<ALL_BINS, true>(r, v, part, f.most, per, weigh, count); });
    else each_part(r, s.first, s.step, [&](f32x4 v, int part) { add_to_bins<ALL_BINS, false>(r, v, part, f.most, per, weigh, bins); });
    __syncthreads();
    for (int i = threadIdx.x; i < ALL_BINS; i += 1024) {
        if (by_count && count[i]) atomicAdd(w.count + i, count[i]);
        if (!by_count && bins[i]) atomicAdd(w.bins + i, bins[i]);
    }
}
// The bin of a row's first border: top_k's, or top_p's alone.
template <int BINS, int THREADS, class S>
__device__ __forceinline__ Found first_border(S& sh, const uint32_t* count, const unsigned long long* bins, const Filter& f, bool by_count,
                                              uint64_t& limit) {
    uint64_t sum;
    return by_count ? find_all<BINS, THREADS>(sh, count, sum, false, [&] { return (uint64_t)f.k - 1; })
                    : find_all<BINS, THREADS>(sh, bins, sum, false, [&] {
                          limit = limit_of(f.top_p, sum);
                          return limit - 1;
                      });
}
// Its list: top_k's bin and all above it, or top_p's bin.
template <class T>
__global__ __launch_bounds__(1024) void share_list_kernel(SampleArgs a, RowSpace* space, int shares) {
    __shared__ struct {
        unsigned long long part[16];
        Found found;
    } sh;
    const Share s(shares);
    const Row<T> r(a, s.row);
    RowSpace& w = space[s.row];
    Filter f = filter_of(a, s.row);
    f.most = most_of(w, shares);
    const bool by_count = f.k < r.n;
    if (f.most == -INFINITY || !(by_count || f.top_p < 1.0f)) return;
    const float per = (float)(f.per * (ALL_BINS / -GONE));
    uint64_t limit;
    const Found at = first_border<ALL_BINS, 1024>(sh, w.count, w.bins, f, by_count, limit);
    each_part(r, s.first, s.step, [&](f32x4 v, int part) {
        add_to_list<ALL_BINS, ALL_LIST>(r, v, part, f.most, per, by_count ? 0 : at.index, at.index, &w.listed, w.key, w.act);
    });
}

// A row's action by a workgroup (WHOLE), or where workgroups share it and its histogram and
// list are in the workspace, the sums of its parts (SUMS), and the action of them (PICK; a
// row whose list was too long is taken whole).
enum Part { WHOLE, SUMS, PICK };
template <class T, int THREADS, int BINS, int LIST, int MOST, Part PART>
__global__ __launch_bounds__(THREADS) void sample_row_kernel(SampleArgs a, RowSpace* space, int shares) {
    constexpr int NW = THREADS / 64;
    __shared__ RowShared<BINS, LIST, MOST / 256 + 1> sh;
    const int64_t row = PART == SUMS ? blockIdx.x / shares : blockIdx.x;
    const int share = PART == SUMS ? blockIdx.x % shares : 0;
    const Row<T> r(a, row);
    const int lane = r.lane, wave = threadIdx.x >> 6, n = r.n, parts = r.parts;
    const Series series;
    Filter f = filter_of(a, row);
    auto weigh = [&](float v) { return weight(v, f, series); };
    auto each = [&](auto&& f) { each_part(r, wave, NW, f); };
    // sums[] of parts first, first + step, ..: g(value) over the values that stay(value, action);
    // g is formed for all of a wave's four values or none, so that its long chains overlap.
    auto sum_parts = [&](int first, int step, unsigned long long* sums, auto&& stay, auto&& g) {
        each_part(r, first, step, [&](f32x4 v, int part) {
            bool some[4], any = false;
#pragma unroll
            for (int j = 0; j < 4; ++j) any |= some[j] = stay(v[j], r.action(part, j));
            uint64_t s = 0;
            if (__any(any)) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint64_t w = g(v[j]);
                    s += some[j] ? w : 0;
                }
                s = wave_sum(s);
            }
            if (lane == 0) sums[part] = s;
        });
    };
    auto sums = [&](auto&& stay, auto&& g) {  // of all parts
        __syncthreads();
        sum_parts(wave, NW, sh.sums, stay, g);
        __syncthreads();
    };
    auto total = [&]() -> uint64_t {  // of the sums, for every lane
        uint64_t s = 0;
        for (int i = lane; i < parts; i += 64) s += sh.sums[i];
        return wave_sum(s);
    };

    if (PART != WHOLE) {
        f.most = most_of(space[row], shares);
    } else {
        float most = -INFINITY;
        each([&](f32x4 v, int) { most = fmaxf(fmaxf(most, fmaxf(v[0], v[1])), fmaxf(v[2], v[3])); });
        f.most = block_most<NW>(most, sh.most);
    }
    if (f.most == -INFINITY) {
        if (PART != SUMS && threadIdx.x == 0) {
            a.action[row] = -1;
            if (a.probability) a.probability[row] = 0.0f;
        }
        return;
    }

    uint32_t key = 0;                  // larger ones stay,
    uint64_t ties = ~0ull, equal = 0;  // and so many of the `equal` ones that are equal
    int end = n;                       // : those before this action
    bool complete = false;             // all that may stay is in the list
    const bool by_count = f.k < n, by_sum = f.top_p < 1.0f;
    const bool known = PART == PICK && space[row].done;
    if (known) {
        key = space[row].border, end = space[row].end;
        for (int i = threadIdx.x; i < parts; i += THREADS) sh.sums[i] = space[row].sums[i];
        __syncthreads();
    } else if (by_count || by_sum) {
        const float per = (float)(f.per * (BINS / -GONE));
        auto bin_at = [&](float v) { return bin_of<BINS>(v, f.most, per); };
        bool in_list = false;  // the bin at hand is in the list
        uint32_t listed = 0;
        uint64_t limit = 0, all;
        Found at;
        auto list = [&](int first, int last) {
            __syncthreads();
            if (threadIdx.x == 0) sh.listed = 0;
            __syncthreads();
            each([&](f32x4 v, int part) { add_to_list<BINS, LIST>(r, v, part, f.most, per, first, last, &sh.listed, sh.key, sh.act); });
            __syncthreads();
            listed = sh.listed;
            in_list = listed <= LIST;
        };
        auto weigh_list = [&] {
            if (by_sum)
                for (uint32_t i = threadIdx.x; i < listed; i += THREADS) sh.weight[i] = weigh(value_of_key(sh.key[i]));
            __syncthreads();
        };
        if (PART == SUMS) {
            at = first_border<BINS, THREADS>(sh, space[row].count, space[row].bins, f, by_count, limit);
            listed = space[row].listed;
            if (listed > LIST) {
                if (share == 0 && threadIdx.x == 0) space[row].done = 0;
                return;
            }
            for (uint32_t i = threadIdx.x; i < listed; i += THREADS) sh.key[i] = space[row].key[i], sh.act[i] = space[row].act[i];
            in_list = true, complete = by_count;
            __syncthreads();
            weigh_list();
        } else {
            for (int i = threadIdx.x; i < BINS; i += THREADS) sh.bins[i] = 0, sh.count[i] = 0;
            __syncthreads();
            if (by_count) each([&](f32x4 v, int part) { add_to_bins<BINS, true>(r, v, part, f.most, per, weigh, sh.count); });
            else each([&](f32x4 v, int part) { add_to_bins<BINS, false>(r, v, part, f.most, per, weigh, sh.bins); });
            at = first_border<BINS, THREADS>(sh, sh.count, sh.bins, f, by_count, limit);
            complete = by_count && at.above + at.level <= LIST;
            if (complete) {
                list(0, at.index);
                weigh_list();
            }
        }

        // The key in the bin `at` at which the sum of weights (or numbers) from the largest on reaches `target`,
        // the sum above it and its own.
        struct Border {
            uint32_t key;
            uint64_t above, own;
        };
        auto border = [&](Found at, uint64_t target, bool weights) {
            if (PART != SUMS && !complete) {
                list(at.index, at.index);
                if (in_list) weigh_list();
            }
            Border b{0, at.above, 0};
            if (in_list) {  // the bin's few, each held against the others
                __syncthreads();
                if (threadIdx.x == 0) sh.few = 0;
                __syncthreads();
                for (uint32_t i = threadIdx.x; i < listed; i += THREADS)
                    if (bin_at(value_of_key(sh.key[i])) == at.index) {
                        const uint32_t k = atomicAdd(&sh.few, 1u);
                        if (k < SMALL) sh.small_key[k] = sh.key[i], sh.small_act[k] = sh.act[i], sh.small_weight[k] = weights ? sh.weight[i] : 1;
                    }
                __syncthreads();
                const uint32_t few = sh.few;
                if (few <= SMALL) {
                    if (threadIdx.x < few) {
                        const uint32_t own = sh.small_key[threadIdx.x];
                        uint64_t above = at.above, same = 0;
                        uint32_t first = ~0u;
#pragma unroll 8
                        for (uint32_t j = 0; j < few; ++j) {
                            const uint32_t o = sh.small_key[j];
                            const uint64_t m = sh.small_weight[j];
                            above += o > own ? m : 0;
                            same += o == own ? m : 0;
                            first = o == own && j < first ? j : first;
                        }
                        if (first == threadIdx.x && above < target && target <= above + same) sh.found = Found{(int)own, above, same};
                    }
                    __syncthreads();
                    return Border{(uint32_t)sh.found.index, sh.found.above, sh.found.level};
                }
            }
            // the bits in which the bin's keys differ at all (a list's): the others need no search
            uint32_t differ = ~0u;
            if (in_list) {
                __syncthreads();
                if (threadIdx.x == 0) sh.few = 0;
                __syncthreads();
                for (uint32_t i = threadIdx.x; i < listed; i += THREADS)
                    if (bin_at(value_of_key(sh.key[i])) == at.index) atomicOr(&sh.few, sh.key[i] ^ sh.small_key[0]);
                __syncthreads();
                differ = sh.few;
                __syncthreads();
                if (threadIdx.x == 0) sh.few = SMALL + 1;
                b.key = sh.small_key[0] & ~differ;
            }
#pragma unroll 1
            for (int shift = 24; shift >= 0; shift -= 8) {
                if ((differ >> shift & 255u) == 0 && shift > 0) continue;
                auto add = [&](uint32_t k, uint64_t m) {
                    if (((uint64_t)(k ^ b.key) >> (shift + 8)) == 0 && m) atomicAdd(&sh.digits[k >> shift & 255u], (unsigned long long)m);
                };
                __syncthreads();
                if (threadIdx.x < 256) sh.digits[threadIdx.x] = 0;
                __syncthreads();
                if (in_list) {
                    for (uint32_t i = threadIdx.x; i < listed; i += THREADS)
                        if (bin_at(value_of_key(sh.key[i])) == at.index) add(sh.key[i], weights ? sh.weight[i] : 1);
                } else {
                    each([&](f32x4 v, int part) {
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            if (bin_at(v[j]) == at.index && r.inside(r.action(part, j))) add(key_of(v[j]), weights ? weigh(v[j]) : 1);
                    });
                }
                const Found got = find_all<256, THREADS>(sh, sh.digits, all, true, [&] { return target - 1 - b.above; });
                b.key |= (uint32_t)got.index << shift;
                b.above += got.above;
                b.own = got.level;
            }
            return b;
        };
        if (by_count) {
            const Border b = border(at, (uint64_t)f.k, false);
            key = b.key, ties = (uint64_t)f.k - b.above, equal = b.own;
        }
        if (by_sum) {
            if (by_count) {  // of the weights that top_k leaves, or (their histogram) of more
                uint64_t left = 0;
                __syncthreads();
                for (int i = threadIdx.x; i < BINS; i += THREADS) sh.bins[i] = 0;
                __syncthreads();
                if (complete) {
                    for (uint32_t i = threadIdx.x; i < listed; i += THREADS) {
                        const uint64_t w = sh.weight[i];
                        if (sh.key[i] > key) left += w;
                        if (w) atomicAdd(&sh.bins[bin_at(value_of_key(sh.key[i]))], (unsigned long long)w);
                    }
                    left = block_sum<NW>(sh, left);
                } else {
                    each([&](f32x4 v, int part) { add_to_bins<BINS, false>(r, v, part, f.most, per, weigh, sh.bins); });
                    sums([&](float v, int) { return key_of(v) > key; }, weigh);
                    left = total();
                }
                limit = limit_of(f.top_p, left + ties * weigh(value_of_key(key)));
                at = find_all<BINS, THREADS>(sh, sh.bins, all, false, [&] { return limit - 1; });
            }
            const Border b = border(at, limit, true);
            const uint64_t w = weigh(value_of_key(b.key)), t = (limit - b.above + w - 1) / w;
            if (!by_count || b.key != key || t < ties) ties = t;
            key = b.key, equal = b.own / w;
        }
        if (ties < equal) {  // the first of the equal ones that does not stay
            const uint32_t few = sh.few;
            if (in_list && few <= SMALL) {
                if (threadIdx.x < few && sh.small_key[threadIdx.x] == key) {
                    const uint32_t own = sh.small_act[threadIdx.x];
                    uint32_t rank = 0;
#pragma unroll 8
                    for (uint32_t j = 0; j < few; ++j) rank += sh.small_key[j] == key && sh.small_act[j] < own;
                    if (rank == ties) sh.end = (int)own;
                }
                __syncthreads();
                end = sh.end;
            } else {
                sums([&](float v, int i) { return key_of(v) == key && r.inside(i); }, [](float) -> uint64_t { return 1; });
                const Found got = find<false>(sh.sums, parts, ties);
                const f32x4 v = values_of(r.load(got.index));
                uint64_t own = 0;
#pragma unroll
                for (int j = 0; j < 4; ++j) own += key_of(v[j]) == key && r.inside(r.action(got.index, j));
                uint64_t at = got.above + wave_running(own) - own;
                int here = -1;
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (key_of(v[j]) == key && r.inside(r.action(got.index, j)) && at++ == ties) here = r.action(got.index, j);
                end = __builtin_amdgcn_readlane(here, __ffsll((unsigned long long)__ballot(here >= 0)) - 1);
            }
        }
        if (complete && PART != SUMS) {
            __syncthreads();
            for (int i = threadIdx.x; i < parts; i += THREADS) sh.sums[i] = 0;
            __syncthreads();
            for (uint32_t i = threadIdx.x; i < listed; i += THREADS) {
                const uint64_t w = by_sum ? sh.weight[i] : weigh(value_of_key(sh.key[i]));
                if (w >= f.least && w && (sh.key[i] > key || (sh.key[i] == key && (int)sh.act[i] < end)))
                    atomicAdd(&sh.sums[((int)sh.act[i] + r.shift) / 256], (unsigned long long)w);
            }
            __syncthreads();
        }
    }
    auto stays = [&](float v, int i) {
        const uint32_t k = key_of(v);
        return k > key || (k == key && i < end);
    };
    auto enough = [&](float v) -> uint64_t {
        const uint64_t w = weigh(v);
        return w >= f.least ? w : 0;
    };
    if (PART == SUMS) {
        sum_parts(share * NW + wave, shares * NW, space[row].sums, stays, enough);
        if (share == 0 && threadIdx.x == 0) space[row].done = 1, space[row].border = key, space[row].end = end;
        return;
    }
    if (!known && !complete) sums(stays, enough);
    if (wave != 0) return;
    const uint64_t sum = total(), at = place_of(a.u[row], sum);
    const Found got = find<false>(sh.sums, parts, at);
    const f32x4 v = values_of(r.load(got.index));
    uint64_t w[4], own = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        w[j] = enough(v[j]);
        if (!stays(v[j], r.action(got.index, j))) w[j] = 0;
        own += w[j];
    }
    uint64_t run = got.above + wave_running(own) - own;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if (run <= at && at < run + w[j]) {
            a.action[row] = r.action(got.index, j);
            if (a.probability) a.probability[row] = (float)((double)w[j] / (double)sum);
        }
        run += w[j];
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
    // few rows of many actions: each shared by workgroups of 16 parts, if the workspace has the place
    int shares = (actions + 3 + 16 * 256 - 1) / (16 * 256);
    if (shares > SHARES) shares = SHARES;
    const bool shared = actions > SHARED_FROM && rows * shares <= 2 * c.cus && ctx_view(ctx, (size_t)rows * sizeof(RowSpace), c) == GORILA_OK;
    auto go = [&](auto t) {
        using T = decltype(t);
        if (threads == 64) {
            sample_wave_kernel<T><<<(unsigned)((rows + 3) / 4), 256, 0, c.stream>>>(a);
        } else if (threads == 256) {
            sample_row_kernel<T, 256, 512, 1024, 2048, WHOLE><<<(unsigned)rows, 256, 0, c.stream>>>(a, nullptr, 0);
        } else if (actions <= 65536 && !shared) {
            sample_row_kernel<T, 1024, 2048, 4096, 65536, WHOLE><<<(unsigned)rows, 1024, 0, c.stream>>>(a, nullptr, 0);
        } else if (shared) {
            RowSpace* space = (RowSpace*)c.ws;
            const unsigned blocks = (unsigned)(rows * shares);
            share_most_kernel<T><<<blocks, 1024, 0, c.stream>>>(a, space, shares);
            share_bins_kernel<T><<<blocks, 1024, 0, c.stream>>>(a, space, shares);
            share_list_kernel<T><<<blocks, 1024, 0, c.stream>>>(a, space, shares);
            sample_row_kernel<T, 1024, ALL_BINS, ALL_LIST, MAX_SAMPLE, SUMS><<<blocks, 1024, 0, c.stream>>>(a, space, shares);
            sample_row_kernel<T, 1024, ALL_BINS, ALL_LIST, MAX_SAMPLE, PICK><<<(unsigned)rows, 1024, 0, c.stream>>>(a, space, shares);
        } else {
            sample_row_kernel<T, 1024, 2048, 4096, MAX_SAMPLE, WHOLE><<<(unsigned)rows, 1024, 0, c.stream>>>(a, nullptr, 0);
        }
    };
    dtype == GORILA_F32 ? go(float{}) : go(uint16_t{});
    return launched();
}

}  // extern "C"
