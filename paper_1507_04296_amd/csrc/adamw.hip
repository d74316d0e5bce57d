// AdamW over many tensors (gorila_adamw, gorila_adamw_values).
//
// Memory bound: fp32 states move 28 bytes an element (fp32 gradients), 8-bit ones 16,
// for 20 and 60 operations.  A wave takes 256 consecutive elements, four a lane, so that
// a block of 8-bit states has its largest value in six steps over the lanes, and a
// workgroup's chunk of elements is found by its number among those of all tensors,
// which travel in the kernel's arguments: a launch for 48 tensors, and nothing to copy.
// The clock is a launch of its own, before: all workgroups read it.
//
// The Q-network's ten tensors (1.69 M elements, fp32): 10.2 us (4.6 TB/s, part of it from
// the cache) and 2.2 for the clock.  52 M elements in 8 bits, bf16 gradients, three sets in
// turn: 144 us with the clock (5.1 TB/s; a large copy, half of whose bytes are written,
// reaches 4.65), a third more with divisions, branches for the tail in every chunk and sums
// through LDS.  Their values: 99 us (5.3 TB/s).
#include "seq.h"

namespace gorila {
namespace {

constexpr int MOST = 48;      // tensors a launch (its arguments hold 4 KB)
constexpr int GROUP = 256;    // elements that share a scale
constexpr int CHUNK = 2048;   // elements a workgroup: 256 lanes of four, twice
constexpr uint64_t GOLDEN = 0x9E3779B97F4A7C15ull;

struct Tensor {
    float* theta;
    const void* grad;
    void *m, *v;
    float *m_scale, *v_scale;
    int64_t n;
    uint64_t place;  // of its first pair of elements among the random numbers
    uint32_t chunk;  // its first among the launch's
    float decay;
};
struct Tensors {
    Tensor t[MOST];
    int count;
};
static_assert(sizeof(Tensors) <= 4032, "the arguments fit a launch's");

struct Rule {
    double* clock;
    const uint8_t* keep;
    float lr, eps, beta1, beta2, rest1, rest2;
    uint64_t seed;
};

__device__ __forceinline__ uint64_t mix(uint64_t z) {  // SplitMix64's output function (Steele, Lea and Flood 2014)
    z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
    z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
    return z ^ (z >> 31);
}

__global__ void clock_kernel(double* clock, const uint8_t* keep, double beta1, double beta2) {
    if (keep && !*keep) return;
    const double t = clock[0] + 1.0;
    clock[0] = t;
    clock[1] = 1.0 - pow(beta1, t);
    clock[2] = 1.0 - pow(beta2, t);
}

// The tensor that holds the workgroup's chunk: the last one that starts at it or before.
__device__ __forceinline__ int tensor_of(const Tensors& s, uint32_t chunk) {
    int lo = 0, hi = s.count;
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (s.t[mid].chunk <= chunk) lo = mid;
        else hi = mid;
    }
    return lo;
}

// Four codes, n of which exist.
__device__ __forceinline__ uint32_t load_codes(const uint8_t* p, int n) {
    if (n >= 4) return load_any<uint32_t>(p);
    uint32_t v = 0;
#pragma unroll
    for (int j = 0; j < 3; ++j)
        if (j < n) v |= (uint32_t)p[j] << (8 * j);
    return v;
}
__device__ __forceinline__ void store_codes(uint8_t* p, uint32_t v, int n) {
    if (n >= 4) return store_any(p, v);
#pragma unroll
    for (int j = 0; j < 3; ++j)
        if (j < n) p[j] = (uint8_t)(v >> (8 * j));
}

// Codes are the upper bits of an fp32 value of 2^-31.75 (m: 2^-15.75) to 1: three bits
// of mantissa, so that a value is off by at most 1/16 of itself before chance
// decides, where linear codes would lose all small ones.
constexpr int LEAST_M = 889, LEAST_V = 761;
__device__ __forceinline__ float value_of(uint32_t code, int least, float scale) {
    const float unit = code ? __uint_as_float((code + least) << 20) : 0.0f;
    return unit * scale;
}
// size / most rounded once, for a scale that a wave shares: by its reciprocal and what the
// first quotient leaves (Markstein 1990), exact while the remainder is (quotients below
// 2^-33 are off, and held as zero anyway).  Scales outside 2^-64 .. 2^124 are divided by.
struct Scale {
    float most, inverse;
    bool far;
    __device__ __forceinline__ explicit Scale(float m) : most(m), inverse(1.0f / m), far(!(m >= 0x1p-64f && m <= 0x1p124f)) {}
    __device__ __forceinline__ float unit(float size) const {
        if (far) return most > 0.0f ? size / most : 0.0f;
        const float q = size * inverse;
        return fmaf(fmaf(-q, most, size), inverse, q);
    }
};
__device__ __forceinline__ int code_of(float unit, uint32_t chance, int least) {
    const int c = (int)((__float_as_uint(unit) + (chance << 4)) >> 20) - least;
    return c < 0 ? 0 : c;
}
// m / (sqrt(v) + eps) to three units of the last place, v from the smallest fp32 value on.  The
// reciprocal takes and gives normal numbers alone: an eps that may lie outside (ODD; a root is
// 0 or 2^-75 to 2^64) has a copy of the code that divides.
bool odd(float eps) { return (eps > 0.0f && eps < 0x1p-126f) || eps > 0x1p125f; }
template <bool ODD>
__device__ __forceinline__ float step_of(float m, float v, float eps) {
    const bool tiny = v < 0x1p-100f;
    const float root = __builtin_amdgcn_sqrtf(tiny ? v * 0x1p64f : v) * (tiny ? 0x1p-32f : 1.0f);
    return ODD ? m / (root + eps) : m * __builtin_amdgcn_rcpf(root + eps);
}
__device__ __forceinline__ float wave_max(float v) {  // of sizes
    return over_wave(v, [](float a, float b) { return fmaxf(a, b); });
}

// G: the gradients' type; BITS: the states'.
template <class G, int BITS, bool ODD>
__global__ __launch_bounds__(256) void adamw_kernel(Tensors s, Rule r) {
// m' and v' are held to the bit as the header says: products and sums are rounded apart
#pragma clang fp contract(off)
    if (r.keep && !*r.keep) return;
    const int which = tensor_of(s, blockIdx.x);
    const Tensor& t = s.t[which];
    const int64_t first = (int64_t)(blockIdx.x - t.chunk) * CHUNK;
    auto chunk = [&](auto whole) {  // a whole chunk, or any
#pragma clang fp contract(off)
        constexpr bool FULL = decltype(whole)::value;
        // all loads first: the stores between could lie anywhere, for the compiler
        constexpr int TURNS = CHUNK / 1024;
        f32x4 theta[TURNS], g[TURNS], m[TURNS], v[TURNS];
        uint32_t cm[TURNS], cv[TURNS];
        float sm[TURNS], sv[TURNS];
#pragma unroll
        for (int k = 0; k < TURNS; ++k) {
            const int64_t at = first + k * 1024 + threadIdx.x * 4, left = t.n - at;
            const int n = FULL || left > 4 ? 4 : left > 0 ? (int)left : 0;
            const int64_t p = n > 0 ? at : 0;
            theta[k] = quad_load(t.theta + p, n);
            g[k] = quad_load((const G*)t.grad + p, n);
            if (BITS == 32) {
                m[k] = quad_load((const float*)t.m + p, n);
                v[k] = quad_load((const float*)t.v + p, n);
            } else {
                cm[k] = load_codes((const uint8_t*)t.m + p, n);
                cv[k] = load_codes((const uint8_t*)t.v + p, n);
                sm[k] = n > 0 ? t.m_scale[p / GROUP] : 0.0f;
                sv[k] = n > 0 ? t.v_scale[p / GROUP] : 0.0f;
            }
        }
        const float c1 = 1.0f / (float)r.clock[1], c2 = 1.0f / (float)r.clock[2];
        const uint64_t key = BITS == 8 ? mix(r.seed + (uint64_t)(int64_t)r.clock[0] * GOLDEN) : 0;
#pragma unroll
        for (int k = 0; k < TURNS; ++k) {
            const int64_t at = first + k * 1024 + threadIdx.x * 4, left = t.n - at;
            const int n = FULL || left > 4 ? 4 : left > 0 ? (int)left : 0;
            if (!FULL && __ballot(n > 0) == 0) break;
            const int64_t p = n > 0 ? at : 0;
            if (BITS == 8) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t c = cm[k] >> (8 * j) & 255u;
                    const float size = value_of(c & 127u, LEAST_M, sm[k]);
                    m[k][j] = c & 128u ? -size : size;
                    v[k][j] = value_of(cv[k] >> (8 * j) & 255u, LEAST_V, sv[k]);
                }
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                m[k][j] = r.beta1 * m[k][j] + r.rest1 * g[k][j];
                v[k][j] = r.beta2 * v[k][j] + r.rest2 * (g[k][j] * g[k][j]);
                theta[k][j] = theta[k][j] - r.lr * (t.decay * theta[k][j] + step_of<ODD>(m[k][j] * c1, v[k][j] * c2, r.eps));
            }
            quad_store(t.theta + p, theta[k], n);
            if (BITS == 32) {
                quad_store((float*)t.m + p, m[k], n);
                quad_store((float*)t.v + p, v[k], n);
            } else {
                float mm = 0.0f, mv = 0.0f, bad_m = 0.0f, bad_v = 0.0f;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (j >= n) m[k][j] = v[k][j] = 0.0f;
                    mm = fmaxf(mm, fabsf(m[k][j])), mv = fmaxf(mv, v[k][j]);
                    bad_m += m[k][j] * 0.0f, bad_v += v[k][j] * 0.0f;
                }
                mm = wave_max(bad_m == bad_m ? mm : INFINITY);
                mv = wave_max(bad_v == bad_v ? mv : INFINITY);
                const Scale scale_m(mm), scale_v(mv);
                uint32_t new_m = 0, new_v = 0;
                const uint64_t pair = t.place + (uint64_t)p / 2;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint64_t z = mix(key + (pair + h + 1) * GOLDEN);
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const int j = 2 * h + i;
                        const uint32_t chance = (uint32_t)(z >> (32 * i));
                        uint32_t a = code_of(scale_m.unit(fabsf(m[k][j])), chance & 0xffffu, LEAST_M), b = code_of(scale_v.unit(v[k][j]), chance >> 16, LEAST_V);
                        if (v[k][j] > 0.0f && b == 0) b = 1;
                        if (m[k][j] < 0.0f) a |= 128u;
                        if (mm == INFINITY) a = 0;
                        if (mv == INFINITY) b = 0;
                        new_m |= a << (8 * j), new_v |= b << (8 * j);
                    }
                }
                store_codes((uint8_t*)t.m + p, new_m, n);
                store_codes((uint8_t*)t.v + p, new_v, n);
                if (n > 0 && (threadIdx.x & 63) == 0) {
                    t.m_scale[p / GROUP] = mm == INFINITY ? NAN : mm;
                    t.v_scale[p / GROUP] = mv == INFINITY ? NAN : mv;
                }
            }
        }
    };
    if (first + CHUNK <= t.n) chunk(std::true_type{});
    else chunk(std::false_type{});
}

// theta and grad: where m's and v's values go.
__global__ __launch_bounds__(256) void values_kernel(Tensors s) {
    const int which = tensor_of(s, blockIdx.x);
    const Tensor& t = s.t[which];
    const int64_t first = (int64_t)(blockIdx.x - t.chunk) * CHUNK;
#pragma unroll
    for (int k = 0; k < CHUNK / 1024; ++k) {
        const int64_t p = first + k * 1024 + threadIdx.x * 4, left = t.n - p;
        if (left <= 0) return;
        const int n = left > 4 ? 4 : (int)left;
        const uint32_t cm = load_codes((const uint8_t*)t.m + p, n), cv = load_codes((const uint8_t*)t.v + p, n);
        const float sm = t.m_scale[p / GROUP], sv = t.v_scale[p / GROUP];
        f32x4 m, v;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t c = cm >> (8 * j) & 255u;
            const float size = value_of(c & 127u, LEAST_M, sm);
            m[j] = c & 128u ? -size : size;
            v[j] = value_of(cv >> (8 * j) & 255u, LEAST_V, sv);
        }
        quad_store(t.theta + p, m, n);
        quad_store((float*)t.grad + p, v, n);
    }
}

// ---- host ----

// Calls launch(tensors, chunks) for the tensors that have elements, MOST or as many chunks
// as a launch holds at a time; fill(from, i, t) sets the addresses.
template <class F, class L>
void by_launch(const gorila_adamw_tensor* tensors, int count, F&& fill, L&& launch) {
    Tensors s{};
    uint64_t chunks = 0, place = 0;
    auto flush = [&] {
        if (s.count) launch(s, (unsigned)chunks);
        s.count = 0, chunks = 0;
    };
    for (int i = 0; i < count; ++i) {
        const int64_t n = tensors[i].n;
        const uint64_t need = (uint64_t)(n + CHUNK - 1) / CHUNK;
        if (need > 0) {
            if (s.count == MOST || !launch_fits((double)(chunks + need), 256)) flush();
            Tensor& t = s.t[s.count];
            t.n = n, t.place = place, t.chunk = (uint32_t)chunks, t.decay = tensors[i].decay;
            fill(tensors[i], i, t);
            ++s.count;
            chunks += need;
        }
        place += (uint64_t)(n + GROUP - 1) / GROUP * (GROUP / 2);
    }
    flush();
}

int check_count(const gorila_adamw_tensor* tensors, int count) {
    if (count < 0 || (count > 0 && !tensors)) return GORILA_EINVAL;
    for (int i = 0; i < count; ++i)
        if (tensors[i].n < 0) return GORILA_EINVAL;
    if (count > GORILA_ADAMW_MAX_TENSORS) return GORILA_EUNSUPPORTED;
    for (int i = 0; i < count; ++i)
        if (!launch_fits((double)((tensors[i].n + CHUNK - 1) / CHUNK), 256)) return GORILA_EUNSUPPORTED;
    return GORILA_OK;
}
// What 8-bit states need of a tensor with elements.
bool held8(const gorila_adamw_tensor& t) { return t.m && t.v && t.m_scale && t.v_scale && at_element(t.m_scale, 4) && at_element(t.v_scale, 4); }

}  // namespace
}  // namespace gorila

using namespace gorila;

extern "C" {

int gorila_adamw(const gorila_adamw_tensor* tensors, int32_t count, int32_t grad_dtype, int32_t state_bits, double* clock,
                 const uint8_t* keep, float lr, double beta1, double beta2, float eps, uint64_t seed, gorila_ctx* ctx) {
    CtxView c;
    int rc = ctx_view(ctx, 0, c);
    if (rc || (rc = check_count(tensors, count))) return rc;
    if (!row_dtype(grad_dtype) || (state_bits != 8 && state_bits != 32) || !clock || !at_element(clock, 8)) return GORILA_EINVAL;
    if (!(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0) || !(eps >= 0.0f && eps < INFINITY) || !(lr >= 0.0f && lr < INFINITY))
        return GORILA_EINVAL;
    const int e = dtype_bytes(grad_dtype);
    for (int i = 0; i < count; ++i) {
        const gorila_adamw_tensor& t = tensors[i];
        if (t.n == 0) continue;
        if (!t.theta || !t.grad || !t.m || !t.v || !at_element(t.theta, 4) || !at_element(t.grad, e)) return GORILA_EINVAL;
        if (state_bits == 8 ? !held8(t) : !at_element(t.m, 4) || !at_element(t.v, 4)) return GORILA_EINVAL;
    }
    Rule r{clock, keep, lr, eps, (float)beta1, (float)beta2, (float)(1.0 - beta1), (float)(1.0 - beta2), seed};
    clock_kernel<<<1, 1, 0, c.stream>>>(clock, keep, beta1, beta2);
    by_launch(
        tensors, count,
        [&](const gorila_adamw_tensor& from, int, Tensor& t) {
            t.theta = from.theta, t.grad = from.grad, t.m = from.m, t.v = from.v, t.m_scale = from.m_scale, t.v_scale = from.v_scale;
        },
        [&](const Tensors& s, unsigned chunks) {
            auto go = [&](auto g, auto bits, auto odd_eps) {
                adamw_kernel<decltype(g), decltype(bits)::value, decltype(odd_eps)::value><<<chunks, 256, 0, c.stream>>>(s, r);
            };
            auto by_bits = [&](auto g, auto odd_eps) {
                using std::integral_constant;
                if (state_bits == 32) go(g, integral_constant<int, 32>{}, odd_eps);
                else go(g, integral_constant<int, 8>{}, odd_eps);
            };
            auto by_type = [&](auto odd_eps) { grad_dtype == GORILA_F32 ? by_bits(float{}, odd_eps) : by_bits(uint16_t{}, odd_eps); };
            odd(eps) ? by_type(std::true_type{}) : by_type(std::false_type{});
        });
    return launched();
}

int gorila_adamw_values(const gorila_adamw_tensor* tensors, int32_t count, float* const* m_out, float* const* v_out, gorila_ctx* ctx) {
    CtxView c;
    int rc = ctx_view(ctx, 0, c);
    if (rc || (rc = check_count(tensors, count))) return rc;
    if (count > 0 && (!m_out || !v_out)) return GORILA_EINVAL;
    for (int i = 0; i < count; ++i)
        if (tensors[i].n > 0 && (!held8(tensors[i]) || !m_out[i] || !v_out[i] || !at_element(m_out[i], 4) || !at_element(v_out[i], 4)))
            return GORILA_EINVAL;
    by_launch(
        tensors, count,
        [&](const gorila_adamw_tensor& from, int i, Tensor& t) {
            t.m = from.m, t.v = from.v, t.m_scale = from.m_scale, t.v_scale = from.v_scale, t.theta = m_out[i], t.grad = v_out[i];
        },
        [&](const Tensors& s, unsigned chunks) { values_kernel<<<chunks, 256, 0, c.stream>>>(s); });
    return launched();
}

}  // extern "C"
