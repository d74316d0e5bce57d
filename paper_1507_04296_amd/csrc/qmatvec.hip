// Products with 4-bit weights and group scales (gorila_quantize_weights,
// gorila_qmatvec).
//
// With few rows the codes are what has to be read, once, at the rate of the memory;
// everything else has to stay below that.  Products run on the matrix unit also for
// one row: there a run of 32 codes costs one instruction, and what is left for the
// vector unit is turning codes into operands, one instruction a code.
//
// A wave takes 16 outputs and 128 codes of each at a time.  Its operands
// want lane l to hold row l % 16, but loaded that way every lane of a load is in a
// line of its own, and the address unit takes a line a cycle (one load of scales:
// 69 cycles of a compute unit).  So loads run along the rows, four lanes a row's 64
// bytes of codes, and pass through the wave's own part of LDS, quads swapped by row
// so that neither side meets a bank twice.  Lanes 16 apart then exchange quarters of
// their codes, so that each instruction reduces over one run of 32, in one group.
//
// Code c as bf16 is 1 + c / 16 = 0x3f80 | c << 3: the weight is 16 (that - 1.5), and
// the sum of 1.5 x comes from the same instruction with a constant operand.  (128 + c
// needs no shifts, but its sums cancel 30 times their rounding instead of 5.)  fp32
// rows are three exact bf16 terms, bf16 rows one; 8-bit rows take the integer
// instruction, whose sums are exact, with c and 8.
//
// The waves of a workgroup share the outputs and split the inputs; their sums are
// added in LDS, in order.
#include "planes.h"
#include "seq.h"

namespace gorila {
namespace {

struct MatvecView {
    const void* x;
    int64_t xs, rows;
    const float* x_scale;
    const uint8_t* codes;
    const float* scales;
    int outputs, inputs, group, chunks, groups;  // chunks: runs of 32 codes a row
    void* y;
};

// Element (lane group g, register j) to (group j, register g); a group is 16 lanes.
__device__ __forceinline__ void transpose_groups(uint32_t (&r)[4]) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const auto v = __builtin_amdgcn_permlane32_swap(r[i], r[i + 2], false, false);
        r[i] = v[0];
        r[i + 2] = v[1];
    }
#pragma unroll
    for (int i = 0; i < 4; i += 2) {
        const auto v = __builtin_amdgcn_permlane16_swap(r[i], r[i + 1], false, false);
        r[i] = v[0];
        r[i + 1] = v[1];
    }
}

// Eight inputs a lane (row l % 16, inputs 8 (l / 16) .. +7 of a run) as operands, in
// the order that the codes' side has them, and the codes' side.
template <class T> struct Side {  // fp32 and bf16
    static constexpr int NP = std::is_same<T, float>::value ? 3 : 1;
    typedef f32x4 Acc;
    struct X { bf16x8 p[NP]; };
    struct W { bf16x8 v; };
    // from LDS; order: 0 4 1 5 2 6 3 7
    static __device__ __forceinline__ X operand(const uint4* row, int piece, int swap) {
        X o;
        if constexpr (NP == 1) {
            constexpr uint32_t LOW = 0x05040100u, HIGH = 0x07060302u;
            const uint4 r = row[piece ^ swap];
            const uint4 q{__builtin_amdgcn_perm(r.z, r.x, LOW), __builtin_amdgcn_perm(r.z, r.x, HIGH),
                          __builtin_amdgcn_perm(r.w, r.y, LOW), __builtin_amdgcn_perm(r.w, r.y, HIGH)};
            o.p[0] = __builtin_bit_cast(bf16x8, q);
        } else {
            const f32x4 a = __builtin_bit_cast(f32x4, row[(2 * piece) ^ swap]), b = __builtin_bit_cast(f32x4, row[(2 * piece + 1) ^ swap]);
            const f32x4 lo{a[0], b[0], a[1], b[1]}, hi{a[2], b[2], a[3], b[3]};
            bf16x4 l[NP], h[NP];
            split4<NP>(lo, l);
            split4<NP>(hi, h);
#pragma unroll
            for (int i = 0; i < NP; ++i) o.p[i] = __builtin_shufflevector(l[i], h[i], 0, 1, 2, 3, 4, 5, 6, 7);
        }
        return o;
    }
    static __device__ __forceinline__ W weights(uint32_t q) {
        constexpr uint32_t M = 0x00780078u, ONE = 0x3f803f80u;
        const uint4 v{(q << 3 & M) | ONE, (q >> 1 & M) | ONE, (q >> 5 & M) | ONE, (q >> 9 & M) | ONE};
        return W{__builtin_bit_cast(bf16x8, v)};
    }
    static __device__ __forceinline__ W offset() {
        constexpr uint32_t C = 0xbfc0bfc0u;  // -1.5
        return W{__builtin_bit_cast(bf16x8, uint4{C, C, C, C})};
    }
    static __device__ __forceinline__ Acc mul(const X& x, const W& w, Acc c) {
#pragma unroll
        for (int i = NP - 1; i >= 0; --i) c = mfma16(x.p[i], w.v, c);
        return c;
    }
    static __device__ __forceinline__ f32x4 sum(Acc a, Acc off) { return (a + off) * 16.0f; }
};
template <> struct Side<int8_t> {
    typedef i32x4 Acc;
    struct X { long v; };
    struct W { long v; };
    // order: 0 2 4 6 1 3 5 7
    static __device__ __forceinline__ X operand(const uint4* row, int piece, int swap) {
        const uint2 r = ((const uint2*)(row + ((piece >> 1) ^ swap)))[piece & 1];
        return X{pack(__builtin_amdgcn_perm(r.y, r.x, 0x06040200u), __builtin_amdgcn_perm(r.y, r.x, 0x07050301u))};
    }
    static __device__ __forceinline__ W weights(uint32_t q) { return W{pack(q & 0x0f0f0f0fu, q >> 4 & 0x0f0f0f0fu)}; }
    static __device__ __forceinline__ W offset() { return W{pack(0xf8f8f8f8u, 0xf8f8f8f8u)}; }  // -8
    static __device__ __forceinline__ Acc mul(const X& x, const W& w, Acc c) { return __builtin_amdgcn_mfma_i32_16x16x32_i8(x.v, w.v, c, 0, 0, 0); }
    static __device__ __forceinline__ f32x4 sum(Acc a, Acc off) {
        a += off;
        return f32x4{(float)a[0], (float)a[1], (float)a[2], (float)a[3]};
    }
    static __device__ __forceinline__ long pack(uint32_t a, uint32_t b) { return (long)((uint64_t)b << 32 | a); }
};

// 16 bytes of a row's inputs, of which the first n elements are there.
template <bool VEC, class T>
__device__ __forceinline__ uint4 input_quad(const T* p, int n) {
    constexpr int E = 16 / sizeof(T);
    if (VEC && n >= E) return *(const uint4*)p;
    T v[E];
#pragma unroll
    for (int i = 0; i < E; ++i) v[i] = i < n ? p[i] : (T)0;
    uint4 r;
    __builtin_memcpy(&r, v, 16);
    return r;
}

// A sum as it stands for y: itself, or where it is no number, formed term by term in 64
// bits.  The kernels add code x and -8 x apart, which are infinities of both signs for an
// infinite x or past fp32's range for a large one, and multiply the zeros past a row's end
// with its last scale.  Slow, and for such rows alone; the view (both kernels' first
// argument) is read again here, or it would be kept in scalar registers that the main
// loops need (fp32, 64 rows and more: 1.5 % of the time, this way 0.9).
template <class T>
__device__ __forceinline__ float sum_of(float sum, int64_t row, int out) {
    if (__builtin_expect(fabsf(sum) < INFINITY, 1)) return sum;
    uint64_t args = (uint64_t)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(args));
    const MatvecView s = *(const MatvecView*)args;
    const T* x = (const T*)s.x + row * s.xs;
    const uint8_t* codes = s.codes + (int64_t)out * s.chunks * 16;
    const float* scales = s.scales + (int64_t)out * s.groups;
    const int shift = s.group == 32 ? 5 : s.group == 64 ? 6 : 7;
    double v = 0.0;
#pragma unroll 1
    for (int k = 0; k < s.inputs; ++k)
        v += (double)row_value(x[k]) * ((double)scales[k >> shift] * (double)((codes[k >> 1] >> (4 * (k & 1)) & 15) - 8));
    return (float)v;
}

constexpr int SUPER = 4;  // runs of 32 codes that a wave takes together
// Of those, loaded together.  (All of them are waited for before the first product: `raw`
// is indexed in a loop that breaks off, so the compiler keeps it in scratch memory, 80
// bytes a lane.)
constexpr int AHEAD = 4;

// What a wave has in LDS, and how many waves a workgroup has at most (one of 150 KB
// of LDS takes 1.5 us longer to start than one of 40).
template <class T, int RT> struct Part {
    uint4 codes[64];                           // [row][quad, swapped by row]
    float scales[64];                          // [row][4]
    uint4 x[RT][16][SUPER * 2 * sizeof(T)];    // [row][quad, swapped by row]
};
template <class T, int RT>
constexpr int most_waves() { return sizeof(Part<T, RT>) * 8 <= 80 * 1024 ? 8 : 4; }

// RT: tiles of 16 rows.  Lanes of outputs that are not there take the last one's and
// store nothing.
template <class T, int RT, bool VEC>
__global__ __launch_bounds__((64 * most_waves<T, RT>())) void matvec_kernel(MatvecView s) {
    using S = Side<T>;
    constexpr int WAVES = most_waves<T, RT>(), XQ = SUPER * 2 * sizeof(T);  // quads a row
    constexpr int ROWS = 64 / XQ, XL = 16 / ROWS;                           // rows a load, loads a tile
    union Lds {
        Part<T, RT> part[WAVES];
        float sums[WAVES][RT][256];
    };
    __shared__ __align__(16) Lds lds;
    const int l = threadIdx.x & 63, lc = l & 15, lg = l >> 4;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;  // the same in a wave
    Part<T, RT>& own = lds.part[w];
    const int o0 = blockIdx.x * 16;
    const int64_t r0 = (int64_t)blockIdx.y * 16 * RT;
    const int supers = (s.chunks + SUPER - 1) / SUPER, per = (supers + waves - 1) / waves;
    const int u0 = w * per, u1 = u0 + per < supers ? u0 + per : supers;
    const int shift = s.group == 32 ? 0 : s.group == 64 ? 1 : 2, last = (1 << shift) - 1;  // runs a group
    f32x4 acc[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) acc[r] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    // this lane's places in the loads: a quarter of an output's codes and scales, a quad
    // of a row's inputs
    const int quarter = l & 3, put = (l & ~3) | (quarter ^ (l >> 4));  // row l / 4, swapped by row / 4
    const int64_t at_out = o0 + (l >> 2) < s.outputs ? o0 + (l >> 2) : s.outputs - 1;
    const uint8_t* codes = s.codes + at_out * s.chunks * 16;
    const float* scales = s.scales + at_out * s.groups;
    const int xq = l % XQ, xr = l / XQ;

    struct In {
        uint4 x[RT][XL];
        float sc;
    };
    auto load_in = [&](int u, In& in) {
        const int k = u * SUPER * 32 + xq * (int)(16 / sizeof(T)), n = s.inputs - k;
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int i = 0; i < XL; ++i) {
                const int64_t row = r0 + 16 * r + ROWS * i + xr;
                in.x[r][i] = uint4{0, 0, 0, 0};
                if (row < s.rows && n > 0) in.x[r][i] = input_quad<VEC>((const T*)s.x + row * s.xs + k, n);
            }
        const int g = (u * SUPER >> shift) + quarter;
        in.sc = scales[g < s.groups ? g : s.groups - 1];  // past the end: times sums of zeros
    };
    auto products = [&](const uint4& raw, const In& in) {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // what was read is read
        __builtin_amdgcn_wave_barrier();
        own.codes[put] = raw;
        own.scales[l] = in.sc;
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int i = 0; i < XL; ++i) {
                const int row = ROWS * i + xr;
                own.x[r][row][xq ^ (row & (XQ - 1))] = in.x[r][i];
            }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        const uint4 v = own.codes[4 * lc + (lg ^ (lc >> 2))];
        uint32_t q[4] = {v.x, v.y, v.z, v.w};
        transpose_groups(q);
        typename S::Acc part[RT], off[RT];
#pragma unroll
        for (int j = 0; j < SUPER; ++j) {
            const typename S::W wt = S::weights(q[j]);
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                if ((j & last) == 0) part[r] = off[r] = typename S::Acc{0, 0, 0, 0};
                const typename S::X x = S::operand(own.x[r][lc], 4 * j + lg, lc & (XQ - 1));
                off[r] = S::mul(x, S::offset(), off[r]);
                part[r] = S::mul(x, wt, part[r]);
            }
            if ((j & last) == last) {
                const float sc = own.scales[4 * lc + (j >> shift)];
#pragma unroll
                for (int r = 0; r < RT; ++r) acc[r] += S::sum(part[r], off[r]) * sc;
            }
        }
    };
    for (int ub = u0; ub < u1; ub += AHEAD) {
        uint4 raw[AHEAD];
#pragma unroll
        for (int d = 0; d < AHEAD; ++d) {
            const int u = ub + d < u1 ? ub + d : u1 - 1;
            const int c = u * SUPER + quarter;
            raw[d] = *(const uint4*)(codes + (int64_t)(c < s.chunks ? c : s.chunks - 1) * 16);  // past the end: times zeros
        }
        In in[2];
        load_in(ub, in[0]);
#pragma unroll
        for (int d = 0; d < AHEAD; ++d) {
            if (ub + d >= u1) break;
            if (d + 1 < AHEAD && ub + d + 1 < u1) load_in(ub + d + 1, in[(d + 1) & 1]);
            products(raw[d], in[d & 1]);
        }
    }
    __syncthreads();
    // rows 4 (l / 16) + e, output l % 16 of a tile
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int e = 0; e < 4; ++e) lds.sums[w][r][(4 * lg + e) * 16 + lc] = acc[r][e];
    __syncthreads();
    for (int e = threadIdx.x; e < RT * 256; e += blockDim.x) {
        const int out = o0 + e % 16;
        const int64_t row = r0 + e / 16;
        if (out >= s.outputs || row >= s.rows) continue;
        float v = 0.0f;
        for (int i = 0; i < waves; ++i) v += lds.sums[i][e / 256][e % 256];
        const int64_t at = row * s.outputs + out;
        if constexpr (std::is_same<T, int8_t>::value) ((float*)s.y)[at] = v * s.x_scale[row];
        else ((T*)s.y)[at] = row_round<T>(sum_of<T>(v, row, out));
    }
}

// ---- one and two rows, and up to four 8-bit ones ----
//
// A lane takes one run of 32 codes of a row of weights and keeps the inputs they meet
// in registers over all its outputs, so that a load of codes (16 bytes a lane, a
// kilobyte in one piece a wave) is all that an output costs beside the products.  fp32:
// a code costs its conversion and one multiply-add a row, counts as 0 .. 15, and 8
// times the sum of the inputs comes off; bf16: pairs as above in dot products of two;
// 8-bit rows: integer dot products of four.  8192 x 8192, one row: fp32 15.2 us, bf16
// 13.6, 8-bit 9.4 (the matrix unit's kernel 38, 30 and 22: its operands cost the
// vector unit more than these products; what the three differ by is the work of a
// code); four rows bf16 37.7, and 20.7 there.

// Inputs of a lane's run, as the products take them, and the sum that the offset costs.
template <class T> struct Run {
    float v[32], off;
    template <bool VEC>
    __device__ __forceinline__ void load(const T* p, int n) {
        float sum = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const f32x4 a = row_load<VEC>(p + (n > 4 * j ? 4 * j : 0), n - 4 * j);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[4 * j + i] = a[i];
            sum += (a[0] + a[1]) + (a[2] + a[3]);
        }
        off = -8.0f * sum;
    }
};
template <> struct Run<uint16_t> {
    bf16x2 v[16];  // of each eight 0 4, 1 5, 2 6, 3 7
    float off;
    template <bool VEC>
    __device__ __forceinline__ void load(const uint16_t* p, int n) {
        float sum = 0.0f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const f32x4 a = row_load<VEC>(p + (n > 8 * j ? 8 * j : 0), n - 8 * j);
            const f32x4 b = row_load<VEC>(p + (n > 8 * j + 4 ? 8 * j + 4 : 0), n - 8 * j - 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) {  // exact: they were bf16
                const uint32_t u = __builtin_amdgcn_perm(__float_as_uint(b[i]), __float_as_uint(a[i]), 0x07060302u);
                v[4 * j + i] = __builtin_bit_cast(bf16x2, u);
            }
            sum += ((a[0] + a[1]) + (a[2] + a[3])) + ((b[0] + b[1]) + (b[2] + b[3]));
        }
        off = -1.5f * sum;
    }
};
template <> struct Run<int8_t> {
    int even[4], odd[4], off;
    template <bool VEC>
    __device__ __forceinline__ void load(const int8_t* p, int n) {
        int sum = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            uint32_t a = 0, b = 0;
            if (VEC && n >= 8 * j + 8) {
                const uint2 u = *(const uint2*)(p + 8 * j);
                a = u.x, b = u.y;
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (8 * j + i < n) a |= (uint32_t)(uint8_t)p[8 * j + i] << (8 * i);
                    if (8 * j + 4 + i < n) b |= (uint32_t)(uint8_t)p[8 * j + 4 + i] << (8 * i);
                }
            }
            even[j] = (int)__builtin_amdgcn_perm(b, a, 0x06040200u);
            odd[j] = (int)__builtin_amdgcn_perm(b, a, 0x07050301u);
            sum = __builtin_amdgcn_sdot4(even[j], 0x01010101, sum, false);
            sum = __builtin_amdgcn_sdot4(odd[j], 0x01010101, sum, false);
        }
        off = -8 * sum;
    }
};

// Sum over the lk lanes of a team (4 .. 64, all of them get it).
__device__ __forceinline__ float team_sum(float v, int lk) {
    auto with = [&](auto ctrl) {
        const int o = __builtin_amdgcn_update_dpp(0, __float_as_int(v), decltype(ctrl)::value, 0xf, 0xf, true);
        v += __int_as_float(o);
    };
    with(std::integral_constant<int, 0xb1>{});              // lanes swapped in pairs
    with(std::integral_constant<int, 0x4e>{});              // pairs in fours
    if (lk > 4) with(std::integral_constant<int, 0x141>{});  // eight mirrored
    if (lk > 8) with(std::integral_constant<int, 0x140>{});  // sixteen mirrored
    if (lk > 16) v += __shfl_xor(v, 16, 64);
    if (lk > 32) v += __shfl_xor(v, 32, 64);
    return v;
}

constexpr int FEW_WAVES = 8;
// Outputs a team takes at a time: what the registers hold beside R rows' inputs.
constexpr int few_outputs(int r) { return r == 4 ? 2 : 4; }

// A wave's lanes form 64 / lk teams of lk lanes; a team takes `batches` times OUT
// outputs, its lanes and those of the other waves the runs of the row in turn.
template <class T, int R, bool VEC>
__global__ __launch_bounds__(64 * FEW_WAVES) void few_rows_kernel(MatvecView s, int lk, int batches) {
    constexpr int OUT = few_outputs(R);
    __shared__ float sums[FEW_WAVES][R * OUT * 16];  // [wave][row, output, team]
    const int l = threadIdx.x & 63, k = l % lk, team = l / lk, teams = 64 / lk;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    const int shift = s.group == 32 ? 0 : s.group == 64 ? 1 : 2;  // runs a group
    const int c0 = w * lk + k, pass = waves * lk, passes = (s.chunks + pass - 1) / pass;
    const int first = (int)blockIdx.x * teams * batches * OUT;  // output of batch 0, team 0
    struct Weights {
        uint4 q[OUT];
        float sc[OUT];
    };
    auto load = [&](int batch, int p, Weights& g) {
        const int c = c0 + p * pass < s.chunks ? c0 + p * pass : s.chunks - 1;  // past the end: times zeros
#pragma unroll
        for (int o = 0; o < OUT; ++o) {
            const int out = first + (batch * teams + team) * OUT + o;
            const int64_t at = out < s.outputs ? out : s.outputs - 1;
            g.q[o] = *(const uint4*)(s.codes + (at * s.chunks + c) * 16);
            g.sc[o] = s.scales[at * s.groups + (c >> shift)];
        }
    };
    Run<T> x[R];
    auto load_x = [&](int p) {
        const int c = c0 + p * pass, n = s.inputs - c * 32;
#pragma unroll
        for (int r = 0; r < R; ++r) x[r].template load<VEC>((const T*)s.x + (r < s.rows ? r : 0) * s.xs + (n > 0 ? c * 32 : 0), n);
    };
    Weights now, next;
    load(0, 0, now);
    load_x(0);
    for (int batch = 0; batch < batches; ++batch) {
        float acc[R][OUT];
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int o = 0; o < OUT; ++o) acc[r][o] = 0.0f;
        for (int p = 0; p < passes; ++p) {
            const bool more = p + 1 < passes || batch + 1 < batches;
            if (more) load(p + 1 < passes ? batch : batch + 1, p + 1 < passes ? p + 1 : 0, next);
#pragma unroll
            for (int o = 0; o < OUT; ++o) {
                const uint32_t qs[4] = {now.q[o].x, now.q[o].y, now.q[o].z, now.q[o].w};
                if constexpr (std::is_same<T, int8_t>::value) {
                    int d[R];
#pragma unroll
                    for (int r = 0; r < R; ++r) d[r] = x[r].off;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int even = (int)(qs[j] & 0x0f0f0f0fu), odd = (int)(qs[j] >> 4 & 0x0f0f0f0fu);
#pragma unroll
                        for (int r = 0; r < R; ++r) d[r] = __builtin_amdgcn_sdot4(x[r].odd[j], odd, __builtin_amdgcn_sdot4(x[r].even[j], even, d[r], false), false);
                    }
#pragma unroll
                    for (int r = 0; r < R; ++r) acc[r][o] = fmaf((float)d[r], now.sc[o], acc[r][o]);
                } else if constexpr (std::is_same<T, uint16_t>::value) {
                    float d[R];
#pragma unroll
                    for (int r = 0; r < R; ++r) d[r] = x[r].off;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const typename Side<T>::W wt = Side<T>::weights(qs[j]);
                        const uint4 pairs = __builtin_bit_cast(uint4, wt.v);
                        const uint32_t pr[4] = {pairs.x, pairs.y, pairs.z, pairs.w};
#pragma unroll
                        for (int i = 0; i < 4; ++i)
#pragma unroll
                            for (int r = 0; r < R; ++r) d[r] = __builtin_amdgcn_fdot2_f32_bf16(x[r].v[4 * j + i], __builtin_bit_cast(bf16x2, pr[i]), d[r], false);
                    }
#pragma unroll
                    for (int r = 0; r < R; ++r) acc[r][o] = fmaf(16.0f * d[r], now.sc[o], acc[r][o]);
                } else {
                    float d[R];
#pragma unroll
                    for (int r = 0; r < R; ++r) d[r] = x[r].off;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const uint32_t even = qs[j] & 0x0f0f0f0fu, odd = qs[j] >> 4 & 0x0f0f0f0fu;
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float ce = (float)(even >> (8 * i) & 255u), co = (float)(odd >> (8 * i) & 255u);
#pragma unroll
                            for (int r = 0; r < R; ++r) d[r] = fmaf(co, x[r].v[8 * j + 2 * i + 1], fmaf(ce, x[r].v[8 * j + 2 * i], d[r]));
                        }
                    }
#pragma unroll
                    for (int r = 0; r < R; ++r) acc[r][o] = fmaf(d[r], now.sc[o], acc[r][o]);
                }
            }
            now = next;
            if (passes > 1 && more) load_x(p + 1 < passes ? p + 1 : 0);
        }
        if (batch > 0) __syncthreads();  // the sums of the batch before are read
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int o = 0; o < OUT; ++o) {
                const float v = team_sum(acc[r][o], lk);
                if (k == 0) sums[w][(r * OUT + o) * teams + team] = v;
            }
        __syncthreads();
        for (int e = threadIdx.x; e < R * OUT * teams; e += blockDim.x) {
            const int r = e / teams / OUT, out = first + (batch * teams + e % teams) * OUT + e / teams % OUT;
            if (r >= s.rows || out >= s.outputs) continue;
            float v = 0.0f;
            for (int i = 0; i < waves; ++i) v += sums[i][e];
            const int64_t at = (int64_t)r * s.outputs + out;
            if constexpr (std::is_same<T, int8_t>::value) ((float*)s.y)[at] = v * s.x_scale[r];
            else ((T*)s.y)[at] = row_round<T>(sum_of<T>(v, r, out));
        }
    }
}

// A lane takes four weights; the lanes of a group find its largest together.
template <class T, bool VEC>
__global__ __launch_bounds__(256) void quantize_kernel(const T* w, int64_t ws, int outputs, int inputs, int group, int chunks,
                                                       int groups, uint8_t* codes, float* scales) {
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int per = groups * (group / 4);  // lanes a row, whole groups
    const int64_t row = id / per;
    const int k = (int)(id % per) * 4, lanes = group / 4;
    const bool on = row < outputs;
    f32x4 v = row_load<VEC>(w + (on && k < inputs ? row * ws + k : 0), on ? inputs - k : 0);
    float most = 0.0f, bad = 0.0f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        most = fmaxf(most, fabsf(v[j]));
        bad += v[j] * 0.0f;
    }
    if (bad != bad) most = INFINITY;
    for (int m = lanes >> 1; m; m >>= 1) most = fmaxf(most, __shfl_xor(most, m, 64));
    if (!on) return;
    const bool fine = most < INFINITY;
    if (k % group == 0) scales[row * groups + k / group] = fine ? most / 7.0f : NAN;
    if (k >= chunks * 32) return;  // past the row's codes
    if (most < TINY) v *= TINY_UP, most *= TINY_UP;
    const float inv = most > 0.0f && fine ? 7.0f / most : 0.0f;
    uint32_t q = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) q |= (uint32_t)(8 + (fine ? (int)rintf(v[j] * inv) : 0)) << (4 * j);
    *(uint16_t*)(codes + row * chunks * 16 + k / 2) = (uint16_t)q;
}

// Inputs and outputs whose sums with a workgroup's are 32 bits: the lanes of eight waves
// take a run of 32 inputs each at a time, a team 8 batches of 64 outputs.
constexpr int MAX_INPUTS = INT32_MAX - 32 * (64 * FEW_WAVES + 1), MAX_OUTPUTS = INT32_MAX - 512;
bool group_size(int g) { return g == 32 || g == 64 || g == 128; }

}  // namespace
}  // namespace gorila

using namespace gorila;

extern "C" {

int gorila_quantize_weights(const void* weights, int64_t weights_stride, int32_t outputs, int32_t inputs, int32_t dtype,
                            int32_t group, uint8_t* codes, float* scales, gorila_ctx* ctx) {
    CtxView c;
    const int rc = ctx_view(ctx, 0, c);
    if (rc) return rc;
    if (!row_dtype(dtype) || outputs < 0 || inputs < 1 || !group_size(group)) return GORILA_EINVAL;
    if (inputs > MAX_INPUTS) return GORILA_EUNSUPPORTED;
    if (outputs == 0) return GORILA_OK;
    const int e = dtype_bytes(dtype);
    if (!weights || !codes || !scales || !at_element(weights, e) || !aligned16(codes) || !at_element(scales, 4)) return GORILA_EINVAL;
    const int chunks = (inputs + 31) / 32, groups = (inputs + group - 1) / group;
    const int64_t lanes = (int64_t)outputs * groups * (group / 4);
    if (!launch_fits((double)lanes + 255, 1)) return GORILA_EUNSUPPORTED;
    const bool vec = !((weights_stride | inputs) & 3) && at_four(weights, e);
    const unsigned grid = (unsigned)((lanes + 255) / 256);
    auto go = [&](auto t, auto al) {
        using T = decltype(t);
        quantize_kernel<T, decltype(al)::value><<<grid, 256, 0, c.stream>>>((const T*)weights, weights_stride, outputs, inputs, group,
                                                                          chunks, groups, codes, scales);
    };
    if (dtype == GORILA_F32) vec ? go(float{}, std::true_type{}) : go(float{}, std::false_type{});
    else vec ? go(uint16_t{}, std::true_type{}) : go(uint16_t{}, std::false_type{});
    return launched();
}

int gorila_qmatvec(const void* x, int64_t x_stride, const float* x_scale, int32_t x_dtype, int64_t rows, const uint8_t* codes,
                   const float* scales, int32_t outputs, int32_t inputs, int32_t group, void* y, gorila_ctx* ctx) {
    CtxView c;
    const int rc = ctx_view(ctx, 0, c);
    if (rc) return rc;
    if (!row_dtype(x_dtype) && x_dtype != GORILA_CODES) return GORILA_EINVAL;
    if (rows < 0 || outputs < 0 || inputs < 1 || !group_size(group)) return GORILA_EINVAL;
    if (rows == 0 || outputs == 0) return GORILA_OK;
    const int e = x_dtype == GORILA_CODES ? 1 : dtype_bytes(x_dtype);
    if (!x || !codes || !scales || !y || (x_dtype == GORILA_CODES && !x_scale)) return GORILA_EINVAL;
    if (!at_element(x, e) || !aligned16(codes) || !at_element(scales, 4) || !at_element(x_scale, 4) ||
        !at_element(y, x_dtype == GORILA_BF16 ? 2 : 4))
        return GORILA_EINVAL;
    if (inputs > MAX_INPUTS || outputs > MAX_OUTPUTS || rows > 65535) return GORILA_EUNSUPPORTED;
    MatvecView v{x, x_stride, rows, x_scale, codes, scales, outputs, inputs, group, (inputs + 31) / 32, (inputs + group - 1) / group, y};
    const int supers = (v.chunks + SUPER - 1) / SUPER, tiles = (outputs + 15) / 16;
    using std::integral_constant;
    bool fits = true;
    auto go = [&](auto t, auto rt, auto al) {
        using T = decltype(t);
        constexpr int RT = decltype(rt)::value;
        int waves = 1;
        while (waves < most_waves<T, RT>() && waves < supers) waves <<= 1;
        fits = launch_fits(tiles, 64 * waves);
        const dim3 grid((unsigned)tiles, (unsigned)((rows + 16 * RT - 1) / (16 * RT)));
        if (fits) matvec_kernel<T, RT, decltype(al)::value><<<grid, 64 * waves, 0, c.stream>>>(v);
    };
    // Rows in as few passes over the codes as the registers allow: 64 8-bit rows at
    // once 38 us for 8192 x 8192, two times 32 54; bf16 82 and 70.
    auto by = [&](auto t, auto al) {
        if constexpr (std::is_same<decltype(t), int8_t>::value)
            if (rows > 32) return go(t, integral_constant<int, 4>{}, al);
        if (rows > 16) go(t, integral_constant<int, 2>{}, al);
        else go(t, integral_constant<int, 1>{}, al);
    };
    auto few = [&](auto t, auto r, auto al) {
        constexpr int R = decltype(r)::value, OUT = few_outputs(R);
        int lk = 4;
        while (lk < 64 && lk < v.chunks) lk <<= 1;
        const int waves = v.chunks <= 64 ? 1 : v.chunks < 64 * FEW_WAVES ? (v.chunks + 63) / 64 : FEW_WAVES;
        // more outputs a team, which share its inputs, where that leaves workgroups enough
        const int teams = 64 / lk, per = teams * OUT;
        int batches = 1;
        while (batches < 8 && (int64_t)(outputs + per - 1) / per * waves > 16 * batches * c.cus) batches <<= 1;
        const int blocks = (outputs + per * batches - 1) / (per * batches);
        fits = launch_fits(blocks, 64 * waves);
        if (fits) few_rows_kernel<decltype(t), R, decltype(al)::value><<<blocks, 64 * waves, 0, c.stream>>>(v, lk, batches);
    };
    auto by_few = [&](auto t, auto al) {
        if (rows == 1) few(t, integral_constant<int, 1>{}, al);
        else if (rows == 2) few(t, integral_constant<int, 2>{}, al);
        else if constexpr (std::is_same<decltype(t), int8_t>::value) few(t, integral_constant<int, 4>{}, al);
    };
    if (rows <= (x_dtype == GORILA_CODES ? 4 : 2)) {
        const bool four = x_dtype == GORILA_CODES ? !(x_stride & 7) && ((uintptr_t)x & 7) == 0 : !((x_stride | inputs) & 3) && at_four(x, e);
        if (x_dtype == GORILA_F32) four ? by_few(float{}, std::true_type{}) : by_few(float{}, std::false_type{});
        else if (x_dtype == GORILA_BF16) four ? by_few(uint16_t{}, std::true_type{}) : by_few(uint16_t{}, std::false_type{});
        else four ? by_few(int8_t{}, std::true_type{}) : by_few(int8_t{}, std::false_type{});
        return fits ? launched() : GORILA_EUNSUPPORTED;
    }
    const bool vec = aligned16(x) && ((x_stride * e) & 15) == 0;
    if (x_dtype == GORILA_F32) vec ? by(float{}, std::true_type{}) : by(float{}, std::false_type{});
    else if (x_dtype == GORILA_BF16) vec ? by(uint16_t{}, std::true_type{}) : by(uint16_t{}, std::false_type{});
    else vec ? by(int8_t{}, std::true_type{}) : by(int8_t{}, std::false_type{});
    return fits ? launched() : GORILA_EUNSUPPORTED;
}

}  // extern "C"
