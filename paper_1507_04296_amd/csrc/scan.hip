// The selective scan (gorila_scan, _backward, _step).
//
// With log-decays g_t = log a_t, G_t their running sum inside a chunk of Q steps,
// v_t = d_t x_t, and the state S before the chunk, one head's chunk is
//   y_t = sum_{s <= t} e^(G_t - G_s) (c_t . b_s) v_s + e^(G_t) S c_t + skip x_t,
//   S'  = e^(G_Q) S + sum_s e^(G_Q - G_s) v_s b_s^T,
// matrix products of Q x Q, Q x state and head_dim x state, formed from LDS on the
// matrix unit (fp32 rows v_mfma_f32_16x16x4_f32, bf16 rows v_mfma_f32_16x16x32_bf16).
// An episode start cuts the chunk: a pair (t, s)
// counts only where both are in one episode, S only for the steps before the first
// start.  Backward, with R the gradient that reaches the state after the chunk and
// F_ts = e^(G_t - G_s) (dy_t . x_s), M_ts = e^(G_t - G_s) (c_t . b_s),
//   dv_s = sum_t M_ts dy_t + w_s R b_s,            w_s = e^(G_Q - G_s)
//   dc_t = sum_s F_ts d_s b_s + e^(G_t) S^T dy_t,
//   db_s = d_s q_s,  q_s = sum_t F_ts c_t + w_s R^T x_s,
//   R'   = e^(G_Q) R + sum_t e^(G_t) dy_t c_t^T,
// and the gradient of g_t is the sum over all that passes from before t to t and
// after: pairs s < t <= u inside the chunk (F_us d_s (c_u . b_s)), the state before
// to the steps from t on, the steps before t to the state behind, and the state
// before to the state behind.  (The shorter sum_{u >= t} (c_u . dc_u - b_u . db_u)
// + <R, S'> is the same number, but cancels what does not pass t: with large step
// sizes its error is thousands of times the gradient's.)
//
// A workgroup of eight waves walks the chunks of one segment of one (sequence,
// head, 64 channels), the state in registers: wave w holds 16 channels (w % 4) and
// half of their states (w / 4).  Where there are few of those, sequences are cut into
// segments whose states are formed first (state_kernel), joined (join_kernel), and
// walked again side by side: a prompt of 8192 steps takes 65 us, where one workgroup a
// head would walk 256 chunks one after the other.
//
// What bounds it is mostly the chain of a chunk (stage, decays, products, walk; four
// barriers forward, seven backward with the states before the chunks walked again).
// fp32, 32 x 128 steps, 16 heads of 64, state 64: forward 28 us, backward 71 us + 8 us
// for the sums over heads, the matrix unit busy 30 % of the time.  bf16, 4 x 1999 steps,
// state 128: states 29 us (46 of both directions), joins 9 us (14), forward 54 us;
// backward 196 us, sums 26 us (131 MB), the matrix unit busy 10 % and less.  There the
// backward also moves 395 MB of workspace (the chunks' states out and in, the parts of
// db and dc), 82 us at the rate of a copy, with one workgroup a compute unit (132 KB of
// LDS, 185 registers and more).
// Chunks of 32 steps: with 64, the products inside a chunk double a step, and the
// backward's LDS holds one workgroup a compute unit at state 64 too.
//
// Masked products multiply by zero, which is no mask for infinities and NaN, so a
// chunk that holds any is walked one step at a time.  Its products still have zeros
// beside them (padded states and channels, the lower terms of bf16 rows' partners), so
// that an infinity may come out as NaN; finite it never becomes within its episode.
#include "planes.h"
#include "seq.h"

namespace gorila {
namespace {

constexpr int Q = 32;    // steps a chunk
constexpr int PW = 64;   // channels a workgroup
constexpr int THREADS = 512;
constexpr int LP = PW + 4, LQ = Q + 4;  // LDS row lengths: 16 lanes' quads on all banks
constexpr float LOG2E = 1.44269504088896341f;

__host__ __device__ inline int padded_state(int n) { return n <= 16 ? 16 : n <= 32 ? 32 : n <= 64 ? 64 : 128; }

struct ScanView {
    const void *x, *dt, *b, *c, *dy;
    int64_t xb, xt, dtb, dtt, bb, bt, cb, ct, dyb, dyt;
    const float *a_log, *dt_bias, *skip, *state;
    const uint8_t* reset;
    int B, T, H, P, G, N;
    int ptiles, vh;       // 64-channel tiles of a head; heads * ptiles
    int nch, cps, nseg;   // chunks, chunks a segment, segments
    void* y;
    float* state_out;
    // segments' states [B][nseg][vh][PW][NP] and decays [B][nseg][vh] (< 0: an
    // episode starts in it)
    float *seg_s, *seg_r, *seg_a;
    // backward
    const float* dstate_out;
    float *chunk_s;             // states before the chunks [B][nch][vh][PW * NP], in the lanes' order
    float *pdb, *pdc;           // [B][nch][vh][Q / 16][NP / 16][64][4], in the lanes' order
    float *pdt;                 // [B][T][vh]
    float *ppar;                // [B][nseg][vh][3]
    void* dx;
    float* dstate;
};

// Position of a workgroup: (sequence, segment, head, channels).
struct Place {
    int b, seg, v, h, p0, pw, grp;
    __device__ Place(const ScanView& s, int id) {
        v = id % s.vh;
        const int r = id / s.vh;
        seg = r % s.nseg;
        b = r / s.nseg;
        h = v / s.ptiles;
        p0 = (v % s.ptiles) * PW;
        pw = s.P - p0 < PW ? s.P - p0 : PW;
        grp = h / (s.H / s.G);
    }
};

__device__ __forceinline__ f32x4 mma(f32x4 a, f32x4 b, f32x4 c) {
#pragma unroll
    for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[j], b[j], c, 0, 0, 0);
    return c;
}
// Operands of 16 rows (columns) and 16 reduction indices: lane l holds row l % 16
// and indices 4 (l / 16) .. +3.  kfrag: the reduction runs along the LDS rows.
__device__ __forceinline__ f32x4 kfrag(const float* s, int ld, int row0, int k0, int l) {
    return *(const f32x4*)(s + (row0 + (l & 15)) * ld + k0 + 4 * (l >> 4));
}
__device__ __forceinline__ f32x4 rfrag(const float* s, int ld, int k0, int col0, int l) {
    const float* p = s + (k0 + 4 * (l >> 4)) * ld + col0 + (l & 15);
    return f32x4{p[0], p[ld], p[2 * ld], p[3 * ld]};
}

// bf16 rows: their values are operands of the bf16 instruction as they are, 16 times
// as fast as the fp32 one.  What is formed from them (states, decayed products) enters
// as three bf16 terms, which hold an fp32 value.  (Two terms, 16 bits: 2^-17 of every
// term, which products that cancel show.)  fp32 rows take the fp32 instruction: three
// terms of both operands would cost the vector unit what the matrix unit saves.
enum Operand { ROWS, FP32 };  // rows' values; fp32 values
// Upper halves of eight values that are bf16.
__device__ __forceinline__ bf16x8 rows_of(f32x4 a, f32x4 b) {
    constexpr uint32_t HIGH = 0x07060302u;
    const uint4 o{__builtin_amdgcn_perm(__float_as_uint(a[1]), __float_as_uint(a[0]), HIGH), __builtin_amdgcn_perm(__float_as_uint(a[3]), __float_as_uint(a[2]), HIGH),
                  __builtin_amdgcn_perm(__float_as_uint(b[1]), __float_as_uint(b[0]), HIGH), __builtin_amdgcn_perm(__float_as_uint(b[3]), __float_as_uint(b[2]), HIGH)};
    return __builtin_bit_cast(bf16x8, o);
}
template <int KIND> struct Terms {
    static constexpr int N = KIND == ROWS ? 1 : 3;
    bf16x8 t[N];
    __device__ __forceinline__ Terms(f32x4 a, f32x4 b) {
        if constexpr (KIND == FP32) {
            bf16x4 p[N], q[N];
            split4<N>(a, p);
            split4<N>(b, q);
#pragma unroll
            for (int i = 0; i < N; ++i) t[i] = __builtin_shufflevector(p[i], q[i], 0, 1, 2, 3, 4, 5, 6, 7);
        } else {
            t[0] = rows_of(a, b);
        }
    }
};
// c + two blocks of 16 reduction indices of a (rows' values) and b, and one block.
template <class T, int KIND>
__device__ __forceinline__ f32x4 mul2(f32x4 a0, f32x4 a1, f32x4 b0, f32x4 b1, f32x4 c) {
    if constexpr (std::is_same<T, float>::value) return mma(a1, b1, mma(a0, b0, c));
    else {
        const Terms<ROWS> a(a0, a1);
        const Terms<KIND> b(b0, b1);
#pragma unroll
        for (int i = Terms<KIND>::N - 1; i >= 0; --i) c = mfma16(a.t[0], b.t[i], c);
        return c;
    }
}
template <class T, int KIND>
__device__ __forceinline__ f32x4 mul2_swapped(f32x4 a0, f32x4 a1, f32x4 b0, f32x4 b1, f32x4 c) {  // b holds the rows' values
    if constexpr (std::is_same<T, float>::value) return mma(a1, b1, mma(a0, b0, c));
    else {
        const Terms<KIND> a(a0, a1);
        const Terms<ROWS> b(b0, b1);
#pragma unroll
        for (int i = Terms<KIND>::N - 1; i >= 0; --i) c = mfma16(a.t[i], b.t[0], c);
        return c;
    }
}
template <class T, int KIND>
__device__ __forceinline__ f32x4 mul1(f32x4 a, f32x4 b, f32x4 c) {
    if constexpr (std::is_same<T, float>::value) return mma(a, b, c);
    else return mul2<T, KIND>(a, f32x4{0.0f, 0.0f, 0.0f, 0.0f}, b, f32x4{0.0f, 0.0f, 0.0f, 0.0f}, c);
}
// Products over N blocks of 16, fa(i) and fb(i) the operands' blocks.
template <class T, int KIND, int N, bool SWAPPED = false, class A, class B>
__device__ __forceinline__ f32x4 product(A&& fa, B&& fb, f32x4 c) {
#pragma unroll
    for (int i = 0; i < N; i += 2) {
        const f32x4 zero{0.0f, 0.0f, 0.0f, 0.0f};
        if constexpr (N == 1 && std::is_same<T, float>::value) c = mma(fa(i), fb(i), c);
        else if constexpr (SWAPPED) c = mul2_swapped<T, KIND>(fa(i), N > 1 ? fa(i + 1) : zero, fb(i), N > 1 ? fb(i + 1) : zero, c);
        else c = mul2<T, KIND>(fa(i), N > 1 ? fa(i + 1) : zero, fb(i), N > 1 ? fb(i + 1) : zero, c);
    }
    return c;
}

// The same with one a (FP32 values) and two b (rows' values).
template <class T, int N, class A, class B>
__device__ __forceinline__ void product_pair(A&& fa, B&& fb, f32x4 (&c)[2]) {
#pragma unroll
    for (int i = 0; i < N; i += 2) {
        const f32x4 zero{0.0f, 0.0f, 0.0f, 0.0f};
        const f32x4 a0 = fa(i), a1 = N > 1 ? fa(i + 1) : zero;
        if constexpr (std::is_same<T, float>::value) {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                c[u] = mma(a0, fb(u, i), c[u]);
                if constexpr (N > 1) c[u] = mma(a1, fb(u, i + 1), c[u]);
            }
        } else {
            const Terms<FP32> a(a0, a1);
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const Terms<ROWS> b(fb(u, i), N > 1 ? fb(u, i + 1) : zero);
#pragma unroll
                for (int k = Terms<FP32>::N - 1; k >= 0; --k) c[u] = mfma16(a.t[k], b.t[0], c[u]);
            }
        }
    }
}

// Q rows of COLS columns on their way from memory to LDS, as they are in memory; rows
// past len and columns past cols are zeros.
template <class T, bool VEC> struct Quad {
    f32x4 v;
    __device__ __forceinline__ void load(const T* p, int n) { v = row_load<VEC>(p, n); }
    __device__ __forceinline__ f32x4 get() const { return v; }
};
template <> struct Quad<uint16_t, true> {
    uint2 v;
    __device__ __forceinline__ void load(const uint16_t* p, int n) {
        v = uint2{0, 0};
        if (n > 0) v = *(const uint2*)p;
    }
    __device__ __forceinline__ f32x4 get() const {
        return f32x4{__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xffff0000u), __uint_as_float(v.y << 16), __uint_as_float(v.y & 0xffff0000u)};
    }
};
template <int COLS, bool VEC, class T>
struct Rows {
    static constexpr int QUADS = COLS * Q / 4, R = (QUADS + THREADS - 1) / THREADS;
    Quad<T, VEC> v[R];
    const T* base;
    int64_t stride;
    int cols;
    static __device__ __forceinline__ int row(int i, int tid) { return (tid + THREADS * i) / (COLS / 4); }
    static __device__ __forceinline__ int col(int i, int tid) { return (tid + THREADS * i) % (COLS / 4) * 4; }
    __device__ __forceinline__ Rows(const T* b, int64_t st, int n) : base(b), stride(st), cols(n) {}
    // The len steps from t on.  The lanes' addresses are formed again each time: kept
    // over the loop they went to scratch memory, and reading them back waited for the
    // loads before.
    __device__ __forceinline__ void load(int t, int len) {
        const T* from = base + t * stride;
        const int tid = opaque((int)threadIdx.x);
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const int r = row(i, tid), c = col(i, tid);
            const bool in = r < len && c < cols;
            v[i].load(from + (in ? r * stride + c : 0), in ? cols - c : 0);
        }
    }
    // Adds 0 to bad, or NaN where a value is not finite.
    __device__ __forceinline__ void store(float* lds, int ld, float& bad) const {
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const f32x4 f = v[i].get();
            if (QUADS % THREADS == 0 || (int)threadIdx.x + THREADS * i < QUADS) *(f32x4*)(lds + row(i, (int)threadIdx.x) * ld + col(i, (int)threadIdx.x)) = f;
            bad += (f[0] * 0.0f + f[1] * 0.0f) + (f[2] * 0.0f + f[3] * 0.0f);
        }
    }
};

// Moves between lanes without LDS.  move<C>: within rows of 16, 0 where there is no
// such lane.
constexpr int DOWN = 0x100, UP = 0x110;  // + n: from the lane n above, n below
template <int C> __device__ __forceinline__ int move(int v) { return __builtin_amdgcn_update_dpp(0, v, C, 0xf, 0xf, true); }
template <int C> __device__ __forceinline__ float move(float v) { return __int_as_float(move<C>(__float_as_int(v))); }
__device__ __forceinline__ int lane_value(int v, int lane) { return __builtin_amdgcn_readlane(v, lane); }
__device__ __forceinline__ float lane_value(float v, int lane) { return __int_as_float(lane_value(__float_as_int(v), lane)); }
// Sum over the row's 16 lanes; over the same lane of the four rows; over the wave (all get it).
__device__ __forceinline__ float sum16(float v) {
    v += move<0xb1>(v);   // lanes swapped in pairs
    v += move<0x4e>(v);   // pairs in fours
    v += move<0x141>(v);  // eight mirrored
    v += move<0x140>(v);  // sixteen mirrored
    return v;
}
__device__ __forceinline__ float sum_rows(float v) {
    const uint32_t u = __float_as_uint(v);
    const auto p = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    const uint32_t q = __float_as_uint(__uint_as_float(p[0]) + __uint_as_float(p[1]));
    const auto r = __builtin_amdgcn_permlane32_swap(q, q, false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float sum64(float v) { return sum_rows(sum16(v)); }

// Step sizes, running log2-decays and episode numbers of a chunk.  A running sum is
// kept as a whole number and a rest within +-1/2, so that the difference of two of
// them is exact to 2^-23 however large both have grown: one sum in fp32 would lose
// what few small steps after a large one differ by.
struct Steps {
    float d[Q];            // step size
    float gi[Q], gf[Q];    // sum of the log2-decays: whole number, rest
    float from[Q], to[Q];  // e^G_t from the state before, e^(G_end - G_t) to the one behind; 0 in another episode
    int ep[Q];             // -1: past the end
    float all;             // from the state before to the one behind
    int last;              // episode of its end; not 0: one starts in it
    int odd;               // a step size is not finite
};
__device__ __forceinline__ float pow2(float v) { return __builtin_amdgcn_exp2f(v); }
constexpr float LEAST_LOG2 = -65536.0f;  // 2^this is zero, and sums of Q of it are whole numbers below 2^24
template <class T> struct StepRegs {  // as they are in memory: a value that is changed here is waited for here
    T raw;
    uint8_t raw_reset;
    __device__ __forceinline__ void load(const T* dt_base, int64_t stride, const uint8_t* rs, int t0, int len, int l) {
        raw = T{0};
        raw_reset = 0;
        if (l < len) {
            raw = dt_base[(int64_t)(t0 + l) * stride];
            if (rs) raw_reset = rs[t0 + l];
        }
    }
    // By the lanes of one wave (lanes past Q take part and store nothing).
    __device__ __forceinline__ void store(Steps& s, float bias, float rate2, int len, int l) const {
        const float v = row_value(raw) + bias;
        const float e = expf(-fabsf(v));
        float d = fmaxf(v, 0.0f) + log1pf(e);
        if (v != v) d = v;
        if (l >= len) d = 0.0f;
        float dec = rate2 * d;
        if (dec < LEAST_LOG2) dec = LEAST_LOG2;
        float gi = rintf(dec), gf = dec - gi;
        int ep = raw_reset != 0;
        static_assert(Q == 32, "two rows of lanes");
        auto add = [&](float iu, float fu, int eu) {
            gf += fu;
            const float r = rintf(gf);
            gi += iu + r;
            gf -= r;
            ep += eu;
        };
        add(move<UP + 1>(gi), move<UP + 1>(gf), move<UP + 1>(ep));
        add(move<UP + 2>(gi), move<UP + 2>(gf), move<UP + 2>(ep));
        add(move<UP + 4>(gi), move<UP + 4>(gf), move<UP + 4>(ep));
        add(move<UP + 8>(gi), move<UP + 8>(gf), move<UP + 8>(ep));
        const float row_gi = lane_value(gi, 15), row_gf = lane_value(gf, 15);
        const int row_ep = lane_value(ep, 15);
        if (l >= 16) add(row_gi, row_gf, row_ep);
        const float end_gi = lane_value(gi, Q - 1), end_gf = lane_value(gf, Q - 1);
        const int end_ep = lane_value(ep, Q - 1);
        if (l < Q) {
            const bool in = l < len;
            s.d[l] = d;
            s.gi[l] = gi;
            s.gf[l] = gf;
            s.ep[l] = in ? ep : -1;
            s.from[l] = in && ep == 0 ? pow2(gi + gf) : 0.0f;
            s.to[l] = in && ep == end_ep ? pow2((end_gi - gi) + (end_gf - gf)) : 0.0f;
        }
        const bool odd = __any(l < Q && d * 0.0f != 0.0f);
        if (l == 0) {
            s.odd = odd;
            s.all = end_ep == 0 ? pow2(end_gi + end_gf) : 0.0f;
            s.last = end_ep;
        }
    }
};

// v times a factor of a Steps where both are of one episode, else 0 whatever v is.  The
// factor itself is no mask: it is also zero where a decay is too small for it, and there
// a v that is not finite stays so.
__device__ __forceinline__ f32x4 masked(f32x4 v, float f, bool one_episode) { return one_episode ? v * f : f32x4{0.0f, 0.0f, 0.0f, 0.0f}; }

// State tiles of a wave: the half h of NT (all of one).
template <int NT> struct Half {
    static constexpr int TILES = NT > 1 ? NT / 2 : 1;
    static __device__ __forceinline__ int first(int h) { return h * TILES; }
    static __device__ __forceinline__ bool on(int h) { return NT > 1 || h == 0; }
};

// acc (rows: states from m on, columns: 16 channels from ch on) = decay * acc + sum
// over steps of weight * m[step][state] * ch[step][channel].  AFTER: the state after
// the chunk from the one before (weights w_s d_s); else the gradient before it from
// the one after (weights e^G).
template <class T, int TILES, bool AFTER>
__device__ __forceinline__ void walk(f32x4 (&acc)[TILES], const float* m, int ldm, const float* ch, const Steps& st, int l) {
    const float all = st.all;
    const bool starts = st.last != 0;
#pragma unroll
    for (int n = 0; n < TILES; ++n) acc[n] = masked(acc[n], all, !starts);
    if (!AFTER && st.ep[0] != 0) return;  // an episode starts with the chunk
    f32x4 v[Q / 16];
#pragma unroll
    for (int kb = 0; kb < Q / 16; ++kb) {
        const int k0 = 16 * kb + 4 * (l >> 4);
        v[kb] = rfrag(ch, LP, 16 * kb, 0, l);
        v[kb] *= AFTER ? *(const f32x4*)(st.to + k0) * *(const f32x4*)(st.d + k0) : *(const f32x4*)(st.from + k0);
    }
#pragma unroll
    for (int n = 0; n < TILES; ++n)
        acc[n] = mul2<T, FP32>(rfrag(m, ldm, 0, 16 * n, l), rfrag(m, ldm, 16, 16 * n, l), v[0], v[1], acc[n]);
}

// Registers <-> state arrays [channel][state] of `ld` states a channel in memory, the
// wave's tiles from channel p0 and state n0 on, of pw channels and n_in states in all.
template <int TILES, bool VEC>
__device__ __forceinline__ void load_state(f32x4 (&acc)[TILES], const float* s, int ld, int pw, int n_in, int p0, int n0, int l) {
    const int p = p0 + (l & 15);
#pragma unroll
    for (int i = 0; i < TILES; ++i) {
        const int n = n0 + 16 * i + 4 * (l >> 4);
        const bool in = s && p < pw && n < n_in;
        acc[i] = row_load<VEC>(in ? s + (int64_t)p * ld + n : s, in ? n_in - n : 0);
    }
}
template <int TILES, bool VEC>
__device__ __forceinline__ void store_state(const f32x4 (&acc)[TILES], float* s, int ld, int pw, int n_in, int p0, int n0, int l) {
    const int p = p0 + (l & 15);
#pragma unroll
    for (int i = 0; i < TILES; ++i) {
        const int n = n0 + 16 * i + 4 * (l >> 4);
        if (p < pw && n < n_in) row_store<VEC>(s + (int64_t)p * ld + n, acc[i], n_in - n);
    }
}
// The same of the workspace's states, in the order of the lanes that hold them:
// [state tile][channel tile][lane][4].  In rows of states, a wave's 16 bytes a lane lie
// on 16 lines, which a load or store takes one after the other.
__device__ __forceinline__ f32x4* own_state(float* s, int p0, int n0, int l) { return (f32x4*)s + ((n0 / 16) * (PW / 16) + p0 / 16) * 64 + l; }
template <int TILES>
__device__ __forceinline__ void load_own(f32x4 (&acc)[TILES], float* s, int p0, int n0, int l) {
#pragma unroll
    for (int i = 0; i < TILES; ++i) acc[i] = own_state(s, p0, n0, l)[i * (PW / 16) * 64];
}
template <int TILES>
__device__ __forceinline__ void store_own(const f32x4 (&acc)[TILES], float* s, int p0, int n0, int l) {
#pragma unroll
    for (int i = 0; i < TILES; ++i) own_state(s, p0, n0, l)[i * (PW / 16) * 64] = acc[i];
}
// To LDS [channel][state].
template <int TILES>
__device__ __forceinline__ void stage_state(const f32x4 (&acc)[TILES], float* s, int ld, int p0, int n0, int l) {
#pragma unroll
    for (int i = 0; i < TILES; ++i) *(f32x4*)(s + (p0 + (l & 15)) * ld + n0 + 16 * i + 4 * (l >> 4)) = acc[i];
}

template <class T>
__device__ __forceinline__ const T* of(const void* p, int64_t off) { return (const T*)p + off; }

// Where a workgroup's data lie.
template <class T> struct Data {
    const T *x, *b, *c, *dy, *dt;
    const uint8_t* reset;
    int64_t state;  // of the caller's states
    float rate2, bias;
    __device__ Data(const ScanView& s, const Place& at) {
        const int64_t h = (int64_t)at.h * s.P + at.p0, g = (int64_t)at.grp * s.N;
        x = of<T>(s.x, at.b * s.xb + h);
        dy = of<T>(s.dy, at.b * s.dyb + h);
        b = of<T>(s.b, at.b * s.bb + g);
        c = of<T>(s.c, at.b * s.cb + g);
        dt = of<T>(s.dt, at.b * s.dtb + at.h);
        reset = s.reset ? s.reset + (int64_t)at.b * s.T : nullptr;
        state = (((int64_t)at.b * s.H + at.h) * s.P + at.p0) * s.N;
        rate2 = -expf(s.a_log[at.h]) * LOG2E;
        bias = s.dt_bias[at.h];
    }
};

// Steps that are walked together: chunks, or, where a chunk holds a value that is not
// finite, its steps one by one.
struct Walk {
    int begin, end;    // of the segment
    int t, len;        // now
    int single;        // end (backward: begin) of the chunk that is walked step by step, or -1
    __device__ Walk(const ScanView& s, int seg) {
        begin = seg * s.cps * Q;
        end = begin + s.cps * Q < s.T ? begin + s.cps * Q : s.T;
        single = -1;
    }
    __device__ int chunk_end(int a) const { return a + Q < end ? a + Q : end; }
    // forward
    __device__ bool start() { t = begin, len = chunk_end(t) - t; return t < end; }
    __device__ void split() { single = t + len, len = 1; }
    __device__ bool next(bool& whole) {  // whole: the chunk that was walked step by step is done
        t += len;
        whole = single >= 0 && t >= single;
        if (whole) single = -1;
        if (t >= end) return false;
        len = single >= 0 ? 1 : chunk_end(t) - t;
        return true;
    }
    // backward
    __device__ int chunk() const { return begin + (t - begin) / Q * Q; }
    __device__ bool start_back() { t = begin + (end > begin ? (end - begin - 1) / Q * Q : 0), len = end - t; return begin < end; }
    __device__ void split_back() { single = t, t += len - 1, len = 1; }
    __device__ bool next_back(bool& whole) {
        whole = single >= 0 && t <= single;
        if (whole) single = -1;
        if (t <= begin) return false;
        if (single >= 0) { t -= 1; }
        else { t = begin + (t - 1 - begin) / Q * Q, len = Q; }
        return true;
    }
};

// Forward over one segment.
template <class T, int NP, bool VEC>
__global__ __launch_bounds__(THREADS, 4) void scan_kernel(ScanView s) {
    constexpr int NT = NP / 16, LN = NP + 4, TILES = Half<NT>::TILES;
    __shared__ __align__(16) float sc[Q * LN], sb[Q * LN], sx[Q * LP], ss[PW * LN], sm[Q * LQ];
    __shared__ __align__(16) Steps st;
    __shared__ int flag;
    const Place at(s, blockIdx.x);
    const Data<T> in(s, at);
    const int tid = threadIdx.x, l = tid & 63, lg = l >> 4, lc = l & 15;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6), wp = w & 3, half = w >> 2, n_own = 16 * Half<NT>::first(half);
    const bool on = Half<NT>::on(half);
    const float skip = s.skip[at.h];
    const int64_t yt = (int64_t)s.H * s.P;
    T* y = (T*)s.y + ((int64_t)at.b * s.T * s.H + at.h) * s.P + at.p0 + (16 * half + lc) * yt + 16 * wp + 4 * lg;

    f32x4 S[TILES];
    if (s.nseg > 1)
        load_own(S, s.seg_s + (((int64_t)at.b * s.nseg + at.seg) * s.vh + at.v) * PW * NP, 16 * wp, on ? n_own : 0, l);
    else
        load_state<TILES, VEC>(S, s.state ? s.state + in.state : nullptr, s.N, at.pw, s.N, 16 * wp, n_own, l);
    if (tid == 0) flag = 0;

    Rows<PW, VEC, T> rx(in.x, s.xt, at.pw);
    Rows<NP, VEC, T> rb(in.b, s.bt, s.N), rc(in.c, s.ct, s.N);
    StepRegs<T> rd;
    Walk at_t(s, at.seg);
    auto load = [&]() {
        rx.load(at_t.t, at_t.len);
        rb.load(at_t.t, at_t.len);
        rc.load(at_t.t, at_t.len);
        if (w == 7) rd.load(in.dt, s.dtt, in.reset, at_t.t, at_t.len, l);
    };
    bool more = at_t.start();
    if (more) load();
    while (more) {
        // What needs no decays, beside the decays (a long chain of a few lanes): what the
        // state gives 16 steps (rows = channels, columns = steps), c_t . b_s of the three
        // tiles with s <= t.
        const int t = 16 * half + lc, si = w >> 1, ti = w > 0;
        f32x4 acc, m;
        for (;;) {  // again where the chunk is to be walked step by step
            __syncthreads();
            float bad = 0.0f;
            rx.store(sx, LP, bad);
            rb.store(sb, LN, bad);
            rc.store(sc, LN, bad);
            if (on) stage_state<TILES>(S, ss, LN, 16 * wp, n_own, l);
            if (bad != bad) flag = 1;
            __syncthreads();
            acc = m = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
            if (w == 7) rd.store(st, in.bias, in.rate2, at_t.len, l);
            acc = product<T, FP32, NT, true>([&](int n) { return kfrag(ss, LN, 16 * wp, 16 * n, l); },
                                              [&](int n) { return kfrag(sc, LN, 16 * half, 16 * n, l); }, acc);
            if (w < 3)
                m = product<T, ROWS, NT>([&](int n) { return kfrag(sb, LN, 16 * si, 16 * n, l); },
                                         [&](int n) { return kfrag(sc, LN, 16 * ti, 16 * n, l); }, m);
            __syncthreads();
            if (at_t.single >= 0 || !(flag || st.odd)) break;
            at_t.split();
            load();
        }
        const int t0 = at_t.t, len = at_t.len;
        bool whole;
        more = at_t.next(whole);
        if (more) load();
        acc = masked(acc, st.from[t], st.ep[t] == 0);
        if (w < 3) {  // decay * (c_t . b_s) * d_s
            const int tm = 16 * ti + lc, q0 = 16 * si + 4 * lg;
            const float gi_t = st.gi[tm], gf_t = st.gf[tm];
            const int et = st.ep[tm];
            const f32x4 gi = *(const f32x4*)(st.gi + q0), gf = *(const f32x4*)(st.gf + q0), d = *(const f32x4*)(st.d + q0);
            const i32x4 ep = *(const i32x4*)(st.ep + q0);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const bool same = tm == q0 + j, behind = tm > q0 + j && ep[j] == et;
                m[j] = same ? m[j] * d[j] : behind ? m[j] * (pow2((gi_t - gi[j]) + (gf_t - gf[j])) * d[j]) : 0.0f;
            }
            *(f32x4*)(sm + tm * LQ + q0) = m;
        }
        if (on) walk<T, TILES, true>(S, sb + n_own, LN, sx + 16 * wp, st, l);
        __syncthreads();
        if (half)
            acc = mul2<T, FP32>(rfrag(sx, LP, 0, 16 * wp, l), rfrag(sx, LP, 16, 16 * wp, l), kfrag(sm, LQ, 16, 0, l), kfrag(sm, LQ, 16, 16, l), acc);
        else
            acc = mul1<T, FP32>(rfrag(sx, LP, 0, 16 * wp, l), kfrag(sm, LQ, 0, 0, l), acc);
        const int p = 16 * wp + 4 * lg;
        if (t < len && p < at.pw) row_store<VEC>(y + t0 * yt, acc + skip * *(const f32x4*)(sx + t * LP + p), at.pw - p);
        if (whole && tid == 0) flag = 0;  // nobody reads it before the next chunk is staged
    }
    if (on && s.state_out && at.seg == s.nseg - 1) store_state<TILES, VEC>(S, s.state_out + in.state, s.N, at.pw, s.N, 16 * wp, n_own, l);
}

// What one segment adds to the state behind it (REV = false: from x and b) or to
// the gradient of the state before it (REV = true: from dy and c), and its decay.
template <class T, int NP, bool VEC, bool REV>
__device__ __forceinline__ void segment_state(const ScanView& s, float* sb, float* sx, Steps* st, int& flag) {
    constexpr int NT = NP / 16, LN = NP + 4, TILES = Half<NT>::TILES;
    const Place at(s, blockIdx.x);
    const Data<T> in(s, at);
    const int tid = threadIdx.x, l = tid & 63;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6), wp = w & 3, half = w >> 2, n_own = 16 * Half<NT>::first(half);
    const bool on = Half<NT>::on(half);
    f32x4 S[TILES];
#pragma unroll
    for (int n = 0; n < TILES; ++n) S[n] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    if (tid == 0) flag = 0;
    float decay = 1.0f;
    bool starts = false;
    const int64_t xt = REV ? s.dyt : s.xt, bt = REV ? s.ct : s.bt;
    Rows<PW, VEC, T> rx(REV ? in.dy : in.x, xt, at.pw);
    Rows<NP, VEC, T> rb(REV ? in.c : in.b, bt, s.N);
    StepRegs<T> rd;
    Walk at_t(s, at.seg);
    auto load = [&]() {
        rx.load(at_t.t, at_t.len);
        rb.load(at_t.t, at_t.len);
        if (w == 7) rd.load(in.dt, s.dtt, in.reset, at_t.t, at_t.len, l);
    };
    // Where nothing stops it, wave 7 forms the decays of the next chunk beside the walk
    // of this one (st[turn ^ 1]).
    int turn = 0;
    auto steps = [&](int to) { rd.store(st[to], in.bias, in.rate2, at_t.len, l); };
    bool more = REV ? at_t.start_back() : at_t.start();
    if (more) {
        load();
        if (w == 7) steps(0);
    }
    while (more) {
        for (;;) {  // again where the chunk is to be walked step by step
            __syncthreads();
            float bad = 0.0f;
            rx.store(sx, LP, bad);
            rb.store(sb, LN, bad);
            if (bad != bad) flag = 1;
            __syncthreads();
            if (at_t.single >= 0 || !(flag || st[turn].odd)) break;
            REV ? at_t.split_back() : at_t.split();
            load();
            __syncthreads();  // everyone has read st[turn]
            if (w == 7) steps(turn);
        }
        bool whole;
        more = REV ? at_t.next_back(whole) : at_t.next(whole);
        if (more) load();
        decay *= st[turn].all;
        starts |= st[turn].last != 0;
        if (on) walk<T, TILES, !REV>(S, sb + n_own, LN, sx + 16 * wp, st[turn], l);
        if (more && w == 7) steps(turn ^ 1);
        turn ^= 1;
        if (whole) {
            __syncthreads();
            if (tid == 0) flag = 0;
        }
    }
    const int64_t o = ((int64_t)at.b * s.nseg + at.seg) * s.vh + at.v;
    if (on) store_own(S, (REV ? s.seg_r : s.seg_s) + o * PW * NP, 16 * wp, n_own, l);
    if (!REV && tid == 0) s.seg_a[o] = starts ? -1.0f : decay;
}

template <class T, int NP, bool VEC>
__global__ __launch_bounds__(THREADS, 4) void state_kernel(ScanView s) {
    __shared__ __align__(16) float sb[Q * (NP + 4)], sx[Q * LP];
    __shared__ __align__(16) Steps st[2];
    __shared__ int flag;
    if (blockIdx.y == 0) segment_state<T, NP, VEC, false>(s, sb, sx, st, flag);
    else segment_state<T, NP, VEC, true>(s, sb, sx, st, flag);
}

// Turns what each segment adds into the state before it (blockIdx.y = 0) or the
// gradient behind it (1), in place, one thread an element.
template <int NP, bool VEC>
__global__ __launch_bounds__(256) void join_kernel(ScanView s) {
    const int e = (blockIdx.x % (PW * NP / 256)) * 256 + threadIdx.x, o = blockIdx.x / (PW * NP / 256);
    const int v = o % s.vh, b = o / s.vh, h = v / s.ptiles;
    // its place in the lanes' order
    const int lane = e / 4 % 64, p = (v % s.ptiles) * PW + e / 256 % (PW / 16) * 16 + lane % 16, n = e / (PW * 16) * 16 + lane / 16 * 4 + e % 4;
    const bool rev = blockIdx.y != 0;
    const float* from = rev ? s.dstate_out : s.state;
    float* seg = (rev ? s.seg_r : s.seg_s) + ((int64_t)b * s.nseg * s.vh + v) * PW * NP + e;
    const float* dec = s.seg_a + (int64_t)b * s.nseg * s.vh + v;
    const int64_t step = (int64_t)s.vh * PW * NP;
    float cur = from && p < s.P && n < s.N ? from[(((int64_t)b * s.H + h) * s.P + p) * s.N + n] : 0.0f;
    constexpr int AHEAD = 8;  // loads in flight
    for (int i0 = 0; i0 < s.nseg; i0 += AHEAD) {
        float own[AHEAD], a[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int at = i0 + i < s.nseg ? i0 + i : s.nseg - 1, k = rev ? s.nseg - 1 - at : at;
            own[i] = seg[k * step], a[i] = dec[k * s.vh];
        }
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            if (i0 + i >= s.nseg) break;
            seg[(rev ? s.nseg - 1 - i0 - i : i0 + i) * step] = cur;
            cur = a[i] < 0.0f ? own[i] : a[i] * cur + own[i];
        }
    }
}

// A lane's part of a state walked without LDS from step t0 to t1, where a chunk has
// values that are not finite (slow, and rare: kept out of the registers of the rest).
template <int TILES> struct Tiles { f32x4 v[TILES]; };
template <int TILES, class T>
__device__ __noinline__ Tiles<TILES> walk_plain(Tiles<TILES> S, const T* x, int64_t xt, const T* b, int64_t bt, int n_left, const T* dt,
                                                int64_t dtt, const uint8_t* reset, float rate2, float bias, int t0, int t1) {
    for (int t = t0; t < t1; ++t) {
        const float v = row_value(dt[t * dtt]) + bias;
        float d = fmaxf(v, 0.0f) + log1pf(expf(-fabsf(v)));
        if (v != v) d = v;
        const float a = pow2(rate2 * d), xv = x ? row_value(x[t * xt]) : 0.0f;
        const bool start = reset && reset[t];
#pragma unroll
        for (int i = 0; i < TILES; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float add = d * xv * (16 * i + j < n_left ? row_value(b[t * bt + 16 * i + j]) : 0.0f);
                S.v[i][j] = start ? add : fmaf(a, S.v[i][j], add);
            }
    }
    return S;
}

// Backward over one segment: forward once for the states before its chunks, then
// back.
template <class T, int NP, bool VEC>
__global__ __launch_bounds__(THREADS, NP > 64 ? 2 : 4) void scan_backward_kernel(ScanView s) {
    constexpr int NT = NP / 16, LN = NP + 4, TILES = Half<NT>::TILES;
    __shared__ __align__(16) float sc[Q * LN], sb[Q * LN], sx[Q * LP], sdy[Q * LP], ss[PW * LN], sr[PW * LN];
    __shared__ __align__(16) float sm[Q * LQ], sf[Q * LQ];
    __shared__ __align__(16) Steps st;
    __shared__ float hc[NT][Q], qb[NT][Q], kb[NT][Q], pairs[3][Q], inner[8];
    __shared__ int flag;
    const Place at(s, blockIdx.x);
    const Data<T> in(s, at);
    const int tid = threadIdx.x, lane = tid & 63;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6), wp = w & 3, half = w >> 2, n_own = 16 * Half<NT>::first(half);
    const bool on = Half<NT>::on(half);
    const int64_t yt = (int64_t)s.H * s.P;
    const int64_t seg0 = (((int64_t)at.b * s.nseg + at.seg) * s.vh + at.v) * PW * NP;
    float* chunk_s = s.chunk_s + ((int64_t)at.b * s.nch * s.vh + at.v) * PW * NP;  // of chunk 0
    const int64_t chunk_step = (int64_t)s.vh * PW * NP;

    Rows<PW, VEC, T> rx(in.x, s.xt, at.pw);
    Rows<NP, VEC, T> rb(in.b, s.bt, s.N);
    StepRegs<T> rd;
    f32x4 R[TILES];
    float decay_sum = 0.0f, bias_sum = 0.0f, skip_sum = 0.0f;  // of the three parameters' gradients
    if (tid == 0) flag = 0;
    Walk at_t(s, at.seg);
    auto load_in = [&]() {
        rx.load(at_t.t, at_t.len);
        rb.load(at_t.t, at_t.len);
        if (w == 7) rd.load(in.dt, s.dtt, in.reset, at_t.t, at_t.len, opaque(lane));
    };
    auto stage_in = [&](int l) {
        float bad = 0.0f;
        rx.store(sx, LP, bad);
        rb.store(sb, LN, bad);
        if (bad != bad) flag = 1;
    };
    auto steps = [&](Steps& to, int l) { rd.store(to, in.bias, in.rate2, at_t.len, l); };
    auto plain_walk = [&](f32x4 (&S)[TILES], int t0, int t1) {
        const int lc = lane & 15, lg = lane >> 4;
        Tiles<TILES> v;
#pragma unroll
        for (int i = 0; i < TILES; ++i) v.v[i] = S[i];
        const int p = 16 * wp + lc, n = n_own + 4 * lg;
        v = walk_plain<TILES, T>(v, p < at.pw ? in.x + p : nullptr, s.xt, in.b + n, s.bt, s.N - n, in.dt, s.dtt, in.reset, in.rate2, in.bias, t0, t1);
#pragma unroll
        for (int i = 0; i < TILES; ++i) S[i] = v.v[i];
    };
    {
        f32x4 S[TILES];
        if (s.nseg > 1)
            load_own(S, s.seg_s + seg0, 16 * wp, on ? n_own : 0, lane);
        else
            load_state<TILES, VEC>(S, s.state ? s.state + in.state : nullptr, s.N, at.pw, s.N, 16 * wp, n_own, lane);
        // Wave 7 forms the decays of the next chunk beside the walk of this one; every
        // other chunk's stand in sf, which is not in use yet.
        static_assert(sizeof(Steps) <= sizeof sf, "a place for the steps");
        if (at_t.start()) {
            load_in();
            if (w == 7 && at_t.len < at_t.end - at_t.t) steps(st, opaque(lane));
            Steps *now = &st, *next = (Steps*)sf;
            for (;;) {
                const int t0 = at_t.t, len = at_t.len;
                if (on) store_own(S, chunk_s + t0 / Q * chunk_step, 16 * wp, n_own, lane);
                bool whole;
                if (t0 + len >= at_t.end) break;  // nobody asks for the state behind the last
                __syncthreads();
                stage_in(opaque(lane));
                __syncthreads();
                const bool plain = flag != 0 || now->odd;
                at_t.next(whole);
                load_in();
                if (plain) {
                    plain_walk(S, t0, t0 + len);
                    __syncthreads();
                    if (tid == 0) flag = 0;
                } else if (on) {
                    walk<T, TILES, true>(S, sb + n_own, LN, sx + 16 * wp, *now, opaque(lane));
                }
                if (w == 7 && at_t.len < at_t.end - at_t.t) steps(*next, opaque(lane));
                Steps* const other = now;
                now = next;
                next = other;
            }
        }
        if (s.nseg > 1)
            load_own(R, s.seg_r + seg0, 16 * wp, on ? n_own : 0, lane);
        else
            load_state<TILES, VEC>(R, s.dstate_out ? s.dstate_out + in.state : nullptr, s.N, at.pw, s.N, 16 * wp, n_own, lane);
    }

    Rows<PW, VEC, T> ry(in.dy, s.dyt, at.pw);
    Rows<NP, VEC, T> rc(in.c, s.ct, s.N);
    f32x4 S[TILES];
    auto load_out = [&]() {
        ry.load(at_t.t, at_t.len);
        rc.load(at_t.t, at_t.len);
    };
    auto load_s = [&]() {
        load_own(S, chunk_s + at_t.chunk() / Q * chunk_step, 16 * wp, on ? n_own : 0, opaque(lane));
    };
    const float skip = s.skip[at.h];
    T* dx = (T*)s.dx + ((int64_t)at.b * s.T * s.H + at.h) * s.P + at.p0;
    const int64_t part0 = ((int64_t)at.b * s.nch * s.vh + at.v) * Q * NP, part_step = (int64_t)s.vh * Q * NP;
    auto load = [&]() {
        load_in();
        load_out();
    };
    // The gradients of a chunk's step sizes and decays, lane = step: by wave 6, beside the
    // next chunk's first products (a long chain of a few lanes).
    float past_d = 0.0f, past_all = 0.0f;
    int past_t = 0, past_len = 0;
    auto finish = [&](int l) {
        const int t = l & (Q - 1);
        float h = 0.0f, k = 0.0f, q = 0.0f;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            h += hc[n][t];
            k += kb[n][t];
            q += qb[n][t];
        }
        k *= past_d;
        h += move<DOWN + 1>(h);  // steps from t on
        h += move<DOWN + 2>(h);
        h += move<DOWN + 4>(h);
        h += move<DOWN + 8>(h);
        const float h16 = lane_value(h, 16);
        if (t < 16) h += h16;
        k += move<UP + 1>(k);  // steps up to t
        k += move<UP + 2>(k);
        k += move<UP + 4>(k);
        k += move<UP + 8>(k);
        const float k15 = lane_value(k, 15), below = move<UP + 1>(k);
        float g = h + (t > 16 ? k15 + below : t == 16 ? k15 : below);
        if (t > 0) g += pairs[1][t];
        if (t > 0 && t < 16) g += pairs[0][t];
        if (t > 16) g += pairs[2][t];
        // without a start in the chunk, the state before it to the one behind it
        if (!(past_all < 0.0f)) g += (((inner[0] + inner[1]) + (inner[2] + inner[3])) + ((inner[4] + inner[5]) + (inner[6] + inner[7]))) * past_all;
        if (l < past_len) {
            // log a = -exp(a_log) d, and d's derivative by dt is 1 - e^-d
            const float rate = in.rate2 / LOG2E, dd = (q + g * rate) * -expm1f(-past_d);
            const float log_a = rate * past_d;
            decay_sum += g * (log_a < LEAST_LOG2 / LOG2E ? LEAST_LOG2 / LOG2E : log_a);
            bias_sum += dd;
            s.pdt[((int64_t)at.b * s.T + past_t + l) * s.vh + at.v] = dd;
        }
        past_len = 0;
    };
    bool more = at_t.start_back();
    if (more) {
        load_out();
        load_s();
    }  // the last chunk's inputs are here
    while (more) {
        // what the lane number decides is decided again for every chunk: kept over the
        // loop it took more scalar registers than there are
        const int l = opaque(lane), lg = l >> 4, lc = l & 15;
        // What needs no decays, beside the decays: the tiles with s <= t of c_t . b_s
        // (waves 0 .. 2) and dy_t . x_s (3 .. 5); rows = s, columns = t.
        const int tile = w < 3 ? w : w - 3, si = tile >> 1, ti = tile > 0;
        const int tm = 16 * ti + lc, q0 = 16 * si + 4 * lg;
        f32x4 f;
        float pass;
        // (Again with a chunk's last step where it is to be walked step by step: in this
        // small loop, or the other loop's registers would be copied at its end, and waited for.)
        for (;;) {
            if (at_t.single >= 0 && on) plain_walk(S, at_t.chunk(), at_t.t);
            __syncthreads();
            stage_in(l);
            float bad = 0.0f;
            ry.store(sdy, LP, bad);
            rc.store(sc, LN, bad);
            pass = 0.0f;  // <R, S>, from the state before to the one behind
            if (on) {
                stage_state<TILES>(R, sr, LN, 16 * wp, n_own, l);
                stage_state<TILES>(S, ss, LN, 16 * wp, n_own, l);
#pragma unroll
                for (int n = 0; n < TILES; ++n) pass += (R[n][0] * S[n][0] + R[n][1] * S[n][1]) + (R[n][2] * S[n][2] + R[n][3] * S[n][3]);
            }
            if (bad != bad) flag = 1;
            __syncthreads();
            f = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
            if (w < 3) {
                f = product<T, ROWS, NT>([&](int n) { return kfrag(sb, LN, 16 * si, 16 * n, l); },
                                         [&](int n) { return kfrag(sc, LN, 16 * ti, 16 * n, l); }, f);
            } else if (w < 6) {
                f = product<T, ROWS, PW / 16>([&](int n) { return kfrag(sx, LP, 16 * si, 16 * n, l); },
                                              [&](int n) { return kfrag(sdy, LP, 16 * ti, 16 * n, l); }, f);
            } else if (w == 7) {
                steps(st, l);
            } else if (past_len) {
                finish(l);
            }
            __syncthreads();
            if (at_t.single >= 0 || !(flag || st.odd)) break;
            at_t.split_back();
            load();
            load_s();
        }
        const int t0 = at_t.t, len = at_t.len;
        bool whole;
        more = at_t.next_back(whole);
        if (more) load();
        load_s();  // after the last chunk too: loaded in a branch, it would be copied, and waited for, at its end
        if (w < 6) {  // M and F
            const float gi_t = st.gi[tm], gf_t = st.gf[tm];
            const int et = st.ep[tm];
            const f32x4 gi = *(const f32x4*)(st.gi + q0), gf = *(const f32x4*)(st.gf + q0);
            const i32x4 ep = *(const i32x4*)(st.ep + q0);
            f32x4 g;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const bool same = tm == q0 + j, behind = tm > q0 + j && ep[j] == et;
                g[j] = same ? f[j] : behind ? f[j] * pow2((gi_t - gi[j]) + (gf_t - gf[j])) : 0.0f;
            }
            *(f32x4*)((w < 3 ? sm : sf) + tm * LQ + q0) = g;
        }
        // What the states around the chunk give dc (of S) and db (of R; rows = state,
        // columns = steps) and dx (of R; rows = channels), meanwhile.  A wave has a tile
        // of one of the two for both halves of the steps, and its own tiles of R for dx:
        // no state is read and split twice.
        constexpr int JOBS = NT == 8 ? 2 : 1;
        f32x4 ja[JOBS][2], xa[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) xa[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int u = 0; u < JOBS; ++u) {
            const bool of_r = NT == 8 ? u : w >= NT;
            const int n = NT == 8 ? w : w % NT;
            const float *m = of_r ? sr : ss, *rows = of_r ? sx : sdy, *by = of_r ? st.to : st.from;
            const int ep = of_r ? st.last : 0;
            ja[u][0] = ja[u][1] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
            if (w < 2 * NT)
                product_pair<T, PW / 16>([&](int k) { return rfrag(m, LN, 16 * k, 16 * n, l); },
                                         [&](int i, int k) { return kfrag(rows, LP, 16 * i, 16 * k, l); }, ja[u]);
#pragma unroll
            for (int i = 0; i < 2; ++i) ja[u][i] = masked(ja[u][i], by[16 * i + lc], st.ep[16 * i + lc] == ep);
        }
        if (on)
            product_pair<T, TILES>([&](int n) { return R[n]; }, [&](int i, int n) { return kfrag(sb, LN, 16 * i, n_own + 16 * n, l); }, xa);
#pragma unroll
        for (int i = 0; i < 2; ++i) xa[i] = masked(xa[i], st.to[16 * i + lc], st.ep[16 * i + lc] == st.last);
        __syncthreads();
        if (w >= 3 && w < 6) {  // what passes from s to t: M F d without F's decay, summed for every step between
            const f32x4 v = *(const f32x4*)(sm + tm * LQ + q0) * f * *(const f32x4*)(st.d + q0);
            f32x4 pre;  // sums over s up to q0 + j
            float run = 0.0f;
#pragma unroll
            for (int j = 0; j < 4; ++j) pre[j] = run += tm > q0 + j ? v[j] : 0.0f;
            const float up = __shfl_up(run, 16, 64);  // and of the lanes with lower s
            float low = lg > 0 ? up : 0.0f;
            const float up2 = __shfl_up(low + run, 32, 64);
            if (lg > 1) low += up2;
            pre += low;
            if (si == ti) {
                // step q0 + j + 1 of this half: sum over t from it on
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float u = sum16(tm > q0 + j ? pre[j] : 0.0f);
                    if (lc == 0 && (q0 + j + 1) % 16) pairs[2 * si][q0 + j + 1] = u;
                }
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) {  // every t is behind step q0 + j + 1
                    const float u = sum16(pre[j]);
                    if (lc == 0) pairs[1][q0 + j + 1] = u;
                }
                float u = __shfl(pre[3], 48 + lc, 64);  // all s, and t from a step of the second half on
                for (int o = 1; o < 16; o <<= 1) {
                    const float down = __shfl_down(u, o, 16);
                    if (lc + o < 16) u += down;
                }
                if (lg == 0 && lc > 0) pairs[1][tm] = u;
            }
        }
        // dx's part for the steps of the wave with the other half of the states
        f32x4* const swap = (f32x4*)sr;
        if (on) swap[w * 64 + l] = half ? xa[0] : xa[1];
        f32x4 xo = half ? xa[1] : xa[0];
#pragma unroll
        for (int u = 0; u < JOBS; ++u) {
            if (w >= 2 * NT) break;
            const bool of_r = NT == 8 ? u : w >= NT;
            const int n = NT == 8 ? w : w % NT, n0 = 16 * n + 4 * lg;
            const float* own = of_r ? sc : sb;
            const f32x4 low = rfrag(own, LN, 0, 16 * n, l), high = rfrag(own, LN, 16, 16 * n, l);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int t = 16 * i + lc;
                f32x4 a = ja[u][i];
                const f32x4 v = *(const f32x4*)((of_r ? sb : sc) + t * LN + n0);
                float h = (a[0] * v[0] + a[1] * v[1]) + (a[2] * v[2] + a[3] * v[3]), bq = 0.0f;
                if (of_r) {  // the steps from this one on
                    if (i) a = mul1<T, FP32>(high, rfrag(sf, LQ, 16, 16, l), a);
                    else a = mul2<T, FP32>(low, high, rfrag(sf, LQ, 0, 0, l), rfrag(sf, LQ, 16, 0, l), a);
                    bq = (a[0] * v[0] + a[1] * v[1]) + (a[2] * v[2] + a[3] * v[3]);
                } else {  // the steps up to this one
                    auto fd = [&](int k) { return kfrag(sf, LQ, 16 * i, 16 * k, l) * *(const f32x4*)(st.d + 16 * k + 4 * lg); };
                    if (i) a = mul2<T, FP32>(low, high, fd(0), fd(1), a);
                    else a = mul1<T, FP32>(low, fd(0), a);
                }
                h = sum_rows(h);
                if (of_r) bq = sum_rows(bq);
                if (lg == 0) {
                    (of_r ? kb : hc)[n][t] = h;
                    if (of_r) qb[n][t] = bq;
                }
                if (t < len && n0 < s.N) {
                    const int at_q = t0 % Q + t;  // in its chunk
                    float* o = (of_r ? s.pdb : s.pdc) + part0 + t0 / Q * part_step;
                    *((f32x4*)o + ((at_q / 16 * NT + n) * 64 + 16 * lg + at_q % 16)) = of_r ? a * st.d[t] : a;
                }
            }
        }
        if (half)
            xo = mul1<T, FP32>(rfrag(sdy, LP, 16, 16 * wp, l), rfrag(sm, LQ, 16, 16, l), xo);
        else
            xo = mul2<T, FP32>(rfrag(sdy, LP, 0, 16 * wp, l), rfrag(sdy, LP, 16, 16 * wp, l), rfrag(sm, LQ, 0, 0, l), rfrag(sm, LQ, 16, 0, l), xo);
        pass = sum64(pass);
        if (l == 0) inner[w] = pass;
        if (on) walk<T, TILES, false>(R, sc + n_own, LN, sdy + 16 * wp, st, l);
        __syncthreads();
        {  // dx
            const int t = 16 * half + lc, p = 16 * wp + 4 * lg;
            if (Half<NT>::on(1 - half)) xo += swap[(w ^ 4) * 64 + l];
            const f32x4 yv = *(const f32x4*)(sdy + t * LP + p), xv = *(const f32x4*)(sx + t * LP + p);
            skip_sum += (yv[0] * xv[0] + yv[1] * xv[1]) + (yv[2] * xv[2] + yv[3] * xv[3]);
            if (t < len && p < at.pw) row_store<VEC>(dx + (t0 + t) * yt + p, xo * st.d[t] + skip * yv, at.pw - p);
        }
        if (w == 6) {
            past_d = st.d[l & (Q - 1)];
            past_all = st.last ? -1.0f : st.all;
            past_t = t0;
            past_len = len;
        }
        if (whole) {
            __syncthreads();
            if (tid == 0) flag = 0;
        }
    }
    if (w == 6 && past_len) finish(lane);
    if (on && s.dstate && at.seg == 0) store_state<TILES, VEC>(R, s.dstate + in.state, s.N, at.pw, s.N, 16 * wp, n_own, lane);
    skip_sum = sum64(skip_sum);
    decay_sum = sum64(decay_sum);
    bias_sum = sum64(bias_sum);
    __syncthreads();
    if (lane == 0) inner[w] = skip_sum;
    __syncthreads();
    if (tid == THREADS - 128) {  // of wave 6
        float* o = s.ppar + (((int64_t)at.b * s.nseg + at.seg) * s.vh + at.v) * 3;
        o[0] = decay_sum;
        o[1] = bias_sum;
        o[2] = ((inner[0] + inner[1]) + (inner[2] + inner[3])) + ((inner[4] + inner[5]) + (inner[6] + inner[7]));
    }
}

// Sums the workgroups' parts, in order: of db and dc over the heads of a group,
// of ddt over a head's tiles (blockIdx.y = 0), and of the parameters over sequences
// and segments (blockIdx.y = 1: a wave a head).
template <class T, bool VEC>
__global__ __launch_bounds__(256) void scan_reduce_kernel(ScanView s, T* db, T* dc, T* ddt, float* da_log, float* ddt_bias,
                                                          float* dskip) {
    if (blockIdx.y == 1) {
        const int h = blockIdx.x * 4 + (threadIdx.x >> 6), l = threadIdx.x & 63;
        if (h >= s.H) return;
        float a[3] = {0.0f, 0.0f, 0.0f};
        const int parts = s.B * s.nseg * s.ptiles;
        for (int i = l; i < parts; i += 64) {
            const float* p = s.ppar + ((int64_t)(i / s.ptiles) * s.vh + h * s.ptiles + i % s.ptiles) * 3;
            a[0] += p[0];
            a[1] += p[1];
            a[2] += p[2];
        }
        for (int o = 32; o; o >>= 1)
            for (int j = 0; j < 3; ++j) a[j] += __shfl_xor(a[j], o, 64);
        if (l == 0) {
            da_log[h] = a[0];
            ddt_bias[h] = a[1];
            dskip[h] = a[2];
        }
        return;
    }
    const int heads = s.vh / s.G, tiles = (s.N + 15) / 16, nt = padded_state(s.N) / 16;
    const int64_t rows = (int64_t)s.B * s.T, total = (int64_t)s.B * s.nch * s.G * (Q / 16) * tiles * 64, part = Q * nt * 4;
    for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < total; e += (int64_t)gridDim.x * 256) {
        const int l = (int)(e & 63), i = (int)(e / 64 / tiles % (Q / 16)), n = (int)(e / 64 % tiles);
        const int64_t r = e / 64 / tiles / (Q / 16), bk = r / s.G;  // (sequence, chunk)
        const int g = (int)(r % s.G), n0 = 16 * n + 4 * (l >> 4);
        const int64_t t = bk % s.nch * Q + 16 * i + (l & 15);
        if (t >= s.T || n0 >= s.N) continue;
        const int64_t o = (bk * s.vh + (int64_t)g * heads) * part + (i * nt + n) * 64 + l;
        f32x4 b{0.0f, 0.0f, 0.0f, 0.0f}, c = b;
        for (int k = 0; k < heads; ++k) {
            b += ((const f32x4*)s.pdb)[o + k * part];
            c += ((const f32x4*)s.pdc)[o + k * part];
        }
        const int64_t to = ((bk / s.nch * s.T + t) * s.G + g) * s.N + n0;
        row_store<VEC>(db + to, b, s.N - n0);
        row_store<VEC>(dc + to, c, s.N - n0);
    }
    for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < rows * s.H; e += (int64_t)gridDim.x * 256) {
        float d = 0.0f;
        for (int i = 0; i < s.ptiles; ++i) d += s.pdt[e * s.ptiles + i];
        ddt[e] = row_round<T>(d);
    }
}

// One step of a row and head: memory bound on the state, read and written once.  A
// workgroup takes 256 / L channels at a time, L = lanes of a channel's states.  1024
// rows, 16 heads of 64, state 64: 125 us, 4.35 TB/s (a large copy: 4.8).
template <class T, bool VEC>
__global__ __launch_bounds__(256) void scan_step_kernel(ScanView s, float* pool, int64_t slots, const int32_t* slot, int lanes,
                                                        int pblocks, unsigned* err) {
    constexpr int V = VEC ? 4 : 1;
    const int id = blockIdx.x, pb = id % pblocks, h = id / pblocks % s.H, row = id / pblocks / s.H;
    const int grp = h / (s.H / s.G), l = threadIdx.x % lanes;
    const T* x = of<T>(s.x, row * s.xb + (int64_t)h * s.P);
    const T* bm = of<T>(s.b, row * s.bb + (int64_t)grp * s.N);
    const T* cm = of<T>(s.c, row * s.cb + (int64_t)grp * s.N);
    const float v = row_value(of<T>(s.dt, row * s.dtb)[h]) + s.dt_bias[h];
    float d = fmaxf(v, 0.0f) + log1pf(expf(-fabsf(v)));
    if (v != v) d = v;
    const float a = expf(-expf(s.a_log[h]) * d), skip = s.skip[h];
    bool reset = s.reset && s.reset[row];
    int64_t at = slot ? slot[row] : row;
    const bool out = at < 0 || at >= slots;
    if (out) {
        if (threadIdx.x == 0 && err) atomicOr(err, ERR_IDX_RANGE);
        reset = true;
        at = 0;
    }
    float* st = pool + (at * s.H + h) * (int64_t)s.P * s.N;
    T* y = (T*)s.y + ((int64_t)row * s.H + h) * s.P;
    const int per = (s.P + pblocks - 1) / pblocks, p1 = (pb + 1) * per < s.P ? (pb + 1) * per : s.P;
    for (int p = pb * per + threadIdx.x / lanes; p < p1; p += 256 / lanes) {
        const float xv = row_value(x[p]), dxv = d * xv;
        float sum = 0.0f;
        for (int n = l * V; n < s.N; n += lanes * V) {
            float* e = st + (int64_t)p * s.N + n;
            float o[V], bv[V], cv[V];
            if (VEC) {
                const f32x4 ov = reset ? f32x4{0.0f, 0.0f, 0.0f, 0.0f} : *(const f32x4*)e, b4 = row_load4(bm + n), c4 = row_load4(cm + n);
                for (int j = 0; j < V; ++j) o[j] = ov[j], bv[j] = b4[j], cv[j] = c4[j];
            } else {
                o[0] = reset ? 0.0f : *e;
                bv[0] = row_value(bm[n]);
                cv[0] = row_value(cm[n]);
            }
#pragma unroll
            for (int j = 0; j < V; ++j) {
                o[j] = reset ? dxv * bv[j] : fmaf(a, o[j], dxv * bv[j]);
                sum = fmaf(o[j], cv[j], sum);
            }
            if (!out) {
                if (VEC) *(f32x4*)e = f32x4{o[0], o[V > 1 ? 1 : 0], o[V > 2 ? 2 : 0], o[V > 3 ? 3 : 0]};
                else *e = o[0];
            }
        }
        for (int m = lanes >> 1; m; m >>= 1) sum += __shfl_xor(sum, m, 64);
        if (l == 0) y[p] = row_round<T>(fmaf(skip, xv, sum));
    }
}

// ---- host ----

// Segments a sequence is cut into: none where the (sequence, head, channels) fill
// the chip, else enough for two workgroups a compute unit, of one chunk at least.
constexpr int FULL = 512;  // workgroups that fill it
// Chunks of sequences that a forward call walks in one segment where the workspace has
// no place for more: the contexts of uncut calls have none, and take smaller ones too.
constexpr int SHORT = 4;
struct Cut {
    int ptiles, vh, nch, cps, nseg;
    Cut(int B, int T, int H, int P) {
        ptiles = (P + PW - 1) / PW;
        vh = H * ptiles;
        nch = (T + Q - 1) / Q;
        const int64_t groups = (int64_t)B * vh;
        const int want = groups > 0 && groups < FULL ? (int)((FULL + groups - 1) / groups) : 1;
        nseg = want < nch ? want : nch;
        if (nseg < 1) nseg = 1;
        cps = nch > 0 ? (nch + nseg - 1) / nseg : 1;
        nseg = nch > 0 ? (nch + cps - 1) / cps : 1;
    }
    void whole() { nseg = 1, cps = nch > 0 ? nch : 1; }
    // Segments of B sequences that have states in the workspace.
    size_t joined(int B) const { return nseg > 1 ? (size_t)B * nseg * vh : 0; }
    // The most of them in any call of up to B sequences of up to nch chunks: calls of
    // g < FULL workgroups are cut, into less than FULL + g segments in all.
    size_t most_joined(int B) const {
        const size_t groups = (size_t)B * vh, cut = groups < FULL ? groups : FULL - 1, all = cut * nch;
        return nch <= 1 ? 0 : all < 2 * FULL ? all : 2 * FULL;
    }
};
struct ScanPlan {
    size_t seg_s, seg_r, seg_a, chunk_s, pdb, pdc, pdt, ppar, total;
    // joined: states of segments; walks: workgroups that walk one.
    ScanPlan(const Cut& k, size_t joined, size_t walks, int B, int T, int N, bool backward) {
        size_t o = 0;
        auto take = [&](size_t floats) { size_t at = o; o += (floats * 4 + 255) / 256 * 256; return at; };
        const size_t state = (size_t)PW * padded_state(N), rows = (size_t)B * T * k.vh;
        seg_s = take(joined * state);
        seg_a = take(joined);
        seg_r = take(backward ? joined * state : 0);
        chunk_s = take(backward ? (size_t)B * k.nch * k.vh * state : 0);
        const size_t parts = backward ? (size_t)B * k.nch * k.vh * Q * padded_state(N) : 0;
        pdb = take(parts);
        pdc = take(parts);
        pdt = take(backward ? rows : 0);
        ppar = take(backward ? walks * 3 : 0);
        total = o;
    }
    ScanPlan(const Cut& k, int B, int T, int N, bool backward)
        : ScanPlan(k, k.joined(B), (size_t)B * k.nseg * k.vh, B, T, N, backward) {}
};

constexpr int MAX_WIDTH = 128, MAX_STATE = 128;
// Sequences and steps whose sums with a segment's are 32 bits.
bool sizes_fit(int batch, int length) { return length <= 1 << 30 && (int64_t)batch * length <= INT32_MAX; }

// The view of valid arguments; `step`: strides along the steps are not used.
int scan_view(const gorila_scan_args* a, bool step, ScanView& v, bool& vec) {
    if (!a || !row_dtype(a->dtype) || a->batch < 0 || a->length < 0 || a->heads < 1 || a->groups < 1) return GORILA_EINVAL;
    if (a->heads % a->groups || a->head_dim < 1 || a->state_dim < 1) return GORILA_EINVAL;
    if (a->head_dim > MAX_WIDTH || a->state_dim > MAX_STATE || a->heads > 65536) return GORILA_EUNSUPPORTED;
    if (!sizes_fit(a->batch, a->length)) return GORILA_EUNSUPPORTED;
    if (!a->a_log || !a->dt_bias || !a->skip) return GORILA_EINVAL;
    if (a->batch > 0 && a->length > 0 && (!a->x || !a->dt || !a->b || !a->c)) return GORILA_EINVAL;
    const int e = dtype_bytes(a->dtype);
    for (const void* p : {a->x, a->dt, a->b, a->c})
        if (!at_element(p, e)) return GORILA_EINVAL;
    for (const void* p : {a->a_log, a->dt_bias, a->skip, a->state})
        if (!at_element(p, 4)) return GORILA_EINVAL;
    v = ScanView{};
    v.x = a->x, v.dt = a->dt, v.b = a->b, v.c = a->c;
    v.xb = a->x_batch_stride, v.xt = a->x_step_stride, v.dtb = a->dt_batch_stride, v.dtt = a->dt_step_stride;
    v.bb = a->b_batch_stride, v.bt = a->b_step_stride, v.cb = a->c_batch_stride, v.ct = a->c_step_stride;
    v.a_log = a->a_log, v.dt_bias = a->dt_bias, v.skip = a->skip, v.state = a->state, v.reset = a->reset;
    v.B = a->batch, v.T = a->length, v.H = a->heads, v.P = a->head_dim, v.G = a->groups, v.N = a->state_dim;
    const int64_t strides = v.xb | v.bb | v.cb | (step ? 0 : v.xt | v.bt | v.ct);
    vec = !((v.P | v.N) & 3) && !(strides & 3) && at_four(a->x, e) && at_four(a->b, e) && at_four(a->c, e) && at_four(a->state, 4);
    return GORILA_OK;
}

void cut_view(ScanView& v, const Cut& k) {
    v.ptiles = k.ptiles, v.vh = k.vh, v.nch = k.nch, v.cps = k.cps, v.nseg = k.nseg;
}

template <class F>
void by_state(int n, F&& f) {
    switch (padded_state(n)) {
        case 16: f(std::integral_constant<int, 16>{}); break;
        case 32: f(std::integral_constant<int, 32>{}); break;
        case 64: f(std::integral_constant<int, 64>{}); break;
        default: f(std::integral_constant<int, 128>{}); break;
    }
}
// Calls f(row type, padded state, whether quads are aligned) as constants.
template <class F>
void by_kind(int dtype, int n, bool vec, F&& f) {
    by_state(n, [&](auto np) {
        if (dtype == GORILA_F32) vec ? f(float{}, np, std::true_type{}) : f(float{}, np, std::false_type{});
        else vec ? f(uint16_t{}, np, std::true_type{}) : f(uint16_t{}, np, std::false_type{});
    });
}

}  // namespace
}  // namespace gorila

using namespace gorila;

extern "C" {

size_t gorila_scan_workspace_bytes(int32_t batch, int32_t length, int32_t heads, int32_t head_dim, int32_t groups,
                                   int32_t state_dim, int32_t backward) {
    if (batch < 0 || length < 0 || heads < 1 || heads > 65536 || groups < 1 || heads % groups) return 0;
    if (head_dim < 1 || head_dim > MAX_WIDTH || state_dim < 1 || state_dim > MAX_STATE || !sizes_fit(batch, length)) return 0;
    const Cut k(batch, length, heads, head_dim);
    // enough for every smaller batch and length too, which may be cut where this is not
    const bool exact = !backward && k.nch <= SHORT;
    const size_t joined = exact ? k.joined(batch) : k.most_joined(batch), all = (size_t)batch * k.vh;
    const size_t own = ScanPlan(k, joined, joined > all ? joined : all, batch, length, state_dim, backward != 0).total;
    return own ? WS_FIXED_BYTES + own : 0;
}

int gorila_scan(const gorila_scan_args* args, void* y, float* state_out, gorila_ctx* ctx) {
    ScanView v;
    CtxView c;
    bool vec;
    int rc = ctx_view(ctx, 0, c);
    if (rc || (rc = scan_view(args, false, v, vec))) return rc;
    if (v.B == 0 || (v.T == 0 && !state_out)) return GORILA_OK;
    if ((v.T > 0 && !y) || !at_element(y, dtype_bytes(args->dtype)) || !at_element(state_out, 4)) return GORILA_EINVAL;
    Cut k(v.B, v.T, v.H, v.P);
    if (k.nch <= SHORT && ctx_view(ctx, ScanPlan(k, v.B, v.T, v.N, false).total, c) == GORILA_EWORKSPACE) k.whole();
    const ScanPlan p(k, v.B, v.T, v.N, false);
    cut_view(v, k);
    const int64_t blocks = (int64_t)v.B * v.nseg * v.vh;
    if (!launch_fits((double)blocks, THREADS)) return GORILA_EUNSUPPORTED;
    if ((rc = ctx_view(ctx, p.total, c))) return rc;
    vec = vec && at_four(y, dtype_bytes(args->dtype)) && at_four(state_out, 4);
    v.y = y;
    v.state_out = state_out;
    v.seg_s = (float*)(c.ws + p.seg_s);
    v.seg_a = (float*)(c.ws + p.seg_a);
    by_kind(args->dtype, v.N, vec, [&](auto t, auto np, auto al) {
        using T = decltype(t);
        constexpr int NP = decltype(np)::value;
        constexpr bool VEC = decltype(al)::value;
        if (v.nseg > 1) {
            state_kernel<T, NP, VEC><<<(unsigned)blocks, THREADS, 0, c.stream>>>(v);
            join_kernel<NP, VEC><<<dim3((unsigned)(v.B * v.vh * (PW * NP / 256)), 1), 256, 0, c.stream>>>(v);
        }
        scan_kernel<T, NP, VEC><<<(unsigned)blocks, THREADS, 0, c.stream>>>(v);
    });
    return launched();
}

int gorila_scan_backward(const gorila_scan_args* args, const void* dy, int64_t dy_batch_stride, int64_t dy_step_stride,
                         const float* dstate_out, void* dx, void* ddt, void* db, void* dc, float* da_log, float* ddt_bias,
                         float* dskip, float* dstate, gorila_ctx* ctx) {
    ScanView v;
    CtxView c;
    bool vec;
    int rc = ctx_view(ctx, 0, c);
    if (rc || (rc = scan_view(args, false, v, vec))) return rc;
    const int e = dtype_bytes(args->dtype);
    if (!da_log || !ddt_bias || !dskip) return GORILA_EINVAL;
    if (v.B > 0 && v.T > 0 && (!dy || !dx || !ddt || !db || !dc)) return GORILA_EINVAL;
    for (const void* p : {dy, (const void*)dx, (const void*)ddt, (const void*)db, (const void*)dc})
        if (!at_element(p, e)) return GORILA_EINVAL;
    for (const float* p : {dstate_out, (const float*)da_log, (const float*)ddt_bias, (const float*)dskip, (const float*)dstate})
        if (!at_element(p, 4)) return GORILA_EINVAL;
    const Cut k(v.B, v.T, v.H, v.P);
    const ScanPlan p(k, v.B, v.T, v.N, true);
    cut_view(v, k);
    const int64_t blocks = (int64_t)v.B * v.nseg * v.vh;
    if (!launch_fits((double)blocks, THREADS)) return GORILA_EUNSUPPORTED;
    if ((rc = ctx_view(ctx, p.total, c))) return rc;
    vec = vec && !((dy_batch_stride | dy_step_stride) & 3) && at_four(dy, e) && at_four(dx, e) && at_four(db, e) && at_four(dc, e) && at_four(dstate_out, 4) && at_four(dstate, 4);
    v.dy = dy;
    v.dyb = dy_batch_stride;
    v.dyt = dy_step_stride;
    v.dstate_out = dstate_out;
    v.dx = dx;
    v.dstate = dstate;
    auto ws = [&](size_t o) { return (float*)(c.ws + o); };
    v.seg_s = ws(p.seg_s), v.seg_a = ws(p.seg_a), v.seg_r = ws(p.seg_r), v.chunk_s = ws(p.chunk_s);
    v.pdb = ws(p.pdb), v.pdc = ws(p.pdc), v.pdt = ws(p.pdt), v.ppar = ws(p.ppar);
    by_kind(args->dtype, v.N, vec, [&](auto t, auto np, auto al) {
        using T = decltype(t);
        constexpr int NP = decltype(np)::value;
        constexpr bool VEC = decltype(al)::value;
        if (blocks > 0) {
            if (v.nseg > 1) {
                state_kernel<T, NP, VEC><<<dim3((unsigned)blocks, 2), THREADS, 0, c.stream>>>(v);
                join_kernel<NP, VEC><<<dim3((unsigned)(v.B * v.vh * (PW * NP / 256)), 2), 256, 0, c.stream>>>(v);
            }
            scan_backward_kernel<T, NP, VEC><<<(unsigned)blocks, THREADS, 0, c.stream>>>(v);
        }
        const int64_t quads = (int64_t)v.B * v.nch * v.G * (Q / 16) * ((v.N + 15) / 16) * 64;
        const int64_t least = (int64_t)v.B * v.T * v.H, per = ((quads > least ? quads : least) + 255) / 256, heads = (v.H + 3) / 4;
        const unsigned gx = (unsigned)(per > 8192 ? 8192 : per);
        scan_reduce_kernel<T, VEC><<<dim3(gx > heads ? gx : (unsigned)heads, 2), 256, 0, c.stream>>>(v, (T*)db, (T*)dc, (T*)ddt, da_log,
                                                                                                   ddt_bias, dskip);
    });
    return launched();
}

int gorila_scan_step(const gorila_scan_args* args, float* state_pool, int64_t slots, const int32_t* slot, void* y,
                     gorila_ctx* ctx) {
    ScanView v;
    CtxView c;
    bool vec;
    int rc = ctx_view(ctx, 0, c);
    if (rc || (rc = scan_view(args, true, v, vec))) return rc;
    if (v.T != 1 || slots < 0) return GORILA_EINVAL;
    if (v.B == 0) return GORILA_OK;
    if (!state_pool || !y || !at_element(state_pool, 4) || !at_element(y, dtype_bytes(args->dtype)) || !at_element(slot, 4))
        return GORILA_EINVAL;
    if (slot ? !c.err : slots < v.B) return slot ? GORILA_EWORKSPACE : GORILA_EINVAL;
    vec = vec && at_four(state_pool, 4);
    v.y = y;
    // lanes of a channel: its quads, up to a wave; channels over more workgroups
    // while there are fewer of them than compute units
    int lanes = 1;
    while (lanes < 64 && lanes * (vec ? 4 : 1) < v.N) lanes <<= 1;
    const int most = (v.P * lanes + 255) / 256;
    int pblocks = 1;
    while (pblocks < most && (int64_t)v.B * v.H * pblocks < 2 * c.cus) pblocks <<= 1;
    if (pblocks > most) pblocks = most;
    const int64_t blocks = (int64_t)v.B * v.H * pblocks;
    if (!launch_fits((double)blocks, 256)) return GORILA_EUNSUPPORTED;
    auto go = [&](auto t, auto al) {
        scan_step_kernel<decltype(t), decltype(al)::value><<<(unsigned)blocks, 256, 0, c.stream>>>(v, state_pool, slots, slot, lanes, pblocks, c.err);
    };
    if (args->dtype == GORILA_F32) vec ? go(float{}, std::true_type{}) : go(float{}, std::false_type{});
    else vec ? go(uint16_t{}, std::true_type{}) : go(uint16_t{}, std::false_type{});
    return launched();
}

}  // extern "C"
