// Norms before and after a block, with the block's gate, its residual scale and the residual stream, forward and backward:
//     y = N_post(a) p + p_bias,   h = x + alpha s sigmoid(t) y,   u = N_pre(h) q + q_bias.
// Statistics, sums and the row itself in 32 bits, each output rounded once.  Bound by memory: forward 3.1 M x 256 bf16 1.29 ms, 6.2 TB/s of
// the 8.0 GB that it has to move (a copy of 4 GB goes at 5.6); backward 600,000 x 256 floats 0.87 ms, 5.6 TB/s of 4.9 GB.
#include <float.h>

#include <algorithm>
#include <type_traits>

#include "common.h"
#include "norm_layout.h"
#include "wave.h"

namespace gas {
namespace {

struct ResidualNorm {
    const char *X, *A, *T;
    int64_t ldx, lda, ldt;
    int gate_cols;                       // 0: no gate, 1: one gate of a row, F: one of every element
    int64_t n;
    int F, post, pre;
    const float *p, *p_bias, *s, *q, *q_bias;
    float alpha, eps;
    char *H, *U;
    int64_t ldh, ldu;
    float* stats;                        // [n][4]: mean and 1 / deviation of a, and of h
    const int32_t* idx;
    char* hist;
    int64_t ld_hist;
    int turns;                           // of a workgroup, RowLanes::kRows rows each
};

template <bool BF>
__device__ __forceinline__ float load_one(const char* p, int64_t i) {
    if constexpr (BF) return __uint_as_float((uint32_t)reinterpret_cast<const uint16_t*>(p)[i] << 16);
    else return reinterpret_cast<const float*>(p)[i];
}
template <bool BF>
__device__ __forceinline__ void store_one(char* p, int64_t i, float v) {
    if constexpr (BF) reinterpret_cast<uint16_t*>(p)[i] = (uint16_t)f32_to_bf16(v);
    else reinterpret_cast<float*>(p)[i] = v;
}
__device__ __forceinline__ float at(const float* v, int f, float otherwise) { return v ? v[f] : otherwise; }

// A gate, g = 1 / (1 + z) with z = exp(-t), and 1 - g = z g, which has its own digits: the difference from 1 has none left where the gate is open
// (1e-3 of it off at t = 10, 0 from t = 17 on).  Where z is an infinity g is 0, and so is every gradient that goes with g (1 - g).
struct Gate { float g, rest; };
__device__ __forceinline__ Gate gate_from(float z, float g) { return {g, fminf(z, FLT_MAX) * g}; }
__device__ __forceinline__ Gate gate_of(float t) {
    const float z = expf(-t);
    return gate_from(z, 1.f / (1.f + z));
}

// Mean and 1 / deviation over the F values that value(f) gives, the same in every lane.
template <class V>
__device__ __forceinline__ void row_stats(int kind, int F, float eps, V value, float* mean, float* r) {
    const int lane = threadIdx.x & 63;
    *mean = 0.f;
    *r = 1.f;
    if (kind == GAS_NORM_NONE) return;
    if (kind == GAS_NORM_LAYER) {
        float sum = 0.f;
        for (int f = lane; f < F; f += 64) sum += value(f);
        *mean = wave_sum(sum) / (float)F;
    }
    float sq = 0.f;
    for (int f = lane; f < F; f += 64) {
        const float d = value(f) - *mean;
        sq = fmaf(d, d, sq);
    }
    *r = 1.f / sqrtf(wave_sum(sq) / (float)F + eps);
}

// Rows that do not fit the registers: a wavefront to a row, element by element, read anew for every sum.
template <bool BF>
__global__ __launch_bounds__(256) void residual_norm_kernel(ResidualNorm c) {
    const int lane = threadIdx.x & 63;
    const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (row >= c.n) return;
    float mean_a = 0.f, r_a = 1.f, mean_h, r_h;
    if (c.A) row_stats(c.post, c.F, c.eps, [&](int f) { return load_one<BF>(c.A, row * c.lda + f); }, &mean_a, &r_a);
    const float row_gate = c.gate_cols == 1 ? gate_of(load_one<BF>(c.T, row * c.ldt)).g : 1.f;
    auto h_of = [&](int f) {
        const float x = load_one<BF>(c.X, row * c.ldx + f);
        if (!c.A) return x;
        const float y = fmaf((load_one<BF>(c.A, row * c.lda + f) - mean_a) * r_a, at(c.p, f, 1.f), at(c.p_bias, f, 0.f));
        const float g = c.gate_cols > 1 ? gate_of(load_one<BF>(c.T, row * c.ldt + f)).g : row_gate;
        return fmaf(c.alpha * at(c.s, f, 1.f) * g, y, x);
    };
    row_stats(c.U || c.hist || c.stats ? c.pre : GAS_NORM_NONE, c.F, c.eps, h_of, &mean_h, &r_h);
    if (c.stats && lane < 4) c.stats[row * 4 + lane] = lane == 0 ? mean_a : lane == 1 ? r_a : lane == 2 ? mean_h : r_h;
    const int64_t to = c.hist ? c.idx[row] : 0;
    for (int f = lane; f < c.F; f += 64) {
        const float h = h_of(f);
        const float u = fmaf((h - mean_h) * r_h, at(c.q, f, 1.f), at(c.q_bias, f, 0.f));
        if (c.H) store_one<BF>(c.H, row * c.ldh + f, h);
        if (c.U) store_one<BF>(c.U, row * c.ldu + f, u);
        if (c.hist) store_one<BF>(c.hist, to * c.ld_hist + f, u);
    }
}

// ---- rows in registers
// Sum over aligned groups of G lanes, in every lane of the group, in the same order everywhere: data-parallel moves within 16 lanes,
// swaps of rows of 16 and of halves beyond.  Through LDS (shuffles) a step takes some 60 cycles, this way some 8.
template <int G>
__device__ __forceinline__ float group_sum(float v) {
    if constexpr (G >= 2) v += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0xB1, 0xf, 0xf, true));     // quad_perm 1 0 3 2
    if constexpr (G >= 4) v += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0x4E, 0xf, 0xf, true));     // quad_perm 2 3 0 1
    if constexpr (G >= 8) v += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0x141, 0xf, 0xf, true));    // row_half_mirror
    if constexpr (G >= 16) v += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0x140, 0xf, 0xf, true));   // row_mirror
    if constexpr (G >= 32) {
        const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(s[0]) + __uint_as_float(s[1]);
    }
    if constexpr (G >= 64) {
        const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(s[0]) + __uint_as_float(s[1]);
    }
    return v;
}
// The same over the lanes with the same place in their groups of G: what the groups of a wavefront have between them.
template <int G>
__device__ __forceinline__ float across_groups(float v) {
    if constexpr (G <= 1) v += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0x121, 0xf, 0xf, true));    // row_ror:1
    if constexpr (G <= 2) v += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0x122, 0xf, 0xf, true));    // row_ror:2
    if constexpr (G <= 4) v += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0x124, 0xf, 0xf, true));    // row_ror:4
    if constexpr (G <= 8) v += other_half(v);                                                                         // row_ror:8
    if constexpr (G <= 16) {
        const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(s[0]) + __uint_as_float(s[1]);
    }
    if constexpr (G <= 32) {
        const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(s[0]) + __uint_as_float(s[1]);
    }
    return v;
}

// How a row lies in the lanes: W = 1: in a team of G lanes, 64 / G rows to a wavefront, four wavefronts to a workgroup; W > 1: in the W
// wavefronts of a workgroup (G = 64).  A lane has P pieces of 16 bytes.  MASK: F is no multiple of a piece; the last piece is the
// row's last 16 bytes then, and what of them the piece before has already is left out of the sums.
template <bool BF, int G, int W, int P, bool MASK>
struct RowLanes {
    static constexpr int E = Elems<BF>::E, EB = BF ? 2 : 4;
    static constexpr int kThreads = W == 1 ? 256 : W * 64;
    static constexpr int kRows = W == 1 ? 4 * (64 / G) : 1;           // of a workgroup at a time
    static constexpr bool kTiny = MASK && G == 1;                     // a row is narrower than a piece: its elements are the piece's last ones, one by one
    static constexpr bool kAlone = G == 64;                           // a wavefront has one row at a time: the loop's bound is enough
    static_assert(W == 1 || G == 64, "several wavefronts have all of their lanes");
    int place, team, c[P], skip[P];      // place in the row's lanes, row among the wavefront's; a piece's first element, and its elements that another piece has
    bool on[P];                          // a lane behind the row's end loads its first piece and neither counts nor stores it
    __device__ __forceinline__ RowLanes(int F) {
        place = W == 1 ? threadIdx.x % G : threadIdx.x;
        team = W == 1 ? (threadIdx.x & 63) / G : 0;
#pragma unroll
        for (int i = 0; i < P; ++i) {
            const Piece piece = piece_of<E, MASK, P>(place + i * G * W, i, F);
            c[i] = piece.c; skip[i] = piece.skip; on[i] = piece.on;
        }
    }
    // the wavefront's first row: the same in all of its lanes, so addresses are a scalar's and a lane's 32 bits
    static __device__ __forceinline__ int64_t first(int turns) {
        return (int64_t)blockIdx.x * turns * kRows + (W == 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * (64 / G) : 0);
    }
    __device__ __forceinline__ auto offset(int64_t ld, int i) const {
        if constexpr (kTiny) return tiny_offset<EB>(team, ld, c[i]);
        else return piece_offset<EB>(team, ld, c[i]);
    }
    // 16 bytes of any alignment: the same load
    typedef u32x4 piece __attribute__((aligned(2)));
    __device__ __forceinline__ void load(const char* m, int64_t ld, int64_t base, u32x4 (&v)[P]) const {
#pragma unroll
        for (int i = 0; i < P; ++i) {
            const char* at = m + base * ld * EB + offset(ld, i);
            if constexpr (kTiny) {
                v[i] = u32x4{0u, 0u, 0u, 0u};
#pragma unroll
                for (int e = 1; e < E; ++e)
                    if (e >= skip[i]) {
                        if constexpr (BF) v[i][e >> 1] |= (uint32_t)reinterpret_cast<const uint16_t*>(at)[e] << (16 * (e & 1));
                        else v[i][e] = reinterpret_cast<const uint32_t*>(at)[e];
                    }
            } else {
                v[i] = __builtin_nontemporal_load(reinterpret_cast<const piece*>(at));
            }
        }
    }
    __device__ __forceinline__ void store(char* m, int64_t ld, int64_t base, const u32x4 (&v)[P]) const {
#pragma unroll
        for (int i = 0; i < P; ++i)
            if (on[i]) store_piece(m + base * ld * EB + offset(ld, i), i, v[i]);
    }
    __device__ __forceinline__ void store_at(char* m, int64_t ld, int64_t row, const u32x4 (&v)[P]) const {
#pragma unroll
        for (int i = 0; i < P; ++i)
            if (on[i]) store_piece(m + (row * ld + c[i]) * EB, i, v[i]);
    }
    // Where an output lies in its input, another wavefront may have stored what this lane then reads as the elements that it does not own:
    // across wavefronts it stores its own only.  Within one, all of a row is read before any of it is stored.
    __device__ __forceinline__ void store_piece(char* at, int i, const u32x4& v) const {
        if constexpr (MASK && (W > 1 || kTiny))
            if (skip[i]) {
#pragma unroll
                for (int e = 1; e < E; ++e)
                    if (e >= skip[i]) {
                        if constexpr (BF) reinterpret_cast<uint16_t*>(at)[e] = (uint16_t)(v[e >> 1] >> (16 * (e & 1)));
                        else reinterpret_cast<uint32_t*>(at)[e] = v[e];
                    }
                return;
            }
        __builtin_nontemporal_store(v, reinterpret_cast<piece*>(at));
    }
    __device__ __forceinline__ void vector(const float* v, float otherwise, float (&x)[P][E]) const {
        typedef f32x4 piece __attribute__((aligned(4)));
#pragma unroll
        for (int i = 0; i < P; ++i)
#pragma unroll
            for (int e = 0; e < E; e += 4) {
                f32x4 w = {otherwise, otherwise, otherwise, otherwise};
                if constexpr (kTiny) {
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (v && e + j >= skip[i]) w[j] = v[c[i] + e + j];
                } else if (v) {
                    w = *reinterpret_cast<const piece*>(v + c[i] + e);
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) x[i][e + j] = w[j];
            }
    }
    // the sum of x over the row's elements of this lane
    __device__ __forceinline__ float own(const float (&x)[P][E]) const {
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < P; ++i) {
            float part = 0.f;
#pragma unroll
            for (int e = 0; e < E; ++e) part += MASK && e < skip[i] ? 0.f : x[i][e];
            sum += on[i] ? part : 0.f;
        }
        return sum;
    }
    __device__ __forceinline__ float own_dot(const float (&x)[P][E], const float (&y)[P][E]) const {
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < P; ++i) {
            float part = 0.f;
#pragma unroll
            for (int e = 0; e < E; ++e) part = fmaf(MASK && e < skip[i] ? 0.f : x[i][e], y[i][e], part);
            sum += on[i] ? part : 0.f;
        }
        return sum;
    }
};

// The vectors of a row's columns, N of them, for the pieces of a lane: in its registers, or, where a lane has several pieces, in LDS (PARKED), from
// where they are read again for every row.
template <class L, int N, int P, int E, bool PARKED>
struct Vectors {
    float held[PARKED ? 1 : N][PARKED ? 1 : P][E];
    f32x4 (*parked)[64];                 // [N * P * E / 4][64]
    __device__ __forceinline__ void set(const L& lanes, int k, const float* v, float otherwise) {
        float x[P][E];
        lanes.vector(v, otherwise, x);
#pragma unroll
        for (int i = 0; i < P; ++i)
#pragma unroll
            for (int e = 0; e < E; ++e)
                if constexpr (!PARKED) held[k][i][e] = x[i][e];
                else if (e % 4 == 0 && threadIdx.x < 64) parked[(k * P + i) * (E / 4) + e / 4][threadIdx.x] = f32x4{x[i][e], x[i][e + 1], x[i][e + 2], x[i][e + 3]};
    }
    __device__ __forceinline__ void get(int k, int i, float (&x)[E]) const {
#pragma unroll
        for (int e = 0; e < E; ++e)
            if constexpr (!PARKED) x[e] = held[k][i][e];
            else x[e] = parked[(k * P + i) * (E / 4) + e / 4][threadIdx.x & 63][e % 4];
    }
};

// N sums over a row at once.  Several wavefronts hand their sums over in LDS, in two places by turns, so one barrier is enough: who writes
// a place again has passed the barrier behind its last reading.
template <int G, int W, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], float (*red)[3][16], int& turn) {
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = group_sum<G>(v[k]);
    if constexpr (W > 1) {
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int k = 0; k < N; ++k) red[turn][k][threadIdx.x >> 6] = v[k];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < N; ++k) {
            float sum = red[turn][k][0];
#pragma unroll
            for (int w = 1; w < W; ++w) sum += red[turn][k][w];
            v[k] = sum;
        }
        turn ^= 1;
    }
}
// exp(-t) as a power of 2: the exponent's rounding and that of its factor move it by up to |t| units (62 at |t| = 80), so it is multiplied by what they left out.
// Costs nothing beside memory: huge rows 1,283 us, without it 1,297, 19,997 x 1,433 bf16 backward 93.1 and 92.4.
__device__ __forceinline__ Gate fast_gate(float t) {
    const float u = t * -1.44269504f, left = fmaf(t, -1.92596299e-8f, fmaf(t, -1.44269504f, -u));
    const float rough = __builtin_amdgcn_exp2f(u);
    const float z = fabsf(t) <= 88.f ? fmaf(rough, left * 0.693147181f, rough) : rough;       // beyond it is an infinity or below the normal numbers
    return gate_from(z, __builtin_amdgcn_rcpf(1.f + z));
}

// z becomes what it is beyond its mean; returns 1 / deviation.
template <class L, int G, int W, int P, int E>
__device__ __forceinline__ float centre(const L& lanes, int kind, int F, float eps, float (&z)[P][E], float* mean, float (*red)[3][16], int& turn) {
    *mean = 0.f;
    if (kind == GAS_NORM_NONE) return 1.f;
    float sum[1];
    if (kind == GAS_NORM_LAYER) {
        sum[0] = lanes.own(z);
        row_sums<G, W>(sum, red, turn);
        *mean = sum[0] / (float)F;
#pragma unroll
        for (int i = 0; i < P; ++i)
#pragma unroll
            for (int e = 0; e < E; ++e) z[i][e] -= *mean;
    }
    sum[0] = lanes.own_dot(z, z);
    row_sums<G, W>(sum, red, turn);
    return rsqrtf(sum[0] / (float)F + eps);
}

// One pass over the rows: the next row of a team is on its way while this one is worked on.  ALL: x, a, h and u are there and no push,
// known beforehand.
template <bool BF, int G, int W, int P, bool MASK, bool ALL>
__global__ __launch_bounds__((RowLanes<BF, G, W, P, MASK>::kThreads)) void residual_norm_rows_kernel(ResidualNorm c) {
    using L = RowLanes<BF, G, W, P, MASK>;
    constexpr int E = L::E;
    __shared__ float red[2][3][16];
    int turn = 0;
    const L lanes(c.F);
    const bool has_a = ALL || c.A, has_h = ALL || c.H, has_u = ALL || c.U, push = !ALL && c.hist;
    const int64_t end = min(c.n, (int64_t)(blockIdx.x + 1) * c.turns * L::kRows);
    int64_t base = L::first(c.turns);
    u32x4 x[P], a[P], t[P];
    float t1;
    int32_t to = 0;
    auto fetch = [&](int64_t base) {
        const int64_t row = base + lanes.team;
        if (L::kAlone || row < c.n) {
            lanes.load(c.X, c.ldx, base, x);
            if (has_a) lanes.load(c.A, c.lda, base, a);
            if (c.gate_cols > 1) lanes.load(c.T, c.ldt, base, t);
            if (c.gate_cols == 1) t1 = load_one<BF>(c.T, row * c.ldt);
            if (push) to = c.idx[row];
        }
    };
    t1 = 0.f;
#pragma unroll
    for (int i = 0; i < P; ++i) x[i] = a[i] = t[i] = u32x4{0u, 0u, 0u, 0u};
    if (base < end) fetch(base);
    constexpr bool kParked = W == 1 && P > 1;
    __shared__ f32x4 parked[kParked ? 5 * P * E / 4 : 1][64];
    Vectors<L, 5, P, E, kParked> vec;
    vec.parked = parked;
    vec.set(lanes, 0, c.p, 1.f);
    vec.set(lanes, 1, c.p_bias, 0.f);
    vec.set(lanes, 2, c.s, 1.f);
    vec.set(lanes, 3, c.q, 1.f);
    vec.set(lanes, 4, c.q_bias, 0.f);
    if constexpr (kParked) __syncthreads();
    const bool normed = has_u || push || c.stats;
    for (; base < end; base += L::kRows) {
        if constexpr (kParked) asm volatile("" ::: "memory");        // what is parked stays there
        const bool live = L::kAlone || base + lanes.team < c.n;
        float h[P][E], y[P][E], g[P][E];
        const float gate = c.alpha * (c.gate_cols == 1 ? fast_gate(t1).g : 1.f);
        const int64_t place = to;
#pragma unroll
        for (int i = 0; i < P; ++i) {
            unpack<BF>(x[i], h[i]);
            unpack<BF>(a[i], y[i]);
            unpack<BF>(t[i], g[i]);
        }
        if (base + L::kRows < end) fetch(base + L::kRows);
        float mean_a = 0.f, r_a = 1.f, mean_h, r_h;
        if (has_a) {
            r_a = centre<L, G, W>(lanes, c.post, c.F, c.eps, y, &mean_a, red, turn);
            if (c.gate_cols > 1) {
#pragma unroll
                for (int i = 0; i < P; ++i)
#pragma unroll
                    for (int e = 0; e < E; ++e) g[i][e] = c.alpha * fast_gate(g[i][e]).g;
            } else {
#pragma unroll
                for (int i = 0; i < P; ++i)
#pragma unroll
                    for (int e = 0; e < E; ++e) g[i][e] = gate;
            }
#pragma unroll
            for (int i = 0; i < P; ++i) {
                float p[E], p_bias[E], s[E];
                vec.get(0, i, p);
                vec.get(1, i, p_bias);
                vec.get(2, i, s);
#pragma unroll
                for (int e = 0; e < E; ++e) h[i][e] = fmaf(g[i][e] * s[e], fmaf(y[i][e] * r_a, p[e], p_bias[e]), h[i][e]);
            }
        }
        u32x4 out[P];
        if (has_h && live) {
#pragma unroll
            for (int i = 0; i < P; ++i) out[i] = pack<BF>(h[i]);
            lanes.store(c.H, c.ldh, base, out);
        }
        if (!normed) continue;
        r_h = centre<L, G, W>(lanes, c.pre, c.F, c.eps, h, &mean_h, red, turn);
        if (!live) continue;
        if (c.stats && lanes.place == 0) reinterpret_cast<f32x4*>(c.stats)[base + lanes.team] = f32x4{mean_a, r_a, mean_h, r_h};
#pragma unroll
        for (int i = 0; i < P; ++i) {
            float q[E], q_bias[E];
            vec.get(3, i, q);
            vec.get(4, i, q_bias);
#pragma unroll
            for (int e = 0; e < E; ++e) h[i][e] = fmaf(h[i][e] * r_h, q[e], q_bias[e]);
            out[i] = pack<BF>(h[i]);
        }
        if (has_u) lanes.store(c.U, c.ldu, base, out);
        if (push) lanes.store_at(c.hist, c.ld_hist, place, out);
    }
}

// Backward.  With hn, an the normed rows, d = gu q, c = dy p and P the means of a layer norm (none otherwise):
//     gx = gh + r_h (d - P d - hn mean(d hn)),   dy = gx alpha s g,   ga = r_a (c - P c - an mean(c an)),
//     gt = dy y (1 - g), summed over the row for one gate of a row.
struct ResidualNormBwd {
    const char *GH, *GU, *H, *A, *T;
    int64_t ldgh, ldgu, ldh, lda, ldt;
    int gate_cols;
    const float* stats;
    int64_t n;
    int F, post, pre;
    const float *p, *p_bias, *s, *q;
    float alpha;
    char *GX, *GA, *GT;
    int64_t ldgx, ldga, ldgt;
    float* sums[5];                      // gradients of p, p_bias, s, q, q_bias, or null
    float* row_sums;                     // [n][2]: means of d and of d hn
    float* partials;                     // [slabs][5][F]
    int slabs, turns;
    int64_t rows_per_slab;
};

struct Element { float hn, gu, e, an, y, dy; Gate gate; };

// What one element's gradients are made of; d_mean, dh_mean: the row's means of d and d hn.
template <bool BF>
__device__ __forceinline__ Element element(const ResidualNormBwd& c, int64_t row, int f, const float* st, float d_mean, float dh_mean) {
    Element v;
    v.gu = c.GU ? load_one<BF>(c.GU, row * c.ldgu + f) : 0.f;
    v.hn = c.GU ? (load_one<BF>(c.H, row * c.ldh + f) - st[2]) * st[3] : 0.f;
    const float d = v.gu * at(c.q, f, 1.f);
    v.e = (c.GH ? load_one<BF>(c.GH, row * c.ldgh + f) : 0.f) + st[3] * (d - d_mean - v.hn * dh_mean);
    v.an = v.y = v.dy = 0.f;
    v.gate = {1.f, 0.f};
    if (c.A) {
        v.an = (load_one<BF>(c.A, row * c.lda + f) - st[0]) * st[1];
        v.y = fmaf(v.an, at(c.p, f, 1.f), at(c.p_bias, f, 0.f));
        if (c.gate_cols) v.gate = gate_of(load_one<BF>(c.T, row * c.ldt + (c.gate_cols == 1 ? 0 : f)));
        v.dy = v.e * c.alpha * at(c.s, f, 1.f) * v.gate.g;
    }
    return v;
}

template <bool BF>
__device__ __forceinline__ void row_stats_of(const ResidualNormBwd& c, int64_t row, float (&st)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) st[i] = c.stats ? c.stats[row * 4 + i] : (i & 1 ? 1.f : 0.f);
}

template <bool BF>
__global__ __launch_bounds__(256) void residual_norm_row_sums_kernel(ResidualNormBwd c) {
    const int lane = threadIdx.x & 63;
    const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (row >= c.n) return;
    float st[4], sd = 0.f, sdh = 0.f;
    row_stats_of<BF>(c, row, st);
    if (c.GU && c.pre != GAS_NORM_NONE)
        for (int f = lane; f < c.F; f += 64) {
            const Element v = element<BF>(c, row, f, st, 0.f, 0.f);
            const float d = v.gu * at(c.q, f, 1.f);
            sd += d;
            sdh = fmaf(d, v.hn, sdh);
        }
    sd = c.pre == GAS_NORM_LAYER ? wave_sum(sd) / (float)c.F : 0.f;
    sdh = wave_sum(sdh) / (float)c.F;
    if (lane < 2) c.row_sums[row * 2 + lane] = lane == 0 ? sd : sdh;
}

// Sums over a slab of rows for 64 columns: a lane has a column, the four wavefronts take the rows in turn.
template <bool BF>
__global__ __launch_bounds__(256) void residual_norm_columns_kernel(ResidualNormBwd c) {
    __shared__ float part[4][5][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int f = blockIdx.x * 64 + lane;
    const int64_t r0 = (int64_t)blockIdx.y * c.rows_per_slab, r1 = r0 + c.rows_per_slab < c.n ? r0 + c.rows_per_slab : c.n;
    float sum[5] = {0.f, 0.f, 0.f, 0.f, 0.f};
    if (f < c.F)
        for (int64_t row = r0 + wave; row < r1; row += 4) {
            float st[4];
            row_stats_of<BF>(c, row, st);
            const Element v = element<BF>(c, row, f, st, c.row_sums[row * 2], c.row_sums[row * 2 + 1]);
            sum[0] = fmaf(v.dy, v.an, sum[0]);
            sum[1] += v.dy;
            sum[2] = fmaf(v.e * c.alpha * v.gate.g, v.y, sum[2]);
            sum[3] = fmaf(v.gu, v.hn, sum[3]);
            sum[4] += v.gu;
        }
#pragma unroll
    for (int k = 0; k < 5; ++k) part[wave][k][lane] = sum[k];
    __syncthreads();
    if (wave == 0 && f < c.F)
#pragma unroll
        for (int k = 0; k < 5; ++k)
            c.partials[((int64_t)blockIdx.y * 5 + k) * c.F + f] = (part[0][k][lane] + part[1][k][lane]) + (part[2][k][lane] + part[3][k][lane]);
}

// The backward pass with the row in registers: every matrix is read once and written once, and a lane keeps the sums of its columns
// over all rows that it takes.  ALL: every input and output is there but the gate's, known beforehand.
template <bool BF, int G, int W, int P, bool MASK, bool ALL>
__global__ __launch_bounds__((RowLanes<BF, G, W, P, MASK>::kThreads)) void residual_norm_bwd_rows_kernel(ResidualNormBwd c) {
    using L = RowLanes<BF, G, W, P, MASK>;
    constexpr int E = L::E;
    __shared__ float red[2][3][16];
    constexpr int kAtOnce = P == 1 ? 5 : 1;              // vectors of sums that share a barrier: 40 KB at most
    __shared__ float columns[W == 1 ? 4 : 1][W == 1 ? kAtOnce : 1][W == 1 ? G * P * E : 1];
    int turn = 0;
    const L lanes(c.F);
    const bool has_gh = ALL || c.GH, has_gu = ALL || c.GU, has_a = ALL || c.A, has_gx = ALL || c.GX, has_ga = ALL || c.GA, has_stats = ALL || c.stats;
    const int64_t end = min(c.n, (int64_t)(blockIdx.x + 1) * c.turns * L::kRows);
    int64_t base = L::first(c.turns);
    u32x4 gh[P], gu[P], h[P], a[P], t[P];
    f32x4 st = {0.f, 1.f, 0.f, 1.f};
    float t1 = 0.f;
#pragma unroll
    for (int i = 0; i < P; ++i) gh[i] = gu[i] = h[i] = a[i] = t[i] = u32x4{0u, 0u, 0u, 0u};
    // What the norm before the next block needs of a row, and what the block needs: each is fetched for the next row when this row's
    // has been used, into the same registers.
    auto fetch_pre = [&](int64_t base) {
        const int64_t row = base + lanes.team;
        if (L::kAlone || row < c.n) {
            if (has_gh) lanes.load(c.GH, c.ldgh, base, gh);
            if (has_gu) lanes.load(c.GU, c.ldgu, base, gu);
            if (has_gu) lanes.load(c.H, c.ldh, base, h);
            if (has_stats) st = reinterpret_cast<const f32x4*>(c.stats)[row];
        } else {                             // a row that is not there adds nothing to the sums
#pragma unroll
            for (int i = 0; i < P; ++i) gh[i] = gu[i] = h[i] = u32x4{0u, 0u, 0u, 0u};
            st = f32x4{0.f, 0.f, 0.f, 0.f};
        }
    };
    auto fetch_post = [&](int64_t base) {
        const int64_t row = base + lanes.team;
        if (L::kAlone || row < c.n) {
            if (has_a) lanes.load(c.A, c.lda, base, a);
            if (c.gate_cols > 1) lanes.load(c.T, c.ldt, base, t);
            if (c.gate_cols == 1) t1 = load_one<BF>(c.T, row * c.ldt);
        } else {
#pragma unroll
            for (int i = 0; i < P; ++i) a[i] = u32x4{0u, 0u, 0u, 0u};
        }
    };
    if (base < end) {
        fetch_pre(base);
        fetch_post(base);
    }
    constexpr bool kParked = W == 1 && P > 1;
    __shared__ f32x4 parked[kParked ? P * E : 1][64];
    Vectors<L, 4, P, E, kParked> vec;
    vec.parked = parked;
    vec.set(lanes, 0, c.p, 1.f);
    vec.set(lanes, 1, c.p_bias, 0.f);
    vec.set(lanes, 2, c.s, 1.f);
    vec.set(lanes, 3, c.q, 1.f);
    if constexpr (kParked) __syncthreads();
    float sum[5][P][E];
#pragma unroll
    for (int k = 0; k < 5; ++k)
#pragma unroll
        for (int i = 0; i < P; ++i)
#pragma unroll
            for (int e = 0; e < E; ++e) sum[k][i][e] = 0.f;
    const float inv_f = 1.f / (float)c.F;
    for (; base < end; base += L::kRows) {
        if constexpr (kParked) asm volatile("" ::: "memory");        // what is parked stays there
        const bool live = L::kAlone || base + lanes.team < c.n;
        const float mean_a = st[0], r_a = st[1], mean_h = st[2], r_h = st[3];
        const Gate row_gate = c.gate_cols == 1 ? fast_gate(t1) : Gate{1.f, 0.f};
        float e_[P][E], hn[P][E], d[P][E];
#pragma unroll
        for (int i = 0; i < P; ++i) {
            unpack<BF>(gh[i], e_[i]);
            unpack<BF>(gu[i], d[i]);
            unpack<BF>(h[i], hn[i]);
        }
        if (base + L::kRows < end) fetch_pre(base + L::kRows);
        if (has_gu) {
            float m[2] = {0.f, 0.f};
#pragma unroll
            for (int i = 0; i < P; ++i) {
                float q[E], part[2] = {0.f, 0.f};
                vec.get(3, i, q);
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    hn[i][e] = (hn[i][e] - mean_h) * r_h;
                    sum[3][i][e] = fmaf(d[i][e], hn[i][e], sum[3][i][e]);
                    sum[4][i][e] += d[i][e];
                    d[i][e] *= q[e];
                    const float counted = MASK && e < lanes.skip[i] ? 0.f : d[i][e];
                    part[0] += counted;
                    part[1] = fmaf(counted, hn[i][e], part[1]);
                }
#pragma unroll
                for (int k = 0; k < 2; ++k) m[k] += lanes.on[i] ? part[k] : 0.f;
            }
            if (c.pre != GAS_NORM_NONE) row_sums<G, W>(m, red, turn);
            m[0] = c.pre == GAS_NORM_LAYER ? m[0] * inv_f : 0.f;
            m[1] = c.pre != GAS_NORM_NONE ? m[1] * inv_f : 0.f;
            const float off = -r_h * m[0], along = -r_h * m[1];
#pragma unroll
            for (int i = 0; i < P; ++i)
#pragma unroll
                for (int e = 0; e < E; ++e) e_[i][e] += fmaf(r_h, d[i][e], fmaf(along, hn[i][e], off));
        }
        u32x4 out[P];
        if (has_gx && live) {
#pragma unroll
            for (int i = 0; i < P; ++i) out[i] = pack<BF>(e_[i]);
            lanes.store(c.GX, c.ldgx, base, out);
        }
        if (!has_a) continue;
        // from here on: d = dy p
        float an[P][E], m[3] = {0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < P; ++i) {
            float g[E], rest[E], p[E], p_bias[E], s[E], part[3] = {0.f, 0.f, 0.f};
            unpack<BF>(a[i], an[i]);
            unpack<BF>(t[i], g);
            vec.get(0, i, p);
            vec.get(1, i, p_bias);
            vec.get(2, i, s);
            if (c.gate_cols > 1) {               // a branch, not a choice of both: 11 issue slots an element
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const Gate gate = fast_gate(g[e]);
                    g[e] = gate.g;
                    rest[e] = gate.rest;
                }
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e) g[e] = row_gate.g;
            }
            float w[E];                          // dy y: of it the gate's gradient is a part
#pragma unroll
            for (int e = 0; e < E; ++e) {
                an[i][e] = (an[i][e] - mean_a) * r_a;
                const float y = fmaf(an[i][e], p[e], p_bias[e]);
                const float branch = e_[i][e] * (c.alpha * g[e]), dy = branch * s[e];
                sum[0][i][e] = fmaf(dy, an[i][e], sum[0][i][e]);
                sum[1][i][e] += dy;
                sum[2][i][e] = fmaf(branch, y, sum[2][i][e]);
                d[i][e] = dy * p[e];
                w[e] = dy * y;
                const float counted = MASK && e < lanes.skip[i] ? 0.f : d[i][e];
                part[0] += counted;
                part[1] = fmaf(counted, an[i][e], part[1]);
            }
            if (c.gate_cols > 1) {
#pragma unroll
                for (int e = 0; e < E; ++e) w[e] *= rest[e];
                out[i] = pack<BF>(w);
            } else if (c.gate_cols == 1) {
#pragma unroll
                for (int e = 0; e < E; ++e) part[2] += MASK && e < lanes.skip[i] ? 0.f : w[e];
                part[2] *= row_gate.rest;
            }
#pragma unroll
            for (int k = 0; k < 3; ++k) m[k] += lanes.on[i] ? part[k] : 0.f;
        }
        if (base + L::kRows < end) fetch_post(base + L::kRows);
        if (c.GT && c.gate_cols > 1 && live) lanes.store(c.GT, c.ldgt, base, out);
        if (c.post != GAS_NORM_NONE || c.gate_cols == 1) row_sums<G, W>(m, red, turn);
        m[0] = c.post == GAS_NORM_LAYER ? m[0] * inv_f : 0.f;
        m[1] = c.post != GAS_NORM_NONE ? m[1] * inv_f : 0.f;
        if (!live) continue;
        if (has_ga) {
            const float off = -r_a * m[0], along = -r_a * m[1];
#pragma unroll
            for (int i = 0; i < P; ++i) {
#pragma unroll
                for (int e = 0; e < E; ++e) d[i][e] = fmaf(r_a, d[i][e], fmaf(along, an[i][e], off));
                out[i] = pack<BF>(d[i]);
            }
            lanes.store(c.GA, c.ldga, base, out);
        }
        if (c.GT && c.gate_cols == 1 && lanes.place == 0) store_one<BF>(c.GT, (base + lanes.team) * c.ldgt, m[2]);
    }
    // the workgroup's sums: across the teams of a wavefront by moves, across its wavefronts in LDS
    float* to = c.partials + (int64_t)blockIdx.x * 5 * c.F;
    const bool only = c.slabs == 1;          // the only workgroup's sums are the sums
    if constexpr (W > 1) {
#pragma unroll
        for (int k = 0; k < 5; ++k)
            if (c.sums[k])
#pragma unroll
                for (int i = 0; i < P; ++i)
                    if (lanes.on[i])
#pragma unroll
                        for (int e = 0; e < E; ++e)
                            if (!MASK || e >= lanes.skip[i]) (only ? c.sums[k] : to + (int64_t)k * c.F)[lanes.c[i] + e] = sum[k][i][e];
    } else {
#pragma unroll
        for (int k0 = 0; k0 < 5; k0 += kAtOnce) {
#pragma unroll
            for (int k = k0; k < k0 + kAtOnce && k < 5; ++k)
#pragma unroll
                for (int i = 0; i < P; ++i)
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        const float v = across_groups<G>(sum[k][i][e]);
                        if ((threadIdx.x & 63) < G && lanes.on[i] && (!MASK || e >= lanes.skip[i]))
                            columns[threadIdx.x >> 6][k - k0][lanes.c[i] + e] = v;
                    }
            __syncthreads();
#pragma unroll
            for (int k = k0; k < k0 + kAtOnce && k < 5; ++k)
                if (c.sums[k])
                    for (int f = threadIdx.x; f < c.F; f += 256)
                        (only ? c.sums[k] : to + (int64_t)k * c.F)[f] = (columns[0][k - k0][f] + columns[1][k - k0][f]) + (columns[2][k - k0][f] + columns[3][k - k0][f]);
            if (k0 + kAtOnce < 5) __syncthreads();
        }
    }
}

// Sums over the workgroups' sums: COLUMNS columns to a workgroup, 1,024 / COLUMNS of the partial rows side by side, added up in order.  Thousands of them
// are added up in two launches, first `per` at a time onto `onto`, by 64 columns so that a load is a stretch of 256 bytes.
template <int COLUMNS>
__global__ __launch_bounds__(1024) void residual_norm_finish_kernel(ResidualNormBwd c, const float* from, int slabs, int per, float* onto) {
    constexpr int kSlots = 1024 / COLUMNS;
    __shared__ float part[kSlots][COLUMNS + 1];
    const int k = blockIdx.y, column = threadIdx.x % COLUMNS, slot = threadIdx.x / COLUMNS, f = blockIdx.x * COLUMNS + column;
    if (!c.sums[k]) return;
    const int first = blockIdx.z * per, end = min(slabs, first + per);
    float sum = 0.f;
    if (f < c.F) {
        const float* at = from + (int64_t)k * c.F + f;
        const int64_t row = (int64_t)5 * c.F;
        for (int j0 = first + slot; j0 < end; j0 += 8 * kSlots) {          // eight on their way at a time
            float x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = j0 + kSlots * i < end ? at[(j0 + kSlots * i) * row] : 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) sum += x[i];
        }
    }
    part[slot][column] = sum;
    __syncthreads();
    for (int o = kSlots / 2; o > 0; o >>= 1) {
        if (slot < o) part[slot][column] += part[slot + o][column];
        __syncthreads();
    }
    if (slot == 0 && f < c.F) (onto ? onto + ((int64_t)blockIdx.z * 5 + k) * c.F : c.sums[k])[f] = part[0][column];
}

template <bool BF>
__global__ __launch_bounds__(256) void residual_norm_bwd_kernel(ResidualNormBwd c) {
    const int lane = threadIdx.x & 63;
    const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (row >= c.n) return;
    float st[4], sc = 0.f, sca = 0.f, sg = 0.f;
    row_stats_of<BF>(c, row, st);
    const float d_mean = c.row_sums[row * 2], dh_mean = c.row_sums[row * 2 + 1];
    if (c.A)
        for (int f = lane; f < c.F; f += 64) {
            const Element v = element<BF>(c, row, f, st, d_mean, dh_mean);
            const float cc = v.dy * at(c.p, f, 1.f);
            sc += cc;
            sca = fmaf(cc, v.an, sca);
            sg = fmaf(v.dy * v.y, v.gate.rest, sg);
        }
    sc = c.post == GAS_NORM_LAYER ? wave_sum(sc) / (float)c.F : 0.f;
    sca = c.post == GAS_NORM_NONE ? 0.f : wave_sum(sca) / (float)c.F;
    sg = wave_sum(sg);
    for (int f = lane; f < c.F; f += 64) {
        const Element v = element<BF>(c, row, f, st, d_mean, dh_mean);
        if (c.GX) store_one<BF>(c.GX, row * c.ldgx + f, v.e);
        if (c.GA) store_one<BF>(c.GA, row * c.ldga + f, st[1] * (v.dy * at(c.p, f, 1.f) - sc - v.an * sca));
        if (c.GT && c.gate_cols != 1) store_one<BF>(c.GT, row * c.ldgt + f, v.dy * v.y * v.gate.rest);
    }
    // after every lane has read the row's gate, which may lie there
    if (c.GT && c.gate_cols == 1 && lane == 0) store_one<BF>(c.GT, row * c.ldgt, sg);
}

constexpr int kSlabs = 256, kSplits = 32;          // kSplits: parts that thousands of partial sums are added up in

template <bool BF, bool MASK, bool ALL, class C>
void launch_rows(const Layout& l, dim3 grid, hipStream_t s, const C& c) {
    constexpr bool kBwd = std::is_same_v<C, ResidualNormBwd>;
#define GAS_ROWS(G, W, P)                                                                                                             \
    if (l.g == G && l.w == W && l.p == P) {                                                                                           \
        const dim3 block(W == 1 ? 256 : W * 64);                                                                                      \
        if constexpr (kBwd) hipLaunchKernelGGL((residual_norm_bwd_rows_kernel<BF, G, W, P, MASK, ALL>), grid, block, 0, s, c);        \
        else hipLaunchKernelGGL((residual_norm_rows_kernel<BF, G, W, P, MASK, ALL>), grid, block, 0, s, c);                           \
        return;                                                                                                                       \
    }
    if constexpr (!ALL) { GAS_ROWS(1, 1, 1) GAS_ROWS(2, 1, 1) GAS_ROWS(4, 1, 1) }
    GAS_ROWS(8, 1, 1) GAS_ROWS(16, 1, 1) GAS_ROWS(32, 1, 1) GAS_ROWS(64, 1, 2) GAS_ROWS(64, 1, 3)
    if constexpr (!(kBwd && ALL)) { GAS_ROWS(64, 1, 1) GAS_ROWS(64, 4, 1) GAS_ROWS(64, 6, 1) GAS_ROWS(64, 8, 1) GAS_ROWS(64, 12, 1) GAS_ROWS(64, 16, 1) }
#undef GAS_ROWS
}
template <class C>
void launch_rows(const Layout& l, bool bf, hipStream_t s, C& c) {
    const dim3 grid((unsigned)l.blocks);
    c.turns = l.turns;
    const bool mask = c.F % (bf ? 8 : 4) != 0;
    bool all;
    // Kernels that know beforehand what there is, us against those that look.  Forward from eight lanes on: 3.1 M x 256 bf16 1,317 and 1,329, 1 M x 100 bf16 189 and 192,
    // 20,000 x 1,433 floats 105 and 109, 8,000 x 8,192 bf16 154 and 157, elsewhere alike.  Backward they have more registers, which pays in teams of 8 to 32 lanes (600,000 x
    // 64 floats 222 and 230, x 128 435 and 442; but x 40 158 and 142) and with several pieces (66,667 x 600 bf16 172 and 181, 19,997 x 1,433 bf16 93 and 100, 200,000 x 400 floats
    // 476 and 478), not with one piece in 64 lanes (300,000 x 512 bf16 476 and 453, 600,000 x 256 floats 884 and 878) nor with several wavefronts (13,333 x 3,000 bf16 168 and
    // 148, 10,000 x 6,000 313 and 232, 8,000 x 8,192 738 and 566).
    if constexpr (std::is_same_v<C, ResidualNormBwd>) all = c.GH && c.GU && c.A && c.GX && c.GA && c.stats && l.w == 1 && (l.g < 64 || l.p > 1);
    else all = c.A && c.H && c.U && !c.hist;
    all = all && l.g >= 8;
#define GAS_ROWS(BF, MASK, ALL) \
    if (bf == BF && mask == MASK && all == ALL) return launch_rows<BF, MASK, ALL>(l, grid, s, c);
    GAS_ROWS(false, false, false) GAS_ROWS(false, false, true) GAS_ROWS(false, true, false) GAS_ROWS(false, true, true)
    GAS_ROWS(true, false, false) GAS_ROWS(true, false, true) GAS_ROWS(true, true, false) GAS_ROWS(true, true, true)
#undef GAS_ROWS
}

gas_status finish_sums(const ResidualNormBwd& c, int slabs, float* spare, hipStream_t s) {
    const float* from = c.partials;
    if (slabs > 1024) {
        const int per = ((slabs + kSplits - 1) / kSplits + 127) / 128 * 128, parts = (slabs + per - 1) / per;
        hipLaunchKernelGGL(residual_norm_finish_kernel<64>, dim3((unsigned)((c.F + 63) / 64), 5, parts), dim3(1024), 0, s, c, from, slabs, per, spare);
        GAS_CHECK_HIP(hipGetLastError());
        from = spare;
        slabs = parts;
    }
    hipLaunchKernelGGL(residual_norm_finish_kernel<16>, dim3((unsigned)((c.F + 15) / 16), 5), dim3(1024), 0, s, c, from, slabs, slabs, nullptr);
    GAS_CHECK_HIP(hipGetLastError());
    return GAS_OK;
}

inline bool valid_norm(int k) { return k == GAS_NORM_NONE || k == GAS_NORM_RMS || k == GAS_NORM_LAYER; }

// Whether rows i of two matrices [n, fa] and [n, fb] share memory: blocks of columns of one matrix lie in each other's span but apart.
bool share(const void* a, int64_t lda, int64_t fa, const void* b, int64_t ldb, int64_t fb, int64_t n, int eb) {
    if (!a || !b || n == 0) return false;
    const int64_t a0 = (int64_t)(uintptr_t)a, b0 = (int64_t)(uintptr_t)b;
    if (a0 + ((n - 1) * lda + fa) * eb <= b0 || b0 + ((n - 1) * ldb + fb) * eb <= a0) return false;
    if (lda != ldb || (b0 - a0) % eb) return true;
    const int64_t ld = lda, d = (((b0 - a0) / eb) % ld + ld) % ld;      // b's first column, counted from a's
    return d < fa || d + fb > ld;
}
bool same(const void* a, int64_t lda, const void* b, int64_t ldb, int64_t n) { return a == b && (lda == ldb || n == 1); }

}  // namespace
}  // namespace gas

using namespace gas;

extern "C" {

gas_status gas_residual_norm(const void* X, int64_t ldx, const void* A, int64_t lda, const void* T, int64_t ldt, int32_t gate_cols,
                             int64_t n_rows, int32_t F, gas_dtype dt, int32_t norm_post, const float* p, const float* p_bias,
                             const float* s, float alpha, int32_t norm_pre, const float* q, const float* q_bias, float eps, void* H,
                             int64_t ldh, void* U, int64_t ldu, float* stats, const int32_t* push_idx, void* push_hist,
                             int64_t n_hist_rows, int64_t ld_push, void* stream) {
    const char* who = "gas_residual_norm";
    if (!valid_dtype(dt)) return fail(GAS_ERR_DTYPE, "%s: unknown dtype %d", who, (int)dt);
    GAS_REQUIRE(n_rows >= 0 && F > 0, "%s: n_rows=%lld F=%d", who, (long long)n_rows, F);
    if (n_rows == 0) return GAS_OK;
    GAS_REQUIRE(X && (H || U || push_hist), "%s: null pointer", who);
    GAS_REQUIRE(valid_norm(norm_post) && valid_norm(norm_pre), "%s: unknown norm %d, %d", who, norm_post, norm_pre);
    GAS_REQUIRE(eps > 0.f && eps < INFINITY, "%s: eps=%g", who, (double)eps);
    GAS_REQUIRE(!stats || aligned16(stats), "%s: the statistics are not aligned to 16 bytes", who);
    GAS_REQUIRE(A || !T, "%s: a gate without a block", who);
    GAS_REQUIRE(!T || gate_cols == 1 || gate_cols == F, "%s: %d gates for rows of %d", who, gate_cols, F);
    GAS_REQUIRE(ldx >= F && (!A || lda >= F) && (!T || ldt >= gate_cols) && (!H || ldh >= F) && (!U || ldu >= F),
                "%s: row stride smaller than the row", who);
    GAS_REQUIRE(!push_idx == !push_hist && (!push_hist || (ld_push >= F && n_hist_rows >= n_rows)), "%s: bad history table for the push", who);
    const int eb = elem_bytes(dt);
    const struct { const void* p; int64_t ld; int cols; } in[3] = {{X, ldx, F}, {A, lda, F}, {T, ldt, gate_cols}};
    const struct { void* p; int64_t ld; } out[2] = {{H, ldh}, {U, ldu}};
    const int64_t table = push_hist ? (n_hist_rows - 1) * ld_push + F : 0;
    for (const auto& o : out)
        for (const auto& i : in)
            GAS_REQUIRE(!share(o.p, o.ld, F, i.p, i.ld, i.cols, n_rows, eb) || (i.cols == F && same(o.p, o.ld, i.p, i.ld, n_rows)),
                        "%s: an output lies in an input", who);
    GAS_REQUIRE(!share(H, ldh, F, U, ldu, F, n_rows, eb), "%s: the outputs share memory", who);
    for (const auto& i : in)
        GAS_REQUIRE(!push_hist || !i.p || !share(push_hist, table, table, i.p, (n_rows - 1) * i.ld + i.cols, (n_rows - 1) * i.ld + i.cols, 1, eb),
                    "%s: the history table lies in an input", who);
    for (const auto& o : out)
        GAS_REQUIRE(!push_hist || !o.p || !share(push_hist, table, table, o.p, (n_rows - 1) * o.ld + F, (n_rows - 1) * o.ld + F, 1, eb),
                    "%s: the history table lies in an output", who);
    ResidualNorm c;
    c.X = static_cast<const char*>(X); c.A = static_cast<const char*>(A); c.T = static_cast<const char*>(T);
    c.ldx = ldx; c.lda = lda; c.ldt = ldt; c.gate_cols = T ? gate_cols : 0;
    c.n = n_rows; c.F = F; c.post = norm_post; c.pre = norm_pre;
    c.p = p; c.p_bias = p_bias; c.s = s; c.q = q; c.q_bias = q_bias; c.alpha = alpha; c.eps = eps;
    c.H = static_cast<char*>(H); c.U = static_cast<char*>(U); c.ldh = ldh; c.ldu = ldu; c.stats = stats;
    c.idx = push_idx; c.hist = static_cast<char*>(push_hist); c.ld_hist = ld_push;
    const Layout l = layout_of(n_rows, F, dt == GAS_BF16, false, std::max({ldx, A ? lda : 0, T ? ldt : 0, H ? ldh : 0, U ? ldu : 0}));
    if (l.w) {
        launch_rows(l, dt == GAS_BF16, (hipStream_t)stream, c);
        GAS_CHECK_HIP(hipGetLastError());
        return GAS_OK;
    }
    const int64_t blocks = (n_rows + 3) / 4;
    GAS_REQUIRE(blocks <= 0xFFFFFFFFLL / 256, "%s: too many rows for one launch", who);
    if (dt == GAS_BF16) hipLaunchKernelGGL(residual_norm_kernel<true>, dim3((unsigned)blocks), dim3(256), 0, (hipStream_t)stream, c);
    else hipLaunchKernelGGL(residual_norm_kernel<false>, dim3((unsigned)blocks), dim3(256), 0, (hipStream_t)stream, c);
    GAS_CHECK_HIP(hipGetLastError());
    return GAS_OK;
}

int64_t gas_residual_norm_bwd_typed_workspace(int64_t n_rows, int32_t F, gas_dtype dt) {
    if (n_rows <= 0 || F <= 0 || !valid_dtype(dt)) return 0;
    const Layout l = layout_of(n_rows, F, dt == GAS_BF16, true, 0);
    return 4 * (l.w ? (l.most_blocks + (l.most_blocks > 1024 ? kSplits : 0)) * 5 * F : (int64_t)kSlabs * 5 * F + 2 * n_rows);
}

int64_t gas_residual_norm_bwd_workspace(int64_t n_rows, int32_t F) {
    return std::max(gas_residual_norm_bwd_typed_workspace(n_rows, F, GAS_F32), gas_residual_norm_bwd_typed_workspace(n_rows, F, GAS_BF16));
}

gas_status gas_residual_norm_bwd(const void* GH, int64_t ldgh, const void* GU, int64_t ldgu, const void* H, int64_t ldh, const void* A,
                                 int64_t lda, const void* T, int64_t ldt, int32_t gate_cols, const float* stats, int64_t n_rows,
                                 int32_t F, gas_dtype dt, int32_t norm_post, const float* p, const float* p_bias, const float* s,
                                 float alpha, int32_t norm_pre, const float* q, void* GX, int64_t ldgx, void* GA, int64_t ldga,
                                 void* GT, int64_t ldgt, float* gp, float* gp_bias, float* gs, float* gq, float* gq_bias,
                                 void* workspace, int64_t workspace_bytes, void* stream) {
    const char* who = "gas_residual_norm_bwd";
    if (!valid_dtype(dt)) return fail(GAS_ERR_DTYPE, "%s: unknown dtype %d", who, (int)dt);
    GAS_REQUIRE(n_rows >= 0 && F > 0, "%s: n_rows=%lld F=%d", who, (long long)n_rows, F);
    hipStream_t st = (hipStream_t)stream;
    const bool sums = gp || gp_bias || gs || gq || gq_bias;
    ResidualNormBwd c;
    c.sums[0] = gp; c.sums[1] = gp_bias; c.sums[2] = gs; c.sums[3] = gq; c.sums[4] = gq_bias;
    c.F = F; c.n = n_rows; c.slabs = 0; c.partials = nullptr;
    if (n_rows == 0) {                        // an empty sum still has to be written
        if (!sums) return GAS_OK;
        return finish_sums(c, 0, nullptr, st);
    }
    GAS_REQUIRE(GH || GU, "%s: null pointer", who);
    GAS_REQUIRE(valid_norm(norm_post) && valid_norm(norm_pre), "%s: unknown norm %d, %d", who, norm_post, norm_pre);
    GAS_REQUIRE(A || !(T || GA || GT || gp || gp_bias || gs), "%s: a block's gradient without the block", who);
    GAS_REQUIRE(T || !GT, "%s: a gate's gradient without the gate", who);
    GAS_REQUIRE(GU || !(gq || gq_bias), "%s: a gain's gradient without the gradient of what it gives", who);
    GAS_REQUIRE(!GU || H, "%s: the gradient of the normed rows without the rows", who);
    GAS_REQUIRE(GX || GA || GT || sums, "%s: null pointer", who);
    GAS_REQUIRE(stats || ((!GU || norm_pre == GAS_NORM_NONE) && (!A || norm_post == GAS_NORM_NONE)), "%s: norms without statistics", who);
    GAS_REQUIRE(!stats || aligned16(stats), "%s: the statistics are not aligned to 16 bytes", who);
    GAS_REQUIRE(!T || gate_cols == 1 || gate_cols == F, "%s: %d gates for rows of %d", who, gate_cols, F);
    GAS_REQUIRE((!GH || ldgh >= F) && (!GU || (ldgu >= F && ldh >= F)) && (!A || lda >= F) && (!T || ldt >= gate_cols) && (!GX || ldgx >= F) &&
                (!GA || ldga >= F) && (!GT || ldgt >= gate_cols), "%s: row stride smaller than the row", who);
    const int eb = elem_bytes(dt);
    const struct { const void* p; int64_t ld; int cols; } in[5] = {{GH, ldgh, F}, {GU, ldgu, F}, {GU ? H : nullptr, ldh, F}, {A, lda, F}, {T, ldt, gate_cols}};
    const struct { void* p; int64_t ld; int cols; } out[3] = {{GX, ldgx, F}, {GA, ldga, F}, {GT, ldgt, gate_cols}};
    for (int o = 0; o < 3; ++o) {
        for (const auto& i : in)
            GAS_REQUIRE(!share(out[o].p, out[o].ld, out[o].cols, i.p, i.ld, i.cols, n_rows, eb) ||
                        (i.cols == out[o].cols && same(out[o].p, out[o].ld, i.p, i.ld, n_rows)), "%s: an output lies in an input", who);
        for (int k = 0; k < o; ++k)
            GAS_REQUIRE(!share(out[o].p, out[o].ld, out[o].cols, out[k].p, out[k].ld, out[k].cols, n_rows, eb), "%s: the outputs share memory", who);
    }
    const int64_t need = gas_residual_norm_bwd_typed_workspace(n_rows, F, dt);
    GAS_REQUIRE(workspace && workspace_bytes >= need, "%s: the workspace has %lld bytes, %lld are needed", who, (long long)workspace_bytes, (long long)need);
    GAS_REQUIRE(aligned16(workspace), "%s: the workspace is not aligned to 16 bytes", who);
    c.GH = static_cast<const char*>(GH); c.GU = static_cast<const char*>(GU); c.H = static_cast<const char*>(H);
    c.A = static_cast<const char*>(A); c.T = static_cast<const char*>(T);
    c.ldgh = ldgh; c.ldgu = ldgu; c.ldh = ldh; c.lda = lda; c.ldt = ldt; c.gate_cols = T ? gate_cols : 0;
    c.stats = stats; c.post = norm_post; c.pre = norm_pre; c.p = p; c.p_bias = p_bias; c.s = s; c.q = q; c.alpha = alpha;
    c.GX = static_cast<char*>(GX); c.GA = static_cast<char*>(GA); c.GT = static_cast<char*>(GT);
    c.ldgx = ldgx; c.ldga = ldga; c.ldgt = ldgt;
    c.partials = static_cast<float*>(workspace);
    const Layout l = layout_of(n_rows, F, dt == GAS_BF16, true, std::max({GH ? ldgh : 0, GU ? std::max(ldgu, ldh) : 0, A ? lda : 0, T ? ldt : 0,
                                                                          GX ? ldgx : 0, GA ? ldga : 0, GT ? ldgt : 0}));
    if (l.w) {
        c.slabs = (int)l.blocks;
        launch_rows(l, dt == GAS_BF16, st, c);
        GAS_CHECK_HIP(hipGetLastError());
        return sums && c.slabs > 1 ? finish_sums(c, c.slabs, c.partials + l.most_blocks * 5 * F, st) : GAS_OK;
    }
    c.row_sums = c.partials + (int64_t)kSlabs * 5 * F;
    c.rows_per_slab = (n_rows + kSlabs - 1) / kSlabs;
    c.slabs = (int)((n_rows + c.rows_per_slab - 1) / c.rows_per_slab);
    const int64_t blocks = (n_rows + 3) / 4;
    GAS_REQUIRE(blocks <= 0xFFFFFFFFLL / 256, "%s: too many rows for one launch", who);
    const bool bf = dt == GAS_BF16;
    hipLaunchKernelGGL(bf ? residual_norm_row_sums_kernel<true> : residual_norm_row_sums_kernel<false>, dim3((unsigned)blocks), dim3(256), 0, st, c);
    GAS_CHECK_HIP(hipGetLastError());
    if (sums) {                               // before the outputs, which may lie where the inputs do
        hipLaunchKernelGGL(bf ? residual_norm_columns_kernel<true> : residual_norm_columns_kernel<false>,
                           dim3((unsigned)((F + 63) / 64), (unsigned)c.slabs), dim3(256), 0, st, c);
        GAS_CHECK_HIP(hipGetLastError());
        const gas_status got = finish_sums(c, c.slabs, nullptr, st);
        if (got != GAS_OK) return got;
    }
    if (GX || GA || GT) {
        hipLaunchKernelGGL(bf ? residual_norm_bwd_kernel<true> : residual_norm_bwd_kernel<false>, dim3((unsigned)blocks), dim3(256), 0, st, c);
        GAS_CHECK_HIP(hipGetLastError());
    }
    return GAS_OK;
}

}  // extern "C"
