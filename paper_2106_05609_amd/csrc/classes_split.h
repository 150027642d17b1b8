// Logits of so few tiles that most of the card would have none, where the sums are long: a workgroup a part of a tile's sums, and the parts
// added up by what reads them.  100 x 2,048 x 1,500 of fp32 is 12 tiles of 384 steps one after another: its loss took 202 us, in sixteen parts 46 (the
// products 19, adding up 5).
#pragma once
#include "classes_logits.h"
#include "classes_vector.h"

namespace gas {
namespace {

struct SplitArgs {
    Layer layer;
    float* parts;                 // [splits][rows][ld]
    int64_t ld, step;             // step: elements of a part
    int32_t width, splits;        // the classes from the first on, a multiple of 256
};

// Lanes end up with four neighbouring classes of one row.
template <class P>
__global__ __launch_bounds__(P::T, 2) void classes_split_kernel(SplitArgs a) {
    constexpr int BB = P::kRowsB, WA = kTileC / 32 / P::TA;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    uint16_t* lds = reinterpret_cast<uint16_t*>(smem);
    const Layer& l = a.layer;
    const int count = l.shape->count, nc = a.width / kTileC, steps = (l.F + P::kStepOf - 1) / P::kStepOf;
    int m0, at;
    if (!tile_of(blockIdx.x, gridDim.x, (count + BB - 1) / BB, nc * a.splits, m0, at)) return;
    m0 *= BB;
    const int c0 = at % nc * kTileC, part = at / nc, per = (steps + a.splits - 1) / a.splits;
    const int first = part * per < steps ? part * per : steps, last = first + per < steps ? first + per : steps;
    const int lane = threadIdx.x & 63, li = lane & 31, lh = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wa0 = (wave % WA) * (32 * P::TA), wb0 = (wave / WA) * (32 * P::TB);
    const TileOperand ob = {l.x + (int64_t)m0 * l.fp, l.fp, l.x_plane, l.most - 1 - m0, l.fp};
    f32x16 acc[P::TA][P::TB];
    P product;
    if constexpr (P::kReadOnce) {
        const typename P::Operand oa = {static_cast<const char*>(l.raw) + (int64_t)c0 * (P::PLANES == 1 ? 2 : 4), l.ld_raw, l.C - c0, l.F};
        product.run(oa, ob, count, first, last, lds, wa0, wb0, acc);
    } else {
        const TileOperand oa = {l.w + c0, l.ldw, l.w_plane, l.cw - 8 - c0, l.F};
        product.run(oa, ob, first, last, l.terms, lds, wa0, wb0, acc);
    }
#pragma unroll
    for (int j = 0; j < P::TB; ++j) {
        const int m = m0 + wb0 + 32 * j + li;
        if (m >= count) continue;
        float* row = a.parts + part * a.step + m * a.ld + c0 + wa0 + 4 * lh;
#pragma unroll
        for (int i = 0; i < P::TA; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *reinterpret_cast<f32x4*>(row + 32 * i + 8 * q) = f32x4{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
    }
}

// Logits that came in parts, row m and class c of part s at p[s step + m ld + c]; the bias is still to be added, or NULL.
struct PartsOfZ {
    const float* p;
    int64_t ld, step;
    int32_t splits;
    const float* bias;
};

// A wavefront a row of 256 classes: the logits, and their statistics if they are asked for
struct JoinArgs {
    PartsOfZ from;
    const Shape* shape;
    int64_t stats;
    float inv_t;                  // 0: one temperature
    float* z;                     // [rows][ld]
    Parts parts;
};
__global__ __launch_bounds__(256) void classes_join_kernel(JoinArgs a) {
    const int lane = threadIdx.x & 63, r = (int)(blockIdx.y * 4 + (threadIdx.x >> 6)), c = (int)(blockIdx.x * kTileC) + 4 * lane;
    if (r >= a.shape->count) return;
    const int64_t at = r * a.from.ld + c;
    f32x4 z = sum_of(reinterpret_cast<const f32x4*>(a.from.p + at), a.from.step / 4, a.from.splits, f32x4{0.f, 0.f, 0.f, 0.f});
    z += *reinterpret_cast<const f32x4*>(a.from.bias + c);
    *reinterpret_cast<f32x4*>(a.z + at) = z;
    if (!a.parts.most) return;
    float most = fmaxf(fmaxf(z[0], z[1]), fmaxf(z[2], z[3])), sum = 0.f, sum_t = 0.f;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor(most, o));
    most = fmaxf(most * kLog2e, kLeastExponent);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const float d = fmaf(z[e], kLog2e, -most);
        sum += exp2_of(d);
        sum_t += exp2_of(d * a.inv_t);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        sum += __shfl_xor(sum, o);
        sum_t += __shfl_xor(sum_t, o);
    }
    if (lane > 0) return;
    const int64_t to = blockIdx.x * a.stats + r;
    a.parts.most[to] = most;
    a.parts.sum[to] = sum;
    if (a.inv_t != 0.f) a.parts.sum_t[to] = sum_t;
}

// Whether up to eight rows are better off in split sums than with the vector units, whose time grows with the rows and F until there are classes enough
// to hide it; forward / backward in us, the vector units first:
//     fp32   1 x 1,024 x 4,000     19 / 44      22 / 39        bf16   1 x 512 x 1,001       19 / 38      24 / 40
//            1 x 2,560 x 4,000     39 / 70      29 / 52               1 x 512 x 1,000       19 / 35      17 / 29
//            1 x 2,560 x 24,000    48 / 174     52 / 166              1 x 2,048 x 4,001     81 / 120     26 / 51
//            4 x 512 x 4,000       19 / 43      22 / 41               4 x 512 x 4,001       24 / 45      25 / 42
//            4 x 1,024 x 4,000     27 / 56      23 / 42               8 x 512 x 64,000      43 / 114     27 / 93
//            8 x 512 x 4,000       24 / 49      23 / 44               8 x 2,048 x 50,000   127 / 243     48 / 158
//            8 x 2,560 x 40,000   104 / 292     96 / 286              8 x 4,096 x 16,000   226 / 292     35 / 99
//            8 x 2,560 x 64,000   139 / 435    133 / 432
// bf16 whose rows are no whole pieces is read once as fp32 is, and so as long in coming.
inline bool few_by_split(int64_t n, int F, int C, gas_dtype dt) {
    const int64_t work = (int64_t)F * (n + 5);
    return dt == GAS_F32 ? work >= 6656 && C <= 4096 * (n + 3) : C % 8 == 0 || work >= 4608;
}
// Parts of the sums for which a tile's are worth it: two workgroups for every unit, of a few steps each. A step of fp32 takes as long as several.
inline int splits_of_few(int64_t n, int F, int C, gas_dtype dt) {
    if (rows_of_tile(n, C) != 64) return 1;
    if (n <= kRowsByVector && !few_by_split(n, F, C, dt)) return 1;
    const int64_t tiles = (n + 63) / 64 * (round_up(C, kTileC) / kTileC), steps = round_up(F, FewRows::kStepOf) / FewRows::kStepOf / (dt == GAS_F32 ? 4 : 8);
    int64_t s = 512 / tiles;
    if (s > steps) s = steps;
    if (s > 32) s = 32;
    return s < 2 ? 1 : (int)s;
}

// Room for the logits of few rows, or for parts of them; neither if they are formed in tiles.
struct FewRoom {
    float *z, *parts;
    int64_t ld, step;
    int32_t splits;
    bool by_vector;               // up to eight rows, by the vector units
};
inline FewRoom lay_out_few(Room& room, int64_t n, int F, int C, gas_dtype dt, bool whole) {
    FewRoom f = {nullptr, nullptr, round_up(C, kTileC), round_up(n, 64) * round_up(C, kTileC), splits_of_few(n, F, C, dt), false};
    f.by_vector = n <= kRowsByVector && f.splits == 1;
    if (f.splits > 1) f.parts = room.take<float>(f.splits * f.step);
    if (f.by_vector || (whole && f.splits > 1)) f.z = room.take<float>((f.by_vector ? n : round_up(n, 64)) * f.ld);
    return f;
}

template <class P>
gas_status launch_split_of(const SplitArgs& a, int64_t n, hipStream_t s) {
    static const gas_status attr = lds_of(classes_split_kernel<P>, P::kLdsBytes);
    if (attr != GAS_OK) return attr;
    const int64_t tiles = (n + 63) / 64 * (a.width / kTileC) * a.splits;
    hipLaunchKernelGGL(classes_split_kernel<P>, dim3((unsigned)round_up(tiles, 8)), dim3(P::T), P::kLdsBytes, s, a);
    GAS_CHECK_HIP(hipGetLastError());
    return GAS_OK;
}
inline gas_status launch_split(const Layer& l, const FewRoom& f, int64_t n, hipStream_t s) {
    const SplitArgs a = {l, f.parts, f.ld, f.step, (int32_t)f.ld, f.splits};
    return l.w ? launch_split_of<FewRows>(a, n, s) : l.terms == 1 ? launch_split_of<FewRowsOnce<true>>(a, n, s) : launch_split_of<FewRowsOnce<false>>(a, n, s);
}
inline gas_status launch_join(const Layer& l, const FewRoom& f, int64_t n, float inv_t, const Parts* parts, hipStream_t s) {
    const JoinArgs a = {{f.parts, f.ld, f.step, f.splits, l.bias}, l.shape, l.stats, inv_t, f.z, parts ? *parts : Parts{}};
    hipLaunchKernelGGL(classes_join_kernel, dim3((unsigned)(f.ld / kTileC), (unsigned)((n + 3) / 4)), dim3(256), 0, s, a);
    GAS_CHECK_HIP(hipGetLastError());
    return GAS_OK;
}

}  // namespace
}  // namespace gas
