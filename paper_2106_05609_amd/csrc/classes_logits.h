// The logits of a tile of 256 classes by BB rows, and what is made of them while they are in registers (classes.h says what they
// are of): a row's statistics, the gradient at them, or those that may be among the largest.
#pragma once
#include "classes.h"

namespace gas {
namespace {

enum { LOGITS_STATS = 0, LOGITS_GRAD = 1, LOGITS_TOP = 2 };

struct LogitsArgs {
    Layer layer;
    Parts parts;
    // targets of the rows that count: one label of weight `info.z` (labels), or entries in the order of their classes
    const int32_t* labels;        // [rows]
    const int2* entries;          // [rows][k]: class, weight
    const uint16_t* starts;       // [rows][class tiles + 1]: entries of the tiles before
    int32_t k, tiles;             // tiles: of all classes
    float inv_t;
    // gradient
    const f32x4* info;            // [rows]: lse, lse at the temperature, weights of their exponentials
    uint16_t* g;                  // [planes][rows][width of a piece]
    int64_t g_plane;
    float* gbias;                 // [row tiles][C up to 256], or NULL
    int64_t cap;                  // elements of a plane of g
    int32_t piece;
    // top
    const float* floor;           // [rows]: the value that a logit has to exceed
    float* z;                     // [rows][width of a piece]
    uint32_t* mask;               // [rows][width / 32]: which logits do, see class_of_bit
    int32_t first, width;         // the piece's first class and its width (a multiple of 256)
    int32_t all;                  // every logit is stored, without bits
    int32_t square;               // the temperature is 2: e^z is the square of e^(z / 2)
    int32_t biased;               // the bias is to be added in every tile, else in the last one alone, which ends beyond the classes
};

// Classes of a piece: as many as the room for the gradient at the logits allows, a multiple of 256.
__device__ __host__ __forceinline__ int piece_width(int64_t cap, int64_t rows, int C) {
    const int64_t cp = ((int64_t)C + 255) / 256 * 256, fit = cap / rows / 256 * 256;
    return (int)(fit < 256 ? 256 : (fit < cp ? fit : cp));
}

template <class P>
__host__ __device__ constexpr int logits_tiles_lds() {                           // operands, then the wavefronts' pieces
    constexpr int pieces = P::T / 64 * 32 * (32 * P::TA + 4) * 4;
    return pieces > P::kLdsBytes ? pieces : P::kLdsBytes;
}

// The class that bit `bit` of a mask's word stands for, from the word's first class.
__device__ __forceinline__ int class_of_bit(int bit) { return acc_row(bit & 15, bit >> 4); }

// KIND: what is made of the logits.  TEMPS: bit 0, exponentials as they are, bit 1, at the temperature.  SPLIT: the gradient goes to
// three planes (fp32).
//
// What passes between lanes goes through a piece of LDS that belongs to the wavefront, 32 rows of its classes at a time: a lane has 64 classes of a
// row in fours, memory wants a row's next to each other (stored as they come, 16 bytes to a row, the gradient took ... of a tile's time), and a
// target's logit lies wherever its class is (found by comparing all 64 it took twice what its sums take).
template <int KIND, int TEMPS, bool SPLIT, class P>
__global__ __launch_bounds__(P::T, 2) void classes_logits_kernel(LogitsArgs a) {
    constexpr int TA = P::TA, TB = P::TB, T = P::T, WA = kTileC / 32 / TA, BB = P::kRowsB, WB = BB / 32 / TB;
    constexpr int kRow = 32 * TA + 4;                                            // floats of a row in the wavefront's piece of LDS
    extern __shared__ __attribute__((aligned(16))) char smem[];
    uint16_t* lds = reinterpret_cast<uint16_t*>(smem);
    float* bias = reinterpret_cast<float*>(smem + logits_tiles_lds<P>());                 // [256]
    int* held = reinterpret_cast<int*>(bias + kTileC);                           // [BB] entries of the row in this tile
    int2* entry = reinterpret_cast<int2*>(held + BB);                            // [BB][kHeldEntries]
    const Layer& l = a.layer;
    const int count = *l.count;
    const int nm = (count + BB - 1) / BB;
    int c_first = a.first, c_end = a.first + a.width, width = a.width;
    if constexpr (KIND == LOGITS_GRAD) {
        if (count == 0) return;
        width = piece_width(a.cap, (int64_t)(count + 255) / 256 * 256, l.C);
        const int64_t from = (int64_t)a.piece * width;
        if (from >= l.C) return;
        c_first = (int)from;
        c_end = c_first + width;
    }
    if (c_end > l.C) c_end = l.C;
    int mt, ct;
    if (!tile_of(blockIdx.x, nm, (c_end - c_first + kTileC - 1) / kTileC, mt, ct)) return;
    const int m0 = mt * BB, c0 = c_first + ct * kTileC, tile = c0 / kTileC;
    const int tid = threadIdx.x, lane = tid & 63, li = lane & 31, lh = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wa0 = (wave % WA) * (32 * TA), wb0 = (wave / WA) * (32 * TB);
    const bool biased = a.biased || c0 + kTileC > l.C;
    const TileOperand oa = {l.w + c0, l.ldw, l.w_plane, l.cw - 8 - c0, l.F};
    const TileOperand ob = {l.x + (int64_t)m0 * l.fp, l.fp, l.x_plane, l.most - 1 - m0, l.fp};
    P product;
    typename P::Walk walk = product.begin(oa, ob, 0, (l.F + P::kStepOf - 1) / P::kStepOf, l.terms, lds);
    if (biased)
        for (int i = tid; i < kTileC; i += T) bias[i] = l.bias[c0 + i];
    if constexpr (KIND != LOGITS_TOP) {
        for (int r = tid; r < BB; r += T) {
            int n = 0;
            const int64_t m = m0 + r;
            if (m < count) {
                if (a.labels) {
                    const int rel = a.labels[m] - c0;
                    if (rel >= 0 && rel < kTileC) {
                        n = 1;
                        entry[r * kHeldEntries] = int2{rel, __float_as_int(KIND == LOGITS_GRAD ? a.info[m][2] : 1.f)};
                    }
                } else {
                    const uint16_t* s = a.starts + m * (a.tiles + 1) + tile;
                    const int from = s[0];
                    n = s[1] - from;
                    const int2* e = a.entries + m * a.k + from;
#pragma unroll
                    for (int j = 0; j < kHeldEntries; ++j)
                        if (j < n) entry[r * kHeldEntries + j] = int2{e[j].x - c0, e[j].y};
                }
            }
            held[r] = n;
        }
    }
    f32x16 acc[TA][TB];
    product.run(walk, oa, ob, lds, wa0, wb0, acc);
    if (biased) {
#pragma unroll
        for (int i = 0; i < TA; ++i) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const f32x4 b = *reinterpret_cast<const f32x4*>(bias + wa0 + 32 * i + 8 * q + 4 * lh);
#pragma unroll
                for (int j = 0; j < TB; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[i][j][4 * q + e] += b[e];
            }
            __builtin_amdgcn_sched_barrier(0);                 // not all of the bias at once: there are no registers for it
        }
    }
    float* mine = reinterpret_cast<float*>(smem) + wave * (32 * kRow);
    auto show = [&](int j) {                                   // the wavefront's rows 32 j .. to its piece of LDS
#pragma unroll
        for (int i = 0; i < TA; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *reinterpret_cast<f32x4*>(mine + li * kRow + 32 * i + 8 * q + 4 * lh) =
                    f32x4{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
    };
    // entries of row r of the tile among the wavefront's classes, by one lane of the row
    auto each_entry = [&](int r, auto&& use) {
        const int n = lh == 0 ? held[r] : 0;
        for (int j = 0; j < n; ++j) {
            int2 e;
            if (j < kHeldEntries) e = entry[r * kHeldEntries + j];
            else {
                const int64_t m = m0 + r;
                e = a.entries[m * a.k + a.starts[m * (a.tiles + 1) + tile] + j];
                e.x -= c0;
            }
            const int rel = e.x - wa0;
            if (rel >= 0 && rel < 32 * TA) use(mine + li * kRow + rel, __int_as_float(e.y));
        }
    };
    if constexpr (KIND == LOGITS_GRAD) {
        constexpr int kOwn = 32 * TA / 64;                     // classes whose sum over the rows a lane has
        float column[kOwn] = {};
#pragma unroll
        for (int j = 0; j < TB; ++j) {
            const int row = wb0 + 32 * j + li;
            const int64_t m = m0 + row;
            // a exp(z - lse) = (a 2^(rest)) 2^(z log2 e - least), least = lse log2 e rounded, which leaves out `rest`
            f32x4 info = {INFINITY, INFINITY, 0.f, 0.f};
            if (m < count) info = a.info[m];
            const float least = info[0] * kLog2e, least_t = info[1] * kLog2e, log2e_t = kLog2e * a.inv_t;
            if (m < count) {
                const double rest_t = (double)least_t - (double)info[1] * (double)kLog2e;
                if (TEMPS == 3 && a.square) info[2] *= exp2_of((float)(2.0 * (double)least_t - (double)info[0] * (double)kLog2e));
                else if (TEMPS & 1) info[2] *= exp2_of((float)((double)least - (double)info[0] * (double)kLog2e));
                if (TEMPS & 2) info[3] *= exp2_of((float)rest_t);
            }
            if (TEMPS == 3 && a.square) {                      // exp(z - lse) = exp(z / 2 - lse_t)^2 exp(2 lse_t - lse)
#pragma unroll
                for (int i = 0; i < TA; ++i)
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const float e = exp2_of(fmaf(acc[i][j][r], log2e_t, -least_t));
                        acc[i][j][r] = e * fmaf(e, info[2], info[3]);
                    }
            } else {
#pragma unroll
                for (int i = 0; i < TA; ++i)
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const float z = acc[i][j][r];
                        float g = 0.f;
                        if constexpr (TEMPS & 1) g = info[2] * exp2_of(fmaf(z, kLog2e, -least));
                        if constexpr (TEMPS & 2) g += info[3] * exp2_of(fmaf(z, log2e_t, -least_t));
                        acc[i][j][r] = g;
                    }
            }
            show(j);
            each_entry(row, [&](float* at, float w) { *at -= w; });
            if (a.gbias)
#pragma unroll
                for (int r = 0; r < 32; ++r)
#pragma unroll
                    for (int e = 0; e < kOwn; ++e) column[e] += mine[r * kRow + kOwn * lane + e];
            // eight classes of a row a lane, so that a row's are next to each other
            constexpr int kLanes = 32 * TA / 8, kRows = 64 / kLanes;
            uint16_t* to = a.g + (int64_t)(m0 + wb0 + 32 * j + lane / kLanes) * width + (c0 - c_first) + wa0 + 8 * (lane % kLanes);
            const float* from = mine + (lane / kLanes) * kRow + 8 * (lane % kLanes);
#pragma unroll
            for (int r = 0; r < 32; r += kRows) {
                const f32x4 v0 = *reinterpret_cast<const f32x4*>(from + r * kRow), v1 = *reinterpret_cast<const f32x4*>(from + r * kRow + 4);
                uint16_t* p = to + (int64_t)r * width;
                if constexpr (SPLIT) {
                    const float v[8] = {v0[0], v0[1], v0[2], v0[3], v1[0], v1[1], v1[2], v1[3]};
                    put8(v, 6, p, a.g_plane, 0);
                } else {
                    *reinterpret_cast<u32x4*>(p) = u32x4{pack_bf16(v0[0], v0[1]), pack_bf16(v0[2], v0[3]), pack_bf16(v1[0], v1[1]), pack_bf16(v1[2], v1[3])};
                }
            }
        }
        if (a.gbias) {
            float* sums = bias;                                // [WB][256], over the bias and what follows it
            __syncthreads();
#pragma unroll
            for (int e = 0; e < kOwn; ++e) sums[(wave / WA) * kTileC + wa0 + kOwn * lane + e] = column[e];
            __syncthreads();
            for (int c = tid; c < kTileC; c += T) {
                float v = sums[c];
#pragma unroll
                for (int w = 1; w < WB; ++w) v += sums[w * kTileC + c];
                a.gbias[(int64_t)mt * ((l.C + 255) / 256 * 256) + c0 + c] = v;
            }
        }
        return;
    }
    if constexpr (KIND == LOGITS_TOP) {
#pragma unroll
        for (int j = 0; j < TB; ++j) {
            const int64_t m = m0 + wb0 + 32 * j + li;
            const bool on = m < count;
            float* row = a.z + m * width + (c0 - c_first) + wa0 + 4 * lh;
            if (a.all) {                                       // columns up to the piece's width are there, beyond the classes too
                if (on)
#pragma unroll
                    for (int i = 0; i < TA; ++i)
#pragma unroll
                        for (int q = 0; q < 4; ++q)
                            *reinterpret_cast<f32x4*>(row + 32 * i + 8 * q) =
                                f32x4{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
                continue;
            }
            const float floor = on ? a.floor[m] : INFINITY;
            uint32_t mask[TA];                                 // bit r of a lane: accumulator r; those of lanes 32 on from bit 16 on
            uint32_t some = 0;
#pragma unroll
            for (int i = 0; i < TA; ++i) {
                const int c = c0 + wa0 + 32 * i;
                uint32_t bits = 0;
#pragma unroll
                for (int r = 15; r >= 0; --r) bits = bits + bits + !(acc[i][j][r] <= floor);
                if (c + 32 > l.C)
                    for (int r = 0; r < 16; ++r)
                        if (c + acc_row(r, lh) >= l.C) bits &= ~(1u << r);
                if (!on) bits = 0;
                mask[i] = bits;
                some |= bits;
            }
            if (__any(some != 0)) {
                show(j);
#pragma unroll
                for (int i = 0; i < TA; ++i)
                    for (uint32_t bits = mask[i]; bits; bits &= bits - 1) {
                        const int at = 32 * i + acc_row(__ffs((int)bits) - 1, 0);
                        row[at] = mine[li * kRow + 4 * lh + at];
                    }
            }
#pragma unroll
            for (int i = 0; i < TA; ++i) {
                const uint32_t other = (uint32_t)__shfl_xor((int)mask[i], 32);
                if (on && lh == 0) a.mask[m * (width / 32) + (c0 - c_first + wa0) / 32 + i] = mask[i] | other << 16;
            }
        }
        if (!a.parts.most) return;
    }
    float* red = bias;                                         // [WA][4][BB], over the bias and what follows it
    float most[TB], sum[TB], sum_t[TB], picked[TB];
#pragma unroll
    for (int j = 0; j < TB; ++j) {
        const int row = wb0 + 32 * j + li;
        most[j] = -INFINITY;
        sum[j] = sum_t[j] = picked[j] = 0.f;
        if constexpr (KIND == LOGITS_STATS) {
            if (__any(held[row] > 0)) {
                show(j);
                each_entry(row, [&](const float* at, float w) { picked[j] = fmaf(w, *at, picked[j]); });
            }
        }
#pragma unroll
        for (int i = 0; i < TA; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) most[j] = fmaxf(most[j], acc[i][j][r]);
        most[j] = fmaxf(most[j], __shfl_xor(most[j], 32));
        most[j] = fmaxf(most[j] * kLog2e, kLeastExponent);
        if (TEMPS == 3 && a.square) {
            const float half = 0.5f * most[j];
#pragma unroll
            for (int i = 0; i < TA; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const float e = exp2_of(fmaf(acc[i][j][r], 0.5f * kLog2e, -half));
                    sum_t[j] += e;
                    sum[j] = fmaf(e, e, sum[j]);
                }
        } else {
#pragma unroll
            for (int i = 0; i < TA; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const float d = fmaf(acc[i][j][r], kLog2e, -most[j]);
                    sum[j] += exp2_of(d);
                    if constexpr (TEMPS & 2) sum_t[j] += exp2_of(d * a.inv_t);
                }
        }
        sum[j] += __shfl_xor(sum[j], 32);
        if constexpr (TEMPS & 2) sum_t[j] += __shfl_xor(sum_t[j], 32);
    }
    int n_held = 0;
    if (KIND == LOGITS_STATS && tid < BB) n_held = held[tid];
    __syncthreads();                                           // everyone is done with the bias and the entries
    if (lh == 0) {
#pragma unroll
        for (int j = 0; j < TB; ++j) {
            float* to = red + (wave % WA) * 4 * BB + wb0 + 32 * j + li;
            to[0] = most[j];
            to[BB] = sum[j];
            to[2 * BB] = sum_t[j];
            to[3 * BB] = picked[j];
        }
    }
    __syncthreads();
    static_assert(BB <= T, "a thread a row");
    if (tid < BB && m0 + tid < count) {
        const int64_t m = m0 + tid;
        float top = red[tid], s = red[BB + tid], st = red[2 * BB + tid], z = red[3 * BB + tid];
#pragma unroll
        for (int w = 1; w < WA; ++w) {
            const float* o = red + w * 4 * BB + tid;
            join(top, s, st, o[0], o[BB], o[2 * BB], a.inv_t);
            z += o[3 * BB];
        }
        const int64_t at = (int64_t)tile * l.most + m;
        a.parts.most[at] = top;
        a.parts.sum[at] = s;
        if constexpr (KIND == LOGITS_STATS) {
            if constexpr (TEMPS & 2) a.parts.sum_t[at] = st;
            if (!a.labels) a.parts.picked[at] = z;
            else if (n_held) a.parts.picked[m] = z;
        }
    }
}

template <class P>
constexpr int logits_lds() {
    constexpr int BB = P::kRowsB, extra = kTileC * 4 + BB * 4 + BB * kHeldEntries * 8, red = kTileC / 32 / P::TA * 4 * BB * 4;
    static_assert(BB / 32 / P::TB * kTileC * 4 <= extra, "the sums of the gradient's columns");
    return logits_tiles_lds<P>() + (extra > red ? extra : red);
}

template <int KIND, int TEMPS, bool SPLIT, class P>
gas_status launch_logits_tile(const LogitsArgs& a, int64_t tiles, hipStream_t s) {
    constexpr int smem = logits_lds<P>();
    static_assert(smem <= 160 * 1024, "LDS of a compute unit");
    static const gas_status attr = lds_of(classes_logits_kernel<KIND, TEMPS, SPLIT, P>, smem);
    if (attr != GAS_OK) return attr;
    const int64_t blocks = (tiles + 7) / 8 * 8;
    GAS_REQUIRE(blocks <= 0x7FFFFFLL, "too many tiles for one launch");
    hipLaunchKernelGGL((classes_logits_kernel<KIND, TEMPS, SPLIT, P>), dim3((unsigned)blocks), dim3(P::T), smem, s, a);
    GAS_CHECK_HIP(hipGetLastError());
    return GAS_OK;
}

// tiles: of rows by classes, at most, for tiles of rows_of_tile(n) rows
using FewRows = TileProduct<kTileC, 64, 4, 1, true, false>;
#ifdef VARIANT_A
constexpr int kRowsTile = 128;
using ManyRows = TileProduct<kTileC, 128, 2, 2, true, false>;
#else
constexpr int kRowsTile = 256;
using ManyRows = TileProduct<kTileC, 256, 2, 4, true, false, 64, 2>;
#endif
// Rows of a tile: 64 where there are no more rows, or where tiles of 256 would leave compute units without any.
inline int rows_of_tile(int64_t n, int C) { return n <= 64 || round_up(n, kRowsTile) / kRowsTile * (round_up(C, kTileC) / kTileC) < 256 ? 64 : kRowsTile; }
template <int KIND, int TEMPS, bool SPLIT = false>
gas_status launch_logits(const LogitsArgs& a, int tile_rows, int64_t tiles, hipStream_t s) {
    if (tile_rows == 64) return launch_logits_tile<KIND, TEMPS, SPLIT, FewRows>(a, tiles, s);
    return launch_logits_tile<KIND, TEMPS, SPLIT, ManyRows>(a, tiles, s);
}

}  // namespace
}  // namespace gas
