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
    int32_t two;                  // statistics: both temperatures; gradient: bit 0 the first, bit 1 the other
    // gradient
    const f32x4* info;            // [rows]: lse, lse at the temperature, weights of their exponentials
    uint16_t* g;                  // [planes][rows][width of a piece]
    int64_t g_plane;
    float* gbias;                 // [row tiles][C up to 256], or NULL
    int64_t cap;                  // elements of a plane of g
    int32_t piece;
    // top
    const float* floor;           // [rows]: NaN, or the value that a logit has to exceed
    float* z;                     // [rows][width of a piece]
    uint32_t* mask;               // [rows][width / 32]: which logits do
    int32_t first, width;         // the piece's first class and its width (a multiple of 256)
};

// Classes of a piece: as many as the room for the gradient at the logits allows, a multiple of 256.
__device__ __host__ __forceinline__ int piece_width(int64_t cap, int64_t rows, int C) {
    const int64_t cp = ((int64_t)C + 255) / 256 * 256, fit = cap / rows / 256 * 256;
    return (int)(fit < 256 ? 256 : (fit < cp ? fit : cp));
}

template <int KIND, int BB, int WA, int WB>
__global__ __launch_bounds__(64 * WA * WB) void classes_logits_kernel(LogitsArgs a) {
    using P = TileProduct<kTileC, BB, WA, WB, true, false>;
    constexpr int TA = P::TA, TB = P::TB, T = P::T;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    uint16_t* lds = reinterpret_cast<uint16_t*>(smem);
    float* bias = reinterpret_cast<float*>(smem + P::kLdsBytes);                 // [256]
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
    P product;
    {
        const int last_c = l.cw - 8 - c0, last_m = l.most - 1 - m0;
        const TileOperand oa = {l.w + c0, l.ldw, l.w_plane, last_c, l.F};
        const TileOperand ob = {l.x + (int64_t)m0 * l.fp, l.fp, l.x_plane, last_m, l.fp};
        product.run(oa, ob, 0, l.fp / kStepK, l.terms, lds, wa0, wb0, acc);
    }
    // entries of row r in this wavefront's classes, one after another: use(index, weight) with the index of the lane's element that it
    // names, or -1
    auto each_entry = [&](int r, auto&& use) {
        const int n = held[r];
        for (int j = 0; __any(j < n); ++j) {
            int2 e = {-1, 0};
            if (j < n) {
                if (j < kHeldEntries) e = entry[r * kHeldEntries + j];
                else {
                    const int64_t m = m0 + r;
                    e = a.entries[m * a.k + a.starts[m * (a.tiles + 1) + tile] + j];
                    e.x -= c0;
                }
            }
            const int rel = e.x - wa0;
            const bool mine = j < n && rel >= 0 && rel < 32 * TA && ((rel >> 2) & 1) == lh;
            if (__any(mine)) use(mine ? (rel >> 5) * 16 + ((rel & 31) >> 3) * 4 + (rel & 3) : -1, __int_as_float(e.y));
        }
    };
#pragma unroll
    for (int i = 0; i < TA; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const f32x4 b = *reinterpret_cast<const f32x4*>(bias + wa0 + 32 * i + 8 * q + 4 * lh);
#pragma unroll
            for (int j = 0; j < TB; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[i][j][4 * q + e] += b[e];
        }
    if constexpr (KIND == LOGITS_GRAD) {
        const int64_t rows = (int64_t)(count + 255) / 256 * 256;
        float column[TA][16];                                  // sums over this lane's rows
#pragma unroll
        for (int i = 0; i < TA; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) column[i][r] = 0.f;
#pragma unroll
        for (int j = 0; j < TB; ++j) {
            const int row = wb0 + 32 * j + li;
            const int64_t m = m0 + row;
            f32x4 info = {INFINITY, INFINITY, 0.f, 0.f};
            if (m < count) info = a.info[m];
#pragma unroll
            for (int i = 0; i < TA; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const float z = acc[i][j][r];
                    float g = 0.f;
                    if (a.two & 1) g = info[2] * exp2_of((z - info[0]) * kLog2e);
                    if (a.two & 2) g += info[3] * exp2_of((z * a.inv_t - info[1]) * kLog2e);
                    acc[i][j][r] = g;
                }
            each_entry(row, [&](int at, float w) {
#pragma unroll
                for (int i = 0; i < TA; ++i)
#pragma unroll
                    for (int r = 0; r < 16; ++r) acc[i][j][r] -= at == 16 * i + r ? w : 0.f;
            });
            if (m >= rows) continue;
            uint16_t* to = a.g + m * width + (c0 - c_first) + wa0 + 4 * lh;
#pragma unroll
            for (int i = 0; i < TA; ++i)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    uint32_t h[2], md[2], lo[2];
#pragma unroll
                    for (int e = 0; e < 2; ++e) split_pair(acc[i][j][4 * q + 2 * e], acc[i][j][4 * q + 2 * e + 1], h[e], md[e], lo[e]);
                    uint16_t* at = to + 32 * i + 8 * q;
                    *reinterpret_cast<u32x2*>(at) = u32x2{h[0], h[1]};
                    if (l.terms > 1) {
                        *reinterpret_cast<u32x2*>(at + a.g_plane) = u32x2{md[0], md[1]};
                        *reinterpret_cast<u32x2*>(at + 2 * a.g_plane) = u32x2{lo[0], lo[1]};
                    }
                }
        }
        if (a.gbias) {
            float* sums = reinterpret_cast<float*>(smem);      // [WB][256]
#pragma unroll
            for (int j = 0; j < TB; ++j)
#pragma unroll
                for (int i = 0; i < TA; ++i)
#pragma unroll
                    for (int r = 0; r < 16; ++r) column[i][r] += acc[i][j][r];
#pragma unroll
            for (int i = 0; i < TA; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    float v = column[i][r];
#pragma unroll
                    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor(v, o);
                    if (li == 0) sums[(wave / WA) * kTileC + wa0 + 32 * i + acc_row(r, lh)] = v;
                }
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
            const float floor = on ? a.floor[m] : 0.f;
#pragma unroll
            for (int i = 0; i < TA; ++i) {
                const int c = c0 + wa0 + 32 * i;
                uint32_t mask = 0;
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (!(acc[i][j][r] <= floor) && c + acc_row(r, lh) < l.C) mask |= 1u << acc_row(r, lh);
                if (!on) mask = 0;
                if (mask) {
                    float* to = a.z + m * width + (c - c_first);
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if (mask >> acc_row(r, lh) & 1) to[acc_row(r, lh)] = acc[i][j][r];
                }
                mask |= (uint32_t)__shfl_xor((int)mask, 32);
                if (on && lh == 0) a.mask[m * (width / 32) + (c - c_first) / 32] = mask;
            }
        }
        if (!a.parts.most) return;
    }
    float* red = reinterpret_cast<float*>(smem);               // [WA][4][BB]
#pragma unroll
    for (int j = 0; j < TB; ++j) {
        const int row = wb0 + 32 * j + li;
        float most = -INFINITY, sum = 0.f, sum_t = 0.f, picked = 0.f;
#pragma unroll
        for (int i = 0; i < TA; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) most = fmaxf(most, acc[i][j][r]);
        most = fmaxf(most, __shfl_xor(most, 32));
        const float base = most == -INFINITY ? 0.f : most;
#pragma unroll
        for (int i = 0; i < TA; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const float d = (acc[i][j][r] - base) * kLog2e;
                sum += exp2_of(d);
                if (KIND == LOGITS_STATS && a.two) sum_t += exp2_of(d * a.inv_t);
            }
        sum += __shfl_xor(sum, 32);
        if constexpr (KIND == LOGITS_STATS) {
            if (a.two) sum_t += __shfl_xor(sum_t, 32);
            each_entry(row, [&](int at, float w) {
                float z = 0.f;
#pragma unroll
                for (int i = 0; i < TA; ++i)
#pragma unroll
                    for (int r = 0; r < 16; ++r) z = at == 16 * i + r ? acc[i][j][r] : z;
                if (at >= 0) picked = fmaf(w, z, picked);
            });
            picked += __shfl_xor(picked, 32);
        }
        if (lh == 0) {
            float* to = red + (wave % WA) * 4 * BB + row;
            to[0] = most;
            to[BB] = sum;
            to[2 * BB] = sum_t;
            to[3 * BB] = picked;
        }
    }
    __syncthreads();
    for (int r = tid; r < BB; r += T) {
        const int64_t m = m0 + r;
        if (m >= count) continue;
        float most = red[r], sum = red[BB + r], sum_t = red[2 * BB + r], picked = red[3 * BB + r];
#pragma unroll
        for (int w = 1; w < WA; ++w) {
            const float* o = red + w * 4 * BB + r;
            join(most, sum, sum_t, o[0], o[BB], o[2 * BB], a.inv_t);
            picked += o[3 * BB];
        }
        const int64_t at = (int64_t)tile * l.most + m;
        a.parts.most[at] = most;
        a.parts.sum[at] = sum;
        if constexpr (KIND == LOGITS_STATS) {
            if (a.two) a.parts.sum_t[at] = sum_t;
            if (!a.labels) a.parts.picked[at] = picked;
            else if (held[r]) a.parts.picked[m] = picked;
        }
    }
}

template <int BB, int WA, int WB>
constexpr int logits_lds() { return TileProduct<kTileC, BB, WA, WB, true, false>::kLdsBytes + kTileC * 4 + BB * 4 + BB * kHeldEntries * 8; }

template <int KIND, int BB, int WA, int WB>
gas_status launch_logits_tile(const LogitsArgs& a, int64_t rows, int64_t tiles_c, hipStream_t s) {
    constexpr int smem = logits_lds<BB, WA, WB>();
    static_assert(smem <= 160 * 1024, "LDS of a compute unit");
    static const gas_status attr = lds_of(classes_logits_kernel<KIND, BB, WA, WB>, smem);
    if (attr != GAS_OK) return attr;
    const int64_t tiles = (rows + BB - 1) / BB * tiles_c, blocks = (tiles + 7) / 8 * 8;
    GAS_REQUIRE(blocks <= 0x7FFFFFLL, "too many tiles for one launch");
    hipLaunchKernelGGL((classes_logits_kernel<KIND, BB, WA, WB>), dim3((unsigned)blocks), dim3(64 * WA * WB), smem, s, a);
    GAS_CHECK_HIP(hipGetLastError());
    return GAS_OK;
}

// rows: at most so many count; tiles_c: tiles of 256 classes of the launch
template <int KIND>
gas_status launch_logits(const LogitsArgs& a, int64_t rows, int64_t tiles_c, hipStream_t s) {
    if (rows <= 64) return launch_logits_tile<KIND, 64, 4, 1>(a, rows, tiles_c, s);
    return launch_logits_tile<KIND, 256, 2, 4>(a, rows, tiles_c, s);
}

}  // namespace
}  // namespace gas
