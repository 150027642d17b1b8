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
    int32_t piece;
    // top
    const float* floor;           // [rows]: the value that a logit has to exceed
    float* z;                     // [rows][width of a piece]
    uint32_t* mask;               // [rows][width / 32]: which logits do, see class_of_bit
    int32_t first, width;         // the piece's first class and its width (a multiple of 256)
    int32_t all;                  // every logit is stored, without bits
    int32_t biased;               // the bias is to be added in every tile, else in the last one alone, which ends beyond the classes
};

// Classes of a piece: as many as the room for the gradient at the logits allows, a multiple of 256.
__device__ __host__ __forceinline__ int piece_width(int64_t cap, int64_t rows, int C) {
    const int64_t cp = ((int64_t)C + 255) / 256 * 256, fit = cap / rows / 256 * 256;
    return (int)(fit < 256 ? 256 : (fit < cp ? fit : cp));
}

// The class that bit `bit` of a mask's word stands for, from the word's first class.
__device__ __forceinline__ int class_of_bit(int bit) { return acc_row(bit & 15, bit >> 4); }

// What a tile's rows and classes bring along, in LDS.
template <int BB>
struct Extras {
    float bias[kTileC];
    f32x4 info[BB];               // see LogitsArgs
    int32_t label[BB];            // or, as bits, the floor
    int2 entry[BB][kHeldEntries];
    int held[BB];                 // entries of the row in this tile
};

// 64 times BYTES from memory to LDS, by a wavefront
template <int BYTES>
__device__ __forceinline__ void bring_lds(const void* from, void* to) {
    const auto* at = (const __attribute__((address_space(1))) void*)(static_cast<const char*>(from) + (threadIdx.x & 63) * BYTES);
    if constexpr (BYTES == 16) __builtin_amdgcn_global_load_lds(at, (__attribute__((address_space(3))) void*)to, 16, 0, 0);
    else __builtin_amdgcn_global_load_lds(at, (__attribute__((address_space(3))) void*)to, 4, 0, 0);
}

// KIND: what is made of the logits.  TEMPS: bit 0, exponentials as they are, bit 1, at the temperature; 4: both where the temperature is 2, e^z as
// the square of e^(z / 2) (an exponential takes the unit as long as four other instructions).  SPLIT: the gradient goes to
// three planes (fp32).
//
// Workgroups of many tiles (STREAM): a tile's work beside its products (7 us of 25 at 512 inputs) begins with the loads of the next tile's first
// step, so that these and what the next tile brings along are there when it is done; workgroups of one tile each waited 3.5 us for theirs.
// Two workgroups on a unit with tiles of 256 by 128, of one tile each, whose work beside the products ran while the other multiplied, took 2 to 8% more.
//
// Bound by the matrix units where the sums are long: 8,192 x 2,048 x 131,072 of bf16 in 3.74 to 3.87 ms are 1,140 to 1,180 TFLOP/s (a product
// of these sizes by the library 1,206), the units busy for 56% of the cycles, at the clock that they are held to. Where they are short it is what is
// made of a logit: 8,000 x 128 x 100,003 with both exponentials takes 474 us, of which the products are 170 and the vector units' instructions some
// 250; the gradients of 16,384 x 512 x 131,072 take 2.89 ms (761 TFLOP/s), a quarter of it for storing 4.3 GB.
//
// What passes between lanes goes through a piece of LDS that belongs to the wavefront, 32 rows of 64 classes at a time, where the last step's operands
// were: a lane has its classes in fours, memory wants a row's next to each other, and a target's logit lies wherever its class is. Four classes of
// row r lie at u ^ (r & 15), u their number, so that neither rows nor columns meet in a bank.
template <int KIND, int TEMPS, bool SPLIT, bool STREAM, class P>
__global__ __launch_bounds__(P::T, 2) void classes_logits_kernel(LogitsArgs a) {
    constexpr int TA = P::TA, TB = P::TB, T = P::T, WA = kTileC / 32 / TA, BB = P::kRowsB, WB = BB / 32 / TB;
    static_assert(TA % 2 == 0 && BB <= T && kTileC <= T, "two blocks of classes at a time; a thread a row, and a class");
    // with one tile all of LDS is free in the end
    static_assert(T / 64 * 32 * 64 * 4 <= (STREAM ? 2 * P::kStage : P::kLdsBytes), "the wavefronts' pieces fit where operands were");
    static_assert(!STREAM || P::kStages == 2, "one part of LDS for the next tile's first step, one for the pieces");
    constexpr int kStores = KIND == LOGITS_GRAD ? TA / 2 * TB * 4 * (SPLIT ? 3 : 1) : 0;      // of every thread at the end of a tile
    extern __shared__ __attribute__((aligned(16))) char smem[];
    uint16_t* lds = reinterpret_cast<uint16_t*>(smem);
    Extras<BB>* extras = reinterpret_cast<Extras<BB>*>(smem + P::kLdsBytes);                  // of this tile and, of many, of the next
    const Layer& l = a.layer;
    const int count = l.shape->count;
    int c_first = a.first, c_end = a.first + a.width, width = a.width;
    if constexpr (KIND == LOGITS_GRAD) {
        width = l.shape->width;
        const int64_t from = (int64_t)a.piece * width;
        if (from >= l.C) return;
        c_first = (int)from;
        c_end = c_first + width;
    }
    if (c_end > l.C) c_end = l.C;
    Tiles tiles(blockIdx.x, gridDim.x, (count + BB - 1) / BB, (c_end - c_first + kTileC - 1) / kTileC);
    if (!tiles.on()) return;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wa0 = (wave % WA) * (32 * TA), wb0 = (wave / WA) * (32 * TB);
    const int steps = (l.F + P::kStepOf - 1) / P::kStepOf;

    struct Place {
        int m0, c0;
        int64_t biased;           // no gap in here: copies of one go through memory
        TileOperand a, b;
    };
    auto place = [&]() {
        Place p;
        tiles.at(p.m0, p.c0);
        p.m0 *= BB;
        p.c0 = c_first + p.c0 * kTileC;
        p.biased = a.biased || p.c0 + kTileC > l.C;
        p.a = TileOperand{l.w + p.c0, l.ldw, l.w_plane, l.cw - 8 - p.c0, l.F};
        p.b = TileOperand{l.x + (int64_t)p.m0 * l.fp, l.fp, l.x_plane, l.most - 1 - p.m0, l.fp};
        return p;
    };
    // What a tile brings along: what lies in memory as it is needed goes straight to LDS ...
    auto bring_extras = [&](int fm0, int fc0, bool fbiased, Extras<BB>* x) __attribute__((always_inline)) {
        if (fbiased && wave == 0) bring_lds<16>(l.bias + fc0, x->bias);
        if constexpr (KIND == LOGITS_GRAD)
            for (int q = wave; q < BB / 64; q += T / 64) bring_lds<16>(a.info + fm0 + 64 * q, x->info + 64 * q);
        const int32_t* each = KIND == LOGITS_TOP ? reinterpret_cast<const int32_t*>(a.floor) : a.labels;
        if (each && !(KIND == LOGITS_TOP && a.all))
            for (int q = T / 64 - 1 - wave; q < BB / 64; q += T / 64) bring_lds<4>(each + fm0 + 64 * q, x->label + 64 * q);
    };
    // ... and a row's entries are fetched by a thread in two goes.  In variables of their own: together they end up in memory.
    static_assert(kHeldEntries == 2, "two entries are fetched");
    int next_n = 0, next_from = 0, class0 = 0, class1 = 0, weight0 = 0, weight1 = 0;
    auto fetch = [&](int fm0, int fc0) __attribute__((always_inline)) {
        if (KIND == LOGITS_TOP || a.labels) return;
        const int64_t m = fm0 + tid;
        int n = 0, from = 0;
        if (tid < BB && m < count) {
            const uint16_t* s = a.starts + m * (a.tiles + 1) + fc0 / kTileC;
            from = s[0];
            n = s[1];
        }
        next_n = n;
        next_from = from;
    };
    auto fetch_entries = [&](int fm0, int fc0) __attribute__((always_inline)) {
        if (KIND == LOGITS_TOP || a.labels) return;
        int2 e0 = {0, 0}, e1 = {0, 0};
        const int2* e = a.entries + (int64_t)(fm0 + tid) * a.k + next_from;
        next_n -= next_from;
        if (next_n > 0) e0 = e[0];
        if (next_n > 1) e1 = e[1];
        class0 = e0.x - fc0;
        weight0 = e0.y;
        class1 = e1.x - fc0;
        weight1 = e1.y;
    };
    auto put = [&](Extras<BB>& x) __attribute__((always_inline)) {
        if (KIND == LOGITS_TOP || a.labels || tid >= BB) return;
        x.held[tid] = next_n;
        x.entry[tid][0] = int2{class0, weight0};
        x.entry[tid][1] = int2{class1, weight1};
    };

    // The last step of a tile and what is made of its logits.  now: the last step's operands, then the wavefronts' pieces (one tile: all of LDS);
    // next: where the next tile's first step goes.
    auto finish = [&](uint16_t* __restrict__ now, uint16_t* __restrict__ next, const Extras<BB>* __restrict__ x, Extras<BB>* __restrict__ nx, const P& product, const Place& p,
                      f32x16 (&acc)[TA][TB], bool more, const Place& np, typename P::Walk& walk) {
        if constexpr (STREAM) {
            if (more) {
                product.bring(walk, np.a, np.b, next);
                product.advance(walk, np.a, np.b);
                bring_extras(np.m0, np.c0, np.biased, nx);
            }
            product.multiply(now, wa0, wb0, acc);
        }
        const int m0 = p.m0, c0 = p.c0, tile = c0 / kTileC;
        // the lane's number anew: addresses made from it here would else be kept from tile to tile, in registers that the products need
        int lane = threadIdx.x & 63;
        asm volatile("" : "+v"(lane));
        const int li = lane & 31, lh = lane >> 5;
        if (p.biased) {
#pragma unroll
            for (int i = 0; i < TA; ++i) {
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const f32x4 b = *reinterpret_cast<const f32x4*>(x->bias + wa0 + 32 * i + 8 * q + 4 * lh);
#pragma unroll
                    for (int j = 0; j < TB; ++j)
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[i][j][4 * q + e] += b[e];
                }
                __builtin_amdgcn_sched_barrier(0);             // not all of the bias at once: there are no registers for it
            }
        }
        if (more) fetch(np.m0, np.c0);
        __builtin_amdgcn_s_waitcnt(0xC07F);                    // this wavefront has read the operands (lgkmcnt 0)
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();                          // all of them have
        asm volatile("" ::: "memory");
        float* mine = reinterpret_cast<float*>(now) + wave * (32 * 64);
        // blocks 2 h and 2 h + 1 of rows 32 j .. to the wavefront's piece
        auto show = [&](int j, int h) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    *reinterpret_cast<f32x4*>(mine + li * 64 + 4 * ((8 * i + 2 * q + lh) ^ (li & 15))) =
                        f32x4{acc[2 * h + i][j][4 * q], acc[2 * h + i][j][4 * q + 1], acc[2 * h + i][j][4 * q + 2], acc[2 * h + i][j][4 * q + 3]};
        };
        auto place_of = [&](int r, int c) { return mine + r * 64 + 4 * ((c >> 2) ^ (r & 15)) + (c & 3); };
        // entries of row r of the tile among the 64 classes of half h, by one lane of the row
        auto each_entry = [&](int r, int h, float of_label, auto&& use) {
            if (a.labels) {
                const int rel = x->label[r] - c0 - wa0 - 64 * h;
                if (lh == 0 && rel >= 0 && rel < 64 && m0 + r < count) use(place_of(li, rel), of_label);
                return;
            }
            const int n = lh == 0 ? x->held[r] : 0;
            const int2 e0 = x->entry[r][0], e1 = x->entry[r][1];
            auto one = [&](const int2& e, bool there) {
                const int rel = e.x - wa0 - 64 * h;
                if (there && rel >= 0 && rel < 64) use(place_of(li, rel), __int_as_float(e.y));
            };
            one(e0, n > 0);
            one(e1, n > 1);
#pragma unroll 1
            for (int j = kHeldEntries; j < n; ++j) {
                const int64_t m = m0 + r;
                int2 e = a.entries[m * a.k + a.starts[m * (a.tiles + 1) + tile] + j];
                e.x -= c0;
                one(e, true);
            }
        };
        if constexpr (KIND == LOGITS_GRAD) {
            float column[TA / 2] = {};                         // sums over the rows of a class a lane, of each half
#pragma unroll
            for (int j = 0; j < TB; ++j) {
                const int row = wb0 + 32 * j + li;
                // a exp(z - lse) = (a 2^(rest)) 2^(z log2 e - least), least = lse log2 e rounded, which leaves out `rest`
                f32x4 info = {INFINITY, INFINITY, 0.f, 0.f};
                if (m0 + row < count) info = x->info[row];
                const float of_label = info[2];
                const float least = info[0] * kLog2e, least_t = info[1] * kLog2e, log2e_t = kLog2e * a.inv_t;
                if (m0 + row < count) {
                    const double rest_t = (double)least_t - (double)info[1] * (double)kLog2e;
                    if (TEMPS == 4) info[2] *= exp2_of((float)(2.0 * (double)least_t - (double)info[0] * (double)kLog2e));
                    else if (TEMPS & 1) info[2] *= exp2_of((float)((double)least - (double)info[0] * (double)kLog2e));
                    if (TEMPS > 1) info[3] *= exp2_of((float)rest_t);
                }
#pragma unroll
                for (int h = 0; h < TA / 2; ++h) {
                    if constexpr (TEMPS == 4) {    // exp(z - lse) = exp(z / 2 - lse_t)^2 exp(2 lse_t - lse)
#pragma unroll
                        for (int i = 2 * h; i < 2 * h + 2; ++i)
#pragma unroll
                            for (int r = 0; r < 16; ++r) {
                                const float e = exp2_of(fmaf(acc[i][j][r], log2e_t, -least_t));
                                acc[i][j][r] = e * fmaf(e, info[2], info[3]);
                            }
                    } else {
#pragma unroll
                        for (int i = 2 * h; i < 2 * h + 2; ++i)
#pragma unroll
                            for (int r = 0; r < 16; ++r) {
                                const float z = acc[i][j][r];
                                float g = 0.f;
                                if constexpr (TEMPS & 1) g = info[2] * exp2_of(fmaf(z, kLog2e, -least));
                                if constexpr (TEMPS & 2) g += info[3] * exp2_of(fmaf(z, log2e_t, -least_t));
                                acc[i][j][r] = g;
                            }
                    }
                    __builtin_amdgcn_sched_barrier(0);
                    show(j, h);
                    __builtin_amdgcn_sched_barrier(0);
                    each_entry(row, h, of_label, [&](float* at, float w) { *at -= w; });
                    if (a.gbias)
#pragma unroll
                        for (int r = 0; r < 32; ++r) column[h] += *place_of(r, lane);
                    // eight classes of a row a lane, so that a row's are next to each other
                    const int r0 = lane / 8, u = 2 * (lane & 7);
                    char* tile_at = reinterpret_cast<char*>(a.g + (int64_t)m0 * width + (c0 - c_first));       // the same for all: offsets are 32 bits
                    const uint32_t to = ((uint32_t)(wb0 + 32 * j + r0) * (uint32_t)width + wa0 + 64 * h + 4 * u) * 2;
#pragma unroll
                    for (int r = 0; r < 32; r += 8) {
                        const float* from = mine + (r0 + r) * 64;
                        const int turn = (r0 + r) & 15;
                        const f32x4 v0 = *reinterpret_cast<const f32x4*>(from + 4 * (u ^ turn)), v1 = *reinterpret_cast<const f32x4*>(from + 4 * ((u + 1) ^ turn));
                        uint16_t* at = reinterpret_cast<uint16_t*>(tile_at + (to + (uint32_t)r * (uint32_t)width * 2));
                        if constexpr (SPLIT) {
                            const float v[8] = {v0[0], v0[1], v0[2], v0[3], v1[0], v1[1], v1[2], v1[3]};
                            put8(v, 6, at, a.g_plane, 0);
                        } else {
                            *reinterpret_cast<u32x4*>(at) = u32x4{pack_bf16(v0[0], v0[1]), pack_bf16(v0[2], v0[3]), pack_bf16(v1[0], v1[1]), pack_bf16(v1[2], v1[3])};
                        }
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
                if (j == 0 && more) fetch_entries(np.m0, np.c0);
            }
            if (a.gbias) {
                float* sums = reinterpret_cast<float*>(now);   // [WB][256], over the pieces
                __syncthreads();
#pragma unroll
                for (int h = 0; h < TA / 2; ++h) sums[(wave / WA) * kTileC + wa0 + 64 * h + lane] = column[h];
                __syncthreads();
                if (tid < kTileC) {
                    float v = sums[tid];
#pragma unroll
                    for (int w = 1; w < WB; ++w) v += sums[w * kTileC + tid];
                    a.gbias[(int64_t)(m0 / BB) * ((l.C + 255) / 256 * 256) + c0 + tid] = v;
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
                if (a.all) {                                   // columns up to the piece's width are there, beyond the classes too
                    if (on)
#pragma unroll
                        for (int i = 0; i < TA; ++i)
#pragma unroll
                            for (int q = 0; q < 4; ++q)
                                *reinterpret_cast<f32x4*>(row + 32 * i + 8 * q) =
                                    f32x4{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
                    continue;
                }
                const float floor = __int_as_float(x->label[wb0 + 32 * j + li]);
                uint32_t mask[TA];                             // bit r of a lane: accumulator r; those of lanes 32 on from bit 16 on
#pragma unroll
                for (int i = 0; i < TA; ++i) {
                    const int c = c0 + wa0 + 32 * i;
                    uint32_t bits = 0;
#pragma unroll
                    for (int r = 15; r >= 0; --r) bits = bits + bits + !(acc[i][j][r] <= floor);
                    if (c + 32 > l.C)
                        for (int r = 0; r < 16; ++r)
                            if (c + acc_row(r, lh) >= l.C) bits &= ~(1u << r);
                    mask[i] = on ? bits : 0u;
                }
#pragma unroll
                for (int h = 0; h < TA / 2; ++h)
                    if (__any((mask[2 * h] | mask[2 * h + 1]) != 0)) {
                        show(j, h);
#pragma unroll
                        for (int i = 0; i < 2; ++i)
                            for (uint32_t bits = mask[2 * h + i]; bits; bits &= bits - 1) {
                                const int at = 32 * i + acc_row(__ffs((int)bits) - 1, 0);
                                row[64 * h + at] = *place_of(li, 4 * lh + at);
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
        float most[TB], sum[TB], sum_t[TB], picked[TB];
#pragma unroll
        for (int j = 0; j < TB; ++j) {
            const int row = wb0 + 32 * j + li;
            most[j] = -INFINITY;
            sum[j] = sum_t[j] = picked[j] = 0.f;
            if constexpr (KIND == LOGITS_STATS) {
                if (__any(a.labels ? (uint32_t)(x->label[row] - c0 - wa0) < 32u * TA : x->held[row] > 0))
#pragma unroll
                    for (int h = 0; h < TA / 2; ++h) {
                        show(j, h);
                        each_entry(row, h, 1.f, [&](const float* at, float w) { picked[j] = fmaf(w, *at, picked[j]); });
                    }
            }
#pragma unroll
            for (int i = 0; i < TA; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) most[j] = fmaxf(most[j], acc[i][j][r]);
            most[j] = fmaxf(most[j], __shfl_xor(most[j], 32));
            most[j] = fmaxf(most[j] * kLog2e, kLeastExponent);
            if constexpr (TEMPS == 4) {
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
            if constexpr (TEMPS > 1) sum_t[j] += __shfl_xor(sum_t[j], 32);
            __builtin_amdgcn_sched_barrier(0);
            if (j == 0 && more) fetch_entries(np.m0, np.c0);
        }
        // the wavefronts' sums through their pieces: 32 TB rows of four values
        if (lh == 0) {
#pragma unroll
            for (int j = 0; j < TB; ++j) *reinterpret_cast<f32x4*>(mine + 4 * (32 * j + li)) = f32x4{most[j], sum[j], sum_t[j], picked[j]};
        }
        __syncthreads();
        if (tid < BB && m0 + tid < count) {
            const int64_t m = m0 + tid;
            auto of = [&](int w) {                             // row tid's values of the w-th wavefront along the classes
                return *reinterpret_cast<const f32x4*>(reinterpret_cast<const float*>(now) + ((tid / (32 * TB)) * WA + w) * (32 * 64) + 4 * (tid % (32 * TB)));
            };
            f32x4 v = of(0);
            float top = v[0], s = v[1], st = v[2], z = v[3];
#pragma unroll
            for (int w = 1; w < WA; ++w) {
                v = of(w);
                join(top, s, st, v[0], v[1], v[2], a.inv_t);
                z += v[3];
            }
            const int64_t at = (int64_t)tile * l.stats + m;
            a.parts.most[at] = top;
            a.parts.sum[at] = s;
            if constexpr (KIND == LOGITS_STATS) {
                if constexpr (TEMPS > 1) a.parts.sum_t[at] = st;
                if (!a.labels) a.parts.picked[at] = z;
                else if ((uint32_t)(x->label[tid] - c0) < (uint32_t)kTileC) a.parts.picked[m] = z;
            }
        }
    };

    P product;
    Place p = place();
    int ring = 0, turn = 0;
    typename P::Walk walk;
    f32x16 acc[TA][TB];
    if constexpr (P::kReadOnce) {
        bring_extras(p.m0, p.c0, p.biased, extras);
        fetch(p.m0, p.c0);
        fetch_entries(p.m0, p.c0);
        put(extras[0]);
        constexpr int eb = P::PLANES == 1 ? 2 : 4;
        const typename P::Operand oa = {static_cast<const char*>(l.raw) + (int64_t)p.c0 * eb, l.ld_raw, l.C - p.c0, l.F};
        product.run(oa, p.b, count, 0, steps, lds, wa0, wb0, acc);
        finish(lds, lds, extras, extras, product, p, acc, false, p, walk);
        return;
    } else {
    if constexpr (STREAM) {
        walk = product.start(p.a, p.b, 0, steps, l.terms);
        product.bring(walk, p.a, p.b, lds);
        product.advance(walk, p.a, p.b);
    } else {
        walk = product.begin(p.a, p.b, 0, steps, l.terms, lds);
    }
    bring_extras(p.m0, p.c0, p.biased, extras);
    fetch(p.m0, p.c0);
    fetch_entries(p.m0, p.c0);
    put(extras[0]);
    if constexpr (!STREAM) {
        product.run(walk, p.a, p.b, lds, wa0, wb0, acc);
        finish(lds, lds, extras, extras, product, p, acc, false, p, walk);
        return;
    }
    for (bool first = true;; first = false) {
        P::clear(acc);
        if (first) product.template steps<0>(walk, p.a, p.b, 1, ring, lds, wa0, wb0, acc);
        else product.template steps<kStores>(walk, p.a, p.b, 1, ring, lds, wa0, wb0, acc);
        // the last step; there is no other where the first one is the last
        if (kStores > 0 && walk.n == 1 && !first) P::template meet<kStores>();
        else P::template meet<0>();
        Place np = p;
        tiles.id += tiles.step;
        const bool more = tiles.on();
        if (more) {
            np = place();
            walk = product.start(np.a, np.b, 0, steps, l.terms);
        }
        finish(lds + ring * P::kStage, lds + (ring ^ 1) * P::kStage, extras + turn, extras + (turn ^ 1), product, p, acc, more, np, walk);
        if (!more) return;
        turn ^= 1;
        put(extras[turn]);
        p = np;
        ring ^= 1;
    }
    }
}

template <bool STREAM, class P>
constexpr int logits_lds() { return P::kLdsBytes + (STREAM ? 2 : 1) * (int)sizeof(Extras<P::kRowsB>); }

template <int KIND, int TEMPS, bool SPLIT, bool STREAM, class P>
gas_status launch_logits_tile(const LogitsArgs& a, int64_t tiles, hipStream_t s) {
    constexpr int smem = logits_lds<STREAM, P>();
    static_assert(smem <= 160 * 1024, "LDS of a compute unit");
    static const gas_status attr = lds_of(classes_logits_kernel<KIND, TEMPS, SPLIT, STREAM, P>, smem);
    if (attr != GAS_OK) return attr;
    GAS_REQUIRE(tiles <= 0x3FFFFFFFLL, "too many tiles for one launch");
    int64_t blocks = (tiles + 7) / 8 * 8;
    if (STREAM && blocks > 256) blocks = 256;                  // one for a compute unit, whose LDS it fills
    GAS_REQUIRE(blocks <= 0x7FFFFFLL, "too many tiles for one launch");
    hipLaunchKernelGGL((classes_logits_kernel<KIND, TEMPS, SPLIT, STREAM, P>), dim3((unsigned)blocks), dim3(P::T), smem, s, a);
    GAS_CHECK_HIP(hipGetLastError());
    return GAS_OK;
}

// tiles: of rows by classes, at most, for tiles of rows_of_tile() rows
using FewRows = TileProduct<kTileC, 64, 4, 1, true, false>;
template <bool BF> using FewRowsOnce = ReadOnceProduct<kTileC, 64, 4, 1, true, BF>;
constexpr int kRowsTile = 256;
using ManyRows = TileProduct<kTileC, kRowsTile, 2, 4, true, false, 64, 2>;
// Rows of a tile: 64 where there are no more rows, or where tiles of 64 are all under way at once, two on a unit; tiles of 256 take less where there would be
// a second round. Forward in us, 64 rows and 256:
//     512 tiles of 64     512 x 1,024 x 16,384 fp32    158   184        512 x 256 x 16,384 bf16    19   22
//     516                 256 x 1,024 x 33,000         286   235        256 x 256 x 33,000         24   22
//     752                 512 x 256 x 24,000            80    66        512 x 1,024 x 24,000       49   41
inline int rows_of_tile(int64_t n, int C) { return n <= 64 || (n + 63) / 64 * (round_up(C, kTileC) / kTileC) <= 512 ? 64 : kRowsTile; }
template <int KIND, int TEMPS, bool SPLIT = false>
gas_status launch_logits(const LogitsArgs& a, int tile_rows, int64_t tiles, hipStream_t s) {
    if (!a.layer.w) {
        // SPLIT goes with fp32
        if (a.layer.terms == 1) {
            if constexpr (!SPLIT) return launch_logits_tile<KIND, TEMPS, SPLIT, false, FewRowsOnce<true>>(a, tiles, s);
        } else if constexpr (SPLIT || KIND != LOGITS_GRAD) {
            return launch_logits_tile<KIND, TEMPS, SPLIT, false, FewRowsOnce<false>>(a, tiles, s);
        }
    }
    if (tile_rows == 64) return launch_logits_tile<KIND, TEMPS, SPLIT, false, FewRows>(a, tiles, s);
    return launch_logits_tile<KIND, TEMPS, SPLIT, true, ManyRows>(a, tiles, s);
}

}  // namespace
}  // namespace gas
