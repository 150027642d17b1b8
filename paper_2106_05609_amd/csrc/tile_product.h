// Products of bf16 matrices by tiles, for the output layer over many classes (classes.hip): the main loop shared by its logits,
// its input gradient and its weight gradient.
//
// A workgroup of WA x WB wavefronts owns BA rows of the first operand by BB rows of the second, sum over k, k in steps of 64 or 32.  An
// operand lies in memory with k contiguous (element (r, k) at p[r ld + k]) or with r contiguous (TURNED: at p[k ld + r]); a turned one is
// put right on its way out of LDS (ds_read_b64_tr_b16: sixteen lanes read four k of sixteen rows, and a lane receives four k of
// one row), so nothing is transposed in memory: the logits read W [F, C] turned and X as it lies, the input gradient W and G as they lie, the
// weight gradient both turned.
// Loads go from memory to LDS without registers (16 bytes a lane), the next step's under way while one is multiplied.  LDS holds
// the lanes' pieces in the order of their numbers, so which piece a lane fetches is exchanged instead: of row r, piece p
// lies at p ^ (r & 7); of a turned operand's k, unit u of 16 bytes at u ^ 4 (k & 3).  Sixteen-byte reads of eight
// neighbouring rows, and the 32 bytes of each of four k, then fall on banks of their own.
//
// fp32 operands come as three bf16 planes (split.h says how and what is dropped): `terms` = 6 products of planes follow one
// another over the same accumulators, the smallest first, so that only the last one's sums round at the result's size.  ReadOnceProduct, which takes all
// six at every step, has accumulators of their own for the small ones.
#pragma once
#include "split.h"

namespace gas {
namespace {

constexpr int kStepK = 64;                        // k are a multiple of it, padded or split

struct TileOperand {
    const uint16_t* p;        // the tile's first row and first k
    int64_t ld, plane;        // in elements
    int last;                 // the last row of the tile that can be read (rows beyond repeat it); turned: the last 8 rows' first
    int k;                    // k that can be read (beyond, the last ones repeat: the other operand has zeros there)
};

template <int BA, int BB, int WA, int WB, bool ATURNED, bool BTURNED, int STEP = 32, int STAGES = 3>
struct TileProduct {
    static constexpr int T = 64 * WA * WB, TA = BA / 32 / WA, TB = BB / 32 / WB;
    static constexpr int kStage = (BA + BB) * STEP;                        // elements
    static constexpr int kStepOf = STEP, kRowsA = BA, kRowsB = BB, kStages = STAGES;
    static constexpr bool kReadOnce = false;
    static constexpr int kLdsBytes = STAGES * kStage * 2;
    static_assert((STEP == 32 || STEP == 64) && (STAGES == 2 || STAGES == 3), "");
    // where piece `piece` of row `row` lies, in pieces of 16 bytes
    static __device__ __forceinline__ int swap(int row) { return STEP == 64 ? row & 7 : (row >> 1) & 3; }
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    typedef short s16x8 __attribute__((ext_vector_type(8)));

    template <int R, bool TURNED>
    struct Loads {
        static constexpr int N = R * STEP / 8 / T;
        static_assert(R * STEP / 8 % T == 0, "every thread brings as many pieces");
        uint32_t at[N];                                                    // bytes from the step's first element
        __device__ __forceinline__ void init(const TileOperand& o) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int q = i * T + (int)threadIdx.x;
                if constexpr (TURNED) {
                    const int kr = q / (R / 8), unit = (q % (R / 8)) ^ (4 * (kr & 3) & (R / 8 - 1));
                    at[i] = (uint32_t)((int64_t)kr * o.ld + (8 * unit < o.last ? 8 * unit : o.last)) * 2;
                } else {
                    const int row = q / (STEP / 8), piece = (q % (STEP / 8)) ^ swap(row);
                    at[i] = (uint32_t)((int64_t)(row < o.last ? row : o.last) * o.ld + 8 * piece) * 2;
                }
            }
        }
        // the STEP k from `from` on, of which `left` can be read
        __device__ __forceinline__ void bring(const uint16_t* from, int64_t ld, int left, uint16_t* to) const {
            const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                uint32_t a = at[i];
                if (left < STEP) {
                    const int q = i * T + (int)threadIdx.x;
                    if constexpr (TURNED) {
                        const int kr = q / (R / 8), over = kr - (left - 1);
                        a -= over > 0 ? (uint32_t)(over * ld * 2) : 0u;
                    } else {
                        const int over = 8 * ((q % (STEP / 8)) ^ swap(q / (STEP / 8))) - (left - 8);
                        a -= over > 0 ? (uint32_t)over * 2 : 0u;
                    }
                }
                __builtin_amdgcn_global_load_lds(
                    (const __attribute__((address_space(1))) void*)(reinterpret_cast<const char*>(from) + a),
                    (__attribute__((address_space(3))) void*)(to + (i * T + wave * 64) * 8), 16, 0, 0);
            }
        }
    };

    template <int R, bool TURNED>
    static __device__ __forceinline__ bf16x8 fragment(const uint16_t* tile, int r0, int kk) {
        const int lane = threadIdx.x & 63, li = lane & 31, lh = lane >> 5;
        if constexpr (TURNED) {
            const int i16 = lane & 15, r = r0 + 16 * ((lane >> 4) & 1) + 4 * (i16 & 3);
            s16x4 h[2];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const int k = 16 * kk + 8 * lh + 4 * t + (i16 >> 2);
                const uint16_t* p = tile + k * R + 8 * ((r >> 3) ^ (4 * (k & 3) & (R / 8 - 1))) + (r & 7);
                h[t] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(p));
            }
            return __builtin_bit_cast(bf16x8, s16x8{h[0][0], h[0][1], h[0][2], h[0][3], h[1][0], h[1][1], h[1][2], h[1][3]});
        } else {
            const int row = r0 + li;
            return *reinterpret_cast<const bf16x8*>(tile + (row * (STEP / 8) + ((2 * kk + lh) ^ swap(row))) * 8);
        }
    }

    Loads<BA, ATURNED> la;
    Loads<BB, BTURNED> lb;

    // One step: the next one's loads, then this one's products.  `now` and `next` are different parts of LDS, which the compiler has to
    // know (__restrict__): it would otherwise wait for the loads before every read of LDS.
    __device__ __forceinline__ void step(const uint16_t* __restrict__ now, uint16_t* __restrict__ next, bool more, const uint16_t* a,
                                         int64_t lda, int left_a, const uint16_t* b, int64_t ldb, int left_b, int wa0, int wb0,
                                         f32x16 (&acc)[TA][TB]) const {
        if (more) {
            la.bring(a, lda, left_a, next);
            lb.bring(b, ldb, left_b, next + BA * STEP);
        }
        multiply(now, wa0, wb0, acc);
    }
    __device__ __forceinline__ void multiply(const uint16_t* now, int wa0, int wb0, f32x16 (&acc)[TA][TB]) const {
#pragma unroll
        for (int kk = 0; kk < STEP / 16; ++kk) {
            bf16x8 fa[TA], fb[TB];
#pragma unroll
            for (int j = 0; j < TB; ++j) fb[j] = fragment<BB, BTURNED>(now + BA * STEP, wb0 + 32 * j, kk);
#pragma unroll
            for (int i = 0; i < TA; ++i) fa[i] = fragment<BA, ATURNED>(now, wa0 + 32 * i, kk);
#pragma unroll
            for (int i = 0; i < TA; ++i)
#pragma unroll
                for (int j = 0; j < TB; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa[i], fb[j], acc[i][j], 0, 0, 0);
        }
    }

    // Where the loads of a sum over `terms` terms of steps [first, last) stand.
    struct Walk {
        const uint16_t *a, *b;
        int64_t step_a, step_b;
        int first, last, k, term, terms, n;               // n: steps of all terms
    };
    static constexpr int kLoads = Loads<BA, ATURNED>::N + Loads<BB, BTURNED>::N;      // of a thread for a step
    static_assert(kLoads * (STAGES - 2) < 64, "the counter of loads under way");

    __device__ __forceinline__ void place(Walk& w, const TileOperand& a, const TileOperand& b) const {
        // planes of the terms, the smallest product first: m m, l h, h l, m h, h m, h h, a nibble a term from the lowest; one term: h h
        const int pa = w.terms == 1 ? 0 : 0x010201 >> (4 * w.term) & 15, pb = w.terms == 1 ? 0 : 0x001021 >> (4 * w.term) & 15;
        w.a = a.p + pa * a.plane + w.first * w.step_a;
        w.b = b.p + pb * b.plane + w.first * w.step_b;
    }
    __device__ __forceinline__ void advance(Walk& w, const TileOperand& a, const TileOperand& b) const {
        if (++w.k == w.last) {
            w.k = w.first;
            if (++w.term < w.terms) place(w, a, b);
        } else {
            w.a += w.step_a;
            w.b += w.step_b;
        }
    }
    __device__ __forceinline__ void bring(const Walk& w, const TileOperand& a, const TileOperand& b, uint16_t* to) const {
        la.bring(w.a, a.ld, a.k - STEP * w.k, to);
        lb.bring(w.b, b.ld, b.k - STEP * w.k, to + BA * STEP);
    }
    // Where the loads of a tile stand before its first step; the loads themselves are begun by bring() and advance().
    __device__ __forceinline__ Walk start(const TileOperand& a, const TileOperand& b, int first, int last, int terms) {
        la.init(a);
        lb.init(b);
        Walk w;
        w.step_a = ATURNED ? STEP * a.ld : STEP;
        w.step_b = BTURNED ? STEP * b.ld : STEP;
        w.first = w.k = first;
        w.last = last;
        w.term = 0;
        w.terms = terms;
        w.n = last > first ? (last - first) * terms : 0;
        place(w, a, b);
        return w;
    }
    // The first steps' loads; other work may follow before run().
    __device__ __forceinline__ Walk begin(const TileOperand& a, const TileOperand& b, int first, int last, int terms, uint16_t* lds) {
        Walk w = start(a, b, first, last, terms);
#pragma unroll
        for (int s = 0; s < STAGES - 1; ++s)
            if (s < w.n) {
                bring(w, a, b, lds + s * kStage);
                advance(w, a, b);
            }
        return w;
    }
    static __device__ __forceinline__ void clear(f32x16 (&acc)[TA][TB]) {
#pragma unroll
        for (int i = 0; i < TA; ++i)
#pragma unroll
            for (int j = 0; j < TB; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
    }
    // Waits until at most N of this thread's memory operations, and none of LDS, are under way; then for everyone.
    template <int N>
    static __device__ __forceinline__ void meet() {
        static_assert(N < 64, "the counter of memory operations under way");
        __builtin_amdgcn_s_waitcnt(0x0070 | (N & 15) | (N >> 4 << 14));
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    }
    // The products of a tile's steps but for the last `keep` ones; ring: where in LDS its first step's operands are, and in the end the next
    // one's.  AFTER: operations that every thread has begun since the loads of the first step.
    template <int AFTER>
    __device__ __forceinline__ void steps(Walk& w, const TileOperand& a, const TileOperand& b, int keep, int& ring, uint16_t* lds, int wa0, int wb0,
                                          f32x16 (&acc)[TA][TB]) const {
#pragma unroll 1
        for (int s = 0; s < w.n - keep; ++s) {
            // this step's loads have arrived (those of the step after it may be under way), everyone is done with the step before
            if (STAGES == 3 && s + 1 < w.n) meet<kLoads>();
            else if (AFTER > 0 && s == 0) meet<AFTER>();
            else meet<0>();
            const bool more = s + STAGES - 1 < w.n;
            int next = ring + STAGES - 1;
            if (next >= STAGES) next -= STAGES;
            step(lds + ring * kStage, lds + next * kStage, more, w.a, a.ld, a.k - STEP * w.k, w.b, b.ld, b.k - STEP * w.k, wa0, wb0, acc);
            if (more) advance(w, a, b);
            ring = ring + 1 == STAGES ? 0 : ring + 1;
        }
    }
    // acc = the products.  Called by every thread; LDS is free for other use afterwards.
    __device__ __forceinline__ void run(Walk& w, const TileOperand& a, const TileOperand& b, uint16_t* lds, int wa0, int wb0, f32x16 (&acc)[TA][TB]) {
        clear(acc);
        int ring = 0;
        steps<0>(w, a, b, 0, ring, lds, wa0, wb0, acc);
        __syncthreads();
    }
    __device__ __forceinline__ void run(const TileOperand& a, const TileOperand& b, int first, int last, int terms, uint16_t* lds, int wa0, int wb0,
                                        f32x16 (&acc)[TA][TB]) {
        Walk w = begin(a, b, first, last, terms, lds);
        run(w, a, b, lds, wa0, wb0, acc);
    }
};

// The same sums where the first operand is read once and used by few rows of the second: packing it beforehand (16 bytes a value
// of fp32 and more, 4 of bf16) would take several times what reading it takes. It is read as it lies, any alignment and width, into
// registers, a step ahead, and goes to LDS in its parts; the second operand's planes are packed.  32 k a step, all terms of a step at once.
// Bound by reading it: the logits of 32 x 2,048 x 131,072 of fp32 take 183 us (5.9 TB/s).  Two or four steps ahead took more registers than there
// are, and 5 to 30% longer.
template <int BA, int BB, int WA, int WB, bool ATURNED, bool BF>
struct ReadOnceProduct {
    static constexpr int T = 64 * WA * WB, TA = BA / 32 / WA, TB = BB / 32 / WB, STEP = 32, PLANES = BF ? 1 : 3;
    static constexpr int kStepOf = STEP, kRowsA = BA, kRowsB = BB, kStages = 1;
    static constexpr int kA = BA * STEP, kB = BB * STEP;                   // elements of a plane
    static constexpr int kStage = PLANES * (kA + kB), kLdsBytes = kStage * 2 > T * 128 ? kStage * 2 : T * 128;      // room for 8 KB a wavefront afterwards
    static constexpr bool kReadOnce = true;
    using Same = TileProduct<BA, BB, WA, WB, ATURNED, false, STEP, 2>;     // where pieces lie in LDS, and how they are read
    static constexpr int NA = kA / 8 / T, NB = PLANES * kB / 8 / T;
    static_assert(kA / 8 % T == 0 && PLANES * kB / 8 % T == 0, "every thread brings as many pieces");
    typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));

    struct Operand {              // element (r, k) of the tile at p[r ld + k], turned at p[k ld + r]; rows and k that are there
        const void* p;
        int64_t ld;
        int rows, k;
    };
    struct Walk {
        int first, last;
    };
    union Piece {
        float f[8];
        u32x4 h;
    };
    Piece va[NA];
    u32x4 vb[NB];
    int blocks;                   // of 32 rows of the second operand that are wanted; the others' products are left out

    __device__ __forceinline__ void fetch(const Operand& a, const TileOperand& b, int k0) {
#pragma unroll
        for (int i = 0; i < NA; ++i) {
            const int q = i * T + (int)threadIdx.x;
            const int major = ATURNED ? q / (BA / 8) : q / (STEP / 8), minor = 8 * (ATURNED ? q % (BA / 8) : q % (STEP / 8));
            // turned: major a k, minor rows; else major a row, minor k
            const int majors = ATURNED ? a.k - k0 : a.rows, minors = ATURNED ? a.rows : a.k - k0;
            const int64_t at = ATURNED ? (int64_t)(k0 + major) * a.ld + minor : (int64_t)major * a.ld + k0 + minor;
            if constexpr (BF) va[i].h = u32x4{0u, 0u, 0u, 0u};
            else
#pragma unroll
                for (int e = 0; e < 8; ++e) va[i].f[e] = 0.f;
            if (major >= majors || minor >= minors) continue;
            if (minor + 8 <= minors) {
                if constexpr (BF) {
                    va[i].h = *reinterpret_cast<const u32x4_any*>(static_cast<const uint16_t*>(a.p) + at);
                } else {
                    const f32x4 x = *reinterpret_cast<const f32x4_any*>(static_cast<const float*>(a.p) + at);
                    const f32x4 y = *reinterpret_cast<const f32x4_any*>(static_cast<const float*>(a.p) + at + 4);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        va[i].f[e] = x[e];
                        va[i].f[4 + e] = y[e];
                    }
                }
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (minor + e < minors) {
                        if constexpr (BF) va[i].h[e / 2] |= (uint32_t)static_cast<const uint16_t*>(a.p)[at + e] << (16 * (e & 1));
                        else va[i].f[e] = static_cast<const float*>(a.p)[at + e];
                    }
            }
        }
        // the second operand: rows and k beyond what is there repeat the last ones, whose products nothing takes or which the first one's zeros meet
#pragma unroll
        for (int i = 0; i < NB; ++i) {
            const int q = i * T + (int)threadIdx.x, plane = q / (kB / 8), row = q % (kB / 8) / (STEP / 8), k = k0 + 8 * (q % (STEP / 8));
            vb[i] = *reinterpret_cast<const u32x4*>(b.p + plane * b.plane + (int64_t)(row < b.last ? row : b.last) * b.ld + (k < b.k - 8 ? k : b.k - 8));
        }
    }
    __device__ __forceinline__ void stage(uint16_t* lds) const {
#pragma unroll
        for (int i = 0; i < NA; ++i) {
            const int q = i * T + (int)threadIdx.x;
            int to;                                                        // in pieces
            if constexpr (ATURNED) {
                const int k = q / (BA / 8);
                to = k * (BA / 8) + ((q % (BA / 8)) ^ (4 * (k & 3) & (BA / 8 - 1)));
            } else {
                const int row = q / (STEP / 8);
                to = row * (STEP / 8) + ((q % (STEP / 8)) ^ Same::swap(row));
            }
            if constexpr (BF) {
                *reinterpret_cast<u32x4*>(lds + 8 * to) = va[i].h;
            } else {
                u32x4 h, m, l;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    uint32_t x, y, z;
                    split_pair(va[i].f[2 * e], va[i].f[2 * e + 1], x, y, z);
                    h[e] = x; m[e] = y; l[e] = z;
                }
                *reinterpret_cast<u32x4*>(lds + 8 * to) = h;
                *reinterpret_cast<u32x4*>(lds + 8 * to + kA) = m;
                *reinterpret_cast<u32x4*>(lds + 8 * to + 2 * kA) = l;
            }
        }
#pragma unroll
        for (int i = 0; i < NB; ++i) {
            const int q = i * T + (int)threadIdx.x, plane = q / (kB / 8), row = q % (kB / 8) / (STEP / 8), piece = q % (STEP / 8);
            *reinterpret_cast<u32x4*>(lds + PLANES * kA + plane * kB + 8 * (row * (STEP / 8) + (piece ^ Same::swap(row)))) = vb[i];
        }
    }
    // acc = the products over steps [first, last) of 32 k, with b's first `rows` rows.  Called by every thread; LDS is free for other use afterwards.
    __device__ __forceinline__ void run(const Operand& a, const TileOperand& b, int rows, int first, int last, uint16_t* lds, int wa0, int wb0,
                                        f32x16 (&acc)[TA][TB]) {
        static_assert(WB == 1, "a wavefront's blocks are the tile's");
        blocks = (rows + 31) / 32;
        // The small products have accumulators of their own, as in linear.hip: with one for all six, each step rounded six times at the sum's size (sums of
        // 2,048 terms were 5.9e-7 off, 2-norm, now 2.3e-7; 32 x 2,048 x 131,072 takes as long, 2 workgroups to a unit either way).
        f32x16 small[TA][TB];
        Same::clear(acc);
        if constexpr (!BF) Same::clear(small);
        if (first < last) fetch(a, b, STEP * first);
#pragma unroll 1
        for (int s = first; s < last; ++s) {
            __syncthreads();                                               // everyone is done with the step before
            stage(lds);
            __syncthreads();
            if (s + 1 < last) fetch(a, b, STEP * (s + 1));
            constexpr int PA[6] = {1, 2, 0, 1, 0, 0}, PB[6] = {1, 0, 2, 0, 1, 0};      // the smallest product first
#pragma unroll
            for (int kk = 0; kk < STEP / 16; ++kk) {
                bf16x8 fa[PLANES][TA], fb[PLANES][TB];
#pragma unroll
                for (int p = 0; p < PLANES; ++p) {
#pragma unroll
                    for (int i = 0; i < TA; ++i) fa[p][i] = Same::template fragment<BA, ATURNED>(lds + p * kA, wa0 + 32 * i, kk);
#pragma unroll
                    for (int j = 0; j < TB; ++j)
                        if (j == 0 || j < blocks) fb[p][j] = Same::template fragment<BB, false>(lds + PLANES * kA + p * kB, wb0 + 32 * j, kk);
                }
#pragma unroll
                for (int j = 0; j < TB; ++j)
                    if (j == 0 || j < blocks)
#pragma unroll
                        for (int t = BF ? 5 : 0; t < 6; ++t)
#pragma unroll
                            for (int i = 0; i < TA; ++i) {
                                f32x16& sum = t < 5 ? small[i][j] : acc[i][j];
                                sum = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa[PA[t]][i], fb[PB[t]][j], sum, 0, 0, 0);
                            }
            }
        }
        if constexpr (!BF) {
#pragma unroll
            for (int i = 0; i < TA; ++i)
#pragma unroll
                for (int j = 0; j < TB; ++j) acc[i][j] += small[i][j];
        }
        __syncthreads();
    }
};

}  // namespace
}  // namespace gas
