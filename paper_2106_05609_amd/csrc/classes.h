// The output layer over many classes, none of whose logits are kept: what its losses (classes.hip) and its top logits
// (classes_top.hip) share.
//     z_i = x_i W + bias,     X [n, F], W [F, C] of fp32 or bf16
// Rows that do not count (no label, no entry of a teacher's) have no product: those that do are numbered one after another on the device
// (`count` of them), and a kernel sized for all of them ends at once where there are none left.  What a later launch's shape
// depends on (the width of a piece of the classes, parts of a split sum) is worked out from `count` in every kernel alike.
#pragma once
#include "tile_product.h"

namespace gas {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kTileC = 256;                       // classes of a tile
constexpr int kMaxClasses = 1 << 22;              // a tile's 256 rows of W then lie within 4 GB
constexpr int kMaxWidth = 1 << 16;
constexpr int64_t kMaxRows = 1 << 25;             // a launch of 64 threads a row
constexpr int kReadOnceRows = 64;                 // up to so many rows W is not packed
constexpr int kCopiedClasses = 1 << 15;           // but for bf16 of no more classes
constexpr int64_t kCopiedElements = 1 << 22;      // and elements
constexpr int kRowsByVector = 8;                  // up to so many rows may be multiplied by the vector units
constexpr int kMaxEntries = 256;                  // of a teacher's row
constexpr int kHeldEntries = 2;                   // of a row in one tile that are fetched before the products

inline int64_t round_up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }

// What follows from the number of rows that count, worked out once on the device.
struct Shape {
    int32_t count, width;         // classes of a piece of the gradient at the logits
    int32_t rows;                 // of it that are stored: `count` up to whole tiles
    int32_t part_rows;            // of a part of GX
    int32_t splits_x, splits_w;   // parts of the sums of GX and GW
};

// What kernels know of the layer.
struct Layer {
    const uint16_t* x;            // [planes][rows up to 256][fp], packed, zero beyond the row and beyond the last row
    const uint16_t* w;            // [planes][F][ldw], columns up to cw readable; or NULL: it is read where and as it lies
    const void* raw;              // W itself, rows of ld_raw
    int64_t ld_raw;
    int64_t ldw, w_plane, x_plane;
    const float* bias;            // [C up to 256], -inf beyond C
    const Shape* shape;
    int32_t F, fp, C, cw, terms, most;     // fp: F up to 64; most: rows up to 256
    int32_t stats;                // rows of the tiles' statistics: up to 16
};

// ---- rows that count

struct Targets {
    const int32_t* labels;        // [n] or NULL
    const int32_t* ids;           // [n, k] or NULL
    const float* values;
    int64_t ld_ids, ld_values, n;
    int32_t k, C;
};

__device__ __forceinline__ bool entry_counts(int32_t id, float v, int C) { return id >= 0 && id < C && !(v == -INFINITY); }

__device__ __forceinline__ bool row_counts(const Targets& t, int64_t i) {
    if (t.labels && t.labels[i] >= 0 && t.labels[i] < t.C) return true;
    if (!t.ids) return false;
    for (int k = 0; k < t.k; ++k)
        if (entry_counts(t.ids[i * t.ld_ids + k], t.values[i * t.ld_values + k], t.C)) return true;
    return false;
}

// ---- packing

// elements 8 at a time into the planes: `to` in elements of a plane
__device__ __forceinline__ void put8(const float (&v)[8], int terms, uint16_t* p, int64_t plane, int64_t at) {
    u32x4 h, m, l;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        uint32_t a, b, c;
        split_pair(v[2 * e], v[2 * e + 1], a, b, c);
        h[e] = a; m[e] = b; l[e] = c;
    }
    *reinterpret_cast<u32x4*>(p + at) = h;
    if (terms > 1) {
        *reinterpret_cast<u32x4*>(p + at + plane) = m;
        *reinterpret_cast<u32x4*>(p + at + 2 * plane) = l;
    }
}

// eight elements of a row of any alignment, zero from `width` on
template <bool BF>
__device__ __forceinline__ void get8(const void* row, int c, int width, float (&v)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        float x = 0.f;
        if (c + e < width) {
            if constexpr (BF) x = __uint_as_float((uint32_t)static_cast<const uint16_t*>(row)[c + e] << 16);
            else x = static_cast<const float*>(row)[c + e];
        }
        v[e] = x;
    }
}

struct PackArgs {
    const void *X, *W, *bias;
    int64_t ldx, ldw, n;
    const int32_t* idx;           // NULL: every row counts
    Shape* shape;                 // written where every row counts
    uint16_t *x, *w;              // w NULL: read where it lies
    float* biasp;
    int64_t x_plane, w_plane;
    int32_t F, fp, C, cw, cp, terms;
    unsigned x_blocks, w_blocks;  // then one workgroup for every 256 of the bias
};

// X's rows, W and the bias as the tile products take them, a workgroup a row or 2048 columns of one
template <bool BF>
__global__ __launch_bounds__(256) void classes_pack_kernel(PackArgs a) {
    constexpr int EB = BF ? 2 : 4;
    unsigned b = blockIdx.x;
    if (b < a.x_blocks) {
        const int64_t count = a.idx ? a.shape->count : a.n;
        if (!a.idx && b == 0 && threadIdx.x == 0) a.shape->count = (int32_t)a.n;
        const int64_t rows = (count + 255) / 256 * 256;
        const int pieces = a.fp / 8;
        for (int64_t q = (int64_t)b * 256 + threadIdx.x; q < rows * pieces; q += (int64_t)a.x_blocks * 256) {
            const int64_t r = q / pieces;
            const int c = (int)(q % pieces) * 8;
            float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            if (r < count) get8<BF>(static_cast<const char*>(a.X) + (a.idx ? a.idx[r] : r) * a.ldx * EB, c, a.F, v);
            put8(v, a.terms, a.x, a.x_plane, r * a.fp + c);
        }
        return;
    }
    b -= a.x_blocks;
    if (b < a.w_blocks) {
        const int pieces = a.cw / 8;
        for (int64_t q = (int64_t)b * 256 + threadIdx.x; q < (int64_t)a.F * pieces; q += (int64_t)a.w_blocks * 256) {
            const int64_t r = q / pieces;
            const int c = (int)(q % pieces) * 8;
            float v[8];
            get8<BF>(static_cast<const char*>(a.W) + r * a.ldw * EB, c, a.C, v);
            put8(v, a.terms, a.w, a.w_plane, r * a.cw + c);
        }
        return;
    }
    b -= a.w_blocks;
    const int c = (int)(b * 256 + threadIdx.x);
    if (c >= a.cp) return;
    float v = -INFINITY;
    if (c < a.C) {
        if (!a.bias) v = 0.f;
        else if constexpr (BF) v = __uint_as_float((uint32_t)static_cast<const uint16_t*>(a.bias)[c] << 16);
        else v = static_cast<const float*>(a.bias)[c];
    }
    a.biasp[c] = v;
}

// ---- which tiles a workgroup has
// Workgroups are dealt to the eight XCDs in turn; each XCD has a contiguous range of the tiles, and in it eight row tiles by all
// column tiles after one another, so that what runs there at a time reads few rows and few columns.  A workgroup takes every so many of its XCD's
// tiles as there are workgroups for it.
struct Tiles {
    uint32_t nm, nc, per, end, id, step;
    __device__ __forceinline__ Tiles(uint32_t block, uint32_t blocks, uint32_t nm_, uint32_t nc_) : nm(nm_), nc(nc_) {
        const uint32_t total = nm * nc;
        per = (total + 7) / 8;
        end = ((block & 7) + 1) * per;
        id = (block & 7) * per + (block >> 3);
        step = blocks >> 3;
        if (end > total) end = total;
    }
    __device__ __forceinline__ bool on() const { return id < end; }
    __device__ __forceinline__ void at(int& m, int& c) const {
        const uint32_t group = id / (8 * nc), in = id - group * (8 * nc), first = group * 8;
        if (nm - first >= 8) {
            m = (int)(first + (in & 7));
            c = (int)(in >> 3);
        } else {
            const uint32_t rows = nm - first;
            c = (int)(in / rows);
            m = (int)(first + in - (uint32_t)c * rows);
        }
    }
};
// The same where every workgroup has one tile at most.
__device__ __forceinline__ bool tile_of(uint32_t block, uint32_t blocks, uint32_t nm, uint32_t nc, int& m, int& c) {
    const Tiles t(block, blocks, nm, nc);
    if (!t.on()) return false;
    t.at(m, c);
    return true;
}

__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

// The number of an accumulator's element along the first operand in its 32 x 32 block.
__device__ __forceinline__ int acc_row(int r, int lh) { return 8 * (r / 4) + 4 * lh + (r % 4); }

// ---- statistics of a row's logits, tile by tile
// The largest one times log2 e, rounded, and the sum of 2 to the logits times log2 e less that: one fused multiply-add each, whose rounding is of
// the difference.  A logit that leaves fp32's range by that factor, below -2.3e38, is as one of -infinity.
struct Parts {
    float *most, *sum, *sum_t, *picked;      // [class tiles][stats rows]; sum_t: at the temperature; picked: sum of weighted target logits
};
constexpr float kLeastExponent = -3.4028234e38f;

// (most, sum, sum_t) holds what was joined so far.
__device__ __forceinline__ void join(float& most, float& sum, float& sum_t, float m, float s, float st, float inv_t) {
    const float top = fmaxf(most, m), a = most - top, b = m - top;
    sum = sum * exp2_of(a) + s * exp2_of(b);
    sum_t = sum_t * exp2_of(a * inv_t) + st * exp2_of(b * inv_t);
    most = top;
}
// The logarithm of a sum so held, at 1 / inv_t; divided by the same rounded log2 e that the logits were multiplied by.
__device__ __forceinline__ float log_of(float most, float sum, float inv_t) {
    return (float)((double)most * (double)inv_t / (double)kLog2e + (double)logf(sum));
}

// v[0], v[step], ... n of them one after another, eight under way at a time
template <class V>
__device__ __forceinline__ V sum_of(const V* v, int64_t step, int n, V sum) {
    for (int p = 0; p < n; p += 8) {
        V part[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) part[u] = v[(p + u < n ? p + u : p) * step];
#pragma unroll
        for (int u = 0; u < 8; ++u)
            if (p + u < n) sum += part[u];
    }
    return sum;
}

inline unsigned blocks_for(int64_t items, int64_t per, int64_t most) {
    const int64_t b = (items + per - 1) / per;
    return (unsigned)(b < 1 ? 1 : (b < most ? b : most));
}

// ---- the workspace, piece after piece
struct Room {
    char* base;
    int64_t used = 0;
    template <class T>
    T* take(int64_t n) {
        T* p = reinterpret_cast<T*>(base + used);
        used += round_up(n * (int64_t)sizeof(T), 256);
        return p;
    }
};

#define GAS_TRY(expr)                       \
    do {                                    \
        const gas_status st_ = (expr);      \
        if (st_ != GAS_OK) return st_;      \
    } while (0)

// The size that a call was told may not depend on where W lies; what is laid out may.
inline gas_status check_room(const char* who, const Room& room, int64_t bytes) {
    GAS_REQUIRE(room.used <= bytes, "%s: the workspace is laid out over %lld bytes, %lld are there", who, (long long)room.used, (long long)bytes);
    return GAS_OK;
}

// The parts of the workspace that every call has, and the layer as its kernels take it.
struct Common {
    Layer layer;
    PackArgs pack;
    int32_t *idx, *pos, *block_counts;
};
inline Common lay_out(Room& room, const void* X, int64_t ldx, int64_t n, int F, const void* W, int64_t ldw, int C, const void* bias,
                      gas_dtype dt, bool compact) {
    Common c = {};
    const int planes = dt == GAS_F32 ? 3 : 1;
    const int64_t most = round_up(n, 256), fp = round_up(F, 64), cp = round_up(C, kTileC);
    // W where it lies if its rows can be read in whole pieces
    const bool in_place = dt == GAS_BF16 && C % 8 == 0 && ldw % 8 == 0 && ldw <= kMaxClasses && aligned16(W);
    // and also, by kernels of their own with one tile of rows, where it is used for no more rows than that tile has; of bf16 a copy of a few MB costs less than
    // reading W through registers. Forward / backward in us, read once and packed:
    //     fp32   9 x 512 x 100,001     75 / 306     237 / 716      bf16   9 x 512 x 100,001     51 / 161     82 / 195
    //            64 x 2,048 x 20,001   76 / 248     195 / 387             64 x 512 x 20,001     37 / 81      41 / 69
    //            64 x 512 x 2,001      30 / 72       34 / 66              64 x 2,048 x 2,001    30 / 79      31 / 56
    //            9 x 128 x 2,001       23 / 46       25 / 43              9 x 512 x 2,001       26 / 55      20 / 43
    //                                                                     9 x 64 x 64,001       16 / 37      21 / 51
    const bool small_copy = dt == GAS_BF16 && n > kRowsByVector && C <= kCopiedClasses && (int64_t)F * C <= kCopiedElements;
    const bool once = !in_place && n <= kReadOnceRows && !small_copy;
    const int64_t cw = in_place ? C : round_up(C, 64);
    c.layer.terms = dt == GAS_F32 ? 6 : 1;
    Shape* shape = room.take<Shape>(1);
    c.idx = compact ? room.take<int32_t>(most) : nullptr;
    c.pos = compact ? room.take<int32_t>(most) : nullptr;
    c.block_counts = compact ? room.take<int32_t>(most / 256) : nullptr;
    uint16_t* x = room.take<uint16_t>(planes * most * fp);
    uint16_t* w = in_place || once ? nullptr : room.take<uint16_t>(planes * (int64_t)F * cw);
    float* biasp = room.take<float>(cp);
    c.layer.x = x;
    c.layer.w = in_place ? static_cast<const uint16_t*>(W) : w;
    c.layer.raw = W;
    c.layer.ld_raw = ldw;
    c.layer.ldw = in_place ? ldw : cw;
    c.layer.w_plane = (int64_t)F * cw;
    c.layer.x_plane = most * fp;
    c.layer.bias = biasp;
    c.layer.shape = shape;
    c.layer.F = F;
    c.layer.fp = (int32_t)fp;
    c.layer.C = C;
    c.layer.cw = (int32_t)cw;
    c.layer.most = (int32_t)most;
    c.layer.stats = (int32_t)round_up(n, 16);
    c.pack = PackArgs{X, W, bias, ldx, ldw, n, c.idx, shape, x, w, biasp, c.layer.x_plane, c.layer.w_plane, F, (int32_t)fp, C, (int32_t)cw,
                      (int32_t)cp, c.layer.terms, blocks_for(most * fp / 8, 256, 4096), in_place || once ? 0u : blocks_for((int64_t)F * cw / 8, 256, 8192)};
    return c;
}

inline gas_status run_pack(const Common& c, gas_dtype dt, hipStream_t s) {
    const unsigned blocks = c.pack.x_blocks + c.pack.w_blocks + (unsigned)(c.pack.cp / 256);
    if (dt == GAS_BF16) hipLaunchKernelGGL(classes_pack_kernel<true>, dim3(blocks), dim3(256), 0, s, c.pack);
    else hipLaunchKernelGGL(classes_pack_kernel<false>, dim3(blocks), dim3(256), 0, s, c.pack);
    GAS_CHECK_HIP(hipGetLastError());
    return GAS_OK;
}

// Checks that every call makes of the layer.
inline gas_status check_layer(const char* who, const void* X, int64_t ldx, int64_t n_rows, int32_t F, const void* W, int64_t ldw, int32_t C,
                              gas_dtype dt) {
    if (!valid_dtype(dt)) return fail(GAS_ERR_DTYPE, "%s: unknown dtype %d", who, (int)dt);
    GAS_REQUIRE(n_rows >= 0 && n_rows <= kMaxRows, "%s: n_rows=%lld, at most 2^25 are taken", who, (long long)n_rows);
    GAS_REQUIRE(F > 0 && F <= kMaxWidth, "%s: F=%d, 1 to 65536 are taken", who, F);
    GAS_REQUIRE(C > 0 && C <= kMaxClasses, "%s: n_classes=%d, 1 to 4194304 are taken", who, C);
    if (n_rows == 0) return GAS_OK;
    GAS_REQUIRE(X && W, "%s: null pointer", who);
    GAS_REQUIRE(ldx >= F && ldw >= C, "%s: row stride smaller than the row", who);
    return GAS_OK;
}

// Memory that a call reads or writes, for its check that no output overlaps anything else.
struct Span {
    const void* p;
    int64_t bytes;
};
inline int64_t span(int64_t rows, int64_t ld, int64_t cols, int bytes) { return rows > 0 ? ((rows - 1) * ld + cols) * bytes : 0; }
template <int NI, int NO>
gas_status check_overlaps(const char* who, const Span (&in)[NI], const Span (&out)[NO]) {
    auto meet = [](const Span& a, const Span& b) {
        const uintptr_t p = reinterpret_cast<uintptr_t>(a.p), q = reinterpret_cast<uintptr_t>(b.p);
        return a.p && b.p && p < q + (uintptr_t)b.bytes && q < p + (uintptr_t)a.bytes;
    };
    for (int i = 0; i < NO; ++i) {
        for (const Span& o : in) GAS_REQUIRE(!meet(out[i], o), "%s: an output overlaps another matrix of the call", who);
        for (int j = 0; j < i; ++j) GAS_REQUIRE(!meet(out[i], out[j]), "%s: two outputs overlap", who);
    }
    return GAS_OK;
}

template <class Kernel>
gas_status lds_of(Kernel kernel, int bytes) {
    GAS_CHECK_HIP(hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes));
    return GAS_OK;
}

}  // namespace
}  // namespace gas
