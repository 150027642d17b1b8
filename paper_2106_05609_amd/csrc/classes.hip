// Losses of an output layer over many classes, forward and backward, without its logits: cross-entropy with labels, and
// distillation from a teacher's top logits (with labels beside them or without).
//
// A row's loss is a (lse - z_y) + b T^2 (sum_k q_k log q_k + lse_T - sum_k q_k z_k / T), its gradient at the logits
//     a exp(z - lse) + b T exp(z / T - lse_T) - w,     w_y += a, w_k += b T q_k:
// both losses are two sums of exponentials and a short list of weighted targets, so one kernel forms either from a tile of logits.
// Forward: tiles of logits leave a row's largest logit, its sums from there and its weighted target logits, which a second kernel
// joins.  Backward: a piece of the classes at a time, the gradient at its logits (formed again from the products) is stored in the
// products' type and multiplied by W and X.
//
// In bf16 that rounds it, a value by up to 2^-9: GX and GW of a distillation are 1.6e-3 off (2-norm; 4,096 x 256 x 65,536), as much as their own rounding to
// bf16 makes, of labels alone 6e-5, as most of what they sum is labels' -1.  Two parts of it would double what the products multiply, 4.3 of the 7 ms that
// 16,384 x 512 x 131,072 takes, and the 4.3 GB that are stored between.

#include "classes_split.h"

namespace gas {
namespace {

// ---- targets of the rows that count

struct RowsArgs {
    Targets t;
    int32_t *idx, *pos;
    Shape* shape;
    int64_t cap;                  // backward: room for the gradient at a piece's logits
    int32_t row_step;             // its rows are a multiple of it
    int32_t once;                 // GX by gx_once_tile
    int32_t nfx, nfw, steps_of;   // tiles of inputs of GX and GW; 64 k of one part are `steps_of` steps (of fp32's six terms)
    const float* lse;             // backward: [n] (labels alone) or [n, 2]
    const float* row_scale;       // backward: [n] or NULL
    float label_weight, temperature;
    int32_t* labels;              // [rows]: labels alone
    f32x4* info;                  // [rows]: see LogitsArgs
    float* entropy;               // [rows]: b T^2 sum q log q
    int2* entries;
    uint16_t* starts;
    int32_t k, tiles;             // k: of a row in `entries`
};

// ---- rows that count, numbered in order

// Row i has number r: what is known of it at once. Labels alone: its label and weight.
__device__ __forceinline__ void number(const RowsArgs& a, int64_t i, int r) {
    a.pos[i] = r;
    if (r < 0) return;
    a.idx[r] = (int32_t)i;
    if (!a.labels) return;
    a.labels[r] = a.t.labels[i];
    a.info[r] = f32x4{a.lse ? a.lse[i] : 0.f, 0.f, a.row_scale ? a.row_scale[i] : 1.f, 0.f};
}

// Parts of a sum whose tiles do not fill the card, each of two steps at least. A part more costs its 256 KB written and read again,
// a fifteenth of a step's time on every unit; a round of tiles on all units some four steps beside its own.
constexpr int kUnits = 256, kMostSplits = 32;
__device__ __host__ inline int splits_of(int tiles, int steps, int steps_of, int units) {
    const int candidates[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, kMostSplits};
    int best = 1;
    int64_t least = 0;
    for (int s : candidates) {
        if (s > 1 && (2 * s > steps || (int64_t)s * tiles > 2 * units)) break;
        const int64_t cost = 16LL * ((tiles * s + units - 1) / units) * ((steps + s - 1) / s * steps_of + 4) + (s > 1 ? (int64_t)s * tiles : 0);
        if (s == 1 || cost < least) {
            best = s;
            least = cost;
        }
    }
    return best;
}
// Of few rows, whose parts are short: two for every unit, of 128 classes at least.
__device__ __host__ inline int splits_once(int tiles, int steps) {
    int s = 2 * kUnits / tiles;
    if (s > steps / 2) s = steps / 2;
    return s < 1 ? 1 : s;
}
// Rows of a part of GX: gx_tile stores 32 at a time, gx_once_tile those that are there.
__device__ __host__ inline int64_t part_rows_of(int64_t rows, bool once) { return once ? rows : (rows + 31) / 32 * 32; }
__device__ __forceinline__ Shape shape_for(const RowsArgs& a, int count) {
    Shape s = {count, 0, 0, 0, 1, 1};
    if (a.cap > 0) {
        const int rows = count > 0 ? (count + 255) / 256 * 256 : 256;
        s.rows = (count + a.row_step - 1) / a.row_step * a.row_step;
        s.part_rows = part_rows_of(s.rows, a.once);
        s.width = piece_width(a.cap, s.rows > 0 ? s.rows : a.row_step, a.t.C);
        // they run beside each other: half of the units for each where both could have a round of their own together
        const int64_t tiles_x = (int64_t)rows / 256 * a.nfx, tiles_w = (int64_t)s.width / 256 * a.nfw;
        const int units = !a.once && tiles_x + tiles_w <= kUnits / 2 ? kUnits / 2 : kUnits;
        s.splits_x = a.once ? splits_once(a.nfx, s.width / kStepK) : splits_of((int)tiles_x, s.width / kStepK, a.steps_of, units);
        s.splits_w = splits_of((int)tiles_w, rows / kStepK, a.steps_of, units);
    }
    return s;
}

// Where there are few rows one workgroup does it all.
constexpr int kFewToNumber = 4096, kFewWithEntries = 1024;
__global__ __launch_bounds__(1024) void classes_number_few_kernel(RowsArgs a) {
    __shared__ int part[2][16];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int before = 0;
    for (int64_t i0 = 0, half = 0; i0 < a.t.n; i0 += 1024, half ^= 1) {
        const int64_t i = i0 + tid;
        const bool on = i < a.t.n && row_counts(a.t, i);
        const uint64_t mask = __ballot(on);
        if (lane == 0) part[half][wave] = __popcll(mask);
        __syncthreads();
        int r = before + __popcll(mask & ((1ull << lane) - 1));
        for (int w = 0; w < 16; ++w) {
            if (w < wave) r += part[half][w];
            before += part[half][w];
        }
        if (i < a.t.n) number(a, i, on ? r : -1);
    }
    if (tid == 0) *a.shape = shape_for(a, before);
}

// Else: rows that count in every 256, then their numbers.
__global__ __launch_bounds__(256) void classes_count_kernel(Targets t, int32_t* block_counts) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const bool on = i < t.n && row_counts(t, i);
    const int n = __syncthreads_count(on);
    if (threadIdx.x == 0) block_counts[blockIdx.x] = n;
}

__global__ __launch_bounds__(256) void classes_number_kernel(RowsArgs a, const int32_t* block_counts) {
    __shared__ int part[4];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int before = 0;
    for (int b = tid; b < (int)blockIdx.x; b += 256) before += block_counts[b];
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) before += __shfl_xor(before, o);
    if (lane == 0) part[wave] = before;
    __syncthreads();
    before = part[0] + part[1] + part[2] + part[3];
    __syncthreads();
    const int64_t i = (int64_t)blockIdx.x * 256 + tid;
    const bool on = i < a.t.n && row_counts(a.t, i);
    const uint64_t mask = __ballot(on);
    if (lane == 0) part[wave] = __popcll(mask);
    __syncthreads();
    int r = before + __popcll(mask & ((1ull << lane) - 1));
    for (int w = 0; w < wave; ++w) r += part[w];
    if (i < a.t.n) number(a, i, on ? r : -1);
    if (blockIdx.x + 1 == gridDim.x && tid == 0) *a.shape = shape_for(a, before + part[0] + part[1] + part[2] + part[3]);
}

// A wavefront a row (16,384 rows of 64 entries 52 us): the teacher's distribution over the entries that are there, the label among them, put in the order of their
// classes by counting how many come before each, and where each tile of classes begins in them.
__global__ __launch_bounds__(64) void classes_entries_kernel(RowsArgs a) {
    constexpr int N = (kMaxEntries + 1 + 63) / 64;
    __shared__ int32_t ids[kMaxEntries + 1], sorted[kMaxEntries + 1];
    const int64_t r = blockIdx.x;
    if (r >= a.shape->count) return;
    const int64_t i = a.idx[r];
    const int lane = threadIdx.x;
    const float inv_t = 1.f / a.temperature;
    int32_t id[N];
    float v[N];
    float most = -INFINITY;
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const int k = lane + 64 * j;
        id[j] = 0x7FFFFFFF;
        v[j] = -INFINITY;
        if (k < a.t.k) {
            const int32_t c = a.t.ids[i * a.t.ld_ids + k];
            const float x = a.t.values[i * a.t.ld_values + k];
            if (entry_counts(c, x, a.t.C)) {
                id[j] = c;
                v[j] = x * inv_t;
                most = fmaxf(most, v[j]);
            }
        }
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor(most, o));
    float total = 0.f, e[N];
#pragma unroll
    for (int j = 0; j < N; ++j) {
        e[j] = id[j] == 0x7FFFFFFF ? 0.f : expf(v[j] - most);
        total += e[j];
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) total += __shfl_xor(total, o);
    const bool some = __any(id[0] != 0x7FFFFFFF || id[1] != 0x7FFFFFFF || id[2] != 0x7FFFFFFF || id[3] != 0x7FFFFFFF || id[4] != 0x7FFFFFFF);
    const int32_t label = a.t.labels ? a.t.labels[i] : -1;
    const bool labelled = label >= 0 && label < a.t.C;
    const float scale = a.row_scale ? a.row_scale[i] : 1.f;
    const float wa = labelled ? a.label_weight * scale : 0.f;
    const float wt = some ? (a.t.labels ? 1.f - a.label_weight : 1.f) * a.temperature * scale : 0.f;
    const float log_total = logf(total);
    float entropy = 0.f;
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const float q = e[j] / total;
        if (id[j] != 0x7FFFFFFF && e[j] != 0.f) entropy = fmaf(q, v[j] - most - log_total, entropy);
        e[j] = wt * q;
        if (id[j] == 0x7FFFFFFF || e[j] == 0.f) {           // nothing is left of it: its logit may be anything
            id[j] = 0x7FFFFFFF;
            e[j] = 0.f;
        }
        const int k = lane + 64 * j;
        if (k == a.t.k && labelled && wa != 0.f) {
            id[j] = label;
            e[j] = wa;
        }
        if (k <= a.t.k) ids[k] = id[j];
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) entropy += __shfl_xor(entropy, o);
    __syncthreads();
    int there = 0;
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const int k = lane + 64 * j;
        if (k > a.t.k) continue;
        int before = 0;
        for (int o = 0; o <= a.t.k; ++o) before += ids[o] < id[j] || (ids[o] == id[j] && o < k);
        sorted[before] = id[j];
        if (before < a.k) a.entries[r * a.k + before] = int2{id[j], __float_as_int(e[j])};
        there += id[j] != 0x7FFFFFFF;
    }
    __syncthreads();
    for (int t = lane; t <= a.tiles; t += 64) {
        int from = 0, to = a.t.k + 1;
        const int64_t c = (int64_t)t * kTileC;
        while (from < to) {
            const int mid = (from + to) / 2;
            if (sorted[mid] < c) from = mid + 1;
            else to = mid;
        }
        a.starts[r * (a.tiles + 1) + t] = (uint16_t)from;
    }
    if (lane == 0) {
        f32x4 info = {0.f, 0.f, wa, wt};
        if (a.lse) {
            info[0] = a.lse[2 * i];
            info[1] = a.lse[2 * i + 1];
        }
        a.info[r] = info;
        a.entropy[r] = wt * a.temperature * entropy;
    }
}

// ---- forward: the rows' statistics joined

struct LossArgs {
    Layer layer;
    Parts parts;
    const int32_t* pos;
    const f32x4* info;            // NULL: labels alone
    const float* entropy;
    int64_t n;
    int32_t tiles, two;
    float inv_t, temperature;
    float *loss, *lse;
    // few rows, whose logits are there: where the targets are
    const float* z;
    int64_t ldz;
    const int32_t* labels;        // [rows], or
    const int2* entries;          // [rows][k]
    int32_t k;
};

// ROWS rows a workgroup, 256 / ROWS threads a row: each joins every so many tiles, then they are joined in a tree. Bound by reading 16 bytes for every 256
// logits: 8,192 x 131,072 takes 22 us
template <int ROWS>
__global__ __launch_bounds__(256) void classes_loss_kernel(LossArgs a) {
    constexpr int PARTS = 256 / ROWS;
    __shared__ float red[4][PARTS][ROWS];
    const int row = threadIdx.x % ROWS, part = threadIdx.x / ROWS;
    const int64_t i = (int64_t)blockIdx.x * ROWS + row;
    const int64_t r = i < a.n ? a.pos[i] : -1;
    float most = kLeastExponent, sum = 0.f, sum_t = 0.f, picked = 0.f;
    if (r >= 0) {
        for (int t = part; t < a.tiles; t += PARTS) {
            const int64_t at = (int64_t)t * a.layer.stats + r;
            join(most, sum, sum_t, a.parts.most[at], a.parts.sum[at], a.two ? a.parts.sum_t[at] : 0.f, a.inv_t);
            if (a.info && !a.z) picked += a.parts.picked[at];
        }
        if (a.z) {
            const float* z = a.z + r * a.ldz;
            if (!a.info) picked = part == 0 ? z[a.labels[r]] : 0.f;
            else
                for (int e = part; e < a.k; e += PARTS) {
                    const int2 one = a.entries[r * a.k + e];
                    if (one.x < a.layer.C) picked = fmaf(__int_as_float(one.y), z[one.x], picked);
                }
        }
    }
    for (int half = PARTS / 2; half > 0; half /= 2) {
        red[0][part][row] = most;
        red[1][part][row] = sum;
        red[2][part][row] = sum_t;
        red[3][part][row] = picked;
        __syncthreads();
        if (part < half) {
            join(most, sum, sum_t, red[0][part + half][row], red[1][part + half][row], red[2][part + half][row], a.inv_t);
            picked += red[3][part + half][row];
        }
        __syncthreads();
    }
    if (part > 0 || i >= a.n) return;
    const float lse = log_of(most, sum, 1.f);
    if (!a.info) {
        a.loss[i] = r < 0 ? 0.f : lse - (a.z ? picked : a.parts.picked[r]);
        a.lse[i] = r < 0 ? 0.f : lse;
        return;
    }
    float loss = 0.f, lse_t = 0.f;
    if (r >= 0) {
        const f32x4 info = a.info[r];
        lse_t = a.two ? log_of(most, sum_t, a.inv_t) : lse;
        if (info[2] != 0.f) loss = info[2] * lse;
        if (info[3] != 0.f) loss = fmaf(info[3] * a.temperature, lse_t, loss) + a.entropy[r];
        loss -= picked;
    }
    a.loss[i] = loss;
    a.lse[2 * i] = r < 0 ? 0.f : lse;
    a.lse[2 * i + 1] = lse_t;
}

// the sum of the rows' losses in a fixed order, in double
__global__ __launch_bounds__(1024) void classes_sum_kernel(const float* x, int64_t n, float* out) {
    __shared__ double part[1024];
    double s = 0.0;
    int64_t i = threadIdx.x;
    for (; i + 7 * 1024 < n; i += 8 * 1024) {
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = x[i + 1024 * j];
#pragma unroll
        for (int j = 0; j < 8; ++j) s += (double)v[j];
    }
    for (; i < n; i += 1024) s += (double)x[i];
    part[threadIdx.x] = s;
    __syncthreads();
    for (int w = 512; w > 0; w >>= 1) {
        if ((int)threadIdx.x < w) part[threadIdx.x] += part[threadIdx.x + w];
        __syncthreads();
    }
    if (threadIdx.x == 0) out[0] = (float)part[0];
}

// ---- backward: the products with the gradient at the logits

struct GradArgs {
    Layer layer;
    const uint16_t* g;
    int64_t g_plane;
    int32_t piece;
    float scale;
    float *part_x, *part_w;       // [split][rows][fp], [split][F][width]; NULL: that gradient is not asked for
    uint32_t x_blocks;            // workgroups for gx, then those for gw
    void* gw;
    int64_t ldgw;
    int32_t gw_bf16;
};

// A piece of the classes.
struct Piece {
    int rows, width, first, cols;            // the piece's first class and how many it has
    __device__ __forceinline__ Piece(const Shape& s, int piece, int C) : rows(s.rows), width(s.width) {
        const int64_t from = (int64_t)piece * s.width;
        first = (int)from;
        cols = from >= C ? 0 : (int)(C - from < s.width ? C - from : s.width);
    }
};

// gx += G W^T over a piece of the classes: lanes end up with four neighbouring inputs of one row
template <class P>
__device__ __forceinline__ void gx_tile(const GradArgs& a, uint32_t block, uint32_t blocks, char* smem) {
    constexpr int BA = P::kRowsA, BB = P::kRowsB, WA = BA / 32 / P::TA;
    const Layer& l = a.layer;
    const Shape shape = *l.shape;
    const Piece s(shape, a.piece, l.C);
    if (s.cols == 0 || s.rows == 0) return;
    const int nm = (s.rows + BB - 1) / BB, nf = (l.fp + BA - 1) / BA, steps = (s.cols + kStepK - 1) / kStepK;
    const int full = s.width / kStepK, splits = shape.splits_x;
    int ft, at;
    if (!tile_of(block, blocks, nf, nm * splits, ft, at)) return;
    const int mt = at % nm, part = at / nm;
    const int per = (full + splits - 1) / splits;
    const int first = part * per < steps ? part * per : steps, last = first + per < steps ? first + per : steps;
    const int m0 = mt * BB, f0 = ft * BA;
    const int tid = threadIdx.x, lane = tid & 63, li = lane & 31, lh = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wa0 = (wave % WA) * (32 * P::TA), wb0 = (wave / WA) * (32 * P::TB);
    f32x16 acc[P::TA][P::TB];
    P product;
    const TileOperand oa = {l.w + (int64_t)f0 * l.ldw + s.first, l.ldw, l.w_plane, l.F - 1 - f0, l.cw - s.first};
    const TileOperand ob = {a.g + (int64_t)m0 * s.width, s.width, a.g_plane, BB < s.rows - m0 ? BB - 1 : s.rows - m0 - 1, s.width};
    const int end = (s.cols + P::kStepOf - 1) / P::kStepOf, from = first * (kStepK / P::kStepOf), to = last * (kStepK / P::kStepOf);
    product.run(oa, ob, from < end ? from : end, to < end ? to : end, l.terms, reinterpret_cast<uint16_t*>(smem), wa0, wb0, acc);
    float* out = a.part_x + (int64_t)part * shape.part_rows * l.fp;
#pragma unroll
    for (int j = 0; j < P::TB; ++j) {
        if (m0 + wb0 + 32 * j >= s.rows) continue;
        float* row = out + (int64_t)(m0 + wb0 + 32 * j + li) * l.fp;
#pragma unroll
        for (int i = 0; i < P::TA; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int f = f0 + wa0 + 32 * i + 8 * q + 4 * lh;
                if (f >= l.fp) continue;
                f32x4 v = {acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
                if (a.piece > 0) v += *reinterpret_cast<const f32x4*>(row + f);
                *reinterpret_cast<f32x4*>(row + f) = v;
            }
    }
}

// The same for few rows and W as it lies
template <class P>
__device__ __forceinline__ void gx_once_tile(const GradArgs& a, uint32_t block, uint32_t blocks, char* smem) {
    constexpr int BA = P::kRowsA, WA = BA / 32 / P::TA;
    const Layer& l = a.layer;
    const Shape shape = *l.shape;
    const Piece s(shape, a.piece, l.C);
    if (s.cols == 0 || s.rows == 0) return;
    const int nf = (l.fp + BA - 1) / BA, full = s.width / P::kStepOf, steps = (s.cols + P::kStepOf - 1) / P::kStepOf, splits = shape.splits_x;
    int ft, part;
    if (!tile_of(block, blocks, nf, splits, ft, part)) return;
    const int per = (full + splits - 1) / splits, first = part * per < steps ? part * per : steps, last = first + per < steps ? first + per : steps;
    const int f0 = ft * BA, lane = threadIdx.x & 63, li = lane & 31, lh = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wa0 = (wave % WA) * (32 * P::TA), wb0 = (wave / WA) * (32 * P::TB);
    constexpr int eb = P::PLANES == 1 ? 2 : 4;
    f32x16 acc[P::TA][P::TB];
    P product;
    const typename P::Operand oa = {static_cast<const char*>(l.raw) + ((int64_t)f0 * l.ld_raw + s.first) * eb, l.ld_raw, l.F - f0, l.C - s.first};
    const TileOperand ob = {a.g, s.width, a.g_plane, s.rows - 1, s.width};
    product.run(oa, ob, shape.count, first, last, reinterpret_cast<uint16_t*>(smem), wa0, wb0, acc);
    float* out = a.part_x + (int64_t)part * shape.part_rows * l.fp;
#pragma unroll
    for (int j = 0; j < P::TB; ++j) {
        const int m = wb0 + 32 * j + li;
        if (m >= s.rows) continue;
        float* row = out + (int64_t)m * l.fp;
#pragma unroll
        for (int i = 0; i < P::TA; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int f = f0 + wa0 + 32 * i + 8 * q + 4 * lh;
                if (f >= l.fp) continue;
                f32x4 v = {acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
                if (a.piece > 0) v += *reinterpret_cast<const f32x4*>(row + f);
                *reinterpret_cast<f32x4*>(row + f) = v;
            }
    }
}
template <class P>
__global__ __launch_bounds__(P::T, 2) void classes_gx_once_kernel(GradArgs a) {
    extern __shared__ __attribute__((aligned(16))) char smem[];
    gx_once_tile<P>(a, blockIdx.x, gridDim.x, smem);
}

__device__ __forceinline__ void put4(void* base, int64_t at, const f32x4& v, int n, bool bf, bool whole) {
    if (bf) {
        uint16_t* p = static_cast<uint16_t*>(base) + at;
        if (whole) *reinterpret_cast<u32x2*>(p) = u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
        else
            for (int e = 0; e < n; ++e) p[e] = (uint16_t)f32_to_bf16(v[e]);
    } else {
        float* p = static_cast<float*>(base) + at;
        if (whole) *reinterpret_cast<f32x4*>(p) = v;
        else
            for (int e = 0; e < n; ++e) p[e] = v[e];
    }
}
// whether four elements from column 4 c of every row are aligned as one
__device__ __host__ __forceinline__ bool fours(const void* p, int64_t ld, bool bf) { return ld % 4 == 0 && (reinterpret_cast<uintptr_t>(p) & (bf ? 7 : 15)) == 0; }

// gw = X^T G of a piece of the classes, or a part of the sum over the rows: lanes end up with four neighbouring classes of one input
template <class P>
__device__ __forceinline__ void gw_tile(const GradArgs& a, uint32_t block, uint32_t blocks, char* smem) {
    constexpr int BB = P::kRowsB, WA = P::kRowsA / 32 / P::TA;
    const Layer& l = a.layer;
    const Shape shape = *l.shape;
    const Piece s(shape, a.piece, l.C);
    if (s.cols == 0) return;
    const int nc = (s.cols + 255) / 256, nf = (l.fp + BB - 1) / BB, steps = (shape.count + kStepK - 1) / kStepK;
    const int splits = shape.splits_w;
    int ft, at;
    if (!tile_of(block, blocks, nf, nc * splits, ft, at)) return;
    const int ct = at % nc, part = at / nc;
    const int per = (steps + splits - 1) / splits;
    const int first = part * per < steps ? part * per : steps, last = first + per < steps ? first + per : steps;
    const int c0 = ct * 256, f0 = ft * BB;
    const int tid = threadIdx.x, lane = tid & 63, li = lane & 31, lh = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wa0 = (wave % WA) * (32 * P::TA), wb0 = (wave / WA) * (32 * P::TB);
    f32x16 acc[P::TA][P::TB];
    P product;
    // the steps end within the rows of G that are stored
    const TileOperand oa = {a.g + c0, s.width, a.g_plane, s.width - 8 - c0, l.most};
    const TileOperand ob = {l.x + f0, l.fp, l.x_plane, l.fp - 8 - f0, l.most};
    product.run(oa, ob, first * (kStepK / P::kStepOf), last * (kStepK / P::kStepOf), l.terms, reinterpret_cast<uint16_t*>(smem), wa0, wb0, acc);
    // A lane has classes of 32 inputs' rows, memory wants a row's next to each other: through 32 rows of 64 classes of LDS that belong to the
    // wavefront (stored as they came, rows of no whole pieces took two bytes from every lane to a row of its own).
    const bool whole = fours(a.gw, a.ldgw, a.gw_bf16) && s.first + c0 + 256 <= s.first + s.cols;
    float* mine = reinterpret_cast<float*>(smem) + wave * (32 * 64);
    static_assert(P::T / 64 * 32 * 64 * 4 <= P::kLdsBytes && P::TA % 2 == 0, "the wavefronts' pieces fit where operands were");
#pragma unroll
    for (int j = 0; j < P::TB; ++j)
#pragma unroll
        for (int h = 0; h < P::TA / 2; ++h) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const f32x16& v = acc[2 * h + i][j];
                    *reinterpret_cast<f32x4*>(mine + li * 64 + 4 * ((8 * i + 2 * q + lh) ^ (li & 15))) = f32x4{v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]};
                }
            const int f_first = f0 + wb0 + 32 * j, c_first = c0 + wa0 + 64 * h;
            if (splits > 1 || whole) {                         // four classes a lane, sixteen lanes a row
                const int u = lane & 15;
#pragma unroll
                for (int r = lane >> 4; r < 32; r += 4) {
                    f32x4 v = *reinterpret_cast<const f32x4*>(mine + r * 64 + 4 * (u ^ (r & 15)));
                    const int f = f_first + r, c = c_first + 4 * u;
                    if (f >= l.F) continue;
                    if (splits > 1) *reinterpret_cast<f32x4*>(a.part_w + ((int64_t)part * l.F + f) * s.width + c) = v;
                    else put4(a.gw, (int64_t)f * a.ldgw + s.first + c, v * a.scale, 4, a.gw_bf16, true);
                }
            } else {                                           // a class a lane
                const int c = c_first + lane;
#pragma unroll 8
                for (int r = 0; r < 32; ++r) {
                    const float v = mine[r * 64 + 4 * ((lane >> 2) ^ (r & 15)) + (lane & 3)] * a.scale;
                    const int f = f_first + r;
                    if (f >= l.F || c >= s.cols) continue;
                    const int64_t at = (int64_t)f * a.ldgw + s.first + c;
                    if (a.gw_bf16) static_cast<uint16_t*>(a.gw)[at] = (uint16_t)f32_to_bf16(v);
                    else static_cast<float*>(a.gw)[at] = v;
                }
            }
        }
}

// Both in one launch: neither fills the card alone where there are few tiles, and one's last tiles run beside the other's first.  Bound by the matrix
// units: 16,384 x 512 x 131,072 of bf16 takes four launches of 1.07 ms, 1,020 TFLOP/s; fp32 is six products, 4,096 x 256 x 65,536 1.86 ms,
// 890 TFLOP/s of them.
template <class PX, class PW>
__global__ __launch_bounds__(PX::T, 2) void classes_products_kernel(GradArgs a) {
    static_assert(PX::T == PW::T, "workgroups of one size");
    extern __shared__ __attribute__((aligned(16))) char smem[];
    if (blockIdx.x < a.x_blocks) gx_tile<PX>(a, blockIdx.x, a.x_blocks, smem);
    else gw_tile<PW>(a, blockIdx.x - a.x_blocks, gridDim.x - a.x_blocks, smem);
}

// ---- backward: the gradient at logits that are there, 64 rows by 64 classes of the piece a workgroup, two classes of two rows a thread. Waits for memory:
// 100 x 1,500 logits of 16 parts take 7 us (with eight rows a thread, one part after another, 44), 1 x 200,003 6
// GROUPS of 32 threads, ROWS rows for each: 64 rows, or the eight of a call that has no more.
template <int GROUPS, int ROWS>
__global__ __launch_bounds__(32 * GROUPS) void classes_grad_few_kernel(LogitsArgs a, PartsOfZ from) {
    constexpr bool kFew = GROUPS * ROWS < 64;
    __shared__ float sums[GROUPS][64];
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    const Layer& l = a.layer;
    const int count = l.shape->count, width = l.shape->width, tid = threadIdx.x, in = (int)(blockIdx.x * 64) + 2 * (tid & 31), group = tid >> 5;
    const int64_t c = (int64_t)a.piece * width + in;
    const int r0 = (int)blockIdx.y * 64;
    if ((int)(blockIdx.x * 64) >= width || c >= from.ld || r0 >= count) return;       // whole workgroups: widths are of whole tiles
    f32x2 z[ROWS], sum = {0.f, 0.f}, bias = {0.f, 0.f};
#pragma unroll
    for (int j = 0; j < ROWS; ++j) {
        const int r = r0 + group + GROUPS * j < count ? r0 + group + GROUPS * j : count - 1;
        z[j] = sum_of(reinterpret_cast<const f32x2*>(from.p + r * from.ld + c), from.step / 2, from.splits, f32x2{0.f, 0.f});
    }
    if (from.bias) bias = *reinterpret_cast<const f32x2*>(from.bias + c);
#pragma unroll
    for (int j = 0; j < ROWS; ++j) {
        const int r = r0 + group + GROUPS * j;
        float g[2] = {0.f, 0.f};                               // zero beyond the rows that count: the sums of gw go on to 64
        if (r < count) {
            const f32x4 info = a.info[r];
            const int label = a.labels ? a.labels[r] : -1;
            int e = 0, end = 0;
            if (!a.labels) {
                const uint16_t* s = a.starts + (int64_t)r * (a.tiles + 1) + c / kTileC;
                e = s[0];
                end = s[1];
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                if (c + i >= l.C) continue;
                const float v = z[j][i] + bias[i];
                if (a.labels || info[2] != 0.f) g[i] = info[2] * exp2_of((v - info[0]) * kLog2e);
                if (!a.labels && info[3] != 0.f) g[i] = fmaf(info[3], exp2_of((v * a.inv_t - info[1]) * kLog2e), g[i]);
                if (c + i == label) g[i] -= info[2];
            }
            for (; e < end; ++e) {
                const int2 one = a.entries[(int64_t)r * a.k + e];
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    if (one.x == c + i) g[i] -= __int_as_float(one.y);
            }
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) sum[i] += g[i];
        if (kFew && r >= count) continue;                      // of few rows they end before
        uint32_t part[3];
        split_pair(g[0], g[1], part[0], part[1], part[2]);
        uint16_t* at = a.g + (int64_t)r * width + in;
        *reinterpret_cast<uint32_t*>(at) = part[0];
        if (l.terms > 1) {
            *reinterpret_cast<uint32_t*>(at + a.g_plane) = part[1];
            *reinterpret_cast<uint32_t*>(at + 2 * a.g_plane) = part[2];
        }
    }
    if (!a.gbias) return;
#pragma unroll
    for (int i = 0; i < 2; ++i) sums[group][2 * (tid & 31) + i] = sum[i];
    __syncthreads();
    if (tid >= 64) return;
    float v = 0.f;
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) v += sums[g][tid];
    a.gbias[blockIdx.y * from.ld + (int64_t)a.piece * width + blockIdx.x * 64 + tid] = v;
}

// ---- backward: gw of up to eight rows by the vector units, 1,024 classes of the piece by 16 inputs a workgroup, four classes a thread.
// Bound by writing it: 1,024 x 200,003 of fp32 takes 147 us (5.6 TB/s); as tiles of matrix products, most of whose rows are none, it took 252
template <int R>
__global__ __launch_bounds__(256) void classes_gw_few_kernel(GradArgs a) {
    typedef float f32x4_here __attribute__((ext_vector_type(4), aligned(4)));
    constexpr int kInputs = 16;
    __shared__ __attribute__((aligned(16))) float xs[kInputs][R];
    const Layer& l = a.layer;
    const Shape shape = *l.shape;
    const Piece s(shape, a.piece, l.C);
    const int planes = l.terms > 1 ? 3 : 1, f0 = (int)blockIdx.y * kInputs, fs = l.F - f0 < kInputs ? l.F - f0 : kInputs;
    // a value is the sum of its parts
    auto whole = [&](const uint16_t* p, int64_t plane) {
        float v = __uint_as_float((uint32_t)p[0] << 16);
        if (planes > 1) v += __uint_as_float((uint32_t)p[plane] << 16) + __uint_as_float((uint32_t)p[2 * plane] << 16);
        return v;
    };
    auto four = [&](const uint16_t* p) {
        const u32x2 v = *reinterpret_cast<const u32x2*>(p);
        return f32x4{bf16_lo(v[0]), bf16_hi(v[0]), bf16_lo(v[1]), bf16_hi(v[1])};
    };
    for (int i = threadIdx.x; i < fs * R; i += 256) {
        const int r = i / fs, f = i % fs;
        xs[f][r] = r < shape.count ? whole(l.x + (int64_t)r * l.fp + f0 + f, l.x_plane) * a.scale : 0.f;
    }
    __syncthreads();
    const int c = (int)(blockIdx.x * 256 + threadIdx.x) * 4, n = s.cols - c < 4 ? s.cols - c : 4;
    if (n <= 0) return;
    f32x4 g[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        g[r] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (r >= shape.count) continue;
        const uint16_t* at = a.g + (int64_t)r * s.width + c;
        g[r] = four(at);
        if (planes > 1) g[r] += four(at + a.g_plane) + four(at + 2 * a.g_plane);
    }
    const bool fours_of_bf16 = a.gw_bf16 && n == 4 && fours(a.gw, a.ldgw, true) && s.first % 4 == 0;
#pragma unroll 4
    for (int f = 0; f < fs; ++f) {
        f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = fmaf(xs[f][r], g[r][e], v[e]);
        const int64_t at = (int64_t)(f0 + f) * a.ldgw + s.first + c;
        if (!a.gw_bf16 && n == 4) *reinterpret_cast<f32x4_here*>(static_cast<float*>(a.gw) + at) = v;
        else put4(a.gw, at, v, n, a.gw_bf16, fours_of_bf16);
    }
}

// ---- backward: what came in parts, added up

struct SumArgs {
    GradArgs g;
    const int32_t* pos;
    int64_t n, ldgx;
    void* gx;
    int32_t gx_bf16;
    const float* part_b;          // [row tiles][C up to 256]
    float* gbias;
    int32_t tile_rows;            // of those row tiles
    int32_t lanes;                // a wavefront's lanes that share a sum of gx: few rows come in up to 512 parts
    uint32_t w_blocks, x_blocks;  // workgroups for gw of this piece, for gx, then one for every 256 of gbias
};

// A row of fours: row q / fours of q.  In 32 bits where that does.
__device__ __forceinline__ void row_of(int64_t q, int64_t total, int fours, int64_t& row, int& at) {
    row = total <= 0xFFFFFFFFLL ? (int64_t)((uint32_t)q / (uint32_t)fours) : q / fours;
    at = (int)(q - row * fours);
}

// gw of a piece if its sum over the rows came in parts; after the last piece gx of every row, zero for those that don't count, and gbias
__global__ __launch_bounds__(256) void classes_sums_kernel(SumArgs a) {
    const Layer& l = a.g.layer;
    const Shape shape = *l.shape;
    uint32_t block = blockIdx.x;
    if (block < a.w_blocks) {
        const Piece s(shape, a.g.piece, l.C);
        if (shape.splits_w == 1 || s.cols == 0) return;
        const int n4 = (s.cols + 3) / 4;
        const bool whole = fours(a.g.gw, a.g.ldgw, a.g.gw_bf16);
        const int64_t total = (int64_t)l.F * n4, step = (int64_t)l.F * s.width / 4;
        for (int64_t q = (int64_t)block * 256 + threadIdx.x; q < total; q += (int64_t)a.w_blocks * 256) {
            int64_t f;
            int c;
            row_of(q, total, n4, f, c);
            c *= 4;
            f32x4 v = sum_of(reinterpret_cast<const f32x4*>(a.g.part_w + f * s.width + c), step, shape.splits_w, f32x4{0.f, 0.f, 0.f, 0.f});
            v *= a.g.scale;
            put4(a.g.gw, f * a.g.ldgw + s.first + c, v, s.cols - c < 4 ? s.cols - c : 4, a.g.gw_bf16, whole && c + 4 <= s.cols);
        }
        return;
    }
    block -= a.w_blocks;
    if (block < a.x_blocks) {
        const int n4 = (l.F + 3) / 4;
        const bool whole = fours(a.gx, a.ldgx, a.gx_bf16);
        const int64_t total = a.n * n4, step = (int64_t)shape.part_rows * l.fp / 4;
        const int part = (int)threadIdx.x & (a.lanes - 1);
        for (int64_t q = ((int64_t)block * 256 + threadIdx.x) / a.lanes; q < total; q += (int64_t)a.x_blocks * 256 / a.lanes) {
            int64_t i;
            int f;
            row_of(q, total, n4, i, f);
            f *= 4;
            f32x4 v = {0.f, 0.f, 0.f, 0.f};
            const int64_t r = a.pos[i];
            if (r >= 0 && part < shape.splits_x)
                v = sum_of(reinterpret_cast<const f32x4*>(a.g.part_x + r * l.fp + f) + part * step, step * a.lanes, (shape.splits_x - 1 - part) / a.lanes + 1, v);
            for (int o = a.lanes / 2; o > 0; o >>= 1)
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] += __shfl_xor(v[e], o);
            if (part > 0) continue;
            v *= a.g.scale;
            put4(a.gx, i * a.ldgx + f, v, l.F - f < 4 ? l.F - f : 4, a.gx_bf16, whole && f + 4 <= l.F);
        }
        return;
    }
    block -= a.x_blocks;
    const int c = (int)(block * 256 + threadIdx.x);
    if (c >= l.C) return;
    const int64_t cp = ((int64_t)l.C + 255) / 256 * 256;
    a.gbias[c] = sum_of(a.part_b + c, cp, (shape.count + a.tile_rows - 1) / a.tile_rows, 0.f) * a.g.scale;
}

// ---- host

struct Call {
    const char* who;
    const void* X;
    int64_t ldx, n;
    int32_t F;
    const void* W;
    int64_t ldw;
    int32_t C;
    const void* bias;
    gas_dtype dt;
    Targets t;
    float temperature, label_weight;
    void* workspace;
    int64_t workspace_bytes;
    hipStream_t s;
};

// The workspace of the targets: RowsArgs' arrays
inline RowsArgs lay_out_rows(Room& room, const Call& c, const Common& common, bool distill) {
    RowsArgs r = {};
    const int64_t most = common.layer.most;
    r.t = c.t;
    r.idx = common.idx;
    r.pos = common.pos;
    r.shape = const_cast<Shape*>(common.layer.shape);
    r.label_weight = c.label_weight;
    r.temperature = c.temperature;
    r.tiles = (int32_t)((c.C + kTileC - 1) / kTileC);
    r.info = room.take<f32x4>(most);
    if (!distill) {
        r.labels = room.take<int32_t>(most);
    } else {
        r.k = c.t.k + 1;
        r.entropy = room.take<float>(most);
        r.entries = room.take<int2>(most * r.k);
        r.starts = room.take<uint16_t>(most * (r.tiles + 1));
    }
    return r;
}

inline gas_status run_rows(const Call& c, const Common& common, const RowsArgs& r, bool distill, bool pack) {
    const unsigned blocks = (unsigned)((c.n + 255) / 256);
    if (c.n <= (distill ? kFewWithEntries : kFewToNumber)) {
        hipLaunchKernelGGL(classes_number_few_kernel, dim3(1), dim3(1024), 0, c.s, r);
    } else {
        hipLaunchKernelGGL(classes_count_kernel, dim3(blocks), dim3(256), 0, c.s, c.t, common.block_counts);
        hipLaunchKernelGGL(classes_number_kernel, dim3(blocks), dim3(256), 0, c.s, r, common.block_counts);
    }
    GAS_CHECK_HIP(hipGetLastError());
    if (distill) {
        hipLaunchKernelGGL(classes_entries_kernel, dim3((unsigned)c.n), dim3(64), 0, c.s, r);
        GAS_CHECK_HIP(hipGetLastError());
    }
    return pack ? run_pack(common, c.dt, c.s) : GAS_OK;
}

// What the forward call needs beside: the tiles' statistics
inline Parts lay_out_parts(Room& room, const Common& common, bool distill) {
    const int64_t tiles = (common.layer.C + kTileC - 1) / kTileC, n = tiles * common.layer.stats;
    Parts p = {};
    p.most = room.take<float>(n);
    p.sum = room.take<float>(n);
    p.sum_t = distill ? room.take<float>(n) : nullptr;
    p.picked = room.take<float>(distill ? n : common.layer.most);
    return p;
}

inline LogitsArgs logits_args(const Call& c, const Common& common, const RowsArgs& r, bool distill) {
    LogitsArgs a = {};
    a.layer = common.layer;
    a.labels = distill ? nullptr : r.labels;
    a.entries = r.entries;
    a.starts = r.starts;
    a.k = r.k;
    a.tiles = r.tiles;
    a.inv_t = 1.f / c.temperature;
    a.info = r.info;
    a.biased = c.bias != nullptr;
    a.first = 0;
    a.width = r.tiles * kTileC;
    return a;
}

inline gas_status run_sum(const float* loss, int64_t n, float* out, hipStream_t s) {
    if (!out) return GAS_OK;
    hipLaunchKernelGGL(classes_sum_kernel, dim3(1), dim3(1024), 0, s, loss, n, out);
    GAS_CHECK_HIP(hipGetLastError());
    return GAS_OK;
}

// Logits of few rows, all of them
gas_status launch_few(const Call& c, const Common& common, float inv_t, float* z, const Parts* parts) {
    const VectorArgs v = {c.X, c.W, c.bias, c.ldx, c.ldw, round_up(c.C, 256), common.layer.stats, common.idx, common.layer.shape, (int32_t)c.n, c.F, c.C, inv_t, z,
                          parts ? *parts : Parts{}};
    return c.dt == GAS_BF16 ? launch_vector<true>(v, c.s) : launch_vector<false>(v, c.s);
}

gas_status forward(const Call& c, bool distill, float* loss, float* sum, float* lse) {
    Room room{static_cast<char*>(c.workspace)};
    const Common common = lay_out(room, c.X, c.ldx, c.n, c.F, c.W, c.ldw, c.C, c.bias, c.dt, true);
    const RowsArgs rows = lay_out_rows(room, c, common, distill);
    const Parts parts = lay_out_parts(room, common, distill);
    const FewRoom f = lay_out_few(room, c.n, c.F, c.C, c.dt, true);
    GAS_TRY(check_room(c.who, room, c.workspace_bytes));
    const bool few = f.by_vector;
    GAS_TRY(run_rows(c, common, rows, distill, !few));
    LogitsArgs a = logits_args(c, common, rows, distill);
    a.parts = parts;
    const bool two = distill && c.temperature != 1.f;
    const int tile = rows_of_tile(c.n, c.C);
    const int64_t tiles = (c.n + tile - 1) / tile * rows.tiles;
    if (few) GAS_TRY(launch_few(c, common, two ? a.inv_t : 0.f, f.z, &parts));
    else if (f.splits > 1) {
        GAS_TRY(launch_split(common.layer, f, c.n, c.s));
        GAS_TRY(launch_join(common.layer, f, c.n, two ? a.inv_t : 0.f, &parts, c.s));
    } else GAS_TRY((!two ? launch_logits<LOGITS_STATS, 1>(a, tile, tiles, c.s) : c.temperature == 2.f ? launch_logits<LOGITS_STATS, 4>(a, tile, tiles, c.s)
                                                                         : launch_logits<LOGITS_STATS, 3>(a, tile, tiles, c.s)));
    const LossArgs l = {common.layer, parts, common.pos, distill ? rows.info : nullptr, rows.entropy, c.n, rows.tiles, two, a.inv_t,
                        c.temperature, loss, lse, f.z, f.ld, rows.labels, rows.entries, rows.k};
    // few rows: more threads for each
    if (c.n <= 2048) hipLaunchKernelGGL(classes_loss_kernel<4>, dim3((unsigned)((c.n + 3) / 4)), dim3(256), 0, c.s, l);
    else hipLaunchKernelGGL(classes_loss_kernel<16>, dim3((unsigned)((c.n + 15) / 16)), dim3(256), 0, c.s, l);
    GAS_CHECK_HIP(hipGetLastError());
    return run_sum(loss, c.n, sum, c.s);
}

// Rows of the gradient at the logits are stored in tiles as they are formed, of up to eight one by one.
inline int row_step_of(int64_t n, int C) { return n <= kRowsByVector ? 1 : rows_of_tile(n, C); }
// Room for the gradient at the logits of a piece, in elements.
constexpr int64_t kPieceElements = 1LL << 29;
inline int64_t piece_cap(int64_t rows, int C) {
    const int64_t all = rows * round_up(C, 256), least = rows * 256;
    const int64_t cap = all < kPieceElements ? all : kPieceElements;
    return cap > least ? cap : least;
}
// Tiles of the two products by inputs: as many of them as leave few out; those of 64 and 128 take LDS more often for what they multiply.
using Gx64 = TileProduct<64, 256, 1, 4, false, false, 64, 2>;
using Gx128 = TileProduct<128, 256, 2, 4, false, false, 64, 2>;
using Gx192 = TileProduct<192, 256, 2, 4, false, false, 64, 2>;
using Gx256 = TileProduct<256, 256, 2, 4, false, false, 64, 2>;
using Gx320 = TileProduct<320, 256, 2, 4, false, false, 64, 2>;
template <bool BF> using GxOnce = ReadOnceProduct<256, 64, 4, 1, false, BF>;
using Gw64 = TileProduct<256, 64, 4, 1, true, true, 64, 2>;
using Gw128 = TileProduct<256, 128, 4, 2, true, true, 64, 2>;
using Gw192 = TileProduct<256, 192, 4, 2, true, true, 64, 2>;
using Gw256 = TileProduct<256, 256, 2, 4, true, true, 64, 2>;
using Gw320 = TileProduct<256, 320, 4, 2, true, true, 64, 2>;
inline int width_of_tile(int64_t fp) {
    const struct { int width, cost; } tiles[] = {{64, 16}, {128, 13}, {192, 11}, {256, 10}, {320, 10}};      // cost of an input, tenths
    int best = 64;
    int64_t least = 0;
    for (const auto& t : tiles) {
        const int64_t cost = (fp + t.width - 1) / t.width * t.width * t.cost;
        if (t.width == 64 || cost <= least) {
            best = t.width;
            least = cost;
        }
    }
    return best;
}

struct Grads {
    void* gx;
    int64_t ldgx;
    void* gw;
    int64_t ldgw;
    gas_dtype dt_gw;
    float* gbias;
    float scale;
    const float *lse, *row_scale;
};

struct BackwardRoom {
    uint16_t* g;
    float *gx, *gw, *gbias;
    int64_t cap;
};
inline BackwardRoom lay_out_backward(Room& room, const Common& common, int64_t n, bool gx, bool gw, bool gbias) {
    BackwardRoom b = {};
    const Layer& l = common.layer;
    const int64_t rows = round_up(n, row_step_of(n, l.C)), cp = round_up(l.C, 256);
    b.cap = piece_cap(rows, l.C);
    b.g = room.take<uint16_t>(b.cap * (l.terms > 1 ? 3 : 1));
    // The most parts that the sums of any number of rows up to n can have (splits_of, splits_once): no more than two tiles of them for a unit, and two steps
    // at least for each.  For few rows, whether W is read by gx_once_tile or lies in whole pieces, which the workspace's size is to do for.
    const int fx = width_of_tile(l.fp);
    auto least = [](int64_t a, int64_t b) { return a < b ? a : b; };
    const int64_t tiles = (l.fp + fx - 1) / fx, steps = cp / kStepK, splits = least(2 * kUnits / tiles, least(kMostSplits, steps / 2));
    int64_t parts_x = least(2 * kUnits / tiles * 256, splits * part_rows_of(rows, false));
    if (parts_x < part_rows_of(rows, false)) parts_x = part_rows_of(rows, false);
    if (n <= kReadOnceRows) {
        const int64_t parts_once = splits_once((l.fp + 255) / 256, (int)steps) * rows;
        if (parts_x < parts_once) parts_x = parts_once;
    }
    b.gx = gx ? room.take<float>(parts_x * l.fp) : nullptr;
    // of up to eight rows GW is formed as a whole
    const int64_t parts_w = n <= kRowsByVector ? 0 : least(2 * kUnits / tiles, least(kMostSplits, l.most / kStepK / 2) * (cp / 256)) * 256;
    b.gw = gw ? room.take<float>(parts_w > 0 ? parts_w * l.F : 1) : nullptr;
    b.gbias = gbias ? room.take<float>((n + rows_of_tile(n, l.C) - 1) / rows_of_tile(n, l.C) * round_up(l.C, 256)) : nullptr;
    return b;
}

template <class PX, class PW>
gas_status launch_products(GradArgs a, int64_t rows, int64_t cols, hipStream_t s) {
    constexpr int smem = PX::kLdsBytes > PW::kLdsBytes ? PX::kLdsBytes : PW::kLdsBytes;
    static_assert(smem <= 160 * 1024, "LDS of a compute unit");
    static const gas_status attr = lds_of(classes_products_kernel<PX, PW>, smem);
    if (attr != GAS_OK) return attr;
    const int64_t fp = a.layer.fp;
    auto blocks_of = [](int64_t tiles) { return (tiles < 2 * kUnits ? 2 * kUnits : tiles + 7) / 8 * 8; };
    const int64_t bx = a.part_x ? blocks_of(rows / PX::kRowsB * ((fp + PX::kRowsA - 1) / PX::kRowsA)) : 0;
    const int64_t bw = a.part_w ? blocks_of(cols / PW::kRowsA * ((fp + PW::kRowsB - 1) / PW::kRowsB)) : 0;
    GAS_REQUIRE(bx + bw <= 0x7FFFFFLL, "too many tiles for one launch");
    a.x_blocks = (uint32_t)bx;
    hipLaunchKernelGGL((classes_products_kernel<PX, PW>), dim3((unsigned)(bx + bw)), dim3(PX::T), smem, s, a);
    GAS_CHECK_HIP(hipGetLastError());
    return GAS_OK;
}

gas_status launch_gw_few(const GradArgs& a, int64_t n, int64_t cols, hipStream_t s) {
    const dim3 grid((unsigned)((cols + 1023) / 1024), (unsigned)((a.layer.F + 15) / 16)), block(256);
    if (n == 1) hipLaunchKernelGGL(classes_gw_few_kernel<1>, grid, block, 0, s, a);
    else if (n == 2) hipLaunchKernelGGL(classes_gw_few_kernel<2>, grid, block, 0, s, a);
    else if (n <= 4) hipLaunchKernelGGL(classes_gw_few_kernel<4>, grid, block, 0, s, a);
    else hipLaunchKernelGGL(classes_gw_few_kernel<8>, grid, block, 0, s, a);
    GAS_CHECK_HIP(hipGetLastError());
    return GAS_OK;
}

template <class P>
gas_status launch_gx_once(const GradArgs& a, hipStream_t s) {
    static const gas_status attr = lds_of(classes_gx_once_kernel<P>, P::kLdsBytes);
    if (attr != GAS_OK) return attr;
    const int tiles = (a.layer.fp + P::kRowsA - 1) / P::kRowsA;
    const unsigned blocks = (unsigned)round_up(tiles > 2 * kUnits ? tiles : 2 * kUnits, 8);
    hipLaunchKernelGGL(classes_gx_once_kernel<P>, dim3(blocks), dim3(P::T), P::kLdsBytes, s, a);
    GAS_CHECK_HIP(hipGetLastError());
    return GAS_OK;
}

template <int TEMPS>
gas_status launch_grad_of(const LogitsArgs& a, int n, int64_t tiles, gas_dtype dt, hipStream_t s) {
    return dt == GAS_F32 ? launch_logits<LOGITS_GRAD, TEMPS, true>(a, n, tiles, s) : launch_logits<LOGITS_GRAD, TEMPS, false>(a, n, tiles, s);
}
gas_status launch_grad(const LogitsArgs& a, int n, int64_t tiles, int temps, gas_dtype dt, hipStream_t s) {
    return temps == 1 ? launch_grad_of<1>(a, n, tiles, dt, s) : temps == 2 ? launch_grad_of<2>(a, n, tiles, dt, s)
           : temps == 3 ? launch_grad_of<3>(a, n, tiles, dt, s) : launch_grad_of<4>(a, n, tiles, dt, s);
}

gas_status backward(const Call& c, bool distill, const Grads& g) {
    Room room{static_cast<char*>(c.workspace)};
    const Common common = lay_out(room, c.X, c.ldx, c.n, c.F, c.W, c.ldw, c.C, c.bias, c.dt, true);
    RowsArgs rows = lay_out_rows(room, c, common, distill);
    const BackwardRoom b = lay_out_backward(room, common, c.n, g.gx, g.gw, g.gbias);
    rows.lse = g.lse;
    rows.row_scale = g.row_scale;
    rows.cap = b.cap;
    rows.row_step = row_step_of(c.n, c.C);
    const int fx = width_of_tile(common.layer.fp);
    rows.once = common.layer.w == nullptr;
    rows.nfw = (int32_t)((common.layer.fp + fx - 1) / fx);
    rows.nfx = rows.once ? (int32_t)((common.layer.fp + 255) / 256) : rows.nfw;
    rows.steps_of = common.layer.terms;
    const FewRoom f = lay_out_few(room, c.n, c.F, c.C, c.dt, false);
    GAS_TRY(check_room(c.who, room, c.workspace_bytes));
    PartsOfZ z = {f.parts, f.ld, f.step, f.splits, common.layer.bias};
    GAS_TRY(run_rows(c, common, rows, distill, true));
    if (f.z) {
        GAS_TRY(launch_few(c, common, 0.f, f.z, nullptr));
        z = PartsOfZ{f.z, f.ld, 0, 1, nullptr};
    } else if (f.parts) {
        GAS_TRY(launch_split(common.layer, f, c.n, c.s));
    }
    const Layer& l = common.layer;
    LogitsArgs a = logits_args(c, common, rows, distill);
    a.g = b.g;
    a.g_plane = b.cap;
    a.gbias = b.gbias;
    GradArgs d = {l, b.g, b.cap, 0, g.scale, b.gx, b.gw, 0, g.gw, g.ldgw, g.dt_gw == GAS_BF16};
    // pieces if every row counts; with fewer of them the pieces are wider and fewer, and launches beyond the last one end at once
    const int tile = rows_of_tile(c.n, c.C);
    const int least = piece_width(b.cap, round_up(c.n, rows.row_step), l.C);
    const int pieces = (c.C + least - 1) / least;
    for (int p = 0; p < pieces; ++p) {
        // the widest that piece p can be, and the most tiles that it can have: width * rows <= cap, or 256 classes
        a.piece = d.piece = p;
        const int64_t rows_most = l.most, cols_most = round_up(c.C, 256);
        const int64_t all = (c.n + tile - 1) / tile * (cols_most / 256), fit = b.cap / (tile * 256);
        if (z.p) {
            const dim3 grid((unsigned)(cols_most / 64), (unsigned)((c.n + 63) / 64));
            if (c.n <= kRowsByVector) hipLaunchKernelGGL((classes_grad_few_kernel<8, 1>), grid, dim3(256), 0, c.s, a, z);
            else hipLaunchKernelGGL((classes_grad_few_kernel<32, 2>), grid, dim3(1024), 0, c.s, a, z);
            GAS_CHECK_HIP(hipGetLastError());
        } else {
            GAS_TRY(launch_grad(a, tile, all < fit ? all : fit, !distill ? 1 : !c.t.labels ? 2 : c.temperature == 2.f ? 4 : 3, c.dt, c.s));
        }
        if (g.gx && rows.once) GAS_TRY(c.dt == GAS_BF16 ? launch_gx_once<GxOnce<true>>(d, c.s) : launch_gx_once<GxOnce<false>>(d, c.s));
        const bool gw_few = g.gw && c.n <= kRowsByVector;
        if (gw_few) GAS_TRY(launch_gw_few(d, c.n, cols_most, c.s));
        if ((g.gx && !rows.once) || (g.gw && !gw_few)) {
            const auto launch = fx == 64 ? launch_products<Gx64, Gw64> : fx == 128 ? launch_products<Gx128, Gw128> : fx == 192 ? launch_products<Gx192, Gw192>
                              : fx == 256 ? launch_products<Gx256, Gw256> : launch_products<Gx320, Gw320>;
            GradArgs both = d;
            if (rows.once) both.part_x = nullptr;
            if (gw_few) both.part_w = nullptr;
            GAS_TRY(launch(both, rows_most, cols_most, c.s));
        }
        const bool last = p + 1 == pieces;
        SumArgs sums = {d, common.pos, c.n, g.ldgx, g.gx, c.dt == GAS_BF16, b.gbias, g.gbias, tile, rows.once ? 32 : 1, 0, 0};
        if (g.gw && !gw_few) sums.w_blocks = blocks_for((int64_t)c.F * ((cols_most + 3) / 4), 256, 2048);
        if (g.gx && last) sums.x_blocks = blocks_for(c.n * ((c.F + 3) / 4), 256 / sums.lanes, 4096);
        const unsigned blocks = sums.w_blocks + sums.x_blocks + (g.gbias && last ? (unsigned)((c.C + 255) / 256) : 0u);
        if (blocks == 0) continue;
        hipLaunchKernelGGL(classes_sums_kernel, dim3(blocks), dim3(256), 0, c.s, sums);
        GAS_CHECK_HIP(hipGetLastError());
    }
    return GAS_OK;
}

__global__ __launch_bounds__(256) void classes_zero_kernel(void* p, int64_t ld, int64_t rows, int64_t cols, int bytes) {
    for (int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x; q < rows * cols; q += (int64_t)gridDim.x * 256) {
        const int64_t at = q / cols * ld + q % cols;
        if (bytes == 2) static_cast<uint16_t*>(p)[at] = 0;
        else static_cast<uint32_t*>(p)[at] = 0;
    }
}
gas_status zero(void* p, int64_t ld, int64_t rows, int64_t cols, int bytes, hipStream_t s) {
    if (!p || rows * cols == 0) return GAS_OK;
    hipLaunchKernelGGL(classes_zero_kernel, dim3(blocks_for(rows * cols, 256, 4096)), dim3(256), 0, s, p, ld, rows, cols, bytes);
    GAS_CHECK_HIP(hipGetLastError());
    return GAS_OK;
}

// bytes of a call, for the widest that its arguments allow
int64_t workspace_of(int64_t n, int32_t F, int32_t C, gas_dtype dt, int32_t k, bool bwd) {
    if (n < 0 || n > kMaxRows || F <= 0 || F > kMaxWidth || C <= 0 || C > kMaxClasses || k < 0 || k > kMaxEntries || !valid_dtype(dt)) return -1;
    if (n == 0) return 0;
    Room room{nullptr};
    Call c = {};
    c.n = n; c.C = C; c.t.k = k;
    const Common common = lay_out(room, nullptr, F, n, F, reinterpret_cast<const void*>(2), C, C, nullptr, dt, true);
    lay_out_rows(room, c, common, k > 0);
    if (bwd) lay_out_backward(room, common, n, true, true, true);
    else lay_out_parts(room, common, k > 0);
    lay_out_few(room, n, F, C, dt, !bwd);
    return room.used;
}

gas_status check_call(const Call& c, bool distill, bool bwd) {
    GAS_TRY(check_layer(c.who, c.X, c.ldx, c.n, c.F, c.W, c.ldw, c.C, c.dt));
    if (distill) {
        GAS_REQUIRE(c.t.k > 0 && c.t.k <= kMaxEntries, "%s: k=%d, 1 to 256 entries of a row are taken", c.who, c.t.k);
        GAS_REQUIRE(c.temperature > 0.f && c.temperature < INFINITY, "%s: temperature=%g", c.who, c.temperature);
        GAS_REQUIRE(c.label_weight >= 0.f && c.label_weight <= 1.f, "%s: label_weight=%g, 0 to 1 are taken", c.who, c.label_weight);
    }
    if (c.n == 0) return GAS_OK;
    if (distill) {
        GAS_REQUIRE(c.t.ids && c.t.values, "%s: null pointer", c.who);
        GAS_REQUIRE(c.t.ld_ids >= c.t.k && c.t.ld_values >= c.t.k, "%s: row stride smaller than the row", c.who);
    } else {
        GAS_REQUIRE(c.t.labels, "%s: null pointer", c.who);
    }
    const int64_t need = workspace_of(c.n, c.F, c.C, c.dt, distill ? c.t.k : 0, bwd);
    GAS_REQUIRE(c.workspace && c.workspace_bytes >= need, "%s: the workspace has %lld bytes, %lld are needed", c.who, (long long)c.workspace_bytes, (long long)need);
    GAS_REQUIRE(aligned16(c.workspace), "%s: the workspace is not 16-byte aligned", c.who);
    return GAS_OK;
}

gas_status run_forward(const Call& c, bool distill, float* loss, float* sum, float* lse) {
    GAS_TRY(check_call(c, distill, false));
    if (c.n == 0) return run_sum(loss, 0, sum, c.s);
    GAS_REQUIRE(loss && lse, "%s: null pointer", c.who);
    const int eb = elem_bytes(c.dt);
    const Span in[] = {
        {c.X, span(c.n, c.ldx, c.F, eb)}, {c.W, span(c.F, c.ldw, c.C, eb)}, {c.bias, (int64_t)c.C * eb}, {c.t.labels, c.n * 4},
        {c.t.ids, span(c.n, c.t.ld_ids, c.t.k, 4)}, {c.t.values, span(c.n, c.t.ld_values, c.t.k, 4)}, {c.workspace, c.workspace_bytes}};
    const Span out[] = {{loss, c.n * 4}, {lse, c.n * (distill ? 8 : 4)}, {sum, 4}};
    GAS_TRY(check_overlaps(c.who, in, out));
    return forward(c, distill, loss, sum, lse);
}

gas_status run_backward(const Call& c, bool distill, const Grads& g) {
    GAS_TRY(check_call(c, distill, true));
    if (!valid_dtype(g.dt_gw) || (g.dt_gw == GAS_BF16 && c.dt == GAS_F32)) return fail(GAS_ERR_DTYPE, "%s: GW is of fp32 or of W's type", c.who);
    GAS_REQUIRE(!g.gw || g.ldgw >= c.C, "%s: row stride smaller than the row", c.who);
    if (c.n == 0) {
        GAS_TRY(zero(g.gw, g.ldgw, c.F, c.C, elem_bytes(g.dt_gw), c.s));
        return zero(g.gbias, c.C, 1, c.C, 4, c.s);
    }
    GAS_REQUIRE(g.lse, "%s: null pointer", c.who);
    GAS_REQUIRE(g.gx || g.gw || g.gbias, "%s: no gradient is asked for", c.who);
    GAS_REQUIRE(!g.gx || g.ldgx >= c.F, "%s: row stride smaller than the row", c.who);
    const int eb = elem_bytes(c.dt);
    const Span in[] = {
        {c.X, span(c.n, c.ldx, c.F, eb)}, {c.W, span(c.F, c.ldw, c.C, eb)}, {c.bias, (int64_t)c.C * eb}, {c.t.labels, c.n * 4},
        {c.t.ids, span(c.n, c.t.ld_ids, c.t.k, 4)}, {c.t.values, span(c.n, c.t.ld_values, c.t.k, 4)}, {g.lse, c.n * (distill ? 8 : 4)},
        {g.row_scale, c.n * 4}, {c.workspace, c.workspace_bytes}};
    const Span out[] = {{g.gx, span(c.n, g.ldgx, c.F, eb)}, {g.gw, span(c.F, g.ldgw, c.C, elem_bytes(g.dt_gw))}, {g.gbias, (int64_t)c.C * 4}};
    GAS_TRY(check_overlaps(c.who, in, out));
    return backward(c, distill, g);
}

}  // namespace
}  // namespace gas

using namespace gas;

extern "C" {

int64_t gas_linear_xent_workspace(int64_t n_rows, int32_t F, int32_t n_classes, gas_dtype dt) { return workspace_of(n_rows, F, n_classes, dt, 0, false); }
int64_t gas_linear_xent_bwd_workspace(int64_t n_rows, int32_t F, int32_t n_classes, gas_dtype dt) { return workspace_of(n_rows, F, n_classes, dt, 0, true); }
int64_t gas_linear_distill_workspace(int64_t n_rows, int32_t F, int32_t n_classes, gas_dtype dt, int32_t k) {
    return k > 0 ? workspace_of(n_rows, F, n_classes, dt, k, false) : -1;
}
int64_t gas_linear_distill_bwd_workspace(int64_t n_rows, int32_t F, int32_t n_classes, gas_dtype dt, int32_t k) {
    return k > 0 ? workspace_of(n_rows, F, n_classes, dt, k, true) : -1;
}

gas_status gas_linear_xent(const void* X, int64_t ldx, int64_t n_rows, int32_t F, const void* W, int64_t ldw, int32_t n_classes,
                           const void* bias, gas_dtype dt, const int32_t* labels, float* loss_rows, float* loss_sum, float* lse,
                           void* workspace, int64_t workspace_bytes, void* stream) {
    const Call c = {"gas_linear_xent", X, ldx, n_rows, F, W, ldw, n_classes, bias, dt, {labels, nullptr, nullptr, 0, 0, n_rows, 0, n_classes}, 1.f, 1.f,
                    workspace, workspace_bytes, (hipStream_t)stream};
    return run_forward(c, false, loss_rows, loss_sum, lse);
}

gas_status gas_linear_xent_bwd(const void* X, int64_t ldx, int64_t n_rows, int32_t F, const void* W, int64_t ldw, int32_t n_classes,
                               const void* bias, gas_dtype dt, const int32_t* labels, const float* lse, float scale,
                               const float* row_scale, void* GX, int64_t ldgx, void* GW, int64_t ldgw, gas_dtype dt_gw, float* gbias,
                               void* workspace, int64_t workspace_bytes, void* stream) {
    const Call c = {"gas_linear_xent_bwd", X, ldx, n_rows, F, W, ldw, n_classes, bias, dt, {labels, nullptr, nullptr, 0, 0, n_rows, 0, n_classes}, 1.f, 1.f,
                    workspace, workspace_bytes, (hipStream_t)stream};
    return run_backward(c, false, Grads{GX, ldgx, GW, ldgw, dt_gw, gbias, scale, lse, row_scale});
}

gas_status gas_linear_distill(const void* X, int64_t ldx, int64_t n_rows, int32_t F, const void* W, int64_t ldw, int32_t n_classes,
                              const void* bias, gas_dtype dt, const int32_t* ids, int64_t ld_ids, const float* values, int64_t ld_values, int32_t k,
                              float temperature, const int32_t* labels, float label_weight, float* loss_rows, float* loss_sum,
                              float* lse, void* workspace, int64_t workspace_bytes, void* stream) {
    const Call c = {"gas_linear_distill", X, ldx, n_rows, F, W, ldw, n_classes, bias, dt, {labels, ids, values, ld_ids, ld_values, n_rows, k, n_classes},
                    temperature, label_weight, workspace, workspace_bytes, (hipStream_t)stream};
    return run_forward(c, true, loss_rows, loss_sum, lse);
}

gas_status gas_linear_distill_bwd(const void* X, int64_t ldx, int64_t n_rows, int32_t F, const void* W, int64_t ldw, int32_t n_classes,
                                  const void* bias, gas_dtype dt, const int32_t* ids, int64_t ld_ids, const float* values, int64_t ld_values, int32_t k,
                                  float temperature, const int32_t* labels, float label_weight, const float* lse, float scale,
                                  const float* row_scale, void* GX, int64_t ldgx, void* GW, int64_t ldgw, gas_dtype dt_gw, float* gbias,
                                  void* workspace, int64_t workspace_bytes, void* stream) {
    const Call c = {"gas_linear_distill_bwd", X, ldx, n_rows, F, W, ldw, n_classes, bias, dt, {labels, ids, values, ld_ids, ld_values, n_rows, k, n_classes},
                    temperature, label_weight, workspace, workspace_bytes, (hipStream_t)stream};
    return run_backward(c, true, Grads{GX, ldgx, GW, ldgw, dt_gw, gbias, scale, lse, row_scale});
}

}  // extern "C"
