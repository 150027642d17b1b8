// The k largest logits of an output layer over many classes, and the logarithm of the sum of all their exponentials, without its logits
// (gas_linear_top).
//
// Few rows (64), and more of so few tiles that their sums are split: all logits of them are stored, 4 bytes beside the 2 F or 4 F of W's column, and
// searched. Up to eight rows that are not better off so have a kernel of their own that reads W as it lies and multiplies by the vector units.
//
// Many rows: the classes are taken in pieces. Of the first, 4,096 classes, all logits are stored; of a later one only those above the row's k-th largest
// of the pieces before (a later class never replaces an equal earlier one), with a bit for each, and a row's list is joined with them. A piece seven
// times as wide as all before leaves about 7 k logits a row in earnest, and all of it if the logits rise with the class, which costs
// time and no more.
//
// A logit and its class make one whole number, larger for larger logits and, of equal ones, for lower classes, so the numbers of a
// row differ and any order of work finds the same k. A NaN counts as less than every number.
#include "classes_split.h"

namespace gas {
namespace {

constexpr int kMostTop = 128;
constexpr int kBuffer = 2048;                     // numbers that a workgroup holds: a row's list, and candidates
constexpr int kFirstPiece = 4096;                 // classes
constexpr int kGrowth = 7;                        // of a piece, to all before
constexpr int64_t kTopElements = 1LL << 29;       // of a piece
constexpr int kFewRows = 64;
constexpr int64_t kMostRows = 1 << 23;            // a launch of 256 threads a row

__device__ __forceinline__ uint64_t key_of(float z, int c) {
    const uint32_t b = __float_as_uint(z == 0.f ? 0.f : z);
    const uint32_t up = z != z ? 0u : (b & 0x80000000u ? ~b : b | 0x80000000u);
    return (uint64_t)up << 32 | (uint32_t)~(uint32_t)c;
}
__device__ __forceinline__ float logit_of(uint64_t key) {
    const uint32_t up = (uint32_t)(key >> 32);
    if (up == 0u) return NAN;
    return __uint_as_float(up & 0x80000000u ? up & 0x7FFFFFFFu : ~up);
}

struct SelectArgs {
    const float* z;
    const uint32_t* mask;
    uint64_t* best;               // [rows][k], the largest first
    float* floor;                 // [rows]
    int32_t first, width, k, last;
    int32_t* ids;
    float* values;
    int64_t ld_ids, ld_values;
};

// The numbers in buf[0, n) put in order, the largest first; n up to kBuffer, and room up to the next power of two
__device__ __forceinline__ void sort_down(uint64_t* buf, int n) {
    int size = 2;
    while (size < n) size *= 2;
    for (int i = n + threadIdx.x; i < size; i += 256) buf[i] = 0;
    __syncthreads();
    for (int span = 2; span <= size; span *= 2)
        for (int step = span / 2; step > 0; step /= 2) {
            for (int p = threadIdx.x; p < size / 2; p += 256) {
                const int i = (p / step) * 2 * step + p % step, j = i + step;
                const uint64_t a = buf[i], b = buf[j];
                if ((a < b) == ((i & span) == 0)) {
                    buf[i] = b;
                    buf[j] = a;
                }
            }
            __syncthreads();
        }
}

// Of the workgroup's numbers, N a thread (0: none), all that can be among the k largest, put in order in buf; how many, or -1 if there is no
// room for them. In each of the four wavefronts k / 4 threads have a largest number of at least `from`, so k numbers are no less.
template <int N>
__device__ __forceinline__ int keep_largest(const uint64_t (&key)[N], int k, uint64_t* buf, uint32_t* part, int* held) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t v = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) v = max(v, (uint32_t)(key[i] >> 32));
#pragma unroll
    for (int span = 2; span <= 64; span *= 2)             // the lanes' in order, the largest first
#pragma unroll
        for (int step = span / 2; step > 0; step /= 2) {
            const uint32_t o = (uint32_t)__shfl_xor((int)v, step);
            v = ((lane & span) == 0) == ((lane & step) == 0) ? max(v, o) : min(v, o);
        }
    v = (uint32_t)__shfl((int)v, (k + 3) / 4 - 1);
    __syncthreads();                                      // buf and part are free
    if (lane == 0) part[wave] = v;
    if (threadIdx.x == 0) *held = 0;
    __syncthreads();
    const uint32_t from = min(min(part[0], part[1]), min(part[2], part[3]));
    int mine = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) mine += key[i] != 0 && (uint32_t)(key[i] >> 32) >= from;
    int to = mine ? atomicAdd(held, mine) : 0;            // in any order: the numbers differ and are put in order below
    __syncthreads();
    const int n = *held;
    if (n > kBuffer) return -1;
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (key[i] != 0 && (uint32_t)(key[i] >> 32) >= from) buf[to++] = key[i];
    __syncthreads();
    sort_down(buf, n);
    return n;
}

// A workgroup a row: its list joined with the logits that a piece left.  8,192 rows of 131,072 classes in four pieces: 330 us, for reading a bit of
// every logit, the logits that they name and the sorting of some 450 a row and piece.
__global__ __launch_bounds__(256) void classes_select_kernel(SelectArgs a) {
    __shared__ uint64_t buf[kBuffer];
    __shared__ int part[4], held;
    const int64_t r = blockIdx.x;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const uint32_t* mask = a.mask + r * (a.width / 32);
    const float* z = a.z + r * a.width;
    int n = a.k;                                          // held in buf, the same in every thread
    uint64_t least = 0;                                   // what a number has to exceed, once the buffer was full
    bool shortened = false;
    for (int i = tid; i < a.k; i += 256) buf[i] = a.best[r * a.k + i];
    __syncthreads();
    auto shorten = [&]() {                                // buf: the k largest, in order
        if (n <= 256) {
            sort_down(buf, n);
        } else {
            uint64_t key[kBuffer / 256];
#pragma unroll
            for (int i = 0; i < kBuffer / 256; ++i) key[i] = tid + 256 * i < n ? buf[tid + 256 * i] : 0;
            n = keep_largest(key, a.k, buf, reinterpret_cast<uint32_t*>(part), &held);
        }
        if (n > a.k) n = a.k;
        least = buf[a.k - 1];                             // k are there: the first piece has more classes
        shortened = true;
        __syncthreads();
    };
    // the candidates among the threads' words, if they fit; how many they are
    auto add = [&](uint32_t word, int at) {
        uint32_t kept = word;                             // all of them exceed the list they came against
        if (shortened) {
            kept = 0;
            for (uint32_t w = word; w; w &= w - 1) {
                const int bit = __ffs((int)w) - 1, c = at * 32 + class_of_bit(bit);
                if (key_of(z[c], a.first + c) > least) kept |= 1u << bit;
            }
        }
        const int mine = __popc(kept);
        int before = mine;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int v = __shfl_up(before, o);
            if (lane >= o) before += v;
        }
        if (lane == 63) part[wave] = before;
        __syncthreads();
        int total = 0;
        for (int w = 0; w < 4; ++w) {
            if (w < wave) before += part[w];
            total += part[w];
        }
        before -= mine;
        if (n + total <= kBuffer) {
            int to = n + before;
            for (uint32_t w = kept; w; w &= w - 1) {
                const int c = at * 32 + class_of_bit(__ffs((int)w) - 1);
                buf[to++] = key_of(z[c], a.first + c);
            }
        }
        __syncthreads();
        return total;
    };
    const int words = a.width / 32;
    for (int w0 = 0; w0 < words; w0 += 256) {
        const int at = w0 + tid;
        const uint32_t word = at < words ? mask[at] : 0u;
        const int total = add(word, at);
        if (n + total <= kBuffer) {
            n += total;
            continue;
        }
        for (int part_ = 0; part_ < 8; ++part_) {         // 32 words at a time: 1,024 candidates at most
            const bool in = tid / 32 == part_;
            int t = add(in ? word : 0u, at);
            if (n + t > kBuffer) {
                shorten();
                t = add(in ? word : 0u, at);
            }
            n += t;
        }
    }
    shorten();
    for (int i = tid; i < a.k; i += 256) {
        const uint64_t key = buf[i];
        a.best[r * a.k + i] = key;
        if (a.last) {
            a.ids[r * a.ld_ids + i] = (int32_t)~(uint32_t)key;
            a.values[r * a.ld_values + i] = logit_of(key);
        }
    }
    if (tid == 0) a.floor[r] = logit_of(buf[a.k - 1]);
}

// ---- all logits of a row, or what is left of its parts, searched

struct PickArgs {
    const float* z;               // logits, class e at e, or
    const uint64_t* keys;         // numbers of the parts before (0: none)
    int64_t ld;
    int32_t n, per, parts, k;     // a part: `per` of the n, at most kPick
    uint64_t* best;               // [rows][parts][k], the largest first, 0 beyond what there is
    float* floor;                 // one part: the k-th largest, may be NULL
    int32_t* ids;                 // the last one: what the call returns, else NULL
    float* values;
    int64_t ld_ids, ld_values;
};
constexpr int kPick = 8192, kPickFew = 2048;           // numbers of a part; few of them where that leaves units without any

// A workgroup a part of a row, N numbers a thread, each read once: 32 rows of 250,000 logits 28 us (1.1 TB/s; half of it is the wavefronts' sorting), then
// 9 us for what is left. Where too many are left (equal logits), numbers go in 256 at a time.
template <bool KEYS, int N>
__global__ __launch_bounds__(256) void classes_pick_kernel(PickArgs a) {
    __shared__ uint64_t buf[kBuffer];
    __shared__ uint32_t part_[4];
    __shared__ int held;
    const int64_t row = blockIdx.x / a.parts;
    const int part = (int)(blockIdx.x % a.parts), first = part * a.per, tid = threadIdx.x;
    const int end = first + a.per < a.n ? first + a.per : a.n, there = end - first, k = a.k < there ? a.k : there;
    auto number = [&](int i) {
        const int e = first + tid + 256 * i;
        if (e >= end) return (uint64_t)0;
        if constexpr (KEYS) return a.keys[row * a.ld + e];
        else return key_of(a.z[row * a.ld + e], e);
    };
    uint64_t key[N];
#pragma unroll
    for (int i = 0; i < N; ++i) key[i] = number(i);
    int n = keep_largest(key, k, buf, part_, &held);
    if (n < 0) {
        uint64_t least = 0;
        n = 0;
        __syncthreads();
        if (tid == 0) held = 0;
        __syncthreads();
#pragma unroll 1
        for (int i = 0; i < N; ++i) {
            const uint64_t one = number(i);
            if (one > least) buf[atomicAdd(&held, 1)] = one;
            __syncthreads();
            n = held;
            if (n + 256 > kBuffer || i + 1 == N) {
                sort_down(buf, n);
                n = n < k ? n : k;
                if (n == k) least = buf[k - 1];
                __syncthreads();
                if (tid == 0) held = n;
            }
            __syncthreads();
        }
    }
    for (int i = tid; i < a.k; i += 256) {
        const uint64_t b = i < n ? buf[i] : 0;
        if (a.best) a.best[((int64_t)row * a.parts + part) * a.k + i] = b;
        if (a.ids) {
            a.ids[row * a.ld_ids + i] = (int32_t)~(uint32_t)b;
            a.values[row * a.ld_values + i] = logit_of(b);
        }
    }
    if (a.floor && tid == 0) a.floor[row] = logit_of(buf[a.k - 1]);
}

// ---- lse of every row: its tiles' statistics joined, by 256 / ROWS threads a row, in a fixed tree
template <int ROWS>
__global__ __launch_bounds__(256) void classes_lse_kernel(Parts parts, int64_t stats, int64_t n, int tiles, float* lse) {
    constexpr int PARTS = 256 / ROWS;
    __shared__ float red[2][PARTS][ROWS];
    const int row = threadIdx.x % ROWS, part = threadIdx.x / ROWS;
    const int64_t r = (int64_t)blockIdx.x * ROWS + row;
    float most = kLeastExponent, sum = 0.f, none = 0.f;
    if (r < n)
        for (int t = part; t < tiles; t += PARTS) join(most, sum, none, parts.most[t * stats + r], parts.sum[t * stats + r], 0.f, 1.f);
    for (int half = PARTS / 2; half > 0; half /= 2) {
        red[0][part][row] = most;
        red[1][part][row] = sum;
        __syncthreads();
        if (part < half) join(most, sum, none, red[0][part + half][row], red[1][part + half][row], 0.f, 1.f);
        __syncthreads();
    }
    if (part == 0 && r < n) lse[r] = log_of(most, sum, 1.f);
}

// Whether all logits are stored: of few rows, and where their sums are split. Pieces whose sums were split in different ways would leave
// equal logits with different last bits, and the higher class could come first. 100 x 1,000 x 9,000 of fp32 takes 79 us, of bf16 44; in pieces, the
// first one's sums split, 162 and 60, no sums split 235 and 66.  Pieces whose own tiles would be split and all classes' would not (100 x 2,000
// x 100,000 of fp32, 1,390 us with a split first piece) take a tenth longer.
inline bool top_whole(int64_t n, int F, int C, gas_dtype dt) { return n <= kFewRows || splits_of_few(n, F, C, dt) > 1; }
inline int64_t top_width(int64_t n, int C, bool whole) {
    const int64_t cp = round_up(C, 256);
    if (whole) return cp;
    int64_t w = kTopElements / n / 256 * 256;
    if (w < kFirstPiece) w = kFirstPiece;
    return w < cp ? w : cp;
}
inline int parts_of(int64_t n, int64_t rows) {
    const int64_t most = rows * n < 128LL * kPick ? kPickFew : kPick;
    return (int)((n + most - 1) / most);
}

struct TopRoom {
    Common common;
    Parts parts;
    float *floor, *z;
    uint32_t* mask;
    uint64_t *best, *other;
    int64_t width;
    bool whole, by_vector;
    FewRoom few;                  // parts of the sums
};
TopRoom lay_out_top(Room& room, const void* X, int64_t ldx, int64_t n, int F, const void* W, int64_t ldw, int C, const void* bias, gas_dtype dt,
                    int k) {
    TopRoom t = {};
    t.by_vector = n <= kRowsByVector && splits_of_few(n, F, C, dt) == 1;
    if (!t.by_vector) t.common = lay_out(room, X, ldx, n, F, W, ldw, C, bias, dt, false);
    else t.common.layer.most = t.common.layer.stats = kRowsByVector;
    const int64_t most = t.common.layer.most, stats = t.common.layer.stats, tiles = (C + kTileC - 1) / kTileC;
    t.whole = top_whole(n, F, C, dt);
    t.width = top_width(n, C, t.whole);
    t.parts.most = room.take<float>(tiles * stats);
    t.parts.sum = room.take<float>(tiles * stats);
    t.floor = room.take<float>(most);
    const int64_t lists = t.whole ? parts_of(C, n) : 1;
    t.best = room.take<uint64_t>(n * lists * k);
    t.other = room.take<uint64_t>(n * lists * k);
    t.z = room.take<float>(n * t.width);
    if (t.whole && !t.by_vector) t.few = lay_out_few(room, n, F, C, dt, false);
    t.few.z = t.z;
    t.mask = room.take<uint32_t>(n * (t.width / 32));
    return t;
}

int64_t top_workspace(int64_t n, int32_t F, int32_t C, gas_dtype dt, int32_t k) {
    if (n < 0 || n > kMostRows || F <= 0 || F > kMaxWidth || C <= 0 || C > kMaxClasses || k <= 0 || k > kMostTop || k > C || !valid_dtype(dt)) return -1;
    if (n == 0) return 0;
    Room room{nullptr};
    lay_out_top(room, nullptr, F, n, F, reinterpret_cast<const void*>(2), C, C, nullptr, dt, k);
    return room.used;
}

}  // namespace
}  // namespace gas

using namespace gas;

extern "C" {

int64_t gas_linear_top_workspace(int64_t n_rows, int32_t F, int32_t n_classes, gas_dtype dt, int32_t k) {
    return top_workspace(n_rows, F, n_classes, dt, k);
}

gas_status gas_linear_top(const void* X, int64_t ldx, int64_t n_rows, int32_t F, const void* W, int64_t ldw, int32_t n_classes,
                          const void* bias, gas_dtype dt, int32_t k, int32_t* ids, int64_t ld_ids, float* values, int64_t ld_values, float* lse,
                          void* workspace, int64_t workspace_bytes, void* stream) {
    const char* who = "gas_linear_top";
    gas_status st = check_layer(who, X, ldx, n_rows, F, W, ldw, n_classes, dt);
    if (st != GAS_OK) return st;
    GAS_REQUIRE(n_rows <= kMostRows, "%s: n_rows=%lld, at most 2^23 are taken", who, (long long)n_rows);
    GAS_REQUIRE(k > 0 && k <= kMostTop && k <= n_classes, "%s: k=%d of %d classes, 1 to 128 are taken", who, k, n_classes);
    if (n_rows == 0) return GAS_OK;
    GAS_REQUIRE(ids && values, "%s: null pointer", who);
    GAS_REQUIRE(ld_ids >= k && ld_values >= k, "%s: row stride smaller than the row", who);
    const int64_t need = top_workspace(n_rows, F, n_classes, dt, k);
    GAS_REQUIRE(workspace && workspace_bytes >= need, "%s: the workspace has %lld bytes, %lld are needed", who, (long long)workspace_bytes, (long long)need);
    GAS_REQUIRE(aligned16(workspace), "%s: the workspace is not 16-byte aligned", who);
    const int eb = elem_bytes(dt);
    const Span in[] = {{X, span(n_rows, ldx, F, eb)}, {W, span(F, ldw, n_classes, eb)}, {bias, (int64_t)n_classes * eb}, {workspace, workspace_bytes}};
    const Span out[] = {{ids, span(n_rows, ld_ids, k, 4)}, {values, span(n_rows, ld_values, k, 4)}, {lse, n_rows * 4}};
    st = check_overlaps(who, in, out);
    if (st != GAS_OK) return st;
    hipStream_t s = (hipStream_t)stream;
    Room room{static_cast<char*>(workspace)};
    const TopRoom t = lay_out_top(room, X, ldx, n_rows, F, W, ldw, n_classes, bias, dt, k);
    GAS_TRY(check_room(who, room, workspace_bytes));
    const int64_t cp = round_up(n_classes, 256);
    const int tiles = (int)(cp / kTileC);
    PickArgs pick = {t.z, nullptr, t.width, n_classes, n_classes, 1, k, t.best, nullptr, nullptr, nullptr, ld_ids, ld_values};
    if (t.by_vector) {
        VectorArgs v = {X, W, bias, ldx, ldw, t.width, t.common.layer.stats, nullptr, nullptr, (int32_t)n_rows, F, n_classes, 0.f, t.z, {}};
        if (lse) v.parts = t.parts;
        st = dt == GAS_BF16 ? launch_vector<true>(v, s) : launch_vector<false>(v, s);
        if (st != GAS_OK) return st;
    } else {
        st = run_pack(t.common, dt, s);
        if (st != GAS_OK) return st;
        LogitsArgs a = {};
        a.layer = t.common.layer;
        if (lse) a.parts = t.parts;
        a.inv_t = 1.f;
        a.biased = bias != nullptr;
        a.tiles = tiles;
        a.floor = t.floor;
        a.z = t.z;
        a.mask = t.mask;
        for (int64_t first = 0, width; first < cp; first += width) {
            width = t.whole ? cp : first == 0 ? kFirstPiece : kGrowth * first;
            if (width > t.width) width = t.width;
            if (first + width > cp) width = cp - first;
            a.first = (int32_t)first;
            a.width = (int32_t)width;
            a.all = first == 0;
            const int tile = rows_of_tile(n_rows, (int)width);
            if (t.few.splits > 1) {
                st = launch_split(a.layer, t.few, n_rows, s);
                if (st == GAS_OK) st = launch_join(a.layer, t.few, n_rows, 0.f, lse ? &t.parts : nullptr, s);
            } else {
                st = launch_logits<LOGITS_TOP, 1>(a, tile, (n_rows + tile - 1) / tile * (width / 256), s);
            }
            if (st != GAS_OK) return st;
            if (t.whole) break;
            const bool last = first + width >= cp;
            if (first == 0) {
                pick.ld = width;
                pick.n = pick.per = (int32_t)(width < n_classes ? width : n_classes);
                pick.floor = t.floor;
                pick.ids = last ? ids : nullptr;
                pick.values = values;
                hipLaunchKernelGGL((classes_pick_kernel<false, kFirstPiece / 256>), dim3((unsigned)n_rows), dim3(256), 0, s, pick);
            } else {
                const SelectArgs sel = {t.z, t.mask, t.best, t.floor, a.first, a.width, k, last, ids, values, ld_ids, ld_values};
                hipLaunchKernelGGL(classes_select_kernel, dim3((unsigned)n_rows), dim3(256), 0, s, sel);
            }
            GAS_CHECK_HIP(hipGetLastError());
        }
    }
    if (t.whole) {                                        // parts of 8,192, and what is left of them, until one is left
        int64_t n = n_classes;
        uint64_t *from = t.best, *to = t.best;
        for (bool keys = false;; keys = true) {
            pick.parts = parts_of(n, n_rows);
            pick.per = (int32_t)round_up((n + pick.parts - 1) / pick.parts, 256);
            pick.parts = (int)((n + pick.per - 1) / pick.per);
            pick.n = (int32_t)n;
            pick.keys = from;
            if (keys) pick.ld = n;
            pick.best = to;
            if (pick.parts == 1) {
                pick.best = nullptr;
                pick.ids = ids;
                pick.values = values;
            }
            const dim3 grid((unsigned)(n_rows * pick.parts));
            const bool few = pick.per <= kPickFew;
            if (keys && few) hipLaunchKernelGGL((classes_pick_kernel<true, kPickFew / 256>), grid, dim3(256), 0, s, pick);
            else if (keys) hipLaunchKernelGGL((classes_pick_kernel<true, kPick / 256>), grid, dim3(256), 0, s, pick);
            else if (few) hipLaunchKernelGGL((classes_pick_kernel<false, kPickFew / 256>), grid, dim3(256), 0, s, pick);
            else hipLaunchKernelGGL((classes_pick_kernel<false, kPick / 256>), grid, dim3(256), 0, s, pick);
            GAS_CHECK_HIP(hipGetLastError());
            if (pick.parts == 1) break;
            n = (int64_t)pick.parts * k;
            from = to;
            to = to == t.best ? t.other : t.best;
        }
    }
    if (lse) {
        const int64_t stats = t.common.layer.stats;
        if (n_rows <= 1024) hipLaunchKernelGGL(classes_lse_kernel<1>, dim3((unsigned)n_rows), dim3(256), 0, s, t.parts, stats, n_rows, tiles, lse);
        else hipLaunchKernelGGL(classes_lse_kernel<16>, dim3((unsigned)((n_rows + 15) / 16)), dim3(256), 0, s, t.parts, stats, n_rows, tiles, lse);
        GAS_CHECK_HIP(hipGetLastError());
    }
    return GAS_OK;
}

}  // extern "C"
