// The k largest logits of an output layer over many classes, and the logarithm of the sum of all their exponentials, without its logits
// (gas_linear_top).
//
// The classes are taken in pieces, each twice as wide as the one before. A tile stores only the logits that may still be among the k
// largest: those above the row's k-th largest of the pieces before (a later class never replaces an equal earlier one), and a bit
// for each. A row's list of k is then joined with what was stored. The first piece is stored whole; of a later one about k logits a row
// are left in earnest, and all of it if the logits rise with the class, which costs time and no more.
//
// A logit and its class make one whole number, larger for larger logits and, of equal ones, for lower classes, so the numbers of a
// row differ and any order of work finds the same k. A NaN counts as less than every number.
#include "classes_logits.h"

namespace gas {
namespace {

constexpr int kMostTop = 128;
constexpr int kBuffer = 2048;                     // numbers that a workgroup holds: a row's list, and candidates
constexpr int kFirstPiece = 4096;                 // classes
constexpr int64_t kTopElements = 1LL << 28;       // of a piece

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

// A workgroup a row: its list joined with the logits that a piece left.
__global__ __launch_bounds__(256) void classes_select_kernel(SelectArgs a) {
    __shared__ uint64_t buf[kBuffer];
    __shared__ int part[4];
    const int64_t r = blockIdx.x;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const uint32_t* mask = a.mask + r * (a.width / 32);
    const float* z = a.z + r * a.width;
    int n = 0;                                            // held in buf, the same in every thread
    uint64_t least = 0;                                   // what a number has to exceed
    if (a.first > 0) {
        for (int i = tid; i < a.k; i += 256) buf[i] = a.best[r * a.k + i];
        n = a.k;
        least = a.best[r * a.k + a.k - 1];
    }
    __syncthreads();
    auto shorten = [&]() {                                // buf: the k largest, in order
        sort_down(buf, n);
        if (n > a.k) n = a.k;
        if (n == a.k) least = buf[a.k - 1];
        __syncthreads();
    };
    // the candidates among the threads' words, if they fit; how many they are
    auto add = [&](uint32_t word, int at) {
        uint32_t kept = 0;
        for (uint32_t w = word; w; w &= w - 1) {
            const int bit = __ffs((int)w) - 1;
            if (key_of(z[at * 32 + bit], a.first + at * 32 + bit) > least) kept |= 1u << bit;
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
                const int bit = __ffs((int)w) - 1;
                buf[to++] = key_of(z[at * 32 + bit], a.first + at * 32 + bit);
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

__global__ __launch_bounds__(256) void classes_floor_kernel(float* floor, int64_t n) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i < n) floor[i] = NAN;
}

// lse of every row: its tiles' statistics joined as for the losses
__global__ __launch_bounds__(256) void classes_lse_kernel(Parts parts, int64_t most_rows, int64_t n, int tiles, float* lse) {
    __shared__ float red[2][16][17];
    const int row = threadIdx.x & 15, part = threadIdx.x >> 4;
    const int64_t r = (int64_t)blockIdx.x * 16 + row;
    float most = kLeastExponent, sum = 0.f, none = 0.f;
    if (r < n)
        for (int t = part; t < tiles; t += 16) join(most, sum, none, parts.most[t * most_rows + r], parts.sum[t * most_rows + r], 0.f, 1.f);
    red[0][part][row] = most;
    red[1][part][row] = sum;
    __syncthreads();
    if (part > 0 || r >= n) return;
    for (int p = 1; p < 16; ++p) join(most, sum, none, red[0][p][row], red[1][p][row], 0.f, 1.f);
    lse[r] = log_of(most, sum, 1.f);
}

inline int64_t top_width(int64_t most, int C) {
    const int64_t cp = round_up(C, 256);
    int64_t w = kTopElements / most / 256 * 256;
    if (w < kFirstPiece) w = kFirstPiece;
    return w < cp ? w : cp;
}

struct TopRoom {
    Common common;
    Parts parts;
    float *floor, *z;
    uint32_t* mask;
    uint64_t* best;
    int64_t width;
};
TopRoom lay_out_top(Room& room, const void* X, int64_t ldx, int64_t n, int F, const void* W, int64_t ldw, int C, const void* bias, gas_dtype dt,
                    int k) {
    TopRoom t = {};
    t.common = lay_out(room, X, ldx, n, F, W, ldw, C, bias, dt, false);
    const int64_t most = t.common.layer.most, tiles = (C + kTileC - 1) / kTileC;
    t.width = top_width(most, C);
    t.parts.most = room.take<float>(tiles * most);
    t.parts.sum = room.take<float>(tiles * most);
    t.floor = room.take<float>(most);
    t.best = room.take<uint64_t>(most * k);
    t.z = room.take<float>(n * t.width);
    t.mask = room.take<uint32_t>(n * (t.width / 32));
    return t;
}

int64_t top_workspace(int64_t n, int32_t F, int32_t C, gas_dtype dt, int32_t k) {
    if (n < 0 || n > (1 << 28) || F <= 0 || F > kMaxWidth || C <= 0 || C > kMaxClasses || k <= 0 || k > kMostTop || k > C || !valid_dtype(dt)) return -1;
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
    st = run_pack(t.common, dt, s);
    if (st != GAS_OK) return st;
    hipLaunchKernelGGL(classes_floor_kernel, dim3((unsigned)((n_rows + 255) / 256)), dim3(256), 0, s, t.floor, n_rows);
    GAS_CHECK_HIP(hipGetLastError());
    LogitsArgs a = {};
    a.layer = t.common.layer;
    if (lse) a.parts = t.parts;
    a.inv_t = 1.f;
    a.biased = bias != nullptr;
    a.tiles = (n_classes + kTileC - 1) / kTileC;
    a.floor = t.floor;
    a.z = t.z;
    a.mask = t.mask;
    const int64_t cp = round_up(n_classes, 256);
    for (int64_t first = 0, width; first < cp; first += width) {
        width = first == 0 ? kFirstPiece : 2 * a.width;
        if (width > t.width) width = t.width;
        if (first + width > cp) width = cp - first;
        a.first = (int32_t)first;
        a.width = (int32_t)width;
        st = launch_logits<LOGITS_TOP, 1>(a, n_rows, (n_rows + rows_of_tile(n_rows) - 1) / rows_of_tile(n_rows) * (width / 256), s);
        if (st != GAS_OK) return st;
        const SelectArgs sel = {t.z, t.mask, t.best, t.floor, a.first, a.width, k, first + width >= cp, ids, values, ld_ids, ld_values};
        hipLaunchKernelGGL(classes_select_kernel, dim3((unsigned)n_rows), dim3(256), 0, s, sel);
        GAS_CHECK_HIP(hipGetLastError());
    }
    if (lse) {
        hipLaunchKernelGGL(classes_lse_kernel, dim3((unsigned)((n_rows + 15) / 16)), dim3(256), 0, s, t.parts, t.common.layer.most, n_rows, a.tiles, lse);
        GAS_CHECK_HIP(hipGetLastError());
    }
    return GAS_OK;
}

}  // extern "C"
