// The step of a model with many tensors: the squared norm of all gradients, and AdamW with states in 32 bits or in 8.
//     g = c dW,  m <- b1 m + (1 - b1) g,  v <- b2 v + (1 - b2) g^2,
//     W <- W - lr wd W - lr (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps)
// Bound by memory, small models by the launches.
#include <algorithm>

#include "common.h"

namespace gas {
namespace {

constexpr int kBlock = 256;                         // elements that share a scale: four for every lane
constexpr int kNormChunk = 32768;                   // elements of a partial sum
// Tensors of a launch: their descriptions fit the 4 KB of a launch's arguments.  Models of few tensors have a launch with room for no more: it is
// copied for every call.
constexpr int kNormTensors = 256, kTensors = 144, kFew = 16;

// Index of the tensor that unit `u` (a block, a chunk) belongs to: the last one whose first unit is not behind it.  The lanes look at 64 at a
// time, so it takes one reading, not one after another.
template <int N>
__device__ __forceinline__ int tensor_of(const uint32_t (&first)[N], int count, uint32_t u) {
    const int lane = threadIdx.x & 63;
    int before = 0;
#pragma unroll
    for (int i = 0; i < (N + 63) / 64; ++i) {
        const int k = i * 64 + lane;
        before += __popcll(__ballot(k < count && first[k < count ? k : 0] <= u));
    }
    return __builtin_amdgcn_readfirstlane(before - 1);
}

// Four elements of any alignment.
typedef f32x4 four_f32 __attribute__((aligned(4)));
typedef u32x2 four_bf16 __attribute__((aligned(2)));

// ---- the squared norm of many tensors
template <int N>
struct NormBatch {
    const float* x[N];
    uint32_t first[N];                              // chunk that the tensor begins with
    uint16_t last[N];                               // elements of its last chunk
    int count;
    uint32_t chunks;
    double* partials;
};

__device__ __forceinline__ double wave_sum64(double v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    return v;
}

// A workgroup to a chunk; sums in 64 bits, for which a product of two floats is exact.  154 M: 89 us, 6.9 TB/s of the 7.1 that reading alone reaches.
template <int N>
__global__ __launch_bounds__(256) void sq_norms_kernel(NormBatch<N> b) {
    __shared__ double part[4];
    const int k = tensor_of(b.first, b.count, blockIdx.x);
    const float* x = b.x[k] + (int64_t)(blockIdx.x - b.first[k]) * kNormChunk;
    const bool whole = blockIdx.x + 1 < (k + 1 < b.count ? b.first[k + 1] : b.chunks);
    const int n = whole ? kNormChunk : b.last[k];
    double s[4] = {0.0, 0.0, 0.0, 0.0};
    int i = 4 * threadIdx.x;
    for (; i + 7 * 1024 + 4 <= n; i += 8 * 1024) {
        f32x4 v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = __builtin_nontemporal_load(reinterpret_cast<const four_f32*>(x + i + 1024 * j));
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[e] = fma((double)v[j][e], (double)v[j][e], s[e]);
    }
    for (; i < n; i += 1024)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const double v = i + e < n ? (double)x[i + e] : 0.0;
            s[e] = fma(v, v, s[e]);
        }
    const double sum = wave_sum64((s[0] + s[1]) + (s[2] + s[3]));
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) b.partials[blockIdx.x] = (part[0] + part[1]) + (part[2] + part[3]);
}

__global__ __launch_bounds__(1024) void sq_norms_finish_kernel(const double* partials, int64_t n, float* out, int32_t* steps) {
    __shared__ double part[16];
    double s[4] = {0.0, 0.0, 0.0, 0.0};
    int64_t i = threadIdx.x;
    for (; i + 3 * 1024 < n; i += 4 * 1024)
#pragma unroll
        for (int j = 0; j < 4; ++j) s[j] += partials[i + 1024 * j];
    for (; i < n; i += 1024) s[0] += partials[i];
    const double sum = wave_sum64((s[0] + s[1]) + (s[2] + s[3]));
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        double all = 0.0;
#pragma unroll
        for (int w = 0; w < 16; ++w) all += part[w];
        const float total = (float)all;
        out[0] = total;
        if (steps && total < INFINITY) ++*steps;    // neither an infinity nor a NaN
    }
}

// ---- AdamW
// From here on every product and sum rounds by itself, but where fmaf is written: states and codes do not depend on what a compiler fuses
// (the _rn intrinsics do not say that: here they are the operators).
#pragma clang fp contract(off)

template <int N>
struct AdamTensors {
    char* W[N];
    const float* g[N];
    uint32_t first[N];                              // block that the tensor begins with, counted from `base`
    float decay[N];                                 // lr times the weight decay
    uint16_t last[N];                               // elements of its last block; kHalf: bf16
    int count;
};
struct AdamStep {
    uint32_t blocks;
    int64_t base;                                   // the launch's first block
    void *m, *v;
    float *scales, *master;
    float b1, b2, rate1, rate2, eps;
    float lr, c1, c2;                               // 1 / (1 - b1^t), 1 / sqrt(1 - b2^t)
    float ln1, ln2;                                 // logarithms of b1, b2, for a step that is read on the device
    uint32_t step;
    const int32_t* steps;
    const float* sq_norm;
    float max_norm;
};
constexpr uint16_t kHalf = 0x8000;

// Two numbers of 16 bits from an element's place in the state and the step: multiplied and folded until every bit of both
// has reached all others.  Shifts and multipliers of the folding are those of C. Wellons' published search for 32-bit mixing functions of low bias (2018); the place's
// high half comes in by a multiplier of A. Appleby's published 32-bit hash finalizer, the step by 2^32 over the golden ratio.
__device__ __forceinline__ uint32_t dice(int64_t place, uint32_t step) {
    uint32_t x = (uint32_t)place + (uint32_t)(place >> 32) * 0x85EBCA6Bu;
    x ^= step * 0x9E3779B9u;
    x = (x ^ (x >> 16)) * 0x7FEB352Du;
    x = (x ^ (x >> 15)) * 0x846CA68Bu;
    return x ^ (x >> 16);
}

// What codes stand for: m = s k |k| / 127^2, v = s (k / 255)^4.  A root of the value is what is cut into equal parts, so small
// ones keep more digits: the smallest m is 1 / 16,129 of the block's largest, the smallest sqrt(v) 1 / 65,025.
__device__ __forceinline__ float decode_m(int k, float s) { return s * ((float)(k * (k < 0 ? -k : k)) * (1.f / 16129.f)); }
__device__ __forceinline__ float decode_v(int k, float s) {
    const float t = (float)(k * k) * (1.f / 65025.f);
    return s * t * t;
}

// x in parts of 1 / TOP^POWER of the block's largest to a code: one of the two next to it, at random so that the expectation of what
// the code stands for is x.  Rounded to nearest a state would stand still: v loses 0.1% a step, a code is 1.6% at least.  The
// root needs no care: at a square either side of it leaves the same code.
template <int POWER, int TOP>
__device__ __forceinline__ int encode(float x, uint32_t die) {
    float r = __builtin_amdgcn_sqrtf(x);
    if constexpr (POWER == 4) r = __builtin_amdgcn_sqrtf(r);
    const float k = fminf(floorf(r), (float)(TOP - 1));
    float lower = k * k, upper = (k + 1.f) * (k + 1.f);
    if constexpr (POWER == 4) { lower *= lower; upper *= upper; }
    return (int)k + (((float)die + 0.5f) * (1.f / 65536.f) * (upper - lower) < x - lower ? 1 : 0);
}

// The largest magnitude of the wavefront's values, by their bits: a NaN is larger than all.  By data-parallel moves within 16 lanes and swaps
// beyond: through LDS the two of a block took 12 steps of some 60 cycles.
__device__ __forceinline__ float largest(const f32x4& x) {
    uint32_t u = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) u = max(u, __float_as_uint(fabsf(x[i])));
    u = max(u, (uint32_t)__builtin_amdgcn_mov_dpp(u, 0xB1, 0xf, 0xf, true));           // quad_perm 1 0 3 2
    u = max(u, (uint32_t)__builtin_amdgcn_mov_dpp(u, 0x4E, 0xf, 0xf, true));           // quad_perm 2 3 0 1
    u = max(u, (uint32_t)__builtin_amdgcn_mov_dpp(u, 0x141, 0xf, 0xf, true));          // row_half_mirror
    u = max(u, (uint32_t)__builtin_amdgcn_mov_dpp(u, 0x140, 0xf, 0xf, true));          // row_mirror
    const auto s = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    u = max(s[0], s[1]);
    const auto t = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return __uint_as_float(max(t[0], t[1]));
}

// A wavefront takes one block.  What it loads waits for nothing that it can do without: the clipping factor comes last.  32 bits: 28 bytes an
// element and some 35 operations: 311 to 340 us for 70 M, 5.8 to 6.3 TB/s, near a copy.  8 bits: 16 (float weights) and some 115, half of them the rounding: 154 M
// bf16 weights with masters, 18 bytes each, 483 to 548 us, 5.1 to 5.7 TB/s, bound by issuing them (2% faster when the compiler may fuse).  Two or four
// blocks to a wavefront (measured while it might): 8 bits, 270,000 elements 17 us, 19 and 25, 16 M 78, 80 and 86, 154 M with their unpacking 665, 651 and 654; 32 bits,
// 154 M 715, 759 and 756.  Roots and quotients are the instructions' own, to one unit in the last place.
template <bool EIGHT, int N>
__global__ __launch_bounds__(256) void adamw_kernel(AdamTensors<N> l, AdamStep b) {
    const int lane = threadIdx.x & 63;
    const uint32_t unit = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (unit >= b.blocks) return;
    const float total = b.sq_norm ? *b.sq_norm : 0.f;
    uint32_t step = b.steps ? (uint32_t)*b.steps : b.step;
    const int k = tensor_of(l.first, l.count, unit);
    const uint32_t next = k + 1 < l.count ? l.first[k + 1] : b.blocks;
    const int64_t e = (int64_t)(unit - l.first[k]) * kBlock + 4 * lane, at = (b.base + unit) * kBlock + 4 * lane;
    const bool half = l.last[k] & kHalf, own = half && b.master;
    const int there = unit + 1 < next ? 4 : (int)(l.last[k] & ~kHalf) - 4 * lane;       // of the lane's four elements
    const uint16_t* w16 = reinterpret_cast<const uint16_t*>(l.W[k]) + e;
    const float* w32 = own ? b.master + at : reinterpret_cast<const float*>(l.W[k]) + e;
    f32x4 g = {0.f, 0.f, 0.f, 0.f}, w = g, m, v;
    uint32_t km, kv;
    f32x2_t scale;
    if (there >= 4) {
        g = __builtin_nontemporal_load(reinterpret_cast<const four_f32*>(l.g[k] + e));
        if (half && !own) {
            const u32x2 x = __builtin_nontemporal_load(reinterpret_cast<const four_bf16*>(w16));
            w = f32x4{bf16_lo(x[0]), bf16_hi(x[0]), bf16_lo(x[1]), bf16_hi(x[1])};
        } else {
            w = __builtin_nontemporal_load(reinterpret_cast<const four_f32*>(w32));
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < there) {
                g[i] = l.g[k][e + i];
                w[i] = half && !own ? __uint_as_float((uint32_t)w16[i] << 16) : w32[i];
            }
    }
    if constexpr (EIGHT) {
        km = __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(reinterpret_cast<const int8_t*>(b.m) + at));
        kv = __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(reinterpret_cast<const uint8_t*>(b.v) + at));
        scale = *reinterpret_cast<const f32x2_t*>(b.scales + 2 * (b.base + unit));
    } else {
        m = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(reinterpret_cast<const float*>(b.m) + at));
        v = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(reinterpret_cast<const float*>(b.v) + at));
    }
    if (!(total < INFINITY)) return;                // the whole call alike
    float c = 1.f, c1 = b.c1, c2 = b.c2;
    if (b.sq_norm) c = fminf(1.f, (float)((double)b.max_norm / (sqrt((double)total) + 1e-6)));
    if (b.steps) {
        c1 = 1.f / -expm1f((float)step * b.ln1);
        c2 = 1.f / sqrtf(-expm1f((float)step * b.ln2));
    }
    if constexpr (EIGHT) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            m[i] = decode_m((int8_t)(km >> (8 * i)), scale[0]);
            v[i] = decode_v((kv >> (8 * i)) & 255u, scale[1]);
        }
    }
    const float decay = l.decay[k], rate = b.lr * c1;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float gi = c * g[i];
        m[i] = m[i] * b.b1 + gi * b.rate1;
        v[i] = v[i] * b.b2 + gi * gi * b.rate2;
        const float change = m[i] * rate * __builtin_amdgcn_rcpf(fmaf(__builtin_amdgcn_sqrtf(v[i]), c2, b.eps));
        w[i] -= fmaf(w[i], decay, change);
    }
    const u32x2 low = {pack_bf16(w[0], w[1]), pack_bf16(w[2], w[3])};
    char* W = l.W[k] + e * (half ? 2 : 4);
    if (own) __builtin_nontemporal_store(w, reinterpret_cast<f32x4*>(b.master + at));
    if (there >= 4) {
        if (half) __builtin_nontemporal_store(low, reinterpret_cast<four_bf16*>(W));
        else __builtin_nontemporal_store(w, reinterpret_cast<four_f32*>(W));
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < there) {
                if (half) reinterpret_cast<uint16_t*>(W)[i] = (uint16_t)(low[i >> 1] >> (16 * (i & 1)));
                else reinterpret_cast<float*>(W)[i] = w[i];
            }
    }
    if constexpr (EIGHT) {
        float sm = largest(m), sv = largest(v);
        // A block with an infinity or a NaN is lost and reads as NaN, all of it: beside an infinite scale no element would move any more, without a word.
        // Below the normal numbers: nothing.
        sm = sm < INFINITY ? (sm < 1.17549435e-38f ? 0.f : sm) : NAN;
        sv = sv < INFINITY ? (sv < 1.17549435e-38f ? 0.f : sv) : NAN;
        const float im = sm > 0.f ? 1.f / sm : 0.f, iv = sv > 0.f ? 1.f / sv : 0.f;
        if (lane == 0) *reinterpret_cast<f32x2_t*>(b.scales + 2 * (b.base + unit)) = f32x2_t{sm, sv};
        km = kv = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t die = dice(at + i, step);
            const int x = encode<2, 127>(fabsf(m[i]) * im * 16129.f, die & 0xFFFFu);
            int z = encode<4, 255>(v[i] * iv * 4228250625.f, die >> 16);
            if (z == 0 && v[i] > 0.f && sv > 0.f) z = 1;        // a denominator never becomes nothing
            km |= (uint32_t)((m[i] < 0.f ? -x : x) & 255) << (8 * i);
            kv |= (uint32_t)z << (8 * i);
        }
        __builtin_nontemporal_store(km, reinterpret_cast<uint32_t*>(reinterpret_cast<int8_t*>(b.m) + at));
        __builtin_nontemporal_store(kv, reinterpret_cast<uint32_t*>(reinterpret_cast<uint8_t*>(b.v) + at));
    } else {
        __builtin_nontemporal_store(m, reinterpret_cast<f32x4*>(reinterpret_cast<float*>(b.m) + at));
        __builtin_nontemporal_store(v, reinterpret_cast<f32x4*>(reinterpret_cast<float*>(b.v) + at));
    }
}

// A wavefront takes four blocks; every instruction stores one stretch of memory (sixteen elements a lane, so that a lane's stores lie next to each
// other and an instruction's do not: 154 M elements to bf16 900 us, so 147, 6.3 TB/s).
template <bool BF>
__global__ __launch_bounds__(256) void adamw_unpack_kernel(const int8_t* m, const uint8_t* v, const float* scales, int64_t blocks, char* m_out, char* v_out) {
    const int lane = threadIdx.x & 63;
    const int64_t unit = ((int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6)) * 4;
    uint32_t km[4], kv[4];
    f32x2_t s[4];
#pragma unroll
    for (int r = 0; r < 4; ++r)
        if (unit + r < blocks) {
            km[r] = __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(m) + (unit + r) * 64 + lane);
            kv[r] = __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(v) + (unit + r) * 64 + lane);
            s[r] = reinterpret_cast<const f32x2_t*>(scales)[unit + r];
        }
#pragma unroll
    for (int r = 0; r < 4; ++r)
        if (unit + r < blocks) {
            f32x4 a, b;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                a[e] = decode_m((int8_t)(km[r] >> (8 * e)), s[r][0]);
                b[e] = decode_v((kv[r] >> (8 * e)) & 255u, s[r][1]);
            }
            const int64_t to = (unit + r) * 64 + lane;
            if constexpr (BF) {
                __builtin_nontemporal_store(u32x2{pack_bf16(a[0], a[1]), pack_bf16(a[2], a[3])}, reinterpret_cast<u32x2*>(m_out) + to);
                __builtin_nontemporal_store(u32x2{pack_bf16(b[0], b[1]), pack_bf16(b[2], b[3])}, reinterpret_cast<u32x2*>(v_out) + to);
            } else {
                __builtin_nontemporal_store(a, reinterpret_cast<f32x4*>(m_out) + to);
                __builtin_nontemporal_store(b, reinterpret_cast<f32x4*>(v_out) + to);
            }
        }
}

// Workgroups of 256 threads: a launch has less than 2^32 threads (beyond them the grid wraps, without an error).
constexpr int64_t kMostGroups = 0xFFFFFFFFLL / 256, kMostBlocks = 4 * kMostGroups;

// Stretches of memory that are apart from each other, in order.
struct Stretches {
    uintptr_t from[kTensors], to[kTensors];
    int count = 0;
    bool add(uintptr_t a, uintptr_t b) {                     // false, and nothing is added, if it meets one that is there
        int i = count;
        while (i > 0 && from[i - 1] >= b) --i;               // most lists are in the order of their addresses already
        if (i > 0 && to[i - 1] > a) return false;
        for (int j = count; j > i; --j) from[j] = from[j - 1], to[j] = to[j - 1];
        from[i] = a; to[i] = b;
        ++count;
        return true;
    }
};

}  // namespace
}  // namespace gas

using namespace gas;

extern "C" {

int64_t gas_sq_norms_workspace(int32_t count, const int64_t* n) {
    int64_t chunks = 0;
    for (int32_t i = 0; n && i < count; ++i)
        if (n[i] > 0) chunks += (n[i] + kNormChunk - 1) / kNormChunk;
    return 8 * chunks;
}

gas_status gas_sq_norms(int32_t count, const float* const* x, const int64_t* n, float* out, int32_t* steps, void* workspace,
                        int64_t workspace_bytes, void* stream) {
    const char* who = "gas_sq_norms";
    GAS_REQUIRE(count >= 0 && (count == 0 || (x && n)), "%s: count=%d", who, count);
    GAS_REQUIRE(out, "%s: null output", who);
    for (int32_t i = 0; i < count; ++i) GAS_REQUIRE(n[i] >= 0 && (n[i] == 0 || x[i]), "%s: tensor %d", who, i);
    const int64_t need = gas_sq_norms_workspace(count, n);
    GAS_REQUIRE(need == 0 || (workspace && workspace_bytes >= need && ((uintptr_t)workspace & 7u) == 0),
                "%s: the workspace has %lld bytes, %lld are needed, from a multiple of 8 on", who, (long long)workspace_bytes, (long long)need);
    GAS_REQUIRE(need / 8 <= kMostGroups, "%s: too many elements", who);
    double* partials = static_cast<double*>(workspace);
    int64_t done = 0;
    for (int32_t i = 0; i < count;) {
        NormBatch<kNormTensors> b;
        b.count = 0;
        b.partials = partials + done;
        int64_t chunks = 0;
        for (; i < count && b.count < kNormTensors; ++i) {
            if (n[i] == 0) continue;
            const int64_t more = (n[i] + kNormChunk - 1) / kNormChunk;
            b.x[b.count] = x[i]; b.first[b.count] = (uint32_t)chunks; b.last[b.count] = (uint16_t)(n[i] - (more - 1) * kNormChunk);
            ++b.count;
            chunks += more;
        }
        if (chunks == 0) continue;
        b.chunks = (uint32_t)chunks;
        if (b.count <= kFew) {
            NormBatch<kFew> few;
            std::copy_n(b.x, b.count, few.x);
            std::copy_n(b.first, b.count, few.first);
            std::copy_n(b.last, b.count, few.last);
            few.count = b.count; few.chunks = b.chunks; few.partials = b.partials;
            hipLaunchKernelGGL(sq_norms_kernel<kFew>, dim3(b.chunks), dim3(256), 0, (hipStream_t)stream, few);
        } else {
            hipLaunchKernelGGL(sq_norms_kernel<kNormTensors>, dim3(b.chunks), dim3(256), 0, (hipStream_t)stream, b);
        }
        GAS_CHECK_HIP(hipGetLastError());
        done += chunks;
    }
    hipLaunchKernelGGL(sq_norms_finish_kernel, dim3(1), dim3(1024), 0, (hipStream_t)stream, partials, done, out, steps);
    GAS_CHECK_HIP(hipGetLastError());
    return GAS_OK;
}

int64_t gas_adamw_elements(int32_t count, const int64_t* n) {
    int64_t blocks = 0;
    for (int32_t i = 0; n && i < count; ++i)
        if (n[i] > 0) blocks += (n[i] + kBlock - 1) / kBlock;
    return blocks * kBlock;
}

gas_status gas_adamw_steps(int32_t count, void* const* W, const int32_t* dtypes, const int64_t* n, const float* const* dW, void* m, void* v,
                           float* scales, float* master, int64_t state_elements, int32_t state_bits, float lr, float rate1, float rate2,
                           float eps, const float* weight_decay, int64_t step, const int32_t* steps, const float* sq_norm, float max_norm,
                           void* stream) {
    const char* who = "gas_adamw_steps";
    GAS_REQUIRE(count >= 0 && (count == 0 || (W && dtypes && n && dW && m && v)), "%s: count=%d", who, count);
    for (int32_t i = 0; i < count; ++i) {
        GAS_REQUIRE(n[i] >= 0 && (n[i] == 0 || (W[i] && dW[i])), "%s: tensor %d", who, i);
        if (!valid_dtype(dtypes[i])) return fail(GAS_ERR_DTYPE, "%s: unknown dtype %d of tensor %d", who, dtypes[i], i);
        GAS_REQUIRE(n[i] <= kMostBlocks * kBlock, "%s: tensor %d is too large", who, i);
    }
    GAS_REQUIRE(state_bits == 8 || state_bits == 32, "%s: states of %d bits", who, state_bits);
    GAS_REQUIRE(state_bits == 32 || scales || count == 0, "%s: states of 8 bits without scales", who);
    GAS_REQUIRE(state_elements >= gas_adamw_elements(count, n), "%s: the state has %lld elements, %lld are needed", who,
                (long long)state_elements, (long long)gas_adamw_elements(count, n));
    GAS_REQUIRE(aligned16(m) && aligned16(v) && aligned16(master) && ((uintptr_t)scales & 7u) == 0, "%s: the state is not aligned to 16 bytes", who);
    GAS_REQUIRE(rate1 > 0.f && rate1 <= 1.f && rate2 > 0.f && rate2 <= 1.f && eps >= 1.17549435e-38f, "%s: beta1=%g beta2=%g eps=%g", who, 1.0 - rate1,
                1.0 - rate2, (double)eps);
    GAS_REQUIRE(steps || (step >= 1 && step <= 0x7FFFFFFF), "%s: step=%lld", who, (long long)step);
    GAS_REQUIRE(!sq_norm || max_norm > 0.f, "%s: max_norm=%g", who, (double)max_norm);
    AdamStep b;
    AdamTensors<kTensors> l;
    b.m = m; b.v = v; b.scales = scales; b.master = master;
    const double beta1 = 1.0 - rate1, beta2 = 1.0 - rate2;
    b.lr = lr; b.b1 = (float)beta1; b.b2 = (float)beta2; b.rate1 = rate1; b.rate2 = rate2; b.eps = eps;
    b.step = (uint32_t)step; b.steps = steps; b.sq_norm = sq_norm; b.max_norm = max_norm;
    b.ln1 = (float)log(beta1); b.ln2 = (float)log(beta2);
    b.c1 = steps ? 1.f : (float)(1.0 / (1.0 - pow(beta1, (double)step)));
    b.c2 = steps ? 1.f : (float)(1.0 / sqrt(1.0 - pow(beta2, (double)step)));
    int64_t base = 0;
    for (int32_t i = 0; i < count;) {
        Stretches taken;
        l.count = 0;
        b.base = base;
        int64_t blocks = 0;
        for (; i < count && l.count < kTensors; ++i) {
            if (n[i] == 0) continue;
            const int64_t more = (n[i] + kBlock - 1) / kBlock;
            const uintptr_t w = (uintptr_t)W[i];
            // memory that an earlier tensor of the launch updates too waits for the next one
            if (blocks + more > kMostBlocks || !taken.add(w, w + n[i] * elem_bytes((gas_dtype)dtypes[i]))) break;
            l.W[l.count] = static_cast<char*>(W[i]); l.g[l.count] = dW[i]; l.first[l.count] = (uint32_t)blocks;
            l.decay[l.count] = weight_decay ? lr * weight_decay[i] : 0.f;
            l.last[l.count] = (uint16_t)(n[i] - (more - 1) * kBlock) | (dtypes[i] == GAS_BF16 ? kHalf : 0);
            ++l.count;
            blocks += more;
        }
        if (blocks == 0) continue;
        b.blocks = (uint32_t)blocks;
        base += blocks;
        const dim3 grid((unsigned)((blocks + 3) / 4));
        if (l.count <= kFew) {
            AdamTensors<kFew> few;
            std::copy_n(l.W, l.count, few.W);
            std::copy_n(l.g, l.count, few.g);
            std::copy_n(l.first, l.count, few.first);
            std::copy_n(l.decay, l.count, few.decay);
            std::copy_n(l.last, l.count, few.last);
            few.count = l.count;
            hipLaunchKernelGGL((state_bits == 8 ? adamw_kernel<true, kFew> : adamw_kernel<false, kFew>), grid, dim3(256), 0, (hipStream_t)stream, few, b);
        } else {
            hipLaunchKernelGGL((state_bits == 8 ? adamw_kernel<true, kTensors> : adamw_kernel<false, kTensors>), grid, dim3(256), 0,
                               (hipStream_t)stream, l, b);
        }
        GAS_CHECK_HIP(hipGetLastError());
    }
    return GAS_OK;
}

gas_status gas_adamw_unpack(const void* m, const void* v, const float* scales, int64_t n, gas_dtype dt, void* m_out, void* v_out, void* stream) {
    const char* who = "gas_adamw_unpack";
    if (!valid_dtype(dt)) return fail(GAS_ERR_DTYPE, "%s: unknown dtype %d", who, (int)dt);
    GAS_REQUIRE(n >= 0 && n % kBlock == 0, "%s: n=%lld", who, (long long)n);
    if (n == 0) return GAS_OK;
    GAS_REQUIRE(m && v && scales && m_out && v_out, "%s: null pointer", who);
    GAS_REQUIRE(aligned16(m) && aligned16(v) && aligned16(m_out) && aligned16(v_out) && ((uintptr_t)scales & 7u) == 0,
                "%s: the state or its values are not aligned to 16 bytes", who);
    GAS_REQUIRE((n + 4095) / 4096 <= kMostGroups, "%s: too many elements for one launch", who);
    hipLaunchKernelGGL(dt == GAS_BF16 ? adamw_unpack_kernel<true> : adamw_unpack_kernel<false>, dim3((unsigned)((n + 4095) / 4096)), dim3(256), 0,
                       (hipStream_t)stream, static_cast<const int8_t*>(m), static_cast<const uint8_t*>(v), scales, n / kBlock, static_cast<char*>(m_out),
                       static_cast<char*>(v_out));
    GAS_CHECK_HIP(hipGetLastError());
    return GAS_OK;
}

}  // extern "C"
