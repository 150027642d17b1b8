// The step of a model with many tensors: the squared norm of all gradients, and AdamW with states in 32 bits or in 8.
//     g = c dW,  m <- b1 m + (1 - b1) g,  v <- b2 v + (1 - b2) g^2,
//     W <- W - lr wd W - lr (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps)
// One wavefront takes the 256 elements that share a scale; both kernels are bound by memory, small models by the launch.
#include "common.h"
#include "wave.h"

namespace gas {
namespace {

constexpr int kTensors = 112;                       // of a launch: their descriptions fit the 4 KB of a launch's arguments
constexpr int kBlock = 256;                         // elements that share a scale: four for every lane
constexpr int kNormChunk = 16384;                   // elements of a partial sum

// Index of the tensor that unit `u` (a block, a chunk) belongs to: the last one whose first unit is not behind it.
template <class T>
__device__ __forceinline__ int tensor_of(const T& b, uint32_t u) {
    int lo = 0, hi = b.count;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (b.first[mid] <= u) lo = mid;
        else hi = mid;
    }
    return lo;
}

// ---- the squared norm of many tensors
struct NormBatch {
    const float* x[kTensors];
    int64_t n[kTensors];
    uint32_t first[kTensors];                       // chunk that the tensor begins with
    int count;
    double* partials;
};

__device__ __forceinline__ double wave_sum64(double v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    return v;
}

__global__ __launch_bounds__(256) void sq_norms_kernel(NormBatch b) {
    __shared__ double part[4];
    const int k = tensor_of(b, blockIdx.x);
    const float* x = b.x[k];
    const int64_t e0 = (int64_t)(blockIdx.x - b.first[k]) * kNormChunk;
    const int64_t e1 = e0 + kNormChunk < b.n[k] ? e0 + kNormChunk : b.n[k];
    double s = 0.0;
    for (int64_t i = e0 + threadIdx.x; i < e1; i += 256) s = fma((double)x[i], (double)x[i], s);
    s = wave_sum64(s);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) b.partials[blockIdx.x] = (part[0] + part[1]) + (part[2] + part[3]);
}

__global__ __launch_bounds__(256) void sq_norms_finish_kernel(const double* partials, int64_t n, float* out, int32_t* steps) {
    __shared__ double part[4];
    double s = 0.0;
    for (int64_t i = threadIdx.x; i < n; i += 256) s += partials[i];
    s = wave_sum64(s);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        const float total = (float)((part[0] + part[1]) + (part[2] + part[3]));
        out[0] = total;
        if (steps && total < INFINITY) ++*steps;    // neither an infinity nor a NaN
    }
}

// ---- AdamW
struct AdamBatch {
    char* W[kTensors];
    const float* g[kTensors];
    int64_t n[kTensors];
    uint32_t first[kTensors];                       // block that the tensor begins with, counted from `base`
    float decay[kTensors];                          // lr times the weight decay
    uint8_t bf[kTensors];
    int count;
    int64_t base;                                   // the launch's first block
    uint32_t blocks;
    void *m, *v;
    float *scales, *master;
    float lr, b1, b2, rate1, rate2, eps;
    float c1, c2;                                   // 1 / (1 - b1^t), 1 / sqrt(1 - b2^t)
    float ln1, ln2;                                 // logarithms of b1, b2, for a step that is read on the device
    uint32_t step;
    const int32_t* steps;
    const float* sq_norm;
    float max_norm;
};

// Two numbers of 16 bits from an element's place in the state and the step: multiplied and folded until every bit of both
// has reached all others.
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

// The largest magnitude of the wavefront's values, by their bits: a NaN is larger than all.
__device__ __forceinline__ float largest(const float (&x)[4]) {
    uint32_t u = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) u = max(u, __float_as_uint(fabsf(x[i])));
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) u = max(u, (uint32_t)__shfl_xor(u, o));
    return __uint_as_float(u);
}

template <bool EIGHT>
__global__ __launch_bounds__(256) void adamw_kernel(AdamBatch b) {
    const uint32_t unit = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (unit >= b.blocks) return;
    float c = 1.f;
    if (b.sq_norm) {
        const float total = *b.sq_norm;
        if (!(total < INFINITY)) return;            // the whole launch alike
        c = fminf(1.f, (float)((double)b.max_norm / (sqrt((double)total) + 1e-6)));
    }
    float c1 = b.c1, c2 = b.c2;
    uint32_t step = b.step;
    if (b.steps) {
        step = (uint32_t)*b.steps;
        c1 = 1.f / -expm1f((float)step * b.ln1);
        c2 = 1.f / sqrtf(-expm1f((float)step * b.ln2));
    }
    const int lane = threadIdx.x & 63, k = tensor_of(b, unit);
    const int64_t e0 = (int64_t)(unit - b.first[k]) * kBlock, s0 = (b.base + unit) * kBlock;
    const int64_t n = b.n[k];
    float m[4], v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t e = e0 + lane + 64 * i, at = s0 + lane + 64 * i;
        m[i] = v[i] = 0.f;
        if (e >= n) continue;
        if constexpr (EIGHT) {
            m[i] = decode_m(reinterpret_cast<const int8_t*>(b.m)[at], b.scales[2 * (b.base + unit)]);
            v[i] = decode_v(reinterpret_cast<const uint8_t*>(b.v)[at], b.scales[2 * (b.base + unit) + 1]);
        } else {
            m[i] = reinterpret_cast<const float*>(b.m)[at];
            v[i] = reinterpret_cast<const float*>(b.v)[at];
        }
        const float g = c * b.g[k][e];
        // every product and sum rounds by itself: the codes do not depend on what a compiler contracts
        m[i] = __fadd_rn(__fmul_rn(m[i], b.b1), __fmul_rn(g, b.rate1));
        v[i] = __fadd_rn(__fmul_rn(v[i], b.b2), __fmul_rn(__fmul_rn(g, g), b.rate2));
        const bool half = b.bf[k];
        float w;
        if (half && b.master) w = b.master[at];
        else w = half ? __uint_as_float((uint32_t)reinterpret_cast<const uint16_t*>(b.W[k])[e] << 16) : reinterpret_cast<const float*>(b.W[k])[e];
        w = w - w * b.decay[k] - m[i] * (b.lr * c1) / (sqrtf(v[i]) * c2 + b.eps);
        if (half && b.master) b.master[at] = w;
        if (half) reinterpret_cast<uint16_t*>(b.W[k])[e] = (uint16_t)f32_to_bf16(w);
        else reinterpret_cast<float*>(b.W[k])[e] = w;
        if constexpr (!EIGHT) {
            reinterpret_cast<float*>(b.m)[at] = m[i];
            reinterpret_cast<float*>(b.v)[at] = v[i];
        }
    }
    if constexpr (EIGHT) {
        float sm = largest(m), sv = largest(v);
        sm = sm < 1.17549435e-38f ? 0.f : sm;       // below the normal numbers: nothing
        sv = sv < 1.17549435e-38f ? 0.f : sv;
        const float im = sm > 0.f ? 1.f / sm : 0.f, iv = sv > 0.f ? 1.f / sv : 0.f;
        if (lane == 0) {
            b.scales[2 * (b.base + unit)] = sm;
            b.scales[2 * (b.base + unit) + 1] = sv;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t e = e0 + lane + 64 * i, at = s0 + lane + 64 * i;
            if (e >= n) continue;
            const uint32_t die = dice(at, step);
            const int km = encode<2, 127>(fabsf(m[i]) * im * 16129.f, die & 0xFFFFu);
            int kv = encode<4, 255>(v[i] * iv * 4228250625.f, die >> 16);
            if (kv == 0 && v[i] > 0.f && sv > 0.f) kv = 1;      // a denominator never becomes nothing
            reinterpret_cast<int8_t*>(b.m)[at] = (int8_t)(m[i] < 0.f ? -km : km);
            reinterpret_cast<uint8_t*>(b.v)[at] = (uint8_t)kv;
        }
    }
}

template <bool BF>
__global__ __launch_bounds__(256) void adamw_unpack_kernel(const int8_t* m, const uint8_t* v, const float* scales, int64_t n, char* m_out, char* v_out) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= n) return;
    const float a = decode_m(m[i], scales[2 * (i / kBlock)]), b = decode_v(v[i], scales[2 * (i / kBlock) + 1]);
    if constexpr (BF) {
        reinterpret_cast<uint16_t*>(m_out)[i] = (uint16_t)f32_to_bf16(a);
        reinterpret_cast<uint16_t*>(v_out)[i] = (uint16_t)f32_to_bf16(b);
    } else {
        reinterpret_cast<float*>(m_out)[i] = a;
        reinterpret_cast<float*>(v_out)[i] = b;
    }
}

constexpr int64_t kMostBlocks = 0x7FFFFFFFLL;

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
    GAS_REQUIRE(need / 8 <= kMostBlocks, "%s: too many elements", who);
    double* partials = static_cast<double*>(workspace);
    int64_t done = 0;
    for (int32_t i = 0; i < count;) {
        NormBatch b;
        b.count = 0;
        b.partials = partials + done;
        int64_t chunks = 0;
        for (; i < count && b.count < kTensors; ++i) {
            if (n[i] == 0) continue;
            b.x[b.count] = x[i]; b.n[b.count] = n[i]; b.first[b.count] = (uint32_t)chunks;
            ++b.count;
            chunks += (n[i] + kNormChunk - 1) / kNormChunk;
        }
        if (chunks == 0) continue;
        hipLaunchKernelGGL(sq_norms_kernel, dim3((unsigned)chunks), dim3(256), 0, (hipStream_t)stream, b);
        GAS_CHECK_HIP(hipGetLastError());
        done += chunks;
    }
    hipLaunchKernelGGL(sq_norms_finish_kernel, dim3(1), dim3(256), 0, (hipStream_t)stream, partials, done, out, steps);
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
    }
    GAS_REQUIRE(state_bits == 8 || state_bits == 32, "%s: states of %d bits", who, state_bits);
    GAS_REQUIRE(state_bits == 32 || scales || count == 0, "%s: states of 8 bits without scales", who);
    GAS_REQUIRE(state_elements >= gas_adamw_elements(count, n), "%s: the state has %lld elements, %lld are needed", who,
                (long long)state_elements, (long long)gas_adamw_elements(count, n));
    GAS_REQUIRE(rate1 > 0.f && rate1 <= 1.f && rate2 > 0.f && rate2 <= 1.f && eps > 0.f, "%s: beta1=%g beta2=%g eps=%g", who, 1.0 - rate1,
                1.0 - rate2, (double)eps);
    GAS_REQUIRE(steps || (step >= 1 && step <= 0x7FFFFFFF), "%s: step=%lld", who, (long long)step);
    GAS_REQUIRE(!sq_norm || max_norm > 0.f, "%s: max_norm=%g", who, (double)max_norm);
    AdamBatch b;
    b.m = m; b.v = v; b.scales = scales; b.master = master;
    const double beta1 = 1.0 - rate1, beta2 = 1.0 - rate2;
    b.lr = lr; b.b1 = (float)beta1; b.b2 = (float)beta2; b.rate1 = rate1; b.rate2 = rate2; b.eps = eps;
    b.step = (uint32_t)step; b.steps = steps; b.sq_norm = sq_norm; b.max_norm = max_norm;
    b.ln1 = (float)log(beta1); b.ln2 = (float)log(beta2);
    b.c1 = steps ? 1.f : (float)(1.0 / (1.0 - pow(beta1, (double)step)));
    b.c2 = steps ? 1.f : (float)(1.0 / sqrt(1.0 - pow(beta2, (double)step)));
    int64_t base = 0;
    for (int32_t i = 0; i < count;) {
        b.count = 0;
        b.base = base;
        int64_t blocks = 0;
        for (; i < count && b.count < kTensors; ++i) {
            if (n[i] == 0) continue;
            const int64_t more = (n[i] + kBlock - 1) / kBlock;
            GAS_REQUIRE(more <= kMostBlocks, "%s: tensor %d is too large", who, i);
            char* w = static_cast<char*>(W[i]);
            const int64_t bytes = n[i] * elem_bytes((gas_dtype)dtypes[i]);
            bool apart = blocks + more <= kMostBlocks;       // memory that an earlier tensor of the launch updates too waits for the next one
            for (int j = 0; j < b.count && apart; ++j) apart = w + bytes <= b.W[j] || b.W[j] + b.n[j] * (b.bf[j] ? 2 : 4) <= w;
            if (!apart) break;
            b.W[b.count] = w; b.g[b.count] = dW[i]; b.n[b.count] = n[i]; b.first[b.count] = (uint32_t)blocks;
            b.decay[b.count] = weight_decay ? lr * weight_decay[i] : 0.f;
            b.bf[b.count] = dtypes[i] == GAS_BF16;
            ++b.count;
            blocks += more;
        }
        if (blocks == 0) continue;
        b.blocks = (uint32_t)blocks;
        base += blocks;
        hipLaunchKernelGGL(state_bits == 8 ? adamw_kernel<true> : adamw_kernel<false>, dim3((unsigned)((blocks + 3) / 4)), dim3(256), 0,
                           (hipStream_t)stream, b);
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
    GAS_REQUIRE(n / 256 <= kMostBlocks, "%s: too many elements for one launch", who);
    hipLaunchKernelGGL(dt == GAS_BF16 ? adamw_unpack_kernel<true> : adamw_unpack_kernel<false>, dim3((unsigned)(n / 256)), dim3(256), 0,
                       (hipStream_t)stream, static_cast<const int8_t*>(m), static_cast<const uint8_t*>(v), scales, n, static_cast<char*>(m_out),
                       static_cast<char*>(v_out));
    GAS_CHECK_HIP(hipGetLastError());
    return GAS_OK;
}

}  // extern "C"
