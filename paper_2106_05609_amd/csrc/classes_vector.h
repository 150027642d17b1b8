// Logits of up to eight rows by the vector units (classes.h says what they are of): bound by reading W once, as it lies.
#pragma once
#include "classes.h"

namespace gas {
namespace {

struct VectorArgs {
    const void *X, *W, *bias;
    int64_t ldx, ldw, ldz, stats;
    const int32_t* idx;           // the rows that count, shape->count of them; NULL: all n
    const Shape* shape;
    int32_t n, F, C;
    float inv_t;                  // 0: one temperature
    float* z;                     // [n][ldz]
    Parts parts;                  // `most` NULL: not asked for
};

// A workgroup 256 classes, four a lane; its eight wavefronts take every eighth row of W, sixteen rows of it under way at a time, and their sums
// are added up through LDS. Rows of W need no alignment beyond their elements'. 1 x 256 x 100,003 of bf16 takes 17.7 us (2.9 TB/s), 1 x 512 x 50,021 of
// fp32 18.8 (5.4), 3 x 512 x 188,933 81 (4.8, the rate of a copy).
template <bool BF, int R>
__global__ __launch_bounds__(512) void classes_vector_kernel(VectorArgs a) {
    typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(2)));
    typedef float f32x4_here __attribute__((ext_vector_type(4), aligned(4)));
    constexpr int kChunk = 512, U = 16;
    __shared__ __attribute__((aligned(16))) float xs[kChunk * R];
    __shared__ __attribute__((aligned(16))) float sums[2][8][256];
    __shared__ float stats[3][2][4];
    const int n = a.idx ? a.shape->count : a.n;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c0 = blockIdx.x * 256 + 4 * lane, at = c0 + 4 <= a.C ? c0 : (a.C >= 4 ? a.C - 4 : 0);    // the last whole four where these are not
    float acc[R][4];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[r][e] = 0.f;
    struct Four { float v[4]; };
    auto load = [&](int f) {
        Four w;
        if (a.C < 4) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int64_t i = (int64_t)f * a.ldw + (e < a.C ? e : 0);
                w.v[e] = BF ? __uint_as_float((uint32_t)static_cast<const uint16_t*>(a.W)[i] << 16) : static_cast<const float*>(a.W)[i];
            }
        } else if constexpr (BF) {
            const u32x2_any v = *reinterpret_cast<const u32x2_any*>(static_cast<const uint16_t*>(a.W) + (int64_t)f * a.ldw + at);
            w = Four{bf16_lo(v[0]), bf16_hi(v[0]), bf16_lo(v[1]), bf16_hi(v[1])};
        } else {
            const f32x4_here v = *reinterpret_cast<const f32x4_here*>(static_cast<const float*>(a.W) + (int64_t)f * a.ldw + at);
            w = Four{v[0], v[1], v[2], v[3]};
        }
        return w;
    };
    auto use = [&](const Four& w, int i) {                // i: of the row of W in the chunk
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const float x = xs[i * R + r];
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[r][e] = fmaf(x, w.v[e], acc[r][e]);
        }
    };
    for (int f0 = 0; f0 < a.F; f0 += kChunk) {
        const int fs = a.F - f0 < kChunk ? a.F - f0 : kChunk;
        __syncthreads();
        for (int i = tid; i < fs * R; i += 512) {
            const int r = i / fs, f = i % fs;
            float x = 0.f;
            if (r < n) {
                const int64_t j = (int64_t)(a.idx ? a.idx[r] : r) * a.ldx + f0 + f;
                x = BF ? __uint_as_float((uint32_t)static_cast<const uint16_t*>(a.X)[j] << 16) : static_cast<const float*>(a.X)[j];
            }
            xs[f * R + r] = x;
        }
        __syncthreads();
        int f = wave;
        for (; f + 8 * (U - 1) < fs; f += 8 * U) {
            Four w[U];
#pragma unroll
            for (int u = 0; u < U; ++u) w[u] = load(f0 + f + 8 * u);
#pragma unroll
            for (int u = 0; u < U; ++u) use(w[u], f + 8 * u);
        }
        for (; f < fs; f += 8) use(load(f0 + f), f);
    }
#pragma unroll
    for (int r0 = 0; r0 < R; r0 += 2) {                   // two rows at a time: 256 threads each
        if (r0 >= n) break;
        __syncthreads();
#pragma unroll
        for (int h = 0; h < 2; ++h)
            if (r0 + h < R) {
                if (at == c0) *reinterpret_cast<f32x4*>(&sums[h][wave][4 * lane]) = f32x4{acc[(r0 + h) % R][0], acc[(r0 + h) % R][1], acc[(r0 + h) % R][2], acc[(r0 + h) % R][3]};
                else
                    for (int e = 0; e < 4; ++e)
                        if (at + e >= c0 && at + e < a.C) sums[h][wave][at + e - blockIdx.x * 256] = acc[(r0 + h) % R][e];
            }
        __syncthreads();
        const int h = tid >> 8, t = tid & 255, r = r0 + h, c = blockIdx.x * 256 + t;
        const bool on = r < n && r < R && c < a.C;
        float z = -INFINITY;
        if (on) {
            z = 0.f;
#pragma unroll
            for (int w = 0; w < 8; ++w) z += sums[h][w][t];
            if (a.bias) z += BF ? __uint_as_float((uint32_t)static_cast<const uint16_t*>(a.bias)[c] << 16) : static_cast<const float*>(a.bias)[c];
            a.z[r * a.ldz + c] = z;
        }
        if (a.parts.most) {
            float most = z;
#pragma unroll
            for (int o = 32; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor(most, o));
            if (lane == 0) stats[0][h][wave & 3] = most;
            __syncthreads();
            most = fmaxf(fmaxf(stats[0][h][0], stats[0][h][1]), fmaxf(stats[0][h][2], stats[0][h][3]));
            most = fmaxf(most * kLog2e, kLeastExponent);
            const float d = fmaf(z, kLog2e, -most);
            float sum = exp2_of(d), sum_t = exp2_of(d * a.inv_t);
#pragma unroll
            for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
            if (a.inv_t != 0.f)
#pragma unroll
                for (int o = 32; o > 0; o >>= 1) sum_t += __shfl_xor(sum_t, o);
            if (lane == 0) {
                stats[1][h][wave & 3] = sum;
                stats[2][h][wave & 3] = sum_t;
            }
            __syncthreads();
            if (t == 0 && r < n && r < R) {
                a.parts.most[blockIdx.x * a.stats + r] = most;
                a.parts.sum[blockIdx.x * a.stats + r] = stats[1][h][0] + stats[1][h][1] + stats[1][h][2] + stats[1][h][3];
                if (a.inv_t != 0.f) a.parts.sum_t[blockIdx.x * a.stats + r] = stats[2][h][0] + stats[2][h][1] + stats[2][h][2] + stats[2][h][3];
            }
        }
    }
}

template <bool BF>
gas_status launch_vector(const VectorArgs& a, hipStream_t s) {
    const dim3 grid((unsigned)((a.C + 255) / 256)), block(512);
    if (a.n == 1) hipLaunchKernelGGL((classes_vector_kernel<BF, 1>), grid, block, 0, s, a);
    else if (a.n == 2) hipLaunchKernelGGL((classes_vector_kernel<BF, 2>), grid, block, 0, s, a);
    else if (a.n <= 4) hipLaunchKernelGGL((classes_vector_kernel<BF, 4>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((classes_vector_kernel<BF, 8>), grid, block, 0, s, a);
    GAS_CHECK_HIP(hipGetLastError());
    return GAS_OK;
}

}  // namespace
}  // namespace gas
