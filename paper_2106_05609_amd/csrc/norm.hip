// Norms before and after a block, with the block's gate, its residual scale and the residual stream, forward and backward:
//     y = N_post(a) p + p_bias,   h = x + alpha s sigmoid(t) y,   u = N_pre(h) q + q_bias.
// One wavefront per row, element by element; statistics, sums and the row itself in 32 bits, each output rounded once.
#include "common.h"
#include "wave.h"

namespace gas {
namespace {

struct ResidualNorm {
    const char *X, *A, *T;
    int64_t ldx, lda, ldt;
    int gate_cols;                       // 0: no gate, 1: one gate of a row, F: one of every element
    int64_t n;
    int F, post, pre;
    const float *p, *p_bias, *s, *q, *q_bias;
    float alpha, eps;
    char *H, *U;
    int64_t ldh, ldu;
    float* stats;                        // [n][4]: mean and 1 / deviation of a, and of h
    const int32_t* idx;
    char* hist;
    int64_t ld_hist;
};

template <bool BF>
__device__ __forceinline__ float load_one(const char* p, int64_t i) {
    if constexpr (BF) return __uint_as_float((uint32_t)reinterpret_cast<const uint16_t*>(p)[i] << 16);
    else return reinterpret_cast<const float*>(p)[i];
}
template <bool BF>
__device__ __forceinline__ void store_one(char* p, int64_t i, float v) {
    if constexpr (BF) reinterpret_cast<uint16_t*>(p)[i] = (uint16_t)f32_to_bf16(v);
    else reinterpret_cast<float*>(p)[i] = v;
}
__device__ __forceinline__ float at(const float* v, int f, float otherwise) { return v ? v[f] : otherwise; }
__device__ __forceinline__ float gate_of(float t) { return 1.f / (1.f + expf(-t)); }

// Mean and 1 / deviation over the F values that value(f) gives, the same in every lane.
template <class V>
__device__ __forceinline__ void row_stats(int kind, int F, float eps, V value, float* mean, float* r) {
    const int lane = threadIdx.x & 63;
    *mean = 0.f;
    *r = 1.f;
    if (kind == GAS_NORM_NONE) return;
    if (kind == GAS_NORM_LAYER) {
        float sum = 0.f;
        for (int f = lane; f < F; f += 64) sum += value(f);
        *mean = wave_sum(sum) / (float)F;
    }
    float sq = 0.f;
    for (int f = lane; f < F; f += 64) {
        const float d = value(f) - *mean;
        sq = fmaf(d, d, sq);
    }
    *r = 1.f / sqrtf(wave_sum(sq) / (float)F + eps);
}

template <bool BF>
__global__ __launch_bounds__(256) void residual_norm_kernel(ResidualNorm c) {
    const int lane = threadIdx.x & 63;
    const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (row >= c.n) return;
    float mean_a = 0.f, r_a = 1.f, mean_h, r_h;
    if (c.A) row_stats(c.post, c.F, c.eps, [&](int f) { return load_one<BF>(c.A, row * c.lda + f); }, &mean_a, &r_a);
    const float row_gate = c.gate_cols == 1 ? gate_of(load_one<BF>(c.T, row * c.ldt)) : 1.f;
    auto h_of = [&](int f) {
        const float x = load_one<BF>(c.X, row * c.ldx + f);
        if (!c.A) return x;
        const float y = fmaf((load_one<BF>(c.A, row * c.lda + f) - mean_a) * r_a, at(c.p, f, 1.f), at(c.p_bias, f, 0.f));
        const float g = c.gate_cols > 1 ? gate_of(load_one<BF>(c.T, row * c.ldt + f)) : row_gate;
        return fmaf(c.alpha * at(c.s, f, 1.f) * g, y, x);
    };
    row_stats(c.U || c.hist || c.stats ? c.pre : GAS_NORM_NONE, c.F, c.eps, h_of, &mean_h, &r_h);
    if (c.stats && lane < 4) c.stats[row * 4 + lane] = lane == 0 ? mean_a : lane == 1 ? r_a : lane == 2 ? mean_h : r_h;
    const int64_t to = c.hist ? c.idx[row] : 0;
    for (int f = lane; f < c.F; f += 64) {
        const float h = h_of(f);
        const float u = fmaf((h - mean_h) * r_h, at(c.q, f, 1.f), at(c.q_bias, f, 0.f));
        if (c.H) store_one<BF>(c.H, row * c.ldh + f, h);
        if (c.U) store_one<BF>(c.U, row * c.ldu + f, u);
        if (c.hist) store_one<BF>(c.hist, to * c.ld_hist + f, u);
    }
}

// Backward.  With hn, an the normed rows, d = gu q, c = dy p and P the means of a layer norm (none otherwise):
//     gx = gh + r_h (d - P d - hn mean(d hn)),   dy = gx alpha s g,   ga = r_a (c - P c - an mean(c an)),
//     gt = dy y (1 - g), summed over the row for one gate of a row.
struct ResidualNormBwd {
    const char *GH, *GU, *H, *A, *T;
    int64_t ldgh, ldgu, ldh, lda, ldt;
    int gate_cols;
    const float* stats;
    int64_t n;
    int F, post, pre;
    const float *p, *p_bias, *s, *q;
    float alpha;
    char *GX, *GA, *GT;
    int64_t ldgx, ldga, ldgt;
    float* sums[5];                      // gradients of p, p_bias, s, q, q_bias, or null
    float* row_sums;                     // [n][2]: means of d and of d hn
    float* partials;                     // [slabs][5][F]
    int slabs;
    int64_t rows_per_slab;
};

struct Element { float hn, gu, e, an, y, g, dy; };

// What one element's gradients are made of; d_mean, dh_mean: the row's means of d and d hn.
template <bool BF>
__device__ __forceinline__ Element element(const ResidualNormBwd& c, int64_t row, int f, const float* st, float d_mean, float dh_mean) {
    Element v;
    v.gu = c.GU ? load_one<BF>(c.GU, row * c.ldgu + f) : 0.f;
    v.hn = c.GU ? (load_one<BF>(c.H, row * c.ldh + f) - st[2]) * st[3] : 0.f;
    const float d = v.gu * at(c.q, f, 1.f);
    v.e = (c.GH ? load_one<BF>(c.GH, row * c.ldgh + f) : 0.f) + st[3] * (d - d_mean - v.hn * dh_mean);
    v.an = v.y = v.dy = 0.f;
    v.g = 1.f;
    if (c.A) {
        v.an = (load_one<BF>(c.A, row * c.lda + f) - st[0]) * st[1];
        v.y = fmaf(v.an, at(c.p, f, 1.f), at(c.p_bias, f, 0.f));
        if (c.gate_cols) v.g = gate_of(load_one<BF>(c.T, row * c.ldt + (c.gate_cols == 1 ? 0 : f)));
        v.dy = v.e * c.alpha * at(c.s, f, 1.f) * v.g;
    }
    return v;
}

template <bool BF>
__device__ __forceinline__ void row_stats_of(const ResidualNormBwd& c, int64_t row, float (&st)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) st[i] = c.stats ? c.stats[row * 4 + i] : (i & 1 ? 1.f : 0.f);
}

template <bool BF>
__global__ __launch_bounds__(256) void residual_norm_row_sums_kernel(ResidualNormBwd c) {
    const int lane = threadIdx.x & 63;
    const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (row >= c.n) return;
    float st[4], sd = 0.f, sdh = 0.f;
    row_stats_of<BF>(c, row, st);
    if (c.GU && c.pre != GAS_NORM_NONE)
        for (int f = lane; f < c.F; f += 64) {
            const Element v = element<BF>(c, row, f, st, 0.f, 0.f);
            const float d = v.gu * at(c.q, f, 1.f);
            sd += d;
            sdh = fmaf(d, v.hn, sdh);
        }
    sd = c.pre == GAS_NORM_LAYER ? wave_sum(sd) / (float)c.F : 0.f;
    sdh = wave_sum(sdh) / (float)c.F;
    if (lane < 2) c.row_sums[row * 2 + lane] = lane == 0 ? sd : sdh;
}

// Sums over a slab of rows for 64 columns: a lane has a column, the four wavefronts take the rows in turn.
template <bool BF>
__global__ __launch_bounds__(256) void residual_norm_columns_kernel(ResidualNormBwd c) {
    __shared__ float part[4][5][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int f = blockIdx.x * 64 + lane;
    const int64_t r0 = (int64_t)blockIdx.y * c.rows_per_slab, r1 = r0 + c.rows_per_slab < c.n ? r0 + c.rows_per_slab : c.n;
    float sum[5] = {0.f, 0.f, 0.f, 0.f, 0.f};
    if (f < c.F)
        for (int64_t row = r0 + wave; row < r1; row += 4) {
            float st[4];
            row_stats_of<BF>(c, row, st);
            const Element v = element<BF>(c, row, f, st, c.row_sums[row * 2], c.row_sums[row * 2 + 1]);
            sum[0] = fmaf(v.dy, v.an, sum[0]);
            sum[1] += v.dy;
            sum[2] = fmaf(v.e * c.alpha * v.g, v.y, sum[2]);
            sum[3] = fmaf(v.gu, v.hn, sum[3]);
            sum[4] += v.gu;
        }
#pragma unroll
    for (int k = 0; k < 5; ++k) part[wave][k][lane] = sum[k];
    __syncthreads();
    if (wave == 0 && f < c.F)
#pragma unroll
        for (int k = 0; k < 5; ++k)
            c.partials[((int64_t)blockIdx.y * 5 + k) * c.F + f] = (part[0][k][lane] + part[1][k][lane]) + (part[2][k][lane] + part[3][k][lane]);
}

__global__ __launch_bounds__(64) void residual_norm_finish_kernel(ResidualNormBwd c) {
    const int f = blockIdx.x * 64 + threadIdx.x, k = blockIdx.y;
    if (f >= c.F || !c.sums[k]) return;
    float sum = 0.f;
    for (int j = 0; j < c.slabs; ++j) sum += c.partials[((int64_t)j * 5 + k) * c.F + f];
    c.sums[k][f] = sum;
}

template <bool BF>
__global__ __launch_bounds__(256) void residual_norm_bwd_kernel(ResidualNormBwd c) {
    const int lane = threadIdx.x & 63;
    const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (row >= c.n) return;
    float st[4], sc = 0.f, sca = 0.f, sg = 0.f;
    row_stats_of<BF>(c, row, st);
    const float d_mean = c.row_sums[row * 2], dh_mean = c.row_sums[row * 2 + 1];
    if (c.A)
        for (int f = lane; f < c.F; f += 64) {
            const Element v = element<BF>(c, row, f, st, d_mean, dh_mean);
            const float cc = v.dy * at(c.p, f, 1.f);
            sc += cc;
            sca = fmaf(cc, v.an, sca);
            sg = fmaf(v.dy * v.y, 1.f - v.g, sg);
        }
    sc = c.post == GAS_NORM_LAYER ? wave_sum(sc) / (float)c.F : 0.f;
    sca = c.post == GAS_NORM_NONE ? 0.f : wave_sum(sca) / (float)c.F;
    sg = wave_sum(sg);
    for (int f = lane; f < c.F; f += 64) {
        const Element v = element<BF>(c, row, f, st, d_mean, dh_mean);
        if (c.GX) store_one<BF>(c.GX, row * c.ldgx + f, v.e);
        if (c.GA) store_one<BF>(c.GA, row * c.ldga + f, st[1] * (v.dy * at(c.p, f, 1.f) - sc - v.an * sca));
        if (c.GT && c.gate_cols != 1) store_one<BF>(c.GT, row * c.ldgt + f, v.dy * v.y * (1.f - v.g));
    }
    // after every lane has read the row's gate, which may lie there
    if (c.GT && c.gate_cols == 1 && lane == 0) store_one<BF>(c.GT, row * c.ldgt, sg);
}

constexpr int kSlabs = 256;

inline bool valid_norm(int k) { return k == GAS_NORM_NONE || k == GAS_NORM_RMS || k == GAS_NORM_LAYER; }

// Whether rows i of two matrices [n, fa] and [n, fb] share memory: blocks of columns of one matrix lie in each other's span but apart.
bool share(const void* a, int64_t lda, int64_t fa, const void* b, int64_t ldb, int64_t fb, int64_t n, int eb) {
    if (!a || !b || n == 0) return false;
    const int64_t a0 = (int64_t)(uintptr_t)a, b0 = (int64_t)(uintptr_t)b;
    if (a0 + ((n - 1) * lda + fa) * eb <= b0 || b0 + ((n - 1) * ldb + fb) * eb <= a0) return false;
    if (lda != ldb || (b0 - a0) % eb) return true;
    const int64_t ld = lda, d = (((b0 - a0) / eb) % ld + ld) % ld;      // b's first column, counted from a's
    return d < fa || d + fb > ld;
}
bool same(const void* a, int64_t lda, const void* b, int64_t ldb, int64_t n) { return a == b && (lda == ldb || n == 1); }

}  // namespace
}  // namespace gas

using namespace gas;

extern "C" {

gas_status gas_residual_norm(const void* X, int64_t ldx, const void* A, int64_t lda, const void* T, int64_t ldt, int32_t gate_cols,
                             int64_t n_rows, int32_t F, gas_dtype dt, int32_t norm_post, const float* p, const float* p_bias,
                             const float* s, float alpha, int32_t norm_pre, const float* q, const float* q_bias, float eps, void* H,
                             int64_t ldh, void* U, int64_t ldu, float* stats, const int32_t* push_idx, void* push_hist,
                             int64_t n_hist_rows, int64_t ld_push, void* stream) {
    const char* who = "gas_residual_norm";
    if (!valid_dtype(dt)) return fail(GAS_ERR_DTYPE, "%s: unknown dtype %d", who, (int)dt);
    GAS_REQUIRE(n_rows >= 0 && F > 0, "%s: n_rows=%lld F=%d", who, (long long)n_rows, F);
    if (n_rows == 0) return GAS_OK;
    GAS_REQUIRE(X && (H || U || push_hist), "%s: null pointer", who);
    GAS_REQUIRE(valid_norm(norm_post) && valid_norm(norm_pre), "%s: unknown norm %d, %d", who, norm_post, norm_pre);
    GAS_REQUIRE(eps > 0.f && eps < INFINITY, "%s: eps=%g", who, (double)eps);
    GAS_REQUIRE(A || !T, "%s: a gate without a block", who);
    GAS_REQUIRE(!T || gate_cols == 1 || gate_cols == F, "%s: %d gates for rows of %d", who, gate_cols, F);
    GAS_REQUIRE(ldx >= F && (!A || lda >= F) && (!T || ldt >= gate_cols) && (!H || ldh >= F) && (!U || ldu >= F),
                "%s: row stride smaller than the row", who);
    GAS_REQUIRE(!push_idx == !push_hist && (!push_hist || (ld_push >= F && n_hist_rows >= n_rows)), "%s: bad history table for the push", who);
    const int eb = elem_bytes(dt);
    const struct { const void* p; int64_t ld; int cols; } in[3] = {{X, ldx, F}, {A, lda, F}, {T, ldt, gate_cols}};
    const struct { void* p; int64_t ld; } out[2] = {{H, ldh}, {U, ldu}};
    const int64_t table = push_hist ? (n_hist_rows - 1) * ld_push + F : 0;
    for (const auto& o : out)
        for (const auto& i : in)
            GAS_REQUIRE(!share(o.p, o.ld, F, i.p, i.ld, i.cols, n_rows, eb) || (i.cols == F && same(o.p, o.ld, i.p, i.ld, n_rows)),
                        "%s: an output lies in an input", who);
    GAS_REQUIRE(!share(H, ldh, F, U, ldu, F, n_rows, eb), "%s: the outputs share memory", who);
    for (const auto& i : in)
        GAS_REQUIRE(!push_hist || !i.p || !share(push_hist, table, table, i.p, (n_rows - 1) * i.ld + i.cols, (n_rows - 1) * i.ld + i.cols, 1, eb),
                    "%s: the history table lies in an input", who);
    for (const auto& o : out)
        GAS_REQUIRE(!push_hist || !o.p || !share(push_hist, table, table, o.p, (n_rows - 1) * o.ld + F, (n_rows - 1) * o.ld + F, 1, eb),
                    "%s: the history table lies in an output", who);
    ResidualNorm c;
    c.X = static_cast<const char*>(X); c.A = static_cast<const char*>(A); c.T = static_cast<const char*>(T);
    c.ldx = ldx; c.lda = lda; c.ldt = ldt; c.gate_cols = T ? gate_cols : 0;
    c.n = n_rows; c.F = F; c.post = norm_post; c.pre = norm_pre;
    c.p = p; c.p_bias = p_bias; c.s = s; c.q = q; c.q_bias = q_bias; c.alpha = alpha; c.eps = eps;
    c.H = static_cast<char*>(H); c.U = static_cast<char*>(U); c.ldh = ldh; c.ldu = ldu; c.stats = stats;
    c.idx = push_idx; c.hist = static_cast<char*>(push_hist); c.ld_hist = ld_push;
    const int64_t blocks = (n_rows + 3) / 4;
    GAS_REQUIRE(blocks <= 0x7FFFFFFFLL, "%s: too many rows for one launch", who);
    if (dt == GAS_BF16) hipLaunchKernelGGL(residual_norm_kernel<true>, dim3((unsigned)blocks), dim3(256), 0, (hipStream_t)stream, c);
    else hipLaunchKernelGGL(residual_norm_kernel<false>, dim3((unsigned)blocks), dim3(256), 0, (hipStream_t)stream, c);
    GAS_CHECK_HIP(hipGetLastError());
    return GAS_OK;
}

int64_t gas_residual_norm_bwd_workspace(int64_t n_rows, int32_t F) {
    if (n_rows <= 0 || F <= 0) return 0;
    return ((int64_t)kSlabs * 5 * F + 2 * n_rows) * 4;
}

gas_status gas_residual_norm_bwd(const void* GH, int64_t ldgh, const void* GU, int64_t ldgu, const void* H, int64_t ldh, const void* A,
                                 int64_t lda, const void* T, int64_t ldt, int32_t gate_cols, const float* stats, int64_t n_rows,
                                 int32_t F, gas_dtype dt, int32_t norm_post, const float* p, const float* p_bias, const float* s,
                                 float alpha, int32_t norm_pre, const float* q, void* GX, int64_t ldgx, void* GA, int64_t ldga,
                                 void* GT, int64_t ldgt, float* gp, float* gp_bias, float* gs, float* gq, float* gq_bias,
                                 void* workspace, int64_t workspace_bytes, void* stream) {
    const char* who = "gas_residual_norm_bwd";
    if (!valid_dtype(dt)) return fail(GAS_ERR_DTYPE, "%s: unknown dtype %d", who, (int)dt);
    GAS_REQUIRE(n_rows >= 0 && F > 0, "%s: n_rows=%lld F=%d", who, (long long)n_rows, F);
    hipStream_t st = (hipStream_t)stream;
    const bool sums = gp || gp_bias || gs || gq || gq_bias;
    ResidualNormBwd c;
    c.sums[0] = gp; c.sums[1] = gp_bias; c.sums[2] = gs; c.sums[3] = gq; c.sums[4] = gq_bias;
    c.F = F; c.n = n_rows; c.slabs = 0; c.partials = nullptr;
    const dim3 finish((unsigned)((F + 63) / 64), 5);
    if (n_rows == 0) {                        // an empty sum still has to be written
        if (!sums) return GAS_OK;
        hipLaunchKernelGGL(residual_norm_finish_kernel, finish, dim3(64), 0, st, c);
        GAS_CHECK_HIP(hipGetLastError());
        return GAS_OK;
    }
    GAS_REQUIRE(GH || GU, "%s: null pointer", who);
    GAS_REQUIRE(valid_norm(norm_post) && valid_norm(norm_pre), "%s: unknown norm %d, %d", who, norm_post, norm_pre);
    GAS_REQUIRE(A || !(T || GA || GT || gp || gp_bias || gs), "%s: a block's gradient without the block", who);
    GAS_REQUIRE(T || !GT, "%s: a gate's gradient without the gate", who);
    GAS_REQUIRE(GU || !(gq || gq_bias), "%s: a gain's gradient without the gradient of what it gives", who);
    GAS_REQUIRE(!GU || H, "%s: the gradient of the normed rows without the rows", who);
    GAS_REQUIRE(GX || GA || GT || sums, "%s: null pointer", who);
    GAS_REQUIRE(stats || ((!GU || norm_pre == GAS_NORM_NONE) && (!A || norm_post == GAS_NORM_NONE)), "%s: norms without statistics", who);
    GAS_REQUIRE(!T || gate_cols == 1 || gate_cols == F, "%s: %d gates for rows of %d", who, gate_cols, F);
    GAS_REQUIRE((!GH || ldgh >= F) && (!GU || (ldgu >= F && ldh >= F)) && (!A || lda >= F) && (!T || ldt >= gate_cols) && (!GX || ldgx >= F) &&
                (!GA || ldga >= F) && (!GT || ldgt >= gate_cols), "%s: row stride smaller than the row", who);
    const int eb = elem_bytes(dt);
    const struct { const void* p; int64_t ld; int cols; } in[5] = {{GH, ldgh, F}, {GU, ldgu, F}, {GU ? H : nullptr, ldh, F}, {A, lda, F}, {T, ldt, gate_cols}};
    const struct { void* p; int64_t ld; int cols; } out[3] = {{GX, ldgx, F}, {GA, ldga, F}, {GT, ldgt, gate_cols}};
    for (int o = 0; o < 3; ++o) {
        for (const auto& i : in)
            GAS_REQUIRE(!share(out[o].p, out[o].ld, out[o].cols, i.p, i.ld, i.cols, n_rows, eb) ||
                        (i.cols == out[o].cols && same(out[o].p, out[o].ld, i.p, i.ld, n_rows)), "%s: an output lies in an input", who);
        for (int k = 0; k < o; ++k)
            GAS_REQUIRE(!share(out[o].p, out[o].ld, out[o].cols, out[k].p, out[k].ld, out[k].cols, n_rows, eb), "%s: the outputs share memory", who);
    }
    GAS_REQUIRE(workspace && workspace_bytes >= gas_residual_norm_bwd_workspace(n_rows, F), "%s: the workspace has %lld bytes, %lld are needed", who,
                (long long)workspace_bytes, (long long)gas_residual_norm_bwd_workspace(n_rows, F));
    GAS_REQUIRE(aligned16(workspace), "%s: the workspace is not aligned to 16 bytes", who);
    c.GH = static_cast<const char*>(GH); c.GU = static_cast<const char*>(GU); c.H = static_cast<const char*>(H);
    c.A = static_cast<const char*>(A); c.T = static_cast<const char*>(T);
    c.ldgh = ldgh; c.ldgu = ldgu; c.ldh = ldh; c.lda = lda; c.ldt = ldt; c.gate_cols = T ? gate_cols : 0;
    c.stats = stats; c.post = norm_post; c.pre = norm_pre; c.p = p; c.p_bias = p_bias; c.s = s; c.q = q; c.alpha = alpha;
    c.GX = static_cast<char*>(GX); c.GA = static_cast<char*>(GA); c.GT = static_cast<char*>(GT);
    c.ldgx = ldgx; c.ldga = ldga; c.ldgt = ldgt;
    c.partials = static_cast<float*>(workspace);
    c.row_sums = c.partials + (int64_t)kSlabs * 5 * F;
    c.rows_per_slab = (n_rows + kSlabs - 1) / kSlabs;
    c.slabs = (int)((n_rows + c.rows_per_slab - 1) / c.rows_per_slab);
    const int64_t blocks = (n_rows + 3) / 4;
    GAS_REQUIRE(blocks <= 0x7FFFFFFFLL, "%s: too many rows for one launch", who);
    const bool bf = dt == GAS_BF16;
    hipLaunchKernelGGL(bf ? residual_norm_row_sums_kernel<true> : residual_norm_row_sums_kernel<false>, dim3((unsigned)blocks), dim3(256), 0, st, c);
    GAS_CHECK_HIP(hipGetLastError());
    if (sums) {                               // before the outputs, which may lie where the inputs do
        hipLaunchKernelGGL(bf ? residual_norm_columns_kernel<true> : residual_norm_columns_kernel<false>,
                           dim3((unsigned)((F + 63) / 64), (unsigned)c.slabs), dim3(256), 0, st, c);
        GAS_CHECK_HIP(hipGetLastError());
        hipLaunchKernelGGL(residual_norm_finish_kernel, finish, dim3(64), 0, st, c);
        GAS_CHECK_HIP(hipGetLastError());
    }
    if (GX || GA || GT) {
        hipLaunchKernelGGL(bf ? residual_norm_bwd_kernel<true> : residual_norm_bwd_kernel<false>, dim3((unsigned)blocks), dim3(256), 0, st, c);
        GAS_CHECK_HIP(hipGetLastError());
    }
    return GAS_OK;
}

}  // extern "C"
