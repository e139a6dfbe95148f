// amsim_norm.hip -- residual root-mean-square norm, forward (with an 8-bit output) and backward, and
// the row quantiser.
//
// Per row of n values:  h = x + r,  rstd = (sum h^2 / n + eps)^(-1/2),  y = h rstd w,
//   scale = max|y| / 127,  q = round(y 127 / max|y|).
// Backward, with g = dy w:  dx = rstd (g - h rstd^2 sum(g h) / n) + dh,  dw = sum over rows dy h rstd.
// All of it in FP32; x, r, dy, h and dh are read once and h, y, q, dx written once, so the kernels are
// bound by memory: a row stays in the registers of the workgroup (or wave) that owns it.
#include "amsim_q8.h"

namespace {

using namespace amsim_q8;

constexpr int64_t kMaxNorm = 32768;  // a row in the registers of 1024 threads

// Sum (or maximum) over the THREADS threads that share a row.  With 64 of them it is one wave's own.
template <int THREADS, bool MAX>
__device__ __forceinline__ float row_reduce(float v, float *lds)
{
    v = MAX ? wave_max_nan(v) : wave_sum(v);
    if constexpr (THREADS == 64) return v;
    constexpr int W = THREADS / 64;
    __syncthreads();  // the last reduction's values have been read
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    float r = lds[0];
#pragma unroll
    for (int w = 1; w < W; ++w) r = MAX ? max_nan(r, lds[w]) : r + lds[w];
    return r;
}

struct FwdArgs {
    const void *x, *r;
    const float *w;
    void *h, *y;
    int8_t *q;
    float *scale, *rstd;
    int64_t rows, n, ldx, ldr, ldh, ldy, ldq;
    float eps;
};

// THREADS threads hold a row in CH chunks of eight values each; with 64, a workgroup of 256 has four rows.
// 8190 x 4096 BF16, residual in, h and 8 bits out: 55 us, 4.3 TB/s.  Quantising 8192 x 4096 BF16: 19 us, 5.3 TB/s.  One
// row: 3 us.  (Workgroups that stay and read their next row ahead: 61 us.)
template <typename T, int THREADS, int CH, bool NORM>
__global__ __launch_bounds__(THREADS == 64 ? 256 : THREADS) void norm_fwd_kernel(FwdArgs a)
{
    constexpr int ROWS = THREADS == 64 ? 4 : 1;
    __shared__ float lds[16];
    const int tid = threadIdx.x % THREADS;
    const int64_t row = int64_t(blockIdx.x) * ROWS + threadIdx.x / THREADS;
    if (row >= a.rows) return;  // whole waves, and no barrier follows for waves that own a row each
    float v[CH][8], w[NORM ? CH : 1][8];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int64_t i = int64_t(c * THREADS + tid) * 8;
        load8(static_cast<const T *>(a.x) + row * a.ldx + i, a.n - i, v[c]);
    }
    if (NORM && a.r) {
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int64_t i = int64_t(c * THREADS + tid) * 8;
            float r[8];
            load8(static_cast<const T *>(a.r) + row * a.ldr + i, a.n - i, r);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[c][e] += r[e];
        }
    }
    if constexpr (NORM) {  // on their way during the reduction
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int64_t i = int64_t(c * THREADS + tid) * 8;
            load8(a.w + i, a.n - i, w[c]);
        }
    }
    if (NORM && a.h) {
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int64_t i = int64_t(c * THREADS + tid) * 8;
            store8(static_cast<T *>(a.h) + row * a.ldh + i, a.n - i, v[c]);
        }
    }
    if constexpr (NORM) {
        float ss = 0.0f;
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int e = 0; e < 8; ++e) ss = __builtin_fmaf(v[c][e], v[c][e], ss);
        ss = row_reduce<THREADS, false>(ss, lds);
        const float rstd = 1.0f / __builtin_sqrtf(ss / float(a.n) + a.eps);
        if (a.rstd && tid == 0) a.rstd[row] = rstd;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int64_t i = int64_t(c * THREADS + tid) * 8;
#pragma unroll
            for (int e = 0; e < 8; ++e) v[c][e] = v[c][e] * rstd * w[c][e];
            if (a.y) store8(static_cast<T *>(a.y) + row * a.ldy + i, a.n - i, v[c]);
        }
    }
    if (!a.q) return;
    float amax = 0.0f;
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) amax = max_nan(__builtin_fabsf(v[c][e]), amax);
    amax = row_reduce<THREADS, true>(amax, lds);
    const Scale s = scale_of(amax);
    if (tid == 0) a.scale[row] = s.scale;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int64_t i = int64_t(c * THREADS + tid) * 8;
        store_q8(a.q + row * a.ldq + i, a.n - i, v[c], s.inv);
    }
}

// Quantises rows longer than the registers hold: the maximum, then the row again.
template <typename T>
__global__ __launch_bounds__(1024) void quantize_long_kernel(FwdArgs a)
{
    __shared__ float lds[16];
    const int64_t row = blockIdx.x;
    const T *x = static_cast<const T *>(a.x) + row * a.ldx;
    float amax = 0.0f;
    for (int64_t i = int64_t(threadIdx.x) * 8; i < a.n; i += 8192) {
        float v[8];
        load8(x + i, a.n - i, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) amax = max_nan(__builtin_fabsf(v[e]), amax);
    }
    const Scale s = scale_of(row_reduce<1024, true>(amax, lds));
    if (threadIdx.x == 0) a.scale[row] = s.scale;
    for (int64_t i = int64_t(threadIdx.x) * 8; i < a.n; i += 8192) {
        float v[8];
        load8(x + i, a.n - i, v);
        store_q8(a.q + row * a.ldq + i, a.n - i, v, s.inv);
    }
}

template <typename T, bool NORM>
void launch_rows(const FwdArgs &a, hipStream_t st)
{
    const dim3 one(static_cast<unsigned>(a.rows)), four(static_cast<unsigned>(ceil_div(a.rows, 4)));
#define FWD(THREADS, CH) \
    hipLaunchKernelGGL((norm_fwd_kernel<T, THREADS, CH, NORM>), THREADS == 64 ? four : one, \
                       dim3(THREADS == 64 ? 256 : THREADS), 0, st, a)
    if (a.n <= 512)
        FWD(64, 1);
    else if (a.n <= 1024)
        FWD(64, 2);
    else if (a.n <= 2048)
        FWD(256, 1);
    else if (a.n <= 4096)
        FWD(256, 2);
    else if (a.n <= 8192 && NORM)  // 57 against 64 us for 8190 x 4097 in bf16; the quantiser 32 against 27 us
        FWD(512, 2);
    else if (a.n <= 8192)
        FWD(256, 4);
    else if (a.n <= 16384)
        FWD(1024, 2);
    else if (a.n <= kMaxNorm)
        FWD(1024, 4);
    else
        hipLaunchKernelGGL((quantize_long_kernel<T>), one, dim3(1024), 0, st, a);
#undef FWD
}

template <typename T, bool NORM>
int launch_fwd(const FwdArgs &a, hipStream_t st)
{
    in_launches(a.rows, [&](int64_t first, unsigned count) {
        FwdArgs p = a;
        const auto from = [&](const void *t, int64_t ld) { return t ? static_cast<const T *>(t) + first * ld : nullptr; };
        const auto to = [&](void *t, int64_t ld) { return t ? static_cast<T *>(t) + first * ld : nullptr; };
        p.x = from(a.x, a.ldx), p.r = from(a.r, a.ldr), p.h = to(a.h, a.ldh), p.y = to(a.y, a.ldy);
        if (a.q) p.q = a.q + first * a.ldq, p.scale = a.scale + first;
        if (a.rstd) p.rstd = a.rstd + first;
        p.rows = count;
        launch_rows<T, NORM>(p, st);
    });
    return launch_status();
}

// ------------------------------------------------------------------ backward -------------

struct BwdArgs {
    const void *dy, *dh, *h;
    const float *w, *rstd;
    void *dx;
    float *part;  // [gridDim.x * ROWS][n]: sums of dy h rstd over each owner's rows
    int64_t rows, n, lddy, lddh, ldh, lddx;
};

// A row stays in registers between the sum and dx, and so do the owner's sums for dw over all of its rows.
// 6000 x 2048 FP32 with dh: 37 us, 5.3 TB/s (192 MB).  (Reading the next row ahead takes registers from
// waves that would hide the latency: 94 against 63 us for 8192 x 4096 BF16.)  Above 16384 elements some of a thread's
// values go to scratch memory: 1024 x 32768 BF16 215 us, three times what 2048 x 16384 takes (74 us), FP32 255 us.
template <typename T, int THREADS, int CH>
__global__ __launch_bounds__(THREADS == 64 ? 256 : THREADS) void norm_bwd_kernel(BwdArgs a)
{
    constexpr int ROWS = THREADS == 64 ? 4 : 1;
    __shared__ float lds[16];
    const int tid = threadIdx.x % THREADS;
    const int64_t owner = int64_t(blockIdx.x) * ROWS + threadIdx.x / THREADS;
    float w[CH][8], dw[CH][8];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int64_t i = int64_t(c * THREADS + tid) * 8;
        load8(a.w + i, a.n - i, w[c]);
#pragma unroll
        for (int e = 0; e < 8; ++e) dw[c][e] = 0.0f;
    }
    for (int64_t row = owner; row < a.rows; row += int64_t(gridDim.x) * ROWS) {
        float g[CH][8], h[CH][8];
        const float rstd = a.rstd[row];
        float dot = 0.0f;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int64_t i = int64_t(c * THREADS + tid) * 8;
            load8(static_cast<const T *>(a.dy) + row * a.lddy + i, a.n - i, g[c]);
            load8(static_cast<const T *>(a.h) + row * a.ldh + i, a.n - i, h[c]);
        }
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                dw[c][e] = __builtin_fmaf(g[c][e], h[c][e] * rstd, dw[c][e]);
                g[c][e] *= w[c][e];
                dot = __builtin_fmaf(g[c][e], h[c][e], dot);
            }
        dot = row_reduce<THREADS, false>(dot, lds);
        const float k = rstd * rstd * dot / float(a.n);
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int64_t i = int64_t(c * THREADS + tid) * 8;
            float d[8];
            if (a.dh) {
                load8(static_cast<const T *>(a.dh) + row * a.lddh + i, a.n - i, d);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) d[e] = 0.0f;
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) d[e] += rstd * (g[c][e] - h[c][e] * k);
            store8(static_cast<T *>(a.dx) + row * a.lddx + i, a.n - i, d);
        }
    }
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int64_t i = int64_t(c * THREADS + tid) * 8;
        store8(a.part + owner * a.n + i, a.n - i, dw[c]);
    }
}

// dw[j] = sum of part[p][j] over the owners: 16 columns to a workgroup (enough of them for a row of 2048 to
// take half the GPU), 64 threads to a column deal out the owners, and their sums are added in a tree.
// (1024 owners of 2048: 4.7 us.)
__global__ __launch_bounds__(1024) void norm_dw_kernel(const float *part, float *dw, int64_t owners, int64_t n)
{
    __shared__ float lds[64][17];
    const int col = threadIdx.x & 15, g = threadIdx.x >> 4;
    const int64_t j = int64_t(blockIdx.x) * 16 + col;
    float s = 0.0f;
    if (j < n) {
#pragma unroll 8
        for (int64_t p = g; p < owners; p += 64) s += part[p * n + j];
    }
    lds[g][col] = s;
    __syncthreads();
#pragma unroll
    for (int w = 32; w > 0; w >>= 1) {
        if (g < w) lds[g][col] += lds[g + w][col];
        __syncthreads();
    }
    if (g == 0 && j < n) dw[j] = lds[0][col];
}

// Owners of rows in the backward pass: enough workgroups to fill the GPU, each with several rows, since
// every owner leaves n partial sums.
struct BwdPlan {
    int64_t groups, owners;
};

BwdPlan plan_bwd(int64_t rows, int64_t n)
{
    const int64_t per = n <= 1024 ? 4 : 1;
    const int64_t groups = ceil_div(rows, per) < 1024 ? ceil_div(rows, per) : 1024;
    return {groups, groups * per};
}

template <typename T>
void launch_bwd(const BwdArgs &a, unsigned groups, hipStream_t st)
{
#define BWD(THREADS, CH) \
    hipLaunchKernelGGL((norm_bwd_kernel<T, THREADS, CH>), dim3(groups), dim3(THREADS == 64 ? 256 : THREADS), 0, st, a)
    if (a.n <= 512)
        BWD(64, 1);
    else if (a.n <= 1024)
        BWD(64, 2);
    else if (a.n <= 2048)
        BWD(256, 1);
    else if (a.n <= 4096)
        BWD(256, 2);
    else if (a.n <= 8192)
        BWD(512, 2);
    else if (a.n <= 16384)
        BWD(1024, 2);
    else
        BWD(1024, 4);
#undef BWD
}

bool bad_rows(int64_t rows, int64_t n) { return rows < 0 || n < 0; }
bool too_large(int64_t rows, int64_t n) { return rows >= int64_t(1) << 31 || n >= int64_t(1) << 31; }

}  // namespace

extern "C" {

int amsim_rmsnorm_fwd(int dtype, int64_t rows, int64_t n, const void *x, int64_t ldx, const void *residual,
                      int64_t ldr, const float *weight, float eps, void *h, int64_t ldh, void *y, int64_t ldy,
                      int8_t *q, int64_t ldq, float *q_scale, float *rstd, void *stream)
{
    if (!valid_type(dtype) || bad_rows(rows, n) || !(eps >= 0.0f)) return AMSIM_ERR_INVALID_ARG;
    if (too_large(rows, n) || n > kMaxNorm) return AMSIM_ERR_UNSUPPORTED;
    if (rows == 0) return AMSIM_OK;
    if (n == 0 || !x || !weight || (!h && !y && !q && !rstd) || (q && !q_scale)) return AMSIM_ERR_INVALID_ARG;
    if (ldx < n || (residual && ldr < n) || (h && ldh < n) || (y && ldy < n) || (q && ldq < n))
        return AMSIM_ERR_INVALID_ARG;
    const FwdArgs a{x, residual, weight, h, y, q, q_scale, rstd, rows, n, ldx, ldr, ldh, ldy, ldq, eps};
    return with_type(dtype, [&](auto t) {
        return launch_fwd<decltype(t), true>(a, static_cast<hipStream_t>(stream));
    });
}

int amsim_quantize_rows(int dtype, int64_t rows, int64_t n, const void *x, int64_t ldx, int8_t *q, int64_t ldq,
                        float *q_scale, void *stream)
{
    if (!valid_type(dtype) || bad_rows(rows, n)) return AMSIM_ERR_INVALID_ARG;
    if (too_large(rows, n)) return AMSIM_ERR_UNSUPPORTED;
    if (rows == 0) return AMSIM_OK;
    if (n == 0 || !x || !q || !q_scale || ldx < n || ldq < n) return AMSIM_ERR_INVALID_ARG;
    FwdArgs a{};
    a.x = x, a.q = q, a.scale = q_scale, a.rows = rows, a.n = n, a.ldx = ldx, a.ldq = ldq;
    return with_type(dtype, [&](auto t) {
        return launch_fwd<decltype(t), false>(a, static_cast<hipStream_t>(stream));
    });
}

int amsim_rmsnorm_bwd_workspace_size(int64_t rows, int64_t n, size_t *bytes)
{
    if (!bytes || bad_rows(rows, n)) return AMSIM_ERR_INVALID_ARG;
    if (too_large(rows, n) || n > kMaxNorm) return AMSIM_ERR_UNSUPPORTED;
    *bytes = size_t(plan_bwd(rows, n).owners) * size_t(n) * sizeof(float);
    return AMSIM_OK;
}

int amsim_rmsnorm_bwd(int dtype, int64_t rows, int64_t n, const void *dy, int64_t lddy, const void *dh, int64_t lddh,
                      const void *h, int64_t ldh, const float *weight, const float *rstd, void *dx, int64_t lddx,
                      float *dw, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!valid_type(dtype)) return AMSIM_ERR_INVALID_ARG;
    size_t need = 0;
    const int rc = amsim_rmsnorm_bwd_workspace_size(rows, n, &need);
    if (rc != AMSIM_OK) return rc;
    if (n == 0) return rows == 0 ? AMSIM_OK : AMSIM_ERR_INVALID_ARG;
    if (!dw) return AMSIM_ERR_INVALID_ARG;
    if (rows > 0) {
        if (!dy || !h || !weight || !rstd || !dx || lddy < n || ldh < n || lddx < n || (dh && lddh < n))
            return AMSIM_ERR_INVALID_ARG;
        if (!workspace || workspace_bytes < need) return AMSIM_ERR_WORKSPACE;
        if (uintptr_t(workspace) & 15) return AMSIM_ERR_INVALID_ARG;
    }
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const BwdPlan plan = plan_bwd(rows, n);
    float *part = static_cast<float *>(workspace);
    if (rows > 0) {
        const BwdArgs a{dy, dh, h, weight, rstd, dx, part, rows, n, lddy, lddh, ldh, lddx};
        with_type(dtype, [&](auto t) {
            launch_bwd<decltype(t)>(a, static_cast<unsigned>(plan.groups), st);
            return AMSIM_OK;
        });
    }
    hipLaunchKernelGGL(norm_dw_kernel, dim3(static_cast<unsigned>(ceil_div(n, 16))), dim3(1024), 0, st, part, dw,
                       plan.owners, n);
    return launch_status();
}

}  // extern "C"
