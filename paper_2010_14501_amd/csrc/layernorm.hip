// Layer norm over rows of x [rows][cols]:
//   mean = sum x / cols,  rstd = 1 / sqrt(sum (x - mean)^2 / cols + eps),  xh = (x - mean) rstd,  y = xh gamma + beta.
// Backward, with g = dy gamma:
//   dx = rstd (g - sum g / cols - xh sum(g xh) / cols),  dgamma = sum over rows of dy xh,  dbeta = sum over rows of dy.
// Bound by memory: forward reads x and writes y, backward reads dy and x and writes dx.  All sums are fp32.
#include <cmath>

#include "../../include/monet_kernels.h"
#include "kernels.hpp"
#include "tile_bf16.hpp"

namespace monet {

namespace {

__device__ __forceinline__ float value(float v) { return v; }
__device__ __forceinline__ float value(unsigned short v) { return bf16_float(v); }
__device__ __forceinline__ void put(float *p, float v, bool add) { *p = add ? *p + v : v; }
__device__ __forceinline__ void put(unsigned short *p, float v, bool add) { *p = float_bf16(add ? bf16_float(*p) + v : v); }

__device__ __forceinline__ float sum_of_256(float v, float *seg) {      // the same in every thread
    for (int w = 32; w; w /= 2) v += __shfl_xor(v, w);
    __syncthreads();
    if (threadIdx.x % 64 == 0) seg[threadIdx.x / 64] = v;
    __syncthreads();
    return (seg[0] + seg[1]) + (seg[2] + seg[3]);
}

// a workgroup to a row, which is read once for each of its sums and once more for the result
template <class T, class P>
__global__ __launch_bounds__(256) void layernorm_fwd_kernel(const T *x, const P *__restrict__ gamma, const P *__restrict__ beta, T *y,
                                                            float2 *__restrict__ stats, int cols, int64_t x_ld, int64_t y_ld, float eps) {
    __shared__ float seg[4];
    const int64_t row = blockIdx.x;
    x += row * x_ld;
    y += row * y_ld;
    float sum = 0.f;
    for (int c = threadIdx.x; c < cols; c += 256) sum += value(x[c]);
    const float mean = sum_of_256(sum, seg) / cols;
    sum = 0.f;
    for (int c = threadIdx.x; c < cols; c += 256) {
        const float d = value(x[c]) - mean;
        sum = fmaf(d, d, sum);
    }
    const float rstd = 1.f / sqrtf(sum_of_256(sum, seg) / cols + eps);
    for (int c = threadIdx.x; c < cols; c += 256)
        put(y + c, fmaf((value(x[c]) - mean) * rstd, gamma ? value(gamma[c]) : 1.f, beta ? value(beta[c]) : 0.f), false);
    if (stats && threadIdx.x == 0) stats[row] = make_float2(mean, rstd);
}

template <class T, class P>
__global__ __launch_bounds__(256) void layernorm_dx_kernel(const T *dy, const T *__restrict__ x, const P *__restrict__ gamma, const float2 *__restrict__ stats,
                                                           T *dx, int cols, int64_t dy_ld, int64_t x_ld, int64_t dx_ld, bool add) {
    __shared__ float seg[4];
    const int64_t row = blockIdx.x;
    dy += row * dy_ld;
    x += row * x_ld;
    dx += row * dx_ld;
    const float mean = stats[row].x, rstd = stats[row].y;
    float a = 0.f, b = 0.f;
    for (int c = threadIdx.x; c < cols; c += 256) {
        const float g = value(dy[c]) * (gamma ? value(gamma[c]) : 1.f);
        a += g;
        b = fmaf(g, (value(x[c]) - mean) * rstd, b);
    }
    a = sum_of_256(a, seg) / cols;
    b = sum_of_256(b, seg) / cols;
    for (int c = threadIdx.x; c < cols; c += 256) {
        const float g = value(dy[c]) * (gamma ? value(gamma[c]) : 1.f);
        put(dx + c, rstd * (g - a - (value(x[c]) - mean) * rstd * b), add);
    }
}

// 64 columns of a range of rows: part[range][0: dgamma, 1: dbeta][cols]
template <class T>
__global__ __launch_bounds__(256) void layernorm_columns_kernel(const T *__restrict__ dy, const T *__restrict__ x, const float2 *__restrict__ stats,
                                                                float *__restrict__ part, int64_t rows, int64_t per, int cols, int64_t dy_ld, int64_t x_ld) {
    __shared__ float sums[2][4][64];
    const int l = threadIdx.x & 63, wave = threadIdx.x / 64, c = blockIdx.x * 64 + l;
    const int64_t from = blockIdx.y * per, to = min(rows, from + per);
    float a = 0.f, b = 0.f;
    if (c < cols)
        for (int64_t r = from + wave; r < to; r += 4) {
            const float d = value(dy[r * dy_ld + c]);
            a = fmaf(d, (value(x[r * x_ld + c]) - stats[r].x) * stats[r].y, a);
            b += d;
        }
    sums[0][wave][l] = a;
    sums[1][wave][l] = b;
    __syncthreads();
    if (wave >= 2 || c >= cols) return;
    part[((int64_t)blockIdx.y * 2 + wave) * cols + c] = (sums[wave][0][l] + sums[wave][1][l]) + (sums[wave][2][l] + sums[wave][3][l]);
}

// the parts' sums: grid y 0 dgamma, 1 dbeta (null: not wanted); four waves take a share of the ranges each, in a fixed order
template <class P>
__global__ __launch_bounds__(256) void layernorm_join_kernel(const float *__restrict__ part, int ranges, int cols, P *dgamma, P *dbeta, int add) {
    __shared__ float sums[4][64];
    const int l = threadIdx.x & 63, wave = threadIdx.x / 64, c = blockIdx.x * 64 + l, which = blockIdx.y;
    P *out = which ? dbeta : dgamma;
    if (!out) return;
    float s = 0.f;
    if (c < cols)
        for (int r = wave; r < ranges; r += 4) s += part[((int64_t)r * 2 + which) * cols + c];
    sums[wave][l] = s;
    __syncthreads();
    if (wave || c >= cols) return;
    put(out + c, (sums[0][l] + sums[1][l]) + (sums[2][l] + sums[3][l]), add >> which & 1);
}

int64_t cut(int64_t n, int64_t by) { return (n + by - 1) / by; }

constexpr int LAYERNORM_COLS = 1 << 20;

int64_t layernorm_ranges(int64_t rows, int cols) {
    return std::min<int64_t>(cut(rows, 32), std::max<int64_t>(1, 1024 / cut(cols, 64)));
}
void layernorm_shape(int dtype, int64_t rows, int cols) {
    if (dtype != MONET_F32 && dtype != MONET_BF16) throw KernelError("layernorm: dtype must be MONET_F32 or MONET_BF16");
    if (rows < 0 || cols < 1) throw KernelError("layernorm: bad shape");
    if (rows >= (1ll << 31) || cols > LAYERNORM_COLS) throw KernelError("layernorm: shape too large");
}
void layernorm_params(int param_dtype) {
    if (param_dtype != MONET_F32 && param_dtype != MONET_BF16) throw KernelError("layernorm: param_dtype must be MONET_F32 or MONET_BF16");
}
void layernorm_tensor(const void *p, int dtype, int64_t ld, int cols) {
    if (!p) throw KernelError("layernorm: null pointer");
    if ((uintptr_t)p % (dtype == MONET_BF16 ? 2 : 4)) throw KernelError("layernorm: pointer not aligned");
    if (ld < cols) throw KernelError("layernorm: row stride below the number of columns");
    if (ld >= (1ll << 31)) throw KernelError("layernorm: row stride too large");
}
void layernorm_param(const void *p, int param_dtype) {      // may be null
    if ((uintptr_t)p % (param_dtype == MONET_BF16 ? 2 : 4)) throw KernelError("layernorm: pointer not aligned");
}

template <class F>
void by_types(int dtype, int param_dtype, F &&f) {
    if (dtype == MONET_F32 && param_dtype == MONET_F32) f(0.f, 0.f);
    else if (dtype == MONET_F32) f(0.f, (unsigned short)0);
    else if (param_dtype == MONET_F32) f((unsigned short)0, 0.f);
    else f((unsigned short)0, (unsigned short)0);
}

}  // namespace

void layernorm_fwd(hipStream_t st, int dtype, int param_dtype, const void *x, const void *gamma, const void *beta, void *y, float *stats, int64_t rows,
                   int cols, int64_t x_ld, int64_t y_ld, float eps) {
    layernorm_shape(dtype, rows, cols);
    layernorm_params(param_dtype);
    if (!(eps > 0.f) || !std::isfinite(eps)) throw KernelError("layernorm: eps must be positive and finite");
    if (!rows) return;
    layernorm_tensor(x, dtype, x_ld, cols);
    layernorm_tensor(y, dtype, y_ld, cols);
    if (x == y && x_ld != y_ld) throw KernelError("layernorm: in place, the row strides must be the same");
    layernorm_param(gamma, param_dtype);
    layernorm_param(beta, param_dtype);
    if ((uintptr_t)stats % 8) throw KernelError("layernorm: stats must be 8-byte aligned");
    by_types(dtype, param_dtype, [&](auto t, auto p) {
        using T = decltype(t);
        using P = decltype(p);
        hipLaunchKernelGGL((layernorm_fwd_kernel<T, P>), dim3((unsigned)rows), dim3(256), 0, st, (const T *)x, (const P *)gamma, (const P *)beta, (T *)y,
                           (float2 *)stats, cols, x_ld, y_ld, eps);
    });
    hip_check(hipGetLastError(), "layernorm launch");
}

size_t layernorm_bwd_workspace_bytes(int dtype, int64_t rows, int cols) {
    layernorm_shape(dtype, rows, cols);
    return (size_t)(layernorm_ranges(rows, cols) * 2 * cols * 4);
}

void layernorm_bwd(hipStream_t st, int dtype, int param_dtype, const void *dy, const void *x, const void *gamma, const float *stats, void *dx, void *dgamma,
                   void *dbeta, int64_t rows, int cols, int64_t dy_ld, int64_t x_ld, int64_t dx_ld, int accumulate, void *ws, size_t ws_bytes) {
    const size_t need = layernorm_bwd_workspace_bytes(dtype, rows, cols);
    layernorm_params(param_dtype);
    if (accumulate & ~7) throw KernelError("layernorm: accumulate has bits 0 to 2");
    if (rows) {
        layernorm_tensor(dy, dtype, dy_ld, cols);
        layernorm_tensor(x, dtype, x_ld, cols);
        if (dx) layernorm_tensor(dx, dtype, dx_ld, cols);
        if (dx == dy && dx_ld != dy_ld) throw KernelError("layernorm: in place, the row strides must be the same");
        if (!stats || (uintptr_t)stats % 8) throw KernelError("layernorm: stats must be given, 8-byte aligned");
    }
    layernorm_param(gamma, param_dtype);
    layernorm_param(dgamma, param_dtype);
    layernorm_param(dbeta, param_dtype);
    const bool columns = dgamma || dbeta;
    if (columns && need) {
        if (!ws || ws_bytes < need) throw KernelError("layernorm: workspace of " + std::to_string(ws_bytes) + " bytes, " + std::to_string(need) + " needed");
        if ((uintptr_t)ws % 256) throw KernelError("layernorm: the workspace must be 256-byte aligned");
    }
    const int64_t ranges = layernorm_ranges(rows, cols);
    by_types(dtype, param_dtype, [&](auto t, auto p) {
        using T = decltype(t);
        using P = decltype(p);
        if (columns) {
            if (rows) {
                hipLaunchKernelGGL(layernorm_columns_kernel<T>, dim3((unsigned)cut(cols, 64), (unsigned)ranges), dim3(256), 0, st, (const T *)dy, (const T *)x,
                                   (const float2 *)stats, (float *)ws, rows, cut(rows, ranges), cols, dy_ld, x_ld);
                hip_check(hipGetLastError(), "layernorm columns launch");
            }
            hipLaunchKernelGGL(layernorm_join_kernel<P>, dim3((unsigned)cut(cols, 64), 2), dim3(256), 0, st, (const float *)ws, (int)ranges, cols, (P *)dgamma,
                               (P *)dbeta, accumulate >> 1);
            hip_check(hipGetLastError(), "layernorm join launch");
        }
        if (dx && rows) {
            hipLaunchKernelGGL((layernorm_dx_kernel<T, P>), dim3((unsigned)rows), dim3(256), 0, st, (const T *)dy, (const T *)x, (const P *)gamma,
                               (const float2 *)stats, (T *)dx, cols, dy_ld, x_ld, dx_ld, accumulate & 1);
            hip_check(hipGetLastError(), "layernorm gradient launch");
        }
    });
}

}  // namespace monet
