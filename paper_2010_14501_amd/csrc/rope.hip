// Rotary positions: pair i of a head, (a, b), is turned by the angle of the token's position t,
//   (a cos - b sin, b cos + a sin) * scale,  angle = t f_i,
// pairs being neighbours (interleaved) or lying rot_dim / 2 apart; the rest of a head stays.  The gradient is turned back by the same angle.
// Bound by memory: x is read and y written.  Angles are reduced in 64 bits: t f_i of a position of a million has lost 16 of fp32's 24 bits.
#include <cmath>

#include "../../include/monet_kernels.h"
#include "kernels.hpp"
#include "tile_bf16.hpp"

namespace monet {

namespace {

constexpr int ROPE_DIM = 512;       // rot_dim, at most
struct RopeFreqs { double turns[ROPE_DIM / 2]; };      // whole turns a position, in the kernel's arguments

__device__ __forceinline__ float value(float v) { return v; }
__device__ __forceinline__ float value(unsigned short v) { return bf16_float(v); }
__device__ __forceinline__ void put(float *p, float v, bool add) { *p = add ? *p + v : v; }
__device__ __forceinline__ void put(unsigned short *p, float v, bool add) { *p = float_bf16(add ? bf16_float(*p) + v : v); }

// cosine and sine of a number of turns: the nearest quarter turn is taken off in 64 bits, what is left is at most an eighth
__device__ __forceinline__ void turn(double turns, float &c, float &s) {
    const double t = 4.0 * (turns - rint(turns)), q = rint(t);
    float cr, sr;
    sincospif(0.5f * (float)(t - q), &sr, &cr);
    const int n = (int)q & 3;
    c = n & 1 ? sr : cr;
    s = n & 1 ? cr : sr;
    if (n == 1 || n == 2) c = -c;
    if (n & 2) s = -s;
}

// a thread to a pair, or to a value that stays
template <class T>
__global__ __launch_bounds__(256) void rope_kernel(const T *x, T *y, const int32_t *__restrict__ positions, const RopeFreqs f, int64_t n, int heads, int dim,
                                                   int rot, int64_t x_ld, int64_t y_ld, int interleaved, float scale, int inverse, int add) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= n) return;
    const int units = dim - rot / 2, u = (int)(i % units), h = (int)(i / units % heads);
    const int64_t t = i / units / heads;
    x += t * x_ld + h * dim;
    y += t * y_ld + h * dim;
    if (u >= rot / 2) {
        const int at = u + rot / 2;
        put(y + at, value(x[at]), add);
        return;
    }
    const int a = interleaved ? 2 * u : u, b = interleaved ? 2 * u + 1 : u + rot / 2;
    float c, s;
    turn((positions ? positions[t] : (int)t) * f.turns[u], c, s);
    c *= scale;
    s *= inverse ? -scale : scale;
    const float va = value(x[a]), vb = value(x[b]);
    put(y + a, va * c - vb * s, add);
    put(y + b, vb * c + va * s, add);
}

}  // namespace

void rope_freqs(double *freqs, int rot_dim, double base, double factor, double original, double low, double high) {
    if (!freqs) throw KernelError("rope_freqs: null pointer");
    if (rot_dim < 2 || rot_dim % 2 || rot_dim > ROPE_DIM) throw KernelError("rope_freqs: rot_dim must be even, 2 to " + std::to_string(ROPE_DIM));
    if (!(base > 0) || !std::isfinite(base)) throw KernelError("rope_freqs: the base must be positive and finite");
    if (!(factor > 0) || !std::isfinite(factor)) throw KernelError("rope_freqs: the factor must be positive and finite");
    const bool blend = low != 0 || high != 0;
    if (blend && !(original > 0 && std::isfinite(original) && low >= 0 && high > low && std::isfinite(high)))
        throw KernelError("rope_freqs: a blend needs original > 0 and 0 <= low < high");
    for (int i = 0; i < rot_dim / 2; ++i) {
        const double f = std::pow(base, -2.0 * i / rot_dim);
        const double keep = blend ? std::min(1.0, std::max(0.0, (original * f / (2 * M_PI) - low) / (high - low))) : 0.0;
        freqs[i] = f * (keep + (1 - keep) / factor);
    }
}

void rope(hipStream_t st, int dtype, const void *x, void *y, const int32_t *positions, const double *freqs, int64_t tokens, int heads, int head_dim,
          int rot_dim, int64_t x_ld, int64_t y_ld, bool interleaved, float scale, bool inverse, bool accumulate) {
    if (dtype != MONET_F32 && dtype != MONET_BF16) throw KernelError("rope: dtype must be MONET_F32 or MONET_BF16");
    if (tokens < 0 || heads < 1 || head_dim < 1) throw KernelError("rope: bad shape");
    if (rot_dim < 2 || rot_dim % 2 || rot_dim > ROPE_DIM || rot_dim > head_dim)
        throw KernelError("rope: rot_dim must be even, 2 to head_dim and at most " + std::to_string(ROPE_DIM));
    if (tokens >= (1ll << 31) || heads > 65536 || head_dim > 65536) throw KernelError("rope: shape too large");
    if (!std::isfinite(scale)) throw KernelError("rope: the scale must be finite");
    if (!freqs) throw KernelError("rope: null pointer");
    RopeFreqs f;
    for (int i = 0; i < ROPE_DIM / 2; ++i) {
        f.turns[i] = i < rot_dim / 2 ? freqs[i] / (2 * M_PI) : 0;
        if (!std::isfinite(f.turns[i])) throw KernelError("rope: frequencies must be finite");
    }
    const int64_t n = tokens * heads * (head_dim - rot_dim / 2);
    if (n >= (1ll << 31) * 128) throw KernelError("rope: shape too large");
    if (!tokens) return;
    const int64_t width = (int64_t)heads * head_dim;
    if (!x || !y) throw KernelError("rope: null pointer");
    if (((uintptr_t)x | (uintptr_t)y) % (dtype == MONET_BF16 ? 2 : 4) || (uintptr_t)positions % 4) throw KernelError("rope: pointer not aligned");
    if (x_ld < width || y_ld < width) throw KernelError("rope: token stride below heads * head_dim");
    if (x_ld >= (1ll << 31) || y_ld >= (1ll << 31)) throw KernelError("rope: token stride too large");
    if (x == y && (x_ld != y_ld || accumulate)) throw KernelError("rope: in place, the token strides must be the same and nothing can be added to");
    const dim3 grid((unsigned)((n + 255) / 256));
    if (dtype == MONET_F32)
        hipLaunchKernelGGL(rope_kernel<float>, grid, dim3(256), 0, st, (const float *)x, (float *)y, positions, f, n, heads, head_dim, rot_dim, x_ld, y_ld,
                           interleaved, scale, inverse, accumulate);
    else
        hipLaunchKernelGGL(rope_kernel<unsigned short>, grid, dim3(256), 0, st, (const unsigned short *)x, (unsigned short *)y, positions, f, n, heads, head_dim,
                           rot_dim, x_ld, y_ld, interleaved, scale, inverse, accumulate);
    hip_check(hipGetLastError(), "rope launch");
}

}  // namespace monet
