// Rotary positions: pair i of a head, (a, b), is turned by the angle of the token's position t,
//   (a cos - b sin, b cos + a sin) * scale,  angle = t f_i,
// pairs being neighbours (interleaved) or lying rot_dim / 2 apart; the rest of a head stays.  The gradient is turned back by the same angle.
// Bound by memory: x is read and y written.  Angles are reduced in 64 bits: t f_i of a position of a million has lost 16 of fp32's 24 bits.
#include <cmath>
#include <type_traits>

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

// A unit of a head: V pairs, two runs of V values (interleaved: one of 2 V), or V values that stay.  A workgroup takes `per_token` units of each of
// `at_once` tokens, up to ROPE_UNITS to a thread: all of them are loaded before the angles of its tokens are computed, each once for all heads.
constexpr int ROPE_UNITS = 4;
template <class T, int V, bool INTERLEAVED>
__global__ __launch_bounds__(256) void rope_kernel(const T *x, T *y, const int32_t *__restrict__ positions, const RopeFreqs f, int64_t tokens, unsigned at_once,
                                                   unsigned units, unsigned per_token, unsigned per_head, unsigned dim, unsigned half, int64_t x_ld, int64_t y_ld,
                                                   float scale, int inverse, int add) {
    extern __shared__ float2 table[];       // [token][pair]: cos, sin
    const int64_t t0 = (int64_t)blockIdx.x * at_once;
    const unsigned here = (unsigned)min((int64_t)at_once, tokens - t0), first = blockIdx.y * per_token, count = min(per_token, units - first);
    T va[ROPE_UNITS][V], vb[ROPE_UNITS][V];
    const auto place = [&](unsigned i, unsigned &token, unsigned &u) {      // of unit i: the offset of its head
        token = i / count;
        const unsigned j = first + i - token * count, h = j / per_head;
        u = j - h * per_head;
        return (int64_t)h * dim;
    };
#pragma unroll
    for (int k = 0; k < ROPE_UNITS; ++k) {
        const unsigned i = k * 256 + threadIdx.x;
        if (i >= here * count) break;
        unsigned token, u;
        const int64_t head = place(i, token, u);
        const T *p = x + (t0 + token) * x_ld + head;
        if (u * V >= half) __builtin_memcpy(va[k], p + half + u * V, sizeof va[k]);
        else if (INTERLEAVED) {
            __builtin_memcpy(va[k], p + 2 * V * u, sizeof va[k]);
            __builtin_memcpy(vb[k], p + 2 * V * u + V, sizeof vb[k]);
        } else {
            __builtin_memcpy(va[k], p + V * u, sizeof va[k]);
            __builtin_memcpy(vb[k], p + half + V * u, sizeof vb[k]);
        }
    }
    for (unsigned i = threadIdx.x; i < here * half; i += 256) {
        const unsigned token = i / half, pair = i - token * half;
        float c, s;
        turn((positions ? positions[t0 + token] : (int)(t0 + token)) * f.turns[pair], c, s);
        table[i] = make_float2(c * scale, s * (inverse ? -scale : scale));
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < ROPE_UNITS; ++k) {
        const unsigned i = k * 256 + threadIdx.x;
        if (i >= here * count) break;
        unsigned token, u;
        const int64_t head = place(i, token, u);
        T *p = y + (t0 + token) * y_ld + head;
        const auto store = [&](T *at, const float (&f)[V]) {
            T v[V];
            if (add) __builtin_memcpy(v, at, sizeof v);
#pragma unroll
            for (int e = 0; e < V; ++e) put(v + e, f[e], add);
            __builtin_memcpy(at, v, sizeof v);
        };
        if (u * V >= half) {
            float stays[V];
#pragma unroll
            for (int e = 0; e < V; ++e) stays[e] = value(va[k][e]);
            store(p + half + u * V, stays);
            continue;
        }
        const float2 *cs = table + token * half + u * V;
        float a[V], b[V];
#pragma unroll
        for (int e = 0; e < V; ++e) {       // pair e: values 2 e and 2 e + 1 of the two runs, or e of each
            const float m = value(INTERLEAVED ? (2 * e < V ? va[k][2 * e % V] : vb[k][2 * e % V]) : va[k][e]);
            const float n = value(INTERLEAVED ? (2 * e + 1 < V ? va[k][(2 * e + 1) % V] : vb[k][(2 * e + 1) % V]) : vb[k][e]);
            const float2 t = cs[e];
            a[e] = m * t.x - n * t.y;
            b[e] = n * t.x + m * t.y;
        }
        if (INTERLEAVED) {
            float low[V], high[V];
#pragma unroll
            for (int e = 0; e < V; ++e) {
                low[e] = e % 2 ? b[e / 2] : a[e / 2];
                high[e] = (e + V) % 2 ? b[(e + V) / 2] : a[(e + V) / 2];
            }
            store(p + 2 * V * u, low);
            store(p + 2 * V * u + V, high);
        } else {
            store(p + V * u, a);
            store(p + half + V * u, b);
        }
    }
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
    const int64_t width = (int64_t)heads * head_dim;
    if (tokens >= 1 << 24 || width >= 1 << 26) throw KernelError("rope: shape too large");
    if (!std::isfinite(scale)) throw KernelError("rope: the scale must be finite");
    if (!freqs) throw KernelError("rope: null pointer");
    RopeFreqs f;
    for (int i = 0; i < ROPE_DIM / 2; ++i) {
        f.turns[i] = i < rot_dim / 2 ? freqs[i] / (2 * M_PI) : 0;
        if (!std::isfinite(f.turns[i])) throw KernelError("rope: frequencies must be finite");
    }
    if (!tokens) return;
    if (!x || !y) throw KernelError("rope: null pointer");
    if (((uintptr_t)x | (uintptr_t)y) % (dtype == MONET_BF16 ? 2 : 4) || (uintptr_t)positions % 4) throw KernelError("rope: pointer not aligned");
    if (x_ld < width || y_ld < width) throw KernelError("rope: token stride below heads * head_dim");
    if (x_ld >= (1ll << 31) || y_ld >= (1ll << 31)) throw KernelError("rope: token stride too large");
    if (x == y && (x_ld != y_ld || accumulate)) throw KernelError("rope: in place, the token strides must be the same and nothing can be added to");
    // the widest pieces that pairs and the rest of a head are whole numbers of; where y is x, the rest is there already
    const int half = rot_dim / 2, rest = head_dim - rot_dim;
    const auto launch = [&](auto t, auto v, auto interleaved_) {
        using T = decltype(t);
        constexpr int V = decltype(v)::value;
        if (half % V || rest % V) return false;
        const unsigned per_head = (unsigned)((half + (x == y ? 0 : rest)) / V), units = per_head * (unsigned)heads, most = 256 * ROPE_UNITS;
        const unsigned per_token = std::min(units, most);
        // several tokens to a workgroup where there are enough of them to fill the card; 8 KB of angles at most
        const unsigned at_once = (unsigned)std::max<int64_t>(1, std::min<int64_t>({most / per_token, tokens / 512, 1024 / half}));
        const dim3 grid((unsigned)((tokens + at_once - 1) / at_once), (units + per_token - 1) / per_token);
        hipLaunchKernelGGL((rope_kernel<T, V, decltype(interleaved_)::value>), grid, dim3(256), at_once * half * sizeof(float2), st, (const T *)x, (T *)y, positions,
                           f, tokens, at_once, units, per_token, per_head, (unsigned)head_dim, (unsigned)half, x_ld, y_ld, scale, inverse, accumulate);
        return true;
    };
    using std::integral_constant;
    const auto with = [&](auto i) {
        if (dtype == MONET_F32)
            return launch(0.f, integral_constant<int, 4>(), i) || launch(0.f, integral_constant<int, 2>(), i) || launch(0.f, integral_constant<int, 1>(), i);
        const unsigned short b = 0;
        return launch(b, integral_constant<int, 8>(), i) || launch(b, integral_constant<int, 4>(), i) || launch(b, integral_constant<int, 2>(), i) ||
               launch(b, integral_constant<int, 1>(), i);
    };
    interleaved ? with(std::true_type()) : with(std::false_type());
    hip_check(hipGetLastError(), "rope launch");
}

}  // namespace monet
