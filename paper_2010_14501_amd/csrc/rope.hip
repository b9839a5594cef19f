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

// A unit of a head: V pairs, two runs of V values that lie `half` (interleaved: V) apart, or up to two neighbouring runs that stay.  A workgroup has
// `at_once` tokens; a thread keeps its unit and its token, with their cosines and sines in registers, and takes every `lanes`-th head, the next
// one's values loaded before this one's are turned.  The angles are computed together, each once for all heads.  Heads and units from two divisions a
// unit instead of a thread, and the angles read from LDS for every unit: 165 us where this takes 124.
template <class T, int V, bool INTERLEAVED>
__global__ __launch_bounds__(256) void rope_kernel(const T *x, T *y, const int32_t *__restrict__ positions, const RopeFreqs f, int64_t tokens, int at_once,
                                                   int lanes, int units, int heads, int dim, int half, int64_t x_ld, int64_t y_ld, float scale, int inverse,
                                                   int add) {
    extern __shared__ float2 table[];       // [token][pair]: cos, sin
    const int64_t t0 = (int64_t)blockIdx.x * at_once;
    const int here = (int)min((int64_t)at_once, tokens - t0), wide = min(256, units - (int)blockIdx.y * 256);
    const unsigned slot = threadIdx.x / (unsigned)wide, token = slot / (unsigned)lanes;
    const int u = blockIdx.y * 256 + threadIdx.x - slot * wide, lane = slot - token * lanes;
    const bool mine = (int)token < here, turns = u * V < half;
    const int at = turns && !INTERLEAVED ? V * u : 2 * V * u, other = turns && !INTERLEAVED ? half : V;
    const bool both = turns || at + 2 * V <= dim;
    const T *from = x + (t0 + token) * x_ld + at;
    T *to = y + (t0 + token) * y_ld + at;
    struct Run { T v[V]; };
    Run a, b;
    const auto load = [&](int h) {
        __builtin_memcpy(&a, from + (int64_t)h * dim, sizeof a);
        if (both) __builtin_memcpy(&b, from + (int64_t)h * dim + other, sizeof b);
    };
    if (mine && lane < heads) load(lane);
    for (unsigned i = threadIdx.x; i < (unsigned)(here * half); i += 256) {
        const unsigned t = i / (unsigned)half, pair = i - t * half;
        float c, s;
        turn((positions ? positions[t0 + t] : (int)(t0 + t)) * f.turns[pair], c, s);
        table[i] = make_float2(c * scale, s * (inverse ? -scale : scale));
    }
    __syncthreads();
    if (!mine) return;
    float2 cs[V];
#pragma unroll
    for (int e = 0; e < V; ++e) cs[e] = turns ? table[token * half + u * V + e] : make_float2(1.f, 0.f);
    for (int h = lane; h < heads; h += lanes) {
        const Run oa = a, ob = b;
        if (h + lanes < heads) load(h + lanes);
        float m[V], n[V];
#pragma unroll
        for (int e = 0; e < V; ++e) {       // pair e: values 2 e and 2 e + 1 of the two runs, or e of each
            const float p = value(INTERLEAVED ? (2 * e < V ? oa.v[2 * e % V] : ob.v[2 * e % V]) : oa.v[e]);
            const float q = value(INTERLEAVED ? (2 * e + 1 < V ? oa.v[(2 * e + 1) % V] : ob.v[(2 * e + 1) % V]) : ob.v[e]);
            m[e] = p * cs[e].x - q * cs[e].y;
            n[e] = p * cs[e].y + q * cs[e].x;
        }
        T *p = to + (int64_t)h * dim;
        Run ra, rb;
        if (add) {
            __builtin_memcpy(&ra, p, sizeof ra);
            if (both) __builtin_memcpy(&rb, p + other, sizeof rb);
        }
#pragma unroll
        for (int e = 0; e < V; ++e) {       // what stays is what it was, whatever lies beside it
            const float lo = INTERLEAVED ? (e % 2 ? n[e / 2] : m[e / 2]) : m[e], hi = INTERLEAVED ? ((e + V) % 2 ? n[(e + V) / 2] : m[(e + V) / 2]) : n[e];
            put(ra.v + e, turns ? lo : value(oa.v[e]), add);
            put(rb.v + e, turns ? hi : value(ob.v[e]), add);
        }
        __builtin_memcpy(p, &ra, sizeof ra);
        if (both) __builtin_memcpy(p + other, &rb, sizeof rb);
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

void rope_check(int64_t tokens, int heads, int head_dim, int rot_dim, float scale) {
    if (tokens < 0 || heads < 1 || head_dim < 1) throw KernelError("rope: bad shape");
    if (rot_dim < 2 || rot_dim % 2 || rot_dim > ROPE_DIM || rot_dim > head_dim)
        throw KernelError("rope: rot_dim must be even, 2 to head_dim and at most " + std::to_string(ROPE_DIM));
    if (tokens >= 1 << 24 || (int64_t)heads * head_dim >= 1 << 24 || head_dim > 1 << 15) throw KernelError("rope: shape too large");
    if (!std::isfinite(scale)) throw KernelError("rope: the scale must be finite");
}

void rope(hipStream_t st, int dtype, const void *x, void *y, const int32_t *positions, const double *freqs, int64_t tokens, int heads, int head_dim,
          int rot_dim, int64_t x_ld, int64_t y_ld, bool interleaved, float scale, bool inverse, bool accumulate) {
    if (dtype != MONET_F32 && dtype != MONET_BF16) throw KernelError("rope: dtype must be MONET_F32 or MONET_BF16");
    rope_check(tokens, heads, head_dim, rot_dim, scale);
    if (!freqs) throw KernelError("rope: null pointer");
    RopeFreqs f;
    for (int i = 0; i < ROPE_DIM / 2; ++i) {
        f.turns[i] = i < rot_dim / 2 ? freqs[i] / (2 * M_PI) : 0;
        if (!std::isfinite(f.turns[i])) throw KernelError("rope: frequencies must be finite");
    }
    if (!tokens) return;
    const int64_t width = (int64_t)heads * head_dim;
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
        const int units = half / V + (x == y ? 0 : (rest / V + 1) / 2), slots = 256 / std::min(units, 256);
        // about two heads to a thread: 16384 tokens, 40 heads, both ways, 124 us in bf16 with 128 wide heads (5.4 TB/s; a plain copy reaches 5.6), 101 with 96
        // wide ones of which 24 turn; three: 127 and 101; six: 134 and 113; fp32 of 96 wide ones, of which 24 turn: two 189, six 218
        const int at_once = (int)std::max<int64_t>(1, std::min<int64_t>({slots, (int64_t)slots * 2 / heads, tokens / 512, 2048 / half}));
        const dim3 grid((unsigned)((tokens + at_once - 1) / at_once), (units + 255) / 256);
        hipLaunchKernelGGL((rope_kernel<T, V, decltype(interleaved_)::value>), grid, dim3(256), at_once * half * sizeof(float2), st, (const T *)x, (T *)y, positions,
                           f, tokens, at_once, slots / at_once, units, heads, head_dim, half, x_ld, y_ld, scale, inverse, accumulate);
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
