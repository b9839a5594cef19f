// Activations held in 8 bits between the forward and the backward pass, and the weight gradient of a linear layer from them.
//
// 32 neighbouring columns of a row share a power of two: code = x / 2^e rounded to nearest (ties to even), e the smallest from -126 up
// with max|x| / 2^e < 127.5.  So no code is beyond 127, the error is at most half a step of 2^e (1/128 to 1/255 of the group's maximum),
// and a code times its power is a bf16 number exactly: the weight gradient's products take it as it is.  A group with an infinity or a
// NaN stands for NaN throughout (codes 0, exponent byte 255: 0 times infinity).
//
// Layout: rows of round_up(cols, 32) codes, zero behind the last column, then rows of one exponent byte (e + 127) per group.
#include <initializer_list>

#include "../../include/monet_kernels.h"
#include "gemm_bf16.hpp"
#include "kernels.hpp"

namespace monet {

namespace {

constexpr int GROUP = 32;

int64_t code_ld(int64_t cols) { return (cols + GROUP - 1) / GROUP * GROUP; }

template <class T> __device__ __forceinline__ float value_of(T v);
template <> __device__ __forceinline__ float value_of(float v) { return v; }
template <> __device__ __forceinline__ float value_of(unsigned short v) { return bf16_float(v); }

// eight neighbouring values; `have` of them exist
template <class T>
__device__ __forceinline__ void load8(const T *p, int have, bool vec, float (&v)[8]) {
    if (vec && have >= 8) {
        if constexpr (sizeof(T) == 4) {
            const float4 a = *(const float4 *)p, b = *(const float4 *)(p + 4);
            v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
        } else {
            const uint4 a = *(const uint4 *)p;
            const unsigned w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(w[i] << 16); v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < have ? value_of(p[i]) : 0.f;
    }
}

// a thread takes eight columns, four threads a group
template <class T>
__global__ __launch_bounds__(256) void act8_pack_kernel(const T *__restrict__ x, int64_t ld, int8_t *__restrict__ code, uint8_t *__restrict__ exps,
                                                        int64_t rows, int cols, int per_row, bool vec) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, row = i / per_row;
    if (row >= rows) return;
    const int c = (int)(i - row * per_row) * 8;
    float v[8];
    load8(x + row * ld + c, cols - c, vec, v);
    unsigned top = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(v[j]) & 0x7fffffffu);
    top = max(top, (unsigned)__shfl_xor((int)top, 1));
    top = max(top, (unsigned)__shfl_xor((int)top, 2));
    const bool bad = top >= 0x7f800000u;
    int e = max((int)(top >> 23) - 133, -126);
    if (__uint_as_float(top) * __uint_as_float((unsigned)(127 - e) << 23) >= 127.5f) ++e;
    const float by = __uint_as_float((unsigned)(127 - e) << 23);
    unsigned w[2] = {0, 0};
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int q = bad ? 0 : (int)rintf(v[j] * by);
        w[j / 4] |= (unsigned)(q & 0xff) << (8 * (j % 4));
    }
    *(uint2 *)(code + row * per_row * 8 + c) = make_uint2(w[0], w[1]);
    if (c % GROUP == 0) exps[row * (per_row / 4) + c / GROUP] = bad ? 255 : (uint8_t)(e + 127);
}

template <class T>
__global__ __launch_bounds__(256) void act8_unpack_kernel(const int8_t *__restrict__ code, const uint8_t *__restrict__ exps, T *__restrict__ y, int64_t ld,
                                                          int64_t rows, int cols, int per_row, bool vec) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, row = i / per_row;
    if (row >= rows) return;
    const int c = (int)(i - row * per_row) * 8, have = cols - c;
    if (have <= 0) return;
    const uint2 w = *(const uint2 *)(code + row * per_row * 8 + c);
    const float by = __uint_as_float((unsigned)exps[row * (per_row / 4) + c / GROUP] << 23);
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = (float)(int8_t)((j < 4 ? w.x : w.y) >> (8 * (j % 4))) * by;
    T *p = y + row * ld + c;
    if (vec && have >= 8) {
        if constexpr (sizeof(T) == 4) {
            *(float4 *)p = make_float4(v[0], v[1], v[2], v[3]);
            *(float4 *)(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
        } else *(uint4 *)p = make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < have) {
                if constexpr (sizeof(T) == 4) p[j] = v[j];
                else p[j] = float_bf16(v[j]);
            }
    }
}

// dw[o][c] = sum over rows of dy[row][o] x[row][c]: both operands run across the reduction (DEEP tiles, tile_bf16.hpp).  The codes become
// bf16 on their way to LDS: a byte u = code + 128 to a float, then u 2^e - 128 2^e in one exact multiply-add.  bf16 dy goes in as it is,
// fp32 dy in three pieces (bf16_pieces.hpp), three instructions a product and nothing lost above 2^-110.
struct Act8Shape {
    const int8_t *code;
    const uint8_t *exps;
    const void *dy;
    float *out;
    int64_t rows, range;       // range: elements between the partial results of two ranges
    int cols, outs, ld, tiles_m, tiles_n;
    int64_t chunk;             // rows of a range
    bool vec, vec_out;
};
template <bool F32, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(WM *WN * 64, WM *WN * 64 / 256) void act8_wgrad_kernel(Act8Shape g) {
    constexpr int THREADS = WM * WN * 64, DEPTH = F32 ? 32 : 64, PLANES = F32 ? 3 : 1, MB = BM / WM / 32, NB = BN / WN / 32;
    constexpr int CODES = BM * DEPTH / 16 / THREADS, PIECES = BN * DEPTH / 8 / THREADS;
    constexpr int A_BYTES = BM * DEPTH * 2, B_BYTES = BN * DEPTH * 2;
    __shared__ __attribute__((aligned(16))) char a_lds[2][A_BYTES], b_lds[2][PLANES][B_BYTES];
    int tm, tn;
    gemm_place(g.tiles_m, g.tiles_n, tm, tn);
    const int c0 = tm * BM, o0 = tn * BN, wave = threadIdx.x / 64, wm = (wave / WN) * (BM / WM), wn = (wave % WN) * (BN / WN);
    const int64_t first = blockIdx.y * g.chunk, last = min(g.rows, first + g.chunk);
    GemmFrags<true, BM, MB> fa;
    GemmFrags<true, BN, NB> fb;
    fa.init(wm);
    fb.init(wn);
    floatx16 acc[MB][NB];
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
    uint4 codes[CODES];
    float scale[CODES];
    typedef typename std::conditional<F32, float, unsigned short>::type T;
    float dy[F32 ? PIECES : 1][8];
    uint4 dyw[F32 ? 1 : PIECES];
    auto fetch = [&](int64_t k0) {
#pragma unroll
        for (int i = 0; i < CODES; ++i) {
            const int piece = i * THREADS + threadIdx.x, kr = piece / (BM / 16), c = c0 + piece % (BM / 16) * 16;
            codes[i] = make_uint4(0, 0, 0, 0);
            scale[i] = 0.f;
            if (k0 + kr < last && c < g.ld) {
                codes[i] = *(const uint4 *)(g.code + (k0 + kr) * g.ld + c);
                scale[i] = __uint_as_float((unsigned)g.exps[(k0 + kr) * (g.ld / GROUP) + c / GROUP] << 23);
            }
        }
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int piece = i * THREADS + threadIdx.x, kr = piece / (BN / 8), o = o0 + piece % (BN / 8) * 8;
            const int have = k0 + kr < last ? g.outs - o : 0;
            const T *p = (const T *)g.dy + (k0 + kr) * g.outs + o;
            if constexpr (F32) load8(p, have, g.vec, dy[i]);
            else {
                if (g.vec) dyw[i] = have >= 8 ? *(const uint4 *)p : make_uint4(0, 0, 0, 0);
                else {
                    unsigned w[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) w[j] = (2 * j < have ? p[2 * j] : 0u) | (2 * j + 1 < have ? (unsigned)p[2 * j + 1] << 16 : 0u);
                    dyw[i] = make_uint4(w[0], w[1], w[2], w[3]);
                }
            }
        }
    };
    auto place = [](int kr, int c, int row_bytes) { return kr * row_bytes + ((((c >> 1) ^ (int)deep_turn(kr)) << 1) | (c & 1)) * 16; };
    auto store = [&](int buf) {
#pragma unroll
        for (int i = 0; i < CODES; ++i) {
            const int piece = i * THREADS + threadIdx.x, kr = piece / (BM / 16), c = piece % (BM / 16) * 2;
            const unsigned w[4] = {codes[i].x ^ 0x80808080u, codes[i].y ^ 0x80808080u, codes[i].z ^ 0x80808080u, codes[i].w ^ 0x80808080u};
            const float s = scale[i], mid = -128.f * s;
            unsigned out[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const unsigned b = w[j / 2] >> (16 * (j % 2));
                const float lo = fmaf((float)(b & 0xffu), s, mid), hi = fmaf((float)((b >> 8) & 0xffu), s, mid);
                out[j] = __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
            }
            char *p = a_lds[buf] + place(kr, c, BM * 2);
            *(uint4 *)p = make_uint4(out[0], out[1], out[2], out[3]);
            *(uint4 *)(p + 16) = make_uint4(out[4], out[5], out[6], out[7]);
        }
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int piece = i * THREADS + threadIdx.x, kr = piece / (BN / 8), at = place(kr, piece % (BN / 8), BN * 2);
            if constexpr (F32) {
                unsigned lost = 0;
                const PieceRow r = split_row(dy[i], lost);
                *(bf16x8 *)(b_lds[buf][0] + at) = r.h;
                *(bf16x8 *)(b_lds[buf][1] + at) = r.m;
                *(bf16x8 *)(b_lds[buf][2] + at) = r.l;
            } else *(uint4 *)(b_lds[buf][0] + at) = dyw[i];
        }
    };
    auto work = [&](int buf) {
        const lds_char *a = (const lds_char *)a_lds[buf];
#pragma unroll
        for (int s = 0; s < DEPTH / 16; ++s) {
            bf16x8 x[MB];
#pragma unroll
            for (int i = 0; i < MB; ++i) x[i] = fa.read(a, s, i);
#pragma unroll
            for (int p = 0; p < PLANES; ++p) {
                bf16x8 y[NB];
#pragma unroll
                for (int j = 0; j < NB; ++j) y[j] = fb.read((const lds_char *)b_lds[buf][p], s, j);
#pragma unroll
                for (int i = 0; i < MB; ++i)
#pragma unroll
                    for (int j = 0; j < NB; ++j) acc[i][j] = mfma_bf16(x[i], y[j], acc[i][j]);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    fetch(first);
    store(0);
    __syncthreads();
    int buf = 0;
    for (int64_t k0 = first; k0 < last; k0 += DEPTH, buf ^= 1) {
        fetch(k0 + DEPTH);       // behind the last step: nothing, as zeros
        work(buf);
        store(buf ^ 1);
        __syncthreads();
    }
    const int l = threadIdx.x & 63;
    float *out = g.out + blockIdx.y * g.range;
#pragma unroll
    for (int j = 0; j < NB; ++j) {
        const int o = o0 + wn + 32 * j + (l & 31);
        if (o >= g.outs) continue;
#pragma unroll
        for (int i = 0; i < MB; ++i)
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
                const int c = c0 + wm + 32 * i + result_row(r, l);
                float *p = out + (int64_t)o * g.cols + c;
                if (g.vec_out && c < g.cols) *(float4 *)p = make_float4(acc[i][j][r], acc[i][j][r + 1], acc[i][j][r + 2], acc[i][j][r + 3]);
                else {
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        if (c + q < g.cols) p[q] = acc[i][j][r + q];
                }
            }
    }
}

void check_shape(int64_t rows, int64_t cols) {
    if (rows < 1 || cols < 1 || cols > (1 << 24) || rows > (1ll << 40) / code_ld(cols)) throw KernelError("act8: bad shape");
}
void check_type(int dtype) {
    if (dtype != MONET_F32 && dtype != MONET_BF16) throw KernelError("act8: dtype must be MONET_F32 or MONET_BF16");
}
void check_tensor(const void *p, size_t align) {
    if (!p) throw KernelError("act8: null pointer");
    if ((uintptr_t)p % align) throw KernelError("act8: pointer not aligned");
}

// Results of few tiles cut the reduction over the rows into ranges until every CU has a workgroup, each of at least 256 rows.
struct WgradPlan { int tile, splits; int64_t chunk; };
WgradPlan wgrad_plan(int64_t rows, int cols, int outs) {
    const int tile = gemm_tile(cols, outs);
    const int64_t tiles = ((cols + tile - 1) / tile) * ((int64_t)(outs + tile - 1) / tile);
    const int64_t splits = std::max<int64_t>(1, std::min<int64_t>({512 / tiles, rows / 256, 64}));
    const int64_t chunk = ((rows + splits - 1) / splits + 63) / 64 * 64;
    return {tile, (int)((rows + chunk - 1) / chunk), chunk};
}

}  // namespace

size_t act8_bytes(int64_t rows, int64_t cols) {
    check_shape(rows, cols);
    return (size_t)(rows * (code_ld(cols) / GROUP) * (GROUP + 1));
}

void act8_pack(hipStream_t st, int dtype, const void *x, int64_t ld, void *code, int64_t rows, int64_t cols) {
    check_type(dtype);
    check_shape(rows, cols);
    const int es = dtype == MONET_F32 ? 4 : 2;
    check_tensor(x, es);
    check_tensor(code, 16);
    if (ld < cols) throw KernelError("act8_pack: row stride below the number of columns");
    const int per_row = (int)(code_ld(cols) / 8);
    const int64_t blocks = (rows * per_row + 255) / 256;
    if (blocks > 0x7fffffff) throw KernelError("act8_pack: too many values");
    const bool vec = (uintptr_t)x % 16 == 0 && ld * es % 16 == 0;
    uint8_t *exps = (uint8_t *)code + rows * code_ld(cols);
    if (dtype == MONET_F32)
        hipLaunchKernelGGL((act8_pack_kernel<float>), dim3((unsigned)blocks), dim3(256), 0, st, (const float *)x, ld, (int8_t *)code, exps, rows, (int)cols, per_row, vec);
    else
        hipLaunchKernelGGL((act8_pack_kernel<unsigned short>), dim3((unsigned)blocks), dim3(256), 0, st, (const unsigned short *)x, ld, (int8_t *)code, exps, rows, (int)cols, per_row, vec);
    hip_check(hipGetLastError(), "act8 pack launch");
}

void act8_unpack(hipStream_t st, int dtype, const void *code, void *y, int64_t ld, int64_t rows, int64_t cols) {
    check_type(dtype);
    check_shape(rows, cols);
    const int es = dtype == MONET_F32 ? 4 : 2;
    check_tensor(y, es);
    check_tensor(code, 16);
    if (ld < cols) throw KernelError("act8_unpack: row stride below the number of columns");
    const int per_row = (int)(code_ld(cols) / 8);
    const int64_t blocks = (rows * per_row + 255) / 256;
    if (blocks > 0x7fffffff) throw KernelError("act8_unpack: too many values");
    const bool vec = (uintptr_t)y % 16 == 0 && ld * es % 16 == 0;
    const uint8_t *exps = (const uint8_t *)code + rows * code_ld(cols);
    if (dtype == MONET_F32)
        hipLaunchKernelGGL((act8_unpack_kernel<float>), dim3((unsigned)blocks), dim3(256), 0, st, (const int8_t *)code, exps, (float *)y, ld, rows, (int)cols, per_row, vec);
    else
        hipLaunchKernelGGL((act8_unpack_kernel<unsigned short>), dim3((unsigned)blocks), dim3(256), 0, st, (const int8_t *)code, exps, (unsigned short *)y, ld, rows, (int)cols, per_row, vec);
    hip_check(hipGetLastError(), "act8 unpack launch");
}

size_t act8_wgrad_workspace_bytes(int dtype, int64_t rows, int64_t cols, int64_t outs) {
    check_type(dtype);
    check_shape(rows, cols);
    check_shape(rows, outs);
    const WgradPlan p = wgrad_plan(rows, (int)cols, (int)outs);
    return p.splits > 1 ? (size_t)p.splits * cols * outs * 4 : 0;
}

void act8_wgrad(hipStream_t st, int dtype, const void *code, const void *dy, float *dw, int64_t rows, int64_t cols, int64_t outs, void *ws, size_t ws_bytes) {
    const size_t need = act8_wgrad_workspace_bytes(dtype, rows, cols, outs);
    const WgradPlan p = wgrad_plan(rows, (int)cols, (int)outs);
    const int es = dtype == MONET_F32 ? 4 : 2;
    check_tensor(code, 16);
    check_tensor(dy, es);
    check_tensor(dw, 4);
    if (need && (!ws || ws_bytes < need)) throw KernelError("act8_wgrad: workspace of " + std::to_string(ws_bytes) + " bytes, " + std::to_string(need) + " needed");
    if (need) check_tensor(ws, 16);
    Act8Shape g{};
    g.code = (const int8_t *)code;
    g.ld = (int)code_ld(cols);
    g.exps = (const uint8_t *)code + rows * g.ld;
    g.dy = dy;
    g.out = p.splits > 1 ? (float *)ws : dw;
    g.rows = rows; g.cols = (int)cols; g.outs = (int)outs;
    g.range = cols * outs;
    g.chunk = p.chunk;
    g.tiles_m = (int)((cols + p.tile - 1) / p.tile);
    g.tiles_n = (int)((outs + p.tile - 1) / p.tile);
    g.vec = (uintptr_t)dy % 16 == 0 && outs * es % 16 == 0;
    g.vec_out = (uintptr_t)g.out % 16 == 0 && cols % 4 == 0;
    if ((int64_t)g.tiles_m * g.tiles_n > 0x7fffffff) throw KernelError("act8_wgrad: result too large");
    const dim3 grid(g.tiles_m * g.tiles_n, p.splits);
    if (dtype == MONET_F32) {
        if (p.tile == 256) hipLaunchKernelGGL((act8_wgrad_kernel<true, 256, 256, 2, 4>), grid, dim3(512), 0, st, g);
        else hipLaunchKernelGGL((act8_wgrad_kernel<true, 128, 128, 2, 2>), grid, dim3(256), 0, st, g);
    } else {
        if (p.tile == 256) hipLaunchKernelGGL((act8_wgrad_kernel<false, 256, 256, 2, 4>), grid, dim3(512), 0, st, g);
        else hipLaunchKernelGGL((act8_wgrad_kernel<false, 128, 128, 2, 2>), grid, dim3(256), 0, st, g);
    }
    hip_check(hipGetLastError(), "act8 weight gradient launch");
    if (p.splits > 1) split_reduce(st, (const float *)ws, dw, cols * outs, p.splits, false);
}

}  // namespace monet
