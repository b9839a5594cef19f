// Activations held in 8 bits between the forward and the backward pass, and the weight gradient of a linear layer from them.
//
// 32 neighbouring columns of a row share a power of two: code = x / 2^e rounded to nearest (ties to even), e the smallest from -126 up
// with max|x| / 2^e < 127.5.  So no code is beyond 127 and the error is at most half a step of 2^e: 1/127.5 to 1/255 of the group's maximum
// where e > -126, 2^-127 where e = -126, however small the maximum.  A code times its power is a bf16 number exactly: the weight gradient's
// products take it as it is.  A group with an infinity or a NaN stands for NaN throughout (codes 0, exponent byte 255: 0 times infinity).
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

// vectors at any address that their elements may have: the hardware takes 16 bytes from and to there
typedef float float4_any __attribute__((ext_vector_type(4), aligned(4)));
typedef unsigned uint4_any __attribute__((ext_vector_type(4), aligned(2)));

// eight neighbouring values; `have` of them exist
template <class T>
__device__ __forceinline__ void load8(const T *p, int have, float (&v)[8]) {
    if (have >= 8) {
        if constexpr (sizeof(T) == 4) {
            const float4_any a = *(const float4_any *)p, b = *(const float4_any *)(p + 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[4 + i] = b[i]; }
        } else {
            const uint4_any a = *(const uint4_any *)p;
#pragma unroll
            for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(a[i] << 16); v[2 * i + 1] = __uint_as_float(a[i] & 0xffff0000u); }
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < have ? value_of(p[i]) : 0.f;
    }
}

// A thread takes eight columns, four threads a group.  Bound by memory: 16384 x 4096 in fp32, 337 MB, 71 to 78 us (4.3 to 4.8 TB/s), and back 56
// (6.0 TB/s, part of it from the last-level cache).
template <class T>
__global__ __launch_bounds__(256) void act8_pack_kernel(const T *__restrict__ x, int64_t ld, int8_t *__restrict__ code, uint8_t *__restrict__ exps,
                                                        int64_t rows, int cols, int per_row) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, row = i / per_row;
    if (row >= rows) return;
    const int c = (int)(i - row * per_row) * 8;
    float v[8];
    load8(x + row * ld + c, cols - c, v);
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
                                                          int64_t rows, int cols, int per_row) {
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
    if (have >= 8) {
        if constexpr (sizeof(T) == 4) {
            *(float4_any *)p = float4_any{v[0], v[1], v[2], v[3]};
            *(float4_any *)(p + 4) = float4_any{v[4], v[5], v[6], v[7]};
        } else *(uint4_any *)p = uint4_any{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
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
// bf16 on their way to LDS: a signed byte to a float, times 2^e, both exact.  (By way of code + 128 and a multiply-add, as many instructions,
// 128 2^e is infinite in groups that reach 2^127.)  bf16 dy goes in as it is, fp32 dy in three pieces (bf16_pieces.hpp), three instructions a
// product and nothing lost above 2^-110.  128 x 128 results to a workgroup of four waves, two workgroups a CU.  One of these has its
// conversions and its barrier while the other one multiplies; that, not memory, bounds it:
// 4096 x 2048 x 1024 37 us in bf16 (470 TFLOP/s), 65 in fp32 (264, times three).
struct Act8Shape {
    const int8_t *code;
    const uint8_t *exps;
    const void *dy;
    float *out;
    int64_t rows, range;       // range: elements between the partial results of two ranges
    int cols, outs, ld, tiles_m, tiles_n;
    int64_t chunk;             // rows of a range
    bool vec_out;
};
// WORDS: dy's rows begin on words, which a buffer's loads need.
template <bool F32, bool WORDS, int BM, int BN, int WM, int WN>
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
    // A step's operands on their way.  What lies behind a row's end, the next row's beginning, only reaches results that are not stored; rows
    // behind the range arrive as zeros.
    struct Held {
        uintx4 codes[CODES], dy[PIECES][F32 ? 2 : 1];
        unsigned exps[CODES];
    } held0, held1;
    typedef typename std::conditional<F32, float, unsigned short>::type T;
    unsigned code_at[CODES], exp_at[CODES], dy_at[PIECES];
#pragma unroll
    for (int i = 0; i < CODES; ++i) {
        const unsigned piece = i * THREADS + threadIdx.x, kr = piece / (BM / 16), c = c0 + piece % (BM / 16) * 16;
        code_at[i] = kr * g.ld + c;
        exp_at[i] = kr * (g.ld / GROUP) + c / GROUP;
    }
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
        const unsigned piece = i * THREADS + threadIdx.x, kr = piece / (BN / 8), o = o0 + piece % (BN / 8) * 8;
        dy_at[i] = (kr * g.outs + o) * sizeof(T);
    }
    auto fetch = [&](Held &h, int64_t k0) {
        const unsigned left = (unsigned)max(min(last - k0, (int64_t)DEPTH), (int64_t)0);
        const __amdgpu_buffer_rsrc_t rc = buffer_of(g.code + k0 * g.ld, left * g.ld), re = buffer_of(g.exps + k0 * (g.ld / GROUP), left * (g.ld / GROUP)),
                                     rd = buffer_of((const T *)g.dy + k0 * g.outs, left * g.outs * (unsigned)sizeof(T));
#pragma unroll
        for (int i = 0; i < CODES; ++i) {
            h.codes[i] = __builtin_bit_cast(uintx4, __builtin_amdgcn_raw_buffer_load_b128(rc, code_at[i], 0, 0));
            h.exps[i] = __builtin_amdgcn_raw_buffer_load_b8(re, exp_at[i], 0, 0);
        }
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            if constexpr (WORDS) {
#pragma unroll
                for (int j = 0; j < (F32 ? 2 : 1); ++j) h.dy[i][j] = __builtin_bit_cast(uintx4, __builtin_amdgcn_raw_buffer_load_b128(rd, dy_at[i] + 16 * j, 0, 0));
            } else {
                const int piece = i * THREADS + threadIdx.x, kr = piece / (BN / 8), o = o0 + piece % (BN / 8) * 8, have = kr < (int)left ? g.outs - o : 0;
                const unsigned short *p = (const unsigned short *)g.dy + (k0 + kr) * g.outs + o;
                if (have >= 8) h.dy[i][0] = *(const uint4_any *)p;
                else {
#pragma unroll
                    for (int j = 0; j < 4; ++j) h.dy[i][0][j] = (2 * j < have ? p[2 * j] : 0u) | (2 * j + 1 < have ? (unsigned)p[2 * j + 1] << 16 : 0u);
                }
            }
        }
    };
    auto place = [](int kr, int c, int row_bytes) { return kr * row_bytes + ((((c >> 1) ^ (int)deep_turn(kr)) << 1) | (c & 1)) * 16; };
    auto store = [&](const Held &h, int buf) {
#pragma unroll
        for (int i = 0; i < CODES; ++i) {
            const int piece = i * THREADS + threadIdx.x, kr = piece / (BM / 16), c = piece % (BM / 16) * 2;
            const float s = __uint_as_float(h.exps[i] << 23);
            unsigned out[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const unsigned b = h.codes[i][j / 2] >> (16 * (j % 2));
                const float lo = (float)(int8_t)b * s, hi = (float)(int8_t)(b >> 8) * s;
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
                float v[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = __uint_as_float(h.dy[i][j / 4][j % 4]);
                const PieceRow r = split_row(v, lost);
                *(bf16x8 *)(b_lds[buf][0] + at) = r.h;
                *(bf16x8 *)(b_lds[buf][1] + at) = r.m;
                *(bf16x8 *)(b_lds[buf][2] + at) = r.l;
            } else *(uintx4 *)(b_lds[buf][0] + at) = h.dy[i][0];
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
    // two steps ahead of the products: a step takes less time than its loads (5003 rows, 1000 columns, 777 outputs, fp32: 46 us, one step ahead 52)
    fetch(held0, first);
    fetch(held1, first + DEPTH);
    store(held0, 0);
    __syncthreads();
    for (int64_t k0 = first; k0 < last; k0 += 2 * DEPTH) {
        fetch(held0, k0 + 2 * DEPTH);
        work(0);
        store(held1, 1);
        __syncthreads();
        fetch(held1, k0 + 3 * DEPTH);
        if (k0 + DEPTH < last) work(1);
        store(held0, 0);
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

// dy as the GEMM takes it: rows of `ld` values, zero behind the last one; fp32 in three planes of pieces.  Eight values a thread.
template <class T>
__global__ __launch_bounds__(256) void act8_planes_kernel(const T *__restrict__ dy, unsigned short *__restrict__ out, int64_t rows, int outs, int ld) {
    const int per_row = ld / 8;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, row = i / per_row, plane = rows * ld;
    if (row >= rows) return;
    const int o = (int)(i - row * per_row) * 8;
    float v[8];
    load8(dy + row * outs + o, outs - o, v);
    unsigned short *p = out + row * ld + o;
    if constexpr (sizeof(T) == 4) {
        unsigned lost = 0;
        const PieceRow r = split_row(v, lost);
        *(bf16x8 *)p = r.h;
        *(bf16x8 *)(p + plane) = r.m;
        *(bf16x8 *)(p + 2 * plane) = r.l;
    } else *(uint4 *)p = make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
}

// out[n][m], one range's partial result behind the other
struct RangeEpilogue {
    float *out;
    int64_t range;
    int add;
    bool vec;
    template <int MB, int NB>
    __device__ __forceinline__ void operator()(floatx16 (&acc)[MB][NB], int m0, int n0, int m, int n) const {
        const int l = threadIdx.x & 63;
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            const int o = n0 + 32 * j + (l & 31);
            if (o >= n) continue;
#pragma unroll
            for (int i = 0; i < MB; ++i)
#pragma unroll
                for (int r = 0; r < 16; r += 4) {
                    const int c = m0 + 32 * i + result_row(r, l);
                    float *p = out + blockIdx.y * range + (int64_t)o * m + c;
                    if (vec) {
                        if (c >= m) continue;
                        float4 v = make_float4(acc[i][j][r], acc[i][j][r + 1], acc[i][j][r + 2], acc[i][j][r + 3]);
                        if (add) { const float4 w = *(const float4 *)p; v.x += w.x; v.y += w.y; v.z += w.z; v.w += w.w; }
                        *(float4 *)p = v;
                    } else {
#pragma unroll
                        for (int q = 0; q < 4; ++q)
                            if (c + q < m) p[q] = acc[i][j][r + q] + (add ? p[q] : 0.f);
                    }
                }
        }
    }
};

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

int64_t up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }

// Two forms.  Direct: one kernel from codes and dy, few launches.  Expanded: the codes as bf16 and dy's planes in the workspace, some rows
// (a turn) at a time, and the GEMM, whose operands then need no register on their way.  Both cut the reduction over the rows into
// ranges where the result has few tiles, until every CU has work, of at least 256 rows each; the ranges' results are added in order.
// Measured, expanded and direct: bf16 8192 x 4096 x 4096 256 and 406 us (1.08 PFLOP/s), 8192 x 2048 x 2048 100 and 110, 4096 x 2048 x 1024
// 47 and 40, 1024 x 512 x 512 15 and 12; fp32 (three products each) 8192 x 4096 x 4096 726 and 824, 16384 x 4096 x 1024 460 and 422,
// 4096 x 1024 x 1024 61 and 42.  So bf16 expands from 40 GFLOP on and fp32 from 200.  The expanded form is bound by the matrix instructions'
// power, the direct one by the conversions and barriers between them.
struct WgradPlan {
    bool expanded, copy;       // copy: dy goes through the workspace (fp32, or rows that are no multiple of 16 bytes)
    int tile, splits, ld, ldo, planes;
    int64_t turn, chunk;       // rows of a turn, of a range
    int64_t code_bytes, dy_bytes, part_bytes;
    int64_t bytes() const { return code_bytes + dy_bytes + part_bytes; }
};
constexpr int64_t ACT8_TURN_BYTES = 256ll << 20;
WgradPlan wgrad_plan(int dtype, int64_t rows, int cols, int outs, bool aligned) {
    WgradPlan p{};
    p.ld = (int)code_ld(cols);
    p.expanded = 2.0 * rows * cols * outs >= (dtype == MONET_F32 ? 2e11 : 4e10) && std::max<int64_t>(p.ld, up(outs, 8)) < GEMM_MOST_LD;
    p.tile = p.expanded ? gemm_tile(cols, outs) : 128;
    p.planes = dtype == MONET_F32 ? 3 : 1;
    p.copy = dtype == MONET_F32 || outs % 8 || !aligned;
    p.ldo = p.copy ? (int)up(outs, 8) : outs;
    p.turn = rows;
    if (p.expanded) {
        const int64_t per_row = 2 * (p.ld + p.planes * up(outs, 8));      // as if dy were copied: turns and ranges do not depend on where it lies
        const int64_t turns = (rows * per_row + ACT8_TURN_BYTES - 1) / ACT8_TURN_BYTES;
        p.turn = up((rows + turns - 1) / turns, 64);
        const int64_t held = std::min(p.turn, rows);
        p.code_bytes = up(held * p.ld * 2, 256);
        p.dy_bytes = p.copy ? up(held * p.ldo * 2 * p.planes, 256) : 0;
    }
    const int64_t tiles = ((cols + p.tile - 1) / p.tile) * ((int64_t)(outs + p.tile - 1) / p.tile), first = std::min(p.turn, rows);
    const int64_t splits = std::max<int64_t>(1, std::min<int64_t>({(p.tile == 256 ? 256 : 512) / tiles, first / 256, 64}));
    p.chunk = up((first + splits - 1) / splits, 64);
    p.splits = (int)((first + p.chunk - 1) / p.chunk);
    p.part_bytes = p.splits > 1 ? up((int64_t)p.splits * cols * outs * 4, 256) : 0;
    if (p.expanded ? !gemm_fits(cols, outs, p.splits, p.ld, up(outs, 8)) : tiles >= 1 << 24) throw KernelError("act8_wgrad: result too large");
    return p;
}

}  // namespace

// a launch of eight values a thread takes less than 2^24 workgroups
void act8_check_values(int64_t rows, int64_t cols) {
    check_shape(rows, cols);
    if ((rows * (code_ld(cols) / 8) + 255) / 256 >= 1 << 24) throw KernelError("act8: too many values");
}

size_t act8_bytes(int64_t rows, int64_t cols) {
    act8_check_values(rows, cols);
    return (size_t)(rows * (code_ld(cols) / GROUP) * (GROUP + 1));
}

void act8_pack(hipStream_t st, int dtype, const void *x, int64_t ld, void *code, int64_t rows, int64_t cols) {
    check_type(dtype);
    act8_check_values(rows, cols);
    const int es = dtype == MONET_F32 ? 4 : 2;
    check_tensor(x, es);
    check_tensor(code, 16);
    if (ld < cols) throw KernelError("act8_pack: row stride below the number of columns");
    const int per_row = (int)(code_ld(cols) / 8);
    const int64_t blocks = (rows * per_row + 255) / 256;
    uint8_t *exps = (uint8_t *)code + rows * code_ld(cols);
    if (dtype == MONET_F32)
        hipLaunchKernelGGL((act8_pack_kernel<float>), dim3((unsigned)blocks), dim3(256), 0, st, (const float *)x, ld, (int8_t *)code, exps, rows, (int)cols, per_row);
    else
        hipLaunchKernelGGL((act8_pack_kernel<unsigned short>), dim3((unsigned)blocks), dim3(256), 0, st, (const unsigned short *)x, ld, (int8_t *)code, exps, rows, (int)cols, per_row);
    hip_check(hipGetLastError(), "act8 pack launch");
}

void act8_unpack(hipStream_t st, int dtype, const void *code, void *y, int64_t ld, int64_t rows, int64_t cols) {
    check_type(dtype);
    act8_check_values(rows, cols);
    const int es = dtype == MONET_F32 ? 4 : 2;
    check_tensor(y, es);
    check_tensor(code, 16);
    if (ld < cols) throw KernelError("act8_unpack: row stride below the number of columns");
    const int per_row = (int)(code_ld(cols) / 8);
    const int64_t blocks = (rows * per_row + 255) / 256;
    const uint8_t *exps = (const uint8_t *)code + rows * code_ld(cols);
    if (dtype == MONET_F32)
        hipLaunchKernelGGL((act8_unpack_kernel<float>), dim3((unsigned)blocks), dim3(256), 0, st, (const int8_t *)code, exps, (float *)y, ld, rows, (int)cols, per_row);
    else
        hipLaunchKernelGGL((act8_unpack_kernel<unsigned short>), dim3((unsigned)blocks), dim3(256), 0, st, (const int8_t *)code, exps, (unsigned short *)y, ld, rows, (int)cols, per_row);
    hip_check(hipGetLastError(), "act8 unpack launch");
}

size_t act8_wgrad_workspace_bytes(int dtype, int64_t rows, int64_t cols, int64_t outs) {
    check_type(dtype);
    check_shape(rows, cols);
    check_shape(rows, outs);
    // rows of dy that begin off a 16-byte boundary are copied: room for that in any case
    return (size_t)wgrad_plan(dtype, rows, (int)cols, (int)outs, false).bytes();
}

void act8_wgrad(hipStream_t st, int dtype, const void *code, const void *dy, float *dw, int64_t rows, int64_t cols, int64_t outs, void *ws, size_t ws_bytes) {
    const size_t need = act8_wgrad_workspace_bytes(dtype, rows, cols, outs);
    const int es = dtype == MONET_F32 ? 4 : 2;
    check_tensor(code, 16);
    check_tensor(dy, es);
    check_tensor(dw, 4);
    if (need && (!ws || ws_bytes < need)) throw KernelError("act8_wgrad: workspace of " + std::to_string(ws_bytes) + " bytes, " + std::to_string(need) + " needed");
    if (need) check_tensor(ws, 256);
    const WgradPlan p = wgrad_plan(dtype, rows, (int)cols, (int)outs, (uintptr_t)dy % 16 == 0);
    float *parts = (float *)ws;
    char *held = (char *)ws + p.part_bytes;
    float *out = p.splits > 1 ? parts : dw;
    const bool vec_out = (uintptr_t)out % 16 == 0 && cols % 4 == 0;
    const int8_t *codes = (const int8_t *)code;
    const uint8_t *exps = (const uint8_t *)code + rows * p.ld;
    if (p.expanded) {
        unsigned short *x = (unsigned short *)held, *planes = (unsigned short *)(held + p.code_bytes);
        for (int64_t row = 0; row < rows; row += p.turn) {
            const int64_t n = std::min(p.turn, rows - row);
            const int per_row = p.ld / 8;
            hipLaunchKernelGGL((act8_unpack_kernel<unsigned short>), dim3((unsigned)((n * per_row + 255) / 256)), dim3(256), 0, st, codes + row * p.ld,
                               exps + row * (p.ld / GROUP), x, (int64_t)p.ld, n, p.ld, per_row);
            hip_check(hipGetLastError(), "act8 expand launch");
            const char *src = (const char *)dy + row * outs * es;
            if (p.copy) {
                const dim3 grid((unsigned)((n * (p.ldo / 8) + 255) / 256));
                if (dtype == MONET_F32) hipLaunchKernelGGL((act8_planes_kernel<float>), grid, dim3(256), 0, st, (const float *)src, planes, n, (int)outs, p.ldo);
                else hipLaunchKernelGGL((act8_planes_kernel<unsigned short>), grid, dim3(256), 0, st, (const unsigned short *)src, planes, n, (int)outs, p.ldo);
                hip_check(hipGetLastError(), "act8 planes launch");
            }
            GemmShape g{};
            g.a = x; g.lda = p.ld;
            g.b = p.copy ? planes : (const unsigned short *)src; g.ldb = p.ldo;
            g.m = (int)cols; g.n = (int)outs; g.k = (int)n;
            g.chunk = (int)p.chunk; g.splits = (int)((n + p.chunk - 1) / p.chunk);
            g.planes = p.planes; g.b_plane = n * p.ldo;
            gemm_bf16<true, true>(st, g, RangeEpilogue{out, cols * outs, row > 0, vec_out}, "act8 weight gradient launch");
        }
    } else {
        Act8Shape g{};
        g.code = codes;
        g.ld = p.ld;
        g.exps = exps;
        g.dy = dy;
        g.out = out;
        g.rows = rows; g.cols = (int)cols; g.outs = (int)outs;
        g.range = cols * outs;
        g.chunk = p.chunk;
        g.tiles_m = (int)((cols + 127) / 128);
        g.tiles_n = (int)((outs + 127) / 128);
        g.vec_out = vec_out;
        const dim3 grid(g.tiles_m * g.tiles_n, p.splits);
        if (dtype == MONET_F32) hipLaunchKernelGGL((act8_wgrad_kernel<true, true, 128, 128, 2, 2>), grid, dim3(256), 0, st, g);
        else if ((uintptr_t)dy % 4 == 0 && outs % 2 == 0) hipLaunchKernelGGL((act8_wgrad_kernel<false, true, 128, 128, 2, 2>), grid, dim3(256), 0, st, g);
        else hipLaunchKernelGGL((act8_wgrad_kernel<false, false, 128, 128, 2, 2>), grid, dim3(256), 0, st, g);
        hip_check(hipGetLastError(), "act8 weight gradient launch");
    }
    if (p.splits > 1) split_reduce(st, parts, dw, cols * outs, p.splits, false);
}

}  // namespace monet
