// C = A B^T on bf16 operands with fp32 sums: the products of the vocabulary loss, and large weight gradients of 8-bit inputs.
//
// The result's rows (m) are the index that is contiguous in memory, its columns (n) the other one, since a lane of the matrix
// instruction holds four neighbouring rows of one column.  Either operand may run along the reduction (WIDE: [row][k]) or across it
// (DEEP: [k][row]); both reach LDS in 16-byte copies that pass no register and are read there without conflicts (tile_bf16.hpp).
//
// Bound by the matrix instructions under the power limit: they alone, from registers, reach 1.4 PFLOP/s in this loop (the clock falls), 8192 x 8192 x
// 4096 0.96 to 1.02, the loss's products of 8192 x 4096 x 131072 1.19 to 1.27 (MFMA pipes busy 60 % of the cycles).  Tried without a gain: operands
// of the next step read early, wave priorities, four stages of 32 indices, copies through registers, four waves of 128 x 128.
#pragma once
#include "kernels.hpp"
#include "tile_bf16.hpp"

namespace monet {

struct GemmShape {
    const unsigned short *a, *b;
    int64_t lda, ldb;       // elements between rows (WIDE) or reduction indices (DEEP); a multiple of 8, below 2^23
    int m, n, k;            // a row of a WIDE operand is zero from k to the next multiple of 8, where a DEEP one's rows end is no matter
    int tiles_m, tiles_n;
    int splits, chunk;      // ranges of the reduction (grid y), `chunk` indices each, a multiple of GEMM_DEPTH
    int planes = 1;         // b is the sum of so many matrices, `b_plane` elements apart (a float's bf16 pieces, bf16_pieces.hpp)
    int64_t b_plane = 0;
};
constexpr int GEMM_DEPTH = 64;      // reduction indices of a step

// one operand's tile of ROWS rows by 64 reduction indices in LDS
template <bool DEEP, int ROWS, int THREADS>
struct GemmTile {
    static constexpr int BYTES = ROWS * GEMM_DEPTH * 2;
    static constexpr int COPIES = BYTES / (THREADS * 16);
    static constexpr int PAIRS = ROWS / 16;       // 32-byte pairs in a row of a deep tile
    unsigned off[COPIES];
    __amdgpu_buffer_rsrc_t whole;                 // WIDE: the tile's rows, the reduction by the scalar offset
    const unsigned short *base;
    int64_t ld;
    int rows, k;
    unsigned whole_bytes;
    __device__ __forceinline__ void init(const unsigned short *p, int64_t ld_, int row0, int rows_all, int k_) {
        ld = ld_; k = k_;
        rows = (min(ROWS, rows_all - row0) + 7) & ~7;
        base = p + (DEEP ? (int64_t)row0 : row0 * ld);
        const int t = threadIdx.x;
#pragma unroll
        for (int i = 0; i < COPIES; ++i) {
            const unsigned piece = i * THREADS + t;
            if (DEEP) {
                const unsigned kr = piece / (2 * PAIRS), c = piece % (2 * PAIRS);
                off[i] = kr * (unsigned)ld * 2 + ((((c >> 1) ^ deep_turn(kr)) << 1) | (c & 1)) * 16;
            } else {
                const unsigned row = piece / 8, c = (piece % 8) ^ wide_turn(row);
                off[i] = row * (unsigned)ld * 2 + c * 16;
            }
        }
        if (!DEEP) {
            whole_bytes = (unsigned)((min(ROWS, rows_all - row0) - 1) * ld + ((k + 7) & ~7)) * 2;
            whole = buffer_of(base, whole_bytes);
        }
    }
    __device__ __forceinline__ void move(int64_t elements) {
        base += elements;
        if (!DEEP) whole = buffer_of(base, whole_bytes);
    }
    __device__ __forceinline__ void copy(lds_char *lds, int k0) const {
        const int wave = threadIdx.x / 64;
        __amdgpu_buffer_rsrc_t r = whole;
        if (DEEP) r = buffer_of(base + k0 * ld, k0 < k ? (unsigned)((min(GEMM_DEPTH, k - k0) - 1) * ld + rows) * 2 : 0u);
#pragma unroll
        for (int i = 0; i < COPIES; ++i) {
            lds_char *to = lds + (i * THREADS + wave * 64) * 16;
            if (DEEP) copy_to_lds(r, to, off[i], 0);
            else {
                const unsigned piece = i * THREADS + threadIdx.x;
                const unsigned kk = ((piece % 8) ^ wide_turn(piece / 8)) * 8;
                copy_to_lds(r, to, k0 + (int)kk < k ? off[i] : BUFFER_ABSENT, k0 * 2);
            }
        }
    }
};

// the fragments of `BLOCKS` x 32 rows from row `first` on
template <bool DEEP, int ROWS, int BLOCKS>
struct GemmFrags {
    unsigned at[DEEP ? BLOCKS : 4];
    __device__ __forceinline__ void init(int first) {
        const unsigned l = threadIdx.x & 63;
        if (DEEP) {
            const unsigned kr = 8 * (l >> 5) + ((l & 15) >> 2);
#pragma unroll
            for (int b = 0; b < BLOCKS; ++b)
                at[b] = kr * ROWS * 2 + ((first / 16 + 2 * b + ((l >> 4) & 1)) ^ deep_turn(kr)) * 32 + (l & 3) * 8;
        } else {
            const unsigned row = first + (l & 31);
#pragma unroll
            for (int s = 0; s < 4; ++s) at[s] = row * 128 + (((2 * s + (l >> 5)) ^ wide_turn(row)) << 4);
        }
    }
    __device__ __forceinline__ bf16x8 read(const lds_char *lds, int s, int b) const {
        if (DEEP) {
            const lds_char *p = lds + at[DEEP ? b : 0] + s * 16 * ROWS * 2;
            return join(read_turned(p), read_turned(p + 4 * ROWS * 2));
        }
        return read_wide(lds + at[DEEP ? 0 : s] + b * 32 * 128);
    }
};

// Which tile a workgroup works on: each XCD (workgroups go round them in turn) takes a connected range of the tiles, walked in strips
// of four columns, so that the 32 tiles it holds at a time share operands in its own L2.
__device__ __forceinline__ void gemm_place(int tiles_m, int tiles_n, int &tm, int &tn) {
    const int all = tiles_m * tiles_n, x = blockIdx.x % 8, y = blockIdx.x / 8;
    const int t = x * (all / 8) + min(x, all % 8) + y;
    const int strip = t / (4 * tiles_m), in = t - strip * 4 * tiles_m, width = min(4, tiles_n - 4 * strip);
    tm = in / width;
    tn = 4 * strip + in % width;
}

// WM x WN waves of (BM / WM) x (BN / WN) results each; two tiles per operand in LDS, the next one on its way while this one is used.
// epi(acc, m0, n0): the wave's results, MB x NB blocks of 32 x 32 from row m0 and column n0 on.
template <int BM, int BN, int WM, int WN, bool A_DEEP, bool B_DEEP, class Epi>
__global__ __launch_bounds__(WM *WN * 64, WM *WN * 64 / 256) void gemm_bf16_kernel(GemmShape g, Epi epi) {
    constexpr int THREADS = WM * WN * 64, MB = BM / WM / 32, NB = BN / WN / 32;
    __shared__ __attribute__((aligned(16))) char a0[BM * GEMM_DEPTH * 2], a1[BM * GEMM_DEPTH * 2], b0[BN * GEMM_DEPTH * 2], b1[BN * GEMM_DEPTH * 2];
    int tm, tn;
    gemm_place(g.tiles_m, g.tiles_n, tm, tn);
    GemmTile<A_DEEP, BM, THREADS> ta;
    GemmTile<B_DEEP, BN, THREADS> tb;
    const int last = min(g.k, (int)(blockIdx.y + 1) * g.chunk);
    ta.init(g.a, g.lda, tm * BM, g.m, last);
    tb.init(g.b, g.ldb, tn * BN, g.n, last);
    const int wave = threadIdx.x / 64, wm = (wave / WN) * (BM / WM), wn = (wave % WN) * (BN / WN);
    GemmFrags<A_DEEP, BM, MB> fa;
    GemmFrags<B_DEEP, BN, NB> fb;
    fa.init(wm);
    fb.init(wn);
    floatx16 acc[MB][NB];
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
    auto work = [&](const lds_char *a, const lds_char *b) {
#pragma unroll
        for (int s = 0; s < GEMM_DEPTH / 16; ++s) {
            bf16x8 x[MB], y[NB];
#pragma unroll
            for (int i = 0; i < MB; ++i) x[i] = fa.read(a, s, i);
#pragma unroll
            for (int j = 0; j < NB; ++j) y[j] = fb.read(b, s, j);
#pragma unroll
            for (int i = 0; i < MB; ++i)
#pragma unroll
                for (int j = 0; j < NB; ++j) acc[i][j] = mfma_bf16(x[i], y[j], acc[i][j]);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    lds_char *la0 = (lds_char *)a0, *la1 = (lds_char *)a1, *lb0 = (lds_char *)b0, *lb1 = (lds_char *)b1;
    const int first = blockIdx.y * g.chunk, each = (last - first + GEMM_DEPTH - 1) / GEMM_DEPTH, steps = each * g.planes;
    // the next step's tiles, plane by plane; a step behind the last one is copied as zeros
    int at = 0, left = g.planes;
    auto fetch = [&](lds_char *a, lds_char *b) {
        if (at == each && left > 1) { at = 0; --left; tb.move(g.b_plane); }
        ta.copy(a, at < each ? first + at * GEMM_DEPTH : last);
        tb.copy(b, at < each ? first + at * GEMM_DEPTH : last);
        ++at;
    };
    fetch(la0, lb0);
    for (int step = 0; step < steps; step += 2) {       // two steps a turn
        copies_arrived();
        fetch(la1, lb1);
        work(la0, lb0);
        copies_arrived();
        fetch(la0, lb0);
        work(la1, lb1);
    }
    copies_arrived();
    epi(acc, tm * BM + wm, tn * BN + wn, g.m, g.n);
}

constexpr int64_t GEMM_MOST_LD = 1 << 23;      // row strides are below this: 256 rows in 32 bits of a buffer's offset

// Tiles of 256 x 256 (8 waves) where they give every CU one, of 128 x 128 (4 waves, two workgroups a CU) otherwise.
inline int gemm_tile(int64_t m, int64_t n, int splits = 1) { return ((m + 255) / 256) * ((n + 255) / 256) * splits >= 256 ? 256 : 128; }
// Whether a launch takes so many tiles (less than 2^32 threads) and the addresses such strides.
inline bool gemm_fits(int64_t m, int64_t n, int splits, int64_t lda, int64_t ldb) {
    const int64_t b = gemm_tile(m, n, splits), tiles = ((m + b - 1) / b) * ((n + b - 1) / b);
    return lda < GEMM_MOST_LD && ldb < GEMM_MOST_LD && lda % 8 == 0 && ldb % 8 == 0 && tiles < (b == 256 ? 1 << 23 : 1 << 24);
}
template <bool A_DEEP, bool B_DEEP, class Epi>
void gemm_bf16(hipStream_t st, GemmShape g, const Epi &epi, const char *what) {
    if (!gemm_fits(g.m, g.n, g.splits, g.lda, g.ldb)) throw KernelError(std::string(what) + ": operand too large");
    const int b = gemm_tile(g.m, g.n, g.splits);
    g.tiles_m = (g.m + b - 1) / b;
    g.tiles_n = (g.n + b - 1) / b;
    const dim3 grid(g.tiles_m * g.tiles_n, g.splits);
    if (b == 256) hipLaunchKernelGGL((gemm_bf16_kernel<256, 256, 2, 4, A_DEEP, B_DEEP, Epi>), grid, dim3(512), 0, st, g, epi);
    else hipLaunchKernelGGL((gemm_bf16_kernel<128, 128, 2, 2, A_DEEP, B_DEEP, Epi>), grid, dim3(256), 0, st, g, epi);
    hip_check(hipGetLastError(), what);
}

}  // namespace monet
