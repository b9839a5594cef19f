// Softmax cross entropy of a linear layer over a large vocabulary, in pieces of the vocabulary: the logits
//   l[t][v] = x[t] . w[v]
// are never kept.  Forward: lse[t] = log sum_v exp l[t][v], loss = mean over the rows that have a label of lse[t] - l[t][label].
// Backward: dl[t][v] = (exp(l[t][v] - lse[t]) - [v == label]) / count, dx = dl w, dw = dl^T x, one piece of dl at a time.
//
// bf16: three matrix products on the bf16 matrix cores (gemm_bf16.hpp).  The first one's epilogue keeps a maximum and a sum of
// exponentials per row and 64 or 128 logits (forward) or writes count * dl, rounded to bf16 (backward: it is the operand of two bf16
// products whose results are rounded to bf16 themselves; the rounding, at most 2^-8 of a value, averages out over the sums.  1 / count
// comes in behind the products: the label's entries p - 1 are near -1 and would otherwise all be rounded the same way).  Sums are fp32.
// fp32: the convolution kernels' products, a piece of logits in the workspace at a time; with few rows two of them on the vector units.
#include <initializer_list>
#include <type_traits>
#include <vector>

#include "../../include/monet_kernels.h"
#include "gemm_bf16.hpp"
#include "kernels.hpp"

namespace monet {

namespace {

constexpr float LOG2E = 1.44269504088896340736f;
__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * LOG2E); }

// Maximum and sum of a set of logits: nothing: (-inf, 0); one infinite: (FLT_MAX, inf), which stays so whatever joins it.
struct Soft { float m, s; };
__device__ __forceinline__ Soft soft_join(Soft a, Soft b) {
    const float m = fmaxf(a.m, b.m);
    if (m == -INFINITY) return {m, a.s + b.s};
    return {m, (a.m == -INFINITY ? a.s : a.s * exp_of(a.m - m)) + (b.m == -INFINITY ? b.s : b.s * exp_of(b.m - m))};
}

// rows of the result are vocabulary entries, columns tokens: a lane has 16 * MB logits of each of its NB tokens
struct CeStatsEpilogue {
    const int32_t *labels;
    float2 *part;           // [vocab / (32 MB)][rows]: a wave's rows together
    float *hit;             // the label's logit
    int rows, vocab;
    template <int MB, int NB>
    __device__ __forceinline__ void operator()(floatx16 (&acc)[MB][NB], int m0, int n0, int, int) const {
        static_assert(MB == 4 || MB == 2, "");
        const int l = threadIdx.x & 63;
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            const int t = n0 + 32 * j + (l & 31);
            const int label = t < rows ? labels[t] : -1;
            float top = -INFINITY, mine = 0.f;
            bool found = false;
#pragma unroll
            for (int i = 0; i < MB; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int v = m0 + 32 * i + result_row(r, l);
                    if (v >= vocab) acc[i][j][r] = -INFINITY;
                    if (v == label) { mine = acc[i][j][r]; found = true; }
                    top = fmaxf(top, acc[i][j][r]);
                }
            if (found && label < vocab) hit[t] = mine;
            top = fmaxf(top, __shfl_xor(top, 32));
            const float base = top == -INFINITY ? 0.f : fminf(top, 3.4028235e38f);
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < MB; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) sum += exp_of(acc[i][j][r] - base);
            sum += __shfl_xor(sum, 32);
            if (top == INFINITY) { top = 3.4028235e38f; sum = INFINITY; }
            if (l < 32 && t < rows && m0 < vocab) part[(int64_t)(m0 / (32 * MB)) * rows + t] = make_float2(top, sum);
        }
    }
};

// count * dl[t][v - v0]; columns behind the vocabulary are zero up to the row's end
struct CeGradEpilogue {
    const int32_t *labels;
    const float *lse;
    unsigned short *dl;
    int64_t ld;
    int rows, piece, v0, vocab;      // `piece` logits from v0 on
    template <int MB, int NB>
    __device__ __forceinline__ void operator()(floatx16 (&acc)[MB][NB], int m0, int n0, int, int) const {
        const int l = threadIdx.x & 63;
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            const int t = n0 + 32 * j + (l & 31);
            if (t >= rows) continue;
            const int label = labels[t];
            const bool has = (unsigned)label < (unsigned)vocab;
            const float ls = lse[t];
            unsigned short *row = dl + t * ld + m0;
#pragma unroll
            for (int i = 0; i < MB; ++i)
#pragma unroll
                for (int r = 0; r < 16; r += 4) {
                    float d[4];
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const int v = m0 + 32 * i + result_row(r + q, l);
                        const float p = exp_of(acc[i][j][r + q] - ls);
                        d[q] = has && v < piece ? p - (v0 + v == label ? 1.f : 0.f) : 0.f;
                    }
                    if (m0 + 32 * i + result_row(r, l) < ld)
                        *(uint2 *)(row + 32 * i + result_row(r, l)) = make_uint2(pack_bf16(d[0], d[1]), pack_bf16(d[2], d[3]));
                }
        }
    }
};

// out[n][m]: fp32 partial results of a range of the reduction, written or added to
struct SumEpilogue {
    float *out;
    int64_t ld, range;      // elements between rows, between ranges
    int add;
    template <int MB, int NB>
    __device__ __forceinline__ void operator()(floatx16 (&acc)[MB][NB], int m0, int n0, int m, int n) const {
        const int l = threadIdx.x & 63;
        float *o = out + blockIdx.y * range;
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            const int c = n0 + 32 * j + (l & 31);
            if (c >= n) continue;
#pragma unroll
            for (int i = 0; i < MB; ++i)
#pragma unroll
                for (int r = 0; r < 16; r += 4) {
                    const int row = m0 + 32 * i + result_row(r, l);
                    if (row >= m) continue;
                    float4 *p = (float4 *)(o + c * ld + row);
                    float4 v = make_float4(acc[i][j][r], acc[i][j][r + 1], acc[i][j][r + 2], acc[i][j][r + 3]);
                    if (add) { const float4 w = *p; v.x += w.x; v.y += w.y; v.z += w.z; v.w += w.w; }
                    *p = v;
                }
        }
    }
};

// out[n][m] = *by times the sums (+ out), rounded to bf16
struct RoundEpilogue {
    unsigned short *out;
    const float *by;
    int64_t ld;
    bool add;
    template <int MB, int NB>
    __device__ __forceinline__ void operator()(floatx16 (&acc)[MB][NB], int m0, int n0, int m, int n) const {
        const int l = threadIdx.x & 63;
        const float f = *by;
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            const int c = n0 + 32 * j + (l & 31);
            if (c >= n) continue;
#pragma unroll
            for (int i = 0; i < MB; ++i)
#pragma unroll
                for (int r = 0; r < 16; r += 4) {
                    const int row = m0 + 32 * i + result_row(r, l);
                    if (row >= m) continue;
                    uint2 *p = (uint2 *)(out + c * ld + row);
                    float v[4] = {acc[i][j][r] * f, acc[i][j][r + 1] * f, acc[i][j][r + 2] * f, acc[i][j][r + 3] * f};
                    if (add) {
                        const uint2 o = *p;
                        v[0] += __uint_as_float(o.x << 16); v[1] += __uint_as_float(o.x & 0xffff0000u);
                        v[2] += __uint_as_float(o.y << 16); v[3] += __uint_as_float(o.y & 0xffff0000u);
                    }
                    *p = make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]));
                }
        }
    }
};

// 16 threads to a token: lse and the row's loss from the parts of its logits.  TOKENS = 64: the only workgroup, which takes the mean as well.
template <int TOKENS>
__global__ __launch_bounds__(TOKENS * 16) void ce_merge_kernel(const float2 *__restrict__ part, int parts, const float *__restrict__ hit,
                                                               const int32_t *__restrict__ labels, float *__restrict__ lse,
                                                               float *__restrict__ row_loss, float *__restrict__ loss, int rows, int vocab) {
    __shared__ Soft seg[16][TOKENS];
    const int l = threadIdx.x % TOKENS, s = threadIdx.x / TOKENS, t = blockIdx.x * TOKENS + l;
    Soft a{-INFINITY, 0.f};
    if (t < rows) {
        int b = s;
        for (; b + 48 < parts; b += 64) {
            float2 v[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) v[q] = part[(int64_t)(b + 16 * q) * rows + t];
#pragma unroll
            for (int q = 0; q < 4; ++q) a = soft_join(a, Soft{v[q].x, v[q].y});
        }
        for (; b < parts; b += 16) {
            const float2 v = part[(int64_t)b * rows + t];
            a = soft_join(a, Soft{v.x, v.y});
        }
    }
    seg[s][l] = a;
    __syncthreads();
    if (s) return;
    float mine = 0.f;
    const bool has = t < rows && (unsigned)labels[t] < (unsigned)vocab;
    if (t < rows) {
        for (int b = 1; b < 16; ++b) a = soft_join(a, seg[b][l]);
        const float ls = a.m + logf(a.s);
        lse[t] = ls;
        mine = has ? ls - hit[t] : 0.f;
        if (TOKENS < 64) row_loss[t] = mine;
    }
    if (TOKENS < 64) return;
    double sum = mine;       // one wave by now
    for (int w = 32; w; w /= 2) sum += __shfl_xor(sum, w);
    const int count = __popcll(__ballot(has));
    if (l == 0) *loss = count ? (float)(sum / count) : 0.f;
}

// the number of rows with a label (inv: its reciprocal, 0 for none) and the mean of their losses; sums in a fixed order
__global__ __launch_bounds__(1024) void ce_mean_kernel(const float *__restrict__ row_loss, const int32_t *__restrict__ labels, int rows, int vocab,
                                                       float *__restrict__ loss, float *__restrict__ inv) {
    __shared__ double sums[1024];
    __shared__ int counts[1024];
    double sum = 0;
    int count = 0;
    for (int t = threadIdx.x; t < rows; t += 1024)
        if ((unsigned)labels[t] < (unsigned)vocab) { ++count; if (row_loss) sum += row_loss[t]; }
    sums[threadIdx.x] = sum;
    counts[threadIdx.x] = count;
    for (int w = 512; w; w /= 2) {
        __syncthreads();
        if ((int)threadIdx.x < w) { sums[threadIdx.x] += sums[threadIdx.x + w]; counts[threadIdx.x] += counts[threadIdx.x + w]; }
    }
    if (threadIdx.x) return;
    if (loss) *loss = counts[0] ? (float)(sums[0] / counts[0]) : 0.f;
    if (inv) *inv = counts[0] ? 1.f / counts[0] : 0.f;
}

// out = *by times the sum over ranges of part (+ out), rounded to bf16; eight values a thread
__global__ __launch_bounds__(256) void ce_round_kernel(const float *__restrict__ part, int ranges, int64_t n, const float *__restrict__ by,
                                                       unsigned short *__restrict__ out, int add) {
    const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
    if (i >= n) return;
    float v[8] = {};
    for (int r = 0; r < ranges; ++r) {
        const float4 a = *(const float4 *)(part + r * n + i), b = *(const float4 *)(part + r * n + i + 4);
        v[0] += a.x; v[1] += a.y; v[2] += a.z; v[3] += a.w; v[4] += b.x; v[5] += b.y; v[6] += b.z; v[7] += b.w;
    }
    const float f = *by;
#pragma unroll
    for (int q = 0; q < 8; ++q) v[q] *= f;
    if (add) {
        const uint4 o = *(const uint4 *)(out + i);
        const unsigned w[4] = {o.x, o.y, o.z, o.w};
#pragma unroll
        for (int q = 0; q < 4; ++q) { v[2 * q] += __uint_as_float(w[q] << 16); v[2 * q + 1] += __uint_as_float(w[q] & 0xffff0000u); }
    }
    *(uint4 *)(out + i) = make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
}

// fp32: maximum and sum of CE_SEGMENT logits of a row's piece (grid y: which), and the label's logit.  The logits are read once, into registers; a
// row's segments go to different workgroups, since there may be a single row (92544 logits of it: 4.6 us, with one workgroup to a row 122).
constexpr int CE_SEGMENT = 4096;
__global__ __launch_bounds__(256) void ce_piece_stats_kernel(const float *__restrict__ logits, int piece, int v0, const int32_t *__restrict__ labels,
                                                             float2 *__restrict__ part, float *__restrict__ hit) {
    __shared__ Soft seg[256];
    const int64_t t = blockIdx.x;
    const float *row = logits + t * piece;
    const int from = blockIdx.y * CE_SEGMENT, to = min(piece, from + CE_SEGMENT);
    float x[CE_SEGMENT / 256], top = -INFINITY;
#pragma unroll
    for (int i = 0; i < CE_SEGMENT / 256; ++i) {
        const int v = from + i * 256 + threadIdx.x;
        x[i] = v < to ? row[v] : -INFINITY;
        top = fmaxf(top, x[i]);
    }
    const float base = top == -INFINITY ? 0.f : fminf(top, 3.4028235e38f);
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < CE_SEGMENT / 256; ++i) sum += exp_of(x[i] - base);      // an index that does not exist: e^-inf, 0
    if (top == INFINITY) { top = 3.4028235e38f; sum = INFINITY; }
    seg[threadIdx.x] = Soft{top, sum};
    for (int w = 128; w; w /= 2) {
        __syncthreads();
        if ((int)threadIdx.x < w) seg[threadIdx.x] = soft_join(seg[threadIdx.x], seg[threadIdx.x + w]);
    }
    if (threadIdx.x) return;
    part[blockIdx.y * (int64_t)gridDim.x + t] = make_float2(seg[0].m, seg[0].s);
    const int label = labels[t] - v0;
    if (label >= from && label < to) hit[t] = row[label];
}
// fp32: dl in the place of the logits.  COUNT: with up to 1024 rows every workgroup counts the labels itself, a launch less.
template <bool COUNT>
__global__ __launch_bounds__(256) void ce_piece_grad_kernel(float *__restrict__ logits, int piece, int v0, const int32_t *__restrict__ labels,
                                                            const float *__restrict__ lse, const float *__restrict__ inv_count, int rows, int vocab) {
    __shared__ int counts[4];
    float inv;
    if (COUNT) {
        int count = 0;
        for (int t = threadIdx.x; t < rows; t += 256) count += (unsigned)labels[t] < (unsigned)vocab;
        for (int w = 32; w; w /= 2) count += __shfl_xor(count, w);
        if (threadIdx.x % 64 == 0) counts[threadIdx.x / 64] = count;
        __syncthreads();
        count = counts[0] + counts[1] + counts[2] + counts[3];
        inv = count ? 1.f / count : 0.f;
    } else inv = *inv_count;
    const int64_t t = blockIdx.x;
    const int v = blockIdx.y * 256 + threadIdx.x;
    if (v >= piece) return;
    const int label = labels[t];
    float *at = logits + t * piece + v;
    *at = (unsigned)label < (unsigned)vocab ? (exp_of(*at - lse[t]) - (v0 + v == label ? 1.f : 0.f)) * inv : 0.f;
}

// fp32 and few rows: dx += dl W, which reads all of W for rows * 2 operations an entry.  A matrix tile would be mostly empty, and its few
// workgroups wait for memory; here a workgroup sums 256 columns over `per` entries of the piece on the vector units, rows from scalar
// registers, and leaves part[range][row][column].  11 rows, 1120 columns, 41104 entries (184 MB): 48 us (3.8 TB/s), the convolutions'
// tiles 91; 1 row, 144 columns, 92544 entries: 9 us, the tiles 188.
// Twice as many rows (grid z) read W twice, which pays where it stays in L2; backward pass of 24 rows, with this kernel and with the tiles, us: 128
// columns and 1009 entries 26 and 33, 512 and 2000 27 and 29, 1024 and 1024 30.5 and 30.9, 1024 and 2048 32 and 31, 2048 and 4000 52 and 45, 4096
// and 32000 575 and 469.  So up to 2^20 weights; of narrower layers also beyond (512 and 16000: 54 and 69; 256 and 32000: 56 and 101), not taken.
constexpr int CE_FEW_ROWS = 16;
template <int ROWS>
__global__ __launch_bounds__(256) void ce_few_rows_kernel(const float *__restrict__ dl, int piece, const float *__restrict__ w, int width, int rows, int per,
                                                          float *__restrict__ part) {
    __shared__ float sums[4][ROWS][256];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), l = threadIdx.x & 63, c0 = blockIdx.x * 256;
    const int from = blockIdx.y * per, to = min(piece, from + per), t0 = blockIdx.z * ROWS;
    int col[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) col[j] = min(c0 + 64 * j + l, width - 1);
    float acc[ROWS][4] = {};
    auto add = [&](int v, auto n) {      // entries v .. v + n - 1; rows that do not exist take the last one's dl and are not stored
        constexpr int N = decltype(n)::value;
        float x[N][4];
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) x[i][j] = w[(int64_t)(v + i) * width + col[j]];
#pragma unroll
        for (int t = 0; t < ROWS; ++t) {
            const float *d = dl + (int64_t)min(t0 + t, rows - 1) * piece + v;
#pragma unroll
            for (int i = 0; i < N; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[t][j] = fmaf(d[i], x[i][j], acc[t][j]);
        }
    };
    int v = from + 4 * wave;
    for (; v + 4 <= to; v += 16) add(v, std::integral_constant<int, 4>());
    for (const int end = min(to, v + 4); v < end; ++v) add(v, std::integral_constant<int, 1>());
#pragma unroll
    for (int t = 0; t < ROWS; ++t)
#pragma unroll
        for (int j = 0; j < 4; ++j) sums[wave][t][64 * j + l] = acc[t][j];
    __syncthreads();
    const int c = threadIdx.x;
    if (c0 + c >= width) return;
    for (int t = 0; t < min(ROWS, rows - t0); ++t)
        part[((int64_t)blockIdx.y * rows + t0 + t) * width + c0 + c] = (sums[0][t][c] + sums[1][t][c]) + (sums[2][t][c] + sums[3][t][c]);
}
// The logits of up to eight rows, bound by reading W as well: a wave takes eight entries, its lanes 256 columns of them at a time; the rows come from the
// vector cache, where a workgroup's waves share them.  Then ROWS x 8 sums over 64 lanes: each step exchanges half of them and keeps the other
// half.  Forward pass, 1 row, 2024 columns, 41311 entries (334 MB): 90 us (3.8 TB/s), with the convolutions' tiles 164; 6 rows, 2552, 38183: 162 and
// 194; but 11 rows, 1120, 41119: 214 and 86, the rows' loads outnumber W's; 3 rows, 64 columns, 500 entries, 16 workgroups: 13.1 and 11.3.
constexpr int CE_FEW_ENTRIES = 8;
template <int ROWS>
__global__ __launch_bounds__(256) void ce_few_logits_kernel(const float *__restrict__ x, const float *__restrict__ w, int width, int rows, int piece,
                                                            float *__restrict__ logits) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), l = threadIdx.x & 63;
    const int v0 = (blockIdx.x * 4 + wave) * CE_FEW_ENTRIES;
    if (v0 >= piece) return;
    float sum[ROWS * CE_FEW_ENTRIES] = {};      // [row][entry]; rows and entries that do not exist repeat the last one and are not stored
    auto add = [&](int c, auto whole) {
        constexpr int N = decltype(whole)::value ? 4 : 1;
        float e[CE_FEW_ENTRIES][N];
#pragma unroll
        for (int i = 0; i < CE_FEW_ENTRIES; ++i)
#pragma unroll
            for (int j = 0; j < N; ++j) e[i][j] = w[(int64_t)min(v0 + i, piece - 1) * width + c + 64 * j];
#pragma unroll
        for (int t = 0; t < ROWS; ++t) {
            const float *row = x + (int64_t)min(t, rows - 1) * width + c;
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const float f = row[64 * j];
#pragma unroll
                for (int i = 0; i < CE_FEW_ENTRIES; ++i) sum[t * CE_FEW_ENTRIES + i] = fmaf(f, e[i][j], sum[t * CE_FEW_ENTRIES + i]);
            }
        }
    };
    int c = l;
    for (; c - l + 256 <= width; c += 256) add(c, std::true_type());
    for (; c < width; c += 64) add(c, std::false_type());
    // lane l ends with the LEFT sums from l * LEFT on, or, of fewer than 64, ALIKE neighbouring lanes with the same one
    constexpr int ALL = ROWS * CE_FEW_ENTRIES, LEFT = ALL > 64 ? ALL / 64 : 1, ALIKE = ALL < 64 ? 64 / ALL : 1;
#pragma unroll
    for (int k = 0; k < 6; ++k) {
        const int step = 32 >> k, n = ALL >> (k + 1);
        const bool high = l & step;
        if (n == 0) sum[0] += __shfl_xor(sum[0], step);
#pragma unroll
        for (int i = 0; i < n; ++i) {
            const float keep = high ? sum[i + n] : sum[i], send = high ? sum[i] : sum[i + n];
            sum[i] = keep + __shfl_xor(send, step);
        }
    }
    if (l % ALIKE) return;
#pragma unroll
    for (int i = 0; i < LEFT; ++i) {
        const int at = l / ALIKE * LEFT + i, t = at / CE_FEW_ENTRIES, v = v0 + at % CE_FEW_ENTRIES;
        if (t < rows && v < piece) logits[(int64_t)t * piece + v] = sum[i];
    }
}
bool ce_few_logits(hipStream_t st, const float *x, const float *w, int width, int rows, int piece, float *logits) {
    if (rows > 8 || piece < 8192) return false;
    const unsigned groups = (unsigned)((piece + 4 * CE_FEW_ENTRIES - 1) / (4 * CE_FEW_ENTRIES));
    if (rows <= 4) hipLaunchKernelGGL(ce_few_logits_kernel<4>, dim3(groups), dim3(256), 0, st, x, w, width, rows, piece, logits);
    else hipLaunchKernelGGL(ce_few_logits_kernel<8>, dim3(groups), dim3(256), 0, st, x, w, width, rows, piece, logits);
    hip_check(hipGetLastError(), "linear_ce logits launch");
    return true;
}

// out (+)= the sum over the ranges of part, in a fixed order: sixteen waves take a share of the ranges each
__global__ __launch_bounds__(1024) void ce_few_rows_join_kernel(const float *__restrict__ part, int ranges, int n, float *__restrict__ out, int add) {
    __shared__ float sums[16][64];
    const int wave = threadIdx.x / 64, l = threadIdx.x & 63, i = blockIdx.x * 64 + l;
    float sum = 0.f;
    if (i < n) {
#pragma unroll 8
        for (int r = wave; r < ranges; r += 16) sum += part[(int64_t)r * n + i];
    }
    sums[wave][l] = sum;
    __syncthreads();
    if (wave || i >= n) return;
#pragma unroll
    for (int w = 1; w < 16; ++w) sum += sums[w][l];
    out[i] = add ? out[i] + sum : sum;
}

int64_t up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }
int64_t cut(int64_t n, int64_t by) { return (n + by - 1) / by; }

constexpr int64_t CE_PIECE_BYTES = 256ll << 20;      // a piece of logits or of their gradient

// Results of few tiles leave CUs idle while their reduction is long: as many ranges as fill the card, of at least `least` indices.
int ce_splits(int64_t tiles, int64_t red, int64_t least) {
    return (int)std::max<int64_t>(1, std::min<int64_t>({256 / std::max<int64_t>(tiles, 1), red / least, 16}));
}

// Ranges of the reduction over a piece in dx = dl W.  Large tiles (gemm_tile) where ranges of 4096 entries or more make whole rounds of one to a CU
// (a range's fp32 sums cost 8 bytes of traffic for each result) and few of their entries lie outside the result: backward pass of 512 rows,
// 2048 columns, 100000 entries 830 us, with small tiles 997; 4096 rows, 2048 columns, 50176 entries 2459 and 2542.  Small ones otherwise:
// 4000 rows, 1600 columns, 50257 entries (112 large tiles; three ranges are 1.3 rounds) 2126 us, with large ones 2248.
int ce_input_ranges(int64_t rows, int64_t width, int piece) {
    const int64_t large = cut(width, 256) * cut(rows, 256), ranges = cut(256, large);
    if (ranges <= 16 && piece / ranges >= 4096 && 5 * rows * width * ranges >= 4 * 65536 * up(large * ranges, 256)) return (int)ranges;
    return ce_splits(cut(width, 128) * cut(rows, 128), piece, 512);
}

// How a call goes through the vocabulary, and its workspace: forward [hit][row_loss][part][product][logits (fp32)], backward
// [inv][dx parts (bf16) or product][dl].
struct CePlan {
    int rows, width, vocab;
    bool bf16;
    int unit = 0;                   // bf16 forward: logits to a part
    int piece = 0;                  // logits of a piece
    int ranges = 1, chunk = 0;      // bf16 backward: of the reduction over a piece in dx
    int64_t product = 0;            // fp32: bytes for the products' partial results
    int64_t fixed = 0, per_col = 0;              // bytes without the pieces, and for each logit of a piece

    int64_t bytes() const { return fixed + per_col * piece; }
    int wgrad_splits(int piece) const { return ce_splits(cut(width, 128) * cut(piece, 128), rows, 64); }
    bool few_rows(int piece) const { return rows <= CE_FEW_ROWS || (rows <= 2 * CE_FEW_ROWS && (int64_t)piece * width <= 1 << 20); }      // twice: where W stays in L2
    int few_per(int piece) const {      // entries of W for a workgroup: four workgroups to a CU
        return (int)up(cut(piece, std::max<int64_t>(1, std::min<int64_t>(1024 / cut(width, 256), cut(piece, 64)))), 16);
    }
    // where the pieces begin, and the vocabulary's end.  fp32: the products read 16 bytes at a time where the piece is a multiple of
    // 16, so what a large vocabulary has over that is a piece of its own
    std::vector<int> pieces() const {
        std::vector<int> at;
        const int tail = !bf16 && vocab > 4096 ? vocab % 16 : 0;
        for (int v = 0; v < vocab - tail; v += piece) at.push_back(v);
        if (tail) at.push_back(vocab - tail);
        at.push_back(vocab);
        return at;
    }
    int64_t parts() const {
        if (bf16) return cut(vocab, unit);
        const std::vector<int> at = pieces();
        int64_t n = 0;
        for (size_t i = 0; i + 1 < at.size(); ++i) n += cut(at[i + 1] - at[i], CE_SEGMENT);
        return n;
    }
};

CePlan ce_plan(bool grad, int dtype, int64_t rows, int width, int vocab) {
    if (dtype != MONET_F32 && dtype != MONET_BF16) throw KernelError("linear_ce: dtype must be MONET_F32 or MONET_BF16");
    if (rows < 1 || width < 1 || vocab < 1) throw KernelError("linear_ce: bad shape");
    const bool bf16 = dtype == MONET_BF16;
    if (bf16 && width % 8) throw KernelError("linear_ce: bf16 needs a width that is a multiple of 8");
    if (rows >= (1 << 24) || width > (1 << 20) || vocab > (1 << 28)) throw KernelError("linear_ce: shape too large");
    CePlan p{(int)rows, width, vocab, bf16};
    if (bf16 && !grad) {
        if (!gemm_fits(vocab, rows, 1, width, width)) throw KernelError("linear_ce: rows * vocab too large");
        p.unit = gemm_tile(vocab, rows) / 2;
        p.fixed = 2 * up(rows * 4, 256) + up(p.parts() * rows * 8, 256);
        return p;
    }
    p.per_col = up(rows * (bf16 ? 2 : 4), 256);
    const int64_t pieces = cut(vocab, std::max<int64_t>(CE_PIECE_BYTES / p.per_col / 256 * 256, 256));
    p.piece = (int)std::min<int64_t>(up(cut(vocab, pieces), 256), 1 << 20);
    if (!bf16) p.piece = std::min<int64_t>({p.piece, vocab, std::max<int64_t>(((1ll << 32) - (1 << 21)) / (4 * (int64_t)width) / 256 * 256, 256)});      // the products address a piece of w with 32 bits
    const ConvShape cs{p.rows, 1, 1, width, p.piece, 1, 1, 1, 0, 1, 1};
    if (!grad) {
        p.product = up((int64_t)conv_workspace_bytes(0, cs, 1), 256);
        p.fixed = 2 * up(rows * 4, 256) + up(p.parts() * rows * 8, 256) + p.product;
        return p;
    }
    p.fixed = 256;
    if (bf16) {
        p.ranges = ce_input_ranges(rows, width, p.piece);
        const int64_t ld = up(p.piece, 8);
        if (!gemm_fits(p.piece, rows, 1, width, width) || !gemm_fits(width, rows, p.ranges, width, ld) || !gemm_fits(width, p.piece, 1, width, ld))
            throw KernelError("linear_ce: rows * width too large");      // before anything is launched
        p.chunk = (int)up(cut(p.piece, p.ranges), GEMM_DEPTH);
        p.ranges = (int)cut(std::min(p.piece, vocab), p.chunk);      // a later piece is no longer than the first
        if (p.ranges > 1 || p.piece < vocab) p.fixed += up(p.ranges * rows * width * 4, 256);
    } else {
        p.product = (int64_t)std::max(conv_workspace_bytes(0, cs, 1), p.few_rows(p.piece) ? 0 : conv_workspace_bytes(1, cs, 1));
        const std::vector<int> at = p.pieces();
        for (size_t i = 0; i + 1 < at.size(); ++i) {
            const int64_t piece = at[i + 1] - at[i], splits = p.wgrad_splits((int)piece);
            if (splits > 1) p.product = std::max(p.product, splits * piece * width * 4);
            if (p.few_rows((int)piece)) p.product = std::max(p.product, cut(piece, p.few_per((int)piece)) * rows * width * 4);
        }
        p.product = up(p.product, 256);
        p.fixed += p.product;
    }
    return p;
}

void check_ws(const CePlan &p, const void *ws, size_t ws_bytes) {
    if (!ws || (int64_t)ws_bytes < p.bytes()) throw KernelError("linear_ce: workspace of " + std::to_string(ws_bytes) + " bytes, " + std::to_string(p.bytes()) + " needed");
    if ((uintptr_t)ws % 256) throw KernelError("linear_ce: the workspace must be 256-byte aligned");
}
void check_aligned(const CePlan &p, std::initializer_list<const void *> ptrs) {
    for (const void *q : ptrs) {
        if (!q) throw KernelError("linear_ce: null pointer");
        if ((uintptr_t)q % (p.bf16 ? 16 : 4)) throw KernelError(p.bf16 ? "linear_ce: bf16 tensors must be 16-byte aligned" : "linear_ce: fp32 tensors must be 4-byte aligned");
    }
}
void check_words(std::initializer_list<const void *> ptrs) {
    for (const void *q : ptrs) {
        if (!q) throw KernelError("linear_ce: null pointer");
        if ((uintptr_t)q % 4) throw KernelError("linear_ce: labels, loss and lse must be 4-byte aligned");
    }
}

GemmShape ce_logits_shape(const CePlan &p, const void *x, const void *w, int v0, int piece) {
    GemmShape g{};
    g.a = (const unsigned short *)w + (int64_t)v0 * p.width;
    g.b = (const unsigned short *)x;
    g.lda = g.ldb = p.width;
    g.m = piece; g.n = p.rows; g.k = p.width;
    g.splits = 1; g.chunk = (int)up(p.width, GEMM_DEPTH);
    return g;
}
ConvShape ce_conv_shape(const CePlan &p, int piece) { return ConvShape{p.rows, 1, 1, p.width, piece, 1, 1, 1, 0, 1, 1}; }

}  // namespace

size_t linear_ce_workspace_bytes(bool grad, int dtype, int64_t rows, int width, int vocab) {
    return (size_t)std::max(ce_plan(grad, dtype, rows, width, vocab).bytes(), ce_plan(false, dtype, rows, width, vocab).bytes());
}

void linear_ce_fwd(hipStream_t st, int dtype, const void *x, const void *w, const int32_t *labels, float *loss, float *lse, int64_t rows,
                   int width, int vocab, void *ws, size_t ws_bytes) {
    const CePlan p = ce_plan(false, dtype, rows, width, vocab);
    check_ws(p, ws, ws_bytes);
    check_aligned(p, {x, w});
    check_words({labels, loss, lse});
    float *hit = (float *)ws, *row_loss = hit + up(rows, 64);
    float2 *part = (float2 *)(row_loss + up(rows, 64));
    if (p.bf16) {
        gemm_bf16<false, false>(st, ce_logits_shape(p, x, w, 0, vocab), CeStatsEpilogue{labels, part, hit, p.rows, vocab}, "linear_ce logits launch");
    } else {
        float *logits = (float *)((char *)ws + p.fixed), *product = p.product ? (float *)((char *)logits - p.product) : nullptr;
        const size_t product_bytes = (size_t)p.product;
        const std::vector<int> at = p.pieces();
        int64_t done = 0;      // parts
        for (size_t i = 0; i + 1 < at.size(); ++i) {
            const int piece = at[i + 1] - at[i], segments = (int)cut(piece, CE_SEGMENT);
            const float *wp = (const float *)w + (int64_t)at[i] * width;
            if (!ce_few_logits(st, (const float *)x, wp, width, p.rows, piece, logits)) conv_fwd(st, (const float *)x, wp, logits, ce_conv_shape(p, piece), 1, product, product_bytes);
            hipLaunchKernelGGL(ce_piece_stats_kernel, dim3(p.rows, segments), dim3(256), 0, st, logits, piece, at[i], labels, part + done * rows, hit);
            hip_check(hipGetLastError(), "linear_ce statistics launch");
            done += segments;
        }
    }
    if (rows <= 64 && rows * p.parts() <= 1 << 14) {      // few enough for one workgroup: a launch less
        hipLaunchKernelGGL(ce_merge_kernel<64>, dim3(1), dim3(1024), 0, st, part, (int)p.parts(), hit, labels, lse, row_loss, loss, p.rows, vocab);
        hip_check(hipGetLastError(), "linear_ce merge launch");
        return;
    }
    hipLaunchKernelGGL(ce_merge_kernel<16>, dim3((unsigned)cut(rows, 16)), dim3(256), 0, st, part, (int)p.parts(), hit, labels, lse, row_loss, loss, p.rows, vocab);
    hip_check(hipGetLastError(), "linear_ce merge launch");
    hipLaunchKernelGGL(ce_mean_kernel, dim3(1), dim3(1024), 0, st, row_loss, labels, p.rows, vocab, loss, (float *)nullptr);
    hip_check(hipGetLastError(), "linear_ce mean launch");
}

void linear_ce_bwd(hipStream_t st, int dtype, const void *x, const void *w, const int32_t *labels, const float *lse, void *dx, void *dw,
                   int64_t rows, int width, int vocab, bool accumulate, void *ws, size_t ws_bytes) {
    const CePlan p = ce_plan(true, dtype, rows, width, vocab);
    check_ws(p, ws, ws_bytes);
    check_aligned(p, {x, w, dx, dw});
    check_words({labels, lse});
    float *inv = (float *)ws;
    const bool count = p.bf16 || rows > 1024;
    if (count) {
        hipLaunchKernelGGL(ce_mean_kernel, dim3(1), dim3(1024), 0, st, (const float *)nullptr, labels, p.rows, vocab, (float *)nullptr, inv);
        hip_check(hipGetLastError(), "linear_ce count launch");
    }
    const std::vector<int> at = p.pieces();
    char *dl = (char *)ws + p.fixed;
    float *parts = (float *)((char *)ws + 256);
    for (size_t i = 0; i + 1 < at.size(); ++i) {
        const int v0 = at[i], piece = at[i + 1] - v0;
        if (p.bf16) {
            unsigned short *d = (unsigned short *)dl;
            const int64_t ld = up(piece, 8);
            gemm_bf16<false, false>(st, ce_logits_shape(p, x, w, v0, piece),
                                    CeGradEpilogue{labels, lse, d, ld, p.rows, piece, v0, vocab}, "linear_ce gradient launch");
            GemmShape g{};
            // dx[t][c] (+)= sum over v of w[v][c] dl[t][v]
            g.a = (const unsigned short *)w + (int64_t)v0 * width; g.lda = width;
            g.b = d; g.ldb = ld;
            g.m = width; g.n = p.rows; g.k = piece;
            g.chunk = p.chunk; g.splits = (int)cut(piece, p.chunk);
            if (p.ranges == 1 && at.size() == 2)      // the workspace holds no sums then
                gemm_bf16<true, false>(st, g, RoundEpilogue{(unsigned short *)dx, inv, width, accumulate}, "linear_ce input gradient launch");
            else {
                gemm_bf16<true, false>(st, g, SumEpilogue{parts, width, rows * width, i > 0}, "linear_ce input gradient launch");
                if (i + 2 == at.size()) {
                    const int64_t n = rows * width;
                    hipLaunchKernelGGL(ce_round_kernel, dim3((unsigned)cut(n, 2048)), dim3(256), 0, st, parts, p.ranges, n, inv, (unsigned short *)dx, accumulate);
                    hip_check(hipGetLastError(), "linear_ce round launch");
                }
            }
            // dw[v][c] = sum over t of x[t][c] dl[t][v]
            g.a = (const unsigned short *)x; g.lda = width;
            g.m = width; g.n = piece; g.k = p.rows;
            g.splits = 1; g.chunk = (int)up(rows, GEMM_DEPTH);
            gemm_bf16<true, true>(st, g, RoundEpilogue{(unsigned short *)dw + (int64_t)v0 * width, inv, width, false}, "linear_ce weight gradient launch");
        } else {
            const ConvShape cs = ce_conv_shape(p, piece);
            const float *wp = (const float *)w + (int64_t)v0 * width;
            float *d = (float *)dl;
            float *product = p.product ? parts : nullptr;
            const size_t product_bytes = (size_t)p.product;
            if (!ce_few_logits(st, (const float *)x, wp, width, p.rows, piece, d)) conv_fwd(st, (const float *)x, wp, d, cs, 1, product, product_bytes);
            hipLaunchKernelGGL((count ? ce_piece_grad_kernel<false> : ce_piece_grad_kernel<true>), dim3(p.rows, (unsigned)cut(piece, 256)), dim3(256), 0, st, d, piece, v0,
                               labels, lse, inv, p.rows, vocab);
            hip_check(hipGetLastError(), "linear_ce gradient launch");
            if (p.few_rows(piece)) {
                const int per = p.few_per(piece), ranges = (int)cut(piece, per), n = p.rows * width;
                const dim3 grid((unsigned)cut(width, 256), ranges);
                if (rows <= 4)
                    hipLaunchKernelGGL(ce_few_rows_kernel<4>, grid, dim3(256), 0, st, d, piece, wp, width, p.rows, per, product);
                else
                    hipLaunchKernelGGL(ce_few_rows_kernel<CE_FEW_ROWS>, dim3(grid.x, grid.y, (unsigned)cut(rows, CE_FEW_ROWS)), dim3(256), 0, st, d, piece, wp, width, p.rows, per, product);
                hip_check(hipGetLastError(), "linear_ce input gradient launch");
                hipLaunchKernelGGL(ce_few_rows_join_kernel, dim3((unsigned)cut(n, 64)), dim3(1024), 0, st, product, ranges, n, (float *)dx, accumulate || i > 0);
                hip_check(hipGetLastError(), "linear_ce input gradient sum launch");
            } else {
                conv_dgrad(st, d, wp, (float *)dx, cs, accumulate || i > 0, 1, product, product_bytes);
            }
            const int splits = p.wgrad_splits(piece);
            conv_wgrad(st, (const float *)x, d, (float *)dw + (int64_t)v0 * width, cs, splits, splits > 1 ? product : nullptr, splits > 1 ? product_bytes : 0);
        }
    }
}

}  // namespace monet
