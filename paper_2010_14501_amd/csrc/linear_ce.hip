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
// The same layer against a teacher's top logits (linear_distill): l / T for l, mass exp(l / T - lse) - (the teacher's probabilities) for dl, T / count for
// 1 / count; the products and the pieces are the same, the teacher's few entries of a row go through kernels of their own.
#include <cmath>
#include <initializer_list>
#include <type_traits>
#include <vector>

#include "../../include/monet_kernels.h"
#include "gemm_bf16.hpp"
#include "kernels.hpp"
#include "wave_sum.hpp"

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

// rows of the result are vocabulary entries, columns tokens: a lane has 16 * MB logits of each of its NB tokens.  LABELS: the label's logit
// is kept as well; otherwise the logits are `by` times the product (1 / temperature).
template <bool LABELS>
struct StatsEpilogue {
    const int32_t *labels;
    float2 *part;           // [vocab / (32 MB)][rows]: a wave's rows together
    float *hit;             // the label's logit
    int rows, vocab;
    float by;
    template <int MB, int NB>
    __device__ __forceinline__ void operator()(floatx16 (&acc)[MB][NB], int m0, int n0, int, int) const {
        static_assert(MB == 4 || MB == 2, "");
        const int l = threadIdx.x & 63;
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            const int t = n0 + 32 * j + (l & 31);
            const int label = LABELS && t < rows ? labels[t] : -1;
            float top = -INFINITY, mine = 0.f;
            bool found = false;
#pragma unroll
            for (int i = 0; i < MB; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int v = m0 + 32 * i + result_row(r, l);
                    if (!LABELS) acc[i][j][r] *= by;
                    if (v >= vocab) acc[i][j][r] = -INFINITY;
                    if (LABELS && v == label) { mine = acc[i][j][r]; found = true; }
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

// The same against a teacher: count / T dl = mass exp(l / T - lse), without the teacher's entries, which distill_entries_kernel puts in.
struct DistillGradEpilogue {
    const float *mass, *lse;
    unsigned short *dl;
    int64_t ld;
    int rows, piece;
    float by;           // 1 / T
    template <int MB, int NB>
    __device__ __forceinline__ void operator()(floatx16 (&acc)[MB][NB], int m0, int n0, int, int) const {
        const int l = threadIdx.x & 63;
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            const int t = n0 + 32 * j + (l & 31);
            if (t >= rows) continue;
            const float m = mass[t], ls = lse[t];
            unsigned short *row = dl + t * ld + m0;
#pragma unroll
            for (int i = 0; i < MB; ++i)
#pragma unroll
                for (int r = 0; r < 16; r += 4) {
                    float d[4];
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        d[q] = m != 0.f && m0 + 32 * i + result_row(r + q, l) < piece ? m * exp_of(acc[i][j][r + q] * by - ls) : 0.f;
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

// 16 threads to a token: lse and the row's loss (LABELS false: lse alone) from the parts of its logits.  TOKENS = 64: the only workgroup, which
// takes the mean as well.
template <int TOKENS, bool LABELS = true>
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
    const bool has = LABELS && t < rows && (unsigned)labels[t] < (unsigned)vocab;
    if (t < rows) {
        for (int b = 1; b < 16; ++b) a = soft_join(a, seg[b][l]);
        const float ls = a.m + logf(a.s);
        lse[t] = ls;
        mine = has ? ls - hit[t] : 0.f;
        if (TOKENS < 64 && LABELS) row_loss[t] = mine;
    }
    if (TOKENS < 64 || !LABELS) return;
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
// LABELS false: `by` times the logits, no label.
constexpr int CE_SEGMENT = 4096;
template <bool LABELS>
__global__ __launch_bounds__(256) void ce_piece_stats_kernel(const float *__restrict__ logits, int piece, int v0, const int32_t *__restrict__ labels,
                                                             float2 *__restrict__ part, float *__restrict__ hit, float by) {
    __shared__ Soft seg[256];
    const int64_t t = blockIdx.x;
    const float *row = logits + t * piece;
    const int from = blockIdx.y * CE_SEGMENT, to = min(piece, from + CE_SEGMENT);
    float x[CE_SEGMENT / 256], top = -INFINITY;
#pragma unroll
    for (int i = 0; i < CE_SEGMENT / 256; ++i) {
        const int v = from + i * 256 + threadIdx.x;
        x[i] = v < to ? (LABELS ? row[v] : row[v] * by) : -INFINITY;
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
    if (!LABELS) return;
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

// ---- against a teacher's top logits
// Entry j of a row is vocabulary index i_j with the teacher's logit t_j; p_j = exp(t_j / T - its normaliser), 0 for an index outside the vocabulary.
//   loss = sum_j p_j (log p_j + lse - z_j),   mass = sum_j p_j,   delta_j = mass exp(z_j - lse) - (sum of p at the same index)
// with z_j = x . w[i_j] / T.  One workgroup to a row; z by a wave's sums over the columns, each in the same order, so that an index that comes
// twice gets the same number twice.  Bound by reading rows * top rows of w, most of them from the caches: 8192 rows, 64 entries, 4096 columns, bf16
// (4.3 GB): 530 us, one entry at a time to each of four waves 640; 1000 rows, 64 entries, 1024 columns (131 MB): 22 us, so 30.
constexpr int DISTILL_TOP = 1024;      // entries of a row, at most
constexpr int DISTILL_TAIL = 16;       // fp32: more than a large vocabulary has over a multiple of 16, below
// N dot products with one x by G lanes, of which this is lane g: 16 bytes at a time, and of a row of floats that is no multiple of four the rest value by
// value.  The sums are in all of the lanes.
template <int G>
__device__ __forceinline__ float distill_lanes_sum(float v) {
    static_assert(G == 16 || G == 64, "");
    return G == 64 ? wave_sum(v) : row_sum(v);
}
template <int G, int N>
__device__ __forceinline__ void distill_dots(const float *x, const float *const (&w)[N], int width, int g, float (&s)[N]) {
    typedef float any __attribute__((ext_vector_type(4), aligned(4)));
    const auto load = [&](int c, any &f, any (&v)[N]) {
        f = *(const any *)(x + c);
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = *(const any *)(w[j] + c);
    };
    const auto add = [&](const any &f, const any (&v)[N]) {
#pragma unroll
        for (int j = 0; j < N; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[j] = fmaf(f[e], v[j][e], s[j]);
    };
    any f0, f1, v0[N], v1[N];       // two steps' loads under way: 63 rows, 139 entries, 2584 columns, bf16 21 us, with one 41
    int c = 4 * g;
    for (; c + 4 * G + 4 <= width; c += 8 * G) {
        load(c, f0, v0);
        load(c + 4 * G, f1, v1);
        add(f0, v0);
        add(f1, v1);
    }
    if (c + 4 <= width) {
        load(c, f0, v0);
        add(f0, v0);
        c += 4 * G;
    }
    for (int e = c; e < min(c + 4, width); ++e)
#pragma unroll
        for (int j = 0; j < N; ++j) s[j] = fmaf(x[e], w[j][e], s[j]);
#pragma unroll
    for (int j = 0; j < N; ++j) s[j] = distill_lanes_sum<G>(s[j]);
}
template <int G, int N>
__device__ __forceinline__ void distill_dots(const unsigned short *x, const unsigned short *const (&w)[N], int width, int g, float (&s)[N]) {
    const auto load = [&](int c, uintx4 &f, uintx4 (&v)[N]) {
        f = *(const uintx4 *)(x + c);
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = *(const uintx4 *)(w[j] + c);
    };
    const auto add = [&](const uintx4 &f, const uintx4 (&v)[N]) {
#pragma unroll
        for (int j = 0; j < N; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                s[j] = fmaf(__uint_as_float(f[q] << 16), __uint_as_float(v[j][q] << 16), s[j]);
                s[j] = fmaf(__uint_as_float(f[q] & 0xffff0000u), __uint_as_float(v[j][q] & 0xffff0000u), s[j]);
            }
    };
    uintx4 f0, f1, v0[N], v1[N];
    int c = 8 * g;
    for (; c + 8 * G < width; c += 16 * G) {
        load(c, f0, v0);
        load(c + 8 * G, f1, v1);
        add(f0, v0);
        add(f1, v1);
    }
    if (c < width) {
        load(c, f0, v0);
        add(f0, v0);
    }
#pragma unroll
    for (int j = 0; j < N; ++j) s[j] = distill_lanes_sum<G>(s[j]);
}
constexpr int DISTILL_WAVES = 8;
template <class T>
__global__ __launch_bounds__(64 * DISTILL_WAVES) void distill_rows_kernel(const T *__restrict__ x, const T *__restrict__ w, const int32_t *__restrict__ index,
                                                                          const float *__restrict__ target, const float *__restrict__ target_lse,
                                                                          const float2 *__restrict__ part, int parts, const float *__restrict__ logits,
                                                                          int piece, int rows, float *__restrict__ lse,
                                                                          float *__restrict__ mass, float *__restrict__ delta, float *__restrict__ row_loss,
                                                                          int width, int vocab, int tail, int top, float heat) {
    __shared__ float z[DISTILL_TOP], last[DISTILL_TAIL];
    __shared__ alignas(16) float p[DISTILL_TOP];
    __shared__ alignas(16) int at[DISTILL_TOP];
    __shared__ uint4 seen[1024];                // a bit for each value of an index's lowest 17 bits
    __shared__ Soft joined[DISTILL_WAVES];
    __shared__ int twice;                       // an index may come more than once
    constexpr int THREADS = 64 * DISTILL_WAVES;
    const int64_t t = blockIdx.x;
    const int wave = threadIdx.x / 64, l = threadIdx.x & 63;
    index += t * top;
    target += t * top;
    if (threadIdx.x == 0) twice = 0;
    for (int j = threadIdx.x; j < 1024; j += THREADS) seen[j] = make_uint4(0, 0, 0, 0);
    // the row's lse from its parts or its logits, unless it is there already
    Soft a{-INFINITY, 0.f};
    const bool joins = part || logits;
    if (logits) {
        constexpr int AHEAD = 8;
        const float *row = logits + t * piece, by = 1.f / heat;
        for (int v0 = threadIdx.x; v0 - (int)threadIdx.x < piece; v0 += AHEAD * THREADS) {
            float f[AHEAD], m = -INFINITY, sum = 0.f;
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) {
                f[i] = v0 + i * THREADS < piece ? row[v0 + i * THREADS] * by : -INFINITY;
                m = fmaxf(m, f[i]);
            }
            const float base = m == -INFINITY ? 0.f : fminf(m, 3.4028235e38f);
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) sum += exp_of(f[i] - base);
            if (m == INFINITY) { m = 3.4028235e38f; sum = INFINITY; }
            a = soft_join(a, Soft{m, sum});
        }
    }
    if (part) {
        for (int b = threadIdx.x; b < parts; b += THREADS) {
            const float2 v = part[(int64_t)b * rows + t];
            a = soft_join(a, Soft{v.x, v.y});
        }
    }
    const int whole = (top + 3) & ~3;       // entries behind the last one have no index and no weight
    for (int j = threadIdx.x; j < whole; j += THREADS) {
        const int v = j < top ? index[j] : -1;
        at[j] = (unsigned)v < (unsigned)vocab ? v : -1;
        if (j >= top) p[j] = 0.f;
    }
    __syncthreads();
    for (int j = threadIdx.x; j < top; j += THREADS) {
        const unsigned v = at[j] & 0x1ffff, bit = 1u << (v & 31);
        if (at[j] >= 0 && (atomicOr((unsigned *)seen + v / 32, bit) & bit)) twice = 1;
    }
    // G lanes to an entry of `end`, N entries at a time; their vocabulary indices are which(j), below 0 for one that is none
    const auto dots = [&](int end, auto lanes, auto n, auto which, float *out) {
        constexpr int G = decltype(lanes)::value, N = decltype(n)::value;
        for (int j0 = N * (threadIdx.x / G); j0 < end; j0 += N * (THREADS / G)) {
            const T *row[N];
            float s[N] = {};
            int some = -1, v[N];
#pragma unroll
            for (int j = 0; j < N; ++j) {
                v[j] = j0 + j < end ? which(j0 + j) : -1;
                if (G == 64) v[j] = __builtin_amdgcn_readfirstlane(v[j]);
                some = max(some, v[j]);
            }
#pragma unroll
            for (int j = 0; j < N; ++j) row[j] = w + (int64_t)max(v[j] < 0 ? some : v[j], 0) * width;      // one that is none repeats another, or the first
            distill_dots<G>(x + t * width, row, some < 0 ? 0 : width, threadIdx.x % G, s);
#pragma unroll
            for (int j = 0; j < N; ++j)
                if (threadIdx.x % G == 0 && j0 + j < end) out[j0 + j] = s[j] / heat;
        }
    };
    // a wave to an entry where the row has its 16 bytes for every lane, else a quarter of one: 64 rows, 99 entries, 160 columns, bf16 13.5 us, with waves 22.6;
    // 1320 rows, 69 entries, 4000 columns 70 and 50
    const auto entry = [&](int j) { return at[j]; };
    using std::integral_constant;
    const integral_constant<int, 16> quarter;
    const integral_constant<int, 64> whole_wave;
    if (width * (int64_t)sizeof(T) >= 1024) {
        if (top >= 32) dots(top, whole_wave, integral_constant<int, 4>(), entry, z);
        else if (top >= 16) dots(top, whole_wave, integral_constant<int, 2>(), entry, z);
        else dots(top, whole_wave, integral_constant<int, 1>(), entry, z);
    } else if (top >= 48) dots(top, quarter, integral_constant<int, 2>(), entry, z);
    else dots(top, quarter, integral_constant<int, 1>(), entry, z);
    if (tail) dots(tail, quarter, integral_constant<int, 1>(), [&](int i) { return vocab - tail + i; }, last);
    if (joins) {
        const float m = wave_max(a.m);
        a = Soft{m, wave_sum(a.m == -INFINITY ? a.s : a.s * exp_of(a.m - m))};
        if (l == 0) joined[wave] = a;
    }
    __syncthreads();
    if (wave) return;
    // the rest is one wave's
    float ls;
    if (joins) {
        a = joined[0];
#pragma unroll
        for (int i = 1; i < DISTILL_WAVES; ++i) a = soft_join(a, joined[i]);
    } else {
        ls = lse[t];
        a = ls == INFINITY ? Soft{3.4028235e38f, INFINITY} : Soft{ls, ls == -INFINITY ? 0.f : 1.f};
    }
    if (joins || tail) {
        for (int j = 0; j < tail; ++j) a = soft_join(a, last[j] == INFINITY ? Soft{3.4028235e38f, INFINITY} : Soft{last[j], 1.f});
        ls = a.m + logf(a.s);
        if (l == 0) lse[t] = ls;
    }
    // log p = (target - most) / T - norm; the difference first, so that the lowest numbers of all do not become infinite
    float most = 0.f, norm;
    if (target_lse) norm = target_lse[t];
    else {
        most = -INFINITY;
        for (int j = l; j < top; j += 64)
            if (at[j] >= 0) most = fmaxf(most, target[j]);
        most = wave_max(most);
        float sum = 0.f;
        for (int j = l; j < top; j += 64)
            if (at[j] >= 0 && target[j] != -INFINITY) sum += expf((target[j] - most) / heat);
        norm = logf(wave_sum(sum));
    }
    float loss = 0.f, m = 0.f;
    for (int j = l; j < top; j += 64) {
        // an entry of weight 0 adds nothing, whatever the row's logits are
        const float logp = (target[j] - most) / heat - norm, pj = at[j] < 0 || target[j] == -INFINITY ? 0.f : expf(logp);
        p[j] = pj;
        m += pj;
        if (pj != 0.f) loss += pj * (logp + (ls - z[j]));
    }
    loss = wave_sum(loss);
    m = wave_sum(m);
    __builtin_amdgcn_wave_barrier();       // p is read by other lanes than wrote it
    const bool search = __builtin_amdgcn_readfirstlane(twice);
    for (int j = l; j < top; j += 64) {
        float d = 0.f;
        if (at[j] >= 0 && m != 0.f) {
            float same = p[j];
            if (search) {
                same = 0.f;
                for (int i = 0; i < whole; i += 4) {
                    const int4 v = *(const int4 *)(at + i);
                    const float4 q = *(const float4 *)(p + i);
                    same += v.x == at[j] ? q.x : 0.f;
                    same += v.y == at[j] ? q.y : 0.f;
                    same += v.z == at[j] ? q.z : 0.f;
                    same += v.w == at[j] ? q.w : 0.f;
                }
            }
            d = m * expf(z[j] - ls) - same;
        }
        delta[t * top + j] = d;
    }
    if (l) return;
    mass[t] = m;
    row_loss[t] = loss;
}
// the rows with weight, and the sum of their losses (row_loss may be null), in the first thread of a workgroup of 64 * WAVES; in a fixed order
template <int WAVES>
__device__ __forceinline__ int distill_count(const float *row_loss, const float *mass, int rows, double &sum) {
    __shared__ double sums[WAVES];
    __shared__ int counts[WAVES];
    int count = 0;
    sum = 0;
    constexpr int AHEAD = 8;       // rows of a thread whose loads are under way together
    for (int t0 = threadIdx.x; t0 < rows; t0 += 64 * WAVES * AHEAD) {
        float m[AHEAD], v[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int t = t0 + 64 * WAVES * i;
            m[i] = t < rows ? mass[t] : 0.f;
            v[i] = row_loss && t < rows ? row_loss[t] : 0.f;
        }
#pragma unroll
        for (int i = 0; i < AHEAD; ++i)
            if (m[i] != 0.f) { ++count; sum += v[i]; }
    }
    for (int k = 32; k; k /= 2) { sum += __shfl_xor(sum, k); count += __shfl_xor(count, k); }
    if (threadIdx.x % 64 == 0) { sums[threadIdx.x / 64] = sum; counts[threadIdx.x / 64] = count; }
    __syncthreads();
    sum = 0;
    count = 0;
    for (int i = 0; i < WAVES; ++i) { sum += sums[i]; count += counts[i]; }
    return count;
}
// T^2 times the mean of the losses of the rows with weight
__global__ __launch_bounds__(1024) void distill_mean_kernel(const float *__restrict__ row_loss, const float *__restrict__ mass, int rows, float heat,
                                                            float *__restrict__ loss) {
    double sum;
    const int count = distill_count<16>(row_loss, mass, rows, sum);
    if (threadIdx.x == 0) *loss = count ? (float)((double)heat * heat * sum / count) : 0.f;
}
__global__ __launch_bounds__(1024) void distill_inv_kernel(const float *__restrict__ mass, int rows, float heat, float *__restrict__ inv) {
    double sum;
    const int count = distill_count<16>(nullptr, mass, rows, sum);
    if (threadIdx.x == 0) *inv = count ? heat / count : 0.f;
}
// bf16: the teacher's entries of a piece, over what the product's epilogue wrote there.  An index that comes twice has the same delta twice.
__global__ __launch_bounds__(256) void distill_entries_kernel(const int32_t *__restrict__ index, const float *__restrict__ delta, int64_t n, int top, int v0,
                                                              int piece, unsigned short *__restrict__ dl, int64_t ld) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
        const int64_t v = (int64_t)index[i] - v0;
        if (v >= 0 && v < piece) dl[i / top * ld + v] = float_bf16(delta[i]);
    }
}
// fp32: dl in the place of a row's 256 logits, then the teacher's entries among them.  COUNT: with up to 64 rows every workgroup counts those with
// weight itself, a launch less (777 rows, 16000 entries: 52 us so, 26 without).
template <bool COUNT>
__global__ __launch_bounds__(256) void distill_piece_grad_kernel(float *__restrict__ logits, int piece, int v0, const float *__restrict__ mass,
                                                                 const float *__restrict__ lse, const int32_t *__restrict__ index,
                                                                 const float *__restrict__ delta, int top, const float *__restrict__ inv, int rows, float heat) {
    const int64_t t = blockIdx.x;
    const int from = blockIdx.y * 256, to = min(piece, from + 256), v = from + threadIdx.x;
    const float m = mass[t], by = 1.f / heat;
    float *row = logits + t * piece;
    const float x = v < to ? row[v] : 0.f;
    float f;
    if (COUNT) {
        double sum;
        const int count = distill_count<4>(nullptr, mass, rows, sum);
        f = count ? heat / count : 0.f;
    } else
        f = *inv;
    if (v < to) row[v] = m != 0.f ? m * exp_of(x * by - lse[t]) * f : 0.f;
    __syncthreads();
    for (int j = threadIdx.x; j < top; j += 256) {
        const int64_t e = (int64_t)index[t * top + j] - v0;
        if (e >= from && e < to) row[e] = delta[t * top + j] * f;
    }
}

// fp32: the `tail` entries that a large vocabulary has over a multiple of 16, from v0 on.  As a piece of their own they took six launches of the matrix
// products, mostly empty tiles: both passes of 100 rows, 512 columns, 5003 entries 149 us, with these kernels 101; 777 rows, 1000 columns, 16001 entries
// 819 and 767.  A workgroup to a row: their logits, dl (kept for dw), and their share of dx, which is there already.
__global__ __launch_bounds__(256) void distill_tail_kernel(const float *__restrict__ x, const float *__restrict__ w, const int32_t *__restrict__ index,
                                                           const float *__restrict__ lse, const float *__restrict__ mass, const float *__restrict__ delta,
                                                           const float *__restrict__ inv, float *__restrict__ dl, float *__restrict__ dx, int rows, int width,
                                                           int v0, int tail, int top, float heat) {
    __shared__ float d[DISTILL_TAIL];
    static_assert(DISTILL_TAIL == 256 / 16, "");
    const int64_t t = blockIdx.x;
    const float m = mass[t], f = *inv;
    x += t * width;
    w += (int64_t)v0 * width;
    // 16 lanes to an entry, or, of up to four, a wave
    const auto entry = [&](auto lanes) {
        constexpr int G = decltype(lanes)::value;
        const int j = threadIdx.x / G;
        const float *row[1] = {w + (int64_t)min(j, tail - 1) * width};
        float s[1] = {};
        if (m != 0.f) distill_dots<G>(x, row, width, threadIdx.x % G, s);
        if (threadIdx.x % G == 0) d[j] = m != 0.f && j < tail ? m * expf(s[0] / heat - lse[t]) * f : 0.f;
    };
    if (tail > 4) entry(std::integral_constant<int, 16>());
    else {
        if (threadIdx.x >= 4 && threadIdx.x < DISTILL_TAIL) d[threadIdx.x] = 0.f;
        entry(std::integral_constant<int, 64>());
    }
    __syncthreads();
    for (int j = threadIdx.x; j < top; j += 256) {
        const int64_t e = (int64_t)index[t * top + j] - v0;
        if (e >= 0 && e < tail) d[e] = delta[t * top + j] * f;
    }
    __syncthreads();
    if (threadIdx.x < DISTILL_TAIL) dl[t * DISTILL_TAIL + threadIdx.x] = d[threadIdx.x];
    for (int c = threadIdx.x; c < width; c += 256) {
        float sum = dx[t * width + c];
        for (int j = 0; j < tail; ++j) sum = fmaf(d[j], w[(int64_t)j * width + c], sum);
        dx[t * width + c] = sum;
    }
}
// 64 columns of dw's last rows over a range of rows (grid y), or, of the only range, the result
__global__ __launch_bounds__(256) void distill_tail_wgrad_kernel(const float *__restrict__ x, const float *__restrict__ dl, int64_t rows, int64_t per, int width, int tail,
                                                                 float *__restrict__ part) {
    __shared__ float sums[4][DISTILL_TAIL][64];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), l = threadIdx.x & 63, c = blockIdx.x * 64 + l;
    const int64_t from = blockIdx.y * per, to = min(rows, from + per);
    float acc[DISTILL_TAIL] = {};
#pragma unroll 4
    for (int64_t t = from + wave; t < to; t += 4) {
        const float v = x[t * width + min(c, width - 1)];
#pragma unroll
        for (int j = 0; j < DISTILL_TAIL; ++j) acc[j] = fmaf(dl[t * DISTILL_TAIL + j], v, acc[j]);
    }
#pragma unroll
    for (int j = 0; j < DISTILL_TAIL; ++j) sums[wave][j][l] = acc[j];
    __syncthreads();
    if (c >= width) return;
    for (int j = wave; j < tail; j += 4)
        part[((int64_t)blockIdx.y * tail + j) * width + c] = (sums[0][j][l] + sums[1][j][l]) + (sums[2][j][l] + sums[3][j][l]);
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

// out (+)= the sum over the ranges of part, in a fixed order: sixteen waves take a share of the ranges each.  T bf16: times *by, rounded.
template <class T = float>
__global__ __launch_bounds__(1024) void ce_few_rows_join_kernel(const float *__restrict__ part, int ranges, int n, T *__restrict__ out, int add, const float *by = nullptr) {
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
    if constexpr (std::is_same<T, float>::value) out[i] = add ? out[i] + sum : sum;
    else out[i] = float_bf16((add ? bf16_float(out[i]) : 0.f) + sum * *by);
}

int64_t up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }
int64_t cut(int64_t n, int64_t by) { return (n + by - 1) / by; }

constexpr int64_t CE_PIECE_BYTES = 256ll << 20;      // a piece of logits or of their gradient

// Results of few tiles leave CUs idle while their reduction is long: as many ranges as fill the card, of at least `least` indices.
int ce_splits(int64_t tiles, int64_t red, int64_t least, int64_t most = 16) {
    return (int)std::max<int64_t>(1, std::min<int64_t>({256 / std::max<int64_t>(tiles, 1), red / least, most}));
}

// Ranges of the reduction over a piece in dx = dl W.  Large tiles (gemm_tile) where ranges of 4096 entries or more make whole rounds of one to a CU
// (a range's fp32 sums cost 8 bytes of traffic for each result) and few of their entries lie outside the result: backward pass of 512 rows,
// 2048 columns, 100000 entries 830 us, with small tiles 997; 4096 rows, 2048 columns, 50176 entries 2459 and 2542.  Small ones otherwise:
// 4000 rows, 1600 columns, 50257 entries (112 large tiles; three ranges are 1.3 rounds) 2126 us, with large ones 2248.
int ce_input_ranges(int64_t rows, int64_t width, int piece, int64_t most) {
    const int64_t large = cut(width, 256) * cut(rows, 256), ranges = cut(256, large);
    if (ranges <= 16 && piece / ranges >= 4096 && 5 * rows * width * ranges >= 4 * 65536 * up(large * ranges, 256)) return (int)ranges;
    return ce_splits(cut(width, 128) * cut(rows, 128), piece, 512, most);
}

// How a call goes through the vocabulary, and its workspace: forward [hit][row_loss][part][product][logits (fp32)], backward
// [inv][dx parts (bf16) or product][dl].
struct CePlan {
    int rows, width, vocab;
    bool bf16;
    int unit = 0;                   // bf16 forward: logits to a part
    int piece = 0;                  // logits of a piece
    int64_t most = 16;              // ranges of the reduction over a piece in dx, at most
    int ranges = 1, chunk = 0;      // bf16 backward: those ranges
    int64_t product = 0;            // fp32: bytes for the products' partial results
    int64_t fixed = 0, per_col = 0;              // bytes without the pieces, and for each logit of a piece

    int64_t bytes() const { return fixed + per_col * piece; }
    int wgrad_splits(int piece) const { return ce_splits(cut(width, 128) * cut(piece, 128), rows, 64); }
    // fp32: ranges in dx where its tiles are so few that `most` of them do not fill the card; 1: what the product chooses by itself, 16 at most.  205 rows, 80
    // columns, 82288 entries: the product 49 us, in 16 ranges 163.  Not where that is fewer: 100 rows, 128 columns, 2000 entries backward 29 us, in 3 ranges
    // of 512 entries or more 45
    int dgrad_splits(int piece) const {
        const int64_t tiles = cut(rows, 128) * (width <= 64 ? 1 : cut(width, 128));
        const int splits = most > 16 && !few_rows(piece) ? ce_splits(tiles, piece, 512, most) : 1;
        return splits > 16 ? splits : 1;
    }
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

CePlan ce_plan(bool grad, int dtype, int64_t rows, int width, int vocab, int64_t most = 16) {
    if (dtype != MONET_F32 && dtype != MONET_BF16) throw KernelError("linear_ce: dtype must be MONET_F32 or MONET_BF16");
    if (rows < 1 || width < 1 || vocab < 1) throw KernelError("linear_ce: bad shape");
    const bool bf16 = dtype == MONET_BF16;
    if (bf16 && width % 8) throw KernelError("linear_ce: bf16 needs a width that is a multiple of 8");
    if (rows >= (1 << 24) || width > (1 << 20) || vocab > (1 << 28)) throw KernelError("linear_ce: shape too large");
    CePlan p{(int)rows, width, vocab, bf16};
    p.most = most;
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
        p.ranges = ce_input_ranges(rows, width, p.piece, most);
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
            if (p.dgrad_splits((int)piece) > 1) p.product = std::max(p.product, p.dgrad_splits((int)piece) * rows * width * 4);
            if (p.few_rows((int)piece)) p.product = std::max(p.product, cut(piece, p.few_per((int)piece)) * rows * width * 4);
        }
        p.product = up(p.product, 256);
        p.fixed += p.product;
    }
    return p;
}

void check_ws(const CePlan &p, const void *ws, size_t ws_bytes, int64_t front = 0) {
    if (!ws || (int64_t)ws_bytes < front + p.bytes())
        throw KernelError("linear_ce: workspace of " + std::to_string(ws_bytes) + " bytes, " + std::to_string(front + p.bytes()) + " needed");
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

// the parts of lse (and the labels' logits) of all logits, which are `by` times the products where there are no labels
// (part null: the logits alone, of the only piece)
template <bool LABELS>
void vocab_stats(hipStream_t st, const CePlan &p, const void *x, const void *w, const int32_t *labels, float2 *part, float *hit, float by, void *ws) {
    if (p.bf16) {
        gemm_bf16<false, false>(st, ce_logits_shape(p, x, w, 0, p.vocab), StatsEpilogue<LABELS>{labels, part, hit, p.rows, p.vocab, by}, "linear_ce logits launch");
        return;
    }
    float *logits = (float *)((char *)ws + p.fixed), *product = p.product ? (float *)((char *)logits - p.product) : nullptr;
    const std::vector<int> at = p.pieces();
    int64_t done = 0;      // parts
    for (size_t i = 0; i + 1 < at.size(); ++i) {
        const int piece = at[i + 1] - at[i], segments = (int)cut(piece, CE_SEGMENT);
        const float *wp = (const float *)w + (int64_t)at[i] * p.width;
        if (!ce_few_logits(st, (const float *)x, wp, p.width, p.rows, piece, logits))
            conv_fwd(st, (const float *)x, wp, logits, ce_conv_shape(p, piece), 1, product, (size_t)p.product);
        if (!LABELS && !part) continue;
        hipLaunchKernelGGL(ce_piece_stats_kernel<LABELS>, dim3(p.rows, segments), dim3(256), 0, st, logits, piece, at[i], labels, part + done * p.rows, hit, by);
        hip_check(hipGetLastError(), "linear_ce statistics launch");
        done += segments;
    }
}

// dx and dw, a piece of the logits' gradient dl at a time.  grad_bf16(g, d, ld, v0, piece) launches the product g with an epilogue that leaves dl / *inv
// in d, rows ld apart; grad_f32(d, v0, piece) puts dl in the place of the logits d.
template <class GradBf16, class GradF32>
void vocab_gradients(hipStream_t st, const CePlan &p, const void *x, const void *w, void *dx, void *dw, bool accumulate, void *ws, const float *inv,
                     GradBf16 &&grad_bf16, GradF32 &&grad_f32) {
    const int64_t rows = p.rows;
    const int width = p.width;
    const std::vector<int> at = p.pieces();
    char *dl = (char *)ws + p.fixed;
    float *parts = (float *)((char *)ws + 256);
    for (size_t i = 0; i + 1 < at.size(); ++i) {
        const int v0 = at[i], piece = at[i + 1] - v0;
        if (p.bf16) {
            unsigned short *d = (unsigned short *)dl;
            const int64_t ld = up(piece, 8);
            grad_bf16(ce_logits_shape(p, x, w, v0, piece), d, ld, v0, piece);
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
                    if (p.ranges > 16)      // few results: 64 rows, 160 columns in 64 ranges 20 us with a thread to eight of them
                        hipLaunchKernelGGL(ce_few_rows_join_kernel<unsigned short>, dim3((unsigned)cut(n, 64)), dim3(1024), 0, st, parts, p.ranges, (int)n,
                                           (unsigned short *)dx, accumulate, (const float *)inv);
                    else
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
            grad_f32(d, v0, piece);
            if (p.few_rows(piece)) {
                const int per = p.few_per(piece), ranges = (int)cut(piece, per), n = p.rows * width;
                const dim3 grid((unsigned)cut(width, 256), ranges);
                if (rows <= 4)
                    hipLaunchKernelGGL(ce_few_rows_kernel<4>, grid, dim3(256), 0, st, d, piece, wp, width, p.rows, per, product);
                else
                    hipLaunchKernelGGL(ce_few_rows_kernel<CE_FEW_ROWS>, dim3(grid.x, grid.y, (unsigned)cut(rows, CE_FEW_ROWS)), dim3(256), 0, st, d, piece, wp, width, p.rows, per, product);
                hip_check(hipGetLastError(), "linear_ce input gradient launch");
                hipLaunchKernelGGL(ce_few_rows_join_kernel<float>, dim3((unsigned)cut(n, 64)), dim3(1024), 0, st, product, ranges, n, (float *)dx, accumulate || i > 0, (const float *)nullptr);
                hip_check(hipGetLastError(), "linear_ce input gradient sum launch");
            } else {
                conv_dgrad(st, d, wp, (float *)dx, cs, accumulate || i > 0, p.dgrad_splits(piece), product, product_bytes);
            }
            const int splits = p.wgrad_splits(piece);
            conv_wgrad(st, (const float *)x, d, (float *)dw + (int64_t)v0 * width, cs, splits, splits > 1 ? product : nullptr, splits > 1 ? product_bytes : 0);
        }
    }
}

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
    vocab_stats<true>(st, p, x, w, labels, part, hit, 1.f, ws);
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
    vocab_gradients(st, p, x, w, dx, dw, accumulate, ws, inv,
        [&](const GemmShape &g, unsigned short *d, int64_t ld, int v0, int piece) {
            gemm_bf16<false, false>(st, g, CeGradEpilogue{labels, lse, d, ld, p.rows, piece, v0, vocab}, "linear_ce gradient launch");
        },
        [&](float *d, int v0, int piece) {
            hipLaunchKernelGGL((count ? ce_piece_grad_kernel<false> : ce_piece_grad_kernel<true>), dim3(p.rows, (unsigned)cut(piece, 256)), dim3(256), 0, st, d, piece, v0,
                               labels, lse, inv, p.rows, vocab);
            hip_check(hipGetLastError(), "linear_ce gradient launch");
        });
}

namespace {
// The entries that the matrix products do not take: with a piece that is no multiple of 16 they read value by value.  Both passes, us, those entries among
// the others and in kernels of their own: 24 rows, 128 columns, 1009 entries 49 and 56; 64, 256 and 1009 59 and 58; 300, 512 and 1001 88 and 80; 690,
// 3856 and 539 244 and 208; 2000, 2000 and 4001 1477 and 928.
int distill_tail(int dtype, int64_t rows, int width, int vocab) {
    const bool large = vocab > 4096 || (vocab >= 64 && rows * width * vocab >= 1 << 24);
    return dtype == MONET_F32 && large ? vocab % DISTILL_TAIL : 0;
}
CePlan distill_plan(bool grad, int dtype, int64_t rows, int width, int vocab, int top) {
    if (top < 1 || top > DISTILL_TOP) throw KernelError("linear_distill: 1 to " + std::to_string(DISTILL_TOP) + " entries a row");
    if (rows < 1 || width < 1 || vocab < 1) throw KernelError("linear_distill: bad shape");
    return ce_plan(grad, dtype, rows, width, vocab - distill_tail(dtype, rows, width, vocab), 64);
}
int64_t distill_tail_ranges(int64_t rows) { return std::max<int64_t>(1, std::min<int64_t>(64, rows / 64)); }
// bytes in front of the plan's: dl of the tail, and dw's parts if there are several
int64_t distill_tail_bytes(bool grad, int dtype, int64_t rows, int width, int vocab) {
    const int64_t tail = distill_tail(dtype, rows, width, vocab), ranges = distill_tail_ranges(rows);
    if (!grad || !tail) return 0;
    return up(rows * DISTILL_TAIL * 4, 256) + (ranges > 1 ? up(ranges * tail * width * 4, 256) : 0);
}
void distill_check(float heat) {
    if (!(heat > 0.f) || !std::isfinite(heat) || !std::isfinite(1.f / heat)) throw KernelError("linear_distill: the temperature must be positive and finite");
}
}  // namespace

size_t linear_distill_workspace_bytes(bool grad, int dtype, int64_t rows, int width, int vocab, int top) {
    const int64_t forward = distill_plan(false, dtype, rows, width, vocab, top).bytes();
    return (size_t)std::max(forward, distill_plan(grad, dtype, rows, width, vocab, top).bytes() + distill_tail_bytes(grad, dtype, rows, width, vocab));
}

void linear_distill_fwd(hipStream_t st, int dtype, const void *x, const void *w, const int32_t *index, const float *target, const float *target_lse,
                        float *loss, float *lse, float *mass, float *delta, int64_t rows, int width, int vocab, int top, float heat, void *ws,
                        size_t ws_bytes) {
    const CePlan p = distill_plan(false, dtype, rows, width, vocab, top);
    distill_check(heat);
    check_ws(p, ws, ws_bytes);
    check_aligned(p, {x, w});
    check_words({index, target, loss, lse, mass, delta});
    if ((uintptr_t)target_lse % 4) throw KernelError("linear_distill: target_lse must be 4-byte aligned");
    float *row_loss = (float *)ws;
    float2 *part = (float2 *)(row_loss + 2 * up(rows, 64));
    // fp32: logits that a row's workgroup takes in one step of its loads need no launch for their statistics (24 rows, 128 columns, 1009 entries, both passes 47 us,
    // with one 50); of more, that launch has them from more workgroups (348 rows, 63168: 113 us together, the rows alone 128)
    const bool direct = !p.bf16 && p.pieces().size() == 2 && p.piece <= 4096;
    if (direct) part = nullptr;
    vocab_stats<false>(st, p, x, w, nullptr, part, nullptr, 1.f / heat, ws);
    // a row's workgroup joins its parts itself, a launch less, where reading 8 bytes from each of as many lines costs little
    const int parts = (int)p.parts();
    const bool merged = !direct && rows * parts > 1 << 19;
    if (merged) {
        hipLaunchKernelGGL((ce_merge_kernel<16, false>), dim3((unsigned)cut(rows, 16)), dim3(256), 0, st, part, parts, nullptr, nullptr, lse, nullptr, nullptr, p.rows, vocab);
        hip_check(hipGetLastError(), "linear_distill merge launch");
    }
    const auto rows_kernel = [&](auto t) {
        using T = decltype(t);
        hipLaunchKernelGGL(distill_rows_kernel<T>, dim3(p.rows), dim3(64 * DISTILL_WAVES), 0, st, (const T *)x, (const T *)w, index, target, target_lse,
                           merged ? nullptr : part, parts, direct ? (const float *)((char *)ws + p.fixed) : nullptr, p.piece, p.rows, lse, mass, delta, row_loss, width, vocab, distill_tail(dtype, rows, width, vocab), top, heat);
        hip_check(hipGetLastError(), "linear_distill rows launch");
    };
    if (p.bf16) rows_kernel((unsigned short)0);
    else rows_kernel(0.f);
    hipLaunchKernelGGL(distill_mean_kernel, dim3(1), dim3(1024), 0, st, row_loss, mass, p.rows, heat, loss);
    hip_check(hipGetLastError(), "linear_distill mean launch");
}

void linear_distill_bwd(hipStream_t st, int dtype, const void *x, const void *w, const int32_t *index, const float *lse, const float *mass,
                        const float *delta, void *dx, void *dw, int64_t rows, int width, int vocab, int top, float heat, bool accumulate, void *ws,
                        size_t ws_bytes) {
    const CePlan p = distill_plan(true, dtype, rows, width, vocab, top);
    const int64_t front = distill_tail_bytes(true, dtype, rows, width, vocab);
    const int tail = distill_tail(dtype, rows, width, vocab);
    distill_check(heat);
    check_ws(p, ws, ws_bytes, front);
    check_aligned(p, {x, w, dx, dw});
    check_words({index, lse, mass, delta});
    float *dl = (float *)ws;
    ws = (char *)ws + front;
    float *inv = (float *)ws;
    const bool count = p.bf16 || rows > 64 || tail;
    if (count) {
        hipLaunchKernelGGL(distill_inv_kernel, dim3(1), dim3(1024), 0, st, mass, p.rows, heat, inv);
        hip_check(hipGetLastError(), "linear_distill count launch");
    }
    vocab_gradients(st, p, x, w, dx, dw, accumulate, ws, inv,
        [&](const GemmShape &g, unsigned short *d, int64_t ld, int v0, int piece) {
            gemm_bf16<false, false>(st, g, DistillGradEpilogue{mass, lse, d, ld, p.rows, piece, 1.f / heat}, "linear_distill gradient launch");
            const int64_t n = rows * top;
            hipLaunchKernelGGL(distill_entries_kernel, dim3((unsigned)std::min<int64_t>(cut(n, 256), 1 << 16)), dim3(256), 0, st, index, delta, n, top, v0, piece, d, ld);
            hip_check(hipGetLastError(), "linear_distill entries launch");
        },
        [&](float *d, int v0, int piece) {
            hipLaunchKernelGGL((count ? distill_piece_grad_kernel<false> : distill_piece_grad_kernel<true>), dim3(p.rows, (unsigned)cut(piece, 256)), dim3(256), 0, st,
                               d, piece, v0, mass, lse, index, delta, top, inv, p.rows, heat);
            hip_check(hipGetLastError(), "linear_distill gradient launch");
        });
    if (!tail) return;
    hipLaunchKernelGGL(distill_tail_kernel, dim3(p.rows), dim3(256), 0, st, (const float *)x, (const float *)w, index, lse, mass, delta, inv, dl, (float *)dx, p.rows,
                       width, vocab - tail, tail, top, heat);
    hip_check(hipGetLastError(), "linear_distill tail launch");
    const int64_t ranges = distill_tail_ranges(rows);
    float *out = (float *)dw + (int64_t)(vocab - tail) * width, *part = ranges > 1 ? dl + up(rows * DISTILL_TAIL, 64) : out;
    hipLaunchKernelGGL(distill_tail_wgrad_kernel, dim3((unsigned)cut(width, 64), (unsigned)ranges), dim3(256), 0, st, (const float *)x, dl, rows, cut(rows, ranges), width,
                       tail, part);
    hip_check(hipGetLastError(), "linear_distill tail launch");
    if (ranges == 1) return;
    hipLaunchKernelGGL(ce_few_rows_join_kernel<float>, dim3((unsigned)cut((int64_t)tail * width, 64)), dim3(1024), 0, st, part, (int)ranges, tail * width, out, 0, (const float *)nullptr);
    hip_check(hipGetLastError(), "linear_distill tail launch");
}


}  // namespace monet
