// Layer norm over rows of x [rows][cols]:
//   mean = sum x / cols,  rstd = 1 / sqrt(sum (x - mean)^2 / cols + eps),  xh = (x - mean) rstd,  y = xh gamma + beta.
// Backward, with g = dy gamma:
//   dx = rstd (g - sum g / cols - xh sum(g xh) / cols),  dgamma = sum over rows of dy xh,  dbeta = sum over rows of dy.
// A mean m from an fp32 sum is off by the sum's rounding, a few 2^-24 of it, which matters where the deviation is much smaller.  Rows with m^2 >= 16 var take a
// third sum over d = x - m, mean = m + sum d / cols and var = sum d^2 / cols - (sum d / cols)^2: equal values are their own mean (48 of 1000.1 with eps 1e-5:
// xh 0, without it 0.02).  In the other rows the mean's error is at most that of five values of a deviation's size.  The comparison costs 2 % of 4096 x 16384
// in bf16; the third sum in all rows cost 9 %.
// Bound by memory: forward reads x and writes y, backward reads dy and x and writes dx.  All sums are fp32; a result is rounded once.
#include <cmath>
#include <type_traits>

#include "../../include/monet_kernels.h"
#include "kernels.hpp"
#include "tile_bf16.hpp"
#include "wave_sum.hpp"

namespace monet {

namespace {

__device__ __forceinline__ void put(float *p, float v, bool add) { *p = add ? *p + v : v; }
__device__ __forceinline__ void put(unsigned short *p, float v, bool add) { *p = float_bf16(add ? bf16_float(*p) + v : v); }

// ---- rows that fit the registers: L lanes to a row (4, 16 or whole waves), each with CH pieces of 16 bytes
template <class T> constexpr int VEC = 16 / sizeof(T);
template <class T, int L, int CH> constexpr int CAPACITY = L * VEC<T> * CH;

// 16 bytes at any address of an element: rows of odd length begin anywhere, and one such load is what aligned ones cost
typedef unsigned uintx4_at2 __attribute__((ext_vector_type(4), aligned(2)));
typedef unsigned uintx4_at4 __attribute__((ext_vector_type(4), aligned(4)));
__device__ __forceinline__ uintx4 load16(const float *p) { return *(const uintx4_at4 *)p; }
__device__ __forceinline__ uintx4 load16(const unsigned short *p) { return *(const uintx4_at2 *)p; }
__device__ __forceinline__ void store16(float *p, uintx4 v) { *(uintx4_at4 *)p = v; }
__device__ __forceinline__ void store16(unsigned short *p, uintx4 v) { *(uintx4_at2 *)p = v; }
__device__ __forceinline__ void unpack(uintx4 v, float (&f)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(v[i]);
}
__device__ __forceinline__ void unpack(uintx4 v, float (&f)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(v[i] << 16); f[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u); }
}
__device__ __forceinline__ uintx4 pack(const float (&f)[4]) {
    uintx4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = __float_as_uint(f[i]);
    return v;
}
__device__ __forceinline__ uintx4 pack(const float (&f)[8]) {
    uintx4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = pack_bf16(f[2 * i], f[2 * i + 1]);
    return v;
}
// A lane's piece of a row.  WHOLE: rows are whole pieces.  MOVED: the last piece is moved back to the row's end (values that two lanes hold are added once,
// and stored twice alike, where a row is in registers before any of it is stored).  SHORT: the row is shorter than a piece and goes value by value.  A piece
// behind the end: nothing.
enum { WHOLE, MOVED, SHORT };
template <class T, int ROWS>
struct Piece {
    int c, from, to;        // values from .. to - 1 count
    bool has;
    __device__ __forceinline__ Piece(int at, int cols) : c(at), from(0), to(VEC<T>), has(at < cols) {
        if (ROWS == MOVED && at + VEC<T> > cols) { c = cols - VEC<T>; from = at - c; }
        if (ROWS == SHORT) to = cols - at;
    }
    __device__ __forceinline__ bool counts(int e) const { return (ROWS != MOVED || e >= from) && (ROWS != SHORT || e < to); }
    __device__ __forceinline__ uintx4 load(const T *row) const {
        if (ROWS != SHORT) return has ? load16(row + c) : uintx4{};
        T v[VEC<T>] = {};
#pragma unroll
        for (int e = 0; e < VEC<T>; ++e)
            if (e < to) v[e] = row[c + e];
        return __builtin_bit_cast(uintx4, v);
    }
    __device__ __forceinline__ float once(float v, int e) const { return counts(e) ? v : 0.f; }
    // alone: a moved piece stores only the values that count, which nobody else reads or stores
    __device__ __forceinline__ void store(T *row, const float (&f)[VEC<T>], bool add, bool alone = false) const {
        if (!has) return;
        if (ROWS != SHORT && !add && !(alone && from)) { store16(row + c, pack(f)); return; }
#pragma unroll
        for (int e = 0; e < VEC<T>; ++e)
            if (counts(e)) put(row + c + e, f[e], add);
    }
    __device__ __forceinline__ void params(const void *p, bool bf16, float missing, float (&f)[VEC<T>]) const {
#pragma unroll
        for (int e = 0; e < VEC<T>; ++e) f[e] = has ? missing : 0.f;
        if (!p || !has) return;
        if (ROWS == SHORT) {
#pragma unroll
            for (int e = 0; e < VEC<T>; ++e)
                if (e < to) f[e] = bf16 ? bf16_float(((const unsigned short *)p)[c + e]) : ((const float *)p)[c + e];
        } else if (bf16) {
            typedef unsigned short half __attribute__((ext_vector_type(VEC<T>)));
            half v;
            __builtin_memcpy(&v, (const unsigned short *)p + c, sizeof v);
#pragma unroll
            for (int e = 0; e < VEC<T>; ++e) f[e] = bf16_float(v[e]);
        } else
            __builtin_memcpy(f, (const float *)p + c, sizeof f);
    }
};

// the sum of the L lanes of a row; `at`: this group's and this sum's place in LDS, not used again before the next barrier but one
template <int L>
__device__ __forceinline__ float group_sum(float v, float *at, int wave) {
    if (L == 4) return quad_sum(v);
    if (L == 16) return row_sum(v);
    v = wave_sum(v);
    if (L == 64) return v;
    if ((threadIdx.x & 63) == 0) at[wave] = v;
    __syncthreads();
    v = at[0];
#pragma unroll
    for (int i = 1; i < L / 64; ++i) v += at[i];
    return v;
}
__device__ __forceinline__ bool far_from_zero(float mean, float var) { return mean * mean >= 16.f * var; }
// the mean and the variance with the mean deviation that was left; a variance beyond fp32 stays
__device__ __forceinline__ void shift(float &mean, float &var, float off) {
    mean += off;
    if (var < INFINITY) var = fmaxf(var - off * off, 0.f);
}
// which of a workgroup's rows a thread works on: the same for a wave where it has a wave or more
template <int L>
__device__ __forceinline__ int group_of() {
    return L >= 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x / 64) / (L / 64) : threadIdx.x / L;
}
template <int L> constexpr int WAVES_OF = L < 64 ? 1 : L / 64;      // of a row

// A workgroup walks over rows with gamma and beta in registers, the next row's loads under way while this one's mean, deviations from it and results are
// computed: two passes over registers, one over memory.  16384 x 4096, bf16: 47 us (5.7 TB/s); with gamma and beta loaded value by value for every row 147;
// a row read three times, value by value, 128.  1023 x 12289, fp32: 21 us (4.7 TB/s).  Short rows share a wave: 327680 x 128, bf16, 16 lanes each 29 us,
// a wave each 82.  Rows of two waves have a workgroup of their own, since only some rows take a third sum behind its barrier: 16384 x 2048, bf16: 24.4 us, two rows to
// a workgroup and no third sum 24.1.
template <int L> constexpr int FWD_THREADS = L <= 64 ? 256 : L;

template <class T, int L, int CH, int ROWS>
__global__ __launch_bounds__(FWD_THREADS<L>) void layernorm_rows_kernel(const T *x, const void *__restrict__ gamma, const void *__restrict__ beta, bool params_bf16,
                                                                        T *y, float2 *__restrict__ stats, int64_t rows, int cols, int64_t x_ld, int64_t y_ld,
                                                                        float eps) {
    constexpr int V = VEC<T>, GROUPS = FWD_THREADS<L> / L;
    __shared__ float sums[3][GROUPS][WAVES_OF<L>];
    const int group = group_of<L>(), l = threadIdx.x % L, lot = threadIdx.x / 64 % WAVES_OF<L>;
    const auto piece = [&](int k) { return Piece<T, ROWS>((k * L + l) * V, cols); };
    float g[CH][V], b[CH][V];
    uintx4 raw[CH], next[CH];
    const auto load = [&](int64_t row, uintx4 (&v)[CH]) {
        const T *x_row = x + min(row, rows - 1) * x_ld;
#pragma unroll
        for (int k = 0; k < CH; ++k) v[k] = piece(k).load(x_row);
    };
    load((int64_t)blockIdx.x * GROUPS + group, raw);
#pragma unroll
    for (int k = 0; k < CH; ++k) {
        piece(k).params(gamma, params_bf16, 1.f, g[k]);
        piece(k).params(beta, params_bf16, 0.f, b[k]);
    }
    const int64_t step = (int64_t)gridDim.x * GROUPS;
    for (int64_t first = (int64_t)blockIdx.x * GROUPS; first < rows; first += step) {
        const int64_t row = first + group;
        if (first + step < rows) load(row + step, next);
        float sum = 0.f;
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            float f[V];
            unpack(raw[k], f);
#pragma unroll
            for (int e = 0; e < V; ++e) sum += piece(k).once(f[e], e);
        }
        float mean = group_sum<L>(sum, sums[0][group], lot) / cols;
        sum = 0.f;
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            float f[V];
            unpack(raw[k], f);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float d = piece(k).has ? piece(k).once(f[e] - mean, e) : 0.f;
                sum = fmaf(d, d, sum);
            }
        }
        float var = group_sum<L>(sum, sums[1][group], lot) / cols;
        static_assert(L < 128 || GROUPS == 1, "the rows of a workgroup would part at a barrier");
        if (far_from_zero(mean, var)) {
            sum = 0.f;
#pragma unroll
            for (int k = 0; k < CH; ++k) {
                float f[V];
                unpack(raw[k], f);
#pragma unroll
                for (int e = 0; e < V; ++e) sum += piece(k).has ? piece(k).once(f[e] - mean, e) : 0.f;
            }
            shift(mean, var, group_sum<L>(sum, sums[2][group], lot) / cols);
        }
        const float rstd = 1.f / sqrtf(var + eps);
        if (row < rows) {
            if (stats && l == 0) stats[row] = make_float2(mean, rstd);
#pragma unroll
            for (int k = 0; k < CH; ++k) {
                float f[V];
                unpack(raw[k], f);
#pragma unroll
                for (int e = 0; e < V; ++e) f[e] = fmaf((f[e] - mean) * rstd, g[k][e], b[k][e]);
                piece(k).store(y + row * y_ld, f, false);
            }
        }
#pragma unroll
        for (int k = 0; k < CH; ++k) raw[k] = next[k];
    }
}

// dx, and this workgroup's rows' part of dgamma and dbeta: a lane's columns are the same in every row, so their sums stay in its registers and dy and x are
// read once for all three results.  Eight waves with up to 32 values of a row to a lane (160 registers of sums, gamma and two rows under way; with 16 waves
// and 128 registers it spilled); as many workgroups as are on the card at once, since each leaves a part of 8 bytes a column.  16384 x 4096, bf16: 84 us
// (4.9 TB/s) and 4.5 for the join of 256 parts; in three kernels that read dy and x twice, value by value, 430.  1023 x 12289, fp32: 45 us, 25 MB of its 256 parts.
template <int L> constexpr int BWD_THREADS = L <= 512 ? 512 : L;
template <class T, int L, int CH, int ROWS>
__global__ __launch_bounds__(BWD_THREADS<L>) void layernorm_rows_bwd_kernel(const T *dy, const T *__restrict__ x, const void *__restrict__ gamma, bool params_bf16,
                                                                            const float2 *__restrict__ stats, T *dx, float *__restrict__ part, int64_t rows,
                                                                            int cols, int64_t dy_ld, int64_t x_ld, int64_t dx_ld, int add, void *dgamma, void *dbeta) {
    constexpr int V = VEC<T>, THREADS = BWD_THREADS<L>, GROUPS = THREADS / L, N = CH * V, W = WAVES_OF<L>;
    constexpr bool AHEAD = L <= 512;      // the next row's loads begin before this one is worked; 16 waves have registers for one row
    __shared__ float sums[2][2][GROUPS][W];
    __shared__ float joined[GROUPS > 1 ? THREADS * N : 1];
    const int group = group_of<L>(), l = threadIdx.x % L, lot = threadIdx.x / 64 % W;
    const float by = 1.f / cols;
    const auto piece = [&](int k) { return Piece<T, ROWS>((k * L + l) * V, cols); };
    float g[N], a[N] = {}, b[N] = {};
#pragma unroll
    for (int k = 0; k < CH; ++k) {
        float f[V];
        piece(k).params(gamma, params_bf16, 1.f, f);
#pragma unroll
        for (int e = 0; e < V; ++e) g[k * V + e] = f[e];
    }
    uintx4 rd[CH], rx[CH], nd[CH], nx[CH];
    float2 st, nst;
    const auto load = [&](int64_t row, uintx4 (&d)[CH], uintx4 (&v)[CH], float2 &s) {
        if (row >= rows) {      // adds nothing: zeros of a row whose mean is 0
#pragma unroll
            for (int k = 0; k < CH; ++k) d[k] = v[k] = uintx4{};
            s = make_float2(0.f, 0.f);
            return;
        }
        s = stats[row];
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            d[k] = piece(k).load(dy + row * dy_ld);
            v[k] = piece(k).load(x + row * x_ld);
        }
    };
    const int64_t step = (int64_t)gridDim.x * GROUPS;
    load((int64_t)blockIdx.x * GROUPS + group, rd, rx, st);
    int turn = 0;
    for (int64_t first = (int64_t)blockIdx.x * GROUPS; first < rows; first += step, turn ^= 1) {
        const int64_t row = first + group;
        if (AHEAD) load(row + step, nd, nx, nst);
        float s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            float d[V], v[V];
            unpack(rd[k], d);
            unpack(rx[k], v);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const int i = k * V + e;
                const float xh = (v[e] - st.x) * st.y, o = piece(k).once(d[e], e), t = o * g[i];
                s1 += t;
                s2 = fmaf(t, xh, s2);
                a[i] = fmaf(o, xh, a[i]);
                b[i] += o;
            }
        }
        if (W == 1) {
            s1 = group_sum<L>(s1, nullptr, 0);
            s2 = group_sum<L>(s2, nullptr, 0);
        } else {      // two places in turn: who still reads the other one has not passed this barrier
            s1 = wave_sum(s1);
            s2 = wave_sum(s2);
            if (threadIdx.x % 64 == 0) { sums[turn][0][group][lot] = s1; sums[turn][1][group][lot] = s2; }
            __syncthreads();
            s1 = sums[turn][0][group][0];
            s2 = sums[turn][1][group][0];
#pragma unroll
            for (int i = 1; i < W; ++i) { s1 += sums[turn][0][group][i]; s2 += sums[turn][1][group][i]; }
        }
        s1 *= by;
        s2 *= by;
        if (dx && row < rows) {
#pragma unroll
            for (int k = 0; k < CH; ++k) {
                float d[V], v[V];
                unpack(rd[k], d);
                unpack(rx[k], v);
#pragma unroll
                for (int e = 0; e < V; ++e) d[e] = st.y * (d[e] * g[k * V + e] - s1 - (v[e] - st.x) * st.y * s2);
                piece(k).store(dx + row * dx_ld, d, add & 1);
            }
        }
        if (AHEAD) {
#pragma unroll
            for (int k = 0; k < CH; ++k) { rd[k] = nd[k]; rx[k] = nx[k]; }
            st = nst;
        } else
            load(row + step, rd, rx, st);
    }
    if (!dgamma && !dbeta) return;
    // the groups' sums, in their order; the only workgroup has the results, no part of them
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        float(&s)[N] = which ? b : a;
        if (L < 64) {      // a wave's rows
#pragma unroll
            for (int k = 32; k >= L; k /= 2)
#pragma unroll
                for (int i = 0; i < N; ++i) s[i] += __shfl_xor(s[i], k);
        }
        if (GROUPS > 1) {
            constexpr int APART = L < 64 ? 64 : L;      // threads from one sum to the next
            if (which) __syncthreads();
#pragma unroll
            for (int i = 0; i < N; ++i) joined[i * THREADS + threadIdx.x] = s[i];
            __syncthreads();
            if (group == 0) {
#pragma unroll
                for (int o = 1; o < THREADS / APART; ++o)
#pragma unroll
                    for (int i = 0; i < N; ++i) s[i] += joined[i * THREADS + o * APART + threadIdx.x];
            }
        }
        void *out = which ? dbeta : dgamma;
        if (group || !out) continue;
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            const Piece<T, ROWS> at = piece(k);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                if (!at.has || !at.counts(e)) continue;
                const int c = at.c + e;
                if (gridDim.x > 1) part[((int64_t)blockIdx.x * 2 + which) * cols + c] = s[k * V + e];
                else if (params_bf16) put((unsigned short *)out + c, s[k * V + e], add >> (1 + which) & 1);
                else put((float *)out + c, s[k * V + e], add >> (1 + which) & 1);
            }
        }
    }
}

// ---- longer rows (more than 16384 columns), which are read again, mostly from L2, for each of their sums; pieces as above: 1000 x 30000 in bf16 forward 37 us,
// backward 77 (3.2 and 2.3 TB/s), where the caches hold the rows from an earlier launch 33 and 68
constexpr int LONG_THREADS = 1024;
__device__ __forceinline__ float long_sum(float v, float *seg) {      // the same in every thread
    v = wave_sum(v);
    __syncthreads();
    if (threadIdx.x % 64 == 0) seg[threadIdx.x / 64] = v;
    __syncthreads();
    v = seg[0];
#pragma unroll
    for (int i = 1; i < LONG_THREADS / 64; ++i) v += seg[i];
    return v;
}
// calls of(value) with a thread's values of a row
template <class T, class F>
__device__ __forceinline__ void long_values(const T *row, int cols, F &&of) {
    constexpr int V = VEC<T>;
    for (int c = threadIdx.x * V; c < cols; c += LONG_THREADS * V) {
        const Piece<T, MOVED> at(c, cols);
        float f[V];
        unpack(at.load(row), f);
#pragma unroll
        for (int e = 0; e < V; ++e)
            if (at.counts(e)) of(f[e]);
    }
}
template <class T>
__global__ __launch_bounds__(LONG_THREADS) void layernorm_fwd_kernel(const T *x, const void *__restrict__ gamma, const void *__restrict__ beta, bool params_bf16,
                                                                     T *y, float2 *__restrict__ stats, int64_t rows, int cols, int64_t x_ld, int64_t y_ld,
                                                                     float eps) {
    constexpr int V = VEC<T>;
    __shared__ float seg[LONG_THREADS / 64];
    for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
        const T *from = x + row * x_ld;
        T *to = y + row * y_ld;
        float sum = 0.f;
        long_values(from, cols, [&](float v) { sum += v; });
        float mean = long_sum(sum, seg) / cols;
        sum = 0.f;
        long_values(from, cols, [&](float v) { sum = fmaf(v - mean, v - mean, sum); });
        float var = long_sum(sum, seg) / cols;
        if (far_from_zero(mean, var)) {
            sum = 0.f;
            long_values(from, cols, [&](float v) { sum += v - mean; });
            shift(mean, var, long_sum(sum, seg) / cols);
        }
        const float rstd = 1.f / sqrtf(var + eps);
        // in place, others read and store their values meanwhile: everybody stores those that nobody else reads for a result
        for (int c = threadIdx.x * V; c < cols; c += LONG_THREADS * V) {
            const Piece<T, MOVED> at(c, cols);
            float f[V], g[V], b[V];
            unpack(at.load(from), f);
            at.params(gamma, params_bf16, 1.f, g);
            at.params(beta, params_bf16, 0.f, b);
#pragma unroll
            for (int e = 0; e < V; ++e) f[e] = fmaf((f[e] - mean) * rstd, g[e], b[e]);
            at.store(to, f, false, true);
        }
        if (stats && threadIdx.x == 0) stats[row] = make_float2(mean, rstd);
    }
}

template <class T>
__global__ __launch_bounds__(LONG_THREADS) void layernorm_dx_kernel(const T *dy, const T *__restrict__ x, const void *__restrict__ gamma, bool params_bf16,
                                                                    const float2 *__restrict__ stats, T *dx, int64_t rows, int cols, int64_t dy_ld, int64_t x_ld,
                                                                    int64_t dx_ld, bool add) {
    constexpr int V = VEC<T>;
    __shared__ float seg[LONG_THREADS / 64];
    for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
        const T *go = dy + row * dy_ld, *from = x + row * x_ld;
        T *to = dx + row * dx_ld;
        const float mean = stats[row].x, rstd = stats[row].y;
        float a = 0.f, b = 0.f;
        for (int c = threadIdx.x * V; c < cols; c += LONG_THREADS * V) {
            const Piece<T, MOVED> at(c, cols);
            float d[V], v[V], g[V];
            unpack(at.load(go), d);
            unpack(at.load(from), v);
            at.params(gamma, params_bf16, 1.f, g);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float t = at.once(d[e], e) * g[e];
                a += t;
                b = fmaf(t, (v[e] - mean) * rstd, b);
            }
        }
        a = long_sum(a, seg) / cols;
        b = long_sum(b, seg) / cols;
        for (int c = threadIdx.x * V; c < cols; c += LONG_THREADS * V) {
            const Piece<T, MOVED> at(c, cols);
            float d[V], v[V], g[V];
            unpack(at.load(go), d);
            unpack(at.load(from), v);
            at.params(gamma, params_bf16, 1.f, g);
#pragma unroll
            for (int e = 0; e < V; ++e) d[e] = rstd * (d[e] * g[e] - a - (v[e] - mean) * rstd * b);
            at.store(to, d, add, true);      // as in the forward pass
        }
    }
}

// 64 pieces of a range of rows: part[range][0: dgamma, 1: dbeta][cols]
template <class T>
__global__ __launch_bounds__(256) void layernorm_columns_kernel(const T *__restrict__ dy, const T *__restrict__ x, const float2 *__restrict__ stats,
                                                                float *__restrict__ part, int64_t rows, int64_t per, int cols, int64_t dy_ld, int64_t x_ld) {
    constexpr int V = VEC<T>;
    __shared__ float sums[2][4][V][64];
    const int l = threadIdx.x & 63, wave = threadIdx.x / 64;
    const Piece<T, MOVED> at((blockIdx.x * 64 + l) * V, cols);
    const int64_t from = blockIdx.y * per, to = min(rows, from + per);
    float a[V] = {}, b[V] = {};
#pragma unroll 2
    for (int64_t r = from + wave; r < to; r += 4) {
        const float2 st = stats[r];
        float d[V], v[V];
        unpack(at.load(dy + r * dy_ld), d);
        unpack(at.load(x + r * x_ld), v);
#pragma unroll
        for (int e = 0; e < V; ++e) {
            a[e] = fmaf(d[e], (v[e] - st.x) * st.y, a[e]);
            b[e] += d[e];
        }
    }
#pragma unroll
    for (int e = 0; e < V; ++e) {
        sums[0][wave][e][l] = a[e];
        sums[1][wave][e][l] = b[e];
    }
    __syncthreads();
    if (wave >= 2 || !at.has) return;
#pragma unroll
    for (int e = 0; e < V; ++e)
        if (at.counts(e))
            part[((int64_t)blockIdx.y * 2 + wave) * cols + at.c + e] =
                (sums[wave][0][e][l] + sums[wave][1][e][l]) + (sums[wave][2][e][l] + sums[wave][3][e][l]);
}

// the parts' sums: grid y 0 dgamma, 1 dbeta (null: not wanted); sixteen waves take a share of the ranges each, in a fixed order
template <class P>
__global__ __launch_bounds__(1024) void layernorm_join_kernel(const float *__restrict__ part, int ranges, int cols, P *dgamma, P *dbeta, int add) {
    __shared__ float sums[16][64];
    const int l = threadIdx.x & 63, wave = threadIdx.x / 64, c = blockIdx.x * 64 + l, which = blockIdx.y;
    P *out = which ? dbeta : dgamma;
    if (!out) return;
    float s = 0.f;
    if (c < cols) {
#pragma unroll 8
        for (int r = wave; r < ranges; r += 16) s += part[((int64_t)r * 2 + which) * cols + c];
    }
    sums[wave][l] = s;
    __syncthreads();
    if (wave || c >= cols) return;
#pragma unroll
    for (int w = 1; w < 16; ++w) s += sums[w][l];
    put(out + c, s, add >> which & 1);
}

int64_t cut(int64_t n, int64_t by) { return (n + by - 1) / by; }

constexpr int LAYERNORM_COLS = 1 << 20;

// Calls f(lanes to a row, pieces of 16 bytes to a lane of it) with the smallest form that a row of a piece or more fits.  BACK: the backward pass.  false: the
// row does not fit.
template <class T, bool BACK, class F>
bool layernorm_form(int cols, F &&f) {
    constexpr int M = BACK ? 4 : 16 / VEC<T>;       // pieces to a lane of a wave or more
    const auto fits = [&](auto l, auto ch) {
        if (cols > CAPACITY<T, decltype(l)::value, decltype(ch)::value>) return false;
        f(l, ch);
        return true;
    };
    using std::integral_constant;
    const integral_constant<int, 1> one;
    const integral_constant<int, 2> two;
    const integral_constant<int, 16> quarter;
    const integral_constant<int, 64> wave;
    const integral_constant<int, M> m;
    if (fits(integral_constant<int, 4>(), one) || fits(quarter, one) || fits(quarter, two) || fits(wave, one) || fits(wave, two) || fits(wave, m) ||
        fits(integral_constant<int, 128>(), m) || fits(integral_constant<int, 256>(), m) || fits(integral_constant<int, 512>(), m))
        return true;
    if constexpr (!BACK || std::is_same<T, float>::value) return fits(integral_constant<int, 1024>(), m);
    else return false;
}
// Calls f(lanes, pieces, WHOLE, MOVED or SHORT) with the form of a row; false: it does not fit the registers
template <class T, bool BACK, class F>
bool layernorm_rows_form(int cols, F &&f) {
    using std::integral_constant;
    if (cols < VEC<T>) {
        f(integral_constant<int, 4>(), integral_constant<int, 1>(), integral_constant<int, SHORT>());
        return true;
    }
    return layernorm_form<T, BACK>(cols, [&](auto l, auto ch) {
        if (cols % VEC<T>) f(l, ch, integral_constant<int, MOVED>());
        else f(l, ch, integral_constant<int, WHOLE>());
    });
}
// Parts of dgamma and dbeta: the workgroups that share the rows of a backward pass (as many as are on the card at once), or, of rows that do not fit
// the registers, ranges of rows
int64_t layernorm_ranges(int dtype, int64_t rows, int cols) {
    int64_t rows_at_once = 0, groups = 0;
    const auto form = [&](auto l, auto ch, auto) {
        constexpr int L = decltype(l)::value, CH = decltype(ch)::value;
        rows_at_once = BWD_THREADS<L> / L;
        groups = L <= 512 && CH * (dtype == MONET_F32 ? 4 : 8) <= 16 ? 512 : 256;
    };
    dtype == MONET_F32 ? layernorm_rows_form<float, true>(cols, form) : layernorm_rows_form<unsigned short, true>(cols, form);
    // few values: one workgroup, which needs no second launch (37 rows of 203 in fp32, both passes: 24 us, with a join 27.5)
    if (rows && rows_at_once && rows * cols <= 1 << 14 && rows <= 8 * rows_at_once) return 1;
    // three turns or more to a workgroup, since a part costs as much as four rows of bf16 (1000 x 8192: backward pass 24 us with two turns, 18.5 with three), unless fewer than
    // 128 workgroups are left
    if (rows_at_once) return std::min({groups, cut(rows, rows_at_once), std::max<int64_t>(128, cut(rows, 3 * rows_at_once))});
    return std::min<int64_t>(cut(rows, 32), std::max<int64_t>(1, 2048 / cut(cols, 64 * (dtype == MONET_F32 ? 4 : 8))));
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

// calls f with a value of the type
template <class F>
void by_type(int dtype, F &&f) {
    if (dtype == MONET_F32) f(0.f);
    else f((unsigned short)0);
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
    by_type(dtype, [&](auto t) {
        using T = decltype(t);
        const bool rows_fit = layernorm_rows_form<T, false>(cols, [&](auto l, auto ch, auto form) {
            constexpr int L = decltype(l)::value, CH = decltype(ch)::value, GROUPS = FWD_THREADS<L> / L;
            hipLaunchKernelGGL((layernorm_rows_kernel<T, L, CH, decltype(form)::value>), dim3((unsigned)std::min<int64_t>(cut(rows, GROUPS), 256 * 1024 / FWD_THREADS<L>)),
                               dim3(FWD_THREADS<L>), 0, st, (const T *)x, gamma, beta, param_dtype == MONET_BF16, (T *)y, (float2 *)stats, rows, cols, x_ld, y_ld,
                               eps);
        });
        if (rows_fit) return;
        hipLaunchKernelGGL(layernorm_fwd_kernel<T>, dim3((unsigned)std::min<int64_t>(rows, 1 << 16)), dim3(LONG_THREADS), 0, st, (const T *)x, gamma, beta,
                           param_dtype == MONET_BF16, (T *)y, (float2 *)stats, rows, cols, x_ld, y_ld, eps);
    });
    hip_check(hipGetLastError(), "layernorm launch");
}

size_t layernorm_bwd_workspace_bytes(int dtype, int64_t rows, int cols) {
    layernorm_shape(dtype, rows, cols);
    return (size_t)(layernorm_ranges(dtype, rows, cols) * 2 * cols * 4);
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
    const int64_t ranges = layernorm_ranges(dtype, rows, cols);
    const auto join = [&] {
        by_type(param_dtype, [&](auto p) {
            using P = decltype(p);
            hipLaunchKernelGGL(layernorm_join_kernel<P>, dim3((unsigned)cut(cols, 64), 2), dim3(1024), 0, st, (const float *)ws, (int)ranges, cols, (P *)dgamma,
                               (P *)dbeta, accumulate >> 1);
        });
        hip_check(hipGetLastError(), "layernorm join launch");
    };
    by_type(dtype, [&](auto t) {
        using T = decltype(t);
        if (!rows) {
            if (columns) join();
            return;
        }
        if (!dx && !columns) return;
        const bool rows_fit = layernorm_rows_form<T, true>(cols, [&](auto l, auto ch, auto form) {
            constexpr int L = decltype(l)::value, CH = decltype(ch)::value;
            hipLaunchKernelGGL((layernorm_rows_bwd_kernel<T, L, CH, decltype(form)::value>), dim3((unsigned)ranges), dim3(BWD_THREADS<L>), 0, st, (const T *)dy,
                               (const T *)x, gamma, param_dtype == MONET_BF16, (const float2 *)stats, (T *)dx, (float *)ws, rows, cols, dy_ld, x_ld, dx_ld,
                               accumulate, dgamma, dbeta);
            hip_check(hipGetLastError(), "layernorm gradients launch");
        });
        if (rows_fit) {
            if (columns && ranges > 1) join();
            return;
        }
        if (columns) {
            hipLaunchKernelGGL(layernorm_columns_kernel<T>, dim3((unsigned)cut(cols, 64 * VEC<T>), (unsigned)ranges), dim3(256), 0, st, (const T *)dy, (const T *)x,
                               (const float2 *)stats, (float *)ws, rows, cut(rows, ranges), cols, dy_ld, x_ld);
            hip_check(hipGetLastError(), "layernorm columns launch");
            join();
        }
        if (dx) {
            hipLaunchKernelGGL(layernorm_dx_kernel<T>, dim3((unsigned)std::min<int64_t>(rows, 1 << 16)), dim3(LONG_THREADS), 0, st, (const T *)dy, (const T *)x, gamma,
                               param_dtype == MONET_BF16, (const float2 *)stats, (T *)dx, rows, cols, dy_ld, x_ld, dx_ld, accumulate & 1);
            hip_check(hipGetLastError(), "layernorm gradient launch");
        }
    });
}

}  // namespace monet
