// Causal attention over packed sequences with grouped heads.
//
//   s[i][j] = scale q[i] . k[j] for j <= i of the same sequence,  lse[i] = log sum_j exp s[i][j],  p = exp(s - lse),  o[i] = sum_j p[i][j] v[j]
//   delta[i] = do[i] . o[i] = sum_j p[i][j] (do[i] . v[j]),  ds = p (do v^T - delta),  dq = scale ds k,  dk = scale ds^T q,  dv = p^T do  (dk, dv summed over a group's heads)
//
// Nothing of size length x length is kept: the forward pass leaves lse, the backward pass computes p again.
//
// The products are worked as their transposes, so that a lane of the matrix instruction holds 16 scores of one row: the row's maximum and
// sum need one exchange between the wave's halves, and the scores leave the first product where the second one reads its operand (the
// order of a reduction's indices is free as long as both operands agree).  The other operand of the second product runs across the
// reduction and is read from LDS by ds_read_b64_tr_b16.
//
// Everything runs on v_mfma_f32_32x32x16_bf16.  bf16: p and ds are rounded to bf16 between the products, at most 2^-8 of a value each.  Rounding
// the results alone leaves them 1.7e-3 off (Frobenius norm; 8 ragged sequences of 8192 rows), with this o is 2.0e-3 and dq and dk are 2.4e-3 off;
// ds in two pieces would take nine products for seven.  fp32: every operand in three bf16 pieces and a product in
// six terms (bf16_pieces.hpp), 2^-24 of it at worst, in 192 cycles where the fp32 instruction takes 512; tiles are split on their way to
// LDS, results in registers.  An infinity comes out as NaN there.  Scores, maxima, sums and gradients are fp32 in both.
//
// Backward is two kernels without atomics, so results do not depend on the order of anything: the first walks along the keys of 128
// rows (dq, and delta on the way), the second along the rows and the group's heads of 128 keys (dk, dv).  That computes the scores
// and do v^T twice, seven products for five; bf16 computes them a third time for a sequence's first 128 rows (FEW_KEYS).
//
// What bounds it, two sequences of 8192 rows, 32 heads of 128 on 8, bf16: forward 1.05 ms (1.05 PFLOP/s), dq 1.5 (1.1 of its three products), dk and
// dv 2.2 (1.0 of four).  MFMA pipes busy 51, 58 and 51 % of the cycles at 1.8 to 1.9 GHz, which the power limit leaves of 2.4; vector instructions
// 43, 36 and 34 %, LDS 38, 39 and 44 % without a conflict.  Eight ragged sequences of as many rows in all keep the pipes busy 38, 41 and 32 % at
// 2.1 GHz: no power limit there, but the longest ways, which end alone.  fp32, one of 4096 rows: 0.84, 1.33 and 2.30 ms (164, 155 and 120 TFLOP/s),
// pipes busy 44, 39 and 29 %; one of 1347 rows and one of 700, 12 heads of 64: 15 to 20 %, with 6 to 10 vector instructions, most of them for the
// pieces, to a matrix instruction.
#include <initializer_list>

#include "../../include/monet_kernels.h"
#include "kernels.hpp"
#include "tile_bf16.hpp"

namespace monet {

namespace {

constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.69314718055994530942f;
typedef float floatx4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ int uniform_wave() { return __builtin_amdgcn_readfirstlane(threadIdx.x / 64); }      // in a scalar register, as is what follows from it

// bf16: delta = sum of p dp, from fp32, in the rows of a sequence before this one; from o, rounded to bf16, in the others.  What rounding o moves delta by
// goes into ds of all keys alike, which few keys do not average out: dq and dk of sequences of a few rows are 2.4e-3 off so, from o throughout 4.2e-3.
// It costs two products more in those rows.  Both backward kernels, 32 / 8 heads of 128: 128 sequences of 64 rows 171 us, without it 161; 64 of 128
// 254 and 227; 142 of 1 to 60 rows 151 and 134; 16 of 512 259 and 255; the eight ragged ones the same.
constexpr int FEW_KEYS = 128;

// The rows of a 32 x 32 result that lie before `limit` are not the lane's key's: their probabilities are 0.  The limit passes through a register of
// its own inside the branch that this stands in, or the compiler compares for every tile what only those on the diagonal need.
__device__ __forceinline__ void clear_before(floatx16 &s, int limit) {
    limit -= 4 * ((threadIdx.x & 63) >> 5);
    asm volatile("" : "+v"(limit));
#pragma unroll
    for (int r = 0; r < 16; ++r)
        if ((r & 3) + 8 * (r >> 2) < limit) s[r] = 0.f;
}

// What a lane holds of an operand at 16 reduction indices, and the product of two of these.
template <class T> struct Piece;
template <> struct Piece<unsigned short> {
    typedef bf16x8 V;
    static constexpr int PLANES = 1;
    static __device__ __forceinline__ V plane(const V &v, int) { return v; }
    static __device__ __forceinline__ floatx16 mma(const V &a, const V &b, floatx16 c) { return mfma_bf16(a, b, c); }
    // results 8 s .. 8 s + 7 of a lane as an operand
    static __device__ __forceinline__ V from_result(const floatx16 &p, int s) {
        const uintx4 w{pack_bf16(p[8 * s], p[8 * s + 1]), pack_bf16(p[8 * s + 2], p[8 * s + 3]), pack_bf16(p[8 * s + 4], p[8 * s + 5]),
                       pack_bf16(p[8 * s + 6], p[8 * s + 7])};
        return __builtin_bit_cast(V, w);
    }
    static __device__ __forceinline__ V load(const unsigned short *p) { return *(const V *)p; }
    static __device__ __forceinline__ float dot(const unsigned short *a, const unsigned short *b) {
        float s = 0.f;
        const uintx4 x = *(const uintx4 *)a, y = *(const uintx4 *)b;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            s += __uint_as_float(x[i] << 16) * __uint_as_float(y[i] << 16);
            s += __uint_as_float(x[i] & 0xffff0000u) * __uint_as_float(y[i] & 0xffff0000u);
        }
        return s;
    }
};
template <> struct Piece<float> {
    typedef PieceRow V;
    static constexpr int PLANES = 3;
    static __device__ __forceinline__ floatx16 mma(const V &a, const V &b, floatx16 c) {
        c = mfma_bf16(a.l, b.h, c);
        c = mfma_bf16(a.h, b.l, c);
        c = mfma_bf16(a.m, b.m, c);
        c = mfma_bf16(a.m, b.h, c);
        c = mfma_bf16(a.h, b.m, c);
        return mfma_bf16(a.h, b.h, c);
    }
    static __device__ __forceinline__ V from_result(const floatx16 &p, int s) {
        const float v[8] = {p[8 * s], p[8 * s + 1], p[8 * s + 2], p[8 * s + 3], p[8 * s + 4], p[8 * s + 5], p[8 * s + 6], p[8 * s + 7]};
        unsigned lost = 0;
        return split_row(v, lost);
    }
    static __device__ __forceinline__ V load(const float *p) {
        const float4 a = *(const float4 *)p, b = *(const float4 *)(p + 4);
        const float v[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
        unsigned lost = 0;
        return split_row(v, lost);
    }
    static __device__ __forceinline__ float dot(const float *a, const float *b) {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) s += a[i] * b[i];
        return s;
    }
};

// A tile of R rows of D values in LDS, as bf16 (fp32: a plane for each piece): strips of 64 columns, each R rows of 128 bytes in eight
// pieces turned by the row (tile_bf16.hpp).
template <class T, int D, int R> struct AttTile;
template <int D, int R>
struct AttTile<unsigned short, D, R> {         // straight from memory to LDS
    // a copy takes 32 rows of a strip; the turns repeat after 16, so a strip's offsets serve all of its copies
    static constexpr int BYTES = R * D * 2, STRIPS = D / 64;
    unsigned off[STRIPS];
    int64_t ld;
    int used;               // bytes of a row that exist
    __device__ __forceinline__ void init(int64_t ld_, int head_dim) {
        ld = ld_;
        used = head_dim * 2;
#pragma unroll
        for (int i = 0; i < STRIPS; ++i) {
            const unsigned row = threadIdx.x / 8, col = i * 128 + (((threadIdx.x % 8) ^ wide_turn(row)) << 4);
            off[i] = (int)col < used ? row * (unsigned)(ld * 2) + col : BUFFER_ABSENT;
        }
    }
    // rows of which `left` exist; the others arrive as zeros
    __device__ __forceinline__ void copy(lds_char *lds, const unsigned short *rows, int left) const {
        const int wave = uniform_wave();
#pragma unroll
        for (int row = 0; row < R; row += 32) {
            const __amdgpu_buffer_rsrc_t r = buffer_of(rows + row * ld, left > row ? (unsigned)((min(left - row, 32) - 1) * ld * 2) + used : 0u);
#pragma unroll
            for (int i = 0; i < STRIPS; ++i) copy_to_lds(r, lds + (i * R + row) * 128 + wave * 1024, off[i], 0);
        }
    }
};
template <int D, int R>
struct AttTile<float, D, R> {                  // through registers, where it is split
    static constexpr int PLANE = R * D * 2, BYTES = 3 * PLANE, COPIES = R * D / (256 * 8);
    float4 held[COPIES][2];
    int64_t ld;
    int head_dim;
    __device__ __forceinline__ void init(int64_t ld_, int head_dim_) {
        ld = ld_;
        head_dim = head_dim_;
    }
    __device__ __forceinline__ void load(const float *rows, int left) {
#pragma unroll
        for (int i = 0; i < COPIES; ++i) {
            const int piece = i * 256 + threadIdx.x, row = piece / (D / 8), col = piece % (D / 8) * 8;
            held[i][0] = held[i][1] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (row < left && col < head_dim) {
                const float *p = rows + row * ld + col;
                held[i][0] = *(const float4 *)p;
                held[i][1] = *(const float4 *)(p + 4);
            }
        }
    }
    __device__ __forceinline__ void store(lds_char *lds) const {
#pragma unroll
        for (int i = 0; i < COPIES; ++i) {
            const int piece = i * 256 + threadIdx.x, row = piece / (D / 8), c = piece % (D / 8);
            const float4 a = held[i][0], b = held[i][1];
            const float v[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
            unsigned lost = 0;
            const PieceRow r = split_row(v, lost);
            lds_char *p = lds + (c >> 3) * R * 128 + row * 128 + (((c & 7) ^ (int)wide_turn(row)) << 4);
            typedef __attribute__((address_space(3))) bf16x8 lds_bf16x8;
            *(lds_bf16x8 *)p = r.h;
            *(lds_bf16x8 *)(p + PLANE) = r.m;
            *(lds_bf16x8 *)(p + 2 * PLANE) = r.l;
        }
    }
};
// where a lane reads such tiles
template <class T, int D, int R>
struct AttReader {
    static constexpr int PLANE = R * D * 2;
    typedef typename Piece<T>::V V;
    unsigned wide_at[4], deep_at[4];
    __device__ __forceinline__ void init() {
        const unsigned l = threadIdx.x & 63, h = l >> 5;
#pragma unroll
        for (int s = 0; s < 4; ++s) wide_at[s] = (l & 31) * 128 + (((2 * s + h) ^ wide_turn(l & 31)) << 4);
#pragma unroll
        for (int p = 0; p < 4; ++p) {      // bit 0: rows + 8, bit 1: columns + 32
            const unsigned row = 4 * h + ((l & 15) >> 2) + 8 * (p & 1), c = 4 * (p >> 1) + 2 * ((l >> 4) & 1) + ((l & 3) >> 1);
            deep_at[p] = row * 128 + ((c ^ wide_turn(row)) << 4) + (l & 1) * 8;
        }
    }
    // rows 32 b + (l & 31), 16 columns from 16 s on
    __device__ __forceinline__ V wide(const lds_char *t, int b, int s) const {
        const lds_char *p = t + wide_at[s & 3] + b * 32 * 128 + (s >> 2) * R * 128;
        if constexpr (sizeof(T) == 2) return read_wide(p);
        else return PieceRow{read_wide(p), read_wide(p + PLANE), read_wide(p + 2 * PLANE)};
    }
    // columns 32 c + (l & 31), the rows of 32 b .. that results of step s hold
    __device__ __forceinline__ V deep(const lds_char *t, int b, int s, int c) const {
        const lds_char *p = t + (c >> 1) * R * 128 + (32 * b + 16 * s) * 128;
        const unsigned x = deep_at[2 * (c & 1)], y = deep_at[2 * (c & 1) + 1];
        if constexpr (sizeof(T) == 2) return join(read_turned(p + x), read_turned(p + y));
        else
            return PieceRow{join(read_turned(p + x), read_turned(p + y)), join(read_turned(p + PLANE + x), read_turned(p + PLANE + y)),
                            join(read_turned(p + 2 * PLANE + x), read_turned(p + 2 * PLANE + y))};
    }
};

// The pieces of row l & 31 of 32 rows (of which `left` exist) straight from memory
template <class T, int D>
struct RowPieces {
    typename Piece<T>::V p[D / 16];
    __device__ __forceinline__ void load(const T *rows, int64_t ld, int left, int head_dim) {
        const int l = threadIdx.x & 63;
        const T *row = rows + (l & 31) * ld;
#pragma unroll
        for (int s = 0; s < D / 16; ++s) {
            const int col = (2 * s + (l >> 5)) * 8;
            p[s] = typename Piece<T>::V{};
            if ((l & 31) < left && col < head_dim) p[s] = Piece<T>::load(row + col);
        }
    }
};

struct AttShape {
    const int32_t *cu;
    int seqs, tokens, heads, kv_heads, head_dim, slots;
    int64_t q_ld, k_ld, v_ld, o_ld;
    float scale;
};

// How a workgroup's four waves share a tile.  PARTS = 1: 32 rows each, every wave takes the whole tile.  PARTS = 2, 4: 64 or 32 rows in all,
// the waves of the same rows take 32 of the tile's columns each and add up what they have at the end: two and four times as many
// workgroups and as short a way for each, for as much more traffic from L2.
template <class T, int D, int PARTS>
struct AttForm {
    static constexpr int ROWS = 128 / PARTS, BLOCKS = sizeof(T) == 2 && PARTS == 1 ? 2 : 1, TILE = 32 * BLOCKS * PARTS;
    static constexpr int PIECES = D / 16, STEPS = 2;
    typedef AttTile<T, D, TILE> Tile;
    // bf16: two tiles of each of two tensors, copied to while the others are read; fp32: one of each, which registers hold the next of
    static constexpr int BUFFERS = sizeof(T) == 2 ? 2 : 1;
    static constexpr bool TWO_GROUPS = 2 * BUFFERS * Tile::BYTES <= 72 << 10;      // two workgroups in a CU's LDS
    static constexpr int AREA = D / 32 * 16 * 256;                       // a wave's results
    static constexpr int RANGE_TILES = sizeof(T) == 2 ? 16 : 6;          // dk, dv: the most tiles of rows to a range
    static constexpr int RANGE_ROWS = RANGE_TILES * TILE;
};

// Sequence s owns the slots from cu[s] / ROWS + s on: at least one for every ROWS rows begun, whatever the lengths, so the grid
// needs no more than tokens / ROWS + seqs slots and a workgroup finds its sequence by a search of 64 at a time.  Offsets are held
// to 0 .. tokens.
template <int ROWS>
__device__ __forceinline__ bool find_rows(const AttShape &a, int slot, int &start, int &len, int &row0) {
    const int lane = threadIdx.x & 63;
    auto at = [&](int s) { return min(max(a.cu[s], 0), a.tokens); };
    int lo = 0, n = a.seqs;
    while (true) {
        const int step = (n + 63) / 64, i = lane * step;
        const unsigned long long ok = __ballot(i < n && at(lo + min(i, n - 1)) / ROWS + lo + i <= slot);
        if (!ok) return false;
        const int last = 63 - __builtin_clzll(ok);
        lo += last * step;
        n = min(step, n - last * step);
        if (n <= 1) break;
    }
    lo = __builtin_amdgcn_readfirstlane(lo);
    start = __builtin_amdgcn_readfirstlane(at(lo));
    len = __builtin_amdgcn_readfirstlane(at(lo + 1)) - start;
    row0 = (slot - (start / ROWS + lo)) * ROWS;
    return row0 < len;
}
// Workgroups go round the eight XCDs in turn.  Where the heads can be dealt out evenly, each XCD gets whole heads, so that a group's keys and
// values stay in one L2.  Otherwise runs of slots (128 rows) are dealt out, the heads of a run side by side: a connected eighth of the slots may
// hold nothing but empty sequences, or the shortest ways of all.  Both backward kernels, fp32, 4096 rows, 4 / 1 heads of 64: 320 us, with
// connected eighths 359, and with 63 empty sequences behind them 332 and 616; but 16 sequences of 256 rows, heads of 128: 128 and 111.
template <int ROWS>
struct AttPlace {
    static constexpr int RUN = 128 / ROWS;
    static unsigned groups(int heads, int slots) {
        if (heads % 8 == 0) return (unsigned)heads * slots;
        const unsigned runs = (unsigned)heads * ((slots + RUN - 1) / RUN);
        return (runs + 7) / 8 * 8 * RUN;
    }
    static __device__ __forceinline__ bool find(int heads, int slots, int &head, int &slot) {
        const int x = blockIdx.x % 8, y = blockIdx.x / 8;
        if (heads % 8 == 0) {
            const int t = x * (heads / 8 * slots) + y;
            head = t / slots;
            slot = t - head * slots;
            return true;
        }
        const int u = y / RUN * 8 + x, run = u / heads;
        head = u - run * heads;
        slot = run * RUN + y % RUN;
        return slot < slots;
    }
};

__device__ __forceinline__ float exchange_max(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float exchange_sum(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// A lane's columns 32 c + result_row of a transposed result to a row in memory, four neighbours at a time
template <class T>
__device__ __forceinline__ void store_block(T *row, int c, const floatx16 &acc, float by, int head_dim, bool add) {
    const int l = threadIdx.x & 63;
#pragma unroll
    for (int r = 0; r < 16; r += 4) {
        const int col = 32 * c + result_row(r, l);
        if (col >= head_dim) continue;
        float v[4] = {acc[r] * by, acc[r + 1] * by, acc[r + 2] * by, acc[r + 3] * by};
        if constexpr (sizeof(T) == 2) {
            uint2 *p = (uint2 *)(row + col);
            if (add) {
                const uint2 o = *p;
                v[0] += __uint_as_float(o.x << 16); v[1] += __uint_as_float(o.x & 0xffff0000u);
                v[2] += __uint_as_float(o.y << 16); v[3] += __uint_as_float(o.y & 0xffff0000u);
            }
            *p = make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]));
        } else {
            float4 *p = (float4 *)(row + col);
            if (add) { const float4 o = *p; v[0] += o.x; v[1] += o.y; v[2] += o.z; v[3] += o.w; }
            *p = make_float4(v[0], v[1], v[2], v[3]);
        }
    }
}

// The PARTS waves of the same rows add up their results (each times its own factor) and store them, D / 32 blocks of columns dealt out
// among them.  area(w): LDS for wave w's results, free by now.
template <class T, int D, int PARTS, class Area>
__device__ __forceinline__ void join_and_store(Area area, const floatx16 (&acc)[D / 32], float factor, T *row, bool exists, float by, int head_dim, bool add) {
    const int l = threadIdx.x & 63, wave = threadIdx.x / 64, part = wave % PARTS;
    if constexpr (PARTS == 1) {
        if (exists) {
#pragma unroll
            for (int c = 0; c < D / 32; ++c) store_block(row, c, acc[c], by * factor, head_dim, add);
        }
        return;
    }
    typedef __attribute__((address_space(3))) float lds_float;
    lds_float *mine = (lds_float *)area(wave);
#pragma unroll
    for (int c = 0; c < D / 32; ++c)
#pragma unroll
        for (int r = 0; r < 16; ++r) mine[(c * 16 + r) * 64 + l] = acc[c][r] * factor;
    __syncthreads();
#pragma unroll
    for (int c = 0; c < D / 32; ++c) {
        if (c % PARTS != part) continue;
        floatx16 sum;
#pragma unroll
        for (int r = 0; r < 16; ++r) sum[r] = 0.f;
#pragma unroll
        for (int i = 0; i < PARTS; ++i) {
            const lds_float *p = (const lds_float *)area(wave - part + i);
#pragma unroll
            for (int r = 0; r < 16; ++r) sum[r] += p[(c * 16 + r) * 64 + l];
        }
        if (exists) store_block(row, c, sum, by, head_dim, add);
    }
}

template <class T, int D, int PARTS>
__global__ __launch_bounds__(256, (AttForm<T, D, PARTS>::TWO_GROUPS ? 2 : 1)) void attention_fwd_kernel(
    AttShape a, const T *__restrict__ q, const T *__restrict__ k, const T *__restrict__ v, T *__restrict__ o, float *__restrict__ lse) {
    typedef AttForm<T, D, PARTS> F;
    typedef typename F::Tile Tile;
    constexpr int R = F::TILE, B = F::BLOCKS, PIECES = F::PIECES, STEPS = F::STEPS;
    __shared__ float stats[2][4][64];
    constexpr int BYTES = Tile::BYTES, SECOND = F::BUFFERS == 2 ? BYTES : 16;
    __shared__ __attribute__((aligned(16))) char k0[BYTES], k1[SECOND], v0[BYTES], v1[SECOND];
    int head, slot, start, len, row0;
    if (!AttPlace<F::ROWS>::find(a.heads, a.slots, head, slot)) return;
    if (!find_rows<F::ROWS>(a, a.slots - 1 - slot, start, len, row0)) return;      // the longest rows first
    const int kv_head = head / (a.heads / a.kv_heads), l = threadIdx.x & 63, wave = threadIdx.x / 64;
    const int part = wave % PARTS, first = row0 + wave / PARTS * 32, row = first + (l & 31);
    Tile tk, tv;
    tk.init(a.k_ld, a.head_dim);
    tv.init(a.v_ld, a.head_dim);
    AttReader<T, D, R> rd;
    rd.init();
    const T *kp = k + start * a.k_ld + (int64_t)kv_head * a.head_dim, *vp = v + start * a.v_ld + (int64_t)kv_head * a.head_dim;
    RowPieces<T, D> qr;
    qr.load(q + (start + first) * a.q_ld + (int64_t)head * a.head_dim, a.q_ld, len - first, a.head_dim);
    const float by = a.scale * LOG2E;
    float top = -INFINITY, sum = 0.f;
    floatx16 acc[D / 32];
#pragma unroll
    for (int c = 0; c < D / 32; ++c)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[c][r] = 0.f;
    const int end = min(len, row0 + F::ROWS);
    auto work = [&](const lds_char *lk, const lds_char *lv, int tile0) {
        const int key0 = tile0 + 32 * B * part;
        if (key0 > first + 31 || key0 >= end) return;
        floatx16 s[B];
#pragma unroll
        for (int b = 0; b < B; ++b) {
#pragma unroll
            for (int r = 0; r < 16; ++r) s[b][r] = 0.f;
#pragma unroll
            for (int p = 0; p < PIECES; ++p) s[b] = Piece<T>::mma(rd.wide(lk, B * part + b, p), qr.p[p], s[b]);
        }
        if (key0 + 32 * B - 1 > first) {
#pragma unroll
            for (int b = 0; b < B; ++b)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (key0 + 32 * b + result_row(r, l) > row) s[b][r] = -INFINITY;
        }
        float most = -INFINITY;
#pragma unroll
        for (int b = 0; b < B; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) most = fmaxf(most, s[b][r]);
        most = exchange_max(most) * by;
        // The sums are kept relative to a maximum that may lie up to 2^8 below the true one: they are only rescaled when it falls
        // further behind, which after the first tiles is rare.
        if (__any(most > top + 8.f)) {
            const float next = fmaxf(top, most), f = top == next ? 1.f : __builtin_amdgcn_exp2f(top - next);
            sum *= f;
#pragma unroll
            for (int c = 0; c < D / 32; ++c)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[c][r] *= f;
            top = next;
        }
        const float base = top == -INFINITY ? 0.f : top;      // no key yet that has a weight: a part of a row may see none, scores may be -infinity
#pragma unroll
        for (int b = 0; b < B; ++b) {
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[b][r] = __builtin_amdgcn_exp2f(s[b][r] * by - base);
                sum += s[b][r];
            }
#pragma unroll
            for (int p = 0; p < STEPS; ++p) {
                const typename Piece<T>::V pr = Piece<T>::from_result(s[b], p);
#pragma unroll
                for (int c = 0; c < D / 32; ++c) acc[c] = Piece<T>::mma(rd.deep(lv, B * part + b, p, c), pr, acc[c]);
            }
        }
    };
    lds_char *lk0 = (lds_char *)k0, *lk1 = (lds_char *)k1, *lv0 = (lds_char *)v0, *lv1 = (lds_char *)v1;
    if constexpr (F::BUFFERS == 2) {
        auto fetch = [&](lds_char *lk, lds_char *lv, int key0) {      // none is under way when the last tile has been used
            if (key0 >= end) return;
            tk.copy(lk, kp + key0 * a.k_ld, len - key0);
            tv.copy(lv, vp + key0 * a.v_ld, len - key0);
        };
        fetch(lk0, lv0, 0);
        for (int key0 = 0; key0 < end; key0 += 2 * R) {
            copies_arrived();
            fetch(lk1, lv1, key0 + R);
            work(lk0, lv0, key0);
            copies_arrived();
            fetch(lk0, lv0, key0 + 2 * R);
            work(lk1, lv1, key0 + R);
        }
    } else {
        tk.load(kp, len);
        tv.load(vp, len);
        for (int key0 = 0; key0 < end; key0 += R) {
            __syncthreads();
            tk.store(lk0);
            tv.store(lv0);
            __syncthreads();
            if (key0 + R < end) {
                tk.load(kp + (key0 + R) * a.k_ld, len - key0 - R);
                tv.load(vp + (key0 + R) * a.v_ld, len - key0 - R);
            }
            work(lk0, lv0, key0);
        }
    }
    sum = exchange_sum(sum);
    float factor = 1.f;
    if constexpr (PARTS > 1) {
        stats[0][wave][l] = top;
        stats[1][wave][l] = sum;
        __syncthreads();             // and everybody is done with the tiles
        const float mine = top;
        top = stats[0][wave - part][l];
#pragma unroll
        for (int i = 1; i < PARTS; ++i) top = fmaxf(top, stats[0][wave - part + i][l]);
        sum = 0.f;
#pragma unroll
        for (int i = 0; i < PARTS; ++i) sum += stats[1][wave - part + i][l] * __builtin_amdgcn_exp2f(stats[0][wave - part + i][l] - top);
        factor = __builtin_amdgcn_exp2f(mine - top);
    }
    auto area = [&](int w) {
        if (F::BUFFERS == 2) return w == 0 ? lk0 : w == 1 ? lk1 : w == 2 ? lv0 : lv1;
        return (w < 2 ? lk0 : lv0) + (w & 1) * F::AREA;
    };
    static_assert(PARTS == 1 || BYTES >= F::AREA * (F::BUFFERS == 2 ? 1 : 2), "");
    if (lse && part == 0 && l < 32 && row < len) lse[(int64_t)head * a.tokens + start + row] = (top + __builtin_amdgcn_logf(sum)) * LN2;
    join_and_store<T, D, PARTS>(area, acc, factor, o + (int64_t)(start + row) * a.o_ld + (int64_t)head * a.head_dim, row < len, 1.f / sum, a.head_dim, false);
}

// dq, and for the other kernel delta and, behind it, lse in powers of two
template <class T, int D, int PARTS>
__global__ __launch_bounds__(256, (AttForm<T, D, PARTS>::TWO_GROUPS && (sizeof(T) == 2 || D == 64) ? 2 : 1)) void attention_dq_kernel(
    AttShape a, const T *__restrict__ go, const T *__restrict__ q, const T *__restrict__ k, const T *__restrict__ v, const T *__restrict__ o,
    const float *__restrict__ lse, T *dq, float *__restrict__ delta, int add) {
    typedef AttForm<T, D, PARTS> F;
    typedef typename F::Tile Tile;
    constexpr int R = F::TILE, B = F::BLOCKS, PIECES = F::PIECES, STEPS = F::STEPS;
    constexpr int BYTES = Tile::BYTES, SECOND = F::BUFFERS == 2 ? BYTES : 16;
    __shared__ __attribute__((aligned(16))) char k0[BYTES], k1[SECOND], v0[BYTES], v1[SECOND];
    int head, slot, start, len, row0;
    if (!AttPlace<F::ROWS>::find(a.heads, a.slots, head, slot)) return;
    if (!find_rows<F::ROWS>(a, a.slots - 1 - slot, start, len, row0)) return;
    const int kv_head = head / (a.heads / a.kv_heads), l = threadIdx.x & 63, wave = threadIdx.x / 64;
    const int part = wave % PARTS, first = row0 + wave / PARTS * 32, row = first + (l & 31);
    Tile tk, tv;
    tk.init(a.k_ld, a.head_dim);
    tv.init(a.v_ld, a.head_dim);
    AttReader<T, D, R> rd;
    rd.init();
    const T *kp = k + start * a.k_ld + (int64_t)kv_head * a.head_dim, *vp = v + start * a.v_ld + (int64_t)kv_head * a.head_dim;
    RowPieces<T, D> qr, gr;
    qr.load(q + (start + first) * a.q_ld + (int64_t)head * a.head_dim, a.q_ld, len - first, a.head_dim);
    gr.load(go + (start + first) * a.o_ld + (int64_t)head * a.head_dim, a.o_ld, len - first, a.head_dim);
    float dot = 0.f;
    if (row < len) {
        const int64_t at = (start + row) * a.o_ld + (int64_t)head * a.head_dim;
#pragma unroll
        for (int p = 0; p < PIECES; ++p) {
            const int col = (2 * p + (l >> 5)) * 8;
            if (col < a.head_dim) dot += Piece<T>::dot(o + at + col, go + at + col);
        }
    }
    dot = exchange_sum(dot);
    const int64_t at = (int64_t)head * a.tokens + start + row;
    const float by = a.scale * LOG2E, ls = row < len ? lse[at] * LOG2E : 0.f;
    const int end = min(len, row0 + F::ROWS);
    if constexpr (sizeof(T) == 2) {
        if (row0 < FEW_KEYS) {
            __shared__ float sums[4][32];
            float sum = 0.f;
            for (int key0 = 0; key0 < end; key0 += R) {
                __syncthreads();
                tk.copy((lds_char *)k0, kp + key0 * a.k_ld, len - key0);
                tv.copy((lds_char *)v0, vp + key0 * a.v_ld, len - key0);
                copies_arrived();
#pragma unroll
                for (int b = 0; b < B; ++b) {
                    floatx16 s, d;
#pragma unroll
                    for (int r = 0; r < 16; ++r) s[r] = d[r] = 0.f;
#pragma unroll
                    for (int p = 0; p < PIECES; ++p) s = Piece<T>::mma(rd.wide((lds_char *)k0, B * part + b, p), qr.p[p], s);
#pragma unroll
                    for (int p = 0; p < PIECES; ++p) d = Piece<T>::mma(rd.wide((lds_char *)v0, B * part + b, p), gr.p[p], d);
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if (key0 + 32 * (B * part + b) + result_row(r, l) <= row) sum += __builtin_amdgcn_exp2f(s[r] * by - ls) * d[r];
                }
            }
            sum = exchange_sum(sum);
            if (l < 32) sums[wave][l] = sum;
            __syncthreads();
            dot = 0.f;
#pragma unroll
            for (int w = 0; w < PARTS; ++w) dot += sums[wave / PARTS * PARTS + w][l & 31];
        }
    }
    if (part == 0 && l < 32 && row < len) {
        delta[at] = dot;
        delta[at + (int64_t)a.heads * a.tokens] = ls;
    }
    floatx16 acc[D / 32];
#pragma unroll
    for (int c = 0; c < D / 32; ++c)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[c][r] = 0.f;
    auto work = [&](const lds_char *lk, const lds_char *lv, int tile0) {
        const int key0 = tile0 + 32 * B * part;
        if (key0 > first + 31 || key0 >= end) return;
        const bool edge = key0 + 32 * B - 1 > first;
#pragma unroll
        for (int b = 0; b < B; ++b) {
            floatx16 s, d;
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] = d[r] = 0.f;
#pragma unroll
            for (int p = 0; p < PIECES; ++p) s = Piece<T>::mma(rd.wide(lk, B * part + b, p), qr.p[p], s);
#pragma unroll
            for (int p = 0; p < PIECES; ++p) d = Piece<T>::mma(rd.wide(lv, B * part + b, p), gr.p[p], d);
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(s[r] * by - ls) * (d[r] - dot);
            if (edge) {
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (key0 + 32 * b + result_row(r, l) > row) s[r] = 0.f;
            }
#pragma unroll
            for (int p = 0; p < STEPS; ++p) {
                const typename Piece<T>::V ds = Piece<T>::from_result(s, p);
#pragma unroll
                for (int c = 0; c < D / 32; ++c) acc[c] = Piece<T>::mma(rd.deep(lk, B * part + b, p, c), ds, acc[c]);
            }
        }
    };
    lds_char *lk0 = (lds_char *)k0, *lk1 = (lds_char *)k1, *lv0 = (lds_char *)v0, *lv1 = (lds_char *)v1;
    if constexpr (F::BUFFERS == 2) {
        auto fetch = [&](lds_char *lk, lds_char *lv, int key0) {      // none is under way when the last tile has been used
            if (key0 >= end) return;
            tk.copy(lk, kp + key0 * a.k_ld, len - key0);
            tv.copy(lv, vp + key0 * a.v_ld, len - key0);
        };
        fetch(lk0, lv0, 0);
        for (int key0 = 0; key0 < end; key0 += 2 * R) {
            copies_arrived();
            fetch(lk1, lv1, key0 + R);
            work(lk0, lv0, key0);
            copies_arrived();
            fetch(lk0, lv0, key0 + 2 * R);
            work(lk1, lv1, key0 + R);
        }
    } else {
        tk.load(kp, len);
        tv.load(vp, len);
        for (int key0 = 0; key0 < end; key0 += R) {
            __syncthreads();
            tk.store(lk0);
            tv.store(lv0);
            __syncthreads();
            if (key0 + R < end) {
                tk.load(kp + (key0 + R) * a.k_ld, len - key0 - R);
                tv.load(vp + (key0 + R) * a.v_ld, len - key0 - R);
            }
            work(lk0, lv0, key0);
        }
    }
    if (PARTS > 1) __syncthreads();      // everybody is done with the tiles
    auto area = [&](int w) {
        if (F::BUFFERS == 2) return w == 0 ? lk0 : w == 1 ? lk1 : w == 2 ? lv0 : lv1;
        return (w < 2 ? lk0 : lv0) + (w & 1) * F::AREA;
    };
    static_assert(PARTS == 1 || BYTES >= F::AREA * (F::BUFFERS == 2 ? 1 : 2), "");
    join_and_store<T, D, PARTS>(area, acc, 1.f, dq + (int64_t)(start + row) * a.q_ld + (int64_t)head * a.head_dim, row < len, a.scale, a.head_dim, add);
}

// dk and dv: a wave holds 32 keys and walks along the rows behind them, head by head of the group.  Where the grid has more than one range (y),
// a way is cut into as many as it has room for: each workgroup takes its share and leaves fp32 sums in `ranges` ([range][token][kv_head]
// [head_dim], dk's and behind them dv's), which attention_join_kernel adds up in order; `counts` tells it a token's number of ranges.  A way too
// short for two is one workgroup's, which writes the results, and the others of its keys end at once.
template <class T, int D, int PARTS>
__global__ __launch_bounds__(256, (AttForm<T, D, PARTS>::TWO_GROUPS && (sizeof(T) == 2 || D == 64) ? 2 : 1)) void attention_dkv_kernel(
    AttShape a, const T *__restrict__ go, const T *__restrict__ q, const T *__restrict__ k, const T *__restrict__ v, const float *__restrict__ delta,
    T *dk, T *dv, int add_k, int add_v, float *__restrict__ ranges, int32_t *__restrict__ counts) {
    typedef AttForm<T, D, PARTS> F;
    typedef typename F::Tile Tile;
    constexpr int R = F::TILE, B = F::BLOCKS, PIECES = F::PIECES, STEPS = F::STEPS;
    constexpr int BYTES = Tile::BYTES, SECOND = F::BUFFERS == 2 ? BYTES : 16;
    __shared__ __attribute__((aligned(16))) char q0[BYTES], q1[SECOND], g0[BYTES], g1[SECOND];
    __shared__ __attribute__((aligned(16))) float stat0[256], stat1[256];      // delta of a tile's rows, their lse
    int kv_head, slot, start, len, key0;
    if (!AttPlace<F::ROWS>::find(a.kv_heads, a.slots, kv_head, slot)) return;
    if (!find_rows<F::ROWS>(a, slot, start, len, key0)) return;
    const int group = a.heads / a.kv_heads, l = threadIdx.x & 63, wave = D > 64 ? threadIdx.x / 64 : uniform_wave();
    const int part = wave % PARTS, first = key0 + wave / PARTS * 32, key = first + (l & 31);
    const int from = key0 / R * R, tiles = (len - from + R - 1) / R, count = min((int)gridDim.y, (tiles * group + F::RANGE_TILES - 1) / F::RANGE_TILES);
    if ((int)blockIdx.y >= count) return;
    Tile tq, tg;
    tq.init(a.q_ld, a.head_dim);
    tg.init(a.o_ld, a.head_dim);
    AttReader<T, D, R> rd;
    rd.init();
    RowPieces<T, D> kr, vr;
    kr.load(k + (start + first) * a.k_ld + (int64_t)kv_head * a.head_dim, a.k_ld, len - first, a.head_dim);
    vr.load(v + (start + first) * a.v_ld + (int64_t)kv_head * a.head_dim, a.v_ld, len - first, a.head_dim);
    const float by = a.scale * LOG2E;
    const int limit = key - 4 * (l >> 5);
    floatx16 ak[D / 32], av[D / 32];
#pragma unroll
    for (int c = 0; c < D / 32; ++c)
#pragma unroll
        for (int r = 0; r < 16; ++r) ak[c][r] = av[c][r] = 0.f;
    const int begin = (int)((int64_t)tiles * group * blockIdx.y / count), all = (int)((int64_t)tiles * group * (blockIdx.y + 1) / count);
    auto place = [&](int t, int &head, int &row) {
        const int g = t / tiles;
        head = kv_head * group + g;
        row = from + (t - g * tiles) * R;
    };
    // fp32: one product's operands at a time, or they do not fit the registers
    auto narrow = [] { if (sizeof(T) == 4) __builtin_amdgcn_sched_barrier(0); };
    auto work = [&](const lds_char *lq, const lds_char *lg, const lds_char *ls, int t) {
        const int row = from + t % tiles * R + 32 * B * part;
        if (t >= all || row + 32 * B - 1 < first || row >= len) return;
        const bool edge = row < first + 31;
#pragma unroll
        for (int b = 0; b < B; ++b) {
            floatx16 s, d;
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] = d[r] = 0.f;
#pragma unroll
            for (int p = 0; p < PIECES; ++p) s = Piece<T>::mma(rd.wide(lq, B * part + b, p), kr.p[p], s);
            narrow();
#pragma unroll
            for (int p = 0; p < PIECES; ++p) d = Piece<T>::mma(rd.wide(lg, B * part + b, p), vr.p[p], d);
            narrow();
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
                const lds_char *at = ls + (32 * (B * part + b) + result_row(r, l)) * 4;
                const floatx4 y = *(const __attribute__((address_space(3))) floatx4 *)at, x = *(const __attribute__((address_space(3))) floatx4 *)(at + 512);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    s[r + j] = __builtin_amdgcn_exp2f(s[r + j] * by - x[j]);
                    if (D > 64 && edge && row + 32 * b + result_row(r + j, 0) < limit) s[r + j] = 0.f;
                    d[r + j] = D > 64 ? s[r + j] * (d[r + j] - y[j]) : d[r + j] - y[j];
                }
            }
            // 64 wide in a branch of its own: 185 us (bf16, two sequences of 4096 rows, 16 heads of 64), in the loop above 229.  128 wide the branch's
            // limit does not fit the registers: 42 spilled in the loop, where a reload waits for the copies under way; the form above none
            if (D <= 64) {
                if (edge) clear_before(s, key - row - 32 * b);
#pragma unroll
                for (int r = 0; r < 16; ++r) d[r] *= s[r];
            }
#pragma unroll
            for (int p = 0; p < STEPS; ++p) {
                const typename Piece<T>::V pr = Piece<T>::from_result(s, p), ds = Piece<T>::from_result(d, p);
#pragma unroll
                for (int c = 0; c < D / 32; ++c) av[c] = Piece<T>::mma(rd.deep(lg, B * part + b, p, c), pr, av[c]);
#pragma unroll
                for (int c = 0; c < D / 32; ++c) ak[c] = Piece<T>::mma(rd.deep(lq, B * part + b, p, c), ds, ak[c]);
                narrow();
            }
        }
    };
    lds_char *lq0 = (lds_char *)q0, *lq1 = (lds_char *)q1, *lg0 = (lds_char *)g0, *lg1 = (lds_char *)g1, *ls0 = (lds_char *)stat0, *ls1 = (lds_char *)stat1;
    if constexpr (F::BUFFERS == 2) {
        auto fetch = [&](lds_char *lq, lds_char *lg, lds_char *ls, int t) {      // none is under way when the last tile has been used
            if (t >= all) return;
            int head, row;
            place(t, head, row);
            tq.copy(lq, q + (start + row) * a.q_ld + (int64_t)head * a.head_dim, len - row);
            tg.copy(lg, go + (start + row) * a.o_ld + (int64_t)head * a.head_dim, len - row);
            // 64 rows' delta (waves 0, 1) and lse (2, 3); rows behind the sequence: 0
            const int w = uniform_wave();
            if (64 * (w & 1) < R) {
                const float *p = delta + (w / 2 * a.heads + head) * (int64_t)a.tokens + start + row;
                const __amdgpu_buffer_rsrc_t r = buffer_of(p, (unsigned)min(len - row, R) * 4);
                __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void *)(ls + w * 256), 4, (64 * (w & 1) + l) * 4, 0, 0, 0);
            }
        };
        fetch(lq0, lg0, ls0, begin);
        for (int t = begin; t < all; t += 2) {
            copies_arrived();
            fetch(lq1, lg1, ls1, t + 1);
            work(lq0, lg0, ls0, t);
            copies_arrived();
            fetch(lq0, lg0, ls0, t + 2);
            work(lq1, lg1, ls1, t + 1);
        }
    } else {
        float stat = 0.f;            // threads 0 .. 127: a row's delta, 128 .. 255: its lse
        const int stat_row = threadIdx.x & 127;
        auto load = [&](int t) {
            int head, row;
            place(t, head, row);
            tq.load(q + (start + row) * a.q_ld + (int64_t)head * a.head_dim, len - row);
            tg.load(go + (start + row) * a.o_ld + (int64_t)head * a.head_dim, len - row);
            stat = stat_row < R && row + stat_row < len ? delta[((int64_t)(threadIdx.x / 128) * a.heads + head) * a.tokens + start + row + stat_row] : 0.f;
        };
        if (begin < all) load(begin);
        for (int t = begin; t < all; ++t) {
            __syncthreads();
            tq.store(lq0);
            tg.store(lg0);
            stat0[threadIdx.x] = stat;
            __syncthreads();
            if (t + 1 < all) load(t + 1);
            work(lq0, lg0, ls0, t);
        }
    }
    auto area = [&](int w) {
        if (F::BUFFERS == 2) return w == 0 ? lq0 : w == 1 ? lq1 : w == 2 ? lg0 : lg1;
        return (w < 2 ? lq0 : lg0) + (w & 1) * F::AREA;
    };
    static_assert(PARTS == 1 || BYTES >= F::AREA * (F::BUFFERS == 2 ? 1 : 2), "");
    if (PARTS > 1) __syncthreads();      // everybody is done with the tiles
    if (ranges && blockIdx.y == 0 && kv_head == 0 && part == 0 && l < 32 && key < len) counts[start + key] = count;
    if (count > 1) {
        float *row = ranges + (((int64_t)blockIdx.y * a.tokens + start + key) * a.kv_heads + kv_head) * a.head_dim;
        join_and_store<float, D, PARTS>(area, ak, 1.f, row, key < len, a.scale, a.head_dim, false);
        if (PARTS > 1) __syncthreads();
        row += (int64_t)gridDim.y * a.tokens * a.kv_heads * a.head_dim;
        join_and_store<float, D, PARTS>(area, av, 1.f, row, key < len, 1.f, a.head_dim, false);
        return;
    }
    join_and_store<T, D, PARTS>(area, ak, 1.f, dk + (int64_t)(start + key) * a.k_ld + (int64_t)kv_head * a.head_dim, key < len, a.scale, a.head_dim, add_k);
    if (PARTS > 1) __syncthreads();
    join_and_store<T, D, PARTS>(area, av, 1.f, dv + (int64_t)(start + key) * a.v_ld + (int64_t)kv_head * a.head_dim, key < len, 1.f, a.head_dim, add_v);
}

// dk (grid y 0) or dv (1) = the sum of its ranges where there is more than one, four values a thread; tokens of no sequence are left alone
template <class T>
__global__ __launch_bounds__(256) void attention_join_kernel(AttShape a, const float *__restrict__ ranges, const int32_t *__restrict__ counts, int most, T *dk,
                                                             T *dv, int add_k, int add_v) {
    const int width = a.kv_heads * a.head_dim, per_row = width / 4;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, row = i / per_row, all = (int64_t)a.tokens * width;
    if (row >= a.tokens || row < a.cu[0] || row >= a.cu[a.seqs]) return;
    const int count = min(counts[row], most);
    if (count < 2) return;
    const int c = (int)(i - row * per_row) * 4;
    const float *p = ranges + (blockIdx.y ? most * all : 0) + row * width + c;
    float4 v = *(const float4 *)p;
    for (int r = 1; r < count; ++r) {
        const float4 w = *(const float4 *)(p + r * all);
        v.x += w.x; v.y += w.y; v.z += w.z; v.w += w.w;
    }
    const bool add = blockIdx.y ? add_v : add_k;
    T *out = blockIdx.y ? dv + row * a.v_ld + c : dk + row * a.k_ld + c;
    if constexpr (sizeof(T) == 2) {
        if (add) {
            const uint2 o = *(const uint2 *)out;
            v.x += __uint_as_float(o.x << 16); v.y += __uint_as_float(o.x & 0xffff0000u);
            v.z += __uint_as_float(o.y << 16); v.w += __uint_as_float(o.y & 0xffff0000u);
        }
        *(uint2 *)out = make_uint2(pack_bf16(v.x, v.y), pack_bf16(v.z, v.w));
    } else {
        if (add) { const float4 o = *(const float4 *)out; v.x += o.x; v.y += o.y; v.z += o.z; v.w += o.w; }
        *(float4 *)out = v;
    }
}

// Rows in front of the first sequence and behind the last one of up to three tensors (grid y): zero.  Nothing to do where the offsets cover
// all tokens, which only the device knows.
struct OutsideRows { float *p[3]; int width[3]; };
__global__ __launch_bounds__(256) void attention_clear_outside_kernel(const int32_t *__restrict__ cu, int seqs, int tokens, OutsideRows r) {
    const int first = min(max(cu[0], 0), tokens), behind = min(max(cu[seqs], first), tokens), per_row = r.width[blockIdx.y] / 4;
    const int64_t all = (int64_t)(first + tokens - behind) * per_row;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
        const int64_t at = i < (int64_t)first * per_row ? i : i + (int64_t)(behind - first) * per_row;
        ((float4 *)r.p[blockIdx.y])[at] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
}

AttShape att_shape(int dtype, const int32_t *cu, int seqs, int64_t tokens, int heads, int kv_heads, int head_dim, int64_t q_ld, int64_t k_ld,
                   int64_t v_ld, int64_t o_ld, float scale) {
    if (dtype != MONET_F32 && dtype != MONET_BF16) throw KernelError("attention: dtype must be MONET_F32 or MONET_BF16");
    if (seqs < 1 || tokens < 0 || heads < 1 || kv_heads < 1 || heads % kv_heads) throw KernelError("attention: bad shape (heads must be a multiple of kv_heads)");
    if (head_dim < 8 || head_dim > 128 || head_dim % 8) throw KernelError("attention: head_dim must be a multiple of 8 between 8 and 128");
    if (!(scale > 0.f) || scale > 1e30f) throw KernelError("attention: scale must be positive and finite");
    const int64_t step = dtype == MONET_BF16 ? 8 : 4;
    for (int64_t ld : {q_ld, o_ld})
        if (ld < (int64_t)heads * head_dim || ld % step || ld >= (1 << 23)) throw KernelError("attention: row strides must hold all heads, be a multiple of 16 bytes and below 2^23 elements");
    for (int64_t ld : {k_ld, v_ld})
        if (ld < (int64_t)kv_heads * head_dim || ld % step || ld >= (1 << 23)) throw KernelError("attention: row strides must hold all heads, be a multiple of 16 bytes and below 2^23 elements");
    // a launch takes less than 2^24 workgroups; what comes on top of a workgroup for 64 rows or a sequence: runs of slots, 32 keys to a workgroup
    if (tokens > 0x7fffffff || (tokens / 64 + seqs + 8) * heads >= (1 << 24) - (1 << 11)) throw KernelError("attention: too many tokens");
    if (!cu) throw KernelError("attention: null pointer");
    if ((uintptr_t)cu % 4) throw KernelError("attention: offsets and lse must be 4-byte aligned");
    return AttShape{cu, seqs, (int)tokens, heads, kv_heads, head_dim, 0, q_ld, k_ld, v_ld, o_ld, scale};
}
void check_tensors(std::initializer_list<const void *> ptrs) {
    for (const void *p : ptrs) {
        if (!p) throw KernelError("attention: null pointer");
        if ((uintptr_t)p % 16) throw KernelError("attention: tensors must be 16-byte aligned");
    }
}
void check_lse(const float *lse) {
    if ((uintptr_t)lse % 4) throw KernelError("attention: offsets and lse must be 4-byte aligned");
}

// Rows of the forward and the first backward kernel: 128 to a workgroup where that gives four workgroups to a CU (fp32 with 128 columns, whose
// tiles take more of LDS: two), 64 below.  How long the sequences are does not matter for it, and the host does not know.  Forward, 64 and 128
// rows: bf16 8 x 16 heads of 512 rows 14.4 and 15.5 us, one sequence of 4000 rows and 8 heads 40 and 51, two of 8192 and 32 heads 1190 and 1084,
// 82 of 100 rows and 32 heads of 128 72 and 56; fp32 4 x 16 heads of 512 rows 28 and 36, one of 4096 and 32 heads of 128 1135 and 813, 205 of 40
// and 32 heads of 128 320 and 213 (where its backward kernel loses what this one gains).
template <class T, int D>
int row_parts(const AttShape &a) {
    const int64_t full = (int64_t)(a.tokens / 128) * a.heads;
    return full >= (sizeof(T) == 4 && D == 128 ? 512 : 1024) ? 1 : 2;
}
// The second backward kernel has fewer workgroups (key heads) with a longer way each (the rows behind a key, of every head of the group).
// Where 128 keys to a workgroup do not give four workgroups to a CU, ways are cut into ranges, each as its own length asks for
// (attention_dkv_kernel): the launch has as many as the longest way there can be, all tokens in one sequence, has room for.  So empty and tiny
// sequences, of which padded offsets have many, take no ranges from a long one.  bf16: with less than one workgroup to a CU, and unless
// sequences of the mean length give ranges for two, a workgroup takes 32 keys.  Both backward kernels, us:
//   bf16, 10000 rows, 4 / 1 heads: uncut 1865, 14 ranges 559, 32 keys in 4 ranges 794;  1024 rows, 8 heads of 64: 47, with 32 keys 28
//   fp32, 2048 ragged rows, 12 / 4 heads of 64: 587 uncut, 16 ranges 158
//   as the mean length has it, and so: bf16, 4000 rows and nine empty sequences, 8 / 1 heads of 64, 291 and 123; 12000 and 255 empty, 4 / 1 heads
//   of 128, 2000 and 770; fp32, 6000 and 63 empty, 16 / 4 heads of 128, 7900 and 4310; 5000, 3, 900 and 2000 rows, 8 / 4 heads of 128, 2450 and
//   2040; but bf16, 32 sequences of 128 rows, 32 / 4 heads of 64, 63 and 74: workgroups that find no range to work on, and a launch to join none
//   bf16, 32 keys in one range and up to two: 4 sequences of 1024 rows, 4 / 4 heads of 128, 61 and 64; 3258 rows, 8 / 8 heads of 40, 77 and 84; 6000
//   and 63 empty, 16 / 4 heads of 128, 1063 and 755
//   bf16, 128 and 32 keys: 256 sequences of 32 rows, 16 / 4 heads of 128, 139 and 187; 16 of 256, 4 / 1 heads of 128, 71 and 42
struct KeyForm { int parts, ranges; };
KeyForm key_form(const AttShape &a, bool fp32) {
    const int64_t full = std::max<int64_t>(1, (int64_t)(a.tokens / 128) * a.kv_heads), group = a.heads / a.kv_heads, mean = a.tokens / a.seqs;
    // ranges until there are 1024 workgroups, if a way of so many rows has room for them
    const auto cut = [](int64_t groups, int64_t way, int64_t least) {
        return std::max<int64_t>(1, std::min<int64_t>({(1024 + groups - 1) / groups, (way + least - 1) / least, 16}));
    };
    const int64_t longest = a.tokens * group;
    if (fp32) return {1, (int)cut(full, longest, AttForm<float, 64, 1>::RANGE_ROWS)};
    constexpr int LEAST = AttForm<unsigned short, 64, 1>::RANGE_ROWS;
    if (full >= 256 || (mean >= 64 && full * std::min<int64_t>(mean * group / LEAST, 16) >= 512)) return {1, full >= 1024 ? 1 : (int)cut(full, longest, LEAST)};
    constexpr int LEAST4 = AttForm<unsigned short, 64, 4>::RANGE_ROWS;
    if (longest < (4 * full >= 512 ? 8 : 2) * LEAST4) return {4, 1};      // two ranges at most, of ways that are not long
    return {4, (int)cut(4 * full, longest, LEAST4)};
}

template <class T, int D, int PARTS>
void fwd_launch(hipStream_t st, AttShape a, const void *q, const void *k, const void *v, void *o, float *lse) {
    a.slots = a.tokens / AttForm<T, D, PARTS>::ROWS + a.seqs;
    hipLaunchKernelGGL((attention_fwd_kernel<T, D, PARTS>), dim3(AttPlace<AttForm<T, D, PARTS>::ROWS>::groups(a.heads, a.slots)), dim3(256), 0, st, a, (const T *)q, (const T *)k, (const T *)v, (T *)o, lse);
    hip_check(hipGetLastError(), "attention forward launch");
}
template <class T, int D>
void fwd_form(hipStream_t st, const AttShape &a, const void *q, const void *k, const void *v, void *o, float *lse) {
    const int parts = row_parts<T, D>(a);
    if (parts == 1) fwd_launch<T, D, 1>(st, a, q, k, v, o, lse);
    else fwd_launch<T, D, 2>(st, a, q, k, v, o, lse);
}
struct BwdArgs {
    const void *go, *q, *k, *v, *o;
    const float *lse;
    void *dq, *dk, *dv;
    float *delta, *ranges;
    int32_t *counts;
    int accumulate;
};
int64_t count_bytes(const AttShape &a) { return ((int64_t)a.tokens * 4 + 255) / 256 * 256; }
int64_t stat_bytes(const AttShape &a) { return (2 * (int64_t)a.heads * a.tokens * 4 + 255) / 256 * 256; }
template <class T, int D, int PARTS>
void dq_launch(hipStream_t st, AttShape a, const BwdArgs &b) {
    a.slots = a.tokens / AttForm<T, D, PARTS>::ROWS + a.seqs;
    hipLaunchKernelGGL((attention_dq_kernel<T, D, PARTS>), dim3(AttPlace<AttForm<T, D, PARTS>::ROWS>::groups(a.heads, a.slots)), dim3(256), 0, st, a, (const T *)b.go, (const T *)b.q, (const T *)b.k,
                       (const T *)b.v, (const T *)b.o, b.lse, (T *)b.dq, b.delta, b.accumulate & 1);
    hip_check(hipGetLastError(), "attention query gradient launch");
}
template <class T, int D, int PARTS>
void dkv_launch(hipStream_t st, AttShape a, const BwdArgs &b, int ranges) {
    a.slots = a.tokens / AttForm<T, D, PARTS>::ROWS + a.seqs;
    hipLaunchKernelGGL((attention_dkv_kernel<T, D, PARTS>), dim3(AttPlace<AttForm<T, D, PARTS>::ROWS>::groups(a.kv_heads, a.slots), ranges), dim3(256), 0, st, a, (const T *)b.go, (const T *)b.q,
                       (const T *)b.k, (const T *)b.v, b.delta, (T *)b.dk, (T *)b.dv, b.accumulate & 2, b.accumulate & 4, ranges > 1 ? b.ranges : nullptr, b.counts);
    hip_check(hipGetLastError(), "attention key gradient launch");
    if (ranges > 1) {
        const int64_t blocks = ((int64_t)a.tokens * a.kv_heads * a.head_dim / 4 + 255) / 256;
        hipLaunchKernelGGL((attention_join_kernel<T>), dim3((unsigned)blocks, 2), dim3(256), 0, st, a, b.ranges, b.counts, ranges, (T *)b.dk, (T *)b.dv,
                           b.accumulate & 2, b.accumulate & 4);
        hip_check(hipGetLastError(), "attention join launch");
    }
}
template <class T, int D>
void bwd_form(hipStream_t st, const AttShape &a, const BwdArgs &b) {
    const int parts = row_parts<T, D>(a);
    if (parts == 1) dq_launch<T, D, 1>(st, a, b);
    else dq_launch<T, D, 2>(st, a, b);
    const KeyForm f = key_form(a, sizeof(T) == 4);
    if (sizeof(T) == 4 || f.parts == 1) dkv_launch<T, D, 1>(st, a, b, f.ranges);
    else if constexpr (sizeof(T) == 2) dkv_launch<T, D, 4>(st, a, b, f.ranges);
}

}  // namespace

void attention_fwd(hipStream_t st, int dtype, const void *q, const void *k, const void *v, void *o, float *lse, const int32_t *cu, int seqs,
                   int64_t tokens, int heads, int kv_heads, int head_dim, int64_t q_ld, int64_t k_ld, int64_t v_ld, int64_t o_ld, float scale) {
    const AttShape a = att_shape(dtype, cu, seqs, tokens, heads, kv_heads, head_dim, q_ld, k_ld, v_ld, o_ld, scale);
    if (!tokens) return;
    check_tensors({q, k, v, o});
    check_lse(lse);
    if (dtype == MONET_BF16) (head_dim <= 64 ? fwd_form<unsigned short, 64> : fwd_form<unsigned short, 128>)(st, a, q, k, v, o, lse);
    else (head_dim <= 64 ? fwd_form<float, 64> : fwd_form<float, 128>)(st, a, q, k, v, o, lse);
}

void attention_clear_outside(hipStream_t st, const int32_t *cu, int seqs, int64_t tokens, std::initializer_list<std::pair<float *, int>> tensors) {
    OutsideRows r{};
    int n = 0;
    for (const auto &t : tensors)
        if (t.first) { r.p[n] = t.first; r.width[n++] = t.second; }
    if (!n || !tokens) return;
    hipLaunchKernelGGL(attention_clear_outside_kernel, dim3(64, n), dim3(256), 0, st, cu, seqs, (int)tokens, r);
    hip_check(hipGetLastError(), "attention clear launch");
}

size_t attention_bwd_workspace_bytes(int dtype, int seqs, int64_t tokens, int heads, int kv_heads, int head_dim) {
    static const int32_t none = 0;
    const AttShape a = att_shape(dtype, &none, seqs, tokens, heads, kv_heads, head_dim, (int64_t)heads * head_dim, (int64_t)kv_heads * head_dim,
              (int64_t)kv_heads * head_dim, (int64_t)heads * head_dim, 1.f);
    const int ranges = key_form(a, dtype == MONET_F32).ranges;
    return (size_t)(stat_bytes(a) + (ranges > 1 ? count_bytes(a) + 2 * (int64_t)ranges * tokens * kv_heads * head_dim * 4 : 0));
}

void attention_bwd(hipStream_t st, int dtype, const void *go, const void *q, const void *k, const void *v, const void *o, const float *lse, void *dq,
                   void *dk, void *dv, const int32_t *cu, int seqs, int64_t tokens, int heads, int kv_heads, int head_dim, int64_t q_ld, int64_t k_ld,
                   int64_t v_ld, int64_t o_ld, float scale, int accumulate, void *ws, size_t ws_bytes) {
    const AttShape a = att_shape(dtype, cu, seqs, tokens, heads, kv_heads, head_dim, q_ld, k_ld, v_ld, o_ld, scale);
    if (!tokens) return;
    check_tensors({go, q, k, v, o, dq, dk, dv});
    if (!lse) throw KernelError("attention: null pointer");
    check_lse(lse);
    if (accumulate & ~7) throw KernelError("attention: accumulate has one bit each for dq, dk and dv");
    if (!ws || ws_bytes < attention_bwd_workspace_bytes(dtype, seqs, tokens, heads, kv_heads, head_dim))
        throw KernelError("attention: workspace too small");
    if ((uintptr_t)ws % 256) throw KernelError("attention: the workspace must be 256-byte aligned");
    char *behind = (char *)ws + stat_bytes(a);
    const BwdArgs b{go, q, k, v, o, lse, dq, dk, dv, (float *)ws, (float *)(behind + count_bytes(a)), (int32_t *)behind, accumulate};
    if (dtype == MONET_BF16) (head_dim <= 64 ? bwd_form<unsigned short, 64> : bwd_form<unsigned short, 128>)(st, a, b);
    else (head_dim <= 64 ? bwd_form<float, 64> : bwd_form<float, 128>)(st, a, b);
}

}  // namespace monet
