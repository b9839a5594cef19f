// Tiles of bf16 matrices in LDS: copies from memory straight into it, and the reads that feed v_mfma_f32_32x32x16_bf16.
#pragma once
#include <hip/hip_runtime.h>

#include "bf16_pieces.hpp"
#include "buffer_addr.hpp"

namespace monet {

typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef short shortx4 __attribute__((ext_vector_type(4)));
typedef unsigned uintx2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) char lds_char;

// A lane of v_mfma_f32_32x32x16_bf16 holds of its operands row (column) l & 31 at reduction indices 8 (l >> 5) .. + 7, and of the
// result column l & 31 at rows result_row(r, l), r = 0 .. 15.
__device__ __forceinline__ int result_row(int r, int lane) { return (r & 3) + 8 * (r >> 2) + 4 * (lane >> 5); }

__device__ __forceinline__ floatx16 mfma_bf16(bf16x8 a, bf16x8 b, floatx16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

// 16 bytes a lane from memory to LDS without a register in between: lane l's arrive at dst + 16 l (dst the same for the wave).
// Absent offsets (buffer_addr.hpp) arrive as zeros.
__device__ __forceinline__ void copy_to_lds(__amdgpu_buffer_rsrc_t r, lds_char *dst, unsigned voff, unsigned soff) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void *)dst, 16, (int)voff, (int)soff, 0, 0);
}

// The workgroup's copies so far are in LDS, and nobody reads any more what was there before.
__device__ __forceinline__ void copies_arrived() {
    __builtin_amdgcn_s_waitcnt(0x0f70);      // vmcnt(0): a barrier alone does not wait for them
    __syncthreads();
}

// Tiles whose rows run along the reduction ("wide": 128 bytes a row).  A read takes 16 bytes at the same place of 32 rows, so the
// eight pieces of a row are turned by the row: every 8 rows (and every 16, over 256 bytes) meet all banks.  So do the 32-byte pairs of
// four rows that a turned read (below) takes of such a tile.
__device__ __forceinline__ unsigned wide_turn(unsigned row) { return (((row & 3) << 1) | ((row >> 2) & 1)) ^ ((row >> 2) & 2); }

// Tiles whose rows run across it ("deep": one reduction index a row, COLS values).  ds_read_b64_tr_b16 gives lane i of 16 the i-th
// of 16 neighbouring columns at four reduction indices; the lanes' addresses are 8-byte pieces of four rows.  The 32-byte pairs of a
// row are turned by 0, 3, 5 or 6, so that the four rows of 16 lanes (and of 32, over 256 bytes) meet all banks.
__device__ __forceinline__ unsigned deep_turn(unsigned row) { return (0x6530u >> (4 * (row & 3))) & 7; }

__device__ __forceinline__ shortx4 read_turned(const lds_char *p) {
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) shortx4 *)p);
}
__device__ __forceinline__ bf16x8 join(shortx4 a, shortx4 b) {
    typedef short shortx8 __attribute__((ext_vector_type(8)));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}
__device__ __forceinline__ bf16x8 read_wide(const lds_char *p) { return *(const __attribute__((address_space(3))) bf16x8 *)p; }

__device__ __forceinline__ float bf16_float(unsigned short v) { return __uint_as_float((unsigned)v << 16); }
__device__ __forceinline__ unsigned short float_bf16(float v) { return (unsigned short)(pack_bf16(v, v) & 0xffffu); }

}  // namespace monet
