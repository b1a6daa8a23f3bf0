// The 4-bit prefix cache: a page holds 32 consecutive rows of one (sequence, key/value head), keys and values.
//
//   offset      content
//   0           key codes    [D / 32 chunks][32 rows][16 bytes]: chunk c of a row holds its channels 32c .. 32c + 31
//   16 D        value codes  [D channels][16 bytes]: the 32 rows of one channel
//   32 D        bf16 key scale [32], key offset [32], value scale [32], value offset [32]
//
// In the 16 bytes of a chunk, value 8w + 2i + h (w, i = 0..3, h = 0, 1) is the nibble at bits 4i + 16h of 32-bit word w,
// so that one shift and one mask give two neighbouring values in the two halves of a register.  A row's code c
// (0..15) stands for scale * (16 + c) + offset: 16 + c is a bf16 or fp16 number of whose mantissa the code is four bits, so
// value codes become numbers by masking them into the pattern of 16, without a conversion.  Key codes mostly go to the
// tensor cores as bytes: c is c 2^-9 in e4m3.
//
// Keys are stored by row and values by channel because that is how the two products of attention consume them with
// 128 keys (S^T = K Q^T) or 128 channels (O^T = V^T P^T) on the rows of the tensor-core operand; in both, the 16-byte
// pieces that neighbouring threads need lie next to each other.
#pragma once

#include <cuda_bf16.h>

#include "common.cuh"

namespace mcsd {

constexpr int kPageRows = 32;
__host__ __device__ constexpr int kv4_page_bytes(int D) { return 32 * D + 256; }
__host__ __device__ constexpr int kv4_values_at(int D) { return 16 * D; }
__host__ __device__ constexpr int kv4_scales_at(int D) { return 32 * D; }

// bit position of value e (0..7) inside its 32-bit word
__host__ __device__ constexpr int kv4_bit(int e) { return 4 * (e >> 1) + 16 * (e & 1); }

__device__ __forceinline__ float bf16_bits_to_f32(uint32_t bits) { return __uint_as_float(bits << 16); }

// scale * (16 + code) + offset: the product has at most 13 significant bits, so the fused form rounds once
__device__ __forceinline__ float kv4_value(uint32_t code, float scale, float offset) {
    return fmaf(scale, (float)(16u + code), offset);
}

}  // namespace mcsd
