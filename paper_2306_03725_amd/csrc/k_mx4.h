// Microscaled 4-bit numbers: what a code and a block's scale stand for.
//
// The slots of a label come in blocks of 32 with a scale 2^(byte - 127) each (byte 255: not a number); a code is a sign bit (8) and one
// of the magnitudes 0, 0.5, 1, 1.5, 2, 3, 4, 6 (2 bits of exponent, 1 of mantissa).  Eight codes make a word, the lowest slot in its
// lowest bits; a label's words are those of ceil(k / 8), codes behind its last slot are 0.
#pragma once
#include "usl_internal.h"

constexpr int MX4_BLOCK = 32;
__host__ __device__ constexpr int mx4_words(int k) { return (k + 7) / 8; }
__host__ __device__ constexpr int mx4_blocks(int k) { return (k + MX4_BLOCK - 1) / MX4_BLOCK; }

// 2^(byte - 127): the byte is the exponent of a float, but 0 (a denormal number) and 255
__device__ __forceinline__ float mx4_scale(uint32_t byte) {
    return __uint_as_float(byte == 255u ? 0x7FC00000u : byte == 0u ? 0x00400000u : byte << 23);
}
// magnitude bits em (3 of them): 0 and 0.5 are the denormal numbers; else exponent em >> 1 and mantissa em & 1
__device__ __forceinline__ float mx4_code(uint32_t code) {
    const uint32_t em = code & 7u, bits = em < 2u ? (em ? 0x3F000000u : 0u) : ((em >> 1) + 126u) << 23 | (em & 1u) << 22;
    return __uint_as_float(bits | (code & 8u) << 28);
}
// slot t of label j
__device__ __forceinline__ float mx4_value(const uint32_t* __restrict__ codes, const uint8_t* __restrict__ scales, int64_t j, int t, int k) {
    return mx4_code(codes[j * mx4_words(k) + t / 8] >> (4 * (t % 8))) * mx4_scale(scales[j * mx4_blocks(k) + t / MX4_BLOCK]);
}
