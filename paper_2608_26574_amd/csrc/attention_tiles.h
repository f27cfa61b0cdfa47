// Images of 64-key K and V^T tiles in LDS and the words that say which block
// keys a row sees, shared by the bf16 attention kernels.
#pragma once

#include "common.h"

namespace dard {

constexpr int kKeys = 64;      // keys per tile

// Eight E4M3 codes (two dwords) -> eight bf16 values, two an instruction (exact:
// at most 4 significant bits, scale 1; a NaN code gives NaN).
__device__ __forceinline__ uint4 e4m3x8_to_bf16x8_scaled(uint32_t lo, uint32_t hi) {
    return make_uint4(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, false)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, true)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, false)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, true)));
}

// 16-byte chunk slots.  The LDS serves a 16-byte read 16 consecutive lanes
// per cycle over 64 banks (256 bytes; measured: an image that separates only
// groups of 8 lanes within 128 bytes kept its conflicts), and each group must
// hit 16 different 4-bank groups; the swizzles below also keep every 8 lanes
// within 128 bytes apart.  With x ^ (x >> 3) a value x in [0, 16) and its
// neighbour x ^ 8 differ in their low three bits.
//   K row r keeps its chunk c (dims 8c..8c+7) in slot c ^ kswz(r): with
//   x = pi(r) % 16, pi swapping bits 2 and 3, kswz = x for DH = 128 (a row
//   is 256 bytes) and (x ^ (x >> 3)) % 8 for DH = 64.  The S^T operand read
//   of lane l takes key row pi(l % 32), so x is l % 16.
//   V^T row d (a dim, 128 bytes) keeps its chunk c (keys 8c..8c+7) in slot
//   c ^ vswz(d), vswz(d) = (d ^ (d >> 3)) % 8; the V^T read of lane l takes
//   row 32j + l % 32.
__device__ __forceinline__ int swap23(int r) { return (r & ~12) | ((r & 4) << 1) | ((r & 8) >> 1); }
template <int DH>
__device__ __forceinline__ int kswz(int r) {
    const int x = swap23(r) & 15;   // rows 32 apart share their swizzle
    return DH == 128 ? x : ((x ^ (x >> 3)) & (DH / 8 - 1));
}
template <int DH>
__device__ __forceinline__ int kslot(int r, int c) { return r * (DH / 8) + (c ^ kswz<DH>(r)); }
__device__ __forceinline__ int vswz(int d) { return (d ^ (d >> 3)) & 7; }
__device__ __forceinline__ int vslot(int d, int c) { return d * (kKeys / 8) + (c ^ vswz(d)); }

// The 2B-bit block visibility of a row, x^j for the set bits j of its take-x
// value X (B <= 256 bits, zero above B), s^j for the clear ones: bits [0, B)
// are X, bits [B, 2B) are NOT X.  block_word gives bits [64 bt, 64 bt + 64),
// the word of block tile bt.
__device__ __forceinline__ uint64_t word_at(const uint64_t (&x)[kBlockWords], int q) {
    uint64_t w = 0ull;
#pragma unroll
    for (int k = 0; k < kBlockWords; ++k) w = q == k ? x[k] : w;
    return w;
}
// Bits [start, start + 64) of X (start may be negative), zero outside [0, B).
__device__ __forceinline__ uint64_t bits64(const uint64_t (&x)[kBlockWords], int B, int start) {
    if (start >= B || start <= -64) return 0ull;
    uint64_t v;
    if (start < 0) {
        v = word_at(x, 0) << (-start);
    } else {
        const int q = start >> 6, sh = start & 63;
        v = word_at(x, q) >> sh;
        if (sh) v |= word_at(x, q + 1) << (64 - sh);
    }
    const int n = B - start;
    return n < 64 ? v & ((1ull << n) - 1) : v;
}
// Bits j of a word with 0 <= start + j < B.
__device__ __forceinline__ uint64_t range_mask(int start, int B) {
    const int lo = start < 0 ? -start : 0;
    const int hi = B - start < 64 ? B - start : 64;
    if (hi <= lo) return 0ull;
    const uint64_t up = hi >= 64 ? ~0ull : (1ull << hi) - 1;
    const uint64_t low = lo >= 64 ? ~0ull : (1ull << lo) - 1;
    return up & ~low;
}
__device__ __forceinline__ uint64_t block_word(const uint64_t (&x)[kBlockWords], int B, int bt) {
    const int s0 = 64 * bt;
    return bits64(x, B, s0) | (~bits64(x, B, s0 - B) & range_mask(s0 - B, B));
}

}  // namespace dard
