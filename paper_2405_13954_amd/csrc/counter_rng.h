// Dropout masks from a counter-based generator: nothing is stored, every
// kernel that needs the mask of an element draws it again.
//
// Element (row, col) of a matrix belongs to the eight-column chunk col / 8;
// Philox4x32 (Salmon et al., SC'11) of the counter (col / 8, row, offset) under
// the key `seed` gives the chunk 128 bits, 16 for each column.  The element is
// kept iff its 16 bits are at least thr = round(65536 p), so with probability
// exactly 1 - thr / 65536, and a kept element is scaled by 65536 / (65536 - thr).
// Seven rounds: the fewest that pass BigCrush in that paper; with ten, the
// adapters' dropped rows would take 1.4 times the integer multiplies, which are
// quarter rate and come close to the memory time.
#pragma once
#include "common.h"

namespace logra {

struct DropArgs {
    uint32_t thr;         // 0: keep everything (and draw nothing)
    float scale;          // 65536 / (65536 - thr)
    uint32_t key[2];      // seed
    uint32_t off[2];      // offset
};

// Philox4x32-7: 128 bits for the counter (x0, x1, x2, x3) under the key (k0, k1).
__device__ __forceinline__ u32x4 philox(uint32_t x0, uint32_t x1, uint32_t x2, uint32_t x3, uint32_t k0, uint32_t k1) {
#pragma unroll
    for (int i = 0; i < 7; ++i) {
        const uint64_t a = static_cast<uint64_t>(x0) * 0xD2511F53u, b = static_cast<uint64_t>(x2) * 0xCD9E8D57u;
        x0 = static_cast<uint32_t>(b >> 32) ^ x1 ^ k0;
        x2 = static_cast<uint32_t>(a >> 32) ^ x3 ^ k1;
        x1 = static_cast<uint32_t>(b);
        x3 = static_cast<uint32_t>(a);
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    u32x4 w;
    w[0] = x0;
    w[1] = x1;
    w[2] = x2;
    w[3] = x3;
    return w;
}

// The 128 bits of chunk (row, chunk): word j holds column 2j in its low half
// and column 2j + 1 in its high half, as a pair of bf16 values is packed.
__device__ __forceinline__ u32x4 drop_bits(const DropArgs &d, uint32_t row, uint32_t chunk) {
    return philox(chunk, row, d.off[0], d.off[1], d.key[0], d.key[1]);
}

// 0xFFFF in each half of w that is kept (half >= thr), 0 in the others.
__device__ __forceinline__ uint32_t keep_mask(uint32_t w, uint32_t thr) {
    typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
    const u16x2 h = __builtin_bit_cast(u16x2, w);
    const uint16_t t = static_cast<uint16_t>(thr);
    const u16x2 below = __builtin_elementwise_sub_sat(u16x2{t, t}, h);   // 0 iff kept
    const u16x2 one = {1, 1};
    return __builtin_bit_cast(uint32_t, static_cast<u16x2>(__builtin_elementwise_min(below, one) - one));
}

// Eight packed bf16 values (columns 8 chunk .. + 7 of `row`) with the dropped
// ones replaced by zeros (a selection: a dropped NaN is a zero); not scaled.
__device__ __forceinline__ u32x4 drop8_bf16(const DropArgs &d, u32x4 v, uint32_t row, uint32_t chunk) {
    const u32x4 w = drop_bits(d, row, chunk);
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] &= keep_mask(w[j], d.thr);
    return v;
}
// Four fp32 values, columns col .. col + 3 (col a multiple of four), likewise.
__device__ __forceinline__ u32x4 drop4_f32(const DropArgs &d, u32x4 v, uint32_t row, uint32_t col) {
    const u32x4 w = drop_bits(d, row, col >> 3);
    const bool high = (col & 4u) != 0;
    const uint32_t a = high ? w[2] : w[0], b = high ? w[3] : w[1];
    v[0] = (a & 0xFFFFu) >= d.thr ? v[0] : 0u;
    v[1] = (a >> 16) >= d.thr ? v[1] : 0u;
    v[2] = (b & 0xFFFFu) >= d.thr ? v[2] : 0u;
    v[3] = (b >> 16) >= d.thr ? v[3] : 0u;
    return v;
}

}  // namespace logra
