// Rows of bf16 or fp32 in 16-byte vectors, and what the row-wise kernels (token and preference loss, layer norm) do with
// them: partial vectors at a row's end, sums and maxima over a workgroup, exponentials.
#pragma once
#include "common.h"

namespace logra {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
constexpr float kLog2e = 1.4426950408889634f;

// exp(z - top); a row without a finite logit uses top = 0 and gets zeros
__device__ __forceinline__ float exp_from(float z, float top) {
    return __builtin_amdgcn_exp2f((z - top) * kLog2e);
}

template <bool BF16>
struct Vec {
    static constexpr int kN = BF16 ? 8 : 4;   // elements in 16 bytes
    __device__ static float get(u32x4 v, int e) {
        if constexpr (BF16) return __uint_as_float((e & 1) ? (v[e >> 1] & 0xFFFF0000u) : (v[e >> 1] << 16));
        return __uint_as_float(v[e]);
    }
    __device__ static u32x4 none() {   // -inf in every slot
        u32x4 v;
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = BF16 ? 0xFF80FF80u : 0xFF800000u;
        return v;
    }
    // the n < kN elements at p, v's in the other slots
    __device__ static u32x4 load(const char *p, int n, u32x4 v = none()) {
#pragma unroll
        for (int e = 0; e < kN; ++e)
            if (e < n) {
                if constexpr (BF16) {
                    const uint32_t h = reinterpret_cast<const uint16_t *>(p)[e];
                    v[e >> 1] = (e & 1) ? ((v[e >> 1] & 0xFFFFu) | (h << 16)) : ((v[e >> 1] & 0xFFFF0000u) | h);
                } else {
                    v[e] = reinterpret_cast<const uint32_t *>(p)[e];
                }
            }
        return v;
    }
    // to nearest, ties to even
    __device__ static u32x4 pack(const float *g) {
        u32x4 v;
        if constexpr (BF16) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                v[j] = __builtin_bit_cast(uint32_t,
                                          bf16x2{static_cast<__bf16>(g[2 * j]), static_cast<__bf16>(g[2 * j + 1])});
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = __float_as_uint(g[j]);
        }
        return v;
    }
    __device__ static void store(char *p, const float *g, int n) { put(p, pack(g), n); }
    // the first n elements of v
    __device__ static void put(char *p, u32x4 v, int n) {
        if (n >= kN) {
            __builtin_nontemporal_store(v, reinterpret_cast<u32x4 *>(p));
            return;
        }
#pragma unroll
        for (int e = 0; e < kN; ++e)
            if (e < n) {
                if constexpr (BF16)
                    reinterpret_cast<uint16_t *>(p)[e] = static_cast<uint16_t>(v[e >> 1] >> (16 * (e & 1)));
                else
                    reinterpret_cast<uint32_t *>(p)[e] = v[e];
            }
    }
};

// Maximum (MAX) or sum of v over the workgroup, the same in every thread, in a
// fixed order.  red: TH / 64 floats; the caller's later use of red is ordered
// by the second barrier.
template <int TH, bool MAX>
__device__ __forceinline__ float group_reduce(float v, float *red) {
#pragma unroll
    for (int m = 32; m; m >>= 1) {
        const float o = __shfl_xor(v, m);
        v = MAX ? fmaxf(v, o) : v + o;
    }
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = red[0];
#pragma unroll
    for (int w = 1; w < TH / 64; ++w) v = MAX ? fmaxf(v, red[w]) : v + red[w];
    __syncthreads();
    return v;
}

}  // namespace logra
