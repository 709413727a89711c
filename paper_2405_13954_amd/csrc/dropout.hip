// out = residual + drop(x): dropout with the mask of counter_rng.h, drawn where
// it is used and never stored.  The backward pass is the same call on the
// gradient.
//
// One thread takes eight-column chunks (16 bytes of bf16, 32 of fp32), each one
// draw of the generator.  The chunks of all rows are one list, cut into
// workgroups of kIter x 256; a thread's loads are all issued before its first
// draw.  Bound by memory: x (and the residual) read once, out written once
// (16,384 x 4096 bf16 with a residual: 69 us, 5.9 TB/s).
#include <cmath>

#include "counter_rng.h"
#include "internal.h"

namespace logra {
namespace {

constexpr int kIter = 4;   // chunks per thread

template <bool BF16>
struct Chunk {
    u32x4 v[BF16 ? 1 : 2];
};

template <bool BF16>
__device__ __forceinline__ Chunk<BF16> load_chunk(const char *p, int n) {
    Chunk<BF16> c;
    if (n >= 8) {
        c.v[0] = ld128_nt(p);
        if constexpr (!BF16) c.v[1] = ld128_nt(p + 16);
        return c;
    }
    uint32_t w[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < n) {
            if constexpr (BF16)
                w[i >> 1] |= static_cast<uint32_t>(reinterpret_cast<const uint16_t *>(p)[i]) << (16 * (i & 1));
            else
                w[i] = reinterpret_cast<const uint32_t *>(p)[i];
        }
#pragma unroll
    for (int j = 0; j < (BF16 ? 4 : 8); ++j) c.v[j >> 2][j & 3] = w[j];
    return c;
}

template <bool BF16>
__device__ __forceinline__ void store_chunk(char *p, const Chunk<BF16> &c, int n) {
    if (n >= 8) {
        __builtin_nontemporal_store(c.v[0], reinterpret_cast<u32x4 *>(p));
        if constexpr (!BF16) __builtin_nontemporal_store(c.v[1], reinterpret_cast<u32x4 *>(p + 16));
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < n) {
            if constexpr (BF16)
                reinterpret_cast<uint16_t *>(p)[i] = static_cast<uint16_t>(c.v[0][i >> 1] >> (16 * (i & 1)));
            else
                reinterpret_cast<uint32_t *>(p)[i] = c.v[i >> 2][i & 3];
        }
}

// x, residual, out may be the same memory: a thread reads its elements before
// it writes them, and no other thread touches them.
template <bool BF16, bool RES>
__global__ __launch_bounds__(256) void k_dropout(const char *x, int64_t ld_x, const char *res, int64_t ld_r, char *out,
                                                 int64_t ld_o, int64_t rows, int cols, uint32_t chunks, uint32_t inv,
                                                 DropArgs d) {
    constexpr int kEs = BF16 ? 2 : 4;
    // the workgroup's first chunk as (row, chunk); within it, chunk numbers fit 32 bits
    const uint64_t first = (blockIdx.x + static_cast<uint64_t>(gridDim.x) * blockIdx.y) * (256 * kIter);
    const int64_t row0 = static_cast<int64_t>(first / chunks);
    const uint32_t c0 = static_cast<uint32_t>(first % chunks);
    int64_t row[kIter];
    uint32_t ch[kIter];
    int n[kIter];
    Chunk<BF16> v[kIter], r[kIter];
#pragma unroll
    for (int i = 0; i < kIter; ++i) {
        const uint32_t at = c0 + threadIdx.x + 256u * i;
        uint32_t q = __umulhi(at, inv);            // floor(at / chunks) or one less
        uint32_t c = at - q * chunks;
        if (c >= chunks) {
            c -= chunks;
            ++q;
        }
        row[i] = row0 + q;
        ch[i] = c;
        n[i] = row[i] < rows ? cols - static_cast<int>(8 * c) : 0;
        if (n[i] > 0) {
            v[i] = load_chunk<BF16>(x + (row[i] * ld_x + 8 * static_cast<int64_t>(c)) * kEs, n[i]);
            if constexpr (RES) r[i] = load_chunk<BF16>(res + (row[i] * ld_r + 8 * static_cast<int64_t>(c)) * kEs, n[i]);
        }
    }
#pragma unroll
    for (int i = 0; i < kIter; ++i) {
        if (n[i] <= 0) continue;
        u32x4 w = {0, 0, 0, 0};
        if (d.thr) w = drop_bits(d, static_cast<uint32_t>(row[i]), ch[i]);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const bool keep = ((w[e >> 1] >> (16 * (e & 1))) & 0xFFFFu) >= d.thr;
            float a, b = 0.f;
            if constexpr (BF16) {
                a = bf16_to_f32(static_cast<bf16_bits>(v[i].v[0][e >> 1] >> (16 * (e & 1))));
                if constexpr (RES) b = bf16_to_f32(static_cast<bf16_bits>(r[i].v[0][e >> 1] >> (16 * (e & 1))));
            } else {
                a = __uint_as_float(v[i].v[e >> 2][e & 3]);
                if constexpr (RES) b = __uint_as_float(r[i].v[e >> 2][e & 3]);
            }
            a = keep ? a * d.scale : 0.f;
            if constexpr (RES) a += b;
            if constexpr (BF16) {
                const uint32_t h = f32_to_bf16_rne(a);
                const uint32_t old = v[i].v[0][e >> 1];
                v[i].v[0][e >> 1] = (e & 1) ? ((old & 0xFFFFu) | (h << 16)) : ((old & 0xFFFF0000u) | h);
            } else {
                v[i].v[e >> 2][e & 3] = __float_as_uint(a);
            }
        }
        store_chunk<BF16>(out + (row[i] * ld_o + 8 * static_cast<int64_t>(ch[i])) * kEs, v[i], n[i]);
    }
}

}  // namespace

DropArgs drop_args(double p, uint64_t seed, uint64_t offset) {
    DropArgs d;
    d.thr = static_cast<uint32_t>(std::nearbyint(p * 65536.0));
    d.scale = 65536.f / static_cast<float>(65536u - d.thr);
    d.key[0] = static_cast<uint32_t>(seed);
    d.key[1] = static_cast<uint32_t>(seed >> 32);
    d.off[0] = static_cast<uint32_t>(offset);
    d.off[1] = static_cast<uint32_t>(offset >> 32);
    return d;
}

hipError_t launch_dropout(const void *x, int64_t ld_x, bool bf16, int64_t rows, int cols, const void *res,
                          int64_t ld_r, void *out, int64_t ld_o, double p, uint64_t seed, uint64_t offset,
                          hipStream_t s) {
    const DropArgs d = drop_args(p, seed, offset);
    const uint32_t chunks = (static_cast<uint32_t>(cols) + 7) / 8;
    const uint64_t groups = (static_cast<uint64_t>(rows) * chunks + 256 * kIter - 1) / (256 * kIter);
    // x spans at most 2^23 workgroups (2^31 threads), y the rest
    const uint32_t gx = static_cast<uint32_t>(groups < (1u << 23) ? groups : (1u << 23));
    const dim3 grid(gx, static_cast<uint32_t>((groups + gx - 1) / gx));
    const uint32_t inv = chunks == 1 ? 0xFFFFFFFFu : static_cast<uint32_t>((uint64_t{1} << 32) / chunks);
    const auto go = [&](auto kernel) {
        kernel<<<grid, 256, 0, s>>>(static_cast<const char *>(x), ld_x, static_cast<const char *>(res), ld_r,
                                    static_cast<char *>(out), ld_o, rows, cols, chunks, inv, d);
    };
    if (bf16)
        res ? go(k_dropout<true, true>) : go(k_dropout<true, false>);
    else
        res ? go(k_dropout<false, true>) : go(k_dropout<false, false>);
    return hipGetLastError();
}

}  // namespace logra
