// Cross-entropy of every token's logits and its gradient:
//
//     loss_t = w_t (lse(z_t) - z_t[target_t]),   dz_t = w_t (softmax(z_t) - onehot(target_t))
//
// One workgroup per token.  A thread keeps NV of its 16-byte vectors of the
// vocabulary packed in registers; the others go by once for the statistics and
// once more, out of the cache, for the gradient.  So memory sees one read of the
// logits and one write of the gradient, which is what bounds it (2,048 tokens of
// 128,000 bf16 logits, a fifth of them masked: 201 us for 0.94 GB, 4.7 TB/s).
// The statistics are one pass: a running maximum and the sum of exp(z - max),
// brought to a new maximum once per four vectors.  Maximum, sum and gradient are
// fp32; z - max is formed before the product with log2(e), so that the likely
// tokens keep their full precision.
#include "common.h"
#include "internal.h"

namespace logra {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
constexpr float kLog2e = 1.4426950408889634f;

// exp(z - top); a row without a finite logit uses top = 0 and gets zeros
__device__ __forceinline__ float exp_from(float z, float top) {
    return __builtin_amdgcn_exp2f((z - top) * kLog2e);
}

template <bool BF16>
struct Vec {
    static constexpr int kN = BF16 ? 8 : 4;   // logits in 16 bytes
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
    // the n < kN logits at p, -inf in the other slots
    __device__ static u32x4 load(const char *p, int n) {
        u32x4 v = none();
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
    __device__ static void store(char *p, const float *g, int n) {
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

__device__ __forceinline__ float row_loss(float top, float total, float w, float zt) {
    // no finite logit: no distribution, and no token of it has a chance
    return total == 0.f ? __builtin_inff() : w * (logf(total) + (top - zt));
}

// MINW: waves on a SIMD that the registers leave room for.
template <bool BF16, int TH, int NV, int MINW>
__global__ __launch_bounds__(TH, MINW) void k_token_loss(const char *logits, int64_t ld, int64_t rows, int vocab,
                                                   const int64_t *target, const float *weight, float *loss,
                                                   char *dlogits, int64_t ld_d) {
    using V = Vec<BF16>;
    constexpr int kEs = BF16 ? 2 : 4, kGroup = 4;
    constexpr float kNone = -__builtin_inff();
    __shared__ float red[TH / 64];
    const int64_t row = blockIdx.x + static_cast<int64_t>(gridDim.x) * blockIdx.y;
    if (row >= rows) return;
    const int64_t t = target[row];
    const float w = weight ? weight[row] : 1.f;
    const char *z = logits + row * ld * kEs;
    char *dz = dlogits ? dlogits + row * ld_d * kEs : nullptr;
    const int n_vec = (vocab + V::kN - 1) / V::kN;
    const int tid = static_cast<int>(threadIdx.x);
    if (t < 0 || t >= vocab || w == 0.f) {   // a masked token: nothing of it is read
        if (tid == 0) loss[row] = 0.f;
        if (dz) {
            const float zero[V::kN] = {};
            for (int i = tid; i < n_vec; i += TH) V::store(dz + static_cast<int64_t>(i) * 16, zero, vocab - i * V::kN);
        }
        return;
    }
    float zt;
    if constexpr (BF16)
        zt = bf16_to_f32(reinterpret_cast<const bf16_bits *>(z)[t]);
    else
        zt = reinterpret_cast<const float *>(z)[t];
    const int n_full = vocab / V::kN, odd = vocab - n_full * V::kN;   // whole vectors; logits of the last, partial one
    const bool tail = odd > 0 && tid == n_full % TH;                  // the thread that has it
    const auto maximum = [&](u32x4 v, float m) {
#pragma unroll
        for (int e = 0; e < V::kN; ++e) m = fmaxf(m, V::get(v, e));
        return m;
    };
    const auto sum = [&](u32x4 v, float m) {
        float q = 0.f;
#pragma unroll
        for (int e = 0; e < V::kN; ++e) q += exp_from(V::get(v, e), m);
        return q;
    };
    // the packed logits are what is kept between the uses of a vector, not their fp32 values or exponentials, which the
    // compiler would otherwise carry over at two registers for each one
    const auto again = [](u32x4 &v) { asm volatile("" : "+v"(v)); };
    const auto load = [&](int i) { return i < n_full ? ld128(z + static_cast<int64_t>(i) * 16) : V::none(); };
    float top = kNone, total = 0.f;   // of the thread's own vectors, a running pair
    const auto take = [&](u32x4 (&v)[kGroup]) {
        float m = top;
#pragma unroll
        for (int j = 0; j < kGroup; ++j) m = maximum(v[j], m);
        const float base = m == kNone ? 0.f : m;
        total *= exp_from(top, base);
#pragma unroll
        for (int j = 0; j < kGroup; ++j) {
            again(v[j]);
            total += sum(v[j], base);
        }
        top = m;
    };
    u32x4 keep[NV / kGroup][kGroup];
#pragma unroll
    for (int k = 0; k < NV; ++k) keep[k / kGroup][k % kGroup] = load(k * TH + tid);
    u32x4 last = V::none();
    if (tail) last = V::load(z + static_cast<int64_t>(n_full) * 16, odd);
    for (int i = NV * TH + tid; i < n_full; i += kGroup * TH) {
        u32x4 v[kGroup];
#pragma unroll
        for (int j = 0; j < kGroup; ++j) v[j] = load(i + j * TH);
        take(v);
    }
#pragma unroll
    for (int k = 0; k < NV / kGroup; ++k) take(keep[k]);
    {
        u32x4 v[kGroup] = {last, V::none(), V::none(), V::none()};
        if (tail) take(v);
    }
    const float mine = top;
    top = group_reduce<TH, true>(mine, red);
    if (top == kNone) top = 0.f;
    total = group_reduce<TH, false>(total * exp_from(mine, top), red);
    if (tid == 0) loss[row] = row_loss(top, total, w, zt);
    if (!dz) return;
    const float f = total == 0.f ? 0.f : w / total, hot = total == 0.f ? 0.f : w;
    const auto gradient = [&](u32x4 v, int i) {
        float g[V::kN];
#pragma unroll
        for (int e = 0; e < V::kN; ++e) g[e] = exp_from(V::get(v, e), top) * f;
        const int hit = static_cast<int>(t) - i * V::kN;
        if (hit >= 0 && hit < V::kN) {   // one vector of the whole token
#pragma unroll
            for (int e = 0; e < V::kN; ++e) g[e] -= e == hit ? hot : 0.f;
        }
        V::store(dz + static_cast<int64_t>(i) * 16, g, vocab - i * V::kN);
    };
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        again(keep[k / kGroup][k % kGroup]);
        if (k * TH + tid < n_full) gradient(keep[k / kGroup][k % kGroup], k * TH + tid);
    }
    for (int i = NV * TH + tid; i < n_full; i += kGroup * TH) {
        u32x4 v[kGroup];
#pragma unroll
        for (int j = 0; j < kGroup; ++j)
            v[j] = i + j * TH < n_full ? ld128_nt(z + static_cast<int64_t>(i + j * TH) * 16) : V::none();
#pragma unroll
        for (int j = 0; j < kGroup; ++j)
            if (i + j * TH < n_full) gradient(v[j], i + j * TH);
    }
    if (tail) gradient(last, n_full);
}

}  // namespace

hipError_t launch_token_loss(const void *logits, int64_t ld, bool bf16, int64_t rows, int vocab, const int64_t *target,
                             const float *weight, float *loss, void *dlogits, int64_t ld_d, hipStream_t s) {
    const uint32_t gx = static_cast<uint32_t>(rows < (1 << 21) ? rows : (1 << 21));
    const dim3 grid(gx, static_cast<uint32_t>((rows + gx - 1) / gx));
    const auto go = [&](auto kernel, int threads) {
        kernel<<<grid, threads, 0, s>>>(static_cast<const char *>(logits), ld, rows, vocab, target, weight, loss,
                                        static_cast<char *>(dlogits), ld_d);
    };
    const int64_t vec = (static_cast<int64_t>(vocab) + (bf16 ? 7 : 3)) / (bf16 ? 8 : 4);
    const auto pick = [&](auto b) {
        constexpr bool B = decltype(b)::value;
        // More tokens than CUs, of a large vocabulary: two workgroups of 1024 threads on a CU, so that one loads or
        // stores while the other computes; otherwise as much as one workgroup has registers for.  us with 4 and with 12
        // kept vectors: bf16, 2,048 tokens of 50,257 logits 81 and 106, 300 tokens 18.6 and 25; 2,048 tokens of 128,000
        // 201 and 198, 300 tokens 41.2 and 40.5, 256 tokens 29 and 26, 200 tokens of 50,257 12.6 and 14.1; fp32,
        // 61 tokens of 50,001 11.1 and 10.0, 2,048 tokens of 50,257 164 and 157.
        if (vec <= 256 * 4) go(k_token_loss<B, 256, 4, 8>, 256);
        else if (vec <= 512 * 4) go(k_token_loss<B, 512, 4, 8>, 512);
        else if (vec <= 1024 * 4 || rows > 256) go(k_token_loss<B, 1024, 4, 8>, 1024);
        else go(k_token_loss<B, 1024, 12, 4>, 1024);
    };
    if (bf16)
        pick(std::true_type{});
    else
        pick(std::false_type{});
    return hipGetLastError();
}

}  // namespace logra
