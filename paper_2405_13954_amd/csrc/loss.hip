// Cross-entropy of every token's logits and its gradient:
//
//     loss_t = w_t (lse(z_t) - z_t[target_t]),   dz_t = w_t (softmax(z_t) - onehot(target_t))
//
// One workgroup per token.  The token's logits are read once and stay packed in
// registers (NV 16-byte vectors a thread) through the three passes over them:
// the maximum, the sum of exp(z - max), and the gradient, so memory sees one
// read and one write of the vocabulary, which is what bounds it.  Vocabularies
// beyond the registers of 1024 threads are read a second time for the gradient,
// maximum and sum being kept as a running pair in the first pass.
// Maximum, sum and gradient are fp32; z - max is formed before the product with
// log2(e), so that the likely tokens keep their full precision.
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
                v[j] = __builtin_bit_cast(uint32_t, bf16x2{static_cast<__bf16>(g[2 * j]), static_cast<__bf16>(g[2 * j + 1])});
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

// NV = 0: the vocabulary does not stay in registers.
template <bool BF16, int TH, int NV>
__global__ __launch_bounds__(TH) void k_token_loss(const char *logits, int64_t ld, int64_t rows, int vocab,
                                                   const int64_t *target, const float *weight, float *loss,
                                                   char *dlogits, int64_t ld_d) {
    using V = Vec<BF16>;
    constexpr int kEs = BF16 ? 2 : 4;
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
    const char *zk = z + static_cast<int64_t>(tid) * 16;
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
    const auto gradient = [&](u32x4 v, int i, float m, float f, float hot) {
        float g[V::kN];
        const int hit = static_cast<int>(t) - i * V::kN;
#pragma unroll
        for (int e = 0; e < V::kN; ++e) {
            g[e] = exp_from(V::get(v, e), m) * f;
            if (e == hit) g[e] -= hot;
        }
        V::store(dz + static_cast<int64_t>(i) * 16, g, vocab - i * V::kN);
    };
    u32x4 last = V::none();
    if (tail) last = V::load(z + static_cast<int64_t>(n_full) * 16, odd);
    float top = maximum(last, kNone), total = 0.f;
    if constexpr (NV > 0) {
        u32x4 v[NV];
        // between the passes: the packed logits are what is kept, not their fp32 values or exponentials, which
        // the compiler would otherwise carry over at two registers for each one
        const auto again = [&](u32x4 (&x)[NV]) {
            asm volatile("" : "+v"(top));
            if constexpr (BF16) {
#pragma unroll
                for (int k = 0; k < NV; ++k) asm volatile("" : "+v"(x[k]));
            }
        };
#pragma unroll
        for (int k = 0; k < NV; ++k) v[k] = k * TH + tid < n_full ? ld128_nt(zk + static_cast<int64_t>(k) * TH * 16) : V::none();
#pragma unroll
        for (int k = 0; k < NV; ++k) top = maximum(v[k], top);
        top = group_reduce<TH, true>(top, red);
        if (top == kNone) top = 0.f;
        again(v);
#pragma unroll
        for (int k = 0; k < NV; ++k) total += sum(v[k], top);
        total = group_reduce<TH, false>(total + sum(last, top), red);
        if (tid == 0) loss[row] = row_loss(top, total, w, zt);
        if (!dz) return;
        const float f = total == 0.f ? 0.f : w / total, hot = total == 0.f ? 0.f : w;
        again(v);
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (k * TH + tid < n_full) gradient(v[k], k * TH + tid, top, f, hot);
        if (tail) gradient(last, n_full, top, f, hot);
    } else {
        // each thread keeps the running maximum and sum of its own vectors
        float mine = top;
        total = mine == kNone ? 0.f : sum(last, mine);
        for (int i = tid; i < n_full; i += TH) {
            const u32x4 v = ld128(z + static_cast<int64_t>(i) * 16);
            const float m = maximum(v, mine), base = m == kNone ? 0.f : m;
            total = total * exp_from(mine, base) + sum(v, base);
            mine = m;
        }
        top = group_reduce<TH, true>(mine, red);
        if (top == kNone) top = 0.f;
        total = group_reduce<TH, false>(total * exp_from(mine, top), red);
        if (tid == 0) loss[row] = row_loss(top, total, w, zt);
        if (!dz) return;
        const float f = total == 0.f ? 0.f : w / total, hot = total == 0.f ? 0.f : w;
        for (int i = tid; i < n_full; i += TH) gradient(ld128(z + static_cast<int64_t>(i) * 16), i, top, f, hot);
        if (tail) gradient(last, n_full, top, f, hot);
    }
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
        if (vec <= 256 * 4) go(k_token_loss<B, 256, 4>, 256);
        else if (vec <= 256 * 8) go(k_token_loss<B, 256, 8>, 256);
        else if (vec <= 512 * 8) go(k_token_loss<B, 512, 8>, 512);
        else if (vec <= 1024 * 8) go(k_token_loss<B, 1024, 8>, 1024);
        else if (vec <= 1024 * 16) go(k_token_loss<B, 1024, 16>, 1024);
        else go(k_token_loss<B, 1024, 0>, 1024);
    };
    if (bf16)
        pick(std::true_type{});
    else
        pick(std::false_type{});
    return hipGetLastError();
}

}  // namespace logra
