// One AdamW step of many tensors, of many models at once:
//
//   c = min(1, max_norm / |g|)             for each group of slices (one model), over all its slices
//   m = b1 m + (1 - b1) c g,   v = b2 v + (1 - b2) (c g)^2
//   p = p (1 - lr decay) - lr (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps),   work = bf16(p)
//
// The plan lists the tensors as chunks of 2,048 elements, each with its pointers, so that a step is one launch over all
// tensors whatever their number and sizes (k_adamw_step: one workgroup a chunk, eight elements a thread), behind a launch
// that squares and adds the gradients (k_adamw_norm: a wave for each chunk) and a small one that turns the sums into each
// group's factors (k_adamw_head).  Bound by memory: 28 bytes an element with fp32 states, 16 with 8-bit ones, 2 more for
// the bf16 copy, and 4 to read the gradient twice where it is clipped.
//
// 8-bit states: blocks of 256 elements share a power-of-two scale, the smallest that brings the block's largest magnitude
// to 1.75 times the largest power of two of the type or below.  m is e4m3.  v is e5m2: gradients of outlying columns are a
// thousand times the others', and their squares need the wider exponent more than the third bit.  Both are rounded at
// random, up with the probability of the part that is cut off: to nearest, a v whose step adds less than half of its last
// bit (an eighth) would never move again.  A v that is not zero keeps at least the smallest code, so that no element divides
// by eps alone.  One last bit of m or v can tip a code, so this path is float64 up to the code; it is still bound by memory.
#include "counter_rng.h"
#include "internal.h"
#include "vec16.h"

namespace logra {
namespace {

constexpr int kTh = 256, kPer = 8;             // elements of a thread
static_assert(kAdamwChunk == kTh * kPer, "a workgroup takes one chunk");
static_assert(kAdamwBlock == 32 * kPer, "a block of the 8-bit states is half a wave's");

// Under-aligned vectors: tensors may be slices of flat buffers, so only the elements themselves are aligned.
typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x4h __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x2b __attribute__((ext_vector_type(2), aligned(1)));

__device__ __forceinline__ void load8(const float *p, int n, float (&x)[kPer]) {
    if (n >= kPer) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const f32x4u v = *reinterpret_cast<const f32x4u *>(p + 4 * k);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[4 * k + e] = v[e];
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < kPer; ++e) x[e] = e < n ? p[e] : 0.f;
}

__device__ __forceinline__ void store8(float *p, int n, const float (&x)[kPer]) {
    if (n >= kPer) {
#pragma unroll
        for (int k = 0; k < 2; ++k)
            *reinterpret_cast<f32x4u *>(p + 4 * k) = f32x4u{x[4 * k], x[4 * k + 1], x[4 * k + 2], x[4 * k + 3]};
        return;
    }
#pragma unroll
    for (int e = 0; e < kPer; ++e)
        if (e < n) p[e] = x[e];
}

__device__ __forceinline__ u32x2b load8(const uint8_t *p, int n) {
    if (n >= kPer) return *reinterpret_cast<const u32x2b *>(p);
    u32x2b v = {0, 0};
#pragma unroll
    for (int e = 0; e < kPer; ++e)
        if (e < n) v[e >> 2] |= static_cast<uint32_t>(p[e]) << (8 * (e & 3));
    return v;
}

__device__ __forceinline__ void store8(uint8_t *p, int n, u32x2b v) {
    if (n >= kPer) {
        *reinterpret_cast<u32x2b *>(p) = v;
        return;
    }
#pragma unroll
    for (int e = 0; e < kPer; ++e)
        if (e < n) p[e] = static_cast<uint8_t>(v[e >> 2] >> (8 * (e & 3)));
}

// What the kernels find at fixed places of the plan's memory, whatever it holds; `room` chunks lie within it.
struct PlanArgs {
    AdamwHeader *header;
    size_t bytes;
    int groups;
    uint32_t room;
    AdamwGroup *group;
    const uint32_t *starts;
    const AdamwChunk *chunks;
};

__device__ __forceinline__ bool is_plan(const PlanArgs &a) {
    const AdamwHeader *h = a.header;
    return h->magic == kAdamwMagic && h->bytes <= a.bytes && h->groups == a.groups && h->chunks <= a.room;
}
__device__ __forceinline__ double *parts_of(const PlanArgs &a) {
    return reinterpret_cast<double *>(reinterpret_cast<char *>(a.header) + adamw_parts_at(a.groups, a.header->chunks));
}

// A wave for each chunk: the sum of its squared gradients in float64, at the chunk's place among its group's.
__global__ __launch_bounds__(kTh) void k_adamw_norm(PlanArgs a) {
    const int lane = static_cast<int>(threadIdx.x & 63);
    const uint32_t c = blockIdx.x * (kTh / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (c >= a.room) return;
    const float *grad = a.chunks[c].grad;   // loaded beside the header; used if this is a plan
    const int count = a.chunks[c].count;
    const uint32_t slot = a.chunks[c].slot;
    if (!is_plan(a) || c >= a.header->chunks) return;
    float g[kAdamwChunk / 64 / 4][4];
#pragma unroll
    for (int i = 0; i < kAdamwChunk / 64 / 4; ++i) {
        const int at = (i * 64 + lane) * 4, n = count - at;
        if (n >= 4) {
            const f32x4u v = *reinterpret_cast<const f32x4u *>(grad + at);
#pragma unroll
            for (int e = 0; e < 4; ++e) g[i][e] = v[e];
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) g[i][e] = e < n ? grad[at + e] : 0.f;
        }
    }
    double s = 0.0;
#pragma unroll
    for (int i = 0; i < kAdamwChunk / 64 / 4; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) s = fma(static_cast<double>(g[i][e]), static_cast<double>(g[i][e]), s);
#pragma unroll
    for (int m = 32; m; m >>= 1) s += __shfl_xor(s, m);
    if (lane == 0) parts_of(a)[slot] = s;
}

// A workgroup for each group: its norm, and what its elements are multiplied by.
__global__ __launch_bounds__(kTh) void k_adamw_head(PlanArgs a, const int64_t *step, AdamwHyper y, bool with_norm,
                                                    const float *lr_scale, float *norms) {
    if (!is_plan(a)) return;
    __shared__ double red[kTh / 64];
    const int group = static_cast<int>(blockIdx.x);
    double clip = 1.0;
    bool skip = false;
    if (with_norm) {
        const uint32_t begin = a.starts[group], end = a.starts[group + 1];
        const double *parts = parts_of(a);
        double s = 0.0;
        for (uint32_t i = begin + threadIdx.x; i < end; i += kTh) s += parts[i];
#pragma unroll
        for (int m = 32; m; m >>= 1) s += __shfl_xor(s, m);
        if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
        __syncthreads();
        const double norm = sqrt(((red[0] + red[1]) + red[2]) + red[3]);
        if (norms && threadIdx.x == 0) norms[group] = static_cast<float>(norm);
        skip = !(norm < __builtin_inf());
        if (y.max_norm > 0.0 && norm > y.max_norm) clip = y.max_norm / norm;
    }
    if (threadIdx.x) return;
    const double t = static_cast<double>(*step + 1);
    const double fix1 = 1.0 - pow(y.beta1, t), fix2 = 1.0 - pow(y.beta2, t);
    // lr lr_scale is one rounding, as a caller's own product of the two would be
    const double lr = static_cast<double>(lr_scale ? static_cast<float>(y.lr) * lr_scale[group] : static_cast<float>(y.lr));
    AdamwGroup &o = a.group[group];
    o.clip = clip;
    o.lr = static_cast<float>(lr);
    o.rate = static_cast<float>(lr / fix1);
    o.root = static_cast<float>(1.0 / sqrt(fix2));
    o.skip = skip;
    o.step = *step + 1;
}

// param after its move.  The hardware's root and reciprocal are within one last bit, and what they make is a correction of
// param; the root of small numbers is taken of a larger one, since the hardware's flushes subnormal ones.
__device__ __forceinline__ float moved(float p, float m, float v, const AdamwGroup &g, float keep, float eps) {
    const bool small = v < 0x1p-96f;
    const float root = __builtin_amdgcn_sqrtf(small ? v * 0x1p64f : v) * (small ? 0x1p-32f : 1.f);
    return fmaf(p, keep, -g.rate * m * __builtin_amdgcn_rcpf(fmaf(root, g.root, eps)));
}

constexpr double kFloatMax = 3.4028234663852886e38;

// |x| as an ordered key: the high word of the double, its last bit set where the low word holds anything, so that 1.75 times
// a power of two and what is above it differ.
__device__ __forceinline__ uint32_t key_of(double x) {
    const uint64_t u = __builtin_bit_cast(uint64_t, x);
    return (static_cast<uint32_t>(u >> 32) & 0x7FFFFFFFu) | (static_cast<uint32_t>(u) != 0 ? 1u : 0u);
}

// The exponent of the block's scale, from the largest key: the scale brings it to 1.75 * 2^HIGH or below.
template <int HIGH>
__device__ __forceinline__ int scale_of(uint32_t key) {
    if (key < 0x00100000u) return 0;   // only zeros (a double that fp32 numbers give is not subnormal)
    const int k = static_cast<int>(key >> 20) - 1023 - HIGH + ((key & 0xFFFFFu) > 0xC0000u ? 1 : 0);
    return k < -126 ? -126 : k;
}

// |x| 2^-k in steps of a float of BITS mantissa bits and exponents from LOW on, rounded up where the part cut off exceeds
// draw / 65536 of a step; as its code.  LEAST: the smallest code of what is not zero.  The leading 21 bits of x, one more
// where there are others, give the number of 65536ths of a step, rounded up.
template <int BITS, int LOW, uint32_t LEAST>
__device__ __forceinline__ uint32_t code_of(double x, int k, uint32_t draw) {
    const uint64_t u = __builtin_bit_cast(uint64_t, x);
    const uint32_t high = static_cast<uint32_t>(u >> 32) & 0x7FFFFFFFu;
    const int e = static_cast<int>(high >> 20) - 1023 - k, under = LOW - e;   // under > 0: below the smallest exponent
    int drop = 4 - BITS + (under > 0 ? under : 0);
    drop = drop < 31 ? drop : 31;
    const uint32_t lead = ((high & 0xFFFFFu) | 0x100000u) + (static_cast<uint32_t>(u) != 0 ? 1u : 0u);
    const uint32_t fixed = (lead + ((1u << drop) - 1u)) >> drop;
    uint32_t n = (fixed + 65535u - draw) >> 16;
    if (LEAST) n = n < LEAST ? LEAST : n;
    n += static_cast<uint32_t>(under > 0 ? 0 : -under) << BITS;
    return high < 0x00100000u ? 0u : n;
}

__device__ __forceinline__ uint32_t half_wave_max(uint32_t v) {
#pragma unroll
    for (int m = 16; m; m >>= 1) {
        const uint32_t o = static_cast<uint32_t>(__shfl_xor(static_cast<int>(v), m));
        v = v > o ? v : o;
    }
    return v;
}

// The largest key of a block's elements that are finite in fp32.
__device__ __forceinline__ uint32_t top_key(const double (&x)[kPer], int n) {
    double top = 0.0;
#pragma unroll
    for (int e = 0; e < kPer; ++e) top = fmax(top, e < n ? fabs(x[e]) : 0.0);   // (the maximum of a NaN and a number is the number)
    if (__builtin_expect(top > kFloatMax, 0)) {
        top = 0.0;
#pragma unroll
        for (int e = 0; e < kPer; ++e) top = fmax(top, e < n && fabs(x[e]) <= kFloatMax ? fabs(x[e]) : 0.0);
    }
    return half_wave_max(key_of(top));
}

__global__ __launch_bounds__(kTh) void k_adamw_step(PlanArgs a, int64_t *step, AdamwHyper y) {
    const AdamwChunk k = a.chunks[blockIdx.x];   // loaded beside the header; used if this is a plan
    if (!is_plan(a)) return;
    // k_adamw_head has read the step, and no workgroup of this launch does
    if (blockIdx.x == 0 && threadIdx.x == 0) *step = a.group->step;
    if (blockIdx.x >= a.header->chunks) return;
    const int at = static_cast<int>(threadIdx.x) * kPer, n = k.count - at;
    float p[kPer], g[kPer];
    load8(k.grad + at, n, g);
    load8(k.param + at, n, p);
    const AdamwGroup o = a.group[k.group];
    const float keep = k.decay ? static_cast<float>(1.0 - static_cast<double>(o.lr) * y.decay) : 1.f;
    const float eps = static_cast<float>(y.eps);
    if (!k.m_scale) {
        float m[kPer], v[kPer];
        load8(static_cast<const float *>(k.m) + at, n, m);
        load8(static_cast<const float *>(k.v) + at, n, v);
        if (o.skip) return;   // a model whose gradient is not finite stays as it is
        const float clip = static_cast<float>(o.clip), b1 = static_cast<float>(y.beta1), b2 = static_cast<float>(y.beta2);
        const float a1 = static_cast<float>(1.0 - y.beta1), a2 = static_cast<float>(1.0 - y.beta2);
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            const float cg = clip * g[e];
            m[e] = fmaf(a1, cg, b1 * m[e]);
            v[e] = fmaf(a2, cg * cg, b2 * v[e]);
            p[e] = moved(p[e], m[e], v[e], o, keep, eps);
        }
        store8(static_cast<float *>(k.m) + at, n, m);
        store8(static_cast<float *>(k.v) + at, n, v);
    } else {
        const int block = at / kAdamwBlock;   // half a wave has it
        const uint32_t i = k.first + static_cast<uint32_t>(at);
        const u32x2b cm = load8(static_cast<const uint8_t *>(k.m) + at, n);
        const u32x2b cv = load8(static_cast<const uint8_t *>(k.v) + at, n);
        const float sm = n > 0 ? k.m_scale[block] : 0.f, sv = n > 0 ? k.v_scale[block] : 0.f;
        if (o.skip) return;
        const double b1 = y.beta1 * sm, b2 = y.beta2 * sv, a1 = (1.0 - y.beta1) * o.clip, a2 = (1.0 - y.beta2) * (o.clip * o.clip);
        double m[kPer], v[kPer];
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            const int w = static_cast<int>(cm[e >> 2]), u = static_cast<int>(cv[e >> 2]);
            const float fm = (e & 3) == 0   ? __builtin_amdgcn_cvt_f32_fp8(w, 0)
                             : (e & 3) == 1 ? __builtin_amdgcn_cvt_f32_fp8(w, 1)
                             : (e & 3) == 2 ? __builtin_amdgcn_cvt_f32_fp8(w, 2)
                                            : __builtin_amdgcn_cvt_f32_fp8(w, 3);
            const float fv = (e & 3) == 0   ? __builtin_amdgcn_cvt_f32_bf8(u, 0)
                             : (e & 3) == 1 ? __builtin_amdgcn_cvt_f32_bf8(u, 1)
                             : (e & 3) == 2 ? __builtin_amdgcn_cvt_f32_bf8(u, 2)
                                            : __builtin_amdgcn_cvt_f32_bf8(u, 3);
            const double ge = static_cast<double>(g[e]);
            m[e] = fma(a1, ge, b1 * static_cast<double>(fm));
            v[e] = fma(a2, ge * ge, b2 * static_cast<double>(fv));
            p[e] = moved(p[e], static_cast<float>(m[e]), static_cast<float>(v[e]), o, keep, eps);
        }
        const int scale_m = scale_of<8>(top_key(m, n)), scale_v = scale_of<15>(top_key(v, n));
        u32x2b out_m = {0, 0}, out_v = {0, 0};
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const u32x4 bits = philox(i / 4 + q, k.slice, k.tensor, static_cast<uint32_t>(o.step), y.key[0], y.key[1]);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const double me = m[4 * q + e], ve = v[4 * q + e];
                uint32_t one = code_of<3, -6, 0>(me, scale_m, bits[e] & 0xFFFFu);
                one |= static_cast<uint32_t>(__builtin_bit_cast(uint64_t, me) >> 56) & 0x80u;
                uint32_t two = code_of<2, -14, 1>(ve, scale_v, bits[e] >> 16);
                one = fabs(me) <= kFloatMax ? one : 0x7Fu;                            // NaN (the type has no infinity)
                two = ve <= kFloatMax ? two : ve > 0.0 ? 0x7Cu : 0x7Fu;   // infinity, NaN
                out_m[q] |= one << (8 * e);
                out_v[q] |= two << (8 * e);
            }
        }
        store8(static_cast<uint8_t *>(k.m) + at, n, out_m);
        store8(static_cast<uint8_t *>(k.v) + at, n, out_v);
        if (n > 0 && (threadIdx.x & 31) == 0) {
            k.m_scale[block] = __uint_as_float(static_cast<uint32_t>(scale_m + 127) << 23);
            k.v_scale[block] = __uint_as_float(static_cast<uint32_t>(scale_v + 127) << 23);
        }
    }
    store8(k.param + at, n, p);
    if (k.work) {
        bf16_bits *work = static_cast<bf16_bits *>(k.work) + at;
        const u32x4 v = Vec<true>::pack(p);
        if (n >= kPer) {
            *reinterpret_cast<u32x4h *>(work) = v;
        } else {
#pragma unroll
            for (int e = 0; e < kPer; ++e)
                if (e < n) work[e] = static_cast<bf16_bits>(v[e >> 1] >> (16 * (e & 1)));
        }
    }
}

}  // namespace

hipError_t launch_adamw_step(void *plan, size_t plan_bytes, int groups, int64_t *step, const AdamwHyper &y,
                             const float *lr_scale, float *norms, hipStream_t s) {
    char *base = static_cast<char *>(plan);
    // as many chunks as the plan's memory has room for
    const size_t room = (plan_bytes - adamw_chunks_at(groups)) / (sizeof(AdamwChunk) + sizeof(double));
    const PlanArgs a = {static_cast<AdamwHeader *>(plan), plan_bytes, groups,
                        static_cast<uint32_t>(room > kMaxAdamwChunks ? kMaxAdamwChunks : room),
                        reinterpret_cast<AdamwGroup *>(base + adamw_groups_at()),
                        reinterpret_cast<const uint32_t *>(base + adamw_starts_at(groups)),
                        reinterpret_cast<const AdamwChunk *>(base + adamw_chunks_at(groups))};
    const bool with_norm = norms || y.max_norm > 0.0;
    if (with_norm) k_adamw_norm<<<(a.room + 3) / 4, kTh, 0, s>>>(a);
    k_adamw_head<<<groups, kTh, 0, s>>>(a, step, y, with_norm, lr_scale, norms);
    k_adamw_step<<<a.room, kTh, 0, s>>>(a, step, y);
    return hipGetLastError();
}

}  // namespace logra
