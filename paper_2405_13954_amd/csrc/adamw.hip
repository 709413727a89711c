// One AdamW step of many tensors, of many models at once:
//
//   c = min(1, max_norm / |g|)             for each group of slices (one model), over all its slices
//   m = b1 m + (1 - b1) c g,   v = b2 v + (1 - b2) (c g)^2
//   p = p (1 - lr decay) - lr (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps),   work = bf16(p)
//
// The plan lists the tensors as chunks of 2,048 elements, each with its pointers, so that a step is one launch over all
// tensors whatever their number and sizes (k_adamw_step: one workgroup a chunk, eight elements a thread), behind a launch
// that squares and adds the gradients (k_adamw_norm: a wave for each chunk) and, for many chunks, a small one that turns the
// sums into each group's factors (k_adamw_head).  Bound by memory: 28 bytes an element with fp32 states, 16 with 8-bit ones,
// 2 more for the bf16 copy, and 4 to read the gradient twice where it is clipped.  10.5 million elements of 15 tensors with
// the copy and clipping, fp32 states: 8 + 5 + 58 us, the last 5.4 TB/s; 42 million with 8-bit states: 30 + 5 + 130 us, 5.8.
// Parameters and states pass by once a step, non-temporal both ways: a line that a load has brought into the cache and a store
// has changed there is written back under the next launch, which was the next step's sum of squares (14 and 47 us then, with
// 54 and 131 for the step).  The gradients are loaded as usual, and what the sum has read of them may still be there.
// Sums and factors in one launch, by the workgroup that is the last to finish, took 77 us for the 14 + 7: every workgroup's
// release of its sum costs some 50 ns, one after the other.
//
// 8-bit states: blocks of 256 elements share a power-of-two scale, the smallest that brings the block's largest magnitude
// to 1.75 times the largest power of two of the type or below.  m is e4m3.  v is e5m2: gradients of outlying columns are a
// thousand times the others', and their squares need the wider exponent more than the third bit.  Both are rounded at
// random, up with the probability of the part that is cut off: to nearest, a v whose step adds less than half of its last
// bit (an eighth) would never move again.  A v that is not zero keeps at least the smallest code, so that no element divides
// by eps alone.  One last bit of m or v can tip a code, so this path is float64 up to the code, each product and sum rounded by
// itself as the formula is written (with beta = 0.9 and few digits in m and the gradient, sums on the very boundary that the random
// bits set are common: some in a million); it is still bound by memory.
#include "counter_rng.h"
#include "internal.h"
#include "vec16.h"

namespace logra {
namespace {

constexpr int kTh = 256, kPer = 8;             // elements of a thread
static_assert(kAdamwChunk == kTh * kPer, "a workgroup takes one chunk");
static_assert(kAdamwBlock == 32 * kPer, "a block of the 8-bit states is half a wave's");

// Under-aligned vectors: tensors may be slices of flat buffers, so only the elements themselves are aligned.  The pointers
// come out of the plan, so the compiler has to be told that they are global memory's.
typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x4h __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x2b __attribute__((ext_vector_type(2), aligned(1)));
template <typename T>
using global_ptr = __attribute__((address_space(1))) T *;
template <typename T, typename P>
__device__ __forceinline__ global_ptr<T> global(P *p) {
    return (global_ptr<T>)(T *)p;
}

// What a launch does not write, through the scalar cache.
template <typename T>
__device__ __forceinline__ T constant(const T *p) {
    struct Words {
        uint32_t w[sizeof(T) / 4];
    } words;
    const auto *from = (const __attribute__((address_space(4))) uint32_t *)reinterpret_cast<const uint32_t *>(p);
#pragma unroll
    for (size_t i = 0; i < sizeof(T) / 4; ++i) words.w[i] = from[i];
    return __builtin_bit_cast(T, words);
}
// Keeps a load in front of the branch that follows, so that both wait at once.
template <typename T>
__device__ __forceinline__ void loaded(T &x) {
    asm volatile("" : "+s"(x));
}

// A thread's elements: kPer of them, or the first n.  ONCE: not read again soon.
template <bool ONCE = true>
__device__ __forceinline__ void load_all(const float *p, int at, float (&x)[kPer]) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const auto *from = global<const f32x4u>(p + at + 4 * k);
        const f32x4u v = ONCE ? __builtin_nontemporal_load(from) : *from;
#pragma unroll
        for (int e = 0; e < 4; ++e) x[4 * k + e] = v[e];
    }
}
__device__ __forceinline__ void load_some(const float *p, int at, int n, float (&x)[kPer]) {
#pragma unroll
    for (int e = 0; e < kPer; ++e) x[e] = e < n ? global<const float>(p)[at + e] : 0.f;
}
__device__ __forceinline__ void store_all(float *p, int at, const float (&x)[kPer]) {
#pragma unroll
    for (int k = 0; k < 2; ++k)
        __builtin_nontemporal_store(f32x4u{x[4 * k], x[4 * k + 1], x[4 * k + 2], x[4 * k + 3]}, global<f32x4u>(p + at + 4 * k));
}
__device__ __forceinline__ void store_some(float *p, int at, int n, const float (&x)[kPer]) {
#pragma unroll
    for (int e = 0; e < kPer; ++e)
        if (e < n) global<float>(p)[at + e] = x[e];
}
__device__ __forceinline__ u32x2b load_all(const uint8_t *p, int at) { return __builtin_nontemporal_load(global<const u32x2b>(p + at)); }
__device__ __forceinline__ u32x2b load_some(const uint8_t *p, int at, int n) {
    u32x2b v = {0, 0};
#pragma unroll
    for (int e = 0; e < kPer; ++e)
        if (e < n) v[e >> 2] |= static_cast<uint32_t>(global<const uint8_t>(p)[at + e]) << (8 * (e & 3));
    return v;
}
__device__ __forceinline__ void store_some(uint8_t *p, int at, int n, u32x2b v) {
#pragma unroll
    for (int e = 0; e < kPer; ++e)
        if (e < n) global<uint8_t>(p)[at + e] = static_cast<uint8_t>(v[e >> 2] >> (8 * (e & 3)));
}

// Up to so many chunks every workgroup adds its group's sums up itself, while its elements are on their way, instead of a
// launch between.  us a step without and with, fp32 and 8-bit states: 76 chunks of one group 9.6 and 8.3, 12.1 and 10.5, 608
// of 8 groups 17.2 and 13.4, 15.4 and 14.4, 1,216 of 16 groups 24.4 and 22.0, 19.5 and 21.6.
constexpr uint32_t kJoinChunks = 1024;

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

// (One load of the whole header: conditions that are looked at one after the other would wait for one load each.)
__device__ __forceinline__ bool is_plan(const PlanArgs &a, const AdamwHeader &h) {
    return (h.magic == kAdamwMagic) & (h.bytes <= a.bytes) & (h.groups == a.groups) & (h.chunks <= a.room);
}
__device__ __forceinline__ double *parts_of(const PlanArgs &a, const AdamwHeader &h) {
    return reinterpret_cast<double *>(reinterpret_cast<char *>(a.header) + adamw_parts_at(a.groups, h.chunks));
}

// A wave for each chunk: the sum of its squared gradients in float64, at the chunk's place among its group's.
__global__ __launch_bounds__(kTh) void k_adamw_norm(PlanArgs a, const int64_t *step) {
    constexpr int kVec = kAdamwChunk / 64 / 4;
    const int lane = static_cast<int>(threadIdx.x & 63);
    const uint32_t c = blockIdx.x * (kTh / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (c >= a.room) return;
    const AdamwHeader h = constant(a.header);
    AdamwChunk k = constant(a.chunks + c);   // loaded beside the header; used if this is a plan
    loaded(k.grad);
    loaded(k.count);
    loaded(k.slot);
    const float *grad = k.grad;
    const int count = k.count;
    if (!is_plan(a, h)) return;
    if (c == 0 && lane == 0) a.group->step = *step + 1;   // where no k_adamw_head writes it
    if (c >= h.chunks) return;
    f32x4 g[kVec];
    if (count == kAdamwChunk) {
#pragma unroll
        for (int i = 0; i < kVec; ++i) g[i] = *global<const f32x4u>(grad + (i * 64 + lane) * 4);
    } else {
#pragma unroll
        for (int i = 0; i < kVec; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int at = (i * 64 + lane) * 4 + e;
                g[i][e] = at < count ? global<const float>(grad)[at] : 0.f;
            }
    }
    double s = 0.0;
#pragma unroll
    for (int i = 0; i < kVec; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) s = fma(static_cast<double>(g[i][e]), static_cast<double>(g[i][e]), s);
#pragma unroll
    for (int m = 32; m; m >>= 1) s += __shfl_xor(s, m);
    if (lane == 0) parts_of(a, h)[k.slot] = s;
}

// What a step asks for besides the plan.
struct StepArgs {
    int64_t *step;
    AdamwHyper y;
    const float *lr_scale;
    float *norms;
};

// A group's sum of squares, from its chunks' in order: the same in every thread.  red: a workgroup's.  meanwhile() is called
// while the first of them are on their way.
template <class Meanwhile>
__device__ __forceinline__ double square_of(const PlanArgs &a, const AdamwHeader &h, uint32_t begin, uint32_t end, double *red,
                                            const Meanwhile &meanwhile) {
    const double *parts = parts_of(a, h);
    double s = 0.0;
    constexpr int kBatch = 8;   // loads on their way together
    double v[kBatch];
    const auto load = [&](uint32_t i) {
#pragma unroll
        for (int j = 0; j < kBatch; ++j) v[j] = i + j * kTh < end ? parts[i + j * kTh] : 0.0;
    };
    const auto add = [&] {
#pragma unroll
        for (int j = 0; j < kBatch; ++j) s += v[j];
    };
    load(begin + threadIdx.x);
    meanwhile();
    add();
    for (uint32_t i = begin + kBatch * kTh + threadIdx.x; i < end; i += kBatch * kTh) {
        load(i);
        add();
    }
#pragma unroll
    for (int m = 32; m; m >>= 1) s += __shfl_xor(s, m);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
    __syncthreads();
    return ((red[0] + red[1]) + red[2]) + red[3];
}

// What a group's elements are multiplied by in step t, but for what its norm decides.
__device__ __forceinline__ AdamwGroup rates_of(const StepArgs &x, int group, int64_t t) {
    const AdamwHyper &y = x.y;
    const double fix1 = 1.0 - pow(y.beta1, static_cast<double>(t)), fix2 = 1.0 - pow(y.beta2, static_cast<double>(t));
    // lr lr_scale is one rounding, as a caller's own product of the two would be
    const double lr = static_cast<double>(x.lr_scale ? static_cast<float>(y.lr) * x.lr_scale[group] : static_cast<float>(y.lr));
    AdamwGroup o;
    o.clip = 1.0;
    o.lr = static_cast<float>(lr);
    o.rate = static_cast<float>(lr / fix1);
    o.root = static_cast<float>(1.0 / sqrt(fix2));
    o.skip = false;
    o.step = t;
    return o;
}
__device__ __forceinline__ void set_norm(AdamwGroup &o, double max_norm, double norm) {
    if (max_norm > 0.0 && norm > max_norm) o.clip = max_norm / norm;
    o.skip = !(norm < __builtin_inf());
}

// A workgroup for each group: its norm, and its record.
__global__ __launch_bounds__(kTh) void k_adamw_head(PlanArgs a, StepArgs x, bool with_norm) {
    const AdamwHeader h = constant(a.header);
    if (!is_plan(a, h)) return;
    __shared__ double red[kTh / 64];
    const int group = static_cast<int>(blockIdx.x);
    const int64_t done = *x.step;
    AdamwGroup o;
    if (with_norm) {
        const double norm = sqrt(square_of(a, h, a.starts[group], a.starts[group + 1], red, [&] { o = rates_of(x, group, done + 1); }));
        set_norm(o, x.y.max_norm, norm);
        if (x.norms && threadIdx.x == 0) x.norms[group] = static_cast<float>(norm);
    } else {
        o = rates_of(x, group, done + 1);
    }
    if (threadIdx.x == 0) a.group[group] = o;
}

// param after its move.  The hardware's root and reciprocal are within one last bit, and what they make is a correction of
// param; the root of small numbers is taken of a larger one, since the hardware's flushes subnormal ones.
__device__ __forceinline__ float moved(float p, float m, float v, const AdamwGroup &g, float keep, float eps) {
    const bool small = v < 0x1p-96f;
    const float root = __builtin_amdgcn_sqrtf(small ? v * 0x1p64f : v) * (small ? 0x1p-32f : 1.f);
    return fmaf(p, keep, -g.rate * m * __builtin_amdgcn_rcpf(fmaf(root, g.root, eps)));
}

// beta state + rest now.
__device__ __forceinline__ double mixed(double beta, double state, double rest, double now) {
#pragma clang fp contract(off)
    const double a = beta * state, b = rest * now;
    return a + b;
}

// The states' codes are made from the high and low words of m and v in float64.  kHuge: the high word of 2^128, from which on
// (and for infinities and NaN) a magnitude is not finite in fp32.
constexpr uint32_t kHuge = 0x47F00000u;
__device__ __forceinline__ uint32_t low_of(double x) { return static_cast<uint32_t>(__builtin_bit_cast(uint64_t, x)); }
__device__ __forceinline__ uint32_t high_of(double x) {   // of |x|
    return static_cast<uint32_t>(__builtin_bit_cast(uint64_t, x) >> 32) & 0x7FFFFFFFu;
}

// The exponent of a block's scale, from the high word of its largest magnitude (its last bit set where the low word holds
// anything): the scale brings it to 1.75 * 2^HIGH or below.
template <int HIGH>
__device__ __forceinline__ int scale_of(uint32_t key) {
    if (key < 0x00100000u) return 0;   // only zeros (a double that fp32 numbers give is not subnormal)
    const int k = static_cast<int>(key >> 20) - 1023 - HIGH + ((key & 0xFFFFFu) > 0xC0000u ? 1 : 0);
    return k < -126 ? -126 : k;
}

// An 8-bit type: BITS of mantissa, exponents from LOW on.  LEAST: the smallest code of what is not zero.
template <int BITS, int LOW, uint32_t LEAST>
struct Code {
    static constexpr int kCut = 4 - BITS;   // bits of the high word below 1 / 65536 of a step

    // The high word of the smallest normal number at the scale 2^k.
    static __device__ __forceinline__ uint32_t normal(int k) { return static_cast<uint32_t>(1023 + LOW + k) << 20; }

    // |x| 2^-k, not below the smallest normal number: x's own bits, rounded up where the part cut off exceeds draw / 65536 of
    // a step.  65535 - draw of these, and one less than a unit of what lies below them, carry exactly then.
    static __device__ __forceinline__ uint32_t of_normal(double x, int k, uint32_t draw) {
        const uint32_t lead = high_of(x) - (normal(k) - 0x100000u) + (low_of(x) != 0 ? 1u : 0u);
        return (lead + ((65535u - draw) << kCut) + ((1u << kCut) - 1u)) >> (16 + kCut);
    }

    // The same for any magnitude that is finite in fp32.
    static __device__ __forceinline__ uint32_t of(double x, int k, uint32_t draw) {
        const uint32_t high = high_of(x);
        if (high >= normal(k)) return of_normal(x, k, draw);
        if (high < 0x00100000u) return 0u;
        int drop = kCut + LOW + k + 1023 - static_cast<int>(high >> 20);
        drop = drop < 31 ? drop : 31;
        const uint32_t lead = ((high & 0xFFFFFu) | 0x100000u) + (low_of(x) != 0 ? 1u : 0u);
        const uint32_t fixed = (lead + ((1u << drop) - 1u)) >> drop, n = (fixed + 65535u - draw) >> 16;
        return n < LEAST ? LEAST : n;
    }
};

__device__ __forceinline__ uint32_t half_wave_max(uint32_t v) {
#pragma unroll
    for (int m = 16; m; m >>= 1) {
        const uint32_t o = static_cast<uint32_t>(__shfl_xor(static_cast<int>(v), m));
        v = v > o ? v : o;
    }
    return v;
}

// The key of a block's largest magnitude that is finite in fp32, from its threads' n elements each.
__device__ __forceinline__ uint32_t top_key(const double (&x)[kPer], int n) {
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
        const uint32_t h = high_of(x[e]), key = e < n && h < kHuge ? h | (low_of(x[e]) != 0 ? 1u : 0u) : 0u;
        top = key > top ? key : top;
    }
    return half_wave_max(top);
}

// The codes of a thread's elements; plain: every one is a normal number of its type.
template <bool PLAIN>
__device__ __forceinline__ void codes_of(const double (&m)[kPer], const double (&v)[kPer], int scale_m, int scale_v,
                                         const u32x4 (&bits)[2], u32x2b &out_m, u32x2b &out_v) {
    using M = Code<3, -6, 0>;    // e4m3
    using S = Code<2, -14, 1>;   // e5m2
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
        const uint32_t w = bits[e >> 2][e & 3];
        uint32_t one = PLAIN ? M::of_normal(m[e], scale_m, w & 0xFFFFu) : M::of(m[e], scale_m, w & 0xFFFFu);
        uint32_t two = PLAIN ? S::of_normal(v[e], scale_v, w >> 16) : S::of(v[e], scale_v, w >> 16);
        one |= static_cast<uint32_t>(__builtin_bit_cast(uint64_t, m[e]) >> 56) & 0x80u;
        if (!PLAIN) {
            one = high_of(m[e]) < kHuge ? one : 0x7Fu;                          // NaN (the type has no infinity)
            two = high_of(v[e]) < kHuge ? two : v[e] > 0.0 ? 0x7Cu : 0x7Fu;     // infinity, NaN
        }
        out_m[e >> 2] |= one << (8 * (e & 3));
        out_v[e >> 2] |= two << (8 * (e & 3));
    }
}

// JOIN: the records are made here, by every workgroup for itself, and not by k_adamw_head.
template <bool JOIN>
__global__ __launch_bounds__(kTh) void k_adamw_step(PlanArgs a, StepArgs x) {
    const AdamwHyper &y = x.y;
    const AdamwHeader h = constant(a.header);
    AdamwChunk k = constant(a.chunks + blockIdx.x);   // loaded beside the header; used if this is a plan
    loaded(k.grad);
    loaded(k.m_scale);
    loaded(k.count);
    if (!is_plan(a, h)) return;
    // the launch before has read the step, and no workgroup of this one does
    if (blockIdx.x == 0 && threadIdx.x == 0) *x.step = a.group->step;
    if (JOIN && blockIdx.x == 0 && x.norms)   // groups without chunks
        for (int group = static_cast<int>(threadIdx.x); group < a.groups; group += kTh)
            if (a.starts[group] == a.starts[group + 1]) x.norms[group] = 0.f;
    if (blockIdx.x >= h.chunks) return;
    const int at = static_cast<int>(threadIdx.x) * kPer, n = k.count - at;
    const auto record = [&] {
        if constexpr (!JOIN) return constant(a.group + k.group);
        __shared__ double red[kTh / 64];
        const uint32_t begin = a.starts[k.group], end = a.starts[k.group + 1];
        __shared__ AdamwGroup rates;   // one wave's work: the powers take as long as a chunk's elements
        const double norm = sqrt(square_of(a, h, begin, end, red, [&] {
            if (threadIdx.x < kTh - 64) return;
            const AdamwGroup of = rates_of(x, static_cast<int>(k.group), a.group->step);
            if (threadIdx.x == kTh - 1) rates = of;
        }));
        AdamwGroup of = rates;
        set_norm(of, y.max_norm, norm);
        if (x.norms && threadIdx.x == 0 && k.slot == begin) x.norms[k.group] = static_cast<float>(norm);
        return of;
    };
    AdamwGroup o;
    if (!JOIN) o = record();
    const auto kept = [&] { return k.decay ? static_cast<float>(1.0 - static_cast<double>(o.lr) * y.decay) : 1.f; };
    const float eps = static_cast<float>(y.eps);
    float p[kPer], g[kPer], keep;
    if (!k.m_scale) {
        float m[kPer], v[kPer];
        float *pm = static_cast<float *>(k.m), *pv = static_cast<float *>(k.v);
        if (n >= kPer) {
            load_all<false>(k.grad, at, g);
            load_all(k.param, at, p);
            load_all(pm, at, m);
            load_all(pv, at, v);
        } else {
            load_some(k.grad, at, n, g);
            load_some(k.param, at, n, p);
            load_some(pm, at, n, m);
            load_some(pv, at, n, v);
        }
        if (JOIN) o = record();   // (while the elements are on their way)
        if (o.skip) return;   // a model whose gradient is not finite stays as it is
        keep = kept();
        const float clip = static_cast<float>(o.clip), b1 = static_cast<float>(y.beta1), b2 = static_cast<float>(y.beta2);
        const float a1 = static_cast<float>(1.0 - y.beta1), a2 = static_cast<float>(1.0 - y.beta2);
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            const float cg = clip * g[e];
            m[e] = fmaf(a1, cg, b1 * m[e]);
            v[e] = fmaf(a2, cg * cg, b2 * v[e]);
            p[e] = moved(p[e], m[e], v[e], o, keep, eps);
        }
        if (n >= kPer) {
            store_all(pm, at, m);
            store_all(pv, at, v);
        } else {
            store_some(pm, at, n, m);
            store_some(pv, at, n, v);
        }
    } else {
        const int block = at / kAdamwBlock;   // half a wave has it
        const uint32_t i = k.first + static_cast<uint32_t>(at);
        uint8_t *pm = static_cast<uint8_t *>(k.m), *pv = static_cast<uint8_t *>(k.v);
        u32x2b cm, cv;
        float sm = 0.f, sv = 0.f;
        if (n >= kPer) {
            load_all<false>(k.grad, at, g);
            load_all(k.param, at, p);
            cm = load_all(pm, at);
            cv = load_all(pv, at);
            sm = global<const float>(k.m_scale)[block];
            sv = global<const float>(k.v_scale)[block];
        } else {
            load_some(k.grad, at, n, g);
            load_some(k.param, at, n, p);
            cm = load_some(pm, at, n);
            cv = load_some(pv, at, n);
            if (n > 0) {
                sm = global<const float>(k.m_scale)[block];
                sv = global<const float>(k.v_scale)[block];
            }
        }
        if (JOIN) o = record();
        if (o.skip) return;
        keep = kept();
        const double a1 = 1.0 - y.beta1, a2 = 1.0 - y.beta2, dm = sm, dv = sv;
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
            const double cg = o.clip * static_cast<double>(g[e]);
            m[e] = mixed(y.beta1, dm * static_cast<double>(fm), a1, cg);
            v[e] = mixed(y.beta2, dv * static_cast<double>(fv), a2, cg * cg);
            p[e] = moved(p[e], static_cast<float>(m[e]), static_cast<float>(v[e]), o, keep, eps);
        }
        // The largest and smallest magnitudes by their high words alone, which is all but always enough.  (Elements past
        // the tensor's end are zeros, unless a scale was not finite.)
        uint32_t top_m = 0, top_v = 0, low_m = ~0u, low_v = ~0u;
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            const uint32_t hm = high_of(m[e]), hv = high_of(v[e]);
            top_m = hm > top_m ? hm : top_m;
            top_v = hv > top_v ? hv : top_v;
            low_m = hm < low_m ? hm : low_m;
            low_v = hv < low_v ? hv : low_v;
        }
        top_m = half_wave_max(top_m);
        top_v = half_wave_max(top_v);
        // not finite, or next to 1.75 times a power of two
        const auto unsure = [](uint32_t top) { return top >= kHuge || (top & 0xFFFFFu) == 0xC0000u; };
        const bool sure = !unsure(top_m) && !unsure(top_v);
        if (__builtin_amdgcn_ballot_w64(!sure)) {
            top_m = top_key(m, n);
            top_v = top_key(v, n);
        }
        const int scale_m = scale_of<8>(top_m), scale_v = scale_of<15>(top_v);
        const bool plain = sure && low_m >= Code<3, -6, 0>::normal(scale_m) && low_v >= Code<2, -14, 1>::normal(scale_v);
        const uint32_t t = static_cast<uint32_t>(o.step);
        const u32x4 bits[2] = {philox(i / 4, k.slice, k.tensor, t, y.key[0], y.key[1]),
                               philox(i / 4 + 1, k.slice, k.tensor, t, y.key[0], y.key[1])};
        u32x2b out_m = {0, 0}, out_v = {0, 0};
        if (__builtin_amdgcn_ballot_w64(!plain) == 0)
            codes_of<true>(m, v, scale_m, scale_v, bits, out_m, out_v);
        else
            codes_of<false>(m, v, scale_m, scale_v, bits, out_m, out_v);
        if (n >= kPer) {
            __builtin_nontemporal_store(out_m, global<u32x2b>(pm + at));
            __builtin_nontemporal_store(out_v, global<u32x2b>(pv + at));
        } else {
            store_some(pm, at, n, out_m);
            store_some(pv, at, n, out_v);
        }
        if (n > 0 && (threadIdx.x & 31) == 0) {
            global<float>(k.m_scale)[block] = __uint_as_float(static_cast<uint32_t>(scale_m + 127) << 23);
            global<float>(k.v_scale)[block] = __uint_as_float(static_cast<uint32_t>(scale_v + 127) << 23);
        }
    }
    const u32x4 w = Vec<true>::pack(p);
    bf16_bits *work = static_cast<bf16_bits *>(k.work);
    if (n >= kPer) {
        store_all(k.param, at, p);
        if (work) __builtin_nontemporal_store((u32x4h)w, global<u32x4h>(work + at));
    } else {
        store_some(k.param, at, n, p);
#pragma unroll
        for (int e = 0; e < kPer; ++e)
            if (work && e < n) global<bf16_bits>(work)[at + e] = static_cast<bf16_bits>(w[e >> 1] >> (16 * (e & 1)));
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
    const StepArgs x = {step, y, lr_scale, norms};
    const bool with_norm = norms || y.max_norm > 0.0;
    if (with_norm) k_adamw_norm<<<(a.room + 3) / 4, kTh, 0, s>>>(a, step);
    if (with_norm && a.room <= kJoinChunks) {
        k_adamw_step<true><<<a.room, kTh, 0, s>>>(a, x);
    } else {
        k_adamw_head<<<groups, kTh, 0, s>>>(a, x, with_norm);
        k_adamw_step<false><<<a.room, kTh, 0, s>>>(a, x);
    }
    return hipGetLastError();
}

}  // namespace logra
