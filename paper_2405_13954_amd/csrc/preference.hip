// The loss of pairs of answers by their log ratios, and the gradient of every logit:
//
//   lp_s = sum over the tokens t of sequence s of (z_t[target_t] - lse(z_t))
//   d    = beta ((lp_chosen - ref_chosen) - (lp_rejected - ref_rejected))
//   loss = w ((1 - e) softplus(-d) + e softplus(d)),   slope = w beta (e - sigma(-d))
//   dz_t = +-slope (onehot - softmax(z_t))             (+ chosen, - rejected)
//
// A token's gradient needs the sums of its whole pair, so the logits go by twice: k_pair_stats forms the maximum and the
// sum of exponentials of ranges of each row, k_pair_sums joins them, adds up each sequence (in float64: the ratio is a
// small difference of large sums) and leaves two factors for every row, and k_pair_grad writes the gradient.  The second
// pass takes the rows from the last to the first, so that those that the 256 MB cache still holds are read from there.  Small
// calls have the second and third launch in one (k_pair_few).
// 2,048 tokens of 128,000 bf16 logits, 0.3 of them masked: 68 + 6 + 128 us for 367, 0 and 891 MB (5.4 and 6.9 TB/s; a copy
// inside the cache reaches 7.2).
#include "internal.h"
#include "vec16.h"

namespace logra {
namespace {

constexpr int kMaxSplits = 16;   // ranges of a row that are summed by workgroups of their own
constexpr int kTh = 256;

// Of one token: its maximum, the sum of exp(z - top) and then, in its place, the factor of the gradient
// dz = factor exp(z - top) + (hot at the target).  Zeros: no gradient.
struct Row {
    float top;
    union {
        float total, factor;
    };
    float hot, unused;
};

struct PairArgs {
    const char *logits;
    int64_t ld, rows;
    const int64_t *target, *offsets;
    float2 *part;   // [rows][splits]: maximum, sum
    float *zt;      // [rows]: the target's logit
    Row *row;       // [rows]
    int vocab, splits, pairs;
};

// Whether the row counts: its target is a token, and it lies in the sequences.
__device__ __forceinline__ bool counts(const PairArgs &a, int64_t row, int64_t t) {
    const int64_t first = a.offsets[0], last = a.offsets[2 * static_cast<int64_t>(a.pairs)];
    return (t >= 0) & (t < a.vocab) & (row >= first) & (row < last);   // (the loads wait together)
}

// Workgroups that take parts of rows: the part in x, the row in y and z.
__device__ __forceinline__ int64_t row_of() { return blockIdx.y + static_cast<int64_t>(gridDim.y) * blockIdx.z; }

template <bool BF16>
__global__ __launch_bounds__(kTh) void k_pair_stats(PairArgs a) {
    using V = Vec<BF16>;
    constexpr int kEs = BF16 ? 2 : 4, kGroup = 4;
    constexpr float kNone = -__builtin_inff();
    __shared__ float red[kTh / 64];
    const int64_t row = row_of();
    const int split = static_cast<int>(blockIdx.x), tid = static_cast<int>(threadIdx.x);
    if (row >= a.rows) return;
    if (split == 0 && tid == 0) a.row[row] = {0.f, 0.f, 0.f, 0.f};   // no gradient, until k_pair_sums says more
    const int64_t t = a.target[row];
    if (!counts(a, row, t)) return;   // nothing of it is read
    const char *z = a.logits + row * a.ld * kEs;
    const int n_full = a.vocab / V::kN, odd = a.vocab - n_full * V::kN;   // whole vectors; logits of the last, partial one
    const int each = (n_full + a.splits - 1) / a.splits, begin = split * each, end = begin + each < n_full ? begin + each : n_full;
    float top = kNone, total = 0.f;
    const auto take = [&](const u32x4 (&v)[kGroup]) {
        float m = top;
#pragma unroll
        for (int j = 0; j < kGroup; ++j)
#pragma unroll
            for (int e = 0; e < V::kN; ++e) m = fmaxf(m, V::get(v[j], e));
        const float base = m == kNone ? 0.f : m;
        total *= exp_from(top, base);
#pragma unroll
        for (int j = 0; j < kGroup; ++j) {
            float q = 0.f;
#pragma unroll
            for (int e = 0; e < V::kN; ++e) q += exp_from(V::get(v[j], e), base);
            total += q;
        }
        top = m;
    };
    int i = begin + tid;
    for (; i + (kGroup - 1) * kTh < end; i += kGroup * kTh) {
        u32x4 v[kGroup];
#pragma unroll
        for (int j = 0; j < kGroup; ++j) v[j] = ld128(z + static_cast<int64_t>(i + j * kTh) * 16);
        take(v);
    }
    const bool tail = odd > 0 && split == a.splits - 1 && tid == kTh - 1;   // the thread that has the partial vector
    if (i < end || tail) {   // (i + 3 kTh is past the end: at most three vectors are left)
        u32x4 v[kGroup];
#pragma unroll
        for (int j = 0; j < kGroup - 1; ++j) v[j] = i + j * kTh < end ? ld128(z + static_cast<int64_t>(i + j * kTh) * 16) : V::none();
        v[kGroup - 1] = V::none();
        if (tail) v[kGroup - 1] = V::load(z + static_cast<int64_t>(n_full) * 16, odd);
        take(v);
    }
    const float mine = top;
    top = group_reduce<kTh, true>(mine, red);
    total = group_reduce<kTh, false>(total * exp_from(mine, top == kNone ? 0.f : top), red);
    if (tid == 0) {
        a.part[row * a.splits + split] = make_float2(top, total);
        if (split == 0) {
            float zt;
            if constexpr (BF16)
                zt = bf16_to_f32(reinterpret_cast<const bf16_bits *>(z)[t]);
            else
                zt = reinterpret_cast<const float *>(z)[t];
            a.zt[row] = zt;
        }
    }
}

// What the pairs are compared by, and what is wanted of them.
struct LossArgs {
    const float *ref, *weight;
    double beta, smoothing;
    float *loss, *logp;
};

// A row's log probability, maximum and sum, from its ranges'.  What it needs is loaded at once, whether the row counts or not.
__device__ __forceinline__ double row_sums(const PairArgs &a, int64_t row, int64_t first, int64_t last, float &top, float &total) {
    constexpr float kNone = -__builtin_inff();
    const int64_t t = a.target[row];
    const float2 *part = a.part + row * a.splits;
    const float zt = a.zt[row];
    float2 p[kMaxSplits];
#pragma unroll
    for (int i = 0; i < kMaxSplits; ++i) p[i] = i < a.splits ? part[i] : make_float2(kNone, 0.f);
    float m = kNone, sum = 0.f;
#pragma unroll
    for (int i = 0; i < kMaxSplits; ++i) m = fmaxf(m, p[i].x);
    top = m == kNone ? 0.f : m;
#pragma unroll
    for (int i = 0; i < kMaxSplits; ++i) sum += p[i].y * exp_from(p[i].x, top);
    if (t < 0 || t >= a.vocab || row < first || row >= last) {   // never written: whatever was loaded is dropped
        total = 0.f;
        return 0.0;
    }
    total = sum;
    // without a finite logit there is no distribution, and no token of it has a chance
    return sum == 0.f ? -__builtin_inf() : static_cast<double>(zt - top) - static_cast<double>(logf(sum));
}

// The log probabilities of a pair's sequences, whose rows are cut[0] .. cut[1] - 1 and cut[1] .. cut[2] - 1, the same in every
// thread; keep(s, first, row, top, total) is called for every row, `first` for each thread's first of sequence s.
template <int TH, class Keep>
__device__ __forceinline__ void pair_sums(const PairArgs &a, const int64_t (&cut)[3], int64_t first, int64_t last,
                                          double (&red)[2][TH / 64], double (&sum)[2], const Keep &keep) {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        double mine = 0.0;
        float m, q;
        const int64_t at = cut[s] + threadIdx.x;
        if (at < cut[s + 1]) {
            mine = row_sums(a, at, first, last, m, q);
            keep(s, true, at, m, q);
        }
        for (int64_t row = at + TH; row < cut[s + 1]; row += TH) {
            mine += row_sums(a, row, first, last, m, q);
            keep(s, false, row, m, q);
        }
#pragma unroll
        for (int k = 32; k; k >>= 1) mine += __shfl_xor(mine, k);
        if ((threadIdx.x & 63) == 0) red[s][threadIdx.x >> 6] = mine;
    }
    __syncthreads();
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        sum[s] = 0.0;
#pragma unroll
        for (int w = 0; w < TH / 64; ++w) sum[s] += red[s][w];
    }
}

__device__ __forceinline__ double softplus(double x) { return fmax(x, 0.0) + log1p(exp(-fabs(x))); }

// The slope of a pair's loss, from its sequences' log probabilities; with `write`, its loss and these are written.
__device__ __forceinline__ double pair_end(const LossArgs &l, int64_t pair, const double (&sum)[2], bool write) {
    const double ratio_c = sum[0] - (l.ref ? static_cast<double>(l.ref[2 * pair]) : 0.0);
    const double ratio_r = sum[1] - (l.ref ? static_cast<double>(l.ref[2 * pair + 1]) : 0.0);
    const double d = l.beta * (ratio_c - ratio_r);
    const double w = l.weight ? static_cast<double>(l.weight[pair]) : 1.0;
    const bool off = w == 0.0;   // a pair that does not count, whatever its logits hold
    if (write) {
        l.logp[2 * pair] = static_cast<float>(sum[0]);
        l.logp[2 * pair + 1] = static_cast<float>(sum[1]);
        const double flipped = l.smoothing > 0.0 ? l.smoothing * softplus(d) : 0.0;
        const double kept = l.smoothing < 1.0 ? (1.0 - l.smoothing) * softplus(-d) : 0.0;
        if (l.loss) l.loss[pair] = off ? 0.f : static_cast<float>(w * (kept + flipped));
    }
    return off ? 0.0 : w * l.beta * (l.smoothing - 1.0 / (1.0 + exp(d)));
}

// What the gradient of a row is made of, of a sequence with this slope.
__device__ __forceinline__ Row factors(float hot, float top, float total) {
    const bool none = total == 0.f || hot == 0.f;
    return {top, none ? 0.f : -hot / total, none ? 0.f : hot, 0.f};
}

// One workgroup per pair.  What was found of a thread's first row of each sequence stays in registers.
template <int kSumTh>
__global__ __launch_bounds__(kSumTh) void k_pair_sums(PairArgs a, LossArgs l) {
    const int64_t pair = blockIdx.x + static_cast<int64_t>(gridDim.x) * blockIdx.y;
    if (pair >= a.pairs) return;
    __shared__ double red[2][kSumTh / 64];
    int64_t cut[3];
    const int64_t first = a.offsets[0], last = a.offsets[2 * static_cast<int64_t>(a.pairs)];
#pragma unroll
    for (int i = 0; i < 3; ++i) {   // whatever the offsets hold, rows outside the logits are not touched
        const int64_t o = a.offsets[2 * pair + i];
        cut[i] = o < 0 ? 0 : o > a.rows ? a.rows : o;
    }
    float top[2] = {0.f, 0.f}, total[2] = {0.f, 0.f};
    double sum[2];
    pair_sums<kSumTh>(a, cut, first, last, red, sum, [&](int s, bool of_thread, int64_t row, float m, float q) {
        if (of_thread) {
            top[s] = m;
            total[s] = q;
        } else {
            a.row[row].top = m;
            a.row[row].total = q;
        }
    });
    const double slope = pair_end(l, pair, sum, threadIdx.x == 0);
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        const float hot = static_cast<float>(s ? -slope : slope);
        const int64_t at = cut[s] + threadIdx.x;
        if (at < cut[s + 1]) a.row[at] = factors(hot, top[s], total[s]);
        for (int64_t row = at + kSumTh; row < cut[s + 1]; row += kSumTh) a.row[row] = factors(hot, a.row[row].top, a.row[row].total);
    }
}

// A workgroup writes kGroup x kTh vectors of one row.  us with two, four and eight vectors a thread: 2,048 rows of 128,000
// bf16 logits 127, 131 and 129, 2,041 rows of 50,257 54, 55 and 65.
constexpr int kGroup = 2;
__device__ __forceinline__ int first_vector() {
    return static_cast<int>(blockIdx.x) * kGroup * kTh + static_cast<int>(threadIdx.x);
}
template <bool BF16>
__device__ __forceinline__ void take_logits(const char *z, int vocab, u32x4 (&v)[kGroup]) {
    using V = Vec<BF16>;
    const int first = first_vector();
    if ((first - static_cast<int>(threadIdx.x) + kGroup * kTh) * V::kN <= vocab) {   // the whole workgroup's vectors are whole
#pragma unroll
        for (int j = 0; j < kGroup; ++j) v[j] = ld128_nt(z + static_cast<int64_t>(first + j * kTh) * 16);
        return;
    }
#pragma unroll
    for (int j = 0; j < kGroup; ++j) {
        const int i = first + j * kTh, n = vocab - i * V::kN;
        v[j] = n >= V::kN ? ld128_nt(z + static_cast<int64_t>(i) * 16)
                          : (n > 0 ? V::load(z + static_cast<int64_t>(i) * 16, n) : V::none());
    }
}
template <bool BF16>
__device__ __forceinline__ void put_zeros(char *dz, int vocab) {
    using V = Vec<BF16>;
#pragma unroll
    for (int j = 0; j < kGroup; ++j) {
        const int i = first_vector() + j * kTh, n = vocab - i * V::kN;
        if (n > 0) V::put(dz + static_cast<int64_t>(i) * 16, u32x4{0, 0, 0, 0}, n);
    }
}
template <bool BF16>
__device__ __forceinline__ void put_gradient(const u32x4 (&v)[kGroup], const Row &r, int t, char *dz, int vocab) {
    using V = Vec<BF16>;
#pragma unroll
    for (int j = 0; j < kGroup; ++j) {
        const int i = first_vector() + j * kTh, n = vocab - i * V::kN;
        if (n <= 0) continue;
        float g[V::kN];
#pragma unroll
        for (int e = 0; e < V::kN; ++e) g[e] = exp_from(V::get(v[j], e), r.top) * r.factor;
        const int hit = t - i * V::kN;
        if (hit >= 0 && hit < V::kN) {
#pragma unroll
            for (int e = 0; e < V::kN; ++e) g[e] += e == hit ? r.hot : 0.f;
        }
        V::store(dz + static_cast<int64_t>(i) * 16, g, n);
    }
}

template <bool BF16>
__global__ __launch_bounds__(kTh) void k_pair_grad(PairArgs a, char *dlogits, int64_t ld_d) {
    constexpr int kEs = BF16 ? 2 : 4;
    const int64_t row = a.rows - 1 - row_of();
    if (row < 0) return;
    char *dz = dlogits + row * ld_d * kEs;
    const Row r = a.row[row];
    if (r.factor == 0.f && r.hot == 0.f) return put_zeros<BF16>(dz, a.vocab);
    u32x4 v[kGroup];
    take_logits<BF16>(a.logits + row * a.ld * kEs, a.vocab, v);
    put_gradient<BF16>(v, r, static_cast<int>(a.target[row]), dz, a.vocab);
}

// Few rows and pairs: the gradient's workgroups add up their row's pair themselves, while its logits are on their way, and one
// for each pair behind them writes the loss.
constexpr int kFewPairs = kTh / 2 - 1;   // a thread for every offset
template <bool BF16>
__global__ __launch_bounds__(kTh) void k_pair_few(PairArgs a, LossArgs l, char *dlogits, int64_t ld_d) {
    constexpr int kEs = BF16 ? 2 : 4;
    __shared__ int64_t cuts[kTh];
    __shared__ double red[2][kTh / 64];
    __shared__ float own[2];
    const int tid = static_cast<int>(threadIdx.x), row = static_cast<int>(a.rows) - 1 - static_cast<int>(blockIdx.y);
    if (row < 0 && blockIdx.x > 0) return;
    const int64_t t = row < 0 ? -1 : a.target[row];
    bool before = false;
    if (tid <= 2 * a.pairs) {
        const int64_t o = a.offsets[tid];
        cuts[tid] = o < 0 ? 0 : o > a.rows ? a.rows : o;
        before = o <= row;
    }
    if (tid < 2) own[tid] = 0.f;
    const int sequence = __syncthreads_count(before) - 1;
    const int64_t first = cuts[0], last = cuts[2 * a.pairs];
    u32x4 v[kGroup];
    if (row >= 0) {
        char *dz = dlogits + row * ld_d * kEs;
        if (t < 0 || t >= a.vocab || row < first || row >= last) return put_zeros<BF16>(dz, a.vocab);   // nothing of it is read
        take_logits<BF16>(a.logits + row * a.ld * kEs, a.vocab, v);
    }
    // (offsets that decrease can give a sequence that the row is not in, but none out of range: the first is not above the
    // row, and the last one is)
    const int pair = row < 0 ? -1 - row : sequence / 2;
    const int64_t cut[3] = {cuts[2 * pair], cuts[2 * pair + 1], cuts[2 * pair + 2]};
    double sum[2];
    pair_sums<kTh>(a, cut, first, last, red, sum, [&](int, bool, int64_t at, float m, float q) {
        if (at == row) {
            own[0] = m;
            own[1] = q;
        }
    });
    const double slope = pair_end(l, pair, sum, row < 0 && tid == 0);
    if (row < 0) return;
    const Row r = factors(static_cast<float>(sequence & 1 ? -slope : slope), own[0], own[1]);
    char *dz = dlogits + row * ld_d * kEs;
    if (r.factor == 0.f && r.hot == 0.f) return put_zeros<BF16>(dz, a.vocab);
    put_gradient<BF16>(v, r, static_cast<int>(t), dz, a.vocab);
}

// Up to so many workgroups of the gradient, where pairs have no more than 128 rows on average, k_pair_few takes the place of
// k_pair_sums and k_pair_grad.  us of a call's kernels with and without: 64 rows of 516 bf16 logits 9.1 and 10.9, 512 rows of
// 5,004 fp32 (1,536 workgroups) 13.0 and 14.7, 128 rows of 32,004 bf16 (1,024) 12.7 and 15.3, 256 (2,048) 19.0 and 18.8, 64 rows
// of 128,004 (2,048) 19.4 and 18.8.  A launch less is also 2.6 us less of the host's time.
constexpr int kFewGroups = 1536;

dim3 grid_of(int parts, int64_t rows) {
    const int64_t z = (rows + 65534) / 65535;
    return dim3(static_cast<uint32_t>(parts), static_cast<uint32_t>((rows + z - 1) / z), static_cast<uint32_t>(z));
}

}  // namespace

size_t preference_ws_bytes(int64_t rows) {
    return align256(rows * kMaxSplits * sizeof(float2)) + align256(rows * sizeof(float)) + align256(rows * sizeof(Row));
}

hipError_t launch_preference_loss(const PreferenceLoss &p, hipStream_t s) {
    const int vec = (p.vocab + (p.bf16 ? 7 : 3)) / (p.bf16 ? 8 : 4);
    // Ranges of 16 vectors a thread; shorter ones, of four at least, where there are few rows: eight workgroups on a CU.
    // us of k_pair_stats with at most 4, 8, 16 and 32: 2,048 rows of 128,000 bf16 logits, 0.3 of them masked, 84, 70, 68
    // and 72; 61 rows of 5,001 fp32 logits 4.0, 4.8, 4.8 and 4.7.
    const auto ranges = [&](int of) { return (vec + of * kTh - 1) / (of * kTh); };
    const int64_t wanted = (2048 + p.rows - 1) / (p.rows > 0 ? p.rows : 1);
    int splits = static_cast<int>(wanted < ranges(4) ? wanted : ranges(4));
    splits = splits > ranges(16) ? splits : ranges(16);
    splits = splits < kMaxSplits ? splits : kMaxSplits;
    char *ws = static_cast<char *>(p.ws);
    PairArgs a = {static_cast<const char *>(p.logits), p.ld, p.rows, p.target, p.offsets, reinterpret_cast<float2 *>(ws),
                  reinterpret_cast<float *>(ws + align256(p.rows * kMaxSplits * sizeof(float2))),
                  reinterpret_cast<Row *>(ws + align256(p.rows * kMaxSplits * sizeof(float2)) + align256(p.rows * sizeof(float))),
                  p.vocab, splits, p.pairs};
    if (p.rows > 0) {
        const dim3 grid = grid_of(splits, p.rows);
        p.bf16 ? k_pair_stats<true><<<grid, kTh, 0, s>>>(a) : k_pair_stats<false><<<grid, kTh, 0, s>>>(a);
    }
    const LossArgs l = {p.ref, p.weight, p.beta, p.smoothing, p.loss, p.logp};
    const int pieces = (vec + kGroup * kTh - 1) / (kGroup * kTh);
    char *dz = static_cast<char *>(p.dlogits);
    if (dz && p.rows > 0 && p.rows * pieces <= kFewGroups && p.pairs <= kFewPairs && p.rows <= 128 * static_cast<int64_t>(p.pairs)) {
        const dim3 grid(static_cast<uint32_t>(pieces), static_cast<uint32_t>(p.rows + p.pairs));
        p.bf16 ? k_pair_few<true><<<grid, kTh, 0, s>>>(a, l, dz, p.ld_d) : k_pair_few<false><<<grid, kTh, 0, s>>>(a, l, dz, p.ld_d);
        return hipGetLastError();
    }
    const auto sums = [&](auto kernel, int threads) {
        const int64_t gx = p.pairs < (1 << 21) ? p.pairs : (1 << 21);
        kernel<<<dim3(static_cast<uint32_t>(gx), static_cast<uint32_t>((p.pairs + gx - 1) / gx)), threads, 0, s>>>(a, l);
    };
    // 256 threads where most sequences have no more rows: 32 pairs in 2,041 rows 5.7 us against 6.1 with 1024, 8 pairs in
    // 2,048 rows 7.4 against 6.4.
    if (p.rows <= 128 * static_cast<int64_t>(p.pairs))
        sums(k_pair_sums<256>, 256);
    else
        sums(k_pair_sums<1024>, 1024);
    if (dz && p.rows > 0) {
        const dim3 grid = grid_of(pieces, p.rows);
        p.bf16 ? k_pair_grad<true><<<grid, kTh, 0, s>>>(a, dz, p.ld_d) : k_pair_grad<false><<<grid, kTh, 0, s>>>(a, dz, p.ld_d);
    }
    return hipGetLastError();
}

}  // namespace logra
