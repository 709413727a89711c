// Layer norm of rows, with or without the mean, and its backward pass:
//
//   forward   h = x + residual,  y = (h - mean) rstd gain + bias,  rstd = 1 / sqrt(mean((h - mean)^2) + eps)
//   backward  xh = (h - mean) rstd,  c = dy gain,  dx = base + rstd (c - avg(c) - xh avg(c xh)),
//             dgain = sum_t dy xh,  dbias = sum_t dy
//
// (rms: mean = 0, and no avg(c).)  A row is held in the registers of a team of threads, each with NV of its 16-byte
// vectors, so memory sees every tensor once, which is what bounds both passes.  The variance is that of the differences
// from the mean, formed after the mean: no cancellation.  Sums and statistics are fp32.  The statistics' terms are scaled by a
// power of two (exact for normal numbers; of smaller terms eps leaves nothing), so that their sums stay near the averages: what
// overflows is an average beyond fp32, and not the sum of a wide row.
//
// Backward: a workgroup walks rows a grid apart and keeps the sums for dgain and dbias of its columns in registers; the
// next row's vectors are loaded before the current row's sums are known.  The workgroups' sums go to the workspace, and a
// second launch adds them in order, so that reruns give the same bits.  Few rows: one launch (k_norm_bwd_few).
//
// 16,384 rows of 4096 bf16 columns without the mean: forward with residual and statistics 94 us for 537 MB (5.7 TB/s),
// backward with base and a fifth of the rows masked 79 + 5 us for 483 MB (5.7).  768 columns with the mean: 16 and 20 + 4 us
// for 91 and 101 MB.
#include "internal.h"
#include "vec16.h"

namespace logra {
namespace {

struct FwdArgs {
    const char *x, *res;
    char *h, *y;
    int64_t ld_x, ld_r, ld_h, ld_y, rows;
    const uint8_t *mask;
    const char *gain, *bias;
    float *mean, *rstd;
    int cols;
    float eps;
    float root, per;   // 2^-k, 4^k / cols for the smallest 4^k >= cols
    bool stream;
};

struct BwdArgs {
    const char *h, *dy, *base;
    char *dx;
    int64_t ld_h, ld_dy, ld_b, ld_dx, rows;
    const uint8_t *mask;
    const char *gain;
    const float *mean, *rstd;
    float *part_g, *part_b;   // [workgroups][cols], or NULL
    int cols;
};

// The workgroups' sums lie in rows of whole vectors.
__host__ __device__ inline int padded(int cols) { return (cols + 3) & ~3; }

constexpr u32x4 kZero4 = {0, 0, 0, 0};

// The vector of n elements at p (n <= 0: zeros, nothing is read).  p need have the elements' alignment only: a gain may be
// one of several models' of an odd width, one behind the other.
typedef uint32_t u32x4e __attribute__((ext_vector_type(4), aligned(2)));
template <bool BF16>
__device__ __forceinline__ u32x4 take(const char *p, int n) {
    if (n >= Vec<BF16>::kN) return *reinterpret_cast<const u32x4e *>(p);
    return n > 0 ? Vec<BF16>::load(p, n, kZero4) : kZero4;
}

// The same for a row that another one follows: row strides are whole vectors, so what a partial vector's load brings
// besides lies between the rows.  first_of drops it where the vector is used, so that the load need not be waited for here.
template <bool BF16, bool STREAM>
__device__ __forceinline__ u32x4 take_inner(const char *p, int n, bool inner) {
    if (n >= Vec<BF16>::kN || (inner && n > 0)) return STREAM ? ld128_nt(p) : ld128(p);
    return n > 0 ? Vec<BF16>::load(p, n, kZero4) : kZero4;
}
// The NV vectors of a thread: those at lane, lane + TPR, ... of a row of `cols` elements.
template <bool BF16, int TPR, int NV, bool STREAM>
__device__ __forceinline__ void take_row(const char *row, int lane, int cols, bool inner, u32x4 (&v)[NV]) {
#pragma unroll
    for (int k = 0; k < NV; ++k)
        v[k] = take_inner<BF16, STREAM>(row + (k * TPR + lane) * 16, cols - (k * TPR + lane) * Vec<BF16>::kN, inner);
}

// The first n elements of v, zeros behind them.
template <bool BF16>
__device__ __forceinline__ u32x4 first_of(u32x4 v, int n) {
    if (n >= Vec<BF16>::kN) return v;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if constexpr (BF16)
            v[j] = n >= 2 * j + 2 ? v[j] : n == 2 * j + 1 ? v[j] & 0xFFFFu : 0u;
        else
            v[j] = n > j ? v[j] : 0u;
    }
    return v;
}

// Sum over a row's team, the same in every thread, in a fixed order.  red: a slot for each wave, of this call alone until
// the next but one barrier.
template <int TPR>
__device__ __forceinline__ float team_sum(float v, float *red) {
#pragma unroll
    for (int m = (TPR < 64 ? TPR : 64) / 2; m; m >>= 1) v += __shfl_xor(v, m);
    if constexpr (TPR > 64) {
        if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
        __syncthreads();
        v = red[0];
#pragma unroll
        for (int w = 1; w < TPR / 64; ++w) v += red[w];
    }
    return v;
}

// The backward pass's two sums (CENTER: both) over a row's team.  red: a slot of each for every wave of the workgroup.
template <int TPR, bool CENTER, int WAVES>
__device__ __forceinline__ void team_sums(float &s1, float &s2, float (&red)[2][WAVES], int team) {
    constexpr int kW = TPR > 64 ? TPR / 64 : 1;
#pragma unroll
    for (int m = (TPR < 64 ? TPR : 64) / 2; m; m >>= 1) {
        s2 += __shfl_xor(s2, m);
        if constexpr (CENTER) s1 += __shfl_xor(s1, m);
    }
    if constexpr (TPR > 64) {
        if ((threadIdx.x & 63) == 0) {
            red[0][threadIdx.x >> 6] = s1;
            red[1][threadIdx.x >> 6] = s2;
        }
        __syncthreads();
        s1 = 0.f;
        s2 = 0.f;
#pragma unroll
        for (int w = 0; w < kW; ++w) {
            if constexpr (CENTER) s1 += red[0][team * kW + w];
            s2 += red[1][team * kW + w];
        }
    }
}

template <bool BF16, int TPR, int NV, bool CENTER>
__global__ __launch_bounds__(TPR <= 64 ? 256 : TPR) void k_norm_fwd(FwdArgs a) {
    using V = Vec<BF16>;
    constexpr int kTeams = TPR <= 64 ? 256 / TPR : 1, kEs = BF16 ? 2 : 4;
    __shared__ float red[2][TPR > 64 ? TPR / 64 : 1];
    const int lane = static_cast<int>(threadIdx.x) % TPR;
    const int64_t row = (blockIdx.x + static_cast<int64_t>(gridDim.x) * blockIdx.y) * kTeams + threadIdx.x / TPR;
    if (row >= a.rows) return;   // (whole teams: one wave or less, or the whole workgroup)
    const char *x = a.x + row * a.ld_x * kEs;
    char *y = a.y + row * a.ld_y * kEs;
    char *h_out = a.h ? a.h + row * a.ld_h * kEs : nullptr;
    if (a.mask && a.mask[row] == 0) {   // nothing of it is read
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int i = k * TPR + lane, n = a.cols - i * V::kN;
            if (n > 0) {
                if (h_out) V::put(h_out + i * 16, kZero4, n);
                V::put(y + i * 16, kZero4, n);
            }
        }
        if (lane == 0) {
            if (a.mean) a.mean[row] = 0.f;
            if (a.rstd) a.rstd[row] = 0.f;
        }
        return;
    }
    const bool inner = row + 1 < a.rows;
    const char *r = a.res + row * a.ld_r * kEs;
    u32x4 h[NV], v[NV];
    if (a.stream) {
        take_row<BF16, TPR, NV, true>(x, lane, a.cols, inner, h);
        if (a.res) take_row<BF16, TPR, NV, true>(r, lane, a.cols, inner, v);
    } else {
        take_row<BF16, TPR, NV, false>(x, lane, a.cols, inner, h);
        if (a.res) take_row<BF16, TPR, NV, false>(r, lane, a.cols, inner, v);
    }
    if (a.res) {
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            float s[V::kN];
#pragma unroll
            for (int e = 0; e < V::kN; ++e) s[e] = V::get(h[k], e) + V::get(v[k], e);
            h[k] = V::pack(s);   // the sum is rounded where it is stored, and the norm is that of the stored sum
        }
    }
#pragma unroll
    for (int k = 0; k < NV; ++k) h[k] = first_of<BF16>(h[k], a.cols - (k * TPR + lane) * V::kN);
    float mean = 0.f;
    if constexpr (CENTER) {
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int e = 0; e < V::kN; ++e) s = fmaf(V::get(h[k], e), a.root * a.root, s);
        mean = team_sum<TPR>(s, red[0]) * a.per;
    }
    float q = 0.f;
    const float level = -mean * a.root;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const int n = a.cols - (k * TPR + lane) * V::kN;
#pragma unroll
        for (int e = 0; e < V::kN; ++e) {
            const float d = fmaf(V::get(h[k], e), a.root, level);   // 2^-k (h - mean), one rounding
            q += e < n ? d * d : 0.f;
        }
    }
    const float var = team_sum<TPR>(q, red[1]) * a.per;
    const float rstd = 1.f / sqrtf(var + a.eps);
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const int i = k * TPR + lane, n = a.cols - i * V::kN;
        if (n <= 0) continue;
        const u32x4 g = a.gain ? take<BF16>(a.gain + i * 16, n) : kZero4;
        const u32x4 b = a.bias ? take<BF16>(a.bias + i * 16, n) : kZero4;
        float o[V::kN];
#pragma unroll
        for (int e = 0; e < V::kN; ++e) {
            const float t = (V::get(h[k], e) - mean) * rstd;
            o[e] = fmaf(t, a.gain ? V::get(g, e) : 1.f, V::get(b, e));
        }
        if (h_out) V::put(h_out + i * 16, h[k], n);
        V::store(y + i * 16, o, n);
    }
    if (lane == 0) {
        if (a.mean) a.mean[row] = mean;
        if (a.rstd) a.rstd[row] = rstd;
    }
}

// -avg(c xh) from avg(c (h - mean)).  A row beyond the range of its statistics (rstd 0) may have any sum, and has none here.
__device__ __forceinline__ float mean_along(float avg, float rstd) { return rstd == 0.f ? 0.f : -avg * rstd; }

// A team's share of one row.
template <int NV>
struct RowPart {
    u32x4 h[NV], dy[NV];
    float mean, rstd;
    bool live;
};

template <bool BF16, int TPR, int NV, bool CENTER, bool STREAM>
__global__ __launch_bounds__(TPR < 512 ? 512 : TPR) void k_norm_bwd(BwdArgs a) {
    using V = Vec<BF16>;
    constexpr int kTh = TPR < 512 ? 512 : TPR, kTeams = kTh / TPR, kEs = BF16 ? 2 : 4;
    constexpr int kCols = TPR * NV * V::kN;
    // What registers are kept for: up to 24 columns of a thread, the next row and the gain in fp32; from 32 on the gain waits
    // in LDS, base is not loaded ahead, and the packed row is unpacked again for dx; a workgroup of 1024 threads loads no row
    // ahead.
    constexpr bool kAhead = TPR < 1024, kTight = NV * V::kN >= 32 || TPR == 1024;
    __shared__ u32x4 gains[kTight ? NV * TPR : 1];
    __shared__ float red[2][2][kTh / 64];          // by parity of the row, sum, wave
    __shared__ __attribute__((aligned(16))) float joined[kTeams > 1 ? kTeams * kCols : 4];
    const int lane = static_cast<int>(threadIdx.x) % TPR, team = static_cast<int>(threadIdx.x) / TPR;
    const int64_t stride = static_cast<int64_t>(gridDim.x) * kTeams;
    const float per = 1.f / static_cast<float>(a.cols);
    float gain[kTight ? 1 : NV][V::kN];
    float dg[NV][V::kN] = {}, db[NV][V::kN] = {};
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const int i = k * TPR + lane;
        const float ones[8] = {1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f};
        const u32x4 v = a.gain ? take<BF16>(a.gain + i * 16, a.cols - i * V::kN) : V::pack(ones);
        if constexpr (kTight) {
            gains[i] = v;   // (read by this thread alone: the teams of such rows are whole workgroups)
        } else {
#pragma unroll
            for (int e = 0; e < V::kN; ++e) gain[k][e] = V::get(v, e);
        }
    }
    const auto gain_of = [&](int k, float (&g)[V::kN]) {
        u32x4 v = kZero4;
        if constexpr (kTight) v = gains[k * TPR + lane];
#pragma unroll
        for (int e = 0; e < V::kN; ++e) g[e] = kTight ? V::get(v, e) : gain[kTight ? 0 : k][e];
    };
    const auto load = [&](int64_t row, RowPart<NV> &p) {
        p.live = row < a.rows && (!a.mask || a.mask[row] != 0);
        p.mean = CENTER && p.live ? a.mean[row] : 0.f;
        p.rstd = p.live ? a.rstd[row] : 0.f;
        const int width = p.live ? a.cols : 0;
        const bool inner = row + 1 < a.rows;
        take_row<BF16, TPR, NV, STREAM>(a.h + row * a.ld_h * kEs, lane, width, inner, p.h);
        take_row<BF16, TPR, NV, STREAM>(a.dy + row * a.ld_dy * kEs, lane, width, inner, p.dy);
    };
    u32x4 base[NV], next_base[NV];
    const auto load_base = [&](int64_t row, u32x4 (&to)[NV]) {
        const int width = row < a.rows && a.base ? a.cols : 0;
        const bool inner = row + 1 < a.rows;
        take_row<BF16, TPR, NV, STREAM>(a.base + row * a.ld_b * kEs, lane, width, inner, to);
    };
    const int64_t rounds = (a.rows + stride - 1) / stride;   // the same for the whole workgroup: there are barriers inside
    int64_t row = static_cast<int64_t>(blockIdx.x) * kTeams + team;
    RowPart<NV> cur, next;
    if (kAhead) load(row, cur);
    if (!kTight) load_base(row, base);
    for (int64_t it = 0; it < rounds; ++it, row += stride) {
        if (!kAhead) load(row, cur);
        if (kTight) load_base(row, base);
        if (it + 1 < rounds) {
            if (kAhead) load(row + stride, next);
            if (!kTight) load_base(row + stride, next_base);
        }
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int n = a.cols - (k * TPR + lane) * V::kN;
            cur.h[k] = first_of<BF16>(cur.h[k], n);
            cur.dy[k] = first_of<BF16>(cur.dy[k], n);
        }
        float s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            float g[V::kN];
            gain_of(k, g);
#pragma unroll
            for (int e = 0; e < V::kN; ++e) {
                const float dy = V::get(cur.dy[k], e), c = dy * g[e];
                const float d = CENTER ? V::get(cur.h[k], e) - cur.mean : V::get(cur.h[k], e), xh = d * cur.rstd;
                if constexpr (CENTER) {
                    s1 += c;
                    db[k][e] += dy;
                }
                s2 = fmaf(c, d, s2);   // (not xh, which may be infinite behind the row's end, where d is -mean and c 0)
                dg[k][e] = fmaf(dy, xh, dg[k][e]);
                if constexpr (!BF16) cur.h[k][e] = __float_as_uint(xh);   // (fp32: xh in the place of h)
            }
            if constexpr (kTight) asm volatile("" : "+v"(cur.h[k]), "+v"(cur.dy[k]));   // not its fp32 values are kept
        }
        team_sums<TPR, CENTER>(s1, s2, red[it & 1], team);   // (the other half may still be read by a slower wave)
        // dx - base = rstd (c - avg(c) - xh avg(c xh)), as it stands: h - mean under one factor, rstd^3 avg(c (h - mean)), would take
        // a cube that leaves fp32 on both sides.  (A masked row has zeros in all, whose products with a gain that is not finite are
        // dropped.)
        const float level = -(s1 * per), along = mean_along(s2 * per, cur.rstd);
        if (a.dx && row < a.rows) {
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                const int i = k * TPR + lane, n = a.cols - i * V::kN;
                if (n <= 0) continue;
                float o[V::kN], g[V::kN];
                gain_of(k, g);
#pragma unroll
                for (int e = 0; e < V::kN; ++e) {
                    const float c = CENTER ? fmaf(V::get(cur.dy[k], e), g[e], level) : V::get(cur.dy[k], e) * g[e];
                    const float at = V::get(cur.h[k], e), xh = BF16 ? (CENTER ? at - cur.mean : at) * cur.rstd : at;
                    const float to = V::get(base[k], e);
                    o[e] = cur.live ? fmaf(fmaf(xh, along, c), cur.rstd, to) : to;
                }
                V::store(a.dx + row * a.ld_dx * kEs + i * 16, o, n);
            }
        }
        if (kAhead) cur = next;
        if constexpr (!kTight) {
#pragma unroll
            for (int k = 0; k < NV; ++k) base[k] = next_base[k];
        }
    }
    const auto write = [&](float (&sum)[NV][V::kN], float *part) {
        if (!part) return;
        float *to = part + static_cast<int64_t>(blockIdx.x) * padded(a.cols);
        if constexpr (kTeams > 1) {   // the teams' sums, added in order
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int e = 0; e < V::kN; e += 4)
                    *reinterpret_cast<f32x4 *>(joined + team * kCols + (k * TPR + lane) * V::kN + e) =
                        f32x4{sum[k][e], sum[k][e + 1], sum[k][e + 2], sum[k][e + 3]};
            __syncthreads();
            for (int c = static_cast<int>(threadIdx.x); c < a.cols; c += kTh) {
                float t = joined[c];
#pragma unroll
                for (int i = 1; i < kTeams; ++i) t += joined[i * kCols + c];
                to[c] = t;
            }
            __syncthreads();
        } else {
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int e = 0; e < V::kN; ++e) {
                    const int c = (k * TPR + lane) * V::kN + e;
                    if (c < a.cols) to[c] = sum[k][e];
                }
        }
    };
    write(dg, a.part_g);
    if constexpr (CENTER) write(db, a.part_b);
}

// The same for few rows in one launch: the first `column_groups` workgroups sum dgain and dbias of their columns over all rows,
// which needs the statistics but no row's sums, and the others' teams take one row each for dx.  h and dy are read twice, and
// the second launch and its wait are saved.
//
// Threads of a workgroup and vectors of a row (64 or 128 bytes) that it sums.  us of 512 rows with 128 threads and four, 512
// and four, 512 and eight, 1024 and eight: 768 bf16 columns 7.4, 4.3, 5.6, 5.2; 4096 columns 12.0, 7.6, 7.9, 7.2; of 4096 fp32
// columns with 1024 threads and two, four, eight vectors: 26.9, 15.0, 10.5.
constexpr int few_threads(int team) { return team < 512 ? 512 : team; }
constexpr int few_vecs(int team) { return team < 1024 ? 4 : 8; }
template <bool BF16, int TH, int VECS, bool CENTER>
__device__ void sum_columns(const BwdArgs &a, float *dgain, float *dbias, bool accumulate) {
    using V = Vec<BF16>;
    constexpr int kEs = BF16 ? 2 : 4, kSlots = TH / VECS, kAhead = 4, kC = VECS * V::kN, kParts = 8;
    static_assert(TH / kC >= kParts, "a thread for every column and part");
    __shared__ __attribute__((aligned(16))) float sums[kSlots][kC + 4];
    __shared__ float joined[kParts][kC];
    const int tid = static_cast<int>(threadIdx.x), slot = tid / VECS, mine = tid % VECS;
    const int i = static_cast<int>(blockIdx.x) * VECS + mine, n = a.cols - i * V::kN;
    float dg[V::kN] = {}, db[V::kN] = {};
    const auto add = [&](u32x4 h, u32x4 dy, float mean, float rstd, bool live) {   // what a masked row holds is dropped
#pragma unroll
        for (int e = 0; e < V::kN; ++e) {
            const float g = V::get(dy, e), d = CENTER ? V::get(h, e) - mean : V::get(h, e);
            dg[e] = live ? fmaf(g, d * rstd, dg[e]) : dg[e];
            if constexpr (CENTER) db[e] += live ? g : 0.f;
        }
    };
    // A partial vector's load brings what lies between the rows besides, for columns that are not stored; behind the last row
    // nothing may lie.
    const char *h_at = a.h + i * 16, *dy_at = a.dy + i * 16;
    const int last = static_cast<int>(a.rows) - 1, whole = n >= V::kN ? last + 1 : n > 0 ? last : 0;
    for (int first = slot; first < whole; first += kAhead * kSlots) {
        u32x4 h[kAhead], dy[kAhead];
        float mean[kAhead], rstd[kAhead];
        uint8_t mask[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            const int64_t row = first + j * kSlots < whole ? first + j * kSlots : first;
            h[j] = ld128(h_at + row * a.ld_h * kEs);
            dy[j] = ld128(dy_at + row * a.ld_dy * kEs);
            mean[j] = CENTER ? a.mean[row] : 0.f;
            rstd[j] = a.rstd[row];
            mask[j] = a.mask ? a.mask[row] : 1;
        }
#pragma unroll
        for (int j = 0; j < kAhead; ++j) add(h[j], dy[j], mean[j], rstd[j], first + j * kSlots < whole && mask[j] != 0);
    }
    if (n > 0 && n < V::kN && slot == last % kSlots)
        add(take<BF16>(h_at + last * a.ld_h * kEs, n), take<BF16>(dy_at + last * a.ld_dy * kEs, n),
            CENTER ? a.mean[last] : 0.f, a.rstd[last], !a.mask || a.mask[last] != 0);
    const auto write = [&](const float (&sum)[V::kN], float *out) {
        if (!out) return;   // (the same for the whole workgroup)
#pragma unroll
        for (int e = 0; e < V::kN; e += 4)
            *reinterpret_cast<f32x4 *>(&sums[slot][mine * V::kN + e]) = f32x4{sum[e], sum[e + 1], sum[e + 2], sum[e + 3]};
        __syncthreads();
        const int c = tid % kC, part = tid / kC;
        if (part < kParts) {
            float t = 0.f;
#pragma unroll
            for (int k = 0; k < kSlots / kParts; ++k) t += sums[part * (kSlots / kParts) + k][c];
            joined[part][c] = t;
        }
        __syncthreads();
        const int column = static_cast<int>(blockIdx.x) * kC + c;
        if (part == 0 && column < a.cols) {
            float t = joined[0][c];
#pragma unroll
            for (int k = 1; k < kParts; ++k) t += joined[k][c];
            out[column] = accumulate ? out[column] + t : t;
        }
        __syncthreads();   // `sums` and `joined` are used again
    };
    write(dg, dgain);
    if constexpr (CENTER) write(db, dbias);
}

template <bool BF16, int TPR, int NV, bool CENTER>
__global__ __launch_bounds__(few_threads(TPR)) void k_norm_bwd_few(BwdArgs a, float *dgain, float *dbias, bool accumulate,
                                                                   int column_groups) {
    using V = Vec<BF16>;
    constexpr int kTh = few_threads(TPR), kTeams = kTh / TPR, kEs = BF16 ? 2 : 4;
    if (static_cast<int>(blockIdx.x) < column_groups) return sum_columns<BF16, kTh, few_vecs(TPR), CENTER>(a, dgain, dbias, accumulate);
    __shared__ float red[2][kTh / 64];
    const int lane = static_cast<int>(threadIdx.x) % TPR;
    const int64_t row = static_cast<int64_t>(static_cast<int>(blockIdx.x) - column_groups) * kTeams + threadIdx.x / TPR;
    const bool in = row < a.rows, inner = row + 1 < a.rows, live = in && (!a.mask || a.mask[row] != 0);
    const int width = live ? a.cols : 0;
    u32x4 h[NV], dy[NV], base[NV], gain[NV];
    take_row<BF16, TPR, NV, false>(a.h + row * a.ld_h * kEs, lane, width, inner, h);
    take_row<BF16, TPR, NV, false>(a.dy + row * a.ld_dy * kEs, lane, width, inner, dy);
    take_row<BF16, TPR, NV, false>(a.base + row * a.ld_b * kEs, lane, in && a.base ? a.cols : 0, inner, base);
    const float ones[8] = {1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f};
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const int i = k * TPR + lane;
        gain[k] = a.gain ? take<BF16>(a.gain + i * 16, a.cols - i * V::kN) : V::pack(ones);
    }
    const float mean = CENTER && live ? a.mean[row] : 0.f, rstd = live ? a.rstd[row] : 0.f;
    float s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const int n = a.cols - (k * TPR + lane) * V::kN;
        h[k] = first_of<BF16>(h[k], n);
        dy[k] = first_of<BF16>(dy[k], n);
#pragma unroll
        for (int e = 0; e < V::kN; ++e) {
            const float c = V::get(dy[k], e) * V::get(gain[k], e);
            if constexpr (CENTER) s1 += c;
            s2 = fmaf(c, V::get(h[k], e) - mean, s2);
        }
    }
    team_sums<TPR, CENTER>(s1, s2, red, static_cast<int>(threadIdx.x) / TPR);
    const float per = 1.f / static_cast<float>(a.cols);
    const float level = -(s1 * per), along = mean_along(s2 * per, rstd);   // as in k_norm_bwd
    if (!in) return;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const int i = k * TPR + lane, n = a.cols - i * V::kN;
        if (n <= 0) continue;
        float o[V::kN];
#pragma unroll
        for (int e = 0; e < V::kN; ++e) {
            const float g = V::get(gain[k], e), to = V::get(base[k], e);
            const float c = CENTER ? fmaf(V::get(dy[k], e), g, level) : V::get(dy[k], e) * g;
            o[e] = live ? fmaf(fmaf((V::get(h[k], e) - mean) * rstd, along, c), rstd, to) : to;
        }
        V::store(a.dx + row * a.ld_dx * kEs + i * 16, o, n);
    }
}

// dgain and dbias from the workgroups' sums: a workgroup takes 32 columns, eight threads of four for each of 32 ranges of
// the parts; the ranges are added in order.  blockIdx.y: 0 dgain, 1 dbias.  256 parts of 4096 columns: 4.8 us.
__global__ __launch_bounds__(256) void k_norm_parts(const float *part_g, const float *part_b, int parts, int cols,
                                                    float *dgain, float *dbias, bool accumulate) {
    constexpr int kSlots = 32, kAhead = 8;
    __shared__ float sums[kSlots][33];
    const float *part = blockIdx.y ? part_b : part_g;
    float *out = blockIdx.y ? dbias : dgain;
    if (!out) return;
    const int quad = threadIdx.x & 7, slot = threadIdx.x >> 3, ld = padded(cols);
    const int c = static_cast<int>(blockIdx.x) * 32 + quad * 4;
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
    if (c < ld) {   // (the last vector of a row may hold unwritten columns, which are not stored)
        const int each = (parts + kSlots - 1) / kSlots, begin = slot * each, end = begin + each < parts ? begin + each : parts;
        for (int i = begin; i < end; i += kAhead) {
            f32x4 v[kAhead];
#pragma unroll
            for (int j = 0; j < kAhead; ++j)
                v[j] = i + j < end ? *reinterpret_cast<const f32x4 *>(part + static_cast<int64_t>(i + j) * ld + c)
                                   : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int j = 0; j < kAhead; ++j) s += v[j];
        }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) sums[slot][quad * 4 + e] = s[e];
    __syncthreads();
    const int mine = static_cast<int>(blockIdx.x) * 32 + threadIdx.x;
    if (threadIdx.x >= 32 || mine >= cols) return;
    float t = 0.f;
    for (int i = 0; i < kSlots; ++i) t += sums[i][threadIdx.x];
    out[mine] = accumulate ? out[mine] + t : t;
}

template <int N>
using int_c = std::integral_constant<int, N>;

// Calls go(team, vectors a thread), as compile-time constants: the smallest team from 32 to LARGEST threads that holds a
// row of `vectors` in at most MOST vectors a thread.
template <int MOST, int LARGEST, int TEAM = 32, class Go>
void with_team(int vectors, const Go &go) {
    constexpr int kLeast = TEAM == 32 ? 1 : MOST / 2 + 1;   // (fewer, and a smaller team would do)
    if constexpr (TEAM < LARGEST) {
        if (vectors > TEAM * MOST) return with_team<MOST, LARGEST, TEAM * 2>(vectors, go);
    }
    const int nv = (vectors + TEAM - 1) / TEAM;
    if constexpr (kLeast <= 1 && MOST >= 1)
        if (nv <= 1) return go(int_c<TEAM>{}, int_c<1>{});
    if constexpr (kLeast <= 2 && MOST >= 2)
        if (nv <= 2) return go(int_c<TEAM>{}, int_c<2>{});
    if constexpr (kLeast <= 3 && MOST >= 3)
        if (nv <= 3) return go(int_c<TEAM>{}, int_c<3>{});
    if constexpr (MOST >= 4) go(int_c<TEAM>{}, int_c<4>{});
}

// Whether a call's matrices are more than the 256 MB cache holds.  Then the loads are non-temporal, as the stores always are:
// a call reads nothing twice, and lines that it would bring into the cache or change there cost its later loads their room.
// (Measured on the norm alone: what the projection that reads y next would gain by ordinary stores is not in these figures.)
// us of the first launch with and without: 16,384 rows
// of 4096 bf16 columns forward 93 and 96, backward 79 and 83; of 768 columns, 91 and 101 MB and the next call on the same
// memory soon, 20.7 and 16, 21.2 and 19.3.
bool beyond_cache(bool bf16, int64_t rows, int cols, int matrices) {
    return static_cast<double>(rows) * cols * (bf16 ? 2 : 4) * matrices > 256.0 * (1 << 20);
}

int vectors_of(bool bf16, int cols) { return (cols + (bf16 ? 7 : 3)) / (bf16 ? 8 : 4); }

// Workgroups of the backward pass: one on each CU, as many as there are rows for.  us with 160, 256, 512 and 768 (base, no
// mask, bf16): 16,384 rows of 4096 columns 111, 96.5, 98 and 102, 2,400 rows 19.9, 17.6, 21.8 and 24.3, 600 rows 9.8, 10.8,
// 12.9 and 12.9, 16,384 rows of 768 22.8, 20.6, 21.8 and 27.4.
constexpr int kBwdGroups = 256;

// Up to so many rows k_norm_bwd_few takes the backward pass.  us of a pass with it and with k_norm_bwd and k_norm_parts, of
// 16, 512, 1,024 and 2,048 rows: 768 bf16 columns with the mean 3.7 and 8.1, 4.3 and 8.4, 7.6 and 8.6, 13.5 and 9.3; 4096 rms
// 3.3 and 6.7, 7.6 and 9.3, 12.0 and 11.3, 20.6 and 15.7; 14,336 rms 4.5 and 14.5, 16.3 and 26.4, 30.4 and 37.4, 62 and 60.
// A launch less is also 2.6 us less of the host's time, which decides at 1,024 rows of 4096; a captured call, which does not pay
// the host, takes those 0.7 us longer.  Where dx takes the place of h or dy there are two launches.
constexpr int kFewRows = 1024;

}  // namespace

size_t norm_ws_bytes(int64_t rows, int cols) {
    // (a workgroup has at least one row)
    const int64_t groups = rows < kBwdGroups ? rows : kBwdGroups;
    return static_cast<size_t>(groups) * padded(cols) * 2 * sizeof(float);
}

hipError_t launch_norm_forward(const NormForward &n, hipStream_t s) {
    float root = 1.f;
    while (1.f / (root * root) < static_cast<float>(n.cols)) root *= 0.5f;
    FwdArgs a = {static_cast<const char *>(n.x), static_cast<const char *>(n.residual), static_cast<char *>(n.h),
                 static_cast<char *>(n.y), n.ld_x, n.ld_res, n.ld_h, n.ld_y, n.rows, n.mask,
                 static_cast<const char *>(n.gain), static_cast<const char *>(n.bias), n.mean, n.rstd, n.cols, n.eps,
                 root, 1.f / (root * root) / static_cast<float>(n.cols),
                 beyond_cache(n.bf16, n.rows, n.cols, 2 + (n.residual ? 1 : 0) + (n.h ? 1 : 0))};
    const int vec = vectors_of(n.bf16, n.cols);
    const auto go = [&](auto t, auto v) {
        constexpr int T = decltype(t)::value, NV = decltype(v)::value;
        const int teams = T <= 64 ? 256 / T : 1;
        const int64_t groups = (n.rows + teams - 1) / teams;
        const uint32_t gx = static_cast<uint32_t>(groups < (1 << 21) ? groups : (1 << 21));
        const dim3 grid(gx, static_cast<uint32_t>((groups + gx - 1) / gx));
        const int th = T <= 64 ? 256 : T;
        if (n.bf16)
            n.rms ? k_norm_fwd<true, T, NV, false><<<grid, th, 0, s>>>(a) : k_norm_fwd<true, T, NV, true><<<grid, th, 0, s>>>(a);
        else
            n.rms ? k_norm_fwd<false, T, NV, false><<<grid, th, 0, s>>>(a) : k_norm_fwd<false, T, NV, true><<<grid, th, 0, s>>>(a);
    };
    // few rows: one vector a thread, for the shortest way through a row; many: four, for fewer threads that wait
    if (n.rows <= 1024 && vec <= 1024)
        with_team<1, 1024>(vec, go);
    else
        with_team<4, 1024>(vec, go);
    return hipGetLastError();
}

// One launch, or, where dx takes the place of what the columns' sums read, one for these before it.
static hipError_t launch_few(const NormBackward &n, hipStream_t s) {
    const int vec = vectors_of(n.bf16, n.cols);
    const BwdArgs a = {static_cast<const char *>(n.h), static_cast<const char *>(n.dy), static_cast<const char *>(n.base),
                       static_cast<char *>(n.dx), n.ld_h, n.ld_dy, n.ld_base, n.ld_dx, n.rows, n.mask,
                       static_cast<const char *>(n.gain), n.mean, n.rstd, nullptr, nullptr, n.cols};
    const bool sums = n.dgain || n.dbias, apart = sums && n.dx && (n.dx == n.h || n.dx == n.dy);
    const auto launch = [&](auto t, auto v, auto is_bf16) {
        constexpr int T = decltype(t)::value, NV = decltype(v)::value, th = few_threads(T), teams = th / T;
        constexpr bool B = decltype(is_bf16)::value;
        const int rows = n.dx ? (static_cast<int>(n.rows) + teams - 1) / teams : 0;
        const int columns = sums ? (vec + few_vecs(T) - 1) / few_vecs(T) : 0;
        const auto run = [&](int groups, int column_groups) {
            if (n.rms)
                k_norm_bwd_few<B, T, NV, false><<<groups, th, 0, s>>>(a, n.dgain, n.dbias, n.accumulate, column_groups);
            else
                k_norm_bwd_few<B, T, NV, true><<<groups, th, 0, s>>>(a, n.dgain, n.dbias, n.accumulate, column_groups);
        };
        if (apart) {
            run(columns, columns);
            run(rows, 0);
        } else {
            run(columns + rows, columns);
        }
    };
    const auto go = [&](auto t, auto v) { n.bf16 ? launch(t, v, std::true_type{}) : launch(t, v, std::false_type{}); };
    if (vec <= 1024)
        with_team<1, 1024>(vec, go);
    else if (vec <= 2 * 1024)
        go(int_c<1024>{}, int_c<2>{});
    else if (vec <= 3 * 1024)   // (fp32)
        launch(int_c<1024>{}, int_c<3>{}, std::false_type{});
    else
        launch(int_c<1024>{}, int_c<4>{}, std::false_type{});
    return hipGetLastError();
}

hipError_t launch_norm_backward(const NormBackward &n, hipStream_t s) {
    if (n.rows > 0 && n.rows <= kFewRows) return launch_few(n, s);
    const int vec = vectors_of(n.bf16, n.cols);
    int groups = 0;   // (without rows: the gradients' sums are empty)
    float *part_g = nullptr, *part_b = nullptr;
    const auto launch = [&](auto t, auto v, auto is_bf16) {
        constexpr int T = decltype(t)::value, NV = decltype(v)::value;
        constexpr bool B = decltype(is_bf16)::value;
        constexpr int th = T < 512 ? 512 : T, teams = th / T;
        const int64_t g = (n.rows + teams - 1) / teams;
        groups = static_cast<int>(g < kBwdGroups ? g : kBwdGroups);
        part_g = n.dgain ? static_cast<float *>(n.ws) : nullptr;
        part_b = n.dbias ? static_cast<float *>(n.ws) + static_cast<int64_t>(groups) * padded(n.cols) : nullptr;
        const BwdArgs a = {static_cast<const char *>(n.h), static_cast<const char *>(n.dy), static_cast<const char *>(n.base),
                           static_cast<char *>(n.dx), n.ld_h, n.ld_dy, n.ld_base, n.ld_dx, n.rows, n.mask,
                           static_cast<const char *>(n.gain), n.mean, n.rstd, part_g, part_b, n.cols};
        const auto run = [&](auto stream) {
            constexpr bool S = decltype(stream)::value;
            n.rms ? k_norm_bwd<B, T, NV, false, S><<<groups, th, 0, s>>>(a) : k_norm_bwd<B, T, NV, true, S><<<groups, th, 0, s>>>(a);
        };
        if (beyond_cache(n.bf16, n.rows, n.cols, 2 + (n.base ? 1 : 0) + (n.dx ? 1 : 0)))
            run(std::true_type{});
        else
            run(std::false_type{});
    };
    const auto go = [&](auto t, auto v) { n.bf16 ? launch(t, v, std::true_type{}) : launch(t, v, std::false_type{}); };
    if (n.rows > 0) {
        if (vec <= 3 * 512)
            with_team<3, 512>(vec, go);
        else if (vec <= 4 * 512)
            go(int_c<512>{}, int_c<4>{});
        else if (vec <= 3 * 1024)   // (fp32)
            launch(int_c<1024>{}, int_c<3>{}, std::false_type{});
        else
            launch(int_c<1024>{}, int_c<4>{}, std::false_type{});
    }
    if (n.dgain || n.dbias)
        k_norm_parts<<<dim3(static_cast<uint32_t>(n.cols + 31) / 32, n.dbias ? 2 : 1), 256, 0, s>>>(
            part_g, part_b, groups, n.cols, n.dgain, n.dbias, n.accumulate);
    return hipGetLastError();
}

}  // namespace logra
