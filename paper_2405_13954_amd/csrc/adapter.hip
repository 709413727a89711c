// Low-rank adapters of many requests at once, beside a shared projection:
//
//     u_t = A_a drop(x_t)                  y_t  = base_t + s_a B_a^T u_t
//     du_t = s_a B_a dy_t                  dx_t = base_t + drop'(A_a^T du_t)
//     dA_a = sum_t du_t drop(x_t)^T        dB_a = s_a sum_t u_t dy_t^T
//
// for rows t of x whose adapter is a (a row without one: y = base, dx = base),
// A [n][rank][n_in] and B [n][rank][n_out], both with the long index
// contiguous as the projections P_in and P_out of this library are.  So the
// forward and the backward pass are made of the same three products:
//
//   shrink   U[t][r]  = sum_j W_a[r][j] v_t[j]                  (x with A, dy with B)
//   expand   out_t[j] = base_t[j] + sum_r U[t][r] W_a[r][j]     (B, then A)
//   grad     dW_a[r][j] = sum_t U[t][r] v_t[j]                  (dy with u, x with du)
//
// All are bound by memory (2 rank multiply-adds for each element of x or y): the
// design has each product read or write every element of x, dy, base and y once,
// and keeps the weights in L2.  Few rows are bound by latency: each product is
// one launch, shared by the two that can run together.
//
//  0. k_plan_*: groups the rows of a batch by adapter, stably (so that sums run
//     in row order, and reruns give the same bits).  Each group starts at a
//     multiple of 32 in the order, and lists of its tiles of 16 and 32 rows let
//     a workgroup find its rows with one load.  Kernels that get memory which is
//     no plan for their sizes do nothing.
//  1. shrink: a workgroup owns a tile of 16 or 32 rows and a range of the long
//     axis, its four waves taking 128-byte pieces of it in turn; the waves' sums
//     are added through LDS.  Few rows: the axis is split over workgroups, whose
//     parts those that read U add, each kernel in a fixed order of its own (of four
//     parts, expand adds the fourth before the second, grad last, so that dx and dA
//     may see a du that differs in its last bits).  16,384 x 4096 bf16 at rank 16: 31 us
//     (4.3 TB/s) with the dropout of x drawn on the way, by the launch's 2048
//     workgroups, 37 without it, by 512.
//  2. expand: a workgroup owns 16 or 32 rows and a slice of columns; W's slice is
//     put in LDS once, and U as MFMA operands.  A bf16 W takes U as two bf16
//     halves (16 significant bits, so that U's rounding stays far below that of
//     the output); rank 16 then fills the 32-deep contraction of one MFMA exactly.
//     fp32 uses fp32 MFMAs.  16,384 x 4096 bf16 at rank 16: 55-58 us for 268 MB
//     (4.7 TB/s; a copy in the same pieces takes 48).
//  3. grad: a workgroup owns a run of an order's blocks of 32 rows and 256 (or 128)
//     columns; a block goes through LDS, where transposed reads (bf16:
//     ds_read_b64_tr_b16) turn it into operands whose contraction runs over
//     rows.  A bf16 v takes U as three bf16 thirds (24 significant bits: the
//     gradients are fp32, so nothing of u and du may be lost).  k_reduce adds the
//     runs' sums in order.
//  Forward: k_shrink, k_expand.  Backward: k_back_dy (du and dB, both of which
//  read dy), k_back_x (dx and dA), k_reduce: 16,384 rows, 4096 + 4096 columns,
//  rank 16, dropout: 47 + 81-84 + 7 us for the 544 MB that the pass cannot do without.
#include "counter_rng.h"
#include "internal.h"

namespace logra {
namespace {

constexpr int kHeights = 2;          // tile lists of 16 << h rows
constexpr int kSeg = 4096;           // rows of one workgroup of the plan's kernels
constexpr int kPlanMagic = 0x4c6f4164;
// Ranges of the long axis in k_shrink at most, which all that read U add up.  At 4096
// columns of x, those pay as much for eight as k_shrink gains, or more (shrink + expand,
// us: 96 rows of 64 adapters to 14336 columns 5.4 + 9.3, with eight 4.5 + 11.7; 8 rows
// 4.0 + 3.5 and 3.3 + 4.6; 300 rows 5.4 + 4.4 and 4.5 + 5.6; 1,999 rows at rank 64 to
// 1024 columns 10.9 + 6.0 and 11.3 + 7.3; with two, 5.0 + 3.4 for 8 rows).  At 14336 columns
// of x eight would be better (1 row 6.1 + 3.6 and 4.7 + 4.4, 16 rows 9.6 + 3.6 and
// 6.3 + 4.5), and more were not measured.
constexpr int kMaxParts = 4;
constexpr int kPad = 32;             // groups start at multiples of this
static_assert(kMaxAdapters + 1 <= 1024, "the plan's kernels have a thread and an LDS word for each group");
static_assert(kMaxAdapterRank <= 16 * 8, "the products take at most eight blocks of ranks");

struct PlanHead {
    int magic, rows, n;
    int tiles_used[kHeights];        // tiles of the adapters
    int tiles_all[kHeights];         // and of the rows without one, which come last
};
struct Tile {
    int group, p0, count, pad;       // adapter, first place in the order, rows; 16 bytes, one load
};

// The plan's memory: head, row of each place (-1: a pad), tile lists, each
// group's first tile in them, and the segments' counts while it is made.
struct PlanView {
    PlanHead *head;
    int *row_of;
    Tile *tiles[kHeights];
    int *first[kHeights];
    int *start;                      // first place of each group, [n + 2]
    int *hist;
    int rows, n;
};

struct PlanLayout {
    size_t row_of, tiles[kHeights], first[kHeights], start, hist, bytes;
};

inline int64_t plan_places(int64_t rows, int n) {
    const int64_t groups = n + 1 < rows ? n + 1 : rows;
    return (rows + (kPad - 1) * groups + kPad - 1) / kPad * kPad;
}
inline int64_t plan_max_tiles(int64_t rows, int n, int h) {
    return (rows >> (4 + h)) + (n + 1 < rows ? n + 1 : rows);
}

PlanLayout plan_layout(int64_t rows, int n) {
    PlanLayout l;
    size_t at = align256(sizeof(PlanHead));
    const auto take = [&](size_t b) {
        const size_t here = at;
        at += align256(b);
        return here;
    };
    l.row_of = take(static_cast<size_t>(plan_places(rows, n)) * 4);
    for (int h = 0; h < kHeights; ++h)
        l.tiles[h] = take(static_cast<size_t>(plan_max_tiles(rows, n, h)) * sizeof(Tile));
    for (int h = 0; h < kHeights; ++h) l.first[h] = take(static_cast<size_t>(n + 2) * 4);
    l.start = take(static_cast<size_t>(n + 2) * 4);
    l.hist = take(static_cast<size_t>((rows + kSeg - 1) / kSeg) * (n + 1) * 4);
    l.bytes = at;
    return l;
}

PlanView plan_view(void *plan, int64_t rows, int n) {
    const PlanLayout l = plan_layout(rows, n);
    char *p = static_cast<char *>(plan);
    PlanView v;
    v.head = reinterpret_cast<PlanHead *>(p);
    v.row_of = reinterpret_cast<int *>(p + l.row_of);
    for (int h = 0; h < kHeights; ++h) {
        v.tiles[h] = reinterpret_cast<Tile *>(p + l.tiles[h]);
        v.first[h] = reinterpret_cast<int *>(p + l.first[h]);
    }
    v.start = reinterpret_cast<int *>(p + l.start);
    v.hist = reinterpret_cast<int *>(p + l.hist);
    v.rows = static_cast<int>(rows);
    v.n = n;
    return v;
}

// What a kernel needs of a plan: one tile list.
struct TileList {
    const PlanHead *head;
    const Tile *tiles;
    const int *row_of;
    int rows, n, h;
};
TileList tile_list(const PlanView &v, int h) { return {v.head, v.tiles[h], v.row_of, v.rows, v.n, h}; }

__device__ __forceinline__ bool is_plan(const PlanHead *h, int rows, int n) {
    return h->magic == kPlanMagic && h->rows == rows && h->n == n;
}
__device__ __forceinline__ int tile_count(const TileList &l, bool all) {
    if (!is_plan(l.head, l.rows, l.n)) return 0;
    return all ? l.head->tiles_all[l.h] : l.head->tiles_used[l.h];
}

// ------------------------------------------------------------------- plan --
__device__ __forceinline__ int group_of(const int *row_adapter, int row, int n) {
    const int a = row_adapter[row];
    return a >= 0 && a < n ? a : n;
}

// The groups of a thread's rows, `step` apart (all loads together); -1 beyond
// the last row.
template <int N>
__device__ __forceinline__ void groups_of(const int *row_adapter, const PlanView &v, int64_t at, int step,
                                          int (&group)[N]) {
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const int64_t row = at + static_cast<int64_t>(k) * step;
        group[k] = row < v.rows ? group_of(row_adapter, static_cast<int>(row), v.n) : -1;
    }
}

__global__ __launch_bounds__(1024) void k_plan_hist(const int *row_adapter, PlanView v) {
    __shared__ int cnt[1024];
    const int g = threadIdx.x;
    int group[kSeg / 1024];
    groups_of(row_adapter, v, static_cast<int64_t>(blockIdx.x) * kSeg + threadIdx.x, 1024, group);
    cnt[g] = 0;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kSeg / 1024; ++k)
        if (group[k] >= 0) atomicAdd(&cnt[group[k]], 1);
    __syncthreads();
    if (g <= v.n) v.hist[static_cast<int64_t>(blockIdx.x) * (v.n + 1) + g] = cnt[g];
}

// Exclusive sum over the workgroup's 1024 threads; `total` gets the whole sum.
__device__ __forceinline__ int scan1024(int x, int *red, int *total) {
    int v = x;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int o = __shfl_up(v, d);
        if ((threadIdx.x & 63) >= static_cast<unsigned>(d)) v += o;
    }
    if ((threadIdx.x & 63) == 63) red[threadIdx.x >> 6] = v;
    __syncthreads();
    int before = 0, all = 0;
    for (int w = 0; w < 16; ++w) {
        if (w < static_cast<int>(threadIdx.x >> 6)) before += red[w];
        all += red[w];
    }
    __syncthreads();
    *total = all;
    return before + v - x;
}

// One thread per group: starts, tile lists, and the segments' counts turned
// into the segments' first places within the group, one segment after the other:
// 5-6 us up to 16,384 rows of some adapters (16 with 1,023), 20 us for 2^18 rows, 68 for
// 2^20, 1.1 ms for 2^24 (2.2 with 1,023 adapters).
__global__ __launch_bounds__(1024) void k_plan_scan(PlanView v, int segs) {
    __shared__ int red[16], lds_first[1025], lds_start[1024], lds_count[1024];
    const int g = threadIdx.x, groups = v.n + 1;
    int count = 0;
    if (g < groups)
        for (int s = 0; s < segs; ++s) {
            int *p = &v.hist[static_cast<int64_t>(s) * groups + g];
            const int c = *p;
            *p = count;
            count += c;
        }
    int total;
    const int start = scan1024((count + kPad - 1) / kPad * kPad, red, &total);
    lds_start[g] = start;
    lds_count[g] = count;
    if (g < groups) {
        v.start[g] = start;
        for (int i = start + count; i < start + (count + kPad - 1) / kPad * kPad; ++i) v.row_of[i] = -1;
    }
    if (g == 0) {
        v.start[groups] = total;
        v.head->magic = kPlanMagic;
        v.head->rows = v.rows;
        v.head->n = v.n;
    }
    for (int h = 0; h < kHeights; ++h) {
        const int height = 16 << h;
        const int first = scan1024((count + height - 1) / height, red, &total);
        lds_first[g] = first;
        if (g < groups) v.first[h][g] = first;
        if (g == v.n) v.head->tiles_used[h] = first;
        if (g == 0) {
            lds_first[1024] = total;
            v.first[h][groups] = total;
            v.head->tiles_all[h] = total;
        }
        __syncthreads();
        for (int t = g; t < total; t += 1024) {
            int lo = 0, hi = groups;   // the last group whose first tile is at or before t
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (lds_first[mid] <= t)
                    lo = mid;
                else
                    hi = mid;
            }
            const int i = t - lds_first[lo], left = lds_count[lo] - i * height;
            v.tiles[h][t] = {lo, lds_start[lo] + i * height, left < height ? left : height, 0};
        }
        __syncthreads();
    }
}

// The wave's lanes with a row of the same group: two groups differ in a bit.
__device__ __forceinline__ uint64_t lanes_alike(int group, uint64_t live, int n) {
    uint64_t same = live;
    for (int bit = 1; bit <= n; bit <<= 1) {
        const uint64_t set = __ballot((group & bit) != 0);
        same &= group & bit ? set : ~set;
    }
    return same;
}

// Places of the rows: each of the 16 waves takes 256 consecutive rows, 64 at a
// time; lanes of one group are ranked by their lane numbers, so a group's rows
// keep their order.  Bound by latency (96 rows of 64 adapters 2.8 us; with a turn
// for each group of the 64 rows, 18).
__global__ __launch_bounds__(1024) void k_plan_scatter(const int *row_adapter, PlanView v) {
    constexpr int kIter = kSeg / 1024;
    __shared__ int next[16][1024];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, g = threadIdx.x;
    const int64_t at = static_cast<int64_t>(blockIdx.x) * kSeg + wave * (kSeg / 16) + lane;
    int group[kIter];
    uint64_t same[kIter] = {};
    groups_of(row_adapter, v, at, 64, group);
    const int before = g <= v.n ? v.start[g] + v.hist[static_cast<int64_t>(blockIdx.x) * (v.n + 1) + g] : 0;
    if (g <= v.n)
        for (int w = 0; w < 16; ++w) next[w][g] = 0;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kIter; ++k) {
        const uint64_t live = __ballot(group[k] >= 0);
        if (!live) break;
        same[k] = lanes_alike(group[k], live, v.n);
        if (group[k] >= 0) atomicAdd(&next[wave][group[k]], 1);
    }
    __syncthreads();
    if (g <= v.n) {
        int p = before;
        for (int w = 0; w < 16; ++w) {
            const int c = next[w][g];
            next[w][g] = p;
            p += c;
        }
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kIter; ++k) {
        volatile int *slot = &next[wave][group[k] < 0 ? 0 : group[k]];
        const int p = *slot, rank = __popcll(same[k] & ((uint64_t{1} << lane) - 1));
        __builtin_amdgcn_wave_barrier();   // every lane has read its group's place
        if (group[k] >= 0) {
            v.row_of[p + rank] = static_cast<int>(at + 64 * k);
            if (rank == 0) *slot = p + __popcll(same[k]);
        }
        __builtin_amdgcn_wave_barrier();
    }
}

// Memory and matrix operands want different lanes.  An operand or result of a
// 16-row block has row t = l % 16 in lane l, and 16 bytes of column group
// g = l / 16: 64-byte pieces of 16 rows.  Memory streams best in 128-byte pieces
// of 8 rows (read + write at 5.6 TB/s against 4.4 to 4.9 for 64-byte ones).  Two
// neighbouring 64-byte pieces of the block, a and b, and the 128-byte pieces of
// its rows 0-7 and 8-15 are turned into each other by one exchange between lanes
// l and l ^ 8.
__device__ __forceinline__ void swap8(u32x4 &a, u32x4 &b) {
    const bool low = (threadIdx.x & 8) == 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const uint32_t send = low ? b[e] : a[e];
        const uint32_t got = static_cast<uint32_t>(
            __builtin_amdgcn_mov_dpp(static_cast<int>(send), 0x128 /* rotate 16 lanes by 8 */, 0xf, 0xf, false));
        if (low)
            b[e] = got;
        else
            a[e] = got;
    }
}
// The lane's place in such a pair: row of the first piece (the second's is 8
// more) and its 16-byte column within the 128 bytes.
__device__ __forceinline__ int pair_row() { return threadIdx.x & 7; }
__device__ __forceinline__ int pair_col() { return ((threadIdx.x >> 3) & 1) * 4 + ((threadIdx.x >> 4) & 3); }

// Grids are lists of blocks in which the tiles are the slow index, so that
// workgroups that run together work on the same rows (4.4 TB/s with the rows as
// the fast one); beyond 2^22 blocks a list goes on in y.
__device__ __forceinline__ uint32_t block_index() { return blockIdx.x + gridDim.x * blockIdx.y; }
inline dim3 block_grid(int64_t blocks) {
    const int64_t x = blocks < (1 << 22) ? blocks : (1 << 22);
    return dim3(static_cast<unsigned>(x), static_cast<unsigned>((blocks + x - 1) / x));
}

__device__ __forceinline__ u32x4 zeros() { return u32x4{0, 0, 0, 0}; }
__device__ __forceinline__ f32x4 zeros4() { return f32x4{0.f, 0.f, 0.f, 0.f}; }
__device__ __forceinline__ f32x4 ldf4(const void *p) { return *reinterpret_cast<const f32x4 *>(p); }
__device__ __forceinline__ float ldf(const void *p) { return *reinterpret_cast<const float *>(p); }
__device__ __forceinline__ void stf4(void *p, f32x4 v) { *reinterpret_cast<f32x4 *>(p) = v; }
__device__ __forceinline__ void st128(void *p, u32x4 v) { *reinterpret_cast<u32x4 *>(p) = v; }
__device__ __forceinline__ void st128_nt(void *p, u32x4 v) {
    __builtin_nontemporal_store(v, reinterpret_cast<u32x4 *>(p));
}

// ----------------------------------------------------------------- shrink --
template <bool BF16>
constexpr int kEs = BF16 ? 2 : 4;
template <bool BF16>
constexpr int kVec = BF16 ? 8 : 4;        // elements in 16 bytes

// One 16-byte piece of both operands: contraction elements 8 (l / 16) .. + 7
// (bf16) or 4 (l / 16) .. + 3 (fp32, one MFMA for each).
template <bool BF16>
__device__ __forceinline__ f32x4 mfma_piece(u32x4 a, u32x4 b, f32x4 c) {
    if constexpr (BF16) return mfma16_bf16(as_bf16x8(a), as_bf16x8(b), c);
    const f32x4 fa = as_f32x4(a), fb = as_f32x4(b);
#pragma unroll
    for (int e = 0; e < 4; ++e) c = mfma16_f32(fa[e], fb[e], c);
    return c;
}

template <bool BF16>
__device__ __forceinline__ u32x4 drop_piece(const DropArgs &d, u32x4 v, uint32_t row, int col) {
    if constexpr (BF16) return drop8_bf16(d, v, row, static_cast<uint32_t>(col) >> 3);
    return drop4_f32(d, v, row, static_cast<uint32_t>(col));
}

struct ShrinkArgs {
    const char *v;
    int64_t ld;
    int width;
    const char *W;
    int rank;
    float *part;              // [splits][places][16 RT]
    int64_t places;
    int splits, per_split;
};
template <int M, int RT>
constexpr int kShrinkLds = 4 * 16 * M * 16 * RT * 4;

// Block `index`: tile and range of the long axis; part = the sum over the range
// of W_a[r][j] drop(v_t[j]).
template <bool BF16, int M, int RT, bool DROP>
__device__ __forceinline__ void shrink(const TileList &list, const ShrinkArgs &a, const DropArgs &d, uint32_t index,
                                       char *lds) {
    constexpr int kRp = 16 * RT, kUnit = 8 * kVec<BF16>;   // 128 bytes of a row
    float(*red)[16 * M][kRp] = reinterpret_cast<float(*)[16 * M][kRp]>(lds);
    const int at = index / a.splits, split = index - at * a.splits;
    if (at >= tile_count(list, false)) return;
    const Tile tile = list.tiles[at];
    const char *v = a.v, *W = a.W;
    const int64_t ld = a.ld;
    const int width = a.width, rank = a.rank;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, t = lane & 15, g = lane >> 4;
    const int begin = split * a.per_split;
    const int end = width - begin < a.per_split ? width : begin + a.per_split;

    // rows of the two 128-byte pieces of each 16-row block
    int row[M][2];
    const char *vp[M][2];
    const char *wp[RT];
#pragma unroll
    for (int m = 0; m < M; ++m)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int i = 16 * m + 8 * h + pair_row();
            row[m][h] = list.row_of[tile.p0 + (i < tile.count ? i : 0)];
            vp[m][h] = v + row[m][h] * ld * kEs<BF16> + 16 * pair_col();
        }
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        const int i = 16 * r + t;
        wp[r] = W + (static_cast<int64_t>(tile.group) * rank + (i < rank ? i : rank - 1)) * width * kEs<BF16> + 16 * g;
    }
    f32x4 acc[M][RT];
#pragma unroll
    for (int m = 0; m < M; ++m)
#pragma unroll
        for (int r = 0; r < RT; ++r) acc[m][r] = zeros4();

    struct Piece {
        u32x4 x[2][M], w[2][RT];
    };
    // the 128-byte piece at column j; `whole`: it ends inside the row
    const auto load = [&](Piece &p, int j, bool whole) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int64_t off = static_cast<int64_t>(j) * kEs<BF16>;
            const bool in_x = whole || j + pair_col() * kVec<BF16> < end;
            const bool in_w = whole || j + (4 * h + g) * kVec<BF16> < end;
#pragma unroll
            for (int m = 0; m < M; ++m) p.x[h][m] = in_x ? ld128_nt(vp[m][h] + off) : zeros();
#pragma unroll
            for (int r = 0; r < RT; ++r) p.w[h][r] = in_w ? ld128(wp[r] + off + 64 * h) : zeros();
        }
    };
    const auto multiply = [&](Piece &p, int j) {
#pragma unroll
        for (int m = 0; m < M; ++m) {
            if constexpr (DROP) {
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    p.x[h][m] = drop_piece<BF16>(d, p.x[h][m], static_cast<uint32_t>(row[m][h]),
                                                 j + pair_col() * kVec<BF16>);
            }
            swap8(p.x[0][m], p.x[1][m]);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int m = 0; m < M; ++m)
#pragma unroll
                for (int r = 0; r < RT; ++r) acc[m][r] = mfma_piece<BF16>(p.w[h][r], p.x[h][m], acc[m][r]);
        }
    };
    int j = begin + wave * kUnit;
    if (j + kUnit <= end) {
        Piece now;
        load(now, j, true);
        for (; j + 5 * kUnit <= end; j += 4 * kUnit) {   // the next piece is on its way while this one is multiplied
            Piece next;
            load(next, j + 4 * kUnit, true);
            multiply(now, j);
            now = next;
        }
        multiply(now, j);
        j += 4 * kUnit;
    }
    if (j < end) {
        Piece last;
        load(last, j, false);
        multiply(last, j);
    }

    // lane holds ranks 16 r + 4 g .. + 3 of row 16 m + t
#pragma unroll
    for (int m = 0; m < M; ++m)
#pragma unroll
        for (int r = 0; r < RT; ++r) stf4(&red[wave][16 * m + t][16 * r + 4 * g], acc[m][r]);
    __syncthreads();
    const float f = DROP ? d.scale : 1.f;
    float *out = a.part + (static_cast<int64_t>(split) * a.places + tile.p0) * kRp;
    for (int i = threadIdx.x; i < 16 * M * kRp / 4; i += 256) {
        const int slot = i / (kRp / 4), r = i % (kRp / 4) * 4;
        if (slot >= tile.count) break;
        f32x4 s = ldf4(&red[0][slot][r]);
#pragma unroll
        for (int w = 1; w < 4; ++w) s += ldf4(&red[w][slot][r]);
#pragma unroll
        for (int e = 0; e < 4; ++e) s[e] = r + e < rank ? s[e] * f : 0.f;
        stf4(out + static_cast<int64_t>(slot) * kRp + r, s);
    }
}

template <bool BF16, int M, int RT, bool DROP>
__global__ __launch_bounds__(256) void k_shrink(TileList list, ShrinkArgs a, DropArgs d) {
    __shared__ __align__(16) char lds[kShrinkLds<M, RT>];
    shrink<BF16, M, RT, DROP>(list, a, d, block_index(), lds);
}

// ----------------------------------------------------------------- expand --
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t pack2(float a, float b) {
    return __builtin_bit_cast(uint32_t, bf16x2{static_cast<__bf16>(a), static_cast<__bf16>(b)});
}
// What rounding f to bf16 leaves over (0 beside an infinity or a NaN, which the
// rounded part carries alone).
__device__ __forceinline__ float left_over(float f) {
    const float h = static_cast<float>(static_cast<__bf16>(f));
    return __builtin_isfinite(h) ? f - h : 0.f;
}

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
__device__ __forceinline__ s16x4 read_tr(uint32_t at) {
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(uintptr_t)at);
}

// Columns of one wave in k_expand: as many as keep W's slice within 40 KB of LDS.
template <bool BF16, int RT>
constexpr int kCols = BF16 ? (RT <= 4 ? 64 : 32) : (RT <= 2 ? 64 : RT <= 4 ? 32 : 16);

struct ExpandArgs {
    const float *part;        // [splits][places][16 RT]
    int splits;
    int64_t places;
    const float *scale;       // [n] or null
    const char *W;
    int rank, width;
    const char *base;
    int64_t ld_b;
    char *out;
    int64_t ld_o;
    float *u_out;             // [rows][rank] or null: the sum of the partials, unscaled
    int slices;               // of kSlice columns
};

template <bool BF16, int RT>
constexpr int kSliceCols = 4 * kCols<BF16, RT>;
template <bool BF16, int RT>
constexpr int kWPitch = kSliceCols<BF16, RT> * kEs<BF16> + (BF16 ? 32 : 16);
// A row of U: bf16 upper halves then lower halves, or fp32.
template <int RT>
constexpr int kURow = 64 * RT + 16;
template <bool BF16, int M, int RT>
constexpr int kExpandLds = 16 * RT * kWPitch<BF16, RT> + 16 * M * kURow<RT>;

// Block `index`: tile of 16 M rows and slice of four waves' columns.
template <bool BF16, int M, int RT, bool DROP>
__device__ __forceinline__ void expand(const TileList &list, const ExpandArgs &a, const DropArgs &d, uint32_t index,
                                       char *lds) {
    constexpr int kRp = 16 * RT, kNw = kCols<BF16, RT>, kSlice = kSliceCols<BF16, RT>, kPitch = kWPitch<BF16, RT>;
    constexpr int kV = kVec<BF16>, kUPitch = kURow<RT>;
    char *lds_w = lds, *lds_u = lds + kRp * kPitch;
    const int at = index / a.slices, slice = index - at * a.slices;
    if (at >= tile_count(list, true)) return;
    const Tile tile = list.tiles[at];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, t = lane & 15, g = lane >> 4;
    const int n0 = slice * kSlice;

    if (tile.group == list.n) {   // rows without an adapter
        if (a.u_out && slice == 0)
            for (int i = threadIdx.x; i < tile.count * a.rank; i += 256)
                a.u_out[static_cast<int64_t>(list.row_of[tile.p0 + i / a.rank]) * a.rank + i % a.rank] = 0.f;
        if (a.out == a.base && a.ld_o == a.ld_b) return;
        for (int i = threadIdx.x; i < tile.count * (kSlice / kV); i += 256) {
            const int64_t row = list.row_of[tile.p0 + i / (kSlice / kV)];
            const int col = n0 + i % (kSlice / kV) * kV;
            if (col >= a.width) continue;
            const u32x4 b = a.base ? ld128_nt(a.base + (row * a.ld_b + col) * kEs<BF16>) : zeros();
            st128_nt(a.out + (row * a.ld_o + col) * kEs<BF16>, b);
        }
        return;
    }

    // Loads return in the order in which they are issued: first what the operands are made of (it comes from L2), then
    // the rows' base (from memory), which is on its way while the operands are put together.
    constexpr int kWVecs = kRp * (kSlice / kV) / 256, kItems = (16 * M * kRp / 4 + 255) / 256, kAhead = 3;
    constexpr int kPairs = kNw * kEs<BF16> / 128, kLoads = kPairs ? 2 : 1, kQ = kPairs ? kPairs : 1;
    // 128-byte pieces of 8 rows (64-byte pieces of 16 rows where the wave has only 64 bytes of columns)
    int row[M][kLoads];
#pragma unroll
    for (int m = 0; m < M; ++m)
#pragma unroll
        for (int h = 0; h < kLoads; ++h) {
            const int i = 16 * m + (kPairs ? 8 * h + pair_row() : t);
            row[m][h] = i < tile.count ? list.row_of[tile.p0 + i] : -1;
        }
    u32x4 w[kWVecs];      // W's slice, zeros beyond the rank and the width
#pragma unroll
    for (int k = 0; k < kWVecs; ++k) {
        const int i = threadIdx.x + 256 * k, r = i / (kSlice / kV), c = i % (kSlice / kV) * kV;
        const bool in = r < a.rank && n0 + c < a.width;
        w[k] = in ? ld128(a.W + ((static_cast<int64_t>(tile.group) * a.rank + r) * a.width + n0 + c) * kEs<BF16>)
                  : zeros();
    }
    // Four ranks of a row, of each split; the fourth split is added at once, and not kept for later (15.2 us, with all
    // kept 15.8, for 96 rows of 64 adapters).
    f32x4 u[kItems][kAhead];
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
        const int i = threadIdx.x + 256 * k, slot = i / (kRp / 4), r = i % (kRp / 4) * 4;
        const float *up = a.part + (static_cast<int64_t>(tile.p0) + slot) * kRp + r;
#pragma unroll
        for (int c = 0; c < kAhead; ++c)
            u[k][c] = slot < tile.count && c < a.splits ? ldf4(up + c * a.places * kRp)
                                                        : zeros4();
        for (int c = kAhead; c < a.splits; ++c)
            if (slot < tile.count) u[k][0] += ldf4(up + c * a.places * kRp);
    }
    const float s = a.scale ? a.scale[tile.group] : 1.f;
    const int w0 = n0 + wave * kNw, col0 = w0 + (kPairs ? pair_col() : g) * kV;
    u32x4 base[M][kQ][kLoads];
#pragma unroll
    for (int m = 0; m < M; ++m)
#pragma unroll
        for (int h = 0; h < kLoads; ++h)
#pragma unroll
            for (int q = 0; q < kQ; ++q) {
                const int col = col0 + 8 * q * kV;
                base[m][q][h] = a.base && row[m][h] >= 0 && col < a.width
                                    ? ld128_nt(a.base + (row[m][h] * a.ld_b + col) * kEs<BF16>)
                                    : zeros();
            }

#pragma unroll
    for (int k = 0; k < kWVecs; ++k) {
        const int i = threadIdx.x + 256 * k, r = i / (kSlice / kV), c = i % (kSlice / kV) * kV;
        st128(lds_w + r * kPitch + c * kEs<BF16>, w[k]);
    }
    // U: the splits' sums, scaled, as operands
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
        const int i = threadIdx.x + 256 * k, slot = i / (kRp / 4), r = i % (kRp / 4) * 4;
        if (slot >= tile.count) break;
        f32x4 v = u[k][0];
#pragma unroll
        for (int c = 1; c < kAhead; ++c) v += u[k][c];
        if (a.u_out && slice == 0) {
            float *o = a.u_out + static_cast<int64_t>(list.row_of[tile.p0 + slot]) * a.rank + r;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (r + e < a.rank) o[e] = v[e];
        }
        v *= s;
        if constexpr (BF16) {
            uint32_t *o = reinterpret_cast<uint32_t *>(lds_u + slot * kUPitch + 2 * r);
            o[0] = pack2(v[0], v[1]);
            o[1] = pack2(v[2], v[3]);
            o[kRp / 2] = pack2(left_over(v[0]), left_over(v[1]));
            o[kRp / 2 + 1] = pack2(left_over(v[2]), left_over(v[3]));
        } else {
            stf4(lds_u + slot * kUPitch + 4 * r, v);
        }
    }
    __syncthreads();

    // MFMA operands from W.  bf16: lane i of the 16 holds the column whose result row is i; result rows 4 g .. + 3
    // of an even and the next odd block are columns 8 g .. + 3 and 8 g + 4 .. + 7 of a 32-column piece, so that a
    // lane ends up with eight neighbouring columns.  Contraction: lanes g = 0, 1 ranks 0-7 and 8-15 with U's upper
    // half, g = 2, 3 the same ranks with its lower half.
    constexpr int kBlocks = kNw / 16;
    u32x4 wf[BF16 ? kBlocks : 1][RT];
    if constexpr (BF16) {
        const uint32_t l0 = lds_addr(lds_w) + static_cast<uint32_t>(wave * kNw * 2);
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                const uint32_t p = l0 + static_cast<uint32_t>((16 * r + 8 * (g & 1) + (t >> 2)) * kPitch +
                                                              (32 * (b >> 1) + 8 * (t & 3) + 4 * (b & 1)) * 2);
                const s16x4 v8[2] = {read_tr(p), read_tr(p + 4 * kPitch)};
                wf[b][r] = __builtin_bit_cast(u32x4, v8);
            }
    }
#pragma unroll
    for (int m = 0; m < M; ++m) {
        if (16 * m >= tile.count) break;
        f32x4 acc[kBlocks];
#pragma unroll
        for (int b = 0; b < kBlocks; ++b) acc[b] = zeros4();
        const char *lu = lds_u + (16 * m + t) * kUPitch;
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            if constexpr (BF16) {
                const u32x4 uf = *reinterpret_cast<const u32x4 *>(lu + (g >> 1) * 2 * kRp + (16 * r + 8 * (g & 1)) * 2);
#pragma unroll
                for (int b = 0; b < kBlocks; ++b) acc[b] = mfma16_bf16(as_bf16x8(wf[b][r]), as_bf16x8(uf), acc[b]);
            } else {
                const f32x4 uf = ldf4(lu + (16 * r + 4 * g) * 4);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const char *lw = lds_w + (16 * r + 4 * g + e) * kPitch + (wave * kNw + t) * 4;
#pragma unroll
                    for (int b = 0; b < kBlocks; ++b)
                        acc[b] = mfma16_f32(ldf(lw + 64 * b), uf[e], acc[b]);
                }
            }
        }
        // block row t, 64-byte piece q: the lane's kV columns at w0 + (4 q + g) kV
        const int own = DROP && 16 * m + t < tile.count ? list.row_of[tile.p0 + 16 * m + t] : 0;
        const auto finish = [&](int q, u32x4 b) {
            float y[kV];
#pragma unroll
            for (int e = 0; e < kV; ++e) y[e] = BF16 ? acc[2 * q + (e >> 2)][e & 3] : acc[q][e];
            if constexpr (DROP) {
                const int col = w0 + (4 * q + g) * kV;
                const u32x4 w = drop_bits(d, static_cast<uint32_t>(own), static_cast<uint32_t>(col) >> 3);
#pragma unroll
                for (int e = 0; e < kV; ++e) {
                    uint32_t word;
                    if constexpr (BF16)
                        word = w[e >> 1];
                    else
                        word = (col & 4) ? w[2 + (e >> 1)] : w[e >> 1];
                    y[e] = ((word >> (16 * (e & 1))) & 0xFFFFu) >= d.thr ? y[e] * d.scale : 0.f;
                }
            }
            u32x4 o;
            if constexpr (BF16) {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    o[e] = pack2(y[2 * e] + __uint_as_float(b[e] << 16),
                                 y[2 * e + 1] + __uint_as_float(b[e] & 0xFFFF0000u));
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) o[e] = __float_as_uint(y[e] + __uint_as_float(b[e]));
            }
            return o;
        };
#pragma unroll
        for (int q = 0; q < kQ; ++q) {
            u32x4 o[2];
            if constexpr (kPairs > 0) {
                swap8(base[m][q][0], base[m][q][1]);
                o[0] = finish(2 * q, base[m][q][0]);
                o[1] = finish(2 * q + 1, base[m][q][1]);
                swap8(o[0], o[1]);
            } else {
                o[0] = finish(0, base[m][0][0]);
            }
            const int col = col0 + 8 * q * kV;
#pragma unroll
            for (int h = 0; h < kLoads; ++h)
                if (row[m][h] >= 0 && col < a.width)
                    st128_nt(a.out + (row[m][h] * a.ld_o + col) * kEs<BF16>, o[h]);
        }
    }
}

template <bool BF16, int M, int RT, bool DROP>
__global__ __launch_bounds__(256) void k_expand(TileList list, ExpandArgs a, DropArgs d) {
    __shared__ __align__(16) char lds[kExpandLds<BF16, M, RT>];
    expand<BF16, M, RT, DROP>(list, a, d, block_index(), lds);
}

// ------------------------------------------------------------------- grad --
// The blocks of 32 places (the tile list of 32 rows) are shared evenly among the
// workgroups of a column slice: run i of n has the blocks from T i / n on.  A run
// may pass from one adapter to the next; each (run, adapter) pair that meets is a
// part of the adapter's sum.  Runs and adapters both only increase, so run +
// adapter numbers the parts, an adapter's parts one after the other.  No run is
// empty: there are at most as many as blocks.
constexpr uint32_t kMaxRuns = 1024;
static_assert((kMaxAdapterRows / 32 + kMaxAdapters) * kMaxRuns <= UINT32_MAX, "products of blocks and runs fit 32 bits");
__device__ __forceinline__ uint32_t run_begin(uint32_t blocks, uint32_t i, uint32_t n) { return blocks * i / n; }
__device__ __forceinline__ uint32_t run_of(uint32_t blocks, uint32_t j, uint32_t n) {
    return ((j + 1) * n - 1) / blocks;
}

struct GradArgs {
    const char *v;            // rows x or dy
    int64_t ld;
    int width, slices;        // of grad_cols columns and grad_tiles blocks of ranks
    const float *U;           // splits = 0: u [rows][rank]; else du in parts [splits][places][rp]
    int splits;
    int64_t places;
    int rank;
    float *part;              // [runs + n][rp][width]
    int runs;
};

// A workgroup of the gradient takes as many columns and ranks as the registers of
// two waves on a SIMD hold: 256 columns, or 128 of fp32 from rank 64 on (the
// backward pass of 300 rows of 4096 + 4096 columns at rank 64: 52 us, with 256
// columns 81; 2,048 rows 99 and 114, 8,192 rows 273 and 285), and of rank 128 one
// half, the other half being another workgroup's, which reads the same rows (bf16,
// 300 rows: 67 us, 99 as one; 2,048 rows 98 and 119, 16,384 rows 410 and 416).
__host__ __device__ constexpr int grad_cols(bool bf16, int rt) { return bf16 || rt < 4 ? 256 : 128; }
__host__ __device__ constexpr int grad_tiles(int rt) { return rt == 8 ? rt / 2 : rt; }
template <int RT>
constexpr int kGradTiles = grad_tiles(RT);
template <bool BF16, int RT>
constexpr int kGradCols = grad_cols(BF16, RT);

// Parts of du that are fetched one by one, and so the splits of the backward
// pass's k_shrink.
__host__ __device__ constexpr int parts_of(int rt) { return rt == 1 ? kMaxParts : 2; }
template <int RT>
constexpr int kParts = parts_of(RT);
constexpr int kGradChunk = 32;   // blocks whose rows are looked up together
template <bool BF16, int RT>
constexpr int kVPitch = kGradCols<BF16, RT> * kEs<BF16> + 32;
template <bool BF16, int RT>
constexpr int kULds = BF16 ? 3 * 16 * RT * 80 : 32 * (64 * RT + 16);
template <bool BF16, int RT>
constexpr int kGradLds = 32 * kVPitch<BF16, RT> + kULds<BF16, kGradTiles<RT>> + kGradChunk * (32 * 4 + 16);

// Block `index`: run, range of ranks and slice of grad_cols columns of v.
template <bool BF16, int ALL, bool DROP>
__device__ __forceinline__ void grad(const TileList &list, const GradArgs &a, const DropArgs &d, uint32_t index,
                                     char *lds) {
    constexpr int RT = kGradTiles<ALL>, kRanges = ALL / RT, kAll = 16 * ALL;   // blocks of ranks: here, in all
    constexpr int kRp = 16 * RT, kV = kVec<BF16>, kPitch = kVPitch<BF16, ALL>;
    constexpr int kNc = kGradCols<BF16, ALL>, kNw = kNc / 4, kBlocks = kNw / 16;   // columns: all, of a wave; its MFMAs
    constexpr int kLoads = 32 * (kNc / kV) / 256;      // 16-byte loads of a thread for 32 rows
    constexpr int kRowsPer = 32 / kLoads;                    // rows that the workgroup loads at once
    // U of 32 places.  bf16: [third][rank][place]; fp32: [place][rank]
    constexpr int kUPitch = BF16 ? 80 : 4 * kRp + 16, kUThird = kRp * kUPitch, kChunk = kGradChunk;
    char *lds_v = lds, *lds_u = lds + 32 * kPitch;
    int *lds_row = reinterpret_cast<int *>(lds_u + kULds<BF16, RT>);
    Tile *lds_tile = reinterpret_cast<Tile *>(lds_row + 32 * kChunk);
    const uint32_t blocks = tile_count(list, false), runs = blocks < static_cast<uint32_t>(a.runs) ? blocks : a.runs;
    const uint32_t run = index / a.slices, slice = index - run * a.slices;
    if (run >= runs) return;
    const int range = kRanges > 1 ? static_cast<int>(slice) * kRanges / a.slices : 0, r0 = range * kRp;
    const int n0 = (static_cast<int>(slice) - range * (a.slices / kRanges)) * kNc;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, t = lane & 15, g = lane >> 4;
    const int end = run_begin(blocks, run + 1, runs);

    const int lr = threadIdx.x / (kNc / kV), lc = threadIdx.x % (kNc / kV) * kV;
    const bool in = n0 + lc < a.width;
    const int ur = threadIdx.x & 15, up = threadIdx.x >> 4;   // rank within 16 and pair of places that the thread loads
    // The next block is on its way while one is multiplied (two ahead measured the same).  Every lane loads: for a pad,
    // and beyond the rank or the width, something of the block's first row or the first column, which is put aside when
    // it is used.
    struct Fetch {
        float u[kParts<RT>][RT][2];
        u32x4 v[kLoads];
    } ahead;
    const int64_t col_bytes = static_cast<int64_t>(in ? n0 + lc : 0) * kEs<BF16>;
    const auto load = [&](Fetch &f, int i) {   // U first: it comes from L2, and loads return in order
        const int first = lds_row[32 * i];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int row = lds_row[32 * i + 2 * up + e];
            const int64_t place = static_cast<int64_t>(lds_tile[i].p0) + (row < 0 ? 0 : 2 * up + e);
            const float *q = a.splits ? a.U + place * kAll + r0 + ur
                                      : a.U + static_cast<int64_t>(row < 0 ? first : row) * a.rank;
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                const int k = r0 + 16 * r + ur, known = k < a.rank ? k : 0;
                f.u[0][r][e] = a.splits ? q[16 * r] : q[known];
#pragma unroll
                for (int c = 1; c < kParts<RT>; ++c) {
                    f.u[c][r][e] = 0.f;
                    if (a.splits > c) f.u[c][r][e] = q[16 * r + c * a.places * kAll];
                }
            }
        }
#pragma unroll
        for (int k = 0; k < kLoads; ++k) {
            const int row = lds_row[32 * i + kRowsPer * k + lr];
            f.v[k] = ld128_nt(a.v + (row < 0 ? first : row) * a.ld * kEs<BF16> + col_bytes);
        }
    };
    f32x4 acc[kBlocks][RT];
    const auto clear = [&] {
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
            for (int r = 0; r < RT; ++r) acc[b][r] = zeros4();
    };
    // lane holds columns 4 g .. + 3 of block b for rank 16 r + t
    const auto flush = [&](int group) {
        float *out = a.part + ((static_cast<int64_t>(run) + group) * kAll + r0) * a.width;
#pragma unroll
        for (int b = 0; b < kBlocks; ++b) {
            const int col = n0 + wave * kNw + 16 * b + 4 * g;
            if (col >= a.width) continue;
#pragma unroll
            for (int r = 0; r < RT; ++r)
                stf4(out + static_cast<int64_t>(16 * r + t) * a.width + col, acc[b][r]);
        }
    };
    clear();
    int group = -1;
    for (int chunk = run_begin(blocks, run, runs); chunk < end; chunk += kChunk) {
        const int count = end - chunk < kChunk ? end - chunk : kChunk;
        __syncthreads();
        if (static_cast<int>(threadIdx.x) < count) lds_tile[threadIdx.x] = list.tiles[chunk + threadIdx.x];
        __syncthreads();
        for (int i = threadIdx.x; i < count * 32; i += 256) {
            const Tile tile = lds_tile[i / 32];
            lds_row[i] = i % 32 < tile.count ? list.row_of[tile.p0 + i % 32] : -1;
        }
        __syncthreads();
        const auto step = [&](Fetch &f, int i) {
            if (lds_tile[i].group != group) {
                if (group >= 0) {
                    flush(group);
                    clear();
                }
                group = lds_tile[i].group;
            }
            if (i) __syncthreads();   // the waves are done with the block before (two in LDS and one barrier: no gain)
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                float q[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    q[e] = f.u[0][r][e];
#pragma unroll
                    for (int c = 1; c < kParts<RT>; ++c) q[e] += f.u[c][r][e];
                    if (lds_row[32 * i + 2 * up + e] < 0 || r0 + 16 * r + ur >= a.rank) q[e] = 0.f;
                }
                if constexpr (BF16) {
#pragma unroll
                    for (int third = 0; third < 3; ++third) {
                        char *to = lds_u + third * kUThird + (16 * r + ur) * kUPitch + 4 * up;
                        *reinterpret_cast<uint32_t *>(to) = pack2(q[0], q[1]);
                        q[0] = left_over(q[0]);
                        q[1] = left_over(q[1]);
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 2; ++e)
                        *reinterpret_cast<float *>(lds_u + (2 * up + e) * kUPitch + (16 * r + ur) * 4) = q[e];
                }
            }
#pragma unroll
            for (int k = 0; k < kLoads; ++k) {
                const int slot = kRowsPer * k + lr, row = lds_row[32 * i + slot];
                if constexpr (DROP) f.v[k] = drop_piece<BF16>(d, f.v[k], static_cast<uint32_t>(row), n0 + lc);
                st128(lds_v + slot * kPitch + lc * kEs<BF16>, in && row >= 0 ? f.v[k] : zeros());
            }
            __syncthreads();
            if (i + 1 < count) load(f, i + 1);
            if constexpr (BF16) {
                u32x4 vf[kBlocks];
                const uint32_t l0 = lds_addr(lds_v) + static_cast<uint32_t>((8 * g + (t >> 2)) * kPitch +
                                                                            (wave * kNw + 4 * (t & 3)) * 2);
#pragma unroll
                for (int b = 0; b < kBlocks; ++b) {
                    const s16x4 v8[2] = {read_tr(l0 + 32 * b), read_tr(l0 + 32 * b + 4 * kPitch)};
                    vf[b] = __builtin_bit_cast(u32x4, v8);
                }
#pragma unroll
                for (int third = 0; third < 3; ++third)
#pragma unroll
                    for (int r = 0; r < RT; ++r) {
                        const u32x4 uf =
                            *reinterpret_cast<const u32x4 *>(lds_u + third * kUThird + (16 * r + t) * kUPitch + 16 * g);
#pragma unroll
                        for (int b = 0; b < kBlocks; ++b)
                            acc[b][r] = mfma16_bf16(as_bf16x8(vf[b]), as_bf16x8(uf), acc[b][r]);
                    }
            } else {
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    float uf[RT];
#pragma unroll
                    for (int r = 0; r < RT; ++r)
                        uf[r] = ldf(lds_u + (4 * k + g) * kUPitch + (16 * r + t) * 4);
#pragma unroll
                    for (int b = 0; b < kBlocks; ++b) {
                        const float vf = ldf(lds_v + (4 * k + g) * kPitch + (wave * kNw + 16 * b + t) * 4);
#pragma unroll
                        for (int r = 0; r < RT; ++r) acc[b][r] = mfma16_f32(vf, uf[r], acc[b][r]);
                    }
                }
            }
        };
        load(ahead, 0);
        for (int i = 0; i < count; ++i) step(ahead, i);
    }
    if (group >= 0) flush(group);
}

// The two launches of the backward pass.  In each, a gradient's blocks come first
// (they are few and long), then those of the product that shares its rows:
// du = B dy beside dB, both of which read dy; then dx beside dA.
//
// At least kWaves waves on a SIMD: the registers of three instead of two at rank
// 64 cost three that spill, and are worth it where there are many rows (16,384 of
// bf16: the backward pass 246 -> 217 us; 2,048: both 60).
template <int RT>
constexpr int kWaves = RT == 4 ? 3 : RT == 8 ? 2 : 1;
template <bool BF16, int M, int RT>
__global__ __launch_bounds__(256, kWaves<RT>) void k_back_dy(TileList blocks, GradArgs g, TileList tiles,
                                                             ShrinkArgs s, DropArgs d) {
    constexpr int kLds = kGradLds<BF16, RT> > kShrinkLds<M, RT> ? kGradLds<BF16, RT> : kShrinkLds<M, RT>;
    __shared__ __align__(16) char lds[kLds];
    const uint32_t index = block_index(), n = g.runs * g.slices;
    if (index < n)
        grad<BF16, RT, false>(blocks, g, d, index, lds);
    else
        shrink<BF16, M, RT, false>(tiles, s, d, index - n, lds);
}
template <bool BF16, int M, int RT, bool DROP>
__global__ __launch_bounds__(256, kWaves<RT>) void k_back_x(TileList blocks, GradArgs g, TileList tiles,
                                                            ExpandArgs e, DropArgs d) {
    constexpr int kLds = kGradLds<BF16, RT> > kExpandLds<BF16, M, RT> ? kGradLds<BF16, RT> : kExpandLds<BF16, M, RT>;
    __shared__ __align__(16) char lds[kLds];
    const uint32_t index = block_index(), n = g.runs * g.slices;
    if (index < n)
        grad<BF16, RT, DROP>(blocks, g, d, index, lds);
    else if (e.out)   // (dx may not be wanted)
        expand<BF16, M, RT, DROP>(tiles, e, d, index - n, lds);
}

struct ReduceJob {
    const float *part;        // [runs + n][rp][width]
    float *dW;                // [n][rank][width]
    const float *scale;       // [n] or null
    float f;
    int width, slices;
};
struct ReduceArgs {
    ReduceJob job[2];
    const PlanHead *head;
    const int *first;         // first block of 32 places of each group
    int rows, n, rank, rp, runs, accumulate;
};

// dW_a[r] (+)= f s_a times the sum of the adapter's parts, in their order; zeros
// for an adapter without rows.
__global__ __launch_bounds__(256) void k_reduce(ReduceArgs a) {
    if (!is_plan(a.head, a.rows, a.n)) return;
    const int which = static_cast<int>(blockIdx.y) >= a.job[0].slices;
    const ReduceJob job = which ? a.job[1] : a.job[0];
    const int col = ((blockIdx.y - (which ? a.job[0].slices : 0)) * 256 + threadIdx.x) * 4;
    if (col >= job.width) return;
    const int ad = blockIdx.x / a.rank, r = blockIdx.x % a.rank;
    const uint32_t j0 = a.first[ad], j1 = a.first[ad + 1], blocks = a.first[a.n];
    f32x4 s = zeros4();
    if (j1 > j0) {
        const uint32_t runs = blocks < static_cast<uint32_t>(a.runs) ? blocks : a.runs;
        const int i0 = run_of(blocks, j0, runs), i1 = run_of(blocks, j1 - 1, runs);
        const float *p = job.part + (static_cast<int64_t>(i0 + ad) * a.rp + r) * job.width + col;
        const int64_t step = static_cast<int64_t>(a.rp) * job.width;
        for (int i = i0; i <= i1; i += 8) {   // eight loads on their way, added in order
            f32x4 v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = i + k <= i1 ? ldf4(p + k * step) : zeros4();
#pragma unroll
            for (int k = 0; k < 8; ++k) s += v[k];
            p += 8 * step;
        }
        s *= job.f * (job.scale ? job.scale[ad] : 1.f);   // (an adapter without rows has zeros whatever its scale)
    }
    float *out = job.dW + static_cast<int64_t>(blockIdx.x) * job.width + col;
    if (a.accumulate) s += ldf4(out);
    stf4(out, s);
}

__global__ __launch_bounds__(256) void k_zero(float *p, int64_t quads) {
    const int64_t i = static_cast<int64_t>(block_index()) * 256 + threadIdx.x;
    if (i < quads) reinterpret_cast<f32x4 *>(p)[i] = zeros4();
}

// ------------------------------------------------------------------- host --
int rank_tiles(int rank) { return rank <= 16 ? 1 : rank <= 32 ? 2 : rank <= 64 ? 4 : 8; }
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Launch shapes, functions of the sizes alone.
struct Shape {
    int rt, rp;
    int64_t places;
    int runs;                     // of the gradients
};

Shape shape_of(int64_t rows, int n_in, int n_out, int rank, int n) {
    Shape s;
    s.rt = rank_tiles(rank);
    s.rp = 16 * s.rt;
    s.places = plan_places(rows, n);
    // runs of the gradients: 1024 workgroups for both together, shared in proportion to their columns, though each has a
    // launch of its own.  16,384 rows at rank 16, dy's launch + x's + k_reduce, with 512, 1024 and 2048 in all: 4096 +
    // 4096 columns 52 + 83 + 5, 47 + 81 + 7 and 59 + 84 + 9 us.  Where the widths differ the narrow side has few
    // workgroups: x of 4096 beside dy of 14336 columns 176 + 115 + 7, 253 + 76 + 7 and 214 + 71 + 10, beside 128,000
    // (one run: 16 workgroups for dA) 1437 + 629 + 18, 1440 + 638 + 18 and, with two runs, 1688 + 229 + 17.
    const int64_t slices = ceil_div(n_in, 256) + ceil_div(n_out, 256);   // (of either type: one workspace)
    // a part costs what rank / 16 blocks do: runs of at least 1.5 times that many (2,047 rows at rank 64: runs of one
    // block took 21 us and their sum 12, runs of six 17 and 6)
    const int64_t least = s.rt == 1 ? 1 : s.rt * 3 / 2, most = ceil_div(plan_max_tiles(rows, n, 1), least);
    const int64_t runs = kMaxRuns / (slices * (s.rt / grad_tiles(s.rt)));
    s.runs = static_cast<int>(runs < 1 ? 1 : runs > most ? most : runs);
    return s;
}

// Tiles of the shrinking product (16 << h rows) and ranges of its long axis: as
// many workgroups as `groups`, if ranges of a kilobyte and tiles of 16 rows give
// them.  Tiles of 32 rows from 192 of their workgroups on (us at 4096 columns of bf16,
// rank 16, 16- and 32-row tiles: 300 rows 5.2-5.6 and 5.8, 1,024 6.8 and 6.4, 1,536
// 6.9 and 6.5, 2,048 9.0 and 9.1, 4,096 14.0 and 12.0; 1,999 rows at rank 64 13.9 and
// 11.0; 509 rows of 768 fp32 4.4 and 5.7).
struct ShrinkShape {
    int h, splits, per;
};
ShrinkShape shrink_shape(int64_t rows, int n, int width, int es, int groups, int most_splits) {
    const int64_t wide = ceil_div(static_cast<int64_t>(width) * es, 1024);
    const int64_t most = wide < most_splits ? wide : most_splits;
    ShrinkShape s;
    s.h = (rows >> 5) * most < 192 ? 0 : 1;
    const int64_t tiles = (rows >> (4 + s.h)) + (n < rows ? n : rows);
    int64_t want = ceil_div(groups, tiles);
    want = want > most ? most : want;
    const int step = 512 / es;   // the four waves' pieces
    s.per = static_cast<int>(ceil_div(ceil_div(width, want), step) * step);
    s.splits = static_cast<int>(ceil_div(width, s.per));
    return s;
}
// The forward pass hides the drawing of its dropout behind more workgroups (16,384 x 4096 at rank 16: 38 us with 512,
// 31 with 2048).  Without it more workgroups gain less, and those that add their parts lose some of that again: 37 + 55
// us with 512, 31 + 58 with 2048 (shrink + expand); the backward pass of the same rows 46 + 81 and 44 + 86.
constexpr int kForwardGroups = 2048, kGroups = 512;

struct WsLayout {
    size_t part, part_a, part_b, bytes;
};
WsLayout ws_layout(const Shape &s, int64_t rows, int n_in, int n_out, int n) {
    WsLayout l;
    size_t at = 0;
    const auto take = [&](size_t b) {
        const size_t here = at;
        at += align256(b);
        return here;
    };
    int splits = 1;
    for (int es = 2; es <= 4; es += 2) {
        const int f = shrink_shape(rows, n, n_in, es, kForwardGroups, kMaxParts).splits,
                  b = shrink_shape(rows, n, n_out, es, kGroups, parts_of(s.rt)).splits;
        splits = f > splits ? f : splits;
        splits = b > splits ? b : splits;
    }
    const size_t parts = static_cast<size_t>(s.runs) + n;
    l.part = take(static_cast<size_t>(s.places) * s.rp * 4 * splits);
    l.part_a = take(parts * s.rp * n_in * 4);
    l.part_b = take(parts * s.rp * n_out * 4);
    l.bytes = at;
    return l;
}

template <typename F>
void with_rank(int rt, F f) {
    switch (rt) {
        case 1: f(std::integral_constant<int, 1>{}); break;
        case 2: f(std::integral_constant<int, 2>{}); break;
        case 4: f(std::integral_constant<int, 4>{}); break;
        default: f(std::integral_constant<int, 8>{}); break;
    }
}
template <typename F>
void with_tile(int h, F f) {
    if (h == 0)
        f(std::integral_constant<int, 1>{});
    else
        f(std::integral_constant<int, 2>{});
}
// Tiles of the expanding product: 32 rows, or 16 where those leave CUs without work (us with 16 and 32 rows, bf16 at
// rank 16 to 4096 columns: 300 rows 4.3 and 4.6, 1,024 6.5 and 6.8, 2,048 10.0 and 11.0, 4,096 17.3 and 17.3; 1,999
// rows to 1024 columns 4.8 and 5.4, at rank 64 5.8 and 6.6; 509 rows to 2304 fp32 columns 6.7 and 10.3).
int expand_height(int64_t rows, int slices) { return (rows >> 5) * slices < 512 ? 0 : 1; }

}  // namespace

size_t adapter_plan_bytes(int64_t rows, int n) { return plan_layout(rows, n).bytes; }

hipError_t launch_adapter_plan(const int *row_adapter, int64_t rows, int n, void *plan, hipStream_t s) {
    const PlanView v = plan_view(plan, rows, n);
    const int segs = static_cast<int>((rows + kSeg - 1) / kSeg);
    k_plan_hist<<<segs, 1024, 0, s>>>(row_adapter, v);
    k_plan_scan<<<1, 1024, 0, s>>>(v, segs);
    k_plan_scatter<<<segs, 1024, 0, s>>>(row_adapter, v);
    return hipGetLastError();
}

size_t adapter_ws_bytes(int64_t rows, int n_in, int n_out, int rank, int n, bool backward) {
    const WsLayout l = ws_layout(shape_of(rows, n_in, n_out, rank, n), rows, n_in, n_out, n);
    return backward ? l.bytes : l.part_a;   // the forward pass has the parts of U alone, which come first
}

hipError_t launch_adapter_forward(const AdapterDims &m, bool bf16, const void *plan, const void *x, int64_t ld_x,
                                  const void *A, const void *B, const float *scale, const void *base, int64_t ld_b,
                                  void *y, int64_t ld_y, float *u, double p, uint64_t seed, uint64_t offset, void *ws,
                                  hipStream_t st) {
    const DropArgs d = drop_args(p, seed, offset);
    const PlanView pv = plan_view(const_cast<void *>(plan), m.rows, m.n);
    const Shape s = shape_of(m.rows, m.n_in, m.n_out, m.rank, m.n);
    const WsLayout l = ws_layout(s, m.rows, m.n_in, m.n_out, m.n);
    float *part = reinterpret_cast<float *>(static_cast<char *>(ws) + l.part);
    const ShrinkShape h = shrink_shape(m.rows, m.n, m.n_in, bf16 ? 2 : 4, d.thr ? kForwardGroups : kGroups, kMaxParts);
    const ShrinkArgs sa = {static_cast<const char *>(x), ld_x, m.n_in, static_cast<const char *>(A), m.rank, part,
                           s.places, h.splits, h.per};
    ExpandArgs e = {part, h.splits, s.places, scale, static_cast<const char *>(B), m.rank, m.n_out,
                    static_cast<const char *>(base), ld_b, static_cast<char *>(y), ld_y, u, 0};
    const auto go = [&](auto b, auto rt) {
        constexpr bool BF16 = decltype(b)::value;
        constexpr int RT = decltype(rt)::value;
        with_tile(h.h, [&](auto mt) {
            constexpr int M = decltype(mt)::value;
            const dim3 grid = block_grid(plan_max_tiles(m.rows, m.n, h.h) * h.splits);
            if (d.thr)
                k_shrink<BF16, M, RT, true><<<grid, 256, 0, st>>>(tile_list(pv, h.h), sa, d);
            else
                k_shrink<BF16, M, RT, false><<<grid, 256, 0, st>>>(tile_list(pv, h.h), sa, d);
        });
        e.slices = static_cast<int>(ceil_div(m.n_out, kSliceCols<BF16, RT>));
        const int he = expand_height(m.rows, e.slices);
        with_tile(he, [&](auto mt) {
            k_expand<BF16, decltype(mt)::value, RT, false>
                <<<block_grid(plan_max_tiles(m.rows, m.n, he) * e.slices), 256, 0, st>>>(tile_list(pv, he), e, d);
        });
    };
    with_rank(s.rt, [&](auto rt) { bf16 ? go(std::true_type{}, rt) : go(std::false_type{}, rt); });
    return hipGetLastError();
}

hipError_t launch_adapter_backward(const AdapterDims &m, bool bf16, const void *plan, const void *x, int64_t ld_x,
                                   const void *dy, int64_t ld_dy, const void *A, const void *B, const float *scale,
                                   const float *u, const void *base, int64_t ld_b, void *dx, int64_t ld_dx, float *dA,
                                   float *dB, bool accumulate, double drop_p, uint64_t seed, uint64_t offset, void *ws,
                                   hipStream_t st) {
    const DropArgs d = drop_args(drop_p, seed, offset);
    if (m.rows == 0) {   // sums over nothing
        if (!accumulate) {
            const int64_t na = static_cast<int64_t>(m.n) * m.rank * m.n_in / 4;
            const int64_t nb = static_cast<int64_t>(m.n) * m.rank * m.n_out / 4;
            k_zero<<<block_grid(ceil_div(na, 256)), 256, 0, st>>>(dA, na);
            k_zero<<<block_grid(ceil_div(nb, 256)), 256, 0, st>>>(dB, nb);
        }
        return hipGetLastError();
    }
    const PlanView pv = plan_view(const_cast<void *>(plan), m.rows, m.n);
    const Shape s = shape_of(m.rows, m.n_in, m.n_out, m.rank, m.n);
    const WsLayout l = ws_layout(s, m.rows, m.n_in, m.n_out, m.n);
    char *w = static_cast<char *>(ws);
    float *part = reinterpret_cast<float *>(w + l.part);
    const ShrinkShape h = shrink_shape(m.rows, m.n, m.n_out, bf16 ? 2 : 4, kGroups, parts_of(s.rt));
    const ShrinkArgs sa = {static_cast<const char *>(dy), ld_dy, m.n_out, static_cast<const char *>(B), m.rank, part,
                           s.places, h.splits, h.per};
    const int cols = grad_cols(bf16, s.rt), ranges = s.rt / grad_tiles(s.rt);
    const GradArgs gb = {static_cast<const char *>(dy), ld_dy, m.n_out,
                         static_cast<int>(ceil_div(m.n_out, cols)) * ranges,
                         u, 0, s.places, m.rank, reinterpret_cast<float *>(w + l.part_b), s.runs};
    const GradArgs ga = {static_cast<const char *>(x), ld_x, m.n_in, static_cast<int>(ceil_div(m.n_in, cols)) * ranges,
                         part, h.splits, s.places, m.rank, reinterpret_cast<float *>(w + l.part_a), s.runs};
    ExpandArgs e = {part, h.splits, s.places, scale, static_cast<const char *>(A), m.rank, m.n_in,
                    static_cast<const char *>(base), ld_b, static_cast<char *>(dx), ld_dx, nullptr, 0};
    const TileList blocks = tile_list(pv, 1);
    const auto go = [&](auto b, auto rt) {
        constexpr bool BF16 = decltype(b)::value;
        constexpr int RT = decltype(rt)::value;
        with_tile(h.h, [&](auto mt) {
            const int64_t n = static_cast<int64_t>(gb.runs) * gb.slices + plan_max_tiles(m.rows, m.n, h.h) * h.splits;
            k_back_dy<BF16, decltype(mt)::value, RT>
                <<<block_grid(n), 256, 0, st>>>(blocks, gb, tile_list(pv, h.h), sa, d);
        });
        e.slices = static_cast<int>(ceil_div(m.n_in, kSliceCols<BF16, RT>));
        const int he = expand_height(m.rows, e.slices);
        with_tile(he, [&](auto mt) {
            constexpr int M = decltype(mt)::value;
            const int64_t n = static_cast<int64_t>(ga.runs) * ga.slices +
                              (dx ? plan_max_tiles(m.rows, m.n, he) * e.slices : 0);
            if (d.thr)
                k_back_x<BF16, M, RT, true><<<block_grid(n), 256, 0, st>>>(blocks, ga, tile_list(pv, he), e, d);
            else
                k_back_x<BF16, M, RT, false><<<block_grid(n), 256, 0, st>>>(blocks, ga, tile_list(pv, he), e, d);
        });
    };
    with_rank(s.rt, [&](auto rt) { bf16 ? go(std::true_type{}, rt) : go(std::false_type{}, rt); });
    ReduceArgs r = {};
    r.job[0] = {gb.part, dB, scale, 1.f, m.n_out, static_cast<int>(ceil_div(m.n_out, 1024))};
    r.job[1] = {ga.part, dA, scale, d.scale, m.n_in, static_cast<int>(ceil_div(m.n_in, 1024))};
    r.head = pv.head;
    r.first = pv.first[1];
    r.runs = s.runs;
    r.rows = pv.rows;
    r.n = m.n;
    r.rank = m.rank;
    r.rp = s.rp;
    r.accumulate = accumulate;
    const dim3 grid(static_cast<unsigned>(m.n * m.rank), static_cast<unsigned>(r.job[0].slices + r.job[1].slices));
    k_reduce<<<grid, 256, 0, st>>>(r);
    return hipGetLastError();
}

}  // namespace logra
