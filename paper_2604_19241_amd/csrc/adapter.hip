// The shared projection with a low-rank adapter for each request, and its gradients (the mathematics: adapter.hpp).
//
// Forward and the gradient of x are one operation: x W + s (x A^T) B and dy W^T + s (dy B^T) A differ in which factor comes
// first and in the form of W, so `x`, `first` and `second` below are x, A, B or dy, B, A; R is the reduction's length and C
// the columns of the result.  The gradients of the factors, dA_a = sum_t g[t]^T x[t] with g = s dy B^T and dB_a = sum_t h[t]^T dy[t] with
// h = s x A^T, are reductions over the tokens of one adapter.
//
// Few tokens (kFewTokens): two launches and no plan.  The first computes x W cut along R into fp32 parts, and the likewise cut h of
// every group of tokens with one adapter, side by side; the second adds the parts, then h B, and rounds once.  Each workgroup finds the
// tokens of its adapter by itself, from a ballot over the ids.
// More tokens: a plan sorts them by adapter (stable, one launch), a launch computes h, and the tiles of the product run on over
// their low-rank part (adapter.hpp).
// No atomic decides an order anywhere: results are the same bits on every run.
#include "adapter.hpp"

#include <algorithm>
#include <type_traits>

namespace uniep {

constexpr int kFewTokens = 512;
constexpr int kFewWords = kFewTokens / 64;
// Rows of a block of the plan: as many tokens of one adapter share the fetch of its first factor.
static int block_rows(int T) { return T >= 16384 ? 64 : 32; }
constexpr int kGradRows = 64;         // rows up to which an adapter's gradients are made row by row (adapter_grad_rows_kernel)
constexpr int kUnit = 64;             // rows of which the plan knows the first and the last segment

// ------------------------------------------------------------------ the plan
// int32 words: [0] blocks, [1] adapters with many rows, [2] adapters with rows, then the arrays.
struct PlanView {
    int32_t* head;
    int32_t* order;      // [T] row -> token: those without an adapter, then by adapter, each in the order of the tokens
    int32_t* start;      // [n + 1] first row of an adapter
    int32_t* ordinal;    // [n] which segment an adapter is
    int32_t* seg;        // [n] segment -> adapter
    int32_t* unit;       // [units][2] segments of the first and the last row of every kUnit rows (-1: no adapter)
    int32_t* many;       // [n] adapters with more than kGradRows rows (as many as head[1] says)
    int32_t* block;      // [blocks][2] first row; rows | (adapter + 1) << 8.  One adapter, one multiple of block_rows
};
static size_t plan_blocks(const moe_adapter_shape_t& s) { return (size_t)s.T / block_rows(s.T) + s.adapters + 2; }
static size_t plan_units(const moe_adapter_shape_t& s) { return ((size_t)s.T + kUnit - 1) / kUnit; }
// (room for blocks of 32 whatever their rows are: with as many adapters no two numbers of tokens have plans of one size, by which the binding knows a plan's own)
static size_t plan_words(const moe_adapter_shape_t& s) {
    return 16 + (size_t)s.T + 4 * (size_t)s.adapters + 1 + 2 * plan_units(s) + 2 * ((size_t)s.T / 32 + s.adapters + 2);
}
static PlanView plan_view(const moe_adapter_shape_t& s, void* plan) {
    PlanView v;
    v.head = (int32_t*)plan;
    v.block = v.head + 16;                       // (pairs first: 8-byte aligned)
    v.unit = v.block + 2 * plan_blocks(s);
    v.order = v.unit + 2 * plan_units(s);
    v.start = v.order + s.T;
    v.ordinal = v.start + s.adapters + 1;
    v.seg = v.ordinal + s.adapters;
    v.many = v.seg + s.adapters;
    return v;
}
// Whether the path for few tokens is taken: up to 256 tokens always, up to 512 unless the product, in tiles of 64 x 64, is large. Measured, us of the forward call and of the training step in a
// graph of ten, few tokens / sorted with the plan (tokens, K x N, ranks, adapters):
//   512, 2048 x 2816,  16,  16     24.4,  58.1 /  33.6,  80.2        400, 7168 x 7168,  16,   2    106.3, 216.7 /  83.5, 164.9
//   512, 2048 x 2816, 128,   2     43.2,  95.0 /  40.8,  87.7        400, 7168 x 7168,  16,  16    104.7, 225.3 /  89.5, 197.5
//   512, 2048 x 2816, 128, 256     57.7, 361.7 /  93.5, 352.2        400, 7168 x 7168, 128,   2    134.4, 298.6 / 102.3, 240.4
//   300, 4096 x 4096, 128,   2     50.4, 109.7 /  54.4, 115.1        300, 7168 x 7168,  16,   2     85.1, 170.2 /  81.6, 159.0
//   512, 4096 x 4096,  16,  16     44.2,  98.9 /  52.8, 118.8        300, 7168 x 7168,  16,  16     83.8, 177.4 /  91.5, 202.5
//   512, 4096 x 4096, 128,   2     61.9, 143.9 /  60.1, 126.5        400, 7168 x 7168, 128,  16    143.8, 361.4 / 232.6, 510.6
// The left column's are not sorted, the right one's are.  The rule knows neither ranks nor adapters and is on the slower side for 300 tokens of 16 adapters (9 to 14 %), by 40 to 60 % where tiles of
// sorted tokens have long low-rank parts (the last line on the right), and by up to 14 % for 512 tokens on few adapters of many ranks (128, 2 on the left).
static bool adapter_few(const moe_adapter_shape_t& s) { return s.T <= kFewTokens / 2 || (s.T <= kFewTokens && (long long)s.T * s.K * s.N <= 8ll << 30); }
bool adapter_needs_plan(const moe_adapter_shape_t& s) { return s.T > kFewTokens; }
// What a plan holds goes by the tokens and the adapters alone, whatever the widths of the shape that it is made with: a plan serves layers of all widths, and up to 512 tokens some
// of them may sort and others not.  (Up to 256 none does.)  Where a shape that sorts is given no plan it makes its own in the workspace, so that the shape alone says which way is taken.
size_t adapter_table_bytes(const moe_adapter_shape_t& s) { return s.T <= kFewTokens / 2 ? 0 : plan_words(s) * 4; }
size_t adapter_plan_bytes(const moe_adapter_shape_t& s) { return adapter_few(s) ? 0 : adapter_table_bytes(s); }

// One workgroup: a counting sort.  Every wave counts a contiguous part of the tokens and later gives its tokens their rows, 64 at a
// time: lanes with the same adapter find each other with a ballot for each bit of the id.
constexpr int kSortWaves = 16;
__global__ void __launch_bounds__(64 * kSortWaves) adapter_plan_kernel(int T, int n, int brows_log2, const int32_t* __restrict__ ids, PlanView v) {
    __shared__ int32_t hist[kSortWaves][kMaxAdapters + 1];
    __shared__ int32_t first[kMaxAdapters + 2];     // rows before bin b (bin 0: no adapter, bin a + 1: adapter a)
    __shared__ int32_t fblock[kMaxAdapters + 2], fseg[kMaxAdapters + 2];
    __shared__ int32_t carry[3][kSortWaves];
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, bins = n + 1;
    const uint64_t below = (1ull << lane) - 1ull;
    for (int b = lane; b < bins; b += 64) hist[w][b] = 0;
    const int part = ((T + kSortWaves - 1) / kSortWaves + 63) & ~63, lo = min(T, w * part), hi = min(T, lo + part);
    // f(token, bin) for this wave's tokens, 64 at a time; the ids of 256 are fetched together while those before them are worked on, and the first are kept
    // (a copy of f for each of 16 fetches, with all ids kept for the second time, was slower: 12 KB of code that runs once)
    auto fetch = [&](int (&a)[4], int t0) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int t = t0 + 64 * i + lane;
            a[i] = t < hi ? ids[t] : -1;
        }
    };
    int start[4];
    fetch(start, lo);
    auto each = [&](auto f) {
        int next[4] = {start[0], start[1], start[2], start[3]};
#pragma unroll 1
        for (int t0 = lo; t0 < hi; t0 += 256) {
            const int a[4] = {next[0], next[1], next[2], next[3]};
            if (t0 + 256 < hi) fetch(next, t0 + 256);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (t0 + 64 * i < hi) f(t0 + 64 * i + lane, (unsigned)a[i] < (unsigned)n ? a[i] + 1 : 0);
        }
    };
    __syncthreads();
    auto count = [&](int t, int b) {   // packed requests: mostly 64 tokens with one adapter
        if (__ballot(t < hi && b == rfl(b)) == ~0ull) {
            if (lane == 0) hist[w][b] += 64;
        } else if (t < hi) {
            atomicAdd(&hist[w][b], 1);
        }
    };
    each(count);
    __syncthreads();
    // bins -> first rows, blocks and segments: thread b has bin b (two at most a thread: 1025 bins)
    int base_rows = 0, base_blocks = 0, base_segs = 0;
    for (int b0 = 0; b0 < bins; b0 += 64 * kSortWaves) {
        const int b = b0 + tid;
        int h[kSortWaves], c = 0;
#pragma unroll
        for (int k = 0; k < kSortWaves; ++k) {
            h[k] = b < bins ? hist[k][b] : 0;
            c += h[k];
        }
        // x's sum over the threads before this one; the waves' totals are exchanged between the two
        auto within = [&](int x, int which) {
            const int p = wave_scan(x);
            if (lane == 63) carry[which][w] = p;
            return p - x;
        };
        auto before = [&](int p, int which, int& base) {
            p += base;
#pragma unroll
            for (int k = 0; k < kSortWaves; ++k) {
                const int u = carry[which][k];
                if (k < w) p += u;
                base += u;
            }
            return p;
        };
        int r0 = within(c, 0), both = within(b > 0 && c > 0 ? 1 | (c > kGradRows) << 16 : 0, 2);   // (up to 1024 of each)
        __syncthreads();
        r0 = before(r0, 0, base_rows);
        both = before(both, 2, base_segs);
        const int s0 = both & 0xffff;
        int k0 = within(c > 0 ? ((r0 + c - 1) >> brows_log2) - (r0 >> brows_log2) + 1 : 0, 1);
        __syncthreads();
        k0 = before(k0, 1, base_blocks);
        if (b < bins) {
            first[b] = r0;
            fblock[b] = k0;
            fseg[b] = s0;
            int at = r0;
#pragma unroll
            for (int k = 0; k < kSortWaves; ++k) {
                hist[k][b] = at;
                at += h[k];
            }
            if (b > 0) {
                v.start[b - 1] = r0;
                v.ordinal[b - 1] = s0;
                if (c > 0) v.seg[s0] = b - 1;
                if (c > kGradRows) v.many[both >> 16] = b - 1;
            }
        }
        __syncthreads();
    }
    if (tid == 0) {
        first[bins] = T;
        fblock[bins] = base_blocks;
        v.start[n] = T;
        v.head[0] = base_blocks;
        v.head[1] = base_segs >> 16;
        v.head[2] = base_segs & 0xffff;
    }
    __syncthreads();
    // rows
    volatile int32_t* mine = hist[w];
    auto place = [&](int t, int b) {
        uint64_t same = __ballot(t < hi);
        if (__ballot(b == rfl(b)) != ~0ull)
            for (int bit = 0; (bins - 1) >> bit; ++bit) {
                const uint64_t m = __ballot((b >> bit) & 1);
                same &= (b >> bit) & 1 ? m : ~m;
            }
        if (t < hi) {
            const int at = mine[b];
            v.order[at + __popcll(same & below)] = t;
            __builtin_amdgcn_wave_barrier();
            if ((same >> lane) == 1ull) mine[b] = at + __popcll(same);   // the last of them
        }
        __builtin_amdgcn_wave_barrier();
    };
    each(place);
    // blocks and units, a wave a bin
    for (int b = w; b < bins; b += kSortWaves) {
        const int r0 = first[b], r1 = first[b + 1], o = b > 0 ? fseg[b] : -1;
        if (r1 <= r0) continue;
        const int q0 = r0 >> brows_log2, q1 = (r1 - 1) >> brows_log2;
        for (int q = q0 + lane; q <= q1; q += 64) {
            const int a = max(r0, q << brows_log2), e = min(r1, (q + 1) << brows_log2);
            v.block[2 * (fblock[b] + q - q0)] = a;
            v.block[2 * (fblock[b] + q - q0) + 1] = (e - a) | b << 8;
        }
        for (int u = r0 / kUnit + lane; u <= (r1 - 1) / kUnit; u += 64) {
            if (u * kUnit >= r0) v.unit[2 * u] = o;
            if (min(T, (u + 1) * kUnit) <= r1) v.unit[2 * u + 1] = o;
        }
    }
}

int adapter_plan_launch(const moe_adapter_shape_t& s, const int32_t* ids, void* plan, hipStream_t st) {
    hipLaunchKernelGGL(adapter_plan_kernel, dim3(1), dim3(64 * kSortWaves), 0, st, s.T, s.adapters, block_rows(s.T) == 64 ? 6 : 5, ids, plan_view(s, plan));
    return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP;
}

// ------------------------------------------------------------------ parameters
struct ProjParams {
    int T, R, C, r, n;
    const char* x;          // [T][ldx bytes]
    size_t ldx;
    const char* w;          // KS: [R][C], KC: [C][R]
    const char* first;      // [n][r][R]
    const char* second;     // [n][r][C]
    const float* scale;     // [n] or NULL
    const int32_t* ids;
    char* y;                // [T][C] bf16, or fp32
    int out_f32;
    float* h;               // [T][r], or NULL where nobody wants it (few tokens)
    // few tokens
    float* part;            // [splits][T][C]
    float* hpart;           // [hsplits][T][r]
    int splits, per_split, hsplits, hper_split;
    int col_tiles, row_tiles, rank_tiles, hgroups;
    int dot_cut;            // workgroups that share 64 ranks of dots
    // more
    PlanView plan;
    char* hx;               // the low-rank rows of every tile (hx_base)
    char* second_t;         // [n][C][r] (KC)
    uint16_t* terms[2];     // backward: [T rows][3][r], h (of the forward call) and this h as three bf16 terms, by row
    const float* h_given;   // the forward call's h
    int tile_rows;
    int span;               // columns of a segment's low-rank part: 2 r, for an fp32 result 3 r
    int blocks;             // at most, of the plan (0: there is none)
    int join_rows;          // adapter_parts_join_kernel: rows of a workgroup
};
struct GradParams {
    int T, r, n, few;
    int W[2];               // columns: dB (of dy, with h), dA (of x, with g)
    const char* x[2];
    size_t ldx[2];
    const float* h[2];      // [T][r]; NULL: hpart (few tokens)
    float* out[2];          // [n][r][W]
    int parts;              // more tokens: into how many parts an adapter's rows are cut at most (GradCut), and the parts' sums, [grad_pieces][r][W] each
    float* part[2];
    int col_tiles[2], rank_tiles;
};

__device__ __forceinline__ int adapter_of(const int32_t* ids, int t, int n) {
    const int a = ids[t];
    return (unsigned)a < (unsigned)n ? a : -1;
}
__device__ __forceinline__ Stages stages_of(int R) { return Stages{R / BK, R % BK}; }

// ------------------------------------------------------------------ few tokens
// Which tokens have adapter `a`: a bit each, in scalar registers.  256 threads, two barriers.
struct Members {
    uint64_t m[kFewWords];
    __device__ __forceinline__ void find(int T, int n, const int32_t* ids, int a, uint64_t* s_mask) {
        const int tid = threadIdx.x;
#pragma unroll
        for (int i = 0; i < kFewWords / 4; ++i) {
            const int t = tid + 256 * i;
            const uint64_t b = __ballot(t < T && adapter_of(ids, t < T ? t : 0, n) == a);
            if ((tid & 63) == 0) s_mask[4 * i + (tid >> 6)] = b;
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kFewWords; ++i) {
            const uint64_t b = s_mask[i];
            m[i] = (uint64_t)(uint32_t)rfl((int)(b >> 32)) << 32 | (uint32_t)rfl((int)b);
        }
    }
    __device__ __forceinline__ int before(int t) const {   // t the same in all threads
        int c = 0;
#pragma unroll
        for (int i = 0; i < kFewWords; ++i) c += __popcll(64 * i + 64 <= t ? m[i] : 64 * i >= t ? 0ull : m[i] & ((1ull << (t & 63)) - 1ull));
        return c;
    }
    __device__ __forceinline__ int count() const { return before(kFewTokens); }
    // the tokens from the `skip`-th on, up to `most`, into list[]; ends with a barrier
    __device__ __forceinline__ void list(int skip, int most, int32_t* list) const {
        const int w = rfl(threadIdx.x >> 6), lane = threadIdx.x & 63;
#pragma unroll
        for (int i = 0; i < kFewWords / 4; ++i) {
            uint64_t mine = 0;
            int k = -skip;
#pragma unroll
            for (int q = 0; q < kFewWords; ++q) {
                if (q < 4 * i + w) k += __popcll(m[q]);
                if (q == 4 * i + w) mine = m[q];
            }
            k += __builtin_amdgcn_mbcnt_hi((uint32_t)(mine >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mine, 0));
            if (((mine >> lane) & 1) && k >= 0 && k < most) list[k] = 64 * (4 * i + w) + lane;
        }
        __syncthreads();
    }
};

// Ranks [j0, j1) of h for up to 4 tokens over [k0, k1) of the reduction, by dot products: wave w has every fourth rank, its lanes 8 elements of 512 each;
// put(m, j, v) is called by one lane.  For so few tokens the tile of 32 rows by 64 ranks that is used for more moves ten times the bytes (the first launch of
// 256 tokens of 256 adapters, 8 ranks of 2048: 19.0 us, with dots 14.3).
constexpr int kDotTokens = 4;
template <class TokenFn, class PutFn>
__device__ __forceinline__ void few_dots(const ProjParams& p, int a, int j0, int j1, int rows, int k0, int k1, TokenFn token, PutFn put) {
    constexpr int kRanks = 4;   // of a wave, at a time
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    for (int j = j0 + w; j < j1; j += 4 * kRanks) {
        const char* const f = p.first + ((size_t)a * p.r + j) * p.R * 2;
        float acc[kRanks][kDotTokens] = {};
        for (int kk = k0 + 8 * lane; kk < k1; kk += 1024) {
            u32x4_t b[2][kRanks], x[2][kDotTokens];
#pragma unroll
            for (int h = 0; h < 2; ++h) {   // (loads first: two runs of k are on their way together)
                const int k = kk + 512 * h;
#pragma unroll
                for (int i = 0; i < kRanks; ++i) {
                    b[h][i] = zero4();
                    if (k < k1 && j + 4 * i < j1) b[h][i] = *(const u32x4_t*)(f + ((size_t)(4 * i) * p.R + k) * 2);
                }
#pragma unroll
                for (int m = 0; m < kDotTokens; ++m) {
                    x[h][m] = zero4();
                    if (k < k1 && m < rows) x[h][m] = *(const u32x4_t*)(p.x + (size_t)token(m) * p.ldx + (size_t)k * 2);
                }
            }
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int m = 0; m < kDotTokens; ++m)
                    if (m < rows)
#pragma unroll
                        for (int i = 0; i < kRanks; ++i)
#pragma unroll
                            for (int q = 0; q < 4; ++q) acc[i][m] += bf16_lo(x[h][m][q]) * bf16_lo(b[h][i][q]) + bf16_hi(x[h][m][q]) * bf16_hi(b[h][i][q]);
        }
#pragma unroll
        for (int i = 0; i < kRanks; ++i)
#pragma unroll
            for (int m = 0; m < kDotTokens; ++m)
                if (m < rows && j + 4 * i < j1) {
                    across<64>(acc[i][m], [](float u, float v) { return u + v; });
                    if (lane == 0) put(m, j + 4 * i, acc[i][m]);
                }
    }
}

// Parts of x W and of h.  Tasks: (column tile, split, row tile), then of h (token, part of a rank tile's dots, rank tile, split), where a workgroup whose token is not every
// 32nd of its adapter's has nothing to do, or (adapter, 32 of its tokens, rank tile, split) where that is fewer.
template <int NRF, int FORM>
__global__ void __launch_bounds__(kSmallThreads) adapter_few_first_kernel(ProjParams p) {
    constexpr int kLds = SmallTile<NRF, 2>::kLds > SmallTile<1, 2>::kLds ? SmallTile<NRF, 2>::kLds : SmallTile<1, 2>::kLds;   // (h: 32 rows)
    __shared__ __attribute__((aligned(512))) char smem[kLds];
    __shared__ uint64_t s_mask[kFewWords];
    __shared__ int32_t s_list[32];
    const Stages all = stages_of(p.R);
    const int nst = all.full + (all.tail > 0);
    int id = blockIdx.x;
    const int pairs = p.col_tiles * p.splits, gemm = pairs * p.row_tiles;
    auto part_of = [&](int s0, int s1) { return Stages{min(all.full, s1) - s0, s1 > all.full ? all.tail : 0}; };
    if (id < gemm) {
        const int pair = id % pairs, rt = id / pairs, ct = pair % p.col_tiles, sp = pair / p.col_tiles;
        const int s0 = sp * p.per_split, s1 = min(nst, s0 + p.per_split);
        const int row0 = rt * 32 * NRF, rows = min(32 * NRF, p.T - row0);
        const Stages st = part_of(s0, s1);
        f32x16_t acc[NRF][2];
        {
            const Lane ln;
            KcStages<NRF, false> lb;
            lb.init(ln, rows, st, [&](int r) { return p.x + (size_t)(row0 + r) * p.ldx + (size_t)s0 * (BK * 2); });
            lb.low.used = 0;
            if constexpr (FORM == kKs) {
                KsStages<2, 64> la;
                la.init(ln, p.w + (size_t)s0 * BK * p.C * 2, 64 * ct, p.C, st);
                small_loop<NRF, 2, kKs>(lb, la, s1 - s0, smem, acc);
            } else {
                KcStages<2, true> la;
                la.init(ln, min(64, p.C - 64 * ct), st, [&](int c) { return p.w + ((size_t)(64 * ct + c) * p.R + (size_t)s0 * BK) * 2; });
                small_loop<NRF, 2, kKc>(lb, la, s1 - s0, smem, acc);
            }
        }
        small_sum<NRF, 2>(smem, acc, [&](int row, int col, const float (&v)[8]) {
            col += 64 * ct;
            if (row >= rows || col >= p.C) return;
            f32x4_t* to = (f32x4_t*)(p.part + ((size_t)sp * p.T + row0 + row) * p.C + col);
            to[0] = f32x4_t{v[0], v[1], v[2], v[3]};
            to[1] = f32x4_t{v[4], v[5], v[6], v[7]};
        });
        return;
    }
    id -= gemm;
    const int t = id % p.hgroups, rest = id / p.hgroups, quarter = rest % p.dot_cut, rt = rest / p.dot_cut % p.rank_tiles, sp = rest / p.dot_cut / p.rank_tiles;
    int a, rows, rank = 0;
    if (p.blocks > 0) {   // sorted: a block of the plan
        if (t >= p.plan.head[0]) return;
        const int row0 = p.plan.block[2 * t], code = p.plan.block[2 * t + 1];
        a = (code >> 8) - 1;
        rows = code & 255;
        if (a < 0) return;
        if ((int)threadIdx.x < rows) s_list[threadIdx.x] = p.plan.order[row0 + threadIdx.x];
        __syncthreads();
    } else {
        const int blocks = (p.T + 31) / 32;
        a = p.hgroups == p.T ? rfl(adapter_of(p.ids, t, p.n)) : t / blocks;
        if (a < 0) return;
        Members mb;
        mb.find(p.T, p.n, p.ids, a, s_mask);
        rank = p.hgroups == p.T ? mb.before(t) : t % blocks * 32;
        if (rank % 32 != 0 || rank >= mb.count()) return;
        mb.list(rank, 32, s_list);
        rows = min(32, mb.count() - rank);
    }
    const int s0 = sp * p.hper_split, s1 = min(nst, s0 + p.hper_split);
    if (rank == 0 && rows <= kDotTokens) {
        float* const out = p.hpart + (size_t)sp * p.T * p.r;
        const int ranks = 64 / p.dot_cut, j0 = 64 * rt + quarter * ranks;
        few_dots(p, a, j0, min(p.r, j0 + ranks), rows, s0 * BK, min(p.R, s1 * BK), [&](int m) { return s_list[m]; },
                 [&](int m, int j, float v) { out[(size_t)s_list[m] * p.r + j] = v; });
        return;
    }
    if (quarter > 0) return;
    const Stages st = part_of(s0, s1);
    f32x16_t acc[1][2];
    {
        const Lane ln;
        KcStages<1, false> lb;
        lb.init(ln, rows, st, [&](int r) { return p.x + (size_t)s_list[r] * p.ldx + (size_t)s0 * (BK * 2); });
        lb.low.used = 0;
        KcStages<2, true> la;
        la.init(ln, min(64, p.r - 64 * rt), st, [&](int j) { return p.first + (((size_t)a * p.r + 64 * rt + j) * p.R + (size_t)s0 * BK) * 2; });
        small_loop<1, 2, kKc>(lb, la, s1 - s0, smem, acc);
    }
    small_sum<1, 2>(smem, acc, [&](int row, int col, const float (&v)[8]) {
        col += 64 * rt;
        if (row >= rows || col >= p.r) return;
        f32x4_t* to = (f32x4_t*)(p.hpart + ((size_t)sp * p.T + s_list[row]) * p.r + col);
        to[0] = f32x4_t{v[0], v[1], v[2], v[3]};
        to[1] = f32x4_t{v[4], v[5], v[6], v[7]};
    });
}

// s h[t][j] from its parts
__device__ __forceinline__ float whole_h(const ProjParams& p, int t, int j, float s) {
    float v = 0.f;
#pragma unroll 8
    for (int k = 0; k < p.hsplits; ++k) v += p.hpart[((size_t)k * p.T + t) * p.r + j];
    return v * s;
}
__device__ __forceinline__ void fma8(float (&acc)[8], float h, u32x4_t b) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        acc[2 * q] += h * bf16_lo(b[q]);
        acc[2 * q + 1] += h * bf16_hi(b[q]);
    }
}

// y of G tokens with one adapter (the last group may have fewer) and 1024 columns, 4 a lane.  (Waves that shared 512 columns and their sums in LDS
// took 11.6 us for 256 tokens of 256 adapters, 8 ranks of 4096 columns each.)
constexpr int kJoinCols = 1024;
template <int G>
struct JoinShared {
    __attribute__((aligned(16))) float h[kMaxRank][G];
    uint64_t mask[kFewWords];
    int32_t list[G];
};
__device__ __forceinline__ void fma4(float (&acc)[4], float h, u32x2_t b) {
    acc[0] += h * bf16_lo(b[0]);
    acc[1] += h * bf16_hi(b[0]);
    acc[2] += h * bf16_lo(b[1]);
    acc[3] += h * bf16_hi(b[1]);
}
template <int G>
__device__ __forceinline__ void join_task(const ProjParams& p, int t, int cb, JoinShared<G>& S) {
    const int tid = threadIdx.x;
    const int a = rfl(adapter_of(p.ids, t, p.n));
    int rows = 1;
    if (G > 1) {
        Members mb;
        mb.find(p.T, p.n, p.ids, a, S.mask);
        const int rank = mb.before(t);
        if (rank % G != 0) return;
        mb.list(rank, G, S.list);
        rows = min(G, mb.count() - rank);
    }
    auto token = [&](int m) { return G == 1 ? t : S.list[m]; };
    const int c = cb * kJoinCols + 4 * tid;
    const bool works = c < p.C;
    const char* const f = p.second + ((size_t)max(a, 0) * p.r * p.C + c) * 2;
    const float* const part = p.part + c;
    // the first loads of everything are on their way together: this kernel is what its dependent loads take
    constexpr int kPreB = 8, kPreP = 8;
    u32x2_t b[kPreB];
    f32x4_t q[kPreP];
#pragma unroll
    for (int i = 0; i < kPreB; ++i) {
        b[i] = u32x2_t{0u, 0u};
        if (works && a >= 0) b[i] = *(const u32x2_t*)(f + (size_t)i * p.C * 2);   // (there are at least 8 ranks)
    }
#pragma unroll
    for (int i = 0; i < kPreP; ++i) {
        q[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        if (works && i < p.splits) q[i] = *(const f32x4_t*)(part + ((size_t)i * p.T + t) * p.C);
    }
    if (a >= 0 || p.h) {
        const float s = a < 0 ? 0.f : p.scale ? p.scale[a] : 1.f;
        for (int i = tid; i < rows * p.r; i += 256) {
            const int m = G == 1 ? 0 : i / p.r, j = i - m * p.r, tok = token(m);
            const float v = a < 0 ? 0.f : whole_h(p, tok, j, s);
            S.h[j][m] = v;
            if (p.h && cb == 0) p.h[(size_t)tok * p.r + j] = v;
        }
        __syncthreads();
    }
    if (!works) return;
    float acc[G][4] = {};
#pragma unroll
    for (int i = 0; i < kPreP; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[0][j] += q[i][j];
#pragma unroll
    for (int m = 0; m < G; ++m)
        if (m < rows)
#pragma unroll 4
            for (int s = m == 0 ? kPreP : 0; s < p.splits; ++s) {
                const f32x4_t u = *(const f32x4_t*)(part + ((size_t)s * p.T + token(m)) * p.C);
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[m][j] += u[j];
            }
    if (a >= 0) {
#pragma unroll
        for (int i = 0; i < kPreB; ++i)
#pragma unroll
            for (int m = 0; m < G; ++m) fma4(acc[m], S.h[i][m], b[i]);   // (rows that are not there: never stored)
#pragma unroll 8
        for (int j = kPreB; j < p.r; ++j) {
            const u32x2_t x = *(const u32x2_t*)(f + (size_t)j * p.C * 2);
#pragma unroll
            for (int m = 0; m < G; ++m) fma4(acc[m], S.h[j][m], x);
        }
    }
#pragma unroll
    for (int m = 0; m < G; ++m)
        if (m < rows) {
            const size_t at = (size_t)token(m) * p.C + c;
            if (p.out_f32) *(f32x4_t*)(p.y + at * 4) = f32x4_t{acc[m][0], acc[m][1], acc[m][2], acc[m][3]};
            else *(u32x2_t*)(p.y + at * 2) = u32x2_t{pack_bf16x2(acc[m][0], acc[m][1]), pack_bf16x2(acc[m][2], acc[m][3])};
        }
}

// Gradients of 8 ranks of one adapter, token by token.  With COLS = 64 or 256 columns a workgroup groups of 16 or 64 lanes share the tokens, and their sums are added in LDS; with 1024
// every lane has its own columns, which keeps the LDS small and the workgroups few where the adapters have few tokens or none (11 tokens, 27 adapters of 64 ranks, 6552 x 464:
// the training step 66 us with 256, 51 with 1024).  (With 512 columns a wave and each wave its own columns or ranks, 256 tokens on 2 adapters of 512 x 1024 were 4
// workgroups that took 128 tokens one after the other: 48 us; with 256 columns 12 workgroups, 11; with 64, where a group's tokens are all fetched at once, 8.)
constexpr int kGradRanks = 8;
// LPR lanes have a token's row.
template <int TOKENS, int COLS>
struct FewGradShared {
    static constexpr int LPR = COLS < 1024 ? COLS / 4 : 256, kGroups = 256 / LPR;
    float h[TOKENS][kGradRanks];
    __attribute__((aligned(16))) float sums[kGroups > 1 ? kGroups : 1][kGroups > 1 ? kGradRanks : 1][kGroups > 1 ? COLS : 4];
    uint64_t mask[kFewWords];
    int32_t list[TOKENS];
};
// Which piece of work `id` is.
struct FewGradTask {
    int which, cb, a, j0;
    __device__ __forceinline__ FewGradTask(const GradParams& g, int id) {
        const int of = g.n * g.rank_tiles * g.col_tiles[0];
        which = id < of ? 0 : 1;
        if (which) id -= of;
        const int rest = id / g.col_tiles[which];
        cb = id % g.col_tiles[which];
        a = rest % g.n;
        j0 = rest / g.n * kGradRanks;
    }
};
// S.list[0 .. count): the adapter's tokens; h4(token, j) = 4 ranks of it from j on.
template <int TOKENS, int COLS, class H4>
__device__ __forceinline__ void few_grad_task(const GradParams& g, const FewGradTask& t, int count, FewGradShared<TOKENS, COLS>& S, H4 h4) {
    constexpr int LPR = FewGradShared<TOKENS, COLS>::LPR, kStep = FewGradShared<TOKENS, COLS>::kGroups, kPre = kStep > 1 ? 8 : 4;
    const int tid = threadIdx.x, k0 = tid / LPR, W = g.W[t.which], c = t.cb * COLS + 4 * (tid % LPR);
    float* const out = g.out[t.which] + ((size_t)t.a * g.r + t.j0) * W;
    float acc[kGradRanks][4] = {};
    if (count > 0) {
        // the first rows of x are on their way while h is fetched
        const size_t ldx = g.ldx[t.which];
        const char* const x = g.x[t.which] + (size_t)min(c, W - 4) * 2;
        u32x2_t pre[kPre];
#pragma unroll
        for (int i = 0; i < kPre; ++i) pre[i] = *(const u32x2_t*)(x + (size_t)S.list[min(k0 + kStep * i, count - 1)] * ldx);
        for (int i = tid; i < 2 * count; i += 256) *(f32x4_t*)&S.h[i >> 1][4 * (i & 1)] = h4(S.list[i >> 1], t.j0 + 4 * (i & 1));
        __syncthreads();
        if (c < W) {
#pragma unroll
            for (int i = 0; i < kPre; ++i)
                if (k0 + kStep * i < count)
#pragma unroll
                    for (int j = 0; j < kGradRanks; ++j) fma4(acc[j], S.h[k0 + kStep * i][j], pre[i]);
#pragma unroll 8
            for (int k = k0 + kStep * kPre; k < count; k += kStep) {
                const u32x2_t b = *(const u32x2_t*)(x + (size_t)S.list[k] * ldx);
#pragma unroll
                for (int j = 0; j < kGradRanks; ++j) fma4(acc[j], S.h[k][j], b);
            }
        }
    }
    if (kStep == 1) {
        if (c < W)
#pragma unroll
            for (int j = 0; j < kGradRanks; ++j) *(f32x4_t*)(out + (size_t)j * W + c) = f32x4_t{acc[j][0], acc[j][1], acc[j][2], acc[j][3]};
        return;
    }
#pragma unroll
    for (int j = 0; j < kGradRanks; ++j) *(f32x4_t*)&S.sums[k0][j][4 * (tid % LPR)] = f32x4_t{acc[j][0], acc[j][1], acc[j][2], acc[j][3]};
    __syncthreads();
    if (c >= W) return;
    // the groups' sums: k0 adds up ranks k0, k0 + kStep ..
#pragma unroll
    for (int j = k0; j < kGradRanks; j += kStep) {
        f32x4_t v = *(const f32x4_t*)&S.sums[0][j][4 * (tid % LPR)];
#pragma unroll
        for (int k = 1; k < kStep; ++k) {
            const f32x4_t o = *(const f32x4_t*)&S.sums[k][j][4 * (tid % LPR)];
#pragma unroll
            for (int q = 0; q < 4; ++q) v[q] += o[q];
        }
        *(f32x4_t*)(out + (size_t)j * W + c) = v;
    }
}
template <int TOKENS, int COLS>
__device__ __forceinline__ void few_tokens_grad_task(const ProjParams& p, const GradParams& g, int id, FewGradShared<TOKENS, COLS>& S) {
    const FewGradTask t(g, id);
    Members mb;
    mb.find(g.T, g.n, p.ids, t.a, S.mask);
    mb.list(0, TOKENS, S.list);
    const float* const h = g.h[t.which];
    const float s = p.scale ? p.scale[t.a] : 1.f;
    few_grad_task(g, t, mb.count(), S, [&](int tok, int j) {
        if (h) return *(const f32x4_t*)(h + (size_t)tok * g.r + j);
        f32x4_t v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
        for (int q = 0; q < p.hsplits; ++q) {
            const f32x4_t u = *(const f32x4_t*)(p.hpart + ((size_t)q * p.T + tok) * p.r + j);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] += u[e];
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] *= s;
        return v;
    });
}

template <int G>
__global__ void __launch_bounds__(256) adapter_few_second_kernel(ProjParams p) {
    __shared__ JoinShared<G> S;
    join_task<G>(p, blockIdx.x % p.T, blockIdx.x / p.T, S);
}
// COLS = 1024: up to kGradRows tokens
template <int G, int COLS>
__global__ void __launch_bounds__(256) adapter_few_second_grad_kernel(ProjParams p, GradParams g, int joins) {
    union Shared {
        JoinShared<G> join;
        FewGradShared<COLS == 1024 ? kGradRows : kFewTokens, COLS> grad;
    };
    __shared__ Shared S;
    const int id = blockIdx.x;
    if (id < joins) join_task<G>(p, id % p.T, id / p.T, S.join);
    else few_tokens_grad_task(p, g, id - joins, S.grad);
}

// ------------------------------------------------------------------ more tokens
// The low-rank rows of tile i (tile_rows rows from tile_rows i on): segments first .. first + count - 1 of the plan.  The tiles before
// it have at most first + i segments together (each may share one with the next), which bounds where it begins.
// A tile with more segments than a quarter of its rows has its low-rank part added row by row instead, after the product: a segment costs the matrix pipe 2 r columns for all
// rows, a row costs the vector unit r of its own (in tiles of 64 x 64 both take as long at some 14 segments, of 256 x 256 at 58).
struct TileLow {
    int first, count, used, ld;   // used, ld: columns; ld a multiple of BK
    bool apart;
    size_t at;                    // first element in hx
};
__device__ __forceinline__ TileLow tile_low(const ProjParams& p, int tile) {
    const int u0 = tile * (p.tile_rows / kUnit), u1 = min((tile + 1) * p.tile_rows, p.T) - 1;
    const int f = p.plan.unit[2 * u0], l = p.plan.unit[2 * (u1 / kUnit) + 1];
    TileLow t;
    t.first = max(f, 0);
    t.count = l < 0 ? 0 : l - t.first + 1;
    t.apart = 4 * t.count > p.tile_rows;
    t.used = t.apart ? 0 : t.count * p.span;
    t.ld = (t.used + BK - 1) / BK * BK;
    t.at = (size_t)p.tile_rows * ((size_t)tile * (p.span + BK) + (size_t)t.first * p.span);
    return t;
}
static size_t hx_bytes(const moe_adapter_shape_t& s, int tile_rows) {
    const size_t tiles = ((size_t)s.T + tile_rows - 1) / tile_rows, segs = (size_t)(s.adapters < s.T ? s.adapters : s.T);
    return 2 * (size_t)tile_rows * (tiles * (3 * (size_t)s.rank + BK) + segs * 3 * (size_t)s.rank);   // (three terms, for an fp32 result)
}

// v as three bf16 terms: the whole 24 bits of an fp32 value
__device__ __forceinline__ void store_terms(uint16_t* to, int r, float (&v)[8]) {
#pragma unroll
    for (int term = 0; term < 3; ++term) {
        float e[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) e[q] = bf16_round(v[q]);
        *(u32x4_t*)(to + term * r) = pack8f(e);
#pragma unroll
        for (int q = 0; q < 8; ++q) v[q] = fabsf(e[q]) < INFINITY ? v[q] - e[q] : 0.f;   // (an infinite value stays one)
    }
}
// h of one block of the plan, as fp32 and as the rows of its tile's low-rank part; behind the blocks, where the factors are wanted
// transposed, 64 columns of one adapter's a workgroup.
template <int NRF, int NCF>
__global__ void __launch_bounds__(kSmallThreads) adapter_low_kernel(ProjParams p) {
    using S = SmallTile<NRF, NCF>;
    __shared__ __attribute__((aligned(512))) char smem[S::kLds];
    const int tid = threadIdx.x;
    if ((int)blockIdx.x >= p.blocks) {
        const int id = blockIdx.x - p.blocks, tiles = (p.C + 63) / 64, a = id / tiles, c0 = id % tiles * 64;
        if (p.plan.start[a] == p.plan.start[a + 1]) return;
        // (a rank's 64 columns as 128 bytes; 2 bytes a lane on both sides of the turn are 4 MB at 64 ranks of 4096 columns and 8 adapters)
        uint16_t(*s)[66] = (uint16_t(*)[66])smem;   // [r][64]
        const uint16_t* from = (const uint16_t*)p.second + (size_t)a * p.r * p.C + c0;
        for (int i = tid; i < p.r * 64; i += kSmallThreads)
            if (c0 + (i & 63) < p.C) s[i >> 6][i & 63] = from[(size_t)(i >> 6) * p.C + (i & 63)];
        __syncthreads();
        uint16_t* to = (uint16_t*)p.second_t + ((size_t)a * p.C + c0) * p.r;
        for (int i = tid; i < p.r * 64; i += kSmallThreads) {
            const int c = i / p.r, j = i - c * p.r;
            if (c0 + c < p.C) to[i] = s[j][c];
        }
        return;
    }
    // every XCD a run of the blocks: those of one adapter fetch its factor into one L2
    const int nb = p.plan.head[0], per = (nb + 7) >> 3, slot = blockIdx.x >> 3, blk = (blockIdx.x & 7) * per + slot;
    if (slot >= per || blk >= nb) return;
    const int row0 = p.plan.block[2 * blk], code = p.plan.block[2 * blk + 1], rows = code & 255, a = (code >> 8) - 1;
    const int tile = row0 / p.tile_rows;
    const TileLow tl = tile_low(p, tile);
    uint16_t* const hx = (uint16_t*)p.hx + tl.at + (size_t)(row0 - tile * p.tile_rows) * tl.ld;
    const int own = a < 0 ? -1 : (p.plan.ordinal[a] - tl.first) * p.span;   // first column of its segment
    for (int i = tid; i < rows * (tl.ld / 8); i += kSmallThreads) {
        const int row = i / (tl.ld / 8), col = 8 * (i - row * (tl.ld / 8));
        if (a < 0 || col < own || col >= own + p.span) *(u32x4_t*)(hx + (size_t)row * tl.ld + col) = zero4();
    }
    if (a < 0) {
        for (int i = tid; i < rows * p.r; i += kSmallThreads) p.h[(size_t)p.plan.order[row0 + i / p.r] * p.r + i % p.r] = 0.f;
        return;
    }
    const Stages st = stages_of(p.R);
    if (p.terms[0])
        for (int i = tid; i < rows * (p.r / 8); i += kSmallThreads) {
            const int row = i / (p.r / 8), col = 8 * (i - row * (p.r / 8));
            const f32x4_t* q = (const f32x4_t*)(p.h_given + (size_t)p.plan.order[row0 + row] * p.r + col);
            float v[8];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                v[j] = q[0][j];
                v[4 + j] = q[1][j];
            }
            store_terms(p.terms[0] + (size_t)(row0 + row) * 3 * p.r + col, p.r, v);
        }
    const float s = p.scale ? p.scale[a] : 1.f;
    // (one copy of what is done with a value, for both ways to it: a launch this short waits for its instructions too)
    const bool dots = rows <= kDotTokens;
    float(*const d)[kMaxRank] = (float(*)[kMaxRank])smem;
    if (dots) {
        few_dots(p, a, 0, p.r, rows, 0, p.R, [&](int m) { return p.plan.order[row0 + m]; }, [&](int m, int j, float v) { d[m][j] = v; });
    } else {
        f32x16_t acc[NRF][NCF];
        const Lane ln;
        KcStages<NRF, false> lb;
        lb.init(ln, rows, st, [&](int r) { return p.x + (size_t)p.plan.order[row0 + r] * p.ldx; });
        lb.low.used = 0;
        KcStages<NCF, true> la;
        la.init(ln, p.r, st, [&](int j) { return p.first + ((size_t)a * p.r + j) * p.R * 2; });
        small_loop<NRF, NCF, kKc>(lb, la, st.full + (st.tail > 0), smem, acc);
        small_put(smem, acc);
    }
    __syncthreads();
#pragma unroll 1
    for (int i = tid; i < rows * (p.r / 8); i += kSmallThreads) {
        const int row = i / (p.r / 8), col = 8 * (i - row * (p.r / 8));
        float h[8], e[8], l[8];
        if (dots) {
#pragma unroll
            for (int j = 0; j < 8; ++j) h[j] = d[row][col + j];
        } else {
            small_get<NRF, NCF>(smem, row, col >> 3, h);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            h[j] *= s;
            e[j] = bf16_round(h[j]);
            l[j] = fabsf(e[j]) < INFINITY ? h[j] - e[j] : 0.f;   // an infinite h stays one
        }
        f32x4_t* to = (f32x4_t*)(p.h + (size_t)p.plan.order[row0 + row] * p.r + col);
        to[0] = f32x4_t{h[0], h[1], h[2], h[3]};
        to[1] = f32x4_t{h[4], h[5], h[6], h[7]};
        const u32x4_t hi = pack8f(e), lo = pack8f(l);
#pragma unroll
        for (int j = 0; j < 8; ++j) l[j] = fabsf(e[j]) < INFINITY ? l[j] - bf16_round(l[j]) : 0.f;
        const u32x4_t rest = pack8f(l);   // the third term: what the first two leave
        if (!tl.apart) {
            uint16_t* x = hx + (size_t)row * tl.ld + own + col;
            *(u32x4_t*)x = hi;
            *(u32x4_t*)(x + p.r) = lo;
            if (p.span > 2 * p.r) *(u32x4_t*)(x + 2 * p.r) = rest;
        }
        if (p.terms[1]) {
            uint16_t* x = p.terms[1] + (size_t)(row0 + row) * 3 * p.r + col;
            *(u32x4_t*)x = hi;
            *(u32x4_t*)(x + p.r) = lo;
            *(u32x4_t*)(x + 2 * p.r) = rest;
        }
    }
}

// The second launch where the product is cut into parts (parts_pay): y of up to 16 rows of the plan and 1024 columns, 4 a thread, and with the first
// columns h and the gradients' terms, as adapter_low_kernel writes them.
constexpr int kPartsRows = 16;
__global__ void __launch_bounds__(256) adapter_parts_join_kernel(ProjParams p) {
    __shared__ float s_h[kPartsRows][kMaxRank];
    __shared__ int32_t s_tok[kPartsRows], s_a[kPartsRows];
    const int tid = threadIdx.x, groups = (p.T + p.join_rows - 1) / p.join_rows, row0 = (int)blockIdx.x % groups * p.join_rows, cb = (int)blockIdx.x / groups;
    const int rows = min(p.join_rows, p.T - row0);
    if (tid < rows) {
        const int t = p.plan.order[row0 + tid];
        s_tok[tid] = t;
        s_a[tid] = adapter_of(p.ids, t, p.n);
    }
    __syncthreads();
#pragma unroll 1
    for (int i = tid; i < rows * (p.r / 8); i += 256) {
        const int m = i / (p.r / 8), col = 8 * (i - m * (p.r / 8)), t = s_tok[m], a = s_a[m];
        float v[8] = {};
        if (a >= 0) {
            const float* const q = p.hpart + (size_t)t * p.r + col;
#pragma unroll 4
            for (int k = 0; k < p.hsplits; ++k) {
                const f32x4_t* const u = (const f32x4_t*)(q + (size_t)k * p.T * p.r);
                const f32x4_t x = u[0], y = u[1];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    v[j] += x[j];
                    v[4 + j] += y[j];
                }
            }
            const float s = p.scale ? p.scale[a] : 1.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] *= s;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) s_h[m][col + j] = v[j];
        if (cb == 0) {
            f32x4_t* const to = (f32x4_t*)(p.h + (size_t)t * p.r + col);
            to[0] = f32x4_t{v[0], v[1], v[2], v[3]};
            to[1] = f32x4_t{v[4], v[5], v[6], v[7]};
            if (p.terms[0]) {
                const size_t at = (size_t)(row0 + m) * 3 * p.r + col;
                store_terms(p.terms[1] + at, p.r, v);
                const f32x4_t* const g = (const f32x4_t*)(p.h_given + (size_t)t * p.r + col);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    v[j] = g[0][j];
                    v[4 + j] = g[1][j];
                }
                store_terms(p.terms[0] + at, p.r, v);
            }
        }
    }
    __syncthreads();
    const int wide = min(256, (p.C + 3) / 4), m = tid / wide, c = (cb * 256 + tid % wide) * 4;
    if (m >= rows || c >= p.C) return;
    const int t = s_tok[m], a = s_a[m];
    float acc[4] = {};
    const float* const part = p.part + (size_t)t * p.C + c;
#pragma unroll 8
    for (int k = 0; k < p.splits; ++k) {
        const f32x4_t u = *(const f32x4_t*)(part + (size_t)k * p.T * p.C);
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[j] += u[j];
    }
    if (a >= 0) {
        const char* const f = p.second + ((size_t)a * p.r * p.C + c) * 2;
#pragma unroll 8
        for (int j = 0; j < p.r; ++j) fma4(acc, s_h[m][j], *(const u32x2_t*)(f + (size_t)j * p.C * 2));
    }
    const size_t at = (size_t)t * p.C + c;
    if (p.out_f32) *(f32x4_t*)(p.y + at * 4) = f32x4_t{acc[0], acc[1], acc[2], acc[3]};
    else *(u32x2_t*)(p.y + at * 2) = u32x2_t{pack_bf16x2(acc[0], acc[1]), pack_bf16x2(acc[2], acc[3])};
}

// sum_j h[j] second[a][j][col ..]: the low-rank part of 8 columns of one row, for tiles with many adapters (tile_low's `apart`) and those in which something is not finite
__device__ __forceinline__ void add_low(const ProjParams& p, int row, int col, float (&v)[8]) {
    const int t = p.plan.order[row], a = adapter_of(p.ids, t, p.n);
    if (a < 0) return;
    for (int j = 0; j < p.r; ++j) fma8(v, p.h[(size_t)t * p.r + j], *(const u32x4_t*)(p.second + (((size_t)a * p.r + j) * p.C + col) * 2));
}
__device__ __forceinline__ void store_y(const ProjParams& p, int row, int col, const float (&v)[8]) {
    const size_t at = (size_t)p.plan.order[row] * p.C + col;
    if (p.out_f32) {
        f32x4_t* to = (f32x4_t*)(p.y + at * 4);
        to[0] = f32x4_t{v[0], v[1], v[2], v[3]};
        to[1] = f32x4_t{v[4], v[5], v[6], v[7]};
    } else {
        *(u32x4_t*)(p.y + at * 2) = pack8f(v);
    }
}
__device__ __forceinline__ bool all_finite(const f32x16_t& a) {
    // (a sum of 0 v: 0 where every v is finite, else NaN)
    float s = 0.f;
#pragma unroll
    for (int v = 0; v < 16; ++v) s += 0.f * a[v];
    return s == 0.f;
}
__device__ __forceinline__ LowRank low_of(const ProjParams& p, const TileLow& t, bool transposed) {
    return LowRank{p.hx + t.at * 2, (uint32_t)t.ld * 2, transposed ? p.second_t : p.second, p.plan.seg + t.first, t.used, p.span, p.r, p.C};
}

// Which tile a workgroup has.  Workgroups go to the eight XCDs in turn; each XCD gets a run of the tiles in an order that has 8 row tiles
// innermost, so that what it has at a time is about 8 x 4 tiles that meet in its L2.
struct TileId {
    int rt, ct;
    __device__ __forceinline__ TileId(const ProjParams& p) {
        const int n = p.row_tiles * p.col_tiles, x = blockIdx.x & 7, slot = blockIdx.x >> 3, per = n >> 3, more = n & 7;
        const int id = x * per + min(x, more) + slot;   // (XCD x has per tiles, the first `more` one more: as many workgroups as go there)
        const int group = 8 * p.col_tiles, g = id / group, in = id - g * group, rows = min(8, p.row_tiles - 8 * g);
        ct = in / rows;
        rt = 8 * g + in - ct * rows;
    }
};

// Tiles of 64 x 64 and of 128 x 128.
// A factor with an infinity or NaN must not reach the rows of other adapters, but 0 times it would: a tile whose sums are not all finite
// is computed again without its low-rank part, which is then added row by row (as is one where x or W is not finite).
template <int FORM, bool MID>
__global__ void __launch_bounds__(MID ? kMidThreads : kSmallThreads) adapter_tile_kernel(ProjParams p) {
    constexpr int kTile = MID ? 128 : 64;
    __shared__ __attribute__((aligned(512))) char smem[MID ? MidTile::kLds : SmallTile<2, 2>::kLds];
    __shared__ int s_bad;
    const TileId at(p);
    const int rt = at.rt, ct = at.ct;
    const int row0 = rt * kTile, rows = min(kTile, p.T - row0), col0 = ct * kTile;
    const TileLow tl = tile_low(p, rt);
    const Stages st = stages_of(p.R);
    const int dense = st.full + (st.tail > 0);
    if (threadIdx.x == 0) s_bad = tl.apart;
    f32x16_t acc[2][2];
#pragma unroll 1
    for (int low = !tl.apart;; low = 0) {
        {
            const Lane ln;
            KcStages<2, false> lb;
            lb.init(ln, rows, st, [&](int r) { return p.x + (size_t)p.plan.order[row0 + r] * p.ldx; });
            lb.low = low_of(p, tl, FORM == kKc);
            const int nk = dense + (low ? tl.ld / BK : 0);
            if constexpr (FORM == kKs) {
                KsStages<2, kTile> la;
                la.init(ln, p.w, col0, p.C, st);
                la.low = lb.low;
                if constexpr (MID) mid_loop<kKs>(lb, la, nk, smem, acc);
                else small_loop<2, 2, kKs>(lb, la, nk, smem, acc);
            } else {
                KcStages<2, true> la;
                la.init(ln, min(kTile, p.C - col0), st, [&](int c) { return p.w + (size_t)(col0 + c) * p.R * 2; });
                la.low = lb.low;
                la.first = col0;
                if constexpr (MID) mid_loop<kKc>(lb, la, nk, smem, acc);
                else small_loop<2, 2, kKc>(lb, la, nk, smem, acc);
            }
        }
        if (!low || tl.count == 0) break;
        const bool ok = all_finite(acc[0][0]) && all_finite(acc[0][1]) && all_finite(acc[1][0]) && all_finite(acc[1][1]);
        if (!ok) s_bad = 1;
        __syncthreads();
        if (!s_bad) break;
    }
    const bool bad = s_bad;
    auto store = [&](int row, int col, float (&v)[8]) {
        col += col0;
        if (row >= rows || col >= p.C) return;
        if (bad) add_low(p, row0 + row, col, v);
        store_y(p, row0 + row, col, v);
    };
    if constexpr (MID) mid_sum(smem, acc, store);
    else small_sum<2, 2>(smem, acc, store);
}

// Tiles of 256 columns and up to 256 rows (mma.hpp's loops).
template <int FORM, class LA>
__device__ __forceinline__ void big_gemm(const ProjParams& p, LA& la, const Lane& ln, int row0, int rows, Stages st, const LowRank& low, int nk, char* smem,
                                         Acc& acc) {
    FragAddr fa;
    frag_addresses<FORM, false>(fa, lds_addr(smem), ln);
    auto row_of = [&](int r) { return p.x + (size_t)p.plan.order[row0 + r] * p.ldx; };
    zero_acc(acc, false);
    const int ntf = active_row_frags(rows);
    if (rows <= kLowRows) {
        KcStages<2, false> lb;
        lb.init(ln, rows, st, row_of);
        lb.low = low;
        if (ntf > 2) mma_low<4, FORM>(lb, la, nk, smem, fa, acc);
        else if (ntf > 0) mma_low<2, FORM>(lb, la, nk, smem, fa, acc);
        else mma_low<0, FORM>(lb, la, nk, smem, fa, acc);
    } else {
        KcStages<4, false> lb;
        lb.init(ln, rows, st, row_of);
        lb.low = low;
        if (ntf > 2) mma_loop<4, 0, FORM, false>(lb, la, nk, smem, fa, acc);
        else mma_loop<2, 0, FORM, false>(lb, la, nk, smem, fa, acc);
    }
}
template <int FORM>
__global__ void __launch_bounds__(kMmaThreads) __attribute__((amdgpu_waves_per_eu(2, 2))) adapter_big_kernel(ProjParams p) {
    __shared__ __attribute__((aligned(512))) char smem[kMmaSmem];
    __shared__ int s_bad;
    const TileId at(p);
    const int rt = at.rt, ct = at.ct;
    const int row0 = rt * p.tile_rows, rows = min(p.tile_rows, p.T - row0), col0 = ct * BN;
    const TileLow tl = tile_low(p, rt);
    const Stages st = stages_of(p.R);
    const int dense = st.full + (st.tail > 0);
    if (threadIdx.x == 0) s_bad = tl.apart;
    Acc acc;
#pragma unroll 1
    for (int low = !tl.apart;; low = 0) {
        const Lane ln;
        const LowRank lr = low_of(p, tl, FORM == kKc);
        const int nk = dense + (low ? tl.ld / BK : 0);
        if constexpr (FORM == kKs) {
            KsStages<4, 256> la;
            la.init(ln, p.w, col0, p.C, st);
            la.low = lr;
            big_gemm<kKs>(p, la, ln, row0, rows, st, lr, nk, smem, acc);
        } else {
            KcStages<4, true> la;
            la.init(ln, min(BN, p.C - col0), st, [&](int c) { return p.w + (size_t)(col0 + c) * p.R * 2; });
            la.low = lr;
            la.first = col0;
            big_gemm<kKc>(p, la, ln, row0, rows, st, lr, nk, smem, acc);
        }
        if (!low || tl.count == 0) break;
        bool ok = true;
#pragma unroll
        for (int tf = 0; tf < 4; ++tf) ok = ok && all_finite(acc.a[tf][0]) && all_finite(acc.a[tf][1]);
        if (!ok) s_bad = 1;
        __syncthreads();
        if (!s_bad) break;
    }
    if (!s_bad && !p.out_f32) {
        store_subtile_bf16<false>(acc, smem, rows, p.C - col0, [&](int row, int col, u32x4_t v) {
            *(u32x4_t*)(p.y + ((size_t)p.plan.order[row0 + row] * p.C + col0 + col) * 2) = v;
        });
        return;
    }
    const Lane ln;
    const bool bad = s_bad;
#pragma unroll
    for (int tf = 0; tf < 4; ++tf)
#pragma unroll
        for (int af = 0; af < 2; ++af)
#pragma unroll
            for (int vg = 0; vg < 2; ++vg) {
                const int row = acc_row(ln, tf), col = col0 + acc_col8(ln, af, vg);
                float v[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = acc.a[tf][af][8 * vg + j];
                if (row < rows && col < p.C) {
                    if (bad) add_low(p, row0 + row, col, v);
                    store_y(p, row0 + row, col, v);
                }
            }
}

// ------------------------------------------------------------------ gradients of the factors, more tokens
// out[a][j][c] = sum over the adapter's rows of h[row][j] x[row][c]: h as three bf16 terms (the sums are returned in fp32; adapter_low_kernel
// has written them row by row), x as it is.  A stage is 64 rows; both operands are KS images, x gathered through the plan; wave w
// takes k-sub-step w of a stage for the whole tile of 32 NRF ranks by 32 NCF columns, as in small_loop.  Rows at and past the last come from the page of zeros.
template <int NRF, int NCF>
struct GradTile {
    static constexpr int kXRow = 64 * NCF, kHRow = 64 * NRF;
    static constexpr int kX = BK * kXRow, kH = BK * kHRow, kStage = kX + 3 * kH;
    static constexpr int kDepth = NRF == 4 ? 2 : 3;
    static constexpr int kSums = 16384 * NCF;   // one fragment of ranks at a time
    static constexpr int kLds = kDepth * kStage > kSums ? kDepth * kStage : kSums;
    static constexpr int kXLoads = kX / 4096, kHLoads = 3 * kH / 4096;   // DMA instructions of a wave
    static constexpr int kList = 2048;          // rows whose tokens are in LDS
};
// swizzle of a KS image with rows of `bytes`
template <int BYTES>
__device__ __forceinline__ int ks_swz(int k) { return BYTES == 64 ? 0 : BYTES == 128 ? (k & 2) << 1 : (k & 3) << 2; }
// N fragments by transposing reads; a fragment's second half lies NEXT bytes behind its first
template <int N, int NEXT>
__device__ __forceinline__ void read_tr(u32x4_t (&f)[N], const uint32_t (&at)[N], uint32_t off) {
    u32x2_t lo[N], hi[N];
    if constexpr (N == 4) {
        const uint32_t a0 = at[0] + off, a1 = at[1] + off, a2 = at[2] + off, a3 = at[3] + off;
        asm volatile("ds_read_b64_tr_b16 %0, %8\n ds_read_b64_tr_b16 %1, %8 offset:%12\n ds_read_b64_tr_b16 %2, %9\n ds_read_b64_tr_b16 %3, %9 offset:%12\n"
                     "ds_read_b64_tr_b16 %4, %10\n ds_read_b64_tr_b16 %5, %10 offset:%12\n ds_read_b64_tr_b16 %6, %11\n ds_read_b64_tr_b16 %7, %11 offset:%12\n"
                     "s_waitcnt lgkmcnt(0)"
                     : "=&v"(lo[0]), "=&v"(hi[0]), "=&v"(lo[1]), "=&v"(hi[1]), "=&v"(lo[2]), "=&v"(hi[2]), "=&v"(lo[3]), "=&v"(hi[3])
                     : "v"(a0), "v"(a1), "v"(a2), "v"(a3), "n"(NEXT) : "memory");
    } else if constexpr (N == 2) {
        const uint32_t a0 = at[0] + off, a1 = at[1] + off;
        asm volatile("ds_read_b64_tr_b16 %0, %4\n ds_read_b64_tr_b16 %1, %4 offset:%6\n ds_read_b64_tr_b16 %2, %5\n ds_read_b64_tr_b16 %3, %5 offset:%6\n"
                     "s_waitcnt lgkmcnt(0)"
                     : "=&v"(lo[0]), "=&v"(hi[0]), "=&v"(lo[1]), "=&v"(hi[1]) : "v"(a0), "v"(a1), "n"(NEXT) : "memory");
    } else {
        const uint32_t a0 = at[0] + off;
        asm volatile("ds_read_b64_tr_b16 %0, %2\n ds_read_b64_tr_b16 %1, %2 offset:%3\n s_waitcnt lgkmcnt(0)"
                     : "=&v"(lo[0]), "=&v"(hi[0]) : "v"(a0), "n"(NEXT) : "memory");
    }
#pragma unroll
    for (int i = 0; i < N; ++i) f[i] = u32x4_t{lo[i][0], lo[i][1], hi[i][0], hi[i][1]};
}

// How the adapters' rows are cut, where g.parts allows it: those with rows (g.few: with more than kGradRows) are known only here, and a batch may be on few of many.  As many parts as give
// every CU a tile, of 512 rows at least; active * eff * tiles <= 256 where eff > 1.
struct GradCut {
    int active, eff;
    __device__ __forceinline__ GradCut(const GradParams& g, const int32_t* head)
        : active(g.few ? head[1] : head[2]), eff(g.parts > 1 ? max(1, min(g.parts, 256 / ((g.col_tiles[0] + g.col_tiles[1]) * max(active, 1)))) : 1) {}
    __device__ __forceinline__ int rows(int count) const { return max(512, ((count + eff - 1) / eff + BK - 1) / BK * BK); }
    __device__ __forceinline__ int pieces(int count) const { return eff > 1 ? (count + rows(count) - 1) / rows(count) : 1; }
};

// Waves 0..3 multiply, waves 4..7 only move operands: with one wave a SIMD for both, its requests (ten a stage, each with an address of its own)
// and its products were done one after the other.
constexpr int kGradThreads = 2 * kSmallThreads;
// g.few: adapters with up to kGradRows rows are left to adapter_grad_rows_kernel.
template <int NRF, int NCF>
__global__ void __launch_bounds__(kGradThreads) adapter_grad_kernel(ProjParams p, GradParams g) {
    using G = GradTile<NRF, NCF>;
    __shared__ __attribute__((aligned(512))) char smem[G::kLds];
    __shared__ int32_t s_tok[G::kList];
    const int tid = threadIdx.x;
    // every XCD a run of the column tiles, adapter by adapter: its workgroups share one adapter's h in their L2, however unlike the adapters are
    const int tiles = g.col_tiles[0] + g.col_tiles[1], per = (tiles + 7) >> 3, slot = blockIdx.x >> 3;
    const GradCut cut(g, p.plan.head);
    const int at = slot / per / cut.eff, piece = slot / per - at * cut.eff;
    if ((g.few || g.parts > 1) && at >= cut.active) return;   // (without rows: left to adapter_grad_rows_kernel or adapter_grad_sum_kernel)
    const int a = g.few ? p.plan.many[at] : g.parts > 1 ? p.plan.seg[at] : at;
    int ct = (blockIdx.x & 7) * per + slot % per;
    if (ct >= tiles) return;
    const int which = ct < g.col_tiles[0] ? 0 : 1;
    if (which) ct -= g.col_tiles[0];
    const int W = g.W[which], c0 = ct * 32 * NCF, r = g.r;
    int row0 = p.plan.start[a], count = p.plan.start[a + 1] - row0;
    float* out = g.out[which] + (size_t)a * r * W;
    if (cut.eff > 1) {
        const int rows = cut.rows(count);
        if (piece * rows >= count) return;
        if (rows < count) out = g.part[which] + (size_t)(at * cut.eff + piece) * r * W;
        row0 += piece * rows;
        count = min(rows, count - piece * rows);
    }
    const Lane ln;
    const int wave = ln.wave_uniform() & 3;
    const bool moves = ln.wave_uniform() >= 4;
    // x: an instruction moves kXRows rows of kXLanes lanes
    constexpr int kXLanes = 4 * NCF, kXRows = 64 / kXLanes, kHLanes = 4 * NRF, kHRows = 64 / kHLanes;
    const int xk = kXRows * G::kXLoads * wave + ln.l / kXLanes;                                  // (+ kXRows i)
    const int xc = (ln.l % kXLanes) ^ ks_swz<G::kXRow>(ln.l / kXLanes);                          // (kXRows is 4 or 8: it does not depend on i)
    const char* const x = g.x[which] + (size_t)min(c0 + 8 * xc, W - 8) * 2;
    const size_t ldx = g.ldx[which];
    const char* const h = (const char*)(p.terms[which] + (size_t)row0 * 3 * r);
    const uint32_t tok0 = lds_addr(s_tok) + xk * 4;
    // h: this lane's row of instruction i, and its chunk from the first row of the stage on
    auto h_row = [&](int i) { return ((G::kHLoads * wave + i) % (4 * NRF)) * kHRows + ln.l / kHLanes; };
    auto h_off = [&](int i) {
        const int k = h_row(i), c = (ln.l % kHLanes) ^ ks_swz<G::kHRow>(k);
        return (k * 3 + (G::kHLoads * wave + i) / (4 * NRF)) * r * 2 + min(c * 16, 2 * r - 16);
    };
    uint32_t oh[G::kHLoads];
#pragma unroll
    for (int i = 0; i < G::kHLoads; ++i) oh[i] = h_off(i);
    auto issue = [&](int k0, int left, char* dst) {   // the 64 rows from row k0 on, of which `left` are there
        int32_t tok[G::kXLoads];
        const uint32_t at = tok0 + (k0 % G::kList) * 4;
        if constexpr (G::kXLoads == 4)
            asm volatile("ds_read_b32 %0, %4\n ds_read_b32 %1, %4 offset:%5\n ds_read_b32 %2, %4 offset:%6\n ds_read_b32 %3, %4 offset:%7\n s_waitcnt lgkmcnt(0)"
                         : "=&v"(tok[0]), "=&v"(tok[1]), "=&v"(tok[2]), "=&v"(tok[3]) : "v"(at), "n"(kXRows * 4), "n"(kXRows * 8), "n"(kXRows * 12) : "memory");
        else
            asm volatile("ds_read_b32 %0, %2\n ds_read_b32 %1, %2 offset:%3\n s_waitcnt lgkmcnt(0)" : "=&v"(tok[0]), "=&v"(tok[1]) : "v"(at), "n"(kXRows * 4) : "memory");
        char* const dx = dst + G::kXLoads * 1024 * wave;
        char* const dh = dst + G::kX + G::kHLoads * 1024 * wave;
        const char* const hs = h + (size_t)k0 * 6 * r;
        if (left >= BK) {
#pragma unroll
            for (int i = 0; i < G::kXLoads; ++i) dma16(x + (size_t)tok[i] * ldx, dx + i * 1024);
#pragma unroll
            for (int i = 0; i < G::kHLoads; ++i) dma16(hs + oh[i], dh + i * 1024);
        } else {
#pragma unroll
            for (int i = 0; i < G::kXLoads; ++i) dma16(xk + i * kXRows < left ? x + (size_t)tok[i] * ldx : zero_chunk(), dx + i * 1024);
#pragma unroll
            for (int i = 0; i < G::kHLoads; ++i) dma16(h_row(i) < left ? hs + oh[i] : zero_chunk(), dh + i * 1024);
        }
    };
    f32x16_t acc[NRF][NCF];
#pragma unroll
    for (int tf = 0; tf < NRF; ++tf)
#pragma unroll
        for (int af = 0; af < NCF; ++af)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[tf][af][v] = 0.f;
    // fragments: x columns in the A role, ranks in the B role
    const int gg = (ln.l >> 4) & 1, e = (ln.l & 15) >> 2, q4 = ln.l & 3, sq = ((q4 & 1) << 1) | (q4 >> 1), krow = 16 * wave + 8 * ln.hf + e;
    uint32_t ax[NCF], ah[NRF];
#pragma unroll
    for (int af = 0; af < NCF; ++af)
        ax[af] = lds_addr(smem) + krow * G::kXRow + (((4 * af + 2 * gg + (sq >> 1)) ^ ks_swz<G::kXRow>(e)) << 4) + (sq & 1) * 8;
#pragma unroll
    for (int tf = 0; tf < NRF; ++tf)
        ah[tf] = lds_addr(smem) + G::kX + krow * G::kHRow + (((4 * tf + 2 * gg + (q4 >> 1)) ^ ks_swz<G::kHRow>(e)) << 4) + (q4 & 1) * 8;
    // (both roles meet at the same barriers: two for each list, one for each stage)
    if (moves) {
        for (int base = 0; base < count; base += G::kList) {
            const int here = min(G::kList, count - base), nst = (here + BK - 1) / BK;
            __syncthreads();   // the stages of the list before have been read
            for (int i = tid - kSmallThreads; i < here; i += kSmallThreads) s_tok[i] = p.plan.order[row0 + base + i];
            __syncthreads();
            for (int t = 0; t < min(G::kDepth - 1, nst); ++t) issue(base + t * BK, here - t * BK, smem + t * G::kStage);
            int next = (G::kDepth - 1) * G::kStage;
            for (int t = 0; t < nst; ++t) {
                if (t + G::kDepth - 2 < nst) asm volatile("s_waitcnt vmcnt(%0)" ::"n"((G::kDepth - 2) * (G::kXLoads + G::kHLoads)) : "memory");
                else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
                __builtin_amdgcn_s_barrier();   // stage t is here, and stage t - 1 has been read
                if (t + G::kDepth - 1 < nst) {
                    issue(base + (t + G::kDepth - 1) * BK, here - (t + G::kDepth - 1) * BK, smem + next);
                    next = next == (G::kDepth - 1) * G::kStage ? 0 : next + G::kStage;
                }
            }
        }
    } else {
        for (int base = 0; base < count; base += G::kList) {
            const int nst = (min(G::kList, count - base) + BK - 1) / BK;
            __syncthreads();
            __syncthreads();
            int at = 0;
            for (int t = 0; t < nst; ++t) {
                __builtin_amdgcn_s_barrier();
                u32x4_t fx[NCF];
                read_tr<NCF, 4 * G::kXRow>(fx, ax, at);
#pragma unroll
                for (int term = 0; term < 3; ++term) {
                    u32x4_t fh[NRF];
                    read_tr<NRF, 4 * G::kHRow>(fh, ah, at + term * G::kH);
                    mfma_tile(fh, fx, acc);
                }
                at = at == (G::kDepth - 1) * G::kStage ? 0 : at + G::kStage;
            }
        }
    }
#pragma unroll
    for (int tf = 0; tf < NRF; ++tf) {
        __syncthreads();
        small_sum<1, NCF, kGradThreads>(smem, *(const f32x16_t(*)[1][NCF])&acc[tf], [&](int row, int col, const float (&v)[8]) {
            row += 32 * tf;
            col += c0;
            if (row >= r || col >= W) return;
            f32x4_t* to = (f32x4_t*)(out + (size_t)row * W + col);
            to[0] = f32x4_t{v[0], v[1], v[2], v[3]};
            to[1] = f32x4_t{v[4], v[5], v[6], v[7]};
        });
    }
}
// The parts' sums, first part first, and zeros for adapters without rows (g.few: adapter_grad_rows_kernel's).
__global__ void __launch_bounds__(256) adapter_grad_sum_kernel(PlanView plan, GradParams g) {
    const GradCut cut(g, plan.head);
    if (g.few && (int)blockIdx.y >= cut.active) return;
    const int a = g.few ? plan.many[blockIdx.y] : blockIdx.y, at = g.few ? blockIdx.y : plan.ordinal[a];
    const int count = plan.start[a + 1] - plan.start[a], pieces = cut.pieces(count);
    if (pieces == 1 && count > 0) return;
    const int n0 = g.r * g.W[0] / 4, n1 = g.r * g.W[1] / 4;
    int i = blockIdx.x * 256 + threadIdx.x;
    const int which = i < n0 ? 0 : 1;
    if (which) i -= n0;
    const int n = which ? n1 : n0;
    if (i >= n) return;
    f32x4_t v = {0.f, 0.f, 0.f, 0.f};
    if (count > 0) {
        const f32x4_t* const q = (const f32x4_t*)g.part[which] + (size_t)at * cut.eff * n + i;
        v = q[0];
#pragma unroll 8
        for (int k = 1; k < pieces; ++k) {
            const f32x4_t u = q[(size_t)k * n];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] += u[e];
        }
    }
    ((f32x4_t*)g.out[which])[(size_t)a * n + i] = v;
}

// The same for adapters with up to kGradRows rows, on the vector unit: a workgroup of the tiles above takes 6 us whatever its rows and has a CU for itself (a training step of 512 tokens on
// 200 adapters of 680 x 480, 16 ranks, 112 us, of 600 with this and the low-rank parts row by row 85).
__global__ void __launch_bounds__(256) adapter_grad_rows_kernel(ProjParams p, GradParams g) {
    __shared__ FewGradShared<kGradRows, 1024> S;
    const FewGradTask t(g, blockIdx.x);
    const int row0 = p.plan.start[t.a], count = p.plan.start[t.a + 1] - row0;
    if (count > kGradRows) return;
    if ((int)threadIdx.x < count) S.list[threadIdx.x] = p.plan.order[row0 + threadIdx.x];
    __syncthreads();
    const float* const h = g.h[t.which];
    few_grad_task(g, t, count, S, [&](int tok, int j) { return *(const f32x4_t*)(h + (size_t)tok * g.r + j); });
}

// ------------------------------------------------------------------ launches
constexpr int kMostSplits = 16;
static int stages_in(int R) { return (R + BK - 1) / BK; }
struct FewPlan {
    int row_frags, col_tiles, row_tiles, rank_tiles, hgroups, dot_cut, splits, per_split, hsplits, hper_split;
};
// Parts of at least 4 stages, as many as give every CU a workgroup but no more than the second launch fetches in two goes; h is cut alike, or into fewer parts where every token may be a group of its own.
static FewPlan few_plan(int T, int R, int C, int r, int n, int blocks = 0) {
    FewPlan f;
    f.row_frags = T <= 32 ? 1 : 2;
    f.col_tiles = (C + 63) / 64;
    f.row_tiles = (T + 32 * f.row_frags - 1) / (32 * f.row_frags);
    f.rank_tiles = (r + 63) / 64;
    const int nst = stages_in(R), tiles = f.col_tiles * f.row_tiles;
    const int want = std::max(1, 256 / tiles);
    f.per_split = std::max({4, (nst + want - 1) / want, (nst + kMostSplits - 1) / kMostSplits});
    f.splits = (nst + f.per_split - 1) / f.per_split;
    f.hgroups = blocks > 0 ? blocks : (int)std::min((long long)T, (long long)n * ((T + 31) / 32));
    f.hper_split = std::max(std::min(f.per_split, 16), (int)(((long long)nst * f.hgroups * f.rank_tiles + 511) / 512));
    f.hsplits = (nst + f.hper_split - 1) / f.hper_split;
    // dots of many ranks: 16 a workgroup (one turn of its waves) while there are up to 512 workgroups.  First launch, us, 64 ranks a workgroup / cut while there are 256, 512, 1024 (tokens, K, N, ranks,
    // adapters): 9, 912, 448, 128, 4 14.1 / 7.4 with 256; 100, 1024, 1024, 64, 200 18.0 / 18.0, 14.0, 14.9; 60, 2048, 2048, 64, 60 19.8 / 19.4, 16.6, 18.6.
    f.dot_cut = 1;
    while (T <= kDotTokens * n && 64 / f.dot_cut > 16 && r > 64 / f.dot_cut / 2 && (long long)f.hgroups * f.rank_tiles * f.hsplits * f.dot_cut <= 512) f.dot_cut *= 2;
    return f;
}
static size_t few_bytes(int T, int R, int C, int r, int n, int blocks = 0) {
    const FewPlan f = few_plan(T, R, C, r, n, blocks);
    return align_up((size_t)f.splits * T * C * 4, 256) + align_up((size_t)f.hsplits * T * r * 4, 256);
}
// Tiles of the product.  A stage of 64 k takes about 0.38 us in tiles of 64 x 64 (two on a CU), 0.6 in tiles of 128 x 128, 1.0 in 128 x 256 and 1.45 in 256 x 256, and what counts
// is how often the CUs have to be filled.  Measured, us of the forward call with each (K, N; 16 ranks, 8 adapters; the choice is the fastest of every line):
//   1021 tokens, 2048 x 2816      34.0   31.3   41.1   56.6        16384, 512 x 256              20.0   16.7   20.8   25.0
//   4099, 2048 x 128              18.3   28.1   38.3   53.6        600, 5000 x 5000             104.5   58.7   90.4  130.2
//   4099, 2048 x 1408             54.3   53.0   43.8   57.7        6000, 1000 x 3000             97.6   81.4   78.6   74.6
//   4099, 1408 x 2048             54.3   57.6   58.6   46.3        2048, 4096 x 4096            119.8   95.1   79.6   99.8
//   8192, 7168 x 2048            361.9  281.4  241.3  214.0        1024, 7168 x 7168            178.5  139.5  117.9  159.4
// (256 x 256 by 4 waves, each with a quarter of 128 x 128 in 256 accumulator registers, moves a quarter less through the LDS and was 1 to 10 % slower: one wave a SIMD
// waits at every barrier.)
struct TileShape {
    int rows, cols;
};
static TileShape tile_shape(int T, int C) {
    struct Form {
        TileShape t;
        int slots, cost;
    };
    static const Form forms[] = {{{256, 256}, 256, 145}, {{128, 256}, 256, 100}, {{128, 128}, 256, 60}, {{64, 64}, 512, 38}};
    TileShape best = {};
    long long least = INT64_MAX;
    for (const Form& f : forms) {
        const long long tiles = ((long long)T + f.t.rows - 1) / f.t.rows * ((C + f.t.cols - 1) / f.t.cols), cost = (tiles + f.slots - 1) / f.slots * f.cost;
        if (cost < least) {
            least = cost;
            best = f.t;
        }
    }
    return best;
}
static size_t hx_most(const moe_adapter_shape_t& s) { return std::max(hx_bytes(s, tile_shape(s.T, s.N).rows), hx_bytes(s, tile_shape(s.T, s.K).rows)); }
// The factors' gradients: columns of a tile; whether adapters with few rows have a kernel of their own (where they have few on average); and into how many parts
// an adapter's rows are cut at most, if it had all of them (3594 tokens on one adapter, 2528 x 264: 30.5 us in one part, 13.5 in 7 with the sum of the parts; 12337 on 2 of 193, 72 x
// 24: 94 in one part, 16).  With less than 8 adapters that fill half of the CUs it would be an empty launch for most batches.
static int grad_cols(int r) { return r > 64 ? 64 : 128; }
static int grad_tiles(const moe_adapter_shape_t& s) { return (s.K + grad_cols(s.rank) - 1) / grad_cols(s.rank) + (s.N + grad_cols(s.rank) - 1) / grad_cols(s.rank); }
static bool grad_rows(const moe_adapter_shape_t& s) { return (long long)s.adapters * kGradRows >= s.T; }
static int grad_pieces(const moe_adapter_shape_t& s) { return 256 / grad_tiles(s); }   // of all adapters together
static int grad_parts(const moe_adapter_shape_t& s) {
    if (s.adapters < 8 && s.adapters * grad_tiles(s) > 128) return 1;
    return std::max(1, std::min(grad_pieces(s), s.T / 512));
}
// Whether a product of sorted tokens is cut along its reduction into fp32 parts, with h beside it, as that of few tokens: long reductions of small results, which
// tiles in one piece leave to a few CUs, behind an equally long h.  Measured, us of the forward call with its plan in a graph of ten, in one piece / in parts (tokens, K, N):
//   2608, 6952,  24   49.7 / 30.6      8192, 2048,  64   31.6 / 31.6  (T C = 512 << 10)      12000, 2048, 128   42.5 / 47.2
//   6793, 5800,  64   52.7 / 44.4      1214, 5720, 840   80.3 / 70.9  (996 << 10)             8192, 2048, 256   39.8 / 53.5
//   4099, 2048, 128   28.2 / 24.0      4099, 2048, 256   33.3 / 34.9  (1025 << 10)            8192, 7168, 256   88.8 / 113.2
//                                      4099, 7168, 256   72.9 / 70.1                          1214, 5720, 1640  83.8 / 93.5
//                                      8192, 2048, 128   32.6 / 38.7  (1024 << 10)
// (the middle column is what lies about the limit: either way within 4 %, but for one line that gains 12 % in parts and one that loses 19)
static bool parts_pay(int T, int R, int C) { return T < 16384 && stages_in(R) >= 24 && (long long)T * C <= 640 << 10; }
static int parts_blocks(const moe_adapter_shape_t& s) { return ((int)plan_blocks(s) + 7) & ~7; }
static size_t parts_bytes(const moe_adapter_shape_t& s, int R, int C) {
    return parts_pay(s.T, R, C) ? few_bytes(s.T, R, C, s.rank, s.adapters, parts_blocks(s)) : 0;
}
static size_t grad_part_at(const moe_adapter_shape_t& s);
static size_t parts_at(const moe_adapter_shape_t& s) {
    const int parts = grad_parts(s);
    return grad_part_at(s) + (parts > 1 ? align_up((size_t)grad_pieces(s) * s.rank * ((size_t)s.K + s.N) * 4, 256) : 0);
}
static size_t many_bytes(const moe_adapter_shape_t& s) { return parts_at(s) + std::max(parts_bytes(s, s.K, s.N), parts_bytes(s, s.N, s.K)); }
static size_t grad_part_at(const moe_adapter_shape_t& s) {
    return align_up(hx_most(s), 256) + align_up((size_t)s.T * s.rank * 4, 256) + align_up((size_t)s.adapters * s.K * s.rank * 2, 256) +
           2 * align_up((size_t)s.T * s.rank * 6, 256);
}
size_t adapter_workspace_bytes(const moe_adapter_shape_t& s) {
    if (s.T == 0) return 256;
    if (adapter_few(s)) return std::max(few_bytes(s.T, s.K, s.N, s.rank, s.adapters), few_bytes(s.T, s.N, s.K, s.rank, s.adapters));
    return many_bytes(s) + (adapter_needs_plan(s) ? 0 : align_up(adapter_table_bytes(s), 256));
}

static void few_params(ProjParams& p, char* ws, FewPlan& f) {
    f = few_plan(p.T, p.R, p.C, p.r, p.n, p.blocks);
    p.part = (float*)ws;
    p.hpart = (float*)(ws + align_up((size_t)f.splits * p.T * p.C * 4, 256));
    p.splits = f.splits, p.per_split = f.per_split, p.hsplits = f.hsplits, p.hper_split = f.hper_split;
    p.col_tiles = f.col_tiles, p.row_tiles = f.row_tiles, p.rank_tiles = f.rank_tiles, p.hgroups = f.hgroups, p.dot_cut = f.dot_cut;
}
template <int FORM>
static void few_first(const ProjParams& p, const FewPlan& f, hipStream_t st) {
    const dim3 grid((unsigned)(f.col_tiles * f.splits * f.row_tiles + f.hgroups * f.rank_tiles * f.hsplits * f.dot_cut));
    if (f.row_frags == 1) hipLaunchKernelGGL((adapter_few_first_kernel<1, FORM>), grid, dim3(kSmallThreads), 0, st, p);
    else hipLaunchKernelGGL((adapter_few_first_kernel<2, FORM>), grid, dim3(kSmallThreads), 0, st, p);
}
static int few_joins(const ProjParams& p) { return p.T * ((p.C + kJoinCols - 1) / kJoinCols); }
// Whether tokens of one adapter share the fetch of its second factor in the second launch.  Measured, us by themselves / in fours (tokens, ranks, columns): 254, 128, 1728
// 11.7 / 17.4; 500, 16, 7168 12.0 / 20.8; 400, 128, 2048 18.3 / 18.9; 250, 64, 7168 17.4 / 16.8; 250, 128, 14336 59.8 / 40.3.
static bool join_groups(const ProjParams& p) { return (long long)p.T * p.r * p.C > 1 << 27; }

template <int FORM>
static int many_launch(ProjParams& p, const moe_adapter_shape_t& s, void* plan, char* ws, hipStream_t st) {
    if (!plan) {   // (up to kFewTokens)
        plan = ws + many_bytes(s);
        const int rc = adapter_plan_launch(s, p.ids, plan, st);
        if (rc != MOE_OK) return rc;
    }
    p.plan = plan_view(s, plan);
    const TileShape tile = tile_shape(p.T, p.C);
    p.tile_rows = tile.rows;
    p.span = (p.out_f32 ? 3 : 2) * p.r;
    p.blocks = parts_blocks(s);
    p.hx = ws;
    char* rest = ws + align_up(hx_most(s), 256);
    if (!p.h) p.h = (float*)rest;
    p.second_t = rest + align_up((size_t)s.T * s.rank * 4, 256);
    if (FORM == kKc) {
        p.terms[0] = (uint16_t*)(p.second_t + align_up((size_t)s.adapters * s.K * s.rank * 2, 256));
        p.terms[1] = (uint16_t*)((char*)p.terms[0] + align_up((size_t)s.T * s.rank * 6, 256));
    }
    if (parts_pay(p.T, p.R, p.C)) {
        FewPlan f;
        few_params(p, ws + parts_at(s), f);
        few_first<FORM>(p, f, st);
        const int wide = (p.C + 3) / 4;
        p.join_rows = std::max(1, std::min(kPartsRows, 256 / wide));
        const unsigned groups = (unsigned)((p.T + p.join_rows - 1) / p.join_rows * ((wide + 255) / 256));
        hipLaunchKernelGGL(adapter_parts_join_kernel, dim3(groups), dim3(256), 0, st, p);
        return MOE_OK;
    }
    const dim3 low((unsigned)(p.blocks + (FORM == kKc ? p.n * ((p.C + 63) / 64) : 0)));
    auto low_launch = [&](auto nrf) {
        if (p.r <= 32) hipLaunchKernelGGL((adapter_low_kernel<nrf.value, 1>), low, dim3(kSmallThreads), 0, st, p);
        else if (p.r <= 64) hipLaunchKernelGGL((adapter_low_kernel<nrf.value, 2>), low, dim3(kSmallThreads), 0, st, p);
        else hipLaunchKernelGGL((adapter_low_kernel<nrf.value, 4>), low, dim3(kSmallThreads), 0, st, p);
    };
    if (block_rows(p.T) == 64) low_launch(std::integral_constant<int, 2>{});
    else low_launch(std::integral_constant<int, 1>{});
    p.row_tiles = (p.T + p.tile_rows - 1) / p.tile_rows;
    p.col_tiles = (p.C + tile.cols - 1) / tile.cols;
    const dim3 grid((unsigned)(p.row_tiles * p.col_tiles));
    if (tile.cols == 64) hipLaunchKernelGGL((adapter_tile_kernel<FORM, false>), grid, dim3(kSmallThreads), 0, st, p);
    else if (tile.cols == 128) hipLaunchKernelGGL((adapter_tile_kernel<FORM, true>), grid, dim3(kMidThreads), 0, st, p);
    else hipLaunchKernelGGL((adapter_big_kernel<FORM>), grid, dim3(kMmaThreads), 0, st, p);
    return MOE_OK;
}

int adapter_forward_launch(const moe_adapter_shape_t& s, const void* x, size_t ldx, const void* w, const void* a, const void* b, const float* scale,
                           const int32_t* ids, void* plan, void* y, int out_f32, float* h, char* ws, hipStream_t st) {
    if (s.T == 0) return MOE_OK;
    ProjParams p = {};
    p.T = s.T, p.R = s.K, p.C = s.N, p.r = s.rank, p.n = s.adapters;
    p.x = (const char*)x, p.ldx = ldx * 2, p.w = (const char*)w, p.first = (const char*)a, p.second = (const char*)b;
    p.scale = scale, p.ids = ids, p.y = (char*)y, p.out_f32 = out_f32, p.h = h;
    if (adapter_few(s)) {
        FewPlan f;
        few_params(p, ws, f);
        few_first<kKs>(p, f, st);
        if (join_groups(p)) hipLaunchKernelGGL((adapter_few_second_kernel<4>), dim3((unsigned)few_joins(p)), dim3(256), 0, st, p);
        else hipLaunchKernelGGL((adapter_few_second_kernel<1>), dim3((unsigned)few_joins(p)), dim3(256), 0, st, p);
    } else {
        const int rc = many_launch<kKs>(p, s, plan, ws, st);
        if (rc != MOE_OK) return rc;
    }
    return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP;
}

// Columns of a workgroup of the factors' gradients of few tokens: 64 where that leaves the CUs a workgroup each.  Backward call with 256 / with 64, us (workgroups of
// 256 columns; tokens, K, N, ranks, adapters): 4 (128, 512 x 512, 8, 1) 12.4 / 10.2, 12 (256, 512 x 1024, 8, 2) 16.7 / 14.0, 56 (512, 2048 x 1408, 16, 2) 31.4 / 22.7, 64 (200,
// 1024 x 1024, 64, 1) 18.7 / 15.9, 96 (80, 1024 x 2048, 8, 8) 11.2 / 11.3, 448 (256, 2048 x 1408, 16, 16) 18.1 / 19.6, 1920 (200, 4096 x 4096, 16, 30) 36.0 / 58.4.
static int few_grad_cols(const moe_adapter_shape_t& s) {
    if (s.T <= kGradRows) return 1024;
    const size_t wide = (size_t)s.adapters * (s.rank / kGradRanks) * ((s.K + 255) / 256 + (s.N + 255) / 256);
    return 4 * wide <= 256 ? 64 : 256;
}

int adapter_backward_launch(const moe_adapter_shape_t& s, const void* dy, size_t lddy, const void* x, size_t ldx, const void* w, const void* a, const void* b,
                            const float* scale, const int32_t* ids, void* plan, const float* h, void* dx, float* da, float* db, char* ws, hipStream_t st) {
    ProjParams p = {};
    p.T = s.T, p.R = s.N, p.C = s.K, p.r = s.rank, p.n = s.adapters;
    p.x = (const char*)dy, p.ldx = lddy * 2, p.w = (const char*)w, p.first = (const char*)b, p.second = (const char*)a;
    p.scale = scale, p.ids = ids, p.y = (char*)dx;
    GradParams g = {};
    g.T = s.T, g.r = s.rank, g.n = s.adapters;
    g.W[0] = s.N, g.W[1] = s.K;
    g.x[0] = (const char*)dy, g.x[1] = (const char*)x;
    g.ldx[0] = lddy * 2, g.ldx[1] = ldx * 2;
    g.h[0] = h;
    g.out[0] = db, g.out[1] = da;
    if (adapter_few(s)) {
        FewPlan f;
        if (s.T > 0) {
            few_params(p, ws, f);
            few_first<kKc>(p, f, st);
        }
        const int joins = s.T > 0 ? few_joins(p) : 0;
        g.rank_tiles = g.r / kGradRanks;
        const int cols = few_grad_cols(s);
        for (int i = 0; i < 2; ++i) g.col_tiles[i] = (g.W[i] + cols - 1) / cols;
        const dim3 grid((unsigned)(joins + g.n * g.rank_tiles * (g.col_tiles[0] + g.col_tiles[1])));
        auto launch = [&](auto width) {
            if (join_groups(p)) hipLaunchKernelGGL((adapter_few_second_grad_kernel<4, width.value>), grid, dim3(256), 0, st, p, g, joins);
            else hipLaunchKernelGGL((adapter_few_second_grad_kernel<1, width.value>), grid, dim3(256), 0, st, p, g, joins);
        };
        if (cols == 1024) launch(std::integral_constant<int, 1024>{});
        else if (cols == 256) launch(std::integral_constant<int, 256>{});
        else launch(std::integral_constant<int, 64>{});
    } else {
        p.h_given = h;
        const int rc = many_launch<kKc>(p, s, plan, ws, st);
        if (rc != MOE_OK) return rc;
        // With so many adapters that they have few rows on average, those that do have are done by a kernel for that
        const bool rows = grad_rows(s);
        g.few = rows;
        g.h[1] = p.h;
        if (rows) {
            g.rank_tiles = g.r / kGradRanks;
            for (int i = 0; i < 2; ++i) g.col_tiles[i] = (g.W[i] + 1023) / 1024;
            hipLaunchKernelGGL(adapter_grad_rows_kernel, dim3((unsigned)(g.n * g.rank_tiles * (g.col_tiles[0] + g.col_tiles[1]))), dim3(256), 0, st, p, g);
        }
        const int cols = grad_cols(p.r);
        for (int i = 0; i < 2; ++i) g.col_tiles[i] = (g.W[i] + cols - 1) / cols;
        g.parts = grad_parts(s);
        g.part[0] = (float*)(ws + grad_part_at(s));
        g.part[1] = g.part[0] + (size_t)grad_pieces(s) * g.r * g.W[0];
        const int most = rows ? std::min(g.n, g.T / (kGradRows + 1)) : g.n;   // adapters that may have to be done
        const dim3 grid((unsigned)(8 * (g.parts > 1 ? std::max(most, grad_pieces(s)) : most) * ((g.col_tiles[0] + g.col_tiles[1] + 7) / 8)));
        if (p.r <= 32) hipLaunchKernelGGL((adapter_grad_kernel<1, 4>), grid, dim3(kGradThreads), 0, st, p, g);
        else if (p.r <= 64) hipLaunchKernelGGL((adapter_grad_kernel<2, 4>), grid, dim3(kGradThreads), 0, st, p, g);
        else hipLaunchKernelGGL((adapter_grad_kernel<4, 2>), grid, dim3(kGradThreads), 0, st, p, g);
        if (g.parts > 1)   // (more adapters than grad_pieces are not cut)
            hipLaunchKernelGGL(adapter_grad_sum_kernel, dim3((unsigned)((g.r * (g.W[0] + g.W[1]) / 4 + 255) / 256), (unsigned)(rows ? std::min(most, grad_pieces(s)) : g.n)), dim3(256), 0, st, p.plan, g);
    }
    return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP;
}

}  // namespace uniep
