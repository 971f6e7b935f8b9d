// Building blocks of the projection with many low-rank adapters: operand loaders whose reduction
// goes on past a dense matrix into the tile's low-rank part, and a 64 x 64 tile for small problems.
//
//   y[t] = x[t] W + s_a (x[t] A_a^T) B_a,   a = ids[t]            [T, K] x [K, N], A_a [r, K], B_a [r, N]
//
// With the rows sorted by adapter a tile of rows holds a few runs ("segments"), and its low-rank part is a
// product over 2 r more columns a segment: the tile's row of h = s x A^T stands, as the bf16 pair hi + lo (an error of
// 2^-17 of the fp32 value: small beside the rounding of a bf16 y), at the columns of its own segment, zeros at the
// others', and B_a stands twice behind W.  For an fp32 y it is three terms, the whole 24 bits, and 3 r columns.  So the matrix pipeline runs on without a second loop: stages of 64
// k are the dense ones, one that holds the rest of K, and then those of the low-rank part.  Every chunk of 16 bytes that
// lies past either is fetched from a page of zeros.
#pragma once
#include "mma.hpp"

namespace uniep {

// (zero-initialised; only read)
__device__ u32x4_t g_zero_page[4];
__device__ __forceinline__ const char* zero_chunk() { return (const char*)g_zero_page; }

// The low-rank part of a tile's reduction.
struct LowRank {
    const char* h;        // [rows of the tile][ld bytes] bf16: the terms (r columns each) of every segment, zeros elsewhere
    uint32_t ld;
    const char* f;        // KS: factors [adapters][r][C]; KC: [adapters][C][r]
    const int32_t* seg;   // adapters of the tile's segments
    int used;             // columns that hold something: `span` a segment
    int span, r, C;
    __device__ __forceinline__ const char* row(int row, int j) const { return h + (size_t)row * ld + (size_t)j * 2; }
    __device__ __forceinline__ const char* ks(int j, int col) const {
        if (j >= used) return zero_chunk();
        const int s = j / span, q = j - s * span;
        return f + (((size_t)seg[s] * r + (q < r ? q : q < 2 * r ? q - r : q - 2 * r)) * C + col) * 2;
    }
    __device__ __forceinline__ const char* kc(int j, int col) const {   // j a multiple of 8, as r is
        if (j >= used) return zero_chunk();
        const int s = j / span, q = j - s * span;
        return f + (((size_t)seg[s] * C + col) * r + (q < r ? q : q < 2 * r ? q - r : q - 2 * r)) * 2;
    }
};

// Stages of a reduction: `full` of 64, one with `tail` (0: none; a multiple of 8), then the low-rank ones.
struct Stages {
    int full, tail;
};

// Operand with k along its memory rows (KC image, 128 bytes a row): DMA instruction i of wave w fills block NI w + i, rows
// 8 (NI w + i) + l / 8.  COLUMNS: the low-rank part holds factors, else h.
template <int NI, bool COLUMNS>
struct KcStages : PlainLoader<KcStages<NI, COLUMNS>> {
    const char* p[NI];   // this lane's chunk in the stage to come
    int left, tail;
    int last;            // last row
    int first;           // COLUMNS: column of row 0
    LowRank low;
    __device__ __forceinline__ bool full() const { return true; }
    static __device__ __forceinline__ int row(const Lane& ln, int i) { return 8 * (NI * ln.w + i) + (ln.l >> 3); }
    static __device__ __forceinline__ int chunk(const Lane& ln, int i) { return (ln.l & 7) ^ ((row(ln, i) >> 1) & 7); }
    // row_of(r) = address of row r's first k; rows past the last alias it
    template <class F>
    __device__ __forceinline__ void init(const Lane& ln, int rows, Stages s, F row_of) {
        left = s.full;
        tail = s.tail;
        last = rows - 1;
#pragma unroll
        for (int i = 0; i < NI; ++i) p[i] = row_of(min(row(ln, i), last)) + chunk(ln, i) * 16;
    }
    // one of the full stages
    __device__ __forceinline__ void issue_full(char* dst) {
        char* d = dst + __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)) * (NI * 1024);
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            dma16(p[i], d + i * 1024);
            p[i] += BK * 2;
        }
        --left;
    }
    __device__ __forceinline__ void issue(char* dst) {
        if (left > 0) {
            issue_full(dst);
        } else {
            char* d = dst + __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)) * (NI * 1024);
            const Lane ln;
            const char* q[NI];
#pragma unroll
            for (int i = 0; i < NI; ++i) {
                const int c = 8 * chunk(ln, i), r = min(row(ln, i), last);
                if (left == 0 && tail > 0) q[i] = c < tail ? p[i] : zero_chunk();
                else {
                    const int j = BK * (-left - (tail > 0 ? 1 : 0)) + c;
                    q[i] = COLUMNS ? low.kc(j, first + r) : low.row(r, j);
                }
            }
#pragma unroll
            for (int i = 0; i < NI; ++i) asm volatile("" : "+v"(q[i]));   // the addresses exist before the first request
#pragma unroll
            for (int i = 0; i < NI; ++i) dma16(q[i], d + i * 1024);
            --left;
        }
    }
};

// Operand whose k is its memory row (KS image, TC columns): a k row is TC / 8 lanes.
template <int NI, int TC>
struct KsStages : PlainLoader<KsStages<NI, TC>> {
    static constexpr int kLanes = TC / 8, kRows = 64 / kLanes;
    const char* p[NI];
    long long step;
    int left, tail, col[2];   // (the chunk depends on i through i % 2 at most)
    LowRank low;
    __device__ __forceinline__ bool full() const { return true; }
    static __device__ __forceinline__ int swz(int k) { return TC == 64 ? (k & 2) << 1 : (k & 3) << 2; }
    static __device__ __forceinline__ int krow(const Lane& ln, int i) { return kRows * (NI * ln.w + i) + ln.l / kLanes; }
    static __device__ __forceinline__ int chunk(const Lane& ln, int i) { return (ln.l % kLanes) ^ swz(krow(ln, i)); }
    // m: the first k row, n columns; columns from `first` on, chunks past the last alias it; k rows below `rows` are there
    __device__ __forceinline__ void init(const Lane& ln, const char* m, int first, int n, Stages s) {
        left = s.full;
        tail = s.tail;
        step = (long long)BK * n * 2;
#pragma unroll
        for (int i = 0; i < 2; ++i) col[i] = min(first + 8 * chunk(ln, i), n - 8);
#pragma unroll
        for (int i = 0; i < NI; ++i) p[i] = m + ((size_t)krow(ln, i) * n + col[i & 1]) * 2;
    }
    __device__ __forceinline__ void issue_full(char* dst) {
        char* d = dst + __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)) * (NI * 1024);
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            dma16(p[i], d + i * 1024);
            p[i] += step;
        }
        --left;
    }
    __device__ __forceinline__ void issue(char* dst) {
        if (left > 0) {
            issue_full(dst);
        } else {
            char* d = dst + __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)) * (NI * 1024);
            const Lane ln;
            const char* q[NI];
#pragma unroll
            for (int i = 0; i < NI; ++i) {
                const int k = krow(ln, i);
                if (left == 0 && tail > 0) q[i] = k < tail ? p[i] : zero_chunk();
                else q[i] = low.ks(BK * (-left - (tail > 0 ? 1 : 0)) + k, col[i & 1]);
            }
#pragma unroll
            for (int i = 0; i < NI; ++i) asm volatile("" : "+v"(q[i]));
#pragma unroll
            for (int i = 0; i < NI; ++i) dma16(q[i], d + i * 1024);
            --left;
        }
    }
};

// ------------------------------------------------------------------ small tiles
// 4 waves, 32 NRF rows by 32 NCF columns.  Every wave has the whole tile in its accumulators and takes one of a stage's four k-sub-steps: a wave with a
// quarter of the tile instead would read each operand's fragments twice, and the LDS is what a small tile is bound by.  The four
// sums are added at the end, wave 0 first.  kDepth stage buffers, all but one on their way; one barrier a stage.  As many buffers as leave
// room for two workgroups on a CU: what a CU draws from memory is what it has on its way over a latency (the low-rank part of 8192 tokens 7168 wide,
// a workgroup a CU, with four buffers of 8 KB 28 us).
constexpr int kSmallThreads = 256;
template <int NRF, int NCF>
struct SmallTile {
    static constexpr int kRowsBytes = 4096 * NRF, kStage = 4096 * (NRF + NCF);
    static constexpr int kDepth = NRF + NCF == 2 ? 8 : NRF + NCF == 3 ? 6 : 4;
    static constexpr int kSums = 16384 * NRF * NCF;   // 4 waves, fp32
    static constexpr int kLds = kDepth * kStage > kSums ? kDepth * kStage : kSums;
};

template <int NRF, int NCF, int FORM>
struct SmallFrags {
    uint32_t b, a[2];
    __device__ __forceinline__ SmallFrags(const Lane& ln, uint32_t lds0) {
        const int kh = ln.hf, w = ln.w;
        b = lds0 + ln.l31 * 128 + (((2 * w + kh) ^ ((ln.l31 >> 1) & 7)) << 4);
        const uint32_t a0 = lds0 + SmallTile<NRF, NCF>::kRowsBytes;
        if (FORM == kKc) {
            const int n = swap23(ln.l31);
            a[0] = a0 + n * 128 + (((2 * w + kh) ^ ((n >> 1) & 7)) << 4);
            a[1] = a[0] + 4096;
        } else {
            static_assert(FORM == kKc || NCF == 2, "");
            const int g = (ln.l >> 4) & 1, e = (ln.l & 15) >> 2, q = ln.l & 3, sq = ((q & 1) << 1) | (q >> 1);
            const uint32_t k = a0 + (16 * w + 8 * kh + e) * 128 + (sq & 1) * 8;
            a[0] = k + (((2 * g + (sq >> 1)) ^ ((e & 2) << 1)) << 4);
            a[1] = k + (((4 + 2 * g + (sq >> 1)) ^ ((e & 2) << 1)) << 4);
        }
    }
    // The wave's fragments of the stage `off` bytes behind the first buffer.  The wait stands in the block that reads: nothing can
    // touch a register that is still being filled.
    __device__ __forceinline__ void read(uint32_t off, u32x4_t (&rb)[NRF], u32x4_t (&ra)[NCF]) const {
        const uint32_t bo = b + off;
        if constexpr (FORM == kKc) {
            const uint32_t ao = a[0] + off;
            if constexpr (NRF == 2 && NCF == 2)
                asm volatile("ds_read_b128 %0, %4\n ds_read_b128 %1, %4 offset:4096\n ds_read_b128 %2, %5\n ds_read_b128 %3, %5 offset:4096\n"
                             "s_waitcnt lgkmcnt(0)" : "=&v"(rb[0]), "=&v"(rb[1]), "=&v"(ra[0]), "=&v"(ra[1]) : "v"(bo), "v"(ao) : "memory");
            else if constexpr (NRF == 1 && NCF == 2)
                asm volatile("ds_read_b128 %0, %3\n ds_read_b128 %1, %4\n ds_read_b128 %2, %4 offset:4096\n"
                             "s_waitcnt lgkmcnt(0)" : "=&v"(rb[0]), "=&v"(ra[0]), "=&v"(ra[1]) : "v"(bo), "v"(ao) : "memory");
            else if constexpr (NRF == 1 && NCF == 4)
                asm volatile("ds_read_b128 %0, %5\n ds_read_b128 %1, %6\n ds_read_b128 %2, %6 offset:4096\n ds_read_b128 %3, %6 offset:8192\n"
                             "ds_read_b128 %4, %6 offset:12288\n s_waitcnt lgkmcnt(0)"
                             : "=&v"(rb[0]), "=&v"(ra[0]), "=&v"(ra[1]), "=&v"(ra[2]), "=&v"(ra[3]) : "v"(bo), "v"(ao) : "memory");
            else if constexpr (NRF == 2 && NCF == 1)
                asm volatile("ds_read_b128 %0, %3\n ds_read_b128 %1, %3 offset:4096\n ds_read_b128 %2, %4\n"
                             "s_waitcnt lgkmcnt(0)" : "=&v"(rb[0]), "=&v"(rb[1]), "=&v"(ra[0]) : "v"(bo), "v"(ao) : "memory");
            else if constexpr (NRF == 2 && NCF == 4)
                asm volatile("ds_read_b128 %0, %6\n ds_read_b128 %1, %6 offset:4096\n ds_read_b128 %2, %7\n ds_read_b128 %3, %7 offset:4096\n"
                             "ds_read_b128 %4, %7 offset:8192\n ds_read_b128 %5, %7 offset:12288\n s_waitcnt lgkmcnt(0)"
                             : "=&v"(rb[0]), "=&v"(rb[1]), "=&v"(ra[0]), "=&v"(ra[1]), "=&v"(ra[2]), "=&v"(ra[3]) : "v"(bo), "v"(ao) : "memory");
            else {
                static_assert(NRF == 1 && NCF == 1, "");
                asm volatile("ds_read_b128 %0, %2\n ds_read_b128 %1, %3\n s_waitcnt lgkmcnt(0)" : "=&v"(rb[0]), "=&v"(ra[0]) : "v"(bo), "v"(ao) : "memory");
            }
        } else {
            const uint32_t a0 = a[0] + off, a1 = a[1] + off;
            u32x2_t l0, h0, l1, h1;
            if constexpr (NRF == 2)
                asm volatile("ds_read_b128 %0, %6\n ds_read_b128 %1, %6 offset:4096\n"
                             "ds_read_b64_tr_b16 %2, %7\n ds_read_b64_tr_b16 %3, %7 offset:512\n"
                             "ds_read_b64_tr_b16 %4, %8\n ds_read_b64_tr_b16 %5, %8 offset:512\n s_waitcnt lgkmcnt(0)"
                             : "=&v"(rb[0]), "=&v"(rb[1]), "=&v"(l0), "=&v"(h0), "=&v"(l1), "=&v"(h1) : "v"(bo), "v"(a0), "v"(a1) : "memory");
            else
                asm volatile("ds_read_b128 %0, %5\n"
                             "ds_read_b64_tr_b16 %1, %6\n ds_read_b64_tr_b16 %2, %6 offset:512\n"
                             "ds_read_b64_tr_b16 %3, %7\n ds_read_b64_tr_b16 %4, %7 offset:512\n s_waitcnt lgkmcnt(0)"
                             : "=&v"(rb[0]), "=&v"(l0), "=&v"(h0), "=&v"(l1), "=&v"(h1) : "v"(bo), "v"(a0), "v"(a1) : "memory");
            ra[0] = u32x4_t{l0[0], l0[1], h0[0], h0[1]};
            ra[1] = u32x4_t{l1[0], l1[1], h1[0], h1[1]};
        }
    }
};

// Runs nk >= 0 stages through DEPTH buffers of STAGE bytes, the rows' image first, and calls multiply(buffer) for each; a wave has REQUESTS requests a
// stage.  One barrier a stage.  Ends with a barrier: the buffers may be written.
template <int DEPTH, int STAGE, int ROWS, int REQUESTS, class LB, class LA, class M>
__device__ __forceinline__ void pipeline(LB& lb, LA& la, int nk, char* smem, M multiply) {
    // (one copy of the requests' code: a launch this short waits for its instructions too)
#pragma unroll 1
    for (int t = 0; t < min(DEPTH - 1, nk); ++t) {
        lb.issue(smem + t * STAGE);
        la.issue(smem + t * STAGE + ROWS);
    }
    int at = 0, next = (DEPTH - 1) * STAGE;   // buffers of stages t and t + DEPTH - 1
    auto step = [&](int& b) { b = b == (DEPTH - 1) * STAGE ? 0 : b + STAGE; };
    // while full stages are left to request: no branch but the loop's
    int t = 0;
    for (int n = lb.left; n > 0; --n, ++t) {
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"((DEPTH - 2) * REQUESTS) : "memory");   // stage t is here when at most those behind it are on their way
        __builtin_amdgcn_s_barrier();
        lb.issue_full(smem + next);   // into the buffer that every wave has read before the barrier
        la.issue_full(smem + next + ROWS);
        step(next);
        multiply(at);
        step(at);
    }
    for (; t < nk; ++t) {
        if (t + DEPTH - 2 < nk) asm volatile("s_waitcnt vmcnt(%0)" ::"n"((DEPTH - 2) * REQUESTS) : "memory");
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        if (t + DEPTH - 1 < nk) {
            lb.issue(smem + next);
            la.issue(smem + next + ROWS);
            step(next);
        }
        multiply(at);
        step(at);
    }
    __builtin_amdgcn_sched_barrier(0);
    __syncthreads();
}
template <int NRF, int NCF>
__device__ __forceinline__ void zero_tile(f32x16_t (&acc)[NRF][NCF]) {
#pragma unroll
    for (int tf = 0; tf < NRF; ++tf)
#pragma unroll
        for (int af = 0; af < NCF; ++af)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[tf][af][v] = 0.f;
}
template <int NRF, int NCF>
__device__ __forceinline__ void mfma_tile(const u32x4_t (&rb)[NRF], const u32x4_t (&ra)[NCF], f32x16_t (&acc)[NRF][NCF]) {
#pragma unroll
    for (int tf = 0; tf < NRF; ++tf)
#pragma unroll
        for (int af = 0; af < NCF; ++af)
            acc[tf][af] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, ra[af]), __builtin_bit_cast(bf16x8_t, rb[tf]),
                                                                  acc[tf][af], 0, 0, 0);
}

// acc = sum over nk >= 0 stages of this wave's sub-step.
template <int NRF, int NCF, int FORM, class LB, class LA>
__device__ __forceinline__ void small_loop(LB& lb, LA& la, int nk, char* smem, f32x16_t (&acc)[NRF][NCF]) {
    using S = SmallTile<NRF, NCF>;
    const SmallFrags<NRF, NCF, FORM> fr(Lane(), lds_addr(smem));
    zero_tile(acc);
    pipeline<S::kDepth, S::kStage, S::kRowsBytes, NRF + NCF>(lb, la, nk, smem, [&](int buffer) {
        u32x4_t rb[NRF], ra[NCF];
        fr.read(buffer, rb, ra);
        mfma_tile(rb, ra, acc);
    });
}

// The tiles of waves 0..3 into LDS, and 8 columns of their sum, wave 0 first.
template <int NRF, int NCF>
__device__ __forceinline__ void small_put(char* smem, const f32x16_t (&acc)[NRF][NCF]) {
    constexpr int kPitch = NCF * 128, kWave = kPitch * 32 * NRF;
    const Lane ln;
    if (ln.w >= 4) return;
    char* base = smem + ln.w * kWave;
#pragma unroll
    for (int tf = 0; tf < NRF; ++tf)
#pragma unroll
        for (int af = 0; af < NCF; ++af)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int row = 32 * tf + ln.l31, piece = 8 * af + 4 * (q >> 1) + 2 * ln.hf + (q & 1);
                *(f32x4_t*)(base + row * kPitch + ((piece ^ (row & 7)) << 4)) =
                    f32x4_t{acc[tf][af][4 * q], acc[tf][af][4 * q + 1], acc[tf][af][4 * q + 2], acc[tf][af][4 * q + 3]};
            }
}
template <int NRF, int NCF>
__device__ __forceinline__ void small_get(const char* smem, int row, int c8, float (&v)[8]) {
    constexpr int kPitch = NCF * 128, kWave = kPitch * 32 * NRF;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int at = row * kPitch + (((2 * c8 + h) ^ (row & 7)) << 4);
        f32x4_t s = *(const f32x4_t*)(smem + at);
#pragma unroll
        for (int w = 1; w < 4; ++w) {
            const f32x4_t o = *(const f32x4_t*)(smem + w * kWave + at);
#pragma unroll
            for (int j = 0; j < 4; ++j) s[j] += o[j];
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) v[4 * h + j] = s[j];
    }
}
// Both, and f(row, column, values) for every run of 8 columns by one of THREADS threads.
template <int NRF, int NCF, int THREADS = kSmallThreads, class F>
__device__ __forceinline__ void small_sum(char* smem, const f32x16_t (&acc)[NRF][NCF], F f) {
    small_put(smem, acc);
    __syncthreads();
#pragma unroll 1
    for (int unit = threadIdx.x; unit < 128 * NRF * NCF; unit += THREADS) {
        float v[8];
        small_get<NRF, NCF>(smem, unit / (4 * NCF), unit % (4 * NCF), v);
        f(unit / (4 * NCF), 8 * (unit % (4 * NCF)), v);
    }
}

// ------------------------------------------------------------------ tiles of 128 x 128
// 8 waves: wave 4 h + 2 r + c has sub-steps 2 h and 2 h + 1 of every stage for a quarter of 64 x 64; the two halves' sums are added at the end.  A
// flop takes half the operand bytes that it takes in tiles of 64 x 64, and those are what a CU draws into its LDS at some 60 bytes a nanosecond.
constexpr int kMidThreads = 512;
struct MidTile {
    static constexpr int kRowsBytes = 16384, kStage = 32768, kDepth = 4, kLds = kDepth * kStage;
};
template <int FORM>
struct MidFrags {
    uint32_t b[2], a[2][2];   // of the wave's two sub-steps; KS: a[0] of the two column fragments
    __device__ __forceinline__ MidFrags(const Lane& ln, uint32_t lds0) {
        const int half = ln.w >> 2, rh = (ln.w >> 1) & 1, ch = ln.w & 1, kh = ln.hf;
        const uint32_t a0 = lds0 + MidTile::kRowsBytes;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int kk = 2 * half + s, n = swap23(ln.l31);
            b[s] = lds0 + (64 * rh + ln.l31) * 128 + (((2 * kk + kh) ^ ((ln.l31 >> 1) & 7)) << 4);
            if (FORM == kKc) {
                a[s][0] = a0 + (64 * ch + n) * 128 + (((2 * kk + kh) ^ ((n >> 1) & 7)) << 4);
                a[s][1] = 0;
            }
        }
        if (FORM != kKc) {
            const int g = (ln.l >> 4) & 1, e = (ln.l & 15) >> 2, q = ln.l & 3, sq = ((q & 1) << 1) | (q >> 1);
#pragma unroll
            for (int af = 0; af < 2; ++af) {
                a[0][af] = a0 + (32 * half + 8 * kh + e) * 256 + (((8 * ch + 4 * af + 2 * g + (sq >> 1)) ^ (e << 2)) << 4) + (sq & 1) * 8;
                a[1][af] = 0;
            }
        }
    }
    template <int S>
    __device__ __forceinline__ void read(uint32_t off, u32x4_t (&rb)[2], u32x4_t (&ra)[2]) const {
        const uint32_t bo = b[S] + off;
        if constexpr (FORM == kKc) {
            const uint32_t ao = a[S][0] + off;
            asm volatile("ds_read_b128 %0, %4\n ds_read_b128 %1, %4 offset:4096\n ds_read_b128 %2, %5\n ds_read_b128 %3, %5 offset:4096\n"
                         "s_waitcnt lgkmcnt(0)" : "=&v"(rb[0]), "=&v"(rb[1]), "=&v"(ra[0]), "=&v"(ra[1]) : "v"(bo), "v"(ao) : "memory");
        } else {
            const uint32_t a0 = a[0][0] + off, a1 = a[0][1] + off;
            u32x2_t l0, h0, l1, h1;
            asm volatile("ds_read_b128 %0, %6\n ds_read_b128 %1, %6 offset:4096\n"
                         "ds_read_b64_tr_b16 %2, %7 offset:%9\n ds_read_b64_tr_b16 %3, %7 offset:%10\n"
                         "ds_read_b64_tr_b16 %4, %8 offset:%9\n ds_read_b64_tr_b16 %5, %8 offset:%10\n s_waitcnt lgkmcnt(0)"
                         : "=&v"(rb[0]), "=&v"(rb[1]), "=&v"(l0), "=&v"(h0), "=&v"(l1), "=&v"(h1)
                         : "v"(bo), "v"(a0), "v"(a1), "n"(S * 4096), "n"(S * 4096 + 1024) : "memory");
            ra[0] = u32x4_t{l0[0], l0[1], h0[0], h0[1]};
            ra[1] = u32x4_t{l1[0], l1[1], h1[0], h1[1]};
        }
    }
};
template <int FORM, class LB, class LA>
__device__ __forceinline__ void mid_loop(LB& lb, LA& la, int nk, char* smem, f32x16_t (&acc)[2][2]) {
    const MidFrags<FORM> fr(Lane(), lds_addr(smem));
    zero_tile(acc);
    pipeline<MidTile::kDepth, MidTile::kStage, MidTile::kRowsBytes, 4>(lb, la, nk, smem, [&](int buffer) {
        u32x4_t rb[2], ra[2];
        fr.template read<0>(buffer, rb, ra);
        mfma_tile(rb, ra, acc);
        fr.template read<1>(buffer, rb, ra);
        mfma_tile(rb, ra, acc);
    });
}
// The two halves' sums, as small_sum.
template <class F>
__device__ __forceinline__ void mid_sum(char* smem, const f32x16_t (&acc)[2][2], F f) {
    constexpr int kPitch = 512, kHalf = 128 * kPitch;
    {
        const Lane ln;
        char* base = smem + (ln.w >> 2) * kHalf;
#pragma unroll
        for (int tf = 0; tf < 2; ++tf)
#pragma unroll
            for (int af = 0; af < 2; ++af)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int row = 64 * ((ln.w >> 1) & 1) + 32 * tf + ln.l31, piece = 16 * (ln.w & 1) + 8 * af + 4 * (q >> 1) + 2 * ln.hf + (q & 1);
                    *(f32x4_t*)(base + row * kPitch + ((piece ^ (row & 7)) << 4)) =
                        f32x4_t{acc[tf][af][4 * q], acc[tf][af][4 * q + 1], acc[tf][af][4 * q + 2], acc[tf][af][4 * q + 3]};
                }
    }
    __syncthreads();
#pragma unroll 1
    for (int unit = threadIdx.x; unit < 2048; unit += kMidThreads) {
        const int row = unit >> 4, c8 = unit & 15;
        float v[8];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int at = row * kPitch + (((2 * c8 + h) ^ (row & 7)) << 4);
            const f32x4_t s = *(const f32x4_t*)(smem + at), o = *(const f32x4_t*)(smem + kHalf + at);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[4 * h + j] = s[j] + o[j];
        }
        f(row, 8 * c8, v);
    }
}

__device__ __forceinline__ u32x4_t pack8f(const float (&v)[8]) {
    return u32x4_t{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
}
__device__ __forceinline__ float bf16_round(float v) { return bf16_lo(pack_bf16x2(v, 0.f) & 0xffffu); }

}  // namespace uniep
