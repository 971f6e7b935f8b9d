// Products of expert-sorted rows with their experts' weights, both in microscaled 4-bit floating point (mx.hpp):
//   product   y[r] = a[src(r)] W_e^T              for the rows r of expert e, offsets[e] <= r < offsets[e + 1]
//   gate_up   h[r] = silu(a[src(r)] Wg_e^T) * (a[src(r)] Wu_e^T), in bf16 or quantised again
// src(r) = perm[r] / k where there is a table (the rows' tokens), else r.
//
// v_mfma_scale_f32_32x32x64_f8f6f4 takes 32 values of a row and one scale a lane: exactly a block.  It runs four times as many products a clock as the bf16 instruction on
// as many bytes, so that a tile needs its operands as fast as a bf16 tile does, for four times the reduction.  Up to some 300 rows an expert the weights, read once from memory, take longer
// than the matrix work.
//
// Tile: 128 rows by 256 columns (gate_up: 128 columns of each weight) by four waves, each with all rows of 64 columns: 4 x 2 accumulators of 32 x 32.  K advances 128 values a stage, 64 bytes
// a row, by DMA into one of three images (24 KB); chunk c of row r lies at c ^ (r / 4 % 4), so that fragments are read without bank conflicts.  Two workgroups share a
// CU (78 KB of LDS and 256 registers a lane each): one's first stages and stores run behind the other's matrix work, as a tile has only K / 128 stages.
// Scales: four stages' bytes of a row are 16 of memory; they are moved a dword a lane into an image of their own, and one LDS read a fragment and four stages hands a lane its row's.
// A lane takes values 32 (2 s + half) .. + 31 of sub-step s, so its scale is byte 2 s + half of the stage's dword: the bytes of its half in two stages' dwords are put into one, of which the
// instruction selects one.
//
// Tiles are listed expert by expert, columns by columns, rows fastest, and dealt to the XCDs in eight runs: the tiles that share weights and rows meet in one L2.
//
// What bounds it.  The instruction alone runs at 6.5 PFLOP/s on normally distributed values, where the chip lowers its clock to 1.65 GHz, and at 9.8 on zeros.  In large tiles the operands' way through
// L2 into LDS takes longer than the matrix work, and the two do not overlap whole.  us with parts of the loop left out (the stores and a tile's ends are in all of them):
//                                                           whole   requests alone   matrix work alone   neither, without reads of LDS
//   gate_up, 8 of 4096 x 14336, 8002 rows (1.88 TFLOP)        529              436                 372                              77
//   gate_up, 256 of 2048 x 768, 512 rows each                 300              257                 206                              69
//   gate_up, 32 of 7168 x 2048, 512 rows each                 314              275                 207                              36
//   product, 128 of 768 x 2048, 512 rows each                 120              102                  84                              58
// Between the ends the first one's matrix work takes 295 us, the instruction's own rate, and its requests 359: 38 million of up to 128 bytes to L2, a fifth of them for the scales' 32 bytes a row.  The
// reads of fragments from LDS cost it 8 us (LDS is busy a quarter of the time, without bank conflicts).  With codes of zero, whose matrix work is done in two thirds, it took 422 us where random ones took
// 510; by the clock that a chip holds it is 510 to 551.  The last one is 111 to 118 with inputs in the cache (93 at best), 110 to 130 from memory, of which 76 are bytes.  37 tokens, 32 experts of 256
// here, 7168 x 2048: 53 to 71 us for the weights of 22 to 26 experts that have rows, 0.34 to 0.40 GB (a large copy: 65 to 77; some come from the cache of 256 MB).
// Slower or nothing: the next tile's first stages requested before the stores (127 us for 121 in the second case), waves that only move operands (152 for 120), tiles of 256 x 256 with 64 bytes a row
// in four images (560 for 516), by four waves of 128 x 128 (548 for 515), with the requests of a stage between its last products (514 to 518 for 510), weights' lines requested into L2 ahead
// (548 for 530), XCDs' runs of equal cost instead of equal count (518 both), the operands' rows that a tile does not have left out (514 both).
#include "mma.hpp"
#include "mx.hpp"

#include <mutex>

namespace uniep {

constexpr int kMxRows = 128, kMxCols = 256;
constexpr int kMxStageK = 128;                       // values
constexpr int kMxImages = 3;
constexpr int kMxThreads = 256;
constexpr int kThinRows = 32;   // see thin_tile
static_assert(kMxStageK == kMxPad, "");

struct MxParams {
    int rows, N, experts;
    int stages;               // K' / 128
    int slots;                // workgroups that run at a time
    int col_tiles, thin_tiles;   // of a row tile, of an expert with few rows
    uint32_t a_rows;
    const uint8_t *a_codes, *a_scales;
    const int32_t* perm;      // or NULL
    int k;
    const uint8_t *w_codes, *w_scales;   // product: the weights; gate_up: the gate's
    const uint8_t *u_codes, *u_scales;   // gate_up: up
    const int32_t* offsets;
    void* y;                  // [rows][N]; gate_up: h, or NULL
    uint8_t *h_codes, *h_scales;
    int f32;
};

// ---- which tile
struct MxTile {
    int expert, row0, rows, col_tile;   // rows: of the tile
    bool thin;                          // the expert has few: col_tile counts narrow ones
};
// A wave's view of the experts: lane l has `per` of them from l * per on.
// Experts with up to so many rows are done in narrow tiles (thin_tile).  A narrow tile takes longer for what it does, its first stages and its sums four times as often, but there are four times as
// many: they pay where wide ones would leave three quarters of the chip idle, and where these would not fill it once, or the reduction is long, if no expert has more than 16 rows (both kinds in
// one launch are slower than either where all CUs have work: 32 experts of 7168 x 2048 with 4 rows on average 120 us).  us, wide tiles / narrow ones up to 32 rows, by the rows of an expert on average:
//   gate_up, 32 of 7168 x 2048        6 experts with a row 39 / 25, 1 85 / 75, 4 95 / 89, 10 104 / 108, 24 105 / 139
//   gate_up, 8 of 4096 x 14336        4 108 / 88, 10 111 / 102, 24 113 / 152
//   product, 8 of 14336 x 4096        1 72 / 46, 24 77 / 64, 48 79 / 82
//   product, 128 of 768 x 2048        15 experts with a row 6.6 / 5.4, 1 17 / 21, 4 23 / 29
//   gate_up, 64 of 1024 x 512         10 experts with a row 7.1 / 4.6, 1 8.1 / 6.6, 4 10.1 / 10.5, 24 10.5 / 14.5
constexpr int kThinAlone = 16;
__device__ __forceinline__ int thin_limit(int stages, int wide_tiles, int slots, bool more) {
    if (4 * wide_tiles <= slots) return kThinRows;
    return !more && (wide_tiles < slots || stages >= 32) ? kThinAlone : 0;
}
template <int ROWS, bool THIN>
struct MxTiles {
    int per, before, total;   // tiles of the lanes before this one
    int row0, n;              // of the lane's only expert (per = 1)
    int thin_rows;
    static __device__ __forceinline__ void rows_of(const MxParams& p, int e, int& row0, int& n) {
        row0 = n = 0;
        if (e >= p.experts) return;
        row0 = min(max(p.offsets[e], 0), p.rows);
        n = min(max(p.offsets[e + 1], row0), p.rows) - row0;
    }
    __device__ __forceinline__ bool thin(int rows) const { return THIN && rows <= thin_rows; }
    __device__ __forceinline__ int tiles_of(const MxParams& p, int rows) const {
        return thin(rows) ? (rows > 0 ? p.thin_tiles : 0) : (rows + ROWS - 1) / ROWS * p.col_tiles;
    }
    // tiles of this lane's experts (`most`: the rows of its largest), and of all up to them
    __device__ __forceinline__ int upto(const MxParams& p, int& mine, int& most) {
        const int lane = threadIdx.x & 63;
        mine = most = 0;
        for (int j = 0; j < per; ++j) {
            if (per > 1) rows_of(p, lane * per + j, row0, n);
            mine += tiles_of(p, n);
            most = max(most, n);
        }
        return wave_scan(mine);
    }
    __device__ __forceinline__ explicit MxTiles(const MxParams& p) {
        int mine, most;
        per = (p.experts + 63) >> 6;
        rows_of(p, threadIdx.x & 63, row0, n);
        thin_rows = -1;   // (all of them wide)
        if (THIN) {
            const int wide = upto(p, mine, most);
            thin_rows = thin_limit(p.stages, __builtin_amdgcn_readlane(wide, 63), p.slots, __ballot(most > kThinAlone) != 0);
        }
        const int all = upto(p, mine, most);
        before = all - mine;
        total = __builtin_amdgcn_readlane(all, 63);
    }
    // tile i of 0 .. total - 1
    __device__ __forceinline__ MxTile find(const MxParams& p, int i) const {
        const int lane = threadIdx.x & 63;
        int l = 63 - __builtin_clzll(__ballot(before <= i));   // (lane 0 has 0)
        int base = __builtin_amdgcn_readlane(before, l), r0 = row0, m = n, e = l;
        if (per > 1) {
            rows_of(p, lane < per ? l * per + lane : p.experts, r0, m);
            const int mine = tiles_of(p, m), first = wave_scan(mine) - mine, at = i - base;
            const int j = 63 - __builtin_clzll(__ballot(lane < per && first <= at));
            base += __builtin_amdgcn_readlane(first, j);
            e = l * per + j;
            l = j;
        }
        MxTile t;
        t.expert = rfl(e);
        const int begin = __builtin_amdgcn_readlane(r0, l), count = __builtin_amdgcn_readlane(m, l);
        const int row_tiles = (count + ROWS - 1) / ROWS, at = i - base;
        t.col_tile = rfl(at / row_tiles);
        const int first = rfl(at - t.col_tile * row_tiles) * ROWS;
        t.row0 = begin + first;
        t.rows = min(count - first, ROWS);
        t.thin = thin(count);
        return t;
    }
};

// Sorted rows -> rows of a.  All are asked for before any is used; one that is out of range is taken from the last row.
template <int N>
__device__ __forceinline__ void mx_sources(const MxParams& p, uint32_t (&r)[N]) {
    if (p.perm) {
#pragma unroll
        for (int i = 0; i < N; ++i) r[i] = (uint32_t)p.perm[r[i]];
#pragma unroll
        for (int i = 0; i < N; ++i) r[i] /= (uint32_t)p.k;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) r[i] = min(r[i], p.a_rows - 1);
}

// ---- operands into LDS
__device__ __forceinline__ void dma4s(glb_ptr_t base, uint32_t off, char* dst) {
    asm volatile("" : "+s"(base), "+v"(off));   // as in dma16s
    __builtin_amdgcn_global_load_lds((glb_void_t*)(base + off), (lds_void_t*)dst, 4, 0, 0);
}
// A pointer that is the same in every lane, in scalar registers.
__device__ __forceinline__ glb_ptr_t uniform(const uint8_t* p) {
    const uint64_t v = (uint64_t)p;
    return (glb_ptr_t)(((uint64_t)(uint32_t)rfl((int)(v >> 32)) << 32) | (uint32_t)rfl((int)v));
}

// Where a wave finds its operands in LDS: of a stage's image the rows at 0 and the columns at kCols; behind IMAGES of them the rows' scales, then the columns'.
template <int ROWS, int COLS>
struct MxPlace {
    static constexpr int kCols = ROWS * 64, kStage = (ROWS + COLS) * 64;
    static constexpr int kScales = kMxImages * kStage, kColScales = kScales + ROWS * 16, kBytes = kColScales + COLS * 16;
};
using MxShared = MxPlace<kMxRows, kMxCols>;   // by the four waves of a workgroup
using MxOwn = MxPlace<kThinRows, 64>;         // a wave's, see thin_tile
constexpr int kMxSmem = MxShared::kBytes;
static_assert(4 * MxOwn::kBytes <= kMxSmem, "");
static_assert(2 * kMxSmem <= 160 * 1024, "");

// A DMA instruction fills 16 rows of an image: lane p the chunk of row p / 4 that belongs at position p % 4; of the scales' image the dword p % 4 of that row.
// A wave moves 32 rows of the tile from `row_at` on and 64 columns of the matrix from `col_first` on (gate_up: 32 of each weight), to the image's rows and columns row_at and col_at; the
// stages `begin` to `end`.  Rows and columns past the last alias it.
template <bool GATE, class P>
struct MxLoader {
    const uint8_t* row[2];            // this lane's chunk in the stage to come
    uint32_t row_scale[2];
    glb_ptr_t col_base[2];            // gate_up: of instructions 0, 1 (gate) and 2, 3 (up)
    glb_ptr_t row_scales, scale_base[2];
    uint32_t col[4];                  // column's first chunk for this lane, from the base
    int t, stages, row_at, col_at;
    __device__ __forceinline__ MxLoader(const MxParams& p, const Lane& ln, const MxTile& tile, int row_at_, int col_at_, int col_first, int begin, int end) {
        const uint32_t pitch = (uint32_t)p.stages * 64;   // of a row's codes; of its scales a sixteenth
        const uint32_t chunk = (ln.l & 3) ^ (ln.l >> 4);
        t = 0;
        stages = end - begin;
        row_at = row_at_, col_at = col_at_;
        row_scales = (glb_ptr_t)p.a_scales;
        uint32_t r[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) r[i] = (uint32_t)(tile.row0 + min(row_at + 16 * i + (ln.l >> 2), tile.rows - 1));
        mx_sources(p, r);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            row[i] = p.a_codes + (size_t)r[i] * pitch + begin * 64 + chunk * 16;
            row_scale[i] = r[i] * (pitch / 16) + begin * 4;
        }
        const size_t expert = (size_t)tile.expert * p.N * pitch + begin * 64;
        col_base[0] = uniform(p.w_codes + expert);
        scale_base[0] = uniform(p.w_scales + expert / 16);
        if (GATE) {
            col_base[1] = uniform(p.u_codes + expert);
            scale_base[1] = uniform(p.u_scales + expert / 16);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) col[i] = (uint32_t)min(col_first + 16 * (GATE ? i & 1 : i) + (ln.l >> 2), p.N - 1) * pitch + chunk * 16;
    }
    // the next stage into the image at `image`; with every fourth stage the scales of it and the next three
    __device__ __forceinline__ void issue(char* smem, uint32_t image) {
        const int l = threadIdx.x & 63;
        if ((t & 3) == 0) {
            const uint32_t at = (uint32_t)min(t + (l & 3), stages - 1) * 4, chunk = (l & 3) ^ (l >> 4);
#pragma unroll
            for (int i = 0; i < 2; ++i) dma4s(row_scales, row_scale[i] + at, smem + P::kScales + (row_at + 16 * i) * 16);
#pragma unroll
            for (int i = 0; i < 4; ++i) dma4s(scale_base[GATE ? i >> 1 : 0], (col[i] >> 4) - chunk + at, smem + P::kColScales + (col_at + 16 * i) * 16);
        }
        char* dst = smem + image;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            dma16((const char*)row[i], dst + (row_at + 16 * i) * 64);
            row[i] += 64;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) dma16s(col_base[GATE ? i >> 1 : 0], col[i], dst + P::kCols + (col_at + 16 * i) * 64);
        col_base[0] += 64;
        if (GATE) col_base[1] += 64;
        ++t;
    }
};
constexpr int kMxRequests = 6;   // of a wave, a stage

// ---- fragments
typedef __attribute__((ext_vector_type(8))) int i32x8_t;
struct MxFrags {
    u32x4_t b[4], a[2];   // rows, columns
};
// A lane's scales of four stages: of stage 2 i + j byte 2 j for its sub-step 0 and 2 j + 1 for sub-step 1.
struct MxScales {
    u32x2_t b[4], a[2];
};
struct MxAddr {
    uint32_t b[2], a[2];   // by sub-step
    uint32_t sb, sa;
    uint32_t pick;         // of two stages' dwords the bytes of this half of the wave
    template <class P>
    __device__ __forceinline__ MxAddr(P, const Lane& ln, char* smem, int col_at) {
        const uint32_t lds0 = lds_addr(smem);
        const int n = col_at + swap23(ln.l31);
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            b[kk] = lds0 + ln.l31 * 64 + (((2 * kk + ln.hf) ^ ((ln.l31 >> 2) & 3)) << 4);
            a[kk] = lds0 + P::kCols + n * 64 + (((2 * kk + ln.hf) ^ ((n >> 2) & 3)) << 4);
        }
        sb = lds0 + P::kScales + ln.l31 * 16;
        sa = lds0 + P::kColScales + n * 16;
        pick = 0x06040200u + 0x01010101u * ln.hf;
    }
};
template <int OFFSET>
__device__ __forceinline__ void read16(u32x4_t& dst, uint32_t addr) {
    asm volatile("ds_read_b128 %0, %1 offset:%2" : "=&v"(dst) : "v"(addr), "n"(OFFSET) : "memory");
}
__device__ __forceinline__ void wait_mx(MxFrags& f) {
    asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(f.b[0]), "+v"(f.b[1]), "+v"(f.b[2]), "+v"(f.b[3]), "+v"(f.a[0]), "+v"(f.a[1])::"memory");
}
__device__ __forceinline__ u32x2_t picked(u32x4_t s, uint32_t pick) {
    return u32x2_t{__builtin_amdgcn_perm(s[1], s[0], pick), __builtin_amdgcn_perm(s[3], s[2], pick)};
}
template <int NTF>
__device__ __forceinline__ void read_scales(MxScales& s, const MxAddr& ad) {
    u32x4_t a0, a1, b0, b1, b2, b3;
    read16<0>(a0, ad.sa);
    read16<512>(a1, ad.sa);
    read16<0>(b0, ad.sb);
    if (NTF > 1) read16<512>(b1, ad.sb);
    if (NTF > 2) read16<1024>(b2, ad.sb);
    if (NTF > 3) read16<1536>(b3, ad.sb);
    asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(a0), "+v"(a1), "+v"(b0), "+v"(b1), "+v"(b2), "+v"(b3)::"memory");
    s.a[0] = picked(a0, ad.pick), s.a[1] = picked(a1, ad.pick), s.b[0] = picked(b0, ad.pick);
    if (NTF > 1) s.b[1] = picked(b1, ad.pick);
    if (NTF > 2) s.b[2] = picked(b2, ad.pick);
    if (NTF > 3) s.b[3] = picked(b3, ad.pick);
}

struct MxAcc {
    f32x16_t a[4][2];
};
// The products of sub-step KK (fragments `cur`, stage S of two) with the reads of `nxt` between them, as in mfma_step_reading.
template <int NTF, int KK, int S>
__device__ __forceinline__ void mx_step(const MxFrags& cur, MxFrags& nxt, uint32_t ad, uint32_t bd, const MxScales& s, MxAcc& acc) {
    auto mm = [&](int tf, int af) {
        const u32x4_t x = cur.a[af], y = cur.b[tf];
        const i32x8_t a = {(int)x[0], (int)x[1], (int)x[2], (int)x[3], 0, 0, 0, 0}, b = {(int)y[0], (int)y[1], (int)y[2], (int)y[3], 0, 0, 0, 0};
        acc.a[tf][af] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, acc.a[tf][af], 4, 4, 2 * S + KK, (int)s.a[af][0], 2 * S + KK, (int)s.b[tf][0]);
    };
    __builtin_amdgcn_sched_barrier(0);
    mm(0, 0);
    __builtin_amdgcn_sched_barrier(0);
    read16<0>(nxt.a[0], ad);
    __builtin_amdgcn_sched_barrier(0);
    mm(0, 1);
    __builtin_amdgcn_sched_barrier(0);
    read16<2048>(nxt.a[1], ad);
    __builtin_amdgcn_sched_barrier(0);
    if (NTF > 1) mm(1, 0);
    __builtin_amdgcn_sched_barrier(0);
    read16<0>(nxt.b[0], bd);
    __builtin_amdgcn_sched_barrier(0);
    if (NTF > 1) mm(1, 1);
    __builtin_amdgcn_sched_barrier(0);
    if (NTF > 1) read16<2048>(nxt.b[1], bd);
    __builtin_amdgcn_sched_barrier(0);
    if (NTF > 2) mm(2, 0);
    __builtin_amdgcn_sched_barrier(0);
    if (NTF > 2) read16<4096>(nxt.b[2], bd);
    __builtin_amdgcn_sched_barrier(0);
    if (NTF > 2) mm(2, 1);
    __builtin_amdgcn_sched_barrier(0);
    if (NTF > 3) read16<6144>(nxt.b[3], bd);
    __builtin_amdgcn_sched_barrier(0);
    if (NTF > 3) mm(3, 0);
    if (NTF > 3) mm(3, 1);
    __builtin_amdgcn_sched_barrier(0);
    // the products stay here: the compiler moved them behind the barrier to come, next to those of the next sub-step
    asm volatile("" : "+v"(acc.a[0][0]), "+v"(acc.a[0][1]));
    if (NTF > 1) asm volatile("" : "+v"(acc.a[1][0]), "+v"(acc.a[1][1]));
    if (NTF > 2) asm volatile("" : "+v"(acc.a[2][0]), "+v"(acc.a[2][1]));
    if (NTF > 3) asm volatile("" : "+v"(acc.a[3][0]), "+v"(acc.a[3][1]));
}

// acc += the tile's product.  Three images: while stage t is multiplied, t + 1 and t + 2 are on their way; t + 3 is requested into t's image behind the barrier that ends
// its reads.  The scales' image is read (stage 4 g) a barrier before it is filled again (with the request of stage 4 g + 4, behind the barrier of stage 4 g + 1).
// P = MxOwn: a wave by itself, whose own order of requests and reads takes the barriers' place.
template <int NTF, bool GATE, class P>
__device__ __forceinline__ void mx_loop(MxLoader<GATE, P>& ld, int nk, char* smem, const MxAddr& ad, MxAcc& acc) {
    auto barrier = [] {
        if (std::is_same<P, MxShared>::value) __builtin_amdgcn_s_barrier();
    };
#pragma unroll
    for (int t = 0; t < kMxImages; ++t)
        if (t < nk) ld.issue(smem, t * P::kStage);
    if (nk > 2) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * kMxRequests) : "memory");
    else if (nk > 1) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kMxRequests) : "memory");
    else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    barrier();
    MxFrags f0, f1;
    MxScales s;
    read_scales<NTF>(s, ad);
    read16<0>(f0.a[0], ad.a[0]);
    read16<2048>(f0.a[1], ad.a[0]);
    read16<0>(f0.b[0], ad.b[0]);
    if (NTF > 1) read16<2048>(f0.b[1], ad.b[0]);
    if (NTF > 2) read16<4096>(f0.b[2], ad.b[0]);
    if (NTF > 3) read16<6144>(f0.b[3], ad.b[0]);
    uint32_t image = 0;
    int t = 0;
    auto stage = [&](auto which) {
        constexpr int S = decltype(which)::value;
        const uint32_t next = image == 2 * P::kStage ? 0 : image + P::kStage;
        wait_mx(f0);
        mx_step<NTF, 0, S>(f0, f1, ad.a[1] + image, ad.b[1] + image, s, acc);
        wait_mx(f1);
        if (t + 1 < nk) {
            if (t + 2 < nk) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(kMxRequests) : "memory");
            else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
            barrier();
            if (t + 3 < nk) ld.issue(smem, image);
        }
        // (behind the last stage it reads what is there)
        mx_step<NTF, 1, S>(f1, f0, ad.a[0] + next, ad.b[0] + next, s, acc);
        image = next;
        ++t;
    };
#pragma unroll 1
    for (int pairs = nk >> 1; pairs > 0; --pairs) {
        stage(std::integral_constant<int, 0>{});
        stage(std::integral_constant<int, 1>{});
        if (t & 2) {
#pragma unroll
            for (int i = 0; i < 2; ++i) s.a[i][0] = s.a[i][1];
#pragma unroll
            for (int i = 0; i < NTF; ++i) s.b[i][0] = s.b[i][1];
        } else if (t < nk) {
            read_scales<NTF>(s, ad);
        }
    }
    if (nk & 1) stage(std::integral_constant<int, 0>{});
    wait_mx(f0);
    barrier();   // every wave has read its last fragments: the images may be refilled
}

// ---- large tiles
// 256 rows by 256 columns (gate_up: 128 of each weight), eight waves of 128 x 64: two thirds of the operand bytes a product, whole lines of 128 bytes (256 values) a row and stage, half the
// barriers; one workgroup a CU.  Wave row m has the rows 64 i + 32 m .. + 31, so that both have work where a tile is not full.  Two images of 64 KB, chunk c of row r at c ^ (r / 2 % 8); four
// sub-steps a stage.  The scales of four stages lie in an image of their own, 32 bytes a row, their halves exchanged where r / 8 is odd.
// K' is a multiple of 128: the last stage may have two sub-steps only; its other half is filled with the first again and not multiplied.
constexpr int kBigThreads = 512;
constexpr int kBigImage = 256 * 128, kBigStage = 2 * kBigImage;
constexpr int kBigScales = 2 * kBigStage;
constexpr int kBigSmem = kBigScales + 512 * 32;
static_assert(kBigSmem <= 160 * 1024, "");
constexpr int kBigRows = 96;   // see mx_large
constexpr int kBigRequests = 8;   // of a wave, a stage, without the scales

// A DMA instruction fills 8 rows of an image, of codes and of scales; wave w moves rows 32 w .. + 31 and as many columns (gate_up: of the gate where w is even).
template <bool GATE>
struct BigLoader {
    const uint8_t* row[4];       // this lane's chunk in the stage to come
    uint32_t col[4];
    glb_ptr_t col_base, rows, row_scales, col_scales;
    int t, blocks, w;            // blocks of 128 values
    static __device__ __forceinline__ uint32_t chunk(int l, int i) { return (l & 7) ^ ((l >> 4) | 4 * (i & 1)); }
    __device__ __forceinline__ void init(const MxParams& p, const Lane& ln, const MxTile& tile) {
        const uint32_t pitch = (uint32_t)p.stages * 64;
        w = ln.wave_uniform();
        t = 0;
        blocks = p.stages;
        const int first = GATE ? tile.col_tile * 128 + 32 * (w >> 1) : tile.col_tile * 256 + 32 * w;
        uint32_t r[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) r[i] = (uint32_t)(tile.row0 + min(32 * w + 8 * i + (ln.l >> 3), tile.rows - 1));
        mx_sources(p, r);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int at = 8 * i + (ln.l >> 3);
            row[i] = p.a_codes + (size_t)r[i] * pitch + chunk(ln.l, i) * 16;
            col[i] = (uint32_t)min(first + at, p.N - 1) * pitch + chunk(ln.l, i) * 16;
        }
        const size_t expert = (size_t)tile.expert * p.N * pitch;
        const bool up = GATE && (w & 1);
        rows = (glb_ptr_t)p.a_codes;
        row_scales = (glb_ptr_t)p.a_scales;
        col_base = uniform((up ? p.u_codes : p.w_codes) + expert);
        col_scales = uniform((up ? p.u_scales : p.w_scales) + expert / 16);
    }
    // this lane, made anew where it is used: what depends on it alone would be kept through the loop, in registers that there are not
    static __device__ __forceinline__ int lane() {
        unsigned l = threadIdx.x;
        asm volatile("" : "+v"(l));
        return (int)(l & 63);
    }
    // 64 bytes back for the lanes that would fetch the second half of a stage that has none
    __device__ __forceinline__ uint32_t back(int l, int i) const { return 2 * t + 1 < blocks ? 0u : (chunk(l, i) & 4) << 4; }
    __device__ __forceinline__ void issue_rows(char* smem, uint32_t image) {
        const int l = lane();
        char* dst = smem + image + w * 4096;
        if ((t & 3) == 0) {
            char* to = smem + kBigScales + w * 1024;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                // a row's scales begin at a sixteenth of where its codes do
                const uint32_t at = (uint32_t)min(2 * t + ((l & 7) ^ 4 * (i & 1)), blocks - 1) * 4 - chunk(l, i);
                dma4s(row_scales, (uint32_t)((uint64_t)((glb_ptr_t)row[i] - rows) >> 4) - 8 * t + at, to + i * 256);
                dma4s(col_scales, (col[i] >> 4) + at, to + 8192 + i * 256);
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            dma16((const char*)row[i] - back(l, i), dst + i * 1024);
            row[i] += 128;
        }
    }
    __device__ __forceinline__ void issue_cols(char* smem, uint32_t image) {
        const int l = lane();
        char* dst = smem + image + kBigImage + w * 4096;
#pragma unroll
        for (int i = 0; i < 4; ++i) dma16s(col_base, col[i] - back(l, i), dst + i * 1024);
        col_base += 128;
        ++t;
    }
};

struct BigAddr {
    uint32_t b, a;   // of sub-step 0; a sub-step's chunks are 2 kk further, before the exchange by the row
    uint32_t sb, sa, pick;
    __device__ __forceinline__ BigAddr(const Lane& ln, char* smem) {
        const uint32_t lds0 = lds_addr(smem);
        const int n = swap23(ln.l31);
        b = lds0 + (32 * ln.wm + ln.l31) * 128 + ((ln.hf ^ ((ln.l31 >> 1) & 7)) << 4);
        a = lds0 + kBigImage + (64 * ln.wn + n) * 128 + ((ln.hf ^ ((n >> 1) & 7)) << 4);
        sb = lds0 + kBigScales + (32 * ln.wm + ln.l31) * 32 + ((ln.l31 >> 3) & 1) * 16;
        sa = lds0 + kBigScales + 8192 + (64 * ln.wn + n) * 32 + ((n >> 3) & 1) * 16;
        pick = 0x06040200u + 0x01010101u * ln.hf;
    }
    template <int KK>
    __device__ __forceinline__ uint32_t row(uint32_t image) const { return (b ^ (KK << 5)) + image; }
    template <int KK>
    __device__ __forceinline__ uint32_t col(uint32_t image) const { return (a ^ (KK << 5)) + image; }
};
// As mx_step; BYTE: of the lane's scales.  ad, bd: where the next fragments are.
template <int NTF, int BYTE, bool READ>
__device__ __forceinline__ void big_step(const MxFrags& cur, MxFrags& nxt, uint32_t ad, uint32_t bd, const MxScales& s, MxAcc& acc) {
    auto mm = [&](int tf, int af) {
        const u32x4_t x = cur.a[af], y = cur.b[tf];
        const i32x8_t a = {(int)x[0], (int)x[1], (int)x[2], (int)x[3], 0, 0, 0, 0}, b = {(int)y[0], (int)y[1], (int)y[2], (int)y[3], 0, 0, 0, 0};
        acc.a[tf][af] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, acc.a[tf][af], 4, 4, BYTE, (int)s.a[af][0], BYTE, (int)s.b[tf][0]);
    };
    __builtin_amdgcn_sched_barrier(0);
    mm(0, 0);
    __builtin_amdgcn_sched_barrier(0);
    if (READ) read16<0>(nxt.a[0], ad);
    __builtin_amdgcn_sched_barrier(0);
    mm(0, 1);
    __builtin_amdgcn_sched_barrier(0);
    if (READ) read16<4096>(nxt.a[1], ad);
    __builtin_amdgcn_sched_barrier(0);
    if (NTF > 1) mm(1, 0);
    __builtin_amdgcn_sched_barrier(0);
    if (READ) read16<0>(nxt.b[0], bd);
    __builtin_amdgcn_sched_barrier(0);
    if (NTF > 1) mm(1, 1);
    __builtin_amdgcn_sched_barrier(0);
    if (READ && NTF > 1) read16<8192>(nxt.b[1], bd);
    __builtin_amdgcn_sched_barrier(0);
    if (NTF > 2) mm(2, 0);
    __builtin_amdgcn_sched_barrier(0);
    if (READ && NTF > 2) read16<16384>(nxt.b[2], bd);
    __builtin_amdgcn_sched_barrier(0);
    if (NTF > 2) mm(2, 1);
    __builtin_amdgcn_sched_barrier(0);
    if (READ && NTF > 3) read16<24576>(nxt.b[3], bd);
    __builtin_amdgcn_sched_barrier(0);
    if (NTF > 3) mm(3, 0);
    if (NTF > 3) mm(3, 1);
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("" : "+v"(acc.a[0][0]), "+v"(acc.a[0][1]));
    if (NTF > 1) asm volatile("" : "+v"(acc.a[1][0]), "+v"(acc.a[1][1]));
    if (NTF > 2) asm volatile("" : "+v"(acc.a[2][0]), "+v"(acc.a[2][1]));
    if (NTF > 3) asm volatile("" : "+v"(acc.a[3][0]), "+v"(acc.a[3][1]));
}
// Stages 0 and 1 are requested together; t + 2 behind the barrier that ends the reads of t, its columns behind the next products.  The scales' image (of stages 4 g .. 4 g + 3) is read at the
// beginning of stages 4 g and 4 g + 2 and requested again with stage 4 g + 4, behind the barrier of stage 4 g + 2.  NTF = 0: a wave without rows moves operands.
template <int NTF, bool GATE>
__device__ __forceinline__ void big_loop(BigLoader<GATE>& ld, int blocks, char* smem, const BigAddr& ad, MxAcc& acc) {
    const int nk = (blocks + 1) >> 1, whole = blocks >> 1;
    ld.issue_rows(smem, 0);
    ld.issue_cols(smem, 0);
    if (nk > 1) {
        ld.issue_rows(smem, kBigStage);
        ld.issue_cols(smem, kBigStage);
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kBigRequests) : "memory");
    } else {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    }
    __builtin_amdgcn_s_barrier();
    MxFrags f0, f1;
    MxScales s;
    auto scales = [&](int t) {
        if (NTF == 0) return;
        const uint32_t half = (t & 2) << 3, sa = ad.sa ^ half, sb = ad.sb ^ half;
        u32x4_t a0, a1, b0, b1, b2, b3;
        read16<0>(a0, sa);
        read16<1024>(a1, sa);
        read16<0>(b0, sb);
        if (NTF > 1) read16<2048>(b1, sb);
        if (NTF > 2) read16<4096>(b2, sb);
        if (NTF > 3) read16<6144>(b3, sb);
        asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(a0), "+v"(a1), "+v"(b0), "+v"(b1), "+v"(b2), "+v"(b3)::"memory");
        s.a[0] = picked(a0, ad.pick), s.a[1] = picked(a1, ad.pick), s.b[0] = picked(b0, ad.pick);
        if (NTF > 1) s.b[1] = picked(b1, ad.pick);
        if (NTF > 2) s.b[2] = picked(b2, ad.pick);
        if (NTF > 3) s.b[3] = picked(b3, ad.pick);
    };
    scales(0);
    if (NTF > 0) {
        read16<0>(f0.a[0], ad.a);
        read16<4096>(f0.a[1], ad.a);
        read16<0>(f0.b[0], ad.b);
        if (NTF > 1) read16<8192>(f0.b[1], ad.b);
        if (NTF > 2) read16<16384>(f0.b[2], ad.b);
        if (NTF > 3) read16<24576>(f0.b[3], ad.b);
    }
#pragma unroll 1
    for (int t = 0; t < whole; ++t) {
        const uint32_t image = (t & 1) * kBigStage, next = kBigStage - image;
        if (NTF > 0) {
            wait_mx(f0);
            big_step<NTF, 0, true>(f0, f1, ad.template col<1>(image), ad.template row<1>(image), s, acc);
            wait_mx(f1);
            big_step<NTF, 1, true>(f1, f0, ad.template col<2>(image), ad.template row<2>(image), s, acc);
            wait_mx(f0);
            big_step<NTF, 2, true>(f0, f1, ad.template col<3>(image), ad.template row<3>(image), s, acc);
            wait_mx(f1);
        }
        if (t + 1 < nk) {
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
            __builtin_amdgcn_s_barrier();
            if (t + 2 < nk) ld.issue_rows(smem, image);
        }
        if (NTF > 0) big_step<NTF, 3, true>(f1, f0, ad.template col<0>(next), ad.template row<0>(next), s, acc);   // (behind the last stage it reads what is there)
        if (t + 2 < nk) ld.issue_cols(smem, image);
        if ((t & 1) == 0) {
#pragma unroll
            for (int i = 0; i < 2; ++i) s.a[i][0] = s.a[i][1];
#pragma unroll
            for (int i = 0; i < NTF; ++i) s.b[i][0] = s.b[i][1];
        } else if (t + 1 < nk) {
            scales(t + 1);
        }
    }
    if (NTF > 0) {
        wait_mx(f0);
        if (blocks & 1) {
            const uint32_t image = (whole & 1) * kBigStage;
            big_step<NTF, 0, true>(f0, f1, ad.template col<1>(image), ad.template row<1>(image), s, acc);
            wait_mx(f1);
            big_step<NTF, 1, false>(f1, f0, 0, 0, s, acc);
        }
    }
    __builtin_amdgcn_s_barrier();   // every wave has read its last fragments: the images may be refilled
}

// ---- what becomes of the accumulators
// BIG: wave row m has the tile's rows 64 i + 32 m .. + 31
template <bool BIG>
__device__ __forceinline__ int mx_tile_row(const Lane& ln, int row) {
    return BIG ? 64 * (row >> 5) + 32 * ln.wm + (row & 31) : row;
}
template <bool BIG>
__device__ __forceinline__ void mx_store(const MxParams& p, const MxTile& t, const MxAcc& acc, char* smem) {
    const Lane ln;
    WaveRepack<8> rp(smem, ln);
    if (!p.f32) {
#pragma unroll
        for (int tf = 0; tf < 4; ++tf)
#pragma unroll
            for (int af = 0; af < 2; ++af)
#pragma unroll
                for (int vg = 0; vg < 2; ++vg) rp.put(32 * tf + ln.l31, 4 * af + 2 * vg + ln.hf, pack8(acc.a[tf][af], vg));
        const int col = t.col_tile * kMxCols + 64 * ln.wn + 8 * rp.get_piece();
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            const int row = mx_tile_row<BIG>(ln, rp.get_row(j));
            const u32x4_t v = rp.get(j);
            if (row < t.rows && col < p.N) store_stream16((uint16_t*)p.y + (size_t)(t.row0 + row) * p.N + col, v);
        }
        return;
    }
#pragma unroll
    for (int af = 0; af < 2; ++af) {
#pragma unroll
        for (int tf = 0; tf < 4; ++tf)
#pragma unroll
            for (int i = 0; i < 4; ++i) {   // four columns: 16 (i / 2) + 8 half + 4 (i % 2)
                u32x4_t v;
#pragma unroll
                for (int q = 0; q < 4; ++q) v[q] = __float_as_uint(acc.a[tf][af][4 * i + q]);
                rp.put(32 * tf + ln.l31, 4 * (i >> 1) + 2 * ln.hf + (i & 1), v);
            }
        const int col = t.col_tile * kMxCols + 64 * ln.wn + 32 * af + 4 * rp.get_piece();
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            const int row = mx_tile_row<BIG>(ln, rp.get_row(j));
            const u32x4_t v = rp.get(j);
            if (row < t.rows && col < p.N) store_stream16((float*)p.y + (size_t)(t.row0 + row) * p.N + col, v);
        }
    }
}

// h of eight columns, rounded to bf16.
__device__ __forceinline__ u32x4_t mx_h8(const f32x16_t& g, const f32x16_t& u, int vg) {
    u32x4_t r;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        float h[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const float x = g[8 * vg + 2 * q + e];
            h[e] = x * sigmoid_f(x) * u[8 * vg + 2 * q + e];
        }
        r[q] = pack_bf16x2(h[0], h[1]);
    }
    return r;
}
template <bool BIG>
__device__ __forceinline__ void mx_store_h(const MxParams& p, const MxTile& t, const MxAcc& acc, char* smem) {
    const Lane ln;
    const int col0 = t.col_tile * (kMxCols / 2) + 32 * ln.wn;
    if (p.y) {
        WaveRepack<4> rp(smem, ln);
#pragma unroll
        for (int tf = 0; tf < 4; ++tf)
#pragma unroll
            for (int vg = 0; vg < 2; ++vg) rp.put(32 * tf + ln.l31, 2 * vg + ln.hf, mx_h8(acc.a[tf][0], acc.a[tf][1], vg));
        const int col = col0 + 8 * rp.get_piece();
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int row = mx_tile_row<BIG>(ln, rp.get_row(j));
            const u32x4_t v = rp.get(j);
            if (row < t.rows && col < p.N) store_stream16((uint16_t*)p.y + (size_t)(t.row0 + row) * p.N + col, v);
        }
        return;
    }
    // The wave's 32 columns are a block: 16 values in either half of the wave.  What is quantised is h as the bf16 result would be, so that both ways
    // to the next product give the same bits (a second rounding of 2^-8 before one of 2^-2).
    // A lane's 8 bytes and a block's byte leave as they are, in pieces of a row; a quarter of the bytes takes as long as the bf16 result.  us, 4 bits / bf16: 8 of 4096 x 14336, 8002 rows 517 / 512; 128 of 2048 x 768, 65536 rows
    // 154 / 153, 8 rows 7.7 / 7.5; 7168 x 2048 for 37 tokens 63 / 63; where the reductions are short, 64 of 512 x 1024, 8192 rows 16.3 / 15.5, 32768 rows 43 / 41.
    const int pitch = mx_padded(p.N);
    if (col0 >= pitch) return;
#pragma unroll
    for (int tf = 0; tf < 4; ++tf) {
        float v[2][8];
        uint32_t m = 0;
#pragma unroll
        for (int vg = 0; vg < 2; ++vg) {
            const u32x4_t h = mx_h8(acc.a[tf][0], acc.a[tf][1], vg);
            const bool in = col0 + 16 * vg + 8 * ln.hf < p.N;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                v[vg][2 * q] = in ? bf16_lo(h[q]) : 0.f;
                v[vg][2 * q + 1] = in ? bf16_hi(h[q]) : 0.f;
                m = max(m, max(mag(v[vg][2 * q]), mag(v[vg][2 * q + 1])));
            }
        }
        const uint32_t byte = mx4_byte(max_halves(m));
        // the halves exchange their outer eights, so that each has eight bytes of the block in a row
        const auto c = __builtin_amdgcn_permlane32_swap(mx4_codes(v[0], byte), mx4_codes(v[1], byte), false, false);
        const int row = mx_tile_row<BIG>(ln, 32 * tf + ln.l31);
        if (row < t.rows) {
            const size_t at = (size_t)(t.row0 + row) * pitch + col0;
            *(u32x2_t*)(p.h_codes + at / 2 + 8 * ln.hf) = u32x2_t{c[0], c[1]};
            if (ln.hf == 0) p.h_scales[at / kMxBlock] = (uint8_t)byte;
        }
    }
}

// ---- few rows
// An expert with up to 32 rows is bound by its weights: a tile is all of its rows by 64 columns (gate_up: 32 of each weight), so that there are enough of them for every CU, and each of the
// four waves has a quarter of the reduction, with images of its own and no barrier.  Their sums are added in LDS in the order of the waves.
constexpr int kThinPitch = 64 + 4;   // floats of a row of a wave's sums
template <bool GATE>
__device__ __forceinline__ void thin_tile(const MxParams& p, const MxTile& t, char* smem) {
    const int each = ((p.stages + 3) / 4 + 1) & ~1;   // (whole lines of 128 bytes)
    MxAcc acc;
#pragma unroll
    for (int af = 0; af < 2; ++af)
#pragma unroll
        for (int v = 0; v < 16; ++v) acc.a[0][af][v] = 0.f;
    const int waves = (p.stages + each - 1) / each;
    {
        const Lane ln;
        const int w = ln.wave_uniform();
        if (w < waves) {
            char* own = smem + w * MxOwn::kBytes;
            const int begin = w * each, end = min(begin + each, p.stages);
            MxLoader<GATE, MxOwn> ld(p, ln, t, 0, 0, (GATE ? 32 : 64) * t.col_tile, begin, end);
            const MxAddr ad(MxOwn{}, ln, own, 0);
            mx_loop<1, GATE>(ld, end - begin, own, ad, acc);
        }
    }
    __syncthreads();   // (the sums take the images' place)
    const Lane ln;
    const int w = ln.wave_uniform();
    float* const sums = (float*)smem;
    if (ln.l31 < t.rows && w < waves)
#pragma unroll
        for (int af = 0; af < 2; ++af)
#pragma unroll
            for (int i = 0; i < 4; ++i)   // columns 16 (i / 2) + 8 half + 4 (i % 2)
                *(f32x4_t*)(sums + (w * kThinRows + ln.l31) * kThinPitch + 32 * af + 16 * (i >> 1) + 8 * ln.hf + 4 * (i & 1)) =
                    f32x4_t{acc.a[0][af][4 * i], acc.a[0][af][4 * i + 1], acc.a[0][af][4 * i + 2], acc.a[0][af][4 * i + 3]};
    __syncthreads();
    auto sum = [&](int row, int c) {
        f32x4_t v = *(const f32x4_t*)(sums + row * kThinPitch + c);
        for (int i = 1; i < waves; ++i) v += *(const f32x4_t*)(sums + (i * kThinRows + row) * kThinPitch + c);
        return v;
    };
    // eight threads a row
    const int r = threadIdx.x >> 3, piece = threadIdx.x & 7;
    if (r < t.rows) {
        const size_t out = (size_t)(t.row0 + r);
        if (!GATE) {
            const int c = 64 * t.col_tile + 8 * piece;
            if (c < p.N) {
                const f32x4_t a = sum(r, 8 * piece), b = sum(r, 8 * piece + 4);
                if (p.f32) {
                    *(f32x4_t*)((float*)p.y + out * p.N + c) = a;
                    *(f32x4_t*)((float*)p.y + out * p.N + c + 4) = b;
                } else {
                    *(u32x4_t*)((uint16_t*)p.y + out * p.N + c) = u32x4_t{pack_bf16x2(a[0], a[1]), pack_bf16x2(a[2], a[3]), pack_bf16x2(b[0], b[1]), pack_bf16x2(b[2], b[3])};
                }
            }
        } else {
            const int c = 32 * t.col_tile + 4 * piece;
            const f32x4_t g = sum(r, 4 * piece), u = sum(r, 32 + 4 * piece);
            float h[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) h[i] = g[i] * sigmoid_f(g[i]) * u[i];
            const u32x2_t b = {pack_bf16x2(h[0], h[1]), pack_bf16x2(h[2], h[3])};
            if (p.y) {
                if (c < p.N) *(u32x2_t*)((uint16_t*)p.y + out * p.N + c) = b;
            } else {
                float v[4] = {bf16_lo(b[0]), bf16_hi(b[0]), bf16_lo(b[1]), bf16_hi(b[1])};
                uint32_t m = 0;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    v[i] = c < p.N ? v[i] : 0.f;
                    m = max(m, mag(v[i]));
                }
                m = max_quad(m);
                m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, m, 0x141, 0xf, 0xf, true));   // row_half_mirror: the other four of the eight
                const uint32_t byte = mx4_byte(m);
                const float s = scale_of(byte);
                uint32_t codes = 0;
                codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, v[0], v[1], s, 0);
                codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, v[2], v[3], s, 1);
                const size_t at = out * mx_padded(p.N) + c;   // (N filled up to a multiple of 128: all of the tile's columns are inside)
                *(uint16_t*)(p.h_codes + at / 2) = (uint16_t)(byte == kMxNan ? 0u : codes);
                if (piece == 0) p.h_scales[at / kMxBlock] = (uint8_t)byte;
            }
        }
    }
}

__device__ __forceinline__ void mx_zero(MxAcc& acc) {
#pragma unroll
    for (int tf = 0; tf < 4; ++tf)
#pragma unroll
        for (int af = 0; af < 2; ++af)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc.a[tf][af][v] = 0.f;
}
// This workgroup's tiles: run(tile) one after the other.
template <int ROWS, bool THIN, class F>
__device__ __forceinline__ void mx_each_tile(const MxParams& p, F run) {
    const MxTiles<ROWS, THIN> tiles(p);
    const int xcd = blockIdx.x % kQueues, each = gridDim.x / kQueues;   // (the grid is a multiple of kQueues)
    const int lo = (int)((long long)tiles.total * xcd / kQueues), hi = (int)((long long)tiles.total * (xcd + 1) / kQueues);
    for (int i = lo + (int)(blockIdx.x / kQueues); i < hi; i += each) {
        run(tiles.find(p, i));
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();   // the stores' LDS is read
    }
}

template <bool GATE>
__global__ void __launch_bounds__(kMxThreads, 2) mx_product_kernel(MxParams p) {
    extern __shared__ __attribute__((aligned(16))) char smem[];
    mx_each_tile<kMxRows, true>(p, [&](const MxTile& t) {
        if (t.thin) {
            thin_tile<GATE>(p, t, smem);
            return;
        }
        MxAcc acc;
        mx_zero(acc);
        {
            const Lane ln;
            const int w = ln.wave_uniform();
            MxLoader<GATE, MxShared> ld(p, ln, t, 32 * w, 64 * w, GATE ? t.col_tile * (kMxCols / 2) + 32 * w : t.col_tile * kMxCols + 64 * w, 0, p.stages);
            const MxAddr ad(MxShared{}, ln, smem, 64 * w);
            const int ntf = (t.rows + 31) >> 5;
            if (ntf == 4) mx_loop<4, GATE>(ld, p.stages, smem, ad, acc);
            else if (ntf == 3) mx_loop<3, GATE>(ld, p.stages, smem, ad, acc);
            else if (ntf == 2) mx_loop<2, GATE>(ld, p.stages, smem, ad, acc);
            else mx_loop<1, GATE>(ld, p.stages, smem, ad, acc);
        }
        if (GATE) mx_store_h<false>(p, t, acc, smem);
        else mx_store<false>(p, t, acc, smem);
    });
}

template <bool GATE>
__global__ void __launch_bounds__(kBigThreads, 2) mx_big_kernel(MxParams p) {
    extern __shared__ __attribute__((aligned(16))) char smem[];
    mx_each_tile<256, false>(p, [&](const MxTile& t) {
        MxAcc acc;
        mx_zero(acc);
        {
            const Lane ln;
            BigLoader<GATE> ld;
            ld.init(p, ln, t);
            const BigAddr ad(ln, smem);
            const int ntf = min(max((t.rows - 32 * (ln.wave_uniform() >> 2) + 63) >> 6, 0), 4);
            if (ntf == 4) big_loop<4, GATE>(ld, p.stages, smem, ad, acc);
            else if (ntf == 3) big_loop<3, GATE>(ld, p.stages, smem, ad, acc);
            else if (ntf == 2) big_loop<2, GATE>(ld, p.stages, smem, ad, acc);
            else if (ntf == 1) big_loop<1, GATE>(ld, p.stages, smem, ad, acc);
            else big_loop<0, GATE>(ld, p.stages, smem, ad, acc);
        }
        if (GATE) mx_store_h<true>(p, t, acc, smem);
        else mx_store<true>(p, t, acc, smem);
    });
}

namespace {
// Launches one of the kernels with as many workgroups as run at a time, or as there can be tiles.  How many run is asked once a device.
template <class K>
int mx_launch(K kernel, int threads, int smem, int (&known)[kMaxDevices], int64_t tiles, MxParams p, hipStream_t st) {
    static std::mutex lock;
    int dev = 0, resident = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= kMaxDevices) return MOE_ERR_HIP;
    {
        std::lock_guard<std::mutex> guard(lock);
        if (known[dev] == 0) {
            int per_cu = 0, cus = 0;
            if (hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, smem) != hipSuccess ||
                hipOccupancyMaxActiveBlocksPerMultiprocessor(&per_cu, kernel, threads, smem) != hipSuccess ||
                hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || per_cu < 1)
                return MOE_ERR_HIP;
            known[dev] = (per_cu * cus + kQueues - 1) / kQueues * kQueues;
        }
        resident = known[dev];
    }
    p.slots = resident;
    const int grid = tiles < resident ? ((int)tiles + kQueues - 1) / kQueues * kQueues : resident;
    hipLaunchKernelGGL(kernel, dim3(grid), dim3(threads), smem, st, p);
    return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP;
}
int g_resident[4][kMaxDevices];

// Large tiles move two thirds of the operands' bytes, but half as many of them run on a CU, one instead of two: they pay in long reductions and in many rounds, and not where they leave CUs idle.
// `large` and `wide`: how often the 256 CUs are filled, were half of every expert's last tile used; the rest of the rule (a tile's time by its stages, what a first round costs more) is fitted to a
// thousand sizes in both kinds, 64 to 1000 rows an expert on average, inputs from memory: 1.4 % above the better kind on average and 11 % in the worst twentieth (ten stages and 96 rows as the limits: 2.9 and 20 %).
// us, 128 x 256 / 256 x 256, by the rows of an expert on average:
//   gate_up, 32 of 7168 x 2048        100 146 / 132, 230 210 / 177, 512 363 / 301, 1000 646 / 506
//   gate_up, 8 of 4096 x 14336        100 139 / 130, 230 201 / 177, 512 356 / 308, 1000 642 / 522
//   gate_up, 256 of 2048 x 768        100 124 / 132, 230 187 / 177, 512 333 / 303, 1000 596 / 519
//   gate_up, 64 of 512 x 1024         100 15 / 24, 230 22 / 26, 512 41 / 47, 1000 72 / 76
//   product, 32 of 1408 x 2048        100 18 / 18, 230 25 / 28, 512 40 / 44, 1000 71 / 73
//   product, 64 of 2048 x 1024        100 23 / 29, 230 34 / 34, 512 62 / 60, 1000 117 / 103
//   product, 128 of 768 x 2048        100 44 / 48, 230 69 / 69, 512 126 / 118, 1000 216 / 204
//   product, 8 of 4096 x 2048         100 21 / 21, 230 22 / 26, 512 37 / 29, 700 40 / 32
// The rows are those that the buffer has room for, as only the device knows how many there are; a share of the experts fills its part of them, and the choice may be the slower one.  Of 144 shares (1/4, 1/8
// and 1/16 of 128 and 256 experts, 256 to 8192 tokens of 8, products of 768 x 2048 and 2048 x 7168, gate_up of 2048 x 768 and 7168 x 2048) 90 are done in large tiles and take 6 % more than in
// the better kind on average, 24 % in the worst twentieth; by the rows that are there it would be 2.5 and 17 %.  us, 128 x 256 / 256 x 256:
//   gate_up, 16 of 128 of 7168 x 2048   256 tokens 53 / 56, 1024 78 / 62, 2048 91 / 93, 8192 200 / 171
//   gate_up, 32 of 256 of 2048 x 768    2048 tokens 15 / 17, 4096 22 / 20, 8192 25 / 35
//   gate_up, 8 of 128 of 7168 x 2048    256 tokens 38 / 48, 2048 46 / 56, 4096 66 / 56
//   product, 32 of 256 of 768 x 2048    4096 tokens 13 / 17, 8192 17 / 20
//   product, 16 of 128 of 2048 x 7168   512 tokens 30 / 34, 2048 42 / 41, 8192 106 / 97
// The 256 CUs are the whole chip's; a part of it as a device of its own would be filled more often than the rule says.
bool mx_large(int rows, int64_t experts, int col_tiles, int stages) {
    if (rows / experts < kBigRows) return false;
    const float large = (rows / 256.f + experts / 2.f) * col_tiles / 256.f, wide = (rows / 128.f + experts / 2.f) * col_tiles / 512.f;
    return (0.56f + 1.5f / stages) * (large + 1.6f) < wide + 0.8f;
}
}  // namespace

int mx_product_launch(const moe_mx_shape_t& s, bool gate, const uint8_t* a_codes, const uint8_t* a_scales, int64_t a_rows, const int32_t* perm, int k,
                      const uint8_t* w_codes, const uint8_t* w_scales, const uint8_t* u_codes, const uint8_t* u_scales, const int32_t* offsets, void* y, int f32,
                      uint8_t* h_codes, uint8_t* h_scales, hipStream_t st) {
    if (s.rows == 0 || a_rows == 0) return MOE_OK;
    MxParams p = {};
    p.rows = s.rows, p.N = s.N, p.experts = s.experts;
    p.stages = mx_padded(s.K) / kMxStageK;
    const int cols = gate ? kMxCols / 2 : kMxCols;
    p.col_tiles = ((h_codes ? mx_padded(s.N) : s.N) + cols - 1) / cols;
    const int narrow = gate ? 32 : 64;
    p.thin_tiles = ((h_codes ? mx_padded(s.N) : s.N) + narrow - 1) / narrow;
    p.a_rows = (uint32_t)a_rows, p.a_codes = a_codes, p.a_scales = a_scales, p.perm = perm, p.k = k;
    p.w_codes = w_codes, p.w_scales = w_scales, p.u_codes = u_codes, p.u_scales = u_scales;
    p.offsets = offsets, p.y = y, p.f32 = f32, p.h_codes = h_codes, p.h_scales = h_scales;
    const int64_t experts = s.experts < s.rows ? s.experts : s.rows;
    if (mx_large(s.rows, experts, p.col_tiles, p.stages)) {
        const int64_t most = (s.rows / 256 + experts) * p.col_tiles;
        return gate ? mx_launch(mx_big_kernel<true>, kBigThreads, kBigSmem, g_resident[3], most, p, st)
                    : mx_launch(mx_big_kernel<false>, kBigThreads, kBigSmem, g_resident[2], most, p, st);
    }
    const int64_t most = (int64_t)s.rows / kMxRows * p.col_tiles + experts * p.thin_tiles;
    return gate ? mx_launch(mx_product_kernel<true>, kMxThreads, kMxSmem, g_resident[1], most, p, st)
                : mx_launch(mx_product_kernel<false>, kMxThreads, kMxSmem, g_resident[0], most, p, st);
}

}  // namespace uniep
