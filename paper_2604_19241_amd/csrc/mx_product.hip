// Products of expert-sorted rows with their experts' weights, both in microscaled 4-bit floating point (mx.hpp):
//   product   y[r] = a[src(r)] W_e^T              for the rows r of expert e, offsets[e] <= r < offsets[e + 1]
//   gate_up   h[r] = silu(a[src(r)] Wg_e^T) * (a[src(r)] Wu_e^T), in bf16 or quantised again
// src(r) = perm[r] / k where there is a table (the rows' tokens), else r.
//
// v_mfma_scale_f32_32x32x64_f8f6f4 takes 32 values of a row and one scale a lane: exactly a block.  It runs four times as many products a clock as the bf16 instruction on
// as many bytes, so that a tile needs its operands as fast as a bf16 tile does, for four times the reduction.  At the row counts of a layer's experts (hundreds) the weights, read once
// from memory, take longer than the matrix work.
//
// Tile: 128 rows by 256 columns (gate_up: 128 columns of each weight) by four waves, each with all rows of 64 columns: 4 x 2 accumulators of 32 x 32.  K advances 128 values a stage, 64 bytes
// a row, by DMA into one of three images (24 KB); chunk c of row r lies at c ^ (r / 4 % 4), so that fragments are read without bank conflicts.  Two workgroups share a
// CU (78 KB of LDS and 256 registers a lane each): one's first stages and stores run behind the other's matrix work, as a tile has only K / 128 stages.
// Scales: four stages' bytes of a row are 16 of memory; they are moved a dword a lane into an image of their own, and one LDS read a fragment and four stages hands a lane its row's.
// A lane takes values 32 (2 s + half) .. + 31 of sub-step s, so its scale is byte 2 s + half of the stage's dword: the dword is shifted by the half once, and the
// instruction selects byte 0 or 2.
//
// Tiles are listed expert by expert, columns by columns, rows fastest, and dealt to the XCDs in eight runs: the tiles that share weights and rows meet in one L2.
#include "mma.hpp"
#include "mx.hpp"

#include <mutex>

namespace uniep {

constexpr int kMxRows = 128, kMxCols = 256;
constexpr int kMxStageK = 128;                       // values
constexpr int kMxRowImage = kMxRows * 64, kMxStage = kMxRowImage + kMxCols * 64;
constexpr int kMxImages = 3;
constexpr int kMxScales = kMxImages * kMxStage;      // where the scales' image lies: 16 bytes a row, then a column
constexpr int kMxSmem = kMxScales + (kMxRows + kMxCols) * 16;
constexpr int kMxThreads = 256;
static_assert(2 * kMxSmem <= 160 * 1024, "");
static_assert(kMxStageK == kMxPad, "");

struct MxParams {
    int rows, N, experts;
    int stages;               // K' / 128
    int col_tiles;
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
};
// A wave's view of the experts: lane l has `per` of them from l * per on.
struct MxTiles {
    int per, before, total;   // tiles of the lanes before this one
    int row0, n;              // of the lane's only expert (per = 1)
    static __device__ __forceinline__ void rows_of(const MxParams& p, int e, int& row0, int& n) {
        row0 = n = 0;
        if (e >= p.experts) return;
        row0 = min(max(p.offsets[e], 0), p.rows);
        n = min(max(p.offsets[e + 1], row0), p.rows) - row0;
    }
    static __device__ __forceinline__ int tiles_of(const MxParams& p, int n) { return (n + kMxRows - 1) / kMxRows * p.col_tiles; }
    __device__ __forceinline__ explicit MxTiles(const MxParams& p) {
        const int lane = threadIdx.x & 63;
        per = (p.experts + 63) >> 6;
        int mine = 0;
        for (int j = 0; j < per; ++j) {
            rows_of(p, lane * per + j, row0, n);
            mine += tiles_of(p, n);
        }
        const int upto = wave_scan(mine);
        before = upto - mine;
        total = __builtin_amdgcn_readlane(upto, 63);
    }
    // tile i of 0 .. total - 1
    __device__ __forceinline__ MxTile find(const MxParams& p, int i) const {
        const int lane = threadIdx.x & 63;
        int l = 63 - __builtin_clzll(__ballot(before <= i));   // (lane 0 has 0)
        int base = __builtin_amdgcn_readlane(before, l), r0 = row0, m = n, e = l;
        if (per > 1) {
            rows_of(p, lane < per ? l * per + lane : p.experts, r0, m);
            const int mine = tiles_of(p, m), upto = wave_scan(mine);
            const int first = upto - mine, at = i - base;
            const int j = 63 - __builtin_clzll(__ballot(lane < per && first <= at));
            base += __builtin_amdgcn_readlane(first, j);
            e = l * per + j;
            l = j;
        }
        MxTile t;
        t.expert = rfl(e);
        const int begin = __builtin_amdgcn_readlane(r0, l), count = __builtin_amdgcn_readlane(m, l);
        const int row_tiles = (count + kMxRows - 1) / kMxRows, at = i - base;
        t.col_tile = rfl(at / row_tiles);
        const int first = rfl(at - t.col_tile * row_tiles) * kMxRows;
        t.row0 = begin + first;
        t.rows = min(count - first, kMxRows);
        return t;
    }
};

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

// A DMA instruction fills 16 rows of an image: lane p the chunk of row p / 4 that belongs at position p % 4; of the scales' image the dword p % 4 of that row.
// Wave w moves rows 32 w .. + 31 and columns 64 w .. + 63.  Rows and columns past the last alias it.
template <bool GATE>
struct MxLoader {
    const uint8_t* row[2];            // this lane's chunk in the stage to come
    uint32_t row_scale[2];
    glb_ptr_t col_base[2];            // gate_up: of instructions 0, 1 (gate) and 2, 3 (up)
    glb_ptr_t row_scales, scale_base[2];
    uint32_t col[4];                  // column's first chunk for this lane, from the base
    int t, stages, w;
    __device__ __forceinline__ MxLoader(const MxParams& p, const Lane& ln, const MxTile& tile) {
        const uint32_t pitch = (uint32_t)p.stages * 64;   // of a row's codes; of its scales a sixteenth
        const uint32_t chunk = (ln.l & 3) ^ (ln.l >> 4);
        w = ln.wave_uniform();
        t = 0;
        stages = p.stages;
        row_scales = (glb_ptr_t)p.a_scales;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            uint32_t r = (uint32_t)(tile.row0 + min(32 * w + 16 * i + (ln.l >> 2), tile.rows - 1));
            if (p.perm) r = (uint32_t)p.perm[r] / (uint32_t)p.k;
            r = min(r, p.a_rows - 1);
            row[i] = p.a_codes + (size_t)r * pitch + chunk * 16;
            row_scale[i] = r * (pitch / 16);
        }
        const size_t expert = (size_t)tile.expert * p.N * pitch;
        col_base[0] = uniform(p.w_codes + expert);
        scale_base[0] = uniform(p.w_scales + expert / 16);
        if (GATE) {
            col_base[1] = uniform(p.u_codes + expert);
            scale_base[1] = uniform(p.u_scales + expert / 16);
        }
        const int first = GATE ? tile.col_tile * (kMxCols / 2) + 32 * w : tile.col_tile * kMxCols + 64 * w;
#pragma unroll
        for (int i = 0; i < 4; ++i) col[i] = (uint32_t)min(first + 16 * (GATE ? i & 1 : i) + (ln.l >> 2), p.N - 1) * pitch + chunk * 16;
    }
    // the next stage into the image at `image`; with every fourth stage the scales of it and the next three
    __device__ __forceinline__ void issue(char* smem, uint32_t image) {
        const int l = threadIdx.x & 63;
        if ((t & 3) == 0) {
            const uint32_t at = (uint32_t)min(t + (l & 3), stages - 1) * 4, chunk = (l & 3) ^ (l >> 4);
            char* dst = smem + kMxScales;
#pragma unroll
            for (int i = 0; i < 2; ++i) dma4s(row_scales, row_scale[i] + at, dst + (2 * w + i) * 256);
#pragma unroll
            for (int i = 0; i < 4; ++i) dma4s(scale_base[GATE ? i >> 1 : 0], (col[i] >> 4) - chunk + at, dst + kMxRows * 16 + (4 * w + i) * 256);
        }
        char* dst = smem + image;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            dma16((const char*)row[i], dst + (2 * w + i) * 1024);
            row[i] += 64;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) dma16s(col_base[GATE ? i >> 1 : 0], col[i], dst + kMxRowImage + (4 * w + i) * 1024);
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
    __device__ __forceinline__ MxAddr(const Lane& ln, char* smem) {
        const uint32_t lds0 = lds_addr(smem);
        const int n = swap23(ln.l31);
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            b[kk] = lds0 + ln.l31 * 64 + (((2 * kk + ln.hf) ^ ((ln.l31 >> 2) & 3)) << 4);
            a[kk] = lds0 + kMxRowImage + (64 * ln.wn + n) * 64 + (((2 * kk + ln.hf) ^ ((n >> 2) & 3)) << 4);
        }
        sb = lds0 + kMxScales + ln.l31 * 16;
        sa = lds0 + kMxScales + (kMxRows + 64 * ln.wn + n) * 16;
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
template <int NTF, bool GATE>
__device__ __forceinline__ void mx_loop(MxLoader<GATE>& ld, int nk, char* smem, const MxAddr& ad, MxAcc& acc) {
#pragma unroll
    for (int t = 0; t < kMxImages; ++t)
        if (t < nk) ld.issue(smem, t * kMxStage);
    if (nk > 2) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * kMxRequests) : "memory");
    else if (nk > 1) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kMxRequests) : "memory");
    else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
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
        const uint32_t next = image == 2 * kMxStage ? 0 : image + kMxStage;
        wait_mx(f0);
        mx_step<NTF, 0, S>(f0, f1, ad.a[1] + image, ad.b[1] + image, s, acc);
        wait_mx(f1);
        if (t + 1 < nk) {
            if (t + 2 < nk) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(kMxRequests) : "memory");
            else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
            __builtin_amdgcn_s_barrier();
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
    __builtin_amdgcn_s_barrier();   // every wave has read its last fragments: the images may be refilled
}

// ---- what becomes of the accumulators
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
            const int row = rp.get_row(j);
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
            const int row = rp.get_row(j);
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
            const int row = rp.get_row(j);
            const u32x4_t v = rp.get(j);
            if (row < t.rows && col < p.N) store_stream16((uint16_t*)p.y + (size_t)(t.row0 + row) * p.N + col, v);
        }
        return;
    }
    // The wave's 32 columns are a block: 16 values in either half of the wave.  What is quantised is h as the bf16 result would be, so that both ways
    // to the next product give the same bits (a second rounding of 2^-8 before one of 2^-2).
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
        const int row = 32 * tf + ln.l31;
        if (row < t.rows) {
            const size_t at = (size_t)(t.row0 + row) * pitch + col0;
            *(u32x2_t*)(p.h_codes + at / 2 + 8 * ln.hf) = u32x2_t{c[0], c[1]};
            if (ln.hf == 0) p.h_scales[at / kMxBlock] = (uint8_t)byte;
        }
    }
}

template <bool GATE>
__global__ void __launch_bounds__(kMxThreads, 2) mx_product_kernel(MxParams p) {
    extern __shared__ __attribute__((aligned(16))) char smem[];
    const MxTiles tiles(p);
    const int xcd = blockIdx.x % kQueues, each = gridDim.x / kQueues;   // (the grid is a multiple of kQueues)
    const int lo = (int)((long long)tiles.total * xcd / kQueues), hi = (int)((long long)tiles.total * (xcd + 1) / kQueues);
    for (int i = lo + (int)(blockIdx.x / kQueues); i < hi; i += each) {
        const MxTile t = tiles.find(p, i);
        MxAcc acc;
#pragma unroll
        for (int tf = 0; tf < 4; ++tf)
#pragma unroll
            for (int af = 0; af < 2; ++af)
#pragma unroll
                for (int v = 0; v < 16; ++v) acc.a[tf][af][v] = 0.f;
        {
            const Lane ln;
            MxLoader<GATE> ld(p, ln, t);
            const MxAddr ad(ln, smem);
            const int ntf = (t.rows + 31) >> 5;
            if (ntf == 4) mx_loop<4, GATE>(ld, p.stages, smem, ad, acc);
            else if (ntf == 3) mx_loop<3, GATE>(ld, p.stages, smem, ad, acc);
            else if (ntf == 2) mx_loop<2, GATE>(ld, p.stages, smem, ad, acc);
            else mx_loop<1, GATE>(ld, p.stages, smem, ad, acc);
        }
        if (GATE) mx_store_h(p, t, acc, smem);
        else mx_store(p, t, acc, smem);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();   // the stores' LDS is read
    }
}

namespace {
// Workgroups that run at a time, asked once a device.
int mx_resident(bool gate, int* out) {
    static std::mutex lock;
    static int known[2][kMaxDevices] = {};
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= kMaxDevices) return MOE_ERR_HIP;
    std::lock_guard<std::mutex> guard(lock);
    int& n = known[gate][dev];
    if (n == 0) {
        const auto fn = gate ? mx_product_kernel<true> : mx_product_kernel<false>;
        int per_cu = 0, cus = 0;
        if (hipFuncSetAttribute((const void*)fn, hipFuncAttributeMaxDynamicSharedMemorySize, kMxSmem) != hipSuccess ||
            hipOccupancyMaxActiveBlocksPerMultiprocessor(&per_cu, fn, kMxThreads, kMxSmem) != hipSuccess ||
            hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || per_cu < 1)
            return MOE_ERR_HIP;
        n = (per_cu * cus + kQueues - 1) / kQueues * kQueues;
    }
    *out = n;
    return MOE_OK;
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
    p.a_rows = (uint32_t)a_rows, p.a_codes = a_codes, p.a_scales = a_scales, p.perm = perm, p.k = k;
    p.w_codes = w_codes, p.w_scales = w_scales, p.u_codes = u_codes, p.u_scales = u_scales;
    p.offsets = offsets, p.y = y, p.f32 = f32, p.h_codes = h_codes, p.h_scales = h_scales;
    int resident = 0;
    const int rc = mx_resident(gate, &resident);
    if (rc != MOE_OK) return rc;
    const int64_t most = ((int64_t)s.rows / kMxRows + (s.experts < s.rows ? s.experts : s.rows)) * p.col_tiles;
    const int grid = most < resident ? ((int)most + kQueues - 1) / kQueues * kQueues : resident;
    if (gate) hipLaunchKernelGGL((mx_product_kernel<true>), dim3(grid), dim3(kMxThreads), kMxSmem, st, p);
    else hipLaunchKernelGGL((mx_product_kernel<false>), dim3(grid), dim3(kMxThreads), kMxSmem, st, p);
    return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP;
}

}  // namespace uniep
