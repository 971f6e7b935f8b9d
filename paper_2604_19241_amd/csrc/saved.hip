// What the forward pass keeps for the backward pass, in 8 bits: G and U of every row in blocks of 32 that share an exponent (mx.hpp), from which
// h = silu(G) U is made again.  The stash's third part, the experts' outputs, is not read by the backward pass and not kept.
//
// 2.06 I bytes a row instead of the stash's 6 I + 2 d, so that the layers of a model can share one stash.  Both directions are copies that change the type:
// they are bound by memory, and what a lane computes for its 16 bytes hides behind it.  65536 rows of 768: packed in 48 us (6.4 TB/s of 305 MB), unpacked in 70 (5.8 TB/s of 406 MB).
//
// Eight bits of an integer, not of a floating-point number with three bits of mantissa: among 32 values of alike size the step of 2^-6 of the largest's
// power of two is closer for all but the smallest, whose errors weigh little (values from a normal distribution: 0.9 % of their norm, e4m3 with the same exponents 2.9 %).
#include "mma.hpp"
#include "mx.hpp"

namespace uniep {

struct SavedParams {
    int I;
    int experts;
    const int32_t* offsets;   // [experts + 1]: the last one is the number of rows
    uint32_t rows;            // that the stash holds
    uint16_t* gu;          // [rows][2 I]
    uint16_t* h;           // [rows][I]
    uint8_t* codes;           // [rows][2 I]
    uint8_t* scales;          // [rows][2 I / 32]
};
constexpr int kSavedThreads = 256;
constexpr int kSavedUnits = 4;   // of 8 values, a thread (65536 rows of 768 packed and unpacked: 2 118 us, 4 119, 8 124; 1542 of 1408 12.2, 12.1, 12.9)

__device__ __forceinline__ uint32_t saved_rows(const SavedParams& p) { return (uint32_t)min((int64_t)max(p.offsets[p.experts], 0), (int64_t)p.rows); }

__global__ void __launch_bounds__(kSavedThreads) saved_pack_kernel(SavedParams p) {
    // four lanes a block: 8 values each.  G and U of all rows are one run of blocks
    const size_t units = (size_t)saved_rows(p) * (p.I / 4), first = (size_t)blockIdx.x * (kSavedThreads * kSavedUnits) + threadIdx.x;
    if (first - threadIdx.x >= units) return;
    u32x4_t u[kSavedUnits];
#pragma unroll
    for (int i = 0; i < kSavedUnits; ++i) {
        const size_t at = first + i * kSavedThreads;
        u[i] = u32x4_t{0u, 0u, 0u, 0u};
        if (at < units) u[i] = __builtin_nontemporal_load((const u32x4_t*)p.gu + at);
    }
#pragma unroll
    for (int i = 0; i < kSavedUnits; ++i) {
        const size_t at = first + i * kSavedThreads;
        float v[8];
        uint32_t m = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v[2 * j] = bf16_lo(u[i][j]);
            v[2 * j + 1] = bf16_hi(u[i][j]);
            m = max(m, max(mag(v[2 * j]), mag(v[2 * j + 1])));
        }
        const uint32_t byte = mx8_byte(max_quad(m));
        u32x2_t c = {0u, 0u};
        if (byte != kMxNan)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int q = (int)fminf(fmaxf(rintf(__builtin_amdgcn_ldexpf(v[j], 6 + 127 - (int)byte)), -127.f), 127.f);
                c[j >> 2] |= (uint32_t)(q & 0xff) << (8 * (j & 3));
            }
        if (at < units) {
            __builtin_nontemporal_store(c, (u32x2_t*)p.codes + at);
            if ((threadIdx.x & 3) == 0) p.scales[at >> 2] = (uint8_t)byte;
        }
    }
}

__device__ __forceinline__ void mx8_values(float (&v)[8], u32x2_t codes, uint32_t byte) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float q = (float)(int8_t)(codes[j >> 2] >> (8 * (j & 3)));
        v[j] = byte == kMxNan ? __uint_as_float(0x7fc00000u) : __builtin_amdgcn_ldexpf(q, (int)byte - 127 - 6);
    }
}
__device__ __forceinline__ u32x4_t packed8(const float (&v)[8]) {
    return u32x4_t{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
}

__global__ void __launch_bounds__(kSavedThreads) saved_unpack_kernel(SavedParams p) {
    const uint32_t per = p.I / 8;   // units of a row's G, and of its U
    const size_t units = (size_t)saved_rows(p) * per, first = (size_t)blockIdx.x * (kSavedThreads * kSavedUnits) + threadIdx.x;
    if (first - threadIdx.x >= units) return;
    u32x2_t c[kSavedUnits][2];
    uint32_t s[kSavedUnits][2];
    size_t at[kSavedUnits];   // G's unit; U's is `per` on
    // rows by one division, and from one unit to the next by what the threads are apart (a division of 64 bits takes as long as the loads)
    size_t row = first >> 32 ? first / per : (uint32_t)first / per;
    uint32_t in = (uint32_t)(first - row * per);
    const uint32_t step_rows = kSavedThreads / per, step_in = kSavedThreads - step_rows * per;
#pragma unroll
    for (int i = 0; i < kSavedUnits; ++i) {
        at[i] = first + i * kSavedThreads < units ? row * 2 * per + in : 0;
        row += step_rows;
        in += step_in;
        if (in >= per) {
            in -= per;
            ++row;
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            c[i][j] = __builtin_nontemporal_load((const u32x2_t*)p.codes + at[i] + j * per);
            s[i][j] = p.scales[(at[i] + j * per) >> 2];
        }
    }
#pragma unroll
    for (int i = 0; i < kSavedUnits; ++i) {
        if (first + i * kSavedThreads >= units) break;
        float g[8], u[8], h[8];
        mx8_values(g, c[i][0], s[i][0]);
        mx8_values(u, c[i][1], s[i][1]);
#pragma unroll
        for (int j = 0; j < 8; ++j) h[j] = g[j] * sigmoid_f(g[j]) * u[j];
        store_stream16((u32x4_t*)p.gu + at[i], packed8(g));
        store_stream16((u32x4_t*)p.gu + at[i] + per, packed8(u));
        store_stream16((u32x4_t*)p.h + first + i * kSavedThreads, packed8(h));
    }
}

namespace {
template <class K>
int saved_launch(K kernel, const moe_shape_t& s, const int32_t* offsets, size_t units, char* gu, char* h, uint8_t* codes, uint8_t* scales, hipStream_t st) {
    if (units == 0) return MOE_OK;
    SavedParams p = {s.I, s.e_count, offsets, (uint32_t)((size_t)s.T * s.k), (uint16_t*)gu, (uint16_t*)h, codes, scales};
    const size_t each = kSavedThreads * kSavedUnits;
    hipLaunchKernelGGL(kernel, dim3((unsigned)((units + each - 1) / each)), dim3(kSavedThreads), 0, st, p);
    return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP;
}
}  // namespace

int saved_pack_launch(const moe_shape_t& s, const int32_t* offsets, const char* gu, uint8_t* codes, uint8_t* scales, hipStream_t st) {
    return saved_launch(saved_pack_kernel, s, offsets, (size_t)s.T * s.k * (s.I / 4), (char*)gu, nullptr, codes, scales, st);
}
int saved_unpack_launch(const moe_shape_t& s, const int32_t* offsets, const uint8_t* codes, const uint8_t* scales, char* gu, char* h, hipStream_t st) {
    return saved_launch(saved_unpack_kernel, s, offsets, (size_t)s.T * s.k * (s.I / 8), gu, h, (uint8_t*)codes, (uint8_t*)scales, st);
}

}  // namespace uniep
