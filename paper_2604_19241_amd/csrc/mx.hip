// Microscaled 4-bit floating point (mx.hpp): activations and weights into it and back.
//
// Codes lie two to a byte, the first in the lower half, K' / 2 bytes a row with K' = K filled up to a multiple of 128 by zeros; exponents K' / 32 bytes a row.
// Both directions are copies that change the type, bound by memory: 8191 rows of 7168 in 27 us (5.5 TB/s of 149 MB) and back in 24, 32 weights of 2048 x 1408 in 42 us (5.6 TB/s of 234 MB) and
// back in 39.
#include "mx.hpp"

namespace uniep {

constexpr int kQuantThreads = 64 * kTailWaves;
constexpr int kQuantUnits = 2;              // of 8 values, a lane: 1024 values a wave (8191 rows of 7168 there and back: 1 54 us, 2 51, 4 54)
constexpr int kQuantCols = 64 * 8 * kQuantUnits;

struct QuantParams {
    const void* x;     // [rows][ld]
    size_t ld;
    uint32_t rows;
    int K;
    uint8_t* codes;    // [rows][K' / 2]
    uint8_t* scales;   // [rows][K' / 32]
};

// Eight values of either type.
template <bool F32>
__device__ __forceinline__ void load8(float (&v)[8], const void* p, size_t at) {
    if (F32) {
        const u32x4_t a = __builtin_nontemporal_load((const u32x4_t*)((const float*)p + at)), b = __builtin_nontemporal_load((const u32x4_t*)((const float*)p + at) + 1);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(a[i]), v[4 + i] = __uint_as_float(b[i]);
    } else {
        const u32x4_t a = __builtin_nontemporal_load((const u32x4_t*)((const uint16_t*)p + at));
#pragma unroll
        for (int i = 0; i < 4; ++i) v[2 * i] = bf16_lo(a[i]), v[2 * i + 1] = bf16_hi(a[i]);
    }
}
__device__ __forceinline__ uint32_t mag8(const float (&v)[8]) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, mag(v[i]));
    return m;
}

// Four lanes a block, 8 values each; a wave a run of columns of one row.
template <bool F32>
__global__ void __launch_bounds__(kQuantThreads) mx_quantize_kernel(QuantParams p, uint32_t first) {
    const uint32_t Kp = mx_padded(p.K), parts = (Kp + kQuantCols - 1) / kQuantCols, id = first + rfl((int)blockIdx.x * kTailWaves + (int)(threadIdx.x >> 6));
    const uint32_t row = id / parts, c0 = (id - row * parts) * kQuantCols + (threadIdx.x & 63) * 8;
    if (row >= p.rows) return;
    float v[kQuantUnits][8] = {};
#pragma unroll
    for (int i = 0; i < kQuantUnits; ++i)
        if (c0 + 512 * i < (uint32_t)p.K) load8<F32>(v[i], p.x, row * p.ld + c0 + 512 * i);
#pragma unroll
    for (int i = 0; i < kQuantUnits; ++i) {
        const uint32_t c = c0 + 512 * i;
        const uint32_t byte = mx4_byte(max_quad(mag8(v[i])));
        if (c >= Kp) continue;   // (whole blocks: Kp is a multiple of 128)
        const size_t at = (size_t)row * Kp + c;
        *(uint32_t*)(p.codes + at / 2) = mx4_codes(v[i], byte);
        if ((threadIdx.x & 3) == 0) p.scales[at / kMxBlock] = (uint8_t)byte;
    }
}

// And back, to bf16 (exact) or fp32.
template <bool F32>
__global__ void __launch_bounds__(kQuantThreads) mx_values_kernel(QuantParams p, uint32_t first) {
    const uint32_t Kp = mx_padded(p.K), parts = (p.K + kQuantCols - 1) / kQuantCols, id = first + rfl((int)blockIdx.x * kTailWaves + (int)(threadIdx.x >> 6));
    const uint32_t row = id / parts, c0 = (id - row * parts) * kQuantCols + (threadIdx.x & 63) * 8;
    if (row >= p.rows) return;
    uint32_t codes[kQuantUnits], bytes[kQuantUnits];
#pragma unroll
    for (int i = 0; i < kQuantUnits; ++i) {
        const size_t at = (size_t)row * Kp + min(c0 + 512 * i, Kp - 8);
        codes[i] = __builtin_nontemporal_load((const uint32_t*)(p.codes + at / 2));
        bytes[i] = p.scales[at / kMxBlock];
    }
#pragma unroll
    for (int i = 0; i < kQuantUnits; ++i) {
        if (c0 + 512 * i >= (uint32_t)p.K) continue;
        const size_t at = (size_t)row * p.ld + c0 + 512 * i;
        float v[8];
        mx4_values(v, codes[i], bytes[i]);
        if (F32) {
            store_stream16((float*)p.x + at, u32x4_t{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])});
            store_stream16((float*)p.x + at + 4, u32x4_t{__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7])});
        } else {
            store_stream16((uint16_t*)p.x + at, u32x4_t{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])});
        }
    }
}

// Weights [K][N] of every expert to codes [N][K']: blocks run along K, the memory rows.  A workgroup has 256 k of 128 columns: a lane 8 k of 8 columns (the 16 bytes of
// 8 loads), a quad of lanes a block of 8 columns, a wave 32 k at a time.  The codes change their order in LDS, so that a column's 128 bytes leave as one line; straight from the
// registers they would be pieces of 16 bytes in 128 lines.
constexpr int kWqK = 256, kWqN = 128;
constexpr int kWqPitch = kWqK / 2 + 16;   // of a column's codes: pieces of neighbouring columns in different banks
struct WeightParams {
    const uint16_t* w;   // [experts][K][N] bf16
    int K, N;
    uint8_t* codes;      // [experts][N][K' / 2]
    uint8_t* scales;     // [experts][N][K' / 32]
};
__global__ void __launch_bounds__(256) mx_quantize_weights_kernel(WeightParams p) {
    __shared__ __attribute__((aligned(16))) uint8_t s_codes[kWqN * kWqPitch];
    __shared__ __attribute__((aligned(8))) uint8_t s_scales[kWqN * (kWqK / kMxBlock)];
    const int Kp = mx_padded(p.K), tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int tiles_n = (p.N + kWqN - 1) / kWqN;
    const size_t expert = blockIdx.y;
    const int k0 = (int)(blockIdx.x / tiles_n) * kWqK, n0 = (int)(blockIdx.x % tiles_n) * kWqN;
    const int cols = lane >> 2, quad = lane & 3;   // columns 8 cols .. + 7, k 8 quad .. + 7 of the block
    const uint16_t* w = p.w + expert * p.K * p.N + n0 + 8 * cols;
#pragma unroll
    for (int b = 0; b < 2; ++b) {
        const int block = 4 * b + wave, k = k0 + kMxBlock * block + 8 * quad;
        u32x4_t u[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            u[i] = u32x4_t{0u, 0u, 0u, 0u};
            if (k + i < p.K && n0 + 8 * cols < p.N) u[i] = __builtin_nontemporal_load((const u32x4_t*)(w + (size_t)(k + i) * p.N));
        }
#pragma unroll
        for (int c = 0; c < 8; ++c) {
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = c & 1 ? bf16_hi(u[i][c >> 1]) : bf16_lo(u[i][c >> 1]);
            const uint32_t byte = mx4_byte(max_quad(mag8(v)));
            const int col = 8 * cols + c;
            *(uint32_t*)(s_codes + col * kWqPitch + block * 16 + quad * 4) = mx4_codes(v, byte);
            if (quad == 0) s_scales[col * (kWqK / kMxBlock) + block] = (uint8_t)byte;
        }
    }
    __syncthreads();
    const int bytes = min(kWqK, Kp - k0) / 2;   // of a column: 64 or 128
#pragma unroll
    for (int i = 0; i < kWqN * 8 / 256; ++i) {
        const int col = (tid >> 3) + 32 * i, at = (tid & 7) * 16;
        if (n0 + col < p.N && at < bytes)
            store_stream16(p.codes + ((expert * p.N + n0 + col) * (size_t)Kp + k0) / 2 + at, *(const u32x4_t*)(s_codes + col * kWqPitch + at));
    }
    const int col = tid >> 1, at = (tid & 1) * 4;
    if (n0 + col < p.N && at * 16 < bytes)
        *(uint32_t*)(p.scales + ((expert * p.N + n0 + col) * (size_t)Kp + k0) / kMxBlock + at) = *(const uint32_t*)(s_scales + col * (kWqK / kMxBlock) + at);
}

int mx_quantize_launch(const void* x, size_t ldx, int f32, int64_t rows, int K, uint8_t* codes, uint8_t* scales, hipStream_t st) {
    if (rows == 0) return MOE_OK;
    const QuantParams p = {x, ldx, (uint32_t)rows, K, codes, scales};
    launch_tail_waves((size_t)rows * ((mx_padded(K) + kQuantCols - 1) / kQuantCols), [&](dim3 grid, uint32_t first) {
        if (f32) hipLaunchKernelGGL((mx_quantize_kernel<true>), grid, dim3(kQuantThreads), 0, st, p, first);
        else hipLaunchKernelGGL((mx_quantize_kernel<false>), grid, dim3(kQuantThreads), 0, st, p, first);
    });
    return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP;
}

int mx_values_launch(const uint8_t* codes, const uint8_t* scales, int64_t rows, int K, void* out, int f32, hipStream_t st) {
    if (rows == 0) return MOE_OK;
    const QuantParams p = {out, (size_t)K, (uint32_t)rows, K, (uint8_t*)codes, (uint8_t*)scales};
    launch_tail_waves((size_t)rows * ((K + kQuantCols - 1) / kQuantCols), [&](dim3 grid, uint32_t first) {
        if (f32) hipLaunchKernelGGL((mx_values_kernel<true>), grid, dim3(kQuantThreads), 0, st, p, first);
        else hipLaunchKernelGGL((mx_values_kernel<false>), grid, dim3(kQuantThreads), 0, st, p, first);
    });
    return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP;
}

int mx_quantize_weights_launch(const void* w, int experts, int K, int N, uint8_t* codes, uint8_t* scales, hipStream_t st) {
    const WeightParams p = {(const uint16_t*)w, K, N, codes, scales};
    const unsigned tiles = (unsigned)((mx_padded(K) + kWqK - 1) / kWqK) * (unsigned)((N + kWqN - 1) / kWqN);
    hipLaunchKernelGGL(mx_quantize_weights_kernel, dim3(tiles, experts), dim3(256), 0, st, p);
    return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP;
}

}  // namespace uniep
