// Tokens copied to the rows of their experts, rows added up for their tokens with the gates' weights, and the gradients of both.
//
// With row(t, j) the row of slot j of token t (moe_route's inv_perm, or any table in which every row stands once at most):
//   dispatch   xs[row(t, j)] = x[t]                     dx[t] = sum_j dxs[row(t, j)]
//   combine    y[t] = sum_j w[t][j] o[row(t, j)]        do[row(t, j)] = w[t][j] dy[t],   dw[t][j] = sum_c dy[t][c] o[row(t, j)][c]
// Slots whose row is outside the buffer have none: nothing is read or written for them.  dx is y with weights of one.  Every wave has a token's run of columns, so two slots that name
// one row leave some of its columns from either token.
//
// Nothing is computed that memory could wait for: every token's side is read or written once (by combine's gradients once for eight slots), by the lanes that have all of its rows, so the k copies of a
// token come from registers and its sum needs no pass over a sorted buffer.  Sums are fp32 in the order of the slots (dw: lanes, then waves), rounded once.
// bf16, 8192 tokens of 2048 with 8 rows each: dispatch 57 us (5.3 TB/s of 302 MB), its gradient 52 (5.9).  fp32, 4099 tokens of 2304 with two rows here on average: combine 21 us (5.5),
// its gradients 36 (5.3).  A large copy: 5.3.  One token: 2.5 us, the launch and two loads in a row.
#include "common.hpp"

namespace uniep {

constexpr int kMoveSlots = 8;   // requested at a time (4: 61 us for 4099 tokens of 2304 fp32, with the gradients, 8: 55)

struct MoveParams {
    int T, k, d;
    int rows;
    const void* token;        // [T][ld]   x, dy
    size_t ld;
    const void* sorted;       // [rows][d] dxs, o
    const int32_t* row_of;    // [T][k]
    const float* w;           // [T][k] or NULL (ones)
    void* out;                // dispatch, do: [rows][d];  dx, y: [T][d]
    float* dw;                // [T][k] or NULL
};

// 16 bytes of either type as fp32.
template <bool F32>
struct Piece {
    static constexpr int kN = F32 ? 4 : 8;
    float v[kN];
    __device__ __forceinline__ explicit Piece(u32x4_t u) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (F32) {
                v[i] = __uint_as_float(u[i]);
            } else {
                v[2 * i] = bf16_lo(u[i]);
                v[2 * i + 1] = bf16_hi(u[i]);
            }
        }
    }
    __device__ __forceinline__ u32x4_t packed() const {
        u32x4_t u;
#pragma unroll
        for (int i = 0; i < 4; ++i) u[i] = F32 ? __float_as_uint(v[i]) : pack_bf16x2(v[2 * i], v[2 * i + 1]);
        return u;
    }
};
template <bool F32>
__device__ __forceinline__ const u32x4_t* piece_at(const void* p, size_t row, size_t ld, int c) {
    return (const u32x4_t*)((const char*)p + (row * ld + c) * (F32 ? 4 : 2));
}

// The wave's token and first column.  V pieces of 16 bytes a lane: the wave has 64 V of them.
template <bool F32, int V>
struct MoveWork {
    static constexpr int kCols = 64 * V * Piece<F32>::kN;
    uint32_t t;
    int c;
    __device__ __forceinline__ MoveWork(const MoveParams& p, uint32_t first) {
        const uint32_t parts = (p.d + kCols - 1) / kCols, id = first + rfl((int)blockIdx.x * kTailWaves + (int)(threadIdx.x >> 6));
        t = id / parts;
        c = (int)(id - t * parts) * kCols + (int)(threadIdx.x & 63) * Piece<F32>::kN;
    }
    __device__ __forceinline__ int col(int i) const { return c + i * 64 * Piece<F32>::kN; }
};

// A token's rows and weights: a lane has a slot, so that they take one request each.
struct Slots {
    int rows;
    float weights;
    __device__ __forceinline__ Slots(const MoveParams& p, size_t t) {
        const int lane = threadIdx.x & 63;
        rows = lane < p.k ? p.row_of[t * p.k + lane] : -1;
        weights = lane < p.k && p.w ? p.w[t * p.k + lane] : 1.f;
    }
    __device__ __forceinline__ int row(int j) const { return __builtin_amdgcn_readlane(rows, j); }
    __device__ __forceinline__ float weight(int j) const { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(weights), j)); }
};

template <bool F32, int V>
__global__ void __launch_bounds__(64 * kTailWaves) dispatch_kernel(MoveParams p, uint32_t first) {
    const MoveWork<F32, V> m(p, first);
    if (m.t >= (uint32_t)p.T) return;
    u32x4_t x[V];
#pragma unroll
    for (int i = 0; i < V; ++i)
        if (m.col(i) < p.d) x[i] = __builtin_nontemporal_load(piece_at<F32>(p.token, m.t, p.ld, m.col(i)));
    const Slots slots(p, m.t);
    for (int j = 0; j < p.k; ++j) {
        const int r = slots.row(j);
        if ((unsigned)r >= (unsigned)p.rows) continue;
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (m.col(i) < p.d) store_stream16((void*)piece_at<F32>(p.out, r, p.d, m.col(i)), x[i]);
    }
}

template <bool F32, int V, bool WEIGHTED>
__global__ void __launch_bounds__(64 * kTailWaves) combine_kernel(MoveParams p, uint32_t first) {
    const MoveWork<F32, V> m(p, first);
    if (m.t >= (uint32_t)p.T) return;
    const Slots slots(p, m.t);
    float sum[V][Piece<F32>::kN] = {};
    for (int j0 = 0; j0 < p.k; j0 += kMoveSlots) {
        u32x4_t o[kMoveSlots][V];
        int r[kMoveSlots];
#pragma unroll
        for (int j = 0; j < kMoveSlots; ++j) r[j] = slots.row(j0 + j);
#pragma unroll
        for (int j = 0; j < kMoveSlots; ++j)
#pragma unroll
            for (int i = 0; i < V; ++i)
                if ((unsigned)r[j] < (unsigned)p.rows && m.col(i) < p.d)
                    o[j][i] = __builtin_nontemporal_load(piece_at<F32>(p.sorted, r[j], p.d, m.col(i)));
#pragma unroll
        for (int j = 0; j < kMoveSlots; ++j) {
            if ((unsigned)r[j] >= (unsigned)p.rows) continue;
            const float w = slots.weight(j0 + j);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const Piece<F32> v(o[j][i]);
#pragma unroll
                for (int e = 0; e < Piece<F32>::kN; ++e) sum[i][e] = WEIGHTED ? fmaf(w, v.v[e], sum[i][e]) : sum[i][e] + v.v[e];
            }
        }
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
        if (m.col(i) >= p.d) continue;
        Piece<F32> y(u32x4_t{0u, 0u, 0u, 0u});
#pragma unroll
        for (int e = 0; e < Piece<F32>::kN; ++e) y.v[e] = sum[i][e];
        store_stream16((void*)piece_at<F32>(p.out, m.t, p.d, m.col(i)), y.packed());
    }
}

// do and dw: a workgroup a token, as dw is a sum over all of its columns.  dy is read once for eight slots and stays in registers between the rows' products and their stores.
// Narrow rows leave threads, or whole waves, without columns, and a token costs its workgroup and its sums all the same.  us, 65536 tokens in bf16, 2 / 8 / 16 rows each: 64 columns 90 / 119 / 213 (combine
// itself 18 / 32 / 51), 256 98 / 141 / 249, 512 109 / 214 / 429, 1024 130 / 430 / 855, 2048 220 / 872 / 1727 (5.1 to 6.1 TB/s).
template <bool F32>
__global__ void __launch_bounds__(64 * kTailWaves) combine_backward_kernel(MoveParams p, uint32_t first) {
    using P = Piece<F32>;
    __shared__ float parts[kTailWaves][kMaxTopK];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const size_t t = first + blockIdx.x;
    const Slots slots(p, t);
    for (int j0 = 0; j0 < p.k; j0 += kMoveSlots) {
        int r[kMoveSlots];
        float w[kMoveSlots], dot[kMoveSlots] = {};
#pragma unroll
        for (int j = 0; j < kMoveSlots; ++j) {
            r[j] = slots.row(j0 + j);
            w[j] = slots.weight(j0 + j);
        }
        for (int c = (int)threadIdx.x * P::kN; c < p.d; c += 64 * kTailWaves * P::kN) {
            const P g(*piece_at<F32>(p.token, t, p.ld, c));
            u32x4_t o[kMoveSlots];
            if (p.dw)
#pragma unroll
                for (int j = 0; j < kMoveSlots; ++j)
                    if ((unsigned)r[j] < (unsigned)p.rows) o[j] = __builtin_nontemporal_load(piece_at<F32>(p.sorted, r[j], p.d, c));
#pragma unroll
            for (int j = 0; j < kMoveSlots; ++j) {
                if ((unsigned)r[j] >= (unsigned)p.rows) continue;
                P d = g;
#pragma unroll
                for (int e = 0; e < P::kN; ++e) d.v[e] *= w[j];
                store_stream16((void*)piece_at<F32>(p.out, r[j], p.d, c), d.packed());
                if (p.dw) {
                    const P v(o[j]);
#pragma unroll
                    for (int e = 0; e < P::kN; ++e) dot[j] = fmaf(g.v[e], v.v[e], dot[j]);
                }
            }
        }
        if (p.dw)
#pragma unroll
            for (int j = 0; j < kMoveSlots; ++j) {
                const float s = wave_sum(dot[j]);
                if (lane == 0) parts[wave][j0 + j] = s;
            }
    }
    if (!p.dw) return;
    __syncthreads();
    if ((int)threadIdx.x < p.k) {
        float s = parts[0][threadIdx.x];
#pragma unroll
        for (int i = 1; i < kTailWaves; ++i) s += parts[i][threadIdx.x];
        p.dw[t * p.k + threadIdx.x] = s;
    }
}

namespace {
MoveParams move_params(const moe_dispatch_shape_t& s, const int32_t* row_of) {
    MoveParams p = {};
    p.T = s.T, p.k = s.k, p.d = s.d, p.rows = s.rows;
    p.row_of = row_of;
    return p;
}
int launched() { return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP; }
template <class F>
void waves_of(const MoveParams& p, int cols, F launch) {
    launch_tail_waves((size_t)p.T * ((p.d + cols - 1) / cols), launch);
}
template <bool F32>
void dispatch(const MoveParams& p, hipStream_t st) {
    constexpr int V = 4;   // (one of 16 bytes a lane, two: 113.8 us for 8192 tokens of 2048 to 8 rows each and back, four 109.7; 256 tokens the same)
    waves_of(p, MoveWork<F32, V>::kCols, [&](dim3 grid, uint32_t first) {
        hipLaunchKernelGGL((dispatch_kernel<F32, V>), grid, dim3(64 * kTailWaves), 0, st, p, first);
    });
}
template <bool F32, bool WEIGHTED>
void combine(const MoveParams& p, hipStream_t st) {
    constexpr int V = 1;   // (two: the same for large batches, a token of 2048 columns on half as many waves)
    waves_of(p, MoveWork<F32, V>::kCols, [&](dim3 grid, uint32_t first) {
        hipLaunchKernelGGL((combine_kernel<F32, V, WEIGHTED>), grid, dim3(64 * kTailWaves), 0, st, p, first);
    });
}
}  // namespace

int dispatch_forward_launch(const moe_dispatch_shape_t& s, const void* x, size_t ldx, int f32, const int32_t* row_of, void* xs, hipStream_t st) {
    if (s.T == 0 || s.rows == 0) return MOE_OK;
    MoveParams p = move_params(s, row_of);
    p.token = x, p.ld = ldx, p.out = xs;
    f32 ? dispatch<true>(p, st) : dispatch<false>(p, st);
    return launched();
}

int combine_forward_launch(const moe_dispatch_shape_t& s, const void* o, int f32, const int32_t* row_of, const float* w, void* y, hipStream_t st) {
    if (s.T == 0) return MOE_OK;
    MoveParams p = move_params(s, row_of);
    p.sorted = o, p.w = w, p.out = y;
    if (w) f32 ? combine<true, true>(p, st) : combine<false, true>(p, st);
    else f32 ? combine<true, false>(p, st) : combine<false, false>(p, st);
    return launched();
}

int combine_backward_launch(const moe_dispatch_shape_t& s, const void* dy, size_t lddy, const void* o, int f32, const int32_t* row_of, const float* w,
                            void* d_o, float* dw, hipStream_t st) {
    if (s.T == 0) return MOE_OK;
    MoveParams p = move_params(s, row_of);
    p.token = dy, p.ld = lddy, p.sorted = o, p.w = w, p.out = d_o, p.dw = dw;
    for (size_t t = 0; t < (size_t)s.T; t += kTailGroups) {
        const dim3 grid((unsigned)(s.T - t < kTailGroups ? s.T - t : kTailGroups));
        if (f32) hipLaunchKernelGGL((combine_backward_kernel<true>), grid, dim3(64 * kTailWaves), 0, st, p, (uint32_t)t);
        else hipLaunchKernelGGL((combine_backward_kernel<false>), grid, dim3(64 * kTailWaves), 0, st, p, (uint32_t)t);
    }
    return launched();
}

}  // namespace uniep
