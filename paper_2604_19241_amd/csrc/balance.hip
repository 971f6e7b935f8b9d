// The router's balance loss and z loss with the count of every expert, and the gradient of the logits.
//
// Over the kept tokens t of sequence s, p[t] = softmax(logits[t]):
//   P[s][e] = sum_t p[t][e]       c[s][e] = slots of these tokens with expert e       f[s][e] = c[s][e] / (k tokens[s])
//   balance = E / n sum_s sum_e f[s][e] P[s][e]          z = 1 / n sum_t lse[t]^2          n = all kept tokens
//   loss = balance_coef balance + z_coef z
// With u the gradient of the loss, counts being constants,
//   dlogits[t][e] = p[t][e] (u balance_coef E / n (f[s][e] - sum_j f[s][j] p[t][j]) + u z_coef 2 / n lse[t])
// for kept tokens, plus w_i (dw_i - sum_j w_j dw_j) at the expert of slot i for every token, where the gates' gradients are given.
//
// Both directions read the logits once and are bound by that: a token's logits stay in the registers of the lanes that share it.
// Sums over tokens are made in a fixed order (lanes, waves, chunks of tokens), so every run gives the same bits.
#include "common.hpp"

#include <type_traits>

namespace uniep {

constexpr int kBalThreads = 256;
constexpr int kBalWaves = kBalThreads / kWave;

struct BalParams {
    int T, E, k, S, chunk, chunks;
    float balance_coef, z_coef;
    const float* logits;
    const int32_t* idx;       // [T][k]
    const int32_t* offsets;   // [S + 1] or NULL (one sequence)
    const uint8_t* mask;      // [T] or NULL
    // forward
    float* loss;              // [3]
    int32_t* counts;          // [S][E]
    int32_t* tokens;          // [S + 1]
    float* prob_sums;         // [S][E]
    float* lse;               // [T]
    // parts: of the tokens of chunk c that sequence s has, at slot c + s (from one part to the next c or s grows, so no two share a slot)
    float* part_p;            // [slots][E]
    int32_t* part_c;          // [slots][E]
    float* part_z;            // [slots]
    int32_t* part_n;          // [slots]
    double* sum_b;            // [S][blocks of experts]
    double* sum_z;            // [S]
    int32_t* ticket;
    // backward
    const float* w;
    const float* dw;
    const float* dloss;
    void* dlogits;
    int out_bf16;
};

__device__ __forceinline__ int seq_begin(const BalParams& p, int s) { return p.offsets ? min(max(p.offsets[s], 0), p.T) : s > 0 ? p.T : 0; }
// last sequence that begins at or before token t
__device__ __forceinline__ int seq_of(const BalParams& p, int t) {
    if (!p.offsets) return 0;
    int lo = 0, hi = p.S - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (p.offsets[mid] <= t) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

// G lanes share a token, each with 4 NV of its experts: runs of 4 where rows are 16-byte aligned, else every G-th.
template <int G, int NV, bool VEC>
struct TokenLanes {
    static constexpr int kValues = 4 * NV;
    int g;
    __device__ __forceinline__ explicit TokenLanes(int lane) : g(lane % G) {}
    __device__ __forceinline__ int expert(int v) const { return VEC ? 4 * (G * (v >> 2) + g) + (v & 3) : G * v + g; }
    // experts past the last: `rest`
    template <class T4, class T1>
    __device__ __forceinline__ void load(const T1* row, int E, T1 rest, T1 (&x)[kValues]) const {
        if (VEC) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int e = 4 * (G * i + g);
                if (e < E) {
                    const T4 u = *(const T4*)(row + e);
#pragma unroll
                    for (int c = 0; c < 4; ++c) x[4 * i + c] = u[c];
                } else {
#pragma unroll
                    for (int c = 0; c < 4; ++c) x[4 * i + c] = rest;
                }
            }
        } else {
#pragma unroll
            for (int v = 0; v < kValues; ++v) {
                const int e = G * v + g;
                x[v] = e < E ? row[e] : rest;
            }
        }
    }
    static __device__ __forceinline__ float sum(float v) {
#pragma unroll
        for (int o = G / 2; o > 0; o >>= 1) v += __shfl_xor(v, o);
        return v;
    }
    static __device__ __forceinline__ float most(float v) {
#pragma unroll
        for (int o = G / 2; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
        return v;
    }
};
typedef __attribute__((ext_vector_type(4))) int32_t i32x4_t;

template <int G, int NV, bool VEC>
__global__ void __launch_bounds__(kBalThreads) balance_forward_kernel(BalParams p) {
    using L = TokenLanes<G, NV, VEC>;
    constexpr int kMost = 4 * G * NV, kGroups = 64 / G;
    __shared__ float s_p[kBalWaves][kMost];
    __shared__ int32_t s_c[kMost];
    __shared__ float s_z[kBalWaves];
    __shared__ int32_t s_n[kBalWaves];
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, E = p.E;
    const L ln(lane);
    const int c = blockIdx.x, c0 = c * p.chunk, c1 = min(p.T, c0 + p.chunk);
    if (c == 0 && tid == 0) *p.ticket = 0;
    for (int s = seq_of(p, c0); s < p.S; ++s) {
        const int from = seq_begin(p, s);
        if (from >= c1) break;
        const int a = max(from, c0), b = min(seq_begin(p, s + 1), c1);
        if (a >= b) continue;
        for (int e = tid; e < E; e += kBalThreads) s_c[e] = 0;
        __syncthreads();
        for (int i = tid; i < (b - a) * p.k; i += kBalThreads) {
            const int t = a + i / p.k, e = p.idx[(size_t)a * p.k + i];
            if ((unsigned)e < (unsigned)E && (!p.mask || p.mask[t])) atomicAdd(&s_c[e], 1);
        }
        float sums[L::kValues] = {}, z = 0.f;
        int n = 0;
        for (int t = a + w * kGroups + lane / G; t < b; t += kBalWaves * kGroups) {
            const bool keep = !p.mask || p.mask[t];
            float m = -INFINITY, total = 1.f, x[L::kValues];
            if (keep) {
                ln.template load<f32x4_t>(p.logits + (size_t)t * E, E, -INFINITY, x);
#pragma unroll
                for (int v = 0; v < L::kValues; ++v) m = fmaxf(m, x[v]);
                m = L::most(m);
                float q = 0.f;
#pragma unroll
                for (int v = 0; v < L::kValues; ++v) {
                    x[v] = ln.expert(v) < E ? __expf(x[v] - m) : 0.f;
                    q += x[v];
                }
                total = L::sum(q);
                const float inv = 1.f / total;
#pragma unroll
                for (int v = 0; v < L::kValues; ++v) sums[v] += x[v] * inv;
            }
            const float lse = keep ? m + logf(total) : -INFINITY;
            if (ln.g == 0) {
                p.lse[t] = lse;
                if (keep) {
                    z += lse * lse;
                    ++n;
                }
            }
        }
        // the groups of a wave, then the waves
#pragma unroll
        for (int o = G; o < 64; o <<= 1) {
#pragma unroll
            for (int v = 0; v < L::kValues; ++v) sums[v] += __shfl_xor(sums[v], o);
            z += __shfl_xor(z, o);
            n += __shfl_xor(n, o);
        }
        if (lane < G) {
#pragma unroll
            for (int v = 0; v < L::kValues; ++v) s_p[w][ln.expert(v)] = sums[v];
            if (lane == 0) {
                s_z[w] = z;
                s_n[w] = n;
            }
        }
        __syncthreads();
        const size_t slot = (size_t)c + s;
        for (int e = tid; e < E; e += kBalThreads) {
            p.part_p[slot * E + e] = ((s_p[0][e] + s_p[1][e]) + s_p[2][e]) + s_p[3][e];
            p.part_c[slot * E + e] = s_c[e];
        }
        if (tid == 0) {
            p.part_z[slot] = ((s_z[0] + s_z[1]) + s_z[2]) + s_z[3];
            p.part_n[slot] = s_n[0] + s_n[1] + s_n[2] + s_n[3];
        }
        __syncthreads();
    }
}

// Sums the parts of one sequence and 32 experts; the workgroup that is last to end adds up the losses.
constexpr int kSumThreads = 1024, kSumExperts = 32, kSumGroups = kSumThreads / kSumExperts;
__global__ void __launch_bounds__(kSumThreads) balance_sum_kernel(BalParams p) {
    __shared__ float s_p[kSumGroups][kSumExperts];
    __shared__ int32_t s_c[kSumGroups][kSumExperts];
    __shared__ double s_d[2][kSumThreads / kWave];
    __shared__ int32_t s_i[kSumThreads / kWave];
    __shared__ int s_last;
    const int tid = threadIdx.x, blocks = (p.E + kSumExperts - 1) / kSumExperts, s = blockIdx.x / blocks, eb = blockIdx.x % blocks;
    const int from = seq_begin(p, s), to = seq_begin(p, s + 1);
    const int first = from / p.chunk, count = to > from ? (to - 1) / p.chunk - first + 1 : 0;
    const int e = eb * kSumExperts + tid % kSumExperts, grp = tid / kSumExperts;
    float sum = 0.f;
    int c = 0;
    if (e < p.E)
#pragma unroll 4
        for (int i = grp; i < count; i += kSumGroups) {
            const size_t slot = (size_t)first + i + s;
            sum += p.part_p[slot * p.E + e];
            c += p.part_c[slot * p.E + e];
        }
    s_p[grp][tid % kSumExperts] = sum;
    s_c[grp][tid % kSumExperts] = c;
    // the kept tokens of the sequence, and its z
    int n = 0;
    double z = 0.0;
    for (int i = tid; i < count; i += kSumThreads) {
        const size_t slot = (size_t)first + i + s;
        n += p.part_n[slot];
        z += (double)p.part_z[slot];
    }
    auto block_sum = [&](double& x, int which) {
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o);
        if ((tid & 63) == 0) s_d[which][tid >> 6] = x;
    };
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) n += __shfl_xor(n, o);
    if ((tid & 63) == 0) s_i[tid >> 6] = n;
    block_sum(z, 0);
    __syncthreads();
    n = 0;
    z = 0.0;
    for (int i = 0; i < kSumThreads / kWave; ++i) {
        n += s_i[i];
        z += s_d[0][i];
    }
    if (tid < kWave) {
        double b = 0.0;
        if (tid < kSumExperts && e < p.E) {
            float ps = 0.f;
            int cs = 0;
#pragma unroll
            for (int i = 0; i < kSumGroups; ++i) {
                ps += s_p[i][tid];
                cs += s_c[i][tid];
            }
            p.prob_sums[(size_t)s * p.E + e] = ps;
            p.counts[(size_t)s * p.E + e] = cs;
            b = (double)cs * ps;
        }
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) b += __shfl_xor(b, o);
        if (tid == 0) {
            p.sum_b[blockIdx.x] = n > 0 ? b / ((double)p.k * n) : 0.0;
            if (eb == 0) {
                p.sum_z[s] = z;
                p.tokens[s] = n;
            }
            __threadfence();
            s_last = atomicAdd(p.ticket, 1) == (int)gridDim.x - 1;
        }
    }
    __syncthreads();
    if (!s_last) return;
    __threadfence();
    double b = 0.0;
    z = 0.0;
    n = 0;
    for (int i = tid; i < (int)gridDim.x; i += kSumThreads) b += __hip_atomic_load(p.sum_b + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    for (int i = tid; i < p.S; i += kSumThreads) {
        z += __hip_atomic_load(p.sum_z + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        n += __hip_atomic_load(p.tokens + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) n += __shfl_xor(n, o);
    block_sum(b, 0);
    block_sum(z, 1);
    if ((tid & 63) == 0) s_i[tid >> 6] = n;
    __syncthreads();
    if (tid == 0) {
        b = z = 0.0;
        n = 0;
        for (int i = 0; i < kSumThreads / kWave; ++i) {
            b += s_d[0][i];
            z += s_d[1][i];
            n += s_i[i];
        }
        const double per = 1.0 / (n > 0 ? n : 1);
        const double balance = p.E * per * b;
        z *= per;
        p.tokens[p.S] = n;
        p.loss[0] = (float)(p.balance_coef * balance + p.z_coef * z);
        p.loss[1] = (float)balance;
        p.loss[2] = (float)z;
    }
}

template <int G, int NV, bool VEC>
__global__ void __launch_bounds__(kBalThreads) balance_backward_kernel(BalParams p) {
    using L = TokenLanes<G, NV, VEC>;
    constexpr int kGroups = 64 / G, kSlots = (kMaxTopK + G - 1) / G;
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, E = p.E;
    const L ln(lane);
    const int c0 = blockIdx.x * p.chunk, c1 = min(p.T, c0 + p.chunk);
    const int all = p.tokens[p.S];
    const float u = *p.dloss, per = 1.f / (float)max(all, 1);
    const float cb = u * p.balance_coef * (float)E * per, cz = u * p.z_coef * 2.f * per;
    int s = -1, end = 0;
    float f[L::kValues];   // cb f[s]
    for (int t0 = c0 + w * kGroups; t0 < c1; t0 += kBalWaves * kGroups) {
        const int t = t0 + lane / G;
        const bool there = t < c1;   // (the lanes of a wave stay together: they exchange the slots)
        float d[L::kValues];
#pragma unroll
        for (int v = 0; v < L::kValues; ++v) d[v] = 0.f;
        const float lse = there ? p.lse[t] : -INFINITY;
        if (lse != -INFINITY) {   // (a token that is not kept)
            if (s < 0 || t >= end) {
                s = seq_of(p, t);
                end = seq_begin(p, s + 1);
                const float scale = cb / ((float)p.k * (float)max(p.tokens[s], 1));
                int32_t cnt[L::kValues];
                ln.template load<i32x4_t>(p.counts + (size_t)s * E, E, 0, cnt);
#pragma unroll
                for (int v = 0; v < L::kValues; ++v) f[v] = scale * (float)cnt[v];
            }
            ln.template load<f32x4_t>(p.logits + (size_t)t * E, E, -INFINITY, d);
            float inner = 0.f;
#pragma unroll
            for (int v = 0; v < L::kValues; ++v) {
                d[v] = ln.expert(v) < E ? __expf(d[v] - lse) : 0.f;
                inner += f[v] * d[v];
            }
            inner = L::sum(inner);
            const float add = cz * lse - inner;
#pragma unroll
            for (int v = 0; v < L::kValues; ++v) d[v] *= f[v] + add;
        }
        if (p.w) {
            int e[kSlots];
            float g[kSlots], mean = 0.f;
#pragma unroll
            for (int i = 0; i < kSlots; ++i) {
                const int j = i * G + ln.g;
                e[i] = -1;
                g[i] = 0.f;
                if (there && j < p.k) {
                    const size_t at = (size_t)t * p.k + j;
                    const int x = p.idx[at];
                    if ((unsigned)x < (unsigned)E) {
                        e[i] = x;
                        g[i] = p.w[at];
                        mean += g[i] * p.dw[at];
                    }
                }
            }
            mean = L::sum(mean);
#pragma unroll
            for (int i = 0; i < kSlots; ++i)
                if (e[i] >= 0) g[i] *= p.dw[(size_t)t * p.k + i * G + ln.g] - mean;
#pragma unroll
            for (int i = 0; i < kSlots; ++i)
                for (int j = 0; j < min(G, p.k - i * G); ++j) {
                    int ej;
                    float gj;
                    if (G == 64) {
                        ej = __builtin_amdgcn_readlane(e[i], j);
                        gj = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(g[i]), j));
                    } else {
                        ej = __shfl(e[i], j, G);
                        gj = __shfl(g[i], j, G);
                    }
#pragma unroll
                    for (int v = 0; v < L::kValues; ++v) d[v] += ln.expert(v) == ej ? gj : 0.f;
                }
        }
        if (!there) continue;
        if (VEC) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int e = 4 * (G * i + ln.g);
                if (e >= E) continue;
                if (p.out_bf16)
                    *(u32x2_t*)((uint16_t*)p.dlogits + (size_t)t * E + e) = u32x2_t{pack_bf16x2(d[4 * i], d[4 * i + 1]), pack_bf16x2(d[4 * i + 2], d[4 * i + 3])};
                else
                    *(f32x4_t*)((float*)p.dlogits + (size_t)t * E + e) = f32x4_t{d[4 * i], d[4 * i + 1], d[4 * i + 2], d[4 * i + 3]};
            }
        } else {
#pragma unroll
            for (int v = 0; v < L::kValues; ++v) {
                const int e = ln.expert(v);
                if (e >= E) continue;
                if (p.out_bf16) ((uint16_t*)p.dlogits)[(size_t)t * E + e] = (uint16_t)(pack_bf16x2(d[v], 0.f) & 0xffffu);
                else ((float*)p.dlogits)[(size_t)t * E + e] = d[v];
            }
        }
    }
}

// ------------------------------------------------------------------ launches
// Tokens of a chunk (one workgroup).
static int chunk_of(const moe_balance_shape_t& s) {
    int chunk = 32;
    while (chunk < 128 && (s.T + chunk - 1) / chunk > 1024) chunk *= 2;
    while (chunk > 4 && (long long)chunk * s.seqs > 4ll * s.T) chunk /= 2;   // a part is a turn of the workgroup: few sequences a chunk
    return chunk;
}
static int sum_blocks(const moe_balance_shape_t& s) { return (s.E + kSumExperts - 1) / kSumExperts; }
struct BalLayout {
    size_t p, c, z, n, b, sz, ticket, total;
};
static BalLayout bal_layout(const moe_balance_shape_t& s) {
    const int chunk = chunk_of(s);
    const size_t slots = ((size_t)s.T + chunk - 1) / chunk + s.seqs;
    BalLayout L;
    size_t at = 0;
    L.p = at, at = align_up(at + slots * s.E * 4, 256);
    L.c = at, at = align_up(at + slots * s.E * 4, 256);
    L.z = at, at = align_up(at + slots * 4, 256);
    L.n = at, at = align_up(at + slots * 4, 256);
    L.b = at, at = align_up(at + (size_t)s.seqs * sum_blocks(s) * 8, 256);
    L.sz = at, at = align_up(at + (size_t)s.seqs * 8, 256);
    L.ticket = at, at += 256;
    L.total = at;
    return L;
}
size_t balance_workspace_bytes(const moe_balance_shape_t& s) { return bal_layout(s).total; }

// f(G, NV, VEC) with constants
template <class F>
static void by_experts(int E, bool vec, F f) {
    auto with = [&](auto g, auto nv) {
        if (vec) f(g, nv, std::true_type{});
        else f(g, nv, std::false_type{});
    };
    if (E <= 8) with(std::integral_constant<int, 2>{}, std::integral_constant<int, 1>{});
    else if (E <= 32) with(std::integral_constant<int, 8>{}, std::integral_constant<int, 1>{});
    else if (E <= 64) with(std::integral_constant<int, 16>{}, std::integral_constant<int, 1>{});
    else if (E <= 128) with(std::integral_constant<int, 32>{}, std::integral_constant<int, 1>{});
    else if (E <= 256) with(std::integral_constant<int, 64>{}, std::integral_constant<int, 1>{});
    else if (E <= 512) with(std::integral_constant<int, 64>{}, std::integral_constant<int, 2>{});
    else with(std::integral_constant<int, 64>{}, std::integral_constant<int, 4>{});
}
static void bal_params(BalParams& p, const moe_balance_shape_t& s) {
    p.T = s.T, p.E = s.E, p.k = s.k, p.S = s.seqs;
    p.balance_coef = s.balance_coef, p.z_coef = s.z_coef;
    p.chunk = chunk_of(s);
    p.chunks = (s.T + p.chunk - 1) / p.chunk;
}
// Whether every row of both can be moved 16 bytes a lane.
static bool rows_aligned(const void* a, const void* b, int E) { return E % 4 == 0 && (((uintptr_t)a | (uintptr_t)b) & 15) == 0; }

__global__ void balance_ticket_kernel(int32_t* ticket) { *ticket = 0; }

int balance_forward_launch(const moe_balance_shape_t& s, const float* logits, const int32_t* idx, const int32_t* offsets, const uint8_t* mask,
                           const moe_balance_stats_t& out, char* ws, hipStream_t st) {
    BalParams p = {};
    bal_params(p, s);
    const BalLayout L = bal_layout(s);
    p.logits = logits, p.idx = idx, p.offsets = offsets, p.mask = mask;
    p.loss = out.loss, p.counts = out.counts, p.tokens = out.tokens, p.prob_sums = out.prob_sums, p.lse = out.lse;
    p.part_p = (float*)(ws + L.p), p.part_c = (int32_t*)(ws + L.c), p.part_z = (float*)(ws + L.z), p.part_n = (int32_t*)(ws + L.n);
    p.sum_b = (double*)(ws + L.b), p.sum_z = (double*)(ws + L.sz), p.ticket = (int32_t*)(ws + L.ticket);
    if (p.chunks > 0)
        by_experts(s.E, rows_aligned(logits, nullptr, s.E), [&](auto g, auto nv, auto vec) {
            hipLaunchKernelGGL((balance_forward_kernel<g.value, nv.value, vec.value>), dim3((unsigned)p.chunks), dim3(kBalThreads), 0, st, p);
        });
    else hipLaunchKernelGGL(balance_ticket_kernel, dim3(1), dim3(1), 0, st, p.ticket);
    hipLaunchKernelGGL(balance_sum_kernel, dim3((unsigned)(s.seqs * sum_blocks(s))), dim3(kSumThreads), 0, st, p);
    return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP;
}

int balance_backward_launch(const moe_balance_shape_t& s, const float* logits, const int32_t* idx, const int32_t* offsets, const moe_balance_stats_t& stats, const float* w, const float* dw, const float* dloss, void* dlogits, int out_bf16,
                            hipStream_t st) {
    if (s.T == 0) return MOE_OK;
    BalParams p = {};
    bal_params(p, s);
    p.logits = logits, p.idx = idx, p.offsets = offsets;
    p.counts = stats.counts, p.tokens = stats.tokens, p.lse = stats.lse;
    p.w = w, p.dw = dw, p.dloss = dloss, p.dlogits = dlogits, p.out_bf16 = out_bf16;
    p.chunk = 32;
    while (p.chunk < 128 && (s.T + p.chunk - 1) / p.chunk > 1024) p.chunk *= 2;
    p.chunks = (s.T + p.chunk - 1) / p.chunk;
    const bool vec = rows_aligned(logits, dlogits, s.E) && ((uintptr_t)stats.counts & 15) == 0;
    by_experts(s.E, vec, [&](auto g, auto nv, auto v) {
        hipLaunchKernelGGL((balance_backward_kernel<g.value, nv.value, v.value>), dim3((unsigned)p.chunks), dim3(kBalThreads), 0, st, p);
    });
    return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP;
}

}  // namespace uniep
