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
    double* part_z;           // [slots]
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
// Last sequence that begins at or before token t, the same in the whole wave, whose lanes look at 64 of them at a time: one load for up to 64 sequences, two
// for 4096 (a search by halves waits for six loads one after the other for 64).
__device__ __forceinline__ int seq_of(const BalParams& p, int t) {
    if (!p.offsets) return 0;
    const int lane = threadIdx.x & 63;
    int lo = 0, n = p.S;   // it is one of lo .. lo + n - 1
    while (n > 1) {
        const int step = (n + 63) >> 6, i = lo + lane * step;
        const int before = __popcll(__ballot(lane * step < n && p.offsets[min(i, p.S - 1)] <= t));
        const int at = max(before - 1, 0) * step;
        lo += at;
        n = min(step, n - at);
    }
    return rfl(lo);
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
    // over the lanes of a token, the same bits in each
    static __device__ __forceinline__ float sum(float v) {
        across<G>(v, [](float a, float b) { return a + b; });
        return v;
    }
    static __device__ __forceinline__ float most(float v) {
        across<G>(v, [](float a, float b) { return fmaxf(a, b); });
        return v;
    }
};
typedef __attribute__((ext_vector_type(4))) int32_t i32x4_t;

__device__ __forceinline__ void write_losses(const BalParams& p, double b, double z, int n) {   // b, z: the sums over all sequences and tokens
    const double per = 1.0 / (n > 0 ? n : 1), balance = p.E * per * b;
    z *= per;
    p.tokens[p.S] = n;
    p.loss[0] = (float)(p.balance_coef * balance + p.z_coef * z);
    p.loss[1] = (float)balance;
    p.loss[2] = (float)z;
}

// With one workgroup (one_launch) it writes the results itself, else the parts that balance_sum_kernel adds.
template <int G, int NV, bool VEC>
__global__ void __launch_bounds__(kBalThreads) balance_forward_kernel(BalParams p) {
    using L = TokenLanes<G, NV, VEC>;
    constexpr int kMost = 4 * G * NV, kGroups = 64 / G, kU = NV == 1 ? (G == 64 ? 8 : 4) : 1, kSlots = (kMaxTopK + G - 1) / G;
    __shared__ float s_p[kBalWaves][kMost];
    __shared__ int32_t s_c[kMost];
    __shared__ double s_z[kBalWaves];
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
        float sums[L::kValues] = {};
        double z = 0.0;   // (squares: in fp32 those of logits beyond 1.8e19, such as a mask's lowest value, would be infinite, and 0 times them NaN)
        int n = 0;
        // U tokens a turn: their loads are on their way together
        for (int t0 = a + w * kGroups + lane / G; t0 < b; t0 += kU * kBalWaves * kGroups) {
            float x[kU][L::kValues];
            int slot[kU][kSlots];
            bool keep[kU];
#pragma unroll
            for (int u = 0; u < kU; ++u) {
                const int t = t0 + u * kBalWaves * kGroups;
                keep[u] = t < b && (!p.mask || p.mask[t]);
            }
            // (fetched whether they are kept or not: behind the mask they would wait for it)
#pragma unroll
            for (int u = 0; u < kU; ++u)
                if (t0 + u * kBalWaves * kGroups < b) {
                    const size_t t = t0 + u * kBalWaves * kGroups;
                    ln.template load<f32x4_t>(p.logits + t * E, E, -INFINITY, x[u]);
#pragma unroll
                    for (int i = 0; i < kSlots; ++i) slot[u][i] = i * G + ln.g < p.k ? p.idx[t * p.k + i * G + ln.g] : -1;
                }
#pragma unroll
            for (int u = 0; u < kU; ++u) {
                const int t = t0 + u * kBalWaves * kGroups;
                float lse = -INFINITY;
                if (keep[u]) {
                    float m = x[u][0];
#pragma unroll
                    for (int v = 1; v < L::kValues; ++v) m = fmaxf(m, x[u][v]);
                    m = L::most(m);
                    float q = 0.f;
#pragma unroll
                    for (int v = 0; v < L::kValues; ++v) {
                        x[u][v] = ln.expert(v) < E ? __expf(x[u][v] - m) : 0.f;
                        q += x[u][v];
                    }
#pragma unroll
                    for (int i = 0; i < kSlots; ++i)
                        if ((unsigned)slot[u][i] < (unsigned)E) atomicAdd(&s_c[slot[u][i]], 1);
                    const float total = L::sum(q), inv = 1.f / total;
#pragma unroll
                    for (int v = 0; v < L::kValues; ++v) sums[v] += x[u][v] * inv;
                    lse = m + logf(total);
                    if (ln.g == 0) {
                        z += (double)lse * lse;
                        ++n;
                    }
                }
                if (ln.g == 0 && t < b) p.lse[t] = lse;
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
        if (gridDim.x == 1 && p.S == 1) {
            __shared__ double s_b[kBalWaves];
            n = s_n[0] + s_n[1] + s_n[2] + s_n[3];
            double bal = 0.0;
            for (int e = tid; e < E; e += kBalThreads) {
                const float sum = ((s_p[0][e] + s_p[1][e]) + s_p[2][e]) + s_p[3][e];
                p.prob_sums[e] = sum;
                p.counts[e] = s_c[e];
                bal += (double)s_c[e] * sum;
            }
#pragma unroll
            for (int o = 32; o > 0; o >>= 1) bal += __shfl_xor(bal, o);
            if (lane == 0) s_b[w] = bal;
            __syncthreads();
            if (tid == 0) {
                p.tokens[0] = n;
                write_losses(p, n > 0 ? (((s_b[0] + s_b[1]) + s_b[2]) + s_b[3]) / ((double)p.k * n) : 0.0, ((s_z[0] + s_z[1]) + s_z[2]) + s_z[3], n);
            }
            return;
        }
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

// Sums the parts of one sequence and `wide` experts (a power of two), 1024 / wide threads an expert; where there are several workgroups, the one that is last
// to end adds up the losses.  What it reads of the others they have written through to memory: a fence each, which writes back an L2, took
// most of the time (61 sequences of 256 experts, 488 workgroups of 32 experts 24 us).
constexpr int kSumThreads = 1024, kSumWaves = kSumThreads / kWave;
__global__ void __launch_bounds__(kSumThreads) balance_sum_kernel(BalParams p, int wide, int blocks) {
    __shared__ double s_p[kSumThreads];
    __shared__ int32_t s_c[kSumThreads];
    __shared__ double s_d[3][kSumWaves];
    __shared__ int32_t s_i[2][kSumWaves];
    __shared__ int s_last;
    const int tid = threadIdx.x, s = blockIdx.x / blocks, eb = blockIdx.x % blocks;
    const int from = seq_begin(p, s), to = seq_begin(p, s + 1);
    const int first = from / p.chunk, count = to > from ? (to - 1) / p.chunk - first + 1 : 0;
    const int lane = tid & (wide - 1), e = eb * wide + lane, grp = tid / wide, groups = kSumThreads / wide;
    auto sum_d = [&](double x, int which) {
        x = wave_sum(x);
        if ((tid & 63) == 0) s_d[which][tid >> 6] = x;
    };
    auto sum_i = [&](int x, int which) {
        x = wave_sum(x);
        if ((tid & 63) == 0) s_i[which][tid >> 6] = x;
    };
    // the kept tokens of the sequence, and its z
    int n = 0;
    double z = 0.0;
    for (int i = tid; i < count; i += kSumThreads) {
        const size_t slot = (size_t)first + i + s;
        n += p.part_n[slot];
        z += p.part_z[slot];
    }
    // (in 64 bits: there are as many parts as the tokens make, and parts that are alike are rounded alike; of 65536 alike, 2048 a thread, sums in fp32 were off by 2.7e-5.
    // The eight parts that a turn fetches are added among themselves first: 131072 tokens, 129 experts 15.9 us, with a 64-bit addition for each 19.8)
    double sum = 0.0;
    int c = 0;
    if (e < p.E) {
        int i = grp;
        for (; i + 7 * groups < count; i += 8 * groups) {
            float v[8];
            int u[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const size_t at = ((size_t)first + i + k * groups + s) * p.E + e;
                v[k] = p.part_p[at];
                u[k] = p.part_c[at];
            }
            sum += (double)(((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7])));
            c += ((u[0] + u[1]) + (u[2] + u[3])) + ((u[4] + u[5]) + (u[6] + u[7]));
        }
        for (; i < count; i += groups) {
            const size_t at = ((size_t)first + i + s) * p.E + e;
            sum += (double)p.part_p[at];
            c += p.part_c[at];
        }
    }
    s_p[tid] = sum;
    s_c[tid] = c;
    sum_i(n, 0);
    sum_d(z, 0);
    __syncthreads();
    double b = 0.0;
    if (tid < wide && e < p.E) {
        sum = 0.0;
        c = 0;
#pragma unroll 8
        for (int i = 0; i < groups; ++i) {
            sum += s_p[i * wide + tid];
            c += s_c[i * wide + tid];
        }
        p.prob_sums[(size_t)s * p.E + e] = (float)sum;
        p.counts[(size_t)s * p.E + e] = c;
        b = (double)c * sum;
    }
    sum_d(b, 1);
    __syncthreads();
    b = z = 0.0;
    n = 0;
    for (int i = 0; i < kSumWaves; ++i) {
        b += s_d[1][i];
        z += s_d[0][i];
        n += s_i[0][i];
    }
    if (n > 0) b /= (double)p.k * n;
    if (tid == 0 && eb == 0) __hip_atomic_store(p.tokens + s, n, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (gridDim.x > 1) {
        if (tid == 0) {
            store_wt8(p.sum_b + blockIdx.x, __builtin_bit_cast(u32x2_t, b));
            if (eb == 0) store_wt8(p.sum_z + s, __builtin_bit_cast(u32x2_t, z));
            wait_stores();
            s_last = __hip_atomic_fetch_add(p.ticket, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (int)gridDim.x - 1;
        }
        __syncthreads();
        if (!s_last) return;
        b = z = 0.0;
        n = 0;
        for (int i = tid; i < (int)gridDim.x; i += kSumThreads) b += __hip_atomic_load(p.sum_b + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        for (int i = tid; i < p.S; i += kSumThreads) {
            z += __hip_atomic_load(p.sum_z + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            n += __hip_atomic_load(p.tokens + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        sum_i(n, 1);
        sum_d(b, 1);
        sum_d(z, 2);
        __syncthreads();
        b = z = 0.0;
        n = 0;
        for (int i = 0; i < kSumWaves; ++i) {
            b += s_d[1][i];
            z += s_d[2][i];
            n += s_i[1][i];
        }
    }
    if (tid == 0) write_losses(p, b, z, n);
}

// The gates' part goes to its experts through a row of LDS that is all zeros between tokens: the lanes of the slots add to it and clear their
// entries again once every lane has read its own.
template <int G, int NV, bool VEC>
__global__ void __launch_bounds__(kBalThreads) balance_backward_kernel(BalParams p) {
    using L = TokenLanes<G, NV, VEC>;
    constexpr int kGroups = 64 / G, kSlots = (kMaxTopK + G - 1) / G, kMost = 4 * G * NV, kU = NV == 1 && G > 8 ? 2 : 1;
    __shared__ __attribute__((aligned(16))) float s_row[kBalWaves * kGroups][kMost];
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, E = p.E;
    const L ln(lane);
    float* const row = s_row[w * kGroups + lane / G];
    const int c0 = blockIdx.x * p.chunk, c1 = min(p.T, c0 + p.chunk);
    const int all = p.tokens[p.S];
    const float up = *p.dloss, per = 1.f / (float)max(all, 1);
    const float cb = up * p.balance_coef * (float)E * per, cz = up * p.z_coef * 2.f * per;
    if (p.w)
#pragma unroll
        for (int v = 0; v < L::kValues; ++v) row[ln.expert(v)] = 0.f;
    int s = seq_of(p, min(c0 + w * kGroups, p.T - 1)), end = -1;   // (of the wave's first token; then every group goes on by itself)
    float f[L::kValues];   // cb f[s]
    for (int t0 = c0 + w * kGroups + lane / G; t0 < c1; t0 += kU * kBalWaves * kGroups) {
        float d[kU][L::kValues], lse[kU], g[kU][kSlots], dw[kU][kSlots];
        int e[kU][kSlots];
#pragma unroll
        for (int u = 0; u < kU; ++u) {
            const int t = t0 + u * kBalWaves * kGroups;
            lse[u] = t < c1 ? p.lse[t] : -INFINITY;   // -inf: a token that is not kept
            if (t < c1) ln.template load<f32x4_t>(p.logits + (size_t)t * E, E, -INFINITY, d[u]);
#pragma unroll
            for (int i = 0; i < kSlots; ++i) {
                const int j = i * G + ln.g;
                e[u][i] = -1;
                g[u][i] = dw[u][i] = 0.f;
                if (p.w && t < c1 && j < p.k) {
                    const size_t at = (size_t)t * p.k + j;
                    e[u][i] = p.idx[at];
                    g[u][i] = p.w[at];
                    dw[u][i] = p.dw[at];
                }
            }
        }
#pragma unroll
        for (int u = 0; u < kU; ++u) {
            const int t = t0 + u * kBalWaves * kGroups;
            if (t >= c1) break;
            if (lse[u] != -INFINITY) {
                if (t >= end) {
                    while ((end = seq_begin(p, s + 1)) <= t && s + 1 < p.S) ++s;
                    const float scale = cb / ((float)p.k * (float)max(p.tokens[s], 1));
                    int32_t cnt[L::kValues];
                    ln.template load<i32x4_t>(p.counts + (size_t)s * E, E, 0, cnt);
#pragma unroll
                    for (int v = 0; v < L::kValues; ++v) f[v] = scale * (float)cnt[v];
                }
                // (divided by their sum: lse has been rounded, which for logits of thousands is a factor of 1e-4 to all of them)
                float inner = 0.f, q = 0.f;
#pragma unroll
                for (int v = 0; v < L::kValues; ++v) {
                    d[u][v] = ln.expert(v) < E ? __expf(d[u][v] - lse[u]) : 0.f;
                    inner += f[v] * d[u][v];
                    q += d[u][v];
                }
                const float inv = 1.f / L::sum(q), add = cz * lse[u] - L::sum(inner) * inv;
#pragma unroll
                for (int v = 0; v < L::kValues; ++v) d[u][v] *= (f[v] + add) * inv;
            } else {
#pragma unroll
                for (int v = 0; v < L::kValues; ++v) d[u][v] = 0.f;
            }
            if (p.w) {
                float mean = 0.f;
#pragma unroll
                for (int i = 0; i < kSlots; ++i) {
                    if ((unsigned)e[u][i] >= (unsigned)E) g[u][i] = 0.f;
                    mean += (unsigned)e[u][i] < (unsigned)E ? g[u][i] * dw[u][i] : 0.f;
                }
                mean = L::sum(mean);
#pragma unroll
                for (int i = 0; i < kSlots; ++i)
                    if ((unsigned)e[u][i] < (unsigned)E) atomicAdd(&row[e[u][i]], g[u][i] * (dw[u][i] - mean));
                asm volatile("" ::: "memory");   // (one wave's LDS operations are done in order)
#pragma unroll
                for (int v = 0; v < L::kValues; v += VEC ? 4 : 1) {
                    if (VEC) {
                        const f32x4_t r = *(const f32x4_t*)&row[ln.expert(v)];
#pragma unroll
                        for (int c = 0; c < 4; ++c) d[u][v + c] += r[c];
                    } else {
                        d[u][v] += row[ln.expert(v)];
                    }
                }
                asm volatile("" ::: "memory");
#pragma unroll
                for (int i = 0; i < kSlots; ++i)
                    if ((unsigned)e[u][i] < (unsigned)E) row[e[u][i]] = 0.f;
                asm volatile("" ::: "memory");
            }
            if (VEC) {
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    const int x = 4 * (G * i + ln.g);
                    if (x >= E) continue;
                    const float* v = &d[u][4 * i];
                    if (p.out_bf16) *(u32x2_t*)((uint16_t*)p.dlogits + (size_t)t * E + x) = u32x2_t{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
                    else *(f32x4_t*)((float*)p.dlogits + (size_t)t * E + x) = f32x4_t{v[0], v[1], v[2], v[3]};
                }
            } else {
#pragma unroll
                for (int v = 0; v < L::kValues; ++v) {
                    const int x = ln.expert(v);
                    if (x >= E) continue;
                    if (p.out_bf16) ((uint16_t*)p.dlogits)[(size_t)t * E + x] = (uint16_t)(pack_bf16x2(d[u][v], 0.f) & 0xffffu);
                    else ((float*)p.dlogits)[(size_t)t * E + x] = d[u][v];
                }
            }
        }
    }
}

// ------------------------------------------------------------------ launches
// Whether one workgroup is the faster way: one sequence, and up to four turns of its four waves (with G lanes a token a wave takes 64 / G tokens, four times, a
// turn).  Measured, us of a pass with the backward call in a graph of ten, in one launch / in two (tokens, experts): 64, 8 6.6 / 10.0; 256, 8 7.8 / 10.7; 1024, 8 (two turns) 10.9 / 11.2;
// 2048, 8 15.3 / 11.5; 512, 32 11.8 / 10.6; 64, 64 7.9 / 10.2; 256, 64 12.2 / 10.7; 64, 128 9.8 / 11.3; 128, 128 13.1 / 12.2; 64, 256 15.0 / 15.1.  With three and four turns the GPU takes longer, by up to
// 4 us; outside a graph a pass takes the host's 13 us, of which a launch is 2.4.
static bool one_launch(const moe_balance_shape_t& s) {
    const int lanes = s.E <= 8 ? 2 : s.E <= 32 ? 8 : s.E <= 64 ? 16 : s.E <= 128 ? 32 : 64;
    return s.seqs == 1 && s.T > 0 && s.E <= 256 && s.T <= 4 * (64 / lanes) * 4 * kBalWaves;
}
// Tokens of a chunk (one workgroup).
static int chunk_of(const moe_balance_shape_t& s) {
    if (one_launch(s)) return s.T;
    int chunk = 32;
    while (chunk < 64 && (s.T + chunk - 1) / chunk > 1024) chunk *= 2;
    while (chunk > 4 && (long long)chunk * s.seqs > 4ll * s.T) chunk /= 2;   // a part is a turn of the workgroup: few sequences a chunk
    return chunk;
}
// Experts of a workgroup of the sum: as many as leave a thread up to 4 parts on average (61 sequences of 256 experts and 34 parts, 488 / 244 / 61 workgroups 11.2 / 8.1 / 10.7 us:
// fewer wait for the longest sequence, more for the ticket).  (One workgroup for 8192 tokens, 128 experts and 257 parts needs no other's sums, and was slower.)
static int sum_wide(const moe_balance_shape_t& s) {
    const long long parts = (s.T + chunk_of(s) - 1) / chunk_of(s) / s.seqs + 1;
    int wide = 32;
    while (wide < s.E && wide * 2 * parts <= 4 * kSumThreads) wide *= 2;
    return wide;
}
static int sum_blocks(const moe_balance_shape_t& s) { return (s.E + sum_wide(s) - 1) / sum_wide(s); }
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
    L.z = at, at = align_up(at + slots * 8, 256);
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
    p.part_p = (float*)(ws + L.p), p.part_c = (int32_t*)(ws + L.c), p.part_z = (double*)(ws + L.z), p.part_n = (int32_t*)(ws + L.n);
    p.sum_b = (double*)(ws + L.b), p.sum_z = (double*)(ws + L.sz), p.ticket = (int32_t*)(ws + L.ticket);
    if (p.chunks > 0)
        by_experts(s.E, rows_aligned(logits, nullptr, s.E), [&](auto g, auto nv, auto vec) {
            hipLaunchKernelGGL((balance_forward_kernel<g.value, nv.value, vec.value>), dim3((unsigned)p.chunks), dim3(kBalThreads), 0, st, p);
        });
    else hipLaunchKernelGGL(balance_ticket_kernel, dim3(1), dim3(1), 0, st, p.ticket);
    if (p.chunks == 1 && s.seqs == 1) return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP;
    hipLaunchKernelGGL(balance_sum_kernel, dim3((unsigned)(s.seqs * sum_blocks(s))), dim3(kSumThreads), 0, st, p, sum_wide(s), sum_blocks(s));
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
    while (p.chunk < 64 && (s.T + p.chunk - 1) / p.chunk > 2048) p.chunk *= 2;
    p.chunks = (s.T + p.chunk - 1) / p.chunk;
    const bool vec = rows_aligned(logits, dlogits, s.E) && ((uintptr_t)stats.counts & 15) == 0;
    by_experts(s.E, vec, [&](auto g, auto nv, auto v) {
        hipLaunchKernelGGL((balance_backward_kernel<g.value, nv.value, v.value>), dim3((unsigned)p.chunks), dim3(kBalThreads), 0, st, p);
    });
    return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP;
}

}  // namespace uniep
