// extern "C" boundary: argument checks, workspace carving, launches.
// Every check happens before anything is enqueued.
#include "common.hpp"

#include <algorithm>

namespace uniep {
size_t route_workspace_bytes(const moe_shape_t& s);
int route_backward_launch(const moe_shape_t& s, const int32_t* topk_idx, const float* topk_w,
                          const float* dtopk_w, float* dlogits, hipStream_t st);
int route_launch(const moe_shape_t& s, const float* logits, const moe_routing_t& out, void* ws,
                 hipStream_t st);
int route_static_launch(const moe_shape_t& s, const float* logits, const moe_routing_t& out,
                        hipStream_t st);
int global_map_launch(const moe_shape_t& s, int W, int rank, const moe_routing_t& r,
                      const int32_t* c_all, const moe_global_map_t& out, void* ws, hipStream_t st);
size_t fwd_workspace_bytes(const moe_shape_t& s);
size_t fwd_ctrl_bytes(const moe_shape_t& s);
int fwd_launch(const moe_shape_t& s, const void* x, const void* w_gate, const void* w_up,
               const void* w_down, const moe_routing_t& r, void* y, char* gu, char* h, char* o,
               char* ws, const moe_opts_t& opts, hipStream_t st);
size_t bwd_workspace_bytes(const moe_shape_t& s, int split_rows);
bool bwd_split_ok(const moe_shape_t& s, int split_rows);
int bwd_launch(const moe_shape_t& s, const void* dy, const void* x, const void* w_gate,
               const void* w_up, const void* w_down, const moe_routing_t& r, const char* gu,
               const char* h, const char* o, void* dx, void* dw_gate, void* dw_up, void* dw_down,
               float* dtopk_w, char* ws, const moe_opts_t& opts, hipStream_t st);
bool adapter_needs_plan(const moe_adapter_shape_t& s);
size_t adapter_plan_bytes(const moe_adapter_shape_t& s);
size_t adapter_table_bytes(const moe_adapter_shape_t& s);
size_t adapter_workspace_bytes(const moe_adapter_shape_t& s);
int adapter_plan_launch(const moe_adapter_shape_t& s, const int32_t* ids, void* plan, hipStream_t st);
int adapter_forward_launch(const moe_adapter_shape_t& s, const void* x, size_t ldx, const void* w, const void* a,
                           const void* b, const float* scale, const int32_t* ids, void* plan, void* y, int out_f32,
                           float* h, char* ws, hipStream_t st);
int adapter_backward_launch(const moe_adapter_shape_t& s, const void* dy, size_t lddy, const void* x, size_t ldx,
                            const void* w, const void* a, const void* b, const float* scale, const int32_t* ids,
                            void* plan, const float* h, void* dx, float* da, float* db, char* ws, hipStream_t st);
size_t balance_workspace_bytes(const moe_balance_shape_t& s);
int balance_forward_launch(const moe_balance_shape_t& s, const float* logits, const int32_t* idx,
                           const int32_t* offsets, const uint8_t* mask, const moe_balance_stats_t& out, char* ws,
                           hipStream_t st);
int balance_backward_launch(const moe_balance_shape_t& s, const float* logits, const int32_t* idx,
                            const int32_t* offsets, const moe_balance_stats_t& stats, const float* w, const float* dw, const float* dloss, void* dlogits, int out_bf16,
                            hipStream_t st);
int dispatch_forward_launch(const moe_dispatch_shape_t& s, const void* x, size_t ldx, int f32, const int32_t* row_of, void* xs, hipStream_t st);
int combine_forward_launch(const moe_dispatch_shape_t& s, const void* o, int f32, const int32_t* row_of, const float* w, void* y, hipStream_t st);
int combine_backward_launch(const moe_dispatch_shape_t& s, const void* dy, size_t lddy, const void* o, int f32, const int32_t* row_of, const float* w,
                            void* d_o, float* dw, hipStream_t st);
int saved_pack_launch(const moe_shape_t& s, const int32_t* offsets, const char* gu, uint8_t* codes, uint8_t* scales, hipStream_t st);
int saved_unpack_launch(const moe_shape_t& s, const int32_t* offsets, const uint8_t* codes, const uint8_t* scales, char* gu, char* h, hipStream_t st);
int mx_quantize_launch(const void* x, size_t ldx, int f32, int64_t rows, int K, uint8_t* codes, uint8_t* scales, hipStream_t st);
int mx_values_launch(const uint8_t* codes, const uint8_t* scales, int64_t rows, int K, void* out, int f32, hipStream_t st);
int mx_quantize_weights_launch(const void* w, int experts, int K, int N, uint8_t* codes, uint8_t* scales, hipStream_t st);
int mx_product_launch(const moe_mx_shape_t& s, bool gate, const uint8_t* a_codes, const uint8_t* a_scales, int64_t a_rows, const int32_t* perm, int k,
                      const uint8_t* w_codes, const uint8_t* w_scales, const uint8_t* u_codes, const uint8_t* u_scales, const int32_t* offsets, void* y, int f32,
                      uint8_t* h_codes, uint8_t* h_scales, hipStream_t st);
}  // namespace uniep

using namespace uniep;

namespace {

int check_shape(const moe_shape_t* s) {
    if (!s) return MOE_ERR_ARG;
    if (s->T < 0 || s->d < 64 || s->I < 64 || s->E < 1 || s->k < 1) return MOE_ERR_SHAPE;
    if (s->k > kMaxTopK || s->E > kMaxExperts || s->k > s->E) return MOE_ERR_SHAPE;
    if (s->e_start < 0 || s->e_count < 1 || s->e_start + s->e_count > s->E) return MOE_ERR_SHAPE;
    if (s->d % 64 != 0 || s->I % 64 != 0) return MOE_ERR_SHAPE;
    if ((int64_t)s->T * s->k >= (1ll << 30)) return MOE_ERR_SHAPE;
    return MOE_OK;
}

// A GEMM task has 16 bits for its column tile, of 256 columns (d) or 128 (I, gate and up side by side).
int check_layer_shape(const moe_shape_t* s) {
    const int rc = check_shape(s);
    if (rc != MOE_OK) return rc;
    return s->d > 65536 * 256 || s->I > 65536 * 128 ? MOE_ERR_SHAPE : MOE_OK;
}

bool aligned(const void* p, size_t a) { return ((uintptr_t)p % a) == 0; }

int check_routing(const moe_routing_t* r, int T) {
    if (!r) return MOE_ERR_ARG;
    if (!r->counts || !r->offsets) return MOE_ERR_ARG;
    if (T > 0 && (!r->topk_idx || !r->topk_w || !r->perm || !r->inv_perm)) return MOE_ERR_ARG;
    if (!aligned(r->topk_idx, 4) || !aligned(r->topk_w, 4) || !aligned(r->counts, 4) ||
        !aligned(r->offsets, 4) || !aligned(r->perm, 4) || !aligned(r->inv_perm, 4))
        return MOE_ERR_ARG;
    return MOE_OK;
}

int check_opts(const moe_opts_t* o, moe_opts_t* out) {
    moe_opts_t d = {};
    if (o) d = *o;
    if (d.schedule < 0 || d.schedule > 3 || d.workers < 0 || d.spin_limit_ms < 0) return MOE_ERR_ARG;
    if (d.tile_rows != 0 && d.tile_rows != 128 && d.tile_rows != 256) return MOE_ERR_ARG;
    if (d.skip_tail != 0 && d.skip_tail != 1) return MOE_ERR_ARG;
    if (d.dw_accumulate != 0 && d.dw_accumulate != 1) return MOE_ERR_ARG;
    if (d.dw_split_rows < 0 || d.dw_split_rows % 64 != 0 || (d.dw_split_rows != 0 && d.dw_split_rows < 256))
        return MOE_ERR_ARG;
    if (d.reserved[0] != 0) return MOE_ERR_ARG;
    *out = d;
    return MOE_OK;
}

int check_adapter_shape(const moe_adapter_shape_t* s) {
    if (!s) return MOE_ERR_ARG;
    if (s->T < 0 || s->T > 1 << 26 || s->adapters < 1 || s->adapters > kMaxAdapters) return MOE_ERR_SHAPE;
    if (s->rank < 8 || s->rank > kMaxRank || s->rank % 8 != 0) return MOE_ERR_SHAPE;
    for (int width : {s->K, s->N}) {
        if (width < 8 || width > 1 << 16 || width % 8 != 0) return MOE_ERR_SHAPE;
        if ((int64_t)s->T * width > (1ll << 38)) return MOE_ERR_SHAPE;
    }
    return MOE_OK;
}
int check_balance_shape(const moe_balance_shape_t* s) {
    if (!s) return MOE_ERR_ARG;
    if (s->T < 0 || s->E < 1 || s->E > kMaxExperts || s->k < 1 || s->k > kMaxTopK || s->k > s->E) return MOE_ERR_SHAPE;
    if ((int64_t)s->T * s->k >= (1ll << 30) || s->seqs < 1 || s->seqs > 65536) return MOE_ERR_SHAPE;
    return MOE_OK;
}
// What both directions of the projection have to be given.
int check_adapter(const moe_adapter_shape_t& s, const void* w, const void* a, const void* b, const float* scale, const int32_t* ids,
                  const void* plan, const void* ws, size_t ws_bytes) {
    if (!w || !a || !b || !ws) return MOE_ERR_ARG;
    if (s.T > 0 && (!ids || (adapter_needs_plan(s) && !plan))) return MOE_ERR_ARG;
    if (!aligned(w, 16) || !aligned(a, 16) || !aligned(b, 16) || !aligned(scale, 4) || !aligned(ids, 4) || !aligned(plan, 16) || !aligned(ws, 256))
        return MOE_ERR_ARG;
    return ws_bytes < adapter_workspace_bytes(s) ? MOE_ERR_WORKSPACE : MOE_OK;
}
bool bad_rows(const moe_adapter_shape_t& s, const void* p, int64_t ld, int width) {
    if (s.T == 0) return false;
    return !p || !aligned(p, 16) || ld < width || ld % 8 != 0 || ld > (1ll << 40) / s.T;
}
int check_balance(const moe_balance_shape_t& s, const float* logits, const int32_t* idx, const int32_t* offsets, const moe_balance_stats_t* st) {
    if (!st || !st->counts || !st->tokens) return MOE_ERR_ARG;
    if (s.T > 0 && (!logits || !idx || !st->lse)) return MOE_ERR_ARG;
    if (!offsets && s.seqs != 1) return MOE_ERR_ARG;
    const void* ptrs[] = {logits, idx, offsets, st->counts, st->tokens, st->lse};
    for (const void* p : ptrs)
        if (!aligned(p, 4)) return MOE_ERR_ARG;
    return MOE_OK;
}

int check_dispatch_shape(const moe_dispatch_shape_t* s) {
    if (!s) return MOE_ERR_ARG;
    if (s->T < 0 || s->k < 1 || s->k > kMaxTopK || (int64_t)s->T * s->k >= (1ll << 30) || s->rows < 0) return MOE_ERR_SHAPE;
    if (s->d < 8 || s->d > 1 << 20 || s->d % 8 != 0 || (int64_t)s->T * s->d > (1ll << 38)) return MOE_ERR_SHAPE;
    return MOE_OK;
}
// What every call that moves tokens has to be given: the token's side (rows ld apart), the rows' side and the table.
int check_move(const moe_dispatch_shape_t& s, const void* tokens, int64_t ld, const void* rows, int f32, const int32_t* row_of) {
    if (f32 != 0 && f32 != 1) return MOE_ERR_ARG;
    if (s.T > 0 && (!tokens || !row_of || ld < s.d || ld % 8 != 0 || ld > (1ll << 40) / s.T)) return MOE_ERR_ARG;
    if (s.T > 0 && s.rows > 0 && !rows) return MOE_ERR_ARG;
    return aligned(tokens, 16) && aligned(rows, 16) && aligned(row_of, 4) ? MOE_OK : MOE_ERR_ARG;
}
int check_packed(const moe_shape_t* s, const moe_routing_t* r, const void* saved, const void* codes, const void* scales) {
    const int rc = check_shape(s);
    if (rc != MOE_OK) return rc;
    if (!r || !r->offsets || !aligned(r->offsets, 4)) return MOE_ERR_ARG;
    if (s->T > 0 && (!saved || !codes || !scales)) return MOE_ERR_ARG;
    return aligned(saved, 256) && aligned(codes, 16) && aligned(scales, 4) ? MOE_OK : MOE_ERR_ARG;
}
int check_mx(int64_t rows, int K) {
    if (rows < 0 || rows >= (1ll << 31) || K < 8 || K > 1 << 16 || K % 8 != 0 || rows * K > (1ll << 36)) return MOE_ERR_SHAPE;
    return MOE_OK;
}
int check_mx_shape(const moe_mx_shape_t* s) {
    if (!s) return MOE_ERR_ARG;
    if (s->rows < 0 || s->rows >= 1 << 30 || s->experts < 1 || s->experts > kMaxExperts) return MOE_ERR_SHAPE;
    for (int width : {s->K, s->N})
        if (width < 8 || width > 1 << 16 || width % 8 != 0 || (int64_t)s->rows * width > (1ll << 36)) return MOE_ERR_SHAPE;
    return (int64_t)s->experts * s->N * s->K > (1ll << 40) ? MOE_ERR_SHAPE : MOE_OK;
}
bool bad_mx(const void* codes, const void* scales, bool any) { return (any && (!codes || !scales)) || !aligned(codes, 16) || !aligned(scales, 16); }

// What both products have to be given; any: there are rows.
int check_mx_operands(const moe_mx_shape_t& s, const void* a_codes, const void* a_scales, int64_t a_rows, const int32_t* perm, int k, const void* w_codes,
                      const void* w_scales, const int32_t* offsets) {
    if (a_rows < 0 || a_rows >= (1ll << 31) || a_rows * ((s.K + 127) / 128 * 128) > (1ll << 36)) return MOE_ERR_SHAPE;   // (a row's scales begin below 2^32)
    if (k < 1 || (perm ? s.rows > 0 && a_rows == 0 : a_rows < s.rows)) return MOE_ERR_ARG;
    if (bad_mx(a_codes, a_scales, s.rows > 0) || bad_mx(w_codes, w_scales, true) || !offsets) return MOE_ERR_ARG;
    return aligned(perm, 4) && aligned(offsets, 4) ? MOE_OK : MOE_ERR_ARG;
}

struct SavedLayout {
    size_t gu, h, o, total;
};
SavedLayout saved_layout(const moe_shape_t& s) {
    const size_t A_cap = (size_t)s.T * s.k;
    SavedLayout L;
    size_t off = 0;
    L.gu = off; off = align_up(off + A_cap * 2 * s.I * 2, 256);
    L.h = off;  off = align_up(off + A_cap * s.I * 2, 256);
    L.o = off;  off = align_up(off + A_cap * s.d * 2, 256);
    L.total = off > 0 ? off : 256;
    return L;
}

}  // namespace

// Plain streaming copy with known HBM traffic (profiler counter calibration).
__global__ void __launch_bounds__(256) calibration_copy_kernel(uniep::u32x4_t* __restrict__ dst,
                                                               const uniep::u32x4_t* __restrict__ src,
                                                               size_t n16) {
    const size_t stride = (size_t)gridDim.x * blockDim.x;
    for (size_t i = (size_t)blockIdx.x * blockDim.x + threadIdx.x; i < n16; i += stride)
        __builtin_nontemporal_store(__builtin_nontemporal_load(src + i), dst + i);
}

// Dependent-free bf16 MFMA stream with non-trivial operands: what the matrix pipes sustain
// when nothing else runs (profiler and bench calibration of the matrix-core ceiling and of
// the shader clock under that load).  clk[0] = shader clocks, clk[1] = 100 MHz ticks that the
// first wave of workgroup 0 spent in the loop.
__global__ void __launch_bounds__(512) calibration_mfma_kernel(int iters, const uint32_t* __restrict__ seed,
                                                               float* __restrict__ sink, long long* clk) {
    using namespace uniep;
    u32x4_t ar, br;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        ar[i] = seed[(threadIdx.x * 4 + i) & 1023];
        br[i] = seed[(threadIdx.x * 4 + i + 512) & 1023];
    }
    const bf16x8_t a = __builtin_bit_cast(bf16x8_t, ar), b = __builtin_bit_cast(bf16x8_t, br);
    f32x16_t acc[8];
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int v = 0; v < 16; ++v) acc[j][v] = 0.f;
    const long long c0 = clock64(), w0 = wall_clock64();
    for (int it = 0; it < iters; ++it) {
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, acc[j], 0, 0, 0);
    }
    const long long c1 = clock64(), w1 = wall_clock64();
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int v = 0; v < 16; ++v) s += acc[j][v];
    if (s == 0.12345f) sink[0] = s;   // keeps the accumulators alive
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        clk[0] = c1 - c0;
        clk[1] = w1 - w0;
    }
}

__global__ void clear_status_kernel(int* ws) { ws[uniep::CTRL_STATUS] = 0; }

extern "C" {

int moe_calibration_copy(void* dst, const void* src, size_t bytes, void* stream) {
    if (!dst || !src || ((uintptr_t)dst & 15) || ((uintptr_t)src & 15) || (bytes & 15)) return MOE_ERR_ARG;
    if (bytes == 0) return MOE_OK;
    const size_t n16 = bytes / 16;
    const int grid = (int)std::min<size_t>((n16 + 255) / 256, 256 * 16);
    hipLaunchKernelGGL(calibration_copy_kernel, dim3(grid), dim3(256), 0, (hipStream_t)stream,
                       (uniep::u32x4_t*)dst, (const uniep::u32x4_t*)src, n16);
    return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP;
}

int moe_calibration_mfma(int32_t workgroups, int32_t waves, int32_t iters, const uint32_t* seed,
                         float* sink, long long* clocks, void* stream) {
    if (!seed || !sink || !clocks || ((uintptr_t)seed & 3) || ((uintptr_t)clocks & 7)) return MOE_ERR_ARG;
    if (workgroups < 1 || workgroups > 65536 || waves < 1 || waves > 8 || iters < 1) return MOE_ERR_ARG;
    hipLaunchKernelGGL(calibration_mfma_kernel, dim3(workgroups), dim3(64 * waves), 0, (hipStream_t)stream,
                       iters, seed, sink, clocks);
    return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP;
}

int moe_workspace_bytes(const moe_shape_t* shape, size_t* route_ws, size_t* fwd_ws, size_t* bwd_ws,
                        size_t* saved_bytes) {
    int rc = check_shape(shape);
    if (rc != MOE_OK) return rc;
    if (route_ws) *route_ws = route_workspace_bytes(*shape);
    if (fwd_ws) *fwd_ws = fwd_workspace_bytes(*shape);
    if (bwd_ws) *bwd_ws = bwd_workspace_bytes(*shape, 0);
    if (saved_bytes) *saved_bytes = saved_layout(*shape).total;
    return MOE_OK;
}

int moe_backward_workspace_bytes(const moe_shape_t* shape, const moe_opts_t* opts, size_t* bwd_ws) {
    int rc = check_shape(shape);
    if (rc != MOE_OK) return rc;
    moe_opts_t o;
    rc = check_opts(opts, &o);
    if (rc != MOE_OK) return rc;
    if (!bwd_ws || !bwd_split_ok(*shape, o.dw_split_rows)) return MOE_ERR_ARG;
    *bwd_ws = bwd_workspace_bytes(*shape, o.dw_split_rows);
    return MOE_OK;
}

int moe_saved_layout(const moe_shape_t* shape, size_t* off_gu, size_t* off_h, size_t* off_o) {
    int rc = check_shape(shape);
    if (rc != MOE_OK) return rc;
    const SavedLayout L = saved_layout(*shape);
    if (off_gu) *off_gu = L.gu;
    if (off_h) *off_h = L.h;
    if (off_o) *off_o = L.o;
    return MOE_OK;
}

int moe_route(const moe_shape_t* shape, const float* logits, const moe_routing_t* out, void* ws,
              size_t ws_bytes, void* stream) {
    int rc = check_shape(shape);
    if (rc != MOE_OK) return rc;
    rc = check_routing(out, shape->T);
    if (rc != MOE_OK) return rc;
    if (!ws || !aligned(ws, 256)) return MOE_ERR_ARG;
    if (shape->T > 0 && (!logits || !aligned(logits, 4))) return MOE_ERR_ARG;
    if (ws_bytes < route_workspace_bytes(*shape)) return MOE_ERR_WORKSPACE;
    return route_launch(*shape, logits, *out, ws, (hipStream_t)stream);
}

int moe_route_static(const moe_shape_t* shape, const float* logits, const moe_routing_t* out,
                     void* stream) {
    int rc = check_shape(shape);
    if (rc != MOE_OK) return rc;
    rc = check_routing(out, shape->T);
    if (rc != MOE_OK) return rc;
    if (shape->T > 0 && (!logits || !aligned(logits, 4))) return MOE_ERR_ARG;
    if (route_workspace_bytes(*shape) > kRouteStaticScratchBytes) return MOE_ERR_WORKSPACE;
    return route_static_launch(*shape, logits, *out, (hipStream_t)stream);
}

int moe_fused_forward(const moe_shape_t* shape, const void* x, const void* w_gate, const void* w_up,
                      const void* w_down, const moe_routing_t* routing, void* y, void* saved,
                      void* ws, size_t ws_bytes, const moe_opts_t* opts, void* stream) {
    int rc = check_layer_shape(shape);
    if (rc != MOE_OK) return rc;
    rc = check_routing(routing, shape->T);
    if (rc != MOE_OK) return rc;
    moe_opts_t o;
    rc = check_opts(opts, &o);
    if (rc != MOE_OK) return rc;
    if (!w_gate || !w_up || !w_down || !ws) return MOE_ERR_ARG;
    if (shape->T > 0 && (!x || !y)) return MOE_ERR_ARG;
    if (!aligned(x, 16) || !aligned(y, 16) || !aligned(w_gate, 16) || !aligned(w_up, 16) ||
        !aligned(w_down, 16) || !aligned(ws, 256) || !aligned(saved, 256))
        return MOE_ERR_ARG;
    if (ws_bytes < fwd_workspace_bytes(*shape)) return MOE_ERR_WORKSPACE;
    if (shape->T == 0) {   // nothing to compute: leave a clean status word for moe_device_status
        hipLaunchKernelGGL(clear_status_kernel, dim3(1), dim3(1), 0, (hipStream_t)stream, (int*)ws);
        return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP;
    }
    char* wsb = (char*)ws;
    char *gu = nullptr, *h, *ob;
    if (saved) {
        const SavedLayout L = saved_layout(*shape);
        gu = (char*)saved + L.gu;
        h = (char*)saved + L.h;
        ob = (char*)saved + L.o;
    } else {
        const size_t A_cap = (size_t)shape->T * shape->k;
        const size_t ctrl = fwd_ctrl_bytes(*shape);
        h = wsb + ctrl;
        ob = h + align_up(A_cap * shape->I * 2, 256);
    }
    return fwd_launch(*shape, x, w_gate, w_up, w_down, *routing, y, gu, h, ob, wsb, o,
                      (hipStream_t)stream);
}

int moe_fused_backward(const moe_shape_t* shape, const void* dy, const void* x, const void* w_gate,
                       const void* w_up, const void* w_down, const moe_routing_t* routing,
                       const void* saved, void* dx, void* dw_gate, void* dw_up, void* dw_down,
                       float* dtopk_w, void* ws, size_t ws_bytes, const moe_opts_t* opts,
                       void* stream) {
    int rc = check_layer_shape(shape);
    if (rc != MOE_OK) return rc;
    rc = check_routing(routing, shape->T);
    if (rc != MOE_OK) return rc;
    moe_opts_t o;
    rc = check_opts(opts, &o);
    if (rc != MOE_OK) return rc;
    if (!w_gate || !w_up || !w_down || !ws || !saved || !dw_gate || !dw_up || !dw_down)
        return MOE_ERR_ARG;
    if (shape->T > 0 && (!x || !dy || !dx)) return MOE_ERR_ARG;
    if (!aligned(x, 16) || !aligned(dy, 16) || !aligned(dx, 16) || !aligned(w_gate, 16) ||
        !aligned(w_up, 16) || !aligned(w_down, 16) || !aligned(dw_gate, 16) ||
        !aligned(dw_up, 16) || !aligned(dw_down, 16) || !aligned(ws, 256) ||
        !aligned(saved, 256) || !aligned(dtopk_w, 4))
        return MOE_ERR_ARG;
    if (!bwd_split_ok(*shape, o.dw_split_rows)) return MOE_ERR_ARG;
    if (ws_bytes < bwd_workspace_bytes(*shape, o.dw_split_rows)) return MOE_ERR_WORKSPACE;
    const SavedLayout L = saved_layout(*shape);
    const char* sv = (const char*)saved;
    return bwd_launch(*shape, dy, x, w_gate, w_up, w_down, *routing, sv + L.gu, sv + L.h, sv + L.o,
                      dx, dw_gate, dw_up, dw_down, dtopk_w, (char*)ws, o,
                      (hipStream_t)stream);
}

int moe_route_backward(const moe_shape_t* shape, const int32_t* topk_idx, const float* topk_w,
                       const float* dtopk_w, float* dlogits, void* stream) {
    int rc = check_shape(shape);
    if (rc != MOE_OK) return rc;
    if (shape->T > 0 && (!topk_idx || !topk_w || !dtopk_w || !dlogits)) return MOE_ERR_ARG;
    if (!aligned(topk_idx, 4) || !aligned(topk_w, 4) || !aligned(dtopk_w, 4) || !aligned(dlogits, 4))
        return MOE_ERR_ARG;
    return route_backward_launch(*shape, topk_idx, topk_w, dtopk_w, dlogits, (hipStream_t)stream);
}

int moe_global_map(const moe_shape_t* shape, int32_t W, int32_t rank, const moe_routing_t* routing,
                   const int32_t* c_all, const moe_global_map_t* out, void* ws, size_t ws_bytes,
                   void* stream) {
    int rc = check_shape(shape);
    if (rc != MOE_OK) return rc;
    if (shape->e_start != 0 || shape->e_count != shape->E) return MOE_ERR_SHAPE;
    if (W < 1 || W > 64 || shape->E % W != 0 || rank < 0 || rank >= W) return MOE_ERR_SHAPE;
    if (!routing || !out || !c_all || !ws) return MOE_ERR_ARG;
    if (!routing->offsets || !out->recv_offsets) return MOE_ERR_ARG;
    if (shape->T > 0 && (!routing->topk_idx || !routing->inv_perm || !out->dst_rank ||
                         !out->dst_expert || !out->dst_off || !out->dst_row || !out->send ||
                         !out->n_dst_ranks))
        return MOE_ERR_ARG;
    const void* ptrs[] = {routing->topk_idx, routing->inv_perm, routing->offsets, c_all,
                          out->dst_rank, out->dst_expert, out->dst_off, out->dst_row, out->send,
                          out->n_dst_ranks, out->recv_offsets, ws};
    for (const void* q : ptrs)
        if (!aligned(q, 4)) return MOE_ERR_ARG;
    if (ws_bytes < (size_t)shape->E * 8) return MOE_ERR_WORKSPACE;
    return global_map_launch(*shape, W, rank, *routing, c_all, *out, ws, (hipStream_t)stream);
}

int moe_adapter_workspace_bytes(const moe_adapter_shape_t* shape, size_t* ws_bytes, size_t* plan_bytes) {
    const int rc = check_adapter_shape(shape);
    if (rc != MOE_OK) return rc;
    if (ws_bytes) *ws_bytes = adapter_workspace_bytes(*shape);
    if (plan_bytes) *plan_bytes = adapter_plan_bytes(*shape);
    return MOE_OK;
}

int moe_adapter_plan(const moe_adapter_shape_t* shape, const int32_t* ids, void* plan, size_t plan_bytes, void* stream) {
    const int rc = check_adapter_shape(shape);
    if (rc != MOE_OK) return rc;
    // a plan that is given is filled or refused, also where this shape's own calls do without: those of a wider one may read it
    const size_t need = adapter_table_bytes(*shape);
    if (need == 0 || (!plan && adapter_plan_bytes(*shape) == 0)) return MOE_OK;
    if (!ids || !plan || !aligned(ids, 4) || !aligned(plan, 16)) return MOE_ERR_ARG;
    if (plan_bytes < need) return MOE_ERR_WORKSPACE;
    return adapter_plan_launch(*shape, ids, plan, (hipStream_t)stream);
}

int moe_adapter_forward(const moe_adapter_shape_t* shape, const void* x, int64_t ldx, const void* w, const void* a, const void* b,
                        const float* scale, const int32_t* ids, const void* plan, void* y, int32_t out_f32, float* h, void* ws,
                        size_t ws_bytes, void* stream) {
    int rc = check_adapter_shape(shape);
    if (rc != MOE_OK) return rc;
    if (bad_rows(*shape, x, ldx, shape->K) || (out_f32 != 0 && out_f32 != 1)) return MOE_ERR_ARG;
    if ((shape->T > 0 && !y) || !aligned(y, 16) || !aligned(h, 16)) return MOE_ERR_ARG;
    rc = check_adapter(*shape, w, a, b, scale, ids, plan, ws, ws_bytes);
    if (rc != MOE_OK) return rc;
    return adapter_forward_launch(*shape, x, (size_t)ldx, w, a, b, scale, ids, (void*)plan, y, out_f32, h, (char*)ws, (hipStream_t)stream);
}

int moe_adapter_backward(const moe_adapter_shape_t* shape, const void* dy, int64_t lddy, const void* x, int64_t ldx, const void* w,
                         const void* a, const void* b, const float* scale, const int32_t* ids, const void* plan, const float* h,
                         void* dx, float* da, float* db, void* ws, size_t ws_bytes, void* stream) {
    int rc = check_adapter_shape(shape);
    if (rc != MOE_OK) return rc;
    if (bad_rows(*shape, dy, lddy, shape->N) || bad_rows(*shape, x, ldx, shape->K)) return MOE_ERR_ARG;
    if (!da || !db || (shape->T > 0 && (!dx || !h))) return MOE_ERR_ARG;
    if (!aligned(dx, 16) || !aligned(da, 16) || !aligned(db, 16) || !aligned(h, 16)) return MOE_ERR_ARG;
    rc = check_adapter(*shape, w, a, b, scale, ids, plan, ws, ws_bytes);
    if (rc != MOE_OK) return rc;
    return adapter_backward_launch(*shape, dy, (size_t)lddy, x, (size_t)ldx, w, a, b, scale, ids, (void*)plan, h, dx, da, db, (char*)ws,
                                   (hipStream_t)stream);
}

int moe_balance_workspace_bytes(const moe_balance_shape_t* shape, size_t* ws_bytes) {
    const int rc = check_balance_shape(shape);
    if (rc != MOE_OK) return rc;
    if (ws_bytes) *ws_bytes = balance_workspace_bytes(*shape);
    return MOE_OK;
}

int moe_balance_forward(const moe_balance_shape_t* shape, const float* logits, const int32_t* topk_idx, const int32_t* seq_offsets,
                        const uint8_t* mask, const moe_balance_stats_t* out, void* ws, size_t ws_bytes, void* stream) {
    int rc = check_balance_shape(shape);
    if (rc != MOE_OK) return rc;
    rc = check_balance(*shape, logits, topk_idx, seq_offsets, out);
    if (rc != MOE_OK) return rc;
    if (!out->loss || !out->prob_sums || !aligned(out->loss, 4) || !aligned(out->prob_sums, 4) || !ws || !aligned(ws, 256)) return MOE_ERR_ARG;
    if (ws_bytes < balance_workspace_bytes(*shape)) return MOE_ERR_WORKSPACE;
    return balance_forward_launch(*shape, logits, topk_idx, seq_offsets, mask, *out, (char*)ws, (hipStream_t)stream);
}

int moe_balance_backward(const moe_balance_shape_t* shape, const float* logits, const int32_t* topk_idx, const int32_t* seq_offsets,
                         const moe_balance_stats_t* stats, const float* topk_w, const float* dtopk_w, const float* dloss, void* dlogits, int32_t out_bf16, void* stream) {
    int rc = check_balance_shape(shape);
    if (rc != MOE_OK) return rc;
    rc = check_balance(*shape, logits, topk_idx, seq_offsets, stats);
    if (rc != MOE_OK) return rc;
    if ((topk_w == nullptr) != (dtopk_w == nullptr) || !aligned(topk_w, 4) || !aligned(dtopk_w, 4)) return MOE_ERR_ARG;
    if (!dloss || !aligned(dloss, 4) || (out_bf16 != 0 && out_bf16 != 1)) return MOE_ERR_ARG;
    if ((shape->T > 0 && !dlogits) || !aligned(dlogits, out_bf16 ? 2 : 4)) return MOE_ERR_ARG;
    return balance_backward_launch(*shape, logits, topk_idx, seq_offsets, *stats, topk_w, dtopk_w, dloss, dlogits, out_bf16,
                                   (hipStream_t)stream);
}

int moe_dispatch_forward(const moe_dispatch_shape_t* shape, const void* x, int64_t ldx, int32_t f32, const int32_t* row_of, void* xs, void* stream) {
    int rc = check_dispatch_shape(shape);
    if (rc != MOE_OK) return rc;
    rc = check_move(*shape, x, ldx, xs, f32, row_of);
    if (rc != MOE_OK) return rc;
    return dispatch_forward_launch(*shape, x, (size_t)ldx, f32, row_of, xs, (hipStream_t)stream);
}

int moe_dispatch_backward(const moe_dispatch_shape_t* shape, const void* dxs, int32_t f32, const int32_t* row_of, void* dx, void* stream) {
    return moe_combine_forward(shape, dxs, f32, row_of, nullptr, dx, stream);
}

int moe_combine_forward(const moe_dispatch_shape_t* shape, const void* o, int32_t f32, const int32_t* row_of, const float* w, void* y, void* stream) {
    int rc = check_dispatch_shape(shape);
    if (rc != MOE_OK) return rc;
    rc = check_move(*shape, y, shape->d, o, f32, row_of);
    if (rc != MOE_OK) return rc;
    if (!aligned(w, 4)) return MOE_ERR_ARG;
    return combine_forward_launch(*shape, o, f32, row_of, w, y, (hipStream_t)stream);
}

int moe_combine_backward(const moe_dispatch_shape_t* shape, const void* dy, int64_t lddy, const void* o, int32_t f32, const int32_t* row_of, const float* w,
                         void* d_o, float* dw, void* stream) {
    int rc = check_dispatch_shape(shape);
    if (rc != MOE_OK) return rc;
    rc = check_move(*shape, dy, lddy, d_o, f32, row_of);
    if (rc != MOE_OK) return rc;
    if ((dw && shape->T > 0 && shape->rows > 0 && !o) || !aligned(o, 16) || !aligned(w, 4) || !aligned(dw, 4)) return MOE_ERR_ARG;
    return combine_backward_launch(*shape, dy, (size_t)lddy, o, f32, row_of, w, d_o, dw, (hipStream_t)stream);
}

int moe_saved_pack(const moe_shape_t* shape, const moe_routing_t* routing, const void* saved, void* codes, void* scales, void* stream) {
    const int rc = check_packed(shape, routing, saved, codes, scales);
    if (rc != MOE_OK) return rc;
    return saved_pack_launch(*shape, routing->offsets, (const char*)saved + saved_layout(*shape).gu, (uint8_t*)codes, (uint8_t*)scales, (hipStream_t)stream);
}

int moe_saved_unpack(const moe_shape_t* shape, const moe_routing_t* routing, const void* codes, const void* scales, void* saved, void* stream) {
    const int rc = check_packed(shape, routing, saved, codes, scales);
    if (rc != MOE_OK) return rc;
    const SavedLayout L = saved_layout(*shape);
    return saved_unpack_launch(*shape, routing->offsets, (const uint8_t*)codes, (const uint8_t*)scales, (char*)saved + L.gu, (char*)saved + L.h, (hipStream_t)stream);
}

int moe_mx_quantize(const void* x, int64_t ldx, int32_t f32, int64_t rows, int32_t K, void* codes, void* scales, void* stream) {
    const int rc = check_mx(rows, K);
    if (rc != MOE_OK) return rc;
    if ((f32 != 0 && f32 != 1) || bad_mx(codes, scales, rows > 0)) return MOE_ERR_ARG;
    if ((rows > 0 && (!x || ldx < K || ldx % 8 != 0 || ldx > (1ll << 40) / rows)) || !aligned(x, 16)) return MOE_ERR_ARG;
    return mx_quantize_launch(x, (size_t)ldx, f32, rows, K, (uint8_t*)codes, (uint8_t*)scales, (hipStream_t)stream);
}

int moe_mx_quantize_weights(const void* w, int32_t experts, int32_t K, int32_t N, void* codes, void* scales, void* stream) {
    if (experts < 1 || experts > kMaxExperts || N < 8 || N > 1 << 16 || N % 8 != 0) return MOE_ERR_SHAPE;
    const int rc = check_mx((int64_t)experts * N, K);
    if (rc != MOE_OK) return rc;
    if (!w || !aligned(w, 16) || bad_mx(codes, scales, true)) return MOE_ERR_ARG;
    return mx_quantize_weights_launch(w, experts, K, N, (uint8_t*)codes, (uint8_t*)scales, (hipStream_t)stream);
}

int moe_mx_values(const void* codes, const void* scales, int64_t rows, int32_t K, void* out, int32_t out_f32, void* stream) {
    const int rc = check_mx(rows, K);
    if (rc != MOE_OK) return rc;
    if ((out_f32 != 0 && out_f32 != 1) || bad_mx(codes, scales, rows > 0) || (rows > 0 && !out) || !aligned(out, 16)) return MOE_ERR_ARG;
    return mx_values_launch((const uint8_t*)codes, (const uint8_t*)scales, rows, K, out, out_f32, (hipStream_t)stream);
}

int moe_mx_product(const moe_mx_shape_t* shape, const void* a_codes, const void* a_scales, int64_t a_rows, const int32_t* perm, int32_t k, const void* w_codes,
                   const void* w_scales, const int32_t* offsets, void* y, int32_t out_f32, void* stream) {
    int rc = check_mx_shape(shape);
    if (rc != MOE_OK) return rc;
    rc = check_mx_operands(*shape, a_codes, a_scales, a_rows, perm, k, w_codes, w_scales, offsets);
    if (rc != MOE_OK) return rc;
    if ((out_f32 != 0 && out_f32 != 1) || (shape->rows > 0 && !y) || !aligned(y, 16)) return MOE_ERR_ARG;
    return mx_product_launch(*shape, false, (const uint8_t*)a_codes, (const uint8_t*)a_scales, a_rows, perm, k, (const uint8_t*)w_codes, (const uint8_t*)w_scales,
                             nullptr, nullptr, offsets, y, out_f32, nullptr, nullptr, (hipStream_t)stream);
}

int moe_mx_gate_up(const moe_mx_shape_t* shape, const void* a_codes, const void* a_scales, int64_t a_rows, const int32_t* perm, int32_t k, const void* gate_codes,
                   const void* gate_scales, const void* up_codes, const void* up_scales, const int32_t* offsets, void* h, void* h_codes, void* h_scales, void* stream) {
    int rc = check_mx_shape(shape);
    if (rc != MOE_OK) return rc;
    rc = check_mx_operands(*shape, a_codes, a_scales, a_rows, perm, k, gate_codes, gate_scales, offsets);
    if (rc != MOE_OK) return rc;
    if (bad_mx(up_codes, up_scales, true) || !aligned(h, 16) || bad_mx(h_codes, h_scales, false)) return MOE_ERR_ARG;
    if ((h && (h_codes || h_scales)) || (!h_codes != !h_scales) || (shape->rows > 0 && !h && !h_codes)) return MOE_ERR_ARG;
    return mx_product_launch(*shape, true, (const uint8_t*)a_codes, (const uint8_t*)a_scales, a_rows, perm, k, (const uint8_t*)gate_codes, (const uint8_t*)gate_scales,
                             (const uint8_t*)up_codes, (const uint8_t*)up_scales, offsets, h, 0, (uint8_t*)h_codes, (uint8_t*)h_scales, (hipStream_t)stream);
}

int moe_device_status(const void* ws, void* stream) {
    if (!ws) return MOE_ERR_ARG;
    if (hipStreamSynchronize((hipStream_t)stream) != hipSuccess) return MOE_ERR_HIP;
    int status = 0;
    if (hipMemcpy(&status, ws, sizeof(int), hipMemcpyDeviceToHost) != hipSuccess) return MOE_ERR_HIP;
    return status == 0 ? MOE_OK : MOE_ERR_DEVICE;
}

const char* moe_status_string(int code) {
    switch (code) {
        case MOE_OK: return "ok";
        case MOE_ERR_ARG: return "bad argument (null or misaligned pointer, bad option)";
        case MOE_ERR_SHAPE: return "shape outside the supported limits";
        case MOE_ERR_WORKSPACE: return "workspace too small (or the problem exceeds the static scratch of moe_route_static)";
        case MOE_ERR_HIP: return "HIP runtime call failed";
        case MOE_ERR_DEVICE: return "a kernel gave up a bounded scoreboard wait";
        default: return "unknown status";
    }
}

}  // extern "C"
