// C ABI for the single operations (mllm_op_*): argument checks, then the same launchers the
// stage uses.  The attention entry points build their tile lists on the host in pinned staging
// memory (a per-thread ring of slots) and copy them into the caller's workspace on the caller's
// stream, in front of the kernel that reads them.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <cstring>
#include <mutex>
#include <string>
#include <utility>
#include <vector>

#include "../../include/mllm_stage.h"
#include "kernels.h"
#include "attn_items.h"
#include "pinned_ring.h"

using namespace mllm;

namespace {

constexpr size_t ALIGN = 256;
size_t align_up(size_t x) { return (x + ALIGN - 1) / ALIGN * ALIGN; }

}  // namespace

// One thread-local error slot for the whole library; it lives beside mllm_last_error().
namespace mllm_detail { void set_last_error(const char* msg); }

namespace {
mllm_status_t op_fail(mllm_status_t st, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  mllm_detail::set_last_error(buf);
  return st;
}

mllm_status_t check_pack(const mllm_pack_t* p) {
  if (!p || !p->cu_seqlens_host || (p->n_segments > 0 && !p->mask_kind_host)) return op_fail(MLLM_ERR_NULL, "pack or its arrays are NULL");
  if (p->n_segments < 0 || p->total_tokens < 0) return op_fail(MLLM_ERR_SHAPE, "negative sizes");
  if (p->cu_seqlens_host[0] != 0) return op_fail(MLLM_ERR_CU_SEQLENS, "cu_seqlens[0] != 0");
  int longest = 0;
  for (int s = 0; s < p->n_segments; s++) {
    int len = p->cu_seqlens_host[s + 1] - p->cu_seqlens_host[s];
    if (len < 0) return op_fail(MLLM_ERR_CU_SEQLENS, "cu_seqlens decreases at segment %d", s);
    longest = std::max(longest, len);
    if (p->mask_kind_host[s] > 1) return op_fail(MLLM_ERR_MASK_KIND, "mask kind %d at segment %d", (int)p->mask_kind_host[s], s);
  }
  if (p->cu_seqlens_host[p->n_segments] != p->total_tokens) return op_fail(MLLM_ERR_CU_SEQLENS, "cu_seqlens does not end at total_tokens");
  if (p->max_seqlen < longest) return op_fail(MLLM_ERR_SHAPE, "max_seqlen below the longest segment");
  return MLLM_OK;
}

mllm_status_t check_attn(const mllm_pack_t* pack, int32_t hq, int32_t hkv, int32_t hd, int64_t qs,
                         int64_t kvs, int64_t os, const void* ws, size_t ws_bytes) {
  mllm_status_t r = check_pack(pack);
  if (r != MLLM_OK) return r;
  if (hd != 64 && hd != 128) return op_fail(MLLM_ERR_UNSUPPORTED, "head_dim must be 64 or 128");
  if (hq <= 0 || hkv <= 0 || hq % hkv) return op_fail(MLLM_ERR_SHAPE, "n_q_heads must be a positive multiple of n_kv_heads");
  if (qs < (int64_t)hq * hd || kvs < (int64_t)hkv * hd || os < (int64_t)hq * hd || qs % 8 || kvs % 8 || os % 8)
    return op_fail(MLLM_ERR_SHAPE, "row strides too small or not multiples of 8");
  if (!ws) return op_fail(MLLM_ERR_NULL, "workspace is NULL");
  if (ws_bytes < mllm_op_attn_workspace_bytes(pack->n_segments, pack->total_tokens, hq)) return op_fail(MLLM_ERR_WORKSPACE, "attention workspace too small");
  return MLLM_OK;
}

#define OP_TRY(expr)                                                                        \
  do {                                                                                      \
    hipError_t e_ = (expr);                                                                 \
    if (e_ != hipSuccess) return op_fail(MLLM_ERR_HIP, "%s: %s", #expr, hipGetErrorString(e_)); \
  } while (0)

// One ring per host thread (the library keeps no other state between op calls); never freed.
PinnedRing& op_staging() {
  thread_local PinnedRing* ring = new PinnedRing();
  return *ring;
}

// The work lists a call needs (forward: query tiles; backward: key tiles too), one behind the other in one copy.
mllm_status_t upload_tiles(const mllm_pack_t* pack, void* ws, AttnArgs& a, bool backward, hipStream_t stream) {
  char* w = (char*)ws;
  const size_t bytes = align_up(attn_list_bytes(*pack, ATTN_FWD_Q_TILE, a.n_q_heads)) +
                       (backward ? attn_list_bytes(*pack, ATTN_BWD_KV_TILE, a.n_kv_heads) : 0);
  PinnedRing& ring = op_staging();
  PinnedRing::Slot* slot = nullptr;
  OP_TRY(ring.acquire(bytes, &slot));
  char* h = (char*)slot->p;
  a.q_grid = build_attn_list(*pack, ATTN_FWD_Q_TILE, false, a.n_kv_heads, a.n_q_heads / a.n_kv_heads, 64, h);
  size_t used = (size_t)a.q_grid * sizeof(AttnItem);
  const size_t koff = align_up(used);
  if (backward) {
    a.kv_grid = build_attn_list(*pack, ATTN_BWD_KV_TILE, true, a.n_kv_heads, a.n_q_heads / a.n_kv_heads,
                                a.head_dim == 64 ? 64 : 32, h + koff);
    used = koff + (size_t)a.kv_grid * sizeof(AttnItem);
  }
  if (used) OP_TRY(hipMemcpyAsync(w, h, used, hipMemcpyHostToDevice, stream));
  OP_TRY(ring.commit(slot, stream));
  a.q_list = w;
  a.kv_list = w + koff;
  double pairs = 0;
  for (int s = 0; s < pack->n_segments; s++) {
    const double len = pack->cu_seqlens_host[s + 1] - pack->cu_seqlens_host[s];
    pairs += pack->mask_kind_host[s] == MLLM_MASK_CAUSAL ? 0.5 * len * len : len * len;
  }
  a.fwd_flops = 4.0 * pairs * a.n_q_heads * a.head_dim;
  return MLLM_OK;
}

}  // namespace

// Scratch of mllm_op_colsum_static, the entry point for callers that cannot allocate: the fp32
// partial column sums that mllm_op_colsum takes as its `partial` argument live in this array
// instead.  Every GPU the library runs on holds its own copy until the process ends.
constexpr size_t STATIC_SCRATCH_BYTES = (size_t)8 << 20;
static __device__ __align__(256) unsigned char scratch[STATIC_SCRATCH_BYTES];

namespace {
constexpr int MAX_DEVICES = 64;
void* g_scratch_ptr[MAX_DEVICES];       // device address of `scratch` on each device, resolved on first use
std::mutex g_scratch_mutex;

// The array's name is only a host-side handle: its device address on the current device comes
// from hipGetSymbolAddress, once per device.
mllm_status_t static_scratch(void** out) {
  int dev = -1;
  OP_TRY(hipGetDevice(&dev));
  if (dev < 0 || dev >= MAX_DEVICES) return op_fail(MLLM_ERR_UNSUPPORTED, "device index %d beyond %d", dev, MAX_DEVICES);
  std::lock_guard<std::mutex> lock(g_scratch_mutex);
  if (!g_scratch_ptr[dev]) {
    void* p = nullptr;
    OP_TRY(hipGetSymbolAddress(&p, HIP_SYMBOL(scratch)));
    if (!p) return op_fail(MLLM_ERR_HIP, "hipGetSymbolAddress returned a null address");
    g_scratch_ptr[dev] = p;
  }
  *out = g_scratch_ptr[dev];
  return MLLM_OK;
}
}  // namespace

extern "C" {

mllm_status_t mllm_op_gemm(const void* a, const void* b, void* c, int64_t m, int64_t n, int64_t k,
                           int a_layout, int b_layout, int out_fp32, int accumulate,
                           const void* bias, const void* residual, void* hip_stream) {
  if (!a || !b || !c) return op_fail(MLLM_ERR_NULL, "a, b or c is NULL");
  if (m < 0 || n < 0 || k < 0) return op_fail(MLLM_ERR_SHAPE, "negative size");
  if ((a_layout | b_layout) & ~1) return op_fail(MLLM_ERR_SHAPE, "layouts must be 0 or 1");
  const int64_t lda = a_layout ? m : k, ldb = b_layout ? k : n;
  if (lda % 8 || ldb % 8 || n % 8) return op_fail(MLLM_ERR_SHAPE, "contiguous dimensions must be multiples of 8");
  if (out_fp32 && residual) return op_fail(MLLM_ERR_UNSUPPORTED, "residual needs a bf16 output");
  if (!out_fp32 && accumulate) return op_fail(MLLM_ERR_UNSUPPORTED, "accumulate needs an fp32 output");
  GemmArgs g;
  g.a = a; g.b = b; g.c = c; g.m = m; g.n = n; g.k = k; g.lda = lda; g.ldb = ldb; g.ldc = n;
  g.a_layout = a_layout; g.b_layout = b_layout; g.out_fp32 = out_fp32; g.accumulate = accumulate;
  g.bias = bias; g.residual = residual; g.ldres = n;
  g.splitk_ws = nullptr; g.splitk_ws_bytes = 0;
  OP_TRY(launch_gemm(g, (hipStream_t)hip_stream));
  return MLLM_OK;
}

mllm_status_t mllm_gemm_form(int64_t m, int64_t n, int64_t k, int a_layout, int b_layout, size_t scratch_bytes,
                             int32_t* tile_rows, int32_t* tile_cols, int32_t* k_parts) {
  if (m < 0 || n < 0 || k < 0) return op_fail(MLLM_ERR_SHAPE, "negative size");
  if ((a_layout | b_layout) & ~1) return op_fail(MLLM_ERR_SHAPE, "layouts must be 0 or 1");
  GemmArgs g{};
  g.m = m; g.n = n; g.k = k; g.lda = a_layout ? m : k; g.ldb = b_layout ? k : n; g.ldc = n;
  g.a_layout = a_layout; g.b_layout = b_layout;
  g.splitk_ws = scratch_bytes ? &g : nullptr;   // only whether there is any
  g.splitk_ws_bytes = scratch_bytes;
  const GemmForm f = gemm_form(g);
  if (tile_rows) *tile_rows = f.tile_rows;
  if (tile_cols) *tile_cols = f.tile_cols;
  if (k_parts) *k_parts = f.k_parts;
  return MLLM_OK;
}

static void linear_bwd_args(GemmArgs& x, GemmArgs& w, int64_t t, int64_t k, int64_t n) {
  x.m = t; x.n = k; x.k = n; x.lda = n; x.ldb = n; x.ldc = k; x.a_layout = 0; x.b_layout = 1;
  w.m = k; w.n = n; w.k = t; w.lda = k; w.ldb = n; w.ldc = n; w.a_layout = 1; w.b_layout = 0; w.out_fp32 = 1;
}

mllm_status_t mllm_op_linear_bwd(const void* dy, const void* x, const void* w, void* dx, void* dw, int64_t t, int64_t k,
                                 int64_t n, int accumulate, const void* swiglu_pre, void* workspace, size_t scratch_bytes,
                                 void* hip_stream) {
  if (!dy || !x || !w || !dx || !dw) return op_fail(MLLM_ERR_NULL, "a tensor pointer is NULL");
  if (t < 0 || k <= 0 || n <= 0) return op_fail(MLLM_ERR_SHAPE, "sizes must be positive");
  if (k % 8 || n % 8) return op_fail(MLLM_ERR_SHAPE, "widths must be multiples of 8");
  if (scratch_bytes && !workspace) return op_fail(MLLM_ERR_NULL, "workspace is NULL");
  if ((uintptr_t)workspace % ALIGN) return op_fail(MLLM_ERR_WORKSPACE, "the workspace must be 256-byte aligned");
  if (swiglu_pre && !gemm_swiglu_bwd_fusable(t, k, n))
    return op_fail(MLLM_ERR_UNSUPPORTED, "the fused form needs n %% 64 == 0 and at least 200 tiles of 256 x 256");
  GemmArgs gx{}, gw{};
  linear_bwd_args(gx, gw, t, k, n);
  gx.a = dy; gx.b = w; gx.c = dx;
  if (swiglu_pre) { gx.c = nullptr; gx.ldc = 2 * k; gx.swiglu_pre = swiglu_pre; gx.swiglu_dpre = dx; }
  gw.a = x; gw.b = dy; gw.c = dw; gw.accumulate = accumulate;
  gx.splitk_ws = gw.splitk_ws = scratch_bytes ? workspace : nullptr;
  gx.splitk_ws_bytes = gw.splitk_ws_bytes = scratch_bytes;
  OP_TRY(launch_linear_bwd(gx, gw, (hipStream_t)hip_stream));
  return MLLM_OK;
}

mllm_status_t mllm_linear_bwd_form(int64_t t, int64_t k, int64_t n, int swiglu, size_t scratch_bytes, int32_t* form,
                                   size_t* scratch_wanted) {
  if (!form) return op_fail(MLLM_ERR_NULL, "form is NULL");
  if (t < 0 || k <= 0 || n <= 0) return op_fail(MLLM_ERR_SHAPE, "sizes must be positive");
  GemmArgs gx{}, gw{};
  linear_bwd_args(gx, gw, t, k, n);
  if (swiglu) gx.swiglu_dpre = &gx;                          // only whether there is one
  gx.splitk_ws = gw.splitk_ws = scratch_bytes ? &gx : nullptr;   // likewise
  gx.splitk_ws_bytes = gw.splitk_ws_bytes = scratch_bytes;
  const LinearBwdForm f = linear_bwd_form(gx, gw);
  const int32_t v[8] = {f.paired, f.x.tile_rows, f.x.tile_cols, f.x.k_parts, f.w.tile_rows, f.w.tile_cols, f.w.k_parts, f.x_first};
  for (int i = 0; i < 8; i++) form[i] = v[i];
  if (scratch_wanted) *scratch_wanted = linear_bwd_ws_bytes(t, k, n, swiglu != 0);
  return MLLM_OK;
}

mllm_status_t mllm_op_gemm_swiglu(const void* x, const void* w_gu, void* pre, void* act, int64_t m,
                                  int64_t f, int64_t k, void* hip_stream) {
  if (!x || !w_gu || !pre || !act) return op_fail(MLLM_ERR_NULL, "a tensor pointer is NULL");
  if (m < 0 || f <= 0 || k <= 0) return op_fail(MLLM_ERR_SHAPE, "sizes must be positive");
  if (!gemm_swiglu_fusable(m, 2 * f, k))
    return op_fail(MLLM_ERR_UNSUPPORTED, "the fused form needs f a multiple of 128, k a multiple of 64 and at least 200 output tiles of 256 x 256");
  GemmArgs g;
  g.a = x; g.b = w_gu; g.c = pre; g.m = m; g.n = 2 * f; g.k = k; g.lda = k; g.ldb = 2 * f; g.ldc = 2 * f;
  g.a_layout = 0; g.b_layout = 0; g.out_fp32 = 0; g.accumulate = 0;
  g.bias = nullptr; g.residual = nullptr; g.ldres = 0;
  g.splitk_ws = nullptr; g.splitk_ws_bytes = 0;
  g.swiglu_act = act;
  OP_TRY(launch_gemm(g, (hipStream_t)hip_stream));
  return MLLM_OK;
}

mllm_status_t mllm_op_gemm_swiglu_bwd(const void* dy, const void* w_d, const void* pre, void* dpre,
                                      int64_t m, int64_t f, int64_t k, void* hip_stream) {
  if (!dy || !w_d || !pre || !dpre) return op_fail(MLLM_ERR_NULL, "a tensor pointer is NULL");
  if (m < 0 || f <= 0 || k <= 0) return op_fail(MLLM_ERR_SHAPE, "sizes must be positive");
  if (!gemm_swiglu_bwd_fusable(m, f, k))
    return op_fail(MLLM_ERR_UNSUPPORTED, "the fused form needs f a multiple of 8, k a multiple of 64 and at least 200 tiles of 256 x 256 of [m, f]");
  GemmArgs g;
  g.a = dy; g.b = w_d; g.c = nullptr; g.m = m; g.n = f; g.k = k; g.lda = k; g.ldb = k; g.ldc = 2 * f;
  g.a_layout = 0; g.b_layout = 1; g.out_fp32 = 0; g.accumulate = 0;
  g.bias = nullptr; g.residual = nullptr; g.ldres = 0;
  g.splitk_ws = nullptr; g.splitk_ws_bytes = 0;
  g.swiglu_pre = pre; g.swiglu_dpre = dpre;
  OP_TRY(launch_gemm(g, (hipStream_t)hip_stream));
  return MLLM_OK;
}

mllm_status_t mllm_op_rope_table(float* table, int64_t n_pos, int32_t head_dim, float rope_base, void* hip_stream) {
  if (!table) return op_fail(MLLM_ERR_NULL, "table is NULL");
  if (n_pos < 0 || head_dim <= 0 || head_dim % 16 || !(rope_base > 1.f)) return op_fail(MLLM_ERR_SHAPE, "bad rope table geometry");
  OP_TRY(launch_rope_table(table, n_pos, head_dim, rope_base, (hipStream_t)hip_stream));
  return MLLM_OK;
}

mllm_status_t mllm_op_gemm_rope(const void* x, const void* w, const void* bias, void* y, int64_t m, int64_t n,
                                int64_t k, const int32_t* pos, const float* rope_table, int64_t rope_cols,
                                int32_t head_dim, void* hip_stream) {
  if (!x || !w || !y || !pos || !rope_table) return op_fail(MLLM_ERR_NULL, "a pointer is NULL");
  if (m < 0 || n <= 0 || k <= 0 || n % 8 || k % 8) return op_fail(MLLM_ERR_SHAPE, "sizes must be positive, n and k multiples of 8");
  if (rope_cols < 0 || rope_cols > n || rope_cols % 128 || (head_dim != 64 && head_dim != 128))
    return op_fail(MLLM_ERR_SHAPE, "rope_cols must be a multiple of 128 within n, head_dim 64 or 128");
  if (!gemm_rope_fusable(m, n, k, head_dim))
    return op_fail(MLLM_ERR_UNSUPPORTED, "the fused form needs k a multiple of 64 and at least 200 output tiles of 256 x 256");
  GemmArgs g;
  g.a = x; g.b = w; g.c = y; g.m = m; g.n = n; g.k = k; g.lda = k; g.ldb = n; g.ldc = n;
  g.a_layout = 0; g.b_layout = 0; g.out_fp32 = 0; g.accumulate = 0;
  g.bias = bias; g.residual = nullptr; g.ldres = 0;
  g.splitk_ws = nullptr; g.splitk_ws_bytes = 0;
  g.rope_table = rope_table; g.rope_pos = pos; g.rope_cols = rope_cols; g.rope_head_dim = head_dim;
  OP_TRY(launch_gemm(g, (hipStream_t)hip_stream));
  return MLLM_OK;
}

mllm_status_t mllm_attn_work_list(const mllm_pack_t* pack, int32_t kv_major, int32_t n_q_heads, int32_t n_kv_heads,
                                  int32_t head_dim, void* out_host, size_t out_bytes, size_t* bytes_needed,
                                  int32_t* grid_out) {
  mllm_status_t r = check_pack(pack);
  if (r != MLLM_OK) return r;
  if (head_dim != 64 && head_dim != 128) return op_fail(MLLM_ERR_UNSUPPORTED, "head_dim must be 64 or 128");
  if (n_q_heads <= 0 || n_kv_heads <= 0 || n_q_heads % n_kv_heads) return op_fail(MLLM_ERR_SHAPE, "n_q_heads must be a positive multiple of n_kv_heads");
  const int tile = kv_major ? ATTN_BWD_KV_TILE : ATTN_FWD_Q_TILE;
  const size_t need = attn_list_bytes(*pack, tile, kv_major ? n_kv_heads : n_q_heads);
  if (bytes_needed) *bytes_needed = need;
  if (!out_host) return MLLM_OK;
  if (out_bytes < need) return op_fail(MLLM_ERR_WORKSPACE, "work list needs %zu bytes, %zu given", need, out_bytes);
  const int grid = build_attn_list(*pack, tile, kv_major != 0, n_kv_heads, n_q_heads / n_kv_heads,
                                   kv_major ? (head_dim == 64 ? 64 : 32) : 64, (char*)out_host);
  if (grid_out) *grid_out = grid;
  return MLLM_OK;
}

size_t mllm_op_attn_workspace_bytes(int32_t n_segments, int32_t total_tokens, int32_t n_q_heads) {
  const size_t max_tiles = (size_t)std::max(0, total_tokens) / 128 + (size_t)std::max(0, n_segments) + 1;
  return 2 * align_up((size_t)ATTN_XCDS * sizeof(AttnItem) * max_tiles * (size_t)std::max(1, n_q_heads));
}

mllm_status_t mllm_op_attn_fwd(const void* q, const void* k, const void* v, void* o, float* lse,
                               const mllm_pack_t* pack, int32_t n_q_heads, int32_t n_kv_heads,
                               int32_t head_dim, int64_t q_stride, int64_t kv_stride,
                               int64_t o_stride, void* workspace, size_t workspace_bytes,
                               void* hip_stream) {
  if (!q || !k || !v || !o || !lse) return op_fail(MLLM_ERR_NULL, "a tensor pointer is NULL");
  mllm_status_t r = check_attn(pack, n_q_heads, n_kv_heads, head_dim, q_stride, kv_stride, o_stride, workspace, workspace_bytes);
  if (r != MLLM_OK) return r;
  AttnArgs a = {};
  a.q = q; a.k = k; a.v = v; a.o = o; a.lse = lse;
  a.q_stride = q_stride; a.kv_stride = kv_stride; a.o_stride = o_stride;
  a.total_tokens = pack->total_tokens; a.n_q_heads = n_q_heads; a.n_kv_heads = n_kv_heads; a.head_dim = head_dim;
  if ((r = upload_tiles(pack, workspace, a, false, (hipStream_t)hip_stream)) != MLLM_OK) return r;
  OP_TRY(launch_attn_fwd(a, (hipStream_t)hip_stream));
  return MLLM_OK;
}

mllm_status_t mllm_op_attn_bwd(const void* q, const void* k, const void* v, const void* o,
                               const float* lse, const void* d_o, void* dq, void* dk, void* dv,
                               float* delta, const mllm_pack_t* pack, int32_t n_q_heads,
                               int32_t n_kv_heads, int32_t head_dim, int64_t q_stride,
                               int64_t kv_stride, int64_t o_stride, void* workspace,
                               size_t workspace_bytes, void* hip_stream) {
  return mllm_op_attn_bwd_rope(q, k, v, o, lse, d_o, dq, dk, dv, delta, pack, n_q_heads, n_kv_heads, head_dim, q_stride,
                               kv_stride, o_stride, nullptr, workspace, workspace_bytes, hip_stream);
}

mllm_status_t mllm_op_attn_bwd_rope(const void* q, const void* k, const void* v, const void* o,
                                    const float* lse, const void* d_o, void* dq, void* dk, void* dv,
                                    float* delta, const mllm_pack_t* pack, int32_t n_q_heads,
                                    int32_t n_kv_heads, int32_t head_dim, int64_t q_stride,
                                    int64_t kv_stride, int64_t o_stride, const float* rope_table,
                                    void* workspace, size_t workspace_bytes, void* hip_stream) {
  if (!q || !k || !v || !o || !lse || !d_o || !dq || !dk || !dv || !delta) return op_fail(MLLM_ERR_NULL, "a tensor pointer is NULL");
  mllm_status_t r = check_attn(pack, n_q_heads, n_kv_heads, head_dim, q_stride, kv_stride, o_stride, workspace, workspace_bytes);
  if (r != MLLM_OK) return r;
  AttnArgs a = {};
  a.q = q; a.k = k; a.v = v; a.o = const_cast<void*>(o); a.lse = const_cast<float*>(lse);
  a.d_o = d_o; a.dq = dq; a.dk = dk; a.dv = dv; a.delta = delta;
  a.rope_table = rope_table;
  a.q_stride = q_stride; a.kv_stride = kv_stride; a.o_stride = o_stride;
  a.total_tokens = pack->total_tokens; a.n_q_heads = n_q_heads; a.n_kv_heads = n_kv_heads; a.head_dim = head_dim;
  if ((r = upload_tiles(pack, workspace, a, true, (hipStream_t)hip_stream)) != MLLM_OK) return r;
  OP_TRY(launch_attn_bwd(a, (hipStream_t)hip_stream));
  return MLLM_OK;
}

mllm_status_t mllm_op_norm_fwd(int kind, const void* x, const void* gamma, const void* beta,
                               void* y, float* stats, int64_t t, int64_t d, float eps,
                               void* hip_stream) {
  if (!x || !gamma || !y || !stats || (kind == 0 && !beta)) return op_fail(MLLM_ERR_NULL, "a pointer is NULL");
  if (kind != 0 && kind != 1) return op_fail(MLLM_ERR_SHAPE, "kind must be 0 or 1");
  if (t < 0 || d <= 0 || d % 8 || d > 8192) return op_fail(MLLM_ERR_SHAPE, "d must be a multiple of 8, at most 8192");
  OP_TRY(launch_norm_fwd(kind, x, gamma, beta, y, stats, t, d, d, eps, (hipStream_t)hip_stream));
  return MLLM_OK;
}

size_t mllm_op_norm_bwd_partial_bytes(int64_t t, int64_t d) {
  return (size_t)norm_bwd_partial_rows(t) * (size_t)d * 4 * 3;
}

mllm_status_t mllm_op_norm_bwd(int kind, const void* dy, const void* x, const void* gamma,
                               const float* stats, const void* dres, void* dx, float* dgamma,
                               float* dbeta, int accumulate, float* partial, int64_t t, int64_t d,
                               void* hip_stream) {
  if (!dy || !x || !gamma || !stats || !dx || !dgamma || !partial || (kind == 0 && !dbeta)) return op_fail(MLLM_ERR_NULL, "a pointer is NULL");
  if (kind != 0 && kind != 1) return op_fail(MLLM_ERR_SHAPE, "kind must be 0 or 1");
  if (t < 0 || d <= 0 || d % 8 || d > 8192) return op_fail(MLLM_ERR_SHAPE, "d must be a multiple of 8, at most 8192");
  PartialSums sums(partial, mllm_op_norm_bwd_partial_bytes(t, d), accumulate);
  OP_TRY(launch_norm_bwd(kind, dy, x, gamma, stats, dres, dx, dgamma, dbeta, sums, t, d, d, (hipStream_t)hip_stream));
  OP_TRY(sums.flush((hipStream_t)hip_stream));
  return MLLM_OK;
}

mllm_status_t mllm_op_norm_bwd_colsum(int kind, const void* dy, const void* x, const void* gamma,
                                      const float* stats, const void* dres, void* dx, float* dgamma,
                                      float* dbeta, float* dx_colsum, int accumulate, float* partial,
                                      int64_t t, int64_t d, void* hip_stream) {
  if (!dy || !x || !gamma || !stats || !dx || !dgamma || !dx_colsum || !partial || (kind == 0 && !dbeta))
    return op_fail(MLLM_ERR_NULL, "a pointer is NULL");
  if (kind != 0 && kind != 1) return op_fail(MLLM_ERR_SHAPE, "kind must be 0 or 1");
  if (t < 0 || d <= 0 || d % 8 || !norm_bwd_colsum_fusable(d))
    return op_fail(MLLM_ERR_SHAPE, "d must be a multiple of 8, at most 1024");
  PartialSums sums(partial, mllm_op_norm_bwd_partial_bytes(t, d), accumulate);
  OP_TRY(launch_norm_bwd(kind, dy, x, gamma, stats, dres, dx, dgamma, dbeta, sums, t, d, d, (hipStream_t)hip_stream, dx_colsum));
  OP_TRY(sums.flush((hipStream_t)hip_stream));
  return MLLM_OK;
}

mllm_status_t mllm_op_rope(void* qk, const int32_t* pos, int64_t t, int64_t row_stride,
                           int64_t col0, int32_t n_heads, int32_t head_dim, float rope_base,
                           int inverse, void* hip_stream) {
  if (!qk || !pos) return op_fail(MLLM_ERR_NULL, "a pointer is NULL");
  if (t < 0 || n_heads < 0 || head_dim <= 0 || head_dim % 16 || row_stride % 8 || col0 % 8 ||
      col0 + (int64_t)n_heads * head_dim > row_stride)
    return op_fail(MLLM_ERR_SHAPE, "bad rope geometry");
  OP_TRY(launch_rope(qk, pos, t, row_stride, col0, n_heads, head_dim, rope_base, inverse, (hipStream_t)hip_stream));
  return MLLM_OK;
}

mllm_status_t mllm_op_act_fwd(int act, const void* pre, void* a, int64_t t, int64_t f, void* hip_stream) {
  if (!pre || !a) return op_fail(MLLM_ERR_NULL, "a pointer is NULL");
  if (act < 0 || act > 2 || t < 0 || f <= 0 || f % 8) return op_fail(MLLM_ERR_SHAPE, "bad activation arguments");
  OP_TRY(launch_act_fwd(act, pre, a, t, f, (hipStream_t)hip_stream));
  return MLLM_OK;
}

mllm_status_t mllm_op_act_bwd(int act, const void* da, const void* pre, void* dpre, int64_t t, int64_t f, void* hip_stream) {
  if (!da || !pre || !dpre) return op_fail(MLLM_ERR_NULL, "a pointer is NULL");
  if (act < 0 || act > 2 || t < 0 || f <= 0 || f % 8) return op_fail(MLLM_ERR_SHAPE, "bad activation arguments");
  OP_TRY(launch_act_bwd(act, da, pre, dpre, t, f, (hipStream_t)hip_stream));
  return MLLM_OK;
}

// What a caller provides (and what the static scratch must hold): a row of sums for every four tokens, at most
// 512.  The kernel takes one for every 16 (colsum_partial_rows).
size_t mllm_op_colsum_partial_bytes(int64_t t, int64_t n) {
  return (size_t)std::max<int64_t>(1, std::min<int64_t>(512, t / 4)) * (size_t)n * 4;
}

mllm_status_t mllm_op_colsum(const void* x, float* out, int accumulate, float* partial, int64_t t, int64_t n, void* hip_stream) {
  if (!x || !out || !partial) return op_fail(MLLM_ERR_NULL, "a pointer is NULL");
  if (t < 0 || n <= 0 || n % 8) return op_fail(MLLM_ERR_SHAPE, "n must be a positive multiple of 8");
  PartialSums sums(partial, mllm_op_colsum_partial_bytes(t, n), accumulate);
  OP_TRY(launch_colsum(x, n, out, sums, t, n, (hipStream_t)hip_stream));
  OP_TRY(sums.flush((hipStream_t)hip_stream));
  return MLLM_OK;
}

size_t mllm_op_colsum_static_max_bytes(void) { return STATIC_SCRATCH_BYTES; }

mllm_status_t mllm_op_colsum_static(const void* x, float* out, int accumulate, int64_t t, int64_t n, void* hip_stream) {
  if (!x || !out) return op_fail(MLLM_ERR_NULL, "a pointer is NULL");
  if (t < 0 || n <= 0 || n % 8) return op_fail(MLLM_ERR_SHAPE, "n must be a positive multiple of 8");
  const size_t need = mllm_op_colsum_partial_bytes(t, n);
  if (need > STATIC_SCRATCH_BYTES)
    return op_fail(MLLM_ERR_WORKSPACE, "a [%lld, %lld] column sum needs %zu bytes of partial sums, the static scratch holds %zu",
                   (long long)t, (long long)n, need, STATIC_SCRATCH_BYTES);
  void* partial = nullptr;
  mllm_status_t r = static_scratch(&partial);
  if (r != MLLM_OK) return r;
  // every partial sum the second kernel reads is written by the first: nothing to clear
  PartialSums sums((float*)partial, need, accumulate);
  OP_TRY(launch_colsum(x, n, out, sums, t, n, (hipStream_t)hip_stream));
  OP_TRY(sums.flush((hipStream_t)hip_stream));
  return MLLM_OK;
}

// What the entry points of the token side ask of a matrix: rows that the 16-byte accesses can take.
static mllm_status_t check_rows(const char* name, const void* p, int64_t width, int64_t stride) {
  if (stride < width || stride % 8) return op_fail(MLLM_ERR_SHAPE, "%s: row stride below its width or not a multiple of 8", name);
  if ((uintptr_t)p % 16) return op_fail(MLLM_ERR_UNSUPPORTED, "%s must start on 16 bytes", name);
  return MLLM_OK;
}
#define CHECK(expr)                        \
  do {                                     \
    const mllm_status_t r_ = (expr);       \
    if (r_ != MLLM_OK) return r_;          \
  } while (0)
constexpr int64_t MAX_ROWS = INT32_MAX;
// The embedding's tokens and ids: int32 in the kernels' lists, and fewer than 2^32 threads in a launch.
constexpr int64_t MAX_TOKENS = 1 << 30, MAX_VOCAB = 1 << 30, MAX_WIDTH = 1 << 20;

static mllm_status_t check_embed(int64_t t, int64_t vocab, int64_t d) {
  if (t < 0 || t > MAX_TOKENS || vocab <= 0 || vocab > MAX_VOCAB) return op_fail(MLLM_ERR_SHAPE, "t must be in 0 .. 2^30 and vocab in 1 .. 2^30");
  if (d <= 0 || d % 8 || d > MAX_WIDTH) return op_fail(MLLM_ERR_SHAPE, "d must be a positive multiple of 8, at most 2^20");
  return MLLM_OK;
}

mllm_status_t mllm_op_embed_fwd(const void* table, int table_fp32, const int32_t* ids, void* y, int64_t t, int64_t vocab,
                                int64_t d, int64_t y_stride, float scale, void* hip_stream) {
  CHECK(check_embed(t, vocab, d));
  if (!table || (t > 0 && (!ids || !y))) return op_fail(MLLM_ERR_NULL, "table, ids or y is NULL");
  CHECK(check_rows("table", table, d, d));
  CHECK(check_rows("y", y, d, y_stride));
  OP_TRY(launch_embed_fwd(table, table_fp32, ids, y, t, vocab, d, y_stride, scale, (hipStream_t)hip_stream));
  return MLLM_OK;
}

size_t mllm_op_embed_bwd_workspace_bytes(int64_t t, int64_t vocab, int64_t d) {
  return t <= 0 || t > MAX_TOKENS || vocab <= 0 || vocab > MAX_VOCAB || d <= 0 || d > MAX_WIDTH ? 0 : embed_bwd_ws_bytes(t, vocab, d);
}

mllm_status_t mllm_op_embed_bwd(const void* dy, const int32_t* ids, float* dtable, int accumulate, int64_t t, int64_t vocab,
                                int64_t d, int64_t dy_stride, float scale, void* workspace, size_t workspace_bytes,
                                void* hip_stream) {
  CHECK(check_embed(t, vocab, d));
  if (!dtable || (t > 0 && (!ids || !dy))) return op_fail(MLLM_ERR_NULL, "dy, ids or dtable is NULL");
  CHECK(check_rows("dy", dy, d, dy_stride));
  CHECK(check_rows("dtable", dtable, d, d));
  const size_t need = mllm_op_embed_bwd_workspace_bytes(t, vocab, d);
  if (need && !workspace) return op_fail(MLLM_ERR_NULL, "workspace is NULL");
  if ((uintptr_t)workspace % ALIGN) return op_fail(MLLM_ERR_WORKSPACE, "the workspace must be 256-byte aligned");
  if (workspace_bytes < need) return op_fail(MLLM_ERR_WORKSPACE, "workspace has %zu bytes, %zu needed", workspace_bytes, need);
  OP_TRY(launch_embed_bwd(dy, ids, dtable, accumulate, t, vocab, d, dy_stride, scale, workspace, (hipStream_t)hip_stream));
  return MLLM_OK;
}

static bool head_counts_fit(int32_t n_q_heads, int32_t n_kv_heads) {
  return n_q_heads > 0 && n_kv_heads > 0 && n_q_heads <= 65536 && n_kv_heads <= 65536;
}

// x, the other matrix that is read (the forward pass has none) and the one that is written.
static mllm_status_t check_qk_norm(const QkNormArgs& a) {
  if (!a.gamma_q || !a.gamma_k || (a.t > 0 && (!a.x || !a.y || !a.dy))) return op_fail(MLLM_ERR_NULL, "a tensor pointer is NULL");
  if (a.rope_table && a.t > 0 && !a.pos) return op_fail(MLLM_ERR_NULL, "pos is NULL");
  if (a.head_dim <= 0 || a.head_dim % 16 || a.head_dim > 256) return op_fail(MLLM_ERR_UNSUPPORTED, "head_dim must be a multiple of 16, at most 256");
  if (!head_counts_fit(a.n_q_heads, a.n_kv_heads))
    return op_fail(MLLM_ERR_SHAPE, "n_q_heads and n_kv_heads must be positive, at most 65536");
  const int64_t heads = (int64_t)a.n_q_heads + a.n_kv_heads, width = heads * a.head_dim;
  // a lane group of up to 16 a head in whole workgroups of 256, and fewer than 2^32 threads in a launch
  if (a.t < 0 || a.t > MAX_ROWS || a.t * heads > ((int64_t)1 << 28) - 16)
    return op_fail(MLLM_ERR_SHAPE, "t must not be negative, t times the heads at most 2^28 - 16");
  if (!(a.eps >= 0.f)) return op_fail(MLLM_ERR_SHAPE, "eps must not be negative");
  if (a.rope_table && a.n_pos < 0) return op_fail(MLLM_ERR_SHAPE, "n_pos must not be negative");
  CHECK(check_rows("x", a.x, width, a.x_stride));
  CHECK(check_rows("dy", a.dy, width, a.dy_stride));
  CHECK(check_rows("the output", a.y, width, a.y_stride));
  if (((uintptr_t)a.gamma_q | (uintptr_t)a.gamma_k | (uintptr_t)a.rope_table) % 16)
    return op_fail(MLLM_ERR_UNSUPPORTED, "gamma_q, gamma_k and rope_table must start on 16 bytes");
  return MLLM_OK;
}

mllm_status_t mllm_op_qk_norm_rope_fwd(const void* x, const void* gamma_q, const void* gamma_k, void* y, const int32_t* pos,
                                       const float* rope_table, int64_t n_pos, int64_t t, int32_t n_q_heads, int32_t n_kv_heads,
                                       int32_t head_dim, int64_t x_stride, int64_t y_stride, float eps, void* hip_stream) {
  const QkNormArgs a = {x, x, y, gamma_q, gamma_k, pos, rope_table, n_pos, t, x_stride, x_stride, y_stride, n_q_heads, n_kv_heads, head_dim, eps};
  CHECK(check_qk_norm(a));
  OP_TRY(launch_qk_norm_fwd(a, (hipStream_t)hip_stream));
  return MLLM_OK;
}

size_t mllm_op_qk_norm_rope_bwd_partial_bytes(int64_t t, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim) {
  return t < 0 || t > MAX_ROWS || !head_counts_fit(n_q_heads, n_kv_heads) || head_dim <= 0 || head_dim > 256 ? 0 : qk_norm_bwd_partial_floats(t, n_q_heads, n_kv_heads, head_dim) * 4;
}

mllm_status_t mllm_op_qk_norm_rope_bwd(const void* dy, const void* x, const void* gamma_q, const void* gamma_k, void* dx,
                                       float* dgamma_q, float* dgamma_k, int accumulate, float* partial, const int32_t* pos,
                                       const float* rope_table, int64_t n_pos, int64_t t, int32_t n_q_heads, int32_t n_kv_heads,
                                       int32_t head_dim, int64_t dy_stride, int64_t x_stride, int64_t dx_stride, float eps,
                                       void* hip_stream) {
  const QkNormArgs a = {x, dy, dx, gamma_q, gamma_k, pos, rope_table, n_pos, t, x_stride, dy_stride, dx_stride, n_q_heads, n_kv_heads, head_dim, eps};
  if (!dgamma_q || !dgamma_k || !partial) return op_fail(MLLM_ERR_NULL, "dgamma_q, dgamma_k or partial is NULL");
  CHECK(check_qk_norm(a));
  if (((uintptr_t)dgamma_q | (uintptr_t)dgamma_k | (uintptr_t)partial) % 16)
    return op_fail(MLLM_ERR_UNSUPPORTED, "dgamma_q, dgamma_k and partial must start on 16 bytes");
  if (dgamma_q != dgamma_k && ranges_overlap(dgamma_q, (int64_t)head_dim * 4, dgamma_k, (int64_t)head_dim * 4))
    return op_fail(MLLM_ERR_UNSUPPORTED, "dgamma_k may be dgamma_q but not overlap it otherwise");
  PartialSums sums(partial, mllm_op_qk_norm_rope_bwd_partial_bytes(t, n_q_heads, n_kv_heads, head_dim), accumulate);
  OP_TRY(launch_qk_norm_bwd(a, dgamma_q, dgamma_k, sums, (hipStream_t)hip_stream));
  OP_TRY(sums.flush((hipStream_t)hip_stream));
  return MLLM_OK;
}

mllm_status_t mllm_op_xent(const void* logits, int logits_fp32, const int32_t* targets, const float* dloss, float* loss,
                           void* dlogits, int64_t t, int32_t vocab, int32_t cols, int64_t logits_stride, int64_t dlogits_stride,
                           float scale, void* hip_stream) {
  if (t < 0 || t > MAX_ROWS) return op_fail(MLLM_ERR_SHAPE, "t must be in 0 .. 2^31 - 1");
  if (vocab <= 0 || cols < vocab || cols % 8 || cols > (1 << 30)) return op_fail(MLLM_ERR_SHAPE, "vocab must be in 1 .. cols, cols a multiple of 8, at most 2^30");
  if (t > 0 && (!logits || !targets || !loss)) return op_fail(MLLM_ERR_NULL, "logits, targets or loss is NULL");
  CHECK(check_rows("logits", logits, cols, logits_stride));
  if (dlogits) {
    CHECK(check_rows("dlogits", dlogits, cols, dlogits_stride));
    const auto span = [&](int64_t stride, int bytes) {
      return (int64_t)std::min<__int128>(((__int128)(t - 1) * stride + cols) * bytes, INT64_MAX / 4);
    };
    const int64_t in = span(logits_stride, logits_fp32 ? 4 : 2), out = span(dlogits_stride, 2);
    if (t > 0 && ranges_overlap(logits, in, dlogits, out) && (dlogits != logits || logits_fp32 || dlogits_stride != logits_stride))
      return op_fail(MLLM_ERR_UNSUPPORTED, "dlogits may be logits (bf16, same stride) but not overlap them otherwise");
  }
  const XentArgs a = {logits, targets, dloss, loss, dlogits, t, logits_stride, dlogits_stride, vocab, cols, scale};
  OP_TRY(launch_xent(a, logits_fp32, (hipStream_t)hip_stream));
  return MLLM_OK;
}

}  // extern "C"

// Positions of packed text and grids.  The walk over the runs, once to check them and once to launch.
namespace {
template <typename Run>
mllm_status_t walk_positions(int32_t n_segments, const int32_t* cu, int32_t n_grids, const int32_t* grids, int64_t* n_pos, Run run) {
  int64_t most = 0;
  int32_t g = 0;
  for (int32_t s = 0; s < n_segments; s++) {
    if (cu[s + 1] < cu[s]) return op_fail(MLLM_ERR_CU_SEQLENS, "cu_seqlens decreases at segment %d", s);
    int64_t row = cu[s], p = 0;
    const int64_t end = cu[s + 1];
    while (row < end) {
      PositionRun r = {(int32_t)row, (int32_t)p, 0, 1, 0};
      const int32_t* grid = grids + 5 * (int64_t)g;
      int64_t to = end, takes, reaches;
      if (g < n_grids && grid[0] < row) return op_fail(MLLM_ERR_INDEX, "grid %d begins before the end of the one in front of it", g);
      if (g < n_grids && grid[0] == row) {
        const int64_t frames = grid[1], height = grid[2], width = grid[3], step = grid[4];
        if (frames <= 0 || height <= 0 || width <= 0 || step < 0) return op_fail(MLLM_ERR_SHAPE, "grid %d: sizes must be positive, the step not negative", g);
        if (height > end - row || width > end - row || frames > end - row || height * width > end - row || frames * height * width > end - row)
          return op_fail(MLLM_ERR_INDEX, "grid %d goes beyond its segment", g);
        r.frame_rows = (int32_t)(height * width);
        r.width = (int32_t)width;
        r.step = (int32_t)step;
        to = row + frames * height * width;
        takes = reaches = std::max((frames - 1) * step + 1, std::max(height, width));
        g++;
      } else {
        if (g < n_grids && grid[0] < end) to = grid[0];
        takes = reaches = to - row;
      }
      if (p + reaches > INT32_MAX) return op_fail(MLLM_ERR_SHAPE, "segment %d: positions beyond 2^31 - 1", s);
      most = std::max(most, p + reaches);
      const mllm_status_t st = run(r, to);
      if (st != MLLM_OK) return st;
      row = to;
      p += takes;
    }
  }
  if (g < n_grids) return op_fail(MLLM_ERR_INDEX, "grid %d begins outside the sequence or inside a segment's end", g);
  if (n_pos) *n_pos = most;
  return MLLM_OK;
}
mllm_status_t check_positions(int32_t n_segments, const int32_t* cu, int32_t n_grids, const int32_t* grids, int64_t* n_pos) {
  if (!cu || (n_grids > 0 && !grids)) return op_fail(MLLM_ERR_NULL, "cu_seqlens or grids is NULL");
  if (n_segments < 0 || n_grids < 0) return op_fail(MLLM_ERR_SHAPE, "negative sizes");
  if (cu[0] != 0) return op_fail(MLLM_ERR_CU_SEQLENS, "cu_seqlens[0] != 0");
  return walk_positions(n_segments, cu, n_grids, grids, n_pos, [](const PositionRun&, int64_t) { return MLLM_OK; });
}
}  // namespace

extern "C" {

mllm_status_t mllm_grid_positions_count(int32_t n_segments, const int32_t* cu_seqlens_host, int32_t n_grids, const int32_t* grids_host, int64_t* n_pos) {
  if (!n_pos) return op_fail(MLLM_ERR_NULL, "n_pos is NULL");
  return check_positions(n_segments, cu_seqlens_host, n_grids, grids_host, n_pos);
}

mllm_status_t mllm_op_grid_positions(int32_t n_segments, const int32_t* cu_seqlens_host, int32_t n_grids, const int32_t* grids_host,
                                     int32_t* pos, int64_t pos_stride, void* hip_stream) {
  CHECK(check_positions(n_segments, cu_seqlens_host, n_grids, grids_host, nullptr));
  const int64_t rows = cu_seqlens_host[n_segments];
  if (rows > 0 && !pos) return op_fail(MLLM_ERR_NULL, "pos is NULL");
  if (pos_stride < rows) return op_fail(MLLM_ERR_SHAPE, "pos_stride below the sequence's rows");
  PositionRun runs[POSITION_RUNS];
  int count = 0;
  return walk_positions(n_segments, cu_seqlens_host, n_grids, grids_host, nullptr, [&](const PositionRun& r, int64_t to) {
    runs[count++] = r;
    if (count == POSITION_RUNS || to == rows) {
      OP_TRY(launch_grid_positions(runs, count, pos, pos_stride, runs[0].row, (int32_t)(to - runs[0].row), (hipStream_t)hip_stream));
      count = 0;
    }
    return MLLM_OK;
  });
}

mllm_status_t mllm_op_rope_freq_table(float* table, int64_t n_pos, int32_t n_pairs, const double* frequencies_host, void* hip_stream) {
  if (!frequencies_host || (n_pos > 0 && !table)) return op_fail(MLLM_ERR_NULL, "table or frequencies is NULL");
  if (n_pairs <= 0 || n_pairs > ROPE_PAIRS) return op_fail(MLLM_ERR_SHAPE, "n_pairs must be in 1 .. %d", ROPE_PAIRS);
  if (n_pos < 0 || n_pos > MAX_ROWS || n_pos * n_pairs >= (int64_t)1 << 31) return op_fail(MLLM_ERR_SHAPE, "n_pos must not be negative, n_pos times n_pairs below 2^31");
  RopeFrequencies f = {};
  for (int i = 0; i < n_pairs; i++) {
    f.frequency[i] = frequencies_host[i];
    if (!std::isfinite(f.frequency[i])) return op_fail(MLLM_ERR_SHAPE, "frequency %d is not finite", i);
  }
  OP_TRY(launch_rope_freq_table(table, n_pos, n_pairs, f, (hipStream_t)hip_stream));
  return MLLM_OK;
}

// Bytes from a matrix's first element to behind its last one (rows of width, stride apart).
static int64_t span_bytes(int64_t t, int64_t width, int64_t stride, int bytes) {
  return t <= 0 ? 0 : (int64_t)std::min<__int128>(((__int128)(t - 1) * stride + width) * bytes, INT64_MAX / 4);
}

// Whether two matrices share a byte.  Rows of the same stride may lie in one another's gaps: columns of one buffer beside each other.
static bool rows_overlap(const void* a, int64_t a_stride, const void* b, int64_t b_stride, int64_t t, int64_t width, int bytes) {
  if (!ranges_overlap(a, span_bytes(t, width, a_stride, bytes), b, span_bytes(t, width, b_stride, bytes))) return false;
  const __int128 row = (__int128)a_stride * bytes, apart = (uintptr_t)b > (uintptr_t)a ? (uintptr_t)b - (uintptr_t)a : (uintptr_t)a - (uintptr_t)b;
  return a_stride != b_stride || apart % row < width * bytes || row - apart % row < width * bytes;
}

mllm_status_t mllm_op_rope_axes(const void* x, void* y, const int32_t* pos, int64_t pos_stride, int32_t n_axes,
                                const uint8_t* pair_axis_host, int32_t n_pairs, const float* table, int64_t n_pos, int64_t t,
                                int32_t n_heads, int32_t head_dim, int64_t x_stride, int64_t y_stride, int inverse, void* hip_stream) {
  if (!pair_axis_host || !table || (t > 0 && n_heads > 0 && (!x || !y || !pos))) return op_fail(MLLM_ERR_NULL, "a pointer is NULL");
  if (t < 0 || t > MAX_ROWS || n_heads < 0 || n_heads > 65535 || n_pos < 0 || n_pos > MAX_ROWS)
    return op_fail(MLLM_ERR_SHAPE, "t, n_heads and n_pos must not be negative, n_heads at most 65535");
  if (head_dim <= 0 || head_dim % 8 || head_dim > 2 * ROPE_PAIRS) return op_fail(MLLM_ERR_UNSUPPORTED, "head_dim must be a multiple of 8, at most %d", 2 * ROPE_PAIRS);
  if (n_pairs <= 0 || n_pairs % 8 || 2 * n_pairs > head_dim) return op_fail(MLLM_ERR_SHAPE, "n_pairs must be a positive multiple of 8, at most head_dim / 2");
  if (n_axes <= 0 || n_axes > ROPE_AXES) return op_fail(MLLM_ERR_UNSUPPORTED, "n_axes must be in 1 .. %d", ROPE_AXES);
  if (n_axes > 1 && pos_stride < t) return op_fail(MLLM_ERR_SHAPE, "pos_stride below t");
  const int64_t width = (int64_t)n_heads * head_dim;
  CHECK(check_rows("x", x, width, x_stride));
  CHECK(check_rows("y", y, width, y_stride));
  if ((uintptr_t)table % 16) return op_fail(MLLM_ERR_UNSUPPORTED, "table must start on 16 bytes");
  if (rows_overlap(x, x_stride, y, y_stride, t, width, 2) && (x != y || x_stride != y_stride))
    return op_fail(MLLM_ERR_UNSUPPORTED, "y may be x (same stride) but not overlap it otherwise");
  const int64_t result = span_bytes(t, width, y_stride, 2);
  bool over = ranges_overlap(y, result, table, n_pos * n_pairs * 8);
  for (int axis = 0; axis < n_axes; axis++) over |= pos && ranges_overlap(y, result, pos + axis * pos_stride, 4 * t);
  if (over) return op_fail(MLLM_ERR_UNSUPPORTED, "y may not overlap positions or table");
  RopeAxesArgs a = {};
  a.x = x; a.y = y; a.pos = pos; a.pos_stride = pos_stride; a.table = table; a.n_pos = n_pos; a.t = t; a.x_stride = x_stride; a.y_stride = y_stride;
  a.n_heads = n_heads; a.head_dim = head_dim; a.n_pairs = n_pairs;
  for (int i = 0; i < n_pairs; i++) {
    if (pair_axis_host[i] >= n_axes) return op_fail(MLLM_ERR_INDEX, "pair %d follows axis %d of %d", i, (int)pair_axis_host[i], n_axes);
    a.axes[i / 16] |= (uint32_t)pair_axis_host[i] << (2 * (i % 16));
  }
  OP_TRY(launch_rope_axes(a, inverse, (hipStream_t)hip_stream));
  return MLLM_OK;
}

// The residual stream between two blocks.
namespace {
mllm_status_t residual_args(const mllm_residual_norm_t* b, int64_t t, int64_t d, ResidualArgs& a) {
  if (!b) return op_fail(MLLM_ERR_NULL, "block is NULL");
  if (t < 0 || t > MAX_ROWS || d <= 0 || d % 8 || d > 8192) return op_fail(MLLM_ERR_SHAPE, "t must not be negative, d a multiple of 8, at most 8192");
  if (b->post_kind < 0 || b->post_kind > MLLM_NORM_NONE || b->pre_kind < 0 || b->pre_kind > MLLM_NORM_NONE) return op_fail(MLLM_ERR_SHAPE, "norm kind out of range");
  if (b->gate_act < 0 || b->gate_act > MLLM_GATE_SIGMOID) return op_fail(MLLM_ERR_SHAPE, "gate_act out of range");
  const auto used = [](int32_t kind, const void* p, int32_t from) { return kind <= from ? p : nullptr; };
  a.post_kind = b->post_kind; a.pre_kind = b->pre_kind; a.gate_act = b->gate_act; a.gate_per_row = b->gate_per_row != 0 && b->gate;
  a.post_eps = b->post_eps; a.pre_eps = b->pre_eps;
  a.post_g = used(b->post_kind, b->post_g, MLLM_NORM_RMS); a.post_b = used(b->post_kind, b->post_b, MLLM_NORM_LAYER);
  a.pre_g = used(b->pre_kind, b->pre_g, MLLM_NORM_RMS); a.pre_b = used(b->pre_kind, b->pre_b, MLLM_NORM_LAYER);
  a.scale = b->scale; a.gate = b->gate; a.t = t; a.d = (int)d;
  const auto lacks = [](int32_t kind, const void* g, const void* s) { return kind != MLLM_NORM_NONE && (!g || (kind == MLLM_NORM_LAYER && !s)); };
  if (lacks(a.post_kind, a.post_g, a.post_b) || lacks(a.pre_kind, a.pre_g, a.pre_b)) return op_fail(MLLM_ERR_NULL, "a norm's gain or shift is NULL");
  if ((a.post_kind != MLLM_NORM_NONE && !(a.post_eps >= 0.f)) || (a.pre_kind != MLLM_NORM_NONE && !(a.pre_eps >= 0.f)))
    return op_fail(MLLM_ERR_SHAPE, "eps must not be negative");
  if (((uintptr_t)a.post_g | (uintptr_t)a.post_b | (uintptr_t)a.pre_g | (uintptr_t)a.pre_b | (uintptr_t)a.scale) % 16)
    return op_fail(MLLM_ERR_UNSUPPORTED, "gains, shifts and scale must start on 16 bytes");
  return MLLM_OK;
}
struct Range { const void* p; int64_t bytes; };
bool any_overlap(Range a, std::initializer_list<Range> others) {
  for (const Range& b : others)
    if (ranges_overlap(a.p, a.bytes, b.p, b.bytes)) return true;
  return false;
}
// The rows of the statistics that the kinds have.
Range statistics_of(const ResidualArgs& a, const float* stats) {
  const bool post = a.post_kind != MLLM_NORM_NONE, pre = a.pre_kind != MLLM_NORM_NONE;
  return {stats && !post ? stats + 2 * a.t : stats, 8 * a.t * (post + pre)};
}
}  // namespace

mllm_status_t mllm_op_residual_norm_fwd(const mllm_residual_norm_t* block, const void* x, const void* o, void* y, void* n, float* stats,
                                        int64_t t, int64_t d, void* hip_stream) {
  ResidualArgs a;
  CHECK(residual_args(block, t, d, a));
  if (a.pre_kind == MLLM_NORM_NONE) n = nullptr;
  const bool keeps = a.post_kind != MLLM_NORM_NONE || a.pre_kind != MLLM_NORM_NONE;
  if (t > 0 && (!x || !o || !y || (keeps && !stats) || (a.pre_kind != MLLM_NORM_NONE && !n))) return op_fail(MLLM_ERR_NULL, "a tensor pointer is NULL");
  if (((uintptr_t)x | (uintptr_t)o | (uintptr_t)y | (uintptr_t)n) % 16) return op_fail(MLLM_ERR_UNSUPPORTED, "x, o, y and n must start on 16 bytes");
  const int64_t bytes = 2 * t * d;
  const Range in[] = {{x, bytes}, {o, bytes}, {a.post_g, 2 * d}, {a.post_b, 2 * d}, {a.scale, 2 * d}, {a.pre_g, 2 * d}, {a.pre_b, 2 * d}, {a.gate, a.gate_per_row ? 4 * t : 4}};
  const Range out[] = {{y, bytes}, {n, bytes}, statistics_of(a, stats)};
  for (int i = 0; i < 3; i++) {
    for (int j = 0; j < 8; j++)
      if (!(i == 0 && j == 0 && x == y) && any_overlap(out[i], {in[j]}))
        return op_fail(MLLM_ERR_UNSUPPORTED, "y may be x; no other output may overlap an input");
    for (int j = 0; j < i; j++)
      if (any_overlap(out[i], {out[j]})) return op_fail(MLLM_ERR_UNSUPPORTED, "two outputs overlap");
  }
  OP_TRY(launch_residual_fwd(a, x, o, y, n, stats, (hipStream_t)hip_stream));
  return MLLM_OK;
}

size_t mllm_op_residual_norm_bwd_partial_bytes(int64_t t, int64_t d) {
  return t < 0 || t > MAX_ROWS || d <= 0 || d % 8 || d > 8192 ? 0 : residual_bwd_partial_floats(t, d) * 4;
}

mllm_status_t mllm_op_residual_norm_bwd(const mllm_residual_norm_t* block, const void* dn, const void* dy, const void* y, const void* o,
                                        const float* stats, void* dx, void* d_o, const mllm_residual_norm_grads_t* grads, int accumulate,
                                        float* partial, int64_t t, int64_t d, void* hip_stream) {
  ResidualArgs a;
  CHECK(residual_args(block, t, d, a));
  if (!grads) return op_fail(MLLM_ERR_NULL, "grads is NULL");
  const bool pre = a.pre_kind != MLLM_NORM_NONE, post = a.post_kind != MLLM_NORM_NONE;
  if (!pre) dn = y = nullptr;
  if (!partial || (t > 0 && (!o || !dx || !d_o || (pre && (!dn || !y)) || (!pre && !dy) || ((pre || post) && !stats))))
    return op_fail(MLLM_ERR_NULL, "a tensor pointer is NULL");
  if (((uintptr_t)dn | (uintptr_t)dy | (uintptr_t)y | (uintptr_t)o | (uintptr_t)dx | (uintptr_t)d_o | (uintptr_t)partial) % 16)
    return op_fail(MLLM_ERR_UNSUPPORTED, "dn, dy, y, o, dx, d_o and partial must start on 16 bytes");
  ResidualGrads g = {post ? grads->post_g : nullptr, a.post_kind == MLLM_NORM_LAYER ? grads->post_b : nullptr, a.scale ? grads->scale : nullptr,
                     pre ? grads->pre_g : nullptr, a.pre_kind == MLLM_NORM_LAYER ? grads->pre_b : nullptr, a.gate ? grads->gate : nullptr};
  if (((uintptr_t)g.post_g | (uintptr_t)g.post_b | (uintptr_t)g.scale | (uintptr_t)g.pre_g | (uintptr_t)g.pre_b) % 16)
    return op_fail(MLLM_ERR_UNSUPPORTED, "gradients of gains, shifts and scale must start on 16 bytes");
  // Workgroups read what others may have written by then: no output shares a byte with an input or another output, but dx and d_o over the gradients that they come from.
  const int64_t bytes = 2 * t * d, gates = a.gate_per_row ? 4 * t : 4;
  const Range in[] = {{dn, bytes}, {dy, bytes}, {y, bytes}, {o, bytes}, statistics_of(a, stats), {a.post_g, 2 * d}, {a.post_b, 2 * d}, {a.scale, 2 * d},
                      {a.pre_g, 2 * d}, {a.pre_b, 2 * d}, {a.gate, gates}};
  const Range out[] = {{dx, bytes}, {d_o, bytes}, {partial, (int64_t)residual_bwd_partial_floats(t, d) * 4}, {g.post_g, 4 * d}, {g.post_b, 4 * d},
                       {g.scale, 4 * d}, {g.pre_g, 4 * d}, {g.pre_b, 4 * d}, {g.gate, gates}};
  for (int i = 0; i < 9; i++) {
    for (int j = 0; j < 11; j++)
      if (!(i < 2 && j < 2 && out[i].p == in[j].p) && any_overlap(out[i], {in[j]}))
        return op_fail(MLLM_ERR_UNSUPPORTED, "dx and d_o may each be dn or dy; no other output may overlap an input");
    for (int j = 0; j < i; j++)
      if (any_overlap(out[i], {out[j]})) return op_fail(MLLM_ERR_UNSUPPORTED, "two outputs overlap");
  }
  OP_TRY(launch_residual_bwd(a, dn, dy, y, o, stats, dx, d_o, g, accumulate, partial, (hipStream_t)hip_stream));
  return MLLM_OK;
}

// Matrices kept in 8 bits.  Nothing that a call reads or writes beside them may share a byte with them.
static mllm_status_t check_kept(const void* q, const void* exponents, int64_t t, int64_t width, std::initializer_list<Range> others, int64_t parts = 1) {
  if ((uintptr_t)q % 16) return op_fail(MLLM_ERR_UNSUPPORTED, "q must start on 16 bytes");
  const Range values = {q, t * width * parts}, bytes = {exponents, t * ((width + 31) / 32) * parts};
  if (any_overlap(values, {bytes}) || any_overlap(values, others) || any_overlap(bytes, others))
    return op_fail(MLLM_ERR_UNSUPPORTED, "q and exponents may not overlap each other or another tensor");
  return MLLM_OK;
}
static mllm_status_t check_keep8(int64_t t, int64_t width, int format) {
  if (t < 0 || t > MAX_ROWS || width <= 0 || width % 8 || width > ((int64_t)1 << 30)) return op_fail(MLLM_ERR_SHAPE, "t must not be negative, the width a positive multiple of 8, at most 2^30");
  if (format != MLLM_KEEP_INT8 && format != MLLM_KEEP_E4M3) return op_fail(MLLM_ERR_SHAPE, "unknown 8-bit format");
  return MLLM_OK;
}

mllm_status_t mllm_op_keep8(const void* x, void* q, void* exponents, int64_t t, int64_t width, int64_t x_stride, int format, void* hip_stream) {
  CHECK(check_keep8(t, width, format));
  if (t > 0 && (!x || !q || !exponents)) return op_fail(MLLM_ERR_NULL, "x, q or exponents is NULL");
  CHECK(check_rows("x", x, width, x_stride));
  CHECK(check_kept(q, exponents, t, width, {{x, span_bytes(t, width, x_stride, 2)}}));
  OP_TRY(launch_keep8(x, q, exponents, t, width, x_stride, format, (hipStream_t)hip_stream));
  return MLLM_OK;
}

mllm_status_t mllm_op_keep8_load(const void* q, const void* exponents, void* y, int64_t t, int64_t width, int64_t y_stride, int format, void* hip_stream) {
  CHECK(check_keep8(t, width, format));
  if (t > 0 && (!y || !q || !exponents)) return op_fail(MLLM_ERR_NULL, "y, q or exponents is NULL");
  CHECK(check_rows("y", y, width, y_stride));
  CHECK(check_kept(q, exponents, t, width, {{y, span_bytes(t, width, y_stride, 2)}}));
  OP_TRY(launch_keep8_load(q, exponents, y, t, width, y_stride, format, (hipStream_t)hip_stream));
  return MLLM_OK;
}

mllm_status_t mllm_op_act_fwd_keep8(int act, const void* pre, void* a, void* q, void* exponents, int64_t t, int64_t f, int format, void* hip_stream) {
  CHECK(check_keep8(t, f, format));
  if (act < 0 || act > 2) return op_fail(MLLM_ERR_SHAPE, "bad activation arguments");
  if (t > 0 && (!pre || !a || !q || !exponents)) return op_fail(MLLM_ERR_NULL, "pre, a, q or exponents is NULL");
  if (((uintptr_t)pre | (uintptr_t)a) % 16) return op_fail(MLLM_ERR_UNSUPPORTED, "pre and a must start on 16 bytes");
  const int64_t halves = act == 2 ? 2 : 1;
  CHECK(check_kept(q, exponents, t, f, {{pre, 2 * halves * t * f}, {a, 2 * t * f}}, halves));
  if (any_overlap({pre, 2 * halves * t * f}, {{a, 2 * t * f}})) return op_fail(MLLM_ERR_UNSUPPORTED, "a may not overlap pre");
  OP_TRY(launch_act_fwd_keep8(act, pre, a, q, exponents, t, f, format, (hipStream_t)hip_stream));
  return MLLM_OK;
}

mllm_status_t mllm_op_act_bwd_keep8(int act, const void* da, const void* q, const void* exponents, void* dpre, void* a, int64_t t, int64_t f, int format,
                                    void* hip_stream) {
  CHECK(check_keep8(t, f, format));
  if (act < 0 || act > 2) return op_fail(MLLM_ERR_SHAPE, "bad activation arguments");
  if (t > 0 && (!q || !exponents || !da != !dpre || (!da && !a))) return op_fail(MLLM_ERR_NULL, "q, exponents, da, dpre or a is NULL");
  if (((uintptr_t)da | (uintptr_t)dpre | (uintptr_t)a) % 16) return op_fail(MLLM_ERR_UNSUPPORTED, "da, dpre and a must start on 16 bytes");
  const int64_t halves = act == 2 ? 2 : 1;
  CHECK(check_kept(q, exponents, t, f, {{da, 2 * t * f}, {dpre, 2 * halves * t * f}, {a, 2 * t * f}}, halves));
  if (any_overlap({dpre, 2 * halves * t * f}, {{a, 2 * t * f}}) || any_overlap({a, 2 * t * f}, {{da, 2 * t * f}}) ||
      (any_overlap({dpre, 2 * halves * t * f}, {{da, 2 * t * f}}) && (dpre != da || halves == 2)))
    return op_fail(MLLM_ERR_UNSUPPORTED, "dpre may be da for the GELU kinds; nothing else may overlap");
  OP_TRY(launch_act_bwd_keep8(act, da, q, exponents, dpre, a, t, f, format, (hipStream_t)hip_stream));
  return MLLM_OK;
}

// The gradient of x contracts over n, which the tile kernel takes in multiples of 64 alone; other widths go to the general kernel, or here get copies of dy and w with
// columns of zeros, in the launch that loads x.  us without and with the copies: 1 x 1000 x 3000 (t x k x n) 34.8 and 15.8, 777 x 256 x 136 15.5 and 11, 777 x 504 x 3000 45 and 23,
// 777 x 7000 x 7000 273 and 211, 2999 x 4096 x 4104 250 and 185, 5000 x 1000 x 3000 104 and 82, 8192 x 520 x 3000 93 and 85, 16000 x 2048 x 1000 166 and 161, 30000 x 4096 x 4104 1990 and 1620.  Many rows of
// narrow x lose, dy being most of what is read: 16000 x 256 x 136 26.6 and 31.9, 16000 x 72 x 7000 115 and 154 (2999 rows 81 and 38).  The border at 512 columns of x is not
// sharp: 16000 x 520 x 3000 160 and 152, 16000 x 1000 x 3000 188 and 201, 30000 x 520 x 3000 258 and 276, 30000 x 1000 x 3000 364 and 373, 30000 x 600 x 136 63 and 54.
constexpr int64_t PADDED_ROWS = 4096, PADDED_WIDTH = 512;
static bool takes_copies(int64_t t, int64_t k, int64_t n) { return n % 64 != 0 && (t <= PADDED_ROWS || k >= PADDED_WIDTH); }
static int64_t padded(int64_t n) { return (n + 63) / 64 * 64; }
static size_t copies_bytes(int64_t t, int64_t k, int64_t n) { return align_up((size_t)t * padded(n) * 2) + align_up((size_t)k * padded(n) * 2); }

size_t mllm_op_linear_bwd_keep8_workspace_bytes(int64_t t, int64_t k, int64_t n) {
  if (t < 0 || t > MAX_ROWS || k <= 0 || n <= 0 || k > ((int64_t)1 << 30) || n > ((int64_t)1 << 30)) return 0;
  const int64_t rows = k >= PADDED_WIDTH ? t : std::min(t, PADDED_ROWS);   // so that a buffer for more rows has room for the copies of fewer
  return align_up((size_t)t * k * 2) + (n % 64 == 0 ? 0 : copies_bytes(rows, k, n)) +
         std::max(linear_bwd_ws_bytes(t, k, n, false), linear_bwd_ws_bytes(t, k, padded(n), false));
}

mllm_status_t mllm_op_linear_bwd_keep8(const void* dy, const void* q, const void* exponents, const void* w, void* dx, void* dw, int64_t t,
                                       int64_t k, int64_t n, int format, int accumulate, void* workspace, size_t workspace_bytes,
                                       void* hip_stream) {
  CHECK(check_keep8(t, k, format));
  if (!dw || !w || (t > 0 && (!dy || !q || !exponents || !dx))) return op_fail(MLLM_ERR_NULL, "a tensor pointer is NULL");
  if (n <= 0 || n % 8 || n > ((int64_t)1 << 30)) return op_fail(MLLM_ERR_SHAPE, "n must be a positive multiple of 8, at most 2^30");
  for (const auto& e : {std::pair<int64_t, int64_t>(t, k), std::pair<int64_t, int64_t>(t, n), std::pair<int64_t, int64_t>(k, n)})
    if (2 * e.first * e.second > GEMM_MAX_OPERAND_BYTES) return op_fail(MLLM_ERR_SHAPE, "an operand of 4 GiB or more");
  const size_t kept = align_up((size_t)t * k * 2);
  if (kept && !workspace) return op_fail(MLLM_ERR_NULL, "workspace is NULL");
  if ((uintptr_t)workspace % ALIGN) return op_fail(MLLM_ERR_WORKSPACE, "the workspace must be 256-byte aligned");
  if (workspace_bytes < kept) return op_fail(MLLM_ERR_WORKSPACE, "workspace has %zu bytes, %zu needed", workspace_bytes, kept);
  if (((uintptr_t)dy | (uintptr_t)w | (uintptr_t)dx | (uintptr_t)dw) % 16) return op_fail(MLLM_ERR_UNSUPPORTED, "dy, w, dx and dw must start on 16 bytes");
  CHECK(check_kept(q, exponents, t, k, {{dx, 2 * t * k}, {dw, 4 * k * n}, {workspace, (int64_t)workspace_bytes}}));
  const Range rx = {dx, 2 * t * k}, rw = {dw, 4 * k * n}, rs = {workspace, (int64_t)workspace_bytes}, in[2] = {{dy, 2 * t * n}, {w, 2 * k * n}};
  if (any_overlap(rx, {rw, rs, in[0], in[1]}) || any_overlap(rw, {rs, in[0], in[1]}) || any_overlap(rs, {in[0], in[1]}))
    return op_fail(MLLM_ERR_UNSUPPORTED, "dx, dw and workspace may not overlap each other or an input");
  if (t == 0) return mllm_op_linear_bwd(w, w, w, dw, dw, 0, k, n, accumulate, nullptr, nullptr, 0, hip_stream);   // no rows: none of the rows' matrices is touched
  const int64_t wide = padded(n);
  const size_t copies = copies_bytes(t, k, n);
  if (!takes_copies(t, k, n) || workspace_bytes < kept + copies || 2 * std::max(t, k) * wide > GEMM_MAX_OPERAND_BYTES) {
    OP_TRY(launch_keep8_load(q, exponents, workspace, t, k, k, format, (hipStream_t)hip_stream));
    return mllm_op_linear_bwd(dy, workspace, w, dx, dw, t, k, n, accumulate, nullptr, (char*)workspace + kept, workspace_bytes - kept, hip_stream);
  }
  char* dy_padded = (char*)workspace + kept;
  char* w_padded = dy_padded + align_up((size_t)t * wide * 2);
  OP_TRY(launch_linear_operands(q, exponents, workspace, dy, dy_padded, w, w_padded, t, k, n, wide, format, (hipStream_t)hip_stream));
  GemmArgs gx{}, gw{};
  linear_bwd_args(gx, gw, t, k, n);
  gx.a = dy_padded; gx.b = w_padded; gx.c = dx; gx.k = gx.lda = gx.ldb = wide;
  gw.a = workspace; gw.b = dy_padded; gw.c = dw; gw.ldb = wide; gw.accumulate = accumulate;
  gx.splitk_ws_bytes = gw.splitk_ws_bytes = workspace_bytes - kept - copies;
  gx.splitk_ws = gw.splitk_ws = gx.splitk_ws_bytes ? (char*)workspace + kept + copies : nullptr;
  OP_TRY(launch_linear_bwd(gx, gw, (hipStream_t)hip_stream));
  return MLLM_OK;
}

}  // extern "C"
