// The residual stream between two blocks of a layer, in one pass over it:
//   u = post(o) * scale * gate      o the block's output; post LayerNorm, RMSNorm or none; scale of every channel; gate of the block or of every row
//   y = x + u                       the stream, stored as bf16
//   n = pre(y)                      what the next block reads: the norm of the stream as it is stored
// and its gradients.  Bound by memory (32768 x 4096 forward 177 us, 6.1 TB/s): o, x, y and n forward, dn, dy, y, o, dx and the gradient of o backward, each once.
#include <algorithm>

#include "common.h"
#include "kernels.h"
#include "rows.h"

namespace mllm {

namespace {

constexpr int LAYER = 0, RMS = 1, NONE = 2;

__device__ __forceinline__ float gate_value(int act, float v) { return act == 1 ? tanhf(v) : act == 2 ? 1.f / (1.f + expf(-v)) : v; }
__device__ __forceinline__ float gate_slope(int act, float v) {   // from the gate itself: 1 - tanh^2 and s (1 - s) have no digits left where they are small
  if (act == 0) return 1.f;
  const float e = expf(act == 1 ? -2.f * fabsf(v) : -fabsf(v)), r = 1.f / (1.f + e);
  return (act == 1 ? 4.f : 1.f) * e * r * r;
}

// A row belongs to `waves` wavefronts (a lane has eight neighbouring columns, so 512 columns a wavefront), a workgroup to `rows` rows:
// wavefront w of the workgroup is wavefront w % waves of row w / waves.  Sums over a row go through LDS where it has several wavefronts;
// every sum has a slot of its own until the next row but one.
constexpr int MAX_WAVES = 16;
struct RowSums { float part[2][2][3][MAX_WAVES]; };   // [parity][first or second exchange][sum][wavefront]
template <int N>
__device__ __forceinline__ void row_sums(float* v, float (*part)[MAX_WAVES], int waves, int wave, int lane) {
#pragma unroll
  for (int i = 0; i < N; i++) v[i] = over_lanes<64, false>(v[i]);
  if (waves == 1) return;
  if (lane == 0)
#pragma unroll
    for (int i = 0; i < N; i++) part[i][wave] = v[i];
  __syncthreads();
  const int first = wave - wave % waves, k = lane & 15;
#pragma unroll
  for (int i = 0; i < N; i++) v[i] = over_lanes<16, false>(k < waves ? part[i][first + k] : 0.f);
}

// (factor, mean) of a norm over the row's values.  LayerNorm takes two exchanges, the mean and then the squares about it (every wavefront's mean and squares joined in
// one exchange: 5125 x 3200 with LayerNorm on both sides 34.9 us, so 33.1).  per = 1 / d: a division is some ten instructions (33.1 -> 30.3, backward 48.7 -> 45.1).
template <int KIND>
__device__ __forceinline__ void statistics(const float* v, bool there, int d, float per, float eps, float (*part)[3][MAX_WAVES], int waves, int wave, int lane,
                                           float& factor, float& mean) {
  factor = 1.f;
  mean = 0.f;
  if (KIND == NONE) return;
  float sum[1];
  if (KIND == LAYER) {
    sum[0] = 0.f;
#pragma unroll
    for (int e = 0; e < 8; e++) sum[0] += v[e];       // zeros behind the row
    row_sums<1>(sum, part[0], waves, wave, lane);
    mean = sum[0] * per;
    mean = fmaf(fmaf(-mean, (float)d, sum[0]), per, mean);   // the remainder, so that a row of equal values has a mean equal to them
  }
  sum[0] = 0.f;
  if (there)
#pragma unroll
    for (int e = 0; e < 8; e++) {
      const float w = v[e] - mean;
      sum[0] += w * w;
    }
  row_sums<1>(sum, part[1], waves, wave, lane);
  factor = rsqrtf(sum[0] * per + eps);
}

__device__ __forceinline__ void load_vector(const bf16_t* p, int c, bool there, float* f) {
  if (p && there) {
    load8(p + 8 * c, f);
  } else {
#pragma unroll
    for (int e = 0; e < 8; e++) f[e] = 0.f;
  }
}

template <int POST, int PRE, bool PAST>
__global__ __launch_bounds__(1024) void residual_fwd_kernel(ResidualArgs a, const bf16_t* x, const bf16_t* __restrict__ o, bf16_t* y,
                                                            bf16_t* __restrict__ n, float* __restrict__ stats, int waves, int rows) {
  __shared__ RowSums sums[2];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = (wave % waves) * 64 + lane, of = wave / waves;
  const bool column = c < a.d >> 3;
  const int64_t step = (int64_t)gridDim.x * rows;
  uint4 qo, qx;
  float gate_in = 0.f;
  auto fetch = [&](int64_t row) __attribute__((always_inline)) {
    qo = qx = make_uint4(0, 0, 0, 0);
    if (row >= a.t) return;
    if (column) {
      qo = load16_once(o + row * a.d + 8 * c);
      qx = load16_once(x + row * a.d + 8 * c);
    }
    if (a.gate) gate_in = a.gate[a.gate_per_row ? row : 0];
  };
  const int64_t first = (int64_t)blockIdx.x * rows;
  fetch(first + of);
  uint4 pg = make_uint4(0, 0, 0, 0), pb = pg, sc = pg, ng = pg, nb = pg;
  if (column) {
    if (POST != NONE) pg = *reinterpret_cast<const uint4*>((const bf16_t*)a.post_g + 8 * c);
    if (POST == LAYER) pb = *reinterpret_cast<const uint4*>((const bf16_t*)a.post_b + 8 * c);
    if (a.scale) sc = *reinterpret_cast<const uint4*>((const bf16_t*)a.scale + 8 * c);
    if (PRE != NONE) ng = *reinterpret_cast<const uint4*>((const bf16_t*)a.pre_g + 8 * c);
    if (PRE == LAYER) nb = *reinterpret_cast<const uint4*>((const bf16_t*)a.pre_b + 8 * c);
  }
  const float per = 1.f / (float)a.d;
  int parity = 0;
  for (int64_t base = first; base < a.t; base += step, parity ^= 1) {    // all wavefronts alike: they meet at barriers
    const int64_t row = base + of, at = row * a.d + 8 * c;
    const bool there = row < a.t && column;
    const float gate = a.gate ? gate_value(a.gate_act, gate_in) : 1.f;
    float v[8], w[8], g[8], b[8];
    unpack8(qo, v);
    unpack8(qx, w);
    fetch(row + step);
    float factor, mean;
    statistics<POST>(v, there, a.d, per, a.post_eps, sums[parity].part[0], waves, wave, lane, factor, mean);
    if (POST != NONE) {
      unpack8(pg, g);
      unpack8(pb, b);
#pragma unroll
      for (int e = 0; e < 8; e++) v[e] = (v[e] - mean) * factor * g[e] + (POST == LAYER ? b[e] : 0.f);
      if (there && c == 0) {
        stats[row] = factor;
        stats[a.t + row] = mean;
      }
    }
    if (a.scale) {
      unpack8(sc, g);
#pragma unroll
      for (int e = 0; e < 8; e++) v[e] *= g[e];
    }
#pragma unroll
    for (int e = 0; e < 8; e++) w[e] = fmaf(v[e], gate, w[e]);
    const uint4 stored = pack8(w);
    if (there) store16<PAST>(y + at, stored);
    if (PRE == NONE) continue;
    unpack8(stored, w);
    statistics<PRE>(w, there, a.d, per, a.pre_eps, sums[parity].part[1], waves, wave, lane, factor, mean);
    unpack8(ng, g);
    unpack8(nb, b);
#pragma unroll
    for (int e = 0; e < 8; e++) w[e] = (w[e] - mean) * factor * g[e] + (PRE == LAYER ? b[e] : 0.f);
    if (there) {
      store16<PAST>(n + at, pack8(w));
      if (c == 0) {
        stats[2 * a.t + row] = factor;
        stats[3 * a.t + row] = mean;
      }
    }
  }
}

// The gradients that follow from the columns' sums A, B, C, D of N columns from col on; a sum that nobody asked for is never used.
struct FinishArgs {
  const float* partial; const float* gate_partial;
  int W, d, sets, accumulate;
  const bf16_t* post_g; const bf16_t* post_b; const bf16_t* scale;
  ResidualGrads g;
};
// (N columns, a multiple of four, from a multiple of N on.)
template <int N>
__device__ __forceinline__ void put_sums(float* out, const float* v, int64_t col, int accumulate) {
  if (!out) return;
#pragma unroll
  for (int e = 0; e < N; e += 4) {
    float4* o = reinterpret_cast<float4*>(out + col + e);
    const float4 old = accumulate ? *o : make_float4(0.f, 0.f, 0.f, 0.f);
    *o = make_float4(v[e] + old.x, v[e + 1] + old.y, v[e + 2] + old.z, v[e + 3] + old.w);
  }
}
template <int N>
__device__ __forceinline__ void columns_of(const bf16_t* p, int64_t col, float* f, float none) {
#pragma unroll
  for (int e = 0; e < N; e += 4) {
    const uint2 u = p ? *reinterpret_cast<const uint2*>(p + col + e) : make_uint2(0, 0);
    f[e] = p ? bf16lo(u.x) : none; f[e + 1] = p ? bf16hi(u.x) : none; f[e + 2] = p ? bf16lo(u.y) : none; f[e + 3] = p ? bf16hi(u.y) : none;
  }
}
template <int N>
__device__ __forceinline__ void put_post(const FinishArgs& a, const float* A, const float* B, int64_t col) {
  float s[N], g[N], b[N], pg[N], pb[N], sc[N];
  columns_of<N>(a.scale, col, s, 1.f);
  columns_of<N>(a.post_g, col, g, 1.f);
  columns_of<N>(a.post_b, col, b, 0.f);
#pragma unroll
  for (int e = 0; e < N; e++) {
    pg[e] = s[e] * A[e];
    pb[e] = s[e] * B[e];
    sc[e] = a.post_b ? fmaf(g[e], A[e], b[e] * B[e]) : g[e] * A[e];
  }
  put_sums<N>(a.g.post_g, pg, col, a.accumulate);
  put_sums<N>(a.g.post_b, pb, col, a.accumulate);
  put_sums<N>(a.g.scale, sc, col, a.accumulate);
}

// Backward.  With h the stream without mean, times its factor, z the same of o (o itself without a norm), g the gate:
//   dY = dy + pre'(dn),  pre'(dn) = factor * (dn pre_g - mean(dn pre_g) - h mean(dn pre_g h));  dx = dY
//   do = post'(dY g scale post_g), or dY g scale without a norm
// and, summed over the rows, A = dY g z and B = dY g of every column: post_g's gradient is scale A, post_b's scale B, the scale's
// post_g A + post_b B; pre_g's and pre_b's are the sums of dn h and dn.  The gate's is the row's sum of dY post(o) scale times its slope.
// A workgroup goes over rows b, b + B, ...; a lane keeps its columns' sums, which go to `partial`, [set][workgroup][d]; the next row's
// operands are requested before a row is worked on.  32768 x 4096 with RMSNorm on both sides 265 us (6.1 TB/s), 5125 x 3200 (LayerNorm in front, scale, gates) 38 (5.2).
template <int POST, int PRE, bool PAST, int THREADS>
__global__ __launch_bounds__(THREADS) void residual_bwd_kernel(ResidualArgs a, const bf16_t* dn, const bf16_t* dy, const bf16_t* __restrict__ y,
                                                            const bf16_t* __restrict__ o, const float* __restrict__ stats, bf16_t* dx, bf16_t* d_o,
                                                            float* __restrict__ gate_rows, float* __restrict__ partial, int waves, int rows, FinishArgs finish) {
  __shared__ RowSums sums;
  __shared__ float joined_columns[8 * 512];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = (wave % waves) * 64 + lane, of = wave / waves;
  const bool column = c < a.d >> 3;
  const int64_t step = (int64_t)gridDim.x * rows;
  float k[8], A[8], Bs[8], C[8], D[8];   // B and D only where a norm has a shift
  uint4 pg = make_uint4(0, 0, 0, 0);
  if (PRE != NONE && column) pg = *reinterpret_cast<const uint4*>((const bf16_t*)a.pre_g + 8 * c);
  {   // k: what dY g is multiplied by on its way through gain and scale
    float g[8], s[8];
    load_vector((const bf16_t*)a.post_g, c, column, g);
    load_vector((const bf16_t*)a.scale, c, column, s);
#pragma unroll
    for (int e = 0; e < 8; e++) {
      k[e] = (a.post_g ? g[e] : 1.f) * (a.scale ? s[e] : 1.f);
      A[e] = Bs[e] = C[e] = D[e] = 0.f;
    }
  }
  float gate_sum = 0.f;
  const float per = 1.f / (float)a.d;
  const bool reads_o = POST != NONE || (finish.sets & 3) || gate_rows;   // with neither, its gradient follows from dx alone (40000 x 3200 250 -> 217 us)
  // THREADS: what the registers are dealt by.  With LayerNorm behind the block and a norm in front of the next one, 1024 threads have none left for the next row's operands (they
  // spill: us requested ahead and not, LayerNorm on both sides, 16384 x 8192 377 and 323, 2999 x 8192 87 and 74, 16384 x 6152 338 and 271).  Rows of 4104 to 6144 columns have
  // a form for 768 threads with room for them (28728 x 4544 483 and 358, on 768 284; 2999 x 6144 72, 59, 50).
  constexpr bool AHEAD = !(THREADS == 1024 && POST == LAYER);
  uint4 qn, qd, qy, qo;
  float f_pre, m_pre, f_post, m_post, gate_in;
  auto fetch = [&](int64_t row) __attribute__((always_inline)) {
    qn = qd = qy = qo = make_uint4(0, 0, 0, 0);
    f_pre = f_post = m_pre = m_post = gate_in = 0.f;
    if (row >= a.t) return;
    const int64_t at = row * a.d + 8 * c;
    if (column) {
      if (PRE != NONE) qn = load16_once(dn + at);
      if (PRE != NONE) qy = load16_once(y + at);
      if (dy) qd = load16_once(dy + at);
      if (reads_o) qo = load16_once(o + at);
    }
    if (PRE != NONE) f_pre = stats[2 * a.t + row];
    if (PRE == LAYER) m_pre = stats[3 * a.t + row];
    if (POST != NONE) f_post = stats[row];
    if (POST == LAYER) m_post = stats[a.t + row];
    if (a.gate) gate_in = a.gate[a.gate_per_row ? row : 0];
  };
  const int64_t first = (int64_t)blockIdx.x * rows;
  if (AHEAD) fetch(first + of);
  int parity = 0;
  for (int64_t base = first; base < a.t; base += step, parity ^= 1) {    // all wavefronts alike: they meet at barriers
    const int64_t row = base + of, at = row * a.d + 8 * c;
    const bool there = row < a.t && column;
    if (!AHEAD) fetch(row);
    const float r1 = f_pre, m1 = m_pre, r2 = f_post, m2 = m_post;
    const float gate_raw = gate_in, gate = a.gate ? gate_value(a.gate_act, gate_in) : 1.f;
    float dY[8], h[8], z[8];
    unpack8(qd, dY);
    unpack8(qo, z);
    float s[3];
    if (PRE != NONE) {
      float dh[8], gain[8];
      unpack8(pg, gain);
      unpack8(qn, dh);
      unpack8(qy, h);
      s[0] = s[1] = 0.f;
#pragma unroll
      for (int e = 0; e < 8; e++) {
        h[e] = (h[e] - m1) * r1;
        C[e] = fmaf(dh[e], h[e], C[e]);
        if (PRE == LAYER) D[e] += dh[e];
        dh[e] *= gain[e];
        s[0] = fmaf(dh[e], h[e], s[0]);
        if (PRE == LAYER) s[1] += dh[e];
      }
      if (AHEAD) fetch(row + step);
      row_sums<PRE == LAYER ? 2 : 1>(s, sums.part[parity][0], waves, wave, lane);
      s[0] *= per;
      s[1] = PRE == LAYER ? s[1] * per : 0.f;
#pragma unroll
      for (int e = 0; e < 8; e++) dY[e] = fmaf(dh[e] - s[1] - h[e] * s[0], r1, dY[e]);
    } else if (AHEAD) {
      fetch(row + step);
    }
    if (there) store16<PAST>(dx + at, pack8(dY));
    s[0] = s[1] = s[2] = 0.f;
    float dz[8];
#pragma unroll
    for (int e = 0; e < 8; e++) {
      if (POST != NONE) z[e] = (z[e] - m2) * r2;
      const float v = dY[e] * gate;
      A[e] = fmaf(v, z[e], A[e]);
      if (POST == LAYER) Bs[e] += v;
      dz[e] = dY[e] * k[e];
      s[0] = fmaf(dz[e], z[e], s[0]);
      if (POST == LAYER) s[1] += dz[e];
    }
    if (POST == LAYER && gate_rows) {   // the norm's shift counts for the gate alone: read again for every row rather than kept
      float b[8], sc[8];
      load_vector((const bf16_t*)a.post_b, c, column, b);
      load_vector((const bf16_t*)a.scale, c, column, sc);
#pragma unroll
      for (int e = 0; e < 8; e++) s[2] = fmaf(dY[e], a.scale ? b[e] * sc[e] : b[e], s[2]);
    }
    if (POST != NONE || a.gate) {
      row_sums<POST == LAYER ? 3 : 1>(s, sums.part[parity][1], waves, wave, lane);
      if (gate_rows && row < a.t) {
        const float v = (s[0] + (POST == LAYER ? s[2] : 0.f)) * gate_slope(a.gate_act, gate_raw);
        if (a.gate_per_row) {
          if (c == 0) gate_rows[row] = v;
        } else {
          gate_sum += v;
        }
      }
    }
    const float t0 = POST != NONE ? s[0] * per : 0.f, t1 = POST == LAYER ? s[1] * per : 0.f;
#pragma unroll
    for (int e = 0; e < 8; e++) {
      if (POST != NONE) dz[e] = (dz[e] - t1 - z[e] * t0) * r2;
      dz[e] *= gate;
    }
    if (there) store16<PAST>(d_o + at, pack8(dz));
  }
  // Sets of sums in the order of the bits of `sets`; the wavefronts of a column add theirs up through LDS.  One workgroup alone finishes them too.
  const int64_t W = gridDim.x;
  int at_set = 0;
#pragma unroll
  for (int set = 0; set < 4; set++) {
    if (!(finish.sets >> set & 1) || (set == 1 && POST != LAYER) || (set == 3 && PRE != LAYER)) continue;   // those are not among the sets
    float* v = set == 0 ? A : set == 1 ? Bs : set == 2 ? C : D;
    if (rows > 1) {
      __syncthreads();
#pragma unroll
      for (int e = 0; e < 8; e++) joined_columns[wave * 512 + e * 64 + lane] = v[e];
      __syncthreads();
      if (of == 0)
        for (int r = 1; r < rows; r++)
#pragma unroll
          for (int e = 0; e < 8; e++) v[e] += joined_columns[(r * waves + wave) * 512 + e * 64 + lane];
    }
    if (of == 0 && column && W > 1) {
      float4* p = reinterpret_cast<float4*>(partial + ((int64_t)at_set * W + blockIdx.x) * a.d + 8 * c);
      p[0] = make_float4(v[0], v[1], v[2], v[3]);
      p[1] = make_float4(v[4], v[5], v[6], v[7]);
    }
    at_set++;
  }
  if (W == 1 && of == 0 && column) {
    if (finish.sets & 3) put_post<8>(finish, A, Bs, 8 * c);
    if (finish.sets & 4) put_sums<8>(finish.g.pre_g, C, 8 * c, finish.accumulate);
    if (finish.sets & 8) put_sums<8>(finish.g.pre_b, D, 8 * c, finish.accumulate);
  }
  if (gate_rows && !a.gate_per_row) {
    __syncthreads();
    if (wave % waves == 0 && lane == 0) joined_columns[of] = gate_sum;
    __syncthreads();
    if (threadIdx.x == 0) {
      float v = 0.f;
      for (int r = 0; r < rows; r++) v += joined_columns[r];
      if (W > 1)
        gate_rows[blockIdx.x] = v;
      else
        *finish.g.gate = v + (finish.accumulate ? *finish.g.gate : 0.f);
    }
  }
}

// The form for a workgroup's threads.  768 is for the kinds that run out of registers on 1024; the others are the same on both (28728 x 4544 RMSNorm on both sides 264 us on either,
// LayerNorm behind the block alone 227; 2999 x 6144 44.9 and 44.8, 39.3 and 38.6).
template <int POST, int PRE, bool PAST>
auto bwd_kernel(int threads) {
  if (threads <= 512) return residual_bwd_kernel<POST, PRE, PAST, 512>;
  if constexpr (POST == LAYER && PRE != NONE)
    if (threads <= 768) return residual_bwd_kernel<POST, PRE, PAST, 768>;
  return residual_bwd_kernel<POST, PRE, PAST, 1024>;
}

// What the sums of the workgroups come to: 32 columns a workgroup, a line of 128 bytes, four of them a lane, and every 32nd workgroup's sums in a group of eight
// lanes, eight of those requested at a time; the groups of a wavefront are added up by exchanges, the wavefronts' sums through LDS.
// Grid y: A and B with the gradients that follow from both, C, D, the shared gate.
__device__ __forceinline__ float over_groups(float v) {   // lanes 8, 16, ... apart
  v += from_lane<0x128>(v);
  auto w = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(w[0]) + __uint_as_float(w[1]);
  w = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(w[0]) + __uint_as_float(w[1]);
}
__device__ __forceinline__ void finish_sum(const float* partial, int W, int d, int64_t col, bool valid, float (*part)[8][4], float* out) {
  const int cg = threadIdx.x & 7, slice = threadIdx.x >> 3, wave = threadIdx.x >> 6;
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
  if (valid)
    for (int p = slice; p < W; p += 8 * 32) {
      float4 v[8];
#pragma unroll
      for (int q = 0; q < 8; q++) v[q] = p + 32 * q < W ? *reinterpret_cast<const float4*>(partial + (int64_t)(p + 32 * q) * d + col) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int q = 0; q < 8; q++) { s.x += v[q].x; s.y += v[q].y; s.z += v[q].z; s.w += v[q].w; }
    }
  s = make_float4(over_groups(s.x), over_groups(s.y), over_groups(s.z), over_groups(s.w));
  if ((threadIdx.x & 63) < 8) *reinterpret_cast<float4*>(part[wave][cg]) = s;
  __syncthreads();
#pragma unroll
  for (int e = 0; e < 4; e++) out[e] = (part[0][cg][e] + part[1][cg][e]) + (part[2][cg][e] + part[3][cg][e]);
}
__global__ __launch_bounds__(256) void residual_finish_kernel(FinishArgs a) {
  __shared__ __align__(16) float part[2][4][8][4];
  const int cg = threadIdx.x & 7, job = blockIdx.y;
  const int64_t col = ((int64_t)blockIdx.x * 8 + cg) * 4;
  const bool valid = col < a.d;
  const bool writes = valid && threadIdx.x < 8;
  if (job == 3) {        // the shared gate: one workgroup
    if (!a.gate_partial || blockIdx.x != 0) return;
    float v = 0.f, *red = &part[0][0][0][0];
    for (int p = threadIdx.x; p < a.W; p += 256) v += a.gate_partial[p];
    v = over_lanes<64, false>(v);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    if (threadIdx.x == 0) *a.g.gate = (red[0] + red[1]) + (red[2] + red[3]) + (a.accumulate ? *a.g.gate : 0.f);
    return;
  }
  const int before = __popc(a.sets & ((1 << (job == 0 ? 0 : job + 1)) - 1));
  const float* sums = a.partial + (int64_t)before * a.W * a.d;
  if (job > 0) {
    if (!(a.sets >> (job + 1) & 1)) return;
    float v[4];
    finish_sum(sums, a.W, a.d, col, valid, part[0], v);
    if (writes) put_sums<4>(job == 1 ? a.g.pre_g : a.g.pre_b, v, col, a.accumulate);
    return;
  }
  if (!(a.sets & 3)) return;
  float A[4] = {0.f, 0.f, 0.f, 0.f}, B[4] = {0.f, 0.f, 0.f, 0.f};
  if (a.sets & 1) {
    finish_sum(sums, a.W, a.d, col, valid, part[0], A);
    sums += (int64_t)a.W * a.d;
  }
  if (a.sets & 2) finish_sum(sums, a.W, a.d, col, valid, part[1], B);
  if (writes) put_post<4>(a, A, B, col);
}

// Wavefronts of a row, rows of a workgroup: eight wavefronts or more.
inline int row_waves(int64_t d) { return (int)ceil_div(d, 512); }
inline int rows_of(int waves) { return std::max(1, 8 / waves); }
// Workgroups, each going over several rows.  Backward one a CU, two where a wavefront has a row of its own (us with 256 and 512: 32768 x 4096 268 and 290,
// 5125 x 3200 42.6 and 43.4, 2999 x 3584 30.7 and 31.6, 777 x 4096 15.9 and 18, 26496 x 1024 64 and 67.6; 30000 x 256 26.7 and 24); with the next row but one requested too,
// the same.  One alone where it has no more to do than twice: it finishes the sums itself, without the second launch (8 x 256 5.8 us, 16 x 256 6.7 and with two 8.3, 4096
// columns of one row 5.4, of two 7.0 and 8.2, of four 9.7 and 8.2).
inline int64_t bwd_workgroups(int64_t t, int64_t d) {
  const int waves = row_waves(d);
  const int64_t blocks = ceil_div(t, rows_of(waves));
  if (blocks <= 2) return 1;
  return std::max<int64_t>(1, std::min<int64_t>(waves == 1 ? 512 : 256, blocks));
}
// Forward as many of 768 as gives all of them the same number of rows (5125 x 3200 25.1 us, with 256 29.2, a row each 29.1; 2999 x 3584 16.5, 20.3, 20.1; 30000 x 256 14.9,
// 19.8, 17.1); where the results go past the caches as backward (32768 x 4096 183, with 768 198, a row each 181; 16000 x 8192 176, 178, 233; 65000 x 2048 178, 198,
// 179; 500000 x 256 with 512 197, 256 262, 768 199).
inline int64_t fwd_workgroups(int64_t t, int64_t d, bool past) {
  const int waves = row_waves(d);
  const int64_t blocks = ceil_div(t, rows_of(waves)), most = !past ? 768 : waves == 1 ? 512 : 256;
  return ceil_div(blocks, ceil_div(blocks, most));
}

}  // namespace

hipError_t launch_residual_fwd(const ResidualArgs& a, const void* x, const void* o, void* y, void* n, float* stats, hipStream_t s) {
  if (a.t == 0) return hipSuccess;
  const int waves = row_waves(a.d), rows = rows_of(waves);
  const bool past = 2 * a.t * a.d >= NT_BYTES;
  const dim3 grid((unsigned)fwd_workgroups(a.t, a.d, past)), block(64 * waves * rows);
  ProfScope prof(PROF_ELEMENTWISE, (a.pre_kind == NONE ? 6.0 : 8.0) * (double)a.t * a.d, s);
#define CALL(POST, PRE)                                                                                                                \
  if (a.post_kind == POST && a.pre_kind == PRE)                                                                                        \
    hipLaunchKernelGGL((past ? residual_fwd_kernel<POST, PRE, true> : residual_fwd_kernel<POST, PRE, false>), grid, block, 0, s, a, (const bf16_t*)x, (const bf16_t*)o, (bf16_t*)y, (bf16_t*)n, stats, waves, rows);
  CALL(LAYER, LAYER) CALL(LAYER, RMS) CALL(LAYER, NONE) CALL(RMS, LAYER) CALL(RMS, RMS) CALL(RMS, NONE) CALL(NONE, LAYER) CALL(NONE, RMS) CALL(NONE, NONE)
#undef CALL
  return hipGetLastError();
}

size_t residual_bwd_partial_floats(int64_t t, int64_t d) { return (size_t)bwd_workgroups(t, d) * (size_t)(4 * d + 1); }

hipError_t launch_residual_bwd(const ResidualArgs& a, const void* dn, const void* dy, const void* y, const void* o, const float* stats, void* dx,
                               void* d_o, const ResidualGrads& g, int accumulate, float* partial, hipStream_t s) {
  const int waves = row_waves(a.d), rows = rows_of(waves);
  const int64_t W = bwd_workgroups(a.t, a.d);
  // which of A, B, C, D anybody asks for
  const int sets = (g.post_g || g.scale ? 1 : 0) | (g.post_b || (g.scale && a.post_b) ? 2 : 0) | (g.pre_g ? 4 : 0) | (g.pre_b ? 8 : 0);
  float* gate_partial = g.gate && !a.gate_per_row ? partial + (size_t)__builtin_popcount(sets) * W * a.d : nullptr;
  float* gate_rows = a.gate_per_row ? g.gate : gate_partial;
  const FinishArgs f = {partial, gate_partial, (int)W, a.d, sets, accumulate, (const bf16_t*)a.post_g, (const bf16_t*)a.post_b, (const bf16_t*)a.scale, g};
  {
    ProfScope prof(PROF_ELEMENTWISE, (4.0 + (dy ? 2 : 0) + (a.pre_kind == NONE ? 0 : 4) + 2) * (double)a.t * a.d, s);
    const bool past = 2 * a.t * a.d >= NT_BYTES;
    const int threads = 64 * waves * rows;
#define CALL(POST, PRE)                                                                                                              \
    if (a.post_kind == POST && a.pre_kind == PRE)                                                                                    \
      hipLaunchKernelGGL((past ? bwd_kernel<POST, PRE, true>(threads) : bwd_kernel<POST, PRE, false>(threads)), dim3((unsigned)W), dim3(threads), 0, s, a, (const bf16_t*)dn, \
                         (const bf16_t*)dy, (const bf16_t*)y, (const bf16_t*)o, stats, (bf16_t*)dx, (bf16_t*)d_o, gate_rows, partial, waves, rows, f);
    CALL(LAYER, LAYER) CALL(LAYER, RMS) CALL(LAYER, NONE) CALL(RMS, LAYER) CALL(RMS, RMS) CALL(RMS, NONE) CALL(NONE, LAYER) CALL(NONE, RMS) CALL(NONE, NONE)
#undef CALL
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (W == 1 || (!sets && !gate_partial)) return hipSuccess;
  ProfScope prof(PROF_ELEMENTWISE, 0.0, s);   // the bytes of the sums are counted with their first stage
  hipLaunchKernelGGL(residual_finish_kernel, dim3((unsigned)ceil_div(a.d, 32), 4), dim3(256), 0, s, f);
  return hipGetLastError();
}

}  // namespace mllm
