// Rotary positions with several axes: the positions of packed text, images and clips on the axes time, height and width, the table of the
// angles for any list of frequencies, and the rotation of heads whose pairs follow different axes.
#include <algorithm>

#include "common.h"
#include "kernels.h"
#include "rows.h"

namespace mllm {

namespace {

// ---------------------------------------------------------------------------------------------
// Positions.  A run is a stretch of text or a grid of frames x height x width rows; the host has walked over the samples and knows where
// every run begins and at which position.  The runs travel as the kernel's argument, so that a call copies nothing and can be captured.
// ---------------------------------------------------------------------------------------------
__global__ __launch_bounds__(256) void grid_positions_kernel(PositionRuns runs, int n, int32_t* __restrict__ pos, int64_t stride, int32_t row0, int32_t rows) {
  const int32_t i = blockIdx.x * 256 + threadIdx.x;
  if (i >= rows) return;
  const int32_t row = row0 + i;
  int lo = 0, hi = n;                       // the last run that begins at or before the row
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (runs.run[mid].row <= row) lo = mid; else hi = mid;
  }
  const PositionRun r = runs.run[lo];
  const int32_t at = row - r.row;
  int32_t a = at, b = at, c = at;
  if (r.frame_rows > 0) {
    const uint32_t frame = (uint32_t)at / (uint32_t)r.frame_rows, in = (uint32_t)at - frame * (uint32_t)r.frame_rows;
    a = (int32_t)frame * r.step;
    b = (int32_t)(in / (uint32_t)r.width);
    c = (int32_t)(in - (uint32_t)b * (uint32_t)r.width);
  }
  pos[row] = r.position + a;
  pos[stride + row] = r.position + b;
  pos[2 * stride + row] = r.position + c;
}

// Row p: the cosines of p * frequency, then the sines (angles and their sines in fp64, as in rope_table_kernel).
__global__ __launch_bounds__(256) void rope_freq_table_kernel(float* __restrict__ table, int64_t n, int pairs, RopeFrequencies f) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= n) return;
  const int64_t p = i / pairs;
  const int pair = (int)(i - p * pairs);
  double sn, cs;
  sincos((double)p * f.frequency[pair], &sn, &cs);
  table[p * 2 * pairs + pair] = (float)cs;
  table[p * 2 * pairs + pairs + pair] = (float)sn;
}

// ---------------------------------------------------------------------------------------------
// Rotation: pair i of a head, its elements i and i + pairs, by the angle of position pos[axis of i][row]; elements from 2 pairs on stay.
// A thread has eight neighbouring pairs of a token and takes them through up to heads_per heads (grid y), four heads' values requested
// before any is stored: their factors, as many bytes as the values of two heads, are then read once for all of them.  Pairs of several
// axes read the eight factors of each axis that is there and keep their own.  Threads behind the pairs' copy what is not rotated.
// ---------------------------------------------------------------------------------------------
template <bool PAST>
__global__ __launch_bounds__(256) void rope_axes_kernel(RopeAxesArgs a, int groups, int tokens_per_block, int heads_per, bool inverse) {
  const int tid = threadIdx.x, of = tid / groups, g = tid - of * groups;
  if (of >= tokens_per_block) return;
  const int rotated = a.n_pairs >> 3, h0 = blockIdx.y * heads_per, h1 = min(h0 + heads_per, a.n_heads);
  const bf16_t* x = (const bf16_t*)a.x;
  bf16_t* y = (bf16_t*)a.y;
  for (int64_t row = (int64_t)blockIdx.x * tokens_per_block + of; row < a.t; row += (int64_t)gridDim.x * tokens_per_block) {
    const bool tail = g >= rotated;
    const int at = tail ? 2 * a.n_pairs + 8 * (g - rotated) : 8 * g;
    float cs[8], sn[8];
    if (!tail) {
#pragma unroll
      for (int e = 0; e < 8; e++) cs[e] = sn[e] = __uint_as_float(0x7fc00000u);
      const uint64_t axes = *reinterpret_cast<const uint64_t*>(a.axis + 8 * g);
      const uint32_t there = a.present[g];
#pragma unroll
      for (int k = 0; k < ROPE_AXES; k++) {
        if (!(there >> k & 1)) continue;
        const int64_t p = a.pos[k * a.pos_stride + row];
        if (p < 0 || p >= a.n_pos) continue;          // those pairs stay NaN
        float c[8], s[8];
        load8(a.table + p * (2 * a.n_pairs) + 8 * g, c);
        load8(a.table + p * (2 * a.n_pairs) + a.n_pairs + 8 * g, s);
#pragma unroll
        for (int e = 0; e < 8; e++) {
          const bool mine = (axes >> (8 * e) & 0xff) == k;
          cs[e] = mine ? c[e] : cs[e];
          sn[e] = mine ? (inverse ? -s[e] : s[e]) : sn[e];
        }
      }
    }
    const bf16_t* src = x + row * a.x_stride + at;
    bf16_t* dst = y + row * a.y_stride + at;
    constexpr int AHEAD = 4;
    for (int h = h0; h < h1; h += AHEAD) {
      uint4 u[AHEAD], v[AHEAD];
#pragma unroll
      for (int j = 0; j < AHEAD; j++) {
        u[j] = v[j] = make_uint4(0, 0, 0, 0);
        if (h + j < h1) {
          u[j] = *reinterpret_cast<const uint4*>(src + (int64_t)(h + j) * a.head_dim);
          if (!tail) v[j] = *reinterpret_cast<const uint4*>(src + (int64_t)(h + j) * a.head_dim + a.n_pairs);
        }
      }
#pragma unroll
      for (int j = 0; j < AHEAD; j++) {
        if (h + j >= h1) break;
        bf16_t* o = dst + (int64_t)(h + j) * a.head_dim;
        if (tail) {
          store16<PAST>(o, u[j]);
          continue;
        }
        float p[8], q[8], r[8], s[8];
        unpack8(u[j], p);
        unpack8(v[j], q);
#pragma unroll
        for (int e = 0; e < 8; e++) {
          r[e] = p[e] * cs[e] - q[e] * sn[e];
          s[e] = q[e] * cs[e] + p[e] * sn[e];
        }
        store16<PAST>(o, pack8(r));
        store16<PAST>(o + a.n_pairs, pack8(s));
      }
    }
  }
}

}  // namespace

hipError_t launch_grid_positions(const PositionRuns& runs, int n, int32_t* pos, int64_t stride, int32_t row0, int32_t rows, hipStream_t s) {
  if (n <= 0 || rows <= 0) return hipSuccess;
  ProfScope prof(PROF_ELEMENTWISE, 12.0 * rows, s);
  hipLaunchKernelGGL(grid_positions_kernel, dim3((unsigned)ceil_div(rows, 256)), dim3(256), 0, s, runs, n, pos, stride, row0, rows);
  return hipGetLastError();
}

hipError_t launch_rope_freq_table(float* table, int64_t n_pos, int32_t n_pairs, const RopeFrequencies& f, hipStream_t s) {
  const int64_t n = n_pos * n_pairs;
  if (n == 0) return hipSuccess;
  ProfScope prof(PROF_ELEMENTWISE, 8.0 * (double)n, s);
  hipLaunchKernelGGL(rope_freq_table_kernel, dim3((unsigned)ceil_div(n, 256)), dim3(256), 0, s, table, n, n_pairs, f);
  return hipGetLastError();
}

hipError_t launch_rope_axes(const RopeAxesArgs& a, int inverse, hipStream_t s) {
  if (a.t == 0 || a.n_heads == 0) return hipSuccess;
  const int groups = a.n_pairs / 8 + (a.y == a.x ? 0 : (a.head_dim - 2 * a.n_pairs) / 8);   // in place the rest is there already
  const int tokens = 256 / groups;
  int heads_per = 8;
  while (heads_per > 1 && ceil_div(a.t, tokens) * ceil_div(a.n_heads, heads_per) < 1024) heads_per /= 2;
  const double values = (double)a.t * a.n_heads * (a.y == a.x ? 2 * a.n_pairs : a.head_dim);
  ProfScope prof(PROF_ELEMENTWISE, 4.0 * values, s);
  const dim3 grid((unsigned)std::min(ceil_div(a.t, tokens), MAX_GRID), (unsigned)ceil_div(a.n_heads, heads_per));
  if (2.0 * values >= NT_BYTES)
    hipLaunchKernelGGL(rope_axes_kernel<true>, grid, dim3(256), 0, s, a, groups, tokens, heads_per, inverse != 0);
  else
    hipLaunchKernelGGL(rope_axes_kernel<false>, grid, dim3(256), 0, s, a, groups, tokens, heads_per, inverse != 0);
  return hipGetLastError();
}

}  // namespace mllm
