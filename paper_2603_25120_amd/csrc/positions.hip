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
// every run begins and at which position.  The runs travel as the kernel's argument, so that a call copies nothing and can be captured.  Bound by the
// launch: 220 rows 1.8 us, 32768 rows of 95 runs 3 to 5.  Few runs travel by themselves: the host copies the whole argument, 4.5 us a call of 192, 3.6 of 24.
// ---------------------------------------------------------------------------------------------
template <int RUNS>
struct PositionRuns { PositionRun run[RUNS]; };
template <int RUNS>
__global__ __launch_bounds__(256) void grid_positions_kernel(PositionRuns<RUNS> runs, int n, int32_t* __restrict__ pos, int64_t stride, int32_t row0, int32_t rows) {
  __shared__ PositionRun run[256];
  run[threadIdx.x].row = INT32_MAX;
  if ((int)threadIdx.x < n) run[threadIdx.x] = runs.run[threadIdx.x];
  __syncthreads();
  const uint32_t i = blockIdx.x * 256u + threadIdx.x;
  if (i >= (uint32_t)rows) return;
  const int32_t row = row0 + (int32_t)i;
  int lo = 0;                               // the last run that begins at or before the row
#pragma unroll
  for (int step = 128; step >= 1; step >>= 1)
    if (run[lo + step].row <= row) lo += step;
  const PositionRun r = run[lo];
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

// Row p: the cosines of p * frequency, then the sines (angles and their sines in fp64, as in rope_table_kernel).  Made once for many calls, and bound by the
// arithmetic: 32768 x 64 pairs 10.2 us, 131072 x 64 29.5, 2^20 x 64 204 (2.6 TB/s of what is written).
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
// Bound by memory.  An item is eight neighbouring pairs of a head (two 16-byte vectors), or eight elements behind them, which are copied.  A workgroup has a
// few whole tokens: their factors, gathered pair by pair from the rows that the axes' positions name, are put into LDS once for all heads, while
// the first items' values are on their way, and its lanes then go over the tokens' items side by side, a wavefront over 2 KB of a row.
// us for 32768 x 40 x 128 (pairs dealt out to three axes) / 26496 x 32 x 64 / 2999 x 32 x 128 / 8192 x 32 x 128 (dealt out): this 112 / 47 / 10.9 / 25, the first at
// 6.0 TB/s; two items a lane in flight 114 / 46 / 10.7 / 26, four 125 / 47 / 12.6 / 28; three times the tokens a workgroup 130 / 56 / 11 / 27; eight pairs of a token a
// thread that goes over its heads, factors in registers: 167 / 51 / 14.8 / 28.
// ---------------------------------------------------------------------------------------------
constexpr int ROPE_LDS = 4096;                 // floats of factors a workgroup holds
struct RopeItems { Division per_token, groups, pairs; int tokens; };   // items of a token and of a head; pairs of a head; tokens of a workgroup
template <bool PAST>
__global__ __launch_bounds__(256) void rope_axes_kernel(RopeAxesArgs a, RopeItems it, bool inverse) {
  __shared__ __align__(16) float factors[ROPE_LDS];   // of every token the cosines, then the sines
  const int tid = threadIdx.x, P = a.n_pairs;
  const int64_t row0 = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * it.tokens;
  if (row0 >= a.t) return;
  const int tokens = a.t - row0 < it.tokens ? (int)(a.t - row0) : it.tokens, items = tokens * (int)it.per_token.divisor;
  const bf16_t* x = (const bf16_t*)a.x + row0 * a.x_stride;
  bf16_t* y = (bf16_t*)a.y + row0 * a.y_stride;
  int token, group, column;
  bool tail;
  uint4 u, v;
  auto fetch = [&](int i) __attribute__((always_inline)) {
    if (i >= items) return;
    token = (int)divide((uint32_t)i, it.per_token);
    const int r = i - token * (int)it.per_token.divisor, h = (int)divide((uint32_t)r, it.groups);
    group = r - h * (int)it.groups.divisor;
    tail = 8 * group >= P;
    column = h * a.head_dim + 8 * group + (tail ? P : 0);
    const bf16_t* src = x + (int64_t)token * a.x_stride + column;
    u = load16_once(src);
    if (!tail) v = load16_once(src + P);
  };
  fetch(tid);
  for (int i = tid; i < tokens * P; i += 256) {
    const int of = (int)divide((uint32_t)i, it.pairs), pair = i - of * P;
    uint32_t axes = a.axes[0];                // from registers: a load here is one more to wait for before those of position and factors
#pragma unroll
    for (int k = 1; k < ROPE_PAIRS / 16; k++) axes = pair >> 4 == k ? a.axes[k] : axes;
    const int64_t p = a.pos[(axes >> (2 * (pair & 15)) & 3) * a.pos_stride + row0 + of];
    float c = __uint_as_float(0x7fc00000u), s = c;
    if (p >= 0 && p < a.n_pos) {
      c = a.table[p * (2 * P) + pair];
      s = a.table[p * (2 * P) + P + pair];
    }
    factors[of * 2 * P + pair] = c;
    factors[of * 2 * P + P + pair] = inverse ? -s : s;
  }
  __syncthreads();
  for (int i = tid; i < items; i += 256) {
    bf16_t* o = y + (int64_t)token * a.y_stride + column;
    if (tail) {
      store16<PAST>(o, u);
    } else {
      float cs[8], sn[8], first[8], second[8], f[8], g[8];
      load8(factors + token * 2 * P + 8 * group, cs);
      load8(factors + token * 2 * P + P + 8 * group, sn);
      unpack8(u, first);
      unpack8(v, second);
#pragma unroll
      for (int e = 0; e < 8; e++) {
        f[e] = first[e] * cs[e] - second[e] * sn[e];
        g[e] = second[e] * cs[e] + first[e] * sn[e];
      }
      store16<PAST>(o, pack8(f));
      store16<PAST>(o + P, pack8(g));
    }
    fetch(i + 256);
  }
}

}  // namespace

namespace {
template <int RUNS>
void launch_positions(const PositionRun* runs, int n, int32_t* pos, int64_t stride, int32_t row0, int32_t rows, hipStream_t s) {
  PositionRuns<RUNS> list;
  for (int i = 0; i < RUNS; i++) list.run[i] = i < n ? runs[i] : PositionRun{INT32_MAX, 0, 0, 1, 0};
  hipLaunchKernelGGL(grid_positions_kernel<RUNS>, dim3((unsigned)ceil_div(rows, 256)), dim3(256), 0, s, list, n, pos, stride, row0, rows);
}
}  // namespace

hipError_t launch_grid_positions(const PositionRun* runs, int n, int32_t* pos, int64_t stride, int32_t row0, int32_t rows, hipStream_t s) {
  if (n <= 0 || rows <= 0) return hipSuccess;
  if (n > POSITION_RUNS) return hipErrorInvalidValue;
  ProfScope prof(PROF_ELEMENTWISE, 12.0 * rows, s);
  if (n <= 24)
    launch_positions<24>(runs, n, pos, stride, row0, rows, s);
  else
    launch_positions<POSITION_RUNS>(runs, n, pos, stride, row0, rows, s);
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
  const int64_t per_token = (int64_t)a.n_heads * groups;
  // two items a thread where a token has fewer, but no fewer than 1024 workgroups
  int64_t tokens = std::min<int64_t>(512 / per_token, ROPE_LDS / (2 * a.n_pairs));
  tokens = std::max<int64_t>(1, std::min(tokens, a.t / 1024));
  const RopeItems it = {division((uint32_t)per_token), division((uint32_t)groups), division((uint32_t)a.n_pairs), (int)tokens};
  const double values = (double)a.t * a.n_heads * (a.y == a.x ? 2 * a.n_pairs : a.head_dim);
  ProfScope prof(PROF_ELEMENTWISE, 4.0 * values, s);
  const int64_t blocks = ceil_div(a.t, tokens);
  const dim3 grid((unsigned)std::min(blocks, MAX_GRID), (unsigned)ceil_div(blocks, MAX_GRID));
  const auto kernel = 2.0 * values >= NT_BYTES ? rope_axes_kernel<true> : rope_axes_kernel<false>;
  hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, a, it, inverse != 0);
  return hipGetLastError();
}

}  // namespace mllm
