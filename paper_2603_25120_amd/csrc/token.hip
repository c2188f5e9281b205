// The token side of a language model: rows of the token table into the packed sequence and the table's gradient, the RMS norm of
// every query and key head with the rotary positions in the same pass and its gradient, and the loss over the vocabulary with the
// gradient of the logits.  All are bound by memory: bf16 (or fp32) storage, fp32 arithmetic, 16-byte accesses, one rounding of each
// result, no atomics on values that are summed.
#include <algorithm>
#include <cmath>

#include "common.h"
#include "kernels.h"

namespace mllm {

namespace {

__device__ __forceinline__ void unpack8(const uint4& u, float* f) {
  f[0] = bf16lo(u.x); f[1] = bf16hi(u.x); f[2] = bf16lo(u.y); f[3] = bf16hi(u.y);
  f[4] = bf16lo(u.z); f[5] = bf16hi(u.z); f[6] = bf16lo(u.w); f[7] = bf16hi(u.w);
}
__device__ __forceinline__ uint4 pack8(const float* f) {
  return make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7]));
}
__device__ __forceinline__ void load8(const float* p, float* f) {
  const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
  f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
}
__device__ __forceinline__ void load8(const bf16_t* p, float* f) { unpack8(*reinterpret_cast<const uint4*>(p), f); }

// Results of NT_BYTES and more, half of the memory-side cache, are stored past the caches: the kernel that reads them next does not find them
// there, and as ordinary stores they displace what is being read (32768 x 4096 rows of the table 72 -> 50 us).  With that kernel behind the call,
// us past the caches and not: norm and rotation with the attention that reads it, 84 MB 151 and 145, 126 MB 206 and 194, 168 MB 246 and 247,
// 252 MB 353 and 359; embedding rows with the norm that reads them, 101 MB 66.5 and 66.8, 134 MB 88 and 91, 201 MB 141 and 144.
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
template <bool PAST>   // (a flag at run time will not do: the compiler makes one ordinary store of both)
__device__ __forceinline__ void store16(void* p, const uint4& v) {
  const u32x4 w = {v.x, v.y, v.z, v.w};
  if (PAST)
    __builtin_nontemporal_store(w, reinterpret_cast<u32x4*>(p));
  else
    *reinterpret_cast<u32x4*>(p) = w;
}
__device__ __forceinline__ uint4 load16_once(const void* p) {   // what nobody reads a second time
  const u32x4 w = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p));
  return make_uint4(w[0], w[1], w[2], w[3]);
}
constexpr int64_t NT_BYTES = (int64_t)128 << 20;

// What 2, 4, 8, 16 or 64 neighbouring lanes hold, added up or the largest, in all of them: exchanges inside the vector unit (through LDS, as
// __shfl_xor goes, a step is some fifty cycles).
template <int CTRL>
__device__ __forceinline__ float from_lane(float v) { return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true)); }
template <bool MAX>
__device__ __forceinline__ float joined(float a, float b) { return MAX ? fmaxf(a, b) : a + b; }
template <int LANES, bool MAX>
__device__ __forceinline__ float over_lanes(float v) {
  static_assert(LANES == 2 || LANES == 4 || LANES == 8 || LANES == 16 || LANES == 64, "whole groups of lanes");
  v = joined<MAX>(v, from_lane<0xb1>(v));                       // the other one of a pair
  if (LANES > 2) v = joined<MAX>(v, from_lane<0x4e>(v));        // the other pair of four
  if (LANES > 4) v = joined<MAX>(v, from_lane<0x141>(v));       // a row's halves mirrored: the other four
  if (LANES > 8) v = joined<MAX>(v, from_lane<0x140>(v));       // a row mirrored: the other eight
  if (LANES > 16) {
    auto w = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = joined<MAX>(__uint_as_float(w[0]), __uint_as_float(w[1]));
    w = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = joined<MAX>(__uint_as_float(w[0]), __uint_as_float(w[1]));
  }
  return v;
}

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
constexpr int64_t MAX_GRID = 1 << 20;   // workgroups along x: a dimension holds fewer than 2^32 threads

// ---------------------------------------------------------------------------------------------
// Rows of the token table: y[t] = scale * table[ids[t]], zeros for ids below 0, NaN for ids that the table does not hold.  LPR lanes
// take a row (of a slice of up to four 16-byte vectors a lane: grid y), so that narrow rows fill the wavefront too.
// ---------------------------------------------------------------------------------------------
constexpr int EMBED_VECS = 4;
template <typename E, int LPR, bool PAST>
__global__ __launch_bounds__(256) void embed_fwd_kernel(const E* __restrict__ table, const int32_t* __restrict__ ids, bf16_t* __restrict__ y,
                                                        int64_t T, int64_t vocab, int nvec, int64_t ldy, float scale) {
  const int lane = threadIdx.x % LPR, c0 = blockIdx.y * (EMBED_VECS * LPR) + lane;
  for (int64_t row = (int64_t)blockIdx.x * (256 / LPR) + threadIdx.x / LPR; row < T; row += (int64_t)gridDim.x * (256 / LPR)) {
    const int32_t id = ids[row];
    const float nothing = id < 0 ? 0.f : __uint_as_float(0x7fc00000u);
    const bool there = id >= 0 && id < vocab;
    const float by = there ? scale : 1.f;                  // a scale that is no number leaves them zero
    const E* src = table + (there ? (int64_t)id * nvec * 8 : 0);
    float v[EMBED_VECS][8];
#pragma unroll
    for (int j = 0; j < EMBED_VECS; j++) {
      const int c = c0 + j * LPR;
#pragma unroll
      for (int e = 0; e < 8; e++) v[j][e] = nothing;
      if (there && c < nvec) load8(src + (int64_t)c * 8, v[j]);
    }
#pragma unroll
    for (int j = 0; j < EMBED_VECS; j++) {
      const int c = c0 + j * LPR;
#pragma unroll
      for (int e = 0; e < 8; e++) v[j][e] *= by;
      if (c < nvec) store16<PAST>(y + row * ldy + (int64_t)c * 8, pack8(v[j]));
    }
  }
}

// ---------------------------------------------------------------------------------------------
// The table's gradient.  The tokens are first brought together by id (embed_sort_kernel), then chunks of the sorted tokens are added up,
// every chunk alike long whatever the ids' frequencies (embed_sum_kernel); ids that go on beyond their chunk leave partial sums, which
// embed_join_kernel adds up chunk after chunk.  All orders are those of the tokens: no atomics on sums, same bits every time.
//
// Sorting: ids are dealt to `buckets` (a power of two, at least 256, at most 1024 ids each) by their lowest bits, so that frequent
// neighbours land in different ones.  A workgroup owns a bucket and reads ALL ids: those of lower buckets only count, which gives its place
// in the list without waiting for any other workgroup (32768 tokens 13.6 us, 2999 5.5).  Each of its 16 wavefronts counts a contiguous piece of the tokens per
// id; from the scan over (id, wavefront) it then places its piece's tokens in their order.  The ids come from L2: 32768 of them are 128 KB.
// It also leaves a bit for every id of its bucket that no token has: with the gradient overwritten, their rows are cleared
// (embed_sum_kernel).
// ---------------------------------------------------------------------------------------------
constexpr int SORT_WAVES = 16, SORT_RANGE = 1024, SORT_IDS = 32;   // RANGE: ids a bucket holds at most
__device__ __forceinline__ int lanes_below(uint64_t mask) { return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0u)); }

__global__ __launch_bounds__(64 * SORT_WAVES) void embed_sort_kernel(const int32_t* __restrict__ ids, int T, int vocab, int log2_buckets,
                                                                     int32_t* __restrict__ order, int32_t* __restrict__ keys, int32_t* __restrict__ total,
                                                                     uint64_t* __restrict__ absent) {
  __shared__ int hist[SORT_WAVES][SORT_RANGE];
  __shared__ int sums[SORT_WAVES], below_of[SORT_WAVES];
  const int bucket = blockIdx.x, mask = (1 << log2_buckets) - 1, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int range = (vocab - bucket + mask) >> log2_buckets;   // ids bucket, bucket + buckets, ... below vocab
  for (int i = threadIdx.x; i < range; i += 64 * SORT_WAVES)
#pragma unroll
    for (int w = 0; w < SORT_WAVES; w++) hist[w][i] = 0;
  __syncthreads();
  const int piece = (int)(((int64_t)T + 64 * SORT_WAVES - 1) / (64 * SORT_WAVES) * 64);
  const int64_t first = (int64_t)wave * piece, end = first + piece < T ? first + piece : T;
  int32_t id[SORT_IDS];   // of 64 SORT_IDS tokens; a piece that is no longer keeps them for the second walk
  auto request = [&](int64_t t0) {
#pragma unroll
    for (int j = 0; j < SORT_IDS; j++) {
      id[j] = -1;
      if (t0 + 64 * (j & ~7) < end && t0 + 64 * j + lane < end) id[j] = ids[t0 + 64 * j + lane];   // by eights: few tokens walk over few registers
    }
  };
  int below = 0;
  for (int64_t t0 = first; t0 < end; t0 += 64 * SORT_IDS) {
    request(t0);
#pragma unroll
    for (int j = 0; j < SORT_IDS; j++) {
      if (t0 + 64 * (j & ~7) >= end) break;
      const bool there = (uint32_t)id[j] < (uint32_t)vocab;
      below += there && (id[j] & mask) < bucket;
      if (there && (id[j] & mask) == bucket) atomicAdd(&hist[wave][id[j] >> log2_buckets], 1);
    }
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) below += __shfl_xor(below, o, 64);
  if (lane == 0) below_of[wave] = below;
  __syncthreads();
  // the scan: thread i has the i-th id of the bucket
  int count = 0;
  if (threadIdx.x < range)
#pragma unroll
    for (int w = 0; w < SORT_WAVES; w++) count += hist[w][threadIdx.x];
  int upto = count;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int v = __shfl_up(upto, o, 64);
    if (lane >= o) upto += v;
  }
  if (lane == 63) sums[wave] = upto;
  __syncthreads();
  int at = upto - count;
#pragma unroll
  for (int w = 0; w < SORT_WAVES; w++) at += below_of[w] + (w < wave ? sums[w] : 0);
  if (T > 0 && bucket == mask && threadIdx.x == 64 * SORT_WAVES - 1) *total = at + count;
  if (threadIdx.x < range)
#pragma unroll
    for (int w = 0; w < SORT_WAVES; w++) {
      const int n = hist[w][threadIdx.x];
      hist[w][threadIdx.x] = at;
      at += n;
    }
  const uint64_t without = __ballot(threadIdx.x < range && count == 0);
  if (lane == 0) absent[bucket * SORT_WAVES + wave] = without;
  __syncthreads();
  for (int64_t t0 = first; t0 < end; t0 += 64 * SORT_IDS) {
    if (piece > 64 * SORT_IDS) request(t0);
#pragma unroll
    for (int j = 0; j < SORT_IDS; j++) {
      if (t0 + 64 * (j & ~7) >= end) break;
      const bool mine = (uint32_t)id[j] < (uint32_t)vocab && (id[j] & mask) == bucket;
      uint64_t left = __ballot(mine);
      while (left) {   // the lanes of one id at a time
        const int32_t v = __builtin_amdgcn_readlane(id[j], __builtin_ctzll(left));
        const uint64_t same = __ballot(mine && id[j] == v);
        int place = 0;
        if (lane == 0) place = atomicAdd(&hist[wave][v >> log2_buckets], __popcll(same));
        place = __builtin_amdgcn_readfirstlane(place) + lanes_below(same);
        if (mine && id[j] == v) {
          order[place] = (int32_t)(t0 + 64 * j + lane);
          keys[place] = v;
        }
        left &= ~same;
      }
    }
  }
}

// Up to 64 tokens, or none: clears the rows of all other ids.  The lanes hold the tokens' ids, the workgroups go over the table in one sweep.
__global__ __launch_bounds__(256) void embed_clear_kernel(float* __restrict__ dtable, int nvec, int64_t n_quads, const int32_t* __restrict__ ids, int T) {
  const int64_t first = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * 256, row0 = first / (2 * nvec), quad = first + threadIdx.x;
  const int row = (int)row0 + (int)((uint32_t)(quad - row0 * (2 * nvec)) / (uint32_t)(2 * nvec)), lane = threadIdx.x & 63;
  const int32_t id = lane < T ? ids[lane] : -1;
  bool clear = quad < n_quads;
  for (int r = __builtin_amdgcn_readfirstlane(row); r <= __builtin_amdgcn_readlane(row, 63); r++)
    if (__ballot(id == r) && row == r) clear = false;
  if (clear) reinterpret_cast<float4*>(dtable)[quad] = make_float4(0.f, 0.f, 0.f, 0.f);
}

// Up to 64 tokens: the lanes hold their ids, and the wavefront of an id's first token (and a slice of 512 columns) adds up its rows.  No sorting and no
// joining: 20 tokens of 256 columns 9.9 us, sorted 14.2; 64 of 2048, added to the gradient, 4 and 14.  (More than a lane's id each would make one
// wavefront's run of rows too long.)
constexpr int EMBED_FEW = 64;
__global__ __launch_bounds__(256) void embed_few_kernel(const bf16_t* __restrict__ dy, const int32_t* __restrict__ ids, float* __restrict__ dtable, int T,
                                                        int vocab, int slices, int nvec, int64_t ld, float scale, int accumulate) {
  const int item = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int token = item / slices, v = (item - token * slices) * 64 + lane;
  if (token >= T) return;
  const int32_t id = lane < T ? ids[lane] : -1, mine = __builtin_amdgcn_readlane(id, token);
  if ((uint32_t)mine >= (uint32_t)vocab) return;
  uint64_t same = __ballot(id == mine);
  if (__builtin_ctzll(same) != token || v >= nvec) return;
  float* o = dtable + ((int64_t)mine * nvec + v) * 8;
  float old[8], acc[8];
#pragma unroll
  for (int e = 0; e < 8; e++) old[e] = acc[e] = 0.f;
  if (accumulate) load8(o, old);
  while (same) {
    constexpr int AHEAD = 8;
    uint4 row[AHEAD];
    int n = 0;
#pragma unroll
    for (int j = 0; j < AHEAD; j++) {
      row[j] = make_uint4(0, 0, 0, 0);
      if (!same) continue;
      row[j] = load16_once(dy + __builtin_ctzll(same) * ld + (int64_t)v * 8);
      same &= same - 1;
      n++;
    }
#pragma unroll
    for (int j = 0; j < AHEAD; j++) {
      if (j >= n) break;
      float f[8];
      unpack8(row[j], f);
#pragma unroll
      for (int e = 0; e < 8; e++) acc[e] += f[e];
    }
  }
#pragma unroll
  for (int e = 0; e < 8; e++) acc[e] = fmaf(scale, acc[e], old[e]);
  reinterpret_cast<float4*>(o)[0] = make_float4(acc[0], acc[1], acc[2], acc[3]);
  reinterpret_cast<float4*>(o)[1] = make_float4(acc[4], acc[5], acc[6], acc[7]);
}

// Adds up a chunk of the sorted tokens: LPR lanes take eight columns each (of a slice of 8 LPR columns) and walk over the chunk's rows, eight
// requested at a time, with what the table holds for the ids that end among them where the sums are added to that (requested
// when its id ended, each such row was waited for by itself: two microbatches of 32768 tokens, half of them images, 4096 columns, 186 -> 138 us).  Where an id ends, the sum goes to
// its row of the table; one that began in an earlier chunk, or goes on in the next one, to the partial sums instead: [0][chunk] or
// [1][chunk].
// Where the table is overwritten, the workgroups behind the sums' clear the rows of the ids that no token has, in one sweep (a row a wavefront:
// 360 us for 131072 rows of 4096 columns, 314 so).  The sums wait for scattered rows of dy meanwhile, so that they cost little beside it, provided that they keep
// few registers, which is why only ACCUMULATE has the table's old rows (76 registers; with the 142 of the other form the clearing has too few
// wavefronts: two microbatches of 32768 tokens into 131072 rows 594 us, 494 so).  With a launch of its own for the clearing the same are 499 us; 2999 tokens
// into 50257 rows of 3584 132, 122 so; 300 into 1000 of 512 17 and 13.
template <int LPR, bool ACCUMULATE>
__global__ __launch_bounds__(256) void embed_sum_kernel(const bf16_t* __restrict__ dy, const int32_t* __restrict__ order, const int32_t* __restrict__ keys,
                                                        const int32_t* __restrict__ total, float* __restrict__ dtable, float* __restrict__ partial,
                                                        int chunk, int n_chunks, int slices, int nvec, int64_t ld, float scale, uint32_t sum_blocks,
                                                        const uint64_t* __restrict__ absent, int log2_buckets, int64_t n_quads) {
  constexpr int AHEAD = 8;
  if (!ACCUMULATE) {
    const int64_t block = (int64_t)blockIdx.y * gridDim.x + blockIdx.x - sum_blocks;
    if (block >= 0) {
      const int64_t first = block * 256, row0 = first / (2 * nvec), quad = first + threadIdx.x;
      const int row = (int)row0 + (int)((uint32_t)(quad - row0 * (2 * nvec)) / (uint32_t)(2 * nvec)), at = row >> log2_buckets;
      if (quad < n_quads && absent[(row & ((1 << log2_buckets) - 1)) * SORT_WAVES + (at >> 6)] >> (at & 63) & 1)
        reinterpret_cast<float4*>(dtable)[quad] = make_float4(0.f, 0.f, 0.f, 0.f);
      return;
    }
  }
  const uint32_t item = blockIdx.x * (256 / LPR) + threadIdx.x / LPR;
  const int c = (int)(item / (uint32_t)slices), v = (int)(item - (uint32_t)c * slices) * LPR + threadIdx.x % LPR;
  const int N = *total;
  const int64_t p0 = (int64_t)c * chunk;
  if (c >= n_chunks || p0 >= N || v >= nvec) return;
  const int n = N - p0 < chunk ? (int)(N - p0) : chunk;
  const int32_t behind = p0 + n < N ? keys[p0 + n] : -1;   // the id that follows the chunk
  bool began_before = c > 0 && keys[p0 - 1] == keys[p0];
  const bf16_t* src = dy + (int64_t)v * 8;
  float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  for (int i = 0; i < n; i += AHEAD) {
    int32_t key[AHEAD + 1];
    uint4 row[AHEAD];
    float old[AHEAD][8];
#pragma unroll
    for (int j = 0; j < AHEAD; j++) {
      const int64_t p = p0 + (i + j < n ? i + j : n - 1);   // behind the chunk's end its last row again
      key[j] = keys[p];
      row[j] = load16_once(src + order[p] * ld);
    }
    key[AHEAD] = i + AHEAD < n ? keys[p0 + i + AHEAD] : behind;
#pragma unroll
    for (int j = 0; j < AHEAD; j++) {
#pragma unroll
      for (int e = 0; e < 8; e++) old[j][e] = 0.f;
      if (ACCUMULATE && i + j < n && key[j] != (i + j + 1 < n ? key[j + 1] : behind)) load8(dtable + ((int64_t)key[j] * nvec + v) * 8, old[j]);
    }
#pragma unroll
    for (int j = 0; j < AHEAD; j++) {
      if (i + j >= n) break;
      float f[8];
      unpack8(row[j], f);
#pragma unroll
      for (int e = 0; e < 8; e++) acc[e] += f[e];
      const bool last = i + j + 1 == n;
      const int32_t next = last ? behind : key[j + 1];
      if (next == key[j] && !last) continue;
      const int slot = began_before ? 0 : next == key[j] ? 1 : 2;   // 2: the table
      float* o = slot < 2 ? partial + (((int64_t)slot * n_chunks + c) * nvec + v) * 8 : dtable + ((int64_t)key[j] * nvec + v) * 8;
#pragma unroll
      for (int e = 0; e < 8; e++) {
        f[e] = slot < 2 ? acc[e] : fmaf(scale, acc[e], old[j][e]);
        acc[e] = 0.f;
      }
      reinterpret_cast<float4*>(o)[0] = make_float4(f[0], f[1], f[2], f[3]);
      reinterpret_cast<float4*>(o)[1] = make_float4(f[4], f[5], f[6], f[7]);
      began_before = false;
    }
  }
}

// An id that begins in a chunk and goes on beyond it: its last partial sum of that chunk and the first ones of the following chunks, as
// many as begin with it.  A wavefront looks at a chunk and has 256 columns; runs of many chunks, ids that a good part of the tokens have, are
// added up by the workgroup's four wavefronts together, a quarter of the chunks each (30000 tokens, 640 columns: 9 us, 20 without).
__device__ __forceinline__ float4 join_sum(const float4* src, int64_t step, int chunks) {
  float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int i = 0; i < chunks; i += 8) {
    float4 f[8];
#pragma unroll
    for (int j = 0; j < 8; j++) f[j] = i + j < chunks ? src[(int64_t)(i + j) * step] : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int j = 0; j < 8; j++) { sum.x += f[j].x; sum.y += f[j].y; sum.z += f[j].z; sum.w += f[j].w; }
  }
  return sum;
}
__global__ __launch_bounds__(256) void embed_join_kernel(const int32_t* __restrict__ keys, const int32_t* __restrict__ total, float* __restrict__ dtable,
                                                         const float* __restrict__ partial, int chunk, int n_chunks, int slices, int nvec, float scale,
                                                         int accumulate) {
  constexpr int LONG = 32;                           // chunks of a run that the four wavefronts share
  __shared__ int2 runs[4];                           // (chunks, id)
  __shared__ float4 part[4][64];
  const int group = (int)(blockIdx.x / (uint32_t)slices), wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int q = (int)(blockIdx.x - (uint32_t)group * slices) * 64 + lane;   // four columns
  const int N = *total;
  const int64_t step = (int64_t)nvec * 2;
  const float4* src = reinterpret_cast<const float4*>(partial) + q;
  const bool there = q < 2 * nvec;
  auto put = [&](int id, const float4& sum) {
    float4* o = reinterpret_cast<float4*>(dtable) + (int64_t)id * step + q;
    const float4 old = accumulate ? *o : make_float4(0.f, 0.f, 0.f, 0.f);
    *o = make_float4(fmaf(scale, sum.x, old.x), fmaf(scale, sum.y, old.y), fmaf(scale, sum.z, old.z), fmaf(scale, sum.w, old.w));
  };
  const int c = group * 4 + wave;
  const int64_t p0 = (int64_t)c * chunk, p1 = p0 + chunk;
  int id = 0, chunks = 0;                            // that begin with the id
  if (c < n_chunks && p1 < N) {
    id = keys[p1 - 1];
    if (keys[p1] == id && !(c > 0 && keys[p0] == id && keys[p0 - 1] == id)) {
      while (true) {
        const int64_t p = p1 + (int64_t)(chunks + lane) * chunk;
        const uint64_t others = ~__ballot(p < N && keys[p] == id);
        if (others) { chunks += __builtin_ctzll(others); break; }
        chunks += 64;
      }
      if (chunks < LONG && there) {
        float4 sum = src[((int64_t)n_chunks + c) * step];
        const float4 rest = join_sum(src + (int64_t)(c + 1) * step, step, chunks);
        sum.x += rest.x; sum.y += rest.y; sum.z += rest.z; sum.w += rest.w;
        put(id, sum);
      }
    }
  }
  if (lane == 0) runs[wave] = make_int2(chunks, id);
  __syncthreads();
  for (int w = 0; w < 4; w++) {
    const int2 run = runs[w];
    if (run.x < LONG) continue;
    const int from = (int)((int64_t)run.x * wave / 4), to = (int)((int64_t)run.x * (wave + 1) / 4), first = group * 4 + w;
    if (there) part[wave][lane] = join_sum(src + (int64_t)(first + 1 + from) * step, step, to - from);
    __syncthreads();
    if (wave == 0 && there) {
      float4 sum = src[((int64_t)n_chunks + first) * step];
#pragma unroll
      for (int k = 0; k < 4; k++) { sum.x += part[k][lane].x; sum.y += part[k][lane].y; sum.z += part[k][lane].z; sum.w += part[k][lane].w; }
      put(run.y, sum);
    }
    __syncthreads();
  }
}

// ---------------------------------------------------------------------------------------------
// Per-head RMS norm and rotation.  A head is held by LPH lanes, eight of its first half's elements and the eight half-split partners
// of these in a lane (so the rotation needs no other lane; a head narrower than 16 LPH leaves lanes idle).  Forward a lane group takes one
// head; the rotary factors, twice the bytes of its values, come from the caches (two heads of a token a group 114 us for 32768 x 40 x 128,
// four 123, one 113).
// ---------------------------------------------------------------------------------------------
// cos and sin of eight pairs of a row's position, NaN for a position outside the table (0 in lanes that hold nothing).
__device__ __forceinline__ void rotary_factors(const float* __restrict__ table, int64_t p, int64_t n_pos, int hd, int i0, bool active, float* cs, float* sn) {
#pragma unroll
  for (int e = 0; e < 8; e++) cs[e] = sn[e] = active ? __uint_as_float(0x7fc00000u) : 0.f;
  if (active && p >= 0 && p < n_pos) {
    load8(table + p * hd + i0, cs);
    load8(table + p * hd + hd / 2 + i0, sn);
  }
}

template <int LPH, bool ROTATE, bool PAST>
__global__ __launch_bounds__(256) void qk_norm_fwd_kernel(QkNormArgs a) {
  const uint32_t n_heads = a.n_q_heads + a.n_kv_heads, unit = blockIdx.x * (256 / LPH) + threadIdx.x / LPH;   // tokens times heads stay below 2^28
  const uint32_t token = unit / n_heads, h = unit - token * n_heads;
  const int64_t t = token;
  if (t >= a.t) return;
  const int i0 = (threadIdx.x % LPH) * 8, half = a.head_dim >> 1;
  const bool active = i0 < half;
  // Requested in front of everything else: loads come back in order, and the factors wait for the position (32768 x 40 x 128 118 -> 113 us).
  const int64_t at = ROTATE ? a.pos[t] : 0;
  uint4 xl = make_uint4(0, 0, 0, 0), xh = xl, gl = xl, gh = xl;
  if (active) {
    const bf16_t* x = (const bf16_t*)a.x + t * a.x_stride + (int64_t)h * a.head_dim + i0;
    const bf16_t* g = (const bf16_t*)((int)h < a.n_q_heads ? a.gamma_q : a.gamma_k) + i0;
    xl = load16_once(x);
    xh = load16_once(x + half);
    gl = *reinterpret_cast<const uint4*>(g);
    gh = *reinterpret_cast<const uint4*>(g + half);
  }
  float cs[8], sn[8], p[8], q[8], gp[8], gq[8], s = 0.f;
  if (ROTATE) rotary_factors(a.rope_table, at, a.n_pos, a.head_dim, i0, active, cs, sn);
  unpack8(xl, p);
  unpack8(xh, q);
  unpack8(gl, gp);
  unpack8(gh, gq);
#pragma unroll
  for (int e = 0; e < 8; e++) s = fmaf(p[e], p[e], fmaf(q[e], q[e], s));
  s = over_lanes<LPH, false>(s);
  if (!active) return;
  const float r = rsqrtf(s / (float)a.head_dim + a.eps);
#pragma unroll
  for (int e = 0; e < 8; e++) {
    const float np = p[e] * r * gp[e], nq = q[e] * r * gq[e];
    p[e] = ROTATE ? np * cs[e] - nq * sn[e] : np;
    q[e] = ROTATE ? nq * cs[e] + np * sn[e] : nq;
  }
  bf16_t* o = (bf16_t*)a.y + t * a.y_stride + (int64_t)h * a.head_dim + i0;
  store16<PAST>(o, pack8(p));
  store16<PAST>(o + half, pack8(q));
}

// Backward: with n = x r and g the gradient of what left the norm (dy turned back), d = g gamma:
// dx = r (d - n mean(d n)), dgamma = sum over tokens and heads of g n.  r is formed anew from x, which has to be read anyway.  The
// first q_blocks workgroups take the query heads, the others the key heads, each walking over its share of the tokens with the sums of
// g n in registers; it leaves one row of partial sums.
// Threads of a workgroup: its row of partial sums stands for more heads than with 256 (5125 x 50 x 128 38.0 and 38.7 us, 32768 x 40 x 128 189
// and 193; with 1024 37.6 and 190, but 22464 x 32 x 64 63 with 512 and 77).
constexpr int QK_THREADS = 512;
template <int LPH, bool ROTATE, bool PAST>
__global__ __launch_bounds__(QK_THREADS) void qk_norm_bwd_kernel(QkNormArgs a, float* __restrict__ partial_q, float* __restrict__ partial_k, int q_blocks) {
  constexpr int GROUPS = QK_THREADS / LPH;
  __shared__ float part[16][QK_THREADS + 4];   // [element][thread]; the sums are read a row of them at a time
  const bool is_q = (int)blockIdx.x < q_blocks;
  const int block = is_q ? blockIdx.x : blockIdx.x - q_blocks, blocks = is_q ? q_blocks : gridDim.x - q_blocks;
  const int l = threadIdx.x % LPH, i0 = l * 8, half = a.head_dim >> 1, col = (is_q ? 0 : a.n_q_heads * a.head_dim) + i0;
  const uint32_t n_heads = is_q ? a.n_q_heads : a.n_kv_heads, units = (uint32_t)a.t * n_heads;   // below 2^28, as forward
  const bool active = i0 < half;
  float g[16], dg[16];
#pragma unroll
  for (int e = 0; e < 16; e++) g[e] = dg[e] = 0.f;
  if (active) {
    const bf16_t* gamma = (const bf16_t*)(is_q ? a.gamma_q : a.gamma_k) + i0;
    load8(gamma, g);
    load8(gamma + half, g + 8);
  }
  const float inv = 1.f / (float)a.head_dim;
  for (uint32_t unit = block * GROUPS + threadIdx.x / LPH; unit < units; unit += blocks * GROUPS) {
    const uint32_t token = unit / n_heads;
    const int64_t t = token, c = col + (int64_t)(unit - token * n_heads) * a.head_dim, at = ROTATE ? a.pos[t] : 0;   // the position first, as forward
    uint4 xl = make_uint4(0, 0, 0, 0), xh = xl, dl = xl, dh = xl;
    if (active) {
      const bf16_t *px = (const bf16_t*)a.x + t * a.x_stride + c, *pd = (const bf16_t*)a.dy + t * a.dy_stride + c;
      xl = load16_once(px);
      xh = load16_once(px + half);
      dl = load16_once(pd);
      dh = load16_once(pd + half);
    }
    float cs[8], sn[8];
    if (ROTATE) rotary_factors(a.rope_table, at, a.n_pos, a.head_dim, i0, active, cs, sn);
    float x[16], d[16], s = 0.f;
    unpack8(xl, x);
    unpack8(xh, x + 8);
    unpack8(dl, d);
    unpack8(dh, d + 8);
    if (ROTATE)
#pragma unroll
      for (int e = 0; e < 8; e++) {
        const float p = d[e], q = d[e + 8];
        d[e] = p * cs[e] + q * sn[e];
        d[e + 8] = q * cs[e] - p * sn[e];
      }
#pragma unroll
    for (int e = 0; e < 16; e++) s = fmaf(x[e], x[e], s);
    const float r = rsqrtf(over_lanes<LPH, false>(s) * inv + a.eps);
    float m = 0.f;
#pragma unroll
    for (int e = 0; e < 16; e++) {
      x[e] *= r;
      const float dn = d[e] * x[e];
      dg[e] += dn;
      d[e] *= g[e];
      m = fmaf(dn, g[e], m);
    }
    m = over_lanes<LPH, false>(m) * inv;
    if (!active) continue;
#pragma unroll
    for (int e = 0; e < 16; e++) d[e] = r * (d[e] - x[e] * m);
    bf16_t* p = (bf16_t*)a.y + t * a.y_stride + c;
    store16<PAST>(p, pack8(d));
    store16<PAST>(p + half, pack8(d + 8));
  }
#pragma unroll
  for (int e = 0; e < 16; e++) part[e][threadIdx.x] = dg[e];
  __syncthreads();
  // a thread adds up an element and a lane of the head over the lane groups
  float* out = (is_q ? partial_q : partial_k) + (int64_t)block * a.head_dim;
  for (int c = threadIdx.x; c < 16 * LPH; c += QK_THREADS) {
    const int e = c / LPH, k = c % LPH, at = k * 8 + (e & 7) + (e < 8 ? 0 : half);
    float sum = 0.f;
#pragma unroll 8
    for (int g = 0; g < GROUPS; g++) sum += part[e][g * LPH + k];
    if (k * 8 < half) out[at] = sum;
  }
}

// ---------------------------------------------------------------------------------------------
// Loss over the vocabulary and its gradient, the row read once: GROUP threads hold up to NV vectors of eight logits each in registers
// from the maximum to the gradient; of a longer row the vectors behind the first GROUP * NV are read again for the gradient.  With the
// maximum m and L = log2(e):  s = sum 2^((x - m) L), loss = log2(s) / L + (m - x[target]), gradient = 2^((x - m) L - log2(s) + log2 |weight|)
// with the weight's sign, and |weight| (2^((x - m) L) / s - 1) at the target.  Every thread sums against its own maximum, so that one exchange
// joins (m, s) of all.
// (x L - m L in one instruction would lose rows of the type's lowest value: m L is beyond the largest number.)
// ---------------------------------------------------------------------------------------------
constexpr float LOG2E = 1.4426950408889634f;
typedef short s16x2 __attribute__((ext_vector_type(2)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float value(bf16_t v) { return __uint_as_float((uint32_t)v << 16); }
__device__ __forceinline__ float value(float v) { return v; }

// Vectors of the compiler's: of four single words it moved some to other registers behind a load, which waits for each by itself.
typedef float f32x4 __attribute__((ext_vector_type(4)));
template <typename E>
struct Logits8;
template <>
struct Logits8<bf16_t> {
  u32x4 u;
  __device__ __forceinline__ void load(const bf16_t* p) { u = *reinterpret_cast<const u32x4*>(p); }
  __device__ __forceinline__ void none() { u = 0xff80ff80u; }   // -inf
  __device__ __forceinline__ void get(float* f) const { unpack8(make_uint4(u[0], u[1], u[2], u[3]), f); }
  // Keeps the compiler from carrying unpacked values from one use to the next (16384 x 32000: 339 us, 343 without).
  __device__ __forceinline__ void settle() { asm volatile("" : "+v"(u)); }
  __device__ __forceinline__ void keep(int n) {   // the first n, 1 to 7
#pragma unroll
    for (int i = 0; i < 4; i++) u[i] = 2 * i + 1 < n ? u[i] : 2 * i < n ? (u[i] & 0xffffu) | 0xff800000u : 0xff80ff80u;
  }
};
template <>
struct Logits8<float> {
  f32x4 a, b;
  __device__ __forceinline__ void load(const float* p) { a = *reinterpret_cast<const f32x4*>(p); b = *reinterpret_cast<const f32x4*>(p + 4); }
  __device__ __forceinline__ void none() { a = b = -INFINITY; }
  __device__ __forceinline__ void settle() {}
  __device__ __forceinline__ void get(float* f) const {
#pragma unroll
    for (int i = 0; i < 8; i++) f[i] = i < 4 ? a[i & 3] : b[i & 3];
  }
  __device__ __forceinline__ void keep(int n) {
#pragma unroll
    for (int i = 0; i < 4; i++) { a[i] = i < n ? a[i] : -INFINITY; b[i] = i + 4 < n ? b[i] : -INFINITY; }
  }
};
// The largest of N vectors.  bf16 in pairs without unpacking: among 16-bit integers numbers at or above zero keep their order and are
// above all others; where there are none, the largest is the smallest unsigned one.
template <int N>
__device__ __forceinline__ float largest(const Logits8<bf16_t>* v) {
  s16x2 m = {-32768, -32768};
#pragma unroll
  for (int j = 0; j < N; j++)
    for (uint32_t w : {v[j].u[0], v[j].u[1], v[j].u[2], v[j].u[3]}) m = __builtin_elementwise_max(m, __builtin_bit_cast(s16x2, w));
  uint32_t top = (uint16_t)(m[0] > m[1] ? m[0] : m[1]);
  if (top & 0x8000u) {
    u16x2 n = {65535, 65535};
#pragma unroll
    for (int j = 0; j < N; j++)
      for (uint32_t w : {v[j].u[0], v[j].u[1], v[j].u[2], v[j].u[3]}) n = __builtin_elementwise_min(n, __builtin_bit_cast(u16x2, w));
    top = n[0] < n[1] ? n[0] : n[1];
  }
  return __uint_as_float(top << 16);
}
template <int N>
__device__ __forceinline__ float largest(const Logits8<float>* v) {
  float m = -INFINITY;
#pragma unroll
  for (int j = 0; j < N; j++) m = fmaxf(fmaxf(fmaxf(fmaxf(v[j].a[0], v[j].a[1]), fmaxf(v[j].a[2], v[j].a[3])), fmaxf(fmaxf(v[j].b[0], v[j].b[1]), fmaxf(v[j].b[2], v[j].b[3]))), m);
  return m;
}

// What a sum against the maximum `from` is worth against `to`, at or above it; a sum of nothing but -inf is none.
__device__ __forceinline__ float rescale(float from, float to) { return from == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((from - to) * LOG2E); }

// PARTS: grid z workgroups a row, each of which reads all of it for the sums and forms one step's gradient (1: all of it).
// A row is added up in the same order by all forms that may take it, which its length alone says: a thread's vectors in units that every one of them
// holds a whole number of, each against the maximum so far.  So its bits do not depend on the rows beside it, nor on what is asked for.
template <typename E, int GROUP, int NV, bool PAST, bool PARTS>
__global__ __launch_bounds__(GROUP < 256 ? 256 : GROUP) void xent_kernel(XentArgs a) {
  constexpr int BLOCK = GROUP < 256 ? 256 : GROUP, WAVES = GROUP / 64;
  __shared__ float2 wave_sums[WAVES];
  const int64_t row = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * (BLOCK / GROUP) + threadIdx.x / GROUP;
  if (row >= a.t) return;                              // the whole group
  const int tid = threadIdx.x % GROUP, nvec = (a.vocab + 7) >> 3, tail = a.vocab & 7;
  const int32_t target = a.targets[row];
  const E* x = (const E*)a.logits + row * a.stride;
  bf16_t* out = a.dlogits ? (bf16_t*)a.dlogits + row * a.dstride : nullptr;
  const int part = PARTS ? blockIdx.z : 0, parts = PARTS ? gridDim.z : 1;
  if (target < 0) {
    if (tid == 0 && part == 0) a.loss[row] = 0.f;
    if (out)
      for (int c = part * GROUP + tid; c < a.cols >> 3; c += parts * GROUP) store16<PAST>(out + (int64_t)c * 8, make_uint4(0, 0, 0, 0));
    return;
  }
  int at = target < a.vocab ? target : 0;
  asm volatile("" : "+v"(at));                         // as a vector load: the next scalar one would wait for it
  const E raw = x[at];
  asm volatile("" ::: "memory");                       // requested in front of the row: waited for behind it, it is 0.7 us of a row's 12 (131072 logits)
  constexpr int STEP = NV * GROUP, UNIT = GROUP < 1024 ? NV : sizeof(E) == 2 ? 4 : 2;
  static_assert(NV % UNIT == 0, "a step holds whole units");
  Logits8<E> v[NV];
  float m = -INFINITY, s = 0.f;
  for (int from = (nvec - 1) / STEP * STEP; from >= 0; from -= STEP) {   // the first vectors last: they are what stays
#pragma unroll
    for (int j = 0; j < NV; j++) {
      const int c = from + tid + j * GROUP;
      v[j].none();
      if (c < nvec) v[j].load(x + (int64_t)c * 8);
    }
    if (tail)
#pragma unroll
      for (int j = 0; j < NV; j++)
        if (from + tid + j * GROUP == nvec - 1) v[j].keep(tail);
#pragma unroll
    for (int u = NV - UNIT; u >= 0; u -= UNIT) {
      const float n = fmaxf(m, largest<UNIT>(v + u)), before = rescale(m, n);
      m = n;
      const float c = m == -INFINITY ? 0.f : m;        // nothing but -inf: s is 0 of no weight
#pragma unroll
      for (int j = u; j < u + UNIT; j++) {
        v[j].settle();
        float f[8];
        v[j].get(f);
#pragma unroll
        for (int e = 0; e < 8; e++) f[e] = __builtin_amdgcn_exp2f((f[e] - c) * LOG2E);
        const float sum = ((f[0] + f[1]) + (f[2] + f[3])) + ((f[4] + f[5]) + (f[6] + f[7]));
        s = j == u ? fmaf(s, before, sum) : s + sum;     // written out, as below: which products it fuses the compiler decides for each form
      }
    }
  }
  // all threads' (m, s) in one (without anything but -inf s ends as 0, and the differences of m below as NaN)
  float top = over_lanes<64, true>(m);
  s *= rescale(m, top);
  asm("" : "+v"(s));
  s = over_lanes<64, false>(s);
  if (WAVES > 1) {
    if ((threadIdx.x & 63) == 0) wave_sums[threadIdx.x >> 6] = make_float2(top, s);
    __syncthreads();
    float2 w[WAVES];
    float most = -INFINITY;
#pragma unroll
    for (int i = 0; i < WAVES; i++) { w[i] = wave_sums[i]; most = fmaxf(most, w[i].x); }
    top = most;
    s = 0.f;
#pragma unroll
    for (int i = 0; i < WAVES; i++) s = fmaf(w[i].y, rescale(w[i].x, top), s);
  }
  const float xt = target < a.vocab ? value(raw) : __uint_as_float(0x7fc00000u);
  if (tid == 0 && part == 0) a.loss[row] = (float)((double)log2f(s) * (1.0 / (double)LOG2E) + ((double)top - (double)xt));
  if (!out) return;
  const float weight = a.scale * (a.dloss ? a.dloss[row] : 1.f), size = fabsf(weight);
  const uint32_t sign = weight < 0.f ? 0x80008000u : 0u;
  const float shift = target < a.vocab ? log2f(size) - log2f(s) : __uint_as_float(0x7fc00000u);
  auto put = [&](int c, const Logits8<E>& u) {
    float f[8];
    u.get(f);
#pragma unroll
    for (int e = 0; e < 8; e++) f[e] = __builtin_amdgcn_exp2f(fmaf(f[e] - top, LOG2E, shift));
    // The target's own is formed without the weight in the exponent, which at a weight of 1/5000 is rounded to 2^-20 of p, and p - 1 of a
    // confident row is little more (1 - p = 1e-4, 1e-5: off by up to 1.3 and 12 % so, by 0.7 and 4 % now, as a p in fp32 is).  Here, where one
    // thread comes by: formed ahead by all, 2999 x 50257 fp32 took 1 % longer.
    if (c == target >> 3) {
      const float hit = size * fmaf(__builtin_amdgcn_exp2f((xt - top) * LOG2E), __builtin_amdgcn_rcpf(s), -1.f);
#pragma unroll
      for (int e = 0; e < 8; e++) f[e] = e == (target & 7) ? hit : f[e];
    }
    if (tail && c == nvec - 1)
#pragma unroll
      for (int e = 0; e < 8; e++) f[e] = e < tail ? f[e] : 0.f;
    uint4 r = pack8(f);
    r.x ^= sign; r.y ^= sign; r.z ^= sign; r.w ^= sign;
    store16<PAST>(out + (int64_t)c * 8, r);
  };
  if (part == 0) {
#pragma unroll
    for (int j = 0; j < NV; j++) {
      v[j].settle();
      if (tid + j * GROUP < nvec) put(tid + j * GROUP, v[j]);
    }
    for (int c = nvec + tid; c < a.cols >> 3; c += GROUP) store16<PAST>(out + (int64_t)c * 8, make_uint4(0, 0, 0, 0));
    if (PARTS && parts > 1) return;
  }
  for (int from = PARTS && part > 0 ? part * STEP : STEP; from < nvec; from += PARTS && parts > 1 ? nvec : STEP) {
#pragma unroll
    for (int j = 0; j < NV; j++)
      if (from + tid + j * GROUP < nvec) v[j].load(x + (int64_t)(from + tid + j * GROUP) * 8);
#pragma unroll
    for (int j = 0; j < NV; j++)
      if (from + tid + j * GROUP < nvec) put(from + tid + j * GROUP, v[j]);
  }
}

}  // namespace

hipError_t launch_embed_fwd(const void* table, int table_fp32, const int32_t* ids, void* y, int64_t t, int64_t vocab, int64_t d, int64_t y_stride,
                            float scale, hipStream_t s) {
  if (t == 0) return hipSuccess;
  const int nvec = (int)(d / 8), lpr = nvec <= 8 ? 8 : nvec <= 16 ? 16 : nvec <= 32 ? 32 : 64;
  const dim3 grid((unsigned)std::min<int64_t>(ceil_div(t, 256 / lpr), MAX_GRID), (unsigned)ceil_div(nvec, EMBED_VECS * lpr));
  ProfScope prof(PROF_ELEMENTWISE, (double)t * (double)d * (table_fp32 ? 6.0 : 4.0), s);
#define CALL(E, L, P) hipLaunchKernelGGL((embed_fwd_kernel<E, L, P>), grid, dim3(256), 0, s, (const E*)table, ids, (bf16_t*)y, t, vocab, nvec, y_stride, scale)
#define CALL_LPR(E, P) \
  do { if (lpr == 8) CALL(E, 8, P); else if (lpr == 16) CALL(E, 16, P); else if (lpr == 32) CALL(E, 32, P); else CALL(E, 64, P); } while (0)
#define CALL_PAST(E) do { if (t * d * 2 >= NT_BYTES) CALL_LPR(E, true); else CALL_LPR(E, false); } while (0)
  if (table_fp32) CALL_PAST(float); else CALL_PAST(bf16_t);
#undef CALL_PAST
#undef CALL_LPR
#undef CALL
  return hipGetLastError();
}

namespace {
// How the sorted tokens are cut: into chunks of 8, 16 or 32, the shortest that make at most 16384 wavefronts.
struct EmbedCut { int lpr, slices, chunk; int64_t chunks; };
EmbedCut embed_cut(int64_t t, int64_t d) {
  EmbedCut c;
  const int64_t nvec = d / 8;
  c.lpr = nvec <= 8 ? 8 : nvec <= 16 ? 16 : nvec <= 32 ? 32 : 64;
  c.slices = (int)ceil_div(nvec, c.lpr);
  c.chunk = 8;
  while (c.chunk < 32 && ceil_div(t, c.chunk) * c.slices * c.lpr > 16384 * 64) c.chunk *= 2;
  c.chunks = ceil_div(t, c.chunk);
  return c;
}
int embed_log2_buckets(int64_t vocab) {
  int n = 8;
  while (ceil_div(vocab, (int64_t)1 << n) > SORT_RANGE) n++;
  return n;
}
size_t align256(size_t n) { return (n + 255) / 256 * 256; }
}  // namespace

// The token order, its ids, their number, a bit for every id; two rows of partial sums a chunk.  Not less for fewer tokens: shorter chunks are never more
// than 16384 wavefronts' worth.  (EMBED_FEW tokens and fewer leave it alone.)
size_t embed_bwd_ws_bytes(int64_t t, int64_t vocab, int64_t d) {
  const EmbedCut c = embed_cut(t, d);
  const int64_t most = std::max(ceil_div(t, 32), std::min<int64_t>(ceil_div(t, 8), 16384 * 64 / c.lpr / c.slices));
  return 2 * align256((size_t)t * 4) + 256 + ((size_t)SORT_WAVES * 8 << embed_log2_buckets(vocab)) + (size_t)2 * most * d * 4;
}

hipError_t launch_embed_bwd(const void* dy, const int32_t* ids, float* dtable, int accumulate, int64_t t, int64_t vocab, int64_t d, int64_t dy_stride,
                            float scale, void* ws, hipStream_t s) {
  const EmbedCut c = embed_cut(t, d);
  const int nvec = (int)(d / 8), log2_buckets = embed_log2_buckets(vocab);
  const bool few = t <= EMBED_FEW;
  char* w = (char*)ws;
  int32_t *order = (int32_t*)w, *keys = (int32_t*)(w + align256((size_t)t * 4)), *total = (int32_t*)(w + 2 * align256((size_t)t * 4));
  uint64_t* absent = (uint64_t*)((char*)total + 256);
  float* partial = (float*)((char*)absent + ((size_t)SORT_WAVES * 8 << log2_buckets));
  if (!few) {
    ProfScope prof(PROF_ELEMENTWISE, 0.0, s);
    hipLaunchKernelGGL(embed_sort_kernel, dim3(1u << log2_buckets), dim3(64 * SORT_WAVES), 0, s, ids, (int)t, (int)vocab, log2_buckets, order, keys, total,
                       absent);
  }
  const int64_t quads = vocab * nvec * 2, clear_blocks = accumulate ? 0 : ceil_div(quads, 256);
  if (few && !accumulate) {
    ProfScope prof(PROF_ELEMENTWISE, (double)vocab * (double)d * 4.0, s);
    const dim3 grid((unsigned)std::min(clear_blocks, MAX_GRID), (unsigned)ceil_div(clear_blocks, MAX_GRID));
    hipLaunchKernelGGL(embed_clear_kernel, grid, dim3(256), 0, s, dtable, nvec, quads, ids, (int)t);
  }
  if (t == 0) return hipGetLastError();
  if (few) {
    ProfScope prof(PROF_ELEMENTWISE, (double)t * (double)d * 2.0, s);
    const int slices = (int)ceil_div(nvec, 64);
    hipLaunchKernelGGL(embed_few_kernel, dim3((unsigned)ceil_div(t * slices, 4)), dim3(256), 0, s, (const bf16_t*)dy, ids, dtable, (int)t, (int)vocab, slices,
                       nvec, dy_stride, scale, accumulate);
    return hipGetLastError();
  }
  {
    ProfScope prof(PROF_ELEMENTWISE, (double)t * (double)d * 2.0 + (accumulate ? 0.0 : (double)vocab * (double)d * 4.0), s);
    // The sums' workgroups all in the grid's first row.
    const int64_t sum_blocks = ceil_div(c.chunks * c.slices, 256 / c.lpr), blocks = sum_blocks + clear_blocks;
    const int64_t along = std::max(sum_blocks, std::min(blocks, MAX_GRID));
    const dim3 grid((unsigned)along, (unsigned)ceil_div(blocks, along));
#define CALL(L, A)                                                                                                                                  \
  hipLaunchKernelGGL((embed_sum_kernel<L, A>), grid, dim3(256), 0, s, (const bf16_t*)dy, order, keys, total, dtable, partial, c.chunk, (int)c.chunks, \
                     c.slices, nvec, dy_stride, scale, (uint32_t)sum_blocks, absent, log2_buckets, quads)
#define CALL_LPR(A) \
  do { if (c.lpr == 8) CALL(8, A); else if (c.lpr == 16) CALL(16, A); else if (c.lpr == 32) CALL(32, A); else CALL(64, A); } while (0)
    if (accumulate) CALL_LPR(true); else CALL_LPR(false);
#undef CALL_LPR
#undef CALL
  }
  ProfScope prof(PROF_ELEMENTWISE, 0.0, s);
  const int slices = (int)ceil_div(nvec, 32);
  hipLaunchKernelGGL(embed_join_kernel, dim3((unsigned)(ceil_div(c.chunks, 4) * slices)), dim3(256), 0, s, keys, total, dtable, partial, c.chunk,
                     (int)c.chunks, slices, nvec, scale, accumulate);
  return hipGetLastError();
}

namespace {
int qk_lanes(int head_dim) { return head_dim <= 32 ? 2 : head_dim <= 64 ? 4 : head_dim <= 128 ? 8 : 16; }
// Workgroups of the backward pass that take `heads` of `all` heads: a lane group walks over some eight heads, within 512 to 4096 workgroups
// for all (32768 x 40 x 128: 2048 195 us, 2560 189; fewer leave the memory idle, more leave more partial sums: 8000 x 12 x 256 with three
// heads a lane group 38.4, with six 32.7).
int64_t qk_bwd_blocks(int64_t t, int heads, int all, int head_dim) {
  const int64_t groups = QK_THREADS / qk_lanes(head_dim), most = std::min<int64_t>(4096, std::max<int64_t>(512, t * all / (8 * groups)));
  return std::max<int64_t>(1, std::min<int64_t>(ceil_div(t * heads, groups), ceil_div(most * heads, all)));
}
}  // namespace

hipError_t launch_qk_norm_fwd(const QkNormArgs& a, hipStream_t s) {
  if (a.t == 0) return hipSuccess;
  const int n_heads = a.n_q_heads + a.n_kv_heads, lph = qk_lanes(a.head_dim);
  ProfScope prof(PROF_ELEMENTWISE, 4.0 * (double)a.t * n_heads * a.head_dim, s);
  const dim3 grid((unsigned)ceil_div(a.t * n_heads, 256 / lph));
  const bool past = a.t * n_heads * a.head_dim * 2 >= NT_BYTES;
#define CALL(L, R)                                                                                    \
  do {                                                                                                \
    if (past) hipLaunchKernelGGL((qk_norm_fwd_kernel<L, R, true>), grid, dim3(256), 0, s, a);         \
    else hipLaunchKernelGGL((qk_norm_fwd_kernel<L, R, false>), grid, dim3(256), 0, s, a);             \
  } while (0)
#define CALL_LPH(R) do { if (lph == 2) CALL(2, R); else if (lph == 4) CALL(4, R); else if (lph == 8) CALL(8, R); else CALL(16, R); } while (0)
  if (a.rope_table) CALL_LPH(true); else CALL_LPH(false);
#undef CALL_LPH
#undef CALL
  return hipGetLastError();
}

size_t qk_norm_bwd_partial_floats(int64_t t, int n_q_heads, int n_kv_heads, int head_dim) {
  const int all = n_q_heads + n_kv_heads;
  return (size_t)((qk_bwd_blocks(t, n_q_heads, all, head_dim) + qk_bwd_blocks(t, n_kv_heads, all, head_dim)) * head_dim);
}

hipError_t launch_qk_norm_bwd(const QkNormArgs& a, float* dgamma_q, float* dgamma_k, PartialSums& sums, hipStream_t s) {
  const int all = a.n_q_heads + a.n_kv_heads, lph = qk_lanes(a.head_dim);
  const int64_t bq = qk_bwd_blocks(a.t, a.n_q_heads, all, a.head_dim), bk = qk_bwd_blocks(a.t, a.n_kv_heads, all, a.head_dim);
  const bool past = a.t * all * a.head_dim * 2 >= NT_BYTES;
  float *pq = nullptr, *pk = nullptr;
  ProfScope prof(PROF_ELEMENTWISE, 6.0 * (double)a.t * all * a.head_dim, s);
#define CALL(L, R, BLOCKS, Q)                                                                                                                         \
  do {                                                                                                                                               \
    if (past) hipLaunchKernelGGL((qk_norm_bwd_kernel<L, R, true>), dim3((unsigned)(BLOCKS)), dim3(QK_THREADS), 0, s, a, pq, pk, (int)(Q));                  \
    else hipLaunchKernelGGL((qk_norm_bwd_kernel<L, R, false>), dim3((unsigned)(BLOCKS)), dim3(QK_THREADS), 0, s, a, pq, pk, (int)(Q));                      \
  } while (0)
#define CALL_R(R, BLOCKS, Q) \
  do { if (lph == 2) CALL(2, R, BLOCKS, Q); else if (lph == 4) CALL(4, R, BLOCKS, Q); else if (lph == 8) CALL(8, R, BLOCKS, Q); else CALL(16, R, BLOCKS, Q); } while (0)
#define CALL_LPH(BLOCKS, Q) \
  do { if (a.rope_table) CALL_R(true, BLOCKS, Q); else CALL_R(false, BLOCKS, Q); } while (0)
  hipError_t e = sums.room((size_t)(bq + bk) * a.head_dim, a.head_dim, {dgamma_q, dgamma_k}, s);
  if (e == hipSuccess) e = sums.take(bq, a.head_dim, {dgamma_q}, s, &pq);
  if (e != hipSuccess) return e;
  const int64_t bytes = (int64_t)a.head_dim * 4;
  if (ranges_overlap(dgamma_q, bytes, dgamma_k, bytes)) {   // one gain for both: the key heads' sums are added to the query heads' in any case
    CALL_LPH(bq, bq);
    if ((e = sums.flush(s)) != hipSuccess) return e;
    const int accumulate = sums.accumulate;
    sums.accumulate = 1;
    e = sums.take(bk, a.head_dim, {dgamma_k}, s, &pk);
    if (e == hipSuccess) {
      CALL_LPH(bk, 0);
      e = sums.flush(s);
    }
    sums.accumulate = accumulate;
    if (e != hipSuccess) return e;
  } else {
    if ((e = sums.take(bk, a.head_dim, {dgamma_k}, s, &pk)) != hipSuccess) return e;
    CALL_LPH(bq + bk, bq);
  }
#undef CALL_LPH
#undef CALL_R
#undef CALL
  return hipGetLastError();
}

hipError_t launch_xent(const XentArgs& a, int logits_fp32, hipStream_t s) {
  if (a.t == 0) return hipSuccess;
  ProfScope prof(PROF_ELEMENTWISE, (double)a.t * ((logits_fp32 ? 4.0 : 2.0) * (double)a.vocab + (a.dlogits ? 2.0 * (double)a.cols : 0.0)), s);
  const int64_t nvec = ceil_div(a.vocab, 8), blocks = nvec <= 256 ? ceil_div(a.t, 4) : a.t;
  dim3 grid((unsigned)std::min(blocks, MAX_GRID), (unsigned)ceil_div(blocks, MAX_GRID));
  const bool past = a.dlogits && a.t * a.cols * 2 >= NT_BYTES;
#define CALL(E, GROUP, NV)                                                                                                  \
  do {                                                                                                                      \
    if (past) hipLaunchKernelGGL((xent_kernel<E, GROUP, NV, true, false>), grid, dim3(GROUP < 256 ? 256 : GROUP), 0, s, a); \
    else hipLaunchKernelGGL((xent_kernel<E, GROUP, NV, false, false>), grid, dim3(GROUP < 256 ? 256 : GROUP), 0, s, a);     \
  } while (0)
  // Threads times vectors that hold a row with the least idle and two workgroups a CU at least where that goes; TB/s of what a pass
  // reads and writes, rows of bf16: 1000 columns 64x2 5.7, 64x4 4.4; 2000 64x4 6.6, 256x2 3.7; 4096 256x2 5.7, 256x4 4.9; 8192 256x4 5.8, 512x4 5.0;
  // 16384 512x4 5.4, 256x8 5.5; 24000 512x8 5.6, 1024x4 5.7; 27000 and 32000 1024x4 5.7 and 6.2, 512x8 5.2 and 5.5; 65536 512x16 5.5, 1024x8 5.1; 96000 (a third
  // of the row read again) 512x16 5.3, 1024x20 4.7; 131072 1024x20 5.1, 512x16 4.9; 256000 1024x20 4.7.  fp32: 1000 64x2 5.8; 4096 256x4 5.9; 16384
  // 512x8 6.2, 1024x8 3.7; 65536 1024x10 5.4, 512x8 5.2; 131072 1024x10 4.7, 512x16 4.6.
  // Few long rows: as many workgroups a row as it has steps, while every one has a CU to itself.  A lone workgroup is bound by its own exponentials,
  // two a logit, of which this spares it most of the second (131072 logits, one row 18.0 -> 14.2 us, fp32 17.7 -> 11.9, 64 rows 21.5 -> 17.2;
  // 260000, 64 rows 37.4 -> 25.9).  Not over the logits themselves, which the other workgroups of the row still read: in place the shorter steps
  // alone are worth 18.3 us for 18.7, 64 rows 21.3 for 21.8, 32 rows of 196608 28.3 for 34.1.
  // The loss alone has nothing to hold a row for and takes shorter steps for any number of rows: 8192 x 131072 350 us for 410, 300 rows 23.7 for 28.4,
  // fp32 2999 x 50257 105 for 111, 1000 x 131072 95 for 104.  (3000 x 70000 113 for 82: those keep 512x16.)
  const int64_t parts = ceil_div(nvec, logits_fp32 ? 4 * 1024 : 8 * 1024);
  if (parts > 1 && (a.t * parts <= 256 || (!a.dlogits && (logits_fp32 || nvec > 12288)))) {
    if (a.dlogits && a.dlogits != a.logits) grid.z = (unsigned)parts;
    if (logits_fp32)
      hipLaunchKernelGGL((xent_kernel<float, 1024, 4, false, true>), grid, dim3(1024), 0, s, a);
    else if (nvec <= 12288)
      hipLaunchKernelGGL((xent_kernel<bf16_t, 512, 16, false, true>), grid, dim3(512), 0, s, a);
    else
      hipLaunchKernelGGL((xent_kernel<bf16_t, 1024, 8, false, true>), grid, dim3(1024), 0, s, a);
  } else if (logits_fp32) {
    if (nvec <= 128) CALL(float, 64, 2); else if (nvec <= 256) CALL(float, 64, 4); else if (nvec <= 1024) CALL(float, 256, 4);
    else if (nvec <= 4096) CALL(float, 512, 8); else CALL(float, 1024, 10);
  } else {
    if (nvec <= 128) CALL(bf16_t, 64, 2); else if (nvec <= 256) CALL(bf16_t, 64, 4); else if (nvec <= 512) CALL(bf16_t, 256, 2);
    else if (nvec <= 1024) CALL(bf16_t, 256, 4); else if (nvec <= 2048) CALL(bf16_t, 512, 4); else if (nvec <= 3300) CALL(bf16_t, 512, 8);
    else if (nvec <= 4096) CALL(bf16_t, 1024, 4); else if (nvec <= 12288) CALL(bf16_t, 512, 16); else CALL(bf16_t, 1024, 20);
  }
#undef CALL
  return hipGetLastError();
}

}  // namespace mllm
