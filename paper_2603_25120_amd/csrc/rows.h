// What the memory-bound kernels of rows of values share: 16-byte accesses, stores past the caches, exchanges between lanes.
#pragma once
#include "common.h"

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

// n / divisor for n < 2^31, by multiplication.
struct Division { uint32_t divisor, factor, shift; };
inline Division division(uint32_t divisor) {
  uint32_t shift = 0;
  while (((uint64_t)1 << shift) < divisor) shift++;
  return {divisor, (uint32_t)((((uint64_t)1 << 32) * (((uint64_t)1 << shift) - divisor)) / divisor + 1), shift};
}
__device__ __forceinline__ uint32_t divide(uint32_t n, const Division& d) { return (__umulhi(n, d.factor) + n) >> d.shift; }

}  // namespace
}  // namespace mllm
