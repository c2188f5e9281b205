// Activations kept in 8 bits from the forward to the backward pass, and their use there.  A row is cut into blocks of 32 neighbouring columns; a
// block has an exponent e, the smallest one (from -112 on) with max |x| <= L 2^e, and its values are x 2^-e rounded to the nearest of the format:
//   int8   whole numbers up to L = 127: an error of at most 2^e / 2, 1/254 of the block's largest value or 1/127 just above a power of two
//   e4m3   L = 448: an error of at most 2^-4 of the value itself, down to 2^-10 2^e
// Powers of two, so that x 2^-e and the way back are exact whatever computes them, and the rounding is the format's alone; the stored byte is
// e + 127.  A block that holds an infinity or a NaN has the byte 255 and comes back as NaN, all of it.
// Bound by memory: a thread has eight columns, four neighbouring lanes a block, whose largest magnitude they exchange inside the vector unit.  Measured (us, TB/s of what
// has to be moved): 8192 x 14336 SwiGLU forward 150, 6.3, backward with the activation again 187, 6.3; GELU 98, 6.0 and 131, 6.3; keeping a matrix 60,
// 5.9, loading it 57, 6.3; 777 x 4096 SwiGLU 6.1 and 7.6 (results past the caches too 5.8 and 5.9, but the products that follow read them).
#include <algorithm>

#include "common.h"
#include "kernels.h"
#include "rows.h"

namespace mllm {

namespace {

constexpr int INT8 = 0, E4M3 = 1;
constexpr int LOWEST = -112;          // below it the values of a block are rounded to multiples of 2^-112 (e4m3 2^-121), so that no step meets subnormal numbers

// The largest magnitude of eight bf16 values, as the bits of a bf16: infinity and NaN are the largest ones.
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ u16x2 larger(uint32_t a, uint32_t b) {
  return __builtin_elementwise_max(__builtin_bit_cast(u16x2, a & 0x7fff7fffu), __builtin_bit_cast(u16x2, b & 0x7fff7fffu));
}
__device__ __forceinline__ uint32_t lane_xor(uint32_t v, bool two) {
  return (uint32_t)(two ? __builtin_amdgcn_update_dpp(0, (int)v, 0x4e, 0xf, 0xf, true) : __builtin_amdgcn_update_dpp(0, (int)v, 0xb1, 0xf, 0xf, true));
}
__device__ __forceinline__ uint32_t block_top(const uint4& u) {
  u16x2 m = __builtin_elementwise_max(larger(u.x, u.y), larger(u.z, u.w));
  uint32_t v = max((uint32_t)m[0], (uint32_t)m[1]);
  v = max(v, lane_xor(v, false));
  return max(v, lane_xor(v, true));
}

// The block's exponent byte.  top = 1.m 2^E: 127 2^e takes it in from e = E - 6 on unless m is all ones, 448 2^e from E - 8 on up to m = .75.
template <int FORMAT>
__device__ __forceinline__ uint32_t exponent_byte(uint32_t top) {
  const int E = (int)(top >> 7) - 127, m = (int)(top & 127);
  const int e = max(FORMAT == INT8 ? E - 6 + (m == 127) : E - 8 + (m > 96), LOWEST);
  return top >= 0x7f80u ? 255u : (uint32_t)(e + 127);
}
__device__ __forceinline__ float scale_of(uint32_t byte) { return byte == 255u ? __uint_as_float(0x7fc00000u) : __uint_as_float(byte << 23); }

// Eight values in 8 bits, and back.
template <int FORMAT>
__device__ __forceinline__ uint2 to8(const uint4& u, uint32_t byte) {
  const float by = byte == 255u ? 0.f : __uint_as_float((254u - byte) << 23);
  float f[8];
  unpack8(u, f);
  uint2 q = make_uint2(0, 0);
  if (byte == 255u) return q;
  if (FORMAT == INT8) {
    uint32_t b[8];
#pragma unroll
    for (int e = 0; e < 8; e++) b[e] = __float_as_uint(fmaf(f[e], by, 12582912.f));     // + 1.5 2^23: the sum's last bits are the nearest whole number
#pragma unroll
    for (int k = 0; k < 2; k++) {
      const uint32_t lo = __builtin_amdgcn_perm(b[4 * k + 1], b[4 * k], 0x0c0c0400u), hi = __builtin_amdgcn_perm(b[4 * k + 3], b[4 * k + 2], 0x0c0c0400u);
      (k ? q.y : q.x) = lo | hi << 16;
    }
  } else {
#pragma unroll
    for (int k = 0; k < 2; k++) {
      int w = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * k] * by, f[4 * k + 1] * by, 0, false);
      w = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * k + 2] * by, f[4 * k + 3] * by, w, true);
      (k ? q.y : q.x) = (uint32_t)w;
    }
  }
  return q;
}
template <int FORMAT>
__device__ __forceinline__ void from8(const uint2& q, uint32_t byte, float* f) {
  const float s = scale_of(byte);
#pragma unroll
  for (int k = 0; k < 2; k++) {
    const uint32_t w = k ? q.y : q.x;
    if (FORMAT == INT8) {
#pragma unroll
      for (int e = 0; e < 4; e++) f[4 * k + e] = (float)((int32_t)(w << (24 - 8 * e)) >> 24) * s;
    } else {
      const f32x2_t lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
      f[4 * k] = lo[0] * s; f[4 * k + 1] = lo[1] * s; f[4 * k + 2] = hi[0] * s; f[4 * k + 3] = hi[1] * s;
    }
  }
}

// ---------------------------------------------------------------------------------------------
// Activations from what they are taken of, relative to their own size also where they are small.
// ---------------------------------------------------------------------------------------------
__device__ __forceinline__ float logistic(float v) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.4426950408889634f * v)); }
// The normal distribution's share below v: of -|v| it is exp(-v^2 / 2) t P(t), t = 1 / (1 + 0.36 |v|), P fitted to 9e-7 of it (least squares on
// 0 <= |v| <= 14, reweighted towards the largest error); phi: its density.
__device__ __forceinline__ float normal_below(float v, float& phi) {
  const float u = fabsf(v), t = __builtin_amdgcn_rcpf(fmaf(0.36f, u, 1.f)), e = __builtin_amdgcn_exp2f(-0.7213475204444817f * v * v);
  float p = fmaf(0.0470579304f, t, -0.179770187f);
  p = fmaf(p, t, 0.180961311f);
  p = fmaf(p, t, 0.0265444126f);
  p = fmaf(p, t, 0.139721021f);
  p = fmaf(p, t, 0.141772136f);
  p = fmaf(p, t, 0.14371307f);
  p *= t * e;
  phi = 0.3989422804014327f * e;
  return v < 0.f ? p : 1.f - p;
}
constexpr int GELU_ERF = 0, GELU_TANH = 1, SWIGLU = 2;
// The activation of one value and its slope; for SwiGLU of gate and up, with both slopes.
template <int ACT>
__device__ __forceinline__ float activate(float v, float up, float& slope, float& slope_up) {
  if (ACT == SWIGLU) {
    const float s = logistic(v), silu = v * s;
    slope = up * fmaf(silu, 1.f - s, s);
    slope_up = silu;
    return silu * up;
  }
  if (ACT == GELU_ERF) {
    float phi;
    const float below = normal_below(v, phi);
    slope = fmaf(v, phi, below);
    return v * below;
  }
  // 0.5 v (1 + tanh u) = v logistic(2 u), u = sqrt(2 / pi) (v + 0.044715 v^3)
  const float v2 = fminf(v * v, 1e30f), s = logistic(1.5957691216057308f * v * fmaf(0.044715f, v2, 1.f));
  slope = fmaf(v * s * (1.f - s), 1.5957691216057308f * fmaf(0.134145f, v2, 1.f), s);
  return v * s;
}

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
// What is kept is read again in the backward pass only: past the caches, whatever its size (SwiGLU forward, 8192 x 4096 47.1 -> 41.6 us).
__device__ __forceinline__ void store8_past(void* p, const uint2& v) {
  const u32x2 w = {v.x, v.y};
  __builtin_nontemporal_store(w, reinterpret_cast<u32x2*>(p));
}
__device__ __forceinline__ uint2 load8_once(const void* p) {
  const u32x2 w = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(p));
  return make_uint2(w[0], w[1]);
}

// ---------------------------------------------------------------------------------------------
// Items of a launch: (row, eight columns), rows filled up to whole blocks of four lanes.
// ---------------------------------------------------------------------------------------------
struct Items { Division per_row; uint32_t count; int nvec; };   // vectors of a row with those behind its end; of the launch; of a row

template <int FORMAT>
__global__ __launch_bounds__(256) void keep8_kernel(const bf16_t* __restrict__ x, uint8_t* __restrict__ q, uint8_t* __restrict__ exponent, Items it,
                                                    int64_t x_stride) {
  const uint32_t i = blockIdx.x * 256u + threadIdx.x, row = divide(i, it.per_row), c = i - row * it.per_row.divisor;
  const bool there = i < it.count && (int)c < it.nvec;
  uint4 u = make_uint4(0, 0, 0, 0);
  if (there) u = load16_once(x + (int64_t)row * x_stride + 8 * c);
  const uint32_t byte = exponent_byte<FORMAT>(block_top(u));
  if (!there) return;
  store8_past(q + ((int64_t)row * it.nvec + c) * 8, to8<FORMAT>(u, byte));
  if ((c & 3) == 0) exponent[(int64_t)row * (it.per_row.divisor >> 2) + (c >> 2)] = (uint8_t)byte;
}

template <int FORMAT, bool PAST>
__global__ __launch_bounds__(256) void keep8_load_kernel(const uint8_t* __restrict__ q, const uint8_t* __restrict__ exponent, bf16_t* __restrict__ y, Items it,
                                                         int64_t y_stride) {
  const uint32_t i = blockIdx.x * 256u + threadIdx.x, row = divide(i, it.per_row), c = i - row * it.per_row.divisor;
  if (i >= it.count || (int)c >= it.nvec) return;
  float f[8];
  from8<FORMAT>(load8_once(q + ((int64_t)row * it.nvec + c) * 8), exponent[(int64_t)row * (it.per_row.divisor >> 2) + (c >> 2)], f);
  store16<PAST>(y + (int64_t)row * y_stride + 8 * c, pack8(f));
}

// What the gradients of a linear map read where its output width is no multiple of 64: x from its kept values, and dy and w with rows of zeros up to one, in one launch.
struct Padded { const bf16_t* src; bf16_t* dst; Division per_row; uint32_t count, first; int nvec; };   // first: its first workgroup; nvec: of a row of src
template <int FORMAT>
__global__ __launch_bounds__(256) void linear_operands_kernel(const uint8_t* __restrict__ q, const uint8_t* __restrict__ exponent, bf16_t* __restrict__ x, Items it,
                                                              Padded dy, Padded w) {
  if (blockIdx.x >= dy.first) {
    const Padded p = blockIdx.x >= w.first ? w : dy;
    const uint32_t i = (blockIdx.x - p.first) * 256u + threadIdx.x, row = divide(i, p.per_row), c = i - row * p.per_row.divisor;
    if (i >= p.count) return;
    uint4 u = make_uint4(0, 0, 0, 0);
    if ((int)c < p.nvec) u = *reinterpret_cast<const uint4*>(p.src + ((int64_t)row * p.nvec + c) * 8);
    store16<false>(p.dst + (int64_t)i * 8, u);
    return;
  }
  const uint32_t i = blockIdx.x * 256u + threadIdx.x, row = divide(i, it.per_row), c = i - row * it.per_row.divisor;
  if (i >= it.count || (int)c >= it.nvec) return;
  float f[8];
  from8<FORMAT>(load8_once(q + ((int64_t)row * it.nvec + c) * 8), exponent[(int64_t)row * (it.per_row.divisor >> 2) + (c >> 2)], f);
  store16<false>(x + ((int64_t)row * it.nvec + c) * 8, pack8(f));
}

// a = act(pre), and pre in 8 bits.  SwiGLU: pre = [gate | up], each half a matrix of its own blocks.
template <int ACT, int FORMAT, bool PAST>
__global__ __launch_bounds__(256) void act_fwd_keep8_kernel(const bf16_t* __restrict__ pre, bf16_t* __restrict__ a, uint8_t* __restrict__ q,
                                                            uint8_t* __restrict__ exponent, Items it) {
  constexpr int H = ACT == SWIGLU ? 2 : 1;
  const uint32_t i = blockIdx.x * 256u + threadIdx.x, row = divide(i, it.per_row), c = i - row * it.per_row.divisor;
  const bool there = i < it.count && (int)c < it.nvec;
  const int blocks = it.per_row.divisor >> 2;
  uint4 u[H];
#pragma unroll
  for (int h = 0; h < H; h++) {
    u[h] = make_uint4(0, 0, 0, 0);
    if (there) u[h] = load16_once(pre + (((int64_t)row * H + h) * it.nvec + c) * 8);
  }
#pragma unroll
  for (int h = 0; h < H; h++) {
    const uint32_t byte = exponent_byte<FORMAT>(block_top(u[h]));
    if (!there) continue;
    store8_past(q + (((int64_t)row * H + h) * it.nvec + c) * 8, to8<FORMAT>(u[h], byte));
    if ((c & 3) == 0) exponent[((int64_t)row * H + h) * blocks + (c >> 2)] = (uint8_t)byte;
  }
  if (!there) return;
  float f[H][8], v[8];
#pragma unroll
  for (int h = 0; h < H; h++) unpack8(u[h], f[h]);
#pragma unroll
  for (int e = 0; e < 8; e++) {
    float slope, slope_up;
    v[e] = activate<ACT>(f[0][e], f[H - 1][e], slope, slope_up);
  }
  store16<PAST>(a + ((int64_t)row * it.nvec + c) * 8, pack8(v));
}

// dpre from da and pre in 8 bits, and (a not null) the activation of those; da and dpre null: the activation alone.
template <int ACT, int FORMAT, bool PAST>
__global__ __launch_bounds__(256) void act_bwd_keep8_kernel(const bf16_t* da, const uint8_t* __restrict__ q, const uint8_t* __restrict__ exponent,
                                                            bf16_t* dpre, bf16_t* __restrict__ a, Items it) {
  constexpr int H = ACT == SWIGLU ? 2 : 1;
  const uint32_t i = blockIdx.x * 256u + threadIdx.x, row = divide(i, it.per_row), c = i - row * it.per_row.divisor;
  if (i >= it.count || (int)c >= it.nvec) return;
  const int blocks = it.per_row.divisor >> 2;
  float f[H][8], d[8], v[8];
  uint4 ud = make_uint4(0, 0, 0, 0);
  if (da) ud = load16_once(da + ((int64_t)row * it.nvec + c) * 8);
#pragma unroll
  for (int h = 0; h < H; h++)
    from8<FORMAT>(load8_once(q + (((int64_t)row * H + h) * it.nvec + c) * 8), exponent[((int64_t)row * H + h) * blocks + (c >> 2)], f[h]);
  unpack8(ud, d);
#pragma unroll
  for (int e = 0; e < 8; e++) {
    float slope, slope_up = 0.f;
    v[e] = activate<ACT>(f[0][e], f[H - 1][e], slope, slope_up);
    f[0][e] = d[e] * slope;
    if (H == 2) f[H - 1][e] = d[e] * slope_up;
  }
  if (a) store16<PAST>(a + ((int64_t)row * it.nvec + c) * 8, pack8(v));
  if (dpre)
#pragma unroll
    for (int h = 0; h < H; h++) store16<PAST>(dpre + (((int64_t)row * H + h) * it.nvec + c) * 8, pack8(f[h]));
}

template <bool PAST>
auto act_fwd_kernel(int act, int format) {
  return act == GELU_ERF    ? (format == INT8 ? act_fwd_keep8_kernel<GELU_ERF, INT8, PAST> : act_fwd_keep8_kernel<GELU_ERF, E4M3, PAST>)
         : act == GELU_TANH ? (format == INT8 ? act_fwd_keep8_kernel<GELU_TANH, INT8, PAST> : act_fwd_keep8_kernel<GELU_TANH, E4M3, PAST>)
                            : (format == INT8 ? act_fwd_keep8_kernel<SWIGLU, INT8, PAST> : act_fwd_keep8_kernel<SWIGLU, E4M3, PAST>);
}
template <bool PAST>
auto act_bwd_kernel(int act, int format) {
  return act == GELU_ERF    ? (format == INT8 ? act_bwd_keep8_kernel<GELU_ERF, INT8, PAST> : act_bwd_keep8_kernel<GELU_ERF, E4M3, PAST>)
         : act == GELU_TANH ? (format == INT8 ? act_bwd_keep8_kernel<GELU_TANH, INT8, PAST> : act_bwd_keep8_kernel<GELU_TANH, E4M3, PAST>)
                            : (format == INT8 ? act_bwd_keep8_kernel<SWIGLU, INT8, PAST> : act_bwd_keep8_kernel<SWIGLU, E4M3, PAST>);
}

// Launches of fewer than 2^31 items each, by rows.
template <typename Launch>
hipError_t by_rows(int64_t t, int64_t width, Launch launch) {
  const int64_t per_row = 4 * ceil_div(width, 32), most = std::max<int64_t>(1, (((int64_t)1 << 31) - 256) / per_row);
  for (int64_t row = 0; row < t; row += most) {
    const int64_t rows = std::min(most, t - row);
    const Items it = {division((uint32_t)per_row), (uint32_t)(rows * per_row), (int)(width / 8)};
    launch(row, it, dim3((unsigned)ceil_div(rows * per_row, 256)));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

hipError_t launch_keep8(const void* x, void* q, void* e, int64_t t, int64_t width, int64_t x_stride, int format, hipStream_t s) {
  ProfScope prof(PROF_ELEMENTWISE, 3.03125 * (double)t * (double)width, s);
  return by_rows(t, width, [&](int64_t row, const Items& it, dim3 grid) {
    const auto kernel = format == INT8 ? keep8_kernel<INT8> : keep8_kernel<E4M3>;
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, (const bf16_t*)x + row * x_stride, (uint8_t*)q + row * width,
                       (uint8_t*)e + row * ceil_div(width, 32), it, x_stride);
  });
}

hipError_t launch_keep8_load(const void* q, const void* e, void* y, int64_t t, int64_t width, int64_t y_stride, int format, hipStream_t s) {
  ProfScope prof(PROF_ELEMENTWISE, 3.03125 * (double)t * (double)width, s);
  const bool past = 2 * t * width >= NT_BYTES;
  return by_rows(t, width, [&](int64_t row, const Items& it, dim3 grid) {
    const auto kernel = format == INT8 ? (past ? keep8_load_kernel<INT8, true> : keep8_load_kernel<INT8, false>) : (past ? keep8_load_kernel<E4M3, true> : keep8_load_kernel<E4M3, false>);
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, (const uint8_t*)q + row * width, (const uint8_t*)e + row * ceil_div(width, 32),
                       (bf16_t*)y + row * y_stride, it, y_stride);
  });
}

hipError_t launch_linear_operands(const void* q, const void* e, void* x, const void* dy, void* dy_padded, const void* w, void* w_padded, int64_t t, int64_t k,
                                  int64_t n, int64_t n_padded, int format, hipStream_t s) {
  const int64_t per_row = 4 * ceil_div(k, 32), items = t * per_row, wide = n_padded / 8;
  if (items >= (int64_t)1 << 31 || t * wide >= (int64_t)1 << 31 || k * wide >= (int64_t)1 << 31) return hipErrorInvalidValue;
  ProfScope prof(PROF_ELEMENTWISE, 3.03125 * (double)t * (double)k + 4.0 * (double)(t + k) * (double)n, s);
  const Items it = {division((uint32_t)per_row), (uint32_t)items, (int)(k / 8)};
  const uint32_t first = (uint32_t)ceil_div(items, 256), second = first + (uint32_t)ceil_div(t * wide, 256);
  const Padded pd = {(const bf16_t*)dy, (bf16_t*)dy_padded, division((uint32_t)wide), (uint32_t)(t * wide), first, (int)(n / 8)};
  const Padded pw = {(const bf16_t*)w, (bf16_t*)w_padded, division((uint32_t)wide), (uint32_t)(k * wide), second, (int)(n / 8)};
  const auto kernel = format == INT8 ? linear_operands_kernel<INT8> : linear_operands_kernel<E4M3>;
  hipLaunchKernelGGL(kernel, dim3(second + (unsigned)ceil_div(k * wide, 256)), dim3(256), 0, s, (const uint8_t*)q, (const uint8_t*)e, (bf16_t*)x, it, pd, pw);
  return hipGetLastError();
}

hipError_t launch_act_fwd_keep8(int act, const void* pre, void* a, void* q, void* e, int64_t t, int64_t f, int format, hipStream_t s) {
  const int64_t halves = act == SWIGLU ? 2 : 1;
  ProfScope prof(PROF_ELEMENTWISE, (2.0 + 3.03125 * halves) * (double)t * (double)f, s);
  const bool past = 2 * t * f >= NT_BYTES;
  return by_rows(t, f, [&](int64_t row, const Items& it, dim3 grid) {
    const auto kernel = past ? act_fwd_kernel<true>(act, format) : act_fwd_kernel<false>(act, format);
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, (const bf16_t*)pre + row * halves * f, (bf16_t*)a + row * f, (uint8_t*)q + row * halves * f,
                       (uint8_t*)e + row * halves * ceil_div(f, 32), it);
  });
}

hipError_t launch_act_bwd_keep8(int act, const void* da, const void* q, const void* e, void* dpre, void* a, int64_t t, int64_t f, int format,
                                hipStream_t s) {
  const int64_t halves = act == SWIGLU ? 2 : 1;
  ProfScope prof(PROF_ELEMENTWISE, (1.03125 * halves + (da ? 2.0 + 2.0 * halves : 0.0) + (a ? 2.0 : 0.0)) * (double)t * (double)f, s);
  const bool past = 2 * ((dpre ? halves : 0) + (a ? 1 : 0)) * t * f >= NT_BYTES;
  return by_rows(t, f, [&](int64_t row, const Items& it, dim3 grid) {
    const auto kernel = past ? act_bwd_kernel<true>(act, format) : act_bwd_kernel<false>(act, format);
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, da ? (const bf16_t*)da + row * f : nullptr, (const uint8_t*)q + row * halves * f,
                       (const uint8_t*)e + row * halves * ceil_div(f, 32), dpre ? (bf16_t*)dpre + row * halves * f : nullptr,
                       a ? (bf16_t*)a + row * f : nullptr, it);
  });
}

}  // namespace mllm
