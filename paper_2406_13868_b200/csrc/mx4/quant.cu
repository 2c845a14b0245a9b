// Plain microscaled 4-bit matrices: quantizers, importer, exporter, dequantizer (formats: include/sdq_mx4.h, layouts: layout.h).
//
// All of them work in units of 8 rows x 128 K, one a warp: lane l has row l / 4, elements 32 (l % 4) .. + 31, so that the codes of a unit are 512
// contiguous bytes and a row's four MXFP4 scales (eight NVFP4 scales) one (two) words of a scale atom.
//
// Bound by DRAM traffic: 2 to 4 bytes an element on one side, 0.53 or 0.56 on the other.
#include <cuda_fp16.h>

#include "../sdq_codec.cuh"
#include "../sdq_internal.h"
#include "layout.h"
#include "../sdq_ptx.cuh"

namespace sdq {
namespace mx4 {

template <int DT> struct Elem;
template <> struct Elem<SDQ_BF16> { using type = __nv_bfloat16; };
template <> struct Elem<SDQ_FP16> { using type = __half; };
template <> struct Elem<SDQ_FP32> { using type = float; };
template <int DT> __device__ __forceinline__ constexpr float type_max() {
  return DT == SDQ_BF16 ? 3.3895313892515355e38f : DT == SDQ_FP16 ? 65504.0f : 3.4028234663852886e38f;
}
template <int DT> __device__ __forceinline__ float to_float(typename Elem<DT>::type x) {
  if constexpr (DT == SDQ_BF16) return __bfloat162float(x);
  else if constexpr (DT == SDQ_FP16) return __half2float(x);
  else return x;
}
template <int DT> __device__ __forceinline__ typename Elem<DT>::type from_float(float x) {
  if constexpr (DT == SDQ_BF16) return __float2bfloat16_rn(x);
  else if constexpr (DT == SDQ_FP16) return __float2half_rn(x);
  else return x;
}

constexpr int Q_WARPS = 8;
constexpr int UNIT_K = 128;
// staging of rows that no vector access fits: one unit, rows 16 bytes apart from their neighbours' banks
template <int DT> struct Stage { static constexpr uint32_t PITCH = UNIT_K * sizeof(typename Elem<DT>::type) + 16, BYTES = 8 * PITCH; };

// this lane's 32 elements of the unit whose first row's unit starts at column k0; `row`: this lane's row (nullptr: none), zeros behind K
template <int DT, bool VEC>
__device__ __forceinline__ void load_unit(float (&v)[32], const typename Elem<DT>::type* row, int64_t k0, int64_t K, uint8_t* stage, uint32_t lane) {
  using T = typename Elem<DT>::type;
  constexpr int PER = 16 / sizeof(T);                      // elements of a 16-byte load
  uint4 raw[32 / PER];
  if constexpr (VEC) {
    const int64_t k = k0 + 32 * (lane & 3);
#pragma unroll
    for (int i = 0; i < 32 / PER; ++i) {
      raw[i] = make_uint4(0, 0, 0, 0);
      if (row && k + i * PER < K) raw[i] = *reinterpret_cast<const uint4*>(row + k + i * PER);
    }
  } else {
    // rows of any alignment: consecutive lanes take consecutive elements, and the unit is turned in shared memory
#pragma unroll
    for (int r = 0; r < 8; ++r) {
      const T* p = reinterpret_cast<const T*>(__shfl_sync(0xffffffffu, (unsigned long long)(uintptr_t)row, 4 * r));
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int64_t k = k0 + 32 * i + lane;
        T x = from_float<DT>(0.0f);
        if (p && k < K) x = p[k];
        *reinterpret_cast<T*>(stage + r * Stage<DT>::PITCH + (32 * i + lane) * sizeof(T)) = x;
      }
    }
    __syncwarp();
    const uint4* s = reinterpret_cast<const uint4*>(stage + (lane >> 2) * Stage<DT>::PITCH + (lane & 3) * 32 * sizeof(T));
#pragma unroll
    for (int i = 0; i < 32 / PER; ++i) raw[i] = s[i];
    __syncwarp();
  }
#pragma unroll
  for (int i = 0; i < 32 / PER; ++i) {
    const uint32_t w[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if constexpr (DT == SDQ_FP32) v[4 * i + j] = __uint_as_float(w[j]);
      else if constexpr (DT == SDQ_BF16) {
        v[8 * i + 2 * j] = __uint_as_float(w[j] << 16);
        v[8 * i + 2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u);
      } else {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[j]));
        v[8 * i + 2 * j] = f.x;
        v[8 * i + 2 * j + 1] = f.y;
      }
    }
  }
}
// larger of a and |x|; a NaN stays
__device__ __forceinline__ float max_abs(float a, float x) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(fabsf(x)));
  return r;
}
// largest magnitude of N elements; where it is an infinity, the elements are limited to the type's largest number first
template <int DT, int FIRST, int N>
__device__ __forceinline__ float block_max(float (&v)[32]) {
  float a = 0.0f;
#pragma unroll
  for (int i = FIRST; i < FIRST + N; ++i) a = max_abs(a, v[i]);
  if (a == INFINITY) {
#pragma unroll
    for (int i = FIRST; i < FIRST + N; ++i) v[i] = fminf(fmaxf(v[i], -type_max<DT>()), type_max<DT>());
    a = type_max<DT>();
  }
  return a;
}

// ---- quotients ---------------------------------------------------------------------------------------------------------
// z = fp32 quotient of a and b, whose exact quotient is about to be rounded to a format of a few bits: z equals a boundary
// between two values of it (its LOW last bits are zero then) only if the exact quotient does, else it is moved by one unit to
// where that lies.  The remainder of a correctly rounded quotient is exact in one fused operation.
template <int LOW>
__device__ __forceinline__ float keep_side(float z, float a, float b) {
  if ((__float_as_uint(z) & ((1u << LOW) - 1u)) == 0u) {
    const float rem = fmaf(-z, b, a);
    if (rem != 0.0f && z != 0.0f) z = __uint_as_float(__float_as_uint(z) + ((rem > 0.0f) == (z > 0.0f) ? 1u : 0xFFFFFFFFu));
  }
  return z;
}
// E4M3 code nearest to a / 6 (a >= 0, at most 2688), at least the smallest positive one unless the block is all zero
__device__ __forceinline__ uint32_t nv_scale_code(float a, bool nonzero) {
  const uint32_t c = e4m3x1(keep_side<19>(__fdiv_rn(a, 6.0f), a, 6.0f));
  return nonzero ? max(c, 1u) : 0u;
}
__device__ __forceinline__ float e4m3_value(uint32_t c) { return __half2float(__half(__nv_cvt_fp8_to_halfraw((__nv_fp8_storage_t)c, __NV_E4M3))); }
// exponent t of a row's factor: smallest integer >= -126 with a <= 2688 * 2^t (2688 = 1.3125 * 2^11); 0 for a row of zeros
__device__ __forceinline__ int nv_row_exp(float a) {
  if (a == 0.0f) return 0;
  const uint32_t b = __float_as_uint(a);
  return max((int)(b >> 23) - 127 - 11 + ((b & 0x7FFFFFu) > 0x280000u ? 1 : 0), -126);
}
__device__ __forceinline__ uint32_t mx_scale_code(float a, bool ceil_rule) {
  const uint32_t b = __float_as_uint(a);
  return (uint32_t)max((int)(b >> 23) - 2 + ((ceil_rule && (b & 0x7FFFFFu) > 0x400000u) ? 1 : 0), 0);
}

// codes of 32 elements, 16 bytes
__device__ __forceinline__ uint4 codes32(const float (&q)[32]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float t[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) t[j] = q[8 * i + j];
    w[i] = e2m1x8(t);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
// MXFP4: codes and the scale's code
template <int DT>
__device__ __forceinline__ uint4 encode_mx(float (&v)[32], bool ceil_rule, uint32_t& scale) {
  const float a = block_max<DT, 0, 32>(v);
  const uint32_t c = mx_scale_code(a, ceil_rule);
  const float inv = pow2_inv_e8m0(min(c, 253u));
#pragma unroll
  for (int i = 0; i < 32; ++i) v[i] *= inv;
  scale = a != a ? 255u : c;
  return codes32(v);
}
// NVFP4: 16 elements as quotients and their scale's code; `down` = 2^-t
template <int DT, int FIRST>
__device__ __forceinline__ uint32_t encode_nv16(float (&v)[32], float down) {
  const float a = block_max<DT, FIRST, 16>(v);
  const uint32_t c = a != a ? 127u : nv_scale_code(a * down, a > 0.0f);
  const float s = e4m3_value(c), r = c ? __frcp_rn(s) : 0.0f;
#pragma unroll
  for (int i = FIRST; i < FIRST + 16; ++i) {
    // y / s correctly rounded (Markstein: quotient estimate, its exact remainder, one correction): ties stay ties
    const float y = v[i] * down, q = y * r;
    // (the remainder taken as q s - y, so that a negative zero stays one)
    const float z = fmaf(-fmaf(q, s, -y), r, q);
    v[i] = DT == SDQ_FP32 ? keep_side<21>(z, y, s) : z;
  }
  return c;
}
// codes and the two scales' codes (in the two low bytes)
template <int DT>
__device__ __forceinline__ uint4 encode_nv(float (&v)[32], float down, uint32_t& scales) {
  scales = encode_nv16<DT, 0>(v, down);
  scales |= encode_nv16<DT, 16>(v, down) << 8;
  return codes32(v);
}

// ---- where a unit lies -------------------------------------------------------------------------------------------------
// `g`: 8-row group (linear: of the matrix; experts: of all padded rows), `u`: 128-K unit
struct Unit { uint8_t* codes; uint8_t* scales; };        // of this lane: 16 B; the row's word of the unit's first atom
template <bool EXPERTS, int FMT>
__device__ __forceinline__ Unit unit_at(uint8_t* buf, int64_t g, int64_t u, int64_t kblocks, uint32_t lane) {
  Unit x;
  const uint32_t rr = (uint32_t)(g & 15) * 8 + (lane >> 2);
  if constexpr (EXPERTS) {
    uint8_t* rec = buf + (size_t)((g >> 4) * kblocks + u) * ERECORD;
    x.codes = rec + (uint32_t)(g & 15) * 512 + (lane & 3) * 128 + (lane >> 2) * 16;
    x.scales = rec + ECODES + atom_off(rr, 0);
  } else {
    uint8_t* rec = buf + (size_t)((g >> 4) * kblocks + (u >> 1)) * record(FMT);
    x.codes = rec + (uint32_t)(g & 15) * 1024 + ((uint32_t)(u & 1) * 4 + (lane & 3)) * 128 + (lane >> 2) * 16;
    x.scales = rec + CODES + (uint32_t)(u & 1) * (atoms(FMT) / 2) * ATOM + atom_off(rr, 0);
  }
  return x;
}
__device__ __forceinline__ void put_codes(const Unit& x, uint4 c) { *reinterpret_cast<uint4*>(x.codes) = c; }
__device__ __forceinline__ uint4 get_codes(const Unit& x) { return *reinterpret_cast<const uint4*>(x.codes); }
// the scales of a row's lanes as words (all lanes of the warp): MXFP4 one byte a lane, NVFP4 two
template <int FMT>
__device__ __forceinline__ void put_scales(const Unit& x, uint32_t s, uint32_t lane, bool on) {
  if constexpr (FMT == SDQ_FMT_MXFP4) {
    uint32_t w = s << (8 * (lane & 3));
    w |= __shfl_xor_sync(0xffffffffu, w, 1);
    w |= __shfl_xor_sync(0xffffffffu, w, 2);
    if (on && (lane & 3) == 0) *reinterpret_cast<uint32_t*>(x.scales) = w;
  } else {
    uint32_t w = s << (16 * (lane & 1));
    w |= __shfl_xor_sync(0xffffffffu, w, 1);
    if (on && (lane & 1) == 0) *reinterpret_cast<uint32_t*>(x.scales + ((lane >> 1) & 1) * ATOM) = w;
  }
}
template <int FMT>
__device__ __forceinline__ uint32_t get_scales(const Unit& x, uint32_t lane) {
  if constexpr (FMT == SDQ_FMT_MXFP4) return x.scales[lane & 3];
  else return *reinterpret_cast<const uint16_t*>(x.scales + ((lane >> 1) & 1) * ATOM + 2 * (lane & 1));
}
// element row of a lane: linear: row 8 g + l / 4; experts: padded rows are none (-1)
template <bool EXPERTS>
__device__ __forceinline__ int64_t element_row(int64_t g, int64_t R, int64_t tiles, uint32_t lane) {
  const int64_t p = g * 8 + (lane >> 2);
  if constexpr (!EXPERTS) return p < R ? p : -1;
  const int64_t e = p / (tiles * ROWS), r = p - e * tiles * ROWS;
  return r < R ? e * R + r : -1;
}

struct Shape { int64_t R, K, ld, tiles, kblocks, units; size_t factors; };          // units: 128-K units along K, padding included

// ---- MXFP4 --------------------------------------------------------------------------------------------------------------
template <int DT, bool EXPERTS, bool VEC>
__global__ void __launch_bounds__(32 * Q_WARPS)
mx4_quantize_kernel(const typename Elem<DT>::type* __restrict__ X, Shape s, int ceil_rule, uint8_t* __restrict__ buf)
{
  __shared__ __align__(16) uint8_t stage[VEC ? 16 : Q_WARPS * Stage<DT>::BYTES];
  const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) ptx::griddep_launch_dependents();
  ptx::griddep_wait();
  const int64_t g = blockIdx.x, r = element_row<EXPERTS>(g, s.R, s.tiles, lane);
  for (int64_t u = (int64_t)blockIdx.y * (blockDim.x >> 5) + warp; u < s.units; u += (int64_t)gridDim.y * (blockDim.x >> 5)) {
    float v[32];
    load_unit<DT, VEC>(v, r < 0 ? nullptr : X + r * s.ld, u * UNIT_K, s.K, stage + (VEC ? 0 : warp * Stage<DT>::BYTES), lane);
    uint32_t sc;
    const uint4 c = encode_mx<DT>(v, ceil_rule != 0, sc);
    const Unit x = unit_at<EXPERTS, SDQ_FMT_MXFP4>(buf, g, u, s.kblocks, lane);
    const bool on = EXPERTS || r >= 0;
    if (on) put_codes(x, c);
    put_scales<SDQ_FMT_MXFP4>(x, sc, lane, on);
  }
}

// ---- NVFP4 --------------------------------------------------------------------------------------------------------------
// One CTA per 8 rows: the rows' maxima first, then every unit again (from L2, where the first pass has left it) to be encoded.
// (staging of fp32 rows: eight warps' is what shared memory has without asking for more)
template <int DT, bool VEC> struct NvWarps { static constexpr int value = !VEC && DT == SDQ_FP32 ? 8 : 16; };
// ONE: rows of at most one unit a warp, which stays in registers between the two passes.  (As a condition on the second load instead of
// a form of its own, ptxas 12.9 at -O1 and above lost the upper elements.)
template <int DT, bool VEC, bool ONE>
__global__ void __launch_bounds__(32 * NvWarps<DT, VEC>::value)
nv4_quantize_kernel(const typename Elem<DT>::type* __restrict__ X, Shape s, uint8_t* __restrict__ buf)
{
  __shared__ __align__(16) uint8_t stage[VEC ? 16 : NvWarps<DT, VEC>::value * Stage<DT>::BYTES];
  __shared__ float s_max[16][8];
  const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
  uint8_t* st = stage + (VEC ? 0 : warp * Stage<DT>::BYTES);
  if (threadIdx.x == 0) ptx::griddep_launch_dependents();
  ptx::griddep_wait();
  const int64_t g = blockIdx.x, r = element_row<false>(g, s.R, s.tiles, lane);
  const typename Elem<DT>::type* row = r < 0 ? nullptr : X + r * s.ld;
  float a = 0.0f;
  float v[32];
  for (int64_t u = warp; u < s.units; u += ONE ? s.units : (int64_t)warps) {
    load_unit<DT, VEC>(v, row, u * UNIT_K, s.K, st, lane);
    // (a NaN's block is marked by its scale; the row's factor goes by the others)
#pragma unroll
    for (int i = 0; i < 32; ++i) a = fmaxf(a, fabsf(v[i]));
  }
  a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, 1));
  a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, 2));
  if ((lane & 3) == 0) s_max[warp][lane >> 2] = a;
  __syncthreads();
  for (uint32_t w = 0; w < warps; ++w) a = fmaxf(a, s_max[w][lane >> 2]);
  const int t = nv_row_exp(fminf(a, type_max<DT>()));
  const float down = pow2_neg(t);
  if (warp == 0 && (lane & 3) == 0 && r >= 0) *reinterpret_cast<float*>(buf + s.factors + (size_t)r * 4) = __uint_as_float((uint32_t)(t + 127) << 23);
  for (int64_t u = warp; u < s.units; u += ONE ? s.units : (int64_t)warps) {
    if constexpr (!ONE) load_unit<DT, VEC>(v, row, u * UNIT_K, s.K, st, lane);
    uint32_t sc;
    const uint4 c = encode_nv<DT>(v, down, sc);
    const Unit x = unit_at<false, SDQ_FMT_NVFP4>(buf, g, u, s.kblocks, lane);
    if (r >= 0) put_codes(x, c);
    put_scales<SDQ_FMT_NVFP4>(x, sc, lane, r >= 0);
  }
}

// ---- import, export ------------------------------------------------------------------------------------------------------
template <int FMT, bool EXPERTS>
__global__ void __launch_bounds__(32 * Q_WARPS)
mx4_import_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, const float* __restrict__ factor, Shape s, uint8_t* __restrict__ buf)
{
  constexpr int PER = FMT == SDQ_FMT_NVFP4 ? 2 : 1;
  const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) ptx::griddep_launch_dependents();
  ptx::griddep_wait();
  const int64_t g = blockIdx.x, r = element_row<EXPERTS>(g, s.R, s.tiles, lane);
  const int64_t kb = (s.K + 1) / 2, nb = FMT == SDQ_FMT_NVFP4 ? (s.K + 15) / 16 : (s.K + 31) / 32;
  for (int64_t u = (int64_t)blockIdx.y * Q_WARPS + warp; u < s.units; u += (int64_t)gridDim.y * Q_WARPS) {
    uint32_t w[4] = {0, 0, 0, 0}, sc = 0;
    if (r >= 0) {
      const int64_t b0 = u * 64 + (lane & 3) * 16;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int64_t b = b0 + i;
        if (b < kb) {
          uint32_t x = codes[r * kb + b];
          if (2 * b + 1 == s.K) x &= 15u;
          w[i / 4] |= x << (8 * (i % 4));
        }
      }
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        const int64_t b = (u * 4 + (lane & 3)) * PER + i;
        if (b < nb) sc |= (uint32_t)scales[r * nb + b] << (8 * i);
      }
    }
    const Unit x = unit_at<EXPERTS, FMT>(buf, g, u, s.kblocks, lane);
    const bool on = EXPERTS || r >= 0;
    if (on) put_codes(x, make_uint4(w[0], w[1], w[2], w[3]));
    put_scales<FMT>(x, sc, lane, on);
  }
  if (FMT == SDQ_FMT_NVFP4 && blockIdx.y == 0 && warp == 0 && (lane & 3) == 0 && r >= 0)
    *reinterpret_cast<float*>(buf + s.factors + (size_t)r * 4) = factor ? factor[r] : 1.0f;
}
template <int FMT, bool EXPERTS>
__global__ void __launch_bounds__(32 * Q_WARPS)
mx4_export_kernel(uint8_t* __restrict__ buf, Shape s, uint8_t* __restrict__ codes, uint8_t* __restrict__ scales, float* __restrict__ factor)
{
  constexpr int PER = FMT == SDQ_FMT_NVFP4 ? 2 : 1;
  const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) ptx::griddep_launch_dependents();
  ptx::griddep_wait();
  const int64_t g = blockIdx.x, r = element_row<EXPERTS>(g, s.R, s.tiles, lane);
  if (r < 0) return;
  const int64_t kb = (s.K + 1) / 2, nb = FMT == SDQ_FMT_NVFP4 ? (s.K + 15) / 16 : (s.K + 31) / 32;
  for (int64_t u = (int64_t)blockIdx.y * Q_WARPS + warp; u < s.units; u += (int64_t)gridDim.y * Q_WARPS) {
    const Unit x = unit_at<EXPERTS, FMT>(buf, g, u, s.kblocks, lane);
    const uint4 c = get_codes(x);
    const uint32_t w[4] = {c.x, c.y, c.z, c.w}, sc = get_scales<FMT>(x, lane);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int64_t b = u * 64 + (lane & 3) * 16 + i;
      if (b < kb) codes[r * kb + b] = (uint8_t)(w[i / 4] >> (8 * (i % 4)));
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int64_t b = (u * 4 + (lane & 3)) * PER + i;
      if (b < nb) scales[r * nb + b] = (uint8_t)(sc >> (8 * i));
    }
  }
  if (FMT == SDQ_FMT_NVFP4 && factor && blockIdx.y == 0 && warp == 0 && (lane & 3) == 0) factor[r] = *reinterpret_cast<const float*>(buf + s.factors + (size_t)r * 4);
}

// ---- dequantization ------------------------------------------------------------------------------------------------------
__device__ __forceinline__ void values8(uint32_t w, float* v) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __half2_raw h = __nv_cvt_fp4x2_to_halfraw2((__nv_fp4x2_storage_t)((w >> (8 * i)) & 0xFFu), __NV_E2M1);
    const float2 f = __half22float2(__half2(h));
    v[2 * i] = f.x;
    v[2 * i + 1] = f.y;
  }
}
__device__ __forceinline__ float e8m0_value(uint32_t c) {
  return c == 255u ? __uint_as_float(0x7FFFFFFFu) : c ? __uint_as_float(c << 23) : __uint_as_float(0x00400000u);
}
template <int DT, int FMT, bool EXPERTS, bool VEC>
__global__ void __launch_bounds__(32 * Q_WARPS)
mx4_dequantize_kernel(uint8_t* __restrict__ buf, Shape s, typename Elem<DT>::type* __restrict__ out)
{
  using T = typename Elem<DT>::type;
  constexpr int PER = 16 / sizeof(T);
  __shared__ __align__(16) uint8_t stage[VEC ? 16 : Q_WARPS * Stage<DT>::BYTES];
  const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) ptx::griddep_launch_dependents();
  ptx::griddep_wait();
  const int64_t g = blockIdx.x, r = element_row<EXPERTS>(g, s.R, s.tiles, lane);
  uint8_t* st = stage + (VEC ? 0 : warp * Stage<DT>::BYTES);
  float f = 1.0f;
  if (FMT == SDQ_FMT_NVFP4 && r >= 0) f = *reinterpret_cast<const float*>(buf + s.factors + (size_t)r * 4);
  for (int64_t u = (int64_t)blockIdx.y * (blockDim.x >> 5) + warp; u < s.units; u += (int64_t)gridDim.y * (blockDim.x >> 5)) {
    float v[32];
    if (r >= 0) {
      const Unit x = unit_at<EXPERTS, FMT>(buf, g, u, s.kblocks, lane);
      const uint4 c = get_codes(x);
      const uint32_t sc = get_scales<FMT>(x, lane);
      values8(c.x, v);
      values8(c.y, v + 8);
      values8(c.z, v + 16);
      values8(c.w, v + 24);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float m = FMT == SDQ_FMT_MXFP4 ? e8m0_value(sc) : e4m3_value((sc >> (8 * h)) & 0xFFu);
#pragma unroll
        for (int i = 16 * h; i < 16 * h + 16; ++i) v[i] = FMT == SDQ_FMT_MXFP4 ? v[i] * m : v[i] * m * f;
      }
    }
    uint4 raw[32 / PER];
#pragma unroll
    for (int i = 0; i < 32 / PER; ++i) {
      uint32_t w[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if constexpr (DT == SDQ_FP32) w[j] = __float_as_uint(v[4 * i + j]);
        else if constexpr (DT == SDQ_BF16) {
          const __nv_bfloat162 b = __floats2bfloat162_rn(v[8 * i + 2 * j], v[8 * i + 2 * j + 1]);
          w[j] = *reinterpret_cast<const uint32_t*>(&b);
        } else {
          const __half2 b = __floats2half2_rn(v[8 * i + 2 * j], v[8 * i + 2 * j + 1]);
          w[j] = *reinterpret_cast<const uint32_t*>(&b);
        }
      }
      raw[i] = make_uint4(w[0], w[1], w[2], w[3]);
    }
    T* row = r < 0 ? nullptr : out + r * s.ld;
    if constexpr (VEC) {
      const int64_t k = u * UNIT_K + 32 * (lane & 3);
#pragma unroll
      for (int i = 0; i < 32 / PER; ++i)
        if (row && k + i * PER < s.K) *reinterpret_cast<uint4*>(row + k + i * PER) = raw[i];
    } else {
      uint4* sp = reinterpret_cast<uint4*>(st + (lane >> 2) * Stage<DT>::PITCH + (lane & 3) * 32 * sizeof(T));
#pragma unroll
      for (int i = 0; i < 32 / PER; ++i) sp[i] = raw[i];
      __syncwarp();
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        T* p = reinterpret_cast<T*>(__shfl_sync(0xffffffffu, (unsigned long long)(uintptr_t)row, 4 * q));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int64_t k = u * UNIT_K + 32 * i + lane;
          if (p && k < s.K) p[k] = *reinterpret_cast<const T*>(st + q * Stage<DT>::PITCH + (32 * i + lane) * sizeof(T));
        }
      }
      __syncwarp();
    }
  }
}

// ---- launches ------------------------------------------------------------------------------------------------------------
static Shape shape_of(int64_t E, int64_t R, int64_t K, int64_t ld, int fmt) {
  const Dims d = dims(E, R, K, fmt);
  Shape s;
  s.R = R; s.K = K; s.ld = ld; s.tiles = d.tiles; s.kblocks = d.kblocks; s.units = E ? d.kblocks : 2 * d.kblocks;
  s.factors = d.factors;
  return s;
}
template <typename... P, typename... A>
static sdq_status_t launch(void (*kern)(P...), dim3 grid, unsigned threads, void* stream, A... args) {
  cudaLaunchConfig_t lc = {};
  lc.gridDim = grid;
  lc.blockDim = dim3(threads);
  lc.stream = (cudaStream_t)stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  lc.attrs = attr;
  lc.numAttrs = 1;
  return launch_status(cudaLaunchKernelEx(&lc, kern, args...));
}
// 8-row groups, one a thread block along x: linear: those that hold rows; experts: of all padded rows
static int64_t groups_of(int64_t E, const Shape& s) { return E ? E * s.tiles * 16 : (s.R + 7) / 8; }
static unsigned blocks_along_k(const Shape& s, int warps) { return (unsigned)((s.units + warps - 1) / warps < 65535 ? (s.units + warps - 1) / warps : 65535); }
// rows a vector access of 16 bytes fits
static bool vectors_fit(const void* p, int64_t ld, int64_t K, int32_t dtype, bool one_row) {
  const int64_t per = 16 / (int64_t)dtype_bytes(dtype);
  return ((uintptr_t)p & 15) == 0 && K % per == 0 && (ld % per == 0 || one_row);
}
static void describe(sdq_mx4_t* out, void* buf, int64_t E, int64_t R, int64_t K, int fmt) {
  const Dims d = dims(E, R, K, fmt);
  out->dev = buf; out->bytes = d.total; out->E = E; out->R = R; out->K = K; out->fmt = fmt; out->reserved = 0;
  out->factors = d.factors;
}
template <int DT>
static sdq_status_t quantize(const void* X, int64_t E, const Shape& s, int fmt, int rule, uint8_t* buf, void* stream) {
  using T = typename Elem<DT>::type;
  const T* x = (const T*)X;
  const bool vec = vectors_fit(X, s.ld, s.K, DT, (E ? E : 1) * s.R == 1);
  const int64_t groups = groups_of(E, s);
  if (groups > 0x7FFFFFFF) return SDQ_ERR_SHAPE;
  if (fmt == SDQ_FMT_NVFP4) {
    const int64_t warps = vec ? NvWarps<DT, true>::value : NvWarps<DT, false>::value;
    const unsigned threads = 32u * (unsigned)(s.units < warps ? s.units : warps);
    auto nv = [&](auto kern) { return launch(kern, dim3((unsigned)groups), threads, stream, x, s, buf); };
    if (s.units <= warps) return vec ? nv(nv4_quantize_kernel<DT, true, true>) : nv(nv4_quantize_kernel<DT, false, true>);
    return vec ? nv(nv4_quantize_kernel<DT, true, false>) : nv(nv4_quantize_kernel<DT, false, false>);
  }
  const dim3 grid((unsigned)groups, blocks_along_k(s, Q_WARPS));
  auto go = [&](auto kern) { return launch(kern, grid, 32 * Q_WARPS, stream, x, s, rule, buf); };
  if (E) return vec ? go(mx4_quantize_kernel<DT, true, true>) : go(mx4_quantize_kernel<DT, true, false>);
  return vec ? go(mx4_quantize_kernel<DT, false, true>) : go(mx4_quantize_kernel<DT, false, false>);
}
static sdq_status_t quantize_any(const void* X, int32_t dtype, int64_t E, int64_t R, int64_t K, int64_t ld, int32_t fmt, int32_t rule, void* buf, size_t bytes,
                                 sdq_mx4_t* out, void* stream) {
  if (!X || !buf || !out || !dtype_ok(dtype) || !fmt_ok(fmt) || (rule != SDQ_SCALE_OCP_FLOOR && rule != SDQ_SCALE_CEIL_NOSAT)) return SDQ_ERR_INVALID_ARG;
  if (!size_ok(E, R, K) || ld < K || ld > ((int64_t)1 << 40)) return SDQ_ERR_SHAPE;
  if (((uintptr_t)X % dtype_bytes(dtype)) || ((uintptr_t)buf & 255)) return SDQ_ERR_ALIGNMENT;
  if (bytes < dims(E, R, K, fmt).total) return SDQ_ERR_BUFFER_TOO_SMALL;
  const Shape s = shape_of(E, R, K, ld, fmt);
  const sdq_status_t st = dtype == SDQ_BF16   ? quantize<SDQ_BF16>(X, E, s, fmt, rule, (uint8_t*)buf, stream)
                          : dtype == SDQ_FP16 ? quantize<SDQ_FP16>(X, E, s, fmt, rule, (uint8_t*)buf, stream)
                                              : quantize<SDQ_FP32>(X, E, s, fmt, rule, (uint8_t*)buf, stream);
  if (st == SDQ_OK) describe(out, buf, E, R, K, fmt);
  return st;
}
static sdq_status_t import_any(const uint8_t* codes, const uint8_t* scales, const float* factor, int64_t E, int64_t R, int64_t K, int32_t fmt, void* buf, size_t bytes,
                               sdq_mx4_t* out, void* stream) {
  if (!codes || !scales || !buf || !out || !fmt_ok(fmt) || (factor && fmt != SDQ_FMT_NVFP4)) return SDQ_ERR_INVALID_ARG;
  if (!size_ok(E, R, K)) return SDQ_ERR_SHAPE;
  if (((uintptr_t)buf & 255) || ((uintptr_t)factor & 3)) return SDQ_ERR_ALIGNMENT;
  if (bytes < dims(E, R, K, fmt).total) return SDQ_ERR_BUFFER_TOO_SMALL;
  const Shape s = shape_of(E, R, K, 0, fmt);
  const int64_t groups = groups_of(E, s);
  if (groups > 0x7FFFFFFF) return SDQ_ERR_SHAPE;
  const dim3 grid((unsigned)groups, blocks_along_k(s, Q_WARPS));
  auto go = [&](auto kern) { return launch(kern, grid, 32 * Q_WARPS, stream, codes, scales, factor, s, (uint8_t*)buf); };
  const sdq_status_t st = E ? go(mx4_import_kernel<SDQ_FMT_MXFP4, true>)
                            : fmt == SDQ_FMT_NVFP4 ? go(mx4_import_kernel<SDQ_FMT_NVFP4, false>) : go(mx4_import_kernel<SDQ_FMT_MXFP4, false>);
  if (st == SDQ_OK) describe(out, buf, E, R, K, fmt);
  return st;
}
template <int DT>
static sdq_status_t dequantize(const sdq_mx4_t* q, void* out, int64_t ldo, void* stream) {
  const Shape s = shape_of(q->E, q->R, q->K, ldo, q->fmt);
  const int64_t groups = groups_of(q->E, s);
  if (groups > 0x7FFFFFFF) return SDQ_ERR_SHAPE;
  const bool vec = vectors_fit(out, ldo, q->K, DT, (q->E ? q->E : 1) * q->R == 1);
  const dim3 grid((unsigned)groups, blocks_along_k(s, Q_WARPS));
  using T = typename Elem<DT>::type;
  auto go = [&](auto kern) { return launch(kern, grid, 32 * Q_WARPS, stream, (uint8_t*)q->dev, s, (T*)out); };
  if (q->E) return vec ? go(mx4_dequantize_kernel<DT, SDQ_FMT_MXFP4, true, true>) : go(mx4_dequantize_kernel<DT, SDQ_FMT_MXFP4, true, false>);
  if (q->fmt == SDQ_FMT_NVFP4) return vec ? go(mx4_dequantize_kernel<DT, SDQ_FMT_NVFP4, false, true>) : go(mx4_dequantize_kernel<DT, SDQ_FMT_NVFP4, false, false>);
  return vec ? go(mx4_dequantize_kernel<DT, SDQ_FMT_MXFP4, false, true>) : go(mx4_dequantize_kernel<DT, SDQ_FMT_MXFP4, false, false>);
}

}  // namespace mx4
}  // namespace sdq

using namespace sdq;

extern "C" sdq_status_t sdq_mx4_size(int64_t R, int64_t K, int32_t fmt, size_t* bytes)
{
  if (!bytes || !mx4::fmt_ok(fmt)) return SDQ_ERR_INVALID_ARG;
  if (!mx4::size_ok(0, R, K)) return SDQ_ERR_SHAPE;
  *bytes = mx4::dims(0, R, K, fmt).total;
  return SDQ_OK;
}

extern "C" sdq_status_t sdq_mx4_experts_size(int64_t E, int64_t R, int64_t K, size_t* bytes)
{
  if (!bytes) return SDQ_ERR_INVALID_ARG;
  if (E < 1 || !mx4::size_ok(E, R, K)) return SDQ_ERR_SHAPE;
  *bytes = mx4::dims(E, R, K, SDQ_FMT_MXFP4).total;
  return SDQ_OK;
}

extern "C" sdq_status_t sdq_mx4_quantize(const void* X, int32_t dtype, int64_t R, int64_t K, int64_t ldx, int32_t fmt, int32_t scale_rule,
                                         void* buf, size_t bytes, sdq_mx4_t* out, void* stream)
{ return mx4::quantize_any(X, dtype, 0, R, K, ldx, fmt, scale_rule, buf, bytes, out, stream); }

extern "C" sdq_status_t sdq_mx4_experts_quantize(const void* W, int32_t dtype, int64_t E, int64_t R, int64_t K, int32_t scale_rule,
                                                 void* buf, size_t bytes, sdq_mx4_t* out, void* stream)
{
  if (E < 1) return SDQ_ERR_SHAPE;
  return mx4::quantize_any(W, dtype, E, R, K, K, SDQ_FMT_MXFP4, scale_rule, buf, bytes, out, stream);
}

extern "C" sdq_status_t sdq_mx4_import(const uint8_t* codes, const uint8_t* scales, const float* factor, int64_t R, int64_t K, int32_t fmt,
                                       void* buf, size_t bytes, sdq_mx4_t* out, void* stream)
{ return mx4::import_any(codes, scales, factor, 0, R, K, fmt, buf, bytes, out, stream); }

extern "C" sdq_status_t sdq_mx4_experts_import(const uint8_t* codes, const uint8_t* scales, int64_t E, int64_t R, int64_t K,
                                               void* buf, size_t bytes, sdq_mx4_t* out, void* stream)
{
  if (E < 1) return SDQ_ERR_SHAPE;
  return mx4::import_any(codes, scales, nullptr, E, R, K, SDQ_FMT_MXFP4, buf, bytes, out, stream);
}

extern "C" sdq_status_t sdq_mx4_export(const sdq_mx4_t* q, uint8_t* codes, uint8_t* scales, float* factor, void* stream)
{
  using namespace mx4;
  if (!desc_ok(q) || !codes || !scales) return SDQ_ERR_INVALID_ARG;
  const Shape s = shape_of(q->E, q->R, q->K, 0, q->fmt);
  const int64_t groups = groups_of(q->E, s);
  if (groups > 0x7FFFFFFF) return SDQ_ERR_SHAPE;
  const dim3 grid((unsigned)groups, blocks_along_k(s, Q_WARPS));
  auto go = [&](auto kern) { return launch(kern, grid, 32 * Q_WARPS, stream, (uint8_t*)q->dev, s, codes, scales, factor); };
  return q->E ? go(mx4_export_kernel<SDQ_FMT_MXFP4, true>)
              : q->fmt == SDQ_FMT_NVFP4 ? go(mx4_export_kernel<SDQ_FMT_NVFP4, false>) : go(mx4_export_kernel<SDQ_FMT_MXFP4, false>);
}

extern "C" sdq_status_t sdq_mx4_dequantize(const sdq_mx4_t* q, void* out, int32_t dtype, int64_t ldo, void* stream)
{
  if (!mx4::desc_ok(q) || !out || !mx4::dtype_ok(dtype)) return SDQ_ERR_INVALID_ARG;
  if (ldo < q->K || ldo > ((int64_t)1 << 40)) return SDQ_ERR_SHAPE;
  if ((uintptr_t)out % mx4::dtype_bytes(dtype)) return SDQ_ERR_ALIGNMENT;
  return dtype == SDQ_BF16   ? mx4::dequantize<SDQ_BF16>(q, out, ldo, stream)
         : dtype == SDQ_FP16 ? mx4::dequantize<SDQ_FP16>(q, out, ldo, stream)
                             : mx4::dequantize<SDQ_FP32>(q, out, ldo, stream);
}
