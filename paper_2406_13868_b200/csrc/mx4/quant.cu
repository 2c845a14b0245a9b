// Plain microscaled 4-bit matrices: quantizers, importer, exporter, dequantizer (formats: include/sdq_mx4.h, layouts: layout.h).
//
// All of them work in units of 8 rows x 128 K, one a warp, as two halves of 64 K: lane l has row l / 4, elements 16 (l % 4) .. + 15 of a half.  An
// access of a lane is 32 bytes (of a 16-bit type) and four lanes have a line of 128; a store of codes writes whole core matrices.
//
// What has to move are 2 to 4 bytes an element on one side and 0.53 or 0.56 on the other.  Dequantizer of many aligned rows: at DRAM's rate (8192 x 11008 38 us,
// its bytes 36).  MXFP4 quantizer: near it (8192 x 4096 18 us under the profiler, bytes 13; DRAM 47 % there).  NVFP4 quantizer of many rows: its encode loop, three
// dependent operations an element for an exact quotient (8192 x 11008 66 us, bytes 36).  Rows off every boundary: the granules' branches and shifts (1000 x
// 4109 7.4 and 4.4 us, bytes 1.6).  Importer and exporter move bytes one by one, once for a checkpoint's matrix: 11008 x 4096 28 and 55 us, 1.7 and
// 0.9 TB/s.  A few rows: a launch
#include <cuda_fp16.h>

#include <type_traits>

#include "../../../include/sdq_diag.h"
#include "../sdq_codec.cuh"
#include "../sdq_internal.h"
#include "layout.h"
#include "pipe.cuh"
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
template <int DT> __device__ __forceinline__ typename Elem<DT>::type from_float(float x) {
  if constexpr (DT == SDQ_BF16) return __float2bfloat16_rn(x);
  else if constexpr (DT == SDQ_FP16) return __float2half_rn(x);
  else return x;
}

constexpr int Q_WARPS = 8;
constexpr int UNIT_K = 128;

// ---- rows in memory ------------------------------------------------------------------------------------------------------
// Rows whose elements lie on 32-byte boundaries are loaded and stored 32 bytes a lane (VEC).  Any others go through the 16-byte granules
// around them: a load takes the granules that overlap its bytes and shifts them into place, a store is turned in shared memory.
// Single elements are only touched where a granule is not whole inside the matrix.
struct Bounds { uintptr_t lo, hi; };                        // first byte of the matrix, and the one behind its last

__device__ __forceinline__ void ld32(uint32_t (&w)[8], const void* p) {
  asm volatile("ld.global.nc.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7]) : "l"(p));
}
__device__ __forceinline__ void st32(void* p, const uint32_t (&w)[8]) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
               : "memory");
}
// 32 bytes at `p`, of which the first `valid` belong to the row (zeros behind them)
template <int ES>
__device__ __forceinline__ void ld32_any(uint32_t (&w)[8], const uint8_t* p, int valid, const Bounds& m) {
  const uintptr_t at = (uintptr_t)p, g = at & ~(uintptr_t)15;
  const uint32_t o = (uint32_t)(at & 15);
  uint32_t x[12];
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    uint4 v = make_uint4(0, 0, 0, 0);
    const uintptr_t q = g + 16 * i;
    if (valid > 0 && q < at + (uintptr_t)valid) {              // (its first byte in front of the row's end; its last one behind `at`)
      if (q >= m.lo && q + 16 <= m.hi) {
        v = *reinterpret_cast<const uint4*>(q);
      } else {
        uint32_t e[4] = {0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < 16 / ES; ++j) {
          const uintptr_t r = q + ES * j;
          if (r >= at && r < at + (uintptr_t)valid) {
            if constexpr (ES == 2) e[j / 2] |= (uint32_t)*reinterpret_cast<const uint16_t*>(r) << (16 * (j & 1));
            else e[j] = *reinterpret_cast<const uint32_t*>(r);
          }
        }
        v = make_uint4(e[0], e[1], e[2], e[3]);
      }
    }
    x[4 * i] = v.x; x[4 * i + 1] = v.y; x[4 * i + 2] = v.z; x[4 * i + 3] = v.w;
  }
  // down by 8, 4 and 2 bytes
#pragma unroll
  for (int i = 0; i < 10; ++i) x[i] = o & 8 ? x[i + 2] : x[i];
#pragma unroll
  for (int i = 0; i < 9; ++i) x[i] = o & 4 ? x[i + 1] : x[i];
#pragma unroll
  for (int i = 0; i < 8; ++i) w[i] = ES == 2 && (o & 2) ? __funnelshift_r(x[i], x[i + 1], 16) : x[i];
#pragma unroll
  for (int i = 0; i < 8; ++i) {                             // what lies behind the row's end
    if (valid < 4 * i + 4) w[i] = ES == 2 && valid == 4 * i + 2 ? w[i] & 0xFFFFu : 0u;
  }
}
// 16 elements of a row from `p`, `n` of which exist
template <int DT, bool VEC>
__device__ __forceinline__ void load16(float (&v)[16], const typename Elem<DT>::type* p, int64_t n, const Bounds& m) {
  constexpr int ES = sizeof(typename Elem<DT>::type), PER = 32 / ES;      // elements of 32 bytes
#pragma unroll
  for (int i = 0; i < 16 / PER; ++i) {
    uint32_t w[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j] = 0;
    const int64_t left = n - i * PER;
    if constexpr (VEC) { if (left > 0) ld32(w, p + i * PER); }
    else ld32_any<ES>(w, reinterpret_cast<const uint8_t*>(p + i * PER), (int)(left < 0 ? 0 : left > PER ? PER : left) * ES, m);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if constexpr (DT == SDQ_FP32) v[8 * i + j] = __uint_as_float(w[j]);
      else if constexpr (DT == SDQ_BF16) {
        v[2 * j] = __uint_as_float(w[j] << 16);
        v[2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u);
      } else {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[j]));
        v[2 * j] = f.x;
        v[2 * j + 1] = f.y;
      }
    }
  }
}
template <int DT>
__device__ __forceinline__ void pack16(uint32_t (&w)[16 * sizeof(typename Elem<DT>::type) / 4], const float (&v)[16]) {
#pragma unroll
  for (int j = 0; j < (int)(16 * sizeof(typename Elem<DT>::type) / 4); ++j) {
    if constexpr (DT == SDQ_FP32) w[j] = __float_as_uint(v[j]);
    else if constexpr (DT == SDQ_BF16) {
      const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * j], v[2 * j + 1]);
      w[j] = *reinterpret_cast<const uint32_t*>(&b);
    } else {
      const __half2 b = __floats2half2_rn(v[2 * j], v[2 * j + 1]);
      w[j] = *reinterpret_cast<const uint32_t*>(&b);
    }
  }
}
// a warp's unit on its way to rows of any alignment: a row's bytes at the offset in a granule that they have in memory
template <int DT> struct Stage { static constexpr uint32_t ROW = UNIT_K * sizeof(typename Elem<DT>::type), PITCH = ROW + 48, BYTES = 8 * PITCH; };
template <int DT>
__device__ __forceinline__ void stage16(uint8_t* st, uint32_t o, uint32_t k, const uint32_t (&w)[16 * sizeof(typename Elem<DT>::type) / 4]) {
  constexpr int W = 16 * sizeof(typename Elem<DT>::type) / 4;
  uint8_t* d = st + o + k * sizeof(typename Elem<DT>::type);
  if (DT != SDQ_FP32 && (o & 2)) {
    *reinterpret_cast<uint16_t*>(d) = (uint16_t)w[0];
#pragma unroll
    for (int j = 0; j + 1 < W; ++j) *reinterpret_cast<uint32_t*>(d + 2 + 4 * j) = __funnelshift_r(w[j], w[j + 1], 16);
    *reinterpret_cast<uint16_t*>(d + 4 * W - 2) = (uint16_t)(w[W - 1] >> 16);
  } else {
#pragma unroll
    for (int j = 0; j < W; ++j) *reinterpret_cast<uint32_t*>(d + 4 * j) = w[j];
  }
}
// stores the staged rows: row r's first byte is row[r] (of lane 4 r), `bytes` of each exist.  Whole granules first, then the elements in front of
// and behind them, one a lane.  (Elements of a granule one after the other by the lane that met it: 1000 x 4109 10.1 us, so 4.4)
template <int DT>
__device__ __forceinline__ void store_staged(const uint8_t* st, typename Elem<DT>::type* row, int bytes, uint32_t lane) {
  using S = Stage<DT>;
  constexpr int ES = sizeof(typename Elem<DT>::type), WHOLE = (int)S::ROW / 16;      // granules of a row, at most
  if (bytes <= 0) return;                                                             // (a unit of nothing but padding)
  __syncwarp();
#pragma unroll
  for (int i = 0; i < 8 * WHOLE / 32; ++i) {
    const int r = (32 * i + (int)lane) / WHOLE, g = (32 * i + (int)lane) % WHOLE;
    const uintptr_t p = (uintptr_t)__shfl_sync(0xffffffffu, (unsigned long long)(uintptr_t)row, 4 * r);
    const int o = (int)(p & 15), at = 16 * (g + (o ? 1 : 0));                          // counted from the first granule's start
    if (p && at + 16 <= o + bytes) *reinterpret_cast<uint4*>(reinterpret_cast<uint8_t*>(p) - o + at) = *reinterpret_cast<const uint4*>(st + r * S::PITCH + at);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = 2 * i + (int)(lane >> 4), e = (int)(lane & 7) * ES;
    const bool tail = lane & 8;
    const uintptr_t p = (uintptr_t)__shfl_sync(0xffffffffu, (unsigned long long)(uintptr_t)row, 4 * r);
    const int o = (int)(p & 15), end = o + bytes, last = end & ~15;                    // `last`: start of the granule the row ends in
    // head: from o to the end of the first granule, if it does not start there; tail: from the last granule's start, if that is another one
    const int at = tail ? last + e : o + e;
    const bool on = tail ? (last > 0 || o == 0) && at < end && e < 16 : o > 0 && at < 16 && at < end;
    if (p && on) {
      uint8_t* d = reinterpret_cast<uint8_t*>(p) - o + at;
      const uint8_t* s = st + r * S::PITCH + at;
      if constexpr (ES == 2) *reinterpret_cast<uint16_t*>(d) = *reinterpret_cast<const uint16_t*>(s);
      else *reinterpret_cast<uint32_t*>(d) = *reinterpret_cast<const uint32_t*>(s);
    }
  }
  __syncwarp();
}
// larger of a and |x|; a NaN stays
__device__ __forceinline__ float max_abs(float a, float x) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(fabsf(x)));
  return r;
}
// largest magnitude of 16 elements (a NaN stays)
__device__ __forceinline__ float max16(const float (&v)[16]) {
  float a = 0.0f;
#pragma unroll
  for (int i = 0; i < 16; ++i) a = max_abs(a, v[i]);
  return a;
}
// infinities as the type's largest number; `a`: the block's largest magnitude
template <int DT>
__device__ __forceinline__ void saturate(float (&v)[16], float& a) {
  if (a == INFINITY) {
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = fminf(fmaxf(v[i], -type_max<DT>()), type_max<DT>());
    a = type_max<DT>();
  }
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
// a / b with r = 1 / b to within a few units: the quotient's estimate, its exact remainder, one correction (Markstein).  An exact quotient of
// few bits comes out as itself, so that ties stay ties.  (The remainder is taken as q b - a, so that a negative zero stays one.)
__device__ __forceinline__ float quotient(float a, float b, float r) {
  const float q = a * r;
  return fmaf(-fmaf(q, b, -a), r, q);
}
// E4M3 code nearest to a / 6 (a >= 0, at most 2688), at least the smallest positive one unless the block is all zero.  Only an fp32 a
// can have a quotient so near to a boundary that rounding puts it there
template <int DT>
__device__ __forceinline__ uint32_t nv_scale_code(float a, bool nonzero) {
  const float z = quotient(a, 6.0f, 1.0f / 6.0f);
  const uint32_t c = e4m3x1(DT == SDQ_FP32 ? keep_side<19>(z, a, 6.0f) : z);
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

// codes of 16 elements, 8 bytes
__device__ __forceinline__ uint2 codes16(const float (&q)[16]) {
  float lo[8], hi[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) { lo[j] = q[j]; hi[j] = q[8 + j]; }
  return make_uint2(e2m1x8(lo), e2m1x8(hi));
}
// MXFP4: 16 elements of a block whose other half the neighbouring lane has
template <int DT>
__device__ __forceinline__ uint2 encode_mx(float (&v)[16], bool ceil_rule, uint32_t& scale) {
  float a = max16(v);
  a = max_abs(a, __shfl_xor_sync(0xffffffffu, a, 1));
  saturate<DT>(v, a);
  const uint32_t c = mx_scale_code(a, ceil_rule);
  const float inv = pow2_inv_e8m0(min(c, 253u));
#pragma unroll
  for (int i = 0; i < 16; ++i) v[i] *= inv;
  scale = a != a ? 255u : c;
  return codes16(v);
}
// NVFP4: the row's factor 2^t, as what its elements are worked on with.  Rows of tiny numbers are lifted by 2^64 first, which keeps
// remainders out of the subnormal range
struct NvRow {
  float lift, down, up;                      // 2^0 or 2^64; 2^-t, 2^t of the lifted row
  __device__ __forceinline__ explicit NvRow(int t) {
    const bool tiny = t < -60;
    lift = tiny ? 18446744073709551616.0f : 1.0f;
    down = pow2_neg(tiny ? t + 64 : t);
    up = pow2_neg(tiny ? -t - 64 : -t);
  }
};
// a block
template <int DT>
__device__ __forceinline__ uint2 encode_nv(float (&v)[16], const NvRow& row, uint32_t& scale) {
  if (row.lift != 1.0f) {
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] *= row.lift;
  }
  float a = max16(v);
  saturate<DT>(v, a);
  scale = a != a ? 127u : nv_scale_code<DT>(a * row.down, a > 0.0f);
  const float s = fminf(e4m3_value(scale), 448.0f) * row.up;          // (a NaN's block: codes as under the largest scale, so that zeros, padding among them, stay zeros)
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(s));
  if (scale == 0u) r = 0.0f;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const float z = quotient(v[i], s, r);
    v[i] = DT == SDQ_FP32 ? keep_side<21>(z, v[i], s) : z;
  }
  return codes16(v);
}

// ---- where a unit lies -------------------------------------------------------------------------------------------------
// `g`: 8-row group (linear: of the matrix; experts: of all padded rows), `u`: 128-K unit
struct Unit { uint8_t* codes; uint8_t* scales; };        // of this lane's eight code bytes of the first half (the second's: 256 further on); the row's word of the unit's first atom
template <bool EXPERTS, int FMT>
__device__ __forceinline__ Unit unit_at(uint8_t* buf, int64_t g, int64_t u, int64_t kblocks, uint32_t lane) {
  Unit x;
  const uint32_t rr = (uint32_t)(g & 15) * 8 + (lane >> 2);
  if constexpr (EXPERTS) {
    uint8_t* rec = buf + (size_t)((g >> 4) * kblocks + u) * ERECORD;
    x.codes = rec + (uint32_t)(g & 15) * 512 + ((lane >> 1) & 1) * 128 + (lane >> 2) * 16 + (lane & 1) * 8;
    x.scales = rec + ECODES + atom_off(rr, 0);
  } else {
    uint8_t* rec = buf + (size_t)((g >> 4) * kblocks + (u >> 1)) * record(FMT);
    x.codes = rec + (uint32_t)(g & 15) * 1024 + ((uint32_t)(u & 1) * 4 + ((lane >> 1) & 1)) * 128 + (lane >> 2) * 16 + (lane & 1) * 8;
    x.scales = rec + CODES + (uint32_t)(u & 1) * (atoms(FMT) / 2) * ATOM + atom_off(rr, 0);
  }
  return x;
}
__device__ __forceinline__ void put_codes(const Unit& x, int half, uint2 c) { *reinterpret_cast<uint2*>(x.codes + 256 * half) = c; }
__device__ __forceinline__ uint2 get_codes(const Unit& x, int half) { return *reinterpret_cast<const uint2*>(x.codes + 256 * half); }
// the scales of a row's lanes as words (all lanes of the warp): MXFP4: two of each half, one word; NVFP4: four of a half, a word each
template <int FMT>
__device__ __forceinline__ void put_scales(const Unit& x, const uint32_t (&s)[2], uint32_t lane, bool on) {
  if constexpr (FMT == SDQ_FMT_MXFP4) {
    uint32_t w = (s[0] | s[1] << 16) << (4 * (lane & 2));             // (both lanes of a pair have its scale)
    w |= __shfl_xor_sync(0xffffffffu, w, 2);
    if (on && (lane & 3) == 0) *reinterpret_cast<uint32_t*>(x.scales) = w;
  } else {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      uint32_t w = s[h] << (8 * (lane & 3));
      w |= __shfl_xor_sync(0xffffffffu, w, 1);
      w |= __shfl_xor_sync(0xffffffffu, w, 2);
      if (on && (lane & 3) == (uint32_t)h) *reinterpret_cast<uint32_t*>(x.scales + h * ATOM) = w;
    }
  }
}
template <int FMT>
__device__ __forceinline__ uint32_t get_scale(const Unit& x, int half, uint32_t lane) {
  return FMT == SDQ_FMT_MXFP4 ? x.scales[2 * half + ((lane >> 1) & 1)] : x.scales[half * ATOM + (lane & 3)];
}
// element row of a lane: linear: row 8 g + l / 4; experts: padded rows are none (-1)
template <bool EXPERTS>
__device__ __forceinline__ int64_t element_row(int64_t g, int64_t R, int64_t tiles, uint32_t lane) {
  const int64_t p = g * 8 + (lane >> 2);
  if constexpr (!EXPERTS) return p < R ? p : -1;
  const int64_t e = p / (tiles * ROWS), r = p - e * tiles * ROWS;
  return r < R ? e * R + r : -1;
}

struct Shape { int64_t R, rows, K, ld, tiles, kblocks, units; size_t factors; };          // rows: of all experts; units: 128-K units along K, padding included

template <int DT>
__device__ __forceinline__ Bounds bounds_of(const typename Elem<DT>::type* X, const Shape& s) {
  return Bounds{(uintptr_t)X, (uintptr_t)(X + (s.rows - 1) * s.ld + s.K)};
}

// ---- MXFP4 --------------------------------------------------------------------------------------------------------------
template <int DT, bool EXPERTS, bool VEC>
__global__ void __launch_bounds__(32 * Q_WARPS)
mx4_quantize_kernel(const typename Elem<DT>::type* __restrict__ X, Shape s, int ceil_rule, uint8_t* __restrict__ buf)
{
  const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  ptx::griddep_wait();
  if (threadIdx.x == 0) ptx::griddep_launch_dependents();       // (behind the wait: see pipe.cuh)
  const int64_t g = blockIdx.x, r = element_row<EXPERTS>(g, s.R, s.tiles, lane);
  const Bounds m = bounds_of<DT>(X, s);
  for (int64_t u = (int64_t)blockIdx.y * (blockDim.x >> 5) + warp; u < s.units; u += (int64_t)gridDim.y * (blockDim.x >> 5)) {
    const int64_t k = u * UNIT_K + 16 * (lane & 3);
    float v[2][16];
#pragma unroll
    for (int h = 0; h < 2; ++h) load16<DT, VEC>(v[h], X + r * s.ld + k + 64 * h, r < 0 ? 0 : s.K - k - 64 * h, m);
    const Unit x = unit_at<EXPERTS, SDQ_FMT_MXFP4>(buf, g, u, s.kblocks, lane);
    const bool on = EXPERTS || r >= 0;
    uint32_t sc[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint2 c = encode_mx<DT>(v[h], ceil_rule != 0, sc[h]);
      if (on) put_codes(x, h, c);
    }
    put_scales<SDQ_FMT_MXFP4>(x, sc, lane, on);
  }
}

// ---- NVFP4 --------------------------------------------------------------------------------------------------------------
// The CTAs of a cluster share the units of 8 rows, NU a warp, which stay in registers while the rows' maxima are exchanged through
// distributed shared memory.  Rows too long for that (LONG) are read twice, by one CTA a group, the second time from L2.
// This CTA's maxima of the eight rows, and where the other CTAs put theirs
constexpr int NV_CTAS = 8;
struct NvMax { float warp[Q_WARPS][8], cta[NV_CTAS][8]; };
__device__ __forceinline__ float max_over_cluster(NvMax& m, float a, uint32_t warp, uint32_t lane, uint32_t warps, uint32_t ctas, uint32_t rank) {
  a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, 1));
  a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, 2));
  if ((lane & 3) == 0) m.warp[warp][lane >> 2] = a;
  __syncthreads();
  if (ctas == 1) {
    for (uint32_t w = 0; w < warps; ++w) a = fmaxf(a, m.warp[w][lane >> 2]);
    return a;
  }
  ptx::cluster_sync();                       // (every CTA has started, too: its shared memory may be written)
  if (threadIdx.x < 8 * ctas) {
    const uint32_t row = threadIdx.x & 7, peer = threadIdx.x >> 3;
    float t = 0.0f;
    for (uint32_t w = 0; w < warps; ++w) t = fmaxf(t, m.warp[w][row]);
    asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(ptx::mapa_u32(ptx::smem_u32(&m.cta[rank][row]), peer)), "f"(t) : "memory");
  }
  ptx::cluster_sync();
  for (uint32_t c = 0; c < ctas; ++c) a = fmaxf(a, m.cta[c][lane >> 2]);
  return a;
}
template <int DT, bool VEC, int NU, bool LONG>
__global__ void __launch_bounds__(32 * Q_WARPS)
nv4_quantize_kernel(const typename Elem<DT>::type* __restrict__ X, Shape s, uint8_t* __restrict__ buf)
{
  __shared__ NvMax mx;
  const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
  ptx::griddep_wait();
  if (threadIdx.x == 0) ptx::griddep_launch_dependents();       // (behind the wait: see pipe.cuh)
  const uint32_t ctas = LONG ? 1u : gridDim.y, rank = LONG ? 0u : blockIdx.y;
  const int64_t g = blockIdx.x, r = element_row<false>(g, s.R, s.tiles, lane);
  const Bounds m = bounds_of<DT>(X, s);
  const typename Elem<DT>::type* row = X + r * s.ld + 16 * (lane & 3);
  const int64_t have = r < 0 ? 0 : s.K - 16 * (lane & 3);
  float a = 0.0f, v[NU][2][16];
  // (a NaN's block is marked by its scale; the row's factor goes by the others)
  if constexpr (LONG) {
    for (int64_t u = warp; u < s.units; u += warps)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        load16<DT, VEC>(v[0][h], row + u * UNIT_K + 64 * h, have - u * UNIT_K - 64 * h, m);
#pragma unroll
        for (int i = 0; i < 16; ++i) a = fmaxf(a, fabsf(v[0][h][i]));
      }
  } else {
#pragma unroll
    for (int n = 0; n < NU; ++n) {
      const int64_t u = (int64_t)(rank + ctas * (warp + warps * n));
#pragma unroll
      for (int h = 0; h < 2; ++h) load16<DT, VEC>(v[n][h], row + u * UNIT_K + 64 * h, have - u * UNIT_K - 64 * h, m);
    }
#pragma unroll
    for (int n = 0; n < NU; ++n)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < 16; ++i) a = fmaxf(a, fabsf(v[n][h][i]));
  }
  a = max_over_cluster(mx, a, warp, lane, warps, ctas, rank);
  const int t = nv_row_exp(fminf(a, type_max<DT>()));
  const NvRow nv(t);
  if (rank == 0 && warp == 0 && (lane & 3) == 0 && r >= 0) *reinterpret_cast<float*>(buf + s.factors + (size_t)r * 4) = __uint_as_float((uint32_t)(t + 127) << 23);
  auto encode = [&](float (&w)[2][16], int64_t u) {
    const Unit x = unit_at<false, SDQ_FMT_NVFP4>(buf, g, u, s.kblocks, lane);
    uint32_t sc[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint2 c = encode_nv<DT>(w[h], nv, sc[h]);
      if (r >= 0) put_codes(x, h, c);
    }
    put_scales<SDQ_FMT_NVFP4>(x, sc, lane, r >= 0);
  };
  if constexpr (LONG) {
    for (int64_t u = warp; u < s.units; u += warps) {
#pragma unroll
      for (int h = 0; h < 2; ++h) load16<DT, VEC>(v[0][h], row + u * UNIT_K + 64 * h, have - u * UNIT_K - 64 * h, m);
      encode(v[0], u);
    }
  } else {
#pragma unroll
    for (int n = 0; n < NU; ++n) {
      const int64_t u = (int64_t)(rank + ctas * (warp + warps * n));
      if (u < s.units) encode(v[n], u);
    }
  }
}

// Many long rows of a 16-bit type: one CTA an SM goes through them RB at a time, the next ones on their way into shared memory (bulk copies)
// while these are read there twice, for the maxima and to be encoded.  A row is read from DRAM once and nothing waits for anybody else.
// us, this and the cluster form: 8192 x 11008 bf16 67 and 99 (rows read again from L2: 82), 4096 x 16384 53 and 71, 512 x 11008 7.8 and 9.8; but 300 x
// 11008 6.1 and 4.7, and where a warp of the cluster form has one unit, 2048 x 4096 10.9 and 9.4, 8192 x 4096 29.0 and 28.5.  Copies and
// maxima alone take 28 of the 66 us at 8192 x 11008, without the encoding 47, without the stores 58: what is left is the encode loop, with issue slots 56 % taken and DRAM 54 %.
constexpr int NS_WARPS = 16, NS_MAX_BUFFERS = 8;
template <int DT, int RB>
__global__ void __launch_bounds__(32 * NS_WARPS)
nv4_quantize_stream_kernel(const typename Elem<DT>::type* __restrict__ X, Shape s, int buffers, uint32_t row_bytes, uint8_t* __restrict__ buf, uint32_t* __restrict__ flags)
{
  using T = typename Elem<DT>::type;
  constexpr int LPR = 32 / RB, RUN = 16 * LPR;               // lanes of a row, elements of it that a warp takes at a time
  extern __shared__ __align__(16) uint8_t ring[];            // [buffer][RB][row_bytes]
  __shared__ uint64_t full[NS_MAX_BUFFERS];
  __shared__ float s_max[2][NS_WARPS][RB];
  const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, rl = lane / LPR, kl = (lane % LPR) * 16;
  const int64_t blocks = (s.R + RB - 1) / RB;
  auto load = [&](int64_t b, int n) {                        // (one thread)
    const int rows = (int)min((int64_t)RB, s.R - b * RB);
    const uint32_t bar = ptx::smem_u32(&full[n]), dst = ptx::smem_u32(ring) + (uint32_t)n * RB * row_bytes;
    expect32(bar, (uint32_t)rows * (uint32_t)s.K * (uint32_t)sizeof(T));
    for (int r = 0; r < rows; ++r) copy32(dst + (uint32_t)r * row_bytes, X + (b * RB + r) * s.ld, (uint32_t)s.K * (uint32_t)sizeof(T), bar);
  };
  if (tid == 0) {
    for (int n = 0; n < buffers; ++n) ptx::mbar_init(&full[n], 1);
    ptx::fence_barrier_init();
  }
  __syncthreads();
  ptx::griddep_wait();
  if (tid == 0) ptx::griddep_launch_dependents();
  if (tid == 0)
    for (int n = 0; n < buffers; ++n)
      if (blockIdx.x + (int64_t)n * gridDim.x < blocks) load(blockIdx.x + (int64_t)n * gridDim.x, n);
  int n = 0, turn = 0;
  uint32_t ph = 0;
  for (int64_t b = blockIdx.x; b < blocks; b += gridDim.x, turn ^= 1) {
    const bool landed = __all_sync(0xffffffffu, wait32(ptx::smem_u32(&full[n]), ph));
    const uint8_t* row = ring + ((uint32_t)n * RB + rl) * row_bytes;
    const int64_t r = b * RB + rl;
    const bool have = r < s.R;
    auto read = [&](float (&v)[16], int64_t k) {             // (K is a multiple of a granule's elements)
      constexpr int PER = 16 / sizeof(T);
#pragma unroll
      for (int i = 0; i < 16 / PER; ++i) {
        uint4 q = make_uint4(0, 0, 0, 0);
        if (have && k + i * PER < s.K) q = *reinterpret_cast<const uint4*>(row + (size_t)(k + i * PER) * sizeof(T));
        const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          static_assert(DT != SDQ_FP32);
          if constexpr (DT == SDQ_BF16) { v[8 * i + 2 * j] = __uint_as_float(w[j] << 16); v[8 * i + 2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u); }
          else { const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[j])); v[8 * i + 2 * j] = f.x; v[8 * i + 2 * j + 1] = f.y; }
        }
      }
    };
    float a = 0.0f, v[16];
    {
      using T2 = typename std::conditional<DT == SDQ_BF16, __nv_bfloat162, __half2>::type;
      auto larger = [](uint32_t m, uint32_t x) {
        x &= 0x7FFF7FFFu;
        const T2 r = __hmax2(*reinterpret_cast<const T2*>(&m), *reinterpret_cast<const T2*>(&x));
        return *reinterpret_cast<const uint32_t*>(&r);
      };
      uint32_t m0 = 0, m1 = 0;
      const int granules = have ? (int)s.K / 8 : 0;
#pragma unroll 4
      for (int k = (int)(warp * LPR + lane % LPR); k < granules; k += NS_WARPS * LPR) {
        const uint4 q = reinterpret_cast<const uint4*>(row)[k];
        m0 = larger(m0, q.x); m1 = larger(m1, q.y); m0 = larger(m0, q.z); m1 = larger(m1, q.w);
      }
      m0 = larger(m0, m1);
      if constexpr (DT == SDQ_BF16) a = fmaxf(__uint_as_float(m0 << 16), __uint_as_float(m0 & 0xFFFF0000u));
      else { const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&m0)); a = fmaxf(f.x, f.y); }
    }
#pragma unroll
    for (int o = 1; o < LPR; o <<= 1) a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, o));
    if (lane % LPR == 0) s_max[turn][warp][rl] = a;
    if (!__syncthreads_and(landed)) {                        // a wait gave up: all warps leave, behind the copies that are still under way
      if (tid == 0) {
        atomicOr(&flags[FLAG_TIMEOUT], 1u);
        for (int i = 0; i < buffers && b + (int64_t)i * gridDim.x < blocks; ++i) {
          (void)wait32(ptx::smem_u32(&full[n]), ph);
          if (++n == buffers) { n = 0; ph ^= 1u; }
        }
      }
      return;
    }
#pragma unroll
    for (int w = 0; w < NS_WARPS; ++w) a = fmaxf(a, s_max[turn][w][rl]);
    const int t = nv_row_exp(fminf(a, type_max<DT>()));
    const NvRow nv(t);
    if (warp == 0 && lane % LPR == 0 && have) *reinterpret_cast<float*>(buf + s.factors + (size_t)r * 4) = __uint_as_float((uint32_t)(t + 127) << 23);
    uint8_t* tile = buf + (size_t)(r / ROWS) * s.kblocks * record(SDQ_FMT_NVFP4);
    const uint32_t rr = (uint32_t)(r % ROWS);
    for (int64_t k = (int64_t)warp * RUN + kl; k < s.units * UNIT_K; k += NS_WARPS * RUN) {      // (padding included)
      read(v, k);
      uint32_t sc;
      const uint2 c = encode_nv<DT>(v, nv, sc);
      uint32_t w = sc << (8 * (lane & 3));
      w |= __shfl_xor_sync(0xffffffffu, w, 1);
      w |= __shfl_xor_sync(0xffffffffu, w, 2);
      if (have) {
        uint8_t* rec = tile + (size_t)(k / KREC) * record(SDQ_FMT_NVFP4);
        const uint32_t kk = (uint32_t)(k % KREC);
        *reinterpret_cast<uint2*>(rec + (rr >> 3) * 1024 + (kk >> 5) * 128 + (rr & 7) * 16 + (kk >> 1 & 8)) = c;
        if ((lane & 3) == 0) *reinterpret_cast<uint32_t*>(rec + CODES + (kk >> 6) * ATOM + atom_off(rr, 0)) = w;
      }
    }
    __syncthreads();                                         // the buffer has been read
    if (tid == 0 && b + (int64_t)buffers * gridDim.x < blocks) load(b + (int64_t)buffers * gridDim.x, n);
    if (++n == buffers) { n = 0; ph ^= 1u; }
  }
}

// ---- import, export ------------------------------------------------------------------------------------------------------
template <int FMT, bool EXPERTS>
__global__ void __launch_bounds__(32 * Q_WARPS)
mx4_import_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, const float* __restrict__ factor, Shape s, uint8_t* __restrict__ buf)
{
  const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  ptx::griddep_wait();
  if (threadIdx.x == 0) ptx::griddep_launch_dependents();       // (behind the wait: see pipe.cuh)
  const int64_t g = blockIdx.x, r = element_row<EXPERTS>(g, s.R, s.tiles, lane);
  const int64_t kb = (s.K + 1) / 2, nb = FMT == SDQ_FMT_NVFP4 ? (s.K + 15) / 16 : (s.K + 31) / 32;
  for (int64_t u = (int64_t)blockIdx.y * Q_WARPS + warp; u < s.units; u += (int64_t)gridDim.y * Q_WARPS) {
    const Unit x = unit_at<EXPERTS, FMT>(buf, g, u, s.kblocks, lane);
    const bool on = EXPERTS || r >= 0;
    uint32_t sc[2] = {0, 0};
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      uint32_t w[2] = {0, 0};
      if (r >= 0) {
        const int64_t b0 = u * 64 + 32 * h + (lane & 3) * 8, sb = FMT == SDQ_FMT_NVFP4 ? u * 8 + 4 * h + (lane & 3) : u * 4 + 2 * h + ((lane >> 1) & 1);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int64_t b = b0 + i;
          if (b < kb) {
            uint32_t c = codes[r * kb + b];
            if (2 * b + 1 == s.K) c &= 15u;
            w[i / 4] |= c << (8 * (i % 4));
          }
        }
        if (sb < nb) sc[h] = scales[r * nb + sb] & (FMT == SDQ_FMT_NVFP4 ? 0x7Fu : 0xFFu);
      }
      if (on) put_codes(x, h, make_uint2(w[0], w[1]));
    }
    put_scales<FMT>(x, sc, lane, on);
  }
  if (FMT == SDQ_FMT_NVFP4 && blockIdx.y == 0 && warp == 0 && (lane & 3) == 0 && r >= 0)
    *reinterpret_cast<float*>(buf + s.factors + (size_t)r * 4) = factor ? factor[r] : 1.0f;
}
template <int FMT, bool EXPERTS>
__global__ void __launch_bounds__(32 * Q_WARPS)
mx4_export_kernel(uint8_t* __restrict__ buf, Shape s, uint8_t* __restrict__ codes, uint8_t* __restrict__ scales, float* __restrict__ factor)
{
  const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  ptx::griddep_wait();
  if (threadIdx.x == 0) ptx::griddep_launch_dependents();       // (behind the wait: see pipe.cuh)
  const int64_t g = blockIdx.x, r = element_row<EXPERTS>(g, s.R, s.tiles, lane);
  if (r < 0) return;
  const int64_t kb = (s.K + 1) / 2, nb = FMT == SDQ_FMT_NVFP4 ? (s.K + 15) / 16 : (s.K + 31) / 32;
  for (int64_t u = (int64_t)blockIdx.y * Q_WARPS + warp; u < s.units; u += (int64_t)gridDim.y * Q_WARPS) {
    const Unit x = unit_at<EXPERTS, FMT>(buf, g, u, s.kblocks, lane);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint2 c = get_codes(x, h);
      const int64_t b0 = u * 64 + 32 * h + (lane & 3) * 8, sb = FMT == SDQ_FMT_NVFP4 ? u * 8 + 4 * h + (lane & 3) : u * 4 + 2 * h + ((lane >> 1) & 1);
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (b0 + i < kb) codes[r * kb + b0 + i] = (uint8_t)((i < 4 ? c.x : c.y) >> (8 * (i % 4)));
      if (sb < nb) scales[r * nb + sb] = (uint8_t)get_scale<FMT>(x, h, lane);      // (MXFP4: both lanes of a pair write the same)
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
  constexpr int W = 16 * sizeof(T) / 4;
  __shared__ __align__(16) uint8_t stage[VEC ? 16 : Q_WARPS * Stage<DT>::BYTES];
  const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  ptx::griddep_wait();
  if (threadIdx.x == 0) ptx::griddep_launch_dependents();       // (behind the wait: see pipe.cuh)
  const int64_t g = blockIdx.x, r = element_row<EXPERTS>(g, s.R, s.tiles, lane);
  uint8_t* st = stage + (VEC ? 0 : warp * Stage<DT>::BYTES);
  float f = 1.0f;
  if (FMT == SDQ_FMT_NVFP4 && r >= 0) f = *reinterpret_cast<const float*>(buf + s.factors + (size_t)r * 4);
  for (int64_t u = (int64_t)blockIdx.y * (blockDim.x >> 5) + warp; u < s.units; u += (int64_t)gridDim.y * (blockDim.x >> 5)) {
    const Unit x = unit_at<EXPERTS, FMT>(buf, g, u, s.kblocks, lane);
    T* row = r < 0 ? nullptr : out + r * s.ld + u * UNIT_K;
    uint2 c[2];
    uint32_t sc[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      c[h] = make_uint2(0, 0);
      sc[h] = 0;
      if (r >= 0) { c[h] = get_codes(x, h); sc[h] = get_scale<FMT>(x, h, lane); }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float v[16];
      values8(c[h].x, v);
      values8(c[h].y, v + 8);
      const float m = FMT == SDQ_FMT_MXFP4 ? e8m0_value(sc[h]) : e4m3_value(sc[h]);
#pragma unroll
      for (int i = 0; i < 16; ++i) v[i] = FMT == SDQ_FMT_MXFP4 ? v[i] * m : v[i] * m * f;
      uint32_t w[W];
      pack16<DT>(w, v);
      const int64_t k = 64 * h + 16 * (lane & 3);
      if constexpr (VEC) {
        constexpr int PER = 32 / sizeof(T);
#pragma unroll
        for (int i = 0; i < W / 8; ++i)
          if (row && u * UNIT_K + k + i * PER < s.K) st32(row + k + i * PER, *reinterpret_cast<const uint32_t(*)[8]>(w + 8 * i));
      } else {
        stage16<DT>(st + (lane >> 2) * Stage<DT>::PITCH, (uint32_t)((uintptr_t)row & 15), (uint32_t)k, w);
      }
    }
    if constexpr (!VEC) store_staged<DT>(st, row, (int)min((int64_t)UNIT_K, s.K - u * UNIT_K) * (int)sizeof(T), lane);
  }
}

// ---- launches ------------------------------------------------------------------------------------------------------------
static Shape shape_of(int64_t E, int64_t R, int64_t K, int64_t ld, int fmt) {
  const Dims d = dims(E, R, K, fmt);
  Shape s;
  s.R = R; s.rows = (E ? E : 1) * R; s.K = K; s.ld = ld; s.tiles = d.tiles; s.kblocks = d.kblocks; s.units = E ? d.kblocks : 2 * d.kblocks;
  s.factors = d.factors;
  return s;
}
template <typename... P, typename... A>
static sdq_status_t launch_as(unsigned cluster, size_t smem, void (*kern)(P...), dim3 grid, unsigned threads, void* stream, A... args) {

  cudaLaunchConfig_t lc = {};
  lc.gridDim = grid;
  lc.blockDim = dim3(threads);
  lc.dynamicSmemBytes = smem;
  lc.stream = (cudaStream_t)stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = 1;
  attr[1].val.clusterDim.y = cluster;
  attr[1].val.clusterDim.z = 1;
  lc.attrs = attr;
  lc.numAttrs = cluster ? 2 : 1;
  return launch_status(cudaLaunchKernelEx(&lc, kern, args...));
}
template <typename... P, typename... A>
static sdq_status_t launch(void (*kern)(P...), dim3 grid, unsigned threads, void* stream, A... args) { return launch_as(0, 0, kern, grid, threads, stream, args...); }
constexpr int NS_SMEM = 227328;              // (beside the kernel's own)
constexpr int64_t NS_FROM = 1 << 22;          // elements from which rows are streamed
// Whether the rows of an NVFP4 matrix of a 16-bit type are streamed through shared memory (rows of a turn; 0: they are not), and in how many
// buffers: rows in 16-byte granules, more than one unit a warp in the cluster form, 2^22 elements of them at least, and two buffers that fit.
// (Rows may have 2^31 bytes: compared in 64 bits.)
struct StreamForm {
  int rows, buffers;
  uint32_t row_bytes;
  size_t shared() const { return (size_t)rows * (size_t)buffers * row_bytes; }
};
static StreamForm stream_form(uintptr_t X, int64_t R, int64_t K, int64_t ld, int dtype) {
  const int64_t es = (int64_t)dtype_bytes(dtype), per = 16 / es, row_bytes = K * es, units = (K + KREC - 1) / KREC * (KREC / UNIT_K);
  if (dtype == SDQ_FP32 || (X & 15) || K % per || ld % per || units <= NV_CTAS * Q_WARPS || row_bytes > NS_SMEM / 4 || R < (NS_FROM + K - 1) / K) return {0, 0, 0};
  const int rows = row_bytes <= NS_SMEM / 8 ? 4 : 2;
  const int64_t buffers = NS_SMEM / (row_bytes * rows);
  return {rows, buffers < NS_MAX_BUFFERS ? (int)buffers : NS_MAX_BUFFERS, (uint32_t)row_bytes};
}
// 8-row groups, one a thread block along x: linear: those that hold rows; experts: of all padded rows
static int64_t groups_of(int64_t E, const Shape& s) { return E ? E * s.tiles * 16 : (s.R + 7) / 8; }
static unsigned blocks_along_k(const Shape& s, int warps) { return (unsigned)((s.units + warps - 1) / warps < 65535 ? (s.units + warps - 1) / warps : 65535); }
// rows whose elements lie on 32-byte boundaries
static bool vectors_fit(const void* p, int64_t ld, int64_t K, int32_t dtype, bool one_row) {
  const int64_t per = 32 / (int64_t)dtype_bytes(dtype);
  return ((uintptr_t)p & 31) == 0 && K % per == 0 && (ld % per == 0 || one_row);
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
    DeviceInfo* d = device_info();
    uint32_t* flags = device_flags();
    if (!d || !flags) return SDQ_ERR_CUDA;
    if constexpr (DT != SDQ_FP32) {
      const StreamForm f = stream_form((uintptr_t)X, s.R, s.K, s.ld, DT);
      if (f.rows) {
        auto stream_rows = [&](auto kern, int bit) {
          if (!(d->mx4_quant_attr & (1u << bit))) {
            if (cudaFuncSetAttribute((const void*)kern, cudaFuncAttributeMaxDynamicSharedMemorySize, NS_SMEM) != cudaSuccess) return launch_status(cudaErrorUnknown);
            d->mx4_quant_attr |= 1u << bit;
          }
          const int64_t blocks = (s.R + f.rows - 1) / f.rows;
          return launch_as(0, f.shared(), kern, dim3((unsigned)(blocks < d->sm_count ? blocks : d->sm_count)), 32 * NS_WARPS, stream, x, s, f.buffers, f.row_bytes,
                           buf, flags);
        };
        return f.rows == 4 ? stream_rows(nv4_quantize_stream_kernel<DT, 4>, 2 * DT) : stream_rows(nv4_quantize_stream_kernel<DT, 2>, 2 * DT + 1);
      }
    }
    // one unit a warp where the CTAs of a cluster have as many warps, else two; short rows take fewer warps
    const int nu = s.units <= NV_CTAS * Q_WARPS ? 1 : 2;
    const int64_t warps = (s.units + nu - 1) / nu, ctas = (warps + Q_WARPS - 1) / Q_WARPS;
    if (ctas > NV_CTAS) return vec ? launch(nv4_quantize_kernel<DT, true, 1, true>, dim3((unsigned)groups), 32 * Q_WARPS, stream, x, s, buf)
                                   : launch(nv4_quantize_kernel<DT, false, 1, true>, dim3((unsigned)groups), 32 * Q_WARPS, stream, x, s, buf);
    auto nv = [&](auto kern) { return launch_as((unsigned)ctas, 0, kern, dim3((unsigned)groups, (unsigned)ctas), 32u * (unsigned)((warps + ctas - 1) / ctas), stream, x, s, buf); };
    if (nu == 1) return vec ? nv(nv4_quantize_kernel<DT, true, 1, false>) : nv(nv4_quantize_kernel<DT, false, 1, false>);
    return vec ? nv(nv4_quantize_kernel<DT, true, 2, false>) : nv(nv4_quantize_kernel<DT, false, 2, false>);
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

extern "C" sdq_status_t sdq_diag_mx4_quantize_rows(uint64_t address, int64_t R, int64_t K, int64_t ldx, int32_t dtype, int32_t* rows, int32_t* buffers, int64_t* shared)
{
  if (!rows || !buffers || !shared || !mx4::dtype_ok(dtype)) return SDQ_ERR_INVALID_ARG;
  if (!mx4::size_ok(0, R, K) || ldx < K) return SDQ_ERR_SHAPE;
  const mx4::StreamForm f = mx4::stream_form((uintptr_t)address, R, K, ldx, dtype);
  *rows = f.rows; *buffers = f.buffers; *shared = (int64_t)f.shared();
  return SDQ_OK;
}
