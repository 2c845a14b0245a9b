// Router of an expert layer: logits of every token over the experts, scores, the k best and their weights, in one launch.
//
// A cluster takes a group of tokens; its CTAs share the experts, a warp forms the logits of one expert for all tokens of the group (the
// expert's row is read once for them).  Products of 16-bit operands are exact in fp32, eight are summed there, everything behind that in
// 64 bits: which expert is chosen then hangs on the inputs, not on the order of a sum.  Each token's logits are gathered in the shared
// memory of one CTA, where one warp scores and chooses.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "../sdq_internal.h"
#include "../sdq_ptx.cuh"
#include "layout.h"

namespace sdq {
namespace mx4 {

constexpr int ROUTE_WARPS = 8, ROUTE_CTAS = 8;
constexpr int ROUTE_MAX_E = 1024, ROUTE_MAX_K = 32;

template <int DT> struct RouteElem;
template <> struct RouteElem<SDQ_BF16> { using type = __nv_bfloat16; };
template <> struct RouteElem<SDQ_FP16> { using type = __half; };
template <> struct RouteElem<SDQ_FP32> { using type = float; };
template <int DT> __device__ __forceinline__ float route_float(typename RouteElem<DT>::type x) {
  if constexpr (DT == SDQ_BF16) return __bfloat162float(x);
  else if constexpr (DT == SDQ_FP16) return __half2float(x);
  else return x;
}
// eight consecutive elements; `n` of them exist (VEC: all or none)
template <int DT, bool VEC>
__device__ __forceinline__ void load8(float (&v)[8], const typename RouteElem<DT>::type* p, int64_t n) {
  using T = typename RouteElem<DT>::type;
  if constexpr (VEC && DT != SDQ_FP32) {
    uint4 r = make_uint4(0, 0, 0, 0);
    if (n > 0) r = __ldg(reinterpret_cast<const uint4*>(p));
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (DT == SDQ_BF16) { v[2 * i] = __uint_as_float(w[i] << 16); v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u); }
      else { const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i])); v[2 * i] = f.x; v[2 * i + 1] = f.y; }
    }
  } else if constexpr (VEC) {
    float4 a = make_float4(0, 0, 0, 0), b = a;
    if (n > 0) { a = __ldg(reinterpret_cast<const float4*>(p)); b = __ldg(reinterpret_cast<const float4*>(p) + 1); }
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < n ? route_float<DT>(p[i]) : 0.0f;
  }
}
// order of doubles as order of integers: of equal ones the two zeros alike, a NaN above everything
__device__ __forceinline__ long long rank_key(double x) {
  if (x != x) return 0x7FFFFFFFFFFFFFFFll;
  const long long b = __double_as_longlong(x + 0.0);
  return b ^ ((b >> 63) & 0x7FFFFFFFFFFFFFFFll);
}
__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
__device__ __forceinline__ void store_to_cta(double* local, uint32_t cta, double v) {
  asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(ptx::mapa_u32(ptx::smem_u32(local), cta)), "d"(v) : "memory");
}

struct RouteParams {
  const void *x, *w;
  const float* bias;
  int32_t* ids;
  float* weights;
  int64_t T, H, ldx, ldw;
  int32_t E, k, sigmoid, renorm, elements;   // elements: doubles of a logit row in shared memory
  float scale;
};

// G tokens a cluster
template <int DT, int G, bool VEC>
__global__ void __launch_bounds__(32 * ROUTE_WARPS)
moe_route_kernel(const __grid_constant__ RouteParams p)
{
  using T = typename RouteElem<DT>::type;
  extern __shared__ double s_logit[];        // [tokens of this CTA][E], then as many keys
  const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  uint32_t ctas;
  asm volatile("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(ctas));
  const uint32_t rank = ptx::cluster_ctarank();
  if (threadIdx.x == 0) ptx::griddep_launch_dependents();
  ptx::griddep_wait();
  const int64_t t0 = (int64_t)(blockIdx.x / ctas) * G;
  const T* X = reinterpret_cast<const T*>(p.x);
  const T* W = reinterpret_cast<const T*>(p.w);
  ptx::cluster_sync();                       // (all CTAs have started: their shared memory may be written)
  for (int e = (int)(rank * ROUTE_WARPS + warp); e < p.E; e += (int)ctas * ROUTE_WARPS) {
    double acc[G];
#pragma unroll
    for (int g = 0; g < G; ++g) acc[g] = 0.0;
#pragma unroll 4
    for (int64_t h = lane * 8; h < p.H; h += 256) {
      float w[8], x[8];
      load8<DT, VEC>(w, W + (int64_t)e * p.ldw + h, p.H - h);
#pragma unroll
      for (int g = 0; g < G; ++g) {
        load8<DT, VEC>(x, X + (t0 + g) * p.ldx + h, t0 + g < p.T ? p.H - h : 0);
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) s = fmaf(w[i], x[i], s);
        acc[g] += (double)s;
      }
    }
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const double l = warp_sum(acc[g]);
      if (lane == 0) store_to_cta(s_logit + (size_t)(g / ctas) * p.elements + e, (uint32_t)g % ctas, l);
    }
  }
  ptx::cluster_sync();
  // token g of the group: CTA g % ctas, warp g / ctas
  const int g = (int)(warp * ctas + rank);
  if (g >= G || t0 + g >= p.T) return;
  double* score = s_logit + (size_t)warp * p.elements;
  long long* key = reinterpret_cast<long long*>(s_logit + (size_t)((G + ctas - 1) / ctas) * p.elements) + (size_t)warp * p.elements;
  // scores: softmax over all experts, or sigmoid
  double sum = 1.0;
  if (!p.sigmoid) {
    double top = -INFINITY;
    for (int e = (int)lane; e < p.E; e += 32) top = fmax(top, score[e]);
#pragma unroll
    for (int o = 16; o; o >>= 1) top = fmax(top, __shfl_xor_sync(0xffffffffu, top, o));
    sum = 0.0;
    for (int e = (int)lane; e < p.E; e += 32) { const double v = exp(score[e] - top); sum += v; score[e] = v; }
    sum = warp_sum(sum);
  }
  for (int e = (int)lane; e < p.E; e += 32) {
    const double v = p.sigmoid ? 1.0 / (1.0 + exp(-score[e])) : score[e] / sum;
    score[e] = v;
    key[e] = rank_key(p.bias ? v + (double)p.bias[e] : v);
  }
  double total = 0.0, mine = 0.0;
  int my_id = 0;
  for (int j = 0; j < p.k; ++j) {
    // the largest key that is left, of equal ones the lowest index
    long long best = (long long)0x8000000000000000ull;
    int at = 0x7FFFFFFF;
    for (int e = (int)lane; e < p.E; e += 32)
      if (key[e] > best) { best = key[e]; at = e; }
#pragma unroll
    for (int o = 16; o; o >>= 1) {
      const long long b = __shfl_xor_sync(0xffffffffu, best, o);
      const int a = __shfl_xor_sync(0xffffffffu, at, o);
      if (b > best || (b == best && a < at)) { best = b; at = a; }
    }
    const double v = score[at];
    total += v;
    if ((int)lane == j) { mine = v; my_id = at; }
    __syncwarp();
    if (lane == 0) key[at] = (long long)0x8000000000000000ull;
    __syncwarp();
  }
  if ((int)lane < p.k) {
    p.ids[(t0 + g) * p.k + lane] = my_id;
    p.weights[(t0 + g) * p.k + lane] = (float)((p.renorm ? mine / total : mine) * (double)p.scale);
  }
}

template <int DT, int G>
static sdq_status_t route(const RouteParams& p, bool vec, void* stream) {
  cudaLaunchConfig_t lc = {};
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = ROUTE_CTAS;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  const int64_t groups = (p.T + G - 1) / G;
  if (groups > 0x7FFFFFFF / ROUTE_CTAS) return SDQ_ERR_SHAPE;
  lc.gridDim = dim3((unsigned)groups * ROUTE_CTAS);
  lc.blockDim = dim3(32 * ROUTE_WARPS);
  lc.dynamicSmemBytes = (size_t)((G + ROUTE_CTAS - 1) / ROUTE_CTAS) * p.elements * 16;
  lc.stream = (cudaStream_t)stream;
  lc.attrs = attr;
  lc.numAttrs = 2;
  return launch_status(vec ? cudaLaunchKernelEx(&lc, moe_route_kernel<DT, G, true>, p) : cudaLaunchKernelEx(&lc, moe_route_kernel<DT, G, false>, p));
}

}  // namespace mx4
}  // namespace sdq

using namespace sdq;

extern "C" sdq_status_t sdq_moe_route(const void* X, int32_t dtype, int64_t T, int64_t H, int64_t ldx, const void* Wr, int64_t E, int64_t ldw,
                                      const float* bias, int32_t k, int32_t scoring, int32_t renorm, float scale,
                                      int32_t* ids, float* weights, void* stream)
{
  using namespace mx4;
  if (!X || !Wr || !ids || !weights || !dtype_ok(dtype) || (scoring != SDQ_ROUTE_SOFTMAX && scoring != SDQ_ROUTE_SIGMOID)) return SDQ_ERR_INVALID_ARG;
  if (T < 1 || H < 1 || E < 1 || E > ROUTE_MAX_E || k < 1 || k > E || k > ROUTE_MAX_K || ldx < H || ldw < H || T > ((int64_t)1 << 40) || H > ((int64_t)1 << 30) ||
      ldx > ((int64_t)1 << 40) || ldw > ((int64_t)1 << 40)) return SDQ_ERR_SHAPE;
  const size_t es = dtype_bytes(dtype);
  if ((uintptr_t)X % es || (uintptr_t)Wr % es || (uintptr_t)bias % 4 || (uintptr_t)ids % 4 || (uintptr_t)weights % 4) return SDQ_ERR_ALIGNMENT;
  const bool vec = !((uintptr_t)X & 15) && !((uintptr_t)Wr & 15) && H % 8 == 0 && (ldx % 8 == 0 || T == 1) && (ldw % 8 == 0 || E == 1);
  const RouteParams p = {X, Wr, bias, ids, weights, T, H, ldx, ldw, (int32_t)E, k, scoring == SDQ_ROUTE_SIGMOID, renorm != 0, (int32_t)(E + 1) / 2 * 2, scale};
  const bool one = T <= 8;
  if (dtype == SDQ_BF16) return one ? route<SDQ_BF16, 1>(p, vec, stream) : route<SDQ_BF16, 4>(p, vec, stream);
  if (dtype == SDQ_FP16) return one ? route<SDQ_FP16, 1>(p, vec, stream) : route<SDQ_FP16, 4>(p, vec, stream);
  return one ? route<SDQ_FP32, 1>(p, vec, stream) : route<SDQ_FP32, 4>(p, vec, stream);
}
