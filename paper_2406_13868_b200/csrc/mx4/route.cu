// Router of an expert layer: logits of every token over the experts, scores, the k best and their weights, in one launch.
//
// A cluster takes a group of tokens; its CTAs share the experts, and K where there are few of them.  Each token's logits are gathered in the
// shared memory of one CTA, which scores and chooses.  Which expert is chosen should hang on the order of a sum as little as
// can be: products of 16-bit operands are exact in fp32, 32 of them are summed there, by the tensor core (mma.sync: sixteen experts x eight
// tokens, a shape that this size of problem fills, where a tcgen05 tile would be all padding), which may cut what it adds, and everything
// behind that in 64 bits.  fp32 operands go through ordinary multiplications, eight to a sum.  So a logit is within 32 2^-23 (16-bit operands) or
// 8 2^-24 (fp32) of the sum of its products' magnitudes, and only experts nearer to each other than that may change places.
#include "../sdq_internal.h"
#include "../sdq_ptx.cuh"
#include "layout.h"
#include "pipe.cuh"

namespace sdq {
namespace mx4 {

constexpr int ROUTE_WARPS = 16, ROUTE_CTAS = 8;
constexpr int ROUTE_MAX_E = 1024, ROUTE_MAX_K = 32;

// A lane's eight elements of a run: consecutive ones where rows can be read in 16-byte granules (VEC), else every LANES-th, so that the
// lanes of a row read next to each other.  `n`: elements from `p` to the row's end.  Predicates and no branch: loads of a batch go out together
// (consecutive elements with branches, and so: 33 tokens x 2047 -> 100 in fp32 26 us and 10, 5 x 333 -> 17 in bf16 6.6 and 4.8, 33 x 2047 -> 100 10.5 and 10.9).
template <bool VEC>
__device__ __forceinline__ void load8(float (&v)[8], const float* p, int64_t n) {
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = 0.0f;
  if constexpr (VEC) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
      asm volatile("{\n.reg .pred p;\nsetp.ne.u32 p, %5, 0;\n@p ld.global.nc.v4.f32 {%0, %1, %2, %3}, [%4];\n}"
                   : "+f"(v[4 * i]), "+f"(v[4 * i + 1]), "+f"(v[4 * i + 2]), "+f"(v[4 * i + 3]) : "l"(p + 4 * i), "r"((uint32_t)(n > 0)));
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      asm volatile("{\n.reg .pred p;\nsetp.ne.u32 p, %2, 0;\n@p ld.global.nc.f32 %0, [%1];\n}" : "+f"(v[i]) : "l"(p + 32 * i), "r"((uint32_t)(32 * i < n)));
  }
}
// order of doubles as order of integers: of equal ones the two zeros alike, a NaN above everything
__device__ __forceinline__ long long rank_key(double x) {
  if (x != x) return 0x7FFFFFFFFFFFFFFFll;
  const long long b = __double_as_longlong(x + 0.0);
  return b ^ ((b >> 63) & 0x7FFFFFFFFFFFFFFFll);
}
// largest of n numbers, a NaN aside (by a warp)
__device__ __noinline__ double largest(const double* v, int n, uint32_t lane) {
  double top = -INFINITY;
  for (int i = (int)lane; i < n; i += 32) top = fmax(top, v[i]);
  for (int o = 16; o; o >>= 1) top = fmax(top, __shfl_xor_sync(0xffffffffu, top, o));
  return top;
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
  int32_t E, k, sigmoid, renorm, elements, splits;   // elements: doubles of a logit row in shared memory; splits: parts of K (16-bit operands)
  float scale;
};

// one token's scores, choices and weights, by all warps of the CTA.  score: [E] logits; key: [E]; red: scratch of ROUTE_WARPS doubles and 2 ROUTE_COUNTED
// words.  A softmax is left undivided where only the order and the ratios of the scores matter.
// Up to ROUTE_COUNTED experts the choice is by counting (64 experts, 6 of them: 4.8 us a call, against 5.6 with six maxima one behind the other; 256
// experts, 8 of them: 12.0 against 9.3).
constexpr int ROUTE_COUNTED = 128;
__device__ __forceinline__ void choose(const RouteParams& p, int64_t t, double* score, long long* key, double* red) {
  const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  constexpr int THREADS = 32 * ROUTE_WARPS;
  int32_t *place = reinterpret_cast<int32_t*>(red + ROUTE_WARPS), *chosen = place + ROUTE_COUNTED;
  double inv = 1.0;
  if (!p.sigmoid) {
    // the exponentials are formed relative to a number near the largest logit: the fp32 one (every warp finds it for itself)
    float top = -INFINITY;
    for (int e = (int)lane; e < p.E; e += 32) top = fmaxf(top, (float)score[e]);
    const int b = __float_as_int(top + 0.0f), k = __reduce_max_sync(0xffffffffu, b ^ (b >> 31 & 0x7FFFFFFF));
    top = __int_as_float(k ^ (k >> 31 & 0x7FFFFFFF));
    // (from 2^30 on fp32 is off by more than 32, and further on by more than exp takes)
    const double top64 = fabsf(top) < 1073741824.0f ? (double)top : largest(score, p.E, lane);
    __syncthreads();                                  // (everybody has read the logits)
    double sum = 0.0;
    for (int e = (int)tid; e < p.E; e += THREADS) { const double v = exp(score[e] - top64); sum += v; score[e] = v; }
    if (!p.renorm || p.bias) {
      sum = warp_sum(sum);
      if (lane == 0) red[warp] = sum;
      __syncthreads();
      sum = red[0];
#pragma unroll
      for (int w = 1; w < ROUTE_WARPS; ++w) sum += red[w];
      inv = 1.0 / sum;
    }
  }
  for (int e = (int)tid; e < p.E; e += THREADS) {
    const double v = p.sigmoid ? 1.0 / (1.0 + exp(-score[e])) : score[e] * inv;
    score[e] = v;
    key[e] = rank_key(p.bias ? v + (double)p.bias[e] : v);
    if (e < ROUTE_COUNTED) place[e] = 0;
  }
  __syncthreads();
  int my_id = 0;
  if (p.E <= ROUTE_COUNTED) {
    // an expert's place is the number of those in front of it: larger keys, and equal ones of a lower index.  THREADS / E threads
    // share an expert's comparisons
    int width = 32;
    while (width < p.E) width *= 2;
    const int e = (int)tid & (width - 1), parts = THREADS / width, part = (int)tid / width;
    if (e < p.E) {
      const long long mine = key[e];
      int n = 0;
#pragma unroll 8
      for (int j = part; j < p.E; j += parts) {
        const long long other = key[j];
        n += other > mine || (other == mine && j < e) ? 1 : 0;
      }
      atomicAdd(&place[e], n);
    }
    __syncthreads();
    if ((int)tid < p.E && place[tid] < p.k) chosen[place[tid]] = (int)tid;
    __syncthreads();
    if (tid >= 32) return;
    if ((int)lane < p.k) my_id = chosen[lane];
  } else {
    if (tid >= 32) return;
    // k times the largest key that is left, of equal ones the lowest index; every lane keeps the best of its own
    constexpr long long NONE = (long long)0x8000000000000000ull;
    long long best = NONE;
    int at = 0x7FFFFFFF;
    auto scan = [&]() {
      best = NONE;
      at = 0x7FFFFFFF;
      for (int e = (int)lane; e < p.E; e += 32)
        if (key[e] > best) { best = key[e]; at = e; }
    };
    scan();
    for (int j = 0; j < p.k; ++j) {
      const int hi = (int)(best >> 32), top = __reduce_max_sync(0xffffffffu, hi);
      const uint32_t lo = hi == top ? (uint32_t)best : 0u, low = __reduce_max_sync(0xffffffffu, lo);
      const int win = __reduce_min_sync(0xffffffffu, hi == top && lo == low ? at : 0x7FFFFFFF);
      if ((int)lane == j) my_id = win;
      if (win == at) { key[win] = NONE; scan(); }
    }
  }
  const double v = (int)lane < p.k ? score[my_id] : 0.0, total = p.renorm ? warp_sum(v) : 1.0;
  if ((int)lane < p.k) {
    p.ids[t * p.k + lane] = my_id;
    p.weights[t * p.k + lane] = (float)(v / total * (double)p.scale);
  }
}

// ---- 16-bit operands ------------------------------------------------------------------------------------------------------------
constexpr int ROUTE_TOKENS = 8;                     // of a cluster: an MMA's columns, and one for each CTA
template <int DT>
__device__ __forceinline__ void mma_16x8x16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  if constexpr (DT == SDQ_BF16)
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
template <bool VEC>
__device__ __forceinline__ uint4 load8_raw(const uint16_t* p, int64_t n) {
  uint32_t w[4] = {0, 0, 0, 0};
  if constexpr (VEC) {
    asm volatile("{\n.reg .pred p;\nsetp.ne.u32 p, %5, 0;\n@p ld.global.nc.v4.u32 {%0, %1, %2, %3}, [%4];\n}"
                 : "+r"(w[0]), "+r"(w[1]), "+r"(w[2]), "+r"(w[3]) : "l"(p), "r"((uint32_t)(n > 0)));
  } else {
    uint16_t e[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      e[i] = 0;
      asm volatile("{\n.reg .pred p;\nsetp.ne.u32 p, %2, 0;\n@p ld.global.nc.u16 %0, [%1];\n}" : "+h"(e[i]) : "l"(p + 4 * i), "r"((uint32_t)(4 * i < n)));
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = (uint32_t)e[2 * i] | (uint32_t)e[2 * i + 1] << 16;
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
// The warps of a CTA share its K.  The K of the operands' fragments is permuted alike, which a sum does not see: lane 4 r + c loads K 8 c .. + 7 of a
// chunk of 32 of rows r and r + 8, one access each (or c, c + 4, ..), and its words 0, 1 and 2, 3 are the fragments of two MMAs.
// TILES tiles of sixteen experts at a time, loads in batches of BATCH chunks.
constexpr int ROUTE_BATCH = 4;
template <int DT, bool VEC, int TILES>
__global__ void __launch_bounds__(32 * ROUTE_WARPS)
moe_route_mma_kernel(const __grid_constant__ RouteParams p)
{
  extern __shared__ double s_logit[];               // [K splits][E], keys [E], sums of the warps
  const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, r = lane >> 2, first = (lane & 3) * (VEC ? 8 : 1);        // (of a chunk)
  const uint32_t rank = ptx::cluster_ctarank();
  const int64_t t0 = (int64_t)(blockIdx.x / ROUTE_CTAS) * ROUTE_TOKENS;
  long long* key = reinterpret_cast<long long*>(s_logit + (size_t)p.splits * p.elements);
  double* red = reinterpret_cast<double*>(key + p.elements);          // [warp][tile][16 experts][8 tokens]
  const uint16_t *X = reinterpret_cast<const uint16_t*>(p.x), *W = reinterpret_cast<const uint16_t*>(p.w);
  // this CTA's tiles and K
  const int tiles = (p.E + 15) / 16, split = p.splits > 1 ? (int)rank / tiles : 0, step = p.splits > 1 ? tiles : ROUTE_CTAS;
  const int chunks = (int)((p.H + 31) / 32), parts = p.splits * ROUTE_WARPS, part = split * ROUTE_WARPS + (int)warp;
  const int c0 = (int)((int64_t)part * chunks / parts), c1 = (int)((int64_t)(part + 1) * chunks / parts);
  cluster_arrive();
  ptx::griddep_wait();
  if (tid == 0) ptx::griddep_launch_dependents();
  const bool token = t0 + r < p.T;
  const uint16_t* x = X + (token ? t0 + r : 0) * p.ldx + first;
  bool waited = false;
  for (int tile = (int)rank - split * tiles; split < p.splits && tile < tiles; tile += TILES * step) {
    const uint16_t* w[TILES][2];
    bool have[TILES][2];
    double acc[TILES][4];
#pragma unroll
    for (int i = 0; i < TILES; ++i) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int e = (tile + i * step) * 16 + (int)r + 8 * j;
        have[i][j] = e < p.E;
        w[i][j] = W + (int64_t)(have[i][j] ? e : 0) * p.ldw + first;
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[i][j] = 0.0;
    }
    for (int c = c0; c < c1; c += ROUTE_BATCH) {
      uint4 b[ROUTE_BATCH], a[ROUTE_BATCH][TILES][2];
#pragma unroll
      for (int q = 0; q < ROUTE_BATCH; ++q) {
        const int64_t h = (int64_t)(c + q) * 32, n = c + q < c1 ? p.H - h - first : 0;
        b[q] = load8_raw<VEC>(x + h, token ? n : 0);
#pragma unroll
        for (int i = 0; i < TILES; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j) a[q][i][j] = load8_raw<VEC>(w[i][j] + h, have[i][j] ? n : 0);
      }
#pragma unroll
      for (int q = 0; q < ROUTE_BATCH; ++q)
#pragma unroll
        for (int i = 0; i < TILES; ++i) {
          const uint4 lo = a[q][i][0], hi = a[q][i][1];
          float d[4] = {0.0f, 0.0f, 0.0f, 0.0f};
          mma_16x8x16<DT>(d, lo.x, hi.x, lo.y, hi.y, b[q].x, b[q].y);
          mma_16x8x16<DT>(d, lo.z, hi.z, lo.w, hi.w, b[q].z, b[q].w);
#pragma unroll
          for (int j = 0; j < 4; ++j) acc[i][j] += (double)d[j];
        }
    }
    // accumulator j of lane 4 r + c: expert r + 8 (j / 2), token 2 c + j % 2
    __syncthreads();                                // (the sums of the tiles in front have been read)
#pragma unroll
    for (int i = 0; i < TILES; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) red[((warp * TILES + i) * 16 + r + 8 * (j >> 1)) * 8 + 2 * (lane & 3) + (j & 1)] = acc[i][j];
    __syncthreads();
    if (!waited) { cluster_wait(); waited = true; }  // all CTAs have started: their shared memory may be written
    for (int q = (int)tid; q < TILES * 128; q += 32 * ROUTE_WARPS) {
      const int e = (tile + (q >> 7) * step) * 16 + ((q >> 3) & 15);
      double s = 0.0;
#pragma unroll
      for (int v = 0; v < ROUTE_WARPS; ++v) s += red[v * TILES * 128 + q];
      if (e < p.E) store_to_cta(s_logit + (size_t)split * p.elements + e, (uint32_t)q & 7u, s);
    }
  }
  if (!waited) cluster_wait();
  ptx::cluster_sync();
  if (t0 + rank >= p.T) return;                     // token `rank` of the group is this CTA's
  if (p.splits > 1) {
    for (int e = (int)tid; e < p.E; e += 32 * ROUTE_WARPS) {
      double s = s_logit[e];
      for (int v = 1; v < p.splits; ++v) s += s_logit[(size_t)v * p.elements + e];
      s_logit[e] = s;
    }
    __syncthreads();
  }
  choose(p, t0 + rank, s_logit, key, red);
}

// ---- fp32 operands: G tokens a cluster --------------------------------------------------------------------------------------------
// A warp takes an expert at a time, its loads in batches (8 tokens x 4096 -> 64: 8.0 us, against 8.9 without; 64 -> 256 60 and 49); a row
// that cannot be read in 16-byte pieces goes element by element.
template <int G, bool VEC>
__global__ void __launch_bounds__(32 * ROUTE_WARPS)
moe_route_kernel(const __grid_constant__ RouteParams p)
{
  static_assert(G <= ROUTE_CTAS);
  extern __shared__ double s_logit[];        // [E], keys [E], sums of the warps
  const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = ptx::cluster_ctarank();
  ptx::griddep_wait();
  if (threadIdx.x == 0) ptx::griddep_launch_dependents();
  const int64_t t0 = (int64_t)(blockIdx.x / ROUTE_CTAS) * G;
  const float *X = reinterpret_cast<const float*>(p.x), *W = reinterpret_cast<const float*>(p.w);
  ptx::cluster_sync();                       // (all CTAs have started: their shared memory may be written)
  for (int e = (int)(rank * ROUTE_WARPS + warp); e < p.E; e += ROUTE_CTAS * ROUTE_WARPS) {
    double acc[G];
#pragma unroll
    for (int g = 0; g < G; ++g) acc[g] = 0.0;
    constexpr int BATCH = G == 1 ? 4 : 2;
    for (int64_t h0 = VEC ? lane * 8 : lane; h0 < p.H; h0 += 256 * BATCH) {
      float w[BATCH][8], x[BATCH][G][8];
#pragma unroll
      for (int q = 0; q < BATCH; ++q) {
        const int64_t h = h0 + 256 * q;
        load8<VEC>(w[q], W + (int64_t)e * p.ldw + h, p.H - h);
#pragma unroll
        for (int g = 0; g < G; ++g) load8<VEC>(x[q][g], X + (t0 + g) * p.ldx + h, t0 + g < p.T ? p.H - h : 0);
      }
#pragma unroll
      for (int q = 0; q < BATCH; ++q)
#pragma unroll
        for (int g = 0; g < G; ++g) {
          float s = 0.0f;
#pragma unroll
          for (int i = 0; i < 8; ++i) s = fmaf(w[q][i], x[q][g][i], s);
          acc[g] += (double)s;
        }
    }
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const double l = warp_sum(acc[g]);
      if (lane == 0) store_to_cta(s_logit + e, (uint32_t)g, l);
    }
  }
  ptx::cluster_sync();
  // token `rank` of the group is this CTA's
  if (rank >= G || t0 + rank >= p.T) return;
  long long* key = reinterpret_cast<long long*>(s_logit + p.elements);
  choose(p, t0 + rank, s_logit, key, reinterpret_cast<double*>(key + p.elements));
}

template <typename K>
static sdq_status_t launch_route(K kern, const RouteParams& p, int64_t groups, size_t smem, void* stream) {
  cudaLaunchConfig_t lc = {};
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = ROUTE_CTAS;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  if (groups > 0x7FFFFFFF / ROUTE_CTAS) return SDQ_ERR_SHAPE;
  lc.gridDim = dim3((unsigned)groups * ROUTE_CTAS);
  lc.blockDim = dim3(32 * ROUTE_WARPS);
  lc.dynamicSmemBytes = smem;
  lc.stream = (cudaStream_t)stream;
  lc.attrs = attr;
  lc.numAttrs = 2;
  return launch_status(cudaLaunchKernelEx(&lc, kern, p));
}
template <int DT>
static sdq_status_t route16(RouteParams p, bool vec, void* stream) {
  const int tiles = (p.E + 15) / 16;
  static_assert(ROUTE_TOKENS == ROUTE_CTAS);
  p.splits = tiles < ROUTE_CTAS ? ROUTE_CTAS / tiles : 1;
  const size_t smem = ((size_t)p.splits + 1) * p.elements * 8 + (size_t)ROUTE_WARPS * (tiles > ROUTE_CTAS ? 2 : 1) * 128 * 8;
  const int64_t groups = (p.T + ROUTE_TOKENS - 1) / ROUTE_TOKENS;
  auto go = [&](auto kern) { return launch_route(kern, p, groups, smem, stream); };
  if (tiles > ROUTE_CTAS) return vec ? go(moe_route_mma_kernel<DT, true, 2>) : go(moe_route_mma_kernel<DT, false, 2>);
  return vec ? go(moe_route_mma_kernel<DT, true, 1>) : go(moe_route_mma_kernel<DT, false, 1>);
}
template <int G>
static sdq_status_t route32(const RouteParams& p, bool vec, void* stream) {
  const size_t smem = 2 * (size_t)p.elements * 8 + ROUTE_WARPS * 8 + 8 * ROUTE_COUNTED;
  const int64_t groups = (p.T + G - 1) / G;
  return vec ? launch_route(moe_route_kernel<G, true>, p, groups, smem, stream) : launch_route(moe_route_kernel<G, false>, p, groups, smem, stream);
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
  const RouteParams p = {X, Wr, bias, ids, weights, T, H, ldx, ldw, (int32_t)E, k, scoring == SDQ_ROUTE_SIGMOID, renorm != 0, (int32_t)(E + 1) / 2 * 2, 1, scale};
  if (dtype == SDQ_BF16) return route16<SDQ_BF16>(p, vec, stream);
  if (dtype == SDQ_FP16) return route16<SDQ_FP16>(p, vec, stream);
  return T <= 8 ? route32<1>(p, vec, stream) : route32<4>(p, vec, stream);      // (few tokens: more clusters)
}
