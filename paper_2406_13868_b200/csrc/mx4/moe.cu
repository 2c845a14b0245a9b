// Expert layer of a few tokens over MXFP4 experts:  Y[t] = sum_j weights[t][j] * W2[e](silu(W1[e] x_t) * W3[e] x_t),  e = ids[t][j].
//
// The chosen experts' weights are what has to be read, each once however many tokens chose it.  They are multiplied as they are, in four
// bits, by activations that are not quantized: the 8-bit block-scaled kind takes E2M1 weights (padded to bytes by the copy into shared
// memory) and E4M3 activations, and an activation is a sum of E4M3 pieces -- with the block's largest magnitude in [128, 256) * 2^s,
//   x = 2^s (p0 + p1 / 16 + p2 / 256),   p0 = e4m3(x / 2^s), p1 = e4m3(16 (x / 2^s - p0)), p2 = e4m3(16 (16 (x / 2^s - p0) - p1)),
// every remainder exact, four significant bits a piece: two pieces hold a bf16 exactly down to 2^-14 of its block's largest
// magnitude (and to 2^-22 of that below), three an fp16 (11 bits) and what silu(.) * (.) leaves to 12 bits.  Pieces are columns of the MMA of their
// own, each with its scale 2^s, 2^(s-4), 2^(s-8), and are added in the epilogue: few tokens leave columns to spare, and the weights are
// fetched into the tensor core once for all of them.
//
// Three launches: the pairs (token, choice) are sorted by expert into units of up to 40 pairs; moe_split_kernel writes X in pieces;
// moe_up_kernel forms silu(W1 x) * (W3 x), 128 rows of both a task, and writes it in pieces; moe_down_kernel forms W2 h, adds up every
// token's pairs in a fixed order and rounds once.  Where tasks are too few for the GPU, the CTAs of a cluster split K and add their fp32
// partial sums through distributed shared memory, in a fixed order.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include <mutex>

#include "../sdq_codec.cuh"
#include "../sdq_internal.h"
#include "../sdq_ptx.cuh"
#include "layout.h"

namespace sdq {
namespace mx4 {

constexpr int MOE_MAX_T = 64, MOE_MAX_K = 32, MOE_MAX_E = 1024;
// Pairs of a unit, at most: three pieces of 40 are 120 columns.  Smaller units where there are fewer tokens bound what a CTA has to have
// room for; a token may name an expert more than once, so that the number of tokens alone bounds nothing.
__host__ __device__ constexpr int unit_pairs(int64_t T) { return T <= 8 ? 8 : T <= 16 ? 16 : 40; }
constexpr int H_PIECES = 3;                     // of silu(.) * (.)

// ---- workspace --------------------------------------------------------------------------------------------------------------
struct MoeUnit { int32_t expert, n, pair0, gx, gh; };        // pairs pair0 .. + n of the sorted list; first 8-row group of its pieces of X and h
struct MoeOffsets {
  size_t pairs, xp, xs, hp, hs, total;
  int32_t gx, gh, sh, si;                                    // 8-row groups of a step (bounds), steps of H and I
};
inline MoeOffsets moe_offsets(int64_t T, int k, int64_t H, int64_t I) {
  MoeOffsets o;
  auto al = [](size_t x) { return (x + 255) & ~(size_t)255; };
  const int64_t P = T * k;                                    // units have at least one pair, and up to 7 rows of padding
  o.sh = (int32_t)((H + KSTEP - 1) / KSTEP);
  o.si = (int32_t)((I + KSTEP - 1) / KSTEP);
  o.gx = (int32_t)((P * 3 + 7 * P) / 8 + 1);
  o.gh = (int32_t)((P * H_PIECES + 7 * P) / 8 + 1);
  o.pairs = 0;
  o.xp = al((size_t)P * 4);
  o.xs = al(o.xp + (size_t)o.sh * o.gx * 1024);
  o.hp = al(o.xs + (size_t)P * o.sh * ATOM);
  o.hs = al(o.hp + (size_t)o.si * o.gh * 1024);
  o.total = al(o.hs + (size_t)P * o.si * ATOM);
  return o;
}

struct MoeParams {
  const void* x;
  const int32_t* ids;
  const float* weights;
  void* y;
  uint8_t* ws;
  MoeOffsets off;
  const uint8_t *s1, *s3, *s2;                                // weight scales
  int64_t ldx, ldy;
  int32_t T, k, E, H, I, tiles_h, tiles_i;                    // row tiles of 128 of an expert's matrices
  int32_t unit, max_units;                                    // unit_pairs; units there can be
  int32_t ring_bytes, tmem_cols;
  uint32_t* flags;
};

// row r (of a unit's columns), byte k (0 .. 127) of a step: inside the unit's groups
__device__ __forceinline__ uint32_t piece_off(uint32_t r, uint32_t k) { return (r >> 3) * 1024 + (k >> 4) * 128 + (r & 7) * 16 + (k & 15); }

// ---- pieces -------------------------------------------------------------------------------------------------------------------
// code c of the block's scale 2^(c - 127): the largest magnitude lands in [128, 256); at least 8, so that the later pieces' scales
// (c - 4, c - 8) are codes too
__device__ __forceinline__ uint32_t piece_scale(uint32_t amax_bits) { return (uint32_t)min(max((int)(amax_bits >> 23) - 7, 8), 247); }
// codes of the pieces of x (scaled by inv = 2^(127 - c)); what is not finite: NaN
template <int P>
__device__ __forceinline__ void pieces(float x, float inv, uint32_t (&c)[P]) {
  float r = x * inv;
  const bool bad = !(fabsf(x) <= 3.4028234663852886e38f);
#pragma unroll
  for (int i = 0; i < P; ++i) {
    c[i] = e4m3x1(r);
    const __half_raw h = __nv_cvt_fp8_to_halfraw((__nv_fp8_storage_t)c[i], __NV_E4M3);
    r = (r - __half2float(__half(h))) * 16.0f;
  }
  if (bad) c[0] = 0x7Fu;
}

// ---- pairs by expert --------------------------------------------------------------------------------------------------------------
// Every CTA of the three kernels makes the list of units for itself, from the ids: that is quicker than to wait for another CTA's.
// `s_n`: [E] pairs of an expert; the warp returns the number of units (all lanes) after calling each(lane's expert, its first unit, pair, group of X,
// group of h)
struct Plan { int units, most; };                // units, pairs of the largest
template <int P, typename F>
__device__ __forceinline__ Plan plan_units(const int32_t* s_n, int E, int unit, uint32_t lane, F each) {
  int4 base = make_int4(0, 0, 0, 0);
  int most = 0;
  for (int e0 = 0; e0 < E; e0 += 32) {
    const int e = e0 + (int)lane, n = e < E ? s_n[e] : 0, full = n / unit, rest = n - full * unit;
    const int4 own = make_int4(full + (rest ? 1 : 0), n, full * (P * unit / 8) + (P * rest + 7) / 8, full * (H_PIECES * unit / 8) + (H_PIECES * rest + 7) / 8);
    int4 v = own;
    most = max(most, n);
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int4 u = make_int4(__shfl_up_sync(0xffffffffu, v.x, o), __shfl_up_sync(0xffffffffu, v.y, o), __shfl_up_sync(0xffffffffu, v.z, o), __shfl_up_sync(0xffffffffu, v.w, o));
      if ((int)lane >= o) { v.x += u.x; v.y += u.y; v.z += u.z; v.w += u.w; }
    }
    if (e < E) each(e, n, make_int4(base.x + v.x - own.x, base.y + v.y - own.y, base.z + v.z - own.z, base.w + v.w - own.w));
    base.x += __shfl_sync(0xffffffffu, v.x, 31); base.y += __shfl_sync(0xffffffffu, v.y, 31);
    base.z += __shfl_sync(0xffffffffu, v.z, 31); base.w += __shfl_sync(0xffffffffu, v.w, 31);
  }
  return Plan{base.x, min(__reduce_max_sync(0xffffffffu, most), unit)};
}
// the units themselves, in shared memory (all threads of the CTA; s_n is scratch of E words)
template <int P>
__device__ __forceinline__ Plan make_units(const MoeParams& p, MoeUnit* s_unit, int32_t* s_n, Plan* s_plan) {
  const uint32_t tid = threadIdx.x, lane = tid & 31;
  for (int e = (int)tid; e < p.E; e += (int)blockDim.x) s_n[e] = 0;
  __syncthreads();
  for (int i = (int)tid; i < p.T * p.k; i += (int)blockDim.x) {
    const int e = p.ids[i];
    if (e >= 0 && e < p.E) atomicAdd(&s_n[e], 1);
  }
  __syncthreads();
  if (tid < 32) {
    const int unit = p.unit;
    const Plan r = plan_units<P>(s_n, p.E, unit, lane, [&](int e, int n, int4 at) {
      for (int u = 0; n > 0; ++u, n -= unit)
        s_unit[at.x + u] = MoeUnit{e, min(n, unit), at.y + u * unit, at.z + u * (P * unit / 8), at.w + u * (H_PIECES * unit / 8)};
    });
    if (lane == 0) *s_plan = r;
  }
  __syncthreads();
  return *s_plan;
}

// ---- X in pieces ------------------------------------------------------------------------------------------------------------------
constexpr int SPLIT_THREADS = 256;
template <int DT>
__global__ void __launch_bounds__(SPLIT_THREADS)
moe_split_kernel(const __grid_constant__ MoeParams p)
{
  constexpr int P = DT == SDQ_BF16 ? 2 : 3;
  extern __shared__ int32_t s_split[];
  const int pairs = p.T * p.k, padded = (pairs + 3) / 4 * 4;
  int32_t* s_id = s_split;                       // expert of a pair (-1: none)
  int32_t* s_rank = s_id + padded;               // its place among the expert's pairs
  int4* s_at = reinterpret_cast<int4*>(s_rank + padded);   // first unit, pair, group of X, group of h
  int32_t* s_n = reinterpret_cast<int32_t*>(s_at + p.E);   // pairs of an expert
  const int tid = (int)threadIdx.x;
  ptx::griddep_wait();
  // (behind the wait: what the next launch reads in front of its own, ids and weights, is complete then)
  if (tid == 0) ptx::griddep_launch_dependents();
  for (int i = tid; i < padded; i += SPLIT_THREADS) {
    const int e = i < pairs ? p.ids[i] : -1;
    s_id[i] = e >= 0 && e < p.E ? e : -1;
  }
  __syncthreads();
  for (int e = tid; e < p.E; e += SPLIT_THREADS) {
    int n = 0;
#pragma unroll 4
    for (int i = 0; i < padded; i += 4) {
      const int4 q = *reinterpret_cast<const int4*>(s_id + i);
      if (q.x == e) s_rank[i] = n++;
      if (q.y == e) s_rank[i + 1] = n++;
      if (q.z == e) s_rank[i + 2] = n++;
      if (q.w == e) s_rank[i + 3] = n++;
    }
    s_n[e] = n;
  }
  __syncthreads();
  if (tid < 32) plan_units<P>(s_n, p.E, p.unit, (uint32_t)tid, [&](int e, int, int4 at) { s_at[e] = at; });
  __syncthreads();
  if (blockIdx.x == 0)
    for (int i = tid; i < pairs; i += SPLIT_THREADS)
      if (s_id[i] >= 0) reinterpret_cast<int32_t*>(p.ws + p.off.pairs)[s_at[s_id[i]].y + s_rank[i]] = i;
  // eight elements of a token a thread; four lanes have a block of 32
  using T = typename std::conditional<DT == SDQ_BF16, __nv_bfloat16, __half>::type;
  const int eighths = 16 * p.off.sh;             // of a row, padded to whole steps
  const bool vec = ((uintptr_t)p.x & 15) == 0 && p.ldx % 8 == 0;
  for (int w = (int)blockIdx.x * SPLIT_THREADS + tid; w < p.T * eighths; w += (int)gridDim.x * SPLIT_THREADS) {   // (a multiple of 16: lanes of a block stay together)
    const int t = w / eighths, b = w - t * eighths, h0 = 8 * b;
    const T* row = reinterpret_cast<const T*>(p.x) + (int64_t)t * p.ldx;
    T e8[8];
    if (vec && h0 + 8 <= p.H) {
      *reinterpret_cast<uint4*>(e8) = *reinterpret_cast<const uint4*>(row + h0);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) e8[i] = h0 + i < p.H ? row[h0 + i] : (T)0.0f;
    }
    float v[8];
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) { v[i] = (float)e8[i]; m = max(m, __float_as_uint(v[i]) & 0x7FFFFFFFu); }
    const uint32_t four = 0xFu << (tid & 28);
    m = max(m, __shfl_xor_sync(four, m, 1));
    m = max(m, __shfl_xor_sync(four, m, 2));
    const uint32_t c = piece_scale(m);
    const float inv = __uint_as_float((254u - c) << 23);
    uint32_t code[P][2];
#pragma unroll
    for (int j = 0; j < P; ++j) code[j][0] = code[j][1] = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      uint32_t q[P];
      pieces<P>(v[i], inv, q);
#pragma unroll
      for (int j = 0; j < P; ++j) code[j][i / 4] |= q[j] << (8 * (i % 4));
    }
    const int step = b >> 4;
    for (int j = 0; j < p.k; ++j) {
      const int i = t * p.k + j, e = s_id[i];
      if (e < 0) continue;
      const int u = s_rank[i] / p.unit, r = s_rank[i] - u * p.unit;
      const int4 at = s_at[e];
      uint8_t* dst = p.ws + p.off.xp + ((size_t)step * p.off.gx + at.z + u * (P * p.unit / 8)) * 1024;
      uint8_t* sc = p.ws + p.off.xs + ((size_t)(at.x + u) * p.off.sh + step) * ATOM;
#pragma unroll
      for (int q = 0; q < P; ++q) {
        *reinterpret_cast<uint2*>(dst + piece_off((uint32_t)(P * r + q), (uint32_t)(h0 & 127))) = make_uint2(code[q][0], code[q][1]);
        if ((b & 3) == q) sc[atom_off((uint32_t)(P * r + q), (uint32_t)((b >> 2) & 3))] = (uint8_t)(c - 4 * q);
      }
    }
  }
}

// ---- what the two products share ------------------------------------------------------------------------------------------------
constexpr int MOE_THREADS = 384;                  // weights' producer, MMA issuer, activations' producer, one that lets the next launch in, eight epilogue warps
constexpr int MOE_MAX_SLOTS = 12;
constexpr uint32_t A_BYTES = 16384;               // an expert's tile and step in shared memory
constexpr uint32_t SMEM_MAX = 232448;
constexpr int CHUNK = 16;                         // tokens the epilogue takes at a time

struct MoeBars {
  uint64_t full[MOE_MAX_SLOTS], empty[MOE_MAX_SLOTS], acc_full[2], acc_empty[2], part_full, part_empty;
  uint32_t tmem, timed_out;
  Plan plan;
};
// (the tensor map's rows are core matrices: 128 of a tile and step)
__device__ __forceinline__ void load_tile(const CUtensorMap* map, uint8_t* dst, int core, uint64_t* bar) {
  asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];" ::"r"(ptx::smem_u32(dst)), "l"(map),
               "r"(ptx::smem_u32(bar)), "r"(0), "r"(core) : "memory");
}
// copies of the scales and the four MMAs (32 K each) of one step; nothing accumulates in front of the first where `acc` is 0
__device__ __forceinline__ void step_mma(uint32_t d, uint32_t a, uint32_t b, uint32_t sfa, uint32_t sfb, const uint32_t (&id)[4], uint32_t acc) {
  const uint64_t da = ptx::smem_desc(a, 128, 1024), db = ptx::smem_desc(b, 128, 1024);
#pragma unroll
  for (uint32_t j = 0; j < 4; ++j) ptx::mma_mxf8(d, da + ((256 * j) >> 4), db + ((256 * j) >> 4), id[j], sfa, sfb, j ? 1u : acc);
}
__device__ __forceinline__ void arrive_cta(uint64_t* bar, uint32_t cta) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(ptx::mapa_u32(ptx::smem_u32(bar), cta)) : "memory");
}
__device__ __forceinline__ float4 load_cta4(const float* local, uint32_t cta) { return ptx::ld_cluster_f32x4(ptx::mapa_u32(ptx::smem_u32(local), cta)); }
// sums of the P pieces of 16 consecutive tokens, this lane's row (columns col .. + 16 P - 1)
template <int P>
__device__ __forceinline__ void load_tokens(uint32_t taddr, float (&s)[16]) {
  uint32_t v[16 * P];
#pragma unroll
  for (int i = 0; i < P; ++i) ptx::tmem_ld_32x32b_x16(taddr + 16u * i, *reinterpret_cast<uint32_t(*)[16]>(v + 16 * i));
  ptx::tmem_ld_wait();
#pragma unroll
  for (int t = 0; t < 16; ++t) {
    s[t] = __uint_as_float(v[P * t + P - 1]);      // (the smallest first)
#pragma unroll
    for (int q = P - 2; q >= 0; --q) s[t] += __uint_as_float(v[P * t + q]);
  }
}

// ---- silu(W1 x) * (W3 x) ----------------------------------------------------------------------------------------------------------
// slot = | tile of W1 | tile of W3 | their scale atoms | columns of X | scale atom |
template <int P>
__global__ void __launch_bounds__(MOE_THREADS)
moe_up_kernel(const __grid_constant__ MoeParams p, const __grid_constant__ CUtensorMap m1, const __grid_constant__ CUtensorMap m3)
{
  extern __shared__ uint8_t smem_raw[];
  uint8_t* sm = smem_raw + ((128 - (ptx::smem_u32(smem_raw) & 127)) & 127);
  __shared__ MoeBars b;
  const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  constexpr uint32_t SL_SF = 2 * A_BYTES, SL_B = SL_SF + 2 * ATOM;
  float* part = reinterpret_cast<float*>(sm + p.ring_bytes);              // [token of the chunk][W1 or W3][128 rows]
  MoeUnit* s_unit = reinterpret_cast<MoeUnit*>(part + CHUNK * 256);
  uint32_t ks;
  asm volatile("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(ks));
  const uint32_t rank = ptx::cluster_ctarank();
  const int cluster = (int)(blockIdx.x / ks), clusters = (int)(gridDim.x / ks);
  const int k0 = (int)(rank * (uint32_t)p.off.sh / ks), steps = (int)((rank + 1) * (uint32_t)p.off.sh / ks) - k0;
  if (warp == 0) {
    if (lane == 0) {
      for (int i = 0; i < MOE_MAX_SLOTS; ++i) { ptx::mbar_init(&b.full[i], 2); ptx::mbar_init(&b.empty[i], 1); }
      for (int i = 0; i < 2; ++i) { ptx::mbar_init(&b.acc_full[i], 1); ptx::mbar_init(&b.acc_empty[i], 8); }
      ptx::mbar_init(&b.part_full, ks);
      ptx::mbar_init(&b.part_empty, ks);
      b.timed_out = 0;
      ptx::fence_barrier_init();
    }
    __syncwarp();
  } else if (warp == 1) {
    ptx::tmem_alloc(&b.tmem, (uint32_t)p.tmem_cols);
  }
  // ids and weights are complete: the launch in front, the split, lets this one in behind its own wait
  const Plan plan = make_units<P>(p, s_unit, reinterpret_cast<int32_t*>(part), &b.plan);
  ptx::tc_fence_before();
  __syncthreads();
  ptx::cluster_sync();
  ptx::tc_fence_after();
  const int tasks = plan.units * p.tiles_i;
  const uint32_t COLS = (uint32_t)(P * plan.most + 15) / 16 * 16;         // columns of the largest unit there is
  const uint32_t SLOT = SL_B + COLS * 128u + ATOM, NSLOT = min((uint32_t)p.ring_bytes / SLOT, (uint32_t)MOE_MAX_SLOTS), SL_SFB = SL_B + COLS * 128u;
  const uint32_t tmem = b.tmem, bufs = 4 * COLS + 32 <= (uint32_t)p.tmem_cols ? 2u : 1u, sets = tmem + 2 * bufs * COLS;
  bool ok = true;
  if (warp == 0) {
    if (lane == 0) {
      uint32_t i = 0, s = 0, ph = 1;
      for (int task = cluster; task < tasks && ok; task += clusters) {
        const int u = task / p.tiles_i, tile = task - u * p.tiles_i;
        size_t at = ((size_t)s_unit[u].expert * p.tiles_i + tile) * p.off.sh + k0;
        for (int k = 0; k < steps; ++k, ++i, ++at) {
          if (i >= NSLOT && !(ok = ptx::mbar_wait(&b.empty[s], ph))) break;
          uint8_t* st = sm + (size_t)s * SLOT;
          // (the tensor copies count the bytes they read: the padding is not written)
          ptx::mbar_expect_tx(&b.full[s], 2 * ECODES + 2 * ATOM);
          load_tile(&m1, st, (int)at * 128, &b.full[s]);
          load_tile(&m3, st + A_BYTES, (int)at * 128, &b.full[s]);
          ptx::bulk_g2s(st + SL_SF, p.s1 + at * ATOM, ATOM, &b.full[s]);
          ptx::bulk_g2s(st + SL_SF + ATOM, p.s3 + at * ATOM, ATOM, &b.full[s]);
          if (++s == NSLOT) { s = 0; ph ^= 1u; }
        }
      }
      if (!ok) atomicOr(&p.flags[FLAG_TIMEOUT], 1u);
    }
    __syncwarp();
  } else if (warp == 3) {
    // the next launch is let in behind the wait: what lies in front of this one is complete for it
    ptx::griddep_wait();
    if (lane == 0) ptx::griddep_launch_dependents();
  } else if (warp == 2) {
    ptx::griddep_wait();                          // X in pieces
    if (lane == 0) {
      uint32_t i = 0, s = 0, ph = 1;
      for (int task = cluster; task < tasks && ok; task += clusters) {
        const int u = task / p.tiles_i;
        const MoeUnit un = s_unit[u];
        const uint32_t bytes = (uint32_t)(P * un.n + 7) / 8 * 1024u;
        const uint8_t *x = p.ws + p.off.xp + ((size_t)k0 * p.off.gx + un.gx) * 1024, *sf = p.ws + p.off.xs + ((size_t)u * p.off.sh + k0) * ATOM;
        for (int k = 0; k < steps; ++k, ++i, x += (size_t)p.off.gx * 1024, sf += ATOM) {
          if (i >= NSLOT && !(ok = ptx::mbar_wait(&b.empty[s], ph))) break;
          uint8_t* st = sm + (size_t)s * SLOT;
          ptx::mbar_expect_tx(&b.full[s], bytes + ATOM);
          ptx::bulk_g2s(st + SL_B, x, bytes, &b.full[s]);
          ptx::bulk_g2s(st + SL_SFB, sf, ATOM, &b.full[s]);
          if (++s == NSLOT) { s = 0; ph ^= 1u; }
        }
      }
      if (!ok) atomicOr(&p.flags[FLAG_TIMEOUT], 1u);
    }
    __syncwarp();
  } else if (warp == 1) {
    if (lane == 0) {
      uint32_t i = 0, t = 0, s = 0, ph = 0;
      for (int task = cluster; task < tasks && ok; task += clusters, ++t) {
        const uint32_t N = (uint32_t)(P * s_unit[task / p.tiles_i].n + 15) / 16 * 16, buf = bufs == 2 ? t & 1u : 0u, use = bufs == 2 ? t >> 1 : t;
        const uint32_t acc = tmem + buf * 2 * COLS;
        uint32_t id[4];
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) id[j] = ptx::idesc_mxf8_e2m1_e4m3(128, N, j);
        if (use > 0 && !(ok = ptx::mbar_wait(&b.acc_empty[buf], (use - 1) & 1u))) break;
        for (int k = 0; k < steps; ++k, ++i) {
          if (!(ok = ptx::mbar_wait(&b.full[s], ph))) break;
          ptx::tc_fence_after();
          const uint32_t st = ptx::smem_u32(sm) + s * SLOT, sf = sets + (i & 1u) * 12u;
          ptx::tc_cp_32x128b_warpx4(sf, ptx::smem_desc(st + SL_SF, 0, 128));
          ptx::tc_cp_32x128b_warpx4(sf + 4, ptx::smem_desc(st + SL_SF + ATOM, 0, 128));
          ptx::tc_cp_32x128b_warpx4(sf + 8, ptx::smem_desc(st + SL_SFB, 0, 128));
          step_mma(acc, st, st + SL_B, sf, sf + 8, id, k ? 1u : 0u);
          step_mma(acc + COLS, st + A_BYTES, st + SL_B, sf + 4, sf + 8, id, k ? 1u : 0u);
          ptx::tc_commit(&b.empty[s]);
          if (++s == NSLOT) { s = 0; ph ^= 1u; }
        }
        if (ok) ptx::tc_commit(&b.acc_full[buf]);
      }
      if (!ok) atomicOr(&p.flags[FLAG_TIMEOUT], 1u);
    }
    __syncwarp();
  } else if (warp >= 4) {
    // Epilogue: warps 4 to 7 read W1's accumulator, 8 to 11 W3's, 16 tokens at a time, into shared memory; then eight lanes have the 32
    // rows of a token that make a block, four rows each (in tensor memory's own order, a row a thread, every code was a store of its own)
    const uint32_t q = warp & 3, which = (warp - 4) >> 2, row = q * 32 + lane, et = tid - 128;
    ptx::griddep_wait();                          // (h of the call in front may still be read)
    volatile uint32_t* timed_out = &b.timed_out;
    uint32_t t = 0, chunks = 0;
    for (int task = cluster; task < tasks; task += clusters, ++t) {
      const int u = task / p.tiles_i, tile = task - u * p.tiles_i;
      const MoeUnit un = s_unit[u];
      const uint32_t buf = bufs == 2 ? t & 1u : 0u, use = bufs == 2 ? t >> 1 : t;
      uint8_t* hp = p.ws + p.off.hp + ((size_t)tile * p.off.gh + un.gh) * 1024;
      uint8_t* hs = p.ws + p.off.hs + ((size_t)u * p.off.si + tile) * ATOM;
      if (et == 0 && !(ok = ptx::mbar_wait(&b.acc_full[buf], use & 1u))) *timed_out = 1u;
      for (int t0 = 0; t0 < un.n; t0 += CHUNK, ++chunks) {
        if (et == 0 && ks > 1 && chunks > 0 && !ptx::mbar_wait_cluster(&b.part_empty, (chunks - 1) & 1u)) { ok = false; *timed_out = 1u; }
        ptx::named_bar_sync(1, 256);
        if (*timed_out) break;
        ptx::tc_fence_after();
        const int n = min(CHUNK, un.n - t0);
        float v[CHUNK];
        load_tokens<P>(tmem + ((q * 32u) << 16) + buf * 2 * COLS + which * COLS + (uint32_t)(P * t0), v);
#pragma unroll
        for (int j = 0; j < CHUNK; ++j)
          if (j < n) part[j * 256 + which * 128 + row] = v[j];
        if (t0 + CHUNK >= un.n) {                 // the accumulator has been read
          ptx::tc_fence_before();
          __syncwarp();
          if (lane == 0) ptx::mbar_arrive(&b.acc_empty[buf]);
        }
        ptx::named_bar_sync(1, 256);
        if (ks > 1) {
          // (one thread's acquire, and the barrier behind it, order the peers' stores before everybody's loads)
          if (et < ks) arrive_cta(&b.part_full, et);
          if (et == 0 && !ptx::mbar_wait_cluster(&b.part_full, chunks & 1u)) { ok = false; *timed_out = 1u; }
          ptx::named_bar_sync(1, 256);
          if (*timed_out) break;
        }
        // (token, block of 32 rows) by (token, block), spread over the cluster's CTAs; eight lanes one
        for (int c = (int)(rank + ks * (et >> 3)); c < 4 * n; c += (int)(32 * ks)) {
          const int tok = c >> 2;
          const uint32_t blk = (uint32_t)c & 3u, r0 = blk * 32 + (et & 7u) * 4;
          const float* src = part + tok * 256 + r0;
          float4 g = make_float4(0, 0, 0, 0), w = g;
          if (ks == 1) {
            g = *reinterpret_cast<const float4*>(src);
            w = *reinterpret_cast<const float4*>(src + 128);
          } else {
            for (uint32_t r = 0; r < ks; ++r) {
              const float4 a = load_cta4(src, r), d = load_cta4(src + 128, r);
              g.x += a.x; g.y += a.y; g.z += a.z; g.w += a.w;
              w.x += d.x; w.y += d.y; w.z += d.z; w.w += d.w;
            }
          }
          const float h[4] = {g.x / (1.0f + expf(-g.x)) * w.x, g.y / (1.0f + expf(-g.y)) * w.y, g.z / (1.0f + expf(-g.z)) * w.z, g.w / (1.0f + expf(-g.w)) * w.w};
          uint32_t m = 0;
#pragma unroll
          for (int j = 0; j < 4; ++j) m = max(m, __float_as_uint(h[j]) & 0x7FFFFFFFu);
          const uint32_t mask = 0xFFu << (lane & 24u);
          m = max(m, __shfl_xor_sync(mask, m, 1));
          m = max(m, __shfl_xor_sync(mask, m, 2));
          m = max(m, __shfl_xor_sync(mask, m, 4));
          const uint32_t sc = piece_scale(m);
          const float inv = __uint_as_float((254u - sc) << 23);
          uint32_t code[H_PIECES] = {0, 0, 0};
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            uint32_t x[H_PIECES];
            pieces<H_PIECES>(h[j], inv, x);
#pragma unroll
            for (int i = 0; i < H_PIECES; ++i) code[i] |= x[i] << (8 * j);
          }
#pragma unroll
          for (uint32_t i = 0; i < H_PIECES; ++i) {
            const uint32_t r = (uint32_t)(H_PIECES * (t0 + tok)) + i;
            *reinterpret_cast<uint32_t*>(hp + piece_off(r, r0)) = code[i];
            if ((et & 7u) == i) hs[atom_off(r, blk)] = (uint8_t)(sc - 4 * i);
          }
        }
        if (ks > 1) {
          ptx::named_bar_sync(1, 256);
          if (et < ks) arrive_cta(&b.part_empty, et);
        }
      }
      if (*timed_out) break;
    }
    if (et == 0 && !ok) atomicOr(&p.flags[FLAG_TIMEOUT], 1u);
    __syncwarp();
  }
  ptx::tc_fence_before();
  __syncthreads();
  ptx::cluster_sync();                             // nobody leaves while its partial sums are being read
  if (warp == 1) ptx::tmem_dealloc(tmem, (uint32_t)p.tmem_cols);
}

// ---- W2 h, and the sum over a token's pairs -------------------------------------------------------------------------------------
// A cluster has one tile of 128 outputs; its CTAs share the steps of all units.  slot = | tile of W2 | scale atom | columns of h | scale atom |
template <int DT>
__global__ void __launch_bounds__(MOE_THREADS)
moe_down_kernel(const __grid_constant__ MoeParams p, const __grid_constant__ CUtensorMap m2)
{
  using T = typename std::conditional<DT == SDQ_BF16, __nv_bfloat16, __half>::type;
  constexpr int P = H_PIECES;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* sm = smem_raw + ((128 - (ptx::smem_u32(smem_raw) & 127)) & 127);
  __shared__ MoeBars b;
  const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  constexpr uint32_t SL_SF = A_BYTES, SL_B = SL_SF + ATOM;
  uint32_t ks;
  asm volatile("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(ks));
  const uint32_t rank = ptx::cluster_ctarank();
  const int tile = (int)(blockIdx.x / ks), pairs = p.T * p.k;
  float* out = reinterpret_cast<float*>(sm + p.ring_bytes);               // [token][128 rows]
  int2* s_pair = reinterpret_cast<int2*>(out + p.T * 128);                // pairs by unit: token, weight
  MoeUnit* s_unit = reinterpret_cast<MoeUnit*>(s_pair + pairs);
  if (warp == 0) {
    if (lane == 0) {
      for (int i = 0; i < MOE_MAX_SLOTS; ++i) { ptx::mbar_init(&b.full[i], 2); ptx::mbar_init(&b.empty[i], 1); }
      for (int i = 0; i < 2; ++i) { ptx::mbar_init(&b.acc_full[i], 1); ptx::mbar_init(&b.acc_empty[i], 4); }
      b.timed_out = 0;
      ptx::fence_barrier_init();
    }
    __syncwarp();
  } else if (warp == 1) {
    ptx::tmem_alloc(&b.tmem, (uint32_t)p.tmem_cols);
  }
  // (as in the launch in front, which lets this one in behind its own wait)
  const Plan plan = make_units<DT == SDQ_BF16 ? 2 : 3>(p, s_unit, reinterpret_cast<int32_t*>(sm), &b.plan);
  for (uint32_t i = tid; i < (uint32_t)p.T * 128u; i += MOE_THREADS) out[i] = 0.0f;
  ptx::fence_proxy_async();                        // (the counts lay where the ring is)
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  const uint32_t COLS = (uint32_t)(P * plan.most + 15) / 16 * 16;
  const uint32_t SLOT = SL_B + COLS * 128u + ATOM, NSLOT = min((uint32_t)p.ring_bytes / SLOT, (uint32_t)MOE_MAX_SLOTS), SL_SFB = SL_B + COLS * 128u;
  const uint32_t tmem = b.tmem, sets = tmem + 2 * COLS;
  const int SI = p.off.si, total = plan.units * SI;                       // steps of a unit, of the tile
  const int g0 = (int)((int64_t)rank * total / ks), g1 = (int)((int64_t)(rank + 1) * total / ks);
  bool ok = true;
  if (warp == 0) {
    if (lane == 0) {
      uint32_t i = 0, s = 0, ph = 1;
      for (int g = g0; g < g1 && ok;) {
        const int u = g / SI, end = min(g1, (u + 1) * SI);
        size_t at = ((size_t)s_unit[u].expert * p.tiles_h + tile) * SI + (g - u * SI);
        for (; g < end; ++g, ++i, ++at) {
          if (i >= NSLOT && !(ok = ptx::mbar_wait(&b.empty[s], ph))) break;
          uint8_t* st = sm + (size_t)s * SLOT;
          ptx::mbar_expect_tx(&b.full[s], ECODES + ATOM);
          load_tile(&m2, st, (int)at * 128, &b.full[s]);
          ptx::bulk_g2s(st + SL_SF, p.s2 + at * ATOM, ATOM, &b.full[s]);
          if (++s == NSLOT) { s = 0; ph ^= 1u; }
        }
      }
      if (!ok) atomicOr(&p.flags[FLAG_TIMEOUT], 1u);
    }
    __syncwarp();
  } else if (warp == 3) {
    // the next launch is let in behind the wait: what lies in front of this one is complete for it
    ptx::griddep_wait();
    if (lane == 0) ptx::griddep_launch_dependents();
  } else if (warp == 2) {
    ptx::griddep_wait();                          // h
    if (lane == 0) {
      uint32_t i = 0, s = 0, ph = 1;
      for (int g = g0; g < g1 && ok;) {
        const int u = g / SI, end = min(g1, (u + 1) * SI), k = g - u * SI;
        const MoeUnit un = s_unit[u];
        const uint32_t bytes = (uint32_t)(P * un.n + 7) / 8 * 1024u;
        const uint8_t *h = p.ws + p.off.hp + ((size_t)k * p.off.gh + un.gh) * 1024, *sf = p.ws + p.off.hs + ((size_t)u * SI + k) * ATOM;
        for (; g < end; ++g, ++i, h += (size_t)p.off.gh * 1024, sf += ATOM) {
          if (i >= NSLOT && !(ok = ptx::mbar_wait(&b.empty[s], ph))) break;
          uint8_t* st = sm + (size_t)s * SLOT;
          ptx::mbar_expect_tx(&b.full[s], bytes + ATOM);
          ptx::bulk_g2s(st + SL_B, h, bytes, &b.full[s]);
          ptx::bulk_g2s(st + SL_SFB, sf, ATOM, &b.full[s]);
          if (++s == NSLOT) { s = 0; ph ^= 1u; }
        }
      }
      if (!ok) atomicOr(&p.flags[FLAG_TIMEOUT], 1u);
    }
    __syncwarp();
  } else if (warp == 1) {
    if (lane == 0) {
      uint32_t seg = 0, i = 0, s = 0, ph = 0;
      for (int g = g0; g < g1 && ok; ++seg) {
        const int u = g / SI, end = min(g1, (u + 1) * SI);
        const uint32_t N = (uint32_t)(P * s_unit[u].n + 15) / 16 * 16, acc = tmem + (seg & 1u) * COLS;
        uint32_t id[4];
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) id[j] = ptx::idesc_mxf8_e2m1_e4m3(128, N, j);
        if (seg > 1 && !(ok = ptx::mbar_wait(&b.acc_empty[seg & 1u], ((seg >> 1) - 1) & 1u))) break;
        for (const int first = g; g < end; ++g, ++i) {
          if (!(ok = ptx::mbar_wait(&b.full[s], ph))) break;
          ptx::tc_fence_after();
          const uint32_t st = ptx::smem_u32(sm) + s * SLOT, sf = sets + (i & 1u) * 8u;
          ptx::tc_cp_32x128b_warpx4(sf, ptx::smem_desc(st + SL_SF, 0, 128));
          ptx::tc_cp_32x128b_warpx4(sf + 4, ptx::smem_desc(st + SL_SFB, 0, 128));
          step_mma(acc, st, st + SL_B, sf, sf + 4, id, g > first ? 1u : 0u);
          ptx::tc_commit(&b.empty[s]);
          if (++s == NSLOT) { s = 0; ph ^= 1u; }
        }
        if (ok) ptx::tc_commit(&b.acc_full[seg & 1u]);
      }
      if (!ok) atomicOr(&p.flags[FLAG_TIMEOUT], 1u);
    }
    __syncwarp();
  } else if (warp >= 4 && warp < 8) {
    const uint32_t q = warp & 3, row = q * 32 + lane, et = tid - 128;
    ptx::griddep_wait();
    for (int i = (int)et; i < pairs; i += 128) {
      // (as many of them as there are in units; the others are not looked at)
      const int pr = min(max(reinterpret_cast<const int32_t*>(p.ws + p.off.pairs)[i], 0), pairs - 1);
      s_pair[i] = make_int2(pr / p.k, __float_as_int(p.weights[pr]));
    }
    volatile uint32_t* timed_out = &b.timed_out;
    uint32_t seg = 0;
    for (int g = g0; g < g1; ++seg) {
      const int u = g / SI;
      g = min(g1, (u + 1) * SI);
      const MoeUnit un = s_unit[u];
      if (et == 0 && !(ok = ptx::mbar_wait(&b.acc_full[seg & 1u], (seg >> 1) & 1u))) *timed_out = 1u;
      ptx::named_bar_sync(1, 128);
      if (*timed_out) break;
      ptx::tc_fence_after();
      for (int t0 = 0; t0 < un.n; t0 += CHUNK) {
        float v[CHUNK];
        load_tokens<P>(tmem + ((q * 32u) << 16) + (seg & 1u) * COLS + (uint32_t)(P * t0), v);
#pragma unroll
        for (int j = 0; j < CHUNK; ++j)
          if (t0 + j < un.n) {
            const int2 pr = s_pair[un.pair0 + t0 + j];
            out[pr.x * 128 + row] += __int_as_float(pr.y) * v[j];
          }
      }
      ptx::tc_fence_before();
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(&b.acc_empty[seg & 1u]);
    }
    if (et == 0 && !ok) atomicOr(&p.flags[FLAG_TIMEOUT], 1u);
    __syncwarp();
  }
  ptx::tc_fence_before();
  __syncthreads();
  ptx::cluster_sync();
  ptx::griddep_wait();                             // (all threads: Y may be in use by a kernel in front)
  for (uint32_t i = tid; i < 32u * (uint32_t)p.T; i += MOE_THREADS) {
    if (i % ks != rank) continue;
    const int t = (int)(i >> 5), r0 = (int)(i & 31u) * 4;
    float4 s = make_float4(0, 0, 0, 0);
    for (uint32_t c = 0; c < ks; ++c) {
      const float4 v = load_cta4(out + t * 128 + r0, c);
      s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
    }
    const int64_t n = (int64_t)tile * 128 + r0;
    T* y = reinterpret_cast<T*>(p.y) + (int64_t)t * p.ldy + n;
    const float v[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (n + j < p.H) y[j] = (T)v[j];
  }
  ptx::cluster_sync();
  if (warp == 1) ptx::tmem_dealloc(tmem, (uint32_t)p.tmem_cols);
}

// ---- launches -----------------------------------------------------------------------------------------------------------------
typedef CUresult (*EncodeTiled)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*, const cuuint32_t*,
                                CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
static EncodeTiled encode_tiled() {
  static std::atomic<void*> fn{nullptr};
  void* f = fn;
  if (!f) {
    cudaDriverEntryPointQueryResult r;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12080, cudaEnableDefault, &r) != cudaSuccess || r != cudaDriverEntryPointSuccess) return nullptr;
    fn = f;
  }
  return (EncodeTiled)f;
}
// an expert matrix's codes as core matrices of 128 elements; 128 of them are a tile's step
static bool tile_map(CUtensorMap* map, const sdq_mx4_t* w) {
  EncodeTiled enc = encode_tiled();
  const Dims d = dims(w->E, w->R, w->K, w->fmt);
  const cuuint64_t dim[2] = {128, (cuuint64_t)w->E * d.tiles * d.kblocks * 128}, stride[1] = {64};
  const cuuint32_t box[2] = {128, 128}, es[2] = {1, 1};
  return enc && enc(map, CU_TENSOR_MAP_DATA_TYPE_16U4_ALIGN16B, 2, w->dev, dim, stride, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE,
                    CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
template <typename K>
static bool with_smem(K kern, DeviceInfo* d, int bit) {
  if (d->moe_attr & (1u << bit)) return true;
  const bool ok = cudaFuncSetAttribute((const void*)kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)SMEM_MAX - 1024) == cudaSuccess;
  if (ok) d->moe_attr |= 1u << bit;
  return ok;
}
struct Launch {
  cudaLaunchConfig_t lc;
  cudaLaunchAttribute attr[2];
  Launch(unsigned grid, unsigned threads, unsigned cluster, size_t smem, void* stream) : lc() {
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    lc.gridDim = dim3(grid);
    lc.blockDim = dim3(threads);
    lc.dynamicSmemBytes = smem;
    lc.stream = (cudaStream_t)stream;
    lc.attrs = attr;
    lc.numAttrs = cluster ? 2 : 1;
  }
};

template <int DT>
static sdq_status_t moe(MoeParams p, const sdq_mx4_t* w1, const sdq_mx4_t* w3, const sdq_mx4_t* w2, DeviceInfo* d, void* stream) {
  constexpr int P = DT == SDQ_BF16 ? 2 : 3;
  CUtensorMap m1, m3, m2;
  if (!tile_map(&m1, w1) || !tile_map(&m3, w3) || !tile_map(&m2, w2)) return SDQ_ERR_CUDA;
  auto up = moe_up_kernel<P>;
  auto down = moe_down_kernel<DT>;
  if (!with_smem(up, d, 2 * DT) || !with_smem(down, d, 2 * DT + 1)) return launch_status(cudaErrorUnknown);
  const int pairs = p.T * p.k;
  p.unit = unit_pairs(p.T);
  p.max_units = (pairs < p.E ? pairs : p.E) + pairs / p.unit;
  // Few tokens: both products in half an SM's shared and tensor memory, so that the second's CTAs run beside the first's and have their weights
  // under way when h comes.  More than 76 KB each in any case: never a third such CTA on an SM, which tensor memory would not serve
  const bool half = p.T <= 16;
  p.tmem_cols = half ? 256 : 512;
  const uint32_t room = (half ? SMEM_MAX / 2 - 1024 : SMEM_MAX) - 1024 - 128;
  {
    const size_t smem = (size_t)(pairs + 3) / 4 * 4 * 8 + (size_t)p.E * 20;
    const int work = p.T * 16 * p.off.sh, blocks = (work + SPLIT_THREADS - 1) / SPLIT_THREADS;
    Launch l((unsigned)(blocks < d->sm_count ? blocks : d->sm_count), SPLIT_THREADS, 0, smem, stream);
    const sdq_status_t st = launch_status(cudaLaunchKernelEx(&l.lc, moe_split_kernel<DT>, p));
    if (st != SDQ_OK) return st;
  }
  {
    const int64_t tasks = (int64_t)p.max_units * p.tiles_i;                // (at most)
    int best = 1;
    int64_t cost = 0;
    for (int ks = 1; ks <= 8 && ks <= p.off.sh; ks *= 2) {
      const int64_t cl = d->sm_count / ks, c = ((tasks + cl - 1) / cl) * ((p.off.sh + ks - 1) / ks + (ks > 1 ? 4 : 2));
      if (ks == 1 || c < cost) { best = ks; cost = c; }
    }
    const uint32_t behind = CHUNK * 1024u + (uint32_t)p.max_units * (uint32_t)sizeof(MoeUnit);
    p.ring_bytes = (int32_t)((room - behind) / 128 * 128);
    const int64_t cl = d->sm_count / best < tasks ? d->sm_count / best : tasks;
    Launch l((unsigned)(cl * best), MOE_THREADS, (unsigned)best, (size_t)p.ring_bytes + behind + 128, stream);
    const sdq_status_t st = launch_status(cudaLaunchKernelEx(&l.lc, up, p, m1, m3));
    if (st != SDQ_OK) return st;
  }
  {
    int ks = 1;
    while (ks < 8 && 2 * ks * p.tiles_h <= d->sm_count) ks *= 2;
    const uint32_t behind = (uint32_t)p.T * 512u + (uint32_t)pairs * 8u + (uint32_t)p.max_units * (uint32_t)sizeof(MoeUnit);
    p.ring_bytes = (int32_t)((room - behind) / 128 * 128);
    Launch l((unsigned)(p.tiles_h * ks), MOE_THREADS, (unsigned)ks, (size_t)p.ring_bytes + behind + 128, stream);
    return launch_status(cudaLaunchKernelEx(&l.lc, down, p, m2));
  }
}
static bool moe_sizes_ok(int64_t T, int32_t k, int64_t H, int64_t I) {
  return T >= 1 && T <= MOE_MAX_T && k >= 1 && k <= MOE_MAX_K && H >= 1 && I >= 1 && H <= (1 << 24) && I <= (1 << 24);
}

}  // namespace mx4
}  // namespace sdq

using namespace sdq;

extern "C" sdq_status_t sdq_mx4_moe_workspace_size(int64_t T, int32_t k, int64_t H, int64_t I, size_t* bytes)
{
  if (!bytes) return SDQ_ERR_INVALID_ARG;
  if (!mx4::moe_sizes_ok(T, k, H, I)) return SDQ_ERR_SHAPE;
  *bytes = mx4::moe_offsets(T, k, H, I).total;
  return SDQ_OK;
}

extern "C" sdq_status_t sdq_mx4_moe(const void* X, int32_t dtype, int64_t T, int64_t H, int64_t ldx, const int32_t* ids, const float* weights, int32_t k,
                                    const sdq_mx4_t* w1, const sdq_mx4_t* w3, const sdq_mx4_t* w2, void* Y, int64_t ldy,
                                    void* ws, size_t ws_bytes, void* stream)
{
  using namespace mx4;
  if (!X || !ids || !weights || !Y || !ws || !desc_ok(w1) || !desc_ok(w3) || !desc_ok(w2) || (dtype != SDQ_BF16 && dtype != SDQ_FP16)) return SDQ_ERR_INVALID_ARG;
  if (!w1->E || !w3->E || !w2->E) return SDQ_ERR_UNSUPPORTED;
  const int64_t E = w1->E, I = w1->R;
  if (!moe_sizes_ok(T, k, H, I) || E > MOE_MAX_E || w1->K != H || w3->E != E || w3->R != I || w3->K != H || w2->E != E || w2->R != H || w2->K != I || ldx < H || ldy < H ||
      ldx > ((int64_t)1 << 40) || ldy > ((int64_t)1 << 40)) return SDQ_ERR_SHAPE;
  if ((uintptr_t)X & 1 || (uintptr_t)Y & 1 || (uintptr_t)ids & 3 || (uintptr_t)weights & 3 || (uintptr_t)ws & 255) return SDQ_ERR_ALIGNMENT;
  const Dims d1 = dims(E, I, H, SDQ_FMT_MXFP4), d2 = dims(E, H, I, SDQ_FMT_MXFP4);
  // (core matrices of a matrix are coordinates of a tensor map)
  if (E * d1.tiles * d1.kblocks * 128 > 0x7FFFFFFF || E * d2.tiles * d2.kblocks * 128 > 0x7FFFFFFF) return SDQ_ERR_SHAPE;
  MoeParams p = {};
  p.off = moe_offsets(T, k, H, I);
  if (ws_bytes < p.off.total) return SDQ_ERR_BUFFER_TOO_SMALL;
  DeviceInfo* d = device_info();
  p.flags = device_flags();
  if (!d || !p.flags) return SDQ_ERR_CUDA;
  p.x = X; p.ids = ids; p.weights = weights; p.y = Y; p.ws = (uint8_t*)ws;
  p.s1 = (const uint8_t*)w1->dev + d1.off1; p.s3 = (const uint8_t*)w3->dev + d1.off1; p.s2 = (const uint8_t*)w2->dev + d2.off1;
  p.ldx = ldx; p.ldy = ldy;
  p.T = (int32_t)T; p.k = k; p.E = (int32_t)E; p.H = (int32_t)H; p.I = (int32_t)I; p.tiles_h = (int32_t)d2.tiles; p.tiles_i = (int32_t)d1.tiles;
  return dtype == SDQ_BF16 ? moe<SDQ_BF16>(p, w1, w3, w2, d, stream) : moe<SDQ_FP16>(p, w1, w3, w2, d, stream);
}
