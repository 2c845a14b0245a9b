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
// Three launches: moe_split_kernel sorts the pairs (token, choice) by expert into units of up to 40 pairs and writes X in pieces;
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
constexpr int UNIT_PAIRS = 40;                  // pairs of a unit: three pieces of each are 120 columns
constexpr int H_PIECES = 3;                     // of silu(.) * (.)

// ---- workspace --------------------------------------------------------------------------------------------------------------
struct MoeUnit { int32_t expert, n, pair0, gx, gh; };        // pairs pair0 .. + n of the sorted list; first 8-row group of its pieces of X and h
struct MoeOffsets {
  size_t units, pairs, xp, xs, hp, hs, total;
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
  o.units = 256;                                             // (in front: number of units, pairs of the largest)
  o.pairs = al(o.units + (size_t)P * sizeof(MoeUnit));
  o.xp = al(o.pairs + (size_t)P * 4);
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
  int32_t ring_bytes;
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

// ---- pairs by expert, X in pieces -----------------------------------------------------------------------------------------------
constexpr int SPLIT_THREADS = 256;
template <int DT>
__global__ void __launch_bounds__(SPLIT_THREADS)
moe_split_kernel(const __grid_constant__ MoeParams p)
{
  constexpr int P = DT == SDQ_BF16 ? 2 : 3;
  extern __shared__ int32_t s_split[];
  const int pairs = p.T * p.k;
  int32_t* s_id = s_split;                       // expert of a pair (-1: none)
  int32_t* s_rank = s_id + pairs;                // its place among the expert's pairs
  int32_t* s_n = s_rank + pairs;                 // pairs of an expert
  int4* s_at = reinterpret_cast<int4*>((reinterpret_cast<uintptr_t>(s_n + p.E) + 15) & ~(uintptr_t)15);   // first unit, pair, group of X, group of h
  const int tid = (int)threadIdx.x, lane = tid & 31;
  if (tid == 0) ptx::griddep_launch_dependents();
  ptx::griddep_wait();
  for (int i = tid; i < pairs; i += SPLIT_THREADS) {
    const int e = p.ids[i];
    s_id[i] = e >= 0 && e < p.E ? e : -1;
  }
  __syncthreads();
  for (int e = tid; e < p.E; e += SPLIT_THREADS) {
    int n = 0;
    for (int i = 0; i < pairs; ++i)
      if (s_id[i] == e) s_rank[i] = n++;
    s_n[e] = n;
  }
  __syncthreads();
  if (tid < 32) {
    int4 base = make_int4(0, 0, 0, 0);
    int most = 0;
    for (int e0 = 0; e0 < p.E; e0 += 32) {
      const int e = e0 + lane, n = e < p.E ? s_n[e] : 0, full = n / UNIT_PAIRS, rest = n - full * UNIT_PAIRS;
      const int4 own = make_int4(full + (rest ? 1 : 0), n, full * (P * UNIT_PAIRS / 8) + (P * rest + 7) / 8, full * (H_PIECES * UNIT_PAIRS / 8) + (H_PIECES * rest + 7) / 8);
      int4 v = own;
      most = max(most, n);
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int4 u = make_int4(__shfl_up_sync(0xffffffffu, v.x, o), __shfl_up_sync(0xffffffffu, v.y, o), __shfl_up_sync(0xffffffffu, v.z, o), __shfl_up_sync(0xffffffffu, v.w, o));
        if (lane >= o) { v.x += u.x; v.y += u.y; v.z += u.z; v.w += u.w; }
      }
      if (e < p.E) s_at[e] = make_int4(base.x + v.x - own.x, base.y + v.y - own.y, base.z + v.z - own.z, base.w + v.w - own.w);
      base.x += __shfl_sync(0xffffffffu, v.x, 31); base.y += __shfl_sync(0xffffffffu, v.y, 31);
      base.z += __shfl_sync(0xffffffffu, v.z, 31); base.w += __shfl_sync(0xffffffffu, v.w, 31);
    }
    most = min(__reduce_max_sync(0xffffffffu, most), UNIT_PAIRS);
    if (blockIdx.x == 0 && lane == 0) *reinterpret_cast<int2*>(p.ws) = make_int2(base.x, most);
  }
  __syncthreads();
  if (blockIdx.x == 0) {
    MoeUnit* units = reinterpret_cast<MoeUnit*>(p.ws + p.off.units);
    for (int e = tid; e < p.E; e += SPLIT_THREADS) {
      const int4 at = s_at[e];
      for (int u = 0, n = s_n[e]; n > 0; ++u, n -= UNIT_PAIRS)
        units[at.x + u] = MoeUnit{e, min(n, UNIT_PAIRS), at.y + u * UNIT_PAIRS, at.z + u * (P * UNIT_PAIRS / 8), at.w + u * (H_PIECES * UNIT_PAIRS / 8)};
    }
    for (int i = tid; i < pairs; i += SPLIT_THREADS)
      if (s_id[i] >= 0) reinterpret_cast<int32_t*>(p.ws + p.off.pairs)[s_at[s_id[i]].y + s_rank[i]] = i;
  }
  // 32 elements of a token a thread
  using T = typename std::conditional<DT == SDQ_BF16, __nv_bfloat16, __half>::type;
  const int blocks = 4 * p.off.sh;               // blocks of 32 of a row, padded to whole steps
  for (int w = (int)blockIdx.x * SPLIT_THREADS + tid; w < p.T * blocks; w += (int)gridDim.x * SPLIT_THREADS) {
    const int t = w / blocks, b = w - t * blocks, h0 = 32 * b;
    const T* row = reinterpret_cast<const T*>(p.x) + (int64_t)t * p.ldx;
    float v[32];
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 32; ++i) {
      v[i] = 0.0f;
      if (h0 + i < p.H) v[i] = (float)row[h0 + i];
      m = max(m, __float_as_uint(v[i]) & 0x7FFFFFFFu);
    }
    const uint32_t c = piece_scale(m);
    const float inv = __uint_as_float((254u - c) << 23);
    uint32_t code[P][8];
#pragma unroll
    for (int i = 0; i < 32; ++i) {
      uint32_t q[P];
      pieces<P>(v[i], inv, q);
#pragma unroll
      for (int j = 0; j < P; ++j) code[j][i / 4] = (i % 4 ? code[j][i / 4] : 0u) | q[j] << (8 * (i % 4));
    }
    const int step = b >> 2;
    for (int j = 0; j < p.k; ++j) {
      const int i = t * p.k + j, e = s_id[i];
      if (e < 0) continue;
      const int u = s_rank[i] / UNIT_PAIRS, r = s_rank[i] - u * UNIT_PAIRS;
      uint8_t* dst = p.ws + p.off.xp + ((size_t)step * p.off.gx + s_at[e].z + u * (P * UNIT_PAIRS / 8)) * 1024;
      uint8_t* sc = p.ws + p.off.xs + ((size_t)(s_at[e].x + u) * p.off.sh + step) * ATOM;
#pragma unroll
      for (int q = 0; q < P; ++q) {
        const uint32_t at = piece_off((uint32_t)(P * r + q), (uint32_t)(h0 & 127));
        *reinterpret_cast<uint4*>(dst + at) = make_uint4(code[q][0], code[q][1], code[q][2], code[q][3]);
        *reinterpret_cast<uint4*>(dst + at + 128) = make_uint4(code[q][4], code[q][5], code[q][6], code[q][7]);
        sc[atom_off((uint32_t)(P * r + q), (uint32_t)(b & 3))] = (uint8_t)(c - 4 * q);
      }
    }
  }
}

// ---- what the two products share ------------------------------------------------------------------------------------------------
constexpr int MOE_THREADS = 192;                  // producer, MMA issuer, four epilogue warps
constexpr int MOE_MAX_SLOTS = 8;
constexpr uint32_t A_BYTES = 16384;               // an expert's tile and step in shared memory
constexpr uint32_t SMEM_MAX = 232448;

// Ring of a product: as many slots as fit, a slot having room for the columns of the largest unit there is (known on the device only).
struct MoeRing { uint32_t cols, slot, slots; };
__device__ __forceinline__ MoeRing moe_ring(const MoeParams& p, int pieces, int steps) {
  MoeRing r;
  const uint32_t n = (uint32_t)reinterpret_cast<const volatile int32_t*>(p.ws)[1];
  r.cols = ((uint32_t)pieces * n + 15u) / 16u * 16u;
  r.slot = 2u * (A_BYTES + ATOM) + (uint32_t)steps * (r.cols * 128u + ATOM);
  r.slots = min((uint32_t)p.ring_bytes / r.slot, (uint32_t)MOE_MAX_SLOTS);
  return r;
}

struct MoeBars {
  uint64_t full[MOE_MAX_SLOTS], empty[MOE_MAX_SLOTS], acc_full, acc_empty, part_full, part_empty;
  uint32_t tmem, timed_out;
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
__device__ __forceinline__ float load_cta(uint32_t saddr, uint32_t cta) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(ptx::mapa_u32(saddr, cta)) : "memory");
  return v;
}
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
  uint32_t ks;
  asm volatile("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(ks));
  const uint32_t rank = ptx::cluster_ctarank();
  const int cluster = (int)(blockIdx.x / ks), clusters = (int)(gridDim.x / ks);
  const int k0 = (int)(rank * (uint32_t)p.off.sh / ks), steps = (int)((rank + 1) * (uint32_t)p.off.sh / ks) - k0;
  if (warp == 0) {
    if (lane == 0) {
      ptx::griddep_launch_dependents();
      for (int i = 0; i < MOE_MAX_SLOTS; ++i) { ptx::mbar_init(&b.full[i], 1); ptx::mbar_init(&b.empty[i], 1); }
      ptx::mbar_init(&b.acc_full, 1);
      ptx::mbar_init(&b.acc_empty, 4);
      ptx::mbar_init(&b.part_full, ks);
      ptx::mbar_init(&b.part_empty, ks);
      b.timed_out = 0;
      ptx::fence_barrier_init();
    }
    __syncwarp();
  } else if (warp == 1) {
    ptx::tmem_alloc(&b.tmem, 512);
  }
  ptx::tc_fence_before();
  __syncthreads();
  ptx::cluster_sync();
  ptx::tc_fence_after();
  const uint32_t tmem = b.tmem, sets = tmem + 256u;
  ptx::griddep_wait();
  const int tasks = *reinterpret_cast<const volatile int32_t*>(p.ws) * p.tiles_i;
  const MoeRing ring = moe_ring(p, P, 1);
  const uint32_t SLOT = ring.slot, NSLOT = ring.slots, SL_SFB = SL_B + ring.cols * 128u;
  const MoeUnit* units = reinterpret_cast<const MoeUnit*>(p.ws + p.off.units);
  bool ok = true;
  if (warp == 0) {
    if (lane == 0) {
      uint32_t i = 0;
      for (int task = cluster; task < tasks && ok; task += clusters) {
        const int u = task / p.tiles_i, tile = task - u * p.tiles_i;
        const MoeUnit un = units[u];
        const size_t at = ((size_t)un.expert * p.tiles_i + tile) * p.off.sh + k0;
        const uint32_t bbytes = (uint32_t)(P * un.n + 7) / 8 * 1024u;
        for (int k = 0; k < steps; ++k, ++i) {
          const uint32_t s = i % NSLOT;
          if (i >= NSLOT && !(ok = ptx::mbar_wait(&b.empty[s], ((i / NSLOT) & 1u) ^ 1u))) break;
          uint8_t* st = sm + (size_t)s * SLOT;
          // (the tensor copies count the bytes they read: the padding is not written)
          ptx::mbar_expect_tx(&b.full[s], 2 * ECODES + 3 * ATOM + bbytes);
          load_tile(&m1, st, (int)(at + k) * 128, &b.full[s]);
          load_tile(&m3, st + A_BYTES, (int)(at + k) * 128, &b.full[s]);
          ptx::bulk_g2s(st + SL_SF, p.s1 + (at + k) * ATOM, ATOM, &b.full[s]);
          ptx::bulk_g2s(st + SL_SF + ATOM, p.s3 + (at + k) * ATOM, ATOM, &b.full[s]);
          ptx::bulk_g2s(st + SL_B, p.ws + p.off.xp + ((size_t)(k0 + k) * p.off.gx + un.gx) * 1024, bbytes, &b.full[s]);
          ptx::bulk_g2s(st + SL_SFB, p.ws + p.off.xs + ((size_t)u * p.off.sh + k0 + k) * ATOM, ATOM, &b.full[s]);
        }
      }
      if (!ok) atomicOr(&p.flags[FLAG_TIMEOUT], 1u);
    }
    __syncwarp();
  } else if (warp == 1) {
    if (lane == 0) {
      uint32_t i = 0, t = 0;
      for (int task = cluster; task < tasks && ok; task += clusters, ++t) {
        const uint32_t N = (uint32_t)(P * units[task / p.tiles_i].n + 15) / 16 * 16;
        uint32_t id[4];
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) id[j] = ptx::idesc_mxf8_e2m1_e4m3(128, N, j);
        if (t > 0 && !(ok = ptx::mbar_wait(&b.acc_empty, (t - 1) & 1u))) break;
        for (int k = 0; k < steps; ++k, ++i) {
          const uint32_t s = i % NSLOT;
          if (!(ok = ptx::mbar_wait(&b.full[s], (i / NSLOT) & 1u))) break;
          ptx::tc_fence_after();
          const uint32_t st = ptx::smem_u32(sm) + s * SLOT, sf = sets + (i & 1u) * 12u;
          ptx::tc_cp_32x128b_warpx4(sf, ptx::smem_desc(st + SL_SF, 0, 128));
          ptx::tc_cp_32x128b_warpx4(sf + 4, ptx::smem_desc(st + SL_SF + ATOM, 0, 128));
          ptx::tc_cp_32x128b_warpx4(sf + 8, ptx::smem_desc(st + SL_SFB, 0, 128));
          step_mma(tmem, st, st + SL_B, sf, sf + 8, id, k ? 1u : 0u);
          step_mma(tmem + 128u, st + A_BYTES, st + SL_B, sf + 4, sf + 8, id, k ? 1u : 0u);
          ptx::tc_commit(&b.empty[s]);
        }
        if (ok) ptx::tc_commit(&b.acc_full);
      }
      if (!ok) atomicOr(&p.flags[FLAG_TIMEOUT], 1u);
    }
    __syncwarp();
  } else {
    const uint32_t q = warp & 3, row = q * 32 + lane, et = tid - 64;
    float* part = reinterpret_cast<float*>(sm + p.ring_bytes);     // K split: [token][W1 or W3][128 rows]
    uint32_t t = 0;
    for (int task = cluster; task < tasks; task += clusters, ++t) {
      const int u = task / p.tiles_i, tile = task - u * p.tiles_i;
      const MoeUnit un = units[u];
      if (et == 0) {
        ok = ptx::mbar_wait(&b.acc_full, t & 1u);
        if (ok && ks > 1 && t > 0) ok = ptx::mbar_wait_cluster(&b.part_empty, (t - 1) & 1u);
        if (!ok) *const_cast<volatile uint32_t*>(&b.timed_out) = 1u;
      }
      ptx::named_bar_sync(1, 128);
      if (*const_cast<volatile uint32_t*>(&b.timed_out)) break;
      ptx::tc_fence_after();
      uint8_t* hp = p.ws + p.off.hp + ((size_t)tile * p.off.gh + un.gh) * 1024;
      uint8_t* hs = p.ws + p.off.hs + ((size_t)u * p.off.si + tile) * ATOM;
      // one token's value of this row: rounded into pieces with the warp's 32 rows as their block
      auto finish = [&](int tok, float g, float v) {
        const float h = g / (1.0f + expf(-g)) * v;
        const uint32_t c = piece_scale(__reduce_max_sync(0xffffffffu, __float_as_uint(h) & 0x7FFFFFFFu));
        uint32_t code[H_PIECES];
        pieces<H_PIECES>(h, __uint_as_float((254u - c) << 23), code);
#pragma unroll
        for (int j = 0; j < H_PIECES; ++j) {
          const uint32_t r = (uint32_t)(H_PIECES * tok + j);
          hp[piece_off(r, row)] = (uint8_t)code[j];
          if (lane == 0) hs[atom_off(r, q)] = (uint8_t)(c - 4 * j);
        }
      };
      const uint32_t ta = tmem + ((q * 32u) << 16);
      for (int t0 = 0; t0 < un.n; t0 += 16) {
        float g[16], v[16];
        load_tokens<P>(ta + (uint32_t)(P * t0), g);
        load_tokens<P>(ta + 128u + (uint32_t)(P * t0), v);
#pragma unroll
        for (int j = 0; j < 16; ++j)
          if (t0 + j < un.n) {
            if (ks > 1) {
              part[(size_t)(t0 + j) * 256 + row] = g[j];
              part[(size_t)(t0 + j) * 256 + 128 + row] = v[j];
            } else {
              finish(t0 + j, g[j], v[j]);
            }
          }
      }
      ptx::tc_fence_before();
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(&b.acc_empty);
      if (ks > 1) {
        ptx::named_bar_sync(1, 128);
        if (et < ks) arrive_cta(&b.part_full, et);
        if (et == 0 && !(ok = ptx::mbar_wait_cluster(&b.part_full, t & 1u))) *const_cast<volatile uint32_t*>(&b.timed_out) = 1u;
        ptx::named_bar_sync(1, 128);
        if (*const_cast<volatile uint32_t*>(&b.timed_out)) break;
        // (the acquire of one thread and the barrier behind it order the peers' stores before everybody's loads)
        for (int tok = (int)rank; tok < un.n; tok += (int)ks) {
          float g = 0.0f, v = 0.0f;
          const uint32_t at = ptx::smem_u32(part + (size_t)tok * 256 + row);
          for (uint32_t c = 0; c < ks; ++c) { g += load_cta(at, c); v += load_cta(at + 512u, c); }
          finish(tok, g, v);
        }
        ptx::named_bar_sync(1, 128);
        if (et < ks) arrive_cta(&b.part_empty, et);
      }
    }
    if (et == 0 && !ok) atomicOr(&p.flags[FLAG_TIMEOUT], 1u);
    __syncwarp();
  }
  ptx::tc_fence_before();
  __syncthreads();
  ptx::cluster_sync();                             // nobody leaves while its partial sums are being read
  if (warp == 1) ptx::tmem_dealloc(tmem, 512);
}

// ---- W2 h, and the sum over a token's pairs -------------------------------------------------------------------------------------
// A cluster has one tile of 128 outputs; its CTAs share the steps of all units.  slot = two steps: | tiles of W2 | their scale atoms |
// columns of h | their scale atoms |
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
  constexpr uint32_t SL_SF = 2 * A_BYTES, SL_B = SL_SF + 2 * ATOM;
  uint32_t ks;
  asm volatile("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(ks));
  const uint32_t rank = ptx::cluster_ctarank();
  const int tile = (int)(blockIdx.x / ks);
  float* out = reinterpret_cast<float*>(sm + p.ring_bytes);       // [token][128 rows]
  for (uint32_t i = tid; i < (uint32_t)p.T * 128u; i += MOE_THREADS) out[i] = 0.0f;
  if (warp == 0) {
    if (lane == 0) {
      ptx::griddep_launch_dependents();
      for (int i = 0; i < MOE_MAX_SLOTS; ++i) { ptx::mbar_init(&b.full[i], 1); ptx::mbar_init(&b.empty[i], 1); }
      ptx::mbar_init(&b.acc_full, 1);
      ptx::mbar_init(&b.acc_empty, 4);
      b.timed_out = 0;
      ptx::fence_barrier_init();
    }
    __syncwarp();
  } else if (warp == 1) {
    ptx::tmem_alloc(&b.tmem, 512);
  }
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  const uint32_t tmem = b.tmem, sets = tmem + 256u;
  ptx::griddep_wait();
  const MoeRing ring = moe_ring(p, P, 2);
  const uint32_t SLOT = ring.slot, NSLOT = ring.slots, B_BYTES = ring.cols * 128u, SL_SFB = SL_B + 2 * B_BYTES;
  const int SI = p.off.si, per = (SI + 1) / 2, total = *reinterpret_cast<const volatile int32_t*>(p.ws) * per;   // stages of a unit, of the tile
  const int g0 = (int)((int64_t)rank * total / ks), g1 = (int)((int64_t)(rank + 1) * total / ks);
  const MoeUnit* units = reinterpret_cast<const MoeUnit*>(p.ws + p.off.units);
  bool ok = true;
  if (warp == 0) {
    if (lane == 0) {
      for (int g = g0; g < g1; ++g) {
        const uint32_t i = (uint32_t)(g - g0), s = i % NSLOT;
        const int u = g / per, k = 2 * (g - u * per), two = k + 1 < SI ? 2 : 1;
        const MoeUnit un = units[u];
        const size_t at = ((size_t)un.expert * p.tiles_h + tile) * SI + k;
        const uint32_t bbytes = (uint32_t)(P * un.n + 7) / 8 * 1024u;
        if (i >= NSLOT && !(ok = ptx::mbar_wait(&b.empty[s], ((i / NSLOT) & 1u) ^ 1u))) break;
        uint8_t* st = sm + (size_t)s * SLOT;
        ptx::mbar_expect_tx(&b.full[s], (uint32_t)two * (ECODES + 2 * ATOM + bbytes));
        ptx::bulk_g2s(st + SL_SF, p.s2 + at * ATOM, (uint32_t)two * ATOM, &b.full[s]);
        ptx::bulk_g2s(st + SL_SFB, p.ws + p.off.hs + ((size_t)u * SI + k) * ATOM, (uint32_t)two * ATOM, &b.full[s]);
        for (int j = 0; j < two; ++j) {
          load_tile(&m2, st + j * A_BYTES, (int)(at + j) * 128, &b.full[s]);
          ptx::bulk_g2s(st + SL_B + j * B_BYTES, p.ws + p.off.hp + ((size_t)(k + j) * p.off.gh + un.gh) * 1024, bbytes, &b.full[s]);
        }
      }
      if (!ok) atomicOr(&p.flags[FLAG_TIMEOUT], 1u);
    }
    __syncwarp();
  } else if (warp == 1) {
    if (lane == 0) {
      uint32_t seg = 0;
      for (int g = g0; g < g1 && ok;) {
        const int u = g / per, end = min(g1, (u + 1) * per);
        const uint32_t N = (uint32_t)(P * units[u].n + 15) / 16 * 16;
        uint32_t id[4];
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) id[j] = ptx::idesc_mxf8_e2m1_e4m3(128, N, j);
        if (seg > 0 && !(ok = ptx::mbar_wait(&b.acc_empty, (seg - 1) & 1u))) break;
        for (const int first = g; g < end; ++g) {
          const uint32_t i = (uint32_t)(g - g0), s = i % NSLOT;
          const int k = 2 * (g - u * per);
          if (!(ok = ptx::mbar_wait(&b.full[s], (i / NSLOT) & 1u))) break;
          ptx::tc_fence_after();
          const uint32_t st = ptx::smem_u32(sm) + s * SLOT, sf = sets + (i & 1u) * 16u;
          for (uint32_t j = 0; j < (k + 1 < SI ? 2u : 1u); ++j) {
            ptx::tc_cp_32x128b_warpx4(sf + 8 * j, ptx::smem_desc(st + SL_SF + j * ATOM, 0, 128));
            ptx::tc_cp_32x128b_warpx4(sf + 8 * j + 4, ptx::smem_desc(st + SL_SFB + j * ATOM, 0, 128));
            step_mma(tmem, st + j * A_BYTES, st + SL_B + j * B_BYTES, sf + 8 * j, sf + 8 * j + 4, id, g > first || j ? 1u : 0u);
          }
          ptx::tc_commit(&b.empty[s]);
        }
        if (ok) { ptx::tc_commit(&b.acc_full); ++seg; }
      }
      if (!ok) atomicOr(&p.flags[FLAG_TIMEOUT], 1u);
    }
    __syncwarp();
  } else {
    const uint32_t q = warp & 3, row = q * 32 + lane, et = tid - 64;
    const int32_t* pairs = reinterpret_cast<const int32_t*>(p.ws + p.off.pairs);
    uint32_t seg = 0;
    for (int g = g0; g < g1; ++seg) {
      const int u = g / per;
      g = min(g1, (u + 1) * per);
      const MoeUnit un = units[u];
      if (et == 0 && !(ok = ptx::mbar_wait(&b.acc_full, seg & 1u))) *const_cast<volatile uint32_t*>(&b.timed_out) = 1u;
      ptx::named_bar_sync(1, 128);
      if (*const_cast<volatile uint32_t*>(&b.timed_out)) break;
      ptx::tc_fence_after();
      for (int t0 = 0; t0 < un.n; t0 += 16) {
        float v[16];
        load_tokens<P>(tmem + ((q * 32u) << 16) + (uint32_t)(P * t0), v);
#pragma unroll
        for (int j = 0; j < 16; ++j)
          if (t0 + j < un.n) {
            const int pair = pairs[un.pair0 + t0 + j];
            out[(size_t)(pair / p.k) * 128 + row] += p.weights[pair] * v[j];
          }
      }
      ptx::tc_fence_before();
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(&b.acc_empty);
    }
    if (et == 0 && !ok) atomicOr(&p.flags[FLAG_TIMEOUT], 1u);
    __syncwarp();
  }
  ptx::tc_fence_before();
  __syncthreads();
  ptx::cluster_sync();
  for (uint32_t i = tid; i < 128u * (uint32_t)p.T; i += MOE_THREADS) {
    const int t = (int)(i >> 7), row = (int)(i & 127u);
    if ((uint32_t)t % ks != rank) continue;
    float s = 0.0f;
    for (uint32_t c = 0; c < ks; ++c) s += load_cta(ptx::smem_u32(out + i), c);
    const int64_t n = (int64_t)tile * 128 + row;
    if (n < p.H) reinterpret_cast<T*>(p.y)[(int64_t)t * p.ldy + n] = (T)s;
  }
  ptx::cluster_sync();
  if (warp == 1) ptx::tmem_dealloc(tmem, 512);
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
  const int n = p.T * p.k < UNIT_PAIRS ? p.T * p.k : UNIT_PAIRS;       // most pairs a unit may have (a token may name an expert twice)
  {
    const size_t smem = (size_t)pairs * 8 + (size_t)p.E * 20 + 16;
    const int work = p.T * 4 * p.off.sh, blocks = (work + SPLIT_THREADS - 1) / SPLIT_THREADS;
    Launch l((unsigned)(blocks < d->sm_count ? blocks : d->sm_count), SPLIT_THREADS, 0, smem, stream);
    const sdq_status_t st = launch_status(cudaLaunchKernelEx(&l.lc, moe_split_kernel<DT>, p));
    if (st != SDQ_OK) return st;
  }
  {
    const int64_t units = (int64_t)(pairs < p.E ? pairs : p.E) + pairs / UNIT_PAIRS, tasks = units * p.tiles_i;   // (at most)
    int best = 1;
    int64_t cost = 0;
    for (int ks = 1; ks <= 8 && ks <= p.off.sh; ks *= 2) {
      const int64_t cl = d->sm_count / ks, c = ((tasks + cl - 1) / cl) * ((p.off.sh + ks - 1) / ks + (ks > 1 ? 4 : 2));
      if (ks == 1 || c < cost) { best = ks; cost = c; }
    }
    const uint32_t parts = best > 1 ? (uint32_t)n * 1024u : 0u;
    p.ring_bytes = (int32_t)((SMEM_MAX - 1024 - 128 - parts) / 128 * 128);
    const int64_t cl = d->sm_count / best < tasks ? d->sm_count / best : tasks;
    Launch l((unsigned)(cl * best), MOE_THREADS, (unsigned)best, (size_t)p.ring_bytes + parts + 128, stream);
    const sdq_status_t st = launch_status(cudaLaunchKernelEx(&l.lc, up, p, m1, m3));
    if (st != SDQ_OK) return st;
  }
  {
    int ks = 1;
    while (ks < 8 && 2 * ks * p.tiles_h <= d->sm_count) ks *= 2;
    const uint32_t outs = (uint32_t)p.T * 512u;
    p.ring_bytes = (int32_t)((SMEM_MAX - 1024 - 128 - outs) / 128 * 128);
    Launch l((unsigned)(p.tiles_h * ks), MOE_THREADS, (unsigned)ks, (size_t)p.ring_bytes + outs + 128, stream);
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
