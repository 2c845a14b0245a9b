// Expert layer of a few tokens over MXFP4 experts:  Y[t] = sum_j weights[t][j] * W2[e](silu(W1[e] x_t) * W3[e] x_t),  e = ids[t][j].
//
// The chosen experts' weights are what has to be read, each once however many tokens chose it.  They are multiplied as they are, in four
// bits, by activations that are not quantized: kind::mxf4 takes E2M1 on both sides, and an activation is a sum of six E2M1 pieces,
//   x = 2^s (p0 + p1 / 8 + .. + p5 / 8^5),   p0 = e2m1(r), r = x / 2^s;   p1 = e2m1(8 (r - p0));   ..
// 2^s such that the block's largest magnitude lies in [2, 4) 2^s.  E2M1 is within 1/2 of every number up to 4, so a remainder, times 8, is again at
// most 4, and every one of them is exact in fp32; what is left behind six pieces is at most 2^-16 2^s.  Pieces are columns of the MMA of their
// own, each with its scale (2^s, 2^(s-3), ..), added up in the epilogue: few tokens leave columns to spare -- an MMA takes 46 clocks for up to
// 64 columns, 64 for 128 -- and the weights are fetched into the tensor core once for all of them.  (Two or three E4M3 pieces under the 8-bit kind
// are as exact, but that kind wants 4-bit operands padded to bytes, twice the shared memory for what is in flight, and twice the
// MMAs: 64 tokens x 8 experts of 4096 x 11008 took 187 us.)
//
// Three launches: the pairs (token, choice) are sorted by expert into units of up to 20 pairs; moe_split_kernel writes X in pieces;
// moe_up_kernel forms silu(W1 x) * (W3 x), 128 rows of both a task, and writes it in pieces; moe_down_kernel forms W2 h, adds up every
// token's pairs in a fixed order and rounds once.  Where tasks are too few for the GPU, the CTAs of a cluster split K and add their fp32
// partial sums through distributed shared memory, in a fixed order.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp4.h>

#include <type_traits>

#include "../sdq_codec.cuh"
#include "../sdq_internal.h"
#include "../sdq_ptx.cuh"
#include "layout.h"
#include "pipe.cuh"

namespace sdq {
namespace mx4 {

constexpr int MOE_MAX_T = 64, MOE_MAX_K = 32, MOE_MAX_E = 1024;
constexpr int PIECES = 6;
// Pairs of a unit, at most: six pieces of 20 are 120 columns, which one scale atom serves.  Smaller units where there are fewer tokens bound
// what a CTA has to have room for; a token may name an expert more than once, so that the number of tokens alone bounds nothing.
// (A unit's pieces are whole groups of eight rows: a multiple of four pairs.)  Sixteen where an expert has eight pairs or fewer in the mean, and so
// seldom more than sixteen
constexpr int unit_pairs(int64_t T, int64_t pairs, int64_t E) { return T <= 8 ? 8 : T <= 16 || pairs <= 8 * E ? 16 : 20; }

// ---- workspace --------------------------------------------------------------------------------------------------------------
struct MoeUnit { int32_t expert, n, pair0, group; };        // pairs pair0 .. + n of the sorted list; first 8-row group of its pieces
struct MoeOffsets {
  size_t pairs, xp, xs, hp, hs, total;
  int32_t groups, sh, si;                                    // 8-row groups of a step (bound), steps of H and I
};
constexpr uint32_t GROUP = 512;                 // bytes of eight rows and a step
inline MoeOffsets moe_offsets(int64_t T, int k, int64_t H, int64_t I) {
  MoeOffsets o;
  auto al = [](size_t x) { return (x + 255) & ~(size_t)255; };
  const int64_t P = T * k;                                    // units have at least one pair, and up to 7 rows of padding
  o.sh = (int32_t)((H + KSTEP - 1) / KSTEP);
  o.si = (int32_t)((I + KSTEP - 1) / KSTEP);
  o.groups = (int32_t)((P * PIECES + 7 * P) / 8 + 1);
  o.pairs = 0;
  o.xp = al((size_t)P * 4);
  o.xs = al(o.xp + (size_t)o.sh * o.groups * GROUP);
  o.hp = al(o.xs + (size_t)P * o.sh * ATOM);
  o.hs = al(o.hp + (size_t)o.si * o.groups * GROUP);
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
  const uint8_t *w1, *w3, *w2;                                // records
  int64_t ldx, ldy;
  int32_t T, k, E, H, I, tiles_h, tiles_i;                    // row tiles of 128 of an expert's matrices
  int32_t unit, max_units;                                    // unit_pairs; units there can be
  int32_t ring_bytes, tmem_cols;
  uint32_t* flags;
};

// row r (of a unit's columns), byte k (0 .. 63) of a step: inside the unit's groups
__device__ __forceinline__ uint32_t piece_off(uint32_t r, uint32_t k) { return (r >> 3) * GROUP + (k >> 4) * 128 + (r & 7) * 16 + (k & 15); }

// ---- pieces -------------------------------------------------------------------------------------------------------------------
// code c of the block's scale 2^(c - 127), its largest magnitude lying in [2, 4) times it; at least 15, so that the later pieces' scales
// (c - 3, .., c - 15) are codes too (blocks whose largest magnitude is below 2^-111 keep what lies above 2^-128)
__device__ __forceinline__ uint32_t piece_scale(uint32_t amax_bits) { return (uint32_t)min(max((int)(amax_bits >> 23) - 1, 15), 253); }
__device__ __forceinline__ float piece_inverse(uint32_t c) { return __uint_as_float((254u - c) << 23); }
// scale code of piece i; a block that holds something not finite: NaN
__device__ __forceinline__ uint32_t piece_code(uint32_t amax_bits, uint32_t c, uint32_t i) { return amax_bits >= 0x7F800000u ? 255u : c - 3u * i; }
// next piece of two remainders: the codes (one byte), and what they leave, times 8
__device__ __forceinline__ uint32_t next_piece(float& a, float& b) {
  const uint32_t c = e2m1x2(a, b);
  const __half2_raw h = __nv_cvt_fp4x2_to_halfraw2((__nv_fp4x2_storage_t)c, __NV_E2M1);
  const float2 f = __half22float2(__half2(h));
  a = (a - f.x) * 8.0f;
  b = (b - f.y) * 8.0f;
  return c;
}

// ---- pairs by expert --------------------------------------------------------------------------------------------------------------
// Every CTA of the three kernels makes the list of units for itself, from the ids: that is quicker than to wait for another CTA's.
// `s_n`: [E] pairs of an expert; the warp calls each(expert, its pairs, its first unit, pair and group)
struct Plan { int units, most; };                // units, pairs of the largest
template <typename F>
__device__ __forceinline__ Plan plan_units(const int32_t* s_n, int E, int unit, uint32_t lane, F each) {
  int3 base = make_int3(0, 0, 0);
  int most = 0;
  for (int e0 = 0; e0 < E; e0 += 32) {
    const int e = e0 + (int)lane, n = e < E ? s_n[e] : 0, full = n / unit, rest = n - full * unit;
    const int3 own = make_int3(full + (rest ? 1 : 0), n, full * (PIECES * unit / 8) + (PIECES * rest + 7) / 8);
    int3 v = own;
    most = max(most, n);
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int3 u = make_int3(__shfl_up_sync(0xffffffffu, v.x, o), __shfl_up_sync(0xffffffffu, v.y, o), __shfl_up_sync(0xffffffffu, v.z, o));
      if ((int)lane >= o) { v.x += u.x; v.y += u.y; v.z += u.z; }
    }
    if (e < E) each(e, n, make_int3(base.x + v.x - own.x, base.y + v.y - own.y, base.z + v.z - own.z));
    base.x += __shfl_sync(0xffffffffu, v.x, 31); base.y += __shfl_sync(0xffffffffu, v.y, 31); base.z += __shfl_sync(0xffffffffu, v.z, 31);
  }
  return Plan{base.x, min(__reduce_max_sync(0xffffffffu, most), unit)};
}
// the units themselves, in shared memory (all threads of the CTA; s_n is scratch of E words)
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
    const Plan r = plan_units(s_n, p.E, unit, lane, [&](int e, int n, int3 at) {
      for (int u = 0; n > 0; ++u, n -= unit) s_unit[at.x + u] = MoeUnit{e, min(n, unit), at.y + u * unit, at.z + u * (PIECES * unit / 8)};
    });
    if (lane == 0) *s_plan = r;
  }
  __syncthreads();
  return *s_plan;
}

// ---- X in pieces ------------------------------------------------------------------------------------------------------------------
// (SPLIT_THREADS: few tokens are spread over more SMs)
template <int DT, int SPLIT_THREADS>
__global__ void __launch_bounds__(SPLIT_THREADS)
moe_split_kernel(const __grid_constant__ MoeParams p)
{
  using T = typename std::conditional<DT == SDQ_BF16, __nv_bfloat16, __half>::type;
  extern __shared__ int32_t s_split[];
  const int pairs = p.T * p.k, padded = (pairs + 3) / 4 * 4;
  int32_t* s_id = s_split;                       // expert of a pair (-1: none)
  int32_t* s_rank = s_id + padded;               // its place among the expert's pairs
  int32_t* s_n = s_rank + padded;                // pairs of an expert
  int3* s_at = reinterpret_cast<int3*>(s_n + p.E);   // an expert's first unit, pair, group
  const int tid = (int)threadIdx.x;
  ptx::griddep_wait();
  // (behind the wait: what the next launch reads in front of its own, ids and weights, is complete then)
  if (tid == 0) ptx::griddep_launch_dependents();
  // eight elements of a token a thread, four lanes have a block of 32; the grid has a thread for each
  const int eighths = 16 * p.off.sh;             // of a row, padded to whole steps
  const int w = (int)blockIdx.x * SPLIT_THREADS + tid, t = w / eighths, b = w - t * eighths, h0 = 8 * b;
  T e8[8];
  if (t < p.T && h0 + 8 <= p.H && ((uintptr_t)p.x & 15) == 0 && p.ldx % 8 == 0) {
    *reinterpret_cast<uint4*>(e8) = *reinterpret_cast<const uint4*>(reinterpret_cast<const T*>(p.x) + (int64_t)t * p.ldx + h0);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) e8[i] = t < p.T && h0 + i < p.H ? reinterpret_cast<const T*>(p.x)[(int64_t)t * p.ldx + h0 + i] : (T)0.0f;
  }
  for (int i = tid; i < padded; i += SPLIT_THREADS) {
    const int e = i < pairs ? p.ids[i] : -1;
    s_id[i] = e >= 0 && e < p.E ? e : -1;
  }
  float v[8];
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) { v[i] = (float)e8[i]; m = max(m, __float_as_uint(v[i]) & 0x7FFFFFFFu); }
  m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
  m = max(m, __shfl_xor_sync(0xffffffffu, m, 2));
  const uint32_t c = piece_scale(m);
  const float inv = piece_inverse(c);
  uint32_t code[PIECES];
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] *= inv;
#pragma unroll
  for (int q = 0; q < PIECES; ++q) {
    code[q] = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) code[q] |= next_piece(v[2 * i], v[2 * i + 1]) << (8 * i);
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
  if (tid < 32) plan_units(s_n, p.E, p.unit, (uint32_t)tid, [&](int e, int, int3 at) { s_at[e] = at; });
  __syncthreads();
  if (blockIdx.x == 0)
    for (int i = tid; i < pairs; i += SPLIT_THREADS)
      if (s_id[i] >= 0) reinterpret_cast<int32_t*>(p.ws + p.off.pairs)[s_at[s_id[i]].y + s_rank[i]] = i;
  if (t >= p.T) return;
  const int step = b >> 4;
  for (int j = 0; j < p.k; ++j) {
    const int i = t * p.k + j, e = s_id[i];
    if (e < 0) continue;
    const int u = s_rank[i] / p.unit, r = s_rank[i] - u * p.unit;
    const int3 at = s_at[e];
    uint8_t* dst = p.ws + p.off.xp + ((size_t)step * p.off.groups + at.z + u * (PIECES * p.unit / 8)) * GROUP;
    uint8_t* sc = p.ws + p.off.xs + ((size_t)(at.x + u) * p.off.sh + step) * ATOM;
#pragma unroll
    for (uint32_t q = 0; q < PIECES; ++q) {
      const uint32_t row = (uint32_t)(PIECES * r) + q;
      *reinterpret_cast<uint32_t*>(dst + piece_off(row, (uint32_t)(h0 & 127) / 2)) = code[q];
      if ((uint32_t)(b & 3) == (q & 3u)) sc[atom_off(row, (uint32_t)((b >> 2) & 3))] = (uint8_t)piece_code(m, c, q);
    }
  }
}

// ---- what the two products share ------------------------------------------------------------------------------------------------
constexpr int MOE_THREADS = 384;                  // weights' producer, MMA issuer, activations' producer, one that lets the next launch in, eight epilogue warps
constexpr int MOE_MAX_SLOTS = 12;
constexpr uint32_t SMEM_MAX = 232448;
constexpr int CHUNK = 8;                          // tokens read from tensor memory at a time

struct MoeBars {
  uint64_t full[MOE_MAX_SLOTS], empty[MOE_MAX_SLOTS], acc_full[2], acc_empty[2], part_full, part_empty;
  uint32_t tmem, timed_out;
  Plan plan;
};
// A producer (one warp): the first lap of the ring at once, a lane a slot, since nothing has to be waited for; then one lane goes on, filling
// a slot when it has been released.  `fill(i, slot's address, barrier)` starts the copies of step i.
template <typename F>
__device__ __forceinline__ void produce(MoeBars& b, const uint8_t* sm, uint32_t slot_bytes, uint32_t slots, uint32_t lane, uint32_t n, uint32_t* flags, F fill) {
  if (lane < slots && lane < n) fill(lane, ptx::smem_u32(sm) + lane * slot_bytes, ptx::smem_u32(&b.full[lane]));
  __syncwarp();
  if (lane == 0) {
    Slot at(b.full, b.empty, sm, 0);
    bool ok = true;
    for (uint32_t i = slots; i < n; ++i) {
      if (!(ok = wait32(at.empty, at.ph))) break;
      fill(i, at.at, at.full);
      at.next(slots, slot_bytes);
    }
    if (!ok) atomicOr(&flags[FLAG_TIMEOUT], 1u);
  }
  __syncwarp();
}
// step counted through a CTA's tasks of `steps` each -> task, step of the task, without a division where it is the one behind the last asked for
struct Walk {
  uint32_t steps, i, t, k;
  __device__ __forceinline__ explicit Walk(uint32_t s) : steps(s), i(0), t(0), k(0) {}
  __device__ __forceinline__ void to(uint32_t j) {
    if (j == i + 1) { ++k; if (k == steps) { k = 0; ++t; } }
    else { t = j / steps; k = j - t * steps; }
    i = j;
  }
};

// the two MMAs (64 K each) of one step; nothing accumulates in front of the first where `acc` is 0
__device__ __forceinline__ void step_mma(uint32_t d, uint64_t da, uint64_t db, uint32_t sfa, uint32_t sfb, uint32_t id0, uint32_t id2, uint32_t acc) {
  ptx::mma_mxf4(d, da, db, id0, sfa, sfb, acc);
  ptx::mma_mxf4(d, da + (256 >> 4), db + (256 >> 4), id2, sfa, sfb, 1u);
}
__device__ __forceinline__ void arrive_cta(uint64_t* bar, uint32_t cta) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(ptx::mapa_u32(ptx::smem_u32(bar), cta)) : "memory");
}
__device__ __forceinline__ float4 load_cta4(const float* local, uint32_t cta) { return ptx::ld_cluster_f32x4(ptx::mapa_u32(ptx::smem_u32(local), cta)); }
// sums of the pieces of eight consecutive tokens, this lane's row (columns from `taddr`)
__device__ __forceinline__ void load_tokens(uint32_t taddr, float (&s)[CHUNK]) {
  uint32_t v[CHUNK * PIECES];
#pragma unroll
  for (int i = 0; i < CHUNK * PIECES / 16; ++i) ptx::tmem_ld_32x32b_x16(taddr + 16u * i, *reinterpret_cast<uint32_t(*)[16]>(v + 16 * i));
  ptx::tmem_ld_wait();
#pragma unroll
  for (int t = 0; t < CHUNK; ++t) {
    s[t] = __uint_as_float(v[PIECES * t + PIECES - 1]);      // (the smallest first)
#pragma unroll
    for (int q = PIECES - 2; q >= 0; --q) s[t] += __uint_as_float(v[PIECES * t + q]);
  }
}

// ---- silu(W1 x) * (W3 x) ----------------------------------------------------------------------------------------------------------
// slot = | record of W1 | record of W3 | columns of X | scale atom |
__global__ void __launch_bounds__(MOE_THREADS)
moe_up_kernel(const __grid_constant__ MoeParams p)
{
  extern __shared__ uint8_t smem_raw[];
  uint8_t* sm = smem_raw + ((128 - (ptx::smem_u32(smem_raw) & 127)) & 127);
  __shared__ MoeBars b;
  const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  constexpr uint32_t SL_B = 2 * ERECORD;
  float* part = reinterpret_cast<float*>(sm + p.ring_bytes);              // [token of the unit][W1 or W3][128 rows]
  MoeUnit* s_unit = reinterpret_cast<MoeUnit*>(part + p.unit * 256);
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
  const Plan plan = make_units(p, s_unit, reinterpret_cast<int32_t*>(part), &b.plan);
  ptx::tc_fence_before();
  __syncthreads();
  ptx::cluster_sync();
  ptx::tc_fence_after();
  const int tasks = plan.units * p.tiles_i;
  const uint32_t n_steps = cluster < tasks ? (uint32_t)((tasks - cluster + clusters - 1) / clusters * steps) : 0u;   // of this CTA
  const uint32_t COLS = (uint32_t)(PIECES * plan.most + 15) / 16 * 16;    // columns of the largest unit there is
  const uint32_t SLOT = SL_B + COLS * 64u + ATOM, NSLOT = min((uint32_t)p.ring_bytes / SLOT, (uint32_t)MOE_MAX_SLOTS), SL_SFB = SL_B + COLS * 64u;
  const uint32_t tmem = b.tmem, bufs = 4 * COLS + 32 <= (uint32_t)p.tmem_cols ? 2u : 1u, sets = tmem + 2 * bufs * COLS;
  bool ok = true;
  if (warp == 0) {
    Walk w((uint32_t)steps);
    auto record = [&](uint32_t i) {               // offset of the step's records
      w.to(i);
      const int task = cluster + (int)w.t * clusters, u = task / p.tiles_i, tile = task - u * p.tiles_i;
      return (((size_t)s_unit[u].expert * p.tiles_i + tile) * p.off.sh + k0 + w.k) * ERECORD;
    };
    produce(b, sm, SLOT, NSLOT, lane, n_steps, p.flags, [&](uint32_t i, uint32_t dst, uint32_t bar) {
      const size_t rec = record(i);
      expect32(bar, 2 * ERECORD);
      copy32(dst, p.w1 + rec, ERECORD, bar);
      copy32(dst + ERECORD, p.w3 + rec, ERECORD, bar);
      // (while the first lap waits for its activations, the second's weights come into L2)
      if (i < NSLOT && i + NSLOT < n_steps) {
        const size_t next = record(i + NSLOT);
        ptx::bulk_prefetch_l2(p.w1 + next, ERECORD);
        ptx::bulk_prefetch_l2(p.w3 + next, ERECORD);
        w.i = i;                                  // (not where the walk goes on)
        w.t = i / (uint32_t)steps;
        w.k = i - w.t * (uint32_t)steps;
      }
    });
  } else if (warp == 3) {
    // the next launch is let in behind the wait: what lies in front of this one is complete for it
    ptx::griddep_wait();
    if (lane == 0) ptx::griddep_launch_dependents();
  } else if (warp == 2) {
    ptx::griddep_wait();                          // X in pieces
    Walk w((uint32_t)steps);
    produce(b, sm, SLOT, NSLOT, lane, n_steps, p.flags, [&](uint32_t i, uint32_t dst, uint32_t bar) {
      w.to(i);
      const uint32_t k = w.k;
      const int u = (cluster + (int)w.t * clusters) / p.tiles_i;
      const MoeUnit un = s_unit[u];
      const uint32_t bytes = (uint32_t)(PIECES * un.n + 7) / 8 * GROUP;
      expect32(bar, bytes + ATOM);
      copy32(dst + SL_B, p.ws + p.off.xp + ((size_t)(k0 + k) * p.off.groups + un.group) * GROUP, bytes, bar);
      copy32(dst + SL_SFB, p.ws + p.off.xs + ((size_t)u * p.off.sh + k0 + k) * ATOM, ATOM, bar);
    });
  } else if (warp == 1) {
    if (lane == 0) {
      Slot at(b.full, b.empty, sm, 0);
      uint32_t t = 0, sf = sets, again = n_steps > NSLOT ? n_steps - NSLOT : 0u;      // slots that will be filled again
      const uint64_t a0 = ptx::smem_desc(at.at, 128, 512), b0 = a0 + (SL_B >> 4), c0 = ptx::smem_desc(at.at, 0, 128), cb0 = c0 + (SL_SFB >> 4);
      uint64_t off = 0;
      for (int task = cluster; task < tasks && ok; task += clusters, ++t) {
        const uint32_t N = (uint32_t)(PIECES * s_unit[task / p.tiles_i].n + 15) / 16 * 16, buf = bufs == 2 ? t & 1u : 0u, use = bufs == 2 ? t >> 1 : t;
        const uint32_t acc = tmem + buf * 2 * COLS;
        const uint32_t id0 = ptx::idesc_block_scaled(128, N, 1, false, 0, 0), id2 = ptx::idesc_block_scaled(128, N, 1, false, 2, 2);
        if (use > 0 && !(ok = ptx::mbar_wait(&b.acc_empty[buf], (use - 1) & 1u))) break;
        for (int k = 0; k < steps; ++k) {
          if (!(ok = wait32(at.full, at.ph))) break;
          ptx::tc_fence_after();
          ptx::tc_cp_32x128b_warpx4(sf, c0 + off + (ECODES >> 4));
          ptx::tc_cp_32x128b_warpx4(sf + 4, c0 + off + ((ERECORD + ECODES) >> 4));
          ptx::tc_cp_32x128b_warpx4(sf + 8, cb0 + off);
          step_mma(acc, a0 + off, b0 + off, sf, sf + 8, id0, id2, k ? 1u : 0u);
          step_mma(acc + COLS, a0 + off + (ERECORD >> 4), b0 + off, sf + 4, sf + 8, id0, id2, k ? 1u : 0u);
          if (again) { --again; commit32(at.empty); }
          sf = sets + (sets + 12u - sf);          // (the other set)
          off += SLOT >> 4;
          at.next(NSLOT, SLOT);
          if (at.s == 0) off = 0;
        }
        if (ok) ptx::tc_commit(&b.acc_full[buf]);
      }
      if (!ok) { atomicOr(&p.flags[FLAG_TIMEOUT], 1u); wait_for_copies(at, NSLOT); }
    }
    __syncwarp();
  } else if (warp >= 4) {
    // Epilogue: warps 4 to 7 read W1's accumulator, 8 to 11 W3's, into shared memory, and hand it back; then eight lanes have the 32 rows of
    // a token that make a block, four rows each (in tensor memory's own order, a row a thread, every code was a store of its own)
    const uint32_t q = warp & 3, which = (warp - 4) >> 2, row = q * 32 + lane, et = tid - 128;
    ptx::griddep_wait();                          // (h of the call in front may still be read)
    volatile uint32_t* timed_out = &b.timed_out;
    uint32_t t = 0;
    for (int task = cluster; task < tasks; task += clusters, ++t) {
      const int u = task / p.tiles_i, tile = task - u * p.tiles_i;
      const MoeUnit un = s_unit[u];
      const uint32_t buf = bufs == 2 ? t & 1u : 0u, use = bufs == 2 ? t >> 1 : t;
      uint8_t* hp = p.ws + p.off.hp + ((size_t)tile * p.off.groups + un.group) * GROUP;
      uint8_t* hs = p.ws + p.off.hs + ((size_t)u * p.off.si + tile) * ATOM;
      if (et == 0) {
        ok = ptx::mbar_wait(&b.acc_full[buf], use & 1u);
        if (ok && ks > 1 && t > 0) ok = ptx::mbar_wait_cluster(&b.part_empty, (t - 1) & 1u);
        if (!ok) *timed_out = 1u;
      }
      ptx::named_bar_sync(1, 256);                // (also: everybody is through with the task in front's sums)
      if (*timed_out) break;
      ptx::tc_fence_after();
      for (int t0 = 0; t0 < un.n; t0 += CHUNK) {
        float v[CHUNK];
        load_tokens(tmem + ((q * 32u) << 16) + buf * 2 * COLS + which * COLS + (uint32_t)(PIECES * t0), v);
#pragma unroll
        for (int j = 0; j < CHUNK; ++j)
          if (t0 + j < un.n) part[(t0 + j) * 256 + which * 128 + row] = v[j];
      }
      ptx::tc_fence_before();
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(&b.acc_empty[buf]);
      ptx::named_bar_sync(1, 256);
      if (ks > 1) {
        // (one thread's acquire, and the barrier behind it, order the peers' stores before everybody's loads)
        if (et < ks) arrive_cta(&b.part_full, et);
        if (et == 0 && !(ok = ptx::mbar_wait_cluster(&b.part_full, t & 1u))) *timed_out = 1u;
        ptx::named_bar_sync(1, 256);
        if (*timed_out) break;
      }
      // (token, block of 32 rows) by (token, block), spread over the cluster's CTAs; eight lanes one
      for (int c = (int)(rank + ks * (et >> 3)); c < 4 * un.n; c += (int)(32 * ks)) {
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
        float h[4] = {g.x / (1.0f + expf(-g.x)) * w.x, g.y / (1.0f + expf(-g.y)) * w.y, g.z / (1.0f + expf(-g.z)) * w.z, g.w / (1.0f + expf(-g.w)) * w.w};
        uint32_t m = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) m = max(m, __float_as_uint(h[j]) & 0x7FFFFFFFu);
        const uint32_t mask = 0xFFu << (lane & 24u);
        m = max(m, __shfl_xor_sync(mask, m, 1));
        m = max(m, __shfl_xor_sync(mask, m, 2));
        m = max(m, __shfl_xor_sync(mask, m, 4));
        const uint32_t sc = piece_scale(m);
        const float inv = piece_inverse(sc);
#pragma unroll
        for (int j = 0; j < 4; ++j) h[j] *= inv;
#pragma unroll
        for (uint32_t i = 0; i < PIECES; ++i) {
          const uint32_t r = (uint32_t)(PIECES * tok) + i, lo = next_piece(h[0], h[1]), hi = next_piece(h[2], h[3]);
          *reinterpret_cast<uint16_t*>(hp + piece_off(r, r0 / 2)) = (uint16_t)(lo | hi << 8);
          if ((et & 7u) == i) hs[atom_off(r, blk)] = (uint8_t)piece_code(m, sc, i);
        }
      }
      if (ks > 1) {
        ptx::named_bar_sync(1, 256);
        if (et < ks) arrive_cta(&b.part_empty, et);
      }
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
// A cluster has one tile of 128 outputs; its CTAs share the steps of all units.  slot = | record of W2 | columns of h | scale atom |
template <int DT>
__global__ void __launch_bounds__(MOE_THREADS, 2)
moe_down_kernel(const __grid_constant__ MoeParams p)
{
  using T = typename std::conditional<DT == SDQ_BF16, __nv_bfloat16, __half>::type;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* sm = smem_raw + ((128 - (ptx::smem_u32(smem_raw) & 127)) & 127);
  __shared__ MoeBars b;
  const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  constexpr uint32_t SL_B = ERECORD;
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
  const Plan plan = make_units(p, s_unit, reinterpret_cast<int32_t*>(sm), &b.plan);
  for (uint32_t i = tid; i < (uint32_t)p.T * 128u; i += MOE_THREADS) out[i] = 0.0f;
  ptx::fence_proxy_async();                        // (the counts lay where the ring is)
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  const uint32_t COLS = (uint32_t)(PIECES * plan.most + 15) / 16 * 16;
  const uint32_t SLOT = SL_B + COLS * 64u + ATOM, NSLOT = min((uint32_t)p.ring_bytes / SLOT, (uint32_t)MOE_MAX_SLOTS), SL_SFB = SL_B + COLS * 64u;
  const uint32_t tmem = b.tmem, bufs = 2 * COLS + 16 <= (uint32_t)p.tmem_cols ? 2u : 1u, sets = tmem + bufs * COLS;
  const int SI = p.off.si, total = plan.units * SI;                       // steps of a unit, of the tile
  const int g0 = (int)((int64_t)rank * total / ks), g1 = (int)((int64_t)(rank + 1) * total / ks);
  bool ok = true;
  if (warp == 0) {
    Walk w((uint32_t)SI);
    produce(b, sm, SLOT, NSLOT, lane, (uint32_t)(g1 - g0), p.flags, [&](uint32_t i, uint32_t dst, uint32_t bar) {
      w.to((uint32_t)g0 + i);
      expect32(bar, ERECORD);
      copy32(dst, p.w2 + (((size_t)s_unit[w.t].expert * p.tiles_h + tile) * SI + w.k) * ERECORD, ERECORD, bar);
    });
  } else if (warp == 3) {
    // the next launch is let in behind the wait: what lies in front of this one is complete for it
    ptx::griddep_wait();
    if (lane == 0) ptx::griddep_launch_dependents();
  } else if (warp == 2) {
    ptx::griddep_wait();                          // h
    Walk w((uint32_t)SI);
    produce(b, sm, SLOT, NSLOT, lane, (uint32_t)(g1 - g0), p.flags, [&](uint32_t i, uint32_t dst, uint32_t bar) {
      w.to((uint32_t)g0 + i);
      const uint32_t u = w.t, k = w.k;
      const MoeUnit un = s_unit[u];
      const uint32_t bytes = (uint32_t)(PIECES * un.n + 7) / 8 * GROUP;
      expect32(bar, bytes + ATOM);
      copy32(dst + SL_B, p.ws + p.off.hp + ((size_t)k * p.off.groups + un.group) * GROUP, bytes, bar);
      copy32(dst + SL_SFB, p.ws + p.off.hs + ((size_t)u * SI + k) * ATOM, ATOM, bar);
    });
  } else if (warp == 1) {
    if (lane == 0) {
      Slot at(b.full, b.empty, sm, 0);
      uint32_t seg = 0, sf = sets, again = (uint32_t)(g1 - g0) > NSLOT ? (uint32_t)(g1 - g0) - NSLOT : 0u;
      const uint64_t a0 = ptx::smem_desc(at.at, 128, 512), b0 = a0 + (SL_B >> 4), ca0 = ptx::smem_desc(at.at + ECODES, 0, 128), cb0 = ptx::smem_desc(at.at + SL_SFB, 0, 128);
      uint64_t off = 0;
      for (int g = g0; g < g1 && ok; ++seg) {
        const int u = g / SI, end = min(g1, (u + 1) * SI);
        const uint32_t N = (uint32_t)(PIECES * s_unit[u].n + 15) / 16 * 16, buf = bufs == 2 ? seg & 1u : 0u, use = bufs == 2 ? seg >> 1 : seg, acc = tmem + buf * COLS;
        const uint32_t id0 = ptx::idesc_block_scaled(128, N, 1, false, 0, 0), id2 = ptx::idesc_block_scaled(128, N, 1, false, 2, 2);
        if (use > 0 && !(ok = ptx::mbar_wait(&b.acc_empty[buf], (use - 1) & 1u))) break;
        for (uint32_t more = 0; g < end; ++g, more = 1) {
          if (!(ok = wait32(at.full, at.ph))) break;
          ptx::tc_fence_after();
          ptx::tc_cp_32x128b_warpx4(sf, ca0 + off);
          ptx::tc_cp_32x128b_warpx4(sf + 4, cb0 + off);
          step_mma(acc, a0 + off, b0 + off, sf, sf + 4, id0, id2, more);
          if (again) { --again; commit32(at.empty); }
          sf = sets + (sets + 8u - sf);
          off += SLOT >> 4;
          at.next(NSLOT, SLOT);
          if (at.s == 0) off = 0;
        }
        if (ok) ptx::tc_commit(&b.acc_full[buf]);
      }
      if (!ok) { atomicOr(&p.flags[FLAG_TIMEOUT], 1u); wait_for_copies(at, NSLOT); }
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
      const uint32_t buf = bufs == 2 ? seg & 1u : 0u, use = bufs == 2 ? seg >> 1 : seg;
      if (et == 0 && !(ok = ptx::mbar_wait(&b.acc_full[buf], use & 1u))) *timed_out = 1u;
      ptx::named_bar_sync(1, 128);
      if (*timed_out) break;
      ptx::tc_fence_after();
      for (int t0 = 0; t0 < un.n; t0 += CHUNK) {
        float v[CHUNK];
        load_tokens(tmem + ((q * 32u) << 16) + buf * COLS + (uint32_t)(PIECES * t0), v);
#pragma unroll
        for (int j = 0; j < CHUNK; ++j)
          if (t0 + j < un.n) {
            const int2 pr = s_pair[un.pair0 + t0 + j];
            out[pr.x * 128 + row] += __int_as_float(pr.y) * v[j];
          }
      }
      ptx::tc_fence_before();
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(&b.acc_empty[buf]);
    }
    if (et == 0 && !ok) atomicOr(&p.flags[FLAG_TIMEOUT], 1u);
    __syncwarp();
  }
  ptx::tc_fence_before();
  __syncthreads();
  ptx::cluster_sync();
  ptx::griddep_wait();                             // (all threads: Y may be in use by a kernel in front)
  // (neighbouring threads of a CTA on neighbouring outputs; dealt out one by one among the CTAs, the loads cost 10 us at 64 tokens)
  for (uint32_t i = rank * MOE_THREADS + tid; i < 32u * (uint32_t)p.T; i += ks * MOE_THREADS) {
    const int t = (int)(i >> 5), r0 = (int)(i & 31u) * 4;
    const float4 s = sum_over_cluster(out + t * 128 + r0, ks);
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
static sdq_status_t moe(MoeParams p, DeviceInfo* d, void* stream) {
  auto up = moe_up_kernel;
  auto down = moe_down_kernel<DT>;
  if (!with_smem(up, d, 0) || !with_smem(down, d, 1 + DT)) return launch_status(cudaErrorUnknown);
  const int pairs = p.T * p.k;
  p.unit = unit_pairs(p.T, pairs, p.E);
  p.max_units = (pairs < p.E ? pairs : p.E) + pairs / p.unit;
  // Few pairs an expert: both products in half an SM's shared and tensor memory, so that two CTAs of the first run on an SM, or the second's CTAs beside the
  // first's, with their weights under way when h comes (shared_for_columns: tensor memory serves whatever an SM has room for)
  const bool half = p.unit <= 16, few = p.T <= 16;
  p.tmem_cols = half ? 256 : 512;
  const uint32_t room = (half ? SMEM_MAX / 2 - 1024 : SMEM_MAX) - 1024 - 128;
  {
    const size_t smem = (size_t)(pairs + 3) / 4 * 4 * 8 + (size_t)p.E * 16;
    const int threads = few ? 64 : 256;
    Launch l((unsigned)((p.T * 16 * (int64_t)p.off.sh + threads - 1) / threads), (unsigned)threads, 0, smem, stream);
    const sdq_status_t st = launch_status(few ? cudaLaunchKernelEx(&l.lc, moe_split_kernel<DT, 64>, p) : cudaLaunchKernelEx(&l.lc, moe_split_kernel<DT, 256>, p));
    if (st != SDQ_OK) return st;
  }
  {
    const int64_t tasks = (int64_t)p.max_units * p.tiles_i;                // (at most)
    // (half an SM each and more tasks than SMs: two CTAs an SM, as in the second product.  us with one and with two: 16 tokens, 8 of 64 experts of
    // 4096 x 1408, 146 and 127, 8 tokens, 2 of 8 of 4096 x 11008, 117 and 108, 1 token, 2 of 8 of 4096 x 14336, 53.6 and 48.3, 3 tokens, 2 of 35 of
    // 2899 x 3121, 36.7 and 32.2; 32 tokens, 2 of 8 of 4096 x 11008, in units of twenty by one CTA 119, of sixteen by two 108, 17 tokens,
    // 8 of 64 of 4096 x 1408, 142 and 121)
    const int64_t at_once = half && tasks > d->sm_count ? 2 * d->sm_count : d->sm_count;
    int best = 1;
    int64_t cost = 0;
    for (int ks = 1; ks <= 8 && ks <= p.off.sh; ks *= 2) {
      const int64_t cl = at_once / ks, c = ((tasks + cl - 1) / cl) * ((p.off.sh + ks - 1) / ks + (ks > 1 ? 4 : 2));
      if (ks == 1 || c < cost) { best = ks; cost = c; }
    }
    const uint32_t behind = (uint32_t)p.unit * 1024u + (uint32_t)p.max_units * (uint32_t)sizeof(MoeUnit);
    p.ring_bytes = (int32_t)((room - behind) / 128 * 128);
    const int64_t cl = at_once / best < tasks ? at_once / best : tasks;
    Launch l((unsigned)(cl * best), MOE_THREADS, (unsigned)best, shared_for_columns((size_t)p.ring_bytes + behind + 128, p.tmem_cols), stream);
    const sdq_status_t st = launch_status(cudaLaunchKernelEx(&l.lc, up, p));
    if (st != SDQ_OK) return st;
  }
  {
    // two CTAs an SM, twice as many as SMs where there is work for them: an SM's two MMA issuers hide each other's trips, and the SMs that
    // have one CTA get the more of the memory's bandwidth (64 tokens, 2 of 8 experts of 4096 x 11008: the layer 147 us with one an SM, 130 with two)
    p.tmem_cols = 256;
    int ks = 1;
    while (ks < 8 && 2 * ks * p.tiles_h <= 2 * d->sm_count && 2 * ks <= p.max_units * p.off.si) ks *= 2;
    const uint32_t room = SMEM_MAX / 2 - 1024 - 1024 - 128, behind = (uint32_t)p.T * 512u + (uint32_t)pairs * 8u + (uint32_t)p.max_units * (uint32_t)sizeof(MoeUnit);
    p.ring_bytes = (int32_t)((room - behind) / 128 * 128);
    Launch l((unsigned)(p.tiles_h * ks), MOE_THREADS, (unsigned)ks, shared_for_columns((size_t)p.ring_bytes + behind + 128, p.tmem_cols), stream);
    return launch_status(cudaLaunchKernelEx(&l.lc, down, p));
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
  if (E * d1.tiles * d1.kblocks > 0x7FFFFFFF || E * d2.tiles * d2.kblocks > 0x7FFFFFFF) return SDQ_ERR_SHAPE;   // (tasks and steps are counted in 32 bits)
  MoeParams p = {};
  p.off = moe_offsets(T, k, H, I);
  if (ws_bytes < p.off.total) return SDQ_ERR_BUFFER_TOO_SMALL;
  DeviceInfo* d = device_info();
  p.flags = device_flags();
  if (!d || !p.flags) return SDQ_ERR_CUDA;
  p.x = X; p.ids = ids; p.weights = weights; p.y = Y; p.ws = (uint8_t*)ws;
  p.w1 = (const uint8_t*)w1->dev; p.w3 = (const uint8_t*)w3->dev; p.w2 = (const uint8_t*)w2->dev;
  p.ldx = ldx; p.ldy = ldy;
  p.T = (int32_t)T; p.k = k; p.E = (int32_t)E; p.H = (int32_t)H; p.I = (int32_t)I; p.tiles_h = (int32_t)d2.tiles; p.tiles_i = (int32_t)d1.tiles;
  return dtype == SDQ_BF16 ? moe<SDQ_BF16>(p, d, stream) : moe<SDQ_FP16>(p, d, stream);
}
