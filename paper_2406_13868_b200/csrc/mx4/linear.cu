// Product of two microscaled 4-bit matrices  Y = Xq Wq^T + bias  on the block-scaled tensor-core kinds
// (kind::mxf4 .block32 for MXFP4, kind::mxf4nvf4 .block16 for NVFP4; fp32 accumulators in tensor memory).
//
// Few tokens (mx4_linear_narrow_kernel): weights stream through, so their rows are the MMA's 128 rows and the tokens its columns.
// The CTAs of a cluster split K of one row tile, keep their fp32 partial tiles in shared memory and sum them there in a fixed
// order: no scratch in global memory, no atomics, the same result every time.
//
// Many tokens (mx4_linear_wide_kernel): CTA pairs, 256 tokens x 256 weight rows a task, K in records of 256.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <type_traits>

#include "../sdq_internal.h"
#include "layout.h"
#include "pipe.cuh"
#include "../sdq_ptx.cuh"

namespace sdq {
namespace mx4 {

struct GemmParams {
  const uint8_t *x, *w;            // records of the activations and of the weights
  const float *fx, *fw;            // row factors (NVFP4)
  const void* bias;
  void* Y;
  uint32_t* flags;
  int64_t M, N, ldy;
  int32_t kb;                      // records along K
  int32_t m_tiles, n_tiles;        // row tiles of 128 of both
  int32_t T;                       // narrow: token columns of a tile
  int32_t wide_rows;               // narrow: rows of Y keep four outputs aligned
  int32_t nslot;
  int32_t pt_m, pt_n, tasks;       // wide: tiles of 256, tasks
};

template <int DT> struct Out;
template <> struct Out<SDQ_BF16> { using type = __nv_bfloat16; };
template <> struct Out<SDQ_FP16> { using type = __half; };
template <> struct Out<SDQ_FP32> { using type = float; };
template <int DT> __device__ __forceinline__ typename Out<DT>::type to_out(float v) {
  if constexpr (DT == SDQ_BF16) return __float2bfloat16_rn(v);
  else if constexpr (DT == SDQ_FP16) return __float2half_rn(v);
  else return v;
}
template <int DT> __device__ __forceinline__ float from_out(typename Out<DT>::type v) {
  if constexpr (DT == SDQ_BF16) return __bfloat162float(v);
  else if constexpr (DT == SDQ_FP16) return __half2float(v);
  else return v;
}

// ---- row factors (NVFP4) ----------------------------------------------------------------------------------------------------
// s fw fx + b.  The product of two factors that both lie in [2^-62, 2^62], or are zero, is a normal number or zero: one multiplication of the sum.
// Others, a whole row's magnitude each, can leave fp32's range together although the output does not, and are applied one after the other: where
// their product is too small the larger one first, where it is too large the smaller one.  s is zero or between 2^-20, the smallest product of two held elements, and 2^53,
// so that nothing in between is lost: factors of a product below 2^-126 have a larger one of at most 2^23 (the smaller one is 2^-149 or more), and s
// times it is a subnormal number only where the output is zero; of a product above 2^128, a smaller one above 1, and s times it is too large only
// where the output is.
__device__ __forceinline__ bool plain_factor(float f) {
  const uint32_t e = __float_as_uint(f) << 1;
  return e == 0u || (e >= (65u << 24) && e <= (189u << 24));
}
__device__ __forceinline__ float apply_factors(float s, float fw, float fx, float b) {
  const float f = fw * fx, mag = fabsf(f), large = fabsf(fw) > fabsf(fx) ? fw : fx, small = fabsf(fw) > fabsf(fx) ? fx : fw;
  if (mag >= 1.17549435e-38f && mag < INFINITY) return fmaf(s, f, b);
  return mag < 1.0f ? fmaf(s * large, small, b) : fmaf(s * small, large, b);      // (a NaN stays one)
}

// ---- few tokens -----------------------------------------------------------------------------------------------------------
constexpr int NARROW_THREADS = 256;                  // weights' producer, MMA issuer, tokens' producer, an idle warp, four epilogue warps
constexpr uint32_t NARROW_TAIL = 256 + 128;          // barriers, and room to align the ring to 128 bytes
constexpr int NARROW_MAX_SLOTS = 12;
// slot = | weight record | codes of T tokens | scale atoms of the tokens |
__host__ __device__ constexpr uint32_t narrow_slot(int fmt, int T) { return record(fmt) + (uint32_t)T * 128u + atoms(fmt) * ATOM; }

template <int FMT, int DT>
__global__ void __launch_bounds__(NARROW_THREADS)
mx4_linear_narrow_kernel(const __grid_constant__ GemmParams p)
{
  using T_out = typename Out<DT>::type;
  constexpr uint32_t NA = atoms(FMT), REC = record(FMT), SET = 8u * NA;       // TMEM columns of one set of scales: 4 NA weights, 4 NA tokens
  extern __shared__ uint8_t smem_raw[];
  uint8_t* sm = smem_raw + ((128 - (ptx::smem_u32(smem_raw) & 127)) & 127);
  const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t T = (uint32_t)p.T, SLOT = narrow_slot(FMT, p.T), NSLOT = (uint32_t)p.nslot;
  uint64_t* full = reinterpret_cast<uint64_t*>(sm + (size_t)NSLOT * SLOT);
  uint64_t* empty = full + NARROW_MAX_SLOTS;
  uint64_t* acc_full = empty + NARROW_MAX_SLOTS;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(acc_full + 1);
  static_assert((2 * NARROW_MAX_SLOTS + 1) * 8 + 4 <= 256);
  uint32_t ks;
  asm volatile("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(ks));
  const uint32_t rank = ptx::cluster_ctarank();
  const int nt = (int)(blockIdx.x / ks), mt = (int)blockIdx.y;
  const int k0 = (int)(rank * (uint32_t)p.kb / ks), n_rec = (int)((rank + 1) * (uint32_t)p.kb / ks) - k0;
  const uint8_t* w = p.w + ((size_t)nt * p.kb + k0) * REC;
  const uint8_t* x = p.x + ((size_t)mt * p.kb + k0) * REC;

  if (warp == 0) {
    if (lane == 0) {
      for (uint32_t i = 0; i < NSLOT; ++i) { ptx::mbar_init(&full[i], 2); ptx::mbar_init(&empty[i], 1); }
      ptx::mbar_init(acc_full, 1);
      ptx::fence_barrier_init();
      // the weights may be what the kernel in front writes: they are brought into L2, which holds what is written, not into
      // shared memory
      for (int i = 0; i < min(n_rec, (int)NSLOT); ++i) ptx::bulk_prefetch_l2(w + (size_t)i * REC, REC);
    }
  } else if (warp == 1) {
    ptx::tmem_alloc(tmem_slot, 256);
  }
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  const uint32_t tmem = *tmem_slot, sets = tmem + 128u;
  ptx::griddep_wait();
  if (tid == 0) ptx::griddep_launch_dependents();

  bool ok = true;
  if (warp == 0 || warp == 2) {
    if (lane == 0) {
      Slot at(full, empty, sm, 1);
      const uint8_t* src = warp ? x : w;
      for (int i = 0; i < n_rec; ++i, src += REC) {
        if (i >= (int)NSLOT && !(ok = wait32(at.empty, at.ph))) break;
        if (warp == 0) {
          expect32(at.full, REC);
          copy32(at.at, src, REC, at.full);
        } else {
          expect32(at.full, T * 128u + NA * ATOM);
          copy32(at.at + REC, src, T * 128u, at.full);
          copy32(at.at + REC + T * 128u, src + CODES, NA * ATOM, at.full);
        }
        at.next(NSLOT, SLOT);
      }
      if (!ok) atomicOr(&p.flags[FLAG_TIMEOUT], 1u);
    }
    __syncwarp();
  } else if (warp == 1) {
    if (lane == 0) {
      // copies to tensor memory and MMAs of one thread execute in issue order: two alternating sets of scales serve all slots
      const uint32_t id0 = ptx::idesc_block_scaled(128, T, 1, false, 0, 0) ^ (FMT == SDQ_FMT_NVFP4 ? 1u << 23 : 0u);
      const uint32_t id2 = ptx::idesc_block_scaled(128, T, 1, false, 2, 2);
      Slot at(full, empty, sm, 0);
      const uint64_t a0 = ptx::smem_desc(at.at, 128, 1024), b0 = ptx::smem_desc(at.at + REC, 128, 1024);
      const uint64_t ca0 = ptx::smem_desc(at.at + CODES, 0, 128), cb0 = ptx::smem_desc(at.at + REC + T * 128u, 0, 128);
      uint64_t off = 0;
      uint32_t sfa = sets;
      for (int i = 0; i < n_rec; ++i) {
        if (!(ok = wait32(at.full, at.ph))) break;
        ptx::tc_fence_after();
        const uint32_t sfb = sfa + 4 * NA;
#pragma unroll
        for (uint32_t a = 0; a < NA; ++a) {
          ptx::tc_cp_32x128b_warpx4(sfa + 4 * a, ca0 + off + a * (ATOM >> 4));
          ptx::tc_cp_32x128b_warpx4(sfb + 4 * a, cb0 + off + a * (ATOM >> 4));
        }
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) {                       // 64 K each: two adjacent core matrices
          const uint32_t acc = i || j ? 1u : 0u;
          if constexpr (FMT == SDQ_FMT_NVFP4) ptx::mma_nvf4(tmem, a0 + off + ((256 * j) >> 4), b0 + off + ((256 * j) >> 4), id0, sfa + 4 * j, sfb + 4 * j, acc);
          else ptx::mma_mxf4(tmem, a0 + off + ((256 * j) >> 4), b0 + off + ((256 * j) >> 4), j & 1 ? id2 : id0, sfa + 4 * (j >> 1), sfb + 4 * (j >> 1), acc);
        }
        commit32(at.empty);
        sfa = sets + (sets + SET - sfa);                         // (the other set)
        off += SLOT >> 4;
        at.next(NSLOT, SLOT);
        if (at.s == 0) off = 0;
      }
      if (ok) ptx::tc_commit(acc_full);
      else { atomicOr(&p.flags[FLAG_TIMEOUT], 1u); wait_for_copies(at, NSLOT); }
    }
    __syncwarp();
  } else if (warp >= 4) {
    // warp w moves TMEM lanes 32 (w % 4) .. (weight rows) to where the ring was: [token][128 rows]
    const uint32_t q = warp & 3;
    ok = ptx::mbar_wait(acc_full, 0);
    if (!__all_sync(0xffffffffu, ok) && lane == 0) atomicOr(&p.flags[FLAG_TIMEOUT], 1u);
    ptx::tc_fence_after();
    float* part = reinterpret_cast<float*>(sm) + q * 32 + lane;
    for (uint32_t c0 = 0; c0 < T; c0 += 32) {
      uint32_t v[2][16];
      ptx::tmem_ld_32x32b_x16(tmem + ((q * 32u) << 16) + c0, v[0]);
      if (c0 + 16 < T) ptx::tmem_ld_32x32b_x16(tmem + ((q * 32u) << 16) + c0 + 16, v[1]);
      ptx::tmem_ld_wait();
#pragma unroll
      for (int j = 0; j < 16; ++j) part[(c0 + j) * ROWS] = __uint_as_float(v[0][j]);
      if (c0 + 16 < T) {
#pragma unroll
        for (int j = 0; j < 16; ++j) part[(c0 + 16 + j) * ROWS] = __uint_as_float(v[1][j]);
      }
    }
    ptx::tc_fence_before();
  }
  // every CTA's partial tile is in place
  if (ks > 1) ptx::cluster_sync(); else __syncthreads();
  {
    const int64_t n0 = (int64_t)nt * ROWS, m0 = (int64_t)mt * 128;
    const uint32_t n = (tid & 31u) * 4;                          // this thread's rows of the tile
    float fw[4], b[4];
    bool plain_w = true;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const bool in = n0 + n + j < p.N;
      fw[j] = FMT == SDQ_FMT_NVFP4 && in ? p.fw[n0 + n + j] : 1.0f;
      plain_w = plain_w && plain_factor(fw[j]);
      b[j] = p.bias && in ? from_out<DT>(reinterpret_cast<const T_out*>(p.bias)[n0 + n + j]) : 0.0f;
    }
    const int valid = (int)min((int64_t)T, p.M - m0);
    const bool whole = n0 + n + 4 <= p.N && p.wide_rows;         // four outputs are one aligned store
    const float* part = reinterpret_cast<const float*>(sm);
    for (int c = (int)(rank + ks * warp); c < valid; c += (int)ks * (NARROW_THREADS / 32)) {
      const float* src = part + c * ROWS + n;
      const float4 s4 = ks > 1 ? sum_over_cluster(src, ks) : *reinterpret_cast<const float4*>(src);
      const float fx = FMT == SDQ_FMT_NVFP4 ? __ldg(p.fx + m0 + c) : 1.0f;
      const float s[4] = {s4.x, s4.y, s4.z, s4.w};
      T_out o[4];
      if (FMT != SDQ_FMT_NVFP4 || (plain_w && plain_factor(fx))) {
#pragma unroll
        for (int j = 0; j < 4; ++j) o[j] = to_out<DT>(fmaf(s[j], FMT == SDQ_FMT_NVFP4 ? fw[j] * fx : 1.0f, b[j]));
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) o[j] = to_out<DT>(apply_factors(s[j], fw[j], fx, b[j]));
      }
      T_out* y = reinterpret_cast<T_out*>(p.Y) + (m0 + c) * p.ldy + n0 + n;
      if (whole) {
        if constexpr (DT == SDQ_FP32) *reinterpret_cast<float4*>(y) = make_float4(o[0], o[1], o[2], o[3]);
        else *reinterpret_cast<uint2*>(y) = *reinterpret_cast<const uint2*>(o);
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (n0 + n + j < p.N) y[j] = o[j];
      }
    }
  }
  if (ks > 1) ptx::cluster_sync();                               // nobody leaves while its partial tile is being read
  if (warp == 1) ptx::tmem_dealloc(tmem, 256);
}

// ---- many tokens ----------------------------------------------------------------------------------------------------------
constexpr int WIDE_THREADS = 512;                    // producer, MMA issuer, one that tells of landed slots, an idle one, eight epilogue, four scale warps
constexpr int WIDE_PAIRS = 4, WIDE_SETS = 4;
// slots of the ring: what shared memory has beside the staging of outputs that are not aligned
__host__ __device__ constexpr int wide_slots(int fmt, bool vec) { return fmt == SDQ_FMT_MXFP4 && vec ? 6 : 5; }
// slot = | token record (codes, scale atoms) | codes of 128 weight rows | scale atoms of both CTAs' weight rows |
__host__ __device__ constexpr uint32_t wide_slot(int fmt) { return record(fmt) + CODES + 2 * atoms(fmt) * ATOM; }
// an arrival on a barrier of the pair's even CTA.  Relaxed: what it tells of, loads from and stores to tensor memory, has completed and been waited
// for, and is ordered by tcgen05's own fences; a releasing arrival would wait for all of the thread's memory operations, a microsecond with a ring's
// copies under way.  It passes nothing on of shared memory: that a slot has landed, warp 2 tells
__device__ __forceinline__ void arrive_leader(uint64_t* bar) {
  asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(ptx::mapa_u32(ptx::smem_u32(bar), 0)) : "memory");
}
constexpr uint32_t WIDE_PITCH = 68;                  // bytes of a staged row of 64
__host__ __device__ constexpr uint32_t wide_tail(bool vec) { return 256u + 2u * 2u * 256u * 4u + (vec ? 0u : 8u * 32u * WIDE_PITCH) + 128u; }

template <int FMT, int DT, bool VEC>
__global__ void __launch_bounds__(WIDE_THREADS)
mx4_linear_wide_kernel(const __grid_constant__ GemmParams p)
{
  using T_out = typename Out<DT>::type;
  constexpr int WIDE_SLOTS = wide_slots(FMT, VEC);
  constexpr uint32_t NA = atoms(FMT), REC = record(FMT), SLOT = wide_slot(FMT), SFA_SET = 4u * NA, SET = 12u * NA;
  static_assert(256 + WIDE_SETS * SET <= 512 && (6 + WIDE_PAIRS + 2 + WIDE_SETS) * 8 + 8 + WIDE_SETS * 4 <= 256);
  constexpr uint32_t SL_B = REC, SL_SF = REC + CODES;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* sm = smem_raw + ((128 - (ptx::smem_u32(smem_raw) & 127)) & 127);
  const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  uint64_t* full = reinterpret_cast<uint64_t*>(sm + WIDE_SLOTS * SLOT);
  uint64_t* empty = full + WIDE_SLOTS;               // [pair of stages % WIDE_PAIRS]: the MMAs that read them have completed
  uint64_t* acc_full = empty + WIDE_PAIRS;
  uint64_t* acc_empty = acc_full + 1;
  uint64_t* ready = acc_empty + 1;                   // [set] leader: slot landed and scales in tensor memory, in both CTAs
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(ready + WIDE_SETS);
  volatile uint32_t* timed_out = tmem_slot + 1;
  uint32_t* told = tmem_slot + 2;                    // [set] leader: where the odd CTA's word that its slot has landed goes
  float* s_fac = reinterpret_cast<float*>(sm + WIDE_SLOTS * SLOT + 256);       // [task parity][factor, bias][256 weight rows]
  uint8_t* s_out = reinterpret_cast<uint8_t*>(s_fac + 4 * 256);
  const uint32_t rank = ptx::cluster_ctarank();
  const int pair = (int)blockIdx.x >> 1, n_pairs = (int)gridDim.x >> 1;
  const int my_tasks = p.tasks > pair ? (p.tasks - pair + n_pairs - 1) / n_pairs : 0;
  const int KB = p.kb;

  if (warp == 0 && lane == 0) {
    for (int i = 0; i < WIDE_SLOTS; ++i) ptx::mbar_init(&full[i], 1);
    for (int i = 0; i < WIDE_SETS; ++i) ptx::mbar_init(&ready[i], 9);
    for (int i = 0; i < WIDE_PAIRS; ++i) ptx::mbar_init(&empty[i], 1);
    ptx::mbar_init(acc_full, 1);
    ptx::mbar_init(acc_empty, 16);
    *timed_out = 0u;
    ptx::fence_barrier_init();
  }
  __syncwarp();
  if (warp == 1) ptx::tmem_alloc_pair(tmem_slot, 512);
  ptx::tc_fence_before();
  __syncthreads();
  ptx::cluster_sync();
  ptx::tc_fence_after();
  const uint32_t tmem = *tmem_slot, sets = tmem + 256u;
  ptx::griddep_wait();
  if (tid == 0) ptx::griddep_launch_dependents();

  // task -> tiles of 256: weight tiles vary fastest inside bands of eight token tiles
  auto tile_of = [&](int task, int& mt, int& nt) {
    const int band = 8 * p.pt_n, b = task / band, r = task - b * band, h = min(8, p.pt_m - 8 * b);
    nt = r / h;
    mt = 8 * b + r - nt * h;
  };
  bool ok = true;
  if (warp == 0) {
    if (lane == 0) {
      int i = 0;                                     // stage, counted through the CTA's tasks
      for (int t = 0; t < my_tasks && ok; ++t) {
        int mt, nt;
        tile_of(pair + t * n_pairs, mt, nt);
        // (an odd number of tiles: the last one is taken twice, and stored once)
        const uint8_t* xa = p.x + (size_t)min(2 * mt + (int)rank, p.m_tiles - 1) * KB * REC;
        const uint8_t* w0 = p.w + (size_t)(2 * nt) * KB * REC;
        const uint8_t* w1 = p.w + (size_t)min(2 * nt + 1, p.n_tiles - 1) * KB * REC;
        const uint8_t* wb = rank ? w1 : w0;
        for (int k = 0; k < KB; ++k, ++i) {
          if (i >= WIDE_SLOTS) {
            const uint32_t q = (uint32_t)(i - WIDE_SLOTS) >> 1;
            if (!(ok = ptx::mbar_wait(&empty[q % WIDE_PAIRS], (q / WIDE_PAIRS) & 1u))) break;
          }
          const uint32_t s = (uint32_t)i % WIDE_SLOTS;
          uint8_t* st = sm + (size_t)s * SLOT;
          const size_t off = (size_t)k * REC;
          ptx::mbar_expect_tx(&full[s], SLOT);
          ptx::bulk_g2s(st, xa + off, REC, &full[s]);
          ptx::bulk_g2s(st + SL_B, wb + off, CODES, &full[s]);
          ptx::bulk_g2s(st + SL_SF, w0 + off + CODES, NA * ATOM, &full[s]);
          ptx::bulk_g2s(st + SL_SF + NA * ATOM, w1 + off + CODES, NA * ATOM, &full[s]);
        }
      }
      if (!ok) atomicOr(&p.flags[FLAG_TIMEOUT], 1u);
    }
    __syncwarp();
  } else if (warp == 1) {
    if (rank == 0 && lane == 0) {
      const uint32_t id0 = ptx::idesc_block_scaled(256, 256, 1, false, 0, 0) ^ (FMT == SDQ_FMT_NVFP4 ? 1u << 23 : 0u);
      const uint32_t id2 = ptx::idesc_block_scaled(256, 256, 1, false, 2, 2);
      const int total = my_tasks * KB;
      const uint64_t a0 = ptx::smem_desc(ptx::smem_u32(sm), 128, 1024), b0 = a0 + (SL_B >> 4);
      uint64_t off = 0;
      int i = 0;
      for (int t = 0; t < my_tasks && ok; ++t) {
        for (int k = 0; k < KB; ++k, ++i) {
          if (!(ok = ptx::mbar_wait_cluster(&ready[i % WIDE_SETS], ((uint32_t)i / WIDE_SETS) & 1u))) break;
          if (k == 0 && t > 0 && !(ok = ptx::mbar_wait_cluster(acc_empty, (uint32_t)(t - 1) & 1u))) break;
          ptx::tc_fence_after();
          const uint32_t sfa = sets + (uint32_t)(i % WIDE_SETS) * SET, sfb = sfa + SFA_SET;
#pragma unroll
          for (uint32_t j = 0; j < 4; ++j) {
            const uint32_t acc = k || j ? 1u : 0u;
            if constexpr (FMT == SDQ_FMT_NVFP4) ptx::mma2_nvf4(tmem, a0 + off + ((256 * j) >> 4), b0 + off + ((256 * j) >> 4), id0, sfa + 4 * j, sfb + 8 * j, acc);
            else ptx::mma2_mxf4(tmem, a0 + off + ((256 * j) >> 4), b0 + off + ((256 * j) >> 4), j & 1 ? id2 : id0, sfa + 4 * (j >> 1), sfb + 8 * (j >> 1), acc);
          }
          // one release for two stages: a pair-wide commit costs the tensor pipe a bubble
          if ((i & 1) && i + 1 < total) ptx::tc2_commit_both(&empty[(uint32_t)(i >> 1) % WIDE_PAIRS], 3);
          if (k == KB - 1) ptx::tc2_commit_both(acc_full, 3);
          off += SLOT >> 4;
          if (off == (uint64_t)(SLOT >> 4) * WIDE_SLOTS) off = 0;
        }
      }
      if (!ok) atomicOr(&p.flags[FLAG_TIMEOUT], 1u);
    }
    __syncwarp();
  } else if (warp == 2) {
    // Tells the thread that issues the MMAs that a slot has landed.  In the leader by an arrival, in the odd CTA by an asynchronous store of a word that
    // this arrival expects: its completion on the leader's barrier is a release at cluster scope, for which nobody waits here.  (A releasing arrival
    // there takes a microsecond under load, 8192 x 4096 -> 11008 265 us against 171, or 195 with two warps in turn; barriers of their own that the
    // issuing thread waits for as well, 190.)  Like the scale warps, not before the barrier's phase in front has completed
    if (lane == 0) {
      const uint32_t bar = ptx::mapa_u32(ptx::smem_u32(ready), 0), at = ptx::mapa_u32(ptx::smem_u32(told), 0);
      const int total = my_tasks * KB;
      Slot at_slot(full, full, sm, 0);
      for (int i = 0; i < total; ++i) {
        ok = wait32(at_slot.full, at_slot.ph);
        if (ok && i >= WIDE_SETS) {
          const uint32_t e = (uint32_t)(i - WIDE_SETS) >> 1;
          ok = ptx::mbar_wait(&empty[e % WIDE_PAIRS], (e / WIDE_PAIRS) & 1u);
        }
        if (!ok) break;
        const uint32_t set = (uint32_t)i % WIDE_SETS;
        if (rank == 0) ptx::mbar_expect_tx(&ready[set], 4);
        else ptx::st_async_u32(at + 4 * set, 0u, bar + 8 * set);
        at_slot.next(WIDE_SLOTS, SLOT);
      }
      if (!ok) { atomicOr(&p.flags[FLAG_TIMEOUT], 1u); wait_for_copies(at_slot, WIDE_SLOTS); }
    }
    __syncwarp();
  } else if (warp >= 12) {
    // Scales of a slot into tensor memory, by ordinary stores of four warps (each its 32 lanes, all the same: what a copy instruction would
    // replicate).  The copies would go through the tensor pipe, in order with its MMAs: 44 clocks each, six (MXFP4) or twelve (NVFP4) of them to
    // four MMAs of 128 -- 850 and 1115 clocks a stage instead of 590.
    const uint32_t q = warp & 3;
    uint32_t s = 0;
    const int total = my_tasks * KB;
    for (int i = 0; i < total; ++i) {
      ok = ptx::mbar_wait(&full[s], ((uint32_t)i / WIDE_SLOTS) & 1u);
      if (ok && i >= WIDE_SETS) {                    // the MMAs that read this set have completed
        const uint32_t e = (uint32_t)(i - WIDE_SETS) >> 1;
        ok = ptx::mbar_wait(&empty[e % WIDE_PAIRS], (e / WIDE_PAIRS) & 1u);
      }
      if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
      const uint8_t* st = sm + (size_t)s * SLOT;
      uint32_t v[12 * NA];                           // SFA, then of every atom the two halves of the weight rows
#pragma unroll
      for (uint32_t a = 0; a < NA; ++a) {
        *reinterpret_cast<uint4*>(v + 4 * a) = *reinterpret_cast<const uint4*>(st + CODES + a * ATOM + lane * 16);
        *reinterpret_cast<uint4*>(v + SFA_SET + 8 * a) = *reinterpret_cast<const uint4*>(st + SL_SF + a * ATOM + lane * 16);
        *reinterpret_cast<uint4*>(v + SFA_SET + 8 * a + 4) = *reinterpret_cast<const uint4*>(st + SL_SF + (NA + a) * ATOM + lane * 16);
      }
      const uint32_t at = sets + (uint32_t)(i % WIDE_SETS) * SET + ((q * 32u) << 16);
#pragma unroll
      for (uint32_t c = 0; c + 16 <= 12 * NA; c += 16) ptx::tmem_st_32x32b_x16(at + c, *reinterpret_cast<const uint32_t(*)[16]>(v + c));
      if constexpr (12 * NA % 16 != 0) {
        static_assert(12 * NA % 16 == 8);
        ptx::tmem_st_32x32b_x4(at + 12 * NA - 8, *reinterpret_cast<const uint32_t(*)[4]>(v + 12 * NA - 8));
        ptx::tmem_st_32x32b_x4(at + 12 * NA - 4, *reinterpret_cast<const uint32_t(*)[4]>(v + 12 * NA - 4));
      }
      ptx::tmem_st_wait();
      ptx::tc_fence_before();
      __syncwarp();
      if (lane == 0) arrive_leader(&ready[i % WIDE_SETS]);
      if (++s == WIDE_SLOTS) s = 0;
    }
    if (!ok && lane == 0) atomicOr(&p.flags[FLAG_TIMEOUT], 1u);
    __syncwarp();
  } else if (warp >= 4) {
    // epilogue: warp w owns TMEM lanes 32 (w % 4) .. (tokens); warps 4 to 7 the first 128 weight rows, 8 to 11 the others.  The
    // accumulator is packed into registers and handed back before anything is stored.
    const uint32_t q = warp & 3, half = (warp - 4) >> 2, et = tid - 128;
    for (int t = 0; t < my_tasks && ok; ++t) {
      int mt, nt;
      tile_of(pair + t * n_pairs, mt, nt);
      const int64_t n0 = (int64_t)nt * 256;
      float* fac = s_fac + (t & 1) * 512;
      {
        const int64_t n = n0 + et;
        fac[et] = FMT == SDQ_FMT_NVFP4 && n < p.N ? __ldg(p.fw + n) : 1.0f;
        fac[256 + et] = p.bias && n < p.N ? from_out<DT>(reinterpret_cast<const T_out*>(p.bias)[n]) : 0.0f;
      }
      const int64_t m = (int64_t)(2 * mt + (int)rank) * ROWS + q * 32 + lane;
      const float fx = FMT == SDQ_FMT_NVFP4 && m < p.M ? __ldg(p.fx + m) : 1.0f;
      if (et == 0 && !ptx::mbar_wait(acc_full, (uint32_t)t & 1u)) *timed_out = 1u;
      // (whether all factors of the CTA's tile are plain ones comes with the barrier)
      bool plain = true;
      if constexpr (FMT == SDQ_FMT_NVFP4) plain = ptx::named_bar_all(1, 256, plain_factor(fac[et]) && plain_factor(fx));
      else ptx::named_bar_sync(1, 256);
      if (*timed_out) { ok = false; break; }
      ptx::tc_fence_after();
      // (four-byte outputs in two parts: what a thread holds is 64 words)
      constexpr int PER = DT == SDQ_FP32 ? 1 : 2, WORDS = 64, COLS = WORDS * PER, PARTS = 128 / COLS;
      const bool stored = 2 * mt + (int)rank < p.m_tiles;        // (not the repeated last tile)
#pragma unroll 1
      for (int part = 0; part < PARTS; ++part) {
        const uint32_t c0 = half * 128u + (uint32_t)(part * COLS);
        uint32_t out[WORDS];
#pragma unroll
        for (int c = 0; c < COLS / 16; ++c) {
          uint32_t v[16];
          ptx::tmem_ld_32x32b_x16(tmem + ((q * 32u) << 16) + c0 + 16u * c, v);
          ptx::tmem_ld_wait();
          if (plain) {
#pragma unroll
            for (int j = 0; j < 16; ++j) {
              const uint32_t col = c0 + 16u * c + j;
              v[j] = __float_as_uint(fmaf(__uint_as_float(v[j]), FMT == SDQ_FMT_NVFP4 ? fac[col] * fx : 1.0f, fac[256 + col]));
            }
          } else {
#pragma unroll
            for (int j = 0; j < 16; ++j) {
              const uint32_t col = c0 + 16u * c + j;
              v[j] = __float_as_uint(apply_factors(__uint_as_float(v[j]), fac[col], fx, fac[256 + col]));
            }
          }
#pragma unroll
          for (int j = 0; j < 16 / PER; ++j) {
            if constexpr (DT == SDQ_FP32) out[16 * c + j] = v[j];
            else if constexpr (DT == SDQ_BF16) {
              const __nv_bfloat162 b = __floats2bfloat162_rn(__uint_as_float(v[2 * j]), __uint_as_float(v[2 * j + 1]));
              out[8 * c + j] = *reinterpret_cast<const uint32_t*>(&b);
            } else {
              const __half2 b = __floats2half2_rn(__uint_as_float(v[2 * j]), __uint_as_float(v[2 * j + 1]));
              out[8 * c + j] = *reinterpret_cast<const uint32_t*>(&b);
            }
          }
        }
        if (part == PARTS - 1) {                                 // the accumulator has been read
          ptx::tc_fence_before();
          __syncwarp();
          if (lane == 0) arrive_leader(acc_empty);
        }
        if (!stored) continue;
        T_out* y = reinterpret_cast<T_out*>(p.Y) + m * p.ldy + n0 + c0;
        const int cols = (int)min((int64_t)COLS, p.N - n0 - (int64_t)c0);
        if constexpr (VEC) {
          if (m < p.M) {
#pragma unroll
            for (int c = 0; c < WORDS / 8; ++c) {                // 32 bytes, one sector, a store
              constexpr int EL = 8 * PER;
              if ((c + 1) * EL <= cols)
                asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(y + c * EL), "r"(out[8 * c]), "r"(out[8 * c + 1]), "r"(out[8 * c + 2]),
                             "r"(out[8 * c + 3]), "r"(out[8 * c + 4]), "r"(out[8 * c + 5]), "r"(out[8 * c + 6]), "r"(out[8 * c + 7]) : "memory");
            }
          }
        } else {
          // any alignment: 64 bytes of 32 tokens at a time turned in shared memory, consecutive lanes store consecutive outputs of a token
          constexpr int EL = 16 * PER, RUN = 32 / EL;            // outputs of a token at a time, tokens a store instruction covers
          uint8_t* st = s_out + (warp - 4) * 32u * WIDE_PITCH;
          const int64_t mw = m - lane;
          const int rows = (int)min((int64_t)32, p.M - mw), col = (int)lane % EL, r0 = (int)lane / EL;
#pragma unroll
          for (int c = 0; c < WORDS / 16; ++c) {
            __syncwarp();
#pragma unroll
            for (int j = 0; j < 16; ++j) *reinterpret_cast<uint32_t*>(st + lane * WIDE_PITCH + 4u * j) = out[16 * c + j];
            __syncwarp();
            if (c * EL + col < cols) {
              T_out* yr = reinterpret_cast<T_out*>(p.Y) + mw * p.ldy + n0 + c0 + c * EL + col;
              for (int r = r0; r < rows; r += RUN) yr[(int64_t)r * p.ldy] = *reinterpret_cast<const T_out*>(st + r * WIDE_PITCH + col * sizeof(T_out));
            }
          }
        }
      }
    }
    if (!ok && lane == 0) atomicOr(&p.flags[FLAG_TIMEOUT], 1u);
    __syncwarp();
  }
  // (a peer may still signal barriers of this CTA, and its MMAs read this CTA's shared memory)
  ptx::tc_fence_before();
  __syncwarp();
  ptx::cluster_sync();
  if (warp == 1) ptx::tmem_dealloc_pair(tmem, 512);
}

// ---- launches ---------------------------------------------------------------------------------------------------------------
template <typename K>
static cudaError_t with_smem(K kern, uint32_t bytes, DeviceInfo* d, int bit) {
  if (d->mx4_attr & (1u << bit)) return cudaSuccess;
  const cudaError_t e = cudaFuncSetAttribute((const void*)kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
  if (e == cudaSuccess) d->mx4_attr |= 1u << bit;
  return e;
}
constexpr uint32_t SMEM_MAX = 232448, NARROW_LEAST = 112640;
static_assert(NARROW_LEAST == shared_for_columns(0, 256) && SMEM_MAX >= shared_for_columns(0, 512));

// CTAs that share K of a row tile in the narrow kernel: as many as keep all of them resident, two an SM, with a tenth left over for clusters
// that do not fit a GPU processing cluster (96 tiles x 3 of K = 4096 took 16.2 us, x 2 11.1); the sum over them is the dearer the more tokens there are
// (128 tokens, 4096 x 4096: four 7.7 us, eight 10.4; 16 tokens, 11008 -> 4096: four 9.8, eight 8.8; 64 tokens, 8192 -> 512: four 6.7, eight 5.4).
static int narrow_split(int64_t tiles, int T, int kb, int sms) {
  int ks = 1;
  for (int k = 2; k <= (T > 32 && 8 * tiles > sms ? 4 : 8) && k <= kb; ++k)
    if (10 * k * tiles <= 18 * sms) ks = k;
  return ks;
}
// Which kernel takes a call of more than 128 tokens: microseconds that each took, as linear functions of what its longest CTA goes through (sweeps
// of 129 to 1500 tokens against 1000 to 11008 rows, K 1000 to 11008, within 15 %).  E.g. MXFP4, narrow and wide: 256 x 4096 -> 4096 10.1 and 11.4, 333 x 4096 -> 11008
// 13.7 and 20.4, 512 x 11008 -> 4096 18.2 and 22.0, 256 x 4096 -> 11008 13.6 and 12.9, 512 x 4096 -> 11008 24.0 and 20.4
static bool narrow_is_faster(int fmt, int64_t tiles, int ks, int64_t wide_tasks, int kb, bool aligned, int sms) {
  const bool nv = fmt == SDQ_FMT_NVFP4;
  const int64_t waves = (tiles * ks + 2 * sms - 1) / (2 * sms), wide_waves = (wide_tasks + sms / 2 - 1) / (sms / 2);
  const double narrow = (double)waves * ((kb <= 8 ? 5.0 : 8.2) + (nv ? 0.55 : 0.44) * (double)((kb + ks - 1) / ks));
  const double wide = (aligned ? 3.4 : 4.9) + (double)wide_waves * (2.2 + (nv ? 0.433 : 0.374) * kb);
  return narrow < wide;
}

template <int FMT, int DT>
static sdq_status_t linear(GemmParams& p, DeviceInfo* d, void* stream) {
  cudaLaunchConfig_t lc = {};
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  lc.attrs = attr;
  lc.numAttrs = 2;
  lc.stream = (cudaStream_t)stream;
  constexpr int BIT = 3 * (FMT * 3 + DT);
  p.T = p.M <= 128 ? (int32_t)(p.M + 15) / 16 * 16 : 128;
  const int64_t tiles = (int64_t)p.n_tiles * p.m_tiles;
  const int ks = narrow_split(tiles, p.T, p.kb, d->sm_count);
  p.pt_m = (p.m_tiles + 1) / 2;
  p.pt_n = (p.n_tiles + 1) / 2;
  const int64_t sector = 32 / (int64_t)dtype_bytes(DT);
  const bool vec = ((uintptr_t)p.Y & 31) == 0 && p.ldy % sector == 0 && p.N % sector == 0;      // rows of Y in whole 32-byte sectors
  if (p.M <= 128 || p.m_tiles <= 65535 && narrow_is_faster(FMT, tiles, ks, (int64_t)p.pt_m * p.pt_n, p.kb, vec, d->sm_count)) {
    const uint32_t slot = narrow_slot(FMT, p.T);
    const uint32_t room = (tiles * ks <= d->sm_count ? SMEM_MAX : SMEM_MAX / 2 - 1024) - NARROW_TAIL;
    const int want = (p.kb + ks - 1) / ks;
    p.nslot = (int32_t)(room / slot);
    if (p.nslot > want) p.nslot = want;
    if (p.nslot > NARROW_MAX_SLOTS) p.nslot = NARROW_MAX_SLOTS;
    if (p.n_tiles > 0x7FFFFFFF / 8) return SDQ_ERR_SHAPE;
    const uint32_t ring = (uint32_t)p.nslot * slot, parts = (uint32_t)p.T * ROWS * 4u;
    // (the partial tile lies where the ring was; the barriers behind both)
    if (parts > ring) p.nslot = (int32_t)((parts + slot - 1) / slot);
    lc.gridDim = dim3((unsigned)(p.n_tiles * ks), (unsigned)p.m_tiles);
    lc.blockDim = dim3(NARROW_THREADS);
    // (nearly half of an SM's at least, for the 256 columns: see shared_for_columns)
    const uint32_t bytes = (uint32_t)p.nslot * slot + NARROW_TAIL;
    lc.dynamicSmemBytes = bytes > NARROW_LEAST ? bytes : NARROW_LEAST;
    attr[1].val.clusterDim.x = (unsigned)ks;
    p.wide_rows = ((uintptr_t)p.Y % (4 * dtype_bytes(DT))) == 0 && (p.ldy % 4 == 0 || p.M == 1);
    auto kern = mx4_linear_narrow_kernel<FMT, DT>;
    if (with_smem(kern, SMEM_MAX, d, BIT) != cudaSuccess) return launch_status(cudaErrorUnknown);
    return launch_status(cudaLaunchKernelEx(&lc, kern, p));
  }
  if ((int64_t)p.pt_m * p.pt_n > 0x3FFFFFFF) return SDQ_ERR_SHAPE;
  p.tasks = p.pt_m * p.pt_n;
  const int pairs = d->sm_count / 2 < p.tasks ? d->sm_count / 2 : p.tasks;
  lc.gridDim = dim3(2 * (unsigned)pairs);
  lc.blockDim = dim3(WIDE_THREADS);
  attr[1].val.clusterDim.x = 2;
  auto go = [&](auto kern, auto v, int bit) {
    constexpr bool V = decltype(v)::value;
    constexpr uint32_t bytes = wide_slots(FMT, V) * wide_slot(FMT) + wide_tail(V);
    static_assert(bytes <= SMEM_MAX, "the ring fits");
    lc.dynamicSmemBytes = SMEM_MAX;                  // (an SM's: nothing else that takes tensor memory is beside it)
    if (with_smem(kern, SMEM_MAX, d, bit) != cudaSuccess) return launch_status(cudaErrorUnknown);
    return launch_status(cudaLaunchKernelEx(&lc, kern, p));
  };
  return vec ? go(mx4_linear_wide_kernel<FMT, DT, true>, std::true_type{}, BIT + 1) : go(mx4_linear_wide_kernel<FMT, DT, false>, std::false_type{}, BIT + 2);
}

}  // namespace mx4
}  // namespace sdq

using namespace sdq;

extern "C" sdq_status_t sdq_mx4_linear(const sdq_mx4_t* Xq, const sdq_mx4_t* Wq, const void* bias, int32_t dtype, void* Y, int64_t ldy, void* stream)
{
  if (!mx4::desc_ok(Xq) || !mx4::desc_ok(Wq) || !Y || !mx4::dtype_ok(dtype)) return SDQ_ERR_INVALID_ARG;
  if (Xq->E || Wq->E || Xq->fmt != Wq->fmt) return SDQ_ERR_UNSUPPORTED;
  if (Xq->K != Wq->K || ldy < Wq->R || ldy > ((int64_t)1 << 40)) return SDQ_ERR_SHAPE;
  const size_t es = mx4::dtype_bytes(dtype);
  if (((uintptr_t)Y % es) || ((uintptr_t)bias % es)) return SDQ_ERR_ALIGNMENT;
  const mx4::Dims dx = mx4::dims(0, Xq->R, Xq->K, Xq->fmt), dw = mx4::dims(0, Wq->R, Wq->K, Wq->fmt);
  if (dx.tiles > 0x3FFFFFFF || dw.tiles > 0x3FFFFFFF) return SDQ_ERR_SHAPE;
  DeviceInfo* d = device_info();
  mx4::GemmParams p = {};
  p.flags = device_flags();
  if (!d || !p.flags) return SDQ_ERR_CUDA;
  p.x = (const uint8_t*)Xq->dev; p.w = (const uint8_t*)Wq->dev;
  p.fx = reinterpret_cast<const float*>(p.x + dx.factors); p.fw = reinterpret_cast<const float*>(p.w + dw.factors);
  p.bias = bias; p.Y = Y; p.M = Xq->R; p.N = Wq->R; p.ldy = ldy;
  p.kb = (int32_t)dx.kblocks; p.m_tiles = (int32_t)dx.tiles; p.n_tiles = (int32_t)dw.tiles;
  auto go = [&](auto fmt) -> sdq_status_t {
    constexpr int F = decltype(fmt)::value;
    return dtype == SDQ_BF16   ? mx4::linear<F, SDQ_BF16>(p, d, stream)
           : dtype == SDQ_FP16 ? mx4::linear<F, SDQ_FP16>(p, d, stream)
                               : mx4::linear<F, SDQ_FP32>(p, d, stream);
  };
  return Xq->fmt == SDQ_FMT_NVFP4 ? go(std::integral_constant<int, SDQ_FMT_NVFP4>{}) : go(std::integral_constant<int, SDQ_FMT_MXFP4>{});
}
