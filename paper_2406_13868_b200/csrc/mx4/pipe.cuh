// The ring's operations on 32-bit shared-memory addresses.  One thread fills a ring and one thread empties it, and a trip of either loop has to be
// shorter than what it moves takes: a thread alone issues an instruction every few clocks, so addresses and descriptors are kept and
// stepped instead of being worked out in every trip.
//
// Every kernel of this directory lets the next launch in behind its own wait for the one in front (griddepcontrol.launch_dependents after
// griddepcontrol.wait).  A launch may then read, in front of its own wait, what was complete before the launch in front of it began to work:
// the library's other products read packed weights there, this directory's expert layer ids and experts' weights.
#pragma once
#include "../sdq_ptx.cuh"

namespace sdq {
namespace mx4 {

__device__ __forceinline__ bool test32(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile("{\n.reg .pred p;\nmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
  return ok != 0;
}
__device__ __forceinline__ bool wait32(uint32_t bar, uint32_t parity, uint32_t limit = 1u << 22) {
  uint32_t ok = test32(bar, parity);
  for (uint32_t i = 0; !ok && i < limit; ++i)
    asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
  return ok != 0;
}
__device__ __forceinline__ void expect32(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy32(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
__device__ __forceinline__ void commit32(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
// the two halves of ptx::cluster_sync
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
// sum over the cluster's CTAs (up to eight), in their order, of the four floats at `local`; all of them are asked for before the first is added
__device__ __forceinline__ float4 sum_over_cluster(const float* local, uint32_t ctas) {
  const uint32_t at = ptx::smem_u32(local);
  float4 v[8];
#pragma unroll
  for (uint32_t c = 0; c < 8; ++c)
    if (c < ctas) v[c] = ptx::ld_cluster_f32x4(ptx::mapa_u32(at, c));
  float4 s = v[0];
#pragma unroll
  for (uint32_t c = 1; c < 8; ++c)
    if (c < ctas) { s.x += v[c].x; s.y += v[c].y; s.z += v[c].z; s.w += v[c].w; }
  return s;
}
// position in a ring of `n` slots: barriers 8 bytes apart, data `size` bytes apart; `ph` flips with every lap
struct Slot {
  uint32_t s, ph, full, empty, at;
  __device__ __forceinline__ Slot(const uint64_t* full0, const uint64_t* empty0, const void* data, uint32_t phase)
      : s(0), ph(phase), full(ptx::smem_u32(full0)), empty(ptx::smem_u32(empty0)), at(ptx::smem_u32(data)) {}
  __device__ __forceinline__ void next(uint32_t n, uint32_t size) {
    ++s; full += 8; empty += 8; at += size;
    if (s == n) { s = 0; ph ^= 1u; full -= 8 * n; empty -= 8 * n; at -= size * n; }
  }
};

// for the thread that empties a ring, whose wait gave up at `at`: waits, with a limit, for the copies that may still be under way, those of a lap from there
// on, so that none is left when the shared memory becomes another thread block's (who calls this is waited for before the thread block can leave)
__device__ __forceinline__ void wait_for_copies(Slot at, uint32_t slots) {
#pragma unroll 1
  for (uint32_t i = 0; i < slots; ++i) {
    (void)wait32(at.full, at.ph, 1u << 16);
    at.next(slots, 0);
  }
}

}  // namespace mx4
}  // namespace sdq
