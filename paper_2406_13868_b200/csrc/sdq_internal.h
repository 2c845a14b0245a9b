// Internals shared by the translation units of the library (not part of the C-ABI).
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>

#include "../../include/sdq.h"

namespace sdq {

// Sticky device-side flag words (one small allocation-free __device__ array per loaded library).
enum { FLAG_TIMEOUT = 1, FLAG_COUNT = 4 };

// device address of the flag words of the current device (nullptr on failure)
uint32_t* device_flags();

// Host-side facts about one device, looked up by the CURRENT device of the calling thread: they differ between the
// GPUs of one process (SM count; function attributes are per context), so nothing of this kind is a process-wide static.
// Threads share the table: sm_count is filled in under a lock, and so are pair_clusters, before clusters_known says so.
struct DeviceInfo {
  int sm_count;            // 0 until queried
  std::atomic<uint32_t> linear_attr;    // 1: the single-CTA GEMM instantiations carry their shared-memory attribute
  std::atomic<uint32_t> pair_attr;      // bit per CTA-pair GEMM instantiation
  std::atomic<uint32_t> diag_attr;      // the copy-rate diagnostic
  std::atomic<uint32_t> group_attr;     // the grouped few-token GEMM
  std::atomic<uint32_t> mx4_attr;       // bit per instantiation of the microscaled 4-bit GEMMs
  std::atomic<uint32_t> mx4_quant_attr; // bit per instantiation of the row-streaming quantizer
  std::atomic<uint32_t> moe_attr;       // the expert layer's kernels
  std::atomic<uint32_t> clusters_known; // 1: pair_clusters is filled in
  int pair_clusters[5];    // CTA-pair GEMM: clusters of k pairs that run at once
};
constexpr int MAX_DEVICES = 64;
// entry of device `dev` (0 <= dev < MAX_DEVICES) in the table; nullptr outside that range
DeviceInfo* device_info_slot(int dev);
// entry of the current device with sm_count filled in (nullptr on failure).  First use per device takes a lock.
DeviceInfo* device_info();

// Dynamic shared memory of a thread block that takes `columns` columns of tensor memory and needs `bytes`: at least so much that its columns are
// there whenever an SM has room for it.  An SM is given thread blocks by their threads, registers and shared memory (228 KB, 1 KB of it
// reserved for each); of its 512 columns of tensor memory whoever places them knows nothing, and a thread block whose columns are taken waits
// for them, without a limit, while its cluster's others may wait for it.  Two clusters, of one launch, of two streams or of a launch that was let in early, could
// so hold the columns that each other's peers wait for.  With a quarter of the shared memory for 128 columns, nearly half for 256 and
// what leaves less than a quarter for 512, no set of thread blocks that an SM has room for asks for more than 512.
constexpr int SM_SHARED = 233472, SHARED_RESERVED = 1024;
constexpr size_t shared_for_columns(size_t bytes, int columns) {
  const size_t least = columns <= 128 ? SM_SHARED / 4 - SHARED_RESERVED : columns <= 256 ? 112640 : 3 * (SM_SHARED / 4);
  return bytes > least ? bytes : least;
}

// status of a launch that returned `e`; takes the thread's last error with it, or the next call would report it as its own
inline sdq_status_t launch_status(cudaError_t e) {
  const cudaError_t last = cudaGetLastError();
  return e == cudaSuccess && last == cudaSuccess ? SDQ_OK : SDQ_ERR_CUDA;
}

// sdq_quantize_act; early_next: the next launch of the stream, the caller's own, may begin and read packed weights before this
// one has waited for its predecessor
sdq_status_t quantize_act(const void* X, int64_t M, int64_t K, int64_t ldx, const sdq_config_t* cfg, void* xq_buf, size_t xq_bytes, sdq_act_t* out,
                          void* stream, bool early_next);

}  // namespace sdq
