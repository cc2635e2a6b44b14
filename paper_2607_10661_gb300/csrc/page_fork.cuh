// Internal launcher of the forks of paged sequences (not part of the C ABI).
#pragma once
#include <cuda_runtime.h>

#include <cstddef>
#include <cstdint>

namespace ptd {
struct PageForkParams {
  int from_batch, to_batch;
  int num_pages, max_pages, page_log2;
  const int32_t* table;        // from: [from_batch][max_pages]
  const int32_t* held;
  const int32_t* free_pages;   // [num_pages]
  const int32_t* free_count;
  int32_t* new_table;          // to: [to_batch][max_pages]
  int32_t* new_held;
  int32_t* new_free_pages;
  int32_t* new_free_count;
  const int32_t* parents;      // [to_batch]
  const int32_t* lens;
  void* k;                     // the cache
  void* v;
  int num_layers;
  int64_t row_bytes;           // of a slot, a multiple of 16
  int32_t* dev_status;
  int32_t* scratch;            // page_fork_scratch_ints() of them
};
// Turns of a CTA that copy a page of K (or V); a call's, to_batch times as many, fit in an int.
int page_copy_chunks(int64_t page_bytes);
size_t page_fork_scratch_ints(int num_pages, int from_batch, int to_batch);
cudaError_t launch_page_fork(const PageForkParams& p, int sms, cudaStream_t stream);
}  // namespace ptd
