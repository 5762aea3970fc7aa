// The cache in pages: launch interface between the C ABI (abi.cu) and its kernels.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

namespace glide {

struct PlanArgs {
  const int32_t *q_len, *kv_len, *held, *n_free;
  int32_t *table, *free_pages;
  int32_t *cu_q, *slots, *positions, *new_kv_len, *new_held, *new_n_free;  // positions may be null
  int B, T, P, W, free_cap;
};

struct PagedAppendArgs {
  void *K, *V;
  const void *k_new, *v_new;
  long long k_stride, v_stride;  // bytes from token to token
  const int32_t* slots;
  long long n_slots;             // n_pages * page_size
  int T, H, page_shift, row_bytes;  // H: cached heads; row_bytes: of one head's row
};

// Packed rows of new tokens that attend to a paged cache, or (table null) to packed keys and values.
struct RowsArgs {
  const void *q, *K, *V;
  void* out;
  void* ws;
  const int32_t* cu;       // [B + 1]
  const int32_t* kv_len;   // [B]; packed: null, the sequence's own length
  const int32_t* table;    // [B, W]; packed: null
  long long q_stride, k_stride, v_stride;  // elements from token to token (K, V: packed only)
  int B, T, H, Hkv, D, W, n_pages, page_shift;
  int max_q, max_kv;
  int dtype;               // 0 bf16, 1 f32
  float scale;
  unsigned flags;
};

cudaError_t launch_page_plan(const PlanArgs& a, cudaStream_t st);
cudaError_t launch_paged_append(const PagedAppendArgs& a, cudaStream_t st);
// On the CUDA cores, every type and size.
cudaError_t launch_rows_fma(const RowsArgs& a, cudaStream_t st);
// Whether that kernel is the fastest one for bf16 rows.
bool rows_fma_leads(const RowsArgs& a);
// bf16, pages, at most 16 query rows for a cached head; cudaErrorNotSupported for others.
cudaError_t launch_paged_few(const RowsArgs& a, cudaStream_t st);
// bf16, at most 128 query heads for a cached head, on the tensor cores; cudaErrorNotSupported for others and beyond 32-bit
// coordinates.
cudaError_t launch_rows_tc(const RowsArgs& a, cudaStream_t st);

size_t rows_workspace_bytes(int B, int H, int Hkv, int D, int T, int max_q, int dtype);

}  // namespace glide
