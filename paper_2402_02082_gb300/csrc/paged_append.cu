// New keys and values into a paged pool by their slots.
//
// A token's rows of all cached heads lie side by side where it comes from and a page apart where it goes, so the work is
// a copy of 16-byte pieces with one division for the head.  What bounds it: HBM for prompts (every byte once in, once
// out), the launch for a decoding step.  16384 tokens of 32 heads of 128, bf16: 83 to 85 us, 6.3 to 6.5 TB/s of a copy's 6.8;
// 64 tokens of 8 heads: 2.5 us.
#include "common.cuh"
#include "device.h"
#include "kernels.h"
#include "paged.h"

namespace glide {
namespace {

constexpr int kAppThreads = 256;

__global__ void __launch_bounds__(kAppThreads) paged_append_kernel(const PagedAppendArgs a, int pieces, int row_shift) {
  pdl_wait();
  const long long total = (long long)a.T * pieces, step = (long long)gridDim.x * kAppThreads;
  for (long long x = (long long)blockIdx.x * kAppThreads + threadIdx.x; x < total; x += step) {
    const int i = (int)(x / pieces), c = (int)(x - (long long)i * pieces);
    const int slot = __ldcg(a.slots + i);
    if (slot < 0 || slot >= a.n_slots) continue;
    const int h = c >> row_shift, piece = c & ((1 << row_shift) - 1);
    const long long page = slot >> a.page_shift, r = slot & ((1 << a.page_shift) - 1);
    const long long to = (((page * a.H + h) << a.page_shift) + r) * a.row_bytes + 16 * piece;
    const uint4 k = *reinterpret_cast<const uint4*>(static_cast<const unsigned char*>(a.k_new) + i * a.k_stride + 16ll * c);
    const uint4 v = *reinterpret_cast<const uint4*>(static_cast<const unsigned char*>(a.v_new) + i * a.v_stride + 16ll * c);
    *reinterpret_cast<uint4*>(static_cast<unsigned char*>(a.K) + to) = k;
    *reinterpret_cast<uint4*>(static_cast<unsigned char*>(a.V) + to) = v;
  }
}

}  // namespace

cudaError_t launch_paged_append(const PagedAppendArgs& a, cudaStream_t st) {
  const int pieces = a.H * a.row_bytes / 16;
  int row_shift = 0;
  while ((16 << row_shift) < a.row_bytes) ++row_shift;
  const long long blocks = ((long long)a.T * pieces + kAppThreads - 1) / kAppThreads;
  const long long most = 16ll * sm_count();
  return launch_pdl(paged_append_kernel, dim3((unsigned)(blocks < most ? blocks : most)), dim3(kAppThreads), 0, st, a, pieces,
                    row_shift);
}

}  // namespace glide
