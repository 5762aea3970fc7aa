// Attention of packed rows of new tokens over a paged cache or over the pack itself, a warp for each row
// and query head on the CUDA cores: fp32, and everything that the tensor-core kernels do not take.
//
// What bounds it.  Every row reads all the keys that it sees, so the calls that it is meant for are the small
// ones in fp32; there the chain of a warp counts: 32 dot products at once (a lane a key), one maximum and
// one sum over the warp, then the values column by column.
#include "kernels.h"
#include "rows_attn.cuh"

namespace glide {
namespace {

constexpr int kRowWarps = 4;

// The sequence of packed row i: the last b with cu[b] <= i.
__device__ __forceinline__ int seq_at(const RowsParams& p, int i) {
  int lo = 0, hi = p.B - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (__ldcg(p.cu + mid) <= i) lo = mid; else hi = mid - 1;
  }
  return lo;
}

template <typename T, int D>
__global__ void __launch_bounds__(kRowWarps * 32) rows_kernel(const RowsParams p) {
  constexpr int kE = D / 32;
  pdl_wait();
  const int lane = threadIdx.x & 31;
  const long long total = (long long)p.T * p.H, step = (long long)gridDim.x * kRowWarps;
  for (long long x = (long long)blockIdx.x * kRowWarps + (threadIdx.x >> 5); x < total; x += step) {
    const int row = (int)(x / p.H), h = (int)(x - (long long)row * p.H);
    const int b = seq_at(p, row);
    const Seq s = seq_of(p, b);
    const int i = row - s.row0;
    if (i < 0 || i >= s.rows) continue;
    const int n = seen(s, i);
    float o[kE];
    if (n > 0) {
      attend_row<T, D>(p, b, s, i, h, n, o);
    } else {
#pragma unroll
      for (int e = 0; e < kE; ++e) o[e] = 0.f;
    }
    store_row<kE>(reinterpret_cast<T*>(p.out) + x * D + lane * kE, o);
  }
}

template <typename T, int D>
cudaError_t launch_typed(const RowsParams& p, cudaStream_t st) {
  const long long blocks = ((long long)p.T * p.H + kRowWarps - 1) / kRowWarps;
  const unsigned grid = (unsigned)(blocks < (1 << 30) ? blocks : (1 << 30));
  return launch_pdl(rows_kernel<T, D>, dim3(grid), dim3(kRowWarps * 32), 0, st, p);
}

}  // namespace

cudaError_t launch_rows_fma(const RowsArgs& a, cudaStream_t st) {
  const RowsParams p = rows_params(a);
  if (a.dtype == 0) return a.D == 128 ? launch_typed<__nv_bfloat16, 128>(p, st) : launch_typed<__nv_bfloat16, 64>(p, st);
  return a.D == 128 ? launch_typed<float, 128>(p, st) : launch_typed<float, 64>(p, st);
}

}  // namespace glide
