// Attention of packed rows of new tokens over a paged cache or over the pack itself, a block for each row and query
// head on the CUDA cores: fp32, and everything that the tensor-core kernels do not take.
//
// What bounds it.  Every row reads all the keys that it sees, so the calls that it is meant for are the small
// ones in fp32; there the chain of a row counts.  Four warps take its keys in turn, 32 at a time, with 16 loads in flight
// each: 32 dot products at once (a lane a key), one maximum and one sum over the warp, then the values column by column;
// the warps' results meet in shared memory.  Two prompts of 60 to 128 tokens, 4 heads of 64: a warp a row 40 us.
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
  __shared__ float part_o[kRowWarps][D], part_m[kRowWarps], part_l[kRowWarps];
  pdl_wait();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const long long total = (long long)p.T * p.H;
  for (long long x = blockIdx.x; x < total; x += gridDim.x) {
    const int row = (int)(x / p.H), h = (int)(x - (long long)row * p.H);
    const int b = seq_at(p, row);
    const Seq s = seq_of(p, b);
    const int i = row - s.row0;
    if (i < 0 || i >= s.rows) continue;
    const int n = seen(s, i);
    RowPart<D> r = no_keys<D>();
    if (n > 0) attend_keys<T, D, 16>(p, b, s, i, h, n, warp * 32, kRowWarps * 32, r);
    __syncthreads();  // the row before has been read
#pragma unroll
    for (int e = 0; e < kE; ++e) part_o[warp][lane * kE + e] = r.o[e];
    if (lane == 0) {
      part_m[warp] = r.m;
      part_l[warp] = r.l;
    }
    __syncthreads();
    if (threadIdx.x < D) {
      float m = -CUDART_INF_F, l = 0.f, o = 0.f;
#pragma unroll
      for (int w = 0; w < kRowWarps; ++w) m = fmaxf(m, part_m[w]);
      const float ref = m == -CUDART_INF_F ? 0.f : m;
#pragma unroll
      for (int w = 0; w < kRowWarps; ++w) {
        float f = fast_exp2(part_m[w] - ref);
        if (part_m[w] != -CUDART_INF_F) f = f < FLT_MIN ? FLT_MIN : f;  // an infinite value keeps its weight (a NaN stays one)
        l += f * part_l[w];
        o += f * part_o[w][threadIdx.x];
      }
      store_one(reinterpret_cast<T*>(p.out) + x * D + threadIdx.x, n > 0 ? o / l : 0.f);
    }
  }
}

template <typename T, int D>
cudaError_t launch_typed(const RowsParams& p, cudaStream_t st) {
  const long long blocks = (long long)p.T * p.H;
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
