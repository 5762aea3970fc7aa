// Attention of packed rows of new tokens over a paged cache or over the pack itself, a block for each row and query
// head on the CUDA cores: fp32, everything that the tensor-core kernels do not take, and bf16 calls of at most 32 keys that
// are small for them (rows_fma_leads).
//
// What bounds it.  Every row reads all the keys that it sees, so the calls that it is meant for are the small ones; there
// the chain of a row counts.  A block's four warps take a row's keys in turn, 32 at a time, with up to 16 loads in flight each:
// 32 dot products at once (a lane a key), one maximum and one sum over the warp, then the values column by column; the
// warps' results meet in shared memory.  Where no row can see more than 32 keys, each warp has a row of its own.
// Two fp32 prompts of 60 to 128 tokens, 4 heads of 64: 9.8 to 10.1 us, 940 blocks where 912 are resident (a warp a row and 4 loads in flight: 40).  Registers are bounded for
// six blocks an SM (four with 128 dims), where the values of eight keys at once fit without spills; 12 or 16 keys do not (prompts of
// 32 tokens, 4 heads of 64: 5.2, 5.4 and 5.5 us; of 115 and 120: 10.6, 12.0 and 11.9).
#include "device.h"
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

// Output rows x = row * H + head = x0, x0 + step, .. by the definition.  (Out of line, after a loop that is done: the kernel keeps its
// registers.  With grids of up to 2^30 blocks there is mostly one row.)
template <typename T, int D, int kRowsAt>
__device__ __noinline__ void define_rows(const RowsParams& p) {
  const long long total = (long long)p.T * p.H;
#pragma unroll 1
  for (long long x = (long long)blockIdx.x * kRowsAt + (kRowsAt > 1 ? threadIdx.x >> 5 : 0); x < total; x += (long long)gridDim.x * kRowsAt) {
    const int row = (int)(x / p.H), h = (int)(x - (long long)row * p.H);
    const int b = seq_at(p, row);
    const Seq s = seq_of(p, b);
    const int i = row - s.row0;
    if (i < 0 || i >= s.rows || seen(s, i) == 0) continue;
    float o[D / 32];
    attend_row<T, D>(p, b, s, i, h, seen(s, i), o);
    store_row<D / 32>(reinterpret_cast<T*>(p.out) + x * D + (threadIdx.x & 31) * (D / 32), o);
  }
}

// kPerRow: warps of a row, 1 or all of the block.
template <typename T, int D, int kPerRow>
__global__ void __launch_bounds__(kRowWarps * 32, D == 64 ? 6 : 4) rows_kernel(const __grid_constant__ RowsParams p) {
  constexpr int kE = D / 32;
  __shared__ float part_o[kRowWarps][D], part_m[kRowWarps], part_l[kRowWarps];
  pdl_wait();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const long long total = (long long)p.T * p.H;
  constexpr int kRowsAt = kRowWarps / kPerRow;
  bool again = false;
  for (long long x = (long long)blockIdx.x * kRowsAt + (kPerRow == 1 ? warp : 0); x < total; x += (long long)gridDim.x * kRowsAt) {
    const int row = (int)(x / p.H), h = (int)(x - (long long)row * p.H);
    const int b = seq_at(p, row);
    const Seq s = seq_of(p, b);
    const int i = row - s.row0;
    if (i < 0 || i >= s.rows) continue;
    const int n = seen(s, i);
    RowPart<D> r = no_keys<D>();
    if (n > 0) attend_keys<T, D>(p, b, s, i, h, n, (kPerRow == 1 ? 0 : warp) * 32, kPerRow * 32, r);
    // A sum of weights that is 0 or NaN makes the row NaN by definition; a result that is not finite beside another sum of
    // weights has to be computed again.
    if constexpr (kPerRow == 1) {
      bool odd = false;
#pragma unroll
      for (int e = 0; e < kE; ++e) {
        r.o[e] = n > 0 ? r.o[e] / r.l : 0.f;
        odd |= !isfinite(r.o[e]);
      }
      store_row<kE>(reinterpret_cast<T*>(p.out) + x * D + lane * kE, r.o);
      again |= __any_sync(0xffffffffu, odd) && r.l > 0.f;
    } else {
#pragma unroll
      for (int e = 0; e < kE; ++e) part_o[warp][lane * kE + e] = r.o[e];
      if (lane == 0) {
        part_m[warp] = r.m;
        part_l[warp] = r.l;
      }
      __syncthreads();
      bool odd = false;
      if (threadIdx.x < D) {
        float m = -CUDART_INF_F, l = 0.f, o = 0.f;
#pragma unroll
        for (int w = 0; w < kRowWarps; ++w) m = fmaxf(m, part_m[w]);
        const float ref = m == -CUDART_INF_F ? 0.f : m;
#pragma unroll
        for (int w = 0; w < kRowWarps; ++w) {
          const float f = fast_exp2(part_m[w] - ref);
          l += f * part_l[w];
          o += f * part_o[w][threadIdx.x];
        }
        o = n > 0 ? o / l : 0.f;
        odd = !isfinite(o) && l > 0.f;
        store_one(reinterpret_cast<T*>(p.out) + x * D + threadIdx.x, o);
      }
      again |= __syncthreads_or(odd) != 0;  // (the row's parts have been read, and its first result is written)
    }
  }
  if (again && (kPerRow == 1 || warp == 0)) define_rows<T, D, kRowsAt>(p);
}

template <typename T, int D>
cudaError_t launch_typed(const RowsParams& p, int keys, cudaStream_t st) {
  const long long rows = (long long)p.T * p.H, blocks = keys <= 32 ? (rows + kRowWarps - 1) / kRowWarps : rows;
  const unsigned grid = (unsigned)(blocks < (1 << 30) ? blocks : (1 << 30));
  if (keys <= 32) return launch_pdl(rows_kernel<T, D, 1>, dim3(grid), dim3(kRowWarps * 32), 0, st, p);
  return launch_pdl(rows_kernel<T, D, kRowWarps>, dim3(grid), dim3(kRowWarps * 32), 0, st, p);
}

constexpr int most_keys(const RowsArgs& a) { return a.table ? a.max_kv : a.max_q; }

}  // namespace

// A row of at most 32 keys is one pass of a warp here, and the tensor-core kernel starts for about 6 us and then has a
// chain of 3.7 us for each of an SM's items (a request's rows of one cached head), however few they are.  Measured, here
// and there, 8 or 32 query heads of 128 over 8 cached: about 2.5 us + 2 ns a row against 6 + 0.025 an item.  Prompts of
// 4 tokens, 8 heads: 1024 rows 4.6 and 12.1 us, 16384 rows 36 and 106; of 32 tokens: 2048 rows 9.2 and 9.1, 8192 rows
// 25 and 12; four heads to a cached one, prompts of 16: 2048 rows 6.6 and 8.9, 8192 rows 19 and 9.  Above 32 keys the
// tensor cores lead almost from the first row on (48 keys: 768 rows 8.5 and 8.8 us, 1920 rows 17 and 9).
// Where launch_paged_few would serve the rows (pages, at most 16 of a cached head), its CTA for each cached head leads until
// they are more than two for an SM; from there, a call of 1200 cached heads, 128 dims: 1 row of 16 keys 6.2 us here and 16.3
// there, 2 of 32 keys 11 and 17, 4 of 16 keys 14 and 18, but 8 of 32 keys 40 and 21.
bool rows_fma_leads(const RowsArgs& a) {
  const long long slabs = (long long)a.B * a.Hkv, slab_rows = (long long)a.max_q * (a.H / a.Hkv);
  if (most_keys(a) > 32) return false;
  if (a.table && slab_rows <= 16) return slabs > 2LL * sm_count() && most_keys(a) * slab_rows <= 64;
  const long long items = slabs * ((slab_rows + 127) / 128);
  return (long long)a.T * a.H <= 2048 + 12 * items;
}

cudaError_t launch_rows_fma(const RowsArgs& a, cudaStream_t st) {
  const RowsParams p = rows_params(a);
  const int keys = most_keys(a);
  if (a.dtype == 0)
    return a.D == 128 ? launch_typed<__nv_bfloat16, 128>(p, keys, st) : launch_typed<__nv_bfloat16, 64>(p, keys, st);
  return a.D == 128 ? launch_typed<float, 128>(p, keys, st) : launch_typed<float, 64>(p, keys, st);
}

}  // namespace glide
