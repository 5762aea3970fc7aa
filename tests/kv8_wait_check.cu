// The bounded waits of the 8-bit cache's tcgen05 kernel (kv8_wait.cuh) made to run out, on barriers that nothing completes,
// with the kernels' own limit of a second.  One CTA of four warps:
//   warp 0  gives up after the limit and raises the abort flag;
//   warp 1  starts half the limit later and is released by the flag, not by its own limit;
//   warp 2  waits on a barrier that completes, and later asks once more with the flag set;
//   warp 3  waits on nothing, and later, with the flag set, on a barrier that never completes.
// Then one thread records the status.  Prints what each waiter saw, the status word and the microseconds since the start.
#include <cstdio>

#include "kv8_wait.cuh"

namespace {

__global__ void __launch_bounds__(128) wait_kernel(unsigned* status, int* saw, unsigned long long* ns) {
  __shared__ uint64_t bar[4];
  __shared__ int abort_flag;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int b = 0; b < 4; ++b) glide::mbar_init(&bar[b], 1);
    abort_flag = 0;
    glide::fence_barrier_init();
  }
  __syncthreads();
  if (threadIdx.x == 64) glide::mbar_arrive(&bar[2]);
  const uint64_t t0 = glide::global_timer_ns();
  int ok = 2;
  if (warp == 0) ok = glide::warp_wait(&bar[0], 0, &abort_flag);
  if (warp == 1) {
    for (int i = 0; i < 1 << 24 && glide::global_timer_ns() - t0 < glide::kWaitLimitNs / 2; ++i) {
    }
    __syncwarp();
    ok = glide::warp_wait(&bar[1], 0, &abort_flag);
  }
  if (warp == 2) ok = glide::warp_wait(&bar[2], 0, &abort_flag);
  __syncwarp();
  if (lane == 0) ns[warp] = glide::global_timer_ns() - t0;
  const bool same = __all_sync(0xffffffffu, ok == __shfl_sync(0xffffffffu, ok, 0));
  if (lane == 0) saw[warp] = same ? ok : -1;
  __syncthreads();
  if (warp >= 2) ok = glide::warp_wait(&bar[warp], 0, &abort_flag);
  if (warp >= 2 && lane == 0) saw[2 + warp] = ok, ns[2 + warp] = glide::global_timer_ns() - t0;
  if (threadIdx.x == 0) glide::record_abort(&abort_flag, status);
}

}  // namespace

int main() {
  struct Out {
    unsigned long long ns[6];
    unsigned status[4];
    int saw[6];
  }* out;
  if (cudaMallocManaged(&out, sizeof(Out)) != cudaSuccess) return 2;
  *out = Out{};
  wait_kernel<<<1, 128>>>(out->status, out->saw, out->ns);
  if (cudaDeviceSynchronize() != cudaSuccess) return 2;
  for (int w = 0; w < 6; ++w) std::printf("%d ", out->saw[w]);
  std::printf("%u", out->status[0]);
  for (int w = 0; w < 6; ++w) std::printf(" %llu", out->ns[w] / 1000);
  std::printf("\n");
  return cudaFree(out) == cudaSuccess ? 0 : 2;
}
