// The waits of the attention of packed rows (wait_watched, warp_wait_watched, put_off in rows_wait.cuh): with a limit of
// 20 ms that is put off for 100 ms they wait as long, and give up 20 ms later.  One CTA of four warps:
//   warp 0, lane 0  waits for what comes at the end of the 100 ms, and gets it;
//   warp 1          as a whole warp, for what never comes: gives up 20 ms behind them, and raises the abort flag;
//   warp 2, lane 0  waits for what never comes too, and gives up by the deadline or by the flag;
//   warp 3          puts the waits off every millisecond for 100, then completes warp 0's barrier.
// Then one thread records the status.  Prints what each waiter saw, the status word and the microseconds.
#include <cstdio>

#include "rows_wait.cuh"

namespace {

constexpr uint32_t kLimitNs = 20000000u;

__global__ void __launch_bounds__(128) wait_kernel(unsigned* status, int* saw, unsigned long long* ns) {
  __shared__ uint64_t bar[3];
  __shared__ glide::Watch watch;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int b = 0; b < 3; ++b) glide::mbar_init(&bar[b], 1);
    watch.abort = 0;
    glide::put_off(&watch, kLimitNs);
    glide::fence_barrier_init();
  }
  __syncthreads();
  const uint64_t t0 = glide::global_timer_ns();
  int ok = 2;
  if (warp == 0 && lane == 0) ok = glide::wait_watched(&bar[0], 0, &watch);
  if (warp == 1) ok = glide::warp_wait_watched(&bar[1], 0, &watch);
  if (warp == 2 && lane == 0) ok = glide::wait_watched(&bar[2], 0, &watch);
  if (warp == 3 && lane == 0) {
    for (int i = 1; i <= 100; ++i) {
      while (glide::global_timer_ns() - t0 < i * 1000000ull) {
      }
      glide::put_off(&watch, kLimitNs);
    }
    glide::mbar_arrive(&bar[0]);
  }
  __syncwarp();
  if (lane == 0) ns[warp] = glide::global_timer_ns() - t0;
  const bool same = __all_sync(0xffffffffu, ok == __shfl_sync(0xffffffffu, ok, 0));
  if (lane == 0) saw[warp] = warp == 1 && !same ? -1 : ok;
  __syncthreads();
  if (warp == 3) {  // a completed phase is seen whatever the flag says
    ok = glide::warp_wait_watched(&bar[0], 0, &watch);
    if (lane == 0) saw[4] = ok;
  }
  if (threadIdx.x == 0) glide::record_abort(&watch.abort, status);
}

}  // namespace

int main() {
  struct Out {
    unsigned long long ns[4];
    unsigned status[4];
    int saw[8];
  }* out;
  if (cudaMallocManaged(&out, sizeof(Out)) != cudaSuccess) return 2;
  *out = Out{};
  wait_kernel<<<1, 128>>>(out->status, out->saw, out->ns);
  if (cudaDeviceSynchronize() != cudaSuccess) return 2;
  std::printf("%d %d %d %d %u", out->saw[0], out->saw[1], out->saw[2], out->saw[4], out->status[0]);
  for (int w = 0; w < 4; ++w) std::printf(" %llu", out->ns[w] / 1000);
  std::printf("\n");
  return cudaFree(out) == cudaSuccess ? 0 : 2;
}
