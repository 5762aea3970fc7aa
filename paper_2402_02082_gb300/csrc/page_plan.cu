// The page tables and slots of a serving step, from the requests' lengths: which pages the requests of a
// step get from the stack of free ones, and where each new token's key and value go.
//
// The mathematics is three running sums over the requests: new tokens (the packed offsets), pages that finished
// requests give back, pages that live ones ask for.  With them every output is a function of its own index:
//   page x of the stack       free[x] below n_free, else a finished request's table entry
//   the y-th page handed out  page avail - 1 - y of that stack
//   page j of request b       its table below held[b], else the (asked before b + j - held[b])-th handed out
// so nothing that is written is read back, and CTAs need not wait for one another: each makes the sums for
// itself and writes its share of the outputs.
//
// What bounds it: latency.  The lengths are a few kB; a step of 32 requests is one CTA with two dependent
// loads (lengths, a page number) and six barriers of its 32 warps: 4.4 us, a launch without work ~2.5.  1024
// requests with 80 thousand new tokens: 6.5 us (0.85 MB).
#include "common.cuh"
#include "device.h"
#include "kernels.h"
#include "paged.h"

namespace glide {
namespace {

constexpr int kPlanThreads = 1024;
static_assert(kPlanThreads >= kMaxBatch, "a thread a request");

// Running sums over the requests before and at one.
struct Sums {
  unsigned tokens;
  int pages;
};
// Tokens count as at most T (below 2^31, so that no sum of two wraps).
__device__ __forceinline__ Sums plus(const Sums& a, const Sums& b, unsigned T) {
  const unsigned t = a.tokens + b.tokens;
  return {t < T ? t : T, a.pages + b.pages};
}
__device__ __forceinline__ Sums scan_warp(Sums v, unsigned T, int lane) {
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    const Sums u = {__shfl_up_sync(0xffffffffu, v.tokens, off), __shfl_up_sync(0xffffffffu, v.pages, off)};
    if (lane >= off) v = plus(u, v, T);
  }
  return v;
}
// Inclusive, over the block's threads; `warps` is the block's own scratch for this call.
__device__ __forceinline__ Sums scan_block(Sums v, unsigned T, Sums* warps) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  v = scan_warp(v, T, lane);
  if (lane == 31) warps[warp] = v;
  __syncthreads();
  if (warp == 0) warps[lane] = scan_warp(lane < (int)(blockDim.x >> 5) ? warps[lane] : Sums{0u, 0}, T, lane);
  __syncthreads();
  return warp > 0 ? plus(warps[warp - 1], v, T) : v;
}

// The last b in [0, B) with at[b] <= x, where at[0] <= x.
__device__ __forceinline__ int last_at_most(const int* at, int B, int x) {
  int lo = 0, hi = B - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (at[mid] <= x) lo = mid; else hi = mid - 1;
  }
  return lo;
}

__global__ void __launch_bounds__(kPlanThreads) page_plan_kernel(const PlanArgs a, int shift) {
  // before request b: new tokens, pages given back, pages asked for
  __shared__ int tok[kMaxBatch + 1], back[kMaxBatch + 1], ask[kMaxBatch + 1];
  __shared__ int kvs[kMaxBatch], helds[kMaxBatch];
  __shared__ bool oks[kMaxBatch];
  __shared__ Sums scratch[2][32];
  __shared__ int s_n_free, s_taken;
  const int tid = threadIdx.x;
  pdl_wait();
  const bool real = tid < a.B;
  const int q = real ? __ldcg(a.q_len + tid) : 0, kv0 = real ? __ldcg(a.kv_len + tid) : 0, held0 = real ? __ldcg(a.held + tid) : 0;
  if (tid == 0) {
    const int n = __ldcg(a.n_free);
    s_n_free = n < 0 ? 0 : (n > a.free_cap ? a.free_cap : n);
    s_taken = 0;
    tok[0] = back[0] = ask[0] = 0;
  }
  const bool done = q < 0;
  const int kv = kv0 < 0 ? 0 : kv0, held = held0 < 0 ? 0 : (held0 > a.W ? a.W : held0);
  const unsigned T = (unsigned)a.T;
  const Sums one = scan_block({q <= 0 ? 0u : ((unsigned)q < T ? (unsigned)q : T), real && done ? held : 0}, T, scratch[0]);
  if (real) {
    tok[tid + 1] = (int)one.tokens;
    back[tid + 1] = one.pages;
    kvs[tid] = kv;
    helds[tid] = held;
  }
  __syncthreads();
  const int m = real ? tok[tid + 1] - tok[tid] : 0;
  const long long most = (long long)kv + m;
  const long long want = (most + a.P - 1) >> shift;
  const bool fits = real && !done && want <= a.W && most <= 0x7fffffffLL;
  const int need = fits && m > 0 && want > held ? (int)want - held : 0;
  const Sums two = scan_block({0u, need}, T, scratch[1]);
  const int n_free = s_n_free;
  const long long on_stack = (long long)n_free + back[a.B];
  const int avail = (int)(on_stack < a.free_cap ? on_stack : a.free_cap);
  const bool ok = fits && (need == 0 || two.pages <= avail);
  if (real) {
    ask[tid + 1] = two.pages;
    oks[tid] = ok;
    if (ok && need > 0) atomicMax(&s_taken, two.pages);  // requests that get pages come before those that are refused some
  }
  __syncthreads();
  const int taken = s_taken;

  const auto stack = [&](int x) {
    if (x < n_free) return __ldcg(a.free_pages + x);
    const int f = last_at_most(back, a.B, x - n_free);
    return __ldcg(a.table + (size_t)f * a.W + (x - n_free - back[f]));
  };
  const auto handed_out = [&](int y) { return stack(avail - 1 - y); };

  if (blockIdx.x == 0) {
    if (real) {
      a.cu_q[tid + 1] = tok[tid + 1];
      a.new_kv_len[tid] = done ? 0 : (ok ? (int)most : kv);
      a.new_held[tid] = done ? 0 : held + (ok ? need : 0);
    }
    if (tid == 0) {
      a.cu_q[0] = 0;
      a.new_n_free[0] = avail - taken;
    }
  }
  const long long x0 = (long long)blockIdx.x * kPlanThreads + tid, step = (long long)gridDim.x * kPlanThreads;
  for (long long x = x0; x < a.T; x += step) {
    const int i = (int)x;
    int slot = -1, pos = 0;
    if (i < tok[a.B]) {
      const int b = last_at_most(tok, a.B, i);
      const long long at = (long long)kvs[b] + (i - tok[b]);
      pos = at < 0x7fffffffLL ? (int)at : 0x7fffffff;
      if (oks[b]) {
        const int j = pos >> shift;
        const int page = j < helds[b] ? __ldcg(a.table + (size_t)b * a.W + j) : handed_out(ask[b] + j - helds[b]);
        const long long s = ((long long)page << shift) + (pos & (a.P - 1));
        slot = page >= 0 && s <= 0x7fffffffLL ? (int)s : -1;
      }
    }
    a.slots[i] = slot;
    if (a.positions) a.positions[i] = pos;
  }
  for (long long y = x0; y < taken; y += step) {
    const int b = last_at_most(ask, a.B, (int)y);
    a.table[(size_t)b * a.W + helds[b] + ((int)y - ask[b])] = handed_out((int)y);
  }
  for (long long x = n_free + x0; x < on_stack && x < a.free_cap; x += step) a.free_pages[x] = stack((int)x);
}

}  // namespace

cudaError_t launch_page_plan(const PlanArgs& a, cudaStream_t st) {
  int shift = 0;
  while ((1 << shift) < a.P) ++shift;
  // a token a thread; finished requests' pages and new table entries ride along
  long long grid = ((long long)a.T + kPlanThreads - 1) / kPlanThreads;
  if (grid < (a.B + 63) / 64) grid = (a.B + 63) / 64;
  if (grid > sm_count()) grid = sm_count();
  return launch_pdl(page_plan_kernel, dim3((unsigned)grid), dim3(kPlanThreads), 0, st, a, shift);
}

}  // namespace glide
