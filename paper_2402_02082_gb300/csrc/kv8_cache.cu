// The 8-bit cache's rows: quantising new ones as they are written, and reading rows back.
//
//   e    = least e with max |x| <= 448 * 2^e over the finite new elements of a block of 64 tokens and
//          head, not below the exponent of rows that the block holds already
//   code = x * 2^-e to the nearest 8-bit float
//
// One CTA takes one block of one slab: its new rows stay in registers between the maximum and the
// rounding, so a new element is read once.  Rows from before are read only where their exponent grows.
#include <cuda_runtime.h>
#include <stdint.h>

#include "common.cuh"
#include "device.h"
#include "kv8.h"

namespace glide {
namespace {

constexpr int kThreads = 256;

struct AppendParams {
  uint8_t *K, *V;
  int8_t *Ke, *Ve;
  const void *k_new, *v_new;
  const int32_t *kv_len, *path, *len;
  int32_t* new_kv_len;
  int layers, B, H, S_cap, n, blocks;  // blocks: those that n rows can touch
};

// The least e with amax <= 448 * 2^e, from the bits of a finite amax >= 0: 448 = 1.75 * 2^8.
__device__ __forceinline__ int block_exponent(uint32_t bits) {
  const int e = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0);
  return kv8_clamp_exp(e);  // zero and subnormal numbers too
}

// Eight consecutive elements as fp32.
__device__ __forceinline__ void load8(const __nv_bfloat16* p, float (&f)[8]) {
  const uint4 w = *reinterpret_cast<const uint4*>(p);
  f[0] = bf16lo(w.x); f[1] = bf16hi(w.x); f[2] = bf16lo(w.y); f[3] = bf16hi(w.y);
  f[4] = bf16lo(w.z); f[5] = bf16hi(w.z); f[6] = bf16lo(w.w); f[7] = bf16hi(w.w);
}
__device__ __forceinline__ void load8(const float* p, float (&f)[8]) {
  const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
  f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w;
  f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
}

__device__ __forceinline__ uint2 encode8(const float (&f)[8], float s) {
  uint2 w;
  w.x = kv8_encode2(f[0] * s, f[1] * s) | (kv8_encode2(f[2] * s, f[3] * s) << 16);
  w.y = kv8_encode2(f[4] * s, f[5] * s) | (kv8_encode2(f[6] * s, f[7] * s) << 16);
  return w;
}

// Grid: x = touched block of (layer, b, h), y = K or V.
template <typename T, int D>
__global__ void __launch_bounds__(kThreads) kv8_append_kernel(const AppendParams p) {
  constexpr int kPerRow = D / 8;                       // threads per row
  constexpr int kRows = kThreads / kPerRow;            // rows per pass
  constexpr int kPasses = kKv8Block / kRows;
  __shared__ uint32_t top[kThreads / 32];
  pdl_wait();
  const int slab = (int)(blockIdx.x / (unsigned)p.blocks), nth = (int)(blockIdx.x - (unsigned)slab * p.blocks);
  const int bh = slab % (p.B * p.H), layer = slab / (p.B * p.H);
  const int b = bh / p.H, h = bh - b * p.H;
  int L = p.kv_len[b];
  L = L < 0 ? 0 : (L > p.S_cap - p.n ? p.S_cap - p.n : L);
  int m = p.n;
  if (p.len) {
    m = p.len[b];
    m = (m < -1 ? -1 : (m > p.n - 1 ? p.n - 1 : m)) + 1;
  }
  if (nth == 0 && blockIdx.y == 0 && layer == 0 && h == 0 && threadIdx.x == 0) p.new_kv_len[b] = L + m;
  const int block = L / kKv8Block + nth;
  const int row0 = block * kKv8Block;
  if (m == 0 || row0 >= L + m) return;
  uint8_t* codes = (blockIdx.y ? p.V : p.K) + ((size_t)slab * p.S_cap + row0) * D;
  int8_t* exps = (blockIdx.y ? p.Ve : p.Ke) + (size_t)slab * kv8_blocks(p.S_cap) + block;
  const T* fresh = static_cast<const T*>(blockIdx.y ? p.v_new : p.k_new) + (size_t)layer * p.B * p.n * p.H * D;

  const int r0 = threadIdx.x / kPerRow, d = (threadIdx.x % kPerRow) * 8;
  float x[kPasses][8];
  uint32_t most = 0;
#pragma unroll
  for (int i = 0; i < kPasses; ++i) {
    const int k = row0 + r0 + i * kRows - L;  // new row
#pragma unroll
    for (int j = 0; j < 8; ++j) x[i][j] = 0.f;
    if (k >= 0 && k < m) {
      int src = k;
      if (p.path) {
        src = p.path[(size_t)b * p.n + k];
        src = src < 0 ? 0 : (src > p.n - 1 ? p.n - 1 : src);
      }
      load8(fresh + (((size_t)b * p.n + src) * p.H + h) * D + d, x[i]);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t a = __float_as_uint(x[i][j]) & 0x7fffffffu;
      if (a < 0x7f800000u && a > most) most = a;
    }
  }
  most = __reduce_max_sync(0xffffffffu, most);
  if ((threadIdx.x & 31) == 0) top[threadIdx.x >> 5] = most;
  const int old = row0 < L ? (int)*exps : kKv8ExpMin;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kThreads / 32; ++w) most = top[w] > most ? top[w] : most;
  int e = block_exponent(most);
  if (row0 < L && old >= e) e = kv8_clamp_exp(old);
  if (threadIdx.x == 0) *exps = (int8_t)e;  // every thread has read the old one before the barrier
  const float s = kv8_pow2(-e);
  const bool grown = row0 < L && e > old;
  const float shrink = grown ? kv8_pow2(old - e < -126 ? -126 : old - e) : 1.f;
#pragma unroll
  for (int i = 0; i < kPasses; ++i) {
    const int r = r0 + i * kRows, k = row0 + r - L;
    uint2* at = reinterpret_cast<uint2*>(codes + (size_t)r * D + d);
    if (k >= 0 && k < m) {
      *at = encode8(x[i], s);
    } else if (k < 0 && grown) {
      const uint2 w = *at;
      float f[8];
      kv8_decode4(w.x, f);
      kv8_decode4(w.y, f + 4);
      *at = encode8(f, shrink);
    }
  }
}

template <typename T, int D>
cudaError_t append(const Kv8AppendArgs& a, cudaStream_t st) {
  AppendParams p;
  p.K = a.K; p.V = a.V; p.Ke = a.Ke; p.Ve = a.Ve; p.k_new = a.k_new; p.v_new = a.v_new;
  p.kv_len = a.kv_len; p.path = a.path; p.len = a.len; p.new_kv_len = a.new_kv_len;
  p.layers = a.layers; p.B = a.B; p.H = a.H; p.S_cap = a.S_cap; p.n = a.n;
  p.blocks = (a.n + kKv8Block - 2) / kKv8Block + 1;
  const long long ctas = (long long)p.blocks * a.layers * a.B * a.H;
  if (ctas > 0x7fffffffll) return cudaErrorNotSupported;
  return launch_pdl(kv8_append_kernel<T, D>, dim3((unsigned)ctas, 2), dim3(kThreads), 0, st, p);
}

struct ReadParams {
  const uint8_t *K, *V;
  const int8_t *Ke, *Ve;
  const int32_t* kv_len;
  void *K_out, *V_out;
  long long chunks;  // 16-code pieces of one output tensor
  int B, H, S_cap, S_out;
};

__device__ __forceinline__ void store16(__nv_bfloat16* p, const float (&f)[16]) {
  uint32_t w[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[i]) : "f"(f[2 * i + 1]), "f"(f[2 * i]));
  }
  reinterpret_cast<uint4*>(p)[0] = make_uint4(w[0], w[1], w[2], w[3]);
  reinterpret_cast<uint4*>(p)[1] = make_uint4(w[4], w[5], w[6], w[7]);
}
__device__ __forceinline__ void store16(float* p, const float (&f)[16]) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
    reinterpret_cast<float4*>(p)[i] = make_float4(f[4 * i], f[4 * i + 1], f[4 * i + 2], f[4 * i + 3]);
}

// A thread takes 16 codes at a time.  Grid: y = K or V.
template <typename T, int D>
__global__ void __launch_bounds__(kThreads) kv8_read_kernel(const ReadParams p) {
  constexpr int kPerRow = D / 16;
  pdl_wait();
  const uint8_t* codes = blockIdx.y ? p.V : p.K;
  const int8_t* exps = blockIdx.y ? p.Ve : p.Ke;
  T* out = static_cast<T*>(blockIdx.y ? p.V_out : p.K_out);
  for (long long c = (long long)blockIdx.x * kThreads + threadIdx.x; c < p.chunks; c += (long long)gridDim.x * kThreads) {
    const long long row = c / kPerRow, slab = row / p.S_out;
    const int t = (int)(row - slab * p.S_out), d = (int)(c % kPerRow) * 16;
    const int b = (int)((slab / p.H) % p.B);
    float f[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) f[i] = 0.f;
    if (t < p.kv_len[b]) {
      const uint4 w = *reinterpret_cast<const uint4*>(codes + ((size_t)slab * p.S_cap + t) * D + d);
      const float s = kv8_pow2(kv8_clamp_exp(exps[slab * kv8_blocks(p.S_cap) + t / kKv8Block]));
      kv8_decode4(w.x, f);
      kv8_decode4(w.y, f + 4);
      kv8_decode4(w.z, f + 8);
      kv8_decode4(w.w, f + 12);
#pragma unroll
      for (int i = 0; i < 16; ++i) f[i] *= s;
    }
    store16(out + ((size_t)row * D + d), f);
  }
}

template <typename T, int D>
cudaError_t read(const Kv8ReadArgs& a, cudaStream_t st) {
  ReadParams p;
  p.K = a.K; p.V = a.V; p.Ke = a.Ke; p.Ve = a.Ve; p.kv_len = a.kv_len; p.K_out = a.K_out; p.V_out = a.V_out;
  p.B = a.B; p.H = a.H; p.S_cap = a.S_cap; p.S_out = a.S_out;
  p.chunks = (long long)a.layers * a.B * a.H * a.S_out * (D / 16);
  long long grid = (p.chunks + kThreads - 1) / kThreads;
  const long long cap = (long long)sm_count() * 32;
  if (grid > cap) grid = cap;
  return launch_pdl(kv8_read_kernel<T, D>, dim3((unsigned)grid, 2), dim3(kThreads), 0, st, p);
}

}  // namespace

cudaError_t launch_kv8_append(const Kv8AppendArgs& a, cudaStream_t st) {
  if (a.dtype == 0) return a.D == 128 ? append<__nv_bfloat16, 128>(a, st) : append<__nv_bfloat16, 64>(a, st);
  return a.D == 128 ? append<float, 128>(a, st) : append<float, 64>(a, st);
}

cudaError_t launch_kv8_read(const Kv8ReadArgs& a, cudaStream_t st) {
  if (a.dtype == 0) return a.D == 128 ? read<__nv_bfloat16, 128>(a, st) : read<__nv_bfloat16, 64>(a, st);
  return a.D == 128 ? read<float, 128>(a, st) : read<float, 64>(a, st);
}

}  // namespace glide
