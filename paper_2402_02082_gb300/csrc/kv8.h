// The 8-bit cache: launch interface between the C ABI (abi.cu) and its kernels, and the device
// helpers that they share.
//
// A code is a signed 8-bit float (4 exponent bits, bias 7, 3 mantissa bits; 0x7f and 0xff are NaN,
// there is no infinity); a block of 64 tokens of a cached head shares a power-of-two exponent.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace glide {

constexpr int kKv8Block = 64;     // tokens that share an exponent
constexpr int kKv8MaxRows = 256;  // query rows per cached head (n x H / H_kv)
constexpr int kKv8ExpMin = -117;  // 2^(-117 - 9), the smallest code's value, is a normal bf16 / fp32 number
constexpr int kKv8ExpMax = 119;   // 448 * 2^119 is below the largest finite one

inline __host__ __device__ int kv8_blocks(int rows) { return (rows + kKv8Block - 1) / kKv8Block; }

struct Kv8AppendArgs {
  uint8_t *K, *V;
  int8_t *Ke, *Ve;
  const void *k_new, *v_new;
  const int32_t* kv_len;
  const int32_t* path;  // or null
  const int32_t* len;   // or null
  int32_t* new_kv_len;
  int layers, B, H, D, S_cap, n;  // H: cached heads
  int dtype;                      // 0 bf16, 1 f32
};

struct Kv8ReadArgs {
  const uint8_t *K, *V;
  const int8_t *Ke, *Ve;
  const int32_t* kv_len;
  void *K_out, *V_out;
  int layers, B, H, D, S_cap, S_out;
  int dtype;
};

struct Kv8AttnArgs {
  const void* q;
  const uint8_t *K, *V;
  const int8_t *Ke, *Ve;
  const void *kt, *vt;      // the tree's own keys and values [B, n, Hkv, D], null without a tree
  const int32_t* parent;    // null without a tree
  const int32_t* kv_len;
  void* out;
  void* ws;
  int B, H, Hkv, D, S_cap, nq, max_kv_len;
  int dtype;                // of q, kt, vt and out: 0 bf16, 1 f32
  float scale;
  int max_ctas;
};

cudaError_t launch_kv8_append(const Kv8AppendArgs& a, cudaStream_t st);
cudaError_t launch_kv8_read(const Kv8ReadArgs& a, cudaStream_t st);
// On the tensor cores, bf16 queries; cudaErrorNotSupported for a cache beyond 32-bit coordinates.
cudaError_t launch_kv8_attn_tc(const Kv8AttnArgs& a, cudaStream_t st);
// Few query rows, bf16, straight from global memory to registers; cudaErrorNotSupported where launch_kv8_attn_tc is
// the one to take.
cudaError_t launch_kv8_few(const Kv8AttnArgs& a, cudaStream_t st);
// On the CUDA cores, fp32 throughout.
cudaError_t launch_kv8_attn_fma(const Kv8AttnArgs& a, cudaStream_t st);
size_t kv8_workspace_bytes(int B, int Hkv, int D, int rows);

#ifdef __CUDACC__
__device__ __forceinline__ float kv8_pow2(int e) { return __int_as_float((e + 127) << 23); }  // |e| <= 126
__device__ __forceinline__ int kv8_clamp_exp(int e) {
  return e < kKv8ExpMin ? kKv8ExpMin : (e > kKv8ExpMax ? kKv8ExpMax : e);
}

// Two codes (the first in the low byte) of two fp32 values: nearest, ties to even, the largest code
// beyond it, NaN for NaN.
__device__ __forceinline__ uint32_t kv8_encode2(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
// Two codes to two fp16 values, exactly.
__device__ __forceinline__ uint32_t kv8_decode2_f16(uint32_t two) {
  uint32_t r;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((uint16_t)two));
  return r;
}
__device__ __forceinline__ float2 kv8_f16pair(uint32_t h) {
  float2 f;
  asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tcvt.f32.f16 %0, l;\n\tcvt.f32.f16 %1, h;\n\t}"
      : "=f"(f.x), "=f"(f.y)
      : "r"(h));
  return f;
}
// Four codes (a 32-bit word, the first in the low byte) to fp32.
__device__ __forceinline__ void kv8_decode4(uint32_t w, float* f) {
  const float2 a = kv8_f16pair(kv8_decode2_f16(w & 0xffffu)), b = kv8_f16pair(kv8_decode2_f16(w >> 16));
  f[0] = a.x;
  f[1] = a.y;
  f[2] = b.x;
  f[3] = b.y;
}
#endif

}  // namespace glide
