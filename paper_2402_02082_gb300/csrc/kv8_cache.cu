// The 8-bit cache's rows: quantising new ones as they are written, and reading rows back.
//
//   e    = least e with max |x| <= 448 * 2^e over the finite new elements of a block of 64 tokens and
//          head, not below the exponent of rows that the block holds already
//   code = x * 2^-e to the nearest 8-bit float
//
// What bounds it.  A prompt's rows are a stream (2 or 4 bytes in, 1 out): one CTA takes a block of K or
// of V of one slab, all its loads in flight at once and kept as they came, so a new element is read once
// between the maximum and the rounding.  Instructions weigh beside the bytes (29.6 us): a maximum over packed
// magnitudes instead of over each element's finite value 37.4 -> 32.9 us for 4 x 32 heads of 2048 bf16 rows, 6.1 TB/s
// (fp32: 51.5 us, 6.5 TB/s).  A round's few rows are latency (the lengths, the path, the rows, the exponent, one after
// another): a warp takes a block, so that all layers and heads fit the GPU at once.  Rows from before are read only where their exponent grows.
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

// Eight consecutive elements, as they lie in memory.
template <typename T>
struct Eight;
template <>
struct Eight<__nv_bfloat16> {
  uint4 w;
  __device__ __forceinline__ void none() { w = make_uint4(0u, 0u, 0u, 0u); }
  __device__ __forceinline__ void load(const __nv_bfloat16* p) { w = __ldcs(reinterpret_cast<const uint4*>(p)); }
  __device__ __forceinline__ void get(float (&f)[8]) const {
    f[0] = bf16lo(w.x); f[1] = bf16hi(w.x); f[2] = bf16lo(w.y); f[3] = bf16hi(w.y);
    f[4] = bf16lo(w.z); f[5] = bf16hi(w.z); f[6] = bf16lo(w.w); f[7] = bf16hi(w.w);
  }
};
template <>
struct Eight<float> {
  float4 a, b;
  __device__ __forceinline__ void none() { a = b = make_float4(0.f, 0.f, 0.f, 0.f); }
  __device__ __forceinline__ void load(const float* p) {
    a = __ldcs(reinterpret_cast<const float4*>(p));
    b = __ldcs(reinterpret_cast<const float4*>(p) + 1);
  }
  __device__ __forceinline__ void get(float (&f)[8]) const {
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w;
    f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
  }
};
// The bits of the largest finite magnitude, or of `most`.
template <typename T>
__device__ __forceinline__ uint32_t top8(const Eight<T>& x, uint32_t most) {
  float f[8];
  x.get(f);
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const uint32_t a = __float_as_uint(f[j]) & 0x7fffffffu;
    most = max(most, a < 0x7f800000u ? a : 0u);
  }
  return most;
}

// The bits of the largest magnitude, infinities and NaN among them; bf16: two magnitudes at a time, as integers.
template <int N>
__device__ __forceinline__ uint32_t top_of_all(const Eight<__nv_bfloat16> (&x)[N]) {
  uint32_t most = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    most = __vmaxu2(most, __vmaxu2(x[i].w.x & 0x7fff7fffu, x[i].w.y & 0x7fff7fffu));
    most = __vmaxu2(most, __vmaxu2(x[i].w.z & 0x7fff7fffu, x[i].w.w & 0x7fff7fffu));
  }
  return max(most << 16, most & 0xffff0000u);
}
template <int N>
__device__ __forceinline__ uint32_t top_of_all(const Eight<float> (&x)[N]) {
  uint32_t most = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    float f[8];
    x[i].get(f);
#pragma unroll
    for (int j = 0; j < 8; ++j) most = max(most, __float_as_uint(f[j]) & 0x7fffffffu);
  }
  return most;
}

__device__ __forceinline__ uint2 encode8(const float (&f)[8], float s) {
  uint2 w;
  w.x = kv8_encode2(f[0] * s, f[1] * s) | (kv8_encode2(f[2] * s, f[3] * s) << 16);
  w.y = kv8_encode2(f[4] * s, f[5] * s) | (kv8_encode2(f[6] * s, f[7] * s) << 16);
  return w;
}
template <typename T>
__device__ __forceinline__ uint2 encode8(const Eight<T>& x, float s) {
  float f[8];
  x.get(f);
  return encode8(f, s);
}

// A block's exponent from its new rows' largest magnitude and, if it holds rows, its old exponent (within the range).
__device__ __forceinline__ int joined_exponent(uint32_t most, bool holds, int old) {
  const int e = block_exponent(most);
  return holds && old >= e ? old : e;
}
// What a grown exponent makes of the codes that a block holds.
__device__ __forceinline__ float shrink_by(int old, int e) { return kv8_pow2(old - e < -126 ? -126 : old - e); }
__device__ __forceinline__ uint2 shrink8(const uint2& w, float by) {
  float f[8];
  kv8_decode4(w.x, f);
  kv8_decode4(w.y, f + 4);
  return encode8(f, by);
}

struct Rows {  // of a sequence: its length so far, and how many join (as many as the slab has room for)
  int L, m;
};
__device__ __forceinline__ Rows rows_of(const AppendParams& p, int b) {
  int L = p.kv_len[b], m = p.len ? p.len[b] : p.n - 1;
  L = L < 0 ? 0 : (L > p.S_cap ? p.S_cap : L);
  m = (m < -1 ? -1 : (m > p.n - 1 ? p.n - 1 : m)) + 1;
  m = m > p.S_cap - L ? p.S_cap - L : m;
  return {L, m};
}
// Where element 0 of new row k of (layer, b, h) lies in k_new / v_new.
__device__ __forceinline__ size_t row_at(const AppendParams& p, int layer, int b, int h, int k, int D) {
  int src = k;
  if (p.path) {
    src = p.path[(size_t)b * p.n + k];
    src = src < 0 ? 0 : (src > p.n - 1 ? p.n - 1 : src);
  }
  return ((((size_t)layer * p.B + b) * p.n + src) * p.H + h) * D;
}

// A CTA takes a touched block of (layer, b, h), of K (blockIdx.y = 0) or of V.
constexpr int kAppendThreads = 128;
template <typename T, int D>
__global__ void __launch_bounds__(kAppendThreads, sizeof(T) == 2 ? 8 : 5) kv8_append_kernel(const AppendParams p) {
  constexpr int kPerRow = D / 8;                   // threads per row
  constexpr int kRows = kAppendThreads / kPerRow;  // rows per pass
  constexpr int kPasses = kKv8Block / kRows;
  constexpr int kW = kAppendThreads / 32;
  __shared__ uint32_t top[2][kW];
  pdl_wait();
  // heads first: CTAs that run together then read whole tokens' rows
  const int bn = (int)(blockIdx.x / (unsigned)p.H), h = (int)(blockIdx.x - (unsigned)bn * p.H);
  const int lb = bn / p.blocks, nth = bn - lb * p.blocks;
  const int layer = lb / p.B, b = lb - layer * p.B, slab = lb * p.H + h;
  const bool is_v = blockIdx.y != 0;
  const Rows r = rows_of(p, b);
  if (!is_v && nth == 0 && layer == 0 && h == 0 && threadIdx.x == 0) p.new_kv_len[b] = r.L + r.m;
  const int block = r.L / kKv8Block + nth, row0 = block * kKv8Block;
  if (r.m == 0 || row0 >= r.L + r.m) return;
  int8_t* const exp = (is_v ? p.Ve : p.Ke) + (size_t)slab * kv8_blocks(p.S_cap) + block;
  const T* const fresh = static_cast<const T*>(is_v ? p.v_new : p.k_new);
  const int rt = threadIdx.x / kPerRow, d = (threadIdx.x % kPerRow) * 8;
  const bool holds = row0 < r.L;
  Eight<T> x[kPasses];
#pragma unroll
  for (int i = 0; i < kPasses; ++i) {
    const int k = row0 + rt + i * kRows - r.L;  // new row
    x[i].none();
    if (k >= 0 && k < r.m) x[i].load(fresh + row_at(p, layer, b, h, k, D) + d);
  }
  const int old_raw = holds ? (int)*exp : 0;
  auto joined = [&](uint32_t mine, int nth) {  // over the CTA
    mine = __reduce_max_sync(0xffffffffu, mine);
    if ((threadIdx.x & 31) == 0) top[nth][threadIdx.x >> 5] = mine;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kW; ++w) mine = max(mine, top[nth][w]);
    return mine;
  };
  uint32_t most = joined(top_of_all(x), 0);
  if (most >= 0x7f800000u) {  // the finite elements decide; looking at each costs too much where all are
    most = 0;
#pragma unroll
    for (int i = 0; i < kPasses; ++i) most = top8(x[i], most);
    most = joined(most, 1);
  }
  const int old = kv8_clamp_exp(old_raw), e = joined_exponent(most, holds, old);
  if (threadIdx.x == 0) *exp = (int8_t)e;  // every thread has read the old one
  const float s = kv8_pow2(-e);
  uint8_t* const codes = (is_v ? p.V : p.K) + ((size_t)slab * p.S_cap + row0) * D + d;
#pragma unroll
  for (int i = 0; i < kPasses; ++i) {
    const int row = rt + i * kRows, k = row0 + row - r.L;
    uint2* at = reinterpret_cast<uint2*>(codes + (size_t)row * D);
    if (k >= 0 && k < r.m)
      *at = encode8(x[i], s);
    else if (k < 0 && holds && e > old)
      *at = shrink8(*at, shrink_by(old, e));
  }
}

// A warp takes a touched block of (layer, b, h), of K or of V: up to 64 new rows.
template <typename T, int D>
__global__ void __launch_bounds__(kThreads) kv8_append_few_kernel(const AppendParams p) {
  constexpr int kPerRow = D / 8, kRows = 32 / kPerRow;  // lanes per row, rows per load
  constexpr int kHeld = 8;                              // loads whose rows stay in registers
  pdl_wait();
  const int lane = threadIdx.x & 31;
  const long long units = 2ll * p.blocks * p.layers * p.B * p.H;
  const long long unit = ((long long)blockIdx.x * kThreads + threadIdx.x) >> 5;
  if (unit >= units) return;
  const int kv = (int)(unit & 1), nth = (int)((unit >> 1) % p.blocks);
  const int slab = (int)((unit >> 1) / p.blocks);
  const int bh = slab % (p.B * p.H), layer = slab / (p.B * p.H);
  const int b = bh / p.H, h = bh - b * p.H;
  const Rows r = rows_of(p, b);
  if (kv == 0 && nth == 0 && layer == 0 && h == 0 && lane == 0) p.new_kv_len[b] = r.L + r.m;
  const int block = r.L / kKv8Block + nth, row0 = block * kKv8Block;
  if (r.m == 0 || row0 >= r.L + r.m) return;
  uint8_t* codes = (kv ? p.V : p.K) + ((size_t)slab * p.S_cap + row0) * D;
  int8_t* exp = (kv ? p.Ve : p.Ke) + (size_t)slab * kv8_blocks(p.S_cap) + block;
  const T* fresh = static_cast<const T*>(kv ? p.v_new : p.k_new);
  const bool holds = row0 < r.L;
  const int old_raw = holds ? (int)*exp : 0;
  // rows first .. last - 1 of the block are new
  const int first = holds ? r.L - row0 : 0, last = min(kKv8Block, r.L + r.m - row0);
  const int rl = lane / kPerRow, d = (lane % kPerRow) * 8;
  auto load = [&](int row) {
    Eight<T> x;
    x.none();
    if (row < last) x.load(fresh + row_at(p, layer, b, h, row0 + row - r.L, D) + d);
    return x;
  };
  Eight<T> x[kHeld];
  uint32_t most = 0;
#pragma unroll
  for (int i = 0; i < kHeld; ++i) x[i] = load(first + rl + i * kRows);
#pragma unroll
  for (int i = 0; i < kHeld; ++i) most = top8(x[i], most);
  for (int row = first + rl + kHeld * kRows; row < last; row += kRows) most = top8(load(row), most);
  most = __reduce_max_sync(0xffffffffu, most);
  const int old = kv8_clamp_exp(old_raw), e = joined_exponent(most, holds, old);
  __syncwarp();
  if (lane == 0) *exp = (int8_t)e;  // every lane has read the old one
  const float s = kv8_pow2(-e);
#pragma unroll
  for (int i = 0; i < kHeld; ++i) {
    const int row = first + rl + i * kRows;
    if (row < last) *reinterpret_cast<uint2*>(codes + (size_t)row * D + d) = encode8(x[i], s);
  }
  for (int row = first + rl + kHeld * kRows; row < last; row += kRows)
    *reinterpret_cast<uint2*>(codes + (size_t)row * D + d) = encode8(load(row), s);
  if (holds && e > old) {
    const float by = shrink_by(old, e);
    for (int row = rl; row < first; row += kRows) {
      uint2* at = reinterpret_cast<uint2*>(codes + (size_t)row * D + d);
      *at = shrink8(*at, by);
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
  const long long blocks = (long long)p.blocks * a.layers * a.B * a.H;
  if (blocks > 0x7fffffffll) return cudaErrorNotSupported;
  // A CTA a block streams; few rows leave most of it idle (5 rows of 33 nodes, 32 layers of 32 heads: 9.6 us, a warp a
  // block 5.5).
  if (a.n <= kKv8Block) {
    const long long ctas = (2 * blocks * 32 + kThreads - 1) / kThreads;
    return launch_pdl(kv8_append_few_kernel<T, D>, dim3((unsigned)ctas), dim3(kThreads), 0, st, p);
  }
  return launch_pdl(kv8_append_kernel<T, D>, dim3((unsigned)blocks, 2), dim3(kAppendThreads), 0, st, p);
}

struct ReadParams {
  const uint8_t *K, *V;
  const int8_t *Ke, *Ve;
  const int32_t* kv_len;
  void *K_out, *V_out;
  int B, H, S_cap, S_out, parts;  // parts: CTAs of a slab
};

__device__ __forceinline__ void store8(__nv_bfloat16* p, const float (&f)[8]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[i]) : "f"(f[2 * i + 1]), "f"(f[2 * i]));
  __stcs(reinterpret_cast<uint4*>(p), make_uint4(w[0], w[1], w[2], w[3]));
}
__device__ __forceinline__ void store8(float* p, const float (&f)[8]) {
  __stcs(reinterpret_cast<float4*>(p), make_float4(f[0], f[1], f[2], f[3]));
  __stcs(reinterpret_cast<float4*>(p) + 1, make_float4(f[4], f[5], f[6], f[7]));
}

// A stream: 1 byte in, 2 or 4 out.  A CTA takes kPieces x 256 pieces of 8 codes of one slab, a thread kPieces of them,
// loaded before any is used (32 heads of 2048 tokens: 1 piece 12.9 us, 2 9.6, 4 9.0, 8 9.1; 4 x 8 heads of 16384:
// 89, 60.5, 59.1, 59.4, of which the bytes are 59; fp32 19.7 and 117.5, bytes 12.3 and 98.7).  Grid: x = part of a slab, y = K or V.
constexpr int kPieces = 4;
template <typename T, int D>
__global__ void __launch_bounds__(kThreads) kv8_read_kernel(const ReadParams p) {
  constexpr int kPerRow = D / 8;
  pdl_wait();
  const int slab = (int)(blockIdx.x / (unsigned)p.parts), part = (int)(blockIdx.x - (unsigned)slab * p.parts);
  const int L = p.kv_len[slab / p.H % p.B];
  const uint8_t* codes = (blockIdx.y ? p.V : p.K) + (size_t)slab * p.S_cap * D;
  const int8_t* exps = (blockIdx.y ? p.Ve : p.Ke) + (size_t)slab * kv8_blocks(p.S_cap);
  T* out = static_cast<T*>(blockIdx.y ? p.V_out : p.K_out) + (size_t)slab * p.S_out * D;
  const int d = (int)(threadIdx.x % kPerRow) * 8, row = part * (kPieces * kThreads / kPerRow) + threadIdx.x / kPerRow;
  uint2 w[kPieces];
  int e[kPieces];
#pragma unroll
  for (int i = 0; i < kPieces; ++i) {
    const int t = row + i * (kThreads / kPerRow);
    w[i] = make_uint2(0u, 0u);
    e[i] = 0;
    if (t < L && t < p.S_out) {
      w[i] = __ldcs(reinterpret_cast<const uint2*>(codes + (size_t)t * D + d));
      e[i] = exps[t / kKv8Block];
    }
  }
#pragma unroll
  for (int i = 0; i < kPieces; ++i) {
    const int t = row + i * (kThreads / kPerRow);
    if (t >= p.S_out) break;
    const float s = kv8_pow2(kv8_clamp_exp(e[i]));
    float f[8];
    kv8_decode4(w[i].x, f);
    kv8_decode4(w[i].y, f + 4);
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] *= s;
    store8(out + (size_t)t * D + d, f);
  }
}

template <typename T, int D>
cudaError_t read(const Kv8ReadArgs& a, cudaStream_t st) {
  constexpr int kRowsOfCta = kPieces * kThreads * 8 / D;
  ReadParams p;
  p.K = a.K; p.V = a.V; p.Ke = a.Ke; p.Ve = a.Ve; p.kv_len = a.kv_len; p.K_out = a.K_out; p.V_out = a.V_out;
  p.B = a.B; p.H = a.H; p.S_cap = a.S_cap; p.S_out = a.S_out;
  p.parts = (a.S_out + kRowsOfCta - 1) / kRowsOfCta;
  const long long ctas = (long long)p.parts * a.layers * a.B * a.H;
  if (ctas > 0x7fffffffll) return cudaErrorNotSupported;
  return launch_pdl(kv8_read_kernel<T, D>, dim3((unsigned)ctas, 2), dim3(kThreads), 0, st, p);
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
