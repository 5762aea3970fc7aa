// Attention over the 8-bit cache on the CUDA cores, for fp32 queries:
//
//   s[r,t]  = q[r] . code_K[t] * 2^eK[t/64] * scale        (cached rows)
//           = q[r] . k_tree[j] * scale                     (nodes j in A_r)
//   out[r]  = sum_t softmax(s[r])_t value_V[t]
//
// A CTA takes kRT query rows of a slab (the rows that share a cached head) and all its keys; its
// warps take tiles of 32 keys in turn.  Lane = key for the scores (the query comes from shared
// memory, the same address in every lane), lane = slice of the head dimension for the values.
// Running maximum, sum and output are kept per warp and joined at the end.
//
// What bounds it: at small sizes a call is a chain of latencies, a tile after the other in each warp.  Sixteen
// warps with two rows keep it short and still share a tile's keys and values
// (8 warps x 4 rows / 16 x 2 / 16 x 1, us: 5 nodes on 4 heads of 64 dims, 128 keys 6.4 / 6.5 / 6.1; 16 nodes on 2 x 2
// cached heads of 1024 42 / 22 / 23; 32 nodes on 2 x 32 heads of 2048 307 / 251 / 816).  Nothing splits a slab's keys over
// CTAs, so few heads leave most of the GPU idle; the fp32 calls on a cache in fp32 do split them, and take less: 8 nodes
// of 2 query heads to each of 2 x 2 cached of 1024 keys 20 us for 8.9, 32 nodes on 2 x 32 heads of 2048 262 for 164.
#include <math_constants.h>

#include "attn_common.cuh"
#include "common.cuh"
#include "device.h"
#include "kv8.h"

namespace glide {
namespace {

constexpr int kWarps = 16;
constexpr int kThreads = kWarps * 32;
constexpr int kRT = 2;  // query rows of a CTA

// Row tile `unit` of all slabs' tiles.
template <int D>
__device__ __forceinline__ void attend(const Kv8AttnArgs& a, unsigned unit, int tiles) {
  constexpr int kPer = D / 32;  // value elements per lane
  __shared__ __align__(16) float q[kRT][D];
  __shared__ float o_all[kWarps][kRT][D];
  __shared__ float m_all[kWarps][kRT], l_all[kWarps][kRT];
  __shared__ unsigned long long sees[kRT];
  __shared__ int up[64];
  __shared__ int odd_values;  // the tree has values that are not finite
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int group = a.H / a.Hkv, rows = a.nq * group;
  const int slab = (int)(unit / (unsigned)tiles), r0 = (int)(unit - (unsigned)slab * tiles) * kRT;
  const int b = slab / a.Hkv, h = slab - b * a.Hkv;
  int L = a.kv_len[b];
  L = L < 0 ? 0 : (L > a.max_kv_len ? a.max_kv_len : L);
  const float* Q = static_cast<const float*>(a.q);
  for (int i = threadIdx.x; i < kRT * D; i += kThreads) {
    const int r = r0 + i / D;
    q[i / D][i % D] = r < rows ? Q[out_row(b, h, r, rows, group, a.H) * D + i % D] : 0.f;
  }
  const int n = a.parent ? a.nq : 0;
  if (threadIdx.x == 0) odd_values = 0;
  if (threadIdx.x < n) up[threadIdx.x] = a.parent[(size_t)b * n + threadIdx.x];
  __syncthreads();
  if (threadIdx.x < kRT && n) {  // the row's node and its ancestors
    unsigned long long set = 0;
    const int r = r0 + threadIdx.x < rows ? r0 + threadIdx.x : rows - 1;
    for (int j = r / group; j >= 0;) {
      set |= 1ull << j;
      j = up[j] < j ? up[j] : -1;
    }
    sees[threadIdx.x] = set;
  }
  __syncthreads();

  const float c = a.scale * kLog2e;
  float m[kRT], l[kRT], o[kRT][kPer];
#pragma unroll
  for (int r = 0; r < kRT; ++r) {
    m[r] = -CUDART_INF_F;
    l[r] = 0.f;
#pragma unroll
    for (int k = 0; k < kPer; ++k) o[r][k] = 0.f;
  }
  // Folds 32 keys in: s are this lane's scores (log2 domain), `seen` which rows see its key, v
  // the exponent's factor of its value row, value(j, f) this lane's slice of key j's value row.
  auto fold = [&](float (&s)[kRT], unsigned seen, float v, int keys, auto value) {
    float w[kRT];
#pragma unroll
    for (int r = 0; r < kRT; ++r) {
      const bool on = (seen >> r) & 1u;
      const float top = fmaxf(m[r], warp_max(on ? s[r] : -CUDART_INF_F));
      const float ref = top == -CUDART_INF_F ? 0.f : top;  // nothing seen yet, or NaN only
      const float p = on ? fast_exp2(s[r] - ref) : 0.f;
      const float keep = m[r] == -CUDART_INF_F ? (l[r] == 0.f ? 0.f : 1.f) : fast_exp2(m[r] - ref);
      l[r] = l[r] * keep + warp_sum(p);
#pragma unroll
      for (int k = 0; k < kPer; ++k) o[r][k] *= keep;
      m[r] = top;
      w[r] = p * v;
    }
    for (int j = 0; j < keys; ++j) {
      float f[kPer];
      value(j, f);
#pragma unroll
      for (int r = 0; r < kRT; ++r) {
        const float pj = __shfl_sync(0xffffffffu, w[r], j);
#pragma unroll
        for (int k = 0; k < kPer; ++k) o[r][k] = fmaf(pj, f[k], o[r][k]);
      }
    }
  };

  const size_t base = (size_t)slab * a.S_cap;
  const int8_t* Ke = a.Ke + (size_t)slab * kv8_blocks(a.S_cap);
  const int8_t* Ve = a.Ve + (size_t)slab * kv8_blocks(a.S_cap);
  const int cached = (L + 31) / 32, all = cached + (n + 31) / 32;
  for (int tile = warp; tile < all; tile += kWarps) {
    float s[kRT];
#pragma unroll
    for (int r = 0; r < kRT; ++r) s[r] = 0.f;
    if (tile < cached) {
      const int t = tile * 32 + lane, at = t < L ? t : L - 1, keys = L - tile * 32 < 32 ? L - tile * 32 : 32;
      const uint8_t* row = a.K + (base + at) * D;
#pragma unroll 2
      for (int d = 0; d < D; d += 16) {
        const uint4 w = *reinterpret_cast<const uint4*>(row + d);
        float f[16];
        kv8_decode4(w.x, f);
        kv8_decode4(w.y, f + 4);
        kv8_decode4(w.z, f + 8);
        kv8_decode4(w.w, f + 12);
#pragma unroll
        for (int r = 0; r < kRT; ++r)
#pragma unroll
          for (int k = 0; k < 16; ++k) s[r] = fmaf(q[r][d + k], f[k], s[r]);
      }
      const float ks = c * kv8_pow2(kv8_clamp_exp(Ke[at / kKv8Block]));
#pragma unroll
      for (int r = 0; r < kRT; ++r) s[r] *= ks;
      const uint8_t* vrow = a.V + (base + tile * 32) * D + lane * kPer;
      fold(s, t < L ? ~0u : 0u, kv8_pow2(kv8_clamp_exp(Ve[at / kKv8Block])), keys, [&](int j, float* f) {
        if constexpr (kPer == 4) {
          kv8_decode4(*reinterpret_cast<const uint32_t*>(vrow + (size_t)j * D), f);
        } else {
          const float2 v = kv8_f16pair(kv8_decode2_f16(*reinterpret_cast<const uint16_t*>(vrow + (size_t)j * D)));
          f[0] = v.x;
          f[1] = v.y;
        }
      });
    } else {
      const int j0 = (tile - cached) * 32, j = j0 + lane, at = j < n ? j : n - 1;
      const float* row = static_cast<const float*>(a.kt) + (((size_t)b * n + at) * a.Hkv + h) * D;
      for (int d = 0; d < D; ++d) {
        const float k = row[d];
#pragma unroll
        for (int r = 0; r < kRT; ++r) s[r] = fmaf(q[r][d], k, s[r]);
      }
      unsigned seen = 0;
#pragma unroll
      for (int r = 0; r < kRT; ++r) {
        s[r] *= c;
        if (j < n && (sees[r] >> j) & 1ull) seen |= 1u << r;
      }
      const float* vt = static_cast<const float*>(a.vt) + (((size_t)b * n + j0) * a.Hkv + h) * D + lane * kPer;
      fold(s, seen, 1.f, n - j0 < 32 ? n - j0 : 32, [&](int i, float* f) {
#pragma unroll
        for (int k = 0; k < kPer; ++k) {
          f[k] = vt[(size_t)i * a.Hkv * D + k];
          // what is not finite must not meet a weight of zero: it is left out here, and put back at the end where it is seen
          if (!isfinite(f[k])) f[k] = 0.f, odd_values = 1;
        }
      });
    }
  }
#pragma unroll
  for (int r = 0; r < kRT; ++r) {
    if (lane == 0) {
      m_all[warp][r] = m[r];
      l_all[warp][r] = l[r];
    }
#pragma unroll
    for (int k = 0; k < kPer; ++k) o_all[warp][r][lane * kPer + k] = o[r][k];
  }
  __syncthreads();
  float* out = static_cast<float*>(a.out);
  for (int i = threadIdx.x; i < kRT * D; i += kThreads) {
    const int r = i / D, d = i % D;
    if (r0 + r >= rows) break;
    float M = -CUDART_INF_F, sum = 0.f, x = 0.f;
    for (int w = 0; w < kWarps; ++w) M = fmaxf(M, m_all[w][r]);
    for (int w = 0; w < kWarps; ++w) {
      const float f = m_all[w][r] == -CUDART_INF_F ? 1.f : fast_exp2(m_all[w][r] - M);  // -inf: nothing, or NaN
      sum += f * l_all[w][r];
      x += f * o_all[w][r][d];
    }
    if (odd_values)
      for (int j = 0; j < n; ++j) {
        const float v = static_cast<const float*>(a.vt)[(((size_t)b * n + j) * a.Hkv + h) * D + d];
        if (!isfinite(v) && (sees[r] >> j) & 1ull) x += v;
      }
    // no keys at all: zeros; scores of -inf alone: NaN
    out[out_row(b, h, r0 + r, rows, group, a.H) * D + d] = all == 0 ? 0.f : x / sum;
  }
}

template <int D>
__global__ void __launch_bounds__(kThreads, 2) kv8_attn_fma_kernel(const Kv8AttnArgs a) {
  const int tiles = (a.nq * (a.H / a.Hkv) + kRT - 1) / kRT;
  const unsigned units = (unsigned)(a.B * a.Hkv) * (unsigned)tiles;
  pdl_wait();
  for (unsigned unit = blockIdx.x; unit < units; unit += gridDim.x) {  // once, unless the caller bounds the CTAs
    attend<D>(a, unit, tiles);
    if (unit + gridDim.x < units) __syncthreads();  // before its shared memory is written again
  }
}

template <int D>
cudaError_t launch(const Kv8AttnArgs& a, cudaStream_t st) {
  const int rows = a.nq * (a.H / a.Hkv);
  long long ctas = (long long)a.B * a.Hkv * ((rows + kRT - 1) / kRT);
  if (a.max_ctas > 0 && ctas > a.max_ctas) ctas = a.max_ctas;
  return launch_pdl(kv8_attn_fma_kernel<D>, dim3((unsigned)ctas), dim3(kThreads), 0, st, a);
}

}  // namespace

cudaError_t launch_kv8_attn_fma(const Kv8AttnArgs& a, cudaStream_t st) {
  return a.D == 128 ? launch<128>(a, st) : launch<64>(a, st);
}

}  // namespace glide
