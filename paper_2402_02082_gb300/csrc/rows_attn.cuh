// One row of attention over a paged cache or packed keys and values, by a warp on the CUDA cores:
// the whole of the simple kernel, and what the tensor-core kernels turn to for a row whose result is
// not finite.
//
// The mathematics: u_t = (q . k_t) scale log2(e), m the running maximum of u, p_t = 2^(u_t - m),
// out = sum p_t v_t / sum p_t, in fp32.  Lane t of a pass takes key t: its dot product needs no exchange;
// for the values lane d takes D / 32 columns.
//
// Two forms.  The plain sums (attend_keys) hold for results that are finite.  They are not finite where a value is
// infinite or NaN (a weight of 0 makes NaN of it), or where a sum passes the type's range although the mean does not.  Then the row
// is computed again by the definition (attend_row): values that are not finite decide their column at any weight but that of
// a score of -inf and are summed apart, the others have their true weight, which may be 0, and are held as the mean so far, which
// never passes its largest term.  A weight below 2^-126 of the largest counts as 0 in both.
#pragma once

#include <cfloat>
#include <cuda_bf16.h>
#include <math_constants.h>

#include "attn_common.cuh"
#include "common.cuh"
#include "paged.h"

namespace glide {
namespace {

struct RowsParams {
  const unsigned char *q, *K, *V;
  unsigned char* out;
  const int *cu, *kv_len, *table;
  long long q_stride, k_stride, v_stride;  // bytes from token to token
  int B, T, H, Hkv, group, W, n_pages, page_shift;
  int max_q, max_kv;
  float scale_log2;
};

__host__ inline RowsParams rows_params(const RowsArgs& a) {
  const int size = a.dtype == 0 ? 2 : 4;
  RowsParams p;
  p.q = static_cast<const unsigned char*>(a.q);
  p.K = static_cast<const unsigned char*>(a.K);
  p.V = static_cast<const unsigned char*>(a.V);
  p.out = static_cast<unsigned char*>(a.out);
  p.cu = a.cu; p.kv_len = a.kv_len; p.table = a.table;
  p.q_stride = a.q_stride * size; p.k_stride = a.k_stride * size; p.v_stride = a.v_stride * size;
  p.B = a.B; p.T = a.T; p.H = a.H; p.Hkv = a.Hkv; p.group = a.H / a.Hkv;
  p.W = a.W; p.n_pages = a.n_pages; p.page_shift = a.page_shift;
  p.max_q = a.max_q; p.max_kv = a.max_kv;
  p.scale_log2 = a.scale * kLog2e;
  return p;
}

__device__ __forceinline__ int clamp_to(int x, int lo, int hi) { return x < lo ? lo : (x > hi ? hi : x); }

// Sequence b's rows and keys: its first row, how many of its rows are served, its rows in all and its keys.
struct Seq {
  int row0, rows, m, kv;
};
__device__ __forceinline__ Seq seq_of(const RowsParams& p, int b) {
  Seq s;
  s.row0 = clamp_to(__ldcg(p.cu + b), 0, p.T);
  s.m = clamp_to(__ldcg(p.cu + b + 1), s.row0, p.T) - s.row0;
  s.rows = s.m < p.max_q ? s.m : p.max_q;
  s.kv = p.table ? clamp_to(__ldcg(p.kv_len + b), 0, p.max_kv) : s.m;
  return s;
}
// Keys that row i of the sequence sees.
__device__ __forceinline__ int seen(const Seq& s, int i) {
  const int n = s.kv - s.m + i + 1;
  return n < 0 ? 0 : n;
}
// The page that holds a request's tokens from page index j on.
__device__ __forceinline__ int page_at(const RowsParams& p, int b, int j) {
  return clamp_to(__ldcg(p.table + (size_t)b * p.W + j), 0, p.n_pages - 1);
}

// Byte offset of key row t of cached head h of sequence b (row0 its first packed row), and of its value row.
template <int kRow>
__device__ __forceinline__ size_t key_at(const RowsParams& p, int b, int row0, int h, int t, long long stride) {
  if (!p.table) return (size_t)((long long)(row0 + t) * stride) + (size_t)h * kRow;
  const int page = page_at(p, b, t >> p.page_shift), r = t & ((1 << p.page_shift) - 1);
  return ((((size_t)page * p.Hkv + h) << p.page_shift) + r) * kRow;
}

// The softmax of some of a row's keys: (max, sum, columns lane * (D / 32) .. of the weighted values).
template <int D>
struct RowPart {
  float m, l, o[D / 32];
};

template <int D>
__device__ __forceinline__ RowPart<D> no_keys() {
  RowPart<D> r;
  r.m = -CUDART_INF_F;
  r.l = 0.f;
#pragma unroll
  for (int e = 0; e < D / 32; ++e) r.o[e] = 0.f;
  return r;
}

// u of key t < n for the query at `q`, cached head hk of sequence b; v_at: where its value is.  kAtOnce: 16-byte pieces loaded at once.
template <typename T, int D, int kAtOnce>
__device__ __forceinline__ float key_score(const RowsParams& p, int b, const Seq& s, int hk, const unsigned char* q, unsigned t,
                                           size_t& v_at) {
  constexpr int kRow = D * (int)sizeof(T), kC = 16 / (int)sizeof(T);
  const unsigned char* k = p.K + key_at<kRow>(p, b, s.row0, hk, (int)t, p.k_stride);
  v_at = key_at<kRow>(p, b, s.row0, hk, (int)t, p.v_stride);
  float acc[2] = {0.f, 0.f};
#pragma unroll kAtOnce
  for (int c = 0; c < D / kC; ++c)
    dot_chunk<T>(*reinterpret_cast<const uint4*>(q + 16 * c), *reinterpret_cast<const uint4*>(k + 16 * c), acc);
  return (acc[0] + acc[1]) * p.scale_log2;
}

// Query head h in row `row0 + i` (row i of sequence b) over its keys first .. first + 31, first + step .., below n > 0.  All
// lanes of a warp.  kAtOnce: loads in flight.  Keys are counted without a sign: n may be 2^31 - 1, and the count passes it by a
// step.
template <typename T, int D>
__device__ __forceinline__ void attend_keys(const RowsParams& p, int b, const Seq& s, int i, int h, unsigned n, unsigned first,
                                            unsigned step, RowPart<D>& r) {
  constexpr int kE = D / 32, kRow = D * (int)sizeof(T), kAtOnce = 8;  // keys whose values are loaded at once
  const int lane = threadIdx.x & 31, hk = h / p.group;
  const unsigned char* q = p.q + (long long)(s.row0 + i) * p.q_stride + (size_t)h * kRow;
#pragma unroll 1
  for (unsigned t0 = first; t0 < n; t0 += step) {
    const unsigned t = t0 + lane;
    float u = -CUDART_INF_F;
    size_t v_at = 0;  // of key t
    if (t < n) u = key_score<T, D, 16>(p, b, s, hk, q, t, v_at);
    const float m_new = fmaxf(r.m, warp_max(u));
    const float m_eff = m_new == -CUDART_INF_F ? 0.f : m_new;
    const float f = fast_exp2(r.m - m_eff), w = fast_exp2(u - m_eff);
    r.l = r.l * f + warp_sum(w);
#pragma unroll
    for (int e = 0; e < kE; ++e) r.o[e] *= f;
    r.m = m_new;
    const int most = n - t0 < 32 ? (int)(n - t0) : 32;
#pragma unroll 1
    for (int j0 = 0; j0 < most; j0 += kAtOnce) {
      float v[kAtOnce][kE];
#pragma unroll
      for (int j = 0; j < kAtOnce; ++j) {
        const size_t at = __shfl_sync(0xffffffffu, v_at, (j0 + j) & 31);
        if (j0 + j < most) load_row_chunk<T, kE>(reinterpret_cast<const T*>(p.V + at) + lane * kE, v[j]);
      }
#pragma unroll
      for (int j = 0; j < kAtOnce; ++j) {
        const float pj = __shfl_sync(0xffffffffu, w, (j0 + j) & 31);
        if (j0 + j >= most) continue;
#pragma unroll
        for (int e = 0; e < kE; ++e) r.o[e] = fmaf(pj, v[j][e], r.o[e]);
      }
    }
  }
}

// The whole row by one warp and the definition: o[e], column lane * (D / 32) + e of the result over the first n > 0 keys.  Called
// where the plain sums are not finite.  step(): once for every 32 keys.  (Inlined: a kernel that splits its registers among its
// warps holds no call.)
struct NoStep {
  __device__ __forceinline__ void operator()() const {}
};
template <typename T, int D, class Step = NoStep>
__device__ __forceinline__ void attend_row(const RowsParams& p, int b, const Seq& s, int i, int h, unsigned n, float (&o)[D / 32],
                                           Step step = {}) {
  constexpr int kE = D / 32, kRow = D * (int)sizeof(T), kAtOnce = 4;
  const int lane = threadIdx.x & 31, hk = h / p.group;
  const unsigned char* q = p.q + (long long)(s.row0 + i) * p.q_stride + (size_t)h * kRow;
  float m = -CUDART_INF_F, l = 0.f, bad[kE];  // bad: the sum of values that are not finite
#pragma unroll
  for (int e = 0; e < kE; ++e) o[e] = bad[e] = 0.f;  // o: half of the mean so far, so that its terms' rounding stays in range too
#pragma unroll 1
  for (unsigned t0 = 0; t0 < n; t0 += 32) {
    step();
    float u = -CUDART_INF_F;
    size_t v_at = 0;
    if (t0 + lane < n) u = key_score<T, D, kAtOnce>(p, b, s, hk, q, t0 + lane, v_at);
    const float m_new = fmaxf(m, warp_max(u));
    const float m_eff = m_new == -CUDART_INF_F ? 0.f : m_new;
    const float before = l * fast_exp2(m - m_eff);
    float w = fast_exp2(u - m_eff);
    l = before + warp_sum(w);  // NaN from the first score that is NaN or +inf on
    const float inv = l > 0.f ? 1.f / l : 0.f, keep = before * inv;
    w *= 0.5f * inv;
    m = m_new;
#pragma unroll
    for (int e = 0; e < kE; ++e) o[e] *= keep;
    const unsigned weighs = __ballot_sync(0xffffffffu, u != -CUDART_INF_F);
    const int most = n - t0 < 32 ? (int)(n - t0) : 32;
#pragma unroll 1
    for (int j0 = 0; j0 < most; j0 += kAtOnce) {
      float v[kAtOnce][kE];
#pragma unroll
      for (int j = 0; j < kAtOnce; ++j) {
        const size_t at = __shfl_sync(0xffffffffu, v_at, (j0 + j) & 31);
        if (j0 + j < most) load_row_chunk<T, kE>(reinterpret_cast<const T*>(p.V + at) + lane * kE, v[j]);
      }
#pragma unroll
      for (int j = 0; j < kAtOnce; ++j) {
        const float pj = __shfl_sync(0xffffffffu, w, (j0 + j) & 31);
        if (j0 + j >= most || !((weighs >> (j0 + j)) & 1u)) continue;
#pragma unroll
        for (int e = 0; e < kE; ++e) {
          const bool finite = fabsf(v[j][e]) <= FLT_MAX;
          o[e] = fmaf(pj, finite ? v[j][e] : 0.f, o[e]);
          bad[e] += finite ? 0.f : v[j][e];
        }
      }
    }
  }
#pragma unroll
  for (int e = 0; e < kE; ++e) {
    const float mean = fmaxf(-FLT_MAX, fminf(2.f * o[e], FLT_MAX));
    o[e] = l > 0.f ? (bad[e] == 0.f ? mean : bad[e]) : CUDART_NAN_F;
  }
}

__device__ __forceinline__ void store_one(float* at, float v) { *at = v; }
__device__ __forceinline__ void store_one(__nv_bfloat16* at, float v) { *at = __float2bfloat16_rn(v); }
template <int kE>
__device__ __forceinline__ void store_row(float* at, const float (&o)[kE]) {
#pragma unroll
  for (int e = 0; e < kE; e += 2) *reinterpret_cast<float2*>(at + e) = make_float2(o[e], o[e + 1]);
}
template <int kE>
__device__ __forceinline__ void store_row(__nv_bfloat16* at, const float (&o)[kE]) {
#pragma unroll
  for (int e = 0; e < kE; e += 2)
    *reinterpret_cast<__nv_bfloat162*>(at + e) = __floats2bfloat162_rn(o[e], o[e + 1]);
}

}  // namespace
}  // namespace glide
