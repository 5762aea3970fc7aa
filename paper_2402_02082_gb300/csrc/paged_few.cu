// Attention over a paged cache for few new tokens (decoding steps, short chain proposals), straight from global memory
// to registers.
//
// What bounds it.  A cached row is read once for at most 16 query rows (new tokens x H / H_kv), so HBM bounds long
// caches and the fixed parts of a call bound short ones.  A cluster of C CTAs serves a slab (a request's cached head and the
// queries that read it) and its 8 C warps take the 16-key tiles in turn: a tile lies in one page, whose number a warp
// loads two tiles ahead; a tile's 8 KB go to registers, the next keys while the warp works on this tile's values.  No
// ring, no barrier until the end; the warps' partial results meet in shared memory, the CTAs' in distributed shared memory, in
// a fixed order.  Clusters start with the longest requests, so that the SMs end together.
// Measured (D = 128, us): 32 requests of 1024 to 16384 keys, 32 heads over 8 cached, 148 to 151 (6.8 TB/s and more, as a copy); six
// new tokens of four requests of 16384, 52 heads, 259 to 268; one request of 2048, 32 heads, 9.9 (33.6 MB, 5 at that rate: the
// launch, the lengths and page numbers, the first loads and the merge, one after another).  9 to 16 rows (one CTA an SM): four new
// tokens of eight requests of 8192, 32 heads over 8, 59.5 (268 MB, 40 at that rate); one token of them, pages of 256, 45.5.  A bound of
// 131072 keys for any of these: no slower.
//
// The mathematics: u = (q . k) scale log2(e), p = 2^(u - m) with m a running maximum, out = sum p v / sum p.  The
// products are warp-level bf16 ones with fp32 sums, keys (and value columns) their 16 rows and queries their 8 columns;
// a weight is rounded to bf16 for the second.  A product's K index may be any permutation that both operands share, so
// a lane's fragments are 16-byte pieces of a row, and the lanes of a load instruction read whole 32-byte sectors:
//   S^T (16 keys x 8 queries): lane (g, t) reads pieces t, t + 4, .. of keys g, g + 8, and of query g
//   O^T (16 dims x 8 queries): lane (g, t) reads pieces g, g + 8 of keys 2t, 2t + 1, 2t + 8, 2t + 9
// The weights of S^T become the second product's operand by a transpose of 8 x 8 within the warp.
// The reference maximum is raised only where a tile's exceeds it by more than 8, so O is seldom rescaled.  The tensor cores' sums lose
// what lies 2^-25 below O with every product, so a warp's O takes in 2^17 keys and then joins fp32 sums in shared memory (the
// mean of 2^24 keys of like weight, a CTA a slab, relative error: -5e-3 without, -1e-4 with it).
//
// A result that is not finite (an infinity or NaN among the values that the row sees, or one that it does not see, in a tile that it
// shares; or an overflow) is computed again by the definition, the row alone, unless its sum of weights is 0 or NaN, which makes
// it NaN.
#include <cuda_bf16.h>
#include <math_constants.h>

#include "device.h"
#include "kernels.h"
#include "rows_attn.cuh"
#include "tc_attn.cuh"

namespace glide {
namespace {

constexpr int kFewWarps = 8;
constexpr int kFewThreads = kFewWarps * 32;
constexpr int kFewKeys = 16;  // keys of a tile: no page is smaller
constexpr int kMaxC = 8;
constexpr unsigned kSpanTiles = 8192;  // tiles of a warp that one O takes in (2^17 keys)
constexpr float kRaise = 8.f;  // log2 of how far a weight may exceed 1

__device__ __forceinline__ void mma_bf16_16x8(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transposed8(uint32_t x) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
  return r;
}
__device__ __forceinline__ void store_pair(float2* at, uint32_t rank, float2 v) {
  uint32_t a;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_u32(at)), "r"(rank));
  asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(a), "f"(v.x), "f"(v.y) : "memory");
}

template <int D, int NT>
struct FewSmem {
  static constexpr int kR = 8 * NT;       // query rows
  static constexpr int kStride = D + 4;   // floats of a partial row: the lanes' stores meet no bank twice
  float red[kFewWarps * kR * kStride];
  float2 stat[kFewWarps * kR];            // (m, l) of each warp
  float2 peer_ml[kMaxC * kR];             // from the cluster's CTAs
  float2 peer_o[kR * D / 2 + kMaxC];      // this CTA's pairs of columns, from each
  uint2 qf[NT * (D / 16) * 32];           // the queries' fragments
  int odd[kR];                            // the row has to be computed again
  int slab_b;
};

template <int D, int NT>
__global__ void __launch_bounds__(kFewThreads, NT == 1 ? 2 : 1) paged_few_kernel(const RowsParams p, int C, int sorted) {
  using M = FewSmem<D, NT>;
  constexpr int kR = M::kR, kStride = M::kStride;
  constexpr int kSteps = D / 16;        // products of S along D, and of O
  constexpr int kPK = D / 32;           // pieces of a key row that a lane reads
  constexpr int kPV = D / 64;           // of a value row
  extern __shared__ unsigned char smem_raw[];
  M& sm = *reinterpret_cast<M*>(smem_raw);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int rank = (int)cluster_rank();
  const int slab = blockIdx.x / C, h = slab % p.Hkv;
  int b = slab / p.Hkv;
  cluster_arrive();  // that every peer's shared memory is there is known when it is written to
  pdl_wait();
  if (sorted) {  // the request of this rank by length, the longest first; B <= the block's threads
    int* len = reinterpret_cast<int*>(sm.red);
    const int mine = threadIdx.x < p.B ? clamp_to(__ldcg(p.kv_len + threadIdx.x), 0, p.max_kv) : 0;
    if (threadIdx.x < p.B) len[threadIdx.x] = mine;
    __syncthreads();
    if (threadIdx.x < p.B) {
      int before = 0;
      for (int x = 0; x < p.B; ++x) before += len[x] > mine || (len[x] == mine && x < threadIdx.x);
      if (before == b) sm.slab_b = threadIdx.x;
    }
    __syncthreads();
    b = sm.slab_b;
  }
  // (keys are counted without a sign: there may be 2^31 - 1 of them, and the count passes that by two steps)
  const unsigned step = C * kFewWarps * kFewKeys;
  unsigned key0 = (rank * kFewWarps + warp) * kFewKeys;
  // (by the bound of the lengths, so that the first numbers are on their way beside the length)
  const auto page_of = [&](unsigned key0) { return key0 < (unsigned)p.max_kv ? page_at(p, b, (int)(key0 >> p.page_shift)) : 0; };
  int page = page_of(key0), page_next = page_of(key0 + step);
  const Seq s = seq_of(p, b);
  const int rows = s.rows * p.group < kR ? s.rows * p.group : kR;
  const unsigned n = rows > 0 ? seen(s, s.rows - 1) : 0;  // keys that some row sees
  const uint64_t pol = policy_evict_first();

  // this lane's pieces of a tile; keys that no row sees are zeros (the pool may hold anything there)
  uint4 kr[2][kPK], vr[4][kPV];
  const auto row_of = [&](const unsigned char* base, int page, unsigned key) {
    return base + ((((size_t)page * p.Hkv + h) << p.page_shift) + (key & ((1 << p.page_shift) - 1))) * (2 * D);
  };
  const auto load_k = [&](int page, unsigned key0) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const unsigned key = key0 + g + 8 * i;
      const unsigned char* at = row_of(p.K, page, key) + 16 * t;
#pragma unroll
      for (int c = 0; c < kPK; ++c) {
        kr[i][c] = make_uint4(0u, 0u, 0u, 0u);
        if (key < n) kr[i][c] = load_once(at + 64 * c, pol);
      }
    }
  };
  const auto load_v = [&](int page, unsigned key0) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const unsigned key = key0 + 8 * (i >> 1) + 2 * t + (i & 1);
      const unsigned char* at = row_of(p.V, page, key) + 16 * g;
#pragma unroll
      for (int c = 0; c < kPV; ++c) {
        vr[i][c] = make_uint4(0u, 0u, 0u, 0u);
        if (key < n) vr[i][c] = load_once(at + 128 * c, pol);
      }
    }
  };
  load_k(page, key0);

  if (warp < NT) {  // the queries' fragments, by a warp for 8 of them
    const int r = 8 * warp + g, i = r / p.group;
    const unsigned char* at = p.q + (long long)(s.row0 + i) * p.q_stride + (size_t)(h * p.group + r - i * p.group) * (2 * D);
#pragma unroll
    for (int c = 0; c < kPK; ++c) {
      uint4 x = make_uint4(0u, 0u, 0u, 0u);
      if (r < rows) x = *reinterpret_cast<const uint4*>(at + 16 * t + 64 * c);
      sm.qf[(warp * kSteps + 2 * c) * 32 + lane] = make_uint2(x.x, x.y);
      sm.qf[(warp * kSteps + 2 * c + 1) * 32 + lane] = make_uint2(x.z, x.w);
    }
  }
  unsigned vis[NT][2];  // keys that rows 2t, 2t + 1 see
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const int r = 8 * nt + 2 * t + x;
      vis[nt][x] = r < rows ? seen(s, r / p.group) : 0;
    }
  const unsigned all_see = rows > 0 ? seen(s, 0) : 0;
  __syncthreads();

  float m[NT][2], l[NT][2], o[kSteps][NT][4];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    m[nt][0] = m[nt][1] = -CUDART_INF_F;
    l[nt][0] = l[nt][1] = 0.f;
#pragma unroll
    for (int j = 0; j < kSteps; ++j)
#pragma unroll
      for (int k = 0; k < 4; ++k) o[j][nt][k] = 0.f;
  }
  unsigned stop = step * kSpanTiles < n ? step * kSpanTiles : n;  // (at most 2^23 keys a span)
  bool first = true;
#pragma unroll 1
  while (true) {
#pragma unroll 1
    for (; key0 < stop; key0 += step) {
      load_v(page, key0);
      float u[NT][4];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int k = 0; k < 4; ++k) u[nt][k] = 0.f;
#pragma unroll
      for (int c = 0; c < kPK; ++c) {
        const uint32_t a0[4] = {kr[0][c].x, kr[1][c].x, kr[0][c].y, kr[1][c].y};
        const uint32_t a1[4] = {kr[0][c].z, kr[1][c].z, kr[0][c].w, kr[1][c].w};
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          const uint2 q0 = sm.qf[(nt * kSteps + 2 * c) * 32 + lane], q1 = sm.qf[(nt * kSteps + 2 * c + 1) * 32 + lane];
          mma_bf16_16x8(u[nt], a0, q0.x, q0.y);
          mma_bf16_16x8(u[nt], a1, q1.x, q1.y);
        }
      }
      load_k(page_next, key0 + step);  // the next tile's keys, under this one's softmax and values
      page = page_next;
      page_next = page_of(key0 + 2 * step);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int k = 0; k < 4; ++k) u[nt][k] *= p.scale_log2;
      if (key0 + kFewKeys > all_see) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int k = 0; k < 4; ++k) u[nt][k] = key0 + g + 4 * (k & 2) < vis[nt][k & 1] ? u[nt][k] : -CUDART_INF_F;
      }
      uint32_t pt[NT][2];
      bool raise = false;
      float top[NT][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          float v = fmaxf(u[nt][x], u[nt][x + 2]);
#pragma unroll
          for (int off = 4; off < 32; off <<= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, off));
          top[nt][x] = v;
          raise |= v > m[nt][x] + kRaise;
        }
      if (__any_sync(0xffffffffu, raise)) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          float f[2];
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const float m_new = top[nt][x] > m[nt][x] + kRaise ? top[nt][x] : m[nt][x];
            f[x] = m[nt][x] == m_new ? 1.f : fast_exp2(m[nt][x] - m_new);
            l[nt][x] *= f[x];
            m[nt][x] = m_new;
          }
#pragma unroll
          for (int j = 0; j < kSteps; ++j) {
            o[j][nt][0] *= f[0];
            o[j][nt][1] *= f[1];
            o[j][nt][2] *= f[0];
            o[j][nt][3] *= f[1];
          }
        }
      }
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const float ref = m[nt][x] == -CUDART_INF_F ? 0.f : m[nt][x];
          u[nt][x] = fast_exp2(u[nt][x] - ref);
          u[nt][x + 2] = fast_exp2(u[nt][x + 2] - ref);
          l[nt][x] += u[nt][x] + u[nt][x + 2];
        }
        pt[nt][0] = transposed8(pack_bf16x2(u[nt][0], u[nt][1]));
        pt[nt][1] = transposed8(pack_bf16x2(u[nt][2], u[nt][3]));
      }
#pragma unroll
      for (int j = 0; j < kSteps; ++j) {
        const int c = j >> 2;
        const auto word = [&](int i) { return (j & 3) == 0 ? vr[i][c].x : (j & 3) == 1 ? vr[i][c].y : (j & 3) == 2 ? vr[i][c].z : vr[i][c].w; };
        // dims 8 (g + 8 c) + 2 (j % 4) and the next are the product's rows g and g + 8
        const uint32_t a[4] = {__byte_perm(word(0), word(1), 0x5410), __byte_perm(word(0), word(1), 0x7632),
                               __byte_perm(word(2), word(3), 0x5410), __byte_perm(word(2), word(3), 0x7632)};
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) mma_bf16_16x8(o[j][nt], a, pt[nt][0], pt[nt][1]);
      }
    }

    // a span's results, and those of the spans before
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int r = 8 * nt + 2 * t + x;
        float f = 0.f;
        if (!first) {
          const float before = sm.stat[warp * kR + r].x;
          f = before == m[nt][x] ? 1.f : fast_exp2(before - m[nt][x]);
        }
#pragma unroll
        for (int j = 0; j < kSteps; ++j) {
          float2* at = reinterpret_cast<float2*>(&sm.red[(warp * kR + r) * kStride + 64 * (j >> 2) + 8 * g + 2 * (j & 3)]);
          float2 sum = make_float2(o[j][nt][x], o[j][nt][x + 2]);
          if (!first) sum = make_float2(sum.x + f * at->x, sum.y + f * at->y);
          *at = sum;
          o[j][nt][x] = o[j][nt][x + 2] = 0.f;
        }
      }
    __syncwarp();
    if (g == 0) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int x = 0; x < 2; ++x) sm.stat[warp * kR + 8 * nt + 2 * t + x].x = m[nt][x];
    }
    __syncwarp();
    if (key0 >= n) break;
    first = false;
    stop = n - stop < step * kSpanTiles ? n : stop + step * kSpanTiles;
  }

  // ---- the warps' results, then the cluster's
  if (threadIdx.x < kR) sm.odd[threadIdx.x] = 0;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int x = 0; x < 2; ++x) {
#pragma unroll
      for (int off = 4; off < 32; off <<= 1) l[nt][x] += __shfl_xor_sync(0xffffffffu, l[nt][x], off);
      if (g == 0) sm.stat[warp * kR + 8 * nt + 2 * t + x].y = l[nt][x];
    }
  __syncthreads();
  // a warp or CTA without a tile has the maximum -inf, zeros, and weight 0
  const auto weight = [](float m_part, float m_all) { return m_part == -CUDART_INF_F ? 0.f : fast_exp2(m_part - m_all); };
  const int pairs = rows * (D / 2), per = (pairs + C - 1) / C;
  cluster_wait();
  for (int i = threadIdx.x; i < pairs; i += kFewThreads) {
    const int r = i / (D / 2), d = 2 * (i % (D / 2));
    float m_all = -CUDART_INF_F, l_all = 0.f;
#pragma unroll
    for (int w = 0; w < kFewWarps; ++w) m_all = fmaxf(m_all, sm.stat[w * kR + r].x);
    float2 sum = make_float2(0.f, 0.f);
#pragma unroll
    for (int w = 0; w < kFewWarps; ++w) {
      const float2 ml = sm.stat[w * kR + r];
      const float f = weight(ml.x, m_all);
      const float2 v = *reinterpret_cast<const float2*>(&sm.red[(w * kR + r) * kStride + d]);
      l_all += ml.x == -CUDART_INF_F ? ml.y : f * ml.y;  // (a NaN stays one)
      sum.x += f * v.x;
      sum.y += f * v.y;
    }
    const int to = i / per;  // the CTA that finishes this pair
    store_pair(&sm.peer_o[rank * per + (i - to * per)], to, sum);
    if (i % per == 0 || d == 0) store_pair(&sm.peer_ml[rank * kR + r], to, make_float2(m_all, l_all));
  }
  cluster_arrive();
  cluster_wait();
  __nv_bfloat16* const out = reinterpret_cast<__nv_bfloat16*>(p.out);
  const auto out_at = [&](int r) {
    const int i = r / p.group;
    return out + ((size_t)(s.row0 + i) * p.H + h * p.group + (r - i * p.group)) * D;
  };
  for (int k = threadIdx.x; k < per; k += kFewThreads) {
    const int i = rank * per + k;
    if (i >= pairs) break;
    const int r = i / (D / 2), d = 2 * (i % (D / 2));
    float m_all = -CUDART_INF_F, l_all = 0.f;
    for (int x = 0; x < C; ++x) m_all = fmaxf(m_all, sm.peer_ml[x * kR + r].x);
    float2 sum = make_float2(0.f, 0.f);
    for (int x = 0; x < C; ++x) {
      const float2 ml = sm.peer_ml[x * kR + r];
      const float f = weight(ml.x, m_all);
      const float2 v = sm.peer_o[x * per + k];
      l_all += ml.x == -CUDART_INF_F ? ml.y : f * ml.y;
      sum.x += f * v.x;
      sum.y += f * v.y;
    }
    if (seen(s, r / p.group) == 0) {
      sum = make_float2(0.f, 0.f);
    } else {
      const float inv = 1.f / l_all;
      sum.x *= inv;
      sum.y *= inv;
      if (l_all > 0.f && !(isfinite(sum.x) && isfinite(sum.y))) sm.odd[r] = 1;
    }
    *reinterpret_cast<uint32_t*>(out_at(r) + d) = pack_bf16x2(sum.x, sum.y);
  }
  __syncthreads();
  for (int r = warp; r < rows; r += kFewWarps) {  // this CTA's columns of the rows that are not finite
    if (!sm.odd[r]) continue;
    float y[D / 32];
    const int i = r / p.group;
    attend_row<__nv_bfloat16, D>(p, b, s, i, h * p.group + r - i * p.group, seen(s, i), y);
#pragma unroll
    for (int e = 0; e < D / 32; e += 2) {
      const int d = lane * (D / 32) + e;
      if ((r * (D / 2) + d / 2) / per == rank) *reinterpret_cast<uint32_t*>(out_at(r) + d) = pack_bf16x2(y[e], y[e + 1]);
    }
  }
}

// CTAs of a slab's cluster, for up to `keys` keys: the C of least estimated time.  A CTA alone streams ~40 GB/s and all of
// them ~7 TB/s, each wave costs its start of ~2.5 us, and the last wave has what is left.  Only the bound of the lengths is
// known here, so a call of several requests is judged by the sum of two: all at the bound, and half of that in the mean
// with one at the bound, which the longest CTA then may decide.  us by C = 1 / 2 / 4 / 8: 208 slabs of 16384 keys 277 / 293 /
// 264 / 268, 256 of 1024 to 16384 keys 201 / 153 / 160 / 180, 512 of up to 1024 keys 39 / 46 / 59 / 92, 32 of 8192
// keys 85 / 47 / 30 / 26, 128 of up to 4096 keys (64 dims) 31 / 22 / 25 / 33.
int pick(long long slabs, long long slots, int keys, int row_bytes, bool several) {
  const float mb = 2e-6f * (float)keys * (float)row_bytes;
  constexpr float kOne = 25.f, kAll = 1.f / 7.f, kStart = 2.5f;  // us per MB: a CTA alone, all together; us
  int best = 1;
  float least = 0.f;
  for (int C = 1; C <= kMaxC; C *= 2) {
    if (C > 1 && C * kFewWarps * kFewKeys >= 2LL * keys) break;  // no tiles for half of the warps
    const long long n = slabs * C, full = n / slots, rest = n - full * slots;
    const float part = mb / (float)C;
    const auto wave = [&](float ctas) { return part * (ctas * kAll > kOne ? ctas * kAll : kOne); };
    const float start = kStart * (float)(full + (rest ? 1 : 0));
    float cost = (float)full * wave((float)slots) + (rest ? wave((float)rest) : 0.f) + start;
    if (several) {
      const float mean = 0.5f * mb * (float)slabs * kAll, longest = part * kOne;
      cost += (mean > longest ? mean : longest) + start;
    }
    if (C == 1 || cost < least) {
      least = cost;
      best = C;
    }
  }
  return best;
}

template <int D, int NT>
cudaError_t launch_typed(const RowsArgs& a, cudaStream_t st) {
  constexpr size_t kSmem = sizeof(FewSmem<D, NT>);
  static PerDevice<int> allowed;
  cudaError_t e = allow_smem(allowed, paged_few_kernel<D, NT>, (int)kSmem);
  if (e != cudaSuccess) return e;
  const long long slabs = (long long)a.B * a.Hkv, slots = (NT == 1 ? 2LL : 1LL) * sm_count();
  const int C = pick(slabs, slots, a.max_kv, 2 * D, a.B > 1);
  if (slabs * C > 0x7fffffffLL) return cudaErrorNotSupported;
  const RowsParams p = rows_params(a);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(slabs * C));
  cfg.blockDim = dim3(kFewThreads);
  cfg.dynamicSmemBytes = kSmem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)C;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  const int sorted = a.B > 1 && a.B <= kFewThreads && slabs * C > slots ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, paged_few_kernel<D, NT>, p, C, sorted);
}

}  // namespace

cudaError_t launch_paged_few(const RowsArgs& a, cudaStream_t st) {
  const long long rows = (long long)a.max_q * (a.H / a.Hkv);
  if (a.dtype != 0 || !a.table || rows > 16) return cudaErrorNotSupported;
  if (rows <= 8) return a.D == 128 ? launch_typed<128, 1>(a, st) : launch_typed<64, 1>(a, st);
  return a.D == 128 ? launch_typed<128, 2>(a, st) : launch_typed<64, 2>(a, st);
}

}  // namespace glide
