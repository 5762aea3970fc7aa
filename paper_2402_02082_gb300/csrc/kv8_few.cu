// Attention over the 8-bit cache for few query rows (draft queries, short chains), straight from global
// memory to registers.
//
// What bounds it.  A cached row is read once for at most 16 query rows, so HBM bounds long caches and the fixed parts of a
// call bound short ones.  The tcgen05 kernel spends ~8 us beside the bytes on barriers, tensor memory, a split table and a
// second kernel for the merge.  Here a cluster of C CTAs serves a slab (a sequence's cached head and the queries that read
// it) and its 8 C warps take the 32-key tiles in turn, without shared memory until the end.
//
// The mathematics is that of the tcgen05 kernel: u = s + eV, m its running maximum, p = 2^(u - m + 8), l = sum p 2^-eV,
// out = (sum p V8) / l.  The products are warp-level fp16 ones with fp32 sums, keys (and value columns) their 16 rows and
// queries their 8 columns: codes are fp16 numbers exactly, so are bf16 queries scaled by a power of two, and a weight is
// held to 2^-12.  A fragment's K index may be any permutation that both operands share, so a lane's fragments are
// consecutive bytes of a row:
//   S^T (16 keys x 8 queries): lane (g, t) reads dims D/4 t .. of key g, and the same dims of query g
//   O^T (16 dims x 8 queries): lane (g, t) reads dims D/8 g .. of keys 2t, 2t + 1, 2t + 8, 2t + 9
// The weights of S^T become the second product's operand by a transpose of 8 x 8 within the warp; rows of both results lie
// in the same lanes, so the running maximum and sum need no exchange but the maximum's over the keys.
#include <cfloat>
#include <cuda_bf16.h>
#include <math_constants.h>

#include "attn_common.cuh"
#include "common.cuh"
#include "device.h"
#include "kv8.h"
#include "tc_attn.cuh"

namespace glide {
namespace {

constexpr int kWarpsF = 8;
constexpr int kThreadsF = kWarpsF * 32;
constexpr int kTKF = 32;  // keys of a tile
constexpr int kMaxC = 8;
constexpr float kLiftF = 8.f;

struct FewParams {
  const __nv_bfloat16 *q, *kt, *vt;
  const uint8_t *K, *V;
  const int8_t *Ke, *Ve;
  const int *kv_len, *parent;
  __nv_bfloat16* out;
  int H, Hkv, S_cap, max_kv_len, n, group, rows, C, blocks;
  float scale_log2;
};

__device__ __forceinline__ void mma_f16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
  return r;
}
__device__ __forceinline__ uint32_t f16pair(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
// Four codes as four fp16 values, exactly.
__device__ __forceinline__ void widen(uint32_t w, uint32_t& a, uint32_t& b) {
  asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, l;\n\tcvt.rn.f16x2.e4m3x2 %1, h;\n\t}"
      : "=r"(a), "=r"(b)
      : "r"(w));
}
// The exponent that brings the largest finite of some bf16 magnitudes (its bits) to at most 448.
__device__ __forceinline__ int exponent_of(uint32_t bits) {
  return kv8_clamp_exp((int)(bits >> 7) - 127 - 8 + ((bits & 0x7fu) > 0x60u ? 1 : 0));
}
__device__ __forceinline__ uint32_t top_pair(uint32_t w, uint32_t most) {
  const uint32_t a = w & 0x7fffu, b = (w >> 16) & 0x7fffu;
  return max(most, max(a < 0x7f80u ? a : 0u, b < 0x7f80u ? b : 0u));
}
// Two bf16 elements times a power of two as fp16; what is not finite stays so.
__device__ __forceinline__ uint32_t scaled_pair(uint32_t w, float s) { return f16pair(bf16lo(w) * s, bf16hi(w) * s); }

// A pair of floats to the same place in CTA `rank`'s shared memory.
__device__ __forceinline__ void store_peer(float2* at, uint32_t rank, float2 v) {
  uint32_t a;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_u32(at)), "r"(rank));
  asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(a), "f"(v.x), "f"(v.y) : "memory");
}

template <int D, int NT>
__global__ void __launch_bounds__(kThreadsF, NT == 1 ? 2 : 1) kv8_few_kernel(const FewParams p) {
  constexpr int kR = 8 * NT;        // query rows
  constexpr int kSteps = D / 16;    // products of S along D
  constexpr int kWK = D / 16;       // 32-bit words of a key row that a lane reads
  constexpr int kWV = D / 32;       // of a value row
  constexpr int kStride = D + 4;    // floats of a partial row: the lanes' stores then meet no bank twice
  extern __shared__ float smem[];
  float* red = smem;                                                        // [warps][kR][kStride]
  float2* stat = reinterpret_cast<float2*>(red + kWarpsF * kR * kStride);   // [warps][kR] (m, l)
  float2* peer_ml = stat + kWarpsF * kR;                                    // [kMaxC][kR] (m, l), from the peers
  float2* peer_o = peer_ml + kMaxC * kR;                                    // [kR D / 2 + kMaxC]: this CTA's pairs, from each
  uint2* qf = reinterpret_cast<uint2*>(peer_o + kR * D / 2 + kMaxC);        // [NT][kSteps][32] the queries' fragments
  float* q_unit = reinterpret_cast<float*>(qf + NT * kSteps * 32);          // [kR] what makes a product log2 units
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int rank = (int)cluster_rank();
  const int slab = blockIdx.x / p.C, b = slab / p.Hkv, h = slab - b * p.Hkv;
  cluster_arrive();  // that every peer's shared memory is there is known when it is written to
  pdl_wait();
  const int L_told = p.kv_len[b];
  const int Lmax = p.max_kv_len;
  const uint64_t pol = policy_evict_first();
  const uint8_t* Kg = p.K + (size_t)slab * p.S_cap * D;
  const uint8_t* Vg = p.V + (size_t)slab * p.S_cap * D;
  const int8_t *Ke = p.Ke + (size_t)slab * p.blocks, *Ve = p.Ve + (size_t)slab * p.blocks;

  // this lane's pieces of a tile: keys g, g + 8, .. of K; of V keys 2t, 2t + 1, 2t + 8, 2t + 9 of each 16.  The first
  // loads do not wait for the length but go by its bound; what lies past the length is masked, and V's made zeros.
  uint32_t kr[4][kWK], vr[8][kWV];
  auto load_k = [&](int key0) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int key = key0 + g + 8 * i;
      const uint8_t* at = Kg + (size_t)key * D + t * (D / 4);
#pragma unroll
      for (int w = 0; w < kWK; w += 4) {
        uint4 x = make_uint4(0u, 0u, 0u, 0u);
        if (key < Lmax) x = load_once(at + 4 * w, pol);
        kr[i][w] = x.x;
        kr[i][w + 1] = x.y;
        kr[i][w + 2] = x.z;
        kr[i][w + 3] = x.w;
      }
    }
  };
  auto load_v = [&](int key0) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int key = key0 + 16 * (i / 4) + 8 * ((i / 2) % 2) + 2 * t + i % 2;
      const uint8_t* at = Vg + (size_t)key * D + g * (D / 8);
      if constexpr (kWV == 4) {
        uint4 x = make_uint4(0u, 0u, 0u, 0u);
        if (key < Lmax) x = load_once(at, pol);
        vr[i][0] = x.x;
        vr[i][1] = x.y;
        vr[i][2] = x.z;
        vr[i][3] = x.w;
      } else {
        uint2 x = make_uint2(0u, 0u);
        if (key < Lmax) x = __ldcs(reinterpret_cast<const uint2*>(at));
        vr[i][0] = x.x;
        vr[i][1] = x.y;
      }
    }
  };
  // A tree is one more tile, of the cluster's last warp, which in clusters of four CTAs or more has no other: its keys,
  // values and parents are loads of their own (32 heads, 2048 keys, 6 nodes: 12.7 us beside a tile, 11.3 alone).
  const bool tree_warp = p.parent && rank == p.C - 1 && warp == kWarpsF - 1;
  const int spare = p.parent && p.C >= 4 ? 1 : 0;
  const int step = (p.C * kWarpsF - spare) * kTKF;
  int key0 = tree_warp && spare ? p.max_kv_len : (rank * kWarpsF + warp) * kTKF;
  int ke = 0, ve = 0;
  auto load_exps = [&](int key) {
    if (key < Lmax) {
      ke = kv8_clamp_exp(Ke[key / kKv8Block]);
      ve = kv8_clamp_exp(Ve[key / kKv8Block]);
    }
  };
  // The tree's own keys (g, g + 8; as K) and values (2t, 2t + 1, 2t + 8, 2t + 9; as V), bf16 as they lie, in the registers
  // that a tile's take.
  auto load_tree = [&] {
    auto put = [](const __nv_bfloat16* at, bool there, uint32_t* w) {
      const uint4 x = there ? *reinterpret_cast<const uint4*>(at) : make_uint4(0u, 0u, 0u, 0u);
      w[0] = x.x;
      w[1] = x.y;
      w[2] = x.z;
      w[3] = x.w;
    };
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int key = g + 8 * i;
      const __nv_bfloat16* at = p.kt + (((size_t)b * p.n + key) * p.Hkv + h) * D + t * (D / 4);
#pragma unroll
      for (int w = 0; w < 2 * kSteps; w += 4) put(at + 2 * w, key < p.n, &kr[2 * i + w / kWK][w % kWK]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int key = 8 * (i / 2) + 2 * t + i % 2;
      const __nv_bfloat16* at = p.vt + (((size_t)b * p.n + key) * p.Hkv + h) * D + g * (D / 8);
      uint32_t w[2 * kWV];
#pragma unroll
      for (int k = 0; k < 2 * kWV; k += 4) put(at + 2 * k, key < p.n, w + k);
#pragma unroll
      for (int k = 0; k < 2 * kWV; ++k) vr[2 * i + k / kWV][k % kWV] = w[k];
    }
  };
  int2 up = make_int2(-1, -1);
  if (tree_warp) {
    up = parents_of(p.parent + (size_t)b * p.n, p.n, lane);
    load_tree();
  } else {
    load_k(key0);
    load_v(key0);
    load_exps(key0);
  }


  // the queries, each scaled by its own power of two, by one warp for 8 of them
  if (warp < NT) {
    const int r = 8 * warp + g, node = r / p.group;
    uint32_t w[2 * kSteps];
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < 2 * kSteps; i += 4) {
      uint4 x = make_uint4(0u, 0u, 0u, 0u);
      if (r < p.rows)
        x = *reinterpret_cast<const uint4*>(
            p.q + (((size_t)b * p.n + node) * p.H + h * p.group + (r - node * p.group)) * D + t * (D / 4) + 2 * i);
      w[i] = x.x;
      w[i + 1] = x.y;
      w[i + 2] = x.z;
      w[i + 3] = x.w;
#pragma unroll
      for (int k = 0; k < 4; ++k) most = top_pair(w[i + k], most);
    }
    most = max(most, __shfl_xor_sync(0xffffffffu, most, 1));
    most = max(most, __shfl_xor_sync(0xffffffffu, most, 2));
    const int e = exponent_of(most);
    const float s = kv8_pow2(-e);
#pragma unroll
    for (int i = 0; i < kSteps; ++i)
      qf[(warp * kSteps + i) * 32 + lane] = make_uint2(scaled_pair(w[2 * i], s), scaled_pair(w[2 * i + 1], s));
    if (t == 0) q_unit[r] = p.scale_log2 * kv8_pow2(e);
  }
  const int L = L_told < 0 ? 0 : (L_told > Lmax ? Lmax : L_told);
  __syncthreads();
  float c[NT][2];  // of rows 2t, 2t + 1
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    c[nt][0] = q_unit[8 * nt + 2 * t];
    c[nt][1] = q_unit[8 * nt + 2 * t + 1];
  }

  float m[NT][2], l[NT][2], o[D / 16][NT][4];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    m[nt][0] = m[nt][1] = -CUDART_INF_F;
    l[nt][0] = l[nt][1] = 0.f;
#pragma unroll
    for (int j = 0; j < D / 16; ++j)
#pragma unroll
      for (int k = 0; k < 4; ++k) o[j][nt][k] = 0.f;
  }
  // A new maximum over `u` (16 KG keys: [group][row tile][key g: rows 2t, 2t + 1; key g + 8: the same]), then the
  // weights, transposed for the second product.  The keys of a cached tile share the exponent e[0]; those of the tree's one
  // group have their own, e[0] of key g and e[1] of key g + 8, so far apart that 2^-e must not meet a weight that has
  // become zero: their terms of l are exponentials of their own.
  auto weigh = [&](auto& u, auto& pt, const int (&e)[2]) {
    constexpr int KG = sizeof(u) / sizeof(u[0]);
    const float inv_v = kv8_pow2(-e[0]);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      float corr[2];
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        float top = fmaxf(u[0][nt][x], u[0][nt][x + 2]);
#pragma unroll
        for (int kg = 1; kg < KG; ++kg) top = fmaxf(top, fmaxf(u[kg][nt][x], u[kg][nt][x + 2]));
#pragma unroll
        for (int off = 4; off < 32; off <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
        top = fmaxf(m[nt][x], top);
        const float ref = (top == -CUDART_INF_F ? 0.f : top) - kLiftF;  // nothing seen yet, or NaN only
        // l holds 2^-eV and so may be far larger than the weights that it sums: it takes 2^(m - top) in two steps, neither
        // of which leaves fp32's range before the result does
        const float half = fast_exp2(0.5f * (m[nt][x] - (ref + kLiftF)));
        corr[x] = half * half;
        l[nt][x] = l[nt][x] == 0.f ? 0.f : l[nt][x] * half * half;
        if constexpr (KG == 1)
          l[nt][x] += fast_exp2(u[0][nt][x] - ref - (float)e[0]) + fast_exp2(u[0][nt][x + 2] - ref - (float)e[1]);
        float sum = 0.f;
#pragma unroll
        for (int kg = 0; kg < KG; ++kg) {
          u[kg][nt][x] = fast_exp2(u[kg][nt][x] - ref);
          u[kg][nt][x + 2] = fast_exp2(u[kg][nt][x + 2] - ref);
          sum += u[kg][nt][x] + u[kg][nt][x + 2];
        }
        if constexpr (KG > 1) l[nt][x] += sum * inv_v;
        m[nt][x] = top;
      }
#pragma unroll
      for (int kg = 0; kg < KG; ++kg) {
        pt[kg][nt][0] = transpose8(f16pair(u[kg][nt][0], u[kg][nt][1]));
        pt[kg][nt][1] = transpose8(f16pair(u[kg][nt][2], u[kg][nt][3]));
      }
#pragma unroll
      for (int j = 0; j < D / 16; ++j) {
        o[j][nt][0] *= corr[0];
        o[j][nt][1] *= corr[1];
        o[j][nt][2] *= corr[0];
        o[j][nt][3] *= corr[1];
      }
    }
  };

  int ref_v = -128;  // the largest value exponent of the cached blocks so far, which every row sees
  // ---- the tree's own keys and values: at most 16
  bool odd_values = false;  // the tree has values that are not finite
  uint32_t* const own_vis = reinterpret_cast<uint32_t*>(red + warp * kR * kStride);  // then: the nodes that each row sees
  if (tree_warp) {
    const int n = p.n;
    // the nodes that node `lane` sees: itself and its ancestors, found by pointer jumping (at most 16 levels)
    uint32_t sees = lane < n ? 1u << lane : 0u;
    int next = lane < n && up.x >= 0 && up.x < lane ? up.x : -1;
#pragma unroll
    for (int round = 0; round < 4; ++round) {
      const int from = next < 0 ? lane : next;
      const uint32_t more = __shfl_sync(0xffffffffu, sees, from);
      const int further = __shfl_sync(0xffffffffu, next, from);
      sees |= more;
      next = next < 0 ? -1 : further;
    }
    uint32_t vis[NT][2];  // the nodes that rows 2t, 2t + 1 see
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int r = 8 * nt + 2 * t + x;
        vis[nt][x] = __shfl_sync(0xffffffffu, sees, r < p.rows ? r / p.group : 0);
      }
    auto kw = [&](int i, int w) { return kr[2 * i + w / kWK][w % kWK]; };
    auto vw = [&](int i, int w) -> uint32_t& { return vr[2 * i + w / kWV][w % kWV]; };
    // keys and values are scaled to fp16, each node's by powers of two of its own: a row that does not see a node must not
    // lose anything to that node's size
    float sk[2], ks[2];  // keys g, g + 8
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      uint32_t most = 0;
#pragma unroll
      for (int w = 0; w < 2 * kSteps; ++w) most = top_pair(kw(i, w), most);
      most = max(most, __shfl_xor_sync(0xffffffffu, most, 1));
      most = max(most, __shfl_xor_sync(0xffffffffu, most, 2));
      const int e = exponent_of(most);
      sk[i] = kv8_pow2(-e);
      ks[i] = kv8_pow2(e);
    }
    float u[1][NT][4];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int k = 0; k < 4; ++k) u[0][nt][k] = 0.f;
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      const uint32_t a[4] = {scaled_pair(kw(0, 2 * s), sk[0]), scaled_pair(kw(1, 2 * s), sk[1]),
                             scaled_pair(kw(0, 2 * s + 1), sk[0]), scaled_pair(kw(1, 2 * s + 1), sk[1])};
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const uint2 q = qf[(nt * kSteps + s) * 32 + lane];
        mma_f16(u[0][nt], a, q.x, q.y);
      }
    }
    bool odd = false;
    int e_v[4];  // of keys 2t, 2t + 1, 2t + 8, 2t + 9
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t most = 0;
#pragma unroll
      for (int w = 0; w < 2 * kWV; ++w) {
        uint32_t& x = vw(i, w);
        // an unseen value that is not finite must not meet a weight of zero: left out here, put back below
        if ((x & 0x7f80u) == 0x7f80u) x &= 0xffff0000u, odd = true;
        if ((x & 0x7f800000u) == 0x7f800000u) x &= 0xffffu, odd = true;
        most = top_pair(x, most);
      }
#pragma unroll
      for (int off = 4; off < 32; off <<= 1) most = max(most, __shfl_xor_sync(0xffffffffu, most, off));
      e_v[i] = max(exponent_of(most), -90);
    }
    int e[2];  // of keys g, g + 8
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int even = __shfl_sync(0xffffffffu, e_v[2 * i], g >> 1), other = __shfl_sync(0xffffffffu, e_v[2 * i + 1], g >> 1);
      e[i] = g & 1 ? other : even;
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float x = fmaf(u[0][nt][k] * ks[k >> 1], c[nt][k & 1], (float)e[k >> 1]);
        u[0][nt][k] = (vis[nt][k & 1] >> (g + 4 * (k & 2))) & 1u ? x : -CUDART_INF_F;
      }
    uint32_t pt[1][NT][2];
    weigh(u, pt, e);
#pragma unroll
    for (int j = 0; j < D / 16; ++j) {
      auto pair = [&](int i, uint32_t& lo, uint32_t& hi) {  // dims 2j, 2j + 1 of two keys
        const float sx = kv8_pow2(-e_v[i]), sy = kv8_pow2(-e_v[i + 1]);
        lo = f16pair(bf16lo(vw(i, j)) * sx, bf16lo(vw(i + 1, j)) * sy);
        hi = f16pair(bf16hi(vw(i, j)) * sx, bf16hi(vw(i + 1, j)) * sy);
      };
      uint32_t a[4];
      pair(0, a[0], a[1]);
      pair(2, a[2], a[3]);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) mma_f16(o[j][nt], a, pt[0][nt][0], pt[0][nt][1]);
    }
    odd_values = __any_sync(0xffffffffu, odd);
    if (odd_values && g == 0) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) own_vis[8 * nt + 2 * t] = vis[nt][0], own_vis[8 * nt + 2 * t + 1] = vis[nt][1];
    }
    load_k(key0);
    load_v(key0);
    load_exps(key0);
  }
#pragma unroll 1
  for (bool first = true; key0 < L; key0 += step, first = false) {
    if (!first) load_v(key0);
    if (key0 + kTKF > L) {  // the last tile
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int key = key0 + 16 * (i / 4) + 8 * ((i / 2) % 2) + 2 * t + i % 2;
#pragma unroll
        for (int w = 0; w < kWV; ++w) vr[i][w] = key < L ? vr[i][w] : 0u;
      }
    }
    float u[2][NT][4];
    const float ks = kv8_pow2(ke);
    ref_v = max(ref_v, ve);
    const int e = max(max(ve, ref_v - 110), -90);  // far smaller blocks count as 2^-110 of the largest
#pragma unroll
    for (int kg = 0; kg < 2; ++kg) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int k = 0; k < 4; ++k) u[kg][nt][k] = 0.f;
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        uint32_t a[4];
        widen(kr[2 * kg][s], a[0], a[2]);
        widen(kr[2 * kg + 1][s], a[1], a[3]);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          const uint2 q = qf[(nt * kSteps + s) * 32 + lane];
          mma_f16(u[kg][nt], a, q.x, q.y);
        }
      }
    }
    load_k(key0 + step);  // the next tile's keys, under this one's softmax and values
    load_exps(key0 + step);
#pragma unroll
    for (int kg = 0; kg < 2; ++kg)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float x = fmaf(u[kg][nt][k] * ks, c[nt][k & 1], (float)e);
          u[kg][nt][k] = key0 + 16 * kg + g + 4 * (k & 2) < L ? x : -CUDART_INF_F;
        }
    uint32_t pt[2][NT][2];
    weigh(u, pt, {e, e});
#pragma unroll
    for (int kg = 0; kg < 2; ++kg)
#pragma unroll
      for (int j = 0; j < D / 16; ++j) {
        // bytes 2j, 2j + 1 of the lane's piece: dims of the product's rows g and g + 8
        const uint32_t pick = j % 2 ? 0x7362u : 0x5140u;
        uint32_t a[4];
        widen(__byte_perm(vr[4 * kg][j / 2], vr[4 * kg + 1][j / 2], pick), a[0], a[1]);
        widen(__byte_perm(vr[4 * kg + 2][j / 2], vr[4 * kg + 3][j / 2], pick), a[2], a[3]);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) mma_f16(o[j][nt], a, pt[kg][nt][0], pt[kg][nt][1]);
      }
  }

  if (odd_values) {  // a visible one decides its column, however small its weight
    __syncwarp();
    uint32_t vis[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) vis[nt][0] = own_vis[8 * nt + 2 * t], vis[nt][1] = own_vis[8 * nt + 2 * t + 1];
    __syncwarp();
#pragma unroll 1
    for (int key = 0; key < p.n; ++key)
#pragma unroll
      for (int j = 0; j < D / 16; ++j)
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          const float v = __bfloat162float(p.vt[(((size_t)b * p.n + key) * p.Hkv + h) * D + g * (D / 8) + 2 * j + y]);
          if (isfinite(v)) continue;
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int x = 0; x < 2; ++x)
              if ((vis[nt][x] >> key) & 1u) o[j][nt][2 * y + x] += v;
        }
  }

  // ---- the warps' results, then the cluster's.  Position 16 j + 2 g + y of a partial row is dim D/8 g + 2 j + y.
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const int r = 8 * nt + 2 * t + x;
#pragma unroll
      for (int off = 4; off < 32; off <<= 1) l[nt][x] += __shfl_xor_sync(0xffffffffu, l[nt][x], off);
      if (g == 0) stat[warp * kR + r] = make_float2(m[nt][x], l[nt][x]);
#pragma unroll
      for (int j = 0; j < D / 16; ++j)
        *reinterpret_cast<float2*>(&red[(warp * kR + r) * kStride + 16 * j + 2 * g]) = make_float2(o[j][nt][x], o[j][nt][x + 2]);
    }
  __syncthreads();
  // The weight of a partial (m, l, o) against the largest M, and its l: in the logarithm, as 2^-eV may take either
  // factor out of fp32's range.  The weight is at least the least normal number: zero times an infinite o were NaN.
  auto weight = [](float2 s, float M, float& L) {
    const float ref = M == -CUDART_INF_F ? 0.f : M;
    if (s.y != 0.f) L += s.x == -CUDART_INF_F ? s.y : fast_exp2(s.x - ref + __log2f(s.y));
    return s.x == -CUDART_INF_F ? 0.f : fmaxf(fast_exp2(s.x - ref), FLT_MIN);
  };
  const int pairs = p.rows * (D / 2), per = (pairs + p.C - 1) / p.C;
  cluster_wait();
  for (int i = threadIdx.x; i < pairs; i += kThreadsF) {
    const int r = i / (D / 2), d = 2 * (i % (D / 2));
    float M = -CUDART_INF_F, Lr = 0.f;
#pragma unroll
    for (int w = 0; w < kWarpsF; ++w) M = fmaxf(M, stat[w * kR + r].x);
    float2 sum = make_float2(0.f, 0.f);
#pragma unroll
    for (int w = 0; w < kWarpsF; ++w) {
      const float f = weight(stat[w * kR + r], M, Lr);
      const float2 v = *reinterpret_cast<const float2*>(&red[(w * kR + r) * kStride + d]);
      sum.x += f * v.x;
      sum.y += f * v.y;
    }
    // to the CTA that finishes this pair: pair i is CTA i / per's
    const int to = i / per;
    store_peer(&peer_o[rank * per + (i - to * per)], to, sum);
    if (i % per == 0 || d == 0) store_peer(&peer_ml[rank * kR + r], to, make_float2(M, Lr));
  }
  cluster_arrive();
  cluster_wait();
  for (int k = threadIdx.x; k < per; k += kThreadsF) {
    const int i = rank * per + k;
    if (i >= pairs) break;
    const int r = i / (D / 2), d = 2 * (i % (D / 2));
    float M = -CUDART_INF_F, Lr = 0.f;
    for (int x = 0; x < p.C; ++x) M = fmaxf(M, peer_ml[x * kR + r].x);
    float2 sum = make_float2(0.f, 0.f);
    for (int x = 0; x < p.C; ++x) {
      const float f = weight(peer_ml[x * kR + r], M, Lr);
      const float2 v = peer_o[x * per + k];
      sum.x += f * v.x;
      sum.y += f * v.y;
    }
    const float inv = L == 0 && !p.parent ? 0.f : 1.f / Lr;  // no keys at all: zeros; scores of -inf alone: NaN
    const int node = r / p.group, dim = (D / 8) * (d % 16 / 2) + 2 * (d / 16);
    *reinterpret_cast<uint32_t*>(p.out + (((size_t)b * p.n + node) * p.H + h * p.group + (r - node * p.group)) * D + dim) =
        pack_bf16x2(sum.x * inv, sum.y * inv);
  }
}

cudaLaunchConfig_t config(long long slabs, int C, size_t smem, cudaStream_t st, cudaLaunchAttribute* attr) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(slabs * C));
  cfg.blockDim = dim3(kThreadsF);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)C;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cfg;
}

template <int D, int NT>
cudaError_t launch_typed(const Kv8AttnArgs& a, cudaStream_t st) {
  constexpr size_t kSmem = sizeof(float) * (kWarpsF * 8 * NT * (D + 4) + 2 * (kWarpsF + kMaxC) * 8 * NT +
                                            8 * NT * D + 2 * kMaxC + NT * (D / 16) * 64 + 8 * NT);
  static PerDevice<int> allowed;
  cudaError_t e = allow_smem(allowed, kv8_few_kernel<D, NT>, (int)kSmem);
  if (e != cudaSuccess) return e;
  const long long slabs = (long long)a.B * a.Hkv, slots = (NT == 1 ? 2LL : 1LL) * sm_count();
  int C = kMaxC;
  while (C > 1 && (slabs * C > slots || (long long)C * kWarpsF * kTKF >= 2LL * a.max_kv_len)) C >>= 1;
  // One wave, and short: with 32 keys a warp at a time and nothing but registers to hold what is on its way, the tcgen05
  // kernel's ring streams faster once the warps have several tiles.  Here / there, us, with the tiles a warp has.  Up to 8
  // rows: 32 heads of 2048 keys (1) 8.9 / 10.6, 4096 (2) 12.2 / 13.1, 6144 (3) 15.1 / 14.8, 16384 (8) 29.3 / 26.2; the
  // GPU half empty, 8 heads of 8192 (4) 13.7 / 17.2, 16384 (8) 21.9 / 17.3; two waves, 8 x 40 heads of 512 17.7 / 14.1.
  // Up to 16 rows: 12 nodes on 32 heads of 4096 (4) 16.5 / 16.8, 6144 (6) 20.8 / 18.5.  Rows of 64 dims are half a tile:
  // 32 heads of 8192 (4) 11.9 / 13.9.
  const long long rounds = (a.max_kv_len + C * kWarpsF * kTKF - 1LL) / (C * kWarpsF * kTKF);
  const int most = NT == 1 && 2 * slabs * C > slots ? 2 : 4;
  if (slabs * C > slots || rounds * D > most * 128LL) return cudaErrorNotSupported;
  if (a.max_ctas > 0 && slabs * C > a.max_ctas) return cudaErrorNotSupported;
  if (slabs * C > 0x7fffffffLL) return cudaErrorNotSupported;
  FewParams p;
  p.q = static_cast<const __nv_bfloat16*>(a.q);
  p.kt = static_cast<const __nv_bfloat16*>(a.kt);
  p.vt = static_cast<const __nv_bfloat16*>(a.vt);
  p.K = a.K; p.V = a.V; p.Ke = a.Ke; p.Ve = a.Ve; p.kv_len = a.kv_len; p.parent = a.parent;
  p.out = static_cast<__nv_bfloat16*>(a.out);
  p.H = a.H; p.Hkv = a.Hkv; p.S_cap = a.S_cap; p.max_kv_len = a.max_kv_len; p.n = a.nq; p.group = a.H / a.Hkv;
  p.rows = a.nq * p.group; p.C = C; p.blocks = kv8_blocks(a.S_cap);
  p.scale_log2 = a.scale * kLog2e;
  cudaLaunchAttribute attr[2];
  const cudaLaunchConfig_t cfg = config(slabs, C, kSmem, st, attr);
  return cudaLaunchKernelEx(&cfg, kv8_few_kernel<D, NT>, p);
}

}  // namespace

cudaError_t launch_kv8_few(const Kv8AttnArgs& a, cudaStream_t st) {
  const int rows = a.nq * (a.H / a.Hkv);
  if (a.dtype != 0 || rows > 16) return cudaErrorNotSupported;
  if (rows <= 8) return a.D == 128 ? launch_typed<128, 1>(a, st) : launch_typed<64, 1>(a, st);
  return a.D == 128 ? launch_typed<128, 2>(a, st) : launch_typed<64, 2>(a, st);
}

}  // namespace glide
