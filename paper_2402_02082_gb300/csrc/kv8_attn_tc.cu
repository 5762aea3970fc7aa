// Attention over the 8-bit cache on the tcgen05 tensor cores: draft queries (cross-attention) and
// tree queries (verification), bf16 in and out, fp32 sums.
//
// The mathematics.  With codes K8, V8 and block exponents eK, eV of key t,
//   s[r,t] = q[r] . K8[t] * 2^eK * scale * log2(e),   u[r,t] = s[r,t] + eV[t]
//   m[r]   = running maximum of u less kLift,    p[r,t] = 2^(u - m)
//   O[r]   = sum_t p[r,t] V8[t],     l[r]   = sum_t p[r,t] 2^-eV[t],    out[r] = O[r] / l[r]
// Taking the value exponent into the weight's exponent leaves the codes as they are: no key or value is scaled, no key is
// widened, and values only where many rows share that work (below).
//
// 8-bit operands without 8-bit results.  A bf16 query has 8 significant bits, two codes' worth: with a row's largest
// element scaled to at most 448, and at least 28, q = hi + lo exactly down to the codes' least step (2^-9, or 2^-13 at 8
// rows, where lo is held 16 times itself).  Weights, up to 16 rows: p <= 430 is hi + lo / 28 to 2^-8.5 of itself, or to 2^-22
// of the row's largest, which is at least 2^8.  More rows: values are widened to fp16 in shared memory, weights rounded
// to fp16 (2^-12 of themselves).  The tree's own bf16 keys and values are a tile of their own, multiplied as bf16
// with bf16 queries and weights; a node's values are scaled by a power of two of its own, which its weight's exponent takes
// as a block's, so that what a row does not see has no say in how finely the rest is held.
//
// Orientation.  Keys are the 128 rows of the MMA and the queries its columns:
//   S^T = K8 Q^T    : M = 128 keys, N = NP, K = D twice (hi, then lo, into the same columns; at 8 rows, less than an MMA's
//                     columns, they lie side by side), both operands K-major
//   O^T += V^T P^T  : M = D, N = NP (2 x NP, hi | lo, where weights are codes), K = keys, both operands M/N-major
// so the tensor work goes with the query rows (NP = 8 .. 64), not with a padded 128, K and V tiles are read from shared
// memory once, and thread = key in the softmax.  A row's maximum then lies across the threads; it is looked for only
// when a weight would pass the largest there is (one vote per tile), which after a slab's first tiles is rare.
//
// Roles: groups of four softmax warps, two copy warps (TMA: K, V), two MMA warps (S, P.V), four warps that widen values
// (17 - 48 rows, and 64 of 64 dims); a persistent grid and the cost-balanced split of the key sequence that the other
// kernels use.  A group takes 8 or 16 of the query rows, thread = key: sixteen softmax warps fill an SM at 64 rows (one
// group of 64 rows spilled: 660 us for 198).  Up to 16 rows two CTAs share an SM, above one has it.  S and P
// have two buffers each.  A buffer's P.V is waited for by the S products' warp alone, whose scores then say to all softmax
// warps that S, P and W are free (each warp waiting for itself: 208 us for 201).  A tree is tile 0 of its slab: the softmax
// warps write its operands while the first copies are on their way.
//
// What bounds it, and what it takes: 64 nodes on 4 x 52 heads of 16384 keys 200 us, 4.4 TB/s of the cache, where the
// bytes alone take 130: a tile of 128 keys costs a CTA 1.14 us (at HBM's rate 0.74), spread over a softmax warp's chain
// of waits, loads, vote, weights and stores; issue slots are a little over half used.  26 nodes there 137 us, 12 nodes
// 135, one query 128.  26 nodes on 8 x 40 heads of 512 - 4096 keys: 56 us (bytes: 32), where a slab's start, in which
// its queries become operands, and the two tiles in which its maxima settle weigh in (23 us where a slab has 128 keys).
// 33 nodes of 4 query heads to a cached one: three row tiles of 44 that read the cache three times, from L2 twice, and
// widen its values three times: 83 us on 4 x 8 cached heads of 16384 keys.
//
// A slab whose keys lie in several CTAs' shares leaves partials (m, l, O) in the workspace and
// kv8_merge_kernel joins them.
#include <cuda.h>
#include <cuda_bf16.h>
#include <math_constants.h>

#include "attn_common.cuh"
#include "common.cuh"
#include "device.h"
#include "kernels.h"
#include "kv8.h"
#include "kv8_wait.cuh"
#include "tc_attn.cuh"
#include "tc_ptx.cuh"
#include "tensor_map.h"

namespace glide {
namespace {

constexpr int kTK = 128;          // keys per tile
constexpr int kTreeKeys = 64;     // rows of the tree tile
constexpr int kMaxStages8 = 6;
constexpr float kPLo = 28.f;         // p = hi + lo / kPLo: of p <= 430 at most 16 are left to lo, 448 its largest code
constexpr int kVExpSpan = 110, kVExpLeast = -90;  // see effective_exp
constexpr int kTreeExpMost = 20;                  // see tree_exp
constexpr float kNoM = -1.f;                      // of a row whose scores in the tree tile are all -inf: it has no m yet
constexpr int kQExpSpan = 3;                      // rows of queries share a power of two if it is within 2^3 of their own

// What a switch of slabs costs a CTA, in tiles (from 1 + np / 32 to 3 + np / 16: within 5% of each other, either way).
__host__ __device__ constexpr int seg_weight8(int np) { return 2 + np / 16; }

// barriers
constexpr int F_K = 0, F_V = 6, E_K = 12, E_V = 18, QFULL8 = 24, SFULL8 = 25, PFULL8 = 27, PVDONE = 29, MDONE8 = 31,
              WFULL = 33, kBars8 = 35;

template <int D, int NP>
struct Cfg {
  // Up to 16 rows: weights as two codes each, and two CTAs an SM, for which widened values leave no shared memory.  More:
  // values widened to fp16, work that the rows share, by warps that work beside the softmax (two codes / widened, us, when
  // this was chosen: 26 nodes on 4 x 52 heads of 16384 keys 145 / 137, on 8 x 40 heads of 512 - 4096 59 / 53, of 1024 35.4 /
  // 34.3, of 128 18.3 / 20.6; 32 nodes on 32 heads of 8192 25.9 / 21.8; 44 nodes on 4 x 52 heads of 16384 182 / 164).
  static constexpr bool kWiden = NP > 16;
  static constexpr float kMost = kWiden ? 15.5f : 8.75f;              // log2 of the largest weight: 2^16, 448 are too large
  static constexpr float kLift = kWiden ? 6.f : 8.f;                  // log2 of the weight of a new maximum
  static constexpr int kRT = NP < 16 ? NP : 16;                    // rows of a softmax group
  static constexpr int kSG = NP / kRT;                                // softmax groups
  static constexpr int kSoft = 128 * kSG;
  // Warps after the softmax: K's copies, V's copies, S products, P.V products.  One thread for both copies or both
  // products sets a slower pace than the stream: a copy or a product keeps its issuer busy for over 100 cycles.
  static constexpr int kCopyK = 4 * kSG, kCopyV = kCopyK + 1, kMmaS = kCopyK + 2, kMmaO = kCopyK + 3,
                       kWideW = kCopyK + 4;                           // the first that widens values
  // Four warps after those widen, beside the softmax (16384 keys, softmax warps / these, us, when this was chosen: 44 nodes
  // on 4 x 52 heads 177 / 164, 33 nodes of 4 query heads to each of 4 x 8 cached 90 / 84.5, 64 nodes on 4 x 52 heads of 64
  // dims 182 / 167).  With 64 rows of 128 dims they and the softmax take longer than the softmax alone: 216 / 200, half
  // each 240.
  static constexpr bool kWideWarps = kWiden && (NP < 64 || D == 64);
  static constexpr int kOwn = kWiden && !kWideWarps ? D / 16 / kSG : 0;  // else: pieces of 16 codes of a softmax group
  static constexpr int kThreads = kSoft + 128 + (kWideWarps ? 128 : 0);
  static constexpr int kCtas = kWiden ? 1 : 2;                        // of an SM
  // Each row's queries are scaled by a power of two of their own: always, or only where one is far smaller than another,
  // which takes the rows' largest and least element at a slab's start and leaves out a product per score (always / so, us:
  // 7 nodes on 4 x 40 heads of 322 - 2583 keys 18.0 / 18.9, 12 rows on 6 x 8 heads of 2005 - 16045 30.5 / 32.5, 33 nodes
  // of 4 query heads on 4 x 8 cached of 16384 83 / 87; 26 nodes on 8 x 40 ragged heads 60 / 57, 64 nodes on 4 x 52 heads
  // of 16384 207 / 199).
  static constexpr bool kRowScales = NP <= 16 || NP == 48;
  static constexpr int kBuf = 2;                                      // S and P buffers
  static constexpr int kNO = kWiden ? NP : 2 * NP;                      // columns of O (few rows: hi | lo)
  // S adds hi and lo up itself, as products along 2 D; 8 columns are less than an MMA has, so there they lie side by side.
  static constexpr bool kSplitS = NP < 16;
  static constexpr float kQLo = kSplitS ? 16.f : 1.f;                 // q = hi + lo / kQLo
  static constexpr int kNS = NP < 16 ? 16 : NP;                         // MMA columns of S
  static constexpr int kPitch = NP <= 16 ? 32 : (NP <= 32 ? 64 : 128);  // bytes of a key's weights
  static constexpr uint32_t kQBytes = 2 * NP * D;
  static constexpr uint32_t kWide = kTK * D * 2;                      // a tile of widened values
  static constexpr uint32_t kPBytes = kTK * kPitch;
  static constexpr uint32_t kTile = kTK * D;
  static constexpr uint32_t off_Q = 0;
  static constexpr uint32_t off_P = (kQBytes + 1023) / 1024 * 1024;
  static constexpr uint32_t off_W = off_P + kBuf * kPBytes;
  static constexpr uint32_t off_K = off_W + (kWiden ? kBuf * kWide : 0);
  static __host__ __device__ uint32_t off_V(int ns) { return off_K + ns * kTile; }
  static __host__ __device__ uint32_t off_small(int ns) { return off_V(ns) + ns * kTile; }
  static constexpr uint32_t kTmemS = kNS == 48 ? 64 : kNS;            // columns of an S buffer
  static constexpr uint32_t kTmemO = kBuf * kTmemS;                   // S buffers from column 0, then O
  static constexpr uint32_t kUsed = kTmemO + kNO;
  static constexpr uint32_t kCols = kUsed <= 32 ? 32 : kUsed <= 64 ? 64 : kUsed <= 128 ? 128 : 256;
};

struct Small {  // per CTA, after the rings
  uint64_t bars[kBars8];
  ShareStart share;
  unsigned long long sees[64];  // the rows' nodes and their ancestors
  alignas(16) float minus_m[64];  // what turns a row's u into its weight's logarithm
  alignas(16) float minus_up[64];  // by how much m rose last, negative; what turns a raw u into the logarithm
  alignas(16) float f[64];      // 2^(-up / 2), or kNoM; at the end 1 / l, or l
  alignas(16) float q_unit[64];    // what makes a row's scores log2 units where its queries have a scale of their own
  alignas(16) float part[4][64];  // per lane quarter: row maxima, row sums
  alignas(4) uint8_t rise[2][4][4];  // tiles in turn, per group and lane quarter: the chunks whose m rises
  alignas(16) int rel[64];                  // a row's place among a sequence's [node, head] rows from the slab's first head, -1: none
  uint2 top[16];                 // per softmax warp: the largest query element, the least of its rows' largest
  int8_t v_exp[kTreeKeys];       // the tree's nodes' value exponents
  uint32_t tmem;
  int abort_flag;
  int odd_values;               // the tree has values that are not finite
};

struct Params8 {
  const __nv_bfloat16 *q, *kt, *vt;
  const int8_t *Ke, *Ve;
  const int *kv_len, *parent;
  __nv_bfloat16* out;
  unsigned* status;
  int2* ranges;
  float* partials;
  int B, H, Hkv, S_cap, max_kv_len, n, group, rows, R, per_tile, tree, ns, blocks;
  float scale_log2;
};

// True in one lane of a converged warp.  The products and copies are issued behind it, by a warp whose loops all lanes
// run: the compiler then knows that one thread issues, and that its operands are the warp's.  Behind `lane == 0` every
// product took its issuer 120 - 210 cycles, behind this 60 - 70 (M = 128, N = 64: 8 fp16 products 978 -> 474 cycles).
__device__ __forceinline__ bool elect_one() {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
  return r != 0;
}
// Named barriers: 1 among all softmax threads, 2 + g within group g.
template <int kThreads>
__device__ __forceinline__ void soft_sync(int id) {
  asm volatile("bar.sync %0, %1;" ::"r"(id), "n"(kThreads) : "memory");
}
// The same, and whether any of the threads says so.
template <int kThreads>
__device__ __forceinline__ bool soft_any(int id, bool x) {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\t"
      "barrier.cta.red.or.pred q, %2, %3, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(r)
      : "r"((uint32_t)x), "r"(id), "n"(kThreads)
      : "memory");
  return r != 0;
}

// Shared-memory matrix descriptor; `pitch` (32, 64, 128 bytes) is the swizzle's width, 8 rows of it the
// stride between groups of 8 rows.
__device__ __forceinline__ uint64_t swizzled_desc(uint32_t saddr, int pitch) {
  const uint64_t mode = pitch == 128 ? 2 : (pitch == 64 ? 4 : 6);
  return (uint64_t)((saddr & 0x3FFFFu) >> 4) | (1ull << 16) | ((uint64_t)((8 * pitch) >> 4) << 32) | (1ull << 46) |
         (mode << 61);
}
// Where byte `c` of row `r` lies in a tile of that pitch.
template <int kPitch>
__device__ __forceinline__ uint32_t swizzled(uint32_t r, uint32_t c) {
  const uint32_t a = r * kPitch + c;
  return a ^ ((a >> 3) & (kPitch == 128 ? 0x70u : (kPitch == 64 ? 0x30u : 0x10u)));
}
// Instruction descriptor of kind::f8f6f4, both operands 8-bit floats of 4 exponent bits, fp32 sums.
__host__ __device__ constexpr uint32_t idesc_f8(int M, int N, bool a_mn, bool b_mn) {
  return (1u << 4) | ((a_mn ? 1u : 0u) << 15) | ((b_mn ? 1u : 0u) << 16) | ((uint32_t)(N >> 3) << 17) |
         ((uint32_t)(M >> 4) << 24);
}
__device__ __forceinline__ void mma_f8(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc,
                                       uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
      "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}

// 8 columns of this thread's TMEM lane (from each of two places), complete on return.  Loads and wait are one block of
// code: results that a later wait makes valid would have to be copied to keep their uses behind it.
__device__ __forceinline__ void tmem_ld8(uint32_t at, uint32_t (&r)[8]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
      : "r"(at)
      : "memory");
}
__device__ __forceinline__ void tmem_ld8x2(uint32_t at, uint32_t at2, uint32_t (&r)[8], uint32_t (&q)[8]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%16];\n\t"
      "tcgen05.ld.sync.aligned.32x32b.x8.b32 {%8, %9, %10, %11, %12, %13, %14, %15}, [%17];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(q[0]),
        "=r"(q[1]), "=r"(q[2]), "=r"(q[3]), "=r"(q[4]), "=r"(q[5]), "=r"(q[6]), "=r"(q[7])
      : "r"(at), "r"(at2)
      : "memory");
}
__device__ __forceinline__ void tmem_st8(uint32_t at, const uint32_t (&r)[8]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(at), "r"(r[0]),
               "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
               : "memory");
}

// Four floats times four in shared memory.
__device__ __forceinline__ void scale4(uint32_t* x, const float* f) {
  const ulonglong2 w = *reinterpret_cast<const ulonglong2*>(f);
  float y[4];
  unf2(f2mul(f2(__uint_as_float(x[0]), __uint_as_float(x[1])), w.x), y[0], y[1]);
  unf2(f2mul(f2(__uint_as_float(x[2]), __uint_as_float(x[3])), w.y), y[2], y[3]);
#pragma unroll
  for (int k = 0; k < 4; ++k) x[k] = __float_as_uint(y[k]);
}
// The largest of a value over the warp; NaN only if all are.
__device__ __forceinline__ float warp_top(float x) {
  float r;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(x));
  return r;
}

// Four weights in [0, 430] (or NaN) as codes hi and lo, p = hi + lo / 28: the fp16 in between has 11 bits.
// One block of code: the halves of a register are then picked by the conversions themselves.
__device__ __forceinline__ void split_weights(float p0, float p1, float p2, float p3, uint32_t& hi, uint32_t& lo) {
  asm("{\n\t.reg .b32 h, g, d;\n\t.reg .b16 a, b, c, e;\n\t"
      "cvt.rn.f16x2.f32 h, %3, %2;\n\t"
      "cvt.rn.f16x2.f32 g, %5, %4;\n\t"
      "cvt.rn.satfinite.e4m3x2.f16x2 a, h;\n\t"
      "cvt.rn.satfinite.e4m3x2.f16x2 b, g;\n\t"
      "mov.b32 %0, {a, b};\n\t"
      "cvt.rn.f16x2.e4m3x2 d, a;\n\t"
      "sub.rn.f16x2 h, h, d;\n\t"
      "cvt.rn.f16x2.e4m3x2 d, b;\n\t"
      "sub.rn.f16x2 g, g, d;\n\t"
      "mul.rn.f16x2 h, h, %6;\n\t"
      "mul.rn.f16x2 g, g, %6;\n\t"
      "cvt.rn.satfinite.e4m3x2.f16x2 c, h;\n\t"
      "cvt.rn.satfinite.e4m3x2.f16x2 e, g;\n\t"
      "mov.b32 %1, {c, e};\n\t}"
      : "=&r"(hi), "=r"(lo)
      : "f"(p0), "f"(p1), "f"(p2), "f"(p3), "r"(0x4f004f00u));  // 28, 28
}
// Four codes as four fp16 values, exactly.
__device__ __forceinline__ void widen4(uint32_t w, uint32_t& a, uint32_t& b) {
  asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, l;\n\tcvt.rn.f16x2.e4m3x2 %1, h;\n\t}"
      : "=r"(a), "=r"(b)
      : "r"(w));
}
// 16 codes as fp16 values to two places of a swizzled row (zeros if they are not there).
__device__ __forceinline__ void widen_piece(const unsigned char* from, unsigned char* row, uint32_t at, bool there) {
  uint4 w = *reinterpret_cast<const uint4*>(from);
  if (!there) w = make_uint4(0u, 0u, 0u, 0u);
  uint4 lo, hi;
  widen4(w.x, lo.x, lo.y);
  widen4(w.y, lo.z, lo.w);
  widen4(w.z, hi.x, hi.y);
  widen4(w.w, hi.z, hi.w);
  *reinterpret_cast<uint4*>(row + at) = lo;
  *reinterpret_cast<uint4*>(row + (at ^ 16)) = hi;
}
__device__ __forceinline__ uint32_t cvt_f16x2(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
// Eight bf16 elements times s as codes hi and lo, x = hi + lo / by; what is not finite becomes NaN.
__device__ __forceinline__ void split8(const uint4& w, float s, float by, uint2& hi, uint2& lo) {
  const uint32_t in[4] = {w.x, w.y, w.z, w.w};
  uint32_t h[4], l[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float a = bf16lo(in[i]) * s, b = bf16hi(in[i]) * s;  // finite ones are at most 448
    a = (in[i] & 0x7f80u) == 0x7f80u ? CUDART_NAN_F : a;
    b = (in[i] & 0x7f800000u) == 0x7f800000u ? CUDART_NAN_F : b;
    h[i] = kv8_encode2(a, b);
    const float2 was = kv8_f16pair(kv8_decode2_f16(h[i]));
    l[i] = kv8_encode2((a - was.x) * by, (b - was.y) * by);
  }
  hi = make_uint2(h[0] | (h[1] << 16), h[2] | (h[3] << 16));
  lo = make_uint2(l[0] | (l[1] << 16), l[2] | (l[3] << 16));
}
// The largest finite magnitude among eight bf16 elements (as its bits).
__device__ __forceinline__ uint32_t top8(const uint4& w) {
  const uint32_t in[4] = {w.x, w.y, w.z, w.w};
  uint32_t most = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t a = in[i] & 0x7fffu, b = (in[i] >> 16) & 0x7fffu;
    most = max(most, max(a < 0x7f80u ? a : 0u, b < 0x7f80u ? b : 0u));
  }
  return most;
}
// The largest magnitude among eight bf16 elements, infinities and NaN among them (as its bits).
__device__ __forceinline__ uint32_t top8_of_all(const uint4& w) {
  const uint32_t m = __vmaxu2(__vmaxu2(w.x & 0x7fff7fffu, w.y & 0x7fff7fffu), __vmaxu2(w.z & 0x7fff7fffu, w.w & 0x7fff7fffu));
  return max(m & 0xffffu, m >> 16);
}
// The largest finite one (which all are but seldom).
__device__ __forceinline__ uint32_t finite_top8(const uint4& w) {
  const uint32_t m = top8_of_all(w);
  return opaque(m >= 0x7f80u) ? top8(w) : m;
}
// Eight bf16 elements with zeros for those that are not finite; says whether there are any.
__device__ __forceinline__ bool drop_odd(uint4& w) {
  uint32_t in[4] = {w.x, w.y, w.z, w.w};
  bool odd = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if ((in[i] & 0x7f80u) == 0x7f80u) in[i] &= 0xffff0000u, odd = true;
    if ((in[i] & 0x7f800000u) == 0x7f800000u) in[i] &= 0xffffu, odd = true;
  }
  w = make_uint4(in[0], in[1], in[2], in[3]);
  return odd;
}
// The least e with x <= 448 * 2^e for the bf16 magnitude x with these bits.
__device__ __forceinline__ int top_exponent(uint32_t bits) {
  return kv8_clamp_exp((int)(bits >> 7) - 127 - 8 + ((bits & 0x7fu) > 0x60u ? 1 : 0));
}

// A block's value exponent as the weights take it.  A block of zero values has the least exponent there is; beside an
// ordinary block its weights would leave fp32's range, and the sum l with them.  So an exponent counts as at least
// 110 below the largest seen, and as -90: its values then show up 2^-102 of that block's largest at most.
__device__ __forceinline__ int effective_exp(int e, int ref) { return max(max(e, ref - kVExpSpan), kVExpLeast); }
// A tree node's value exponent, from the bits of its largest value: its own, as most rows do not see the node, but at least
// the cached blocks' (so that the first of these do not raise m).  Its values are multiplied as bf16, whose range lets the
// exponent stay within 110 of any other's.
__device__ __forceinline__ int tree_exp(uint32_t bits, int ref) {
  return min(max(max(top_exponent(bits), ref), kVExpLeast), kTreeExpMost);
}

template <int D, int NP>
__global__ void __launch_bounds__(Cfg<D, NP>::kThreads, Cfg<D, NP>::kCtas)
    kv8_attn_tc_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                       const Params8 p) {
  using C = Cfg<D, NP>;
  constexpr int RT = C::kRT, kSoft = C::kSoft, kBuf = C::kBuf;
  extern __shared__ unsigned char smem_raw[];
  unsigned char* base = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  const int ns = p.ns;
  const uint32_t off_V = C::off_V(ns);
  Small& sm = *reinterpret_cast<Small*>(base + C::off_small(ns));
  uint64_t* bars = sm.bars;
  volatile int* abort_flag = &sm.abort_flag;
  BatchTiles bt;
  bt.start = reinterpret_cast<long long*>(&sm + 1);
  bt.len = reinterpret_cast<int*>(bt.start + p.B + 1);
  bt.ntiles = bt.len + p.B;
  bt.plen = bt.ntiles + p.B;
  bt.sidx = bt.plen + p.B;
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    tc::prefetch_tmap(&tmK);
    tc::prefetch_tmap(&tmV);
    for (int b = 0; b < kBars8; ++b) {
      const bool soft = b == QFULL8 || (b >= PFULL8 && b < PVDONE), v_read = b >= E_V && b < QFULL8;
      mbar_init(&bars[b], soft || (v_read && C::kOwn) ? 4 * C::kSG : b >= WFULL || (v_read && C::kWideWarps) ? 4 : 1);
    }
    *abort_flag = 0;
    fence_barrier_init();
  }
  const int G = gridDim.x / p.R, x = blockIdx.x / p.R, y = blockIdx.x - x * p.R;
  const int row0 = y * p.per_tile, rows_here = min(p.per_tile, p.rows - row0);
  const int weight = seg_weight8(NP);
  if (threadIdx.x < 64) {
    const int r = threadIdx.x, node = (row0 + r) / p.group;
    sm.rel[r] = r < rows_here ? node * p.H + (row0 + r - node * p.group) : -1;
  }
  if (warp == 0) {
    wait_and_build_share(bt, p.kv_len, p.B, p.Hkv, p.max_kv_len, p.tree ? kTK : 0, kTK, G, weight, x, &sm.share);
    __syncwarp();
  } else {
    pdl_wait();
  }
  if (warp == C::kMmaS) {
    tc::tmem_alloc(&sm.tmem, C::kCols);
    tc::tmem_relinquish();
  }
  tc::fence_before_sync();
  __syncthreads();
  tc::fence_after_sync();
  const uint32_t tmem = sm.tmem;
  SegWalk s;
  s.start(bt, sm.share);

  if (warp == C::kCopyK || warp == C::kCopyV) {
    // -------------------------------------------------------------- copies
    const bool is_k = warp == C::kCopyK;
    const CUtensorMap* map = is_k ? &tmK : &tmV;
    uint64_t *full = &bars[is_k ? F_K : F_V], *empty = &bars[is_k ? E_K : E_V];
    unsigned char* dst = base + (is_k ? C::off_K : off_V);
    // one reader per tile: evict it first; R row tiles read each tile R times
    const uint64_t policy = p.R == 1 ? policy_evict_first() : policy_evict_normal();
    int st = 0;
    uint32_t phase = 1, out = 0, par = 0;  // out, par by stage: a copy issued, and the parity of its last one
    bool ok = true;
    for (; s.any() && ok; s.next(bt, p.Hkv)) {
      int row = (s.b * p.Hkv + s.h) * p.S_cap + (s.t0 - p.tree) * kTK;
      for (int t = s.t0; t < s.t1; ++t, row += kTK) {
        if (p.tree && t == 0) {  // the tree's: the softmax warps write it, K's part into K's ring
          if (C::kWiden && !is_k) continue;  // its values go into W
        } else {
          ok = warp_wait(&empty[st], phase, abort_flag);
          if (!ok) break;
          if (elect_one()) {
            mbar_arrive_expect_tx(&full[st], C::kTile);
            tc::tma_load_2d(dst + st * C::kTile, map, 0, row, &full[st], policy);
          }
          __syncwarp();
          out |= 1u << st;
          par = (par & ~(1u << st)) | ((phase ^ 1u) << st);
        }
        if (++st == ns) {
          st = 0;
          phase ^= 1;
        }
      }
    }
    if (!ok && lane == 0)  // aborted: issued copies land before the CTA exits
      for (int k = 0; k < ns; ++k)
        if ((out >> k) & 1u) mbar_drain(&full[k], (par >> k) & 1u);
  } else if (warp == C::kMmaS) {
    // ---------------------------------------------------------- S products
    constexpr uint32_t idS = idesc_f8(128, C::kNS, false, false);
    constexpr uint32_t idT = tc::idesc_bf16_f32(128, C::kNS, false, false);
    const uint64_t dQ = swizzled_desc(smem_u32(base + C::off_Q), D);
    const uint64_t dK0 = swizzled_desc(smem_u32(base + C::off_K), D);
    int st = 0, seg = 0, i = 0;
    uint32_t phase = 0;
    bool ok = true;
    for (; s.any() && ok; s.next(bt, p.Hkv), ++seg) {
      ok = warp_wait(&bars[QFULL8], seg & 1, abort_flag);
      for (int t = s.t0; t < s.t1 && ok; ++t, ++i) {
        const int buf = i % kBuf;
        // P.V of the tile that had the buffers is done: its scores were read before its weights were written, so S is free;
        // and these scores will tell the softmax that P and W are (one warp waits here for all of its warps).
        ok = warp_wait(&bars[F_K + st], phase, abort_flag) &&
             (i < kBuf || warp_wait(&bars[PVDONE + buf], (i - kBuf) / kBuf & 1, abort_flag));
        if (!ok) break;
        tc::fence_after_sync();
        const uint32_t tS = tmem + buf * C::kTmemS;
        if (p.tree && t == 0) {  // bf16 keys [D / 64][64 keys][64], bf16 queries [D / 64][kNS][64] in P's place
          const uint64_t dA = tc::sw128_desc(smem_u32(base + C::off_K + st * C::kTile), 16, 1024);
          const uint64_t dB = tc::sw128_desc(smem_u32(base + C::off_P + buf * C::kPBytes), 16, 1024);
          if (elect_one()) {
#pragma unroll
            for (int k = 0; k < D / 16; ++k)
              tc::mma_bf16(tS, dA + desc_step((k / 4) * kTreeKeys * 128 + (k % 4) * 32),
                           dB + desc_step((k / 4) * C::kNS * 128 + (k % 4) * 32), idT, k > 0);
            tc::mma_commit(&bars[SFULL8 + buf]);
            tc::mma_commit(&bars[E_K + st]);
          }
        } else {
          const uint64_t dK = dK0 + (uint64_t)st * desc_step(C::kTile);
          if (elect_one()) {
#pragma unroll
            for (int k = 0; k < D / 32; ++k) mma_f8(tS, dK + desc_step(32 * k), dQ + desc_step(32 * k), idS, k > 0);
            if (!C::kSplitS) {
#pragma unroll
              for (int k = 0; k < D / 32; ++k)
                mma_f8(tS, dK + desc_step(32 * k), dQ + desc_step(NP * D + 32 * k), idS, 1);
            }
            tc::mma_commit(&bars[SFULL8 + buf]);
            tc::mma_commit(&bars[E_K + st]);
          }
        }
        __syncwarp();
        if (++st == ns) {
          st = 0;
          phase ^= 1;
        }
      }
    }
    if (elect_one()) tc::mma_commit(&bars[MDONE8]);  // every MMA finished before TMEM is released
    __syncwarp();
    mbar_drain(&bars[MDONE8], 0);
  } else if (warp == C::kMmaO) {
    // -------------------------------------------------------- P.V products
    if (y == 0) write_ranges(bt, p.B, p.Hkv, G, weight, p.ranges, x * 32 + lane, G * 32);
    __syncwarp();
    constexpr uint32_t id8 = idesc_f8(D, C::kNO, true, true);
    constexpr uint32_t idT = tc::idesc_bf16_f32(D, C::kNS, true, true);
    constexpr uint32_t id16 = idT & ~((1u << 7) | (1u << 10));  // fp16 for bf16
    constexpr int kPitchP = C::kPitch;
    const uint64_t dP0 = swizzled_desc(smem_u32(base + C::off_P), kPitchP);
    const uint32_t values = smem_u32(base + (C::kWiden ? C::off_W : off_V));
    const uint64_t dV0 = C::kWiden ? tc::sw128_desc(values, kTK * 128, 1024) : swizzled_desc(values, D);
    const uint64_t dT0 = tc::sw128_desc(values, kTreeKeys * 128, 1024);
    int i = 0, st = 0;
    uint32_t phase = 0;
    bool ok = true;
    for (; s.any() && ok; s.next(bt, p.Hkv)) {
      for (int t = s.t0; t < s.t1; ++t, ++i) {
        const int buf = i % kBuf;
        // O of the segment before is read before the first weights of this one are written
        ok = (C::kOwn || warp_wait(C::kWiden ? &bars[WFULL + buf] : &bars[F_V + st], C::kWiden ? i / kBuf & 1 : phase,
                                   abort_flag)) &&
             warp_wait(&bars[PFULL8 + buf], i / kBuf & 1, abort_flag);
        if (!ok) break;
        tc::fence_after_sync();
        const uint64_t dP = dP0 + (uint64_t)buf * desc_step(C::kPBytes);
        const uint64_t at = C::kWiden ? (uint64_t)buf * desc_step(C::kWide) : (uint64_t)st * desc_step(C::kTile);
        const uint32_t tO = tmem + C::kTmemO;
        const uint32_t acc = t > s.t0 ? 1u : 0u;
        if (elect_one()) {
          if (p.tree && t == 0) {
#pragma unroll
            for (int k = 0; k < kTreeKeys / 16; ++k)
              tc::mma_bf16(tO, dT0 + at + desc_step(k * 16 * 128), dP + desc_step(k * 16 * kPitchP), idT, k > 0);
          } else if (C::kWiden) {
#pragma unroll
            for (int k = 0; k < kTK / 16; ++k)
              tc::mma_bf16(tO, dV0 + at + desc_step(k * 16 * 128), dP + desc_step(k * 16 * kPitchP), id16,
                           k > 0 ? 1u : acc);
          } else {
#pragma unroll
            for (int k = 0; k < kTK / 32; ++k)
              mma_f8(tO, dV0 + at + desc_step(k * 32 * D), dP + desc_step(k * 32 * kPitchP), id8, k > 0 ? 1u : acc);
          }
          tc::mma_commit(&bars[PVDONE + buf]);
          if (!C::kWiden) tc::mma_commit(&bars[E_V + st]);
        }
        __syncwarp();
        if (!C::kWiden && ++st == ns) {
          st = 0;
          phase ^= 1;
        }
      }
    }
    if (elect_one()) tc::mma_commit(&bars[MDONE8 + 1]);
    __syncwarp();
    mbar_drain(&bars[MDONE8 + 1], 0);
  } else if (C::kWideWarps && warp >= C::kWideW) {
    // ------------------------------------------------- values as fp16, exactly
    // Thread = key; zeros past the end (what lies there may be NaN, and zero times NaN is no zero).
    const int key = (warp - C::kWideW) * 32 + lane;
    const uint32_t x128 = (key & 7) << 4, xD = D == 128 ? x128 : ((key >> 1) & 3) << 4;
    int st = 0, i = 0;
    uint32_t phase = 0;
    bool ok = true;
    for (; s.any() && ok; s.next(bt, p.Hkv)) {
      const int plen = bt.plen[s.b];
      for (int t = s.t0; t < s.t1; ++t, ++i) {
        const int buf = i % kBuf;
        if (i >= kBuf) ok = warp_wait(&bars[PVDONE + buf], (i - kBuf) / kBuf & 1, abort_flag);
        if (!ok) break;
        if (!(p.tree && t == 0)) {  // the tree's are the softmax warps' to write
          ok = warp_wait(&bars[F_V + st], phase, abort_flag);
          if (!ok) break;
          const unsigned char* from = base + off_V + st * C::kTile + key * D;
          unsigned char* to = base + C::off_W + buf * C::kWide + key * 128;
          const bool there = (t - p.tree) * kTK + key < plen;
#pragma unroll
          for (int j = 0; j < D / 16; ++j)
            widen_piece(from + ((j * 16) ^ xD), to + (j / 4) * kTK * 128, (j % 4 * 32) ^ x128, there);
          __syncwarp();
          if (lane == 0) mbar_arrive(&bars[E_V + st]);
          if (++st == ns) {
            st = 0;
            phase ^= 1;
          }
        }
        tc::fence_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(&bars[WFULL + buf]);
      }
    }
  } else {
    // ------------------------------------------------------------- softmax
    const int sid = threadIdx.x, tid = sid & 127, group = warp >> 2;
    // tid: the key of a tile, and the value column of O^T; r_own: the group's first query row
    const int r_own = group * RT, quarter = warp & 3, gbar = 2 + group;
    const uint32_t lane_addr = tmem + ((uint32_t)(quarter * 32) << 16);
    const uint32_t tO = lane_addr + C::kTmemO + r_own;
    const uint32_t v_mix = (group * 16) ^ ((tid & 7) << 4), w_mix = (group * 32) ^ ((tid & 7) << 4);
    const uint32_t p_row = tid * C::kPitch,
                   p_mix = C::kPitch == 128 ? (tid & 7) << 4 : (C::kPitch == 64 ? ((tid >> 1) & 3) << 4 : ((tid >> 2) & 1) << 4);
    bool dead = false;
    int st = 0, vst = 0, i = 0;  // stages of K (and V, where values are not widened) and V, tiles so far
    int sees_b = -1;             // the sequence that sm.sees is of
    uint32_t ring = 0, v_ring = 0;
    // P.V of tile j of this CTA is done
    auto wait_pv = [&](int j) {
      if (j >= 0) dead |= !warp_wait(&bars[PVDONE + j % C::kBuf], j / C::kBuf & 1, abort_flag);
    };
    if (!p.tree) {  // zeros for sequences without cached keys
      const long long per = (long long)p.n * p.H * D;
      for (int b = 0; b < p.B; ++b)
        if (bt.ntiles[b] == 0)
          for (long long e = (long long)blockIdx.x * kSoft + sid; e < per; e += (long long)gridDim.x * kSoft)
            p.out[b * per + e] = __float2bfloat16_rn(0.f);
    }
    for (; s.any(); s.next(bt, p.Hkv)) {
      const int plen = bt.plen[s.b], slab = s.b * p.Hkv + s.h;
      const bool tree_here = p.tree && s.t0 == 0;
      const int8_t *Ke = p.Ke + (size_t)slab * p.blocks, *Ve = p.Ve + (size_t)slab * p.blocks;
      const int used = kv8_blocks(plen);
      // What 32 blocks (16 tiles) make of scores and weights, a lane's own: the upper halves of the fp32 numbers 2^eK
      // (low half) and eV (high half), and 2^-eV.
      uint32_t scales = 0;
      float inv = 0.f;
      int ref = -128;
      auto fetch = [&](int block) {
        const int at = min(block + lane, used - 1);
        return make_int2(Ke[at], Ve[at]);
      };
      auto set_scales = [&](int2 raw) {
        const int ek = kv8_clamp_exp(raw.x), ev = kv8_clamp_exp(raw.y);
        ref = max(ref, __reduce_max_sync(0xffffffffu, ev));
        const int e = effective_exp(ev, ref);
        scales = (uint32_t)(ek + 127) << 7 | (__float_as_uint((float)e) & 0xffff0000u);
        inv = kv8_pow2(-e);
      };
      // Everything that the segment's start reads from global memory is on its way before any of it is used.
      int2 raw = make_int2(0, 0), up = make_int2(-1, -1);
      if (used > 0) raw = fetch(tree_here ? 0 : 2 * (s.t0 - p.tree));
      const bool walk = tree_here && s.b != sees_b;  // the rows' ancestors, the same for a sequence's heads
      if (walk && quarter == 0) up = parents_of(p.parent + (size_t)s.b * p.n, p.n, lane);

      // ---- the segment's queries, and the tree's own keys and values, as operands
      const int first_tile = i;
      float a_q = 1.f;    // what makes a score of S and of 2^eK
      bool apart = true;  // each row's queries are scaled by a power of two of its own
      {
        constexpr int kPerRow = D / 8, kQ = (NP * kPerRow + kSoft - 1) / kSoft,
                      kT = (kTreeKeys * kPerRow + kSoft - 1) / kSoft;
        const uint4 none = make_uint4(0u, 0u, 0u, 0u);
        auto over_row = [](uint32_t x) {  // the largest of a row's pieces, which kPerRow neighbouring lanes have
          uint32_t r = 0;
#pragma unroll
          for (int g = 0; g < 32 / kPerRow; ++g) {
            const bool mine = (threadIdx.x & 31) / kPerRow == g;
            const uint32_t y = __reduce_max_sync(0xffffffffu, mine ? x : 0u);
            r = mine ? y : r;
          }
          return r;
        };
        uint4 q[kQ], kt[kT], v[kT];
        uint32_t most = 0, least = ~0u, row_top[kQ];
        const size_t q0 = (size_t)s.b * p.n * p.H + (size_t)s.h * p.group;
#pragma unroll
        for (int i = 0; i < kQ; ++i) {
          const int c = sid + i * kSoft, r = c / kPerRow;
          q[i] = none;
          if (r < rows_here) q[i] = reinterpret_cast<const uint4*>(p.q + (q0 + sm.rel[r]) * D)[c % kPerRow];
        }
        if (tree_here) {
#pragma unroll
          for (int i = 0; i < kT; ++i) {
            const int c = sid + i * kSoft, r = c / kPerRow, d = c % kPerRow * 8;
            kt[i] = v[i] = none;
            if (r < p.n) {  // p.n <= kTreeKeys
              const size_t at = (((size_t)s.b * p.n + r) * p.Hkv + s.h) * D + d;
              kt[i] = *reinterpret_cast<const uint4*>(p.kt + at);
              v[i] = *reinterpret_cast<const uint4*>(p.vt + at);
            }
          }
        }
        if constexpr (!C::kRowScales) {
#pragma unroll
          for (int i = 0; i < kQ; ++i) {
            row_top[i] = over_row(finite_top8(q[i]));
            most = max(most, row_top[i]);
            if (row_top[i] != 0) least = min(least, row_top[i]);
          }
        }
        // Byte of element d of row r in a bf16 operand of `rows` rows: 64 elements (128 bytes) a row and part.
        auto in_bf16 = [](int r, int d, int rows) { return (d / 64) * rows * 128 + swizzled<128>(r, (d % 64) * 2); };
        bool odd = false;
        if (tree_here) {
          dead |= !warp_wait(&bars[E_K + st], ring ^ 1, abort_flag);
          if (!C::kWiden) dead |= !warp_wait(&bars[E_V + st], ring ^ 1, abort_flag);
          unsigned char* kd = base + C::off_K + st * C::kTile;
#pragma unroll
          for (int i = 0; i < kT; ++i) {
            const int c = sid + i * kSoft, r = c / kPerRow, d = c % kPerRow * 8;
            if (kTreeKeys * kPerRow % kSoft != 0 && r >= kTreeKeys) continue;
            *reinterpret_cast<uint4*>(kd + in_bf16(r, d, kTreeKeys)) = kt[i];
          }
#pragma unroll
          for (int i = 0; i < kT; ++i)
            // An unseen value that is not finite must not meet a weight of zero: it is left out here, and put
            // back at the end where it is seen.
            if (opaque(top8_of_all(v[i]) >= 0x7f80u)) odd |= drop_odd(v[i]);
          unsigned char* qd = base + C::off_P + first_tile % C::kBuf * C::kPBytes;  // P of this tile comes later
#pragma unroll
          for (int i = 0; i < kQ; ++i) {
            const int c = sid + i * kSoft, r = c / kPerRow, d = c % kPerRow * 8;
            if (r < NP) *reinterpret_cast<uint4*>(qd + in_bf16(r, d, C::kNS)) = q[i];
          }
          if (NP < C::kNS && sid < (C::kNS - NP) * kPerRow)
            *reinterpret_cast<uint4*>(qd + in_bf16(NP + sid / kPerRow, sid % kPerRow * 8, C::kNS)) = none;
        }
        if (!C::kRowScales) {
          most = __reduce_max_sync(0xffffffffu, most);
          least = __reduce_min_sync(0xffffffffu, least);
          if (lane == 0) sm.top[warp] = make_uint2(most, least);
        }
        const bool odd_any = soft_any<kSoft>(1, odd);  // a barrier too
        if (sid == 0) sm.odd_values = odd_any;
#pragma unroll
        for (int w = 0; w < (C::kRowScales ? 0 : 4 * C::kSG); ++w) {
          most = max(most, sm.top[w].x);
          least = min(least, sm.top[w].y);
        }
        if (used > 0) set_scales(raw);
        if (tree_here) {
          unsigned char* vd =  // W's buffer is free, as P's is
              base + (C::kWiden ? C::off_W + first_tile % kBuf * C::kWide : off_V + st * C::kTile);
#pragma unroll
          for (int i = 0; i < kT; ++i) {
            const int c = sid + i * kSoft, r = c / kPerRow, d = c % kPerRow * 8;
            if (kTreeKeys * kPerRow % kSoft != 0 && r >= kTreeKeys) continue;  // whole warps
            int e = kVExpLeast;
            e = tree_exp(over_row(top8_of_all(v[i])), ref);
            const float vs = kv8_pow2(-e);
            const uint4 w = v[i];
            *reinterpret_cast<uint4*>(vd + in_bf16(r, d, kTreeKeys)) =
                make_uint4(pack_bf16x2(bf16lo(w.x) * vs, bf16hi(w.x) * vs), pack_bf16x2(bf16lo(w.y) * vs, bf16hi(w.y) * vs),
                           pack_bf16x2(bf16lo(w.z) * vs, bf16hi(w.z) * vs), pack_bf16x2(bf16lo(w.w) * vs, bf16hi(w.w) * vs));
            if (d == 0) sm.v_exp[r] = (int8_t)e;
          }
        }
        // The rows' largest elements decide one power of two, unless a row is so small that its codes would be coarse.
        int q_exp = 0;
        if constexpr (!C::kRowScales) {
          q_exp = top_exponent(most);
          apart = most != 0 && top_exponent(least) < q_exp - kQExpSpan;
          if (!apart) a_q = p.scale_log2 * kv8_pow2(q_exp);
        }
#pragma unroll
        for (int i = 0; i < kQ; ++i) {
          const int c = sid + i * kSoft, r = c / kPerRow, d = c % kPerRow * 8;
          const uint32_t top = C::kRowScales ? over_row(finite_top8(q[i])) : row_top[i];
          if (r < NP) {
            const int e = apart ? top_exponent(top) : q_exp;
            uint2 hi, lo;
            split8(q[i], kv8_pow2(-e), C::kQLo, hi, lo);
            if (d == 0) sm.q_unit[r] = p.scale_log2 * kv8_pow2(e);
            *reinterpret_cast<uint2*>(base + C::off_Q + swizzled<D>(r, d)) = hi;
            *reinterpret_cast<uint2*>(base + C::off_Q + swizzled<D>(NP + r, d)) = lo;
          }
        }
        tc::fence_async_smem();
        soft_sync<kSoft>(1);
        if (lane == 0) mbar_arrive(&bars[QFULL8]);
        if (tree_here && sid == 0) {
          mbar_arrive(&bars[F_K + st]);
          if (!C::kWiden) mbar_arrive(&bars[F_V + st]);
        }
      }

      uint64_t l2[RT / 2];  // pairs of rows
#pragma unroll
      for (int k = 0; k < RT / 2; ++k) l2[k] = 0ull;
      if (walk) {  // while the first product runs
        if (quarter == 0) {
          const int r = r_own + lane;
          const unsigned long long set = ancestors(up, p.n, r < rows_here ? (row0 + r) / p.group : 0, true, lane);
          if (lane < RT) sm.sees[r] = set;
        }
        sees_b = s.b;
        soft_sync<128>(gbar);
      }
      int nth = 0;  // of the blocks whose scales the lanes hold
      auto scales_of = [&](float& a, float& ef, float& inv_v) {  // the next cached tile's
        const uint32_t mine = __shfl_sync(0xffffffffu, scales, nth + (tid >> 6));
        inv_v = __shfl_sync(0xffffffffu, inv, nth + (tid >> 6));
        a = a_q * __uint_as_float(mine << 16);
        ef = __uint_as_float(mine & 0xffff0000u);
        nth += 2;
      };
      auto first_scales = [&](float& a, float& ef, float& inv_v) {  // the segment's first tile's
        if (tree_here) {
          a = p.scale_log2;
          ef = 0.f;  // each key has its own: below
          inv_v = 1.f;
        } else {
          scales_of(a, ef, inv_v);
        }
      };
      // Where one CTA has an SM, a tile's scales are made ready during the tile before it (44 nodes on 4 x 52 heads of
      // 16384 keys: 164 -> 161 us);
      // two have no registers for that (12 nodes on 8 x 40 heads of 1024 keys: 28.2 -> 30.5).
      float a_next, ef_next, inv_next;
      if (C::kWiden) first_scales(a_next, ef_next, inv_next);
      int late = -1;  // the tile that gives an m to rows that the tree's, with infinite keys, left without
      for (int t = s.t0; t < s.t1; ++t, ++i) {
        const bool is_tree = p.tree && t == 0, first = t == s.t0, raw = first || t == late;
        const int key0 = (t - p.tree) * kTK, buf = i % kBuf;
        if (opaque(nth == 32)) {  // the next 16 tiles' (past a slab's last block: that one's, for nothing)
          set_scales(fetch((t + (C::kWiden ? 1 : 0) - p.tree) * (kTK / kKv8Block)));
          nth = 0;
        }
        float a, ef, inv_v;
        if (C::kWiden)
          a = a_next, ef = ef_next, inv_v = inv_next;
        else if (first)
          first_scales(a, ef, inv_v);
        else
          scales_of(a, ef, inv_v);
        dead |= !warp_wait(&bars[SFULL8 + buf], i / C::kBuf & 1, abort_flag);
        tc::fence_after_sync();
        if (C::kOwn && !is_tree) {  // this group's pieces of the key's values
          dead |= !warp_wait(&bars[F_V + vst], v_ring, abort_flag);
          const unsigned char* from = base + off_V + vst * C::kTile + tid * D;
          unsigned char* to = base + C::off_W + buf * C::kWide + tid * 128;
#pragma unroll
          for (int j = 0; j < C::kOwn; ++j)  // four groups, 128 dims: of 4 pieces in a half row, group's is its own
            widen_piece(from + (v_mix ^ (j * 64)), to + j * kTK * 128, w_mix, key0 + tid < plen);
          __syncwarp();
          if (lane == 0) mbar_arrive(&bars[E_V + vst]);
          if (++vst == ns) {
            vst = 0;
            v_ring ^= 1;
          }
        }
        // ---- u = S a + e, less m (none yet in a segment's first tile)
        float u[RT];
        const uint32_t tS = lane_addr + buf * C::kTmemS + r_own;
        if (!C::kWiden && NP >= 16 && opaque(is_tree)) {  // this tile starts O, and its product leaves the lower parts out
          const uint32_t none[8] = {};
#pragma unroll 1
          for (int c = 0; c < RT; c += 8) tmem_st8(tO + NP + c, none);
          tc::tmem_wait_st();
        }
        {
#pragma unroll
          for (int c = 0; c < RT; c += 16) {
            constexpr int CH = 8;
            uint32_t x[CH], z[CH];  // split: hi, lo; else rows c .. c + 7, rows c + 8 .. c + 15
            tmem_ld8x2(tS + c, tS + c + (C::kSplitS ? NP : 8), x, z);
            if (opaque(apart && !is_tree)) {  // the rows' own scales; the tree's queries are not scaled
#pragma unroll
              for (int k = 0; k < CH; k += 4) {
                scale4(x + k, &sm.q_unit[r_own + c + k]);
                scale4(z + k, &sm.q_unit[r_own + c + (C::kSplitS ? 0 : 8) + k]);
              }
            } else if (C::kSplitS) {  // columns without a query, NaN for an infinite key
#pragma unroll
              for (int k = 0; k < CH; ++k) z[k] = 0u;
            }
            const uint64_t a2 = f2(a, a), ef2 = f2(ef, ef);
            auto pair = [](const uint32_t* x) { return f2(__uint_as_float(x[0]), __uint_as_float(x[1])); };
#pragma unroll
            for (int k = 0; k < CH; k += 2) {
              if constexpr (C::kSplitS) {
                const uint64_t lo2 = f2(a / C::kQLo, a / C::kQLo);
                unf2(ffma2(pair(x + k), a2, ffma2(pair(z + k), lo2, ef2)), u[c + k], u[c + k + 1]);
              } else {
                unf2(ffma2(pair(x + k), a2, ef2), u[c + k], u[c + k + 1]);
                if (c + 8 + k < RT) unf2(ffma2(pair(z + k), a2, ef2), u[c + 8 + k], u[c + 9 + k]);
              }
            }
          }
        }
        if (opaque(is_tree || key0 + kTK > plen)) {  // which rows see this thread's key
          uint32_t vis = key0 + tid < plen ? ~0u : 0u;
          if (is_tree) {
            const float e = (float)sm.v_exp[tid % kTreeKeys];
#pragma unroll
            for (int k = 0; k < RT; ++k) u[k] += e;
            vis = 0;
            if (tid < p.n)
#pragma unroll 4
              for (int r = 0; r < RT; ++r) vis |= (uint32_t)((sm.sees[r_own + r] >> tid) & 1ull) << r;
          }
#pragma unroll
          for (int k = 0; k < RT; ++k) u[k] = (vis >> k) & 1u ? u[k] : -CUDART_INF_F;
        }
        if (C::kWiden) scales_of(a_next, ef_next, inv_next);
        uint32_t rise = (1u << RT / 8) - 1u;  // by chunks of 8 rows
        if (!raw) {
          rise = 0;
#pragma unroll
          for (int c = 0; c < RT; c += 8) {
            float top = -CUDART_INF_F;
#pragma unroll
            for (int k = c; k < c + 8; k += 4) {
              const ulonglong2 m = *reinterpret_cast<const ulonglong2*>(&sm.minus_m[r_own + k]);
              unf2(fadd2(f2(u[k], u[k + 1]), m.x), u[k], u[k + 1]);
              unf2(fadd2(f2(u[k + 2], u[k + 3]), m.y), u[k + 2], u[k + 3]);
              top = fmax3(fmax3(top, u[k], u[k + 1]), u[k + 2], u[k + 3]);
            }
            if (top > C::kMost) rise |= 1u << c / 8;
          }
          rise = __reduce_or_sync(0xffffffffu, rise);
          if (lane == 0) sm.rise[t & 1][group][quarter] = (uint8_t)rise;
          soft_sync<128>(gbar);
          rise = *reinterpret_cast<const uint32_t*>(sm.rise[t & 1][group]);
          rise = (rise | rise >> 16);
          rise = (rise | rise >> 8) & 0xffu;
        }
        // A new m for the rows whose weights would pass the largest code.  l holds 2^-eV and so may be far larger than the
        // weights that it sums: it takes 2^-up in two steps, neither of which leaves fp32's range before the result does.
        if (opaque(rise != 0)) {
#pragma unroll
          for (int c = 0; c < RT; c += 8) {
            if (!((rise >> c / 8) & 1u)) continue;
            float mine = 0.f;  // lane k: the largest of row c + k
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              const float v = warp_top(u[c + k]);
              mine = lane == k ? v : mine;
            }
            if (lane < 8) sm.part[quarter][r_own + c + lane] = mine;
          }
          soft_sync<128>(gbar);
          if (tid < RT && (rise >> tid / 8) & 1u) {
            const int r = r_own + tid;
            const float top = fmaxf(fmaxf(sm.part[0][r], sm.part[1][r]), fmaxf(sm.part[2][r], sm.part[3][r]));
            // a row with nothing but NaN has no m, and keeps none
            float up = first || top > C::kMost || top != top ? top - C::kLift : 0.f, f = first ? 0.f : fast_exp2(-0.5f * up);
            const float was = first ? 0.f : sm.minus_m[r];
            float add = -up;
            if (opaque(t == late)) {  // u holds no m yet
              const bool fresh = sm.f[r] == kNoM;
              const float now = top + was;
              up = fresh || now > C::kMost || now != now ? now - C::kLift : 0.f;
              f = fresh ? 0.f : fast_exp2(-0.5f * up);
              add = was - up;
            }
            if (opaque(first && top == -CUDART_INF_F)) up = add = 0.f, f = kNoM;
            sm.minus_m[r] = was - up;
            sm.minus_up[r] = add;
            sm.f[r] = f;
          }
          soft_sync<128>(gbar);
#pragma unroll
          for (int c = 0; c < RT; c += 8) {
            if (!((rise >> c / 8) & 1u)) continue;
#pragma unroll
            for (int k = c; k < c + 8; ++k) {
              u[k] += sm.minus_up[r_own + k];
              if (k % 2 == 0) {
                const uint64_t f = *reinterpret_cast<const uint64_t*>(&sm.f[r_own + k]);
                l2[k / 2] = f2mul(f2mul(l2[k / 2], f), f);
              }
            }
          }
          if (opaque(is_tree) && __any_sync(0xffffffffu, sm.f[r_own + lane % RT] == kNoM)) late = 1;
        }

        // ---- weights: p = 2^(u - m), l += p 2^-e, in bf16 beside the tree's bf16 values, in fp16 beside widened
        // ones, else as two codes
        unsigned char* const p_to = base + C::off_P + buf * C::kPBytes + p_row;
        if (opaque(is_tree)) {
          const float inv_v = kv8_pow2(-sm.v_exp[tid % kTreeKeys]);
#pragma unroll
          for (int c = 0; c < RT; c += 8) {
            uint32_t w[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const float v0 = fast_exp2(u[c + 2 * k]), v1 = fast_exp2(u[c + 2 * k + 1]);
              l2[c / 2 + k] = ffma2(f2(v0, v1), f2(inv_v, inv_v), l2[c / 2 + k]);
              w[k] = pack_bf16x2(v0, v1);
            }
            *reinterpret_cast<uint4*>(p_to + ((2 * (r_own + c)) ^ p_mix)) = make_uint4(w[0], w[1], w[2], w[3]);
          }
          if (NP < C::kNS) *reinterpret_cast<uint4*>(p_to + ((2 * NP) ^ p_mix)) = make_uint4(0u, 0u, 0u, 0u);
        } else if constexpr (C::kWiden) {
#pragma unroll
          for (int c = 0; c < RT; c += 8) {
            uint32_t w[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const float v0 = fast_exp2(u[c + 2 * k]), v1 = fast_exp2(u[c + 2 * k + 1]);
              l2[c / 2 + k] = ffma2(f2(v0, v1), f2(inv_v, inv_v), l2[c / 2 + k]);
              w[k] = cvt_f16x2(v0, v1);
            }
            *reinterpret_cast<uint4*>(p_to + ((2 * (r_own + c)) ^ p_mix)) = make_uint4(w[0], w[1], w[2], w[3]);
          }
        } else {
          uint32_t hw[RT / 4], lw[RT / 4];
#pragma unroll
          for (int k = 0; k < RT / 4; ++k) {
            const float v0 = fast_exp2(u[4 * k]), v1 = fast_exp2(u[4 * k + 1]);
            const float v2 = fast_exp2(u[4 * k + 2]), v3 = fast_exp2(u[4 * k + 3]);
            l2[2 * k] = ffma2(f2(v0, v1), f2(inv_v, inv_v), l2[2 * k]);
            l2[2 * k + 1] = ffma2(f2(v2, v3), f2(inv_v, inv_v), l2[2 * k + 1]);
            split_weights(v0, v1, v2, v3, hw[k], lw[k]);
          }
          if constexpr (NP == 8) {
            *reinterpret_cast<uint4*>(p_to + p_mix) = make_uint4(hw[0], hw[1], lw[0], lw[1]);
          } else {
            *reinterpret_cast<uint4*>(p_to + (r_own ^ p_mix)) = make_uint4(hw[0], hw[1], hw[2], hw[3]);
            *reinterpret_cast<uint4*>(p_to + ((NP + r_own) ^ p_mix)) = make_uint4(lw[0], lw[1], lw[2], lw[3]);
          }
          if (opaque(key0 + kTK > plen)) {  // value rows past the end may hold NaN: zero times NaN is no zero
            dead |= !warp_wait(&bars[F_V + st], ring, abort_flag);
            if (key0 + tid >= plen) {
              uint4* row = reinterpret_cast<uint4*>(base + off_V + st * C::kTile + tid * D);
#pragma unroll
              for (int c = 0; c < D / 16; ++c) row[c] = make_uint4(0u, 0u, 0u, 0u);
            }
          }
        }
        if (opaque(rise != 0 && !first)) {  // what O holds so far, to the new m, before this tile's P.V adds to it
          wait_pv(i - 1);
          tc::fence_after_sync();
#pragma unroll 1
          for (int c = 0; c < RT; c += 8) {
            if (!((rise >> c / 8) & 1u)) continue;
            uint32_t o[8];
#pragma unroll 1
            for (int half = 0; half < (C::kWiden ? 1 : 2); ++half) {
              tmem_ld8(tO + half * NP + c, o);
#pragma unroll
              for (int k = 0; k < 8; ++k)
                o[k] = __float_as_uint(__uint_as_float(o[k]) * sm.f[r_own + c + k] * sm.f[r_own + c + k]);
              tmem_st8(tO + half * NP + c, o);
            }
          }
          tc::tmem_wait_st();
        }
        tc::fence_async_smem();
        tc::fence_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive(&bars[PFULL8 + buf]);
        if (++st == ns) {
          st = 0;
          ring ^= 1;
        }
      }

      // ---- the segment's end: l over the threads, then O / l or a partial
      {
        float l[RT];
#pragma unroll
        for (int k = 0; k < RT / 2; ++k) unf2(l2[k], l[2 * k], l[2 * k + 1]);
        // Halving exchanges, while the rows can be halved: each leaves a lane half as many rows, summed over
        // twice as many lanes.
        int r0 = 0;
#pragma unroll
        for (int off = 16, cnt = RT; off >= 1; off >>= 1) {
          if (cnt % 2 == 0) {
            const bool upper = (lane & off) != 0;
            cnt /= 2;
#pragma unroll
            for (int j = 0; j < RT / 2; ++j) {
              if (j < cnt) {
                const float send = upper ? l[j] : l[j + cnt], keep = upper ? l[j + cnt] : l[j];
                l[j] = keep + __shfl_xor_sync(0xffffffffu, send, off);
              }
            }
            r0 += upper ? cnt : 0;
          } else {
#pragma unroll
            for (int j = 0; j < RT / 2; ++j)
              if (j < cnt) l[j] += __shfl_xor_sync(0xffffffffu, l[j], off);
          }
          if (off == 1)
#pragma unroll
            for (int j = 0; j < RT / 2; ++j)
              if (j < cnt) sm.part[quarter][r_own + r0 + j] = l[j];
        }
      }
      soft_sync<128>(gbar);
      const bool whole = s.whole(bt);
      if (tid < RT) {
        const int r = r_own + tid;
        const float sum = (sm.part[0][r] + sm.part[1][r]) + (sm.part[2][r] + sm.part[3][r]);
        sm.f[r] = whole ? 1.f / sum : sum;
      }
      soft_sync<128>(gbar);
      wait_pv(i - 1);
      tc::fence_after_sync();
      // D = 64: an accumulator of 64 rows keeps rows 16 w .. 16 w + 15 in lanes 32 w .. 32 w + 15
      const int d = D == 128 ? tid : quarter * 16 + lane;
      const bool has = D == 128 || lane < 16;
      const bool odd = tree_here && sm.odd_values;
      float* part = partial_slot(p.partials, x + slab, p.rows, D) + (size_t)row0 * (D + 2);
      const size_t o0 = (size_t)s.b * p.n * p.H + (size_t)s.h * p.group;
      if (!whole && tid < RT && !dead && sm.rel[r_own + tid] >= 0)
        *reinterpret_cast<float2*>(part + (size_t)(r_own + tid) * (D + 2)) =
            make_float2(sm.f[r_own + tid] == 0.f ? -CUDART_INF_F : -sm.minus_m[r_own + tid], sm.f[r_own + tid]);
      const bool live = has && !dead;
#pragma unroll 1
      for (int c = 0; c < RT; c += 8) {
        uint32_t acc[8], low[8];
        float o[8];
        if (C::kWiden)
          tmem_ld8(tO + c, acc);
        else
          tmem_ld8x2(tO + c, tO + NP + c, acc, low);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          o[k] = __uint_as_float(acc[k]);
          if (!C::kWiden) o[k] = fmaf(__uint_as_float(low[k]), 1.f / kPLo, o[k]);
        }
        if (opaque(odd) && live) {  // a visible value that is not finite decides its column
#pragma unroll 1
          for (int j = 0; j < p.n; ++j) {
            const float v = __bfloat162float(p.vt[(((size_t)s.b * p.n + j) * p.Hkv + s.h) * D + d]);
            if (isfinite(v)) continue;
#pragma unroll
            for (int k = 0; k < 8; ++k)
              if ((sm.sees[r_own + c + k] >> j) & 1ull) o[k] += v;
          }
        }
        const int4 ra = *reinterpret_cast<const int4*>(&sm.rel[r_own + c]),
                   rb = *reinterpret_cast<const int4*>(&sm.rel[r_own + c + 4]);
        const int rel[8] = {ra.x, ra.y, ra.z, ra.w, rb.x, rb.y, rb.z, rb.w};
        if (whole) {
          const float4 fa = *reinterpret_cast<const float4*>(&sm.f[r_own + c]),
                       fb = *reinterpret_cast<const float4*>(&sm.f[r_own + c + 4]);
          const float f[8] = {fa.x, fa.y, fa.z, fa.w, fb.x, fb.y, fb.z, fb.w};
          __nv_bfloat16* to = p.out + o0 * D + d;
#pragma unroll
          for (int k = 0; k < 8; ++k)
            if (live && rel[k] >= 0) to[(size_t)rel[k] * D] = __float2bfloat16_rn(o[k] * f[k]);
        } else {
          float* to = part + (size_t)(r_own + c) * (D + 2) + 2 + d;
#pragma unroll
          for (int k = 0; k < 8; ++k)
            if (live && rel[k] >= 0) to[k * (D + 2)] = o[k];
        }
      }
      tc::fence_before_sync();
      soft_sync<kSoft>(1);  // m, f, sees and O are free for the next segment
    }
  }

  __syncwarp();
  tc::fence_before_sync();
  __syncthreads();
  if (threadIdx.x == 0) record_abort(abort_flag, p.status);
  if (warp == C::kMmaS) {
    tc::fence_after_sync();
    tc::tmem_dealloc(tmem, C::kCols);
  }
}

// Joins the partials of every split slab, one warp per query row: with M the largest m,
//   out = sum_c 2^(m_c - M) o_c / sum_c 2^(m_c - M) l_c.
// l is a sum of 2^-eV, so its share's weight is taken in the logarithm: either may leave fp32's range.  An o's weight
// is at least the least number there is: zero times an infinite o, of an infinite value, were NaN.
constexpr int kMergeW = 8;
template <int D>
__global__ void __launch_bounds__(kMergeW * 32) kv8_merge_kernel(const int2* ranges, const float* partials,
                                                                 __nv_bfloat16* out, int BH, int rows, int group,
                                                                 int Hq, int Hkv) {
  constexpr int kPairs = D / 64;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const float least = __int_as_float(1);
  const int lane = threadIdx.x & 31;
  const unsigned total = (unsigned)BH * (unsigned)rows, step = gridDim.x * kMergeW;
  pdl_wait();
  for (unsigned wr = blockIdx.x * kMergeW + (threadIdx.x >> 5); wr < total; wr += step) {
    const int bh = (int)(wr / (unsigned)rows), r = (int)(wr - (unsigned)bh * (unsigned)rows);
    const int b = bh / Hkv, h = bh - b * Hkv;
    const int2 rg = __ldcg(&ranges[bh]);
    if (rg.x < 0) continue;
    const size_t stride = (size_t)rows * (D + 2);
    const float* row0 = partials + (size_t)(rg.x + bh) * stride + (size_t)r * (D + 2);
    const int shares = rg.y - rg.x + 1;
    float M = -CUDART_INF_F, L = 0.f;
    float2 acc[kPairs];
#pragma unroll
    for (int k = 0; k < kPairs; ++k) acc[k] = make_float2(0.f, 0.f);
    for (int c0 = 0; c0 < shares; c0 += 8) {
      float2 ml[8], o[8][kPairs];
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const float* pr = row0 + (size_t)(c0 + u < shares ? c0 + u : c0) * stride;
        ml[u] = __ldcg(reinterpret_cast<const float2*>(pr));
#pragma unroll
        for (int k = 0; k < kPairs; ++k) o[u][k] = __ldcg(reinterpret_cast<const float2*>(pr + 2 + 64 * k + 2 * lane));
      }
      float now = M;
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if (c0 + u < shares) now = fmaxf(now, ml[u].x);
      const float f = M == -CUDART_INF_F ? 0.f : fmaxf(fast_exp2(M - now), least);
      if (M != -CUDART_INF_F) {
        L = L > 0.f ? fast_exp2(M - now + __log2f(L)) : L;
#pragma unroll
        for (int k = 0; k < kPairs; ++k) acc[k] = make_float2(acc[k].x * f, acc[k].y * f);
      }
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        if (c0 + u >= shares) break;
        const float w = fmaxf(fast_exp2(ml[u].x - now), least);
        L += fast_exp2(ml[u].x - now + __log2f(ml[u].y));
#pragma unroll
        for (int k = 0; k < kPairs; ++k) {
          acc[k].x += w * o[u][k].x;
          acc[k].y += w * o[u][k].y;
        }
      }
      M = now;
    }
    const float inv = 1.f / L;
    __nv_bfloat16* dst = out + out_row(b, h, r, rows, group, Hq) * D;
#pragma unroll
    for (int k = 0; k < kPairs; ++k)
      *reinterpret_cast<uint32_t*>(dst + 64 * k + 2 * lane) = pack_bf16x2(acc[k].x * inv, acc[k].y * inv);
  }
}

// ------------------------------------------------------------------- host
// A [rows, D] matrix of codes in boxes of kTK whole rows, swizzled by the row's width.
bool make_code_map(CUtensorMap* m, const void* base, long long rows, int D) {
  PFN_cuTensorMapEncodeTiled_v12000 fn = tensor_map_encoder();
  if (!fn) return false;
  const cuuint64_t dims[2] = {(cuuint64_t)D, (cuuint64_t)rows};
  const cuuint64_t strides[1] = {(cuuint64_t)D};
  const cuuint32_t box[2] = {(cuuint32_t)D, kTK};
  const cuuint32_t es[2] = {1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(base), dims, strides, box, es,
            CU_TENSOR_MAP_INTERLEAVE_NONE, D == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

constexpr int kMaxShares = 1024;

template <int D, int NP>
cudaError_t launch_np(const Kv8AttnArgs& a, int R, int per_tile, cudaStream_t st) {
  using C = Cfg<D, NP>;
  static PerDevice<int> allowed;
  const int limit = smem_optin_bytes();
  cudaError_t e = allow_smem(allowed, kv8_attn_tc_kernel<D, NP>, limit);
  if (e != cudaSuccess) return e;
  auto bytes = [&](int ns) {
    return (size_t)1024 + C::off_small(ns) + sizeof(Small) + (size_t)(a.B + 1) * 8 + (size_t)(4 * a.B + 1) * 4;
  };
  int ns = kMaxStages8;  // as many stages as let the SM's CTAs share it (228 KB, 1 KB of it each CTA's own)
  while (ns > 2 && bytes(ns) > (size_t)(limit + 1024) / C::kCtas - 1024) --ns;
  if (bytes(ns) > (size_t)limit) return cudaErrorNotSupported;
  CUtensorMap mk, mv;
  const long long rows = (long long)a.B * a.Hkv * a.S_cap;
  if (!make_code_map(&mk, a.K, rows, D) || !make_code_map(&mv, a.V, rows, D)) return cudaErrorNotSupported;
  const int tree = a.parent != nullptr;
  const long long tiles = (long long)a.B * a.Hkv * ((a.max_kv_len + kTK - 1) / kTK + tree);
  long long G = (a.max_ctas > 0 ? a.max_ctas : C::kCtas * sm_count()) / R;
  if (G > kMaxShares) G = kMaxShares;
  if (G > tiles) G = tiles;
  if (G < 1) G = 1;
  Params8 p;
  p.q = static_cast<const __nv_bfloat16*>(a.q);
  p.kt = static_cast<const __nv_bfloat16*>(a.kt);
  p.vt = static_cast<const __nv_bfloat16*>(a.vt);
  p.Ke = a.Ke; p.Ve = a.Ve; p.kv_len = a.kv_len; p.parent = a.parent;
  p.out = static_cast<__nv_bfloat16*>(a.out);
  unsigned char* ws = static_cast<unsigned char*>(a.ws);
  p.status = reinterpret_cast<unsigned*>(ws);
  p.ranges = reinterpret_cast<int2*>(ws + WsLayout::kZeros);
  p.partials = reinterpret_cast<float*>(ws + WsLayout::align(WsLayout::kZeros + 8 * (size_t)a.B * a.Hkv));
  p.B = a.B; p.H = a.H; p.Hkv = a.Hkv; p.S_cap = a.S_cap; p.max_kv_len = a.max_kv_len; p.n = a.nq;
  p.group = a.H / a.Hkv; p.rows = a.nq * p.group; p.R = R; p.per_tile = per_tile; p.tree = tree; p.ns = ns;
  p.blocks = kv8_blocks(a.S_cap);
  p.scale_log2 = a.scale * kLog2e;
  e = launch_pdl(kv8_attn_tc_kernel<D, NP>, dim3((unsigned)(G * R)), dim3(C::kThreads), bytes(ns), st, mk, mv, p);
  if (e != cudaSuccess) return e;
  long long grid = ((long long)a.B * a.Hkv * p.rows + kMergeW - 1) / kMergeW;
  if (grid > 8LL * sm_count()) grid = 8LL * sm_count();
  return launch_pdl(kv8_merge_kernel<D>, dim3((unsigned)grid), dim3(kMergeW * 32), 0, st, p.ranges, p.partials, p.out,
                    a.B * a.Hkv, p.rows, p.group, a.H, a.Hkv);
}

template <int D>
cudaError_t launch_d(const Kv8AttnArgs& a, cudaStream_t st) {
  const int rows = a.nq * (a.H / a.Hkv);
  const int R = (rows + 63) / 64, per = (rows + R - 1) / R;
  if (per <= 8) return launch_np<D, 8>(a, R, per, st);
  if (per <= 16) return launch_np<D, 16>(a, R, per, st);
  if (per <= 32) return launch_np<D, 32>(a, R, per, st);
  if (per <= 48) return launch_np<D, 48>(a, R, per, st);
  return launch_np<D, 64>(a, R, per, st);
}

}  // namespace

size_t kv8_workspace_bytes(int B, int Hkv, int D, int rows) {
  return WsLayout::align(WsLayout::kZeros + 8 * (size_t)B * Hkv) +
         ((size_t)kMaxShares + (size_t)B * Hkv) * rows * (D + 2) * sizeof(float);
}

cudaError_t launch_kv8_attn_tc(const Kv8AttnArgs& a, cudaStream_t st) {
  if (a.dtype != 0) return cudaErrorNotSupported;
  // 32-bit TMA coordinates and tile counts
  if ((long long)a.B * a.Hkv * a.S_cap > 0x7fffffffLL - kTK) return cudaErrorNotSupported;
  return a.D == 128 ? launch_d<128>(a, st) : launch_d<64>(a, st);
}

}  // namespace glide
