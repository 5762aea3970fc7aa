// Attention of packed rows of new tokens (chunks over a paged cache, whole prompts over themselves) on the tcgen05
// tensor cores.
//
// The mathematics: row i of a sequence's m new tokens sees its keys t <= kv - m + i.  u = (q . k) scale log2(e),
// p = 2^(u - r) with r a running reference maximum, out = sum p v / sum p:
//   S = Q K^T   : M = 128 rows, N = 128 keys, K = D, operands in shared memory (128-byte swizzle)
//   O += P V    : M = 128, N = D, K = 128 keys, P (bf16) in tensor memory over its S, V in shared memory
// A row tile packs the H / H_kv query heads that share a cached head: row r is token r / group, head r % group, so
// 128 / group tokens and every key once for the whole group.
//
// What bounds it: the tensor pipe, two products of ~520 cycles for a row tile and 128 keys, as long as nothing waits.  A
// work item therefore has two row tiles, each with a softmax group of four warps, a product issuer and its S and O in tensor
// memory: while one tile's scores are exponentiated the pipe works on the other's.  A thread holds its row of 128
// scores in registers (one read of S), and hands P over in two halves of 64 keys, so that P V starts under the
// second half's exponentials.  Both tiles use the same K and V stages: half the loads of one tile alone.
//
// Work items are (cached head, 2 x 128 / group tokens, keys), claimed from a counter: cached heads in groups whose keys and
// values together stay in L2, in them the row tiles with the most keys first, so that the SMs end together.  Where there are
// fewer than two items for an SM, an item's keys are cut into chunks; partial results (max, sum, o) go through the
// workspace, and the warp that finishes an item's last chunk merges its rows in the chunks' order.
//
// Roles (512 threads, one CTA per SM):
//   warps 0-3, 4-7  softmax of row tile 0 and 1, one thread a row; they rescale O where the reference is raised (by
//                   more than 8, so seldom).
//   warps 8-11      results: a TMEM lane quarter each of both tiles, O / l through 4 KB of shared memory in whole rows.
//   warp 12         claims items, loads Q and K (a page's rows at a time, or 128 packed rows); warp 13 loads V and clears its
//                   rows past an item's last visible key.
//   warps 14, 15    the products of row tile 0 and 1 (lane 0).
// S of a tile overwrites P of the tile before, so its issuer waits for that P V to complete; O is only touched by
// the softmax warps between that point and their hand-over of P.
//
// A result that is not finite (an infinity or NaN that the row sees, or one that it does not see, in a tile
// that it shares) is computed again by the definition, the row alone.
#include <cuda.h>
#include <cuda_bf16.h>
#include <math_constants.h>

#include "device.h"
#include "kernels.h"
#include "rows_attn.cuh"
#include "tc_attn.cuh"
#include "tc_ptx.cuh"
#include "tensor_map.h"

namespace glide {
namespace {

constexpr int kBM = 128;          // rows of a row tile (MMA rows, TMEM lanes)
constexpr int kBN = 128;          // keys of a tile
constexpr int kOutWarp0 = 8;
constexpr int kKWarp = 12;
constexpr int kVWarp = 13;
constexpr int kMmaWarp0 = 14;
constexpr int kTcThreads = 512;
constexpr int kTmemCols = 512;
constexpr uint32_t kAtom = 128 * 128;  // one 128-byte-swizzle atom of 128 rows
constexpr float kRescaleLog2 = 8.0f;
constexpr int kItemSlots = 2;
constexpr int kItemReaders = 15;       // warps that read an item beside the one that makes it
constexpr int kMaxGrid = 160;
constexpr int kMaxChunks = 3 * kMaxGrid;  // partial slots: below 2 grids of items and one grid more of chunks
constexpr int kMinChunkTiles = 4;
constexpr int kSortMost = 128;         // sequences that are taken in the order of their keys
constexpr long long kL2Bytes = 48ll << 20;

// Workspace: status word, the claim counter and the count of finished CTAs in the header, arrival counters [chunk slot]
// [quarter], then partial slots.
constexpr size_t kCountOff = WsLayout::kHeader;
constexpr size_t kPartOff = (kCountOff + kMaxChunks * 4 * sizeof(unsigned) + 255) / 256 * 256;

struct Bars {
  uint64_t kfull[4], kempty[4], vfull[4], vempty[4], vclr[4];
  uint64_t qfull[2], qempty[2], sfull[2], pfull[2][2], pvdone[2], olast[2], ofree[2], lready[2], lfree[2];
  uint64_t itemfull[kItemSlots], itemempty[kItemSlots];
  uint64_t drained[2];
};

struct TcItem {
  int b;                  // -1: no more
  int h, row0, m, kv, rows, pos0;
  int t0, te0, te1;       // key tiles of the two row tiles: [t0, te0) and [t0, te1)
  int klen;               // keys that some row of the item sees
  int chunks, chunk, slot, slot_step;  // chunks of the item, this one, its partial slot, slots from chunk to chunk
  __device__ __forceinline__ int end() const { return te0 > te1 ? te0 : te1; }
  __device__ __forceinline__ int stop(int g) const { return g ? te1 : te0; }
};

template <int D>
struct TcCfg {
  static constexpr int kHalves = D / 64;
  static constexpr uint32_t kTile = kHalves * kAtom;  // 128 rows x D
  static constexpr unsigned kNS = D == 128 ? 2 : 4;   // stages of the K ring and of the V ring
  static constexpr uint32_t off_Q = 0;
  static constexpr uint32_t off_K = 2 * kTile;
  static constexpr uint32_t off_V = off_K + kNS * kTile;
  static constexpr uint32_t off_stage = off_V + kNS * kTile;  // 4 KB for each of the result warps
  static constexpr uint32_t off_bar = off_stage + 4 * 4096;
  static constexpr uint32_t off_item = off_bar + sizeof(Bars);
  static constexpr uint32_t off_misc = (off_item + kItemSlots * sizeof(TcItem) + 15) / 16 * 16;
  static constexpr uint32_t off_ml = off_misc + 64;                 // [tile][row] maxima, then sums
  static constexpr uint32_t off_order = off_ml + 2 * 2 * kBM * 4;
  static constexpr size_t kSmem = 1024 + off_order + kSortMost * 4;
  static_assert(kSmem <= 227 * 1024, "shared memory");
  static constexpr uint32_t kColS = 0, kColO = 2 * kBN;             // TMEM columns: S0, S1, O0, O1
  static_assert(kColO + 2 * D <= kTmemCols, "TMEM columns");
};

struct TcParams {
  RowsParams r;
  unsigned char* ws;
  int tokens;      // of a row tile: 128 / group
  int box_rows;    // key rows of one TMA box: a page's, at most 128
  int part_rows;   // rows of a partial slot: 128 or 256
};

struct Misc {
  uint32_t tmem;
  int abort;
  int head_group;      // cached heads that are worked on together
  int chunk_tiles;     // key tiles of a chunk
  int entries;         // (sequence, row tiles, chunk) triples
  int levels;          // the most row tile pairs of a sequence
  long long sum[3];
};

// Row-tile pairs of a sequence, and the keys that the last row of pair x sees.
__device__ __forceinline__ int pairs_of(const Seq& s, int tokens) { return (s.rows + 2 * tokens - 1) / (2 * tokens); }
__device__ __forceinline__ int keys_of(const Seq& s, int tokens, int x) {
  const int last = (x + 1) * 2 * tokens;
  return seen(s, (last < s.rows ? last : s.rows) - 1);
}
__device__ __forceinline__ int chunks_of(const Seq& s, int tokens, int x, int chunk_tiles) {
  if (x >= pairs_of(s, tokens)) return 0;
  const int nt = (keys_of(s, tokens, x) + kBN - 1) / kBN;
  return nt <= chunk_tiles ? 1 : (nt + chunk_tiles - 1) / chunk_tiles;
}

template <int N>
__device__ __forceinline__ void tc_regs_up() {
  asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N) : "memory");
}
template <int N>
__device__ __forceinline__ void tc_regs_down() {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N) : "memory");
}

// The items as every other warp reads them.
struct ItemReader {
  unsigned n = 0;
  __device__ __forceinline__ bool next(Bars* bars, const TcItem* items, TcItem& it, volatile int* abort, int lane) {
    const unsigned slot = n % kItemSlots, phase = (n / kItemSlots) & 1;
    ++n;
    if (!warp_wait_small(&bars->itemfull[slot], phase, abort)) return false;
    it = items[slot];
    __syncwarp();
    if (lane == 0) mbar_arrive(&bars->itemempty[slot]);
    return it.b >= 0;
  }
};

template <int D>
__global__ void __launch_bounds__(kTcThreads, 1)
    rows_tc_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                   const __grid_constant__ CUtensorMap tmV, const TcParams p) {
  using C = TcCfg<D>;
  extern __shared__ unsigned char smem_raw[];
  unsigned char* base = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  Bars* bars = reinterpret_cast<Bars*>(base + C::off_bar);
  TcItem* items = reinterpret_cast<TcItem*>(base + C::off_item);
  Misc* misc = reinterpret_cast<Misc*>(base + C::off_misc);
  float* m_row = reinterpret_cast<float*>(base + C::off_ml);
  float* l_row = m_row + 2 * kBM;
  int* order = reinterpret_cast<int*>(base + C::off_order);
  volatile int* abort_flag = &misc->abort;
  unsigned* status = reinterpret_cast<unsigned*>(p.ws);
  unsigned* claim = reinterpret_cast<unsigned*>(p.ws + WsLayout::kClaimOff);
  unsigned* finished = reinterpret_cast<unsigned*>(p.ws + WsLayout::kDoneOff);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const RowsParams& rp = p.r;
  if (threadIdx.x == 0) {
    const auto init = [](uint64_t* b, int n, int count) {
#pragma unroll 1
      for (int i = 0; i < n; ++i) mbar_init(b + i, count);
    };
    init(bars->kfull, 4, 1);
    init(bars->kempty, 4, 2);
    init(bars->vfull, 4, 1);
    init(bars->vempty, 4, 2);
    init(bars->vclr, 4, 1);
    init(bars->qfull, 2, 1);
    init(bars->qempty, 2, 1);
    init(bars->sfull, 2, 1);
    init(&bars->pfull[0][0], 4, 4);
    init(bars->pvdone, 2, 1);
    init(bars->olast, 2, 1);
    init(bars->ofree, 2, 4);
    init(bars->lready, 2, 4);
    init(bars->lfree, 2, 4);
    init(bars->itemfull, kItemSlots, 1);
    init(bars->itemempty, kItemSlots, kItemReaders);
    init(bars->drained, 2, 1);
    misc->abort = 0;
    misc->levels = 0;
    misc->sum[0] = misc->sum[1] = misc->sum[2] = 0;
    fence_barrier_init();
  }
  __syncthreads();
  pdl_wait();  // every global access and the TMEM allocation come after it
  if (warp == kKWarp) {
    tc::tmem_alloc(&misc->tmem, kTmemCols);
    tc::tmem_relinquish();
  }
  // ---- the plan of the call: what all CTAs find alike from the lengths
  {
    long long pairs = 0, units = 0, keys = 0;
    int levels = 0;
#pragma unroll 1
    for (int b = threadIdx.x; b < rp.B; b += kTcThreads) {
      const Seq s = seq_of(rp, b);
      const int n = pairs_of(s, p.tokens);
      const int mean = s.kv - s.m + (s.rows + 1) / 2;
      pairs += n;
      units += (long long)n * (((mean > 0 ? mean : 0) + kBN) / kBN);
      keys += s.kv;
      levels = n > levels ? n : levels;
    }
    if (pairs) {
      atomicAdd(reinterpret_cast<unsigned long long*>(&misc->sum[0]), (unsigned long long)pairs);
      atomicAdd(reinterpret_cast<unsigned long long*>(&misc->sum[1]), (unsigned long long)units);
      atomicAdd(reinterpret_cast<unsigned long long*>(&misc->sum[2]), (unsigned long long)keys);
      atomicMax(&misc->levels, levels);
    }
    if (rp.B <= kSortMost && threadIdx.x < rp.B) {  // the most keys first
      const int mine = seq_of(rp, threadIdx.x).kv;
      int before = 0;
#pragma unroll 1
      for (int x = 0; x < rp.B; ++x) {
        const int other = seq_of(rp, x).kv;
        before += other > mine || (other == mine && x < threadIdx.x);
      }
      order[before] = threadIdx.x;
    }
    __syncthreads();
    const long long n_items = misc->sum[0] * rp.Hkv, n_units = misc->sum[1] * rp.Hkv;
    int chunk = 0x7fffffff;
    if (n_items < 2ll * gridDim.x) {  // an SM's share of the key tiles
      const long long c = (n_units + gridDim.x - 1) / gridDim.x;
      chunk = c < kMinChunkTiles ? kMinChunkTiles : (int)c;
    }
    if (threadIdx.x == 0) {
      const long long bytes = misc->sum[2] * D * 4;  // keys and values of a cached head
      const long long g = bytes > 0 ? kL2Bytes / bytes : rp.Hkv;
      misc->head_group = (int)(g < 1 ? 1 : (g > rp.Hkv ? rp.Hkv : g));
    }
    // whole items need no slots; chunks grow until there is one for each (no more than the items, then)
#pragma unroll 1
    while (true) {
      int entries = 0;
#pragma unroll 1
      for (int b = threadIdx.x; b < rp.B; b += kTcThreads) {
        const Seq s = seq_of(rp, b);
        const int n = pairs_of(s, p.tokens);
        if (chunk == 0x7fffffff) {
          entries += n;
        } else {
#pragma unroll 1
          for (int x = 0; x < n; ++x) entries += chunks_of(s, p.tokens, x, chunk);
        }
      }
      if (threadIdx.x == 0) misc->entries = 0;
      __syncthreads();
      if (entries) atomicAdd(&misc->entries, entries);
      __syncthreads();
      const int total = misc->entries;
      __syncthreads();
      if (chunk == 0x7fffffff || (long long)total * rp.Hkv <= kMaxChunks) break;
      chunk = chunk > 0x3fffffff ? 0x7ffffffe : 2 * chunk;
    }
    if (threadIdx.x == 0) misc->chunk_tiles = chunk;
  }
  tc::fence_before_sync();
  __syncthreads();
  tc::fence_after_sync();
  const uint32_t tmem = misc->tmem;

  if (warp >= kKWarp) {
    tc_regs_down<56>();
    if (warp == kKWarp || warp == kVWarp) {
      // ------------------------------------------------------------ loads
      const bool keys = warp == kKWarp;
      const uint64_t pol_q = policy_evict_first(), pol_kv = policy_evict_last();
      const CUtensorMap* map = keys ? &tmK : &tmV;
      if (lane == 0) {
        tc::prefetch_tmap(map);
        if (keys) tc::prefetch_tmap(&tmQ);
      }
      unsigned char* ring = base + (keys ? C::off_K : C::off_V);
      uint64_t* full = keys ? bars->kfull : bars->vfull;
      uint64_t* empty = keys ? bars->kempty : bars->vempty;
      unsigned st = 0, phase = 1, issued = 0, q_issued[2] = {0, 0};
      bool ok = true;
      // the items: made here (by the K warp) or read
      ItemReader reader;
      unsigned made = 0;
      int level = misc->levels - 1, block = 0, acc = 0, group_at = 0;
      const int entries = misc->entries, head_group = misc->head_group, chunk_tiles = misc->chunk_tiles;
      const long long claims = (long long)entries * rp.Hkv;
      unsigned next = blockIdx.x;
      TcItem it;
      while (ok) {
        if (keys) {
          const unsigned c = next;
          if (lane == 0) next = gridDim.x + atomicAdd(claim, 1u);
          next = __shfl_sync(0xffffffffu, next, 0);
          it.b = -1;
          if ((long long)c < claims) {
            const long long per_group = (long long)entries * head_group;
            const int hg = (int)(c / per_group), in_group = (int)(c - hg * per_group);
            const int left = rp.Hkv - hg * head_group, heads = left < head_group ? left : head_group;
            const int e = in_group / heads;
            if (hg != group_at) {
              group_at = hg;
              level = misc->levels - 1;
              block = acc = 0;
            }
            // entry e: level by level from the last rows on, in a level by sequence
#pragma unroll 1
            while (level >= 0) {
              const int at = block * 32 + lane;
              int n = 0, b = 0;
              Seq s = {0, 0, 0, 0};
              if (at < rp.B) {
                b = rp.B <= kSortMost ? order[at] : at;
                s = seq_of(rp, b);
                n = chunks_of(s, p.tokens, level, chunk_tiles);
              }
              int upto = n;
#pragma unroll
              for (int off = 1; off < 32; off <<= 1) {
                const int u = __shfl_up_sync(0xffffffffu, upto, off);
                if (lane >= off) upto += u;
              }
              const int total = __shfl_sync(0xffffffffu, upto, 31);
              if (e < acc + total) {
                const int who = __ffs(__ballot_sync(0xffffffffu, e < acc + upto)) - 1;
                it.b = __shfl_sync(0xffffffffu, b, who);
                it.chunks = __shfl_sync(0xffffffffu, n, who);
                it.chunk = e - acc - (__shfl_sync(0xffffffffu, upto, who) - it.chunks);
                it.row0 = __shfl_sync(0xffffffffu, s.row0, who);
                it.m = __shfl_sync(0xffffffffu, s.m, who);
                it.kv = __shfl_sync(0xffffffffu, s.kv, who);
                it.rows = __shfl_sync(0xffffffffu, s.rows, who);
                break;
              }
              acc += total;
              if (++block * 32 >= rp.B) {
                block = 0;
                --level;
              }
            }
            if (it.b >= 0) {
              it.h = hg * head_group + (in_group - e * heads);
              it.pos0 = level * 2 * p.tokens;
              const Seq s = {it.row0, it.rows, it.m, it.kv};
              it.klen = keys_of(s, p.tokens, level);
              it.slot = (int)c;
              it.slot_step = heads;
              it.t0 = it.chunks > 1 ? it.chunk * chunk_tiles : 0;
              const int nt = (it.klen + kBN - 1) / kBN;
              const int end = it.chunks > 1 && nt - it.t0 > chunk_tiles ? it.t0 + chunk_tiles : nt;
#pragma unroll
              for (int g = 0; g < 2; ++g) {
                const int first = it.pos0 + g * p.tokens, stop = first + p.tokens;
                int n = 0;
                if (first < it.rows) n = (seen(s, (stop < it.rows ? stop : it.rows) - 1) + kBN - 1) / kBN;
                n = n < end ? n : end;
                (g ? it.te1 : it.te0) = n > it.t0 ? n : it.t0;
              }
            }
          }
          const unsigned slot = made % kItemSlots;
          ok = warp_wait_small(&bars->itemempty[slot], ((made / kItemSlots) & 1) ^ 1, abort_flag);
          if (!ok) break;
          ++made;
          if (lane == 0) {
            items[slot] = it;
            mbar_arrive(&bars->itemfull[slot]);
          }
          __syncwarp();
          if (it.b < 0) break;
#pragma unroll
          for (int g = 0; g < 2; ++g) {
            if (it.stop(g) == it.t0) continue;
            ok = warp_wait_small(&bars->qempty[g], (q_issued[g] & 1) ^ 1, abort_flag);
            if (!ok) break;
            if (lane == 0) {
              mbar_arrive_expect_tx(&bars->qfull[g], (uint32_t)(C::kHalves * p.tokens * rp.group * 128));
              for (int hd = 0; hd < C::kHalves; ++hd)
                tc::tma_load_3d(base + C::off_Q + g * C::kTile + hd * kAtom, &tmQ, hd * 64, it.h * rp.group,
                                it.row0 + it.pos0 + g * p.tokens, &bars->qfull[g], pol_q);
            }
            __syncwarp();
            ++q_issued[g];
          }
          if (!ok) break;
        } else if (!reader.next(bars, items, it, abort_flag, lane)) {
          break;
        }
        const int end = it.end();
#pragma unroll 1
        for (int t = it.t0; t < end; ++t) {
          ok = warp_wait_small(&empty[st], phase, abort_flag);
          if (!ok) break;
          unsigned char* dst = ring + st * C::kTile;
          const int left = it.klen - t * kBN;
          if (!rp.table) {
            if (lane == 0) {
              mbar_arrive_expect_tx(&full[st], C::kTile);
              for (int hd = 0; hd < C::kHalves; ++hd)
                tc::tma_load_3d(dst + hd * kAtom, map, hd * 64, it.h, it.row0 + t * kBN, &full[st], pol_kv);
            }
          } else {
            // the pages that hold keys of this tile: a lane for each box
            const int need = left < kBN ? left : kBN, boxes = (need + p.box_rows - 1) / p.box_rows;
            if (lane == 0) mbar_arrive_expect_tx(&full[st], (uint32_t)(boxes * C::kHalves * p.box_rows * 128));
            __syncwarp();
            const int x = lane / C::kHalves, hd = lane - x * C::kHalves;
            if (x < boxes) {
              const int key = t * kBN + x * p.box_rows;
              const int page = page_at(rp, it.b, key >> rp.page_shift);
              tc::tma_load_3d(dst + hd * kAtom + x * p.box_rows * 128, map, hd * 64, key & ((1 << rp.page_shift) - 1),
                              page * rp.Hkv + it.h, &full[st], pol_kv);
            }
          }
          __syncwarp();
          ++issued;
          if (!keys && left < kBN) {  // the item's last V tile: clear its rows past the last visible key
            ok = warp_wait_small(&full[st], phase ^ 1, abort_flag);
            if (!ok) break;
#pragma unroll 1
            for (int idx = left * C::kHalves * 8 + lane; idx < kBN * C::kHalves * 8; idx += 32)
              *reinterpret_cast<uint4*>(dst + ((idx >> 3) % C::kHalves) * kAtom + idx / (C::kHalves * 8) * 128 +
                                        (idx & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
            tc::fence_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(&bars->vclr[st]);
          }
          if (++st == C::kNS) {
            st = 0;
            phase ^= 1;
          }
        }
      }
      if (!ok) {  // aborted: let issued loads land before the CTA exits
        for (unsigned j = issued > C::kNS ? issued - C::kNS : 0; j < issued; ++j)
          mbar_drain(&full[j % C::kNS], (j / C::kNS) & 1);
        for (int g = 0; g < 2; ++g)
          if (q_issued[g]) mbar_drain(&bars->qfull[g], (q_issued[g] - 1) & 1);
      }
    } else {
      // ------------------------------------------------------------ products of row tile g
      const int g = warp - kMmaWarp0;
      constexpr uint32_t idS = tc::idesc_bf16_f32(kBM, kBN, false, false);
      constexpr uint32_t idO = tc::idesc_bf16_f32(kBM, D, false, true);
      const uint64_t dQ = tc::sw128_desc(smem_u32(base + C::off_Q + g * C::kTile), 16, 1024);
      const uint64_t dK0 = tc::sw128_desc(smem_u32(base + C::off_K), 16, 1024);
      const uint64_t dV0 = tc::sw128_desc(smem_u32(base + C::off_V), kAtom, 1024);
      const uint32_t colS = tmem + C::kColS + g * kBN, colO = tmem + C::kColO + g * D;
      unsigned st = 0, phase = 0, cleared = 0;  // both rings move together: one K and one V tile a step
      unsigned n_q = 0, n_tiles = 0, n_items = 0;
      bool ok = true;
      ItemReader reader;
      TcItem it;
      while (ok && reader.next(bars, items, it, abort_flag, lane)) {
        const int end = it.end(), mine = it.stop(g);
        if (lane == 0) {
          if (mine > it.t0) {
            ok = mbar_wait_small(&bars->qfull[g], n_q & 1, abort_flag);
            ++n_q;
          }
#pragma unroll 1
          for (int t = it.t0; ok && t < end; ++t) {
            const bool clear = it.klen - t * kBN < kBN;
            ok = mbar_wait_small(&bars->kfull[st], phase, abort_flag);
            if (!ok) break;
            if (t < mine) {
              // S over the P of the tile before, which its P V has read
              if (n_tiles > 0) ok = mbar_wait_small(&bars->pvdone[g], (n_tiles - 1) & 1, abort_flag);
              if (!ok) break;
              tc::fence_after_sync();
              const uint64_t dK = dK0 + st * desc_step(C::kTile);
#pragma unroll
              for (int ks = 0; ks < D / 16; ++ks) {
                const uint64_t step = desc_step((ks >> 2) * kAtom + (ks & 3) * 32);
                tc::mma_bf16(colS, dQ + step, dK + step, idS, ks > 0 ? 1u : 0u);
              }
              tc::mma_commit(&bars->sfull[g]);
              tc::mma_commit(&bars->kempty[st]);
              if (t == mine - 1) tc::mma_commit(&bars->qempty[g]);
              ok = mbar_wait_small(&bars->vfull[st], phase, abort_flag);
              if (ok && clear) ok = mbar_wait_small(&bars->vclr[st], (cleared >> st) & 1, abort_flag);
              if (ok && t == it.t0 && n_items > 0) ok = mbar_wait_small(&bars->ofree[g], (n_items - 1) & 1, abort_flag);
              const uint64_t dV = dV0 + st * desc_step(C::kTile);
#pragma unroll
              for (int half = 0; half < 2; ++half) {
                ok = ok && mbar_wait_small(&bars->pfull[g][half], n_tiles & 1, abort_flag);
                if (!ok) break;
                tc::fence_after_sync();
#pragma unroll
                for (int ks = 4 * half; ks < 4 * half + 4; ++ks)
                  tc::mma_bf16_ts(colO, colS + ks * 8, dV + desc_step(ks * 16 * 128), idO, ks > 0 || t > it.t0 ? 1u : 0u);
              }
              if (!ok) break;
              tc::mma_commit(&bars->vempty[st]);
              tc::mma_commit(&bars->pvdone[g]);
              if (t == mine - 1) tc::mma_commit(&bars->olast[g]);
              ++n_tiles;
            } else {  // the other row tile's alone
              mbar_arrive(&bars->kempty[st]);
              ok = mbar_wait_small(&bars->vfull[st], phase, abort_flag);
              if (!ok) break;
              mbar_arrive(&bars->vempty[st]);
            }
            if (clear) cleared ^= 1u << st;
            if (++st == C::kNS) {
              st = 0;
              phase ^= 1;
            }
          }
          if (mine > it.t0) ++n_items;
        }
        ok = __shfl_sync(0xffffffffu, ok ? 1 : 0, 0) != 0;
      }
      if (lane == 0) {  // every product finished before TMEM is released
        tc::mma_commit(&bars->drained[g]);
        mbar_drain(&bars->drained[g], 0);
      }
    }
  } else if (warp >= kOutWarp0) {
    tc_regs_down<104>();
    // -------------------------------------------------------------- results
    const int quarter = warp - kOutWarp0;
    unsigned char* stage = base + C::off_stage + quarter * 4096;
    const int r = quarter * 32 + lane;
    const int token = r / rp.group;
    const uint32_t lane_base = tmem + ((uint32_t)(quarter * 32) << 16);
    __nv_bfloat16* out = reinterpret_cast<__nv_bfloat16*>(rp.out);
    float* parts = reinterpret_cast<float*>(p.ws + kPartOff);
    const size_t slot_floats = (size_t)p.part_rows * (D + 2);
    unsigned n_l = 0, o_phase = 0;  // bit g: parity of the items with tiles of row tile g
    ItemReader reader;
    TcItem it;
    bool ok = true;
    while (ok && reader.next(bars, items, it, abort_flag, lane)) {
      const Seq s = {it.row0, it.rows, it.m, it.kv};
      const bool split = it.chunks > 1;
#pragma unroll 1
      for (int g = 0; g < 2 && ok; ++g) {
        ok = warp_wait_small(&bars->lready[g], n_l & 1, abort_flag);
        if (!ok) break;
        const float mx = m_row[g * kBM + r], l = l_row[g * kBM + r];
        __syncwarp();
        if (lane == 0) mbar_arrive(&bars->lfree[g]);
        const int pos = it.pos0 + g * p.tokens + token;
        const bool valid = token < p.tokens && pos < it.rows;
        const int sees = valid ? seen(s, pos) : 0;
        const bool tiles = it.stop(g) > it.t0;
        if (tiles) {
          ok = warp_wait_small(&bars->olast[g], (o_phase >> g) & 1, abort_flag);
          o_phase ^= 1u << g;
          if (!ok) break;
          tc::fence_after_sync();
        }
        const unsigned any = __ballot_sync(0xffffffffu, valid);
        bool odd = false;
        const float inv = split ? 1.f : 1.f / l;
        float* part = parts + it.slot * slot_floats + (size_t)(g * kBM + quarter * 32) * (D + 2);
        // 32 columns at a time as fp32 (a partial result) or 64 as bf16: 128 bytes a row in the stage, 16-byte piece e of row
        // x at e ^ (x & 7)
        const auto flush = [&](int col) {
          __syncwarp();
#pragma unroll 1
          for (int x = lane >> 3; x < 32; x += 4) {
            if (!((any >> x) & 1u)) continue;
            const int e = lane & 7;
            const uint4 v = *reinterpret_cast<const uint4*>(stage + x * 128 + ((e ^ (x & 7)) << 4));
            if (split) {
              float* at = part + (size_t)x * (D + 2) + 2 + col + 4 * e;  // (rows are 8-byte aligned)
              *reinterpret_cast<uint2*>(at) = make_uint2(v.x, v.y);
              *reinterpret_cast<uint2*>(at + 2) = make_uint2(v.z, v.w);
            } else {
              const int xr = quarter * 32 + x, xt = xr / rp.group;
              *reinterpret_cast<uint4*>(out + ((size_t)(it.row0 + it.pos0 + g * p.tokens + xt) * rp.H + it.h * rp.group +
                                               (xr - xt * rp.group)) * D + col + 8 * e) = v;
            }
          }
          __syncwarp();
        };
#pragma unroll 1
        for (int c = 0; c < D / 32; ++c) {
          uint32_t o[32];
          if (tiles) {
            tc::tmem_ld32(lane_base + C::kColO + g * D + c * 32, o);
            tc::tmem_wait_ld();
          }
          if (c == D / 32 - 1 && tiles) {
            tc::fence_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive(&bars->ofree[g]);
          }
          if (!tiles || sees == 0) {
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] = 0u;
          }
          if (any == 0) continue;
          if (split) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
              *reinterpret_cast<uint4*>(stage + lane * 128 + ((e ^ (lane & 7)) << 4)) =
                  make_uint4(o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]);
            flush(c * 32);
          } else {
            if (sees > 0) {
#pragma unroll
              for (int e = 0; e < 32; ++e) {
                const float v = __uint_as_float(o[e]) * inv;
                odd |= !isfinite(v);
                o[e] = __float_as_uint(v);
              }
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const uint32_t* a = o + 8 * e;
              *reinterpret_cast<uint4*>(stage + lane * 128 + (((4 * (c & 1) + e) ^ (lane & 7)) << 4)) =
                  make_uint4(pack_bf16x2(__uint_as_float(a[0]), __uint_as_float(a[1])),
                             pack_bf16x2(__uint_as_float(a[2]), __uint_as_float(a[3])),
                             pack_bf16x2(__uint_as_float(a[4]), __uint_as_float(a[5])),
                             pack_bf16x2(__uint_as_float(a[6]), __uint_as_float(a[7])));
            }
            if (c & 1) flush((c - 1) * 32);
          }
        }
        if (split) {
          if (valid) *reinterpret_cast<float2*>(part + (size_t)lane * (D + 2)) = make_float2(tiles ? mx : -CUDART_INF_F, tiles ? l : 0.f);
        } else {
          unsigned again = __ballot_sync(0xffffffffu, odd && valid);
#pragma unroll 1
          while (again) {
            const int x = __ffs(again) - 1;
            again &= again - 1;
            const int xr = quarter * 32 + x, xt = xr / rp.group, xp = it.pos0 + g * p.tokens + xt;
            const int head = it.h * rp.group + (xr - xt * rp.group);
            float y[D / 32];
            attend_row<__nv_bfloat16, D>(rp, it.b, s, xp, head, seen(s, xp), y);
            store_row<D / 32>(out + ((size_t)(it.row0 + xp) * rp.H + head) * D + lane * (D / 32), y);
          }
        }
      }
      ++n_l;
      if (!ok || !split) continue;
      // ---- this chunk's rows are there; the warp that completes the item's count merges its quarter's rows
      __threadfence();
      __syncwarp();
      unsigned* count = reinterpret_cast<unsigned*>(p.ws + kCountOff) + (size_t)(it.slot - it.chunk * it.slot_step) * 4 + quarter;
      unsigned before = 0;
      if (lane == 0) before = atomicAdd(count, 1u);
      before = __shfl_sync(0xffffffffu, before, 0);
      if (before != (unsigned)it.chunks - 1u) continue;
      __threadfence();
      if (lane == 0) *count = 0u;
#pragma unroll 1
      for (int y = 0; y < 64; ++y) {
        const int g = y >> 5, xr = quarter * 32 + (y & 31), xt = xr / rp.group, xp = it.pos0 + g * p.tokens + xt;
        if (xt >= p.tokens || xp >= it.rows) continue;
        const int head = it.h * rp.group + (xr - xt * rp.group);
        __nv_bfloat16* at = out + ((size_t)(it.row0 + xp) * rp.H + head) * D + lane * (D / 32);
        float v[D / 32];
#pragma unroll
        for (int e = 0; e < D / 32; ++e) v[e] = 0.f;
        const int sees = seen(s, xp);
        if (sees > 0) {
          const float* row = parts + (size_t)(it.slot - it.chunk * it.slot_step) * slot_floats + (size_t)(g * kBM + xr) * (D + 2);
          const size_t step = (size_t)it.slot_step * slot_floats;
          float m_all = -CUDART_INF_F, l_all = 0.f;
#pragma unroll 1
          for (int c = lane; c < it.chunks; c += 32) m_all = fmaxf(m_all, __ldcg(row + c * step));
          m_all = warp_max(m_all);
#pragma unroll 4
          for (int c = 0; c < it.chunks; ++c) {
            const float2 ml = __ldcg(reinterpret_cast<const float2*>(row + c * step));
            const float f = ml.x == -CUDART_INF_F ? 0.f : fast_exp2(ml.x - m_all);
            l_all += ml.x == -CUDART_INF_F ? ml.y : f * ml.y;  // (a NaN stays one)
#pragma unroll
            for (int e = 0; e < D / 32; e += 2) {
              const float2 o = __ldcg(reinterpret_cast<const float2*>(row + c * step + 2 + lane * (D / 32) + e));
              v[e] += f * o.x;
              v[e + 1] += f * o.y;
            }
          }
          bool odd = false;
#pragma unroll
          for (int e = 0; e < D / 32; ++e) {
            v[e] /= l_all;
            odd |= !isfinite(v[e]);
          }
          if (__any_sync(0xffffffffu, odd)) attend_row<__nv_bfloat16, D>(rp, it.b, s, xp, head, sees, v);
        }
        store_row<D / 32>(at, v);
      }
    }
  } else {
    tc_regs_up<176>();
    // -------------------------------------------------------------- softmax of row tile g
    const int g = warp >> 2, quarter = warp & 3;
    const int r = quarter * 32 + lane;
    const int token = r / rp.group;
    const uint32_t lane_base = tmem + ((uint32_t)(quarter * 32) << 16);
    const uint32_t s_col = lane_base + C::kColS + g * kBN, o_col = lane_base + C::kColO + g * D;
    const float sl2 = rp.scale_log2;
    const uint64_t sc2 = f2(sl2, sl2);
    unsigned n_tiles = 0, n_items = 0;
    ItemReader reader;
    TcItem it;
    bool ok = true;
    while (ok && reader.next(bars, items, it, abort_flag, lane)) {
      const Seq s = {it.row0, it.rows, it.m, it.kv};
      const int pos = it.pos0 + g * p.tokens + token;
      const int limit = token < p.tokens && pos < it.rows ? seen(s, pos) : 0;  // keys that this row sees
      const int all_see = seen(s, it.pos0 + g * p.tokens);                     // that every row of the tile sees
      float m = -CUDART_INF_F, l = 0.f;
#pragma unroll 1
      for (int t = it.t0; t < it.stop(g); ++t, ++n_tiles) {
        ok = warp_wait_small(&bars->sfull[g], n_tiles & 1, abort_flag);
        if (!ok) break;
        tc::fence_after_sync();
        uint32_t sv[128];
#pragma unroll
        for (int c = 0; c < 4; ++c) tc::tmem_ld32(s_col + 32 * c, *reinterpret_cast<uint32_t(*)[32]>(sv + 32 * c));
        tc::tmem_wait_ld();
        if ((t + 1) * kBN > all_see) {
          const int nv = limit - t * kBN;
#pragma unroll
          for (int e = 0; e < 128; ++e) sv[e] = e < nv ? sv[e] : 0xff800000u;
        }
        float mx[4] = {-CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F};
#pragma unroll
        for (int e = 0; e < 128; e += 8)
#pragma unroll
          for (int q = 0; q < 4; ++q) mx[q] = fmax3(mx[q], __uint_as_float(sv[e + 2 * q]), __uint_as_float(sv[e + 2 * q + 1]));
        const float tmax = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * sl2;
        const bool need = tmax > m + kRescaleLog2;
        if (__any_sync(0xffffffffu, need)) {
          const float m_new = need ? tmax : m;
          const float f = m == m_new ? 1.f : fast_exp2(m - m_new);
          l *= f;
          m = m_new;
          if (t > it.t0) {
#pragma unroll 1
            for (int c = 0; c < opaque(D / 16); ++c) {
              uint32_t o[16];
              tc::tmem_ld16(o_col + c * 16, o);
              tc::tmem_wait_ld();
#pragma unroll
              for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
              tc::tmem_st16(o_col + c * 16, o);
            }
            tc::tmem_wait_st();
          }
        }
        const float ref = m == -CUDART_INF_F ? 0.f : m;
        const uint64_t nm2 = f2(-ref, -ref);
        uint64_t acc[4] = {0ull, 0ull, 0ull, 0ull};
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          uint32_t pk[32];
#pragma unroll
          for (int e = 0; e < 32; ++e) {
            float x0, x1;
            unf2(ffma2(f2(__uint_as_float(sv[64 * half + 2 * e]), __uint_as_float(sv[64 * half + 2 * e + 1])), sc2, nm2), x0, x1);
            const float p0 = fast_exp2(x0), p1 = fast_exp2(x1);
            acc[e & 3] = fadd2(acc[e & 3], f2(p0, p1));
            pk[e] = pack_bf16x2(p0, p1);
          }
          tc::tmem_st32(s_col + 32 * half, pk);
          tc::tmem_wait_st();
          tc::fence_before_sync();
          __syncwarp();
          if (lane == 0) mbar_arrive(&bars->pfull[g][half]);
        }
        float a0, a1, b0, b1;
        unf2(fadd2(acc[0], acc[1]), a0, a1);
        unf2(fadd2(acc[2], acc[3]), b0, b1);
        l += (a0 + a1) + (b0 + b1);
      }
      if (!ok) break;
      ok = warp_wait_small(&bars->lfree[g], (n_items & 1) ^ 1, abort_flag);
      if (!ok) break;
      m_row[g * kBM + r] = m;
      l_row[g * kBM + r] = l;
      __syncwarp();
      if (lane == 0) mbar_arrive(&bars->lready[g]);
      ++n_items;
    }
  }

  __syncwarp();
  tc::fence_before_sync();
  __syncthreads();
  if (threadIdx.x == 0) {
    record_abort(abort_flag, status);
    if (atomicAdd(finished, 1u) == gridDim.x - 1) {  // the counters back to zero for the next call
      *claim = 0u;
      *finished = 0u;
    }
  }
  if (warp == kKWarp) {
    tc::fence_after_sync();
    tc::tmem_dealloc(tmem, kTmemCols);
  }
}

// [d2, d1, d0] bf16 rows with strides of their own, in boxes of 64 x box1 x box2 with the 128-byte swizzle.
bool rows_map(CUtensorMap* m, const void* base, long long d0, long long d1, long long d2, long long stride1, long long stride2,
              int box1, int box2) {
  PFN_cuTensorMapEncodeTiled_v12000 fn = tensor_map_encoder();
  if (!fn) return false;
  const cuuint64_t dims[3] = {(cuuint64_t)d0, (cuuint64_t)d1, (cuuint64_t)d2};
  const cuuint64_t strides[2] = {(cuuint64_t)stride1 * 2, (cuuint64_t)stride2 * 2};
  const cuuint32_t box[3] = {64, (cuuint32_t)box1, (cuuint32_t)box2};
  const cuuint32_t es[3] = {1, 1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, box, es,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

int part_rows(int max_q, int group) { return max_q <= kBM / group ? kBM : 2 * kBM; }

template <int D>
cudaError_t launch_typed(const RowsArgs& a, cudaStream_t st) {
  using C = TcCfg<D>;
  static PerDevice<int> allowed;
  cudaError_t e = allow_smem(allowed, rows_tc_kernel<D>, (int)C::kSmem);
  if (e != cudaSuccess) return e;
  TcParams p;
  p.r = rows_params(a);
  p.ws = static_cast<unsigned char*>(a.ws);
  const int group = p.r.group;
  p.tokens = kBM / group;
  p.part_rows = part_rows(a.max_q, group);
  CUtensorMap mq, mk, mv;
  if (!rows_map(&mq, a.q, D, a.H, a.T, D, a.q_stride, group, p.tokens)) return cudaErrorNotSupported;
  if (a.table) {
    const int P = 1 << a.page_shift;
    p.box_rows = P < kBN ? P : kBN;
    const long long slabs = (long long)a.n_pages * a.Hkv;
    if (slabs > 0x7fffffffLL) return cudaErrorNotSupported;  // 32-bit TMA coordinates
    if (!rows_map(&mk, a.K, D, P, slabs, D, (long long)P * D, p.box_rows, 1) ||
        !rows_map(&mv, a.V, D, P, slabs, D, (long long)P * D, p.box_rows, 1))
      return cudaErrorNotSupported;
  } else {
    p.box_rows = kBN;
    if (!rows_map(&mk, a.K, D, a.Hkv, a.T, D, a.k_stride, 1, kBN) || !rows_map(&mv, a.V, D, a.Hkv, a.T, D, a.v_stride, 1, kBN))
      return cudaErrorNotSupported;
  }
  // claims, their counter's reach past the last one, and token coordinates past the last row stay in 32 bits
  const long long most = ((long long)a.T / (2 * p.tokens) + a.B) * a.Hkv;
  if (most > 0x7fffffffLL - 2 * kMaxGrid || (long long)a.T + 4 * kBM > 0x7fffffffLL || (long long)a.max_kv + kBN > 0x7fffffffLL)
    return cudaErrorNotSupported;
  int G = sm_count() < kMaxGrid ? sm_count() : kMaxGrid;
  return launch_pdl(rows_tc_kernel<D>, dim3((unsigned)G), dim3(kTcThreads), C::kSmem, st, mq, mk, mv, p);
}

}  // namespace

size_t rows_workspace_bytes(int B, int H, int Hkv, int D, int T, int max_q, int dtype) {
  (void)B;
  (void)T;
  if (dtype != 0 || H / Hkv > kBM) return WsLayout::kHeader;
  return kPartOff + (size_t)kMaxChunks * part_rows(max_q, H / Hkv) * (D + 2) * sizeof(float);
}

cudaError_t launch_rows_tc(const RowsArgs& a, cudaStream_t st) {
  if (a.dtype != 0 || a.H / a.Hkv > kBM) return cudaErrorNotSupported;
  return a.D == 128 ? launch_typed<128>(a, st) : launch_typed<64>(a, st);
}

}  // namespace glide
