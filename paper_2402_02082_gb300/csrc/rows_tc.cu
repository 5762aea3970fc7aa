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
// What bounds it: a row tile and 128 keys of 128 take two products of ~520 cycles, in which S reads 64 KB of shared memory
// and P V 32, while the loads write 64 (1250 cycles at 128 bytes a cycle); ~1430 cycles a tile measured.  At D = 64, half
// of all that, ~1300: so the chain of a tile (S, the softmax of a row by one thread, P V, and the hand-overs between), which
// takes three times the products, counts as much.  Tensor memory holds three S buffers beside O: S of tile i + 3 waits for
// P V of tile i.  Two softmax groups of four warps take the key tiles in turn; the reference maximum passes from tile to
// tile, so from group to group, through shared memory; a group keeps its own sum and takes it to the item's last reference at
// the end.  Of a long prompt's cycles the tensor pipe is busy in 66% (D = 64: 37%), issue in 47, the exponentials' pipe in
// 33.  Slower: a third softmax group (+7%), one eighth of the exponentials as polynomials (+3%), four S buffers of 96 keys
// (long prompts +1.5%, paged calls up to +20%, prompts of 1000 tokens -5%).
// An item costs 3000 to 4000 cycles beside its tiles, and a call ~9 us: 7000 cycles from the plan to the first scores, most
// of them latency (lengths, code that runs once, queries, keys).
//
// Measured (bf16, D = 128; us): a prompt of 16384 tokens, 32 heads over 8 cached, 1340, and 1490 to 1530 call after call under the
// power limit (1.64 and 1.44 to 1.48 PFLOP/s of visible pairs); four of 2048, 32 heads, 120 to 132 (1.04 to 1.15); 24 of up to
// 333, 52 heads, 56.5; eight requests of up to 512 new tokens over 512 to 4096 keys, 40 heads, 105 to 108, the same with a bound
// of 131072 or (a kernel of its own) 262144 keys.  A prompt of 8192, 32 heads over 8: 361, and 298 with 64 dims.
//
// The tensor cores' sums lose what lies 2^-25 below O with every product (measured), which the sum of a row's weights does not.  So
// one O takes in 2^17 keys at most: an item of more goes in segments, whose (max, sum, o) the result warps fold in fp32 in the
// workspace.  The mean of 2^22 keys of like weight, relative error: -2.5e-2 in one O, -5e-5 in segments; of 2^24, -0.1 and -5e-5.
//
// Work items are (cached head, 128 / group tokens, keys), claimed from a counter: cached heads in groups whose keys and
// values together stay in L2, in them the row tiles with the most keys first; the short ones of all heads come last, so
// that the SMs end together.  Where there are fewer than two items for an SM, an item's keys may be cut into chunks, as many
// as cost least (split_cost); their partial results (max, sum, o) go through the workspace, rows side by side, and a second
// kernel merges them in the chunks' order.
//
// Code size counts: what does not stay in the instruction cache is fetched again by every role at every item.  A form of
// this kernel with two row tiles a CTA, a softmax group each and rows of 128 scores in registers, unrolled, took 6000
// cycles to write an item's rows and lost more to that than it gained by sharing the key tiles.
//
// Roles (512 threads, one CTA per SM):
//   warps 0-7    softmax, two groups of four: warp w reads TMEM lane quarter w % 4, one thread a row, of the tiles of
//                parity w / 4; they rescale O where the reference is raised (by more than 8, so seldom).
//   warp 8       claims items and makes them, up to two ahead; loads Q (two items' worth) and K (a page's rows at a time,
//                or 128 packed rows); warp 11 loads V and clears its rows past an item's last visible key.
//   warp 9       S issue, warp 10 P V issue (lane 0).
//   warps 12-15  results: a TMEM lane quarter each, O / l through 4 KB of shared memory in whole rows.
//
// A result that is not finite (an infinity or NaN among the values that the row sees, or one that it does not see, in a tile that it
// shares; or an overflow) is computed again by the definition, the row alone, unless its sum of weights is 0 or NaN, which makes
// it NaN.  The other warps' waits are put off meanwhile.  A NaN among the keys costs nothing; where all rows of a prompt of 16384
// tokens, four heads, see an infinite value, each is computed again by one warp: 1.07 s.
#include <cuda.h>
#include <cuda_bf16.h>
#include <math_constants.h>

#include "device.h"
#include "kernels.h"
#include "rows_attn.cuh"
#include "rows_wait.cuh"
#include "tc_attn.cuh"
#include "tc_ptx.cuh"
#include "tensor_map.h"

namespace glide {
namespace {

constexpr int kBM = 128;          // rows of a row tile (MMA rows, TMEM lanes)
constexpr int kBN = 128;          // keys of a tile
constexpr int kKWarp = 8;
constexpr int kSWarp = 9;
constexpr int kVWarp = 11;
constexpr int kOutWarp0 = 12;
constexpr int kTcThreads = 512;
constexpr int kTmemCols = 512;
constexpr uint32_t kAtom = 128 * 128;  // one 128-byte-swizzle atom of 128 rows
constexpr float kRescaleLog2 = 8.0f;
constexpr int kSBufs = 3;
constexpr int kItemSlots = 4;
constexpr int kItemReaders = 15;       // warps that read an item beside the one that makes it
constexpr int kMaxGrid = 160;
constexpr int kMaxChunks = 3 * kMaxGrid;  // partial slots: below 2 grids of items and one grid more of chunks
constexpr int kFewTiles = 12;          // key tiles of an item that are not worth a second kernel
constexpr int kSortMost = 128;         // sequences that are taken in the order of their keys
constexpr int kListMost = 3000;        // entries (sequence, row tile, chunk) that are listed in shared memory
constexpr int kLevelMost = 4096;       // row tiles of a sequence that a list entry holds
constexpr long long kL2Bytes = 48ll << 20;
constexpr int kManyKeys = 1 << 24;     // that no part of L2 holds; sums of two for each lane of a warp stay in 32 bits
constexpr int kSegTiles = 1024;        // key tiles that one O takes in (2^17 keys)
constexpr int kLateTenths = 4;         // items with at most this part of the longest one's key tiles are left to the end

// Workspace: in the header the status word, the claim counter, the count of finished CTAs, and for the merge the count of
// items in chunks and that of its finished CTAs.  Behind the bytes that are zero between calls, those items and partial slots of [D + 2][128 rows] floats: a row's maximum, its sum, its columns.
struct PartItem {
  int b, h, row0, m, kv, rows, pos0, chunks, slot, slot_step;
};
constexpr size_t kPartsOff = 64, kMergedOff = 96;
constexpr size_t kPartItemsBytes = (2 * kMaxGrid * sizeof(PartItem) + 255) / 256 * 256;
constexpr int kSplitCount = 11;  // chunks of the longest item that are tried: 2 .. 6, 8, 10, 12, 16, 20, 24
constexpr int kMergeTiles = 7;
constexpr int kAlone = 4;  // row tiles of a sequence that one lane counts
// The cost of n items of at most `tiles` key tiles on G SMs, in key tiles: an item takes 3 beside its own, a chunk 5, and
// the merge and its launch 7.  us without chunks and with: 256 new tokens over 6000 keys, 32 heads over 8 cached 51 and
// 39; 16 over 16384 121 and 28; two requests of 64 over 16384, 32 heads 128 and 94; 512 over 4000, 52 heads 65 and 75.
__host__ __device__ constexpr int rounds_cost(int n, int G, int tiles) { return (n + G - 1) / G * (tiles + 3); }
__host__ __device__ constexpr int split_cost(int n, int G, int tiles) {
  return n > kMaxChunks ? 0x7fffffff : rounds_cost(n, G, tiles + 2) + kMergeTiles;
}
__host__ __device__ constexpr int split_of(int i) { return i < 5 ? i + 2 : (i < 8 ? 2 * i - 2 : 4 * (i - 4)); }

struct Bars {
  uint64_t kfull[4], vfull;  // vfull: of a V tile whose end is cleared before P meets it
  uint64_t qfull[2], qempty[2];  // qempty: the result warps are done with what was the queries' place
  uint64_t sfull[kSBufs];  // S is there, and its K stage free
  uint64_t pvfull[kSBufs]; // P and the V tile that it meets are there
  uint64_t bfree[kSBufs];  // P V has read both, and added to O
  uint64_t olast, ofree, lready, lfree;
  uint64_t turn[4][2];    // [quarter][tile parity]: a tile's reference is there
  uint64_t itemfull[kItemSlots], itemempty[kItemSlots];
  uint64_t drained[2];
};

constexpr int kMore = 1, kAfter = 2;
struct TcItem {
  int b;                  // -1: no more
  int h, row0, m, kv, rows, pos0;
  int t0, te;             // key tiles (of this segment)
  int segment;            // kMore: segments of the item follow, kAfter: some came before
  int klen;               // keys that some row of the item sees
  int chunks, chunk, slot, slot_step;  // chunks of the item, this one, its partial slot, slots from chunk to chunk
};

struct Misc {
  Watch watch;
  uint32_t tmem;
  int head_group;      // cached heads that are worked on together
  int chunk_tiles;     // key tiles of a chunk
  int entries;         // (sequence, row tiles, chunk) triples
  int levels;          // the most row tiles of a sequence
  int listed;          // the entries are in the list
  int grouped;         // entries that are taken head group by head group; the rest follow for all heads
  long long sum[2];
  int longest;         // key tiles of the item with the most
  int4 splits[kSplitCount];  // by chunks of the longest item: entries, key tiles of a chunk, cost
};

template <int D>
struct TcCfg {
  static constexpr int kHalves = D / 64;
  static constexpr uint32_t kTile = kHalves * kAtom;  // 128 rows x D
  // stages of the K ring and of the V ring; no more than S buffers, whose barriers say when a stage is free
  static constexpr unsigned kNS = D == 128 ? 2 : 3;
  static_assert(kNS <= kSBufs, "stage release");
  static constexpr uint32_t off_Q = 0;                // two items' queries
  static constexpr uint32_t off_K = 2 * kTile;
  static constexpr uint32_t off_V = off_K + kNS * kTile;
  static constexpr uint32_t off_bar = off_V + kNS * kTile;
  static constexpr uint32_t off_item = off_bar + sizeof(Bars);
  static constexpr uint32_t off_misc = (off_item + kItemSlots * sizeof(TcItem) + 15) / 16 * 16;
  static constexpr uint32_t off_rows = off_misc + sizeof(Misc);      // [row] references, then sums [group][row], then final
  static constexpr uint32_t off_table = off_rows + 4 * kBM * 4;     // lengths, in the order in which they are taken
  static constexpr uint32_t off_rowat = off_table + kSortMost * 16;  // elements from a row tile's first row to its rows
  static constexpr uint32_t off_order = off_rowat + kBM * 4;
  static constexpr uint32_t off_list = off_order + kSortMost * 4;
  static constexpr size_t kSmem = 1024 + off_list + kListMost * 4;
  static_assert(kSmem <= 227 * 1024, "shared memory");
  static constexpr uint32_t kColO = kSBufs * kBN;                   // TMEM columns: three S buffers, O
  static_assert(kColO + D <= kTmemCols, "TMEM columns");
};

struct TcParams {
  RowsParams r;
  unsigned char *ws, *scratch;
  int may_split;   // a merge kernel follows
  int tokens;      // of a row tile: 128 / group
  unsigned by_tokens, by_heads;  // reciprocals, of H_kv the second
  int box_rows;    // key rows of one TMA box: a page's, at most 128
};

// n / d and the remainder by a multiplication, for n < 2^31 and r = reciprocal(d): the estimate is the quotient or one less.
__host__ __device__ __forceinline__ unsigned reciprocal(unsigned d) { return d ? 0xffffffffu / d : 0u; }
__device__ __forceinline__ unsigned divide(unsigned n, unsigned d, unsigned r, unsigned& rest) {
  unsigned q = __umulhi(n, r);
  rest = n - q * d;
  if (rest >= d) {
    rest -= d;
    ++q;
  }
  return q;
}

// Row tiles of a sequence, and the keys that the last row of tile x sees.
__device__ __forceinline__ int tiles_of(const Seq& s, int tokens, unsigned by_tokens) {
  unsigned rest;
  return s.rows > 0 ? (int)divide((unsigned)(s.rows - 1), tokens, by_tokens, rest) + 1 : 0;
}
__device__ __forceinline__ int keys_of(const Seq& s, int tokens, int x) {
  const int last = (x + 1) * tokens;
  return seen(s, (last < s.rows ? last : s.rows) - 1);
}
__device__ __forceinline__ int chunks_of(const Seq& s, int tokens, int x, int chunk_tiles) {
  if (x * tokens >= s.rows) return 0;
  const int nt = (keys_of(s, tokens, x) + kBN - 1) / kBN;
  return nt <= chunk_tiles ? 1 : (nt + chunk_tiles - 1) / chunk_tiles;
}

// The first row tile of `most` with at least `count` key tiles (`most`: none).
__device__ __forceinline__ int first_tile(const Seq& s, int most, int tokens, unsigned by_tokens, int count) {
  if (count > 0 && (most == 0 || keys_of(s, tokens, most - 1) <= (count - 1) * kBN)) return most;
  const int need = (count - 1) * kBN - (s.kv - s.m);  // of its tokens, counted from the sequence's first: more than these
  unsigned rest;
  return count <= 0 || need < 0 ? 0 : (int)divide((unsigned)need, tokens, by_tokens, rest);
}

template <int N>
__device__ __forceinline__ void tc_regs_up() {
  asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N) : "memory");
}
template <int N>
__device__ __forceinline__ void tc_regs_down() {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N) : "memory");
}

// The items as every other warp reads them: a slot is the warp's until it lets go.
struct ItemReader {
  unsigned n = 0;
  __device__ __forceinline__ const TcItem* next(Bars* bars, const TcItem* items, Watch* watch) {
    const unsigned slot = n % kItemSlots;
    if (!warp_wait_watched(&bars->itemfull[slot], (n / kItemSlots) & 1, watch)) return nullptr;
    return items[slot].b >= 0 ? items + slot : nullptr;
  }
  __device__ __forceinline__ void release(Bars* bars, int lane) {
    __syncwarp();
    if (lane == 0) mbar_arrive(&bars->itemempty[n % kItemSlots]);
    ++n;
  }
};

// A key tile in shared memory is made of 8-row x 128-byte swizzle atoms: row r, half hd of D (64 columns) at
//   packed   hd * 16 KB + r * 128       (a 4-D box of 64 columns x 128 rows x halves)
//   pages    (r / 8) * (halves KB) + hd KB + (r % 8) * 128   (a page's rows are one box of 64 columns x 8 rows x halves x
//            groups of 8 rows)
// so a box brings all of D, and the products' descriptors differ in two strides alone.
template <int D>
struct KeyTile {
  static constexpr uint32_t kHalves = D / 64;
  uint32_t group, half;  // bytes from 8 rows to the next, and from half to half
  __device__ __forceinline__ explicit KeyTile(bool packed) : group(packed ? 1024 : kHalves * 1024), half(packed ? kAtom : 1024) {}
  __device__ __forceinline__ uint32_t at(int row, int hd) const { return (row >> 3) * group + hd * half + (row & 7) * 128; }
};

// The box of a key tile that this lane loads: a page's keys of the tile, or 128 packed rows.
struct Boxes {
  int at, shift;  // this lane's first row in a tile; log2 of a box's rows
  __device__ __forceinline__ Boxes(const TcParams& p, int lane) {
    shift = 31 - __clz(p.box_rows);
    at = lane << shift;
  }
  __device__ __forceinline__ bool any(int left) const { return at < kBN && at < left; }  // left: keys from the tile on
  __device__ __forceinline__ uint32_t bytes(int left, bool packed, int row_bytes) const {
    const int rows = left < kBN && !packed ? (left + (1 << shift) - 1) >> shift << shift : kBN;
    return (uint32_t)(rows * row_bytes);
  }
  // coordinates (y, w) of the lane's box, for key tile t of the item: packed rows and the head, or 0 and the group of 8 rows
  __device__ __forceinline__ int2 where(const RowsParams& r, int b, int h, int row0, int t) const {
    const int key = t * kBN + at;
    if (!r.table) return make_int2(row0 + key, h);
    const int row = key & ((1 << r.page_shift) - 1);
    return make_int2(0, (((page_at(r, b, key >> r.page_shift) * r.Hkv + h) << r.page_shift) + row) >> 3);
  }
};

// kLong: items may have more than kSegTiles key tiles.  (Short prompts take 57 us without the code for that, 58 with it.)
template <int D, bool kLong>
__global__ void __launch_bounds__(kTcThreads, 1)
    rows_tc_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                   const __grid_constant__ CUtensorMap tmV, const TcParams p) {
  using C = TcCfg<D>;
  extern __shared__ unsigned char smem_raw[];
  unsigned char* base = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  Bars* bars = reinterpret_cast<Bars*>(base + C::off_bar);
  TcItem* items = reinterpret_cast<TcItem*>(base + C::off_item);
  Misc* misc = reinterpret_cast<Misc*>(base + C::off_misc);
  float* m_ref = reinterpret_cast<float*>(base + C::off_rows);  // the running reference, from one softmax group to the other
  float* l_row = m_ref + kBM;                                   // [group][row] sums
  float* m_row = m_ref + 3 * kBM;                               // the item's last reference
  Seq* table = reinterpret_cast<Seq*>(base + C::off_table);
  int* order = reinterpret_cast<int*>(base + C::off_order);
  uint32_t* list = reinterpret_cast<uint32_t*>(base + C::off_list);
  int* row_at = reinterpret_cast<int*>(base + C::off_rowat);
  Watch* watch = &misc->watch;
  unsigned* status = reinterpret_cast<unsigned*>(p.ws);
  unsigned* claim = reinterpret_cast<unsigned*>(p.ws + WsLayout::kClaimOff);
  unsigned* finished = reinterpret_cast<unsigned*>(p.ws + WsLayout::kDoneOff);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const RowsParams& rp = p.r;
  {  // a warp a kind, a lane a barrier
    int w = 0;
    const auto init = [&](uint64_t* b, int n, int count) {
      if (warp == w++ && lane < n) mbar_init(b + lane, count);
    };
    init(bars->kfull, 4, 1);
    init(&bars->vfull, 1, 1);
    init(bars->qfull, 2, 1);
    init(bars->qempty, 2, 4);
    init(bars->sfull, kSBufs, 1);
    init(bars->pvfull, kSBufs, 5);  // four softmax warps and the load
    init(bars->bfree, kSBufs, 1);
    init(&bars->olast, 1, 1);
    init(&bars->ofree, 1, 4);
    init(&bars->lready, 1, 8);
    init(&bars->lfree, 1, 4);
    init(&bars->turn[0][0], 8, 1);
    init(bars->itemfull, kItemSlots, 1);
    init(bars->itemempty, kItemSlots, kItemReaders);
    init(bars->drained, 2, 1);
    if (warp == 15) {
      if (lane == 0) {
        misc->watch.abort = 0;
        misc->levels = 0;
        misc->listed = 0;
        misc->longest = 0;
        misc->sum[0] = misc->sum[1] = 0;
      }
    }
    fence_barrier_init();
  }
  __syncthreads();
  pdl_wait();  // every global access and the TMEM allocation come after it
  unsigned next = 0;  // the claim of the second item, under way beside the plan
  if (warp == kKWarp) {
    if (lane == 0) next = atomicAdd(claim, 1u);
    tc::tmem_alloc(&misc->tmem, kTmemCols);
    tc::tmem_relinquish();
  }
  if (threadIdx.x < kBM) row_at[threadIdx.x] = (threadIdx.x / rp.group * rp.H + threadIdx.x % rp.group) * D;
  // ---- the plan of the call: what all CTAs find alike from the lengths
  {
    unsigned tiles = 0, keys = 0;
    int levels = 0, longest = 0;
    if (rp.B <= kSortMost && threadIdx.x < rp.B) table[threadIdx.x] = seq_of(rp, threadIdx.x);
#pragma unroll 1
    for (int b = threadIdx.x; b < rp.B; b += kTcThreads) {
      const Seq s = seq_of(rp, b);
      const int n = tiles_of(s, p.tokens, p.by_tokens);
      if (n == 0) continue;
      tiles += n;
      keys += s.kv < kManyKeys ? s.kv : kManyKeys;
      levels = n > levels ? n : levels;
      const int nt = (keys_of(s, p.tokens, n - 1) + kBN - 1) / kBN;
      longest = nt > longest ? nt : longest;
    }
    if (warp * 32 < rp.B) {  // (atomics of a warp's lanes on one word would go one by one)
      tiles = __reduce_add_sync(0xffffffffu, tiles);
      keys = __reduce_add_sync(0xffffffffu, keys);
      levels = __reduce_max_sync(0xffffffffu, levels);
      longest = __reduce_max_sync(0xffffffffu, longest);
      if (lane == 0) {
        atomicAdd(reinterpret_cast<unsigned long long*>(&misc->sum[0]), (unsigned long long)tiles);
        atomicAdd(reinterpret_cast<unsigned long long*>(&misc->sum[1]), (unsigned long long)keys);
        atomicMax(&misc->levels, levels);
        atomicMax(&misc->longest, longest);
      }
    }
    __syncthreads();
    if (rp.B <= kSortMost) {  // the most keys first, four threads a sequence
      static_assert(4 * kSortMost <= kTcThreads, "threads of the sort");
      const int at = threadIdx.x >> 2;
      Seq mine = {0, 0, 0, 0};
      int before = 0;
      if (at < rp.B) {
        mine = table[at];
#pragma unroll 4
        for (int x = threadIdx.x & 3; x < rp.B; x += 4) before += table[x].kv > mine.kv || (table[x].kv == mine.kv && x < at);
      }
      before += __shfl_xor_sync(0xffffffffu, before, 1);
      before += __shfl_xor_sync(0xffffffffu, before, 2);
      __syncthreads();
      if (at < rp.B && (threadIdx.x & 3) == 0) {
        table[before] = mine;
        order[before] = at;
      }
    }
    int chunk = 0x7fffffff;
    long long entries = misc->sum[0];
    const int G = gridDim.x;
    longest = misc->longest;
    if (p.may_split && entries * rp.Hkv < 2ll * G && longest > kFewTiles) {
      // The number of chunks of the longest item whose rounds over the SMs cost least.
      // A warp a number of chunks; a lane a sequence, or where it has many row tiles, all lanes that sequence.
      if (warp < kSplitCount) {
        const int c = (longest + split_of(warp) - 1) / split_of(warp);
        int n = 0;
#pragma unroll 1
        for (int b0 = 0; b0 < rp.B; b0 += 32) {
          const int at = b0 + lane;
          Seq s = {0, 0, 0, 0};
          if (at < rp.B) s = rp.B <= kSortMost ? table[at] : seq_of(rp, at);
          const int most = tiles_of(s, p.tokens, p.by_tokens);
          if (most <= kAlone) {
#pragma unroll 1
            for (int x = 0; x < most; ++x) n += chunks_of(s, p.tokens, x, c);
          }
          unsigned rest = __ballot_sync(0xffffffffu, most > kAlone);
#pragma unroll 1
          while (rest) {
            const int who = __ffs(rest) - 1;
            rest &= rest - 1;
            const Seq o = {0, __shfl_sync(0xffffffffu, s.rows, who), __shfl_sync(0xffffffffu, s.m, who), __shfl_sync(0xffffffffu, s.kv, who)};
#pragma unroll 1
            for (int x = lane; x * p.tokens < o.rows; x += 32) n += chunks_of(o, p.tokens, x, c);
          }
        }
        n = __reduce_add_sync(0xffffffffu, n);
        const int items = n * rp.Hkv;
        if (lane == 0) misc->splits[warp] = make_int4(n, c, split_cost(items, G, c), 0);
      }
      __syncthreads();
      int least = rounds_cost((int)entries * rp.Hkv, G, longest);
#pragma unroll 1
      for (int i = 0; i < kSplitCount; ++i) {
        const int4 x = misc->splits[i];
        if (x.z >= least) continue;
        least = x.z;
        chunk = x.y;
        entries = x.x;
      }
    }
    if (threadIdx.x == 0) {
      const long long bytes = misc->sum[1] * D * 4;  // keys and values of a cached head
      const long long g = bytes > 0 ? kL2Bytes / bytes : rp.Hkv;
      misc->head_group = (int)(g < 1 ? 1 : (g > rp.Hkv ? rp.Hkv : g));
      misc->chunk_tiles = chunk;
      misc->entries = (int)entries;
      misc->grouped = (int)entries;
    }
    __syncthreads();
    // The list of entries, where a CTA makes several items: those with the most key tiles first (so that the SMs end
    // together), among them by sequence, row tile and chunk.  A group of lanes a count of key tiles, a lane of it a
    // sequence; the entries before are one for each row tile of more key tiles than the count and each chunk before its last.
    if (misc->entries <= kListMost && misc->levels <= kLevelMost && longest < kLevelMost &&
        (entries * rp.Hkv > 2 * G || misc->levels > 8)) {
      const int wide = rp.B >= 32 ? 5 : 32 - __clz(rp.B - 1), width = 1 << wide, sub = lane & (width - 1);  // B = 1: one lane
      const int at_once = kTcThreads >> wide;
#pragma unroll 1
      for (int count0 = 0; count0 <= longest; count0 += at_once) {
        const int count = count0 + (threadIdx.x >> wide);
        const bool some = count <= longest;
        const int pieces = count <= chunk ? 1 : (count + chunk - 1) / chunk;
        int to = 0;
#pragma unroll 1
        for (int pass = 0; pass < 2; ++pass) {
#pragma unroll 1
          for (int b0 = 0; b0 < rp.B; b0 += width) {
            const int at = b0 + sub;
            int x = 0, n = 0;
            if (some && at < rp.B) {
              const Seq s = rp.B <= kSortMost ? table[at] : seq_of(rp, at);
              const int most = tiles_of(s, p.tokens, p.by_tokens);
              const int more = first_tile(s, most, p.tokens, p.by_tokens, count + 1);
              if (pass) {  // row tiles x .. more - 1 have `count` key tiles
                x = first_tile(s, most, p.tokens, p.by_tokens, count);
                n = (more - x) * pieces;
              } else {
                n = most - more;
#pragma unroll 1
                for (int j = chunk; j < longest; j += chunk)  // (a chunk is longer than that, or far from overflow)
                  n += most - first_tile(s, most, p.tokens, p.by_tokens, (j > count ? j : count) + 1);
              }
            }
            int upto = n;
#pragma unroll 1
            for (int off = 1; off < width; off <<= 1) {
              const int u = __shfl_up_sync(0xffffffffu, upto, off, width);
              if (sub >= off) upto += u;
            }
            if (pass) {
              uint32_t* put = list + to + upto - n;
              int piece = 0;
#pragma unroll 1
              for (int c = 0; c < n; ++c) {
                put[c] = (uint32_t)at | (uint32_t)x << 10 | (uint32_t)piece << 22;
                if (++piece == pieces) {
                  piece = 0;
                  ++x;
                }
              }
            }
            to += __shfl_sync(0xffffffffu, upto, width - 1, width);
          }
          if (!pass && sub == 0 && count == longest * kLateTenths / 10) misc->grouped = to;
        }
      }
      if (threadIdx.x == 0) misc->listed = 1;
    }
  }
  if (threadIdx.x == 0) put_off(watch);  // (the kernel before, which pdl_wait waits for, may have taken any time)
  tc::fence_before_sync();
  __syncthreads();
  tc::fence_after_sync();
  const uint32_t tmem = misc->tmem;

  if (warp >= kKWarp && warp < kOutWarp0) {
    tc_regs_down<104>();
    if (warp == kKWarp) {
      // ------------------------------------------------------------ items, Q and K
      const uint64_t pol_q = policy_evict_first(), pol_k = policy_evict_last();
      if (lane < 2) tc::prefetch_tmap(lane == 0 ? &tmQ : &tmK);
      const Boxes box(p, lane);
      const KeyTile<D> lay(!rp.table);
      const int entries = misc->entries, head_group = misc->head_group, chunk_tiles = misc->chunk_tiles;
      const unsigned claims = (unsigned)entries * rp.Hkv, per_group = (unsigned)misc->grouped * head_group;  // below 2^31
      const unsigned in_groups = (unsigned)misc->grouped * rp.Hkv;
      const bool one_group = head_group == rp.Hkv;
      const unsigned by_group = one_group ? 0u : reciprocal(per_group), by_heads = one_group ? p.by_heads : reciprocal(head_group),
                     by_last = one_group ? 0u : reciprocal(rp.Hkv % head_group);
      int level = misc->levels - 1, block = 0, acc = 0, group_at = 0;
      bool first = true;
      unsigned made = 0, cur = 0;  // items made, and the one whose keys are loaded
      unsigned st = 0, k_issued = 0, q_issued = 0;
      bool ok = true, more = true, started = false, rest = false;
      int end = 0;  // of the last item made; rest: it has more segments
      int b = 0, h = 0, row0 = 0, klen = 0, t = 0, te = 0;  // of that item
#pragma unroll 1
      while (ok) {
        // the next item when there is none, and up to two ahead once the first keys of one are on their way
        if (more && made < cur + (started ? 3u : 1u)) {
          TcItem it;
          if (kLong && rest) {
            it = items[(made - 1) % kItemSlots];
            it.t0 = it.te;
            it.segment = kAfter;
          } else {
            const unsigned c = first ? blockIdx.x : gridDim.x + __shfl_sync(0xffffffffu, next, 0);
            if (lane == 0 && !first && c < claims) next = atomicAdd(claim, 1u);  // needed for the item after this one
            first = false;
            it.b = -1;
            if (c < claims) {
              unsigned in_group = 0, in_entry;
              int hg = 0, heads = rp.Hkv, e;
              if (c < in_groups) {
                if (one_group) in_group = c;
                else hg = (int)divide(c, per_group, by_group, in_group);
                const int left = rp.Hkv - hg * head_group;
                heads = left < head_group ? left : head_group;
                e = (int)divide(in_group, heads, left < head_group ? by_last : by_heads, in_entry);
              } else {
                e = misc->grouped + (int)divide(c - in_groups, rp.Hkv, p.by_heads, in_entry);
              }
              if (misc->listed) {
                const uint32_t x = list[e];
                const int at = x & 1023;
                level = (x >> 10) & 4095;
                it.chunk = x >> 22;
                const Seq s = rp.B <= kSortMost ? table[at] : seq_of(rp, at);
                it.b = rp.B <= kSortMost ? order[at] : at;
                it.row0 = s.row0;
                it.m = s.m;
                it.kv = s.kv;
                it.rows = s.rows;
                it.chunks = chunks_of(s, p.tokens, level, chunk_tiles);
              } else {
              if (hg != group_at) {
                group_at = hg;
                level = misc->levels - 1;
                block = acc = 0;
              }
              // entry e, found by the counts (many sequences or very long ones)
#pragma unroll 1
              while (level >= 0) {
                const int at = block * 32 + lane;
                int n = 0;
                Seq s = {0, 0, 0, 0};
                if (at < rp.B) {
                  s = rp.B <= kSortMost ? table[at] : seq_of(rp, at);
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
                  it.b = __shfl_sync(0xffffffffu, at, who);
                  if (rp.B <= kSortMost) it.b = order[it.b];
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
              }
              if (it.b >= 0) {
                it.h = hg * head_group + (int)in_entry;
                it.pos0 = level * p.tokens;
                const Seq s = {it.row0, it.rows, it.m, it.kv};
                it.klen = keys_of(s, p.tokens, level);
                // a slot for each item of a call that has chunks (kMaxChunks at most), one for each CTA of another
                it.slot = chunk_tiles < 0x7fffffff ? (int)c : (int)blockIdx.x;
                it.slot_step = heads;
                it.t0 = it.chunks > 1 ? it.chunk * chunk_tiles : 0;
                const int nt = (it.klen + kBN - 1) / kBN;
                end = it.chunks > 1 && nt - it.t0 > chunk_tiles ? it.t0 + chunk_tiles : nt;
                it.segment = 0;
              }
            }
          }
          it.te = end;
          if constexpr (kLong) {
            rest = it.b >= 0 && end - it.t0 > kSegTiles;
            if (rest) {
              it.te = it.t0 + kSegTiles;
              it.segment |= kMore;
            }
          }
          const unsigned slot = made % kItemSlots;
          ok = warp_wait_watched(&bars->itemempty[slot], ((made / kItemSlots) & 1) ^ 1, watch);
          if (!ok) break;
          if (lane == 0) {
            put_off(watch);
            items[slot] = it;
            mbar_arrive(&bars->itemfull[slot]);
          }
          __syncwarp();
          if (it.b < 0) {
            more = false;
            continue;
          }
          ++made;
          if (lane < C::kHalves && it.te > it.t0)  // what the loads will find in L2
            tc::tma_prefetch_l2_3d(&tmQ, lane * 64, it.h * rp.group, it.row0 + it.pos0);
          continue;
        }
        if (!started) {
          if (cur == made) break;  // no more
          const TcItem& it = items[cur % kItemSlots];
          b = it.b; h = it.h; row0 = it.row0; klen = it.klen; t = it.t0; te = it.te;
          if (t == te) {
            ++cur;
            continue;
          }
          const unsigned qb = q_issued & 1;
          ok = warp_wait_watched(&bars->qempty[qb], ((q_issued >> 1) & 1) ^ 1, watch);
          if (!ok) break;
          if (lane == 0) mbar_arrive_expect_tx(&bars->qfull[qb], (uint32_t)(C::kHalves * p.tokens * rp.group * 128));
          __syncwarp();
          if (lane < C::kHalves)
            tc::tma_load_3d(base + C::off_Q + qb * C::kTile + lane * kAtom, &tmQ, lane * 64, h * rp.group, row0 + it.pos0,
                            &bars->qfull[qb], pol_q);
          ++q_issued;
          started = true;
        }
        const int left = klen - t * kBN;
        const int2 x = box.any(left) ? box.where(rp, b, h, row0, t) : make_int2(0, 0);
        if (k_issued >= C::kNS) {  // S of the tile that had the stage
          const unsigned j = k_issued - C::kNS;
          ok = warp_wait_watched(&bars->sfull[j % kSBufs], (j / kSBufs) & 1, watch);
          if (!ok) break;
        }
        if (lane == 0) mbar_arrive_expect_tx(&bars->kfull[st], box.bytes(left, !rp.table, 2 * D));
        __syncwarp();
        if (box.any(left))
          tc::tma_load_4d(base + C::off_K + st * C::kTile + lay.at(box.at, 0), &tmK, 0, x.x, 0, x.y, &bars->kfull[st], pol_k);
        __syncwarp();
        ++k_issued;
        if (++st == C::kNS) st = 0;
        if (++t == te) {
          started = false;
          ++cur;
        }
      }
      // The CTA has made its last claim, and the fence waits for it (of a CTA without an item nothing has looked at the result): the
      // last CTA sets the counters back to zero for the next call.  Here, under the last item's work; at the end of the kernel
      // the fences cost 0.9 us.
      if (lane == 0) {
        __threadfence();
        if (atomicAdd(finished, 1u) == gridDim.x - 1) {
          __threadfence();
          *claim = 0u;
          *finished = 0u;
        }
      }
      if (!ok) {  // aborted: let issued loads land before the CTA exits
        for (unsigned j = k_issued > C::kNS ? k_issued - C::kNS : 0; j < k_issued; ++j)
          mbar_drain(bars->kfull + j % C::kNS, (j / C::kNS) & 1);
        for (unsigned j = q_issued > 2 ? q_issued - 2 : 0; j < q_issued; ++j) mbar_drain(&bars->qfull[j & 1], (j >> 1) & 1);
      }
    } else if (warp == kVWarp) {
      // ------------------------------------------------------------ V
      const uint64_t pol_v = policy_evict_last();
      if (lane == 0) tc::prefetch_tmap(&tmV);
      const Boxes box(p, lane);
      const KeyTile<D> lay(!rp.table);
      unsigned st = 0, v_issued = 0, n_clear = 0;
      bool ok = true;
      ItemReader reader;
      while (ok) {
        const TcItem* at = reader.next(bars, items, watch);
        if (!at) break;
        const int b = at->b, h = at->h, row0 = at->row0, klen = at->klen, t0 = at->t0, te = at->te;
        reader.release(bars, lane);
#pragma unroll 1
        for (int t = t0; t < te; ++t) {
          const int left = klen - t * kBN;
          const int2 x = box.any(left) ? box.where(rp, b, h, row0, t) : make_int2(0, 0);
          if (v_issued >= C::kNS) {  // P V of the tile that had the stage
            const unsigned j = v_issued - C::kNS;
            ok = warp_wait_watched(&bars->bfree[j % kSBufs], (j / kSBufs) & 1, watch);
            if (!ok) break;
          }
          const unsigned bi = v_issued % kSBufs;
          uint64_t* full = left < kBN ? &bars->vfull : &bars->pvfull[bi];
          if (lane == 0) mbar_arrive_expect_tx(full, box.bytes(left, !rp.table, 2 * D));
          __syncwarp();
          unsigned char* dst = base + C::off_V + st * C::kTile;
          if (box.any(left))
            tc::tma_load_4d(dst + lay.at(box.at, 0), &tmV, 0, x.x, 0, x.y, full, pol_v);
          __syncwarp();
          ++v_issued;
          if (left < kBN) {  // the item's last V tile: clear its rows past the last visible key
            ok = warp_wait_watched(&bars->vfull, n_clear & 1, watch);
            if (!ok) break;
            ++n_clear;
#pragma unroll 1
            for (int idx = left * C::kHalves * 8 + lane; idx < kBN * C::kHalves * 8; idx += 32)
              *reinterpret_cast<uint4*>(dst + lay.at(idx / (C::kHalves * 8), (idx >> 3) % C::kHalves) + (idx & 7) * 16) =
                  make_uint4(0u, 0u, 0u, 0u);
            tc::fence_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(&bars->pvfull[bi]);
          }
          if (++st == C::kNS) st = 0;
        }
      }
      if (!ok) {  // aborted: let issued loads land (a barrier that P never completes is waited for until its limit)
        for (unsigned j = v_issued > C::kNS ? v_issued - C::kNS : 0; j < v_issued; ++j)
          mbar_drain(&bars->pvfull[j % kSBufs], (j / kSBufs) & 1);
      }
    } else {
      // ------------------------------------------------------------ products
      const bool scores = warp == kSWarp;
      constexpr uint32_t idS = tc::idesc_bf16_f32(kBM, kBN, false, false);
      constexpr uint32_t idO = tc::idesc_bf16_f32(kBM, D, false, true);
      const uint64_t dQ0 = tc::sw128_desc(smem_u32(base + C::off_Q), 16, 1024);
      const KeyTile<D> lay(!rp.table);
      const uint64_t dK0 = tc::sw128_desc(smem_u32(base + C::off_K), 16, lay.group);
      const uint64_t dV0 = tc::sw128_desc(smem_u32(base + C::off_V), lay.half, lay.group);
      const uint64_t k_half = desc_step(lay.half), v_step = desc_step(2 * lay.group);  // 64 columns on; 16 keys on
      unsigned st = 0, phase = 0, bi = 0, b_phase = 0, n_items = 0;
      uint32_t col = tmem;
      bool ok = true;
      ItemReader reader;
      while (ok) {
        const TcItem* at = reader.next(bars, items, watch);
        if (!at) break;
        const int nt = at->te - at->t0;
        reader.release(bars, lane);
        if (nt == 0) continue;
        if (lane == 0) {
          if (scores) {
            // S(i) = Q K(i)^T into buffer i % 3, once P V of tile i - 3 has read that buffer
            const uint64_t dQ = dQ0 + (n_items & 1) * desc_step(C::kTile);
            ok = wait_watched(&bars->qfull[n_items & 1], (n_items >> 1) & 1, watch);
#pragma unroll 1
            for (int t = nt; ok && t > 0; --t) {
              ok = wait_watched(&bars->kfull[st], phase, watch) &&
                   wait_watched(&bars->bfree[bi], b_phase ^ 1, watch);
              if (!ok) break;
              tc::fence_after_sync();
              const uint64_t dK = dK0 + st * desc_step(C::kTile);
#pragma unroll
              for (int ks = 0; ks < D / 16; ++ks) {
                const uint64_t step = desc_step((ks & 3) * 32);
                tc::mma_bf16(col, dQ + desc_step((ks >> 2) * kAtom) + step, dK + (ks >> 2) * k_half + step, idS, ks > 0 ? 1u : 0u);
              }
              tc::mma_commit(&bars->sfull[bi]);
              if (++st == C::kNS) {
                st = 0;
                phase ^= 1;
              }
              col += kBN;
              if (++bi == kSBufs) {
                bi = 0;
                b_phase ^= 1;
                col = tmem;
              }
            }
          } else {
            // O (+)= P(i) V(i), P in the first 64 columns of buffer i % 3
            if (n_items > 0) ok = wait_watched(&bars->ofree, (n_items - 1) & 1, watch);
            uint32_t acc = 0;
#pragma unroll 1
            for (int t = nt; ok && t > 0; --t) {
              ok = wait_watched(&bars->pvfull[bi], b_phase, watch);
              if (!ok) break;
              tc::fence_after_sync();
              const uint64_t dV = dV0 + st * desc_step(C::kTile);
#pragma unroll
              for (int ks = 0; ks < kBN / 16; ++ks)
                tc::mma_bf16_ts(tmem + C::kColO, col + ks * 8, dV + ks * v_step, idO, ks > 0 ? 1u : acc);
              acc = 1;
              tc::mma_commit(&bars->bfree[bi]);
              if (t == 1) tc::mma_commit(&bars->olast);
              if (++st == C::kNS) {
                st = 0;
                phase ^= 1;
              }
              col += kBN;
              if (++bi == kSBufs) {
                bi = 0;
                b_phase ^= 1;
                col = tmem;
              }
            }
          }
        }
        ++n_items;
        ok = __shfl_sync(0xffffffffu, ok ? 1 : 0, 0) != 0;
      }
      if (lane == 0) {  // every product finished before TMEM is released
        uint64_t* bar = &bars->drained[scores ? 0 : 1];
        tc::mma_commit(bar);
        mbar_drain(bar, 0);
      }
    }
  } else if (warp >= kOutWarp0) {
    tc_regs_up<136>();
    // -------------------------------------------------------------- results
    const int quarter = warp - kOutWarp0;
    const int r = quarter * 32 + lane;
    const int token = r / rp.group;
    const uint32_t o_col = tmem + ((uint32_t)(quarter * 32) << 16) + C::kColO;
    __nv_bfloat16* out = reinterpret_cast<__nv_bfloat16*>(rp.out);
    float* parts = reinterpret_cast<float*>(p.scratch + kPartItemsBytes);
    constexpr size_t slot_floats = (size_t)kBM * (D + 2);
    unsigned n_items = 0;  // with tiles
    ItemReader reader;
    bool ok = true;
    while (ok) {
      const TcItem* item = reader.next(bars, items, watch);
      if (!item) break;
      const TcItem& it = *item;  // let go at the item's end
      const Seq s = {it.row0, it.rows, it.m, it.kv};
      const bool split = it.chunks > 1, keep = split || (kLong && (it.segment & kMore));  // keep: the results stay in the slot
      unsigned again = 0;  // rows whose result is not finite
      const int pos = it.pos0 + token;
      const bool valid = token < p.tokens && pos < it.rows;
      const int sees = valid ? seen(s, pos) : 0;
      const unsigned any = __ballot_sync(0xffffffffu, valid);
      if (it.te == it.t0) {  // no row sees a key: zeros
#pragma unroll 1
        for (int x = 0; x < 32; ++x)
          if ((any >> x) & 1u) {
            const int xr = quarter * 32 + x, xt = xr / rp.group;
            float y[D / 32];
#pragma unroll
            for (int e = 0; e < D / 32; ++e) y[e] = 0.f;
            store_row<D / 32>(out + ((size_t)(it.row0 + it.pos0 + xt) * rp.H + it.h * rp.group + (xr - xt * rp.group)) * D + lane * (D / 32), y);
          }
        reader.release(bars, lane);
        continue;
      }
      ok = warp_wait_watched(&bars->lready, n_items & 1, watch);
      if (!ok) break;
      if (lane == 0) put_off(watch);
      float l = l_row[r] + l_row[kBM + r], mx = m_row[r];
      __syncwarp();
      if (lane == 0) mbar_arrive(&bars->lfree);
      ok = warp_wait_watched(&bars->olast, n_items & 1, watch);
      if (!ok) break;
      ++n_items;
      tc::fence_after_sync();
      // O, 32 columns at a time, through what was the place of the item's queries (S is done with them), then out in whole
      // rows.  bf16: 16-byte piece e of row x at e ^ (x & 7) of its 256 (D = 64: 128) bytes; rolled loops (code size).
      unsigned char* stage = base + C::off_Q + ((n_items - 1) & 1) * C::kTile + quarter * 32 * (2 * D);
      float* part = parts + it.slot * slot_floats + r;
      if (kLong && (it.segment & kAfter)) {  // what this thread left there joins O
        const float m_before = part[0], top = fmaxf(mx, m_before);
        const float f = mx == top ? 1.f : fast_exp2(mx - top);  // (without a maximum: zeros, or NaN to stay)
        const float f_before = m_before == top ? 1.f : fast_exp2(m_before - top);
        l = f * l + f_before * part[kBM];
        mx = top;
#pragma unroll 1
        for (int c = 0; c < opaque(D / 32); ++c) {
          uint32_t o[32];
          tc::tmem_ld32(o_col + c * 32, o);
          tc::tmem_wait_ld();
#pragma unroll
          for (int e = 0; e < 32; ++e)
            o[e] = __float_as_uint(f * __uint_as_float(o[e]) + f_before * part[(2 + 32 * c + e) * kBM]);
          tc::tmem_st32(o_col + c * 32, o);
        }
        tc::tmem_wait_st();
      }
      const float inv = keep ? 1.f : sees > 0 ? 1.f / l : 0.f;
      const uint64_t inv2 = f2(inv, inv);
      uint64_t odd2 = 0ull;  // NaN once a result is not finite
#pragma unroll 1
      for (int c = 0; c < opaque(D / 32); ++c) {
        uint32_t o[32];
        tc::tmem_ld32(o_col + c * 32, o);
        tc::tmem_wait_ld();
        if (keep) {  // a partial result: fp32, rows side by side
          float* at = part + (2 + 32 * c) * kBM;
#pragma unroll
          for (int e = 0; e < 32; ++e) at[e * kBM] = __uint_as_float(o[e]);
          continue;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          uint32_t w[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const uint32_t* a = o + 8 * e + 2 * k;
            const uint64_t v = ffma2(f2(__uint_as_float(a[0]), __uint_as_float(a[1])), inv2, 0ull);
            odd2 = ffma2(v, 0ull, odd2);
            float lo, hi;
            unf2(v, lo, hi);
            w[k] = sees ? pack_bf16x2(lo, hi) : 0u;
          }
          *reinterpret_cast<uint4*>(stage + lane * (2 * D) + (((4 * c + e) ^ (lane & 7)) << 4)) = make_uint4(w[0], w[1], w[2], w[3]);
        }
      }
      tc::fence_before_sync();
      __syncwarp();
      if (lane == 0) mbar_arrive(&bars->ofree);
      if (keep) {
        part[0] = mx;
        part[kBM] = l;
        if (split && !(kLong && (it.segment & kMore)) && it.chunk == 0 && quarter == 0 && lane == 0) {
          const unsigned n = atomicAdd(reinterpret_cast<unsigned*>(p.ws + kPartsOff), 1u);
          reinterpret_cast<PartItem*>(p.scratch)[n] = {it.b, it.h, it.row0, it.m, it.kv, it.rows, it.pos0, it.chunks, it.slot, it.slot_step};
        }
      } else {
        constexpr int kPieces = D / 8, kRowsAt = 32 / kPieces;  // of a row; rows that the warp writes at once
        const int e = lane % kPieces;
        __nv_bfloat16* const to = out + ((size_t)(it.row0 + it.pos0) * rp.H + it.h * rp.group) * D + 8 * e;
#pragma unroll 8
        for (int x = lane / kPieces; x < 32; x += kRowsAt) {
          const uint4 v = *reinterpret_cast<const uint4*>(stage + x * (2 * D) + ((e ^ (x & 7)) << 4));
          if ((any >> x) & 1u) *reinterpret_cast<uint4*>(to + row_at[quarter * 32 + x]) = v;
        }
        float lo, hi;
        unf2(odd2, lo, hi);
        again = __ballot_sync(0xffffffffu, sees > 0 && l > 0.f && !(lo == 0.f && hi == 0.f));
        tc::fence_async_smem();  // the next queries come by the asynchronous proxy
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&bars->qempty[(n_items - 1) & 1]);
#pragma unroll 1
      while (again) {
        const int x = __ffs(again) - 1;
        again &= again - 1;
        __syncwarp();  // the row's first result is written
        const int xr = quarter * 32 + x, xt = xr / rp.group, xp = it.pos0 + xt;
        const int head = it.h * rp.group + (xr - xt * rp.group);
        float y[D / 32];
        attend_row<__nv_bfloat16, D>(rp, it.b, s, xp, head, seen(s, xp), y, [&] {
          if (lane == 0) put_off(watch);
        });
        store_row<D / 32>(out + ((size_t)(it.row0 + xp) * rp.H + head) * D + lane * (D / 32), y);
      }
      reader.release(bars, lane);
    }
  } else {
    tc_regs_up<136>();
    // -------------------------------------------------------------- softmax
    const int grp = warp >> 2, quarter = warp & 3;  // this group's tiles: CTA-local index parity grp
    const int r = quarter * 32 + lane;
    const int token = r / rp.group;
    const uint32_t lane_base = tmem + ((uint32_t)(quarter * 32) << 16);
    const float sl2 = rp.scale_log2;
    const uint64_t sc2 = f2(sl2, sl2);
    unsigned i = 0, n_items = 0;  // CTA-local tile, items with tiles
    ItemReader reader;
    bool ok = true;
    while (ok) {
      const TcItem* at = reader.next(bars, items, watch);
      if (!at) break;
      const Seq s = {at->row0, at->rows, at->m, at->kv};
      const int pos = at->pos0 + token;
      const int limit = token < p.tokens && pos < s.rows ? seen(s, pos) : 0;  // keys that this row sees
      const int all_see = seen(s, at->pos0);                                  // that every row of the tile sees
      const int t0 = at->t0, nt = at->te - t0;
      reader.release(bars, lane);
      if (nt == 0) continue;
      float m = -CUDART_INF_F, l = 0.f;  // the sum over this group's tiles and the reference that it is taken against
#pragma unroll 1
      for (int t = (int)((i ^ grp) & 1u); t < nt; t += 2) {
        const unsigned ti = i + t, bi = ti % kSBufs;
        const uint32_t s_col = lane_base + bi * kBN;
        ok = warp_wait_watched(&bars->sfull[bi], (ti / kSBufs) & 1, watch);
        if (!ok) break;
        tc::fence_after_sync();
        // keys that this row does not see: -inf (a suffix of the tile), written back in the 32-key chunks that have one
        const int key0 = (t0 + t) * kBN;
        if (key0 + kBN > all_see) {
          const int nv = limit - key0, nv_min = __reduce_min_sync(0xffffffffu, nv), nv_max = __reduce_max_sync(0xffffffffu, nv);
#pragma unroll 1
          for (int c = nv_min < 0 ? 0 : nv_min >> 5; c < opaque(kBN / 32); ++c) {
            uint32_t o[32];
            if (32 * c < nv_max) {
              tc::tmem_ld32(s_col + c * 32, o);
              tc::tmem_wait_ld();
            }
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] = 32 * c + e < nv ? o[e] : 0xff800000u;
            tc::tmem_st32(s_col + c * 32, o);
          }
          tc::tmem_wait_st();
        }
        // The scores are read from TMEM twice, 64 at a time in rolled loops (row max, then exponentials).
        float mx[4] = {-CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F};
#pragma unroll 1
        for (int half = 0; half < opaque(2); ++half) {
          uint32_t sv[64];
          tc::tmem_ld32(s_col + half * 64, *reinterpret_cast<uint32_t(*)[32]>(sv));
          tc::tmem_ld32(s_col + half * 64 + 32, *reinterpret_cast<uint32_t(*)[32]>(sv + 32));
          tc::tmem_wait_ld();
#pragma unroll
          for (int e = 0; e < 64; e += 8)
#pragma unroll
            for (int q = 0; q < 4; ++q) mx[q] = fmax3(mx[q], __uint_as_float(sv[e + 2 * q]), __uint_as_float(sv[e + 2 * q + 1]));
        }
        const float tmax = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * sl2;
        // The reference passes from tile to tile, so from group to group (one slot: a thread reads its row's before it writes
        // the next).
        float m_prev = -CUDART_INF_F;
        if (t > 0) {
          ok = warp_wait_watched(&bars->turn[quarter][(ti - 1) & 1], ((ti - 1) >> 1) & 1, watch);
          if (!ok) break;
          m_prev = m_ref[r];
        }
        const bool need = tmax > m_prev + kRescaleLog2;
        const float m_used = need ? tmax : m_prev;
        m_ref[r] = m_used;
        __syncwarp();
        if (lane == 0) mbar_arrive(&bars->turn[quarter][ti & 1]);
        if (__any_sync(0xffffffffu, need) && t > 0) {
          // O holds P V of this item's earlier tiles, the other group's last one included: rescale it
          const unsigned before = ti - 1;
          ok = warp_wait_watched(&bars->bfree[before % kSBufs], (before / kSBufs) & 1, watch);
          if (!ok) break;
          const float f = need ? fast_exp2(m_prev - m_used) : 1.f;
          tc::fence_after_sync();
#pragma unroll 1
          for (int c = 0; c < opaque(D / 32); ++c) {
            uint32_t o[32];
            tc::tmem_ld32(lane_base + C::kColO + c * 32, o);
            tc::tmem_wait_ld();
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
            tc::tmem_st32(lane_base + C::kColO + c * 32, o);
          }
          tc::tmem_wait_st();
        }
        if (m != m_used) {
          l *= fast_exp2(m - m_used);  // 0 while there is no sum
          m = m_used;
        }
        const float ref = m_used == -CUDART_INF_F ? 0.f : m_used;
        const uint64_t nm2 = f2(-ref, -ref);
        uint64_t acc[4] = {0ull, 0ull, 0ull, 0ull};
#pragma unroll 1
        for (int half = 0; half < opaque(2); ++half) {
          uint32_t sv[64], pk[32];
          tc::tmem_ld32(s_col + half * 64, *reinterpret_cast<uint32_t(*)[32]>(sv));
          tc::tmem_ld32(s_col + half * 64 + 32, *reinterpret_cast<uint32_t(*)[32]>(sv + 32));
          tc::tmem_wait_ld();
#pragma unroll
          for (int e = 0; e < 32; ++e) {
            float x0, x1;
            unf2(ffma2(f2(__uint_as_float(sv[2 * e]), __uint_as_float(sv[2 * e + 1])), sc2, nm2), x0, x1);
            const float p0 = fast_exp2(x0), p1 = fast_exp2(x1);
            acc[e & 3] = fadd2(acc[e & 3], f2(p0, p1));
            pk[e] = pack_bf16x2(p0, p1);
          }
          tc::tmem_st32(s_col + 32 * half, pk);  // over scores already read
        }
        tc::tmem_wait_st();
        tc::fence_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive(&bars->pvfull[bi]);
        float a0, a1, b0, b1;
        unf2(fadd2(acc[0], acc[1]), a0, a1);
        unf2(fadd2(acc[2], acc[3]), b0, b1);
        l += (a0 + a1) + (b0 + b1);
      }
      if (!ok) break;
      i += nt;
      if (((i ^ grp) & 1u) == 0) {  // the other group had the last tile: take this sum to its reference
        ok = warp_wait_watched(&bars->turn[quarter][(i - 1) & 1], ((i - 1) >> 1) & 1, watch);
        if (!ok) break;
        const float m_last = m_ref[r];
        if (m != m_last) l *= fast_exp2(m - m_last);
        m = m_last;
      }
      // to the result warps, once they have read the item before
      ok = warp_wait_watched(&bars->lfree, (n_items & 1) ^ 1, watch);
      if (!ok) break;
      l_row[grp * kBM + r] = l;
      if (((i ^ grp) & 1u) != 0) m_row[r] = m;
      __syncwarp();
      if (lane == 0) mbar_arrive(&bars->lready);
      ++n_items;
    }
  }

  __syncwarp();
  tc::fence_before_sync();
  __syncthreads();
  if (threadIdx.x == 0) record_abort(&watch->abort, status);
  if (warp == kKWarp) {
    tc::fence_after_sync();
    tc::tmem_dealloc(tmem, kTmemCols);
  }
}

// The items in chunks: a warp for 32 rows and kCols columns of one, a lane a row, four chunks' loads in flight.
//   out = sum_c 2^(m_c - M) o_c / sum_c 2^(m_c - M) l_c,  M = max_c m_c, in the order of the chunks
// Sixteen columns write whole 32-byte sectors of a row; eight make twice the tasks, for few items in many chunks.  Two
// requests of up to 512 new tokens, 40 heads (a call, us): 4 columns and eight chunks 91, eight 82, sixteen 78; one of 16
// tokens over 16384 keys, 32 heads over 8 cached: 32.8, 32.4 and 33.8.
constexpr int kMergeThreads = 256;
template <int D, int kCols>
__device__ __forceinline__ void merge_parts(const TcParams& p, int n) {
  constexpr int kTasks = kBM / 32 * (D / kCols), kAtOnce = 4;
  const RowsParams& rp = p.r;
  const int lane = threadIdx.x & 31;
  const float* parts = reinterpret_cast<const float*>(p.scratch + kPartItemsBytes);
  __nv_bfloat16* out = reinterpret_cast<__nv_bfloat16*>(rp.out);
  const int warps = gridDim.x * (kMergeThreads / 32);
#pragma unroll 1
  for (int task = blockIdx.x * (kMergeThreads / 32) + (threadIdx.x >> 5); task < n * kTasks; task += warps) {
    PartItem it;
    constexpr int kWords = sizeof(PartItem) / 4;
#pragma unroll
    for (int e = 0; e < kWords; ++e) reinterpret_cast<int*>(&it)[e] = __ldcg(reinterpret_cast<const int*>(p.scratch) + task / kTasks * kWords + e);
    const int rest = task % kTasks, r = rest / (D / kCols) * 32 + lane, col = rest % (D / kCols) * kCols;
    const int token = r / rp.group, pos = it.pos0 + token, head = it.h * rp.group + (r - token * rp.group);
    const bool valid = token < p.tokens && pos < it.rows;
    if (!__any_sync(0xffffffffu, valid)) continue;
    const Seq s = {it.row0, it.rows, it.m, it.kv};
    const float* at = parts + (size_t)it.slot * kBM * (D + 2) + r;
    const size_t step = (size_t)it.slot_step * kBM * (D + 2);
    float m = -CUDART_INF_F, l = 0.f, v[kCols];
#pragma unroll
    for (int e = 0; e < kCols; ++e) v[e] = 0.f;
#pragma unroll 1
    for (int c0 = 0; c0 < it.chunks; c0 += kAtOnce) {
      float mc[kAtOnce], lc[kAtOnce], o[kAtOnce][kCols];
#pragma unroll
      for (int c = 0; c < kAtOnce; ++c) {
        const float* from = at + (c0 + c) * step;
        const bool there = c0 + c < it.chunks;
        mc[c] = there ? __ldcg(from) : -CUDART_INF_F;
        lc[c] = there ? __ldcg(from + kBM) : 0.f;
#pragma unroll
        for (int e = 0; e < kCols; ++e) o[c][e] = there ? __ldcg(from + (2 + col + e) * kBM) : 0.f;
      }
      float top = m;
#pragma unroll
      for (int c = 0; c < kAtOnce; ++c) top = fmaxf(top, mc[c]);
      const float old = m == -CUDART_INF_F ? 1.f : fast_exp2(m - top);  // (sums without a maximum: zeros, or NaN to stay)
      l *= old;
#pragma unroll
      for (int e = 0; e < kCols; ++e) v[e] *= old;
#pragma unroll
      for (int c = 0; c < kAtOnce; ++c) {
        const float f = mc[c] == -CUDART_INF_F ? 0.f : fast_exp2(mc[c] - top);
        l += mc[c] == -CUDART_INF_F ? lc[c] : f * lc[c];
#pragma unroll
        for (int e = 0; e < kCols; ++e) v[e] += f * o[c][e];
      }
      m = top;
    }
    const int sees = valid ? seen(s, pos) : 0;
    bool odd = false;
#pragma unroll
    for (int e = 0; e < kCols; ++e) {
      v[e] = sees > 0 ? v[e] / l : 0.f;
      odd |= !isfinite(v[e]) && l > 0.f;
    }
    __nv_bfloat16* to = out + ((size_t)(it.row0 + pos) * rp.H + head) * D + col;
    if (valid)
#pragma unroll
      for (int e = 0; e < kCols; e += 8)
        *reinterpret_cast<uint4*>(to + e) = make_uint4(pack_bf16x2(v[e], v[e + 1]), pack_bf16x2(v[e + 2], v[e + 3]),
                                                       pack_bf16x2(v[e + 4], v[e + 5]), pack_bf16x2(v[e + 6], v[e + 7]));
    unsigned again = __ballot_sync(0xffffffffu, odd);  // by the definition, this warp's columns
#pragma unroll 1
    while (again) {
      const int x = __ffs(again) - 1, xr = rest / (D / kCols) * 32 + x, xt = xr / rp.group, xp = it.pos0 + xt;
      const int xh = it.h * rp.group + (xr - xt * rp.group);
      again &= again - 1;
      __syncwarp();  // the row's first result is written
      float y[D / 32];
      attend_row<__nv_bfloat16, D>(rp, it.b, s, xp, xh, seen(s, xp), y);
      const int first = lane * (D / 32);
      if (first >= col && first < col + kCols) store_row<D / 32>(out + ((size_t)(it.row0 + xp) * rp.H + xh) * D + first, y);
    }
  }
}

template <int D>
__global__ void __launch_bounds__(kMergeThreads) rows_merge_kernel(const TcParams p) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");  // the next call's start overlaps the merge
  pdl_wait();
  const int n = (int)__ldcg(reinterpret_cast<const unsigned*>(p.ws + kPartsOff));
  constexpr int kWide = kBM / 32 * (D / 16);  // tasks of an item
  if (n * kWide >= (int)gridDim.x * (kMergeThreads / 32) / 2) merge_parts<D, 16>(p, n);
  else merge_parts<D, 8>(p, n);
  __syncthreads();
  if (threadIdx.x == 0) {
    unsigned* merged = reinterpret_cast<unsigned*>(p.ws + kMergedOff);
    if (atomicAdd(merged, 1u) == gridDim.x - 1) {  // the counts back to zero for the next call
      *merged = 0u;
      *reinterpret_cast<unsigned*>(p.ws + kPartsOff) = 0u;
    }
  }
}

// bf16 keys or values in boxes of 64 columns x box1 x halves of D x box3 with the 128-byte swizzle; strides in elements.
bool keys_map(CUtensorMap* m, const void* base, int halves, long long d1, long long stride1, int box1, long long d3,
              long long stride3, int box3) {
  PFN_cuTensorMapEncodeTiled_v12000 fn = tensor_map_encoder();
  if (!fn) return false;
  const cuuint64_t dims[4] = {64, (cuuint64_t)d1, (cuuint64_t)halves, (cuuint64_t)d3};
  const cuuint64_t strides[3] = {(cuuint64_t)stride1 * 2, 128, (cuuint64_t)stride3 * 2};
  const cuuint32_t box[4] = {64, (cuuint32_t)box1, (cuuint32_t)halves, (cuuint32_t)box3};
  const cuuint32_t es[4] = {1, 1, 1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(base), dims, strides, box, es,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
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

// Key tiles of the longest item, by the bounds that the host has.
long long most_tiles(const RowsArgs& a) { return ((long long)(a.table ? a.max_kv : a.max_q) + kBN - 1) / kBN; }

template <int D, bool kLong>
cudaError_t launch_typed(const RowsArgs& a, cudaStream_t st) {
  using C = TcCfg<D>;
  static PerDevice<int> allowed;
  cudaError_t e = allow_smem(allowed, rows_tc_kernel<D, kLong>, (int)C::kSmem);
  if (e != cudaSuccess) return e;
  TcParams p;
  p.r = rows_params(a);
  p.ws = static_cast<unsigned char*>(a.ws);
  p.scratch = p.ws + WsLayout::kZeros;
  const int group = p.r.group;
  p.tokens = kBM / group;
  p.by_tokens = reciprocal(p.tokens);
  p.by_heads = reciprocal(a.Hkv);
  CUtensorMap mq, mk, mv;
  if (!rows_map(&mq, a.q, D, a.H, a.T, D, a.q_stride, group, p.tokens)) return cudaErrorNotSupported;
  if (a.table) {
    const int P = 1 << a.page_shift;
    p.box_rows = P < kBN ? P : kBN;
    const long long groups = (long long)a.n_pages * a.Hkv * (P / 8);  // of 8 rows
    if (groups > 0x7fffffffLL / 8) return cudaErrorNotSupported;  // 32-bit TMA coordinates
    if (!keys_map(&mk, a.K, C::kHalves, 8, D, 8, groups, 8 * D, p.box_rows / 8) ||
        !keys_map(&mv, a.V, C::kHalves, 8, D, 8, groups, 8 * D, p.box_rows / 8))
      return cudaErrorNotSupported;
  } else {
    p.box_rows = kBN;
    if (!keys_map(&mk, a.K, C::kHalves, a.T, a.k_stride, kBN, a.Hkv, D, 1) ||
        !keys_map(&mv, a.V, C::kHalves, a.T, a.v_stride, kBN, a.Hkv, D, 1))
      return cudaErrorNotSupported;
  }
  // claims, their counter's reach past the last one, and token coordinates past the last row stay in 32 bits
  const long long most = ((long long)a.T / p.tokens + a.B) * a.Hkv;
  if (most > 0x7fffffffLL - 2 * kMaxGrid || (long long)a.T + 4 * kBM > 0x7fffffffLL || (long long)a.max_kv + kBN > 0x7fffffffLL)
    return cudaErrorNotSupported;
  int G = sm_count() < kMaxGrid ? sm_count() : kMaxGrid;
  // Few enough items that some may be cut, by what the host knows of them
  const long long longest = most_tiles(a);
  p.may_split = 2 * most < 5ll * G && longest > kFewTiles;
  if (p.may_split && a.B == 1) {  // one sequence's items are known here, and so is a merge that would have nothing to do
    const int items = (a.max_q + p.tokens - 1) / p.tokens * a.Hkv, least = rounds_cost(items, G, (int)longest);
    p.may_split = 0;
    for (int i = 0; i < kSplitCount && items < 2 * G; ++i) {
      const int c = (int)((longest + split_of(i) - 1) / split_of(i)), n = (int)((longest + c - 1) / c);
      p.may_split |= split_cost(items * n, G, c) < least;
    }
  }
  e = launch_pdl(rows_tc_kernel<D, kLong>, dim3((unsigned)G), dim3(kTcThreads), C::kSmem, st, mq, mk, mv, p);
  if (e != cudaSuccess || !p.may_split) return e;
  return launch_pdl(rows_merge_kernel<D>, dim3((unsigned)(2 * G)), dim3(kMergeThreads), 0, st, p);
}

}  // namespace

size_t rows_workspace_bytes(int B, int H, int Hkv, int D, int T, int max_q, int dtype) {
  (void)B;
  (void)T;
  (void)max_q;
  if (dtype != 0 || H / Hkv > kBM) return WsLayout::kHeader;
  return WsLayout::kZeros + kPartItemsBytes + (size_t)kMaxChunks * kBM * (D + 2) * sizeof(float);
}

cudaError_t launch_rows_tc(const RowsArgs& a, cudaStream_t st) {
  if (a.dtype != 0 || a.H / a.Hkv > kBM) return cudaErrorNotSupported;
  if (most_tiles(a) > kSegTiles) return a.D == 128 ? launch_typed<128, true>(a, st) : launch_typed<64, true>(a, st);
  return a.D == 128 ? launch_typed<128, false>(a, st) : launch_typed<64, false>(a, st);
}

}  // namespace glide
