// slicemoe_mx4_product: rows of microscaled 4-bit activations times the matrices of the experts that a routing list names.
//
// The product is computed transposed, D[weight row, token] (128 weight rows x up to 224 tokens): the weights' rows are the fixed
// side of the tensor instruction, so that a tile with one token costs what it reads and no more.  An item is a block of 128
// weight rows times a tile of one expert's tokens; one persistent CTA per SM takes every grid'th item.  Steps of 256 values of K go
// through a ring in shared memory by bulk copies (the packed layout is the operand layout, and so is that of placed token rows),
// scales on to tensor memory by tcgen05.cp, four tcgen05.mma (kind mxf4, a scale per 32 values) a step.  Two accumulators in tensor
// memory: one is drained while the other fills.
//
// Sums are fp32 in tensor memory and rounded once.  Which column of a tile a token has does not enter its sum, so a row's
// result does not depend on the rest of the call.
//
// Bound and measured (B200, in a graph).  One token, gated, 6 experts of 1408 x 2048: 7.4 us where the weights come from HBM, 6.1 where L2
// still holds them; their 18.4 MB take 2.8 at the copy rate, the rest are latencies.  16 tokens that name 39 experts (119 MB): 24.3 us =
// 4.9 TB/s, and 22.2 from L2: 5.8 items to a CTA, so that some end early.  64 tokens, 59 experts: 33.6 us = 5.4 TB/s, the way from HBM.  2,048
// tokens x 4 of 60, gated: 56 us, HBM (184 MB of weights), the placing of the rows ahead, and ramp and tail.  8,192 x 6, 2048 x 1408: 125 us =
// 2.3 PFLOP/s (140 where it goes on for tenths of a second, at the power limit's clocks): 20 us of placing, and the drain.  An item of 224
// tokens is 5.5 steps of 711 clocks of shared-memory traffic (47 KB come in and 44 KB are read at 128 bytes a clock; its products take 448), 3,900,
// which the drain's exchanges and 4-byte stores, on the same way, are longer than.
#include "decode_common.cuh"
#include "mx4.cuh"

namespace slicemoe {

// The head of a workspace: as far as slicemoe_get_status and slicemoe_workspace_set_wait go it is that of the layer calls (WsHeader in
// decode.cu: status at 8, the switch at 12, the limit at 16).
struct MpHeader {
  unsigned unused0, unused1;
  unsigned status;
  unsigned extra_arrivals;  // != 0: the weights are never brought, and the waits for them run out
  unsigned long long wait_cycles;
};
static_assert(offsetof(MpHeader, status) == 8 && offsetof(MpHeader, extra_arrivals) == 12 && offsetof(MpHeader, wait_cycles) == 16, "WsHeader");
constexpr int kMpMaxExperts = 1024;
constexpr int64_t kMpMaxPairs = 1 << 24;
constexpr int kMpTile = 224, kMpLeastTile = 32;  // most tokens of a tile; of a narrow one
constexpr int kMpFew = 512;          // up to so many pairs, and
constexpr int kMpResident = 96 * 1024;  // so many bytes of token rows, every CTA keeps all rows and plans for itself
constexpr int kMpSortPairs = 4096;   // else: pairs of a block of the kernel that ranks them
constexpr int kMpPlaceAll = 8192;    // pairs up to which the kernel that places them ranks them too
constexpr int kMpSortThreads = 1024, kMpPlaceThreads = 256;

// An expert's rows are cut into as few tiles as they fit, of equal size (a multiple of 16).
struct MpTiles {
  int n, each;
};
__host__ __device__ inline MpTiles mp_tiles(int rows, int tile) {
  MpTiles t;
  t.n = (rows + tile - 1) / tile;
  t.each = t.n ? ((rows + t.n - 1) / t.n + 15) & ~15 : 0;
  return t;
}
// Most rows of a tile.  An expert has at most T rows where no token names one twice: wider tiles would only take room from the ring.  And
// narrower ones, down to kMpLeastTile, while there are no more items than SMs: they are drained side by side then, and their
// weights come from L2 for all but the first.  (483 tokens, 3 experts of 335 x 768, gated: 10.8 us in tiles of 161, 8.0 in tiles of 32.
// Past the number of SMs it turns round: 2,854 tokens x 3 of 3 experts of 282 x 1,280, 18.0 us in 117 items, 21.9 in 153.)
inline int mp_tile(int T, int pairs, int E, int row_blocks, int sms) {
  int tile = T >= kMpTile ? kMpTile : (T + 15) & ~15;
  const int used = pairs < E ? pairs : E, rows = (pairs + used - 1) / used;
  while (tile > kMpLeastTile && (int64_t)used * ((rows + tile - 17) / (tile - 16)) * row_blocks <= sms) tile -= 16;
  return tile;
}

// Token rows lie as the tensor instruction takes an operand: by steps of 256 values, in a step a row's 128 bytes after the other, their eight
// pieces of 16 bytes swapped about by the row (piece c at c ^ (row % 8): the 128-byte swizzle).  Eight rows begin at a multiple of 1024.
constexpr int kMpStepChunks = 4;  // chunks of 64 values a step
constexpr int kMpRowBytes = kMpStepChunks * kMxChunk / 2;
__host__ __device__ inline int mp_steps(int K) { return (mx_chunks(K) + kMpStepChunks - 1) / kMpStepChunks; }
__device__ __forceinline__ uint32_t mp_piece(uint32_t rows, uint32_t row, uint32_t piece) {  // where a piece of 16 bytes lies in a tile
  return (piece >> 3) * rows * kMpRowBytes + row * kMpRowBytes + ((piece ^ row) & 7) * 16;
}

// Workspace: header; ranks of the pairs among the block's of their expert, and the blocks' counts; rows, tiles and tiles' rows before each
// expert; the pairs by expert; token rows in the operand layout.  Every part grows with each argument, so that a workspace serves smaller calls.
struct MpLayout {
  size_t rank, hist, first, list, scale, codes, total;
  int blocks;
};
__host__ __device__ inline MpLayout mp_layout(int T, int k, int E, int K) {
  auto up = [](size_t v) { return (v + 255) & ~(size_t)255; };
  // tiles, of the narrowest kind; one above 128 rows has two blocks of scales, and there are fewer than half as many of those
  const int64_t pairs = (int64_t)T * k, tiles = (pairs / kMpLeastTile > k ? pairs / kMpLeastTile : k) + 2 * (pairs < E ? pairs : E) + 2;
  MpLayout l;
  l.blocks = (int)((pairs + kMpSortPairs - 1) / kMpSortPairs);
  l.rank = 256;
  l.hist = l.rank + up(pairs * sizeof(int));
  l.first = l.hist + up((size_t)l.blocks * E * sizeof(int));
  l.list = l.first + up((size_t)3 * (E + 1) * sizeof(int));
  l.scale = l.list + up(pairs * sizeof(int));
  l.codes = l.scale + up((size_t)tiles * mx_atoms(K) * kMxAtomBytes);
  l.total = l.codes + up((size_t)(pairs + 16 * tiles) * mp_steps(K) * kMpRowBytes);
  return l;
}

// ---- pairs by expert, and their rows into tiles --------------------------------------------------------------------
// Exclusive scans over the block of three values per thread, side by side; total gets the sums.
template <int THREADS>
__device__ __forceinline__ void mp_scan3(int (&v)[3], int (*s)[3], int (&total)[3]) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int inc[3] = {v[0], v[1], v[2]};
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    int a[3];
#pragma unroll
    for (int i = 0; i < 3; ++i) a[i] = __shfl_up_sync(0xffffffffu, inc[i], off);
#pragma unroll
    for (int i = 0; i < 3; ++i)
      if (lane >= off) inc[i] += a[i];
  }
  __syncthreads();
  if (lane == 31) s[warp][0] = inc[0], s[warp][1] = inc[1], s[warp][2] = inc[2];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    const int w = lane < THREADS / 32 ? s[lane][i] : 0, before = lane < warp ? w : 0;
    total[i] = __reduce_add_sync(0xffffffffu, w);
    v[i] = __reduce_add_sync(0xffffffffu, before) + inc[i] - v[i];
  }
}

struct MpSortParams {
  const int32_t* ids;
  int pairs, E;
  int* rank;
  int* hist;  // [block][E]
  MpHeader* head;
};
// A pair's rank among the block's of its expert is what the counting atomic returns.  (It depends on the atomics' order; which column
// of a tile a pair gets does not enter its result.)
__global__ void __launch_bounds__(kMpSortThreads) mp_sort_kernel(const MpSortParams p) {
  __shared__ int s_count[kMpMaxExperts];
  mx_dep_launch();
  const int tid = threadIdx.x;
  s_count[tid] = 0;
  mx_dep_wait();
  __syncthreads();
  constexpr int kEach = kMpSortPairs / kMpSortThreads;
  const int base = blockIdx.x * kMpSortPairs + tid;
  int e[kEach];
  bool bad = false;
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int at = base + i * kMpSortThreads;
    e[i] = at < p.pairs ? __ldcg(p.ids + at) : -1;
    bad |= at < p.pairs && (unsigned)e[i] >= (unsigned)p.E;
  }
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int at = base + i * kMpSortThreads;
    if (at < p.pairs) p.rank[at] = (unsigned)e[i] < (unsigned)p.E ? atomicAdd(&s_count[e[i]], 1) : -1;
  }
  __syncthreads();
  if (tid < p.E) p.hist[(size_t)blockIdx.x * p.E + tid] = s_count[tid];
  if (bad) atomicOr(&p.head->status, (unsigned)SLICEMOE_STATUS_BAD_EXPERT_ID);
}

struct MpPlaceParams {
  const int32_t* ids;  // NULL: all of expert 0, in order
  const int *rank, *hist;
  const uint8_t *codes, *scale;
  int *first, *list;    // first: [3][E + 1], rows, tiles and tiles' rows before an expert
  uint8_t *t_codes, *t_scale;
  int pairs, E, blocks, chunk, tile, k, x_per_pair, K;
  MpHeader* head;
};
// Each pair's row to its place in its tile; scales as those of packed weights.  A block takes `chunk` pairs of one block of ranks: where they
// go is worked out by a thread each, then a warp moves two or four rows at a time.  A row is read in runs of 512 bytes and written in runs of
// 128, which is what the swizzled operand layout keeps together.  (Without the swizzle a row's pieces of 16 bytes lie apart: 9 us
// for 8,192 rows of 2,048 values and 28 for 49,152 of 1,408, in whichever order the rows are taken.)
constexpr int kMpPlaceChunk = 128;
struct MpPlace {
  uint32_t x, code, scale, row;  // row of x (all ones: none); rows, and blocks of scales, before the tile; rows of the tile << 16 | row in it
};
// FEW: no kernel has ranked the pairs; every block looks at all of them and takes 32 of them itself, which saves a launch.  That pays while all
// blocks are resident together, two to an SM: 296 of them, 9,472 pairs.  Products in a graph, so / by two launches, in us:
//   pairs                               1,024          4,096          8,192          10,240         16,384
//   16 experts, 256 x 512            8.1 /  9.1    10.0 / 10.8    12.2 / 12.7    16.9 / 13.5    25.3 / 17.3
//   64 experts, 256 x 256            8.7 /  9.3    11.3 / 12.0    13.7 / 14.2    19.0 / 15.4    24.7 / 16.5
//   60 experts, gated 1408 x 2048   38.8 / 41.7    42.6 / 45.3    49.2 / 51.7    60.1 / 57.4    86.5 / 78.9
//   64 experts, 2048 x 1408         26.0 / 29.5    29.1 / 33.1    35.7 / 37.8    44.5 / 41.3    63.3 / 56.1
//   256 experts, 512 x 2048         34.8 / 37.3    36.7 / 39.8    40.1 / 42.2    46.7 / 43.5    53.9 / 46.1
template <bool FEW>
__global__ void __launch_bounds__(FEW ? 2 * kMpPlaceThreads : kMpPlaceThreads, FEW ? 2 : 4) mp_place_kernel(const MpPlaceParams p) {
  constexpr int kThreads = FEW ? 2 * kMpPlaceThreads : kMpPlaceThreads, kRows = FEW ? 2 : 4;
  __shared__ int s_first[kMpMaxExperts], s_before[kMpMaxExperts], s_count[kMpMaxExperts], s_tile[kMpMaxExperts], s_row[kMpMaxExperts], s_sums[32][3];
  __shared__ MpPlace s_place[kMpPlaceChunk];
  mx_dep_launch();
  if constexpr (FEW)
    for (int e = threadIdx.x; e < p.E; e += kThreads) s_count[e] = s_before[e] = 0;
  mx_dep_wait();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int base = blockIdx.x * p.chunk, me = base / kMpSortPairs;
  int own = -1, own_rank = 0;
  if constexpr (FEW) {
    __syncthreads();
    if (tid < 32 && base + tid < p.pairs) own = __ldcg(p.ids + base + tid);
    constexpr int kAhead = 8;
    bool bad = false;
    for (int i0 = tid; i0 < p.pairs; i0 += kAhead * kThreads) {
      int id[kAhead];
#pragma unroll
      for (int i = 0; i < kAhead; ++i) id[i] = i0 + i * kThreads < p.pairs ? __ldcg(p.ids + i0 + i * kThreads) : -1;
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        const int at = i0 + i * kThreads;
        if ((unsigned)id[i] < (unsigned)p.E) {
          atomicAdd(&s_count[id[i]], 1);
          if (at < base) atomicAdd(&s_before[id[i]], 1);
        } else {
          bad |= at < p.pairs;
        }
      }
    }
    if (bad && blockIdx.x == 0) atomicOr(&p.head->status, (unsigned)SLICEMOE_STATUS_BAD_EXPERT_ID);
    __syncthreads();
  }
  int sum[3] = {};
  for (int e0 = 0; e0 < p.E; e0 += kThreads) {
    const int e = e0 + tid;
    int count = 0, before = 0;
    if (e < p.E) {
      if constexpr (FEW) {
        count = s_count[e], before = s_before[e];
      } else if (p.ids) {
#pragma unroll 8
        for (int b = 0; b < p.blocks; ++b) {
          const int n = __ldcg(p.hist + (size_t)b * p.E + e);
          count += n;
          before += b < me ? n : 0;
        }
      } else {
        count = p.pairs;
      }
    }
    const MpTiles t = mp_tiles(count, p.tile);
    int v[3] = {count, t.n, t.n * t.each}, total[3];
    mp_scan3<kThreads>(v, s_sums, total);
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      v[i] += sum[i];
      sum[i] += total[i];
    }
    if (e < p.E) {
      s_first[e] = v[0], s_before[e] = before, s_count[e] = count, s_tile[e] = v[1], s_row[e] = v[2];
      if (blockIdx.x == 0) p.first[e] = v[0], p.first[p.E + 1 + e] = v[1], p.first[2 * (p.E + 1) + e] = v[2];
    }
  }
  if (blockIdx.x == 0 && tid == 0) p.first[p.E] = sum[0], p.first[2 * p.E + 1] = sum[1];
  const int atoms = mx_atoms(p.K), pieces = 2 * mx_chunks(p.K), kbytes = p.K >> 1, halves = (p.tile + 127) >> 7, steps = mp_steps(p.K);
  for (int c0 = 0; c0 < p.chunk; c0 += kMpPlaceChunk) {
    const int here = min(kMpPlaceChunk, p.chunk - c0);
    if constexpr (FEW) {
      if (warp == 0) own_rank = __popc(__match_any_sync(0xffffffffu, own) & ((1u << lane) - 1u));  // in their order
    }
    __syncthreads();
    if (tid < here) {
      const int pair = base + c0 + tid;
      MpPlace at = {0xffffffffu, 0, 0, 0};
      if (pair < p.pairs) {
        int e = own, rank = own_rank;
        if constexpr (!FEW) e = p.ids ? __ldcg(p.ids + pair) : 0, rank = p.ids ? __ldcg(p.rank + pair) : pair;
        if ((unsigned)e < (unsigned)p.E) {
          const int pos = p.ids ? s_before[e] + rank : pair, count = s_count[e];
          const MpTiles t = count <= p.tile ? MpTiles{1, (count + 15) & ~15} : mp_tiles(count, p.tile);
          const int tile = t.n == 1 ? 0 : pos / t.each;
          at.x = p.x_per_pair ? pair : pair / p.k;
          at.code = s_row[e] + tile * t.each;
          at.scale = s_tile[e] + tile;
          at.row = t.each << 16 | (pos - tile * t.each);
          p.list[s_first[e] + pos] = pair;
        }
      }
      s_place[tid] = at;
    }
    __syncthreads();
    for (int i = warp * kRows; i < here; i += kThreads / 32 * kRows) {
      // loads first, then stores: left to itself the compiler cannot know that they do not overlap, and waits for each
      for (int q = lane; q < pieces; q += 32) {
        uint4 v[kRows];
#pragma unroll
        for (int l = 0; l < kRows; ++l) {
          const uint32_t x = s_place[i + l].x;
          v[l] = ~x && q * 16 < kbytes ? __ldcg(reinterpret_cast<const uint4*>(p.codes + (size_t)x * kbytes) + q) : make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int l = 0; l < kRows; ++l) {
          const MpPlace at = s_place[i + l];
          if (~at.x) *reinterpret_cast<uint4*>(p.t_codes + (size_t)at.code * steps * kMpRowBytes + mp_piece(at.row >> 16, at.row & 0xffffu, q)) = v[l];
        }
      }
      for (int j = lane; j < atoms; j += 32) {
        const int left = (p.K >> 5) - 4 * j;
        uint32_t w[kRows];
#pragma unroll
        for (int l = 0; l < kRows; ++l) {
          const uint32_t x = s_place[i + l].x;
          w[l] = ~x ? __ldcg(reinterpret_cast<const uint32_t*>(p.scale + (size_t)x * (4 * atoms)) + j) : 0u;
        }
#pragma unroll
        for (int l = 0; l < kRows; ++l) {
          const MpPlace at = s_place[i + l];
          const uint32_t r = at.row & 0xffffu;
          if (left < 4) w[l] &= (1u << (8 * left)) - 1u;  // bytes beyond the row's end
          if (~at.x)
            *reinterpret_cast<uint32_t*>(p.t_scale + (((size_t)at.scale * atoms + j) * halves + (r >> 7)) * kMxAtomBytes + (r & 31) * 16 +
                                         ((r >> 5) & 3) * 4) = w[l];
        }
      }
    }
  }
}

// ---- the product ----------------------------------------------------------------------------------------------------
constexpr int kMpWeightWarp = 0, kMpMmaWarp = 1, kMpPlanWarp = 2, kMpTileWarp = 3, kMpFirstDrain = 4, kMpDrainWarps = 8;  // the fourth brings placed tiles, or helps to lay out resident rows
constexpr int kMpThreads = 32 * (kMpFirstDrain + kMpDrainWarps);
constexpr int kMpTable = 128;                // table entries that a CTA keeps in shared memory
constexpr int kMpSlots = 4, kMpMaxStages = 12;
constexpr int kMpTmemCols = 512;
constexpr int kMpScaleCol = 2 * kMpTile;     // behind the two accumulators: scales of two steps, 8 + 16 columns each
constexpr int kMpScaleCols = 24;
static_assert(kMpScaleCol + 2 * kMpScaleCols <= kMpTmemCols, "tensor memory");
constexpr int kMpABytes = kMpStepChunks * kMxChunkBytes, kMpAScaleBytes = kMpStepChunks / 2 * kMxAtomBytes;

struct MpItem {
  const uint8_t *codes, *scale;      // the row block's weights
  const uint8_t *t_codes, *t_scale;  // the placed tile
  int n;         // columns, a multiple of 16; < 0: no more items
  int rows;      // rows of the tile as it lies, a multiple of 16
  int rb;        // row block
  uint32_t groups;  // the sixteens of columns that hold pairs of the item
};
struct __align__(16) MpSmem {
  unsigned long long full[kMpMaxStages], free_[kMpMaxStages];
  unsigned long long acc_full[2], acc_free[2], item_known[kMpSlots], item_full[kMpSlots], item_free[kMpSlots], resident, drain;
  uint32_t tmem;
  int pad0;
  int dead, pad1;
  unsigned long long limit;  // 8 bytes behind dead
  MpItem item[kMpSlots];
  alignas(16) int pair[kMpSlots][kMpTile];  // of a column; -1: none; read four at a time
  slicemoe_mx4_mat mats[kMpTable];
  int first[kMpMaxExperts + 1];  // rows before an expert
  int tiles[kMpMaxExperts + 1];  // tiles before it
  int padded[kMpMaxExperts];     // rows of the tiles before it
  uint32_t place[2][kMpMaxStages];  // where the steps under way begin, as either filler knows it
  int key[kMpFew], tile[kMpFew]; // of a pair, and of a tile, where the CTA plans for itself: expert, and how often the token named it before << 16
};
static_assert(offsetof(MpSmem, pair) % 16 == 0 && kMpTile % 4 == 0 && offsetof(MpSmem, mats) % 8 == 0, "alignment");
static_assert(offsetof(MpSmem, limit) == offsetof(MpSmem, dead) + 8, "wait_limit()");
constexpr int kMpFixed = (int)((sizeof(MpSmem) + 1023) / 1024 * 1024);
constexpr int kMpSmem = 227 * 1024;  // all of it, whatever the call: one CTA to an SM, since each takes all of tensor memory

// A step in the ring: weights, their scales, token rows, their scales.  Steps lie one behind the other, each as long as its item's
// tile needs, and start again at 0 where the next does not fit: who fills and who reads work out the same places.
__host__ __device__ constexpr uint32_t mp_step_bytes(int rows, int halves) {
  return kMpABytes + kMpAScaleBytes + rows * kMpRowBytes + halves * kMpAScaleBytes;
}
__device__ __forceinline__ uint32_t mp_next_place(uint32_t& head, uint32_t bytes, uint32_t ring) {
  const uint32_t at = head + bytes <= ring ? head : 0;
  head = at + bytes;
  return at;
}

struct MpParams {
  const slicemoe_mx4_mat* mats;
  const uint8_t* codes;
  const uint8_t* scale;
  const int32_t* ids;
  void* out;
  MpHeader* head;
  const int *first, *list;             // of the placed rows
  const uint8_t *t_codes, *t_scale;
  int E, N, K, gated, T, k, x_per_pair;
  uint32_t k_inverse;    // ceil(2^32 / k), for k > 1
  int tile;              // most tokens of a tile, a multiple of 16; resident: all rows
  int resident;          // bytes of resident rows and their scales
  int stages, ring;      // steps that may be under way, and the bytes that they share
  int row_blocks;
};

// Operand descriptors without swizzle: 8 rows x 16 bytes one after the other, 128 bytes on to the next eight rows (weights and all scales
// alike), `lead` bytes to the next 16 bytes of a row.  The upper half is the same for all.
constexpr uint32_t kMpDescHigh = (128 >> 4) | 1u << 14, kMpDescSwizzled = (1024 >> 4) | 1u << 14 | 2u << 29;
__device__ __forceinline__ uint64_t mp_desc(uint32_t low) { return (uint64_t)kMpDescHigh << 32 | low; }
// Of token rows: 128-byte swizzle, 1024 bytes to the next eight rows.
__device__ __forceinline__ uint64_t mp_desc_rows(uint32_t low) { return (uint64_t)kMpDescSwizzled << 32 | low; }
// E2M1 x E2M1, E8M0 scales, M 128, N tokens.  Bits 29 and 4: which pair of the four scale bytes, see mp_mma.
__device__ __forceinline__ uint32_t mp_idesc(int n) {
  return (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | (1u << 23) | ((uint32_t)(kMxRows >> 4) << 24);
}
__device__ __forceinline__ bool mp_elect() {
  uint32_t p;
  asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}" : "=r"(p));
  return p != 0;
}
__device__ __forceinline__ void mp_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sa, uint32_t sb, uint32_t acc) {
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.b32 p, %6, 0;\n"
      " tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(acc)
      : "memory");
}
// 32 rows x 16 bytes of shared memory to four columns, the same in all four quarters of the lanes.
__device__ __forceinline__ void mp_copy_scales(uint32_t tmem, uint64_t desc) {
  asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
}
__device__ __forceinline__ void mp_commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void mp_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void mp_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void mp_ld16(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];\n"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
        "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void mp_bulk(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar)
               : "memory");
}
// By a whole warp; every lane gets the same answer.
__device__ __forceinline__ bool mp_wait(const void* bar, uint32_t parity, MpSmem* s, unsigned* status) {
  return __all_sync(0xffffffffu, mbar_wait(smem_u32(bar), parity, &s->dead, status));
}
// silu(g) u.  __expf(-g) is off by (2 + 1.2 |g|) 2^-23, which enters with the weight of e^-g / (1 + e^-g); |silu(g)| (2 + 1.2 |g|) times
// that weight stays below 1.3 |g|: an error of 1.3 x 2^-23 |g u|, no more than that of the sums behind g and u (each of at least
// 32 products).  __fdividef adds 2 ulp, and gives 0 for e^-g above 2^126, where the quotient is below 2^-119.
__device__ __forceinline__ float mp_gated(float g, float u) { return __fdividef(g, 1.0f + __expf(-g)) * u; }

template <class O>
__device__ __forceinline__ uint32_t mp_pack2(float a, float b) {
  const O e[2] = {mx_from_float<O>(a), mx_from_float<O>(b)};
  uint32_t w;
  memcpy(&w, e, 4);
  return w;
}

// PLACED: token rows come tile by tile, as mp_place_kernel has laid them out.  Else all rows of the call are resident in shared memory, and
// an item's tile is all of them: the tensor instruction takes hardly longer for the columns that no pair of the item uses, and
// nothing has to be gathered.
template <class O, bool GATED, bool PLACED>
__global__ void __launch_bounds__(kMpThreads, 1) mp_product_kernel(const MpParams p) {
  extern __shared__ __align__(1024) uint8_t mp_smem[];
  MpSmem* s = reinterpret_cast<MpSmem*>(mp_smem);
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  const int chunks = mx_chunks(p.K), atoms = mx_atoms(p.K), steps = (chunks + kMpStepChunks - 1) / kMpStepChunks;
  const int halves = (p.tile + 127) >> 7;  // scale blocks of 128 tokens
  const uint32_t rows_at = smem_u32(mp_smem) + kMpFixed, ring = rows_at + p.resident;
  unsigned* status = &p.head->status;

  mx_dep_launch();
  if (warp == kMpMmaWarp) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&s->tmem)), "r"(kMpTmemCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  } else if (warp == kMpPlanWarp) {
    if (lane == 0) {
      s->dead = 0;
      const unsigned long long cycles = __ldcg(&p.head->wait_cycles);
      s->limit = cycles ? cycles : kWaitCycles;
    }
  } else if (warp >= kMpFirstDrain && warp < kMpFirstDrain + 2) {
    // one barrier to a thread: they lie one behind the other in the order of MpSmem
    const int i = tid - 32 * kMpFirstDrain;
    constexpr int kRing = 2 * kMpMaxStages, kAll = kRing + 4 + 3 * kMpSlots + 2;
    static_assert(kAll <= 64 && offsetof(MpSmem, drain) == 8 * (kAll - 1), "barriers");
    int arrivals = i < kMpMaxStages && PLACED ? 2 : 1;
    if (i >= kRing + 2 && i < kRing + 4) arrivals = kMpDrainWarps;
    if (i >= kRing + 4 + 2 * kMpSlots && i < kRing + 4 + 3 * kMpSlots) arrivals = (PLACED ? 3 : 2) + kMpDrainWarps;
    if (i == kAll - 2) arrivals = kMpDrainWarps + 1;
    if (i < kAll) mbar_init(smem_u32(&s->full[0] + i), arrivals);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  const int pairs = p.T * p.k;
  if (!PLACED && pairs > 32)
    for (int e = tid; e < p.E; e += kMpThreads) s->first[e] = 0;
  mp_fence_before();
  __syncthreads();
  mp_fence_after();
  const uint32_t tmem = s->tmem;

  if (!PLACED && pairs > 32) {
    // more pairs than lanes: all warps look at them.  A tile of an expert takes one pair of a token; first[] counts its tiles
    mx_dep_wait();
    for (int i = tid; i < pairs; i += kMpThreads) {
      int e = p.ids ? __ldcg(p.ids + i) : 0;
      if ((unsigned)e >= (unsigned)p.E) {
        e = -1;
        if (blockIdx.x == 0) atomicOr(status, (unsigned)SLICEMOE_STATUS_BAD_EXPERT_ID);
      }
      s->tile[i] = e;
    }
    __syncthreads();
    for (int i = tid; i < pairs; i += kMpThreads) {
      const int e = s->tile[i], t0 = p.k > 1 ? (int)__umulhi((uint32_t)i, p.k_inverse) * p.k : i;
      int before = 0;
      for (int j = t0; j < i; ++j) before += s->tile[j] == e;
      s->key[i] = e < 0 ? -1 : e | before << 16;
      if (e >= 0) atomicMax(&s->first[e], before + 1);
    }
    __syncthreads();
  }
  if (warp == kMpPlanWarp) {
    // ---- the plan: rows by expert, then which item is next, and its rows.  One warp does it, the others wait for their first item: with
    // few pairs that is a chain of latencies which barriers of the whole CTA would only lengthen ----
    int at = blockIdx.x / p.row_blocks, rest = blockIdx.x - at * p.row_blocks;  // an item's place among the tiles
    const int at_step = gridDim.x / p.row_blocks, rest_step = gridDim.x - at_step * p.row_blocks;
    int total_tiles = 0;
    if (p.E <= kMpTable) {
      // the table does not change between launches: it is asked for while the kernel before is still at work
      constexpr int kWords = sizeof(slicemoe_mx4_mat) / 8, kAhead = 8;
      for (int i0 = lane; i0 < p.E * kWords; i0 += 32 * kAhead) {
        unsigned long long w[kAhead];
#pragma unroll
        for (int a = 0; a < kAhead; ++a)
          if (i0 + 32 * a < p.E * kWords) w[a] = __ldg(reinterpret_cast<const unsigned long long*>(p.mats) + i0 + 32 * a);
#pragma unroll
        for (int a = 0; a < kAhead; ++a)
          if (i0 + 32 * a < p.E * kWords) reinterpret_cast<unsigned long long*>(s->mats)[i0 + 32 * a] = w[a];
      }
    }
    mx_dep_wait();
    if constexpr (PLACED) {
      for (int e = lane; e <= p.E; e += 32) {
        s->first[e] = __ldcg(p.first + e);
        s->tiles[e] = __ldcg(p.first + p.E + 1 + e);
        if (e < p.E) s->padded[e] = __ldcg(p.first + 2 * (p.E + 1) + e);
      }
    } else if (pairs <= 32) {
      int e = -1;
      if (lane < pairs) {
        e = p.ids ? __ldcg(p.ids + lane) : 0;
        if ((unsigned)e >= (unsigned)p.E) {
          e = -1;
          if (blockIdx.x == 0) atomicOr(status, (unsigned)SLICEMOE_STATUS_BAD_EXPERT_ID);
        }
      }
      const unsigned lower = (1u << lane) - 1u, token = p.k > 1 ? ~0u << (__umulhi((uint32_t)lane, p.k_inverse) * p.k) : ~0u << lane;
      const unsigned same = __match_any_sync(0xffffffffu, e);  // by all lanes, whatever they hold
      const int key = e < 0 ? -1 : e | __popc(same & lower & token) << 16;
      const unsigned alike = __match_any_sync(0xffffffffu, key);
      const bool leads = key >= 0 && (alike & lower) == 0;
      const unsigned all = __ballot_sync(0xffffffffu, leads);
      s->key[lane] = key;
      if (leads) s->tile[__popc(all & lower)] = key;
      total_tiles = __popc(all);
    } else {
      for (int e0 = 0; e0 < p.E; e0 += 32) {
        const int e = e0 + lane, count = e < p.E ? s->first[e] : 0;
        int inc = count;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
          const int o = __shfl_up_sync(0xffffffffu, inc, off);
          if (lane >= off) inc += o;
        }
        for (int m = 0; m < count; ++m) s->tile[total_tiles + inc - count + m] = e | m << 16;
        total_tiles += __shfl_sync(0xffffffffu, inc, 31);
      }
    }
    __syncwarp();
    if constexpr (PLACED) total_tiles = s->tiles[p.E];
    uint32_t slot = 0, turn = 0;
    for (;; at += at_step, rest += rest_step) {
      if (rest >= p.row_blocks) rest -= p.row_blocks, ++at;
      if (!mp_wait(&s->item_free[slot], turn ^ 1u, s, status)) break;
      if (at >= total_tiles) {
        if (lane == 0) {
          s->item[slot].n = -1;
          mbar_arrive(smem_u32(&s->item_known[slot]));
          mbar_arrive(smem_u32(&s->item_full[slot]));
        }
        break;
      }
      int e, key = 0;
      if constexpr (PLACED) {  // the last expert whose first tile is not above the item's; two steps of 32 lanes
        e = 32 * (__popc(__ballot_sync(0xffffffffu, lane * 32 < p.E && s->tiles[lane * 32] <= at)) - 1);
        e += __popc(__ballot_sync(0xffffffffu, e + lane < p.E && s->tiles[e + lane] <= at)) - 1;
      } else {
        key = s->tile[at];
        e = key & 0xffff;
      }
      const slicemoe_mx4_mat m = p.E <= kMpTable ? s->mats[e] : p.mats[e];
      if (!m.codes || !m.scale || m.N != p.N || m.K != p.K || (m.gated != 0) != GATED) {
        if (lane == 0) atomicOr(status, (unsigned)SLICEMOE_STATUS_BAD_EXPERT_ID);
        continue;
      }
      // first what the weights and the products need, then where the results go
      MpItem* item = &s->item[slot];
      int rb = rest, list_at = 0, n = 0, n16 = p.tile;
      if constexpr (PLACED) {
        // of an expert's items a row block's tiles come one after the other: its weights are in L2 for all but the first
        const int first = s->first[e], count = s->first[e + 1] - first, e_tile = s->tiles[e];
        const MpTiles tt = count <= p.tile ? MpTiles{1, (count + 15) & ~15} : mp_tiles(count, p.tile);
        const int local = (at - e_tile) * p.row_blocks + rest;
        rb = tt.n == 1 ? local : local / tt.n;
        const int t = local - rb * tt.n, r0 = t * tt.each;
        n = min(tt.each, count - r0), n16 = (n + 15) & ~15, list_at = first + r0;
        if (lane == 0) {
          item->t_codes = p.t_codes + (size_t)(s->padded[e] + r0) * steps * kMpRowBytes;
          item->t_scale = p.t_scale + (size_t)(e_tile + t) * atoms * halves * kMxAtomBytes;
          item->rows = tt.each;
        }
      } else if (lane == 0) {
        item->rows = p.tile;
      }
      if (lane == 0) {
        item->n = n16;
        item->codes = m.codes + (size_t)rb * chunks * kMxChunkBytes;
        item->scale = m.scale + (size_t)rb * atoms * kMxAtomBytes;
        item->rb = rb;
        mbar_arrive(smem_u32(&s->item_known[slot]));
      }
      uint32_t groups = (1u << (n16 >> 4)) - 1u;
      if constexpr (PLACED) {
        for (int i = lane; i < n16; i += 32) s->pair[slot][i] = i < n ? __ldcg(p.list + list_at + i) : -1;
      } else {
        for (int i = lane; i < p.tile; i += 32) s->pair[slot][i] = -1;
        __syncwarp();
        groups = 0;
        for (int i = lane; i < pairs; i += 32)
          if (s->key[i] == key) {
            const int row = p.x_per_pair ? i : (int)__umulhi((uint32_t)i, p.k_inverse);
            s->pair[slot][row] = i;
            groups |= 1u << (row >> 4);
          }
        groups = __reduce_or_sync(0xffffffffu, groups);
      }
      if (lane == 0) item->groups = groups;
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&s->item_full[slot]));
      if (++slot == kMpSlots) slot = 0, turn ^= 1u;
    }
  } else if (warp == kMpWeightWarp || (PLACED && warp == kMpTileWarp)) {
    // ---- weights by one warp, placed tiles by another.  One thread, and the compiler knows it: addresses stay on the uniform datapath ----
    const bool tiles = PLACED && warp == kMpTileWarp;
    if (mp_elect()) {
      uint32_t* place = s->place[tiles ? 1 : 0];
      uint32_t slot = 0, turn = 0, st = 0, head = 0;
      uint32_t live = 0, old = 0, old_ph = 0;  // steps not known to be consumed, the oldest one's barrier
      uint32_t filled = 0;
      mx_dep_wait();  // first of all, like every role: the time that the kernel before still takes does not count against the waits' limit
      const bool bring = __ldcg(&p.head->extra_arrivals) == 0;
      if constexpr (PLACED) asm volatile("fence.proxy.async;" ::: "memory");  // the tiles were written by ordinary stores
      bool ok = true;
      while (ok && (ok = mbar_wait(smem_u32(&s->item_known[slot]), turn, &s->dead, status))) {
        const MpItem item = s->item[slot];
        if (item.n < 0) break;
        const uint32_t bytes = PLACED ? mp_step_bytes(item.rows, halves) : kMpABytes + kMpAScaleBytes, t_step = item.rows * kMpRowBytes;
        for (int i = 0; i < steps; ++i) {
          uint32_t at;
          for (;;) {
            at = head + bytes <= (uint32_t)p.ring ? head : 0;
            if (live == 0) break;
            // what is live lies in [tail, head), or in [tail, ...) and [0, head) where it has started again at 0
            const uint32_t tail = place[old];
            const bool room = head > tail ? at == head || bytes <= tail : at == head && head + bytes <= tail;
            if (room && live < (uint32_t)p.stages) break;
            if (!(ok = mbar_wait(smem_u32(&s->free_[old]), old_ph, &s->dead, status))) break;
            --live;
            if (++old == (uint32_t)p.stages) old = 0, old_ph ^= 1u;
          }
          if (!ok) break;
          head = at + bytes;
          place[st] = at;
          ++live;
          if (bring) {
            const int c = min(kMpStepChunks, chunks - i * kMpStepChunks), a = (c + 1) >> 1;
            const uint32_t dst = ring + at, bar = smem_u32(&s->full[st]);
            if (tiles) {
              const uint32_t t_dst = dst + kMpABytes + kMpAScaleBytes, s_bytes = a * halves * kMxAtomBytes;
              mbar_arrive_expect_tx(bar, t_step + s_bytes);
              mp_bulk(t_dst, item.t_codes + (size_t)i * t_step, t_step, bar);
              mp_bulk(t_dst + t_step, item.t_scale + (size_t)i * halves * kMpAScaleBytes, s_bytes, bar);
            } else {
              mbar_arrive_expect_tx(bar, c * kMxChunkBytes + a * kMxAtomBytes);
              mp_bulk(dst, item.codes + (size_t)i * kMpABytes, c * kMxChunkBytes, bar);
              mp_bulk(dst + kMpABytes, item.scale + (size_t)i * kMpAScaleBytes, a * kMxAtomBytes, bar);
            }
            ++filled;
          }
          if (++st == (uint32_t)p.stages) st = 0;
        }
        if (!ok) break;
        mbar_arrive(smem_u32(&s->item_free[slot]));
        if (++slot == kMpSlots) slot = 0, turn ^= 1u;
      }
      // what is on its way lands before the CTA ends, also where another role has given up
      for (uint32_t i = 1; i <= min(filled, (uint32_t)p.stages); ++i) {
        const uint32_t f = filled - i, b = f % p.stages, par = (f / p.stages) & 1u;
        const long long t0 = clock64();
        while (!mbar_try(smem_u32(&s->full[b]), par) && clock64() - t0 < 4000000ll) {
        }
      }
    }
    __syncwarp();
  } else if (warp == kMpMmaWarp) {
    // ---- products.  One thread too.  (With descriptors made in ordinary registers a step's twelve instructions took it 700 clocks, more
    // than the weights take to arrive; 285 with warp-wide waits.) ----
    if (mp_elect()) {
      uint32_t slot = 0, turn = 0, st = 0, ph = 0, acc = 0, acc_ph = 0, flip = 0, head = 0;
      mx_dep_wait();
      bool ok = PLACED || mbar_wait(smem_u32(&s->resident), 0, &s->dead, status);
      while (ok && (ok = mbar_wait(smem_u32(&s->item_known[slot]), turn, &s->dead, status))) {
        const int n = s->item[slot].n, rows = s->item[slot].rows;
        if (n < 0) break;
        const uint32_t idesc = mp_idesc(n), d = tmem + acc * kMpTile;
        const bool wide = n > 128;
        const uint32_t b_bytes = rows * kMpRowBytes, bytes = PLACED ? mp_step_bytes(rows, halves) : kMpABytes + kMpAScaleBytes;
        if (!(ok = mbar_wait(smem_u32(&s->acc_free[acc]), acc_ph ^ 1u, &s->dead, status))) break;
        mp_fence_after();
        for (int i = 0; i < steps; ++i) {
          if (!(ok = mbar_wait(smem_u32(&s->full[st]), ph, &s->dead, status))) break;
          mp_fence_after();
          const int c = chunks - i * kMpStepChunks;  // chunks of the step, if below four
          const uint32_t at = ring + mp_next_place(head, bytes, p.ring), b_at = PLACED ? at + kMpABytes + kMpAScaleBytes : rows_at + i * b_bytes;
          const uint32_t la = (at >> 4) + ((kMxRows * 16 >> 4) << 16), lb = (b_at >> 4) + (1u << 16);
          const uint32_t s_at = PLACED ? b_at + b_bytes : rows_at + steps * b_bytes + i * halves * kMpAScaleBytes;
          const uint32_t lsa = (at + kMpABytes) >> 4, lsb = s_at >> 4, next = halves * (kMxAtomBytes >> 4);
          const uint32_t sa = tmem + kMpScaleCol + flip * kMpScaleCols, sb = sa + 8;
          mp_copy_scales(sa, mp_desc(lsa));
          mp_copy_scales(sb, mp_desc(lsb));
          if (wide) mp_copy_scales(sb + 4, mp_desc(lsb + (kMxAtomBytes >> 4)));
          if (c > 2) {
            mp_copy_scales(sa + 4, mp_desc(lsa + (kMxAtomBytes >> 4)));
            mp_copy_scales(sb + 8, mp_desc(lsb + next));
            if (wide) mp_copy_scales(sb + 12, mp_desc(lsb + next + (kMxAtomBytes >> 4)));
          }
#pragma unroll
          for (int j = 0; j < kMpStepChunks; ++j)
            if (j < c) {
              constexpr uint32_t kHigh = 2u << 29 | 2u << 4;  // the upper two of the four scale bytes
              mp_mma(d, mp_desc(la + j * (kMxChunkBytes >> 4)), mp_desc_rows(lb + j * (kMxChunk / 2 >> 4)), j & 1 ? idesc | kHigh : idesc, sa + 4 * (j >> 1),
                     sb + 8 * (j >> 1), (uint32_t)(i | j));
            }
          mp_commit(smem_u32(&s->free_[st]));
          flip ^= 1u;
          if (++st == (uint32_t)p.stages) st = 0, ph ^= 1u;
        }
        if (!ok) break;
        mp_commit(smem_u32(&s->acc_full[acc]));
        mbar_arrive(smem_u32(&s->item_free[slot]));
        if (++slot == kMpSlots) slot = 0, turn ^= 1u;
        if (acc ^= 1u; acc == 0) acc_ph ^= 1u;
      }
      // every instruction issued is done before tensor memory is given back
      mp_commit(smem_u32(&s->drain));
      const long long t0 = clock64();
      while (!mbar_try(smem_u32(&s->drain), 0) && clock64() - t0 < 4000000ll) {
      }
    }
    __syncwarp();
  } else {
    if constexpr (!PLACED) {
      // ---- all rows of the call into the operand layout, 512 bytes of a row at a time ----
      mx_dep_wait();
      const int rows = p.x_per_pair ? pairs : p.T, kbytes = p.K >> 1, pieces = 2 * chunks, scales = rows_at + steps * p.tile * kMpRowBytes;
      const int runs = (pieces + 31) >> 5;
      for (int i = warp - 3; i < rows * runs; i += kMpDrainWarps + 1) {
        const int r = i / runs, q = (i - r * runs) * 32 + lane;
        if (q < pieces) {  // beyond the row's end zeros; all of a lane's copies are under way at once
          const uint8_t* src = p.codes + (size_t)r * kbytes;
          const bool in = q * 16 < kbytes;
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(rows_at + mp_piece(p.tile, r, q)), "l"(in ? src + q * 16 : src),
                       "r"(in ? 16u : 0u)
                       : "memory");
        }
      }
      constexpr int kStride = 32 * (kMpDrainWarps + 1), kAhead = 4;
      for (int i0 = (warp - 3) * 32 + lane; i0 < rows * atoms; i0 += kAhead * kStride) {
        uint32_t w[kAhead];
#pragma unroll
        for (int a = 0; a < kAhead; ++a)
          if (i0 + a * kStride < rows * atoms) w[a] = __ldcg(reinterpret_cast<const uint32_t*>(p.scale) + i0 + a * kStride);
#pragma unroll
        for (int a = 0; a < kAhead; ++a) {
          const int i = i0 + a * kStride;
          if (i >= rows * atoms) break;
          const int r = i / atoms, j = i - r * atoms, left = (p.K >> 5) - 4 * j;
          const uint32_t v = left < 4 ? w[a] & ((1u << (8 * left)) - 1u) : w[a];  // bytes beyond the row's end
          asm volatile("st.shared.b32 [%0], %1;" ::"r"(scales + (j * halves + (r >> 7)) * kMxAtomBytes + (r & 31) * 16 + ((r >> 5) & 3) * 4), "r"(v) : "memory");
        }
      }
      asm volatile("cp.async.wait_all;" ::: "memory");
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&s->resident));
    }
    if (warp >= kMpFirstDrain) {
    // ---- results: a warp reads 32 weight rows, 16 tokens at a time, every other sixteen that is in use ----
    const int quarter = warp & 3, half = (warp - kMpFirstDrain) >> 2;
    uint32_t slot = 0, turn = 0, acc = 0, acc_ph = 0;
    bool ok = true;
    O* out = static_cast<O*>(p.out);
    mx_dep_wait();
    while (ok && (ok = mp_wait(&s->item_full[slot], turn, s, status))) {
      const int rb = s->item[slot].rb;
      uint32_t groups = s->item[slot].groups;
      if (s->item[slot].n < 0) break;
      if (!(ok = mp_wait(&s->acc_full[acc], acc_ph, s, status))) break;
      mp_fence_after();
      const uint32_t d = tmem + ((uint32_t)(quarter * 32) << 16) + acc * kMpTile;
      if (half) groups &= groups - 1u;
      while (groups) {
        const int c0 = 16 * (__ffs(groups) - 1);
        groups &= groups - 1u;
        groups &= groups - 1u;
        uint32_t r[16];
        mp_ld16(d + c0, r);
        const int* pairs = &s->pair[slot][c0];
        // Results of 16 bits leave as pairs of columns: two tokens' values in a word, half of the words exchanged with the neighbouring
        // lane, and each lane has both columns of half of the tokens.  Exchanges and stores go the way that the products' operands
        // take out of shared memory, and are what a long prompt's drain waits for: with an exchange for every word it took 5,700
        // clocks an item of 224 tokens, more than the products.
        const bool odd = lane & 1;
        if constexpr (GATED) {
          // lanes 0 to 15 hold gate, 16 to 31 up of the same columns of the result: of two tokens, the lower lanes take the first
          const bool hi = lane & 16;
          const int col = rb * 64 + quarter * 16 + (lane & 15);
          float h[8];  // of tokens 2 i + hi
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float v0 = __uint_as_float(r[2 * i]), v1 = __uint_as_float(r[2 * i + 1]);
            const float got = __shfl_xor_sync(0xffffffffu, hi ? v0 : v1, 16);
            h[i] = mp_gated(hi ? got : v0, hi ? v1 : got);
          }
          if (sizeof(O) == 2 && (p.N & 1) == 0) {
            uint32_t w[4], got[2];
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = mp_pack2<O>(h[2 * i], h[2 * i + 1]);
#pragma unroll
            for (int i = 0; i < 2; ++i) got[i] = __shfl_xor_sync(0xffffffffu, odd ? w[i] : w[2 + i], 1);
            const int4 a = *reinterpret_cast<const int4*>(pairs + (odd ? 8 : 0)), b = *reinterpret_cast<const int4*>(pairs + (odd ? 12 : 4));
            const int pr[4] = {hi ? a.y : a.x, hi ? a.w : a.z, hi ? b.y : b.x, hi ? b.w : b.z};
            if (col < p.N) {
              O* at = out + (col & ~1);
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const uint32_t mine = odd ? w[2 + (i >> 1)] : w[i >> 1], first = odd ? got[i >> 1] : mine, second = odd ? mine : got[i >> 1];
                if (pr[i] >= 0) *reinterpret_cast<uint32_t*>(at + (size_t)pr[i] * p.N) = __byte_perm(first, second, i & 1 ? 0x7632 : 0x5410);
              }
            }
          } else if (col < p.N) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
              if (const int pair = pairs[2 * i + (hi ? 1 : 0)]; pair >= 0) out[(size_t)pair * p.N + col] = mx_from_float<O>(h[i]);
          }
        } else {
          const int col = rb * kMxRows + quarter * 32 + lane;
          if (sizeof(O) == 2 && (p.N & 1) == 0) {
            uint32_t w[8], got[4];
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = mp_pack2<O>(__uint_as_float(r[2 * i]), __uint_as_float(r[2 * i + 1]));
#pragma unroll
            for (int i = 0; i < 4; ++i) got[i] = __shfl_xor_sync(0xffffffffu, odd ? w[i] : w[4 + i], 1);
            const int4 a = *reinterpret_cast<const int4*>(pairs + (odd ? 8 : 0)), b = *reinterpret_cast<const int4*>(pairs + (odd ? 12 : 4));
            const int pr[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
            if (col < p.N) {
              O* at = out + (col & ~1);
#pragma unroll
              for (int i = 0; i < 8; ++i) {
                const uint32_t mine = odd ? w[4 + (i >> 1)] : w[i >> 1], first = odd ? got[i >> 1] : mine, second = odd ? mine : got[i >> 1];
                if (pr[i] >= 0) *reinterpret_cast<uint32_t*>(at + (size_t)pr[i] * p.N) = __byte_perm(first, second, i & 1 ? 0x7632 : 0x5410);
              }
            }
          } else if (col < p.N) {
#pragma unroll
            for (int i = 0; i < 16; ++i)
              if (const int pair = pairs[i]; pair >= 0) out[(size_t)pair * p.N + col] = mx_from_float<O>(__uint_as_float(r[i]));
          }
        }
      }
      mp_fence_before();
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(smem_u32(&s->acc_free[acc]));
        mbar_arrive(smem_u32(&s->item_free[slot]));
      }
      if (++slot == kMpSlots) slot = 0, turn ^= 1u;
      if (acc ^= 1u; acc == 0) acc_ph ^= 1u;
    }
    }
  }
  mp_fence_before();
  __syncthreads();
  mp_fence_after();
  if (warp == kMpMmaWarp) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kMpTmemCols) : "memory");
}

// SMs of the current device.
static int mp_sm_count(int* sms) {
  static int count[64];
  int dev = 0;
  SM_CUDA_TRY(cudaGetDevice(&dev));
  if (dev < 0 || dev >= 64) return SLICEMOE_E_UNSUPPORTED;
  if (!count[dev]) SM_CUDA_TRY(cudaDeviceGetAttribute(&count[dev], cudaDevAttrMultiProcessorCount, dev));
  *sms = count[dev];
  return SLICEMOE_OK;
}
template <class O, bool GATED, bool PLACED>
static int mp_launch(const MpParams& p, int ctas, cudaStream_t st) {
  static bool attr_set[64];
  int dev = 0;
  SM_CUDA_TRY(cudaGetDevice(&dev));
  if (!attr_set[dev]) {  // mp_sm_count() has looked at the device's number
    SM_CUDA_TRY(cudaFuncSetAttribute(mp_product_kernel<O, GATED, PLACED>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMpSmem));
    attr_set[dev] = true;
  }
  return mx_launch(mp_product_kernel<O, GATED, PLACED>, dim3(ctas), kMpThreads, (size_t)kMpSmem, st, MpParams(p));
}
template <class O>
static int mp_launch_as(const MpParams& p, int ctas, cudaStream_t st) {
  if (p.t_codes) return p.gated ? mp_launch<O, true, true>(p, ctas, st) : mp_launch<O, false, true>(p, ctas, st);
  return p.gated ? mp_launch<O, true, false>(p, ctas, st) : mp_launch<O, false, false>(p, ctas, st);
}

}  // namespace slicemoe

using namespace slicemoe;

extern "C" size_t slicemoe_mx4_workspace_bytes(int T, int k, int n_experts, int K) {
  if (T <= 0 || k < 1 || k > SLICEMOE_MAX_TOP_K || n_experts <= 0 || n_experts > kMpMaxExperts || (int64_t)T * k > kMpMaxPairs) return 0;
  if (K <= 0 || K % kMxBlock || K > kMxMaxK) return 0;
  return mp_layout(T, k, n_experts, K).total;
}

extern "C" int slicemoe_mx4_workspace_init(void* workspace, size_t workspace_bytes, void* stream) {
  if (!workspace || workspace_bytes < 256 || !mx_aligned(workspace, 256)) return SLICEMOE_E_INVALID_ARG;
  SM_CUDA_TRY(cudaMemsetAsync(workspace, 0, 256, (cudaStream_t)stream));
  return SLICEMOE_OK;
}

extern "C" int slicemoe_mx4_product(const slicemoe_mx4_mat* mats, int n_experts, int N, int K, int gated, const uint8_t* codes,
                                    const uint8_t* scale, int T, int k, int x_per_pair, const int32_t* ids, void* out, int dtype, void* workspace,
                                    size_t workspace_bytes, void* stream) {
  if (!mats || !codes || !scale || !out || !workspace) return SLICEMOE_E_INVALID_ARG;
  if (n_experts <= 0 || N <= 0 || K <= 0 || K % kMxBlock || T <= 0 || k < 1 || (!ids && k != 1)) return SLICEMOE_E_INVALID_ARG;
  if (n_experts > kMpMaxExperts || N > kMxMaxN || K > kMxMaxK || k > SLICEMOE_MAX_TOP_K || (int64_t)T * k > kMpMaxPairs || !mx_dtype(dtype))
    return SLICEMOE_E_UNSUPPORTED;
  const int pairs = T * k, E = ids ? n_experts : 1;
  const MpLayout l = mp_layout(T, k, E, K);
  if (!mx_aligned(mats, 8) || !mx_aligned(codes, 16) || !mx_aligned(scale, 4) || !mx_aligned(out, 16) || !mx_aligned(ids, 4) ||
      !mx_aligned(workspace, 256) || workspace_bytes < l.total)
    return SLICEMOE_E_INVALID_ARG;
  cudaStream_t st = (cudaStream_t)stream;
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  MpParams p = {};
  p.mats = mats;
  p.codes = codes;
  p.scale = scale;
  p.ids = ids;
  p.out = out;
  p.head = reinterpret_cast<MpHeader*>(ws);
  p.E = E;
  p.N = N;
  p.K = K;
  p.gated = gated;
  p.T = T;
  p.k = k;
  p.x_per_pair = x_per_pair || k == 1;
  p.k_inverse = k > 1 ? (uint32_t)((0x100000000ull + k - 1) / k) : 0;
  // Resident where all rows fit: no launches ahead, and nothing to gather.
  const int rows = p.x_per_pair ? pairs : T, rows16 = (rows + 15) & ~15;
  const int64_t held = (int64_t)rows16 * mp_steps(K) * kMpRowBytes + (int64_t)mx_atoms(K) * ((rows16 + 127) / 128) * kMxAtomBytes;
  const bool placed = pairs > kMpFew || rows16 > kMpTile || held > kMpResident;
  int sms = 0;
  const int rc_sms = mp_sm_count(&sms);
  if (rc_sms != SLICEMOE_OK) return rc_sms;
  p.row_blocks = mx_row_blocks(N, gated);
  p.tile = placed ? mp_tile(T, pairs, E, p.row_blocks, sms) : rows16;
  p.resident = placed ? 0 : (int)((held + 1023) & ~1023);
  p.ring = kMpSmem - kMpFixed - p.resident;
  p.stages = kMpMaxStages;
  if (!placed && p.stages > p.ring / (kMpABytes + kMpAScaleBytes)) p.stages = p.ring / (kMpABytes + kMpAScaleBytes);
  const int64_t tiles = placed ? (int64_t)pairs / p.tile + (pairs < E ? pairs : E) : pairs, items = tiles * p.row_blocks;
  if (items > INT32_MAX) return SLICEMOE_E_UNSUPPORTED;
  if (placed) {
    int *rank = reinterpret_cast<int*>(ws + l.rank), *hist = reinterpret_cast<int*>(ws + l.hist), *first = reinterpret_cast<int*>(ws + l.first),
        *list = reinterpret_cast<int*>(ws + l.list);
    const bool few = ids && pairs <= kMpPlaceAll;
    if (ids && !few) {
      const int rc = mx_launch(mp_sort_kernel, dim3(l.blocks), kMpSortThreads, 0, st, MpSortParams{ids, pairs, E, rank, hist, p.head});
      if (rc != SLICEMOE_OK) return rc;
    }
    int chunk = 32;  // pairs of a block: more where there are blocks enough to fill the device
    while (!few && chunk < kMpSortPairs && pairs / chunk > 148 * 6) chunk *= 2;
    const MpPlaceParams pp = {ids, rank, hist, codes, scale, first, list, ws + l.codes, ws + l.scale, pairs, E, l.blocks, chunk, p.tile, k, p.x_per_pair, K, p.head};
    const int rc = mx_launch(few ? mp_place_kernel<true> : mp_place_kernel<false>, dim3((pairs + chunk - 1) / chunk),
                             (unsigned)(few ? 2 * kMpPlaceThreads : kMpPlaceThreads), 0, st, MpPlaceParams(pp));
    if (rc != SLICEMOE_OK) return rc;
    p.first = first;
    p.list = list;
    p.t_codes = ws + l.codes;
    p.t_scale = ws + l.scale;
  }
  const int ctas = items < sms ? (int)items : sms;
  if (dtype == SLICEMOE_F32) return mp_launch_as<float>(p, ctas, st);
  if (dtype == SLICEMOE_BF16) return mp_launch_as<__nv_bfloat16>(p, ctas, st);
  return mp_launch_as<__half>(p, ctas, st);
}
