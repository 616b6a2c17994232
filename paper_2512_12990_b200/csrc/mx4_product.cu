// slicemoe_mx4_product: rows of microscaled 4-bit activations times the matrices of the experts that a routing list names.
//
// The product is computed transposed, D[weight row, token] (128 weight rows x up to 224 tokens): the weights' rows are the fixed
// side of the tensor instruction, so that a tile with one token costs what it reads and no more.  An item is a block of 128
// weight rows times a tile of one expert's tokens; one persistent CTA per SM takes every grid'th item.  Steps of 256 values of K go through a
// ring in shared memory: weights and their scales by bulk copies (the packed layout is the operand layout), token rows gathered by
// cp.async, scales on to tensor memory by tcgen05.cp, four tcgen05.mma (kind mxf4, a scale per 32 values) a step.  Two
// accumulators in tensor memory: one is drained while the other fills.
//
// Sums are fp32 in tensor memory and rounded once.  Which column of a tile a token has does not enter its sum, so a row's
// result does not depend on the rest of the call.
#include "decode_common.cuh"
#include "mx4.cuh"

namespace slicemoe {

// The head of a workspace: as far as slicemoe_get_status and slicemoe_workspace_set_wait go it is that of the layer calls.
struct MpHeader {
  unsigned unused0, unused1;
  unsigned status;
  unsigned extra_arrivals;  // != 0: the weights are never brought, and the waits for them run out
  unsigned long long wait_cycles;
};
constexpr int kMpMaxExperts = 1024;
constexpr int64_t kMpMaxPairs = 1 << 24;
constexpr int kMpInline = 512;       // up to here every CTA sorts the pairs itself; above, a kernel before does
constexpr int kMpSortPairs = 4096;   // pairs of a block of that kernel
constexpr int kMpSortThreads = 1024;

// Workspace: header, rows before each expert, the pairs by expert; and the same of each block where there is more than one.
struct MpLayout {
  size_t first, list, block_first, block_list, total;
  int blocks;
};
__host__ __device__ inline MpLayout mp_layout(int64_t pairs, int E) {
  auto up = [](size_t v) { return (v + 255) & ~(size_t)255; };
  MpLayout l;
  l.blocks = (int)((pairs + kMpSortPairs - 1) / kMpSortPairs);
  const bool many = l.blocks > 1;
  l.first = 256;
  l.list = l.first + up((E + 1) * sizeof(int));
  l.block_first = l.list + up(pairs * sizeof(int));
  l.block_list = l.block_first + (many ? up((size_t)l.blocks * (E + 1) * sizeof(int)) : 0);
  l.total = l.block_list + (many ? up(pairs * sizeof(int)) : 0);
  return l;
}

// ---- pairs by expert ----------------------------------------------------------------------------------------------
// Exclusive scan over the block of one value per thread; *total gets the sum.  s: one int per warp.
template <int THREADS>
__device__ __forceinline__ int mp_scan(int v, int* s, int* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int inc = v;
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    const int a = __shfl_up_sync(0xffffffffu, inc, off);
    if (lane >= off) inc += a;
  }
  __syncthreads();
  if (lane == 31) s[warp] = inc;
  __syncthreads();
  const int w = lane < THREADS / 32 ? s[lane] : 0;
  *total = __reduce_add_sync(0xffffffffu, w);
  return __reduce_add_sync(0xffffffffu, lane < warp ? w : 0) + inc - v;
}

struct MpSortParams {
  const int32_t* ids;
  int pairs, E;
  int* first;  // [block][E + 1]
  int* list;   // [block][kMpSortPairs]
  MpHeader* head;
};
// A block's pairs by expert: a pair's rank among the block's of its expert is what the counting atomic returns.  (The order within an
// expert depends on the atomics' order; which column of a tile a pair gets does not enter its result.)
__global__ void __launch_bounds__(kMpSortThreads) mp_sort_kernel(const MpSortParams p) {
  __shared__ int s_first[kMpMaxExperts + 1], s_sums[32];
  mx_dep_launch();
  const int tid = threadIdx.x;
  s_first[tid] = 0;
  if (tid == 0) s_first[kMpMaxExperts] = 0;
  mx_dep_wait();
  __syncthreads();
  const int base = blockIdx.x * kMpSortPairs;
  constexpr int kEach = kMpSortPairs / kMpSortThreads;
  int e[kEach], rank[kEach];
  bool bad = false;
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int at = base + i * kMpSortThreads + tid;
    e[i] = at < p.pairs ? __ldcg(p.ids + at) : -1;
    bad |= at < p.pairs && (unsigned)e[i] >= (unsigned)p.E;
  }
#pragma unroll
  for (int i = 0; i < kEach; ++i) rank[i] = (unsigned)e[i] < (unsigned)p.E ? atomicAdd(&s_first[e[i]], 1) : 0;
  __syncthreads();
  int total;
  const int before = mp_scan<kMpSortThreads>(s_first[tid], s_sums, &total);
  s_first[tid] = before;
  if (tid == 0) s_first[kMpMaxExperts] = total;
  __syncthreads();
  for (int i = tid; i <= p.E; i += kMpSortThreads) p.first[(size_t)blockIdx.x * (p.E + 1) + i] = s_first[i];
#pragma unroll
  for (int i = 0; i < kEach; ++i)
    if ((unsigned)e[i] < (unsigned)p.E) p.list[base + s_first[e[i]] + rank[i]] = base + i * kMpSortThreads + tid;
  if (bad) atomicOr(&p.head->status, (unsigned)SLICEMOE_STATUS_BAD_EXPERT_ID);
}

struct MpMergeParams {
  const int *block_first, *block_list;
  int blocks, E;
  int *first, *list;
};
// The blocks' lists one behind the other: block b moves its own, an expert's pairs behind those of the blocks before.
__global__ void __launch_bounds__(kMpSortThreads) mp_merge_kernel(const MpMergeParams p) {
  __shared__ int s_at[kMpMaxExperts], s_sums[32];
  mx_dep_launch();
  mx_dep_wait();
  const int tid = threadIdx.x, me = blockIdx.x;
  int count = 0, before = 0, mine = 0;
  if (tid < p.E)
    for (int b = 0; b < p.blocks; ++b) {
      const int* f = p.block_first + (size_t)b * (p.E + 1) + tid;
      const int lo = __ldcg(f), n = __ldcg(f + 1) - lo;
      if (b < me) before += n;
      if (b == me) mine = lo;
      count += n;
    }
  int total;
  const int first = mp_scan<kMpSortThreads>(count, s_sums, &total);
  if (me == 0 && tid <= p.E) p.first[tid] = first;
  if (me == 0 && p.E == kMpSortThreads && tid == 0) p.first[p.E] = total;
  s_at[tid] = first + before - mine;  // what to add to a place in the block's list
  __syncthreads();
  const int* src = p.block_list + (size_t)me * kMpSortPairs;
  const int n = __ldcg(p.block_first + (size_t)me * (p.E + 1) + p.E);
  for (int i = tid; i < n; i += kMpSortThreads) {
    int lo = 0, hi = p.E - 1;  // the last expert whose first place is not above i
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (__ldcg(p.block_first + (size_t)me * (p.E + 1) + mid) <= i) lo = mid; else hi = mid - 1;
    }
    p.list[s_at[lo] + i] = __ldcg(src + i);
  }
}

// ---- the product ----------------------------------------------------------------------------------------------------
constexpr int kMpTile = 224;                 // most tokens of a tile
constexpr int kMpStepChunks = 4;             // chunks of 64 values a step
constexpr int kMpGatherWarps = 6, kMpDrainWarps = 8;
constexpr int kMpWeightWarp = 0, kMpMmaWarp = 1, kMpFirstGather = 2, kMpFirstDrain = 8;
constexpr int kMpThreads = 32 * (kMpFirstDrain + kMpDrainWarps);
constexpr int kMpPlanWarp = kMpFirstDrain + kMpDrainWarps;  // one more warp
constexpr int kMpAllThreads = kMpThreads + 32;
constexpr int kMpSlots = 4, kMpMaxStages = 8;
constexpr int kMpTmemCols = 512;
constexpr int kMpScaleCol = 2 * kMpTile;     // behind the two accumulators: scales of two steps, 8 + 16 columns each
constexpr int kMpScaleCols = 24;
static_assert(kMpScaleCol + 2 * kMpScaleCols <= kMpTmemCols, "tensor memory");
constexpr int kMpABytes = kMpStepChunks * kMxChunkBytes, kMpAScaleBytes = kMpStepChunks / 2 * kMxAtomBytes;

struct MpItem {
  const uint8_t *codes, *scale;
  int n;         // tokens; < 0: no more items
  int rb;        // row block
  int pad_[2];
};
struct __align__(16) MpSmem {
  unsigned long long full_a[kMpMaxStages], full_b[kMpMaxStages], free_[kMpMaxStages];
  unsigned long long acc_full[2], acc_free[2], item_full[kMpSlots], item_free[kMpSlots], drain;
  uint32_t tmem;
  int pad0;
  int dead, pad1;
  unsigned long long limit;  // 8 bytes behind dead
  MpItem item[kMpSlots];
  int pair[kMpSlots][kMpTile], row[kMpSlots][kMpTile];
  int first[kMpMaxExperts + 1];  // rows before an expert
  int items[kMpMaxExperts + 1];  // items before it
  int list[kMpInline];
  int sums[32];
};
static_assert(offsetof(MpSmem, limit) == offsetof(MpSmem, dead) + 8, "wait_limit()");
constexpr int kMpFixed = (int)((sizeof(MpSmem) + 127) / 128 * 128);
constexpr int kMpSmemMax = 227 * 1024, kMpSmemMin = 116 * 1024;  // one CTA to an SM: each takes all of tensor memory

struct MpParams {
  const slicemoe_mx4_mat* mats;
  const uint8_t* codes;
  const uint8_t* scale;
  const int32_t* ids;
  void* out;
  MpHeader* head;
  const int *first, *list;
  int E, N, K, gated, T, k, x_per_pair;
  int tile, stages;      // most tokens of a tile here, a multiple of 16; steps of the ring
  int row_blocks;
};

__device__ __forceinline__ uint64_t mp_desc(uint32_t addr, uint32_t lead, uint32_t stride) {  // no swizzle
  return (uint64_t)((addr & 0x3FFFF) >> 4) | (uint64_t)(lead >> 4) << 16 | (uint64_t)(stride >> 4) << 32 | (uint64_t)1 << 46;
}
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
__device__ __forceinline__ void mp_cp16(uint32_t dst, const void* src, uint32_t bytes) {  // bytes 0: zeros
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
// By a whole warp; every lane gets the same answer.
__device__ __forceinline__ bool mp_wait(const void* bar, uint32_t parity, MpSmem* s, unsigned* status) {
  return __all_sync(0xffffffffu, mbar_wait(smem_u32(bar), parity, &s->dead, status));
}
__device__ __forceinline__ float mp_silu(float v) { return v / (1.0f + expf(-v)); }

template <class O>
__device__ __forceinline__ uint32_t mp_pack2(float a, float b) {
  const O e[2] = {mx_from_float<O>(a), mx_from_float<O>(b)};
  uint32_t w;
  memcpy(&w, e, 4);
  return w;
}

template <class O, bool GATED>
__global__ void __launch_bounds__(kMpAllThreads, 1) mp_product_kernel(const MpParams p) {
  extern __shared__ __align__(128) uint8_t mp_smem[];
  MpSmem* s = reinterpret_cast<MpSmem*>(mp_smem);
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  const int chunks = mx_chunks(p.K), atoms = mx_atoms(p.K), steps = (chunks + kMpStepChunks - 1) / kMpStepChunks;
  const int halves = (p.tile + 127) >> 7;  // scale blocks of 128 tokens
  const uint32_t b_bytes = p.tile * (kMpStepChunks * kMxChunk / 2), stage_bytes = kMpABytes + kMpAScaleBytes + b_bytes + halves * kMpAScaleBytes;
  const uint32_t ring = smem_u32(mp_smem) + kMpFixed;
  unsigned* status = &p.head->status;

  mx_dep_launch();
  if (tid == 0) {
    for (int i = 0; i < kMpMaxStages; ++i) {
      mbar_init(smem_u32(&s->full_a[i]), 1);
      mbar_init(smem_u32(&s->full_b[i]), 1);
      mbar_init(smem_u32(&s->free_[i]), 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(smem_u32(&s->acc_full[i]), 1);
      mbar_init(smem_u32(&s->acc_free[i]), kMpDrainWarps);
    }
    for (int i = 0; i < kMpSlots; ++i) {
      mbar_init(smem_u32(&s->item_full[i]), 1);
      mbar_init(smem_u32(&s->item_free[i]), 2 + kMpGatherWarps + kMpDrainWarps);
    }
    mbar_init(smem_u32(&s->drain), 1);
    s->dead = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kMpMmaWarp) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&s->tmem)), "r"(kMpTmemCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  // the table does not change between launches: it is read while the kernel before is still at work
  bool fits[(kMpMaxExperts + kMpAllThreads - 1) / kMpAllThreads];
  constexpr int kEach = sizeof(fits) / sizeof(fits[0]);
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int e = i * kMpAllThreads + tid;
    fits[i] = false;
    if (e < p.E) {
      const slicemoe_mx4_mat m = p.mats[e];
      fits[i] = m.codes && m.scale && m.N == p.N && m.K == p.K && (m.gated != 0) == GATED;
      s->first[e] = 0;
    }
  }
  mx_dep_wait();
  if (tid == 0) s->limit = p.head->wait_cycles ? p.head->wait_cycles : kWaitCycles;
  const bool own_list = p.ids && !p.list;
  int total_rows = p.T;
  if (own_list) {  // few pairs: by expert, here
    const int pairs = p.T * p.k;
    __syncthreads();
    const int e = tid < pairs ? __ldcg(p.ids + tid) : -1;
    const bool named = (unsigned)e < (unsigned)p.E;
    // in the order of the list, warp after warp: all CTAs must deal the same pairs to the same tiles
    int rank = 0;
    const unsigned same = __match_any_sync(0xffffffffu, e), lower = same & ((1u << lane) - 1u);
    for (int w = 0; w * 32 < pairs; ++w) {
      if (warp == w && named) rank = s->first[e] + __popc(lower);
      __syncwarp();
      if (warp == w && named && lower == 0) s->first[e] += __popc(same);
      __syncthreads();
    }
    if (tid < pairs && !named && blockIdx.x == 0) atomicOr(status, (unsigned)SLICEMOE_STATUS_BAD_EXPERT_ID);
    int count[kEach], before[kEach], base = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int x = i * kMpAllThreads + tid;
      count[i] = x < p.E ? s->first[x] : 0;
      before[i] = 0;
      if (i * kMpAllThreads < p.E) {
        int total;
        before[i] = base + mp_scan<kMpAllThreads>(count[i], s->sums, &total);
        base += total;
      }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int x = i * kMpAllThreads + tid;
      if (x < p.E) s->first[x] = before[i];
    }
    total_rows = base;
    __syncthreads();
    if (named) s->list[s->first[e] + rank] = tid;
  } else if (p.list) {
    for (int i = tid; i < p.E; i += kMpAllThreads) s->first[i] = __ldcg(p.first + i);
    total_rows = __ldcg(p.first + p.E);
  } else {
    for (int i = tid; i < p.E; i += kMpAllThreads) s->first[i] = i ? p.T : 0;
  }
  if (tid == 0) s->first[p.E] = total_rows;
  __syncthreads();
  int total_items = 0;
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int e = i * kMpAllThreads + tid;
    if (i * kMpAllThreads >= p.E) break;
    int n = e < p.E ? s->first[e + 1] - s->first[e] : 0;
    if (n > 0 && !fits[i]) {
      n = 0;
      if (blockIdx.x == 0) atomicOr(status, (unsigned)SLICEMOE_STATUS_BAD_EXPERT_ID);
    }
    int total;
    const int before = mp_scan<kMpAllThreads>((n + p.tile - 1) / p.tile * p.row_blocks, s->sums, &total);
    if (e < p.E) s->items[e] = total_items + before;
    total_items += total;
  }
  if (tid == 0) s->items[p.E] = total_items;
  mp_fence_before();
  __syncthreads();
  mp_fence_after();
  const uint32_t tmem = s->tmem;

  if (warp == kMpPlanWarp) {
    // ---- which item is next, and its rows ----
    uint32_t slot = 0, turn = 0;
    bool ok = true;
    for (int it = blockIdx.x;; it += gridDim.x) {
      ok = mp_wait(&s->item_free[slot], turn ^ 1u, s, status);
      if (!ok) break;
      if (it >= total_items) {
        if (lane == 0) s->item[slot].n = -1;
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&s->item_full[slot]));
        break;
      }
      int lo = 0;  // the last expert whose first item is not above `it`; two steps of 32 lanes
      const int cut = lane * 32;
      lo = 32 * (__popc(__ballot_sync(0xffffffffu, cut < p.E && s->items[cut] <= it)) - 1);
      lo += __popc(__ballot_sync(0xffffffffu, lo + lane < p.E && s->items[lo + lane] <= it)) - 1;
      const slicemoe_mx4_mat* m = p.mats + lo;
      const uint8_t *codes = m->codes, *scale = m->scale;
      const int first = s->first[lo], count = s->first[lo + 1] - first, local = it - s->items[lo];
      const int tiles = (count + p.tile - 1) / p.tile, rb = local / tiles, t = local - rb * tiles;
      const int each = ((count + tiles - 1) / tiles + 15) & ~15, r0 = t * each, n = min(each, count - r0);
      for (int i = lane; i < n; i += 32) {
        const int at = first + r0 + i;
        const int pair = own_list ? s->list[at] : p.list ? __ldcg(p.list + at) : at;
        s->pair[slot][i] = pair;
        s->row[slot][i] = p.x_per_pair ? pair : pair / p.k;
      }
      if (lane == 0) {
        s->item[slot].codes = codes + (size_t)rb * chunks * kMxChunkBytes;
        s->item[slot].scale = scale + (size_t)rb * atoms * kMxAtomBytes;
        s->item[slot].n = n;
        s->item[slot].rb = rb;
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&s->item_full[slot]));
      if (++slot == kMpSlots) slot = 0, turn ^= 1u;
    }
  } else if (warp == kMpWeightWarp) {
    // ---- weights ----
    uint32_t slot = 0, turn = 0, st = 0, ph = 0, filled = 0;
    const bool bring = p.head->extra_arrivals == 0;
    bool ok = true;
    while (ok && (ok = mp_wait(&s->item_full[slot], turn, s, status))) {
      const MpItem item = s->item[slot];
      if (item.n < 0) break;
      for (int i = 0; i < steps; ++i) {
        if (!(ok = mp_wait(&s->free_[st], ph ^ 1u, s, status))) break;
        const int c = min(kMpStepChunks, chunks - i * kMpStepChunks), a = (c + 1) >> 1;
        if (bring && mp_elect()) {
          const uint32_t dst = ring + st * stage_bytes, bar = smem_u32(&s->full_a[st]);
          mbar_arrive_expect_tx(bar, c * kMxChunkBytes + a * kMxAtomBytes);
          mp_bulk(dst, item.codes + (size_t)i * kMpABytes, c * kMxChunkBytes, bar);
          mp_bulk(dst + kMpABytes, item.scale + (size_t)i * kMpAScaleBytes, a * kMxAtomBytes, bar);
        }
        __syncwarp();
        ++filled;
        if (++st == (uint32_t)p.stages) st = 0, ph ^= 1u;
      }
      if (!ok) break;
      if (lane == 0) mbar_arrive(smem_u32(&s->item_free[slot]));
      if (++slot == kMpSlots) slot = 0, turn ^= 1u;
    }
    if (bring) {  // what is on its way lands before the CTA ends, also where another role has given up
      const uint32_t mine = min(filled, (uint32_t)p.stages);
      for (uint32_t i = 0; i < mine; ++i) {
        const uint32_t f = filled - 1 - i, b = f % p.stages, par = (f / p.stages) & 1u;
        const long long t0 = clock64();
        while (!mbar_try(smem_u32(&s->full_a[b]), par) && clock64() - t0 < 4000000ll) {
        }
      }
    }
  } else if (warp == kMpMmaWarp) {
    // ---- products ----
    uint32_t slot = 0, turn = 0, st = 0, ph = 0, acc = 0, acc_ph = 0, flip = 0;
    bool ok = true;
    while (ok && (ok = mp_wait(&s->item_full[slot], turn, s, status))) {
      const int n = s->item[slot].n;
      if (n < 0) break;
      const uint32_t idesc = mp_idesc((n + 15) & ~15), d = tmem + acc * kMpTile;
      const int blocks = (n + 127) >> 7;
      if (!(ok = mp_wait(&s->acc_free[acc], acc_ph ^ 1u, s, status))) break;
      mp_fence_after();
      for (int i = 0; i < steps; ++i) {
        if (!(ok = mp_wait(&s->full_a[st], ph, s, status))) break;
        if (!(ok = mp_wait(&s->full_b[st], ph, s, status))) break;
        mp_fence_after();
        const int c = min(kMpStepChunks, chunks - i * kMpStepChunks), a = (c + 1) >> 1;
        if (mp_elect()) {
          const uint32_t at = ring + st * stage_bytes, b_at = at + kMpABytes + kMpAScaleBytes, bs_at = b_at + b_bytes;
          const uint32_t sa = tmem + kMpScaleCol + flip * kMpScaleCols, sb = sa + 8;
          for (int j = 0; j < a; ++j) {
            mp_copy_scales(sa + 4 * j, mp_desc(at + kMpABytes + j * kMxAtomBytes, 0, 128));
            for (int h = 0; h < blocks; ++h) mp_copy_scales(sb + 8 * j + 4 * h, mp_desc(bs_at + (j * halves + h) * kMxAtomBytes, 0, 128));
          }
          for (int j = 0; j < c; ++j) {
            const uint32_t half = (uint32_t)(j & 1) * 2u;
            mp_mma(d, mp_desc(at + j * kMxChunkBytes, kMxRows * 16, 128), mp_desc(b_at + j * p.tile * 32, p.tile * 16, 128),
                   idesc | half << 29 | half << 4, sa + 4 * (j >> 1), sb + 8 * (j >> 1), (i | j) != 0);
          }
          mp_commit(smem_u32(&s->free_[st]));
          if (i == steps - 1) mp_commit(smem_u32(&s->acc_full[acc]));
        }
        __syncwarp();
        flip ^= 1u;
        if (++st == (uint32_t)p.stages) st = 0, ph ^= 1u;
      }
      if (!ok) break;
      if (lane == 0) mbar_arrive(smem_u32(&s->item_free[slot]));
      if (++slot == kMpSlots) slot = 0, turn ^= 1u;
      if (acc ^= 1u; acc == 0) acc_ph ^= 1u;
    }
    // every instruction issued is done before tensor memory is given back
    if (mp_elect()) mp_commit(smem_u32(&s->drain));
    __syncwarp();
    const long long t0 = clock64();
    while (!mbar_try(smem_u32(&s->drain), 0) && clock64() - t0 < 4000000ll) {
    }
  } else if (warp < kMpFirstDrain) {
    // ---- token rows: the warps bring the steps in turn ----
    const int me = warp - kMpFirstGather;
    uint32_t slot = 0, turn = 0, st = 0, ph = 0;
    // No more warps take turns than the ring has steps.  A warp's next step is then at most one round of the ring ahead of one that
    // it has waited for, and the parity of a barrier tells it what it needs: with more it could be two rounds ahead.
    const int gathers = min(kMpGatherWarps, p.stages);
    int next = 0;  // whose turn the step is
    bool ok = true;
    const int pitch = 4 * atoms, kbytes = p.K >> 1;
    while (ok && (ok = mp_wait(&s->item_full[slot], turn, s, status))) {
      const int n = s->item[slot].n;
      if (n < 0) break;
      const int *rows = s->row[slot];
      for (int i = 0; i < steps; ++i) {
        if (next == me) {
          if (!(ok = mp_wait(&s->free_[st], ph ^ 1u, s, status))) break;
          const int c = min(kMpStepChunks, chunks - i * kMpStepChunks), a = (c + 1) >> 1;
          const uint32_t dst = ring + st * stage_bytes + kMpABytes + kMpAScaleBytes, sdst = dst + b_bytes;
          // scales: a word of four per row and 128 values, bytes beyond the row's end cleared
          for (int r = lane; r < n; r += 32) {
            const uint8_t* src = p.scale + (size_t)rows[r] * pitch + i * (2 * kMpStepChunks);
            for (int j = 0; j < a; ++j) {
              uint32_t w = __ldcg(reinterpret_cast<const uint32_t*>(src) + j);
              const int left = (p.K >> 5) - (i * (kMpStepChunks / 2) + j) * 4;
              if (left < 4) w &= (1u << (8 * left)) - 1u;
              asm volatile("st.shared.b32 [%0], %1;" ::"r"(sdst + (j * halves + (r >> 7)) * kMxAtomBytes + (r & 31) * 16 + ((r >> 5) & 3) * 4), "r"(w) : "memory");
            }
          }
          // codes: eight rows x four pieces of 16 bytes a step of the warp; a shared-memory write is eight rows side by side
          for (int r = lane & 7; r < n; r += 8) {
            const uint8_t* src = p.codes + (size_t)rows[r] * kbytes;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const int piece = (lane >> 3) + 4 * h, at = i * (kMpStepChunks * kMxChunk / 2) + piece * 16;
              if (piece < 2 * c) {
                const bool in = at < kbytes;
                mp_cp16(dst + (piece >> 1) * p.tile * 32 + (piece & 1) * p.tile * 16 + r * 16, in ? src + at : src, in ? 16u : 0u);
              }
            }
          }
          asm volatile("cp.async.wait_all;" ::: "memory");
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_u32(&s->full_b[st]));
        }
        if (++next == gathers) next = 0;
        if (++st == (uint32_t)p.stages) st = 0, ph ^= 1u;
      }
      if (!ok) break;
      if (lane == 0) mbar_arrive(smem_u32(&s->item_free[slot]));
      if (++slot == kMpSlots) slot = 0, turn ^= 1u;
    }
  } else {
    // ---- results: a warp reads 32 weight rows, 16 tokens at a time, every other sixteen ----
    const int quarter = warp & 3, half = (warp - kMpFirstDrain) >> 2;
    uint32_t slot = 0, turn = 0, acc = 0, acc_ph = 0;
    bool ok = true;
    O* out = static_cast<O*>(p.out);
    while (ok && (ok = mp_wait(&s->item_full[slot], turn, s, status))) {
      const int n = s->item[slot].n, rb = s->item[slot].rb;
      if (n < 0) break;
      if (!(ok = mp_wait(&s->acc_full[acc], acc_ph, s, status))) break;
      mp_fence_after();
      const uint32_t d = tmem + ((uint32_t)(quarter * 32) << 16) + acc * kMpTile;
      for (int c0 = 16 * half; c0 < n; c0 += 32) {
        uint32_t r[16];
        mp_ld16(d + c0, r);
        const int4* pairs = reinterpret_cast<const int4*>(&s->pair[slot][c0]);
        int pr[16];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int4 v = pairs[i];
          pr[4 * i] = v.x, pr[4 * i + 1] = v.y, pr[4 * i + 2] = v.z, pr[4 * i + 3] = v.w;
        }
        if constexpr (GATED) {
          // lanes 0 to 15 hold gate, 16 to 31 up of the same columns of the result: of two tokens, the lower lanes take the first
          const bool hi = lane & 16;
          const int col = rb * 64 + quarter * 16 + (lane & 15);
#pragma unroll
          for (int i = 0; i < 16; i += 2) {
            const float v0 = __uint_as_float(r[i]), v1 = __uint_as_float(r[i + 1]);
            const float got = __shfl_xor_sync(0xffffffffu, hi ? v0 : v1, 16);
            const float g = hi ? got : v0, u = hi ? v1 : got;
            if (c0 + i + (hi ? 1 : 0) < n && col < p.N) out[(size_t)(hi ? pr[i + 1] : pr[i]) * p.N + col] = mx_from_float<O>(mp_silu(g) * u);
          }
        } else {
          const int col = rb * kMxRows + quarter * 32 + lane;
          if (sizeof(O) == 2 && (p.N & 1) == 0) {  // two columns of one token to a lane
            const bool hi = lane & 1;
#pragma unroll
            for (int i = 0; i < 16; i += 2) {
              const float v0 = __uint_as_float(r[i]), v1 = __uint_as_float(r[i + 1]);
              const float got = __shfl_xor_sync(0xffffffffu, hi ? v0 : v1, 1);
              if (c0 + i + (hi ? 1 : 0) < n && col < p.N)
                *reinterpret_cast<uint32_t*>(out + (size_t)(hi ? pr[i + 1] : pr[i]) * p.N + (col & ~1)) = mp_pack2<O>(hi ? got : v0, hi ? v1 : got);
            }
          } else {
#pragma unroll
            for (int i = 0; i < 16; ++i)
              if (c0 + i < n && col < p.N) out[(size_t)pr[i] * p.N + col] = mx_from_float<O>(__uint_as_float(r[i]));
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
  mp_fence_before();
  __syncthreads();
  mp_fence_after();
  if (warp == kMpMmaWarp) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kMpTmemCols) : "memory");
}

template <class O, bool GATED>
static int mp_launch(const MpParams& p, int items, cudaStream_t st) {
  static bool attr_set[64];
  static int sm_count[64];
  int dev = 0;
  SM_CUDA_TRY(cudaGetDevice(&dev));
  if (dev < 0 || dev >= 64) return SLICEMOE_E_UNSUPPORTED;
  if (!attr_set[dev]) {
    SM_CUDA_TRY(cudaFuncSetAttribute(mp_product_kernel<O, GATED>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMpSmemMax));
    SM_CUDA_TRY(cudaDeviceGetAttribute(&sm_count[dev], cudaDevAttrMultiProcessorCount, dev));
    attr_set[dev] = true;
  }
  const int stage = kMpABytes + kMpAScaleBytes + p.tile * (kMpStepChunks * kMxChunk / 2) + (p.tile + 127) / 128 * kMpAScaleBytes;
  const int smem = kMpFixed + p.stages * stage;
  return mx_launch(mp_product_kernel<O, GATED>, dim3(items < sm_count[dev] ? items : sm_count[dev]), kMpAllThreads,
                   (size_t)(smem > kMpSmemMin ? smem : kMpSmemMin), st, MpParams(p));
}
template <class O>
static int mp_launch_as(const MpParams& p, int items, cudaStream_t st) {
  return p.gated ? mp_launch<O, true>(p, items, st) : mp_launch<O, false>(p, items, st);
}

}  // namespace slicemoe

using namespace slicemoe;

extern "C" size_t slicemoe_mx4_workspace_bytes(int T, int k, int n_experts) {
  if (T <= 0 || k < 1 || k > SLICEMOE_MAX_TOP_K || n_experts <= 0 || n_experts > kMpMaxExperts || (int64_t)T * k > kMpMaxPairs) return 0;
  return mp_layout((int64_t)T * k, n_experts).total;
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
  const int pairs = T * k;
  const MpLayout l = mp_layout(pairs, n_experts);
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
  p.E = ids ? n_experts : 1;
  p.N = N;
  p.K = K;
  p.gated = gated;
  p.T = T;
  p.k = k;
  p.x_per_pair = x_per_pair;
  // an expert has at most T rows where no token names one twice: wider tiles would only take room from the ring
  p.tile = T >= kMpTile ? kMpTile : (T + 15) & ~15;
  const int stage = kMpABytes + kMpAScaleBytes + p.tile * (kMpStepChunks * kMxChunk / 2) + (p.tile + 127) / 128 * kMpAScaleBytes;
  p.stages = (kMpSmemMax - kMpFixed) / stage;
  if (p.stages > kMpMaxStages) p.stages = kMpMaxStages;
  p.row_blocks = mx_row_blocks(N, gated);
  const int64_t tiles = (int64_t)pairs / p.tile + (pairs < p.E ? pairs : p.E), items = tiles * p.row_blocks;
  if (items > INT32_MAX) return SLICEMOE_E_UNSUPPORTED;
  if (ids && pairs > kMpInline) {
    int* first = reinterpret_cast<int*>(ws + l.first);
    int* list = reinterpret_cast<int*>(ws + l.list);
    int* block_first = l.blocks > 1 ? reinterpret_cast<int*>(ws + l.block_first) : first;
    int* block_list = l.blocks > 1 ? reinterpret_cast<int*>(ws + l.block_list) : list;
    int rc = mx_launch(mp_sort_kernel, dim3(l.blocks), kMpSortThreads, 0, st, MpSortParams{ids, pairs, n_experts, block_first, block_list, p.head});
    if (rc != SLICEMOE_OK) return rc;
    if (l.blocks > 1) {
      rc = mx_launch(mp_merge_kernel, dim3(l.blocks), kMpSortThreads, 0, st, MpMergeParams{block_first, block_list, l.blocks, n_experts, first, list});
      if (rc != SLICEMOE_OK) return rc;
    }
    p.first = first;
    p.list = list;
  }
  if (dtype == SLICEMOE_F32) return mp_launch_as<float>(p, (int)items, st);
  if (dtype == SLICEMOE_BF16) return mp_launch_as<__nv_bfloat16>(p, (int)items, st);
  return mp_launch_as<__half>(p, (int)items, st);
}
