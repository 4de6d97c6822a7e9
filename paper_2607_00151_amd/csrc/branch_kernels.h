// Pages of branches: forks of cached contexts, the counts of the tables that
// list each slot, the list of free slots, and the compaction of a pool.
//
// A slot's count is the number of table entries that name it.  Counts are
// raised and lowered by integer atomics, whose order does not show.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "branch_plan.h"
#include "common.h"
#include "kv_kernels.h"
#include "rope_kernels.h"

namespace sa {

constexpr int kCountError = 8;         // error flag: a count that does not fit the tables

// ---------------------------------------------------------------- fork

struct ForkArgs {
  uint16_t* k_pool;
  uint16_t* v_pool;
  const ForkChild* children;
  const int32_t* dst_indptr;   // [C + 1] plan copy of the destination table offsets
  const int32_t* copies;       // [n_copies] children with a partial page
  const int32_t* src_indptr;
  const int32_t* src_indices;
  const int32_t* fresh;
  int32_t* out_indptr;
  int32_t* out_indices;
  int32_t* ref;                // nullable
  int32_t* err;
  int64_t num_slots;
  int64_t slot_elems;
  int64_t layer_elems;
  int32_t n_dst, C, n_copies, table_blocks, Hkv, P;
};

// Blocks 0 .. table_blocks - 1 write the destination table, a thread per entry,
// and raise its slots' counts; the others copy the valid rows of one child's
// partial page, of K or of V, in one layer.  Bound by trips to memory (children,
// parent's table, count): 64 children of 16 contexts, 83K entries, two layers,
// 5.6 us; 7.4 where every child's entry raised the shared page's count itself.
__global__ __launch_bounds__(256) void fork_kernel(ForkArgs a) {
  const int tid = threadIdx.x;
  if ((int)blockIdx.x < a.table_blocks) {
    const int e = blockIdx.x * 256 + tid;
    if (e <= a.C) a.out_indptr[e] = a.dst_indptr[e];
    // the child of the wave's first entry, and of each lane's from there on
    const int first = __builtin_amdgcn_readfirstlane(e);
    if (first >= a.n_dst) return;
    int c = __builtin_amdgcn_readfirstlane(wave_find_seq(a.dst_indptr, a.C, first));
    if (e >= a.n_dst) return;
    if (a.dst_indptr[c + 1] <= min(first + 63, a.n_dst - 1)) c += find_seq(a.dst_indptr + c, a.C - c, e);
    const ForkChild ch = a.children[c];
    const int j = e - ch.dst0;
    int32_t slot = -1;
    if (j < ch.full) {
      const int32_t base = a.src_indptr[ch.parent];
      if (j < a.src_indptr[ch.parent + 1] - base) slot = a.src_indices[base + j];
    } else {
      slot = a.fresh[ch.fresh0 + j - ch.full];
    }
    a.out_indices[e] = slot;
    if (slot < 0 || (int64_t)slot >= a.num_slots) {
      atomicOr(a.err, 4);
    } else if (a.ref != nullptr) {
      // a shared page is in use already, a fresh slot is not
      if (j >= ch.full) {
        if (atomicAdd(a.ref + slot, 1) != 0) atomicOr(a.err, kCountError);
      } else if (ch.raise > 0 && atomicAdd(a.ref + slot, ch.raise) < 1) {
        atomicOr(a.err, kCountError);
      }
    }
    return;
  }
  const int u = blockIdx.x - a.table_blocks;
  const int which = u & 1;
  const int layer = (u >> 1) / a.n_copies;
  const ForkChild ch = a.children[a.copies[(u >> 1) - layer * a.n_copies]];
  const int32_t base = a.src_indptr[ch.parent];
  const int32_t s = ch.full < a.src_indptr[ch.parent + 1] - base ? a.src_indices[base + ch.full] : -1;
  const int32_t d = a.fresh[ch.fresh0];
  if (s < 0 || (int64_t)s >= a.num_slots || d < 0 || (int64_t)d >= a.num_slots) {
    if (tid == 0) atomicOr(a.err, 4);
    return;
  }
  uint16_t* const pool = (which ? a.v_pool : a.k_pool) + layer * a.layer_elems;
  const uint16_t* const src = pool + s * a.slot_elems;
  uint16_t* const dst = pool + d * a.slot_elems;
  const int per_head = ch.rows * 16;                       // 16-byte chunks of a head's valid rows
  const int n = a.Hkv * per_head;
  constexpr int kDepth = 4;
  for (int c0 = tid; c0 < n; c0 += 256 * kDepth) {
    u32x4 x[kDepth];
    int off[kDepth];
#pragma unroll
    for (int i = 0; i < kDepth; ++i) {
      const int c = c0 + 256 * i, head = c / per_head;
      off[i] = head * a.P * kHD + (c - head * per_head) * 8;
      if (c < n) x[i] = ld_u32x4(src + off[i]);
    }
#pragma unroll
    for (int i = 0; i < kDepth; ++i)
      if (c0 + 256 * i < n) st_u32x4(dst + off[i], x[i]);
  }
}

// ---------------------------------------------------------------- counts

struct CountArgs {
  const int32_t* indptr;       // [batch + 1]
  const int32_t* indices;
  int32_t* ref;
  int32_t* err;
  int64_t num_slots;
  int64_t max_entries;         // entries that indices holds
  int32_t batch;
};

// Every entry of the tables raises (kUp) or lowers its slot's count.  A count
// never falls below zero: an entry that finds none left puts it back and raises
// the error flag.
template <bool kUp>
__device__ __forceinline__ void count_entries(const CountArgs& a) {
  const int64_t lo = a.indptr[0], hi = a.indptr[a.batch];
  if (lo < 0 || hi < lo || hi > a.max_entries) {
    if (blockIdx.x == 0 && threadIdx.x == 0) atomicOr(a.err, 4);
    return;
  }
  const int64_t stride = (int64_t)gridDim.x * blockDim.x;
  for (int64_t e = lo + (int64_t)blockIdx.x * blockDim.x + threadIdx.x; e < hi; e += stride) {
    const int32_t slot = a.indices[e];
    if (slot < 0 || (int64_t)slot >= a.num_slots) {
      atomicOr(a.err, 4);
    } else if (kUp) {
      atomicAdd(a.ref + slot, 1);
    } else if (atomicSub(a.ref + slot, 1) <= 0) {
      atomicAdd(a.ref + slot, 1);
      atomicOr(a.err, kCountError);
    }
  }
}

template <bool kUp>
__global__ __launch_bounds__(256) void count_kernel(CountArgs a) {
  count_entries<kUp>(a);
}

// ---------------------------------------------------------------- scans over the slots
//
// A list of slots in order needs, for each chunk of slots, how many of those
// before it are listed: a launch leaves each chunk's number, and the next one's
// blocks add up the numbers before theirs.  A pool of one chunk needs no counting
// launch.  Bound by trips to memory: 37K slots 4.2 us each launch, against 14 in one
// launch whose blocks all count the slots before their own.

constexpr int kScanThreads = 512;
constexpr int kScanPer = 8;                                 // slots per thread
constexpr int kScanWaves = kScanThreads / 64;
constexpr int kScanChunk = kScanThreads * kScanPer;

// A wave has 512 slots in a row, lane l slots l, 64 + l, ...: loads and stores of
// whole lines, and a slot's place among the wave's listed ones by ballots.
__device__ __forceinline__ int scan_slot(int i) {
  return blockIdx.x * kScanChunk + (threadIdx.x >> 6) * (64 * kScanPer) + i * 64 + (threadIdx.x & 63);
}
__device__ __forceinline__ int lanes_before(uint64_t mask) {
  return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0u));
}

struct ScanRoom {
  int own[kScanWaves], before[kScanWaves], all[kScanWaves];
};

// Of the listed slots (mask[i]: lanes whose i-th slot is): those before this
// wave's (x) and all of the pool's (y).  counts: the chunks' numbers, or null with
// one chunk.  Every thread of the block takes part.
__device__ __forceinline__ int2 scan_block(const uint64_t (&mask)[kScanPer], const int32_t* counts, int chunks,
                                           ScanRoom& room) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int own = 0;
#pragma unroll
  for (int i = 0; i < kScanPer; ++i) own += __popcll(mask[i]);
  int before = 0, all = 0;
  if (counts != nullptr) {
    for (int k = threadIdx.x; k < chunks; k += kScanThreads) {
      const int x = counts[k];
      all += x;
      if (k < (int)blockIdx.x) before += x;
    }
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) {
      before += __shfl_xor(before, d);
      all += __shfl_xor(all, d);
    }
  } else {
    all = own;
  }
  if (lane == 0) {
    room.own[wave] = own;
    room.before[wave] = before;
    room.all[wave] = all;
  }
  __syncthreads();
  int2 n = {0, 0};
#pragma unroll
  for (int k = 0; k < kScanWaves; ++k) {
    n.x += room.before[k] + (k < wave ? room.own[k] : 0);
    n.y += room.all[k];
  }
  __syncthreads();                                          // the room may be used again
  return n;
}

// A chunk's number of listed slots.
__device__ __forceinline__ void count_block(const uint64_t (&mask)[kScanPer], int32_t* count, ScanRoom& room) {
  int own = 0;
#pragma unroll
  for (int i = 0; i < kScanPer; ++i) own += __popcll(mask[i]);
  if ((threadIdx.x & 63) == 0) room.own[threadIdx.x >> 6] = own;
  __syncthreads();
  if (threadIdx.x == 0) {
    int n = 0;
    for (int k = 0; k < kScanWaves; ++k) n += room.own[k];
    *count = n;
  }
  __syncthreads();
}

struct FreeArgs {
  const int32_t* ref;
  int32_t* free_list;          // [num_slots]
  int32_t* num_free;
  int32_t* counts;             // [chunks] free slots of each chunk; null: there is one
  int32_t num_slots, chunks;
};

__device__ __forceinline__ void idle_slots(const FreeArgs& a, uint64_t (&mask)[kScanPer]) {
  bool idle[kScanPer];
#pragma unroll
  for (int i = 0; i < kScanPer; ++i) {
    const int s = scan_slot(i);
    // at device scope: where the counts were lowered by this same launch
    idle[i] = s < a.num_slots && __hip_atomic_load(a.ref + s, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) <= 0;
  }
#pragma unroll
  for (int i = 0; i < kScanPer; ++i) mask[i] = __ballot(idle[i]);
}

__global__ __launch_bounds__(kScanThreads) void free_count_kernel(FreeArgs a) {
  __shared__ ScanRoom room;
  uint64_t mask[kScanPer];
  idle_slots(a, mask);
  count_block(mask, a.counts + blockIdx.x, room);
}

// The slots without a count, ascending, then -1 up to num_slots.
__device__ __forceinline__ void list_idle(const FreeArgs& a, ScanRoom& room) {
  uint64_t mask[kScanPer];
  idle_slots(a, mask);
  const int2 n = scan_block(mask, a.counts, a.chunks, room);
  int at = n.x;
#pragma unroll
  for (int i = 0; i < kScanPer; ++i) {
    const int s = scan_slot(i);
    if ((mask[i] >> (threadIdx.x & 63)) & 1) a.free_list[at + lanes_before(mask[i])] = s;
    at += __popcll(mask[i]);
    if (s < a.num_slots && s >= n.y) a.free_list[s] = -1;
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) *a.num_free = n.y;
}

__global__ __launch_bounds__(kScanThreads) void free_list_kernel(FreeArgs a) {
  __shared__ ScanRoom room;
  list_idle(a, room);
}

// A small pool's whole release in one block: its entries lower the counts, and
// once the atomics have returned the block lists the slots.  What it saves is the
// host's work of a launch; each thread's atomics follow one another, so it is for
// few entries.  A call of it and of the two launches, us, 1295 slots: 16 entries
// 6.5 and 8.9, 1020 7.7 and 9.1, 2048 8.9 and 9.1, 4096 11.8 and 9.2; 4096 slots:
// 6.4 and 9.0, 8.3 and 9.2, 9.7 and 9.1, 13.0 and 9.1.  (Replayed from a graph, which
// has no host's work to save, it takes 5.6 and 5.3, 7.5 and 6.1 at 1295 slots.)
constexpr int64_t kOneBlockEntries = 1536;

__global__ __launch_bounds__(kScanThreads) void release_small_kernel(CountArgs c, FreeArgs a) {
  __shared__ ScanRoom room;
  count_entries<false>(c);
  __threadfence();
  __syncthreads();
  list_idle(a, room);
}

// ---------------------------------------------------------------- compaction

struct CompactArgs {
  uint16_t* k_pool;
  uint16_t* v_pool;
  const int32_t* ref;
  int32_t* ref_out;
  const int32_t* indices;
  int32_t* indices_out;
  int32_t* slot_map;           // [num_slots]
  int32_t* moved;              // [2] pages moved, pages left from the limit on
  int32_t* err;
  int32_t* counts;             // [2][chunks] holes and movers of each chunk; null: there is one
  int32_t* rank;               // [num_slots], see compact_rank_kernel
  int32_t* hole;               // [num_slots] slot of each hole, by rank
  int32_t* mover;              // [num_slots]
  int32_t* mover_ref;          // [num_slots]
  int64_t slot_elems;
  int64_t layer_elems;
  int64_t num_entries;
  int32_t num_slots, limit, chunks, num_layers;
};

// Holes are the free slots below the limit, movers the slots in use from it on.
__device__ __forceinline__ void holes_and_movers(const CompactArgs& a, int (&count)[kScanPer], uint64_t (&hole)[kScanPer],
                                                 uint64_t (&mover)[kScanPer]) {
#pragma unroll
  for (int i = 0; i < kScanPer; ++i) {
    const int s = scan_slot(i);
    count[i] = s < a.num_slots ? a.ref[s] : 0;
  }
#pragma unroll
  for (int i = 0; i < kScanPer; ++i) {
    const int s = scan_slot(i);
    hole[i] = __ballot(s < a.limit && count[i] <= 0);
    mover[i] = __ballot(s >= a.limit && count[i] > 0);
  }
}

__global__ __launch_bounds__(kScanThreads) void compact_count_kernel(CompactArgs a) {
  __shared__ ScanRoom room;
  int count[kScanPer];
  uint64_t hole[kScanPer], mover[kScanPer];
  holes_and_movers(a, count, hole, mover);
  count_block(hole, a.counts + blockIdx.x, room);
  count_block(mover, a.counts + a.chunks + blockIdx.x, room);
}

// Ranks of holes and movers, of which the first min(holes, movers) take part.
// rank[s]: the rank of a hole or mover that takes part, else kStays for a slot
// in use and kIdle for one that is not.
constexpr int kStays = -1, kIdle = -2;

__global__ __launch_bounds__(kScanThreads) void compact_rank_kernel(CompactArgs a) {
  __shared__ ScanRoom room;
  int count[kScanPer];
  uint64_t hole[kScanPer], mover[kScanPer];
  holes_and_movers(a, count, hole, mover);
  const int2 hs = scan_block(hole, a.counts, a.chunks, room);
  const int2 ms = scan_block(mover, a.counts == nullptr ? nullptr : a.counts + a.chunks, a.chunks, room);
  const int n = min(hs.y, ms.y);
  int h = hs.x, m = ms.x;
#pragma unroll
  for (int i = 0; i < kScanPer; ++i) {
    const int s = scan_slot(i);
    int rank = count[i] > 0 ? kStays : kIdle;
    if ((hole[i] >> (threadIdx.x & 63)) & 1) {
      const int at = h + lanes_before(hole[i]);
      if (at < n) {
        rank = at;
        a.hole[at] = s;
      }
    } else if ((mover[i] >> (threadIdx.x & 63)) & 1) {
      const int at = m + lanes_before(mover[i]);
      if (at < n) {
        rank = at;
        a.mover[at] = s;
        a.mover_ref[at] = count[i];
      }
    }
    h += __popcll(hole[i]);
    m += __popcll(mover[i]);
    if (s < a.num_slots) a.rank[s] = rank;
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    a.moved[0] = n;
    a.moved[1] = ms.y - n;
  }
}

// Where a slot's page goes: itself, a hole, or -1 for a slot not in use.  Reads
// only what compact_rank_kernel left, so that counts may be rewritten meanwhile.
__device__ __forceinline__ int new_slot(const CompactArgs& a, int s) {
  const int r = a.rank[s];
  return r == kStays ? s : r >= 0 && s >= a.limit ? a.hole[r] : -1;
}

// The counts, the map and the table, a thread per slot or entry; and the pages:
// unit u is K or V of one moved page in one layer.  Bound by HBM: 1.7 GB in 314 us
// (5.5 TB/s), 268 MB in 48; units of half a page or blocks of 512 threads are
// within 2% of that.
__global__ __launch_bounds__(256) void compact_move_kernel(CompactArgs a) {
  const int64_t stride = (int64_t)gridDim.x * 256;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < a.num_slots; i += stride) {
    const int s = (int)i, r = a.rank[s];
    a.slot_map[s] = new_slot(a, s);
    a.ref_out[s] = r < 0 ? a.ref[s] : s < a.limit ? a.mover_ref[r] : 0;
  }
  for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < a.num_entries; e += stride) {
    const int32_t s = a.indices[e];
    int32_t to = s;
    if (s < 0 || s >= a.num_slots) {
      atomicOr(a.err, 4);
    } else {
      to = new_slot(a, s);
      if (to < 0) atomicOr(a.err, kCountError);
    }
    a.indices_out[e] = to;
  }
  const int n = a.moved[0];
  const int chunks = (int)(a.slot_elems / 8);
  for (int64_t u = blockIdx.x; u < (int64_t)n * a.num_layers * 2; u += gridDim.x) {
    const int64_t page = u >> 1;
    const int layer = (int)(page / n), i = (int)(page - (int64_t)layer * n);
    uint16_t* const pool = ((u & 1) ? a.v_pool : a.k_pool) + layer * a.layer_elems;
    const uint16_t* const src = pool + a.mover[i] * a.slot_elems;
    uint16_t* const dst = pool + a.hole[i] * a.slot_elems;
    constexpr int kDepth = 8;
    for (int c0 = threadIdx.x; c0 < chunks; c0 += 256 * kDepth) {
      u32x4 x[kDepth];
#pragma unroll
      for (int j = 0; j < kDepth; ++j)
        if (c0 + 256 * j < chunks) x[j] = ld_stream(src + (c0 + 256 * j) * 8);
#pragma unroll
      for (int j = 0; j < kDepth; ++j)
        if (c0 + 256 * j < chunks) st_stream(dst + (c0 + 256 * j) * 8, x[j]);
    }
  }
}

}  // namespace sa
