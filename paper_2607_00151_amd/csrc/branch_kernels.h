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
// partial page, of K or of V, in one layer.
__global__ __launch_bounds__(256) void fork_kernel(ForkArgs a) {
  const int tid = threadIdx.x;
  if ((int)blockIdx.x < a.table_blocks) {
    const int e = blockIdx.x * 256 + tid;
    if (e <= a.C) a.out_indptr[e] = a.dst_indptr[e];
    if (e >= a.n_dst) return;
    const ForkChild ch = a.children[find_seq(a.dst_indptr, a.C, e)];
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
      const int old = atomicAdd(a.ref + slot, 1);
      if (j < ch.full ? old < 1 : old != 0) atomicOr(a.err, kCountError);
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
__global__ __launch_bounds__(256) void count_kernel(CountArgs a) {
  const int64_t lo = a.indptr[0], hi = a.indptr[a.batch];
  if (lo < 0 || hi < lo || hi > a.max_entries) {
    if (blockIdx.x == 0 && threadIdx.x == 0) atomicOr(a.err, 4);
    return;
  }
  for (int64_t e = lo + (int64_t)blockIdx.x * 256 + threadIdx.x; e < hi; e += (int64_t)gridDim.x * 256) {
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

// ---------------------------------------------------------------- scans over the slots
//
// A list of slots in order needs, for each chunk of slots, how many of those
// before it are listed: a launch leaves each chunk's number, and the next one's
// blocks add up the numbers before theirs.  A pool of one chunk needs no counting
// launch.  (Every block counting all slots before its own instead: 14 us against
// 7.5 for both launches at 28K slots.)

constexpr int kScanThreads = 512;
constexpr int kScanPer = 8;                                 // slots per thread
constexpr int kScanChunk = kScanThreads * kScanPer;

// Sums of two numbers over the block; every thread gets them.
__device__ __forceinline__ int2 block_sum(int2 x, int2* room) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) {
    x.x += __shfl_xor(x.x, d);
    x.y += __shfl_xor(x.y, d);
  }
  __syncthreads();
  if (lane == 0) room[wave] = x;
  __syncthreads();
  int2 s = {0, 0};
#pragma unroll
  for (int k = 0; k < kScanThreads / 64; ++k) {
    s.x += room[k].x;
    s.y += room[k].y;
  }
  return s;
}

// Sum over the threads before this one.
__device__ __forceinline__ int block_before(int x, int2* room) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int inc = x;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int y = __shfl_up(inc, d);
    if (lane >= d) inc += y;
  }
  __syncthreads();
  if (lane == 63) room[wave].x = inc;
  __syncthreads();
  int s = inc - x;
  for (int k = 0; k < wave; ++k) s += room[k].x;
  return s;
}

// Listed slots before this block's chunk (x) and in all (y), from the chunks'
// numbers or, with one chunk, from the thread's own.
__device__ __forceinline__ int2 count_listed(const int32_t* counts, int chunks, int own, int2* room) {
  int2 n = {0, 0};
  if (counts == nullptr) n.y = own;
  else
    for (int k = threadIdx.x; k < chunks; k += kScanThreads) {
      const int x = counts[k];
      n.y += x;
      if (k < (int)blockIdx.x) n.x += x;
    }
  return block_sum(n, room);
}

struct FreeArgs {
  const int32_t* ref;
  int32_t* free_list;          // [num_slots]
  int32_t* num_free;
  int32_t* counts;             // [chunks] free slots of each chunk; null: there is one
  int32_t num_slots, chunks;
};

__global__ __launch_bounds__(kScanThreads) void free_count_kernel(FreeArgs a) {
  __shared__ int2 room[kScanThreads / 64];
  const int s0 = blockIdx.x * kScanChunk + threadIdx.x;
  int2 n = {0, 0};
#pragma unroll
  for (int i = 0; i < kScanPer; ++i) {
    const int s = s0 + i * kScanThreads;
    n.x += s < a.num_slots && a.ref[s] == 0;
  }
  n = block_sum(n, room);
  if (threadIdx.x == 0) a.counts[blockIdx.x] = n.x;
}

// The slots without a count, ascending, then -1 up to num_slots.
__global__ __launch_bounds__(kScanThreads) void free_list_kernel(FreeArgs a) {
  __shared__ int2 room[kScanThreads / 64];
  const int s0 = blockIdx.x * kScanChunk + threadIdx.x * kScanPer;
  unsigned idle = 0;
#pragma unroll
  for (int i = 0; i < kScanPer; ++i) idle |= (unsigned)(s0 + i < a.num_slots && a.ref[s0 + i] == 0) << i;
  const int2 n = count_listed(a.counts, a.chunks, __popc(idle), room);
  int at = n.x + block_before(__popc(idle), room);
#pragma unroll
  for (int i = 0; i < kScanPer; ++i) {
    if ((idle >> i) & 1) a.free_list[at++] = s0 + i;
    if (s0 + i < a.num_slots && s0 + i >= n.y) a.free_list[s0 + i] = -1;
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) *a.num_free = n.y;
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
__device__ __forceinline__ bool is_hole(const CompactArgs& a, int s) { return s < a.limit && a.ref[s] <= 0; }
__device__ __forceinline__ bool is_mover(const CompactArgs& a, int s) {
  return s >= a.limit && s < a.num_slots && a.ref[s] > 0;
}

__global__ __launch_bounds__(kScanThreads) void compact_count_kernel(CompactArgs a) {
  __shared__ int2 room[kScanThreads / 64];
  const int s0 = blockIdx.x * kScanChunk + threadIdx.x;
  int2 n = {0, 0};
#pragma unroll
  for (int i = 0; i < kScanPer; ++i) {
    n.x += is_hole(a, s0 + i * kScanThreads);
    n.y += is_mover(a, s0 + i * kScanThreads);
  }
  n = block_sum(n, room);
  if (threadIdx.x == 0) {
    a.counts[blockIdx.x] = n.x;
    a.counts[a.chunks + blockIdx.x] = n.y;
  }
}

// Ranks of holes and movers, of which the first min(holes, movers) take part.
// rank[s]: the rank of a hole or mover that takes part, else kStays for a slot
// in use and kIdle for one that is not.
constexpr int kStays = -1, kIdle = -2;

__global__ __launch_bounds__(kScanThreads) void compact_rank_kernel(CompactArgs a) {
  __shared__ int2 room[kScanThreads / 64];
  const int s0 = blockIdx.x * kScanChunk + threadIdx.x * kScanPer;
  int count[kScanPer];
  unsigned hole = 0, mover = 0;
#pragma unroll
  for (int i = 0; i < kScanPer; ++i) {
    count[i] = s0 + i < a.num_slots ? a.ref[s0 + i] : 0;
    hole |= (unsigned)(s0 + i < a.limit && count[i] <= 0) << i;
    mover |= (unsigned)(s0 + i >= a.limit && count[i] > 0) << i;
  }
  const int2 hs = count_listed(a.counts, a.chunks, __popc(hole), room);
  const int2 ms = count_listed(a.counts == nullptr ? nullptr : a.counts + a.chunks, a.chunks, __popc(mover), room);
  const int n = min(hs.y, ms.y);
  int h = hs.x + block_before(__popc(hole), room);
  int m = ms.x + block_before(__popc(mover), room);
#pragma unroll
  for (int i = 0; i < kScanPer; ++i) {
    const int s = s0 + i;
    if (s >= a.num_slots) break;
    int rank = count[i] > 0 ? kStays : kIdle;
    if ((hole >> i) & 1) {
      if (h < n) {
        rank = h;
        a.hole[h] = s;
      }
      ++h;
    } else if ((mover >> i) & 1) {
      if (m < n) {
        rank = m;
        a.mover[m] = s;
        a.mover_ref[m] = count[i];
      }
      ++m;
    }
    a.rank[s] = rank;
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
// unit u is K or V of one moved page in one layer.
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
