// Attention of a batch whose members share a prefix (sa_shared_prefix_attn).
//
// For one query row with key sets A (the shared prefix) and B (its sequence's
// own keys), each again cut into parts p,
//   L = log2 sum_p 2^(L_p),   O = sum_p 2^(L_p - L) O_p,
// O_p and L_p the normalised output and log2-sum-exp over part p alone.  No row
// of a group is masked inside the shared prefix, so the rows of all its members
// pack into 128-row tiles over it: its keys and values are read once per tile
// instead of once per member, and the matrix work of the padded rows goes.  One
// launch makes all parts (the members' rows lie next to each other in Q, so a
// prefix tile is an item of attn_pipe_kernel's body whose "sequence" is the
// whole group), a second joins them row by row.
//
// Probabilities are rounded to bf16 for the PV product (its matrix instruction's
// operand), as in attn_pipe.h; scores, sums, partials and their join are fp32.
//
// Bound by HBM for one token per member (32 of 16K keys, 32/8 heads: 110 MB in 25
// us and the merge's 7, against 154 by the segment attention), by the matrix
// cores and the softmax beside them from some 200 rows on (64 of 64K, 64/8 heads: 139
// GFLOP in 175 us and 14, the shortest 150 and 12, against 1155).
#pragma once

#include "attn_pipe.h"
#include "branch_plan.h"

namespace sa {

template <int P, bool kPoolRsrc>
__global__ __launch_bounds__(256, 2) void attn_shared_kernel(AttnArgs a) {
  __shared__ __attribute__((aligned(1024))) uint8_t k_lds0[kTileBytes], k_lds1[kTileBytes];
  __shared__ __attribute__((aligned(1024))) uint8_t v_lds0[kTileBytes], v_lds1[kTileBytes];
  __shared__ float dec_stats[2 * 4 * kDecRows + 1];
  const AttnItem it = ld_uniform(a.items + blockIdx.x);
  if (it.kv_begin >= it.kv_end) return;                     // padding item
  const SeqDesc sd{it.q_start, it.q_len, it.kv_len, 0};
  const PipeLds L{(lds_u8*)k_lds0, (lds_u8*)k_lds1, (lds_u8*)v_lds0, (lds_u8*)v_lds1,
                  nullptr, nullptr, nullptr, nullptr, nullptr};
  const int rows = it.q_len * a.G;
  if (rows <= 16)
    decode_group<P, true, 1, true>(a, it, (lds_u8*)k_lds0, (lds_u8*)k_lds1, (lds_u8*)v_lds0, (lds_u8*)v_lds1,
                                   (lds_f32*)dec_stats);
  else if (rows <= kDecRows)
    decode_group<P, true, 2, true>(a, it, (lds_u8*)k_lds0, (lds_u8*)k_lds1, (lds_u8*)v_lds0, (lds_u8*)v_lds1,
                                   (lds_f32*)dec_stats);
  else
    pipe_group<P, kPoolRsrc, 1, 0, false, true, true>(a, it, sd, L);
}

struct MergeRowsArgs {
  const float* part_o;       // [part rows][kHD]
  const float* part_lse;     // [part rows], log2
  const MergeUnit* units;
  uint16_t* o;
  float* lse;                // nullable
  int32_t Hq, Hkv, G, block_rows;
};

__device__ __forceinline__ float half_max(float x) {
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) x = fmaxf(x, __shfl_xor(x, d));
  return x;
}
__device__ __forceinline__ float half_sum(float x) {
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) x += __shfl_xor(x, d);
  return x;
}

// Block ((unit, KV head), y): rows block_rows y .. of the unit, 8 / block_rows half waves
// (32 threads, four d each) per row, which share the row's parts and meet in LDS.
// A half wave takes its parts 32 at a time: lane c has the c-th one's weight, and
// the partial rows are loaded eight ahead of their use.  With block_rows = 1, 2,
// 4 or 8 by the most parts of a row (merge_block_rows) a half wave has at most
// about eight parts, whose loads are all in flight at once: the launch is bound
// by that latency.  32 branches of 16K, 30 parts a row:
// 13.4 us with a row's loads one after another, 7.
__global__ __launch_bounds__(256) void merge_rows_kernel(MergeRowsArgs a) {
  __shared__ f32x4 red[8][32];
  __shared__ float red_m[8], red_den[8];
  const int unit = blockIdx.x / a.Hkv, kvh = blockIdx.x - unit * a.Hkv;
  const MergeUnit u = ld_uniform(a.units + unit);
  const int r0 = blockIdx.y * a.block_rows;
  if (r0 >= u.n) return;
  const int lane = threadIdx.x & 63, hw = threadIdx.x >> 5, c = threadIdx.x & 31;
  const int nsub = 8 / a.block_rows;
  const int sub = hw % nsub;
  const int r = r0 + hw / nsub;
  const bool mine = r < u.n;
  const int np = mine ? u.a_n + u.b_n : 0;
  auto row_of = [&](int s) {
    return r + (s < u.a_n ? (int64_t)u.a_row + ((int64_t)kvh * u.a_n + s) * u.a_stride
                          : (int64_t)u.b_row + ((int64_t)kvh * u.b_n + s - u.a_n) * u.b_stride);
  };
  float mx = -INFINITY, den = 0.f;
  f32x4 num = f32x4{};
  constexpr int kAhead = 8;
  for (int s0 = sub; s0 < np; s0 += 32 * nsub) {
    const int n = min(32, (np - s0 + nsub - 1) / nsub);      // parts of this round
    f32x4 x[kAhead];
    auto load = [&](int k0) {
#pragma unroll
      for (int k = 0; k < kAhead; ++k)
        if (k0 + k < n) x[k] = *(const f32x4*)(a.part_o + row_of(s0 + (k0 + k) * nsub) * kHD + 4 * c);
    };
    load(0);
    const float l = c < n ? a.part_lse[row_of(s0 + c * nsub)] : -INFINITY;
    const float m_new = fmaxf(mx, half_max(l));
    const float off = m_new == -INFINITY ? 0.f : m_new;
    const float f = exp2f_fast(mx - off), w = exp2f_fast(l - off);
    num *= f;
    den = den * f + half_sum(w);
    mx = m_new;
    for (int k0 = 0; k0 < n; k0 += kAhead) {
#pragma unroll
      for (int k = 0; k < kAhead; ++k)
        if (k0 + k < n) num += __shfl(w, (lane & 32) + k0 + k) * x[k];
      load(k0 + kAhead);
    }
  }
  if (nsub > 1) {
    red[hw][c] = num;
    if (c == 0) {
      red_m[hw] = mx;
      red_den[hw] = den;
    }
    __syncthreads();
    if (!mine || sub != 0) return;
    float all = mx;
    for (int k = 1; k < nsub; ++k) all = fmaxf(all, red_m[hw + k]);
    const float off = all == -INFINITY ? 0.f : all;
    float f = exp2f_fast(mx - off);
    num *= f;
    den *= f;
    for (int k = 1; k < nsub; ++k) {
      f = exp2f_fast(red_m[hw + k] - off);
      num += f * red[hw + k][c];
      den += f * red_den[hw + k];
    }
    mx = all;
  }
  if (!mine) return;
  const float inv = den > 0.f ? 1.f / den : 0.f;
  const int row = u.r0 + r, tok = row / a.G;
  const int64_t orow = (int64_t)(u.q_start + tok) * a.Hq + kvh * a.G + (row - tok * a.G);
  st_bf16x4(a.o + orow * kHD + 4 * c, num[0] * inv, num[1] * inv, num[2] * inv, num[3] * inv);
  if (a.lse != nullptr && c == 0)
    a.lse[orow] = den == 0.f ? -INFINITY : (mx + __builtin_amdgcn_logf(den)) * 0.69314718055994531f;
}

}  // namespace sa
