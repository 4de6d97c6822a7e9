// Attention over a cache of 4 bits (sa_kvq_attn).
//
// Row i of a sequence sees keys j < limit_i (its position, or every key where there
// is no mask):
//   s_j = c q . k_j,  m = max s_j,  O = sum 2^(s_j - m) v_j / l,  l = sum 2^(s_j - m)
// with c = scale log2 e, in one pass with m, l and O carried and rescaled when scores outgrow m.
//
// Up to 32 rows, scores are bf16 products of converted keys (a 4-bit value is a bf16 one) with
// the query rows, so exact but for the fp32 sum.  They cost nothing there, where HBM bounds:
// 259 us for 64 contexts of 4K to 32K keys, 257 with the pieces below.
// More rows take them from the block-scaled matrix instruction (16x16x128), which has
// the keys as they lie in the cache: lane l's operand is the 16 code bytes of key
// l % 16, block l / 16, with that block's scale byte.  The query goes in as three 6-bit floats
// per value (e2m3, scales 2^e, 2^(e-4), 2^(e-10) per 32 dims, each the rounded rest of the one
// before): the bf16 value itself from 2^-6 of the block's largest on, others to 2^-14 of it.  c is
// multiplied in behind the product, in fp32.  Against a bf16 product the matrix work is 3/4
// and the conversion goes; two 8-bit pieces would cost 4/4 and lose 2^-14 in the instruction's
// sum (measured).  In rows whose dims are of one size next to none are inexact (of normal
// ones 0.2 of 32), but beside an outlier all can be, and what keys of zeros at the outlier
// leave of a score is then off by as much as it is.  An item with a row of which pieces would
// lose more than kvq_coarse allows takes bf16 products (none of 16 thousand items of 128 normal
// rows, one in 2000 of rows with two-sided exponential values, most where a dim is 8 times the
// others): 2048 rows x 4 heads behind 8K keys, 254 to 258 us, take 305 so.
// Values have a scale per key and 32 dims, which a sum over keys cannot take in that
// instruction: they are converted to bf16 (exactly; 2 per v_cvt), laid out in LDS and
// read back transposed for the 16x16x32 bf16 product.  Probabilities are rounded to
// bf16 for it, as in attn_pipe.h; everything else is fp32.
//
// An item is a tile of packed rows of one KV head (row r: token r / G, head kvh G + r % G)
// over a range of keys.  Up to 32 rows: the block's four waves take a quarter of the keys
// each, with their own m, l, O and LDS and no barrier until the end, the next tile of 64
// keys (8.7 KB) in registers before the present one is computed.  More rows: the waves
// share them out and go over the keys together (kvq_split_rows).
//
// Bound by HBM for one token a sequence: 64 contexts of 4K to 32K keys, 32/8 heads, 1.39 GB
// in 259 us, 5.4 TB/s; 96 equal ones of 16K 5.7.  From some 64 rows on by the matrix cores
// and the softmax beside them: 2048 rows x 4 heads behind 8K keys, 309 GFLOP in 254 to 258 us (1.21
// PFLOP/s, matrix cores busy 47% of the time), which the bf16 cache's attention takes 262 to 268 for.
#pragma once

#include "attn_pipe.h"
#include "kvq_kernels.h"
#include "kvq_plan.h"

#include <type_traits>

namespace sa {

struct KvqAttnArgs {
  const uint16_t* q;
  const uint8_t* k;          // pools, offset to the layer
  const uint8_t* v;
  uint16_t* o;
  float* lse;                // nullable
  float* part_o;             // [part rows][kHD]
  float* part_lse;           // [part rows], log2
  const KvqItem* items;
  int32_t* count;            // arrivals of the parts that a launch joins itself, zero between launches
  const int32_t* indptr;
  const int32_t* indices;
  int32_t* err;
  int32_t num_slots, Hq, Hkv, G;
  int32_t causal;
  float c;                   // softmax scale times log2 e
};

// A head's page through a resource, which holds nothing where the slot is -1: zeros then.
typedef __amdgpu_buffer_rsrc_t KvqPage;
__device__ __forceinline__ KvqPage kvq_page(const uint8_t* pool, int32_t slot, int64_t slot_bytes, int64_t head_at,
                                            int64_t page_bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(pool + (int64_t)max(slot, 0) * slot_bytes + head_at),
                                           (short)0, slot >= 0 ? (int)page_bytes : 0, 0x00020000);
}
__device__ __forceinline__ u32x4 kvq_load_codes(KvqPage page, uint32_t at) {
  return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(page, at, 0, 0));
}
__device__ __forceinline__ uint32_t kvq_load_scale(KvqPage page, uint32_t at) {
  return (uint8_t)__builtin_amdgcn_raw_buffer_load_b8(page, at, 0, 0);
}

typedef uint32_t u32x6 __attribute__((ext_vector_type(6)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x32 __attribute__((ext_vector_type(32)));

// 32 dims of a query row as three 6-bit pieces; scales: their bytes (255: the block holds
// an infinity or a NaN).  The rests' arithmetic is exact.  With S the first piece's scale, the largest
// dim is 3.75 to 7.5 S, and the first rest is at most S / 4, of a bf16 value with 4 bits
// behind those taken: two pieces, the second from S / 128 on, hold dims from S on exactly.  The
// rest of others is at most S / 2^8, 4 of the third piece's units: it comes to S / 2^13 at most
// (half its largest step), and to nothing from S / 2^5 on.  Without c: c times a bf16 value is
// none, and three pieces of it leave 20 times as much of normal rows.
__device__ __forceinline__ void kvq_split_q(const uint16_t* p, u32x6 (&piece)[3], int& scales) {
  u32x4 w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = ld_u32x4(p + 8 * i);
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) top = max(top, max(w[i][e] & 0x7FFF0000u, (w[i][e] << 16) & 0x7FFF0000u));
  const bool fine = top < 0x7F800000u;
  const int s = max((int)((top + 0x100000u) >> 23) - 2, 11);   // 7.5: the format's largest
  f32x16 even, odd;                                          // dims 2 i and 2 i + 1, as the conversion takes them
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const uint32_t two = fine ? w[i >> 2][i & 3] : 0u;
    even[i] = __uint_as_float(two << 16);
    odd[i] = __uint_as_float(two & 0xFFFF0000u);
  }
  constexpr int kDown[3] = {0, 4, 10};
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    const float unit = __uint_as_float((uint32_t)(s - kDown[k]) << 23);
    const auto six = __builtin_amdgcn_cvt_scalef32_2xpk16_fp6_f32(even, odd, unit);
    piece[k] = __builtin_bit_cast(u32x6, six);
    if (k == 2) break;
    const f32x32 back = __builtin_amdgcn_cvt_scalef32_pk32_f32_fp6(six, unit);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      even[i] -= back[2 * i];
      odd[i] -= back[2 * i + 1];
    }
  }
  scales = fine ? s | (s - kDown[1]) << 8 | (s - kDown[2]) << 16 : 0xFFFFFF;
}

// Whether pieces would not do for 32 dims of a row.  Of a scale S they do not hold those dims that are
// no multiple of S / 2^13, and each of these is off by that at most; together it may be 2^-14
// of the magnitudes of all dims but the largest.
__device__ __forceinline__ bool kvq_coarse(const uint16_t* p) {
  u32x4 w[4];
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    w[i] = ld_u32x4(p + 8 * i);
#pragma unroll
    for (int e = 0; e < 4; ++e) top = max(top, max(w[i][e] & 0x7FFF0000u, (w[i][e] << 16) & 0x7FFF0000u));
  }
  const int n = 127 + 13 - max((int)((top + 0x100000u) >> 23) - 2, 11);   // x 2^13 / S is x 2^n
  int rests = 0;
  float sum = -__builtin_ldexpf(__uint_as_float(top), n);
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const uint32_t two = w[i >> 2][i & 3];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const float x = __builtin_ldexpf(__uint_as_float(e == 0 ? two << 16 & 0x7FFFFFFFu : two & 0x7FFF0000u), n);
      rests += __builtin_amdgcn_fractf(x) != 0.f;
      sum += x;
    }
  }
  return top < 0x7F800000u && (float)(rests << 14) > sum;
}

// 16 keys (codes and scale byte kScale of `scales`) times 16 query rows in pieces, the
// smallest first.
template <int kScale>
__device__ __forceinline__ f32x4 kvq_scores(u32x4 key, uint32_t scales, const u32x6 (&q)[3], int q_scales) {
  const i32x8 a = {(int)key[0], (int)key[1], (int)key[2], (int)key[3], 0, 0, 0, 0};
  auto piece = [&](const u32x6& w) __attribute__((always_inline)) {
    return i32x8{(int)w[0], (int)w[1], (int)w[2], (int)w[3], (int)w[4], (int)w[5], 0, 0};
  };
  f32x4 s = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, piece(q[2]), f32x4{}, 4, 2, kScale, (int)scales, 2, q_scales);
  s = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, piece(q[1]), s, 4, 2, kScale, (int)scales, 1, q_scales);
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, piece(q[0]), s, 4, 2, kScale, (int)scales, 0, q_scales);
}

// The dims as they are, all NaN where one is an infinity or a NaN: keys of zeros would make a
// NaN of an infinity, others not.
__device__ __forceinline__ void kvq_load_q(const uint16_t* p, bf16x8 (&q)[4]) {
  u32x4 w[4];
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    w[i] = ld_u32x4(p + 8 * i);
#pragma unroll
    for (int e = 0; e < 4; ++e) top = max(top, max(w[i][e] & 0x7FFF0000u, (w[i][e] << 16) & 0x7FFF0000u));
  }
  const uint32_t spoiled = top < 0x7F800000u ? 0u : 0x7FFF7FFFu;
#pragma unroll
  for (int i = 0; i < 4; ++i) q[i] = __builtin_bit_cast(bf16x8, w[i] | spoiled);
}

// 16 keys, converted, times bf16 query rows: exact products.  Element e of a lane's operands of
// product j is dim 32 (lane / 16) + 8 j + e.
template <int kNB>
__device__ __forceinline__ void kvq_scores_bf16(u32x4 codes, uint32_t scale, const bf16x8 (&q)[kNB][4], int kb,
                                                f32x4 (&x)[kNB][4]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t w = codes[j];
    const bf16x8 key = __builtin_bit_cast(bf16x8, kvq_values(w, scale));
#pragma unroll
    for (int nb = 0; nb < kNB; ++nb)
      x[nb][kb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(key, q[nb][j], j == 0 ? f32x4{} : x[nb][kb], 0, 0, 0);
  }
}

__device__ __forceinline__ float row4_max(float x) {         // over the lanes that share lane % 16, NaN if any is
  auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = vmax(__uint_as_float(r[0]), __uint_as_float(r[1]));
  r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return vmax(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float row4_sum(float x) {
  auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Of 8 codes those whose values no bf16 holds (4 and 6 under a scale byte of 253, 2 and more under
// 254: infinities), others 0.
__device__ __forceinline__ uint32_t kvq_beyond(uint32_t w, uint32_t scale) {
  const uint32_t two = w >> 2 & 0x11111111u;
  return w & (scale == 254 ? two : scale == 253 ? two & w >> 1 : 0u) * 15u;
}
// A key's infinities of one block of 32 dims, which stayed out of the product, where the row sees it.
__device__ __forceinline__ void kvq_add_beyond(f32x4 (&o)[8], bool sees, int block, u32x4 codes, int g) {
#pragma unroll
  for (int db = 0; db < 8; ++db) {                           // dims 16 db + 4 g + i
    if (db >> 1 != block || !sees) continue;
    const uint32_t lo = codes[2 * (db & 1)], hi = codes[2 * (db & 1) + 1];
    const uint32_t four = (g & 2 ? hi : lo) >> (16 * (g & 1));
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (four >> (4 * i) & 4) o[db][i] += four >> (4 * i) & 8 ? -INFINITY : INFINITY;
  }
}

constexpr int kKvqWaves = 4;
// How far (log2) scores may outgrow a row's offset before l and O are rescaled: weights
// then reach 2^8, which their rounding to bf16, relative as it is, does not notice.  Moved
// at every growth, some row of a wave moves in 45% of the tiles of 8K keys.  Where the
// waves split the rows no maximum is taken at all as long as the weights a lane has added up
// for a row come to no more than kKvqMost; where they split the keys, l and O are rescaled
// beyond kKvqMostOfKeys too.  A row's weights then never come to 2^18, and values below 2^110 to no
// infinite sum, over any number of keys.  An offset goes to the maximum, or beyond it by
// as many powers of two as bring the row's weights below 2^10.
constexpr float kKvqLag = 8.f, kKvqMostOfKeys = 8192.f, kKvqMost = 32768.f;
__device__ __forceinline__ float kvq_offset(float m, float top, float l) {
  return vmax(top, m + (float)max(__builtin_amdgcn_frexp_expf(row4_sum(l)) - 10, 0));
}
// Bytes of a key's bf16 values in LDS: 32 more than they take, so that the 8 keys x 32
// bytes of half a wave's transposed reads, and the 8 rows' chunks of a quarter's
// writes, lie in different banks.
constexpr int kKvqVRow = kHD * 2 + 32;
constexpr int kKvqHalf = 32 * kKvqVRow;      // 32 keys: one wave's LDS where the waves split the keys

typedef __attribute__((address_space(3))) float KvqStats[2][kKvqWaves][16];   // of 16 rows: m and l of each wave

// One tile of 64 keys as loaded: 16-key block kb, lane l key l % 16, block l / 16 of its dims.
struct KvqTile {
  u32x4 k[4], v[4];
  uint32_t ks[4], vs[4];
};

// Partial results of a tile's parts and their join by the one that counts itself last.
// The parts run on different XCDs, whose L2s do not see each other's ordinary stores
// before the launch ends: they are stored and loaded at device scope, counted once the
// stores are acknowledged, and nothing waits.  Sums are in the parts' order, whichever
// ends last.
struct KvqParts {
  __amdgpu_buffer_rsrc_t o, lse;             // of all parts: row n of the tile in part s is s * rows + n
};
__device__ __forceinline__ KvqParts kvq_parts(const KvqAttnArgs& a, const KvqItem& it, int rows) {
  return {__builtin_amdgcn_make_buffer_rsrc(a.part_o + (int64_t)it.part0 * kHD, (short)0, it.n_parts * rows * kHD * 4, 0x00020000),
          __builtin_amdgcn_make_buffer_rsrc(a.part_lse + it.part0, (short)0, it.n_parts * rows * 4, 0x00020000)};
}
constexpr uint32_t kKvqNoRow = 0x400000;     // a row beyond the resources: nothing is read
static_assert(kKvqMostJoin < (int)kKvqNoRow / 2, "rows of a tile's parts");

// Counts at counter c; true for the last of the tile's parts, which puts the counter back.
__device__ __forceinline__ bool kvq_arrive(const KvqAttnArgs& a, const KvqItem& it, int c) {
  int32_t* const cnt = a.count + it.counter + c;
  const bool last = __hip_atomic_fetch_add(cnt, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == it.n_parts - 1;
  if (last) __hip_atomic_store(cnt, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return last;
}

__device__ __forceinline__ int64_t kvq_out_row(const KvqAttnArgs& a, const KvqItem& it, int r) {
  const int row = it.row0 + r, tok = row / a.G;
  return (int64_t)(it.q_start + tok) * a.Hq + it.kvh * a.G + (row - tok * a.G);
}

// Rows first .. first + n - 1 (n up to 16) of a part whose block has them whole: thread (r, ch)
// has 8 dims of row first + r.  In the block that ends last every thread takes 8 dims of a
// row and every nsub-th part of it.
__device__ __forceinline__ void kvq_join(const KvqAttnArgs& a, const KvqItem& it, int rows, int first, int n, int r, int ch,
                                         f32x4 o0, f32x4 o1, float log2sum, lds_u8* lds) {
  const int tid = threadIdx.x;
  const KvqParts parts = kvq_parts(a, it, rows);
  __attribute__((address_space(3))) int32_t* const flag = (__attribute__((address_space(3))) int32_t*)lds;
  if (r < n) {
    const uint32_t at = (uint32_t)(it.part - it.part0 + first + r);
    part_st4(parts.o, at * (kHD * 4) + ch * 32, o0);
    part_st4(parts.o, at * (kHD * 4) + ch * 32 + 16, o1);
    if (ch == 0) part_st1(parts.lse, at * 4, 0, log2sum);
  }
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0x0070);                        // vmcnt(0): my stores are acknowledged
  __syncthreads();
  if (tid == 0) *flag = kvq_arrive(a, it, first >> 4);
  __syncthreads();
  if (*flag == 0) return;
  const int nsub = 16 / n, slot = tid >> 4, sub = slot / n, row = slot - sub * n;
  const bool mine = sub < nsub;
  float top = -INFINITY, den = 0.f;
  f32x4 num[2] = {};
  constexpr int kAhead = 4;
  for (int s0 = sub; s0 < it.n_parts && mine; s0 += kAhead * nsub) {
    f32x4 x[kAhead][2];
    float lse[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int s = s0 + k * nsub;
      const uint32_t at = s < it.n_parts ? (uint32_t)(s * rows + first + row) : kKvqNoRow;
      lse[k] = part_ld1(parts.lse, at * 4, 0);
      x[k][0] = part_ld4(parts.o, at * (kHD * 4) + ch * 32, 0);
      x[k][1] = part_ld4(parts.o, at * (kHD * 4) + ch * 32 + 16, 0);
    }
    float m = top;
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      if (s0 + k * nsub >= it.n_parts) lse[k] = -INFINITY;
      m = fmaxf(m, lse[k]);
    }
    const float off = m == -INFINITY ? 0.f : m;
    const float f = exp2f_fast(top - off);
    top = m;
    den *= f;
    num[0] *= f;
    num[1] *= f;
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const float w = exp2f_fast(lse[k] - off);
      den += w;
      num[0] += w * x[k][0];
      num[1] += w * x[k][1];
    }
  }
  typedef __attribute__((address_space(3))) float lds_f;
  lds_f* const red = (lds_f*)(lds + 64);                     // [slot][ch][10]
  if (nsub > 1) {
    lds_f* const my = red + tid * 10;
    my[0] = top;
    my[1] = den;
#pragma unroll
    for (int e = 0; e < 8; ++e) my[2 + e] = num[e >> 2][e & 3];
    __syncthreads();
    if (sub > 0) return;
    float all = top;
    for (int k = 1; k < nsub; ++k) all = fmaxf(all, red[((k * n + row) * 16 + ch) * 10]);
    const float off = all == -INFINITY ? 0.f : all;
    float f = exp2f_fast(top - off);
    den *= f;
    num[0] *= f;
    num[1] *= f;
    for (int k = 1; k < nsub; ++k) {
      const lds_f* const x = red + ((k * n + row) * 16 + ch) * 10;
      f = exp2f_fast(x[0] - off);
      den += f * x[1];
#pragma unroll
      for (int e = 0; e < 8; ++e) num[e >> 2][e & 3] += f * x[2 + e];
    }
    top = all;
  }
  if (!mine) return;
  const float inv = den == 0.f ? 0.f : 1.f / den;
  const int64_t orow = kvq_out_row(a, it, first + row);
  bf16x8 out;
#pragma unroll
  for (int e = 0; e < 8; ++e) out[e] = (__bf16)(num[e >> 2][e & 3] * inv);
  *(bf16x8*)(a.o + orow * kHD + 8 * ch) = out;
  if (a.lse != nullptr && ch == 0)
    a.lse[orow] = den == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(den)) * 0.69314718055994531f;
}

template <int P, int kNB>
__device__ __forceinline__ void kvq_split_keys(const KvqAttnArgs& a, const KvqItem& it, lds_u8* lds, KvqStats* stats_p) {
  static_assert(P == 16 || P == 32, "page size");
  auto& stats = *stats_p;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = lane >> 4, r16 = lane & 15;
  const int G = a.G, rows = min(it.q_len * G - it.row0, 16 * kNB);
  const int pre = it.kv_len - it.q_len;
  const int32_t pt_base = ld_uniform(a.indptr + it.seq);
  const int32_t pt_count = ld_uniform(a.indptr + it.seq + 1) - pt_base;
  lds_u8* const vbuf = lds + wave * kKvqHalf;

  // this wave's tiles
  constexpr int kKeys = 64;
  const int t_lo = it.kv_begin / kKeys, t_hi = (it.kv_end + kKeys - 1) / kKeys;
  const int per = (t_hi - t_lo + kKvqWaves - 1) / kKvqWaves;
  const int t0 = min(t_lo + wave * per, t_hi), t1 = min(t0 + per, t_hi);

  // slots of 64 pages from page pg0 on, one a lane; -1 where a page is missing or outside the pool
  bool bad = false;
  int pg0 = t0 * (kKeys / P);
  auto load_slots = [&]() __attribute__((always_inline)) {
    const int pg = pg0 + lane;
    const bool need = (int64_t)pg * P < min(it.kv_end, t1 * kKeys);
    int32_t s = need && pg < pt_count ? a.indices[pt_base + pg] : -1;
    s = s >= 0 && s < a.num_slots ? s : -1;
    bad |= need && s < 0;
    return s;
  };
  int32_t slots = load_slots();

  const uint32_t code_off = (uint32_t)(r16 * kKvqCodes + g * 16), scale_off = (uint32_t)(P * kKvqCodes + r16 * 4 + g);
  const int64_t page_bytes = (int64_t)P * kKvqRow, slot_bytes = a.Hkv * page_bytes;
  auto load_tile = [&](int t, KvqTile& x) __attribute__((always_inline)) {
    if (t * (kKeys / P) - pg0 >= 64) {
      pg0 = t * (kKeys / P);
      slots = load_slots();
    }
#pragma unroll
    for (int kb = 0; kb < 4; ++kb) {
      const int32_t s = __builtin_amdgcn_readlane(slots, t * (kKeys / P) - pg0 + kb * 16 / P);
      constexpr int kIn[4] = {0, 16 % P, 32 % P, 48 % P};    // the block's first row in its page
      const KvqPage k = kvq_page(a.k, s, slot_bytes, it.kvh * page_bytes, page_bytes);
      const KvqPage v = kvq_page(a.v, s, slot_bytes, it.kvh * page_bytes, page_bytes);
      x.k[kb] = kvq_load_codes(k, code_off + kIn[kb] * kKvqCodes);
      x.v[kb] = kvq_load_codes(v, code_off + kIn[kb] * kKvqCodes);
      x.ks[kb] = kvq_load_scale(k, scale_off + kIn[kb] * 4);
      x.vs[kb] = kvq_load_scale(v, scale_off + kIn[kb] * 4);
    }
  };
  const int tr_at = (4 * g + (r16 >> 2)) * kKvqVRow + 8 * (r16 & 3);   // this lane's source of a transposed read
  KvqTile now, next;
  if (t0 < t1) load_tile(t0, now);

  // every wave holds the same rows: row r16 of each 16-row block, dims 32 g on
  bf16x8 q[kNB][4];
  int limit[kNB];
#pragma unroll
  for (int nb = 0; nb < kNB; ++nb) {
    const int rr = it.row0 + min(16 * nb + r16, rows - 1);
    const int tok = rr / G;
    const int head = it.kvh * G + (rr - tok * G);
    limit[nb] = min(it.kv_end, a.causal ? pre + tok + 1 : it.kv_len);
    kvq_load_q(a.q + ((int64_t)(it.q_start + tok) * a.Hq + head) * kHD + g * 32, q[nb]);
  }
  // keys below are seen by all rows
  const int all_see = min(it.kv_end, a.causal ? pre + it.row0 / G + 1 : it.kv_len);

  f32x4 o[kNB][8];                                           // dims 16 db + 4 g + i of row r16
  float m[kNB], l[kNB];
  uint32_t poison[kNB];                                      // blocks of 32 dims in which the row met a NaN value
#pragma unroll
  for (int nb = 0; nb < kNB; ++nb) {
    m[nb] = -INFINITY;
    l[nb] = 0.f;
    poison[nb] = 0;
#pragma unroll
    for (int db = 0; db < 8; ++db) o[nb][db] = f32x4{};
  }

  for (int t = t0; t < t1; ++t) {
    if (t + 1 < t1) load_tile(t + 1, next);
    const int key0 = t * kKeys;
    const bool masked = key0 + kKeys > all_see;
    if (masked) {
      // Values that no row sees are zeros; a NaN that some rows see is kept out of the
      // product, where it would reach the others, and put into those rows at the end, an
      // infinity added to them here.
#pragma unroll
      for (int kb = 0; kb < 4; ++kb) {
        const int key = key0 + 16 * kb + r16;
        if (key >= it.kv_end) {
          now.v[kb] = u32x4{};
          now.vs[kb] = 127;
        }
        for (uint64_t hit = __ballot(now.vs[kb] == 255); hit != 0; hit &= hit - 1) {
          const int from = __builtin_ctzll(hit);
#pragma unroll
          for (int nb = 0; nb < kNB; ++nb)
            if (key0 + 16 * kb + (from & 15) < limit[nb]) poison[nb] |= 1u << (from >> 4);
        }
        if (now.vs[kb] == 255) {
          now.v[kb] = u32x4{};
          now.vs[kb] = 127;
        }
        if (const uint64_t some = __ballot(now.vs[kb] > 252)) {
          u32x4 far;
#pragma unroll
          for (int j = 0; j < 4; ++j) far[j] = kvq_beyond(now.v[kb][j], now.vs[kb]);
          now.v[kb] ^= far;
          for (uint64_t hit = some; hit != 0; hit &= hit - 1) {
            const int from = __builtin_ctzll(hit);
            u32x4 codes;
#pragma unroll
            for (int j = 0; j < 4; ++j) codes[j] = (uint32_t)__builtin_amdgcn_readlane((int)far[j], from);
#pragma unroll
            for (int nb = 0; nb < kNB; ++nb)
              kvq_add_beyond(o[nb], key0 + 16 * kb + (from & 15) < limit[nb], from >> 4, codes, g);
          }
        }
      }
    }
    bf16x8 p[kNB][2];
    f32x4 x[kNB][4];
#pragma unroll
    for (int kb = 0; kb < 4; ++kb) kvq_scores_bf16(now.k[kb], now.ks[kb], q, kb, x);
#pragma unroll
    for (int nb = 0; nb < kNB; ++nb) {
      f32x4(&s)[4] = x[nb];
      if (masked) {
#pragma unroll
        for (int kb = 0; kb < 4; ++kb)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (key0 + 16 * kb + 4 * g + i >= limit[nb]) s[kb][i] = -INFINITY;
      }
      float top = s[0][0];
#pragma unroll
      for (int j = 1; j < 16; ++j) top = vmax(top, s[j >> 2][j & 3]);
      float grown = vmax(m[nb], row4_max(top) * a.c);
      if (__ballot(!(grown <= m[nb] + kKvqLag) | !(l[nb] <= kKvqMostOfKeys))) {
        grown = kvq_offset(m[nb], grown, l[nb]);
        // a row that had met no key has nothing but this tile's infinities
        const float f = m[nb] == -INFINITY ? 1.f : exp2f_fast(m[nb] - grown);
        l[nb] *= f;
#pragma unroll
        for (int db = 0; db < 8; ++db) o[nb][db] *= f;
        m[nb] = grown;
      }
      const float off = m[nb] == -INFINITY ? 0.f : m[nb];
#pragma unroll
      for (int kb = 0; kb < 4; ++kb)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float e = exp2f_fast(__builtin_fmaf(s[kb][i], a.c, -off));
          l[nb] += e;
          p[nb][kb >> 1][4 * (kb & 1) + i] = (__bf16)e;
        }
    }
    // O^T += V^T P^T, 32 keys at a time.  Element j of a lane's operands is key
    // 16 (j / 4) + 4 g + j % 4 of them.
#pragma unroll
    for (int half = 0; half < 2; ++half) {
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        const u32x4 w = now.v[2 * half + kb];
#pragma unroll
        for (int j = 0; j < 4; ++j)
          *(__attribute__((address_space(3))) u32x4*)(vbuf + (16 * kb + r16) * kKvqVRow + 64 * g + 16 * j) =
              kvq_values(w[j], now.vs[2 * half + kb]);
      }
#pragma unroll
      for (int db = 0; db < 8; ++db) {
        bf16x8 v;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
          const auto four = lds_read_tr(vbuf + tr_at + 16 * kb * kKvqVRow + 32 * db);
#pragma unroll
          for (int i = 0; i < 4; ++i) v[4 * kb + i] = four[i];
        }
#pragma unroll
        for (int nb = 0; nb < kNB; ++nb)
          o[nb][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, p[nb][half], o[nb][db], 0, 0, 0);
      }
    }
    now = next;
  }
  if (__ballot(bad) != 0 && lane == 0) atomicOr(a.err, 1);

  // the four waves' results, 16 rows at a time: each wave's rows in its own LDS
#pragma unroll
  for (int nb = 0; nb < kNB; ++nb) {
    if (nb > 0) __syncthreads();
#pragma unroll
    for (int db = 0; db < 8; ++db) {
      if (poison[nb] >> (db >> 1) & 1) o[nb][db] = f32x4{NAN, NAN, NAN, NAN};
      *(__attribute__((address_space(3))) f32x4*)(vbuf + r16 * (kHD * 4) + (((4 * db + g) ^ r16) << 4)) = o[nb][db];
    }
    l[nb] = row4_sum(l[nb]);
    if (g == 0) {
      stats[0][wave][r16] = m[nb];
      stats[1][wave][r16] = l[nb];
    }
    __syncthreads();
    const int r = tid >> 4, ch = tid & 15;                   // row, 8 dims
    float top = stats[0][0][r];
#pragma unroll
    for (int w = 1; w < kKvqWaves; ++w) top = vmax(top, stats[0][w][r]);
    const float off = top == -INFINITY ? 0.f : top;
    float den = 0.f;
    f32x4 num[2] = {};
#pragma unroll
    for (int w = 0; w < kKvqWaves; ++w) {
      const float f = exp2f_fast(stats[0][w][r] - off);
      den += f * stats[1][w][r];
#pragma unroll
      for (int i = 0; i < 2; ++i)
        num[i] += f * *(__attribute__((address_space(3))) f32x4*)(lds + w * kKvqHalf + r * (kHD * 4) + (((2 * ch + i) ^ r) << 4));
    }
    const float inv = den == 0.f ? 0.f : 1.f / den;
    const float log2sum = den == 0.f ? -INFINITY : top + __builtin_amdgcn_logf(den);
    if (it.counter >= 0) {
      __syncthreads();                                       // the waves' results have been read
      if (16 * nb < rows) kvq_join(a, it, rows, 16 * nb, min(16, rows - 16 * nb), r, ch, num[0] * inv, num[1] * inv, log2sum, lds);
      continue;
    }
    if (16 * nb + r >= rows) continue;
    if (it.part >= 0) {
      const int64_t at = (int64_t)it.part + 16 * nb + r;
      *(f32x4*)(a.part_o + at * kHD + 8 * ch) = num[0] * inv;
      *(f32x4*)(a.part_o + at * kHD + 8 * ch + 4) = num[1] * inv;
      if (ch == 0) a.part_lse[at] = log2sum;
    } else {
      const int64_t at = kvq_out_row(a, it, 16 * nb + r);
      bf16x8 out;
#pragma unroll
      for (int e = 0; e < 8; ++e) out[e] = (__bf16)(num[e >> 2][e & 3] * inv);
      *(bf16x8*)(a.o + at * kHD + 8 * ch) = out;
      if (a.lse != nullptr && ch == 0) a.lse[at] = log2sum * 0.69314718055994531f;
    }
  }
}

// Items of up to 64 kNB rows whose four waves hold 16 kNB rows each and go over the
// same keys together: the tile's values are converted once, a quarter by each wave.
//
// A step makes the scores of tile t + 1 while the probabilities of tile t are taken, and
// then O += P V of tile t while the values of t + 1 are converted: matrix and vector
// instructions of one wave, each independent of the other's.  Behind the barrier of step
// t - 1 LDS holds the values of tile t (bf16) and the keys of t + 1 (codes, or bf16); step t
// writes the values of t + 1 and the keys of t + 2 from registers, whose loads were issued
// a step before.
constexpr int kKvqTile = 64 * kKvqVRow;
constexpr int kKvqKRow = kHD * 2 + 16;       // a key's bf16 values: 16 rows' 16-byte chunks in all banks
template <bool kExact>
struct KvqRowsLds {                          // kExact: keys converted, for bf16 products; else codes
  uint8_t v[2][kKvqTile];
  uint8_t k[2][64 * (kExact ? kKvqKRow : kKvqCodes)];
  uint64_t nan[2][4];        // masked tiles: bit 16 g + r16 of a 16-key block, a value block that is NaN
  uint64_t some[2][4];       // the same, one that may hold infinities, and
  const uint8_t* page[2][4]; // the pages that those 16 keys lie in
  uint32_t ks[2][64];        // codes: lane (key r16, block g): the scale bytes of the four 16-key blocks
};

// Whether the item has a row for which pieces would not do: for all four waves, which share the
// keys' form in LDS.
template <int kNB>
__device__ __forceinline__ bool kvq_any_coarse(const KvqAttnArgs& a, const KvqItem& it,
                                               __attribute__((address_space(3))) int* votes) {
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 4, r16 = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rows = min(it.q_len * a.G - it.row0, 64 * kNB);
  bool coarse = false;
#pragma unroll
  for (int nb = 0; nb < kNB; ++nb) {
    const int rr = it.row0 + min(16 * kNB * wave + 16 * nb + r16, rows - 1), tok = rr / a.G;
    coarse |= kvq_coarse(a.q + ((int64_t)(it.q_start + tok) * a.Hq + it.kvh * a.G + (rr - tok * a.G)) * kHD + g * 32);
  }
  const bool any = __ballot(coarse) != 0;
  if (lane == 0) votes[wave] = any;
  __syncthreads();
  return __builtin_amdgcn_readfirstlane(votes[0] | votes[1] | votes[2] | votes[3]) != 0;
}

template <int P, int kNB, bool kExact>
__device__ __forceinline__ void kvq_split_rows(const KvqAttnArgs& a, const KvqItem& it,
                                               __attribute__((address_space(3))) KvqRowsLds<kExact>* lds) {
  static_assert(P == 16 || P == 32, "page size");
  constexpr int kTile = kKvqTile;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = lane >> 4, r16 = lane & 15;
  const int G = a.G, rows = min(it.q_len * G - it.row0, 64 * kNB);
  const int pre = it.kv_len - it.q_len;
  const int32_t pt_base = ld_uniform(a.indptr + it.seq);
  const int32_t pt_count = ld_uniform(a.indptr + it.seq + 1) - pt_base;
  constexpr int kKeys = 64;
  const int t0 = it.kv_begin / kKeys, t1 = (it.kv_end + kKeys - 1) / kKeys;
  // keys below are seen by all rows of the item
  const int all_see = min(it.kv_end, a.causal ? pre + it.row0 / G + 1 : it.kv_len);

  // This wave stages 16-key block `wave` of every tile; lane i has the slot of tile ts + i.
  // Keys run a tile or two ahead of values, so the values' slots follow the keys'.
  bool bad = false;
  auto load_slots = [&](int ts) __attribute__((always_inline)) {
    const int64_t key = (int64_t)(ts + lane) * kKeys + 16 * wave;
    const bool need = key < it.kv_end;
    const int pg = (int)(key / P);
    int32_t s = need && pg < pt_count ? a.indices[pt_base + pg] : -1;
    s = s >= 0 && s < a.num_slots ? s : -1;
    bad |= need && s < 0;
    return s;
  };
  int ts_k = t0, ts_v = t0;
  int32_t slots_k = load_slots(t0), slots_v = slots_k;
  // the slots of the keys of tile t and the values of tile t - 1 are at hand
  auto need_slots = [&](int t) __attribute__((always_inline)) {
    if (t - 1 - ts_v >= 64) {
      ts_v = ts_k;
      slots_v = slots_k;
    }
    if (t - ts_k >= 64) {
      ts_k = t;
      slots_k = load_slots(t);
    }
  };
  const int in = (16 * wave) % P;
  const uint32_t code_off = (uint32_t)((in + r16) * kKvqCodes + g * 16);
  const uint32_t scale_off = (uint32_t)(P * kKvqCodes + (in + r16) * 4 + g);
  const int64_t page_bytes = (int64_t)P * kKvqRow;
  struct Staged {
    u32x4 codes;
    uint32_t scale;
  };
  const int64_t slot_bytes = a.Hkv * page_bytes;
  auto load = [&](const uint8_t* pool, int32_t s, Staged& x) __attribute__((always_inline)) {
    const KvqPage page = kvq_page(pool, s, slot_bytes, it.kvh * page_bytes, page_bytes);
    x.codes = kvq_load_codes(page, code_off);
    x.scale = kvq_load_scale(page, scale_off);
  };
  auto load_k = [&](int t, Staged& x) __attribute__((always_inline)) {
    load(a.k, __builtin_amdgcn_readlane(slots_k, (t - ts_k) & 63), x);
  };
  auto load_v = [&](int t, Staged& x) __attribute__((always_inline)) {
    load(a.v, __builtin_amdgcn_readlane(slots_v, (t - ts_v) & 63), x);
  };
  lds_u8* const v0 = (lds_u8*)lds->v;
  lds_u8* const k0 = (lds_u8*)lds->k;
  auto put = [&](lds_u8* row, const Staged& x) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      *(__attribute__((address_space(3))) u32x4*)(row + 64 * g + 16 * j) = kvq_values(x.codes[j], x.scale);
  };
  auto put_k = [&](int b, const Staged& x) __attribute__((always_inline)) {
    lds_u8* const k = k0 + b * sizeof(lds->k[0]);
    if constexpr (kExact) {
      put(k + (16 * wave + r16) * kKvqKRow, x);
    } else {
      *(__attribute__((address_space(3))) u32x4*)(k + wave * 1024 + lane * 16) = x.codes;
      ((lds_u8*)lds->ks)[b * 256 + lane * 4 + wave] = (uint8_t)x.scale;
    }
  };
  auto put_v = [&](int b, const Staged& x) __attribute__((always_inline)) {
    put(v0 + b * kTile + (16 * wave + r16) * kKvqVRow, x);
  };
  // of a tile that is masked for some row: values that no row sees are zeros, and NaN
  // blocks and infinities, which would reach rows that do not see them, go round the product
  auto filter_v = [&](int t, int b, Staged& x) __attribute__((always_inline)) {
    if (t * kKeys + 16 * wave + r16 >= it.kv_end) x = Staged{u32x4{}, 127};
    const uint64_t hit = __ballot(x.scale == 255);
    if (lane == 0) lds->nan[b][wave] = hit;
    if (x.scale == 255) x = Staged{u32x4{}, 127};
    const uint64_t some = __ballot(x.scale > 252);
    if (lane == 0) lds->some[b][wave] = some;
    if (some != 0) {
      if (lane == 0)
        lds->page[b][wave] = a.v + __builtin_amdgcn_readlane(slots_v, (t - ts_v) & 63) * slot_bytes + it.kvh * page_bytes;
#pragma unroll
      for (int j = 0; j < 4; ++j) x.codes[j] ^= kvq_beyond(x.codes[j], x.scale);
    }
  };

  Staged kx, vx;
  if (t0 < t1) {
    load_k(t0, kx);
    load_v(t0, vx);
  }

  // this wave's rows: row r16 of each 16-row block, dims 32 g on
  const int wrow = 16 * kNB * wave;
  u32x6 pieces[kNB][3];
  bf16x8 q[kNB][4];
  int scales[kNB], limit[kNB];
#pragma unroll
  for (int nb = 0; nb < kNB; ++nb) {
    const int rr = it.row0 + min(wrow + 16 * nb + r16, rows - 1);
    const int tok = rr / G;
    const int head = it.kvh * G + (rr - tok * G);
    limit[nb] = min(it.kv_end, a.causal ? pre + tok + 1 : it.kv_len);
    const uint16_t* const row = a.q + ((int64_t)(it.q_start + tok) * a.Hq + head) * kHD + g * 32;
    if constexpr (kExact) kvq_load_q(row, q[nb]);
    else kvq_split_q(row, pieces[nb], scales[nb]);
  }
  const int wave_sees = min(it.kv_end, a.causal ? pre + (it.row0 + min(wrow, rows - 1)) / G + 1 : it.kv_len);

  f32x4 o[kNB][8];
  float m[kNB], l[kNB], off[kNB], most[kNB];   // off: m, or 0 where the row has met no key
  uint32_t poison[kNB];
#pragma unroll
  for (int nb = 0; nb < kNB; ++nb) {
    m[nb] = -INFINITY;
    l[nb] = 0.f;
    off[nb] = 0.f;
    most[nb] = -1.f;
    poison[nb] = 0;
#pragma unroll
    for (int db = 0; db < 8; ++db) o[nb][db] = f32x4{};
  }

  auto scores = [&](int b, f32x4 (&x)[kNB][4]) __attribute__((always_inline)) {
    if constexpr (kExact) {
      const lds_u8* const k = k0 + b * sizeof(lds->k[0]) + r16 * kKvqKRow + 64 * g;
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int kb = 0; kb < 4; ++kb) {
          const bf16x8 key = *(const __attribute__((address_space(3))) bf16x8*)(k + 16 * kb * kKvqKRow + 16 * j);
#pragma unroll
          for (int nb = 0; nb < kNB; ++nb)
            x[nb][kb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(key, q[nb][j], j == 0 ? f32x4{} : x[nb][kb], 0, 0, 0);
        }
    } else {
      const uint32_t ks = lds->ks[b][lane];
      const lds_u8* const k = k0 + b * sizeof(lds->k[0]) + lane * 16;
      u32x4 key[4];
#pragma unroll
      for (int kb = 0; kb < 4; ++kb) key[kb] = *(const __attribute__((address_space(3))) u32x4*)(k + kb * 1024);
#pragma unroll
      for (int nb = 0; nb < kNB; ++nb) {
        x[nb][0] = kvq_scores<0>(key[0], ks, pieces[nb], scales[nb]);
        x[nb][1] = kvq_scores<1>(key[1], ks, pieces[nb], scales[nb]);
        x[nb][2] = kvq_scores<2>(key[2], ks, pieces[nb], scales[nb]);
        x[nb][3] = kvq_scores<3>(key[3], ks, pieces[nb], scales[nb]);
      }
    }
  };
  // m, l and O moved to the maxima of a tile's scores
  auto settle = [&](const f32x4 (&x)[kNB][4]) __attribute__((always_inline)) {
#pragma unroll
    for (int nb = 0; nb < kNB; ++nb) {
      float top = x[nb][0][0];
#pragma unroll
      for (int j = 1; j < 16; ++j) top = vmax(top, x[nb][j >> 2][j & 3]);
      top = kvq_offset(m[nb], vmax(m[nb], row4_max(top) * a.c), l[nb]);
      const bool met = top != -INFINITY;
      off[nb] = met ? top : 0.f;
      most[nb] = met ? kKvqMost : -1.f;
      const float f = exp2f_fast(m[nb] - off[nb]);
      l[nb] *= f;
#pragma unroll
      for (int db = 0; db < 8; ++db) o[nb][db] *= f;
      m[nb] = top;
    }
  };
  // P of a tile's scores, from the offsets as they are.  Only where a lane's weights come to more than
  // kKvqMost, or its row has met no key, m, l and O are moved to the maxima and P is taken again: 34
  // vector instructions less in a step, which pays for c behind the product (measured together: 246 us for
  // 2048 rows x 4 heads behind 8K keys, 266 with maxima, 250 with c in the query).  ahead: the scores of the next
  // tile, which the compiler else moves behind the branch, away from the exponentials.
  auto weigh = [&](const f32x4 (&x)[kNB][4], bf16x8 (&p)[kNB][2], const f32x4 (*ahead)[4]) __attribute__((always_inline)) {
    float sum[kNB];
    auto weights = [&]() __attribute__((always_inline)) {
#pragma unroll
      for (int nb = 0; nb < kNB; ++nb) {
        float part[2] = {0.f, 0.f};
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          const float e = exp2f_fast(__builtin_fmaf(x[nb][j >> 2][j & 3], a.c, -off[nb]));
          part[j & 1] += e;
          p[nb][j >> 3][j & 7] = (__bf16)e;
        }
        sum[nb] = part[0] + part[1];
      }
    };
    weights();
    if (ahead != nullptr) {
#pragma unroll
      for (int nb = 0; nb < kNB; ++nb)
#pragma unroll
        for (int kb = 0; kb < 4; ++kb) asm volatile("" ::"v"(ahead[nb][kb]));
    }
    bool far = false;
#pragma unroll
    for (int nb = 0; nb < kNB; ++nb) far |= !(l[nb] + sum[nb] <= most[nb]);
    if (__ballot(far)) {
      settle(x);
      weights();
    }
#pragma unroll
    for (int nb = 0; nb < kNB; ++nb) l[nb] += sum[nb];
  };
  auto product = [&](int b, const bf16x8 (&p)[kNB][2]) __attribute__((always_inline)) {
    const lds_u8* const vt = v0 + b * kTile + (4 * g + (r16 >> 2)) * kKvqVRow + 8 * (r16 & 3);
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
      for (int db = 0; db < 8; ++db) {
        bf16x8 v;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
          const auto four = lds_read_tr(vt + (32 * half + 16 * kb) * kKvqVRow + 32 * db);
#pragma unroll
          for (int i = 0; i < 4; ++i) v[4 * kb + i] = four[i];
        }
#pragma unroll
        for (int nb = 0; nb < kNB; ++nb)
          o[nb][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, p[nb][half], o[nb][db], 0, 0, 0);
      }
  };
  auto mask = [&](int t, f32x4 (&x)[kNB][4]) __attribute__((always_inline)) {
#pragma unroll
    for (int nb = 0; nb < kNB; ++nb)
#pragma unroll
      for (int j = 0; j < 16; ++j)
        if (t * kKeys + 16 * (j >> 2) + 4 * g + (j & 3) >= limit[nb]) x[nb][j >> 2][j & 3] = -INFINITY;
  };

  f32x4 s[2][kNB][4];
  if (t0 < t1) {
    if ((t0 + 1) * kKeys > all_see) filter_v(t0, 0, vx);
    put_k(0, kx);
    put_v(0, vx);
    if (t0 + 1 < t1) load_k(t0 + 1, kx);
    lds_barrier();
    scores(0, s[0]);
    if ((t0 + 1) * kKeys > wave_sees) mask(t0, s[0]);
    settle(s[0]);
    if (t0 + 1 < t1) {
      put_k(1, kx);
      load_v(t0 + 1, vx);
      if (t0 + 2 < t1) load_k(t0 + 2, kx);
    }
    lds_barrier();
  }
  // steps whose tile and the next one all rows see: no branch but the slots' and the rescale's, so that the
  // compiler mixes their instructions; keys and values behind the item's last tile are loaded as zeros
  auto plain = [&](int t, auto buf) __attribute__((always_inline)) {
    constexpr int b = decltype(buf)::value;
    need_slots(t + 3);
    bf16x8 p[kNB][2];
    scores(b ^ 1, s[b ^ 1]);
    weigh(s[b], p, s[b ^ 1]);
    put_v(b ^ 1, vx);
    put_k(b, kx);
    load_v(t + 2, vx);
    load_k(t + 3, kx);
    product(b, p);
    lds_barrier();
  };
  int t = t0;
  for (const int end = min(t1, all_see / kKeys) - 1; t + 1 < end; t += 2) {
    plain(t, std::integral_constant<int, 0>{});
    plain(t + 1, std::integral_constant<int, 1>{});
  }
  for (; t < t1; ++t) {
    const int b = (t - t0) & 1;
    bf16x8 p[kNB][2];
    if (t + 1 < t1) scores(b ^ 1, s[1]);
    weigh(s[0], p, nullptr);
    product(b, p);
    if ((t + 1) * kKeys > all_see) {
#pragma unroll
      for (int kb = 0; kb < 4; ++kb)
        for (uint64_t hit = lds->nan[b][kb]; hit != 0; hit &= hit - 1) {
          const int from = __builtin_ctzll(hit);
#pragma unroll
          for (int nb = 0; nb < kNB; ++nb)
            if (t * kKeys + 16 * kb + (from & 15) < limit[nb]) poison[nb] |= 1u << (from >> 4);
        }
#pragma nounroll
      for (int kb = 0; kb < 4; ++kb)
        for (uint64_t hit = lds->some[b][kb]; hit != 0; hit &= hit - 1) {
          const int from = __builtin_ctzll(hit);
          const int row = (16 * kb) % P + (from & 15), block = from >> 4;
          const uint8_t* const page = lds->page[b][kb];
          const uint32_t scale = page[P * kKvqCodes + row * 4 + block];
          u32x4 codes = ld_u32x4((const uint16_t*)(page + row * kKvqCodes + block * 16));
#pragma unroll
          for (int j = 0; j < 4; ++j) codes[j] = kvq_beyond(codes[j], scale);
#pragma unroll
          for (int nb = 0; nb < kNB; ++nb)
            kvq_add_beyond(o[nb], t * kKeys + 16 * kb + (from & 15) < limit[nb], block, codes, g);
        }
    }
    if (t + 1 < t1) {
      if ((t + 2) * kKeys > all_see) filter_v(t + 1, b ^ 1, vx);
      put_v(b ^ 1, vx);
      if (t + 2 < t1) {
        put_k(b, kx);
        need_slots(t + 3);
        load_v(t + 2, vx);
        if (t + 3 < t1) load_k(t + 3, kx);
      }
      if ((t + 2) * kKeys > wave_sees) mask(t + 1, s[1]);
    }
#pragma unroll
    for (int nb = 0; nb < kNB; ++nb)
#pragma unroll
      for (int kb = 0; kb < 4; ++kb) s[0][nb][kb] = s[1][nb][kb];
    lds_barrier();
  }
  if (__ballot(bad) != 0 && lane == 0) atomicOr(a.err, 1);

  // this wave's rows: out, or as a part, which the wave that ends last joins with the others
  float log2sum[kNB];
#pragma unroll
  for (int nb = 0; nb < kNB; ++nb) {
    const float den = row4_sum(l[nb]);
    const float inv = den == 0.f ? 0.f : 1.f / den;
    log2sum[nb] = den == 0.f ? -INFINITY : m[nb] + __builtin_amdgcn_logf(den);
#pragma unroll
    for (int db = 0; db < 8; ++db)
      o[nb][db] = poison[nb] >> (db >> 1) & 1 ? f32x4{NAN, NAN, NAN, NAN} : o[nb][db] * inv;
  }
  if (wrow >= rows) return;
  if (it.counter >= 0) {
    const KvqParts parts = kvq_parts(a, it, rows);
#pragma unroll
    for (int nb = 0; nb < kNB; ++nb) {
      const int r = wrow + 16 * nb + r16;
      if (r >= rows) continue;
      const uint32_t at = (uint32_t)(it.part - it.part0 + r);
#pragma unroll
      for (int db = 0; db < 8; ++db) part_st4(parts.o, at * (kHD * 4) + db * 64 + g * 16, o[nb][db]);
      if (g == 0) part_st1(parts.lse, at * 4, 0, log2sum[nb]);
    }
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0070);                      // vmcnt(0): this wave's stores are acknowledged
    asm volatile("" ::: "memory");
    int last = 0;
    if (lane == 0) last = kvq_arrive(a, it, wave);
    if (__builtin_amdgcn_readfirstlane(last) == 0) return;
    asm volatile("" ::: "memory");
#pragma unroll
    for (int nb = 0; nb < kNB; ++nb) {
      const int r = wrow + 16 * nb + r16;
      const uint32_t row = r < rows ? (uint32_t)r : kKvqNoRow;
      float top = -INFINITY, den = 0.f;
      for (int s = 0; s < it.n_parts; ++s) top = fmaxf(top, part_ld1(parts.lse, (row + s * rows) * 4, 0));
      const float off = top == -INFINITY ? 0.f : top;
      f32x4 num[8] = {};
      for (int s = 0; s < it.n_parts; ++s) {
        const uint32_t at = row + s * rows;
        f32x4 x[8];
#pragma unroll
        for (int db = 0; db < 8; ++db) x[db] = part_ld4(parts.o, at * (kHD * 4) + db * 64 + g * 16, 0);
        const float w = exp2f_fast(part_ld1(parts.lse, at * 4, 0) - off);
        den += w;
#pragma unroll
        for (int db = 0; db < 8; ++db) num[db] += w * x[db];
      }
      const float inv = den == 0.f ? 0.f : 1.f / den;
      log2sum[nb] = den == 0.f ? -INFINITY : top + __builtin_amdgcn_logf(den);
#pragma unroll
      for (int db = 0; db < 8; ++db) o[nb][db] = num[db] * inv;
    }
  }
#pragma unroll
  for (int nb = 0; nb < kNB; ++nb) {
    const int r = wrow + 16 * nb + r16;
    if (r >= rows) continue;
    const bool part = it.part >= 0 && it.counter < 0;
    const int64_t at = part ? (int64_t)it.part + r : kvq_out_row(a, it, r);
#pragma unroll
    for (int db = 0; db < 8; ++db) {
      const f32x4 x = o[nb][db];
      if (part) *(f32x4*)(a.part_o + at * kHD + 16 * db + 4 * g) = x;
      else st_bf16x4(a.o + at * kHD + 16 * db + 4 * g, x[0], x[1], x[2], x[3]);
    }
    if (g == 0) {
      if (part) a.part_lse[at] = log2sum[nb];
      else if (a.lse != nullptr) a.lse[at] = log2sum[nb] * 0.69314718055994531f;
    }
  }
}

// Items of so few keys take bf16 products unasked: the vote's trip to memory is some 2 us.  Over
// 30 drawn batches with row tiles, against pieces without a vote: every item asked 1.12 times
// the time (1.27 at the worst), those of more than 256 keys 1.045, 512 1.035, 1024 1.041, 2048 1.05.
constexpr int kKvqShort = 512;
// Asked beforehand: a vote inside the loop's function, or both forms under one loop, cost the
// pieces' loop registers (64 and 85 spilled; 257 us for 2048 rows x 4 heads so, 415 else).
template <int P, int kNB>
__device__ __forceinline__ void kvq_rows(const KvqAttnArgs& a, const KvqItem& it, lds_u8* lds, KvqStats* stats) {
  if (it.kv_end - it.kv_begin <= kKvqShort || kvq_any_coarse<kNB>(a, it, (__attribute__((address_space(3))) int*)stats))
    kvq_split_rows<P, kNB, true>(a, it, (__attribute__((address_space(3))) KvqRowsLds<true>*)lds);
  else
    kvq_split_rows<P, kNB, false>(a, it, (__attribute__((address_space(3))) KvqRowsLds<false>*)lds);
}

// A launch of items of up to 16 rows alone: three blocks on a CU.
template <int P>
__global__ __launch_bounds__(256, 3) void attn_kvq_few_kernel(KvqAttnArgs a) {
  __shared__ __attribute__((aligned(1024))) uint8_t lds[kKvqWaves * kKvqHalf];
  __shared__ float stats[2][kKvqWaves][16];
  const KvqItem it = ld_uniform(a.items + blockIdx.x);
  kvq_split_keys<P, 1>(a, it, (lds_u8*)lds, (KvqStats*)stats);
}

// Items of every class (kvq_plan.h).
template <int P>
__global__ __launch_bounds__(256, 2) void attn_kvq_kernel(KvqAttnArgs a) {
  constexpr int kBytes = std::max<int>(std::max(sizeof(KvqRowsLds<false>), sizeof(KvqRowsLds<true>)), kKvqWaves * kKvqHalf);
  __shared__ __attribute__((aligned(1024))) uint8_t lds[kBytes];
  __shared__ float stats[2][kKvqWaves][16];
  const KvqItem it = ld_uniform(a.items + blockIdx.x);
  if (it.cls == 0) kvq_split_keys<P, 1>(a, it, (lds_u8*)lds, (KvqStats*)stats);
  else if (it.cls == 1) kvq_split_keys<P, 2>(a, it, (lds_u8*)lds, (KvqStats*)stats);
  else if (it.cls == 2) kvq_rows<P, 1>(a, it, (lds_u8*)lds, (KvqStats*)stats);
  else kvq_rows<P, 2>(a, it, (lds_u8*)lds, (KvqStats*)stats);
}

}  // namespace sa
