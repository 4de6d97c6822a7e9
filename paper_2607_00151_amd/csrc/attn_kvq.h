// Attention over a cache of 4 bits (sa_kvq_attn).
//
// Row i of a sequence sees keys j < limit_i (its position, or every key where there
// is no mask):
//   s_j = scale q . k_j,  m = max s_j,  O = sum 2^(s_j - m) v_j / l,  l = sum 2^(s_j - m)
// in the exp2 domain, in one pass with m, l and O carried and rescaled when m grows.
//
// Scores come out of the block-scaled matrix instruction (16x16x128), which takes
// the keys as they lie in the cache: lane l's operand is the 16 code bytes of key
// l % 16, block l / 16, with that block's scale byte, so a wave's load of 16 keys is
// one contiguous KB.  The query goes in as three 6-bit floats per value (e2m3, scales
// 2^e, 2^(e-4), 2^(e-8) per 32 dims, each the rounded rest of the one before), which
// together are the bf16 value to 2^-14 of its block's largest: against a bf16 product
// of converted keys the matrix work is 3/4 and the conversion goes, and two 8-bit
// pieces would cost 4/4 and lose 2^-14 in the instruction's sum (measured).
// Values have a scale per key and 32 dims, which a sum over keys cannot take in that
// instruction: they are converted to bf16 (exactly; 2 per v_cvt), laid out in LDS and
// read back transposed for the 16x16x32 bf16 product.  Probabilities are rounded to
// bf16 for it, as in attn_pipe.h; everything else is fp32.
//
// An item is up to 16 kNB packed rows of one KV head (row r: token r / G, head
// kvh G + r % G) over a range of keys.  Its four waves take a quarter of the keys
// each, with their own m, l, O and LDS and no barrier until the end; the next tile of
// 64 keys (8.7 KB) is in registers before the present one is computed.
#pragma once

#include "attn_pipe.h"
#include "kvq_kernels.h"
#include "kvq_plan.h"

namespace sa {

struct KvqAttnArgs {
  const uint16_t* q;
  const uint8_t* k;          // pools, offset to the layer
  const uint8_t* v;
  uint16_t* o;
  float* lse;                // nullable
  float* part_o;             // [part rows][kHD]
  float* part_lse;           // [part rows], log2
  const AttnItem* items;
  const int32_t* indptr;
  const int32_t* indices;
  int32_t* err;
  int32_t num_slots, Hq, Hkv, G;
  int32_t causal;
  float c;                   // softmax scale times log2 e
};

// What absent pages read as: codes and scale bytes of 0.
static __device__ uint8_t kvq_zero_page[32 * kKvqRow];

typedef uint32_t u32x6 __attribute__((ext_vector_type(6)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x32 __attribute__((ext_vector_type(32)));

// 32 dims of a query row as three 6-bit pieces; scales: their bytes (255: the block holds
// an infinity or a NaN).
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
  const int s = max((int)(top >> 23) - 2, 10);               // the block's largest is 4 to 8 times the scale
  bf16x32 x;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const bf16x2 two = __builtin_bit_cast(bf16x2, fine ? w[i][e] : 0u);
      x[8 * i + 2 * e] = two[0];
      x[8 * i + 2 * e + 1] = two[1];
    }
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    const float unit = __uint_as_float((uint32_t)(s - 4 * k) << 23);
    piece[k] = __builtin_bit_cast(u32x6, __builtin_amdgcn_cvt_scalef32_pk32_fp6_bf16(x, unit));
    if (k == 2) break;
    const bf16x32 back = __builtin_amdgcn_cvt_scalef32_pk32_bf16_fp6(__builtin_bit_cast(decltype(__builtin_amdgcn_cvt_scalef32_pk32_fp6_bf16(x, unit)), piece[k]), unit);
#pragma unroll
    for (int d = 0; d < 32; ++d) x[d] = (__bf16)((float)x[d] - (float)back[d]);   // exact: at most x's own bits are left
  }
  scales = fine ? s | (s - 4) << 8 | (s - 8) << 16 : 0xFFFFFF;
}

// S += 16 keys (codes and scale byte kScale of `scales`) times 16 query rows in pieces,
// the smallest first.
template <int kScale>
__device__ __forceinline__ f32x4 kvq_scores(u32x4 key, uint32_t scales, const u32x6 (&q)[3], int q_scales) {
  const i32x8 a = {(int)key[0], (int)key[1], (int)key[2], (int)key[3], 0, 0, 0, 0};
  f32x4 s{};
  auto piece = [&](const u32x6& w) __attribute__((always_inline)) {
    return i32x8{(int)w[0], (int)w[1], (int)w[2], (int)w[3], (int)w[4], (int)w[5], 0, 0};
  };
  s = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, piece(q[2]), s, 4, 2, kScale, (int)scales, 2, q_scales);
  s = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, piece(q[1]), s, 4, 2, kScale, (int)scales, 1, q_scales);
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, piece(q[0]), s, 4, 2, kScale, (int)scales, 0, q_scales);
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

constexpr int kKvqWaves = 4;
constexpr int kKvqHalf = 32 * kHD * 2;       // 32 keys of bf16 values: one wave's LDS

// One tile of 64 keys as loaded: 16-key block kb, lane l key l % 16, block l / 16 of its dims.
struct KvqTile {
  u32x4 k[4], v[4];
  uint32_t ks[4], vs[4];
};

template <int P, int kNB>
__global__ __launch_bounds__(256, kNB == 1 ? 3 : kNB == 2 ? 2 : 1) void attn_kvq_kernel(KvqAttnArgs a) {
  static_assert(P == 16 || P == 32, "page size");
  __shared__ __attribute__((aligned(1024))) uint8_t lds[kKvqWaves * kKvqHalf];
  __shared__ float stats[2][kKvqWaves][16];
  const AttnItem it = ld_uniform(a.items + blockIdx.x);
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = lane >> 4, r16 = lane & 15;
  const int G = a.G, rows = min(it.q_len * G - it.row0, 16 * kNB);
  const int pre = it.kv_len - it.q_len;
  const int32_t pt_base = ld_uniform(a.indptr + it.seq);
  const int32_t pt_count = ld_uniform(a.indptr + it.seq + 1) - pt_base;
  lds_u8* const vbuf = (lds_u8*)lds + wave * kKvqHalf;

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
  const int64_t page_bytes = (int64_t)P * kKvqRow;
  auto load_tile = [&](int t, KvqTile& x) __attribute__((always_inline)) {
    if (t * (kKeys / P) - pg0 >= 64) {
      pg0 = t * (kKeys / P);
      slots = load_slots();
    }
#pragma unroll
    for (int kb = 0; kb < 4; ++kb) {
      const int32_t s = __builtin_amdgcn_readlane(slots, t * (kKeys / P) - pg0 + kb * 16 / P);
      const int64_t at = ((int64_t)s * a.Hkv + it.kvh) * page_bytes;
      const uint8_t* const kp = s >= 0 ? a.k + at : kvq_zero_page;
      const uint8_t* const vp = s >= 0 ? a.v + at : kvq_zero_page;
      constexpr int kIn[4] = {0, 16 % P, 32 % P, 48 % P};    // the block's first row in its page
      x.k[kb] = *(const u32x4*)(kp + code_off + kIn[kb] * kKvqCodes);
      x.v[kb] = *(const u32x4*)(vp + code_off + kIn[kb] * kKvqCodes);
      x.ks[kb] = kp[scale_off + kIn[kb] * 4];
      x.vs[kb] = vp[scale_off + kIn[kb] * 4];
    }
  };
  KvqTile now, next;
  if (t0 < t1) load_tile(t0, now);

  // every wave holds the same rows: row r16 of each 16-row block, dims 32 g on
  u32x6 q[kNB][3];
  int qs[kNB], limit[kNB];
#pragma unroll
  for (int nb = 0; nb < kNB; ++nb) {
    const int rr = it.row0 + min(16 * nb + r16, rows - 1);
    const int tok = rr / G;
    const int head = it.kvh * G + (rr - tok * G);
    limit[nb] = min(it.kv_end, a.causal ? pre + tok + 1 : it.kv_len);
    kvq_split_q(a.q + ((int64_t)(it.q_start + tok) * a.Hq + head) * kHD + g * 32, q[nb], qs[nb]);
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
      // product, where it would reach the others, and put into those rows at the end.
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
      }
    }
    bf16x8 p[kNB][2];
#pragma unroll
    for (int nb = 0; nb < kNB; ++nb) {
      f32x4 s[4];
#pragma unroll
      for (int kb = 0; kb < 4; ++kb) {
        s[kb] = kvq_scores<0>(now.k[kb], now.ks[kb], q[nb], qs[nb]);
      }
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
      const float grown = vmax(m[nb], row4_max(top) * a.c);
      if (__ballot(!(grown == m[nb]))) {
        const float f = exp2f_fast(m[nb] - (grown == -INFINITY ? 0.f : grown));
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
    // 16 (j / 4) + 4 g + j % 4 of them.  16-byte chunks of an LDS row are XORed by its
    // key, so that a column of 16 rows' chunks, and the transposed reads of 16 rows x 32
    // bytes, touch every bank alike.
#pragma unroll
    for (int half = 0; half < 2; ++half) {
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        const u32x4 w = now.v[2 * half + kb];
        lds_u8* const row = vbuf + (16 * kb + r16) * (kHD * 2);
#pragma unroll
        for (int j = 0; j < 4; ++j)
          *(__attribute__((address_space(3))) u32x4*)(row + (((4 * g + j) ^ r16) << 4)) = kvq_values(w[j], now.vs[2 * half + kb]);
      }
      const int tr_key = 4 * g + (r16 >> 2);
#pragma unroll
      for (int db = 0; db < 8; ++db) {
        bf16x8 v;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
          const auto four = lds_read_tr(vbuf + (16 * kb + tr_key) * (kHD * 2) + (((2 * db + ((r16 >> 1) & 1)) ^ tr_key) << 4) +
                                    (r16 & 1) * 8);
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
    if (16 * nb + r >= rows) continue;
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
        num[i] += f * *(__attribute__((address_space(3))) f32x4*)((lds_u8*)lds + w * kKvqHalf + r * (kHD * 4) + (((2 * ch + i) ^ r) << 4));
    }
    const float inv = den == 0.f ? 0.f : 1.f / den;
    const float log2sum = den == 0.f ? -INFINITY : top + __builtin_amdgcn_logf(den);
    if (it.part >= 0) {
      const int64_t at = (int64_t)it.part + 16 * nb + r;
      *(f32x4*)(a.part_o + at * kHD + 8 * ch) = num[0] * inv;
      *(f32x4*)(a.part_o + at * kHD + 8 * ch + 4) = num[1] * inv;
      if (ch == 0) a.part_lse[at] = log2sum;
    } else {
      const int row = it.row0 + 16 * nb + r, tok = row / G;
      const int64_t at = (int64_t)(it.q_start + tok) * a.Hq + it.kvh * G + (row - tok * G);
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
// A step makes the scores of tile t + 1 while the probabilities of tile t are taken,
// and then O += P V of tile t with the row maxima of t + 1: matrix and vector
// instructions of one wave, each independent of the other's.  Behind the barrier of
// step t - 1 LDS holds the values of tile t (bf16) and the codes of the keys of t + 1;
// step t writes the values of t + 1 and the keys of t + 2 from registers, whose
// loads were issued a step before.
template <int P, int kNB>
__global__ __launch_bounds__(256, 2) void attn_kvq_rows_kernel(KvqAttnArgs a) {
  static_assert(P == 16 || P == 32, "page size");
  constexpr int kTile = 64 * kHD * 2, kKeyBytes = 64 * kKvqCodes;
  __shared__ __attribute__((aligned(1024))) uint8_t v_lds[2][kTile];
  __shared__ __attribute__((aligned(1024))) uint8_t k_lds[2][kKeyBytes];
  __shared__ uint32_t ks_lds[2][64];           // lane (key r16, block g): the scale bytes of the four 16-key blocks
  __shared__ uint64_t nan_lds[2][4];           // masked tiles: bit 16 g + r16 of a 16-key block, a value block that is NaN
  const AttnItem it = ld_uniform(a.items + blockIdx.x);
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

  // this wave stages 16-key block `wave` of every tile; lane i has the slot of tile ts + i
  bool bad = false;
  int ts = t0;
  auto load_slots = [&]() __attribute__((always_inline)) {
    const int64_t key = (int64_t)(ts + lane) * kKeys + 16 * wave;
    const bool need = key < it.kv_end;
    const int pg = (int)(key / P);
    int32_t s = need && pg < pt_count ? a.indices[pt_base + pg] : -1;
    s = s >= 0 && s < a.num_slots ? s : -1;
    bad |= need && s < 0;
    return s;
  };
  int32_t slots = load_slots();
  int ts_next = ts;                            // tiles ask for their slots in order, keys two before values
  int32_t slots_next = slots;
  const int in = (16 * wave) % P;
  const uint32_t code_off = (uint32_t)((in + r16) * kKvqCodes + g * 16);
  const uint32_t scale_off = (uint32_t)(P * kKvqCodes + (in + r16) * 4 + g);
  const int64_t page_bytes = (int64_t)P * kKvqRow;
  struct Staged {
    u32x4 codes;
    uint32_t scale;
  };
  auto load = [&](const uint8_t* pool, int32_t s, Staged& x) __attribute__((always_inline)) {
    const uint8_t* const p = s >= 0 ? pool + ((int64_t)s * a.Hkv + it.kvh) * page_bytes : kvq_zero_page;
    x.codes = *(const u32x4*)(p + code_off);
    x.scale = p[scale_off];
  };
  // keys run ahead of values: their slots are refilled first, the values' follow when they get there
  auto load_k = [&](int t, Staged& x) __attribute__((always_inline)) {
    if (t - ts_next >= 64) {
      ts = ts_next = t;
      slots_next = load_slots();
    }
    load(a.k, __builtin_amdgcn_readlane(slots_next, (t - ts_next) & 63), x);
  };
  int ts_v = t0;
  auto load_v = [&](int t, Staged& x) __attribute__((always_inline)) {
    if (t - ts_v >= 64) {
      ts_v = ts_next;
      slots = slots_next;
    }
    load(a.v, __builtin_amdgcn_readlane(slots, (t - ts_v) & 63), x);
  };
  lds_u8* const v0 = (lds_u8*)v_lds;
  lds_u8* const k0 = (lds_u8*)k_lds;
  auto put_k = [&](int b, const Staged& x) __attribute__((always_inline)) {
    *(__attribute__((address_space(3))) u32x4*)(k0 + b * kKeyBytes + wave * 1024 + lane * 16) = x.codes;
    ((lds_u8*)ks_lds)[b * 256 + lane * 4 + wave] = (uint8_t)x.scale;
  };
  auto put_v = [&](int t, int b, Staged x) __attribute__((always_inline)) {
    if ((t + 1) * kKeys > all_see) {
      // values that no row sees are zeros; NaN blocks that some rows see go round the product
      if (t * kKeys + 16 * wave + r16 >= it.kv_end) x = Staged{u32x4{}, 127};
      const uint64_t hit = __ballot(x.scale == 255);
      if (lane == 0) nan_lds[b][wave] = hit;
      if (x.scale == 255) x = Staged{u32x4{}, 127};
    }
    lds_u8* const row = v0 + b * kTile + (16 * wave + r16) * (kHD * 2);
#pragma unroll
    for (int j = 0; j < 4; ++j)
      *(__attribute__((address_space(3))) u32x4*)(row + (((4 * g + j) ^ r16) << 4)) = kvq_values(x.codes[j], x.scale);
  };

  Staged kx, vx;
  if (t0 < t1) {
    load_k(t0, kx);
    load_v(t0, vx);
  }

  // this wave's rows: row r16 of each 16-row block, dims 32 g on
  const int wrow = 16 * kNB * wave;
  u32x6 q[kNB][3];
  int qs[kNB], limit[kNB];
#pragma unroll
  for (int nb = 0; nb < kNB; ++nb) {
    const int rr = it.row0 + min(wrow + 16 * nb + r16, rows - 1);
    const int tok = rr / G;
    const int head = it.kvh * G + (rr - tok * G);
    limit[nb] = min(it.kv_end, a.causal ? pre + tok + 1 : it.kv_len);
    kvq_split_q(a.q + ((int64_t)(it.q_start + tok) * a.Hq + head) * kHD + g * 32, q[nb], qs[nb]);
  }
  const int wave_sees = min(it.kv_end, a.causal ? pre + (it.row0 + min(wrow, rows - 1)) / G + 1 : it.kv_len);

  f32x4 o[kNB][8];
  float m[kNB], l[kNB];
  uint32_t poison[kNB];
#pragma unroll
  for (int nb = 0; nb < kNB; ++nb) {
    m[nb] = -INFINITY;
    l[nb] = 0.f;
    poison[nb] = 0;
#pragma unroll
    for (int db = 0; db < 8; ++db) o[nb][db] = f32x4{};
  }

  f32x4 s[kNB][4];
  auto scores = [&](int b, f32x4 (&x)[kNB][4]) __attribute__((always_inline)) {
    const uint32_t scales = ((__attribute__((address_space(3))) uint32_t*)ks_lds)[b * 64 + lane];
    const lds_u8* const k = k0 + b * kKeyBytes + lane * 16;
    u32x4 key[4];
#pragma unroll
    for (int kb = 0; kb < 4; ++kb) key[kb] = *(const __attribute__((address_space(3))) u32x4*)(k + kb * 1024);
#pragma unroll
    for (int nb = 0; nb < kNB; ++nb) {
      x[nb][0] = kvq_scores<0>(key[0], scales, q[nb], qs[nb]);
      x[nb][1] = kvq_scores<1>(key[1], scales, q[nb], qs[nb]);
      x[nb][2] = kvq_scores<2>(key[2], scales, q[nb], qs[nb]);
      x[nb][3] = kvq_scores<3>(key[3], scales, q[nb], qs[nb]);
    }
  };
  // m, l and O moved to the maxima of new scores
  auto settle = [&](const float (&top)[kNB]) __attribute__((always_inline)) {
    float grown[kNB];
    bool moves = false;
#pragma unroll
    for (int nb = 0; nb < kNB; ++nb) {
      grown[nb] = vmax(m[nb], row4_max(top[nb]) * a.c);
      moves |= !(grown[nb] == m[nb]);
    }
    if (__ballot(moves)) {
#pragma unroll
      for (int nb = 0; nb < kNB; ++nb) {
        const float f = exp2f_fast(m[nb] - (grown[nb] == -INFINITY ? 0.f : grown[nb]));
        l[nb] *= f;
#pragma unroll
        for (int db = 0; db < 8; ++db) o[nb][db] *= f;
        m[nb] = grown[nb];
      }
    }
  };
  auto maxima = [&](const f32x4 (&x)[kNB][4], float (&top)[kNB]) __attribute__((always_inline)) {
#pragma unroll
    for (int nb = 0; nb < kNB; ++nb) {
      top[nb] = x[nb][0][0];
#pragma unroll
      for (int j = 1; j < 16; ++j) top[nb] = vmax(top[nb], x[nb][j >> 2][j & 3]);
    }
  };
  auto mask = [&](int t, f32x4 (&x)[kNB][4]) __attribute__((always_inline)) {
#pragma unroll
    for (int nb = 0; nb < kNB; ++nb)
#pragma unroll
      for (int j = 0; j < 16; ++j)
        if (t * kKeys + 16 * (j >> 2) + 4 * g + (j & 3) >= limit[nb]) x[nb][j >> 2][j & 3] = -INFINITY;
  };

  if (t0 < t1) {
    put_k(0, kx);
    put_v(t0, 0, vx);
    if (t0 + 1 < t1) load_k(t0 + 1, kx);
    lds_barrier();
    scores(0, s);
    if ((t0 + 1) * kKeys > wave_sees) mask(t0, s);
    float top[kNB];
    maxima(s, top);
    settle(top);
    if (t0 + 1 < t1) {
      put_k(1, kx);
      load_v(t0 + 1, vx);
      if (t0 + 2 < t1) load_k(t0 + 2, kx);
    }
    lds_barrier();
  }
  for (int t = t0; t < t1; ++t) {
    const int b = (t - t0) & 1;
    // scores of the next tile (of whatever LDS holds behind the last one: not used)
    f32x4 s_next[kNB][4];
    scores(b ^ 1, s_next);
    bf16x8 p[kNB][2];
#pragma unroll
    for (int nb = 0; nb < kNB; ++nb) {
      const float off = m[nb] == -INFINITY ? 0.f : m[nb];
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        const float e = exp2f_fast(__builtin_fmaf(s[nb][j >> 2][j & 3], a.c, -off));
        l[nb] += e;
        p[nb][j >> 3][j & 7] = (__bf16)e;
      }
    }
    const lds_u8* const vt = v0 + b * kTile;
    const int tr_key = 4 * g + (r16 >> 2);
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
      for (int db = 0; db < 8; ++db) {
        bf16x8 v;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
          const auto four = lds_read_tr(vt + (32 * half + 16 * kb + tr_key) * (kHD * 2) +
                                        (((2 * db + ((r16 >> 1) & 1)) ^ tr_key) << 4) + (r16 & 1) * 8);
#pragma unroll
          for (int i = 0; i < 4; ++i) v[4 * kb + i] = four[i];
        }
#pragma unroll
        for (int nb = 0; nb < kNB; ++nb)
          o[nb][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, p[nb][half], o[nb][db], 0, 0, 0);
      }
    if ((t + 1) * kKeys > all_see) {
#pragma unroll
      for (int kb = 0; kb < 4; ++kb)
        for (uint64_t hit = nan_lds[b][kb]; hit != 0; hit &= hit - 1) {
          const int from = __builtin_ctzll(hit);
#pragma unroll
          for (int nb = 0; nb < kNB; ++nb)
            if (t * kKeys + 16 * kb + (from & 15) < limit[nb]) poison[nb] |= 1u << (from >> 4);
        }
    }
    if (t + 1 < t1) {
      put_v(t + 1, b ^ 1, vx);
      if (t + 2 < t1) {
        put_k(b, kx);
        load_v(t + 2, vx);
        if (t + 3 < t1) load_k(t + 3, kx);
      }
      if ((t + 2) * kKeys > wave_sees) mask(t + 1, s_next);
      float top[kNB];
      maxima(s_next, top);
      settle(top);
    }
#pragma unroll
    for (int nb = 0; nb < kNB; ++nb)
#pragma unroll
      for (int kb = 0; kb < 4; ++kb) s[nb][kb] = s_next[nb][kb];
    lds_barrier();
  }
  if (__ballot(bad) != 0 && lane == 0) atomicOr(a.err, 1);

#pragma unroll
  for (int nb = 0; nb < kNB; ++nb) {
    const int r = wrow + 16 * nb + r16;
    const float den = row4_sum(l[nb]);
    if (r >= rows) continue;
    const float inv = den == 0.f ? 0.f : 1.f / den;
    const float log2sum = den == 0.f ? -INFINITY : m[nb] + __builtin_amdgcn_logf(den);
    const int row = it.row0 + r, tok = row / G;
    const int64_t at = it.part >= 0 ? (int64_t)it.part + r : (int64_t)(it.q_start + tok) * a.Hq + it.kvh * G + (row - tok * G);
#pragma unroll
    for (int db = 0; db < 8; ++db) {
      f32x4 x = o[nb][db] * inv;
      if (poison[nb] >> (db >> 1) & 1) x = f32x4{NAN, NAN, NAN, NAN};
      if (it.part >= 0) *(f32x4*)(a.part_o + at * kHD + 16 * db + 4 * g) = x;
      else st_bf16x4(a.o + at * kHD + 16 * db + 4 * g, x[0], x[1], x[2], x[3]);
    }
    if (g == 0) {
      if (it.part >= 0) a.part_lse[at] = log2sum;
      else if (a.lse != nullptr) a.lse[at] = log2sum * 0.69314718055994531f;
    }
  }
}

}  // namespace sa
