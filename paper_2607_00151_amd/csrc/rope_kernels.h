// Append of a segment's rows with the norms of its query and key heads and
// their rotation by position (sa_kv_append_rope).
//
// For one head row x of 128 values, weights w and pairs (i, j) of dims with
// angle a = pos * inv_freq:
//   y = x * rsqrt(mean x^2 + eps) * (w + offset)          (where there are weights)
//   (y_i, y_j) <- (y_i cos a - y_j sin a, y_j cos a + y_i sin a)
// in fp32, rounded once to bf16.
//
// Angles: a position can be millions and inv_freq 1, where an fp32 product is
// off by whole turns.  Frequencies are therefore kept in turns per position as
// 64-bit binary fractions; position times fraction modulo 2^64 is the exact
// phase (one integer multiply), of which the top 32 bits, signed, go to fp32 and
// to v_sin / v_cos, whose arguments are turns.
//
// Bytes are the floor (2 * 256 per head row, read and written once), but at 16
// lanes of 16 bytes a row the vector instructions per row come close behind, so
// everything that depends only on token and dim is made once per wave: with
// G = w + offset, r = rsqrt(...) and the partner's value p (of the same row)
//   out = r * (x * (G cos) + p * (+-G' sin)),
// the two products per dim of one token, for query and for key heads.  A wave
// takes 16 head rows at a time of one token, the next 16 in flight, for as many
// rounds as leave the chip enough waves; the sum of squares is a 4-step DPP
// reduction within a row's 16 lanes.  40.7K tokens of 48 head rows (1.0 GB): 237 us
// with everything per row, 190 so, 175 (5.7 TB/s) with kStream; 64 tokens 5 us.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "common.h"
#include "kvq_kernels.h"
#include "kv_kernels.h"
#include "plan.h"

namespace sa {

struct RopeArgs {
  const uint16_t* q;         // token t, head h at t * q_stride + h * 128
  const uint16_t* k;
  const uint16_t* v;
  int64_t q_stride, k_stride, v_stride;
  uint16_t* q_out;           // [T][Hq][128]
  uint16_t* k_pool;          // offset to the layer
  uint16_t* v_pool;
  uint8_t* kq_pool;          // the same of 4 bits
  uint8_t* vq_pool;
  const uint16_t* q_weight;  // [128] or null
  const uint16_t* k_weight;
  const int32_t* tok_begin;  // [B + 1]
  const int32_t* start;      // [B] cache position of each sequence's first new token
  const int32_t* pos;        // [B] its position for the rotation
  const int32_t* indptr;
  const int32_t* indices;
  int32_t* err;
  int64_t num_slots;
  int32_t T, B, Hq, Hkv, P;
  int32_t rot;
  int32_t rounds;            // rounds of kRopeRows head rows per wave
  float eps, offset;
  const uint64_t* freq;      // [rot / 2] turns per position, as fractions of 2^64
  const int32_t* axis;       // [rot / 2] axis of each pair, and
  const int32_t* axis_pos;   // the tokens' positions on axis i from i * axis_stride on
  int64_t axis_stride;
  int32_t num_axes;
};

constexpr int kRopeRows = 16;        // head rows of a round: 4 loads of 16 bytes per lane

// Largest b with tok_begin[b] <= t, by the whole wave: 64 probes per round.
__device__ __forceinline__ int wave_find_seq(const int32_t* tok_begin, int B, int t) {
  const int lane = threadIdx.x & 63;
  int lo = 0, n = B;                                        // answer in [lo, lo + n)
  while (n > 1) {
    const int step = (n + 63) >> 6;
    const int i = lo + lane * step;
    const bool at_most = i < lo + n && tok_begin[i] <= t;
    const int k = __popcll(__ballot(at_most)) - 1;          // offsets ascend: the hits are a prefix of the lanes
    lo += k * step;
    n = min(step, n - k * step);
  }
  return lo;
}

// Sine and cosine of a phase in fractions of 2^64 of a turn, to some 2^-45: the nearest
// quarter turn goes by symmetry, the rest, up to an eighth, by the Taylor series up to the
// 13th and 14th power.
__device__ __forceinline__ void turn_sincos(uint64_t phase, double& sine, double& cosine) {
  const uint32_t quarter = (uint32_t)((phase + (uint64_t(1) << 61)) >> 62);
  const double a = (double)(int64_t)(phase - ((uint64_t)quarter << 62)) * 3.4061215800304785e-19;   // 2 pi / 2^64
  const double x = a * a;
  double s = __builtin_fma(x, 1. / 6227020800., -1. / 39916800.);
  s = __builtin_fma(x, s, 1. / 362880.);
  s = __builtin_fma(x, s, -1. / 5040.);
  s = __builtin_fma(x, s, 1. / 120.);
  s = __builtin_fma(x, s, -1. / 6.);
  s = __builtin_fma(a * x, s, a);
  double c = __builtin_fma(x, -1. / 87178291200., 1. / 479001600.);
  c = __builtin_fma(x, c, -1. / 3628800.);
  c = __builtin_fma(x, c, 1. / 40320.);
  c = __builtin_fma(x, c, -1. / 720.);
  c = __builtin_fma(x, c, 1. / 24.);
  c = __builtin_fma(x, c, -0.5);
  c = __builtin_fma(x, c, 1.);
  sine = quarter & 1 ? c : s;
  cosine = quarter & 1 ? s : c;
  if (quarter & 2) sine = -sine;
  if ((quarter + 1) & 2) cosine = -cosine;
}

typedef double f64x2 __attribute__((ext_vector_type(2)));

template <int kCtrl>
__device__ __forceinline__ float row16(float x) {
  return __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(x), kCtrl, 0xF, 0xF, true));
}
template <int kCtrl>
__device__ __forceinline__ uint32_t row16u(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_mov_dpp((int)x, kCtrl, 0xF, 0xF, true);
}
// over the 16 lanes that share lane / 16
__device__ __forceinline__ float row16_sum(float x) {
  x += row16<0xB1>(x);       // lane ^ 1
  x += row16<0x4E>(x);       // lane ^ 2
  x += row16<0x124>(x);      // 4 lanes on
  x += row16<0x128>(x);      // 8 lanes on
  return x;
}
__device__ __forceinline__ double row16_sum(double x) {
  auto add = [&](auto ctrl) __attribute__((always_inline)) {
    const uint64_t w = __builtin_bit_cast(uint64_t, x);
    const uint64_t lo = row16u<decltype(ctrl)::value>((uint32_t)w), hi = row16u<decltype(ctrl)::value>((uint32_t)(w >> 32));
    x += __builtin_bit_cast(double, hi << 32 | lo);
  };
  add(std::integral_constant<int, 0xB1>{});
  add(std::integral_constant<int, 0x4E>{});
  add(std::integral_constant<int, 0x124>{});
  add(std::integral_constant<int, 0x128>{});
  return x;
}

// To fp32 with the last bit set where anything is cut off, so that no later rounding finds
// a tie that is none.
__device__ __forceinline__ float rounded_to_odd(double z) {
  const float f = (float)z;
  const double rest = z - (double)f;
  const uint32_t w = __float_as_uint(f);
  const bool odd = (w & 1) != 0 || rest == 0. || f == 0.f || !(fabsf(f) < INFINITY);
  return odd ? f : __uint_as_float((rest > 0.) == (f > 0.f) ? w + 1 : w - 1);
}

// out = r (x own + p other), p the pair's other value
struct RopeCoef {
  float own[8], other[8];
  bool normed;
};

__device__ __forceinline__ void unpack8(u32x4 w, float (&x)[8]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    x[2 * e] = __uint_as_float(w[e] << 16);
    x[2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u);
  }
}

// kPair: where a dim's partner is -- in the same lane (dims 2d, 2d + 1), 8 lanes
// on (d, d + 64: a DPP rotation), or in any lane of the row (a permute).
enum RopePair { kPairInLane, kPairFull, kPairAny };

// kStream: rows read and written past the caches' use of them (non-temporal), for
// calls that move more than the Infinity Cache holds.  With and without, us:
// 40.7K tokens of 48 head rows (1.0 GB) 174, 190; 16384 (0.4 GB) 72, 79; below it
// the rows a call leaves in the cache are worth more -- 8192 tokens (0.2 GB) 37,
// 33.5; 4096 with the segment's attention behind them 197.5, 193.8.
constexpr int64_t kRopeStreamBytes = int64_t(256) << 20;

// kAxes: each pair turns by the position on its own axis, of a few per token.  The
// token's positions are loaded by as many lanes beside the axis numbers, not behind
// them, and handed round.
//
// kKvq: key and value rows go into pages of 4 bits (kvq_kernels.h): a lane's 8 dims are
// a quarter of a block, so the scale is a maximum over 4 lanes.  Keys are normed and
// rotated in 64 bits, since a value by a tie between two elements moves by a whole step:
// of 10 million values of fp32 results about one does.  16 requests of 512 to 4096 new
// tokens with the pages read back take 220 us so, 200 in fp32; with the coefficients of
// the keys held in 64 bits 227, and with fewer rounds to a wave 253 and more.  With
// nothing to norm or rotate the keys are the input's bits.
template <RopePair kPair, bool kStream, bool kAxes = false, bool kKvq = false>
__global__ __launch_bounds__(256) void rope_append_kernel(RopeArgs a) {
  const int lane = threadIdx.x & 63;
  const int c = lane & 15, sub = lane >> 4;                 // 16-byte chunk of the row, row within a load
  const int n_qk = a.Hq + a.Hkv, n_rows = n_qk + a.Hkv;
  const int rows_wave = a.rounds * kRopeRows;
  const int per_tok = (n_rows + rows_wave - 1) / rows_wave;
  const int64_t w = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (w >= (int64_t)a.T * per_tok) return;
  const int t = (int)(w / per_tok);
  const int row_begin = (int)(w - (int64_t)t * per_tok) * rows_wave;
  const int row_end = min(row_begin + rows_wave, n_rows);

  const uint16_t* const qt = a.q + t * a.q_stride + c * 8;
  const uint16_t* const kt = a.k + t * a.k_stride + c * 8 - a.Hq * kHD;
  const uint16_t* const vt = a.v + t * a.v_stride + c * 8 - n_qk * kHD;
  auto load = [&](int row0, u32x4 (&x)[4]) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = row0 + 4 * i + sub;
      if (row >= row_end) continue;
      const uint16_t* const p = (row < a.Hq ? qt : row < n_qk ? kt : vt) + row * kHD;
      x[i] = kStream ? ld_stream(p) : ld_u32x4(p);
    }
  };
  auto store = [&](uint16_t* p, u32x4 v) __attribute__((always_inline)) {
    if constexpr (kStream) st_stream(p, v);
    else st_u32x4(p, v);
  };
  u32x4 x[4];
  load(row_begin, x);
  int32_t token_pos = 0;
  if constexpr (kAxes) token_pos = lane < a.num_axes ? a.axis_pos[lane * a.axis_stride + t] : 0;

  const int b = __builtin_amdgcn_readfirstlane(wave_find_seq(a.tok_begin, a.B, t));
  const int step = t - a.tok_begin[b];
  // where the token's key and value rows go
  const int at = a.start[b] + step;
  const int page = at / a.P, prow = at - page * a.P;
  int32_t slot = -1;
  if (row_end > a.Hq) {
    const int32_t base = a.indptr[b];
    if (page < a.indptr[b + 1] - base) slot = a.indices[base + page];
    if (slot < 0 || (int64_t)slot >= a.num_slots) {
      slot = -1;
      if (lane == 0) atomicOr(a.err, 2);
    }
  }

  // this lane's partner lane and its pairs' cosines and signed sines
  const int hl = a.rot >> 4;                                // lanes of each half (pairs of halves)
  const bool rotates = kPair == kPairFull ? true : kPair == kPairAny ? c < 2 * hl : 8 * c < a.rot;
  const bool upper = kPair == kPairFull ? c >= 8 : kPair == kPairAny && c >= hl;
  const int partner = kPair == kPairInLane || !rotates ? c : kPair == kPairFull ? c ^ 8 : upper ? c - hl : c + hl;
  uint32_t pos = 0;
  if constexpr (!kAxes) pos = (uint32_t)(a.pos[b] + step);
  float cs[8], sn[8];
  f64x2* turns = nullptr;                                   // of this wave: cosine and sine of each pair
  if constexpr (kKvq) {
    // lane j works pair j out, and the lanes of its dims read it
    __shared__ f64x2 lds[4][64];
    turns = lds[threadIdx.x >> 6];
    const bool mine = 2 * lane < a.rot;
    if constexpr (kAxes) pos = (uint32_t)__shfl(token_pos, mine ? a.axis[lane] : 0);
    if (mine) {
      double s, co;
      turn_sincos(a.freq[lane] * (kAxes ? (uint64_t)(int64_t)(int32_t)pos : (uint64_t)pos), s, co);
      turns[lane] = f64x2{co, s};
    }
    asm volatile("" ::: "memory");
    __builtin_amdgcn_wave_barrier();
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    if (kPair == kPairInLane && (e & 1)) {
      cs[e] = cs[e - 1];
      sn[e] = -sn[e - 1];
      continue;
    }
    const int j = kPair == kPairInLane ? 4 * c + e / 2 : 8 * (upper ? partner : c) + e;
    cs[e] = 1;
    sn[e] = 0;
    if constexpr (kAxes && !kKvq) pos = (uint32_t)__shfl(token_pos, rotates ? a.axis[j] : 0);
    if (rotates) {
      float s;
      if constexpr (kKvq) {
        const f64x2 both = turns[j];
        cs[e] = (float)both[0];
        s = (float)both[1];
      } else {
        const uint64_t f = a.freq[j];
        uint32_t phase = __umulhi((uint32_t)f, pos) + (uint32_t)(f >> 32) * pos;
        if constexpr (kAxes) phase -= (int32_t)pos < 0 ? (uint32_t)f : 0u;   // pos stands for pos - 2^32
        const float turns = (float)(int32_t)phase * 2.3283064365386963e-10f;   // 2^-32
        cs[e] = __builtin_amdgcn_cosf(turns);
        s = __builtin_amdgcn_sinf(turns);
      }
      sn[e] = upper ? s : -s;
    }
  }
  auto coefs = [&](const uint16_t* wt) __attribute__((always_inline)) {
    RopeCoef k;
    k.normed = wt != nullptr;
    float g[8], h[8];
    if (k.normed) {
      unpack8(ld_u32x4(wt + c * 8), g);
      unpack8(ld_u32x4(wt + partner * 8), h);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float own = k.normed ? g[e] + a.offset : 1.f;
      const float other = k.normed ? h[kPair == kPairInLane ? e ^ 1 : e] + a.offset : 1.f;
      k.own[e] = own * cs[e];
      k.other[e] = other * sn[e];
    }
    return k;
  };
  auto partners = [&](u32x4 raw, const float (&y)[8], float (&p)[8]) __attribute__((always_inline)) {
    if constexpr (kPair == kPairInLane) {
#pragma unroll
      for (int e = 0; e < 8; ++e) p[e] = rotates ? y[e ^ 1] : 0.f;
    } else {
      u32x4 o;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if constexpr (kPair == kPairFull)
          o[e] = (uint32_t)__builtin_amdgcn_mov_dpp((int)raw[e], 0x128, 0xF, 0xF, true);   // 8 lanes on
        else
          o[e] = rotates ? (uint32_t)__shfl((int)raw[e], (lane & 48) + partner) : 0u;
      }
      unpack8(o, p);
    }
  };
  auto turn = [&](u32x4 raw, const RopeCoef& k, float (&z)[8]) __attribute__((always_inline)) {
    float y[8], p[8];
    unpack8(raw, y);
    partners(raw, y, p);
    float r = 1.f;
    if (k.normed) {
      float ss[2] = {0.f, 0.f};
#pragma unroll
      for (int e = 0; e < 8; ++e) ss[e & 1] = __builtin_fmaf(y[e], y[e], ss[e & 1]);
      r = __builtin_amdgcn_rsqf(row16_sum(ss[0] + ss[1]) * (1.f / kHD) + a.eps);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      z[e] = __builtin_fmaf(y[e], k.own[e], p[e] * k.other[e]);
      if (k.normed) z[e] = r * z[e];
    }
  };
  // the same of a key row in 64 bits, its coefficients made where they are used
  auto turn_key = [&](u32x4 raw, u32x4 own, u32x4 other, float (&z)[8]) __attribute__((always_inline)) {
    float y[8], p[8], g[8], h[8];
    unpack8(raw, y);
    partners(raw, y, p);
    unpack8(own, g);
    unpack8(other, h);
    double r = 1.;
    if (a.k_weight != nullptr) {
      double ss[2] = {0., 0.};
#pragma unroll
      for (int e = 0; e < 8; ++e) ss[e & 1] = __builtin_fma((double)y[e], (double)y[e], ss[e & 1]);
      const double x = row16_sum(ss[0] + ss[1]) * (1. / kHD) + (double)a.eps;
      r = __builtin_amdgcn_rsq(x);
      r = __builtin_fma(0.5 * r, __builtin_fma(-x * r, r, 1.), r);   // a Newton step behind v_rsq's 2^-26
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      double own_e = 1., other_e = 1.;
      if (a.k_weight != nullptr) {
        own_e = (double)g[e] + (double)a.offset;
        other_e = (double)h[kPair == kPairInLane ? e ^ 1 : e] + (double)a.offset;
      }
      f64x2 both = {1., 0.};
      if (rotates) both = turns[kPair == kPairInLane ? 4 * c + e / 2 : 8 * (upper ? partner : c) + e];
      const bool plus = kPair == kPairInLane ? e & 1 : upper;
      const double v = __builtin_fma((double)y[e], own_e * both[0], (plus ? (double)p[e] : -(double)p[e]) * (other_e * both[1]));
      z[e] = rounded_to_odd(r * v);
    }
  };
  auto rounded = [](const float (&z)[8]) __attribute__((always_inline)) {
    typedef __bf16 b8 __attribute__((ext_vector_type(8)));
    b8 out;
#pragma unroll
    for (int e = 0; e < 8; ++e) out[e] = (__bf16)z[e];
    return __builtin_bit_cast(u32x4, out);
  };
  // a row into its page of 4 bits; rows of other lanes may be none of this pool's (`mine`)
  auto store4 = [&](uint8_t* pool, int head, uint32_t codes, uint32_t scale, bool mine) __attribute__((always_inline)) {
    if (!mine) return;
    uint8_t* const p = pool + ((int64_t)slot * a.Hkv + head) * a.P * kKvqRow;
    *(uint32_t*)(p + prow * kKvqCodes + c * 4) = codes;
    uint32_t scales = scale << (8 * (c >> 2));               // the row's four bytes from its four blocks
    scales |= row16u<0x124>(scales);
    scales |= row16u<0x128>(scales);
    if (c == 0) *(uint32_t*)(p + a.P * kKvqCodes + prow * 4) = scales;
  };

  uint16_t* const q_out = a.q_out + (int64_t)t * a.Hq * kHD + c * 8;
  const int64_t page_at = ((int64_t)slot * a.Hkv * a.P + prow) * kHD + c * 8;
  RopeCoef cq, ck;
  u32x4 key_own{}, key_other{};
  if (row_begin < a.Hq) cq = coefs(a.q_weight);
  if (row_end > a.Hq && row_begin < n_qk) {
    if constexpr (!kKvq) {
      ck = coefs(a.k_weight);
    } else if (a.k_weight != nullptr) {
      key_own = ld_u32x4(a.k_weight + c * 8);
      key_other = ld_u32x4(a.k_weight + partner * 8);
    }
  }
  for (int row0 = row_begin; row0 < row_end; row0 += kRopeRows) {
    u32x4 next[4];
    load(row0 + kRopeRows, next);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int first = row0 + 4 * i, row = first + sub;    // first: the same for the whole wave
      float z[8];
      if (first < a.Hq) {
        turn(x[i], cq, z);
        if (row < a.Hq) store(q_out + row * kHD, rounded(z));
      }
      if constexpr (kKvq) {
        uint32_t codes, scale;
        if (first + 3 >= a.Hq && first < n_qk) {
          if (a.rot == 0 && a.k_weight == nullptr) {
            codes = kvq_codes_bf16(x[i], scale);
          } else {
            turn_key(x[i], key_own, key_other, z);
            codes = kvq_codes(z, scale);
          }
          store4(a.kq_pool, row - a.Hq, codes, scale, row >= a.Hq && row < n_qk && slot >= 0);
        }
        if (first + 3 >= n_qk) {
          codes = kvq_codes_bf16(x[i], scale);
          store4(a.vq_pool, row - n_qk, codes, scale, row >= n_qk && row < row_end && slot >= 0);
        }
      } else {
        if (first + 3 >= a.Hq && first < n_qk) {
          turn(x[i], ck, z);
          if (row >= a.Hq && row < n_qk && slot >= 0)
            store(a.k_pool + page_at + (int64_t)(row - a.Hq) * a.P * kHD, rounded(z));
        }
        if (first + 3 >= n_qk && row >= n_qk && row < row_end && slot >= 0)
          store(a.v_pool + page_at + (int64_t)(row - n_qk) * a.P * kHD, x[i]);
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = next[i];
  }
}

}  // namespace sa
