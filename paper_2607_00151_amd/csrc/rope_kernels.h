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

// Sine and cosine of a phase in fractions of 2^32 of a turn, to about an fp32 rounding:
// the nearest quarter turn goes by symmetry, the rest, up to an eighth, by the Taylor
// series up to the 9th and 10th power (what is left out is below 2^-28).  v_sin and v_cos
// are off by some 2^-21, which a rounding to bf16 hides but which decides more of the ties
// between two elements of 4 bits, a whole step apart.
__device__ __forceinline__ void turn_sincos(uint32_t phase, float& sine, float& cosine) {
  const uint32_t quarter = (phase + 0x20000000u) >> 30;
  const float a = (float)(int32_t)(phase - (quarter << 30)) * 1.4629180792671596e-9f;   // 2 pi / 2^32
  const float x = a * a;
  float s = __builtin_fmaf(x, 2.7557319e-6f, -1.9841270e-4f);
  s = __builtin_fmaf(x, s, 8.3333333e-3f);
  s = __builtin_fmaf(x, s, -1.6666667e-1f);
  s = __builtin_fmaf(a * x, s, a);
  float c = __builtin_fmaf(x, -2.7557319e-7f, 2.4801587e-5f);
  c = __builtin_fmaf(x, c, -1.3888889e-3f);
  c = __builtin_fmaf(x, c, 4.1666667e-2f);
  c = __builtin_fmaf(x, c, -0.5f);
  c = __builtin_fmaf(x, c, 1.f);
  sine = quarter & 1 ? c : s;
  cosine = quarter & 1 ? s : c;
  if (quarter & 2) sine = -sine;
  if ((quarter + 1) & 2) cosine = -cosine;
}

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
// kKvq: key and value rows go into pages of 4 bits (kvq_kernels.h), keys from the fp32
// results: a lane's 8 dims are a quarter of a block, so the scale is a maximum over
// 4 lanes.  With Hq = 0 and nothing to norm or rotate the keys are the input's bits.
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
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    if (kPair == kPairInLane && (e & 1)) {
      cs[e] = cs[e - 1];
      sn[e] = -sn[e - 1];
      continue;
    }
    const int j = kPair == kPairInLane ? 4 * c + e / 2 : 8 * (upper ? partner : c) + e;
    cs[e] = 1.f;
    sn[e] = 0.f;
    if constexpr (kAxes) pos = (uint32_t)__shfl(token_pos, rotates ? a.axis[j] : 0);
    if (rotates) {
      const uint64_t f = a.freq[j];
      uint32_t phase = __umulhi((uint32_t)f, pos) + (uint32_t)(f >> 32) * pos;
      if constexpr (kAxes) phase -= (int32_t)pos < 0 ? (uint32_t)f : 0u;   // pos stands for pos - 2^32
      float s;
      if constexpr (kKvq) {
        turn_sincos(phase, s, cs[e]);
      } else {
        const float turns = (float)(int32_t)phase * 2.3283064365386963e-10f;   // 2^-32
        cs[e] = __builtin_amdgcn_cosf(turns);
        s = __builtin_amdgcn_sinf(turns);
      }
      sn[e] = upper ? s : -s;
    }
  }
  // out = r * (x * own + p * other)
  struct Coef {
    float own[8], other[8];
    bool normed;
  };
  auto coefs = [&](const uint16_t* wt) __attribute__((always_inline)) {
    Coef k;
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
  auto turn = [&](u32x4 raw, const Coef& k, float (&z)[8]) __attribute__((always_inline)) {
    float y[8], p[8];
    unpack8(raw, y);
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
  Coef cq, ck;
  if (row_begin < a.Hq) cq = coefs(a.q_weight);
  if (row_end > a.Hq && row_begin < n_qk) ck = coefs(a.k_weight);
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
          if (a.rot == 0 && !ck.normed) {
            codes = kvq_codes_bf16(x[i], scale);
          } else {
            turn(x[i], ck, z);
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
