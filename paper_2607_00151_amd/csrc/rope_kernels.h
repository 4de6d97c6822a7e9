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
// Bytes are all this does (2 * 256 per head row, read and written once): a row is
// 16 lanes of 16 bytes, a wave takes 16 rows of one token, all its loads first.
// The sum of squares is a 4-step DPP reduction within the 16 lanes, and the
// sines and cosines, which depend only on token and dim, are made once per lane
// for the wave's rows.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "common.h"
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
  int32_t half_lanes;        // pairs (d, d + rot/2): rot / 16; interleaved: unused
  int32_t rot;
  float eps, offset;
  uint64_t freq[64];         // turns per position, as a fraction of 2^64
};

constexpr int kRopeRows = 16;        // head rows per wave: 4 loads of 16 bytes per lane

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

template <int kCtrl>
__device__ __forceinline__ float row16(float x) {
  return __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(x), kCtrl, 0xF, 0xF, true));
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

template <bool kInterleaved>
__global__ __launch_bounds__(256) void rope_append_kernel(RopeArgs a) {
  const int lane = threadIdx.x & 63;
  const int c = lane & 15, sub = lane >> 4;                 // 16-byte chunk of the row, row within a load
  const int n_rows = a.Hq + 2 * a.Hkv;
  const int per_tok = (n_rows + kRopeRows - 1) / kRopeRows;
  const int64_t w = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (w >= (int64_t)a.T * per_tok) return;
  const int t = (int)(w / per_tok);
  const int row0 = (int)(w - (int64_t)t * per_tok) * kRopeRows;

  u32x4 x[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int row = row0 + 4 * i + sub;
    if (row < a.Hq) x[i] = ld_u32x4(a.q + t * a.q_stride + row * kHD + c * 8);
    else if (row < a.Hq + a.Hkv) x[i] = ld_u32x4(a.k + t * a.k_stride + (row - a.Hq) * kHD + c * 8);
    else if (row < n_rows) x[i] = ld_u32x4(a.v + t * a.v_stride + (row - a.Hq - a.Hkv) * kHD + c * 8);
    else x[i] = u32x4{0u, 0u, 0u, 0u};
  }
  const int b = __builtin_amdgcn_readfirstlane(wave_find_seq(a.tok_begin, a.B, t));
  const int step = t - a.tok_begin[b];
  // where the token's key and value rows go
  const int at = a.start[b] + step;
  const int page = at / a.P, prow = at - page * a.P;
  int32_t slot = -1;
  if (row0 + kRopeRows > a.Hq) {
    const int32_t base = a.indptr[b];
    if (page < a.indptr[b + 1] - base) slot = a.indices[base + page];
    if (slot < 0 || (int64_t)slot >= a.num_slots) {
      slot = -1;
      if (lane == 0) atomicOr(a.err, 2);
    }
  }
  // cosines and sines of this lane's pairs
  constexpr int kPairs = kInterleaved ? 4 : 8;
  const int hl = a.half_lanes;
  const bool rotates = kInterleaved ? true : c < 2 * hl;
  const bool upper = !kInterleaved && c >= hl;
  const uint32_t pos = (uint32_t)(a.pos[b] + step);
  float cs[kPairs], sn[kPairs];
#pragma unroll
  for (int e = 0; e < kPairs; ++e) {
    const int j = kInterleaved ? 4 * c + e : 8 * (upper ? c - hl : c) + e;
    const bool on = kInterleaved ? 2 * j < a.rot : rotates;
    const uint64_t phase = on ? a.freq[j] * pos : 0;
    const float turns = (float)(int32_t)(phase >> 32) * 2.3283064365386963e-10f;   // 2^-32
    cs[e] = __builtin_amdgcn_cosf(turns);
    sn[e] = __builtin_amdgcn_sinf(turns);
    if (upper) sn[e] = -sn[e];                              // own * cos - partner * sin, the sign of the upper half
  }
  const int partner = kInterleaved ? lane : (sub << 4) + (!rotates ? c : upper ? c - hl : c + hl);

#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int row = row0 + 4 * i + sub;
    const bool is_q = row < a.Hq, is_k = !is_q && row < a.Hq + a.Hkv;
    u32x4 other;
    if constexpr (!kInterleaved)
#pragma unroll
      for (int e = 0; e < 4; ++e) other[e] = (uint32_t)__shfl((int)x[i][e], partner);
    float y[8], z[8];
    unpack8(x[i], y);
    const uint16_t* wt = is_q ? a.q_weight : a.k_weight;
    float ss = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) ss = __builtin_fmaf(y[e], y[e], ss);
    ss = row16_sum(ss);
    const bool normed = (is_q || is_k) && wt != nullptr;
    const float r = __builtin_amdgcn_rsqf(ss * (1.f / kHD) + a.eps);
    if (normed) {
      float g[8];
      unpack8(ld_u32x4(wt + c * 8), g);
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = y[e] * r * (g[e] + a.offset);
    }
    if constexpr (kInterleaved) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        z[2 * e] = y[2 * e] * cs[e] - y[2 * e + 1] * sn[e];
        z[2 * e + 1] = y[2 * e + 1] * cs[e] + y[2 * e] * sn[e];
      }
    } else {
      float p[8];
      unpack8(other, p);
      if (normed) {
        float g[8];
        unpack8(ld_u32x4(wt + (partner & 15) * 8), g);
#pragma unroll
        for (int e = 0; e < 8; ++e) p[e] = p[e] * r * (g[e] + a.offset);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) z[e] = rotates ? y[e] * cs[e] - p[e] * sn[e] : y[e];
    }
    typedef __bf16 b8 __attribute__((ext_vector_type(8)));
    b8 out;
#pragma unroll
    for (int e = 0; e < 8; ++e) out[e] = (__bf16)z[e];
    const u32x4 turned = __builtin_bit_cast(u32x4, out);
    if (is_q)
      st_u32x4(a.q_out + ((int64_t)t * a.Hq + row) * kHD + c * 8, turned);
    else if (row < n_rows && slot >= 0) {
      const int head = row - a.Hq - (is_k ? 0 : a.Hkv);
      const int64_t dst = (((int64_t)slot * a.Hkv + head) * a.P + prow) * kHD + c * 8;
      st_u32x4((is_k ? a.k_pool : a.v_pool) + dst, is_k ? turned : x[i]);
    }
  }
}

}  // namespace sa
