// A cache of 4 bits: its format, and the conversion of pages between a bf16 pool
// and a pool of 4 bits (sa_kvq_pack, sa_kvq_unpack).
//
// A head row of 128 is four blocks of 32 neighbouring dims.  A block has a scale
// byte s, worth 2^(s - 127), and 32 elements of 4 bits: a sign, two bits of
// exponent and one of mantissa, 0 0.5 1 1.5 2 3 4 6.  With amax the block's largest
// magnitude,
//   s = exponent of amax rounded half up to one bit behind the point, less 2,
// so that 3.5 <= amax / 2^(s - 127) < 7 (the last binade's upper end rounds to 6),
// and elements are rounded to the nearest, ties to the even code.  amax itself is then
// off by 1/5 at most (5 goes to 4; cutting off at 6 takes up to 1/7); by its exponent alone,
// without rounding, 6 would cut off up to a quarter.  Powers of two make every step exact: x / 2^(s - 127) has
// x's bits, so the codes do not depend on who computes them.  s is held to 1 .. 252:
// below, elements are under 2^-127 anyway; above, 4 times the scale is no bf16 number.
// A block that holds an infinity or a NaN is 255 with codes of 0: NaN throughout.
//
// A page of one head: P rows of 64 code bytes (the even dim in a byte's low half),
// then P rows of 4 scale bytes; a slot holds its heads' pages back to back.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "common.h"
#include "kv_kernels.h"
#include "plan.h"

namespace sa {

constexpr int kKvqRow = 68;          // bytes of a head row
constexpr int kKvqCodes = 64;        // of which codes

__device__ __forceinline__ uint32_t quad_max(uint32_t x) {    // over the 4 lanes that share lane / 4
  x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0xB1, 0xF, 0xF, true));   // lane ^ 1
  return max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x4E, 0xF, 0xF, true));   // lane ^ 2
}

// The scale byte of a block from the bits of its largest magnitude (fp32, sign cleared).
__device__ __forceinline__ uint32_t kvq_scale(uint32_t top) {
  const int s = (int)((top + 0x200000u) >> 23) - 2;
  return top < 0x7F800000u ? (uint32_t)min(max(s, 1), 252) : 255u;
}

// Codes of 8 neighbouring dims, whose block lies in 4 lanes; s: the block's scale byte.
__device__ __forceinline__ uint32_t kvq_codes(const float (&x)[8], uint32_t& s) {
  uint32_t top = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(x[e]) & 0x7FFFFFFFu);
  s = kvq_scale(quad_max(top));
  const float scale = __uint_as_float(s << 23);
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], scale, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], scale, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], scale, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], scale, 3);
  return s == 255u ? 0u : w;
}

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// The same of 8 bf16 values as they lie in memory.
__device__ __forceinline__ uint32_t kvq_codes_bf16(u32x4 x, uint32_t& s) {
  typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
  u16x2 m = {0, 0};
#pragma unroll
  for (int e = 0; e < 4; ++e) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, x[e] & 0x7FFF7FFFu));
  s = kvq_scale(quad_max((uint32_t)max(m[0], m[1]) << 16));
  const float scale = __uint_as_float(s << 23);
  const uint32_t x0 = x[0], x1 = x[1], x2 = x[2], x3 = x[3];   // a bit cast of x[i] itself would read x[0]
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, x0), scale, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, x1), scale, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, x2), scale, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, x3), scale, 3);
  return s == 255u ? 0u : w;
}

// The bf16 values of 8 codes.
__device__ __forceinline__ u32x4 kvq_values(uint32_t w, uint32_t s) {
  const float scale = __uint_as_float(s << 23);
  u32x4 x;
  x[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0));
  x[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1));
  x[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2));
  x[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3));
  return x;
}

struct KvqConvArgs {
  uint16_t* k;               // bf16 pools [layers][num_slots][Hkv][P][128]
  uint16_t* v;
  uint8_t* k4;               // pools of 4 bits [layers][num_slots4][Hkv][P * 68]
  uint8_t* v4;
  const int32_t* slots;      // [pages] of the bf16 pools
  const int32_t* slots4;     // [pages] of the pools of 4 bits
  int32_t* err;
  int64_t num_slots, num_slots4;
  int32_t Hkv, P;
};

// Block (page, 2 layer + K or V).  A wave takes 16 rows at a time, which lie in one
// head's page: lane l holds chunk l % 16 (8 dims) of rows 4 i + l / 16, so a block
// of 32 dims is 4 neighbouring lanes, and both sides' accesses are contiguous.
// Of the 4 scale bytes that its lanes hold alike per row group, lane l keeps row
// 4 (l % 4) + l / 16's: the 16 rows' 64 scale bytes go out in one store.
//
// Bound by HBM: 512 pages x 32 layers (1.07 GB of bf16, 0.29 of 4 bits) to 4 bits and back
// take 468 us, 5.8 TB/s (487 where every pass has other pages; 559 seen on another card),
// with the bf16 rows read and written past the caches' use of them and two groups of rows in
// flight; 506 us, where it is 468, with ordinary loads and stores, one group at a time.  One
// or four groups, and codes transposed to 16 bytes a lane, are within 1.5% of it.
template <bool kPack>
__global__ __launch_bounds__(256) void kvq_convert_kernel(KvqConvArgs a) {
  const int lane = threadIdx.x & 63, c = lane & 15, sub = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int page = blockIdx.x, layer = blockIdx.y >> 1;
  const bool is_v = blockIdx.y & 1;
  const int32_t s = ld_uniform(a.slots + page), s4 = ld_uniform(a.slots4 + page);
  if (s < 0 || s >= a.num_slots || s4 < 0 || s4 >= a.num_slots4) {
    if (threadIdx.x == 0) atomicOr(a.err, 4);
    return;
  }
  const int rows = a.Hkv * a.P;
  uint16_t* const x = (is_v ? a.v : a.k) + ((int64_t)layer * a.num_slots + s) * rows * kHD;
  uint8_t* const x4 = (is_v ? a.v4 : a.k4) + ((int64_t)layer * a.num_slots4 + s4) * rows * kKvqRow;
  // rows r0 on: where this lane's first row, codes and scale bytes are
  struct At {
    uint16_t* x;
    uint8_t *codes, *scales;
  };
  auto at = [&](int r0) __attribute__((always_inline)) {
    const int head = r0 / a.P, in = r0 - head * a.P;
    uint8_t* const page4 = x4 + (int64_t)head * a.P * kKvqRow;
    return At{x + (int64_t)(r0 + sub) * kHD + c * 8, page4 + (in + sub) * kKvqCodes + c * 4,
              page4 + a.P * kKvqCodes + in * 4};
  };
  constexpr int kDepth = 2;                                  // groups of 16 rows in flight
  for (int r0 = wave * 16; r0 < rows; r0 += kDepth * 64) {
    if constexpr (kPack) {
      u32x4 v[kDepth][4];
#pragma unroll
      for (int n = 0; n < kDepth; ++n) {
        if (r0 + 64 * n >= rows) break;
        const At p = at(r0 + 64 * n);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[n][i] = ld_stream(p.x + 4 * i * kHD);
      }
#pragma unroll
      for (int n = 0; n < kDepth; ++n) {
        if (r0 + 64 * n >= rows) break;
        const At p = at(r0 + 64 * n);
        uint32_t mine = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint32_t sc;
          const uint32_t w = kvq_codes_bf16(v[n][i], sc);
          *(uint32_t*)(p.codes + 4 * i * kKvqCodes) = w;
          if ((c & 3) == i) mine = sc;
        }
        p.scales[(4 * (c & 3) + sub) * 4 + (c >> 2)] = (uint8_t)mine;
      }
    } else {
      uint32_t w[kDepth][4], sc[kDepth][4];
#pragma unroll
      for (int n = 0; n < kDepth; ++n) {
        if (r0 + 64 * n >= rows) break;
        const At p = at(r0 + 64 * n);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          w[n][i] = *(const uint32_t*)(p.codes + 4 * i * kKvqCodes);
          sc[n][i] = p.scales[(4 * i + sub) * 4 + (c >> 2)];
        }
      }
#pragma unroll
      for (int n = 0; n < kDepth; ++n) {
        if (r0 + 64 * n >= rows) break;
        const At p = at(r0 + 64 * n);
#pragma unroll
        for (int i = 0; i < 4; ++i) st_stream(p.x + 4 * i * kHD, kvq_values(w[n][i], sc[n][i]));
      }
    }
  }
}

}  // namespace sa
