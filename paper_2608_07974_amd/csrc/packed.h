// Device side of the packed format (include/zl_layer.h): e4m3 codes with a
// power-of-two scale per 32 columns.  A lane holds 8 consecutive columns, four
// consecutive lanes a block, so the block's maximum is two DPP moves.
#pragma once

#include "common.h"

namespace zl {

constexpr int PW = 8;    // columns per lane
constexpr int PBLK = 32; // columns per scale

__device__ __forceinline__ uint32_t quad_max(uint32_t m) {
  m = max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0xB1, 0xF, 0xF, true));  // lane ^ 1
  return max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x4E, 0xF, 0xF, true));  // lane ^ 2
}

// Packs the 8 values of this lane; all four lanes of a block take part, with
// zeros past the row's end.  Returns the codes (low bytes first) and leaves the
// scale byte in sb.  The scale: 2^e with e = the exponent of the block's
// maximum less 8, one more where its fraction is above 1.75 (448 = 1.75 * 2^8).
// Scaling by a power of two is exact; the conversion rounds to nearest even.
__device__ __forceinline__ uint2 pack8(const float (&v)[PW], uint32_t& sb) {
  uint32_t m = 0;
#pragma unroll
  for (int k = 0; k < PW; ++k) m = max(m, __float_as_uint(v[k]) & 0x7fffffffu);
  m = quad_max(m);
  float w[PW];
  if (m <= 0x7f600000u) {  // 1.75 * 2^127: every value is finite and within the largest block
    int e = (int)(m >> 23) - 135 + ((m & 0x7fffffu) > 0x600000u ? 1 : 0);
    e = max(e, -117);
    sb = (uint32_t)(e + 127);
    const float inv = __uint_as_float((uint32_t)(127 - e) << 23);
#pragma unroll
    for (int k = 0; k < PW; ++k) w[k] = v[k] * inv;
  } else {  // scale from the finite values, the others become NaN
    m = 0;
#pragma unroll
    for (int k = 0; k < PW; ++k) {
      const uint32_t a = __float_as_uint(v[k]) & 0x7fffffffu;
      m = max(m, a < 0x7f800000u ? a : 0u);
    }
    m = quad_max(m);
    int e = (int)(m >> 23) - 135 + ((m & 0x7fffffu) > 0x600000u ? 1 : 0);
    e = min(max(e, -117), 119);
    sb = (uint32_t)(e + 127);
    const float inv = __uint_as_float((uint32_t)(127 - e) << 23);
#pragma unroll
    for (int k = 0; k < PW; ++k) {
      const uint32_t a = __float_as_uint(v[k]) & 0x7fffffffu;
      w[k] = a < 0x7f800000u ? fminf(fmaxf(v[k] * inv, -448.f), 448.f) : __uint_as_float(0x7fc00000u);
    }
  }
  uint2 c;
  c.x = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(w[0], w[1], 0, false);
  c.x = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(w[2], w[3], (int)c.x, true);
  c.y = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(w[4], w[5], 0, false);
  c.y = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(w[6], w[7], (int)c.y, true);
  return c;
}

// 2^(b - 127): bytes 1 .. 254 are the exponent field, 0 is subnormal, 255 NaN.
__device__ __forceinline__ float scale_of(uint32_t b) {
  return __uint_as_float(b == 0 ? 0x00400000u : b == 255 ? 0x7fc00000u : b << 23);
}

__device__ __forceinline__ void unpack8(const uint2 c, const uint32_t sb, float (&v)[PW]) {
  const float s = scale_of(sb);
  const f32x2_t a = __builtin_amdgcn_cvt_pk_f32_fp8((int)c.x, false);
  const f32x2_t b = __builtin_amdgcn_cvt_pk_f32_fp8((int)c.x, true);
  const f32x2_t d = __builtin_amdgcn_cvt_pk_f32_fp8((int)c.y, false);
  const f32x2_t f = __builtin_amdgcn_cvt_pk_f32_fp8((int)c.y, true);
  v[0] = a[0] * s; v[1] = a[1] * s; v[2] = b[0] * s; v[3] = b[1] * s;
  v[4] = d[0] * s; v[5] = d[1] * s; v[6] = f[0] * s; v[7] = f[1] * s;
}

// 8 consecutive elements of an fp32 or bf16 row as they lie in memory (16-byte
// aligned), and as numbers.  Element i + c: where i is the same for all lanes,
// the address is a scalar base and a 32-bit lane offset.
template <typename T>
__device__ __forceinline__ const T* at(const void* p, int64_t byte, uint32_t lane_byte) {
  return reinterpret_cast<const T*>(static_cast<const char*>(p) + byte + lane_byte);
}
template <typename T>
__device__ __forceinline__ T* at(void* p, int64_t byte, uint32_t lane_byte) {
  return reinterpret_cast<T*>(static_cast<char*>(p) + byte + lane_byte);
}
// NT: streaming accesses.  An access of 16 (codes 8) bytes per lane writes whole
// lines then; fp32 stores, 32 bytes per lane in two accesses, would not (rotary
// of 16384 x 5120 fp32: 138 us, streaming 173) and never stream.
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
template <bool BF> struct Raw8;
template <> struct Raw8<true> {
  uint4 a;
  __device__ __forceinline__ void zero() { a = make_uint4(0, 0, 0, 0); }
  template <bool NT = false>
  __device__ __forceinline__ void load(const void* p, int64_t i, uint32_t c = 0) {
    const u32x4_t* q = at<u32x4_t>(p, i * 2, c * 2);
    a = __builtin_bit_cast(uint4, NT ? __builtin_nontemporal_load(q) : *q);
  }
  __device__ __forceinline__ void get(float (&v)[PW]) const {
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      v[2 * k] = __uint_as_float(w[k] << 16);
      v[2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u);
    }
  }
};
template <> struct Raw8<false> {
  float4 a, b;
  __device__ __forceinline__ void zero() { a = b = make_float4(0.f, 0.f, 0.f, 0.f); }
  template <bool NT = false>
  __device__ __forceinline__ void load(const void* p, int64_t i, uint32_t c = 0) {
    const float4* q = at<float4>(p, i * 4, c * 4);
    a = q[0];
    b = q[1];
  }
  __device__ __forceinline__ void get(float (&v)[PW]) const {
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  }
};
// Rounded to nearest even where the type is bf16.
template <bool BF, bool NT = false>
__device__ __forceinline__ void store8(void* p, int64_t i, uint32_t c, const float (&v)[PW]) {
  if constexpr (BF) {
    const u32x4_t w = {pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
    u32x4_t* q = at<u32x4_t>(p, i * 2, c * 2);
    if (NT) __builtin_nontemporal_store(w, q);
    else *q = w;
  } else {
    float4* q = at<float4>(p, i * 4, c * 4);
    q[0] = make_float4(v[0], v[1], v[2], v[3]);
    q[1] = make_float4(v[4], v[5], v[6], v[7]);
  }
}

// The same for the 8 codes and the scale byte of a lane.
struct RawP {
  uint2 c;
  uint32_t s;
  __device__ __forceinline__ void zero() { c = make_uint2(0, 0); s = 127; }
  __device__ __forceinline__ void load(const zl_packed& p, int64_t r, uint32_t col) {
    c = *at<uint2>(static_cast<const void*>(p.codes), r * p.ld_codes, col);
    s = *at<uint8_t>(static_cast<const void*>(p.scales), r * p.ld_scales, col / PBLK);
  }
  __device__ __forceinline__ void get(float (&v)[PW]) const { unpack8(c, s, v); }
};
// Stores the codes of a lane and, from the block's first lane, the scale.
template <bool NT = false>
__device__ __forceinline__ void store_packed(const zl_packed& p, int64_t r, uint32_t col, uint2 c, uint32_t sb) {
  u32x2_t* q = at<u32x2_t>(p.codes, r * p.ld_codes, col);
  const u32x2_t w = {c.x, c.y};
  if (NT) __builtin_nontemporal_store(w, q);
  else *q = w;
  if ((col & (PBLK - 1)) == 0) *at<uint8_t>(p.scales, r * p.ld_scales, col / PBLK) = (uint8_t)sb;
}

}  // namespace zl
