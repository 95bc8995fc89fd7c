// Shared by the attention kernels over pages (tq_pages_attend.hip, tq_pages_attend_prompt.hip); the mathematics is described in the first.
#pragma once
#include "tq_pages.h"

namespace tq {

constexpr float BASE = 7.f, HEAD = 8.f;  // weights up to 2^15 of fp16's 2^16
constexpr float LN2 = 0.69314718055994530942f;

__device__ __forceinline__ float swap_max(float v) {  // over the four lanes that share lane % 16
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float swap_sum(float v) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// eight codes as bf16 / fp16, exactly
template <int CT>
__device__ __forceinline__ bf16x8_t codes_bf16(uint32_t lo, uint32_t hi) {
  union {
    bf16x2_t h[4];
    uint32_t w[4];
    bf16x8_t v;
  } u;
  if constexpr (CT == kPageE4m3) {
    u.h[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)lo, 1.f, false);
    u.h[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)lo, 1.f, true);
    u.h[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)hi, 1.f, false);
    u.h[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)hi, 1.f, true);
  } else {
    asm("" : "+v"(lo), "+v"(hi));  // (whole words: else the compiler carries a tile through the loop a byte a register)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t w = (i < 2 ? lo : hi) >> (16 * (i & 1));
      u.w[i] = __builtin_amdgcn_perm(__float_as_uint((float)(int8_t)(w >> 8)), __float_as_uint((float)(int8_t)w), 0x07060302u);
    }
  }
  return u.v;
}
template <int CT>
__device__ __forceinline__ half8_t codes_fp16(uint32_t lo, uint32_t hi) {
  union {
    half2_t h[4];
    half8_t v;
  } u;
  if constexpr (CT == kPageE4m3) {
    u.h[0] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)lo, 1.f, false);
    u.h[1] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)lo, 1.f, true);
    u.h[2] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)hi, 1.f, false);
    u.h[3] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)hi, 1.f, true);
  } else {
    asm("" : "+v"(lo), "+v"(hi));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t w = (i < 2 ? lo : hi) >> (16 * (i & 1));
      u.h[i] = __builtin_convertvector(float2_t{(float)(int8_t)w, (float)(int8_t)(w >> 8)}, half2_t);
    }
  }
  return u.v;
}

// coordinates [first, first + N) of an output row: the sums over the weights' sum
template <int N, bool F32>
__device__ __forceinline__ void store_row(const PagesRows& out, int64_t row, int head, int first, const float (&y)[N], float sum) {
  const float inv = sum != 0.f ? 1.f / sum : 0.f;
  const int64_t at = row * out.ld_row + head * out.ld_head + first;
  if constexpr (F32) {
    typedef float vec __attribute__((ext_vector_type(N < 4 ? N : 4)));
#pragma unroll
    for (int c = 0; c < N; c += 4) {
      vec z;
#pragma unroll
      for (int i = 0; i < (N < 4 ? N : 4); ++i) z[i] = y[c + i] * inv;
      *reinterpret_cast<vec*>(static_cast<float*>(const_cast<void*>(out.p)) + at + c) = z;
    }
  } else {
    typedef __bf16 vec __attribute__((ext_vector_type(N < 8 ? N : 8)));
#pragma unroll
    for (int c = 0; c < N; c += 8) {
      vec z;
#pragma unroll
      for (int i = 0; i < (N < 8 ? N : 8); ++i) z[i] = (__bf16)(y[c + i] * inv);
      *reinterpret_cast<vec*>(static_cast<uint16_t*>(const_cast<void*>(out.p)) + at + c) = z;
    }
  }
}
__device__ __forceinline__ float log_sum(float M, float sum) { return sum != 0.f ? (__builtin_amdgcn_logf(sum) + (M - BASE)) * LN2 : -INFINITY; }

// bytes that are the NaN of e4m3, as 0xff
__device__ __forceinline__ uint32_t nan_bytes(uint32_t w) {
  return ((((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) >> 7) * 255u;
}

// Beyond every position that a row or a stored token has here: rows further on count as at the last one before it, and the tokens from it on
// (fewer than 128 below 2^31) are not there.  What is no page lies at it, seen by no row; 127 above it is still an int.
constexpr int NOWHERE = 0x7fffff80;
__device__ __forceinline__ int row_position(int64_t at) { return (int)max(min(at, (int64_t)NOWHERE - 1), (int64_t)-1); }

// One subtile of 16 keys, as a lane of a wavefront that looks up 64 at a time knows it.
struct Subtile {
  int at;        // its place in the pool in units of 16 tokens, -1: its page is none
  int pos;       // of its first token (NOWHERE where its page is none)
  float ks, lv, iv;  // scale of its keys, base-2 logarithm and inverse of that of its values
};
__device__ __forceinline__ Subtile no_subtile() { return Subtile{-1, NOWHERE, 1.f, 0.f, 1.f}; }
// the 16 tokens from position `off` of place i of a table's row on, head h
__device__ __forceinline__ Subtile find_subtile(const PagesView& c, const int32_t* table, int width, int h, int i, int off) {
  Subtile t = no_subtile();
  const int64_t pos = ((int64_t)i << c.log2_page) + off;
  if (i < 0 || i >= width || pos >= NOWHERE) return t;
  const int p = table[i];
  if (p < 0 || p >= c.n_pages) return t;
  const int64_t block = (int64_t)p * c.heads + h;
  t.at = (int)(((block << c.log2_page) + off) >> 4);
  t.pos = (int)pos;
  t.ks = c.k_scale[block];
  const float vs = c.v_scale[block];
  t.lv = __builtin_amdgcn_logf(vs);
  t.iv = 1.f / vs;
  // A scale that is none (a page that nothing was appended to) makes the rows that see it NaN, by their logits: an unseen key has the
  // weight 0, which must not meet 1 / 0 or NaN.
  if (!(t.iv > 0.f && t.iv < INFINITY)) t.lv = __builtin_nanf(""), t.iv = 0.f;
  return t;
}
__device__ __forceinline__ float lane_value(float v, int lane) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), lane)); }

}  // namespace tq
