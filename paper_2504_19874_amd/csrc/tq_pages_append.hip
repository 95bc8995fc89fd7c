// New keys and values into pages of 8-bit codes.
//
// A workgroup has one page of one head that gets a row, its keys or its values (blockIdx.z): amax over the new rows, from it the
// scale 2^e; the codes of tokens that were there are rounded to a scale that grew (the factor is a power of two: exact in fp32, one
// rounding to the code); then the new rows' codes, and of keys the page's bounds.  A row is read once (kept in registers while
// a thread has no more than HELD vectors of eight values), a code written once: bound by memory, for a few tokens by
// the launch and the chain lens -> table -> scale -> codes.
#include <cfloat>

#include "tq_pages.h"

namespace tq {

namespace {

constexpr int HELD = 4;
constexpr float BF16_MAX = 3.38953139e38f;

typedef uint16_t ushort2_t __attribute__((ext_vector_type(2)));

template <bool F32>
struct Vec8 {
  uint4_t w[F32 ? 2 : 1];
  __device__ __forceinline__ void load(const void* p, int64_t at) {
    if constexpr (F32) {
      w[0] = *reinterpret_cast<const uint4_t*>(static_cast<const float*>(p) + at);
      w[1] = *reinterpret_cast<const uint4_t*>(static_cast<const float*>(p) + at + 4);
    } else {
      w[0] = *reinterpret_cast<const uint4_t*>(static_cast<const uint16_t*>(p) + at);
    }
  }
  // the larger of `most` and the values' magnitudes: of fp32 their bits; of bf16 two at a time, to be taken apart by unpacked()
  __device__ __forceinline__ uint32_t top(uint32_t most) const {
    if constexpr (F32) {
#pragma unroll
      for (int i = 0; i < 8; ++i) most = max(most, w[i >> 2][i & 3] & 0x7fffffffu);
      return most;
    } else {
      ushort2_t m = __builtin_bit_cast(ushort2_t, most);
#pragma unroll
      for (int i = 0; i < 4; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(ushort2_t, w[0][i] & 0x7fff7fffu));
      return __builtin_bit_cast(uint32_t, m);
    }
  }
  static __device__ __forceinline__ uint32_t unpacked(uint32_t most) { return F32 ? most : max(most & 0xffff0000u, most << 16); }
  __device__ __forceinline__ float operator[](int i) const {
    if constexpr (F32) return __uint_as_float(w[i >> 2][i & 3]);
    else return __uint_as_float((i & 1) ? w[0][i >> 1] & 0xffff0000u : w[0][i >> 1] << 16);
  }
};

// the exponent of the smallest power of two s with amax / s <= the largest code
template <int CT>
__device__ __forceinline__ int scale_exponent(float amax) {
  constexpr uint32_t top_mantissa = CT == kPageE4m3 ? 0x600000u : 0x7e0000u;  // 448 = 1.75 * 2^8, 127 = 1.984375 * 2^6
  constexpr int top_exponent = CT == kPageE4m3 ? 8 : 6;
  const uint32_t b = __float_as_uint(amax);
  if (b < 0x00800000u) return kPageScaleLow;  // zero and what is below the normal range
  const int e = (int)(b >> 23) - 127 - top_exponent + ((b & 0x7fffffu) > top_mantissa ? 1 : 0);
  return e < kPageScaleLow ? kPageScaleLow : e > kPageScaleHigh ? kPageScaleHigh : e;
}
__device__ __forceinline__ float pow2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// an fp32 value to the next bf16 below (above), as fp32
__device__ __forceinline__ float outward(float x, bool down) {
  x = fminf(fmaxf(x, -BF16_MAX), BF16_MAX);
  const uint32_t b = __float_as_uint(x);
  const bool away = (b & 0xffffu) != 0 && ((b >> 31) != 0) == down;
  return __uint_as_float((b & 0xffff0000u) + (away ? 0x10000u : 0u));
}

template <int D, int CT, bool F32, int THREADS>
__global__ __launch_bounds__(THREADS) void pages_append_kernel(const PagesView c, const BatchView b, const PagesRows kr, const PagesRows vr,
                                                              const Divide pages_each) {
  constexpr int COLS = D / 8, LINES = THREADS / COLS;  // threads of a row, rows at a time
  __shared__ uint32_t red_s[THREADS / 64];
  __shared__ float edge_s[2][LINES][D];
  const int tid = threadIdx.x, col = tid % COLS, line = tid / COLS;
  const uint32_t seq = pages_each.of(blockIdx.x);
  const int s = (int)seq, h = blockIdx.y;
  const bool values = blockIdx.z != 0;
  const int page = 1 << c.log2_page;
  const int len = b.lens[s], count = b.count(s);
  const int64_t begin = (int64_t)len - count;  // position of the sequence's first row
  const int64_t first = begin > 0 ? begin : 0;
  const int64_t index = (first >> c.log2_page) + pages_each.rest(blockIdx.x, seq), at = index << c.log2_page;
  // positions [lo, hi) of this page are new (no more than max_new rows of a sequence are taken)
  const int64_t end = count > b.max_new ? begin + b.max_new : (int64_t)len;
  const int64_t row0 = b.first_row(s);
  int64_t lo = first > at ? first : at, hi = end < at + page ? end : at + page;
  if (row0 + (lo - begin) < 0) lo = begin - row0;
  if (row0 + (hi - begin) > b.n_rows) hi = b.n_rows - row0 + begin;
  if (lo >= hi || index >= b.width) return;
  const int p = b.table[(int64_t)s * b.table_stride + index];
  if (p < 0 || p >= c.n_pages) return;
  const int had = (int)(lo - at), rows = (int)(hi - lo);
  const int64_t block = (int64_t)p * c.heads + h;
  uint8_t* const codes = (values ? c.v : c.k) + ((block << c.log2_page) * D);
  float* const scale = (values ? c.v_scale : c.k_scale) + block;
  const float before = had > 0 ? *scale : 0.f;
  const PagesRows& x = values ? vr : kr;
  const int64_t from = (row0 + (lo - begin)) * x.ld_row + h * x.ld_head + 8 * col;
  const int mine = rows > line ? (rows - line + LINES - 1) / LINES : 0;  // vectors of this thread: rows line, line + LINES, ...
  const bool bounds = !values && c.bounds != nullptr;

  // the largest magnitude, as bits (those of what is not finite above all others), and of keys the channels' ends
  Vec8<F32> held[HELD];
  uint32_t top = 0;
  float low[8], high[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) low[i] = INFINITY, high[i] = -INFINITY;
  for (int j0 = 0; j0 < mine; j0 += HELD) {
#pragma unroll
    for (int u = 0; u < HELD; ++u)
      if (j0 + u < mine) held[u].load(x.p, from + (int64_t)(line + (j0 + u) * LINES) * x.ld_row);
#pragma unroll
    for (int u = 0; u < HELD; ++u)
      if (j0 + u < mine) {
        top = held[u].top(top);
        if (bounds)
#pragma unroll
          for (int i = 0; i < 8; ++i) low[i] = fminf(low[i], held[u][i]), high[i] = fmaxf(high[i], held[u][i]);  // (a NaN is passed over)
      }
  }
  top = Vec8<F32>::unpacked(top);
  const auto larger = [](uint32_t p, uint32_t q) { return p > q ? p : q; };
  top = over_wavefront(top, larger);
  if ((tid & 63) == 0) red_s[tid >> 6] = top;
  if (bounds)
#pragma unroll
    for (int i = 0; i < 8; ++i) edge_s[0][line][8 * col + i] = low[i], edge_s[1][line][8 * col + i] = high[i];
  __syncthreads();
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w) top = larger(top, red_s[w]);
  const bool clean = top < 0x7f800000u;  // every value is finite
  float amax = __uint_as_float(top);
  if (!clean) {
    amax = 0.f;
    for (int j = 0; j < mine; ++j) {
      held[0].load(x.p, from + (int64_t)(line + j * LINES) * x.ld_row);
#pragma unroll
      for (int i = 0; i < 8; ++i) amax = fmaxf(amax, fabsf(held[0][i]) <= FLT_MAX ? fabsf(held[0][i]) : 0.f);
    }
    amax = over_wavefront(amax, [](float p, float q) { return fmaxf(p, q); });
    __syncthreads();
    if ((tid & 63) == 0) red_s[tid >> 6] = __float_as_uint(amax);
    __syncthreads();
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) amax = fmaxf(amax, __uint_as_float(red_s[w]));
  }
  // a power of two: what was there (of any kind, if append has not made it) is taken up to one
  const uint32_t was = __float_as_uint(before);
  const bool old = had > 0 && was >= 0x00800000u && was < 0x7e800000u;
  int e = scale_exponent<CT>(amax);
  const bool beyond = e == kPageScaleHigh;  // (values may be larger than the largest code)
  if (old) e = max(e, (int)(was >> 23) - 127 + ((was & 0x7fffffu) != 0 ? 1 : 0));
  const float after = pow2(e), inv = pow2(-e);
  if (tid == 0) *scale = after;

  if (old && after != before) {
    const float factor = before * inv;
    for (int i = tid * 16; i < had * D; i += THREADS * 16) {
      uint4_t w = *reinterpret_cast<const uint4_t*>(codes + i);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float y[4];
        page_decode<CT>(w[j], y);
#pragma unroll
        for (int k = 0; k < 4; ++k) y[k] *= factor;
        w[j] = page_encode<CT>(y);
      }
      *reinterpret_cast<uint4_t*>(codes + i) = w;
    }
  }

  const auto store = [&](auto encode) {
    for (int j0 = 0; j0 < mine; j0 += HELD) {
      if (mine > HELD || !clean) {
#pragma unroll
        for (int u = 0; u < HELD; ++u)
          if (j0 + u < mine) held[u].load(x.p, from + (int64_t)(line + (j0 + u) * LINES) * x.ld_row);
      }
#pragma unroll
      for (int u = 0; u < HELD; ++u)
        if (j0 + u < mine) {
          uint2_t w;
          w[0] = encode(held[u][0], held[u][1], held[u][2], held[u][3]);
          w[1] = encode(held[u][4], held[u][5], held[u][6], held[u][7]);
          *reinterpret_cast<uint2_t*>(codes + (int64_t)(had + line + (j0 + u) * LINES) * D + 8 * col) = w;
        }
    }
  };
  if (clean && !beyond) {
    store([&](float p, float q, float r, float t) {
      if constexpr (CT == kPageE4m3) {
        const int w = __builtin_amdgcn_cvt_pk_fp8_f32(p * inv, q * inv, 0, false);
        return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(r * inv, t * inv, w, true);
      } else {
        // 1.5 * 2^23 above: the sum is rounded to a whole number, ties to even, whose two's complement ends its bits
        constexpr float up = 12582912.f;
        const uint32_t a0 = __float_as_uint(fmaf(p, inv, up)), a1 = __float_as_uint(fmaf(q, inv, up));
        const uint32_t a2 = __float_as_uint(fmaf(r, inv, up)), a3 = __float_as_uint(fmaf(t, inv, up));
        return __builtin_amdgcn_perm(__builtin_amdgcn_perm(a3, a2, 0x0c0c0400u), __builtin_amdgcn_perm(a1, a0, 0x0c0c0400u), 0x05040100u);
      }
    });
  } else {
    store([&](float p, float q, float r, float t) { return page_encode<CT>({p * inv, q * inv, r * inv, t * inv}); });
  }

  if (bounds)
    for (int j = tid; j < D; j += THREADS) {
      float lower = INFINITY, upper = -INFINITY;
      for (int n = 0; n < (rows < LINES ? rows : LINES); ++n) {
        lower = fminf(lower, edge_s[0][n][j]);
        upper = fmaxf(upper, edge_s[1][n][j]);
      }
      if (lower > upper) lower = upper = 0.f;  // nothing but NaN
      uint16_t* const to = c.bounds + block * (2 * D);
      lower = outward(lower, true), upper = outward(upper, false);
      if (had > 0) {
        lower = fminf(lower, __uint_as_float((uint32_t)to[j] << 16));
        upper = fmaxf(upper, __uint_as_float((uint32_t)to[D + j] << 16));
      }
      to[j] = (uint16_t)(__float_as_uint(lower) >> 16);
      to[D + j] = (uint16_t)(__float_as_uint(upper) >> 16);
    }
}

template <int D, int CT, bool F32>
hipError_t launch(const PagesView& c, const BatchView& b, const PagesRows& k, const PagesRows& v, hipStream_t s) {
  // max_new rows from any position on lie in no more than this many pages, and a sequence has no more than width
  int64_t pages_each = (((int64_t)b.max_new + (1 << c.log2_page) - 2) >> c.log2_page) + 1;
  if (pages_each > b.width) pages_each = b.width;
  if (!grid_fits(b.n_seqs * pages_each, 256)) return hipErrorInvalidConfiguration;
  const dim3 grid((unsigned)(b.n_seqs * pages_each), (unsigned)c.heads, 2);
  hipLaunchKernelGGL((pages_append_kernel<D, CT, F32, 256>), grid, dim3(256), 0, s, c, b, k, v, Divide(pages_each));
  return hipGetLastError();
}

template <int D>
hipError_t launch_d(int type, bool f32, const PagesView& c, const BatchView& b, const PagesRows& k, const PagesRows& v, hipStream_t s) {
  if (type == kPageI8) return f32 ? launch<D, kPageI8, true>(c, b, k, v, s) : launch<D, kPageI8, false>(c, b, k, v, s);
  return f32 ? launch<D, kPageE4m3, true>(c, b, k, v, s) : launch<D, kPageE4m3, false>(c, b, k, v, s);
}

}  // namespace

hipError_t launch_pages_append(int d, int type, bool f32, const PagesView& c, const BatchView& b, const PagesRows& k, const PagesRows& v,
                               hipStream_t s) {
  if (d == 64) return launch_d<64>(type, f32, c, b, k, v, s);
  if (d == 128) return launch_d<128>(type, f32, c, b, k, v, s);
  return launch_d<256>(type, f32, c, b, k, v, s);
}

}  // namespace tq
