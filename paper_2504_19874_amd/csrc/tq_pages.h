// Shared by the kernels of the 8-bit paged cache (tq_pages_*.hip).
#pragma once
#include "tq_internal.h"
#include "tq_pages_plan.h"

namespace tq {

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
typedef _Float16 half8_t __attribute__((ext_vector_type(8)));
typedef float float2_t __attribute__((ext_vector_type(2)));
typedef float float4_t __attribute__((ext_vector_type(4)));
typedef uint32_t uint2_t __attribute__((ext_vector_type(2)));
typedef uint32_t uint4_t __attribute__((ext_vector_type(4)));

constexpr int kPageE4m3 = TQ_PAGE_E4M3, kPageI8 = TQ_PAGE_I8;
constexpr int kPageScaleLow = -40, kPageScaleHigh = 40;  // exponents of the scales that append makes

// A call's cache and batch as the kernels take them (tq_pages, tq_batch).
struct PagesView {
  uint8_t *k, *v;
  float *k_scale, *v_scale;
  uint16_t* bounds;
  int32_t* refs;
  int n_pages, heads, log2_page;
};
struct BatchView {
  int32_t *table, *lens;
  const int32_t* starts;
  int64_t table_stride, n_rows;
  int width, n_seqs, max_new;
  // first row of sequence s, and its rows (no more than max_new of them are worked on)
  __device__ __forceinline__ int64_t first_row(int s) const { return starts != nullptr ? starts[s] : (int64_t)s * max_new; }
  __device__ __forceinline__ int count(int s) const { return starts != nullptr ? starts[s + 1] - starts[s] : max_new; }
};

// Numbers below 2^31 (2^31 + 2 for divisors below 2^30) over one that the host knows: a product's upper half, a sum and a shift (scalar where the number is; the compiler's own
// division of two registers is some thirty vector instructions, of 64 bits over a hundred, in front of a kernel's first load).
struct Divide {
  uint32_t mul, shift, by;
  Divide() = default;
  explicit Divide(int64_t d) : mul(0), shift(0), by((uint32_t)(d > 0 ? d : 1)) {
    while ((1ull << shift) < by) ++shift;
    mul = (uint32_t)(((1ull << 32) * ((1ull << shift) - by)) / by + 1);
  }
  __device__ __forceinline__ uint32_t of(uint32_t n) const { return (__umulhi(n, mul) + n) >> shift; }
  __device__ __forceinline__ uint32_t rest(uint32_t n, uint32_t quotient) const { return n - quotient * by; }
};

// One launch takes this many workgroups: it counts the threads of a dimension in 32 bits.
inline bool grid_fits(int64_t blocks, int threads) { return blocks * threads <= 0xffffffffll; }

// Rows of keys, values, queries or outputs.
struct PagesRows {
  const void* p;
  int64_t ld_row, ld_head;
};

// codes of one dword as fp32
template <int CT>
__device__ __forceinline__ void page_decode(uint32_t w, float (&x)[4]) {
  if constexpr (CT == kPageE4m3) {
    const float2_t a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    x[0] = a[0], x[1] = a[1], x[2] = b[0], x[3] = b[1];
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = (float)(int8_t)(w >> (8 * i));
  }
}
// four values over their scale as codes: to nearest, ties to even, the largest code beyond it; NaN stays NaN in e4m3 and is 0 in int8
template <int CT>
__device__ __forceinline__ uint32_t page_encode(const float (&x)[4]) {
  constexpr float top = CT == kPageE4m3 ? 448.f : 127.f;
  float y[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    y[i] = fminf(fmaxf(x[i], -top), top);
    if (x[i] != x[i]) y[i] = CT == kPageE4m3 ? x[i] : 0.f;
  }
  if constexpr (CT == kPageE4m3) {
    const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], lo, true);
  } else {
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) w |= ((uint32_t)(int)rintf(y[i]) & 0xffu) << (8 * i);
    return w;
  }
}

struct PagesAttendArgs {
  PagesView c;
  BatchView b;
  PagesRows q, out;
  float* lse;
  const int32_t* chosen;
  int n_chosen;
  int group;  // query heads that read a head of the cache
  float scale2, scale2_rest;  // log2(e) scale as a sum of two
  int window;  // of tokens that a row sees; INT_MAX: all
  int splits;   // ranges that the keys of a unit are cut into
  bool prompt;  // the kernel for prompts
  int tiles;    // of 16 rows to a workgroup of the other kernel
  float* part;  // what they leave, [n_rows][query heads][splits][4 + d]; with one range unused
  Divide by_splits, by_tiles, by_heads, by_new, by_group, by_queries;  // (tiles of rows: of the kernel that is taken; query heads)
};
inline PagesAttendSizes pages_attend_sizes(const BatchView& b, int heads, int group, bool chosen, int n_chosen, int log2_page, int window) {
  return PagesAttendSizes{b.n_seqs, b.max_new, b.width, heads, group, chosen, n_chosen, log2_page, window};
}
size_t pages_attend_part_bytes(int d, const BatchView& b, int heads, int group, int splits);
hipError_t launch_pages_attend(int d, int type, bool f32, const PagesAttendArgs& a, hipStream_t s);
// many rows of bf16 queries (tq_pages_attend_prompt.hip)
hipError_t launch_pages_attend_prompt(int d, int type, const PagesAttendArgs& a, hipStream_t s);

// The launches below return hipErrorInvalidConfiguration, and have launched nothing, where a grid does not fit.
hipError_t launch_pages_append(int d, int type, bool f32, const PagesView& c, const BatchView& b, const PagesRows& k, const PagesRows& v,
                               hipStream_t s);

struct PagesSelectArgs {
  PagesView c;
  BatchView b;
  PagesRows q;
  int group, keep_first, keep_last, n_chosen;
  int32_t* chosen;
  float* scores;  // [n_rows][heads][width]
  Divide by_heads, by_new, by_blocks;  // (blocks: workgroups that score the pages of a row and head)
};
hipError_t launch_pages_select(int d, bool f32, const PagesSelectArgs& a, hipStream_t s);
bool pages_pick_fits(const BatchView& b, int heads);  // the grid of the choice itself

hipError_t launch_pages_reserve(const PagesView& c, const BatchView& b, int32_t* list, int32_t* missing, hipStream_t s);
hipError_t launch_pages_fork(const PagesView& c, const BatchView& b, int d, const int32_t* parents, const int32_t* children, int n, int32_t* list,
                             int32_t* pairs, int32_t* missing, hipStream_t s);  // pairs: 2 n, 8-byte aligned
hipError_t launch_pages_free(const PagesView& c, const BatchView& b, const int32_t* rows, int n, hipStream_t s);
hipError_t launch_pages_compact(const PagesView& c, const BatchView& b, int d, int32_t* plan, int32_t* move, int32_t* at, int32_t* n_live, hipStream_t s);
hipError_t launch_pages_copy(const PagesView& c, int d, const int32_t* src, const int32_t* dst, int64_t n, hipStream_t s);

}  // namespace tq
