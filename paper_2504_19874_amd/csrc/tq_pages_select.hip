// Choosing pages by the bounds of their keys.
//
// No key k of a page with bounds lo <= k <= hi has <q, k> above sum_j max(q_j lo_j, q_j hi_j).  The sums are taken in 64 bits (a
// product of two bf16 values is exact there, and so is the sum of a page's products unless they are 2^30 apart) and rounded to fp32
// once: which page is chosen does not depend on the order of a sum.
//
// pages_score_kernel writes one word for every page that a row may choose, ordered like its rank: 0 no page, 1 NaN, then the
// scores' bits in an order of unsigned numbers, all ones for pages that are kept.  pages_pick_kernel finds the n_chosen-th
// largest word byte by byte (counts of the words that share the bytes found so far) and writes the places of what is above it, and
// of as many equal ones as there is room for, lowest first.
#include "tq_pages.h"

namespace tq {

namespace {

constexpr int HEADS_AT_ONCE = 4;

__device__ __forceinline__ float load_value(const void* p, int64_t at, bool f32) {
  return f32 ? static_cast<const float*>(p)[at] : __uint_as_float((uint32_t)static_cast<const uint16_t*>(p)[at] << 16);
}

template <int D, bool F32>
__global__ __launch_bounds__(256) void pages_score_kernel(const PagesSelectArgs a, const int blocks) {
  __shared__ double q_s[HEADS_AT_ONCE][D];
  const int heads = a.c.heads;
  const int place = (int)(blockIdx.x % (unsigned)blocks) * 256 + threadIdx.x;
  unsigned unit = blockIdx.x / (unsigned)blocks;
  const int h = (int)(unit % (unsigned)heads);
  unit /= (unsigned)heads;
  const int s = (int)(unit / (unsigned)a.b.max_new), t = (int)(unit % (unsigned)a.b.max_new);
  const int whole = a.b.count(s);
  const int64_t row = a.b.first_row(s) + t;
  if (t >= whole || row < 0 || row >= a.b.n_rows) return;
  const int pos = a.b.lens[s] - whole + t;
  const int last = pos >= 0 ? pos >> a.c.log2_page : -1;
  const bool open = place <= last && place < a.b.width;
  const int p = open ? a.b.table[(int64_t)s * a.b.table_stride + place] : -1;
  const bool there = open && p >= 0 && p < a.c.n_pages;
  const uint16_t* const lo = a.c.bounds + ((int64_t)(there ? p : 0) * heads + h) * (2 * D);
  float best = -INFINITY;
  bool nan = false;
  for (int g0 = 0; g0 < a.group; g0 += HEADS_AT_ONCE) {
    __syncthreads();
    for (int i = threadIdx.x; i < HEADS_AT_ONCE * D; i += 256) {
      const int g = g0 + i / D < a.group ? g0 + i / D : a.group - 1;
      q_s[i / D][i % D] = (double)load_value(a.q.p, row * a.q.ld_row + (h * a.group + g) * a.q.ld_head + i % D, F32);
    }
    __syncthreads();
    double sum[HEADS_AT_ONCE] = {};
    if (there)
      for (int j = 0; j < D; ++j) {
        const double x = (double)__uint_as_float((uint32_t)lo[j] << 16), y = (double)__uint_as_float((uint32_t)lo[D + j] << 16);
#pragma unroll
        for (int g = 0; g < HEADS_AT_ONCE; ++g) {
          const double f = q_s[g][j];
          sum[g] += f > 0. ? f * y : f * x;
        }
      }
#pragma unroll
    for (int g = 0; g < HEADS_AT_ONCE; ++g) {
      const float v = (float)sum[g];
      nan |= v != v;
      best = fmaxf(best, v);
    }
  }
  if (place >= a.b.width) return;
  uint32_t word = 0;
  if (there) {
    const uint32_t b = __float_as_uint(best + 0.f);
    word = nan ? 1u : b ^ ((b >> 31) ? 0xffffffffu : 0x80000000u);
    if (place < a.keep_first || place > last - a.keep_last) word = 0xffffffffu;
  }
  reinterpret_cast<uint32_t*>(a.scores)[(row * heads + h) * a.b.width + place] = word;
}

template <int THREADS>
__global__ __launch_bounds__(THREADS) void pages_pick_kernel(const PagesSelectArgs a) {
  constexpr int WAVES = THREADS / 64;
  __shared__ int count_s[256];
  __shared__ int found_s[3];  // byte of the last wanted word, words above it, words of this byte
  __shared__ int above_s[WAVES], equal_s[WAVES];
  const int heads = a.c.heads, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  unsigned unit = blockIdx.x;
  const int h = (int)(unit % (unsigned)heads);
  unit /= (unsigned)heads;
  const int s = (int)(unit / (unsigned)a.b.max_new), t = (int)(unit % (unsigned)a.b.max_new);
  const int whole = a.b.count(s);
  const int64_t row = a.b.first_row(s) + t;
  if (t >= whole || row < 0 || row >= a.b.n_rows) return;
  const int pos = a.b.lens[s] - whole + t;
  const int n = pos >= 0 ? min((pos >> a.c.log2_page) + 1, a.b.width) : 0;
  const uint32_t* const words = reinterpret_cast<const uint32_t*>(a.scores) + (row * heads + h) * a.b.width;
  int32_t* const out = a.chosen + (row * heads + h) * a.n_chosen;

  // the n_chosen-th largest word: `bar`; `room` of its equals are taken
  uint32_t bar = 0, known = 0;
  int room = a.n_chosen;
  for (int shift = 24; shift >= 0; shift -= 8) {
    for (int i = tid; i < 256; i += THREADS) count_s[i] = 0;
    __syncthreads();
    for (int i = tid; i < n; i += THREADS) {
      const uint32_t w = words[i];
      if (w != 0 && (w & known) == bar) atomicAdd(&count_s[(w >> shift) & 255], 1);
    }
    __syncthreads();
    if (wave == 0) {
      // from the highest byte down: lane holds bytes 255 - 4 lane - 0..3
      int c[4], sum = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) c[i] = count_s[255 - 4 * lane - i], sum += c[i];
      int upto = sum;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int v = __shfl_up(upto, o);
        if (lane >= o) upto += v;
      }
      const int total = __shfl(upto, 63);
      if (lane == 0 && total < room) found_s[0] = -1;  // fewer pages than places: all of them
      int over = upto - sum;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (over < room && over + c[i] >= room) found_s[0] = 255 - 4 * lane - i, found_s[1] = over;
        over += c[i];
      }
    }
    __syncthreads();
    if (found_s[0] < 0) {  // (only before the first byte is known)
      bar = 0;
      room = 0;
      break;
    }
    bar |= (uint32_t)found_s[0] << shift;
    known |= 0xffu << shift;
    room -= found_s[1];
    __syncthreads();
  }

  int above = 0, equal = 0;  // of the places before this block of THREADS
  for (int i0 = 0; i0 < n; i0 += THREADS) {
    const uint32_t w = i0 + tid < n ? words[i0 + tid] : 0;
    const uint64_t more = __builtin_amdgcn_ballot_w64(w > bar), same = __builtin_amdgcn_ballot_w64(w == bar && w != 0);
    __syncthreads();
    if (lane == 0) above_s[wave] = __popcll(more), equal_s[wave] = __popcll(same);
    __syncthreads();
    const uint64_t before = (1ull << lane) - 1;
    int more_before = above + __popcll(more & before), same_before = equal + __popcll(same & before);
#pragma unroll
    for (int v = 0; v < WAVES; ++v) {
      if (v < wave) more_before += above_s[v], same_before += equal_s[v];
      above += above_s[v];
      equal += equal_s[v];
    }
    const bool take = w > bar || (w == bar && w != 0 && same_before < room);
    if (take) out[more_before + min(same_before, room)] = i0 + tid;
  }
  for (int i = above + min(equal, room) + tid; i < a.n_chosen; i += THREADS) out[i] = -1;
}

template <int D>
hipError_t launch(bool f32, const PagesSelectArgs& a, hipStream_t s) {
  const int64_t units = (int64_t)a.b.n_seqs * a.b.max_new * a.c.heads;
  const int blocks = (a.b.width + 255) / 256;
  const dim3 grid((unsigned)(units * blocks));
  if (blocks > 0) {
    if (f32) hipLaunchKernelGGL((pages_score_kernel<D, true>), grid, dim3(256), 0, s, a, blocks);
    else hipLaunchKernelGGL((pages_score_kernel<D, false>), grid, dim3(256), 0, s, a, blocks);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (a.b.width > 2048) hipLaunchKernelGGL((pages_pick_kernel<1024>), dim3((unsigned)units), dim3(1024), 0, s, a);
  else hipLaunchKernelGGL((pages_pick_kernel<256>), dim3((unsigned)units), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_pages_select(int d, bool f32, const PagesSelectArgs& a, hipStream_t s) {
  return d == 64 ? launch<64>(f32, a, s) : d == 128 ? launch<128>(f32, a, s) : launch<256>(f32, a, s);
}

}  // namespace tq
