// Choosing pages by the bounds of their keys.
//
// No key k with lo <= k <= hi has <q, k> above sum_j max(q_j lo_j, q_j hi_j): none of a page's keys as they were appended; their codes may lie
// beyond by a rounding.  The sums are taken in 64 bits (a
// product of two bf16 values is exact there, and so is the sum of a page's products unless they are 2^30 apart) and rounded to fp32
// once: which page is chosen does not depend on the order of a sum.
//
// pages_score_kernel writes one word for every page that a row may choose, ordered like its rank: 0 no page, 1 NaN, then the
// scores' bits in an order of unsigned numbers, all ones for pages that are kept.  Sixteen lanes share a page (a lane has d / 16
// channels of both bounds) and add up by halves: of 16 sums (4 pages of a lane group x 4 query heads) every lane ends with one.
// 2048 pages of four rows, 8 x 4 heads of d = 128, 33.6 MB: 10.6 us, 3.2 TB/s; the wavefronts wait 81 % of their time (SQ_WAIT_ANY), vector
// instructions take 4.5 us at four cycles each.  A thread to a page instead read 512 bytes apart.
// pages_pick_kernel finds the n_chosen-th largest word by its leading bits (counts of up to 256 values of the next eight, from the first
// bit on in which the words differ) and writes the places of what is above it, and of as many equal ones as there is room for,
// lowest first.
#include "tq_pages.h"

namespace tq {

namespace {

__device__ __forceinline__ float load_value(const void* p, int64_t at, bool f32) {
  return f32 ? static_cast<const float*>(p)[at] : __uint_as_float((uint32_t)static_cast<const uint16_t*>(p)[at] << 16);
}

template <int CTRL>
__device__ __forceinline__ double dpp(double v) {
  const uint64_t b = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)b, CTRL, 0xf, 0xf, true);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(b >> 32), CTRL, 0xf, 0xf, true);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}
constexpr int XOR1 = 0xB1, XOR2 = 0x4E, HALF_MIRROR = 0x141, ROR8 = 0x128;

// N sums over 16 lanes, one step: the lane whose bit S is set keeps the upper half of the sums, its partner (CTRL, in which bit S is
// the other) the lower half; a single sum is added in both
template <int S, int CTRL, int N, int V>
__device__ __forceinline__ void add_halves(double (&v)[V]) {
  const bool upper = (threadIdx.x & S) != 0;
  if constexpr (N == 1) {
    v[0] += dpp<CTRL>(v[0]);
  } else {
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
      const double mine = upper ? v[i + N / 2] : v[i], other = upper ? v[i] : v[i + N / 2];
      v[i] = mine + dpp<CTRL>(other);
    }
  }
}

constexpr int pages_at_once(int heads) { return heads == 1 ? 8 : 4; }  // of a group of 16 lanes: 8 sums, or 16 for four heads

template <int D, bool F32, int G>
__global__ __launch_bounds__(256) void pages_score_kernel(const PagesSelectArgs a, const int steps) {
  constexpr int C = D / 16;                 // channels of a lane
  constexpr int U = pages_at_once(G), V = U * G;
  __shared__ double q_s[G][C][16][2];  // what is positive of a query's value, and what is negative: q_j > 0 ? q_j upper_j : q_j lower_j is a sum of two
  const int heads = a.c.heads, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, j = lane & 15, lanes = lane >> 4;
  const uint32_t unit = a.by_blocks.of(blockIdx.x), new_row = a.by_heads.of(unit);
  const int block = (int)a.by_blocks.rest(blockIdx.x, unit), h = (int)a.by_heads.rest(unit, new_row);
  const int s = (int)a.by_new.of(new_row), t = (int)a.by_new.rest(new_row, (uint32_t)s);
  const int whole = a.b.count(s);
  const int64_t row = a.b.first_row(s) + t;
  if (t >= whole || row < 0 || row >= a.b.n_rows) return;
  const int64_t pos = (int64_t)a.b.lens[s] - whole + t;
  const int last = pos >= 0 ? (int)(pos >> a.c.log2_page) : -1;
  const int n = min(last + 1, a.b.width);
  // a wavefront: `steps` times 4 U pages
  const int first = (block * 4 + wave) * steps * (4 * U);
  if (block * 4 * steps * (4 * U) >= n) return;  // (the whole workgroup)
  const int32_t* const table = a.b.table + (int64_t)s * a.b.table_stride;
  uint32_t* const words = reinterpret_cast<uint32_t*>(a.scores) + (row * heads + h) * a.b.width;

  const auto stage = [&](int g0) {
    for (int i = threadIdx.x; i < G * D; i += 256) {
      const int g = g0 + i / D < a.group ? g0 + i / D : a.group - 1, c = i % D;
      const double x = (double)load_value(a.q.p, row * a.q.ld_row + (h * a.group + g) * a.q.ld_head + c, F32);
      q_s[i / D][c % C][c / C][0] = x > 0. ? x : 0.;
      q_s[i / D][c % C][c / C][1] = x > 0. ? 0. : x;  // (NaN is kept)
    }
    __syncthreads();
  };
  if (a.group <= G) stage(0);

  // A page's sum as the definition has it, by one lane: the sum of two above has 0 * inf where the side that is not taken has no bound.
  const auto defined = [&](int p, int g) {
    const uint16_t* const from = a.c.bounds + ((int64_t)p * heads + h) * (2 * D);
    double sum = 0.;
    for (int c0 = 0; c0 < D && sum == sum; c0 += 8) {
      const uint4_t low = *reinterpret_cast<const uint4_t*>(from + c0), high = *reinterpret_cast<const uint4_t*>(from + D + c0);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int c = c0 + i;
        const double x = q_s[g][c % C][c / C][0] + q_s[g][c % C][c / C][1];
        const float l = __uint_as_float((i & 1) ? low[i >> 1] & 0xffff0000u : low[i >> 1] << 16);
        const float u = __uint_as_float((i & 1) ? high[i >> 1] & 0xffff0000u : high[i >> 1] << 16);
        if (x != x || l != l || u != u) sum = __builtin_nan("");
        else if (x != 0.) sum = fma(x, (double)(x > 0. ? u : l), sum);
      }
    }
    return (float)sum;
  };

  for (int step = 0; step < steps; ++step) {
    const int base = first + step * (4 * U);
    bool there[U];
    uint32_t lo[U][C / 2], hi[U][C / 2];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int place = base + 4 * u + lanes, p = place < n ? table[place] : -1;
      there[u] = p >= 0 && p < a.c.n_pages;
      const uint16_t* const from = a.c.bounds + ((int64_t)(there[u] ? p : 0) * heads + h) * (2 * D) + j * C;
#pragma unroll
      for (int c = 0; c < C / 2; c += 4 < C / 2 ? 4 : C / 2) {
        if constexpr (C == 4) {
          *reinterpret_cast<uint2_t*>(&lo[u][c]) = *reinterpret_cast<const uint2_t*>(from + 2 * c);
          *reinterpret_cast<uint2_t*>(&hi[u][c]) = *reinterpret_cast<const uint2_t*>(from + D + 2 * c);
        } else {
          *reinterpret_cast<uint4_t*>(&lo[u][c]) = *reinterpret_cast<const uint4_t*>(from + 2 * c);
          *reinterpret_cast<uint4_t*>(&hi[u][c]) = *reinterpret_cast<const uint4_t*>(from + D + 2 * c);
        }
      }
    }
    float best = -INFINITY;
    bool nan = false;
    for (int g0 = 0; g0 < a.group; g0 += G) {
      if (a.group > G) {
        __syncthreads();
        stage(g0);
      }
      // (else the compiler turns all channels before the loop over the heads, into 64 to 256 registers)
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int c = 0; c < C / 2; ++c) asm("" : "+v"(lo[u][c]), "+v"(hi[u][c]));
      double sum[V] = {};
#pragma unroll
      for (int c = 0; c < C; ++c) {
        double low[U], high[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          low[u] = (double)__uint_as_float((c & 1) ? lo[u][c / 2] & 0xffff0000u : lo[u][c / 2] << 16);
          high[u] = (double)__uint_as_float((c & 1) ? hi[u][c / 2] & 0xffff0000u : hi[u][c / 2] << 16);
        }
#pragma unroll
        for (int g = 0; g < G; ++g) {
          const double above = q_s[g][c][j][0], below = q_s[g][c][j][1];
#pragma unroll
          for (int u = 0; u < U; ++u) sum[u * G + g] = fma(above, high[u], fma(below, low[u], sum[u * G + g]));
        }
      }
      add_halves<8, ROR8, V>(sum);
      add_halves<4, HALF_MIRROR, V / 2>(sum);
      add_halves<2, XOR2, V / 4>(sum);
      add_halves<1, XOR1, V / 8>(sum);
      // lane j (of eight sums: lanes 2 i and 2 i + 1) has the sum of page sum / G of the lane group and head sum % G
      float v = (float)sum[0];
      if (v != v) {
        const int i = V == 16 ? j : j >> 1, place = base + 4 * (i / G) + lanes, p = place < n ? table[place] : -1;
        if (p >= 0 && p < a.c.n_pages) v = defined(p, i % G);
      }
      nan |= v != v;
      best = fmaxf(best, v);
    }
    uint32_t rank = nan ? 1u : 0u;
    if (rank == 0) {
      const uint32_t bits = __float_as_uint(best + 0.f);
      rank = bits ^ ((bits >> 31) ? 0xffffffffu : 0x80000000u);
    }
    // the best of the heads; a NaN of one is the page's
    constexpr int HEAD_BITS = G == 1 ? 0 : G == 2 ? 2 : 3;  // lane bits that are the head's
    const auto merge = [&](uint32_t x) { rank = rank == 1u || x == 1u ? 1u : max(rank, x); };
    if constexpr ((HEAD_BITS & 1) != 0) merge((uint32_t)__builtin_amdgcn_update_dpp(0, (int)rank, XOR1, 0xf, 0xf, true));
    if constexpr ((HEAD_BITS & 2) != 0) merge((uint32_t)__builtin_amdgcn_update_dpp(0, (int)rank, XOR2, 0xf, 0xf, true));
    const int u = (V == 16 ? j : j >> 1) / G, place = base + 4 * u + lanes;
    bool is = false;
#pragma unroll
    for (int i = 0; i < U; ++i) is = i == u ? there[i] : is;
    if (place < a.keep_first || place > last - a.keep_last) rank = 0xffffffffu;
    if ((j & (16 / U - 1)) == 0 && place < n) words[place] = is ? rank : 0u;
  }
}

// sums of the lanes up to and with this one
__device__ __forceinline__ int scan_wavefront(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);  // row_shr 1, 2, 4, 8
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);  // the last lane of a row to the next, of two rows to the next two
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);
  return v;
}

template <int THREADS, int HELD>
__global__ __launch_bounds__(THREADS) void pages_pick_kernel(const PagesSelectArgs a) {
  constexpr int WAVES = THREADS / 64;
  __shared__ int count_s[4][256];
  static_assert(HELD * WAVES <= 64, "a lane for each");
  __shared__ int sum_s[64];
  __shared__ int kept_s[2][WAVES];
  __shared__ uint32_t range_s[2][WAVES];
  const int heads = a.c.heads, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const uint32_t new_row = a.by_heads.of(blockIdx.x);
  const int h = (int)a.by_heads.rest(blockIdx.x, new_row), s = (int)a.by_new.of(new_row), t = (int)a.by_new.rest(new_row, (uint32_t)s);
  const int whole = a.b.count(s);
  const int64_t row = a.b.first_row(s) + t;
  if (t >= whole || row < 0 || row >= a.b.n_rows) return;
  const uint32_t* const words = reinterpret_cast<const uint32_t*>(a.scores) + (row * heads + h) * a.b.width;
  int32_t* const out = a.chosen + (row * heads + h) * a.n_chosen;

  // places tid, tid + THREADS, ..: the first HELD of a thread in registers
  uint32_t held[HELD];
#pragma unroll
  for (int i = 0; i < HELD; ++i) held[i] = i * THREADS + tid < a.b.width ? words[i * THREADS + tid] : 0u;
  const int64_t pos = (int64_t)a.b.lens[s] - whole + t;
  const int n = pos >= 0 ? min((int)(pos >> a.c.log2_page) + 1, a.b.width) : 0;
#pragma unroll
  for (int i = 0; i < HELD; ++i) held[i] = i * THREADS + tid < n ? held[i] : 0u;  // (behind the row's last page nothing has been written)
  const auto each = [&](auto f) {
#pragma unroll
    for (int i = 0; i < HELD; ++i) f(held[i]);
    for (int i = HELD * THREADS + tid; i < n; i += THREADS) f(words[i]);
  };
  for (int i = tid; i < 4 * 256; i += THREADS) count_s[i >> 8][i & 255] = 0;

  // pages that are kept, others, and the others' range
  int kept = 0, others = 0;
  uint32_t least = 0xffffffffu, most = 0;
  each([&](uint32_t w) {
    const bool other = w != 0 && w != 0xffffffffu;
    kept += w == 0xffffffffu ? 1 : 0;
    others += other ? 1 : 0;
    least = min(least, other ? w : 0xffffffffu), most = max(most, other ? w : 0u);
  });
  const auto add = [](int x, int y) { return x + y; };
  kept = over_wavefront(kept, add), others = over_wavefront(others, add);
  least = over_wavefront(least, [](uint32_t x, uint32_t y) { return x < y ? x : y; });
  most = over_wavefront(most, [](uint32_t x, uint32_t y) { return x > y ? x : y; });
  if (lane == 0) kept_s[0][wave] = kept, kept_s[1][wave] = others, range_s[0][wave] = least, range_s[1][wave] = most;
  __syncthreads();
  kept = others = 0;
#pragma unroll
  for (int v = 0; v < WAVES; ++v) kept += kept_s[0][v], others += kept_s[1][v], least = min(least, range_s[0][v]), most = max(most, range_s[1][v]);

  // what is taken: kept pages, words whose bits from `shift` on are above `bar`, and the first `room` places of those that equal it
  uint32_t bar = 0;
  int shift = 0, room = a.n_chosen - kept;
  if (room == 0) {
    bar = 0xffffffffu;
  } else if (others > room) {
    shift = least == most ? 0 : 32 - __builtin_clz(least ^ most);
    bar = shift < 32 ? most >> shift : 0u;
    for (int pass = 0; shift > 0; ++pass) {
      const int bits = shift < 8 ? shift : 8, next = shift - bits;
      each([&](uint32_t w) {
        if (w != 0 && w != 0xffffffffu && (shift == 32 || (w >> shift) == bar)) atomicAdd(&count_s[pass][(w >> next) & ((1u << bits) - 1)], 1);
      });
      __syncthreads();
      // every wavefront for itself, from the highest value down: lane holds 255 - 4 lane - 0..3
      int c[4], sum = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) c[i] = count_s[pass][255 - 4 * lane - i], sum += c[i];
      const int upto = scan_wavefront(sum);
      int over = upto - sum, value = 0, here = 0, many = 0;
      bool mine = false;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (over < room && over + c[i] >= room) mine = true, value = 255 - 4 * lane - i, here = over, many = c[i];
        over += c[i];
      }
      const int from = __builtin_ctzll(__builtin_amdgcn_ballot_w64(mine));  // one lane has it: there are at least `room` of these words
      value = __builtin_amdgcn_readlane(value, from), here = __builtin_amdgcn_readlane(here, from), many = __builtin_amdgcn_readlane(many, from);
      bar = (shift == 32 ? 0u : bar << bits) | (uint32_t)value;
      room -= here;
      shift = next;
      if (many == room) break;  // all of them
    }
  }

  const auto over = [&](uint32_t w) { return w == 0xffffffffu || (w != 0 && (w >> shift) > bar); };
  const auto level = [&](uint32_t w) { return w != 0 && w != 0xffffffffu && (w >> shift) == bar; };
  const uint64_t before = (1ull << lane) - 1;
  int above = 0, equal = 0;  // of the places so far
  for (int i0 = 0; i0 < n; i0 += HELD * THREADS) {
    if (i0 > 0) {
#pragma unroll
      for (int i = 0; i < HELD; ++i) held[i] = i0 + i * THREADS + tid < n ? words[i0 + i * THREADS + tid] : 0u;
    }
    __syncthreads();
    // 64 places each in the order of the places: those above the bar in the lower half of a word, its equals in the upper
    uint64_t more[HELD], same[HELD];
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
      more[i] = __builtin_amdgcn_ballot_w64(over(held[i])), same[i] = __builtin_amdgcn_ballot_w64(level(held[i]));
      if (lane == 0) sum_s[i * WAVES + wave] = __popcll(more[i]) | __popcll(same[i]) << 16;
    }
    __syncthreads();
    const int own = lane < HELD * WAVES ? sum_s[lane] : 0;
    int upto = scan_wavefront(own);
    const int all = __builtin_amdgcn_readlane(upto, HELD * WAVES - 1);
    upto -= own;
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
      const int start = __builtin_amdgcn_readlane(upto, i * WAVES + wave);
      const int more_before = above + (start & 0xffff) + __popcll(more[i] & before), same_before = equal + (start >> 16) + __popcll(same[i] & before);
      if (over(held[i]) || (level(held[i]) && same_before < room)) out[more_before + min(same_before, room)] = i0 + i * THREADS + tid;
    }
    above += all & 0xffff, equal += all >> 16;
  }
  for (int i = above + min(equal, room) + tid; i < a.n_chosen; i += THREADS) out[i] = -1;
}

// of a workgroup that chooses from `width` pages
int pick_threads(int width) { return width > 4096 ? 1024 : width > 1024 ? 512 : 256; }

template <int D, bool F32, int G>
hipError_t launch_score(PagesSelectArgs a, int64_t units, hipStream_t s) {
  // a wavefront takes a step (16 or 32 pages), up to eight where that leaves three workgroups for a compute unit.  Four rows of 8 heads and
  // 2048 pages, both kernels: one 25.2 us, two 21.2, three and more 19.3
  constexpr int per = 4 * 4 * pages_at_once(G);
  const int64_t all = (a.b.width + per - 1) / per;
  int64_t steps = units * all / (3 * device_cu_count());
  steps = steps < 1 ? 1 : steps > 8 ? 8 : steps;
  const int64_t blocks = (all + steps - 1) / steps;
  if (!grid_fits(units * blocks, 256)) return hipErrorInvalidConfiguration;
  a.by_blocks = Divide(blocks);
  hipLaunchKernelGGL((pages_score_kernel<D, F32, G>), dim3((unsigned)(units * blocks)), dim3(256), 0, s, a, (int)steps);
  return hipGetLastError();
}
template <int D, bool F32>
hipError_t launch_score_g(const PagesSelectArgs& a, int64_t units, hipStream_t s) {
  if (a.group == 1) return launch_score<D, F32, 1>(a, units, s);
  if (a.group == 2) return launch_score<D, F32, 2>(a, units, s);
  return launch_score<D, F32, 4>(a, units, s);
}

template <int D>
hipError_t launch(bool f32, PagesSelectArgs a, hipStream_t s) {
  a.by_heads = Divide(a.c.heads), a.by_new = Divide(a.b.max_new);
  const int64_t units = (int64_t)a.b.n_seqs * a.b.max_new * a.c.heads;
  if (!pages_pick_fits(a.b, a.c.heads)) return hipErrorInvalidConfiguration;
  if (a.b.width > 0) {
    const hipError_t e = f32 ? launch_score_g<D, true>(a, units, s) : launch_score_g<D, false>(a, units, s);
    if (e != hipSuccess) return e;
  }
  const dim3 grid((unsigned)units);
  const int threads = pick_threads(a.b.width);
  if (threads == 1024) hipLaunchKernelGGL((pages_pick_kernel<1024, 4>), grid, dim3(1024), 0, s, a);
  else if (threads == 512) hipLaunchKernelGGL((pages_pick_kernel<512, 8>), grid, dim3(512), 0, s, a);
  else hipLaunchKernelGGL((pages_pick_kernel<256, 4>), grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace

bool pages_pick_fits(const BatchView& b, int heads) { return grid_fits((int64_t)b.n_seqs * b.max_new * heads, pick_threads(b.width)); }

hipError_t launch_pages_select(int d, bool f32, const PagesSelectArgs& a, hipStream_t s) {
  return d == 64 ? launch<64>(f32, a, s) : d == 128 ? launch<128>(f32, a, s) : launch<256>(f32, a, s);
}

}  // namespace tq
