// Attention over pages of 8-bit keys and values.
//
//   out = sum_j softmax_j(scale <q, k_j>) v_j,  one pass over the keys with the running maximum and sum of the softmax.
//
// A wavefront has 16 rows (of one sequence and head of the cache: its new tokens times the query heads that read this head) and walks
// the keys in tiles of 32, two subtiles of 16; a subtile never leaves a page.  Products on v_mfma_f32_16x16x32:
//   S^T = K Q^T    A = 16 keys, B = 16 rows.  The codes are exact in bf16; so is a bf16 query, an fp32 one is three bf16 pieces.
//                  Lane (r = lane % 16, g = lane / 16) has row r of a subtile's keys, bytes [g d / 4, (g + 1) d / 4): which
//                  coordinate is which k of the product does not matter as long as both sides agree.
//   O^T += V^T P^T A = 16 coordinates, B = 16 rows, k = 32 keys.  S^T leaves lane (r, g) with the weights of row r and the keys
//                  4 g + 0..3 of both subtiles, which are eight k of this product already: no weight changes its lane.  The lane
//                  fetches the same eight keys' coordinates [r d / 16, (r + 1) d / 16) and turns them by 4 x 4 bytes in
//                  registers.  The codes are exact in fp16; the weights are fp16 (two pieces for an fp32 output).
// With C the base-2 logarithm, lane sums and frames are:  x = log2(e) scale s + log2(v_scale) - M + BASE,  w = 2^x,
// O = sum w c_v,  l = sum w / v_scale; M is the largest log2(e) scale s + log2(v_scale) so far or up to HEAD below it (a new M costs
// a pass over O, so it is taken only where a weight would leave fp16's range).  The scale of a value block sits in the exponent of
// its weights and never costs a product.  With |log2 v_scale| <= 40 what a weight that underflows (2^-126, the largest is 2^BASE or
// more) would add to l is less than 2^-50 of it.
#include "tq_pages_attend.h"

namespace tq {

namespace {

// a tile on its way: 32 keys and values, and what its two subtiles are
template <int D>
struct Tile {
  uint32_t k[2][D / 16], v[8][D / 64];
  int pos[2];             // of the subtile's first token (NOWHERE where its page is none)
  float ks[2], lv[2], iv[2];  // scale of its keys, base-2 logarithm and inverse of that of its values
};

constexpr int WAVES = kPagesAttendWaves;

// What a range of keys leaves for pages_join_kernel: [0] M, [1] l, [4, 4 + D) O.
template <int D>
constexpr int kPart = 4 + D;

// What a wavefront does: R tiles of 16 rows of a unit (a sequence and head; a row and head where the pages are chosen) against keys.
template <int D, int CT, bool F32, int R>
struct Walk {
  static constexpr int KS = D / 32;  // k steps of S, and pieces of eight bytes of a lane's keys
  static constexpr int VE = D / 16;  // coordinates of a lane's values
  static constexpr int QP = F32 ? 3 : 1;

  const PagesAttendArgs& a;
  int lane, r, g, heads, h;
  // the unit's rows; of the lane's own rows positions, and the tiles' smallest and largest
  int rows, t0;
  int64_t row0;
  int pos[R], pos_lo, pos_hi;
  // keys [lo, hi) of the sequence, or of the chosen pages put together
  int lo, hi;
  const int32_t *table, *list;
  bool listed;
  // a lane knows one subtile of the next 64
  int begin;
  Subtile sub;
  bf16x8_t q[R][QP][KS];
  float4_t o[R][VE];
  float l[R], M[R], shift[R], limit[R];  // shift = BASE - M, limit: of x before a new M is taken

  __device__ __forceinline__ explicit Walk(const PagesAttendArgs& args) : a(args) {}

  __device__ __forceinline__ int token_of(int m) const { return (int)a.by_group.of((uint32_t)m); }
  __device__ __forceinline__ int64_t row_of(int m) const { return row0 + t0 + token_of(m); }
  __device__ __forceinline__ int head_of(int m) const { return h * a.group + m - token_of(m) * a.group; }

  // the unit and its rows [first, first + 16 R); false: there are none
  __device__ __forceinline__ bool start(unsigned unit, int first_row) {
    lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    heads = a.c.heads;
    const uint32_t rest = a.by_heads.of(unit);
    h = (int)a.by_heads.rest(unit, rest);
    const int s = a.chosen != nullptr ? (int)a.by_new.of(rest) : (int)rest;
    t0 = a.chosen != nullptr ? (int)a.by_new.rest(rest, (uint32_t)s) : 0;
    const int whole = a.b.count(s), count = min(whole, a.b.max_new);
    rows = (a.chosen != nullptr ? (t0 < count ? 1 : 0) : count) * a.group;
    if (first_row >= rows) return false;
    const int len = a.b.lens[s];
    row0 = a.b.first_row(s);
    const int64_t at0 = (int64_t)len - whole + t0;
    pos_lo = row_position(at0 + token_of(first_row)), pos_hi = row_position(at0 + token_of(min(first_row + 16 * R - 1, rows - 1)));
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int m = min(first_row + 16 * i + r, rows - 1);
      const int64_t row = row_of(m);
      const bool there = first_row + 16 * i + r < rows && row >= 0 && row < a.b.n_rows;
      pos[i] = row_position(at0 + token_of(m));
      load_query(i, there, row * a.q.ld_row + head_of(m) * a.q.ld_head + g * (D / 4));
#pragma unroll
      for (int e = 0; e < VE; ++e) o[i][e] = float4_t{0.f, 0.f, 0.f, 0.f};
      l[i] = 0.f, M[i] = -INFINITY, shift[i] = 0.f, limit[i] = -3e38f;
    }
    const int64_t bound = (int64_t)a.b.width << a.c.log2_page;
    lo = 0;
    if (a.chosen != nullptr) {
      hi = a.n_chosen << a.c.log2_page;  // (at most 2^31 - 128: tq_pages_attend)
    } else {
      hi = (int)min((int64_t)pos_hi + 1, bound);
      lo = (int)max((int64_t)0, (int64_t)pos_lo - a.window + 1) & ~31;
    }
    table = a.b.table + (int64_t)s * a.b.table_stride;
    list = a.chosen != nullptr ? a.chosen + ((row0 + t0) * heads + h) * a.n_chosen : nullptr;
    listed = a.chosen == nullptr || (row0 + t0 >= 0 && row0 + t0 < a.b.n_rows);
    return true;
  }
  __device__ __forceinline__ int tiles() const { return hi > lo ? (hi - lo + 31) >> 5 : 0; }

  __device__ __forceinline__ void load_query(int i, bool there, int64_t from) {
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      const int64_t at = from + 8 * k;
      if constexpr (F32) {
        float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (there) {
          const float4_t u = *reinterpret_cast<const float4_t*>(static_cast<const float*>(a.q.p) + at);
          const float4_t w = *reinterpret_cast<const float4_t*>(static_cast<const float*>(a.q.p) + at + 4);
#pragma unroll
          for (int e = 0; e < 4; ++e) x[e] = u[e], x[4 + e] = w[e];
        }
        // three pieces of eight bits: what a rounding leaves is exact in fp32 (an infinite value's pieces: itself and NaN)
#pragma unroll
        for (int p = 0; p < 3; ++p)
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            q[i][p][k][e] = (__bf16)x[e];
            x[e] -= (float)q[i][p][k][e];
          }
      } else {
        union {
          uint4_t w;
          bf16x8_t v;
        } u;
        u.w = uint4_t{0, 0, 0, 0};
        if (there) u.w = *reinterpret_cast<const uint4_t*>(static_cast<const uint16_t*>(a.q.p) + at);
        q[i][0][k] = u.v;
      }
    }
  }

  __device__ __forceinline__ void look_up(int first) {
    const int64_t at = (int64_t)lo + 16 * ((int64_t)2 * first + lane);
    sub = no_subtile();
    if (at < hi && listed) {
      const int i = (int)(at >> a.c.log2_page);
      sub = find_subtile(a.c, table, a.b.width, h, list != nullptr ? list[i] : i, (int)at & ((1 << a.c.log2_page) - 1));
    }
  }

  __device__ __forceinline__ void load(Tile<D>& b, int i) {
    if (((i - begin) & 31) == 0) look_up(i);
    const int from = ((i - begin) & 31) << 1;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int at = __builtin_amdgcn_readlane(sub.at, from + u);
      const int64_t off = (int64_t)(at < 0 ? 0 : at) * (16 * D);  // where there is no page, the pool's first bytes, unused
      const uint8_t* const kp = a.c.k + off + r * D + g * (D / 4);
#pragma unroll
      for (int j = 0; j < D / 64; ++j) *reinterpret_cast<uint4_t*>(&b.k[u][4 * j]) = *reinterpret_cast<const uint4_t*>(kp + 16 * j);
      const uint8_t* const vp = a.c.v + off + 4 * g * D + r * VE;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        uint32_t* const to = b.v[4 * u + j];
        if constexpr (D == 64) to[0] = *reinterpret_cast<const uint32_t*>(vp + j * D);
        if constexpr (D == 128) *reinterpret_cast<uint2_t*>(to) = *reinterpret_cast<const uint2_t*>(vp + j * D);
        if constexpr (D == 256) *reinterpret_cast<uint4_t*>(to) = *reinterpret_cast<const uint4_t*>(vp + j * D);
      }
    }
    // (behind the loads: these wait for the scales)
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      b.pos[u] = __builtin_amdgcn_readlane(sub.pos, from + u);
      b.ks[u] = lane_value(sub.ks, from + u), b.lv[u] = lane_value(sub.lv, from + u), b.iv[u] = lane_value(sub.iv, from + u);
    }
  }

  // x of row tile i: base-2 logarithms of its weights in the frame
  __device__ __forceinline__ void exponents(float (&x)[8], const float4_t (&acc)[2], const Tile<D>& b, int i, uint32_t hidden) const {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const float ch = b.ks[u] * a.scale2, cl = b.ks[u] * a.scale2_rest, add = b.lv[u] + shift[i];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[4 * u + e] = fmaf(acc[u][e], ch, add);
        if (F32) x[4 * u + e] = fmaf(acc[u][e], cl, x[4 * u + e]);
      }
    }
    if (hidden != 0) {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if ((hidden >> j) & 1) x[j] = -INFINITY;
    }
  }

  __device__ __forceinline__ void step(Tile<D>& b) {
    float4_t acc[R][2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
#pragma unroll
      for (int i = 0; i < R; ++i) acc[i][u] = float4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        const bf16x8_t f = codes_bf16<CT>(b.k[u][2 * k], b.k[u][2 * k + 1]);
#pragma unroll
        for (int i = 0; i < R; ++i)
#pragma unroll
          for (int p = QP - 1; p >= 0; --p) acc[i][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, q[i][p][k], acc[i][u], 0, 0, 0);
      }
    }
    // all rows see the whole tile, or some do not
    const bool inner = max(b.pos[0], b.pos[1]) + 15 <= pos_lo && (int64_t)min(b.pos[0], b.pos[1]) > (int64_t)pos_hi - a.window;
    uint32_t poison = 0;
    if (CT == kPageE4m3 && !inner) {
      // 0 * NaN is NaN: a NaN among the values leaves the product, and comes back by the weights of the rows that see it
      uint32_t any = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int w = 0; w < D / 64; ++w) any |= nan_bytes(b.v[j][w]);
      if (__builtin_amdgcn_ballot_w64(any != 0) != 0) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          uint32_t here = 0;
#pragma unroll
          for (int w = 0; w < D / 64; ++w) {
            const uint32_t n = nan_bytes(b.v[j][w]);
            b.v[j][w] &= ~n;
            here |= n;
          }
          const uint64_t lanes = __builtin_amdgcn_ballot_w64(here != 0);
          poison |= ((lanes >> (16 * g)) & 0xffffu) != 0 ? 1u << j : 0u;
        }
      }
    }
    half8_t p_hi[R], p_lo[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
      uint32_t hidden = 0;  // bit j: key j is not seen
      if (!inner) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int key = b.pos[j >> 2] + 4 * g + (j & 3);
          const bool seen = key <= pos[i] && (int64_t)key > (int64_t)pos[i] - a.window;
          hidden |= seen ? 0u : 1u << j;
          if (seen && ((poison >> j) & 1)) acc[i][j >> 2][j & 3] = __builtin_nanf("");
        }
      }
      float x[8];
      exponents(x, acc[i], b, i, hidden);
      float top = x[0];
#pragma unroll
      for (int j = 1; j < 8; ++j) top = fmaxf(top, x[j]);
      if (__builtin_amdgcn_ballot_w64(top > limit[i]) != 0) {
        const float next = fmaxf(M[i], swap_max(top) - shift[i]);
        const float down = M[i] == next || M[i] == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(M[i] - next);
        if (next != -INFINITY) {
          M[i] = next;
          shift[i] = BASE - next;
          limit[i] = BASE + HEAD;
        }
        l[i] *= down;
#pragma unroll
        for (int e = 0; e < VE; ++e) o[i][e] *= down;
        exponents(x, acc[i], b, i, hidden);
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float w = __builtin_amdgcn_exp2f(x[j]);
        l[i] = fmaf(w, b.iv[j >> 2], l[i]);
        p_hi[i][j] = (_Float16)w;
        if (F32) p_lo[i][j] = (_Float16)(w - (float)p_hi[i][j]);
      }
    }
#pragma unroll
    for (int e4 = 0; e4 < VE / 4; ++e4) {
      uint32_t turned[2][4];  // [subtile][coordinate]: four keys
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const uint32_t w0 = b.v[4 * u][e4], w1 = b.v[4 * u + 1][e4], w2 = b.v[4 * u + 2][e4], w3 = b.v[4 * u + 3][e4];
        const uint32_t a0 = __builtin_amdgcn_perm(w1, w0, 0x05010400u), a1 = __builtin_amdgcn_perm(w1, w0, 0x07030602u);
        const uint32_t b0 = __builtin_amdgcn_perm(w3, w2, 0x05010400u), b1 = __builtin_amdgcn_perm(w3, w2, 0x07030602u);
        turned[u][0] = __builtin_amdgcn_perm(b0, a0, 0x05040100u);
        turned[u][1] = __builtin_amdgcn_perm(b0, a0, 0x07060302u);
        turned[u][2] = __builtin_amdgcn_perm(b1, a1, 0x05040100u);
        turned[u][3] = __builtin_amdgcn_perm(b1, a1, 0x07060302u);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const half8_t f = codes_fp16<CT>(turned[0][e], turned[1][e]);
#pragma unroll
        for (int i = 0; i < R; ++i) {
          float4_t& to = o[i][4 * e4 + e];
          if (F32) to = __builtin_amdgcn_mfma_f32_16x16x32_f16(f, p_lo[i], to, 0, 0, 0);
          to = __builtin_amdgcn_mfma_f32_16x16x32_f16(f, p_hi[i], to, 0, 0, 0);
        }
      }
    }
  }

  // tiles [from, to); the next tile is asked for before a tile's products
  __device__ __forceinline__ void run(int from, int to) {
    begin = from;
    Tile<D> one, two;
    if (from < to) load(one, from);
    for (int i = from; i < to; i += 2) {
      if (i + 1 < to) load(two, i + 1);
      step(one);
      if (i + 1 < to) {
        if (i + 2 < to) load(one, i + 2);
        step(two);
      }
    }
  }
};

// One unit and 16 R rows to a workgroup, whose wavefronts share the keys of one range.
template <int D, int CT, bool F32, int R>
__global__ __launch_bounds__(64 * WAVES) void pages_attend_kernel(const PagesAttendArgs a) {
  constexpr int VE = D / 16;
  __shared__ float o_s[2][16][D + 4];
  __shared__ float ml_s[WAVES][16][2];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t ranged = a.by_splits.of(blockIdx.x), unit = a.by_tiles.of(ranged);
  const int split = (int)a.by_splits.rest(blockIdx.x, ranged), tile = (int)a.by_tiles.rest(ranged, unit);
  Walk<D, CT, F32, R> w(a);
  if (!w.start(unit, 16 * R * tile)) return;
  // this wavefront's tiles: an equal part of them, in one piece
  const int tiles = w.tiles(), each = (tiles + a.splits * WAVES - 1) / (a.splits * WAVES);
  const int begin = (split * WAVES + wave) * each;
  w.run(begin, min(begin + each, tiles));
  const int r = w.r, g = w.g, heads = w.heads, group = a.group;
#pragma unroll
  for (int i16 = 0; i16 < R; ++i16) {
    if (i16 > 0) __syncthreads();  // the sums of the 16 rows before are still read
    const float M = w.M[i16], l = swap_sum(w.l[i16]);

    // The wavefronts' sums in one frame.  Lane (r, g): row r, coordinates [g d / 4, (g + 1) d / 4): o[e][i] is coordinate g d / 4 + i d / 16 + e
    if (g == 0) ml_s[wave][r][0] = M, ml_s[wave][r][1] = l;
    __syncthreads();
    float top = ml_s[0][r][0];
#pragma unroll
    for (int i = 1; i < WAVES; ++i) top = fmaxf(top, ml_s[i][r][0]);
    const float down = M == -INFINITY && l == 0.f ? 0.f : M == top ? 1.f : __builtin_amdgcn_exp2f(M - top);
    float* const mine_s = &o_s[wave & 1][r][g * (D / 4)];
    for (int pair = 0; pair < WAVES; pair += 2) {
      if ((wave & ~1) == pair) {
#pragma unroll
        for (int c = 0; c < D / 4; c += 4) {
          float4_t y = {};
          if (pair != 0) y = *reinterpret_cast<const float4_t*>(mine_s + c);
#pragma unroll
          for (int i = 0; i < 4; ++i) y[i] += w.o[i16][(c + i) % VE][(c + i) / VE] * down;
          *reinterpret_cast<float4_t*>(mine_s + c) = y;
        }
      }
      __syncthreads();
    }

    // thread: one row, D / 16 coordinates of it
    const int out_r = threadIdx.x >> 4, first = (threadIdx.x & 15) * VE;
    const int m2 = (tile * R + i16) * 16 + out_r;
    if (m2 >= w.rows) continue;
    const int64_t row2 = w.row_of(m2);
    const int head2 = w.head_of(m2);
    if (row2 < 0 || row2 >= a.b.n_rows) continue;
    float m = ml_s[0][out_r][0], sum = 0.f;
#pragma unroll
    for (int i = 1; i < WAVES; ++i) m = fmaxf(m, ml_s[i][out_r][0]);
#pragma unroll
    for (int i = 0; i < WAVES; ++i) {
      const float mw = ml_s[i][out_r][0], lw = ml_s[i][out_r][1];
      sum += lw == 0.f ? 0.f : mw == m ? lw : lw * __builtin_amdgcn_exp2f(mw - m);
    }
    float y[VE];
#pragma unroll
    for (int c = 0; c < VE; c += 4) {
      const float4_t u = *reinterpret_cast<const float4_t*>(&o_s[0][out_r][first + c]), v = *reinterpret_cast<const float4_t*>(&o_s[1][out_r][first + c]);
#pragma unroll
      for (int i = 0; i < 4; ++i) y[c + i] = u[i] + v[i];
    }
    if (a.splits > 1) {
      float* const part = a.part + ((row2 * heads * group + head2) * a.splits + split) * kPart<D>;
#pragma unroll
      for (int c = 0; c < VE; c += 4) *reinterpret_cast<float4_t*>(part + 4 + first + c) = float4_t{y[c], y[c + 1], y[c + 2], y[c + 3]};
      if (first == 0) part[0] = m, part[1] = sum;
      continue;
    }
    store_row<VE, F32>(a.out, row2, head2, first, y, sum);
    if (a.lse != nullptr && first == 0) a.lse[row2 * heads * group + head2] = log_sum(m, sum);
  }
}

// The ranges of keys of a row and head in one frame: one wavefront for up to 16 of them, four (WIDE) for up to 64, 16 to each
// (32 ranges of 32 rows 4.0 -> 3.6 us, traced).
template <int D, bool F32, bool WIDE>
__global__ __launch_bounds__(256) void pages_join_kernel(const PagesAttendArgs a) {
  constexpr int VE = D / 64;
  __shared__ float y_s[WIDE ? 4 : 1][WIDE ? D + 4 : 1];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), heads = a.c.heads * a.group;
  const uint32_t item = WIDE ? blockIdx.x : blockIdx.x * 4 + (uint32_t)wave, token = a.by_queries.of(item);
  const int head = (int)a.by_queries.rest(item, token), s = (int)a.by_new.of(token), t = (int)a.by_new.rest(token, (uint32_t)s);
  if (s >= a.b.n_seqs || t >= a.b.count(s)) return;
  const int64_t row = a.b.first_row(s) + t;
  if (row < 0 || row >= a.b.n_rows) return;
  const int i0 = WIDE ? 16 * wave : 0, n = min(a.splits - i0, 16);  // this wavefront's ranges
  const float* const part = a.part + ((row * heads + head) * a.splits + i0) * kPart<D>;
  // everything is asked for before anything is waited for
  float x[16][VE];
  float m = -INFINITY, l = 0.f;
  if (n > 0) {
    if (lane < n) m = part[lane * kPart<D>], l = part[lane * kPart<D> + 1];
#pragma unroll
    for (int u = 0; u < 16; ++u)
#pragma unroll
      for (int c = 0; c < VE; ++c) x[u][c] = part[(u < n ? u : 0) * kPart<D> + 4 + lane * VE + c];
  }
  float top = over_wavefront(m, [](float p, float q) { return fmaxf(p, q); });
  const float f = l == 0.f ? 0.f : m == top ? 1.f : __builtin_amdgcn_exp2f(m - top);
  float sum = over_wavefront(f * l, [](float p, float q) { return p + q; });
  float y[VE] = {};
  if (n > 0) {
#pragma unroll
    for (int u = 0; u < 16; ++u) {
      const float w = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(f), u));  // (0 behind the last range)
#pragma unroll
      for (int c = 0; c < VE; ++c) y[c] = fmaf(w, x[u][c], y[c]);
    }
  }
  if constexpr (WIDE) {
#pragma unroll
    for (int c = 0; c < VE; ++c) y_s[wave][4 + lane * VE + c] = y[c];
    if (lane == 0) y_s[wave][0] = top, y_s[wave][1] = sum;
    __syncthreads();
    if (wave != 0) return;
    float mw[4], lw[4];
#pragma unroll
    for (int w = 0; w < 4; ++w) mw[w] = y_s[w][0], lw[w] = y_s[w][1];
    top = fmaxf(fmaxf(mw[0], mw[1]), fmaxf(mw[2], mw[3]));
    sum = 0.f;
#pragma unroll
    for (int c = 0; c < VE; ++c) y[c] = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float fw = lw[w] == 0.f ? 0.f : mw[w] == top ? 1.f : __builtin_amdgcn_exp2f(mw[w] - top);
      sum = fmaf(fw, lw[w], sum);
#pragma unroll
      for (int c = 0; c < VE; ++c) y[c] = fmaf(fw, y_s[w][4 + lane * VE + c], y[c]);
    }
  }
  store_row<VE, F32>(a.out, row, head, lane * VE, y, sum);
  if (a.lse != nullptr && lane == 0) a.lse[row * heads + head] = log_sum(top, sum);
}

template <int D, bool F32>
void launch_join(const PagesAttendArgs& a, hipStream_t s) {
  const int64_t items = (int64_t)a.b.n_seqs * a.b.max_new * a.c.heads * a.group;
  if (a.splits > 16) hipLaunchKernelGGL((pages_join_kernel<D, F32, true>), dim3((unsigned)items), dim3(256), 0, s, a);
  else hipLaunchKernelGGL((pages_join_kernel<D, F32, false>), dim3((unsigned)((items + 3) / 4)), dim3(256), 0, s, a);
}

template <int D, int CT>
hipError_t launch(bool f32, PagesAttendArgs a, hipStream_t s) {
  const int64_t rows = (a.chosen != nullptr ? 1 : (int64_t)a.b.max_new) * a.group, per = a.prompt ? pages_prompt_rows(D) : 16 * a.tiles;
  a.by_splits = Divide(a.splits), a.by_tiles = Divide((rows + per - 1) / per);
  a.by_heads = Divide(a.c.heads), a.by_new = Divide(a.b.max_new), a.by_group = Divide(a.group), a.by_queries = Divide(a.c.heads * a.group);
  hipError_t e;
  if (a.prompt) {
    e = launch_pages_attend_prompt(D, CT, a, s);
  } else {
    const int64_t blocks = pages_attend_units(pages_attend_sizes(a.b, a.c.heads, a.group, a.chosen != nullptr, a.n_chosen, a.c.log2_page, a.window), a.tiles) * a.splits;
    if (!grid_fits(blocks, 64 * WAVES)) return hipErrorInvalidConfiguration;
    const dim3 grid((unsigned)blocks);
    if (a.tiles == 2) {
      if constexpr (D == 128) hipLaunchKernelGGL((pages_attend_kernel<D, CT, false, 2>), grid, dim3(64 * WAVES), 0, s, a);
    } else {
      if (f32) hipLaunchKernelGGL((pages_attend_kernel<D, CT, true, 1>), grid, dim3(64 * WAVES), 0, s, a);
      else hipLaunchKernelGGL((pages_attend_kernel<D, CT, false, 1>), grid, dim3(64 * WAVES), 0, s, a);
    }
    e = hipGetLastError();
  }
  if (e != hipSuccess || a.splits == 1) return e;
  if (f32) launch_join<D, true>(a, s);
  else launch_join<D, false>(a, s);
  return hipGetLastError();
}

}  // namespace

size_t pages_attend_part_bytes(int d, const BatchView& b, int heads, int group, int splits) {
  return splits > 1 ? (size_t)b.n_rows * heads * group * splits * (4 + d) * sizeof(float) : 0;
}

hipError_t launch_pages_attend(int d, int type, bool f32, const PagesAttendArgs& a, hipStream_t s) {
  const bool i8 = type == kPageI8;
  if (d == 64) return i8 ? launch<64, kPageI8>(f32, a, s) : launch<64, kPageE4m3>(f32, a, s);
  if (d == 128) return i8 ? launch<128, kPageI8>(f32, a, s) : launch<128, kPageE4m3>(f32, a, s);
  return i8 ? launch<256, kPageI8>(f32, a, s) : launch<256, kPageE4m3>(f32, a, s);
}

}  // namespace tq
