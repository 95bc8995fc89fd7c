// Attention over pages for prompts: many rows of bf16 queries.
//
// The mathematics is that of tq_pages_attend.hip.  Here a workgroup has 256 rows (d = 256: 128) of a sequence and head, 32 to a wavefront, and all
// wavefronts share one tile of 128 keys (d = 256: 64) in LDS, as 16-bit operands: turning codes into operands (and values by 4 x 4 bytes) is
// vector work that eight wavefronts would do eight times.  Products on v_mfma_f32_32x32x16, S^T = K Q^T and O^T += V^T P^T:
// lane (r = lane % 32, b = lane / 32) has row r and of 16 keys 4 b + 0..3 and 8 + 4 b + 0..3 in both, so weights stay in
// their lane.  LDS holds fragments in the order in which the lanes read them (16 bytes a lane, 1 KB a product):
//   keys    [32 keys][16 coordinates][lane]: lane (key, half of the coordinates), its place XOR the coordinates' number, so that eight
//           lanes that write one key's fragments meet eight groups of banks
//   values  [16 keys][d tile][lane]: d tile t has the coordinates (d / 32) i + t; a lane fetches d / 32 coordinates of eight keys and
//           writes a fragment to each d tile (d = 64: four coordinates, two to each, and half a wavefront has a subtile of 16 keys)
// Wavefronts 0..3 take the values of two subtiles of 16 keys each (d = 256: one), 4..7 the keys.  The next tile is fetched while a tile is multiplied
// and written to the other half of LDS: one barrier a tile.
//
// What bounds it: matrix and vector instructions.  With two wavefronts to a SIMD four fused multiply-adds behind a product hide (14.2 ns, the
// product alone 13.7), more of them hide in part (8: 19.9, apart 22.7) and then hardly at all (16: 29.7, apart 30.8); this kernel has
// 6.5 vector instructions to a product, so that what counts is their number.  Of the SIMDs' cycles the matrix cores are busy in 46 %
// (SQ_VALU_MFMA_BUSY_CYCLES), vector and matrix instructions issue in 51 % (SQ_ACTIVE_INST_VALU).  Tiles of 128 keys have half the barriers, addresses and masks of tiles of 64: 8192 tokens of which 2048 are new, 4
// sequences of 8 x 4 heads, d = 64 784 -> 620 us, d = 128 1012 -> 970 (on one card); d = 256 1614 -> 1390 (two sequences) by what
// is no longer carried through the loop in registers.  Logits of the next 32 keys multiplied between the exponentials: 7-15 % slower.
#include "tq_pages_attend.h"

namespace tq {

namespace {

typedef float float16_t __attribute__((ext_vector_type(16)));

constexpr int WAVES = 8;
// d = 256: two wavefronts share 32 rows, each with half of the output's coordinates (and all of S, which is cheaper than its exchange)
template <int D>
constexpr int kShare = D == 256 ? 2 : 1;
template <int D>
constexpr int kRows = pages_prompt_rows(D);

// subtiles of 16 keys of a tile: LDS holds two tiles (d = 64: 16 are not faster)
template <int D>
constexpr int kSubtiles = D == 256 ? 4 : 8;

template <int D, int CT>
__global__ __launch_bounds__(64 * WAVES) void pages_attend_prompt_kernel(const PagesAttendArgs a) {
  constexpr int KS = D / 16;             // k steps of S
  constexpr int ROWS = kRows<D>;
  static_assert(ROWS == 32 * WAVES / kShare<D>, "32 rows to a wavefront, or to two");
  constexpr int DA = D / 32, DT = DA / kShare<D>;  // d tiles, and those of a wavefront
  constexpr int KC = D == 64 ? 4 : D == 128 ? 8 : 4;  // fragments of keys that a lane holds at a time (d = 256: 8 cost 8 % by spills)
  constexpr int VW = D == 256 ? 2 : 1;   // words of a key's values that a lane turns
  constexpr int T = kSubtiles<D>, SW = T / 4;  // subtiles of 16 keys of a tile, and those of a wavefront that turns codes
  constexpr int VQ = D == 64 ? 1 : SW;   // ... one after the other (d = 64: half a wavefront has one)
  constexpr int KL = D / 64;             // 16-byte loads of a lane's keys of a subtile
  constexpr int TILE = 16 * T * D * 2 / 16;  // fragments of a tile's keys, as many of its values
  extern __shared__ uint4_t lds[];       // [2][keys, values][TILE]
  __shared__ uint16_t poison_s[2][T];    // of a subtile's keys: those with a NaN among their values
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 31, b = lane >> 5;
  const int heads = a.c.heads, group = a.group;
  const int row_tiles = (int)a.by_tiles.by;
  // the row tiles of a unit read the same keys: on one XCD (workgroups go to the eight of them in turn), the longest first
  const unsigned units = (unsigned)a.b.n_seqs * (unsigned)heads, each_unit = (unsigned)(row_tiles * a.splits);
  unsigned unit, part_of;
  if (units % 8 == 0) unit = (blockIdx.x >> 3) / each_unit * 8 + (blockIdx.x & 7), part_of = (blockIdx.x >> 3) % each_unit;
  else unit = blockIdx.x / each_unit, part_of = blockIdx.x % each_unit;
  const int split = (int)(part_of % (unsigned)a.splits), first = (row_tiles - 1 - (int)(part_of / (unsigned)a.splits)) * ROWS;
  const int h = (int)(unit % (unsigned)heads), s = (int)(unit / (unsigned)heads);
  const int whole = a.b.count(s), rows = min(whole, a.b.max_new) * group;
  if (first >= rows) return;
  const int len = a.b.lens[s];
  const int64_t row0 = a.b.first_row(s);
  const auto token_of = [&](int m) { return (int)a.by_group.of((uint32_t)m); };
  const int64_t at0 = (int64_t)len - whole;

  const int rows_of = kShare<D> == 1 ? wave : wave & 3, dh = kShare<D> == 1 ? 0 : wave >> 2;  // which 32 rows, which part of the coordinates
  const int m = min(first + 32 * rows_of + r, rows - 1);
  const int64_t row = row0 + token_of(m);
  const int head = h * group + m - token_of(m) * group;
  const bool there = first + 32 * rows_of + r < rows && row >= 0 && row < a.b.n_rows;
  const auto position_of = [&](int m) { return row_position(at0 + token_of(m)); };
  const int pos = position_of(m);
  const int pos_lo = position_of(first), pos_hi = position_of(min(first + ROWS - 1, rows - 1));  // of the workgroup
  const int mine_lo = position_of(min(first + 32 * rows_of, rows - 1)), mine_hi = position_of(min(first + 32 * rows_of + 31, rows - 1));

  bf16x8_t q[KS];
#pragma unroll
  for (int k = 0; k < KS; ++k) {
    union {
      uint4_t w;
      bf16x8_t v;
    } u;
    u.w = uint4_t{0, 0, 0, 0};
    if (there) u.w = *reinterpret_cast<const uint4_t*>(static_cast<const uint16_t*>(a.q.p) + row * a.q.ld_row + head * a.q.ld_head + 16 * k + 8 * b);
    q[k] = u.v;
  }

  const bool busy = first + 32 * rows_of < rows;  // (without rows a wavefront only turns codes: 66 rows, 16 sequences of 2000, 44.8 -> 40.2 us)
  const int64_t bound = (int64_t)a.b.width << a.c.log2_page;
  const int hi = (int)min((int64_t)pos_hi + 1, bound);
  const int lo = (int)max((int64_t)0, (int64_t)pos_lo - a.window + 1) & ~63;
  const int all_tiles = hi > lo ? (int)(((int64_t)hi - lo + 16 * T - 1) / (16 * T)) : 0, each = (all_tiles + a.splits - 1) / a.splits;
  const int begin = min(split * each, all_tiles), tiles = min(begin + each, all_tiles) - begin;  // this range's
  const int32_t* const table = a.b.table + (int64_t)s * a.b.table_stride;

  Subtile sub = no_subtile();  // a lane knows one subtile of the next 64
  uint64_t partly = 0;         // those that not all of the workgroup's rows see whole
  const auto look_up = [&](int tile) {
    const int64_t at = (int64_t)lo + 16 * ((int64_t)T * (begin + tile) + lane);
    sub = no_subtile();
    if (at < hi) sub = find_subtile(a.c, table, a.b.width, h, (int)(at >> a.c.log2_page), (int)at & ((1 << a.c.log2_page) - 1));
    partly = __builtin_amdgcn_ballot_w64(sub.pos + 15 > pos_lo || (int64_t)sub.pos <= (int64_t)pos_hi - a.window);
    sub.ks *= a.scale2;
  };
  const auto place = [&](int tile, int u) { return (tile & (64 / T - 1)) * T + u; };  // the lane that knows subtile u
  // a lane's part of the next tile: wavefronts 0..3 values, 4..7 keys, of SW subtiles
  uint32_t raw[(8 * VW * VQ > 4 * KL * SW ? 8 * VW * VQ : 4 * KL * SW)];
  const bool has_values = wave < 4;
  const int dq = D == 64 ? r & 15 : r;
  const auto fetch = [&](int tile) {
    int64_t off[SW];
#pragma unroll
    for (int q = 0; q < SW; ++q) off[q] = (int64_t)max(__builtin_amdgcn_readlane(sub.at, place(tile, SW * (wave & 3) + q)), 0) * (16 * D);
    if (has_values) {
#pragma unroll
      for (int q = 0; q < VQ; ++q) {
        const uint8_t* const p = a.c.v + (D != 64 || r < 16 ? off[q] : off[SW - 1]) + 4 * VW * dq;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const uint8_t* const from = p + (4 * b + (j & 3) + (j >> 2) * 8) * D;
          if constexpr (VW == 1) {
            raw[8 * q + j] = *reinterpret_cast<const uint32_t*>(from);
          } else {
            const uint2_t two = *reinterpret_cast<const uint2_t*>(from);
            raw[j] = two[0], raw[8 + j] = two[1];
          }
        }
      }
    } else {
#pragma unroll
      for (int q = 0; q < SW; ++q) {
        const uint8_t* const p = a.c.k + off[q] + 16 * lane;  // 16 keys of d bytes in one piece
#pragma unroll
        for (int j = 0; j < KL; ++j) *reinterpret_cast<uint4_t*>(&raw[4 * (KL * q + j)]) = *reinterpret_cast<const uint4_t*>(p + 1024 * j);
      }
    }
  };
  const auto put = [&](int half, bool masked) {
    if (has_values) {
#pragma unroll
      for (int q = 0; q < VQ; ++q) {
        const int sb = SW * (wave & 3) + (D == 64 ? r >> 4 : q);
        if (CT == kPageE4m3 && masked) {
          uint32_t flags[SW] = {};
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            uint32_t n = 0;
#pragma unroll
            for (int v = 0; v < VW; ++v) {
              const uint32_t bytes = nan_bytes(raw[8 * (VW * q + v) + j]);
              raw[8 * (VW * q + v) + j] &= ~bytes;
              n |= bytes;
            }
            const uint64_t lanes = __builtin_amdgcn_ballot_w64(n != 0);
            const int key = (j & 3) + (j >> 2) * 8;
#pragma unroll
            for (int u = 0; u < (D == 64 ? SW : 1); ++u) {
              const uint32_t half_of = D == 64 ? 0xffffu << 16 * u : 0xffffffffu;
              flags[u] |= ((uint32_t)lanes & half_of) != 0 ? 1u << key : 0u;
              flags[u] |= ((uint32_t)(lanes >> 32) & half_of) != 0 ? 16u << key : 0u;
            }
          }
          if (lane == 0)
#pragma unroll
            for (int u = 0; u < (D == 64 ? SW : 1); ++u) poison_s[half][SW * (wave & 3) + q + u] = (uint16_t)flags[u];
        }
        uint4_t* const to = lds + (2 * half + 1) * TILE + sb * (DA * 64) + 32 * b;
#pragma unroll
        for (int v = 0; v < VW; ++v) {
          uint32_t turned[2][4];
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const uint32_t *const w = raw + 8 * (VW * q + v) + 4 * u;
            const uint32_t a0 = __builtin_amdgcn_perm(w[1], w[0], 0x05010400u), a1 = __builtin_amdgcn_perm(w[1], w[0], 0x07030602u);
            const uint32_t b0 = __builtin_amdgcn_perm(w[3], w[2], 0x05010400u), b1 = __builtin_amdgcn_perm(w[3], w[2], 0x07030602u);
            turned[u][0] = __builtin_amdgcn_perm(b0, a0, 0x05040100u);
            turned[u][1] = __builtin_amdgcn_perm(b0, a0, 0x07060302u);
            turned[u][2] = __builtin_amdgcn_perm(b1, a1, 0x05040100u);
            turned[u][3] = __builtin_amdgcn_perm(b1, a1, 0x07060302u);
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint4_t f = __builtin_bit_cast(uint4_t, codes_fp16<CT>(turned[0][e], turned[1][e]));
            // coordinate 4 VW dq + 4 v + e = (d / 32) i + t
            if constexpr (D == 64) to[(e & 1) * 64 + 2 * dq + (e >> 1)] = f;
            else to[(4 * v + e) * 64 + dq] = f;
          }
        }
      }
    } else {
      uint4_t* const to = lds + 2 * half * TILE;
#pragma unroll
      for (int q = 0; q < SW; ++q)
#pragma unroll
        for (int j = 0; j < KL; ++j) {
          // bytes [16 lane + 1024 j, + 16) of the subtile: key, and 16 of its coordinates
          const int byte = 16 * lane + 1024 * j, key = 16 * (SW * (wave & 3) + q) + byte / D, step = byte % D / 16;
          const uint32_t* const w = raw + 4 * (KL * q + j);
          uint4_t* const at = to + ((key >> 5) * KS + step) * 64;
          at[(key & 31) ^ (step & 7)] = __builtin_bit_cast(uint4_t, codes_bf16<CT>(w[0], w[1]));
          at[(32 + (key & 31)) ^ (step & 7)] = __builtin_bit_cast(uint4_t, codes_bf16<CT>(w[2], w[3]));
        }
    }
  };

  float16_t o[DT];
#pragma unroll
  for (int t = 0; t < DT; ++t)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[t][i] = 0.f;
  float l = 0.f, M = -INFINITY, shift = 0.f, limit = -3e38f;

  const auto is_masked = [&](int tile) { return ((partly >> place(tile, 0)) & ((1u << T) - 1)) != 0; };

  const auto step = [&](int half, int tile, int tile_pos, const float (&ks)[T], const float (&lv)[T], const float (&iv)[T], bool masked) {
    const uint4_t* const keys = lds + 2 * half * TILE;
    const uint4_t* const values = keys + TILE;
    // Fragments are fetched a phase ahead of their products (a product takes 32 cycles, a fetch over 100), and the barriers keep them there
    uint4_t kf[KC], vf[DT];
    const auto fetch_keys = [&](int kt, int k0) {
#pragma unroll
      for (int k = 0; k < KC; ++k) kf[k] = keys[(kt * KS + k0 + k) * 64 + (lane ^ ((k0 + k) & 7))];
    };
    fetch_keys(0, 0);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int kt = 0; kt < T / 2; ++kt) {
      float16_t acc;
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[i] = 0.f;
#pragma unroll
      for (int k0 = 0; k0 < KS; k0 += KC) {
        if (k0 > 0) fetch_keys(kt, k0);
#pragma unroll
        for (int k = 0; k < KC; ++k) acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, kf[k]), q[k0 + k], acc, 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int i = 0; i < DT; ++i) vf[i] = values[((2 * kt + i / DT) * DA + dh * DT + i % DT) * 64 + lane];
      __builtin_amdgcn_sched_barrier(0);
      uint32_t hidden = 0;  // bit i: key 8 (i / 4) + 4 b + i % 4 is not seen
      if (masked) {
        const int sp[2] = {__builtin_amdgcn_readlane(tile_pos, place(tile, 2 * kt)), __builtin_amdgcn_readlane(tile_pos, place(tile, 2 * kt + 1))};
        const bool inner = max(sp[0], sp[1]) + 15 <= mine_lo && (int64_t)min(sp[0], sp[1]) > (int64_t)mine_hi - a.window;
        uint32_t poison = 0;
        if (CT == kPageE4m3) poison = (uint32_t)poison_s[half][2 * kt] | (uint32_t)poison_s[half][2 * kt + 1] << 16;
        if (!inner || poison != 0) {
          int b4 = 4 * b;
          asm volatile("" : "+v"(b4));  // (else sixteen positions are carried through the loop)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int in = 8 * (i >> 2) + b4 + (i & 3), key = sp[i >> 3] + (in & 15);
            const bool seen = key <= pos && (int64_t)key > (int64_t)pos - a.window;
            hidden |= seen ? 0u : 1u << i;
            if (seen && ((poison >> in) & 1)) acc[i] = __builtin_nanf("");
          }
        }
      }
      float x[16];
      const auto exponents = [&] {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const float ch = ks[2 * kt + u], add = lv[2 * kt + u] + shift;
#pragma unroll
          for (int i = 0; i < 8; ++i) x[8 * u + i] = fmaf(acc[8 * u + i], ch, add);
        }
        if (hidden != 0) {
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if ((hidden >> i) & 1) x[i] = -INFINITY;
        }
      };
      exponents();
      float top = x[0];
#pragma unroll
      for (int i = 1; i < 16; ++i) top = fmaxf(top, x[i]);
      if (__builtin_amdgcn_ballot_w64(top > limit) != 0) {
        const auto two = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
        const float next = fmaxf(M, fmaxf(__uint_as_float(two[0]), __uint_as_float(two[1])) - shift);
        const float down = M == next || M == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(M - next);
        if (next != -INFINITY) {
          M = next;
#pragma unroll
          for (int i = 0; i < 16; ++i) x[i] += BASE - next - shift;
          shift = BASE - next;
          limit = BASE + HEAD;
        }
        l *= down;
#pragma unroll
        for (int t = 0; t < DT; ++t) o[t] *= down;
      }
      half8_t p[2];
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float w = __builtin_amdgcn_exp2f(x[i]);
        l = fmaf(w, iv[2 * kt + (i >> 3)], l);
        p[i >> 3][i & 7] = (_Float16)w;
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int t = 0; t < DT; ++t) o[t] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8_t, vf[t]), p[0], o[t], 0, 0, 0), vf[t] = values[((2 * kt + 1) * DA + dh * DT + t) * 64 + lane];
      __builtin_amdgcn_sched_barrier(0);
      if (kt + 1 < T / 2) fetch_keys(kt + 1, 0);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int t = 0; t < DT; ++t) o[t] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8_t, vf[t]), p[1], o[t], 0, 0, 0);
    }
  };

  if (tiles > 0) {
    look_up(0);
    fetch(0);
    bool masked = is_masked(0);
    put(0, masked);
    __syncthreads();
    for (int n = 0; n < tiles; ++n) {
      const int tile_pos = sub.pos;
      float ks[T], lv[T], iv[T];
#pragma unroll
      for (int u = 0; u < T; ++u) {
        const int from = place(n, u);
        ks[u] = lane_value(sub.ks, from), lv[u] = lane_value(sub.lv, from), iv[u] = lane_value(sub.iv, from);
      }
      bool next_masked = false;
      if (n + 1 < tiles) {
        if (place(n + 1, 0) == 0) look_up(n + 1);
        next_masked = is_masked(n + 1);
        fetch(n + 1);
      }
      if (busy) step(n & 1, n, tile_pos, ks, lv, iv, masked);
      if (n + 1 < tiles) put((n + 1) & 1, next_masked);
      masked = next_masked;
      __syncthreads();
    }
  }

  const auto two = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
  const float sum = __uint_as_float(two[0]) + __uint_as_float(two[1]);
  if (!there) return;
  // o[t][i] is coordinate (d / 32) (8 (i / 4) + 4 b + i % 4) + t, of the second part 4 more: in one piece for four i, or for one where
  // wavefronts share the coordinates
  constexpr int N = kShare<D> == 1 ? 4 * DT : DT;
#pragma unroll
  for (int c = 0; c < 16 * DT / N; ++c) {
    float y[N];
#pragma unroll
    for (int i = 0; i < N / DT; ++i)
#pragma unroll
      for (int t = 0; t < DT; ++t) y[i * DT + t] = o[t][c * (N / DT) + i];
    const int i0 = c * (N / DT), at = DA * (8 * (i0 >> 2) + 4 * b + (i0 & 3)) + dh * DT;
    if (a.splits == 1) {
      store_row<N, false>(a.out, row, head, at, y, sum);
    } else {
      float* const part = a.part + ((row * heads * group + head) * a.splits + split) * (4 + D);
#pragma unroll
      for (int i = 0; i < N; i += 4) *reinterpret_cast<float4_t*>(part + 4 + at + i) = float4_t{y[i], y[i + 1], y[i + 2], y[i + 3]};
      if (c == 0 && b == 0 && dh == 0) part[0] = M, part[1] = sum;
    }
  }
  if (a.splits > 1) return;
  if (a.lse != nullptr && b == 0 && dh == 0) a.lse[row * heads * group + head] = log_sum(M, sum);
}

template <int D, int CT>
hipError_t launch(const PagesAttendArgs& a, hipStream_t s) {
  const int64_t row_tiles = ((int64_t)a.b.max_new * a.group + kRows<D> - 1) / kRows<D>, blocks = (int64_t)a.b.n_seqs * a.c.heads * row_tiles * a.splits;
  if (!grid_fits(blocks, 64 * WAVES)) return hipErrorInvalidConfiguration;
  constexpr int bytes = 2 * 2 * 16 * kSubtiles<D> * D * 2;
  static LdsLimit limit;
  const void* const kernel = reinterpret_cast<const void*>(&pages_attend_prompt_kernel<D, CT>);
  const hipError_t e = raise_lds_limit(limit, kernel, bytes);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((pages_attend_prompt_kernel<D, CT>), dim3((unsigned)blocks), dim3(64 * WAVES), bytes, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_pages_attend_prompt(int d, int type, const PagesAttendArgs& a, hipStream_t s) {
  if (type == kPageI8) return d == 64 ? launch<64, kPageI8>(a, s) : d == 128 ? launch<128, kPageI8>(a, s) : launch<256, kPageI8>(a, s);
  return d == 64 ? launch<64, kPageE4m3>(a, s) : d == 128 ? launch<128, kPageE4m3>(a, s) : launch<256, kPageE4m3>(a, s);
}

}  // namespace tq
