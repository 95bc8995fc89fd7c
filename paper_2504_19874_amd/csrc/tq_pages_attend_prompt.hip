// Attention over pages for prompts: many rows of bf16 queries.
//
// The mathematics is that of tq_pages_attend.hip.  Here a workgroup has 256 rows (d = 256: 128) of a sequence and head, 32 to a wavefront, and all
// wavefronts share one tile of 64 keys in LDS, as 16-bit operands: turning codes into operands (and values by 4 x 4 bytes) is
// vector work that eight wavefronts would do eight times.  Products on v_mfma_f32_32x32x16, S^T = K Q^T and O^T += V^T P^T:
// lane (r = lane % 32, b = lane / 32) has row r and of 16 keys 4 b + 0..3 and 8 + 4 b + 0..3 in both, so weights stay in
// their lane.  LDS holds fragments in the order in which the lanes read them (16 bytes a lane, 1 KB a product):
//   keys    [32 keys][16 coordinates][lane]: lane (key, half of the coordinates), its place XOR the coordinates' number, so that eight
//           lanes that write one key's fragments meet eight groups of banks
//   values  [16 keys][d tile][lane]: d tile T has the coordinates (d / 32) i + T; a lane fetches d / 32 coordinates of eight keys and
//           writes a fragment to each d tile (d = 64: four coordinates, two to each)
// Wavefronts 0..3 take the values of one subtile of 16 keys each, 4..7 the keys.  The next tile is fetched while a tile is multiplied
// and written to the other half of LDS: one barrier a tile.
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

template <int D, int CT>
__global__ __launch_bounds__(64 * WAVES) void pages_attend_prompt_kernel(const PagesAttendArgs a) {
  constexpr int KS = D / 16;             // k steps of S
  constexpr int ROWS = kRows<D>;
  static_assert(ROWS == 32 * WAVES / kShare<D>, "32 rows to a wavefront, or to two");
  constexpr int DA = D / 32, DT = DA / kShare<D>;  // d tiles, and those of a wavefront
  constexpr int KC = D == 64 ? 4 : D == 128 ? 8 : 4;  // fragments of keys that a lane holds at a time (d = 256: 8 cost 8 % by spills)
  constexpr int VW = D == 256 ? 2 : 1;   // words of a key's values that a lane turns
  constexpr int KL = D / 64;             // 16-byte loads of a lane's keys
  constexpr int TILE = 64 * D * 2 / 16;  // fragments of a tile's keys, as many of its values
  extern __shared__ uint4_t lds[];       // [2][keys, values][TILE]
  __shared__ uint16_t poison_s[2][4];    // of a subtile's keys: those with a NaN among their values
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
  const int at0 = len - whole;

  const int rows_of = kShare<D> == 1 ? wave : wave & 3, dh = kShare<D> == 1 ? 0 : wave >> 2;  // which 32 rows, which part of the coordinates
  const int m = min(first + 32 * rows_of + r, rows - 1);
  const int64_t row = row0 + token_of(m);
  const int head = h * group + m - token_of(m) * group;
  const bool there = first + 32 * rows_of + r < rows && row >= 0 && row < a.b.n_rows;
  const int pos = at0 + token_of(m);
  const int pos_lo = at0 + token_of(first), pos_hi = at0 + token_of(min(first + ROWS - 1, rows - 1));  // of the workgroup
  const int mine_lo = at0 + token_of(min(first + 32 * rows_of, rows - 1)), mine_hi = at0 + token_of(min(first + 32 * rows_of + 31, rows - 1));

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

  const int64_t bound = (int64_t)a.b.width << a.c.log2_page;
  const int hi = (int)min((int64_t)pos_hi + 1, min(bound, (int64_t)INT_MAX - 128));
  const int lo = (int)max((int64_t)0, (int64_t)pos_lo - a.window + 1) & ~63;
  const int all_tiles = hi > lo ? (hi - lo + 63) >> 6 : 0, each = (all_tiles + a.splits - 1) / a.splits;
  const int begin = min(split * each, all_tiles), tiles = min(begin + each, all_tiles) - begin;  // this range's
  const int32_t* const table = a.b.table + (int64_t)s * a.b.table_stride;

  Subtile sub = no_subtile();  // a lane knows one subtile of the next 64
  const auto look_up = [&](int tile) {
    const int64_t at = (int64_t)lo + 16 * ((int64_t)4 * (begin + tile) + lane);
    sub = no_subtile();
    if (at < hi) sub = find_subtile(a.c, table, a.b.width, h, (int)(at >> a.c.log2_page), (int)at & ((1 << a.c.log2_page) - 1));
  };
  // a lane's part of the next tile: wavefronts 0..3 values, 4..7 keys, of subtile wave % 4
  uint32_t raw[8 * VW > 4 * KL ? 8 * VW : 4 * KL];
  const bool has_values = wave < 4;
  const int dq = D == 64 ? r & 15 : r;
  const auto fetch = [&](int tile) {
    const int at = __builtin_amdgcn_readlane(sub.at, ((tile & 15) << 2) + (wave & 3));
    const int64_t off = (int64_t)(at < 0 ? 0 : at) * (16 * D);
    if (has_values) {
      if (D != 64 || r < 16) {
        const uint8_t* const p = a.c.v + off + 4 * VW * dq;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const uint8_t* const from = p + (4 * b + (j & 3) + (j >> 2) * 8) * D;
          if constexpr (VW == 1) {
            raw[j] = *reinterpret_cast<const uint32_t*>(from);
          } else {
            const uint2_t two = *reinterpret_cast<const uint2_t*>(from);
            raw[j] = two[0], raw[8 + j] = two[1];
          }
        }
      }
    } else {
      const uint8_t* const p = a.c.k + off + 16 * lane;  // 16 keys of d bytes in one piece
#pragma unroll
      for (int j = 0; j < KL; ++j) *reinterpret_cast<uint4_t*>(&raw[4 * j]) = *reinterpret_cast<const uint4_t*>(p + 1024 * j);
    }
  };
  const auto put = [&](int half, bool masked) {
    const int sb = wave & 3;
    if (has_values) {
      if (CT == kPageE4m3 && masked) {
        uint32_t flags = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          uint32_t n = 0;
          if (D != 64 || r < 16)
#pragma unroll
            for (int v = 0; v < VW; ++v) {
              const uint32_t bytes = nan_bytes(raw[8 * v + j]);
              raw[8 * v + j] &= ~bytes;
              n |= bytes;
            }
          const uint64_t lanes = __builtin_amdgcn_ballot_w64(n != 0);
          const int key = (j & 3) + (j >> 2) * 8;
          flags |= ((uint32_t)lanes != 0 ? 1u << key : 0u) | ((uint32_t)(lanes >> 32) != 0 ? 16u << key : 0u);
        }
        if (lane == 0) poison_s[half][sb] = (uint16_t)flags;
      }
      if (D != 64 || r < 16) {
        uint4_t* const to = lds + (2 * half + 1) * TILE + sb * (DA * 64) + 32 * b;
#pragma unroll
        for (int v = 0; v < VW; ++v) {
          uint32_t turned[2][4];
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const uint32_t *const w = raw + 8 * v + 4 * u;
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
            // coordinate 4 VW dq + 4 v + e = (d / 32) i + T
            if constexpr (D == 64) to[(e & 1) * 64 + 2 * dq + (e >> 1)] = f;
            else to[(4 * v + e) * 64 + dq] = f;
          }
        }
      }
    } else {
      uint4_t* const to = lds + 2 * half * TILE;
#pragma unroll
      for (int j = 0; j < KL; ++j) {
        // bytes [16 lane + 1024 j, + 16) of the subtile: key, and 16 of its coordinates
        const int byte = 16 * lane + 1024 * j, key = 16 * sb + byte / D, step = byte % D / 16;
        union {
          bf16x8_t v;
          uint4_t w;
        } f0, f1;
        f0.v = codes_bf16<CT>(raw[4 * j], raw[4 * j + 1]);
        f1.v = codes_bf16<CT>(raw[4 * j + 2], raw[4 * j + 3]);
        uint4_t* const at = to + ((key >> 5) * KS + step) * 64;
        at[(key & 31) ^ (step & 7)] = f0.w;
        at[(32 + (key & 31)) ^ (step & 7)] = f1.w;
      }
    }
  };

  float16_t o[DT];
#pragma unroll
  for (int t = 0; t < DT; ++t)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[t][i] = 0.f;
  float l = 0.f, M = -INFINITY, shift = 0.f, limit = -3e38f;

  // where not all of the workgroup's rows see all of a tile: its subtiles' positions from the lanes that know them
  const auto tile_pos = [&](int tile, int u) { return __builtin_amdgcn_readlane(sub.pos, ((tile & 15) << 2) + u); };
  const auto is_masked = [&](int tile) {
    const int p0 = tile_pos(tile, 0), p1 = tile_pos(tile, 1), p2 = tile_pos(tile, 2), p3 = tile_pos(tile, 3);
    return max(max(p0, p1), max(p2, p3)) + 15 > pos_lo || (int64_t)min(min(p0, p1), min(p2, p3)) <= (int64_t)pos_hi - a.window;
  };

  const auto step = [&](int half, const int (&sp)[4], const float (&ks)[4], const float (&lv)[4], const float (&iv)[4], bool masked) {
    const uint4_t* const keys = lds + 2 * half * TILE;
    const uint4_t* const values = keys + TILE;
    // Fragments are fetched a phase ahead of their products (a product takes 32 cycles, a fetch over 100), and the barriers keep them there
    uint4_t kf[KC], vf[2 * DT];
    const auto fetch_keys = [&](int kt, int k0) {
#pragma unroll
      for (int k = 0; k < KC; ++k) kf[k] = keys[(kt * KS + k0 + k) * 64 + (lane ^ ((k0 + k) & 7))];
    };
    fetch_keys(0, 0);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
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
      for (int i = 0; i < 2 * DT; ++i) vf[i] = values[((2 * kt + i / DT) * DA + dh * DT + i % DT) * 64 + lane];
      __builtin_amdgcn_sched_barrier(0);
      uint32_t hidden = 0;  // bit i: key 8 (i / 4) + 4 b + i % 4 is not seen
      if (masked) {
        const bool inner = max(sp[2 * kt], sp[2 * kt + 1]) + 15 <= mine_lo && (int64_t)min(sp[2 * kt], sp[2 * kt + 1]) > (int64_t)mine_hi - a.window;
        uint32_t poison = 0;
        if (CT == kPageE4m3) poison = (uint32_t)poison_s[half][2 * kt] | (uint32_t)poison_s[half][2 * kt + 1] << 16;
        if (!inner || poison != 0) {
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int in = 8 * (i >> 2) + 4 * b + (i & 3), key = sp[2 * kt + (i >> 3)] + (in & 15);
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
          const float ch = ks[2 * kt + u] * a.scale2, add = lv[2 * kt + u] + shift;
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
          shift = BASE - next;
          limit = BASE + HEAD;
        }
        l *= down;
#pragma unroll
        for (int t = 0; t < DT; ++t) o[t] *= down;
        exponents();
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
      for (int t = 0; t < DT; ++t) o[t] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8_t, vf[t]), p[0], o[t], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
      if (kt == 0) fetch_keys(1, 0);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int t = 0; t < DT; ++t) o[t] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8_t, vf[DT + t]), p[1], o[t], 0, 0, 0);
    }
  };

  if (tiles > 0) {
    look_up(0);
    fetch(0);
    bool masked = is_masked(0);
    put(0, masked);
    __syncthreads();
    for (int n = 0; n < tiles; ++n) {
      int sp[4];
      float ks[4], lv[4], iv[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int from = ((n & 15) << 2) + u;
        sp[u] = __builtin_amdgcn_readlane(sub.pos, from);
        ks[u] = lane_value(sub.ks, from), lv[u] = lane_value(sub.lv, from), iv[u] = lane_value(sub.iv, from);
      }
      bool next_masked = false;
      if (n + 1 < tiles) {
        if (((n + 1) & 15) == 0) look_up(n + 1);
        next_masked = is_masked(n + 1);
        fetch(n + 1);
      }
      step(n & 1, sp, ks, lv, iv, masked);
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
  constexpr int bytes = 2 * 2 * 64 * D * 2;
  static LdsLimit limit;
  const void* const kernel = reinterpret_cast<const void*>(&pages_attend_prompt_kernel<D, CT>);
  const hipError_t e = raise_lds_limit(limit, kernel, bytes);
  if (e != hipSuccess) return e;
  const int64_t row_tiles = ((int64_t)a.b.max_new * a.group + kRows<D> - 1) / kRows<D>;
  hipLaunchKernelGGL((pages_attend_prompt_kernel<D, CT>), dim3((unsigned)((int64_t)a.b.n_seqs * a.c.heads * row_tiles * a.splits)), dim3(64 * WAVES), bytes, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_pages_attend_prompt(int d, int type, const PagesAttendArgs& a, hipStream_t s) {
  if (type == kPageI8) return d == 64 ? launch<64, kPageI8>(a, s) : d == 128 ? launch<128, kPageI8>(a, s) : launch<256, kPageI8>(a, s);
  return d == 64 ? launch<64, kPageE4m3>(a, s) : d == 128 ? launch<128, kPageE4m3>(a, s) : launch<256, kPageE4m3>(a, s);
}

}  // namespace tq
