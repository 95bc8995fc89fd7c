// The page pool: giving out pages, forking and ending sequences, making the pool dense.
//
// One workgroup reads tables, lengths and reference counts in order and hands out ranks by prefix sums, so that which page goes where does
// not depend on the order of execution.  It looks at 1024 counts at a time, from page 0 until it has enough: 64 rows that want a page
// of a pool that is full to nine tenths take 2.5 us where it has 4096 pages, 39 where 65536, 660 where 2^20 (rows that want none 3.4
// us in any); making the pool dense reads all counts twice, 7.8, 55 and 840 us.  Pages are then moved by as many
// workgroups as there are pieces of PIECE bytes: bound by memory, 2 bytes moved for a byte.
#include "tq_pages.h"

namespace tq {

namespace {

constexpr int THREADS = 1024, WAVES = THREADS / 64;
constexpr int PIECE = 16384;  // bytes of keys or values that a workgroup moves

// exclusive count of `flag` over the workgroup's threads in order, on top of `base`, which moves on by the total
__device__ __forceinline__ int rank_of(bool flag, int& base, int* wave_s) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint64_t set = __builtin_amdgcn_ballot_w64(flag);
  __syncthreads();  // wave_s may still be read
  if (lane == 0) wave_s[wave] = __popcll(set);
  __syncthreads();
  int mine = base + __popcll(set & ((1ull << lane) - 1));
  for (int v = 0; v < WAVES; ++v) {
    if (v < wave) mine += wave_s[v];
    base += wave_s[v];
  }
  return mine;
}

// the lowest free pages, up to `want` of them, into `list`; returns how many there are
__device__ __forceinline__ int free_pages(const PagesView& c, int want, int32_t* list, int* wave_s) {
  int found = 0;
  for (int p0 = 0; p0 < c.n_pages && found < want; p0 += THREADS) {
    const int p = p0 + threadIdx.x;
    const bool is = p < c.n_pages && c.refs[p] <= 0;
    const int rank = rank_of(is, found, wave_s);
    if (is && rank < want) list[rank] = p;
  }
  __syncthreads();  // the list is read by other threads
  return min(found, want);
}

__device__ __forceinline__ bool is_page(const PagesView& c, int p) { return p >= 0 && p < c.n_pages; }

__global__ __launch_bounds__(THREADS) void pages_reserve_kernel(const PagesView c, const BatchView b, const Divide each, int32_t* list,
                                                               int32_t* missing) {
  __shared__ int wave_s[WAVES];
  __shared__ int lost_s;  // entries that hold tokens before the new ones, which had no page to go to: a free one has somebody else's
  const uint32_t items = (uint32_t)b.n_seqs * each.by;
  const auto entry = [&](uint32_t item, bool count) -> int32_t* {
    if (item >= items) return nullptr;
    const uint32_t s = each.of(item);
    const int64_t len = b.lens[s], most = max(min(b.count((int)s), b.max_new), 0), from = len > most ? len - most : 0;
    const int64_t i = (from >> c.log2_page) + each.rest(item, s);
    if (most == 0 || (i << c.log2_page) >= len || i >= b.width) return nullptr;
    int32_t* const e = b.table + (int64_t)s * b.table_stride + i;
    if (is_page(c, *e)) return nullptr;
    if ((i << c.log2_page) >= from) return e;
    if (count) atomicAdd(&lost_s, 1);
    return nullptr;
  };
  if (threadIdx.x == 0) lost_s = 0;
  __syncthreads();
  int want = 0;
  for (uint32_t i = 0; i < items; i += THREADS) rank_of(entry(i + threadIdx.x, true) != nullptr, want, wave_s);
  const int got = free_pages(c, want, list, wave_s);
  int at = 0;
  for (uint32_t i = 0; i < items; i += THREADS) {
    int32_t* const e = entry(i + threadIdx.x, false);
    const int rank = rank_of(e != nullptr, at, wave_s);
    if (e != nullptr) {
      const int p = rank < got ? list[rank] : -1;
      *e = p;
      if (p >= 0) c.refs[p] = 1;
    }
  }
  if (threadIdx.x == 0 && missing != nullptr) *missing = want - got + lost_s;
}

// What fork i does, written by the first kernel for the second: the tokens of its parent (-1: it is skipped) and the free page that the
// last of them are copied into (-1: none).
struct Fork {
  int32_t len, fresh;
};

__global__ __launch_bounds__(THREADS) void pages_fork_kernel(const PagesView c, const BatchView b, const int32_t* parents, const int32_t* children,
                                                            const int n, int32_t* list, Fork* forks, int32_t* missing) {
  __shared__ int wave_s[WAVES];
  const auto is_row = [&](int s) { return s >= 0 && s < b.n_seqs; };
  // Of the entries with one child the first counts: i - n, below every length, in the child's place.  A child that holds tokens is left alone.
  for (int i = threadIdx.x; i < n; i += THREADS) {
    const int p = parents[i], s = children[i];
    forks[i] = Fork{-1, -1};
    if (is_row(p) && is_row(s) && p != s && b.lens[s] <= 0) {
      forks[i].len = max(b.lens[p], 0);
      if (b.lens[s] != 0) b.lens[s] = 0;  // (a length below zero is none; it must not stand before an entry's number)
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += THREADS)
    if (forks[i].len >= 0) atomicMin(&b.lens[children[i]], i - n);
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += THREADS)
    if (forks[i].len >= 0 && b.lens[children[i]] != i - n) forks[i].len = -1;
  __syncthreads();
  // the page of a parent's last tokens, if that is not full
  const auto wants = [&](int i) {
    if (i >= n || forks[i].len < 0) return false;
    const int full = forks[i].len >> c.log2_page;
    return (forks[i].len & ((1 << c.log2_page) - 1)) != 0 && full < b.width && is_page(c, b.table[(int64_t)parents[i] * b.table_stride + full]);
  };
  int want = 0;
  for (int i = 0; i < n; i += THREADS) rank_of(wants(i + (int)threadIdx.x), want, wave_s);
  const int got = free_pages(c, want, list, wave_s);
  int at = 0;
  for (int i0 = 0; i0 < n; i0 += THREADS) {
    const int i = i0 + (int)threadIdx.x;
    const bool is = wants(i);
    const int rank = rank_of(is, at, wave_s);
    if (is && rank < got) {
      forks[i].fresh = list[rank];
      c.refs[list[rank]] = 1;
    }
  }
  if (threadIdx.x == 0 && missing != nullptr) *missing = want - got;
}

// pieces of a page: of its keys, as many of its values, one with scales and bounds
__host__ __device__ inline int pieces_of(const PagesView& c, int d) { return 2 * (((c.heads << c.log2_page) * d + PIECE - 1) / PIECE) + 1; }

__device__ __forceinline__ void copy_piece(const PagesView& c, int d, int from, int to, int piece) {
  const int64_t bytes = (int64_t)(c.heads << c.log2_page) * d;
  const int half = (pieces_of(c, d) - 1) / 2;
  if (piece < 2 * half) {
    uint8_t* const x = piece < half ? c.k : c.v;
    const int64_t first = (int64_t)(piece < half ? piece : piece - half) * PIECE, last = first + PIECE < bytes ? first + PIECE : bytes;
    const uint4_t* const src = reinterpret_cast<const uint4_t*>(x + from * bytes);
    uint4_t* const dst = reinterpret_cast<uint4_t*>(x + to * bytes);
    for (int64_t i = first / 16 + threadIdx.x; i < last / 16; i += blockDim.x) dst[i] = src[i];
    return;
  }
  for (int i = threadIdx.x; i < c.heads; i += blockDim.x) {
    c.k_scale[(int64_t)to * c.heads + i] = c.k_scale[(int64_t)from * c.heads + i];
    c.v_scale[(int64_t)to * c.heads + i] = c.v_scale[(int64_t)from * c.heads + i];
  }
  if (c.bounds != nullptr) {
    const int64_t n = (int64_t)c.heads * 2 * d;  // bf16 values
    const uint4_t* const src = reinterpret_cast<const uint4_t*>(c.bounds + from * n);
    uint4_t* const dst = reinterpret_cast<uint4_t*>(c.bounds + to * n);
    for (int64_t i = threadIdx.x; i < n / 8; i += blockDim.x) dst[i] = src[i];
  }
}

// fork i: its table row, the counts of the pages that it shares (blockIdx.y 0), and its last page's content
__global__ __launch_bounds__(256) void pages_fork_rows_kernel(const PagesView c, const BatchView b, const int32_t* parents, const int32_t* children,
                                                             const Fork* forks, const int d) {
  const int i = blockIdx.x, piece = (int)blockIdx.y - 1;
  const Fork f = forks[i];
  if (f.len < 0) return;
  const int32_t* const src = b.table + (int64_t)parents[i] * b.table_stride;
  const int full = min(f.len >> c.log2_page, b.width);
  if (piece >= 0) {
    if (f.fresh >= 0) copy_piece(c, d, src[full], f.fresh, piece);
    return;
  }
  int32_t* const dst = b.table + (int64_t)children[i] * b.table_stride;
  for (int j = threadIdx.x; j < b.width; j += 256) {
    int p = -1;
    if (j < full) {
      p = src[j];
      if (is_page(c, p)) atomicAdd(&c.refs[p], 1);
    } else if (j == full) {
      p = f.fresh;
    }
    dst[j] = p;
  }
  if (threadIdx.x == 0) b.lens[children[i]] = f.len;
}

__global__ __launch_bounds__(256) void pages_free_kernel(const PagesView c, const BatchView b, const int32_t* rows) {
  const int s = rows[blockIdx.x];
  if (s < 0 || s >= b.n_seqs) return;
  int32_t* const row = b.table + (int64_t)s * b.table_stride;
  for (int j = threadIdx.x; j < b.width; j += 256) {
    const int p = atomicExch(&row[j], -1);  // (a row that is in the list twice gives its pages back once)
    if (is_page(c, p)) atomicSub(&c.refs[p], 1);
  }
  if (threadIdx.x == 0) b.lens[s] = 0;
}

// plan[0]: pages to move, plan[1]: pages in use; move[2 i], move[2 i + 1]: from, to; at[p]: where a page of plan[1] and above goes
__global__ __launch_bounds__(THREADS) void pages_compact_kernel(const PagesView c, int32_t* plan, int32_t* move, int32_t* at, int32_t* n_live) {
  __shared__ int wave_s[WAVES];
  int live = 0;
  for (int p0 = 0; p0 < c.n_pages; p0 += THREADS) {
    const int p = p0 + (int)threadIdx.x;
    rank_of(p < c.n_pages && c.refs[p] > 0, live, wave_s);
  }
  int holes = 0, moves = 0;
  for (int p0 = 0; p0 < c.n_pages; p0 += THREADS) {
    const int p = p0 + (int)threadIdx.x;
    const bool used = p < c.n_pages && c.refs[p] > 0;
    const bool hole = p < live && !used, goes = p >= live && used;
    if (p0 < live) {
      const int rank = rank_of(hole, holes, wave_s);
      if (hole) move[2 * rank + 1] = p;
    }
    if (p0 + THREADS > live) {
      const int rank = rank_of(goes, moves, wave_s);
      if (goes) move[2 * rank] = p;
      else if (p >= live && p < c.n_pages) at[p] = -1;
    }
  }
  if (threadIdx.x == 0) {
    plan[0] = moves;
    plan[1] = live;
    if (n_live != nullptr) *n_live = live;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < moves; i += THREADS) at[move[2 * i]] = move[2 * i + 1];
}

// the table's rows (blockIdx.y 0), and the pieces of the pages that move
__global__ __launch_bounds__(256) void pages_move_kernel(const PagesView c, const BatchView b, const int32_t* plan, const int32_t* move,
                                                        const int32_t* at, const int d) {
  const int moves = plan[0], live = plan[1], piece = (int)blockIdx.y - 1;
  if (piece < 0) {  // the table
    for (int s = blockIdx.x; s < b.n_seqs; s += gridDim.x) {
      int32_t* const row = b.table + (int64_t)s * b.table_stride;
      for (int j = threadIdx.x; j < b.width; j += 256) {
        const int p = row[j];
        if (p >= live && p < c.n_pages) row[j] = at[p];
      }
    }
    return;
  }
  for (int i = blockIdx.x; i < moves; i += gridDim.x) {
    const int from = move[2 * i], to = move[2 * i + 1];
    if (piece == 0 && threadIdx.x == 0) {
      c.refs[to] = c.refs[from];
      c.refs[from] = 0;
    }
    copy_piece(c, d, from, to, piece);
  }
}

__global__ __launch_bounds__(256) void pages_copy_kernel(const PagesView c, const int32_t* src, const int32_t* dst, const int64_t n, const int d) {
  for (int64_t i = blockIdx.x; i < n; i += gridDim.x) {
    const int from = src[i], to = dst[i];
    if (is_page(c, from) && is_page(c, to) && from != to) copy_piece(c, d, from, to, blockIdx.y);
  }
}

}  // namespace

hipError_t launch_pages_copy(const PagesView& c, int d, const int32_t* src, const int32_t* dst, int64_t n, hipStream_t s) {
  const dim3 grid((unsigned)(n < 65536 ? n : 65536), (unsigned)pieces_of(c, d));
  hipLaunchKernelGGL(pages_copy_kernel, grid, dim3(256), 0, s, c, src, dst, n, d);
  return hipGetLastError();
}

hipError_t launch_pages_reserve(const PagesView& c, const BatchView& b, int32_t* list, int32_t* missing, hipStream_t s) {
  // max_new positions lie in no more pages than this, nor in more than a sequence has entries
  int64_t each = (((int64_t)b.max_new + (1 << c.log2_page) - 2) >> c.log2_page) + 1;
  each = each < b.width ? each : b.width > 0 ? b.width : 1;
  hipLaunchKernelGGL(pages_reserve_kernel, dim3(1), dim3(THREADS), 0, s, c, b, Divide(each), list, missing);
  return hipGetLastError();
}

hipError_t launch_pages_fork(const PagesView& c, const BatchView& b, int d, const int32_t* parents, const int32_t* children, int n, int32_t* list,
                             int32_t* pairs, int32_t* missing, hipStream_t s) {
  Fork* const forks = reinterpret_cast<Fork*>(pairs);
  hipLaunchKernelGGL(pages_fork_kernel, dim3(1), dim3(THREADS), 0, s, c, b, parents, children, n, list, forks, missing);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || n == 0) return e;
  const dim3 grid((unsigned)n, (unsigned)pieces_of(c, d) + 1);
  hipLaunchKernelGGL(pages_fork_rows_kernel, grid, dim3(256), 0, s, c, b, parents, children, forks, d);
  return hipGetLastError();
}

hipError_t launch_pages_free(const PagesView& c, const BatchView& b, const int32_t* rows, int n, hipStream_t s) {
  hipLaunchKernelGGL(pages_free_kernel, dim3((unsigned)n), dim3(256), 0, s, c, b, rows);
  return hipGetLastError();
}

hipError_t launch_pages_compact(const PagesView& c, const BatchView& b, int d, int32_t* plan, int32_t* move, int32_t* at, int32_t* n_live, hipStream_t s) {
  hipLaunchKernelGGL(pages_compact_kernel, dim3(1), dim3(THREADS), 0, s, c, plan, move, at, n_live);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int64_t pairs = c.n_pages / 2 > b.n_seqs ? c.n_pages / 2 : b.n_seqs;
  if (pairs > 0) {
    const dim3 grid((unsigned)(pairs < 2048 ? pairs : 2048), (unsigned)pieces_of(c, d) + 1);
    hipLaunchKernelGGL(pages_move_kernel, grid, dim3(256), 0, s, c, b, plan, move, at, d);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace tq
