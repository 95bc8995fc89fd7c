// Which kernel attends over pages, and into how many ranges the keys are cut: by sizes that the host knows.  (No HIP here: the tests ask it too.)
#pragma once
#include <algorithm>
#include <cstdint>

namespace tq {

constexpr int kPagesAttendWaves = 4;  // wavefronts of a workgroup of the kernel for few rows: each has a part of its keys
constexpr int pages_prompt_rows(int d) { return d == 256 ? 128 : 256; }  // to a workgroup of the kernel for prompts

struct PagesAttendSizes {
  int64_t n_seqs, max_new, width;
  int heads, group;  // of the cache; query heads that read one
  bool chosen;
  int64_t n_chosen;
  int log2_page;
  int64_t window;  // of tokens that a row sees; INT_MAX: all
  int64_t rows() const { return (chosen ? 1 : max_new) * group; }  // of a unit: a sequence and head, or a row and head
};
struct PagesAttendPlan {
  bool prompt;  // the kernel for prompts
  int splits, tiles;  // ranges of keys; tiles of 16 rows to a workgroup of the other kernel
};

// workgroups of one range each: sequences (or rows) times heads times tiles of query rows
inline int64_t pages_attend_units(const PagesAttendSizes& n, int tiles) {
  return n.n_seqs * n.heads * (n.chosen ? n.max_new : 1) * ((n.rows() + 16 * tiles - 1) / (16 * tiles));
}

inline PagesAttendPlan pages_attend_plan(int d, bool f32, const PagesAttendSizes& n, int64_t cus) {
  int64_t keys = (n.chosen ? n.n_chosen : n.width) << n.log2_page;
  if (!n.chosen && n.window + n.max_new < keys) keys = n.window + n.max_new;
  const int64_t rows = n.rows();
  PagesAttendPlan plan = {false, 1, 1};
  // More than 16 rows of bf16 queries, d = 128, and keys enough for every compute unit: 32 rows to a workgroup, which fetches and turns a tile
  // once for them.  us with 16 / 32 rows, 8 x 4 heads after 4096 tokens: 64 sequences of 8 rows 154 / 121, of 16 288 / 205, eight of 8
  // 30.1 / 25.6, one 12.9 / 14.3, one after 60000 37.0 / 34.3.  (d = 64: 27.0 / 27.3 for 16 sequences of 8 rows)
  if (rows > 16 && !f32 && d == 128 && pages_attend_units(n, 1) * keys >= 2048 * cus) plan.tiles = 2;
  const int64_t units = pages_attend_units(n, plan.tiles);
  if (units == 0) return plan;
  // Prompts.  The kernel for them shares a tile between 256 rows; ranges of no fewer than 1024 keys, as many as give no
  // compute unit a second workgroup, and taken where half of them (d = 256: three quarters) have one.
  // us there / in the kernel below (8 x 4 heads, d = 128): 4 x 2048 new tokens of 8192 930 / 2506, 512 of 4096 64 / 98, 128 of 4096 34 / 34, 512
  // of 512 24 / 22; 64 sequences of 4096 with 8 new tokens each (32 rows) 264 / 121, 16 (64 rows) 263 / 205, 32 279 / 577;
  // d = 256, where a workgroup has 128 rows: 427 of 1191 129 / 153, 500 of 1000 72 / 64
  const int64_t block = pages_prompt_rows(d), blocks = n.n_seqs * n.heads * ((rows + block - 1) / block);
  if (!n.chosen && !f32 && rows > 64) {
    const int64_t fill = cus / blocks, most = (keys + 1023) / 1024;
    plan.splits = (int)std::min(std::max(std::min(fill, most), (int64_t)1), (int64_t)16);
    plan.prompt = (d == 256 ? 4 : 6) * blocks * plan.splits >= 3 * cus;
    if (plan.prompt) return plan;
  }
  // As many ranges as give no compute unit a second workgroup while others have one (us by workgroups, 8 x 4 heads: 5 sequences of 8000
  // tokens 240 20.6, 280 24.3; 12 sequences 192 38.8, 288 44.2; 9 of 4000, d = 256, 216 31.0, 288 43.7).  Or as many as give every unit no
  // more than two: for d = 64, whose workgroups need half the registers and have half the bytes on their way (14 of 4000: 224 18.5, 448
  // 16.3; 24: 192 25.4, 384 23.0), and for few long ranges, where that fills the card better (20 of 8000: 160 74, 480 59) or evens out
  // lengths that differ (12, 14, 24 of 1000-8000: 192 37.0, 480 32.5; 224 37.1, 448 29.4; 192 60.0, 384 49.7; all of 8000: 37.8, 36.7; 39.3, 40.4;
  // 76.7, 81.9).  And as many as give them four where one range is more than one workgroup each and much less than two (36 sequences of 8000:
  // 288 138, 864 118, of 1000-8000 95, 81; d = 256 278, 231).
  const int64_t once = std::max(cus / units, (int64_t)1), twice = std::max((units > cus && 4 * units < 7 * cus ? 4 : 2) * cus / units, (int64_t)1);
  int64_t splits = once;
  if (d == 64 ? keys >= 512 * twice : once < 4 && (units > cus || (d == 128 && plan.tiles == 1)) && keys >= (twice == 2 ? 1536 : 1024) * twice) splits = twice;
  splits = std::min(std::min(splits, (keys + 32 * kPagesAttendWaves - 1) / (32 * kPagesAttendWaves)), (int64_t)64);  // (no more than there are tiles for their wavefronts)
  // The second launch has to be earned (one range / many, 8 x 4 heads: one token after 512 8.2 / 9.3, 768 9.6 / 9.2; 16 sequences, two
  // ranges, 1150 13.8 / 13.7, 1400 15.6 / 15.4; d = 256 384 9.7 / 10.4, 448 11.1 / 10.6)
  plan.splits = splits > 1 && keys * (splits - 1) > (d == 256 ? 320 : 640) * splits ? (int)splits : 1;
  return plan;
}

}  // namespace tq
