// Prints, for every line "d f32 n_seqs max_new width heads group chosen n_chosen page window cus" of its input, which kernel attends over
// pages (1: the one for prompts), into how many ranges the keys are cut, and the tiles of 16 rows to a workgroup of the other kernel.
#include <climits>
#include <cstdio>

#include "../../paper_2504_19874_amd/csrc/tq_pages_plan.h"

int main() {
  long long d, f32, seqs, most, width, heads, group, chosen, n_chosen, page, window, cus;
  while (std::scanf("%lld %lld %lld %lld %lld %lld %lld %lld %lld %lld %lld %lld", &d, &f32, &seqs, &most, &width, &heads, &group, &chosen, &n_chosen, &page, &window, &cus) == 12) {
    int log2_page = 0;
    while ((1 << log2_page) < page) ++log2_page;
    const tq::PagesAttendSizes n{seqs, most, width, (int)heads, (int)group, chosen != 0, n_chosen, log2_page, window > 0 ? window : INT_MAX};
    const tq::PagesAttendPlan p = tq::pages_attend_plan((int)d, f32 != 0, n, cus);
    std::printf("%d %d %d\n", p.prompt ? 1 : 0, p.splits, p.tiles);
  }
  return 0;
}
