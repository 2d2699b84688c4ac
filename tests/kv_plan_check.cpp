// Sweeps the launch plans of the paged cache's attention on the host.  kv_plan_check RULE prints
// the first size that breaks the rule and returns 1, or returns 0.
//   covers   what a call's plan writes fits into the workspace of its sizes
#include <stdio.h>
#include <string.h>

#include "kv_plan.h"

using namespace kv;

static const int kKeep = 4096;       // pages of a selection's lists at most
static const int kHeads[] = {1, 2, 3, 8}, kGroups[] = {1, 4, 16, 64}, kDims[] = {128, 256};
static const int kPages[] = {32, 64, 128, 256};

static bool fits(int heads, int group, int d, int page, long tokens, int batch, int max_pages, int m) {
  const int hq = heads * group;
  const int64_t need = ws_need(heads, page, d, tokens, hq, batch, max_pages, kKeep);
  const Plan p = m ? plan_sel(heads, page, d, tokens, group, m)
                   : plan_dense(heads, page, d, tokens, batch, group, max_pages);
  if (part_bytes(tokens, hq, d, p.splits) <= need) return true;
  printf("heads %d group %d d %d page %d tokens %ld batch %d max_pages %d m %d: %d ranges take %lld "
         "bytes of %lld\n", heads, group, d, page, tokens, batch, max_pages, m, p.splits,
         (long long)part_bytes(tokens, hq, d, p.splits), (long long)need);
  return false;
}

static int covers() {
  for (int heads : kHeads)
    for (int group : kGroups)
      for (int d : kDims)
        for (int page : kPages)
          for (long tokens = 1; tokens <= 700; tokens += tokens < 140 ? 1 : 37) {
            // lists of every length; a table of one page has the smallest score rows
            for (int m = 1; m <= kKeep; m += m < 600 ? 1 : 7)
              if (!fits(heads, group, d, page, tokens, 1, 1, m)) return 1;
            for (int batch = 1; batch <= tokens; batch = batch * 2 + 1)
              for (int max_pages = 1; max_pages < 100000; max_pages = max_pages * 3 / 2 + 1)
                if (!fits(heads, group, d, page, tokens, batch, max_pages, 0)) return 1;
          }
  return 0;
}

int main(int argc, char** argv) {
  if (argc == 2 && !strcmp(argv[1], "covers")) return covers();
  return 2;
}
