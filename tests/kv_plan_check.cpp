// Sweeps the launch plans of the paged cache's attention on the host.  kv_plan_check RULE prints
// the first size that breaks the rule and returns 1, or returns 0.
//   covers   what a call's plan writes fits into the workspace of its sizes
//   grows    a workspace for larger sizes serves smaller ones
//   launches the largest calls of up to 2^24 rows fit into a launch of fewer than 2^32 threads
#include <stdio.h>
#include <string.h>

#include <initializer_list>

#include "kv_plan.h"

using namespace kv;

static const int kKeep = 4096;       // pages of a selection's lists at most
static const int kHeads[] = {1, 2, 3, 5, 8, 16}, kGroups[] = {1, 4, 16, 64}, kDims[] = {128, 256};
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
          for (long tokens = 1; tokens <= 2100; tokens += tokens < 140 ? 1 : tokens < 1100 ? 37 : 333) {
            // lists of every length; a table of one page has the smallest score rows
            for (int m = 1; m <= kKeep; m += m < 600 ? 1 : 7)
              if (!fits(heads, group, d, page, tokens, 1, 1, m)) return 1;
            for (int batch = 1; batch <= tokens; batch = batch * 2 + 1)
              for (int max_pages = 1; max_pages < 100000; max_pages = max_pages * 3 / 2 + 1)
                if (!fits(heads, group, d, page, tokens, batch, max_pages, 0)) return 1;
          }
  return 0;
}

static int64_t need_of(int heads, int group, int d, int page, long tokens, int batch, int max_pages) {
  return ws_need(heads, page, d, tokens, heads * group, batch, max_pages, kKeep);
}

// along every size, the others held
static int grows() {
  static const long kTokens[] = {1, 2, 5, 16, 17, 33, 64, 65, 100, 255, 512, 1000, 2047, 2048, 20000};
  static const int kBatches[] = {1, 2, 3, 8, 64, 1000}, kWidths[] = {1, 3, 16, 32, 100, 2048, 60000};
  for (int heads = 1; heads <= 16; ++heads)
    for (int d : kDims)
      for (int page : kPages)
        for (int group = 1; group <= 64; ++group) {
          for (int batch : kBatches)
            for (int width : kWidths) {
              int64_t last = 0;
              for (long tokens : kTokens) {
                const int64_t need = need_of(heads, group, d, page, tokens, batch, width);
                if (need < last ||
                    need < need_of(heads, group > 1 ? group - 1 : 1, d, page, tokens, batch, width) ||
                    need < need_of(heads, group, d, page, tokens - 1, batch, width) ||
                    need < need_of(heads, group, d, page, tokens, batch > 1 ? batch - 1 : 1, width) ||
                    need < need_of(heads, group, d, page, tokens, batch, width > 1 ? width - 1 : 1)) {
                  printf("heads %d group %d d %d page %d tokens %ld batch %d max_pages %d: %lld bytes, "
                         "more for a smaller size\n", heads, group, d, page, tokens, batch, width,
                         (long long)need);
                  return 1;
                }
                last = need;
              }
            }
          if (group > 4 && heads > 2) group += 6;
        }
  // every count of tokens and of sequences of some shapes
  for (int heads : {1, 2, 8})
    for (int group : {1, 4, 7})
      for (int d : kDims)
        for (int width : {32, 2048}) {
          int64_t last = 0;
          for (long tokens = 0; tokens <= 9000; ++tokens) {
            const int64_t need = need_of(heads, group, d, 64, tokens, 1, width);
            if (need < last) return printf("tokens %ld heads %d group %d\n", tokens, heads, group), 1;
            last = need;
          }
          last = 0;
          for (int batch = 1; batch <= 3000; ++batch) {
            const int64_t need = need_of(heads, group, d, 64, 3000, batch, width);
            if (need < last) return printf("batch %d heads %d group %d\n", batch, heads, group), 1;
            last = need;
          }
        }
  return 0;
}

static int launches() {
  for (int heads : {1, 2, 3})
    for (int group : {1, 2, 3})
      for (int d : kDims)
        for (int page : kPages)
          for (long tokens = 1 << 20; tokens * heads * group < 1 << 24; tokens += tokens / 3 + 1)
            for (int n : {1, 2, 5, 16, 60}) {
              const Plan plans[] = {plan_sel(heads, page, d, tokens, group, n),
                                    plan_dense(heads, page, d, tokens, 1 << 20, group, n)};
              for (const Plan& p : plans) {
                const int threads = p.rt > 0 ? 64 * p.waves : 2 * p.rows;
                if (p.items * heads * p.splits >= 1 << 24) continue;       // refused in any case
                if (p.items * heads * p.splits * threads >= 1LL << 32)
                  return printf("heads %d group %d d %d page %d tokens %ld pages %d: %lld workgroups of %d\n",
                                heads, group, d, page, tokens, n,
                                (long long)(p.items * heads * p.splits), threads), 1;
              }
            }
  return 0;
}

int main(int argc, char** argv) {
  if (argc == 2 && !strcmp(argv[1], "covers")) return covers();
  if (argc == 2 && !strcmp(argv[1], "grows")) return grows();
  if (argc == 2 && !strcmp(argv[1], "launches")) return launches();
  return 2;
}
