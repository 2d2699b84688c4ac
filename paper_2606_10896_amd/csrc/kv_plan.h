// Launch plans of the paged cache's attention and the workspace they need: host arithmetic on
// sizes, without a GPU header, so that a test can compile and sweep it.
#ifndef KV_PLAN_H
#define KV_PLAN_H

#include <stdint.h>

namespace kv {

constexpr int kCUs = 256;
// partial results of a row at most: 1024 keys each at 131,072 keys
constexpr int kMaxSplits = 128;
// a launch has fewer than 2^32 threads: so many workgroups of 256
constexpr int64_t kMaxThreads = ((int64_t)1 << 32) - 1;
constexpr int64_t kMaxBlocks = ((int64_t)1 << 24) - 1;

constexpr int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Row tiles and key ranges of an attention call.
struct Plan {
  int waves;               // k_attend_few: 4, or 8 for a whole row tile's keys in one workgroup
  int rt;                  // k_attend_few: 16 rt rows a tile, 0 if it is k_attend_tile
  int rows;                // k_attend_tile: rows of a tile
  int64_t items;           // row tiles of a head
  int tiles_token;
  int chunk, splits;
};

// Key ranges of k_attend_few: enough workgroups for every CU to hold two, whatever a range's
// length (a workgroup's first loads take as long as some steps: 8 sequences of 4000 keys, 4
// tokens and 32 rows each: 66 us in ranges of 128 keys, 32 in ranges of 512), and more where
// ranges stay above 1024 keys, which evens out ragged lengths (64 sequences of up to 32,768 keys:
// 811 us with 1024 workgroups, 686 with 2048, 657 with 4096, 652 with 8192).
inline int64_t few_ranges(int64_t tiles, int64_t keys) {
  if (tiles < 1) tiles = 1;          // the workspace of no tokens is asked for, too
  const int64_t fill = cdiv(2 * kCUs, tiles), even = cdiv(32 * kCUs, tiles);
  const int64_t long_ones = keys / 1024;
  int64_t want = even < long_ones ? even : long_ones;
  if (want < fill) want = fill;
  return want > kMaxSplits ? kMaxSplits : want;
}

// rows of a tile above 64 are shared through LDS (k_attend_tile)
inline int few_rows(int64_t rows, int d) { return rows <= 16 ? 1 : rows <= 32 || d > 128 ? 2 : 4; }

// One workgroup of eight waves takes all keys of a row tile where these are few or there are
// tiles for half of the CUs: nothing to join, one launch less.  (2048 keys, whole and split with
// its join: 256 tiles 45 us, 48; 32 tiles 35 us, 18; 8 tiles of 1000 keys 21 us, 13.)  From 2^23
// tiles on a launch holds no eight waves for each.
inline bool whole_rows(int64_t keys, int64_t tiles, int rt, int d) {
  return rt == 1 && d <= 128 && tiles * 512 <= kMaxThreads && keys <= (tiles >= kCUs / 2 ? 2048 : 512);
}

inline Plan plan_dense(int heads, int page, int d, int64_t tokens, int32_t batch, int group,
                       int32_t max_pages) {
  Plan p{};
  const int64_t keys = (int64_t)max_pages * page;
  const int64_t rows = cdiv(tokens, batch) * group;
  int64_t want, unit;
  if (rows > 64) {
    // eight waves share a step's operands from 65 to 128 dimensions (2048 tokens on 34,816 keys:
    // 0.98 ms, 1.11 in workgroups of four waves; 512 on 8512: 93 us, 136), but not for prompts
    // that are most of their own context, whose few steps a tile of 128 rows ends earlier at the
    // diagonal (32 heads on 8, eight waves and four: 2 prompts of 700 tokens 52 us, 32; 4: 57, 47;
    // 16: 181, 151; one of 2000 97, 90; 8 of 2000 415, 395; but 4 of 500 33, 35).  Up to 64 the
    // vector part takes longer than the matrix part, and three workgroups of four waves a CU hide
    // more of it (prompts of 4000 tokens with a window, when it was chosen: 0.21 ms, 0.23); above
    // 128 there are registers for four waves
    const bool prompt = keys <= 2048 && keys * batch <= 2 * tokens;
    p.rows = rows > 128 && d > 64 && d <= 128 && !prompt ? 256 : 128;
    const int64_t tiles = tokens * group / p.rows;
    p.items = tiles + batch;
    // one workgroup a CU; keys are split where there are fewer row tiles than that
    want = cdiv(kCUs, (tiles > 0 ? tiles : 1) * heads);
    unit = 512;
  } else {
    p.rt = few_rows(rows, d);
    p.items = tokens * group / (16 * p.rt) + batch;
    want = few_ranges(p.items * heads, keys);
    unit = 128;                      // a step of 32 keys for every wave
    p.waves = whole_rows(keys, p.items * heads, p.rt, d) ? 8 : 4;
    if (p.waves == 8) want = 1;
  }
  if (want > kMaxSplits) want = kMaxSplits;
  const int64_t chunk = cdiv(cdiv(keys, want), unit) * unit;
  p.chunk = (int)chunk;
  p.splits = (int)cdiv(keys, chunk);
  return p;
}

inline Plan plan_sel(int heads, int page, int d, int64_t tokens, int group, int32_t m) {
  Plan p{};
  p.rt = few_rows(group, d);
  p.tiles_token = (int)cdiv(group, 16 * p.rt);
  p.items = tokens * p.tiles_token;
  int64_t want = few_ranges(p.items * heads, (int64_t)m * page);
  p.waves = whole_rows((int64_t)m * page, p.items * heads, p.rt, d) ? 8 : 4;
  if (p.waves == 8) want = 1;
  const int least = page >= 128 ? 1 : 128 / page;
  int64_t chunk = cdiv(m, want);
  if (chunk < least) chunk = least;
  p.chunk = (int)chunk;
  p.splits = (int)cdiv(m, chunk);
  return p;
}

inline int64_t plan_threads(const Plan& p, int heads) {
  return p.items * heads * p.splits * (p.rt > 0 ? 64 * p.waves : 2 * p.rows);
}

inline int64_t part_bytes(int64_t tokens, int hq, int d, int splits) {
  return splits <= 1 ? 0 : (int64_t)splits * tokens * hq * (d + 2) * 4;
}

inline int64_t score_row(int32_t max_pages) { return cdiv(max_pages, 4) * 4; }

// The workspace is sized for every call of up to its sizes, not for one plan: fewer rows make
// more ranges (17 tokens of 32 heads on 8 may take no partial results, 16 tokens 128 ranges), and
// a list of m pages makes ceil(m / ceil(m / want)) of them, which does not grow with m (2016
// entries may make 126 ranges where 4096 make 125).
//
// Each kind of plan makes s > 1 ranges only for tiles * heads <= a / (s - 1), a + 1 being the
// workgroups it wants: it makes up to ceil((a + 1) / tiles) ranges.  A tile has at most c rows, so a
// head has at most f(s) = c (a / ((s - 1) heads) + extra) of them.  most_rows returns the largest
// s min(rows, f(s)) with 2 <= s <= most.  f falls with s, and s f(s) is convex: the largest value is at
// the last s with f(s) >= rows, at the one after it, or at the end.
inline int64_t most_rows(int64_t rows, int64_t c, int64_t a, int extra, int heads, int64_t most) {
  if (most > kMaxSplits) most = kMaxSplits;
  if (most > a / heads + 1) most = a / heads + 1;       // at least one tile
  if (most < 2) return 0;
  const auto all = [&](int64_t s) { return cdiv(s * c * a, (s - 1) * heads) + s * c * extra; };
  // f(s) >= rows for s - 1 <= c a / (heads (rows - c extra))
  const int64_t over = heads * (rows - c * extra);
  int64_t s1 = over > 0 ? c * a / over + 1 : most;
  if (s1 >= most) return most * rows;
  int64_t res = s1 >= 2 ? s1 * rows : 0;
  const int64_t next = all(s1 >= 2 ? s1 + 1 : 2), last = all(most);
  if (next > res) res = next;
  return last > res ? last : res;
}

inline int64_t ws_need(int heads, int page, int d, int64_t tokens, int hq, int32_t batch,
                       int32_t max_pages, int32_t max_keep) {
  const int group = hq / heads;
  const int64_t keys = (int64_t)max_pages * page, rows = tokens * group;
  // k_attend_few, at most 64 rows a sequence: floor(rows / (16 rt)) + batch tiles, batch at least
  // rows / 64; ranges have 128 keys, and 1024 beyond the first two workgroups a CU
  const int64_t few = rows < 64 * (int64_t)batch ? rows : 64 * (int64_t)batch;
  const int64_t c = d > 128 ? 22 : 32;       // 1 / (1 / (16 rt) + 1 / 64), rounded up
  const int64_t long_ones = keys / 1024;
  int64_t part = most_rows(few, c, 2 * kCUs - 1, 1, heads, cdiv(keys, 128));
  const auto more = [&](int64_t v) { part = v > part ? v : part; };
  more(most_rows(few, c, 32 * kCUs - 1, 1, heads, long_ones));
  // k_attend_tile: tiles of up to 256 rows, ranges of 512 keys
  more(most_rows(rows, 256, kCUs - 1, 1, heads, cdiv(keys, 512)));
  // selected pages: whole tiles a token
  const int64_t per = 16 * few_rows(group, d), ct = group < per ? group : per;
  const int64_t kept = (int64_t)max_keep * page;
  more(most_rows(rows, ct, 2 * kCUs - 1, 0, heads, kMaxSplits));
  more(most_rows(rows, ct, 32 * kCUs - 1, 0, heads, kept / 1024));
  const int64_t scores = tokens * heads * score_row(max_pages) * 4;
  part *= (int64_t)heads * (d + 2) * 4;
  return cdiv((part > scores ? part : scores) + 256, 256) * 256;
}

}  // namespace kv

#endif  // KV_PLAN_H
