// Pages of the key/value cache as a pool, for AMD Instinct MI355X (gfx950): copying, forking,
// growing and compacting.
//
// ref[p] counts the table entries that name page p, over all tables; 0 is a free page.  Every
// decision is taken on the GPU from the counts and tables, in an order that the sizes fix: atomics
// add and take minima of whole numbers, and give out slots of a hash table and of the list of copies,
// whose order no result depends on.
//
// Free and used pages are ranked by words: 64 pages make one by one ballot, a lane keeps a word, and a
// page's rank is a sum over words plus a bit count.

#include <hip/hip_runtime.h>

#include <limits.h>
#include <stdint.h>

#include "flashgmm.h"
#include "kv_host.h"
#include "kv_plan.h"

namespace {

using namespace kv;

constexpr int kWaves = 16;                        // of a workgroup that ranks pages
constexpr int kSpan = kWaves * 64 * 64;           // pages that it ranks at a time, at most

__device__ __forceinline__ int pages_of(int keys, int shift) {
  return keys <= 0 ? 0 : (keys >> shift) + ((keys & ((1 << shift) - 1)) != 0);
}

// ---------------------------------------------------------------- copies
struct Pages {
  char* k;
  char* v;
  char* box;
  float* scale;
  int pages;
};

struct CopyArgs {
  Pages src, dst;
  int bytes;                  // of a page's keys, and of its values: up to 2^27
  int box_bytes, heads;
  const int32_t* from;
  const int32_t* to;
  const int32_t* count;       // pairs, or null: n
  int n;
};

// Work items of a pair: `parts` of its keys, as many of its values, and its box.  A thread moves 16
// bytes in each of kSteps steps, all loads before the stores, streamed past the caches.  Sizes within a
// page are 32-bit: hipcc (ROCm 7.2) took the shorter of two uniform 64-bit lengths from a flag that its
// comparison does not set, and an incomplete part was copied whole.
template <int kThreads, int kSteps>
__device__ __forceinline__ void copy_items(const CopyArgs& a, int block, int blocks) {
  typedef uint32_t V __attribute__((ext_vector_type(4)));
  constexpr int kBytes = kThreads * 16, kPart = kBytes * kSteps;
  const int n = a.count ? *a.count : a.n;
  const int parts = (a.bytes + kPart - 1) / kPart, per = 2 * parts + (a.dst.box != nullptr);
  const int step_pair = blocks / per, step_part = blocks - step_pair * per;
  int pair = block / per, part = block - pair * per;
  while (pair < n) {
    const int from = a.from[pair], to = a.to[pair];
    if (from >= 0 && from < a.src.pages && to >= 0 && to < a.dst.pages) {
      if (part < 2 * parts) {
        const bool values = part >= parts;
        const int at = (values ? part - parts : part) * kPart + threadIdx.x * 16;
        const char* f = (values ? a.src.v : a.src.k) + (int64_t)from * a.bytes + at;
        char* t = (values ? a.dst.v : a.dst.k) + (int64_t)to * a.bytes + at;
        V v[kSteps];
#pragma unroll
        for (int i = 0; i < kSteps; ++i)
          if (at + i * kBytes < a.bytes)
            v[i] = __builtin_nontemporal_load(reinterpret_cast<const V*>(f + i * kBytes));
#pragma unroll
        for (int i = 0; i < kSteps; ++i)
          if (at + i * kBytes < a.bytes)
            __builtin_nontemporal_store(v[i], reinterpret_cast<V*>(t + i * kBytes));
      } else {
        const char* f = a.src.box + (int64_t)from * a.box_bytes;
        char* t = a.dst.box + (int64_t)to * a.box_bytes;
        for (int at = threadIdx.x * 16; at < a.box_bytes; at += kBytes)
          *reinterpret_cast<V*>(t + at) = *reinterpret_cast<const V*>(f + at);
        for (int i = threadIdx.x; i < a.heads; i += kThreads)
          a.dst.scale[(int64_t)to * a.heads + i] = a.src.scale[(int64_t)from * a.heads + i];
      }
    }
    pair += step_pair;
    part += step_part;
    if (part >= per) {
      part -= per;
      ++pair;
    }
  }
}

// The number of pairs is known to the host: a workgroup an item, in the order of the addresses.
// Bound by bytes: 2048 pages of 256 KiB between two caches 190 us, 5.7 TB/s (a plain 2 GiB copy: 4.96).
// With four accesses a thread 232 us, and without streaming past the caches 4 % more.
__global__ __launch_bounds__(256) void k_kv_copy(CopyArgs a) {
  copy_items<256, 1>(a, blockIdx.x, gridDim.x);
}

// It is not: few workgroups with more in flight each, as empty ones cost (compacting, 1049 pages of 256
// KiB of up to 2120: 105 us, 5.3 TB/s; a workgroup an item 128).
template <int kThreads, int kSteps>
__global__ __launch_bounds__(kThreads) void k_kv_copy_some(CopyArgs a) {
  copy_items<kThreads, kSteps>(a, blockIdx.x, gridDim.x);
}

// ---------------------------------------------------------------- fork
struct ForkArgs {
  int32_t* ref;
  int cache_pages, shift;
  const int32_t* total;
  const int32_t* pages;
  int64_t stride;
  int batch, max_pages;
  const int32_t* parent;
  const int32_t* keep;
  int rows, release;
  int32_t* total_out;
  int32_t* pages_out;
  int64_t out_stride;
  int out_max;
  int span;                   // entries of a workgroup
};

__device__ __forceinline__ void count(const ForkArgs& a, int page, int by) {
  if (page >= 0 && page < a.cache_pages) atomicAdd(a.ref + page, by);
}

// Is p among the first n parents?  The same answer in every thread.
__device__ __forceinline__ bool named(const ForkArgs& a, int p, int n) {
  for (int i0 = 0; i0 < n; i0 += 4096) {
    bool hit = false;
#pragma unroll
    for (int k = 0; k < 16; ++k) {
      const int i = i0 + k * 256 + threadIdx.x;
      hit |= i < n && a.parent[min(i, n - 1)] == p;
    }
    if (__syncthreads_or(hit)) return true;
  }
  return false;
}

// Workgroups of a new row copy its parent's entries, those of an old row without a child give up
// its pages.  An old row's counts pass to its first child, so that rows that go on alone change
// none.  Bound by latency (parent, total, parents, entries, counts) and by atomics: 7.5 us for 512
// rows of up to 512 pages, 3.2 for 20 rows.
__global__ __launch_bounds__(256) void k_kv_fork(ForkArgs a) {
  const int row = blockIdx.x;
  const int e0 = blockIdx.y * a.span, e1 = e0 + a.span;
  if (row >= a.rows) {
    const int b = row - a.rows;
    const int n = min(pages_of(a.total[b], a.shift), a.max_pages);
    if (e0 >= n || named(a, b, a.rows)) return;
    for (int e = e0 + threadIdx.x; e < min(e1, n); e += 256) count(a, a.pages[b * a.stride + e], -1);
    return;
  }
  const int p = a.parent[row];
  const bool ok = p >= 0 && p < a.batch;
  const int have = ok ? max(a.total[p], 0) : 0;
  const int kept = a.keep ? min(have, max(a.keep[row], 0)) : have;
  const int nold = min(pages_of(have, a.shift), a.max_pages);
  const int n = min(pages_of(kept, a.shift), a.max_pages);
  if (blockIdx.y == 0 && threadIdx.x == 0) a.total_out[row] = kept;
  const bool heir = a.release && ok && e0 < nold && !named(a, p, row);
  for (int e = e0 + threadIdx.x; e < min(e1, a.out_max); e += 256) {
    int page = -1;
    if (e < n) {
      page = a.pages[p * a.stride + e];
      if (!heir) count(a, page, 1);
    } else if (heir && e < nold) {
      count(a, a.pages[p * a.stride + e], -1);
    }
    a.pages_out[row * a.out_stride + e] = page;
  }
}

// ---------------------------------------------------------------- ranks of pages
// lane `i`'s value, of a lane that is the same for the wave
__device__ __forceinline__ uint64_t lane_value(uint64_t v, int i) {
  return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), i) << 32 |
         (uint32_t)__builtin_amdgcn_readlane((int)v, i);
}
// set bits of the lanes before
__device__ __forceinline__ int below(uint64_t bits) {
  return __builtin_amdgcn_mbcnt_hi((uint32_t)(bits >> 32),
                                   __builtin_amdgcn_mbcnt_lo((uint32_t)bits, 0));
}

// Inclusive sum over the wave's lanes.
template <typename T>
__device__ __forceinline__ T wave_sum(T v) {
  const int lane = threadIdx.x & 63;
  for (int o = 1; o < 64; o <<= 1) {
    const T p = __shfl_up(v, o);
    if (lane >= o) v += p;
  }
  return v;
}

// Exclusive sum over the workgroup's threads, in their order, and the sum of all.
template <typename T>
__device__ __forceinline__ T group_sum(T v, T* tmp, T* all) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const T incl = wave_sum(v);
  __syncthreads();
  if (lane == 63) tmp[w] = incl;
  __syncthreads();
  T before = 0, total = 0;
  for (int i = 0; i < kWaves; ++i) {
    if (i < w) before += tmp[i];
    total += tmp[i];
  }
  *all = total;
  return before + incl - v;
}

// Words of the pages from `first` on: wave w's words are those of its `words` x 64 pages in a
// row, word i of them in lane i; a bit is set where the page is used.
template <int kFlight>
__device__ __forceinline__ uint64_t load_words(const int32_t* ref, int pages, int base, int words) {
  const int lane = threadIdx.x & 63;
  uint64_t mine = 0;
  for (int i = 0; i < words; i += kFlight) {
    int v[kFlight];                  // loads in flight
#pragma unroll
    for (int j = 0; j < kFlight; ++j) v[j] = ref[min(base + (i + j) * 64, pages - 1)];
#pragma unroll
    for (int j = 0; j < kFlight; ++j) {
      const uint64_t bits = __ballot(i + j < words && base + (i + j) * 64 < pages && v[j] > 0);
      if (lane == i + j) mine = bits;
    }
  }
  return mine;
}
__device__ __forceinline__ uint64_t load_words(const int32_t* ref, int pages, int first, int words) {
  const int base = first + (int)(threadIdx.x >> 6) * words * 64 + (int)(threadIdx.x & 63);
  return words > 8 ? load_words<32>(ref, pages, base, words) : load_words<4>(ref, pages, base, words);
}
__device__ __forceinline__ int words_of(int pages) {
  return pages >= kSpan ? 64 : (pages + 64 * kWaves - 1) / (64 * kWaves);
}

// Used pages of the spans of 1024 `words` pages, a workgroup each.
__global__ __launch_bounds__(64 * kWaves) void k_kv_count(const int32_t* ref, int pages, int words,
                                                          int32_t* counts) {
  __shared__ int tmp[kWaves];
  int all;
  group_sum((int)__popcll(load_words(ref, pages, (int)blockIdx.x * 64 * kWaves * words, words)), tmp,
            &all);
  if (threadIdx.x == 0) counts[blockIdx.x] = all;
}

// ---------------------------------------------------------------- grow
struct GrowArgs {
  int32_t* ref;
  int cache_pages, shift;
  const int32_t* held;
  const int32_t* total;
  int32_t* pages;
  int64_t stride;
  int batch, max_pages;
  int32_t* short_by;
  // workspace
  int32_t* count;             // copies
  int32_t* from;              // [batch]
  int32_t* to;                // [batch]
  int32_t* base;              // [batch] pages needed by the rows before
  int32_t* cow;               // [batch] the shared page that the row writes into, or -1
  int32_t* first;             // [cache pages] first row that writes into a shared page
  int32_t* writers;           // [cache pages] rows that do
  int32_t* free_list;         // [cache pages]
  const int32_t* counts;      // used pages of every kSpan pages of a larger pool, or null
};

__device__ __forceinline__ int load_agent(const int32_t* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ void store_agent(int32_t* p, int v) {
  __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// The shared page that a row writes into, or -1.
__device__ __forceinline__ int shared_page(const GrowArgs& a, int r, int held, int total) {
  if (held <= 0 || total <= held || (held & ((1 << a.shift) - 1)) == 0) return -1;
  const int e = held >> a.shift;
  if (e >= a.max_pages) return -1;
  const int p = a.pages[r * a.stride + e];
  return p >= 0 && p < a.cache_pages && a.ref[p] > 1 ? p : -1;
}
__device__ __forceinline__ int fresh_pages(const GrowArgs& a, int held, int total) {
  return max(0, min(pages_of(total, a.shift), a.max_pages) - pages_of(held, a.shift));
}

// Free pages of a span, a word of 64 in a lane.
__device__ __forceinline__ uint64_t free_words(const GrowArgs& a, int first, int words) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int p0 = first + (w * words + lane) * 64;
  uint64_t bits = 0;
  if (lane < words && p0 < a.cache_pages)
    bits = a.cache_pages - p0 >= 64 ? ~0ull : (1ull << (a.cache_pages - p0)) - 1;
  return bits & ~load_words(a.ref, a.cache_pages, first, words);
}

constexpr int kRows = 64 * kWaves;     // rows that a workgroup takes at once
constexpr int kSlots = 2 * kRows;      // of their table of shared pages
constexpr int kList = 4096;            // free pages kept in LDS

// One workgroup takes all decisions: what a row needs, which free pages there are, who gets which.
// Bound by the latency of that chain, 8.0 us for 512 rows that share pages, 5.8 for 9 rows and 1108
// pages, and by the counts' 64 bytes a clock of one CU (65,536 pages: 12 us, 8192: 6.5).
// kFew: up to kRows rows, which stay in LDS; else they pass through the workspace (512 rows: 11 us).
template <bool kFew>
__global__ __launch_bounds__(64 * kWaves) void k_kv_grow(GrowArgs a) {
  __shared__ int tmp[kWaves];
  __shared__ int64_t tmp64[kWaves];
  __shared__ int copies;
  __shared__ int slot_page[kFew ? kSlots : 1], slot_first[kFew ? kSlots : 1], slot_rows[kFew ? kSlots : 1];
  __shared__ int row_base[kFew ? kRows : 1], row_held[kFew ? kRows : 1], row_cow[kFew ? kRows : 1];
  __shared__ int list[kList];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  int64_t want = 0;
  uint64_t bits = 0;
  const int words0 = words_of(a.cache_pages);
  if (tid == 0) copies = 0;
  // what a row needs; of the rows that write into one shared page, the first keeps it if no other
  // row holds it
  if constexpr (kFew) {
    const bool in = tid < a.batch;
    const int held = in ? a.held[tid] : 0, total = in ? a.total[tid] : 0;
    bits = free_words(a, 0, words0);                 // needed later: under way meanwhile
    for (int i = tid; i < kSlots; i += kRows) {
      slot_page[i] = -1;
      slot_first[i] = INT_MAX;
      slot_rows[i] = 0;
    }
    const int p = in ? shared_page(a, tid, held, total) : -1;
    const int holders = p >= 0 ? a.ref[p] : 0;
    __syncthreads();
    int slot = (int)((uint32_t)p * 2654435761u >> 21);
    if (p >= 0) {
      for (;; slot = (slot + 1) & (kSlots - 1)) {    // half of the slots stay empty
        const int was = atomicCAS(slot_page + slot, -1, p);
        if (was == -1 || was == p) break;
      }
      atomicMin(slot_first + slot, tid);
      atomicAdd(slot_rows + slot, 1);
    }
    __syncthreads();
    const bool keeps = p >= 0 && holders <= slot_rows[slot] && slot_first[slot] == tid;
    const int cow = keeps ? -1 : p;
    const int64_t before =
        group_sum((int64_t)fresh_pages(a, held, total) + (cow >= 0), tmp64, &want);
    row_base[tid] = (int)min(before, (int64_t)INT_MAX);
    row_held[tid] = held;
    row_cow[tid] = cow;
  } else {
    for (int r = tid; r < a.batch; r += kRows) {
      const int p = shared_page(a, r, a.held[r], a.total[r]);
      a.cow[r] = p;
      if (p >= 0) {
        store_agent(a.first + p, INT_MAX);
        store_agent(a.writers + p, 0);
      }
    }
    __syncthreads();
    for (int r = tid; r < a.batch; r += kRows) {
      const int p = a.cow[r];
      if (p >= 0) {
        atomicMin(a.first + p, r);
        atomicAdd(a.writers + p, 1);
      }
    }
    __syncthreads();
    for (int r0 = 0; r0 < a.batch; r0 += kRows) {
      const int r = r0 + tid;
      int64_t need = 0;               // up to 2^25 a row
      if (r < a.batch) {
        need = fresh_pages(a, a.held[r], a.total[r]);
        const int p = a.cow[r];
        if (p >= 0) {
          if (a.ref[p] <= load_agent(a.writers + p) && load_agent(a.first + p) == r) a.cow[r] = -1;
          else ++need;
        }
      }
      int64_t all;
      const int64_t before = group_sum(need, tmp64, &all);
      // a sum past the pool's size is capped: what it says is that the pool is short
      if (r < a.batch) a.base[r] = (int)min(want + before, (int64_t)INT_MAX);
      want += all;
    }
    bits = free_words(a, 0, words0);
  }
  // the first `want` free pages
  int64_t have = 0;
  for (int first = 0; first < a.cache_pages && have < want; first += kSpan) {
    const int words = words_of(a.cache_pages - first);
    if (a.counts && a.counts[first / kSpan] == min(kSpan, a.cache_pages - first)) continue;
    if (first > 0) bits = free_words(a, first, words);
    int all;
    const int rank = group_sum((int)__popcll(bits), tmp, &all);
    for (int i = 0; i < words; ++i) {
      const uint64_t b = lane_value(bits, i);
      const int64_t at = have + __builtin_amdgcn_readlane(rank, i);
      if (at >= want) break;
      const int64_t k = at + below(b);
      if ((b >> lane & 1) && k < want) {
        const int page = first + (w * words + i) * 64 + lane;
        if (k < kList) list[k] = page;
        else a.free_list[k] = page;
      }
    }
    have += all;
  }
  if (tid == 0) a.short_by[0] = have < want ? (int)min(want - have, (int64_t)INT_MAX) : 0;
  __syncthreads();
  if (have >= want) {
    const int* base = kFew ? row_base : a.base;
    for (int k = tid; k < want; k += kRows) {
      int lo = 0, hi = a.batch;        // the last row with base <= k
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (base[mid] <= k) lo = mid;
        else hi = mid;
      }
      const int page = k < kList ? list[k] : a.free_list[k];
      int i = k - base[lo];
      const int held = kFew ? row_held[lo] : a.held[lo], old = kFew ? row_cow[lo] : a.cow[lo];
      if (old >= 0 && i-- == 0) {
        const int c = atomicAdd(&copies, 1);
        a.from[c] = old;
        a.to[c] = page;
        atomicSub(a.ref + old, 1);
        a.pages[lo * a.stride + (held >> a.shift)] = page;
      } else {
        a.pages[lo * a.stride + pages_of(held, a.shift) + i] = page;
      }
      a.ref[page] = 1;
    }
  }
  __syncthreads();
  if (tid == 0) a.count[0] = copies;
}

// ---------------------------------------------------------------- compact
struct CompactArgs {
  int32_t* ref;
  int cache_pages, shift;
  const int32_t* total;
  int32_t* pages;
  int64_t stride;
  int batch, max_pages;
  int32_t* where;
  int32_t* used;
  // workspace
  int32_t* count;             // pages moved
  int32_t* from;              // [cache pages / 2]
  int32_t* to;
  int32_t* counts;            // [spans] used pages, not with one span
  int words, spans;           // a workgroup has 1024 words pages
};

// With U used pages, those at U and above go to the free ones below, in order.  A workgroup a span
// finds the places of its pages from the spans' counts: the k-th free page below U is to[k], the
// k-th used one from U on from[k], which is noted as -2 - k until it has moved.  5 us for 4240 pages;
// one workgroup for a pool of 2^20 took 2 ms.
__global__ __launch_bounds__(64 * kWaves) void k_kv_places(CompactArgs a) {
  __shared__ int tmp[kWaves];
  __shared__ int prefix[64 * kWaves];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, span = 64 * kWaves * a.words;
  const int first = blockIdx.x * span;
  const uint64_t bits = load_words(a.ref, a.cache_pages, first, a.words);
  int used, all, rank = group_sum((int)__popcll(bits), tmp, &used);
  int below_u;                         // used pages below U
  uint64_t bits_u = bits;
  int at_u = 0;                        // first page of the span that holds page U
  if (a.spans > 1) {
    const int before = group_sum(tid < a.spans ? a.counts[tid] : 0, tmp, &used);
    prefix[tid] = before;
    __syncthreads();
    rank += prefix[blockIdx.x];
    at_u = min(used / span, a.spans - 1) * span;
    bits_u = load_words(a.ref, a.cache_pages, at_u, a.words);
    below_u = prefix[at_u / span];
  } else {
    below_u = 0;
  }
  const int p0 = at_u + (w * a.words + lane) * 64;
  if (lane >= a.words || p0 >= used) bits_u = 0;
  else if (used - p0 < 64) bits_u &= (1ull << (used - p0)) - 1;
  group_sum((int)__popcll(bits_u), tmp, &all);
  below_u += all;
  for (int i = 0; i < a.words; ++i) {
    const uint64_t b = lane_value(bits, i);
    const int p = first + (w * a.words + i) * 64 + lane;
    const int before = __builtin_amdgcn_readlane(rank, i) + below(b);
    if (p >= a.cache_pages) continue;
    const bool in = b >> lane & 1;
    int place = in ? p : -1;
    if (p < used && !in) a.to[p - before] = p;
    if (p >= used && in) {
      a.from[before - below_u] = p;
      place = -2 - (before - below_u);
    }
    a.where[p] = place;
  }
  if (blockIdx.x == 0 && tid == 0) {
    a.used[0] = used;
    a.count[0] = used - below_u;
  }
}

// The first `blocks` workgroups copy and note the new places, the others rewrite the tables: a part of
// a row, an entry a thread.  A place that is being noted reads as either of two that say the same.
template <int kThreads, int kSteps>
__global__ __launch_bounds__(kThreads) void k_kv_move(CopyArgs c, CompactArgs a, int blocks,
                                                      int spans) {
  if ((int)blockIdx.x < blocks) {
    const int moves = *a.count;
    for (int i = blockIdx.x * kThreads + threadIdx.x; i < moves; i += blocks * kThreads) {
      const int from = a.from[i], to = a.to[i];
      a.where[from] = to;
      a.ref[to] = a.ref[from];
      a.ref[from] = 0;
    }
    copy_items<kThreads, kSteps>(c, blockIdx.x, blocks);
    return;
  }
  const int item = (int)blockIdx.x - blocks, row = item / spans;
  const int e = (item - row * spans) * kThreads + (int)threadIdx.x;
  if (e >= min(pages_of(a.total[row], a.shift), a.max_pages)) return;
  const int p = a.pages[(int64_t)row * a.stride + e];
  if (p < 0 || p >= a.cache_pages) return;
  const int place = a.where[p];
  const int to = place < -1 ? a.to[-2 - place] : place;
  if (to >= 0 && to != p) a.pages[(int64_t)row * a.stride + e] = to;
}

// ---------------------------------------------------------------- host
Pages pages_at(const gmm_kv_cache* c) {
  return Pages{(char*)c->k, (char*)c->v, (char*)c->box, c->box_scale, c->pages};
}

void set_copy(const gmm_kv_cache* src, const gmm_kv_cache* dst, CopyArgs* a) {
  a->src = pages_at(src);
  a->dst = pages_at(dst);
  a->bytes = dst->heads * dst->page * dst->d * 2;
  a->box_bytes = dst->heads * 2 * dst->d;
  a->heads = dst->heads;
}

// The number of pages to copy is known on the GPU: up to two workgroups a CU of 1024 threads, as many
// threads in smaller ones where a page's keys leave most of 1024 idle.
constexpr int kSmallPage = 8192;

// workgroups for up to `pairs` pages, `units` of 16 bytes an item
int64_t copy_blocks(const CopyArgs& a, int64_t pairs, int units) {
  const int64_t items = pairs * (2 * cdiv(a.bytes, units * 16) + 1);
  const int64_t most = a.bytes > kSmallPage ? 8 * kCUs : 32 * kCUs;
  return items < most ? items : most;
}

int64_t pool_need(const gmm_kv_cache* c, int32_t batch) {
  return cdiv(256 + 4 * (3 * (int64_t)c->pages + 4 * (int64_t)batch + 64 + 1024), 256) * 256;
}

int check_tables(const gmm_kv_cache* c, int32_t batch, int32_t max_pages, int64_t stride) {
  if (batch < 1 || max_pages < 1 || stride < max_pages) return GMM_ERR_INVALID_ARG;
  if ((int64_t)max_pages * c->page > (1 << 30) || batch > GMM_KV_MAX_ROWS || c->pages > GMM_KV_MAX_POOL)
    return GMM_ERR_UNSUPPORTED;
  return GMM_OK;
}

int64_t table_bytes(int64_t rows, int64_t stride, int32_t max_pages) {
  return rows < 1 ? 0 : ((rows - 1) * stride + max_pages) * 4;
}

}  // namespace

extern "C" {

int gmm_kv_copy(const gmm_kv_cache* src, const gmm_kv_cache* dst, const int32_t* src_pages,
                const int32_t* dst_pages, int64_t n, hipStream_t stream) {
  int rc = check_cache(src);
  if (rc != GMM_OK) return rc;
  rc = check_cache(dst);
  if (rc != GMM_OK) return rc;
  if (src->heads != dst->heads || src->page != dst->page || src->d != dst->d ||
      src->dtype != dst->dtype || (src->box == nullptr) != (dst->box == nullptr) || n < 0)
    return GMM_ERR_INVALID_ARG;
  if (n > (1 << 30)) return GMM_ERR_UNSUPPORTED;
  if (n == 0) return GMM_OK;
  if (!src_pages || !dst_pages) return GMM_ERR_INVALID_ARG;
  CopyArgs a{};
  set_copy(src, dst, &a);
  a.from = src_pages;
  a.to = dst_pages;
  a.n = (int)n;
  const int64_t items = n * (2 * cdiv(a.bytes, 4096) + (a.dst.box != nullptr));
  hipLaunchKernelGGL(k_kv_copy, dim3((unsigned)(items < (1 << 20) ? items : 1 << 20)), dim3(256), 0,
                     stream, a);
  return launch_status();
}

int gmm_kv_fork(const gmm_kv_cache* cache, int32_t* ref, const int32_t* total,
                const int32_t* pages, int32_t batch, int32_t max_pages, int64_t pages_stride,
                const int32_t* parent, const int32_t* keep, int32_t rows, int32_t release,
                int32_t* total_out, int32_t* pages_out, int32_t out_max_pages,
                int64_t out_stride, hipStream_t stream) {
  int rc = check_cache(cache);
  if (rc != GMM_OK) return rc;
  rc = check_tables(cache, batch, max_pages, pages_stride);
  if (rc != GMM_OK) return rc;
  if (!ref || !total || !pages || rows < 0) return GMM_ERR_INVALID_ARG;
  if (rows > GMM_KV_MAX_ROWS) return GMM_ERR_UNSUPPORTED;
  if (rows > 0) {
    if (!parent || !total_out || !pages_out || out_max_pages < max_pages ||
        out_stride < out_max_pages)
      return GMM_ERR_INVALID_ARG;
    if ((int64_t)out_max_pages * cache->page > (1 << 30)) return GMM_ERR_UNSUPPORTED;
    // what is read or counted while the new tables are written
    const int64_t wide = table_bytes(rows, out_stride, out_max_pages);
    const auto hit = [&](const void* p, int64_t bytes) {
      return p && (overlap(p, bytes, total_out, 4 * (int64_t)rows) || overlap(p, bytes, pages_out, wide));
    };
    if (hit(pages, table_bytes(batch, pages_stride, max_pages)) || hit(total, 4 * (int64_t)batch) ||
        hit(parent, 4 * (int64_t)rows) || hit(keep, 4 * (int64_t)rows) ||
        hit(ref, 4 * (int64_t)cache->pages) || overlap(total_out, 4 * (int64_t)rows, pages_out, wide))
      return GMM_ERR_INVALID_ARG;
  }
  ForkArgs a{};
  a.ref = ref;
  a.cache_pages = cache->pages;
  a.shift = log2i(cache->page);
  a.total = total;
  a.pages = pages;
  a.stride = pages_stride;
  a.batch = batch;
  a.max_pages = max_pages;
  a.parent = parent;
  a.keep = keep;
  a.rows = rows;
  a.release = release != 0;
  a.total_out = total_out;
  a.pages_out = pages_out;
  a.out_stride = out_stride;
  a.out_max = out_max_pages;
  const int64_t blocks = (int64_t)rows + (release ? batch : 0);
  if (blocks == 0) return GMM_OK;
  const int64_t width = rows > 0 ? out_max_pages : max_pages;
  // up to 256 workgroups a row
  a.span = 1024;
  while (cdiv(width, a.span) > 256 || blocks * cdiv(width, a.span) > kMaxBlocks) a.span *= 2;
  hipLaunchKernelGGL(k_kv_fork, dim3((unsigned)blocks, (unsigned)cdiv(width, a.span)), dim3(256),
                     0, stream, a);
  return launch_status();
}

size_t gmm_kv_pool_workspace_bytes(const gmm_kv_cache* cache, int32_t batch) {
  if (check_cache(cache) != GMM_OK || check_tables(cache, batch, 1, 1) != GMM_OK) return 0;
  return (size_t)pool_need(cache, batch);
}

int gmm_kv_grow(const gmm_kv_cache* cache, int32_t* ref, const int32_t* held,
                const int32_t* total, int32_t* pages, int32_t batch, int32_t max_pages,
                int64_t pages_stride, int32_t* short_by, void* ws, size_t ws_bytes,
                hipStream_t stream) {
  int rc = check_cache(cache);
  if (rc != GMM_OK) return rc;
  rc = check_tables(cache, batch, max_pages, pages_stride);
  if (rc != GMM_OK) return rc;
  if (!ref || !held || !total || !pages || !short_by) return GMM_ERR_INVALID_ARG;
  rc = check_kv_ws(ws, ws_bytes, pool_need(cache, batch));
  if (rc != GMM_OK) return rc;
  GrowArgs a{};
  a.ref = ref;
  a.cache_pages = cache->pages;
  a.shift = log2i(cache->page);
  a.held = held;
  a.total = total;
  a.pages = pages;
  a.stride = pages_stride;
  a.batch = batch;
  a.max_pages = max_pages;
  a.short_by = short_by;
  a.count = (int32_t*)ws;
  a.from = a.count + 64;
  a.to = a.from + batch;
  a.base = a.to + batch;
  a.cow = a.base + batch;
  a.first = a.cow + batch;
  a.writers = a.first + cache->pages;
  a.free_list = a.writers + cache->pages;
  if (cache->pages > kSpan) {
    // up to 1024 spans; full ones are passed over
    int32_t* counts = a.free_list + cache->pages;
    a.counts = counts;
    hipLaunchKernelGGL(k_kv_count, dim3((unsigned)cdiv(cache->pages, kSpan)), dim3(64 * kWaves), 0,
                       stream, ref, cache->pages, kSpan / (64 * kWaves), counts);
  }
  if (batch <= kRows) hipLaunchKernelGGL(k_kv_grow<true>, dim3(1), dim3(kRows), 0, stream, a);
  else hipLaunchKernelGGL(k_kv_grow<false>, dim3(1), dim3(kRows), 0, stream, a);
  CopyArgs c{};
  set_copy(cache, cache, &c);
  c.from = a.from;
  c.to = a.to;
  c.count = a.count;
  const auto copy = [&](auto kernel, int threads, int steps) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)copy_blocks(c, batch, threads * steps)), dim3(threads), 0,
                       stream, c);
  };
  if (c.bytes > kSmallPage) copy(k_kv_copy_some<1024, 4>, 1024, 4);
  else copy(k_kv_copy_some<256, 2>, 256, 2);
  return launch_status();
}

int gmm_kv_compact(const gmm_kv_cache* cache, int32_t* ref, const int32_t* total, int32_t* pages,
                   int32_t batch, int32_t max_pages, int64_t pages_stride, int32_t* where,
                   int32_t* used, void* ws, size_t ws_bytes, hipStream_t stream) {
  int rc = check_cache(cache);
  if (rc != GMM_OK) return rc;
  rc = check_tables(cache, batch, max_pages, pages_stride);
  if (rc != GMM_OK) return rc;
  if (!ref || !total || !pages || !where || !used) return GMM_ERR_INVALID_ARG;
  rc = check_kv_ws(ws, ws_bytes, pool_need(cache, batch));
  if (rc != GMM_OK) return rc;
  CompactArgs a{};
  a.ref = ref;
  a.cache_pages = cache->pages;
  a.shift = log2i(cache->page);
  a.total = total;
  a.pages = pages;
  a.stride = pages_stride;
  a.batch = batch;
  a.max_pages = max_pages;
  a.where = where;
  a.used = used;
  a.count = (int32_t*)ws;
  a.from = a.count + 64;
  a.to = a.from + cache->pages;
  a.counts = a.to + cache->pages;
  // one span up to 16,384 pages; else spans of 4096, at most 1024 of them
  a.words = (int)cdiv(cache->pages, 64 * kWaves);
  if (a.words > 16) {
    const int least = (int)cdiv(a.words, 1024);
    a.words = least > 4 ? least : 4;
  }
  a.spans = (int)cdiv(cache->pages, 64 * kWaves * a.words);
  CopyArgs c{};
  set_copy(cache, cache, &c);
  c.from = a.from;
  c.to = a.to;
  c.count = a.count;
  const auto move = [&](auto kernel, int threads, int steps) -> int {
    const int64_t spans = cdiv(max_pages, threads);
    const int64_t blocks = copy_blocks(c, cdiv(cache->pages, 2), threads * steps);
    if ((blocks + batch * spans) * threads > kMaxThreads) return GMM_ERR_UNSUPPORTED;
    if (a.spans > 1)
      hipLaunchKernelGGL(k_kv_count, dim3((unsigned)a.spans), dim3(64 * kWaves), 0, stream, ref,
                         cache->pages, a.words, a.counts);
    hipLaunchKernelGGL(k_kv_places, dim3((unsigned)a.spans), dim3(64 * kWaves), 0, stream, a);
    hipLaunchKernelGGL(kernel, dim3((unsigned)(blocks + batch * spans)), dim3(threads), 0, stream, c, a,
                       (int)blocks, (int)spans);
    return launch_status();
  };
  if (c.bytes > kSmallPage) return move(k_kv_move<1024, 4>, 1024, 4);
  return move(k_kv_move<256, 2>, 256, 2);
}

}  // extern "C"
