// Pages of the key/value cache as a pool, for AMD Instinct MI355X (gfx950): copying, forking,
// growing and compacting.
//
// ref[p] counts the table entries that name page p, over all tables; 0 is a free page.  Every
// decision is taken on the GPU from the counts and tables, in an order that the sizes fix: the
// only atomics are sums and minima of whole numbers, whose result does not depend on theirs.
//
// The free (or used) pages are found by one workgroup: 64 pages make a word by one ballot, a
// lane keeps a word, and a page's rank among the free ones is a sum over words plus a bit count.

#include <hip/hip_runtime.h>

#include <limits.h>
#include <stdint.h>

#include "flashgmm.h"
#include "kv_host.h"
#include "kv_plan.h"

namespace {

using namespace kv;

constexpr int kWaves = 16;                        // of the workgroup that ranks pages
constexpr int kSpan = kWaves * 64 * 64;           // pages it ranks at a time
constexpr int kPart = 16384;                      // bytes of a copy's work item

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
  int parts;                  // work items of a page's keys
  const int32_t* from;
  const int32_t* to;
  const int32_t* count;       // pairs, or null: n
  int n;
};

__device__ __forceinline__ void copy_part(const char* from, char* to, int n) {
  const uint4* f = reinterpret_cast<const uint4*>(from);
  uint4* t = reinterpret_cast<uint4*>(to);
  if (n == kPart / 16) {
    uint4 v[kPart / 4096];
#pragma unroll
    for (int i = 0; i < kPart / 4096; ++i) v[i] = f[threadIdx.x + i * 256];
#pragma unroll
    for (int i = 0; i < kPart / 4096; ++i) t[threadIdx.x + i * 256] = v[i];
  } else {
    for (int i = threadIdx.x; i < n; i += 256) t[i] = f[i];
  }
}

// Work items 2 parts a pair: kPart bytes of the keys or of the values; the first also the box.
__device__ __forceinline__ void copy_items(const CopyArgs& a, int block, int blocks) {
  // a workgroup's items: `blocks` apart, counted in pairs and parts, without a division each
  const int n = a.count ? *a.count : a.n, per = 2 * a.parts;
  const int step_pair = blocks / per, step_part = blocks - step_pair * per;
  int pair = block / per, next = block - pair * per;
  while (pair < n) {
    const int at_pair = pair;
    int part = next;
    pair += step_pair;
    next += step_part;
    if (next >= per) {
      next -= per;
      ++pair;
    }
    const int from = a.from[at_pair], to = a.to[at_pair];
    if (from < 0 || from >= a.src.pages || to < 0 || to >= a.dst.pages) continue;
    if (part == 0 && a.dst.box) {
      const uint4* f = reinterpret_cast<const uint4*>(a.src.box + (int64_t)from * a.box_bytes);
      uint4* t = reinterpret_cast<uint4*>(a.dst.box + (int64_t)to * a.box_bytes);
      for (int i = threadIdx.x; i < a.box_bytes / 16; i += 256) t[i] = f[i];
      for (int i = threadIdx.x; i < a.heads; i += 256)
        a.dst.scale[(int64_t)to * a.heads + i] = a.src.scale[(int64_t)from * a.heads + i];
    }
    const bool values = part >= a.parts;
    if (values) part -= a.parts;
    const int at = part * kPart;
    copy_part((values ? a.src.v : a.src.k) + (int64_t)from * a.bytes + at,
              (values ? a.dst.v : a.dst.k) + (int64_t)to * a.bytes + at,
              min(a.bytes - at, kPart) / 16);
  }
}

__global__ __launch_bounds__(256) void k_kv_copy(CopyArgs a) {
  copy_items(a, blockIdx.x, gridDim.x);
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
  bool hit = false;
  for (int i = threadIdx.x; i < n; i += 256) hit |= a.parent[i] == p;
  return __syncthreads_or(hit);
}

// Workgroups of a new row copy its parent's entries, those of an old row without a child give up
// its pages.  An old row's counts pass to its first child, so that rows that go on alone change
// none.
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
__device__ __forceinline__ uint64_t load_words(const int32_t* ref, int pages, int first, int words) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int base = first + w * words * 64 + lane;
  uint64_t mine = 0;
  for (int i = 0; i < words; i += 8) {
    int v[8];                        // eight loads in flight
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = ref[min(base + (i + j) * 64, pages - 1)];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint64_t bits = __ballot(i + j < words && base + (i + j) * 64 < pages && v[j] > 0);
      if (lane == i + j) mine = bits;
    }
  }
  return mine;
}
__device__ __forceinline__ int words_of(int pages) {
  return pages >= kSpan ? 64 : (pages + 64 * kWaves - 1) / (64 * kWaves);
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
  int32_t* base;              // [batch + 1] pages needed by the rows before
  int32_t* cow;               // [batch] the shared page that the row writes into, or -1
  int32_t* first;             // [cache pages] first row that writes into a shared page
  int32_t* writers;           // [cache pages] rows that do
  int32_t* free_list;         // [cache pages]
};

__device__ __forceinline__ int load_agent(const int32_t* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ void store_agent(int32_t* p, int v) {
  __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
// what a thread of the workgroup wrote to memory is seen by all after it
__device__ __forceinline__ void memory_barrier() {
  __threadfence();
  __syncthreads();
}

// The shared page that row r writes into, or -1.
__device__ __forceinline__ int shared_page(const GrowArgs& a, int r) {
  const int held = a.held[r], total = a.total[r];
  if (held <= 0 || total <= held || (held & ((1 << a.shift) - 1)) == 0) return -1;
  const int e = held >> a.shift;
  if (e >= a.max_pages) return -1;
  const int p = a.pages[r * a.stride + e];
  return p >= 0 && p < a.cache_pages && a.ref[p] > 1 ? p : -1;
}

__global__ __launch_bounds__(64 * kWaves) void k_kv_grow(GrowArgs a) {
  __shared__ int tmp[kWaves];
  __shared__ int64_t tmp64[kWaves];
  __shared__ int copies;
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  if (tid == 0) copies = 0;
  // rows that write into one page: their number and the first of them
  for (int r = tid; r < a.batch; r += 64 * kWaves) {
    const int p = shared_page(a, r);
    a.cow[r] = p;
    if (p >= 0) {
      store_agent(a.first + p, INT_MAX);
      store_agent(a.writers + p, 0);
    }
  }
  memory_barrier();
  for (int r = tid; r < a.batch; r += 64 * kWaves) {
    const int p = a.cow[r];
    if (p >= 0) {
      atomicMin(a.first + p, r);
      atomicAdd(a.writers + p, 1);
    }
  }
  memory_barrier();
  // pages that every row needs; the first writer keeps the page if no other row holds it
  int64_t want = 0;
  for (int r0 = 0; r0 < a.batch; r0 += 64 * kWaves) {
    const int r = r0 + tid;
    int64_t need = 0;               // up to 2^25 a row
    if (r < a.batch) {
      need = max(0, min(pages_of(a.total[r], a.shift), a.max_pages) - pages_of(a.held[r], a.shift));
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
  if (tid == 0) a.base[a.batch] = (int)min(want, (int64_t)INT_MAX);
  // the first `want` free pages
  int64_t have = 0;
  for (int first = 0; first < a.cache_pages && have < want; first += kSpan) {
    const int words = words_of(a.cache_pages - first);
    const int p0 = first + (w * words + lane) * 64;        // pages of the lane's word
    uint64_t bits = 0;
    if (lane < words && p0 < a.cache_pages)
      bits = a.cache_pages - p0 >= 64 ? ~0ull : (1ull << (a.cache_pages - p0)) - 1;
    bits &= ~load_words(a.ref, a.cache_pages, first, words);
    int all;
    int rank = group_sum((int)__popcll(bits), tmp, &all);
    for (int i = 0; i < words; ++i) {
      const uint64_t b = __shfl(bits, i);
      const int64_t at = have + __shfl(rank, i);
      if (at >= want) break;
      const int64_t k = at + __popcll(b & ((1ull << lane) - 1));
      if ((b >> lane & 1) && k < want) a.free_list[k] = first + (w * words + i) * 64 + lane;
    }
    have += all;
  }
  if (tid == 0) a.short_by[0] = have < want ? (int)min(want - have, (int64_t)INT_MAX) : 0;
  memory_barrier();
  if (have >= want) {
    for (int k = tid; k < want; k += 64 * kWaves) {
      int lo = 0, hi = a.batch;        // the last row with base <= k
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (a.base[mid] <= k) lo = mid;
        else hi = mid;
      }
      const int page = a.free_list[k];
      int i = k - a.base[lo];
      const int held = a.held[lo], old = a.cow[lo];
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
  int32_t* count;             // pages moved
  int32_t* from;              // [cache pages / 2]
  int32_t* to;
};

// With U used pages, those at U and above go to the free ones below, in order.
__global__ __launch_bounds__(64 * kWaves) void k_kv_compact(CompactArgs a) {
  __shared__ int tmp[kWaves];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  int used = 0;
  for (int first = 0; first < a.cache_pages; first += kSpan) {
    int all;
    group_sum((int)__popcll(load_words(a.ref, a.cache_pages, first,
                                       words_of(a.cache_pages - first))),
              tmp, &all);
    used += all;
  }
  int below = 0, moves = 0;            // used pages before; pages moved
  bool passed = false;                 // is `used` behind: moves is known then
  for (int first = 0; first < a.cache_pages; first += kSpan) {
    const int words = words_of(a.cache_pages - first);
    const uint64_t bits = load_words(a.ref, a.cache_pages, first, words);
    int all;
    const int rank = below + group_sum((int)__popcll(bits), tmp, &all);
    if (!passed && used <= first + kSpan) {
      // free pages below `used`: those before the word that holds it, and in it
      __shared__ int holes;
      const int p0 = first + (w * words + lane) * 64;
      if (tid == 0) holes = used - (below + all);       // `used` at or behind the last word
      __syncthreads();
      if (lane < words && p0 <= used && used < p0 + 64)
        holes = used - (rank + __popcll(bits & ((1ull << (used - p0)) - 1)));
      __syncthreads();
      moves = holes;
      passed = true;
    }
    for (int i = 0; i < words; ++i) {
      const uint64_t b = __shfl(bits, i);
      const int before = __shfl(rank, i) + __popcll(b & ((1ull << lane) - 1));
      const int p = first + (w * words + i) * 64 + lane;
      if (p >= a.cache_pages) continue;
      const bool in = b >> lane & 1;
      a.where[p] = in ? p : -1;
      if (p < used && !in) a.to[p - before] = p;
      if (p >= used && in) a.from[before - (used - moves)] = p;
    }
    below += all;
  }
  memory_barrier();
  for (int i = tid; i < moves; i += 64 * kWaves) {
    const int from = a.from[i], to = a.to[i];
    a.where[from] = to;
    a.ref[to] = a.ref[from];
    a.ref[from] = 0;
  }
  if (tid == 0) {
    a.used[0] = used;
    a.count[0] = moves;
  }
}

// The first `blocks` workgroups copy, the others rewrite the tables: a row, 1024 entries each.
__global__ __launch_bounds__(256) void k_kv_move(CopyArgs c, CompactArgs a, int blocks,
                                                 int spans) {
  if ((int)blockIdx.x < blocks) {
    copy_items(c, blockIdx.x, blocks);
    return;
  }
  const int item = (int)blockIdx.x - blocks, row = item / spans;
  const int e0 = (item - row * spans) * 1024;
  const int n = min(pages_of(a.total[row], a.shift), a.max_pages);
  for (int e = e0 + threadIdx.x; e < min(n, e0 + 1024); e += 256) {
    const int p = a.pages[(int64_t)row * a.stride + e];
    if (p < 0 || p >= a.cache_pages) continue;
    const int to = a.where[p];
    if (to >= 0 && to != p) a.pages[(int64_t)row * a.stride + e] = to;
  }
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
  a->parts = (int)cdiv(a->bytes, kPart);
}

int64_t copy_blocks(const CopyArgs& a, int64_t pairs) {
  const int64_t items = pairs * 2 * a.parts, most = 16 * kCUs;
  return items < most ? items : most;
}

int64_t pool_need(const gmm_kv_cache* c, int32_t batch) {
  return cdiv(256 + 4 * (3 * (int64_t)c->pages + 4 * (int64_t)batch + 64), 256) * 256;
}

int check_tables(const gmm_kv_cache* c, int32_t batch, int32_t max_pages, int64_t stride) {
  if (batch < 1 || max_pages < 1 || stride < max_pages) return GMM_ERR_INVALID_ARG;
  if ((int64_t)max_pages * c->page > (1 << 30) || batch > GMM_KV_MAX_ROWS || c->pages > (1 << 30))
    return GMM_ERR_UNSUPPORTED;
  return GMM_OK;
}

// do [a, a + na) and [b, b + nb) share a byte?
bool overlap(const void* a, int64_t na, const void* b, int64_t nb) {
  const char *p = (const char*)a, *q = (const char*)b;
  return p < q + nb && q < p + na;
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
  hipLaunchKernelGGL(k_kv_copy, dim3((unsigned)copy_blocks(a, n)), dim3(256), 0, stream, a);
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
    // the old tables are read while the new ones are written
    if (overlap(pages, table_bytes(batch, pages_stride, max_pages), pages_out,
                table_bytes(rows, out_stride, out_max_pages)) ||
        overlap(total, 4 * (int64_t)batch, total_out, 4 * (int64_t)rows))
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
  a.cow = a.base + batch + 1;
  a.first = a.cow + batch;
  a.writers = a.first + cache->pages;
  a.free_list = a.writers + cache->pages;
  hipLaunchKernelGGL(k_kv_grow, dim3(1), dim3(64 * kWaves), 0, stream, a);
  CopyArgs c{};
  set_copy(cache, cache, &c);
  c.from = a.from;
  c.to = a.to;
  c.count = a.count;
  hipLaunchKernelGGL(k_kv_copy, dim3((unsigned)copy_blocks(c, batch)), dim3(256), 0, stream, c);
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
  hipLaunchKernelGGL(k_kv_compact, dim3(1), dim3(64 * kWaves), 0, stream, a);
  CopyArgs c{};
  set_copy(cache, cache, &c);
  c.from = a.from;
  c.to = a.to;
  c.count = a.count;
  const int spans = (int)cdiv(max_pages, 1024);
  const int64_t blocks = copy_blocks(c, cdiv(cache->pages, 2));
  if (blocks + (int64_t)batch * spans > kMaxBlocks) return GMM_ERR_UNSUPPORTED;
  hipLaunchKernelGGL(k_kv_move, dim3((unsigned)(blocks + (int64_t)batch * spans)), dim3(256), 0,
                     stream, c, a, (int)blocks, spans);
  return launch_status();
}

}  // extern "C"
