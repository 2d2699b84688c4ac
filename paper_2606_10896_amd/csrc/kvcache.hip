// Paged key/value cache for AMD Instinct MI355X (gfx950): rotary positions, appending,
// selection of pages by a cheap score, attention of new tokens over the cache.
//
// Attention is the E-step's pattern with other operands: a row's softmax weights are
// responsibilities of equal isotropic components at the keys, formed with a running maximum
// and sum (base 2) and contracted with the values in the same pass; the rows x keys matrix is
// never stored.
//
// Cache layout.  A page holds its keys as rows [page, d] and its values transposed, [d, page].
// Both products then take their cache operand in the register order of the matrix
// instructions straight from memory, 16 bytes a lane, with nothing exchanged between lanes:
//   S^T = K Q^T      A rows = keys: lane l holds 8 consecutive dimensions of key l % 16
//   O^T = V^T P^T    A rows = dimensions: lane l holds 8 consecutive keys of dimension l % 16
// The accumulator of the first product (lane: one query row, 4 keys) is the B operand of the
// second (lane: one query row, 8 keys) when the keys of two 16-key tiles are interleaved in
// groups of 4: row r of tile t is key 8 (r / 4) + 4 t + r % 4 of the 32.
//
// Results are bitwise reproducible: key ranges are fixed by the sizes, their partial results
// are joined in order.  The only atomics are integer counts in LDS.

#include <hip/hip_runtime.h>

#include <float.h>
#include <math.h>
#include <stdint.h>

#include <type_traits>

#include "flashgmm.h"
#include "kv_host.h"
#include "kv_plan.h"

namespace {

using namespace kv;

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
// 1/127 rounded to fp32
constexpr float kInv127 = 1.0f / 127.0f;

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

template <typename T> struct Vec8;
template <> struct Vec8<__bf16> { typedef bf16x8 type; };
template <> struct Vec8<_Float16> { typedef f16x8 type; };

// 16x16x32: lane l holds A[l % 16][8 (l / 16) + e] and B[8 (l / 16) + e][l % 16], e = 0..7,
// and D[4 (l / 16) + i][l % 16], i = 0..3
__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mfma16(f16x8 a, f16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

// 32x32x16: lane l holds A[l % 32][8 (l / 32) + e] and B[8 (l / 32) + e][l % 32], e = 0..7, and
// D[8 (i / 4) + 4 (l / 32) + i % 4][l % 32], i = 0..15
__device__ __forceinline__ f32x16 mfma32(bf16x8 a, bf16x8 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mfma32(f16x8 a, f16x8 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}

__device__ __forceinline__ float exp2_fast(float v) { return __builtin_amdgcn_exp2f(v); }
__device__ __forceinline__ float log2_fast(float v) { return __builtin_amdgcn_logf(v); }

template <typename V>
__device__ __forceinline__ V load16(const void* p) {
  static_assert(sizeof(V) == 16, "16 bytes");
  const uint4 u = *reinterpret_cast<const uint4*>(p);
  return __builtin_bit_cast(V, u);
}

// 8 elements each at at(0) .. at(N - 1) of a caller's rows; vec: these allow 16-byte loads.  The
// loads are issued before any is waited for.
template <typename T, int N, typename At>
__device__ __forceinline__ void load_rows8(typename Vec8<T>::type* v, At at, int vec) {
  if (vec) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = load16<typename Vec8<T>::type>(at(i));
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const T* p = at(i);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[i][e] = p[e];
    }
  }
}

// Barrier for what goes through LDS: unlike __syncthreads it does not wait for global stores.
__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// ---------------------------------------------------------------- sequences
// The tables are read in the constant address space: nothing writes them while a kernel runs,
// and loads at wave-uniform addresses go through the scalar cache.
typedef const __attribute__((address_space(4))) int32_t* Table;

struct Seqs {
  Table cu;
  Table total;
  Table pages;
  int64_t stride;
  int batch, max_pages;
  int page_shift;   // log2 of the page size
  int cache_pages;
};

// Work items are numbered over all sequences without a table made beforehand: sequence b's
// items start at first(b) = floor(cu[b] mul / div) + slack b, which leaves room for
// ceil(n mul / div) items (slack 1), or one more (slack 2), for its n tokens; with slack 2 at
// min(first(b), cu[b]), as a token makes at most one item.  The sequence of an item is the last b
// with first(b) <= item: a search by the whole wave, 64 sequences a step.
__device__ __forceinline__ int64_t first_of(int64_t row0, int b, int mul, int div, int slack) {
  const int64_t f = row0 * mul / div + (int64_t)slack * b;
  return slack == 2 ? min(f, row0) : f;
}
__device__ __forceinline__ int64_t first_item(const Seqs& s, int b, int mul, int div, int slack) {
  return first_of(s.cu[b], b, mul, div, slack);
}
struct Seq {
  int b, row0, n, total;     // index, first row, new tokens, keys with them
};
__device__ __forceinline__ Seq find_seq(const Seqs& s, int64_t item, int mul, int div, int slack) {
  int lo = 0, hi = s.batch;            // the answer is in [lo, hi)
  const int lane = threadIdx.x & 63;
  while (hi - lo > 64) {
    const int step = (hi - lo + 63) / 64;
    const int b = lo + lane * step;
    const bool in = b < hi && first_item(s, b, mul, div, slack) <= item;
    const int cnt = __popcll(__ballot(in));    // first() grows with b: a prefix of the lanes
    lo += (cnt > 0 ? cnt - 1 : 0) * step;
    hi = min(hi, lo + step);
  }
  Seq q;
  if (hi - lo == 1) {
    q.b = __builtin_amdgcn_readfirstlane(lo);
    q.row0 = s.cu[q.b];
    q.n = s.cu[q.b + 1] - q.row0;
    q.total = s.total[q.b];
  } else {                             // a sequence a lane: its numbers come along
    const int b = min(lo + lane, hi - 1);
    const int row0 = s.cu[b], next = s.cu[b + 1], total = s.total[b];
    const bool in = lo + lane < hi && first_of(row0, b, mul, div, slack) <= item;
    const int i = max(__popcll(__ballot(in)) - 1, 0);
    q.b = __builtin_amdgcn_readfirstlane(lo) + i;
    q.row0 = __builtin_amdgcn_readlane(row0, i);
    q.n = __builtin_amdgcn_readlane(next, i) - q.row0;
    q.total = __builtin_amdgcn_readlane(total, i);
  }
  return q;
}

// physical page of a sequence's logical page, -1 if there is none
__device__ __forceinline__ int phys_page(const Seqs& s, int b, int lp) {
  if (lp < 0 || lp >= s.max_pages) return -1;
  const int p = s.pages[(int64_t)b * s.stride + lp];
  return (unsigned)p < (unsigned)s.cache_pages ? p : -1;
}

// ---------------------------------------------------------------- rotation
// A head's row is handled in units of 2 W elements: pair units (W pairs each), then units of
// the dimensions past rot.  A unit is two runs of W elements, at o0 and o1.
struct RopeShape {
  const float* table;
  int positions, rot, inverse;
};

template <int W>
struct Unit {
  int o0, o1;
  int pair;       // first pair, -1 for a unit past rot
  __device__ __forceinline__ Unit(int u, int rot, bool inter) {
    const int h = rot >> 1, hu = h / W;
    if (u < hu && !inter) {
      o0 = u * W;
      o1 = h + u * W;
    } else {
      o0 = u * 2 * W;                 // hu pair units cover 2 W hu = rot dimensions
      o1 = o0 + W;
    }
    pair = u < hu ? u * W : -1;
  }
};

// a unit's elements, as one vector: an array that two branches fill would be kept in memory
template <typename T, int W>
using UnitV = T __attribute__((ext_vector_type(2 * W)));

// W elements at p into / from the elements `at` .. at + W - 1 of v
template <typename T, int W, typename V>
__device__ __forceinline__ void load_run(const T* p, V& v, int at) {
  if constexpr (W == 1) {
    v[at] = p[0];
  } else {
    constexpr int E = 16 / sizeof(T);
    typedef T Run __attribute__((ext_vector_type(E)));
#pragma unroll
    for (int i = 0; i < W / E; ++i) {
      const Run r = load16<Run>(p + i * E);
#pragma unroll
      for (int e = 0; e < E; ++e) v[at + i * E + e] = r[e];
    }
  }
}
template <typename T, int W, typename V>
__device__ __forceinline__ void store_run(T* p, const V& v, int at) {
  if constexpr (W == 1) {
    p[0] = v[at];
  } else {
    constexpr int E = 16 / sizeof(T);
    typedef T Run __attribute__((ext_vector_type(E)));
#pragma unroll
    for (int i = 0; i < W / E; ++i) {
      Run r;
#pragma unroll
      for (int e = 0; e < E; ++e) r[e] = v[at + i * E + e];
      *reinterpret_cast<uint4*>(p + i * E) = __builtin_bit_cast(uint4, r);
    }
  }
}

// v: the unit's 2 W elements, in place.  Products and sums are rounded one by one, as the
// formula is written, so that the result does not depend on where a compiler contracts.  The
// layout is a template argument: with a run-time one the compiler joins both branches into
// one with run-time indexes into v.
template <typename T, int W, bool INTER>
__device__ __forceinline__ void rotate_unit(UnitV<T, W>& v, int pair, int pos, const RopeShape& r) {
#pragma clang fp contract(off)
  if (pair < 0 || pos < 0) return;
  UnitV<float, W> cs = UnitV<float, W>(__builtin_nanf(""));      // cosines, then sines
  if (pos < r.positions) {
    const float* row = r.table + (int64_t)pos * r.rot + pair;
    load_run<float, W>(row, cs, 0);
    load_run<float, W>(row + (r.rot >> 1), cs, W);
  }
#pragma unroll
  for (int i = 0; i < W; ++i) {
    const int ia = INTER ? 2 * i : i, ib = INTER ? 2 * i + 1 : i + W;
    const float a = (float)v[ia], b = (float)v[ib], c = cs[i];
    const float sn = r.inverse ? -cs[W + i] : cs[W + i];
    v[ia] = (T)(a * c - b * sn);
    v[ib] = (T)(b * c + a * sn);
  }
}

template <typename T, int W, bool INTER>
__device__ __forceinline__ void rope_unit(const T* x, T* out, int u, int pos, const RopeShape& r) {
  const Unit<W> un(u, r.rot, INTER);
  UnitV<T, W> v;
  load_run<T, W>(x + un.o0, v, 0);
  load_run<T, W>(x + un.o1, v, W);
  rotate_unit<T, W, INTER>(v, un.pair, pos, r);
  store_run<T, W>(out + un.o0, v, 0);
  store_run<T, W>(out + un.o1, v, W);
}

__global__ __launch_bounds__(256) void k_rope_table(const double* __restrict__ freq, int half,
                                                    double scale, int64_t positions,
                                                    float* __restrict__ table) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= positions * half) return;
  const int64_t p = i / half;
  const int j = (int)(i - p * half);
  double s, c;
  sincos((double)p * freq[j], &s, &c);
  table[p * 2 * half + j] = (float)(scale * c);
  table[p * 2 * half + half + j] = (float)(scale * s);
}

// A unit a thread: 16 elements (W = 8: 16-byte accesses) where rot, d, the strides and the
// addresses allow it, else one pair.  An odd count of dimensions past rot ends in a unit of its
// own (W = 1).  Bound by the bytes: 8192 x 32 x 128 bf16, half rotated, 28.5 us a call, 4.8 TB/s
// (a 2 GiB copy: 5.0); a single token's 40 heads take 2 us.
template <typename T, int W, bool INTER>
__global__ __launch_bounds__(256) void k_rope(const T* x, int64_t xt, int64_t xh, T* out,
                                              int64_t ot, int64_t oh, uint32_t items, int heads,
                                              int d, const int32_t* __restrict__ pos,
                                              RopeShape r) {
  const uint32_t i = blockIdx.x * 256 + threadIdx.x;
  if (i >= items) return;
  const uint32_t units = (d + 2 * W - 1) / (2 * W);
  const uint32_t row = i / units, t = row / heads;
  const int u = i - row * units, h = row - t * heads;
  const T* xr = x + t * xt + (int64_t)h * xh;
  T* orow = out + t * ot + (int64_t)h * oh;
  if (W == 1 && 2 * u + 1 >= d && u >= (r.rot >> 1)) {
    orow[d - 1] = xr[d - 1];
    return;
  }
  rope_unit<T, W, INTER>(xr, orow, u, pos[t], r);
}

// ---------------------------------------------------------------- append
struct AppendArgs {
  Seqs s;
  void* ck;
  void* cv;
  int8_t* box;
  float* box_scale;
  int heads, page, d;
  const void* k;
  int64_t kt, kh;
  const void* v;
  int64_t vt, vh;
  int v_vec;                 // value rows can be read 16 bytes at a time
  const int32_t* pos;
  RopeShape rope;            // table null: no rotation
  const void* q;
  int64_t qt, qh;
  void* qo;
  int64_t qot, qoh;
  int hq;
  int per;                   // heads a workgroup takes: 1, 2 or 4
  int64_t page_blocks;       // workgroups of pages; the rest rotate queries
  uint32_t q_items;          // units of all queries
};

// One workgroup a (page touched, `per` heads): the page's new keys are rotated and stored, its
// new values stored transposed, and its box formed from all its keys, the older ones read back
// (a page of 64 keys of 128 dimensions is 16 KB, so a single new token moves 8 KB on average
// for a box that saves reading that page in every later step in which it is not selected).
// Small pages share a workgroup, 128 or 64 threads a head.  The queries' rotation rides along in
// workgroups of its own: one launch for the step.  Bound by the bytes for prompts (7498 tokens, 16
// heads of 64: 28 us, about 130 MB), for single tokens by the chain sequence, page, keys, barrier
// (64 sequences, 8 heads of 128: 9.4 us).
template <typename T, int W, bool INTER>
__global__ __launch_bounds__(256) void k_kv_append(AppendArgs a) {
  typedef typename Vec8<T>::type V8;
  if ((int64_t)blockIdx.x >= a.page_blocks) {
    const uint32_t first = (uint32_t)(blockIdx.x - a.page_blocks) * 256;
    const uint32_t i = first + threadIdx.x;
    const uint32_t units = a.d / (2 * W), row_units = units * a.hq;
    if (first >= a.q_items) return;
    const uint32_t t = min(i, a.q_items - 1) / row_units;
    int p;
    if (a.pos) {
      p = a.pos[t];
    } else {
      // the sequence of the wave's first row, then of this thread's
      int b = find_seq(a.s, __builtin_amdgcn_readfirstlane(t), 1, 1, 0).b;
      while (b + 1 < a.s.batch && a.s.cu[b + 1] <= (int)t) ++b;
      p = a.s.total[b] - (a.s.cu[b + 1] - (int)t);
    }
    if (i >= a.q_items) return;
    const int h = (i - t * row_units) / units, u = i % units;
    rope_unit<T, W, INTER>((const T*)a.q + t * a.qt + (int64_t)h * a.qh,
                           (T*)a.qo + t * a.qot + (int64_t)h * a.qoh, u, p, a.rope);
    return;
  }
  constexpr int kBatch = W == 1 ? 8 : 2;             // rows in flight a thread
  __shared__ T red[256 * 2 * W * 2];
  __shared__ float wmax[4];
  __shared__ int wbad[4];
  const int threads = 256 / a.per;                   // of a head: whole waves
  const int hsub = threadIdx.x / threads, tid = threadIdx.x - hsub * threads;
  const int head_blocks = (a.heads + a.per - 1) / a.per;
  const int head = (int)(blockIdx.x % head_blocks) * a.per + hsub;
  const bool live = head < a.heads;
  const int64_t item = blockIdx.x / head_blocks;
  const int P = a.page, d = a.d;
  const Seq sq = find_seq(a.s, item, 1, P, 2);
  const int b = sq.b, row0 = sq.row0, n = sq.n, total = sq.total;
  if (n <= 0) return;
  const int64_t s0l = (int64_t)total - n;
  const int s0 = s0l < 0 ? 0 : (int)s0l;                 // first new slot that exists
  const int64_t lp64 = (s0 >> a.s.page_shift) + (item - first_of(row0, b, 1, P, 2));
  if ((lp64 << a.s.page_shift) >= total) return;
  const int lp = (int)lp64;
  const int phys = phys_page(a.s, b, lp);
  if (phys < 0) return;
  const int first = lp << a.s.page_shift;                // first slot of the page
  const int filled = min(P, total - first);
  const int begin = max(0, s0 - first);                  // new keys: begin .. filled - 1
  const int64_t ph = (int64_t)phys * a.heads + (live ? head : 0);
  const int64_t in0 = row0 + ((int64_t)first - s0l);     // input row of the page's slot 0

  // keys
  T* ckp = (T*)a.ck + ph * P * d;
  const T* kin = (const T*)a.k + (int64_t)(live ? head : 0) * a.kh;
  const int units = d / (2 * W), groups = threads / units;
  const int u = tid % units, g = tid / units;
  const Unit<W> un(u, a.rope.rot, INTER);
  UnitV<float, W> hi = -INFINITY, lo = INFINITY;
  bool bad = false;
  const int from = a.box ? 0 : begin;
  if (live && g < groups) {
    for (int sb = from + g; sb < filled; sb += kBatch * groups) {
      UnitV<T, W> v[kBatch];
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        const int s = min(sb + j * groups, filled - 1);
        const T* kr = s < begin ? ckp + (int64_t)s * d : kin + (in0 + s) * a.kt;
        load_run<T, W>(kr + un.o0, v[j], 0);
        load_run<T, W>(kr + un.o1, v[j], W);
      }
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        const int s = sb + j * groups;
        if (s >= filled) break;
        if (s >= begin) {
          if (a.rope.table)
            rotate_unit<T, W, INTER>(v[j], un.pair, a.pos ? a.pos[in0 + s] : first + s, a.rope);
          store_run<T, W>(ckp + (int64_t)s * d + un.o0, v[j], 0);
          store_run<T, W>(ckp + (int64_t)s * d + un.o1, v[j], W);
        }
#pragma unroll
        for (int e = 0; e < 2 * W; ++e) {
          const float f = (float)v[j][e];
          bad |= !(fabsf(f) <= FLT_MAX);
          hi[e] = fmaxf(hi[e], f);
          lo[e] = fminf(lo[e], f);
        }
      }
    }
  }

  // values: 8 slots x 8 dimensions a thread, slots fastest over the lanes, so that a dimension's
  // run of slots is written in whole lines
  {
    T* cvp = (T*)a.cv + ph * d * P;
    const T* vin = (const T*)a.v + (int64_t)(live ? head : 0) * a.vh;
    const int g0 = begin >> 3, ng = ((filled + 7) >> 3) - g0, blocks = live ? ng * (d >> 3) : 0;
    for (int i = tid; i < blocks; i += threads) {
      const int c = i / ng, sg = (g0 + i - c * ng) << 3;
      const bool whole = sg >= begin && sg + 8 <= filled;
      V8 blk[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        blk[j] = V8((T)0.0f);
        if (sg + j >= begin && sg + j < filled)
          load_rows8<T, 1>(&blk[j], [&](int) { return vin + (in0 + sg + j) * a.vt + c * 8; },
                           a.v_vec);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        T* dst = cvp + (int64_t)(c * 8 + e) * P + sg;
        if (whole) {
          V8 col;
#pragma unroll
          for (int j = 0; j < 8; ++j) col[j] = blk[j][e];
          *reinterpret_cast<uint4*>(dst) = __builtin_bit_cast(uint4, col);
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (sg + j >= begin && sg + j < filled) dst[j] = blk[j][e];
        }
      }
    }
  }
  if (!a.box) return;

  // box: the keys are of type T, so their bounds are kept in T without rounding; a row of 2 d
  // entries (upper, then lower bounds) for every group
  T* hred = red + hsub * threads * 4 * W;
  if (live && g < groups) {
#pragma unroll
    for (int e = 0; e < 2 * W; ++e) {
      const int dim = (e < W ? un.o0 : un.o1 - W) + e;
      hred[g * 2 * d + dim] = (T)hi[e];
      hred[g * 2 * d + d + dim] = (T)lo[e];
    }
  }
  // this head's waves agree on its largest magnitude; up to 512 / 64 bounds a thread
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint64_t any = __ballot(bad);
  if (lane == 0) wbad[wave] = any != 0;
  lds_barrier();
  const int rounds = (2 * d + threads - 1) / threads;
  float m = 0.0f;
  for (int r = 0; r < rounds; ++r) {
    const int t = tid + r * threads;
    if (!live || t >= 2 * d) continue;
    const float sign = t < d ? 1.0f : -1.0f;
    float x = -INFINITY;
    for (int j = 0; j < groups; ++j) x = fmaxf(x, sign * (float)hred[j * 2 * d + t]);
    m = fmaxf(m, fabsf(x));
    hred[t] = (T)(sign * x);             // row 0 becomes the page's (its entry is read)
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
  if (lane == 0) wmax[wave] = m;
  lds_barrier();
  const int w0 = hsub * (threads >> 6);
  int any_bad = 0;
  for (int w = w0; w < w0 + (threads >> 6); ++w) {
    m = fmaxf(m, wmax[w]);
    any_bad |= wbad[w];
  }
  if (!live) return;
  const float unit = any_bad ? INFINITY : m * kInv127;
  for (int t = tid; t < 2 * d; t += threads) {
    const float x = (float)hred[t];
    float q = 0.0f;
    if (!any_bad && unit > 0.0f)
      q = t < d ? ceilf(__fdiv_rn(x, unit)) : floorf(__fdiv_rn(x, unit));
    a.box[ph * 2 * d + t] = (int8_t)(int)fminf(127.0f, fmaxf(-127.0f, q));
  }
  if (tid == 0) a.box_scale[ph] = unit;
}

// ---------------------------------------------------------------- selection
struct SelectArgs {
  Seqs s;
  const int8_t* box;
  const float* box_scale;
  const void* q;
  int64_t qt, qh;
  int q_vec;
  int heads, group, d;
  int col_shift;             // log2 of the columns a token takes in a 16-column tile
  int col_tiles;             // 16-column tiles a token takes (1 unless group > 16)
  float* score;              // [tokens * heads][row]
  int64_t row;
  int parts;                 // workgroups a row of tiles takes
  int rounds;                // of 256 pages each
};

__device__ __forceinline__ float score_of(float query_unit, float page_unit, int dot) {
#pragma clang fp contract(off)
  return query_unit * page_unit * (float)dot + 0.0f;      // -0 becomes 0
}

// Scores: [pages x 2 d] . [2 d x (token, query head)] in 8-bit integers on 16x16x64 MFMA, the
// boxes (upper | lower bounds) straight from memory in operand order, the queries (positive |
// negative parts) through LDS.  A wave takes 64 pages: their numbers are one load, their boxes
// (8 KB at a time at d = 128) are in flight while the queries are rounded to 8 bits.  S: 64-byte
// steps of a box.  Bound by the boxes' bytes, 2 d + 4 a (page, head), and the loads before them:
// 32 sequences of up to 2049 pages, 8 heads of 128, 19.4 us, 2.5 TB/s; a few sequences of a few
// hundred pages 7.7 us.
template <typename T, int S>
__global__ __launch_bounds__(256, S <= 4 ? 4 : 2) void k_select_score(SelectArgs a) {
  typedef typename Vec8<T>::type V8;
  constexpr int TB = S <= 2 ? 4 : 2;        // 16-page tiles in flight
  extern __shared__ int8_t q8[];            // [col_tiles * 16][2 d + 16], then the units [.]
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int per = 16 >> a.col_shift;        // tokens a tile holds
  // heads fastest: a page's boxes of all heads are neighbours in memory
  const int head = blockIdx.x % a.heads;
  const int part_no = blockIdx.x / a.heads % a.parts;
  const int64_t item = blockIdx.x / a.heads / a.parts;
  const Seq sq = find_seq(a.s, item, 1, per, 1);
  const int b = sq.b, row0 = sq.row0, n = sq.n;
  const int tok0 = (int)(item - first_of(row0, b, 1, per, 1)) * per;
  if (tok0 >= n) return;
  const int toks = min(per, n - tok0);
  const int64_t total = min((int64_t)sq.total, (int64_t)a.s.max_pages << a.s.page_shift);
  const int64_t last = min(total - 1, (int64_t)sq.total - n + tok0 + toks - 1);
  const int visible = last < 0 ? 0 : (int)(last >> a.s.page_shift) + 1;
  if (part_no * a.rounds * 256 >= visible) return;

  // queries: 16 threads a column, runs of 8 dimensions part, part + 16
  const int d = a.d, cols = a.col_tiles * 16, stride = 2 * d + 16;
  float* unit = reinterpret_cast<float*>(q8 + (size_t)cols * stride);
  const int part = tid & 15;
  V8 qv[2];
  const auto head_of = [&](int c) { return (c & ~15) + (c & ((1 << a.col_shift) - 1)); };
  const auto live_col = [&](int c) {
    return ((c & 15) >> a.col_shift) < toks && head_of(c) < a.group;
  };
  const auto load_column = [&](int c) {
    const bool live = live_col(c);
    const T* qr = (const T*)a.q +
                  (int64_t)(row0 + tok0 + (live ? (c & 15) >> a.col_shift : 0)) * a.qt +
                  (int64_t)(head * a.group + (live ? head_of(c) : 0)) * a.qh;
    load_rows8<T, 2>(qv, [&](int j) { return qr + min(8 * (part + 16 * j), d - 8); }, a.q_vec);
#pragma unroll
    for (int j = 0; j < 2; ++j)
      if (!live || 8 * (part + 16 * j) >= d) qv[j] = V8((T)0.0f);
  };
  const auto round_column = [&](int c) {
    float m = 0.0f;
    int bad = 0;
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float f = fabsf((float)qv[j][e]);
        bad |= !(f <= FLT_MAX);
        m = fmaxf(m, f);
      }
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) {
      m = fmaxf(m, __shfl_xor(m, o));
      bad |= __shfl_xor(bad, o);
    }
    const float un = bad ? INFINITY : m * kInv127;
    const bool zero = bad || !(un > 0.0f);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int at = 8 * (part + 16 * j);
      if (at >= d) continue;
      uint64_t up = 0, dn = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float f = zero ? 0.0f : rintf(__fdiv_rn((float)qv[j][e], un));
        up |= (uint64_t)(uint8_t)(int8_t)(int)fmaxf(f, 0.0f) << (8 * e);
        dn |= (uint64_t)(uint8_t)(int8_t)(int)fminf(f, 0.0f) << (8 * e);
      }
      *reinterpret_cast<uint64_t*>(q8 + (size_t)c * stride + at) = up;
      *reinterpret_cast<uint64_t*>(q8 + (size_t)c * stride + d + at) = dn;
    }
    if (part == 0) unit[c] = live_col(c) ? un : -1.0f;       // -1: no query in this column
  };
  load_column(tid >> 4);

  // this wave's pages, one a lane
  const auto page_at = [&](int round) {
    const int p = ((part_no * a.rounds + round) * 4 + wave) * 64 + lane;
    return p < visible ? phys_page(a.s, b, p) : -1;
  };
  int p0 = 0, phys = page_at(0), ahead = -1;        // ahead: the next round's
  float sp = 0.0f;
  const auto take_pages = [&](int round) {
    p0 = ((part_no * a.rounds + round) * 4 + wave) * 64;
    if (round > 0) phys = ahead;
    sp = a.box_scale[(int64_t)max(phys, 0) * a.heads + head];
    ahead = round + 1 < a.rounds ? page_at(round + 1) : -1;
  };
  const int n16 = lane & 15, g = lane >> 4;
  i32x4 bx[TB][S];
  const auto load_boxes = [&](int t0) {
#pragma unroll
    for (int t = 0; t < TB; ++t) {
      const int64_t rec = (int64_t)max(__shfl(phys, 16 * (t0 + t) + n16), 0) * a.heads + head;
#pragma unroll
      for (int st = 0; st < S; ++st)               // past the end: times 0 below
        bx[t][st] = load16<i32x4>(a.box + rec * 2 * d + min(64 * st + 16 * g, 2 * d - 16));
    }
  };
  take_pages(0);
  if (p0 < visible) load_boxes(0);
  for (int c0 = 0; c0 < cols; c0 += 16) {
    if (c0 > 0) load_column(c0 + (tid >> 4));
    round_column(c0 + (tid >> 4));
  }
  __syncthreads();

  for (int round = 0; round < a.rounds; ++round) {
    if (round > 0) take_pages(round);
    if (p0 >= visible) break;
    for (int t0 = 0; t0 < 4; t0 += TB) {
      if (p0 + 16 * t0 >= visible) break;
      if (t0 > 0 || round > 0) load_boxes(t0);
      float best[TB][4];
#pragma unroll
      for (int t = 0; t < TB; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) best[t][i] = -FLT_MAX;
      for (int ct = 0; ct < a.col_tiles; ++ct) {
        const int8_t* qc = q8 + (size_t)(ct * 16 + n16) * stride;
        i32x4 qf[S];
#pragma unroll
        for (int st = 0; st < S; ++st) {
          const int off = 64 * st + 16 * g;
          qf[st] = i32x4{0, 0, 0, 0};
          if (off < 2 * d) qf[st] = *reinterpret_cast<const i32x4*>(qc + off);
        }
        const float un = unit[ct * 16 + n16];
#pragma unroll
        for (int t = 0; t < TB; ++t) {
          i32x4 acc = {0, 0, 0, 0};
#pragma unroll
          for (int st = 0; st < S; ++st)
            acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(bx[t][st], qf[st], acc, 0, 0, 0);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float v = score_of(un, __shfl(sp, 16 * (t0 + t) + 4 * g + i), acc[i]);
            v = v != v ? INFINITY : v;       // a page or query that has no bound comes first
            best[t][i] = un < 0.0f ? best[t][i] : fmaxf(best[t][i], v);
          }
        }
      }
      for (int o = 1; o < (1 << a.col_shift); o <<= 1)
#pragma unroll
        for (int t = 0; t < TB; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) best[t][i] = fmaxf(best[t][i], __shfl_xor(best[t][i], o));
      // entries out of range hold no key: below every score
      const uint64_t none = __ballot(phys < 0);
      if (none != 0) {
#pragma unroll
        for (int t = 0; t < TB; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (none >> (16 * (t0 + t) + 4 * g + i) & 1) best[t][i] = -INFINITY;
      }
      const int tt = n16 >> a.col_shift;
      if ((n16 & ((1 << a.col_shift) - 1)) == 0 && tt < toks) {
        float* out = a.score + ((int64_t)(row0 + tok0 + tt) * a.heads + head) * a.row;
#pragma unroll
        for (int t = 0; t < TB; ++t) {
          const int at = p0 + 16 * (t0 + t) + 4 * g;
          if (at < a.row)
            *reinterpret_cast<float4*>(out + at) =
                make_float4(best[t][0], best[t][1], best[t][2], best[t][3]);
        }
      }
    }
  }
}

// order-preserving integer of a score, above 0
__device__ __forceinline__ uint32_t score_key(float v) {
  const uint32_t u = __float_as_uint(v);
  return u ^ ((u >> 31) ? 0xFFFFFFFFu : 0x80000000u);
}

// The m best pages of a row, one workgroup a row, PT pages a thread in registers (of 64, which
// tables of more than 16,384 pages need, a part is spilled: 1024 threads have 128 each).  The m-th
// largest key is bracketed by counting the keys at or above three values between the bounds
// (ballots, no atomics) until a count is m or the bounds meet; then the pages above it and the
// lowest ones equal to it are written in page order.  Bound by the rounds' latency: about ten,
// a barrier each: 7.6 us at up to 2049 pages, m = 32, 6.4 at a few hundred.
template <int NT, int PT>
__global__ __launch_bounds__(NT) void k_select_top(Seqs s, const float* __restrict__ score,
                                                   int64_t row, int heads, int m, int keep_first,
                                                   int keep_last, int32_t* __restrict__ idx) {
  constexpr int NW = NT / 64;
  __shared__ int cnt[2][NW][3];
  __shared__ uint32_t ext[NW][2];
  __shared__ int scan[NW];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t r = blockIdx.x, t = r / heads;
  const Seq sq = find_seq(s, t, 1, 1, 0);
  const int64_t slot = (int64_t)sq.total - (sq.row0 + sq.n - t);
  const int64_t nv64 = slot < 0 ? 0 : (slot >> s.page_shift) + 1;
  const int nv = (int)min(nv64, (int64_t)s.max_pages);
  int32_t* out = idx + r * m;
  if (nv <= m) {                          // all that hold keys
    int at = 0;
    for (int i0 = 0; i0 < nv; i0 += NT) {
      const int i = i0 + tid;
      const bool in = i < nv && phys_page(s, sq.b, i) >= 0;
      const uint64_t any = __ballot(in);
      int mine = at + __popcll(any & ((1ull << lane) - 1));
      if constexpr (NW == 1) {
        at += __popcll(any);
      } else {
        if (lane == 0) scan[wave] = __popcll(any);
        __syncthreads();
#pragma unroll
        for (int w = 0; w < NW; ++w) {
          if (w < wave) mine += scan[w];
          at += scan[w];
        }
        __syncthreads();
      }
      if (in) out[mine] = i;
    }
    for (int i = at + tid; i < m; i += NT) out[i] = -1;
    return;
  }
  const float* sc = score + r * row;
  const int first = tid * PT;
  uint32_t key[PT];                       // 0: no page; kept pages have the largest one
  uint32_t kmin = 0xFFFFFFFFu, kmax = 0;
#pragma unroll
  for (int i = 0; i < PT; i += 4) {
    float4 v = make_float4(0, 0, 0, 0);
    if (first + i < nv) v = *reinterpret_cast<const float4*>(sc + first + i);
    const float f[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int p = first + i + j;
      const bool keep = p < keep_first || p >= nv - keep_last;
      const bool none = p >= nv || f[j] == -INFINITY;       // past the last, or out of range
      const uint32_t k = score_key(f[j]);
      key[i + j] = none ? 0 : keep ? 0xFFFFFFFFu : k;
      if (!none && !keep) {
        kmin = min(kmin, k);
        kmax = max(kmax, k);
      }
    }
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    kmin = min(kmin, (uint32_t)__shfl_xor((int)kmin, o));
    kmax = max(kmax, (uint32_t)__shfl_xor((int)kmax, o));
  }
  if (lane == 0) {
    ext[wave][0] = kmin;
    ext[wave][1] = kmax;
  }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < NW; ++w) {
    kmin = min(kmin, ext[w][0]);
    kmax = max(kmax, ext[w][1]);
  }
  // counts of keys >= c0, c1, c2 over the workgroup
  int buf = 0;
  const auto count = [&](uint32_t c0, uint32_t c1, uint32_t c2, int* n) {
    n[0] = n[1] = n[2] = 0;
    if constexpr (PT <= 16) {
#pragma unroll
      for (int i = 0; i < PT; ++i) {
        n[0] += __popcll(__ballot(key[i] >= c0));
        n[1] += __popcll(__ballot(key[i] >= c1));
        n[2] += __popcll(__ballot(key[i] >= c2));
      }
    } else {                              // one reduction over the lanes for many keys
#pragma unroll
      for (int i = 0; i < PT; ++i) {
        n[0] += key[i] >= c0;
        n[1] += key[i] >= c1;
        n[2] += key[i] >= c2;
      }
#pragma unroll
      for (int o = 32; o > 0; o >>= 1)
#pragma unroll
        for (int j = 0; j < 3; ++j) n[j] += __shfl_xor(n[j], o);
    }
    if (lane == 0)
#pragma unroll
      for (int j = 0; j < 3; ++j) cnt[buf][wave][j] = n[j];
    __syncthreads();
    n[0] = n[1] = n[2] = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w)
#pragma unroll
      for (int j = 0; j < 3; ++j) n[j] += cnt[buf][w][j];
    buf ^= 1;
  };
  // more than m keys are >= lo, less than m are >= hi (or m or fewer hold keys: all are taken; the
  // kept ones are at most m)
  uint32_t lo = kmin, hi = kmax + 1, above = 0;       // above: take every key > above
  int ties = 0, n[3];
  bool exact = false;
  count(hi, 1, 1, n);
  int n_hi = n[0];
  const int held = n[1];
  if (held <= m) {
    exact = true;
  } else if (n_hi == m) {
    above = hi - 1;
    exact = true;
  }
  while (!exact && hi - lo > 1) {
    const uint32_t q = max((hi - lo) >> 2, 1u);
    const uint32_t c0 = lo + q, c1 = min(lo + 2 * q, hi), c2 = min(lo + 3 * q, hi);
    count(c0, c1, c2, n);
    exact = true;
    if (n[0] == m) above = c0 - 1;
    else if (n[1] == m) above = c1 - 1;
    else if (n[2] == m) above = c2 - 1;
    else exact = false;
    if (n[0] < m) {
      hi = c0;
      n_hi = n[0];
    } else if (n[1] < m) {
      lo = c0;
      hi = c1;
      n_hi = n[1];
    } else if (n[2] < m) {
      lo = c1;
      hi = c2;
      n_hi = n[2];
    } else {
      lo = c2;
    }
  }
  if (!exact) {                           // the m-th key is lo: some of those equal to it go in
    above = lo;
    ties = m - n_hi;
  }
  // ranks in page order: a thread's pages are consecutive
  const auto before = [&](int mine) {
    int incl = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int v = __shfl_up(incl, o);
      if (lane >= o) incl += v;
    }
    __syncthreads();
    if (lane == 63) scan[wave] = incl;
    __syncthreads();
    int base = incl - mine;
    for (int w = 0; w < wave; ++w) base += scan[w];
    return base;
  };
  int eq = 0, left = 0;
  if (ties > 0) {
#pragma unroll
    for (int i = 0; i < PT; ++i) eq += key[i] == above;
    left = ties - before(eq);
  }
  uint32_t take[(PT + 31) / 32] = {};
  int taken = 0;
#pragma unroll
  for (int i = 0; i < PT; ++i) {
    bool in = key[i] > above;
    if (key[i] == above && left > 0 && ties > 0) {
      in = true;
      --left;
    }
    take[i >> 5] |= (uint32_t)in << (i & 31);
    taken += in;
  }
  int at = before(taken);
#pragma unroll
  for (int i = 0; i < PT; ++i)
    if ((take[i >> 5] >> (i & 31) & 1) && at < m) out[at++] = first + i;
  for (int i = held + tid; i < m; i += NT) out[i] = -1;
}

// ---------------------------------------------------------------- attention
// fp16 has no weights below 2^-25 (half its smallest number), and a million of them may weigh as
// much as the largest one.  Weights of fp16 caches are formed 2^15 times as large by
// k_attend_few, where they are at most 1 otherwise (2^-40 of the largest still counts), and 2^7
// times by k_attend_tile, where a step's may add up to 2^8 (2^-32).  The sums carry the same factor,
// and a row's maximum is given lower by its logarithm, so the joins need not know of it.
template <typename T> constexpr float kFewShift = std::is_same<T, _Float16>::value ? 15.0f : 0.0f;
template <typename T> constexpr float kTileShift = std::is_same<T, _Float16>::value ? 7.0f : 0.0f;

struct AttendArgs {
  Seqs s;
  const void* k;
  const void* v;
  int heads, group, d;
  const void* q;
  int64_t qt, qh;
  int q_vec;
  float scale2;              // scale log2(e)
  int window;
  const int32_t* sel;
  int m;
  void* out;
  float* lse;
  int hq;
  int64_t tokens;
  int chunk;                 // keys (or list entries) a workgroup takes
  int splits;                // 1: results go to out, else partial results
  float* part_o;             // [splits][tokens * hq][d], not divided by the sum
  float* part_ml;            // [splits][tokens * hq][2]: maximum (base 2), sum
  int tiles_token;           // selection: row tiles a (token, head) takes
};

// a row's share of a key range in which it sees no key; r: row of the (sequence, head)
__device__ __forceinline__ void mark_empty(const AttendArgs& a, int split, int row0, int r,
                                           int head) {
  const int ti = r / a.group, hh = r - ti * a.group;
  const int64_t orow = (int64_t)(row0 + ti) * a.hq + head * a.group + hh;
  float* ml = a.part_ml + ((int64_t)split * a.tokens * a.hq + orow) * 2;
  ml[0] = -INFINITY;
  ml[1] = 0.0f;
}

// Values that some rows of a tile do not see pass through the same matrix product as those they do
// see, with a weight of 0, and 0 times a NaN or an infinity would reach them.  Where a step of
// 32 keys holds such keys (later tokens', or of windows that have moved on: before `low` or from
// `from` on), the kernels put 0 for every value that is not finite, and if there was any,
// add_not_finite gives it to the rows that see it: a positive weight times it is itself.  A result
// that is no number although the row's sum is one starts from 0 and gets what the row sees of all
// keys (an infinity times the rest of a weight's rounding, which may be 0 or negative, is not what
// the row holds).
__device__ __forceinline__ bool mixed_step(int key0, int from, int low) {
  return key0 + 32 > from || key0 < low;
}

// The signs of a word's two elements are set where the exponent is all ones, of an infinity or a
// NaN: adding the lowest exponent bit carries.
template <typename T>
__device__ __forceinline__ uint32_t not_finite_signs(uint32_t w) {
  constexpr bool f16 = std::is_same<T, _Float16>::value;
  return ((w & (f16 ? 0x7C007C00u : 0x7F807F80u)) + (f16 ? 0x04000400u : 0x00800080u)) & 0x80008000u;
}

// Puts 0 in N operands of 8 slots from key for what is not finite, and for slots from `end` on,
// which may hold anything; returns 0 unless a key before `end` had such a value.
template <typename T, int N>
__device__ __forceinline__ uint32_t put_zeros(typename Vec8<T>::type* v, int key, int end) {
  uint4 u[N];
#pragma unroll
  for (int i = 0; i < N; ++i) u[i] = __builtin_bit_cast(uint4, v[i]);
  uint32_t any = 0;
  const auto word = [&](int j, auto at) {
    const int k = key + 2 * j;
    const uint32_t held = k + 1 < end ? 0xFFFFFFFFu : k < end ? 0xFFFFu : 0u;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      uint32_t& w = at(u[i]);
      w &= held;
      const uint32_t bad = not_finite_signs<T>(w) >> 15;
      any |= bad;
      asm volatile("" : "+v"(any));      // one after another: a tree would keep all in registers
      w &= ~((bad << 16) - bad);
    }
  };
  word(0, [](uint4& x) -> uint32_t& { return x.x; });
  word(1, [](uint4& x) -> uint32_t& { return x.y; });
  word(2, [](uint4& x) -> uint32_t& { return x.z; });
  word(3, [](uint4& x) -> uint32_t& { return x.w; });
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = __builtin_bit_cast(typename Vec8<T>::type, u[i]);
  return any;
}

// A workgroup's tile, kept in LDS for what comes after its loop.
struct Tile {
  int b, row0, n, total;     // of its sequence
  int r0, rows, tok;         // its rows, of the sequence's; its token (selection)
};

// The kernel's arguments, read again where they are used.
__device__ __forceinline__ const AttendArgs& args_again() {
  auto* p = (const __attribute__((address_space(4))) AttendArgs*)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  return *(const AttendArgs*)p;
}

// The rows of a tile, ra .. rb - 1, that a dimension's results have got an infinity of one sign
// for: those before lo and those from hi on.  (A NaN is both signs.)
struct Had {
  int lo, hi;
  __device__ __forceinline__ void take(int first, int last) {
    if (first <= lo) lo = max(lo, last);
    if (last >= hi) hi = min(hi, first);
  }
};

// x, not finite, is added to dimension dim of the results of the rows that see the key, unless they
// have got it: the same again changes nothing.
template <typename T>
__device__ __forceinline__ void add_to_rows(const Tile& tile, int ra, int rb, int key, int dim, float x,
                                            Had& pos, Had& neg) {
  const AttendArgs& a = args_again();
  const int64_t slot0 = (int64_t)tile.total - tile.n;
  const int first = (int)max((int64_t)ra, (key - slot0) * a.group - tile.r0);
  const int last = a.window > 0
      ? (int)min((int64_t)rb, (key + (int64_t)a.window - slot0) * a.group - tile.r0) : rb;
  if (first >= last) return;
  const bool p = !(x < 0.0f), n = !(x > 0.0f);
  const int begin = max(first, min(p ? pos.lo : rb, n ? neg.lo : rb));
  const int end = min(last, max(p ? pos.hi : ra, n ? neg.hi : ra));
#pragma unroll 1
  for (int r = begin; r < end; ++r) {
    const int rr = tile.r0 + r, ti = rr / a.group;
    const int64_t orow = (int64_t)(tile.row0 + ti) * a.hq + blockIdx.x % a.heads * a.group +
                         (rr - ti * a.group);
    if (a.splits == 1) {
      T* o = (T*)a.out + orow * a.d + dim;
      *o = (T)((float)*o + x);
    } else {
      a.part_o[((int64_t)blockIdx.y * a.tokens * a.hq + orow) * a.d + dim] += x;
    }
  }
  if (p) pos.take(first, last);
  if (n) neg.take(first, last);
}

// By a wave, for the rows ra .. rb - 1 of the workgroup's tile; whole: over all its keys, and not
// only those of mixed steps.  It is rare: what it needs is read again, so that
// nothing is kept for it in registers through a kernel's loop.
template <typename T, bool SEL>
__device__ void add_not_finite(const Tile& tile, int ra, int rb, bool whole) {
  const AttendArgs& a = args_again();
  __threadfence_block();               // other lanes wrote the rows
  const int lane = threadIdx.x & 63, P = 1 << a.s.page_shift, d = a.d;
  const int head = blockIdx.x % a.heads, split = blockIdx.y, sub_shift = a.s.page_shift - 5;
  const int b = __builtin_amdgcn_readfirstlane(tile.b);
  const int total = __builtin_amdgcn_readfirstlane(tile.total);
  const int n = __builtin_amdgcn_readfirstlane(tile.n);
  const int r0 = __builtin_amdgcn_readfirstlane(tile.r0);
  const int32_t* list = nullptr;
  int st0, st1, kend, from, low = 0;
  {
    const int rows = __builtin_amdgcn_readfirstlane(tile.rows);
    const int64_t first = (int64_t)total - n + r0 / a.group;          // slots of the first and last row
    const int64_t last = SEL ? first : (int64_t)total - n + (r0 + rows - 1) / a.group;
    const int64_t held = min((int64_t)total, (int64_t)a.s.max_pages << a.s.page_shift);
    if constexpr (SEL) {               // all rows are one token's
      kend = (int)max((int64_t)0, min(held, first + 1));
      st0 = (split * a.chunk) << sub_shift;
      st1 = min((split + 1) * a.chunk, a.m) << sub_shift;
      list = a.sel + ((int64_t)__builtin_amdgcn_readfirstlane(tile.tok) * a.heads + head) * a.m;
    } else {
      const int64_t klo = a.window > 0 ? max((int64_t)0, first - a.window + 1) : 0;
      kend = (int)max((int64_t)0, min(min(held, last + 1), ((int64_t)split + 1) * a.chunk));
      st0 = (int)(max((int64_t)split * a.chunk, klo) >> 5);
      st1 = (kend + 31) >> 5;
      if (a.window > 0) low = (int)max((int64_t)0, last - a.window + 1);
    }
    from = (int)max((int64_t)0, min(first + 1, (int64_t)kend));
  }
#pragma unroll 1
  for (int dim = lane; dim - lane < d; dim += 64) {
    Had pos{ra, rb}, neg{ra, rb};
#pragma unroll 1
    for (int st = st0; st < st1; ++st) {
      if (__ballot(dim < d && (pos.lo < pos.hi || neg.lo < neg.hi)) == 0) break;
      int64_t key64 = (int64_t)st << 5;
      if constexpr (SEL)
        key64 = ((int64_t)list[st >> sub_shift] << a.s.page_shift) + 32 * (st & ((1 << sub_shift) - 1));
      if (key64 < 0 || key64 >= kend) continue;
      const int key0 = (int)key64;
      if (!whole && !mixed_step(key0, from, low)) continue;
      const int phys = phys_page(a.s, b, key0 >> a.s.page_shift);
      if (phys < 0 || dim >= d) continue;
      const T* v = (const T*)a.v + (((int64_t)phys * a.heads + head) * d + dim) * P + (key0 & (P - 1));
#pragma unroll 1
      for (int at = 0; at < 32; at += 8) {
        const uint4 u = load16<uint4>(v + at);
        if ((not_finite_signs<T>(u.x) | not_finite_signs<T>(u.y) | not_finite_signs<T>(u.z) |
             not_finite_signs<T>(u.w)) == 0)
          continue;
#pragma unroll 1
        for (int e = at; e < at + 8 && key0 + e < kend; ++e)
          if (!(fabsf((float)v[e]) <= FLT_MAX))
            add_to_rows<T>(tile, ra, rb, key0 + e, dim, (float)v[e], pos, neg);
      }
    }
  }
}

// A few query rows (16 RT: tokens x heads of a group) against a range of keys; the NW waves take
// every NW-th step of 32 keys each, straight from memory into matrix operands, and are joined at
// the end.  Every byte of the cache is read by one wave once, so LDS would only add a trip.  The
// page numbers of 64 steps are one load, a lane a step; while a step is computed the next one's
// operands are in flight (16 KB at d = 128) where registers allow it.  Bound by the cache's bytes,
// for short contexts by the chain of loads: sequence, page numbers, keys.  64 sequences of up to
// 32,768 keys, 32 heads on 8 of 128: 634 us a call, 5.5 TB/s; one token on 1000 keys 8.2 us.  The
// rest of the weights' rounding as a second product costs nothing (634 us without) and brings the
// error from 1.3 times the result's rounding to that rounding.
template <typename T, int NS, int RT, bool SEL, int NW>
__global__ __launch_bounds__(64 * NW, NS * RT <= 6 ? 2 : 1) void k_attend_few(AttendArgs a) {
  typedef typename Vec8<T>::type V8;
  constexpr int ND = 2 * NS;                 // 16-dimension tiles of the result
  constexpr int R = 16 * RT;
  constexpr int BUF = NS * RT <= 4 ? 2 : 1;  // steps in registers
  __shared__ float sm[NW][R], sl[NW][R];
  __shared__ int spoilt[NW];                 // a value of a mixed step is not finite
  __shared__ Tile tile;
  __shared__ f32x4 so[NW / 2][ND][64];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n16 = lane & 15, g = lane >> 4;
  const int head = blockIdx.x % a.heads;
  const int64_t item = blockIdx.x / a.heads;
  const int split = blockIdx.y;
  const int P = 1 << a.s.page_shift, d = a.d, G = a.group;

  Seq sq;
  int r0, rows;
  int64_t tok = 0;
  if constexpr (SEL) {
    tok = item / a.tiles_token;
    sq = find_seq(a.s, tok, 1, 1, 0);
    r0 = (int)(tok - sq.row0) * G + (int)(item - tok * a.tiles_token) * R;
    rows = min(R, (int)(tok - sq.row0 + 1) * G - r0);
  } else {
    sq = find_seq(a.s, item, G, R, 1);
    const int64_t rr = (item - first_of(sq.row0, sq.b, G, R, 1)) * R;
    if (rr >= (int64_t)sq.n * G) return;
    r0 = (int)rr;
    rows = (int)min((int64_t)R, (int64_t)sq.n * G - rr);
  }
  const int b = sq.b, row0 = sq.row0, n = sq.n, total = sq.total;
  // keys that exist for this sequence, and the tile's: [klo, khi)
  const int64_t held = min((int64_t)total, (int64_t)a.s.max_pages << a.s.page_shift);
  const int khi = (int)max((int64_t)0, min(held, (int64_t)total - n + (r0 + rows - 1) / G + 1));
  const int klo = a.window > 0
      ? (int)max((int64_t)0, (int64_t)total - n + r0 / G - a.window + 1) : 0;
  // mixed steps (selected pages: all rows are one token's)
  int from = khi, low0 = 0;
  if constexpr (!SEL) {
    from = (int)max((int64_t)0, min((int64_t)khi, (int64_t)total - n + r0 / G + 1));
    if (a.window > 0)
      low0 = (int)max((int64_t)0, (int64_t)total - n + (r0 + rows - 1) / G - a.window + 1);
  }
  // steps of 32 keys: [st0, st1) in units of 32 keys, or of (list entry, part of its page)
  int st0, st1;
  const int sub_shift = a.s.page_shift - 5;
  if constexpr (SEL) {
    st0 = (split * a.chunk) << sub_shift;
    st1 = min((split + 1) * a.chunk, a.m) << sub_shift;
  } else {
    const int64_t c0 = (int64_t)split * a.chunk, c1 = c0 + a.chunk;
    if (c0 >= khi || c1 <= klo) {
      if (a.splits > 1) {
        if (tid < rows) mark_empty(a, split, row0, r0 + tid, head);
        return;
      }
      st0 = st1 = 0;                        // rows that see no key: zeros
    } else {
      st0 = (int)(max(c0, (int64_t)klo) >> 5);
      st1 = (int)((min(c1, (int64_t)khi) + 31) >> 5);
    }
  }

  if (lane == 0) tile = Tile{b, row0, n, total, r0, rows, (int)tok};
  uint32_t not_finite = 0;                   // not 0: a value of a mixed step
  // this wave's steps, 64 at a time: a lane's page and first key
  const int32_t* list = SEL ? a.sel + (tok * a.heads + head) * a.m : nullptr;
  int ahead = st0 + wave, lphys = -1, lkey = 0;
  uint64_t todo = 0;
  const auto refill = [&] {
    const int st = ahead + NW * lane;
    lphys = -1;
    if (st < st1 && st >= st0) {
      if constexpr (SEL) {
        const int lp = list[st >> sub_shift];
        const int64_t key = ((int64_t)lp << a.s.page_shift) + 32 * (st & ((1 << sub_shift) - 1));
        if (lp >= 0 && key < khi) {
          lphys = phys_page(a.s, b, lp);
          lkey = (int)key;
        }
      } else {
        lkey = st << 5;
        lphys = phys_page(a.s, b, lkey >> a.s.page_shift);
      }
    }
    ahead += NW * 64;
    todo = __ballot(lphys >= 0);
  };
  // the next step's lane, -1 if there is none
  const auto next = [&] {
    while (todo == 0 && ahead < st1) refill();
    const int i = todo == 0 ? -1 : __ffsll((unsigned long long)todo) - 1;
    todo &= todo - 1;
    return __builtin_amdgcn_readfirstlane(i);
  };
  // addresses: a uniform part and the lane's own bytes.  The last 32 dimensions of a row that is
  // no multiple of 32 wide overlap those before; queries are 0 where they do.
  const char* kc = (const char*)a.k + (int64_t)head * P * d * 2;
  const char* vc = (const char*)a.v + (int64_t)head * P * d * 2;
  const uint32_t klane = ((8 * (n16 >> 2) + (n16 & 3)) * d + min(8 * g, d - 8)) * 2;
  const uint32_t vlane = (n16 * P + 8 * g) * 2;
  const auto dims_at = [&](int s) { return max(0, min(32 * s, d - 32)); };
  V8 kf[BUF][2][NS], vf[BUF][ND];
  int key[BUF];
  const auto load = [&](int i, auto buf) {
    constexpr int B = decltype(buf)::value;
    const int phys = __builtin_amdgcn_readlane(lphys, i);
    key[B] = __builtin_amdgcn_readlane(lkey, i);
    const int64_t rec = (int64_t)phys * a.heads * P * d * 2;
    const int off = key[B] & (P - 1);
    const char* kp = kc + rec + off * d * 2;
    const char* vp = vc + rec + off * 2;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int s = 0; s < NS; ++s)
        kf[B][t][s] = load16<V8>(kp + (4 * t * d + dims_at(s)) * 2 + klane);
#pragma unroll
    for (int dt = 0; dt < ND; ++dt)
      vf[B][dt] = load16<V8>(vp + min(16 * dt, d - 16) * P * 2 + vlane);
  };
  constexpr std::integral_constant<int, 0> first{};
  constexpr std::integral_constant<int, BUF - 1> second{};
  int cur = next();
  if (BUF == 2 && cur >= 0) load(cur, first);

  int lim[RT], low[RT];
  V8 qf[RT][NS];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int r = rt * 16 + n16;
    const bool live = r < rows;
    const int rr = r0 + (live ? r : 0), ti = rr / G, hh = rr - ti * G;
    const int64_t slot = (int64_t)total - n + ti;
    lim[rt] = live ? (int)max((int64_t)-1, min(slot, held - 1)) : -1;
    low[rt] = a.window > 0 ? (int)max((int64_t)0, slot - a.window + 1) : 0;
    const T* qr = (const T*)a.q + (int64_t)(row0 + ti) * a.qt + (int64_t)(head * G + hh) * a.qh;
    load_rows8<T, NS>(qf[rt], [&](int s) { return qr + min(dims_at(s) + 8 * g, d - 8); }, a.q_vec);
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      const int dim = dims_at(s) + 8 * g;
      if (dim >= d || dim < 32 * s) qf[rt][s] = V8((T)0.0f);
    }
  }

  f32x4 o[RT][ND];
  float mx[RT], sum[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    mx[rt] = -INFINITY;
    sum[rt] = 0.0f;
#pragma unroll
    for (int dt = 0; dt < ND; ++dt) o[rt][dt] = f32x4{0, 0, 0, 0};
  }
  const auto compute = [&](auto buf) {
    constexpr int B = decltype(buf)::value;
    if (mixed_step(key[B], from, low0)) not_finite |= put_zeros<T, ND>(vf[B], key[B] + 8 * g, khi);
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      f32x4 sc[2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        sc[t] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int s = 0; s < NS; ++s) sc[t] = mfma16(kf[B][t][s], qf[rt][s], sc[t]);
      }
      float m = mx[rt];
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int kk = key[B] + 8 * g + 4 * t + i;
          const float v = sc[t][i] * a.scale2;
          sc[t][i] = kk <= lim[rt] && kk >= low[rt] ? v : -INFINITY;
          m = fmaxf(m, sc[t][i]);
        }
      m = fmaxf(m, __shfl_xor(m, 16));
      m = fmaxf(m, __shfl_xor(m, 32));
      const float base = m == -INFINITY ? 0.0f : m;
      const float alpha = exp2_fast(mx[rt] - base);
      mx[rt] = m;
      // weights in [0, 1] (times 2^kFewShift) for the matrix product: rounded to T, and what the
      // rounding leaves (the matrix unit waits for memory here, a second product costs nothing)
      V8 p, rest;
      float z = 0.0f;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float e = exp2_fast(sc[t][i] - base + kFewShift<T>);
          z += e;
          p[4 * t + i] = (T)e;
          rest[4 * t + i] = (T)(e - (float)p[4 * t + i]);
        }
      sum[rt] = sum[rt] * alpha + z;
#pragma unroll
      for (int dt = 0; dt < ND; ++dt) {
        o[rt][dt] *= alpha;
        o[rt][dt] = mfma16(vf[B][dt], rest, o[rt][dt]);
        o[rt][dt] = mfma16(vf[B][dt], p, o[rt][dt]);
      }
    }
  };
  if constexpr (BUF == 2) {
    while (cur >= 0) {
      const int nxt = next();
      if (nxt >= 0) load(nxt, second);
      compute(first);
      if (nxt < 0) break;
      cur = next();
      if (cur >= 0) load(cur, first);
      compute(second);
    }
  } else {
    while (cur >= 0) {
      load(cur, first);
      cur = next();
      compute(first);
    }
  }

  // arguments once more: kept through the loop, they would cost it registers
  const AttendArgs ar = args_again();
  // join the waves
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    sum[rt] += __shfl_xor(sum[rt], 16);
    sum[rt] += __shfl_xor(sum[rt], 32);
    if (g == 0) {
      sm[wave][rt * 16 + n16] = mx[rt];
      sl[wave][rt * 16 + n16] = sum[rt];
    }
  }
  const uint64_t any_lane = __ballot(not_finite != 0);
  if (lane == 0) spoilt[wave] = any_lane != 0;
  __syncthreads();
  const int tile_rows = __builtin_amdgcn_readfirstlane(tile.rows);
  bool no_number = false;                  // a result is none, though its row's sum is
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int c = rt * 16 + n16;
    float mm = sm[0][c];
#pragma unroll
    for (int w = 1; w < NW; ++w) mm = fmaxf(mm, sm[w][c]);
    const float base = mm == -INFINITY ? 0.0f : mm;
    float z = 0.0f;
#pragma unroll
    for (int w = 0; w < NW; ++w) z += sl[w][c] * exp2_fast(sm[w][c] - base);
    const float f = exp2_fast(mx[rt] - base);
#pragma unroll
    for (int dt = 0; dt < ND; ++dt) o[rt][dt] *= f;
    // halves: the upper waves hand their sums to the lower ones
#pragma unroll
    for (int h = NW / 2; h >= 1; h /= 2) {
      if (wave >= h && wave < 2 * h)
#pragma unroll
        for (int dt = 0; dt < ND; ++dt) so[wave - h][dt][lane] = o[rt][dt];
      __syncthreads();
      if (wave < h)
#pragma unroll
        for (int dt = 0; dt < ND; ++dt) o[rt][dt] += so[wave][dt][lane];
      __syncthreads();
    }
    if (wave != 0) continue;
    bool none = false;
    float zero = 0.0f;                     // NaN where a result is not finite
#pragma unroll
    for (int dt = 0; dt < ND; ++dt)
#pragma unroll
      for (int i = 0; i < 4; ++i) zero = fmaf(o[rt][dt][i], 0.0f, zero);
    if (zero != 0.0f && z > 0.0f) {
#pragma unroll
      for (int dt = 0; dt < ND; ++dt)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          none |= o[rt][dt][i] != o[rt][dt][i];
          o[rt][dt][i] = o[rt][dt][i] != o[rt][dt][i] ? 0.0f : o[rt][dt][i];
        }
    }
    no_number |= __ballot(none && c < tile_rows) != 0;
    if (c < tile_rows) {
      const int rr = tile.r0 + c, ti = rr / ar.group, hh = rr - ti * ar.group;
      const int64_t orow = (int64_t)(tile.row0 + ti) * ar.hq + blockIdx.x % ar.heads * ar.group + hh;
      const int64_t pr = (int64_t)blockIdx.y * ar.tokens * ar.hq + orow;
      const float inv = z > 0.0f ? 1.0f / z : 0.0f;
#pragma unroll
      for (int dt = 0; dt < ND; ++dt) {
        const f32x4 v = o[rt][dt];
        const int dim = 16 * dt + 4 * g;
        if (dim >= ar.d) continue;
        if (ar.splits == 1) {
          alignas(8) T w[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) w[i] = (T)(z > 0.0f ? v[i] * inv : z);
          *reinterpret_cast<uint2*>((T*)ar.out + orow * ar.d + dim) = *reinterpret_cast<uint2*>(w);
        } else {
          *reinterpret_cast<f32x4*>(ar.part_o + pr * ar.d + dim) = v;
        }
      }
      if (g == 0) {
        if (ar.splits == 1) {
          if (ar.lse)
            ar.lse[orow] = z > 0.0f ? (mm - kFewShift<T> + log2_fast(z)) * kLn2
                                   : (z == 0.0f ? -INFINITY : z);
        } else {
          float* ml = ar.part_ml + pr * 2;
          ml[0] = mm - kFewShift<T>;
          ml[1] = z;
        }
      }
    }
  }
  if (wave != 0) return;
  int any = 0;
#pragma unroll
  for (int w = 0; w < NW; ++w) any |= spoilt[w];
  if (no_number || __builtin_amdgcn_readfirstlane(any) != 0)
    add_not_finite<T, SEL>(tile, 0, tile_rows, no_number);
}

// Many query rows (NW waves x 32) against a range of keys.  Steps of 64 keys (32 with four waves)
// pass through LDS, where the waves share them; a wave holds its queries (B operands) and results
// in registers.
//
// A turn of the loop has a matrix part, the products of step p - 1 and the scores of step p, and
// a vector part, the weights of a step; between them the operands of the step after are passed
// on.  Eight waves are two on every SIMD, one of either half of the workgroup: the first half
// runs matrix(p), vector(p), the second half vector(p - 1), matrix(p), so that one wave's matrix
// part meets the other's vector part.  (Four waves leave that to chance: two workgroups share a
// CU.)
//
// Keys and values have two LDS slots each, filled from registers that were loaded a turn
// earlier: every wave reads keys p and values p - 1 in turn p and writes keys p + 1 and
// values p, and a barrier ends the turn.
//
// The running maximum is only moved (and the results rescaled) when a step's weights at the old
// one add up to more than 2^8, or a row sees its first key: a common factor cancels in the end,
// and weights up to 2^8 are as exact as those up to 1.  So most steps need no maximum at all.
// A weight is 2^(score scale - maximum), one fma, as long as the rounding of the maximum, a product
// with the scale itself, is small against 1.  Once a maximum passes 2^10 the wave keeps them
// unscaled and takes the difference before the scaling, where it is exact for the largest scores,
// whatever their size (fp32 neighbours at 2^33 lie 1024 apart, and a rounded maximum would make
// weights of 2^512, or none).
//
// Rows of the score tile are keys in the order that makes its accumulator the B operand of the
// second product: row r is key r with bits 2 and 3 exchanged.
//
// 2048 tokens on 34,816 keys, 32 heads on 8 of 128: 997 us a call, 1137 TFLOP/s (a product of 8192^3
// 1274): matrix unit busy 56 % of the cycles, vector unit 42, LDS 35.  Up to 64 dimensions the
// vector unit bounds it (51 %, matrix unit 28): prompts with a window, 178 us.
template <typename T, int ND, int NW>
__global__ __launch_bounds__(64 * NW, ND <= 2 ? 3 : ND <= 4 ? 2 : 1) void k_attend_tile(AttendArgs a) {
  typedef typename Vec8<T>::type V8;
  constexpr int NT = 64 * NW;
  constexpr int HV = NW == 8 ? 2 : 1;             // 32-key blocks of a step
  constexpr int KEYS = 32 * HV;
  constexpr int CD = 4 * ND;                      // 16-byte chunks of a key's row
  constexpr int CK = CD <= 8 ? 8 : (CD + 15) / 16 * 16;   // and the LDS row's
  constexpr int KX = CK <= 8 ? 7 : 15;            // chunk c of row r is kept at c ^ (r & KX)
  constexpr int NS = 2 * ND;                      // 16-dimension steps of the scores
  constexpr int KCH = 32 * CD;                    // chunks of a block's keys, and of its values
  constexpr int PER = (KCH + NT - 1) / NT;
  constexpr int R = 32 * NW;
  __shared__ V8 ks[2][HV][32 * CK];
  __shared__ V8 vs[2][HV][KCH];
  __shared__ int spoilt;                          // a value of a mixed step is not finite
  __shared__ Tile tile;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c32 = lane & 31, half = lane >> 5;
  const int head = blockIdx.x % a.heads;
  // later tiles see more keys: they start first
  const int64_t item = (int64_t)(gridDim.x / a.heads) - 1 - blockIdx.x / a.heads;
  const int split = blockIdx.y;
  const int P = 1 << a.s.page_shift, d = a.d, G = a.group;

  const Seq sq = find_seq(a.s, item, G, R, 1);
  const int b = sq.b, row0 = sq.row0, n = sq.n, total = sq.total;
  const int64_t rr0 = (item - first_of(row0, b, G, R, 1)) * R;
  if (rr0 >= (int64_t)n * G) return;
  const int r0 = (int)rr0;
  const int rows = (int)min((int64_t)R, (int64_t)n * G - rr0);
  const int held = (int)min((int64_t)total, (int64_t)a.s.max_pages << a.s.page_shift);
  const int64_t khi64 = min((int64_t)held, (int64_t)total - n + (r0 + rows - 1) / G + 1);
  const int64_t klo = a.window > 0 ? max((int64_t)0, (int64_t)total - n + r0 / G - a.window + 1) : 0;
  const int64_t k0 = (int64_t)split * a.chunk, k1 = k0 + a.chunk;
  int kbeg = 0, steps = 0;                        // steps of KEYS keys from key kbeg
  if (k0 < khi64 && k1 > klo) {
    kbeg = (int)(max(k0, klo) / KEYS) * KEYS;
    steps = (int)cdiv(min(k1, khi64) - kbeg, KEYS);
  } else if (a.splits > 1) {
    if (tid < rows) mark_empty(a, split, row0, r0 + tid, head);
    return;
  }
  const int kend = (int)min(k1, khi64);           // first key that is not this workgroup's
  const int from = (int)max((int64_t)0, min((int64_t)total - n + r0 / G + 1, (int64_t)kend));
  const int low0 = a.window > 0      // mixed steps
      ? (int)max((int64_t)0, (int64_t)total - n + (r0 + rows - 1) / G - a.window + 1) : 0;

  // queries, slots of this wave's rows
  V8 qf[NS];
  int lim, low;
  const int wr0 = wave * 32;
  {
    const int r = wr0 + c32;
    const bool live = r < rows;
    const int rr = r0 + (live ? r : 0), ti = rr / G, hh = rr - ti * G;
    const int64_t slot = (int64_t)total - n + ti;
    lim = live ? (int)max((int64_t)-1, min(slot, (int64_t)kend - 1)) : -1;
    low = a.window > 0 && live ? (int)max((int64_t)0, slot - a.window + 1) : 0;
    const T* qr = (const T*)a.q + (int64_t)(row0 + ti) * a.qt + (int64_t)(head * G + hh) * a.qh;
    load_rows8<T, NS>(qf, [&](int s) { return qr + min(16 * s + 8 * half, d - 8); }, a.q_vec);
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      const bool zero = 16 * s + 8 * half >= d || a.scale2 == 0.0f;
#pragma unroll
      for (int e = 0; e < 8; ++e)
        qf[s][e] = zero ? (T)0.0f : a.scale2 < 0.0f ? -qf[s][e] : qf[s][e];
    }
  }
  // the scale's sign is in the queries, and so is a scale of 0: a masked score, -inf, stays -inf
  const float sc2 = a.scale2 != 0.0f ? fabsf(a.scale2) : 1.0f;
  // keys wlow .. wlim are seen by every row of the wave: steps among them need no mask
  int wlim = -1, wlow = 0;
  if (wr0 < rows) {
    const int last = min(wr0 + 32, rows) - 1;
    const int64_t s_first = (int64_t)total - n + (r0 + wr0) / G;
    const int64_t s_last = (int64_t)total - n + (r0 + last) / G;
    wlim = (int)max((int64_t)-1, min(s_first, (int64_t)kend - 1));
    wlow = a.window > 0 ? (int)max((int64_t)0, s_last - a.window + 1) : 0;
  }

  // where this thread's chunks of a block's keys and values come from (bytes) and go to
  uint32_t kg[PER], vg[PER];
  int kl[PER], vl[PER];
  const int vkey = 8 * (tid & 3);              // of a thread's values: NT is a multiple of 4
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const int i = min(tid + NT * j, KCH - 1);
    const int key = i / CD, c = i - key * CD;
    const int row = (key & 0x13) | ((key & 4) << 1) | ((key & 8) >> 1);
    kg[j] = (key * d + min(8 * c, d - 8)) * 2;
    kl[j] = row * CK + (c ^ (row & KX));
    const int dim = i >> 2, cv = i & 3;
    vg[j] = (min(dim, d - 1) * P + 8 * cv) * 2;
    vl[j] = dim * 4 + (cv ^ ((dim >> 2) & 3));
  }
  const auto mine = [&](int j) { return KCH % NT == 0 || tid + NT * j < KCH; };

  // A block (32 keys): its page, raw as long as nothing waits for the load; then the byte
  // offset of its record and how many of its keys exist
  struct Block {
    int64_t rec;       // of the page's keys and values
    int off;           // first key's slot
    int live;
  };
  const Table prow = a.s.pages + (int64_t)b * a.s.stride;
  const int kcap = steps > 0 ? kend - 1 : 0;
  const auto raw_page = [&](int step, int hv) {
    return prow[min(kbeg + step * KEYS + 32 * hv, kcap) >> a.s.page_shift];
  };
  const int64_t page_bytes = (int64_t)a.heads * P * d * 2;
  const auto block_of = [&](int step, int hv, int raw) {
    Block k;
    const int key = kbeg + step * KEYS + 32 * hv;
    const bool ok = (unsigned)raw < (unsigned)a.s.cache_pages;
    k.rec = (ok ? raw : 0) * page_bytes;
    k.off = key & (P - 1);
    k.live = ok ? kend - key : 0;
    return k;
  };
  const char* kc = (const char*)a.k + (int64_t)head * P * d * 2;
  const char* vc = (const char*)a.v + (int64_t)head * P * d * 2;
  V8 kreg[HV][PER], vreg[HV][PER];
  const auto load_k = [&](const Block* k) {
#pragma unroll
    for (int hv = 0; hv < HV; ++hv)
#pragma unroll
      for (int j = 0; j < PER; ++j)
        kreg[hv][j] = load16<V8>(kc + k[hv].rec + k[hv].off * d * 2 + kg[j]);
  };
  const auto load_v = [&](const Block* k) {
#pragma unroll
    for (int hv = 0; hv < HV; ++hv)
#pragma unroll
      for (int j = 0; j < PER; ++j)
        vreg[hv][j] = load16<V8>(vc + k[hv].rec + k[hv].off * 2 + vg[j]);
  };
  const auto store_k = [&](int slot) {
#pragma unroll
    for (int hv = 0; hv < HV; ++hv)
#pragma unroll
      for (int j = 0; j < PER; ++j)
        if (mine(j)) ks[slot][hv][kl[j]] = kreg[hv][j];
  };
  const auto store_v = [&](int slot, const Block* k, int key0) {
#pragma unroll
    for (int hv = 0; hv < HV; ++hv) {
      const int kb = key0 + 32 * hv;
      if (k[hv].live < 32 || mixed_step(kb, from, low0))
        if (put_zeros<T, PER>(vreg[hv], kb + vkey, kb + k[hv].live) != 0) spoilt = 1;
#pragma unroll
      for (int j = 0; j < PER; ++j)
        if (mine(j)) vs[slot][hv][vl[j]] = vreg[hv][j];
    }
  };

  f32x16 o[ND], sc[HV];
  V8 pw[HV][2];
  float mx = -INFINITY, sum = 0.0f;
  bool coarse = false;                            // of the wave: mx is unscaled
#pragma unroll
  for (int hv = 0; hv < HV; ++hv) pw[hv][0] = pw[hv][1] = V8((T)0.0f);
#pragma unroll
  for (int dt = 0; dt < ND; ++dt) o[dt] = f32x16(0.0f);
  const auto products = [&](int slot) {
#pragma unroll
    for (int hv = 0; hv < HV; ++hv)
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int dt = 0; dt < ND; ++dt) {
          const V8 vf = vs[slot][hv][(32 * dt + c32) * 4 + ((2 * u + half) ^ ((c32 >> 2) & 3))];
          o[dt] = mfma32(vf, pw[hv][u], o[dt]);
        }
  };

  const auto matrix = [&](auto parity) {
    constexpr int cur = decltype(parity)::value;
    // nothing of the vector part, nor the scalar loads of page numbers, moves between these
    // products: a scalar load in flight turns every wait for an operand into one for all of them
    __builtin_amdgcn_sched_barrier(0);
    constexpr int NP = HV * 2 * ND, M = NP + NS * HV;       // products of weights, then of scores
    const auto operand = [&](int i) {
      if (i < NP) {
        const int hv = i / (2 * ND), u = i / ND % 2, dt = i % ND;
        return vs[cur ^ 1][hv][(32 * dt + c32) * 4 + ((2 * u + half) ^ ((c32 >> 2) & 3))];
      }
      const int s = (i - NP) / HV, hv = (i - NP) % HV;
      return ks[cur][hv][c32 * CK + ((2 * s + half) ^ (c32 & KX))];
    };
#pragma unroll
    for (int hv = 0; hv < HV; ++hv) sc[hv] = f32x16(0.0f);
    // operands are read a few products ahead, in this order also where the compiler keeps to the
    // source's (short of registers it does: every product then waits for its operand, 8 % of a
    // chunk's time)
    V8 op[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) op[i] = operand(i);
#pragma unroll
    for (int i = 0; i < M; ++i) {
      if (i < NP) o[i % ND] = mfma32(op[i & 3], pw[i / (2 * ND)][i / ND % 2], o[i % ND]);
      else sc[(i - NP) % HV] = mfma32(op[i & 3], qf[(i - NP) / HV], sc[(i - NP) % HV]);
      if (i + 4 < M) op[i & 3] = operand(i + 4);
    }
    __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
    for (int i = 0; i < HV * 4 * ND; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  // blocks of the steps p, p + 1, p + 2, raw pages of step p + 3
  Block b0[HV], b1[HV], b2[HV];
  int raw[HV];
  const auto pass_on = [&](int p, auto parity) {
    constexpr int cur = decltype(parity)::value;
    store_k(cur ^ 1);
    store_v(cur, b0, kbeg + p * KEYS);
    load_k(b2);
    load_v(b1);
#pragma unroll
    for (int hv = 0; hv < HV; ++hv) {
      b0[hv] = b1[hv];
      b1[hv] = b2[hv];
      b2[hv] = block_of(p + 3, hv, raw[hv]);
      raw[hv] = raw_page(p + 4, hv);
    }
  };
  const auto vector = [&](int p, const int* live) {
    const int key0 = kbeg + p * KEYS;
    bool edge = key0 + KEYS - 1 > wlim || key0 < wlow;
#pragma unroll
    for (int hv = 0; hv < HV; ++hv) edge |= live[hv] < 32;
    if (edge) {
#pragma unroll
      for (int hv = 0; hv < HV; ++hv)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int kk = 16 * (i >> 3) + 8 * half + (i & 7), key = key0 + 32 * hv + kk;
          const bool see = kk < live[hv] && key <= lim && key >= low;
          sc[hv][i] = see ? sc[hv][i] : -INFINITY;
        }
    }
    // weights at the present maximum; their sum says whether it has to move
    constexpr float shift = kTileShift<T>, limit = shift > 0.0f ? 0x1p15f : 0x1p8f;
    const auto weights = [&](float base) {
      float z = 0.0f;
#pragma unroll
      for (int hv = 0; hv < HV; ++hv)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const float e = exp2_fast(__fmaf_rn(sc[hv][i], sc2, -base));
          z += e;
          pw[hv][i >> 3][i & 7] = (T)e;        // rounded for the matrix product
        }
      return z;
    };
    float z = 0.0f;
    bool move = coarse || __ballot(mx == -INFINITY && lim >= key0) != 0;
    if (!move) {
      z = weights(mx == -INFINITY ? 0.0f : mx - shift);
      move = __ballot(!(z <= limit)) != 0;
    }
    if (move) {
      float top = sc[0][0];
#pragma unroll
      for (int hv = 0; hv < HV; ++hv)
#pragma unroll
        for (int i = 0; i < 16; ++i) top = fmaxf(top, sc[hv][i]);
      top = fmaxf(top, __shfl_xor(top, 32));
      float m = fmaxf(mx, top * sc2);
      if (!coarse && __ballot(m > -INFINITY && !(fabsf(m) <= 1024.0f)) != 0) {
        coarse = true;
        mx /= sc2;                       // of at most 2^10: off by no more than 2^-13 when scaled
      }
      if (coarse) m = fmaxf(mx, top);
      const float f = m == -INFINITY ? 1.0f : exp2_fast(coarse ? (mx - m) * sc2 : mx - m);
      mx = m;
      sum *= f;
#pragma unroll
      for (int dt = 0; dt < ND; ++dt) o[dt] *= f;
      float base = m == -INFINITY ? 0.0f : m;
      if (coarse) {
#pragma unroll
        for (int hv = 0; hv < HV; ++hv) sc[hv] -= base;
        base = 0.0f;
      }
      z = weights(base - shift);
    }
    sum += z;
    // the weights are formed in this part, and not where they are next used
#pragma unroll
    for (int hv = 0; hv < HV; ++hv) asm volatile("" : "+v"(pw[hv][0]), "+v"(pw[hv][1]));
    __builtin_amdgcn_sched_barrier(0);
  };

  if (tid == 0) {
    spoilt = 0;
    tile = Tile{b, row0, n, total, r0, rows, 0};
  }
  if (steps == 0) __syncthreads();
  if (steps > 0) {
#pragma unroll
    for (int hv = 0; hv < HV; ++hv) {
      b0[hv] = block_of(0, hv, raw_page(0, hv));
      b1[hv] = block_of(1, hv, raw_page(1, hv));
      b2[hv] = block_of(2, hv, raw_page(2, hv));
      raw[hv] = raw_page(3, hv);
    }
    load_k(b0);
    load_v(b0);
    store_k(0);
    // the values of "step -1" are read before any are written: zeros
#pragma unroll
    for (int hv = 0; hv < HV; ++hv)
#pragma unroll
      for (int j = 0; j < PER; ++j)
        if (mine(j)) vs[1][hv][vl[j]] = V8((T)0.0f);
    load_k(b1);
    __syncthreads();
    constexpr std::integral_constant<int, 0> even{};
    constexpr std::integral_constant<int, 1> odd{};
    int live[HV];
    const auto keep_live = [&] {
#pragma unroll
      for (int hv = 0; hv < HV; ++hv) live[hv] = b0[hv].live;
    };
    // an odd count of steps ends in one without keys
    if (NW == 4 || wave < NW / 2) {
      for (int p = 0; p < steps; p += 2) {
        matrix(even);
        keep_live();
        pass_on(p, even);
        vector(p, live);
        __syncthreads();
        matrix(odd);
        keep_live();
        pass_on(p + 1, odd);
        vector(p + 1, live);
        __syncthreads();
      }
    } else {
      for (int p = 0; p < steps; p += 2) {
        if (p > 0) vector(p - 1, live);
        keep_live();
        pass_on(p, even);
        matrix(even);
        __syncthreads();
        vector(p, live);
        keep_live();
        pass_on(p + 1, odd);
        matrix(odd);
        __syncthreads();
      }
      vector((steps + 1) / 2 * 2 - 1, live);
    }
    products(1);
  }

  const float z = sum + __shfl_xor(sum, 32), top = (coarse ? mx * sc2 : mx) - kTileShift<T>;
  // arguments and tile once more: kept through the loop, they would cost it registers
  const AttendArgs ar = args_again();
  const int tile_rows = __builtin_amdgcn_readfirstlane(tile.rows);
  const int r = wr0 + c32;
  bool no_number = false;                  // a result is none, though its row's sum is
  float zero = 0.0f;                       // NaN where a result is not finite
#pragma unroll
  for (int dt = 0; dt < ND; ++dt)
#pragma unroll
    for (int i = 0; i < 16; ++i) zero = fmaf(o[dt][i], 0.0f, zero);
  if (zero != 0.0f && z > 0.0f) {
#pragma unroll
    for (int dt = 0; dt < ND; ++dt)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        no_number |= o[dt][i] != o[dt][i];
        o[dt][i] = o[dt][i] != o[dt][i] ? 0.0f : o[dt][i];
      }
  }
  if (r < tile_rows) {
    const int rr = tile.r0 + r, ti = rr / ar.group, hh = rr - ti * ar.group;
    const int64_t orow = (int64_t)(tile.row0 + ti) * ar.hq + blockIdx.x % ar.heads * ar.group + hh;
    const int64_t pr = (int64_t)blockIdx.y * ar.tokens * ar.hq + orow;
    const float inv = z > 0.0f ? 1.0f / z : 0.0f;
#pragma unroll
    for (int dt = 0; dt < ND; ++dt)
#pragma unroll
      for (int i4 = 0; i4 < 4; ++i4) {
        const int dim = 32 * dt + 8 * i4 + 4 * half;
        if (dim >= ar.d) continue;
        if (ar.splits == 1) {
          alignas(8) T w[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) w[i] = (T)(z > 0.0f ? o[dt][4 * i4 + i] * inv : z);
          *reinterpret_cast<uint2*>((T*)ar.out + orow * ar.d + dim) = *reinterpret_cast<uint2*>(w);
        } else {
          f32x4 v;
#pragma unroll
          for (int i = 0; i < 4; ++i) v[i] = o[dt][4 * i4 + i];
          *reinterpret_cast<f32x4*>(ar.part_o + pr * ar.d + dim) = v;
        }
      }
    if (half == 0) {
      if (ar.splits == 1) {
        if (ar.lse) ar.lse[orow] = z > 0.0f ? (top + log2_fast(z)) * kLn2 : (z == 0.0f ? -INFINITY : z);
      } else {
        ar.part_ml[pr * 2] = top;
        ar.part_ml[pr * 2 + 1] = z;
      }
    }
  }
  no_number = __ballot(no_number && r < tile_rows) != 0;
  if (wr0 < tile_rows && (no_number || spoilt != 0))
    add_not_finite<T, false>(tile, wr0, min(wr0 + 32, tile_rows), no_number);
}

// Joins the partial results of the key ranges, in their order.  Ranges without a key of the row
// have a sum of 0 and are skipped: nothing was written for them.
template <typename T>
__device__ __forceinline__ void store_row4(const AttendArgs& a, int64_t orow, int dim, f32x4 acc,
                                           float z) {
  alignas(8) T w[4];
  const float inv = 1.0f / z;
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = (T)(z > 0.0f ? acc[i] * inv : z);
  *reinterpret_cast<uint2*>((T*)a.out + orow * a.d + dim) = *reinterpret_cast<uint2*>(w);
}
__device__ __forceinline__ void store_lse(const AttendArgs& a, int64_t orow, float mm, float z) {
  if (a.lse) a.lse[orow] = z > 0.0f ? (mm + log2_fast(z)) * kLn2 : (z == 0.0f ? -INFINITY : z);
}

// A range's weight, from its maximum and sum; 0 without a key, and -0 where the weight is too small
// for fp32: what is not finite there still reaches the row.
__device__ __forceinline__ float join_weight(float2 v, float mm) {
  const float f = v.y != 0.0f ? exp2_fast(v.x - mm) : 0.0f;   // mm is finite where one is not 0
  return f == 0.0f && v.y != 0.0f ? -0.0f : f;
}
__device__ __forceinline__ bool has_keys(float w) { return __float_as_uint(w) != 0; }

// up to 16 ranges: a wave a row, 4 dimensions a lane
template <typename T>
__global__ __launch_bounds__(256) void k_attend_join(AttendArgs a) {
  const int lane = threadIdx.x & 63;
  const int64_t orow = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int64_t nrows = a.tokens * a.hq;
  if (orow >= nrows) return;
  const float2* ml = reinterpret_cast<const float2*>(a.part_ml) + orow;
  const float2 v = lane < a.splits ? ml[lane * nrows] : make_float2(-INFINITY, 0.0f);
  float mm = v.x;
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) mm = fmaxf(mm, __shfl_xor(mm, o));
  mm = __shfl(mm, 0);
  const float f = join_weight(v, mm);
  float z = f * v.y;
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) z += __shfl_xor(z, o);
  z = __shfl(z, 0);
  f32x4 acc = {0, 0, 0, 0};
  const float* po = a.part_o + orow * a.d + min(lane * 4, a.d - 4);
  for (int c0 = 0; c0 < a.splits; c0 += 8) {       // eight loads in flight
    f32x4 o[8];
    float w[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      w[j] = c0 + j < a.splits ? __shfl(f, c0 + j) : 0.0f;
      o[j] = f32x4{0, 0, 0, 0};
      if (has_keys(w[j])) o[j] = *reinterpret_cast<const f32x4*>(po + (c0 + j) * nrows * a.d);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) acc += w[j] * o[j];
  }
  if (lane * 4 < a.d) store_row4<T>(a, orow, lane * 4, acc, z);
  if (lane == 0) store_lse(a, orow, mm, z);
}

// up to kMaxSplits ranges: a workgroup a row, every eighth (d <= 128) or fourth range a group of
// lanes, the groups' sums in order
template <typename T>
__global__ __launch_bounds__(256) void k_attend_join_many(AttendArgs a) {
  __shared__ float w[kMaxSplits], red[4][2];
  __shared__ f32x4 so[256];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t orow = blockIdx.x, nrows = a.tokens * a.hq;
  const float2* ml = reinterpret_cast<const float2*>(a.part_ml) + orow;
  const float2 v = tid < a.splits ? ml[tid * nrows] : make_float2(-INFINITY, 0.0f);
  float mm = v.x;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) mm = fmaxf(mm, __shfl_xor(mm, o));
  if (lane == 0) red[wave][0] = mm;
  __syncthreads();
  mm = fmaxf(fmaxf(red[0][0], red[1][0]), fmaxf(red[2][0], red[3][0]));
  const float f = join_weight(v, mm);
  if (tid < kMaxSplits) w[tid] = f;
  float z = f * v.y;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) z += __shfl_xor(z, o);
  if (lane == 0) red[wave][1] = z;
  __syncthreads();
  z = red[0][1] + red[1][1] + red[2][1] + red[3][1];
  const int width = a.d <= 128 ? 32 : 64, groups = 256 / width;
  const int at = tid % width * 4;
  const float* po = a.part_o + orow * a.d + min(at, a.d - 4);
  f32x4 acc = {0, 0, 0, 0};
  for (int c0 = tid / width; c0 < a.splits; c0 += 8 * groups) {
    f32x4 o[8];
    float f8[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int c = c0 + j * groups;
      f8[j] = c < a.splits ? w[c] : 0.0f;
      o[j] = f32x4{0, 0, 0, 0};
      if (has_keys(f8[j])) o[j] = *reinterpret_cast<const f32x4*>(po + c * nrows * a.d);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) acc += f8[j] * o[j];
  }
  so[tid] = acc;
  __syncthreads();
  if (tid >= width) return;
  for (int g = 1; g < groups; ++g) acc += so[g * width + tid];
  if (at < a.d) store_row4<T>(a, orow, at, acc, z);
  if (tid == 0) store_lse(a, orow, mm, z);
}

// ---------------------------------------------------------------- host
int check_seqs(const gmm_kv_cache* c, const gmm_kv_batch* s, int64_t tokens, Seqs* o) {
  if (!s || !s->cu || !s->total || !s->pages) return GMM_ERR_INVALID_ARG;
  if (s->batch < 1 || s->max_pages < 1 || s->pages_stride < s->max_pages || tokens < 0)
    return GMM_ERR_INVALID_ARG;
  // slots, and those of steps past the last, are 32-bit; rows (tokens x heads) too
  if ((int64_t)s->max_pages * c->page > (1 << 30) || tokens > (1 << 24) || s->batch > (1 << 20))
    return GMM_ERR_UNSUPPORTED;
  *o = Seqs{(Table)(uintptr_t)s->cu, (Table)(uintptr_t)s->total, (Table)(uintptr_t)s->pages,
            s->pages_stride, s->batch, s->max_pages, log2i(c->page),
            c->pages};
  return GMM_OK;
}

int check_heads(const gmm_kv_cache* c, int32_t hq) {
  if (hq < 1 || hq % c->heads) return GMM_ERR_INVALID_ARG;
  if (hq > GMM_KV_MAX_HEADS || hq / c->heads > GMM_KV_MAX_GROUP) return GMM_ERR_UNSUPPORTED;
  return GMM_OK;
}

int64_t ws_need(const gmm_kv_cache* c, int64_t tokens, int hq, int32_t batch, int32_t max_pages) {
  return kv::ws_need(c->heads, c->page, c->d, tokens, hq, batch, max_pages, GMM_KV_MAX_KEEP);
}

template <typename T>
void launch_append(const AppendArgs& a, bool vec, bool inter, int64_t blocks, hipStream_t st) {
  const dim3 grid((unsigned)blocks);
  if (vec && inter) hipLaunchKernelGGL((k_kv_append<T, 8, true>), grid, dim3(256), 0, st, a);
  else if (vec) hipLaunchKernelGGL((k_kv_append<T, 8, false>), grid, dim3(256), 0, st, a);
  else if (inter) hipLaunchKernelGGL((k_kv_append<T, 1, true>), grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL((k_kv_append<T, 1, false>), grid, dim3(256), 0, st, a);
}

template <typename T, int NS, int RT>
void launch_few(const AttendArgs& a, const Plan& p, hipStream_t st) {
  const dim3 grid((unsigned)(p.items * a.heads), (unsigned)p.splits);
  const auto run = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, dim3(64 * p.waves), 0, st, a);
  };
  if constexpr (RT == 1 && NS <= 4) {
    if (p.waves == 8) {
      if (a.sel) run(k_attend_few<T, NS, RT, true, 8>);
      else run(k_attend_few<T, NS, RT, false, 8>);
      return;
    }
  }
  if (a.sel) run(k_attend_few<T, NS, RT, true, 4>);
  else run(k_attend_few<T, NS, RT, false, 4>);
}

template <typename T, int NS>
void launch_few_rt(const AttendArgs& a, const Plan& p, hipStream_t st) {
  if (p.rt == 1) launch_few<T, NS, 1>(a, p, st);
  else if (p.rt == 2) launch_few<T, NS, 2>(a, p, st);
  else if constexpr (NS <= 4) launch_few<T, NS, 4>(a, p, st);
}

template <typename T, int ND>
void launch_tile(const AttendArgs& a, const Plan& p, hipStream_t st) {
  const dim3 grid((unsigned)(p.items * a.heads), (unsigned)p.splits);
  if constexpr (ND == 3 || ND == 4) {
    if (p.rows == 256) {
      hipLaunchKernelGGL((k_attend_tile<T, ND, 8>), grid, dim3(512), 0, st, a);
      return;
    }
  }
  hipLaunchKernelGGL((k_attend_tile<T, ND, 4>), grid, dim3(256), 0, st, a);
}

template <typename T>
void launch_attend(const AttendArgs& a, const Plan& p, hipStream_t st) {
  if (p.rows > 0) {
    if (a.d <= 64) launch_tile<T, 2>(a, p, st);
    else if (a.d <= 96) launch_tile<T, 3>(a, p, st);
    else if (a.d <= 128) launch_tile<T, 4>(a, p, st);
    else if (a.d <= 192) launch_tile<T, 6>(a, p, st);
    else launch_tile<T, 8>(a, p, st);
  } else if (a.d <= 64) launch_few_rt<T, 2>(a, p, st);
  else if (a.d <= 128) launch_few_rt<T, 4>(a, p, st);
  else if (a.d <= 192) launch_few_rt<T, 6>(a, p, st);
  else launch_few_rt<T, 8>(a, p, st);
  if (a.splits > 1) {
    if (a.splits > 16)
      hipLaunchKernelGGL((k_attend_join_many<T>), dim3((unsigned)(a.tokens * a.hq)), dim3(256), 0,
                         st, a);
    else
      hipLaunchKernelGGL((k_attend_join<T>), dim3((unsigned)cdiv(a.tokens * a.hq, 4)),
                         dim3(256), 0, st, a);
  }
}

template <typename T>
int launch_rope(const void* x, int64_t xt, int64_t xh, void* out, int64_t ot, int64_t oh,
                int64_t tokens, int heads, int d, const int32_t* pos, const RopeShape& r, bool inter,
                hipStream_t st) {
  const bool vec = r.rot % 16 == 0 && d % 16 == 0 && aligned16(x) && aligned16(out) &&
                   aligned16(r.table) && (xt | xh | ot | oh) % 8 == 0;
  const int w = vec ? 8 : 1;
  const int64_t items = tokens * heads * cdiv(d, 2 * w), blocks = cdiv(items, 256);
  if (blocks > kMaxBlocks) return GMM_ERR_UNSUPPORTED;
  const auto run = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(256), 0, st, (const T*)x, xt, xh,
                       (T*)out, ot, oh, (uint32_t)items, heads, d, pos, r);
  };
  if (vec && inter) run(k_rope<T, 8, true>);
  else if (vec) run(k_rope<T, 8, false>);
  else if (inter) run(k_rope<T, 1, true>);
  else run(k_rope<T, 1, false>);
  return launch_status();
}

}  // namespace

extern "C" {

int gmm_rope_table(const double* freq, int32_t half, double scale, int32_t positions,
                   float* table, hipStream_t stream) {
  if (!freq || !table || half < 1 || positions < 1 || !isfinite(scale)) return GMM_ERR_INVALID_ARG;
  const int64_t blocks = cdiv((int64_t)positions * half, 256);
  if (half > GMM_MAX_D / 2 || blocks > kMaxBlocks) return GMM_ERR_UNSUPPORTED;
  hipLaunchKernelGGL(k_rope_table, dim3((unsigned)blocks), dim3(256), 0, stream, freq, half,
                     scale, (int64_t)positions, table);
  return launch_status();
}

int gmm_rope(const void* x, int64_t x_token_stride, int64_t x_head_stride, void* out,
             int64_t out_token_stride, int64_t out_head_stride, int64_t tokens, int32_t heads,
             int32_t d, int32_t dtype, const int32_t* pos, const float* table, int32_t positions,
             int32_t rot, int32_t interleaved, int32_t inverse, hipStream_t stream) {
  if (tokens < 0 || heads < 1 || d < 2 || positions < 1 || rot < 2 || rot > d || rot % 2)
    return GMM_ERR_INVALID_ARG;
  if (dtype != GMM_F32 && dtype != GMM_BF16 && dtype != GMM_F16) return GMM_ERR_UNSUPPORTED;
  if (d > GMM_MAX_D || heads > GMM_KV_MAX_HEADS || tokens > (1 << 24)) return GMM_ERR_UNSUPPORTED;
  if (tokens == 0) return GMM_OK;
  if (!x || !out || !pos || !table) return GMM_ERR_INVALID_ARG;
  const RopeShape r{table, positions, rot, inverse != 0};
  if (dtype == GMM_F32)
    return launch_rope<float>(x, x_token_stride, x_head_stride, out, out_token_stride,
                              out_head_stride, tokens, heads, d, pos, r, interleaved != 0,
                               stream);
  if (dtype == GMM_BF16)
    return launch_rope<__bf16>(x, x_token_stride, x_head_stride, out, out_token_stride,
                               out_head_stride, tokens, heads, d, pos, r, interleaved != 0,
                               stream);
  return launch_rope<_Float16>(x, x_token_stride, x_head_stride, out, out_token_stride,
                               out_head_stride, tokens, heads, d, pos, r, interleaved != 0,
                               stream);
}

int gmm_kv_append(const gmm_kv_cache* cache, const gmm_kv_batch* seqs, int64_t tokens,
                  const void* k, int64_t k_token_stride, int64_t k_head_stride, const void* v,
                  int64_t v_token_stride, int64_t v_head_stride, const int32_t* pos,
                  const float* table, int32_t positions, int32_t rot, int32_t interleaved,
                  const void* q, int64_t q_token_stride, int64_t q_head_stride, void* q_out,
                  int64_t qo_token_stride, int64_t qo_head_stride, int32_t hq,
                  hipStream_t stream) {
  int rc = check_cache(cache);
  if (rc != GMM_OK) return rc;
  AppendArgs a{};
  rc = check_seqs(cache, seqs, tokens, &a.s);
  if (rc != GMM_OK) return rc;
  const int d = cache->d;
  if (table && (positions < 1 || rot < 2 || rot > d || rot % 2)) return GMM_ERR_INVALID_ARG;
  if (q) {
    if (!table || !q_out) return GMM_ERR_INVALID_ARG;
    rc = check_heads(cache, hq);
    if (rc != GMM_OK) return rc;
  }
  if (tokens == 0) return GMM_OK;
  if (!k || !v) return GMM_ERR_INVALID_ARG;
  a.ck = cache->k;
  a.cv = cache->v;
  a.box = cache->box;
  a.box_scale = cache->box_scale;
  a.heads = cache->heads;
  a.page = cache->page;
  a.d = d;
  a.k = k;
  a.kt = k_token_stride;
  a.kh = k_head_stride;
  a.v = v;
  a.vt = v_token_stride;
  a.vh = v_head_stride;
  a.v_vec = aligned16(v) && (v_token_stride | v_head_stride) % 8 == 0;
  a.pos = pos;
  a.rope = RopeShape{table, table ? positions : 0, table ? rot : 0, 0};
  a.q = q;
  a.qt = q_token_stride;
  a.qh = q_head_stride;
  a.qo = q_out;
  a.qot = qo_token_stride;
  a.qoh = qo_head_stride;
  a.hq = q ? hq : 0;
  // 16-byte accesses where the rotated width, strides and addresses allow them, else single
  // pairs
  const bool vec = a.rope.rot % 16 == 0 && aligned16(k) &&
                   (k_token_stride | k_head_stride) % 8 == 0 && aligned16(table) &&
                   (!q || (aligned16(q) && aligned16(q_out) &&
                           (q_token_stride | q_head_stride | qo_token_stride | qo_head_stride) % 8 == 0));
  const int w = vec ? 8 : 1;
  const int64_t q_items = q ? tokens * hq * (d / (2 * w)) : 0;
  // a head's page has page * d / (8 w) units of keys: two for each of its threads
  const int size = cache->page * d;
  a.per = size >= 8192 ? 1 : size >= 4096 ? 2 : 4;
  while (a.per > 1 && 256 / a.per < d / (2 * w)) a.per /= 2;
  int64_t pages = tokens / cache->page + 2 * (int64_t)seqs->batch;
  if (pages > tokens) pages = tokens;
  a.page_blocks = pages * cdiv(cache->heads, a.per);
  const int64_t blocks = a.page_blocks + cdiv(q_items, 256);
  if (blocks > kMaxBlocks) return GMM_ERR_UNSUPPORTED;
  a.q_items = (uint32_t)q_items;
  const bool inter = table && interleaved;
  if (cache->dtype == GMM_BF16) launch_append<__bf16>(a, vec, inter, blocks, stream);
  else launch_append<_Float16>(a, vec, inter, blocks, stream);
  return launch_status();
}

size_t gmm_kv_workspace_bytes(const gmm_kv_cache* cache, int64_t tokens, int32_t hq,
                              int32_t batch, int32_t max_pages) {
  if (check_cache(cache) != GMM_OK || check_heads(cache, hq) != GMM_OK) return 0;
  if (tokens < 0 || tokens > (1 << 24) || batch < 1 || batch > (1 << 20) || max_pages < 1 ||
      (int64_t)max_pages * cache->page > (1 << 30))
    return 0;
  return (size_t)ws_need(cache, tokens, hq, batch, max_pages);
}

int gmm_kv_select(const gmm_kv_cache* cache, const gmm_kv_batch* seqs, int64_t tokens,
                  const void* q, int64_t q_token_stride, int64_t q_head_stride, int32_t hq,
                  int32_t m, int32_t keep_first, int32_t keep_last, int32_t* idx, void* ws,
                  size_t ws_bytes, hipStream_t stream) {
  int rc = check_cache(cache);
  if (rc != GMM_OK) return rc;
  SelectArgs a{};
  rc = check_seqs(cache, seqs, tokens, &a.s);
  if (rc != GMM_OK) return rc;
  rc = check_heads(cache, hq);
  if (rc != GMM_OK) return rc;
  if (!cache->box || m < 1 || keep_first < 0 || keep_last < 1) return GMM_ERR_INVALID_ARG;
  if (m > GMM_KV_MAX_KEEP || seqs->max_pages > GMM_KV_MAX_PAGES) return GMM_ERR_UNSUPPORTED;
  if ((int64_t)keep_first + keep_last > m) return GMM_ERR_INVALID_ARG;
  if (tokens == 0) return GMM_OK;
  if (!q || !idx) return GMM_ERR_INVALID_ARG;
  rc = check_kv_ws(ws, ws_bytes, ws_need(cache, tokens, hq, seqs->batch, seqs->max_pages));
  if (rc != GMM_OK) return rc;
  a.box = cache->box;
  a.box_scale = cache->box_scale;
  a.q = q;
  a.qt = q_token_stride;
  a.qh = q_head_stride;
  a.q_vec = aligned16(q) && (q_token_stride | q_head_stride) % 8 == 0;
  a.heads = cache->heads;
  a.group = hq / cache->heads;
  a.d = cache->d;
  a.col_shift = a.group >= 16 ? 4 : log2i(a.group);
  a.col_tiles = (int)cdiv(a.group, 16);
  a.score = (float*)ws;
  a.row = score_row(seqs->max_pages);
  const int per = 16 >> a.col_shift;
  const int64_t items = tokens / per + seqs->batch;
  // about four workgroups a CU: what a workgroup does first takes as long as a round of pages
  const int64_t parts = cdiv(seqs->max_pages, 256);
  const int64_t rounds = cdiv(parts * items * cache->heads, 4 * kCUs);
  a.rounds = (int)(rounds < 1 ? 1 : rounds > 8 ? 8 : rounds);
  a.parts = (int)cdiv(parts, a.rounds);
  const int64_t blocks = a.parts * items * cache->heads, rows = tokens * cache->heads;
  // a row's workgroup has up to 1024 threads
  if (blocks > kMaxBlocks || rows > kMaxBlocks / 4) return GMM_ERR_UNSUPPORTED;
  const size_t lds = (size_t)a.col_tiles * 16 * (2 * a.d + 16 + 4);
  const auto run_score = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(256), lds, stream, a);
  };
  const bool bf = cache->dtype == GMM_BF16;
  if (a.d <= 64) bf ? run_score(k_select_score<__bf16, 2>) : run_score(k_select_score<_Float16, 2>);
  else if (a.d <= 128) bf ? run_score(k_select_score<__bf16, 4>) : run_score(k_select_score<_Float16, 4>);
  else bf ? run_score(k_select_score<__bf16, 8>) : run_score(k_select_score<_Float16, 8>);
  const auto run_top = [&](auto kernel, int threads) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)rows), dim3(threads), 0, stream, a.s, a.score,
                       a.row, a.heads, m, keep_first, keep_last, idx);
  };
  if (seqs->max_pages <= 512) run_top(k_select_top<64, 8>, 64);
  else if (seqs->max_pages <= 2048) run_top(k_select_top<256, 8>, 256);
  else if (seqs->max_pages <= 16384) run_top(k_select_top<1024, 16>, 1024);
  else run_top(k_select_top<1024, 64>, 1024);
  return launch_status();
}

int gmm_kv_attend(const gmm_kv_cache* cache, const gmm_kv_batch* seqs, int64_t tokens,
                  const void* q, int64_t q_token_stride, int64_t q_head_stride, int32_t hq,
                  float scale, int32_t window, const int32_t* sel, int32_t m, void* out,
                  float* lse, void* ws, size_t ws_bytes, hipStream_t stream) {
  int rc = check_cache(cache);
  if (rc != GMM_OK) return rc;
  AttendArgs a{};
  rc = check_seqs(cache, seqs, tokens, &a.s);
  if (rc != GMM_OK) return rc;
  rc = check_heads(cache, hq);
  if (rc != GMM_OK) return rc;
  if (!isfinite(scale) || window < 0 || (sel ? m < 1 || window != 0 : m != 0))
    return GMM_ERR_INVALID_ARG;
  if (m > GMM_KV_MAX_KEEP) return GMM_ERR_UNSUPPORTED;
  if (tokens == 0) return GMM_OK;
  if (!q || !out || ((uintptr_t)out & 7)) return GMM_ERR_INVALID_ARG;
  const int group = hq / cache->heads;
  const Plan p = sel ? plan_sel(cache->heads, cache->page, cache->d, tokens, group, m)
                     : plan_dense(cache->heads, cache->page, cache->d, tokens, seqs->batch, group,
                                  seqs->max_pages);
  // the documented size, and, whatever that is, what this launch writes
  int64_t need = ws_need(cache, tokens, hq, seqs->batch, seqs->max_pages);
  const int64_t own = part_bytes(tokens, hq, cache->d, p.splits);
  if (own > need) need = own;
  rc = check_kv_ws(ws, ws_bytes, need);
  if (rc != GMM_OK) return rc;
  a.k = cache->k;
  a.v = cache->v;
  a.heads = cache->heads;
  a.group = group;
  a.d = cache->d;
  a.q = q;
  a.qt = q_token_stride;
  a.qh = q_head_stride;
  a.q_vec = aligned16(q) && (q_token_stride | q_head_stride) % 8 == 0;
  a.scale2 = scale * kLog2e;
  a.window = window;
  a.sel = sel;
  a.m = m;
  a.out = out;
  a.lse = lse;
  a.hq = hq;
  a.tokens = tokens;
  a.chunk = p.chunk;
  a.splits = p.splits;
  a.tiles_token = p.tiles_token;
  a.part_o = (float*)ws;
  a.part_ml = a.part_o + (int64_t)p.splits * tokens * hq * a.d;
  if (plan_threads(p, a.heads) > kMaxThreads || p.splits > 65535 || tokens * hq > kMaxBlocks)
    return GMM_ERR_UNSUPPORTED;
  if (cache->dtype == GMM_BF16) launch_attend<__bf16>(a, p, stream);
  else launch_attend<_Float16>(a, p, stream);
  return launch_status();
}

}  // extern "C"
