// Beam search's selection over beams and vocabulary for AMD Instinct MI355X (gfx950).
//
// A beam's words are scored by the log-softmax of its logits, l = s + (a x - log Z), log Z the
// log-sum-exp over the words, and the m largest w l over all beams of a sequence are taken, ties
// to the lower (beam, word).  The logits are read once: a wave takes a run of kRun words and
// leaves their maximum and the sum of exponentials relative to it.  log Z joins a beam's runs.
// Then the m best words lie in the m runs with the largest (w l of the maximum, lower run first):
// any word of another run comes after the m maxima of those.  Only they are read again.
//
// w l grows with x within a beam (a, w > 0; roundings keep the order), so a run's maximum of x is
// its maximum of w l, also after rounding.  Scores are compared in fp64.

#include <hip/hip_runtime.h>

#include <float.h>
#include <limits.h>
#include <math.h>
#include <stdint.h>

#include "flashgmm.h"
#include "kv_host.h"
#include "kv_plan.h"

namespace {

using namespace kv;

constexpr double kLog2eD = 1.4426950408889634;
constexpr double kLn2D = 0.6931471805599453;
constexpr int kRun = 2048;        // words of a run

struct BeamArgs {
  const void* x;
  int64_t seq_stride, beam_stride;
  const float* score;
  const float* weight;        // or null
  const uint8_t* done;        // or null
  const uint32_t* mask;       // or null
  int64_t mask_stride;
  double scale;
  float c;                    // scale log2(e)
  float above_c;              // the power of 2 above it
  int beams, vocab, runs, m, eos, rows;
  float2* part;               // [rows, runs]: maximum, sum
  float* out_score;
  int32_t* out_parent;
  int32_t* out_token;
  uint8_t* out_done;
};

__device__ __forceinline__ bool finite(float v) { return fabsf(v) < INFINITY; }

// A lane's value from another lane of the wave, by the data path of the vector instructions; lanes
// without a source get `old`.  The steps below join 2, 4, 8, 16 lanes (row_shr), rows of 16
// (row_bcast:15) and halves (row_bcast:31); lane 63 holds the result.
template <int kCtrl>
__device__ __forceinline__ uint32_t dpp(uint32_t old, uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp((int)old, (int)v, kCtrl, 0xf, 0xf, false);
}
template <typename Op>
__device__ __forceinline__ uint32_t wave_join(uint32_t v, uint32_t none, Op op) {
  v = op(v, dpp<0x111>(none, v));
  v = op(v, dpp<0x112>(none, v));
  v = op(v, dpp<0x114>(none, v));
  v = op(v, dpp<0x118>(none, v));
  v = op(v, dpp<0x142>(none, v));
  v = op(v, dpp<0x143>(none, v));
  return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
  return wave_join(v, 0u, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
}
__device__ __forceinline__ uint32_t bits_of(float v) { return __builtin_bit_cast(uint32_t, v); }
__device__ __forceinline__ float float_of(uint32_t v) { return __builtin_bit_cast(float, v); }
__device__ __forceinline__ float wave_max(float v) {
  return float_of(wave_join(bits_of(v), bits_of(-INFINITY), [](uint32_t a, uint32_t b) {
    return bits_of(fmaxf(float_of(a), float_of(b)));
  }));
}
__device__ __forceinline__ float wave_sum(float v) {
  return float_of(wave_join(bits_of(v), 0u, [](uint32_t a, uint32_t b) {
    return bits_of(float_of(a) + float_of(b));
  }));
}
// lane `i`'s value, of a lane that is the same for the wave
__device__ __forceinline__ uint64_t lane_value(uint64_t v, int i) {
  return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), i) << 32 |
         (uint32_t)__builtin_amdgcn_readlane((int)v, i);
}
template <int kCtrl>
__device__ __forceinline__ double add_from(double v) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  return v + __builtin_bit_cast(double, (uint64_t)dpp<kCtrl>(0, (uint32_t)(u >> 32)) << 32 |
                                            dpp<kCtrl>(0, (uint32_t)u));
}
__device__ __forceinline__ double wave_sum(double v) {
  v = add_from<0x111>(v);
  v = add_from<0x112>(v);
  v = add_from<0x114>(v);
  v = add_from<0x118>(v);
  v = add_from<0x142>(v);
  v = add_from<0x143>(v);
  return __builtin_bit_cast(double, lane_value(__builtin_bit_cast(uint64_t, v), 63));
}
// sum over the lanes up to this one
__device__ __forceinline__ int lanes_sum(int v) {
  v += (int)dpp<0x111>(0, v);
  v += (int)dpp<0x112>(0, v);
  v += (int)dpp<0x114>(0, v);
  v += (int)dpp<0x118>(0, v);
  // rows of 16 lanes: the sum of the first and of the third to the next, that of the first half
  // to the second
  v += (int)__builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);
  v += (int)__builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);
  return v;
}
// What lanes of the wave wrote to LDS is read by others after it: in order, without a barrier.
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}
// the lane's bit
__device__ __forceinline__ int from_mask(uint64_t mask) {
  return (int)(mask >> (threadIdx.x & 63) & 1);
}
// set bits of the lanes before
__device__ __forceinline__ int below(uint64_t bits) {
  return __builtin_amdgcn_mbcnt_hi((uint32_t)(bits >> 32),
                                   __builtin_amdgcn_mbcnt_lo((uint32_t)bits, 0));
}

// A word's logit in fp32.  (By its bits, of bf16: the compiler would take maxima in bf16, rounding each.)
__device__ __forceinline__ float logit(float x) { return x; }
__device__ __forceinline__ float logit(_Float16 x) { return (float)x; }
__device__ __forceinline__ float logit(__bf16 x) {
  return float_of((uint32_t)__builtin_bit_cast(uint16_t, x) << 16);
}

// 16 bytes of words: at an address that is a multiple of an element only, past the vocabulary
// -inf, and -inf where the mask forbids
template <typename T>
struct Words {
  static constexpr int N = 16 / sizeof(T);
  typedef T V __attribute__((ext_vector_type(N)));
  typedef V Unaligned __attribute__((aligned(sizeof(T))));
  static constexpr int kSteps = kRun / (64 * N);       // of a run

  __device__ __forceinline__ static int at(int run, int step) {
    return run * kRun + (step * 64 + (int)(threadIdx.x & 63)) * N;
  }
  V v[kSteps];
  uint32_t bits[kSteps];

  // Issues the loads of a run.
  __device__ __forceinline__ void fetch(const BeamArgs& a, const T* x, const uint32_t* mask, int run) {
    if (mask) {
#pragma unroll
      for (int i = 0; i < kSteps; ++i) bits[i] = mask[min(at(run, i), a.vocab - 1) >> 5];
    }
    if ((run + 1) * kRun <= a.vocab) {
#pragma unroll
      for (int i = 0; i < kSteps; ++i)
        v[i] = __builtin_nontemporal_load(reinterpret_cast<const Unaligned*>(x + at(run, i)));
    } else {
#pragma unroll
      for (int i = 0; i < kSteps; ++i) {
        const int p = at(run, i);
#pragma unroll
        for (int e = 0; e < N; ++e) v[i][e] = (T)-INFINITY;
        if (p + N <= a.vocab) v[i] = *reinterpret_cast<const Unaligned*>(x + p);
      }
    }
  }
  // The words of an incomplete vector, and those that are forbidden.
  __device__ __forceinline__ void finish(const BeamArgs& a, const T* x, const uint32_t* mask, int run) {
    const int last = a.vocab & -N;
    if (last < a.vocab && last / kRun == run) {
      V t;
#pragma unroll
      for (int e = 0; e < N; ++e) {
        t[e] = (T)-INFINITY;
        if (last + e < a.vocab) t[e] = x[last + e];
      }
#pragma unroll
      for (int i = 0; i < kSteps; ++i)
        if (at(run, i) == last) v[i] = t;
    }
    if (!mask) return;
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      const uint32_t b = bits[i] >> (at(run, i) & 31);
#pragma unroll
      for (int e = 0; e < N; ++e) v[i][e] = b >> e & 1 ? v[i][e] : (T)-INFINITY;
    }
  }
};

template <typename T>
__device__ __forceinline__ const T* row_of(const BeamArgs& a, int row) {
  const int b = (uint32_t)row / (uint32_t)a.beams;
  return (const T*)a.x + b * a.seq_stride + (row - b * a.beams) * a.beam_stride;
}
__device__ __forceinline__ const uint32_t* mask_of(const BeamArgs& a, int row) {
  return a.mask ? a.mask + row * a.mask_stride : nullptr;
}

// The power of 2 to which a run's sum is relative, by its largest logit: its exponent, rounded to a
// whole number, so that joining runs does not round.  The product in fp32 is off by up to 32 below 2^30,
// which the sum carries.  From there on (`large`) more than that, and the sum is relative to the logit
// itself: the next smaller one is 2^-24 of it below, an exponent of -64, and its weight does not count.
__device__ __forceinline__ bool large(const BeamArgs& a, float x) { return !(fabsf(x * a.c) < 0x1p30f); }
__device__ __forceinline__ double unit_of(const BeamArgs& a, float x) {
  return large(a, x) ? (double)x * (double)a.c : (double)rintf(x * a.c);
}

// A wave a run: its maximum and sum of exponentials.  A NaN or +infinity makes the sum NaN.
//
// Bound by bytes: 61 us for 64 x 16 beams of 131,072 fp32 words, a fifth of them finished (7.0 TB/s);
// 32 x 8 of bf16 words 13.3 us (5.0 TB/s; the vector unit needs about 7).  Many short waves in the
// order of the addresses read faster than waves of eight runs with the next under way (81 us), loads
// past the caches faster than others (71).
template <typename T>
__global__ __launch_bounds__(256) void k_beam_run(BeamArgs a) {
  const int lane = threadIdx.x & 63;
  const int item = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
  const int row = (uint32_t)item / (uint32_t)a.runs, run = item - row * a.runs;
  if (row >= a.rows) return;
  const float score = a.score[row];
  const int done = a.done ? a.done[row] : 0;       // both loads together
  if (!finite(score) | (done != 0)) return;
  typedef Words<T> W;
  const T* x = row_of<T>(a, row);
  const uint32_t* mask = mask_of(a, row);
  W words;
  words.fetch(a, x, mask, run);
  words.finish(a, x, mask, run);
  float mx = -INFINITY;
#pragma unroll
  for (int i = 0; i < W::kSteps; ++i)
#pragma unroll
    for (int e = 0; e < W::N; ++e) mx = fmaxf(mx, (float)words.v[i][e]);
  mx = wave_max(mx);
  // Exponents by one multiply-add, whose product is not rounded.  Of large logits those below the
  // maximum need only be far from 0: a power of 2 leaves the maximum's product exact, that above
  // the factor or, where products could pass the type's range (differences of 2^75 and more), 2^-64.
  const bool far = large(a, mx);
  const float c = !far ? a.c : fabsf(mx) < 0x1p100f ? a.above_c : 0x1p-64f;
  const float unit = !(mx > -INFINITY) ? 0.f : far ? mx * c : rintf(mx * c);
  float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < W::kSteps; ++i)
#pragma unroll
    for (int e = 0; e < W::N; ++e)
      sum[e & 3] += __builtin_amdgcn_exp2f(fmaf((float)words.v[i][e], c, -unit));
  const float z = wave_sum((sum[0] + sum[1]) + (sum[2] + sum[3]));
  if (lane == 0) a.part[(int64_t)row * a.runs + run] = make_float2(mx, z);
}

// ---------------------------------------------------------------- the best of many
// Scores as whole numbers of the same order; 0 is no candidate.
__device__ __forceinline__ uint64_t ordered(double v) {
  const int64_t u = __builtin_bit_cast(int64_t, v + 0.0);      // -0 is 0
  return (uint64_t)(u ^ (u >> 63 | INT64_MIN));
}
__device__ __forceinline__ double value_of(uint64_t k) {
  const int64_t u = (int64_t)k;
  return __builtin_bit_cast(double, u < 0 ? u ^ INT64_MIN : ~u);
}

// What pick() takes of the numbers given to it: those above `least`, and the first `ties` equal to it.
struct Picked {
  uint64_t least;
  int ties, count;
  // a number that comes later, behind these in order, is among the best only from here on
  __device__ __forceinline__ uint64_t floor() const { return least + (ties != INT_MAX); }
};

// The m largest of the numbers in v (64 a step; 0 is none), ties to the first in the order of
// steps and lanes: the threshold is built bit by bit from the first bit in which the numbers
// differ, until m numbers reach it.  Some ten rounds for scores.  Equal numbers (logits of 8
// bits, say) never give m: every few rounds one of those still in question is tried.
template <int C>
__device__ __forceinline__ Picked pick(const uint64_t* v, int m) {
  const auto reach = [&](uint64_t t) {
    int n = 0;
#pragma unroll
    for (int c = 0; c < C; ++c) n += __popcll(__ballot(v[c] >= t));
    return n;
  };
  int n = reach(1);
  if (n <= m) return Picked{1, INT_MAX, n};
  uint32_t hi = 0, lo = 0;             // of the upper halves: the largest, the smallest's complement
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const uint32_t h = (uint32_t)(v[c] >> 32);
    hi = max(hi, h);
    lo = max(lo, v[c] ? ~h : 0u);
  }
  hi = wave_max(hi);
  lo = ~wave_max(lo);
  // bits above the first that differs are those of every number
  uint32_t diff = hi ^ lo;
  uint64_t t = (uint64_t)hi << 32, step = (uint64_t)1 << 32;        // the bit above the next one to try
  if (diff) {
    const int top = 31 - __builtin_clz(diff);
    t = top == 31 ? 0 : (uint64_t)(hi >> (top + 1) << (top + 1)) << 32;
    step <<= top;                                    // the first to try
  } else {
    step >>= 1;
  }
  for (int rounds = 10; step; rounds = 5) {
    do {
      const uint64_t up = t | step;
      step >>= 1;
      n = reach(up);
      t = n >= m ? up : t;
    } while (n != m && step && --rounds);
    if (n == m) return Picked{t, INT_MAX, m};
    uint64_t probe = 0;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const uint64_t in = __ballot(v[c] >= t && v[c] - t < 2 * step);
      if (probe == 0 && in) probe = lane_value(v[c], __builtin_ctzll(in));
    }
    const int more = reach(probe + 1);
    if (probe && more < m && reach(probe) >= m) return Picked{probe, m - more, m};
  }
  return Picked{t, m - reach(t + 1), m};
}

// How many of a list of 64 numbers in LDS, of which v is number `lane`, are in front of it: larger, or
// equal and before.  Every lane reads the same addresses, eight numbers a step; those from n on
// are 0.
__device__ __forceinline__ int place_of(const uint64_t* list, uint64_t v, int n) {
  typedef uint64_t Two __attribute__((ext_vector_type(2)));
  int place = 0;
  for (int i = 0; i < n; i += 8) {
    Two t[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) t[k] = *reinterpret_cast<const Two*>(list + i + 2 * k);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const uint64_t u = t[k / 2][k % 2];
      place += from_mask(__ballot(u > v) | (__ballot(u >= v) & ~1ull << (i + k)));
    }
  }
  return place;
}
// How many of a list of 64 numbers below 2^31 are larger than v; those from n on are 0.  (By the sign of
// a difference: a comparison's result would pass through scalar registers, with a wait for each.)
__device__ __forceinline__ int larger_than(const uint32_t* list, uint32_t v, int n) {
  typedef uint32_t Four __attribute__((ext_vector_type(4)));
  int count = 0;
  for (int i = 0; i < n; i += 16) {
    Four t[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) t[k] = *reinterpret_cast<const Four*>(list + i + 4 * k);
#pragma unroll
    for (int k = 0; k < 16; ++k) count += (v - t[k / 4][k % 4]) >> 31;
  }
  return count;
}

// Is v among what was picked?  `seen`: numbers equal to `least` in the steps before.
__device__ __forceinline__ bool taken(const Picked& p, uint64_t v, int* seen) {
  const uint64_t same = __ballot(v == p.least && v != 0);
  const bool in = v > p.least ||
                  (v == p.least && v != 0 && *seen + below(same) < p.ties);
  *seen += __popcll(same);
  return in;
}

constexpr int kChunk = 1024;           // runs looked at together
constexpr int kLane = 1 + kChunk / 64; // and the best before: of a lane, odd for the banks of LDS
constexpr int kBuffer = GMM_BEAM_MAX + 256;       // words that a wave holds

// A wave's words so far: score, and beam * vocab + word.
struct Found {
  uint64_t key[kBuffer];
  uint32_t at[kBuffer];
};

struct Join {
  double logz[GMM_BEAM_MAX];           // log sum exp(scale (x - top))
  double weight[GMM_BEAM_MAX];
  float top[GMM_BEAM_MAX];             // a beam's largest logit
  float score[GMM_BEAM_MAX];
  int kind[GMM_BEAM_MAX];              // 0: no candidate, 1: live, 2: finished
  // scores of the best runs so far, then of a chunk of runs; at the end, of the waves' words
  uint32_t hi[64 * kLane], lo[64 * kLane];
  uint32_t word[64 * 16];
  int run[64];                         // the best runs, in order
  alignas(16) uint64_t list[64];       // what few() leaves
  alignas(16) uint32_t tops[64];
  int list_at[64];
  uint64_t least;
  int kept;
};

template <int NW>
struct JoinOf : Join {
  int count[NW];
  Found found[NW];
};

// l of a live beam's logit, from its difference to the largest: products of large logits would
// cancel, and not alike everywhere (multiply and add may be fused)
__device__ __forceinline__ double total_of(const BeamArgs& a, const Join& s, int j, float x) {
  return (double)s.score[j] + fma(a.scale, (double)x - (double)s.top[j], -s.logz[j]);
}
__device__ __forceinline__ uint64_t key_of(const BeamArgs& a, const Join& s, int j, float x) {
  return x > -INFINITY ? ordered(s.weight[j] * total_of(a, s, j, x)) : 0;
}

// the score of a run's largest logit
__device__ __forceinline__ uint64_t run_key(const BeamArgs& a, const Join& s, int j, int run, float x) {
  if (s.kind[j] == 1) return key_of(a, s, j, x);
  // a finished beam has one run, that of its end word
  return s.kind[j] == 2 && run == a.eos / kRun ? ordered(s.weight[j] * (double)s.score[j]) : 0;
}

// A logit below which no word of beam j has the score `floor`: the logit of that score in fp32, less
// what its roundings may be (each of the four terms has a few units of 2^-24, of its size; 2^-150 of a
// product that has too few bits in fp32 is 2^-110 of l).  The smallest number, which -infinity does not
// reach, if there is none, and for weights whose reciprocal or product may be past the range of fp32.
__device__ __forceinline__ float logit_of(const BeamArgs& a, const Join& s, int j, uint64_t floor) {
  const float w = (float)s.weight[j];
  if (floor <= 1 || !(w >= 0x1p-40f && w <= 0x1p64f)) return -FLT_MAX;
  const float l = (float)value_of(floor) * __builtin_amdgcn_rcpf(w);
  const float z = (float)s.logz[j], inv = __builtin_amdgcn_rcpf((float)a.scale);
  const float x = s.top[j] + ((l - s.score[j]) + z) * inv;
  const float less = ((fabsf(l) + fabsf(s.score[j]) + fabsf(z)) * 0x1p-20f + 1e-30f) * inv +
                     fabsf(x) * 0x1p-20f;
  return x - less > -FLT_MAX ? x - less : -FLT_MAX;      // also for what is no number
}

// All runs of the sequence fit a chunk, those of a beam a wave: their scores are formed with log Z.
__device__ __forceinline__ bool one_chunk(const BeamArgs& a) {
  return a.runs <= 64 && a.beams * a.runs <= kChunk;
}
__device__ __forceinline__ void put_run(Join& s, int i, uint64_t key) {
  s.hi[i] = (uint32_t)(key >> 32);
  s.lo[i] = (uint32_t)key;
}

// log Z of up to two beams of a wave, j and j + NW: their loads go together
template <int NW>
__device__ __forceinline__ void join_beams(const BeamArgs& a, Join& s, int row0, int j0) {
  const int lane = threadIdx.x & 63;
  float sc[2], wt[2];
  int fin[2];
  float2 v[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int row = row0 + min(j0 + i * NW, a.beams - 1);
    sc[i] = a.score[row];
    wt[i] = a.weight ? a.weight[row] : 1.f;
    fin[i] = a.done ? a.done[row] : 0;
    v[i] = a.part[(int64_t)row * a.runs + min(lane, a.runs - 1)];
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int j = j0 + i * NW;
    if (j >= a.beams) break;
    int kind = finite(sc[i]) && wt[i] > 0.f && finite(wt[i]) ? fin[i] ? 2 : 1 : 0;
    double logz = 0.0;
    float mx = -INFINITY;
    if (kind == 1) {
      const float2* p = a.part + (int64_t)(row0 + j) * a.runs;
      float2 u = v[i];
      if (lane < a.runs) mx = u.x;
      for (int r = lane + 64; r < a.runs; r += 64) mx = fmaxf(mx, p[r].x);
      mx = wave_max(mx);
      double z = 0.0;
      const double unit = unit_of(a, mx);
      for (int r = lane; r < a.runs; r += 64) {
        if (r >= 64) u = p[r];
        // a run without a word adds its sum, 0, or NaN
        z += ldexp((double)u.y, u.x > -INFINITY ? (int)fmax(unit_of(a, u.x) - unit, -2000.0) : 0);
      }
      z = wave_sum(z);
      logz = log(z) + (large(a, mx) ? 0.0 : (unit - (double)a.c * (double)mx) * kLn2D);
      if (!finite(mx) || !(z > 0.0 && z < (double)INFINITY)) kind = 0;   // no word, NaN or +infinity
    }
    if (lane == 0) {
      s.logz[j] = logz;
      s.weight[j] = wt[i];
      s.top[j] = mx;
      s.score[j] = sc[i];
      s.kind[j] = kind;
    }
    wave_sync();                       // all of this is read by the other lanes
    if (one_chunk(a) && lane < a.runs) put_run(s, j * a.runs + lane, run_key(a, s, j, lane, v[i].x));
  }
}

// Those of a lane's numbers (bits of `more`, and of `same`, which equal the threshold) that were
// picked: of the equal ones the first `ties`, lane after lane.
__device__ __forceinline__ uint32_t taken(uint32_t more, uint32_t same, int ties) {
  const int n = __popc(same);
  int left = ties == INT_MAX ? n : ties - (lanes_sum(n) - n);
  for (int k = n; k > max(left, 0); --k) same &= ~(0x80000000u >> __builtin_clz(same));
  return more | same;
}

// Up to 64 of the first n numbers of s.hi / s.lo, the m largest among them, by one wave: the numbers into
// s.list, where they were into s.list_at, in order; returns how many.  First those that reach a
// threshold in their upper halves.  Few results: the m-th largest of the lanes' maxima, which are m
// of the numbers, found by counting (8 of 512: 1900 cycles; bit by bit 4500 where numbers are equal).
// Many: built bit by bit until m numbers reach it and 64 at most (64 of 480: 6900 cycles; 14,000 by
// maxima, as too many are left).
__device__ __forceinline__ int few(Join& s, int n, int m) {
  const int lane = threadIdx.x & 63;
  // as many of a lane as leave 6 m lanes: a lane's maximum is cheaper than its place
  const int per = max((n + 63) / 64, min(kLane, n / (6 * m))) | 1, first = lane * per;
  const auto has = [&](int c) { return c < per && first + c < n; };
  uint32_t h[kLane], hi = 0, more = 0, same = 0, least = 1;
#pragma unroll
  for (int c = 0; c < kLane; ++c) h[c] = s.hi[min(first, 63 * kLane) + c];
#pragma unroll
  for (int c = 0; c < kLane; ++c) {
    h[c] = has(c) ? h[c] : 0;
    hi = max(hi, h[c]);
  }
  if (m <= 16) {
    s.tops[lane] = hi >> 1;
    wave_sync();
    const int larger = larger_than(s.tops, hi >> 1, (n + per - 1) / per);
    // the smallest of those that fewer than m are larger than; a number is not 0 in this half
    least = max(~wave_max(larger < m ? ~(hi & ~1u) : 0u), 1u);
  } else if (n > 64) {
    uint32_t lo = 0;                   // the smallest's complement
#pragma unroll
    for (int c = 0; c < kLane; ++c) lo = max(lo, h[c] ? ~h[c] : 0u);
    hi = wave_max(hi);
    lo = ~wave_max(lo);
    uint32_t step = hi == lo ? 0 : 0x80000000u >> __builtin_clz(hi ^ lo);
    least = max(step ? hi & ~(2 * step - 1) : hi, 1u);
    while (step) {
      int k = 0;
#pragma unroll
      for (int c = 0; c < kLane; ++c) k += __popcll(__ballot(h[c] >= (least | step)));
      if (k >= m) least |= step;
      step = k >= m && k <= 64 ? 0 : step >> 1;
    }
  }
#pragma unroll
  for (int c = 0; c < kLane; ++c) more |= (uint32_t)(h[c] >= least) << c;
  int upto = lanes_sum(__popc(more)), all = __builtin_amdgcn_readlane(upto, 63);
  if (all > 64) {                      // many of one size
    uint64_t v[kLane];
#pragma unroll
    for (int c = 0; c < kLane; ++c) v[c] = has(c) ? (uint64_t)h[c] << 32 | s.lo[first + c] : 0;
    const Picked q = pick<kLane>(v, m);
    more = 0;
#pragma unroll
    for (int c = 0; c < kLane; ++c) {
      more |= (uint32_t)(v[c] > q.least) << c;
      same |= (uint32_t)(v[c] && v[c] == q.least) << c;
    }
    more = taken(more, same, q.ties);
    upto = lanes_sum(__popc(more));
    all = q.count;
  }
  s.list[lane] = 0;
  wave_sync();
  for (int at = upto - __popc(more); more; more &= more - 1) {
    const int i = first + __builtin_ctz(more);
    s.list[at] = (uint64_t)s.hi[i] << 32 | s.lo[i];
    s.list_at[at++] = i;
  }
  wave_sync();
  return all;
}

// The best of the first n of s.hi / s.lo (`kept` runs, then those from `base` on), by one wave.
__device__ __forceinline__ void pick_runs(const BeamArgs& a, Join& s, int base, int kept, int n) {
  const int lane = threadIdx.x & 63, all = few(s, n, a.m);
  const uint64_t key = s.list[lane];
  const int i = lane < all ? s.list_at[lane] : 0, run = i < kept ? s.run[i] : base + i - kept;
  const int place = place_of(s.list, key, all);
  const bool in = lane < all && place < a.m;
  const uint64_t bal = __ballot(in), last = __ballot(in && place == a.m - 1);
  wave_sync();
  if (in) {
    const int at = below(bal);
    s.hi[at] = (uint32_t)(key >> 32);
    s.lo[at] = (uint32_t)key;
    s.run[at] = run;
  }
  if (lane == 0) {
    s.kept = __popcll(bal);
    // the m-th run's score, 1 as long as there are fewer
    s.least = last ? lane_value(key, __builtin_ctzll(last)) : 1;
  }
}

// The m best runs of the sequence, in order, into s.run, their scores into s.hi / s.lo, their number
// into s.kept, and the m-th one's score into s.least.
template <int NW>
__device__ __forceinline__ void best_runs(const BeamArgs& a, Join& s, int row0) {
  const int tid = threadIdx.x;
  const int runs = a.beams * a.runs;
  const float inv = 1.f / (float)a.runs;
  const float2* part = a.part + (int64_t)row0 * a.runs;
  int kept = 0;
  uint64_t least = 1;
  for (int base = 0; base < runs; base += kChunk) {
    if (!one_chunk(a)) {
      bool any = false;
      for (int t = tid; t < min(kChunk, runs - base); t += 64 * NW) {
        const int i = base + t, j = (int)(((float)i + 0.5f) * inv);    // i / runs: exact below 2^21
        uint64_t k = run_key(a, s, j, i - j * a.runs, part[i].x);
        // an equal one is behind the m kept
        if (k < least || (kept == a.m && k == least)) k = 0;
        put_run(s, kept + t, k);
        any |= k != 0;
      }
      if (!__syncthreads_or(any) && base > 0) continue;
    }
    if (tid < 64) pick_runs(a, s, base, kept, kept + min(kChunk, runs - base));
    __syncthreads();
    kept = s.kept;
    least = s.least;
  }
}

// Leaves the m best of a wave's n words, in their order.
__device__ __forceinline__ Picked keep_words(Found& f, int n, int m) {
  constexpr int C = kBuffer / 64;
  const int lane = threadIdx.x & 63;
  wave_sync();
  uint64_t v[C];
  uint32_t at[C];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const bool in = c * 64 + lane < n;
    v[c] = in ? f.key[c * 64 + lane] : 0;
    at[c] = in ? f.at[c * 64 + lane] : 0;
  }
  const Picked p = pick<C>(v, m);
  int k = 0, seen = 0;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const bool in = taken(p, v[c], &seen);
    const uint64_t bal = __ballot(in);
    if (in) {
      f.key[k + below(bal)] = v[c];
      f.at[k + below(bal)] = at[c];
    }
    k += __popcll(bal);
  }
  wave_sync();
  return p;
}

// A workgroup of NW waves a sequence: log Z of its beams, its m best runs, their m best words.
//
// Bound by latency, of memory three times (runs, and their words twice as far) and of some 1500
// instructions of one wave: 8.6 us for 8 beams and 8 results, 13.0 for 16, 6.6 for 4.  Few
// instructions count here, so the m best are found by thresholds and counts: sorting networks of 64
// (key, index) pairs took 24 and 41 us.  What costs is the way of a comparison's result through
// scalar registers, hence signs of differences where the numbers allow it.
//
// Waves: as many as beams or results, 4, 8 or 16.  More find a part of the words each (16 beams: 14.6
// us in 8 waves, 13.0 in 16), fewer leave room for other sequences (1000 of 4 beams: whole call 19 us
// in 4 waves, 26 in 8, 44 in 16).
template <typename T, int NW>
__global__ __launch_bounds__(64 * NW, 4) void k_beam_join(BeamArgs a) {
  __shared__ JoinOf<NW> s;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row0 = blockIdx.x * a.beams;
  for (int j = w; j < a.beams; j += 2 * NW) join_beams<NW>(a, s, row0, j);
  __syncthreads();
  best_runs<NW>(a, s, row0);

  // the words that reach the m-th best run's maximum; a wave takes neighbouring runs, so that
  // the waves' words, one after the other, are in order
  typedef Words<T> W;
  Found& buf = s.found[w];
  uint64_t floor = s.least;
  int held = 0;
  const int q1 = (w + 1) * s.kept / NW;
  for (int q = w * s.kept / NW; q < q1; ++q) {
    const int gid = __builtin_amdgcn_readfirstlane(s.run[q]);
    const int j = gid / a.runs, r = gid - j * a.runs;
    W words;
    // parts of the run with words that may count: 256 neighbours, half of the lanes of 16-bit words
    constexpr int kHalves = W::N / 4;
    uint32_t parts = 0;
    float least = -INFINITY;
    if (s.kind[j] == 2) {
      parts = 1;
    } else {
      const T* x = row_of<T>(a, row0 + j);
      words.fetch(a, x, mask_of(a, row0 + j), r);
      words.finish(a, x, mask_of(a, row0 + j), r);
      least = logit_of(a, s, j, floor);
#pragma unroll
      for (int i = 0; i < W::kSteps; ++i) {
        float mx = logit(words.v[i][0]);
#pragma unroll
        for (int e = 1; e < W::N; ++e) mx = fmaxf(mx, logit(words.v[i][e]));
        const uint64_t bal = __ballot(mx >= least);
        if constexpr (kHalves == 2)
          parts |= (uint32_t)((uint32_t)bal != 0) << 2 * i | (uint32_t)(bal >> 32 != 0) << (2 * i + 1);
        else
          parts |= (uint32_t)(bal != 0) << i;
      }
    }
    while (parts) {
      const int part = __builtin_ctz(parts), i = part / kHalves;
      parts &= parts - 1;
      if (s.kind[j] == 2) {
        if (lane == 0) {
          buf.key[held] = (uint64_t)s.hi[q] << 32 | s.lo[q];
          buf.at[held] = (uint32_t)j * a.vocab + a.eos;
        }
        ++held;
      } else {
        typename W::V x = words.v[0];
#pragma unroll
        for (int c = 1; c < W::kSteps; ++c)
          if (c == i) x = words.v[c];
        // in the order of the words: those of the lanes before, then of this one.  What passes for
        // its logit but has not the score is held as none.
        uint32_t pass = 0;
#pragma unroll
        for (int e = 0; e < W::N; ++e) pass |= (uint32_t)(logit(x[e]) >= least) << e;
        if (kHalves == 2 && lane / 32 != part % kHalves) pass = 0;
        const int upto = lanes_sum(__popc(pass));
        for (int at = held + upto - __popc(pass); pass; pass &= pass - 1) {
          const int e = __builtin_ctz(pass);
          float y = logit(x[0]);
#pragma unroll
          for (int c = 1; c < W::N; ++c) y = c == e ? logit(x[c]) : y;
          const uint64_t key = key_of(a, s, j, y);
          buf.key[at] = key < floor ? 0 : key;
          buf.at[at++] = (uint32_t)j * a.vocab + W::at(r, i) + e;
        }
        held += __builtin_amdgcn_readlane(upto, 63);
      }
      if (held > GMM_BEAM_MAX) {
        const Picked p = keep_words(buf, held, a.m);
        held = p.count;
        if (held == a.m) floor = max(floor, p.floor());
      }
    }
  }
  if (lane == 0) s.count[w] = held;
  __syncthreads();

  // all waves' words, one after the other, and of them the best by one wave
  uint64_t key = 0;
  uint32_t word = 0;
  const int upto = lanes_sum(lane < NW ? s.count[lane] : 0);
  int total = __builtin_amdgcn_readlane(upto, NW - 1);
  if (total <= 64 || NW > 8) {
    if (lane < held) {
      const int at = __builtin_amdgcn_readlane(upto, w) - held + lane;
      s.hi[at] = (uint32_t)(buf.key[lane] >> 32);
      s.lo[at] = (uint32_t)buf.key[lane];
      s.word[at] = buf.at[lane];
    }
    __syncthreads();
    if (w != 0) return;
    if (total <= 64) {
      if (lane < total) {
        key = (uint64_t)s.hi[lane] << 32 | s.lo[lane];
        word = s.word[lane];
      }
    } else if constexpr (NW > 8) {
      total = few(s, total, a.m);
      key = s.list[lane];
      word = lane < total ? s.word[s.list_at[lane]] : 0;
    }
  } else if constexpr (NW <= 8) {
    if (w != 0) return;
    uint64_t v[NW];
    uint32_t all[NW];
#pragma unroll
    for (int c = 0; c < NW; ++c) {
      const bool in = lane < s.count[c];
      v[c] = in ? s.found[c].key[lane] : 0;
      all[c] = in ? s.found[c].at[lane] : 0;
    }
    const Picked p = pick<NW>(v, a.m);
    int k = 0, seen = 0;
#pragma unroll
    for (int c = 0; c < NW; ++c) {
      const bool in = taken(p, v[c], &seen);
      const uint64_t bal = __ballot(in);
      if (in) {
        buf.key[k + below(bal)] = v[c];
        buf.at[k + below(bal)] = all[c];
      }
      k += __popcll(bal);
    }
    total = p.count;
    wave_sync();
    if (lane < total) {
      key = buf.key[lane];
      word = buf.at[lane];
    }
  }
  s.list[lane] = key;
  wave_sync();
  const int place = place_of(s.list, key, total), found = __popcll(__ballot(key != 0));
  const int64_t o = (int64_t)blockIdx.x * a.m;
  if (key != 0 && place < a.m) {
    const int j = (int)(word / (uint32_t)a.vocab), v = (int)(word - (uint32_t)j * a.vocab);
    const bool fin = s.kind[j] == 2;
    // l from w l, whose rounding in 64 bits is far below that of the result
    a.out_score[o + place] = fin ? s.score[j] : (float)(value_of(key) / s.weight[j]);
    a.out_parent[o + place] = (int32_t)(row0 + j);
    a.out_token[o + place] = v;
    if (a.out_done) a.out_done[o + place] = fin || v == a.eos;
  }
  if (lane >= found && lane < a.m) {
    a.out_score[o + lane] = -INFINITY;
    a.out_parent[o + lane] = -1;
    a.out_token[o + lane] = -1;
    if (a.out_done) a.out_done[o + lane] = 0;
  }
}

// ---------------------------------------------------------------- host
bool shape_ok(int32_t batch, int32_t beams, int32_t vocab) {
  return beams <= GMM_BEAM_MAX && vocab <= GMM_BEAM_MAX_VOCAB &&
         (int64_t)batch * beams <= (1 << 24) && (int64_t)batch * 1024 <= kMaxThreads &&
         (int64_t)batch * beams * cdiv(vocab, kRun) <= 4 * kMaxBlocks;
}

int64_t need(int32_t batch, int32_t beams, int32_t vocab) {
  return cdiv((int64_t)batch * beams * cdiv(vocab, kRun) * (int64_t)sizeof(float2), 256) * 256;
}

template <typename T>
int launch(const BeamArgs& a, int batch, hipStream_t st) {
  hipLaunchKernelGGL((k_beam_run<T>), dim3((unsigned)cdiv((int64_t)a.rows * a.runs, 4)), dim3(256),
                     0, st, a);
  const int most = a.beams > a.m ? a.beams : a.m;
  const auto join = [&](auto kernel, int waves) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)batch), dim3(64 * waves), 0, st, a);
  };
  if (most <= 4) join(k_beam_join<T, 4>, 4);
  else if (most <= 8) join(k_beam_join<T, 8>, 8);
  else join(k_beam_join<T, 16>, 16);
  return launch_status();
}

}  // namespace

extern "C" {

size_t gmm_beam_workspace_bytes(int32_t batch, int32_t beams, int32_t vocab) {
  if (batch < 1 || beams < 1 || vocab < 1 || !shape_ok(batch, beams, vocab)) return 0;
  return (size_t)need(batch, beams, vocab);
}

int gmm_beam_select(const void* logits, int32_t dtype, int64_t seq_stride, int64_t beam_stride,
                    int32_t batch, int32_t beams, int32_t vocab, const float* score,
                    const float* weight, const uint8_t* done, int32_t eos, const int32_t* mask,
                    int64_t mask_stride, double scale, int32_t m, float* out_score,
                    int32_t* out_parent, int32_t* out_token, uint8_t* out_done, void* ws,
                    size_t ws_bytes, hipStream_t stream) {
  if (batch < 0 || beams < 1 || vocab < 1 || m < 1 || eos >= vocab) return GMM_ERR_INVALID_ARG;
  if (dtype != GMM_F32 && dtype != GMM_BF16 && dtype != GMM_F16) return GMM_ERR_UNSUPPORTED;
  if (m > GMM_BEAM_MAX || !shape_ok(batch, beams, vocab)) return GMM_ERR_UNSUPPORTED;
  if (!(scale >= 1e-6 && scale <= 1e6)) return GMM_ERR_INVALID_ARG;
  if (done && (eos < 0 || !out_done)) return GMM_ERR_INVALID_ARG;
  if (mask && mask_stride < cdiv(vocab, 32)) return GMM_ERR_INVALID_ARG;
  if (batch == 0) return GMM_OK;
  if (!logits || !score || !out_score || !out_parent || !out_token) return GMM_ERR_INVALID_ARG;
  // rows are read by elements of this size
  if ((uintptr_t)logits % (dtype == GMM_F32 ? 4 : 2)) return GMM_ERR_INVALID_ARG;
  // a sequence's results may take the place of what was read for them, not of another's
  const int64_t rows = (int64_t)batch * beams, places = (int64_t)batch * m;
  const auto spoils = [&](const void* out, const void* in, int size) {
    return out && in && !(out == in && m == beams) && overlap(out, places * size, in, rows * size);
  };
  if (spoils(out_score, score, 4) || spoils(out_score, weight, 4) || spoils(out_done, done, 1))
    return GMM_ERR_INVALID_ARG;
  const int rc = check_kv_ws(ws, ws_bytes, need(batch, beams, vocab));
  if (rc != GMM_OK) return rc;
  // nor that of anything else that is read or written
  const struct { const void* at; int64_t bytes; } all[] = {
      {out_score, places * 4}, {out_done, places}, {out_parent, places * 4}, {out_token, places * 4},
      {score, rows * 4}, {weight, rows * 4}, {done, rows}};
  for (int i = 0; i < 4; ++i)
    for (int j = i + 1; j < 7; ++j) {
      const bool own_place = i == 0 ? j == 4 || j == 5 : i == 1 && j == 6;      // looked at above
      if (!own_place && all[i].at && all[j].at && overlap(all[i].at, all[i].bytes, all[j].at, all[j].bytes))
        return GMM_ERR_INVALID_ARG;
    }
  BeamArgs a{};
  a.x = logits;
  a.seq_stride = seq_stride;
  a.beam_stride = beam_stride;
  a.score = score;
  a.weight = weight;
  a.done = done;
  a.mask = (const uint32_t*)mask;
  a.mask_stride = mask_stride;
  a.scale = scale;
  a.c = (float)(scale * kLog2eD);
  int above;
  frexp(a.c, &above);
  a.above_c = ldexpf(1.f, above);
  a.beams = beams;
  a.vocab = vocab;
  a.runs = (int)cdiv(vocab, kRun);
  a.m = m;
  a.eos = eos;
  a.rows = batch * beams;
  a.part = (float2*)ws;
  a.out_score = out_score;
  a.out_parent = out_parent;
  a.out_token = out_token;
  a.out_done = out_done;
  if (dtype == GMM_F32) return launch<float>(a, batch, stream);
  if (dtype == GMM_BF16) return launch<__bf16>(a, batch, stream);
  return launch<_Float16>(a, batch, stream);
}

}  // extern "C"
