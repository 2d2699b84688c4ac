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

#include <math.h>
#include <stdint.h>

#include "flashgmm.h"
#include "kv_host.h"
#include "kv_plan.h"

namespace {

using namespace kv;

constexpr double kLog2eD = 1.4426950408889634;
constexpr int kRun = 2048;        // words of a run
constexpr int kJoinWaves = 8;     // waves of a sequence's workgroup
constexpr uint32_t kNone = 0xffffffffu;

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
  int beams, vocab, runs, m, eos;
  int64_t rows;
  float2* part;               // [rows, runs]: maximum, sum
  float* out_score;
  int32_t* out_parent;
  int32_t* out_token;
  uint8_t* out_done;
};

__device__ __forceinline__ bool finite(float v) { return fabsf(v) < INFINITY; }

// 16 bytes of a row, whose address is a multiple of an element only
template <typename T>
__device__ __forceinline__ void load_vec(const T* p, float* o) {
  constexpr int N = 16 / sizeof(T);
  typedef T V __attribute__((ext_vector_type(N), aligned(sizeof(T))));
  const V v = *reinterpret_cast<const V*>(p);
#pragma unroll
  for (int e = 0; e < N; ++e) o[e] = (float)v[e];
}

// Words at .. at + N - 1 of a beam; -inf past the vocabulary and where the mask forbids them.
template <typename T>
__device__ __forceinline__ void load_words(const BeamArgs& a, const T* x, const uint32_t* mask,
                                           int at, float* o) {
  constexpr int N = 16 / sizeof(T);
  if (at + N <= a.vocab) {
    load_vec<T>(x + at, o);
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e) o[e] = at + e < a.vocab ? (float)x[at + e] : -INFINITY;
  }
  if (mask && at < a.vocab) {
    const uint32_t bits = mask[at >> 5] >> (at & 31);
#pragma unroll
    for (int e = 0; e < N; ++e) o[e] = bits >> e & 1 ? o[e] : -INFINITY;
  }
}

template <typename T>
__device__ __forceinline__ const T* row_of(const BeamArgs& a, int64_t row) {
  const int64_t b = row / a.beams;
  return (const T*)a.x + b * a.seq_stride + (row - b * a.beams) * a.beam_stride;
}
__device__ __forceinline__ const uint32_t* mask_of(const BeamArgs& a, int64_t row) {
  return a.mask ? a.mask + row * a.mask_stride : nullptr;
}

// A wave a run: its maximum and sum of exponentials.  A NaN or +infinity makes the sum NaN.
template <typename T>
__global__ __launch_bounds__(256) void k_beam_run(BeamArgs a) {
  const int lane = threadIdx.x & 63;
  const int64_t item = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int64_t row = item / a.runs;
  if (row >= a.rows) return;
  if (!finite(a.score[row]) || (a.done && a.done[row])) return;
  constexpr int N = 16 / sizeof(T), L = kRun / (64 * N);
  const int run = (int)(item - row * a.runs);
  const T* x = row_of<T>(a, row);
  const uint32_t* mask = mask_of(a, row);
  float v[L][N];
#pragma unroll
  for (int i = 0; i < L; ++i)
    load_words<T>(a, x, mask, run * kRun + (i * 64 + lane) * N, v[i]);
  float mx = -INFINITY;
#pragma unroll
  for (int i = 0; i < L; ++i)
#pragma unroll
    for (int e = 0; e < N; ++e) mx = fmaxf(mx, v[i][e]);
  for (int o = 32; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor(mx, o));
  const float base = mx > -INFINITY ? mx : 0.f;
  // the difference before the product: its rounding, not that of a large maximum's product
  float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < L; ++i)
#pragma unroll
    for (int e = 0; e < N; ++e) sum[e & 3] += __builtin_amdgcn_exp2f((v[i][e] - base) * a.c);
  float z = (sum[0] + sum[1]) + (sum[2] + sum[3]);
  for (int o = 32; o > 0; o >>= 1) z += __shfl_xor(z, o);
  if (lane == 0) a.part[item] = make_float2(mx, z);
}

// ---------------------------------------------------------------- sorted lists
// A wave's list: lane i holds the i-th best of what it has seen, by (key, lower index).
struct Entry {
  double key;
  uint32_t at;
};
__device__ __forceinline__ Entry no_entry() { return Entry{-INFINITY, kNone}; }
__device__ __forceinline__ bool before(const Entry& a, const Entry& b) {
  return a.key > b.key || (a.key == b.key && a.at < b.at);
}
__device__ __forceinline__ Entry shuffle_xor(const Entry& e, int o) {
  return Entry{__shfl_xor(e.key, o), (uint32_t)__shfl_xor((int)e.at, o)};
}
__device__ __forceinline__ Entry shuffle(const Entry& e, int lane) {
  return Entry{__shfl(e.key, lane), (uint32_t)__shfl((int)e.at, lane)};
}
__device__ __forceinline__ void stage(Entry& e, int o, bool up) {
  const Entry p = shuffle_xor(e, o);
  const bool low = (threadIdx.x & o) == 0;
  if (before(p, e) == (low != up)) e = p;
}
// bitonic: 64 entries in any order
__device__ __forceinline__ void sort64(Entry& e) {
  for (int k = 2; k <= 64; k <<= 1)
    for (int o = k >> 1; o > 0; o >>= 1) stage(e, o, (threadIdx.x & k & 63) != 0);
}
// the 64 best of two sorted lists
__device__ __forceinline__ void merge64(Entry& a, const Entry& b) {
  const Entry r = shuffle(b, 63 - (threadIdx.x & 63));
  if (before(r, a)) a = r;
  for (int o = 32; o > 0; o >>= 1) stage(a, o, false);
}

struct Join {
  double key[kJoinWaves][64];
  uint32_t at[kJoinWaves][64];
  float top[GMM_BEAM_MAX];          // a beam's largest logit
  double logz[GMM_BEAM_MAX];        // log sum exp(scale (x - top))
  float score[GMM_BEAM_MAX];
  double weight[GMM_BEAM_MAX];
  int kind[GMM_BEAM_MAX];           // 0: no candidate, 1: live, 2: finished
  Entry buf[kJoinWaves][128];
};

// the waves' lists into wave 0's; all lists are the joined one afterwards
__device__ __forceinline__ void join_lists(Join& s, Entry& e) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  for (int n = kJoinWaves; n > 1; n >>= 1) {
    s.key[w][lane] = e.key;
    s.at[w][lane] = e.at;
    __syncthreads();
    if (w < n / 2) merge64(e, Entry{s.key[w + n / 2][lane], s.at[w + n / 2][lane]});
    __syncthreads();
  }
  s.key[w][lane] = e.key;
  s.at[w][lane] = e.at;
  __syncthreads();
  e = Entry{s.key[0][lane], s.at[0][lane]};
  __syncthreads();
}

// l of a live beam's logit, from its difference to the largest: products of large logits would
// cancel, and not alike everywhere (multiply and add may be fused)
__device__ __forceinline__ double total_of(const BeamArgs& a, const Join& s, int j, float x) {
  return (double)s.score[j] + fma(a.scale, (double)x - (double)s.top[j], -s.logz[j]);
}
__device__ __forceinline__ double key_of(const BeamArgs& a, const Join& s, int j, float x) {
  return x > -INFINITY ? s.weight[j] * total_of(a, s, j, x) : -INFINITY;
}

// A workgroup a sequence: log Z of its beams, its m best runs, their m best words.
template <typename T>
__global__ __launch_bounds__(64 * kJoinWaves) void k_beam_join(BeamArgs a) {
  __shared__ Join s;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int64_t row0 = (int64_t)blockIdx.x * a.beams;
  for (int j = w; j < a.beams; j += kJoinWaves) {
    const float sc = a.score[row0 + j];
    int kind = finite(sc) ? a.done && a.done[row0 + j] ? 2 : 1 : 0;
    double logz = 0.0;
    float mx = -INFINITY;
    if (kind == 1) {
      const float2* p = a.part + (row0 + j) * a.runs;
      for (int r = lane; r < a.runs; r += 64) mx = fmaxf(mx, p[r].x);
      for (int o = 32; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor(mx, o));
      double z = 0.0;
      for (int r = lane; r < a.runs; r += 64) {
        const float2 v = p[r];
        // a run without a word adds its sum, 0, or NaN
        z += (double)(v.y * (v.x > -INFINITY ? __builtin_amdgcn_exp2f((v.x - mx) * a.c) : 1.f));
      }
      for (int o = 32; o > 0; o >>= 1) z += __shfl_xor(z, o);
      logz = log(z);
      if (!finite(mx) || !(z > 0.0)) kind = 0;     // no word, NaN or +infinity
    }
    if (lane == 0) {
      s.top[j] = mx;
      s.logz[j] = logz;
      s.score[j] = sc;
      const float wt = a.weight ? a.weight[row0 + j] : 1.f;
      s.weight[j] = wt;
      s.kind[j] = wt > 0.f && finite(wt) ? kind : 0;
    }
  }
  __syncthreads();

  // runs, numbered over the beams; a finished beam's is the one of its end word
  Entry top = no_entry();
  const int runs = a.beams * a.runs;
  for (int c = w * 64; c < runs; c += 64 * kJoinWaves) {
    Entry e = no_entry();
    if (c + lane < runs) {
      const int j = (c + lane) / a.runs, r = c + lane - j * a.runs;
      e.at = c + lane;
      if (s.kind[j] == 1) e.key = key_of(a, s, j, a.part[row0 * a.runs + c + lane].x);
      else if (s.kind[j] == 2 && r == a.eos / kRun) e.key = s.weight[j] * (double)s.score[j];
    }
    if (c >= 64 * kJoinWaves && !__ballot(before(e, shuffle(top, 63)))) continue;
    sort64(e);
    merge64(top, e);
  }
  join_lists(s, top);
  const int found = __popcll(__ballot(lane < a.m && top.key > -INFINITY));
  const double least = found == a.m ? __shfl(top.key, a.m - 1) : -INFINITY;

  // their words; index: beam * vocab + word
  constexpr int N = 16 / sizeof(T);
  Entry best = no_entry();
  int held = 0;                     // entries of the wave's buffer
  Entry* buf = s.buf[w];
  const auto flush = [&](int n) {
    Entry e = lane < n ? buf[lane] : no_entry();
    sort64(e);
    merge64(best, e);
  };
  for (int q = w; q < found; q += kJoinWaves) {
    const int gid = __shfl((int)top.at, q);
    const int j = gid / a.runs, r = gid - j * a.runs;
    const int64_t row = row0 + j;
    if (s.kind[j] == 2) {
      if (lane == 0) buf[held] = Entry{s.weight[j] * (double)s.score[j],
                                       (uint32_t)j * (uint32_t)a.vocab + (uint32_t)a.eos};
      if (++held >= 64) {
        flush(64);
        held -= 64;
      }
      continue;
    }
    const T* x = row_of<T>(a, row);
    const uint32_t* mask = mask_of(a, row);
    for (int i = 0; i < kRun / (64 * N); ++i) {
      const int at = r * kRun + (i * 64 + lane) * N;
      float v[N];
      load_words<T>(a, x, mask, at, v);
      const Entry last = shuffle(best, a.m - 1);
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const Entry c{key_of(a, s, j, v[e]), (uint32_t)j * (uint32_t)a.vocab + (uint32_t)(at + e)};
        const bool in = c.key > -INFINITY && c.key >= least && before(c, last);
        const uint64_t bal = __ballot(in);
        if (!bal) continue;
        if (in) buf[held + __popcll(bal & ((1ull << lane) - 1))] = c;
        held += __popcll(bal);
        if (held >= 64) {
          flush(64);
          held -= 64;
          if (lane < held) buf[lane] = buf[64 + lane];
        }
      }
    }
  }
  if (held > 0) flush(held);
  join_lists(s, best);
  if (w != 0 || lane >= a.m) return;
  const int64_t o = (int64_t)blockIdx.x * a.m + lane;
  if (!(best.key > -INFINITY)) {
    a.out_score[o] = -INFINITY;
    a.out_parent[o] = -1;
    a.out_token[o] = -1;
    if (a.out_done) a.out_done[o] = 0;
    return;
  }
  const int j = (int)(best.at / (uint32_t)a.vocab), word = (int)(best.at - (uint32_t)j * a.vocab);
  const bool fin = s.kind[j] == 2;
  a.out_score[o] = fin ? s.score[j]
                       : (float)total_of(a, s, j, (float)row_of<T>(a, row0 + j)[word]);
  a.out_parent[o] = (int32_t)(row0 + j);
  a.out_token[o] = word;
  if (a.out_done) a.out_done[o] = fin || word == a.eos;
}

// ---------------------------------------------------------------- host
bool shape_ok(int32_t batch, int32_t beams, int32_t vocab) {
  return beams <= GMM_BEAM_MAX && vocab <= GMM_BEAM_MAX_VOCAB &&
         (int64_t)batch * beams <= (1 << 24) &&
         (int64_t)batch * beams * cdiv(vocab, kRun) <= 4 * kMaxBlocks;
}

int64_t need(int32_t batch, int32_t beams, int32_t vocab) {
  return cdiv((int64_t)batch * beams * cdiv(vocab, kRun) * (int64_t)sizeof(float2), 256) * 256;
}

template <typename T>
int launch(const BeamArgs& a, int batch, hipStream_t st) {
  hipLaunchKernelGGL((k_beam_run<T>), dim3((unsigned)cdiv(a.rows * a.runs, 4)), dim3(256), 0, st,
                     a);
  hipLaunchKernelGGL((k_beam_join<T>), dim3((unsigned)batch), dim3(64 * kJoinWaves), 0, st, a);
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
  const int rc = check_kv_ws(ws, ws_bytes, need(batch, beams, vocab));
  if (rc != GMM_OK) return rc;
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
  a.beams = beams;
  a.vocab = vocab;
  a.runs = (int)cdiv(vocab, kRun);
  a.m = m;
  a.eos = eos;
  a.rows = (int64_t)batch * beams;
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
