// Host-side checks that the paged cache's calls share.
#ifndef KV_HOST_H
#define KV_HOST_H

#include <hip/hip_runtime.h>

#include <stdint.h>

#include "flashgmm.h"

namespace kv {

inline int launch_status() {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? GMM_OK : GMM_ERR_DEVICE;
}

inline bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }
inline bool is_pow2(int64_t v) { return v > 0 && (v & (v - 1)) == 0; }
inline int log2i(int v) {
  int s = 0;
  while ((1 << s) < v) ++s;
  return s;
}

inline int check_cache(const gmm_kv_cache* c) {
  if (!c || !c->k || !c->v) return GMM_ERR_INVALID_ARG;
  if (c->pages < 1 || c->heads < 1 || c->page < 1 || c->d < 1) return GMM_ERR_INVALID_ARG;
  if (!aligned16(c->k) || !aligned16(c->v) || !aligned16(c->box)) return GMM_ERR_INVALID_ARG;
  if ((c->box == nullptr) != (c->box_scale == nullptr)) return GMM_ERR_INVALID_ARG;
  if (c->dtype != GMM_BF16 && c->dtype != GMM_F16) return GMM_ERR_UNSUPPORTED;
  if (c->d % 16 || c->d > GMM_KV_MAX_D || !is_pow2(c->page) || c->page < 32 || c->page > 256 ||
      c->heads > GMM_KV_MAX_HEADS)
    return GMM_ERR_UNSUPPORTED;
  return GMM_OK;
}

inline int check_kv_ws(void* ws, size_t have, int64_t need) {
  if (!ws || ((uintptr_t)ws & 255) || (int64_t)have < need) return GMM_ERR_WORKSPACE;
  return GMM_OK;
}

// do [a, a + na) and [b, b + nb) share a byte?
inline bool overlap(const void* a, int64_t na, const void* b, int64_t nb) {
  const char *p = (const char*)a, *q = (const char*)b;
  return p < q + nb && q < p + na;
}

}  // namespace kv

#endif  // KV_HOST_H
