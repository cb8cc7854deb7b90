// The paged key / value cache of a rank's local KV heads: checks shared by the calls that write and read it (not part of the ABI).
#ifndef NTP_KV_CACHE_H_
#define NTP_KV_CACHE_H_

#include <stdint.h>

#include "ntp.h"

namespace ntp {

inline bool off16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) != 0; }

inline int check_kv_cache(const ntp_kv_cache_t* c, int32_t kv_cnt, int32_t head_dim) {
  if (!c || c->n_pages < 0 || c->page_stride < 0 || (c->n_pages > 0 && (!c->K || !c->V))) return NTP_ERR_INVALID_ARG;
  if (c->page_size < 16 || c->page_size > 65536 || (c->page_size & (c->page_size - 1)) || c->n_pages > 0x7fffffffll) return NTP_ERR_UNSUPPORTED;
  if (c->page_stride < int64_t(kv_cnt) * c->page_size * head_dim) return NTP_ERR_INVALID_ARG;
  if (off16(c->K) || off16(c->V) || c->page_stride % 8) return NTP_ERR_ALIGNMENT;
  return NTP_OK;
}

inline int32_t log2_of(int32_t power) {
  int32_t n = 0;
  while ((1 << n) < power) ++n;
  return n;
}

}  // namespace ntp

#endif  // NTP_KV_CACHE_H_
