// The paged key / value cache of a rank's local KV heads: checks shared by the calls that write and read it (not part of the ABI).
#ifndef NTP_KV_CACHE_H_
#define NTP_KV_CACHE_H_

#include <stdint.h>

#include <cstdlib>

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

// The same of pages in either format.
inline int check_kv_pages(const ntp_kv_pages_t* p, int32_t kv_cnt, int32_t head_dim) {
  if (!p || (p->format != NTP_KV_BF16 && p->format != NTP_KV_E4M3)) return NTP_ERR_INVALID_ARG;
  const ntp_kv_cache_t c{p->K, p->V, p->n_pages, p->page_stride, p->page_size};
  const int st = check_kv_cache(&c, kv_cnt, head_dim);
  if (st != NTP_OK || p->format == NTP_KV_BF16) return st;
  if ((p->n_pages > 0 && (!p->K_exp || !p->V_exp)) || p->exp_stride < int64_t(kv_cnt) * p->page_size) return NTP_ERR_INVALID_ARG;
  if (off16(p->K_exp) || off16(p->V_exp) || p->exp_stride % 16 || p->page_stride % 16) return NTP_ERR_ALIGNMENT;
  return NTP_OK;
}

// Whether two views of bf16 rows share an element.  With one leading dimension their columns are compared, modulo it: row i of a lies i - j leading dimensions
// and the bases' distance from row j of b.  With two of them the whole spans are.
inline bool rows_overlap(const void* a, int64_t lda, int64_t wa, const void* b, int64_t ldb, int64_t wb, int64_t rows) {
  const char *p = static_cast<const char*>(a), *q = static_cast<const char*>(b);
  if (!p || !q || wa == 0 || wb == 0 || p >= q + ((rows - 1) * ldb + wb) * 2 || q >= p + ((rows - 1) * lda + wa) * 2) return false;
  if (lda != ldb || rows == 1) return true;
  const int64_t off = (p - q) / 2;
  int64_t column = off % lda, row = off / lda;  // of a's first element in b
  if (column < 0) column += lda, --row;
  // a's rows begin in b's at that column (row 0 of a in row `row` of b), and reach into the next ones' where they pass the leading dimension
  return (column < wb && std::llabs(row) < rows) || (column + wa > lda && std::llabs(row + 1) < rows);
}

inline int32_t log2_of(int32_t power) {
  int32_t n = 0;
  while ((1 << n) < power) ++n;
  return n;
}

}  // namespace ntp

#endif  // NTP_KV_CACHE_H_
