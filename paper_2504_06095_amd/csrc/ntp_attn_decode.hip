// Attention of one new token per sequence over the paged key / value cache (ntp_attn_decode_shard): for sequence s and query head j
//   C[s, j] = sum_t p_t V[t] / sum_t p_t,   p_t = exp(q_j . K[t] / sqrt(d) - max),   t over the sequence's tokens.
// One pass over the keys with a running maximum and sum.  Every key and value is used by the query heads of one KV head only, 4 d bytes for
// 4 d operations a query head: HBM bounds it.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "ntp_internal.h"
#include "ntp_kv_cache.h"

namespace {

using ntp::off16;
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;

struct DecodeArgs {
  const uint16_t *Q, *K, *V;
  const int32_t *table, *lengths;
  uint16_t* C;
  float* LSE;
  int64_t ldq, ldc, ldt, page_stride, n_pages;
  int32_t n_seq, max_len, q_cnt, q_off, kv_off, group, page_size, page_log2;
  float scale_log2;  // log2(e) / sqrt(d)
};

__device__ __forceinline__ float bf_lo(uint32_t v) { return __builtin_bit_cast(float, v << 16); }
__device__ __forceinline__ float bf_hi(uint32_t v) { return __builtin_bit_cast(float, v & 0xffff0000u); }

// One workgroup per (sequence, query head): D / 8 lanes share a key, 16 bytes each.
template <int D>
__global__ __launch_bounds__(kThreads) void attn_decode_kernel(const DecodeArgs a) {
  constexpr int LPK = D / 8, KEYS = kThreads / LPK;  // lanes per key, keys at a time
  __shared__ float part[KEYS][D + 2];
  const int head = blockIdx.x % a.q_cnt, seq = blockIdx.x / a.q_cnt;
  const int g = (a.q_off + head) / a.group - a.kv_off;
  const int len = std::min(a.lengths[seq], a.max_len);
  const int sub = threadIdx.x % LPK, slot = threadIdx.x / LPK;
  const u32x4 qr = *reinterpret_cast<const u32x4*>(a.Q + int64_t(seq) * a.ldq + int64_t(head) * D + sub * 8);
  float q[8], acc[8] = {}, m = -INFINITY, l = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    q[2 * i] = bf_lo(qr[i]) * a.scale_log2;
    q[2 * i + 1] = bf_hi(qr[i]) * a.scale_log2;
  }
  for (int key = slot; key < len; key += KEYS) {
    const int page = a.table[int64_t(seq) * a.ldt + (key >> a.page_log2)];
    if (page < 0 || page >= a.n_pages) continue;
    const int64_t at = int64_t(page) * a.page_stride + (int64_t(g) * a.page_size + (key & (a.page_size - 1))) * D + sub * 8;
    const u32x4 k = *reinterpret_cast<const u32x4*>(a.K + at), v = *reinterpret_cast<const u32x4*>(a.V + at);
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) s = fmaf(q[2 * i], bf_lo(k[i]), fmaf(q[2 * i + 1], bf_hi(k[i]), s));
#pragma unroll
    for (int x = 1; x < LPK; x *= 2) s += __shfl_xor(s, x);
    const float m_new = fmaxf(m, s), m_use = m_new == -INFINITY ? 0.f : m_new;  // (no score above -inf so far: weights of 0)
    const float alpha = exp2f(m - m_use), p = exp2f(s - m_use);
    l = l * alpha + p;
    m = m_new;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      acc[2 * i] = fmaf(acc[2 * i], alpha, p * bf_lo(v[i]));
      acc[2 * i + 1] = fmaf(acc[2 * i + 1], alpha, p * bf_hi(v[i]));
    }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) part[slot][sub * 8 + i] = acc[i];
  if (sub == 0) {
    part[slot][D] = m;
    part[slot][D + 1] = l;
  }
  __syncthreads();
  if (threadIdx.x >= D) return;
  float top = -INFINITY, sum = 0.f, o = 0.f;
  for (int i = 0; i < KEYS; ++i) top = fmaxf(top, part[i][D]);
  if (top == -INFINITY) top = 0.f;
  for (int i = 0; i < KEYS; ++i) {
    const float w = exp2f(part[i][D] - top);
    sum = fmaf(w, part[i][D + 1], sum);
    o = fmaf(w, part[i][threadIdx.x], o);
  }
  a.C[int64_t(seq) * a.ldc + int64_t(head) * D + threadIdx.x] = __builtin_bit_cast(uint16_t, static_cast<__bf16>(sum == 0.f ? 0.f : o / sum));
  if (a.LSE && threadIdx.x == 0) a.LSE[int64_t(head) * a.n_seq + seq] = (top + log2f(sum)) * 0.6931471805599453f;
}

int check_decode_shape(const ntp_attn_decode_shape_t* s) {
  if (!s || s->n_seq < 0 || s->max_len < 0 || s->q_cnt < 0 || s->kv_cnt < 0 || s->q_off < 0 || s->kv_off < 0 || s->group < 1) return NTP_ERR_INVALID_ARG;
  if (s->head_dim != 64 && s->head_dim != 128) return NTP_ERR_UNSUPPORTED;
  if (int64_t(s->n_seq) * s->q_cnt > 0x7fffffffll || int64_t(s->q_off) + s->q_cnt > 0x7fffffffll) return NTP_ERR_UNSUPPORTED;
  // the KV heads of the local query heads ascend: the first and the last must be local
  if (s->q_cnt > 0) {
    const int64_t first = int64_t(s->q_off) / s->group - s->kv_off, last = (int64_t(s->q_off) + s->q_cnt - 1) / s->group - s->kv_off;
    if (first < 0 || last >= s->kv_cnt) return NTP_ERR_INVALID_ARG;
  }
  return NTP_OK;
}

}  // namespace

int ntp::attn_decode_workspace_wish(const ntp_handle*, const ntp_attn_decode_shape_t* s, int64_t* bytes) {
  if (check_decode_shape(s) != NTP_OK) return NTP_ERR_INVALID_ARG;
  *bytes = 0;
  return NTP_OK;
}

extern "C" int ntp_attn_decode_shard(ntp_handle_t* h, const ntp_attn_decode_shape_t* s, const ntp_kv_cache_t* cache, const void* Q, int64_t ldq,
                                     const int32_t* block_table, int64_t ldt, const int32_t* lengths, void* C, int64_t ldc, float* LSE,
                                     void* stream) {
  int st = check_decode_shape(s);
  if (st != NTP_OK) return st;
  if (!h || (st = ntp::check_kv_cache(cache, s->kv_cnt, s->head_dim)) != NTP_OK) return h ? st : NTP_ERR_INVALID_ARG;
  if (s->n_seq == 0 || s->q_cnt == 0) return NTP_OK;
  const int64_t w = int64_t(s->q_cnt) * s->head_dim, pages = (int64_t(s->max_len) + cache->page_size - 1) / cache->page_size;
  if (!Q || !C || !lengths || (!block_table && pages > 0) || ldq < w || ldc < w || ldt < pages) return NTP_ERR_INVALID_ARG;
  auto off4 = [](const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3) != 0; };
  if (off16(Q) || off16(C) || ldq % 8 || ldc % 8 || off4(block_table) || off4(lengths) || off4(LSE)) return NTP_ERR_ALIGNMENT;
  if (h->device < 0) return NTP_ERR_NO_DEVICE;
  DecodeArgs a{};
  a.Q = static_cast<const uint16_t*>(Q), a.K = static_cast<const uint16_t*>(cache->K), a.V = static_cast<const uint16_t*>(cache->V);
  a.table = block_table, a.lengths = lengths, a.C = static_cast<uint16_t*>(C), a.LSE = LSE;
  a.ldq = ldq, a.ldc = ldc, a.ldt = ldt, a.page_stride = cache->page_stride, a.n_pages = cache->n_pages;
  a.n_seq = s->n_seq, a.max_len = s->max_len, a.q_cnt = s->q_cnt, a.q_off = s->q_off, a.kv_off = s->kv_off, a.group = s->group;
  a.page_size = cache->page_size, a.page_log2 = ntp::log2_of(cache->page_size);
  a.scale_log2 = float(1.4426950408889634 / std::sqrt(double(s->head_dim)));
  hipStream_t hs = static_cast<hipStream_t>(stream);
  if (ntp::timing_on(h)) ntp::timing_begin(h, stream, "attn_decode", 4.0 * s->n_seq * double(s->max_len) * s->head_dim * s->q_cnt, 0.0);
  const dim3 grid(uint32_t(int64_t(s->n_seq) * s->q_cnt));
  if (s->head_dim == 128) hipLaunchKernelGGL(attn_decode_kernel<128>, grid, dim3(kThreads), 0, hs, a);
  else hipLaunchKernelGGL(attn_decode_kernel<64>, grid, dim3(kThreads), 0, hs, a);
  const bool ok = hipGetLastError() == hipSuccess;
  ntp::timing_end(h, stream);
  return ok ? NTP_OK : NTP_ERR_LAUNCH;
}
