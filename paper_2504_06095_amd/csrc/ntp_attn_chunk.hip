// Attention of chunks of new tokens over the paged cache (ntp_attn_chunk_shard).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "ntp_gemm_kernels.h"
#include "ntp_internal.h"
#include "ntp_kv_cache.h"

namespace {

using ntp::off16;

struct ChunkArgs {
  const uint16_t* Q;
  const unsigned char *K, *V;
  const uint8_t *K_exp, *V_exp;
  const int32_t *starts, *table, *lengths;
  uint16_t* C;
  float* LSE;
  int64_t M, ldq, ldc, ldt, page_stride, exp_stride;
  int32_t n_pages, n_seq, max_new, max_len, q_cnt, q_off, kv_off, group, page_size, page_log2;
  float scale_log2;
};

template <int D, bool FP8>
__global__ __launch_bounds__(256) void attn_chunk_plain_kernel(const ChunkArgs a) {
  constexpr int N = D / 64;
  const int lane = threadIdx.x & 63;
  const int64_t id = int64_t(blockIdx.x) * 4 + (threadIdx.x >> 6);
  if (id >= a.M * a.q_cnt) return;
  const int64_t row = id / a.q_cnt;
  const int head = int(id % a.q_cnt), g = (a.q_off + head) / a.group - a.kv_off;
  int s = -1, start = 0, n = 0;
  if (!a.starts) s = int(row), start = int(row), n = 1;
  else
    for (int i = 0; i < a.n_seq; ++i) {
      const int64_t lo = std::min<int64_t>(std::max(a.starts[i], 0), a.M), hi = std::min<int64_t>(std::max(a.starts[i + 1], 0), a.M);
      if (row >= lo && row < hi) s = i, start = int(lo), n = int(hi - lo);
    }
  if (s < 0 || row - start >= a.max_new) return;
  const int seen = std::min(a.lengths[s], a.max_len) - n + int(row - start) + 1;
  float q[N], acc[N];
  for (int i = 0; i < N; ++i) q[i] = __builtin_bit_cast(float, uint32_t(a.Q[row * a.ldq + int64_t(head) * D + lane * N + i]) << 16), acc[i] = 0.f;
  float m = -INFINITY, l = 0.f;
  for (int t = 0; t < seen; ++t) {
    const int page = a.table[int64_t(s) * a.ldt + (t >> a.page_log2)];
    if (page < 0 || page >= a.n_pages) continue;
    const int64_t in = int64_t(g) * a.page_size + (t & (a.page_size - 1)), at = int64_t(page) * a.page_stride + in * D + lane * N;
    float k[N], v[N];
    for (int i = 0; i < N; ++i) {
      if constexpr (FP8) {
        const uint32_t e = a.K_exp[int64_t(page) * a.exp_stride + in], f = a.V_exp[int64_t(page) * a.exp_stride + in];
        k[i] = __builtin_amdgcn_cvt_f32_fp8(a.K[at + i], 0) * __builtin_bit_cast(float, e << 23);
        v[i] = __builtin_amdgcn_cvt_f32_fp8(a.V[at + i], 0) * __builtin_bit_cast(float, f << 23);
      } else {
        k[i] = __builtin_bit_cast(float, uint32_t(reinterpret_cast<const uint16_t*>(a.K)[at + i]) << 16);
        v[i] = __builtin_bit_cast(float, uint32_t(reinterpret_cast<const uint16_t*>(a.V)[at + i]) << 16);
      }
    }
    float x = 0.f;
    for (int i = 0; i < N; ++i) x = fmaf(q[i], k[i], x);
    for (int d = 1; d < 64; d *= 2) x += __shfl_xor(x, d);
    x *= a.scale_log2;
    const float mn = fmaxf(m, x), use = mn == -INFINITY ? 0.f : mn, al = exp2f(m - use), p = exp2f(x - use);
    l = l * al + p;
    for (int i = 0; i < N; ++i) acc[i] = acc[i] * al + p * v[i];
    m = mn;
  }
  const float inv = l == 0.f ? 0.f : 1.0f / l;
  for (int i = 0; i < N; ++i) a.C[row * a.ldc + int64_t(head) * D + lane * N + i] = ntp_gemm::f32_to_bf16(acc[i] * inv);
  if (lane == 0 && a.LSE) a.LSE[int64_t(head) * a.M + row] = (m == -INFINITY ? -INFINITY : m + log2f(l)) * 0.6931471805599453f;
}

int check_chunk_shape(const ntp_attn_chunk_shape_t* s) {
  if (!s || s->M < 0 || s->n_seq < 0 || s->max_new < 0 || s->max_len < 0 || s->q_cnt < 0 || s->kv_cnt < 0 || s->q_off < 0 || s->kv_off < 0 || s->group < 1) return NTP_ERR_INVALID_ARG;
  if (s->head_dim != 64 && s->head_dim != 128) return NTP_ERR_UNSUPPORTED;
  if (s->max_len > 1 << 30 || int64_t(s->q_off) + s->q_cnt > 0x7fffffffll || s->M > 0x7fffffffll || s->M * std::max(s->q_cnt, 1) > 0x7fffffffll ||
      int64_t(s->n_seq) * ((int64_t(s->max_len) + 63) / 64 + 1) * std::max(s->kv_cnt, 1) > 0x7fffffffll)
    return NTP_ERR_UNSUPPORTED;
  // the KV heads of the local query heads ascend: the first and the last must be local
  if (s->q_cnt > 0) {
    const int64_t first = int64_t(s->q_off) / s->group - s->kv_off, last = (int64_t(s->q_off) + s->q_cnt - 1) / s->group - s->kv_off;
    if (first < 0 || last >= s->kv_cnt) return NTP_ERR_INVALID_ARG;
  }
  return NTP_OK;
}

}  // namespace

int ntp::attn_chunk_workspace_wish(const ntp_handle* h, const ntp_attn_chunk_shape_t* s, int64_t* bytes) {
  if (check_chunk_shape(s) != NTP_OK) return NTP_ERR_INVALID_ARG;
  *bytes = 0;
  return NTP_OK;
}

extern "C" int ntp_attn_chunk_shard(ntp_handle_t* h, const ntp_attn_chunk_shape_t* s, const ntp_kv_pages_t* pages, const void* Q, int64_t ldq, const int32_t* row_starts,
                                    const int32_t* block_table, int64_t ldt, const int32_t* lengths, void* C, int64_t ldc, float* LSE, void* stream) {
  if (!h) return NTP_ERR_INVALID_ARG;
  int st = check_chunk_shape(s);
  if (st != NTP_OK || (st = ntp::check_kv_pages(pages, s->kv_cnt, s->head_dim)) != NTP_OK) return st;
  if (!row_starts && s->M != s->n_seq) return NTP_ERR_INVALID_ARG;
  if (s->n_seq == 0 || s->M == 0 || s->q_cnt == 0 || s->max_new == 0) return NTP_OK;
  const int64_t w = int64_t(s->q_cnt) * s->head_dim, used = (int64_t(s->max_len) + pages->page_size - 1) / pages->page_size;
  if (!Q || !C || !lengths || (!block_table && used > 0) || ldq < w || ldc < w || ldt < used) return NTP_ERR_INVALID_ARG;
  auto off4 = [](const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3) != 0; };
  if (off16(Q) || off16(C) || ldq % 8 || ldc % 8 || off4(row_starts) || off4(block_table) || off4(lengths) || off4(LSE)) return NTP_ERR_ALIGNMENT;
  if (h->device < 0) return NTP_ERR_NO_DEVICE;
  ChunkArgs a{};
  a.Q = static_cast<const uint16_t*>(Q), a.K = static_cast<const unsigned char*>(pages->K), a.V = static_cast<const unsigned char*>(pages->V);
  a.K_exp = static_cast<const uint8_t*>(pages->K_exp), a.V_exp = static_cast<const uint8_t*>(pages->V_exp);
  a.starts = row_starts, a.table = block_table, a.lengths = lengths, a.C = static_cast<uint16_t*>(C), a.LSE = LSE;
  a.M = s->M, a.ldq = ldq, a.ldc = ldc, a.ldt = ldt, a.page_stride = pages->page_stride, a.exp_stride = pages->exp_stride, a.n_pages = int32_t(pages->n_pages);
  a.n_seq = s->n_seq, a.max_new = s->max_new, a.max_len = s->max_len, a.q_cnt = s->q_cnt, a.q_off = s->q_off, a.kv_off = s->kv_off, a.group = s->group;
  a.page_size = pages->page_size, a.page_log2 = ntp::log2_of(pages->page_size);
  a.scale_log2 = float(1.4426950408889634 / std::sqrt(double(s->head_dim)));
  hipStream_t hs = static_cast<hipStream_t>(stream);
  const bool fp8 = pages->format == NTP_KV_E4M3;
  const dim3 grid{uint32_t((s->M * s->q_cnt + 3) / 4)};
  if (ntp::timing_on(h)) ntp::timing_begin(h, stream, fp8 ? "attn_chunk8" : "attn_chunk", 4.0 * double(s->M) * double(s->max_len) * s->head_dim * s->q_cnt, 0.0);
  if (s->head_dim == 128 && fp8) hipLaunchKernelGGL((attn_chunk_plain_kernel<128, true>), grid, dim3(256), 0, hs, a);
  else if (s->head_dim == 128) hipLaunchKernelGGL((attn_chunk_plain_kernel<128, false>), grid, dim3(256), 0, hs, a);
  else if (fp8) hipLaunchKernelGGL((attn_chunk_plain_kernel<64, true>), grid, dim3(256), 0, hs, a);
  else hipLaunchKernelGGL((attn_chunk_plain_kernel<64, false>), grid, dim3(256), 0, hs, a);
  const bool ok = hipGetLastError() == hipSuccess;
  ntp::timing_end(h, stream);
  return ok ? NTP_OK : NTP_ERR_LAUNCH;
}
