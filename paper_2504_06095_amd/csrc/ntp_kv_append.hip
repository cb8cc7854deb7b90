// Rotation of the query and key heads and appending of keys and values to the paged cache (ntp_kv_append_shard).
//
// Pair i of a head, (x1, x2), becomes (x1 cos a - x2 sin a, x2 cos a + x1 sin a) with a = position * inv_freq[i]: the angle is formed and reduced to
// less than half a turn in fp64 (positions of 10^5 times a frequency of 1 leave fp32 two digits), its sine and cosine are fp32.  A workgroup takes a few
// tokens, computes their sines and cosines once for all heads, and then streams the heads; what bounds it is HBM (6 operations a pair), and at a
// few tokens the launch itself.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "ntp_internal.h"
#include "ntp_kv_cache.h"

namespace {

using ntp::off16;
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256, kMaxTokens = 8, kMaxPairs = 64;

struct AppendArgs {
  const uint16_t* QKV;
  uint16_t *Qout, *Kout, *K, *V;
  const int32_t* positions;
  const int64_t* slots;
  const double* inv_freq;
  int64_t M, ldqkv, ldq, ldk, page_stride, n_slots;
  int32_t q_cnt, kv_cnt, head_dim, rotary_dim, interleaved, page_size, page_log2;
  int32_t tokens;  // per workgroup
};

__device__ __forceinline__ float bf_lo(uint32_t v) { return __builtin_bit_cast(float, v << 16); }
__device__ __forceinline__ float bf_hi(uint32_t v) { return __builtin_bit_cast(float, v & 0xffff0000u); }
__device__ __forceinline__ uint32_t bf_pack(float lo, float hi) {  // round to nearest even
  return uint32_t(__builtin_bit_cast(uint16_t, static_cast<__bf16>(lo))) | uint32_t(__builtin_bit_cast(uint16_t, static_cast<__bf16>(hi))) << 16;
}

__global__ __launch_bounds__(kThreads) void kv_append_kernel(const AppendArgs a) {
  __shared__ float2 cs[kMaxTokens][kMaxPairs];
  const int64_t row0 = int64_t(blockIdx.x) * a.tokens;
  const int rows = int(std::min<int64_t>(a.tokens, a.M - row0));
  const int half = a.rotary_dim / 2;
  for (int i = threadIdx.x; i < rows * half; i += kThreads) {
    const int t = i / half, p = i % half;
    double turns = double(a.positions[row0 + t]) * a.inv_freq[p] * 0.15915494309189533577;  // 1 / (2 pi)
    turns -= rint(turns);
    float s, c;
    sincospif(2.0f * float(turns), &s, &c);
    cs[t][p] = float2{c, s};
  }
  __syncthreads();
  const int per_head = a.head_dim / 16;  // pairs of 16-byte chunks
  const int heads = a.q_cnt + 2 * a.kv_cnt, per_row = heads * per_head;
  const int rot = a.rotary_dim / 16;
  for (int i = threadIdx.x; i < rows * per_row; i += kThreads) {
    const int t = i / per_row, head = i % per_row / per_head, j = i % per_head;
    const int64_t row = row0 + t;
    const bool is_q = head < a.q_cnt, is_v = head >= a.q_cnt + a.kv_cnt;
    const int g = is_v ? head - a.q_cnt - a.kv_cnt : head - a.q_cnt;
    const bool rotate = !is_v && j < rot;
    // the two chunks: pairs number 8 j .. 8 j + 7, or two chunks behind the rotated part
    int c0 = rot * 2 + (j - rot) * 2, c1 = c0 + 1;
    if (rotate) {
      c0 = a.interleaved ? 2 * j : j;
      c1 = a.interleaved ? 2 * j + 1 : j + rot;
    } else if (is_v) {
      c0 = j;
      c1 = j + per_head;
    }
    uint16_t *d0 = nullptr, *d1 = nullptr;
    if (is_q && a.Qout) d0 = a.Qout + row * a.ldq + int64_t(head) * a.head_dim;
    if (!is_q && !is_v && a.Kout) d0 = a.Kout + row * a.ldk + int64_t(g) * a.head_dim;
    if (!is_q && a.slots) {
      const int64_t slot = a.slots[row];
      if (slot >= 0 && slot < a.n_slots)
        d1 = (is_v ? a.V : a.K) + (slot >> a.page_log2) * a.page_stride + (int64_t(g) * a.page_size + (slot & (a.page_size - 1))) * a.head_dim;
    }
    if (!d0 && !d1) continue;
    const uint16_t* src = a.QKV + row * a.ldqkv + int64_t(head) * a.head_dim;
    u32x4 x = *reinterpret_cast<const u32x4*>(src + c0 * 8), y = *reinterpret_cast<const u32x4*>(src + c1 * 8);
    if (rotate) {
      float2 r[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) r[k] = cs[t][8 * j + k];
      u32x4 u, w;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (a.interleaved) {  // words are pairs: x holds numbers 8 j .. 8 j + 3, y the next four
          const float xl = bf_lo(x[k]), xh = bf_hi(x[k]), yl = bf_lo(y[k]), yh = bf_hi(y[k]);
          u[k] = bf_pack(xl * r[k].x - xh * r[k].y, xh * r[k].x + xl * r[k].y);
          w[k] = bf_pack(yl * r[k + 4].x - yh * r[k + 4].y, yh * r[k + 4].x + yl * r[k + 4].y);
        } else {
          const float xl = bf_lo(x[k]), xh = bf_hi(x[k]), yl = bf_lo(y[k]), yh = bf_hi(y[k]);
          const float2 lo = r[2 * k], hi = r[2 * k + 1];
          u[k] = bf_pack(xl * lo.x - yl * lo.y, xh * hi.x - yh * hi.y);
          w[k] = bf_pack(yl * lo.x + xl * lo.y, yh * hi.x + xh * hi.y);
        }
      }
      x = u;
      y = w;
    }
    if (d0) {
      *reinterpret_cast<u32x4*>(d0 + c0 * 8) = x;
      *reinterpret_cast<u32x4*>(d0 + c1 * 8) = y;
    }
    if (d1) {
      *reinterpret_cast<u32x4*>(d1 + c0 * 8) = x;
      *reinterpret_cast<u32x4*>(d1 + c1 * 8) = y;
    }
  }
}

// Two views of rows may share memory only by being the same columns.
bool overlap(const void* a, int64_t lda, int64_t wa, const void* b, int64_t ldb, int64_t wb, int64_t rows) {
  const char *p = static_cast<const char*>(a), *q = static_cast<const char*>(b);
  return p && q && p < q + ((rows - 1) * ldb + wb) * 2 && q < p + ((rows - 1) * lda + wa) * 2;
}

}  // namespace

extern "C" int ntp_kv_append_shard(ntp_handle_t* h, const ntp_kv_append_shape_t* s, const ntp_kv_cache_t* cache, const void* QKV, int64_t ldqkv,
                                   const int32_t* positions, const int64_t* slots, const double* inv_freq, void* Qout, int64_t ldq, void* Kout,
                                   int64_t ldk, void* stream) {
  if (!h || !s || s->M < 0 || s->q_cnt < 0 || s->kv_cnt < 0 || s->rotary_dim < 0 || (s->M > 0 && (cache != nullptr) != (slots != nullptr))) return NTP_ERR_INVALID_ARG;
  if (s->head_dim != 64 && s->head_dim != 128) return NTP_ERR_UNSUPPORTED;
  if (s->rotary_dim > s->head_dim || s->rotary_dim % 16) return NTP_ERR_INVALID_ARG;
  const int64_t d = s->head_dim, wq = s->q_cnt * d, wk = s->kv_cnt * d, w = wq + 2 * wk;
  if (s->M > 0x7fffffffll || w > 0x7fffffffll / 16) return NTP_ERR_UNSUPPORTED;
  if (cache) {
    const int st = ntp::check_kv_cache(cache, s->kv_cnt, s->head_dim);
    if (st != NTP_OK) return st;
  }
  if (s->M == 0 || w == 0 || (!Qout && !Kout && !cache)) return NTP_OK;
  if (!QKV || (s->rotary_dim > 0 && (!positions || !inv_freq)) || ldqkv < w || (Qout && ldq < wq) || (Kout && ldk < wk)) return NTP_ERR_INVALID_ARG;
  if (off16(QKV) || off16(Qout) || off16(Kout) || ldqkv % 8 || (Qout && ldq % 8) || (Kout && ldk % 8) || (reinterpret_cast<uintptr_t>(positions) & 3) ||
      (reinterpret_cast<uintptr_t>(slots) & 7) || (reinterpret_cast<uintptr_t>(inv_freq) & 7))
    return NTP_ERR_ALIGNMENT;
  const uint16_t* in = static_cast<const uint16_t*>(QKV);
  const bool one = s->M == 1;  // (a leading dimension does not count then)
  if ((overlap(Qout, ldq, wq, QKV, ldqkv, w, s->M) && (Qout != QKV || (ldq != ldqkv && !one))) ||
      (overlap(Kout, ldk, wk, QKV, ldqkv, w, s->M) && (Kout != in + wq || (ldk != ldqkv && !one))))
    return NTP_ERR_INVALID_ARG;
  if (h->device < 0) return NTP_ERR_NO_DEVICE;
  AppendArgs a{};
  a.QKV = in, a.Qout = static_cast<uint16_t*>(Qout), a.Kout = static_cast<uint16_t*>(Kout);
  a.positions = positions, a.inv_freq = inv_freq;
  if (cache) {
    a.K = static_cast<uint16_t*>(cache->K), a.V = static_cast<uint16_t*>(cache->V), a.slots = slots;
    a.page_stride = cache->page_stride, a.page_size = cache->page_size, a.page_log2 = ntp::log2_of(cache->page_size);
    a.n_slots = cache->n_pages * cache->page_size;
  }
  a.M = s->M, a.ldqkv = ldqkv, a.ldq = ldq, a.ldk = ldk;
  a.q_cnt = s->q_cnt, a.kv_cnt = s->kv_cnt, a.head_dim = s->head_dim, a.rotary_dim = s->rotary_dim, a.interleaved = s->interleaved != 0;
  a.tokens = 1;
  hipStream_t hs = static_cast<hipStream_t>(stream);
  if (ntp::timing_on(h))
    ntp::timing_begin(h, stream, "kv_append", 0.0, 2.0 * double(s->M) * double(w + (Qout ? wq : 0) + (Kout ? wk : 0) + (cache ? 2 * wk : 0)));
  hipLaunchKernelGGL(kv_append_kernel, dim3(uint32_t((s->M + a.tokens - 1) / a.tokens)), dim3(kThreads), 0, hs, a);
  const bool ok = hipGetLastError() == hipSuccess;
  ntp::timing_end(h, stream);
  return ok ? NTP_OK : NTP_ERR_LAUNCH;
}
