// Rotation of the query and key heads and appending of keys and values to the paged cache (ntp_kv_append_shard).
//
// Pair i of a head, (x1, x2), becomes (x1 cos a - x2 sin a, x2 cos a + x1 sin a) with a = position * inv_freq[i]: the angle is formed and reduced to
// less than half a turn in fp64 (positions of 10^5 times a frequency of 1 leave fp32 two digits), its sine and cosine are fp32.  A workgroup takes a few
// tokens, computes their sines and cosines once for all heads, and then streams the heads, 32 bytes an item; what bounds it is HBM (6 operations a pair; 8192 tokens,
// 42 heads of 128: 206 MB in 32 us, 6.4 TB/s), and at a few tokens the launch itself (64 tokens, 5 heads: 3.0 us).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <cstdlib>

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

__device__ __forceinline__ u32x4 load_16(const uint16_t* p) { return *reinterpret_cast<const u32x4*>(p); }
// Past the caches: a prompt's rows fit none of them (8192 tokens, 42 heads of 128: 45 -> 32 us; small launches do not care).  Loads stay as they are: the
// two chunks of a pair take half of a cache line each, which would be fetched twice (42 us).
__device__ __forceinline__ void store_16(uint16_t* p, u32x4 v) { __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(p)); }

constexpr int kItems = 2;  // of a thread, whose loads go out together

// Where a pair of 16-byte chunks of a head comes from and goes to.
struct Item {
  const uint16_t* src;
  uint16_t *out, *cache;  // (NULL: nowhere)
  int c0, c1;             // elements in the head
  const float2* angles;   // sine and cosine of its eight pairs; NULL: not rotated
};

__global__ __launch_bounds__(kThreads) void kv_append_kernel(const AppendArgs a) {
  __shared__ float2 cs[kMaxTokens][kMaxPairs];
  __shared__ int64_t slot_of[kMaxTokens];
  const int64_t row0 = int64_t(blockIdx.x) * a.tokens;
  const int rows = int(std::min<int64_t>(a.tokens, a.M - row0));
  const int half = a.rotary_dim / 2;
  if (int(threadIdx.x) < rows) slot_of[threadIdx.x] = a.slots ? a.slots[row0 + threadIdx.x] : -1;
  for (int i = threadIdx.x; i < rows * half; i += kThreads) {
    const int t = i / half, p = i % half;
    double turns = double(a.positions[row0 + t]) * a.inv_freq[p] * 0.15915494309189533577;  // 1 / (2 pi)
    turns -= rint(turns);
    float s, c;
    sincospif(2.0f * float(turns), &s, &c);
    cs[t][p] = float2{c, s};
  }
  __syncthreads();
  const int log2_head = a.head_dim == 128 ? 3 : 2, per_head = 1 << log2_head;  // pairs of chunks in a head
  const int per_row = (a.q_cnt + 2 * a.kv_cnt) << log2_head, rot = a.rotary_dim / 16;
  // item `at` of row t of the workgroup: head by head, the pairs of chunks in order
  auto describe = [&](int t, int at) {
    Item it{};
    const int head = at >> log2_head, j = at & (per_head - 1);
    const int64_t row = row0 + t;
    const bool is_q = head < a.q_cnt, is_v = head >= a.q_cnt + a.kv_cnt, rotate = !is_v && j < rot;
    const int g = is_v ? head - a.q_cnt - a.kv_cnt : head - a.q_cnt;
    // pairs number 8 j .. 8 j + 7, or two chunks behind the rotated part
    it.c0 = (rotate ? (a.interleaved ? 2 * j : j) : is_v ? j : 2 * j) * 8;
    it.c1 = (rotate ? (a.interleaved ? 2 * j + 1 : j + rot) : is_v ? j + per_head : 2 * j + 1) * 8;
    if (rotate) it.angles = &cs[t][8 * j];
    it.src = a.QKV + row * a.ldqkv + int64_t(head) * a.head_dim;
    if (is_q && a.Qout) it.out = a.Qout + row * a.ldq + int64_t(head) * a.head_dim;
    if (!is_q && !is_v && a.Kout) it.out = a.Kout + row * a.ldk + int64_t(g) * a.head_dim;
    const int64_t slot = slot_of[t];
    if (!is_q && slot >= 0 && slot < a.n_slots)
      it.cache = (is_v ? a.V : a.K) + (slot >> a.page_log2) * a.page_stride + (int64_t(g) * a.page_size + (slot & (a.page_size - 1))) * a.head_dim;
    return it;
  };
  int t = int(threadIdx.x) / per_row, at = int(threadIdx.x) % per_row;
  const int dt = kThreads / per_row, dat = kThreads % per_row;
  while (t < rows) {
    Item it[kItems];
    u32x4 x[kItems], y[kItems];
#pragma unroll
    for (int n = 0; n < kItems; ++n) {
      it[n] = Item{};
      if (t < rows) it[n] = describe(t, at);
      if (it[n].out || it[n].cache) {
        x[n] = load_16(it[n].src + it[n].c0);
        y[n] = load_16(it[n].src + it[n].c1);
      }
      t += dt;
      at += dat;
      if (at >= per_row) {
        at -= per_row;
        ++t;
      }
    }
#pragma unroll
    for (int n = 0; n < kItems; ++n) {
      if (it[n].angles) {
        u32x4 u, w;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float xl = bf_lo(x[n][k]), xh = bf_hi(x[n][k]), yl = bf_lo(y[n][k]), yh = bf_hi(y[n][k]);
          if (a.interleaved) {  // words are pairs: x holds numbers 8 j .. 8 j + 3, y the next four
            const float2 p = it[n].angles[k], q = it[n].angles[k + 4];
            u[k] = bf_pack(xl * p.x - xh * p.y, xh * p.x + xl * p.y);
            w[k] = bf_pack(yl * q.x - yh * q.y, yh * q.x + yl * q.y);
          } else {
            const float2 p = it[n].angles[2 * k], q = it[n].angles[2 * k + 1];
            u[k] = bf_pack(xl * p.x - yl * p.y, xh * q.x - yh * q.y);
            w[k] = bf_pack(yl * p.x + xl * p.y, yh * q.x + xh * q.y);
          }
        }
        x[n] = u;
        y[n] = w;
      }
      if (it[n].out) {
        store_16(it[n].out + it[n].c0, x[n]);
        store_16(it[n].out + it[n].c1, y[n]);
      }
      if (it[n].cache) {
        store_16(it[n].cache + it[n].c0, x[n]);
        store_16(it[n].cache + it[n].c1, y[n]);
      }
    }
  }
}

// Whether two views of bf16 rows share an element.  With one leading dimension their columns are compared, modulo it: row i of a lies i - j leading dimensions
// and the bases' distance from row j of b.  With two of them the whole spans are.
bool overlap(const void* a, int64_t lda, int64_t wa, const void* b, int64_t ldb, int64_t wb, int64_t rows) {
  const char *p = static_cast<const char*>(a), *q = static_cast<const char*>(b);
  if (!p || !q || wa == 0 || wb == 0 || p >= q + ((rows - 1) * ldb + wb) * 2 || q >= p + ((rows - 1) * lda + wa) * 2) return false;
  if (lda != ldb || rows == 1) return true;
  const int64_t off = (p - q) / 2;
  int64_t column = off % lda, row = off / lda;  // of a's first element in b
  if (column < 0) column += lda, --row;
  // a's rows begin in b's at that column (row 0 of a in row `row` of b), and reach into the next ones' where they pass the leading dimension
  return (column < wb && std::abs(row) < rows) || (column + wa > lda && std::abs(row + 1) < rows);
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
      (overlap(Kout, ldk, wk, QKV, ldqkv, w, s->M) && (Kout != in + wq || (ldk != ldqkv && !one))) || overlap(Qout, ldq, wq, Kout, ldk, wk, s->M))
    return NTP_ERR_INVALID_ARG;
  const int64_t per_row = (w / d) * (d / 16), most = std::max<int64_t>(1, std::min(int64_t(kMaxTokens), 384 / per_row));  // items of a row; tokens of a workgroup
  if ((s->M + most - 1) / most * kThreads > 0xffffffffll) return NTP_ERR_UNSUPPORTED;  // a launch counts its threads in 32 bits
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
  // at least an item for every thread where rows are short, as long as there are two workgroups for every compute unit (8192 tokens, 5 heads: 1 / 4 / 8 tokens a
  // workgroup 10.3 / 6.4 / 6.7 us, 20 heads: 1 / 2 / 4 tokens 16.6 / 15.7 / 16.0 us, 42 heads: 32 / 35 / 36 us)
  a.tokens = int32_t(std::max<int64_t>(1, std::min(most, s->M / (2 * h->compute_units))));
  hipStream_t hs = static_cast<hipStream_t>(stream);
  if (ntp::timing_on(h))
    ntp::timing_begin(h, stream, "kv_append", 0.0, 2.0 * double(s->M) * double(w + (Qout ? wq : 0) + (Kout ? wk : 0) + (cache ? 2 * wk : 0)));
  hipLaunchKernelGGL(kv_append_kernel, dim3(uint32_t((s->M + a.tokens - 1) / a.tokens)), dim3(kThreads), 0, hs, a);
  const bool ok = hipGetLastError() == hipSuccess;
  ntp::timing_end(h, stream);
  return ok ? NTP_OK : NTP_ERR_LAUNCH;
}
