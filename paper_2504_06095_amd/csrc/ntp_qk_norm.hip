// Norms of query and key heads with the rotation, the append to pages of either format in the same pass (ntp_qk_norm_append_shard), and their gradient
// (ntp_qk_norm_shard_bwd).
//
// Forward: x -> R(x rstd .* gamma), rstd = 1 / sqrt(sum x^2 / d + eps), R the rotation of ntp_kv_append.hip; a head is 8 lanes (d = 64: 4) of 16 elements, so its sums
// and its maximum are three (two) lane exchanges and the row is read once.  8-bit pages: e = the smallest exponent with max <= 448 * 2^e, stored are the e4m3
// numbers nearest to the values times 2^-e, which is exact: the only rounding is e4m3's, half a step of 2^-4.
// Backward: with u = R^T dy, xh = x rstd and w = u .* gamma:  dx = rstd (w - xh (w . xh) / d),  dgamma = sum over tokens and heads of u .* xh.  rstd is formed again
// from x, which the gradient reads anyway: nothing is kept by the forward call.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "ntp_internal.h"
#include "ntp_kv_cache.h"

namespace {

using ntp::off16;
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256, kMaxTokens = 8, kMaxPairs = 64;

__device__ __forceinline__ float bf_lo(uint32_t v) { return __builtin_bit_cast(float, v << 16); }
__device__ __forceinline__ float bf_hi(uint32_t v) { return __builtin_bit_cast(float, v & 0xffff0000u); }
__device__ __forceinline__ uint32_t bf_pack(float lo, float hi) {  // round to nearest even
  return uint32_t(__builtin_bit_cast(uint16_t, static_cast<__bf16>(lo))) | uint32_t(__builtin_bit_cast(uint16_t, static_cast<__bf16>(hi))) << 16;
}
__device__ __forceinline__ u32x4 load_16(const uint16_t* p) { return *reinterpret_cast<const u32x4*>(p); }
__device__ __forceinline__ void store_16(uint16_t* p, u32x4 v) { __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(p)); }
__device__ __forceinline__ void unpack(u32x4 v, float (&f)[8]) {
#pragma unroll
  for (int k = 0; k < 4; ++k) f[2 * k] = bf_lo(v[k]), f[2 * k + 1] = bf_hi(v[k]);
}
__device__ __forceinline__ u32x4 pack(const float (&f)[8]) { return u32x4{bf_pack(f[0], f[1]), bf_pack(f[2], f[3]), bf_pack(f[4], f[5]), bf_pack(f[6], f[7])}; }

// Over the 4 or 8 lanes of a head, left in all of them: lanes 1 and 2 apart, then the quads of 8 lanes.
template <int CTRL>
__device__ __forceinline__ float from(float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, false));
}
template <int D, typename F>
__device__ __forceinline__ float over_head(float v, F&& f) {
  v = f(v, from<0xb1>(v));
  v = f(v, from<0x4e>(v));
  if constexpr (D == 128) v = f(v, from<0x141>(v));
  return v;
}
__device__ __forceinline__ float add(float a, float b) { return a + b; }
// Sum over the lanes of a wavefront with the same number in their heads, left in all of them.
template <int D>
__device__ __forceinline__ float over_same(float v) {
  v += from<0x128>(v);  // rows of 16 lanes, turned by 8 (and by 4)
  if constexpr (D == 64) v += from<0x124>(v);
  {
    const uint32_t x = __builtin_bit_cast(uint32_t, v);
    const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    const uint32_t r0 = r[0], r1 = r[1];
    v = __builtin_bit_cast(float, r0) + __builtin_bit_cast(float, r1);
  }
  const uint32_t x = __builtin_bit_cast(uint32_t, v);
  const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
  const uint32_t r0 = r[0], r1 = r[1];
  return __builtin_bit_cast(float, r0) + __builtin_bit_cast(float, r1);
}

// cos and sin of the positions' angles of a workgroup's tokens, formed and reduced to less than half a turn in fp64
__device__ __forceinline__ void angles(float2 (*cs)[kMaxPairs], const int32_t* positions, const double* inv_freq, int64_t row0, int rows, int half) {
  for (int i = threadIdx.x; i < rows * half; i += kThreads) {
    const int t = i / half, p = i % half;
    double turns = double(positions[row0 + t]) * inv_freq[p] * 0.15915494309189533577;  // 1 / (2 pi)
    turns -= rint(turns);
    float s, c;
    sincospif(2.0f * float(turns), &s, &c);
    cs[t][p] = float2{c, s};
  }
}

// The pairs of 8 + 8 elements of a lane (chunks c0 and c1 of its head) turned by their angles, or back by -1.
__device__ __forceinline__ void turn(float (&x)[8], float (&y)[8], const float2* cs, bool interleaved, float sign) {
  if (interleaved) {  // neighbours: x holds pairs 0 .. 3, y the next four
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float2 p = cs[k], q = cs[k + 4];
      const float ps = sign * p.y, qs = sign * q.y, x0 = x[2 * k], x1 = x[2 * k + 1], y0 = y[2 * k], y1 = y[2 * k + 1];
      x[2 * k] = x0 * p.x - x1 * ps, x[2 * k + 1] = x1 * p.x + x0 * ps;
      y[2 * k] = y0 * q.x - y1 * qs, y[2 * k + 1] = y1 * q.x + y0 * qs;
    }
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float2 p = cs[k];
      const float s = sign * p.y, a = x[k], b = y[k];
      x[k] = a * p.x - b * s, y[k] = b * p.x + a * s;
    }
  }
}

struct AppendArgs {
  const uint16_t *QKV, *q_gamma, *k_gamma;
  uint16_t *Qout, *Kout;
  unsigned char *K, *V;  // pages
  uint8_t *K_exp, *V_exp;
  const int32_t* positions;
  const int64_t* slots;
  const double* inv_freq;
  int64_t M, ldqkv, ldq, ldk, page_stride, exp_stride, n_slots;
  int32_t q_cnt, kv_cnt, rotary_dim, interleaved, page_size, page_log2, tokens;
  float eps;
};

// 8 values as e4m3, in units of the power of two `down` is the reciprocal of; what is not finite becomes NaN
__device__ __forceinline__ u32x2 to_e4m3(const float (&f)[8], float down) {
  u32x2 out;
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    float u[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      u[k] = f[4 * w + k] * down;
      u[k] = __builtin_fmaf(u[k], 0.0f, u[k]);  // infinities to NaN
    }
    const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(u[0], u[1], 0, false);
    out[w] = uint32_t(__builtin_amdgcn_cvt_pk_fp8_f32(u[2], u[3], lo, true));
  }
  return out;
}

template <int D, bool FP8>
__global__ __launch_bounds__(kThreads) void qk_norm_append_kernel(const AppendArgs a) {
  constexpr int kHead = D / 16, kLog2 = D == 128 ? 3 : 2;  // lanes of a head
  __shared__ float2 cs[kMaxTokens][kMaxPairs];
  __shared__ int64_t slot_of[kMaxTokens];
  const int64_t row0 = int64_t(blockIdx.x) * a.tokens;
  const int rows = int(std::min<int64_t>(a.tokens, a.M - row0));
  const int j = int(threadIdx.x) & (kHead - 1), rot = a.rotary_dim / 16;
  const bool turned = j < rot;
  // this lane's 8 + 8 elements of a query or key head: pairs number 8 j .. 8 j + 7, or two chunks behind the rotated part; of a value head
  const int c0 = (turned ? (a.interleaved ? 2 * j : j) : 2 * j) * 8, c1 = (turned ? (a.interleaved ? 2 * j + 1 : j + rot) : 2 * j + 1) * 8;
  const int v0 = j * 8, v1 = (j + kHead) * 8;
  const int heads = a.q_cnt + 2 * a.kv_cnt, per_row = heads << kLog2;
  int t = int(threadIdx.x) / per_row, at = int(threadIdx.x) % per_row;
  const int dt = kThreads / per_row, dat = kThreads % per_row;
  constexpr int kItems = 2;  // of a thread, whose loads go out together; the first ones before the angles are formed
  int tn[kItems], hn[kItems];
  u32x4 xw[kItems], yw[kItems];
  auto fetch = [&] {
#pragma unroll
    for (int n = 0; n < kItems; ++n) {
      tn[n] = t, hn[n] = at >> kLog2;
      if (t < rows) {
        const bool v = hn[n] >= a.q_cnt + a.kv_cnt;
        const uint16_t* const src = a.QKV + (row0 + t) * a.ldqkv + int64_t(hn[n]) * D;
        xw[n] = load_16(src + (v ? v0 : c0));
        yw[n] = load_16(src + (v ? v1 : c1));
      }
      t += dt;
      at += dat;
      if (at >= per_row) at -= per_row, ++t;
    }
  };
  fetch();
  if (int(threadIdx.x) < rows) slot_of[threadIdx.x] = a.slots ? a.slots[row0 + threadIdx.x] : -1;
  u32x4 gq0{}, gq1{}, gk0{}, gk1{};
  if (a.q_gamma) gq0 = load_16(a.q_gamma + c0), gq1 = load_16(a.q_gamma + c1);
  if (a.k_gamma) gk0 = load_16(a.k_gamma + c0), gk1 = load_16(a.k_gamma + c1);
  angles(cs, a.positions, a.inv_freq, row0, rows, a.rotary_dim / 2);
  __syncthreads();

  while (tn[0] < rows) {
#pragma unroll
    for (int n = 0; n < kItems; ++n) {
      if (tn[n] >= rows) continue;  // (all lanes of a head together)
      const int head = hn[n];
      const int64_t row = row0 + tn[n];
      const bool is_q = head < a.q_cnt, is_v = head >= a.q_cnt + a.kv_cnt;
      const bool norm = is_q ? a.q_gamma != nullptr : !is_v && a.k_gamma != nullptr;
      float x[8], y[8];
      unpack(xw[n], x);
      unpack(yw[n], y);
      if (norm) {
        float ss = 0.f;
#pragma unroll
        for (int k = 0; k < 8; ++k) ss = fmaf(x[k], x[k], fmaf(y[k], y[k], ss));
        ss = over_head<D>(ss, add);
        const float rstd = rsqrtf(ss * (1.0f / D) + a.eps);
        float g[8];
        unpack(is_q ? gq0 : gk0, g);
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = x[k] * rstd * g[k];
        unpack(is_q ? gq1 : gk1, g);
#pragma unroll
        for (int k = 0; k < 8; ++k) y[k] = y[k] * rstd * g[k];
      }
      if (turned && !is_v) turn(x, y, &cs[tn[n]][8 * j], a.interleaved, 1.0f);
      const bool changed = norm || (turned && !is_v);  // (what is copied is copied bit for bit)
      const u32x4 xb = changed ? pack(x) : xw[n], yb = changed ? pack(y) : yw[n];
      const int g = is_v ? head - a.q_cnt - a.kv_cnt : head - a.q_cnt;
      uint16_t* const out = is_q ? (a.Qout ? a.Qout + row * a.ldq + int64_t(head) * D : nullptr) : !is_v && a.Kout ? a.Kout + row * a.ldk + int64_t(g) * D : nullptr;
      if (out) {
        store_16(out + c0, xb);
        store_16(out + c1, yb);
      }
      const int64_t slot = slot_of[tn[n]];
      if (is_q || slot < 0 || slot >= a.n_slots) continue;
      const int64_t page = slot >> a.page_log2, in_head = int64_t(g) * a.page_size + (slot & (a.page_size - 1)), place = page * a.page_stride + in_head * D;
      const int p0 = is_v ? v0 : c0, p1 = is_v ? v1 : c1;
      if constexpr (!FP8) {
        uint16_t* const to = reinterpret_cast<uint16_t*>(is_v ? a.V : a.K) + place;
        store_16(to + p0, xb);
        store_16(to + p1, yb);
      } else {
        float top = 0.f;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const float p = fabsf(x[k]), q = fabsf(y[k]);
          top = fmaxf(top, fmaxf(p < INFINITY ? p : 0.f, q < INFINITY ? q : 0.f));
        }
        top = over_head<D>(top, [](float p, float q) { return fmaxf(p, q); });
        // 448 = 1.75 * 2^8: one more than the exponent of top / 2^8 where its mantissa is above 1.75
        int code = int((__builtin_bit_cast(uint32_t, top) + 0x1fffffu) >> 23) - 8;
        code = top == 0.f ? 127 : std::max(code, 16);
        const float down = __builtin_bit_cast(float, uint32_t(254 - code) << 23);
        unsigned char* const to = (is_v ? a.V : a.K) + place;
        *reinterpret_cast<u32x2*>(to + p0) = to_e4m3(x, down);
        *reinterpret_cast<u32x2*>(to + p1) = to_e4m3(y, down);
        if (j == 0) (is_v ? a.V_exp : a.K_exp)[page * a.exp_stride + in_head] = uint8_t(code);
      }
    }
    fetch();
  }
}

// ---- gradient ---------------------------------------------------------------------------------------
// The query heads' part and the key heads' have workgroups of their own (fewer registers than sums of both gammas in one: 4 wavefronts a SIMD more).
struct BwdSide {
  const uint16_t *x, *up, *gamma;  // the first head's columns of QKV, its gradient, and the weights of its norm (NULL: none)
  uint16_t* out;                   // the first head's columns of dQKV
  float* d_gamma;                  // where parts is NULL: one workgroup of the side writes it itself; NULL: not wanted
  int64_t ldup;
  int32_t heads, tokens, wgs, wanted;  // heads; tokens of a workgroup at a time; workgroups; whether the gamma's gradient is formed
};
struct BwdArgs {
  BwdSide q, k;
  float* parts;  // [workgroup][D] partial sums of the gammas' gradients
  const int32_t* positions;
  const double* inv_freq;
  int64_t M, ldx, ldout;
  int32_t rotary_dim, interleaved, accumulate, store;
  float eps;
};

template <int D>
__global__ __launch_bounds__(kThreads) void qk_norm_bwd_kernel(const BwdArgs a) {
  constexpr int kHead = D / 16, kLog2 = D == 128 ? 3 : 2;
  __shared__ float2 cs[kMaxTokens][kMaxPairs];
  __shared__ float sums[kThreads / 64][D];
  const bool is_q = int(blockIdx.x) < a.q.wgs;
  const BwdSide& s = is_q ? a.q : a.k;
  const int wg = int(blockIdx.x) - (is_q ? 0 : a.q.wgs);
  const int j = int(threadIdx.x) & (kHead - 1), rot = a.rotary_dim / 16;
  const bool turned = j < rot;
  const int c0 = (turned ? (a.interleaved ? 2 * j : j) : 2 * j) * 8, c1 = (turned ? (a.interleaved ? 2 * j + 1 : j + rot) : 2 * j + 1) * 8;
  u32x4 gw0{}, gw1{};
  if (s.gamma) gw0 = load_16(s.gamma + c0), gw1 = load_16(s.gamma + c1);
  float dg[16] = {};
  const int per_row = s.heads << kLog2;
  const int dt = kThreads / per_row, dat = kThreads % per_row;
  for (int64_t row0 = int64_t(wg) * s.tokens; row0 < a.M; row0 += int64_t(s.wgs) * s.tokens) {
    const int rows = int(std::min<int64_t>(s.tokens, a.M - row0));
    int t = int(threadIdx.x) / per_row, at = int(threadIdx.x) % per_row;
    u32x4 xw[4];
    auto fetch = [&] {
      if (t >= rows) return;
      const int64_t row = row0 + t, col = int64_t(at >> kLog2) * D;
      const uint16_t *const src = s.x + row * a.ldx + col, *const up = s.up + row * s.ldup + col;
      xw[0] = load_16(src + c0), xw[1] = load_16(src + c1), xw[2] = load_16(up + c0), xw[3] = load_16(up + c1);
    };
    fetch();  // (on its way while the angles are formed)
    __syncthreads();  // the angles of the rows before have been used
    angles(cs, a.positions, a.inv_freq, row0, rows, a.rotary_dim / 2);
    __syncthreads();
    while (t < rows) {
      float x[8], y[8], u[8], w[8];
      unpack(xw[0], x);
      unpack(xw[1], y);
      unpack(xw[2], u);
      unpack(xw[3], w);
      uint16_t* const out = s.out + (row0 + t) * a.ldout + int64_t(at >> kLog2) * D;
      const float2* const angle = &cs[t][8 * j];
      t += dt;
      at += dat;
      if (at >= per_row) at -= per_row, ++t;
      fetch();
      if (turned) turn(u, w, angle, a.interleaved, -1.0f);
      if (s.gamma) {
        float g0[8], g1[8], ss = 0.f, dot = 0.f;
        unpack(gw0, g0);
        unpack(gw1, g1);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          ss = fmaf(x[k], x[k], fmaf(y[k], y[k], ss));
          dot = fmaf(u[k] * g0[k], x[k], fmaf(w[k] * g1[k], y[k], dot));
        }
        ss = over_head<D>(ss, add);
        dot = over_head<D>(dot, add);
        const float rstd = rsqrtf(ss * (1.0f / D) + a.eps), mean = dot * rstd * (1.0f / D);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const float xh = x[k] * rstd, yh = y[k] * rstd;
          dg[k] = fmaf(u[k], xh, dg[k]), dg[8 + k] = fmaf(w[k], yh, dg[8 + k]);
          u[k] = (u[k] * g0[k] - xh * mean) * rstd;
          w[k] = (w[k] * g1[k] - yh * mean) * rstd;
        }
      }
      if (a.store) {
        store_16(out + c0, pack(u));
        store_16(out + c1, pack(w));
      }
    }
  }
  if (!s.wanted) return;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
#pragma unroll
  for (int k = 0; k < 16; ++k) dg[k] = over_same<D>(dg[k]);
  if (lane < kHead) {
#pragma unroll
    for (int k = 0; k < 8; ++k) sums[wave][c0 + k] = dg[k], sums[wave][c1 + k] = dg[8 + k];
  }
  __syncthreads();
  const int c = threadIdx.x;
  if (c >= D) return;
  const float v = (sums[0][c] + sums[1][c]) + (sums[2][c] + sums[3][c]);
  if (a.parts) a.parts[int64_t(blockIdx.x) * D + c] = v;
  else s.d_gamma[c] = a.accumulate ? s.d_gamma[c] + v : v;
}

// Adds up the partial sums of one gamma's gradient (blockIdx.y; the first n_q are the query heads'), 16 columns a workgroup, 64 of them side by side.
constexpr int kSumThreads = 1024;
template <int D>
__global__ __launch_bounds__(kSumThreads) void qk_norm_sum_kernel(const float* parts, int n_q, int n_k, float* d_q, float* d_k, int accumulate) {
  __shared__ float rows[64][17];
  float* const out = blockIdx.y == 0 ? d_q : d_k;
  if (!out) return;
  const int n = blockIdx.y == 0 ? n_q : n_k, c = threadIdx.x & 15, r = threadIdx.x >> 4, col = int(blockIdx.x) * 16 + c;
  parts += blockIdx.y == 0 ? 0 : int64_t(n_q) * D;
  float sum = 0.f;
#pragma unroll 8
  for (int i = r; i < n; i += 64) sum += parts[int64_t(i) * D + col];
  rows[r][c] = sum;
  __syncthreads();
  for (int half = 32; half > 0; half /= 2) {
    if (r < half) rows[r][c] += rows[r + half][c];
    __syncthreads();
  }
  if (r == 0) out[col] = accumulate ? out[col] + rows[0][c] : rows[0][c];
}

int check_shape(const ntp_kv_append_shape_t* s) {
  if (!s || s->M < 0 || s->q_cnt < 0 || s->kv_cnt < 0 || s->rotary_dim < 0) return NTP_ERR_INVALID_ARG;
  if (s->head_dim != 64 && s->head_dim != 128) return NTP_ERR_UNSUPPORTED;
  if (s->rotary_dim > s->head_dim || s->rotary_dim % 16) return NTP_ERR_INVALID_ARG;
  const int64_t w = (s->q_cnt + 2 * int64_t(s->kv_cnt)) * s->head_dim;
  return s->M > 0x7fffffffll || w > 0x7fffffffll / 16 ? NTP_ERR_UNSUPPORTED : NTP_OK;
}
int check_norm(const ntp_qk_norm_t* n) {
  if (!n || (!n->q_gamma && !n->k_gamma)) return NTP_OK;
  if (!(n->eps > 0.f) || !std::isfinite(n->eps)) return NTP_ERR_INVALID_ARG;
  return off16(n->q_gamma) || off16(n->k_gamma) ? NTP_ERR_ALIGNMENT : NTP_OK;
}
bool off(const void* p, int bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) != 0; }
// Tokens of a workgroup: at least an item for every thread where rows are short (as ntp_kv_append.hip), as long as there are `wgs` workgroups.
int32_t tokens_of(int64_t M, int64_t items_per_row, int64_t wgs) {
  const int64_t most = std::max<int64_t>(1, std::min<int64_t>(kMaxTokens, 384 / std::max<int64_t>(items_per_row, 1)));
  return int32_t(std::max<int64_t>(1, std::min(most, M / wgs)));
}

// Workgroups of both sides of the gradient, in proportion to their heads: up to four on every compute unit.
void bwd_sides(const ntp_handle* h, const ntp_kv_append_shape_t* s, BwdSide* q, BwdSide* k) {
  const int64_t all = 4 * int64_t(h->compute_units), heads = std::max(s->q_cnt + s->kv_cnt, 1);
  auto side = [&](BwdSide* d, int32_t n) {
    const int64_t room = std::max<int64_t>(1, all * n / heads);
    d->heads = n;
    d->tokens = tokens_of(s->M, int64_t(n) * (s->head_dim / 16), std::max<int64_t>(1, room / 2));
    d->wgs = n == 0 ? 0 : int32_t(std::min<int64_t>((s->M + d->tokens - 1) / d->tokens, room));
  };
  side(q, s->q_cnt);
  side(k, s->kv_cnt);
}

}  // namespace

int ntp::qk_norm_workspace_wish(const ntp_handle* h, const ntp_kv_append_shape_t* s, int64_t* bytes) {
  const int st = check_shape(s);
  if (st != NTP_OK) return NTP_ERR_INVALID_ARG;
  BwdSide q{}, k{};
  bwd_sides(h, s, &q, &k);
  *bytes = s->M == 0 || q.wgs + k.wgs <= 2 ? 0 : int64_t(q.wgs + k.wgs) * s->head_dim * 4;
  return NTP_OK;
}

extern "C" int ntp_qk_norm_append_shard(ntp_handle_t* h, const ntp_kv_append_shape_t* s, const ntp_qk_norm_t* norm, const ntp_kv_pages_t* pages, const void* QKV,
                                        int64_t ldqkv, const int32_t* positions, const int64_t* slots, const double* inv_freq, void* Qout, int64_t ldq, void* Kout,
                                        int64_t ldk, void* stream) {
  if (!h) return NTP_ERR_INVALID_ARG;
  int st = check_shape(s);
  if (st != NTP_OK || (st = check_norm(norm)) != NTP_OK) return st;
  if (s->M > 0 && (pages != nullptr) != (slots != nullptr)) return NTP_ERR_INVALID_ARG;
  if (pages && (st = ntp::check_kv_pages(pages, s->kv_cnt, s->head_dim)) != NTP_OK) return st;
  const int64_t d = s->head_dim, wq = s->q_cnt * d, wk = s->kv_cnt * d, w = wq + 2 * wk;
  if (s->M == 0 || w == 0 || (!Qout && !Kout && !pages)) return NTP_OK;
  if (!QKV || (s->rotary_dim > 0 && (!positions || !inv_freq)) || ldqkv < w || (Qout && ldq < wq) || (Kout && ldk < wk)) return NTP_ERR_INVALID_ARG;
  if (off16(QKV) || off16(Qout) || off16(Kout) || ldqkv % 8 || (Qout && ldq % 8) || (Kout && ldk % 8) || off(positions, 4) || off(slots, 8) || off(inv_freq, 8))
    return NTP_ERR_ALIGNMENT;
  const uint16_t* in = static_cast<const uint16_t*>(QKV);
  const bool one = s->M == 1;  // (a leading dimension does not count then)
  if ((ntp::rows_overlap(Qout, ldq, wq, QKV, ldqkv, w, s->M) && (Qout != QKV || (ldq != ldqkv && !one))) ||
      (ntp::rows_overlap(Kout, ldk, wk, QKV, ldqkv, w, s->M) && (Kout != in + wq || (ldk != ldqkv && !one))) || ntp::rows_overlap(Qout, ldq, wq, Kout, ldk, wk, s->M))
    return NTP_ERR_INVALID_ARG;
  AppendArgs a{};
  a.tokens = tokens_of(s->M, w / 16, 2 * int64_t(h->compute_units));
  if ((s->M + a.tokens - 1) / a.tokens * kThreads > 0xffffffffll) return NTP_ERR_UNSUPPORTED;  // a launch counts its threads in 32 bits
  if (h->device < 0) return NTP_ERR_NO_DEVICE;
  a.QKV = in, a.Qout = static_cast<uint16_t*>(Qout), a.Kout = static_cast<uint16_t*>(Kout);
  a.positions = positions, a.inv_freq = inv_freq;
  if (norm) a.q_gamma = static_cast<const uint16_t*>(norm->q_gamma), a.k_gamma = static_cast<const uint16_t*>(norm->k_gamma), a.eps = norm->eps;
  const bool fp8 = pages && pages->format == NTP_KV_E4M3;
  if (pages) {
    a.K = static_cast<unsigned char*>(pages->K), a.V = static_cast<unsigned char*>(pages->V), a.slots = slots;
    a.K_exp = static_cast<uint8_t*>(pages->K_exp), a.V_exp = static_cast<uint8_t*>(pages->V_exp);
    a.page_stride = pages->page_stride, a.exp_stride = pages->exp_stride, a.page_size = pages->page_size, a.page_log2 = ntp::log2_of(pages->page_size);
    a.n_slots = pages->n_pages * pages->page_size;
  }
  a.M = s->M, a.ldqkv = ldqkv, a.ldq = ldq, a.ldk = ldk;
  a.q_cnt = s->q_cnt, a.kv_cnt = s->kv_cnt, a.rotary_dim = s->rotary_dim, a.interleaved = s->interleaved != 0;
  hipStream_t hs = static_cast<hipStream_t>(stream);
  if (ntp::timing_on(h))
    ntp::timing_begin(h, stream, fp8 ? "qk_norm_append8" : "qk_norm_append", 0.0,
                      2.0 * double(s->M) * double(w + (Qout ? wq : 0) + (Kout ? wk : 0)) + double(s->M) * double(pages ? 2 * wk : 0) * (fp8 ? 1 : 2));
  const dim3 grid{uint32_t((s->M + a.tokens - 1) / a.tokens)};
  if (d == 128 && fp8) hipLaunchKernelGGL((qk_norm_append_kernel<128, true>), grid, dim3(kThreads), 0, hs, a);
  else if (d == 128) hipLaunchKernelGGL((qk_norm_append_kernel<128, false>), grid, dim3(kThreads), 0, hs, a);
  else if (fp8) hipLaunchKernelGGL((qk_norm_append_kernel<64, true>), grid, dim3(kThreads), 0, hs, a);
  else hipLaunchKernelGGL((qk_norm_append_kernel<64, false>), grid, dim3(kThreads), 0, hs, a);
  const bool ok = hipGetLastError() == hipSuccess;
  ntp::timing_end(h, stream);
  return ok ? NTP_OK : NTP_ERR_LAUNCH;
}

extern "C" int ntp_qk_norm_shard_bwd(ntp_handle_t* h, const ntp_kv_append_shape_t* s, const ntp_qk_norm_t* norm, const void* QKV, int64_t ldqkv, const void* dQ,
                                     int64_t lddq, const void* dK, int64_t lddk, const int32_t* positions, const double* inv_freq, void* dQKV, int64_t lddqkv,
                                     float* d_q_gamma, float* d_k_gamma, int32_t accumulate, void* stream) {
  if (!h) return NTP_ERR_INVALID_ARG;
  int st = check_shape(s);
  if (st != NTP_OK || (st = check_norm(norm)) != NTP_OK) return st;
  if ((d_q_gamma && (!norm || !norm->q_gamma)) || (d_k_gamma && (!norm || !norm->k_gamma))) return NTP_ERR_INVALID_ARG;
  const int64_t d = s->head_dim, wq = s->q_cnt * d, wk = s->kv_cnt * d, w = wq + 2 * wk;
  if (off(d_q_gamma, 4) || off(d_k_gamma, 4)) return NTP_ERR_ALIGNMENT;
  const bool rows = s->M > 0 && wq + wk > 0;
  if (rows) {
    if (!QKV || !dQKV || (wq > 0 && !dQ) || (wk > 0 && !dK) || (s->rotary_dim > 0 && (!positions || !inv_freq)) || ldqkv < w || lddqkv < w || (wq > 0 && lddq < wq) ||
        (wk > 0 && lddk < wk))
      return NTP_ERR_INVALID_ARG;
    if (off16(QKV) || off16(dQ) || off16(dK) || off16(dQKV) || ldqkv % 8 || (wq > 0 && lddq % 8) || (wk > 0 && lddk % 8) || lddqkv % 8 || off(positions, 4) || off(inv_freq, 8))
      return NTP_ERR_ALIGNMENT;
    uint16_t* const out = static_cast<uint16_t*>(dQKV);
    const bool one = s->M == 1;
    if (ntp::rows_overlap(dQKV, lddqkv, wq + wk, QKV, ldqkv, wq + wk, s->M) ||
        (ntp::rows_overlap(dQKV, lddqkv, wq + wk, dQ, lddq, wq, s->M) && (dQ != dQKV || (lddq != lddqkv && !one))) ||
        (ntp::rows_overlap(dQKV, lddqkv, wq + wk, dK, lddk, wk, s->M) && (dK != out + wq || (lddk != lddqkv && !one))))
      return NTP_ERR_INVALID_ARG;
  } else if (!d_q_gamma && !d_k_gamma) {
    return NTP_OK;
  }
  if (h->device < 0) return NTP_ERR_NO_DEVICE;
  BwdArgs a{};
  bwd_sides(h, s, &a.q, &a.k);
  a.q.x = static_cast<const uint16_t*>(QKV), a.k.x = a.q.x + wq, a.q.up = static_cast<const uint16_t*>(dQ), a.k.up = static_cast<const uint16_t*>(dK);
  a.q.out = static_cast<uint16_t*>(dQKV), a.k.out = a.q.out + wq, a.q.ldup = lddq, a.k.ldup = lddk;
  if (norm) a.q.gamma = static_cast<const uint16_t*>(norm->q_gamma), a.k.gamma = static_cast<const uint16_t*>(norm->k_gamma), a.eps = norm->eps;
  a.positions = positions, a.inv_freq = inv_freq, a.M = rows ? s->M : 0, a.ldx = ldqkv, a.ldout = lddqkv;
  a.rotary_dim = s->rotary_dim, a.interleaved = s->interleaved != 0, a.accumulate = accumulate;
  if (!rows) a.q.wgs = a.k.wgs = 0;
  hipStream_t hs = static_cast<hipStream_t>(stream);
  const bool sums = d_q_gamma || d_k_gamma, few = a.q.wgs <= 1 && a.k.wgs <= 1, room = h->workspace && h->workspace_bytes >= int64_t(a.q.wgs + a.k.wgs) * d * 4;
  auto launch = [&] {
    const dim3 grid{uint32_t(a.q.wgs + a.k.wgs)};
    if (d == 128) hipLaunchKernelGGL(qk_norm_bwd_kernel<128>, grid, dim3(kThreads), 0, hs, a);
    else hipLaunchKernelGGL(qk_norm_bwd_kernel<64>, grid, dim3(kThreads), 0, hs, a);
    return hipGetLastError() == hipSuccess;
  };
  auto add_up = [&](float* d_q, float* d_k) {
    const dim3 grid{uint32_t(d / 16), 2};
    if (d == 128) hipLaunchKernelGGL(qk_norm_sum_kernel<128>, grid, dim3(kSumThreads), 0, hs, a.parts, a.q.wgs, a.k.wgs, d_q, d_k, accumulate);
    else hipLaunchKernelGGL(qk_norm_sum_kernel<64>, grid, dim3(kSumThreads), 0, hs, a.parts, a.q.wgs, a.k.wgs, d_q, d_k, accumulate);
    return hipGetLastError() == hipSuccess;
  };
  if (ntp::timing_on(h)) ntp::timing_begin(h, stream, "qk_norm_bwd", 0.0, 6.0 * double(a.M) * double(wq + wk));
  bool ok = true;
  a.store = 1;
  a.q.wanted = d_q_gamma != nullptr, a.k.wanted = d_k_gamma != nullptr;
  if (sums && room && !few) {
    a.parts = static_cast<float*>(h->workspace);
    ok = launch() && add_up(d_q_gamma, d_k_gamma);
  } else {
    if (sums) {
      float* const none_q = a.q.wgs == 0 ? d_q_gamma : nullptr;  // a sum over no heads or no tokens
      float* const none_k = a.k.wgs == 0 ? d_k_gamma : nullptr;
      if (none_q || none_k) ok = add_up(none_q, none_k);
      a.q.d_gamma = d_q_gamma, a.k.d_gamma = d_k_gamma;
      if (!few) {  // one workgroup of each side forms them, before dQKV may take the place of dQ and dK
        const int32_t n_q = a.q.wgs, n_k = a.k.wgs;
        a.q.wgs = std::min(n_q, 1), a.k.wgs = std::min(n_k, 1), a.store = 0;
        ok = ok && launch();
        a.q.wgs = n_q, a.k.wgs = n_k, a.store = 1, a.q.wanted = a.k.wanted = 0;
      }
    }
    if (a.q.wgs + a.k.wgs > 0) ok = ok && launch();
  }
  ntp::timing_end(h, stream);
  return ok ? NTP_OK : NTP_ERR_LAUNCH;
}
