// Norms of query and key heads with the rotation, the append to pages of either format in the same pass (ntp_qk_norm_append_shard), and their gradient
// (ntp_qk_norm_shard_bwd).
//
// Forward: x -> R(x rstd .* gamma), rstd = 1 / sqrt(sum x^2 / d + eps), R the rotation of ntp_kv_append.hip; a head is 8 lanes (d = 64: 4) of 16 elements, so its sums
// and its maximum are three (two) lane exchanges and the row is read once.  8-bit pages: e = the smallest exponent with max <= 448 * 2^e, stored are the e4m3
// numbers nearest to the values times 2^-e, which is exact: the only rounding is e4m3's, half a step of 2^-4.
// Backward: with u = R^T dy, xh = x rstd and w = u .* gamma:  dx = rstd (w - xh (w . xh) / d),  dgamma = sum over tokens and heads of u .* xh.  rstd is formed again
// from x, which the gradient reads anyway: nothing is kept by the forward call.
//
// HBM bounds both: 8192 tokens, 14 heads of 128 of each kind, into 8-bit pages 32-35 us (5.0-5.5 TB/s; the vector unit issues for 86 % of it), into bf16 ones 32 (6.4), the gradient at 405B shape 26 us (5.1 TB/s) and 5
// in the second launch; small calls cost their launch (4 us).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <functional>

#include "ntp_internal.h"
#include "ntp_kv_cache.h"

namespace {

using ntp::off16;
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kMaxThreads = 1024, kMaxTokens = 8, kMaxPairs = 64;

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
// (what was unpacked from v before is unpacked again, and holds no registers in between)
__device__ __forceinline__ void anew(u32x4& v) {
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("" : "+v"(v));
#endif
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
__device__ __forceinline__ void angles(float2 (*cs)[kMaxPairs], const int32_t* positions, const double* inv_freq, int row0, int M, int tokens, int half, bool exact) {
  const int rows = min(tokens, M - row0);
#pragma unroll 1
  for (int i = threadIdx.x; i < rows * half; i += int(blockDim.x)) {
    const int t = i / half, p = i % half;
    double turns = double(positions[row0 + t]) * inv_freq[p] * 0.15915494309189533577;  // 1 / (2 pi)
    turns -= rint(turns);
    float s, c;
    const float near = float(turns);
    sincospif(2.0f * near, &s, &c);
    // What that rounding left of the angle, up to 9e-8, more than sine and cosine are rounded by.  Without norms the call is ntp_kv_append_shard's, bit for bit, which goes without.
    const float rest = exact ? float(turns - double(near)) * 6.28318530717958648f : 0.f;
    cs[t][p] = float2{fmaf(-s, rest, c), fmaf(c, rest, s)};
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

// How a workgroup takes its tokens: `tokens` at a time, kHead = head_dim / 16 lanes a head, so that a thread has one head of one of them and its weights in registers; rows of more
// heads than a workgroup has room for in several passes.  The next tokens' elements are on their way while these are worked on.
struct Deal {
  int32_t heads, tokens, threads, wgs;
};
template <int D>
struct Place {
  static constexpr int kHead = D / 16;
  int j, token, head, stride;  // number in the head, token of the workgroup's, head, heads of a pass
  int c0, c1;                  // a rotated head's elements: pairs number 8 j .. 8 j + 7, or two chunks behind the rotated part
  bool turned;
  __device__ __forceinline__ Place(const Deal& d, int rotary_dim, int interleaved) {
    j = int(threadIdx.x) & (kHead - 1);
    stride = min(d.heads, d.threads / kHead);
    token = (int(threadIdx.x) / kHead) / stride;
    head = (int(threadIdx.x) / kHead) % stride;
    const int rot = rotary_dim / 16;
    turned = j < rot;
    c0 = (turned ? (interleaved ? 2 * j : j) : 2 * j) * 8;
    c1 = (turned ? (interleaved ? 2 * j + 1 : j + rot) : 2 * j + 1) * 8;
  }
};

struct AppendArgs {
  Deal deal;
  const uint16_t *QKV, *q_gamma, *k_gamma;
  uint16_t *Qout, *Kout;
  unsigned char *K, *V;  // pages
  uint8_t *K_exp, *V_exp;
  const int32_t* positions;
  const int64_t* slots;
  const double* inv_freq;
  int64_t M, ldqkv, ldq, ldk, page_stride, exp_stride, n_slots;
  int32_t q_cnt, kv_cnt, rotary_dim, interleaved, page_size, page_log2;
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

// In units of 2^120 the number 256, next to values above 248, would be 2^128, which neither fp32 nor bf16 holds: 240 instead.  Codes 0x78 become 0x77; there are none between them and NaN.
__device__ __forceinline__ void most_240(u32x2& v, bool where) {
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    const uint32_t high = ((v[w] & 0x78787878u) + 0x08080808u) >> 7, nan = ((v[w] & 0x07070707u) + 0x01010101u) >> 3;
    v[w] -= where ? high & ~nan & 0x01010101u : 0u;
  }
}

template <int D, bool FP8>
__global__ __launch_bounds__(kMaxThreads) void qk_norm_append_kernel(const AppendArgs a) {
  __shared__ float2 cs[2][kMaxTokens][kMaxPairs];
  const Place<D> at(a.deal, a.rotary_dim, a.interleaved);
  const int M = int(a.M), step = int(gridDim.x) * a.deal.tokens, half = a.rotary_dim / 2;
  const bool exact = a.q_gamma || a.k_gamma;
  for (int head = at.head; head - at.head < a.deal.heads; head += at.stride) {  // (one pass but for very many heads)
    const bool is_q = head < a.q_cnt, is_v = head >= a.q_cnt + a.kv_cnt, mine = head < a.deal.heads && at.token < a.deal.tokens;
    const uint16_t* const gamma = is_q ? a.q_gamma : is_v ? nullptr : a.k_gamma;
    const bool turned = at.turned && !is_v;
    const int c0 = is_v ? at.j * 8 : at.c0, c1 = is_v ? (at.j + at.kHead) * 8 : at.c1, g = is_q ? head : head - a.q_cnt - (is_v ? a.kv_cnt : 0);
    u32x4 gw0{}, gw1{};
    if (gamma && mine) gw0 = load_16(gamma + c0), gw1 = load_16(gamma + c1);
    u32x4 xw{}, yw{};
    int64_t slot = -1;
    int row0 = int(blockIdx.x) * a.deal.tokens;
    // (not formed from the row each time: 64-bit products)
    const int64_t first = row0 + at.token, ldout = is_q ? a.ldq : a.ldk;
    const uint16_t* src = a.QKV + first * a.ldqkv + int64_t(head) * D;
    uint16_t* const out0 = is_q ? a.Qout : is_v ? nullptr : a.Kout;
    uint16_t* out = out0 + first * ldout + int64_t(g) * D;
    auto fetch = [&] {
      if (mine && row0 + at.token < M) {
        xw = load_16(src + c0);
        yw = load_16(src + c1);
        if (!is_q && a.slots) slot = a.slots[row0 + at.token];
      }
      src += int64_t(step) * a.ldqkv;
    };
    fetch();
    __syncthreads();  // (the pass before has used the angles)
    if (row0 < M) angles(cs[0], a.positions, a.inv_freq, row0, M, a.deal.tokens, half, exact);
    for (int buf = 0; row0 < M; buf ^= 1) {
      __syncthreads();
      const bool there = mine && row0 + at.token < M;
      const int64_t to_slot = slot;
      u32x4 xr = xw, yr = yw;
      row0 += step;
      fetch();
      if (there) {  // (all lanes of a head together)
        float x[8], y[8];
        unpack(xr, x);
        unpack(yr, y);
        if (gamma) {
          float ss = 0.f;
#pragma unroll
          for (int k = 0; k < 8; ++k) ss = fmaf(x[k], x[k], fmaf(y[k], y[k], ss));
          ss = over_head<D>(ss, add);
          // (products of two bf16 numbers are exact; a step of Newton's takes the reciprocal root from one step of fp32 to half of one: e4m3 borders show what fp32 loses)
          const float mean = ss * (1.0f / D) + a.eps, root = rsqrtf(mean);
          const float rstd = mean < INFINITY ? fmaf(0.5f * root, fmaf(-mean * root, root, 1.0f), root) : root;
          float w[8];
          unpack(gw0, w);
#pragma unroll
          for (int k = 0; k < 8; ++k) x[k] = x[k] * w[k] * rstd;
          unpack(gw1, w);
#pragma unroll
          for (int k = 0; k < 8; ++k) y[k] = y[k] * w[k] * rstd;
        }
        if (turned) turn(x, y, &cs[buf][at.token][8 * at.j], a.interleaved, 1.0f);
        const bool changed = gamma || turned;  // (what is copied is copied bit for bit)
        const u32x4 xb = changed ? pack(x) : xr, yb = changed ? pack(y) : yr;
        if (out0) {
          store_16(out + c0, xb);
          store_16(out + c1, yb);
        }
        if (!is_q && to_slot >= 0 && to_slot < a.n_slots) {
          const int64_t page = to_slot >> a.page_log2, in_head = int64_t(g) * a.page_size + (to_slot & (a.page_size - 1)), place = page * a.page_stride + in_head * D;
          if constexpr (!FP8) {
            uint16_t* const to = reinterpret_cast<uint16_t*>(is_v ? a.V : a.K) + place;
            store_16(to + c0, xb);
            store_16(to + c1, yb);
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
            code = top == 0.f ? 127 : max(code, 16);
            const float down = __builtin_bit_cast(float, uint32_t(254 - code) << 23);
            unsigned char* const to = (is_v ? a.V : a.K) + place;
            u32x2 x8 = to_e4m3(x, down), y8 = to_e4m3(y, down);
            if (__any(code > 246)) most_240(x8, code > 246), most_240(y8, code > 246);  // (nearly no wavefront)
            *reinterpret_cast<u32x2*>(to + c0) = x8;
            *reinterpret_cast<u32x2*>(to + c1) = y8;
            if (at.j == 0) (is_v ? a.V_exp : a.K_exp)[page * a.exp_stride + in_head] = uint8_t(code);
          }
        }
      }
      out += int64_t(step) * ldout;
      if (row0 < M) angles(cs[buf ^ 1], a.positions, a.inv_freq, row0, M, a.deal.tokens, half, exact);
    }
  }
}

// ---- gradient ---------------------------------------------------------------------------------------
struct BwdArgs {
  Deal deal;
  const uint16_t *QKV, *dQ, *dK, *q_gamma, *k_gamma;
  uint16_t* dQKV;            // NULL: the gammas' gradients alone
  float* parts;              // [workgroup][2][D] partial sums of the gammas' gradients
  float *d_q, *d_k;          // where parts is NULL: one workgroup writes what is wanted of them itself
  const int32_t* positions;
  const double* inv_freq;
  int64_t M, ldqkv, lddq, lddk, lddqkv;
  int32_t q_cnt, rotary_dim, interleaved, accumulate;
  float eps;
};

template <int D>
__global__ __launch_bounds__(kMaxThreads) void qk_norm_bwd_kernel(const BwdArgs a) {
  __shared__ float2 cs[2][kMaxTokens][kMaxPairs];
  __shared__ float sums[kMaxThreads / 64][2][D];
  const Place<D> at(a.deal, a.rotary_dim, a.interleaved);
  const int M = int(a.M), step = int(gridDim.x) * a.deal.tokens;
  const int half = a.rotary_dim / 2, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const bool wanted = a.parts || a.d_q || a.d_k, exact = a.q_gamma || a.k_gamma;
  if (wanted)
    for (int i = lane; i < 2 * D; i += 64) sums[wave][i / D][i % D] = 0.f;
  for (int head = at.head; head - at.head < a.deal.heads; head += at.stride) {  // (one pass but for very many heads)
    const bool is_q = head < a.q_cnt, mine = head < a.deal.heads && at.token < a.deal.tokens;
    const uint16_t* const gamma = is_q ? a.q_gamma : a.k_gamma;
    u32x4 gw0{}, gw1{};
    if (gamma && mine) gw0 = load_16(gamma + at.c0), gw1 = load_16(gamma + at.c1);
    float dg[16] = {};
    u32x4 xw{}, yw{}, uw{}, ww{};
    int row0 = int(blockIdx.x) * a.deal.tokens;
    // (not formed from the row each time: three 64-bit products)
    const int64_t first = row0 + at.token, up_step = int64_t(step) * (is_q ? a.lddq : a.lddk);
    const uint16_t* src = a.QKV + first * a.ldqkv + int64_t(head) * D;
    const uint16_t* up = is_q ? a.dQ + first * a.lddq + int64_t(head) * D : a.dK + first * a.lddk + int64_t(head - a.q_cnt) * D;
    uint16_t* out = a.dQKV + first * a.lddqkv + int64_t(head) * D;
    auto fetch = [&] {
      if (mine && row0 + at.token < M) xw = load_16(src + at.c0), yw = load_16(src + at.c1), uw = load_16(up + at.c0), ww = load_16(up + at.c1);
      src += int64_t(step) * a.ldqkv, up += up_step;
    };
    fetch();
    __syncthreads();  // (the pass before has used the angles)
    if (row0 < M) angles(cs[0], a.positions, a.inv_freq, row0, M, a.deal.tokens, half, exact);
    for (int buf = 0; row0 < M; buf ^= 1) {
      __syncthreads();
      const bool there = mine && row0 + at.token < M;
      u32x4 xr = xw, yr = yw;
      float x[8], y[8], u[8], w[8];
      unpack(uw, u);
      unpack(ww, w);
      row0 += step;
      fetch();
      if (there) {
        if (at.turned) turn(u, w, &cs[buf][at.token][8 * at.j], a.interleaved, -1.0f);
        if (gamma) {
          float g0[8], g1[8], ss = 0.f, dot = 0.f;
          unpack(xr, x);
          unpack(yr, y);
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
          anew(xr), anew(yr), anew(gw0), anew(gw1);
          unpack(xr, x);
          unpack(yr, y);
          unpack(gw0, g0);
          unpack(gw1, g1);
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const float xh = x[k] * rstd, yh = y[k] * rstd;
            dg[k] = fmaf(u[k], xh, dg[k]), dg[8 + k] = fmaf(w[k], yh, dg[8 + k]);
            u[k] = (u[k] * g0[k] - xh * mean) * rstd;
            w[k] = (w[k] * g1[k] - yh * mean) * rstd;
          }
        }
        if (a.dQKV) {
          store_16(out + at.c0, pack(u));
          store_16(out + at.c1, pack(w));
        }
      }
      out += int64_t(step) * a.lddqkv;
      if (row0 < M) angles(cs[buf ^ 1], a.positions, a.inv_freq, row0, M, a.deal.tokens, half, exact);
    }
    if (wanted) {  // heads of both kinds may stand in a wavefront: one kind after the other
#pragma unroll
      for (int kind = 0; kind < 2; ++kind) {
        if (!__any(mine && is_q == (kind == 0))) continue;
#pragma unroll
        for (int k = 0; k < 16; ++k) {
          const float v = over_same<D>(mine && is_q == (kind == 0) ? dg[k] : 0.f);
          if (lane < at.kHead) sums[wave][kind][(k < 8 ? at.c0 : at.c1 - 8) + k] += v;
        }
      }
    }
  }
  if (!wanted) return;
  __syncthreads();
  const int waves = int(blockDim.x) >> 6;
  for (int i = threadIdx.x; i < 2 * D; i += int(blockDim.x)) {
    const int kind = i / D, c = i % D;
    float v = 0.f;
    for (int k = 0; k < waves; ++k) v += sums[k][kind][c];
    float* const out = kind ? a.d_k : a.d_q;
    if (a.parts) a.parts[int64_t(blockIdx.x) * 2 * D + i] = v;
    else if (out) out[c] = a.accumulate ? out[c] + v : v;
  }
}

// Adds up n partial sums of one gamma's gradient (blockIdx.y), 16 columns a workgroup, 64 of them side by side.
template <int D>
__global__ __launch_bounds__(kMaxThreads) void qk_norm_sum_kernel(const float* parts, int n, float* d_q, float* d_k, int accumulate) {
  __shared__ float rows[64][17];
  float* const out = blockIdx.y == 0 ? d_q : d_k;
  if (!out) return;
  const int c = threadIdx.x & 15, r = threadIdx.x >> 4, col = int(blockIdx.x) * 16 + c;
  float sum = 0.f;
#pragma unroll 8
  for (int i = r; i < n; i += 64) sum += parts[int64_t(i) * 2 * D + blockIdx.y * D + col];
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
  return s->M > 0x7fffffffll - (1 << 20) || w > 0x7fffffffll / 16 ? NTP_ERR_UNSUPPORTED : NTP_OK;
}
int check_norm(const ntp_qk_norm_t* n) {
  if (!n || (!n->q_gamma && !n->k_gamma)) return NTP_OK;
  if (!(n->eps > 0.f) || !std::isfinite(n->eps)) return NTP_ERR_INVALID_ARG;
  return off16(n->q_gamma) || off16(n->k_gamma) ? NTP_ERR_ALIGNMENT : NTP_OK;
}
bool off(const void* p, int bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) != 0; }
constexpr int kAppendRoom = 2048, kBwdRoom = 1024;  // threads of a compute unit's workgroups
// Tokens at a time: as many as leave few of the workgroup's threads without a head, and fill half of the largest workgroup, as long as there are two workgroups for every compute
// unit; as many workgroups as the compute units have room for.
Deal deal_of(const ntp_handle* h, int64_t M, int32_t heads, int32_t head_dim, int32_t room) {
  Deal d{heads, 1, kMaxThreads, 0};
  const int64_t lanes = int64_t(heads) * (head_dim / 16);
  if (lanes == 0 || M == 0) return d;
  double best = 0;
  for (int32_t t = 1; t <= kMaxTokens && (t == 1 || (lanes * t <= kMaxThreads && M / t >= 2 * int64_t(h->compute_units))); ++t) {
    const int64_t threads = std::min<int64_t>(kMaxThreads, (lanes * t + 63) / 64 * 64);
    const double used = lanes > kMaxThreads ? 1.0 : double(lanes * t) / double(threads);
    if (used > best + 0.02 || (used > best - 0.02 && threads <= kMaxThreads / 2)) best = std::max(best, used), d.tokens = t, d.threads = int32_t(threads);
  }
  d.wgs = int32_t(std::min<int64_t>((M + d.tokens - 1) / d.tokens, int64_t(h->compute_units) * std::max(1, room / d.threads)));
  return d;
}

}  // namespace

int ntp::qk_norm_workspace_wish(const ntp_handle* h, const ntp_kv_append_shape_t* s, int64_t* bytes) {
  const int st = check_shape(s);
  if (st != NTP_OK) return NTP_ERR_INVALID_ARG;
  const Deal d = deal_of(h, s->M, s->q_cnt + s->kv_cnt, s->head_dim, kBwdRoom);
  *bytes = d.wgs <= 1 ? 0 : int64_t(d.wgs) * 2 * s->head_dim * 4;
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
  a.deal = deal_of(h, s->M, int32_t(w / d), s->head_dim, kAppendRoom);
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
  const dim3 grid{uint32_t(a.deal.wgs)}, block{uint32_t(a.deal.threads)};
  if (d == 128 && fp8) hipLaunchKernelGGL((qk_norm_append_kernel<128, true>), grid, block, 0, hs, a);
  else if (d == 128) hipLaunchKernelGGL((qk_norm_append_kernel<128, false>), grid, block, 0, hs, a);
  else if (fp8) hipLaunchKernelGGL((qk_norm_append_kernel<64, true>), grid, block, 0, hs, a);
  else hipLaunchKernelGGL((qk_norm_append_kernel<64, false>), grid, block, 0, hs, a);
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
  if (d_q_gamma && d_k_gamma && std::less<>{}(d_q_gamma, d_k_gamma + d) && std::less<>{}(d_k_gamma, d_q_gamma + d)) return NTP_ERR_INVALID_ARG;  // (they are written side by side)
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
  a.deal = deal_of(h, rows ? s->M : 0, s->q_cnt + s->kv_cnt, s->head_dim, kBwdRoom);
  a.QKV = static_cast<const uint16_t*>(QKV), a.dQ = static_cast<const uint16_t*>(dQ), a.dK = static_cast<const uint16_t*>(dK), a.dQKV = static_cast<uint16_t*>(dQKV);
  if (norm) a.q_gamma = static_cast<const uint16_t*>(norm->q_gamma), a.k_gamma = static_cast<const uint16_t*>(norm->k_gamma), a.eps = norm->eps;
  a.positions = positions, a.inv_freq = inv_freq, a.M = rows ? s->M : 0, a.ldqkv = ldqkv, a.lddq = lddq, a.lddk = lddk, a.lddqkv = lddqkv;
  a.q_cnt = s->q_cnt, a.rotary_dim = s->rotary_dim, a.interleaved = s->interleaved != 0, a.accumulate = accumulate;
  hipStream_t hs = static_cast<hipStream_t>(stream);
  const int32_t n = a.deal.wgs;
  const bool sums = d_q_gamma || d_k_gamma, room = h->workspace && h->workspace_bytes >= int64_t(n) * 2 * d * 4;
  auto launch = [&](int32_t wgs) {
    const dim3 grid{uint32_t(wgs)}, block{uint32_t(a.deal.threads)};
    if (d == 128) hipLaunchKernelGGL(qk_norm_bwd_kernel<128>, grid, block, 0, hs, a);
    else hipLaunchKernelGGL(qk_norm_bwd_kernel<64>, grid, block, 0, hs, a);
    return hipGetLastError() == hipSuccess;
  };
  auto add_up = [&] {
    const dim3 grid{uint32_t(d / 16), 2}, block{kMaxThreads};
    if (d == 128) hipLaunchKernelGGL(qk_norm_sum_kernel<128>, grid, block, 0, hs, a.parts, n, d_q_gamma, d_k_gamma, accumulate);
    else hipLaunchKernelGGL(qk_norm_sum_kernel<64>, grid, block, 0, hs, a.parts, n, d_q_gamma, d_k_gamma, accumulate);
    return hipGetLastError() == hipSuccess;
  };
  if (ntp::timing_on(h)) ntp::timing_begin(h, stream, "qk_norm_bwd", 0.0, 6.0 * double(a.M) * double(wq + wk));
  bool ok = true;
  if (n == 0) {  // a sum of nothing
    ok = add_up();
  } else if (sums && n > 1 && room) {
    a.parts = static_cast<float*>(h->workspace);
    ok = launch(n) && add_up();
  } else {
    if (sums) {  // one workgroup forms them, before dQKV may take the place of dQ and dK
      a.d_q = d_q_gamma, a.d_k = d_k_gamma;
      if (n > 1) a.dQKV = nullptr;
      ok = launch(1);
      a.d_q = a.d_k = nullptr, a.dQKV = static_cast<uint16_t*>(dQKV);
    }
    if (!sums || n > 1) ok = ok && launch(n);
  }
  ntp::timing_end(h, stream);
  return ok ? NTP_OK : NTP_ERR_LAUNCH;
}
