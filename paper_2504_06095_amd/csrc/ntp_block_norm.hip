// Norms of a block with its gate and residual, forward and backward (ntp_block_norm_fwd, ntp_block_norm_bwd).
//
// Per row of H elements (t = Z or X', per norm):  hat = (t - mean) rstd,  mean = sum t / H (0 for RMS),  rstd = (sum (t - mean)^2 / H + eps)^-1/2
//   r = hat_z gp + bp (or Z),   X' = a X + b g r,   Y = hat_x gn + bn.
// Backward, from the rows' mean and rstd that the forward call kept:
//   u = dY gn,  G = dX' + rstd_x (u - mean_H(u) - hat_x mean_H(u hat_x))          (mean_H(u) for the layer norm only)
//   dX = a G,   dr = b G g,   dg = b G r,   v = dr gp,   dZ = rstd_z (v - mean_H(v) - hat_z mean_H(v hat_z))
//   dgn = sum dY hat_x,  dbn = sum dY,  dgp = sum dr hat_z,  dbp = sum dr,  and dg summed likewise for a gate per channel (sums over the rows).
//
// One workgroup takes a row at a time; a thread holds the row's 16-byte chunks tid, tid + threads, ... in registers, so that every matrix is read and
// written once.  What bounds both directions is HBM: 8 to 18 bytes an element against some 20 operations.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "ntp_internal.h"

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kMaxThreads = 1024, kMaxWaves = kMaxThreads / 64;
constexpr int kVectors = 5;  // gradients that are sums over the rows: gp, bp, gate, gn, bn
constexpr int64_t kMaxH = 32768;

struct NormArgs {
  const void* X;  // X (forward) or X' (backward)
  const uint16_t* Z;
  void* Xout;     // forward: X'; backward: dX
  uint16_t* Y;    // forward: Y;  backward: dZ
  const void* dXout;
  const uint16_t* dY;
  float* Stats;
  const uint16_t *pg, *pb, *gate, *ng, *nb;
  uint16_t* dgate_rows;  // NTP_GATE_TOKEN
  float* sums[kVectors];  // where the sums over the rows go (NULL: not wanted)
  float* parts;           // [groups][wanted sums][H] partial sums; NULL with one group, whose sums go to `sums`
  int64_t ldx, ldz, ldxo, ldy, lddxo, lddy, ldgate, lddgate, M;
  int32_t H, layer, gate_kind, xf32, accumulate, n_sums;
  float eps, a, b, inv_h;
};

__device__ __forceinline__ float bf_lo(uint32_t v) { return __builtin_bit_cast(float, v << 16); }
__device__ __forceinline__ float bf_hi(uint32_t v) { return __builtin_bit_cast(float, v & 0xffff0000u); }
__device__ __forceinline__ uint32_t bf_pack(float lo, float hi) {  // round to nearest even
  return uint32_t(__builtin_bit_cast(uint16_t, static_cast<__bf16>(lo))) | uint32_t(__builtin_bit_cast(uint16_t, static_cast<__bf16>(hi))) << 16;
}
__device__ __forceinline__ void load8(const uint16_t* p, float (&v)[8]) {
  const u32x4 r = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = bf_lo(r[i]);
    v[2 * i + 1] = bf_hi(r[i]);
  }
}
__device__ __forceinline__ void store8(uint16_t* p, const float (&v)[8]) {
  u32x4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = bf_pack(v[2 * i], v[2 * i + 1]);
  *reinterpret_cast<u32x4*>(p) = r;
}
// elements `at` .. `at` + 7 of a bf16 or fp32 matrix
__device__ __forceinline__ void load8x(const void* p, int64_t at, int f32, float (&v)[8]) {
  if (f32) {
    const f32x4* q = reinterpret_cast<const f32x4*>(static_cast<const float*>(p) + at);
    const f32x4 lo = q[0], hi = q[1];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[i] = lo[i];
      v[4 + i] = hi[i];
    }
  } else {
    load8(static_cast<const uint16_t*>(p) + at, v);
  }
}
__device__ __forceinline__ void store8x(void* p, int64_t at, int f32, const float (&v)[8]) {
  if (f32) {
    f32x4* q = reinterpret_cast<f32x4*>(static_cast<float*>(p) + at);
    q[0] = f32x4{v[0], v[1], v[2], v[3]};
    q[1] = f32x4{v[4], v[5], v[6], v[7]};
  } else {
    store8(static_cast<uint16_t*>(p) + at, v);
  }
}

// Sum over the wavefront, left in all lanes: inside 16 lanes by data-parallel moves (lane ^ 1, ^ 2, mirrored eight, mirrored sixteen), then the
// 16-lane rows and the halves trade places in registers.
template <int CTRL>
__device__ __forceinline__ float dpp_add(float v) {
  const int x = __builtin_bit_cast(int, v);
  return v + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, x, CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float wave_sum(float v) {
  v = dpp_add<0xB1>(v);
  v = dpp_add<0x4E>(v);
  v = dpp_add<0x141>(v);
  v = dpp_add<0x140>(v);
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

// Sums of N values over the workgroup, in the order of the wavefronts.  `turn` alternates between two sets of slots: a set is written again only
// after a barrier that every thread reaches behind its reads of it.
template <int N>
__device__ __forceinline__ void block_sum(float (&v)[N], float (*slots)[kMaxWaves][2], int& turn) {
  const int waves = blockDim.x >> 6;
#pragma unroll
  for (int n = 0; n < N; ++n) v[n] = wave_sum(v[n]);
  if (waves == 1) return;
  if ((threadIdx.x & 63) == 0) {
#pragma unroll
    for (int n = 0; n < N; ++n) slots[turn][threadIdx.x >> 6][n] = v[n];
  }
  __syncthreads();
#pragma unroll
  for (int n = 0; n < N; ++n) v[n] = 0.f;
  for (int w = 0; w < waves; ++w)
#pragma unroll
    for (int n = 0; n < N; ++n) v[n] += slots[turn][w][n];
  turn ^= 1;
}

// Mean and rstd of a row held in registers (columns behind H hold zeros).
template <int V>
__device__ __forceinline__ void row_stats(const NormArgs& a, const float (&t)[V][8], float& mean, float& rstd, float (*slots)[kMaxWaves][2], int& turn) {
  float s[1];
  mean = 0.f;
  if (a.layer) {
    s[0] = 0.f;
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int i = 0; i < 8; ++i) s[0] += t[v][i];
    block_sum<1>(s, slots, turn);
    mean = s[0] * a.inv_h;
  }
  s[0] = 0.f;
#pragma unroll
  for (int v = 0; v < V; ++v)
    if (int(threadIdx.x + v * blockDim.x) * 8 < a.H) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float d = t[v][i] - mean;
        s[0] = fmaf(d, d, s[0]);
      }
    }
  block_sum<1>(s, slots, turn);
  rstd = 1.0f / sqrtf(fmaf(s[0], a.inv_h, a.eps));
}

template <int V>
__global__ __launch_bounds__(kMaxThreads) void block_norm_fwd_kernel(const NormArgs a) {
  __shared__ float slots[2][kMaxWaves][2];
  int turn = 0;
  for (int64_t row = blockIdx.x; row < a.M; row += gridDim.x) {
    float x[V][8], z[V][8];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int c = int(threadIdx.x + v * blockDim.x) * 8;
#pragma unroll
      for (int i = 0; i < 8; ++i) x[v][i] = z[v][i] = 0.f;
      if (c < a.H) {
        load8x(a.X, row * a.ldx + c, a.xf32, x[v]);
        if (a.Z) load8(a.Z + row * a.ldz + c, z[v]);
      }
    }
    if (a.Z) {
      if (a.pg) {
        float mean, rstd;
        row_stats<V>(a, z, mean, rstd, slots, turn);
        if (a.Stats && threadIdx.x == 0) {
          a.Stats[row] = mean;
          a.Stats[a.M + row] = rstd;
        }
#pragma unroll
        for (int v = 0; v < V; ++v) {
          const int c = int(threadIdx.x + v * blockDim.x) * 8;
          if (c < a.H) {
            float g[8], b[8] = {};
            load8(a.pg + c, g);
            if (a.pb) load8(a.pb + c, b);
#pragma unroll
            for (int i = 0; i < 8; ++i) z[v][i] = fmaf((z[v][i] - mean) * rstd, g[i], b[i]);
          }
        }
      }
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const int c = int(threadIdx.x + v * blockDim.x) * 8;
        if (c < a.H) {
          float g[8];
          if (a.gate_kind != NTP_GATE_NONE) {
            load8(a.gate + (a.gate_kind == NTP_GATE_TOKEN ? row * a.ldgate : 0) + c, g);
#pragma unroll
            for (int i = 0; i < 8; ++i) z[v][i] *= g[i];
          }
#pragma unroll
          for (int i = 0; i < 8; ++i) x[v][i] = fmaf(a.a, x[v][i], a.b * z[v][i]);
          if (a.Xout) store8x(a.Xout, row * a.ldxo + c, a.xf32, x[v]);
        }
      }
    }
    if (a.ng) {
      float mean, rstd;
      row_stats<V>(a, x, mean, rstd, slots, turn);
      if (a.Stats && threadIdx.x == 0) {
        a.Stats[2 * a.M + row] = mean;
        a.Stats[3 * a.M + row] = rstd;
      }
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const int c = int(threadIdx.x + v * blockDim.x) * 8;
        if (c < a.H) {
          float g[8], b[8] = {}, y[8];
          load8(a.ng + c, g);
          if (a.nb) load8(a.nb + c, b);
#pragma unroll
          for (int i = 0; i < 8; ++i) y[i] = fmaf((x[v][i] - mean) * rstd, g[i], b[i]);
          store8(a.Y + row * a.ldy + c, y);
        }
      }
    }
  }
}

// Rows row0 .. row1 - 1 of a group; the sums over them stay in registers until the end.
template <int V>
__global__ __launch_bounds__(kMaxThreads) void block_norm_bwd_kernel(const NormArgs a) {
  __shared__ float slots[2][kMaxWaves][2];
  int turn = 0;
  float acc[kVectors][V][8] = {};
  const int64_t row0 = a.M * blockIdx.x / gridDim.x, row1 = a.M * (blockIdx.x + 1) / gridDim.x;
  for (int64_t row = row0; row < row1; ++row) {
    float G[V][8], x[V][8], z[V][8];
    float s[2] = {0.f, 0.f};
    const float mz = a.pg ? a.Stats[row] : 0.f, rz = a.pg ? a.Stats[a.M + row] : 1.f;
    const float mx = a.ng ? a.Stats[2 * a.M + row] : 0.f, rx = a.ng ? a.Stats[3 * a.M + row] : 0.f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int c = int(threadIdx.x + v * blockDim.x) * 8;
#pragma unroll
      for (int i = 0; i < 8; ++i) G[v][i] = x[v][i] = z[v][i] = 0.f;
      if (c < a.H) {
        if (a.dXout) load8x(a.dXout, row * a.lddxo + c, a.xf32, G[v]);
        if (a.Z) load8(a.Z + row * a.ldz + c, z[v]);
        if (a.ng) {
          float dy[8], g[8];
          load8(a.dY + row * a.lddy + c, dy);
          load8x(a.X, row * a.ldx + c, a.xf32, x[v]);
          load8(a.ng + c, g);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            x[v][i] = (x[v][i] - mx) * rx;  // hat_x
            acc[3][v][i] = fmaf(dy[i], x[v][i], acc[3][v][i]);
            acc[4][v][i] += dy[i];
            const float u = dy[i] * g[i];
            s[0] += u;
            s[1] = fmaf(u, x[v][i], s[1]);
            G[v][i] = fmaf(u, rx, G[v][i]);
          }
        }
      }
    }
    if (a.ng) {
      block_sum<2>(s, slots, turn);
      const float m0 = a.layer ? s[0] * a.inv_h * rx : 0.f, m1 = s[1] * a.inv_h * rx;
#pragma unroll
      for (int v = 0; v < V; ++v)
#pragma unroll
        for (int i = 0; i < 8; ++i) G[v][i] -= fmaf(x[v][i], m1, m0);
    }
    s[0] = s[1] = 0.f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int c = int(threadIdx.x + v * blockDim.x) * 8;
      if (c < a.H) {
        float o[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = a.a * G[v][i];
        store8x(a.Xout, row * a.ldxo + c, a.xf32, o);
        if (a.Y) {
          float g[8], p[8], q[8] = {};
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            G[v][i] *= a.b;
            p[i] = 1.f;
            z[v][i] = (z[v][i] - mz) * rz;  // hat_z, or Z itself
          }
          if (a.pg) load8(a.pg + c, p);
          if (a.pb) load8(a.pb + c, q);
          if (a.gate_kind != NTP_GATE_NONE) {
            load8(a.gate + (a.gate_kind == NTP_GATE_TOKEN ? row * a.ldgate : 0) + c, g);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const float dg = G[v][i] * fmaf(z[v][i], p[i], q[i]);
              acc[2][v][i] += dg;
              o[i] = dg;
              G[v][i] *= g[i];  // dr
            }
            if (a.dgate_rows) store8(a.dgate_rows + row * a.lddgate + c, o);
          }
          if (a.pg) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              acc[0][v][i] = fmaf(G[v][i], z[v][i], acc[0][v][i]);
              acc[1][v][i] += G[v][i];
              G[v][i] *= p[i];  // v
              s[0] += G[v][i];
              s[1] = fmaf(G[v][i], z[v][i], s[1]);
            }
          }
        }
      }
    }
    if (a.Y) {
      float m0 = 0.f, m1 = 0.f;
      if (a.pg) {
        block_sum<2>(s, slots, turn);
        m0 = a.layer ? s[0] * a.inv_h : 0.f;
        m1 = s[1] * a.inv_h;
      }
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const int c = int(threadIdx.x + v * blockDim.x) * 8;
        if (c < a.H) {
          float o[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) o[i] = (G[v][i] - fmaf(z[v][i], m1, m0)) * rz;
          store8(a.Y + row * a.ldy + c, o);
        }
      }
    }
  }
  int n = 0;
#pragma unroll
  for (int k = 0; k < kVectors; ++k) {
    if (!a.sums[k]) continue;
    float* dst = a.parts ? a.parts + (int64_t(blockIdx.x) * a.n_sums + n) * a.H : a.sums[k];
    ++n;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int c = int(threadIdx.x + v * blockDim.x) * 8;
      if (c < a.H) {
        f32x4* q = reinterpret_cast<f32x4*>(dst + c);
        f32x4 lo = {acc[k][v][0], acc[k][v][1], acc[k][v][2], acc[k][v][3]}, hi = {acc[k][v][4], acc[k][v][5], acc[k][v][6], acc[k][v][7]};
        if (!a.parts && a.accumulate) {
          lo += q[0];
          hi += q[1];
        }
        q[0] = lo;
        q[1] = hi;
      }
    }
  }
}

// The groups' partial sums added up in order: thread = one column of one vector.
__global__ __launch_bounds__(256) void block_norm_sum_kernel(const NormArgs a, int groups) {
  const int64_t at = int64_t(blockIdx.x) * 256 + threadIdx.x;
  if (at >= int64_t(a.n_sums) * a.H) return;
  const int n = int(at / a.H), c = int(at % a.H);
  float s = 0.f;
  for (int g = 0; g < groups; ++g) s += a.parts[(int64_t(g) * a.n_sums + n) * a.H + c];
  int k = 0;
  for (int left = n; k < kVectors; ++k)
    if (a.sums[k] && left-- == 0) break;
  a.sums[k][c] = a.accumulate ? a.sums[k][c] + s : s;
}

int check_norm_shape(const ntp_block_norm_shape_t* s) {
  if (!s || s->M < 0 || s->H < 0 || (s->norm != NTP_NORM_RMS && s->norm != NTP_NORM_LAYER) || s->gate < NTP_GATE_NONE || s->gate > NTP_GATE_TOKEN ||
      !(s->eps > 0.f) || !std::isfinite(s->eps) || !std::isfinite(s->residual_scale) || !std::isfinite(s->branch_scale))
    return NTP_ERR_INVALID_ARG;
  if (s->H % 8) return NTP_ERR_ALIGNMENT;
  if (s->H > kMaxH || s->M > 0x7fffffffll) return NTP_ERR_UNSUPPORTED;
  return NTP_OK;
}

// Rows of weights and their gate: what may and what must be there (branch: there is a Z).
int check_weights(const ntp_block_norm_shape_t* s, const ntp_block_norm_weights_t* w, bool branch) {
  if (!w || (w->post_beta && !w->post_gamma) || (w->pre_beta && !w->pre_gamma) || (s->gate != NTP_GATE_NONE) != (w->gate != nullptr) ||
      (!branch && (w->post_gamma || w->gate)) || (s->gate == NTP_GATE_TOKEN && w->ldgate < s->H))
    return NTP_ERR_INVALID_ARG;
  return NTP_OK;
}

bool off16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) != 0; }

// Rows are one workgroup's: at most two chunks of 8 columns a thread, four beyond 16384 columns.
int norm_threads(int64_t H) {
  const int64_t chunks = H / 8, v = chunks > 2 * kMaxThreads ? 4 : 2;
  return int(((chunks + v - 1) / v + 63) / 64 * 64);
}

// Workgroups that share out the rows of a backward call, each with partial sums of its own: one per compute unit.
int64_t norm_groups(const ntp_handle* h, const ntp_block_norm_shape_t* s) { return std::max<int64_t>(1, std::min<int64_t>(s->M, h->compute_units)); }

}  // namespace

int ntp::block_norm_workspace_wish(const ntp_handle* h, const ntp_block_norm_shape_t* s, int64_t* bytes) {
  if (check_norm_shape(s) != NTP_OK) return NTP_ERR_INVALID_ARG;
  const int64_t groups = norm_groups(h, s);
  *bytes = groups > 1 ? groups * kVectors * s->H * 4 : 0;
  return NTP_OK;
}

extern "C" int ntp_block_norm_fwd(ntp_handle_t* h, const ntp_block_norm_shape_t* s, const ntp_block_norm_weights_t* w, const void* X, int64_t ldx,
                                  const void* Z, int64_t ldz, void* Xout, int64_t ldxo, void* Y, int64_t ldy, float* Stats, void* stream) {
  int st = check_norm_shape(s);
  if (st != NTP_OK) return st;
  if (!h || (st = check_weights(s, w, Z != nullptr || s->M == 0)) != NTP_OK) return NTP_ERR_INVALID_ARG;  // (matrices without rows may be NULL)
  if (s->M == 0 || s->H == 0) return NTP_OK;
  if ((w->pre_gamma != nullptr) != (Y != nullptr) || (Xout && !Z)) return NTP_ERR_INVALID_ARG;
  if (!X || (!Xout && !Y)) return NTP_ERR_INVALID_ARG;
  if (ldx < s->H || (Z && ldz < s->H) || (Xout && ldxo < s->H) || (Y && ldy < s->H) || (Xout == X && ldxo != ldx)) return NTP_ERR_INVALID_ARG;
  const int64_t xm = s->residual_fp32 ? 4 : 8;
  if (off16(X) || off16(Z) || off16(Xout) || off16(Y) || off16(w->post_gamma) || off16(w->post_beta) || off16(w->gate) || off16(w->pre_gamma) ||
      off16(w->pre_beta) || ldx % xm || (Z && ldz % 8) || (Xout && ldxo % xm) || (Y && ldy % 8) || (s->gate == NTP_GATE_TOKEN && w->ldgate % 8) ||
      (reinterpret_cast<uintptr_t>(Stats) & 3))
    return NTP_ERR_ALIGNMENT;
  if (h->device < 0) return NTP_ERR_NO_DEVICE;
  NormArgs a{};
  a.X = X, a.Z = static_cast<const uint16_t*>(Z), a.Xout = Xout, a.Y = static_cast<uint16_t*>(Y), a.Stats = Stats;
  a.pg = static_cast<const uint16_t*>(w->post_gamma), a.pb = static_cast<const uint16_t*>(w->post_beta), a.gate = static_cast<const uint16_t*>(w->gate);
  a.ng = static_cast<const uint16_t*>(w->pre_gamma), a.nb = static_cast<const uint16_t*>(w->pre_beta);
  a.ldx = ldx, a.ldz = ldz, a.ldxo = ldxo, a.ldy = ldy, a.ldgate = w->ldgate, a.M = s->M;
  a.H = int32_t(s->H), a.layer = s->norm == NTP_NORM_LAYER, a.gate_kind = s->gate, a.xf32 = s->residual_fp32 != 0;
  a.eps = s->eps, a.a = s->residual_scale, a.b = s->branch_scale, a.inv_h = float(1.0 / double(s->H));
  hipStream_t hs = static_cast<hipStream_t>(stream);
  if (ntp::timing_on(h)) {
    const double n = double(s->M) * double(s->H), rt = a.xf32 ? 4 : 2;
    ntp::timing_begin(h, stream, "block_norm_fwd", 0.0, n * (rt + (Z ? 2 : 0) + (Xout ? rt : 0) + (Y ? 2 : 0) + (s->gate == NTP_GATE_TOKEN ? 2 : 0)));
  }
  const dim3 grid(uint32_t(s->M)), block(uint32_t(norm_threads(s->H)));
  if (s->H > 2 * 8 * kMaxThreads) hipLaunchKernelGGL(block_norm_fwd_kernel<4>, grid, block, 0, hs, a);
  else hipLaunchKernelGGL(block_norm_fwd_kernel<2>, grid, block, 0, hs, a);
  const bool ok = hipGetLastError() == hipSuccess;
  ntp::timing_end(h, stream);
  return ok ? NTP_OK : NTP_ERR_LAUNCH;
}

extern "C" int ntp_block_norm_bwd(ntp_handle_t* h, const ntp_block_norm_shape_t* s, const ntp_block_norm_weights_t* w, const void* dXout, int64_t lddxo,
                                  const void* dY, int64_t lddy, const void* Xout, int64_t ldxo, const void* Z, int64_t ldz, const float* Stats, void* dX,
                                  int64_t lddx, void* dZ, int64_t lddz, const ntp_block_norm_grads_t* grads, int32_t accumulate, void* stream) {
  int st = check_norm_shape(s);
  if (st != NTP_OK) return st;
  if (!h || !grads || (st = check_weights(s, w, dZ != nullptr || s->M == 0)) != NTP_OK) return NTP_ERR_INVALID_ARG;
  const bool post = w->post_gamma, pre = w->pre_gamma, gate = s->gate != NTP_GATE_NONE, reads_z = post || gate;
  if ((s->M > 0 && pre != (dY != nullptr)) || (!post && (grads->post_gamma || grads->post_beta)) || (!pre && (grads->pre_gamma || grads->pre_beta)) ||
      (!gate && grads->gate) || (grads->post_beta && !w->post_beta) || (grads->pre_beta && !w->pre_beta))
    return NTP_ERR_INVALID_ARG;
  if (s->H == 0) return NTP_OK;
  const bool token = s->gate == NTP_GATE_TOKEN;
  if (s->M > 0) {
    if (!dX || (pre && !Xout) || (reads_z && !Z) || ((post || pre) && !Stats)) return NTP_ERR_INVALID_ARG;
    if (lddx < s->H || (dXout && lddxo < s->H) || (pre && (lddy < s->H || ldxo < s->H)) || (reads_z && ldz < s->H) || (dZ && lddz < s->H) ||
        (token && grads->gate && grads->ldgate < s->H) || (dX == dXout && lddx != lddxo))
      return NTP_ERR_INVALID_ARG;
  }
  const int64_t xm = s->residual_fp32 ? 4 : 8;
  if (off16(dXout) || off16(dY) || off16(Xout) || off16(Z) || off16(dX) || off16(dZ) || off16(w->post_gamma) || off16(w->post_beta) || off16(w->gate) ||
      off16(w->pre_gamma) || off16(w->pre_beta) || off16(grads->post_gamma) || off16(grads->post_beta) || off16(grads->gate) || off16(grads->pre_gamma) ||
      off16(grads->pre_beta) || lddx % xm || (dXout && lddxo % xm) || (pre && (lddy % 8 || ldxo % xm)) || (reads_z && ldz % 8) || (dZ && lddz % 8) ||
      (token && (w->ldgate % 8 || (grads->gate && grads->ldgate % 8))) || (reinterpret_cast<uintptr_t>(Stats) & 3))
    return NTP_ERR_ALIGNMENT;
  if (h->device < 0) return NTP_ERR_NO_DEVICE;
  NormArgs a{};
  a.X = pre ? Xout : nullptr, a.Z = reads_z ? static_cast<const uint16_t*>(Z) : nullptr, a.Xout = dX, a.Y = static_cast<uint16_t*>(dZ);
  a.dXout = dXout, a.dY = static_cast<const uint16_t*>(dY), a.Stats = const_cast<float*>(Stats);
  a.pg = static_cast<const uint16_t*>(w->post_gamma), a.pb = static_cast<const uint16_t*>(w->post_beta), a.gate = static_cast<const uint16_t*>(w->gate);
  a.ng = static_cast<const uint16_t*>(w->pre_gamma);
  a.ldx = ldxo, a.ldz = ldz, a.ldxo = lddx, a.ldy = lddz, a.lddxo = lddxo, a.lddy = lddy, a.ldgate = w->ldgate, a.lddgate = grads->ldgate, a.M = s->M;
  a.H = int32_t(s->H), a.layer = s->norm == NTP_NORM_LAYER, a.gate_kind = s->gate, a.xf32 = s->residual_fp32 != 0, a.accumulate = accumulate != 0;
  a.a = dZ ? s->residual_scale : 1.0f, a.b = s->branch_scale, a.inv_h = float(1.0 / double(s->H));
  a.dgate_rows = token ? static_cast<uint16_t*>(grads->gate) : nullptr;
  a.sums[0] = grads->post_gamma, a.sums[1] = grads->post_beta, a.sums[2] = token ? nullptr : static_cast<float*>(grads->gate);
  a.sums[3] = grads->pre_gamma, a.sums[4] = grads->pre_beta;
  for (const float* p : a.sums) a.n_sums += p != nullptr;
  if (s->M == 0 && (a.n_sums == 0 || accumulate)) return NTP_OK;  // (the sums over no rows are zeros)
  int64_t groups = norm_groups(h, s);
  if (a.n_sums > 0) {
    groups = std::min<int64_t>(groups, h->workspace ? h->workspace_bytes / (int64_t(a.n_sums) * s->H * 4) : 0);
    a.parts = groups > 1 ? static_cast<float*>(h->workspace) : nullptr;
    groups = std::max<int64_t>(groups, 1);
  }
  hipStream_t hs = static_cast<hipStream_t>(stream);
  if (ntp::timing_on(h)) {
    const double n = double(s->M) * double(s->H), rt = a.xf32 ? 4 : 2;
    ntp::timing_begin(h, stream, "block_norm_bwd", 0.0,
                      n * (rt + (dXout ? rt : 0) + (pre ? 2 + rt : 0) + (a.Z ? 2 : 0) + (dZ ? 2 : 0) + (token ? 2 : 0) + (a.dgate_rows ? 2 : 0)));
  }
  const dim3 grid{uint32_t(groups)}, block(uint32_t(norm_threads(s->H)));
  if (s->H > 2 * 8 * kMaxThreads) hipLaunchKernelGGL(block_norm_bwd_kernel<4>, grid, block, 0, hs, a);
  else hipLaunchKernelGGL(block_norm_bwd_kernel<2>, grid, block, 0, hs, a);
  bool ok = hipGetLastError() == hipSuccess;
  if (ok && a.parts) {
    hipLaunchKernelGGL(block_norm_sum_kernel, dim3(uint32_t((int64_t(a.n_sums) * s->H + 255) / 256)), dim3(256), 0, hs, a, int(groups));
    ok = hipGetLastError() == hipSuccess;
  }
  ntp::timing_end(h, stream);
  return ok ? NTP_OK : NTP_ERR_LAUNCH;
}
