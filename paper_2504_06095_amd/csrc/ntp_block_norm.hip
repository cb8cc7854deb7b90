// Norms of a block with its gate and residual, forward and backward (ntp_block_norm_fwd, ntp_block_norm_bwd).
//
// Per row of H elements (t = Z or X', per norm):  hat = (t - mean) rstd,  mean = sum t / H (0 for RMS),  rstd = (sum (t - mean)^2 / H + eps)^-1/2
//   r = hat_z gp + bp (or Z),   X' = a X + b g r,   Y = hat_x gn + bn.
// Backward, from the rows' mean and rstd that the forward call kept:
//   u = dY gn,  G = dX' + rstd_x (u - mean_H(u) - hat_x mean_H(u hat_x))          (mean_H(u) for the layer norm only)
//   dX = a G,   dr = b G g,   dg = b G r,   v = dr gp,   dZ = rstd_z (v - mean_H(v) - hat_z mean_H(v hat_z))
//   dgn = sum dY hat_x,  dbn = sum dY,  dgp = sum dr hat_z,  dbp = sum dr,  and dg summed likewise for a gate per channel (sums over the rows).
//
// A row belongs to T threads (a power of two from 64 to 1024), which hold its 16-byte chunks tid, tid + T, ... in registers (V a thread), so that
// every matrix is read and written once; a workgroup takes several rows side by side where T is small.  What bounds both directions is HBM: 8 to 18 bytes an
// element against some 20 to 40 operations.  The backward kernel is persistent, one workgroup per compute unit that takes every gridDim-th set of rows, because the sums over
// the rows stay in its registers until the end; the next row's loads are in flight while this one's sums go round.  Measured: forward 8192 x 16384 188 us with a bf16
// residual stream (5.7 TB/s), 285 with an fp32 one (5.7), with a gate per token 234 and 347 (5.7, 5.4), 2048 x 12288 bf16 36 us (5.6); where a row leaves threads idle (T is a power
// of two) 4096 x 9216 68 (4.5), 4096 x 8456 66 (4.2), 8192 x 5120 66 (5.1).  Backward 8192 x 16384 with both norms and a gate 288 us (5.6), 4099 x 6144, fp32, 93 us (4.9 with a last turn
// of 3 rows for 256 workgroups); rows of more than 16384 columns are slow (block_norm_bwd_long_kernel).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <type_traits>

#include "ntp_internal.h"

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kMaxThreads = 1024, kMaxWaves = kMaxThreads / 64;
constexpr int kFwdThreads = 256, kBwdThreads = 512;  // of a workgroup, where a row has no more of its own
constexpr int kMaxV = 4;
constexpr int kSideBySide = 4;  // chunks of column sums in the LDS together (64 KB)
constexpr int kVectors = 5;  // gradients that are sums over the rows: gp, bp, gate, gn, bn
constexpr int64_t kMaxH = int64_t(kMaxThreads) * kMaxV * 8;

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
  int32_t H, layer, gate_kind, xf32, accumulate, n_sums, t_log2;  // (1 << t_log2: threads of a row)
  float eps, a, b, inv_h;
};

__device__ __forceinline__ float bf_lo(uint32_t v) { return __builtin_bit_cast(float, v << 16); }
__device__ __forceinline__ float bf_hi(uint32_t v) { return __builtin_bit_cast(float, v & 0xffff0000u); }
__device__ __forceinline__ uint32_t bf_pack(float lo, float hi) {  // round to nearest even
  return uint32_t(__builtin_bit_cast(uint16_t, static_cast<__bf16>(lo))) | uint32_t(__builtin_bit_cast(uint16_t, static_cast<__bf16>(hi))) << 16;
}
__device__ __forceinline__ void unpack8(u32x4 r, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = bf_lo(r[i]);
    v[2 * i + 1] = bf_hi(r[i]);
  }
}
__device__ __forceinline__ u32x4 pack8(const float (&v)[8]) {
  u32x4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = bf_pack(v[2 * i], v[2 * i + 1]);
  return r;
}

// A row of a matrix as a buffer view: what lies behind its H columns reads as zeros and is not written, so that the kernels have no branches
// (a wait for loads behind which a branch may or may not have issued stores would wait for these too).
__device__ __forceinline__ __amdgpu_buffer_rsrc_t row_view(const void* base, int64_t at, int elem, int columns) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(static_cast<const char*>(base) + at * elem), 0, columns * elem, 0x00020000);
}
// Rows go past the caches (NT: non-temporal) where a thread has more than one chunk: in the forward call many rows, or rows of more than 8192 columns however few; in the
// backward call all rows of more than 512 columns.  In large launches, whose matrices no cache holds until they are used again, it pays (8192 x 16384 forward 225 -> 202 us, backward
// 456 -> 376 us); what it costs the reader of a Y that the last-level cache would have kept was not measured.
template <bool NT>
__device__ __forceinline__ u32x4 load_16(__amdgpu_buffer_rsrc_t rs, uint32_t off) {
  return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rs, off, 0, NT ? 2 : 0));
}
template <bool NT>
__device__ __forceinline__ u32x2 load_8(__amdgpu_buffer_rsrc_t rs, uint32_t off) {
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(rs, off, 0, NT ? 2 : 0));
}
template <bool NT>
__device__ __forceinline__ void store_16(__amdgpu_buffer_rsrc_t rs, uint32_t off, u32x4 v) {
  __builtin_amdgcn_raw_buffer_store_b128(v, rs, off, 0, NT ? 2 : 0);
}
template <bool NT>
__device__ __forceinline__ void store_8(__amdgpu_buffer_rsrc_t rs, uint32_t off, u32x2 v) {
  __builtin_amdgcn_raw_buffer_store_b64(v, rs, off, 0, NT ? 2 : 0);
}

// The eight columns of a thread's chunk v: c0 .. c0 + 3 and c1 .. c1 + 3.  With a bf16 residual stream they are neighbours, 16 bytes of a row; with an fp32 one
// the wavefront's 512 columns are dealt out twice by fours, so that each instruction takes whole cache lines of fp32 rows (32 bytes a lane by two instructions took half of
// every line each: 4099 x 6144 backward 105 -> 102 us, 8192 x 16384 forward in bf16 with views 200 -> 192 us).
template <bool F32>
struct Cols {
  int c0, c1;
  __device__ __forceinline__ Cols(int tid, int v, int t_log2) {
    c0 = F32 ? ((tid & ~63) + (v << t_log2)) * 8 + (tid & 63) * 4 : (tid + (v << t_log2)) * 8;
    c1 = F32 ? c0 + 256 : c0 + 4;
  }
};
template <bool F32, bool NT>
__device__ __forceinline__ u32x4 load_bf(__amdgpu_buffer_rsrc_t rs, const Cols<F32>& c) {  // of a bf16 row
  if constexpr (!F32) return load_16<NT>(rs, uint32_t(c.c0) * 2);
  const u32x2 lo = load_8<NT>(rs, uint32_t(c.c0) * 2), hi = load_8<NT>(rs, uint32_t(c.c1) * 2);
  return u32x4{lo[0], lo[1], hi[0], hi[1]};
}
template <bool F32, bool NT>
__device__ __forceinline__ void store_bf(__amdgpu_buffer_rsrc_t rs, const Cols<F32>& c, const float (&v)[8]) {
  const u32x4 r = pack8(v);
  if constexpr (!F32) {
    store_16<NT>(rs, uint32_t(c.c0) * 2, r);
  } else {
    store_8<NT>(rs, uint32_t(c.c0) * 2, u32x2{r[0], r[1]});
    store_8<NT>(rs, uint32_t(c.c1) * 2, u32x2{r[2], r[3]});
  }
}
// Eight elements of the residual stream, bf16 or fp32, as they lie in memory.
template <bool F32>
struct Raw {
  u32x4 w[F32 ? 2 : 1];
  template <bool NT>
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t rs, const Cols<F32>& c) {
    w[0] = load_16<NT>(rs, uint32_t(c.c0) * (F32 ? 4 : 2));
    if constexpr (F32) w[1] = load_16<NT>(rs, uint32_t(c.c1) * 4);
  }
  __device__ __forceinline__ void get(float (&v)[8]) const {
    if constexpr (F32) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t lo = w[0][i], hi = w[1][i];
        v[i] = __builtin_bit_cast(float, lo);
        v[4 + i] = __builtin_bit_cast(float, hi);
      }
    } else {
      unpack8(w[0], v);
    }
  }
};
template <bool F32, bool NT>
__device__ __forceinline__ void store_x(__amdgpu_buffer_rsrc_t rs, const Cols<F32>& c, const float (&v)[8]) {
  if constexpr (F32) {
    u32x4 lo, hi;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      lo[i] = __builtin_bit_cast(uint32_t, v[i]);
      hi[i] = __builtin_bit_cast(uint32_t, v[4 + i]);
    }
    store_16<NT>(rs, uint32_t(c.c0) * 4, lo);
    store_16<NT>(rs, uint32_t(c.c1) * 4, hi);
  } else {
    store_bf<F32, NT>(rs, c, v);
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

// Sums of N values over the threads of a row, in the order of their wavefronts.  `turn` alternates between two sets of slots: a set is written
// again only after a barrier that every thread reaches behind its reads of it.
template <int N>
__device__ __forceinline__ void row_sum(int t_log2, float (&v)[N], float (*slots)[kMaxWaves][2], int& turn) {
#pragma unroll
  for (int n = 0; n < N; ++n) v[n] = wave_sum(v[n]);
  const int waves = 1 << (t_log2 - 6);
  if (waves == 1) return;
  const int wave = threadIdx.x >> 6, first = wave & ~(waves - 1);
  if ((threadIdx.x & 63) == 0) {
#pragma unroll
    for (int n = 0; n < N; ++n) slots[turn][wave][n] = v[n];
  }
  __syncthreads();
#pragma unroll
  for (int n = 0; n < N; ++n) v[n] = 0.f;
  for (int w = 0; w < waves; w += 2) {  // (two wavefronts a read)
    const f32x4 s = *reinterpret_cast<const f32x4*>(&slots[turn][first + w][0]);
    v[0] += s[0];
    v[0] += s[2];
    if constexpr (N > 1) {
      v[1] += s[1];
      v[1] += s[3];
    }
  }
  turn ^= 1;
}

// Mean and rstd of a row held in registers (columns behind H hold zeros).
template <int V, bool XF32>
__device__ __forceinline__ void row_stats(const NormArgs& a, int tid, const float (&t)[V][8], float& mean, float& rstd, float (*slots)[kMaxWaves][2], int& turn) {
  float s[1];
  mean = 0.f;
  if (a.layer) {
    s[0] = 0.f;
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int i = 0; i < 8; ++i) s[0] += t[v][i];
    row_sum<1>(a.t_log2, s, slots, turn);
    mean = s[0] * a.inv_h;
  }
  s[0] = 0.f;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const Cols<XF32> c(tid, v, a.t_log2);
#pragma unroll
    for (int half = 0; half < 2; ++half)
      if ((half ? c.c1 : c.c0) < a.H) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float d = t[v][half * 4 + i] - mean;
          s[0] = fmaf(d, d, s[0]);
        }
      }
  }
  row_sum<1>(a.t_log2, s, slots, turn);
  rstd = 1.0f / sqrtf(fmaf(s[0], a.inv_h, a.eps));
}

template <int V, bool XF32>
__global__ __launch_bounds__(kMaxThreads) void block_norm_fwd_kernel(const NormArgs a) {
  constexpr bool NT = V > 1;
  constexpr int XB = XF32 ? 4 : 2;
  __shared__ __attribute__((aligned(16))) float slots[2][kMaxWaves][2];
  int turn = 0;
  const int tid = threadIdx.x & ((1 << a.t_log2) - 1);
  const int lane_row = __builtin_amdgcn_readfirstlane(threadIdx.x >> a.t_log2);  // (T is a multiple of the wavefront)
  const int64_t row = (int64_t(blockIdx.x) * blockDim.x >> a.t_log2) + lane_row;
  const bool on = row < a.M;
  const int width = on ? a.H : 0;
  auto vec = [&](const uint16_t* p, int v, float (&o)[8]) { unpack8(load_bf<XF32, false>(row_view(p, 0, 2, a.H), Cols<XF32>(tid, v, a.t_log2)), o); };
  float x[V][8], z[V][8];
  const __amdgpu_buffer_rsrc_t vx = row_view(a.X, row * a.ldx, XB, width), vz = row_view(a.Z, row * a.ldz, 2, a.Z ? width : 0);
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const Cols<XF32> c(tid, v, a.t_log2);
    Raw<XF32> r;
    r.template load<NT>(vx, c);
    r.get(x[v]);
    if (a.Z) unpack8(load_bf<XF32, NT>(vz, c), z[v]);
  }
  if (a.Z) {
    if (a.pg) {
      float mean, rstd;
      row_stats<V, XF32>(a, tid, z, mean, rstd, slots, turn);
      if (a.Stats && on && tid == 0) {
        a.Stats[row] = mean;
        a.Stats[a.M + row] = rstd;
      }
#pragma unroll
      for (int v = 0; v < V; ++v) {
        float g[8], b[8] = {};
        vec(a.pg, v, g);
        if (a.pb) vec(a.pb, v, b);
#pragma unroll
        for (int i = 0; i < 8; ++i) z[v][i] = fmaf((z[v][i] - mean) * rstd, g[i], b[i]);
      }
    }
    const __amdgpu_buffer_rsrc_t vo = row_view(a.Xout, row * a.ldxo, XB, a.Xout ? width : 0);
    const bool token = a.gate_kind == NTP_GATE_TOKEN;
    const __amdgpu_buffer_rsrc_t vg = row_view(a.gate, token ? row * a.ldgate : 0, 2, token ? width : a.gate_kind == NTP_GATE_CHANNEL ? a.H : 0);
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const Cols<XF32> c(tid, v, a.t_log2);
      if (a.gate_kind != NTP_GATE_NONE) {
        float g[8];
        unpack8(load_bf<XF32, false>(vg, c), g);
#pragma unroll
        for (int i = 0; i < 8; ++i) z[v][i] *= g[i];
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) x[v][i] = fmaf(a.a, x[v][i], a.b * z[v][i]);
      if (a.Xout) store_x<XF32, NT>(vo, c, x[v]);
    }
  }
  if (a.ng) {
    float mean, rstd;
    row_stats<V, XF32>(a, tid, x, mean, rstd, slots, turn);
    if (a.Stats && on && tid == 0) {
      a.Stats[2 * a.M + row] = mean;
      a.Stats[3 * a.M + row] = rstd;
    }
    const __amdgpu_buffer_rsrc_t vy = row_view(a.Y, row * a.ldy, 2, width);
#pragma unroll
    for (int v = 0; v < V; ++v) {
      float g[8], b[8] = {}, y[8];
      vec(a.ng, v, g);
      if (a.nb) vec(a.nb, v, b);
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = fmaf((x[v][i] - mean) * rstd, g[i], b[i]);
      store_bf<XF32, NT>(vy, Cols<XF32>(tid, v, a.t_log2), y);
    }
  }
}

// Which sums over the rows a backward kernel holds, by kind: 0 nothing behind the block (no norm, no gate: Z is not read), 1 no gate or one per channel, no
// betas, 2 the same with betas, 3 a gate per token.  Numbers into NormArgs::sums.  A kind holds all its sums, also those that a call has no vector for (3 both betas', 0 the one
// before the next block, 2 both where there is one).  They are fp32: at most one addition a row of the workgroup's share, without a workspace one for every row.
constexpr int kSums[4] = {2, 3, 5, 4};
__device__ constexpr int kSumOf[4][kVectors] = {{3, 4, -1, -1, -1}, {0, 2, 3, -1, -1}, {0, 1, 2, 3, 4}, {0, 1, 3, 4, -1}};

// Workgroup = every gridDim.x-th set of blockDim.x / T rows (neighbouring workgroups read neighbouring rows at the same time: contiguous shares lay a power of two
// apart in memory, 8192 x 12288 212 -> 185 us).  The vectors (gn, gp, the gate per channel, bp) lie in the LDS, for rows of at most
// kBwdThreads * kMaxV chunks: loads of them from memory would be waited for together with the next row's, which are issued before.
template <int V, bool XF32, int KIND, bool LONG>
__device__ __forceinline__ void bwd_body(const NormArgs& a) {
  constexpr bool BRANCH = KIND > 0, BIAS = KIND != 1, TOKEN = KIND == 3;
  constexpr int PG = 0, PB = 1, GT = KIND == 1 ? 1 : 2, NG = KIND == 0 ? 0 : KIND == 2 ? 3 : 2, NB = KIND == 0 ? 1 : KIND == 2 ? 4 : 3;
  constexpr int XB = XF32 ? 4 : 2;
  constexpr bool NT = V > 1;
  __shared__ __attribute__((aligned(16))) float slots[2][kMaxWaves][2];
  extern __shared__ __attribute__((aligned(16))) u32x4 vectors[];  // [4][V * T] chunks: gn, gp, gate, bp; behind the rows: kSideBySide sums of each thread's chunk
  int turn = 0;
  const int T = 1 << a.t_log2, tid = threadIdx.x & (T - 1), n_rows = blockDim.x >> a.t_log2;
  const int lane_row = __builtin_amdgcn_readfirstlane(threadIdx.x >> a.t_log2);  // (T is a multiple of the wavefront)
  const uint16_t* const vec_ptr[4] = {a.ng, a.pg, TOKEN ? nullptr : a.gate, a.pb};
  auto vec = [&](int which, int v, float (&o)[8]) {
    if constexpr (LONG) unpack8(load_bf<XF32, false>(row_view(vec_ptr[which], 0, 2, a.H), Cols<XF32>(tid, v, a.t_log2)), o);
    else unpack8(vectors[(which * V + v) * T + tid], o);
  };
  if constexpr (!LONG) {  // (all on their way before the first goes to the LDS: 4096 x 16384 with betas 290 -> 264 us with what that does to the registers, 8192 x 8192 163 -> 159)
    constexpr int N = KIND == 0 ? 1 : KIND == 1 ? 3 : 4;
    u32x4 r[N][V];
#pragma unroll
    for (int which = 0; which < N; ++which)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const int c = threadIdx.x + i * kBwdThreads;
        if (i * kBwdThreads < V * T) r[which][i] = load_bf<XF32, false>(row_view(vec_ptr[which], 0, 2, vec_ptr[which] ? a.H : 0), Cols<XF32>(c & (T - 1), c >> a.t_log2, a.t_log2));
      }
#pragma unroll
    for (int which = 0; which < N; ++which)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const int c = threadIdx.x + i * kBwdThreads;
        if (c < V * T) vectors[which * V * T + c] = r[which][i];
      }
    __syncthreads();
  }
  float acc[kSums[KIND]][V][8] = {};
  const int64_t row0 = int64_t(blockIdx.x) * n_rows, row1 = a.M, stride = int64_t(gridDim.x) * n_rows;
  Raw<XF32> rx[V], rd[V];
  u32x4 ry[V];
  float st[4] = {0.f, 1.f, 0.f, 1.f}, nst[4] = {0.f, 1.f, 0.f, 1.f};
  __amdgpu_buffer_rsrc_t vd, vy, vx;
  auto next_row = [&](int64_t row) {
    const bool there = row < row1;
    const int width = there ? a.H : 0;
    row = there ? row : 0;
    if (BRANCH && a.pg) nst[0] = a.Stats[row], nst[1] = a.Stats[a.M + row];
    if (a.ng) nst[2] = a.Stats[2 * a.M + row], nst[3] = a.Stats[3 * a.M + row];
    vd = row_view(a.dXout, row * a.lddxo, XB, a.dXout ? width : 0);
    vy = row_view(a.dY, row * a.lddy, 2, a.ng ? width : 0);
    vx = row_view(a.X, row * a.ldx, XB, a.ng ? width : 0);
  };
  auto load_chunk = [&](int v) {
    ry[v] = load_bf<XF32, NT>(vy, Cols<XF32>(tid, v, a.t_log2));
  };
  auto load_d = [&](int v) { rd[v].template load<NT>(vd, Cols<XF32>(tid, v, a.t_log2)); };
  auto load_x = [&](int v) { rx[v].template load<NT>(vx, Cols<XF32>(tid, v, a.t_log2)); };
  // (four chunks with five sums, with a gate per token or in fp32 leave no registers for the next row, and three in fp32 with one of the others: 4096 x 16384 with
  // betas 390 -> 293 us, 4096 x 12288 in fp32 with betas 214 -> 193, with a gate per token 217 -> 209)
  constexpr bool AHEAD = V < 3 || (V == 3 ? KIND < 2 || !XF32 : KIND < 2 && !XF32);
  if (AHEAD && row0 < row1) {  // (without rows nothing may be read)
    next_row(row0 + lane_row);
#pragma unroll
    for (int v = 0; v < V; ++v) {
      load_chunk(v);
      load_x(v);
      load_d(v);
    }
  }
  for (int64_t base = row0; base < row1; base += stride) {
    const int64_t row = base + lane_row;
    const int width = row < row1 ? a.H : 0;
    float G[V][8], s[2] = {0.f, 0.f};
    u32x4 rz[V], rg[V];
    if constexpr (!AHEAD) {
      next_row(row);
#pragma unroll
      for (int v = 0; v < V; ++v) {
        load_chunk(v);
        load_x(v);
        load_d(v);
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) st[i] = nst[i];
    if constexpr (BRANCH) {
      const __amdgpu_buffer_rsrc_t vz = row_view(a.Z, row * a.ldz, 2, width), vg = row_view(a.gate, row * a.ldgate, 2, TOKEN ? width : 0);
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const Cols<XF32> c(tid, v, a.t_log2);
        rz[v] = load_bf<XF32, NT>(vz, c);
        if constexpr (TOKEN) rg[v] = load_bf<XF32, NT>(vg, c);
      }
    }
    if constexpr (AHEAD) next_row(row + stride);
#pragma unroll
    for (int v = 0; v < V; ++v) {  // a chunk's loads of the next row go out as soon as it is taken from its registers
      rd[v].get(G[v]);
      if (a.ng) {
        float dy[8], x[8], g[8];
        unpack8(ry[v], dy);
        rx[v].get(x);
        vec(0, v, g);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float h = (x[i] - st[2]) * st[3];  // hat_x
          acc[NG][v][i] = fmaf(dy[i], h, acc[NG][v][i]);
          if constexpr (BIAS) acc[NB][v][i] += dy[i];
          const float u = dy[i] * g[i];
          s[0] += u;
          s[1] = fmaf(u, h, s[1]);
          G[v][i] = fmaf(u, st[3], G[v][i]);
        }
      }
      if constexpr (AHEAD) load_chunk(v);
      if constexpr (AHEAD && !BRANCH) load_d(v);
    }
    if (a.ng) {
      row_sum<2>(a.t_log2, s, slots, turn);
      const float m0 = a.layer ? s[0] * a.inv_h * st[3] : 0.f, m1 = s[1] * a.inv_h * st[3];
#pragma unroll
      for (int v = 0; v < V; ++v) {
        float x[8];
        rx[v].get(x);
#pragma unroll
        for (int i = 0; i < 8; ++i) G[v][i] -= fmaf((x[i] - st[2]) * st[3], m1, m0);
        if constexpr (AHEAD) load_x(v);
      }
    }
    s[0] = s[1] = 0.f;
    const __amdgpu_buffer_rsrc_t vdx = row_view(a.Xout, row * a.ldxo, XB, width), vdz = row_view(a.Y, row * a.ldy, 2, a.Y ? width : 0),
                                 vdg = row_view(a.dgate_rows, row * a.lddgate, 2, a.dgate_rows ? width : 0);
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const Cols<XF32> c(tid, v, a.t_log2);
      float o[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) o[i] = a.a * G[v][i];
      store_x<XF32, NT>(vdx, c, o);
      if (!BRANCH && a.Y) {
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = a.b * G[v][i];
        store_bf<XF32, NT>(vdz, c, o);
      }
      if constexpr (BRANCH) {
        float z[8], p[8], q[8] = {};
        unpack8(rz[v], z);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          G[v][i] *= a.b;
          p[i] = 1.f;
          z[i] = (z[i] - st[0]) * st[1];  // hat_z, or Z itself
        }
        if (a.pg) vec(1, v, p);
        if (KIND != 1 && a.pb) vec(3, v, q);
        if (TOKEN || a.gate) {
          float g[8];
          if constexpr (TOKEN) unpack8(rg[v], g);
          else vec(2, v, g);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            o[i] = G[v][i] * fmaf(z[i], p[i], q[i]);
            if constexpr (!TOKEN) acc[GT][v][i] += o[i];
            G[v][i] *= g[i];  // dr
          }
          if (TOKEN && a.dgate_rows) store_bf<XF32, NT>(vdg, c, o);
        }
        if (a.pg) {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            acc[PG][v][i] = fmaf(G[v][i], z[i], acc[PG][v][i]);
            if constexpr (KIND != 1) acc[PB][v][i] += G[v][i];
            G[v][i] *= p[i];  // v
            s[0] += G[v][i];
            s[1] = fmaf(G[v][i], z[i], s[1]);
          }
        }
      }
    }
    if constexpr (BRANCH) {
      if (a.pg) {
        row_sum<2>(a.t_log2, s, slots, turn);
        const float m0 = a.layer ? s[0] * a.inv_h : 0.f, m1 = s[1] * a.inv_h;
#pragma unroll
        for (int v = 0; v < V; ++v) {
          float z[8], o[8];
          if constexpr (AHEAD) load_d(v);
          unpack8(rz[v], z);
#pragma unroll
          for (int i = 0; i < 8; ++i) o[i] = (G[v][i] - fmaf((z[i] - st[0]) * st[1], m1, m0)) * st[1];
          store_bf<XF32, NT>(vdz, Cols<XF32>(tid, v, a.t_log2), o);
        }
      } else {  // (a loop of its own: dZ = dr, whatever Z is, which may be infinite)
#pragma unroll
        for (int v = 0; v < V; ++v) {
          if constexpr (AHEAD) load_d(v);
          store_bf<XF32, NT>(vdz, Cols<XF32>(tid, v, a.t_log2), G[v]);
        }
      }
    }
  }
  // the workgroup's sums go out; where rows lie side by side they are added up in order before, kSideBySide chunks at a time by all threads (one at a time by the
  // first row's threads: 12075 x 1016 41.4 us, so 40.4; 4096 x 16384 264, so 256)
  if (a.n_sums == 0) return;
  float* dst[kSums[KIND]];
  int n = 0;
#pragma unroll
  for (int k = 0; k < kSums[KIND]; ++k) {
    float* const out = a.sums[kSumOf[KIND][k]];
    dst[k] = out && a.parts ? a.parts + (int64_t(blockIdx.x) * a.n_sums + n) * a.H : out;
    n += out != nullptr;
  }
  auto put = [&](float* to, int at, f32x4 s) {
    f32x4* q = reinterpret_cast<f32x4*>(to + at);
    if (to && at < a.H) *q = !a.parts && a.accumulate ? *q + s : s;
  };
  if (LONG || n_rows == 1) {
#pragma unroll
    for (int k = 0; k < kSums[KIND]; ++k)
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const Cols<XF32> c(tid, v, a.t_log2);
        put(dst[k], c.c0, f32x4{acc[k][v][0], acc[k][v][1], acc[k][v][2], acc[k][v][3]});
        put(dst[k], c.c1, f32x4{acc[k][v][4], acc[k][v][5], acc[k][v][6], acc[k][v][7]});
      }
    return;
  }
  f32x4* const side = reinterpret_cast<f32x4*>(vectors);  // [kSideBySide][2][threads]
#pragma unroll
  for (int first = 0; first < kSums[KIND] * V; first += kSideBySide) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kSideBySide; ++i)
      if (first + i < kSums[KIND] * V) {
        const float* const s = acc[(first + i) / V][(first + i) % V];
        side[(i * 2 + 0) * kBwdThreads + threadIdx.x] = f32x4{s[0], s[1], s[2], s[3]};
        side[(i * 2 + 1) * kBwdThreads + threadIdx.x] = f32x4{s[4], s[5], s[6], s[7]};
      }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kSideBySide; ++i)
      if (first + i < kSums[KIND] * V && dst[(first + i) / V])
        for (int o = threadIdx.x; o < 2 * T; o += kBwdThreads) {
          const int half = o >> a.t_log2, at = o & (T - 1);
          f32x4 s = side[(i * 2 + half) * kBwdThreads + at];
          for (int r = 1; r < n_rows; ++r) s += side[(i * 2 + half) * kBwdThreads + r * T + at];
          const Cols<XF32> c(at, (first + i) % V, a.t_log2);
          put(dst[(first + i) / V], half ? c.c1 : c.c0, s);
        }
  }
}

template <int V, bool XF32, int KIND>
__global__ __launch_bounds__(kBwdThreads) void block_norm_bwd_kernel(const NormArgs a) {
  bwd_body<V, XF32, KIND, false>(a);
}
// Rows of more than kBwdThreads * kMaxV chunks: 1024 threads leave 128 registers each, of which the sums alone would take 64 to 160, so that all of these kernels keep
// part of them in memory (312 to 740 bytes a lane).  2048 x 20480 444 us (floor 83), with betas 570-690, in fp32 509 and 690 (floor 124); 2048 x 32768 505 (132), 649, 547 (198), 786.
template <int V, bool XF32, int KIND>
__global__ __launch_bounds__(kMaxThreads) void block_norm_bwd_long_kernel(const NormArgs a) {
  bwd_body<V, XF32, KIND, true>(a);
}

// The groups' partial sums added up in a fixed order: 16 lanes hold 64 columns, 16 threads of a column take every 16th group; then these in order.
__global__ __launch_bounds__(256) void block_norm_sum_kernel(const NormArgs a, int groups) {
  __shared__ f32x4 lds[16][16];
  const int lane = threadIdx.x & 15, part = threadIdx.x >> 4;
  const int64_t width = int64_t(a.n_sums) * a.H, at = (int64_t(blockIdx.x) * 16 + lane) * 4;
  f32x4 s = {0.f, 0.f, 0.f, 0.f};
  if (at < width)
#pragma unroll 4
    for (int g = part; g < groups; g += 16) s += *reinterpret_cast<const f32x4*>(a.parts + int64_t(g) * width + at);
  lds[part][lane] = s;
  __syncthreads();
  if (part > 0 || at >= width) return;
  for (int i = 1; i < 16; ++i) s += lds[i][lane];
  const int n = int(at / a.H), c = int(at % a.H);
  int k = 0;
  for (int left = n; k < kVectors; ++k)
    if (a.sums[k] && left-- == 0) break;
  f32x4* q = reinterpret_cast<f32x4*>(a.sums[k] + c);
  *q = a.accumulate ? *q + s : s;
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

// Threads of a row (their logarithm): as few as hold it with kMaxV chunks each.
int norm_t_log2(int64_t H) {
  int n = 6;
  while ((int64_t(8 * kMaxV) << n) < H) ++n;
  return n;
}
int norm_chunks(int64_t H, int t_log2) { return int((H / 8 + (int64_t(1) << t_log2) - 1) >> t_log2); }

// Backward: two chunks a thread rather than four where a workgroup has the threads (8192 x 8192: norm, gate and betas 375 -> 164 us, fp32 271 -> 211; without
// either the same).
int norm_bwd_t_log2(int64_t H) {
  const int n = norm_t_log2(H);
  return norm_chunks(H, n) == kMaxV && (2 << n) <= kBwdThreads ? n + 1 : n;
}

// Workgroups that share out the rows of a backward call, each with partial sums of its own: one per compute unit.
int64_t norm_groups(const ntp_handle* h, const ntp_block_norm_shape_t* s) {
  const int64_t at_once = std::max<int64_t>(1, kBwdThreads >> norm_bwd_t_log2(s->H));
  return std::max<int64_t>(1, std::min<int64_t>((s->M + at_once - 1) / at_once, h->compute_units));
}

// f with the number of chunks a thread holds as a constant
template <typename F>
void by_chunks(int v, F&& f) {
  if (v <= 1) f(std::integral_constant<int, 1>{});
  else if (v == 2) f(std::integral_constant<int, 2>{});
  else if (v == 3) f(std::integral_constant<int, 3>{});
  else f(std::integral_constant<int, 4>{});
}

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
  if (((s->M + 3) << norm_t_log2(s->H)) > 0xffffffffll) return NTP_ERR_UNSUPPORTED;  // a launch counts its threads in 32 bits
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
  // few rows: more threads each, down to one chunk a thread, while the compute units have room for them
  int t_log2 = norm_t_log2(s->H);
  while (norm_chunks(s->H, t_log2) > 1 && (2 << t_log2) <= kMaxThreads && (s->M << t_log2) * 2 <= int64_t(h->compute_units) * kMaxThreads) ++t_log2;
  a.t_log2 = t_log2;
  const int threads = std::max(kFwdThreads, 1 << t_log2), rows = threads >> t_log2;
  const dim3 grid(uint32_t((s->M + rows - 1) / rows)), block{uint32_t(threads)};
  auto launch = [&](auto v) {
    if (a.xf32) hipLaunchKernelGGL((block_norm_fwd_kernel<decltype(v)::value, true>), grid, block, 0, hs, a);
    else hipLaunchKernelGGL((block_norm_fwd_kernel<decltype(v)::value, false>), grid, block, 0, hs, a);
  };
  by_chunks(norm_chunks(s->H, t_log2), launch);
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
  a.t_log2 = norm_bwd_t_log2(s->H);
  const bool bias = w->post_beta || w->pre_beta;
  const int threads = std::max(kBwdThreads, 1 << a.t_log2);
  const dim3 grid{uint32_t(groups)}, block{uint32_t(threads)};
  auto launch = [&](auto v, auto f32, auto kind) {
    constexpr int V = decltype(v)::value, KIND = decltype(kind)::value;
    constexpr bool F32 = decltype(f32)::value;
    if (threads > kBwdThreads) hipLaunchKernelGGL((block_norm_bwd_long_kernel<kMaxV, F32, KIND>), grid, block, 0, hs, a);
    else hipLaunchKernelGGL((block_norm_bwd_kernel<V, F32, KIND>), grid, block, uint32_t(std::max((KIND == 0 ? 1 : KIND == 1 ? 3 : 4) * (V << a.t_log2) * 16, (1 << a.t_log2) < threads ? kSideBySide * kBwdThreads * 32 : 0)), hs, a);
  };
  using std::integral_constant;
  by_chunks(norm_chunks(s->H, a.t_log2), [&](auto v) {
    auto by_kind = [&](auto f32) {
      if (!reads_z) launch(v, f32, integral_constant<int, 0>{});
      else if (token) launch(v, f32, integral_constant<int, 3>{});
      else if (!bias) launch(v, f32, integral_constant<int, 1>{});
      else launch(v, f32, integral_constant<int, 2>{});
    };
    if (a.xf32) by_kind(std::true_type{});
    else by_kind(std::false_type{});
  });
  bool ok = hipGetLastError() == hipSuccess;
  if (ok && a.parts) {
    hipLaunchKernelGGL(block_norm_sum_kernel, dim3(uint32_t((int64_t(a.n_sums) * s->H + 63) / 64)), dim3(256), 0, hs, a, int(groups));
    ok = hipGetLastError() == hipSuccess;
  }
  ntp::timing_end(h, stream);
  return ok ? NTP_OK : NTP_ERR_LAUNCH;
}
