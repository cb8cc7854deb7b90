// Attention of one new token per sequence over the paged key / value cache (ntp_attn_decode_shard): for sequence s and query head j
//   C[s, j] = sum_t p_t V[t] / sum_t p_t,   p_t = exp(q_j . K[t] / sqrt(d) - max),   t over the sequence's tokens.
// One pass over the keys with a running maximum and sum.  Every key and value is read once, 4 d bytes for 4 d operations a query head: HBM bounds it.
//
// The work of a call is a line of steps, sequence by sequence, in it unit by unit (a KV head with up to 16 of its query heads), a unit's steps along its tokens; a step is
// one tile (8 KB of keys, 8 KB of values) for each of a workgroup's four wavefronts.  With a workspace the line is cut into equal shares, two workgroups per compute
// unit, from the lengths on the device: lengths that differ, or that lie far below max_len, leave no workgroup idle.  A workgroup writes the units that lie wholly in
// its share and leaves partial results of the one it begins inside and the one it ends inside, which a second kernel joins.  Without a workspace
// a workgroup takes one unit.
//
// The wavefronts of a workgroup have a running maximum and sum of their own and put their results together at the end of a unit.  Both products run on the
// 16x16x32 bf16 matrix instruction with the query head on the lane axis (S^T = K Q^T, O^T += V^T P^T), the scores go from the one to the other in
// registers.  With one query head 15 of 16 columns are idle: matrix work is far from the bound, 24 instructions a tile (8 for the
// scores, 8 each for the weights and their rest) against 16 KB from HBM.  A KV head with more than 16 query heads is several units, each of which reads its keys and values (64
// sequences of up to 8192, one KV head of 128: 16 query heads 31 us, 32 52, 64 98).
// Both matrices go through a part of the LDS that is the wavefront's own, by DMA, so that nothing but a unit's end needs a barrier.  The loads are non-temporal: a cache line is
// used once (equal lengths of 4096, 14 heads, 64 sequences: 326 -> 292 us, 6.4 TB/s).
//
// A page holds a multiple of 16 tokens, so 16 tokens of one head are one contiguous block; each block is a buffer view of its own that ends with the
// sequence: what lies behind the last token, or in a page that does not exist, reads as zeros and never reaches the products (it may be NaN).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <type_traits>

#include "ntp_gemm_kernels.h"
#include "ntp_gemm_ring.h"
#include "ntp_internal.h"
#include "ntp_kv_cache.h"

namespace {

using ntp::off16;
using ntp_gemm::bf16x8;
using ntp_gemm::f32x4;
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256, kWaves = 4, kBlock = 16;  // kBlock: tokens of a contiguous block
constexpr int kMaxShares = 1024;
constexpr int64_t kMaxGrid = 0xffffffffll / kThreads;   // workgroups: a launch counts its threads in 32 bits
constexpr int kTileBytes = 8192;                        // of keys, and of values, per tile
template <int D>
constexpr int kTile = kTileBytes / (2 * D);  // tokens per tile: 32 or 64
template <int D>
constexpr int kStep = kWaves * kTile<D>;     // tokens per step

struct DecodeArgs {
  const uint16_t *Q, *K, *V;
  const int32_t *table, *lengths;
  uint16_t* C;
  float* LSE;
  // shares of the line of steps: per workgroup two partial results (of the unit it begins inside and the one it ends inside) of 16 query heads each:
  // maximum (log2 units) and sum, and the D unnormalised outputs.  NULL: workgroup = unit
  float2* part_sums;
  float* part_rows;
  int64_t ldq, ldc, ldt, page_stride;
  int32_t n_pages, n_seq, max_len, q_cnt, q_off, kv_off, group, page_size, page_log2;
  int32_t kv_first, kv_used, head_tiles;  // local KV heads that are read; 16-head tiles of a KV head's query heads
  int32_t shares, join_rows;              // join_rows: see attn_decode_join_kernel
  float scale_log2;                       // log2(e) / sqrt(d)
};

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// Maximum / sum over the four lanes l % 16 + {0, 16, 32, 48}, left in all four: the 16-lane rows, then the halves trade places in registers.
template <typename F>
__device__ __forceinline__ float over_rows(float v, F&& f) {
  {
    const uint32_t x = __builtin_bit_cast(uint32_t, v);
    const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    const uint32_t r0 = r[0], r1 = r[1];
    v = f(__builtin_bit_cast(float, r0), __builtin_bit_cast(float, r1));
  }
  const uint32_t x = __builtin_bit_cast(uint32_t, v);
  const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
  const uint32_t r0 = r[0], r1 = r[1];
  return f(__builtin_bit_cast(float, r0), __builtin_bit_cast(float, r1));
}

// `bytes` bytes at p; what lies behind them reads as zeros.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t view(const uint16_t* p, int bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(p), 0, bytes, 0x00020000);
}
__device__ __forceinline__ void dma_16(__amdgpu_buffer_rsrc_t rs, unsigned char* dst, uint32_t off) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (ntp_gemm::lds_void*)dst, 16, off, 0, 0, 2);
}
// All but the last N vector memory instructions have finished.
template <int N>
__device__ __forceinline__ void dma_left() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
// What was loaded is there: the compiler's own wait for it stands here and not in a loop, where it would take in the DMA that is in flight.
template <typename V>
__device__ __forceinline__ void arrived(V& v) {
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("" : "+v"(v));
#endif
}

template <int OFF>
__device__ __forceinline__ u32x4 lds_b128(uint32_t addr) {
#if !defined(__HIP_DEVICE_COMPILE__)
  return u32x4{};
#else
  u32x4 v;
  asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(v) : "v"(addr), "n"(OFF) : "memory");
  return v;
#endif
}
template <int OFF>
__device__ __forceinline__ u32x2 lds_tr_b64(uint32_t addr) {
#if !defined(__HIP_DEVICE_COMPILE__)
  return u32x2{};
#else
  u32x2 v;
  asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(v) : "v"(addr), "n"(OFF) : "memory");
  return v;
#endif
}
// The reads requested before have arrived: every later use of their registers depends on this wait.
template <int N, typename V>
__device__ __forceinline__ void lds_reads_done(V (&r)[N]) {
  static_assert(N % 8 == 0, "");
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("s_waitcnt lgkmcnt(0)"
               : "+v"(r[0]), "+v"(r[1]), "+v"(r[2]), "+v"(r[3]), "+v"(r[4]), "+v"(r[5]), "+v"(r[6]), "+v"(r[7])
               :
               : "memory");
#pragma unroll
  for (int i = 8; i < N; i += 8)
    asm volatile("" : "+v"(r[i]), "+v"(r[i + 1]), "+v"(r[i + 2]), "+v"(r[i + 3]), "+v"(r[i + 4]), "+v"(r[i + 5]), "+v"(r[i + 6]), "+v"(r[i + 7]) : : "memory");
#endif
}

template <int... Is, typename F>
__device__ __forceinline__ void unrolled(std::integer_sequence<int, Is...>, F&& f) {
  (f(std::integral_constant<int, Is>{}), ...);
}

// Rows of D values in the LDS hold their 16-byte chunks permuted: chunk c of row r sits at slot c ^ swz(r), so that the rows that a transposing read
// touches per cycle lie on distinct banks (as the attention core's tiles).
template <int D>
__device__ __forceinline__ uint32_t swz(int r) {
  return D == 128 ? uint32_t((r & 7) << 1) : uint32_t(((r >> 1) & 3) << 1);
}

// Steps of a sequence's unit: at least one, which writes the zeros of a sequence without tokens.
template <int D>
__device__ __forceinline__ int steps_of(const DecodeArgs& a, int len) {
  return std::max(1, (std::min(len, a.max_len) + kStep<D> - 1) / kStep<D>);
}
// Inclusive sum over the wavefront's lanes: inside rows of 16 lanes, then the rows' last values are passed on.
template <int CTRL, int ROWS>
__device__ __forceinline__ int dpp_add(int v) {
  return v + __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, false);
}
__device__ __forceinline__ int sum_upto(int v) {
  v = dpp_add<0x111, 0xf>(v);  // shifted by 1, 2, 4, 8 lanes
  v = dpp_add<0x112, 0xf>(v);
  v = dpp_add<0x114, 0xf>(v);
  v = dpp_add<0x118, 0xf>(v);
  v = dpp_add<0x142, 0xa>(v);  // lane 15 of a row to the next one: rows 1 and 3
  v = dpp_add<0x143, 0xc>(v);  // lane 31 to rows 2 and 3
  return v;
}

// The line of steps: 64 sequences at a time in the lanes of a wavefront (every wavefront for itself).
template <int D>
struct Line {
  int len, upto;        // of this lane's sequence base + lane: its length, and the steps of a unit up to and with it
  int base, before;     // the first of the 64, and the steps of the sequences before it
  int per_seq, total;   // units of a sequence; steps of the line
  int shares, q, r;     // share w has q steps, the first r shares one more
  __device__ __forceinline__ void load(const DecodeArgs& a, int from) {
    const int i = from + int(threadIdx.x & 63);
    base = from;
    len = i < a.n_seq ? a.lengths[i] : 0;
    upto = sum_upto(i < a.n_seq ? steps_of<D>(a, len) : 0);
  }
  __device__ __forceinline__ int last() const { return __builtin_amdgcn_readlane(upto, 63); }
  // steps of a unit of kAtOnce sequences, this lane's and all lanes'; the loads go out together
  static constexpr int kAtOnce = 512;
  __device__ __forceinline__ static int lane_steps(const DecodeArgs& a, int from) {
    int n[kAtOnce / 64], sum = 0;
#pragma unroll
    for (int k = 0; k < kAtOnce / 64; ++k) {
      const int i = from + k * 64 + int(threadIdx.x & 63);
      n[k] = i < a.n_seq ? a.lengths[i] : 0;
    }
#pragma unroll
    for (int k = 0; k < kAtOnce / 64; ++k) sum += from + k * 64 + int(threadIdx.x & 63) < a.n_seq ? steps_of<D>(a, n[k]) : 0;
    return sum;
  }
  __device__ __forceinline__ static int all_steps(int lane_sum) { return __builtin_amdgcn_readlane(sum_upto(lane_sum), 63); }
  // the whole line, and how it is cut; the first 64 sequences
  __device__ __forceinline__ void measure(const DecodeArgs& a) {
    before = 0;
    load(a, 0);
    int steps = last();
    if (a.n_seq > 64) {
      int sum = 0;
      for (int from = 0; from < a.n_seq; from += kAtOnce) sum += lane_steps(a, from);
      steps = all_steps(sum);
    }
    total = steps * per_seq;
    shares = std::min(a.shares, total);  // (one step at least for each)
    q = total / shares;
    r = total % shares;
  }
  // from the first 64 sequences to the one with step x of the line, and its unit and the number in it: by kAtOnce, then by 64 (4096 sequences of up to
  // 400 tokens, one KV head: 64 by 64, and every query head's workgroup joining, 470 us; so 133)
  __device__ __forceinline__ void seek(const DecodeArgs& a, int x, int& seq, int& unit, int& step) {
    int from = 0;
    while (from < a.n_seq - kAtOnce) {
      const int n = all_steps(lane_steps(a, from));
      if ((before + n) * per_seq > x) break;
      before += n;
      from += kAtOnce;
    }
    if (from > 0) load(a, from);
    uint64_t behind;
    while ((behind = __ballot((before + upto) * per_seq > x)) == 0) next64(a);
    seq = base + __builtin_ctzll(behind);
    const int steps = steps_of<D>(a, length(seq)), rest = x - steps_before(seq) * per_seq;
    unit = rest / steps;
    step = rest % steps;
  }
  __device__ __forceinline__ int begin(int w) const { return w * q + std::min(w, r); }
  __device__ __forceinline__ int share_of(int x) const { return x < r * (q + 1) ? x / (q + 1) : r + (x - r * (q + 1)) / q; }
  __device__ __forceinline__ void next64(const DecodeArgs& a) {
    before += last();
    load(a, base + 64);
  }
  __device__ __forceinline__ int length(int seq) const { return __builtin_amdgcn_readlane(len, seq - base); }
  // steps of the sequences before seq, one of the 64
  __device__ __forceinline__ int steps_before(int seq) const { return before + (seq > base ? __builtin_amdgcn_readlane(upto, seq - base - 1) : 0); }
};

// This unit's KV head and its local query heads j0 .. j1 - 1.
struct Heads {
  int g, j0, j1;
  __device__ __forceinline__ Heads(const DecodeArgs& a, int unit) {
    const int tile = unit % a.head_tiles;
    g = a.kv_first + unit / a.head_tiles;
    const int64_t first = int64_t(a.kv_off + g) * a.group - a.q_off;
    j0 = int(std::max<int64_t>(first, 0)) + tile * 16;
    j1 = int(std::min<int64_t>(std::min<int64_t>(first + a.group, a.q_cnt), j0 + 16));
  }
};

template <int D>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2))) void attn_decode_kernel(const DecodeArgs a) {
  constexpr int KS = D / 32, DB = D / 16;           // K-steps of the score product, 16-column blocks of the output
  constexpr int T = kTile<D>, NB = T / kBlock;      // tokens and blocks per tile
  constexpr int BLOCK_BYTES = kBlock * D * 2, DMA = BLOCK_BYTES / 1024;  // DMA instructions per block
  constexpr int ROW = D + 4;                        // floats of a wavefront's result row: outputs, maximum, sum
  constexpr int LDS = kWaves * std::max(2 * kTileBytes, 16 * ROW * 4);
  __shared__ __attribute__((aligned(1024))) unsigned char lds[LDS];

  const int lane = threadIdx.x & 63, lq = lane & 15, lh = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  unsigned char* const sK = lds + wave * 2 * kTileBytes;
  unsigned char* const sV = sK + kTileBytes;
  const uint32_t lK = uint32_t(reinterpret_cast<uintptr_t>(sK)), lV = lK + kTileBytes;

  // lane offsets: DMA of a block's chunks, key fragments (row lane % 16, columns lane / 16 * 8 on), transposing reads
  uint32_t voff[DMA], row[KS], col[DB];
#pragma unroll
  for (int i = 0; i < DMA; ++i) {
    const int p = i * 64 + lane, row = p / (D / 8), slot = p % (D / 8);
    voff[i] = uint32_t(row * D * 2) + ((uint32_t(slot) ^ swz<D>(row)) * 16u);
  }
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) row[ks] = lK + uint32_t(lq * D * 2) + ((uint32_t(ks * 4 + lh) ^ swz<D>(lq)) * 16u);
  const int rv = lh * 4 + (lq >> 2);
#pragma unroll
  for (int db = 0; db < DB; ++db) col[db] = lV + uint32_t(rv * D * 2) + uint32_t(lq & 1) * 8u + ((uint32_t(db * 2 + ((lq & 3) >> 1)) ^ swz<D>(rv)) * 16u);

  // this workgroup's steps x .. x_end - 1 of the line; x lies in unit `unit` of sequence seq, `step` steps behind the unit's first
  Line<D> line;
  line.per_seq = a.kv_used * a.head_tiles;
  int x, x_end, seq, unit, step;
  if (a.part_rows) {
    line.measure(a);
    if (int(blockIdx.x) >= line.shares) return;
    x = line.begin(blockIdx.x);
    x_end = line.begin(blockIdx.x + 1);
    line.seek(a, x, seq, unit, step);
  } else {
    seq = int(blockIdx.x) / line.per_seq;
    unit = int(blockIdx.x) % line.per_seq;
    line.before = 0;
    line.load(a, seq & ~63);
    x = step = 0;
    x_end = steps_of<D>(a, line.length(seq));
  }

  // (said to be the same in every lane: the buffer views below are made from them)
  x = uniform(x), x_end = uniform(x_end), seq = uniform(seq), unit = uniform(unit), step = uniform(step);
  for (bool first = true; x < x_end; first = false) {
  const int len = std::min(line.length(seq), a.max_len), steps = steps_of<D>(a, len), n_steps = std::min(steps - step, x_end - x);
  const int k_lo = step * kStep<D>, k_hi = std::min(len, k_lo + n_steps * kStep<D>);
  const Heads hd(a, unit);
  const int g = hd.g, j0 = hd.j0, j1 = hd.j1;  // (j0 >= j1: a last tile of 16 that a part of a group does not reach)

  bf16x8 qf[KS] = {};  // operand B[k][j]: j = query head (lane % 16), k = 8 consecutive columns
  if (j0 + lq < j1) {
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks] = *reinterpret_cast<const bf16x8*>(a.Q + int64_t(seq) * a.ldq + int64_t(j0 + lq) * D + ks * 32 + lh * 8);
  }

  f32x4 acc[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) acc[db] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m_run = -INFINITY, l_run = 0.f;

  // Page numbers of 64 of the wavefront's blocks, one a lane: its tile number i is tile i * kWaves + wave of the share's tokens.
  constexpr int PER = 64 / NB;  // tiles per set of page numbers
  const int32_t* const row_of_table = a.table + int64_t(seq) * a.ldt;
  auto pages_from = [&](int i) {
    const int key = k_lo + ((i + lane / NB) * kWaves + wave) * T + (lane % NB) * kBlock;
    return key < k_hi ? row_of_table[key >> a.page_log2] : -1;
  };
  int32_t pages = pages_from(0);
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) arrived(qf[ks]);
  arrived(pages);
  const int n_tiles = j0 < j1 ? std::max(0, (k_hi - k_lo + T - 1) / T) : 0;
  const int mine = (n_tiles - wave + kWaves - 1) / kWaves;  // tiles of this wavefront
  // DMA of one matrix of tile i; number of tokens of each block that count
  auto request = [&](const uint16_t* base, unsigned char* to, int i, int (&valid)[NB]) {
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const int key = k_lo + (i * kWaves + wave) * T + b * kBlock;
      const int page = __builtin_amdgcn_readlane(pages, (i % PER) * NB + b);
      const bool there = page >= 0 && page < a.n_pages;
      valid[b] = uniform(there ? std::min(std::max(k_hi - key, 0), kBlock) : 0);
      const int64_t at = there ? int64_t(page) * a.page_stride + (int64_t(g) * a.page_size + (key & (a.page_size - 1))) * D : 0;
      const __amdgpu_buffer_rsrc_t rs = view(base + at, valid[b] * D * 2);
#pragma unroll
      for (int j = 0; j < DMA; ++j) dma_16(rs, to + b * BLOCK_BYTES + j * 1024, voff[j]);
    }
  };
  // One tile of keys and one of values in the LDS: the next keys are requested when this tile's have been read into registers, the next values
  // likewise, so that there is always one or the other in flight.
  constexpr int IN_FLIGHT = NB * DMA;
  int valid[NB], next[NB];
  if (mine > 0) {
    request(a.K, sK, 0, valid);
    request(a.V, sV, 0, valid);
  }
  auto tile = [&](int i, auto last) {
    constexpr bool MORE = !decltype(last)::value;
    dma_left<IN_FLIGHT>();  // the keys are there
    u32x4 kf[NB * KS];
    unrolled(std::make_integer_sequence<int, NB * KS>{}, [&](auto n) {
      constexpr int blk = decltype(n)::value / KS, ks = decltype(n)::value % KS;
      kf[decltype(n)::value] = lds_b128<blk * BLOCK_BYTES>(row[ks]);
    });
    lds_reads_done(kf);
    if constexpr (MORE) {
      if ((i + 1) % PER == 0) {
        pages = pages_from(i + 1);
        arrived(pages);
      }
      request(a.K, sK, i + 1, next);
    }
    // scores, transposed: st[b][r] = score of query head lane % 16 with token key0 + b * 16 + lane / 16 * 4 + r
    f32x4 st[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      st[b] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) st[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kf[b * KS + ks]), qf[ks], st[b], 0, 0, 0);
      if (valid[b] < kBlock) {
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (lh * 4 + r >= valid[b]) st[b][r] = -INFINITY;
      }
    }
    float mx = -INFINITY;
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int r = 0; r < 4; ++r) mx = fmaxf(mx, st[b][r]);
    mx = over_rows(mx, [](float x, float y) { return fmaxf(x, y); }) * a.scale_log2;
    const float m_new = fmaxf(m_run, mx), m_use = m_new == -INFINITY ? 0.f : m_new;  // (no score above -inf so far: weights of 0)
    const float alpha = fast_exp2(m_run - m_use);
    float ls = 0.f;
    // weights as operand B of the second product, per 32 tokens: bf16, and what that leaves, rounded to bf16 too, in a product of its own.  Together they are within 2^-17 of
    // the fp32 weight; an output is a mean of values by these weights, rounded to 2^-8, and a weight has the error of its fp32 score anyway (about 2^-20 for scores of 10)
    bf16x8 pf[NB / 2], pr[NB / 2];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float p = fast_exp2(fmaf(st[b][r], a.scale_log2, -m_use));
        ls += p;
        const __bf16 top = static_cast<__bf16>(p);
        pf[b / 2][(b & 1) * 4 + r] = top;
        pr[b / 2][(b & 1) * 4 + r] = static_cast<__bf16>(p - static_cast<float>(top));
      }
    l_run = l_run * alpha + ls;  // of this lane's tokens; the four lane groups are added at the end
    m_run = m_new;
    if (__any(alpha != 1.0f)) {
#pragma unroll
      for (int db = 0; db < DB; ++db) acc[db] *= alpha;
    }
    dma_left<MORE ? IN_FLIGHT : 0>();  // the values are there
    u32x2 vf[16];  // [(db * NB / 2 + s2) * 2 + half]
    unrolled(std::make_integer_sequence<int, 16>{}, [&](auto n) {
      constexpr int db = decltype(n)::value / NB, q = decltype(n)::value % NB;
      vf[decltype(n)::value] = lds_tr_b64<q * BLOCK_BYTES>(col[db]);
    });
    lds_reads_done(vf);
    if constexpr (MORE) request(a.V, sV, i + 1, next);
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int s2 = 0; s2 < NB / 2; ++s2) {
        const u32x2 lo = vf[db * NB + s2 * 2], hi = vf[db * NB + s2 * 2 + 1];
        const u32x4 both = {lo[0], lo[1], hi[0], hi[1]};
        acc[db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, both), pf[s2], acc[db], 0, 0, 0);
        acc[db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, both), pr[s2], acc[db], 0, 0, 0);
      }
    if constexpr (MORE) {
#pragma unroll
      for (int b = 0; b < NB; ++b) valid[b] = next[b];
    }
  };
  for (int i = 0; i + 1 < mine; ++i) tile(i, std::false_type{});
  if (mine > 0) tile(mine - 1, std::true_type{});

  // the wavefronts' results, one row per query head
  l_run = over_rows(l_run, [](float x, float y) { return x + y; });
  __syncthreads();
  float* const result = reinterpret_cast<float*>(lds) + (wave * 16 + lq) * ROW;
#pragma unroll
  for (int db = 0; db < DB; ++db) *reinterpret_cast<f32x4*>(result + db * 16 + lh * 4) = acc[db];
  if (lh == 0) {
    result[D] = m_run;
    result[D + 1] = l_run;
  }
  __syncthreads();
  const bool whole = n_steps == steps;
  const int64_t slot = (int64_t(blockIdx.x) * 2 + !first) * 16;
  const int r16 = threadIdx.x >> 4, c0 = (threadIdx.x & 15) * 4, head = j0 + r16;
  if (head < j1) {
    const float* const res = reinterpret_cast<const float*>(lds) + r16 * ROW;
    float top = -INFINITY, w[kWaves], sum = 0.f;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) top = fmaxf(top, res[i * 16 * ROW + D]);
    const float base = top == -INFINITY ? 0.f : top;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) {
      w[i] = fast_exp2(res[i * 16 * ROW + D] - base);
      sum = fmaf(w[i], res[i * 16 * ROW + D + 1], sum);
    }
    const float inv = sum == 0.f ? 0.f : 1.0f / sum;
#pragma unroll
    for (int c = c0; c < D; c += 64) {
      f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < kWaves; ++i) o += w[i] * *reinterpret_cast<const f32x4*>(res + i * 16 * ROW + c);
      if (!whole) {
        *reinterpret_cast<f32x4*>(a.part_rows + (slot + r16) * D + c) = o;
      } else {
        ntp_gemm::u16x4 out;
#pragma unroll
        for (int r = 0; r < 4; ++r) out[r] = ntp_gemm::f32_to_bf16(o[r] * inv);
        *reinterpret_cast<ntp_gemm::u16x4*>(a.C + int64_t(seq) * a.ldc + int64_t(head) * D + c) = out;
      }
    }
    if (c0 == 0) {
      if (!whole) a.part_sums[slot + r16] = float2{top, sum};
      else if (a.LSE) a.LSE[int64_t(head) * a.n_seq + seq] = (base + log2f(sum)) * 0.6931471805599453f;
    }
  }
  x += n_steps;
  step = 0;
  if (++unit == line.per_seq) {
    unit = 0;
    if (++seq == line.base + 64 && x < x_end) line.next64(a);
  }
  __syncthreads();  // the results have been read: the next unit's tiles may come
  }
}

// The partial results of one (sequence, query head) put together, where its unit does not lie in one share: the threads form the parts' weights, then W / 4 lanes hold
// W of the outputs and 1024 / W groups of them take the parts in turn (their loads do not depend on each other).  W: all D, or kFewColumns in a workgroup each where a
// unit can lie in 32 shares or more, so that each group has few parts (one sequence of 32768, 8 KV heads: 28.7 -> 27.1 us with the attention; of 1021 in 8 shares 8.2, and
// 8.9 if it were).
constexpr int kFewColumns = 32;
template <int D, int W>
__global__ __launch_bounds__(kThreads) void attn_decode_join_kernel(const DecodeArgs a) {
  constexpr int L = W / 4, G = kThreads / L, N = kMaxShares / kThreads;
  const int job = int(blockIdx.x) / (D / W), col0 = int(blockIdx.x) % (D / W) * W;
  __shared__ float weight[kMaxShares], wave_max[kWaves], wave_sum[kWaves];
  __shared__ f32x4 rows[G][L];
  Line<D> line;
  line.per_seq = a.kv_used * a.head_tiles;
  line.measure(a);
  int seq, head, r16, w0, begin;  // the head's row in its unit's 16, the share in which the unit begins, and its first step
  if (a.join_rows == 0) {  // workgroup = (sequence, query head)
    seq = job / a.q_cnt;
    head = job % a.q_cnt;
    const int kv = (a.q_off + head) / a.group - a.kv_off, unit0 = (kv - a.kv_first) * a.head_tiles;
    const int in_group = head - Heads(a, unit0).j0;
    r16 = in_group % 16;
    while (seq >= line.base + 64) line.next64(a);
    begin = line.steps_before(seq) * line.per_seq + (unit0 + in_group / 16) * steps_of<D>(a, line.length(seq));
    w0 = line.share_of(begin);
  } else {  // workgroup = (border between two shares, row): the first border inside a unit
    const int w = job / a.join_rows + 1;
    if (w >= line.shares) return;
    const int x = line.begin(w);
    int unit, step;
    line.seek(a, x, seq, unit, step);
    begin = x - step;
    w0 = w - 1;
    if (step == 0 || line.begin(w0) > begin) return;
    const Heads hd(a, unit);
    r16 = job % a.join_rows;
    head = hd.j0 + r16;
    if (head >= hd.j1) return;
  }
  const int steps = steps_of<D>(a, line.length(seq)), used = line.share_of(begin + steps - 1) - w0 + 1;
  if (used == 1) return;  // written whole
  // part p is what share w0 + p left: of the unit that it begins inside, but for a first share that begins before the unit
  const int late = line.begin(w0) < begin;
  auto slot = [&](int p) { return (int64_t(w0 + p) * 2 + (p == 0 ? late : 0)) * 16 + r16; };
  const int grp = threadIdx.x / L, c = threadIdx.x % L;
  auto part_row = [&](int p) { return *reinterpret_cast<const f32x4*>(a.part_rows + slot(p) * D + col0 + c * 4); };
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  if (grp < used) o = part_row(grp);  // (on its way while the weights are formed)
  float2 ms[N];
  float top = -INFINITY, sum = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int p = int(threadIdx.x) + i * kThreads;
    ms[i] = p < used ? a.part_sums[slot(p)] : float2{-INFINITY, 0.f};
    top = fmaxf(top, ms[i].x);
  }
  auto wave_all = [](float v, auto f) {
#pragma unroll
    for (int d = 1; d < 16; d *= 2) v = f(v, __shfl_xor(v, d));
    return over_rows(v, f);
  };
  top = wave_all(top, [](float p, float q) { return fmaxf(p, q); });
  if ((threadIdx.x & 63) == 0) wave_max[threadIdx.x >> 6] = top;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kWaves; ++i) top = fmaxf(top, wave_max[i]);
  const float base = top == -INFINITY ? 0.f : top;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float w = fast_exp2(ms[i].x - base);
    sum = fmaf(w, ms[i].y, sum);
    weight[threadIdx.x + i * kThreads] = w;
  }
  sum = wave_all(sum, [](float p, float q) { return p + q; });
  if ((threadIdx.x & 63) == 0) wave_sum[threadIdx.x >> 6] = sum;
  __syncthreads();
  if (grp < used) o *= weight[grp];
#pragma unroll 8
  for (int p = grp + G; p < used; p += G) o += weight[p] * part_row(p);
  rows[grp][c] = o;
  __syncthreads();
  if (grp > 0) return;
  sum = wave_sum[0];
#pragma unroll
  for (int i = 1; i < kWaves; ++i) sum += wave_sum[i];
#pragma unroll
  for (int i = 1; i < G; ++i) o += rows[i][c];
  const float inv = sum == 0.f ? 0.f : 1.0f / sum;
  ntp_gemm::u16x4 out;
#pragma unroll
  for (int r = 0; r < 4; ++r) out[r] = ntp_gemm::f32_to_bf16(o[r] * inv);
  *reinterpret_cast<ntp_gemm::u16x4*>(a.C + int64_t(seq) * a.ldc + int64_t(head) * D + col0 + c * 4) = out;
  if (a.LSE && col0 + c == 0) a.LSE[int64_t(head) * a.n_seq + seq] = (base + log2f(sum)) * 0.6931471805599453f;
}

int check_decode_shape(const ntp_attn_decode_shape_t* s) {
  if (!s || s->n_seq < 0 || s->max_len < 0 || s->q_cnt < 0 || s->kv_cnt < 0 || s->q_off < 0 || s->kv_off < 0 || s->group < 1) return NTP_ERR_INVALID_ARG;
  if (s->head_dim != 64 && s->head_dim != 128) return NTP_ERR_UNSUPPORTED;
  if (s->max_len > 1 << 30 || int64_t(s->n_seq) * s->q_cnt > 0x7fffffffll || int64_t(s->q_off) + s->q_cnt > 0x7fffffffll) return NTP_ERR_UNSUPPORTED;
  // the KV heads of the local query heads ascend: the first and the last must be local
  if (s->q_cnt > 0) {
    const int64_t first = int64_t(s->q_off) / s->group - s->kv_off, last = (int64_t(s->q_off) + s->q_cnt - 1) / s->group - s->kv_off;
    if (first < 0 || last >= s->kv_cnt) return NTP_ERR_INVALID_ARG;
  }
  return NTP_OK;
}

struct DecodeChoice {
  int32_t kv_first, kv_used, head_tiles, shares;  // shares: 0 where workgroup = unit
  int64_t units, ws_bytes;
};

// How a call is cut: into two shares per compute unit (a workgroup's tiles take 64 KB of the LDS), but no more than there can be steps.  Not where units are too short
// for the join's launch to pay: of at most 4 steps, or 8 where half the compute units have one (one sequence, one KV head, 512 tokens 7.2 us whole and 8.2 cut, 1021
// tokens 10.5 / 8.3; 8 KV heads, 1024 tokens: 16 sequences 15.3 / 17.1, 64 42.4 / 45.7, of up to 1024 29.2 / 33.7; 2048 tokens: 16 sequences of up to 2048 24.9 / 19.2).
// Longer units are cut also where there are many, since the lengths are not known here: 512 sequences, 8 KV heads, max_len 8192: lengths of 1 .. 8192 1337 / 1250 us,
// 1 .. 400 69 / 86, 1 .. 200 and one of 8192 116 / 59.
DecodeChoice choose_decode(const ntp_handle* h, int64_t ws_bytes, const ntp_attn_decode_shape_t* s) {
  DecodeChoice c{};
  if (s->q_cnt == 0 || s->n_seq == 0) return c;
  c.kv_first = s->q_off / s->group - s->kv_off;
  c.kv_used = (s->q_off + s->q_cnt - 1) / s->group - s->kv_off - c.kv_first + 1;
  c.head_tiles = (std::min(s->group, s->q_cnt) + 15) / 16;
  c.units = int64_t(c.kv_used) * c.head_tiles * s->n_seq;
  const int64_t step = s->head_dim == 128 ? kStep<128> : kStep<64>, steps = std::max<int64_t>((s->max_len + step - 1) / step, 1);
  if (steps <= 4 || (steps <= 8 && c.units >= h->compute_units / 2) || steps * c.units > 0x7fffffffll) return c;
  const int64_t shares = std::min<int64_t>(std::min(2 * int64_t(h->compute_units), steps * c.units), kMaxShares);
  const int64_t bytes = shares * 2 * 16 * (s->head_dim + 2) * 4;
  if (bytes <= ws_bytes) {
    c.shares = int32_t(shares);
    c.ws_bytes = bytes;
  }
  return c;
}

}  // namespace

int ntp::attn_decode_workspace_wish(const ntp_handle* h, const ntp_attn_decode_shape_t* s, int64_t* bytes) {
  if (check_decode_shape(s) != NTP_OK) return NTP_ERR_INVALID_ARG;
  *bytes = choose_decode(h, INT64_MAX, s).ws_bytes;
  return NTP_OK;
}

extern "C" int ntp_attn_decode_shard(ntp_handle_t* h, const ntp_attn_decode_shape_t* s, const ntp_kv_cache_t* cache, const void* Q, int64_t ldq,
                                     const int32_t* block_table, int64_t ldt, const int32_t* lengths, void* C, int64_t ldc, float* LSE,
                                     void* stream) {
  int st = check_decode_shape(s);
  if (st != NTP_OK) return st;
  if (!h || (st = ntp::check_kv_cache(cache, s->kv_cnt, s->head_dim)) != NTP_OK) return h ? st : NTP_ERR_INVALID_ARG;
  if (s->n_seq == 0 || s->q_cnt == 0) return NTP_OK;
  if (int64_t(s->n_seq) * s->q_cnt > kMaxGrid) return NTP_ERR_UNSUPPORTED;
  const int64_t w = int64_t(s->q_cnt) * s->head_dim, pages = (int64_t(s->max_len) + cache->page_size - 1) / cache->page_size;
  if (!Q || !C || !lengths || (!block_table && pages > 0) || ldq < w || ldc < w || ldt < pages) return NTP_ERR_INVALID_ARG;
  auto off4 = [](const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3) != 0; };
  if (off16(Q) || off16(C) || ldq % 8 || ldc % 8 || off4(block_table) || off4(lengths) || off4(LSE)) return NTP_ERR_ALIGNMENT;
  if (h->device < 0) return NTP_ERR_NO_DEVICE;
  const DecodeChoice c = choose_decode(h, h->workspace ? h->workspace_bytes : 0, s);
  DecodeArgs a{};
  a.Q = static_cast<const uint16_t*>(Q), a.K = static_cast<const uint16_t*>(cache->K), a.V = static_cast<const uint16_t*>(cache->V);
  a.table = block_table, a.lengths = lengths, a.C = static_cast<uint16_t*>(C), a.LSE = LSE;
  if (c.shares > 0) {
    a.part_rows = static_cast<float*>(h->workspace);
    a.part_sums = reinterpret_cast<float2*>(a.part_rows + int64_t(c.shares) * 2 * 16 * s->head_dim);
  }
  a.ldq = ldq, a.ldc = ldc, a.ldt = ldt, a.page_stride = cache->page_stride, a.n_pages = int32_t(cache->n_pages);
  a.n_seq = s->n_seq, a.max_len = s->max_len, a.q_cnt = s->q_cnt, a.q_off = s->q_off, a.kv_off = s->kv_off, a.group = s->group;
  a.page_size = cache->page_size, a.page_log2 = ntp::log2_of(cache->page_size);
  a.kv_first = c.kv_first, a.kv_used = c.kv_used, a.head_tiles = c.head_tiles, a.shares = c.shares;
  a.scale_log2 = float(1.4426950408889634 / std::sqrt(double(s->head_dim)));
  hipStream_t hs = static_cast<hipStream_t>(stream);
  if (ntp::timing_on(h))
    ntp::timing_begin(h, stream, c.shares > 0 ? "attn_decode_cut" : "attn_decode", 4.0 * s->n_seq * double(s->max_len) * s->head_dim * s->q_cnt, 0.0);
  // Joined per (sequence, query head), or per border between shares where that is fewer workgroups: many sequences, of which few are cut
  // (1024 sequences of 1 .. 400 tokens, 32 heads over 8 KV heads: 276 -> 170 us with the search of 512 sequences at a time).
  const int32_t rows = std::min(16, std::min(s->group, s->q_cnt));
  int64_t n_joins = int64_t(s->n_seq) * s->q_cnt;
  if (c.shares > 0 && n_joins > int64_t(c.shares - 1) * rows) {
    a.join_rows = rows;
    n_joins = int64_t(c.shares - 1) * rows;
  }
  const dim3 grid{uint32_t(c.shares > 0 ? c.shares : c.units)}, joins{uint32_t(n_joins)}, split{uint32_t(n_joins * (s->head_dim / kFewColumns))};
  if (s->head_dim == 128) hipLaunchKernelGGL(attn_decode_kernel<128>, grid, dim3(kThreads), 0, hs, a);
  else hipLaunchKernelGGL(attn_decode_kernel<64>, grid, dim3(kThreads), 0, hs, a);
  bool ok = hipGetLastError() == hipSuccess;
  if (ok && c.shares > 1) {
    const bool few = c.shares >= 32 * c.units;
    if (s->head_dim == 128) {
      if (few) hipLaunchKernelGGL((attn_decode_join_kernel<128, kFewColumns>), split, dim3(kThreads), 0, hs, a);
      else hipLaunchKernelGGL((attn_decode_join_kernel<128, 128>), joins, dim3(kThreads), 0, hs, a);
    } else {
      if (few) hipLaunchKernelGGL((attn_decode_join_kernel<64, kFewColumns>), split, dim3(kThreads), 0, hs, a);
      else hipLaunchKernelGGL((attn_decode_join_kernel<64, 64>), joins, dim3(kThreads), 0, hs, a);
    }
    ok = hipGetLastError() == hipSuccess;
  }
  ntp::timing_end(h, stream);
  return ok ? NTP_OK : NTP_ERR_LAUNCH;
}
