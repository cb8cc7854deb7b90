// What the parts of the attention of chunks of new tokens share: arguments, and which rows and tokens a sequence has (not part of the ABI).
#ifndef NTP_ATTN_CHUNK_H_
#define NTP_ATTN_CHUNK_H_

#include "ntp_attn_lds.h"

namespace ntp_chunk {

using namespace ntp_attn;
using ntp_gemm::bf16x8;
using ntp_gemm::f32x4;

constexpr int kThreads = 256, kWaves = 4, kBlock = 16;  // kBlock: tokens that are contiguous in a page
constexpr int kMaxShares = 512;                         // of the line of steps (ntp_attn_chunk_rows.h)
constexpr int kTileRows = 128, kTileKeys = 64;          // of ntp_attn_chunk_tiles.h

struct ChunkArgs {
  const uint16_t* Q;
  const unsigned char *K, *V;
  const uint8_t *K_exp, *V_exp;
  const int32_t *starts, *table, *lengths;
  uint16_t* C;
  float* LSE;
  // workspace; NULL: not cut.  Per share of the line two partial results (of the unit it begins inside and the one it ends inside), of `cap` rows each: maximum (log2 units) and
  // sum, and the D unnormalised outputs
  float2* part_sums;
  float* part_rows;
  int32_t* plan;      // how the row tiles' walks are cut: units, pieces, key tiles of a piece
  float* tile_parts;  // per piece of a tile's walk its rows: D unnormalised outputs, maximum and sum, two unused
  int64_t ldq, ldc, ldt, page_stride, exp_stride;
  int32_t M, n_pages, n_seq, max_new, max_len, q_cnt, q_off, kv_off, group, page_size, page_log2;
  int32_t kv_first, kv_used, gmax;  // local KV heads that are read; the most local query heads of one
  int32_t g_first, g_last;          // those of the first and of the last
  int32_t cap;                      // sequences of up to so many rows (tokens x gmax) go by ntp_attn_chunk_rows.h, the others by ntp_attn_chunk_tiles.h
  int32_t shares, tile_wgs;         // shares that the line is cut into at most; workgroups of a launch of both kinds that take row tiles (the first ones)
  int32_t slots;                    // workgroups that the device has room for, which walks are cut for (into up to twice as many pieces); 0: never
  int32_t parts;                    // 0, or that many pieces of the longest walk (NTP_OPT_ATTN_PARTS)
  float scale_log2;                 // log2(e) / sqrt(d)
};

// A sequence's first row, its rows, and its tokens; none where i is behind the last.  No branch, so that all loads, also those of several sequences, go out together.
__device__ __forceinline__ void extent(const ChunkArgs& a, int i, int& start, int& n, int& len) {
  const int at = min(i, a.n_seq - 1);
  const bool packed = a.starts != nullptr, there = i < a.n_seq;
  const int32_t* const starts = packed ? a.starts : a.lengths;  // (anything that may be read)
  const int tokens = a.lengths[at], from = starts[at], to = starts[packed ? at + 1 : at];
  start = packed ? min(max(from, 0), a.M) : at;
  n = packed ? max(min(max(to, 0), a.M) - start, 0) : 1;
  n = there ? n : 0;
  len = there ? min(max(tokens, 0), a.max_len) : 0;
}

// The local query heads j0 .. j1 - 1 of a local KV head.
struct Heads {
  int j0, j1;
  __device__ __forceinline__ Heads(const ChunkArgs& a, int g) {
    const int64_t first = int64_t(a.kv_off + g) * a.group - a.q_off;
    j0 = int(first > 0 ? first : 0);
    const int64_t end = first + a.group;
    j1 = int(end < a.q_cnt ? end : a.q_cnt);
  }
};

__device__ __forceinline__ float power_of(uint32_t code) { return __builtin_bit_cast(float, code << 23); }  // 2^(code - 127)

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
// Eight e4m3 numbers times a power of two, which bf16 holds exactly.
__device__ __forceinline__ bf16x8 from_e4m3(u32x2 v, float power) {
  bf16x8 out;
#if defined(__HIP_DEVICE_COMPILE__)
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    const bf16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[w], power, false), hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[w], power, true);
    out[4 * w] = lo[0], out[4 * w + 1] = lo[1], out[4 * w + 2] = hi[0], out[4 * w + 3] = hi[1];
  }
#endif
  return out;
}

__device__ __forceinline__ float larger(float x, float y) { return fmaxf(x, y); }
__device__ __forceinline__ float added(float x, float y) { return x + y; }

}  // namespace ntp_chunk

#endif  // NTP_ATTN_CHUNK_H_
