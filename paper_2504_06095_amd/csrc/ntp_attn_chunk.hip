// Attention of chunks of new tokens over the paged cache (ntp_attn_chunk_shard): row i of a sequence's n new ones sees its first len - n + i + 1 tokens,
//   C[row, j] = sum_t p_t V[t] / sum_t p_t,   p_t = exp(q_j . K[t] / sqrt(d) - max).
// One pass over the tokens with a running maximum and sum.  Sequences of up to 32 rows (new tokens x query heads of a KV head) are bound by HBM and go by
// ntp_attn_chunk_rows.h, the others by the matrix instructions and by ntp_attn_chunk_tiles.h; one launch holds workgroups of both kinds, since which sequences are which only the device
// knows, and one more joins what was cut.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "ntp_attn_chunk_rows.h"
#include "ntp_attn_chunk_tiles.h"
#include "ntp_internal.h"
#include "ntp_kv_cache.h"

namespace {

using namespace ntp_chunk;
using ntp::off16;

template <int D, bool FP8, int QB>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2))) void chunk_rows_kernel(const ChunkArgs a) {
  __shared__ __attribute__((aligned(1024))) unsigned char lds[kRowLds<D, QB>];
  chunk_rows<D, FP8, QB>(a, int(blockIdx.x), lds);
}

template <int D, bool FP8>
__global__ __attribute__((amdgpu_flat_work_group_size(kThreads, kThreads), amdgpu_waves_per_eu(2, 2))) void chunk_both_kernel(const ChunkArgs a) {
  __shared__ __attribute__((aligned(1024))) unsigned char lds[std::max(kRowLds<D, 2>, kTileLds<D>)];
  // (the row tiles first: their walks are the longest, and what reads from HBM alone fills the compute units that they leave)
  if (int(blockIdx.x) < a.tile_wgs) chunk_tiles<D, FP8>(a, int(blockIdx.x), lds);
  else chunk_rows<D, FP8, 2>(a, int(blockIdx.x) - a.tile_wgs, lds);
}

template <int D, bool FP8>
__global__ __attribute__((amdgpu_flat_work_group_size(kThreads, kThreads), amdgpu_waves_per_eu(kPlaces<D, FP8>, kPlaces<D, FP8>))) void chunk_tiles_kernel(const ChunkArgs a) {
  __shared__ __attribute__((aligned(1024))) unsigned char lds[kTileLds<D>];
  chunk_tiles<D, FP8>(a, int(blockIdx.x), lds);
}

// Workgroups: first those of the line's units, then those of the row tiles.
enum { kByBorder, kByUnit, kLengthy };  // border between shares and some rows; unit and some rows; unit, row and some columns
struct Joins {
  int32_t kind, rows, row_jobs;  // rows of a unit; workgroups for the units
};
template <int D, bool FP8, int QB>
__global__ __launch_bounds__(kThreads) void chunk_join_kernel(const ChunkArgs a, const Joins j) {
  constexpr int STEP = RowFormat<D, FP8, QB>::STEP, R = 16 * QB;
  const int wg = int(blockIdx.x);
  if (wg < j.row_jobs) {
    constexpr int SPLIT = D / kFewColumns, AT_ONCE = kThreads / (D / 4);
    if (j.kind == kLengthy) {
      chunk_rows_join_long<D, STEP, R>(a, wg / SPLIT / j.rows, wg / SPLIT % j.rows, wg % SPLIT * kFewColumns);
    } else {
      const int per = (j.rows + AT_ONCE - 1) / AT_ONCE;
      CutUnit u;
      if (j.kind == kByUnit ? u.by_number<STEP>(a, wg / per) : u.by_border<STEP>(a, wg / per + 1)) chunk_rows_join_short<D, R>(a, u, wg % per * AT_ONCE);
    }
  } else {
    chunk_tiles_join<D>(a, wg - j.row_jobs, int(gridDim.x) - j.row_jobs);
  }
}

int check_chunk_shape(const ntp_attn_chunk_shape_t* s) {
  if (!s || s->M < 0 || s->n_seq < 0 || s->max_new < 0 || s->max_len < 0 || s->q_cnt < 0 || s->kv_cnt < 0 || s->q_off < 0 || s->kv_off < 0 || s->group < 1) return NTP_ERR_INVALID_ARG;
  if (s->head_dim != 64 && s->head_dim != 128) return NTP_ERR_UNSUPPORTED;
  if (s->max_len > 1 << 30 || int64_t(s->q_off) + s->q_cnt > 0x7fffffffll || s->M > 0x7fffffffll || s->M * std::max(s->q_cnt, 1) > 0x7fffffffll ||
      int64_t(s->n_seq) * ((int64_t(s->max_len) + 63) / 64 + 1) * std::max(s->kv_cnt, 1) > 0x7fffffffll || s->q_cnt > 1 << 20)
    return NTP_ERR_UNSUPPORTED;
  // row tiles are counted in 32 bits, also where row_starts gives every sequence as many rows as there may be
  const int64_t per_seq = std::min<int64_t>(s->max_new, s->M) * s->q_cnt / kTileRows + s->kv_cnt;
  if (per_seq > 0x7fffffffll / std::max(s->n_seq, 1)) return NTP_ERR_UNSUPPORTED;
  // the KV heads of the local query heads ascend: the first and the last must be local
  if (s->q_cnt > 0) {
    const int64_t first = int64_t(s->q_off) / s->group - s->kv_off, last = (int64_t(s->q_off) + s->q_cnt - 1) / s->group - s->kv_off;
    if (first < 0 || last >= s->kv_cnt) return NTP_ERR_INVALID_ARG;
  }
  return NTP_OK;
}

struct ChunkChoice {
  int32_t kv_first, kv_used, gmax, g_first, g_last, cap, qb;
  int64_t row_wgs;                  // workgroups that take sequences of few rows
  int32_t shares, rows;             // shares of their line (0: workgroup = unit); most rows of a unit
  int64_t units;                    // such units at most
  int64_t tiles;                    // (sequence, KV head, row tile)s of the others at most
  int64_t tile_wgs;                 // workgroups for them
  int32_t slots;                    // workgroups that the device has room for: walks are cut for these (0: never), into twice as many at most
  int64_t ws_rows, ws_bytes;        // bytes of the line's partial results, and of all
};

ChunkChoice choose_chunk(const ntp_handle* h, int64_t ws_bytes, const ntp_attn_chunk_shape_t* s, bool fp8) {
  ChunkChoice c{};
  const int64_t most = std::min<int64_t>(s->max_new, s->M);  // rows of a sequence
  if (s->q_cnt == 0 || s->n_seq == 0 || most == 0) return c;
  c.kv_first = s->q_off / s->group - s->kv_off;
  c.kv_used = (s->q_off + s->q_cnt - 1) / s->group - s->kv_off - c.kv_first + 1;
  c.g_first = std::min(s->group - s->q_off % s->group, s->q_cnt);
  c.g_last = c.kv_used > 1 ? (s->q_off + s->q_cnt - 1) % s->group + 1 : c.g_first;
  c.gmax = c.kv_used > 2 ? s->group : std::max(c.g_first, c.g_last);
  c.qb = most * c.gmax <= 16 ? 1 : 2;
  const bool tiles = most * c.gmax > 32;
  c.cap = tiles && (s->n_seq == 1 || c.gmax > 32) ? 0 : 16 * c.qb;
  if (c.cap > 0) {
    c.units = int64_t(s->n_seq) * c.kv_used;
    c.rows = int32_t(std::min<int64_t>(c.cap, most * c.gmax));
  }
  if (tiles) {
    const int64_t seqs = std::min<int64_t>(s->n_seq, s->M * c.gmax / (c.cap + 1));  // that are not of few rows
    auto tiles_of = [&](int32_t G) { return std::min<int64_t>(s->n_seq * ((most * G + kTileRows - 1) / kTileRows), s->M * G / kTileRows + seqs); };
    c.tiles = tiles_of(c.g_first) + std::max(c.kv_used - 2, 0) * tiles_of(c.gmax) + (c.kv_used > 1 ? tiles_of(c.g_last) : 0);
  }
  const int64_t step = s->head_dim == 128 ? 128 : 256, steps = std::max<int64_t>((s->max_len + step - 1) / step, 1);  // (8-bit steps of up to 16 rows are twice as long)
  if (c.units > 0 && steps > 4 && (steps > 8 || c.units < h->compute_units / 2)) {
    c.shares = int32_t(std::min<int64_t>(std::min((tiles ? 1 : 2) * int64_t(h->compute_units), steps * c.units), kMaxShares));
    c.ws_rows = (int64_t(c.shares) * 2 * c.cap * (s->head_dim + 2) * 4 + 255) / 256 * 256;
  }
  if (tiles && s->max_len > kMinPiece * kTileKeys) c.slots = (s->head_dim == 64 && c.cap == 0 && !fp8 ? kPlaces<64, false> : kPlaces<128, false>) * h->compute_units;
  c.ws_bytes = c.ws_rows + (c.slots > 0 ? 256 + int64_t(2 * c.slots) * kTileRows * (s->head_dim + kPartPad) * 4 : 0);
  if (c.ws_bytes > ws_bytes) c.shares = c.slots = 0, c.ws_rows = c.ws_bytes = 0;
  c.row_wgs = c.shares > 0 ? c.shares : c.units;
  if (tiles) c.tile_wgs = (std::max<int64_t>(c.tiles, 2 * c.slots) + 8 * kRun - 1) / (8 * kRun) * (8 * kRun);
  return c;
}

}  // namespace

int ntp::attn_chunk_workspace_wish(const ntp_handle* h, const ntp_attn_chunk_shape_t* s, int64_t* bytes) {
  if (check_chunk_shape(s) != NTP_OK) return NTP_ERR_INVALID_ARG;
  *bytes = std::max(choose_chunk(h, INT64_MAX, s, false).ws_bytes, choose_chunk(h, INT64_MAX, s, true).ws_bytes);
  return NTP_OK;
}

namespace {

constexpr int kJoinWgs = 1024;  // that join row tiles

template <int D, bool FP8>
bool launch_chunk(const ChunkArgs& a, const ChunkChoice& c, hipStream_t hs) {
  const dim3 grid{uint32_t(c.row_wgs + c.tile_wgs)}, block{kThreads};
  if (c.tiles > 0 && c.cap > 0) hipLaunchKernelGGL((chunk_both_kernel<D, FP8>), grid, block, 0, hs, a);
  else if (c.tiles > 0) hipLaunchKernelGGL((chunk_tiles_kernel<D, FP8>), grid, block, 0, hs, a);
  else if (c.qb == 1) hipLaunchKernelGGL((chunk_rows_kernel<D, FP8, 1>), grid, block, 0, hs, a);
  else hipLaunchKernelGGL((chunk_rows_kernel<D, FP8, 2>), grid, block, 0, hs, a);
  if (hipGetLastError() != hipSuccess) return false;
  if (c.shares <= 1 && c.slots == 0) return true;
  constexpr int AT_ONCE = kThreads / (D / 4);
  const int64_t per = (c.rows + AT_ONCE - 1) / AT_ONCE;
  Joins j{c.shares >= 32 * c.units ? kLengthy : c.units < c.shares ? kByUnit : kByBorder, c.rows, 0};
  if (c.shares > 1) j.row_jobs = int32_t(j.kind == kLengthy ? c.units * c.rows * (D / kFewColumns) : (j.kind == kByUnit ? c.units : c.shares - 1) * per);
  const int64_t tile_jobs = c.slots > 0 ? std::min<int64_t>(kJoinWgs, c.tiles * (kTileRows / 2)) : 0;
  const dim3 jobs{uint32_t(j.row_jobs + tile_jobs)};
  if (c.qb == 1) hipLaunchKernelGGL((chunk_join_kernel<D, FP8, 1>), jobs, block, 0, hs, a, j);
  else hipLaunchKernelGGL((chunk_join_kernel<D, FP8, 2>), jobs, block, 0, hs, a, j);
  return hipGetLastError() == hipSuccess;
}

}  // namespace

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
  const bool fp8 = pages->format == NTP_KV_E4M3;
  const ChunkChoice c = choose_chunk(h, h->workspace ? h->workspace_bytes : 0, s, fp8);
  if (c.row_wgs + c.tile_wgs > 0xffffffffll / kThreads) return NTP_ERR_UNSUPPORTED;  // a launch counts its threads in 32 bits
  if (h->device < 0) return NTP_ERR_NO_DEVICE;
  ChunkArgs a{};
  a.Q = static_cast<const uint16_t*>(Q), a.K = static_cast<const unsigned char*>(pages->K), a.V = static_cast<const unsigned char*>(pages->V);
  a.K_exp = static_cast<const uint8_t*>(pages->K_exp), a.V_exp = static_cast<const uint8_t*>(pages->V_exp);
  a.starts = row_starts, a.table = block_table, a.lengths = lengths, a.C = static_cast<uint16_t*>(C), a.LSE = LSE;
  if (c.shares > 0) {
    a.part_rows = static_cast<float*>(h->workspace);
    a.part_sums = reinterpret_cast<float2*>(a.part_rows + int64_t(c.shares) * 2 * c.cap * s->head_dim);
  }
  if (c.slots > 0) {
    a.plan = reinterpret_cast<int32_t*>(static_cast<char*>(h->workspace) + c.ws_rows);
    a.tile_parts = reinterpret_cast<float*>(a.plan + 64);
  }
  a.ldq = ldq, a.ldc = ldc, a.ldt = ldt, a.page_stride = pages->page_stride, a.exp_stride = pages->exp_stride;
  a.M = int32_t(s->M), a.n_pages = int32_t(pages->n_pages), a.n_seq = s->n_seq, a.max_new = s->max_new, a.max_len = s->max_len;
  a.q_cnt = s->q_cnt, a.q_off = s->q_off, a.kv_off = s->kv_off, a.group = s->group, a.page_size = pages->page_size, a.page_log2 = ntp::log2_of(pages->page_size);
  a.kv_first = c.kv_first, a.kv_used = c.kv_used, a.gmax = c.gmax, a.g_first = c.g_first, a.g_last = c.g_last, a.cap = c.cap, a.shares = c.shares, a.tile_wgs = int32_t(c.tile_wgs), a.slots = c.slots, a.parts = int32_t(h->opt[NTP_OPT_ATTN_PARTS]);
  a.scale_log2 = float(1.4426950408889634 / std::sqrt(double(s->head_dim)));
  hipStream_t hs = static_cast<hipStream_t>(stream);
  if (ntp::timing_on(h)) ntp::timing_begin(h, stream, fp8 ? "attn_chunk8" : "attn_chunk", 0.0, 0.0);  // (lengths are on the device)
  const bool ok = s->head_dim == 128 ? (fp8 ? launch_chunk<128, true>(a, c, hs) : launch_chunk<128, false>(a, c, hs))
                                     : (fp8 ? launch_chunk<64, true>(a, c, hs) : launch_chunk<64, false>(a, c, hs));
  ntp::timing_end(h, stream);
  return ok ? NTP_OK : NTP_ERR_LAUNCH;
}
