// Chunk attention, sequences of many rows: 4 d operations a (row, token) on the matrix pipe, about five vector instructions beside them for the softmax, which bound it together (512
// tokens behind 130560, 16 heads on one KV head: bf16 472 us, 1.16 PFLOP/s, 8 bits 513, the pipe busy for 44 % and the vector unit for 53 % of it; one prompt of 8192 tokens, 14 heads:
// 234 us, 1.03 PFLOP/s; d = 64: 162 us).
//
// A workgroup takes 128 rows (token i, head h of a KV head's G: number i G + h) of a sequence and KV head, a wavefront 32 of them in two blocks of 16, and walks over the
// tokens that they see in tiles of 64, which all wavefronts share: two buffers a matrix, one barrier a tile, two workgroups a compute unit.  Grouped heads stand in one tile,
// so that 16 query heads on one KV head read its tokens once and not 16 times.  bf16 tiles come by DMA, wavefront w the tile's block w of 16 tokens (a page holds at least
// 16); 8-bit ones through registers, where they become bf16 (exact: e4m3 times a power of two) before the LDS, once for all wavefronts: converted where fragments
// are read it would be four times the work, on the vector unit that the softmax needs.
//
// Where a batch has fewer tiles than the GPU has room for, walks are cut into pieces, by the lengths on the device, whose partial results a second kernel joins
// (512 tokens behind 130560: 64 tiles in 512 pieces; their join 9 us).  Up to 64 sequences, one a lane, are looked at together: whole walks go longest first, and the best of several cuts is
// taken.  Of more, whole walks go as they stand in the batch (64 prompts of up to 512 tokens, 14 heads: 97 us, 65: 108) and one cut is tried.
#ifndef NTP_ATTN_CHUNK_TILES_H_
#define NTP_ATTN_CHUNK_TILES_H_

#include "ntp_attn_chunk.h"

namespace ntp_chunk {

constexpr int kMinPiece = 4;  // key tiles of a piece at least
constexpr int kPartPad = 4;   // floats behind a partial row's outputs: maximum, sum
constexpr int kRun = 4;       // neighbouring pieces, which read the same tokens, that stay on one XCD
template <int D, bool FP8>
constexpr int kPlaces = D == 64 && !FP8 ? 3 : 2;  // workgroups that a compute unit has room for (8-bit tiles of 64 columns: a third takes registers that a walk needs)

// Of a sequence's KV heads: the first and the last that are read may be read by a part of their group only.
struct PerHead {
  int first, middle, last;
  __device__ __forceinline__ int all(const ChunkArgs& a, int times = 1) const { return times * (first + max(a.kv_used - 2, 0) * middle + (a.kv_used > 1 ? last : 0)); }
  // entry x of all heads', `times` of them for each here: its head and the number in it
  __device__ __forceinline__ int find(const ChunkArgs& a, int times, int& x) const {
    if (x < times * first) return 0;
    x -= times * first;
    const int m = middle > 0 ? min(x / (times * middle), max(a.kv_used - 2, 0)) : max(a.kv_used - 2, 0);
    x -= m * times * middle;
    return 1 + m;
  }
  __device__ __forceinline__ int of(const ChunkArgs& a, int head) const { return head == 0 ? first : head < a.kv_used - 1 ? middle : last; }
};

// Row tiles, by KV head, and key tiles (of its last row) of a sequence; no row tiles where it is one of few rows.
__device__ __forceinline__ void tiles_of(const ChunkArgs& a, int n, int len, PerHead& tiles, int& walk) {
  const int used = min(n, a.max_new);
  tiles = PerHead{0, 0, 0};
  if (used > a.cap / a.gmax) {
    auto rows = [&](int G) { return int((int64_t(used) * G + kTileRows - 1) / kTileRows); };
    tiles = PerHead{rows(a.g_first), rows(a.gmax), rows(a.g_last)};
  }
  walk = max(1, (max(len - n + used, 0) + kTileKeys - 1) / kTileKeys);
}

// How the batch's walks are cut, and the piece with number x of them.  Pieces are numbered sequence by sequence, in it KV head by KV head, piece by piece, row tile by row tile from the
// last (the longest walk) on; all tiles of a sequence are cut into the same number.
struct TilePlan {
  int units, total, piece_tiles;  // (sequence, KV head, row tile)s; pieces; key tiles of a piece at most (0: whole)
  int start, n, len, walk;         // this lane's sequence of 64
  PerHead tiles;
  __device__ __forceinline__ void load(const ChunkArgs& a, int i) {
    extent(a, i, start, n, len);
    tiles_of(a, n, len, tiles, walk);
  }
  // (in fp32: a count one too high where walks are of millions of tiles is the same everywhere)
  __device__ __forceinline__ int cut() const { return piece_tiles == 0 ? 1 : int((float(walk) - 0.5f) * __builtin_amdgcn_rcpf(float(piece_tiles))) + 1; }
  static constexpr int kAtOnce = 256;  // sequences whose loads go out together
  // of the sequences from .. from + kAtOnce - 1: units and pieces of this lane's
  __device__ __forceinline__ void sums(const ChunkArgs& a, int from, int& count, int& pieces) {
    count = pieces = 0;
#pragma unroll
    for (int k = 0; k < kAtOnce / 64; ++k) {
      TilePlan p;
      p.load(a, from + k * 64 + int(threadIdx.x & 63));
      p.piece_tiles = piece_tiles;
      count += p.tiles.all(a);
      pieces += p.tiles.all(a, p.cut());
    }
  }
  __device__ __forceinline__ static int all(int v) { return __builtin_amdgcn_readlane(sum_upto(v), 63); }
  // A call's time by an estimate, in key tiles of two workgroups on a compute unit (2.06 us; 1.6 us of one alone), for walks cut into pieces: rounds of whole pieces, or what list
  // scheduling takes at most, a round's way in and out, and partial results written and read again (47 ns a piece).  Taken is the best of whole walks and six cuts.
  template <int D>
  __device__ __forceinline__ void make(const ChunkArgs& a) {
    piece_tiles = 0;
    int count = 0;
    float work = 0.f, most = 0.f;
    load(a, threadIdx.x & 63);
    auto add = [&](const TilePlan& p) {
      const int c = p.tiles.all(a);
      count += c;
      const int used = min(p.n, a.max_new), rows = min(used, max(p.len - p.n + used, 0));  // (rows that see something)
      work += float(c) * (float(p.walk) - float(rows) * (0.5f / kTileKeys));  // (half a triangle less)
      if (c > 0) most = fmaxf(most, float(p.walk));
    };
    if (a.n_seq <= 64) {
      add(*this);
    } else {
      for (int from = 0; from < a.n_seq; from += kAtOnce) {
#pragma unroll
        for (int k = 0; k < kAtOnce / 64; ++k) {
          TilePlan p;
          p.load(a, from + k * 64 + int(threadIdx.x & 63));
          add(p);
        }
      }
    }
    units = total = all(count);
    if (a.slots == 0 || units == 0 || units >= 2 * a.slots) return;
    work = over_wave(work, added), most = over_wave(most, larger);
    const float slots = float(a.slots), share = work / slots;
    if (a.parts == 1 || (a.parts == 0 && most <= 1.3f * share)) return;  // (longest first, whole walks end together)
    if (a.n_seq > 64) {  // (not looked at piece by piece)
      if (a.parts == 0 && (units >= a.slots || most <= 1.5f * share)) return;
      piece_tiles = max(kMinPiece, int(ceilf(a.parts > 0 ? most / float(a.parts) : share)));
      int pieces = 0, c, p;
      for (int from = 0; from < a.n_seq; from += kAtOnce) {
        sums(a, from, c, p);
        pieces += p;
      }
      total = all(pieces);
      if (total <= 2 * a.slots) return;
      piece_tiles = 0, total = units;
      return;
    }
    const auto longest_of = [&] { return over_wave(tiles.all(a) > 0 ? float(walk) * __builtin_amdgcn_rcpf(float(cut())) : 0.0f, larger); };
    auto estimate = [&](float longest, int all_pieces) {
      const float pieces = float(all_pieces), rounds = ceilf(pieces / slots);
      const float walks = 2.0f * pieces <= slots ? 0.78f * longest : fminf(rounds * longest, fmaxf(longest, share + 0.5f * longest));
      return walks + 3.0f * rounds + (all_pieces > units ? pieces * (1.0f / 45) : 0.0f);
    };
    float best = estimate(most, units);
    int best_tiles = 0;
    if (a.parts > 1) best = INFINITY;
    // each wavefront looks at every fourth cut
    __shared__ float best_of[kWaves];
    __shared__ int tiles_of_best[kWaves], total_of_best[kWaves];
    const int wave = uniform(threadIdx.x >> 6);
    for (int j = wave; j < (a.parts > 0 ? 1 : 6); j += kWaves) {
      const float S = a.parts > 0 ? most / float(a.parts) : j < 3 ? most / float(j + 2) : work / (j == 3 ? slots : j == 4 ? 0.5f * slots : fmaxf(slots - float(units), 1.0f));
      piece_tiles = max(kMinPiece, int(ceilf(S)));
      const int pieces = all(tiles.all(a, cut()));
      if (pieces > 2 * a.slots || pieces == units) continue;
      const float t = estimate(longest_of(), pieces);
      if (t < best) best = t, best_tiles = piece_tiles, total = pieces;
    }
    if ((threadIdx.x & 63) == 0) best_of[wave] = best, tiles_of_best[wave] = best_tiles, total_of_best[wave] = total;
    __syncthreads();
    best = best_of[0], best_tiles = tiles_of_best[0], total = total_of_best[0];
#pragma unroll
    for (int k = 1; k < kWaves; ++k)
      if (best_of[k] < best) best = best_of[k], best_tiles = tiles_of_best[k], total = total_of_best[k];
    piece_tiles = uniform(best_tiles), total = uniform(total);
  }
  // Row tiles of this lane's sequence whose walks have `least` key tiles or more: row tile t's last row is min(rows, 128 (t + 1)) - 1, of token len - n + row / G.
  __device__ __forceinline__ PerHead tiles_from(const ChunkArgs& a, int least) const {
    const int used = min(n, a.max_new), m = (least - 1) * kTileKeys - (len - n);  // (tokens of the chunk behind which the walk is so long)
    if (least <= 0 || m <= 0) return tiles;
    if (m >= used) return PerHead{0, 0, 0};
    auto from = [&](int t, int G) { return t > 0 ? t - (m * G + kTileRows) / kTileRows + 1 : 0; };
    return PerHead{from(tiles.first, a.g_first), from(tiles.middle, a.gmax), from(tiles.last, a.g_last)};
  }
  static constexpr int kLevel = 8;  // key tiles
  // x < total: its sequence, KV head, row tile, and piece.  Whole walks of up to 64 sequences come longest first, whosever they are, by levels of their lengths: tiles of a
  // level are numbered sequence by sequence, head by head.
  int seq, head, tile, piece, n_pieces, seq_start, seq_n, seq_len;
  __device__ __forceinline__ void find(const ChunkArgs& a, int x) {
    if (piece_tiles == 0 && a.n_seq <= 64) {
      auto upto = [&](int level) { return all(tiles_from(a, level * kLevel).all(a)); };
      // the level: the highest with more than x tiles in it and above it (none has `hi`: no walk is longer than max_len's)
      int lo = 0, hi = (a.max_len + kTileKeys - 1) / kTileKeys / kLevel + 1, longer = 0;
      while (hi - lo > 1) {
        const int mid = (lo + hi) / 2, count = upto(mid);
        if (count > x) lo = mid;
        else hi = mid, longer = count;
      }
      const PerHead above = tiles_from(a, (lo + 1) * kLevel), from = tiles_from(a, lo * kLevel);
      const PerHead here = {from.first - above.first, from.middle - above.middle, from.last - above.last};
      const int mine = here.all(a), sum = sum_upto(mine);
      const int at = __builtin_ctzll(__ballot(longer + sum > x));
      auto of = [&](int v) { return __builtin_amdgcn_readlane(v, at); };
      const PerHead h = {of(here.first), of(here.middle), of(here.last)}, up = {of(above.first), of(above.middle), of(above.last)}, t = {of(tiles.first), of(tiles.middle), of(tiles.last)};
      int rest = x - longer - (of(sum) - of(mine));
      n_pieces = 1, piece = 0;
      head = h.find(a, 1, rest);
      tile = t.of(a, head) - 1 - up.of(a, head) - rest;
      seq = at, seq_start = of(start), seq_n = of(n), seq_len = of(len);
      return;
    }
    int from = 0, before = 0;
    if (a.n_seq > 64) {
      for (; from < a.n_seq - kAtOnce; from += kAtOnce) {
        int c, p;
        sums(a, from, c, p);
        p = all(p);
        if (before + p > x) break;
        before += p;
      }
      load(a, from + int(threadIdx.x & 63));
    }
    for (;;) {
      const int mine = tiles.all(a, cut()), upto = sum_upto(mine);
      const uint64_t behind = __ballot(before + upto > x);
      if (behind) {
        const int at = __builtin_ctzll(behind);
        auto of = [&](int v) { return __builtin_amdgcn_readlane(v, at); };
        const PerHead h = {of(tiles.first), of(tiles.middle), of(tiles.last)};
        n_pieces = of(cut());
        int rest = x - before - (of(upto) - of(mine));
        head = h.find(a, n_pieces, rest);
        const int t = h.of(a, head);
        tile = t - 1 - rest % t;
        piece = rest / t;
        seq = from + at, seq_start = of(start), seq_n = of(n), seq_len = of(len);
        return;
      }
      before += __builtin_amdgcn_readlane(upto, 63);
      from += 64;
      load(a, from + int(threadIdx.x & 63));
    }
  }
  // unit < units: the same of it, and the number of its first piece; the unit's pieces lie `tiles_there` apart.  -1: there is no such unit
  int tiles_there;
  __device__ __forceinline__ int find_unit(const ChunkArgs& a, int unit) {
    int from = 0, before = 0, pieces = 0;
    if (a.n_seq > 64) {
      for (; from < a.n_seq - kAtOnce; from += kAtOnce) {
        int c, p;
        sums(a, from, c, p);
        c = all(c);
        if (before + c > unit) break;
        before += c;
        pieces += all(p);
      }
      load(a, from + int(threadIdx.x & 63));
    }
    for (; from < a.n_seq;) {
      const int mine = tiles.all(a), cut_up = tiles.all(a, cut()), upto = sum_upto(mine), pieces_upto = sum_upto(cut_up);
      const uint64_t behind = __ballot(before + upto > unit);
      if (behind) {
        const int at = __builtin_ctzll(behind);
        auto of = [&](int v) { return __builtin_amdgcn_readlane(v, at); };
        const PerHead h = {of(tiles.first), of(tiles.middle), of(tiles.last)};
        n_pieces = of(cut());
        const int number = unit - before - (of(upto) - of(mine));
        int place = number;
        head = h.find(a, 1, place);
        tiles_there = h.of(a, head);
        tile = tiles_there - 1 - place;
        seq_start = of(start), seq_n = of(n);
        return pieces + of(pieces_upto) - of(cut_up) + (number - place) * n_pieces + place;
      }
      before += __builtin_amdgcn_readlane(upto, 63);
      pieces += __builtin_amdgcn_readlane(pieces_upto, 63);
      from += 64;
      load(a, from + int(threadIdx.x & 63));
    }
    return -1;
  }
};

template <int D>
constexpr int kTileLds = 4 * kTileKeys * D * 2;

template <int D>
__device__ __forceinline__ uint32_t tile_swz(int r) {
  return D == 128 ? uint32_t((r & 7) << 1) : uint32_t(((r >> 1) & 3) << 1);
}

template <int D, bool FP8>
__device__ __forceinline__ void chunk_tiles(const ChunkArgs& a, const int wg, unsigned char* const lds) {
  constexpr int KS = D / 32, DB = D / 16, QB = 2;
  constexpr int TILE = kTileKeys * D * 2, BLOCK = kBlock * D * 2;  // bytes in the LDS
  constexpr int NI = BLOCK / 1024;                                 // DMA instructions per wavefront, matrix and tile
  constexpr int NL = FP8 ? kBlock * D / 1024 : 1;                  // or loads of 16 8-bit elements a lane
  const int lane = threadIdx.x & 63, lq = lane & 15, lh = lane >> 4;
  const int wave = uniform(threadIdx.x >> 6);

  TilePlan plan;
  plan.make<D>(a);
  if (wg == 0 && threadIdx.x == 0 && a.plan) a.plan[0] = plan.units, a.plan[1] = plan.total, a.plan[2] = plan.piece_tiles;  // for the kernel that joins
  // Runs of pieces on one XCD (workgroup b runs on XCD b % 8, and there on shader engine b / 8 % 4), turned by one with every eight of them and inside, so that no XCD and no
  // engine has all the long ones (four sequences of 2048 tokens, 14 heads: without the second, compute units ended after 67 to 103 us)
  const int in_xcd = wg / 8, round = in_xcd / kRun;
  const int id = uniform((round * 8 + ((wg - round) & 7)) * kRun + (in_xcd + round) % kRun);
  if (id >= plan.total) return;
  plan.find(a, id);
  const int seq = uniform(plan.seq), start = uniform(plan.seq_start), n = uniform(plan.seq_n), len = uniform(plan.seq_len), used = min(n, a.max_new);
  const int g = a.kv_first + uniform(plan.head), n_pieces = uniform(plan.n_pieces), piece = uniform(plan.piece);
  const Heads hd(a, g);
  const int G = uniform(hd.j1 - hd.j0), j0 = uniform(hd.j0), rows = used * G, row0 = uniform(plan.tile) * kTileRows;
  if (row0 >= rows) return;  // (a KV head that only a part of its group reads)
  const int end = max(len - n + (min(rows, row0 + kTileRows) - 1) / G + 1, 0);  // tokens that the tile's last row sees
  const int walk = (end + kTileKeys - 1) / kTileKeys;
  const int t_lo = int(int64_t(piece) * walk / n_pieces), t_hi = int(int64_t(piece + 1) * walk / n_pieces);

  // the tile's row r is of token token0 + (rest0 + r) / G; the quotient of such small numbers by a product with the reciprocal
  const int token0 = row0 / G, rest0 = row0 - token0 * G;
  const float per_G = 1.0f / float(G);
  auto token_of = [&](int r) { return token0 + int((float(rest0 + r) + 0.5f) * per_G); };

  // this wavefront's rows: their queries, and how many tokens they see
  const int w0 = row0 + wave * 16 * QB;
  const int all_see = len - n + token_of(wave * 16 * QB) + 1, most = w0 < rows ? len - n + token_of(min(rows - row0, wave * 16 * QB + 16 * QB) - 1) + 1 : 0;
  // Page numbers of 16 tiles' four blocks, one a lane, and which of them there are not; the next 16 tiles' are on their way.
  const int32_t* const row_of_table = a.table + int64_t(seq) * a.ldt;
  const __amdgpu_buffer_rsrc_t of_table = view(row_of_table, ((end + a.page_size - 1) >> a.page_log2) * 4);  // (reads behind it give 0)
  auto pages_from = [&](int t) {
    const int key = (t + lane / 4) * kTileKeys + (lane & 3) * kBlock;
    return int32_t(__builtin_amdgcn_raw_buffer_load_b32(of_table, (key >> a.page_log2) * 4, 0, 0));
  };
  auto missing = [&](int pg) { return __ballot(pg < 0 || pg >= a.n_pages); };
  int32_t pages = pages_from(t_lo), pages_next = pages_from(t_lo + 16);
  // (the queries behind them: the first tile is requested before these are there)
  bf16x8 qf[QB][KS];
  int sees[QB];
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    const int rr = w0 + qb * 16 + lq, at = min(rr, rows - 1), i = token_of(at - row0), j = j0 + at - i * G;
    sees[qb] = rr < rows ? len - n + i + 1 : 0;  // (rows behind the last: its queries, which see nothing)
    const uint16_t* const q = a.Q + int64_t(start + i) * a.ldq + int64_t(j) * D + lh * 8;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[qb][ks] = *reinterpret_cast<const bf16x8*>(q + ks * 32);
  }
  f32x4 acc[QB][DB];
  float m_run[QB], l_run[QB];
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
#pragma unroll
    for (int db = 0; db < DB; ++db) acc[qb][db] = f32x4{0.f, 0.f, 0.f, 0.f};
    m_run[qb] = -INFINITY, l_run[qb] = 0.f;
  }

  arrived(pages);
  uint64_t bad = missing(pages), bad_now = bad;  // (bad_now: of the tiles that are multiplied, which follow those that are requested)

  // this wavefront's block of tile t: where it is, and how many of its tokens count
  auto place = [&](int t, int& valid, int64_t& page, int64_t& in) {
    const int key = t * kTileKeys + wave * kBlock;
    const int pg = __builtin_amdgcn_readlane(pages, (((t - t_lo) & 15) << 2) + wave);
    const bool there = pg >= 0 && pg < a.n_pages;
    valid = uniform(there ? min(max(end - key, 0), kBlock) : 0);
    page = there ? pg : 0;
    in = there ? int64_t(g) * a.page_size + (key & (a.page_size - 1)) : 0;
  };
  auto turn_pages = [&](int t) {  // before tile t is requested
    if (((t - t_lo) & 15) == 0 && t > t_lo) {
      pages = pages_next;
      arrived(pages);
      bad = missing(pages);
      pages_next = pages_from(t + 16);
    }
  };
  unsigned char* const sK = lds;
  unsigned char* const sV = lds + 2 * TILE;
  uint32_t voff[NI];
#pragma unroll
  for (int j = 0; j < NI; ++j) {
    const int p = j * 64 + lane, row = p / (D / 8), slot = p % (D / 8);
    voff[j] = uint32_t(row * D * 2) + ((uint32_t(slot) ^ tile_swz<D>(row)) * 16u);
  }
  auto request = [&](int t, int buf) {  // bf16: by DMA
    int valid;
    int64_t page, in;
    place(t, valid, page, in);
    const int64_t at = (page * a.page_stride + in * D) * 2;
    const __amdgpu_buffer_rsrc_t rk = view(a.K + at, valid * D * 2), rv = view(a.V + at, valid * D * 2);
#pragma unroll
    for (int j = 0; j < NI; ++j) {
      dma_16_shared(rk, sK + buf * TILE + wave * BLOCK + j * 1024, voff[j]);
      dma_16_shared(rv, sV + buf * TILE + wave * BLOCK + j * 1024, voff[j]);
    }
  };
  u32x4 k8[NL], v8[NL];  // 8 bits: 16 elements of a token, and its powers of two
  uint32_t ke[NL], ve[NL];
  auto fetch = [&](int t) {
    int valid;
    int64_t page, in;
    place(t, valid, page, in);
    const int64_t at = page * a.page_stride + in * D, ex = page * a.exp_stride + in;
    const __amdgpu_buffer_rsrc_t rk = view(a.K + at, valid * D), rv = view(a.V + at, valid * D), rke = view(a.K_exp + ex, valid), rve = view(a.V_exp + ex, valid);
#pragma unroll
    for (int j = 0; j < NL; ++j) {
      const int p = j * 64 + lane, row = p / (D / 16);
      k8[j] = __builtin_amdgcn_raw_buffer_load_b128(rk, p * 16, 0, 0);
      v8[j] = __builtin_amdgcn_raw_buffer_load_b128(rv, p * 16, 0, 0);
      ke[j] = __builtin_amdgcn_raw_buffer_load_b8(rke, row, 0, 0);
      ve[j] = __builtin_amdgcn_raw_buffer_load_b8(rve, row, 0, 0);
    }
  };
  auto convert = [&](int buf) {
#pragma unroll
    for (int j = 0; j < NL; ++j) {
      const int p = j * 64 + lane, row = p / (D / 16), c = p % (D / 16);
      const uint32_t to = uint32_t(buf * TILE + wave * BLOCK + row * D * 2) + ((uint32_t(2 * c) ^ tile_swz<D>(row)) * 16u);
      const float pk = power_of(ke[j]), pv = power_of(ve[j]);
      bf16x8* const dk = reinterpret_cast<bf16x8*>(sK + to);
      bf16x8* const dv = reinterpret_cast<bf16x8*>(sV + to);
      dk[0] = from_e4m3(u32x2{k8[j][0], k8[j][1]}, pk);
      dk[1] = from_e4m3(u32x2{k8[j][2], k8[j][3]}, pk);
      dv[0] = from_e4m3(u32x2{v8[j][0], v8[j][1]}, pv);
      dv[1] = from_e4m3(u32x2{v8[j][2], v8[j][3]}, pv);
    }
  };

  uint32_t ak[KS], av[DB];
  {
    const uint32_t kbase = uint32_t(reinterpret_cast<uintptr_t>(sK)) + uint32_t(lq * D * 2), xk = tile_swz<D>(lq);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) ak[ks] = kbase + ((uint32_t(ks * 4 + lh) ^ xk) * 16u);
    const int rv = lh * 4 + (lq >> 2);
    const uint32_t vbase = uint32_t(reinterpret_cast<uintptr_t>(sV)) + uint32_t(rv * D * 2) + uint32_t(lq & 1) * 8u, xv = tile_swz<D>(rv);
#pragma unroll
    for (int db = 0; db < DB; ++db) av[db] = vbase + ((uint32_t(db * 2 + ((lq & 3) >> 1)) ^ xv) * 16u);
  }

  // Two wavefronts share a SIMD, and would go through their matrix instructions, and then their softmax, together.  With a priority for each phase, the highest for the last product, one comes
  // before the other and the other one's vector work falls under its matrix instructions (one sequence of 8192 tokens, 14 heads: 251 us with one priority for both products -> 235; 512
  // tokens behind 130560, 16 heads: 514 -> 487).  8-bit pages: what turns the next tile to bf16 waits for the softmax too (512 tokens behind 130560: 558 -> 540, so 520; bf16 of 64 columns,
  // which has none of it: 164 -> 172, so not there).
  constexpr int FIRST = FP8 ? 2 : 1, SOFTMAX = FP8 ? 1 : 0, SECOND = 3;
  // one key tile out of buffer BUF (a compile-time constant, so that every LDS offset is an immediate)
  auto tile_step = [&](auto bufc, int t) {
    constexpr int BUF = decltype(bufc)::value;
    constexpr int BO = BUF * TILE;
    if constexpr (!FP8) dma_left<0>();  // this wavefront's share of tile t has landed ...
    __syncthreads();                    // ... and everyone's; everyone has finished reading tile t - 1 in the other buffer
    if (((t - t_lo) & 15) == 0) bad_now = bad;
    if (t + 1 < t_hi) {
      if constexpr (FP8) {
        convert(BUF ^ 1);
        if (t + 2 < t_hi) {
          turn_pages(t + 2);
          fetch(t + 2);
        }
      } else {
        turn_pages(t + 1);
        request(t + 1, BUF ^ 1);
      }
    }
    const int kv0 = t * kTileKeys;
    if (kv0 >= most) return;  // every token of the tile lies behind what this wavefront's last row sees
    // scores, transposed: st[kb][qb][r] = score of row qb * 16 + lane % 16 with token kv0 + kb * 16 + lane / 16 * 4 + r; eight key fragments at a time, the next ones read under
    // the matrix instructions of the ones before
    constexpr int KG = KS / 2, PER = 4 / KG;  // groups of reads, blocks of 16 tokens in one
    u32x4 kf[KG][8];
    auto k_reads = [&](auto grp) {
      unrolled(std::make_integer_sequence<int, 8>{}, [&](auto c) {
        constexpr int q = decltype(grp)::value, kb = q * PER + decltype(c)::value / KS, ks = decltype(c)::value % KS;
        kf[q][decltype(c)::value] = lds_b128<BO + kb * BLOCK>(ak[ks]);
      });
    };
    f32x4 st[4][QB];
    auto k_products = [&](auto grp) {
      constexpr int q = decltype(grp)::value;
      // (a product of every block in turn: none waits for the one before)
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
#pragma unroll
        for (int k = 0; k < PER; ++k)
#pragma unroll
          for (int qb = 0; qb < QB; ++qb)
            st[q * PER + k][qb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kf[q][k * KS + ks]), qf[qb][ks],
                                                                          ks == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : st[q * PER + k][qb], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    // value fragments, eight reads (two 16-column blocks) a group: [group][(db % 2) * 4 + kb], tokens kb * 16 ..
    constexpr int VG = DB / 2;
    u32x2 vf[VG][8];
    auto v_reads = [&](auto grp) {
      unrolled(std::make_integer_sequence<int, 8>{}, [&](auto c) {
        constexpr int q = decltype(grp)::value, db = q * 2 + decltype(c)::value / 4, kb = decltype(c)::value % 4;
        vf[q][decltype(c)::value] = lds_tr_b64<BO + kb * BLOCK>(av[db]);
      });
    };
    using I0 = std::integral_constant<int, 0>;
    using I1 = std::integral_constant<int, 1>;
    k_reads(I0{});
    lds_reads_done(kf[0]);
    __builtin_amdgcn_s_setprio(FIRST);
    if constexpr (KG == 2) {
      k_reads(I1{});
      k_products(I0{});
      lds_reads_done(kf[1]);
    }
    v_reads(I0{});
    v_reads(I1{});
    k_products(std::integral_constant<int, KG - 1>{});
    __builtin_amdgcn_s_setprio(SOFTMAX);

    const uint32_t gone = uint32_t(bad_now >> (((t - t_lo) & 15) << 2)) & 15u;  // blocks whose pages there are not
    const bool edge = kv0 + kTileKeys > all_see || w0 + 16 * QB > rows;
    if (gone != 0) {
#pragma unroll
      for (int kb = 0; kb < 4; ++kb)
        if ((gone >> kb) & 1u) {
#pragma unroll
          for (int qb = 0; qb < QB; ++qb) st[kb][qb] = f32x4{-INFINITY, -INFINITY, -INFINITY, -INFINITY};
        }
    }
    bf16x8 pf[QB][2];
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
      if (edge) {
        const int room = sees[qb] - kv0 - lh * 4;
#pragma unroll
        for (int kb = 0; kb < 4; ++kb)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (kb * 16 + r >= room) st[kb][qb][r] = -INFINITY;
      }
      float mx = -INFINITY;
#pragma unroll
      for (int kb = 0; kb < 4; ++kb)
#pragma unroll
        for (int r = 0; r < 4; ++r) mx = fmaxf(mx, st[kb][qb][r]);
      mx = over_rows(mx, larger) * a.scale_log2;
      // The reference that weights are relative to moves only where a score passes it by a factor of 2^8: a row's maximum moves with most of its first tiles, and each time all
      // of its outputs would be scaled (57 vector instructions a block; prompts of up to 2048 tokens 106 -> 100 us).  Weights of up to 2^8 are as exact as those of up to 1.
      const bool moves = mx > m_run[qb] + 8.0f;
      if (__any(moves)) {
        const float m_new = moves ? mx : m_run[qb];
        const float alpha = m_new == -INFINITY ? 1.0f : fast_exp2(m_run[qb] - m_new);
        l_run[qb] *= alpha;
        m_run[qb] = m_new;
#pragma unroll
        for (int db = 0; db < DB; ++db) acc[qb][db] *= alpha;
      }
      const float m_use = m_run[qb] == -INFINITY ? 0.f : m_run[qb];  // (no score above -inf so far: weights of 0)
      float ls = 0.f;
      float pr[4][4];
#pragma unroll
      for (int kb = 0; kb < 4; ++kb)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          pr[kb][r] = fast_exp2(fmaf(st[kb][qb][r], a.scale_log2, -m_use));
          ls += pr[kb][r];
        }
      l_run[qb] += ls;
      // weights as bf16: half a step of 2^-8 each, of a mean of values that is rounded to the same (errors against 64 bits 0.0017 to 0.0023, of fp32 weights 0.0015 to 0.0017); what that leaves in a
      // product of its own, as for few rows, would be half as many matrix instructions again on the pipe that bounds this
#pragma unroll
      for (int s2 = 0; s2 < 2; ++s2)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          pf[qb][s2][r] = static_cast<__bf16>(pr[2 * s2][r]);
          pf[qb][s2][4 + r] = static_cast<__bf16>(pr[2 * s2 + 1][r]);
        }
    }
    // O^T += V^T P^T (token slots of a 32-token step in the order the scores sit in the registers); every group of reads lands under the matrix instructions of the group before it
    auto v_products = [&](auto grp) {
      constexpr int q = decltype(grp)::value;
#pragma unroll
      for (int s2 = 0; s2 < 2; ++s2) {
#pragma unroll
        for (int d2 = 0; d2 < 2; ++d2) {
          const u32x2 lo = vf[q][d2 * 4 + s2 * 2], hi = vf[q][d2 * 4 + s2 * 2 + 1];
          const u32x4 both = {lo[0], lo[1], hi[0], hi[1]};
#pragma unroll
          for (int qb = 0; qb < QB; ++qb)
            acc[qb][q * 2 + d2] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, both), pf[qb][s2], acc[qb][q * 2 + d2], 0, 0, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    lds_reads_done(vf[0]);
    lds_reads_tied(vf[1]);
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_setprio(SECOND);
    if constexpr (VG == 4) {
      using I2 = std::integral_constant<int, 2>;
      using I3 = std::integral_constant<int, 3>;
      v_reads(I2{});
      v_products(I0{});
      v_reads(I3{});
      v_products(I1{});
      lds_reads_left<8>(vf[2]);
      v_products(I2{});
      lds_reads_done(vf[3]);
      v_products(I3{});
    } else {
      v_products(I0{});
      v_products(I1{});
    }
    __builtin_amdgcn_s_setprio(0);
  };

  if (t_lo < t_hi) {
    if constexpr (FP8) {
      fetch(t_lo);
      convert(0);
      if (t_lo + 1 < t_hi) fetch(t_lo + 1);
    } else {
      request(t_lo, 0);
    }
  }
#pragma unroll
  for (int qb = 0; qb < QB; ++qb)
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) arrived(qf[qb][ks]);
  for (int t = t_lo; t < t_hi; t += 2) {
    tile_step(std::integral_constant<int, 0>{}, t);
    if (t + 1 < t_hi) tile_step(std::integral_constant<int, 1>{}, t + 1);
  }

#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    const int rr = w0 + qb * 16 + lq, i = token_of(rr - row0), j = j0 + rr - i * G;
    const float l = over_rows(l_run[qb], added);
    if (n_pieces > 1) {
      float* const to = a.tile_parts + (int64_t(id) * kTileRows + (rr - row0)) * (D + kPartPad);
#pragma unroll
      for (int db = 0; db < DB; ++db) *reinterpret_cast<f32x4*>(to + db * 16 + lh * 4) = acc[qb][db];
      if (lh == 0) to[D] = m_run[qb], to[D + 1] = l;
      continue;
    }
    // through the LDS, so that whole rows are stored: 16-byte chunk c of the wavefront's row r at slot c ^ swz(r)
    const float inv = l == 0.f ? 0.f : 1.0f / l;
    if (qb == 0) __syncthreads();  // the last tile has been read
    int l16 = lane;
    arrived(l16);
    const int q16 = l16 & 15, h4 = l16 >> 4;
    unsigned char* const to = lds + (wave * 32 + qb * 16 + q16) * D * 2 + (h4 & 1) * 8;
#pragma unroll
    for (int db = 0; db < DB; ++db) {
      ntp_gemm::u16x4 o;
#pragma unroll
      for (int r = 0; r < 4; ++r) o[r] = ntp_gemm::f32_to_bf16(acc[qb][db][r] * inv);
      *reinterpret_cast<ntp_gemm::u16x4*>(to + ((uint32_t(db * 2 + (h4 >> 1)) ^ tile_swz<D>(q16)) * 16u)) = o;
    }
    if (rr < rows && lh == 0 && a.LSE) a.LSE[int64_t(j) * a.M + start + i] = ((l == 0.f ? 0.f : m_run[qb]) + log2f(l)) * 0.6931471805599453f;
  }
  if (n_pieces > 1) return;
  constexpr int CH = D / 8, PER = 64 / CH;  // chunks of a row, rows of a store
  int l64 = threadIdx.x & 63;
  arrived(l64);  // (what follows from it is not worth registers through the walk)
#pragma unroll
  for (int k = 0; k < 32 / PER; ++k) {
    const int r = k * PER + l64 / CH, c = l64 % CH, rr = w0 + r, i = token_of(rr - row0), j = j0 + rr - i * G;
    if (rr < rows)
      *reinterpret_cast<u32x4*>(a.C + int64_t(start + i) * a.ldc + int64_t(j) * D + c * 8) =
          *reinterpret_cast<const u32x4*>(lds + (wave * 32 + r) * D * 2 + ((uint32_t(c) ^ tile_swz<D>(r & 15)) * 16u));
  }
}

// The pieces of row tiles put together: workgroup number wg of n takes every n-th of (unit, some of its rows).  D / 8 lanes a row, eight pieces' loads at a time; where there are
// more pieces, several groups of lanes take a row's pieces in turn.
template <int D>
__device__ __forceinline__ void chunk_tiles_join(const ChunkArgs& a, const int wg, const int n_wgs) {
  constexpr int L = D / 8, G = kThreads / L, W = D + kPartPad, AT_ONCE = 8;  // lanes of a row, groups of lanes, floats of a partial row
  __shared__ f32x4 rows_of[G][L][2];
  __shared__ float2 sums_of[G];
  TilePlan plan;
  plan.units = a.plan[0], plan.total = a.plan[1], plan.piece_tiles = a.plan[2];
  // (Numbers that something else wrote there, a call on another stream with the same workspace, must not lead out of it: this and the test of the last piece's place.)
  if (plan.total == plan.units || plan.units < 0 || plan.units >= 2 * a.slots) return;
  plan.load(a, threadIdx.x & 63);
  const int grp = threadIdx.x / L, c = int(threadIdx.x) % L * 8;
  int ways = 1;  // groups of lanes of a row
  while (ways < G && plan.total > ways * AT_ONCE * plan.units) ways *= 2;
  const int per_unit = kTileRows / (G / ways), way = grp % ways;
  for (int job = wg; job < plan.units * per_unit; job += n_wgs) {
    const int first = plan.find_unit(a, job / per_unit), np = plan.n_pieces;
    if (first < 0 || np <= 1 || first + int64_t(np - 1) * plan.tiles_there >= 2 * a.slots) continue;
    const Heads hd(a, a.kv_first + plan.head);
    const int heads = hd.j1 - hd.j0, in_tile = job % per_unit * (G / ways) + grp / ways, rr = plan.tile * kTileRows + in_tile;
    const bool there = rr < min(plan.seq_n, a.max_new) * heads;
    const float* const p0 = a.tile_parts + (int64_t(first) * kTileRows + in_tile) * W;
    const int64_t next = int64_t(plan.tiles_there) * kTileRows * W;
    float top = -INFINITY, sum = 0.f;
    f32x4 lo = {0.f, 0.f, 0.f, 0.f}, hi = lo;
    for (int p = way; there && p < np; p += ways * AT_ONCE) {
      float m[AT_ONCE], l[AT_ONCE];
      f32x4 x[AT_ONCE], y[AT_ONCE];
#pragma unroll
      for (int k = 0; k < AT_ONCE; ++k) {
        m[k] = -INFINITY, l[k] = 0.f, x[k] = y[k] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (p + k * ways < np) {
          const float* const q = p0 + (p + k * ways) * next;
          m[k] = q[D], l[k] = q[D + 1], x[k] = *reinterpret_cast<const f32x4*>(q + c), y[k] = *reinterpret_cast<const f32x4*>(q + c + 4);
        }
      }
      float more = top;
#pragma unroll
      for (int k = 0; k < AT_ONCE; ++k) more = fmaxf(more, m[k]);
      const float base = more == -INFINITY ? 0.f : more, old = fast_exp2(top - base);
      sum *= old, lo *= old, hi *= old, top = more;
#pragma unroll
      for (int k = 0; k < AT_ONCE; ++k) {
        const float w = fast_exp2(m[k] - base);
        sum = fmaf(w, l[k], sum), lo += w * x[k], hi += w * y[k];
      }
    }
    if (ways > 1) {  // (the same in the whole workgroup)
      rows_of[grp][c / 8][0] = lo, rows_of[grp][c / 8][1] = hi;
      if (c == 0) sums_of[grp] = float2{top, sum};
      __syncthreads();
      if (way == 0) {
        for (int k = 1; k < ways; ++k) top = fmaxf(top, sums_of[grp + k].x);
        const float base = top == -INFINITY ? 0.f : top;
        sum = 0.f, lo = hi = f32x4{0.f, 0.f, 0.f, 0.f};
        for (int k = 0; k < ways; ++k) {
          const float w = fast_exp2(sums_of[grp + k].x - base);
          sum = fmaf(w, sums_of[grp + k].y, sum), lo += w * rows_of[grp + k][c / 8][0], hi += w * rows_of[grp + k][c / 8][1];
        }
      }
      __syncthreads();
      if (way > 0) continue;
    }
    if (!there) continue;
    const float inv = sum == 0.f ? 0.f : 1.0f / sum;
    u32x4 out;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      out[k] = uint32_t(ntp_gemm::f32_to_bf16(lo[2 * k] * inv)) | uint32_t(ntp_gemm::f32_to_bf16(lo[2 * k + 1] * inv)) << 16;
      out[2 + k] = uint32_t(ntp_gemm::f32_to_bf16(hi[2 * k] * inv)) | uint32_t(ntp_gemm::f32_to_bf16(hi[2 * k + 1] * inv)) << 16;
    }
    const int i = rr / heads, j = hd.j0 + rr - i * heads;
    *reinterpret_cast<u32x4*>(a.C + int64_t(plan.seq_start + i) * a.ldc + int64_t(j) * D + c) = out;
    if (c == 0 && a.LSE) a.LSE[int64_t(j) * a.M + plan.seq_start + i] = ((top == -INFINITY ? 0.f : top) + log2f(sum)) * 0.6931471805599453f;
  }
}

}  // namespace ntp_chunk

#endif  // NTP_ATTN_CHUNK_TILES_H_
