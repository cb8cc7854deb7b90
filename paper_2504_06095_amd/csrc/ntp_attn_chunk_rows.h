// Chunk attention, sequences of few rows (tokens x query heads of a KV head: up to 16 or 32): every key and value is read once for all of them, HBM bounds it (one new token of 64
// sequences of up to 8192, 14 heads, 8 bits: 163 us and 5 in the join, 6.1 TB/s; four tokens of 32 sequences of up to 4100, 8 heads on one: 14 and 4, latency).
//
// A unit is a sequence and KV head; its rows (token i, head h: number i G + h) are the columns of the matrix instruction, as in ntp_attn_decode.hip: both products run on the
// 16x16x32 bf16 instruction with the row on the lane axis (S^T = K Q^T, O^T += V^T P^T), one or two blocks of 16 rows a wavefront.  The units' steps form a line, which is cut into equal shares, two workgroups per
// compute unit, from the lengths on the device; units that are cut are joined by a second kernel.  A wavefront has tiles of its own (8 KB of keys, 8 KB of values) that come by
// DMA, so that nothing but a unit's end needs a barrier.  8-bit pages: twice the tokens a tile; the token's power of two goes into the key's conversion to bf16
// (exact) and, for values, into the weight.
#ifndef NTP_ATTN_CHUNK_ROWS_H_
#define NTP_ATTN_CHUNK_ROWS_H_

#include "ntp_attn_chunk.h"

namespace ntp_chunk {

constexpr int kRowTileBytes = 8192;  // of keys, and of values, per wavefront's tile, at most

template <int D, bool FP8, int QB>
struct RowFormat {
  static constexpr int ROWB = FP8 ? D : 2 * D, CHUNKS = ROWB / 16;  // bytes and 16-byte chunks of a token
  // tokens and blocks of a tile; with two blocks of rows an 8-bit tile is half as long, or the registers of its scores, weights and converted fragments run out
  static constexpr int T = kRowTileBytes / ROWB / (FP8 && QB == 2 ? 2 : 1), NB = T / kBlock;
  static constexpr int BLOCK = kBlock * ROWB, DMA = BLOCK / 1024;   // bytes and DMA instructions of a block
  static constexpr int STEP = kWaves * T;                           // tokens of a step
  // Chunk c of row r of a block sits at slot c ^ swz, so that the rows that a read touches per cycle lie on distinct banks: 16 rows' fragments of 16 (8-bit: 8) bytes of keys;
  // 8 rows of 32 bytes, or of 8-bit values 8 rows of 16 bytes of this block and as many of the next (p: the block's number is odd).
  __device__ static __forceinline__ uint32_t swz_k(int r) {
    if constexpr (FP8) return D == 128 ? uint32_t((r >> 1) & 7) : uint32_t((r >> 2) & 3);
    else return D == 128 ? uint32_t((r & 7) << 1) : uint32_t(((r >> 1) & 3) << 1);
  }
  __device__ static __forceinline__ uint32_t swz_v(int r, int p) {
    if constexpr (FP8) return D == 128 ? uint32_t(((r >> 1) & 3) | (p << 2)) : uint32_t(((r >> 2) & 1) | (p << 1));
    else return swz_k(r);
  }
};

// Steps of a sequence's unit: none where it is not of few rows, else at least one, which writes zeros where nothing is seen.
template <int STEP>
__device__ __forceinline__ int row_steps(const ChunkArgs& a, int n, int len) {
  const int used = min(n, a.max_new);
  if (used == 0 || used > a.cap / a.gmax) return 0;
  return max(1, (max(len - n + used, 0) + STEP - 1) / STEP);
}

// The line of steps: 64 sequences at a time in the lanes of a wavefront (every wavefront for itself).
template <int STEP>
struct RowLine {
  int start, n, len, mine, upto;  // of this lane's sequence base + lane: rows, tokens, a unit's steps, and those of the sequences up to and with it
  int base, before;               // the first of the 64, and the steps of a unit of the sequences before it
  int per_seq, total;             // units of a sequence; steps of the line
  int shares, q, r;               // share w has q steps, the first r shares one more
  __device__ __forceinline__ void load(const ChunkArgs& a, int from) {
    const int i = from + int(threadIdx.x & 63);
    base = from;
    extent(a, i, start, n, len);
    mine = row_steps<STEP>(a, n, len);
    upto = sum_upto(mine);
  }
  __device__ __forceinline__ int last() const { return __builtin_amdgcn_readlane(upto, 63); }
  static constexpr int kAtOnce = 256;  // sequences whose loads go out together
  __device__ __forceinline__ static int all_steps(const ChunkArgs& a, int from) {
    int sum = 0;
#pragma unroll
    for (int k = 0; k < kAtOnce / 64; ++k) {
      const int i = from + k * 64 + int(threadIdx.x & 63);
      int s, n, len;
      extent(a, i, s, n, len);
      sum += row_steps<STEP>(a, n, len);
    }
    return __builtin_amdgcn_readlane(sum_upto(sum), 63);
  }
  // the whole line, and how it is cut; the first 64 sequences
  __device__ __forceinline__ void measure(const ChunkArgs& a) {
    before = 0;
    per_seq = a.kv_used;
    load(a, 0);
    int steps = last();
    if (a.n_seq > 64) {
      steps = 0;
      for (int from = 0; from < a.n_seq; from += kAtOnce) steps += all_steps(a, from);
    }
    total = steps * per_seq;
    shares = max(min(a.shares, max(total / 2, min(total, a.shares / 2))), 1);  // (of one step only where compute units would be left over)
    q = total / shares;
    r = total % shares;
  }
  // from the first 64 sequences to the one with step x < total of the line, and its unit and the number in it
  __device__ __forceinline__ void seek(const ChunkArgs& a, int x, int& seq, int& unit, int& step) {
    int from = 0;
    while (from < a.n_seq - kAtOnce) {
      const int steps = all_steps(a, from);
      if ((before + steps) * per_seq > x) break;
      before += steps;
      from += kAtOnce;
    }
    if (from > 0) load(a, from);
    uint64_t behind;
    while ((behind = __ballot((before + upto) * per_seq > x)) == 0) next64(a);
    const int at = __builtin_ctzll(behind);
    seq = base + at;
    const int steps = __builtin_amdgcn_readlane(mine, at), rest = x - (before + __builtin_amdgcn_readlane(upto, at) - steps) * per_seq;
    unit = rest / steps;
    step = rest % steps;
  }
  __device__ __forceinline__ int begin(int w) const { return w * q + min(w, r); }
  __device__ __forceinline__ int share_of(int x) const { return x < r * (q + 1) ? x / (q + 1) : r + (x - r * (q + 1)) / q; }
  __device__ __forceinline__ void next64(const ChunkArgs& a) {
    before += last();
    load(a, base + 64);
  }
  // the next sequence with steps; there is one
  __device__ __forceinline__ int next(const ChunkArgs& a, int seq) {
    uint64_t more = __ballot(mine > 0 && base + int(threadIdx.x & 63) > seq);
    while (more == 0) {
      next64(a);
      more = __ballot(mine > 0);
    }
    return base + __builtin_ctzll(more);
  }
  __device__ __forceinline__ int of(int v, int seq) const { return __builtin_amdgcn_readlane(v, seq - base); }
};

template <int D, int QB>
constexpr int kRowLds = kWaves * (2 * kRowTileBytes > 16 * QB * (D + 4) * 4 ? 2 * kRowTileBytes : 16 * QB * (D + 4) * 4);

template <int D, bool FP8, int QB>
__device__ __forceinline__ void chunk_rows(const ChunkArgs& a, const int wg, unsigned char* const lds) {
  using F = RowFormat<D, FP8, QB>;
  constexpr int KS = D / 32, DB = D / 16;  // K-steps of the score product, 16-column blocks of the output
  constexpr int T = F::T, NB = F::NB, STEP = F::STEP, ROW = D + 4, R = 16 * QB;
  constexpr int KR = NB * KS, VR = FP8 ? DB * NB / 2 : DB * NB;  // LDS reads of a tile
  using KFrag = std::conditional_t<FP8, u32x2, u32x4>;
  const int lane = threadIdx.x & 63, lq = lane & 15, lh = lane >> 4;
  const int wave = uniform(threadIdx.x >> 6);
  unsigned char* const sK = lds + wave * 2 * kRowTileBytes;
  unsigned char* const sV = sK + kRowTileBytes;
  const uint32_t lK = uint32_t(reinterpret_cast<uintptr_t>(sK)), lV = lK + kRowTileBytes;

  // lane offsets: DMA of a block's chunks (8-bit values: of an even and of an odd block), key fragments (row lane % 16, columns lane / 16 * 8 on), transposing reads
  constexpr int PV = FP8 ? 2 : 1;
  uint32_t koff[F::DMA], voff[PV][F::DMA], row[KS], col[DB];
#pragma unroll
  for (int i = 0; i < F::DMA; ++i) {
    const int p = i * 64 + lane, rw = p / F::CHUNKS, slot = p % F::CHUNKS;
    koff[i] = uint32_t(rw * F::ROWB) + ((uint32_t(slot) ^ F::swz_k(rw)) * 16u);
#pragma unroll
    for (int o = 0; o < PV; ++o) voff[o][i] = uint32_t(rw * F::ROWB) + ((uint32_t(slot) ^ F::swz_v(rw, o)) * 16u);
  }
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) {
    if constexpr (FP8) row[ks] = lK + uint32_t(lq * F::ROWB) + ((uint32_t(ks * 2 + (lh >> 1)) ^ F::swz_k(lq)) * 16u) + uint32_t(lh & 1) * 8u;
    else row[ks] = lK + uint32_t(lq * F::ROWB) + ((uint32_t(ks * 4 + lh) ^ F::swz_k(lq)) * 16u);
  }
#pragma unroll
  for (int db = 0; db < DB; ++db) {
    if constexpr (FP8) {  // eight rows: four of a block, the same four of the next
      const int p = lq >> 3, rv = lh * 4 + ((lq >> 1) & 3);
      col[db] = lV + uint32_t(p * F::BLOCK + rv * F::ROWB) + ((uint32_t(db) ^ F::swz_v(rv, p)) * 16u) + uint32_t(lq & 1) * 8u;
    } else {
      const int rv = lh * 4 + (lq >> 2);
      col[db] = lV + uint32_t(rv * F::ROWB) + uint32_t(lq & 1) * 8u + ((uint32_t(db * 2 + ((lq & 3) >> 1)) ^ F::swz_v(rv, 0)) * 16u);
    }
  }

  // this workgroup's steps x .. x_end - 1 of the line; x lies in unit `unit` of sequence seq, `step` steps behind the unit's first
  RowLine<STEP> line;
  line.per_seq = a.kv_used;
  int x, x_end, seq, unit, step;
  if (a.part_rows) {
    line.measure(a);
    if (wg >= line.shares || line.total == 0) return;
    x = line.begin(wg);
    x_end = line.begin(wg + 1);
    line.seek(a, x, seq, unit, step);
  } else {
    seq = wg / line.per_seq;
    unit = wg % line.per_seq;
    line.before = 0;
    line.load(a, seq & ~63);
    x = step = 0;
    x_end = line.of(line.mine, seq);
  }
  // (said to be the same in every lane: the buffer views below are made from them)
  x = uniform(x), x_end = uniform(x_end), seq = uniform(seq), unit = uniform(unit), step = uniform(step);
  for (bool first = true; x < x_end; first = false) {
  const int start = line.of(line.start, seq), n = line.of(line.n, seq), len = line.of(line.len, seq), steps = line.of(line.mine, seq);
  const int n_steps = min(steps - step, x_end - x), used = min(n, a.max_new);
  const int k_lo = step * STEP, k_hi = min(max(len - n + used, 0), k_lo + n_steps * STEP);
  const int g = a.kv_first + unit;
  const Heads hd(a, g);
  const int G = hd.j1 - hd.j0, rows = used * G;

  // rows qb * 16 + lane % 16: their queries (operand B[k][row], k = 8 consecutive columns), and how many tokens they see
  bf16x8 qf[QB][KS];
  int sees[QB];
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    const int rr = qb * 16 + lq, i = rr / G, j = hd.j0 + rr - i * G;
    sees[qb] = rr < rows ? len - n + i + 1 : 0;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[qb][ks] = bf16x8{};
    if (rr < rows) {
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) qf[qb][ks] = *reinterpret_cast<const bf16x8*>(a.Q + int64_t(start + i) * a.ldq + int64_t(j) * D + ks * 32 + lh * 8);
    }
  }
  const int all_see = len - n + 1;  // tokens that every row sees

  f32x4 acc[QB][DB];
  float m_run[QB], l_run[QB];
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
#pragma unroll
    for (int db = 0; db < DB; ++db) acc[qb][db] = f32x4{0.f, 0.f, 0.f, 0.f};
    m_run[qb] = -INFINITY, l_run[qb] = 0.f;
  }

  // Page numbers of 64 of the wavefront's blocks, one a lane: its tile number i is tile i * kWaves + wave of the share's tokens.
  constexpr int PER = 64 / NB;  // tiles per set of page numbers
  const int32_t* const row_of_table = a.table + int64_t(seq) * a.ldt;
  auto pages_from = [&](int i) {
    const int key = k_lo + ((i + lane / NB) * kWaves + wave) * T + (lane % NB) * kBlock;
    return key < k_hi ? row_of_table[key >> a.page_log2] : -1;
  };
  int32_t pages = pages_from(0);
#pragma unroll
  for (int qb = 0; qb < QB; ++qb)
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) arrived(qf[qb][ks]);
  arrived(pages);
  const int n_tiles = rows > 0 ? max(0, (k_hi - k_lo + T - 1) / T) : 0;
  const int mine = (n_tiles - wave + kWaves - 1) / kWaves;  // tiles of this wavefront
  // DMA of one matrix of tile i; number of tokens of each block that count
  auto place = [&](int i, int b, int& valid, int64_t& page, int64_t& in) {
    const int key = k_lo + (i * kWaves + wave) * T + b * kBlock;
    const int pg = __builtin_amdgcn_readlane(pages, (i % PER) * NB + b);
    const bool there = pg >= 0 && pg < a.n_pages;
    valid = uniform(there ? min(max(k_hi - key, 0), kBlock) : 0);
    page = there ? pg : 0;
    in = there ? int64_t(g) * a.page_size + (key & (a.page_size - 1)) : 0;
  };
  auto request = [&](const unsigned char* base, unsigned char* to, auto values, int i, int (&valid)[NB]) {
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      int64_t page, in;
      place(i, b, valid[b], page, in);
      const __amdgpu_buffer_rsrc_t rs = view(base + page * a.page_stride * (FP8 ? 1 : 2) + in * F::ROWB, valid[b] * F::ROWB);
#pragma unroll
      for (int j = 0; j < F::DMA; ++j) dma_16(rs, to + b * F::BLOCK + j * 1024, decltype(values)::value ? voff[PV == 2 ? b & 1 : 0][j] : koff[j]);
    }
  };
  // the tokens' powers of two: of key lane % 16 of each block, and of values lane / 16 * 4 .. + 3
  uint32_t ke[NB] = {}, ve[NB] = {};
  auto powers = [&](int i) {
    if constexpr (FP8) {
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        int valid;
        int64_t page, in;
        place(i, b, valid, page, in);
        ke[b] = ve[b] = 0;
        if (valid > 0) {
          const int64_t at = page * a.exp_stride + in;
          ke[b] = a.K_exp[at + lq];
          ve[b] = *reinterpret_cast<const uint32_t*>(a.V_exp + at + lh * 4);
        }
      }
    }
  };
  // One tile of keys and one of values in the LDS: the next keys are requested when this tile's have been read into registers, the next values
  // likewise, so that there is always one or the other in flight.
  constexpr int IN_FLIGHT = NB * F::DMA;
  int valid[NB], next[NB];
  if (mine > 0) {
    powers(0);
#pragma unroll
    for (int b = 0; b < NB; ++b) arrived(ke[b]), arrived(ve[b]);
    request(a.K, sK, std::false_type{}, 0, valid);
    request(a.V, sV, std::true_type{}, 0, valid);
  }
  auto tile = [&](int i, auto last) {
    constexpr bool MORE = !decltype(last)::value;
    float pk[NB], pv[NB][4];
    if constexpr (FP8) {
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        pk[b] = power_of(ke[b]);
#pragma unroll
        for (int r = 0; r < 4; ++r) pv[b][r] = power_of((ve[b] >> (8 * r)) & 0xffu);
      }
    }
    dma_left<IN_FLIGHT>();  // the keys are there
    KFrag kf[KR];
    unrolled(std::make_integer_sequence<int, KR>{}, [&](auto c) {
      constexpr int blk = decltype(c)::value / KS, ks = decltype(c)::value % KS;
      if constexpr (FP8) kf[decltype(c)::value] = lds_b64<blk * F::BLOCK>(row[ks]);
      else kf[decltype(c)::value] = lds_b128<blk * F::BLOCK>(row[ks]);
    });
    lds_reads_done(kf);
    if constexpr (MORE) {
      if ((i + 1) % PER == 0) {
        pages = pages_from(i + 1);
        arrived(pages);
      }
      powers(i + 1);
      request(a.K, sK, std::false_type{}, i + 1, next);
    }
    // scores, transposed: st[qb][b][r] = score of row qb * 16 + lane % 16 with token key0 + b * 16 + lane / 16 * 4 + r
    const int key0 = k_lo + (i * kWaves + wave) * T;
    f32x4 st[QB][NB];
    bool edge = key0 + T > all_see;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) st[qb][b] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        bf16x8 k8;
        if constexpr (FP8) k8 = from_e4m3(kf[b * KS + ks], pk[b]);
        else k8 = __builtin_bit_cast(bf16x8, kf[b * KS + ks]);
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) st[qb][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k8, qf[qb][ks], st[qb][b], 0, 0, 0);
      }
      edge = edge || valid[b] < kBlock;
    }
    if (edge) {
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int t = b * kBlock + lh * 4 + r;
          const bool there = lh * 4 + r < valid[b];
          if constexpr (FP8) pv[b][r] = there ? pv[b][r] : 0.f;  // (the byte behind the last token may be any)
#pragma unroll
          for (int qb = 0; qb < QB; ++qb)
            if (!there || key0 + t >= sees[qb]) st[qb][b][r] = -INFINITY;
        }
    }
    // weights as operand B of the second product, per 32 tokens: bf16, and what that leaves, rounded to bf16 too, in a product of its own (as ntp_attn_decode.hip): 2^-16 of a weight
    // is lost, whatever else is in the batch.  The matrix pipe has room for it: HBM and latency bound these walks (four tokens of 32 sequences, 8 heads on one: 17.8 -> 18.1 us with the rest)
    bf16x8 pf[QB][NB / 2], pr[QB][NB / 2];
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
      float mx = -INFINITY;
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int r = 0; r < 4; ++r) mx = fmaxf(mx, st[qb][b][r]);
      mx = over_rows(mx, larger) * a.scale_log2;
      const float m_new = fmaxf(m_run[qb], mx), m_use = m_new == -INFINITY ? 0.f : m_new;  // (no score above -inf so far: weights of 0)
      const float alpha = fast_exp2(m_run[qb] - m_use);
      float ls = 0.f;
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          float p = fast_exp2(fmaf(st[qb][b][r], a.scale_log2, -m_use));
          ls += p;
          if constexpr (FP8) p *= pv[b][r];
          const __bf16 top = static_cast<__bf16>(p);
          pf[qb][b / 2][(b & 1) * 4 + r] = top;
          pr[qb][b / 2][(b & 1) * 4 + r] = static_cast<__bf16>(p - static_cast<float>(top));
        }
      l_run[qb] = l_run[qb] * alpha + ls;  // of this lane's tokens; the four lane groups are added at the end
      m_run[qb] = m_new;
      if (__any(alpha != 1.0f)) {
#pragma unroll
        for (int db = 0; db < DB; ++db) acc[qb][db] *= alpha;
      }
    }
    dma_left<MORE ? IN_FLIGHT : 0>();  // the values are there
    u32x2 vf[VR];
    unrolled(std::make_integer_sequence<int, VR>{}, [&](auto c) {
      if constexpr (FP8) {  // [db * NB / 2 + s2]
        constexpr int db = decltype(c)::value / (NB / 2), s2 = decltype(c)::value % (NB / 2);
        vf[decltype(c)::value] = lds_tr8_b64<s2 * 2 * F::BLOCK>(col[db]);
      } else {  // [(db * NB / 2 + s2) * 2 + half]
        constexpr int db = decltype(c)::value / NB, q = decltype(c)::value % NB;
        vf[decltype(c)::value] = lds_tr_b64<q * F::BLOCK>(col[db]);
      }
    });
    lds_reads_done(vf);
    if constexpr (MORE) request(a.V, sV, std::true_type{}, i + 1, next);
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int s2 = 0; s2 < NB / 2; ++s2) {
        bf16x8 v8;
        if constexpr (FP8) {
          v8 = from_e4m3(vf[db * (NB / 2) + s2], 1.0f);
        } else {
          const u32x2 lo = vf[db * NB + s2 * 2], hi = vf[db * NB + s2 * 2 + 1];
          v8 = __builtin_bit_cast(bf16x8, u32x4{lo[0], lo[1], hi[0], hi[1]});
        }
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) {
          acc[qb][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v8, pf[qb][s2], acc[qb][db], 0, 0, 0);
          acc[qb][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v8, pr[qb][s2], acc[qb][db], 0, 0, 0);
        }
      }
    if constexpr (MORE) {
#pragma unroll
      for (int b = 0; b < NB; ++b) valid[b] = next[b];
    }
  };
  for (int i = 0; i + 1 < mine; ++i) tile(i, std::false_type{});
  if (mine > 0) tile(mine - 1, std::true_type{});

  // the wavefronts' results, one line per row
  __syncthreads();
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    const float l = over_rows(l_run[qb], added);
    float* const result = reinterpret_cast<float*>(lds) + (wave * R + qb * 16 + lq) * ROW;
#pragma unroll
    for (int db = 0; db < DB; ++db) *reinterpret_cast<f32x4*>(result + db * 16 + lh * 4) = acc[qb][db];
    if (lh == 0) {
      result[D] = m_run[qb];
      result[D + 1] = l;
    }
  }
  __syncthreads();
  const bool whole = n_steps == steps;
  const int64_t slot = (int64_t(wg) * 2 + !first) * R;
  const int c0 = (threadIdx.x & 15) * 4;
  for (int rr = threadIdx.x >> 4; rr < rows; rr += 16) {
    const float* const res = reinterpret_cast<const float*>(lds) + rr * ROW;
    const int i = rr / G, j = hd.j0 + rr - i * G;
    float top = -INFINITY, w[kWaves], sum = 0.f;
#pragma unroll
    for (int k = 0; k < kWaves; ++k) top = fmaxf(top, res[k * R * ROW + D]);
    const float base = top == -INFINITY ? 0.f : top;
#pragma unroll
    for (int k = 0; k < kWaves; ++k) {
      w[k] = fast_exp2(res[k * R * ROW + D] - base);
      sum = fmaf(w[k], res[k * R * ROW + D + 1], sum);
    }
    const float inv = sum == 0.f ? 0.f : 1.0f / sum;
#pragma unroll
    for (int c = c0; c < D; c += 64) {
      f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < kWaves; ++k) o += w[k] * *reinterpret_cast<const f32x4*>(res + k * R * ROW + c);
      if (!whole) {
        *reinterpret_cast<f32x4*>(a.part_rows + (slot + rr) * D + c) = o;
      } else {
        ntp_gemm::u16x4 out;
#pragma unroll
        for (int k = 0; k < 4; ++k) out[k] = ntp_gemm::f32_to_bf16(o[k] * inv);
        *reinterpret_cast<ntp_gemm::u16x4*>(a.C + int64_t(start + i) * a.ldc + int64_t(j) * D + c) = out;
      }
    }
    if (c0 == 0) {
      if (!whole) a.part_sums[slot + rr] = float2{top, sum};
      else if (a.LSE) a.LSE[int64_t(j) * a.M + start + i] = (base + log2f(sum)) * 0.6931471805599453f;
    }
  }
  x += n_steps;
  step = 0;
  if (++unit == line.per_seq) {
    unit = 0;
    if (x < x_end) seq = uniform(line.next(a, seq));
  }
  __syncthreads();  // the results have been read: the next unit's tiles may come
  }
}

// The partial results of a unit that does not lie in one share, put together.  Part p of it is what share w0 + p left: of the unit that it begins inside, but for a first share that
// begins before the unit.
struct CutUnit {
  int start, rows, G, j0, parts, w0, late;
  template <int STEP>
  __device__ __forceinline__ void set(const ChunkArgs& a, const RowLine<STEP>& line, int seq, int unit, int begin) {
    const int steps = line.of(line.mine, seq);
    const Heads hd(a, a.kv_first + unit);
    start = line.of(line.start, seq), G = hd.j1 - hd.j0, j0 = hd.j0, rows = min(line.of(line.n, seq), a.max_new) * G;
    w0 = line.share_of(begin);
    late = line.begin(w0) < begin;
    parts = line.share_of(begin + steps - 1) - w0 + 1;
  }
  // unit `number` of the batch (sequence by sequence, KV head by KV head); whether it is cut
  template <int STEP>
  __device__ __forceinline__ bool by_number(const ChunkArgs& a, int number) {
    RowLine<STEP> line;
    line.measure(a);
    const int seq = number / line.per_seq, unit = number % line.per_seq;
    while (seq >= line.base + 64) line.next64(a);
    const int steps = line.of(line.mine, seq);
    if (steps == 0) return false;
    set(a, line, seq, unit, (line.before + line.of(line.upto, seq) - steps) * line.per_seq + unit * steps);
    return parts > 1;
  }
  // the unit with the border between shares w - 1 and w in it, if that is the unit's first
  template <int STEP>
  __device__ __forceinline__ bool by_border(const ChunkArgs& a, int w) {
    RowLine<STEP> line;
    line.measure(a);
    if (w >= line.shares || line.total == 0) return false;
    const int x = line.begin(w);
    int seq, unit, step;
    line.seek(a, x, seq, unit, step);
    if (step == 0 || line.begin(w - 1) > x - step) return false;
    set(a, line, seq, unit, x - step);
    return true;
  }
  __device__ __forceinline__ int64_t slot(int p, int R) const { return (int64_t(w0 + p) * 2 + (p == 0 ? late : 0)) * R; }
};
__device__ __forceinline__ void store_row(const ChunkArgs& a, const CutUnit& u, int rr, int col, int D, f32x4 o, float base, float sum) {
  const int i = rr / u.G, j = u.j0 + rr - i * u.G;
  const float inv = sum == 0.f ? 0.f : 1.0f / sum;
  ntp_gemm::u16x4 out;
#pragma unroll
  for (int k = 0; k < 4; ++k) out[k] = ntp_gemm::f32_to_bf16(o[k] * inv);
  *reinterpret_cast<ntp_gemm::u16x4*>(a.C + int64_t(u.start + i) * a.ldc + int64_t(j) * D + col) = out;
  if (a.LSE && col == 0) a.LSE[int64_t(j) * a.M + u.start + i] = (base + log2f(sum)) * 0.6931471805599453f;
}

// Few units of many parts: workgroup = (unit, row, 32 of the columns); the threads form the parts' weights, then 8 lanes hold the outputs and 32 groups of them take the parts in turn.
constexpr int kFewColumns = 32;
template <int D, int STEP, int R>
__device__ __forceinline__ void chunk_rows_join_long(const ChunkArgs& a, const int number, const int rr, const int col0) {
  constexpr int L = kFewColumns / 4, GR = kThreads / L, N = kMaxShares / kThreads;
  __shared__ float weight[kMaxShares], wave_max[kWaves], wave_sum[kWaves];
  __shared__ f32x4 sums[GR][L];
  CutUnit u;
  if (!u.by_number<STEP>(a, number) || rr >= u.rows) return;
  const int grp = threadIdx.x / L, c = col0 + int(threadIdx.x) % L * 4;
  auto part_row = [&](int p) { return *reinterpret_cast<const f32x4*>(a.part_rows + (u.slot(p, R) + rr) * D + c); };
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  if (grp < u.parts) o = part_row(grp);  // (on its way while the weights are formed)
  float2 ms[N];
  float top = -INFINITY, sum = 0.f;
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const int p = int(threadIdx.x) + k * kThreads;
    ms[k] = p < u.parts ? a.part_sums[u.slot(p, R) + rr] : float2{-INFINITY, 0.f};
    top = fmaxf(top, ms[k].x);
  }
  auto wave_all = [](float v, auto f) {
#pragma unroll
    for (int d = 1; d < 16; d *= 2) v = f(v, __shfl_xor(v, d));
    return over_rows(v, f);
  };
  top = wave_all(top, larger);
  if ((threadIdx.x & 63) == 0) wave_max[threadIdx.x >> 6] = top;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kWaves; ++k) top = fmaxf(top, wave_max[k]);
  const float base = top == -INFINITY ? 0.f : top;
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const float wt = fast_exp2(ms[k].x - base);
    sum = fmaf(wt, ms[k].y, sum);
    weight[threadIdx.x + k * kThreads] = wt;
  }
  sum = wave_all(sum, added);
  if ((threadIdx.x & 63) == 0) wave_sum[threadIdx.x >> 6] = sum;
  __syncthreads();
  if (grp < u.parts) o *= weight[grp];
#pragma unroll 8
  for (int p = grp + GR; p < u.parts; p += GR) o += weight[p] * part_row(p);
  sums[grp][c / 4 % L] = o;
  __syncthreads();
  if (grp > 0) return;
  sum = wave_sum[0];
#pragma unroll
  for (int k = 1; k < kWaves; ++k) sum += wave_sum[k];
#pragma unroll
  for (int k = 1; k < GR; ++k) o += sums[k][c / 4 % L];
  store_row(a, u, rr, c, D, o, base, sum);
}

// Some rows of a unit of few parts, D / 4 lanes a row.
template <int D, int R>
__device__ __forceinline__ void chunk_rows_join_short(const ChunkArgs& a, const CutUnit& u, const int row0) {
  constexpr int L = D / 4;
  const int rr = row0 + int(threadIdx.x) / L, c = int(threadIdx.x) % L * 4;
  if (rr >= u.rows) return;
  constexpr int AT_ONCE = 16;  // parts whose loads go out together
  float top = -INFINITY, sum = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  for (int p = 0; p < u.parts; p += AT_ONCE) {
    float2 ms[AT_ONCE];
    f32x4 x[AT_ONCE];
#pragma unroll
    for (int k = 0; k < AT_ONCE; ++k) {
      ms[k] = float2{-INFINITY, 0.f}, x[k] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (p + k < u.parts) {
        const int64_t at = u.slot(p + k, R) + rr;
        ms[k] = a.part_sums[at];
        x[k] = *reinterpret_cast<const f32x4*>(a.part_rows + at * D + c);
      }
    }
    float more = top;
#pragma unroll
    for (int k = 0; k < AT_ONCE; ++k) more = fmaxf(more, ms[k].x);
    const float base = more == -INFINITY ? 0.f : more, old = fast_exp2(top - base);
    sum *= old, o *= old, top = more;
#pragma unroll
    for (int k = 0; k < AT_ONCE; ++k) {
      const float wt = fast_exp2(ms[k].x - base);
      sum = fmaf(wt, ms[k].y, sum), o += wt * x[k];
    }
  }
  store_row(a, u, rr, c, D, o, top == -INFINITY ? 0.f : top, sum);
}

}  // namespace ntp_chunk

#endif  // NTP_ATTN_CHUNK_ROWS_H_
