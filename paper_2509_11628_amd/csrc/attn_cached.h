// What the kernels of attention over 8-bit pages share: their arguments, how the work is dealt, and widening.
#pragma once

#include "attn_lane.h"
#include "deal.h"
#include "operators.h"

namespace speca {

constexpr int PAGE = SPECA_KV_PAGE;

// four e4m3 bytes x a power of two -> four bf16
__device__ inline void widen(uint32_t b, float scale, uint32_t* out) {
  const bf16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, false), hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, true);
  out[0] = *reinterpret_cast<const uint32_t*>(&lo);
  out[1] = *reinterpret_cast<const uint32_t*>(&hi);
}
// What the join needs to know of a sequence.
struct Share {                      // tiles of few rows
  int32_t splits, tiles;
  int64_t slot;                     // of its first unit; a sequence of one split has none
};
struct alignas(16) Stretch {        // tiles of 128 rows
  int64_t from, per;                // position of its first tile, positions of a block
  int32_t tiles, pages;
  int32_t splits;                   // of every tile, one position each; 0: as the borders of the blocks have it
};
struct CachedArgs {
  const uint8_t *k, *v;
  const float *k_scale, *v_scale;
  const uint16_t* q;
  uint16_t* out;
  int64_t ldq, ldo;
  Packed seqs;
  const int32_t *lens, *table;
  void* shares;                     // Share or Stretch of every sequence, for the join
  float *part, *stats;              // of splits, by slot: O [rows of a tile][HD], and maximum and sum [2][rows]
  int32_t table_ld, pages, kv_heads, group;
  int32_t max_len, resident, least_pages, slots;
  int32_t causal, wide;             // wide: queries at whole 16 bytes, outputs at whole 8
  float scale_log2e;
};

// How the work of few rows is dealt.  The host knows no lengths, so every wave works it out from the lists on the device, 64 sequences at a time.  A
// unit is one row tile of one key head over one split of its sequence's range of pages; ranges longer than split_pages, which deal.h chooses, are
// split evenly.
struct Deal {
  int tiles, pages;                 // of the lane's sequence in the first 64
  int64_t units;                    // of all
  int split_pages;
};
template <int ROWS>
__device__ inline void deal_sequence(const CachedArgs& g, int s, int* tiles, int* pages) {
  const int at = min(s, g.seqs.n - 1);        // (loads without a branch: those of several rounds go out together)
  int start, n;
  packed_rows(g.seqs, at, &start, &n);
  const int len = g.lens[at];
  *tiles = s < g.seqs.n ? static_cast<int>((static_cast<int64_t>(n) * g.group + ROWS - 1) / ROWS) : 0;
  *pages = s < g.seqs.n && len > 0 ? (min(len, g.max_len) + PAGE - 1) / PAGE : 0;
}
// a lane's value, in scalar registers: what follows from it is worked out once per wave
__device__ inline int64_t of_lane(int64_t x, int lane) {
  const uint32_t lo = __builtin_amdgcn_readlane(static_cast<int>(x), lane), hi = __builtin_amdgcn_readlane(static_cast<int>(x >> 32), lane);
  return static_cast<int64_t>(static_cast<uint64_t>(hi) << 32 | lo);
}
// over the lanes that have a sequence (the others hold 0): `lanes` of them
__device__ inline int64_t sum_of_wave(int64_t x, int lanes) {
  for (int off = 1; off < lanes && off < 64; off <<= 1) x += __shfl_xor(x, off, 64);
  return of_lane(x, 0);
}
__device__ inline int max_of_wave(int x, int lanes) {
  for (int off = 1; off < lanes && off < 64; off <<= 1) x = max(x, __shfl_xor(x, off, 64));
  return __builtin_amdgcn_readlane(x, 0);
}
template <int ROWS>
__device__ inline Deal deal(const CachedArgs& g) {
  const int lane = threadIdx.x & 63;
  Deal d;
  deal_sequence<ROWS>(g, lane, &d.tiles, &d.pages);
  int64_t work = static_cast<int64_t>(d.tiles) * d.pages, whole = d.tiles;
  int tiles, pages;
#pragma unroll 4
  for (int s0 = 64; s0 < g.seqs.n; s0 += 64) {
    deal_sequence<ROWS>(g, s0 + lane, &tiles, &pages);
    work += static_cast<int64_t>(tiles) * pages;
    whole += tiles;
  }
  work = sum_of_wave(work, g.seqs.n) * g.kv_heads;
  whole = sum_of_wave(whole, g.seqs.n) * g.kv_heads;
  auto count = [&](int split_pages, int64_t* units, int* longest) {
    int splits = splits_of(d.pages, split_pages), most = d.tiles ? (d.pages + splits - 1) / splits : 0;
    int64_t sum = static_cast<int64_t>(d.tiles) * splits;
#pragma unroll 4
    for (int s0 = 64; s0 < g.seqs.n; s0 += 64) {
      deal_sequence<ROWS>(g, s0 + lane, &tiles, &pages);
      splits = splits_of(pages, split_pages);
      sum += static_cast<int64_t>(tiles) * splits;
      if (tiles) most = max(most, (pages + splits - 1) / splits);
    }
    *units = sum_of_wave(sum, g.seqs.n) * g.kv_heads;
    if (longest) *longest = max_of_wave(most, g.seqs.n);
  };
  const Cut cut = cut_few_rows(work, whole, g.resident, g.least_pages, (g.max_len + PAGE - 1) / PAGE, count);
  d.split_pages = cut.split_pages;
  d.units = cut.units;
  return d;
}
// Sequence of unit u, u's number within it and the slot of its first unit.  (u rises through tiles first, then splits, then heads: blocks
// that run side by side read the same keys.)  With `shares` every sequence's are written down instead.
struct Found {
  int seq, tiles, splits, at;
  int each;                         // pages of a split
  int64_t slot;
};
// Unit of this block in a round of the grid, or -1.  Blocks b, b + 8, ... run on the same XCD: each XCD gets a run of the round's units,
// which share keys, and as many as the others.  (With the XCDs filled one after the other, us: 256 tokens over 4096 and over 1024, 16 heads
// of 72, 52 instead of 43; one token of 8 sequences of up to 43 654, 16 heads over 2, 20.6 instead of 17.9.)
__device__ inline int64_t unit_of_block(int64_t round, int64_t units) {
  const int64_t done = round * gridDim.x;
  const int here = static_cast<int>(min(units - done, static_cast<int64_t>(gridDim.x))), b = blockIdx.x;
  if (gridDim.x % 8) return b < here ? done + b : -1;
  const int each = (here + 7) / 8, at = b % 8 * each + b / 8;
  return b / 8 < each && at < here ? done + at : -1;
}
// Where a search has come to: the units of a block rise, so the next one begins there (one token of 1024 sequences of about 300: 267 -> 191 us).
struct Place {
  int s0 = 0;
  int64_t before = 0, slots = 0;    // units and slots of the sequences ahead of s0
};
template <int ROWS>
__device__ inline Found find_unit(const CachedArgs& g, const Deal& d, int64_t u, Share* shares, Place* from) {
  const int lane = threadIdx.x & 63;
  Found f{-1, 0, 1, 0, 0, 0};
  int64_t before = from->before, slots = from->slots;
  for (int s0 = from->s0; s0 < g.seqs.n; s0 += 64) {
    int tiles, pages;                 // (looked up again: kept, they would take two registers of every lane through a unit's work)
    deal_sequence<ROWS>(g, s0 + lane, &tiles, &pages);
    const int splits = splits_of(pages, d.split_pages), lanes = g.seqs.n - s0;
    const int64_t mine = static_cast<int64_t>(tiles) * splits * g.kv_heads, mine_slots = splits > 1 ? mine : 0;
    int64_t upto = mine, upto_slots = mine_slots;
    for (int off = 1; off < lanes && off < 64; off <<= 1) {
      const int64_t a = __shfl_up(upto, off, 64), b = __shfl_up(upto_slots, off, 64);
      if (lane >= off) { upto += a; upto_slots += b; }
    }
    if (shares) {
      if (lane < lanes) shares[s0 + lane] = {splits, tiles, slots + upto_slots - mine_slots};
    } else {
      const uint64_t hit = __ballot(lane < lanes && before + upto > u);
      if (hit) {
        const int l = __builtin_ctzll(hit);
        f.seq = s0 + l;
        f.tiles = __builtin_amdgcn_readlane(tiles, l);
        f.splits = __builtin_amdgcn_readlane(splits, l);
        f.each = (__builtin_amdgcn_readlane(pages, l) + f.splits - 1) / f.splits;
        f.at = static_cast<int>(u - before - of_lane(upto - mine, l));
        f.slot = slots + of_lane(upto_slots - mine_slots, l);
        *from = {s0, before, slots};
        return f;
      }
    }
    const int last = lanes < 64 ? lanes - 1 : 63;
    before += of_lane(upto, last);
    slots += of_lane(upto_slots, last);
  }
  return f;
}

// Keys that new token `tok` of n sees, of `held` in the sequence of which the first `len` count.
__device__ inline int keys_of(const CachedArgs& g, int held, int len, int n, int tok) { return g.causal ? max(0, min(len, held - n + tok + 1)) : len; }

// How the work of tiles of 128 rows is dealt.  The tiles stand in line, sequence by sequence, head by head.
//   Borders: a tile is as long as its pages and kTileCost positions more, and block k takes positions k per .. (k + 1) per - 1, so that all
// blocks that fit on the chip end together.  A border less than kLeastPart pages from either end of a tile's pages moves to that end of the
// tile.  What a block has of a tile that it shares with others goes to slot 2 k (it begins at the border of block k) or 2 k + 1.
//   Units: a position is a tile, or one of its even splits of at least kLeastPages pages, and its number is its slot.  Taken where one round
// of them ends sooner (few tiles: 256 tokens over 4096 and over 1024, 16 heads of 72: 43 us), and where no sequence is longer than
// kLeastPages pages: then nothing is split, and a block takes every so many.
// With whole rounds of even splits instead of borders (us): a frame of 1590 tokens over 27 286, 24 heads of 128, 648 instead of 618; a prompt of
// 4096 tokens over itself, causal, 32 heads over 8 of 128, 286 instead of 174; 512 tokens over 8192, the same heads, 124 instead of 106.  A tile's
// cost of 6 or 9 positions instead of 4 is no faster.
//   Causal tiles count with all pages of their sequence, though the early ones of a prompt see few: what they do not see is skipped, and a block
// whose part it was is done early.  Where a part is shorter than two tiles that leaves much of the chip without work (3000 tokens over themselves, 12
// heads of 128, 114 us; 2000, 24 heads, 106; 4096, 32 heads over 8, two tiles a part, 175; the packed kernel takes 65, 48 and 149).
constexpr int kTileCost = 4, kLeastPart = 8, kLeastPages = 16;
// Causal tiles see the more pages the later they are: the first, the last, the second, ... so that neighbours have the same work together.
__device__ inline int tile_in_line(int j, int tiles, bool causal) { return !causal ? j : j & 1 ? tiles - 1 - (j >> 1) : j >> 1; }
__device__ inline int place_in_line(int tile, int tiles, bool causal) { return !causal ? tile : tile < (tiles + 1) / 2 ? 2 * tile : 2 * (tiles - 1 - tile) + 1; }

// 128 rows a tile, head_dim 64, 72 or 128 (attn_cached_tile.hip).
void launch_attention_cached_tile(const CachedArgs& g, int head_dim, unsigned blocks, hipStream_t st);

}  // namespace speca
