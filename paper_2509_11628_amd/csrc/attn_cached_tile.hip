// Attention over 8-bit pages for many rows: the heads of a frame of new tokens.
//
// One block = 128 rows of one (sequence, key head), 4 waves x 32; a page of 64 keys is one tile.  A row is one query head of one new token.
// The four waves share a page through LDS, where it lies widened to bf16 (exactly: scales are powers of two), so each value is widened
// once per 128 rows: the matrix instructions, not the conversions, are what is left.  The schedule is the one of the bf16 tiles without a
// cache: scores of the next page under the exponentials of this one, pinned around every pair of matrix instructions.
//
// Bytes go to registers while the tile before is worked on and to LDS (two buffers each of keys and values) in the tile after, spread over
// its second contraction.  Keys lie row-major, 16-byte chunks permuted as in the tiles without a cache.  Values arrive by dimension, as the
// page stores them: 16 bytes are one dimension's keys of one lane group, in the order in which S^T hands them on.  Their two widened halves
// go to place [half][tile of 16 dimensions][lane], so a fragment is one read of 16 bytes per lane, all lanes in a row.
//
// What bounds it: the vector unit (exponentials, maxima, widening; 55 % busy, the matrix unit 39 %, LDS 12 %) and what waves wait for, at two
// blocks per unit.  A frame of 1590 tokens over 27 286, 24 heads of 128: 615 to 630 us with the join, 845 to 865 TFLOP/s.  On the way there, us:
// widening in every wave's registers instead (rows of 64 a wave) 1150; through LDS 950; without bank conflicts of the writes 745 with those
// of the values, 683 with those of the keys gone; without registers that spill to memory, whose restores wait for the bytes on their way, 647
// (three or four fragments ahead instead of two spill again: 650 and 715; keys in units of 8 bytes, which spares the turn below, 802).
#include <type_traits>

#include "attn_cached.h"

namespace speca {

namespace {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
union Frag {
  uint32_t u[4];
  uint4 q;
  bf16x8 v;
};

template <int HD>
__device__ inline int key_chunk(int c, int r) {
  return HD == 128 ? c ^ (r & 15) : HD == 64 ? c ^ (r & 7) ^ ((r >> 3) & 1) : c;
}

// Place of dimension l of lane group g among the 64 chunks of a value fragment: the 16 lanes {0-3, 12-15, 20-27} and so on that a read of
// 16 bytes takes at a time hit different banks, and so do 8 threads that write four groups of two dimensions.
__device__ inline int value_place(int l, int g) { return g * 16 + (l ^ (2 * g)); }

// a value that all lanes read, in a scalar register
__device__ inline float scalar(const float* p) { return *reinterpret_cast<const __attribute__((address_space(4))) float*>(reinterpret_cast<uintptr_t>(p)); }

constexpr int ROWS = 128;

// Quotient of values that no lane differs in, below 2^31 as a rule, where the division is a quarter as long.
__device__ inline int64_t quotient(int64_t a, int64_t b) {
  if (((a | b) >> 31) == 0) return static_cast<uint32_t>(a) / static_cast<uint32_t>(b);
  return a / b;
}
__device__ inline int64_t rounded_up(int64_t a, int64_t b) { return quotient(a + b - 1, b); }

// Tiles and pages of sequence s0 + lane; those of the first 64 lie in LDS, where every wave has written them for itself.
typedef int Lists[64][2];
__device__ inline void look_up(const CachedArgs& g, const Lists& lists, int s0, int* tiles, int* pages) {
  const int lane = threadIdx.x & 63;
  if (s0 == 0) {
    *tiles = lists[lane][0];
    *pages = lists[lane][1];
  } else {
    deal_sequence<ROWS>(g, s0 + lane, tiles, pages);
  }
}

// The line of the tiles (attn_cached.h).
struct Line {
  int64_t length, per;
  int split_pages;                  // of units; 0: borders
};
__device__ inline Line lay_out(const CachedArgs& g, const Lists& lists) {
  int64_t count = 0, work = 0;
  int longest = 0;
#pragma unroll 4
  for (int s0 = 0; s0 < g.seqs.n; s0 += 64) {
    int tiles, pages;
    look_up(g, lists, s0, &tiles, &pages);
    work += static_cast<int64_t>(tiles) * pages;
    count += tiles;
    if (tiles) longest = max(longest, pages);
  }
  longest = max_of_wave(longest, g.seqs.n);
  count = sum_of_wave(count, g.seqs.n) * g.kv_heads;
  if (longest <= kLeastPages || !g.shares) return {count, 1, 0x7FFFFFFF};
  work = sum_of_wave(work, g.seqs.n) * g.kv_heads;
  const int64_t weight = work + count * kTileCost;
  const int64_t per = max(static_cast<int64_t>(kLeastPages), rounded_up(weight, g.resident)), room = g.resident - count;
  int split_pages = kLeastPages;
  for (int turn = 0; turn < 2 && room > 0; ++turn) {
    int64_t units = 0;
    int most = 0;
#pragma unroll 4
    for (int s0 = 0; s0 < g.seqs.n; s0 += 64) {
      int tiles, pages;
      look_up(g, lists, s0, &tiles, &pages);
      const int splits = splits_of(pages, split_pages);
      units += static_cast<int64_t>(tiles) * splits;
      if (tiles) most = max(most, (pages + splits - 1) / splits);
    }
    units = sum_of_wave(units, g.seqs.n) * g.kv_heads;
    most = max_of_wave(most, g.seqs.n);
    // (a block between borders has parts of two tiles as a rule)
    if (units <= g.resident && most <= per + kTileCost) return {units, 1, split_pages};
    split_pages = pages_of_split(rounded_up(work, room), kLeastPages, longest);
  }
  return {weight, per, 0};
}
// The sequence whose tiles hold position x, or seq = -1.  With `all` every sequence's stretch is written down instead.
struct Spot {
  int seq, tiles, pages;
  int64_t from;                     // position of its first tile
};
__device__ inline int width(const Line& l, int pages) { return l.split_pages ? splits_of(pages, l.split_pages) : pages + kTileCost; }
__device__ inline Spot seek(const CachedArgs& g, const Line& l, const Lists& lists, int64_t x, Stretch* all) {
  const int lane = threadIdx.x & 63;
  int64_t before = 0;
  for (int s0 = 0; s0 < g.seqs.n; s0 += 64) {
    int tiles, pages;
    look_up(g, lists, s0, &tiles, &pages);
    const int lanes = g.seqs.n - s0;
    const int64_t mine = static_cast<int64_t>(tiles) * g.kv_heads * width(l, pages);
    int64_t upto = mine;
    for (int off = 1; off < lanes && off < 64; off <<= 1) {
      const int64_t a = __shfl_up(upto, off, 64);
      if (lane >= off) upto += a;
    }
    if (all) {
      if (lane < lanes) all[s0 + lane] = {before + upto - mine, l.per, tiles, pages, l.split_pages ? width(l, pages) : 0};
    } else {
      const uint64_t hit = __ballot(lane < lanes && before + upto > x);
      if (hit) {
        const int at = __builtin_ctzll(hit);
        return {s0 + at, static_cast<int>(__builtin_amdgcn_readlane(tiles, at)), static_cast<int>(__builtin_amdgcn_readlane(pages, at)), before + of_lane(upto - mine, at)};
      }
    }
    before += of_lane(upto, lanes < 64 ? lanes - 1 : 63);
  }
  return {-1, 0, 0, 0};
}
// where the border at position x is
__device__ inline int64_t border(const CachedArgs& g, const Line& l, const Lists& lists, int64_t x) {
  if (l.split_pages || x >= l.length) return min(x, l.length);
  const Spot p = seek(g, l, lists, x, nullptr);
  if (p.seq < 0) return l.length;
  const int64_t w = width(l, p.pages), at = p.from + quotient(x - p.from, w) * w;
  return x - at < kLeastPart ? at : at + p.pages - x < kLeastPart ? at + w : x;
}

template <int HD>
__global__ __launch_bounds__(256, 2) void attention_cached_tile_kernel(const CachedArgs g) {
  constexpr int CH = HD / 8;                  // chunks of 8 values of a key
  constexpr int KS = (HD + 31) / 32;          // steps of 32 columns of q k^T
  constexpr int DT = (HD + 15) / 16;          // tiles of 16 dims of O^T
  constexpr bool KW = CH % 8 == 0;            // keys: units of 16 bytes (two chunks) per thread, or of 8 (head_dim 72)
  constexpr int KU = KW ? CH / 8 : (64 * CH + 255) / 256;
  constexpr int VU = (4 * HD + 255) / 256;    // 16-byte units of a value page per thread
  constexpr int KTILE = 64 * HD, VTILE = 2 * DT * 64 * 8;        // elements
  __shared__ __align__(16) uint16_t smem[2 * KTILE + 2 * VTILE + 8];
  __shared__ volatile int64_t reached[4][2];  // of every wave: position in the line, end of the block's part (not needed while a tile is worked on)
  __shared__ Lists lists;
  __shared__ int odd_unit;                    // last of the block's units in which a page that some row does not see all of holds a NaN
  uint16_t* Ks = smem;
  uint16_t* Vs = smem + 2 * KTILE;
  uint16_t* zero = smem + 2 * KTILE + 2 * VTILE;

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l16 = lane & 15, g4 = lane >> 4;
  if (tid < 8) zero[tid] = 0;
  if (tid == 0) odd_unit = -1;
  if (DT * 16 > HD)                           // dimensions beyond the head: zeros, for results that are not stored
    for (int i = tid; i < 2 * VTILE / 8; i += 256) reinterpret_cast<uint4*>(Vs)[i] = make_uint4(0, 0, 0, 0);
  const float scale_log2e = g.scale_log2e;

  int krd[KS];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) krd[ks] = l16 * HD + (key_chunk<HD>(4 * ks + g4, l16) << 3);
  auto key_frag = [&](int kb, int ks, int m) {
    const uint16_t* kc = Ks + kb * KTILE + m * 16 * HD + krd[ks];
    if (4 * ks + 3 >= CH && 4 * ks + g4 >= CH) kc = zero;
    return *reinterpret_cast<const bf16x8*>(kc);
  };
  const int vplace = value_place(l16, g4);
  auto value_frag = [&](int vb, int u, int dt) { return *reinterpret_cast<const bf16x8*>(Vs + vb * VTILE + ((u * DT + dt) * 64 + vplace) * 8); };

  {
    int tiles, pages;
    deal_sequence<ROWS>(g, lane, &tiles, &pages);
    lists[lane][0] = tiles;
    lists[lane][1] = pages;
    asm volatile("" ::: "memory");
  }
  const Line line = lay_out(g, lists);
  int number = 0;                             // of the block's unit
  const int64_t blocks = rounded_up(line.length, line.per);
  for (int round = 0; static_cast<int64_t>(round) * gridDim.x < blocks; ++round) {
    const int64_t block = unit_of_block(round, blocks);
    if (block < 0) continue;
    reached[wave][0] = border(g, line, lists, block * line.per);
    reached[wave][1] = border(g, line, lists, (block + 1) * line.per);
    for (;;) {
      const int64_t pos = of_lane(reached[wave][0], 0), stop = of_lane(reached[wave][1], 0);
      if (pos >= stop) break;
      const Spot f = seek(g, line, lists, pos, nullptr);
      if (f.seq < 0) break;
      const int wide = width(line, f.pages);
      const int64_t index = quotient(pos - f.from, wide), at = f.from + index * wide;
      const int head = static_cast<int>(quotient(index, f.tiles)), row_tile = tile_in_line(static_cast<int>(index - static_cast<int64_t>(head) * f.tiles), f.tiles, g.causal);
      int first = static_cast<int>(pos - at), last;                               // pages
      bool shared;                                                                // with other blocks
      int64_t until, slot;
      if (line.split_pages) {
        const int each = (f.pages + wide - 1) / wide;
        until = pos + 1;
        first *= each;
        last = min(first + each, f.pages);
        shared = wide > 1;
        slot = pos;
      } else {
        until = min(stop, at + wide);
        last = until < at + wide ? static_cast<int>(until - at) : f.pages;
        shared = first > 0 || until < at + wide;
        slot = 2 * block + (first > 0 ? 0 : 1);
      }
      reached[wave][0] = until;
      if (shared && slot >= g.slots) continue;                                    // (offsets that overlap: there is no room for their sums)
      int start, n;
      packed_rows(g.seqs, f.seq, &start, &n);
      start = __builtin_amdgcn_readfirstlane(start);
      n = __builtin_amdgcn_readfirstlane(n);
      const int64_t r0 = static_cast<int64_t>(row_tile) * ROWS, rows = static_cast<int64_t>(n) * g.group;
      const int held = max(0, static_cast<int>(__builtin_amdgcn_readfirstlane(g.lens[f.seq]))), len = min(held, g.max_len);

      // rows 32 wave + 16 i + l16: token, head, number of keys that it sees
      auto place = [&](int i, int* tok, int64_t* column) {
        const int64_t r = min(r0 + wave * 32 + i * 16 + l16, rows - 1);
        *tok = static_cast<int>(r / g.group);
        *column = (static_cast<int64_t>(head) * g.group + (r - static_cast<int64_t>(*tok) * g.group)) * HD;
      };
      int lim[2];
      const int last_tok = static_cast<int>((min(r0 + ROWS, rows) - 1) / g.group), first_tok = static_cast<int>(r0 / g.group);
      const int most = keys_of(g, held, len, n, last_tok), least = keys_of(g, held, len, n, first_tok);
      const int begin = first, end = min(last, (most + PAGE - 1) / PAGE);
      const bool active = r0 + wave * 32 < rows;

      bf16x8 qf[KS][2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        int tok;
        int64_t column;
        place(i, &tok, &column);
        lim[i] = keys_of(g, held, len, n, tok);
        const uint16_t* qp = g.q + (static_cast<int64_t>(start) + tok) * g.ldq + column;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
          Frag x;
          x.q = make_uint4(0, 0, 0, 0);
          const int d = s * 32 + g4 * 8;
          if (d < HD) {
            if (g.wide) x.q = *reinterpret_cast<const uint4*>(qp + d);
            else {
#pragma unroll
              for (int j = 0; j < 4; ++j) x.u[j] = qp[d + 2 * j] | static_cast<uint32_t>(qp[d + 2 * j + 1]) << 16;
            }
          }
          qf[s][i] = x.v;
        }
      }

      // Numbers of the unit's pages, 64 at a time, one a lane (lengths are bounded by the table's row).  One that is not held is worked on
      // like the others, with some page's bytes, none of which any row sees.
      const int32_t* table = g.table + static_cast<int64_t>(f.seq) * g.table_ld;
      const int tiles = end - begin;
      int ids = -1;
      int cache_pages = g.pages;
      asm("" : "+s"(cache_pages));
      auto number_of = [&](int t) {             // t rises
        if ((t & 63) == 0) ids = t + lane < tiles ? table[begin + t + lane] : -1;
        const int page = __builtin_amdgcn_readlane(ids, t & 63);
        return page < 0 || page >= cache_pages ? -1 : page;
      };

      // Staging: 8-byte units of the keys, 16-byte units of the values, linear in the page.
      typedef std::conditional_t<KW, u32x4, u32x2> KeyUnit;
      KeyUnit ka[KU];
      u32x4 va[VU];
      float kscale = 0.0f, vscale = 0.0f;
      // Through buffer descriptors of a page: one register of offsets serves keys and values, and what lies beyond the page reads as zeros.
      // (the addresses as values of their own: as parts of the arguments the compiler keeps and restores whole groups of them)
      uint64_t k_at = reinterpret_cast<uint64_t>(g.k + static_cast<int64_t>(head) * (PAGE * HD)), v_at = reinterpret_cast<uint64_t>(g.v + static_cast<int64_t>(head) * (PAGE * HD));
      uint64_t ks_at = reinterpret_cast<uint64_t>(g.k_scale + head), vs_at = reinterpret_cast<uint64_t>(g.v_scale + head);
      uint32_t heads = g.kv_heads;
      asm("" : "+s"(k_at), "+s"(v_at), "+s"(ks_at), "+s"(vs_at), "+s"(heads));
      auto load_k = [&](int page) {
        const uint64_t at = static_cast<uint64_t>(page < 0 ? 0 : page) * heads;
        kscale = scalar(reinterpret_cast<const float*>(ks_at + at * 4));
        const auto from = __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<uint8_t*>(k_at + at * (PAGE * HD)), 0, PAGE * HD, 0x00020000);
#pragma unroll
        for (int u = 0; u < KU; ++u) {
          if constexpr (KW) ka[u] = __builtin_amdgcn_raw_buffer_load_b128(from, tid * 16, 4096 * u, 0);
          else ka[u] = __builtin_amdgcn_raw_buffer_load_b64(from, tid * 8, 2048 * u, 0);
        }
      };
      auto load_v = [&](int page) {
        const uint64_t at = static_cast<uint64_t>(page < 0 ? 0 : page) * heads;
        vscale = scalar(reinterpret_cast<const float*>(vs_at + at * 4));
        const auto from = __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<uint8_t*>(v_at + at * (PAGE * HD)), 0, PAGE * HD, 0x00020000);
#pragma unroll
        for (int u = 0; u < VU; ++u) va[u] = __builtin_amdgcn_raw_buffer_load_b128(from, tid * 16, 4096 * u, 0);
      };
      auto stage_k = [&](int buf, int u) {
        if constexpr (KW) {                     // rows CH / 2 units long: 512 / CH rows further with every u, which leaves the permutation as it is
          const int r = tid / (CH / 2), p = 2 * (tid % (CH / 2));
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            Frag x;
            // every other four threads write their second chunk first: 8 threads then hit different banks
            const bool turn = (tid & 4) != 0;
            widen(turn ? ka[u][2 - 2 * h] : ka[u][2 * h], kscale, x.u);
            widen(turn ? ka[u][3 - 2 * h] : ka[u][2 * h + 1], kscale, x.u + 2);
            *reinterpret_cast<uint4*>(Ks + buf * KTILE + r * HD + (key_chunk<HD>(p + (turn ? 1 - h : h), r) << 3) + u * (512 / CH) * HD) = x.q;
          }
        } else {
          const int c = tid + 256 * u, r = static_cast<unsigned>(c) / CH, p = c - r * CH;
          if (c >= 64 * CH) return;
          Frag x;
          widen(ka[u][0], kscale, x.u);
          widen(ka[u][1], kscale, x.u + 2);
          *reinterpret_cast<uint4*>(Ks + buf * KTILE + r * HD + (key_chunk<HD>(p, r) << 3)) = x.q;
        }
      };
      // Whether some row does not see all of page `at` of the sequence, which is page `page` of the cache.
      auto is_edge = [&](int at, int page) { return (at + 1) * PAGE > least || page < 0; };
      // What is done once to the values of such a page: bytes past the last token, whatever they
      // are, become 0, and so does a NaN, which must not meet the probability 0 of a row that does not see it.  The rows that do get it at
      // the end.
      auto edge_v = [&](int at, int page) {
        if (page < 0) vscale = 1.0f;            // (a scale that is no number would not leave the zeros zeros)
#pragma unroll
        for (int u = 0; u < VU; ++u) {
          const int left = (page < 0 ? 0 : len) - (at * PAGE + 4 * (tid & 3));
          uint32_t any = 0;
#pragma unroll
          for (int m = 0; m < 4; ++m) {
            const int c = left - 16 * m;
            va[u][m] &= c >= 4 ? ~0u : c <= 0 ? 0u : (1u << (8 * c)) - 1u;
            const uint32_t nan = ((va[u][m] & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u;
            va[u][m] &= ~((nan >> 7) * 0xFFu);
            any |= nan;
          }
          if (any && (4 * HD % 256 == 0 || tid + 256 * u < 4 * HD)) odd_unit = number;
        }
      };
      auto stage_v = [&](int buf, int u, int half) {
        if (4 * HD % 256 != 0 && tid + 256 * u >= 4 * HD) return;
        const int d = tid >> 2, grp = tid & 3;  // and 64 dimensions further with every u
        Frag x;
        widen(va[u][2 * half], vscale, x.u);
        widen(va[u][2 * half + 1], vscale, x.u + 2);
        *reinterpret_cast<uint4*>(Vs + buf * VTILE + ((d >> 4) * 64 + value_place(d & 15, grp)) * 8 + (half * DT + 4 * u) * 512) = x.q;
      };

      floatx4 o[DT][2];
#pragma unroll
      for (int i = 0; i < DT; ++i)
#pragma unroll
        for (int e = 0; e < 2; ++e) o[i][e] = floatx4{};
      // Online softmax.  A lane's scores of a tile: s[m][i][e], key 16 m + 4 g4 + e, row 16 i + l16.
      float mref[2] = {-INFINITY, -INFINITY}, moff[2] = {}, lrun[2] = {}, psum[2] = {}, corr[2] = {1.0f, 1.0f}, tmax[2];
      bool moved = false, seen[2] = {false, false};
      auto maximum = [&](const floatx4 (&s)[4][2], int from, int to) {
#pragma unroll
        for (int i = from; i < to; ++i) tmax[(i >> 2) & 1] = fmaxf(tmax[(i >> 2) & 1], s[i >> 3][(i >> 2) & 1][i & 3]);
      };
      auto reference = [&](int at, int page) {
        moved = false;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const float mnew = fmaxf(mref[i], max_of_groups(tmax[i]));
          moff[i] = mnew == -INFINITY ? 0.0f : mnew * scale_log2e;     // no finite score yet: weights 0
          corr[i] = fast_exp2(mref[i] * scale_log2e - moff[i]);
          moved |= mnew != mref[i];
          mref[i] = mnew;
          seen[i] |= page >= 0 && at * PAGE < lim[i];
        }
      };
      auto probabilities = [&](floatx4 (&s)[4][2], int from, int to) {
#pragma unroll
        for (int i = from; i < to; ++i) {
          const int m = i >> 3, e = (i >> 2) & 1;
          const float p = fast_exp2(fmaf(s[m][e][i & 3], scale_log2e, -moff[e]));
          s[m][e][i & 3] = p;
          psum[e] += p;
        }
      };
      // P^T of keys 32 u .. 32 u + 31, rounded to bf16 for the matrix instructions; the sum, in fp32, has them unrounded
      auto pack = [&](const floatx4 (&s)[4][2], int u, int i) {
        Frag x;
        x.q = make_uint4(cvt_pk_bf16(s[2 * u][i][0], s[2 * u][i][1]), cvt_pk_bf16(s[2 * u][i][2], s[2 * u][i][3]),
                         cvt_pk_bf16(s[2 * u + 1][i][0], s[2 * u + 1][i][1]), cvt_pk_bf16(s[2 * u + 1][i][2], s[2 * u + 1][i][3]));
        return x.v;
      };
      auto mask = [&](floatx4 (&s)[4][2], int at, int page) {          // keys that a row does not see
        const int left[2] = {page < 0 ? 0 : lim[0] - at * PAGE - 4 * g4, page < 0 ? 0 : lim[1] - at * PAGE - 4 * g4};
#pragma unroll
        for (int i = 0; i < 32; ++i)
          if ((i >> 3) * 16 + (i & 3) >= left[(i >> 2) & 1]) s[i >> 3][(i >> 2) & 1][i & 3] = -INFINITY;
      };

#define SPECA_PIN() __builtin_amdgcn_sched_barrier(0)
// LDS reads and writes done, then everybody; the bytes on their way from memory stay on their way
#define SPECA_TURN()                                        \
  {                                                         \
      __builtin_amdgcn_s_waitcnt(0xC07F);                     \
      asm volatile("" ::: "memory");                          \
      __builtin_amdgcn_s_barrier();                           \
      asm volatile("" ::: "memory");                          \
      SPECA_PIN();                                            \
  }
      constexpr int NS = 4 * KS, NV = 2 * DT, RA = 2, NP = 20;
      // Tile in buffer `buf`, whose scores lie in sc with their reference known.  NEXT: its successor is page at1 of the sequence, page1 of
      // the cache, whose keys lie in the other buffer and whose values are in va; page2 is the one behind it, whose keys are in ka, and page3
      // the one behind that.  (Where there is none, some page is loaded and staged, and not used.)
      auto tile = [&](floatx4 (&sc)[4][2], floatx4 (&sn)[4][2], int buf, int at1, int page1, int page2, int page3, auto next_tag) {
        constexpr bool NEXT = decltype(next_tag)::value;
        bf16x8 kf[NS], vf[NV], pf[2][2];
        const bool edge = NEXT && is_edge(at1, page1);
        if (edge) edge_v(at1, page1);
        constexpr int STEPS = KU + 2 * VU + 1;
        auto staging = [&](int i) {
          if constexpr (NEXT) {
            if (i < KU) stage_k(buf, i);
            else if (i < KU + 2 * VU) stage_v(1 - buf, (i - KU) >> 1, (i - KU) & 1);
            else { load_k(page3); load_v(page2); }
          }
        };
        if (active) {
          if constexpr (NEXT) {
#pragma unroll
            for (int i = 0; i < RA; ++i) kf[i] = key_frag(1 - buf, i >> 2, i & 3);
            SPECA_PIN();
          }
          if (__any(moved)) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              lrun[i] *= corr[i];
#pragma unroll
              for (int dt = 0; dt < DT; ++dt) o[dt][i] *= corr[i];
            }
          }
          psum[0] = psum[1] = 0.0f;
          if constexpr (NEXT) {
#pragma unroll
            for (int i = 0; i < NS; ++i) {
              if (i + RA < NS) kf[i + RA] = key_frag(1 - buf, (i + RA) >> 2, (i + RA) & 3);
              else vf[i + RA - NS] = value_frag(buf, (i + RA - NS) / DT, (i + RA - NS) % DT);
              if (i >= NS - 2) pf[0][i - NS + 2] = pack(sc, 0, i - NS + 2);
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                probabilities(sc, (2 * i + e) * NP / (2 * NS), (2 * i + e + 1) * NP / (2 * NS));
                SPECA_PIN();
                sn[i & 3][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[i], qf[i >> 2][e], i < 4 ? floatx4{} : sn[i & 3][e], 0, 0, 0);
                SPECA_PIN();
              }
            }
          } else {
#pragma unroll
            for (int i = 0; i < RA; ++i) vf[i] = value_frag(buf, i / DT, i % DT);
            probabilities(sc, 0, NP);
#pragma unroll
            for (int e = 0; e < 2; ++e) pf[0][e] = pack(sc, 0, e);
          }
          tmax[0] = tmax[1] = -INFINITY;
#pragma unroll
          for (int i = 0; i < NV; ++i) {
            if (i + RA < NV) vf[i + RA] = value_frag(buf, (i + RA) / DT, (i + RA) % DT);
            if (i >= DT - 1 && i <= DT) pf[1][i - DT + 1] = pack(sc, 1, i - DT + 1);
            if (i < STEPS) staging(i);
            if constexpr (NEXT) {
              if (i == DT && edge) mask(sn, at1, page1);
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              if (i < DT) probabilities(sc, NP + (2 * i + e) * (32 - NP) / (2 * DT - 1), i + 1 == DT && e ? 32 : NP + (2 * i + e + 1) * (32 - NP) / (2 * DT - 1));
              else if constexpr (NEXT) maximum(sn, (2 * (i - DT) + e) * 32 / (2 * DT), (2 * (i - DT) + e + 1) * 32 / (2 * DT));
              SPECA_PIN();
              o[i % DT][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[i], pf[i / DT][e], o[i % DT][e], 0, 0, 0);
              SPECA_PIN();
            }
          }
#pragma unroll
          for (int i = NV; i < STEPS; ++i) staging(i);
#pragma unroll
          for (int e = 0; e < 2; ++e) lrun[e] += psum[e];
          if constexpr (NEXT) reference(at1, page1);
        } else {
#pragma unroll
          for (int i = 0; i < STEPS; ++i) staging(i);
        }
      };

      // Keys are loaded three pages ahead and staged two ahead, values one less.
      floatx4 sa[4][2], sb[4][2];
      if (tiles > 0) {
        int page0 = number_of(0), page1 = tiles > 1 ? number_of(1) : -1, page2 = tiles > 2 ? number_of(2) : -1;
        load_k(page0);
        load_v(page0);
        SPECA_TURN()                            // the unit before is through with LDS, and the zeros of the first are written
#pragma unroll
        for (int u = 0; u < KU; ++u) stage_k(0, u);
        load_k(page1);
        if (is_edge(begin, page0)) edge_v(begin, page0);
#pragma unroll
        for (int u = 0; u < VU; ++u)
#pragma unroll
          for (int h = 0; h < 2; ++h) stage_v(0, u, h);
        load_v(page1);
#pragma unroll
        for (int u = 0; u < KU; ++u) stage_k(1, u);
        load_k(page2);
        SPECA_TURN()
        if (active) {
#pragma unroll
          for (int i = 0; i < NS; ++i) {
            const bf16x8 kf = key_frag(0, i >> 2, i & 3);
#pragma unroll
            for (int e = 0; e < 2; ++e) sa[i & 3][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[i >> 2][e], i < 4 ? floatx4{} : sa[i & 3][e], 0, 0, 0);
          }
          if (is_edge(begin, page0)) mask(sa, begin, page0);
          tmax[0] = tmax[1] = -INFINITY;
          maximum(sa, 0, 32);
          reference(begin, page0);
        }
        // buffers alternate, and so do the two sets of scores
#define SPECA_TILE(PAR, SC, SN)                                                               \
  {                                                                                           \
      const int page3 = t + PAR + 3 < tiles ? number_of(t + PAR + 3) : -1;                      \
      SPECA_TURN()                                                                              \
      tile(SC, SN, PAR, begin + t + PAR + 1, page1, page2, page3, std::true_type());            \
      page1 = page2; page2 = page3;                                                             \
  }
        int t = 0;
        for (; t + 2 < tiles; t += 2) {
          SPECA_TILE(0, sa, sb)
          SPECA_TILE(1, sb, sa)
        }
        if (t + 1 < tiles) {
          SPECA_TILE(0, sa, sb)
          ++t;
#pragma unroll
          for (int m = 0; m < 4; ++m)
#pragma unroll
            for (int e = 0; e < 2; ++e) sa[m][e] = sb[m][e];
        }
#undef SPECA_TILE
        SPECA_TURN()
        tile(sa, sb, t & 1, 0, 0, 0, 0, std::false_type());
        if (odd_unit == number) {               // (written ahead of the last turn)
          for (int at = max(begin, least / PAGE); at < end; ++at) {
            const int page = table[at];
            if (page < 0 || page >= g.pages) continue;
            const uint8_t* v = g.v + (static_cast<int64_t>(page) * g.kv_heads + head) * (PAGE * HD);
#pragma unroll
            for (int dt = 0; dt < DT; ++dt)
#pragma unroll
              for (int q = 0; q < 4; ++q) {
                const int d = dt * 16 + 4 * g4 + q < HD ? dt * 16 + 4 * g4 + q : HD - 1;
                bool hit[2] = {false, false};
#pragma unroll 1
                for (int c = 0; c < PAGE; ++c)
                  if ((v[d * PAGE + c] & 0x7F) == 0x7F) {
                    const int key = at * PAGE + 16 * (c >> 2 & 3) + 4 * (c >> 4) + (c & 3);
                    hit[0] |= key < lim[0];
                    hit[1] |= key < lim[1];
                  }
#pragma unroll
                for (int e = 0; e < 2; ++e)
                  if (hit[e]) o[dt][e][q] = __uint_as_float(0x7FC00000u);
              }
          }
        }
      }
      ++number;
#undef SPECA_TURN
#undef SPECA_PIN

      if (!active) continue;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int r = wave * 32 + i * 16 + l16;
        float total = sum_of_groups(lrun[i]);
        // keys were there, none with a score above -inf: that has no softmax.  No keys: 0
        if (mref[i] == -INFINITY) total = seen[i] ? __uint_as_float(0x7FC00000u) : 0.0f;
        if (shared && g4 == 0) {
          g.stats[slot * 2 * ROWS + r] = mref[i];
          g.stats[slot * 2 * ROWS + ROWS + r] = total;
        }
        const float inv = total == 0.0f ? 0.0f : 1.0f / total;
        int tok;
        int64_t column;
        place(i, &tok, &column);
        uint16_t* op = g.out + (static_cast<int64_t>(start) + tok) * g.ldo + column + 4 * g4;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
          if (dt * 16 + 4 * g4 >= HD) continue;
          if (shared) {
            *reinterpret_cast<floatx4*>(g.part + (slot * ROWS + r) * HD + dt * 16 + 4 * g4) = o[dt][i];
          } else if (r0 + r < rows) {
            uint16_t* to = op + dt * 16;
            const uint32_t a = cvt_pk_bf16(o[dt][i][0] * inv, o[dt][i][1] * inv), b = cvt_pk_bf16(o[dt][i][2] * inv, o[dt][i][3] * inv);
            if (g.wide) *reinterpret_cast<uint2*>(to) = make_uint2(a, b);
            else { to[0] = static_cast<uint16_t>(a); to[1] = static_cast<uint16_t>(a >> 16); to[2] = static_cast<uint16_t>(b); to[3] = static_cast<uint16_t>(b >> 16); }
          }
        }
      }
    }
  }
  if (g.shares && blockIdx.x == 0 && wave == 0) seek(g, line, lists, 0, static_cast<Stretch*>(g.shares));
}

}  // namespace

void launch_attention_cached_tile(const CachedArgs& g, int head_dim, unsigned blocks, hipStream_t st) {
  if (head_dim == 64) attention_cached_tile_kernel<64><<<blocks, 256, 0, st>>>(g);
  else if (head_dim == 72) attention_cached_tile_kernel<72><<<blocks, 256, 0, st>>>(g);
  else attention_cached_tile_kernel<128><<<blocks, 256, 0, st>>>(g);
}

}  // namespace speca
