// Attention of new tokens over keys and values in 8-bit pages: few rows, and the join of split ranges.
//
// One block = 16 NQ rows of one (sequence, key head); a row is one query head of one new token, so the heads that share a key head share its
// reads.  Four waves take the pages w, w + 4, ... of the block's range with an online softmax of their own and merge at the end; where rows
// are few, the range of keys is split over blocks as well (attn_cached.h), whose sums a second launch joins.
//   S^T[key][row] = K q^T,  O^T[d][row] += V^T P^T   (bf16 16x16x32 instructions, keys and values widened from e4m3 under their page's
// scale, exactly: the scale is a power of two)
// Nothing goes through LDS on its way: a page's layout is the operands' one.  Lane (l, g) of an operand wants 8 of 32 columns of key 16 m +
// l; it takes 16 bytes at 16 g, which serve two instructions (the order of the columns is a dummy, q follows it).  Of value dimension d it
// wants the keys in the order in which S^T holds them (4 g .. 4 g + 3 of every 16), which is how the page stores them: 16 bytes per
// dimension.  A page's bytes are asked for as soon as the registers of the page before are free: 16 KB per wave and 128 columns, 128 KB per
// unit, always under way.
//
// What bounds it: memory.  One token of 8 sequences of 257 to 65 000 tokens, 32 heads over 8 of 128: 90 us for 437 MB, 4.9 TB/s (a large
// copy moves 5.0); of 1024 of about 1000 413 us for 2.2 GB.  Short ones are a chain of waits: lists, table, bytes, the four waves' sums;
// four sequences of 1 to 1200 tokens take 13 us.
#include <algorithm>
#include <cmath>

#include "attn_cached.h"
#include "gemm.h"

namespace speca {

namespace {

typedef uint32_t u32x4_at8 __attribute__((ext_vector_type(4), aligned(8)));       // head size 72: rows of 72 bytes
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

union Frag {
  uint32_t u[4];
  bf16x8 v;
};

template <int HD, int NQ>
__global__ __launch_bounds__(256, 2) void attention_cached_kernel(const CachedArgs g) {
  constexpr int FULL = HD / 64, REM = HD % 64;
  constexpr int KS = 2 * FULL + (REM ? 1 : 0);     // steps of 32 columns
  constexpr int DT = (HD + 15) / 16;
  constexpr int ROWS = 16 * NQ;
  static_assert(REM <= 32 && REM % 8 == 0, "head_dim");
  __shared__ __align__(16) floatx4 merge[4][DT * NQ][64];
  __shared__ float stat_m[4][ROWS], stat_l[4][ROWS], stat_seen[4][ROWS];

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l16 = lane & 15, g4 = lane >> 4;
  const Deal d = deal<ROWS>(g);
  if (g.shares && blockIdx.x == 0 && wave == 0) {
    Place all;
    find_unit<ROWS>(g, d, 0, static_cast<Share*>(g.shares), &all);
  }
  Place search;
  for (int64_t round = 0; round * gridDim.x < d.units; ++round) {
    const int64_t unit = unit_of_block(round, d.units);
    if (unit < 0) continue;
    const Found f = find_unit<ROWS>(g, d, unit, nullptr, &search);
    if (f.seq < 0 || (f.splits > 1 && f.slot + f.at >= g.slots)) continue;        // (offsets that overlap: there is no room for their sums)
    const int tile = f.at % f.tiles, split = f.at / f.tiles % f.splits, head = f.at / f.tiles / f.splits, seq = f.seq;
    int start, n;
    packed_rows(g.seqs, seq, &start, &n);
    const int64_t r0 = static_cast<int64_t>(tile) * ROWS, rows = static_cast<int64_t>(n) * g.group;
    const int held = max(0, g.lens[seq]), len = min(held, g.max_len);

    // rows 16 i + l16: token, head, number of keys that it sees
    int tok[NQ], sub[NQ], lim[NQ];
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
      const int64_t r = r0 + i * 16 + l16 < rows ? r0 + i * 16 + l16 : rows - 1;
      tok[i] = static_cast<int>(r / g.group);
      sub[i] = static_cast<int>(r - static_cast<int64_t>(tok[i]) * g.group);
      lim[i] = keys_of(g, held, len, n, tok[i]);
    }
    const int last_tok = static_cast<int>((min(r0 + ROWS, rows) - 1) / g.group), first_tok = static_cast<int>(r0 / g.group);
    const int most = keys_of(g, held, len, n, last_tok), least = keys_of(g, held, len, n, first_tok);
    const int begin = split * f.each, end = min(begin + f.each, (most + PAGE - 1) / PAGE);

    bf16x8 qf[KS][NQ];
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
      const uint16_t* qp = g.q + (static_cast<int64_t>(start) + tok[i]) * g.ldq + (static_cast<int64_t>(head) * g.group + sub[i]) * HD;
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        const int d = s < 2 * FULL ? (s / 2) * 64 + g4 * 16 + (s % 2) * 8 : 64 * FULL + g4 * 8;
        Frag f;
        f.u[0] = f.u[1] = f.u[2] = f.u[3] = 0;
        if (d < HD) {
          if (g.wide) {
            const uint4 w = *reinterpret_cast<const uint4*>(qp + d);
            f.u[0] = w.x; f.u[1] = w.y; f.u[2] = w.z; f.u[3] = w.w;
          } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) f.u[j] = qp[d + 2 * j] | static_cast<uint32_t>(qp[d + 2 * j + 1]) << 16;
          }
        }
        qf[s][i] = f.v;
      }
    }

    floatx4 o[DT][NQ];
    float mref[NQ], lrun[NQ];
    bool seen[NQ];
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
      mref[i] = -INFINITY;
      lrun[i] = 0.0f;
      seen[i] = false;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) o[dt][i] = floatx4{};
    }

    const int32_t* table = g.table + static_cast<int64_t>(seq) * g.table_ld;
    u32x4 kr[4][FULL ? FULL : 1], vr[DT];
    u32x2 kx[4];
    float ks = 0.0f, vs = 0.0f;
    auto load_k = [&](int page) {
      const int64_t unit = static_cast<int64_t>(page) * g.kv_heads + head;
      const uint8_t* p = g.k + unit * (PAGE * HD) + l16 * HD;
      ks = g.k_scale[unit];
#pragma unroll
      for (int m = 0; m < 4; ++m) {
#pragma unroll
        for (int j = 0; j < FULL; ++j) kr[m][j] = *reinterpret_cast<const u32x4_at8*>(p + m * 16 * HD + j * 64 + g4 * 16);
        if constexpr (REM > 0) {
          kx[m] = u32x2{0, 0};
          if (g4 * 8 < REM) kx[m] = *reinterpret_cast<const u32x2*>(p + m * 16 * HD + FULL * 64 + g4 * 8);
        }
      }
    };
    auto load_v = [&](int page) {
      const int64_t unit = static_cast<int64_t>(page) * g.kv_heads + head;
      const uint8_t* p = g.v + unit * (PAGE * HD) + g4 * 16;
      vs = g.v_scale[unit];
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        const int d = dt * 16 + l16;
        vr[dt] = *reinterpret_cast<const u32x4*>(p + (d < HD ? d : HD - 1) * PAGE);        // beyond the head: any, never stored
      }
    };
    // Numbers of the wave's next 64 pages, one a lane; those that are not held are passed over.  (Lengths are bounded by the table's row.)
    int ids = -1, j = begin + wave, ids_from = j;
    auto fetch_ids = [&] {
      ids_from = j;
      const int at = j + 4 * lane;
      ids = at < end ? table[at] : -1;
      if (ids >= g.pages) ids = -1;
    };
    auto page_at = [&] {                             // of j, or of the first one held behind it
      for (;;) {
        if (j >= end) return -1;
        if (j - ids_from >= 256) fetch_ids();
        const uint64_t held = __ballot(ids >= 0) >> ((j - ids_from) >> 2);
        if (held) {
          j += 4 * __builtin_ctzll(held);
          return __builtin_amdgcn_readlane(ids, (j - ids_from) >> 2);
        }
        j = ids_from + 256;
      }
    };
    fetch_ids();
    int page = page_at();
    if (page >= 0) {
      load_k(page);
      load_v(page);
    }
    while (page >= 0) {
      const int here = j;
      j += 4;
      const int next = page_at();
      const float vscale = vs;
      floatx4 s[4][NQ];
#pragma unroll
      for (int m = 0; m < 4; ++m) {
#pragma unroll
        for (int t = 0; t < KS; ++t) {
          Frag f;
          if (t < 2 * FULL) {
            widen(kr[m][t / 2][2 * (t % 2)], ks, f.u);
            widen(kr[m][t / 2][2 * (t % 2) + 1], ks, f.u + 2);
          } else {
            widen(kx[m][0], ks, f.u);
            widen(kx[m][1], ks, f.u + 2);
          }
#pragma unroll
          for (int i = 0; i < NQ; ++i) s[m][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f.v, qf[t][i], t ? s[m][i] : floatx4{}, 0, 0, 0);
        }
      }
      if (next >= 0) load_k(next);                   // its operands are in registers by now
      const bool edge = (here + 1) * PAGE > least;
      bool odd = false;                              // the page holds a NaN that some row does not see
      if (edge) {
#pragma unroll
        for (int i = 0; i < NQ; ++i) {
#pragma unroll
          for (int m = 0; m < 4; ++m)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (here * PAGE + 16 * m + 4 * g4 + e >= lim[i]) s[m][i][e] = -INFINITY;
        }
#pragma unroll
        for (int m = 0; m < 4; ++m) {                // bytes past the last token: whatever they are, 0 now
          const int c = len - (here * PAGE + 16 * m + 4 * g4);
          const uint32_t keep = c >= 4 ? ~0u : c <= 0 ? 0u : (1u << (8 * c)) - 1u;
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) {
            vr[dt][m] &= keep;
            odd |= (((vr[dt][m] & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u) != 0;
          }
        }
        odd = __any(odd);
      }
      bool moved = false;
      float corr[NQ];
#pragma unroll
      for (int i = 0; i < NQ; ++i) {
        float top = -INFINITY;
#pragma unroll
        for (int m = 0; m < 4; ++m)
#pragma unroll
          for (int e = 0; e < 4; ++e) top = fmaxf(top, s[m][i][e]);
        const float mnew = fmaxf(mref[i], max_of_groups(top));
        const float moff = mnew == -INFINITY ? 0.0f : mnew * g.scale_log2e;          // no finite score yet: weights 0
        corr[i] = fast_exp2(mref[i] * g.scale_log2e - moff);
        moved |= mnew != mref[i];
        mref[i] = mnew;
        seen[i] |= here * PAGE < lim[i];
        float sum = 0.0f;
#pragma unroll
        for (int m = 0; m < 4; ++m)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float p = fast_exp2(fmaf(s[m][i][e], g.scale_log2e, -moff));
            s[m][i][e] = p;
            sum += p;
          }
        lrun[i] = lrun[i] * corr[i] + sum;
      }
      if (__any(moved)) {
#pragma unroll
        for (int i = 0; i < NQ; ++i)
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) o[dt][i] *= corr[i];
      }
      if (odd) {
        // A NaN counts for the rows that see it and must not meet the probability 0 of the others: it is taken out of the page, and a
        // product of the places of NaN with the places that a row sees says where it belongs.
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
          floatx4 hit[NQ];
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            Frag a;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const uint32_t w = vr[dt][2 * u + h], nan = ((w & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u;
              a.u[2 * h] = (nan & 0x80u ? 0x3F80u : 0u) | (nan & 0x8000u ? 0x3F800000u : 0u);
              a.u[2 * h + 1] = (nan & 0x800000u ? 0x3F80u : 0u) | (nan & 0x80000000u ? 0x3F800000u : 0u);
              vr[dt][2 * u + h] = w & ~((nan >> 7) * 0xFFu);
            }
#pragma unroll
            for (int i = 0; i < NQ; ++i) {
              Frag b;
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const int key = here * PAGE + 16 * (2 * u + e / 2) + 4 * g4 + 2 * (e % 2);
                b.u[e] = (key < lim[i] ? 0x3F80u : 0u) | (key + 1 < lim[i] ? 0x3F800000u : 0u);
              }
              hit[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v, b.v, u ? hit[i] : floatx4{}, 0, 0, 0);
            }
          }
#pragma unroll
          for (int i = 0; i < NQ; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (hit[i][e] > 0.0f) o[dt][i][e] = __uint_as_float(0x7FC00000u);
        }
      }
      bf16x8 pf[2][NQ];                              // rounded to bf16 for the matrix instructions; their sum, in fp32, has them unrounded
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < NQ; ++i) {
          Frag f;
          f.u[0] = cvt_pk_bf16(s[2 * u][i][0], s[2 * u][i][1]);
          f.u[1] = cvt_pk_bf16(s[2 * u][i][2], s[2 * u][i][3]);
          f.u[2] = cvt_pk_bf16(s[2 * u + 1][i][0], s[2 * u + 1][i][1]);
          f.u[3] = cvt_pk_bf16(s[2 * u + 1][i][2], s[2 * u + 1][i][3]);
          pf[u][i] = f.v;
        }
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          Frag f;
          widen(vr[dt][2 * u], vscale, f.u);
          widen(vr[dt][2 * u + 1], vscale, f.u + 2);
#pragma unroll
          for (int i = 0; i < NQ; ++i) o[dt][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f.v, pf[u][i], o[dt][i], 0, 0, 0);
        }
      if (next >= 0) load_v(next);
      page = next;
    }

    // together: everything relative to the largest maximum of the four waves; wave w sums the dimensions of tiles w, w + 4, ...
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
      const float l = sum_of_groups(lrun[i]);
      if (g4 == 0) {
        stat_m[wave][i * 16 + l16] = mref[i];
        stat_l[wave][i * 16 + l16] = l;
        stat_seen[wave][i * 16 + l16] = seen[i] ? 1.0f : 0.0f;
      }
    }
    __syncthreads();
    float top[NQ], total[NQ];
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
      const int r = i * 16 + l16;
      top[i] = fmaxf(fmaxf(stat_m[0][r], stat_m[1][r]), fmaxf(stat_m[2][r], stat_m[3][r]));
      const float off = top[i] == -INFINITY ? 0.0f : top[i] * g.scale_log2e;
      total[i] = 0.0f;
#pragma unroll
      for (int w = 0; w < 4; ++w) total[i] += stat_l[w][r] * fast_exp2(stat_m[w][r] * g.scale_log2e - off);
      // keys were there, none with a score above -inf: that has no softmax.  No keys: 0
      if (top[i] == -INFINITY) total[i] = stat_seen[0][r] + stat_seen[1][r] + stat_seen[2][r] + stat_seen[3][r] > 0.0f ? __uint_as_float(0x7FC00000u) : 0.0f;
      const float f = fast_exp2(mref[i] * g.scale_log2e - off);
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) merge[wave][dt * NQ + i][lane] = o[dt][i] * f;
    }
    __syncthreads();
    const int64_t slot = f.slot + f.at;
    if (f.splits > 1 && wave == 0 && g4 == 0) {
#pragma unroll
      for (int i = 0; i < NQ; ++i) {
        g.stats[slot * 2 * ROWS + i * 16 + l16] = top[i];
        g.stats[slot * 2 * ROWS + ROWS + i * 16 + l16] = total[i];
      }
    }
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      if (dt % 4 != wave) continue;
      const int d = dt * 16 + 4 * g4;
      if (d >= HD) continue;
#pragma unroll
      for (int i = 0; i < NQ; ++i) {
        const floatx4 v = (merge[0][dt * NQ + i][lane] + merge[1][dt * NQ + i][lane]) + (merge[2][dt * NQ + i][lane] + merge[3][dt * NQ + i][lane]);
        if (f.splits > 1) {
          *reinterpret_cast<floatx4*>(g.part + (slot * ROWS + i * 16 + l16) * HD + d) = v;
        } else if (r0 + i * 16 + l16 < rows) {
          uint16_t* op = g.out + (static_cast<int64_t>(start) + tok[i]) * g.ldo + (static_cast<int64_t>(head) * g.group + sub[i]) * HD + d;
          const float inv = total[i] == 0.0f ? 0.0f : 1.0f / total[i];
          const uint32_t a = cvt_pk_bf16(v[0] * inv, v[1] * inv), b = cvt_pk_bf16(v[2] * inv, v[3] * inv);
          if (g.wide) *reinterpret_cast<uint2*>(op) = make_uint2(a, b);
          else { op[0] = static_cast<uint16_t>(a); op[1] = static_cast<uint16_t>(a >> 16); op[2] = static_cast<uint16_t>(b); op[3] = static_cast<uint16_t>(b >> 16); }
        }
      }
    }
    __syncthreads();                                 // the next unit writes the statistics again
  }
}

// Joins the splits of the rows of a tile of ROWS, four rows at a time, `quads` times per block: wave w sums the splits w, w + WAVES, ... in
// their order, then the waves' sums are added.  Lane: four columns of rows lane / 32 and 2 + lane / 32.
template <int HD, int ROWS, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void attention_cached_join_kernel(const CachedArgs g, int quads) {
  constexpr int C = HD / 4;                        // lanes of a row
  static_assert(C <= 32, "two rows a wave");
  __shared__ float tops[WAVES][4];
  __shared__ __align__(16) floatx4 sums[WAVES][4][C];
  __shared__ float totals[WAVES][4];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int parts = ROWS / 4 / quads, part = blockIdx.x % parts, rest = blockIdx.x / parts, head = rest % g.kv_heads, tile = rest / g.kv_heads;
  const int seq = packed_find(g.seqs, tile, g.group, ROWS, 0);
  int start, n;
  packed_rows(g.seqs, seq, &start, &n);
  const int64_t r0 = static_cast<int64_t>(tile - packed_first_tile(g.seqs, seq, g.group, ROWS, 0)) * ROWS, rows = static_cast<int64_t>(n) * g.group;
  if (r0 < 0 || r0 + part * quads * 4 >= rows) return;
  int splits;
  int64_t first, next;                             // slot of the first split, and what lies between the second's and the others'
  int64_t second;
  if constexpr (ROWS == 128) {
    const Stretch f = static_cast<const Stretch*>(g.shares)[seq];
    const int64_t place = static_cast<int64_t>(head) * f.tiles + place_in_line(static_cast<int>(r0 / ROWS), f.tiles, g.causal);
    if (f.splits) {
      splits = f.splits;
      first = f.from + place * splits;
      second = first + 1;
      next = 1;
      if (splits == 1 || first + splits > g.slots) return;
    } else {
      const int64_t at = f.from + place * (f.pages + kTileCost);
      const int64_t lo = (at + kLeastPart + f.per - 1) / f.per, hi = (at + f.pages - kLeastPart) / f.per;       // borders inside the tile
      if (hi < lo || 2 * hi >= g.slots) return;
      splits = static_cast<int>(hi - lo + 2);
      first = 2 * lo - 1;
      second = 2 * lo;
      next = 2;
    }
  } else {
    const Share f = static_cast<const Share*>(g.shares)[seq];
    if (f.splits == 1 || f.slot + static_cast<int64_t>(f.tiles) * f.splits * g.kv_heads > g.slots) return;
    splits = f.splits;
    first = f.slot + static_cast<int64_t>(head) * f.splits * f.tiles + r0 / ROWS;
    second = first + f.tiles;
    next = f.tiles;
  }
  auto slot_of = [&](int s) { return s == 0 ? first : second + (s - 1) * next; };
  for (int quad = part * quads; quad < (part + 1) * quads && r0 + quad * 4 < rows; ++quad) {
    auto stat = [&](int s, int which, int r) { return g.stats[(slot_of(s) * 2 + which) * ROWS + quad * 4 + r]; };

    float top = -INFINITY;                           // of row lane % 4, over the splits of this lane, then of all
    for (int s = tid >> 2; s < splits; s += 16 * WAVES) top = fmaxf(top, stat(s, 0, tid & 3));
    for (int off = 4; off < 64; off <<= 1) top = fmaxf(top, __shfl_xor(top, off, 64));
    if (lane < 4) tops[wave][lane] = top;
    __syncthreads();
    const int col = lane & 31;
    float m[2], off[2], total[2] = {};
    floatx4 v[2] = {};
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int r = 2 * half + (lane >> 5);
      m[half] = tops[0][r];
#pragma unroll
      for (int w = 1; w < WAVES; ++w) m[half] = fmaxf(m[half], tops[w][r]);
      off[half] = m[half] == -INFINITY ? 0.0f : m[half] * g.scale_log2e;
    }
#pragma unroll 8
    for (int s = wave; s < splits; s += WAVES)
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const int r = 2 * half + (lane >> 5);
        const float ms = stat(s, 0, r), l = stat(s, 1, r);
        const floatx4 x = *reinterpret_cast<const floatx4*>(g.part + (slot_of(s) * ROWS + quad * 4 + r) * HD + 4 * (col < C ? col : 0));
        // a split without a finite score has weight 0, unless all are so: then NaN where keys were seen, 0 elsewhere
        const float w = ms == -INFINITY ? (m[half] == -INFINITY ? 1.0f : 0.0f) : fast_exp2(ms * g.scale_log2e - off[half]);
        total[half] += ms == -INFINITY && w == 0.0f ? 0.0f : l * w;
        v[half] += x * w;
      }
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int r = 2 * half + (lane >> 5);
      if (col < C) sums[wave][r][col] = v[half];
      if (col == 0) totals[wave][r] = total[half];
    }
    __syncthreads();
    const int r = tid / C, c = tid - r * C;
    if (tid < 4 * C && r0 + quad * 4 + r < rows) {
      floatx4 v = sums[0][r][c];
      float total = totals[0][r];
#pragma unroll
      for (int w = 1; w < WAVES; ++w) {
        v += sums[w][r][c];
        total += totals[w][r];
      }
      const int64_t row = r0 + quad * 4 + r;
      const int tok = static_cast<int>(row / g.group), sub = static_cast<int>(row - static_cast<int64_t>(tok) * g.group);
      uint16_t* op = g.out + (static_cast<int64_t>(start) + tok) * g.ldo + (static_cast<int64_t>(head) * g.group + sub) * HD + 4 * c;
      const float inv = total == 0.0f ? 0.0f : 1.0f / total;
      const uint32_t a = cvt_pk_bf16(v[0] * inv, v[1] * inv), b = cvt_pk_bf16(v[2] * inv, v[3] * inv);
      if (g.wide) *reinterpret_cast<uint2*>(op) = make_uint2(a, b);
      else { op[0] = static_cast<uint16_t>(a); op[1] = static_cast<uint16_t>(a >> 16); op[2] = static_cast<uint16_t>(b); op[3] = static_cast<uint16_t>(b >> 16); }
    }
    __syncthreads();
  }
}

struct Plan {
  int rows;                         // of a tile
  int resident, least_pages;
  int64_t tiles, units;             // at most
  int64_t slots;                    // at most; 0: no sequence is long enough to be split
  int64_t part_bytes, stat_bytes, bytes;
};
Plan plan_of(int n_seqs, int total, int max_len, int heads, int kv_heads, int head_dim) {
  Plan p{};
  const int group = heads / kv_heads;
  const int64_t rows = static_cast<int64_t>(total) * group, mean = (rows + n_seqs - 1) / n_seqs, pages = (static_cast<int64_t>(max_len) + PAGE - 1) / PAGE;
  p.rows = mean <= 16 ? 16 : mean <= 32 || head_dim < 64 ? 32 : 128;
  p.tiles = rows / p.rows + n_seqs;
  p.resident = 2 * compute_units();
  // Fewer pages a unit spread a call over more blocks; what begins, ends and joins one costs as much as a few pages.  Few rows: 8 (33 tokens
  // of 13 sequences of up to 9756, 28 heads over 4: 20.9 us, 22.1 with 6, 23.9 with 4, 27.5 with 24), but no splits at all, and no second
  // launch, where no sequence can have more than 20 pages.  One token each, 32 heads over 8 of 128, us uncut / in splits of 8: one sequence of 16
  // pages 11.4 / 14.9, of 20 12.4 / 15.0, 21 13.0 / 15.2, 24 13.6 / 15.3, 32 16.3 / 14.9, 64 26.7 / 15.3; four of 20 13.4 / 15.0, 24 14.9 / 15.0, 32
  // 17.3 / 15.2, 128 48.9 / 21.7; sixteen, which fill half the chip, 20 14.7 / 18.8, 64 29.1 / 31.8, 128 50.7 / 51.7.  (The bound is max_len's, for
  // the host knows no lengths: a bound far above them costs the second launch, 11 to 15 us for short ones.)
  p.least_pages = p.rows == 128 ? kLeastPages : pages <= 20 ? 20 : 8;
  const int64_t whole = p.tiles * kv_heads;
  if (pages > p.least_pages) {
    p.slots = p.rows == 128 ? 2 * std::min<int64_t>(p.resident, (whole * (pages + kTileCost) + kLeastPages - 1) / kLeastPages)
                            : std::min<int64_t>(4 * p.resident, whole * ((pages + p.least_pages - 1) / p.least_pages));
    p.part_bytes = p.slots * p.rows * head_dim * static_cast<int64_t>(sizeof(float));
    p.stat_bytes = p.slots * 2 * p.rows * static_cast<int64_t>(sizeof(float));
    p.bytes = p.part_bytes + p.stat_bytes + n_seqs * static_cast<int64_t>(std::max(sizeof(Share), sizeof(Stretch)));
  }
  p.units = whole + p.slots;
  return p;
}

// Rows to join, four by four, and how many fours a block takes: one while that leaves the chip room, else 32 rows.
int64_t join_quads(const Plan& p, int kv_heads) { return p.tiles * kv_heads * (p.rows / 4); }
int join_each(const Plan& p, int kv_heads) { return join_quads(p, kv_heads) > 8 * p.resident ? std::min(p.rows / 4, 8) : 1; }

template <int HD, int ROWS>
void launch_join(const CachedArgs& g, const Plan& p, hipStream_t st) {
  if (!p.slots) return;
  const int64_t quads = join_quads(p, g.kv_heads);
  const int each = join_each(p, g.kv_heads);
  // Where few rows are joined, by 16 waves: a chain of waits, shorter the fewer splits a wave has (four tokens over 39 656, 28 heads over 4:
  // 29.5 -> 25.0 us).  With more rows than the chip holds such blocks 4 are better (6 tokens over up to 12 234, 24 heads: 27.6 us, 31.3).
  const unsigned blocks = static_cast<unsigned>(quads / each);
  if (quads <= p.resident) attention_cached_join_kernel<HD, ROWS, 16><<<blocks, 1024, 0, st>>>(g, each);
  else attention_cached_join_kernel<HD, ROWS, 4><<<blocks, 256, 0, st>>>(g, each);
}
template <int HD>
void launch_hd(const CachedArgs& g, const Plan& p, hipStream_t st) {
  const unsigned blocks = static_cast<unsigned>(std::min<int64_t>(p.units, p.resident));
  if (p.rows == 16) {
    attention_cached_kernel<HD, 1><<<blocks, 256, 0, st>>>(g);
    launch_join<HD, 16>(g, p, st);
  } else if (p.rows == 32) {
    attention_cached_kernel<HD, 2><<<blocks, 256, 0, st>>>(g);
    launch_join<HD, 32>(g, p, st);
  } else if constexpr (HD >= 64) {
    launch_attention_cached_tile(g, HD, blocks, st);
    launch_join<HD, 128>(g, p, st);
  }
}

bool sizes_ok(int n_seqs, int total, int max_len, int heads, int kv_heads, int head_dim) {
  return n_seqs >= 1 && total >= 0 && max_len >= 0 && max_len <= (1 << 30) && heads >= 1 && heads <= 65536 && kv_heads >= 1 && heads % kv_heads == 0 &&
         (head_dim == 16 || head_dim == 32 || head_dim == 64 || head_dim == 72 || head_dim == 128);
}

}  // namespace

int64_t attention_cached_workspace(int n_seqs, int total, int max_len, int heads, int kv_heads, int head_dim) {
  if (!sizes_ok(n_seqs, total, max_len, heads, kv_heads, head_dim)) return -1;
  return total == 0 ? 0 : plan_of(n_seqs, total, max_len, heads, kv_heads, head_dim).bytes;
}

Error launch_attention_cached(int dtype, const speca_kv_cache& c, const speca_kv_table& t, const CachedAttention& a, void* workspace,
                              int64_t workspace_bytes, hipStream_t st) {
  const char* who = "speca_attention_cached";
  if (dtype == SPECA_F32) SPECA_FAIL(SPECA_EUNSUPPORTED, "%s: bf16 only", who);
  if (dtype != SPECA_BF16) SPECA_FAIL(SPECA_EINVAL, "%s: dtype = %d", who, dtype);
  SPECA_TRY(check_kv_cache(who, c, t));
  if (!a.q || !a.out || !a.seqs.cu || !a.lens) SPECA_FAIL(SPECA_EINVAL, "%s: q, out, starts and lens must not be NULL", who);
  if (a.heads < 1 || a.heads > 65536 || a.heads % c.kv_heads) SPECA_FAIL(SPECA_EINVAL, "%s: %d heads over %d key heads", who, a.heads, c.kv_heads);
  if (!sizes_ok(a.seqs.n, a.seqs.total, a.max_len, a.heads, c.kv_heads, c.head_dim))
    SPECA_FAIL(SPECA_EINVAL, "%s: n_seqs = %d, total = %d, max_len = %d", who, a.seqs.n, a.seqs.total, a.max_len);
  const int64_t w = static_cast<int64_t>(a.heads) * c.head_dim, most = int64_t{1} << 40;
  if (a.ldq < w || a.ldo < w || a.ldq > most || a.ldo > most)
    SPECA_FAIL(SPECA_EINVAL, "%s: tokens %lld and %lld elements apart, heads need %lld", who, static_cast<long long>(a.ldq), static_cast<long long>(a.ldo), static_cast<long long>(w));
  const uintptr_t at = reinterpret_cast<uintptr_t>(a.q), to = reinterpret_cast<uintptr_t>(a.out);
  if (at % 2 || to % 2 || (reinterpret_cast<uintptr_t>(a.seqs.cu) | reinterpret_cast<uintptr_t>(a.lens)) % 4) SPECA_FAIL(SPECA_EINVAL, "%s: a pointer is not aligned to its type", who);
  if (!(a.scale >= 0.0f) || !std::isfinite(a.scale)) SPECA_FAIL(SPECA_EINVAL, "%s: scale = %g", who, a.scale);
  if (a.seqs.total == 0) return ok();
  const Plan p = plan_of(a.seqs.n, a.seqs.total, a.max_len, a.heads, c.kv_heads, c.head_dim);
  if (join_quads(p, c.kv_heads) > 0x7FFFFFFF || (p.slots && join_quads(p, c.kv_heads) / join_each(p, c.kv_heads) > kMaxBlocks))
    SPECA_FAIL(SPECA_EINVAL, "%s: %d tokens of %d heads are too many for one call", who, a.seqs.total, a.heads);
  if (p.bytes && (!workspace || workspace_bytes < p.bytes || reinterpret_cast<uintptr_t>(workspace) % 16))
    SPECA_FAIL(SPECA_EINVAL, "%s: a workspace of %lld bytes, 16-byte aligned, is needed (given: %lld)", who, static_cast<long long>(p.bytes), static_cast<long long>(workspace ? workspace_bytes : 0));
  CachedArgs g;
  g.k = static_cast<const uint8_t*>(c.k); g.v = static_cast<const uint8_t*>(c.v);
  g.k_scale = c.k_scale; g.v_scale = c.v_scale;
  g.q = static_cast<const uint16_t*>(a.q); g.out = static_cast<uint16_t*>(a.out);
  g.ldq = a.ldq; g.ldo = a.ldo;
  g.seqs = a.seqs;
  g.lens = a.lens; g.table = t.page;
  g.part = static_cast<float*>(workspace);
  g.stats = p.bytes ? reinterpret_cast<float*>(static_cast<char*>(workspace) + p.part_bytes) : nullptr;
  g.shares = p.bytes ? static_cast<char*>(workspace) + p.part_bytes + p.stat_bytes : nullptr;
  g.table_ld = t.ld; g.pages = c.pages; g.kv_heads = c.kv_heads; g.group = a.heads / c.kv_heads;
  g.max_len = static_cast<int>(std::min<int64_t>(a.max_len, static_cast<int64_t>(t.ld) * PAGE));
  g.resident = p.resident; g.least_pages = p.least_pages; g.slots = static_cast<int32_t>(p.slots);
  g.causal = a.causal;
  g.wide = at % 16 == 0 && a.ldq % 8 == 0 && to % 8 == 0 && a.ldo % 4 == 0;
  g.scale_log2e = 1.4426950408889634f * (a.scale == 0.0f ? 1.0f / std::sqrt(static_cast<float>(c.head_dim)) : a.scale);
  switch (c.head_dim) {
    case 16: launch_hd<16>(g, p, st); break;
    case 32: launch_hd<32>(g, p, st); break;
    case 64: launch_hd<64>(g, p, st); break;
    case 72: launch_hd<72>(g, p, st); break;
    default: launch_hd<128>(g, p, st); break;
  }
  SPECA_HIP(hipGetLastError());
  return ok();
}

}  // namespace speca
