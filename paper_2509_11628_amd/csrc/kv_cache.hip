// Keys and values in 8 bits: storing packed tokens into pages, and reading them back.
//
// A page holds 64 tokens of one head under one scale 2^e, the smallest with amax <= 448 * 2^e over what was stored.  e follows from the bits
// of amax: 448 = 1.75 * 2^8, so e = exponent(amax) - 8, and one more where the mantissa is above 1.75.
//
// A page and head is one block's, for keys and for values each: amax needs all of its new tokens, and the bytes that stay need the old scale.
// Bound by memory and by the chain of waits of one block (place, tokens, maximum, bytes).  Storing 2512 tokens of 24 heads of 128 in bf16
// takes 15 us, loading them back 11 (46 MB each way); 16 single tokens of 8 heads 6 and 4.  One value per thread at a time took 51 and 30,
// 14 and 12.  In fp32 17 and 46 us (78 MB each way; a row's two halves of 16 bytes go out one after the other), 6 and 7.
#include "operators.h"

namespace speca {

namespace {

constexpr int PAGE = SPECA_KV_PAGE;
constexpr int kLowest = -100, kHighest = 119;       // of e; 448 * 2^119 is the largest that fp32 holds

// eight values at 16- (fp32) or 16-byte (bf16) boundaries, or one at a time
__device__ inline void ld8(const float* p, bool wide, float (&v)[8]) {
  if (wide) {
    const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = p[i];
  }
}
__device__ inline void ld8(const bf16_t* p, bool wide, float (&v)[8]) {
  if (wide) {
    const uint4 a = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(w[i] << 16); v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u); }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = bf16_to_f32(p[i].bits);
  }
}
__device__ inline void st8(float* p, bool wide, const float (&v)[8]) {
  if (wide) {
    *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
    *reinterpret_cast<float4*>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) p[i] = v[i];
  }
}
// (e4m3 x 2^e is a bf16 value: its upper half is all of it)
__device__ inline void st8(bf16_t* p, bool wide, const float (&v)[8]) {
  if (wide) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __float_as_uint(v[2 * i]) >> 16 | (__float_as_uint(v[2 * i + 1]) & 0xFFFF0000u);
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) p[i].bits = static_cast<uint16_t>(__float_as_uint(v[i]) >> 16);
  }
}

__device__ inline float power(int e) { return __uint_as_float(static_cast<uint32_t>(e + 127) << 23); }
__device__ inline int scale_exponent(uint32_t amax_bits) {          // of a finite value >= 0
  const int e = static_cast<int>(amax_bits >> 23) - 127 - 8 + ((amax_bits & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return amax_bits == 0 || e < kLowest ? kLowest : e > kHighest ? kHighest : e;
}
// Four values to e4m3, nearest even; they are scaled already.  The conversion makes NaN of what lies beyond 448, so that is cut off first;
// NaN passes the comparisons.
__device__ inline float cut(float v) { return v > 448.0f ? 448.0f : v < -448.0f ? -448.0f : v; }
__device__ inline uint32_t encode4(float a, float b, float c, float d) {
  const int low = __builtin_amdgcn_cvt_pk_fp8_f32(cut(a), cut(b), 0, false);
  return __builtin_amdgcn_cvt_pk_fp8_f32(cut(c), cut(d), low, true);
}
__device__ inline void decode4(uint32_t w, float s, float* v) {
  v[0] = __builtin_amdgcn_cvt_f32_fp8(w, 0) * s;
  v[1] = __builtin_amdgcn_cvt_f32_fp8(w, 1) * s;
  v[2] = __builtin_amdgcn_cvt_f32_fp8(w, 2) * s;
  v[3] = __builtin_amdgcn_cvt_f32_fp8(w, 3) * s;
}
// the bytes of a word whose tokens t .. t + 3 lie in [lo, hi)
__device__ inline uint32_t bytes_between(int t, int lo, int hi) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) m |= t + i >= lo && t + i < hi ? 0xFFu << (8 * i) : 0u;
  return m;
}

struct Args {
  uint8_t *k, *v;
  float *k_scale, *v_scale;
  int32_t pages, heads, hd;
  const int32_t* table;
  int32_t table_ld;
  const int32_t* from;              // first token in the cache of each sequence's run
  void *x, *y;                      // packed k and v
  int64_t ldx, ldy;
  Packed seqs;
  bool wide_x, wide_y;              // eight features of a token lie at whole 16 bytes
};

// Where a block works: page `page` of the cache (or < 0: nothing to do), whose places [lo, hi) are the rows row .. of the packed tensors.
struct Place {
  int page, lo, hi;
  int64_t row;
};
__device__ inline Place find_place(const Args& g, int tile) {
  Place p{-1, 0, 0, 0};
  const int seq = packed_find(g.seqs, tile, 1, PAGE, 1);
  int start, n;
  packed_rows(g.seqs, seq, &start, &n);
  const int j = tile - packed_first_tile(g.seqs, seq, 1, PAGE, 1);              // j-th page that the run touches
  const int64_t from = g.from[seq], first = from / PAGE + j, end = from + n;
  if (from < 0 || j < 0 || n == 0 || first * PAGE >= end) return p;
  p.lo = first * PAGE < from ? static_cast<int>(from - first * PAGE) : 0;
  p.hi = end - first * PAGE < PAGE ? static_cast<int>(end - first * PAGE) : PAGE;
  p.row = start + first * PAGE + p.lo - from;
  p.page = first < g.table_ld ? g.table[static_cast<int64_t>(seq) * g.table_ld + first] : -2;
  if (p.page < 0 || p.page >= g.pages) p.page = -2;                             // not held
  return p;
}

// One block: the keys (blockIdx.y == 0) or values of one head of one page.  A thread has four consecutive tokens of eight features, which are
// four consecutive bytes of eight rows of a value page; threads next to each other go along the page's rows (features of keys, tokens of
// values).
struct Unit {
  int t, d;                         // first token of the page, first feature
  bool live;
};
__device__ inline Unit unit_of(bool values, int hd) {
  const int u = threadIdx.x, ch = hd / 8;
  Unit x;
  x.live = u < 16 * ch;
  const int group = values ? u & 15 : u / ch;
  x.d = 8 * (values ? u >> 4 : u - group * ch);
  // values: the word at place 16 g + 4 m holds tokens 16 m + 4 g ..
  x.t = values ? 16 * (group & 3) + 4 * (group >> 2) : 4 * group;
  return x;
}

template <typename T>
__global__ __launch_bounds__(256) void kv_store_kernel(const Args g) {
  const int head = blockIdx.x % g.heads;
  const Place p = find_place(g, blockIdx.x / g.heads);
  if (p.page < 0) return;
  const bool values = blockIdx.y != 0, wide = values ? g.wide_y : g.wide_x;
  const int64_t at = static_cast<int64_t>(p.page) * g.heads + head;
  uint8_t* page = (values ? g.v : g.k) + at * PAGE * g.hd;
  float* scale = (values ? g.v_scale : g.k_scale) + at;
  const int64_t ld = values ? g.ldy : g.ldx;
  const Unit u = unit_of(values, g.hd);
  const T* x = static_cast<const T*>(values ? g.y : g.x) + p.row * ld + static_cast<int64_t>(head) * g.hd + u.d;
  const float old = p.lo > 0 ? *scale : 0.0f;

  float v[4][8];
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int t = u.t + i;
    if (u.live && t >= p.lo && t < p.hi) {
      ld8(x + (t - p.lo) * ld, wide, v[i]);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] = 0.0f;
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t b = __float_as_uint(v[i][j]) & 0x7FFFFFFFu;
      if (b < 0x7F800000u && b > top) top = b;
    }
  __shared__ uint32_t tops[4];
  for (int off = 32; off; off >>= 1) {
    const uint32_t o = __shfl_xor(top, off, 64);
    top = o > top ? o : top;
  }
  if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = top;
  __syncthreads();                                   // (and everybody has read the old scale)
  top = max(max(tops[0], tops[1]), max(tops[2], tops[3]));
  float s = power(scale_exponent(top));
  if (old > s) s = old;
  if (threadIdx.x == 0) *scale = s;
  const float inv = 1.0f / s, again = old / s;
  // tokens that were there stay as they are unless the scale rises
  if (!u.live || (u.t + 4 <= p.lo && again == 1.0f)) return;
  const uint32_t keep = bytes_between(u.t, 0, p.lo);
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) v[i][j] *= inv;
  auto kept = [&](uint32_t w) {
    if (again == 1.0f) return w;
    float f[4];
    decode4(w, again, f);
    return encode4(f[0], f[1], f[2], f[3]);
  };
  if (values) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      uint32_t* to = reinterpret_cast<uint32_t*>(page + (u.d + j) * PAGE + 16 * (u.t >> 2 & 3) + 4 * (u.t >> 4));
      uint32_t w = encode4(v[0][j], v[1][j], v[2][j], v[3][j]) & ~keep;
      if (keep) w |= kept(*to) & keep;
      *to = w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint2* to = reinterpret_cast<uint2*>(page + (u.t + i) * g.hd + u.d);
      if (keep >> (8 * i) & 1) {
        if (again == 1.0f) continue;
        const uint2 w = *to;
        *to = make_uint2(kept(w.x), kept(w.y));
      } else {
        *to = make_uint2(encode4(v[i][0], v[i][1], v[i][2], v[i][3]), encode4(v[i][4], v[i][5], v[i][6], v[i][7]));
      }
    }
  }
}

template <typename T>
__global__ __launch_bounds__(256) void kv_load_kernel(const Args g) {
  const int head = blockIdx.x % g.heads;
  const Place p = find_place(g, blockIdx.x / g.heads);
  if (p.page == -1) return;
  const bool values = blockIdx.y != 0, wide = values ? g.wide_y : g.wide_x, held = p.page >= 0;
  const int64_t at = static_cast<int64_t>(held ? p.page : 0) * g.heads + head;
  const uint8_t* page = (values ? g.v : g.k) + at * PAGE * g.hd;
  const int64_t ld = values ? g.ldy : g.ldx;
  const Unit u = unit_of(values, g.hd);
  if (!u.live || u.t + 4 <= p.lo || u.t >= p.hi) return;
  const float s = (values ? g.v_scale : g.k_scale)[at];
  T* x = static_cast<T*>(values ? g.y : g.x) + p.row * ld + static_cast<int64_t>(head) * g.hd + u.d;
  float v[4][8] = {};
  if (held) {
    if (values) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        float f[4];
        decode4(*reinterpret_cast<const uint32_t*>(page + (u.d + j) * PAGE + 16 * (u.t >> 2 & 3) + 4 * (u.t >> 4)), s, f);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i][j] = f[i];
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint2 w = *reinterpret_cast<const uint2*>(page + (u.t + i) * g.hd + u.d);
        decode4(w.x, s, v[i]);
        decode4(w.y, s, v[i] + 4);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (u.t + i >= p.lo && u.t + i < p.hi) st8(x + (u.t + i - p.lo) * ld, wide, v[i]);
}

Error check(const char* who, int dtype, const speca_kv_cache& c, const speca_kv_table& t, const void* from, const void* k, int64_t ldk,
            const void* v, int64_t ldv, const Packed& seqs) {
  if (dtype != SPECA_F32 && dtype != SPECA_BF16) SPECA_FAIL(SPECA_EINVAL, "%s: dtype = %d", who, dtype);
  SPECA_TRY(check_kv_cache(who, c, t));
  if (!from || !k || !v || !seqs.cu) SPECA_FAIL(SPECA_EINVAL, "%s: k, v, starts and the first tokens must not be NULL", who);
  if (seqs.n < 1 || seqs.total < 0) SPECA_FAIL(SPECA_EINVAL, "%s: n_seqs = %d, total = %d", who, seqs.n, seqs.total);
  const int64_t w = static_cast<int64_t>(c.kv_heads) * c.head_dim, most = int64_t{1} << 40;
  if (ldk < w || ldv < w || ldk > most || ldv > most)
    SPECA_FAIL(SPECA_EINVAL, "%s: tokens %lld and %lld elements apart, heads need %lld", who, static_cast<long long>(ldk), static_cast<long long>(ldv), static_cast<long long>(w));
  if ((reinterpret_cast<uintptr_t>(k) | reinterpret_cast<uintptr_t>(v)) % dtype_size(dtype) || (reinterpret_cast<uintptr_t>(from) | reinterpret_cast<uintptr_t>(seqs.cu)) % 4)
    SPECA_FAIL(SPECA_EINVAL, "%s: a pointer is not aligned to its type", who);
  return ok();
}

Args make_args(int dtype, const speca_kv_cache& c, const speca_kv_table& t, const int32_t* from, void* k, int64_t ldk, void* v, int64_t ldv, const Packed& seqs) {
  const int64_t esz = static_cast<int64_t>(dtype_size(dtype));
  const bool wide_k = (reinterpret_cast<uintptr_t>(k) | static_cast<uintptr_t>(ldk * esz)) % 16 == 0, wide_v = (reinterpret_cast<uintptr_t>(v) | static_cast<uintptr_t>(ldv * esz)) % 16 == 0;
  return {static_cast<uint8_t*>(c.k), static_cast<uint8_t*>(c.v), c.k_scale, c.v_scale, c.pages, c.kv_heads, c.head_dim, t.page, t.ld, from, k, v, ldk, ldv, seqs, wide_k, wide_v};
}

Error grid_of(const char* who, const Args& g, dim3* grid) {
  const int64_t blocks = packed_tiles(g.seqs, 1, PAGE, 1) * g.heads;
  if (blocks > kMaxBlocks) SPECA_FAIL(SPECA_EINVAL, "%s: %d tokens of %d heads are too many for one call", who, g.seqs.total, g.heads);
  *grid = dim3(static_cast<unsigned>(blocks), 2);
  return ok();
}

}  // namespace

Error check_kv_cache(const char* who, const speca_kv_cache& c, const speca_kv_table& t) {
  if (!c.k || !c.v || !c.k_scale || !c.v_scale || !t.page) SPECA_FAIL(SPECA_EINVAL, "%s: the cache's tensors and the table must not be NULL", who);
  if (c.pages < 1 || c.kv_heads < 1 || c.kv_heads > 65536 || t.ld < 1) SPECA_FAIL(SPECA_EINVAL, "%s: %d pages, %d key heads, table rows of %d", who, c.pages, c.kv_heads, t.ld);
  if (c.head_dim != 16 && c.head_dim != 32 && c.head_dim != 64 && c.head_dim != 72 && c.head_dim != 128)
    SPECA_FAIL(SPECA_EUNSUPPORTED, "%s: head_dim %d (supported: 16, 32, 64, 72, 128)", who, c.head_dim);
  if ((reinterpret_cast<uintptr_t>(c.k) | reinterpret_cast<uintptr_t>(c.v)) % 16) SPECA_FAIL(SPECA_EINVAL, "%s: pages must be 16-byte aligned", who);
  if ((reinterpret_cast<uintptr_t>(c.k_scale) | reinterpret_cast<uintptr_t>(c.v_scale) | reinterpret_cast<uintptr_t>(t.page)) % 4)
    SPECA_FAIL(SPECA_EINVAL, "%s: a pointer is not aligned to its type", who);
  return ok();
}

Error launch_kv_store(int dtype, const speca_kv_cache& c, const speca_kv_table& t, const int32_t* past, const void* k, int64_t ldk,
                      const void* v, int64_t ldv, const Packed& seqs, hipStream_t st) {
  SPECA_TRY(check("speca_kv_store", dtype, c, t, past, k, ldk, v, ldv, seqs));
  if (seqs.total == 0) return ok();
  const Args g = make_args(dtype, c, t, past, const_cast<void*>(k), ldk, const_cast<void*>(v), ldv, seqs);
  dim3 grid;
  SPECA_TRY(grid_of("speca_kv_store", g, &grid));
  if (dtype == SPECA_BF16) kv_store_kernel<bf16_t><<<grid, 256, 0, st>>>(g);
  else kv_store_kernel<float><<<grid, 256, 0, st>>>(g);
  SPECA_HIP(hipGetLastError());
  return ok();
}

Error launch_kv_load(int dtype, const speca_kv_cache& c, const speca_kv_table& t, const int32_t* first, void* k, int64_t ldk, void* v,
                     int64_t ldv, const Packed& seqs, hipStream_t st) {
  SPECA_TRY(check("speca_kv_load", dtype, c, t, first, k, ldk, v, ldv, seqs));
  if (seqs.total == 0) return ok();
  const Args g = make_args(dtype, c, t, first, k, ldk, v, ldv, seqs);
  dim3 grid;
  SPECA_TRY(grid_of("speca_kv_load", g, &grid));
  if (dtype == SPECA_BF16) kv_load_kernel<bf16_t><<<grid, 256, 0, st>>>(g);
  else kv_load_kernel<float><<<grid, 256, 0, st>>>(g);
  SPECA_HIP(hipGetLastError());
  return ok();
}

}  // namespace speca
