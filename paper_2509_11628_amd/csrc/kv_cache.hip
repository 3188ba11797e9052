// Keys and values in 8 bits: storing packed tokens into pages, and reading them back.
//
// A page holds 64 tokens of one head under one scale 2^e, the smallest with amax <= 448 * 2^e over what was stored.  e follows from the bits
// of amax: 448 = 1.75 * 2^8, so e = exponent(amax) - 8, and one more where the mantissa is above 1.75.
#include "operators.h"

namespace speca {

namespace {

constexpr int PAGE = SPECA_KV_PAGE;
constexpr int kLowest = -100, kHighest = 119;       // of e; 448 * 2^119 is the largest that fp32 holds

__device__ inline float ld_f32(const float* p) { return *p; }
__device__ inline float ld_f32(const bf16_t* p) { return bf16_to_f32(p->bits); }
__device__ inline void st_f32(float* p, float v) { *p = v; }
__device__ inline void st_f32(bf16_t* p, float v) { p->bits = static_cast<uint16_t>(__float_as_uint(v) >> 16); }       // e4m3 x 2^e: exact

__device__ inline float power(int e) { return __uint_as_float(static_cast<uint32_t>(e + 127) << 23); }
__device__ inline int scale_exponent(uint32_t amax_bits) {          // of a finite value >= 0
  const int e = static_cast<int>(amax_bits >> 23) - 127 - 8 + ((amax_bits & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return amax_bits == 0 || e < kLowest ? kLowest : e > kHighest ? kHighest : e;
}
// to e4m3, nearest even; v is scaled already.  The conversion makes NaN of what lies beyond 448, so that is cut off first; NaN passes the
// comparisons.
__device__ inline uint8_t encode(float v) {
  v = v > 448.0f ? 448.0f : v < -448.0f ? -448.0f : v;
  return static_cast<uint8_t>(__builtin_amdgcn_cvt_pk_fp8_f32(v, v, 0, false));
}
__device__ inline float decode(uint8_t b) { return __builtin_amdgcn_cvt_f32_fp8(b, 0); }

// place of token t of a page in a row of the value page
__device__ inline int value_place(int t) { return 16 * ((t >> 2) & 3) + 4 * (t >> 4) + (t & 3); }

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

// One block: the keys (blockIdx.y == 0) or values of one head of one page.
template <typename T>
__global__ __launch_bounds__(256) void kv_store_kernel(const Args g) {
  const int head = blockIdx.x % g.heads;
  const Place p = find_place(g, blockIdx.x / g.heads);
  if (p.page < 0) return;
  const bool values = blockIdx.y != 0;
  const int64_t unit = static_cast<int64_t>(p.page) * g.heads + head;
  uint8_t* page = (values ? g.v : g.k) + unit * PAGE * g.hd;
  float* scale = (values ? g.v_scale : g.k_scale) + unit;
  const int64_t ld = values ? g.ldy : g.ldx;
  const T* x = static_cast<const T*>(values ? g.y : g.x) + p.row * ld + static_cast<int64_t>(head) * g.hd;
  const int n = (p.hi - p.lo) * g.hd;

  uint32_t top = 0;
  for (int i = threadIdx.x; i < n; i += 256) {
    const int t = i / g.hd, d = i - t * g.hd;
    const uint32_t b = __float_as_uint(ld_f32(x + t * ld + d)) & 0x7FFFFFFFu;
    if (b < 0x7F800000u && b > top) top = b;
  }
  __shared__ uint32_t tops[4];
  for (int off = 32; off; off >>= 1) {
    const uint32_t o = __shfl_xor(top, off, 64);
    top = o > top ? o : top;
  }
  if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = top;
  __syncthreads();
  top = max(max(tops[0], tops[1]), max(tops[2], tops[3]));
  float s = power(scale_exponent(top));
  const float old = p.lo > 0 ? *scale : 0.0f;
  if (old > s) s = old;
  const float inv = 1.0f / s, again = old / s;
  __syncthreads();                                   // everybody has read the old scale
  for (int i = threadIdx.x; i < PAGE * g.hd; i += 256) {
    int t, d;
    if (values) {
      d = i / PAGE;
      const int at = i - d * PAGE;
      t = 16 * ((at >> 2) & 3) + 4 * (at >> 4) + (at & 3);      // value_place turned round: the two fields of two bits change places
    } else {
      t = i / g.hd;
      d = i - t * g.hd;
    }
    uint8_t b = 0;
    if (t < p.lo) {
      if (again == 1.0f) continue;
      b = encode(decode(page[i]) * again);
    } else if (t < p.hi) {
      b = encode(ld_f32(x + (t - p.lo) * ld + d) * inv);
    }
    page[i] = b;
  }
  if (threadIdx.x == 0) *scale = s;
}

template <typename T>
__global__ __launch_bounds__(256) void kv_load_kernel(const Args g) {
  const int head = blockIdx.x % g.heads;
  const Place p = find_place(g, blockIdx.x / g.heads);
  if (p.page == -1) return;
  const bool values = blockIdx.y != 0;
  const int64_t unit = static_cast<int64_t>(p.page) * g.heads + head;
  const uint8_t* page = (values ? g.v : g.k) + unit * PAGE * g.hd;
  const float s = p.page < 0 ? 0.0f : (values ? g.v_scale : g.k_scale)[unit];
  const int64_t ld = values ? g.ldy : g.ldx;
  T* x = static_cast<T*>(values ? g.y : g.x) + p.row * ld + static_cast<int64_t>(head) * g.hd;
  for (int i = threadIdx.x; i < (p.hi - p.lo) * g.hd; i += 256) {
    const int t = i / g.hd, d = i - t * g.hd;
    float v = 0.0f;
    if (p.page >= 0) v = decode(page[values ? d * PAGE + value_place(p.lo + t) : (p.lo + t) * g.hd + d]) * s;
    st_f32(x + t * ld + d, v);
  }
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

Args make_args(const speca_kv_cache& c, const speca_kv_table& t, const int32_t* from, void* k, int64_t ldk, void* v, int64_t ldv, const Packed& seqs) {
  return {static_cast<uint8_t*>(c.k), static_cast<uint8_t*>(c.v), c.k_scale, c.v_scale, c.pages, c.kv_heads, c.head_dim, t.page, t.ld, from, k, v, ldk, ldv, seqs};
}

Error grid_of(const char* who, const Args& g, dim3* grid) {
  const int64_t blocks = packed_tiles(g.seqs, 1, PAGE, 1) * g.heads;
  if (blocks > 0x7FFFFFFF) SPECA_FAIL(SPECA_EINVAL, "%s: %d tokens of %d heads are too many for one call", who, g.seqs.total, g.heads);
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
  const Args g = make_args(c, t, past, const_cast<void*>(k), ldk, const_cast<void*>(v), ldv, seqs);
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
  const Args g = make_args(c, t, first, k, ldk, v, ldv, seqs);
  dim3 grid;
  SPECA_TRY(grid_of("speca_kv_load", g, &grid));
  if (dtype == SPECA_BF16) kv_load_kernel<bf16_t><<<grid, 256, 0, st>>>(g);
  else kv_load_kernel<float><<<grid, 256, 0, st>>>(g);
  SPECA_HIP(hipGetLastError());
  return ok();
}

}  // namespace speca
