// Launchers of the operators around attention that stand on their own (speca_rope_axes, speca_attention_packed, speca_kv_store,
// speca_kv_load, speca_attention_cached).  Each checks what its kernel and grid assume and enqueues on the given stream.
#pragma once

#include "common.h"

namespace speca {

// Blocks of 256 threads that one launch may have: fewer than 2^32 threads along a dimension.
constexpr int64_t kMaxBlocks = 0xFFFFFFFF / 256;

Error launch_rope_axes(int dtype, const speca_rope& rope, const int32_t* positions, int64_t tokens, int head_dim, float eps,
                       const speca_rope_io& q, const speca_rope_io* k, hipStream_t st);

// Sequences laid end to end: sequence s holds the rows cu[s] .. cu[s + 1] of `total` (cu on the device).
struct Packed {
  const int32_t* cu;
  int32_t n;
  int32_t total;
};

struct PackedAttention {
  const void *q, *k, *v;
  void* out;
  int64_t ldq, ldk, ldv, ldo;      // elements from one token to the next
  Packed seqs;
  int32_t heads, kv_heads, head_dim;
  bool causal;
  float scale;
};
Error launch_attention_packed(int dtype, const PackedAttention& a, hipStream_t st);
// The kernels behind it, arguments checked, scale given: bf16 tiles (attn_mfma.hip) where alignment and strides allow, the fp32 matrix
// instructions otherwise.
bool attention_packed_mfma_supported(const PackedAttention& a);
Error launch_attention_packed_mfma(const PackedAttention& a, hipStream_t st);
Error launch_attention_packed_f32(int dtype, const PackedAttention& a, hipStream_t st);

Error check_kv_cache(const char* who, const speca_kv_cache& c, const speca_kv_table& t);
Error launch_kv_store(int dtype, const speca_kv_cache& c, const speca_kv_table& t, const int32_t* past, const void* k, int64_t ldk,
                      const void* v, int64_t ldv, const Packed& seqs, hipStream_t st);
Error launch_kv_load(int dtype, const speca_kv_cache& c, const speca_kv_table& t, const int32_t* first, void* k, int64_t ldk, void* v,
                     int64_t ldv, const Packed& seqs, hipStream_t st);

struct CachedAttention {
  const void* q;
  void* out;
  int64_t ldq, ldo;
  Packed seqs;                     // the new tokens
  const int32_t* lens;             // tokens in the cache
  int32_t max_len;                 // none is longer
  int32_t heads;
  bool causal;
  float scale;
};
int64_t attention_cached_workspace(int n_seqs, int total, int max_len, int heads, int kv_heads, int head_dim);      // -1: no valid sizes
Error launch_attention_cached(int dtype, const speca_kv_cache& c, const speca_kv_table& t, const CachedAttention& a, void* workspace,
                              int64_t workspace_bytes, hipStream_t st);

// ---- device side ------------------------------------------------------------------------------------------------------

// Rows of sequence s, as far as the buffer goes: offsets that are no offsets read nothing outside it.
__device__ inline void packed_rows(const Packed& p, int s, int* start, int* len) {
  const int a = p.cu[s], b = p.cu[s + 1];
  *start = a < 0 ? 0 : a < p.total ? a : p.total;
  const int e = b < *start ? *start : b < p.total ? b : p.total;
  *len = e - *start;
}

// A grid of rows / tile + n tiles has room for every sequence's own tiles, and where a sequence's tiles begin follows from its offset
// alone: tile t belongs to the last sequence with cu[s] * mul / tile + s <= t.  So the host needs no lengths, and a block finds its place
// in one or two rounds of 64 offsets at a time.  `extra`: tiles that a sequence may need beyond ceil(rows / tile).
__device__ inline int packed_first_tile(const Packed& p, int s, int mul, int tile, int extra) {
  int a = p.cu[s];
  a = a < 0 ? 0 : a < p.total ? a : p.total;
  return static_cast<int>(static_cast<int64_t>(a) * mul / tile) + s * (1 + extra);
}
__device__ inline int packed_find(const Packed& p, int t, int mul, int tile, int extra) {
  const int lane = threadIdx.x & 63;
  int lo = 0, size = p.n;
  while (size > 1) {
    const int step = (size + 63) / 64, i = lo + lane * step;
    const bool below = lane * step < size && packed_first_tile(p, i, mul, tile, extra) <= t;
    const int n = __popcll(__ballot(below));          // offsets rise, so the ones at or below t come first
    if (n == 0) return lo;
    lo += (n - 1) * step;
    size = size - (n - 1) * step < step ? size - (n - 1) * step : step;
  }
  return __builtin_amdgcn_readfirstlane(lo);
}
inline int64_t packed_tiles(const Packed& p, int mul, int tile, int extra) {
  return static_cast<int64_t>(p.total) * mul / tile + static_cast<int64_t>(p.n) * (1 + extra);
}

}  // namespace speca
