// Attention inside each of several packed sequences: arguments, and which kernel takes them.
#include <cmath>

#include "operators.h"

namespace speca {

Error launch_attention_packed(int dtype, const PackedAttention& given, hipStream_t st) {
  PackedAttention a = given;
  const char* who = "speca_attention_packed";
  if (dtype != SPECA_F32 && dtype != SPECA_BF16) SPECA_FAIL(SPECA_EINVAL, "%s: dtype = %d", who, dtype);
  if (!a.q || !a.k || !a.v || !a.out || !a.seqs.cu) SPECA_FAIL(SPECA_EINVAL, "%s: q, k, v, out and starts must not be NULL", who);
  if (a.seqs.n < 1 || a.seqs.total < 0) SPECA_FAIL(SPECA_EINVAL, "%s: n_seqs = %d, total = %d", who, a.seqs.n, a.seqs.total);
  if (a.heads < 1 || a.kv_heads < 1 || a.heads > 65536 || a.heads % a.kv_heads) SPECA_FAIL(SPECA_EINVAL, "%s: %d heads over %d key heads", who, a.heads, a.kv_heads);
  if (a.head_dim != 16 && a.head_dim != 32 && a.head_dim != 64 && a.head_dim != 72 && a.head_dim != 128)
    SPECA_FAIL(SPECA_EUNSUPPORTED, "%s: head_dim %d (supported: 16, 32, 64, 72, 128)", who, a.head_dim);
  const int64_t wq = static_cast<int64_t>(a.heads) * a.head_dim, wk = static_cast<int64_t>(a.kv_heads) * a.head_dim, most = int64_t{1} << 40;
  if (a.ldq < wq || a.ldo < wq || a.ldk < wk || a.ldv < wk || a.ldq > most || a.ldo > most || a.ldk > most || a.ldv > most)
    SPECA_FAIL(SPECA_EINVAL, "%s: tokens %lld, %lld, %lld and %lld elements apart, heads need %lld and %lld", who, static_cast<long long>(a.ldq),
               static_cast<long long>(a.ldk), static_cast<long long>(a.ldv), static_cast<long long>(a.ldo), static_cast<long long>(wq), static_cast<long long>(wk));
  if ((reinterpret_cast<uintptr_t>(a.q) | reinterpret_cast<uintptr_t>(a.k) | reinterpret_cast<uintptr_t>(a.v) | reinterpret_cast<uintptr_t>(a.out)) % dtype_size(dtype) ||
      reinterpret_cast<uintptr_t>(a.seqs.cu) % 4)
    SPECA_FAIL(SPECA_EINVAL, "%s: a pointer is not aligned to its type", who);
  if (!(a.scale >= 0.0f) || !std::isfinite(a.scale)) SPECA_FAIL(SPECA_EINVAL, "%s: scale = %g", who, a.scale);
  if (a.seqs.total == 0) return ok();
  if (a.scale == 0.0f) a.scale = 1.0f / std::sqrt(static_cast<float>(a.head_dim));
  if (dtype == SPECA_BF16 && attention_packed_mfma_supported(a)) return launch_attention_packed_mfma(a, st);
  return launch_attention_packed_f32(dtype, a, st);
}

}  // namespace speca
