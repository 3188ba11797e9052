// Attention of packed sequences on the fp32 matrix instructions: fp32 tensors, and bf16 ones that the bf16 kernel does not take.
//
// One block = 16 QT queries of one (sequence, head); its four waves take the 16-key tiles w, w + 4, ... with an online softmax of their own
// and merge at the end.  Transposed products: S^T[key][query] leaves lane l with keys 4 (l / 16) .. + 3 of query l % 16, which is the
// second operand of the O^T product as it stands (instruction r takes keys 4 q + r).  The head dimension is dealt to the 16-row tiles of
// O^T in pieces of four (tile i % 4 of group i / 4 owns dimensions 64 g + 4 row + i), so a lane's values are 16-byte pieces of V and of the
// output. T = storage type of q, k, v and the output; arithmetic is fp32.
//
// What bounds it: issue, not memory.  Sequences of 1024, 77, 777 and 256 tokens, 6 heads of 64: 38 us, 69 TFLOP/s.  The matrix unit is busy
// for 54 % of a block's life and the vector unit for 36 %; waves spend 65 % of theirs waiting for their turn at them and 18 % for data; with
// every key and value from a wave's first four tiles, which then lie in its cache, the time is the same.  The 804 blocks leave some units
// four where others have three.  The exponential is the hardware's instruction alone, off by about a unit in the last place.
#include "attn_lane.h"
#include "operators.h"

namespace speca {

namespace {


__device__ __forceinline__ floatx4 mfma4(float a, float b, floatx4 c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }
template <bool WIDE>
__device__ inline floatx4 ld_quad(const float* p) {
  if constexpr (WIDE) return *reinterpret_cast<const floatx4*>(p);
  return floatx4{p[0], p[1], p[2], p[3]};
}
template <bool WIDE>
__device__ inline floatx4 ld_quad(const bf16_t* p) {
  if constexpr (WIDE) {
    const uint2 f = *reinterpret_cast<const uint2*>(p);
    return floatx4{__uint_as_float(f.x << 16), __uint_as_float(f.x & 0xFFFF0000u), __uint_as_float(f.y << 16), __uint_as_float(f.y & 0xFFFF0000u)};
  }
  return floatx4{bf16_to_f32(p[0].bits), bf16_to_f32(p[1].bits), bf16_to_f32(p[2].bits), bf16_to_f32(p[3].bits)};
}
__device__ inline float ld_one(const float* p) { return *p; }
__device__ inline float ld_one(const bf16_t* p) { return bf16_to_f32(p->bits); }
template <bool WIDE>
__device__ inline void st_quad(float* p, floatx4 v) {
  if constexpr (WIDE) *reinterpret_cast<floatx4*>(p) = v;
  else { p[0] = v[0]; p[1] = v[1]; p[2] = v[2]; p[3] = v[3]; }
}
template <bool WIDE>
__device__ inline void st_quad(bf16_t* p, floatx4 v) {
  const uint32_t a = cvt_pk_bf16(v[0], v[1]), b = cvt_pk_bf16(v[2], v[3]);
  if constexpr (WIDE) *reinterpret_cast<uint2*>(p) = make_uint2(a, b);
  else {
    p[0].bits = static_cast<uint16_t>(a); p[1].bits = static_cast<uint16_t>(a >> 16);
    p[2].bits = static_cast<uint16_t>(b); p[3].bits = static_cast<uint16_t>(b >> 16);
  }
}
__device__ inline bool finite(float v) { return (__float_as_uint(v) & 0x7F800000u) != 0x7F800000u; }

struct Args {
  PackedAttention a;
  int32_t group;            // query heads of a key head
  float scale_log2e;
};

// WIDE: every quad of a head lies at a whole quad (16 bytes in fp32, 8 in bf16).
template <typename T, int HD, int QT, bool CAUSAL, bool WIDE>
__global__ __launch_bounds__(256) void attention_packed_f32_kernel(const Args g) {
  constexpr int KS = (HD + 15) / 16;              // steps of 16 dimensions in q k^T
  constexpr int G = HD / 64;                      // groups of four tiles of O^T (64 dimensions)
  constexpr int REM = HD - 64 * G;                // what is left: 8, 16 or 32 dimensions in tiles of 16
  constexpr int RT = (REM + 15) / 16;
  constexpr int DT = 4 * G + RT;
  static_assert(HD % 8 == 0 && (REM == 0 || REM == 8 || REM == 16 || REM == 32), "head_dim");
  constexpr int OST = 16 * DT + 4;                // floats per query in the merge buffer
  __shared__ __align__(16) float merge[3][16 * OST];
  __shared__ float stats[4][2][16];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l16 = lane & 15, g4 = lane >> 4;
  const int head = blockIdx.x % g.a.heads, tile = blockIdx.x / g.a.heads;
  const int seq = packed_find(g.a.seqs, tile, 1, 16 * QT, 0);
  int start, n;
  packed_rows(g.a.seqs, seq, &start, &n);
  const int q0 = (tile - packed_first_tile(g.a.seqs, seq, 1, 16 * QT, 0)) * 16 * QT;
  if (q0 < 0 || q0 >= n) return;
  const float scale_log2e = g.scale_log2e;
  const T* qb = static_cast<const T*>(g.a.q) + start * g.a.ldq + head * HD;
  const T* kb = static_cast<const T*>(g.a.k) + start * g.a.ldk + head / g.group * HD;
  const T* vb = static_cast<const T*>(g.a.v) + start * g.a.ldv + head / g.group * HD;
  const floatx4 zero = {0.f, 0.f, 0.f, 0.f};

  floatx4 qf[QT][KS];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const int q = q0 + t * 16 + l16;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const int d = s * 16 + g4 * 4;
      qf[t][s] = d < HD ? ld_quad<WIDE>(qb + static_cast<int64_t>(q < n ? q : n - 1) * g.a.ldq + d) : zero;
    }
  }
  floatx4 o[QT][DT];
  float mrun[QT], lrun[QT];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    mrun[t] = -INFINITY; lrun[t] = 0.0f;
#pragma unroll
    for (int i = 0; i < DT; ++i) o[t][i] = zero;
  }
  const int keys = CAUSAL ? min(n, q0 + 16 * QT) : n;           // that any query of the block sees
  const int ntiles = (keys + 15) / 16;
  floatx4 kf[KS];
  auto load_k = [&](int kt) {
    int key = kt * 16 + l16;
    key = key < n ? key : n - 1;
    const T* p = kb + static_cast<int64_t>(key) * g.a.ldk + g4 * 4;
#pragma unroll
    for (int s = 0; s < KS; ++s) kf[s] = s * 16 + g4 * 4 < HD ? ld_quad<WIDE>(p + s * 16) : zero;
  };
  if (wave < ntiles) load_k(wave);
  for (int kt = wave; kt < ntiles; kt += 4) {
    // this tile's values, on their way during the scores
    floatx4 vf[4][G > 0 ? G : 1];
    float vr[4][RT > 0 ? RT : 1];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      int key = kt * 16 + g4 * 4 + r;
      key = key < n ? key : n - 1;
      const T* p = vb + static_cast<int64_t>(key) * g.a.ldv;
#pragma unroll
      for (int j = 0; j < G; ++j) vf[r][j] = ld_quad<WIDE>(p + j * 64 + l16 * 4);
#pragma unroll
      for (int i = 0; i < RT; ++i) vr[r][i] = i * 16 + l16 < REM ? ld_one(p + 64 * G + i * 16 + l16) : 0.0f;
    }
    floatx4 s[QT];
#pragma unroll
    for (int t = 0; t < QT; ++t) s[t] = zero;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int t = 0; t < QT; ++t) s[t] = mfma4(kf[ks][c], qf[t][ks][c], s[t]);
    if (kt + 4 < ntiles) load_k(kt + 4);
    if (kt * 16 + 16 > n) {                        // keys past the end: probability 0, which must not meet an infinite value
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        if (kt * 16 + g4 * 4 + r < n) continue;
#pragma unroll
        for (int j = 0; j < G; ++j) vf[r][j] = zero;
#pragma unroll
        for (int i = 0; i < RT; ++i) vr[r][i] = 0.0f;
      }
    }
    const bool edge = kt * 16 + 16 > (CAUSAL ? min(n, q0 + 1) : n);          // some query does not see all of the tile
    // A value that is no number must not meet the probability 0 of a query that does not see it.  The tiles that causal queries see in part
    // are looked through; where one is found, it is taken out of the products and counted for the queries that see it.
    auto value = [&](int r, int i) { return i < 4 * G ? vf[r][G > 0 ? i / 4 : 0][i % 4] : vr[r][RT > 0 ? i - 4 * G : 0]; };
    bool odd = false;
    if (CAUSAL && edge) {
#pragma unroll
      for (int r = 0; r < 4; ++r) {
#pragma unroll
        for (int j = 0; j < G; ++j) odd |= !(finite(vf[r][j][0]) && finite(vf[r][j][1]) && finite(vf[r][j][2]) && finite(vf[r][j][3]));
#pragma unroll
        for (int i = 0; i < RT; ++i) odd |= !finite(vr[r][i]);
      }
      odd = __any(odd);
    }
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      if (edge) {
        const int last = CAUSAL ? min(n - 1, q0 + t * 16 + l16) : n - 1;
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (kt * 16 + g4 * 4 + r > last) s[t][r] = -INFINITY;
      }
      float tmax = fmaxf(fmaxf(s[t][0], s[t][1]), fmaxf(s[t][2], s[t][3]));
      tmax = fmaxf(tmax, __shfl_xor(tmax, 16, 64));
      tmax = fmaxf(tmax, __shfl_xor(tmax, 32, 64));
      const float mnew = fmaxf(mrun[t], tmax);
      // nothing but scores of -inf so far: weight 0, and not -inf - (-inf).  Only a query whose every score is -inf has no softmax; the merge
      // makes that NaN.
      const float moff = mnew == -INFINITY ? 0.0f : mnew * scale_log2e;
      const float corr = __builtin_amdgcn_exp2f(fmaf(mrun[t], scale_log2e, -moff));     // the first tile: exp2(-inf) = 0
      float p[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) p[r] = __builtin_amdgcn_exp2f(fmaf(s[t][r], scale_log2e, -moff));
      lrun[t] = fmaf(lrun[t], corr, (p[0] + p[1]) + (p[2] + p[3]));
      mrun[t] = mnew;
#pragma unroll
      for (int i = 0; i < DT; ++i) o[t][i] *= corr;
      if (CAUSAL && odd) {
        // products of the places of +inf, -inf and NaN with the places that a query sees say where they belong
        const int last = min(n - 1, q0 + t * 16 + l16);
#pragma unroll
        for (int i = 0; i < DT; ++i) {
          floatx4 plus = zero, minus = zero, none = zero;
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const float v = value(r, i), sees = kt * 16 + g4 * 4 + r <= last ? 1.0f : 0.0f;
            plus = mfma4(v == INFINITY ? 1.0f : 0.0f, sees, plus);
            minus = mfma4(v == -INFINITY ? 1.0f : 0.0f, sees, minus);
            none = mfma4(v != v ? 1.0f : 0.0f, sees, none);
            o[t][i] = mfma4(finite(v) ? v : 0.0f, p[r], o[t][i]);
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if (plus[e] > 0.0f) o[t][i][e] += INFINITY;
            if (minus[e] > 0.0f) o[t][i][e] -= INFINITY;
            if (none[e] > 0.0f) o[t][i][e] = __uint_as_float(0x7FC00000u);
          }
        }
        continue;
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) {
#pragma unroll
        for (int i = 0; i < 4 * G; ++i) o[t][i] = mfma4(vf[r][i / 4][i % 4], p[r], o[t][i]);
#pragma unroll
        for (int i = 0; i < RT; ++i) o[t][4 * G + i] = mfma4(vr[r][i], p[r], o[t][4 * G + i]);
      }
    }
  }
  // merge in wave order: every wave scales its sums to the common maximum; waves 1 .. 3 hand theirs over in LDS
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    float l = lrun[t];
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
    if (t > 0) __syncthreads();
    if (lane < 16) { stats[wave][0][l16] = mrun[t]; stats[wave][1][l16] = l; }
    __syncthreads();
    const float m = fmaxf(fmaxf(stats[0][0][l16], stats[1][0][l16]), fmaxf(stats[2][0][l16], stats[3][0][l16]));
    float f[4], lsum = 0.0f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      f[w] = __builtin_amdgcn_exp2f((stats[w][0][l16] - m) * scale_log2e);            // a wave without a tile: exp2(-inf) = 0
      lsum = fmaf(stats[w][1][l16], f[w], lsum);
    }
    const float mine = wave == 0 ? f[0] : wave == 1 ? f[1] : wave == 2 ? f[2] : f[3];
    if (wave > 0) {
#pragma unroll
      for (int i = 0; i < DT; ++i) *reinterpret_cast<floatx4*>(&merge[wave - 1][l16 * OST + i * 16 + g4 * 4]) = o[t][i] * mine;
    }
    __syncthreads();
    if (wave == 0) {
      const float inv = 1.0f / lsum;
      const int q = q0 + t * 16 + l16;
#pragma unroll
      for (int i = 0; i < DT; ++i) {
        floatx4 v = o[t][i] * mine;
#pragma unroll
        for (int w = 0; w < 3; ++w) v += *reinterpret_cast<const floatx4*>(&merge[w][l16 * OST + i * 16 + g4 * 4]);
        o[t][i] = v * inv;
      }
      if (q < n) {
        T* op = static_cast<T*>(g.a.out) + (static_cast<int64_t>(start) + q) * g.a.ldo + head * HD;
        // accumulator r of tile i of group j is dimension 64 j + 4 (4 g4 + r) + i
#pragma unroll
        for (int j = 0; j < G; ++j)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            st_quad<WIDE>(op + j * 64 + 4 * (4 * g4 + r), floatx4{o[t][4 * j][r], o[t][4 * j + 1][r], o[t][4 * j + 2][r], o[t][4 * j + 3][r]});
#pragma unroll
        for (int i = 0; i < RT; ++i) {
          const int d = i * 16 + g4 * 4;
          if (d < REM) st_quad<WIDE>(op + 64 * G + d, o[t][4 * G + i]);
        }
      }
    }
  }
}

template <typename T, int HD, int QT>
void launch_qt(const Args& g, bool wide, unsigned blocks, hipStream_t st) {
  if (g.a.causal && wide) attention_packed_f32_kernel<T, HD, QT, true, true><<<blocks, 256, 0, st>>>(g);
  else if (g.a.causal) attention_packed_f32_kernel<T, HD, QT, true, false><<<blocks, 256, 0, st>>>(g);
  else if (wide) attention_packed_f32_kernel<T, HD, QT, false, true><<<blocks, 256, 0, st>>>(g);
  else attention_packed_f32_kernel<T, HD, QT, false, false><<<blocks, 256, 0, st>>>(g);
}

template <typename T, int HD>
Error launch_hd(const Args& g, hipStream_t st) {
  const PackedAttention& a = g.a;
  const uintptr_t at = reinterpret_cast<uintptr_t>(a.q) | reinterpret_cast<uintptr_t>(a.k) | reinterpret_cast<uintptr_t>(a.v) | reinterpret_cast<uintptr_t>(a.out);
  const bool wide = at % (4 * sizeof(T)) == 0 && (a.ldq | a.ldk | a.ldv | a.ldo) % 4 == 0;
  // 32 queries per block read every key and value half as often; 16 keep the chip busy when there are few blocks, and waste less where sequences or
  // what causal queries see end.  us, 32 / 16: up to 512 blocks 16 are never slower (396 blocks, the sequences above, 47 / 42; 192 blocks 104 / 86);
  // beyond, without mask, 16 heads of 72 over 4096 tokens 858 / 1059, 8 of 16 124 / 140, 24 of 128 2081 / 2128, 4 x 1024 tokens of 6 heads of 64
  // 75 / 72, 20 x 300 of 24 of 128 374 / 307; causal, 16 heads of 72 over 4096 588 / 676, 24 of 128 1413 / 1230, 6 of 64 217 / 164.
  const bool two = static_cast<int64_t>(a.seqs.total / 32) * a.heads >= 512;
  const int64_t blocks = packed_tiles(a.seqs, 1, two ? 32 : 16, 0) * a.heads;
  if (blocks > kMaxBlocks) SPECA_FAIL(SPECA_EINVAL, "speca_attention_packed: %d tokens of %d heads are too many for one call", a.seqs.total, a.heads);
  if (two) launch_qt<T, HD, 2>(g, wide, static_cast<unsigned>(blocks), st);
  else launch_qt<T, HD, 1>(g, wide, static_cast<unsigned>(blocks), st);
  SPECA_HIP(hipGetLastError());
  return ok();
}

template <typename T>
Error launch_t(const Args& g, hipStream_t st) {
  switch (g.a.head_dim) {
    case 16: return launch_hd<T, 16>(g, st);
    case 32: return launch_hd<T, 32>(g, st);
    case 64: return launch_hd<T, 64>(g, st);
    case 72: return launch_hd<T, 72>(g, st);
    case 128: return launch_hd<T, 128>(g, st);
  }
  SPECA_FAIL(SPECA_EUNSUPPORTED, "speca_attention_packed: head_dim %d (supported: 16, 32, 64, 72, 128)", g.a.head_dim);
}

}  // namespace

Error launch_attention_packed_f32(int dtype, const PackedAttention& a, hipStream_t st) {
  Args g;
  g.a = a;
  g.group = a.heads / a.kv_heads;
  g.scale_log2e = 1.4426950408889634f * a.scale;
  return dtype == SPECA_BF16 ? launch_t<bf16_t>(g, st) : launch_t<float>(g, st);
}

}  // namespace speca
