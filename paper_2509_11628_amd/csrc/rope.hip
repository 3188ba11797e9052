// Rotary positions with several axes on packed queries and keys, behind the RMS norm of every head where there is one.
//
//   y = x / sqrt(mean(x^2) + eps) * w      (a, b) -> (a cos - b sin, a sin + b cos),  angle = position[axis] * rate[pair]
//
// Bound by memory: every value is read and written once, at 6 operations.  What is not memory is the angle: position x rate is formed in
// 64 bits and in turns, of which only the fraction counts, so a position of 10^6 keeps an angle of 10^-9; one lane forms its pairs' sines once
// and uses them for every head of the token that its wave works on.
#include <algorithm>
#include <cmath>

#include "gemm.h"
#include "attn_lane.h"
#include "operators.h"

namespace speca {

namespace {

constexpr int kMaxHead = 128;


struct RopeSide {
  const void* x;
  void* out;
  const void* norm;
  int64_t ldx, ldo;
};
struct RopeArgs {
  RopeSide side[2];                 // q, k
  const int32_t* positions;
  int64_t tokens;
  int32_t axes, hd, rotated;        // rotated: features that turn
  int32_t heads, total_heads;       // of q, of q and k
  int32_t lanes_per_head;           // power of two, at least hd / (2 VP)
  int32_t heads_per_wave;           // multiple of 64 / lanes_per_head
  int32_t chunks;                   // waves per token
  float eps;
  double rate[kMaxHead / 2];        // turns per position of a pair
  uint8_t axis[kMaxHead / 2];
};

// VP values in one access (4: 16 or 8 bytes; 1: one element)
template <int VP>
__device__ inline void rope_read(const float* p, float (&v)[VP]) {
  if constexpr (VP == 4) {
    const float4 f = *reinterpret_cast<const float4*>(p);
    v[0] = f.x; v[1] = f.y; v[2] = f.z; v[3] = f.w;
  } else {
    v[0] = *p;
  }
}
template <int VP>
__device__ inline void rope_read(const bf16_t* p, float (&v)[VP]) {
  if constexpr (VP == 4) {
    const uint2 f = *reinterpret_cast<const uint2*>(p);
    v[0] = __uint_as_float(f.x << 16); v[1] = __uint_as_float(f.x & 0xFFFF0000u);
    v[2] = __uint_as_float(f.y << 16); v[3] = __uint_as_float(f.y & 0xFFFF0000u);
  } else {
    v[0] = bf16_to_f32(p->bits);
  }
}
template <int VP>
__device__ inline void rope_write(float* p, const float (&v)[VP]) {
  if constexpr (VP == 4) *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
  else *p = v[0];
}
template <int VP>
__device__ inline void rope_write(bf16_t* p, const float (&v)[VP]) {
  if constexpr (VP == 4) *reinterpret_cast<uint2*>(p) = make_uint2(cvt_pk_bf16(v[0], v[1]), cvt_pk_bf16(v[2], v[3]));
  else p->bits = static_cast<uint16_t>(cvt_pk_bf16(v[0], v[0]));
}

// One wave = one token and heads_per_wave of its heads; a lane owns VP pairs of a head and a wave's lanes hold 64 / lanes_per_head heads at a
// time.  The pieces of a lane are VP features at lo and VP at hi: with HALVES the two sides of its pairs, otherwise neighbours, of which
// features 2j and 2j + 1 are a pair.
template <typename T, int VP, bool HALVES>
__global__ __launch_bounds__(256) void rope_axes_kernel(const RopeArgs g) {
  const int lane = threadIdx.x & 63;
  const int64_t item = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6);
  const int64_t tok = item / g.chunks;
  if (tok >= g.tokens) return;
  const int chunk = static_cast<int>(item - tok * g.chunks);
  const int u = lane & (g.lanes_per_head - 1), sub = lane / g.lanes_per_head, per = 64 / g.lanes_per_head;
  const int units = g.hd / (2 * VP), pairs = g.rotated / 2;
  const bool live = u < units;
  int lo = u * 2 * VP, hi = lo + VP;
  if (HALVES && u * VP < pairs) { lo = u * VP; hi = pairs + lo; }

  float cs[VP], sn[VP];
#pragma unroll
  for (int j = 0; j < VP; ++j) {
    const int pair = u * VP + j;
    cs[j] = 1.0f;
    sn[j] = 0.0f;
    if (pair < pairs) {
      const double turns = static_cast<double>(g.positions[tok * g.axes + g.axis[pair]]) * g.rate[pair];
      sincospif(2.0f * static_cast<float>(turns - rint(turns)), &sn[j], &cs[j]);
    }
  }
  const int end = min(g.total_heads, (chunk + 1) * g.heads_per_wave);
  for (int h = chunk * g.heads_per_wave + sub; h < end; h += per) {
    const RopeSide& s = g.side[h < g.heads ? 0 : 1];
    const int64_t at = static_cast<int64_t>(h < g.heads ? h : h - g.heads) * g.hd;
    const T* x = static_cast<const T*>(s.x) + tok * s.ldx + at;
    T* out = static_cast<T*>(s.out) + tok * s.ldo + at;
    float a[VP] = {}, b[VP] = {};
    if (live) { rope_read<VP>(x + lo, a); rope_read<VP>(x + hi, b); }
    if (s.norm) {
      float sum = 0.0f;
#pragma unroll
      for (int j = 0; j < VP; ++j) sum += a[j] * a[j] + b[j] * b[j];
      for (int off = g.lanes_per_head >> 1; off; off >>= 1) sum += __shfl_xor(sum, off, 64);
      const float r = 1.0f / sqrtf(sum / static_cast<float>(g.hd) + g.eps);
      float wa[VP] = {}, wb[VP] = {};
      if (live) { rope_read<VP>(static_cast<const T*>(s.norm) + lo, wa); rope_read<VP>(static_cast<const T*>(s.norm) + hi, wb); }
#pragma unroll
      for (int j = 0; j < VP; ++j) { a[j] *= r * wa[j]; b[j] *= r * wb[j]; }
    }
    if (!live) continue;
    if constexpr (HALVES || VP == 1) {
#pragma unroll
      for (int j = 0; j < VP; ++j) {
        const float c = a[j] * cs[j] - b[j] * sn[j];
        b[j] = a[j] * sn[j] + b[j] * cs[j];
        a[j] = c;
      }
    } else {
#pragma unroll
      for (int j = 0; j < VP; j += 2) {
        const float c = a[j] * cs[j / 2] - a[j + 1] * sn[j / 2], d = b[j] * cs[VP / 2 + j / 2] - b[j + 1] * sn[VP / 2 + j / 2];
        a[j + 1] = a[j] * sn[j / 2] + a[j + 1] * cs[j / 2];
        b[j + 1] = b[j] * sn[VP / 2 + j / 2] + b[j + 1] * cs[VP / 2 + j / 2];
        a[j] = c;
        b[j] = d;
      }
    }
    rope_write<VP>(out + lo, a);
    rope_write<VP>(out + hi, b);
  }
}

template <typename T>
void launch_t(const RopeArgs& g, bool halves, unsigned blocks, hipStream_t st) {
  if (halves) rope_axes_kernel<T, 1, true><<<blocks, 256, 0, st>>>(g);
  else rope_axes_kernel<T, 1, false><<<blocks, 256, 0, st>>>(g);
}

Error check_side(const char* name, int dtype, const speca_rope_io& s, int hd) {
  const size_t esz = dtype_size(dtype);
  if (!s.x || !s.out) SPECA_FAIL(SPECA_EINVAL, "speca_rope_axes: %s: x and out must not be NULL", name);
  if (s.heads < 1 || s.heads > 65536) SPECA_FAIL(SPECA_EINVAL, "speca_rope_axes: %s: heads = %d", name, s.heads);
  const int64_t width = static_cast<int64_t>(s.heads) * hd;
  if (s.ldx < width || s.ldo < width || s.ldx > (int64_t{1} << 40) || s.ldo > (int64_t{1} << 40))
    SPECA_FAIL(SPECA_EINVAL, "speca_rope_axes: %s: tokens %lld and %lld elements apart, heads need %lld", name, static_cast<long long>(s.ldx),
               static_cast<long long>(s.ldo), static_cast<long long>(width));
  if (s.x == s.out && s.ldx != s.ldo) SPECA_FAIL(SPECA_EINVAL, "speca_rope_axes: %s: in place with two strides", name);
  if ((reinterpret_cast<uintptr_t>(s.x) | reinterpret_cast<uintptr_t>(s.out) | reinterpret_cast<uintptr_t>(s.norm)) % esz)
    SPECA_FAIL(SPECA_EINVAL, "speca_rope_axes: %s: a pointer is not aligned to its type", name);
  return ok();
}

}  // namespace

Error launch_rope_axes(int dtype, const speca_rope& rope, const int32_t* positions, int64_t tokens, int head_dim, float eps,
                       const speca_rope_io& q, const speca_rope_io* k, hipStream_t st) {
  if (dtype != SPECA_F32 && dtype != SPECA_BF16) SPECA_FAIL(SPECA_EINVAL, "speca_rope_axes: dtype = %d", dtype);
  if (head_dim < 2 || head_dim > kMaxHead || head_dim % 2) SPECA_FAIL(SPECA_EINVAL, "speca_rope_axes: head_dim = %d (even, 2..%d)", head_dim, kMaxHead);
  if (rope.axes < 1 || rope.axes > SPECA_ROPE_MAX_AXES) SPECA_FAIL(SPECA_EINVAL, "speca_rope_axes: axes = %d (1..%d)", rope.axes, SPECA_ROPE_MAX_AXES);
  if (rope.pairing != SPECA_ROPE_ADJACENT && rope.pairing != SPECA_ROPE_HALVES) SPECA_FAIL(SPECA_EINVAL, "speca_rope_axes: pairing = %d", rope.pairing);
  if (rope.spectrum != SPECA_ROPE_PER_AXIS && rope.spectrum != SPECA_ROPE_JOINT) SPECA_FAIL(SPECA_EINVAL, "speca_rope_axes: spectrum = %d", rope.spectrum);
  int rotated = 0;
  for (int a = 0; a < rope.axes; ++a) {
    if (rope.dims[a] < 2 || rope.dims[a] % 2 || rope.dims[a] > head_dim) SPECA_FAIL(SPECA_EINVAL, "speca_rope_axes: dims[%d] = %d", a, rope.dims[a]);
    if (!(rope.theta[a] > 0.0f) || !std::isfinite(rope.theta[a])) SPECA_FAIL(SPECA_EINVAL, "speca_rope_axes: theta[%d] = %g", a, rope.theta[a]);
    if (!std::isfinite(rope.scale[a])) SPECA_FAIL(SPECA_EINVAL, "speca_rope_axes: scale[%d] = %g", a, rope.scale[a]);
    rotated += rope.dims[a];
  }
  if (rotated > head_dim) SPECA_FAIL(SPECA_EINVAL, "speca_rope_axes: %d features turn, a head has %d", rotated, head_dim);
  if (tokens < 0 || tokens > 0x7FFFFFFF) SPECA_FAIL(SPECA_EINVAL, "speca_rope_axes: tokens = %lld", static_cast<long long>(tokens));
  if (!(eps >= 0.0f) || !std::isfinite(eps)) SPECA_FAIL(SPECA_EINVAL, "speca_rope_axes: eps = %g", eps);
  SPECA_TRY(check_side("q", dtype, q, head_dim));
  if (k) SPECA_TRY(check_side("k", dtype, *k, head_dim));
  if (!positions) SPECA_FAIL(SPECA_EINVAL, "speca_rope_axes: positions is NULL");
  if (tokens == 0) return ok();

  RopeArgs g;
  g.side[0] = {q.x, q.out, q.norm, q.ldx, q.ldo};
  g.side[1] = k ? RopeSide{k->x, k->out, k->norm, k->ldx, k->ldo} : g.side[0];
  g.positions = positions;
  g.tokens = tokens;
  g.axes = rope.axes;
  g.hd = head_dim;
  g.rotated = rotated;
  g.heads = q.heads;
  g.total_heads = q.heads + (k ? k->heads : 0);
  g.eps = eps;
  // rates by repeated multiplication: 128 steps of half a bit of 2^-53 each, far below what a fraction of a turn shows
  int pair = 0;
  for (int a = 0; a < rope.axes; ++a) {
    const bool own = rope.spectrum == SPECA_ROPE_PER_AXIS;
    const double base = own ? rope.theta[a] : rope.theta[0], ratio = std::pow(base, -2.0 / (own ? rope.dims[a] : rotated));
    double r = own || pair == 0 ? 1.0 : std::pow(ratio, pair);
    for (int j = 0; j < rope.dims[a] / 2; ++j, ++pair, r *= ratio) {
      g.rate[pair] = r * rope.scale[a] / 6.283185307179586476925;
      g.axis[pair] = static_cast<uint8_t>(a);
    }
  }
  g.lanes_per_head = 1;
  while (g.lanes_per_head < head_dim / 2 && g.lanes_per_head < 64) g.lanes_per_head *= 2;
  const int per = 64 / g.lanes_per_head;
  const int steps = (g.total_heads + per - 1) / per;
  g.chunks = steps;
  g.heads_per_wave = per;
  const int64_t blocks = (tokens * g.chunks + 3) / 4;
  if (blocks > 0x7FFFFFFF) SPECA_FAIL(SPECA_EINVAL, "speca_rope_axes: %lld tokens are too many for one call", static_cast<long long>(tokens));
  if (dtype == SPECA_BF16) launch_t<bf16_t>(g, rope.pairing == SPECA_ROPE_HALVES, static_cast<unsigned>(blocks), st);
  else launch_t<float>(g, rope.pairing == SPECA_ROPE_HALVES, static_cast<unsigned>(blocks), st);
  SPECA_HIP(hipGetLastError());
  return ok();
}

}  // namespace speca
