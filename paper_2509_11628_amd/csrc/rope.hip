// Rotary positions with several axes on packed queries and keys, behind the RMS norm of every head where there is one.
//
//   y = x / sqrt(mean(x^2) + eps) * w      (a, b) -> (a cos - b sin, a sin + b cos),  angle = position[axis] * rate[pair]
//
// Bound by memory: every value is read and written once, at 6 operations.  27 286 tokens of 24 + 24 heads of 128 with norm: 141 us, 4.8
// TB/s (a large copy moves 5.05).  What is not memory is the angle: position x rate is formed in 64 bits and in turns, of which only the
// fraction counts (exact to 10^-9 of a turn at positions of 10^6); that is rounded to 32 bits for sine and cosine, half a step of at most 2^-26
// of a turn, 10^-7 radians at any position, about what the products lose in fp32 and far below a step of bf16.  The lanes that hold the same
// pairs of several heads share the work on it (184 us before that and before the token's addresses were scalar).
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
  int32_t steps_per_wave;           // of 64 / lanes_per_head heads
  int32_t chunks;                   // waves per token
  float eps, per_feature;           // 1 / hd
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

// VP values at p + lo and VP at p + hi; ahead of the loads, or behind the stores, of a pair of neighbours (ADJACENT) one access of both
template <int VP, bool HALVES, typename T>
__device__ inline void rope_load(const T* p, uint32_t lo, uint32_t hi, float (&a)[VP], float (&b)[VP]) {
  rope_read<VP>(p + lo, a);
  rope_read<VP>(p + (HALVES || VP == 1 ? hi : lo + VP), b);
}
template <int VP, bool HALVES, typename T>
__device__ inline void rope_store(T* p, uint32_t lo, uint32_t hi, const float (&a)[VP], const float (&b)[VP]) {
  rope_write<VP>(p + lo, a);
  rope_write<VP>(p + (HALVES || VP == 1 ? hi : lo + VP), b);
}

// One wave = one token and some of its heads, steps of 64 / lanes_per_head heads of q, then of k; a lane owns VP pairs of a head.  Its
// pieces are VP features at lo and VP at hi: with HALVES the two sides of its pairs, otherwise neighbours, of which features 2j and 2j + 1
// are a pair. What belongs to the token or the step is in scalar registers, so a lane's addresses are one offset each.
template <typename T, int VP, bool HALVES, bool NORM>
__global__ __launch_bounds__(256) void rope_axes_kernel(const RopeArgs g) {
  constexpr int UN = 4;
  const int lane = threadIdx.x & 63;
  const int64_t item = static_cast<int64_t>(blockIdx.x) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t tok = item / g.chunks;
  if (tok >= g.tokens) return;
  const int chunk = static_cast<int>(item - tok * g.chunks);
  const int u = lane & (g.lanes_per_head - 1), sub = lane / g.lanes_per_head, per = 64 / g.lanes_per_head;
  const int units = g.hd / (2 * VP), pairs = g.rotated / 2;
  const bool live = u < units;
  uint32_t lo = u * 2 * VP, hi = lo + VP;
  if (HALVES && u * VP < pairs) { lo = u * VP; hi = pairs + lo; }
  lo += sub * g.hd;
  hi += sub * g.hd;

  // The lanes that hold the same pairs of several heads share the work on their angles where there are four of them or more.
  float cs[VP], sn[VP];
  auto angle = [&](int pair, float* c, float* s) {
    *c = 1.0f;
    *s = 0.0f;
    if (pair < pairs) {
      const double turns = static_cast<double>(g.positions[tok * g.axes + g.axis[pair]]) * g.rate[pair];
      sincospif(2.0f * static_cast<float>(turns - rint(turns)), s, c);
    }
  };
  if (VP == 4 && per >= 4) {
    float c, s;
    angle(u * VP + (sub & 3), &c, &s);
#pragma unroll
    for (int j = 0; j < VP; ++j) {
      cs[j] = __shfl(c, j * g.lanes_per_head + u, 64);
      sn[j] = __shfl(s, j * g.lanes_per_head + u, 64);
    }
  } else {
#pragma unroll
    for (int j = 0; j < VP; ++j) angle(u * VP + j, &cs[j], &sn[j]);
  }

  // Only pairs that turn: by an angle of 0 a feature would not stay as it is, since 0 x its neighbour is NaN where that is infinite or NaN.
  // (Selected: as branches 146 us instead of 141.)
  auto turn = [](bool turns, float& a, float& b, float c, float s) {
    const float x = fmaf(a, c, -(b * s)), y = fmaf(a, s, b * c);
    a = turns ? x : a;
    b = turns ? y : b;
  };

  int first = chunk * g.steps_per_wave, last = first + g.steps_per_wave;       // steps of this wave, counted from the side's first
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    const RopeSide& s = g.side[which];
    const int heads = which ? g.total_heads - g.heads : g.heads, steps = (heads + per - 1) / per;
    const int from = first < 0 ? 0 : first, to = last < steps ? last : steps;
    first -= steps;
    last -= steps;
    if (from >= to) continue;
    const bool norm = NORM && s.norm;
    float wa[VP] = {}, wb[VP] = {};
    if (norm && live) rope_load<VP, HALVES>(static_cast<const T*>(s.norm), lo - sub * g.hd, hi - sub * g.hd, wa, wb);
    const T* x = static_cast<const T*>(s.x) + tok * s.ldx;
    T* out = static_cast<T*>(s.out) + tok * s.ldo;
    // UN steps at a time: that many loads are on their way before the first is waited for
    for (int s0 = from; s0 < to; s0 += UN) {
      float a[UN][VP], b[UN][VP];
#pragma unroll
      for (int i = 0; i < UN; ++i) {
        const int step = s0 + i;
#pragma unroll
        for (int j = 0; j < VP; ++j) a[i][j] = b[i][j] = 0.0f;
        if (step < to && live && step * per + sub < heads) rope_load<VP, HALVES>(x + step * per * g.hd, lo, hi, a[i], b[i]);
      }
      if (norm) {
        float sum[UN];
#pragma unroll
        for (int i = 0; i < UN; ++i) {
          // pair by pair, then pairs 1, 2, 4, ... apart: the same order, and the same bits, whether a lane holds one pair or four
          if constexpr (VP == 1) {
            sum[i] = fmaf(a[i][0], a[i][0], b[i][0] * b[i][0]);
          } else {
            const bool across = HALVES && u * VP < pairs;
            float t[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const float x0 = across ? a[i][j] : j < 2 ? a[i][2 * j] : b[i][2 * j - 4], x1 = across ? b[i][j] : j < 2 ? a[i][2 * j + 1] : b[i][2 * j - 3];
              t[j] = fmaf(x0, x0, x1 * x1);
            }
            sum[i] = (t[0] + t[1]) + (t[2] + t[3]);
          }
        }
        for (int off = 1; off < g.lanes_per_head; off <<= 1)
#pragma unroll
          for (int i = 0; i < UN; ++i) sum[i] += __shfl_xor(sum[i], off, 64);
#pragma unroll
        for (int i = 0; i < UN; ++i) {
          const float r = rsqrtf(fmaf(sum[i], g.per_feature, g.eps));
#pragma unroll
          for (int j = 0; j < VP; ++j) { a[i][j] *= r * wa[j]; b[i][j] *= r * wb[j]; }
        }
      }
#pragma unroll
      for (int i = 0; i < UN; ++i) {
        const int step = s0 + i;
        if (step >= to) break;
        float(&p)[VP] = a[i];
        float(&q)[VP] = b[i];
        if constexpr (HALVES || VP == 1) {
#pragma unroll
          for (int j = 0; j < VP; ++j) turn(u * VP < pairs, p[j], q[j], cs[j], sn[j]);
        } else {
#pragma unroll
          for (int j = 0; j < VP; ++j) {
            float(&x)[VP] = j < VP / 2 ? p : q;
            turn(u * VP + j < pairs, x[2 * j % VP], x[2 * j % VP + 1], cs[j], sn[j]);
          }
        }
        if (live && step * per + sub < heads) rope_store<VP, HALVES>(out + step * per * g.hd, lo, hi, p, q);
      }
    }
  }
}

template <typename T, int VP>
void launch_vp(const RopeArgs& g, bool halves, unsigned blocks, hipStream_t st) {
  const bool norm = g.side[0].norm || g.side[1].norm;
  if (halves && norm) rope_axes_kernel<T, VP, true, true><<<blocks, 256, 0, st>>>(g);
  else if (halves) rope_axes_kernel<T, VP, true, false><<<blocks, 256, 0, st>>>(g);
  else if (norm) rope_axes_kernel<T, VP, false, true><<<blocks, 256, 0, st>>>(g);
  else rope_axes_kernel<T, VP, false, false><<<blocks, 256, 0, st>>>(g);
}

template <typename T>
void launch_t(const RopeArgs& g, int vp, bool halves, unsigned blocks, hipStream_t st) {
  if (vp == 4) launch_vp<T, 4>(g, halves, blocks, st);
  else launch_vp<T, 1>(g, halves, blocks, st);
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
  if (!positions || reinterpret_cast<uintptr_t>(positions) % 4) SPECA_FAIL(SPECA_EINVAL, "speca_rope_axes: positions is NULL or not aligned to int32");
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
  g.per_feature = 1.0f / static_cast<float>(head_dim);
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
  // Four pairs a lane where every piece of four features lies at a whole piece (16 bytes in fp32, 8 in bf16), one pair otherwise (140
  // and 620 us for 27 286 tokens of 48 heads of 128).  With HALVES the pairs of a lane must end with the rotation, and what does not turn
  // has to be whole lanes too.
  const size_t piece = 4 * dtype_size(dtype);
  uintptr_t at = 0;
  for (const RopeSide& s : g.side)
    at |= reinterpret_cast<uintptr_t>(s.x) | reinterpret_cast<uintptr_t>(s.out) | reinterpret_cast<uintptr_t>(s.norm) | static_cast<uintptr_t>(s.ldx * dtype_size(dtype)) |
          static_cast<uintptr_t>(s.ldo * dtype_size(dtype));
  const bool halves = rope.pairing == SPECA_ROPE_HALVES;
  const int vp = at % piece == 0 && head_dim % 8 == 0 && (!halves || rotated % 8 == 0) ? 4 : 1;
  g.lanes_per_head = 1;
  while (g.lanes_per_head < head_dim / (2 * vp)) g.lanes_per_head *= 2;
  // A wave takes all heads of its token where there are tokens enough for 8 waves per SIMD; with fewer, the heads are dealt to as many waves.
  const int per = 64 / g.lanes_per_head, steps = (g.heads + per - 1) / per + (g.total_heads - g.heads + per - 1) / per;
  const int64_t waves = int64_t{32} * compute_units();
  g.chunks = static_cast<int>(std::min<int64_t>(steps, std::max<int64_t>(1, (waves + tokens - 1) / tokens)));
  g.steps_per_wave = (steps + g.chunks - 1) / g.chunks;
  g.chunks = (steps + g.steps_per_wave - 1) / g.steps_per_wave;
  const int64_t blocks = (tokens * g.chunks + 3) / 4;
  if (blocks > kMaxBlocks) SPECA_FAIL(SPECA_EINVAL, "speca_rope_axes: %lld tokens are too many for one call", static_cast<long long>(tokens));
  if (dtype == SPECA_BF16) launch_t<bf16_t>(g, vp, halves, static_cast<unsigned>(blocks), st);
  else launch_t<float>(g, vp, halves, static_cast<unsigned>(blocks), st);
  SPECA_HIP(hipGetLastError());
  return ok();
}

}  // namespace speca
