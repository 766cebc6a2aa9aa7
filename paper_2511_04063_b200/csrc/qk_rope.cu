// Queries and keys of each head (dq_qk_norm_rope): root-mean-square norm, rotation by position, Hadamard rotation, in one pass.
//
//   h = x / sqrt(mean x^2 + eps) gamma;  (a, b) -> (a cos t - b sin t, b cos t + a sin t), t = position inv_freq[i];  y = h H / sqrt(D)
//
// A lane holds 16 values of a head, D / 16 lanes a head.  Its two pieces of eight are chosen so that every rotated pair lies in one
// lane: 8 l and rot / 2 + 8 l for pairs of halves, neighbours otherwise.  The Hadamard rotation is a butterfly over the bits of the
// index, whichever of them are a lane's own (16 values: four) and whichever are the lane's number (one exchange of all values
// each: with 8 values a lane it would be four exchanges for D = 128 instead of three).
//
// A CTA takes one token (or a part of its heads), so that its angles are formed once, in 64 bits: position x inv_freq is exact
// there up to 2^-53, and at position 10^6 a product in fp32 would be off by 0.06.
#include "kv_common.cuh"

namespace dq {
namespace kv {
namespace {

using mx::Vec8;
using mx::from_f32;
using mx::to_f32;

constexpr int THREADS = 256;

template <typename T, bool VEC>
__device__ __forceinline__ void load8(Vec8<T>& v, const T* p) {
  if constexpr (VEC) v.load(p);
  else
#pragma unroll
  for (int i = 0; i < 4; ++i) v.set_pair(i, make_float2(to_f32(p[2 * i]), to_f32(p[2 * i + 1])));
}
template <typename T, bool VEC>
__device__ __forceinline__ void store8(const Vec8<T>& v, T* p) {
  if constexpr (VEC) v.store(p);
  else
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = v.pair(i);
    p[2 * i] = from_f32<T>(f.x);
    p[2 * i + 1] = from_f32<T>(f.y);
  }
}
template <typename T>
__device__ __forceinline__ void scale_by(float (&x)[16], const void* gamma, int fp32, int a, int b, float by) {
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int at = (i < 8 ? a : b - 8) + i;
    const float g = !gamma ? 1.f : fp32 ? reinterpret_cast<const float*>(gamma)[at] : to_f32(reinterpret_cast<const T*>(gamma)[at]);
    x[i] = x[i] * by * g;
  }
}

// LANES: lanes a head; those past D / 16 hold nothing.
template <typename T, int LANES, bool VEC>
__global__ void __launch_bounds__(THREADS) rope_kernel(const RopeArgs a) {
  __shared__ float s_cos[128], s_sin[128];
  __shared__ float s_turn[THREADS * 16];
  constexpr int GROUPS = THREADS / LANES;
  const int64_t t = blockIdx.x / a.splits;
  const int part = blockIdx.x % a.splits;
  const int l = threadIdx.x % LANES, g = threadIdx.x / LANES;
  const int half = a.rot >> 1;
  const bool halves = !(a.flags & DQ_QK_NEIGHBOURS), norm = a.flags & DQ_QK_NORM, hadamard = a.flags & DQ_QK_HADAMARD;
  const bool held = l * 16 < a.dim, rotated = l * 16 < a.rot;
  const int at_a = halves && rotated ? 8 * l : 16 * l, at_b = halves && rotated ? half + 8 * l : 16 * l + 8;
  const int heads = a.q.heads + a.k.heads;

  auto row = [&](const Heads& q, const Heads& k, int j) {
    const Heads& x = j < q.heads ? q : k;
    return reinterpret_cast<T*>(x.p) + t * x.token + (j < q.heads ? j : j - q.heads) * x.head;
  };
  Vec8<T> va, vb;
  va.clear(); vb.clear();
  auto fetch = [&](int j) {
    if (j < heads && held) {
      const T* p = row(a.q, a.k, j);
      load8<T, VEC>(va, p + at_a);
      load8<T, VEC>(vb, p + at_b);
    }
  };
  mx::wait_for_previous();
  int j = part * GROUPS + g;
  fetch(j);
  if (half) {
    for (int i = threadIdx.x; i < half; i += THREADS) {
      const double turn = (double)a.positions[t] * (double)a.inv_freq[i];
      constexpr double TWO_PI = 6.283185307179586476925;
      float s, c;
      sincosf((float)(turn - rint(turn / TWO_PI) * TWO_PI), &s, &c);
      s_cos[i] = c;
      s_sin[i] = s;
    }
    __syncthreads();
  }
  float cs[16];   // cos and sin of this lane's eight pairs, the same for all heads
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    cs[i] = rotated ? s_cos[8 * l + i] : 1.f;
    cs[8 + i] = rotated ? s_sin[8 * l + i] : 0.f;
  }
  // all lanes of a warp go round equally often: they exchange values
  for (int first = part * GROUPS; first < heads; first += a.splits * GROUPS, j += a.splits * GROUPS) {
    float x[16];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 p = va.pair(i), q = vb.pair(i);
      x[2 * i] = p.x; x[2 * i + 1] = p.y;
      x[8 + 2 * i] = q.x; x[8 + 2 * i + 1] = q.y;
    }
    fetch(j + a.splits * GROUPS);
    if (norm) {
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < 16; ++i) sum += x[i] * x[i];
#pragma unroll
      for (int d = 1; d < LANES; d <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
      const float by = rsqrtf(sum / (float)a.dim + a.eps);
      if (held) scale_by<T>(x, j < a.q.heads ? a.q_gamma : a.k_gamma, a.gamma_fp32, at_a, at_b, by);
    }
    if (half) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int p = halves ? i : 2 * i, q = halves ? 8 + i : 2 * i + 1;
        const float u = x[p] * cs[i] - x[q] * cs[8 + i], v = x[q] * cs[i] + x[p] * cs[8 + i];
        if (rotated) { x[p] = u; x[q] = v; }
      }
    }
    int to_a = at_a, to_b = at_b;
    if (hadamard) {
      if (halves && half && a.rot < a.dim) {   // lanes that hold different bits of the index: to neighbours first
        float* turn = s_turn + (threadIdx.x - l) * 16;
        if (held)
#pragma unroll
          for (int i = 0; i < 16; ++i) turn[(i < 8 ? at_a : at_b - 8) + i] = x[i];
        __syncwarp();
        to_a = 16 * l; to_b = 16 * l + 8;
        if (held)
#pragma unroll
          for (int i = 0; i < 16; ++i) x[i] = turn[to_a + i];
        __syncwarp();
      }
#pragma unroll
      for (int d = 1; d < 16; d <<= 1)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (!(i & d)) { const float u = x[i], v = x[i + d]; x[i] = u + v; x[i + d] = u - v; }
#pragma unroll
      for (int d = 1; d < LANES; d <<= 1)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const float v = __shfl_xor_sync(0xffffffffu, x[i], d);
          x[i] = (l & d) ? v - x[i] : x[i] + v;
        }
      const float by = rsqrtf((float)a.dim);
#pragma unroll
      for (int i = 0; i < 16; ++i) x[i] *= by;
    }
    if (j < heads && held) {
      Vec8<T> ya, yb;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        ya.set_pair(i, make_float2(x[2 * i], x[2 * i + 1]));
        yb.set_pair(i, make_float2(x[8 + 2 * i], x[8 + 2 * i + 1]));
      }
      T* p = row(a.q_out, a.k_out, j);
      store8<T, VEC>(ya, p + to_a);
      store8<T, VEC>(yb, p + to_b);
    }
  }
  mx::allow_next();
}

}  // namespace

dq_status rope(cudaStream_t stream, int dtype, const RopeArgs& in) {
  RopeArgs a = in;
  const bool vec = a.q.vec && a.q_out.vec && (!a.k.heads || (a.k.vec && a.k_out.vec));
  const int lanes = a.dim <= 64 ? 4 : a.dim <= 128 ? 8 : 16;
  const int groups = THREADS / lanes, parts = (a.q.heads + a.k.heads + groups - 1) / groups;
  // Few tokens: a CTA for each set of heads, so that none goes round twice; many: one CTA a token forms its angles once.
  a.splits = a.tokens * parts <= 592 ? parts : 1;
  mx::LaunchConfig c(stream, a.tokens * a.splits, THREADS);
  return by_type(dtype, [&](auto t) {
    using T = decltype(t);
    if (lanes == 4) return vec ? mx::launch(c, rope_kernel<T, 4, true>, a) : mx::launch(c, rope_kernel<T, 4, false>, a);
    if (lanes == 8) return vec ? mx::launch(c, rope_kernel<T, 8, true>, a) : mx::launch(c, rope_kernel<T, 8, false>, a);
    return vec ? mx::launch(c, rope_kernel<T, 16, true>, a) : mx::launch(c, rope_kernel<T, 16, false>, a);
  });
}

}  // namespace kv
}  // namespace dq
