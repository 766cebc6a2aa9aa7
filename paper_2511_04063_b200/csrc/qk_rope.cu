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

constexpr int MAX_THREADS = 256, MIN_CTAS = 3;   // (80 registers: at 120, as the compiler would, 16384 x 72 heads take 247 us, at 64 192)

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
// A lane's 16 values of gamma.
template <typename G>
__device__ __forceinline__ void load_gamma(float2 (&x)[8], const G* gamma, bool vec, int a, int b) {
  Vec8<G> v, w;
  if (vec) {
    v.load(gamma + a);
    w.load(gamma + b);
  } else {
    load8<G, false>(v, gamma + a);
    load8<G, false>(w, gamma + b);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) { x[i] = v.pair(i); x[4 + i] = w.pair(i); }
}

// LANES: lanes a head; those past D / 16 hold nothing.  A CTA takes every (splits x groups)-th head of one token.
template <typename T, int LANES, bool VEC>
__global__ void __launch_bounds__(MAX_THREADS, MIN_CTAS) rope_kernel(const RopeArgs a) {
  __shared__ float s_cos[128], s_sin[128];
  __shared__ float s_turn[MAX_THREADS * 16];
  const int groups = blockDim.x / LANES, stride = a.splits * groups;
  const int64_t t = blockIdx.x / a.splits;
  const int part = blockIdx.x % a.splits;
  const int l = threadIdx.x % LANES;
  const int half = a.rot >> 1;
  const bool halves = !(a.flags & DQ_QK_NEIGHBOURS), norm = a.flags & DQ_QK_NORM, hadamard = a.flags & DQ_QK_HADAMARD;
  const bool held = l * 16 < a.dim, rotated = l * 16 < a.rot;
  const int at_a = halves && rotated ? 8 * l : 16 * l, at_b = halves && rotated ? half + 8 * l : 16 * l + 8;
  const int q_heads = a.q.heads, heads = q_heads + a.k.heads;
  T* const q0 = reinterpret_cast<T*>(a.q.p) + t * a.q.token;
  T* const k0 = reinterpret_cast<T*>(a.k.p) + t * a.k.token - (int64_t)q_heads * a.k.head;
  T* const q1 = reinterpret_cast<T*>(a.q_out.p) + t * a.q_out.token;
  T* const k1 = reinterpret_cast<T*>(a.k_out.p) + t * a.k_out.token - (int64_t)q_heads * a.k_out.head;
  Vec8<T> va, vb;
  va.clear(); vb.clear();
  auto fetch = [&](int j) {
    if (j < heads && held) {
      const T* p = j < q_heads ? q0 + j * a.q.head : k0 + j * a.k.head;
      load8<T, VEC>(va, p + at_a);
      load8<T, VEC>(vb, p + at_b);
    }
  };
  mx::wait_for_previous();
  mx::allow_next();
  int j = part * groups + threadIdx.x / LANES;
  fetch(j);
  float2 gamma[8];
  const void* gammas_of = nullptr;                                     // whose gamma that is
  auto fetch_gamma = [&]() {
    const void* mine = j < q_heads ? a.q_gamma : a.k_gamma;
    if (!mine)
#pragma unroll
      for (int i = 0; i < 8; ++i) gamma[i] = both(1.f);
    else if (a.gamma_fp32) load_gamma(gamma, reinterpret_cast<const float*>(mine), a.gamma_vec, at_a, at_b);
    else load_gamma(gamma, reinterpret_cast<const T*>(mine), a.gamma_vec, at_a, at_b);
    gammas_of = mine;
  };
  if (norm && held) fetch_gamma();
  if (half) {
    for (int i = threadIdx.x; i < half; i += blockDim.x) {
      constexpr double TURNS = 0.15915494309189533577;                  // 1 / (2 pi)
      const double turn = (double)a.positions[t] * (double)a.inv_freq[i] * TURNS;
      float s, c;
      sincospif(2.f * (float)(turn - rint(turn)), &s, &c);
      s_cos[i] = c;
      s_sin[i] = s;
    }
    __syncthreads();
  }
  float2 cosine[4], sine[4];                                           // of this lane's eight pairs, the same for all heads
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    cosine[i] = rotated ? make_float2(s_cos[8 * l + 2 * i], s_cos[8 * l + 2 * i + 1]) : both(1.f);
    sine[i] = rotated ? make_float2(s_sin[8 * l + 2 * i], s_sin[8 * l + 2 * i + 1]) : both(0.f);
  }
  const float over = 1.f / (float)a.dim;
  const float down = hadamard ? rsqrtf((float)a.dim) : 1.f;            // (everything behind the norm is linear)
  // all lanes of a warp go round equally often: they exchange values
  for (int first = j - (threadIdx.x % 32) / LANES; first < heads; first += stride, j += stride) {
    float2 x[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[i] = va.pair(i); x[4 + i] = vb.pair(i); }
    fetch(j + stride);
    if (norm) {
      float2 sum = mul2(x[0], x[0]);
#pragma unroll
      for (int i = 1; i < 8; ++i) sum = fma2(x[i], x[i], sum);
      float s = sum.x + sum.y;
#pragma unroll
      for (int d = 1; d < LANES; d <<= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
      const float by = rsqrtf(s * over + a.eps) * down;
      if (held && (j < q_heads ? a.q_gamma : a.k_gamma) != gammas_of) fetch_gamma();
      if (held)
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = mul2(mul2(x[i], both(by)), gamma[i]);
    } else if (hadamard) {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = mul2(x[i], both(down));
    }
    if (rotated) {
      if (halves)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float2 p = x[i], q = x[4 + i], minus = make_float2(-sine[i].x, -sine[i].y);
          x[i] = fma2(q, minus, mul2(p, cosine[i]));
          x[4 + i] = fma2(p, sine[i], mul2(q, cosine[i]));
        }
      else
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float c = i & 1 ? cosine[i >> 1].y : cosine[i >> 1].x, s = i & 1 ? sine[i >> 1].y : sine[i >> 1].x;
          x[i] = fma2(make_float2(x[i].y, x[i].x), make_float2(-s, s), mul2(x[i], both(c)));
        }
    }
    int to_a = at_a, to_b = at_b;
    if (hadamard) {
      if (halves && half && a.rot < a.dim) {   // lanes that hold different bits of the index: to neighbours first
        float* turn = s_turn + (threadIdx.x - l) * 16;
        if (held)
#pragma unroll
          for (int i = 0; i < 8; ++i) *reinterpret_cast<float2*>(turn + (i < 4 ? at_a : at_b - 8) + 2 * i) = x[i];
        __syncwarp();
        to_a = 16 * l; to_b = 16 * l + 8;
        if (held)
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] = *reinterpret_cast<const float2*>(turn + to_a + 2 * i);
        __syncwarp();
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = make_float2(x[i].x + x[i].y, x[i].x - x[i].y);
#pragma unroll
      for (int d = 1; d < 8; d <<= 1)
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (!(i & d)) {
            const float2 u = x[i], v = x[i + d];
            x[i] = add2(u, v);
            x[i + d] = fma2(v, both(-1.f), u);
          }
#pragma unroll
      for (int d = 1; d < LANES; d <<= 1) {
        const float2 sign = both((l & d) ? -1.f : 1.f);
#pragma unroll
        for (int i = 0; i < 8; ++i)
          x[i] = fma2(x[i], sign, make_float2(__shfl_xor_sync(0xffffffffu, x[i].x, d), __shfl_xor_sync(0xffffffffu, x[i].y, d)));
      }
    }
    if (j < heads && held) {
      Vec8<T> ya, yb;
#pragma unroll
      for (int i = 0; i < 4; ++i) { ya.set_pair(i, x[i]); yb.set_pair(i, x[4 + i]); }
      T* p = j < q_heads ? q1 + j * a.q_out.head : k1 + j * a.k_out.head;
      store8<T, VEC>(ya, p + to_a);
      store8<T, VEC>(yb, p + to_b);
    }
  }
}

}  // namespace

dq_status rope(cudaStream_t stream, int dtype, const RopeArgs& in) {
  RopeArgs a = in;
  const bool vec = a.q.vec && a.q_out.vec && (!a.k.heads || (a.k.vec && a.k_out.vec));
  const int lanes = a.dim <= 64 ? 4 : a.dim <= 128 ? 8 : 16;
  // Few tokens: a CTA for each set of heads, so that none goes round twice; many: one CTA a token forms its angles once, with as many
  // lanes as leave the fewest idle in the last round.
  const int heads = a.q.heads + a.k.heads, at_once = 32 / lanes, most = MAX_THREADS / lanes, rounds = (heads + most - 1) / most;
  a.gamma_vec = (((uintptr_t)a.q_gamma | (uintptr_t)a.k_gamma) & 15) == 0;
  a.splits = a.tokens * rounds <= 592 ? rounds : 1;
  const int groups = ((heads + rounds - 1) / rounds + at_once - 1) / at_once * at_once;
  mx::LaunchConfig c(stream, a.tokens * a.splits, groups * lanes);
  return by_type(dtype, [&](auto t) {
    using T = decltype(t);
    if (lanes == 4) return vec ? mx::launch(c, rope_kernel<T, 4, true>, a) : mx::launch(c, rope_kernel<T, 4, false>, a);
    if (lanes == 8) return vec ? mx::launch(c, rope_kernel<T, 8, true>, a) : mx::launch(c, rope_kernel<T, 8, false>, a);
    return vec ? mx::launch(c, rope_kernel<T, 16, true>, a) : mx::launch(c, rope_kernel<T, 16, false>, a);
  });
}

}  // namespace kv
}  // namespace dq
