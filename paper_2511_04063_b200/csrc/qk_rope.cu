// Queries and keys of each head (dq_qk_norm_rope): root-mean-square norm, rotation by position, Hadamard rotation, in one pass.
//
//   h = x / sqrt(mean x^2 + eps) gamma;  (a, b) -> (a cos t - b sin t, b cos t + a sin t), t = position inv_freq[i];  y = h H / sqrt(D)
//
// A lane holds 16 values of a head, D / 16 lanes a head, chosen so that every rotated pair lies in one lane: the pieces 8 l and
// rot / 2 + 8 l for pairs of halves, 16 l for neighbours.  With the Hadamard rotation, a butterfly over the bits of the index, they are
// eight pairs of neighbours D / 8 apart (through shared memory where the rotated pairs do not allow it): four bits are a lane's own,
// then the lanes exchange their values once, through shared memory, take 16 neighbours each, and the other bits are their own.  (An
// exchange of all values for each of those bits took 187 us for 16384 tokens of 72 heads of 128 when this took 170, before a warp took a token.)
//
// A warp takes all heads of a token where there are many, so that its angles are formed once, in 64 bits: position x inv_freq is exact
// there up to 2^-53, and at position 10^6 a product in fp32 would be off by 0.06.
//
// With the Hadamard rotation 16384 x 72 heads of 128 take 145 us, 4.15 TB/s: 340 instructions for 16 values a lane are about as long as the
// bytes, and neither is full (a scheduler issues 60 % of the time, with 34 % of an SM's warps and one head's loads ahead): latency.  Without it
// 16384 x 40 heads take 72 us, 4.7 TB/s.  Few tokens: latency (2.7 us).
#include "kv_common.cuh"

namespace dq {
namespace kv {
namespace {

using mx::Vec8;
using mx::from_f32;
using mx::to_f32;

constexpr int MAX_THREADS = 256, MIN_CTAS = 3;   // (80 registers: the compiler alone would take 120)

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
// Eight pairs of neighbours, STEP values apart.
template <typename T, bool VEC, int STEP>
__device__ __forceinline__ void load_pairs(Vec8<T>& a, Vec8<T>& b, const T* p) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    Vec8<T>& v = j < 4 ? a : b;
    const T* q = p + j * STEP;
    if constexpr (!VEC) v.set_pair(j & 3, make_float2(to_f32(q[0]), to_f32(q[1])));
    else if constexpr (sizeof(T) == 4) v.set_pair(j & 3, *reinterpret_cast<const float2*>(q));
    else v.w[j & 3] = *reinterpret_cast<const uint32_t*>(q);
  }
}
// A lane's 16 values of gamma.
template <bool SPREAD, int STEP, typename G>
__device__ __forceinline__ void load_gamma(float2 (&x)[8], const G* gamma, bool vec, int a, int b, int l) {
  Vec8<G> v, w;
  if (SPREAD) {
    if (vec) load_pairs<G, true, STEP>(v, w, gamma + 2 * l);
    else load_pairs<G, false, STEP>(v, w, gamma + 2 * l);
  } else if (vec) {
    v.load(gamma + a);
    w.load(gamma + b);
  } else {
    load8<G, false>(v, gamma + a);
    load8<G, false>(w, gamma + b);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) { x[i] = v.pair(i); x[4 + i] = w.pair(i); }
}

// A butterfly between x[j] and x[j + D].
template <int D>
__device__ __forceinline__ void butterfly(float2 (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (!(i & D)) {
      const float2 u = x[i], v = x[i + D];
      x[i] = add2(u, v);
      x[i + D] = fma2(v, both(-1.f), u);
    }
}

// LANES: lanes a head; those past D / 16 hold nothing.  A CTA takes every splits-th set of heads of one token.  SPREAD: a lane's
// values are pairs of neighbours, D / 8 apart, with the Hadamard rotation.
template <typename T, int LANES, bool VEC, bool SPREAD>
__global__ void __launch_bounds__(MAX_THREADS, MIN_CTAS) rope_kernel(const RopeArgs a) {
  __shared__ float s_cos[128], s_sin[128];
  // a head's values in pieces of four, the q-th at q ^ (q / 8 % 4), and its begin so that neither way has bank conflicts
  constexpr int STEP = 2 * LANES, PITCH = LANES * 16 + (LANES == 4 ? 8 : LANES == 8 ? 16 : 0);
  extern __shared__ __align__(16) float s_turn[];                       // [blockDim.x / LANES][PITCH]
  const int groups = blockDim.x / LANES, stride = a.splits * groups;
  const int64_t t = blockIdx.x / a.splits;
  const int part = blockIdx.x % a.splits;
  const int l = threadIdx.x % LANES;
  const int half = a.rot >> 1;
  const bool halves = !(a.flags & DQ_QK_NEIGHBOURS), norm = a.flags & DQ_QK_NORM, hadamard = SPREAD || (a.flags & DQ_QK_HADAMARD);
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
      if constexpr (SPREAD) load_pairs<T, VEC, STEP>(va, vb, p + 2 * l);
      else {
        load8<T, VEC>(va, p + at_a);
        load8<T, VEC>(vb, p + at_b);
      }
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
    else if (a.gamma_fp32) load_gamma<SPREAD, STEP>(gamma, reinterpret_cast<const float*>(mine), a.gamma_vec, at_a, at_b, l);
    else load_gamma<SPREAD, STEP>(gamma, reinterpret_cast<const T*>(mine), a.gamma_vec, at_a, at_b, l);
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
  const int apart = SPREAD && halves ? half / STEP : 0;                // x[j] and x[j + apart] are rotated together
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    cosine[i] = both(1.f);
    sine[i] = both(0.f);
    if constexpr (!SPREAD) {
      if (rotated) {
        cosine[i] = make_float2(s_cos[8 * l + 2 * i], s_cos[8 * l + 2 * i + 1]);
        sine[i] = make_float2(s_sin[8 * l + 2 * i], s_sin[8 * l + 2 * i + 1]);
      }
    } else if (halves) {
      if (i < apart) {
        cosine[i] = make_float2(s_cos[STEP * i + 2 * l], s_cos[STEP * i + 2 * l + 1]);
        sine[i] = make_float2(s_sin[STEP * i + 2 * l], s_sin[STEP * i + 2 * l + 1]);
      }
    } else {
      const int at0 = LANES * 2 * i + l, at1 = at0 + LANES;
      if (at0 < half) { cosine[i].x = s_cos[at0]; sine[i].x = s_sin[at0]; }
      if (at1 < half) { cosine[i].y = s_cos[at1]; sine[i].y = s_sin[at1]; }
    }
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
    auto turn_pair = [&](float2& p, float2& q, int i) {
      const float2 u = p, v = q;
      p = fma2(v, make_float2(-sine[i].x, -sine[i].y), mul2(u, cosine[i]));
      q = fma2(u, sine[i], mul2(v, cosine[i]));
    };
    if (SPREAD ? half != 0 : rotated) {
      if (!halves) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float c = i & 1 ? cosine[i >> 1].y : cosine[i >> 1].x, s = i & 1 ? sine[i >> 1].y : sine[i >> 1].x;
          x[i] = fma2(make_float2(x[i].y, x[i].x), make_float2(-s, s), mul2(x[i], both(c)));
        }
      } else if (!SPREAD || apart == 4) {
#pragma unroll
        for (int i = 0; i < 4; ++i) turn_pair(x[i], x[4 + i], i);
      } else if (apart == 2) {
        turn_pair(x[0], x[2], 0);
        turn_pair(x[1], x[3], 1);
      } else turn_pair(x[0], x[1], 0);
    }
    int to_a = at_a, to_b = at_b;
    if (hadamard) {
      // The index's lowest bit and its three highest are the lane's own, the others the lane's number: four stages; then the lane takes
      // 16 neighbours, and the bits above the lowest are its own.
      float* const row = s_turn + threadIdx.x / LANES * PITCH;
      auto piece = [&](int q) { return reinterpret_cast<float4*>(row) + (q ^ (q >> 3 & 3)); };
      auto pairs = [&](int i) { return reinterpret_cast<float2*>(piece((STEP / 4) * i + (l >> 1))) + (l & 1); };
      if constexpr (!SPREAD) {
        if (held)
#pragma unroll
          for (int i = 0; i < 4; ++i) *piece((i < 2 ? at_a : at_b - 8) / 4 + i) = make_float4(x[2 * i].x, x[2 * i].y, x[2 * i + 1].x, x[2 * i + 1].y);
        __syncwarp();
        if (held)
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] = *pairs(i);
        __syncwarp();
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = make_float2(x[i].x + x[i].y, x[i].x - x[i].y);
      butterfly<1>(x);
      butterfly<2>(x);
      butterfly<4>(x);
      if (held)
#pragma unroll
        for (int i = 0; i < 8; ++i) *pairs(i) = x[i];
      __syncwarp();
      to_a = 16 * l; to_b = 16 * l + 8;
      if (held)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float4 v = *piece(4 * l + i);
          x[2 * i] = make_float2(v.x, v.y);
          x[2 * i + 1] = make_float2(v.z, v.w);
        }
      __syncwarp();
      butterfly<1>(x);
      butterfly<2>(x);
      if (LANES >= 8) butterfly<4>(x);
      if (LANES == 16) {   // the fifth bit
        const float2 sign = both((l & 1) ? -1.f : 1.f);
#pragma unroll
        for (int i = 0; i < 8; ++i)
          x[i] = fma2(x[i], sign, make_float2(__shfl_xor_sync(0xffffffffu, x[i].x, 1), __shfl_xor_sync(0xffffffffu, x[i].y, 1)));
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

dq_status rope(cudaStream_t stream, const mx::Device& dev, int dtype, const RopeArgs& in) {
  RopeArgs a = in;
  const bool vec = a.q.vec && a.q_out.vec && (!a.k.heads || (a.k.vec && a.k_out.vec));
  const int lanes = a.dim <= 64 ? 4 : a.dim <= 128 ? 8 : 16;
  // Many tokens: a warp each, so that angles, gamma and addresses are formed once for as many heads as can be (16384 tokens of 72 heads:
  // 145 us, by six warps 171; 2048 tokens 25 us by one, 20.5 by three, 22.5 by six).  Few: warps enough for 48 an SM, and from 8 on
  // CTAs enough that no warp goes round twice.
  const int heads = a.q.heads + a.k.heads, at_once = 32 / lanes;
  const int warps = (int)max((int64_t)1, min((int64_t)MAX_THREADS / 32, (int64_t)dev.sms * 48 / a.tokens));
  const int most = warps * at_once, rounds = (heads + most - 1) / most;
  a.gamma_vec = (((uintptr_t)a.q_gamma | (uintptr_t)a.k_gamma) & 15) == 0;
  a.splits = a.tokens * rounds <= dev.sms * 4 ? rounds : 1;
  const int groups = ((heads + rounds - 1) / rounds + at_once - 1) / at_once * at_once;
  const int pitch = lanes * 16 + (lanes == 4 ? 8 : lanes == 8 ? 16 : 0);
  mx::LaunchConfig c(stream, a.tokens * a.splits, groups * lanes, a.flags & DQ_QK_HADAMARD ? groups * pitch * 4 : 0);
  // with a Hadamard rotation, where the rotated pairs lie in one lane so: neighbours, or rot of D, D / 2 or D / 4
  const int pair = a.flags & DQ_QK_NEIGHBOURS ? 0 : a.rot / 2, step = 2 * lanes;
  const bool spread = (a.flags & DQ_QK_HADAMARD) && (pair == 0 || pair == step || pair == 2 * step || pair == 4 * step);
  auto launch = [&](auto t, auto lanes, auto vec) {
    using T = decltype(t);
    constexpr int LANES = decltype(lanes)::value;
    constexpr bool VEC = decltype(vec)::value != 0;
    return spread ? mx::launch(c, rope_kernel<T, LANES, VEC, true>, a) : mx::launch(c, rope_kernel<T, LANES, VEC, false>, a);
  };
  return by_type(dtype, [&](auto t) {
    auto by_lanes = [&](auto vec) {
      if (lanes == 4) return launch(t, Number<4>(), vec);
      return lanes == 8 ? launch(t, Number<8>(), vec) : launch(t, Number<16>(), vec);
    };
    return vec ? by_lanes(Number<1>()) : by_lanes(Number<0>());
  });
}

}  // namespace kv
}  // namespace dq
