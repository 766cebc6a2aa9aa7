// The key/value cache in 4 bits: writing (dq_kv_append), reading back (dq_kv_dequantize) and eviction (dq_kv_evict).
//
// Quantiser, for the D values of a token's key or value in one head:
//     offset = the largest bf16 number <= min x,   scale = the smallest bf16 number >= (max x - offset) / 15,
//     code = rint((x - offset) / scale), 0 where scale is 0
// Rounding outwards keeps every value inside the grid, so no code is clamped, and bf16's range is that of the inputs.  A head
// with a NaN or an infinity, or a range past fp32's, gets a scale of NaN and reads back as NaN.
//
// Bound by HBM and instructions alike: 2 D bytes read and D / 2 + 4 written for each key and each value in 16 bits (and 2 D where the
// values that the codes stand for are asked for).  A lane takes 16 values, D / 16 lanes a head; a CTA takes some tokens, for which it
// finds sequence, slot and page first.  12 prompts of up to 2048 tokens, 40 heads of 128, fp16, with the values: 148 to 153 us, 4.8 TB/s, a
// scheduler issues 70 % of the time (207 us without the next head's values on their way and the packed arithmetic).
#include "kv_common.cuh"

namespace dq {
namespace kv {
namespace {

using mx::Vec8;
using mx::from_f32;
using mx::to_f32;

constexpr int THREADS = 256;
constexpr int TILE = 32;      // tokens of a CTA at most

__device__ __forceinline__ float bf16_below(float v) {
  const uint32_t w = __float_as_uint(v), cut = w & 0xffff0000u;
  return __uint_as_float((int)w < 0 && cut != w ? cut + 0x10000u : cut);
}

template <typename T>
__device__ __forceinline__ void load16(Vec8<T>& a, Vec8<T>& b, const T* p, bool vec) {
  if (vec) {
    a.load(p);
    b.load(p + 8);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      a.set_pair(i, make_float2(to_f32(p[2 * i]), to_f32(p[2 * i + 1])));
      b.set_pair(i, make_float2(to_f32(p[8 + 2 * i]), to_f32(p[8 + 2 * i + 1])));
    }
  }
}
template <typename T>
__device__ __forceinline__ void store16(const float2 (&x)[8], T* p, bool vec) {
  if (vec) {
    Vec8<T> a, b;
#pragma unroll
    for (int i = 0; i < 4; ++i) { a.set_pair(i, x[i]); b.set_pair(i, x[4 + i]); }
    a.store(p);
    b.store(p + 8);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) { p[2 * i] = from_f32<T>(x[i].x); p[2 * i + 1] = from_f32<T>(x[i].y); }
  }
}

__device__ __forceinline__ float min_nan(float a, float b) { float d; asm("min.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b)); return d; }
__device__ __forceinline__ float max_nan(float a, float b) { float d; asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b)); return d; }

// Where the tokens of a CTA lie: the first kv head's group of a token's slot (null: in no page), and whether it is a sequence's.
struct Place { uint8_t* group; int in_group, there; };
__device__ __forceinline__ Place place_of(const AppendArgs& a, int64_t t, int dim) {
  Place at{nullptr, 0, 0};
  const int b = t < a.batch.tokens ? a.batch.sequence(t) : -1;
  if (b < 0) return at;
  int64_t first;
  int n;
  a.batch.range(b, first, n);
  if (t < first || t >= first + n) return at;
  at.there = 1;
  const int length = a.cache.length(b);
  const int64_t slot = length - n + (t - first);
  if (slot < 0) return at;
  at.in_group = (int)slot & (GROUP - 1);
  const int64_t page = a.cache.page_of(b, (int)slot);
  if (page >= 0) at.group = a.cache.group_at(page, 0, (int)slot, dim);
  if (a.slot_positions)
    for (int h = 0; h < a.cache.heads; ++h)
      a.slot_positions[((int64_t)b * a.cache.heads + h) * a.ld_slots + slot] = a.positions ? a.positions[t] : (int)slot;
  return at;
}

// WRITE: values are quantised into the cache; otherwise read back from it.
template <typename T, int DIM, bool WRITE>
__global__ void __launch_bounds__(THREADS) append_kernel(const AppendArgs a, int tile) {
  constexpr int LANES = DIM / 16, GROUPS = THREADS / LANES, HALF = GROUP * (DIM / 2 + 4);
  __shared__ Place s_place[TILE];
  const int l = threadIdx.x % LANES;
  const int64_t t0 = (int64_t)blockIdx.x * tile;
  const int heads = a.cache.heads, jobs = tile * 2 * heads;
  mx::wait_for_previous();
  mx::allow_next();
  if ((int)threadIdx.x < tile) s_place[threadIdx.x] = place_of(a, t0 + threadIdx.x, DIM);
  __syncthreads();
  struct Job { int i, which; };                                // a tile's token; a head's key, or from `heads` on its value
  const int i_step = GROUPS / (2 * heads), which_step = GROUPS % (2 * heads);
  auto next = [&](Job k) {
    k.i += i_step;
    k.which += which_step;
    if (k.which >= 2 * heads) { k.which -= 2 * heads; ++k.i; }
    return k;
  };
  Vec8<T> va, vb;                                              // the next job's values
  auto fetch = [&](const Job& k) {
    va.clear();
    vb.clear();
    if (!WRITE || k.i >= tile || !s_place[k.i].there) return;
    const Heads& src = k.which >= heads ? a.v : a.k;
    load16<T>(va, vb, reinterpret_cast<const T*>(src.p) + (t0 + k.i) * src.token + (k.which >= heads ? k.which - heads : k.which) * src.head + l * 16, src.vec);
  };
  Job job{(int)(threadIdx.x / LANES) / (2 * heads), (int)(threadIdx.x / LANES) % (2 * heads)};
  fetch(job);
  for (int j0 = 0; j0 < jobs; j0 += GROUPS, job = next(job)) {   // all lanes of a warp go round equally often
    const int i = job.i, which = job.which;
    const bool value = which >= heads;
    const int h = value ? which - heads : which;
    const Place at = i < tile ? s_place[i] : Place{nullptr, 0, 0};
    const Heads& src = value ? a.v : a.k;
    const int64_t t = t0 + i;
    uint8_t* group = at.group ? at.group + h * a.cache.page_bytes + (value ? HALF : 0) : nullptr;
    float2 x[8];
    if constexpr (!WRITE) {
      if (!at.there) continue;
      float scale = 0.f, offset = 0.f;
      uint2 w = make_uint2(0u, 0u);
      if (group) {
        w = *reinterpret_cast<const uint2*>(group + at.in_group * (DIM / 2) + l * 8);
        const uint32_t p = *reinterpret_cast<const uint32_t*>(group + GROUP * (DIM / 2) + at.in_group * 4);
        scale = scale_of(p);
        offset = offset_of(p);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {                              // (scale times a code is exact)
        const uint32_t c = (e < 4 ? w.x : w.y) >> (8 * (e & 3));
        x[e] = fma2(make_float2((float)(c & 15u), (float)((c >> 4) & 15u)), both(scale), both(offset));
      }
      store16<T>(x, reinterpret_cast<T*>(src.p) + t * src.token + h * src.head + l * 16, src.vec);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) { x[e] = va.pair(e); x[4 + e] = vb.pair(e); }
      fetch(next(job));
      float lo = x[0].x, hi = x[0].x;                            // NaN if any value is
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        lo = min_nan(lo, min_nan(x[e].x, x[e].y));
        hi = max_nan(hi, max_nan(x[e].x, x[e].y));
      }
#pragma unroll
      for (int d = 1; d < LANES; d <<= 1) {
        lo = min_nan(lo, __shfl_xor_sync(0xffffffffu, lo, d));
        hi = max_nan(hi, __shfl_xor_sync(0xffffffffu, hi, d));
      }
      float offset = bf16_below(lo + 0.f);                       // (-0 becomes 0)
      float scale = 0.f - bf16_below(-((hi - offset) / 15.f));
      constexpr float LARGEST = 3.402823466e38f;
      const bool good = lo >= -LARGEST && hi <= LARGEST && scale <= LARGEST;
      uint32_t w[2] = {0u, 0u};
      if (good && scale > 0.f) {
        // A sum with 1.5 2^23 rounds to an integer, which stands in its lowest bits.  The quotient by the reciprocal is off by two
        // roundings, 15 x 2 x 2^-24 at most: near a half, where that could decide, and where the reciprocal might be out of range, the
        // division itself.
        constexpr float MAGIC = 12582912.f;
        constexpr uint32_t BITS = 0x4b400000u;
        const float inverse = 1.f / scale;
        float2 d[8], c[8];
        const float near = scale > 1e-36f ? 0.49999f : -1.f;
        constexpr uint32_t ALL = BITS * 0x11111111u;             // what the eight sums' upper bits add up to
        w[0] = w[1] = 0u - ALL;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          d[e] = add2(x[e], both(-offset));
          float2 sum = fma2(d[e], both(inverse), both(MAGIC));
          c[e] = add2(sum, both(-MAGIC));
          const float2 rest = fma2(d[e], both(inverse), make_float2(-c[e].x, -c[e].y));
          if (!(fmaxf(fabsf(rest.x), fabsf(rest.y)) <= near)) {   // (inputs of 16 bits often lie at a half exactly)
            sum = make_float2(rintf(__fdiv_rn(d[e].x, scale)) + MAGIC, rintf(__fdiv_rn(d[e].y, scale)) + MAGIC);
            c[e] = add2(sum, both(-MAGIC));
          }
          w[e >> 2] += __float_as_uint(sum.x) * (1u << (8 * (e & 3))) + __float_as_uint(sum.y) * (16u << (8 * (e & 3)));
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = fma2(c[e], both(scale), both(offset));
      } else {
        if (!good) scale = offset = __uint_as_float(0x7fc00000u);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = both(offset);
      }
      if (group) {
        *reinterpret_cast<uint2*>(group + at.in_group * (DIM / 2) + l * 8) = make_uint2(w[0], w[1]);
        if (l == 0)
          *reinterpret_cast<uint32_t*>(group + GROUP * (DIM / 2) + at.in_group * 4) =
              (__float_as_uint(scale) >> 16) | (__float_as_uint(offset) & 0xffff0000u);
      }
      const Heads& dst = value ? a.v_values : a.k_values;
      if (at.there && dst.p) store16<T>(x, reinterpret_cast<T*>(dst.p) + t * dst.token + h * dst.head + l * 16, dst.vec);
    }
  }
}

template <bool WRITE>
dq_status run_append(cudaStream_t stream, const mx::Device& dev, int dtype, int dim, const AppendArgs& a) {
  // A CTA's search of sequences and pages (a chain of five loads or so) is paid once a tile: as many tokens as leave four CTAs an SM.
  const int64_t at_once = 4 * (int64_t)dev.sms, waves = (a.batch.tokens + TILE * at_once - 1) / (TILE * at_once);
  const int tile = (int)max((int64_t)1, min((int64_t)TILE, (a.batch.tokens + waves * at_once - 1) / (waves * at_once)));
  return by_type(dtype, [&](auto t) {
    using T = decltype(t);
    return by_dim(dim, [&](auto d) {
      mx::LaunchConfig c(stream, (a.batch.tokens + tile - 1) / tile, THREADS);
      return mx::launch(c, append_kernel<T, decltype(d)::value, WRITE>, a, tile);
    });
  });
}

// ------------------------------------------------------------------------------------------------ eviction
// One CTA for each (sequence, kv head) finds the `keep` slots that stay: the order is (protected, weight, lower slot first).  A
// radix selection over the weights' order-preserving bits, 8 at a time, finds the key of the last one that stays and how many of
// its equals do.  A warp takes neighbouring slots, 32 at a time, and keeps their keys in registers, so that a row is read twice, votes
// number the equals, holes and movers of a warp and one scan each those of the warps before (rows of more than 32768 slots go round
// in blocks of that, and read their keys again).  Slots from `keep` on that stay move into the slots below that do not, the i-th into the i-th: what is moved is
// read from slots that nothing writes, so no order between the moves is needed, and a sequence that is over its budget by a
// few tokens moves a few.  A slot without a page has nothing to move: where its turn is a slot with one, what is there stays.
//
// 32 sequences up to 16384 slots, 8 heads of 128, 4096 stay: 119 to 121 us, 57 for the choice (256 rows are 1.7 waves of CTAs; half the
// threads a CTA were slower) and 52 for the moves (72 bytes at either end, in whole sectors 2.0 times the bytes).  One sequence over by
// eight: 9.9 us on the GPU, two launches and the choice's chain of counts.
constexpr int SELECT = 1024, PER_THREAD = 32, BLOCK = SELECT * PER_THREAD;

__device__ __forceinline__ uint32_t order_key(float w, int position, int64_t guarded_above) {
  if ((int64_t)position > guarded_above) return 0xffffffffu;
  if (w != w) return 0u;
  const uint32_t u = __float_as_uint(w + 0.f);                 // (-0 becomes 0)
  return (int)u < 0 ? ~u : u | 0x80000000u;
}

__global__ void __launch_bounds__(SELECT, 1) evict_select_kernel(const EvictArgs a) {
  __shared__ int s_count[2][256], s_pick[2], s_newest[SELECT / 32];
  __shared__ int64_t s_scan[SELECT / 32];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int64_t row = blockIdx.x;                              // sequence x heads + head
  const int b = (int)(row / a.cache.heads);
  if (tid < 256) s_count[0][tid] = 0;
  mx::wait_for_previous();
  mx::allow_next();
  const int n = a.cache.length(b), keep = min(n, a.keep);
  const float* weights = a.weights + row * a.ld_slots;
  const int* positions = a.positions + row * a.ld_slots;
  int* ws = a.workspace + row * evict_stride(a.keep);
  const int per = min(PER_THREAD, (n + SELECT - 1) / SELECT);   // slots of a thread in each block: mine + 32 j
  const int mine = warp * per * 32 + lane;
  int64_t guarded_above = 0;
  uint32_t last = 0u;      // the key of the last slot that stays
  int equals = n;          // how many slots with that key stay
  uint32_t key[PER_THREAD];
  auto load_keys = [&](int base) {
#pragma unroll
    for (int j = 0; j < PER_THREAD; ++j) {
      if (j >= per) break;
      const int i = base + mine + 32 * j;
      key[j] = i < n ? order_key(weights[i], positions[i], guarded_above) : 0u;
    }
  };
  if (n > keep) {
    int newest = INT_MIN;
    for (int i = tid; i < n; i += SELECT) newest = max(newest, positions[i]);
    newest = __reduce_max_sync(0xffffffffu, newest);
    if (lane == 0) s_newest[warp] = newest;
    __syncthreads();
    newest = __reduce_max_sync(0xffffffffu, lane < SELECT / 32 ? s_newest[lane] : INT_MIN);
    guarded_above = (int64_t)newest - a.recent;
    load_keys(0);
    int wanted = keep;
    for (int shift = 24, now = 0; shift >= 0; shift -= 8, now ^= 1) {
      const uint32_t known = shift == 24 ? 0u : 0xffffffffu << (shift + 8);
      for (int base = 0; base < n; base += BLOCK) {
        if (n > BLOCK) load_keys(base);
#pragma unroll
        for (int j = 0; j < PER_THREAD; ++j) {
          if (j >= per) break;
          if (base + mine + 32 * j < n && (key[j] & known) == last) atomicAdd(&s_count[now][(key[j] >> shift) & 255u], 1);
        }
      }
      if (tid < 256) s_count[now ^ 1][tid] = 0;
      __syncthreads();
      if (warp == 0) {   // from the largest digit down: the first at which the count reaches what is wanted
        int sum = 0;
        int c[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += c[i] = s_count[now][255 - (lane * 8 + i)];
        int upto = sum;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
          const int v = __shfl_up_sync(0xffffffffu, upto, d);
          if (lane >= d) upto += v;
        }
        int before = upto - sum;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if (before < wanted && before + c[i] >= wanted) { s_pick[0] = 255 - (lane * 8 + i); s_pick[1] = wanted - before; }
          before += c[i];
        }
      }
      __syncthreads();
      last |= (uint32_t)s_pick[0] << shift;
      wanted = s_pick[1];
    }
    equals = wanted;
  }
  float* weights_out = a.weights_out + row * a.ld_slots;
  int* positions_out = a.positions_out + row * a.ld_slots;
  // The sum over the warps before this one of a count that is the same in all lanes of a warp; two kinds in one number, 21 bits each
  // (a block has 2^15 slots).
  auto scan = [&](int64_t of_mine, int64_t& all) {
    __syncthreads();
    if (lane == 0) s_scan[warp] = of_mine;
    __syncthreads();
    const int64_t of_warp = lane < SELECT / 32 ? s_scan[lane] : 0;
    int64_t upto = of_warp;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int64_t v = __shfl_up_sync(0xffffffffu, upto, d);
      if (lane >= d) upto += v;
    }
    all = __shfl_sync(0xffffffffu, upto, 31);
    return __shfl_sync(0xffffffffu, upto - of_warp, warp);
  };
  constexpr int64_t MASK = ((int64_t)1 << 21) - 1;
  const uint32_t below = (1u << lane) - 1u;
  int same = 0, holes = 0, movers = 0;                          // in the blocks so far
  for (int base = 0; base < n; base += BLOCK) {
    if (n > keep && n > BLOCK) load_keys(base);
    int64_t all;
    uint32_t stays = 0u;                                        // bit j
    if (n > keep) {
      int count = 0;
#pragma unroll
      for (int j = 0; j < PER_THREAD; ++j) {
        if (j >= per) break;
        count += __popc(__ballot_sync(0xffffffffu, base + mine + 32 * j < n && key[j] == last));
      }
      int before = same + (int)scan(count, all);
      same += (int)all;
#pragma unroll
      for (int j = 0; j < PER_THREAD; ++j) {
        if (j >= per) break;
        const bool there = base + mine + 32 * j < n, equal = there && key[j] == last;
        const uint32_t votes = __ballot_sync(0xffffffffu, equal);
        if (there && (key[j] > last || (equal && before + __popc(votes & below) < equals))) stays |= 1u << j;
        before += __popc(votes);
      }
    } else {
#pragma unroll
      for (int j = 0; j < PER_THREAD; ++j) {
        if (j >= per) break;
        if (base + mine + 32 * j < n) stays |= 1u << j;
      }
    }
    int64_t kinds = 0;
#pragma unroll
    for (int j = 0; j < PER_THREAD; ++j) {
      if (j >= per) break;
      const int i = base + mine + 32 * j;
      const bool stay = stays >> j & 1u;
      kinds += __popc(__ballot_sync(0xffffffffu, i < keep && !stay)) + ((int64_t)__popc(__ballot_sync(0xffffffffu, i >= keep && stay)) << 21);
    }
    const int64_t at = scan(kinds, all);
    int hole = holes + (int)(at & MASK), mover = movers + (int)(at >> 21);
    holes += (int)(all & MASK);
    movers += (int)(all >> 21);
#pragma unroll
    for (int j = 0; j < PER_THREAD; ++j) {
      if (j >= per) break;
      const int i = base + mine + 32 * j;
      const bool stay = stays >> j & 1u, is_hole = i < keep && !stay, is_mover = i >= keep && stay;
      const uint32_t h_votes = __ballot_sync(0xffffffffu, is_hole), m_votes = __ballot_sync(0xffffffffu, is_mover);
      if (is_hole) ws[4 + 2 * (hole + __popc(h_votes & below)) + 1] = i;
      if (is_mover) ws[4 + 2 * (mover + __popc(m_votes & below))] = i;
      if (stay && i < keep) {
        weights_out[i] = weights[i];
        positions_out[i] = positions[i];
      }
      hole += __popc(h_votes);
      mover += __popc(m_votes);
    }
  }
  if (tid == 0) ws[0] = movers;
  __syncthreads();
  for (int i = tid; i < movers; i += SELECT) {
    // (without codes to bring along, the slot's weight and position must not come to lie on another token's)
    const int from = ws[4 + 2 * i], to = ws[4 + 2 * i + 1];
    float w = weights[from];
    int position = positions[from];
    if (a.cache.page_of(b, from) < 0 && a.cache.page_of(b, to) >= 0) {
      w = weights[to];
      position = positions[to];
    }
    weights_out[to] = w;
    positions_out[to] = position;
  }
}

template <int DIM>
__global__ void __launch_bounds__(THREADS) evict_move_kernel(const EvictArgs a, int parts) {
  constexpr int LANES = DIM / 16, GROUPS = THREADS / LANES, HALF = GROUP * (DIM / 2 + 4);
  const int64_t row = blockIdx.x / parts;
  const int part = blockIdx.x % parts, b = (int)(row / a.cache.heads), h = (int)(row % a.cache.heads);
  const int l = threadIdx.x % LANES;
  mx::wait_for_previous();
  mx::allow_next();
  const int* ws = a.workspace + row * evict_stride(a.keep);
  const int moves = ws[0];
  const int half = l >= LANES / 2 ? HALF : 0, chunk = l % (LANES / 2);
  constexpr int AT_ONCE = 4;                                   // moves whose chains of loads go side by side
  for (int i0 = part * GROUPS + threadIdx.x / LANES; i0 < moves; i0 += AT_ONCE * parts * GROUPS) {
    const uint8_t* src[AT_ONCE];
    uint8_t* dst[AT_ONCE];
    int f[AT_ONCE], t[AT_ONCE];
#pragma unroll
    for (int x = 0; x < AT_ONCE; ++x) {
      const int i = i0 + x * parts * GROUPS;
      src[x] = nullptr;
      if (i >= moves) continue;
      const int from = ws[4 + 2 * i], to = ws[4 + 2 * i + 1];
      const int64_t from_page = a.cache.page_of(b, from), to_page = a.cache.page_of(b, to);
      if (from_page < 0 || to_page < 0) continue;
      src[x] = a.cache.group_at(from_page, h, from, DIM) + half;
      dst[x] = a.cache.group_at(to_page, h, to, DIM) + half;
      f[x] = from & (GROUP - 1);
      t[x] = to & (GROUP - 1);
    }
    uint4 codes[AT_ONCE];
    uint32_t p[AT_ONCE];
#pragma unroll
    for (int x = 0; x < AT_ONCE; ++x)
      if (src[x]) {
        codes[x] = *reinterpret_cast<const uint4*>(src[x] + f[x] * (DIM / 2) + chunk * 16);
        if (chunk == 0) p[x] = *reinterpret_cast<const uint32_t*>(src[x] + GROUP * (DIM / 2) + f[x] * 4);
      }
#pragma unroll
    for (int x = 0; x < AT_ONCE; ++x)
      if (src[x]) {
        *reinterpret_cast<uint4*>(dst[x] + t[x] * (DIM / 2) + chunk * 16) = codes[x];
        if (chunk == 0) *reinterpret_cast<uint32_t*>(dst[x] + GROUP * (DIM / 2) + t[x] * 4) = p[x];
      }
  }
  if (h == 0 && part == 0 && threadIdx.x == 0) a.lengths_out[b] = min(a.cache.length(b), a.keep);   // (may be the lengths themselves)
}

}  // namespace

dq_status append(cudaStream_t stream, const mx::Device& dev, int dtype, int dim, const AppendArgs& a) {
  return run_append<true>(stream, dev, dtype, dim, a);
}
dq_status dequantize(cudaStream_t stream, const mx::Device& dev, int dtype, int dim, const AppendArgs& a) {
  return run_append<false>(stream, dev, dtype, dim, a);
}

dq_status evict(cudaStream_t stream, const mx::Device& dev, int dim, const EvictArgs& a) {
  const int64_t rows = (int64_t)a.cache.n_seqs * a.cache.heads;
  {
    mx::LaunchConfig c(stream, rows, SELECT);
    DQ_CHECK(mx::launch(c, evict_select_kernel, a));
  }
  // eight CTAs an SM at most, and none without a round of moves
  const int groups = THREADS / (dim / 16);
  const int parts = (int)max((int64_t)1, min((int64_t)(a.keep + groups - 1) / groups, (8 * (int64_t)dev.sms + rows - 1) / rows));
  mx::LaunchConfig c(stream, rows * parts, THREADS);
  return by_dim(dim, [&](auto d) { return mx::launch(c, evict_move_kernel<decltype(d)::value>, a, parts); });
}

}  // namespace kv
}  // namespace dq
