// Attention over a key/value cache in 4 bits (dq_kv_attention) and the weight each cached token received
// (dq_kv_attention_weights).
//
//     S = scale q k^T over the slots a query sees,   O = softmax(S) v,   lse = log sum exp S
//
// With k = ks c + ko for codes c = 0 .. 15,   q . k = ks (q . c) + ko sum q   and   sum_t p_t v_t = sum_t (p_t vs_t) c_t + sum_t p_t vo_t:
// the matrix instructions multiply the codes, and the parameters enter once for each key.  Four bits alone are an fp16 number,
// the subnormal c 2^-24 (c 2^-20 four bits further up), which the tensor cores multiply exactly: one AND turns two codes into two
// operands, and the powers of two are taken out with the parameters.  (Bits or'ed into the mantissa of 1024, less 1032, are three
// instructions; with them a token over 131072 slots took 107 us.)
//
// The keys are the rows (M) of the instructions and the query rows their columns (N = 8), so that the eight or fewer query heads
// of a kv head fill a tile: S^T = K Q^T, O^T = V^T P^T with mma.m16n8k16.  Any order of the dimensions serves the first product
// as long as Q has the same, any order of the keys the second as long as P has: a thread takes neighbouring codes of a key, as
// they lie, in both.  P^T comes out of the first product transposed and is turned by movmatrix.
//
// Roundings to 16 bits.  A query row is multiplied by a power of two that brings its largest value to 2^14 and rounded to fp16: exact
// for fp16's 11 and bf16's 8 bits, save values below 2^-24 of the largest.  P vs is divided by the power of two of the stage's
// largest vs and rounded to fp16 (2^-11 a term; below 2^-20 of the row's largest 2^-31 of it).  A stage's sum of P vs c starts
// from zero and is added in fp32: the instructions' own sums truncate, which over a long axis would add up.
#include "kv_common.cuh"
#include "tc_gemm.cuh"

namespace dq {
namespace kv {
namespace {

constexpr float LOG2E = 1.44269504088896f, LN2 = 0.693147180559945f;
constexpr int STAGE = 2 * GROUP;   // keys of a pipeline stage: the maximum of a row is looked at once for 32 keys

__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// Two codes as fp16 numbers, c 2^-24: bits 0-3 and 16-19; c 2^-20: bits 4-7 and 20-23.
__device__ __forceinline__ uint32_t low_codes(uint32_t w) { return w & 0x000f000fu; }
__device__ __forceinline__ uint32_t high_codes(uint32_t w) { return w & 0x00f000f0u; }
__device__ __forceinline__ uint32_t transposed(uint32_t v) {
  uint32_t d;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(v));
  return d;
}
__device__ __forceinline__ float exp2_of(float v) {
  float d;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(d) : "f"(v));
  return d;
}
__device__ __forceinline__ uint32_t half_pair(float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
template <int WORDS>
__device__ __forceinline__ void load_words(uint32_t (&w)[WORDS], const uint8_t* p) {
  if (WORDS == 1) w[0] = *reinterpret_cast<const uint32_t*>(p);
  if (WORDS == 2) { const uint2 v = *reinterpret_cast<const uint2*>(p); w[0] = v.x; w[WORDS > 1 ? 1 : 0] = v.y; }
  if (WORDS >= 4)
#pragma unroll
    for (int i = 0; i + 3 < WORDS; i += 4) {
      const uint4 v = reinterpret_cast<const uint4*>(p)[i >> 2];
      w[i] = v.x; w[i + 1] = v.y; w[i + 2] = v.z; w[i + 3] = v.w;
    }
}
// The key (of a group's 16) that is row r of the first product and index r of the second's reduction.  Rows 2 a and 2 a + 1 lie
// 64 bytes apart modulo 128 so that a quarter of a warp reads its keys without bank conflicts.
__device__ __forceinline__ int key_of(int r) { const int c = (r & 7) >> 1; return (r & 8) + ((r & 1) ? (c ^ 1) + 4 : c); }

// Eight values of a row, zeros where there is none.
template <typename T>
__device__ __forceinline__ void load_values(float (&v)[8], const T* p, bool there, bool vec) {
  mx::Vec8<T> x;
  x.clear();
  if (there) {
    if (vec) x.load(p);
    else
#pragma unroll
      for (int i = 0; i < 4; ++i) x.set_pair(i, make_float2(mx::to_f32(p[2 * i]), mx::to_f32(p[2 * i + 1])));
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = x.pair(i);
    v[2 * i] = f.x; v[2 * i + 1] = f.y;
  }
}

// A warp's query rows: tile of 8 NT rows (row r: token r / group, head r % group) as B fragments.  Dimensions whose codes lie four
// bits up are held 2^-4 smaller.  For the columns 2 c and 2 c + 1: `by`, what takes the powers of two out of a product, and the
// sum of the row.
template <typename T, int DIM, int NT>
struct Queries {
  static constexpr int WORDS = DIM / 32;
  uint32_t b[NT][WORDS][4];
  float by[NT][2], sum[NT][2];
  __device__ __forceinline__ void load(const Heads& q, int64_t first, int rows, int row0, int h, int group, int lane) {
    const int c = lane & 3;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int r = row0 + nt * 8 + (lane >> 2);
      const bool there = r < rows;
      const int i = there ? r / group : 0;
      const T* p = reinterpret_cast<const T*>(q.p) + (first + i) * q.token + (int64_t)(h * group + (there ? r - i * group : 0)) * q.head;
      float v[WORDS][8], s = 0.f, most = 0.f;
#pragma unroll
      for (int w = 0; w < WORDS; ++w) {
        load_values<T>(v[w], p + (c * WORDS + w) * 8, there, q.vec);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          s += v[w][e];
          most = fmaxf(most, fabsf(v[w][e]));
        }
      }
      s += __shfl_xor_sync(0xffffffffu, s, 1);
      s += __shfl_xor_sync(0xffffffffu, s, 2);
      most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 1));
      most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 2));
      // the largest value's exponent field, within what keeps both factors normal numbers; a row that is not finite stays so
      const int field = min(max((int)mx::exponent_field(most), 14), 244);
      const float up = __uint_as_float((uint32_t)(268 - field) << 23), up4 = up * 0.0625f;
#pragma unroll
      for (int w = 0; w < WORDS; ++w)
#pragma unroll
        for (int e = 0; e < 4; ++e) b[nt][w][e] = half_pair(v[w][e] * (e & 1 ? up4 : up), v[w][e + 4] * (e & 1 ? up4 : up));
      const float down = __uint_as_float((uint32_t)(field + 10) << 23);   // 2^24 / up
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        sum[nt][j] = __shfl_sync(0xffffffffu, s, c * 8 + 4 * j);
        by[nt][j] = __shfl_sync(0xffffffffu, down, c * 8 + 4 * j);
      }
    }
  }
};

// (q . c) of a group's 16 keys and the tile's rows, without q.by: acc[nt] = (key_of(g), columns 2 c, 2 c + 1), (key_of(g + 8), the same).
template <typename T, int DIM, int NT>
__device__ __forceinline__ void key_products(float (&acc)[NT][4], const uint8_t* codes, const Queries<T, DIM, NT>& q, int lane) {
  constexpr int WORDS = DIM / 32;
  const int g = lane >> 2, c = lane & 3;
  uint32_t k0[WORDS], k1[WORDS];
  load_words<WORDS>(k0, codes + key_of(g) * (DIM / 2) + c * (DIM / 8));
  load_words<WORDS>(k1, codes + key_of(g + 8) * (DIM / 2) + c * (DIM / 8));
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[nt][i] = 0.f;
#pragma unroll
  for (int w = 0; w < WORDS; ++w)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const uint32_t x0 = k0[w] >> (8 * e), x1 = k1[w] >> (8 * e);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
        mma(acc[nt], low_codes(x0), low_codes(x1), high_codes(x0), high_codes(x1), q.b[nt][w][2 * e], q.b[nt][w][2 * e + 1]);
    }
}

// What an item of work is: a tile of query rows of a sequence and kv head, with `stages` stages of keys.
struct Item {
  int b, h, tile;
  int64_t first;
  int n, length, rows, tiles;
  int64_t stages;
};

// Sequence b's units of work: every tile of rows of every kv head, with the stages of its keys (one at least: rows that see
// nothing are written too).
template <int ROWS>
__device__ __forceinline__ void describe(Item& it, const AttentionArgs& a, int b) {
  it.b = b;
  a.batch.range(b, it.first, it.n);
  it.length = a.cache.length(b);
  it.rows = it.n * a.group;
  it.tiles = (it.rows + ROWS - 1) / ROWS;
  it.stages = max(1, (it.length + STAGE - 1) / STAGE);
}

// ------------------------------------------------------------------------------------------------ few rows
// A CTA takes an equal share of all stages of all items, whatever the sequences' lengths, and its warps take them in turn, each with its
// own maximum, sum and O^T, joined in shared memory at an item's end.  A warp brings its stages in by bulk copies into two places of
// its own: while it works on one the other is on its way, across items too.  An item that crosses CTAs is left in the workspace in parts,
// and the CTA that finishes last joins them, in order.
template <int DIM, int NT>
struct Few {
  static constexpr int ROWS = 8 * NT;
  static constexpr int WARPS = DIM == 256 || (DIM == 128 && NT == 2) ? 8 : 16;
  static constexpr int SLOTS = 2;
  static constexpr int THREADS = WARPS * 32;
  static constexpr int GROUP_BYTES = GROUP * (DIM + 8), STAGE_BYTES = 2 * GROUP_BYTES;
  static constexpr int PAD = DIM + 4;                                  // floats of a row of O, against bank conflicts
  static constexpr int RING_BYTES = WARPS * SLOTS * STAGE_BYTES;
  static constexpr int JOIN_BYTES = WARPS * ROWS * PAD * 4;
  static constexpr int SMEM = RING_BYTES + JOIN_BYTES;
  static constexpr int PART = ROWS * (DIM + 2);                        // floats of a part in the workspace: O, maxima, sums
};
constexpr int MAX_CTAS = 256;
constexpr int TICKET_BYTES = MAX_CTAS * 4;
constexpr int LEAST_STAGES = 8;                                        // of a CTA
constexpr float SLACK = 8.f;                                           // a maximum may grow by this (in powers of two) before O is rescaled

// A walk over the items in the order (sequence, head, tile).
template <int ROWS>
struct Walk {
  Item it;
  int seq;
  int64_t index, begin;                                                // of the sequence's items; the item's first unit
  __device__ __forceinline__ void start(const AttentionArgs& a, const Share& s) {
    seq = s.seq;
    describe<ROWS>(it, a, seq);
    index = (s.lo - s.before) / it.stages;
    begin = s.before + index * it.stages;
  }
  __device__ __forceinline__ void next(const AttentionArgs& a) {
    begin += it.stages;
    if (++index < (int64_t)it.tiles * a.cache.heads) return;
    index = 0;
    do {
      if (++seq == a.batch.n_seqs) return;
      describe<ROWS>(it, a, seq);
    } while (it.tiles == 0);
  }
};

template <typename T, int DIM, int NT>
__global__ void __launch_bounds__(Few<DIM, NT>::THREADS, 1) few_kernel(const AttentionArgs a) {
  using F = Few<DIM, NT>;
  constexpr int ROWS = F::ROWS, WARPS = F::WARPS, SLOTS = F::SLOTS, VW = DIM / 64;
  extern __shared__ __align__(128) uint8_t smem[];
  float* joined = reinterpret_cast<float*>(smem + F::RING_BYTES);
  __shared__ __align__(8) uint64_t s_full[WARPS][SLOTS];
  __shared__ int s_valid[WARPS][SLOTS];
  struct Fetch { Walk<ROWS> walk; int64_t unit; int issued; };
  __shared__ Fetch s_fetch[WARPS];                                     // of what a warp brings in next; its first lane's
  __shared__ Share s_share;
  __shared__ int64_t s_sums[WARPS];
  __shared__ float s_max[WARPS][ROWS], s_sum[WARPS][ROWS];
  __shared__ int s_last;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (tid < WARPS * SLOTS) tc::mbar_init(tc::smem_u32(&s_full[0][0]) + tid * 8, 1);
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  mx::wait_for_previous();
  mx::allow_next();
  find_share(&s_share, a.batch.n_seqs, LEAST_STAGES, s_sums, [&](int b) {
    Item it;
    describe<ROWS>(it, a, b);
    return (int64_t)it.tiles * a.cache.heads * it.stages;
  });
  const Share share = s_share;
  if (share.lo >= share.hi) return;

  const uint32_t full0 = tc::smem_u32(&s_full[warp][0]);
  uint8_t* const ring = smem + warp * SLOTS * F::STAGE_BYTES;
  Walk<ROWS> at;
  at.start(a, share);
  auto fetch = [&](Fetch& f) {                                          // the warp's next stage, by its first lane
    if (f.unit >= share.hi) return;
    while (f.unit >= f.walk.begin + f.walk.it.stages) f.walk.next(a);
    const Item& it = f.walk.it;
    const int h = (int)(f.walk.index / it.tiles), slot = (int)(f.unit - f.walk.begin) * STAGE, place = f.issued % SLOTS;
    const int64_t p0 = slot < it.length ? a.cache.page_of(it.b, slot) : -1;
    const int64_t p1 = slot + GROUP < it.length ? a.cache.shift > 4 ? p0 : a.cache.page_of(it.b, slot + GROUP) : -1;
    const bool joint = a.cache.shift > 4 && p1 >= 0;                    // both groups in one page, one behind the other
    const uint32_t dst = tc::smem_u32(ring + place * F::STAGE_BYTES), bar = full0 + place * 8;
    auto copy = [&](uint32_t to, const uint8_t* from, uint32_t bytes) {
      asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                   ::"r"(to), "l"(from), "r"(bytes), "r"(bar) : "memory");
    };
    s_valid[warp][place] = (p0 >= 0 ? 1 : 0) | (p1 >= 0 ? 2 : 0);
    tc::mbar_expect_tx(bar, ((p0 >= 0) + (p1 >= 0)) * F::GROUP_BYTES);
    if (p0 >= 0) copy(dst, a.cache.group_at(p0, h, slot, DIM), joint ? F::STAGE_BYTES : F::GROUP_BYTES);
    if (p1 >= 0 && !joint) copy(dst + F::GROUP_BYTES, a.cache.group_at(p1, h, slot + GROUP, DIM), F::GROUP_BYTES);
    f.unit += WARPS;
    ++f.issued;
  };
  if (lane == 0) {
    Fetch& f = s_fetch[warp];
    f.walk = at;
    f.unit = share.lo + warp;
    f.issued = 0;
    for (int i = 0; i < SLOTS; ++i) fetch(f);
  }
  __syncwarp();

  const int g = lane >> 2, c = lane & 3;
  const float to_log2 = a.scale * LOG2E;
  bool alive = true;
  int turn = 0;                                                         // stages of this warp so far
  Queries<T, DIM, NT> q;
  int64_t unit = share.lo + warp;                                       // this warp's next
  while (true) {
    const Item& it = at.it;
    const int64_t begin = at.begin;
    const int h = (int)(at.index / it.tiles), row0 = (int)(at.index % it.tiles) * ROWS;
    const bool starts = begin >= share.lo, ends = begin + it.stages <= share.hi;
    const int64_t until = min(begin + it.stages, share.hi);
    float top[NT][2], sum[NT][2], off[NT][2], o[NT][VW * 4][4];
    int sees[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        top[nt][j] = -INFINITY; sum[nt][j] = off[nt][j] = 0.f;
        const int r = row0 + nt * 8 + 2 * c + j;
        sees[nt][j] = r < it.rows ? max(it.length - it.n + r / a.group + 1, 0) : 0;
      }
    // all valid rows see the stages before the first row's end, none those past the last one's
    const int least = max(it.length - it.n + row0 / a.group + 1, 0);
    const int most = max(it.length - it.n + (min(row0 + ROWS, it.rows) - 1) / a.group + 1, 0);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int i = 0; i < VW * 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) o[nt][i][j] = 0.f;
    if (unit < until) q.load(a.q, it.first, it.rows, row0, h, a.group, lane);

    for (; unit < until; unit += WARPS) {
      const int place = turn % SLOTS;
      if (alive) alive = __all_sync(0xffffffffu, tc::mbar_wait(full0 + place * 8, (uint32_t)(turn / SLOTS) & 1u, a.d_status));
      if (!alive) continue;
      const int slot0 = (int)(unit - begin) * STAGE;
      if (slot0 < most) {
        const uint8_t* stage = ring + place * F::STAGE_BYTES;
        const int valid = s_valid[warp][place];
        const bool masked = slot0 + STAGE > least || valid != 3;
        float s[2][NT][4];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const uint8_t* group = stage + u * F::GROUP_BYTES;
          key_products<T, DIM, NT>(s[u], group, q, lane);
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const uint32_t p = *reinterpret_cast<const uint32_t*>(group + GROUP * (DIM / 2) + key_of(g + 8 * e) * 4);
            const float ks = scale_of(p) * to_log2, ko = offset_of(p) * to_log2;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int j = 0; j < 2; ++j) s[u][nt][2 * e + j] = s[u][nt][2 * e + j] * (ks * q.by[nt][j]) + ko * q.sum[nt][j];
          }
        }
        uint32_t vp[2][2];                                              // the values' parameters; a masked key's may be anything
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int e = 0; e < 2; ++e)
            vp[u][e] = *reinterpret_cast<const uint32_t*>(stage + u * F::GROUP_BYTES + GROUP * (DIM + 4) + key_of(g + 8 * e) * 4);
        if (masked)
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const int slot = (valid >> u & 1) ? slot0 + u * GROUP + key_of(g + 8 * e) : INT_MAX;
              if (slot >= it.length) vp[u][e] = 0u;
#pragma unroll
              for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int j = 0; j < 2; ++j)
                  if (slot >= sees[nt][j]) s[u][nt][2 * e + j] = -INFINITY;
            }
        // maxima over the stage's keys; O is rescaled where one has grown by more than SLACK
        bool grown = false;
        float now[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            float m = fmaxf(fmaxf(s[0][nt][j], s[0][nt][2 + j]), fmaxf(s[1][nt][j], s[1][nt][2 + j]));
            m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 4));
            m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 8));
            m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 16));
            now[nt][j] = m;
            grown |= m > top[nt][j] + SLACK;
          }
        if (__any_sync(0xffffffffu, grown))
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              const float m = fmaxf(top[nt][j], now[nt][j]);
              const float by = top[nt][j] == -INFINITY ? (sum[nt][j] == 0.f ? 0.f : 1.f) : exp2_of(top[nt][j] - m);
              top[nt][j] = m;
              sum[nt][j] *= by;
              off[nt][j] *= by;
#pragma unroll
              for (int i = 0; i < VW * 4; ++i) {
                o[nt][i][j] *= by;
                o[nt][i][2 + j] *= by;
              }
            }
        // the exponent field of the stage's largest vs (a NaN's does not count): vs 2^(6 - field + 127) < 2^7, and with p < 2^SLACK
        // P stays below 2^15
        uint32_t field = 7u;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const uint32_t f = vp[u][e] >> 7 & 255u;
            field = max(field, f == 255u ? 0u : f);
          }
        field = __reduce_max_sync(0xffffffffu, field);
        const float shrink = __uint_as_float((260u - field) << 23), grow = __uint_as_float((field - 6u) << 23);
        float part[NT][VW * 4][4];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int i = 0; i < VW * 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) part[nt][i][j] = 0.f;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const uint8_t* group = stage + u * F::GROUP_BYTES + GROUP * (DIM / 2 + 4);
          uint32_t b[NT][2];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float vs = scale_of(vp[u][e]) * shrink, vo = offset_of(vp[u][e]);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              float pv[2];
#pragma unroll
              for (int j = 0; j < 2; ++j) {
                const float x = s[u][nt][2 * e + j], m = top[nt][j];
                const float p = exp2_of(x - (m == -INFINITY ? 0.f : m));
                const bool gone = masked && x == -INFINITY;              // (its value may be a NaN that others see)
                sum[nt][j] += p;
                off[nt][j] += gone ? 0.f : p * vo;
                pv[j] = gone ? 0.f : p * vs;
              }
              b[nt][e] = transposed(half_pair(pv[0], pv[1]));
            }
          }
          uint32_t x[4][VW];
#pragma unroll
          for (int i = 0; i < 4; ++i) load_words<VW>(x[i], group + key_of(2 * c + (i & 1) + 8 * (i >> 1)) * (DIM / 2) + g * (DIM / 16));
#pragma unroll
          for (int w = 0; w < VW; ++w) {
            const uint32_t lo01 = __byte_perm(x[0][w], x[1][w], 0x5410), hi01 = __byte_perm(x[0][w], x[1][w], 0x7632);
            const uint32_t lo23 = __byte_perm(x[2][w], x[3][w], 0x5410), hi23 = __byte_perm(x[2][w], x[3][w], 0x7632);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const uint32_t a0 = lo01 >> (i & 2 ? 8 : 0), a1 = hi01 >> (i & 2 ? 8 : 0), a2 = lo23 >> (i & 2 ? 8 : 0), a3 = hi23 >> (i & 2 ? 8 : 0);
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) {
                if (i & 1) mma(part[nt][w * 4 + i], high_codes(a0), high_codes(a1), high_codes(a2), high_codes(a3), b[nt][0], b[nt][1]);
                else mma(part[nt][w * 4 + i], low_codes(a0), low_codes(a1), low_codes(a2), low_codes(a3), b[nt][0], b[nt][1]);
              }
            }
          }
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int i = 0; i < VW * 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) o[nt][i][j] += part[nt][i][j] * grow;
      }
      ++turn;
      __syncwarp();                                                     // all lanes have read the stage
      if (lane == 0) fetch(s_fetch[warp]);
      __syncwarp();
    }

    // ---- the item's rows over the warps
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) {
          sum[nt][j] += __shfl_xor_sync(0xffffffffu, sum[nt][j], d);
          off[nt][j] += __shfl_xor_sync(0xffffffffu, off[nt][j], d);
        }
        if (g == 0) { s_max[warp][nt * 8 + 2 * c + j] = top[nt][j]; s_sum[warp][nt * 8 + 2 * c + j] = sum[nt][j]; }
      }
    __syncthreads();
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int r = nt * 8 + 2 * c + j;
        if (s_sum[warp][r] == 0.f) continue;
        float m = -INFINITY;
        for (int w = 0; w < WARPS; ++w) m = fmaxf(m, s_max[w][r]);
        const float by = top[nt][j] == -INFINITY ? 1.f : exp2_of(top[nt][j] - m);
        float* row = joined + (warp * ROWS + r) * F::PAD + g * (DIM / 8);
        constexpr float LOW = 16777216.f, HIGH = 1048576.f;             // 2^24 and 2^20: of the codes
#pragma unroll
        for (int i = 0; i < VW; ++i)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float4 v;
            v.x = (o[nt][4 * i][2 * e + j] * LOW + off[nt][j]) * by; v.y = (o[nt][4 * i + 1][2 * e + j] * HIGH + off[nt][j]) * by;
            v.z = (o[nt][4 * i + 2][2 * e + j] * LOW + off[nt][j]) * by; v.w = (o[nt][4 * i + 3][2 * e + j] * HIGH + off[nt][j]) * by;
            *reinterpret_cast<float4*>(row + 8 * i + 4 * e) = v;
          }
      }
    __syncthreads();
    const int cta = blockIdx.x;
    const int first_cta = starts ? cta : cta_of(begin, share.total, share.ctas);
    const int last_cta = ends ? cta : cta_of(begin + it.stages - 1, share.total, share.ctas);
    const bool whole = first_cta == last_cta;
    float* parts = reinterpret_cast<float*>(a.workspace + TICKET_BYTES);
    auto part_of = [&](int i) { return parts + ((int64_t)i * 2 + (i == first_cta ? 1 : 0)) * F::PART; };
    auto write = [&](int r, int d, float4 v, float m, float l) {         // row r of the tile, dimensions d .. d + 3
      const int row = row0 + r;
      if (row >= it.rows) return;
      const int i = row / a.group, head = h * a.group + row - i * a.group;
      const float by = l == 0.f ? 0.f : 1.f / l;
      T* p = reinterpret_cast<T*>(a.out.p) + (it.first + i) * a.out.token + head * a.out.head + d;
      T y[4] = {mx::from_f32<T>(v.x * by), mx::from_f32<T>(v.y * by), mx::from_f32<T>(v.z * by), mx::from_f32<T>(v.w * by)};
      if (a.out.vec) { uint2 w; memcpy(&w, y, 8); *reinterpret_cast<uint2*>(p) = w; }
      else
#pragma unroll
        for (int e = 0; e < 4; ++e) p[e] = y[e];
      if (d == 0 && a.lse) a.lse[(it.first + i) * a.q.heads + head] = l == 0.f ? -INFINITY : (m + log2f(l)) * LN2;
    };
    for (int x = tid; x < ROWS * (DIM / 4); x += WARPS * 32) {
      const int r = x / (DIM / 4), d = x % (DIM / 4) * 4;
      float m = -INFINITY, l = 0.f;
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int w = 0; w < WARPS; ++w) m = fmaxf(m, s_max[w][r]);
      for (int w = 0; w < WARPS; ++w) {
        if (s_sum[w][r] == 0.f) continue;
        l += s_sum[w][r] * (s_max[w][r] == -INFINITY ? 1.f : exp2_of(s_max[w][r] - m));
        const float4 t = *reinterpret_cast<const float4*>(joined + (w * ROWS + r) * F::PAD + d);
        v.x += t.x; v.y += t.y; v.z += t.z; v.w += t.w;
      }
      if (whole) { write(r, d, v, m, l); continue; }
      float* p = part_of(cta);
      __stcg(reinterpret_cast<float4*>(p + r * DIM + d), v);
      if (d == 0) { __stcg(p + ROWS * DIM + r, m); __stcg(p + ROWS * (DIM + 1) + r, l); }
    }
    if (!whole) {
      int* ticket = reinterpret_cast<int*>(a.workspace) + first_cta;
      __threadfence();
      __syncthreads();
      if (tid == 0) s_last = atomicAdd(ticket, 1) == last_cta - first_cta;
      __syncthreads();
      if (s_last) {
        __threadfence();
        if (tid == 0) *ticket = 0;                                       // for the next call
        for (int x = tid; x < ROWS * (DIM / 4); x += WARPS * 32) {
          const int r = x / (DIM / 4), d = x % (DIM / 4) * 4;
          float m = -INFINITY, l = 0.f;
          float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
          for (int i = first_cta; i <= last_cta; ++i) m = fmaxf(m, __ldcg(part_of(i) + ROWS * DIM + r));
#pragma unroll 4
          for (int i = first_cta; i <= last_cta; ++i) {
            const float* p = part_of(i);
            const float pl = __ldcg(p + ROWS * (DIM + 1) + r), pm = __ldcg(p + ROWS * DIM + r);
            const float4 t = __ldcg(reinterpret_cast<const float4*>(p + r * DIM + d));
            const float by = pl == 0.f ? 0.f : pm == -INFINITY ? 1.f : exp2_of(pm - m);
            l += pl * by;
            v.x += t.x * by; v.y += t.y * by; v.z += t.z * by; v.w += t.w * by;
          }
          write(r, d, v, m, l);
        }
      }
    }
    __syncthreads();
    if (begin + it.stages >= share.hi) break;
    at.next(a);
  }
  if (!alive && lane == 0)   // no copy is left on its way into memory that may go to another CTA
    for (int i = turn; i < s_fetch[warp].issued; ++i) tc::mbar_wait(full0 + (i % SLOTS) * 8, (uint32_t)(i / SLOTS) & 1u, a.d_status);
}

template <typename T, int DIM, int NT>
dq_status run_few(cudaStream_t stream, const mx::Device& dev, const AttentionArgs& a) {
  using F = Few<DIM, NT>;
  static SmemOptIn opted;
  DQ_CHECK(opt_in_dynamic_smem(few_kernel<T, DIM, NT>, F::SMEM, opted));
  // no more CTAs than the cache can hold work for
  const int64_t rows = a.batch.tokens * a.group, tiles = rows / F::ROWS + a.batch.n_seqs;
  const int64_t stages = max((int64_t)1, ((int64_t)a.cache.width << a.cache.shift) / STAGE);
  const int64_t most = (tiles * a.cache.heads * stages + LEAST_STAGES - 1) / LEAST_STAGES;
  mx::LaunchConfig c(stream, min((int64_t)min(dev.sms, MAX_CTAS), max((int64_t)1, most)), F::THREADS, F::SMEM);
  return mx::launch(c, few_kernel<T, DIM, NT>, a);
}

// ------------------------------------------------------------------------------------------------ weights
// W[slot] = (old slot ? W[slot] : 0) + sum over the kv head's query rows of exp(S - lse): the first product again, with the
// rows' sums known.  A CTA takes tiles of 128 keys, a warp 16 of them for all rows, so that each weight is summed by one warp in
// one order.
constexpr int W_WARPS = 8, W_TILE = W_WARPS * GROUP;

template <typename T, int DIM>
__global__ void __launch_bounds__(W_WARPS * 32) weights_kernel(const AttentionArgs a) {
  __shared__ Share s_share;
  __shared__ int64_t s_sums[W_WARPS];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, c = lane & 3;
  const float to_log2 = a.scale * LOG2E;
  mx::wait_for_previous();
  find_share(&s_share, a.batch.n_seqs, 1, s_sums, [&](int b) { return (int64_t)a.cache.heads * ((a.cache.length(b) + W_TILE - 1) / W_TILE); });
  const Share share = s_share;
  int seq = share.seq;
  int64_t before = share.before;
  for (int64_t unit = share.lo; unit < share.hi; ++unit) {
    int length = a.cache.length(seq);
    int64_t tiles = (length + W_TILE - 1) / W_TILE;
    while (unit >= before + tiles * a.cache.heads) {
      before += tiles * a.cache.heads;
      length = a.cache.length(++seq);
      tiles = (length + W_TILE - 1) / W_TILE;
    }
    int64_t first;
    int n;
    a.batch.range(seq, first, n);
    const int h = (int)((unit - before) / tiles), rows = n * a.group;
    const int slot0 = (int)((unit - before) % tiles) * W_TILE + warp * GROUP;
    if (slot0 >= length) continue;
    const int64_t page = a.cache.page_of(seq, slot0);
    float got[2] = {0.f, 0.f};
    if (page >= 0) {
      const uint8_t* group = a.cache.group_at(page, h, slot0, DIM);
      float ks[2], ko[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const uint32_t p = *reinterpret_cast<const uint32_t*>(group + GROUP * (DIM / 2) + key_of(g + 8 * e) * 4);
        ks[e] = scale_of(p) * to_log2;
        ko[e] = offset_of(p) * to_log2;
      }
      // rows before the first one that sees slot0 see nothing here
      const int row_first = max(0, slot0 - (length - n)) * a.group / 8 * 8;
      for (int row0 = row_first; row0 < rows; row0 += 8) {
        Queries<T, DIM, 1> q;
        q.load(a.q, first, rows, row0, h, a.group, lane);
        float s[1][4];
        key_products<T, DIM, 1>(s, group, q, lane);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int r = row0 + 2 * c + j;
          if (r >= rows) continue;
          const int i = r / a.group, sees = length - n + i + 1;
          const float lse = a.lse[(first + i) * a.q.heads + h * a.group + r - i * a.group] * LOG2E;
#pragma unroll
          for (int e = 0; e < 2; ++e)
            if (slot0 + key_of(g + 8 * e) < sees) got[e] += exp2_of(s[0][2 * e + j] * (ks[e] * q.by[0][j]) + (ko[e] * q.sum[0][j] - lse));
        }
      }
    }
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      got[e] += __shfl_xor_sync(0xffffffffu, got[e], 1);
      got[e] += __shfl_xor_sync(0xffffffffu, got[e], 2);
      const int slot = slot0 + key_of(g + 8 * e);
      if (c == 0 && slot < length) {
        const int64_t at = ((int64_t)seq * a.cache.heads + h) * a.ld_slots + slot;
        a.weights_out[at] = (a.weights && slot < length - n ? a.weights[at] : 0.f) + got[e];
      }
    }
  }
  mx::allow_next();
}

}  // namespace

int64_t attention_workspace(int dim) { return TICKET_BYTES + (int64_t)MAX_CTAS * 2 * 16 * (dim + 2) * 4; }

dq_status attention(cudaStream_t stream, const mx::Device& dev, int dtype, int dim, const AttentionArgs& a) {
  auto by_rows = [&](auto t) {
    using T = decltype(t);
    const bool two = a.batch.tokens * a.group > (int64_t)8 * a.batch.n_seqs;
    if (dim == 64) return two ? run_few<T, 64, 2>(stream, dev, a) : run_few<T, 64, 1>(stream, dev, a);
    if (dim == 128) return two ? run_few<T, 128, 2>(stream, dev, a) : run_few<T, 128, 1>(stream, dev, a);
    return run_few<T, 256, 1>(stream, dev, a);
  };
  return dtype == DQ_BF16 ? by_rows(__nv_bfloat16()) : by_rows(__half());
}

dq_status attention_weights(cudaStream_t stream, const mx::Device& dev, int dtype, int dim, const AttentionArgs& a) {
  const int64_t most = (int64_t)a.cache.n_seqs * a.cache.heads * ((((int64_t)a.cache.width << a.cache.shift) + W_TILE - 1) / W_TILE);
  mx::LaunchConfig c(stream, min((int64_t)dev.sms * 4, max((int64_t)1, most)), W_WARPS * 32);
  auto run = [&](auto t) {
    using T = decltype(t);
    return by_dim(dim, [&](auto d) { return mx::launch(c, weights_kernel<T, decltype(d)::value>, a); });
  };
  return dtype == DQ_BF16 ? run(__nv_bfloat16()) : run(__half());
}

}  // namespace kv
}  // namespace dq
