// Attention over a key/value cache in 4 bits (dq_kv_attention) and the weight each cached token received
// (dq_kv_attention_weights).
//
//     S = scale q k^T over the slots a query sees,   O = softmax(S) v,   lse = log sum exp S
//
// With k = ks c + ko for codes c = 0 .. 15,   q . k = ks (q . (c - 8)) + (ko + 8 ks) sum q,   and
// sum_t p_t v_t = sum_t (p_t vs_t) (c_t - 8) + sum_t p_t (vo_t + 8 vs_t):   the matrix instructions multiply the codes, centred so
// that the sums stay small, and the parameters enter once for each key.  c - 8 is formed in place: four bits or'ed into the
// mantissa of 128 (bf16) or 1024 (fp16), less 136 or 1032.
//
// The keys are the rows (M) of the instructions and the query rows their columns (N = 8), so that the eight or fewer query heads
// of a kv head fill a tile: S^T = K Q^T, O^T = V^T P^T with mma.m16n8k16.  Any order of the dimensions serves the first product
// as long as Q has the same, any order of the keys the second as long as P has: a thread takes neighbouring codes of a key, as
// they lie, in both.  P^T comes out of the first product transposed and is turned by movmatrix.
// P vs is rounded to bf16 for the second product (relative error 2^-9 a term, as the output's own rounding); for fp16 queries it
// is held in two bf16 numbers (2^-17), because the output has 11 bits.
#include <type_traits>

#include "kv_common.cuh"
#include "tc_gemm.cuh"

namespace dq {
namespace kv {
namespace {

constexpr float LOG2E = 1.44269504088896f, LN2 = 0.693147180559945f;
constexpr int STAGE = 2 * GROUP;   // keys of a pipeline stage: the maximum of a row is looked at once for 32 keys

template <typename T>
__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1);
template <>
__device__ __forceinline__ void mma<__nv_bfloat16>(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
template <>
__device__ __forceinline__ void mma<__half>(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// Codes in bits 0-3 and 16-19, as c - 8.
template <typename T> __device__ __forceinline__ uint32_t centred(uint32_t w);
template <> __device__ __forceinline__ uint32_t centred<__nv_bfloat16>(uint32_t w) {
  const uint32_t v = (w & 0x000f000fu) | 0x43004300u, eight = 0x43084308u;   // 136
  const __nv_bfloat162 d = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&v), *reinterpret_cast<const __nv_bfloat162*>(&eight));
  return *reinterpret_cast<const uint32_t*>(&d);
}
template <> __device__ __forceinline__ uint32_t centred<__half>(uint32_t w) {
  const uint32_t v = (w & 0x000f000fu) | 0x64006400u, eight = 0x64086408u;   // 1032
  const __half2 d = __hsub2(*reinterpret_cast<const __half2*>(&v), *reinterpret_cast<const __half2*>(&eight));
  return *reinterpret_cast<const uint32_t*>(&d);
}
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
__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
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

// Eight query values as B fragments of a word's two k steps: (d, d + 4) for d = 0 .. 3.
template <typename T>
__device__ __forceinline__ void query_words(uint32_t (&b)[4], float& sum, const T* p, bool there, bool vec) {
  uint32_t w[4] = {0u, 0u, 0u, 0u};
  if (there) {
    if (vec) {
      const uint4 v = *reinterpret_cast<const uint4*>(p);
      w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        w[i] = (uint32_t)reinterpret_cast<const uint16_t*>(p)[2 * i] | ((uint32_t)reinterpret_cast<const uint16_t*>(p)[2 * i + 1] << 16);
    }
  }
  b[0] = __byte_perm(w[0], w[2], 0x5410);
  b[1] = __byte_perm(w[0], w[2], 0x7632);
  b[2] = __byte_perm(w[1], w[3], 0x5410);
  b[3] = __byte_perm(w[1], w[3], 0x7632);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    T v[2];
    memcpy(v, &w[i], 4);
    sum += mx::to_f32(v[0]) + mx::to_f32(v[1]);
  }
}

// A warp's query rows: tile of 8 NT rows (row r: token r / group, head r % group) as B fragments, and the sums of columns 2 c, 2 c + 1.
template <typename T, int DIM, int NT>
struct Queries {
  static constexpr int WORDS = DIM / 32;
  uint32_t b[NT][WORDS][4];
  float sum[NT][2];
  __device__ __forceinline__ void load(const Heads& q, int64_t first, int rows, int row0, int h, int group, int lane) {
    const int c = lane & 3;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int r = row0 + nt * 8 + (lane >> 2);
      const bool there = r < rows;
      const int i = there ? r / group : 0;
      const T* p = reinterpret_cast<const T*>(q.p) + (first + i) * q.token + (int64_t)(h * group + (there ? r - i * group : 0)) * q.head;
      float s = 0.f;
#pragma unroll
      for (int w = 0; w < WORDS; ++w) query_words<T>(b[nt][w], s, p + (c * WORDS + w) * 8, there, q.vec);
      s += __shfl_xor_sync(0xffffffffu, s, 1);
      s += __shfl_xor_sync(0xffffffffu, s, 2);
      sum[nt][0] = __shfl_sync(0xffffffffu, s, c * 8);
      sum[nt][1] = __shfl_sync(0xffffffffu, s, c * 8 + 4);
    }
  }
};

// q . (c - 8) of a group's 16 keys and the tile's rows: acc[nt] = (key_of(g), columns 2 c, 2 c + 1), (key_of(g + 8), the same).
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
      const uint32_t a0 = centred<T>(k0[w] >> (8 * e)), a1 = centred<T>(k1[w] >> (8 * e));
      const uint32_t a2 = centred<T>(k0[w] >> (8 * e + 4)), a3 = centred<T>(k1[w] >> (8 * e + 4));
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) mma<T>(acc[nt], a0, a1, a2, a3, q.b[nt][w][2 * e], q.b[nt][w][2 * e + 1]);
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
// A CTA takes an equal share of all stages of all items, whatever the sequences' lengths: one producer warp brings groups in by bulk copies, a
// ring of stages ahead; each of the other warps takes whole stages in turn, with its own maximum, sum and O^T, joined in shared memory at an
// item's end.  An item that crosses CTAs is left in the workspace in parts, and the CTA that finishes last joins them, in order.
template <int DIM, int NT>
struct Few {
  static constexpr int ROWS = 8 * NT;
  static constexpr int WARPS = DIM == 256 || (DIM == 128 && NT == 2) ? 8 : 16;
  static constexpr int SLOTS = DIM == 256 ? 16 : 32;
  static constexpr int THREADS = (WARPS + 1) * 32;
  static constexpr int GROUP_BYTES = GROUP * (DIM + 8), STAGE_BYTES = 2 * GROUP_BYTES;
  static constexpr int PAD = DIM + 4;                                  // floats of a row of O, against bank conflicts
  static constexpr int JOIN_BYTES = WARPS * ROWS * PAD * 4;
  static constexpr int SMEM = SLOTS * STAGE_BYTES + JOIN_BYTES;
  static constexpr int PART = ROWS * (DIM + 2);                        // floats of a part in the workspace: O, maxima, sums
};
constexpr int MAX_CTAS = 256;
constexpr int TICKET_BYTES = MAX_CTAS * 4;
constexpr int LEAST_STAGES = 8;                                        // of a CTA
constexpr float SLACK = 8.f;                                           // a maximum may grow by this (in powers of two) before O is rescaled

template <typename T, int DIM, int NT>
__global__ void __launch_bounds__(Few<DIM, NT>::THREADS, 1) few_kernel(const AttentionArgs a) {
  using F = Few<DIM, NT>;
  constexpr int ROWS = F::ROWS, WARPS = F::WARPS, SLOTS = F::SLOTS, VW = DIM / 64;
  extern __shared__ __align__(128) uint8_t smem[];
  float* joined = reinterpret_cast<float*>(smem + SLOTS * F::STAGE_BYTES);
  __shared__ __align__(8) uint64_t s_full[SLOTS], s_empty[SLOTS];
  __shared__ int s_valid[SLOTS];
  __shared__ Share s_share;
  __shared__ int64_t s_sums[WARPS + 1];
  __shared__ float s_max[WARPS][ROWS], s_sum[WARPS][ROWS];
  __shared__ int s_last;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const uint32_t full0 = tc::smem_u32(s_full), empty0 = tc::smem_u32(s_empty);
  if (tid < SLOTS) {
    tc::mbar_init(full0 + tid * 8, 1);
    tc::mbar_init(empty0 + tid * 8, 1);
  }
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

  // Items in the order (sequence, head, tile); both kinds of warps walk the same way.
  Item it;
  int seq = share.seq;
  describe<ROWS>(it, a, seq);
  int64_t index = (share.lo - share.before) / it.stages;                // of the sequence's items
  int64_t begin = share.before + index * it.stages;                     // the item's first unit
  auto next = [&]() {
    begin += it.stages;
    if (++index == (int64_t)it.tiles * a.cache.heads) {
      index = 0;
      do {
        if (++seq == a.batch.n_seqs) return;
        describe<ROWS>(it, a, seq);
      } while (it.tiles == 0);
    }
  };
  int64_t count = 0;                                                    // stages of this CTA so far

  if (warp == WARPS) {   // ------------------------------------------------ producer
    bool alive = true;
    while (alive) {
      const int h = (int)(index / it.tiles);
      const int64_t s0 = max(begin, share.lo) - begin, s1 = min(begin + it.stages, share.hi) - begin;
      for (int64_t at = s0; at < s1 && alive; at += 32) {               // a lane looks a stage's pages up
        int64_t page[2] = {-1, -1};
        const int slot0 = (int)(at + lane) * STAGE;
        if (at + lane < s1) {
          if (slot0 < it.length) page[0] = a.cache.page_of(it.b, slot0);
          if (slot0 + GROUP < it.length) page[1] = a.cache.shift > 4 ? page[0] : a.cache.page_of(it.b, slot0 + GROUP);
        }
        for (int j = 0; j < 32 && at + j < s1; ++j, ++count) {
          const int ring = (int)(count % SLOTS);
          const int64_t p0 = __shfl_sync(0xffffffffu, page[0], j), p1 = __shfl_sync(0xffffffffu, page[1], j);
          alive = __all_sync(0xffffffffu, tc::mbar_wait(empty0 + ring * 8, (uint32_t)(count / SLOTS + 1) & 1u, a.d_status));
          if (!alive) break;
          if (lane == 0) {
            const int slot = (int)(at + j) * STAGE;
            const uint32_t dst = tc::smem_u32(smem + ring * F::STAGE_BYTES), bar = full0 + ring * 8;
            auto copy = [&](uint32_t to, const uint8_t* from, uint32_t bytes) {
              asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                           ::"r"(to), "l"(from), "r"(bytes), "r"(bar) : "memory");
            };
            const bool joint = a.cache.shift > 4 && p1 >= 0;             // both groups in one page, one behind the other
            s_valid[ring] = (p0 >= 0 ? 1 : 0) | (p1 >= 0 ? 2 : 0);
            tc::mbar_expect_tx(bar, ((p0 >= 0) + (p1 >= 0)) * F::GROUP_BYTES);
            if (p0 >= 0) copy(dst, a.cache.group_at(p0, h, slot, DIM), joint ? F::STAGE_BYTES : F::GROUP_BYTES);
            if (p1 >= 0 && !joint) copy(dst + F::GROUP_BYTES, a.cache.group_at(p1, h, slot + GROUP, DIM), F::GROUP_BYTES);
          }
          __syncwarp();
        }
      }
      if (begin + it.stages >= share.hi) break;
      next();
    }
    if (!alive)   // no copy is left on its way into memory that may go to another CTA
      for (int64_t j = max((int64_t)0, count - SLOTS); j < count; ++j)
        tc::mbar_wait(full0 + (int)(j % SLOTS) * 8, (uint32_t)(j / SLOTS) & 1u, a.d_status);
    return;
  }

  // ------------------------------------------------------------------------ the others
  const int g = lane >> 2, c = lane & 3;
  const float to_log2 = a.scale * LOG2E;
  auto sync = [&]() { asm volatile("bar.sync 1, %0;" ::"n"(WARPS * 32) : "memory"); };
  bool alive = true;
  Queries<T, DIM, NT> q;
  while (true) {
    const int h = (int)(index / it.tiles), row0 = (int)(index % it.tiles) * ROWS;
    const int64_t s0 = max(begin, share.lo) - begin, s1 = min(begin + it.stages, share.hi) - begin;
    const bool starts = begin >= share.lo, ends = begin + it.stages <= share.hi;
    int64_t k = s0 + (warp - count % WARPS + WARPS) % WARPS;            // this warp's first stage of the segment
    int64_t n_count = count + (k - s0);
    count += s1 - s0;
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
    if (k < s1) q.load(a.q, it.first, it.rows, row0, h, a.group, lane);

    for (; k < s1; k += WARPS, n_count += WARPS) {
      const int ring = (int)(n_count % SLOTS);
      if (alive) alive = __all_sync(0xffffffffu, tc::mbar_wait(full0 + ring * 8, (uint32_t)(n_count / SLOTS) & 1u, a.d_status));
      const int slot0 = (int)k * STAGE;
      if (alive && slot0 < most) {
        const uint8_t* stage = smem + ring * F::STAGE_BYTES;
        const int valid = s_valid[ring];
        const bool masked = slot0 + STAGE > least || valid != 3;
        float s[2][NT][4];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const uint8_t* group = stage + u * F::GROUP_BYTES;
          key_products<T, DIM, NT>(s[u], group, q, lane);
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const uint32_t p = *reinterpret_cast<const uint32_t*>(group + GROUP * (DIM / 2) + key_of(g + 8 * e) * 4);
            const float ks = scale_of(p) * to_log2, kz = offset_of(p) * to_log2 + 8.f * ks;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int j = 0; j < 2; ++j) s[u][nt][2 * e + j] = s[u][nt][2 * e + j] * ks + kz * q.sum[nt][j];
          }
        }
        if (masked)
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const int slot = (valid >> u & 1) ? slot0 + u * GROUP + key_of(g + 8 * e) : INT_MAX;
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
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const uint8_t* group = stage + u * F::GROUP_BYTES + GROUP * (DIM / 2 + 4);
          uint32_t b[NT][2], b_low[NT][2];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const uint32_t w = *reinterpret_cast<const uint32_t*>(group + GROUP * (DIM / 2) + key_of(g + 8 * e) * 4);
            const float vs = scale_of(w), vz = offset_of(w) + 8.f * vs;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              float pv[2];
#pragma unroll
              for (int j = 0; j < 2; ++j) {
                const float x = s[u][nt][2 * e + j], m = top[nt][j];
                const float p = exp2_of(x - (m == -INFINITY ? 0.f : m));
                const bool gone = masked && x == -INFINITY;              // its parameters may be anything
                sum[nt][j] += p;
                off[nt][j] += gone ? 0.f : p * vz;
                pv[j] = gone ? 0.f : p * vs;
              }
              const uint32_t high = bf16_pair(pv[0], pv[1]);
              b[nt][e] = transposed(high);
              if (!std::is_same<T, __nv_bfloat16>::value)
                b_low[nt][e] = transposed(bf16_pair(pv[0] - scale_of(high), pv[1] - offset_of(high)));
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
              const uint32_t a0 = centred<__nv_bfloat16>(lo01 >> (4 * i)), a1 = centred<__nv_bfloat16>(hi01 >> (4 * i));
              const uint32_t a2 = centred<__nv_bfloat16>(lo23 >> (4 * i)), a3 = centred<__nv_bfloat16>(hi23 >> (4 * i));
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) {
                mma<__nv_bfloat16>(o[nt][w * 4 + i], a0, a1, a2, a3, b[nt][0], b[nt][1]);
                if (!std::is_same<T, __nv_bfloat16>::value) mma<__nv_bfloat16>(o[nt][w * 4 + i], a0, a1, a2, a3, b_low[nt][0], b_low[nt][1]);
              }
            }
          }
        }
      }
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(empty0 + ring * 8);
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
    sync();
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
#pragma unroll
        for (int i = 0; i < VW; ++i) {
          float4 v;
          v.x = (o[nt][4 * i][j] + off[nt][j]) * by; v.y = (o[nt][4 * i + 1][j] + off[nt][j]) * by;
          v.z = (o[nt][4 * i + 2][j] + off[nt][j]) * by; v.w = (o[nt][4 * i + 3][j] + off[nt][j]) * by;
          *reinterpret_cast<float4*>(row + 8 * i) = v;
          v.x = (o[nt][4 * i][2 + j] + off[nt][j]) * by; v.y = (o[nt][4 * i + 1][2 + j] + off[nt][j]) * by;
          v.z = (o[nt][4 * i + 2][2 + j] + off[nt][j]) * by; v.w = (o[nt][4 * i + 3][2 + j] + off[nt][j]) * by;
          *reinterpret_cast<float4*>(row + 8 * i + 4) = v;
        }
      }
    sync();
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
      sync();
      if (tid == 0) s_last = atomicAdd(ticket, 1) == last_cta - first_cta;
      sync();
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
    sync();
    if (begin + it.stages >= share.hi) break;
    next();
  }
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
      float ks[2], kz[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const uint32_t p = *reinterpret_cast<const uint32_t*>(group + GROUP * (DIM / 2) + key_of(g + 8 * e) * 4);
        ks[e] = scale_of(p) * to_log2;
        kz[e] = offset_of(p) * to_log2 + 8.f * ks[e];
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
            if (slot0 + key_of(g + 8 * e) < sees) got[e] += exp2_of(s[0][2 * e + j] * ks[e] + kz[e] * q.sum[0][j] - lse);
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
