// Attention over a key/value cache in 4 bits (dq_kv_attention) and the weight each cached token received
// (dq_kv_attention_weights).
//
//     S = scale q k^T over the slots a query sees,   O = softmax(S) v,   lse = log sum exp S
//
// With k = ks c + ko for codes c = 0 .. 15,   q . k = ks (q . c) + ko sum q   and   sum_t p_t v_t = sum_t (p_t vs_t) (c_t - 8) + sum_t p_t (vo_t + 8 vs_t):
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
// for fp16's 11 and bf16's 8 bits, save values below 2^-24 of the largest.  P vs is divided by the power of two of the largest vs so
// far and rounded to fp16 (2^-11 a term; below 2^-20 of the row's largest 2^-31 of it).  The values' codes are centred (one more
// instruction, in a pipe that has room) because the instructions' own sums truncate: over a long axis sums of 0 .. 15 would drift.
#include "kv_common.cuh"
#include "tc_gemm.cuh"

namespace dq {
namespace kv {
namespace {

constexpr int STAGE = 2 * GROUP;   // keys of a pipeline stage: the maximum of a row is looked at once for 32 keys

__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma(float2 (&d)[2], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0].x), "+f"(d[0].y), "+f"(d[1].x), "+f"(d[1].y) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// The same with a sum that starts from zero.
__device__ __forceinline__ void mma_first(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
               : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ uint32_t transposed(uint32_t v) {
  uint32_t d;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(v));
  return d;
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
__device__ __forceinline__ void load_values(float2 (&v)[4], const T* p, bool there, bool vec) {
  mx::Vec8<T> x;
  x.clear();
  if (there) {
    if (vec) x.load(p);
    else
#pragma unroll
      for (int i = 0; i < 4; ++i) x.set_pair(i, make_float2(mx::to_f32(p[2 * i]), mx::to_f32(p[2 * i + 1])));
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = x.pair(i);
}

// Eight query rows from row0 on (row r: token r / group, head r % group) as B fragments.  Dimensions whose codes lie four bits up
// are held 2^-4 smaller.  For the columns 2 c and 2 c + 1: `by`, what takes the powers of two out of a product, and the sum of the
// row, both times scale log2 e.
template <typename T, int DIM>
struct Queries {
  static constexpr int WORDS = DIM / 32;
  uint4 b[WORDS];
  float2 by, sum;
  __device__ __forceinline__ void load(const AttentionArgs& a, int64_t first, int rows, int row0, int h, int lane) {
    const int c = lane & 3, r = row0 + (lane >> 2);
    const bool there = r < rows;
    const int i = there ? a.token_of(r) : 0;
    const T* p = reinterpret_cast<const T*>(a.q.p) + (first + i) * a.q.token + (int64_t)(h * a.group + (there ? r - i * a.group : 0)) * a.q.head;
    const float factor = a.scale * LOG2E;
    float2 v[WORDS][4], sums = both(0.f);
    float most = 0.f;
#pragma unroll
    for (int w = 0; w < WORDS; ++w) {
      load_values<T>(v[w], p + (c * WORDS + w) * 8, there, a.q.vec);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        sums = add2(sums, v[w][e]);
        most = fmaxf(most, fmaxf(fabsf(v[w][e].x), fabsf(v[w][e].y)));
      }
    }
    float s = sums.x + sums.y;
    s += __shfl_xor_sync(0xffffffffu, s, 1);
    s += __shfl_xor_sync(0xffffffffu, s, 2);
    most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 1));
    most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 2));
    // the largest value's exponent field, within what keeps both factors normal numbers; a row that is not finite stays so
    const int field = min(max((int)mx::exponent_field(most), 14), 244);
    const float up = __uint_as_float((uint32_t)(268 - field) << 23), up4 = up * 0.0625f;
    const float2 ups = make_float2(up, up4);
#pragma unroll
    for (int w = 0; w < WORDS; ++w) {
      const float2 d01 = mul2(v[w][0], ups), d23 = mul2(v[w][1], ups), d45 = mul2(v[w][2], ups), d67 = mul2(v[w][3], ups);
      b[w] = make_uint4(half_pair(d01.x, d45.x), half_pair(d01.y, d45.y), half_pair(d23.x, d67.x), half_pair(d23.y, d67.y));
    }
    const float down = __uint_as_float((uint32_t)(field + 10) << 23);   // 2^24 / up
    sum = make_float2(__shfl_sync(0xffffffffu, s, c * 8) * factor, __shfl_sync(0xffffffffu, s, c * 8 + 4) * factor);
    by = make_float2(__shfl_sync(0xffffffffu, down, c * 8) * factor, __shfl_sync(0xffffffffu, down, c * 8 + 4) * factor);
  }
};

// (q . c) of the 16 keys of N groups and the tile's rows, without q.by: acc[u][nt][e] = key_of(g + 8 e), columns 2 c, 2 c + 1.
// query(nt, w): the B fragments of a word.  Two sums a group side by side, because each instruction waits for the one that its sum
// comes from.
template <int DIM, int NT, int N, int STRIDE, typename Q>
__device__ __forceinline__ void key_products(float2 (&acc)[N][NT][2], const uint8_t* codes, Q query, int lane) {
  constexpr int WORDS = DIM / 32;
  const int g = lane >> 2, c = lane & 3;
  uint32_t k[N][2][WORDS];
#pragma unroll
  for (int u = 0; u < N; ++u)
#pragma unroll
    for (int e = 0; e < 2; ++e)
      load_words<WORDS>(k[u][e], codes + u * STRIDE + key_of(g + 8 * e) * (DIM / 2) + c * (DIM / 8));
  float d[N][2][NT][4];
#pragma unroll
  for (int w = 0; w < WORDS; ++w)
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const uint4 b = query(nt, w);
#pragma unroll
      for (int u = 0; u < N; ++u)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const uint32_t x0 = k[u][0][w] >> (8 * e), x1 = k[u][1][w] >> (8 * e), b0 = e ? b.z : b.x, b1 = e ? b.w : b.y;
          if (w == 0) mma_first(d[u][e][nt], low_codes(x0), low_codes(x1), high_codes(x0), high_codes(x1), b0, b1);
          else mma(d[u][e][nt], low_codes(x0), low_codes(x1), high_codes(x0), high_codes(x1), b0, b1);
        }
    }
#pragma unroll
  for (int u = 0; u < N; ++u)
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int e = 0; e < 2; ++e)
        acc[u][nt][e] = add2(make_float2(d[u][0][nt][2 * e], d[u][0][nt][2 * e + 1]), make_float2(d[u][1][nt][2 * e], d[u][1][nt][2 * e + 1]));
}

// An item of work is a tile of ROWS query rows of a sequence and kv head; it has `stages` stages of keys (one at least: rows that see
// nothing are written too).  ROWS 0: all rows, and no item without keys.
template <int ROWS>
struct Sequence {
  int64_t first;
  int n, length, tiles, stages;
  __device__ __forceinline__ void describe(const AttentionArgs& a, int b) {
    a.batch.range(b, first, n);
    length = a.cache.length(b);
    stages = (length + STAGE - 1) / STAGE;
    if constexpr (ROWS == 0) tiles = min(stages, 1);
    else {
      tiles = (int)(((int64_t)n * a.group + ROWS - 1) / ROWS);
      stages = max(stages, 1);
    }
  }
  __device__ __forceinline__ int64_t units(const AttentionArgs& a) const { return (int64_t)tiles * a.cache.heads * stages; }
};

// A walk over the items in the order (sequence, head, tile).
template <int ROWS>
struct Walk {
  Sequence<ROWS> s;
  int b, h, tile;
  int64_t begin;                                                       // the item's first unit
  __device__ __forceinline__ void start(const AttentionArgs& a, const Share& share) {
    b = share.seq;
    s.describe(a, b);
    const int64_t index = quotient(share.lo - share.before, s.stages);   // of the sequence's items
    h = (int)quotient(index, s.tiles);
    tile = (int)(index - (int64_t)h * s.tiles);
    begin = share.before + index * s.stages;
  }
  __device__ __forceinline__ void next(const AttentionArgs& a) {
    begin += s.stages;
    if (++tile < s.tiles) return;
    tile = 0;
    if (++h < a.cache.heads) return;
    h = 0;
    do {
      if (++b == a.batch.n_seqs) return;
      s.describe(a, b);
    } while (s.tiles == 0);
  }
  // the slots of the item that are a CTA's
  __device__ __forceinline__ int end(const Share& share) const { return (int)(min(begin + s.stages, share.hi) - begin) * STAGE; }
};

// A warp's stages of its CTA's share, every WARPS-th, brought into PLACES places of its own by bulk copies ahead of their use, across
// items.  KEYS: without the values.
template <int DIM, int ROWS, int WARPS, int PLACES, bool KEYS>
struct Stream {
  static constexpr int WHOLE = GROUP * (DIM + 8), GROUP_BYTES = KEYS ? WHOLE / 2 : WHOLE, STAGE_BYTES = 2 * GROUP_BYTES;
  struct List {                                                         // in shared memory
    const uint8_t* group[32][2];                                        // of the next stages (null: no page)
    uint64_t full[PLACES];                                              // barriers: a place has been filled
    int valid[PLACES];                                                  // which of its groups have been
    int used, left, issued;                                             // of the list
    int slot, end;                                                      // within the item, behind the list
    Walk<ROWS> walk;
  };
  const AttentionArgs& a;
  const Share& share;
  List& f;
  uint8_t* ring;
  int lane, turn = 0;                                                   // stages so far
  bool alive = true;

  __device__ __forceinline__ uint32_t bar(int place) const { return tc::smem_u32(&f.full[place]); }
  __device__ __forceinline__ int place() const { return turn % PLACES; }
  __device__ __forceinline__ const uint8_t* stage() const { return ring + place() * STAGE_BYTES; }

  // A lane looks the pages of one of the next 32 stages of an item up.
  __device__ __forceinline__ void refill() {
    int slot = f.slot;
    while (slot >= f.end && f.walk.begin + f.walk.s.stages < share.hi) {
      __syncwarp();
      if (lane == 0) {
        slot -= f.walk.s.stages * STAGE;                                // (the warp's stages go on through all items)
        f.walk.next(a);
        f.end = f.walk.end(share);
        f.slot = slot;
      }
      __syncwarp();
      slot = f.slot;
    }
    const Walk<ROWS>& w = f.walk;
    const int mine = slot + lane * (WARPS * STAGE), length = w.s.length;
    const uint8_t *p0 = nullptr, *p1 = nullptr;
    if (mine < min(f.end, length)) {
      const int64_t page = a.cache.page_of(w.b, mine);
      if (page >= 0) p0 = a.cache.group_at(page, w.h, mine, DIM);
      if (mine + GROUP < length) {
        if (a.cache.shift > 4) p1 = p0 ? p0 + WHOLE : nullptr;
        else {
          const int64_t other = a.cache.page_of(w.b, mine + GROUP);
          if (other >= 0) p1 = a.cache.group_at(other, w.h, mine + GROUP, DIM);
        }
      }
    }
    f.group[lane][0] = p0;
    f.group[lane][1] = p1;
    const int left = slot < f.end ? (f.end - slot + WARPS * STAGE - 1) / (WARPS * STAGE) : 0;
    __syncwarp();
    if (lane == 0) {
      f.left = min(left, 32);
      f.used = 0;
      f.slot = slot + f.left * (WARPS * STAGE);
    }
    __syncwarp();
  }
  // The warp's next stage, if there is one, into a place that no lane reads any more.
  __device__ __forceinline__ void fetch(int place) {
    if (f.used == f.left) refill();
    const int i = f.used;
    if (i == f.left) return;
    __syncwarp();
    if (lane == 0) {
      const uint8_t *p0 = f.group[i][0], *p1 = f.group[i][1];
      const uint32_t dst = tc::smem_u32(ring + place * STAGE_BYTES), full = bar(place);
      auto copy = [&](uint32_t to, const uint8_t* from, uint32_t bytes) {
        asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                     ::"r"(to), "l"(from), "r"(bytes), "r"(full) : "memory");
      };
      f.used = i + 1;
      ++f.issued;
      f.valid[place] = (p0 ? 1 : 0) | (p1 ? 2 : 0);
      tc::mbar_expect_tx(full, ((p0 ? 1 : 0) + (p1 ? 1 : 0)) * GROUP_BYTES);
      if (!KEYS && p0 && p1 == p0 + WHOLE) copy(dst, p0, STAGE_BYTES);   // one behind the other
      else {
        if (p0) copy(dst, p0, GROUP_BYTES);
        if (p1) copy(dst + GROUP_BYTES, p1, GROUP_BYTES);
      }
    }
    __syncwarp();
  }
  // From the first slot of the share's first item that is this warp's.  The barriers are ready.
  __device__ __forceinline__ void start(const Walk<ROWS>& walk, int slot) {
    if (lane == 0) {
      f.walk = walk;
      f.slot = slot; f.end = walk.end(share); f.used = f.left = f.issued = 0;
    }
    __syncwarp();
    for (int i = 0; i < PLACES; ++i) fetch(i);
  }
  // Whether the warp's next stage is there.
  __device__ __forceinline__ bool wait() {
    if (alive) alive = __all_sync(0xffffffffu, tc::mbar_wait(bar(place()), (uint32_t)(turn / PLACES) & 1u, a.d_status));
    return alive;
  }
  // After a wait that gave up: no copy is left on its way into memory that may go to another CTA.
  __device__ __forceinline__ void end() {
    if (!alive && lane == 0)
      for (int i = turn; i < f.issued; ++i) tc::mbar_wait(bar(i % PLACES), (uint32_t)(i / PLACES) & 1u, a.d_status);
  }
};

// ------------------------------------------------------------------------------------------------ few rows
// A CTA takes an equal share of all stages of all items, whatever the sequences' lengths, and its warps take them in turn, each with its
// own maximum, sum and O^T, joined in shared memory at an item's end.  A warp brings its stages in by bulk copies into two places of
// its own: while it works on one the other is on its way, across items too.  An item that crosses CTAs is left in the workspace in parts,
// and the CTA that finishes last joins them, in order.
//
// Where the cache is long no unit is full (integer pipe 56 % of its cycles, issue 54 %, HBM 65 % of the copy rate): with 16 or 12 warps an SM
// the chain inside a stage, from codes over product, maxima and exponentials to the second product, is what is waited for.  64 ragged
// sequences up to 16384 slots, 8 kv heads of 128, 168 us, 4.25 TB/s.  131072 slots of one sequence: 46 us, 3.1 TB/s, of which 10 are start and
// join.  1024 slots: 10.9 us, a chain of table, codes, products, ticket and parts.
template <int DIM, int NT>
struct Few {
  static constexpr int ROWS = 8 * NT;
  // two CTAs an SM: while one joins its warps the other works (64 ragged sequences up to 16384 slots: 171 us when this was chosen; one CTA of twice the
  // warps 190; more warps of fewer registers, 20 or 18 an SM, 185 and 200)
  static constexpr int WARPS = DIM * NT > 128 ? 6 : 8, PER_SM = 2;
  static constexpr int PLACES = 2;
  static constexpr int THREADS = WARPS * 32;
  using Stages = Stream<DIM, ROWS, WARPS, PLACES, false>;
  static constexpr int GROUP_BYTES = Stages::GROUP_BYTES, STAGE_BYTES = Stages::STAGE_BYTES;
  static constexpr int PAD = DIM + 4;                                  // floats of a row of O, against bank conflicts
  static_assert(8 * PAD * 4 <= STAGE_BYTES, "a warp leaves eight rows of O where its last stage was");
  static constexpr int SMEM = WARPS * PLACES * STAGE_BYTES;
  static constexpr int PART = ROWS * (DIM + 2);                        // floats of a part in the workspace: O, maxima, sums
};
constexpr int LEAST_STAGES = 8;                                        // of a CTA
constexpr float SLACK = 8.f;                                           // a maximum may grow by this (in powers of two) before O is rescaled

template <typename T, int DIM, int NT>
__global__ void __launch_bounds__(Few<DIM, NT>::THREADS, Few<DIM, NT>::PER_SM) few_kernel(const AttentionArgs a) {
  using F = Few<DIM, NT>;
  constexpr int ROWS = F::ROWS, WARPS = F::WARPS, PLACES = F::PLACES, VW = DIM / 64;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ typename F::Stages::List s_list[WARPS];
  __shared__ Share s_share;
  __shared__ int64_t s_sums[WARPS];
  __shared__ float s_max[WARPS][ROWS], s_sum[WARPS][ROWS];
  __shared__ int s_place[WARPS];                                       // the place that a warp's O is left in
  __shared__ uint4 s_query[2][NT][DIM / 32][32];                       // this item's queries and the next one's
  __shared__ float2 s_by[2][NT][4], s_qsum[2][NT][4];
  __shared__ float s_join[WARPS * 32 / ROWS][ROWS];
  __shared__ int s_last;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (tid < WARPS * PLACES) tc::mbar_init(tc::smem_u32(&s_list[tid / PLACES].full[tid % PLACES]), 1);
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  mx::wait_for_previous();
  mx::allow_next();
  const Share share = find_share(&s_share, a.batch.n_seqs, LEAST_STAGES, s_sums, [&](int b) {
    Sequence<ROWS> s;
    s.describe(a, b);
    return s.units(a);
  });
  if (share.lo >= share.hi) return;

  __syncthreads();                                                      // the barriers are ready
  Walk<ROWS> at;
  at.start(a, share);
  int slot0 = (int)(share.lo - at.begin + warp) * STAGE;                // this warp's next, within the item
  typename F::Stages stages{a, share, s_list[warp], smem + warp * PLACES * F::STAGE_BYTES, lane};
  stages.start(at, slot0);

  const int g = lane >> 2, c = lane & 3;
  int page = 0;                                                         // of the queries
  auto load_queries = [&](const Walk<ROWS>& w, int into) {              // by the first NT warps
    if (warp >= NT) return;
    Queries<T, DIM> q;
    q.load(a, w.s.first, w.s.n * a.group, w.tile * ROWS + warp * 8, w.h, lane);
#pragma unroll
    for (int i = 0; i < DIM / 32; ++i) s_query[into][warp][i][lane] = q.b[i];
    if (g == 0) {
      s_by[into][warp][c] = q.by;
      s_qsum[into][warp][c] = q.sum;
    }
  };
  load_queries(at, 0);
  __syncthreads();
  while (true) {
    const int64_t begin = at.begin, first = at.s.first;
    const int h = at.h, row0 = at.tile * ROWS, rows = at.s.n * a.group, length = at.s.length;
    const bool starts = begin >= share.lo, ends = begin + at.s.stages <= share.hi;
    const int end = at.end(share);
    float top[NT][2];
    float2 sum[NT], off[NT], o[NT][VW * 4][2];
    int sees[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        top[nt][j] = -INFINITY;
        sum[nt] = off[nt] = both(0.f);
        const int r = row0 + nt * 8 + 2 * c + j;
        sees[nt][j] = r < rows ? max(length - at.s.n + a.token_of(r) + 1, 0) : 0;
      }
    // all valid rows see the stages before the first row's end, none those past the last one's
    const int least = max(length - at.s.n + a.token_of(row0) + 1, 0);
    const int most = max(length - at.s.n + a.token_of(min(row0 + ROWS, rows) - 1) + 1, 0);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int i = 0; i < VW * 4; ++i)
#pragma unroll
        for (int e = 0; e < 2; ++e) o[nt][i][e] = both(0.f);
    float2 q_by[NT], q_sum[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) { q_by[nt] = s_by[page][nt][c]; q_sum[nt] = s_qsum[page][nt][c]; }
    uint32_t scale_field = 7u;                                          // the largest vs's so far
    bool left = false;                                                  // a place is free for O, and not filled again yet

    for (; slot0 < end; slot0 += WARPS * STAGE) {
      if (!stages.wait()) continue;
      const int place = stages.place();
      if (slot0 < most) {
        const uint8_t* stage = stages.stage();
        const int valid = s_list[warp].valid[place];
        const bool masked = slot0 + STAGE > least || valid != 3;
        float2 s[2][NT][2];
        key_products<DIM, NT, 2, F::GROUP_BYTES>(s, stage, [&](int nt, int w) { return s_query[page][nt][w][lane]; }, lane);
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const uint32_t p = *reinterpret_cast<const uint32_t*>(stage + u * F::GROUP_BYTES + GROUP * (DIM / 2) + key_of(g + 8 * e) * 4);
            const float ks = scale_of(p), ko = offset_of(p);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) s[u][nt][e] = fma2(s[u][nt][e], mul2(both(ks), q_by[nt]), mul2(both(ko), q_sum[nt]));
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
              if (slot >= length) vp[u][e] = 0u;
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) {
                if (slot >= sees[nt][0]) s[u][nt][e].x = -INFINITY;
                if (slot >= sees[nt][1]) s[u][nt][e].y = -INFINITY;
              }
            }
        // the exponent field of the stage's largest vs: vs 2^(6 - scale_field + 127) < 2^7, and with p < 2^SLACK P stays below 2^15
        uint32_t field = max(max(vp[0][0] & 0x7f80u, vp[0][1] & 0x7f80u), max(vp[1][0] & 0x7f80u, vp[1][1] & 0x7f80u));
        field = __reduce_max_sync(0xffffffffu, field) >> 7;
        const bool odd = field == 255u;
        if (odd) {                                                      // a NaN does not count: not all rows may see it
          field = 0u;
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const uint32_t f = vp[u][e] >> 7 & 255u;
              field = max(field, f == 255u ? 0u : f);
            }
          field = __reduce_max_sync(0xffffffffu, field);
        }
        // maxima over the stage's keys; O is rescaled where one has grown by more than SLACK, or the largest vs
        bool grown = field > scale_field;
        float now[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            auto at_j = [&](int u, int e) { return j ? s[u][nt][e].y : s[u][nt][e].x; };
            float m = fmaxf(fmaxf(at_j(0, 0), at_j(0, 1)), fmaxf(at_j(1, 0), at_j(1, 1)));
            m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 4));
            m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 8));
            m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 16));
            now[nt][j] = m;
            grown |= m > top[nt][j] + SLACK;
          }
        if (__any_sync(0xffffffffu, grown)) {
          const uint32_t wider = max(field, scale_field) - scale_field;
          const float scaled = wider > 126u ? 0.f : __uint_as_float((127u - wider) << 23);
          scale_field += wider;
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            float by[2];
            const float l[2] = {sum[nt].x, sum[nt].y};
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              const float m = fmaxf(top[nt][j], now[nt][j]);
              by[j] = top[nt][j] == -INFINITY ? (l[j] == 0.f ? 0.f : 1.f) : exp2_of(top[nt][j] - m);
              top[nt][j] = m;
            }
            float2 f = make_float2(by[0], by[1]);
            sum[nt] = mul2(sum[nt], f);
            off[nt] = mul2(off[nt], f);
            f = mul2(f, both(scaled));
#pragma unroll
            for (int i = 0; i < VW * 4; ++i)
#pragma unroll
              for (int e = 0; e < 2; ++e) o[nt][i][e] = mul2(o[nt][i][e], f);
          }
        }
        const float shrink = __uint_as_float((260u - scale_field) << 23);
        float2 base[NT];                                                // less the maximum
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
          base[nt] = make_float2(top[nt][0] == -INFINITY ? 0.f : -top[nt][0], top[nt][1] == -INFINITY ? 0.f : -top[nt][1]);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const uint8_t* group = stage + u * F::GROUP_BYTES + GROUP * (DIM / 2 + 4);
          uint32_t b[NT][2];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float v1 = scale_of(vp[u][e]), vs = v1 * shrink, vo = offset_of(vp[u][e]) + 8.f * v1;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              float2 p = add2(s[u][nt][e], base[nt]), r, v;
              p = make_float2(exp2_of(p.x), exp2_of(p.y));
              sum[nt] = add2(sum[nt], p);
              if (!odd) {
                off[nt] = fma2(p, both(vo), off[nt]);
                v = mul2(p, both(vs));
              } else {                                                  // (a NaN times the zero of a row that does not see it)
                const bool x = masked && s[u][nt][e].x == -INFINITY, y = masked && s[u][nt][e].y == -INFINITY;
                r = make_float2(x ? 0.f : p.x * vo, y ? 0.f : p.y * vo);
                off[nt] = add2(off[nt], r);
                v = make_float2(x ? 0.f : p.x * vs, y ? 0.f : p.y * vs);
              }
              b[nt][e] = transposed(half_pair(v.x, v.y));
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
                if (i & 1) mma(o[nt][w * 4 + i], high_centred(a0), high_centred(a1), high_centred(a2), high_centred(a3), b[nt][0], b[nt][1]);
                else mma(o[nt][w * 4 + i], low_centred(a0), low_centred(a1), low_centred(a2), low_centred(a3), b[nt][0], b[nt][1]);
              }
            }
          }
        }
      }
      ++stages.turn;
      __syncwarp();                                                     // all lanes have read the stage
      left = slot0 + WARPS * STAGE >= end;                              // the last one's place takes O first
      if (!left) stages.fetch(place);
    }

    // ---- the item's rows over the warps
    float l[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int d = 4; d < 32; d <<= 1) {
        sum[nt] = add2(sum[nt], make_float2(__shfl_xor_sync(0xffffffffu, sum[nt].x, d), __shfl_xor_sync(0xffffffffu, sum[nt].y, d)));
        off[nt] = add2(off[nt], make_float2(__shfl_xor_sync(0xffffffffu, off[nt].x, d), __shfl_xor_sync(0xffffffffu, off[nt].y, d)));
      }
      l[nt][0] = sum[nt].x; l[nt][1] = sum[nt].y;
      if (g == 0)
#pragma unroll
        for (int j = 0; j < 2; ++j) { s_max[warp][nt * 8 + 2 * c + j] = top[nt][j]; s_sum[warp][nt * 8 + 2 * c + j] = l[nt][j]; }
    }
    const int place = (stages.turn + PLACES - 1) % PLACES;                       // of the last stage
    if (lane == 0) s_place[warp] = place;
    const bool more = begin + at.s.stages < share.hi;
    if (more && warp < NT) {
      Walk<ROWS> following = at;
      following.next(a);
      load_queries(following, page ^ 1);
    }
    __syncthreads();
    const int cta = blockIdx.x;
    const int first_cta = starts ? cta : cta_of(begin, share.total, share.ctas);
    const int last_cta = ends ? cta : cta_of(begin + at.s.stages - 1, share.total, share.ctas);
    const bool whole = first_cta == last_cta;
    float* parts = reinterpret_cast<float*>(a.workspace + TICKET_BYTES);
    auto part_of = [&](int i) { return parts + ((int64_t)i * 2 + (i == first_cta ? 1 : 0)) * F::PART; };
    auto write = [&](int r, int d, float4 v, float m, float l) {         // row r of the tile, dimensions d .. d + 3
      const int row = row0 + r;
      if (row >= rows) return;
      const int i = a.token_of(row), head = h * a.group + row - i * a.group;
      const float by = l == 0.f ? 0.f : 1.f / l;
      T* p = reinterpret_cast<T*>(a.out.p) + (first + i) * a.out.token + head * a.out.head + d;
      T y[4] = {mx::from_f32<T>(v.x * by), mx::from_f32<T>(v.y * by), mx::from_f32<T>(v.z * by), mx::from_f32<T>(v.w * by)};
      if (a.out.vec) { uint2 w; memcpy(&w, y, 8); *reinterpret_cast<uint2*>(p) = w; }
      else
#pragma unroll
        for (int e = 0; e < 4; ++e) p[e] = y[e];
      if (d == 0 && a.lse) a.lse[(first + i) * a.q.heads + head] = l == 0.f ? -INFINITY : (m + log2f(l)) * LN2;
    };
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int r = nt * 8 + 2 * c + j;
        if (l[nt][j] == 0.f) continue;
        float m = -INFINITY;
        for (int w = 0; w < WARPS; ++w) m = fmaxf(m, s_max[w][r]);
        const float by = top[nt][j] == -INFINITY ? 1.f : exp2_of(top[nt][j] - m);
        float* row = reinterpret_cast<float*>(stages.ring + place * F::STAGE_BYTES) + (2 * c + j) * F::PAD + g * (DIM / 8);
        // out of the codes' 2^24 and 2^20, and the scales' power of two
        const float grow = __uint_as_float((scale_field - 6u) << 23) * by, o0 = (j ? off[nt].y : off[nt].x) * by;
        constexpr float LOW = 16777216.f, HIGH = 1048576.f;             // (apart from grow, with which they may leave fp32's range)
#pragma unroll
        for (int i = 0; i < VW; ++i)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            auto at_j = [&](int k) { const float2 v = o[nt][4 * i + k][e]; return j ? v.y : v.x; };
            *reinterpret_cast<float4*>(row + 8 * i + 4 * e) =
                make_float4(at_j(0) * LOW * grow + o0, at_j(1) * HIGH * grow + o0, at_j(2) * LOW * grow + o0, at_j(3) * HIGH * grow + o0);
          }
      }
      __syncthreads();
      for (int x = tid; x < 8 * (DIM / 4); x += WARPS * 32) {
        const int r = nt * 8 + x / (DIM / 4), d = x % (DIM / 4) * 4;
        float m = -INFINITY, all = 0.f;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int w = 0; w < WARPS; ++w) m = fmaxf(m, s_max[w][r]);
#pragma unroll
        for (int w = 0; w < WARPS; ++w) {
          if (s_sum[w][r] == 0.f) continue;
          all += s_sum[w][r] * (s_max[w][r] == -INFINITY ? 1.f : exp2_of(s_max[w][r] - m));
          const float4 t = *reinterpret_cast<const float4*>(reinterpret_cast<const float*>(smem + (w * PLACES + s_place[w]) * F::STAGE_BYTES) +
                                                            (x / (DIM / 4)) * F::PAD + d);
          v.x += t.x; v.y += t.y; v.z += t.z; v.w += t.w;
        }
        if (whole) { write(r, d, v, m, all); continue; }
        float* p = part_of(cta);
        __stcg(reinterpret_cast<float4*>(p + r * DIM + d), v);
        if (d == 0) { __stcg(p + ROWS * DIM + r, m); __stcg(p + ROWS * (DIM + 1) + r, all); }
      }
      if (!whole && nt == NT - 1) __threadfence();
      __syncthreads();
    }
    if (left) {                                                         // the stage after next comes where O was
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      stages.fetch(place);
    }
    if (!whole) {
      int* ticket = reinterpret_cast<int*>(a.workspace) + first_cta;
      if (tid == 0) s_last = atomicAdd(ticket, 1) == last_cta - first_cta;
      __syncthreads();
      if (s_last) {
        __threadfence();
        if (tid == 0) *ticket = 0;                                       // for the next call
        // each row's maximum and sum, over the parts by many threads; then O
        constexpr int AT_ONCE = WARPS * 32 / ROWS;
        const int row = tid % ROWS, mine = tid / ROWS;
        float m = -INFINITY, all = 0.f;
        for (int i = first_cta + mine; i <= last_cta; i += AT_ONCE) m = fmaxf(m, __ldcg(part_of(i) + ROWS * DIM + row));
        s_join[mine][row] = m;
        __syncthreads();
        for (int i = 0; i < AT_ONCE; ++i) m = fmaxf(m, s_join[i][row]);
        __syncthreads();
        for (int i = first_cta + mine; i <= last_cta; i += AT_ONCE) {
          const float pm = __ldcg(part_of(i) + ROWS * DIM + row), pl = __ldcg(part_of(i) + ROWS * (DIM + 1) + row);
          all += pl == 0.f ? 0.f : pl * (pm == -INFINITY ? 1.f : exp2_of(pm - m));
        }
        s_join[mine][row] = all;
        if (mine == 0) s_max[0][row] = m;
        __syncthreads();
        for (int x = tid; x < ROWS * (DIM / 4); x += WARPS * 32) {
          const int r = x / (DIM / 4), d = x % (DIM / 4) * 4;
          float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
          m = s_max[0][r];
#pragma unroll 8
          for (int i = first_cta; i <= last_cta; ++i) {
            const float pm = __ldcg(part_of(i) + ROWS * DIM + r);
            const float4 t = __ldcg(reinterpret_cast<const float4*>(part_of(i) + r * DIM + d));
            const float by = pm == -INFINITY ? 1.f : exp2_of(pm - m);    // (where there is no sum O is zero)
            v.x += t.x * by; v.y += t.y * by; v.z += t.z * by; v.w += t.w * by;
          }
          all = 0.f;
          for (int i = 0; i < AT_ONCE; ++i) all += s_join[i][r];
          write(r, d, v, m, all);
        }
        __syncthreads();
      }
    }
    page ^= 1;
    if (begin + at.s.stages >= share.hi) break;
    slot0 -= at.s.stages * STAGE;
    at.next(a);
  }
  stages.end();
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
  mx::LaunchConfig c(stream, min((int64_t)min(dev.sms, MAX_SMS) * F::PER_SM, max((int64_t)1, most)), F::THREADS, F::SMEM);
  return mx::launch(c, few_kernel<T, DIM, NT>, a);
}

// ------------------------------------------------------------------------------------------------ weights
// W[slot] = (old slot ? W[slot] : 0) + sum over the kv head's query rows of exp(S - lse): the first product again, with the
// rows' sums known.  Each weight is summed in one order, whatever the run.

// A tile of 8 rows in shared memory, as the product and the exponentials want it.
template <int DIM>
struct Rows {
  uint4 b[DIM / 32][32];
  float2 by[4], sum[4], minus_lse[4];                                  // of columns 2 c, 2 c + 1; no row: an lse of infinity
  int2 sees[4];
  int least, most;                                                     // slots that all rows see, that any does
  template <typename T>
  __device__ __forceinline__ void bring(const AttentionArgs& a, int64_t first, int n, int length, int h, int r0, int lane) {
    const int rows = n * a.group, c = lane & 3;
    Queries<T, DIM> q;
    q.load(a, first, rows, r0, h, lane);
#pragma unroll
    for (int w = 0; w < DIM / 32; ++w) b[w][lane] = q.b[w];
    if (lane < 4) {
      float lse[2];
      int slots[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int r = r0 + 2 * c + j, t = a.token_of(r);
        lse[j] = r < rows ? a.lse[(first + t) * a.q.heads + h * a.group + r - t * a.group] * -LOG2E : -INFINITY;
        slots[j] = r < rows ? length - n + t + 1 : 0;
      }
      by[c] = q.by;
      sum[c] = q.sum;
      minus_lse[c] = make_float2(lse[0], lse[1]);
      sees[c] = make_int2(slots[0], slots[1]);
      if (c == 0) {
        least = slots[0];
        most = r0 < rows ? length - n + a.token_of(min(r0 + 8, rows) - 1) + 1 : 0;
      }
    }
  }
  // The probabilities of products s of a key (parameters ks, ko), added to got.
  __device__ __forceinline__ void add(float2& got, float2 s, float2 ks, float2 ko, int slot, bool masked, int c) const {
    const float2 x = fma2(s, mul2(ks, by[c]), fma2(ko, sum[c], minus_lse[c]));
    float2 p = make_float2(exp2_of(x.x), exp2_of(x.y));
    if (masked) {
      if (slot >= sees[c].x) p.x = 0.f;
      if (slot >= sees[c].y) p.y = 0.f;
    }
    got = add2(got, p);
  }
};
// A weight from the lanes of its key: the sum of their columns.
__device__ __forceinline__ float over_columns(float2 got) {
  float w = got.x + got.y;
  w += __shfl_xor_sync(0xffffffffu, w, 1);
  return w + __shfl_xor_sync(0xffffffffu, w, 2);
}

// Few rows: the keys come as in few_kernel; the first two tiles of rows lie in shared memory, of this item and the next.  There is nothing to
// join, as a weight is its key's.  16 sequences up to 8192 slots, 8 kv heads of 128: 23 us on the GPU, 2.3 TB/s; the bytes take 8, and which part of
// the rest is start, lookup of pages, queries or the first copies has not been measured.
template <int DIM>
struct FewWeights {
  static constexpr int WARPS = DIM == 256 ? 8 : 10, PER_SM = 2, PLACES = DIM == 256 ? 2 : 4, TILES = 2;
  using Stages = Stream<DIM, 0, WARPS, PLACES, true>;
  static constexpr int SMEM = WARPS * PLACES * Stages::STAGE_BYTES;
};
template <typename T, int DIM>
__global__ void __launch_bounds__(FewWeights<DIM>::WARPS * 32, FewWeights<DIM>::PER_SM) few_weights_kernel(const AttentionArgs a) {
  using F = FewWeights<DIM>;
  using Stages = typename F::Stages;
  constexpr int WARPS = F::WARPS, PLACES = F::PLACES;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ typename Stages::List s_list[WARPS];
  __shared__ Rows<DIM> s_rows[2][F::TILES];
  __shared__ Share s_share;
  __shared__ int64_t s_sums[WARPS];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, c = lane & 3;
  if (tid < WARPS * PLACES) tc::mbar_init(tc::smem_u32(&s_list[tid / PLACES].full[tid % PLACES]), 1);
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  mx::wait_for_previous();
  mx::allow_next();
  const Share share = find_share(&s_share, a.batch.n_seqs, LEAST_STAGES, s_sums, [&](int b) {
    Sequence<0> s;
    s.describe(a, b);
    return s.units(a);
  });
  if (share.lo >= share.hi) return;
  __syncthreads();                                                      // the barriers are ready
  Walk<0> at;
  at.start(a, share);
  int slot0 = (int)(share.lo - at.begin + warp) * STAGE, page = 0;
  Stages stages{a, share, s_list[warp], smem + warp * PLACES * Stages::STAGE_BYTES, lane};
  stages.start(at, slot0);
  auto bring = [&](const Walk<0>& w, int into) {
    if (warp < F::TILES) s_rows[into][warp].template bring<T>(a, w.s.first, w.s.n, w.s.length, w.h, warp * 8, lane);
  };
  bring(at, 0);
  __syncthreads();
  while (true) {
    const int n = at.s.n, rows = n * a.group, length = at.s.length, end = at.end(share);
    const int64_t row = ((int64_t)at.b * a.cache.heads + at.h) * a.ld_slots;
    for (; slot0 < end; slot0 += WARPS * STAGE) {
      // the weights that are added to: lane l has that of key l of the stage
      const float old = a.weights && slot0 + lane < length - n ? a.weights[row + slot0 + lane] : 0.f;
      if (!stages.wait()) continue;
      const uint8_t* stage = stages.stage();
      const int valid = s_list[warp].valid[stages.place()];
      float2 got[2][2] = {};
      float ks[2][2], ko[2][2];
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const uint32_t p = *reinterpret_cast<const uint32_t*>(stage + u * Stages::GROUP_BYTES + GROUP * (DIM / 2) + key_of(g + 8 * e) * 4);
          ks[u][e] = scale_of(p);
          ko[u][e] = offset_of(p);
        }
      auto add = [&](const Rows<DIM>& r) {
        if (r.most <= slot0) return;
        float2 s[2][1][2];
        key_products<DIM, 1, 2, Stages::GROUP_BYTES>(s, stage, [&](int, int w) { return r.b[w][lane]; }, lane);
        const bool masked = slot0 + STAGE > r.least;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int e = 0; e < 2; ++e) r.add(got[u][e], s[u][0][e], both(ks[u][e]), both(ko[u][e]), slot0 + u * GROUP + key_of(g + 8 * e), masked, c);
      };
      for (int i = 0; i < min(F::TILES, (rows + 7) / 8); ++i) add(s_rows[page][i]);
      for (int r0 = 8 * F::TILES; r0 < rows; r0 += 8) {                 // a sequence with more rows than most have
        Queries<T, DIM> q;
        q.load(a, at.s.first, rows, r0, at.h, lane);
        float2 s[2][1][2];
        key_products<DIM, 1, 2, Stages::GROUP_BYTES>(s, stage, [&](int, int w) { return q.b[w]; }, lane);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int r = r0 + 2 * c + j, t = a.token_of(r), sees = r < rows ? length - n + t + 1 : 0;
          const float lse = r < rows ? a.lse[(at.s.first + t) * a.q.heads + at.h * a.group + r - t * a.group] * LOG2E : 0.f;
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const float x = (j ? s[u][0][e].y : s[u][0][e].x) * (ks[u][e] * (j ? q.by.y : q.by.x)) + (ko[u][e] * (j ? q.sum.y : q.sum.x) - lse);
              if (slot0 + u * GROUP + key_of(g + 8 * e) < sees) got[u][e].x += exp2_of(x);
            }
        }
      }
      // from the lanes of the keys' rows to a lane a key
      float mine = 0.f;
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float w = over_columns(got[u][e]);
          // key_of(r) for r = 8 e + g: c' = r / 2 % 4 for even r, (c' ^ 1) + 4 for odd ones
          const int key = lane & 15, low = key & 7, from = low < 4 ? 2 * low : 2 * ((low - 4) ^ 1) + 1;
          const float v = __shfl_sync(0xffffffffu, w, from * 4);
          if ((lane >> 4) == u && ((key >> 3) & 1) == e) mine = (valid >> u & 1) ? v : 0.f;
        }
      if (slot0 + lane < length) a.weights_out[row + slot0 + lane] = old + mine;
      const int place = stages.place();
      ++stages.turn;
      __syncwarp();
      stages.fetch(place);
    }
    if (at.begin + at.s.stages >= share.hi) break;
    slot0 -= at.s.stages * STAGE;
    at.next(a);
    bring(at, page ^ 1);
    page ^= 1;
    __syncthreads();
  }
  stages.end();
}

// Many rows: exponentials (16 a cycle and SM) are a quarter of the time, no unit is full (issue 35 %, tensor cores 22 %).  A warp holds 32 keys as fragments (D =
// 256: 16) and goes over the rows, 128 at a time from shared memory.  Bringing rows in costs a warp several times what a tile of them
// does afterwards, so the warps of a CTA hold different keys; the CTAs of a cluster hold the same and take blocks of 128 rows in turn.
// Where that leaves too few units for all SMs, `sets` warps of a CTA share keys too, and take a block's tiles in turn.  2 x 777 queries
// of 16 heads of 64 over 8191 slots: 123 us, of which exponentials are 28; one CTA for each block of keys, without clusters, 213.
template <int DIM>
struct ManyWeights {
  static constexpr int WARPS = DIM == 64 ? 16 : 12, N = DIM == 256 ? 1 : 2, WORDS = DIM / 32;
  static constexpr int KEYS = WARPS * N * GROUP;                       // of a CTA whose warps all have keys of their own
  static constexpr int TILES = 16;                                     // of 8 rows, in shared memory at once
  static constexpr int SMEM = 2 * TILES * (int)sizeof(Rows<DIM>);
};
__device__ __forceinline__ float load_of_rank(const float* p, int rank) {
  uint32_t at;
  float v;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(tc::smem_u32(p)), "r"(rank));
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(at) : "memory");
  return v;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
template <typename T, int DIM>
__global__ void __launch_bounds__(ManyWeights<DIM>::WARPS * 32, 1) many_weights_kernel(const AttentionArgs a, int cluster) {
  using W = ManyWeights<DIM>;
  constexpr int WARPS = W::WARPS, N = W::N, WORDS = W::WORDS, AT_ONCE = W::TILES * 8;
  extern __shared__ __align__(128) uint8_t smem[];
  Rows<DIM>* const rows_at = reinterpret_cast<Rows<DIM>*>(smem);       // [2][TILES]
  __shared__ Share s_share;
  __shared__ int64_t s_sums[WARPS];
  __shared__ float s_got[WARPS][N][2][8];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, c = lane & 3;
  mx::wait_for_previous();
  mx::allow_next();
  auto share_of = [&](int keys) {
    return find_share(&s_share, a.batch.n_seqs, 1, s_sums, [&](int b) { return (int64_t)a.cache.heads * ((a.cache.length(b) + keys - 1) / keys); });
  };
  int sets = 1;
  Share share = share_of(W::KEYS);
  const int clusters = gridDim.x / cluster, rank = blockIdx.x % cluster;
  while (sets < 4 && share.total * sets < clusters) sets *= 2;
  if (sets > 1) {
    __syncthreads();
    share = share_of(W::KEYS / sets);
  }
  // the clusters take the units in turn: neighbours cost about the same, the sequences do not
  const int keys = W::KEYS / sets, set = warp % sets;
  int seq = 0, n = 0, length = 0, tiles = 0;
  int64_t first = 0, before = 0;
  auto describe = [&]() {
    length = a.cache.length(seq);
    tiles = (length + keys - 1) / keys;
    a.batch.range(seq, first, n);
  };
  describe();
  for (int64_t unit = blockIdx.x / cluster; unit < share.total; unit += clusters) {
    while (unit >= before + (int64_t)tiles * a.cache.heads) {
      before += (int64_t)tiles * a.cache.heads;
      ++seq;
      describe();
    }
    const int h = (int)((unit - before) / tiles), tile = (int)((unit - before) - (int64_t)h * tiles);
    const int rows = n * a.group, base = tile * keys, slot0 = base + (warp / sets) * N * GROUP;
    // this warp's keys, as fragments
    uint32_t k[N][WORDS][2][4];
    float2 ks[N][2], ko[N][2];
    bool there[N];
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const int slot = slot0 + u * GROUP;
      const int64_t page = slot < length ? a.cache.page_of(seq, slot) : -1;
      there[u] = page >= 0;
      uint32_t x[2][WORDS], p[2] = {0u, 0u};
#pragma unroll
      for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int w = 0; w < WORDS; ++w) x[e][w] = 0u;
      if (there[u]) {
        const uint8_t* group = a.cache.group_at(page, h, slot, DIM);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          load_words<WORDS>(x[e], group + key_of(g + 8 * e) * (DIM / 2) + c * (DIM / 8));
          p[e] = *reinterpret_cast<const uint32_t*>(group + GROUP * (DIM / 2) + key_of(g + 8 * e) * 4);
        }
      }
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        ks[u][e] = both(scale_of(p[e]));
        ko[u][e] = both(offset_of(p[e]));
      }
#pragma unroll
      for (int w = 0; w < WORDS; ++w)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          k[u][w][e][0] = low_codes(x[0][w] >> (8 * e)); k[u][w][e][1] = low_codes(x[1][w] >> (8 * e));
          k[u][w][e][2] = high_codes(x[0][w] >> (8 * e)); k[u][w][e][3] = high_codes(x[1][w] >> (8 * e));
        }
    }
    float2 got[N][2];
#pragma unroll
    for (int u = 0; u < N; ++u) got[u][0] = got[u][1] = both(0.f);
    auto bring = [&](int row0, int into) {                              // rows row0 .. row0 + 127
      for (int i = warp; i < W::TILES && row0 + i * 8 < rows; i += WARPS)
        rows_at[into * W::TILES + i].template bring<T>(a, first, n, length, h, row0 + i * 8, lane);
    };
    // rows before the first one that sees these keys see nothing of them
    const int row_first = (int)(max((int64_t)0, (int64_t)base - (length - n)) * a.group / AT_ONCE + rank) * AT_ONCE, step = cluster * AT_ONCE;
    int page = 0;
    __syncthreads();
    bring(row_first, 0);
    __syncthreads();
    for (int row0 = row_first; row0 < rows; row0 += step, page ^= 1) {
      if (row0 + step < rows) bring(row0 + step, page ^ 1);
      const int count = min(W::TILES, (rows - row0 + 7) / 8);
      for (int i = set; i < count; i += sets) {
        const Rows<DIM>& q = rows_at[page * W::TILES + i];
        if (q.most <= slot0) continue;
        float d[N][2][4];
#pragma unroll
        for (int w = 0; w < WORDS; ++w) {
          const uint4 b = q.b[w][lane];
#pragma unroll
          for (int u = 0; u < N; ++u)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const uint32_t* x = k[u][w][e];
              if (w == 0) mma_first(d[u][e], x[0], x[1], x[2], x[3], e ? b.z : b.x, e ? b.w : b.y);
              else mma(d[u][e], x[0], x[1], x[2], x[3], e ? b.z : b.x, e ? b.w : b.y);
            }
        }
        const bool masked = slot0 + N * GROUP > q.least;
#pragma unroll
        for (int u = 0; u < N; ++u)
#pragma unroll
          for (int e = 0; e < 2; ++e)
            q.add(got[u][e], add2(make_float2(d[u][0][2 * e], d[u][0][2 * e + 1]), make_float2(d[u][1][2 * e], d[u][1][2 * e + 1])), ks[u][e],
                  ko[u][e], slot0 + u * GROUP + key_of(g + 8 * e), masked, c);
      }
      if (row0 + step < rows) __syncthreads();
    }
#pragma unroll
    for (int u = 0; u < N; ++u)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float w = over_columns(got[u][e]);
        if (c == 0) s_got[warp][u][e][g] = there[u] ? w : 0.f;
      }
    if (cluster > 1) cluster_sync();
    else __syncthreads();
    if (set == 0 && rank == 0 && c == 0)
#pragma unroll
      for (int u = 0; u < N; ++u)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int slot = slot0 + u * GROUP + key_of(g + 8 * e);
          if (slot < length) {
            const int64_t at = ((int64_t)seq * a.cache.heads + h) * a.ld_slots + slot;
            float w = a.weights && slot < length - n ? a.weights[at] : 0.f;
            for (int i = 0; i < sets; ++i)
              for (int r = 0; r < cluster; ++r) w += cluster > 1 ? load_of_rank(&s_got[warp + i][u][e][g], r) : s_got[warp + i][u][e][g];
            a.weights_out[at] = w;
          }
        }
    if (cluster > 1) cluster_sync();                                    // the others' sums have been read
  }
}

}  // namespace

int64_t attention_workspace(int dim) {
  return TICKET_BYTES + max((int64_t)MAX_CTAS * 2 * 16 * (dim + 2), MAX_SMS * prompt_part(dim)) * 4;
}

// Which of the two, for all sequences of a call, by their rows on average (the host does not know `starts`; a batch of decoding sequences and
// one long chunk is right either way, but the chunk, or the others, may take several times what the other kernel would): what 128 keys of
// every sequence take.  A CTA of prompt_kernel needs 2.5 us for them whatever part of its 256 rows
// there is, and as its items are not of equal length about half as much again; few_kernel takes 9.5 ns for each 16 rows, balanced over
// all SMs.  32 sequences of up to 2048 slots, 4 kv heads of 64, 80 rows on average: 44 and 68 us.  Where prompt_kernel's items are few
// it cuts their keys and joins the parts, which pays from 128 rows on (256 for D = 256, whose items are half as large): one sequence
// of 16384, 8 kv heads, 256 rows 72 and 106 us; 8 of up to 8192, 80 rows on average 169 and 121, 160 rows 175 and 221.
static bool prompt_is_faster(const mx::Device& dev, int dim, const AttentionArgs& a) {
  const int64_t rows = a.batch.tokens * a.group / a.batch.n_seqs, tile = dim == 256 ? 128 : 256;
  const int64_t items = a.batch.n_seqs * a.cache.heads * ((rows + tile - 1) / tile);
  if (rows >= (dim == 256 ? 256 : 128)) return true;
  if (rows < 64 || items < dev.sms / 2) return false;
  const int64_t sixteens = (a.batch.tokens * a.group / 16 + a.batch.n_seqs / 2) * a.cache.heads;
  return 3900 * ((items + dev.sms - 1) / dev.sms) < sixteens * 19 / 2;
}

dq_status attention(cudaStream_t stream, const mx::Device& dev, int dtype, int dim, const AttentionArgs& a) {
  if (prompt_is_faster(dev, dim, a)) return prompt_attention(stream, dev, dtype, dim, a);
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
  // up to two tiles of rows a sequence, on average: the keys' way from HBM is what takes time
  const bool few = a.batch.tokens * a.group <= (int64_t)16 * a.cache.n_seqs;
  const int64_t slots = (int64_t)a.cache.width << a.cache.shift, rows = (int64_t)a.cache.n_seqs * a.cache.heads;
  auto run = [&](auto t) {
    using T = decltype(t);
    return by_dim(dim, [&](auto d) {
      constexpr int DIM = decltype(d)::value;
      static SmemOptIn opted_few, opted_many;
      if (few) {
        using F = FewWeights<DIM>;
        DQ_CHECK(opt_in_dynamic_smem(few_weights_kernel<T, DIM>, F::SMEM, opted_few));
        const int64_t most = (rows * ((slots + STAGE - 1) / STAGE) + LEAST_STAGES - 1) / LEAST_STAGES;
        mx::LaunchConfig c(stream, min((int64_t)dev.sms * F::PER_SM, max((int64_t)1, most)), F::WARPS * 32, F::SMEM);
        return mx::launch(c, few_weights_kernel<T, DIM>, a);
      }
      using W = ManyWeights<DIM>;
      DQ_CHECK(opt_in_dynamic_smem(many_weights_kernel<T, DIM>, W::SMEM, opted_many));
      // CTAs of a cluster: two blocks of rows or more for each
      const int64_t each = a.batch.tokens * a.group / a.cache.n_seqs;
      const int cluster = each >= 8 * W::TILES * 8 ? 4 : each >= 4 * W::TILES * 8 ? 2 : 1;
      const int64_t units = max((int64_t)1, rows * ((slots * 4 + W::KEYS - 1) / W::KEYS));
      // no more clusters than run at once: they find their SMs together, 33 or so of four and not 37
      struct Clusters { int most[5]; };
      static PerDevice<Clusters> known;
      Clusters clusters;
      DQ_CHECK((dq_status)known.get(dev.index, clusters, [&](Clusters& out) -> int {
        out.most[1] = dev.sms;
        for (int s = 2; s <= 4; s *= 2) {
          mx::LaunchConfig config(nullptr, s, W::WARPS * 32, W::SMEM, s);
          DQ_CHECK_CUDA(cudaOccupancyMaxActiveClusters(&out.most[s], many_weights_kernel<T, DIM>, &config.cfg));
        }
        return DQ_OK;
      }));
      mx::LaunchConfig c(stream, min((int64_t)max(clusters.most[cluster], 1), units) * cluster, W::WARPS * 32, W::SMEM, cluster);
      return mx::launch(c, many_weights_kernel<T, DIM>, a, cluster);
    });
  };
  return dtype == DQ_BF16 ? run(__nv_bfloat16()) : run(__half());
}

}  // namespace kv
}  // namespace dq
