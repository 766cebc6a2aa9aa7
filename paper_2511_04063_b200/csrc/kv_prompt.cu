// Attention over a key/value cache in 4 bits for many query rows (a prompt's chunk), on the tensor cores' tcgen05 instructions.
//
// A CTA takes 256 query rows (D = 256: 128) of a sequence and kv head, in tiles of M = 128, and goes over the keys 128 at a time:
//     S = Q K^T (128 x 128, tensor memory),  P = exp(S - m) vs (fp16, over S in tensor memory),  O += P V (tensor memory)
// The operands are the codes, as in kv_attention.cu: fp16 subnormals c 2^-24, the values' less 8; keys' parameters are applied to S,
// the values' to P, sum_t p_t (vo_t + 8 vs_t) is added at the end.  Four bits become 16 on their way from global to shared memory:
// eight codes are one word and, as (0, 4), (1, 5), (2, 6), (3, 7), one 16-byte piece of a row, swizzled as the instructions want
// it; Q's dimensions are put in the same order, and the output's taken out of it.  Keys and values have the same layout, [token][64
// dimensions], read K-major by the first product and MN-major by the second.
//
// Warps: four for each tile of rows (a thread a row: scores, exponentials, P, O's rescaling), four that unpack (a thread a key), one
// that issues the products.  While one tile's rows are in the softmax the other's products run.  4096 queries of 32 heads over 16384
// slots: 570 us of products at the measured rate, 430 us of exponentials at 16 a cycle and SM.
#include "kv_common.cuh"
#include "tc_gemm.cuh"

namespace dq {
namespace kv {
namespace {

constexpr int KEYS = 128;                 // of a key tile
constexpr float SLACK = 8.f;              // a maximum may grow by this (in powers of two) before O is rescaled

template <int DIM>
struct Prompt {
  static constexpr int TILES = DIM == 256 ? 1 : 2;                     // of 128 rows
  static constexpr int STAGES = DIM == 64 ? 3 : DIM == 128 ? 2 : 1;    // of keys and values
  static constexpr int ROWS = TILES * 128;
  static constexpr int UNPACK = 4 * TILES, ISSUE = UNPACK + 4, THREADS = 32 * (ISSUE + 4);   // first warps of the roles
  // registers of a thread of each role's four warps; together no more than the launch's (65536 / THREADS each)
  static constexpr int ROW_REGS = DIM == 256 ? 224 : 192, UNPACK_REGS = DIM == 256 ? 152 : 80, ISSUE_REGS = 48;
  static_assert(TILES * ROW_REGS + UNPACK_REGS + ISSUE_REGS <= 65536 / THREADS / 8 * 8 * (TILES + 2), "");
  static constexpr int TILE_BYTES = 128 * DIM * 2, BOX = 128 * 128;    // a box: 128 rows of 64 values
  static constexpr int Q_AT = 0, K_AT = TILES * TILE_BYTES, V_AT = K_AT + STAGES * TILE_BYTES, END = V_AT + STAGES * TILE_BYTES;
  static constexpr int SMEM = END + 1024;
  static constexpr uint32_t O_COLUMN = TILES * 128;                    // of tensor memory, behind the scores
  static constexpr int PART = ROWS * (DIM + 2);
};

struct alignas(16) Params {                                            // of a key tile; read in 16-byte pieces
  float ks[KEYS], ko[KEYS], vs[KEYS], vo[KEYS];
  uint32_t field;                                                      // exponent field of the largest vs so far
  uint32_t valid;                                                      // groups of 16 keys that have a page
};

__device__ __forceinline__ bool elect_one() {
  uint32_t e;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(e));
  return e != 0;
}
// fp16 operands, fp32 sums: instruction descriptor of M = 128, N = n
__host__ __device__ constexpr uint32_t idesc_f16(int n) { return (1u << 4) | ((uint32_t)(n >> 3) << 17) | (8u << 24); }
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
               ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
               ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t at, const uint32_t* r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
               ::"r"(at), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
               "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void store16(uint32_t at, const uint4& v) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
// The 16-byte piece of dimensions 8 w .. 8 w + 7 of a row, in a tile of 128 rows.
__device__ __forceinline__ uint32_t piece_at(uint32_t tile, int row, int w) {
  return tile + (uint32_t)((w >> 3) * Prompt<128>::BOX + row * 128 + (((w & 7) ^ (row & 7)) << 4));
}

template <int N> __device__ __forceinline__ void more_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N> __device__ __forceinline__ void fewer_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }

template <typename T, int DIM>
__global__ void __launch_bounds__(Prompt<DIM>::THREADS, 1) prompt_kernel(const AttentionArgs a, int splits) {
  using P = Prompt<DIM>;
  constexpr int TILES = P::TILES, STAGES = P::STAGES, WORDS = DIM / 8;
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(16) Params s_params[STAGES];
  __shared__ __align__(8) uint64_t s_bars[2 + 4 * STAGES + 3 * TILES];
  __shared__ uint32_t s_tmem;
  __shared__ uint32_t s_fields[4];
  __shared__ Share s_share;
  __shared__ int64_t s_sums[P::THREADS / 32];
  __shared__ int s_last;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const uint32_t smem = (tc::smem_u32(smem_raw) + 1023u) & ~1023u, bars = tc::smem_u32(s_bars);
  auto bar = [&](int i) { return bars + 8u * (uint32_t)i; };
  const uint32_t q_full = bar(0), drained = bar(1);
  auto k_full = [&](int s) { return bar(2 + s); };
  auto k_empty = [&](int s) { return bar(2 + STAGES + s); };
  auto v_full = [&](int s) { return bar(2 + 2 * STAGES + s); };
  auto v_empty = [&](int s) { return bar(2 + 3 * STAGES + s); };
  auto s_full = [&](int m) { return bar(2 + 4 * STAGES + m); };
  auto p_full = [&](int m) { return bar(2 + 4 * STAGES + TILES + m); };
  auto pv_done = [&](int m) { return bar(2 + 4 * STAGES + 2 * TILES + m); };
  if (tid == 0) {
    tc::mbar_init(q_full, 4 * TILES);
    tc::mbar_init(drained, 1);
    for (int s = 0; s < STAGES; ++s) {
      tc::mbar_init(k_full(s), 4);
      tc::mbar_init(k_empty(s), 1);
      tc::mbar_init(v_full(s), 4);
      tc::mbar_init(v_empty(s), 1);
    }
    for (int m = 0; m < TILES; ++m) {
      tc::mbar_init(s_full(m), 1);
      tc::mbar_init(p_full(m), 4);
      tc::mbar_init(pv_done(m), 1);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  mx::wait_for_previous();
  mx::allow_next();
  // an item (or a part of its keys) a CTA: the grid has at least as many
  find_share(&s_share, a.batch.n_seqs, 1, s_sums, [&](int b) {
    int64_t first;
    int n;
    a.batch.range(b, first, n);
    return (((int64_t)n * a.group + P::ROWS - 1) / P::ROWS) * a.cache.heads * splits;
  });
  const Share share = s_share;
  if (share.lo >= share.hi) return;
  const int b = share.seq;
  int64_t first;
  int n;
  a.batch.range(b, first, n);
  const int rows = n * a.group, length = a.cache.length(b), row_tiles = (rows + P::ROWS - 1) / P::ROWS;
  // the tiles that see the most keys first
  const int item = (int)((share.lo - share.before) / splits), part = (int)((share.lo - share.before) % splits);
  const int h = item % a.cache.heads, row0 = (row_tiles - 1 - item / a.cache.heads) * P::ROWS;
  const int most = max(length - n + a.token_of(min(row0 + P::ROWS, rows) - 1) + 1, 0);
  const int all_tiles = (most + KEYS - 1) / KEYS;
  const int tile0 = (int)((int64_t)all_tiles * part / splits), key_tiles = (int)((int64_t)all_tiles * (part + 1) / splits) - tile0;
  if (warp == P::ISSUE) tc::tmem_alloc(tc::smem_u32(&s_tmem), 512);
  tc::tc_fence_before();
  __syncthreads();
  tc::tc_fence_after();
  const uint32_t tmem = s_tmem;

  bool ok = true;
  if (warp >= P::ISSUE) {   // ------------------------------------------------ products, by one warp
    fewer_registers<P::ISSUE_REGS>();   // (all four warps of a role: registers move by fours)
    if (warp == P::ISSUE) {
      auto wait = [&](uint32_t at, int phase) { return __all_sync(0xffffffffu, tc::mbar_wait(at, (uint32_t)phase & 1u, a.d_status)); };
      constexpr uint32_t SCORES = idesc_f16(KEYS), VALUES = idesc_f16(DIM) | tc::IDESC_B_MN_MAJOR;
      auto scores = [&](int m, int i) {
        const uint64_t q = tc::make_kmajor_sw128_desc(smem + P::Q_AT + m * P::TILE_BYTES);
        const uint64_t k = tc::make_kmajor_sw128_desc(smem + P::K_AT + (i % STAGES) * P::TILE_BYTES);
        if (elect_one()) {
#pragma unroll
          for (int s = 0; s < DIM / 16; ++s) {
            const uint32_t step = ((s >> 2) * P::BOX + (s & 3) * 32) >> 4;
            mma_ss(tmem + m * 128, q + step, k + step, SCORES, s > 0);
          }
          tc::umma_commit(s_full(m));
        }
        __syncwarp();
      };
      auto commit = [&](uint32_t at) {
        if (elect_one()) tc::umma_commit(at);
        __syncwarp();
      };
      if (key_tiles > 0) ok = wait(q_full, 0) && wait(k_full(0), 0);
      tc::tc_fence_after();
      if (ok && key_tiles > 0) {
        for (int m = 0; m < TILES; ++m) scores(m, 0);
        commit(k_empty(0));
      }
      for (int i = 0; i < key_tiles && ok; ++i) {
        const int s = i % STAGES, s1 = (i + 1) % STAGES;
        const uint64_t v = tc::make_mnmajor_sw128_desc(smem + P::V_AT + s * P::TILE_BYTES, P::BOX);
        ok = wait(v_full(s), i / STAGES);
        for (int m = 0; m < TILES && ok; ++m) {
          ok = wait(p_full(m), i);
          if (!ok) break;
          tc::tc_fence_after();
          if (elect_one()) {
#pragma unroll
            for (int k = 0; k < KEYS / 16; ++k)
              mma_ts(tmem + P::O_COLUMN + m * DIM, tmem + m * 128 + (k >> 1) * 32 + (k & 1) * 8, v + ((k * 16 * 128) >> 4), VALUES, i > 0 || k > 0);
            tc::umma_commit(pv_done(m));
          }
          __syncwarp();
          if (m == TILES - 1) commit(v_empty(s));
          if (i + 1 < key_tiles) {   // the next scores go over this P: it has to have been read
            if (m == 0) ok = wait(k_full(s1), (i + 1) / STAGES);
            ok = ok && wait(pv_done(m), i);
            if (!ok) break;
            tc::tc_fence_after();
            scores(m, i + 1);
            if (m == TILES - 1) commit(k_empty(s1));
          }
        }
      }
      commit(drained);   // nothing is in flight when tensor and shared memory are given up
      ok = wait(drained, 0) && ok;
    }
  } else if (warp >= P::UNPACK) {   // ---------------------------------------- codes to operands
    if constexpr (P::UNPACK_REGS < 65536 / P::THREADS / 8 * 8) fewer_registers<P::UNPACK_REGS>();
    const int t = tid - P::UNPACK * 32, w4 = warp - P::UNPACK;
    uint32_t k[WORDS], v[WORDS], kp = 0u, vp = 0u;
    bool there = false;
    auto fetch = [&](int i) {
      const int slot = (tile0 + i) * KEYS + t;
      const int64_t page = slot < length ? a.cache.page_of(b, slot) : -1;
      there = page >= 0;
      kp = vp = 0u;
      if (!there) return;
      const uint8_t* group = a.cache.group_at(page, h, slot, DIM);
      const int at = slot & (GROUP - 1);
#pragma unroll
      for (int w = 0; w < WORDS; w += 4) {
        const uint4 x = *reinterpret_cast<const uint4*>(group + at * (DIM / 2) + w * 4);
        const uint4 y = *reinterpret_cast<const uint4*>(group + GROUP * (DIM / 2 + 4) + at * (DIM / 2) + w * 4);
        k[w] = x.x; k[w + 1] = x.y; k[w + 2] = x.z; k[w + 3] = x.w;
        v[w] = y.x; v[w + 1] = y.y; v[w + 2] = y.z; v[w + 3] = y.w;
      }
      kp = *reinterpret_cast<const uint32_t*>(group + GROUP * (DIM / 2) + at * 4);
      vp = *reinterpret_cast<const uint32_t*>(group + GROUP * (DIM + 4) + at * 4);
    };
#pragma unroll
    for (int w = 0; w < WORDS; ++w) k[w] = v[w] = 0u;
    uint32_t field = 7u;
    if (key_tiles > 0) fetch(0);
    auto wait = [&](uint32_t at, int phase) { return __all_sync(0xffffffffu, tc::mbar_wait(at, (uint32_t)phase & 1u, a.d_status)); };
    // After a wait that gave up these warps go on without waiting: they meet at barriers of their own.
    for (int i = 0; i < key_tiles; ++i) {
      const int s = i % STAGES, turn = i / STAGES;
      ok = ok && wait(k_empty(s), turn + 1);
      const uint32_t k_tile = smem + P::K_AT + s * P::TILE_BYTES, v_tile = smem + P::V_AT + s * P::TILE_BYTES;
#pragma unroll
      for (int w = 0; w < WORDS; ++w) {
        const uint32_t x = k[w], y = x >> 8;
        store16(piece_at(k_tile, t, w), make_uint4(low_codes(x), high_codes(x), low_codes(y), high_codes(y)));
      }
      fence_async();
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(k_full(s));
      ok = ok && wait(v_empty(s), turn + 1);
      // (a NaN's field does not count: not all rows may see it)
      const uint32_t mine = vp >> 7 & 255u;
      const uint32_t largest = __reduce_max_sync(0xffffffffu, mine == 255u ? 0u : mine), votes = __ballot_sync(0xffffffffu, there);
      if (lane == 0) s_fields[w4] = largest | (votes & 1u) << 16 | (votes >> 16 & 1u) << 17;
      asm volatile("bar.sync 1, 128;" ::: "memory");
      uint32_t valid = 0u;
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        field = max(field, s_fields[x] & 255u);
        valid |= (s_fields[x] >> 16) << (2 * x);
      }
      asm volatile("bar.sync 1, 128;" ::: "memory");
      Params& p = s_params[s];
      const float vs = scale_of(vp);
      p.ks[t] = scale_of(kp);
      p.ko[t] = offset_of(kp);
      p.vs[t] = vs * __uint_as_float((260u - field) << 23);            // below 2^7
      p.vo[t] = offset_of(vp) + 8.f * vs;
      if (t == 0) { p.field = field; p.valid = valid; }
#pragma unroll
      for (int w = 0; w < WORDS; ++w) {
        const uint32_t x = v[w], y = x >> 8;
        store16(piece_at(v_tile, t, w), make_uint4(low_centred(x), high_centred(x), low_centred(y), high_centred(y)));
      }
      fence_async();
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(v_full(s));
      if (i + 1 < key_tiles) fetch(i + 1);
    }
  } else {   // ---------------------------------------------------------------- rows
    more_registers<P::ROW_REGS>();
    const int m = warp >> 2, r = (warp & 3) * 32 + lane, row = row0 + m * 128 + r;
    const bool there = row < rows;
    const int token = there ? a.token_of(row) : 0, head = h * a.group + (there ? row - token * a.group : 0);
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t s_at = tmem + lanes + m * 128, o_at = tmem + lanes + P::O_COLUMN + m * DIM;
    auto wait = [&](uint32_t at, int phase) { return __all_sync(0xffffffffu, tc::mbar_wait(at, (uint32_t)phase & 1u, a.d_status)); };
    // the row into shared memory, times a power of two that brings its largest value to 2^14 (odd dimensions 2^-4 less, as their codes
    // lie four bits up), and with the scale's sign
    float by, sum_by;
    {
      const T* p = reinterpret_cast<const T*>(a.q.p) + (first + token) * a.q.token + (int64_t)head * a.q.head;
      float most_q = 0.f, sum = 0.f;
      auto load = [&](int w) {
        mx::Vec8<T> x;
        x.clear();
        if (there) {
          if (a.q.vec) x.load(p + w * 8);
          else
#pragma unroll
            for (int e = 0; e < 4; ++e) x.set_pair(e, make_float2(mx::to_f32(p[w * 8 + 2 * e]), mx::to_f32(p[w * 8 + 2 * e + 1])));
        }
        return x;
      };
#pragma unroll 4
      for (int w = 0; w < WORDS; ++w) {
        const mx::Vec8<T> x = load(w);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 f = x.pair(e);
          sum += f.x + f.y;
          most_q = fmaxf(most_q, fmaxf(fabsf(f.x), fabsf(f.y)));
        }
      }
      const int field = min(max((int)mx::exponent_field(most_q), 14), 244);
      const float sign = a.scale < 0.f ? -1.f : 1.f;
      const float up = __uint_as_float((uint32_t)(268 - field) << 23) * sign, up4 = up * 0.0625f;
      by = fmaxf(__uint_as_float((uint32_t)(field + 10) << 23) * fabsf(a.scale) * LOG2E, 1.2e-38f);   // (not zero: it meets infinities)
      sum_by = sum * sign * (fabsf(a.scale) * LOG2E) / by;
      const uint32_t tile = smem + P::Q_AT + m * P::TILE_BYTES;
#pragma unroll 4
      for (int w = 0; w < WORDS; ++w) {
        const mx::Vec8<T> x = load(w);
        const float2 d01 = x.pair(0), d23 = x.pair(1), d45 = x.pair(2), d67 = x.pair(3);
        store16(piece_at(tile, r, w), make_uint4(half_pair(d01.x * up, d45.x * up), half_pair(d01.y * up4, d45.y * up4),
                                                 half_pair(d23.x * up, d67.x * up), half_pair(d23.y * up4, d67.y * up4)));
      }
      fence_async();
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(q_full);
    }
    const int sees = there ? max(length - n + token + 1, 0) : 0;
    // what all rows of the warp that there are see
    const int least = __reduce_min_sync(0xffffffffu, there ? sees : INT_MAX);
    float top = -INFINITY;
    float2 sum = both(0.f), off = both(0.f);
    uint32_t field = 7u;
    for (int i = 0; i < key_tiles && ok; ++i) {
      const int s = i % STAGES, slot0 = (tile0 + i) * KEYS;
      ok = wait(v_full(s), i / STAGES) && wait(s_full(m), i);
      if (!ok) break;
      tc::tc_fence_after();
      const Params& p = s_params[s];
      const uint32_t valid = p.valid;
      const bool masked = slot0 + KEYS > least || valid != 255u;
      uint32_t raw[4][32];
#pragma unroll
      for (int c = 0; c < 4; ++c) tc::tmem_ld32(s_at + 32 * c, raw[c]);
      float2 x[KEYS / 2];                                               // scores, without `by`
      float now = -INFINITY;
      tc::tmem_ld_wait();
#pragma unroll
      for (int e = 0; e < KEYS / 4; ++e) {
        const float4 ks = *reinterpret_cast<const float4*>(p.ks + 4 * e), ko = *reinterpret_cast<const float4*>(p.ko + 4 * e);
        const uint32_t* v = &raw[e >> 3][(e & 7) * 4];
        x[2 * e] = fma2(make_float2(ko.x, ko.y), both(sum_by), mul2(make_float2(__uint_as_float(v[0]), __uint_as_float(v[1])), make_float2(ks.x, ks.y)));
        x[2 * e + 1] = fma2(make_float2(ko.z, ko.w), both(sum_by), mul2(make_float2(__uint_as_float(v[2]), __uint_as_float(v[3])), make_float2(ks.z, ks.w)));
      }
      if (masked)
#pragma unroll
        for (int e = 0; e < KEYS / 2; ++e) {
          const bool none = !(valid >> (e >> 3) & 1u);
          if (none || slot0 + 2 * e >= sees) x[e].x = -INFINITY;
          if (none || slot0 + 2 * e + 1 >= sees) x[e].y = -INFINITY;
        }
#pragma unroll
      for (int e = 0; e < KEYS / 2; ++e) now = fmaxf(now, fmaxf(x[e].x, x[e].y));
      now *= by;
      const uint32_t wider = p.field - field;
      field = p.field;
      if (__any_sync(0xffffffffu, now > top + SLACK) || wider) {
        const float old = top;
        top = fmaxf(top, now);
        const float f = old == -INFINITY ? (sum.x + sum.y == 0.f ? 0.f : 1.f) : exp2_of(old - top);
        sum = mul2(sum, both(f));
        off = mul2(off, both(f));
        if (i > 0) {
          const float o_by = wider > 126u ? 0.f : f * __uint_as_float((127u - wider) << 23);
#pragma unroll 1
          for (int c = 0; c < DIM; c += 16) {
            uint32_t v[16];
            tc::tmem_ld16(o_at + c, v);
            tc::tmem_ld_wait();
#pragma unroll
            for (int e = 0; e < 16; ++e) v[e] = __float_as_uint(__uint_as_float(v[e]) * o_by);
            tmem_st16(o_at + c, v);
          }
        }
      }
      const float base = top == -INFINITY ? 0.f : -top;
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        uint32_t packed[16];
#pragma unroll
        for (int e = 0; e < 16; e += 2) {
          const float4 vs = *reinterpret_cast<const float4*>(p.vs + 32 * c + 2 * e), vo = *reinterpret_cast<const float4*>(p.vo + 32 * c + 2 * e);
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const float2 u = j ? make_float2(vs.z, vs.w) : make_float2(vs.x, vs.y), o = j ? make_float2(vo.z, vo.w) : make_float2(vo.x, vo.y);
            const float2 z = x[16 * c + e + j];
            float2 q = fma2(z, both(by), both(base)), pv, po;
            q = make_float2(exp2_of(q.x), exp2_of(q.y));
            sum = add2(sum, q);
            pv = mul2(q, u);
            if (!masked) off = fma2(q, o, off);
            else {   // (a NaN times the zero of a row that does not see it)
              po = mul2(q, o);
              if (z.x == -INFINITY) pv.x = po.x = 0.f;
              if (z.y == -INFINITY) pv.y = po.y = 0.f;
              off = add2(off, po);
            }
            packed[e + j] = half_pair(pv.x, pv.y);
          }
        }
        tmem_st16(s_at + 32 * c, packed);
      }
      tmem_st_wait();
      tc::tc_fence_before();
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(p_full(m));
    }
    if (ok && key_tiles > 0) ok = wait(pv_done(m), key_tiles - 1);
    tc::tc_fence_after();
    if (ok) {
      const float l = sum.x + sum.y, o0 = off.x + off.y;
      const float grow = __uint_as_float((field - 6u) << 23);
      const float low = key_tiles > 0 ? grow * 16777216.f : 0.f, high = key_tiles > 0 ? grow * 1048576.f : 0.f;
      float* part_at = reinterpret_cast<float*>(a.workspace + TICKET_BYTES) + (int64_t)blockIdx.x * P::PART;
      const float over = l == 0.f ? 0.f : 1.f / l;
      T* out = reinterpret_cast<T*>(a.out.p) + (first + token) * a.out.token + (int64_t)head * a.out.head;
#pragma unroll 1
      for (int c = 0; c < DIM; c += 16) {
        uint32_t v[16];
        tc::tmem_ld16(o_at + c, v);
        tc::tmem_ld_wait();
#pragma unroll
        for (int e = 0; e < 16; e += 8) {
          // a piece's columns are the dimensions 0, 4, 1, 5, 2, 6, 3, 7
          float d[8];
#pragma unroll
          for (int x = 0; x < 8; ++x) {
            const float o = key_tiles > 0 ? __uint_as_float(v[e + x]) : 0.f;
            d[(x >> 1) + 4 * (x & 1)] = o * (x & 2 ? high : low) + o0;
          }
          if (splits > 1) {
            // (by column, rows side by side: the joining CTA reads them so)
#pragma unroll
            for (int x = 0; x < 8; ++x) __stcg(part_at + (int64_t)(c + e + x) * P::ROWS + m * 128 + r, d[x]);
          } else if (there) {
            mx::Vec8<T> y;
#pragma unroll
            for (int x = 0; x < 4; ++x) y.set_pair(x, make_float2(d[2 * x] * over, d[2 * x + 1] * over));
            if (a.out.vec) y.store(out + c + e);
            else
#pragma unroll
              for (int x = 0; x < 8; ++x) out[c + e + x] = mx::from_f32<T>(d[x] * over);
          }
        }
      }
      if (splits > 1) {
        __stcg(part_at + (int64_t)DIM * P::ROWS + m * 128 + r, top);
        __stcg(part_at + (int64_t)(DIM + 1) * P::ROWS + m * 128 + r, l);
        __threadfence();
      } else if (there && a.lse) a.lse[(first + token) * a.q.heads + head] = l == 0.f ? -INFINITY : (top + log2f(l)) * LN2;
    }
    tc::tc_fence_before();
    if (splits > 1) {   // the CTA that finishes an item last joins its parts, in order; a thread a row (only these warps have registers)
      int* ticket = reinterpret_cast<int*>(a.workspace) + (blockIdx.x - part);
      asm volatile("bar.sync 2, %0;" ::"n"(P::ROWS) : "memory");
      if (tid == 0) s_last = atomicAdd(ticket, 1) == splits - 1;
      asm volatile("bar.sync 2, %0;" ::"n"(P::ROWS) : "memory");
      if (s_last) {
        __threadfence();
        if (tid == 0) *ticket = 0;
        if (there) {
          const float* parts = reinterpret_cast<const float*>(a.workspace + TICKET_BYTES) + (int64_t)(blockIdx.x - part) * P::PART + m * 128 + r;
          float all_top = -INFINITY, l = 0.f;
          for (int i = 0; i < splits; ++i) all_top = fmaxf(all_top, __ldcg(parts + (int64_t)i * P::PART + (int64_t)DIM * P::ROWS));
          for (int i = 0; i < splits; ++i) {
            const float* p = parts + (int64_t)i * P::PART;
            const float pl = __ldcg(p + (int64_t)(DIM + 1) * P::ROWS), pm = __ldcg(p + (int64_t)DIM * P::ROWS);
            l += pl == 0.f ? 0.f : pl * (pm == -INFINITY ? 1.f : exp2_of(pm - all_top));
          }
          const float over = l == 0.f ? 0.f : 1.f / l;
          T* out = reinterpret_cast<T*>(a.out.p) + (first + token) * a.out.token + (int64_t)head * a.out.head;
          if (a.lse) a.lse[(first + token) * a.q.heads + head] = l == 0.f ? -INFINITY : (all_top + log2f(l)) * LN2;
#pragma unroll 1
          for (int d = 0; d < DIM; d += 16) {
            float o[16] = {};
            for (int i = 0; i < splits; ++i) {
              const float* p = parts + (int64_t)i * P::PART;
              const float pm = __ldcg(p + (int64_t)DIM * P::ROWS);
              const float f = pm == -INFINITY ? 1.f : exp2_of(pm - all_top);   // (where there is no sum O is zero)
#pragma unroll
              for (int x = 0; x < 16; ++x) o[x] += __ldcg(p + (int64_t)(d + x) * P::ROWS) * f;
            }
#pragma unroll
            for (int x = 0; x < 16; ++x) out[d + x] = mx::from_f32<T>(o[x] * over);
          }
        }
      }
    }
  }
  __syncthreads();
  if (warp == P::ISSUE) {
    tc::tc_fence_after();
    tc::tmem_dealloc(tmem, 512);
  }
}

template <typename T, int DIM>
dq_status run(cudaStream_t stream, const mx::Device& dev, const AttentionArgs& a) {
  using P = Prompt<DIM>;
  static SmemOptIn opted;
  DQ_CHECK(opt_in_dynamic_smem(prompt_kernel<T, DIM>, P::SMEM, opted));
  const int64_t items = (a.batch.tokens * a.group / P::ROWS + a.batch.n_seqs) * a.cache.heads;
  // Fewer items than SMs: their keys are cut, in pieces that are worth a CTA's way (4 tiles).
  const int64_t key_tiles = max((int64_t)1, (((int64_t)a.cache.width << a.cache.shift) + KEYS - 1) / KEYS);
  const int64_t splits = items >= dev.sms ? 1 : max((int64_t)1, min((int64_t)min(dev.sms, MAX_SMS) / items, key_tiles / 4));
  mx::LaunchConfig c(stream, items * splits, P::THREADS, P::SMEM);
  return mx::launch(c, prompt_kernel<T, DIM>, a, (int)splits);
}

}  // namespace

dq_status prompt_attention(cudaStream_t stream, const mx::Device& dev, int dtype, int dim, const AttentionArgs& a) {
  auto by_type = [&](auto t) {
    using T = decltype(t);
    return by_dim(dim, [&](auto d) { return run<T, decltype(d)::value>(stream, dev, a); });
  };
  return dtype == DQ_BF16 ? by_type(__nv_bfloat16()) : by_type(__half());
}

}  // namespace kv
}  // namespace dq
