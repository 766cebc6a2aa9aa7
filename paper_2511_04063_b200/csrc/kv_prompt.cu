// Attention over a key/value cache in 4 bits for many query rows (a prompt's chunk), on the tensor cores' tcgen05 instructions.
//
// A CTA takes 256 query rows (D = 256: 128) of a sequence and kv head, in tiles of M = 128, and goes over the keys 128 at a time:
//     S = Q K^T (128 x 128, tensor memory),  P = exp(S - m) (fp16, tensor memory),  O += P V (tensor memory)
// Four bits become 16 on their way from global to shared memory.  A code alone is the fp16 subnormal c 2^-24, and one multiply-add
// makes it  ks (c - 8)  for a key: 8 bits of scale times 3 of code.  What is left of a key, (ko + 8 ks) times the sum of the query,
// is added to the score in fp32.  A value becomes  vs c + vo,  rounded to fp16 (2^-11, as P is).  The factor of a code is 2^24 times a
// scale, so the largest scale of a tile is held between 2^-10 and 2^-9, seen by a row or not, and fp16's least step is 2^-14 of it: keys are exact
// where their scales are within 2^-7 of the tile's largest, and an element of a smaller one is off by up to 2^-14 of the largest (two
// roundings), as an element of a value is of the largest so far (or 2^-28 of the largest value, where that is far above its scale).  Codes
// shifted to the upper bits of the mantissa, each by itself, would leave 2^-20; they took 1110 us instead of 1079 for the case below, and
// 429 instead of 414 for D = 256.  Parameters are applied here, by a
// thread a key, because a thread of the softmax meets every key: read from shared memory for each of them, four numbers a key took
// 4100 cycles of a key tile's 10000.  Powers of two keep all of it in fp16's range: the largest ks of a tile below 2^-9, the values by the
// largest so far, the rows of Q with their largest value at 2^14.  Eight codes are one word and, as (0, 4), (1, 5), (2, 6), (3, 7), one
// 16-byte piece of a row, swizzled as the instructions want it; Q's dimensions are put in the same order, and the output's taken out
// of it.  Keys and values have the same layout, [token][64 dimensions], read K-major by the first product and MN-major by the second.
//
// Warps: four for each tile of rows (a thread a row: scores, exponentials, P, O's rescaling), four that unpack (a thread a key), one
// that issues the products.  While one tile's rows are in the softmax the other's products run.  The two tiles share one place for S,
// which is free again as soon as its rows have it in registers, so that a tile's next scores are there when its softmax is done (P over
// S, and the next scores behind its product: 1110 us for the case below when this took 1061; a warp for each tile's products 1577, because
// instructions of two sums take turns; S in halves of 64 keys with a place each 1353: 64 columns take as long as 128).
//
// 4096 queries of 32 heads of 128 over 16384 slots: 1077 to 1122 us in a long row of calls (1061 in a short one, cool), 51 to 53 % of the
// measured rate; 570 us of products at that rate (562 measured with nothing between them) and 430 us of exponentials at 16 a cycle and SM.  Left
// out of a copy that took 1061: exponentials 1020 us, the unpackers' stores 980, both and all reads of scores 794.  The rest is the way from product to
// softmax and back, and the last round of CTAs: 512 items of 97 to 128 key tiles, the longest first, end on 148 SMs after 441 tiles, where an
// even share is 389.
#include "kv_common.cuh"
#include "tc_gemm.cuh"

namespace dq {
namespace kv {
namespace {

constexpr int KEYS = 128;                 // of a key tile
constexpr float SLACK = 8.f;              // a maximum may grow by this (in powers of two) before O is rescaled
constexpr float LIFT = 6.f;               // P is held 2^6 larger: with SLACK below 2^14, and 2^-20 of the largest is a normal number yet

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
  static constexpr uint32_t P_COLUMN = KEYS, O_COLUMN = 2 * KEYS;      // of tensor memory, behind the scores of one tile
  static constexpr int PART = ROWS * (DIM + 2);
};

struct alignas(16) Params {                                            // of a key tile; read in 16-byte pieces
  float kz[KEYS];                                                      // (ko + 8 ks) 2^-10 / grow
  float grow;                                                          // power of two of the tile's scores, which are 2^-10 of it
  uint32_t field;                                                      // the values' power of two: exponent field, the largest so far
  uint32_t valid;                                                      // groups of 16 keys that have a page
  int odd;                                                             // the first key whose value is a NaN
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
  __shared__ __align__(8) uint64_t s_bars[3 + (2 + 2 * TILES) * STAGES + 2 * TILES];
  __shared__ uint32_t s_tmem;
  __shared__ uint32_t s_keys[2][4], s_values[2][4];
  __shared__ int s_odd[2][4];
  __shared__ Share s_share;
  __shared__ int64_t s_sums[P::THREADS / 32];
  __shared__ int s_last;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const uint32_t smem = (tc::smem_u32(smem_raw) + 1023u) & ~1023u, bars = tc::smem_u32(s_bars);
  auto bar = [&](int i) { return bars + 8u * (uint32_t)i; };
  const uint32_t q_full = bar(0), drained = bar(1);
  auto k_full = [&](int s) { return bar(2 + s); };
  auto v_full = [&](int s) { return bar(2 + STAGES + s); };
  // of a tile of rows and a stage: the scores are there, and the keys read; the values' product is done, and P and the values read
  auto s_full = [&](int m, int s) { return bar(2 + 2 * STAGES + m * STAGES + s); };
  auto pv_done = [&](int m, int s) { return bar(2 + 2 * STAGES + (TILES + m) * STAGES + s); };
  auto p_half = [&](int m) { return bar(2 + (2 + 2 * TILES) * STAGES + m); };
  auto p_full = [&](int m) { return bar(2 + (2 + 2 * TILES) * STAGES + TILES + m); };
  const uint32_t s_taken = bar(2 + (2 + 2 * TILES) * STAGES + 2 * TILES);   // the scores are in registers
  if (tid == 0) {
    tc::mbar_init(q_full, 4 * TILES);
    tc::mbar_init(drained, 1);
    tc::mbar_init(s_taken, 4);
    for (int s = 0; s < STAGES; ++s) {
      tc::mbar_init(k_full(s), 4);
      tc::mbar_init(v_full(s), 4);
      for (int m = 0; m < TILES; ++m) {
        tc::mbar_init(s_full(m, s), 1);
        tc::mbar_init(pv_done(m, s), 1);
      }
    }
    for (int m = 0; m < TILES; ++m) {
      tc::mbar_init(p_half(m), 4);
      tc::mbar_init(p_full(m), 4);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  mx::wait_for_previous();
  mx::allow_next();
  // an item (or a part of its keys) a CTA: the grid has at least as many
  const Share share = find_share(&s_share, a.batch.n_seqs, 1, s_sums, [&](int b) {
    int64_t first;
    int n;
    a.batch.range(b, first, n);
    return (((int64_t)n * a.group + P::ROWS - 1) / P::ROWS) * a.cache.heads * splits;
  });
  if (share.lo >= share.hi || share.total > gridDim.x) return;   // (more than the grid was made for: starts that decrease)
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
      const int items = key_tiles * TILES;
      auto scores = [&](int item) {                                     // of tiles (item / TILES) of keys and (item % TILES) of rows
        const int i = item / TILES, m = item % TILES, s = i % STAGES;
        if (m == 0) ok = wait(k_full(s), i / STAGES);
        if (item > 0) ok = ok && wait(s_taken, item - 1);
        if (!ok) return;
        tc::tc_fence_after();
        const uint64_t q = tc::make_kmajor_sw128_desc(smem + P::Q_AT + m * P::TILE_BYTES);
        const uint64_t k = tc::make_kmajor_sw128_desc(smem + P::K_AT + s * P::TILE_BYTES);
        if (elect_one()) {
#pragma unroll
          for (int x = 0; x < DIM / 16; ++x) {
            const uint32_t step = ((x >> 2) * P::BOX + (x & 3) * 32) >> 4;
            mma_ss(tmem, q + step, k + step, SCORES, x > 0);
          }
          tc::umma_commit(s_full(m, s));
        }
        __syncwarp();
      };
      if (items > 0) {
        ok = wait(q_full, 0);
        for (int item = 0; item < 2 * TILES - 1 && item < items && ok; ++item) scores(item);
      }
      for (int i = 0; i < key_tiles && ok; ++i) {
        const int s = i % STAGES;
        const uint64_t v = tc::make_mnmajor_sw128_desc(smem + P::V_AT + s * P::TILE_BYTES, P::BOX);
        ok = wait(v_full(s), i / STAGES);
        for (int m = 0; m < TILES && ok; ++m) {
          auto values = [&](int half) {
            tc::tc_fence_after();
            if (elect_one()) {
#pragma unroll
              for (int x = 4 * half; x < 4 * half + 4; ++x)
                mma_ts(tmem + P::O_COLUMN + m * DIM, tmem + P::P_COLUMN + m * (KEYS / 2) + x * 8, v + ((x * 16 * 128) >> 4), VALUES, i > 0 || x > 0);
              if (half) tc::umma_commit(pv_done(m, s));
            }
            __syncwarp();
          };
          ok = wait(p_half(m), i);                                      // the first keys' P, while the others' is formed
          if (!ok) break;
          values(0);
          ok = wait(p_full(m), i);
          if (!ok) break;
          values(1);
          // (of two tiles, these rows have their next scores already, the other's have not)
          const int next = i * TILES + m + 2 * TILES - 1;
          if (next < items) scores(next);
        }
      }
      if (elect_one()) tc::umma_commit(drained);   // nothing is in flight when tensor and shared memory are given up
      __syncwarp();
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
    uint32_t field = 10u;
    if (key_tiles > 0) fetch(0);
    auto wait = [&](uint32_t at, int phase) { return __all_sync(0xffffffffu, tc::mbar_wait(at, (uint32_t)phase & 1u, a.d_status)); };
    // eight codes times a factor (`high`: of the codes four bits up) plus an offset, as a piece of a row
    auto store = [&](uint32_t at, uint32_t x, __half2 low, __half2 high, __half2 offset) {
      auto value = [&](uint32_t code, __half2 by) {
        const __half2 r = __hfma2(*reinterpret_cast<const __half2*>(&code), by, offset);
        return *reinterpret_cast<const uint32_t*>(&r);
      };
      const uint32_t y = x >> 8;
      store16(at, make_uint4(value(low_codes(x), low), value(high_codes(x), high), value(low_codes(y), low), value(high_codes(y), high)));
    };
    // After a wait that gave up these warps go on without waiting: they meet at barriers of their own.
    for (int i = 0; i < key_tiles; ++i) {
      const int s = i % STAGES, turn = i / STAGES;
      const float ks = scale_of(kp), kz = offset_of(kp) + 8.f * ks, vs = scale_of(vp), vo = offset_of(vp);
      // exponent fields of the tile's largest ks, and of what the values are divided by: vs below 2, values below 2^16, both held 2^10
      // smaller.  (That factor stands apart: with it the powers of two of the largest numbers would leave fp32's range.)  A NaN does
      // not count, and a value that is one is held as zero: not all rows may see it.
      auto nan_of = [](float v) { return !(fabsf(v) <= 3.402823466e38f); };
      const bool nan = nan_of(vs) || nan_of(vo);
      // (and kz within 2^91, where a tile's scales are small or zero)
      const int k_field = nan_of(ks) || nan_of(kz) ? 0 : max((int)(kp >> 7 & 255u), (int)mx::exponent_field(kz) - 100), spread = (int)(vp >> 7 & 255u);
      const int size = (int)max(mx::exponent_field(vo), mx::exponent_field(fmaf(15.f, vs, vo))) - 14;
      const uint32_t k_most = __reduce_max_sync(0xffffffffu, (uint32_t)k_field);
      const uint32_t v_most = __reduce_max_sync(0xffffffffu, nan ? 0u : (uint32_t)max(spread, size));
      const uint32_t votes = __ballot_sync(0xffffffffu, there), odd = __ballot_sync(0xffffffffu, nan);
      if (lane == 0) {
        s_keys[i & 1][w4] = k_most;
        s_values[i & 1][w4] = v_most | (votes & 1u) << 16 | (votes >> 16 & 1u) << 17;
        s_odd[i & 1][w4] = odd ? (tile0 + i) * KEYS + w4 * 32 + __ffs(odd) - 1 : INT_MAX;
      }
      asm volatile("bar.sync 1, 128;" ::: "memory");
      uint32_t valid = 0u, key_field = 10u;
      int first_odd = INT_MAX;
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        key_field = max(key_field, s_keys[i & 1][x]);
        field = max(field, s_values[i & 1][x] & 0xffffu);
        valid |= (s_values[i & 1][x] >> 16) << (2 * x);
        first_odd = min(first_odd, s_odd[i & 1][x]);
      }
      key_field = min(key_field, 253u);
      field = min(field, 253u);
      const float k_by = __uint_as_float((254u - key_field) << 23), v_by = __uint_as_float((254u - field) << 23);
      const uint32_t k_tile = smem + P::K_AT + s * P::TILE_BYTES, v_tile = smem + P::V_AT + s * P::TILE_BYTES;
      constexpr float SMALLER = 1.f / 1024.f, LOW = SMALLER * 16777216.f, HIGH = SMALLER * 1048576.f;   // (2^24 and 2^20: of the codes)
      ok = ok && wait(s_full(TILES - 1, s), turn + 1);
      {
        const float by = ks * k_by;
        const __half2 low = __float2half2_rn(by * LOW), high = __float2half2_rn(by * HIGH), offset = __float2half2_rn(-8.f * SMALLER * by);
#pragma unroll
        for (int w = 0; w < WORDS; ++w) store(piece_at(k_tile, t, w), k[w], low, high, offset);
      }
      fence_async();
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(k_full(s));
      ok = ok && wait(pv_done(TILES - 1, s), turn + 1);
      Params& p = s_params[s];
      p.kz[t] = kz * k_by * SMALLER;
      if (t == 0) {
        p.grow = __uint_as_float(key_field << 23);
        p.field = field;
        p.valid = valid;
        p.odd = first_odd;
      }
      {
        const float by = nan ? 0.f : vs * v_by;
        const __half2 low = __float2half2_rn(by * LOW), high = __float2half2_rn(by * HIGH), offset = __float2half2_rn(nan ? 0.f : vo * v_by * SMALLER);
#pragma unroll
        for (int w = 0; w < WORDS; ++w) store(piece_at(v_tile, t, w), v[w], low, high, offset);
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
    const uint32_t s_at = tmem + lanes, p_at = tmem + lanes + P::P_COLUMN + m * (KEYS / 2), o_at = tmem + lanes + P::O_COLUMN + m * DIM;
    auto wait = [&](uint32_t at, int phase) { return __all_sync(0xffffffffu, tc::mbar_wait(at, (uint32_t)phase & 1u, a.d_status)); };
    // the row into shared memory, times a power of two that brings its largest value to 2^14, and with the scale's sign
    float by, sum_by;
    {
      const T* p = reinterpret_cast<const T*>(a.q.p) + (first + token) * a.q.token + (int64_t)head * a.q.head;
      float most_q = 0.f, sum = 0.f;
      mx::Vec8<T> x[WORDS];                                             // (all of the row's loads at once)
#pragma unroll
      for (int w = 0; w < WORDS; ++w) {
        x[w].clear();
        if (there) {
          if (a.q.vec) x[w].load(p + w * 8);
          else
#pragma unroll
            for (int e = 0; e < 4; ++e) x[w].set_pair(e, make_float2(mx::to_f32(p[w * 8 + 2 * e]), mx::to_f32(p[w * 8 + 2 * e + 1])));
        }
      }
#pragma unroll
      for (int w = 0; w < WORDS; ++w)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 f = x[w].pair(e);
          sum += f.x + f.y;
          most_q = fmaxf(most_q, fmaxf(fabsf(f.x), fabsf(f.y)));
        }
      const int field = min(max((int)mx::exponent_field(most_q), 15), 244);
      const float up = __uint_as_float((uint32_t)(268 - field) << 23) * (a.scale < 0.f ? -1.f : 1.f);
      by = __uint_as_float((uint32_t)(field - 4) << 23) * fabsf(a.scale) * LOG2E;   // (the scores' 2^10 with it)
      sum_by = sum * up;
      const uint32_t tile = smem + P::Q_AT + m * P::TILE_BYTES;
#pragma unroll
      for (int w = 0; w < WORDS; ++w) {
        const float2 d01 = x[w].pair(0), d23 = x[w].pair(1), d45 = x[w].pair(2), d67 = x[w].pair(3);
        store16(piece_at(tile, r, w), make_uint4(half_pair(d01.x * up, d45.x * up), half_pair(d01.y * up, d45.y * up),
                                                 half_pair(d23.x * up, d67.x * up), half_pair(d23.y * up, d67.y * up)));
      }
      fence_async();
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(q_full);
    }
    const int sees = there ? max(length - n + token + 1, 0) : 0;
    // what all rows of the warp that there are see
    const int least = __reduce_min_sync(0xffffffffu, there ? sees : INT_MAX);
    float top = -INFINITY;
    float2 sum = both(0.f);
    uint32_t field = 10u;
    bool odd = false;                                                   // the row sees a value that is a NaN
    for (int i = 0; i < key_tiles && ok; ++i) {
      const int s = i % STAGES, slot0 = (tile0 + i) * KEYS;
      ok = wait(v_full(s), i / STAGES) && wait(s_full(m, s), i / STAGES);
      if (!ok) break;
      tc::tc_fence_after();
      const Params& p = s_params[s];
      const uint32_t valid = p.valid;
      const bool masked = slot0 + KEYS > least || valid != 255u;
      uint32_t raw[4][32];
#pragma unroll
      for (int c = 0; c < 4; ++c) tc::tmem_ld32(s_at + 32 * c, raw[c]);
      float2 x[KEYS / 2];                                               // scores, without `tile_by`
      float tile_by = by * p.grow;
      odd |= p.odd < sees;
      tc::tmem_ld_wait();
      tc::tc_fence_before();
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(s_taken);
#pragma unroll
      for (int e = 0; e < KEYS / 4; ++e) {
        const float4 kz = *reinterpret_cast<const float4*>(p.kz + 4 * e);
        const uint32_t* v = &raw[e >> 3][(e & 7) * 4];
        x[2 * e] = fma2(make_float2(kz.x, kz.y), both(sum_by), make_float2(__uint_as_float(v[0]), __uint_as_float(v[1])));
        x[2 * e + 1] = fma2(make_float2(kz.z, kz.w), both(sum_by), make_float2(__uint_as_float(v[2]), __uint_as_float(v[3])));
      }
      if (masked) {   // behind the factor, which may be zero: a row of zeros, keys without a range, a scale of zero
#pragma unroll
        for (int e = 0; e < KEYS / 2; ++e) {
          const bool none = !(valid >> (e >> 3) & 1u);
          x[e] = mul2(x[e], both(tile_by));
          if (none || slot0 + 2 * e >= sees) x[e].x = -INFINITY;
          if (none || slot0 + 2 * e + 1 >= sees) x[e].y = -INFINITY;
        }
        tile_by = 1.f;
      }
      // (four chains: in one, each maximum waits for the one before)
      float most_of[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
      for (int e = 0; e < KEYS / 2; ++e) most_of[e & 3] = fmaxf(most_of[e & 3], fmaxf(x[e].x, x[e].y));
      const float now = fmaxf(fmaxf(most_of[0], most_of[1]), fmaxf(most_of[2], most_of[3])) * tile_by;
      if (i > 0) {   // P and O are this thread's again
        ok = wait(pv_done(m, (i - 1) % STAGES), (i - 1) / STAGES);
        if (!ok) break;
        tc::tc_fence_after();
      }
      const uint32_t wider = p.field - field;
      field = p.field;
      if (__any_sync(0xffffffffu, now > top + SLACK) || wider) {
        const float old = top;
        top = fmaxf(top, now);
        const float f = old == -INFINITY ? (sum.x + sum.y == 0.f ? 0.f : 1.f) : exp2_of(old - top);
        sum = mul2(sum, both(f));
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
      const float base = top == -INFINITY ? 0.f : LIFT - top;
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        uint32_t packed[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          float2 q = fma2(x[16 * c + e], both(tile_by), both(base));
          q = make_float2(exp2_of(q.x), exp2_of(q.y));
          sum = add2(sum, q);
          packed[e] = half_pair(q.x, q.y);
        }
        tmem_st16(p_at + 16 * c, packed);
        if (c & 1) {
          tmem_st_wait();
          tc::tc_fence_before();
          __syncwarp();
          if (lane == 0) tc::mbar_arrive(c == 1 ? p_half(m) : p_full(m));
        }
      }
    }
    if (ok && key_tiles > 0) ok = wait(pv_done(m, (key_tiles - 1) % STAGES), (key_tiles - 1) / STAGES);
    tc::tc_fence_after();
    if (ok) {
      const float l = sum.x + sum.y;
      const float grow = odd ? __uint_as_float(0x7fc00000u) : __uint_as_float(field << 23);
      float* part_at = reinterpret_cast<float*>(a.workspace + TICKET_BYTES) + (int64_t)blockIdx.x * P::PART;
      const float over = l == 0.f ? 0.f : 1024.f / l;                     // (the values' 2^10; a mean of them is in range, their sum may not be)
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
            d[(x >> 1) + 4 * (x & 1)] = (key_tiles > 0 ? __uint_as_float(v[e + x]) * over : 0.f) * grow;
          }
          if (splits > 1) {
            // (by column, rows side by side: the joining CTA reads them so)
#pragma unroll
            for (int x = 0; x < 8; ++x) __stcg(part_at + (int64_t)(c + e + x) * P::ROWS + m * 128 + r, d[x]);
          } else if (there) {
            mx::Vec8<T> y;
#pragma unroll
            for (int x = 0; x < 4; ++x) y.set_pair(x, make_float2(d[2 * x], d[2 * x + 1]));
            if (a.out.vec) y.store(out + c + e);
            else
#pragma unroll
              for (int x = 0; x < 8; ++x) out[c + e + x] = mx::from_f32<T>(d[x]);
          }
        }
      }
      if (splits > 1) {
        __stcg(part_at + (int64_t)DIM * P::ROWS + m * 128 + r, top - LIFT);
        __stcg(part_at + (int64_t)(DIM + 1) * P::ROWS + m * 128 + r, l);
        __threadfence();
      } else if (there && a.lse) a.lse[(first + token) * a.q.heads + head] = l == 0.f ? -INFINITY : (top - LIFT + log2f(l)) * LN2;
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
          float* parts = reinterpret_cast<float*>(a.workspace + TICKET_BYTES) + (int64_t)(blockIdx.x - part) * P::PART + m * 128 + r;
          float all_top = -INFINITY, l = 0.f;
          for (int i = 0; i < splits; ++i) all_top = fmaxf(all_top, __ldcg(parts + (int64_t)i * P::PART + (int64_t)DIM * P::ROWS));
          for (int i = 0; i < splits; ++i) {                              // (a part's sum takes its maximum's place)
            float* p = parts + (int64_t)i * P::PART;
            const float pl = __ldcg(p + (int64_t)(DIM + 1) * P::ROWS), pm = __ldcg(p + (int64_t)DIM * P::ROWS);
            const float f = pl == 0.f ? 0.f : pl * (pm == -INFINITY ? 1.f : exp2_of(pm - all_top));
            __stcg(p + (int64_t)DIM * P::ROWS, f);
            l += f;
          }
          const float over = l == 0.f ? 0.f : 1.f / l;
          T* out = reinterpret_cast<T*>(a.out.p) + (first + token) * a.out.token + (int64_t)head * a.out.head;
          if (a.lse) a.lse[(first + token) * a.q.heads + head] = l == 0.f ? -INFINITY : (all_top + log2f(l)) * LN2;
#pragma unroll 1
          for (int d = 0; d < DIM; d += 16) {
            float o[16] = {};
#pragma unroll 4
            for (int i = 0; i < splits; ++i) {
              const float* p = parts + (int64_t)i * P::PART;
              const float f = __ldcg(p + (int64_t)DIM * P::ROWS) * over;   // the part's share of the mean
#pragma unroll
              for (int x = 0; x < 16; ++x) o[x] += __ldcg(p + (int64_t)(d + x) * P::ROWS) * f;
            }
#pragma unroll
            for (int w = 0; w < 16; w += 8) {
              mx::Vec8<T> y;
#pragma unroll
              for (int x = 0; x < 4; ++x) y.set_pair(x, make_float2(o[w + 2 * x], o[w + 2 * x + 1]));
              if (a.out.vec) y.store(out + d + w);
              else
#pragma unroll
                for (int x = 0; x < 8; ++x) out[d + w + x] = mx::from_f32<T>(o[w + x]);
            }
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
