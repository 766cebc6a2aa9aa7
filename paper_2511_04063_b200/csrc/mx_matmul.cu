// Product of microscaled operands (dq_mx_matmul, dq_mx_linear):  Y[m][n] = sum_k A[m][k] W[n][k].
//
// The tensor cores take the elements and the block scales as they are held: D[n][m] (weight rows are the MMA's M, tokens
// its N) accumulates  2^(sW + sA - 254) q_W q_A  in fp32 tensor memory; nothing is dequantised.  4-bit activations use
// kind::mxf4 (64 values per MMA step), 8-bit ones kind::mxf8f6f4 (32 per step), for which the copy engine spreads the
// weights' 4-bit codes to one 16-byte slot per 16 values while it brings them into shared memory.
//
// Two kernels.  cluster_kernel, for few tokens, is bound by bringing the weights in, by the MMAs that consume them and by the
// latency at both ends: an MMA takes about 140 cycles whatever its N is (each adds to the sum of the one before it; whether
// that or the pipe sets the time was not measured), 4 KB of 4-bit weights an SM.  16 x 8192 x 8192, weights from HBM: 8.8 us at
// 4 bits, 4.1 of them an SM's 55 MMAs; 9.8 at 8 bits, whose MMAs hold half as much and are twice as many; the weights alone need
// 5.5 us of HBM.  pair_kernel, for many, is bound by the tensor cores: 84 % (4 bits) and 87 % (8 bits) of their cycles active,
// 16384 x 8192 x 8192 in 365 to 373 us (6000 TFLOP/s) and 734 to 742 us (3000) from a cool start, and by the 1000 W power limit
// (1.25 to 1.4 GHz, 408 to 430 and 832 to 865 us) when it lasts.
#include "mx_common.cuh"
#include "tc_host.cuh"

namespace dq {
namespace mx {
namespace {

using namespace tc;
using tc2::cluster_ctarank;
using tc2::cluster_sync_all;

struct Params {
  void* y; int64_t ldy; int y_dtype;
  int y_vec;               // Y's rows start on 16-byte boundaries
  int64_t m, n;            // tokens, weight rows
  int n_blocks, m_blocks;  // tiles
  int stages;              // pipeline steps of the whole reduction
  int splits;              // CTAs of a cluster that share a tile's reduction
  int weights_first;       // the kernel before this one writes no weights: the first may be read before its end
  const void* x; int64_t ldx; int64_t k; int x_vec;   // FUSED: activations; every row in whole 16-byte pieces
  int* d_status;
  uint64_t wait_ns;        // limit of every wait
  int64_t fail_step;       // self-test: the issuer's wait for this pipeline step is one for a barrier that nothing arrives at
};

// A pipeline step: 128 bytes of every row, as the MMAs read them: 256 4-bit values, or 128 8-bit ones.  Every stage of shared
// memory has its own columns of tensor memory for the scales of the step that it holds: whoever fills the stage has waited
// for the MMAs that read both, so the issuer needs no wait of its own before it copies new scales there.
template <bool A8> struct Step {
  static constexpr int KT = A8 ? 1 : 2;                    // scale tiles along k
  static constexpr int MMAS = 4;                           // MMA steps of 32 bytes
};

// One lane of a converged warp, always the same.  The instructions of the copy engine and the tensor cores take uniform
// registers; behind `lane == 0` the compiler has to assume a divergent warp and each of them costs the issuer 60 cycles.
__device__ __forceinline__ bool elect_one() {
  uint32_t e;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(e));
  return e != 0;
}
__device__ __forceinline__ void tma_load_2d(uint32_t dst, const CUtensorMap* map, uint32_t bar, int c0, int c1) {
  asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
               ::"r"(dst), "l"((uint64_t)map), "r"(bar), "r"(c0), "r"(c1) : "memory");
}
// A wait of a whole warp, which goes on or gives up together.
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, const Params& p) {
  return __all_sync(0xffffffffu, mbar_wait(bar, parity, p.d_status, p.wait_ns));
}
// After the issuer has given up waiting, at its step i: steps before i have landed, of the others up to STAGES may be on their
// way (the producer needs a free stage for more, and none comes free).  They have to land before the shared memory may go to
// another CTA or be used for something else.  Steps that the producer never got to run out.
template <int STAGES, typename Full>
__device__ __forceinline__ void await_loads(int64_t i, int64_t steps, Full full, const Params& p) {
  for (int64_t j = i; j < steps && j < i + STAGES; ++j) mbar_wait(full((int)(j % STAGES)), (uint32_t)(j / STAGES) & 1u, p.d_status, p.wait_ns);
}
// Scales: 32 rows of 16 bytes, copied to the same 4 columns of all four 32-lane quarters of tensor memory.
__device__ __forceinline__ uint64_t scale_desc(uint32_t smem_addr) {
  return (uint64_t)((smem_addr & 0x3FFFFu) >> 4) | ((uint64_t)(128 >> 4) << 32) | ((uint64_t)1 << 46);
}
template <int GROUP>
__device__ __forceinline__ void copy_scales(uint32_t taddr, uint64_t desc) {
  if (GROUP == 1) asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
  else asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
}
template <int GROUP, bool A8>
__device__ __forceinline__ void mma_scaled(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sa, uint32_t sb,
                                           uint32_t accumulate) {
#define DQ_MX_MMA(G, KIND)                                                                                     \
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\t"                                               \
               "tcgen05.mma.cta_group::" #G ".kind::" KIND ".block_scale.block32 [%0], %1, %2, %3, [%4], [%5], p;\n\t}" \
               ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(accumulate) : "memory")
  if (GROUP == 1) { if (A8) DQ_MX_MMA(1, "mxf8f6f4"); else DQ_MX_MMA(1, "mxf4"); }
  else { if (A8) DQ_MX_MMA(2, "mxf8f6f4"); else DQ_MX_MMA(2, "mxf4"); }
#undef DQ_MX_MMA
}
// Instruction descriptor of the block-scaled kinds: M = weight rows (E2M1), N = tokens (E2M1 or E4M3), E8M0 scales.
template <bool A8>
__host__ __device__ constexpr uint32_t scaled_idesc(int m, int n) {
  const uint32_t w_format = A8 ? 5u : 1u, a_format = A8 ? 0u : 1u;
  return (w_format << 7) | (a_format << 10) | ((uint32_t)(n >> 3) << 17) | (1u << 23) | ((uint32_t)(m >> 4) << 24);
}
// Which byte of a 32-bit scale column MMA step `s` of a pipeline step reads (both operands alike): mxf4 two blocks of a
// column's four per step, mxf8f6f4 one.
template <bool A8>
__device__ __forceinline__ uint32_t scale_select(int s) {
  const uint32_t id = A8 ? (uint32_t)s : 2u * (uint32_t)(s & 1);
  return (id << 29) | (id << 4);
}

__device__ __forceinline__ void store_value(const Params& p, int64_t at, float v) {
  if (p.y_dtype == DQ_BF16) reinterpret_cast<__nv_bfloat16*>(p.y)[at] = __float2bfloat16_rn(v);
  else if (p.y_dtype == DQ_FP16) reinterpret_cast<__half*>(p.y)[at] = __float2half_rn(v);
  else reinterpret_cast<float*>(p.y)[at] = v;
}
__device__ __forceinline__ void store_four(const Params& p, int64_t at, const float4& v) {
  if (p.y_dtype == DQ_FP32) { *reinterpret_cast<float4*>(reinterpret_cast<float*>(p.y) + at) = v; return; }
  uint2 w;
  if (p.y_dtype == DQ_BF16) {
    const __nv_bfloat162 a = __floats2bfloat162_rn(v.x, v.y), b = __floats2bfloat162_rn(v.z, v.w);
    w = make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
  } else {
    const __half2 a = __floats2half2_rn(v.x, v.y), b = __floats2half2_rn(v.z, v.w);
    w = make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
  }
  *reinterpret_cast<uint2*>(reinterpret_cast<uint16_t*>(p.y) + at) = w;
}

// ------------------------------------------------------------------------------------------------ one tile per cluster
// Few tokens: a tile of 128 weight rows x BN tokens, its reduction shared by the CTAs of a cluster.  What bounds it is
// bringing the weights in; `splits` is chosen so that every SM brings some.  The CTAs leave their fp32 partial sums in
// shared memory and each adds up a part of the columns over the cluster, in the order of the ranks: the result does not
// depend on which CTA ends first.
//
// FUSED (dq_mx_linear): the tokens come as T and every CTA quantises the part of them that it multiplies, which stays in shared
// memory for its whole reduction, while the first weights are on their way.
template <int BN, bool A8, bool FUSED>
struct ClusterSmem {
  static constexpr int KT = Step<A8>::KT;
  static constexpr int W_BYTES = 128 * 128;
  static constexpr int W_LOADED = A8 ? W_BYTES / 2 : W_BYTES;   // (codes that are spread count as they lie in memory)
  static constexpr int X_BYTES = BN * 128;
  static_assert(BN <= 128, "one tile of token scales");
  static constexpr int SF_BYTES = KT * TILE_BYTES;              // of one operand
  static constexpr int RING_X = FUSED ? 0 : X_BYTES + SF_BYTES;
  static constexpr int STAGE_BYTES = (W_BYTES + SF_BYTES + RING_X + 1023) / 1024 * 1024;
  static constexpr int STAGE_LOADED = W_LOADED + SF_BYTES + RING_X;
  static constexpr int PARTIAL_BYTES = BN * 128 * 4;
  static constexpr int STAGES = BN <= 32 ? 5 : 6;
  static_assert(PARTIAL_BYTES <= STAGES * STAGE_BYTES, "the partial sums reuse the stages");
  static constexpr int FIXED = STAGES * STAGE_BYTES + 1024 + 256;
  static constexpr int RESIDENT = FUSED ? X_BYTES + SF_BYTES : 0;   // and for each step of a CTA's reduction
  static constexpr int SCALE_COLS = 4 * KT * 2;
  static constexpr int NEED = BN + STAGES * SCALE_COLS;
  static constexpr int TMEM = NEED <= 64 ? 64 : (NEED <= 128 ? 128 : (NEED <= 256 ? 256 : 512));
  static constexpr int THREADS = FUSED ? 320 : 192;
};
constexpr int MAX_SMEM = 232448;

__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&v)[16]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
               : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]),
                 "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
               : "r"(taddr) : "memory");
}
__device__ __forceinline__ float4 ld_cluster_f4(uint32_t addr, uint32_t rank) {
  uint32_t remote;
  float4 v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"(addr), "r"(rank));
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(remote) : "memory");
  return v;
}

// Arrives at the cluster's barrier once the warp's reads of its peers' shared memory have been performed, which is what `bits` has
// to depend on: every lane's goes into a vote, and the arrival takes the vote's outcome.  The arrival itself is relaxed, it orders
// nothing; a releasing one waits for the fence and the stores to Y, too (16 x 8192 x 8192, 4 and 8 bits: 8.8 and 9.8 us so, 9.1
// and 10.0 to 10.3 released; 256 x 8192 x 1000, 8 bits: 8.7 and 9.3; 32 x 4096 x 4096, 8 bits, weights in L2: 4.5 and 4.9 to 5.3).
__device__ __forceinline__ void cluster_arrive_after(uint32_t bits) {
  const int unusual = __any_sync(0xffffffffu, bits == 0x7fdb97c5u);
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.s32 p, %0, 0;\n\t@p nanosleep.u32 1;\n\tbarrier.cluster.arrive.relaxed.aligned;\n\t}"
               ::"r"(unusual) : "memory");
}
// Rows [0, m) x values [c0, c0 + 8 groups) of X as a CTA's resident operand: codes of step i at codes + i X_BYTES in the K-major
// 128-byte-swizzled order of the MMA's operands, its scale tiles at scales + i SF_BYTES.  A warp takes 256 values of a row at
// a time, the `warps` warps in turn.
template <int BN, bool A8, typename T>
__device__ __forceinline__ void quantize_resident(const Params& p, uint8_t* codes, uint8_t* scales, int c0, int groups, int warp, int warps,
                                                  int lane) {
  using L = ClusterSmem<BN, A8, true>;
  constexpr int FMT = A8 ? DQ_MXFP8 : DQ_MXFP4, BYTES = Codes8<FMT>::BYTES, PER_STEP = 128 / BYTES;
  constexpr int AT_ONCE = 4;
  const T* X = reinterpret_cast<const T*>(p.x);
  const int pieces = (groups + 31) / 32, m = (int)p.m;
  int row = warp / pieces, piece = warp % pieces;            // of the next load; then of the next store
  auto step_on = [&](int& r, int& c) {
    for (c += warps; c >= pieces; c -= pieces) ++r;
  };
  while (row < m) {
    Vec8<T> v[AT_ONCE];
    int r = row, c = piece;
#pragma unroll
    for (int u = 0; u < AT_ONCE; ++u) {
      const int at = c0 + (c * 32 + lane) * 8;
      v[u].clear();
      if (r < m && c * 32 + lane < groups) {
        if (!p.x_vec) load_each(v[u], X + r * p.ldx, at, (int)p.k);
        else if (at < p.k) v[u].load(X + r * p.ldx + at);
      }
      step_on(r, c);
    }
#pragma unroll
    for (int u = 0; u < AT_ONCE; ++u) {
      if (row >= m) break;                                   // (whole warps)
      const uint32_t s = scale_code<FMT>(block_exponent(v[u].exponent()));
      Codes8<FMT> q;
      q.encode(v[u], s);
      const int g = piece * 32 + lane;
      if (g < groups) {
        const int step = g / PER_STEP, byte = g % PER_STEP * BYTES, block = g / 4;
        q.store(codes + step * L::X_BYTES + row * 128 + ((((byte >> 4) ^ row) & 7) << 4) + (byte & 15));
        if ((lane & 3) == 0) scales[block / 4 * TILE_BYTES + (row & 31) * 16 + (row >> 5) * 4 + (block & 3)] = (uint8_t)s;
      }
      step_on(row, piece);
    }
  }
}

// (Two CTAs an SM where shared memory has room for them: the registers have to do, too.)
template <int BN, bool A8, bool FUSED, typename T>
__global__ void __launch_bounds__(ClusterSmem<BN, A8, FUSED>::THREADS, 2) 
cluster_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_ws,
               const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_xs, const Params p) {
  using L = ClusterSmem<BN, A8, FUSED>;
  constexpr int STAGES = L::STAGES, KT = L::KT;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t bars = base + STAGES * L::STAGE_BYTES;
  auto full = [&](int s) { return bars + 8u * s; };
  auto empty = [&](int s) { return bars + 8u * (STAGES + s); };
  const uint32_t done = bars + 8u * (2 * STAGES), held = done + 8u, never = held + 8u, tmem_slot = never + 8u;
  const uint32_t res = (bars + 256u + 1023u) & ~1023u;       // FUSED: the resident tokens, then their scales
  uint8_t* smem = smem_raw + (base - smem_u32(smem_raw));

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = p.splits > 1 ? (int)cluster_ctarank() : 0;
  const int tile = blockIdx.x / p.splits;
  const int nb = tile % p.n_blocks, mb = tile / p.n_blocks;
  const int k0 = (int)((int64_t)rank * p.stages / p.splits), kn = (int)((int64_t)(rank + 1) * p.stages / p.splits) - k0;
  const uint32_t res_sf = res + (uint32_t)kn * L::X_BYTES;

  if (threadIdx.x == 0) {
    for (int s = 0; s < STAGES; ++s) { mbar_init(full(s), 1); mbar_init(empty(s), 1); }
    mbar_init(done, 1);
    mbar_init(held, L::THREADS / 32 - 2);
    mbar_init(never, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    prefetch_tensormap(&map_w); prefetch_tensormap(&map_ws);
    if (!FUSED) { prefetch_tensormap(&map_x); prefetch_tensormap(&map_xs); }
  }
  if (warp == 1) tmem_alloc(tmem_slot, L::TMEM);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *reinterpret_cast<const uint32_t*>(smem + (tmem_slot - base));

  if (warp == 0) {
    if (elect_one()) {
      auto weights = [&](int i) {
        const int s = i % STAGES;
        const uint32_t at = base + s * L::STAGE_BYTES;
        mbar_expect_tx(full(s), L::STAGE_LOADED);
        tma_load_2d(at, &map_w, full(s), (k0 + i) * 128, nb * 128);
        tma_load_3d(at + L::W_BYTES, &map_ws, full(s), 0, (k0 + i) * KT, nb);
      };
      auto tokens = [&](int i) {
        const int s = i % STAGES;
        const uint32_t at = base + s * L::STAGE_BYTES + L::W_BYTES + L::SF_BYTES;
        if (FUSED) return;
        tma_load_2d(at, &map_x, full(s), (k0 + i) * 128, mb * BN);
        tma_load_3d(at + L::X_BYTES, &map_xs, full(s), 0, (k0 + i) * KT, mb * BN / 128);
      };
      const int ahead = kn < STAGES ? kn : STAGES;
      if (!p.weights_first) wait_for_previous();
      for (int i = 0; i < ahead; ++i) weights(i);
      if (p.weights_first) wait_for_previous();
      allow_next();
      for (int i = 0; i < ahead; ++i) tokens(i);
      for (int i = ahead; i < kn; ++i) {
        if (!mbar_wait(empty(i % STAGES), (uint32_t)(i / STAGES - 1) & 1u, p.d_status, p.wait_ns)) break;   // (the issuer awaits the loads)
        weights(i);
        tokens(i);
      }
    }
    __syncwarp();
  } else if (warp == 1) {
    constexpr uint32_t IDESC = scaled_idesc<A8>(128, BN);
    wait_for_previous();                                     // (the limits of the waits below do not count that kernel's time)
    // One thread waits and issues: what it decides needs no agreement, and a step is shorter than where the warp waits together
    // (64 x 8192 x 11008, 8 bits: 17.8 us against 22.2; 16 x 8192 x 8192: 10.0 against 10.6, both with a
    // releasing arrival at the end).
    if (elect_one()) {
      auto wait = [&](uint32_t bar, uint32_t parity) { return mbar_wait(bar, parity, p.d_status, p.wait_ns); };
      const int stop = p.fail_step < kn ? (int)p.fail_step : kn;
      bool ok = !FUSED || wait(held, 0);
      int i = 0;
      for (; i < stop && ok; ++i) {
        const int st = i % STAGES;
        ok = wait(full(st), (uint32_t)(i / STAGES) & 1u);
        if (!ok) break;
        tc_fence_after();
        const uint32_t sw = tmem + BN + (uint32_t)st * L::SCALE_COLS, sx = sw + 4 * KT;
        const uint32_t at = base + st * L::STAGE_BYTES, ws = at + L::W_BYTES;
        const uint32_t x = FUSED ? res + i * L::X_BYTES : ws + L::SF_BYTES, xs = FUSED ? res_sf + i * L::SF_BYTES : x + L::X_BYTES;
#pragma unroll
        for (int t = 0; t < KT; ++t) {
          copy_scales<1>(sw + 4 * t, scale_desc(ws + t * TILE_BYTES));
          copy_scales<1>(sx + 4 * t, scale_desc(xs + t * TILE_BYTES));
        }
        const uint64_t a = make_kmajor_sw128_desc(at), b = make_kmajor_sw128_desc(x);
#pragma unroll
        for (int m = 0; m < Step<A8>::MMAS; ++m) {
          const int t = A8 ? 0 : m >> 1;
          mma_scaled<1, A8>(tmem, a + 2 * m, b + 2 * m, IDESC | scale_select<A8>(m), sw + 4 * t, sx + 4 * t, (i | m) ? 1u : 0u);
        }
        umma_commit(empty(st));
      }
      if (ok && stop < kn) ok = wait(never, 0);
      if (!ok) await_loads<STAGES>(i, kn, full, p);
      umma_commit(done);
      if (!ok) wait(done, 0);                                // (the MMAs that were issued have ended)
    }
    __syncwarp();
  } else {
    wait_for_previous();
    if constexpr (FUSED) {
      const int values = A8 ? 128 : 256;                     // of a step
      quantize_resident<BN, A8, T>(p, smem + (res - base), smem + (res_sf - base), k0 * values, kn * (values / 8),
                                   warp - 2, L::THREADS / 32 - 2, lane);
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0) mbar_arrive(held);
    }
    if (warp < 6) {
      const int q = warp & 3;
      // every MMA has completed, so the stages are free: partial sums as [token][128 weight rows]
      const bool complete = warp_wait(done, 0, p);
      tc_fence_after();
      float* part = reinterpret_cast<float*>(smem);
      for (int c = 0; c < BN && complete; c += 16) {
        uint32_t v[16];
        tmem_ld16(tmem + ((uint32_t)(q * 32) << 16) + (uint32_t)c, v);
        tmem_ld_wait();
#pragma unroll
        for (int e = 0; e < 16; ++e) part[(c + e) * 128 + q * 32 + lane] = __uint_as_float(v[e]);
      }
      tc_fence_before();
    }
  }
  if (p.splits > 1) cluster_sync_all(); else __syncthreads();

  // Y[token][4 weight rows] by all threads; the columns are dealt over the cluster
  const int64_t left = p.m - (int64_t)mb * BN;
  const int cols = left < BN ? (int)left : BN;
  const int c0 = rank * cols / p.splits, c1 = (rank + 1) * cols / p.splits;
  const int64_t n0 = (int64_t)nb * 128;
  const int esize = p.y_dtype == DQ_FP32 ? 4 : 2;
  const bool vec = (((uintptr_t)p.y | (uintptr_t)(p.ldy * esize)) & (uintptr_t)(4 * esize - 1)) == 0;
  auto store = [&](int i, const float4& s) {                 // piece i of [token][32 pieces of four weight rows]
    const int c = i >> 5;
    const int64_t n = n0 + (i & 31) * 4, at = ((int64_t)mb * BN + c) * p.ldy + n;
    if (vec && n + 4 <= p.n) { store_four(p, at, s); return; }
    const float e[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) if (n + j < p.n) store_value(p, at + j, e[j]);
  };
  if (p.splits == 1) {
    for (int i = threadIdx.x; i < cols * 32; i += blockDim.x) store(i, reinterpret_cast<const float4*>(smem)[i]);
    tc_fence_before();
    __syncthreads();
  } else {
    // All loads of two pieces at once: one at a time they cost the cluster's latency each (128 x 4096 x 4096: 9.7 us
    // then, 8.4 so).  Pieces past Y's edge are neither loaded nor stored.  What was loaded is gathered in `bits`: the peers may
    // leave, and their shared memory with them, once the barrier at the end says that this CTA has read it.
    constexpr int AT_ONCE = 2, MOST = 8;
    uint32_t bits = 0;
    for (int i0 = (int)threadIdx.x + c0 * 32; i0 < c1 * 32; i0 += AT_ONCE * blockDim.x) {
      float4 v[AT_ONCE][MOST];
      auto wanted = [&](int i) { return i < c1 * 32 && n0 + (i & 31) * 4 < p.n; };
#pragma unroll
      for (int u = 0; u < AT_ONCE; ++u) {
        const int i = i0 + u * (int)blockDim.x;
        const uint32_t at = base + (uint32_t)i * 16u;        // [token][32 pieces]
#pragma unroll
        for (int r = 0; r < MOST; ++r)
          if (r < p.splits && wanted(i)) v[u][r] = ld_cluster_f4(at, (uint32_t)r);
      }
#pragma unroll
      for (int u = 0; u < AT_ONCE; ++u) {
        const int i = i0 + u * (int)blockDim.x;
        if (!wanted(i)) continue;
        float4 s = v[u][0];
#pragma unroll
        for (int r = 1; r < MOST; ++r)
          if (r < p.splits) { s.x += v[u][r].x; s.y += v[u][r].y; s.z += v[u][r].z; s.w += v[u][r].w; }
        bits ^= __float_as_uint(s.x) ^ __float_as_uint(s.y) ^ __float_as_uint(s.z) ^ __float_as_uint(s.w);
        store(i, s);
      }
    }
    tc_fence_before();
    __syncwarp();
    cluster_arrive_after(bits);
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  }
  if (warp == 1) { tc_fence_after(); tmem_dealloc(tmem, L::TMEM); }
}

// ------------------------------------------------------------------------------------------------ persistent pairs
// Many tokens: CTA pairs walk over tiles of 256 weight rows x 256 tokens with cta_group::2, each CTA staging half of both
// operands (64 bytes of shared memory per SM and cycle at the 4-bit rate, where one CTA alone would need 96 for a tile of
// 128 x 256).  Two accumulators of 256 columns do not fit beside five stages' 24 (8 bits: 12) columns of scales: the second
// accumulator starts 136 (196) columns after the first.  The epilogue of a tile takes the columns that both cover into
// registers first, and the next tile's MMAs start once those are free.
template <bool A8>
struct PairSmem {
  static constexpr int KT = Step<A8>::KT;
  static constexpr int W_BYTES = 128 * 128;
  static constexpr int W_LOADED = A8 ? W_BYTES / 2 : W_BYTES;
  static constexpr int X_BYTES = 128 * 128;
  static constexpr int SF_BYTES = KT * TILE_BYTES * 3;     // its 128 weight rows', all 256 tokens'
  static constexpr int STAGE_BYTES = (W_BYTES + X_BYTES + SF_BYTES + 1023) / 1024 * 1024;
  static constexpr int STAGES = 5;
  static constexpr int SCALE_COLS = 12 * KT;
  static constexpr int SCALES = 512 - STAGES * SCALE_COLS;        // first column of the scales
  static constexpr int ACC_STRIDE = SCALES - 256;                 // column where the second accumulator starts
  static constexpr int SHARED = (256 - ACC_STRIDE + 31) / 32 * 32;   // columns both accumulators cover, to a multiple of 32
  static constexpr int EPI_BYTES = 4 * 8192;                      // two buffers for each group of epilogue warps
  static constexpr int TOTAL = STAGES * STAGE_BYTES + EPI_BYTES + 1024 + 256;
};
constexpr int PAIR_GROUP = 8;                              // weight tiles that consecutive tiles go over before the next tokens

__device__ __forceinline__ void tma_load_2d_pair(uint32_t dst, const CUtensorMap* map, uint32_t bar, int c0, int c1) {
  asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
               ::"r"(dst), "l"((uint64_t)map), "r"(bar & tc2::PEER_MASK), "r"(c0), "r"(c1) : "memory");
}

// One arrival on this CTA's barrier once every MMA of the pair issued so far has completed.
__device__ __forceinline__ void commit_leader(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}

// The pieces of 32 columns (tokens from m0 on) x 128 lanes (weight rows) that a group of four epilogue warps takes to Y.  Where
// Y's rows are aligned they leave through shared memory as rows of 128 values, written by the copy engine, which also clips
// them at Y's edges: whole 256-byte rows, where the warps' own stores would write 64 bytes of a row at a time (8192 x 1024 x 8192: 37.8 us against 45.3,
// 16384 x 256 x 8192: 60.0 against 70.4).
// Each group has two buffers of 8 KB, a piece of a 4-byte type goes in two parts.
constexpr int PIECE_BYTES = 8192;
// Whether all 128 threads at the barrier say yes.
__device__ __forceinline__ bool agree(int barrier, bool yes) {
  uint32_t all;
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbar.red.and.pred q, %2, 128, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
               : "=r"(all) : "r"((uint32_t)yes), "r"(barrier) : "memory");
  return all != 0;
}
template <typename T>
struct Output {
  static constexpr int PASS = PIECE_BYTES / 128 / sizeof(T);   // tokens of a buffer
  const CUtensorMap* map;
  uint8_t* buffers;
  int group, q, lane, turn = 0;
  __device__ __forceinline__ void piece(const Params& p, const uint32_t (&v)[32], int64_t n0, int64_t m0) {
    if (p.y_vec) {
      const bool one = q == 2 && lane == 0;                     // (the group's first warp)
#pragma unroll
      for (int e0 = 0; e0 < 32; e0 += PASS, turn ^= 1) {
        T* s = reinterpret_cast<T*>(buffers + turn * PIECE_BYTES);
        if (one) asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");   // the buffer's last piece has been read
        asm volatile("bar.sync %0, 128;" ::"r"(1 + group) : "memory");
#pragma unroll
        for (int e = 0; e < PASS; ++e) s[e * 128 + q * 32 + lane] = from_f32<T>(__uint_as_float(v[e0 + e]));
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        asm volatile("bar.sync %0, 128;" ::"r"(1 + group) : "memory");
        if (one) {
          asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%2, %3}], [%1];"
                       ::"l"((uint64_t)map), "r"(smem_u32(s)), "r"((int)n0), "r"((int)(m0 + e0)) : "memory");
          asm volatile("cp.async.bulk.commit_group;" ::: "memory");
        }
      }
      return;
    }
    const int64_t n = n0 + q * 32 + lane, left = p.m - m0;
    if (n < p.n) {
      T* to = reinterpret_cast<T*>(p.y) + m0 * p.ldy + n;
#pragma unroll
      for (int e = 0; e < 32; ++e, to += p.ldy)
        if (e < left) *to = from_f32<T>(__uint_as_float(v[e]));
    }
  }
  __device__ __forceinline__ void finish(const Params& p) const {   // before the shared memory goes away
    if (p.y_vec && q == 2 && lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
  }
};

constexpr int PAIR_THREADS = 320;                          // producer, issuer, eight epilogue warps
template <bool A8, typename T>
__global__ void __launch_bounds__(PAIR_THREADS, 1)
pair_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_ws,
            const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_xs,
            const __grid_constant__ CUtensorMap map_y, const Params p) {
  using L = PairSmem<A8>;
  constexpr int STAGES = L::STAGES, KT = L::KT;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t epi = base + STAGES * L::STAGE_BYTES, bars = epi + L::EPI_BYTES;
  auto full = [&](int s) { return bars + 8u * s; };
  auto empty = [&](int s) { return bars + 8u * (STAGES + s); };
  auto ready = [&](int a) { return bars + 8u * (2 * STAGES + a); };          // accumulator a is complete
  const uint32_t drained = bars + 8u * (2 * STAGES + 2);                     // the columns it shares are read
  const uint32_t ended = drained + 8u, never = ended + 8u, tmem_slot = never + 8u;   // after a wait that ran out: no MMA is left
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();
  const bool leader = rank == 0;

  if (threadIdx.x == 0) {
    for (int s = 0; s < STAGES; ++s) { mbar_init(full(s), 1); mbar_init(empty(s), 1); }
    mbar_init(ready(0), 1); mbar_init(ready(1), 1);
    mbar_init(drained, 16);
    mbar_init(ended, 1); mbar_init(never, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    prefetch_tensormap(&map_w); prefetch_tensormap(&map_ws); prefetch_tensormap(&map_x); prefetch_tensormap(&map_xs);
  }
  if (warp == 1) tc2::tmem_alloc_pair(tmem_slot, 512);
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();
  tc_fence_after();
  const uint32_t tmem = *reinterpret_cast<const uint32_t*>(smem_raw + (tmem_slot - smem_u32(smem_raw)));

  const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
  const int tiles = p.n_blocks * p.m_blocks;
  auto tile_of = [&](int u, int& nb, int& mb) {
    const int group = u / (PAIR_GROUP * p.m_blocks), r = u % (PAIR_GROUP * p.m_blocks);
    const int left = p.n_blocks - group * PAIR_GROUP, wide = left < PAIR_GROUP ? left : PAIR_GROUP;
    nb = group * PAIR_GROUP + r % wide;
    mb = r / wide;
  };

  if (warp == 0) {
    if (elect_one()) {
      auto weights = [&](int s, int k, int nb) {
        const uint32_t at = base + s * L::STAGE_BYTES;
        if (leader) mbar_expect_tx(full(s), 2 * (L::W_LOADED + L::X_BYTES + L::SF_BYTES));
        tma_load_2d_pair(at, &map_w, full(s), k * 128, nb * 256 + (int)rank * 128);
        tc2::tma_load_3d_pair(at + L::W_BYTES + L::X_BYTES, &map_ws, full(s), 0, k * KT, nb * 2 + (int)rank);
      };
      auto tokens = [&](int s, int k, int mb) {
        const uint32_t at = base + s * L::STAGE_BYTES + L::W_BYTES;
        tma_load_2d_pair(at, &map_x, full(s), k * 128, mb * 256 + (int)rank * 128);
        tc2::tma_load_3d_pair(at + L::X_BYTES + KT * TILE_BYTES, &map_xs, full(s), 0, k * KT, mb * 2);
      };
      const int ahead = p.stages < STAGES ? p.stages : STAGES;   // steps of the first tile that need no free stage
      int nb, mb;
      tile_of(pair, nb, mb);
      if (!p.weights_first) wait_for_previous();
      for (int k = 0; k < ahead; ++k) weights(k, k, nb);
      if (p.weights_first) wait_for_previous();
      allow_next();
      for (int k = 0; k < ahead; ++k) tokens(k, k, mb);
      int s = ahead % STAGES, round = ahead / STAGES;            // stage, and how often it was used
      bool ok = true;
      for (int u = pair, k = ahead; u < tiles && ok; u += pairs, k = 0) {
        tile_of(u, nb, mb);
        for (; k < p.stages; ++k) {
          if (round > 0 && !mbar_wait(empty(s), (uint32_t)(round - 1) & 1u, p.d_status, p.wait_ns)) { ok = false; break; }
          weights(s, k, nb);
          tokens(s, k, mb);
          if (++s == STAGES) { s = 0; ++round; }
        }
      }
    }
    __syncwarp();
  } else if (warp == 1) {
    if (leader) {
      constexpr uint32_t IDESC = scaled_idesc<A8>(256, 256);
      wait_for_previous();                                   // (the limits of the waits below do not count that kernel's time)
      const int mine = pair < tiles ? (tiles - pair + pairs - 1) / pairs : 0;
      const int64_t steps = (int64_t)mine * p.stages;
      int stage = 0;
      uint32_t phase = 0;
      int k = 0, t = 0;                                      // step of the tile, tile
      // (the warp waits together: one thread that waits and issues, as in the other kernel, takes 11 cycles more a step here)
      const int64_t stop = p.fail_step < steps ? p.fail_step : steps;
      int64_t i = 0;
      for (; i < stop; ++i) {
        if (!warp_wait(full(stage), phase, p)) break;
        if (k == 0 && t >= 1 && !warp_wait(drained, (uint32_t)(t - 1) & 1u, p)) break;
        tc_fence_after();
        if (elect_one()) {
          const uint32_t acc = tmem + (uint32_t)((t & 1) * L::ACC_STRIDE);
          const uint32_t sw = tmem + L::SCALES + (uint32_t)stage * L::SCALE_COLS, sx = sw + 4 * KT;
          const uint32_t at = base + (uint32_t)stage * L::STAGE_BYTES, sf = at + L::W_BYTES + L::X_BYTES;
#pragma unroll
          for (int j = 0; j < KT; ++j) {
            copy_scales<2>(sw + 4 * j, scale_desc(sf + j * TILE_BYTES));
            copy_scales<2>(sx + 8 * j, scale_desc(sf + (KT + j) * TILE_BYTES));
            copy_scales<2>(sx + 8 * j + 4, scale_desc(sf + (2 * KT + j) * TILE_BYTES));
          }
          const uint64_t a = make_kmajor_sw128_desc(at), b = make_kmajor_sw128_desc(at + L::W_BYTES);
#pragma unroll
          for (int m = 0; m < Step<A8>::MMAS; ++m) {
            const int j = A8 ? 0 : m >> 1;
            mma_scaled<2, A8>(acc, a + 2 * m, b + 2 * m, IDESC | scale_select<A8>(m), sw + 4 * j, sx + 8 * j, (k | m) ? 1u : 0u);
          }
          tc2::umma_commit_pair(empty(stage));
          if (k + 1 == p.stages) tc2::umma_commit_pair(ready(t & 1));
        }
        __syncwarp();
        if (++stage == STAGES) { stage = 0; phase ^= 1u; }
        if (++k == p.stages) { k = 0; ++t; }
      }
      if (i == stop && stop < steps) warp_wait(never, 0, p);
      if (i < steps) {                                       // gave up: both CTAs' loads arrive at the leader's barriers
        await_loads<STAGES>(i, steps, full, p);
        __syncwarp();
        if (elect_one()) commit_leader(ended);
        __syncwarp();
        warp_wait(ended, 0, p);
      }
    }
    __syncwarp();
  } else {
    // Two warps for each quarter of the tensor-memory lanes; they take turns at the tile's eight pieces of 32 columns,
    // those that both accumulators cover first (accumulator 0 ends with them, accumulator 1 begins with them).
    constexpr int SHARED = L::SHARED / 32;
    wait_for_previous();
    const int q = warp & 3, half = (warp - 2) >> 2;
    Output<T> out{&map_y, smem_raw + (epi - smem_u32(smem_raw)) + half * 2 * PIECE_BYTES, half, q, lane};
    int t = 0;
    for (int u = pair; u < tiles; u += pairs, ++t) {
      int nb, mb;
      tile_of(u, nb, mb);
      const int a = t & 1;
      // (the four warps of a group go on or leave together: they meet at barriers below)
      if (!agree(1 + half, mbar_wait(ready(a), (uint32_t)(t >> 1) & 1u, p.d_status, p.wait_ns))) break;
      tc_fence_after();
      const int64_t n0 = (int64_t)nb * 256 + rank * 128, m0 = (int64_t)mb * 256;
      const uint32_t acc = tmem + ((uint32_t)(q * 32) << 16) + (uint32_t)(a * L::ACC_STRIDE);
      const int first = a == 0 ? 8 - SHARED : 0;
      auto column = [&](int i) { return ((first + i) & 7) * 32; };
      uint32_t v[2][32];
      tmem_ld32(acc + (uint32_t)column(half), v[0]);
      tmem_ld32(acc + (uint32_t)column(half + 2), v[1]);
      tmem_ld_wait();
      static_assert(SHARED <= 4, "the first two pieces of both warps cover the shared columns");
      tc_fence_before();
      __syncwarp();
      if (lane == 0) tc2::mbar_arrive_leader(drained);
      out.piece(p, v[0], n0, m0 + column(half));
      tmem_ld32(acc + (uint32_t)column(half + 4), v[0]);     // (on its way during the next stores)
      out.piece(p, v[1], n0, m0 + column(half + 2));
      tmem_ld_wait();
      tmem_ld32(acc + (uint32_t)column(half + 6), v[1]);
      out.piece(p, v[0], n0, m0 + column(half + 4));
      tmem_ld_wait();
      out.piece(p, v[1], n0, m0 + column(half + 6));
    }
    out.finish(p);
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();
  if (warp == 1) { tc_fence_after(); tc2::tmem_dealloc_pair(tmem, 512); }
}

// ------------------------------------------------------------------------------------------------ host
// Codes as rows of bytes; `spread`: 4-bit codes that arrive as 16 values per 16-byte slot (coordinates in values).
dq_status codes_map(CUtensorMap* m, const uint8_t* codes, int fmt, int64_t rows, int64_t k, int box_rows, bool spread) {
  tch::EncodeFn fn = tch::get_encode_fn();
  if (!fn) return DQ_ERR_CUDA;
  const cuuint64_t bytes = (cuuint64_t)row_bytes(fmt, k);
  cuuint64_t dims[2] = {spread ? (cuuint64_t)(k_tiles(k) * KTILE) : bytes, (cuuint64_t)rows};
  cuuint64_t strides[1] = {bytes};
  cuuint32_t box[2] = {128, (cuuint32_t)box_rows};
  cuuint32_t ones[2] = {1, 1};
  const CUresult r = fn(m, spread ? CU_TENSOR_MAP_DATA_TYPE_16U4_ALIGN16B : CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, (void*)codes, dims,
                        strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                        CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? DQ_OK : DQ_ERR_CUDA;
}
// Scale tiles [row tile][k tile][512 bytes]; a box past the last k tile reads zeros, which scale zeros.
dq_status scales_map(CUtensorMap* m, const uint8_t* scales, int64_t rows, int64_t k, int kt, int row_tiles) {
  tch::EncodeFn fn = tch::get_encode_fn();
  if (!fn) return DQ_ERR_CUDA;
  cuuint64_t dims[3] = {TILE_BYTES / 4, (cuuint64_t)k_tiles(k), (cuuint64_t)((rows + ROW_TILE - 1) / ROW_TILE)};
  cuuint64_t strides[2] = {TILE_BYTES, (cuuint64_t)(k_tiles(k) * TILE_BYTES)};
  cuuint32_t box[3] = {TILE_BYTES / 4, (cuuint32_t)kt, (cuuint32_t)row_tiles};
  cuuint32_t ones[3] = {1, 1, 1};
  const CUresult r = fn(m, CU_TENSOR_MAP_DATA_TYPE_UINT32, 3, (void*)scales, dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                        CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? DQ_OK : DQ_ERR_CUDA;
}

// Y as boxes of 128 weight rows x `tokens`; only where its rows are 16-byte aligned.
dq_status output_map(CUtensorMap* m, void* y, int dtype, int64_t rows, int64_t n, int64_t ldy, int tokens) {
  tch::EncodeFn fn = tch::get_encode_fn();
  if (!fn) return DQ_ERR_CUDA;
  const CUtensorMapDataType type = dtype == DQ_FP32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
                                   : dtype == DQ_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
  cuuint64_t dims[2] = {(cuuint64_t)n, (cuuint64_t)rows};
  cuuint64_t strides[1] = {(cuuint64_t)ldy * (dtype == DQ_FP32 ? 4 : 2)};
  cuuint32_t box[2] = {128, (cuuint32_t)tokens};
  cuuint32_t ones[2] = {1, 1};
  const CUresult r = fn(m, type, 2, y, dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE,
                        CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? DQ_OK : DQ_ERR_CUDA;
}

struct Operands {
  int a_fmt;
  const uint8_t *a_codes, *a_scales, *w_codes, *w_scales;
  int64_t m, n, k;
  void* y; int y_dtype; int64_t ldy;
  bool weights_first = false;
  const void* x = nullptr; int64_t ldx = 0; int x_vec = 0;   // unquantised activations
  int64_t fail_step = INT64_MAX; uint64_t wait_ns = WAIT_LIMIT_NS;  // self-test
};

Params params(const Device& dev, const Operands& o, int rows, int tokens, int kt) {
  Params p{};
  p.y = o.y; p.ldy = o.ldy; p.y_dtype = o.y_dtype; p.m = o.m; p.n = o.n; p.k = o.k;
  p.n_blocks = (int)((o.n + rows - 1) / rows); p.m_blocks = (int)((o.m + tokens - 1) / tokens);
  p.stages = (int)((k_tiles(o.k) + kt - 1) / kt);
  p.splits = 1; p.weights_first = o.weights_first; p.d_status = dev.d_status;
  p.x = o.x; p.ldx = o.ldx; p.x_vec = o.x_vec;
  p.wait_ns = o.wait_ns; p.fail_step = o.fail_step;
  return p;
}

template <int BN, bool A8, bool FUSED>
int cluster_smem(int stages, int splits) {
  using L = ClusterSmem<BN, A8, FUSED>;
  return L::FIXED + (FUSED ? 1024 + (stages + splits - 1) / splits * L::RESIDENT : 0);
}

// Into how many CTAs the reduction of each of `tiles` tiles is split, in powers of two (the kernel takes any number up to 8;
// others were not measured): as many as run at once, until every SM has one; where shared memory has room for two on an SM, up
// to 32 tokens, until it has two, whose latencies hide each other's, as long as each keeps eight steps.  16 x 8192 x 8192 at
// 4 bits: 8.8 us with two CTAs of 8 steps an SM, 9.9 with one of 16.  Any limit from 4 to 8 steps does: 1 x 1024 x 8192 at
// 4 bits takes 2.9 us with either and 3.5 with none, 16 x 2048 x 8192 at 8 bits 5.4 with 8 and 5.2 with 4, the others the
// same.  Clusters have to find their SMs together: of 8 CTAs with an SM each, 15 run at once, not 18.  FUSED: at least as
// many as make the tokens fit.
template <int BN, bool A8, bool FUSED, typename T>
dq_status choose_splits(const Device& dev, int64_t tiles, int stages, int& splits) {
  using L = ClusterSmem<BN, A8, FUSED>;
  struct Clusters { int most[9]; };                          // that run at once with an SM a CTA, by their size
  static PerDevice<Clusters> known;
  constexpr int ALONE = L::FIXED > MAX_SMEM / 2 + 1024 ? L::FIXED : MAX_SMEM / 2 + 1024;   // shared memory that leaves no room for two
  auto kern = cluster_kernel<BN, A8, FUSED, T>;
  Clusters clusters;
  DQ_CHECK((dq_status)known.get(dev.index, clusters, [kern](Clusters& c) -> int {
    DQ_CHECK_CUDA(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, FUSED ? MAX_SMEM : ALONE));
    for (int s = 2; s <= 8; s *= 2) {
      LaunchConfig config(nullptr, s, L::THREADS, ALONE, s);
      DQ_CHECK_CUDA(cudaOccupancyMaxActiveClusters(&c.most[s], kern, &config.cfg));
    }
    return DQ_OK;
  }));
  splits = 1;
  for (int s = 2; s <= 8 && s <= stages; s *= 2) {
    const int smem = cluster_smem<BN, A8, FUSED>(stages, s);
    const bool two = smem <= MAX_SMEM / 2 - 1024 && stages >= s * 8;
    if (cluster_smem<BN, A8, FUSED>(stages, splits) > MAX_SMEM || tiles <= (two ? 2 : 1) * clusters.most[s]) splits = s;
  }
  return DQ_OK;
}

template <int BN, bool A8, bool FUSED, typename T>
dq_status launch_cluster(cudaStream_t stream, const Device& dev, const Operands& o) {
  using L = ClusterSmem<BN, A8, FUSED>;
  CUtensorMap w, ws, x = {}, xs = {};
  Params p = params(dev, o, 128, BN, L::KT);
  const int64_t tiles = (int64_t)p.n_blocks * p.m_blocks;
  DQ_CHECK((choose_splits<BN, A8, FUSED, T>(dev, tiles, p.stages, p.splits)));
  const int smem = cluster_smem<BN, A8, FUSED>(p.stages, p.splits);
  if (tiles * p.splits > 0x7fffffff || smem > MAX_SMEM) return DQ_ERR_UNSUPPORTED;
  // FUSED: more than 8192 values a CTA cost more than the launch that they save (linear says how much)
  if (FUSED && o.m > 1 && o.m * ((p.stages + p.splits - 1) / p.splits) * (L::KT * KTILE) > 8192) return DQ_ERR_UNSUPPORTED;
  DQ_CHECK(codes_map(&w, o.w_codes, DQ_MXFP4, o.n, o.k, 128, A8));
  DQ_CHECK(scales_map(&ws, o.w_scales, o.n, o.k, L::KT, 1));
  if (!FUSED) {
    DQ_CHECK(codes_map(&x, o.a_codes, o.a_fmt, o.m, o.k, BN, false));
    DQ_CHECK(scales_map(&xs, o.a_scales, o.m, o.k, L::KT, 1));
  }
  return launch(LaunchConfig(stream, tiles * p.splits, L::THREADS, smem, p.splits), cluster_kernel<BN, A8, FUSED, T>, w, ws, x, xs, p);
}

template <bool A8, typename T>
dq_status launch_pair(cudaStream_t stream, const Device& dev, const Operands& o) {
  using L = PairSmem<A8>;
  CUtensorMap w, ws, x, xs, y = {};
  DQ_CHECK(codes_map(&w, o.w_codes, DQ_MXFP4, o.n, o.k, 128, A8));
  DQ_CHECK(codes_map(&x, o.a_codes, o.a_fmt, o.m, o.k, 128, false));
  DQ_CHECK(scales_map(&ws, o.w_scales, o.n, o.k, L::KT, 1));
  DQ_CHECK(scales_map(&xs, o.a_scales, o.m, o.k, L::KT, 2));
  Params p = params(dev, o, 256, 256, L::KT);
  p.y_vec = (((uintptr_t)o.y | (uintptr_t)(o.ldy * (int64_t)sizeof(T))) & 15) == 0;
  if (p.y_vec) DQ_CHECK(output_map(&y, o.y, o.y_dtype, o.m, o.n, o.ldy, Output<T>::PASS));
  const int64_t tiles = (int64_t)p.n_blocks * p.m_blocks;
  if (tiles * PAIR_GROUP > 0x7fffffff) return DQ_ERR_UNSUPPORTED;
  const int pairs = tiles < dev.sms / 2 ? (int)tiles : dev.sms / 2;
  static SmemOptIn attr;
  auto kern = pair_kernel<A8, T>;
  DQ_CHECK(opt_in_dynamic_smem(kern, L::TOTAL, attr));
  return launch(LaunchConfig(stream, 2 * pairs, PAIR_THREADS, L::TOTAL, 2), kern, w, ws, x, xs, y, p);
}

// Which kernel.  Up to 64 tokens a cluster's tile: weights are what counts, and a pair's tile would be three quarters empty.
// Above, pairs unless their one tile after another is longer than a cluster's share of the reduction.  Measured (4 to 50 us,
// k 256 to 8192, n 512 to 13824, 80 to 1536 tokens): a pair's step took 0.28 us, a cluster CTA's 0.38, and its epilogue over the
// cluster as long as five of the pair's steps; with more tiles than SMs the clusters lose everywhere.  Both sides, us, 8 bits:
// 256 x 8192 x 1000 clusters 8.7, pairs 22.6; 128 x 4096 x 4096 8.2 and 13.9; 256 x 8192 x 11008 35.3 and 26.4.  A cluster's step has
// become shorter since, and near the border the rule still takes pairs where clusters would win: 100 x 2048 x 11008 8.8 and
// 10.0, 300 x 4096 x 5120 12.5 and 15.0, 333 x 5111 x 5001 14.7 and 18.1 (4 bits: 11.0 and 12.0).
template <bool A8>
dq_status cluster_is_faster(const Device& dev, const Operands& o, bool& yes) {
  constexpr int KT = Step<A8>::KT;
  const int64_t steps = (k_tiles(o.k) + KT - 1) / KT;
  const int64_t tiles = (o.n + 127) / 128 * ((o.m + 127) / 128), pair_tiles = (o.n + 255) / 256 * ((o.m + 255) / 256);
  const int64_t pairs = dev.sms / 2, waves = (pair_tiles + pairs - 1) / pairs;
  int splits = 1;
  yes = o.m <= 64;
  if (yes || tiles > dev.sms) return DQ_OK;
  DQ_CHECK((choose_splits<128, A8, false, float>(dev, tiles, (int)steps, splits)));
  yes = 4 * ((steps + splits - 1) / splits) + 15 < 3 * waves * steps;
  return DQ_OK;
}

template <bool A8>
dq_status product(cudaStream_t stream, const Device& dev, const Operands& o) {
  bool cluster = false;
  DQ_CHECK(cluster_is_faster<A8>(dev, o, cluster));
  if (cluster) {
    if (o.m <= 16) return launch_cluster<16, A8, false, float>(stream, dev, o);
    if (o.m <= 32) return launch_cluster<32, A8, false, float>(stream, dev, o);
    if (o.m <= 64) return launch_cluster<64, A8, false, float>(stream, dev, o);
    return launch_cluster<128, A8, false, float>(stream, dev, o);
  }
  if (o.y_dtype == DQ_BF16) return launch_pair<A8, __nv_bfloat16>(stream, dev, o);
  if (o.y_dtype == DQ_FP16) return launch_pair<A8, __half>(stream, dev, o);
  return launch_pair<A8, float>(stream, dev, o);
}

dq_status run(cudaStream_t stream, const Device& dev, const Operands& o) {
  return o.a_fmt == DQ_MXFP4 ? product<false>(stream, dev, o) : product<true>(stream, dev, o);
}
template <bool A8>
dq_status fused(cudaStream_t stream, const Device& dev, const Operands& o, int x_dtype) {
  if (x_dtype == DQ_BF16) return launch_cluster<16, A8, true, __nv_bfloat16>(stream, dev, o);
  if (x_dtype == DQ_FP16) return launch_cluster<16, A8, true, __half>(stream, dev, o);
  return launch_cluster<16, A8, true, float>(stream, dev, o);
}

}  // namespace

dq_status matmul(cudaStream_t stream, int a_fmt, const uint8_t* a_codes, const uint8_t* a_scales, int64_t m,
                 const uint8_t* w_codes, const uint8_t* w_scales, int64_t n, int64_t k, void* Y, int y_dtype, int64_t ldy) {
  Device dev;
  DQ_CHECK(current_device(dev));
  return run(stream, dev, Operands{a_fmt, a_codes, a_scales, w_codes, w_scales, m, n, k, Y, y_dtype, ldy});
}

dq_status matmul_giving_up(cudaStream_t stream, int a_fmt, const uint8_t* a_codes, const uint8_t* a_scales, int64_t m,
                           const uint8_t* w_codes, const uint8_t* w_scales, int64_t n, int64_t k, void* Y, int y_dtype, int64_t ldy,
                           int64_t step, uint64_t limit_ns) {
  Device dev;
  DQ_CHECK(current_device(dev));
  Operands o{a_fmt, a_codes, a_scales, w_codes, w_scales, m, n, k, Y, y_dtype, ldy};
  o.fail_step = step; o.wait_ns = limit_ns;
  return run(stream, dev, o);
}

dq_status linear(cudaStream_t stream, const void* X, int x_dtype, int64_t m, int64_t k, int64_t ldx, int a_fmt,
                 const uint8_t* w_codes, const uint8_t* w_scales, int64_t n, void* Y, int y_dtype, int64_t ldy,
                 uint8_t* workspace) {
  Device dev;
  DQ_CHECK(current_device(dev));
  uint8_t* scales = workspace + m * row_bytes(a_fmt, k);
  Operands o{a_fmt, workspace, scales, w_codes, w_scales, m, n, k, Y, y_dtype, ldy};
  // Few tokens are quantised by the product's own CTAs, each the part that it multiplies, where that part is small: the CTAs of
  // all weight tiles repeat the work.  Weights from HBM, 4 bits, one launch against two: k = n = 4096, 1024 values a token and
  // CTA, 1 token 4.7 us against 6.1, 8 tokens 5.7 against 6.0, 16 tokens 7.5 against 6.0; k = 1024, n = 4096, 256 values, 16 tokens
  // 4.2 against 4.3; k = n = 8192, 8 tokens 10.9 against 10.1.
  if (m <= 16) {
    o.x = X; o.ldx = ldx;
    o.x_vec = whole_pieces(X, ldx, k, x_dtype);
    const dq_status st = a_fmt == DQ_MXFP4 ? fused<false>(stream, dev, o, x_dtype) : fused<true>(stream, dev, o, x_dtype);
    if (st != DQ_ERR_UNSUPPORTED) return st;                 // (too many values for that, or for their shared memory)
  }
  DQ_CHECK(quantize(stream, X, x_dtype, m, k, ldx, a_fmt, workspace, scales, nullptr, 0));
  o.weights_first = true;
  return run(stream, dev, o);
}

}  // namespace mx
}  // namespace dq
