// Microscaled quantisation: activations or weights to codes and scales (dq_mx_quantize), back to values
// (dq_mx_dequantize), and the root-mean-square norm with the residual's addition in front of it
// (dq_rmsnorm_quantize).  All three are bound by HBM: one read and one write of everything.  Share of the measured copy rate,
// counting every byte once, over several GPUs: 16384 x 4096 bf16 to 4 bits with values 49 to 51 us, 91 to 95 %, codes and
// scales alone 33.4 us, 78 %, back 38.5 us, 67 %; norm of 65536 x 8192 bf16 with residual, sum and values 766 to 803 us, 92 to
// 97 %; 100000 x 128 to 4 bits with values 10.5 to 11.0 us, 80 to 84 %; 5000 x 5111 fp32 (unaligned rows) to 8 bits with values
// 41 to 43 us, 83 to 86 %, the norm of 5000 x 5111 bf16 57 to 62 us, 56 to 62 %.
#include <type_traits>

#include "mx_common.cuh"

namespace dq {
namespace mx {

static __device__ int g_mx_status;

dq_status current_device(Device& out) {
  static PerDevice<Device> known;
  int dev = -1;
  DQ_CHECK_CUDA(cudaGetDevice(&dev));
  if (dev < 0 || dev >= MAX_DEVICES) return DQ_ERR_UNSUPPORTED;
  return (dq_status)known.get(dev, out, [dev](Device& d) -> int {
    int major = 0;
    void* p = nullptr;
    DQ_CHECK_CUDA(cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev));
    if (major != 10) return DQ_ERR_UNSUPPORTED;
    DQ_CHECK_CUDA(cudaDeviceGetAttribute(&d.sms, cudaDevAttrMultiProcessorCount, dev));
    DQ_CHECK_CUDA(cudaGetSymbolAddress(&p, g_mx_status));
    d.d_status = (int*)p;
    d.index = dev;
    return DQ_OK;
  });
}

namespace {

// A warp takes 256 columns of a row at a time (LANES 16: half a warp 128), eight consecutive ones a lane, four lanes a block of
// 32.  WHOLE: rows come in 16-byte pieces, eight values are one or two loads, and a lane's eight columns exist all or not
// at all.  Otherwise the lanes read and write neighbouring values and turn them in shared memory: one by one from each lane's
// own eight columns every load would touch 32 different sectors (5000 x 5111 fp32 to 8 bits: 93 us, 41.5 so).  Rows of k = 0
// columns are neither read nor written and count as zeros; all lanes of a warp make the same calls.
constexpr int PIECE = 256;
template <typename T, bool WHOLE, int LANES>
struct Piece {
  using Raw = Vec8<T>;                       // what a lane fetches
  static __device__ __forceinline__ void fetch(Raw& x, const T* row, int c0, int k, int lane) {
    x.clear();
    if (c0 + lane * 8 < k) x.load(row + c0 + lane * 8);
  }
  static __device__ __forceinline__ const Vec8<T>& turned(const Raw& x, int, T*) { return x; }
  static __device__ __forceinline__ void store(const Vec8<T>& v, T* row, int c0, int k, int lane, T*) {
    if (c0 + lane * 8 < k) v.store(row + c0 + lane * 8);
  }
};
template <typename T, int LANES>
struct Piece<T, false, LANES> {
  struct Raw { T x[8]; };                    // every LANES-th value
  static __device__ __forceinline__ void fetch(Raw& x, const T* row, int c0, int k, int lane) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x.x[i] = c0 + i * LANES + lane < k ? row[c0 + i * LANES + lane] : from_f32<T>(0.f);
  }
  static __device__ __forceinline__ Vec8<T> turned(const Raw& x, int lane, T* turn) {
    Vec8<T> v;
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 8; ++i) turn[i * LANES + lane] = x.x[i];
    __syncwarp();
    v.load(turn + lane * 8);
    return v;
  }
  static __device__ __forceinline__ void store(const Vec8<T>& v, T* row, int c0, int k, int lane, T* turn) {
    __syncwarp();
    v.store(turn + lane * 8);
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c0 + i * LANES + lane < k) row[c0 + i * LANES + lane] = turn[i * LANES + lane];
  }
};

// One warp: rows {i, i + 32, i + 64, i + 96} of a row tile x 256 columns.  The four rows are the ones whose scales are
// neighbours, so a k tile's 16 scale bytes leave in one piece, and their four independent loads per lane are what keeps HBM
// busy.  Every lane has read its values before it writes any, and reads no other lane's (!WHOLE: its warp has, and no other
// warp's): the values may go back to where X lies.  A CTA's eight warps lie side by side, 2^wide of them along the columns.
// NARROW: rows of at most 128 columns, the other half warp takes the next four rows.
constexpr int Q_WARPS = 8;
template <typename T, int FMT, bool WHOLE, bool NARROW>
__global__ void __launch_bounds__(32 * Q_WARPS)
quantize_kernel(const T* X, int64_t rows, int k, int64_t ldx, int wide, uint8_t* __restrict__ codes, uint8_t* __restrict__ scales,
                T* values, int64_t ldv) {
  __shared__ __align__(16) T turn[WHOLE ? 1 : Q_WARPS][WHOLE ? 8 : PIECE];
  wait_for_previous();
  allow_next();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, half = NARROW ? lane >> 4 : 0, place = NARROW ? lane & 15 : lane;
  const int ktiles = (k + KTILE - 1) / KTILE;
  const int c0 = NARROW ? 0 : (((int)blockIdx.y << wide) + (warp & ((1 << wide) - 1))) * PIECE, c = c0 + place * 8;
  const int64_t g = NARROW ? ((int64_t)blockIdx.x * Q_WARPS + warp) * 2 + half : (int64_t)blockIdx.x * (Q_WARPS >> wide) + (warp >> wide);
  const int64_t tile = rows < 32 ? 0 : g >> 5;
  const int64_t i = rows < 32 ? g : g & 31, r0 = tile * ROW_TILE + i;
  if (c0 >= ktiles * KTILE || __all_sync(0xffffffffu, r0 >= rows)) return;   // (whole warps)
  const bool in = c < ktiles * KTILE && r0 < rows;
  using P = Piece<T, WHOLE, NARROW ? 16 : 32>;
  T* stage = turn[WHOLE ? 0 : warp] + (WHOLE ? 0 : half * KTILE);
  // Half warps with rows of their own and shared memory between their lanes go through all four rows together; else a warp
  // skips the rows that do not exist (16384 x 4096 to 4 bits: 49.3 us, 52.5 if it does not).
  constexpr bool ALL = NARROW && !WHOLE;
  auto exists = [&](int j) { return r0 + 32 * j < rows; };
  auto columns = [&](int j) { return ALL && !exists(j) ? 0 : k; };
  Vec8<T> v[4];
  {
    typename P::Raw x[4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (ALL || exists(j)) P::fetch(x[j], X + (r0 + 32 * j) * ldx, c0, columns(j), place);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (ALL || exists(j)) v[j] = P::turned(x[j], place, stage);
      else v[j].clear();
    }
  }
  const uint32_t e01 = block_exponent(v[0].exponent() | v[1].exponent() << 16);
  const uint32_t e23 = block_exponent(v[2].exponent() | v[3].exponent() << 16);
  const uint32_t e[4] = {e01 & 0xffffu, e01 >> 16, e23 & 0xffffu, e23 >> 16};
  const int64_t pitch = row_bytes(FMT, k);
  uint8_t* to = codes + r0 * pitch + c / 8 * Codes8<FMT>::BYTES;
  uint32_t mine = 0;                                          // scale of row (lane % 4) of the four
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t s = scale_code<FMT>(e[j]);
    if ((lane & 3) == j) mine = s;
    if (ALL || exists(j)) {
      Codes8<FMT> q;
      q.encode(v[j], s);
      if (in && (!ALL || exists(j))) q.store(to + 32 * j * pitch);
      if (values) {
        q.decode(s, v[j]);
        P::store(v[j], values + (r0 + 32 * j) * ldv, c0, columns(j), place, stage);
      }
    }
  }
  // four blocks x four rows of a k tile sit in 16 lanes; lane 4 b + j has the scale of (block b, row j)
  mine <<= 8 * ((lane >> 2) & 3);
  mine |= __shfl_xor_sync(0xffffffffu, mine, 4);
  mine |= __shfl_xor_sync(0xffffffffu, mine, 8);
  if (in && (lane & 12) == 0)
    *reinterpret_cast<uint32_t*>(scales + (tile * ktiles + c / KTILE) * TILE_BYTES + i * 16 + (lane & 3) * 4) = mine;
}

// A warp per 256 columns of a row.
template <typename T, int FMT, bool WHOLE>
__global__ void __launch_bounds__(32 * Q_WARPS)
dequantize_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, int64_t rows, int k, int wide, T* __restrict__ Y,
                  int64_t ldy) {
  __shared__ __align__(16) T turn[WHOLE ? 1 : Q_WARPS][WHOLE ? 8 : PIECE];
  wait_for_previous();
  allow_next();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int c0 = (((int)blockIdx.y << wide) + (warp & ((1 << wide) - 1))) * PIECE, c = c0 + lane * 8;
  const int64_t r = (int64_t)blockIdx.x * (Q_WARPS >> wide) + (warp >> wide);
  if (c0 >= k || r >= rows) return;                           // (whole warps)
  Vec8<T> v;
  v.clear();
  if (c < k) {
    Codes8<FMT> q;
    q.load(codes + r * row_bytes(FMT, k) + c / 8 * Codes8<FMT>::BYTES);
    q.decode(scales[scale_offset(r, c / BLOCK, k_tiles(k))], v);
  }
  Piece<T, WHOLE, 32>::store(v, Y + r * ldy, c0, k, lane, turn[WHOLE ? 0 : warp]);
}

// ------------------------------------------------------------------------------------------------ norm
// A row belongs to `warps` warps, each with V pieces of 256 columns that stay in registers between the sum of squares and the
// scaling, so x and the residual are read once.  One warp a row: eight rows a CTA, no barrier; else one row a CTA.
// NARROW (V = 1): rows of at most 128 columns, half a warp each.
template <typename T, typename G, int FMT, int V, bool WHOLE, bool NARROW>
__global__ void __launch_bounds__(V == 1 ? 1024 : 512)
rmsnorm_kernel(const T* X, int64_t rows, int k, int64_t ldx, const T* residual, int64_t ldr, const G* gamma, float eps,
                               uint8_t* __restrict__ codes, uint8_t* __restrict__ scales, T* sum, int64_t lds, T* values, int64_t ldv,
                               int warps) {
  extern __shared__ __align__(16) uint8_t turn[];             // !WHOLE: 1 KB a warp
  __shared__ float part[32];
  wait_for_previous();
  allow_next();
  static_assert(!NARROW || V == 1, "one piece");
  constexpr int LANES = NARROW ? 16 : 32;
  using P = Piece<T, WHOLE, LANES>;
  const int w = threadIdx.x >> 5, lane = NARROW ? threadIdx.x & 15 : threadIdx.x & 31;
  int64_t r = warps == 1 ? (int64_t)blockIdx.x * (blockDim.x >> 5) + w : blockIdx.x;
  if (NARROW) r = r * 2 + (threadIdx.x >> 4 & 1);
  if (__all_sync(0xffffffffu, r >= rows)) return;             // (whole warps; with more than one a row, whole CTAs)
  const bool live = !NARROW || r < rows;                      // (the half of a last warp that has no row repeats the last one)
  if (NARROW && !live) r = rows - 1;
  const int kw = live ? k : 0;                                // columns that are written
  const int first = warps == 1 ? 0 : w;
  T* stage = reinterpret_cast<T*>(turn + (WHOLE ? 0 : w * 1024 + (NARROW ? (threadIdx.x >> 4 & 1) * 512 : 0)));
  G* g_stage = reinterpret_cast<G*>(stage);
  auto column = [&](int u) { return (u * warps + first) * PIECE; };
  float2 h[V][4];
  float2 ss = make_float2(0.f, 0.f);
  {
    typename P::Raw x[V], b[V];
#pragma unroll
    for (int u = 0; u < V; ++u) P::fetch(x[u], X + r * ldx, column(u), k, lane);
    if (residual) {
#pragma unroll
      for (int u = 0; u < V; ++u) P::fetch(b[u], residual + r * ldr, column(u), k, lane);
    }
#pragma unroll
    for (int u = 0; u < V; ++u) {
      const Vec8<T> v = P::turned(x[u], lane, stage);
#pragma unroll
      for (int i = 0; i < 4; ++i) h[u][i] = v.pair(i);
    }
    if (residual) {
#pragma unroll
      for (int u = 0; u < V; ++u) {
        const Vec8<T> v = P::turned(b[u], lane, stage);
#pragma unroll
        for (int i = 0; i < 4; ++i) h[u][i] = add2(h[u][i], v.pair(i));
      }
    }
  }
#pragma unroll
  for (int u = 0; u < V; ++u) {
#pragma unroll
    for (int i = 0; i < 4; ++i) ss = add2(ss, mul2(h[u][i], h[u][i]));
    if (sum) {
      Vec8<T> s;
#pragma unroll
      for (int i = 0; i < 4; ++i) s.set_pair(i, h[u][i]);
      P::store(s, sum + r * lds, column(u), kw, lane, stage);
    }
  }
  float all = ss.x + ss.y;
#pragma unroll
  for (int o = NARROW ? 8 : 16; o >= 1; o >>= 1) all += __shfl_xor_sync(0xffffffffu, all, o);
  if (warps > 1) {
    if (lane == 0) part[w] = all;
    __syncthreads();
    all = lane < warps ? part[lane] : 0.f;
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) all += __shfl_xor_sync(0xffffffffu, all, o);
  }
  const float rstd = rsqrtf(all / (float)k + eps);
  const int ktiles = (k + KTILE - 1) / KTILE;
  uint8_t* to = codes + r * row_bytes(FMT, k);
#pragma unroll
  for (int u = 0; u < V; ++u) {
    const int c0 = column(u), c = c0 + lane * 8;
    if (c0 >= ktiles * KTILE) break;                          // (whole warps)
    Vec8<float> y;
    Vec8<G> g;
    if (gamma) {
      typename Piece<G, WHOLE, LANES>::Raw x;
      Piece<G, WHOLE, LANES>::fetch(x, gamma, c0, k, lane);
      g = Piece<G, WHOLE, LANES>::turned(x, lane, g_stage);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f = mul2(h[u][i], make_float2(rstd, rstd));
      y.set_pair(i, gamma ? mul2(f, g.pair(i)) : f);
    }
    if (c >= k) y.clear();       // padding: not a value, whatever the row's statistics are
    else if (!WHOLE && c + 8 > k) {
#pragma unroll
      for (int e = 0; e < 8; ++e) if (c + e >= k) y.v[e] = 0.f;
    }
    uint32_t s = scale_code<FMT>(block_exponent(y.exponent()));
    Codes8<FMT> q;
    q.encode(y, s);
    const bool in = c < ktiles * KTILE && live;
    if (in) q.store(to + c / 8 * Codes8<FMT>::BYTES);
    if (values) {
      Vec8<T> d;
      q.decode(s, d);
      P::store(d, values + r * ldv, c0, kw, lane, stage);
    }
    s <<= 8 * ((lane >> 2) & 3);
    s |= __shfl_xor_sync(0xffffffffu, s, 4);
    s |= __shfl_xor_sync(0xffffffffu, s, 8);
    if (in && (lane & 15) == 0) *reinterpret_cast<uint32_t*>(scales + scale_offset(r, c / BLOCK, ktiles)) = s;
  }
}

template <typename F>
dq_status by_type(int dtype, F f) {
  if (dtype == DQ_FP32) return f(float{});
  if (dtype == DQ_BF16) return f(__nv_bfloat16{});
  if (dtype == DQ_FP16) return f(__half{});
  return DQ_ERR_INVALID_ARG;
}
template <int FMT> struct Fmt { static constexpr int value = FMT; };
template <typename F>
dq_status by_format(int fmt, F f) {
  if (fmt == DQ_MXFP4) return f(Fmt<DQ_MXFP4>{});
  if (fmt == DQ_MXFP8) return f(Fmt<DQ_MXFP8>{});
  return DQ_ERR_INVALID_ARG;
}

}  // namespace

namespace {
// Warps of a CTA that lie along the columns: as many as there are pieces, up to all (as a power of two).
inline int columns_wide(int64_t pieces) { return pieces >= 8 ? 3 : pieces >= 4 ? 2 : pieces >= 2 ? 1 : 0; }
inline dq_status grid(LaunchConfig& c, int64_t pieces, int64_t row_groups, int wide) {
  const int64_t x = (row_groups + (Q_WARPS >> wide) - 1) / (Q_WARPS >> wide), y = (pieces + (1 << wide) - 1) >> wide;
  if (x > 0x7fffffff || y > 65535) return DQ_ERR_UNSUPPORTED;
  c.cfg.gridDim = dim3((unsigned)x, (unsigned)y);
  return DQ_OK;
}
template <typename F>
dq_status by_flag(bool flag, F f) { return flag ? f(std::true_type{}) : f(std::false_type{}); }
}  // namespace

dq_status quantize(cudaStream_t stream, const void* X, int x_dtype, int64_t rows, int64_t k, int64_t ldx, int fmt,
                   uint8_t* codes, uint8_t* scales, void* values, int64_t ldv) {
  const bool whole = whole_pieces(X, ldx, k, x_dtype) && (!values || whole_pieces(values, ldv, k, x_dtype));
  const int64_t pieces = (k_tiles(k) * KTILE + PIECE - 1) / PIECE;
  const int64_t groups = rows < 32 ? rows : (rows + ROW_TILE - 1) / ROW_TILE * 32;
  const int wide = columns_wide(pieces);
  const bool narrow = k <= KTILE;
  LaunchConfig c(stream, 1, 32 * Q_WARPS);
  DQ_CHECK(grid(c, pieces, narrow ? (groups + 1) / 2 : groups, wide));
  return by_type(x_dtype, [&](auto t) {
    using T = decltype(t);
    return by_format(fmt, [&](auto f) {
      constexpr int FMT = decltype(f)::value;
      auto run = [&](auto kern) { return launch(c, kern, (const T*)X, rows, (int)k, ldx, wide, codes, scales, (T*)values, ldv); };
      if (narrow) return whole ? run(quantize_kernel<T, FMT, true, true>) : run(quantize_kernel<T, FMT, false, true>);
      return whole ? run(quantize_kernel<T, FMT, true, false>) : run(quantize_kernel<T, FMT, false, false>);
    });
  });
}

dq_status dequantize(cudaStream_t stream, int fmt, const uint8_t* codes, const uint8_t* scales, int64_t rows, int64_t k,
                     void* Y, int y_dtype, int64_t ldy) {
  const int64_t pieces = (k + PIECE - 1) / PIECE;
  const int wide = columns_wide(pieces);
  LaunchConfig c(stream, 1, 32 * Q_WARPS);
  DQ_CHECK(grid(c, pieces, rows, wide));
  return by_type(y_dtype, [&](auto t) {
    using T = decltype(t);
    return by_format(fmt, [&](auto f) {
      return by_flag(whole_pieces(Y, ldy, k, y_dtype), [&](auto v) {
        return launch(c, dequantize_kernel<T, decltype(f)::value, decltype(v)::value>, codes, scales, rows, (int)k, wide, (T*)Y, ldy);
      });
    });
  });
}

dq_status rmsnorm_quantize(cudaStream_t stream, const void* X, int dtype, int64_t rows, int64_t k, int64_t ldx,
                           const void* residual, int64_t ldr, const void* gamma, int gamma_dtype, float eps, int fmt,
                           uint8_t* codes, uint8_t* scales, void* sum, int64_t lds, void* values, int64_t ldv) {
  const bool whole = whole_pieces(X, ldx, k, dtype) && (!residual || whole_pieces(residual, ldr, k, dtype)) &&
                     (!sum || whole_pieces(sum, lds, k, dtype)) && (!values || whole_pieces(values, ldv, k, dtype)) &&
                     (!gamma || whole_pieces(gamma, 0, k, gamma_dtype));
  const int pieces = (int)((k_tiles(k) * KTILE + PIECE - 1) / PIECE);
  if (pieces > 4 * 32) return DQ_ERR_UNSUPPORTED;             // 32768 columns: a row has to stay in one CTA's registers
  Device dev;
  DQ_CHECK(current_device(dev));
  // Pieces a warp: one where there are few rows (latency), else four, or two where four would leave too few warps to keep HBM
  // busy or the rows are not in whole pieces (4096 x 1024: 9.4 us with two, 11.4 with four; 16384 x 8192: 185 with four,
  // 207 with two; 5000 x 5111: 62 with two, 73 with four); eight where a CTA of 16 warps would not hold the row.  Between 592
  // and about 5000 rows of whole pieces, where four begin, neither is better throughout: 1200 x 4096 12.7 us with four and 10.9
  // with two, 1777 x 5120 18.3 and 18.0, 600 x 5120 7.7 and 8.8, 3000 x 8192 39.7 and 42.1; from 9000 rows on four are
  // better by 6 to 12 %, except for rows of 1280 and 2560 values (two better by 5 % and by nothing).
  const bool few = rows <= 4 * dev.sms || (pieces <= 4 && rows <= 64 * dev.sms);
  const int V = pieces == 1 || (rows <= 2 * dev.sms && pieces <= 32) ? 1
                : pieces == 2 || (pieces <= 32 && (few || !whole)) ? 2 : pieces <= 64 ? 4 : 8;
  const int warps = (pieces + V - 1) / V;
  const int threads = warps == 1 ? 256 : warps * 32;
  const bool narrow = k <= KTILE;
  const int64_t ctas = warps > 1 ? rows : narrow ? (rows + 15) / 16 : (rows + 7) / 8;
  LaunchConfig c(stream, ctas, threads, whole ? 0 : threads * 32);
  return by_type(dtype, [&](auto t) {
    using T = decltype(t);
    return by_format(fmt, [&](auto f) {
      constexpr int FMT = decltype(f)::value;
      return by_flag(whole, [&](auto wh) {
        constexpr bool WHOLE = decltype(wh)::value;
        auto run = [&](auto g, auto kern) {
          using G = decltype(g);
          return launch(c, kern, (const T*)X, rows, (int)k, ldx, (const T*)residual, ldr, (const G*)gamma, eps, codes, scales,
                        (T*)sum, lds, (T*)values, ldv, warps);
        };
        auto with_gamma = [&](auto g) {
          using G = decltype(g);
          if (narrow) return run(g, rmsnorm_kernel<T, G, FMT, 1, WHOLE, true>);
          if (V == 1) return run(g, rmsnorm_kernel<T, G, FMT, 1, WHOLE, false>);
          if (V == 2) return run(g, rmsnorm_kernel<T, G, FMT, 2, WHOLE, false>);
          if (V == 4) return run(g, rmsnorm_kernel<T, G, FMT, 4, WHOLE, false>);
          return run(g, rmsnorm_kernel<T, G, FMT, 8, WHOLE, false>);
        };
        if (gamma && gamma_dtype == DQ_FP32) return with_gamma(float{});
        return with_gamma(T{});
      });
    });
  });
}

}  // namespace mx
}  // namespace dq
