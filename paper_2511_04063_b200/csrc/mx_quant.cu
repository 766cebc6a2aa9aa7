// Microscaled quantisation: activations or weights to codes and scales (dq_mx_quantize), back to values
// (dq_mx_dequantize), and the root-mean-square norm with the residual's addition in front of it
// (dq_rmsnorm_quantize).  All three are bound by HBM: one read and one write of everything.
#include "mx_common.cuh"

namespace dq {
namespace mx {

static __device__ int g_mx_status;

dq_status current_device(Device& out) {
  static Device known[64];
  static bool done[64] = {};
  int dev = -1;
  DQ_CHECK_CUDA(cudaGetDevice(&dev));
  if (dev < 0 || dev >= 64) return DQ_ERR_UNSUPPORTED;
  if (!done[dev]) {
    int major = 0;
    Device d;
    void* p = nullptr;
    DQ_CHECK_CUDA(cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev));
    if (major != 10) return DQ_ERR_UNSUPPORTED;
    DQ_CHECK_CUDA(cudaDeviceGetAttribute(&d.sms, cudaDevAttrMultiProcessorCount, dev));
    DQ_CHECK_CUDA(cudaGetSymbolAddress(&p, g_mx_status));
    d.d_status = (int*)p;
    known[dev] = d;
    done[dev] = true;
  }
  out = known[dev];
  return DQ_OK;
}

namespace {

inline int type_bytes(int dtype) { return dtype == DQ_FP32 ? 4 : 2; }
// Whether every row of a matrix starts on a 16-byte boundary.
inline bool rows_aligned(const void* p, int64_t ld, int dtype) {
  return ((uintptr_t)p & 15) == 0 && (ld * type_bytes(dtype)) % 16 == 0;
}

// One warp: rows {i, i + 32, i + 64, i + 96} of a row tile x 256 columns, 8 values of each row per lane.  The four rows
// are the ones whose scales are neighbours, so a k tile's 16 scale bytes leave in one piece, and their four independent
// 16-byte loads per lane are what keeps HBM busy.  Every lane has read its values before it writes any, and reads no
// other lane's: the values may go back to where X lies.
constexpr int Q_COLS = 256;
template <typename T, int FMT>
__global__ void __launch_bounds__(256) quantize_kernel(const T* X, int64_t rows, int64_t k, int64_t ldx, int row_groups,
                                                       int64_t col_chunks, uint8_t* __restrict__ codes, uint8_t* __restrict__ scales,
                                                       T* values, int64_t ldv, int x_vec, int v_vec) {
  wait_for_previous();
  allow_next();
  const int lane = threadIdx.x & 31;
  const int64_t w = (int64_t)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
  const int64_t ktiles = k_tiles(k);
  const int64_t chunk = w % col_chunks, g = w / col_chunks;
  const int64_t i = g % row_groups, tile = g / row_groups;
  if (tile * ROW_TILE >= rows) return;                        // (whole warps)
  const int64_t c = chunk * Q_COLS + lane * 8;
  const bool in = c < ktiles * KTILE;
  float v[4][8];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int64_t r = tile * ROW_TILE + 32 * j + i;
    if (r < rows) load8(X + r * ldx, c, k, x_vec, v[j]);
    else {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[j][e] = 0.f;
    }
  }
  uint32_t mine = 0;                                          // scale of row (lane % 4) of the four
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int64_t r = tile * ROW_TILE + 32 * j + i;
    Codes8<FMT> q;
    const uint32_t s = encode_block<FMT>(v[j], q);
    if ((lane & 3) == j) mine = s;
    if (r < rows && in) {
      q.store(codes + r * row_bytes(FMT, k) + c / 8 * Codes8<FMT>::BYTES);
      if (values) {
        float y[8];
        q.decode(scale_value(s), y);
        store8(values + r * ldv, c, k, v_vec, y);
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

template <typename T, int FMT>
__global__ void __launch_bounds__(256) dequantize_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales,
                                                         int64_t rows, int64_t k, T* __restrict__ Y, int64_t ldy, int vec) {
  wait_for_previous();
  allow_next();
  const int64_t groups = (k + 7) / 8;
  const int64_t at = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  const int64_t r = at / groups, c = at % groups * 8;
  if (r >= rows) return;
  Codes8<FMT> q;
  q.load(codes + r * row_bytes(FMT, k) + c / 8 * Codes8<FMT>::BYTES);
  float v[8];
  q.decode(scale_value(scales[scale_offset(r, c / BLOCK, k_tiles(k))]), v);
  store8(Y + r * ldy, c, k, vec, v);
}

// ------------------------------------------------------------------------------------------------ norm
// A row belongs to a group of `threads_per_row` threads (whole warps); V vectors of 8 values a thread stay in registers
// between the sum of squares and the scaling, so x and the residual are read once.
template <typename T, typename G, int FMT, int V>
__global__ void rmsnorm_kernel(const T* X, int64_t rows, int64_t k, int64_t ldx, const T* residual, int64_t ldr,
                               const G* __restrict__ gamma, float eps, uint8_t* __restrict__ codes, uint8_t* __restrict__ scales,
                               T* sum, int64_t lds, T* values, int64_t ldv, int threads_per_row, int vec, int g_vec) {
  __shared__ float part[32];
  wait_for_previous();
  allow_next();
  const int row_in_cta = threadIdx.x / threads_per_row, t = threadIdx.x % threads_per_row;
  const int lane = threadIdx.x & 31, warps = threads_per_row >> 5, warp0 = row_in_cta * warps;
  const int64_t r = (int64_t)blockIdx.x * (blockDim.x / threads_per_row) + row_in_cta;
  const bool live = r < rows;
  float h[V][8];
  float ss = 0.f;
#pragma unroll
  for (int u = 0; u < V; ++u) {
    const int64_t c = ((int64_t)u * threads_per_row + t) * 8;
    if (live) load8(X + r * ldx, c, k, vec, h[u]);
    else {
#pragma unroll
      for (int e = 0; e < 8; ++e) h[u][e] = 0.f;
    }
    if (residual && live) {
      float b[8];
      load8(residual + r * ldr, c, k, vec, b);
#pragma unroll
      for (int e = 0; e < 8; ++e) h[u][e] += b[e];
    }
  }
#pragma unroll
  for (int u = 0; u < V; ++u) {
    const int64_t c = ((int64_t)u * threads_per_row + t) * 8;
    if (sum && live) store8(sum + r * lds, c, k, vec, h[u]);
#pragma unroll
    for (int e = 0; e < 8; ++e) ss += h[u][e] * h[u][e];
  }
#pragma unroll
  for (int o = 16; o >= 1; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
  if (warps > 1) {
    if (lane == 0) part[warp0 + (t >> 5)] = ss;
    __syncthreads();
    ss = 0.f;
    for (int i = 0; i < warps; ++i) ss += part[warp0 + i];
  }
  const float rstd = rsqrtf(ss / (float)k + eps);
  const int64_t ktiles = k_tiles(k);
#pragma unroll
  for (int u = 0; u < V; ++u) {
    const int64_t c = ((int64_t)u * threads_per_row + t) * 8;
    float y[8];
    if (gamma) {
      load8(gamma, c, k, g_vec, y);
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = h[u][e] * rstd * y[e];
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = h[u][e] * rstd;
    }
    if (c >= k) {      // padding: not a value, whatever the row's statistics are
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = 0.f;
    }
    Codes8<FMT> q;
    uint32_t s = encode_block<FMT>(y, q);
    if (live && c < ktiles * KTILE) {
      q.store(codes + r * row_bytes(FMT, k) + c / 8 * Codes8<FMT>::BYTES);
      if (values) {
        float d[8];
        q.decode(scale_value(s), d);
        store8(values + r * ldv, c, k, vec, d);
      }
    }
    s <<= 8 * ((lane >> 2) & 3);
    s |= __shfl_xor_sync(0xffffffffu, s, 4);
    s |= __shfl_xor_sync(0xffffffffu, s, 8);
    if (live && c < ktiles * KTILE && (lane & 15) == 0)
      *reinterpret_cast<uint32_t*>(scales + scale_offset(r, c / BLOCK, ktiles)) = s;
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

dq_status quantize(cudaStream_t stream, const void* X, int x_dtype, int64_t rows, int64_t k, int64_t ldx, int fmt,
                   uint8_t* codes, uint8_t* scales, void* values, int64_t ldv) {
  return by_type(x_dtype, [&](auto t) {
    using T = decltype(t);
    return by_format(fmt, [&](auto f) {
      constexpr int FMT = decltype(f)::value;
      const int64_t chunks = (k_tiles(k) * KTILE + Q_COLS - 1) / Q_COLS;
      const int groups = (int)(rows < 32 ? rows : 32);
      const int64_t warps = (rows + ROW_TILE - 1) / ROW_TILE * groups * chunks;
      const int threads = 256;
      const int64_t ctas = (warps + threads / 32 - 1) / (threads / 32);
      if (ctas > 0x7fffffff) return DQ_ERR_UNSUPPORTED;
      return launch(LaunchConfig(stream, ctas, threads), quantize_kernel<T, FMT>, (const T*)X, rows, k, ldx, groups, chunks, codes,
                    scales, (T*)values, ldv, rows_aligned(X, ldx, x_dtype), rows_aligned(values, ldv, x_dtype));
    });
  });
}

dq_status dequantize(cudaStream_t stream, int fmt, const uint8_t* codes, const uint8_t* scales, int64_t rows, int64_t k,
                     void* Y, int y_dtype, int64_t ldy) {
  return by_type(y_dtype, [&](auto t) {
    using T = decltype(t);
    return by_format(fmt, [&](auto f) {
      constexpr int FMT = decltype(f)::value;
      const int64_t ctas = (rows * ((k + 7) / 8) + 255) / 256;
      if (ctas > 0x7fffffff) return DQ_ERR_UNSUPPORTED;
      return launch(LaunchConfig(stream, ctas, 256), dequantize_kernel<T, FMT>, codes, scales, rows, k, (T*)Y, ldy,
                    rows_aligned(Y, ldy, y_dtype));
    });
  });
}

dq_status rmsnorm_quantize(cudaStream_t stream, const void* X, int dtype, int64_t rows, int64_t k, int64_t ldx,
                           const void* residual, int64_t ldr, const void* gamma, int gamma_dtype, float eps, int fmt,
                           uint8_t* codes, uint8_t* scales, void* sum, int64_t lds, void* values, int64_t ldv) {
  const bool vec = rows_aligned(X, ldx, dtype) && (!residual || rows_aligned(residual, ldr, dtype)) &&
                   (!sum || rows_aligned(sum, lds, dtype)) && (!values || rows_aligned(values, ldv, dtype));
  const bool g_vec = ((uintptr_t)gamma & 15) == 0;
  const int64_t groups = k_tiles(k) * (KTILE / 8);
  if (groups > 4 * 1024) return DQ_ERR_UNSUPPORTED;           // 32768 columns: a row has to stay in one CTA's registers
  const int V = groups <= 1024 ? (groups <= 64 ? 1 : 2) : 4;
  const int per_row = (int)((groups + 32 * V - 1) / (32 * V)) * 32;
  const int rows_per_cta = per_row >= 128 ? 1 : 128 / per_row;
  const int64_t ctas = (rows + rows_per_cta - 1) / rows_per_cta;
  if (ctas > 0x7fffffff) return DQ_ERR_UNSUPPORTED;
  return by_type(dtype, [&](auto t) {
    using T = decltype(t);
    return by_format(fmt, [&](auto f) {
      constexpr int FMT = decltype(f)::value;
      auto run = [&](auto g, auto kern) {
        using G = decltype(g);
        return launch(LaunchConfig(stream, ctas, per_row * rows_per_cta), kern, (const T*)X, rows, k, ldx, (const T*)residual, ldr,
                      (const G*)gamma, eps, codes, scales, (T*)sum, lds, (T*)values, ldv, per_row, vec, g_vec);
      };
      auto with_gamma = [&](auto g) {
        using G = decltype(g);
        if (V == 1) return run(g, rmsnorm_kernel<T, G, FMT, 1>);
        if (V == 2) return run(g, rmsnorm_kernel<T, G, FMT, 2>);
        return run(g, rmsnorm_kernel<T, G, FMT, 4>);
      };
      if (gamma && gamma_dtype == DQ_FP32) return with_gamma(float{});
      return with_gamma(T{});
    });
  });
}

}  // namespace mx
}  // namespace dq
