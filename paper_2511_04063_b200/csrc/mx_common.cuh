// Shared device code of the microscaled operators (mx_quant.cu, mx_matmul.cu): the block format, its conversions and
// the addresses of its scales.
//
// A row of k values is cut into blocks of 32.  A block is held as one power of two, the E8M0 byte
//     s = max(exponent field of max|x| - EMAX, 0)            (value 2^(s - 127); 0xFF is NaN)
// and 32 elements q = RNE(x 2^(127 - s)), saturated, of type E2M1 (EMAX 2, largest 6) or E4M3 (EMAX 8, largest 448).
// The exponent field of a float is floor(log2) + 127 for every normal number and 0 below, so the shared exponent is
// floor(log2 max|x|) - EMAX, clamped at 2^-127, without a logarithm.  A block that holds a NaN or an infinity has
// an exponent field of 255: its scale becomes NaN and with it every value of the block.
#pragma once
#include <cuda_fp16.h>

#include "common.cuh"
#include "per_device.h"

namespace dq {
namespace mx {

constexpr int BLOCK = 32;          // values that share a scale
constexpr int KTILE = 128;         // values of a scale tile (4 blocks); rows of codes are padded to it
constexpr int ROW_TILE = 128;      // rows of a scale tile
constexpr int TILE_BYTES = 512;    // 128 rows x 4 scales

inline __host__ __device__ int64_t k_tiles(int64_t k) { return (k + KTILE - 1) / KTILE; }
inline __host__ __device__ int64_t row_bytes(int fmt, int64_t k) { return k_tiles(k) * (fmt == DQ_MXFP4 ? 64 : 128); }
inline int64_t scale_bytes(int64_t rows, int64_t k) { return (rows + ROW_TILE - 1) / ROW_TILE * k_tiles(k) * TILE_BYTES; }

// Byte of the scale of (row, block): tiles of 128 rows x 4 blocks, [row tile][k tile][row % 32][row / 32 % 4][block % 4].
// This is the order in which the block-scaled MMA wants the scales in tensor memory: 32 lanes x 4 columns of 4 bytes.
__device__ __forceinline__ int64_t scale_offset(int64_t row, int64_t block, int64_t ktiles) {
  return ((row >> 7) * ktiles + (block >> 2)) * TILE_BYTES + (row & 31) * 16 + ((row >> 5) & 3) * 4 + (block & 3);
}

// Two products in one instruction.
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 d;
  asm("{\n\t.reg .b64 a, b, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmul.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 d;
  asm("{\n\t.reg .b64 a, b, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tadd.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
// Magnitude of the larger one, NaN if either is (with a sign that means nothing).
__device__ __forceinline__ float larger(float a, float b) {
  float d;
  asm("max.NaN.xorsign.abs.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
  return d;
}
__device__ __forceinline__ uint32_t exponent_field(float v) { return (__float_as_uint(v) >> 23) & 255u; }

// Eight consecutive values as they lie in memory.  exponent() is the exponent field, as a float's, of the largest
// magnitude: all that the scale of a block needs of its values; 255 if one of them is not finite.
template <typename T> struct Vec8;
template <> struct Vec8<float> {
  float v[8];
  __device__ __forceinline__ void load(const float* p) {
    const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  }
  __device__ __forceinline__ void store(float* p) const {
    reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = 0.f;
  }
  __device__ __forceinline__ float2 pair(int i) const { return make_float2(v[2 * i], v[2 * i + 1]); }
  __device__ __forceinline__ void set_pair(int i, float2 f) { v[2 * i] = f.x; v[2 * i + 1] = f.y; }
  __device__ __forceinline__ uint32_t exponent() const {
    return exponent_field(larger(larger(larger(v[0], v[1]), larger(v[2], v[3])), larger(larger(v[4], v[5]), larger(v[6], v[7]))));
  }
};
struct Words8 {   // of a 16-bit type
  uint32_t w[4];
  __device__ __forceinline__ void load(const void* p) {
    const uint4 a = *reinterpret_cast<const uint4*>(p);
    w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w;
  }
  __device__ __forceinline__ void store(void* p) const { *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]); }
  __device__ __forceinline__ void clear() { w[0] = w[1] = w[2] = w[3] = 0u; }
  // magnitudes order like their bits, NaN above infinity above all
  __device__ __forceinline__ uint32_t largest() const {
    constexpr uint32_t ABS = 0x7fff7fffu;
    const uint32_t m = __vmaxu2(__vmaxu2(w[0] & ABS, w[1] & ABS), __vmaxu2(w[2] & ABS, w[3] & ABS));
    return max(m >> 16, m & 0xffffu);
  }
};
template <> struct Vec8<__nv_bfloat16> : Words8 {
  __device__ __forceinline__ float2 pair(int i) const { return make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u)); }
  __device__ __forceinline__ void set_pair(int i, float2 f) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(f.x, f.y);
    w[i] = *reinterpret_cast<const uint32_t*>(&h);
  }
  __device__ __forceinline__ uint32_t exponent() const { return largest() >> 7; }
};
template <> struct Vec8<__half> : Words8 {
  __device__ __forceinline__ float2 pair(int i) const { return __half22float2(*reinterpret_cast<const __half2*>(&w[i])); }
  __device__ __forceinline__ void set_pair(int i, float2 f) {
    const __half2 h = __floats2half2_rn(f.x, f.y);
    w[i] = *reinterpret_cast<const uint32_t*>(&h);
  }
  __device__ __forceinline__ uint32_t exponent() const { return exponent_field(__half2float(__ushort_as_half((unsigned short)largest()))); }
};
__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }

// Eight values of a row of k starting at column c, one by one; what lies past the row's end is zero.
template <typename T>
__device__ __forceinline__ void load_each(Vec8<T>& v, const T* row, int c, int k) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
    v.set_pair(i, make_float2(c + 2 * i < k ? to_f32(row[c + 2 * i]) : 0.f, c + 2 * i + 1 < k ? to_f32(row[c + 2 * i + 1]) : 0.f));
}

// The four lanes that hold a block agree on its largest exponent (two packed in 16 bits each: two blocks at once).
__device__ __forceinline__ uint32_t block_exponent(uint32_t e) {
  e = __vmaxu2(e, __shfl_xor_sync(0xffffffffu, e, 1));
  return __vmaxu2(e, __shfl_xor_sync(0xffffffffu, e, 2));
}
template <int FMT>
__device__ __forceinline__ uint32_t scale_code(uint32_t exponent) {
  constexpr int EMAX = (FMT == DQ_MXFP4) ? 2 : 8;
  return exponent == 255u ? 255u : (uint32_t)max((int)exponent - EMAX, 0);
}
// 2^(127 - s): what the values are multiplied with (0 for a NaN block, whose elements are held as zeros).
__device__ __forceinline__ float inverse_scale(uint32_t s) { return s == 255u ? 0.f : __uint_as_float((254u - s) << 23); }
// 2^(s - 127)
__device__ __forceinline__ float scale_value(uint32_t s) {
  return __uint_as_float(s == 0u ? 0x00400000u : (s == 255u ? 0x7fffffffu : s << 23));
}

// Eight elements: E2M1 packed into 4 bytes (element 0 in the lowest bits), E4M3 into 8.  The conversions of a pair put
// their first operand into the upper half.  Rounding is to nearest even, saturating.  A block whose scale is NaN is held as
// zeros (its values times an inverse scale of 0 may be NaN, which the conversion would turn into numbers).
template <int FMT> struct Codes8;
template <> struct Codes8<DQ_MXFP4> {
  static constexpr int BYTES = 4;
  uint32_t w;
  template <typename T>
  __device__ __forceinline__ void encode(const Vec8<T>& v, uint32_t s) {
    const float inv = inverse_scale(s);
    float2 f[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = mul2(v.pair(i), make_float2(inv, inv));
    asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b0, %2, %1;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b1, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b2, %6, %5;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b3, %8, %7;\n\t"
        "mov.b32 %0, {b0, b1, b2, b3};\n\t}"
        : "=r"(w) : "f"(f[0].x), "f"(f[0].y), "f"(f[1].x), "f"(f[1].y), "f"(f[2].x), "f"(f[2].y), "f"(f[3].x), "f"(f[3].y));
    if (s == 255u) w = 0u;
  }
  template <typename T>
  __device__ __forceinline__ void decode(uint32_t s, Vec8<T>& v) const {
    uint32_t h[4];
    asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\tmov.b32 {b0, b1, b2, b3}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, b0;\n\t"
        "cvt.rn.f16x2.e2m1x2 %1, b1;\n\t"
        "cvt.rn.f16x2.e2m1x2 %2, b2;\n\t"
        "cvt.rn.f16x2.e2m1x2 %3, b3;\n\t}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(w));
    const float f = scale_value(s);
#pragma unroll
    for (int i = 0; i < 4; ++i) v.set_pair(i, mul2(__half22float2(*reinterpret_cast<const __half2*>(&h[i])), make_float2(f, f)));
  }
  __device__ __forceinline__ void store(uint8_t* p) const { *reinterpret_cast<uint32_t*>(p) = w; }
  __device__ __forceinline__ void load(const uint8_t* p) { w = *reinterpret_cast<const uint32_t*>(p); }
};
template <> struct Codes8<DQ_MXFP8> {
  static constexpr int BYTES = 8;
  uint32_t w[2];
  template <typename T>
  __device__ __forceinline__ void encode(const Vec8<T>& v, uint32_t s) {
    const float inv = inverse_scale(s);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float2 a = mul2(v.pair(2 * i), make_float2(inv, inv)), b = mul2(v.pair(2 * i + 1), make_float2(inv, inv));
      asm("{\n\t.reg .b16 a, b;\n\t"
          "cvt.rn.satfinite.e4m3x2.f32 a, %2, %1;\n\t"
          "cvt.rn.satfinite.e4m3x2.f32 b, %4, %3;\n\t"
          "mov.b32 %0, {a, b};\n\t}"
          : "=r"(w[i]) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
      if (s == 255u) w[i] = 0u;
    }
  }
  template <typename T>
  __device__ __forceinline__ void decode(uint32_t s, Vec8<T>& v) const {
    const float f = scale_value(s);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      uint32_t h0, h1;
      asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\t"
          "cvt.rn.f16x2.e4m3x2 %0, a;\n\t"
          "cvt.rn.f16x2.e4m3x2 %1, b;\n\t}"
          : "=r"(h0), "=r"(h1) : "r"(w[i]));
      v.set_pair(2 * i, mul2(__half22float2(*reinterpret_cast<const __half2*>(&h0)), make_float2(f, f)));
      v.set_pair(2 * i + 1, mul2(__half22float2(*reinterpret_cast<const __half2*>(&h1)), make_float2(f, f)));
    }
  }
  __device__ __forceinline__ void store(uint8_t* p) const { *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]); }
  __device__ __forceinline__ void load(const uint8_t* p) {
    const uint2 a = *reinterpret_cast<const uint2*>(p);
    w[0] = a.x; w[1] = a.y;
  }
};

// Programmatic dependent launch, used by every kernel here: a kernel may be scheduled while the one before it still runs, does
// what touches no memory, and waits for that kernel's end (and for all before it) with `wait_for_previous` before it reads or
// writes anything.  Only then does it allow its own successor to be scheduled, so that whatever a successor reads before its
// own wait can only have been written by the kernel directly before it.
__device__ __forceinline__ void wait_for_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void allow_next() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

struct LaunchConfig {
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute at[2];
  LaunchConfig(const LaunchConfig&) = delete;                 // (cfg points into it)
  LaunchConfig(cudaStream_t stream, int64_t ctas, int threads, int smem = 0, int cluster = 1) {
    cfg.gridDim = dim3((unsigned)ctas); cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = (size_t)smem; cfg.stream = stream;
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = (unsigned)cluster; at[1].val.clusterDim.y = 1; at[1].val.clusterDim.z = 1;
    cfg.attrs = at; cfg.numAttrs = cluster > 1 ? 2 : 1;
  }
};
template <typename... P, typename... A>
inline dq_status launch(const LaunchConfig& c, void (*kern)(P...), A&&... args) {
  return cudaLaunchKernelEx(&c.cfg, kern, static_cast<P>(args)...) == cudaSuccess ? DQ_OK : DQ_ERR_CUDA;
}

// Whether a matrix can be read and written in pieces of eight values: each row starts on a 16-byte boundary and ends with one.
inline bool whole_pieces(const void* p, int64_t ld, int64_t k, int dtype) {
  return ((uintptr_t)p & 15) == 0 && (ld * (dtype == DQ_FP32 ? 4 : 2)) % 16 == 0 && k % 8 == 0;
}

// What an entry point knows of the current device; 0 where it is none that the kernels were built for.
struct Device {
  int index = 0, sms = 0;
  int* d_status = nullptr;   // the operators' status word (dq_mx_status)
};
dq_status current_device(Device& out);

// dq_mx_quantize's work, used by dq_mx_linear too
dq_status quantize(cudaStream_t stream, const void* X, int x_dtype, int64_t rows, int64_t k, int64_t ldx, int fmt,
                   uint8_t* codes, uint8_t* scales, void* values, int64_t ldv);
dq_status dequantize(cudaStream_t stream, int fmt, const uint8_t* codes, const uint8_t* scales, int64_t rows, int64_t k,
                     void* Y, int y_dtype, int64_t ldy);
dq_status rmsnorm_quantize(cudaStream_t stream, const void* X, int dtype, int64_t rows, int64_t k, int64_t ldx,
                           const void* residual, int64_t ldr, const void* gamma, int gamma_dtype, float eps, int fmt,
                           uint8_t* codes, uint8_t* scales, void* sum, int64_t lds, void* values, int64_t ldv);
dq_status matmul(cudaStream_t stream, int a_fmt, const uint8_t* a_codes, const uint8_t* a_scales, int64_t m,
                 const uint8_t* w_codes, const uint8_t* w_scales, int64_t n, int64_t k, void* Y, int y_dtype, int64_t ldy);
// the product whose issuing warp gives up waiting at a pipeline step (dq_mx_selftest_bounded_wait)
dq_status matmul_giving_up(cudaStream_t stream, int a_fmt, const uint8_t* a_codes, const uint8_t* a_scales, int64_t m,
                           const uint8_t* w_codes, const uint8_t* w_scales, int64_t n, int64_t k, void* Y, int y_dtype, int64_t ldy,
                           int64_t step, uint64_t limit_ns);
dq_status linear(cudaStream_t stream, const void* X, int x_dtype, int64_t m, int64_t k, int64_t ldx, int a_fmt,
                 const uint8_t* w_codes, const uint8_t* w_scales, int64_t n, void* Y, int y_dtype, int64_t ldy,
                 uint8_t* workspace);

}  // namespace mx
}  // namespace dq
