// Shared device code of the key/value cache in 4 bits (qk_rope.cu, kv_cache.cu, kv_attention.cu): where a slot lies, the codes'
// conversion, and how work over ragged sequences is cut into equal parts.
//
// A page holds page_size tokens of every kv head: [page][head][group of 16 tokens][bytes].  A group is
//     key codes [16][D / 2], key parameters [16] (scale, offset), value codes [16][D / 2], value parameters [16]
// with bf16 parameters and two codes a byte, the even dimension in the low half; value = offset + scale code.  A group is what a
// warp's matrix instruction takes at once, lies in one piece (16 (D + 8) bytes, a multiple of 128), and two neighbours of a page
// are one bulk copy whatever the page's size.
#pragma once
#include "mx_common.cuh"

namespace dq {
namespace kv {

constexpr int GROUP = 16;

inline __host__ __device__ int64_t group_bytes(int dim) { return (int64_t)GROUP * (dim + 8); }

struct Cache {
  uint8_t* pages;
  int64_t n_pages, page_bytes;   // bytes of a page of one head
  const int* table;              // [n_seqs][width]
  const int* lengths;
  int n_seqs, width, heads, shift;   // page_size == 1 << shift

  __device__ __forceinline__ int length(int b) const { return min(max(lengths[b], 0), width << shift); }
  // The page of one of a sequence's slots, -1 where the table names none.
  __device__ __forceinline__ int64_t page_of(int b, int slot) const {
    const int64_t page = table[(int64_t)b * width + (slot >> shift)];
    return page < 0 || page >= n_pages ? -1 : page;
  }
  __device__ __forceinline__ uint8_t* group_at(int64_t page, int h, int slot, int dim) const {
    return pages + (page * heads + h) * page_bytes + ((slot & ((1 << shift) - 1)) >> 4) * group_bytes(dim);
  }
};

// A tensor [token][head][dim] with contiguous values and strides counted in values.
struct Heads {
  void* p = nullptr;
  int64_t token = 0, head = 0;
  int heads = 0;
  int vec = 0;   // every head starts on a 16-byte boundary
};

// The tokens of a call: sequence b has those from starts[b] up to starts[b + 1], or `each` of them.
struct Batch {
  const int* starts;
  int64_t tokens;
  int each, n_seqs;
  __device__ __forceinline__ void range(int b, int64_t& first, int& n) const {
    if (!starts) { first = (int64_t)b * each; n = each; return; }
    first = min(max((int64_t)starts[b], (int64_t)0), tokens);
    n = (int)max(min((int64_t)starts[b + 1], tokens) - first, (int64_t)0);
  }
  // The sequence of a token, -1 if it belongs to none.
  __device__ __forceinline__ int sequence(int64_t t) const {
    if (!starts) return (int)(t / each);
    int lo = 0, hi = n_seqs + 1;             // the first start above t
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (starts[mid] <= t) lo = mid + 1; else hi = mid;
    }
    return lo == 0 || lo == n_seqs + 1 ? -1 : lo - 1;
  }
};

// The parameters' two bf16 numbers.
__device__ __forceinline__ float scale_of(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float offset_of(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// Work on a device that is cut into equal parts, one for each CTA: sequence b is cost(b) units long.
struct Share {
  int64_t total, lo, hi;   // all units, this CTA's
  int ctas;                // that have some
  int seq;                 // the sequence in which this CTA begins, and the units before it
  int64_t before;
};
// Quotients of non-negative numbers, mostly small ones (a 64-bit division is 70 instructions, a 32-bit one 20).
__device__ __forceinline__ int64_t quotient(int64_t a, int64_t b) {
  return (uint64_t)(a | b) >> 32 ? a / b : (int64_t)((uint32_t)a / (uint32_t)b);
}
// The CTA that has unit x: lo(i) = floor(i total / ctas).
__device__ __forceinline__ int cta_of(int64_t x, int64_t total, int ctas) { return (int)quotient((x + 1) * ctas - 1, total); }

// Two fp32 operations in one instruction.
using mx::add2;
using mx::mul2;
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("{\n\t.reg .b64 a, b, c, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmov.b64 c, {%6, %7};\n\tfma.rn.f32x2 d, a, b, c;\n\t"
      "mov.b64 {%0, %1}, d;\n\t}"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return d;
}
__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }

constexpr float LOG2E = 1.44269504088896f, LN2 = 0.693147180559945f;
__device__ __forceinline__ float exp2_of(float v) {
  float d;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(d) : "f"(v));
  return d;
}
__device__ __forceinline__ uint32_t half_pair(float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
// Two codes as fp16 numbers, c 2^-24: bits 0-3 and 16-19; c 2^-20: bits 4-7 and 20-23.
__device__ __forceinline__ uint32_t low_codes(uint32_t w) { return w & 0x000f000fu; }
__device__ __forceinline__ uint32_t high_codes(uint32_t w) { return w & 0x00f000f0u; }
// The same less 8.
__device__ __forceinline__ uint32_t less(uint32_t w, uint32_t eight) {
  const __half2 d = __hsub2(*reinterpret_cast<const __half2*>(&w), *reinterpret_cast<const __half2*>(&eight));
  return *reinterpret_cast<const uint32_t*>(&d);
}
__device__ __forceinline__ uint32_t low_centred(uint32_t w) { return less(low_codes(w), 0x00080008u); }
__device__ __forceinline__ uint32_t high_centred(uint32_t w) { return less(high_codes(w), 0x00800080u); }

// The share of this CTA, for all of its threads together.  `least`: units that are worth a CTA.
template <typename F>
__device__ __forceinline__ Share find_share(Share* out, int n_seqs, int64_t least, int64_t* warp_sums, F cost) {
  Share s{};
  auto take = [&](int64_t total) {
    s.total = total;
    s.ctas = (int)min((int64_t)gridDim.x, max((int64_t)1, quotient(total + least - 1, least)));
    const int64_t i = blockIdx.x;
    s.lo = i < s.ctas ? quotient(i * total, s.ctas) : 0;
    s.hi = i < s.ctas ? quotient((i + 1) * total, s.ctas) : 0;
  };
  const int tid = threadIdx.x, lane = tid & 31, threads = blockDim.x, warps = threads >> 5;
  auto upto = [&](int64_t sum) {                                        // the sum over the lanes up to this one
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int64_t v = __shfl_up_sync(0xffffffffu, sum, d);
      if (lane >= d) sum += v;
    }
    return sum;
  };
  if (n_seqs <= 32) {   // every warp for itself
    const int64_t c = lane < n_seqs ? cost(lane) : 0, sum = upto(c);
    take(__shfl_sync(0xffffffffu, sum, 31));
    const uint32_t votes = __ballot_sync(0xffffffffu, c > 0 && s.lo >= sum - c && s.lo < sum);
    s.seq = votes ? __ffs(votes) - 1 : 0;
    s.before = __shfl_sync(0xffffffffu, sum - c, s.seq);
    return s;
  }
  const int64_t once = tid < n_seqs ? cost(tid) : 0;   // (kept where there are no more sequences than threads)
  int64_t base = 0;
  for (int pass = 0; pass < 2; ++pass) {
    if (pass) {
      take(base);
      base = 0;
    }
    for (int b0 = 0; b0 < n_seqs; b0 += threads) {
      const int b = b0 + tid;
      const int64_t c = b0 == 0 ? once : b < n_seqs ? cost(b) : 0;
      const int64_t sum = upto(c);
      __syncthreads();
      if (lane == 31) warp_sums[tid >> 5] = sum;
      __syncthreads();
      int64_t all = 0, mine = 0;
      for (int w = 0; w < warps; ++w) {
        if (w == (tid >> 5)) mine = all;
        all += warp_sums[w];
      }
      if (pass && c > 0) {
        const int64_t begin = base + mine + sum - c;
        if (s.lo >= begin && s.lo < begin + c && s.lo < s.hi) { s.seq = b; s.before = begin; *out = s; }
      }
      base += all;
    }
  }
  if (tid == 0 && s.lo >= s.hi) { s.seq = 0; s.before = 0; *out = s; }
  __syncthreads();
  return *out;
}

inline bool pieces(const void* p, int64_t token, int64_t head, int dtype) {
  const int size = dtype == DQ_FP32 ? 4 : 2;
  return ((uintptr_t)p & 15) == 0 && token * size % 16 == 0 && head * size % 16 == 0;
}

template <typename F>
inline dq_status by_type(int dtype, F f) {
  if (dtype == DQ_BF16) return f(__nv_bfloat16());
  if (dtype == DQ_FP16) return f(__half());
  return f(float());
}
template <int N> struct Number { static constexpr int value = N; };
template <typename F>
inline dq_status by_dim(int dim, F f) {
  if (dim == 64) return f(Number<64>());
  if (dim == 128) return f(Number<128>());
  return f(Number<256>());
}

struct RopeArgs {
  Heads q, k, q_out, k_out;
  int64_t tokens;
  int dim, rot;
  const int* positions;
  const float* inv_freq;
  const void *q_gamma, *k_gamma;
  int gamma_fp32, gamma_vec, flags, splits;
  float eps;
};
dq_status rope(cudaStream_t stream, const mx::Device& dev, int dtype, const RopeArgs& a);

struct AppendArgs {
  Heads k, v, k_values, v_values;
  Cache cache;
  Batch batch;
  const int* positions;
  int* slot_positions;
  int64_t ld_slots;
};
dq_status append(cudaStream_t stream, const mx::Device& dev, int dtype, int dim, const AppendArgs& a);
dq_status dequantize(cudaStream_t stream, const mx::Device& dev, int dtype, int dim, const AppendArgs& a);   // k and v are written

struct AttentionArgs {
  Heads q, out;
  Cache cache;
  Batch batch;
  float scale;
  float* lse;              // [tokens][q heads]
  uint8_t* workspace;
  const float* weights;    // [n_seqs][kv heads][ld_slots]
  float* weights_out;
  int64_t ld_slots;
  int group, group_shift;  // query heads of a kv head; their logarithm, -1 if they are no power of two
  int* d_status;
  // the token of a kv head's query row: rows are (token, head of the group)
  __device__ __forceinline__ int token_of(int row) const { return group_shift >= 0 ? row >> group_shift : row / group; }
};
// dq_kv_attention's workspace: a counter for each CTA (zero between calls), then parts of items that several CTAs work on.
constexpr int MAX_SMS = 160, MAX_CTAS = 2 * MAX_SMS, TICKET_BYTES = MAX_CTAS * 4;
inline int64_t prompt_part(int dim) { return (int64_t)(dim == 256 ? 128 : 256) * (dim + 2); }   // floats of a part
int64_t attention_workspace(int dim);
// the same for many query rows a sequence
dq_status prompt_attention(cudaStream_t stream, const mx::Device& dev, int dtype, int dim, const AttentionArgs& a);
dq_status attention(cudaStream_t stream, const mx::Device& dev, int dtype, int dim, const AttentionArgs& a);
dq_status attention_weights(cudaStream_t stream, const mx::Device& dev, int dtype, int dim, const AttentionArgs& a);

struct EvictArgs {
  Cache cache;
  const float* weights;
  const int* positions;
  int64_t ld_slots;
  int keep, recent;
  float* weights_out;
  int* positions_out;
  int* lengths_out;
  int* workspace;
};
inline __host__ __device__ int64_t evict_stride(int keep) { return 4 + 2 * (int64_t)keep; }   // ints of a (sequence, head): the number of moves, (from, to)
dq_status evict(cudaStream_t stream, const mx::Device& dev, int dim, const EvictArgs& a);

}  // namespace kv
}  // namespace dq
