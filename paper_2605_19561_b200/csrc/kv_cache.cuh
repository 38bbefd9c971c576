// A key/value cache in 4 bits: its pages, and the kernels that write new tokens into them and read tokens back.
//
// One page of one head holds page_tokens tokens:  key codes [page_tokens][D / 2] | key scale bytes [page_tokens][D / B] | value codes |
// value scale bytes, B = 32 (MXFP4, MXINT4) or 16 (NVFP4), codes and scale rules those of the library's quantizers.  Nothing is tiled or
// permuted: a page is written token by token and read by 16-byte pieces, and the attention kernels take their operands apart with
// ldmatrix, which wants whole rows.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include "mxint4_quantize.cuh"
#include "nvfp4_quantize.cuh"
#include "quantize.cuh"
#include "sm100_ptx.cuh"

namespace torq {

constexpr int kErrPage = 8;              // TORQ_ERR_PAGE

struct KvView {
  uint8_t* pages;
  const int32_t* table;                  // [batch][width]
  const int32_t* lengths;                // [batch], the new tokens included
  const int32_t* starts;                 // [batch + 1], or null: one new token each
  int batch, num_pages, width, page_shift, heads, dim, tokens;
  int head_bytes, k_scales, v_codes, v_scales;   // of one head's page; where its parts begin
  int64_t page_bytes;                    // of all heads
  float k_ts, v_ts;                      // NVFP4: tensor scales
  int* err_word;
};

__host__ __device__ constexpr int kv_block(int fmt) { return fmt == FMT_NVFP4 ? 16 : 32; }

__device__ __forceinline__ void kv_bad_page(const KvView& c) { atomicCAS(c.err_word, 0, kErrPage); }
// Tokens of sequence b in the cache.  A length that the table has no room for is an error; what has room is used.
__device__ __forceinline__ int kv_length(const KvView& c, int b) {
  const int n = c.lengths[b];
  const int64_t most = (int64_t)c.width << c.page_shift;
  if (n > most) kv_bad_page(c);
  return n < 0 ? 0 : (n > most ? (int)most : n);
}
// The new tokens of sequence b are rows [first, first + count) of the batch and its last ones in the cache.
__device__ __forceinline__ void kv_new_tokens(const KvView& c, int b, int& first, int& count) {
  if (!c.starts) {
    first = b;
    count = b < c.tokens ? 1 : 0;
    return;
  }
  const int lo = c.starts[b], hi = c.starts[b + 1];
  first = lo < 0 ? 0 : (lo > c.tokens ? c.tokens : lo);
  const int end = hi < first ? first : (hi > c.tokens ? c.tokens : hi);
  count = end - first;
}
// The sequence of row i, or -1: the last b with starts[b] <= i, if i lies before starts[b + 1].
__device__ __forceinline__ int kv_sequence_of(const KvView& c, int i) {
  if (!c.starts) return i < c.batch ? i : -1;
  int lo = 0, hi = c.batch;              // starts[lo] <= i < starts[hi], where that is so for 0 and batch
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (c.starts[mid] <= i) lo = mid;
    else hi = mid;
  }
  return c.starts[lo] <= i && i < c.starts[lo + 1] ? lo : -1;
}
// The page of token j of sequence b (j within the table's room), or -1 with the error latched.
__device__ __forceinline__ int kv_page(const KvView& c, const int32_t* table, int width, int b, int j) {
  const int page = table[(int64_t)b * width + (j >> c.page_shift)];
  if ((unsigned)page < (unsigned)c.num_pages) return page;
  kv_bad_page(c);
  return -1;
}
__device__ __forceinline__ uint8_t* kv_head_page(const KvView& c, int page, int head) {
  return c.pages + (int64_t)page * c.page_bytes + (int64_t)head * c.head_bytes;
}

// Eight values -> eight codes in a word; the lanes of a block (4, NVFP4: 2) agree on its scale byte.
template <int FMT>
__device__ __forceinline__ uint32_t kv_quantize8(const float (&v)[8], float tensor_scale, uint32_t& sbyte) {
  float amax = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) amax = fmaxf(amax, fabsf(v[i]));
  amax = fmaxf(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, 1));
  float r;
  if constexpr (FMT == FMT_NVFP4) {
    nv_block_scale(amax, nv_scale(tensor_scale), sbyte, r);
  } else {
    amax = fmaxf(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, 2));
    block_scale(amax, sbyte, r);
  }
  float q[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) q[i] = FMT == FMT_MXINT4 ? int4_round(__fmul_rn(v[i], r)) : __fmul_rn(v[i], r);
  if constexpr (FMT == FMT_MXINT4) return pack8_int4(q);
  return pack8_e2m1(q[0], q[1], q[2], q[3], q[4], q[5], q[6], q[7]);
}
// Eight codes -> the numbers without their scale.
template <int FMT>
__device__ __forceinline__ void kv_codes8(uint32_t w, float (&v)[8]) {
  if constexpr (FMT == FMT_MXINT4) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (float)(((int32_t)(w << (28 - 4 * i))) >> 28);
  } else {
    uint32_t h[4];
    asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\tmov.b32 {b0, b1, b2, b3}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, b0;\n\tcvt.rn.f16x2.e2m1x2 %1, b1;\n\tcvt.rn.f16x2.e2m1x2 %2, b2;\n\tcvt.rn.f16x2.e2m1x2 %3, b3;\n\t}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(w));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h[i]));
      v[2 * i] = f.x;
      v[2 * i + 1] = f.y;
    }
  }
}
// A scale byte as a number.  E8M0: 2^(byte - 127), byte 0 a subnormal.
template <int FMT>
__device__ __forceinline__ float kv_scale(uint32_t byte, float tensor_scale) {
  if constexpr (FMT == FMT_NVFP4) return __fmul_rn(e4m3_to_float(byte), tensor_scale);
  return __uint_as_float(byte ? byte << 23 : 0x00400000u);
}

__device__ __forceinline__ void kv_load8(const float* p, float (&v)[8]) {
  const uint4 a = load_once(p), b = load_once(p + 4);
  const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(w[i]);
}
__device__ __forceinline__ void kv_load8(const __nv_bfloat16* p, float (&v)[8]) {
  const uint4 a = load_once(p);
  const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(w[i] << 16);
    v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
  }
}

// Where the slots of TOKENS rows of the batch are, from row `first` on: the first thread of the CTA for each finds its page (its head 0), the others wait
// for it.  -1: no place.
struct KvSlot {
  int64_t page;                          // bytes from the beginning of the pages
  int slot;
};
template <int TOKENS>
__device__ __forceinline__ void kv_find_slots(const KvView& c, int first, KvSlot* slots) {
  if (threadIdx.x < TOKENS) {
    const int i = first + (int)threadIdx.x, b = i < c.tokens ? kv_sequence_of(c, i) : -1;
    KvSlot s = {-1, 0};
    if (b >= 0) {
      int row, count;
      kv_new_tokens(c, b, row, count);
      const int j = kv_length(c, b) - count + (i - row);
      if (j >= 0) {                      // a token before the start of its sequence (more new ones than its length) has no slot
        const int page = kv_page(c, c.table, c.width, b, j);
        if (page >= 0) s.page = page * c.page_bytes;
        s.slot = j & ((1 << c.page_shift) - 1);
      }
    }
    slots[threadIdx.x] = s;
  }
  __syncthreads();
}

// A CTA takes TOKENS new tokens at a time, all heads, keys and values; a thread eight elements of a row of each.  (A thread to eight elements anywhere, each
// finding its slot: 13040 tokens of 8 x 128 NVFP4 47 us.)
template <int FMT, typename T, int TOKENS>
__global__ void __launch_bounds__(256) kv_append_kernel(const KvView c, const T* K, const T* V, int64_t k_stride, int64_t v_stride) {
  griddep_wait_and_launch();
  __shared__ KvSlot slots[2][TOKENS];
  const int shift = 31 - __clz(c.dim / 8), work = 2 * c.heads << shift, lane = threadIdx.x & 31;
  int buffer = 0;
  for (int first = blockIdx.x * TOKENS; first < c.tokens; first += gridDim.x * TOKENS, buffer ^= 1) {
    bool found = false;
    for (int at = threadIdx.x; at - lane < work; at += 256) {
      const int e = at & ((1 << shift) - 1), head2 = at >> shift;
      const bool value = head2 >= c.heads;
      const int head = value ? head2 - c.heads : head2;
      const T* from = (value ? V : K) + head * c.dim + e * 8;
      const int64_t stride = value ? v_stride : k_stride;
      float v[TOKENS][8];
#pragma unroll
      for (int u = 0; u < TOKENS; ++u) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[u][i] = 0.f;
        if (at < work && first + u < c.tokens) kv_load8(from + (first + u) * stride, v[u]);
      }
      if (!found) kv_find_slots<TOKENS>(c, first, slots[buffer]);          // by all threads: the loops of all warps have a first turn
      found = true;
#pragma unroll
      for (int u = 0; u < TOKENS; ++u) {
        uint32_t sbyte;
        const uint32_t codes = kv_quantize8<FMT>(v[u], value ? c.v_ts : c.k_ts, sbyte);
        const KvSlot s = slots[buffer][u];
        if (s.page < 0 || at >= work) continue;          // the shuffles are behind
        uint8_t* p = c.pages + s.page + (int64_t)head * c.head_bytes;
        *reinterpret_cast<uint32_t*>(p + (value ? c.v_codes : 0) + s.slot * (c.dim / 2) + e * 4) = codes;
        constexpr int lanes = kv_block(FMT) / 8;
        if (e % lanes == 0) p[(value ? c.v_scales : c.k_scales) + s.slot * (c.dim / kv_block(FMT)) + e / lanes] = (uint8_t)sbyte;
      }
    }
    if (!found) kv_find_slots<TOKENS>(c, first, slots[buffer]);            // warps without work
  }
}

__device__ __forceinline__ void kv_store8(float* p, const float (&v)[8]) {
  reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
}
__device__ __forceinline__ void kv_store8(__nv_bfloat16* p, const float (&v)[8]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[i]) : "f"(v[2 * i + 1]), "f"(v[2 * i]));
  *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}

// The same slots read: rows [tokens][heads][dim] of both, zeros for a token without a slot.
template <int FMT, typename T, int TOKENS>
__global__ void __launch_bounds__(256) kv_read_kernel(const KvView c, T* K, T* V) {
  griddep_wait_and_launch();
  __shared__ KvSlot slots[2][TOKENS];
  const int shift = 31 - __clz(c.dim / 8), work = 2 * c.heads << shift;
  int buffer = 0;
  for (int first = blockIdx.x * TOKENS; first < c.tokens; first += gridDim.x * TOKENS, buffer ^= 1) {
    kv_find_slots<TOKENS>(c, first, slots[buffer]);
    for (int at = threadIdx.x; at < work; at += 256) {
      const int e = at & ((1 << shift) - 1), head2 = at >> shift;
      const bool value = head2 >= c.heads;
      const int head = value ? head2 - c.heads : head2;
      uint32_t codes[TOKENS], sbyte[TOKENS];
#pragma unroll
      for (int u = 0; u < TOKENS; ++u) {
        const KvSlot s = slots[buffer][u];
        codes[u] = sbyte[u] = 0;
        if (s.page < 0) continue;
        const uint8_t* p = c.pages + s.page + (int64_t)head * c.head_bytes;
        codes[u] = *reinterpret_cast<const uint32_t*>(p + (value ? c.v_codes : 0) + s.slot * (c.dim / 2) + e * 4);
        sbyte[u] = p[(value ? c.v_scales : c.k_scales) + s.slot * (c.dim / kv_block(FMT)) + e * 8 / kv_block(FMT)];
      }
      const float ts = value ? c.v_ts : c.k_ts;
      T* to = (value ? V : K) + ((int64_t)first * c.heads + head) * c.dim + e * 8;
#pragma unroll
      for (int u = 0; u < TOKENS; ++u) {
        if (first + u >= c.tokens) break;
        float v[8];
        kv_codes8<FMT>(codes[u], v);
        const float scale = kv_scale<FMT>(sbyte[u], 1.f);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = v[i] * scale * ts;              // code and scale byte multiply exactly
        kv_store8(to + (int64_t)u * c.heads * c.dim, v);
      }
    }
  }
}

}  // namespace torq
