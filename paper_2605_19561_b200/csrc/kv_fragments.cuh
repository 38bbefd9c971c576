// Operands of warp-level matrix instructions (m16n8k16, float16, sums in float32) from cached keys and values.
//
// Cached tokens are the rows of the instruction (m) and queries its columns (n = 8):  S^T = K Q^T,  then  O^T = V^T P^T  with features as rows.
// A row of codes in shared memory is D / 32 chunks of 16 bytes, 32 codes each.  ldmatrix on the packed codes hands lane (g, t) = (lane / 4, lane % 4)
// four bytes of a chunk of token g: eight codes, which become four pairs of float16, the A operands of two instructions.  Which code meets which
// k index does not matter as long as the queries' operand has the same order.  The transposing form hands it the two bytes (four codes) at place g of
// tokens 2t and 2t + 1: four pairs over tokens, again A operands, rows being features.  So nothing is moved between lanes and the cache keeps the
// plain layout.
// Chunks are swizzled so that the eight rows of an ldmatrix lie in different banks.
//
// Codes are exact in float16.  MXFP4 and MXINT4: a chunk is one scale block, so the products of a chunk get their scale (a power of two with
// float32's range) as float32; the values' scales are taken relative to the largest in their 32 features so far, 2^(e - E + 12) in float16, exact for
// scales down to 2^-26 of the largest (below they count as zero).  NVFP4: the codes times their E4M3 scale are exact in float16 (6 bits).
#pragma once
#include "kv_cache.cuh"

namespace torq {

template <int D>
__device__ __forceinline__ int kv_swizzled(int row, int chunk) {
  constexpr int CH = D / 32;
  return row * CH + (chunk ^ ((row / (8 / CH)) & (CH - 1)));
}
__device__ __forceinline__ void cp_async_16(uint32_t dst, const void* src, int bytes) {   // what is not copied of the 16 bytes becomes zero
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(__cvta_generic_to_global(src)), "r"(bytes) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void ldmatrix_x4(uint32_t saddr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(saddr) : "memory");
}
__device__ __forceinline__ void ldmatrix_x4_t(uint32_t saddr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(saddr) : "memory");
}
__device__ __forceinline__ uint32_t movmatrix_t(uint32_t v) {
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
// d = a b + c
__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1, const float (&c)[4]) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %11, %12, %13};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(c[0]), "f"(c[1]), "f"(c[2]), "f"(c[3]));
}
__device__ __forceinline__ float ex2(float v) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ uint32_t mul_f16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ uint32_t add_f16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("add.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ uint32_t fma_f16x2(uint32_t a, uint32_t b, uint32_t c) {
  uint32_t r;
  asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(c));
  return r;
}
// Two E4M3 bytes (the low ones of `bytes`) -> two float16.
__device__ __forceinline__ uint32_t e4m3x2_f16x2(uint32_t bytes) {
  uint32_t r;
  asm("{\n\t.reg .b16 t, u;\n\tmov.b32 {t, u}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, t;\n\t}" : "=r"(r) : "r"(bytes));
  return r;
}
// Integer nibbles: n ^ 8 = n + 8 in the mantissa of 1024 (or, four bits higher, sixteen times in it), and the offset taken off again.
__device__ __forceinline__ void int4_pairs(uint32_t w, uint32_t (&o)[4]) {
  const uint32_t x = w ^ 0x88888888u, y = x >> 8;
  const uint32_t off = 0xE408E408u, sixteenth = 0x2C002C00u, off16 = 0xD480D480u;      // -1032, 1 / 16, -72
  o[0] = add_f16x2((x & 0x000F000Fu) | 0x64006400u, off);
  o[1] = fma_f16x2((x & 0x00F000F0u) | 0x64006400u, sixteenth, off16);
  o[2] = add_f16x2((y & 0x000F000Fu) | 0x64006400u, off);
  o[3] = fma_f16x2((y & 0x00F000F0u) | 0x64006400u, sixteenth, off16);
}
// Eight codes of one token -> four pairs in the order of kv_query_order.
template <int FMT>
__device__ __forceinline__ void kv_key_pairs(uint32_t w, uint32_t (&o)[4]) {
  if constexpr (FMT == FMT_MXINT4) {
    int4_pairs(w, o);
  } else {
    asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\tmov.b32 {b0, b1, b2, b3}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, b0;\n\tcvt.rn.f16x2.e2m1x2 %1, b1;\n\tcvt.rn.f16x2.e2m1x2 %2, b2;\n\tcvt.rn.f16x2.e2m1x2 %3, b3;\n\t}"
        : "=r"(o[0]), "=r"(o[1]), "=r"(o[2]), "=r"(o[3]) : "r"(w));
  }
}
// The second element of pair i is element kv_query_order<FMT>(i, 1) of the eight.
template <int FMT>
__device__ constexpr int kv_query_order(int pair, int half) { return FMT == FMT_MXINT4 ? pair + 4 * half : 2 * pair + half; }

// Four codes of token 2t (low half) and of token 2t + 1 -> four pairs (code i of both).
template <int FMT>
__device__ __forceinline__ void kv_value_pairs(uint32_t u, uint32_t (&o)[4]) {
  if constexpr (FMT == FMT_MXINT4) {
    int4_pairs(u, o);
  } else {
    // byte 2 gets code 0 (odd: code 1) of both tokens, byte 3 code 2 (3); by products, since shifts run where the conversions do
    const uint32_t even = (u & 0x0F0F0F0Fu) * 0x00010010u, odd = (u & 0xF0F0F0F0u) * 0x00001001u;
    asm("{\n\t.reg .b8 b0, b1, b2, b3, c0, c1, c2, c3;\n\tmov.b32 {b0, b1, b2, b3}, %4;\n\tmov.b32 {c0, c1, c2, c3}, %5;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, b2;\n\tcvt.rn.f16x2.e2m1x2 %1, c2;\n\tcvt.rn.f16x2.e2m1x2 %2, b3;\n\tcvt.rn.f16x2.e2m1x2 %3, c3;\n\t}"
        : "=r"(o[0]), "=r"(o[1]), "=r"(o[2]), "=r"(o[3]) : "r"(even), "r"(odd));
  }
}

// Scale bytes of one token, `N` of them, from shared memory as words.
template <int N>
__device__ __forceinline__ void kv_scale_words(const uint8_t* p, uint32_t (&w)[(N + 3) / 4]) {
  if constexpr (N == 2) w[0] = *reinterpret_cast<const uint16_t*>(p);
  else if constexpr (N == 4) w[0] = *reinterpret_cast<const uint32_t*>(p);
  else if constexpr (N == 8) {
    const uint2 v = *reinterpret_cast<const uint2*>(p);
    w[0] = v.x;
    w[1] = v.y;
  } else {
    const uint4 v = *reinterpret_cast<const uint4*>(p);
    w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
  }
}
// Scales are made ready once per token, by the lane that has its number, instead of by every lane that needs them (eight for a value's, four for a
// key's), and kept beside the ring.  Keys: float32 per chunk; NVFP4: a pair of equal float16 per block, the blocks of even and of odd
// number apart (lane (g, t) needs block 2 c + t / 2).  Values: float16, tokens in the order 0 1 8 9 2 3 10 11 ... of every sixteen: the pairs that a
// lane needs lie together.
template <int FMT, int D>
struct KvScaleRoom {
  static constexpr int CH = D / 32, SB = D / kv_block(FMT);
  static constexpr int KEYS = 32 * SB * 4, VALUES = 32 * SB * 2, BYTES = KEYS + VALUES;
};
template <int N>
__device__ __forceinline__ void store_words(uint8_t* p, const uint32_t* w) {
  if constexpr (N == 2) *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
  else *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}
template <int N>
__device__ __forceinline__ void load_words(const uint8_t* p, uint32_t* w) {
  if constexpr (N == 2) {
    const uint2 v = *reinterpret_cast<const uint2*>(p);
    w[0] = v.x; w[1] = v.y;
  } else {
    const uint4 v = *reinterpret_cast<const uint4*>(p);
    w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
  }
}
// The scale bytes of key `token` of the 32 (E8M0 byte 0 counts as zero).  Queries are scaled up, so their products with a large key may pass float32 though
// the score does not.  Where a byte is 192 or more (2^65), which is seldom, all 32 keys are taken 2^(E - 191) times smaller, E the largest byte of the tokens
// that may be seen (`seen`: whether this one may; the others count as zero then), and the power of two to be multiplied back is returned, the same for all lanes.
// So the sums stay below 2^64 times 2^26, that of 256 products of a code (8 at most) and an element of a query (2^15).
template <int FMT, int D>
__device__ __forceinline__ float kv_ready_key_scales(const uint8_t* scales, int token, bool seen, uint8_t* room) {
  constexpr int CH = D / 32, SB = D / kv_block(FMT), V = CH < 4 ? CH : 4;
  uint32_t w[(SB + 3) / 4];
  kv_scale_words<SB>(scales + token * SB, w);
  float back = 1.f;
  if constexpr (FMT != FMT_NVFP4) {
    uint32_t high = 0;
#pragma unroll
    for (int i = 0; i < (SB + 3) / 4; ++i) high |= w[i] & w[i] << 1;
    if (__any_sync(0xFFFFFFFFu, (high & 0x80808080u) != 0)) {
      uint32_t most = 0;
#pragma unroll
      for (int i = 0; i < (SB + 3) / 4; ++i) {
        if (!seen) w[i] = 0;
        most = __vmaxu4(most, w[i]);
      }
      most = max(max(most & 0xFFu, most >> 8 & 0xFFu), max(most >> 16 & 0xFFu, most >> 24));
      const uint32_t top = __reduce_max_sync(0xFFFFFFFFu, most), down = top > 191u ? top - 191u : 0u;
#pragma unroll
      for (int i = 0; i < (SB + 3) / 4; ++i) w[i] = __vsubus4(w[i], down * 0x01010101u);
      back = __uint_as_float((127u + down) << 23);
    }
  }
  uint32_t even[CH], odd[CH];
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    if constexpr (FMT == FMT_NVFP4) {
      const uint32_t f = e4m3x2_f16x2(w[c / 2] >> (16 * (c & 1)));
      even[c] = __byte_perm(f, 0, 0x1010);
      odd[c] = __byte_perm(f, 0, 0x3232);
    } else {
      const int at = 8 * (c % 4);
      even[c] = (at < 24 ? w[c / 4] << (23 - at) : w[c / 4] >> 1) & 0x7F800000u;
    }
  }
#pragma unroll
  for (int c = 0; c < CH; c += V) {
    store_words<V>(room + (c / V * 32 + token) * (4 * V), even + c);
    if constexpr (FMT == FMT_NVFP4) store_words<V>(room + KvScaleRoom<FMT, D>::KEYS / 2 + (c / V * 32 + token) * (4 * V), odd + c);
  }
  return back;
}
// ... as lane t needs them.
template <int FMT, int D>
__device__ __forceinline__ void kv_key_scales(const uint8_t* room, int token, int t, uint32_t (&f)[D / 32]) {
  constexpr int CH = D / 32, V = CH < 4 ? CH : 4;
  if (FMT == FMT_NVFP4) room += (t >> 1) * (KvScaleRoom<FMT, D>::KEYS / 2);
#pragma unroll
  for (int c = 0; c < CH; c += V) load_words<V>(room + (c / V * 32 + token) * (4 * V), f + c);
}
__device__ __forceinline__ int kv_value_order(int token) { return (token & 16) | (token & 6) << 1 | (token & 8) >> 2 | (token & 1); }

// The queries' operand of a warp: lane (g, t) holds of row g the elements 32 c + 8 t ... + 7 of every chunk, as four registers.
template <int D>
struct KvQuery {
  uint32_t q[D / 32][4];
};
// A row into float16, times a power of two that brings its largest magnitude to [2^14, 2^15): float16 then keeps all bits of a
// bfloat16 down to 2^-21 of the largest, and nothing is off by more than 2^-39 of it.  Returns the factor to be multiplied back, of row g.
template <int FMT, int D>
__device__ __forceinline__ float kv_scale_query(const uint4 (&raw)[D / 32], KvQuery<D>& out) {
  uint32_t top = 0;
#pragma unroll
  for (int c = 0; c < D / 32; ++c)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t w = (&raw[c].x)[i] & 0x7FFF7FFFu;
      top = max(top, max(w >> 16, w & 0xFFFFu));
    }
  top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
  top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
  const uint32_t ef = top >> 7, field = ef > 15 ? 268u - ef : 253u;
  const float mul = __uint_as_float(field << 23);
#pragma unroll
  for (int c = 0; c < D / 32; ++c) {
    float v[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float((&raw[c].x)[i] << 16) * mul;
      v[2 * i + 1] = __uint_as_float((&raw[c].x)[i] & 0xFFFF0000u) * mul;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) out.q[c][i] = pack_f16(v[kv_query_order<FMT>(i, 0)], v[kv_query_order<FMT>(i, 1)]);
  }
  return __uint_as_float((254u - field) << 23);
}
// Row `p`, null: zeros.
template <int FMT, int D>
__device__ __forceinline__ float kv_load_query(const __nv_bfloat16* p, int t, KvQuery<D>& out) {
  uint4 raw[D / 32];
#pragma unroll
  for (int c = 0; c < D / 32; ++c) raw[c] = p ? load_once(p + 32 * c + 8 * t) : make_uint4(0, 0, 0, 0);
  return kv_scale_query<FMT, D>(raw, out);
}

// Scores of 16 cached tokens (rows first_row ... of the tile at `keys`, their scales made ready in `room`) with NT groups of eight queries:
// s[n][0, 1] token g, queries 2t and 2t + 1 of group n; s[n][2, 3] token g + 8.
template <int FMT, int D, int NT>
__device__ __forceinline__ void kv_tile_scores(uint32_t keys, const uint8_t* room, int first_row, int lane, const KvQuery<D> (&q)[NT], float (&s)[NT][4]) {
  constexpr int CH = D / 32;
  const int g = lane >> 2, t = lane & 3;
  uint32_t fa[CH], fb[CH];
  kv_key_scales<FMT, D>(room, first_row + g, t, fa);
  kv_key_scales<FMT, D>(room, first_row + g + 8, t, fb);
  const float zero[4] = {};
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int i = 0; i < 4; ++i) s[n][i] = 0.f;
#pragma unroll
  for (int c2 = 0; c2 < CH; c2 += 2) {
    uint32_t raw[4];
    ldmatrix_x4(keys + 16 * kv_swizzled<D>(first_row + (lane & 15), c2 + (lane >> 4)), raw);
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int c = c2 + e;
      uint32_t a[4], b[4];
      kv_key_pairs<FMT>(raw[2 * e], a);
      kv_key_pairs<FMT>(raw[2 * e + 1], b);
      if constexpr (FMT == FMT_NVFP4) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          a[i] = mul_f16x2(a[i], fa[c]);
          b[i] = mul_f16x2(b[i], fb[c]);
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          mma_f16(s[n], a[0], b[0], a[1], b[1], q[n].q[c][0], q[n].q[c][1], s[n]);
          mma_f16(s[n], a[2], b[2], a[3], b[3], q[n].q[c][2], q[n].q[c][3], s[n]);
        }
      } else {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          float x[4];
          mma_f16(x, a[0], b[0], a[1], b[1], q[n].q[c][0], q[n].q[c][1], zero);
          mma_f16(x, a[2], b[2], a[3], b[3], q[n].q[c][2], q[n].q[c][3], x);
          s[n][0] += x[0] * __uint_as_float(fa[c]);
          s[n][1] += x[1] * __uint_as_float(fa[c]);
          s[n][2] += x[2] * __uint_as_float(fb[c]);
          s[n][3] += x[3] * __uint_as_float(fb[c]);
        }
      }
    }
  }
}

}  // namespace torq
