// The 8-bit KV cache: block layout, code conversion and the per-call view of a step's rows, shared by
// the append and the attention kernels.
//
// A block is (layer, page of 16 tokens, KV head): 16 * DH e4m3 codes of K, 16 * DH of V, 32 bytes of
// scales.  Both parts are stored in the order in which a lane (g = lane / 4, t = lane % 4) of an
// m16n8k16 instruction needs them, so that a fragment is a 16-byte load from shared memory without
// bank conflicts:
//   K  [DH/64][16 tokens][64]: lane (g, t) takes 16 consecutive dimensions of token g and of token g + 8,
//      four k-steps' worth of rows g and g + 8 of the A operand (K is A, queries are B: the order of the
//      dimensions inside the contraction is free as long as both operands agree)
//   V  [DH/32][dim % 8][t][(dim % 32) / 8][tokens 2t, 2t+1, 2t+8, 2t+9]: lane (g, t) takes, for dimensions
//      g, g + 8, g + 16, g + 24 of 32, the four tokens that an A operand row (V^T) holds at columns
//      2t, 2t+1, 2t+8, 2t+9
#pragma once
#include <cuda_fp8.h>

#include "hb_internal.h"
#include "ptx.cuh"

namespace hb_kv8 {

constexpr int PAGE = 16;
constexpr int E_MIN = -32, E_MAX = 24;   // exponents of a block's scale

template <int DH>
struct Block {
  static constexpr int V_OFF = 16 * DH;
  static constexpr int HDR = 32 * DH;        // float scale of K, float scale of V
  static constexpr int BYTES = 32 * DH + 32; // a multiple of 32: blocks stay sector-aligned and 16-byte copies line up
};
inline size_t block_bytes(int dh) { return static_cast<size_t>(32 * dh + 32); }

// The step's rows and the cache, as the kernels see them.
struct Rows {
  const hb_seg* segs;
  const int32_t* page_ids;
  const int32_t* row_seg;
  int32_t n_segs, n_page_ids, n_rows, max_q_len, max_keys;
  int32_t n_pages, Hkv, G;
  uint8_t* arena;         // this layer's pages
  int64_t page_stride;    // bytes: Hkv blocks
  uint32_t* status;
};

// A segment's own fields agree with each other and with the bounds of the call (nothing it names lies
// outside the arrays); 64-bit sums, because the fields come from device memory unchecked.
__device__ __forceinline__ bool seg_ok(const Rows& r, int q_start, int q_len, int pos_start, int pt_start, int pt_len) {
  const long long keys = static_cast<long long>(pos_start) + q_len;
  return q_start >= 0 && q_len >= 0 && pos_start >= 0 && pt_start >= 0 && pt_len >= 0 &&
         static_cast<long long>(q_start) + q_len <= r.n_rows && q_len <= r.max_q_len && keys <= r.max_keys &&
         static_cast<long long>(pt_start) + pt_len <= r.n_page_ids && (keys + PAGE - 1) / PAGE <= pt_len;
}

// Four codes -> four fp16 (exact): low two -> lo, high two -> hi.
__device__ __forceinline__ void e4m3x4_to_half2x2(uint32_t w, uint32_t& lo, uint32_t& hi) {
  asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}"
      : "=r"(lo), "=r"(hi) : "r"(w));
}
// NaN in V.  A weight of zero does not keep a NaN out of a sum, so where a page holds keys that some rows must not
// see, NaN codes are replaced by zero and the rows that do see such a token become NaN as a whole (elsewhere
// NaN takes its way through the sum, into its own dimensions).
// Zeroes the NaN codes (0x7f, 0xff) of a word; returns a bit (the lowest) for each of its bytes that was one.
__device__ __forceinline__ uint32_t drop_nan(uint32_t& w) {
  const uint32_t bits = (((w & 0x7f7f7f7fu) + 0x01010101u) >> 7) & 0x01010101u;
  w &= ~(bits * 0xffu);
  return bits;
}
// The tokens of a page that the warp's lanes have found NaN in: bytes are tokens 2t, 2t+1, 2t+8, 2t+9; every lane gets bit
// `token` for each.
__device__ __forceinline__ uint32_t nan_tokens(uint32_t bytes, int t) {
  const uint32_t mine = ((bytes & 1u) | ((bytes >> 7) & 2u)) << (2 * t) | (((bytes >> 16) & 1u) | ((bytes >> 23) & 2u)) << (2 * t + 8);
  return __reduce_or_sync(0xffffffffu, mine);
}

// Two floats -> two codes (first in the low byte): round to nearest even, saturating, NaN stays NaN.
__device__ __forceinline__ uint32_t floats_to_e4m3x2(float a, float b) {
  uint32_t r;
  asm("{\n\t.reg .b16 c;\n\tcvt.rn.satfinite.e4m3x2.f32 c, %2, %1;\n\tcvt.u32.u16 %0, c;\n\t}" : "=r"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ uint32_t floats_to_e4m3x4(float a, float b, float c, float d) {
  return floats_to_e4m3x2(a, b) | (floats_to_e4m3x2(c, d) << 16);
}
// Smallest e with amax <= 448 * 2^e = 1.75 * 2^(e + 8), clamped; amax >= 0 and not NaN.
__device__ __forceinline__ int scale_exponent(float amax) {
  const uint32_t u = __float_as_uint(amax);
  const int e = static_cast<int>(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
  return max(E_MIN, min(E_MAX, e));   // zero and fp32 subnormals land on E_MIN
}
__device__ __forceinline__ float pow2f(int e) { return __uint_as_float(static_cast<uint32_t>(e + 127) << 23); }   // -126 <= e <= 127
__device__ __forceinline__ int exponent_of(float s) { return static_cast<int>((__float_as_uint(s) >> 23) & 0xffu) - 127; }

// Untiled bulk copy global -> shared memory, completing on an mbarrier.  16-byte aligned, a multiple of 16 bytes.
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
               ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
__device__ __forceinline__ uint4 lds128(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr));
  return v;
}

}  // namespace hb_kv8
