// Products with scales, bias, activation and residual in the epilogue (hb_linear), and the same with a weight per run of
// rows (hb_linear_grouped):  C = act(a_scale w_scale A W^T + bias) + residual.
//
// The products run on the tcgen05 tensor cores with the WEIGHT rows ("features") as the M side of the instruction and
// the rows of A ("tokens") as its N side: 128 features per CTA whatever the number of tokens, and N follows the tokens of
// the tile in steps of 16, so that one decode row costs one row's worth of loads and a group that ends inside a tile costs
// what it holds.  Operands are moved and multiplied as bytes: a k-block is 128 bytes of K (64 elements of 16
// bits, 128 of 8), a row of the 128-byte swizzle, and four instructions of 32 bytes each; only the instruction's kind differs.
//
//   warp 0   TMA: the tile's weight rows and token rows of one k-block per stage
//   warp 1   issues the MMAs; two accumulators in tensor memory where a CTA walks several tiles.  The whole warp walks the stages
//            and one elected thread issues: with one thread walking, the compiler has to prove the instructions' operands
//            uniform one by one, and a k-block of one CTA took 0.43 us instead of 0.20 (the 4096 x 28672 x 4096 case 435 -> 357 us).
//   others   epilogue: a warp takes 32 features x 32 tokens, a feature per lane, applies scales, bias and activation, adds the
//            residual that a TMA copy brought meanwhile, and sends the block out by another
//
//   CG = 2     a pair of CTAs per 256 x 256 tile (cta_group::2), persistent: many tokens
//   CG = 1     one CTA per 128 x BT tile; persistent, or a cluster of four or eight CTAs that share the tile's K range (few tiles):
//              each computes its share, hands the partial sums of the tokens of rank r to CTA r, which adds them in rank order
//   few rows   linear_narrow_kernel below
//
// What bounds it (one B200, 148 SMs): 4096 x 28672 x 4096 e4m3 with SwiGLU 310 - 330 us, 2.9 - 3.1 PFLOP/s, the tensor pipe and the
// power limit (a k-block takes 512 cycles of it); 64 rows of 28672 x 4096 e4m3 26 us and eight such weights 151 us, HBM
// (4.6 and 6.2 TB/s); 2048^3 fp16 onto fp32 28 us, one wave of tiles: filling, 32 k-blocks, and an epilogue that nothing hides.
//
// Groups: every CTA reads the bounds, drops those that are no good and numbers the token tiles of the others; a weight is a
// three-dimensional tensor map, so that a tile never sees the next group's rows.
#include <cuda_fp8.h>
#include <math.h>

#include <type_traits>

#include "hb_internal.h"
#include "ptx.cuh"

namespace {

constexpr int BF = 128;                 // features per CTA
constexpr int BKB = 128;                // bytes of K per k-block
constexpr int MAX_STAGES = 12;
// The tensor cores cut what falls off the end of a running sum, always towards zero: per instruction (32 bytes of K) 2^-26 of the sum where
// its terms have both signs, up to 2^-23.4 where they have one (fp16; K = 4096 in four shares: 5.9e-6).  So a chain of additions in one
// accumulator is bounded: where a whole tile is one CTA's, sums leave tensor memory after SEG_BLOCKS k-blocks and are added in registers
// (fp32 outputs; 16-bit outputs from KEEP_16 k-blocks on, where the loss comes near a fifth of their half step, 9e-5); tiles whose K is
// shared and the kernel for few rows are taken only where a share is at most KEEP_32 or KEEP_16 k-blocks (2.4e-5 at worst, or 9e-5).
constexpr int SEG_BLOCKS = 10;
constexpr int KEEP_32 = 64, KEEP_16 = 256;
constexpr uint64_t WAIT_LIMIT_NS = 2000000000ull;   // 2 s

struct LinArgs {
  hb_linear_args l;
  const int32_t* start;
  int32_t n_groups;
  int32_t f_tiles;       // tiles of BF * CG features
  int32_t k_blocks;
  int32_t band;          // token tiles walked together over all features
  int32_t stages;
  int32_t c_tma, res_tma;   // rows on 16-byte boundaries: the TMA moves whole blocks
  int32_t c_vec, res_vec;   // bytes of an access where it does not
  int32_t bufs, buf_bytes;  // blocks of results that an epilogue warp has in shared memory, and their size
  uint32_t* status;
};

// x Phi(x), with the complement of erf after Abramowitz and Stegun 7.1.26: erfc(u) = (a1 t + .. + a5 t^5) exp(-u^2), t = 1 / (1 + p u),
// u >= 0, off by at most 1.5e-7, which is 2^-23 |x| here (of GELU itself 0.2 % at x = -5 and 2 % at -10).  Half the instructions of erff, and no branches.
__device__ __forceinline__ float gelu(float x) {
  const float u = fabsf(x) * 0.70710678f, t = __fdividef(1.0f, fmaf(0.3275911f, u, 1.0f));
  float p = fmaf(1.061405429f, t, -1.453152027f);
  p = fmaf(p, t, 1.421413741f);
  p = fmaf(p, t, -0.284496736f);
  p = fmaf(p, t, 0.254829592f) * t;
  const float tail = 0.5f * p * __expf(-u * u);          // Phi(-|x|)
  return x * (x < 0.0f ? tail : 1.0f - tail);
}

// exp and division on the special-function unit: 2^-21 of |z| or less; an exponential that overflows gives the limit, 0.
template <int N, int SIZE>
__device__ __forceinline__ void activate(float (&z)[SIZE], int act) {
  switch (act) {
    case HB_ACT_RELU:
#pragma unroll
      for (int i = 0; i < N; ++i) z[i] = z[i] < 0.0f ? 0.0f : z[i];
      break;
    case HB_ACT_SILU:
#pragma unroll
      for (int i = 0; i < N; ++i) z[i] = __fdividef(z[i], 1.0f + __expf(-z[i]));
      break;
    case HB_ACT_GELU:
#pragma unroll
      for (int i = 0; i < N; ++i) z[i] = gelu(z[i]);
      break;
    case HB_ACT_GELU_TANH:   // (1 + tanh u) / 2 = 1 / (1 + e^-2u)
#pragma unroll
      for (int i = 0; i < N; ++i) z[i] = __fdividef(z[i], 1.0f + __expf(-1.5957691216f * (z[i] + 0.044715f * z[i] * z[i] * z[i])));
      break;
    default: break;
  }
}

// A warp's block of results, 32 features (one per lane) of 32 tokens, on its way out.  It is laid down in shared memory as
// [token][column] (16 columns where gated pairs became one) and leaves by one TMA copy; where rows of C or of the residual do not
// start on 16-byte boundaries, or the block holds rows of another group or the end of rows off such a boundary, the warp copies it
// with the widest accesses that the alignment allows.  The residual comes in the same way, into the same place, ahead of the sums.
struct Block {
  const LinArgs& a;
  char* mem;            // this block in shared memory, and its address there
  uint32_t buf;
  bool issuer;          // the thread that issues the warp's copies, and waits for them
  int lane, row0, tokens, col0;   // first row and how many are this group's; first output column

  __device__ __forceinline__ int width() const { return a.l.gated ? 16 : 32; }
  // columns that exist
  __device__ __forceinline__ int cols() const { return min(width(), (a.l.gated ? a.l.n >> 1 : a.l.n) - col0); }
  __device__ __forceinline__ bool whole() const { return tokens == 32 || row0 + tokens == a.l.m; }   // no row of another group

  template <int V>
  static __device__ __forceinline__ void copy_in(const char* g, uint32_t s, char* m) {
    if constexpr (V == 16) cp_async16(s, g, true);
    else if constexpr (V >= 4) cp_async_small<V>(s, g, true);
    else *reinterpret_cast<unsigned short*>(m) = *reinterpret_cast<const unsigned short*>(g);
  }
  // the block's rows, V bytes per lane and access, between shared memory and `base`
  template <int V, bool OUT>
  __device__ __forceinline__ void copy_v(char* base, int64_t stride_bytes, int size) const {
    const int shift = (a.l.gated ? 4 : 5) + (size == 4 ? 2 : 1) - (V == 16 ? 4 : V == 8 ? 3 : V == 4 ? 2 : 1);   // log2 of the lanes per row
    const int token = lane >> shift, at = (lane - (token << shift)) * V, step = 32 >> shift;   // first token, byte in its row, tokens per pass
    if (at >= cols() * size) return;        // (V divides the row's bytes)
    char* g = base + (row0 + token) * stride_bytes + col0 * size + at;
    using Small = typename std::conditional<V == 4, uint32_t, unsigned short>::type;
    using Vec = typename std::conditional<V == 16, uint4, typename std::conditional<V == 8, uint2, Small>::type>::type;
    int s = lane * V;
    stride_bytes *= step;
#pragma unroll 8
    for (int i = token; i < tokens; i += step, g += stride_bytes, s += 32 * V) {
      if constexpr (OUT) *reinterpret_cast<Vec*>(g) = *reinterpret_cast<const Vec*>(mem + s);
      else copy_in<V>(g, buf + s, mem + s);
    }
  }
  template <bool OUT>
  __device__ __forceinline__ void copy(void* base, int64_t stride, int dtype, int vec) const {
    const int size = dtype == HB_DTYPE_F32 ? 4 : 2;
    char* p = static_cast<char*>(base);
    if (vec == 16) copy_v<16, OUT>(p, stride * size, size);
    else if (vec == 8) copy_v<8, OUT>(p, stride * size, size);
    else if (vec == 4) copy_v<4, OUT>(p, stride * size, size);
    else copy_v<2, OUT>(p, stride * size, size);
  }

  // starts the residual's copy; `bar` is a barrier of this buffer
  __device__ __forceinline__ void fetch(const CUtensorMap* map, uint32_t bar) const {
    if (a.res_tma) {
      fence_async_smem();      // what the lanes did to the buffer comes before the copy
      __syncwarp();
      if (issuer) {
        mbar_arrive_expect_tx(bar, 32 * width() * (a.l.residual_dtype == HB_DTYPE_F32 ? 4 : 2));
        tma_load_2d(buf, map, bar, col0, row0);
      }
    } else {
      copy<false>(const_cast<void*>(a.l.residual), a.l.residual_stride, a.l.residual_dtype, a.res_vec);
      cp_async_commit();
    }
  }
  // element e of a lane is token e, or 2 e + (lane & 1) where pairs of lanes became one column (NE = 16)
  template <int NE, typename T>
  __device__ __forceinline__ T* place(int e) const {
    return reinterpret_cast<T*>(mem) + (NE == 32 ? e * 32 + lane : (2 * e + (lane & 1)) * 16 + (lane >> 1));
  }
  template <int NE>
  __device__ __forceinline__ void add_residual(float (&z)[32]) const {
    if (a.l.residual_dtype == HB_DTYPE_F32) {
#pragma unroll
      for (int e = 0; e < NE; ++e) z[e] += *place<NE, float>(e);
    } else {
      const bool bf16 = a.l.residual_dtype == HB_DTYPE_BF16;
#pragma unroll
      for (int e = 0; e < NE; ++e) {
        const unsigned short v = *place<NE, unsigned short>(e);
        z[e] += bf16 ? __uint_as_float(static_cast<uint32_t>(v) << 16) : __half2float(__ushort_as_half(v));
      }
    }
  }
  template <int NE>
  __device__ __forceinline__ void lay_down(const float (&z)[32]) const {
    if (a.l.c_dtype == HB_DTYPE_F32) {
#pragma unroll
      for (int e = 0; e < NE; ++e) *place<NE, float>(e) = z[e];
    } else {
      const bool bf16 = a.l.c_dtype == HB_DTYPE_BF16;
#pragma unroll
      for (int e = 0; e < NE; e += 2) {
        const uint32_t w = bf16 ? pack_bf16x2(z[e], z[e + 1]) : pack_f16x2_satfinite(z[e], z[e + 1]);
        *place<NE, unsigned short>(e) = static_cast<unsigned short>(w);
        *place<NE, unsigned short>(e + 1) = static_cast<unsigned short>(w >> 16);
      }
    }
  }
  // gate in the even lane, up in the odd one: afterwards z[0 .. 15] are gates and z[16 .. 31] ups, of the even tokens in the even
  // lane and of the odd ones in the odd lane
  __device__ __forceinline__ void pair(float (&z)[32]) const {
    float g[16], u[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      const float other = __shfl_xor_sync(0xffffffffu, lane & 1 ? z[2 * j] : z[2 * j + 1], 1);
      g[j] = lane & 1 ? other : z[2 * j];
      u[j] = lane & 1 ? z[2 * j + 1] : other;
    }
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      z[j] = g[j];
      z[16 + j] = u[j];
    }
  }
  // z = factor * token scale * sum + bias; `scales`: 32 floats of this warp in shared memory, this lane holds its token's in `as`
  __device__ __forceinline__ void scale(float (&z)[32], float factor, float bias, float as, float* scales) const {
    if (a.l.a_scale) {
      scales[lane] = as;
      __syncwarp();
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float4 q = *reinterpret_cast<const float4*>(scales + 4 * j);
        z[4 * j] = fmaf(z[4 * j], q.x * factor, bias);
        z[4 * j + 1] = fmaf(z[4 * j + 1], q.y * factor, bias);
        z[4 * j + 2] = fmaf(z[4 * j + 2], q.z * factor, bias);
        z[4 * j + 3] = fmaf(z[4 * j + 3], q.w * factor, bias);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 32; ++j) z[j] = fmaf(z[j], factor, bias);
    }
  }
  template <int NE, typename Arrived>
  __device__ __forceinline__ void compute(float (&z)[32], Arrived arrived) const {
    if constexpr (NE == 16) pair(z);
    activate<NE>(z, a.l.act);
    if constexpr (NE == 16) {
#pragma unroll
      for (int e = 0; e < NE; ++e) z[e] *= z[16 + e];
    }
    arrived();      // the residual, if there is one; if not, the buffer is free
    if (a.l.residual) {
      add_residual<NE>(z);
      __syncwarp();
    }
    lay_down<NE>(z);
  }
  template <typename Arrived>
  __device__ __forceinline__ void finish(float (&z)[32], float factor, float bias, float as, float* scales, const CUtensorMap* map,
                                         Arrived arrived) const {
    scale(z, factor, bias, as, scales);
    if (a.l.gated) compute<16>(z, arrived);
    else compute<32>(z, arrived);
    // (a copy's rows end on 16-byte boundaries, whatever the tensor map says of their length: it would write behind C's)
    if (a.c_tma && whole() && (cols() >= width() || cols() * (a.l.c_dtype == HB_DTYPE_F32 ? 4 : 2) % 16 == 0)) {
      fence_async_smem();
      __syncwarp();
      if (issuer) tma_store_2d(map, buf, col0, row0);
    } else {
      __syncwarp();
      copy<true>(a.l.c, a.l.c_stride, a.l.c_dtype, a.c_vec);
      __syncwarp();
    }
    if (issuer) tma_store_commit();   // one group per block, empty or not: waits count them
  }
};

// N tokens' values of a lane's feature, written where they belong (few tokens: no need for blocks).  Token e is row0 + e * step,
// the first `count` exist; as[e]: their scales.  All loads come before the first store, which might alias them.
template <int N>
__device__ __forceinline__ void finish_tokens(const hb_linear_args& l, float (&z)[N], const float (&as)[N], float factor, float bias, int row0,
                                              int step, int count, int feature, int lane) {
  const bool keep = feature < l.n && !(l.gated && (lane & 1));
  const int col = l.gated ? feature >> 1 : feature;
  float res[N];
#pragma unroll
  for (int e = 0; e < N; ++e) {
    res[e] = 0.0f;
    if (l.residual && keep && e < count) {
      const int64_t at = (row0 + e * step) * l.residual_stride + col;
      if (l.residual_dtype == HB_DTYPE_F32) res[e] = static_cast<const float*>(l.residual)[at];
      else if (l.residual_dtype == HB_DTYPE_BF16) res[e] = __bfloat162float(static_cast<const __nv_bfloat16*>(l.residual)[at]);
      else res[e] = __half2float(static_cast<const __half*>(l.residual)[at]);
    }
    z[e] = fmaf(z[e], as[e] * factor, bias);
  }
  if (l.gated) {
    float up[N];
#pragma unroll
    for (int e = 0; e < N; ++e) up[e] = __shfl_xor_sync(0xffffffffu, z[e], 1);
    activate<N>(z, l.act);
#pragma unroll
    for (int e = 0; e < N; ++e) z[e] *= up[e];
  } else {
    activate<N>(z, l.act);
  }
#pragma unroll
  for (int e = 0; e < N; ++e) {
    if (!keep || e >= count) continue;
    const int64_t at = (row0 + e * step) * l.c_stride + col;
    const float v = l.residual ? z[e] + res[e] : z[e];
    if (l.c_dtype == HB_DTYPE_F32) static_cast<float*>(l.c)[at] = v;
    else if (l.c_dtype == HB_DTYPE_BF16) static_cast<__nv_bfloat16*>(l.c)[at] = __float2bfloat16_rn(v);
    else static_cast<__half*>(l.c)[at] = __float2half_rn(sat_half_range(v));
  }
}

// Which tile an item is.  lo / pre: first row and first token tile of each group (a group that is dropped has none).
struct Tile {
  int group, row0, rows, feature_tile;
};
template <int BT>
__device__ __forceinline__ Tile tile_of(const LinArgs& a, const int* lo, const int* hi, const int* pre, int item) {
  int b = 0;
  if (a.n_groups > 1) {
    const int q = item / a.f_tiles;
    int e = a.n_groups;            // last group whose first tile is <= q
    while (e - b > 1) {
      const int mid = (b + e) >> 1;
      if (pre[mid] <= q) b = mid; else e = mid;
    }
  }
  const int tiles = pre[b + 1] - pre[b];
  int local = item - pre[b] * a.f_tiles, first = 0, height = tiles;
  if (a.band < tiles) {            // features over bands of token tiles, tokens fastest inside a band
    const int per_band = a.band * a.f_tiles, band = local / per_band;
    local -= band * per_band;
    first = band * a.band;
    height = min(a.band, tiles - first);
  }
  Tile t;
  t.group = b;
  t.feature_tile = local / height;
  t.row0 = lo[b] + (first + local - t.feature_tile * height) * BT;
  t.rows = min(BT, hi[b] - t.row0);
  return t;
}

// One warp fills the group table: bounds that start below an earlier bound, end before they start or leave the rows are dropped.
template <int BT>
__device__ __forceinline__ void number_tiles(const LinArgs& a, int lane, int* g_lo, int* g_hi, int* g_pre) {
  int most = 0, tiles_before = 0;
  for (int e0 = 0; e0 < a.n_groups; e0 += 32) {
    const int e = e0 + lane;
    int lo = 0, hi = a.l.m;
    if (a.start) {
      lo = e < a.n_groups ? a.start[e] : 0;
      hi = e < a.n_groups ? a.start[e + 1] : 0;
    }
    int before = max(lo, 0);     // the largest bound up to and with this one
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, before, o);
      if (lane >= o) before = max(before, v);
    }
    int earlier = __shfl_up_sync(0xffffffffu, before, 1);
    earlier = lane == 0 ? most : max(earlier, most);
    const bool good = lo >= earlier && hi >= lo && hi <= a.l.m;
    if (e < a.n_groups && !good && blockIdx.x == 0) atomicOr(a.status, HB_DEV_GROUP_BAD_INDEX);
    const int tiles = e < a.n_groups && good ? (hi - lo + BT - 1) / BT : 0;
    int sum = tiles;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, sum, o);
      if (lane >= o) sum += v;
    }
    if (e < a.n_groups) {
      g_lo[e] = lo;
      g_hi[e] = hi;
      g_pre[e] = tiles_before + sum - tiles;
    }
    most = max(most, __shfl_sync(0xffffffffu, before, 31));
    tiles_before += __shfl_sync(0xffffffffu, sum, 31);
  }
  if (lane == 0) g_pre[a.n_groups] = tiles_before;
}

// The four instructions of a k-block, 32 bytes of K each (+2 in the descriptors' address field); `fresh`: the sums start from nothing.
template <int CG, bool F8>
__device__ __forceinline__ void issue_block(uint32_t d, uint64_t wdesc, uint64_t adesc, uint32_t idesc, uint32_t fresh) {
#pragma unroll
  for (int k = 0; k < BKB / 32; ++k) {
    const uint32_t more = k == 0 ? fresh ^ 1u : 1u;
    if constexpr (CG == 2) {
      if constexpr (F8) umma_ss_f8_cg2(d, wdesc + 2u * k, adesc + 2u * k, idesc, more);
      else umma_ss_cg2(d, wdesc + 2u * k, adesc + 2u * k, idesc, more);
    } else {
      if constexpr (F8) umma_ss_f8(d, wdesc + 2u * k, adesc + 2u * k, idesc, more);
      else umma_ss(d, wdesc + 2u * k, adesc + 2u * k, idesc, more);
    }
  }
}

// How a persistent CTA's epilogue works.  PLAIN: 8 warps, a residual ahead.  LONG: tensor memory holds a tile's sums for SEG_BLOCKS k-blocks
// at a time, and registers (of 16 warps) add them up, where additions round; the pairs' 18 warps leave 96 registers a thread, of which two
// blocks of sums take 64, and some 300 bytes a thread are spilled.  SHORT: 16 warps, for products of so few k-blocks that the
// results bound them (4096 x 4096 x 64 fp16: 17.9 us, with 8 warps 19.8; at K = 4096 the 8 warps' larger ring wins by 2 %).
enum { PLAIN = 0, LONG = 1, SHORT = 2 };

template <int CG, int BT, int MODE>
struct Shape {
  static constexpr int TOKENS = BT / CG;                        // token rows a CTA holds per stage
  static constexpr int BOX = TOKENS < 64 ? TOKENS : 64;         // token rows per copy
  static constexpr int W_BYTES = BF * BKB;
  // epilogue warps: four per 32 tokens of the tile, up to 8 or 16; a warp has BT / 32 / PARTS blocks of 32 tokens
  static constexpr int MOST = MODE == PLAIN ? 8 : 16;
  static constexpr int EPI_WARPS = BT / 8 < MOST ? BT / 8 : MOST;
  static constexpr int PARTS = EPI_WARPS / 4;
  static constexpr int THREADS = 64 + EPI_WARPS * 32;
  // full, empty, tfull, tempty, one per buffer; two words; to a multiple of 32
  static constexpr int BAR_BYTES = 8 * (2 * MAX_STAGES + 4 + 2 * 16) + 8 + 24;
  static constexpr int SCALE_BYTES = EPI_WARPS * 32 * 4;
  static constexpr int STAGE_BYTES = W_BYTES + TOKENS * BKB;
};

// Adds 32 columns of one lane to z, 16 at a time: registers are short.
__device__ __forceinline__ void add_sums(uint32_t at, float (&z)[32]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    uint32_t r[16];
    tmem_ld16(at + static_cast<uint32_t>(i * 16), r);
    tmem_ld_wait();
#pragma unroll
    for (int j = 0; j < 16; ++j) z[i * 16 + j] += __uint_as_float(r[j]);
  }
}
__device__ __forceinline__ void read_sums(uint32_t at, float (&z)[32]) {
  tmem_ld32(at, reinterpret_cast<uint32_t(&)[32]>(z));
  tmem_ld_wait();
}

// SPLIT: the CTAs of a cluster share one tile's K range (CG = 1), two CTAs per SM; otherwise one persistent CTA per SM.
template <int CG, int BT, bool SPLIT, int MODE>
__global__ void __launch_bounds__(Shape<CG, BT, MODE>::THREADS, SPLIT ? 2 : 1)
linear_kernel(const __grid_constant__ CUtensorMap tm_w, const __grid_constant__ CUtensorMap tm_a, const __grid_constant__ CUtensorMap tm_c,
              const __grid_constant__ CUtensorMap tm_res, const LinArgs a) {
  using S = Shape<CG, BT, MODE>;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* smem_gen = smem_raw + (smem_base - smem_u32(smem_raw));
  const int stages = a.stages;
  const uint32_t cluster = cluster_nctarank();
  const uint32_t rank = cluster_ctarank();
  const int splits = SPLIT ? static_cast<int>(cluster) : 1;   // CTAs that share a tile's K range
  const bool leader = CG == 1 || rank == 0u;
  const int worker = static_cast<int>(blockIdx.x / cluster), n_workers = static_cast<int>(gridDim.x / cluster);
  // shared memory: stages, the epilogue's blocks and scales, barriers and two words, the group table
  const int stage_bytes = stages * S::STAGE_BYTES;
  const int out_bytes = SPLIT ? 0 : S::EPI_WARPS * a.bufs * a.buf_bytes + S::SCALE_BYTES;
  const uint32_t bar_base = smem_base + stage_bytes + out_bytes;
  uint8_t* bar_gen = smem_gen + stage_bytes + out_bytes;
  auto full_bar = [&](int s) { return bar_base + 8u * s; };
  auto empty_bar = [&](int s) { return bar_base + 8u * (MAX_STAGES + s); };
  auto tfull_bar = [&](int i) { return bar_base + 8u * (2 * MAX_STAGES + i); };
  auto tempty_bar = [&](int i) { return bar_base + 8u * (2 * MAX_STAGES + 2 + i); };
  auto buf_bar = [&](int i) { return bar_base + 8u * (2 * MAX_STAGES + 4 + i); };
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bar_gen + 8 * (2 * MAX_STAGES + 4 + 2 * 16));
  volatile uint32_t* abort_flag = tmem_slot + 1;
  int* g_lo = reinterpret_cast<int*>(bar_gen + S::BAR_BYTES);
  int* g_hi = g_lo + a.n_groups;
  int* g_pre = g_hi + a.n_groups;   // [n_groups + 1]
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  constexpr uint32_t tmem_cols = SPLIT ? BT : 2 * BT;   // one accumulator where a CTA has one tile

  if (threadIdx.x == 0) {
    for (int s = 0; s < stages; ++s) {
      mbar_init(full_bar(s), 1);
      mbar_init(empty_bar(s), 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(tfull_bar(i), 1);
      mbar_init(tempty_bar(i), S::EPI_WARPS * CG);
    }
    if constexpr (!SPLIT) {
      for (int i = 0; i < S::EPI_WARPS * a.bufs; ++i) mbar_init(buf_bar(i), 1);
    }
    *abort_flag = 0u;
    mbar_init_fence();
  }
  if (threadIdx.x == 32 * 2) {
    tma_prefetch_map(&tm_w);
    tma_prefetch_map(&tm_a);
  }
  if (warp == 1) {
    if constexpr (CG == 2) {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(tmem_cols) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(tmem_cols) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
  }
  // (what precedes touches this CTA's shared and tensor memory only and may run while the previous kernel drains)
  grid_dep_wait();
  if (warp == 2) number_tiles<BT>(a, lane, g_lo, g_hi, g_pre);
  tc_fence_before();
  __syncthreads();
  if (cluster > 1) cluster_sync();   // the peers' barriers are initialised before anything signals them
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  grid_dep_launch();
  const int total = g_pre[a.n_groups] * a.f_tiles;
  // this CTA's share of K
  const int kb0 = SPLIT ? static_cast<int>(static_cast<int64_t>(rank) * a.k_blocks / splits) : 0;
  const int kb1 = SPLIT ? static_cast<int>(static_cast<int64_t>(rank + 1) * a.k_blocks / splits) : a.k_blocks;
  // tokens of the MMA: the tile's, rounded up to what the instruction takes (and halves of the pair to its row groups)
  auto mma_n = [](int rows) { return CG == 2 ? (rows + 31) / 32 * 32 : (rows + 15) / 16 * 16; };

  auto give_up = [&]() {
    *abort_flag = 1u;
    if constexpr (CG == 2) st_cluster_u32(map_to_rank(smem_u32(const_cast<uint32_t*>(abort_flag)), rank ^ 1u), 1u);
  };

  if (warp == 0) {
    // ---------------- TMA producer ----------------
    // (the whole warp walks, one elected thread issues: see the MMA issuer)
    int stage = 0;
    uint32_t phase = 0;
    bool ok = true;
    const bool issuer = elect_one();
    for (int item = worker; ok && item < total; item += n_workers) {
      const Tile t = tile_of<BT>(a, g_lo, g_hi, g_pre, item);
      const int n = mma_n(t.rows) / CG;                       // token rows of this CTA
      const int boxes = __shfl_sync(0xffffffffu, (n + S::BOX - 1) / S::BOX, 0);
      const int f0 = __shfl_sync(0xffffffffu, (t.feature_tile * CG + (CG == 2 ? static_cast<int>(rank) : 0)) * BF, 0);
      const int r0 = __shfl_sync(0xffffffffu, t.row0 + (CG == 2 ? static_cast<int>(rank) * n : 0), 0);
      const int group = __shfl_sync(0xffffffffu, t.group, 0);
      const uint32_t bytes = static_cast<uint32_t>(S::W_BYTES + boxes * S::BOX * BKB);
      for (int kb = kb0; kb < kb1; ++kb) {
        ok = __all_sync(0xffffffffu, mbar_wait(empty_bar(stage), phase ^ 1u, abort_flag, WAIT_LIMIT_NS));
        if (!ok) { give_up(); break; }
        const uint32_t w_dst = smem_base + stage * S::STAGE_BYTES, a_dst = w_dst + S::W_BYTES;
        if (issuer) {
          if constexpr (CG == 2) {
            // the data of both CTAs is accounted on the leader's barrier
            const uint32_t bar = map_to_rank(full_bar(stage), 0u);
            if (leader) mbar_arrive_expect_tx(full_bar(stage), 2u * bytes);
            tma_load_3d_cg2(w_dst, &tm_w, bar, kb * BKB, f0, group);
            for (int b = 0; b < boxes; ++b) tma_load_2d_cg2(a_dst + b * S::BOX * BKB, &tm_a, bar, kb * BKB, r0 + b * S::BOX);
          } else {
            mbar_arrive_expect_tx(full_bar(stage), bytes);
            tma_load_3d(w_dst, &tm_w, full_bar(stage), kb * BKB, f0, group);
            for (int b = 0; b < boxes; ++b) tma_load_2d(a_dst + b * S::BOX * BKB, &tm_a, full_bar(stage), kb * BKB, r0 + b * S::BOX);
          }
        }
        __syncwarp();
        if (++stage == stages) { stage = 0; phase ^= 1u; }
      }
    }
    if (!ok) {
      // give copies already in flight time to land before shared memory is released
      for (int i = 0; i < 200; ++i) __nanosleep(1000);
    }
    __syncwarp();
  } else if (warp == 1) {
    // ---------------- MMA issuer (leader CTA only) ----------------
    // The whole warp walks the stages and one elected thread issues, so that what the instructions take from
    // uniform registers is uniform for the compiler too.
    if (leader) {
      int stage = 0, acc = 0;
      uint32_t phase = 0, acc_phase = 0;
      bool ok = true;
      const bool f8 = a.l.ab_dtype == HB_DTYPE_E4M3;
      const uint32_t format = a.l.ab_dtype == HB_DTYPE_BF16 ? (1u << 7 | 1u << 10) : 0u;   // bf16 operands; f16 and e4m3 are format 0 of their kinds
      const bool issuer = elect_one();
      bool ready = false;
      for (int item = worker; ok && item < total; item += n_workers) {
        const int rows = __shfl_sync(0xffffffffu, tile_of<BT>(a, g_lo, g_hi, g_pre, item).rows, 0);
        const uint32_t idesc = make_idesc_f16(BF * CG, mma_n(rows), false) | format;
        for (int seg0 = kb0; ok && seg0 < kb1; seg0 += MODE == LONG ? SEG_BLOCKS : kb1 - kb0) {
          const int seg1 = MODE == LONG ? min(seg0 + SEG_BLOCKS, kb1) : kb1;
          ok = __all_sync(0xffffffffu, mbar_wait(tempty_bar(acc), acc_phase ^ 1u, abort_flag, WAIT_LIMIT_NS));
          if (!ok) { give_up(); break; }
          tc_fence_after();
          const uint32_t d = __shfl_sync(0xffffffffu, tmem_base, 0) + static_cast<uint32_t>(acc * BT);
          for (int kb = seg0; kb < seg1; ++kb) {
            if (!ready) ok = __all_sync(0xffffffffu, mbar_wait(full_bar(stage), phase, abort_flag, WAIT_LIMIT_NS));
            if (!ok) { give_up(); break; }
            tc_fence_after();
            const uint32_t w_addr = smem_base + stage * S::STAGE_BYTES;
            const uint64_t wdesc = make_desc(w_addr, 16, 1024), adesc = make_desc(w_addr + S::W_BYTES, 16, 1024);
            const uint32_t done_bar = empty_bar(stage);
            // A look at the next stage's barrier costs over 100 cycles: it is under way while these products are issued.
            if (++stage == stages) { stage = 0; phase ^= 1u; }
            const bool next = mbar_test(full_bar(stage), phase);
            if (issuer) {
              const uint32_t fresh = kb == seg0 ? 1u : 0u;
              if (f8) issue_block<CG, true>(d, wdesc, adesc, idesc, fresh);
              else issue_block<CG, false>(d, wdesc, adesc, idesc, fresh);
              if constexpr (CG == 2) umma_commit_cg2(done_bar);
              else umma_commit(done_bar);
            }
            ready = __all_sync(0xffffffffu, next);
          }
          if (!ok) break;
          if (issuer) {
            if constexpr (CG == 2) umma_commit_cg2(tfull_bar(acc));
            else umma_commit(tfull_bar(acc));
          }
          __syncwarp();
          if (++acc == 2) { acc = 0; acc_phase ^= 1u; }
        }
      }
    }
    __syncwarp();
  } else if constexpr (!SPLIT) {
    // ---------------- epilogue ----------------
    const int quarter = warp & 3;            // tensor memory lanes [32 quarter, 32 quarter + 32) belong to this warp
    const int part = (warp - 2) >> 2;        // which blocks of 32 tokens
    const int ew = warp - 2;
    const uint32_t bufs = smem_base + stage_bytes + ew * a.bufs * a.buf_bytes;
    char* buf_mem = reinterpret_cast<char*>(smem_gen + stage_bytes + ew * a.bufs * a.buf_bytes);
    const bool issuer = elect_one();
    float* scales = reinterpret_cast<float*>(smem_gen + stage_bytes + S::EPI_WARPS * a.bufs * a.buf_bytes) + ew * 32;
    uint32_t buf_phase = 0;                  // a bit per buffer: parity of its next residual
    int buf = 0;
    bool fetched = false;                    // the residual of the next tile's first block is under way
    int acc = 0;
    uint32_t acc_phase = 0;
    bool ok = true;
    // this warp has read the accumulator: the next sums may go there
    auto release = [&]() {
      tc_fence_before();
      __syncwarp();
      if (lane == 0) {
        if constexpr (CG == 2) mbar_arrive_cluster(map_to_rank(tempty_bar(acc), 0u));
        else mbar_arrive(tempty_bar(acc));
      }
      if (++acc == 2) { acc = 0; acc_phase ^= 1u; }
    };
    auto wait_sums = [&]() {
      ok = __all_sync(0xffffffffu, mbar_wait(tfull_bar(acc), acc_phase, abort_flag, WAIT_LIMIT_NS));
      tc_fence_after();
    };
    auto feature_of = [&](const Tile& of) { return (of.feature_tile * CG + (CG == 2 ? static_cast<int>(rank) : 0)) * BF + quarter * 32; };
    Tile ahead = {};
    if (worker < total) ahead = tile_of<BT>(a, g_lo, g_hi, g_pre, worker);
    for (int item = worker; ok && item < total; item += n_workers) {
      const Tile t = ahead;
      ahead.rows = 0;                        // none
      if (item + n_workers < total) ahead = tile_of<BT>(a, g_lo, g_hi, g_pre, item + n_workers);
      const int f0 = feature_of(t);
      const bool mine = f0 + lane < a.l.n;
      const int64_t f_at = static_cast<int64_t>(t.group) * a.l.n + f0 + lane;
      const float factor = mine && a.l.w_scale ? a.l.w_scale[f_at] : 1.0f, bias = mine && a.l.bias ? a.l.bias[f_at] : 0.0f;
      auto block_at = [&](const Tile& tile, int feature, int c, int i) {
        return Block{a, buf_mem + i * a.buf_bytes, bufs + static_cast<uint32_t>(i * a.buf_bytes), issuer, lane, tile.row0 + c,
                     min(32, tile.rows - c), a.l.gated ? feature >> 1 : feature};
      };
      auto block_of = [&](int c, int i) { return block_at(t, f0, c, i); };
      // buffer i can be written: what was copied out of it has been read
      auto free_buffer = [&]() {
        if (issuer) {
          if (MODE == PLAIN) tma_store_wait_read<1>();   // (two buffers, or three where the next residual goes into one meanwhile)
          else tma_store_wait_read<0>();                 // (one, or two)
        }
        __syncwarp();
      };
      // the residual is in buffer i; without one the buffer is free
      auto arrived = [&](int i, bool newest) {
        if (!a.l.residual) {
          free_buffer();
        } else if (a.res_tma) {
          const bool got = mbar_wait(buf_bar(ew * a.bufs + i), (buf_phase >> i) & 1u, abort_flag, WAIT_LIMIT_NS);
          ok = __all_sync(0xffffffffu, got) && ok;
          buf_phase ^= 1u << i;
        } else {
          if (newest) cp_async_wait<0>(); else cp_async_wait<1>();
          __syncwarp();
        }
      };
      auto scale_of = [&](int c) { return a.l.a_scale && c + lane < t.rows ? a.l.a_scale[t.row0 + c + lane] : 1.0f; };
      // blocks of 32 tokens of this warp that exist
      const int pieces = f0 < a.l.n ? (t.rows - part * 32 + S::PARTS * 32 - 1) / (S::PARTS * 32) : 0;
      auto column = [&](int acc_i, int c) {
        return tmem_base + (static_cast<uint32_t>(quarter * 32) << 16) + static_cast<uint32_t>(acc_i * BT + c);
      };
      if constexpr (MODE == LONG) {
        constexpr int PIECES = BT / 32 / S::PARTS;
        float z[PIECES][32];
#pragma unroll
        for (int p = 0; p < PIECES; ++p)
#pragma unroll
          for (int j = 0; j < 32; ++j) z[p][j] = 0.0f;
        if (a.l.residual && pieces > 0) {
          free_buffer();
          block_of(part * 32, 0).fetch(&tm_res, buf_bar(ew));
        }
        for (int seg = kb0; seg < kb1; seg += SEG_BLOCKS) {
          wait_sums();
          if (!ok) { give_up(); break; }
#pragma unroll
          for (int p = 0; p < PIECES; ++p)
            if (p < pieces) add_sums(column(acc, (part + p * S::PARTS) * 32), z[p]);
          release();
        }
        if (!ok) break;
#pragma unroll
        for (int p = 0; p < PIECES; ++p) {
          if (p < pieces) {
            const int c = (part + p * S::PARTS) * 32;
            const Block o = block_of(c, 0);
            if (a.l.residual && p > 0) {
              free_buffer();
              o.fetch(&tm_res, buf_bar(ew));
            }
            o.finish(z[p], factor, bias, scale_of(c), scales, &tm_c, [&]() { arrived(0, true); });
          }
        }
        if (!__all_sync(0xffffffffu, ok)) { ok = false; give_up(); break; }
      } else {
        if (pieces <= 0) wait_sums();
        float as = scale_of(part * 32);
        // the residual of block c of tile `of` is under way while the sums before it are finished
        auto fetch_next = [&](const Tile& of, int feature, int c, int i) {
          free_buffer();
          block_at(of, feature, c, i).fetch(&tm_res, buf_bar(ew * a.bufs + i));
        };
        if (a.l.residual && pieces > 0 && !fetched) fetch_next(t, f0, part * 32, buf);
        fetched = false;
#pragma unroll 1
        for (int p = 0; p < pieces; ++p) {
          const int c = (part + p * S::PARTS) * 32, next = c + S::PARTS * 32, next_buf = buf + 1 == a.bufs ? 0 : buf + 1;
          float z[32];
          const float as_now = as;
          bool more = false;
          if (p + 1 < pieces) {
            as = scale_of(next);
            if (a.l.residual) {
              fetch_next(t, f0, next, next_buf);
              more = true;
            }
          } else if (a.l.residual && part * 32 < ahead.rows && feature_of(ahead) < a.l.n) {
            fetch_next(ahead, feature_of(ahead), part * 32, next_buf);
            more = fetched = true;
          }
          if (p == 0) wait_sums();
          if (!ok) break;
          read_sums(column(acc, c), z);
          if (p + 1 == pieces) release();
          block_of(c, buf).finish(z, factor, bias, as_now, scales, &tm_c, [&]() { arrived(buf, !more); });
          buf = next_buf;
        }
        if (pieces <= 0 && ok) release();
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) { give_up(); break; }
      }
    }
    if (issuer) tma_store_wait_all();        // shared memory stays until it has been read
  } else if (worker < total) {
    mbar_wait(tfull_bar(0), 0u, abort_flag, WAIT_LIMIT_NS);
    __syncwarp();
    tc_fence_after();
  }
  if constexpr (SPLIT) {
    // The partial sums [source][token][feature] of the tokens that a CTA finishes go where its stages were, once every CTA of the
    // cluster is through with them.  What the last step reads from global memory is read ahead.
    const bool busy = worker < total;
    Tile t = {};
    int per = 1, own = 0;                                     // tokens of each CTA, and of this one
    const int quarter = warp & 3, slot = (warp - 2) >> 2;     // epilogue warps: features, and every S::PARTS-th token from `slot`
    constexpr int AHEAD = 8;                                  // tokens finished at a time
    float factor = 1.0f, bias = 0.0f, as[AHEAD];
    int feature = 0, first = 0;                               // first row of this warp
    auto read_scales = [&](int i) {
#pragma unroll
      for (int e = 0; e < AHEAD; ++e) as[e] = a.l.a_scale && i + e * S::PARTS < own ? a.l.a_scale[first + (i + e * S::PARTS)] : 1.0f;
    };
    if (busy) {
      t = tile_of<BT>(a, g_lo, g_hi, g_pre, worker);
      per = (t.rows + splits - 1) / splits;
      own = min(per, t.rows - static_cast<int>(rank) * per);
      feature = t.feature_tile * BF + quarter * 32 + lane;
      const int64_t f_at = static_cast<int64_t>(t.group) * a.l.n + feature;
      if (warp >= 2 && feature < a.l.n) {
        if (a.l.w_scale) factor = a.l.w_scale[f_at];
        if (a.l.bias) bias = a.l.bias[f_at];
      }
      first = t.row0 + static_cast<int>(rank) * per;
      if (warp >= 2) read_scales(slot);
    }
    __syncthreads();
    cluster_sync();
    if (busy && warp >= 2) {
      const uint32_t mine = smem_base + (rank * per * BF + quarter * 32 + lane) * 4;
#pragma unroll 1
      for (int c = slot * 32; c < t.rows; c += S::PARTS * 32) {
        float r[32];
        read_sums(tmem_base + (static_cast<uint32_t>(quarter * 32) << 16) + static_cast<uint32_t>(c), r);
        int owner = c / per, at = c - owner * per;
        uint32_t to = map_to_rank(mine, owner);
#pragma unroll
        for (int j = 0; j < 32; ++j) {
          if (c + j < t.rows) {
            st_cluster_f32(to + at * BF * 4, r[j]);
            if (++at == per && c + j + 1 < t.rows) {
              at = 0;
              to = map_to_rank(mine, ++owner);
            }
          }
        }
      }
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync();
    if (busy && warp >= 2 && !*abort_flag) {
      const float* part = reinterpret_cast<const float*>(smem_gen) + quarter * 32 + lane;
      for (int i = slot; i < own; i += AHEAD * S::PARTS) {
        float z[AHEAD] = {};
        const int count = (own - i + S::PARTS - 1) / S::PARTS;
        for (int src = 0; src < splits; ++src)
#pragma unroll
          for (int e = 0; e < AHEAD; ++e)
            if (e < count) z[e] += part[(src * per + i + e * S::PARTS) * BF];
        if (i != slot) read_scales(i);
        finish_tokens<AHEAD>(a.l, z, as, factor, bias, first + i, S::PARTS, count, feature, lane);
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  // no CTA of a pair leaves (or frees tensor memory) while its peer may still read its shared memory or signal it
  if constexpr (CG == 2) cluster_sync();
  if (threadIdx.x == 0 && *abort_flag) atomicOr(a.status, HB_DEV_LINEAR_WAIT_EXPIRED);
  if (warp == 1) {
    tc_fence_after();
    if constexpr (CG == 2)
      asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(tmem_cols) : "memory");
    else
      asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(tmem_cols) : "memory");
  }
}

// ---- few tokens --------------------------------------------------------------------------------------
//
// A handful of rows is bound by the weight's bytes and by latency: a tensor memory tile costs some 2 us before and behind its
// products whatever it holds.  Here a block takes 16 MT features, its warps take every eighth 64 bytes of K, fragments are
// loaded straight from global memory (16 bytes of a row per lane: which byte of K meets which is the same for both operands, and
// their order is free), and the partial sums of the warps meet in shared memory in a fixed order.

constexpr int NARROW_WARPS = 8;

template <bool F8>
__device__ __forceinline__ void mma_16x8(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1, bool bf16) {
  if constexpr (F8) {
    asm volatile(
        "mma.sync.aligned.m16n8k32.row.col.f32.e4m3.e4m3.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  } else if (bf16) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  } else {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  }
}
// 16 bytes of a row at byte `at` of `k_bytes`; zeros behind its end and where there is no row.
template <bool STREAM>
__device__ __forceinline__ uint4 piece(const uint8_t* row, int at, int k_bytes) {
  uint4 q = make_uint4(0u, 0u, 0u, 0u);
  if (row == nullptr || at >= k_bytes) return q;
  if (at + 16 <= k_bytes) {
    if constexpr (STREAM) {
      asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(q.x), "=r"(q.y), "=r"(q.z), "=r"(q.w) : "l"(row + at));
    } else {
      q = *reinterpret_cast<const uint4*>(row + at);
    }
    return q;
  }
  uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
  for (int i = 0; i < 15; ++i)
    if (at + i < k_bytes) w[i / 4] |= static_cast<uint32_t>(row[at + i]) << (8 * (i & 3));
  return make_uint4(w[0], w[1], w[2], w[3]);
}

template <int MT, int NT, bool F8>
__global__ void __launch_bounds__(NARROW_WARPS * 32, 2) linear_narrow_kernel(const LinArgs a, int64_t w_group_bytes) {
  constexpr int BT = 8 * NT, FE = 16 * MT, STEPS = MT * NT == 1 ? 8 : MT * NT == 2 ? 4 : 2;   // 64-byte pieces under way
  extern __shared__ uint8_t smem_raw[];
  float* part = reinterpret_cast<float*>(smem_raw);                // [warp][token][feature]
  int* g_lo = reinterpret_cast<int*>(smem_raw + NARROW_WARPS * BT * FE * 4);
  int* g_hi = g_lo + a.n_groups;
  int* g_pre = g_hi + a.n_groups;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t4 = lane & 3;
  grid_dep_wait();
  grid_dep_launch();
  if (warp == 0) number_tiles<BT>(a, lane, g_lo, g_hi, g_pre);
  __syncthreads();
  if (static_cast<int>(blockIdx.x) >= g_pre[a.n_groups] * a.f_tiles) return;
  const Tile t = tile_of<BT>(a, g_lo, g_hi, g_pre, blockIdx.x);
  const hb_linear_args& l = a.l;
  const int size = F8 ? 1 : 2, k_bytes = l.k * size, f0 = t.feature_tile * FE;
  const bool bf16 = l.ab_dtype == HB_DTYPE_BF16;
  const uint8_t* wr[2 * MT];
  const uint8_t* ar[NT];
#pragma unroll
  for (int i = 0; i < 2 * MT; ++i) {
    const int f = f0 + 8 * i + g;
    wr[i] = f < l.n ? static_cast<const uint8_t*>(l.w) + t.group * w_group_bytes + f * l.w_stride * size : nullptr;
  }
#pragma unroll
  for (int i = 0; i < NT; ++i) ar[i] = 8 * i + g < t.rows ? static_cast<const uint8_t*>(l.a) + (t.row0 + 8 * i + g) * l.a_stride * size : nullptr;
  // what the last step reads from global memory, ahead of the products
  constexpr int PER_WARP = 32 / FE;        // tokens a warp finishes at a time, every STEP-th of them
  constexpr int STEP = NARROW_WARPS * PER_WARP, MINE = (BT + STEP - 1) / STEP;
  const int feature = f0 + lane % FE;
  const int64_t f_at = static_cast<int64_t>(t.group) * l.n + feature;
  const bool exists = feature < l.n;
  const float factor = exists && l.w_scale ? l.w_scale[f_at] : 1.0f, bias = exists && l.bias ? l.bias[f_at] : 0.0f;
  const int token0 = warp * PER_WARP + lane / FE;
  const int count = token0 < t.rows ? (t.rows - token0 + STEP - 1) / STEP : 0;
  float as[MINE];
#pragma unroll
  for (int e = 0; e < MINE; ++e) as[e] = l.a_scale && e < count ? l.a_scale[t.row0 + token0 + e * STEP] : 1.0f;
  float c[MT][NT][4] = {};
  for (int k0 = warp * 64; k0 < k_bytes; k0 += NARROW_WARPS * 64 * STEPS) {
    uint4 wq[STEPS][2 * MT], aq[STEPS][NT];
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      const int at = k0 + s * NARROW_WARPS * 64 + t4 * 16;
#pragma unroll
      for (int i = 0; i < 2 * MT; ++i) wq[s][i] = piece<true>(wr[i], at, k_bytes);
#pragma unroll
      for (int i = 0; i < NT; ++i) aq[s][i] = piece<false>(ar[i], at, k_bytes);
    }
#pragma unroll
    for (int s = 0; s < STEPS; ++s)
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          mma_16x8<F8>(c[m][n], wq[s][2 * m].x, wq[s][2 * m + 1].x, wq[s][2 * m].y, wq[s][2 * m + 1].y, aq[s][n].x, aq[s][n].y, bf16);
          mma_16x8<F8>(c[m][n], wq[s][2 * m].z, wq[s][2 * m + 1].z, wq[s][2 * m].w, wq[s][2 * m + 1].w, aq[s][n].z, aq[s][n].w, bf16);
        }
  }
  // lane (g, t4) holds features g and g + 8 of tokens 2 t4 and 2 t4 + 1
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        part[(warp * BT + 8 * n + 2 * t4 + (i & 1)) * FE + 16 * m + g + 8 * (i >> 1)] = c[m][n][i];
  __syncthreads();
  float z[MINE];
#pragma unroll
  for (int e = 0; e < MINE; ++e) {
    z[e] = 0.0f;
    if (token0 + e * STEP < BT)
#pragma unroll
      for (int w = 0; w < NARROW_WARPS; ++w) z[e] += part[(w * BT + token0 + e * STEP) * FE + lane % FE];
  }
  finish_tokens<MINE>(l, z, as, factor, bias, t.row0 + token0, STEP, count, feature, lane);
}

bool on(const void* p, int bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }

int check(const hb_ctx* c, const hb_linear_args* l) {
  if (!c || !l || l->m < 0 || l->n < 1 || l->k < 1) return HB_ERR_BAD_ARG;
  if (l->ab_dtype != HB_DTYPE_F16 && l->ab_dtype != HB_DTYPE_BF16 && l->ab_dtype != HB_DTYPE_E4M3) return HB_ERR_BAD_ARG;
  if (!hb_float_type(l->c_dtype) || (l->residual && !hb_float_type(l->residual_dtype))) return HB_ERR_BAD_ARG;
  if (l->act < HB_ACT_NONE || l->act > HB_ACT_GELU_TANH || (l->gated != 0 && l->gated != 1) || (l->gated && l->n % 2)) return HB_ERR_BAD_ARG;
  if (l->m > (1 << 26) || l->n > (1 << 26) || l->k > (1 << 26)) return HB_ERR_TOO_LARGE;
  const int ab = hb_elem_bytes(l->ab_dtype), cols = l->gated ? l->n / 2 : l->n;
  if (l->a_stride < l->k || l->w_stride < l->k || l->c_stride < cols || (l->residual && l->residual_stride < cols)) return HB_ERR_BAD_ARG;
  if (l->a_stride > (1ll << 36) || l->w_stride > (1ll << 36) || l->c_stride > (1ll << 36) || (l->residual && l->residual_stride > (1ll << 36)))
    return HB_ERR_TOO_LARGE;
  if (!on(l->a, 16) || !on(l->w, 16) || (l->a_stride * ab) % 16 || (l->w_stride * ab) % 16) return HB_ERR_BAD_ARG;
  if (!on(l->c, hb_elem_bytes(l->c_dtype)) || (l->residual && !on(l->residual, hb_elem_bytes(l->residual_dtype))) || !on(l->a_scale, 4) ||
      !on(l->w_scale, 4) || !on(l->bias, 4))
    return HB_ERR_BAD_ARG;
  if (l->m > 0 && (!l->a || !l->w || !l->c)) return HB_ERR_BAD_ARG;
  return HB_OK;
}

// Largest access (up to 16 bytes) that fits the rows' alignment and length.
int row_vector(const void* p, int64_t stride, int size, int cols) {
  int v = 16;
  while (v > size && (!on(p, v) || (stride * size) % v || (static_cast<int64_t>(cols) * size) % v)) v /= 2;
  return v;
}

template <int CG, int BT, bool SPLIT, int MODE>
int launch_as(const hb_linear_args& l, LinArgs a, int splits, int num_sms, int64_t w_group_stride, cudaStream_t s, bool pdl) {
  using S = Shape<CG, BT, MODE>;
  const int ab = hb_elem_bytes(l.ab_dtype);
  CUtensorMap tw, ta;
  const uint64_t k_bytes = static_cast<uint64_t>(l.k) * ab;
  int rc = hb_tmap_bytes(&tw, l.w, k_bytes, l.n, a.n_groups, l.w_stride * ab, (a.start ? w_group_stride : l.w_stride) * ab, BKB, BF);
  if (rc != HB_OK) return rc;
  if ((rc = hb_tmap_bytes(&ta, l.a, k_bytes, l.m, 0, l.a_stride * ab, 0, BKB, S::BOX)) != HB_OK) return rc;
  a.f_tiles = (l.n + BF * CG - 1) / (BF * CG);
  // tokens fastest over a band of at most 30 MB of A, which stays in L2 while the features pass
  const int64_t band = (30ll << 20) / (static_cast<int64_t>(BT) * static_cast<int64_t>(k_bytes));
  a.band = static_cast<int>(band < 1 ? 1 : band > (1 << 20) ? (1 << 20) : band);
  const int64_t token_tiles = (l.m + BT - 1) / BT + (a.start ? (a.n_groups < l.m ? a.n_groups : l.m) : 0);   // at most
  const int64_t items = token_tiles * a.f_tiles;
  if (items > (1ll << 30)) return HB_ERR_TOO_LARGE;
  const int table = 4 * (3 * a.n_groups + 1);
  // results: TMA copies where rows start on 16-byte boundaries
  const int width = l.gated ? 16 : 32, cols = l.gated ? l.n / 2 : l.n;
  const int cs = hb_elem_bytes(l.c_dtype), rs = l.residual ? hb_elem_bytes(l.residual_dtype) : 0;
  CUtensorMap tc = ta, tr = ta;
  if constexpr (!SPLIT) {
    a.c_vec = row_vector(l.c, l.c_stride, cs, cols);
    a.c_tma = on(l.c, 16) && (l.c_stride * cs) % 16 == 0;
    if (a.c_tma && (rc = hb_tmap_block(&tc, l.c, l.c_dtype, cols, l.m, l.c_stride * cs, width, 32)) != HB_OK) return rc;
    if (l.residual) {
      a.res_vec = row_vector(l.residual, l.residual_stride, rs, cols);
      a.res_tma = on(l.residual, 16) && (l.residual_stride * rs) % 16 == 0;
      if (a.res_tma && (rc = hb_tmap_block(&tr, l.residual, l.residual_dtype, cols, l.m, l.residual_stride * rs, width, 32)) != HB_OK) return rc;
    }
  }
  a.bufs = (MODE == PLAIN ? 2 : 1) + (MODE != LONG && l.residual ? 1 : 0);
  a.buf_bytes = 32 * width * (cs > rs ? cs : rs);
  const int fixed = 1024 + S::BAR_BYTES + (SPLIT ? 0 : S::EPI_WARPS * a.bufs * a.buf_bytes + S::SCALE_BYTES) + table;
  const int room = (SPLIT ? 113 : 227) * 1024;
  a.stages = (room - fixed) / S::STAGE_BYTES;
  if (a.stages > MAX_STAGES) a.stages = MAX_STAGES;
  const int smem = fixed + a.stages * S::STAGE_BYTES;
  static DynSmemState configured;
  auto kern = linear_kernel<CG, BT, SPLIT, MODE>;
  if (hb_ensure_dyn_smem(reinterpret_cast<const void*>(kern), configured, smem) != HB_OK) return HB_ERR_CUDA;
  int64_t workers = items;
  if (!SPLIT && workers > num_sms / CG) workers = num_sms / CG;
  cudaLaunchConfig_t cfg = {};
  const int cluster = CG == 2 ? 2 : splits;
  cfg.gridDim = dim3(static_cast<unsigned>(workers * cluster));
  cfg.blockDim = dim3(S::THREADS);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = cluster;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = pdl ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kern, tw, ta, tc, tr, a) == cudaSuccess ? HB_OK : HB_ERR_CUDA;
}

template <int MT, int NT, bool F8>
int launch_narrow_as(const hb_linear_args& l, LinArgs a, int64_t w_group_stride, cudaStream_t s, bool pdl) {
  constexpr int BT = 8 * NT, FE = 16 * MT;
  a.f_tiles = (l.n + FE - 1) / FE;
  a.band = 1 << 20;
  const int64_t items = ((l.m + BT - 1) / BT + (a.start ? (a.n_groups < l.m ? a.n_groups : l.m) : 0)) * static_cast<int64_t>(a.f_tiles);
  if (items > (1ll << 30)) return HB_ERR_TOO_LARGE;
  const int smem = NARROW_WARPS * BT * FE * 4 + 4 * (3 * a.n_groups + 1);
  return hb_launch_kernel(linear_narrow_kernel<MT, NT, F8>, static_cast<unsigned>(items), NARROW_WARPS * 32, smem, s, pdl, a,
                          w_group_stride * static_cast<int64_t>(F8 ? 1 : 2));
}
template <int MT, int NT>
int launch_narrow(const hb_linear_args& l, const LinArgs& a, int64_t w_group_stride, cudaStream_t s, bool pdl) {
  return l.ab_dtype == HB_DTYPE_E4M3 ? launch_narrow_as<MT, NT, true>(l, a, w_group_stride, s, pdl)
                                     : launch_narrow_as<MT, NT, false>(l, a, w_group_stride, s, pdl);
}

int k_blocks_of(const hb_linear_args& l) { return static_cast<int>((static_cast<int64_t>(l.k) * hb_elem_bytes(l.ab_dtype) + BKB - 1) / BKB); }

// How the epilogue of an unshared tile of `tokens` works.
int mode_of(const hb_linear_args& l, int k_blocks, int tokens) {
  if (k_blocks > (l.c_dtype == HB_DTYPE_F32 ? SEG_BLOCKS : KEEP_16)) return LONG;
  return tokens >= 128 && k_blocks <= (tokens == 128 ? 8 : 12) ? SHORT : PLAIN;
}

template <int CG, int BT, bool SPLIT>
int launch(const hb_linear_args& l, const LinArgs& a, int splits, int num_sms, int64_t w_group_stride, cudaStream_t s, bool pdl) {
  if constexpr (!SPLIT) {
    const int mode = mode_of(l, a.k_blocks, BT);
    if (mode == LONG) return launch_as<CG, BT, SPLIT, LONG>(l, a, splits, num_sms, w_group_stride, s, pdl);
    if constexpr (BT >= 128) {
      if (mode == SHORT) return launch_as<CG, BT, SPLIT, SHORT>(l, a, splits, num_sms, w_group_stride, s, pdl);
    }
  }
  return launch_as<CG, BT, SPLIT, PLAIN>(l, a, splits, num_sms, w_group_stride, s, pdl);
}

// Which kernel: tokens of a tile (8, 16: linear_narrow_kernel; 32 .. 128: one CTA per tile; 256: a pair), and `share`: 16-feature
// blocks of a narrow tile, or the CTAs that share a tile's K.
struct Variant {
  int tokens, share;
  float us, own;   // the estimate, and the same without what every variant waits for, the weights
};

// Each variant's time in microseconds from the sizes, with what was measured on a B200 (n, k from 300 x 1000 to 28672 x 4096 and
// 1024 x 8192, 1 to 4000 rows, both operand widths); the least wins.  What it decides, both sides measured (us):
//   8 rows, 2048 x 2048, 16 bits    narrow 5.2, one CTA per tile 11.3, four per tile 9.5
//   8 rows, 28672 x 4096, 8 bits    narrow 31.6, one CTA per tile 26.6, pairs 28.0
//   64 rows, 28672 x 4096, 8 bits   one CTA per tile of 64 27.3, pairs 28.7
//   64 rows, 1024 x 8192, 16 bits   narrow 19.0, one CTA per tile 31.1, eight per tile 13.7
//   300 rows, 4096 x 4096, 16 bits  128 tokens 21.4, pairs 27.5
//   2000 rows, 4096 x 4096, 16 bits 128 tokens 69.2, pairs 52.4
Variant pick_variant(const hb_linear_args& l, int n_groups, int k_blocks, bool grouped, int sms) {
  const int groups = n_groups < l.m ? n_groups : l.m;                       // at most so many have rows
  const float rows = static_cast<float>(l.m) / groups, k_bytes = k_blocks * static_cast<float>(BKB);
  const float weight_us = groups * k_bytes * l.n / 5.9e6f;                   // the weights' bytes at 5.9 TB/s
  // token tiles; groups end anywhere, half a tile each is left over
  auto token_tiles = [&](int bt) {
    if (!grouped) return static_cast<float>((l.m + bt - 1) / bt);
    const float t = static_cast<float>(l.m) / bt + 0.5f * groups;
    return t > groups ? t : static_cast<float>(groups);
  };
  auto ceil_div = [](float x, float y) { return ceilf(x / y); };
  Variant best = {256, 1, 1e30f, 1e30f};
  auto offer = [&](int tokens, int share, float us, float own) {
    if (us < best.us || (us == best.us && own < best.own)) best = {tokens, share, us, own};
  };
  const int keep = l.c_dtype == HB_DTYPE_F32 ? KEEP_32 : KEEP_16;            // k-blocks in one accumulator, at most
  if (rows <= 64.0f && k_blocks <= NARROW_WARPS * keep) {
    for (int nt = 1; nt <= 2; ++nt)
      for (int mt = 1; mt <= 2; ++mt) {
        const float blocks = ceil_div(l.n, 16 * mt) * token_tiles(8 * nt);
        const float rounds = ceil_div(k_bytes, 512.0f * (mt * nt == 1 ? 8 : mt * nt == 2 ? 4 : 2));   // of loads that wait for each other
        const float waves = ceil_div(blocks, 2 * sms);
        const float latency = rounds * (mt * nt == 1 ? 2.1f : mt * nt == 2 ? 1.7f : 1.4f), bytes = blocks * (16 * mt + 8 * nt) * k_bytes / 6e6f;
        const float us = 1.0f + waves * (1.0f + mt) + (waves * latency > bytes ? waves * latency : bytes);
        offer(8 * nt, mt, us, us);
      }
  }
  const bool f8 = l.ab_dtype == HB_DTYPE_E4M3;
  for (int bt = 32; bt <= 256; bt *= 2) {
    if (bt > 32 && bt < 256 && rows <= bt / 2) continue;                     // a smaller tile holds them
    if (bt < 128 && rows > 4 * bt) continue;
    const float features = ceil_div(l.n, bt == 256 ? 2 * BF : BF), tiles = features * token_tiles(bt);
    const float block_us = bt <= 64 ? 0.205f : bt == 128 ? (f8 ? 0.25f : 0.22f) : 0.28f;   // a k-block's products
    const float out_us = bt == 32 ? 0.9f : bt == 64 ? 1.25f : bt == 128 ? 2.0f : 4.0f;      // a tile's epilogue
    const float main_us = k_blocks * block_us, waves = ceil_div(tiles, bt == 256 ? sms / 2 : sms);
    const float us = 4.2f + main_us + out_us + (waves - 1.0f) * (main_us > out_us ? main_us : out_us);
    offer(bt, 1, us > weight_us + 4.5f ? us : weight_us + 4.5f, us);   // (of several bound by the weights: the one with most to spare)
    if (bt == 256) break;
    for (int s = 4; s <= 8 && s <= k_blocks; s *= 2) {                         // (two never paid)
      const float ctas = tiles * s, held = rows < bt ? rows : static_cast<float>(bt);
      if (ctas > 2 * sms) break;                                               // all at once, two per SM, or not at all
      if (ceil_div(k_blocks, s) > keep) continue;
      const float share_us = ceil_div(k_blocks, s) * (ctas > sms ? 0.45f : 0.3f);
      const float split_us = share_us > weight_us ? share_us : weight_us;
      const float split = 7.8f + split_us + held / 128.0f * (2.0f + 12.0f / s);
      offer(bt, s, split, split);
    }
  }
  return best;
}

}  // namespace

extern "C" int hb_linear_variant(const hb_linear_args* l, int32_t n_groups, int32_t num_sms, int32_t* out) {
  if (!l || !out || l->m < 1 || l->n < 1 || l->k < 1 || n_groups < 0 || num_sms < 1) return HB_ERR_BAD_ARG;
  if (l->m > (1 << 26) || l->n > (1 << 26) || l->k > (1 << 26) || n_groups > HB_LINEAR_MAX_GROUPS) return HB_ERR_TOO_LARGE;
  const int k_blocks = k_blocks_of(*l);
  const Variant v = pick_variant(*l, n_groups > 0 ? n_groups : 1, k_blocks, n_groups > 0, num_sms);
  out[0] = v.tokens;
  out[1] = v.share;
  out[2] = v.tokens >= 32 && v.share == 1 ? mode_of(*l, k_blocks, v.tokens) : PLAIN;
  return HB_OK;
}

int hb_launch_linear(hb_ctx* c, const hb_linear_args& l, const int32_t* group_start, int n_groups, int64_t w_group_stride,
                     cudaStream_t s, bool pdl) {
  LinArgs a = {};
  a.l = l;
  a.start = group_start;
  a.n_groups = n_groups;
  a.status = c->status;
  a.k_blocks = k_blocks_of(l);
  const int sms = c->num_sms;
  const Variant v = pick_variant(l, n_groups, a.k_blocks, group_start != nullptr, sms);
  switch (v.tokens * 10 + v.share) {
    case 81: return launch_narrow<1, 1>(l, a, w_group_stride, s, pdl);
    case 82: return launch_narrow<2, 1>(l, a, w_group_stride, s, pdl);
    case 161: return launch_narrow<1, 2>(l, a, w_group_stride, s, pdl);
    case 162: return launch_narrow<2, 2>(l, a, w_group_stride, s, pdl);
    case 321: return launch<1, 32, false>(l, a, 1, sms, w_group_stride, s, pdl);
    case 641: return launch<1, 64, false>(l, a, 1, sms, w_group_stride, s, pdl);
    case 1281: return launch<1, 128, false>(l, a, 1, sms, w_group_stride, s, pdl);
    case 2561: return launch<2, 256, false>(l, a, 1, sms, w_group_stride, s, pdl);
    default: break;
  }
  if (v.tokens == 32) return launch<1, 32, true>(l, a, v.share, sms, w_group_stride, s, pdl);
  if (v.tokens == 64) return launch<1, 64, true>(l, a, v.share, sms, w_group_stride, s, pdl);
  return launch<1, 128, true>(l, a, v.share, sms, w_group_stride, s, pdl);
}

extern "C" int hb_linear(hb_ctx* c, const hb_linear_args* l, void* stream) {
  int rc = check(c, l);
  if (rc != HB_OK || l->m == 0) return rc;
  if ((rc = hb_wrong_device(c)) != HB_OK) return rc;
  return hb_launch_linear(c, *l, nullptr, 1, 0, static_cast<cudaStream_t>(stream), false);
}

extern "C" int hb_linear_grouped(hb_ctx* c, const hb_linear_args* l, const int32_t* group_start, int32_t n_groups,
                                 int64_t w_group_stride, void* stream) {
  int rc = check(c, l);
  if (rc != HB_OK) return rc;
  if (n_groups < 1 || !on(group_start, 4) || w_group_stride < static_cast<int64_t>(l->n - 1) * l->w_stride + l->k) return HB_ERR_BAD_ARG;
  if (n_groups > HB_LINEAR_MAX_GROUPS || w_group_stride > (1ll << 36)) return HB_ERR_TOO_LARGE;
  if ((w_group_stride * hb_elem_bytes(l->ab_dtype)) % 16) return HB_ERR_BAD_ARG;
  if (l->m == 0) return HB_OK;
  if (!group_start) return HB_ERR_BAD_ARG;
  if ((rc = hb_wrong_device(c)) != HB_OK) return rc;
  return hb_launch_linear(c, *l, group_start, n_groups, w_group_stride, static_cast<cudaStream_t>(stream), false);
}
