// Products with scales, bias, activation and residual in the epilogue (hb_linear), and the same with a weight per run of
// rows (hb_linear_grouped):  C = act(a_scale w_scale A W^T + bias) + residual.
//
// The products run on the tcgen05 tensor cores with the WEIGHT rows ("features") as the M side of the instruction and
// the rows of A ("tokens") as its N side: 128 features per CTA whatever the number of tokens, and N follows the tokens of
// the tile in steps of 16, so that one decode row costs one row's worth of loads and a group that ends inside a tile costs
// what it holds.  Operands are moved and multiplied as bytes: a k-block is 128 bytes of K (64 elements of 16
// bits, 128 of 8), a row of the 128-byte swizzle, and four instructions of 32 bytes each; only the instruction's kind differs.
//
//   warp 0     TMA: the tile's weight rows and token rows of one k-block per stage
//   warp 1     one thread issues the MMAs; accumulators in tensor memory, two of them where a CTA walks several tiles
//   warps 2-9  epilogue: a warp reads 32 features x 32 tokens, turns them through shared memory, and finishes four adjacent
//              features of a token per thread
//
//   CG = 2     a pair of CTAs per 256 x 256 tile (cta_group::2), persistent: many tokens
//   CG = 1     one CTA per 128 x BT tile; persistent, or a cluster of S CTAs that share the tile's K range (few tiles): each
//              computes its share, hands the partial sums of the tokens of rank r to CTA r, which adds them in rank order
//
// Groups: every CTA reads the bounds, drops those that are no good and numbers the token tiles of the others; a weight is a
// three-dimensional tensor map, so that a tile never sees the next group's rows.
#include <cuda_fp8.h>

#include "hb_internal.h"
#include "ptx.cuh"

namespace {

constexpr int BF = 128;                 // features per CTA
constexpr int BKB = 128;                // bytes of K per k-block
constexpr int NUM_THREADS = 320;
constexpr int EPI_WARPS = 8;
constexpr int MAX_STAGES = 8;
constexpr int STG_PITCH = 36;           // floats between tokens in a warp's staging block (16 tokens x 32 features)
constexpr int STG_BYTES = EPI_WARPS * 16 * STG_PITCH * 4;
constexpr int BAR_BYTES = 256;
constexpr uint64_t WAIT_LIMIT_NS = 2000000000ull;   // 2 s

struct LinArgs {
  hb_linear_args l;
  const int32_t* start;
  int32_t n_groups;
  int32_t f_tiles;       // tiles of BF * CG features
  int32_t k_blocks;
  int32_t band;          // token tiles walked together over all features
  int32_t stages;
  int32_t wide;          // outputs and residual in vectors
  uint32_t* status;
};

__device__ __forceinline__ float activate(float z, int act) {
  switch (act) {
    case HB_ACT_RELU: return z != z ? z : fmaxf(z, 0.0f);
    case HB_ACT_SILU: return z / (1.0f + __expf(-z));
    case HB_ACT_GELU: return 0.5f * z * (1.0f + erff(z * 0.70710678f));
    case HB_ACT_GELU_TANH: return z / (1.0f + __expf(-1.5957691216f * (z + 0.044715f * z * z * z)));   // (1 + tanh u) / 2 = 1 / (1 + e^-2u)
    default: return z;
  }
}

// N (2 or 4) consecutive values of a row, as vectors or one by one up to `valid`.
template <int N>
__device__ __forceinline__ void read_values(const void* p, int64_t at, int dtype, bool wide, int valid, float (&v)[N]) {
  if (dtype == HB_DTYPE_F32) {
    const float* q = static_cast<const float*>(p) + at;
    if (wide) {
      if constexpr (N == 4) {
        const float4 f = *reinterpret_cast<const float4*>(q);
        v[0] = f.x; v[1] = f.y; v[2] = f.z; v[3] = f.w;
      } else {
        const float2 f = *reinterpret_cast<const float2*>(q);
        v[0] = f.x; v[1] = f.y;
      }
      return;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = i < valid ? q[i] : 0.0f;
    return;
  }
  uint32_t w[N / 2];
  const unsigned short* q = static_cast<const unsigned short*>(p) + at;
  if (wide) {
#pragma unroll
    for (int i = 0; i < N / 2; ++i) w[i] = 0u;
    if constexpr (N == 4) {
      const uint2 u = *reinterpret_cast<const uint2*>(q);
      w[0] = u.x; w[1] = u.y;
    } else {
      w[0] = *reinterpret_cast<const uint32_t*>(q);
    }
  } else {
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
      w[i] = 2 * i < valid ? q[2 * i] : 0u;
      if (2 * i + 1 < valid) w[i] |= static_cast<uint32_t>(q[2 * i + 1]) << 16;
    }
  }
#pragma unroll
  for (int i = 0; i < N / 2; ++i) {
    if (dtype == HB_DTYPE_BF16) {
      v[2 * i] = __uint_as_float(w[i] << 16);
      v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    } else {
      const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
      v[2 * i] = f.x;
      v[2 * i + 1] = f.y;
    }
  }
}
template <int N>
__device__ __forceinline__ void write_values(void* p, int64_t at, int dtype, bool wide, int valid, const float (&v)[N]) {
  if (dtype == HB_DTYPE_F32) {
    float* q = static_cast<float*>(p) + at;
    if (wide) {
      if constexpr (N == 4) *reinterpret_cast<float4*>(q) = make_float4(v[0], v[1], v[2], v[3]);
      else *reinterpret_cast<float2*>(q) = make_float2(v[0], v[1]);
      return;
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (i < valid) q[i] = v[i];
    return;
  }
  uint32_t w[N / 2];
#pragma unroll
  for (int i = 0; i < N / 2; ++i) {
    if (dtype == HB_DTYPE_BF16) {
      const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&b);
    } else {
      w[i] = pack_half2_sat(v[2 * i], v[2 * i + 1]);
    }
  }
  unsigned short* q = static_cast<unsigned short*>(p) + at;
  if (wide) {
    if constexpr (N == 4) *reinterpret_cast<uint2*>(q) = make_uint2(w[0], w[1]);
    else *reinterpret_cast<uint32_t*>(q) = w[0];
    return;
  }
#pragma unroll
  for (int i = 0; i < N; ++i)
    if (i < valid) q[i] = static_cast<unsigned short>(w[i / 2] >> (16 * (i & 1)));
}

// Four adjacent features: their factors and biases, read once per tile, and what is done with a token's four sums.
struct Features {
  float scale[4], bias[4];
  int f0, valid;      // first feature; how many of the four exist
  __device__ __forceinline__ void init(const hb_linear_args& l, int group, int f) {
    f0 = f;
    valid = min(4, l.n - f);
    const int64_t at = static_cast<int64_t>(group) * l.n + f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      scale[i] = i < valid && l.w_scale ? l.w_scale[at + i] : 1.0f;
      bias[i] = i < valid && l.bias ? l.bias[at + i] : 0.0f;
    }
  }
  __device__ __forceinline__ void finish(const LinArgs& a, int row, float (&acc)[4]) const {
    const hb_linear_args& l = a.l;
    if (valid <= 0) return;
    const float as = l.a_scale ? l.a_scale[row] : 1.0f;
    const bool wide = a.wide != 0;
    float z[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) z[i] = fmaf(acc[i], as * scale[i], bias[i]);
    if (l.gated) {
      float v[2] = {activate(z[0], l.act) * z[1], activate(z[2], l.act) * z[3]};
      if (l.residual) {
        float r[2];
        read_values<2>(l.residual, row * l.residual_stride + f0 / 2, l.residual_dtype, wide, valid / 2, r);
        v[0] += r[0];
        v[1] += r[1];
      }
      write_values<2>(l.c, row * l.c_stride + f0 / 2, l.c_dtype, wide, valid / 2, v);
    } else {
      float v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = activate(z[i], l.act);
      if (l.residual) {
        float r[4];
        read_values<4>(l.residual, row * l.residual_stride + f0, l.residual_dtype, wide, valid, r);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] += r[i];
      }
      write_values<4>(l.c, row * l.c_stride + f0, l.c_dtype, wide, valid, v);
    }
  }
};

// Which tile an item is.  lo / pre: first row and first token tile of each group (a group that is dropped has none).
struct Tile {
  int group, row0, rows, feature_tile;
};
template <int BT>
__device__ __forceinline__ Tile tile_of(const LinArgs& a, const int* lo, const int* hi, const int* pre, int item) {
  const int q = item / a.f_tiles;
  int b = 0, e = a.n_groups;     // last group whose first tile is <= q
  while (e - b > 1) {
    const int mid = (b + e) >> 1;
    if (pre[mid] <= q) b = mid; else e = mid;
  }
  const int tiles = pre[b + 1] - pre[b];
  const int local = item - pre[b] * a.f_tiles;
  // features over bands of token tiles, tokens fastest inside a band
  const int per_band = a.band * a.f_tiles;
  const int band = local / per_band, in_band = local - band * per_band;
  const int height = min(a.band, tiles - band * a.band);
  Tile t;
  t.group = b;
  t.feature_tile = in_band / height;
  t.row0 = lo[b] + (band * a.band + in_band - t.feature_tile * height) * BT;
  t.rows = min(BT, hi[b] - t.row0);
  return t;
}

template <int CG, int BT>
struct Shape {
  static constexpr int TOKENS = BT / CG;                        // token rows a CTA holds per stage
  static constexpr int BOX = TOKENS < 64 ? TOKENS : 64;         // token rows per copy
  static constexpr int W_BYTES = BF * BKB;
  static constexpr int STAGE_BYTES = W_BYTES + TOKENS * BKB;
};

template <int CG, int BT>
__global__ void __launch_bounds__(NUM_THREADS, CG == 2 ? 1 : 2)
linear_kernel(const __grid_constant__ CUtensorMap tm_w, const __grid_constant__ CUtensorMap tm_a, const LinArgs a) {
  using S = Shape<CG, BT>;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* smem_gen = smem_raw + (smem_base - smem_u32(smem_raw));
  const int stages = a.stages;
  const uint32_t cluster = cluster_nctarank();
  const uint32_t rank = cluster_ctarank();
  const int splits = CG == 2 ? 1 : static_cast<int>(cluster);   // CTAs that share a tile's K range
  const bool leader = CG == 1 || rank == 0u;
  const int worker = static_cast<int>(blockIdx.x / cluster), n_workers = static_cast<int>(gridDim.x / cluster);
  // shared memory: stages, barriers and two words, the epilogue's staging blocks, the group table
  const uint32_t bar_base = smem_base + stages * S::STAGE_BYTES;
  uint8_t* bar_gen = smem_gen + stages * S::STAGE_BYTES;
  auto full_bar = [&](int s) { return bar_base + 8u * s; };
  auto empty_bar = [&](int s) { return bar_base + 8u * (MAX_STAGES + s); };
  auto tfull_bar = [&](int i) { return bar_base + 8u * (2 * MAX_STAGES + i); };
  auto tempty_bar = [&](int i) { return bar_base + 8u * (2 * MAX_STAGES + 2 + i); };
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bar_gen + 8 * (2 * MAX_STAGES + 4));
  volatile uint32_t* abort_flag = tmem_slot + 1;
  float* staging = reinterpret_cast<float*>(bar_gen + BAR_BYTES);
  int* g_lo = reinterpret_cast<int*>(bar_gen + BAR_BYTES + (splits > 1 ? 0 : STG_BYTES));
  int* g_hi = g_lo + a.n_groups;
  int* g_pre = g_hi + a.n_groups;   // [n_groups + 1]
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t tmem_cols = splits > 1 ? (BT < 32 ? 32 : BT) : (2 * BT);   // one accumulator where a CTA has one tile

  if (threadIdx.x == 0) {
    for (int s = 0; s < stages; ++s) {
      mbar_init(full_bar(s), 1);
      mbar_init(empty_bar(s), 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(tfull_bar(i), 1);
      mbar_init(tempty_bar(i), EPI_WARPS * CG);
    }
    *abort_flag = 0u;
    mbar_init_fence();
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
  if (warp == 2) {
    // the group table: bounds that start below an earlier bound, end before they start or leave the rows are dropped
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
  tc_fence_before();
  __syncthreads();
  if (cluster > 1) cluster_sync();   // the peers' barriers are initialised before anything signals them
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  grid_dep_launch();
  const int total = g_pre[a.n_groups] * a.f_tiles;
  // this CTA's share of K
  const int kb0 = splits > 1 ? static_cast<int>(static_cast<int64_t>(rank) * a.k_blocks / splits) : 0;
  const int kb1 = splits > 1 ? static_cast<int>(static_cast<int64_t>(rank + 1) * a.k_blocks / splits) : a.k_blocks;
  // tokens of the MMA: the tile's, rounded up to what the instruction takes (and halves of the pair to its row groups)
  auto mma_n = [](int rows) { return CG == 2 ? (rows + 31) / 32 * 32 : (rows + 15) / 16 * 16; };

  auto give_up = [&]() {
    *abort_flag = 1u;
    if constexpr (CG == 2) st_cluster_u32(map_to_rank(smem_u32(const_cast<uint32_t*>(abort_flag)), rank ^ 1u), 1u);
  };

  if (warp == 0) {
    // ---------------- TMA producer ----------------
    if (lane == 0) {
      int stage = 0;
      uint32_t phase = 0;
      bool ok = true;
      for (int item = worker; ok && item < total; item += n_workers) {
        const Tile t = tile_of<BT>(a, g_lo, g_hi, g_pre, item);
        const int n = mma_n(t.rows) / CG;                       // token rows of this CTA
        const int boxes = (n + S::BOX - 1) / S::BOX;
        const int f0 = (t.feature_tile * CG + (CG == 2 ? static_cast<int>(rank) : 0)) * BF;
        const int r0 = t.row0 + (CG == 2 ? static_cast<int>(rank) * n : 0);
        const uint32_t bytes = static_cast<uint32_t>(S::W_BYTES + boxes * S::BOX * BKB);
        for (int kb = kb0; kb < kb1; ++kb) {
          if (!mbar_wait(empty_bar(stage), phase ^ 1u, abort_flag, WAIT_LIMIT_NS)) { ok = false; give_up(); break; }
          const uint32_t w_dst = smem_base + stage * S::STAGE_BYTES, a_dst = w_dst + S::W_BYTES;
          if constexpr (CG == 2) {
            // the data of both CTAs is accounted on the leader's barrier
            const uint32_t bar = map_to_rank(full_bar(stage), 0u);
            if (leader) mbar_arrive_expect_tx(full_bar(stage), 2u * bytes);
            tma_load_3d_cg2(w_dst, &tm_w, bar, kb * BKB, f0, t.group);
            for (int b = 0; b < boxes; ++b) tma_load_2d_cg2(a_dst + b * S::BOX * BKB, &tm_a, bar, kb * BKB, r0 + b * S::BOX);
          } else {
            mbar_arrive_expect_tx(full_bar(stage), bytes);
            tma_load_3d(w_dst, &tm_w, full_bar(stage), kb * BKB, f0, t.group);
            for (int b = 0; b < boxes; ++b) tma_load_2d(a_dst + b * S::BOX * BKB, &tm_a, full_bar(stage), kb * BKB, r0 + b * S::BOX);
          }
          if (++stage == stages) { stage = 0; phase ^= 1u; }
        }
      }
      if (!ok) {
        // give copies already in flight time to land before shared memory is released
        for (int i = 0; i < 200; ++i) __nanosleep(1000);
      }
    }
    __syncwarp();
  } else if (warp == 1) {
    // ---------------- MMA issuer (leader CTA only) ----------------
    if (lane == 0 && leader) {
      int stage = 0, acc = 0;
      uint32_t phase = 0, acc_phase = 0;
      bool ok = true;
      const bool f8 = a.l.ab_dtype == HB_DTYPE_E4M3;
      const uint32_t format = a.l.ab_dtype == HB_DTYPE_BF16 ? (1u << 7 | 1u << 10) : 0u;   // bf16 operands; f16 and e4m3 are format 0 of their kinds
      for (int item = worker; ok && item < total; item += n_workers) {
        const Tile t = tile_of<BT>(a, g_lo, g_hi, g_pre, item);
        const uint32_t idesc = make_idesc_f16(BF * CG, mma_n(t.rows), false) | format;
        if (!mbar_wait(tempty_bar(acc), acc_phase ^ 1u, abort_flag, WAIT_LIMIT_NS)) { ok = false; give_up(); break; }
        tc_fence_after();
        const uint32_t d = tmem_base + static_cast<uint32_t>(acc * BT);
        for (int kb = kb0; kb < kb1; ++kb) {
          if (!mbar_wait(full_bar(stage), phase, abort_flag, WAIT_LIMIT_NS)) { ok = false; give_up(); break; }
          tc_fence_after();
          const uint32_t w_addr = smem_base + stage * S::STAGE_BYTES;
          const uint64_t wdesc = make_desc(w_addr, 16, 1024), adesc = make_desc(w_addr + S::W_BYTES, 16, 1024);
#pragma unroll
          for (int k = 0; k < BKB / 32; ++k) {
            const uint32_t more = (kb > kb0 || k > 0) ? 1u : 0u;   // 32 bytes along K = +2 in the descriptors' address field
            if constexpr (CG == 2) {
              if (f8) umma_ss_f8_cg2(d, wdesc + 2u * k, adesc + 2u * k, idesc, more);
              else umma_ss_cg2(d, wdesc + 2u * k, adesc + 2u * k, idesc, more);
            } else {
              if (f8) umma_ss_f8(d, wdesc + 2u * k, adesc + 2u * k, idesc, more);
              else umma_ss(d, wdesc + 2u * k, adesc + 2u * k, idesc, more);
            }
          }
          if constexpr (CG == 2) umma_commit_cg2(empty_bar(stage));
          else umma_commit(empty_bar(stage));
          if (++stage == stages) { stage = 0; phase ^= 1u; }
        }
        if (!ok) break;
        if constexpr (CG == 2) umma_commit_cg2(tfull_bar(acc));
        else umma_commit(tfull_bar(acc));
        if (++acc == 2) { acc = 0; acc_phase ^= 1u; }
      }
    }
    __syncwarp();
  } else if (splits == 1) {
    // ---------------- epilogue (warps 2..9) ----------------
    const int quarter = warp & 3;            // tensor memory lanes [32 quarter, 32 quarter + 32) belong to this warp
    const int half = (warp - 2) >> 2;        // which of every two blocks of 32 tokens
    float* stg = staging + (warp - 2) * 16 * STG_PITCH;
    const int fq = (lane & 7) * 4, tk = lane >> 3;
    int acc = 0;
    uint32_t acc_phase = 0;
    bool ok = true;
    for (int item = worker; ok && item < total; item += n_workers) {
      const Tile t = tile_of<BT>(a, g_lo, g_hi, g_pre, item);
      const int f0 = (t.feature_tile * CG + (CG == 2 ? static_cast<int>(rank) : 0)) * BF + quarter * 32;
      Features ft;
      ft.init(a.l, t.group, f0 + fq);
      if (!mbar_wait(tfull_bar(acc), acc_phase, abort_flag, WAIT_LIMIT_NS)) { ok = false; give_up(); break; }
      tc_fence_after();
      const uint32_t t_row = tmem_base + (static_cast<uint32_t>(quarter * 32) << 16) + static_cast<uint32_t>(acc * BT);
#pragma unroll 1
      for (int c = half * 32; c < t.rows; c += 64) {
        uint32_t r[32];
        tmem_ld32(t_row + static_cast<uint32_t>(c), r);
        tmem_ld_wait();
#pragma unroll
        for (int p = 0; p < 2; ++p) {
#pragma unroll
          for (int j = 0; j < 16; ++j) stg[j * STG_PITCH + lane] = __uint_as_float(r[p * 16 + j]);
          __syncwarp();
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int token = c + p * 16 + i * 4 + tk;
            if (token < t.rows) {
              const float4 v = *reinterpret_cast<const float4*>(stg + (i * 4 + tk) * STG_PITCH + fq);
              float s[4] = {v.x, v.y, v.z, v.w};
              ft.finish(a, t.row0 + token, s);
            }
          }
          __syncwarp();
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) {
        if constexpr (CG == 2) mbar_arrive_cluster(map_to_rank(tempty_bar(acc), 0u));
        else mbar_arrive(tempty_bar(acc));
      }
      if (++acc == 2) { acc = 0; acc_phase ^= 1u; }
    }
  } else if (worker < total) {
    mbar_wait(tfull_bar(0), 0u, abort_flag, WAIT_LIMIT_NS);
    __syncwarp();
    tc_fence_after();
  }
  if constexpr (CG == 1) {
    if (splits > 1) {
      // every CTA of the cluster is through with its stages: they take the partial sums [source][token][feature] of the
      // tokens that this CTA finishes
      __syncthreads();
      cluster_sync();
      if (worker < total) {
        const Tile t = tile_of<BT>(a, g_lo, g_hi, g_pre, worker);
        const int per = (t.rows + splits - 1) / splits;     // tokens of each CTA
        if (warp >= 2) {
          const int quarter = warp & 3, half = (warp - 2) >> 2;
          const uint32_t t_row = tmem_base + (static_cast<uint32_t>(quarter * 32) << 16);
          const uint32_t mine = smem_base + (rank * per * BF + quarter * 32 + lane) * 4;
#pragma unroll 1
          for (int c = half * 32; c < t.rows; c += 64) {
            uint32_t r[32];
            tmem_ld32(t_row + static_cast<uint32_t>(c), r);
            tmem_ld_wait();
#pragma unroll
            for (int j = 0; j < 32; ++j) {
              if (c + j < t.rows) {
                const int owner = (c + j) / per;
                st_cluster_f32(map_to_rank(mine + (c + j - owner * per) * BF * 4, owner), __uint_as_float(r[j]));
              }
            }
          }
        }
      }
      tc_fence_before();
      __syncthreads();
      cluster_sync();
      if (worker < total && !*abort_flag) {
        const Tile t = tile_of<BT>(a, g_lo, g_hi, g_pre, worker);
        const int per = (t.rows + splits - 1) / splits;
        Features ft;
        ft.init(a.l, t.group, t.feature_tile * BF + lane * 4);
        const float* part = reinterpret_cast<const float*>(smem_gen);
        for (int i = warp; i < per && static_cast<int>(rank) * per + i < t.rows; i += NUM_THREADS / 32) {
          float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
          for (int src = 0; src < splits; ++src) {
            const float4 v = *reinterpret_cast<const float4*>(part + (src * per + i) * BF + lane * 4);
            s[0] += v.x; s[1] += v.y; s[2] += v.z; s[3] += v.w;
          }
          ft.finish(a, t.row0 + static_cast<int>(rank) * per + i, s);
        }
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

int elem_bytes(int dtype) { return dtype == HB_DTYPE_F32 ? 4 : dtype == HB_DTYPE_E4M3 ? 1 : 2; }
bool float_type(int dtype) { return dtype == HB_DTYPE_F32 || dtype == HB_DTYPE_F16 || dtype == HB_DTYPE_BF16; }
bool on(const void* p, int bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }

int check(const hb_ctx* c, const hb_linear_args* l) {
  if (!c || !l || l->m < 0 || l->n < 1 || l->k < 1) return HB_ERR_BAD_ARG;
  if (l->ab_dtype != HB_DTYPE_F16 && l->ab_dtype != HB_DTYPE_BF16 && l->ab_dtype != HB_DTYPE_E4M3) return HB_ERR_BAD_ARG;
  if (!float_type(l->c_dtype) || (l->residual && !float_type(l->residual_dtype))) return HB_ERR_BAD_ARG;
  if (l->act < HB_ACT_NONE || l->act > HB_ACT_GELU_TANH || (l->gated != 0 && l->gated != 1) || (l->gated && l->n % 2)) return HB_ERR_BAD_ARG;
  if (l->m > (1 << 26) || l->n > (1 << 26) || l->k > (1 << 26)) return HB_ERR_TOO_LARGE;
  const int ab = elem_bytes(l->ab_dtype), cols = l->gated ? l->n / 2 : l->n;
  if (l->a_stride < l->k || l->w_stride < l->k || l->c_stride < cols || (l->residual && l->residual_stride < cols)) return HB_ERR_BAD_ARG;
  if (l->a_stride > (1ll << 36) || l->w_stride > (1ll << 36)) return HB_ERR_TOO_LARGE;
  if (!on(l->a, 16) || !on(l->w, 16) || (l->a_stride * ab) % 16 || (l->w_stride * ab) % 16) return HB_ERR_BAD_ARG;
  if (!on(l->c, elem_bytes(l->c_dtype)) || (l->residual && !on(l->residual, elem_bytes(l->residual_dtype))) || !on(l->a_scale, 4) ||
      !on(l->w_scale, 4) || !on(l->bias, 4))
    return HB_ERR_BAD_ARG;
  if (l->m > 0 && (!l->a || !l->w || !l->c)) return HB_ERR_BAD_ARG;
  return HB_OK;
}

int wrong_device(const hb_ctx* c) {
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess) return HB_ERR_CUDA;
  return dev == c->device ? HB_OK : HB_ERR_BAD_ARG;   // launches go to the current device
}

}  // namespace

namespace {

template <int CG, int BT>
int launch(const hb_linear_args& l, LinArgs a, int splits, int num_sms, int64_t w_group_stride, cudaStream_t s, bool pdl) {
  using S = Shape<CG, BT>;
  const int ab = elem_bytes(l.ab_dtype);
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
  const int fixed = 1024 + BAR_BYTES + (splits > 1 ? 0 : STG_BYTES) + table;
  const int room = (splits > 1 ? 113 : 227) * 1024;
  a.stages = (room - fixed) / S::STAGE_BYTES;
  if (a.stages > MAX_STAGES) a.stages = MAX_STAGES;
  const int smem = fixed + a.stages * S::STAGE_BYTES;
  static DynSmemState configured;
  auto kern = linear_kernel<CG, BT>;
  if (hb_ensure_dyn_smem(reinterpret_cast<const void*>(kern), configured, smem) != HB_OK) return HB_ERR_CUDA;
  int64_t workers = items;
  if (splits == 1 && workers > num_sms / CG) workers = num_sms / CG;
  cudaLaunchConfig_t cfg = {};
  const int cluster = CG == 2 ? 2 : splits;
  cfg.gridDim = dim3(static_cast<unsigned>(workers * cluster));
  cfg.blockDim = dim3(NUM_THREADS);
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
  return cudaLaunchKernelEx(&cfg, kern, tw, ta, a) == cudaSuccess ? HB_OK : HB_ERR_CUDA;
}

}  // namespace

int hb_launch_linear(hb_ctx* c, const hb_linear_args& l, const int32_t* group_start, int n_groups, int64_t w_group_stride,
                     cudaStream_t s, bool pdl) {
  LinArgs a = {};
  a.l = l;
  a.start = group_start;
  a.n_groups = n_groups;
  a.status = c->status;
  a.k_blocks = static_cast<int>((static_cast<int64_t>(l.k) * elem_bytes(l.ab_dtype) + BKB - 1) / BKB);
  const int per = l.gated ? 2 : 4, cb = elem_bytes(l.c_dtype) * per;
  auto rows_on = [](const void* p, int64_t stride, int size, int bytes) { return on(p, bytes) && (stride * size) % bytes == 0; };
  a.wide = l.n % 4 == 0 && rows_on(l.c, l.c_stride, elem_bytes(l.c_dtype), cb) &&
           (!l.residual || rows_on(l.residual, l.residual_stride, elem_bytes(l.residual_dtype), elem_bytes(l.residual_dtype) * per));
  const int avg = (l.m + n_groups - 1) / n_groups;
  const int sms = c->num_sms;
  if (avg > 128) return launch<2, 256>(l, a, 1, sms, w_group_stride, s, pdl);
  const int bt = avg <= 32 ? 32 : avg <= 64 ? 64 : 128;
  const int64_t tiles = static_cast<int64_t>((l.n + BF - 1) / BF) * ((l.m + bt - 1) / bt);
  int splits = 1;
  while (splits < 8 && tiles * splits * 2 <= 2 * sms && 2 * splits <= a.k_blocks) splits *= 2;
  if (bt == 32) return launch<1, 32>(l, a, splits, sms, w_group_stride, s, pdl);
  if (bt == 64) return launch<1, 64>(l, a, splits, sms, w_group_stride, s, pdl);
  return launch<1, 128>(l, a, splits, sms, w_group_stride, s, pdl);
}

extern "C" int hb_linear(hb_ctx* c, const hb_linear_args* l, void* stream) {
  int rc = check(c, l);
  if (rc != HB_OK || l->m == 0) return rc;
  if ((rc = wrong_device(c)) != HB_OK) return rc;
  return hb_launch_linear(c, *l, nullptr, 1, 0, static_cast<cudaStream_t>(stream), false);
}

extern "C" int hb_linear_grouped(hb_ctx* c, const hb_linear_args* l, const int32_t* group_start, int32_t n_groups,
                                 int64_t w_group_stride, void* stream) {
  int rc = check(c, l);
  if (rc != HB_OK) return rc;
  if (n_groups < 1 || !on(group_start, 4) || w_group_stride < static_cast<int64_t>(l->n - 1) * l->w_stride + l->k) return HB_ERR_BAD_ARG;
  if (n_groups > HB_LINEAR_MAX_GROUPS || w_group_stride > (1ll << 36)) return HB_ERR_TOO_LARGE;
  if ((w_group_stride * elem_bytes(l->ab_dtype)) % 16) return HB_ERR_BAD_ARG;
  if (l->m == 0) return HB_OK;
  if (!group_start) return HB_ERR_BAD_ARG;
  if ((rc = wrong_device(c)) != HB_OK) return rc;
  return hb_launch_linear(c, *l, group_start, n_groups, w_group_stride, static_cast<cudaStream_t>(stream), false);
}
