// Chunk rows over the 8-bit cache on the tcgen05 tensor cores (the segments of more than 16 columns).
//
// One CTA per SM stays resident and takes items: 256 query rows (256 / G consecutive tokens x the G query
// heads of one KV head) of one segment against every key they may see, in tiles of 64 keys (4 pages).
// The rows form two tiles A and B of 128 that alternate: while the tensor cores work for one, the softmax
// warps of the other compute.  Both use each converted key tile.  14 warps:
//   warp 0      bulk copies of page blocks (codes and scales) into a ring
//   warp 1      issues tcgen05.mma: S_X = Q_X K^T (128 x 64) and O_X += P_X V (128 x DH), kind::f16, fp32 in
//               tensor memory
//   warps 2-5   conversion e4m3 -> fp16 (exact), one page each: K into [key][dim] rows, V into [dim][key] rows
//               of 128 bytes with the 128-byte swizzle, the layouts the matrix descriptors expect.  V is
//               stored by dimension so that the four codes of a word stay together; the order of the 16
//               keys inside a page that this gives is used for the columns of P too
//   warps 6-9   softmax of A, one thread per row (= tensor-memory lane); warps 10-13 the same for B
// Tensor memory (512 columns): O_A, O_B (fp32), S_A, S_B (fp32, 64 columns each), Q_A, Q_B (fp16, the A operand
// of S).  P_X (fp16) takes the place of S_X once its row has been read, and is the A operand of O_X: neither Q
// nor P is read through shared memory, whose bandwidth goes to K, V and the conversion.
//   order of the tensor cores' work:  S_A(0) S_B(0) | PV_A(0) S_A(1) PV_B(0) S_B(1) | PV_A(1) S_A(2) ...
// K's scale multiplies the fp32 scores (one factor per 16 columns); V's exponent goes into the exponent of
// P, as in the decode body.  O is rescaled only when a row's maximum has grown by more than 2^8.
// Bound by the two chains of dependent steps: 64 keys take a row tile about 2130 to 2420 cycles (scores 840 to 1110 until they
// are there and 160 to read, maximum 370 to 400, exponentials and P 745 to 760), of which the tensor cores work 1090 for both
// tiles together and the exponential unit 1020; with Q there tensor memory has no room for a third tile or a second S (Q in shared
// memory and key tiles of 128 were not tried).  8 chunks of 257 to 512 rows over 0 to 2048 earlier keys (74.5 GFLOP) 130 us =
// 574 TFLOP/s; one prompt of 4096 rows 180 us = 765 TFLOP/s; the chunks with heads of 64 109 us = 341 TFLOP/s.  An item's start and end (look-up 1000 cycles, Q 4400, last P V 800, store 3600) weigh more on short
// contexts.  Measured slower: Q and O through a stage in shared memory with whole lines, the next item's Q ahead (138 us
// against 128); Q_B in shared memory and two S per tile (150); two warps that issue MMAs (161); exponentials against the old
// maximum while the new one is taken (131).
// Every wait is bounded; on expiry the CTA raises a status bit, stores nothing more, frees its tensor memory
// and leaves.
#pragma once
#include "kv8.cuh"

namespace hb_kv8_tc {

using namespace hb_kv8;

constexpr int THREADS = 448;
constexpr int BM = 128, ROWS = 2 * BM;   // rows of a tile, of an item
constexpr int BN = 64, PAGES = BN / PAGE;
constexpr int RAW = 3, CV = 3;           // stages of the ring of codes, of converted tiles
// Items with a bad page, by round.  The copies run ahead of an item's last store by at most RAW + CV + 1 key tiles, so
// by no more items: a slot is not used again before it has been read.
constexpr int BAD = 8;
static_assert(BAD > RAW + CV + 1 && (BAD & (BAD - 1)) == 0, "slots of bad items");
constexpr uint64_t WAIT_NS = 1000000000ull;
// Least factor of the scores (the smallest normal float): zero times the -inf of a key that a row must not see would be
// NaN.  Scores are below 2^32, so that neither it nor anything smaller leaves anything of them.
constexpr float FACTOR_MIN = 1.1754944e-38f;
// A weight's exponent is formed in one step, score * factor + (e - m), whose product is not rounded, while m came from a
// rounded one, so that it may end above its bound by 2^-23 of m.  Up to 2^20 that is no more than the score's own rounding;
// further out the weights could leave fp16 (from 2^24 on), and the scores are rounded first, as in the maximum.
constexpr float FAR = 1048576.0f;

template <int DH>
struct Cfg {
  static constexpr int TILE = BN * DH * 2;              // bytes of a converted K (or V) tile
  static constexpr int RAW_BYTES = PAGES * Block<DH>::BYTES;
  static constexpr int RAW_OFF = CV * 2 * TILE;
  static constexpr int SC_OFF = RAW_OFF + RAW * RAW_BYTES;   // float2 [CV][PAGES]: factor of the scores, exponent of V
  static constexpr int NAN_OFF = SC_OFF + CV * PAGES * 8;    // uint32 [CV][PAGES]: tokens whose V holds NaN (see nan_tokens)
  static constexpr int BAR_OFF = NAN_OFF + CV * PAGES * 4;
  static constexpr int N_BARS = 2 * RAW + 2 * CV + 10;   // raw, cv (full, empty); for A and B: S full, P ready (two halves), Q ready, O full
  static constexpr int MISC_OFF = BAR_OFF + N_BARS * 8;      // abort flag, tensor-memory base, warp sums, bad items
  static constexpr int FIXED = MISC_OFF + 128 + BAD * 4;
  static constexpr int O_COL = 0, S_COL = 256, Q_COL = 384;
};

// One lane of the warp issues; the operands are the same in all of them, so that they stay in uniform registers
// (35 and 67 cycles an instruction at N = 64 and 128, against about 100 from a divergent branch).
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "elect.sync _|q, 0xffffffff;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
      ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(acc) : "memory");
}
__device__ __forceinline__ void commit(uint32_t bar) {
  asm volatile(
      "{\n\t.reg .pred q;\n\t"
      "elect.sync _|q, 0xffffffff;\n\t"
      "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(bar) : "memory");
}

__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
      ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
        "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}

struct TcItem {
  Seg g;
  int seg, head;
  int row0, n_rows;      // rows [row0, row0 + n_rows) of the segment's q_len * G
  int tiles[2];          // key tiles of A and of B (0: no rows)
  int key1;              // keys the item needs (those of its last row)
  int all_see;           // last key that all of its rows see
};

__device__ __forceinline__ int tc_blocks(const Rows& r, const Seg& g) {
  const int cols = g.q_len * r.G;
  return cols > 16 ? (cols + ROWS - 1) / ROWS : 0;
}

// Items in the order of their cost: with few of them (up to MAX_SORTED blocks of rows, each for all KV heads) a
// block that got two long ones would be the last by far (84 key tiles where 52 are the mean, in a step of 8
// chunks over contexts of 0 to 2048).  The blocks take them in rounds, every other round backwards.
constexpr int MAX_SORTED = 512;

__device__ __forceinline__ int item_of(const uint16_t* order, int total, int n_heads, int round) {
  const int t = round * gridDim.x + ((round & 1) ? gridDim.x - 1 - blockIdx.x : blockIdx.x);
  if (t >= total) return -1;
  return order ? order[t / n_heads] * n_heads + t % n_heads : t;
}

__device__ __forceinline__ void tc_item(const Rows& r, const int* prefix, int idx, TcItem& it) {
  it.seg = find_seg(prefix, r.n_segs, idx);
  load_seg(r, it.seg, it.g);
  const int at = idx - prefix[it.seg], nb = tc_blocks(r, it.g);
  it.head = at % r.Hkv;
  const int blk = nb - 1 - at / r.Hkv;      // the last rows see the most keys: first
  it.row0 = blk * ROWS;
  it.n_rows = min(ROWS, it.g.q_len * r.G - it.row0);
  const int last_a = min(it.n_rows, BM) - 1;
  it.tiles[0] = (it.g.pos_start + (it.row0 + last_a) / r.G + 1 + BN - 1) / BN;
  it.key1 = it.g.pos_start + (it.row0 + it.n_rows - 1) / r.G + 1;
  it.all_see = it.g.pos_start + it.row0 / r.G;
  it.tiles[1] = it.n_rows > BM ? (it.key1 + BN - 1) / BN : 0;
}

template <int DH>
__global__ void __launch_bounds__(THREADS, 1)
kv8_chunk_kernel(const AttnParams p) {
  using C = Cfg<DH>;
  extern __shared__ __align__(1024) uint8_t smem[];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t base = smem_u32(smem), bars = base + C::BAR_OFF;
  auto raw_full = [&](int s) { return bars + 8u * s; };
  auto raw_empty = [&](int s) { return bars + 8u * (RAW + s); };
  auto cv_full = [&](int s) { return bars + 8u * (2 * RAW + s); };
  auto cv_empty = [&](int s) { return bars + 8u * (2 * RAW + CV + s); };
  const uint32_t s_full0 = bars + 8u * (2 * RAW + 2 * CV), p_ready0 = s_full0 + 16u, q_ready0 = p_ready0 + 32u, o_full0 = q_ready0 + 16u;
  volatile uint32_t* abort_flag = reinterpret_cast<volatile uint32_t*>(smem + C::MISC_OFF);
  volatile int* bad_items = reinterpret_cast<volatile int*>(smem + C::MISC_OFF + 128);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + C::MISC_OFF + 8);
  int* warp_sums = reinterpret_cast<int*>(smem + C::MISC_OFF + 64);
  int* prefix = reinterpret_cast<int*>(smem + C::FIXED);
  if (base & 1023u) {   // the swizzled tiles need it; the same in every thread
    grid_dep_wait();
    if (tid == 0) atomicOr(p.r.status, HB_DEV_ATTN_BAD_INDEX);
    return;
  }
  if (tid == 0) {
    for (int s = 0; s < RAW; ++s) { mbar_init(raw_full(s), 1); mbar_init(raw_empty(s), 4); }
    for (int s = 0; s < CV; ++s) { mbar_init(cv_full(s), 4); mbar_init(cv_empty(s), 1); }
    for (int x = 0; x < 2; ++x) {
      mbar_init(s_full0 + 8u * x, 1);
      mbar_init(p_ready0 + 16u * x, 4);
      mbar_init(p_ready0 + 16u * x + 8u, 4);
      mbar_init(q_ready0 + 8u * x, 4);
      mbar_init(o_full0 + 8u * x, 1);
    }
    *abort_flag = 0u;
    for (int i = 0; i < BAD; ++i) bad_items[i] = -1;
    mbar_init_fence();
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(tmem_slot)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  // A block may take its SM, its barriers and its tensor memory while the decode kernel drains; what it reads (the
  // segments, the queries, the pages appended by the launch before) is only sure to be there behind the wait.  That the
  // decode blocks have waited for it themselves orders the execution, and makes nothing visible here.
  grid_dep_wait();
  const int total = build_prefix<THREADS>(p.r, prefix, warp_sums, [&](const Seg& g) { return tc_blocks(p.r, g) * p.r.Hkv; }, false);
  const uint16_t* order = nullptr;
  const int n_blocks = total / p.r.Hkv;
  if (n_blocks <= MAX_SORTED && total > static_cast<int>(gridDim.x)) {
    uint16_t* cost = reinterpret_cast<uint16_t*>(prefix + p.r.n_segs + 1);
    uint16_t* sorted = cost + MAX_SORTED;
    for (int i = tid; i < n_blocks; i += THREADS) {
      TcItem it;
      tc_item(p.r, prefix, i * p.r.Hkv, it);
      cost[i] = static_cast<uint16_t>(min(65535, max(it.tiles[0], it.tiles[1]) * 2 - (it.tiles[1] == 0)));
    }
    __syncthreads();
    for (int i = tid; i < n_blocks; i += THREADS) {
      const int mine = cost[i];
      int rank = 0;
      for (int k = 0; k < n_blocks; ++k) rank += cost[k] > mine || (cost[k] == mine && k < i);
      sorted[rank] = static_cast<uint16_t>(i);
    }
    order = sorted;
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  // What follows waits for this kernel's end.  It may start only now that every block has its tensor memory: a block of a
  // later kernel that held some while it waited would keep a block here from starting.
  grid_dep_launch();

  if (warp == 0) {
    // ---------------- page blocks ----------------
    uint32_t n = 0;   // tiles asked for so far
    bool ok = true;
    for (int round = 0, idx; ok && (idx = item_of(order, total, p.r.Hkv, round)) >= 0; ++round) {
      TcItem it;
      tc_item(p.r, prefix, idx, it);
      const int n_pg = (it.key1 + PAGE - 1) / PAGE, n_tiles = (n_pg + PAGES - 1) / PAGES;
      const int32_t* ids = p.r.page_ids + it.g.pt_start;
      int have = 0, cur = 0, nxt = lane < n_pg ? __ldg(ids + lane) : 0;   // 32 page ids, one per lane, 32 more on the way
      for (int j = 0; j < n_tiles; ++j, ++n) {
        if (j * PAGES == have) {
          cur = nxt;
          const bool bad = have + lane < n_pg && (cur < 0 || cur >= p.r.n_pages);
          if (bad) {   // reported; the item runs on another page and its rows are not stored
            atomicOr(p.r.status, HB_DEV_ATTN_BAD_INDEX);
            bad_items[round & (BAD - 1)] = idx;
            cur = 0;
          }
          have += 32;
          nxt = have + lane < n_pg ? __ldg(ids + have + lane) : 0;
        }
        const int st = n % RAW, here = min(PAGES, n_pg - j * PAGES);
        if (!__all_sync(0xffffffffu, mbar_wait(raw_empty(st), ((n / RAW) & 1u) ^ 1u, abort_flag, WAIT_NS))) { ok = false; break; }
        const int page = __shfl_sync(0xffffffffu, cur, (j * PAGES + min(lane, here - 1)) & 31);
        if (lane == 0) mbar_arrive_expect_tx(raw_full(st), static_cast<uint32_t>(here) * Block<DH>::BYTES);
        __syncwarp();
        if (lane < here)
          bulk_load(base + C::RAW_OFF + st * C::RAW_BYTES + lane * Block<DH>::BYTES,
                    p.r.arena + page * p.r.page_stride + static_cast<int64_t>(it.head) * Block<DH>::BYTES, Block<DH>::BYTES, raw_full(st));
      }
    }
  } else if (warp == 1) {
    // ---------------- tensor cores ----------------
    constexpr uint32_t idesc_s = make_idesc_f16(BM, BN, false), idesc_o = make_idesc_f16(BM, DH, false);
    uint32_t n = 0, n_p[2] = {0, 0}, n_q[2] = {0, 0};   // key tiles, P tiles, Q tiles consumed
    bool ok = true;
    auto wait = [&](uint32_t bar, uint32_t parity) {
      if (ok && !__all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag, WAIT_NS))) ok = false;
      return ok;
    };
    auto issue_s = [&](int x, uint32_t tile) {
      const uint32_t k_tile = base + (tile % CV) * 2 * C::TILE;
#pragma unroll
      for (int ks = 0; ks < DH / 16; ++ks)
        mma_ts(tmem + C::S_COL + x * BN, tmem + C::Q_COL + x * (DH / 2) + ks * 8, make_desc(k_tile + (ks >> 2) * (BN * 128) + (ks & 3) * 32, 16, 1024),
               idesc_s, ks > 0 ? 1u : 0u);
      commit(s_full0 + 8u * x);
    };
    for (int round = 0, idx; ok && (idx = item_of(order, total, p.r.Hkv, round)) >= 0; ++round) {
      TcItem it;
      tc_item(p.r, prefix, idx, it);
      const int n_tiles = max(it.tiles[0], it.tiles[1]);
      if (!wait(cv_full(n % CV), (n / CV) & 1u)) break;
      for (int x = 0; x < 2; ++x)
        if (it.tiles[x] > 0) {
          if (!wait(q_ready0 + 8u * x, n_q[x] & 1u)) break;
          ++n_q[x];
          tc_fence_after();
          issue_s(x, n);
        }
      for (int j = 0; j < n_tiles && ok; ++j, ++n) {
        const bool more = j + 1 < n_tiles;
        if (more && !wait(cv_full((n + 1) % CV), ((n + 1) / CV) & 1u)) break;
        const uint32_t v_tile = base + (n % CV) * 2 * C::TILE + C::TILE;
        for (int x = 0; x < 2 && ok; ++x) {
          if (j < it.tiles[x]) {
#pragma unroll
            for (int ks = 0; ks < BN / 16; ++ks) {
              if (ks % 2 == 0) {   // each half of P has its own barrier
                if (!wait(p_ready0 + 16u * x + 4u * ks, n_p[x] & 1u)) break;
                tc_fence_after();
              }
              mma_ts(tmem + C::O_COL + x * DH, tmem + C::S_COL + x * BN + ks * 8, make_desc(v_tile + ks * 32, 16, 1024), idesc_o, (j > 0 || ks > 0) ? 1u : 0u);
            }
            if (!ok) break;
            ++n_p[x];
            if (j + 1 == it.tiles[x]) commit(o_full0 + 8u * x);
          }
          if (x == 1) commit(cv_empty(n % CV));   // both tiles' reads of this key tile are in front of it
          if (j + 1 < it.tiles[x]) issue_s(x, n + 1);
        }
      }
    }
  } else if (warp < 6) {
    // ---------------- conversion: one page of every tile per warp ----------------
    const int pg = warp - 2;
    uint32_t n = 0;
    bool ok = true;
    // lanes of a half warp take dimensions whose rows of V^T differ in their swizzle and in their bank of the
    // codes: 0, 3, 4, 7 and 1, 2, 5, 6
    const int i4 = (lane >> 2) & 3, vd = lane < 16 ? (i4 == 0 ? 0 : i4 == 1 ? 3 : i4 == 2 ? 4 : 7) : (i4 == 0 ? 1 : i4 == 1 ? 2 : i4 == 2 ? 5 : 6), vt = lane & 3;
    for (int round = 0, idx; ok && (idx = item_of(order, total, p.r.Hkv, round)) >= 0; ++round) {
      TcItem it;
      tc_item(p.r, prefix, idx, it);
      const int n_tiles = (it.key1 + BN - 1) / BN;
      for (int j = 0; j < n_tiles; ++j, ++n) {
        const int rs = n % RAW, cs = n % CV;
        if (!__all_sync(0xffffffffu, mbar_wait(raw_full(rs), (n / RAW) & 1u, abort_flag, WAIT_NS) &&
                                         mbar_wait(cv_empty(cs), ((n / CV) & 1u) ^ 1u, abort_flag, WAIT_NS))) { ok = false; break; }
        const int key = j * BN + pg * PAGE, left = it.key1 - key;   // keys of this page that count
        const uint32_t src = base + C::RAW_OFF + rs * C::RAW_BYTES + pg * Block<DH>::BYTES;
        uint8_t* k_tile = smem + cs * 2 * C::TILE;
        uint8_t* v_tile = k_tile + C::TILE;
        float2 sc = make_float2(1.0f, 0.0f);
        if (left > 0) {
          asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(sc.x), "=f"(sc.y) : "r"(src + Block<DH>::HDR));
          sc.x = fmaxf(sc.x * p.scale_log2, FACTOR_MIN);
          sc.y = static_cast<float>(exponent_of(sc.y));
        }
        if (lane == 0) *reinterpret_cast<float2*>(smem + C::SC_OFF + (cs * PAGES + pg) * 8) = sc;
        const bool hidden = key + PAGE - 1 > it.all_see;   // some rows must not see all of this page
        uint32_t nan_bytes = 0;
#pragma unroll
        for (int i = 0; i < DH / 32; ++i) {
          const int hf = i >> 1, u = (i & 1) * 32 + lane, tok = u >> 2, q = u & 3;
          uint4 c = lds128(src + hf * 1024 + tok * 64 + q * 16);
          if (left <= 0) c = make_uint4(0u, 0u, 0u, 0u);   // (no copy has written this part of the stage)
          uint4 a, b;
          e4m3x4_to_half2x2(c.x, a.x, a.y);
          e4m3x4_to_half2x2(c.y, a.z, a.w);
          e4m3x4_to_half2x2(c.z, b.x, b.y);
          e4m3x4_to_half2x2(c.w, b.z, b.w);
          uint8_t* row = k_tile + hf * (BN * 128) + (pg * PAGE + tok) * 128;
          *reinterpret_cast<uint4*>(row + (((2 * q) ^ (tok & 7)) << 4)) = a;
          *reinterpret_cast<uint4*>(row + (((2 * q + 1) ^ (tok & 7)) << 4)) = b;
        }
        // codes of V behind the last key become zero: 0 * NaN would reach the rows
        uint32_t keep = 0xffffffffu;
        if (left < PAGE)
          keep = (2 * vt < left ? 0xffu : 0u) | (2 * vt + 1 < left ? 0xff00u : 0u) | (2 * vt + 8 < left ? 0xff0000u : 0u) |
                 (2 * vt + 9 < left ? 0xff000000u : 0u);
#pragma unroll
        for (int c = 0; c < DH / 32; ++c) {
          const uint4 v = lds128(src + Block<DH>::V_OFF + c * 512 + (vd * 4 + vt) * 16);
          uint32_t w[4] = {v.x & keep, v.y & keep, v.z & keep, v.w & keep};
          if (hidden) {
#pragma unroll
            for (int e = 0; e < 4; ++e) nan_bytes |= drop_nan(w[e]);
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            uint2 h;
            e4m3x4_to_half2x2(w[e], h.x, h.y);
            *reinterpret_cast<uint2*>(v_tile + (c * 32 + e * 8 + vd) * 128 + (((pg * 2 + (vt >> 1)) ^ vd) << 4) + (vt & 1) * 8) = h;
          }
        }
        if (hidden) nan_bytes = nan_tokens(nan_bytes, vt);
        if (lane == 0) *reinterpret_cast<uint32_t*>(smem + C::NAN_OFF + (cs * PAGES + pg) * 4) = nan_bytes;
        fence_async_smem();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(raw_empty(rs));
          mbar_arrive(cv_full(cs));
        }
      }
    }
  } else {
    // ---------------- softmax: one thread per row ----------------
    const int x = warp < 10 ? 0 : 1, quarter = warp & 3, rr = quarter * 32 + lane;
    const uint32_t t_lane = tmem + (static_cast<uint32_t>(quarter * 32) << 16);
    const uint32_t t_s = t_lane + C::S_COL + x * BN, t_o = t_lane + C::O_COL + x * DH, t_q = t_lane + C::Q_COL + x * (DH / 2);
    uint32_t n = 0, n_s = 0, n_o = 0;   // key tiles of all items so far, S tiles and outputs of this row tile
    bool ok = true;
    auto wait = [&](uint32_t bar, uint32_t parity) {
      if (ok && !__all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag, WAIT_NS))) ok = false;
      return ok;
    };
    for (int round = 0, idx; ok && (idx = item_of(order, total, p.r.Hkv, round)) >= 0; ++round) {
      TcItem it;
      tc_item(p.r, prefix, idx, it);
      const int row = x * BM + rr;
      const bool valid = row < it.n_rows;
      const int r = it.row0 + (valid ? row : 0), G = p.r.G;
      const int pos = valid ? it.g.pos_start + r / G : -1;
      const int tok = it.g.q_start + r / G, head = it.head * G + r % G;
      const int n_tiles = it.tiles[x], all_tiles = max(it.tiles[0], it.tiles[1]);
      if (n_tiles > 0) {
        const uint4* src = reinterpret_cast<const uint4*>(p.q + tok * p.q_stride + head * DH);
#pragma unroll
        for (int c = 0; c < DH / 2; c += 32) {
          uint32_t qr[32];
#pragma unroll
          for (int v = 0; v < 8; ++v) {
            const uint4 q4 = valid ? __ldg(src + c / 4 + v) : make_uint4(0u, 0u, 0u, 0u);
            qr[v * 4 + 0] = q4.x; qr[v * 4 + 1] = q4.y; qr[v * 4 + 2] = q4.z; qr[v * 4 + 3] = q4.w;
          }
          tmem_st32(t_q + c, qr);
        }
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        // (only for items with rows: a softmax group without any would run ahead of the barrier's phases)
        if (lane == 0) mbar_arrive(q_ready0 + 8u * x);
      }
      float m = -INFINITY, l = 0.0f;
      bool far = false;   // a row of the warp has its maximum beyond FAR
      for (int j = 0; j < n_tiles; ++j) {
        if (!wait(s_full0 + 8u * x, n_s & 1u)) break;
        ++n_s;
        tc_fence_after();
        uint32_t sr[2][32];
        tmem_ld32(t_s, sr[0]);
        tmem_ld32(t_s + 32, sr[1]);
        float2 sc[PAGES];
#pragma unroll
        for (int g = 0; g < PAGES; ++g) sc[g] = *reinterpret_cast<const float2*>(smem + C::SC_OFF + (((n + j) % CV) * PAGES + g) * 8);
        tmem_ld_wait();
        const int key = j * BN;
        if (key + BN - 1 > it.all_see) {   // NaN codes of V were dropped where some row must not see them
          bool sees_nan = false;
#pragma unroll
          for (int g = 0; g < PAGES; ++g) {
            const int last = min(pos - key - g * PAGE, PAGE - 1);   // the row sees tokens 0 .. last of the page
            if (last >= 0) sees_nan |= (*reinterpret_cast<const uint32_t*>(smem + C::NAN_OFF + (((n + j) % CV) * PAGES + g) * 4) & ((2u << last) - 1u)) != 0;
          }
          if (sees_nan) l = __uint_as_float(0x7fc00000u);
        }
        if (key + BN - 1 > pos) {   // the diagonal, or rows of nobody
          const int last = pos - key;
#pragma unroll
          for (int i = 0; i < BN; ++i)
            if (i > last) sr[i >> 5][i & 31] = 0xff800000u;   // -inf
        }
        float mx = -INFINITY;
#pragma unroll
        for (int g = 0; g < PAGES; ++g) {
          float a = __uint_as_float(sr[g >> 1][(g & 1) * PAGE]), b = __uint_as_float(sr[g >> 1][(g & 1) * PAGE + 1]);
#pragma unroll
          for (int i = 2; i < PAGE; i += 4) {   // (three-input maxima)
            a = fmaxf(fmaxf(a, __uint_as_float(sr[g >> 1][(g & 1) * PAGE + i])), __uint_as_float(sr[g >> 1][(g & 1) * PAGE + i + 1]));
            if (i + 2 < PAGE)
              b = fmaxf(fmaxf(b, __uint_as_float(sr[g >> 1][(g & 1) * PAGE + i + 2])), __uint_as_float(sr[g >> 1][(g & 1) * PAGE + i + 3]));
          }
          a = fmaxf(a, b);
          mx = fmaxf(mx, a == -INFINITY ? a : fmaf(a, sc[g].x, sc[g].y));
        }
        // P stays below 2^14: its reference lies 6 below the maximum it was taken from
        const bool grow = mx > m + 14.0f || (m == -INFINITY && mx > -INFINITY);
        if (__any_sync(0xffffffffu, grow || far)) {
          const float m_new = grow ? mx - 6.0f : m;
          const float f = grow ? ex2_approx(m - m_new) : 1.0f;   // -inf -> 0
          if (j > 0) {   // (S of this tile was issued behind the last P V: O is complete)
#pragma unroll 1
            for (int c = 0; c < DH; c += 32) {
              uint32_t o[32];
              tmem_ld32(t_o + c, o);
              tmem_ld_wait();
#pragma unroll
              for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
              tmem_st32(t_o + c, o);
            }
          }
          l *= f;
          m = m_new;
          far = __any_sync(0xffffffffu, m > FAR || (m < -FAR && m > -INFINITY));
          if (far) {   // exponents out of rounded scores (e, taken off here, is added below: a rounding of 2^-16 at most)
            const float ref = m == -INFINITY ? 0.0f : m;
#pragma unroll
            for (int g = 0; g < PAGES; ++g) {
#pragma unroll
              for (int i = 0; i < PAGE; ++i) {
                uint32_t& s = sr[g >> 1][(g & 1) * PAGE + i];
                s = __float_as_uint(fmaf(__uint_as_float(s), sc[g].x, sc[g].y) - ref - sc[g].y);
              }
              sc[g].x = 1.0f;
            }
          }
        }
        const float neg_m = far || m == -INFINITY ? 0.0f : -m;
#pragma unroll
        for (int h = 0; h < 2; ++h) {   // two pages, then the other two: the first half of P V starts early
          uint32_t pk[16];
#pragma unroll
          for (int g2 = 0; g2 < 2; ++g2) {
            const int g = h * 2 + g2;
            const uint64_t mul = pack2(sc[g].x, sc[g].x), add = pack2(sc[g].y + neg_m, sc[g].y + neg_m);
            float w[PAGE];
            uint64_t sum[2] = {0, 0};
#pragma unroll
            for (int i = 0; i < PAGE; i += 2) {
              float u, v;
              unpack2(fma2(pack2(__uint_as_float(sr[h][g2 * PAGE + i]), __uint_as_float(sr[h][g2 * PAGE + i + 1])), mul, add), u, v);
              w[i] = ex2_approx(u);
              w[i + 1] = ex2_approx(v);
              sum[(i >> 1) & 1] = add2(sum[(i >> 1) & 1], pack2(w[i], w[i + 1]));
            }
            float u, v;
            unpack2(add2(sum[0], sum[1]), u, v);
            l = fmaf(u + v, pow2f(max(-126, min(126, static_cast<int>(-sc[g].y)))), l);
#pragma unroll
            for (int t = 0; t < 4; ++t) {   // the order of the keys in V^T's rows: 2t, 2t+1, 2t+8, 2t+9
              pk[g2 * 8 + 2 * t] = pack_half2(w[2 * t], w[2 * t + 1]);
              pk[g2 * 8 + 2 * t + 1] = pack_half2(w[2 * t + 8], w[2 * t + 9]);
            }
          }
          tmem_st16(t_s + h * 16, pk);
          tmem_st_wait();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(p_ready0 + 16u * x + 8u * h);
        }
      }
      n += all_tiles;
      if (n_tiles > 0 && wait(o_full0 + 8u * x, n_o & 1u)) {
        ++n_o;
        tc_fence_after();
        const float inv = l > 0.0f || l != l ? 1.0f / l : 0.0f;
        const bool store = valid && bad_items[round & (BAD - 1)] != idx;
        __half* dst = p.out + tok * p.out_stride + head * DH;
#pragma unroll 1
        for (int c = 0; c < DH; c += 32) {
          uint32_t o[32];
          tmem_ld32(t_o + c, o);
          tmem_ld_wait();
          if (store) {
#pragma unroll
            for (int v = 0; v < 4; ++v) {
              uint4 h;
              h.x = pack_half2_sat(__uint_as_float(o[v * 8 + 0]) * inv, __uint_as_float(o[v * 8 + 1]) * inv);
              h.y = pack_half2_sat(__uint_as_float(o[v * 8 + 2]) * inv, __uint_as_float(o[v * 8 + 3]) * inv);
              h.z = pack_half2_sat(__uint_as_float(o[v * 8 + 4]) * inv, __uint_as_float(o[v * 8 + 5]) * inv);
              h.w = pack_half2_sat(__uint_as_float(o[v * 8 + 6]) * inv, __uint_as_float(o[v * 8 + 7]) * inv);
              *reinterpret_cast<uint4*>(dst + c + v * 8) = h;
            }
          }
        }
        tc_fence_before();
      }
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (*abort_flag) {
    if (tid == 0) atomicOr(p.r.status, HB_DEV_ATTN_WAIT_EXPIRED);
    for (int i = 0; i < 200; ++i) __nanosleep(1000);   // let requested copies and issued work land
    __syncthreads();
  }
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
  }
}

}  // namespace hb_kv8_tc
