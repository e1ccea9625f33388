// Appending a step's rows to the 8-bit KV cache: RMS norm of every query and key head (optional), rotary
// positions over the first rot_dim dimensions, q stored as fp16, k and v quantised to e4m3 with one
// power-of-two scale per (page, KV head), K and V apart.
//
//   q, k:  y = x / sqrt(mean(x^2) + eps) * gain;  (y_a, y_b) <- (y_a c - y_b s, y_b c + y_a s)
//   block: e = smallest exponent with max |y| <= 448 * 2^e over its new rows (and its old exponent, if the
//          page already holds rows);  code = e4m3(y * 2^-e)
//
// Query warps take 8 heads of one row: norm, rotation, store.  The scale of a block
// of the cache needs all of its new rows at once, so a key / value task is one KV head of one page: the first
// row of its segment in that page (the leader) and the up to 16 rows that follow it.  DH / 8 lanes
// share a row, 8 dimensions each: 16-byte loads; the rotary partner (i + rot_dim / 2) sits at the same place of
// another lane.
//   All segments of up to SMALL_ROWS rows (decode): a warp per row and task, in one wave of blocks; a row that
//     does not lead has no key / value task.  Latency decides: 64 rows of the 7B shape 3.2 us.
//   Otherwise resident blocks walk over two kinds of tasks.  A page with more than SMALL_ROWS new rows is a
//     block's: each of the four warps has four of its slots, w has 2w, 2w + 1, 2w + 8, 2w + 9, the tokens of
//     whole words of V, so that a page that starts afresh is written in words out of registers.  SHARE tasks
//     look at the same 16 rows, find such leaders and share what they have to do (looking costs two
//     dependent loads, so few look).  A page with fewer new rows goes to the query warps of its leader.
//     4096 rows in 8 chunks, 32 / 8 heads of 128, norms and halves: 40.7 us = 2.32 TB/s (30.6 us without norms, in pairs;
//     26 where the pages begin with the rows).  No unit is full: the chain row, segment, page id, old scale and the
//     rows themselves decides, with the 16 warps per SM that 128 registers allow.  16 heads a warp 41.6 us, and 21.6
//     against 18.2 for 64 decode rows and 6 chunks; the rotary tables of both rows of a lane at once (spilled) 50.
#include <algorithm>

#include "kv8.cuh"

namespace {

using namespace hb_kv8;

constexpr int WARPS = 4;
constexpr int SMALL_ROWS = 3, SHARE = 8, HEADS = 8;   // see above

struct AppendParams {
  Rows r;
  const __half* qkv;
  __half* q_out;
  int64_t qkv_stride, q_stride;
  const __nv_bfloat16 *q_gain, *k_gain;
  float eps;
  const float *cos, *sin;
  int32_t rope_rows, rot, Hq;
};

__device__ __forceinline__ void unpack8(const uint4& v, float (&x)[8]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
    x[2 * i] = f.x;
    x[2 * i + 1] = f.y;
  }
}

// The rotary factors of a row for a lane's 8 dimensions: four pairs, or eight halves of pairs.
struct Turn {
  float c[8], s[8];
  int other;     // HALVES: lane that holds the partners
  bool turns;
};

template <int DH, bool HALVES>
__device__ __forceinline__ void load_turn(const AppendParams& p, int pos, int d0, Turn& t) {
  constexpr int LPR = DH / 8;
  const int lane = threadIdx.x & 31, sub = lane & (LPR - 1), half = p.rot >> 1;
  t.turns = d0 < p.rot;
  t.other = lane;
  if (!t.turns) return;
  const bool low = d0 < half;
  const size_t at = static_cast<size_t>(pos) * half + (HALVES ? (low ? d0 : d0 - half) : d0 >> 1);
  const float4* cp = reinterpret_cast<const float4*>(p.cos + at);
  const float4* sp = reinterpret_cast<const float4*>(p.sin + at);
  const float4 c0 = __ldg(cp), s0 = __ldg(sp);
  t.c[0] = c0.x; t.c[1] = c0.y; t.c[2] = c0.z; t.c[3] = c0.w;
  t.s[0] = s0.x; t.s[1] = s0.y; t.s[2] = s0.z; t.s[3] = s0.w;
  if (HALVES) {
    const float4 c1 = __ldg(cp + 1), s1 = __ldg(sp + 1);
    t.c[4] = c1.x; t.c[5] = c1.y; t.c[6] = c1.z; t.c[7] = c1.w;
    t.s[4] = s1.x; t.s[5] = s1.y; t.s[6] = s1.z; t.s[7] = s1.w;
    // half is a multiple of 8, so the partners are the same 8 elements of the lane half / 8 away
    t.other = (lane & ~(LPR - 1)) | (low ? sub + (half >> 3) : sub - (half >> 3));
    if (low) {
#pragma unroll
      for (int i = 0; i < 8; ++i) t.s[i] = -t.s[i];
    }
  }
}

// One row's head: norm (if there is a gain) and rotation.  All lanes of the warp.
template <int DH, bool HALVES>
__device__ __forceinline__ void norm_rotate(const AppendParams& p, const float (&g)[8], bool has_gain, const Turn& t, float (&x)[8]) {
  constexpr int LPR = DH / 8;
  if (has_gain) {
    uint64_t sq = 0;
#pragma unroll
    for (int i = 0; i < 8; i += 2) sq = fma2(pack2(x[i], x[i + 1]), pack2(x[i], x[i + 1]), sq);
    float ss, s1;
    unpack2(sq, ss, s1);
    ss += s1;
#pragma unroll
    for (int o = LPR / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
    const float inv = __frsqrt_rn(ss * (1.0f / DH) + p.eps);
#pragma unroll
    for (int i = 0; i < 8; i += 2) unpack2(mul2(mul2(pack2(x[i], x[i + 1]), pack2(inv, inv)), pack2(g[i], g[i + 1])), x[i], x[i + 1]);
  }
  if (p.rot == 0) return;
  if (!HALVES) {
    if (t.turns) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float a = x[2 * i], b = x[2 * i + 1];
        const uint64_t turned = mul2(pack2(-b, a), pack2(t.s[i], t.s[i]));
        unpack2(fma2(pack2(a, b), pack2(t.c[i], t.c[i]), turned), x[2 * i], x[2 * i + 1]);
      }
    }
  } else {
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = __shfl_sync(0xffffffffu, x[i], t.other);
    if (t.turns) {
#pragma unroll
      for (int i = 0; i < 8; i += 2)
        unpack2(fma2(pack2(x[i], x[i + 1]), pack2(t.c[i], t.c[i + 1]), mul2(pack2(y[i], y[i + 1]), pack2(t.s[i], t.s[i + 1]))), x[i], x[i + 1]);
    }
  }
}

__device__ __forceinline__ void load_gain(const __nv_bfloat16* gain, int d0, float (&g)[8]) {
  if (!gain) return;
  const uint4 v = __ldg(reinterpret_cast<const uint4*>(gain + d0));
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    g[2 * i] = __uint_as_float(w[i] << 16);
    g[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}

// Sixteen codes again under a larger scale (f = old scale / new scale = 2^(e_old - e_new) <= 1).
__device__ __forceinline__ uint4 rescale16(uint4 v, float f) {
  uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t lo, hi;
    e4m3x4_to_half2x2(w[i], lo, hi);
    const float2 a = __half22float2(*reinterpret_cast<__half2*>(&lo)), b = __half22float2(*reinterpret_cast<__half2*>(&hi));
    w[i] = floats_to_e4m3x4(a.x * f, a.y * f, b.x * f, b.y * f);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// Byte of (token, dimension d0 + i) in a block's V part.
__device__ __forceinline__ int v_byte(int tok, int d0, int i) {
  return (d0 >> 5) * 512 + (i * 4 + ((tok & 7) >> 1)) * 16 + ((d0 & 31) >> 3) * 4 + (tok >> 3) * 2 + (tok & 1);
}

struct RowAt { int seg, q_start, q_len, pos_start, pt_start; };

// Segment of a row; false for padding and for what does not fit together (*bad).
__device__ __forceinline__ bool locate(const AppendParams& p, int row, RowAt& a, bool* bad) {
  *bad = false;
  a.seg = __ldg(p.r.row_seg + row);
  if (a.seg == -1) return false;
  bool ok = a.seg >= 0 && a.seg < p.r.n_segs;
  if (ok) {
    const int4 u = __ldg(reinterpret_cast<const int4*>(p.r.segs + a.seg));      // kind, q_start, q_len, pos_start
    const int4 v = __ldg(reinterpret_cast<const int4*>(p.r.segs + a.seg) + 1);  // pt_start, pt_len, pool_slot, pool_mode
    a.q_start = u.y; a.q_len = u.z; a.pos_start = u.w; a.pt_start = v.x;
    ok = seg_ok(p.r, u.y, u.z, u.w, v.x, v.y) && row >= u.y && row - u.y < u.z && (p.rot == 0 || u.w + u.z <= p.rope_rows);
  }
  *bad = !ok;
  return ok;
}

// Whether a row is its segment's first in its page, and the rows from it on that share the page.
__device__ __forceinline__ bool leads(const RowAt& a, int row) {
  const int j = row - a.q_start;
  return j == 0 || ((a.pos_start + j) & (PAGE - 1)) == 0;
}
__device__ __forceinline__ int new_rows(const RowAt& a, int row) {
  const int j = row - a.q_start;
  return min(PAGE - ((a.pos_start + j) & (PAGE - 1)), a.q_len - j);
}

// HEADS query heads of a row from head0 on; false for rows of nobody.
template <int DH, bool HALVES>
__device__ __forceinline__ bool query_task(const AppendParams& p, int row, int head0, RowAt& a) {
  constexpr int LPR = DH / 8, RPW = 32 / LPR, ITERS = HEADS / RPW;
  const int lane = threadIdx.x & 31, which = lane / LPR, d0 = (lane & (LPR - 1)) * 8;
  const __half* src = p.qkv + row * p.qkv_stride + d0;
  // all of the warp's loads are in flight together, and while the row's segment and position are looked up
  uint4 raw[ITERS];
#pragma unroll
  for (int it = 0; it < ITERS; ++it) {
    const int head = head0 + it * RPW + which;
    raw[it] = head < p.Hq ? *reinterpret_cast<const uint4*>(src + head * DH) : make_uint4(0u, 0u, 0u, 0u);
  }
  bool bad;
  if (!locate(p, row, a, &bad)) {
    if (bad && lane == 0) atomicOr(p.r.status, HB_DEV_APPEND_BAD_INDEX);
    return false;
  }
  Turn t;
  load_turn<DH, HALVES>(p, a.pos_start + row - a.q_start, d0, t);
  float g[8] = {};
  load_gain(p.q_gain, d0, g);
  __half* dst = p.q_out + row * p.q_stride + d0;
#pragma unroll
  for (int it = 0; it < ITERS; ++it) {
    if (head0 + it * RPW >= p.Hq) break;
    const int head = head0 + it * RPW + which;
    float x[8];
    unpack8(raw[it], x);
    norm_rotate<DH, HALVES>(p, g, p.q_gain != nullptr, t, x);
    if (head < p.Hq) {
      uint4 o;
      o.x = pack_half2_sat2(x[0], x[1]); o.y = pack_half2_sat2(x[2], x[3]);
      o.z = pack_half2_sat2(x[4], x[5]); o.w = pack_half2_sat2(x[6], x[7]);
      *reinterpret_cast<uint4*>(dst + head * DH) = o;
    }
  }
  return true;
}

// A lane's share of one page's new rows: which of the page's slots they go to, and which are there.  The whole
// block works on a page (four slots per warp), or (SMALL) one warp (its rows in order).
template <int DH, bool SMALL>
struct Slots {
  static constexpr int LPR = DH / 8, RPW = 32 / LPR, ITERS = SMALL ? (SMALL_ROWS + RPW - 1) / RPW : 4 / RPW;
  int tid, warp, which, d0, slot0;
  bool have[ITERS];
  __device__ __forceinline__ Slots(int slot0_, int n_new) : slot0(slot0_) {
    tid = SMALL ? threadIdx.x & 31 : threadIdx.x;
    warp = tid >> 5;
    which = (tid & 31) / LPR;
    d0 = (tid & (LPR - 1)) * 8;
#pragma unroll
    for (int it = 0; it < ITERS; ++it) have[it] = at(it) >= slot0 && at(it) < slot0 + n_new;
  }
  __device__ __forceinline__ int at(int it) const {
    return SMALL ? slot0 + it * RPW + which : DH == 128 ? 2 * warp + which + 8 * it : 2 * warp + (which & 1) + 8 * (which >> 1);
  }
  // the rows' 8 dimensions of one head; `src` points at the leader's
  __device__ __forceinline__ void load(const __half* src, int64_t stride, uint4 (&raw)[ITERS]) const {
#pragma unroll
    for (int it = 0; it < ITERS; ++it)
      raw[it] = have[it] ? *reinterpret_cast<const uint4*>(src + d0 + (at(it) - slot0) * stride) : make_uint4(0u, 0u, 0u, 0u);
  }
  static __device__ __forceinline__ void sync() {
    if (SMALL) __syncwarp(); else __syncthreads();
  }
};

template <int N>
__device__ __forceinline__ float amax_of(const float (&x)[N][8]) {   // over the warp (NaN does not count; absent rows are zero)
  float m = 0.0f;
#pragma unroll
  for (int it = 0; it < N; ++it)
#pragma unroll
    for (int c = 0; c < 8; ++c) m = fmaxf(m, fabsf(x[it][c]));
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  return m;
}

// Quantises the rows x into one part (K or V) of a block.  amax is over all of the part's new rows; everyone has
// read the old exponent.
template <int DH, bool SMALL, bool IS_V>
__device__ __forceinline__ void store_part(const Slots<DH, SMALL>& sl, uint8_t* block, int e_old, float amax,
                                           const float (&x)[Slots<DH, SMALL>::ITERS][8]) {
  using S = Slots<DH, SMALL>;
  const bool fresh = sl.slot0 == 0;
  const int e = max(e_old, scale_exponent(amax)), d0 = sl.d0;
  const float inv = pow2f(-e);
  const bool grew = !fresh && e > e_old;
  if (sl.tid == 0 && (fresh || grew)) reinterpret_cast<float*>(block + Block<DH>::HDR)[IS_V ? 1 : 0] = pow2f(e);
  uint8_t* part = block + (IS_V ? Block<DH>::V_OFF : 0);
  if (grew || (SMALL && fresh)) {   // the part's codes again, under the new scale (or zeros); then the new rows' on top
    for (int c = sl.tid; c < DH; c += SMALL ? 32 : WARPS * 32) {
      uint4* at = reinterpret_cast<uint4*>(part) + c;
      *at = SMALL && fresh ? make_uint4(0u, 0u, 0u, 0u) : rescale16(*at, pow2f(e_old - e));
    }
    S::sync();
  }
  if (!IS_V) {
    // token rows of 64 dimensions: 8 codes per lane and row; the slots without a row of a fresh page become zero
    uint8_t* dst = part + (d0 >> 6) * 1024 + (d0 & 63);
#pragma unroll
    for (int it = 0; it < S::ITERS; ++it) {
      uint2 codes = make_uint2(floats_to_e4m3x4(x[it][0] * inv, x[it][1] * inv, x[it][2] * inv, x[it][3] * inv),
                               floats_to_e4m3x4(x[it][4] * inv, x[it][5] * inv, x[it][6] * inv, x[it][7] * inv));
      if (!sl.have[it]) codes = make_uint2(0u, 0u);   // (norm and rotation may have made NaN of the zeros of no row)
      if (sl.have[it] || (fresh && !SMALL)) *reinterpret_cast<uint2*>(dst + sl.at(it) * 64) = codes;
    }
  } else if (SMALL || !fresh) {
#pragma unroll
    for (int it = 0; it < S::ITERS; ++it) {
      if (sl.have[it]) {
#pragma unroll
        for (int c = 0; c < 8; c += 2) {
          const uint32_t two = floats_to_e4m3x2(x[it][c] * inv, x[it][c + 1] * inv);
          part[v_byte(sl.at(it), d0, c)] = static_cast<uint8_t>(two);
          part[v_byte(sl.at(it), d0, c + 1)] = static_cast<uint8_t>(two >> 8);
        }
      }
    }
  } else {
    // Word (dimension, t = warp) holds the warp's four tokens.  Each exchange with the lane that has the neighbouring
    // token (then, for DH = 64, the token 8 further) leaves a lane with half the dimensions and twice the bytes.
    constexpr int LPR = S::LPR;
    const bool odd = sl.which & 1;
    uint32_t u[8];   // this lane's bytes of the words: 0 and 2 (DH = 128), or 0 (DH = 64)
#pragma unroll
    for (int c = 0; c < 8; c += 2) {
      const uint32_t lo = floats_to_e4m3x2(x[0][c] * inv, x[0][c + 1] * inv);
      u[c] = lo & 0xffu;
      u[c + 1] = lo >> 8;
      if (DH == 128) {
        const uint32_t hi = floats_to_e4m3x2(x[S::ITERS - 1][c] * inv, x[S::ITERS - 1][c + 1] * inv);
        u[c] |= (hi & 0xffu) << 16;
        u[c + 1] |= (hi >> 8) << 16;
      }
    }
    uint32_t w[4];   // dimensions (odd ? 4 : 0) + 0 .. 3
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const uint32_t theirs = __shfl_xor_sync(0xffffffffu, odd ? u[c] : u[c + 4], LPR), mine = odd ? u[c + 4] : u[c];
      w[c] = odd ? (theirs | (mine << 8)) : (mine | (theirs << 8));
    }
    uint8_t* dst = part + (d0 >> 5) * 512 + ((odd ? 16 : 0) + sl.warp) * 16 + ((d0 & 31) >> 3) * 4;   // + 64 per dimension
    if (DH == 128) {
#pragma unroll
      for (int c = 0; c < 4; ++c) *reinterpret_cast<uint32_t*>(dst + c * 64) = w[c];
    } else {
      const bool up = sl.which >> 1;
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const uint32_t theirs = __shfl_xor_sync(0xffffffffu, up ? w[c] : w[c + 2], 2 * LPR), mine = up ? w[c + 2] : w[c];
        *reinterpret_cast<uint32_t*>(dst + (c + (up ? 2 : 0)) * 64) = up ? (theirs | (mine << 16)) : (mine | (theirs << 16));
      }
    }
  }
}

// The leader's block of one KV head, or null (and a report) if its page is none.
template <int DH>
__device__ __forceinline__ uint8_t* block_of(const AppendParams& p, const RowAt& a, int pos, int hk, bool report) {
  const int page = __ldg(p.r.page_ids + a.pt_start + pos / PAGE);
  if (page < 0 || page >= p.r.n_pages) {
    if (report) atomicOr(p.r.status, HB_DEV_APPEND_BAD_INDEX);
    return nullptr;
  }
  return p.r.arena + page * p.r.page_stride + static_cast<int64_t>(hk) * Block<DH>::BYTES;
}

template <int DH>
__device__ __forceinline__ int old_exponent(const uint8_t* block, int slot0, int is_v) {
  return slot0 == 0 ? E_MIN : max(E_MIN, min(E_MAX, exponent_of(reinterpret_cast<const float*>(block + Block<DH>::HDR)[is_v])));
}

// (One row after the other: the tables of both would not leave enough registers for the queries.)
template <int DH, bool HALVES, int N>
__device__ __forceinline__ void key_rows(const AppendParams& p, const int (&pos)[N], int d0, const uint4 (&raw)[N], float (&x)[N][8]) {
  float g[8] = {};
  load_gain(p.k_gain, d0, g);
#pragma unroll
  for (int it = 0; it < N; ++it) {
    Turn t;
    load_turn<DH, HALVES>(p, pos[it], d0, t);
    unpack8(raw[it], x[it]);
    norm_rotate<DH, HALVES>(p, g, p.k_gain != nullptr, t, x[it]);
  }
}

// One warp: K or V of one KV head, the rows (SMALL_ROWS at most) of a leader, `row`, that share its page.
template <int DH, bool HALVES, bool IS_V>
__device__ __forceinline__ void small_task(const AppendParams& p, int row, const RowAt& a, int hk) {
  using S = Slots<DH, true>;
  const int pos = a.pos_start + row - a.q_start;
  const S sl(pos & (PAGE - 1), new_rows(a, row));
  uint4 raw[S::ITERS];
  sl.load(p.qkv + row * p.qkv_stride + static_cast<int64_t>(p.Hq + (IS_V ? p.r.Hkv : 0) + hk) * DH, p.qkv_stride, raw);
  uint8_t* block = block_of<DH>(p, a, pos, hk, sl.tid == 0);
  if (!block) return;
  const int e_old = old_exponent<DH>(block, sl.slot0, IS_V ? 1 : 0);
  float x[S::ITERS][8];
  if (IS_V) {
#pragma unroll
    for (int it = 0; it < S::ITERS; ++it) unpack8(raw[it], x[it]);
  } else {
    int at[S::ITERS];
#pragma unroll
    for (int it = 0; it < S::ITERS; ++it) at[it] = sl.have[it] ? pos - sl.slot0 + sl.at(it) : pos;
    key_rows<DH, HALVES>(p, at, sl.d0, raw, x);
  }
  const float amax = amax_of(x);
  __syncwarp();   // every lane has read the old scale
  store_part<DH, true, IS_V>(sl, block, e_old, amax, x);
}

// The whole block: K and V of one KV head, the rows of a leader that share its page.
template <int DH, bool HALVES>
__device__ __forceinline__ void page_task(const AppendParams& p, int row, const RowAt& a, int hk, float2* warp_max) {
  using S = Slots<DH, false>;
  const int pos = a.pos_start + row - a.q_start;
  const S sl(pos & (PAGE - 1), new_rows(a, row));
  uint4 raw_k[S::ITERS], raw_v[S::ITERS];
  const __half* src = p.qkv + row * p.qkv_stride + static_cast<int64_t>(p.Hq + hk) * DH;
  sl.load(src, p.qkv_stride, raw_k);
  sl.load(src + p.r.Hkv * DH, p.qkv_stride, raw_v);
  uint8_t* block = block_of<DH>(p, a, pos, hk, sl.tid == 0);
  if (!block) return;   // (the same in every thread)
  const int ek = old_exponent<DH>(block, sl.slot0, 0), ev = old_exponent<DH>(block, sl.slot0, 1);
  float xk[S::ITERS][8], xv[S::ITERS][8];
  int at[S::ITERS];
#pragma unroll
  for (int it = 0; it < S::ITERS; ++it) {
    at[it] = sl.have[it] ? pos - sl.slot0 + sl.at(it) : pos;
  }
  key_rows<DH, HALVES>(p, at, sl.d0, raw_k, xk);
#pragma unroll
  for (int it = 0; it < S::ITERS; ++it) unpack8(raw_v[it], xv[it]);
  float2 m = make_float2(amax_of(xk), amax_of(xv));
  __syncthreads();   // the maxima of the block's last task have been read
  if ((threadIdx.x & 31) == 0) warp_max[sl.warp] = m;
  __syncthreads();   // (and the old scales, by everyone)
  m = warp_max[0];
#pragma unroll
  for (int w = 1; w < WARPS; ++w) m = make_float2(fmaxf(m.x, warp_max[w].x), fmaxf(m.y, warp_max[w].y));
  store_part<DH, false, false>(sl, block, ek, m.x, xk);
  store_part<DH, false, true>(sl, block, ev, m.y, xv);
}

template <int DH, bool HALVES>
__global__ void __launch_bounds__(WARPS * 32)
kv8_append_small_kernel(const AppendParams p, const int q_per_row, const int tasks) {
  grid_dep_wait();
  grid_dep_launch();
  const int64_t at = static_cast<int64_t>(blockIdx.x) * WARPS + (threadIdx.x >> 5);
  const int row = static_cast<int>(at / tasks), task = static_cast<int>(at % tasks);
  if (row >= p.r.n_rows) return;
  RowAt a;
  if (task < q_per_row) {
    query_task<DH, HALVES>(p, row, task * HEADS, a);
    return;
  }
  bool bad;
  if (!locate(p, row, a, &bad)) return;   // (bad rows are reported by the query warps)
  if (!leads(a, row)) return;
  const int kv = task - q_per_row;
  if (kv < p.r.Hkv) small_task<DH, HALVES, false>(p, row, a, kv);
  else small_task<DH, HALVES, true>(p, row, a, kv - p.r.Hkv);
}

template <int DH, bool HALVES>
__global__ void __launch_bounds__(WARPS * 32, 4)
kv8_append_kernel(const AppendParams p, const int q_per_row, const int q_tasks, const int n_tasks) {
  grid_dep_wait();
  grid_dep_launch();
  __shared__ float2 warp_max[WARPS];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, n_kv = 2 * p.r.Hkv;
  for (int task = blockIdx.x; task < n_tasks; task += gridDim.x) {   // (the query tasks first: some lead to long chains)
    if (task < q_tasks) {
      const int64_t at = static_cast<int64_t>(task) * WARPS + warp;
      const int row = static_cast<int>(at / q_per_row), share = static_cast<int>(at % q_per_row);
      RowAt a;
      if (row >= p.r.n_rows || !query_task<DH, HALVES>(p, row, share * HEADS, a)) continue;
      if (!leads(a, row) || new_rows(a, row) > SMALL_ROWS) continue;
      for (int kv = share; kv < n_kv; kv += q_per_row) {
        if (kv < p.r.Hkv) small_task<DH, HALVES, false>(p, row, a, kv);
        else small_task<DH, HALVES, true>(p, row, a, kv - p.r.Hkv);
      }
      continue;
    }
    const int row0 = (task - q_tasks) / SHARE * 16;
    RowAt mine = {};
    bool bad, lead = false;
    if (lane < 16 && row0 + lane < p.r.n_rows && locate(p, row0 + lane, mine, &bad))   // (bad rows are reported by the query warps)
      lead = leads(mine, row0 + lane) && new_rows(mine, row0 + lane) > SMALL_ROWS;
    const uint32_t leaders = __ballot_sync(0xffffffffu, lead);   // the same in every warp
    const int n = __popc(leaders) * p.r.Hkv;
    for (int i = (task - q_tasks) % SHARE; i < n; i += SHARE) {
      const int l = __fns(leaders, 0, i / p.r.Hkv + 1);
      RowAt a;
      a.seg = 0;
      a.q_start = __shfl_sync(0xffffffffu, mine.q_start, l);
      a.q_len = __shfl_sync(0xffffffffu, mine.q_len, l);
      a.pos_start = __shfl_sync(0xffffffffu, mine.pos_start, l);
      a.pt_start = __shfl_sync(0xffffffffu, mine.pt_start, l);
      page_task<DH, HALVES>(p, row0 + l, a, i % p.r.Hkv, warp_max);
    }
  }
}

template <int DH, bool HALVES>
int launch(const AppendParams& p, int num_sms, cudaStream_t s, bool pdl) {
  const long long rows = p.r.n_rows;
  if (p.r.max_q_len <= SMALL_ROWS) {
    const int q_per_row = (p.Hq + HEADS - 1) / HEADS, tasks = q_per_row + 2 * p.r.Hkv;
    const long long blocks = (rows * tasks + WARPS - 1) / WARPS;
    if (blocks > 0x7fffffffll) return HB_ERR_TOO_LARGE;
    return hb_launch_kernel(kv8_append_small_kernel<DH, HALVES>, static_cast<unsigned>(blocks), WARPS * 32, 0, s, pdl, p, q_per_row, tasks);
  }
  const int q_per_row = (p.Hq + HEADS - 1) / HEADS;
  const long long q_tasks = (rows * q_per_row + WARPS - 1) / WARPS, n_tasks = q_tasks + (rows + 15) / 16 * SHARE;
  if (n_tasks > 0x7fffffffll) return HB_ERR_TOO_LARGE;
  return hb_launch_kernel(kv8_append_kernel<DH, HALVES>, static_cast<unsigned>(std::min<long long>(n_tasks, 4ll * num_sms)), WARPS * 32, 0, s, pdl,
                          p, q_per_row, static_cast<int>(q_tasks), static_cast<int>(n_tasks));
}

}  // namespace

int hb_launch_kv8_append(hb_ctx* c, const hb_kv8::Rows& r, const hb_append_args& a, cudaStream_t s, bool pdl) {
  AppendParams p;
  p.r = r;
  p.qkv = static_cast<const __half*>(a.qkv);
  p.q_out = static_cast<__half*>(a.q_out);
  p.qkv_stride = a.qkv_stride;
  p.q_stride = a.q_stride;
  p.q_gain = static_cast<const __nv_bfloat16*>(a.q_gain);
  p.k_gain = static_cast<const __nv_bfloat16*>(a.k_gain);
  p.eps = a.norm_eps;
  p.cos = a.rope_cos;
  p.sin = a.rope_sin;
  p.rope_rows = a.rope_rows;
  p.rot = a.rot_dim;
  p.Hq = c->cfg.n_heads;
  const bool halves = a.rope_layout == HB_ROPE_HALVES;
  if (c->cfg.head_dim == 64) return halves ? launch<64, true>(p, c->num_sms, s, pdl) : launch<64, false>(p, c->num_sms, s, pdl);
  if (c->cfg.head_dim == 128) return halves ? launch<128, true>(p, c->num_sms, s, pdl) : launch<128, false>(p, c->num_sms, s, pdl);
  return HB_ERR_UNSUPPORTED;
}
