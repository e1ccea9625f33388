// Attention over the 8-bit paged KV cache (causal, grouped query heads, ragged segments).
//
//   s_ij = scale * q_i . k_j (j <= pos_i);  o_i = sum_j softmax(s_i)_j v_j
//
// A segment has q_len * G columns for one KV head (G = Hq / Hkv; column c = row c / G, head c % G).  Segments of
// up to 16 (decode rows) take the body in this file, their keys cut into splits whose number depends on
// the segment's own length only; larger ones take the tcgen05 body of kv8_attention_tc.cuh in a launch
// of its own.  Each block walks items b, b + grid, ...; the segment of an item is found in a prefix sum
// over the segments that the block forms itself, so that nothing about the batch has to be known on the
// host and a captured launch follows the arrays.
//
// One decode item: four warps share the columns and take every fourth page.  A warp fetches a page's block of
// this KV head (K, V and scales: 2 - 4 KiB, contiguous) with one bulk copy into its own ring and
// computes transposed, so that the 16 keys of the page fill the 16 rows of the matrix instruction
// whatever G is:
//   S^T[16 keys, 8 cols] = K[16, DH] Q^T          A = codes of K converted to fp16 (exact), B = q
//   O^T[DH, 8 cols]     += V^T[DH, 16] P^T[16, 8]  A = codes of V, B = P^T (one 8 x 8 transpose per 8 keys)
// The scale of K multiplies the fp32 scores.  The scale 2^e of V is folded into the exponent: P holds
// 2^(s - m + e) with m the running maximum of s + e over the keys, and the sum takes 2^-e back out, so
// neither scale is ever rounded.
// Bound by HBM: 64 rows, 32 / 8 heads of 128, contexts of 512 to 4096 (300 MB) 64.5 us = 4.65 TB/s, ramp and tail
// included; 256 rows at 2048 keys 196 us = 5.5 TB/s.  The difference is the deal of the items: splits are equal within a segment
// only, and with contexts that differ the fullest block has 1.30 times the mean (its SM 1.10 times).  One row over 600 keys takes
// 10.1 us: the launches and one chain of look-ups, pages and join.  Splits of at least 512 keys, at most 64 (128 of them
// for contexts of 64 Ki keys: 102 us against 93, the join then reads twice the records).  Four blocks per SM with two pages per warp in flight: 63 us;
// three blocks with more stages 72; five (96 registers, spilled) 77.
#include <algorithm>

#include "kv8.cuh"

namespace {

using namespace hb_kv8;

constexpr int DEC_WARPS = 4;
constexpr int DEC_THREADS = DEC_WARPS * 32;
constexpr int STAGES = 2;   // page blocks of a warp in flight or in use: 16 warps of an SM keep up to 128 KiB
constexpr int TILE_COLS = 16;
constexpr int MIN_SPLIT_KEYS = 512, MAX_SPLITS = 64;
constexpr int MAX_SEGS = 8192;
constexpr uint64_t WAIT_NS = 1000000000ull;

struct AttnParams {
  Rows r;
  const __half* q;
  __half* out;
  int64_t q_stride, out_stride;
  float scale_log2;
  int32_t min_split;    // keys of a split, unless the segment is so long that it would have more than MAX_SPLITS
  int32_t max_splits;   // no segment has more
  int32_t by_row;       // how the records of a column are numbered: see record()
  float* part_o;        // [column][max_splits][DH]: weighted sums relative to their maximum
  float2* part_ml;      // [column][max_splits]: maximum (log2), sum
};

// Keys per split of a segment with `keys` keys: as few splits of at most min_split keys as there can be (no
// more than MAX_SPLITS), of equal size, a multiple of the 64 keys that the four warps take in turn.
__device__ __forceinline__ int split_keys(const AttnParams& p, int keys) {
  const int n = min(MAX_SPLITS, max(1, (keys + p.min_split - 1) / p.min_split));
  return ((keys + n - 1) / n + 63) / 64 * 64;
}
__device__ __forceinline__ int n_splits(const AttnParams& p, int keys) {
  const int per = split_keys(p, keys);
  return keys <= per ? 1 : (keys - 1) / per + 1;
}
// No segment of up to max_keys keys has more splits.
inline int splits_bound(int max_keys, int min_split) { return std::max(1, std::min(MAX_SPLITS, max_keys / min_split + 1)); }
// Columns that can have records: every row's heads, or 16 for each segment and KV head, whichever is less.
inline size_t record_columns(int n_rows, int n_segs, int n_kv_heads, int group, bool* by_row) {
  const size_t rows = static_cast<size_t>(n_rows) * n_kv_heads * group, segs = static_cast<size_t>(n_segs) * n_kv_heads * TILE_COLS;
  *by_row = rows <= segs;
  return std::min(rows, segs);
}

struct Seg { int q_start, q_len, pos_start, pt_start; };

__device__ __forceinline__ bool load_seg(const Rows& r, int s, Seg& g) {
  const int4 a = __ldg(reinterpret_cast<const int4*>(r.segs + s));
  const int4 b = __ldg(reinterpret_cast<const int4*>(r.segs + s) + 1);
  g.q_start = a.y; g.q_len = a.z; g.pos_start = a.w; g.pt_start = b.x;
  return seg_ok(r, g.q_start, g.q_len, g.pos_start, g.pt_start, b.y);
}

// Splits of a segment of the decode body: one to 16 columns (0: no rows, or rows for the chunk body).
__device__ __forceinline__ int splits_of(const AttnParams& p, const Seg& g) {
  const int cols = g.q_len * p.r.G;
  return cols < 1 || cols > TILE_COLS ? 0 : n_splits(p, g.pos_start + g.q_len);
}
// First record of column c of a segment's KV head.
__device__ __forceinline__ int64_t record(const AttnParams& p, int seg, const Seg& g, int head, int c) {
  const int64_t column = p.by_row ? static_cast<int64_t>(g.q_start + c / p.r.G) * (p.r.Hkv * p.r.G) + head * p.r.G + c % p.r.G
                                  : (static_cast<int64_t>(seg) * p.r.Hkv + head) * TILE_COLS + c;
  return column * p.max_splits;
}

// Segment that item idx belongs to: prefix[s] <= idx < prefix[s + 1].
__device__ __forceinline__ int find_seg(const int* prefix, int n_segs, int idx) {
  int lo = 0, hi = n_segs;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (prefix[mid] <= idx) lo = mid; else hi = mid;
  }
  return lo;
}

struct Item {
  Seg g;
  int seg, head, split, ns;
  int n_cols;
  int key0, key1;     // keys [key0, key1) of this split
  int all_see;        // last key of the split that every column sees
};

__device__ __forceinline__ void find_item(const AttnParams& p, const int* prefix, int idx, Item& it) {
  it.seg = find_seg(prefix, p.r.n_segs, idx);
  load_seg(p.r, it.seg, it.g);
  const int keys = it.g.pos_start + it.g.q_len, at = idx - prefix[it.seg];
  it.ns = splits_of(p, it.g);
  it.head = at % p.r.Hkv;
  it.split = at / p.r.Hkv;
  it.n_cols = it.g.q_len * p.r.G;
  const int per = it.ns > 1 ? split_keys(p, keys) : keys;
  it.key0 = it.split * per;
  it.key1 = min(keys, it.key0 + per);
  it.all_see = min(it.key1 - 1, it.g.pos_start);
}

// prefix[s] = items before segment s (items(segment) each); returns the total.  All threads of the block; ends
// with a barrier.
template <int THREADS, class F>
__device__ int build_prefix(const Rows& r, int* prefix, int* warp_sums, F&& items_of, bool report) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, n = r.n_segs;
  const int per = (n + THREADS - 1) / THREADS, from = min(n, tid * per), to = min(n, from + per);
  int sum = 0;
  for (int s = from; s < to; ++s) {
    Seg g;
    int items = 0;
    if (load_seg(r, s, g)) items = items_of(g);
    else if (report && blockIdx.x == 0) atomicOr(r.status, HB_DEV_ATTN_BAD_INDEX);
    prefix[s] = sum;
    sum += items;
  }
  int incl = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int v = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += v;
  }
  if (lane == 31) warp_sums[warp] = incl;
  __syncthreads();
  int base = incl - sum, total = 0;
#pragma unroll
  for (int w = 0; w < THREADS / 32; ++w) {
    if (w < warp) base += warp_sums[w];
    total += warp_sums[w];
  }
  for (int s = from; s < to; ++s) prefix[s] += base;
  if (tid == 0) prefix[n] = total;
  __syncthreads();
  return total;
}

}  // namespace

#include "kv8_attention_tc.cuh"

namespace {

template <int DH>
struct DecCfg {
  static constexpr int BLK = Block<DH>::BYTES;
  static constexpr int RING = DEC_WARPS * STAGES * BLK;
  static constexpr int ROW = 64 + 4;   // floats per column of the merge buffer (the odd quarter keeps the stores conflict-free)
  static constexpr int MERGE = DEC_WARPS * 8 * ROW * 4;          // 64 dimensions of one 8-column tile at a time
  static constexpr int ML = DEC_WARPS * TILE_COLS * 8;
  static constexpr int BARS = DEC_WARPS * STAGES * 8;
  static constexpr int FIXED = RING + MERGE + ML + BARS + 64;
};

__device__ __forceinline__ uint32_t transpose8x8(uint32_t v) {
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}

// What a warp keeps of its columns: the lane holds columns 8 nt + 2t and 8 nt + 2t + 1.
template <int DH, int NT>
struct State {
  uint32_t q[NT][DH / 16][2];
  float o[NT][DH / 16][4];
  float m[NT][2], l[NT][2];
  int lim[NT][2];   // last visible key of the lane's columns, -1 for unused ones
};

template <int DH, int NT>
__device__ __forceinline__ void begin(const AttnParams& p, const Item& it, State<DH, NT>& st) {
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int c = nt * 8 + g;
    const int col = min(c, it.n_cols - 1);
    const __half* src = p.q + (it.g.q_start + col / p.r.G) * p.q_stride + (it.head * p.r.G + col % p.r.G) * DH + t * 16;
#pragma unroll
    for (int hf = 0; hf < DH / 64; ++hf) {
      uint4 a = make_uint4(0u, 0u, 0u, 0u), b = a;
      if (c < it.n_cols) {
        a = __ldg(reinterpret_cast<const uint4*>(src + hf * 64));
        b = __ldg(reinterpret_cast<const uint4*>(src + hf * 64) + 1);
      }
      st.q[nt][hf * 4 + 0][0] = a.x; st.q[nt][hf * 4 + 0][1] = a.y;
      st.q[nt][hf * 4 + 1][0] = a.z; st.q[nt][hf * 4 + 1][1] = a.w;
      st.q[nt][hf * 4 + 2][0] = b.x; st.q[nt][hf * 4 + 2][1] = b.y;
      st.q[nt][hf * 4 + 3][0] = b.z; st.q[nt][hf * 4 + 3][1] = b.w;
    }
#pragma unroll
    for (int mt = 0; mt < DH / 16; ++mt) st.o[nt][mt][0] = st.o[nt][mt][1] = st.o[nt][mt][2] = st.o[nt][mt][3] = 0.0f;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int cc = nt * 8 + 2 * t + e;
      st.m[nt][e] = -INFINITY;
      st.l[nt][e] = 0.0f;
      st.lim[nt][e] = cc < it.n_cols ? min(it.key1 - 1, it.g.pos_start + cc / p.r.G) : -1;
    }
  }
}

// Replaces the NaN codes of a page's V by zero, in shared memory; returns a bit for each token that had one.  The warp.
template <int DH>
__device__ __noinline__ uint32_t drop_nan_page(uint32_t blk) {
  const int lane = threadIdx.x & 31;
  uint32_t bytes = 0;
#pragma unroll 1
  for (int c = 0; c < DH / 32; ++c) {
    const uint32_t at = blk + Block<DH>::V_OFF + c * 512 + lane * 16;
    uint4 v = lds128(at);
    const uint32_t here = drop_nan(v.x) | drop_nan(v.y) | drop_nan(v.z) | drop_nan(v.w);
    if (here) asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
    bytes |= here;
  }
  bytes = nan_tokens(bytes, lane & 3);
  if (bytes) fence_async_smem();   // the next copy into this stage comes behind these stores
  return bytes;
}

// One page (16 keys from `key`) out of shared memory at `blk`.
template <int DH, int NT>
__device__ __forceinline__ void page_step(const AttnParams& p, const Item& it, uint32_t blk, int key, State<DH, NT>& st) {
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  float ks, vs;
  asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(ks), "=f"(vs) : "r"(blk + Block<DH>::HDR));
  ks *= p.scale_log2;
  const int ev = exponent_of(vs);
  const float fev = static_cast<float>(ev), back = pow2f(max(-126, min(126, -ev)));
  // (two chains of accumulation: a matrix instruction waits for the one before it on the same sum)
  float s[NT][4], s1[NT][4];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) s[nt][0] = s[nt][1] = s[nt][2] = s[nt][3] = s1[nt][0] = s1[nt][1] = s1[nt][2] = s1[nt][3] = 0.0f;
#pragma unroll
  for (int hf = 0; hf < DH / 64; ++hf) {
    const uint4 ka = lds128(blk + hf * 1024 + g * 64 + t * 16), kb = lds128(blk + hf * 1024 + (g + 8) * 64 + t * 16);
    const uint32_t wa[4] = {ka.x, ka.y, ka.z, ka.w}, wb[4] = {kb.x, kb.y, kb.z, kb.w};
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      uint32_t a[4];
      e4m3x4_to_half2x2(wa[w], a[0], a[2]);
      e4m3x4_to_half2x2(wb[w], a[1], a[3]);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) mma_f16((w & 1) ? s1[nt] : s[nt], a, st.q[nt][hf * 4 + w][0], st.q[nt][hf * 4 + w][1]);
    }
  }
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int e = 0; e < 4; ++e) s[nt][e] += s1[nt][e];
  // scores in the log2 domain, plus V's exponent; invisible keys (only in pages that reach behind the last key
  // that every column sees) -inf
  const bool masked = key + PAGE - 1 > it.all_see;
  bool grow = false;
  float mx[NT][2];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      s[nt][e] = fmaf(s[nt][e], ks, fev);
      s[nt][2 + e] = fmaf(s[nt][2 + e], ks, fev);
      if (masked) {
        if (key + g > st.lim[nt][e]) s[nt][e] = -INFINITY;
        if (key + g + 8 > st.lim[nt][e]) s[nt][2 + e] = -INFINITY;
      }
      float m = fmaxf(s[nt][e], s[nt][2 + e]);
      m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 4));
      m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 8));
      m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 16));
      mx[nt][e] = m;
      grow |= m > st.m[nt][e] + 13.0f || (st.m[nt][e] == -INFINITY && m > -INFINITY);
    }
  }
  // The reference maximum moves only when a column's maximum has grown by more than 2^13 over it.  It is
  // kept 6 below the maximum it was taken from, so that P lies in [0, 2^13]: the small probabilities of a
  // long context stay normal fp16 numbers down to 2^-20 of the largest.
  if (__any_sync(0xffffffffu, grow)) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      float f[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float m_new = mx[nt][e] - 6.0f;
        const bool up = mx[nt][e] > -INFINITY && !(m_new <= st.m[nt][e]);
        f[e] = up ? ex2_approx(st.m[nt][e] - m_new) : 1.0f;   // -inf -> 0
        if (up) st.m[nt][e] = m_new;
        st.l[nt][e] *= f[e];
      }
#pragma unroll
      for (int mt = 0; mt < DH / 16; ++mt) {
        st.o[nt][mt][0] *= f[0]; st.o[nt][mt][1] *= f[1];
        st.o[nt][mt][2] *= f[0]; st.o[nt][mt][3] *= f[1];
      }
    }
  }
  // a page that reaches behind what the first row sees, in a segment of several rows: NaN codes of V go (in place)
  if (key + PAGE - 1 > it.g.pos_start && it.g.q_len > 1) {
    const uint32_t nan_at = drop_nan_page<DH>(blk);
    if (nan_at) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int last = min(st.lim[nt][e] - key, PAGE - 1);   // the column sees tokens 0 .. last of the page
          if (last >= 0 && (nan_at & ((2u << last) - 1u))) st.l[nt][e] = __uint_as_float(0x7fc00000u);
        }
    }
  }
  uint32_t pt[NT][2];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    float w[4];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const float m = st.m[nt][e] == -INFINITY ? 0.0f : st.m[nt][e];
      w[e] = ex2_approx(s[nt][e] - m);
      w[2 + e] = ex2_approx(s[nt][2 + e] - m);
      st.l[nt][e] = fmaf(w[e] + w[2 + e], back, st.l[nt][e]);
    }
    pt[nt][0] = transpose8x8(pack_half2(w[0], w[1]));
    pt[nt][1] = transpose8x8(pack_half2(w[2], w[3]));
  }
  // tokens past the request's last key hold whatever was there: their codes become zero (0 * NaN is NaN)
  uint32_t keep = 0xffffffffu;
  const int left = it.g.pos_start + it.g.q_len - key;
  const bool short_page = left < PAGE;
  if (short_page) {
    keep = (2 * t < left ? 0xffu : 0u) | (2 * t + 1 < left ? 0xff00u : 0u) | (2 * t + 8 < left ? 0xff0000u : 0u) |
           (2 * t + 9 < left ? 0xff000000u : 0u);
  }
#pragma unroll
  for (int c = 0; c < DH / 32; ++c) {
    const uint4 v = lds128(blk + Block<DH>::V_OFF + c * 512 + lane * 16);
    uint32_t wv[4] = {v.x, v.y, v.z, v.w};
    if (short_page) {
#pragma unroll
      for (int w = 0; w < 4; ++w) wv[w] &= keep;
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      uint32_t a[4];
      e4m3x4_to_half2x2(wv[2 * h], a[0], a[2]);
      e4m3x4_to_half2x2(wv[2 * h + 1], a[1], a[3]);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) mma_f16(st.o[nt][c * 2 + h], a, pt[nt][0], pt[nt][1]);
    }
  }
}

// A warp's ring of page blocks.  n counts the copies asked for, c those consumed, over the block's life.
struct Ring {
  uint32_t buf, bar;
  uint32_t n, c;
};

template <int DH>
__device__ __forceinline__ void request(const AttnParams& p, Ring& ring, int page, int head) {
  // every lane; lane 0 issues
  const uint32_t st = ring.n % STAGES;
  if ((threadIdx.x & 31) == 0) {
    const uint32_t bar = ring.bar + 8u * st;
    mbar_arrive_expect_tx(bar, Block<DH>::BYTES);
    bulk_load(ring.buf + st * Block<DH>::BYTES,
              p.r.arena + page * p.r.page_stride + static_cast<int64_t>(head) * Block<DH>::BYTES, Block<DH>::BYTES, bar);
  }
  ++ring.n;
}

// A warp's pages of an item: every fourth.
__device__ __forceinline__ int warp_pages(const Item& it) {
  const int warp = threadIdx.x >> 5, n = (it.key1 + PAGE - 1) / PAGE - it.key0 / PAGE;
  return n > warp ? (n - warp + DEC_WARPS - 1) / DEC_WARPS : 0;
}
// Page ids of the warp's pages [batch, batch + 32) of an item, one per lane (lanes behind the last page: 0).
__device__ __forceinline__ int load_ids(const AttnParams& p, const Item& it, int batch) {
  const int i = batch + (threadIdx.x & 31);
  return i < warp_pages(it) ? __ldg(p.r.page_ids + it.g.pt_start + it.key0 / PAGE + (threadIdx.x >> 5) + i * DEC_WARPS) : 0;
}
// Checks a batch of n ids (or 32, if there are more) and asks for its first pages.  False (and a report) if one is no
// page: nothing is asked for.  Which lanes have an id follows from n: no value of an id stands for "none".
template <int DH>
__device__ __forceinline__ bool start_batch(const AttnParams& p, const Item& it, int id, int n, Ring& ring) {
  const int lane = threadIdx.x & 31;
  if (__any_sync(0xffffffffu, lane < n && (id < 0 || id >= p.r.n_pages))) {
    if (lane == 0) atomicOr(p.r.status, HB_DEV_ATTN_BAD_INDEX);
    return false;
  }
  for (int i = 0; i < min(n, STAGES); ++i) request<DH>(p, ring, __shfl_sync(0xffffffffu, id, i), it.head);
  return true;
}

// One item; its first batch of pages (`id`) has been started (`ok`).  `before_join` runs when the last page has
// been computed: it starts the next item's pages, which then arrive while the warps are joined.
template <int DH, int NT, class F>
__device__ __forceinline__ bool run_item(const AttnParams& p, const Item& it, int id, bool ok, Ring& ring, uint8_t* smem, volatile uint32_t* abort_flag,
                                         F&& before_join) {
  using C = DecCfg<DH>;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
  State<DH, NT> st;
  begin<DH, NT>(p, it, st);
  const int mine = warp_pages(it), pg0 = it.key0 / PAGE + warp;
  for (int batch = 0; batch < mine && ok; batch += 32) {
    const int nb = min(32, mine - batch);
    if (batch > 0) {
      id = load_ids(p, it, batch);
      ok = start_batch<DH>(p, it, id, nb, ring);
      if (!ok) break;
    }
    for (int i = 0; i < nb; ++i) {
      const uint32_t sg = ring.c % STAGES;
      if (!__all_sync(0xffffffffu, mbar_wait(ring.bar + 8u * sg, (ring.c / STAGES) & 1u, abort_flag, WAIT_NS))) { ok = false; break; }
      page_step<DH, NT>(p, it, ring.buf + sg * Block<DH>::BYTES, (pg0 + (batch + i) * DEC_WARPS) * PAGE, st);
      ++ring.c;
      __syncwarp();   // every lane has read the stage
      if (i + STAGES < nb) request<DH>(p, ring, __shfl_sync(0xffffffffu, id, i + STAGES), it.head);
    }
  }
  if (!*abort_flag) before_join();
  // ---- join the four warps: common maximum, then the weighted sums through shared memory ----
  float* merge = reinterpret_cast<float*>(smem + C::RING);
  float2* ml = reinterpret_cast<float2*>(smem + C::RING + C::MERGE);
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      float l = st.l[nt][e];
      l += __shfl_xor_sync(0xffffffffu, l, 4);
      l += __shfl_xor_sync(0xffffffffu, l, 8);
      l += __shfl_xor_sync(0xffffffffu, l, 16);
      if (g == 0) ml[warp * TILE_COLS + nt * 8 + 2 * t + e] = make_float2(st.m[nt][e], l);
    }
  const bool all_ok = __syncthreads_and(ok) != 0;
  if (!all_ok && it.ns > 1 && tid < it.n_cols)   // a negative sum tells the join to leave the row alone
    p.part_ml[record(p, it.seg, it.g, it.head, tid) + it.split] = make_float2(-INFINITY, -1.0f);
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    float f[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      float m = -INFINITY;
#pragma unroll
      for (int w = 0; w < DEC_WARPS; ++w) m = fmaxf(m, ml[w * TILE_COLS + nt * 8 + 2 * t + e].x);
      f[e] = st.m[nt][e] == -INFINITY ? 0.0f : ex2_approx(st.m[nt][e] - m);
    }
#pragma unroll
    for (int hf = 0; hf < DH / 64; ++hf) {
      float* mine_at = merge + (warp * 8 + 2 * t) * C::ROW + g;
#pragma unroll
      for (int m4 = 0; m4 < 4; ++m4) {
        const int mt = hf * 4 + m4;
        mine_at[m4 * 16] = st.o[nt][mt][0] * f[0];
        mine_at[C::ROW + m4 * 16] = st.o[nt][mt][1] * f[1];
        mine_at[m4 * 16 + 8] = st.o[nt][mt][2] * f[0];
        mine_at[C::ROW + m4 * 16 + 8] = st.o[nt][mt][3] * f[1];
      }
      __syncthreads();
      if (all_ok) {
        // two neighbouring dimensions per thread
#pragma unroll
        for (int u = tid; u < 8 * 32; u += DEC_THREADS) {
          const int cc = u / 32, d = (u % 32) * 2, c = nt * 8 + cc;
          if (c >= it.n_cols) continue;
          float m = -INFINITY, l = 0.0f, x = 0.0f, y = 0.0f;
#pragma unroll
          for (int w = 0; w < DEC_WARPS; ++w) m = fmaxf(m, ml[w * TILE_COLS + c].x);
#pragma unroll
          for (int w = 0; w < DEC_WARPS; ++w) {
            const float2 a = ml[w * TILE_COLS + c];
            if (a.x > -INFINITY) l = fmaf(a.y, ex2_approx(a.x - m), l);
            const float2 b = *reinterpret_cast<const float2*>(merge + (w * 8 + cc) * C::ROW + d);
            x += b.x;
            y += b.y;
          }
          if (it.ns == 1) {
            const float inv = l > 0.0f || l != l ? 1.0f / l : 0.0f;
            __half* dst = p.out + (it.g.q_start + c / p.r.G) * p.out_stride + (it.head * p.r.G + c % p.r.G) * DH + hf * 64 + d;
            *reinterpret_cast<uint32_t*>(dst) = pack_half2_sat(x * inv, y * inv);
          } else {
            const int64_t rec = record(p, it.seg, it.g, it.head, c) + it.split;
            *reinterpret_cast<float2*>(p.part_o + rec * DH + hf * 64 + d) = make_float2(x, y);
            if (hf == 0 && d == 0) p.part_ml[rec] = make_float2(m, l);
          }
        }
      }
      __syncthreads();
    }
  }
  return all_ok;
}

// MAX_NT: 8-column tiles that a segment of the launch may have.  With one the blocks need fewer registers, and
// one more fits an SM; the arithmetic of a segment is the same in both.
template <int DH, int MAX_NT>
__global__ void __launch_bounds__(DEC_THREADS, MAX_NT == 1 ? 4 : 3)
kv8_attend_kernel(const AttnParams p) {
  grid_dep_wait();
  grid_dep_launch();   // (what follows waits for this kernel's end before it reads or writes)
  using C = DecCfg<DH>;
  extern __shared__ __align__(128) uint8_t smem[];
  const int tid = threadIdx.x, warp = tid >> 5;
  uint8_t* tail = smem + C::RING + C::MERGE + C::ML;
  volatile uint32_t* abort_flag = reinterpret_cast<volatile uint32_t*>(tail + C::BARS);
  int* warp_sums = reinterpret_cast<int*>(tail + C::BARS + 16);
  int* prefix = reinterpret_cast<int*>(smem + C::FIXED);
  Ring ring;
  ring.buf = smem_u32(smem) + warp * STAGES * C::BLK;
  ring.bar = smem_u32(tail) + warp * STAGES * 8;
  ring.n = ring.c = 0;
  if (tid < DEC_WARPS * STAGES) mbar_init(smem_u32(tail) + 8u * tid, 1);
  if (tid == 0) *abort_flag = 0u;
  mbar_init_fence();
  const int total = build_prefix<DEC_THREADS>(p.r, prefix, warp_sums, [&](const Seg& g) { return splits_of(p, g) * p.r.Hkv; }, true);   // its barriers publish the initialisation
  Item it;
  int id = 0;
  bool ok = true;
  if (static_cast<int>(blockIdx.x) < total) {
    find_item(p, prefix, blockIdx.x, it);
    id = load_ids(p, it, 0);
    ok = start_batch<DH>(p, it, id, warp_pages(it), ring);
  }
  for (int idx = blockIdx.x; idx < total; idx += gridDim.x) {
    // the next item and its page ids are looked up before this one's pages are computed
    const int next = idx + gridDim.x;
    Item nit = it;
    int nid = 0;
    bool nok = true;
    if (next < total) {
      find_item(p, prefix, next, nit);
      nid = load_ids(p, nit, 0);
    }
    auto start_next = [&]() {
      if (next < total) nok = start_batch<DH>(p, nit, nid, warp_pages(nit), ring);
    };
    // (a bad page id costs its item only)
    if (MAX_NT == 1 || it.n_cols <= 8) run_item<DH, 1>(p, it, id, ok, ring, smem, abort_flag, start_next);
    else run_item<DH, MAX_NT>(p, it, id, ok, ring, smem, abort_flag, start_next);
    it = nit;
    id = nid;
    ok = nok;
    if (*abort_flag) {
      // a wait ran out: report, let requested copies land, leave
      if (tid == 0) {
        atomicOr(p.r.status, HB_DEV_ATTN_WAIT_EXPIRED);
        for (int i = 0; i < 200; ++i) __nanosleep(1000);
      }
      __syncthreads();
      break;
    }
  }
}

// Joins the splits of one segment and KV head, a column per warp, in split order.
constexpr int JOIN_WARPS = 4;
template <int DH>
__global__ void __launch_bounds__(JOIN_WARPS * 32)
kv8_join_kernel(const AttnParams p) {
  grid_dep_wait();   // (the segments as much as the records)
  grid_dep_launch();
  const int seg = blockIdx.x / p.r.Hkv, head = blockIdx.x % p.r.Hkv, lane = threadIdx.x & 31;
  Seg g;
  const int ns = load_seg(p.r, seg, g) ? splits_of(p, g) : 0;
  if (ns <= 1) return;
  constexpr int V = DH / 32;   // dimensions per lane
  for (int c = threadIdx.x >> 5; c < g.q_len * p.r.G; c += JOIN_WARPS) {
    const int64_t rec = record(p, seg, g, head, c);
    // the splits' maxima and sums, up to two per lane
    constexpr int N = MAX_SPLITS / 32;
    float2 ml[N];
    float m = -INFINITY;
    bool gone = false;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      ml[i] = lane + 32 * i < ns ? p.part_ml[rec + lane + 32 * i] : make_float2(-INFINITY, 0.0f);
      gone |= ml[i].y < 0.0f;
      m = fmaxf(m, ml[i].x);
    }
    if (__any_sync(0xffffffffu, gone)) continue;   // a split that was given up
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    float l = 0.0f, x[V] = {};
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float fm = ml[i].x > -INFINITY ? ex2_approx(ml[i].x - m) : 0.0f;
      const int here = min(32, ns - 32 * i);
#pragma unroll 4
      for (int s = 0; s < here; ++s) {
        const float f = __shfl_sync(0xffffffffu, fm, s);
        l = fmaf(__shfl_sync(0xffffffffu, ml[i].y, s), f, l);
        const float* src = p.part_o + (rec + 32 * i + s) * DH + lane * V;
        if (V == 4) {
          const float4 v = *reinterpret_cast<const float4*>(src);
          x[0] = fmaf(v.x, f, x[0]); x[1] = fmaf(v.y, f, x[1]); x[2 % V] = fmaf(v.z, f, x[2 % V]); x[3 % V] = fmaf(v.w, f, x[3 % V]);
        } else {
          const float2 v = *reinterpret_cast<const float2*>(src);
          x[0] = fmaf(v.x, f, x[0]); x[1] = fmaf(v.y, f, x[1]);
        }
      }
    }
    const float inv = l > 0.0f || l != l ? 1.0f / l : 0.0f;
    __half* dst = p.out + (g.q_start + c / p.r.G) * p.out_stride + (head * p.r.G + c % p.r.G) * DH + lane * V;
#pragma unroll
    for (int i = 0; i < V; i += 2) *reinterpret_cast<uint32_t*>(dst + i) = pack_half2_sat(x[i] * inv, x[i + 1] * inv);
  }
}

template <int DH>
int launch(const AttnParams& p, int num_sms, cudaStream_t s, bool pdl, int* launches) {
  static DynSmemState configured[2];
  const int smem = DecCfg<DH>::FIXED + (p.r.n_segs + 1) * 4;
  if (smem > 227 * 1024) return HB_ERR_TOO_LARGE;
  const long long cols_bound = static_cast<long long>(p.r.max_q_len) * p.r.G;
  const bool narrow = cols_bound <= 8;
  auto kern = narrow ? kv8_attend_kernel<DH, 1> : kv8_attend_kernel<DH, 2>;
  if (hb_ensure_dyn_smem(reinterpret_cast<const void*>(kern), configured[narrow], smem) != HB_OK) return HB_ERR_CUDA;
  // no more blocks than the bounds of the call allow items
  const long long most = static_cast<long long>(p.r.n_segs) * p.r.Hkv * p.max_splits;
  int rc = hb_launch_kernel(kern, static_cast<unsigned>(std::min<long long>(most, (narrow ? 4ll : 3ll) * num_sms)), DEC_THREADS, smem, s, pdl, p);
  *launches = 1;
  if (rc == HB_OK && cols_bound > TILE_COLS) {   // segments for the chunk body are possible
    static DynSmemState tc_configured;
    const int tc_smem = hb_kv8_tc::Cfg<DH>::FIXED + (p.r.n_segs + 1) * 4 + hb_kv8_tc::MAX_SORTED * 4;
    if (tc_smem > 227 * 1024) return HB_ERR_TOO_LARGE;
    auto tc = hb_kv8_tc::kv8_chunk_kernel<DH>;
    if (hb_ensure_dyn_smem(reinterpret_cast<const void*>(tc), tc_configured, tc_smem) != HB_OK) return HB_ERR_CUDA;
    const long long tc_most = static_cast<long long>(p.r.n_segs) * p.r.Hkv * ((cols_bound + hb_kv8_tc::ROWS - 1) / hb_kv8_tc::ROWS);
    rc = hb_launch_kernel(tc, static_cast<unsigned>(std::min<long long>(tc_most, num_sms)), hb_kv8_tc::THREADS, tc_smem, s, true, p);
    ++*launches;
  }
  if (rc != HB_OK || p.max_splits == 1) return rc;
  ++*launches;
  return hb_launch_kernel(kv8_join_kernel<DH>, static_cast<unsigned>(p.r.n_segs) * p.r.Hkv, JOIN_WARPS * 32, 0, s, true, p);
}

}  // namespace

int hb_kv8_max_segs() { return MAX_SEGS; }
int hb_kv8_min_split_keys() { return MIN_SPLIT_KEYS; }

size_t hb_kv8_attention_scratch(const hb_model_cfg& cfg, int n_rows, int n_segs, int max_keys, int min_split) {
  const int splits = splits_bound(max_keys, min_split);
  bool by_row;
  const size_t columns = record_columns(n_rows, n_segs, cfg.n_kv_heads, cfg.n_heads / cfg.n_kv_heads, &by_row);
  return splits > 1 ? columns * splits * (static_cast<size_t>(cfg.head_dim) * 4 + 8) : 0;
}

int hb_launch_kv8_attention(hb_ctx* c, const hb_kv8::Rows& r, const void* q, int64_t q_stride, void* out, int64_t out_stride,
                            float scale, int min_split, void* workspace, cudaStream_t s, bool pdl, int* launches) {
  AttnParams p;
  p.r = r;
  p.q = static_cast<const __half*>(q);
  p.out = static_cast<__half*>(out);
  p.q_stride = q_stride;
  p.out_stride = out_stride;
  p.scale_log2 = scale * 1.4426950408889634f;
  p.min_split = min_split;
  p.max_splits = splits_bound(r.max_keys, min_split);
  bool by_row;
  const size_t columns = record_columns(r.n_rows, r.n_segs, r.Hkv, r.G, &by_row);
  p.by_row = by_row ? 1 : 0;
  p.part_o = static_cast<float*>(workspace);
  p.part_ml = reinterpret_cast<float2*>(p.part_o + columns * p.max_splits * c->cfg.head_dim);
  if (c->cfg.head_dim == 64) return launch<64>(p, c->num_sms, s, pdl, launches);
  if (c->cfg.head_dim == 128) return launch<128>(p, c->num_sms, s, pdl, launches);
  return HB_ERR_UNSUPPORTED;
}
