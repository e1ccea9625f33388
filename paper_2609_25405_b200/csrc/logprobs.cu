// Scoring of logits rows: log probability of a given token, entropy, the k best alternatives, in one pass
// over the logits.
//
//   m = max x,  T = sum over all but one maximum of e^(x - m),  S = sum (x - m) e^(x - m)
//   log p_i = (x_i - m) - log1p(T);   H = log1p(T) - S / (1 + T)
// The maximum's own term is the 1 of 1 + T and is never added to the small ones: a row that is nearly
// certain keeps its entropy to full relative precision.
//
// A row is cut into chunks of 16 KiB, four of them make a slice that a CTA holds in shared memory at a time
// (bulk copies), and up to 8 parts of whole slices make the row.  The parts are joined in order, whoever
// computed them: with few rows a cluster shares a row, with many one CTA takes all its parts, and the bits
// are the same.  With a slice at hand the CTA passes over it three times: its maximum (while the chunks
// arrive), the two sums relative to that maximum, the logits that can be alternatives.  Then the next
// slice's chunks are asked for.  Bound by HBM for many rows: three CTAs per SM keep up to 192 KiB in
// flight and overlap each other's loads, sums and selections.  400 rows of 128256 in fp32: 39 us = 5.3 TB/s without
// alternatives, 54 us with 20 (about 20 instructions per logit in all, issue slots 59 % busy).  2048 rows of 32000 in
// fp16: 33 us = 4.0 TB/s; there the one exponential per logit on the 16-per-clock unit takes 15 of them.  One
// row of 128256 takes 8.3 us: a cluster of 8, one slice each, and the join.
//
// Alternatives are compared as 64-bit keys: the logit's bits made orderable, then the complement of its
// index, so that all keys differ, equal logits rank by index, and nothing depends on the order in which
// threads arrive.  The k-th largest of the maxima of 64 groups of four threads bounds the k-th best from
// below; what reaches it (a few more than k) is collected and ranked.  If ties or a hostile arrangement
// let too many through, the bound is taken over keys instead; if even that lets too many through, or NaN has to be
// ranked, the k best are found one by one.
#include <algorithm>

#include "hb_internal.h"
#include "ptx.cuh"

namespace {

constexpr int THREADS = 256, WARPS = THREADS / 32;
constexpr int MAX_VOCAB = 1 << 20;
constexpr int MAX_K = HB_LOGPROBS_MAX_K;
constexpr int GROUPS = THREADS / 4;
constexpr int MAX_PARTS = 8;
constexpr float LOG2E = 1.4426950408889634f;
static_assert(GROUPS >= MAX_K, "the bound needs k groups");

constexpr int CHUNK = 16384, CHUNKS = 4;             // bytes of a chunk, chunks a CTA holds
constexpr int VECS = CHUNK / (THREADS * 16);          // 16-byte vectors of a chunk per thread
constexpr int CAP = 512;                              // candidates that can be ranked at once
constexpr uint64_t WAIT_NS = 1000000000ull;
template <typename T>
struct Shape {
  static constexpr int V = 16 / static_cast<int>(sizeof(T)), PER_CHUNK = CHUNK / static_cast<int>(sizeof(T));
};

struct Params {
  const void* logits;
  int64_t row_stride;
  int n_rows, vocab, k, parts;
  const int32_t* tokens;
  float *out_logprob, *out_entropy, *out_top_logprobs;
  int32_t* out_top_ids;
  uint32_t* status;
};

struct Rec { float m, T, S; };   // m = -inf: no logit above -inf so far (T and S are 0, or NaN)

__device__ __forceinline__ float max_nan(float a, float b) {   // NaN if either is
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

__device__ __forceinline__ Rec join(Rec a, Rec b) {
  if (b.m > a.m) { const Rec t = a; a = b; b = t; }
  if (b.m == -INFINITY) return Rec{a.m, a.T + b.T, a.S + b.S};
  // (far below the maximum nothing is left of b; the clamp keeps d finite: masks of the type's lowest value)
  const float d = max_nan(b.m - a.m, -200.0f), f = expf(d), w = 1.0f + b.T;
  return Rec{a.m, fmaf(f, w, a.T), fmaf(f, fmaf(d, w, b.S), a.S)};
}

// Orderable bits of a logit; NaN below -inf, both zeros alike (-0 + 0 is +0).
__device__ __forceinline__ uint32_t order(float x) {
  const uint32_t u = __float_as_uint(x + 0.0f);
  return x != x ? 0u : (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
__device__ __forceinline__ uint64_t make_key(float x, int idx) { return (static_cast<uint64_t>(order(x)) << 32) | static_cast<uint32_t>(~idx); }
__device__ __forceinline__ float key_value(uint64_t key) {
  const uint32_t o = static_cast<uint32_t>(key >> 32);
  return o == 0u ? __uint_as_float(0x7fc00000u) : __uint_as_float((o & 0x80000000u) ? (o & 0x7fffffffu) : ~o);
}

__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T from_f(float v);
template <> __device__ __forceinline__ float from_f<float>(float v) { return v; }
template <> __device__ __forceinline__ __half from_f<__half>(float v) { return __float2half_rn(v); }
// max over the warp of a value that is not NaN
__device__ __forceinline__ float warp_max(float v) {
  float r;
  asm("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
  return r;
}

// The 16 bytes of a chunk's vector as floats.
template <typename T>
__device__ __forceinline__ void widen(const uint4& raw, float (&x)[Shape<T>::V]) {
  const T* e = reinterpret_cast<const T*>(&raw);
#pragma unroll
  for (int j = 0; j < Shape<T>::V; ++j) x[j] = to_f(e[j]);
}
// Largest of a vector's logits; a NaN does not count (-inf if there is nothing else).
template <typename T>
__device__ __forceinline__ float vector_max(const uint4& raw);
template <>
__device__ __forceinline__ float vector_max<float>(const uint4& raw) {
  return fmaxf(fmaxf(__uint_as_float(raw.x), __uint_as_float(raw.y)), fmaxf(__uint_as_float(raw.z), __uint_as_float(raw.w)));
}
template <>
__device__ __forceinline__ float vector_max<__half>(const uint4& raw) {
  const __half2* h = reinterpret_cast<const __half2*>(&raw);
  const __half2 m = __hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3]));
  return fmaxf(__low2float(m), __high2float(m));
}

// Threads per key when n keys are ranked against each other.
__device__ __forceinline__ int share(int n) { return n <= THREADS / 8 ? 8 : n <= THREADS / 4 ? 4 : n <= THREADS / 2 ? 2 : 1; }

// The k largest of keys[0 .. n) (all different, 0 = none) into best[], best first.  All threads; the caller
// separates the calls by barriers.
__device__ __forceinline__ void rank_keys(const uint64_t* keys, int n, int k, uint64_t* best) {
  const int per = share(n), part = threadIdx.x & (per - 1);
  for (int i0 = 0; i0 < n; i0 += THREADS / per) {
    const int i = i0 + threadIdx.x / per;
    const uint64_t mine = i < n ? keys[i] : ~0ull;
    int above = 0;
#pragma unroll 4
    for (int j = part; j < n; j += per) above += keys[j] > mine;
    for (int o = 1; o < per; o <<= 1) above += __shfl_xor_sync(0xffffffffu, above, o);
    if (part == 0 && i < n && mine != 0 && above < k) best[above] = mine;
  }
}

// TOP: alternatives are asked for (p.k > 0); scoring alone does without the code that looks for them.
template <typename T, bool ALIGNED, bool TOP>
__global__ void __launch_bounds__(THREADS, 3)
logprobs_kernel(const Params p) {
  using H = Shape<T>;
  constexpr int V = H::V;
  extern __shared__ __align__(128) uint8_t smem[];       // CHUNKS chunks
  __shared__ uint64_t cand[CAP];
  __shared__ uint64_t lists[2][MAX_K];                   // best of this CTA's slice; they swap roles
  __shared__ uint64_t gathered[2][MAX_PARTS * MAX_K];  // rank 0: every rank's list, rows alternating
  __shared__ Rec recs[2][MAX_PARTS];                     // rank 0: every part's record
  __shared__ uint64_t group_max[GROUPS];
  __shared__ uint64_t key_bound;
  __shared__ float val_bound, warp_val[WARPS], warp_s[WARPS], warp_q[WARPS];
  __shared__ int n_cand;
  __shared__ uint64_t bars[CHUNKS];
  __shared__ uint32_t abort_flag;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  uint32_t rank, size;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(size));
  const int n_chunks = (p.vocab + H::PER_CHUNK - 1) / H::PER_CHUNK, per_part = (n_chunks + p.parts - 1) / p.parts;
  const int parts_here = p.parts / static_cast<int>(size), part0 = static_cast<int>(rank) * parts_here, part1 = part0 + parts_here;
  const uint32_t bar0 = smem_u32(bars), smem0 = smem_u32(smem);
  if (tid == 0) {
    for (int c = 0; c < CHUNKS; ++c) mbar_init(bar0 + 8 * c, 1);
    abort_flag = 0u;
    mbar_init_fence();
  }
  __syncthreads();
  // Up to CHUNKS chunks of `row` from c0 on, none from `to` on, into shared memory.  One thread copies whole
  // 16-byte pieces; what is left of the last chunk is filled up by everyone in `complete`.
  auto request = [&](int row, int c0, int to) {
    if (ALIGNED && tid == 0) {
      for (int c = 0; c < CHUNKS && c0 + c < to; ++c) {
        const long long left = static_cast<long long>(p.vocab - (c0 + c) * H::PER_CHUNK) * static_cast<int>(sizeof(T));
        const uint32_t bytes = left >= CHUNK ? CHUNK : static_cast<uint32_t>(left) & ~15u;
        mbar_arrive_expect_tx(bar0 + 8 * c, bytes);
        if (bytes)
          asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                       ::"r"(smem0 + c * CHUNK), "l"(static_cast<const T*>(p.logits) + row * p.row_stride + static_cast<int64_t>(c0 + c) * H::PER_CHUNK),
                         "r"(bytes), "r"(bar0 + 8 * c) : "memory");
      }
    }
  };
  // Elements of chunk slot c that no copy brings: the row's last few (or all, if rows are not aligned), -inf behind them.
  auto complete = [&](const T* logits, int c0, int to) {
    T* dst = reinterpret_cast<T*>(smem);
    for (int c = 0; c < CHUNKS && c0 + c < to; ++c) {
      const int base = (c0 + c) * H::PER_CHUNK, here = min(H::PER_CHUNK, p.vocab - base);
      for (int i = (ALIGNED ? here & ~(V - 1) : 0) + tid; i < H::PER_CHUNK; i += THREADS)
        dst[c * H::PER_CHUNK + i] = i < here ? logits[base + i] : from_f<T>(-INFINITY);
    }
  };
  uint32_t phases = 0;   // one bit per chunk slot
  int buf = 0;
  const int n_clusters = gridDim.x / size;
  int row = blockIdx.x / size;
  auto first_of = [&](int part) { return min(n_chunks, part * per_part); };
  if (row < p.n_rows) request(row, first_of(part0), first_of(part0 + 1));
  // rank 0's shared memory may be written once its CTA has started
  if (size > 1) cluster_sync();
  for (; row < p.n_rows; row += n_clusters, buf ^= 1) {
    const T* logits = static_cast<const T*>(p.logits) + row * p.row_stride;
    Rec rec{-INFINITY, 0.0f, 0.0f};
    int cur = 0, have = 0, part = part0, c0 = first_of(part0), to = first_of(part0 + 1);
    for (bool more = true; more;) {
      const int held = min(CHUNKS, to - c0);   // (a part behind the last chunk has none)
      const bool part_ends = c0 + CHUNKS >= to, row_ends = part_ends && part + 1 == part1;
      const int next_part = part_ends ? part + 1 : part, next_c0 = part_ends ? first_of(part + 1) : c0 + CHUNKS;
      auto ask_next = [&]() {
        if (!row_ends) request(row, next_c0, first_of(next_part + 1));
        else if (row + n_clusters < p.n_rows) request(row + n_clusters, first_of(part0), first_of(part0 + 1));
      };
      complete(logits, c0, to);
      // ---- the slice's maximum ----
      float mx = -INFINITY;
      if (!ALIGNED || p.vocab < (c0 + held) * H::PER_CHUNK) __syncthreads();   // what `complete` wrote
      for (int c = 0; c < held; ++c) {
        if (ALIGNED) mbar_wait(bar0 + 8 * c, (phases >> c) & 1u, &abort_flag, WAIT_NS);     // (expired: reported at the end)
        const uint4* vec = reinterpret_cast<const uint4*>(smem + c * CHUNK) + tid;
#pragma unroll
        for (int v = 0; v < VECS; ++v) mx = fmaxf(mx, vector_max<T>(vec[v * THREADS]));
      }
      phases ^= (1u << held) - 1u;
      if (mx != mx) mx = -INFINITY;
      {
        const float w = warp_max(mx);
        if (lane == 0) warp_val[warp] = w;
        if (TOP) {
          float g = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
          g = fmaxf(g, __shfl_xor_sync(0xffffffffu, g, 2));
          if ((tid & 3) == 0) group_max[tid >> 2] = order(g);
        }
        if (tid == 0) { n_cand = 0; val_bound = -INFINITY; }
      }
      __syncthreads();
      float M = warp_val[0];
#pragma unroll
      for (int w = 1; w < WARPS; ++w) M = fmaxf(M, warp_val[w]);
      const float ref = M == -INFINITY ? 0.0f : M;
      // Only logits that reach `low` (and then keys above `floor_key`) can be alternatives: the k-th best so far,
      // or, while there are fewer, the k-th largest group maximum (equal ones by group).
      const bool listed = TOP && have == p.k;
      uint64_t floor_key = 0;
      float low = INFINITY;
      if (TOP && listed) {
        floor_key = lists[cur][p.k - 1];
        low = key_value(floor_key);
        if (low != low) low = -INFINITY;   // (NaN is among them)
      } else if (TOP) {
        const uint64_t mine = group_max[tid >> 2];
        int above = 0;
#pragma unroll
        for (int i = 0; i < GROUPS / 4; ++i) {
          const int g = i * 4 + (tid & 3);
          above += group_max[g] > mine || (group_max[g] == mine && g < (tid >> 2));
        }
        above += __shfl_xor_sync(0xffffffffu, above, 1);
        above += __shfl_xor_sync(0xffffffffu, above, 2);
        if ((tid & 3) == 0 && above == p.k - 1) val_bound = key_value(mine << 32);
        __syncthreads();
        low = val_bound;
      }
      auto keep = [&](float x, int idx, uint64_t bound) {
        if (idx < p.vocab) {
          const uint64_t key = make_key(x, idx);
          if (key > bound) {
            const int place = atomicAdd(&n_cand, 1);
            if (place < CAP - MAX_K) cand[place] = key;
          }
        }
      };
      // ---- the sums, and the logits that reach the bound ----
      const bool reaches = TOP && mx >= low;
      float s, q;
      {
        // two logits per instruction.  Below -200 the exponential is zero; the clamp keeps -inf out of the
        // product, and NaN comes through
        uint64_t s2[2] = {0, 0}, q2[2] = {0, 0};
        const uint64_t minus = pack2(-ref, -ref), log2e = pack2(LOG2E, LOG2E);
        for (int c = 0; c < held; ++c) {
          const uint4* vec = reinterpret_cast<const uint4*>(smem + c * CHUNK) + tid;
#pragma unroll
          for (int v = 0; v < VECS; ++v) {
            float x[V];
            const uint4 raw = vec[v * THREADS];
            widen<T>(raw, x);
            if (reaches && vector_max<T>(raw) >= low) {
#pragma unroll
              for (int e = 0; e < V; ++e)
                if (x[e] >= low) keep(x[e], (c0 + c) * H::PER_CHUNK + (v * THREADS + tid) * V + e, floor_key);
            }
#pragma unroll
            for (int e = 0; e < V; e += 2) {
              float a, b;
              unpack2(add2(pack2(x[e], x[e + 1]), minus), a, b);
              const uint64_t d = pack2(max_nan(a, -200.0f), max_nan(b, -200.0f));
              unpack2(mul2(d, log2e), a, b);
              const uint64_t w = pack2(ex2_approx(a), ex2_approx(b));
              s2[(e / 2) & 1] = add2(s2[(e / 2) & 1], w);
              q2[(e / 2) & 1] = fma2(d, w, q2[(e / 2) & 1]);
            }
          }
        }
        float a, b;
        unpack2(add2(s2[0], s2[1]), a, b);
        s = a + b;
        unpack2(add2(q2[0], q2[1]), a, b);
        q = a + b;
      }
      {
        // both over the warp: the lower half of the lanes goes on with s, the upper half with q
        const bool up = lane >= 16;
        float v = (up ? q : s) + __shfl_xor_sync(0xffffffffu, up ? s : q, 16);
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        if (lane == 0) warp_s[warp] = v;
        if (lane == 16) warp_q[warp] = v;
      }
      fence_async_smem();   // this slice's accesses to shared memory, before copies into it
      __syncthreads();
      int n = n_cand;
      s = warp_s[0];
      q = warp_q[0];
#pragma unroll
      for (int w = 1; w < WARPS; ++w) { s += warp_s[w]; q += warp_q[w]; }
      // One of the maxima is the 1 of 1 + T.  While the rest is not small against it, it can be taken off
      // the sum; else the sum is formed again without the maxima, which are counted.
      float T_ = M == -INFINITY ? s : s - 1.0f;
      bool reread = false;   // the slice was read after the last barrier
      if (M > -INFINITY && T_ < 0.25f) {
        reread = true;
        float tops = 0.0f, small = 0.0f;
        for (int c = 0; c < held; ++c) {
          const uint4* vec = reinterpret_cast<const uint4*>(smem + c * CHUNK) + tid;
          for (int v = 0; v < VECS; ++v) {
            float x[V];
            widen<T>(vec[v * THREADS], x);
#pragma unroll
            for (int e = 0; e < V; ++e) {
              const float d = max_nan(x[e] - ref, -200.0f);
              tops += d == 0.0f ? 1.0f : 0.0f;
              small += d == 0.0f ? 0.0f : ex2_approx(d * LOG2E);
            }
          }
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
          small += __shfl_xor_sync(0xffffffffu, small, o);
          tops += __shfl_xor_sync(0xffffffffu, tops, o);
        }
        __syncthreads();
        if (lane == 0) { warp_s[warp] = small; warp_val[warp] = tops; }
        __syncthreads();
        T_ = 0.0f;
        tops = -1.0f;
        for (int w = 0; w < WARPS; ++w) { T_ += warp_s[w]; tops += warp_val[w]; }
        T_ += tops;
      }
      rec = join(rec, Rec{M, T_, q});
      // ---- alternatives ----
      if (TOP) {
        // largest key of this thread that is below `limit` (0: none)
        auto best_below = [&](uint64_t limit) {
          uint64_t best = 0;
          for (int c = 0; c < held; ++c)
            for (int v = 0; v < VECS; ++v) {
              float x[V];
              widen<T>(reinterpret_cast<const uint4*>(smem + c * CHUNK)[v * THREADS + tid], x);
#pragma unroll
              for (int e = 0; e < V; ++e) {
                const int idx = (c0 + c) * H::PER_CHUNK + (v * THREADS + tid) * V + e;
                const uint64_t key = make_key(x[e], idx);
                if (idx < p.vocab && key < limit && key > best) best = key;
              }
            }
          return best;
        };
        if (n > CAP - MAX_K) {
          reread = true;
          // too many reach it: a bound over keys, which are all different
          __syncthreads();
          uint64_t best = reaches ? best_below(~0ull) : 0ull;
          best = max(best, __shfl_xor_sync(0xffffffffu, best, 1));
          best = max(best, __shfl_xor_sync(0xffffffffu, best, 2));
          if ((tid & 3) == 0) group_max[tid >> 2] = best;
          if (tid == 0) { n_cand = 0; key_bound = 0; }
          __syncthreads();
          const uint64_t mine = group_max[tid >> 2];
          int above = 0;
          for (int g = tid & 3; g < GROUPS; g += 4) above += group_max[g] > mine;
          above += __shfl_xor_sync(0xffffffffu, above, 1);
          above += __shfl_xor_sync(0xffffffffu, above, 2);
          if ((tid & 3) == 0 && mine != 0 && above == p.k - 1) key_bound = mine - 1;
          __syncthreads();
          const uint64_t bound = max(floor_key, key_bound);
          if (reaches)
            for (int c = 0; c < held; ++c)
              for (int v = 0; v < VECS; ++v) {
                float x[V];
                widen<T>(reinterpret_cast<const uint4*>(smem + c * CHUNK)[v * THREADS + tid], x);
#pragma unroll
                for (int e = 0; e < V; ++e)
                  if (x[e] >= low) keep(x[e], (c0 + c) * H::PER_CHUNK + (v * THREADS + tid) * V + e, bound);
              }
          __syncthreads();
          n = n_cand;
        }
        const int there = min(min(to * H::PER_CHUNK, p.vocab) - c0 * H::PER_CHUNK, held * H::PER_CHUNK);   // logits of this slice
        if (n > CAP - MAX_K || (!listed && n < min(p.k, there))) {
          // one by one
          reread = true;
          uint64_t limit = ~0ull;
          int found = 0;
          for (; found < p.k; ++found) {
            uint64_t best = best_below(limit);
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) best = max(best, __shfl_xor_sync(0xffffffffu, best, o));
            __syncthreads();
            if (lane == 0) group_max[warp] = best;
            __syncthreads();
            for (int w = 0; w < WARPS; ++w) best = max(best, group_max[w]);
            if (best == 0) break;
            if (tid == 0) cand[found] = best;
            limit = best;
          }
          n = found;
        }
      }
      if (reread) {
        fence_async_smem();
        __syncthreads();
      }
      ask_next();   // nobody needs the slice any more
      if (TOP && n > 0) {
        // rank what was collected and what earlier slices left
        if (tid < have) cand[n + tid] = lists[cur][tid];
        if (tid < MAX_K) lists[cur ^ 1][tid] = 0;
        __syncthreads();
        rank_keys(cand, n + have, p.k, lists[cur ^ 1]);
        cur ^= 1;
        have = min(p.k, n + have);
        __syncthreads();
      }
      if (part_ends) {   // its record goes to rank 0
        if (tid == 0) {
          const uint32_t rec_to = map_to_rank(smem_u32(&recs[buf][part]), 0);
          st_cluster_u32(rec_to, __float_as_uint(rec.m));
          st_cluster_u32(rec_to + 4, __float_as_uint(rec.T));
          st_cluster_u32(rec_to + 8, __float_as_uint(rec.S));
        }
        rec = Rec{-INFINITY, 0.0f, 0.0f};
      }
      more = !row_ends;
      part = next_part;
      c0 = next_c0;
      to = first_of(part + 1);
    }
    // ---- rank 0 joins the parts ----
    if (size > 1) {
      const uint32_t list_to = map_to_rank(smem_u32(&gathered[buf][rank * p.k]), 0);
      if (tid < p.k) {
        const uint64_t key = tid < have ? lists[cur][tid] : 0ull;
        st_cluster_u32(list_to + tid * 8, static_cast<uint32_t>(key));
        st_cluster_u32(list_to + tid * 8 + 4, static_cast<uint32_t>(key >> 32));
      }
      cluster_sync();
      if (rank != 0) continue;
    } else {
      __syncthreads();
    }
    rec = recs[buf][0];
    for (int v = 1; v < p.parts; ++v) rec = join(rec, recs[buf][v]);
    if (size > 1) {
      if (TOP) {
        rank_keys(gathered[buf], static_cast<int>(size) * p.k, p.k, lists[cur]);
        __syncthreads();
      }
    }
    const float nan = __uint_as_float(0x7fc00000u);
    const bool none = rec.m == -INFINITY;
    const float log_sum = none ? nan : log1pf(rec.T);
    if (tid == 32) {
      if (p.out_entropy) p.out_entropy[row] = none ? nan : log_sum - rec.S / (1.0f + rec.T);
      if (p.out_logprob) {
        const int tok = p.tokens[row];
        float lp = 0.0f;
        if (tok >= p.vocab) {
          lp = nan;
          atomicOr(p.status, HB_DEV_TOKEN_BAD_INDEX);
        } else if (tok >= 0) {
          lp = (to_f(logits[tok]) - rec.m) - log_sum;
        }
        p.out_logprob[row] = lp;
      }
    }
    if (tid < p.k) {
      const uint64_t key = lists[cur][tid];
      p.out_top_ids[static_cast<int64_t>(row) * p.k + tid] = static_cast<int32_t>(~static_cast<uint32_t>(key));
      p.out_top_logprobs[static_cast<int64_t>(row) * p.k + tid] = (key_value(key) - rec.m) - log_sum;
    }
  }
  if (abort_flag) {   // a copy did not arrive: report it, let others land
    if (tid == 0) atomicOr(p.status, HB_DEV_LOGPROBS_WAIT_EXPIRED);
    for (int i = 0; i < 200; ++i) __nanosleep(1000);
  }
}

template <typename T, bool ALIGNED>
int launch(Params p, int num_sms, cudaStream_t s) {
  // one part per slice, up to 8 (a power of two, so that clusters of every size share them evenly)
  const int chunks = (p.vocab + Shape<T>::PER_CHUNK - 1) / Shape<T>::PER_CHUNK;
  p.parts = 1;
  while (p.parts < MAX_PARTS && p.parts * CHUNKS < chunks) p.parts *= 2;
  // three CTAs per SM walk over the rows; a row is shared while the rows alone would leave some of them out
  int size = 1;
  while (size < p.parts && 2ll * size * p.n_rows <= 3ll * num_sms) size *= 2;
  const int clusters = std::min(p.n_rows, std::max(1, 3 * num_sms / size));
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(clusters) * size);
  cfg.blockDim = dim3(THREADS);
  const int smem = CHUNKS * CHUNK;
  static DynSmemState configured[2];
  auto kern = p.k > 0 ? logprobs_kernel<T, ALIGNED, true> : logprobs_kernel<T, ALIGNED, false>;
  if (hb_ensure_dyn_smem(reinterpret_cast<const void*>(kern), configured[p.k > 0], smem) != HB_OK) return HB_ERR_CUDA;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = size;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kern, p) == cudaSuccess ? HB_OK : HB_ERR_CUDA;
}

}  // namespace

extern "C" int hb_logprobs(hb_ctx* c, const void* logits, int32_t dtype, int32_t n_rows, int32_t vocab, int64_t row_stride,
                           const int32_t* tokens, int32_t k, float* out_logprob, float* out_entropy, int32_t* out_top_ids,
                           float* out_top_logprobs, void* stream) {
  if (!c || n_rows < 0 || vocab < 1 || row_stride < vocab || k < 0 || k > MAX_K || k > vocab) return HB_ERR_BAD_ARG;
  if (dtype != HB_DTYPE_F32 && dtype != HB_DTYPE_F16) return HB_ERR_BAD_ARG;
  if ((tokens != nullptr) != (out_logprob != nullptr)) return HB_ERR_BAD_ARG;
  if (vocab > MAX_VOCAB || n_rows > (1 << 27)) return HB_ERR_TOO_LARGE;
  const uintptr_t esz = dtype == HB_DTYPE_F32 ? 4 : 2, base = reinterpret_cast<uintptr_t>(logits);
  if (base % esz || ((reinterpret_cast<uintptr_t>(tokens) | reinterpret_cast<uintptr_t>(out_logprob) | reinterpret_cast<uintptr_t>(out_entropy) |
                      reinterpret_cast<uintptr_t>(out_top_ids) | reinterpret_cast<uintptr_t>(out_top_logprobs)) & 3u))
    return HB_ERR_BAD_ARG;
  if (n_rows == 0) return HB_OK;
  if (!logits || (k > 0 && (!out_top_ids || !out_top_logprobs))) return HB_ERR_BAD_ARG;
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess) return HB_ERR_CUDA;
  if (dev != c->device) return HB_ERR_BAD_ARG;
  const Params p{logits, row_stride, n_rows, vocab, k, 1, tokens, out_logprob, out_entropy, out_top_logprobs, out_top_ids, c->status};
  const bool aligned = base % 16 == 0 && (row_stride * static_cast<int64_t>(esz)) % 16 == 0;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (dtype == HB_DTYPE_F32) return aligned ? launch<float, true>(p, c->num_sms, s) : launch<float, false>(p, c->num_sms, s);
  return aligned ? launch<__half, true>(p, c->num_sms, s) : launch<__half, false>(p, c->num_sms, s);
}
