// Scoring of logits rows: log probability of a given token, entropy, the k best alternatives, in one pass
// over the logits.
//
//   m = max x,  T = sum over all but one maximum of e^(x - m),  S = sum (x - m) e^(x - m)
//   log p_i = (x_i - m) - log1p(T);   H = log1p(T) - S / (1 + T)
// The maximum's own term is the 1 of 1 + T and is never added to the small ones: a row that is nearly
// certain keeps its entropy to full relative precision.
//
// A row is cut into tiles of 4096 logits, 16 per thread, which stay in registers; a cluster of up to 8 CTAs
// shares a row when there are few rows (tile t belongs to rank t mod cluster size).  Every warp leaves
// one (m, T, S) record per tile, relative to its own maximum, in the shared memory of the cluster's rank
// 0, which joins all records in an order that depends on the vocabulary alone: no row's bits depend on how many
// rows there are.
//
// The k best are kept as 64-bit keys: the logit's bits made orderable, then the complement of its index, so
// that all keys differ, equal logits rank by index, and nothing depends on the order in which threads
// arrive.  Of a tile only the logits above the k-th best so far matter, after the first tile rarely any.
// When many threads hold one (the first tile; logits in ascending order) a bound is made out of the tile
// itself: the k-th largest of the 64 maxima of four threads each.  No more than k groups reach it, so at
// most 64 k logits pass: the buffer cannot overflow whatever the logits are.
#include <algorithm>

#include "hb_internal.h"
#include "ptx.cuh"

namespace {

constexpr int THREADS = 256, WARPS = THREADS / 32;
constexpr int PER = 16, TILE = THREADS * PER;
constexpr int MAX_VOCAB = 1 << 20, MAX_TILES = MAX_VOCAB / TILE;
constexpr int MAX_K = HB_LOGPROBS_MAX_K;
constexpr int GROUPS = THREADS / 4;
constexpr int CAP = MAX_K * 4 * PER;   // candidates of one tile
constexpr int MAX_CLUSTER = 8;
constexpr float LOG2E = 1.4426950408889634f;
static_assert(GROUPS >= MAX_K, "the bound needs k groups");

struct Params {
  const void* logits;
  int64_t row_stride;
  int vocab, k;
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

// Orderable bits of a logit; NaN below -inf.
__device__ __forceinline__ uint32_t order(float x) {
  const uint32_t u = __float_as_uint(x);
  return x != x ? 0u : (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
__device__ __forceinline__ uint64_t make_key(float x, int idx) { return (static_cast<uint64_t>(order(x)) << 32) | static_cast<uint32_t>(~idx); }
__device__ __forceinline__ float key_value(uint64_t key) {
  const uint32_t o = static_cast<uint32_t>(key >> 32);
  return o == 0u ? __uint_as_float(0x7fc00000u) : __uint_as_float((o & 0x80000000u) ? (o & 0x7fffffffu) : ~o);
}

__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(__half v) { return __half2float(v); }
// Index inside the tile of a thread's element e: 16-byte vectors, neighbouring threads side by side.
template <typename T>
__device__ __forceinline__ int at(int e) {
  constexpr int V = 16 / static_cast<int>(sizeof(T));
  return (e / V) * (THREADS * V) + static_cast<int>(threadIdx.x) * V + e % V;
}

// A tile into registers; elements beyond the vocabulary become -inf.
template <typename T, bool ALIGNED>
__device__ __forceinline__ void load_tile(const T* row, int base, int vocab, float (&x)[PER]) {
  constexpr int V = 16 / static_cast<int>(sizeof(T));
#pragma unroll
  for (int v = 0; v < PER / V; ++v) {
    const int i0 = base + at<T>(v * V);
    if (ALIGNED && i0 + V <= vocab) {
      const uint4 raw = __ldcs(reinterpret_cast<const uint4*>(row + i0));   // read once
      const T* p = reinterpret_cast<const T*>(&raw);
#pragma unroll
      for (int j = 0; j < V; ++j) x[v * V + j] = to_f(p[j]);
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j) x[v * V + j] = i0 + j < vocab ? to_f(row[i0 + j]) : -INFINITY;
    }
  }
}

template <typename T, bool ALIGNED>
__global__ void __launch_bounds__(THREADS)
logprobs_kernel(const Params p) {
  __shared__ float recs[MAX_TILES * WARPS * 3];          // rank 0's are used
  __shared__ uint64_t cand[CAP];
  __shared__ uint64_t lists[2][MAX_K];                   // best so far, sorted; they swap roles
  __shared__ uint64_t gathered[MAX_CLUSTER * MAX_K];     // rank 0: every rank's list
  __shared__ uint64_t group_max[GROUPS];
  __shared__ uint64_t bound;
  __shared__ int n_cand;
  __shared__ Rec warp_recs[WARPS];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  uint32_t rank, size;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(size));
  const int row = blockIdx.x / size;
  const T* logits = static_cast<const T*>(p.logits) + row * p.row_stride;
  const int n_tiles = (p.vocab + TILE - 1) / TILE;
  // rank 0's shared memory may be written once its CTA has started
  if (size > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  if (tid == 0) n_cand = 0;
  __syncthreads();
  const uint32_t recs0 = map_to_rank(smem_u32(recs), 0);
  uint64_t worst = 0;     // the k-th best key so far (0: fewer than k yet)
  int cur = 0, have = 0;
  bool started = size == 1;
  for (int t = rank; t < n_tiles; t += size) {
    float x[PER];
    const int base = t * TILE;
    load_tile<T, ALIGNED>(logits, base, p.vocab, x);
    float mx = x[0];
#pragma unroll
    for (int e = 1; e < PER; ++e) mx = fmaxf(mx, x[e]);      // (a NaN does not count)
    if (mx != mx) mx = -INFINITY;
    float M = mx;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
    const float ref = M == -INFINITY ? 0.0f : M;
    float s = 0.0f, d1 = 0.0f, n = 0.0f;
    if (mx < M || M == -INFINITY) {
#pragma unroll
      for (int e = 0; e < PER; ++e) {
        // below -200 the exponential is zero; the clamp keeps -inf out of the product, and NaN comes through
        const float d = max_nan(x[e] - ref, -200.0f), w = ex2_approx(d * LOG2E);
        s += w;
        d1 = fmaf(d, w, d1);
      }
    } else {   // this thread holds a maximum: count those apart
#pragma unroll
      for (int e = 0; e < PER; ++e) {
        const float d = max_nan(x[e] - ref, -200.0f), w = ex2_approx(d * LOG2E);
        const bool top = d == 0.0f;
        n += top ? 1.0f : 0.0f;
        s += top ? 0.0f : w;
        d1 = fmaf(d, w, d1);
      }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      s += __shfl_xor_sync(0xffffffffu, s, o);
      d1 += __shfl_xor_sync(0xffffffffu, d1, o);
      n += __shfl_xor_sync(0xffffffffu, n, o);
    }
    if (!started) {
      asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
      started = true;
    }
    if (lane == 0) {
      const uint32_t dst = recs0 + static_cast<uint32_t>((t * WARPS + warp) * 12);
      const float T_ = M == -INFINITY ? s : s + (n - 1.0f);
      st_cluster_u32(dst, __float_as_uint(M));
      st_cluster_u32(dst + 4, __float_as_uint(T_));
      st_cluster_u32(dst + 8, __float_as_uint(d1));
    }
    if (p.k == 0) continue;
    // ---- alternatives ----
    uint64_t floor_key = worst;
    const int full = __syncthreads_count(order(mx) >= static_cast<uint32_t>(worst >> 32));
    if (full == 0) continue;
    if (full * PER > CAP) {
      uint64_t best = 0;
#pragma unroll
      for (int e = 0; e < PER; ++e) {
        const int idx = base + at<T>(e);
        if (idx < p.vocab) {
          const uint64_t key = make_key(x[e], idx);
          best = key > best ? key : best;
        }
      }
#pragma unroll
      for (int o = 1; o < 4; o <<= 1) {
        const uint64_t other = __shfl_xor_sync(0xffffffffu, best, o);
        best = other > best ? other : best;
      }
      if ((tid & 3) == 0) group_max[tid >> 2] = best;
      __syncthreads();
      if (tid < GROUPS) {
        const uint64_t mine = group_max[tid];
        int above = 0;
#pragma unroll 8
        for (int g = 0; g < GROUPS; ++g) above += group_max[g] > mine || (group_max[g] == mine && g < tid);   // empty groups are all 0
        if (above == p.k - 1) bound = mine;
      }
      __syncthreads();
      if (bound > 0 && bound - 1 > floor_key) floor_key = bound - 1;   // keys equal to the bound pass
    }
    if (order(mx) >= static_cast<uint32_t>(floor_key >> 32)) {
#pragma unroll
      for (int e = 0; e < PER; ++e) {
        const int idx = base + at<T>(e);
        if (idx < p.vocab) {
          const uint64_t key = make_key(x[e], idx);
          if (key > floor_key) {
            const int place = atomicAdd(&n_cand, 1);
            if (place < CAP) cand[place] = key;   // (never beyond it: see the top of the file)
          }
        }
      }
    }
    __syncthreads();
    const int nc = min(n_cand, CAP), total = nc + have;
    for (int i = tid; i < total; i += THREADS) {
      const uint64_t mine = i < nc ? cand[i] : lists[cur][i - nc];
      int above = 0;
      for (int j = 0; j < nc; ++j) above += cand[j] > mine;
      for (int j = 0; j < have; ++j) above += lists[cur][j] > mine;
      if (above < p.k) lists[cur ^ 1][above] = mine;
    }
    __syncthreads();
    if (tid == 0) n_cand = 0;
    cur ^= 1;
    have = min(p.k, total);
    worst = have == p.k ? lists[cur][p.k - 1] : 0;
    __syncthreads();   // (n_cand is zero before anyone adds to it)
  }
  if (size > 1) {
    if (!started) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    const uint32_t dst = map_to_rank(smem_u32(gathered), 0);
    for (int i = tid; i < p.k; i += THREADS) {
      const uint64_t key = i < have ? lists[cur][i] : 0ull;
      st_cluster_u32(dst + (rank * MAX_K + i) * 8, static_cast<uint32_t>(key));
      st_cluster_u32(dst + (rank * MAX_K + i) * 8 + 4, static_cast<uint32_t>(key >> 32));
    }
    cluster_sync();
    if (rank != 0) return;
  } else {
    for (int i = tid; i < p.k; i += THREADS) gathered[i] = i < have ? lists[cur][i] : 0ull;
    __syncthreads();
  }
  // ---- rank 0: join the records, then the lists ----
  Rec r{-INFINITY, 0.0f, 0.0f};
  for (int i = tid; i < n_tiles * WARPS; i += THREADS) r = join(r, Rec{recs[i * 3], recs[i * 3 + 1], recs[i * 3 + 2]});
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const Rec other{__shfl_down_sync(0xffffffffu, r.m, o), __shfl_down_sync(0xffffffffu, r.T, o), __shfl_down_sync(0xffffffffu, r.S, o)};
    r = join(r, other);
  }
  if (lane == 0) warp_recs[warp] = r;
  __syncthreads();
  r = warp_recs[0];
#pragma unroll
  for (int w = 1; w < WARPS; ++w) r = join(r, warp_recs[w]);
  const float nan = __uint_as_float(0x7fc00000u);
  const bool none = r.m == -INFINITY;
  const float log_sum = none ? nan : log1pf(r.T);
  if (tid == 0) {
    if (p.out_entropy) p.out_entropy[row] = none ? nan : log_sum - r.S / (1.0f + r.T);
    if (p.out_logprob && p.tokens) {
      const int tok = p.tokens[row];
      float lp = 0.0f;
      if (tok >= p.vocab) {
        lp = nan;
        atomicOr(p.status, HB_DEV_TOKEN_BAD_INDEX);
      } else if (tok >= 0) {
        lp = (to_f(logits[tok]) - r.m) - log_sum;
      }
      p.out_logprob[row] = lp;
    }
  }
  const int n_lists = static_cast<int>(size) * p.k;
  for (int i = tid; i < n_lists; i += THREADS) {
    const uint64_t mine = gathered[(i / p.k) * MAX_K + i % p.k];
    if (mine == 0) continue;
    int above = 0;
    for (uint32_t c = 0; c < size; ++c)
      for (int j = 0; j < p.k; ++j) above += gathered[c * MAX_K + j] > mine;
    if (above < p.k) {
      p.out_top_ids[static_cast<int64_t>(row) * p.k + above] = static_cast<int32_t>(~static_cast<uint32_t>(mine));
      p.out_top_logprobs[static_cast<int64_t>(row) * p.k + above] = (key_value(mine) - r.m) - log_sum;
    }
  }
}

template <typename T, bool ALIGNED>
int launch(const Params& p, int n_rows, int num_sms, cudaStream_t s) {
  // a cluster per row while the rows alone leave SMs without four blocks; never more CTAs than tiles
  const int tiles = (p.vocab + TILE - 1) / TILE;
  int size = 1;
  while (size < MAX_CLUSTER && size * 2 <= tiles && static_cast<long long>(n_rows) * size < 4ll * num_sms) size *= 2;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(n_rows) * size);
  cfg.blockDim = dim3(THREADS);
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = size;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, logprobs_kernel<T, ALIGNED>, p) == cudaSuccess ? HB_OK : HB_ERR_CUDA;
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
  const Params p{logits, row_stride, vocab, k, tokens, out_logprob, out_entropy, out_top_logprobs, out_top_ids, c->status};
  const bool aligned = base % 16 == 0 && (row_stride * static_cast<int64_t>(esz)) % 16 == 0;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (dtype == HB_DTYPE_F32) return aligned ? launch<float, true>(p, n_rows, c->num_sms, s) : launch<float, false>(p, n_rows, c->num_sms, s);
  return aligned ? launch<__half, true>(p, n_rows, c->num_sms, s) : launch<__half, false>(p, n_rows, c->num_sms, s);
}
