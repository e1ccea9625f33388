// Appending a step's rows to the 8-bit KV cache: RMS norm of every query and key head (optional), rotary
// positions over the first rot_dim dimensions, q stored as fp16, k and v quantised to e4m3 with one
// power-of-two scale per (page, KV head), K and V apart.
//
//   q, k:  y = x / sqrt(mean(x^2) + eps) * gain;  (y_a, y_b) <- (y_a c - y_b s, y_b c + y_a s)
//   block: e = smallest exponent with max |y| <= 448 * 2^e over its new rows (and its old exponent, if the
//          page already holds rows);  code = e4m3(y * 2^-e)
//
// One warp per (row, task).  A task is 32 / (DH / 8) query heads of the row, or one KV head's K, or one KV
// head's V.  The scale of a block needs all of its new rows at once, so the KV tasks run only for rows
// that are the first of their segment in their page, and take the up to 16 rows that follow.  DH / 8
// lanes share a row, 8 dimensions each: 16-byte loads, the rotary partner (i + rot_dim / 2) sits at the
// same place of another lane.
#include "kv8.cuh"

namespace {

using namespace hb_kv8;

constexpr int WARPS = 8;

struct AppendParams {
  Rows r;
  const __half* qkv;
  __half* q_out;
  int64_t qkv_stride, q_stride;
  const __nv_bfloat16 *q_gain, *k_gain;
  float eps;
  const float *cos, *sin;
  int32_t rope_rows, rot, halves, Hq;
};

__device__ __forceinline__ void load8(const __half* p, float (&x)[8]) {
  const uint4 v = *reinterpret_cast<const uint4*>(p);
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
    x[2 * i] = f.x;
    x[2 * i + 1] = f.y;
  }
}

// One row's head, 8 dimensions per lane (dimensions d0 .. d0 + 7): norm and rotation.  The DH / 8 lanes of a
// row run this together; the shuffles stay inside them.
template <int DH>
__device__ __forceinline__ void norm_rotate(const AppendParams& p, const float (&g)[8], bool has_gain, int pos, int d0,
                                            float (&x)[8]) {
  constexpr int LPR = DH / 8;
  if (has_gain) {
    float ss = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) ss = fmaf(x[i], x[i], ss);
#pragma unroll
    for (int o = LPR / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
    const float inv = __frsqrt_rn(ss * (1.0f / DH) + p.eps);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = x[i] * inv * g[i];
  }
  if (p.rot == 0) return;
  const int half = p.rot >> 1;
  const bool turns = d0 < p.rot;
  if (!p.halves) {
    if (turns) {
      const size_t at = static_cast<size_t>(pos) * half + (d0 >> 1);
      const float4 c = __ldg(reinterpret_cast<const float4*>(p.cos + at)), s = __ldg(reinterpret_cast<const float4*>(p.sin + at));
      const float cc[4] = {c.x, c.y, c.z, c.w}, sn[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float a = x[2 * i], b = x[2 * i + 1];
        x[2 * i] = fmaf(a, cc[i], -b * sn[i]);
        x[2 * i + 1] = fmaf(b, cc[i], a * sn[i]);
      }
    }
  } else {
    const int lane = threadIdx.x & 31, sub = lane & (LPR - 1);
    const bool low = d0 < half;
    // half is a multiple of 8, so the partners are the same 8 elements of the lane half / 8 away
    const int other = (lane & ~(LPR - 1)) | (turns ? (low ? sub + (half >> 3) : sub - (half >> 3)) : sub);
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = __shfl_sync(0xffffffffu, x[i], other);
    if (turns) {
      const size_t at = static_cast<size_t>(pos) * half + (low ? d0 : d0 - half);
      const float4* cp = reinterpret_cast<const float4*>(p.cos + at);
      const float4* sp = reinterpret_cast<const float4*>(p.sin + at);
      const float4 c0 = __ldg(cp), c1 = __ldg(cp + 1), s0 = __ldg(sp), s1 = __ldg(sp + 1);
      const float cc[8] = {c0.x, c0.y, c0.z, c0.w, c1.x, c1.y, c1.z, c1.w};
      const float sn[8] = {s0.x, s0.y, s0.z, s0.w, s1.x, s1.y, s1.z, s1.w};
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = fmaf(x[i], cc[i], low ? -y[i] * sn[i] : y[i] * sn[i]);
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

// Sixteen codes stored again under a scale 2^-shrink_log2 times as large (f = 2^(e_old - e_new) <= 1).
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

template <int DH>
__global__ void __launch_bounds__(WARPS * 32)
kv8_append_kernel(const AppendParams p, const int q_tasks, const int n_tasks, const int groups) {
  grid_dep_wait();
  grid_dep_launch();
  constexpr int LPR = DH / 8, RPW = 32 / LPR, ITERS = 16 / RPW;
  __shared__ uint4 v_stage[WARPS][DH];   // 16 * DH bytes per warp: one block's V part
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int row = blockIdx.x / groups, task = (blockIdx.x % groups) * WARPS + warp;
  if (task >= n_tasks) return;
  const int sg = __ldg(p.r.row_seg + row);
  if (sg == -1) return;   // padding
  bool ok = sg >= 0 && sg < p.r.n_segs;
  int q_start = 0, q_len = 0, pos_start = 0, pt_start = 0;
  if (ok) {
    const int4 a = __ldg(reinterpret_cast<const int4*>(p.r.segs + sg));      // kind, q_start, q_len, pos_start
    const int4 b = __ldg(reinterpret_cast<const int4*>(p.r.segs + sg) + 1);  // pt_start, pt_len, pool_slot, pool_mode
    q_start = a.y; q_len = a.z; pos_start = a.w; pt_start = b.x;
    ok = seg_ok(p.r, q_start, q_len, pos_start, pt_start, b.y) && row >= q_start && row - q_start < q_len &&
         (p.rot == 0 || pos_start + q_len <= p.rope_rows);
  }
  const int sub = lane & (LPR - 1), which = lane / LPR, d0 = sub * 8;
  if (task < q_tasks) {
    if (!ok) {
      if (lane == 0) atomicOr(p.r.status, HB_DEV_APPEND_BAD_INDEX);
      return;
    }
    const int head = task * RPW + which;
    float x[8] = {}, g[8] = {};
    const bool mine = head < p.Hq;
    if (mine) load8(p.qkv + row * p.qkv_stride + head * DH + d0, x);
    load_gain(p.q_gain, d0, g);
    norm_rotate<DH>(p, g, p.q_gain != nullptr, pos_start + row - q_start, d0, x);
    if (mine) {
      uint4 o;
      o.x = pack_half2_sat(x[0], x[1]); o.y = pack_half2_sat(x[2], x[3]);
      o.z = pack_half2_sat(x[4], x[5]); o.w = pack_half2_sat(x[6], x[7]);
      *reinterpret_cast<uint4*>(p.q_out + row * p.q_stride + head * DH + d0) = o;
    }
    return;
  }
  // ---- one KV head's K or V: only the first of the segment's rows in its page ----
  if (!ok) return;   // reported by the query tasks
  const int j = row - q_start, pos = pos_start + j;
  const int slot0 = pos & (PAGE - 1);
  if (j > 0 && slot0 > 0) return;
  const int page = __ldg(p.r.page_ids + pt_start + pos / PAGE);
  if (page < 0 || page >= p.r.n_pages) {
    if (lane == 0) atomicOr(p.r.status, HB_DEV_APPEND_BAD_INDEX);
    return;
  }
  const int kv_task = task - q_tasks;
  const bool is_v = kv_task >= p.r.Hkv;
  const int hk = is_v ? kv_task - p.r.Hkv : kv_task;
  const int n_new = min(PAGE - slot0, q_len - j);
  uint8_t* block = p.r.arena + page * p.r.page_stride + static_cast<int64_t>(hk) * Block<DH>::BYTES;
  float* scale_at = reinterpret_cast<float*>(block + Block<DH>::HDR) + (is_v ? 1 : 0);
  const bool fresh = slot0 == 0;
  const int e_old = fresh ? E_MIN : max(E_MIN, min(E_MAX, exponent_of(*scale_at)));
  const __half* src = p.qkv + row * p.qkv_stride + static_cast<int64_t>(p.Hq + (is_v ? p.r.Hkv : 0) + hk) * DH + d0;
  float x[ITERS][8];
  float g[8] = {};
  if (!is_v) load_gain(p.k_gain, d0, g);
  float amax = 0.0f;
#pragma unroll
  for (int it = 0; it < ITERS; ++it) {
    if (it * RPW >= n_new) break;
    const int i = it * RPW + which;
#pragma unroll
    for (int c = 0; c < 8; ++c) x[it][c] = 0.0f;
    if (i < n_new) load8(src + i * p.qkv_stride, x[it]);
  }
#pragma unroll
  for (int it = 0; it < ITERS; ++it) {
    if (it * RPW >= n_new) break;
    const int i = it * RPW + which;
    if (!is_v) norm_rotate<DH>(p, g, p.k_gain != nullptr, pos + min(i, n_new - 1), d0, x[it]);
#pragma unroll
    for (int c = 0; c < 8; ++c) amax = fmaxf(amax, fabsf(x[it][c]));   // (NaN does not count)
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
  const int e = max(e_old, scale_exponent(amax));
  const float inv = pow2f(-e), shrink = pow2f(e_old - e);
  const bool grew = !fresh && e > e_old;
  __syncwarp();   // every lane has read the old scale
  if (lane == 0 && (fresh || grew)) *scale_at = pow2f(e);
  if (!is_v) {
    // token rows of 64 dimensions: 8 codes per lane and row
    uint8_t* dst = block + (d0 >> 6) * 1024 + (d0 & 63);
    if (grew) {
      for (int c = lane; c < DH; c += 32) {
        uint4* at = reinterpret_cast<uint4*>(block) + c;
        *at = rescale16(*at, shrink);
      }
      __syncwarp();
    }
#pragma unroll
    for (int it = 0; it < ITERS; ++it) {
      const int i = it * RPW + which;
      uint2 w = make_uint2(0u, 0u);
      if (it * RPW < n_new) {
        w.x = floats_to_e4m3x4(x[it][0] * inv, x[it][1] * inv, x[it][2] * inv, x[it][3] * inv);
        w.y = floats_to_e4m3x4(x[it][4] * inv, x[it][5] * inv, x[it][6] * inv, x[it][7] * inv);
      }
      // (the rows past the last one of a fresh page are zero)
      if (i < n_new) *reinterpret_cast<uint2*>(dst + (slot0 + i) * 64) = w;
      else if (fresh) *reinterpret_cast<uint2*>(dst + i * 64) = make_uint2(0u, 0u);
    }
    return;
  }
  uint8_t* vblock = block + Block<DH>::V_OFF;
  if (!fresh && !grew) {
    // the block keeps its scale: only the new rows' bytes are written
#pragma unroll
    for (int it = 0; it < ITERS; ++it) {
      if (it * RPW >= n_new) break;
      const int i = it * RPW + which;
      if (i < n_new) {
#pragma unroll
        for (int c = 0; c < 8; c += 2) {
          const uint32_t two = floats_to_e4m3x2(x[it][c] * inv, x[it][c + 1] * inv);
          vblock[v_byte(slot0 + i, d0, c)] = static_cast<uint8_t>(two);
          vblock[v_byte(slot0 + i, d0, c + 1)] = static_cast<uint8_t>(two >> 8);
        }
      }
    }
    return;
  }
  // whole V part through shared memory: what is there under the new scale (or zeros), the new bytes on top
  uint4* stage = v_stage[warp];
  for (int c = lane; c < DH; c += 32)
    stage[c] = fresh ? make_uint4(0u, 0u, 0u, 0u) : rescale16(reinterpret_cast<const uint4*>(vblock)[c], shrink);
  __syncwarp();
  uint8_t* bytes = reinterpret_cast<uint8_t*>(stage);
#pragma unroll
  for (int it = 0; it < ITERS; ++it) {
    if (it * RPW >= n_new) break;
    const int i = it * RPW + which;
    if (i < n_new) {
#pragma unroll
      for (int c = 0; c < 8; c += 2) {
        const uint32_t two = floats_to_e4m3x2(x[it][c] * inv, x[it][c + 1] * inv);
        bytes[v_byte(slot0 + i, d0, c)] = static_cast<uint8_t>(two);
        bytes[v_byte(slot0 + i, d0, c + 1)] = static_cast<uint8_t>(two >> 8);
      }
    }
  }
  __syncwarp();
  for (int c = lane; c < DH; c += 32) reinterpret_cast<uint4*>(vblock)[c] = stage[c];
}

template <int DH>
int launch(const AppendParams& p, cudaStream_t s, bool pdl) {
  const int rpw = 32 / (DH / 8);
  const int q_tasks = (p.Hq + rpw - 1) / rpw, n_tasks = q_tasks + 2 * p.r.Hkv, groups = (n_tasks + WARPS - 1) / WARPS;
  const long long grid = static_cast<long long>(p.r.n_rows) * groups;
  if (grid > 0x7fffffffll) return HB_ERR_TOO_LARGE;
  return hb_launch_kernel(kv8_append_kernel<DH>, static_cast<unsigned>(grid), WARPS * 32, 0, s, pdl, p, q_tasks, n_tasks, groups);
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
  p.halves = a.rope_layout == HB_ROPE_HALVES ? 1 : 0;
  p.Hq = c->cfg.n_heads;
  if (c->cfg.head_dim == 64) return launch<64>(p, s, pdl);
  if (c->cfg.head_dim == 128) return launch<128>(p, s, pdl);
  return HB_ERR_UNSUPPORTED;
}
