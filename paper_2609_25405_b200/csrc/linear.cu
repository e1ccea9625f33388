// Products with scales, bias, activation and residual in the epilogue (hb_linear), and the same with a weight per run of
// rows (hb_linear_grouped):  C = act(a_scale w_scale A W^T + bias) + residual.
//
// First form: a 64 x 64 tile per block, 4 x 4 results per thread, operands converted to fp32 in shared memory.
#include <cuda_fp8.h>

#include "hb_internal.h"
#include "ptx.cuh"

namespace {

constexpr int TILE = 64, KT = 16;

struct LinArgs {
  hb_linear_args l;
  const int32_t* start;
  int64_t w_group_stride;
  int32_t n_groups;
  uint32_t* status;
};

__device__ __forceinline__ float read_as_float(const void* p, int64_t at, int dtype) {
  switch (dtype) {
    case HB_DTYPE_F32: return static_cast<const float*>(p)[at];
    case HB_DTYPE_F16: return __half2float(static_cast<const __half*>(p)[at]);
    case HB_DTYPE_BF16: return __bfloat162float(static_cast<const __nv_bfloat16*>(p)[at]);
    default: return static_cast<float>(static_cast<const __nv_fp8_e4m3*>(p)[at]);
  }
}
__device__ __forceinline__ void write_from_float(void* p, int64_t at, int dtype, float v) {
  if (dtype == HB_DTYPE_F32) static_cast<float*>(p)[at] = v;
  else if (dtype == HB_DTYPE_F16) static_cast<__half*>(p)[at] = __float2half_rn(sat_half_range(v));
  else static_cast<__nv_bfloat16*>(p)[at] = __float2bfloat16_rn(v);
}
__device__ __forceinline__ float activate(float z, int act) {
  switch (act) {
    case HB_ACT_RELU: return z != z ? z : fmaxf(z, 0.0f);
    case HB_ACT_SILU: return z / (1.0f + expf(-z));
    case HB_ACT_GELU: return 0.5f * z * (1.0f + erff(z * 0.70710678f));
    case HB_ACT_GELU_TANH: return 0.5f * z * (1.0f + tanhf(0.79788456f * (z + 0.044715f * z * z * z)));
    default: return z;
  }
}

__global__ void __launch_bounds__(256) linear_kernel(const LinArgs a) {
  const hb_linear_args& l = a.l;
  __shared__ float sa[KT][TILE + 1], sw[KT][TILE + 1];
  // the group and row tile of this block
  int lo = 0, hi = l.m, g = 0, tile = blockIdx.y;
  if (a.start) {
    int most = 0;   // largest bound so far: no row belongs to two groups
    for (g = 0; g < a.n_groups; ++g) {
      lo = a.start[g];
      hi = a.start[g + 1];
      const bool good = lo >= most && hi >= lo && hi <= l.m;
      most = max(most, max(lo, 0));
      if (!good) {
        if (threadIdx.x == 0) atomicOr(a.status, HB_DEV_GROUP_BAD_INDEX);
        continue;
      }
      const int tiles = (hi - lo + TILE - 1) / TILE;
      if (tile < tiles) break;
      tile -= tiles;
    }
    if (g == a.n_groups) return;
  }
  const int m0 = lo + tile * TILE, n0 = blockIdx.x * TILE;
  if (m0 >= hi) return;
  const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
  float acc[4][4] = {};
  for (int k0 = 0; k0 < l.k; k0 += KT) {
    for (int i = threadIdx.x; i < TILE * KT; i += 256) {
      const int row = i / KT, k = i % KT;
      const bool kin = k0 + k < l.k;
      sa[k][row] = kin && m0 + row < hi ? read_as_float(l.a, (m0 + row) * l.a_stride + k0 + k, l.ab_dtype) : 0.0f;
      sw[k][row] = kin && n0 + row < l.n ? read_as_float(l.w, g * a.w_group_stride + (n0 + row) * l.w_stride + k0 + k, l.ab_dtype) : 0.0f;
    }
    __syncthreads();
    for (int k = 0; k < KT; ++k)
      for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(sa[k][ty * 4 + i], sw[k][tx * 4 + j], acc[i][j]);
    __syncthreads();
  }
  for (int i = 0; i < 4; ++i) {
    const int row = m0 + ty * 4 + i;
    if (row >= hi) break;
    const float as = l.a_scale ? l.a_scale[row] : 1.0f;
    float z[4];
    for (int j = 0; j < 4; ++j) {
      const int col = n0 + tx * 4 + j;
      if (col >= l.n) break;
      z[j] = acc[i][j] * as * (l.w_scale ? l.w_scale[static_cast<int64_t>(g) * l.n + col] : 1.0f) +
             (l.bias ? l.bias[static_cast<int64_t>(g) * l.n + col] : 0.0f);
      int out_col = col;
      float v;
      if (l.gated) {
        if (!(j & 1)) continue;
        out_col = col / 2;
        v = activate(z[j - 1], l.act) * z[j];
      } else {
        v = activate(z[j], l.act);
      }
      if (l.residual) v += read_as_float(l.residual, row * l.residual_stride + out_col, l.residual_dtype);
      write_from_float(l.c, row * l.c_stride + out_col, l.c_dtype, v);
    }
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

int hb_launch_linear(hb_ctx* c, const hb_linear_args& l, const int32_t* group_start, int n_groups, int64_t w_group_stride,
                     cudaStream_t s, bool pdl) {
  const LinArgs a{l, group_start, w_group_stride, n_groups, c->status};
  linear_kernel<<<dim3((l.n + TILE - 1) / TILE, (l.m + TILE - 1) / TILE + (group_start ? n_groups : 0)), 256, 0, s>>>(a);
  return cudaGetLastError() == cudaSuccess ? HB_OK : HB_ERR_CUDA;
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
