// Row operators in front of the projections: residual addition + RMSNorm + gain (hb_norm) and rows to
// 8 bits (hb_quant_rows).
//
//   s = x + residual;  y = s * rsqrt(mean(s^2) + eps) * gain;  E4M3: scale = max |y| / 448, code = y / scale
//
// Both are bound by the bytes of their rows: every element is read once, held in registers in fp32, and
// written once.  The largest |y| is rstd * max |s * gain| with rstd > 0, so the sum of squares and the maximum
// come out of ONE reduction and an 8-bit output needs no second pass over the row.
#include <cuda_fp8.h>

#include "hb_internal.h"
#include "ptx.cuh"

namespace {

struct RowArgs {
  const void* x;
  const void* res;
  void* sum;
  const __nv_bfloat16* gain;
  void* y;
  float* scale;
  const int32_t* index;
  uint32_t* status;
  int64_t x_stride, res_stride, sum_stride, y_stride;
  int32_t n_rows, n_src, d;
  int32_t x_bf16, res_bf16, y_dtype;
  float eps;
};

__device__ __forceinline__ float from16(uint32_t bits16, int bf16) {
  return bf16 ? __uint_as_float(bits16 << 16) : __half2float(__ushort_as_half(static_cast<unsigned short>(bits16)));
}
__device__ __forceinline__ uint32_t to16(float v, int bf16) {
  return bf16 ? __bfloat16_as_ushort(__float2bfloat16_rn(v)) : __half_as_ushort(__float2half_rn(sat_half_range(v)));
}
__device__ __forceinline__ uint32_t to_e4m3(float v) { return __nv_cvt_float_to_fp8(v, __NV_SATFINITE, __NV_E4M3); }

// E consecutive elements of BYTES each, as loaded.
template <int E, int BYTES>
struct Raw {
  static constexpr int WORDS = (E * BYTES + 3) / 4;
  uint32_t w[WORDS];
  __device__ __forceinline__ void load(const void* row, int at) {
    const char* p = static_cast<const char*>(row) + static_cast<size_t>(at) * BYTES;
    if constexpr (E * BYTES >= 16) {
#pragma unroll
      for (int i = 0; i < WORDS / 4; ++i) {
        const uint4 q = reinterpret_cast<const uint4*>(p)[i];
        w[4 * i] = q.x; w[4 * i + 1] = q.y; w[4 * i + 2] = q.z; w[4 * i + 3] = q.w;
      }
    } else if constexpr (E * BYTES == 4) {
      w[0] = *reinterpret_cast<const uint32_t*>(p);
    } else {
      w[0] = *reinterpret_cast<const unsigned short*>(p);
    }
  }
  __device__ __forceinline__ float get(int i, int bf16) const {
    if constexpr (BYTES == 4) return __uint_as_float(w[i]);
    else return from16((w[i / 2] >> (16 * (i & 1))) & 0xffffu, bf16);
  }
};

// One row per T threads, NV vectors of E elements a thread (E = 8: wide accesses, E = 1: rows at any alignment).
// XB / RB: bytes of an element of x and of the residual (0 = none).  NORM: false for hb_quant_rows.
template <int XB, int RB, int T, int NV, int E, bool NORM>
__global__ void __launch_bounds__(T == 32 ? 256 : T) row_kernel(const RowArgs a) {
  grid_dep_wait();
  grid_dep_launch();
  constexpr int ROWS = T == 32 ? 8 : 1;   // rows per block
  const int tid = threadIdx.x % T, lane = threadIdx.x & 31;
  const int64_t r = static_cast<int64_t>(blockIdx.x) * ROWS + threadIdx.x / T;
  if (r >= a.n_rows) return;
  int64_t src = r;
  if (!NORM && a.index) {
    const int i = a.index[r];
    if (i < 0 || i >= a.n_src) {
      if (i >= 0 && tid == 0) atomicOr(a.status, HB_DEV_ROW_BAD_INDEX);
      return;
    }
    src = i;
  }
  const char* x = static_cast<const char*>(a.x) + src * a.x_stride * XB;
  const char* res = RB ? static_cast<const char*>(a.res) + r * a.res_stride * RB : nullptr;
  Raw<E, XB> rx[NV];
  Raw<E, RB ? RB : 4> rr[RB ? NV : 1];
  Raw<E, 2> rg[NORM ? NV : 1];
  const bool has_gain = NORM && a.gain;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int at = (tid + i * T) * E;
    if (at < a.d) {
      rx[i].load(x, at);
      if constexpr (RB != 0) rr[i].load(res, at);
      if constexpr (NORM) {
        if (has_gain) rg[i].load(a.gain, at);
      }
    }
  }
  float s[NV][E];
  float ss = 0.0f;
  uint32_t top = 0u;   // largest magnitude as bits: their order is that of the values, and NaN comes out on top
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const bool in = (tid + i * T) * E < a.d;
#pragma unroll
    for (int j = 0; j < E; ++j) {
      float v = rx[i].get(j, a.x_bf16);
      if constexpr (RB != 0) v += rr[i].get(j, a.res_bf16);
      if (!in) v = 0.0f;
      s[i][j] = v;
      float w = v;
      if constexpr (NORM) {
        ss = fmaf(v, v, ss);
        if (has_gain && in) w *= rg[i].get(j, 1);
      }
      top = max(top, __float_as_uint(w) & 0x7fffffffu);
    }
  }
  if constexpr (RB != 0) {
    if (a.sum) {
      char* out = static_cast<char*>(a.sum) + r * a.sum_stride * RB;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int at = (tid + i * T) * E;
        if (at < a.d) {
          if constexpr (E == 1) {
            if constexpr (RB == 4) reinterpret_cast<float*>(out)[at] = s[i][0];
            else reinterpret_cast<unsigned short*>(out)[at] = static_cast<unsigned short>(to16(s[i][0], a.res_bf16));
          } else if constexpr (RB == 4) {
            float4* o = reinterpret_cast<float4*>(out + static_cast<size_t>(at) * 4);
            o[0] = make_float4(s[i][0], s[i][1], s[i][2], s[i][3]);
            o[1] = make_float4(s[i][4], s[i][5], s[i][6], s[i][7]);
          } else {
            uint32_t w[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = to16(s[i][2 * j], a.res_bf16) | to16(s[i][2 * j + 1], a.res_bf16) << 16;
            *reinterpret_cast<uint4*>(out + static_cast<size_t>(at) * 2) = make_uint4(w[0], w[1], w[2], w[3]);
          }
        }
      }
    }
  }
  // over the row
  if constexpr (NORM) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
  }
  top = __reduce_max_sync(0xffffffffu, top);
  if constexpr (T > 32) {
    __shared__ float red_s[32];
    __shared__ uint32_t red_t[32];
    if (lane == 0) {
      red_s[threadIdx.x >> 5] = ss;
      red_t[threadIdx.x >> 5] = top;
    }
    __syncthreads();
    if constexpr (NORM) {
      ss = lane < T / 32 ? red_s[lane] : 0.0f;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
    }
    top = __reduce_max_sync(0xffffffffu, lane < T / 32 ? red_t[lane] : 0u);
  }
  const float rstd = NORM ? rsqrtf(ss / static_cast<float>(a.d) + a.eps) : 1.0f;
  float inv = 1.0f;
  if (a.y_dtype == HB_DTYPE_E4M3) {
    const float amax = __uint_as_float(top) * rstd;
    const bool finite = amax <= 3.402823466e38f;   // (false for NaN too)
    const float m = fmaxf(amax, 7.888609052210118e-31f);   // 2^-100: 448 / m is finite
    inv = finite ? 448.0f / m : __int_as_float(0x7fffffff);
    if (tid == 0) a.scale[r] = finite ? m / 448.0f : __int_as_float(0x7fffffff);
  }
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int at = (tid + i * T) * E;
    if (at >= a.d) continue;
    float v[E];
#pragma unroll
    for (int j = 0; j < E; ++j) {
      v[j] = s[i][j];
      if constexpr (NORM) {
        v[j] *= rstd;
        if (has_gain) v[j] *= rg[i].get(j, 1);
      }
    }
    if (a.y_dtype == HB_DTYPE_E4M3) {
      char* y = static_cast<char*>(a.y) + r * a.y_stride + at;
      if constexpr (E == 1) {
        *y = static_cast<char>(to_e4m3(v[0] * inv));
      } else {
        uint32_t w[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const __nv_fp8x2_storage_t lo = __nv_cvt_float2_to_fp8x2(make_float2(v[4 * j] * inv, v[4 * j + 1] * inv), __NV_SATFINITE, __NV_E4M3);
          const __nv_fp8x2_storage_t hi = __nv_cvt_float2_to_fp8x2(make_float2(v[4 * j + 2] * inv, v[4 * j + 3] * inv), __NV_SATFINITE, __NV_E4M3);
          w[j] = lo | static_cast<uint32_t>(hi) << 16;
        }
        *reinterpret_cast<uint2*>(y) = make_uint2(w[0], w[1]);
      }
    } else if (a.y_dtype == HB_DTYPE_F32) {
      float* y = static_cast<float*>(a.y) + r * a.y_stride + at;
      if constexpr (E == 1) {
        *y = v[0];
      } else {
        reinterpret_cast<float4*>(y)[0] = make_float4(v[0], v[1], v[2], v[3]);
        reinterpret_cast<float4*>(y)[1] = make_float4(v[4], v[5], v[6], v[7]);
      }
    } else {
      const int bf16 = a.y_dtype == HB_DTYPE_BF16;
      unsigned short* y = static_cast<unsigned short*>(a.y) + r * a.y_stride + at;
      if constexpr (E == 1) {
        *y = static_cast<unsigned short>(to16(v[0], bf16));
      } else {
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = to16(v[2 * j], bf16) | to16(v[2 * j + 1], bf16) << 16;
        *reinterpret_cast<uint4*>(y) = make_uint4(w[0], w[1], w[2], w[3]);
      }
    }
  }
}

template <int XB, int RB, int T, int NV, int E, bool NORM>
int launch(const RowArgs& a, cudaStream_t s, bool pdl) {
  const unsigned grid = T == 32 ? (a.n_rows + 7) / 8 : a.n_rows;
  return hb_launch_kernel(row_kernel<XB, RB, T, NV, E, NORM>, grid, T == 32 ? 256 : T, 0, s, pdl, a);
}

template <int XB, int RB, bool NORM>
int launch_size(const RowArgs& a, bool wide, cudaStream_t s, bool pdl) {
  if (!wide) {
    if (a.d <= 256) return launch<XB, RB, 32, 8, 1, NORM>(a, s, pdl);
    if (a.d <= 2048) return launch<XB, RB, 256, 8, 1, NORM>(a, s, pdl);
    if (a.d <= 8192) return launch<XB, RB, 1024, 8, 1, NORM>(a, s, pdl);
    return launch<XB, RB, 1024, 32, 1, NORM>(a, s, pdl);
  }
  if (a.d <= 256) return launch<XB, RB, 32, 1, 8, NORM>(a, s, pdl);
  if (a.d <= 1024) return launch<XB, RB, 32, 4, 8, NORM>(a, s, pdl);
  if (a.d <= 2048) return launch<XB, RB, 256, 1, 8, NORM>(a, s, pdl);
  if (a.d <= 4096) return launch<XB, RB, 512, 1, 8, NORM>(a, s, pdl);
  if (a.d <= 8192) return launch<XB, RB, 1024, 1, 8, NORM>(a, s, pdl);
  if (a.d <= 16384) return launch<XB, RB, 1024, 2, 8, NORM>(a, s, pdl);
  return launch<XB, RB, 1024, 4, 8, NORM>(a, s, pdl);
}

int elem_bytes(int dtype) { return dtype == HB_DTYPE_F32 ? 4 : dtype == HB_DTYPE_E4M3 ? 1 : 2; }
bool float_type(int dtype) { return dtype == HB_DTYPE_F32 || dtype == HB_DTYPE_F16 || dtype == HB_DTYPE_BF16; }
// Every row starts on a boundary of `bytes`.
bool rows_on(const void* p, int64_t stride, int size, int bytes) {
  return reinterpret_cast<uintptr_t>(p) % bytes == 0 && (stride * size) % bytes == 0;
}

int wrong_device(const hb_ctx* c) {
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess) return HB_ERR_CUDA;
  return dev == c->device ? HB_OK : HB_ERR_BAD_ARG;   // launches go to the current device
}

}  // namespace

int hb_launch_norm(hb_ctx* c, const hb_norm_args& n, cudaStream_t s, bool pdl) {
  RowArgs a = {};
  a.x = n.x; a.res = n.residual; a.sum = n.sum_out; a.gain = static_cast<const __nv_bfloat16*>(n.gain); a.y = n.y; a.scale = n.y_scale;
  a.status = c->status;
  a.x_stride = n.x_stride; a.res_stride = n.residual_stride; a.sum_stride = n.sum_stride; a.y_stride = n.y_stride;
  a.n_rows = n.n_rows; a.n_src = n.n_rows; a.d = n.d;
  a.x_bf16 = n.x_dtype == HB_DTYPE_BF16; a.res_bf16 = n.residual_dtype == HB_DTYPE_BF16; a.y_dtype = n.y_dtype; a.eps = n.eps;
  const int xb = elem_bytes(n.x_dtype), rb = n.residual ? elem_bytes(n.residual_dtype) : 0, yb = elem_bytes(n.y_dtype);
  const bool wide = n.d % 8 == 0 && rows_on(n.x, n.x_stride, xb, 16) && rows_on(n.gain, 0, 2, 16) && rows_on(n.y, n.y_stride, yb, yb == 1 ? 8 : 16) &&
                    (!rb || (rows_on(n.residual, n.residual_stride, rb, 16) && rows_on(n.sum_out, n.sum_stride, rb, 16)));
  if (xb == 4) {
    if (rb == 0) return launch_size<4, 0, true>(a, wide, s, pdl);
    return rb == 4 ? launch_size<4, 4, true>(a, wide, s, pdl) : launch_size<4, 2, true>(a, wide, s, pdl);
  }
  if (rb == 0) return launch_size<2, 0, true>(a, wide, s, pdl);
  return rb == 4 ? launch_size<2, 4, true>(a, wide, s, pdl) : launch_size<2, 2, true>(a, wide, s, pdl);
}

int hb_launch_quant_rows(hb_ctx* c, const void* x, int x_dtype, int64_t x_stride, int n_src, const int32_t* index, int n_rows, int d,
                         void* codes, int64_t codes_stride, float* scale, cudaStream_t s, bool pdl) {
  RowArgs a = {};
  a.x = x; a.y = codes; a.scale = scale; a.index = index; a.status = c->status;
  a.x_stride = x_stride; a.y_stride = codes_stride;
  a.n_rows = n_rows; a.n_src = n_src; a.d = d;
  a.x_bf16 = x_dtype == HB_DTYPE_BF16; a.y_dtype = HB_DTYPE_E4M3;
  const int xb = elem_bytes(x_dtype);
  const bool wide = d % 8 == 0 && rows_on(x, x_stride, xb, 16) && rows_on(codes, codes_stride, 1, 8);
  return xb == 4 ? launch_size<4, 0, false>(a, wide, s, pdl) : launch_size<2, 0, false>(a, wide, s, pdl);
}

extern "C" int hb_norm(hb_ctx* c, const hb_norm_args* n, void* stream) {
  if (!c || !n || n->n_rows < 0 || n->d < 1 || !(n->eps >= 0.0f)) return HB_ERR_BAD_ARG;
  if (!float_type(n->x_dtype) || (n->residual && !float_type(n->residual_dtype)) || (!float_type(n->y_dtype) && n->y_dtype != HB_DTYPE_E4M3))
    return HB_ERR_BAD_ARG;
  if ((n->sum_out && !n->residual) || (n->y_scale && n->y_dtype != HB_DTYPE_E4M3)) return HB_ERR_BAD_ARG;
  if (n->d > HB_NORM_MAX_D) return HB_ERR_TOO_LARGE;
  if (n->x_stride < n->d || n->y_stride < n->d || (n->residual && n->residual_stride < n->d) || (n->sum_out && n->sum_stride < n->d))
    return HB_ERR_BAD_ARG;
  const int xb = elem_bytes(n->x_dtype), rb = n->residual ? elem_bytes(n->residual_dtype) : 1;
  if (!rows_on(n->x, 0, 1, xb) || !rows_on(n->residual, 0, 1, rb) || !rows_on(n->sum_out, 0, 1, rb) || !rows_on(n->gain, 0, 1, 2) ||
      !rows_on(n->y, 0, 1, elem_bytes(n->y_dtype)) || !rows_on(n->y_scale, 0, 1, 4))
    return HB_ERR_BAD_ARG;
  if (n->n_rows == 0) return HB_OK;
  if (!n->x || !n->y || (n->y_dtype == HB_DTYPE_E4M3 && !n->y_scale)) return HB_ERR_BAD_ARG;
  const int rc = wrong_device(c);
  return rc != HB_OK ? rc : hb_launch_norm(c, *n, static_cast<cudaStream_t>(stream), false);
}

extern "C" int hb_quant_rows(hb_ctx* c, const void* x, int32_t x_dtype, int64_t x_stride, int32_t n_src, const int32_t* index,
                             int32_t n_rows, int32_t d, void* codes, int64_t codes_stride, float* scale, void* stream) {
  if (!c || n_rows < 0 || n_src < 0 || d < 1 || !float_type(x_dtype) || (!index && n_src < n_rows)) return HB_ERR_BAD_ARG;
  if (d > HB_NORM_MAX_D) return HB_ERR_TOO_LARGE;
  if (x_stride < d || codes_stride < d) return HB_ERR_BAD_ARG;
  if (!rows_on(x, 0, 1, elem_bytes(x_dtype)) || !rows_on(index, 0, 1, 4) || !rows_on(scale, 0, 1, 4)) return HB_ERR_BAD_ARG;
  if (n_rows == 0) return HB_OK;
  if ((!x && n_src > 0) || !codes || !scale) return HB_ERR_BAD_ARG;
  const int rc = wrong_device(c);
  return rc != HB_OK ? rc
                     : hb_launch_quant_rows(c, x, x_dtype, x_stride, n_src, index, n_rows, d, codes, codes_stride, scale,
                                            static_cast<cudaStream_t>(stream), false);
}
