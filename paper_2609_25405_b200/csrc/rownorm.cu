// Row operators in front of the projections: residual addition + RMSNorm + gain (hb_norm) and rows to
// 8 bits (hb_quant_rows).
//
//   s = x + residual;  y = s * rsqrt(mean(s^2) + eps) * gain;  E4M3: scale = max |y| / 448, code = y / scale
//
// Both are bound by the bytes of their rows: every element is read once, held in registers in fp32, and
// written once.  The largest |y| is rstd * max |s * gain| with rstd > 0, so the sum of squares and the maximum
// come out of ONE reduction and an 8-bit output needs no second pass over the row.
//
// Measured (one B200; 6.46 TB/s is a copy): 4096 rows of 4096, fp16 + fp32 to fp32 and codes, 29 - 31 us = 6.0 - 6.4 TB/s; 2048 rows of
// 16384, 20000 and 32768 the same way 70, 104 and 143 us = 5.3, 4.3 and 5.2 TB/s (with a residual more than 16384 columns spill 70 to
// 270 bytes a thread); 4096 rows of 14336
// fp16 to codes 35.6 us = 4.9 TB/s (gathered 38.9); rows off every boundary (4096 of 4097, fp16 + fp32 to codes) 52 us = 3.5 TB/s, with
// one element per access 88; arrays aligned differently, which have to: 2048 rows of 8000 55 us, of 20000 389 us = 1.2 TB/s
// (32 values a thread and array, 80 to 860 bytes of them spilled).
#include <cuda_fp8.h>

#include <initializer_list>

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
  int32_t lead0, lead_step;   // elements between a 16-byte boundary and the start of row r: (lead0 + r lead_step) mod 8
  int32_t turned, y_lead0, y_lead_step;   // hb_quant_rows: codes not aligned as x is go through `turned` bytes of shared memory per row
  float eps;
  int32_t report;             // of a row's scale and, where rows are fp16, of a largest magnitude that may be a saturated one
};

__device__ __forceinline__ float from16(uint32_t bits16, int bf16) {
  return bf16 ? __uint_as_float(bits16 << 16) : __half2float(__ushort_as_half(static_cast<unsigned short>(bits16)));
}

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
  // the elements that lie in 0 .. d - 1 one by one
  __device__ __forceinline__ void load_some(const void* row, int at, int d) {
#pragma unroll
    for (int i = 0; i < WORDS; ++i) w[i] = 0u;
#pragma unroll
    for (int j = 0; j < E; ++j) {
      if (at + j < 0 || at + j >= d) continue;
      if constexpr (BYTES == 4) w[j] = static_cast<const uint32_t*>(row)[at + j];
      else w[j / 2] |= static_cast<uint32_t>(static_cast<const unsigned short*>(row)[at + j]) << (16 * (j & 1));
    }
  }
  __device__ __forceinline__ float get(int i, int bf16) const {
    if constexpr (BYTES == 4) return __uint_as_float(w[i]);
    else return from16((w[i / 2] >> (16 * (i & 1))) & 0xffffu, bf16);
  }
};

// Stores E values of a row from element `at` on, in one access or (some) those that lie in 0 .. d - 1 one by one.
template <int E>
__device__ __forceinline__ void put(void* row, int64_t at, int dtype, bool whole, int d, const float (&v)[E]) {
  if constexpr (E == 8) {
    if (whole) {
      if (dtype == HB_DTYPE_E4M3) {
        uint32_t w[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const __nv_fp8x2_storage_t lo = __nv_cvt_float2_to_fp8x2(make_float2(v[4 * j], v[4 * j + 1]), __NV_SATFINITE, __NV_E4M3);
          const __nv_fp8x2_storage_t hi = __nv_cvt_float2_to_fp8x2(make_float2(v[4 * j + 2], v[4 * j + 3]), __NV_SATFINITE, __NV_E4M3);
          w[j] = lo | static_cast<uint32_t>(hi) << 16;
        }
        *reinterpret_cast<uint2*>(static_cast<char*>(row) + at) = make_uint2(w[0], w[1]);
      } else if (dtype == HB_DTYPE_F32) {
        float4* o = reinterpret_cast<float4*>(static_cast<float*>(row) + at);
        o[0] = make_float4(v[0], v[1], v[2], v[3]);
        o[1] = make_float4(v[4], v[5], v[6], v[7]);
      } else {
        const bool bf16 = dtype == HB_DTYPE_BF16;
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = bf16 ? pack_bf16x2(v[2 * j], v[2 * j + 1]) : pack_f16x2_satfinite(v[2 * j], v[2 * j + 1]);
        *reinterpret_cast<uint4*>(static_cast<unsigned short*>(row) + at) = make_uint4(w[0], w[1], w[2], w[3]);
      }
      return;
    }
  }
#pragma unroll
  for (int j = 0; j < E; ++j) {
    if (at + j < 0 || at + j >= d) continue;
    if (dtype == HB_DTYPE_E4M3) static_cast<unsigned char*>(row)[at + j] = __nv_cvt_float_to_fp8(v[j], __NV_SATFINITE, __NV_E4M3);
    else if (dtype == HB_DTYPE_F32) static_cast<float*>(row)[at + j] = v[j];
    else if (dtype == HB_DTYPE_BF16) static_cast<__nv_bfloat16*>(row)[at + j] = __float2bfloat16_rn(v[j]);
    else static_cast<__half*>(row)[at + j] = __float2half_rn(sat_half_range(v[j]));
  }
}

// One row per T threads, NV vectors of E elements a thread.  E = 8: wide accesses; vector v holds elements 8 v - lead .. 8 v - lead + 7,
// where `lead` elements lie between a 16-byte boundary and the row's start, so that rows of any length stay wide but for their
// first and last vector.  E = 1: rows whose arrays are not aligned alike.
// XB / RB: bytes of an element of x and of the residual (0 = none).  NORM: false for hb_quant_rows.
// x / unit for the elements of a row, |x| <= 448 unit (1 + 2^-23): a product with the reciprocal, corrected once by its remainder
// (Markstein 1990).  Before its own rounding the result is within 2^-46 of the quotient, so it has the quotient's e4m3 code
// unless the quotient lies that near the middle of two floats beside a border of codes; the units for which one does
// were all tried (2136 cases), and the codes are the same there too.  Rows of tiny values are lifted by a power of two, or the
// remainder would fall below fp32's range.  (4096 x 14336 fp16: 35.6 us; a division per element 48, the reciprocal alone 34.0, with a
// code in 10^5 beside the right one.)
struct Quotient {
  float unit, minus_recip, minus_lift;
  __device__ __forceinline__ Quotient(float u, float largest) {
    const float lift = largest < 9.094947017729282e-13f ? 1.152921504606846976e18f : 1.0f;   // 2^-40, 2^60
    unit = u * lift;
    minus_recip = -__frcp_rn(unit);
    minus_lift = -lift;
  }
  // (the sign of a zero stays)
  template <int E>
  __device__ __forceinline__ void operator()(float (&x)[E]) const {
    if constexpr (E == 1) {
      const float n = x[0] * minus_lift, q = n * minus_recip;
      x[0] = fmaf(fmaf(q, unit, n), minus_recip, q);
    } else {
      const uint64_t l2 = pack2(minus_lift, minus_lift), r2 = pack2(minus_recip, minus_recip), u2 = pack2(unit, unit);
#pragma unroll
      for (int i = 0; i < E; i += 2) {
        const uint64_t n = mul2(pack2(x[i], x[i + 1]), l2), q = mul2(n, r2);
        unpack2(fma2(fma2(q, u2, n), r2, q), x[i], x[i + 1]);
      }
    }
  }
};

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
  const int lead = E == 8 ? static_cast<int>((a.lead0 + src * a.lead_step) & 7) : 0;
  const char* x = static_cast<const char*>(a.x) + src * a.x_stride * XB;
  const char* res = RB ? static_cast<const char*>(a.res) + r * a.res_stride * RB : nullptr;
  auto first = [&](int i) { return (tid + i * T) * E - lead; };
  auto some = [&](int at) { return at < a.d && at + E > 0; };          // any of the vector's elements exists
  auto whole = [&](int at) { return at >= 0 && at + E <= a.d; };
  Raw<E, XB> rx[NV];
  Raw<E, RB ? RB : 4> rr[RB ? NV : 1];
  Raw<E, 2> rg[NORM ? NV : 1];
  const bool has_gain = NORM && a.gain;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int at = first(i);
    if (whole(at)) {
      rx[i].load(x, at);
      if constexpr (RB != 0) rr[i].load(res, at);
    } else {
      rx[i].load_some(x, at, a.d);
      if constexpr (RB != 0) rr[i].load_some(res, at, a.d);
    }
    if constexpr (NORM) {
      if (has_gain) {
        if (lead == 0 && whole(at)) rg[i].load(a.gain, at);
        else rg[i].load_some(a.gain, at, a.d);
      }
    }
  }
  float s[NORM ? NV : 1][E];
  float ss = 0.0f;
  uint32_t top = 0u;   // largest magnitude as bits: their order is that of the values, and NaN comes out on top
  if constexpr (!NORM && XB == 2) {
    uint32_t two = 0u;   // (16-bit values as they are, two at a time)
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int j = 0; j < Raw<E, XB>::WORDS; ++j) two = max_u16x2(two, rx[i].w[j] & 0x7fff7fffu);
    top = __float_as_uint(from16(max(two >> 16, two & 0xffffu), a.x_bf16)) & 0x7fffffffu;
  }
#pragma unroll
  for (int i = 0; i < ((!NORM && XB == 2) ? 0 : NV); ++i) {
#pragma unroll
    for (int j = 0; j < E; ++j) {
      float v = rx[i].get(j, a.x_bf16);
      if constexpr (RB != 0) v += rr[i].get(j, a.res_bf16);
      if constexpr (NORM) {
        s[i][j] = v;
        ss = fmaf(v, v, ss);
        if (has_gain) v *= rg[i].get(j, 1);
      }
      top = max(top, __float_as_uint(v) & 0x7fffffffu);
    }
  }
  if constexpr (RB != 0) {
    if (a.sum) {
      char* out = static_cast<char*>(a.sum) + r * a.sum_stride * RB;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int at = first(i);
        if (some(at)) put<E>(out, at, RB == 4 ? HB_DTYPE_F32 : a.res_bf16 ? HB_DTYPE_BF16 : HB_DTYPE_F16, whole(at), a.d, s[i]);
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
  float inv = 1.0f, unit = 1.0f, m = 1.0f;
  if (a.y_dtype == HB_DTYPE_E4M3) {
    const float amax = __uint_as_float(top) * rstd;
    const bool finite = amax <= 3.402823466e38f;   // (false for NaN too)
    m = fmaxf(amax, 7.888609052210118e-31f);   // 2^-100: 448 / m is finite
    inv = finite ? 448.0f / m : __int_as_float(0x7fffffff);
    unit = finite ? m * (1.0f / 448.0f) : __int_as_float(0x7fffffff);   // (within 2^-23; bit for bit PyTorch's m / 448)
    if (tid == 0) {
      a.scale[r] = unit;
      if (a.report && (!finite || (!NORM && XB == 2 && !a.x_bf16 && amax >= 65504.0f))) atomicOr(a.status, HB_DEV_F16_RANGE);
    }
  }
  // Rows as they came have values next to borders of codes far more often than chance has it (few bits, ratios of small
  // numbers): their codes are the quotient's by the scale that is handed out.  A norm's values carry errors of their own.
  const Quotient over_unit(unit, m);
  if constexpr (!NORM && E == 8) {
    if (a.turned) {
      // codes where the boundaries of their own row lie, then out in 8-byte accesses
      extern __shared__ __align__(16) unsigned char codes[];
      const int y_lead = static_cast<int>((a.y_lead0 + r * a.y_lead_step) & 7);
      unsigned char* mine = codes + threadIdx.x / T * a.turned;
      unsigned char* y = static_cast<unsigned char*>(a.y) + r * a.y_stride;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int at = first(i);
        float v[E];
#pragma unroll
        for (int j = 0; j < E; ++j) v[j] = rx[i].get(j, a.x_bf16);
        over_unit(v);
#pragma unroll
        for (int j = 0; j < E; ++j)
          if (at + j >= 0 && at + j < a.d) mine[y_lead + at + j] = __nv_cvt_float_to_fp8(v[j], __NV_SATFINITE, __NV_E4M3);
      }
      if constexpr (T == 32) __syncwarp();
      else __syncthreads();
      for (int i = tid * 8; i < y_lead + a.d; i += T * 8) {
        const int at = i - y_lead;
        if (whole(at)) {
          *reinterpret_cast<uint2*>(y + at) = *reinterpret_cast<const uint2*>(mine + i);
        } else {
          for (int j = 0; j < 8; ++j)
            if (at + j >= 0 && at + j < a.d) y[at + j] = mine[i + j];
        }
      }
      return;
    }
  }
  char* y = static_cast<char*>(a.y) + r * a.y_stride * (a.y_dtype == HB_DTYPE_E4M3 ? 1 : a.y_dtype == HB_DTYPE_F32 ? 4 : 2);
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int at = first(i);
    if (!some(at)) continue;
    float v[E];
#pragma unroll
    for (int j = 0; j < E; ++j) {
      if constexpr (NORM) {
        v[j] = s[i][j] * rstd;
        if (has_gain) v[j] *= rg[i].get(j, 1);
        v[j] *= inv;
      } else {
        v[j] = rx[i].get(j, a.x_bf16);     // (kept as loaded: half the registers)
      }
    }
    if constexpr (!NORM) over_unit(v);
    put<E>(y, at, a.y_dtype, whole(at), a.d, v);
  }
}

template <int XB, int RB, int T, int NV, int E, bool NORM>
int launch(const RowArgs& a, cudaStream_t s, bool pdl) {
  const unsigned rows = static_cast<unsigned>(a.n_rows), grid = T == 32 ? (rows + 7) / 8 : rows;   // (n_rows may be the largest int)
  return hb_launch_kernel(row_kernel<XB, RB, T, NV, E, NORM>, grid, T == 32 ? 256 : T, (T == 32 ? 8 : 1) * a.turned, s, pdl, a);
}

// Threads of a row and vectors of a thread.  An SM needs some 40 KB under way: where a vector is few bytes (no residual), four a
// thread reach that if there are enough rows (8192 fp16 to codes, 4096 rows: 18.9 us, with one or two a thread 27.7); otherwise
// more threads do (4096 fp16 + fp32 to codes, 4096 rows: 28.9 us = 6.4 TB/s, 99 % of the copy rate).
template <int XB, int RB, bool NORM>
int launch_size(const RowArgs& a, bool wide, bool many, cudaStream_t s, bool pdl) {
  if (!wide) {
    if constexpr (!NORM) return launch<XB, RB, 1024, 32, 1, NORM>(a, s, pdl);   // (only the last few lengths)
    if (a.d <= 256) return launch<XB, RB, 32, 8, 1, NORM>(a, s, pdl);
    if (a.d <= 2048) return launch<XB, RB, 256, 8, 1, NORM>(a, s, pdl);
    if (a.d <= 8192) return launch<XB, RB, 1024, 8, 1, NORM>(a, s, pdl);
    return launch<XB, RB, 1024, 32, 1, NORM>(a, s, pdl);
  }
  const int d = a.d + ((a.lead0 | a.lead_step) & 7 ? 7 : 0);     // with the elements in front of the row
  if (d <= 256) return launch<XB, RB, 32, 1, 8, NORM>(a, s, pdl);
  if (d <= 512) return launch<XB, RB, 32, 2, 8, NORM>(a, s, pdl);
  if (d <= 1024) return launch<XB, RB, 32, 4, 8, NORM>(a, s, pdl);
  if constexpr ((XB == 2 || !NORM) && RB == 0) {
    if (many) {
      if (d <= 2048) return launch<XB, RB, 64, 4, 8, NORM>(a, s, pdl);
      if (d <= 4096) return launch<XB, RB, 128, 4, 8, NORM>(a, s, pdl);
      if (d <= 8192) return launch<XB, RB, 256, 4, 8, NORM>(a, s, pdl);
      if (d <= 16384) return launch<XB, RB, 512, 4, 8, NORM>(a, s, pdl);
    }
  }
  if (d <= 2048) return launch<XB, RB, 256, 1, 8, NORM>(a, s, pdl);
  if (d <= 4096) return launch<XB, RB, 512, 1, 8, NORM>(a, s, pdl);
  if (d <= 8192) return launch<XB, RB, 512, 2, 8, NORM>(a, s, pdl);
  if (d <= 16384) return launch<XB, RB, 1024, 2, 8, NORM>(a, s, pdl);
  if (d <= 32768) return launch<XB, RB, 1024, 4, 8, NORM>(a, s, pdl);
  return launch<XB, RB, 1024, 32, 1, NORM>(a, s, pdl);   // (the last few lengths, off a boundary)
}

// The rows of one array: first element, elements between rows, bytes of an element.
struct Rows {
  const void* p;
  int64_t stride;
  int size;
};
// Whether the arrays of a call are aligned alike, so that one `lead` per row serves them all: a wide access takes 8 elements of 1 or
// 2 bytes from a boundary of as many, or 4 of 4 bytes.
bool aligned_alike(std::initializer_list<Rows> arrays, RowArgs* a) {
  const Rows* ref = arrays.begin();
  for (const Rows& x : arrays)
    if (x.p && x.size < 4) ref = &x;
  const int64_t lead = reinterpret_cast<uintptr_t>(ref->p) / ref->size % 8, step = ref->stride % 8;
  for (const Rows& x : arrays) {
    const int64_t unit = x.size == 4 ? 4 : 8;
    if (!x.p) continue;
    if ((reinterpret_cast<uintptr_t>(x.p) / x.size) % unit != static_cast<uint64_t>(lead % unit) || x.stride % unit != step % unit) return false;
  }
  a->lead0 = static_cast<int32_t>(lead);
  a->lead_step = static_cast<int32_t>(step);
  return true;
}

// Every row starts on a boundary of `bytes`.
bool rows_on(const void* p, int64_t stride, int size, int bytes) {
  return reinterpret_cast<uintptr_t>(p) % bytes == 0 && (stride * size) % bytes == 0;
}

}  // namespace

int hb_launch_norm(hb_ctx* c, const hb_norm_args& n, cudaStream_t s, bool pdl, bool report) {
  if (n.d > HB_NORM_MAX_D) return HB_ERR_TOO_LARGE;   // (no variant covers more)
  RowArgs a = {};
  a.x = n.x; a.res = n.residual; a.sum = n.sum_out; a.gain = static_cast<const __nv_bfloat16*>(n.gain); a.y = n.y; a.scale = n.y_scale;
  a.status = c->status; a.report = report;
  a.x_stride = n.x_stride; a.res_stride = n.residual_stride; a.sum_stride = n.sum_stride; a.y_stride = n.y_stride;
  a.n_rows = n.n_rows; a.n_src = n.n_rows; a.d = n.d;
  a.x_bf16 = n.x_dtype == HB_DTYPE_BF16; a.res_bf16 = n.residual_dtype == HB_DTYPE_BF16; a.y_dtype = n.y_dtype; a.eps = n.eps;
  const int xb = hb_elem_bytes(n.x_dtype), rb = n.residual ? hb_elem_bytes(n.residual_dtype) : 0, yb = hb_elem_bytes(n.y_dtype);
  const bool wide = rows_on(n.gain, 0, 2, 16) &&
                    aligned_alike({{n.x, n.x_stride, xb}, {n.residual, n.residual_stride, rb ? rb : 1},
                                   {n.sum_out, n.sum_stride, rb ? rb : 1}, {n.y, n.y_stride, yb}}, &a);
  const bool many = n.n_rows >= 2 * c->num_sms;
  if (xb == 4) {
    if (rb == 0) return launch_size<4, 0, true>(a, wide, many, s, pdl);
    return rb == 4 ? launch_size<4, 4, true>(a, wide, many, s, pdl) : launch_size<4, 2, true>(a, wide, many, s, pdl);
  }
  if (rb == 0) return launch_size<2, 0, true>(a, wide, many, s, pdl);
  return rb == 4 ? launch_size<2, 4, true>(a, wide, many, s, pdl) : launch_size<2, 2, true>(a, wide, many, s, pdl);
}

int hb_launch_quant_rows(hb_ctx* c, const void* x, int x_dtype, int64_t x_stride, int n_src, const int32_t* index, int n_rows, int d,
                         void* codes, int64_t codes_stride, float* scale, cudaStream_t s, bool pdl, bool report) {
  if (d > HB_NORM_MAX_D) return HB_ERR_TOO_LARGE;
  RowArgs a = {};
  a.x = x; a.y = codes; a.scale = scale; a.index = index; a.status = c->status; a.report = report;
  a.x_stride = x_stride; a.y_stride = codes_stride;
  a.n_rows = n_rows; a.n_src = n_src; a.d = d;
  a.x_bf16 = x_dtype == HB_DTYPE_BF16; a.y_dtype = HB_DTYPE_E4M3;
  const int xb = hb_elem_bytes(x_dtype);
  if (!aligned_alike({{x, x_stride, xb}, {codes, codes_stride, 1}}, &a) || (index && a.lead_step)) {   // (an index breaks the step)
    a.y_lead0 = static_cast<int32_t>(reinterpret_cast<uintptr_t>(codes) % 8);
    a.y_lead_step = static_cast<int32_t>(codes_stride % 8);
    a.turned = (d + 7 + 15) / 16 * 16;
    aligned_alike({{x, x_stride, xb}}, &a);
  }
  const bool wide = ((a.lead0 | a.lead_step) & 7) == 0 || d + 7 <= HB_NORM_MAX_D;
  if (!wide) a.turned = 0;
  const bool many = n_rows >= 2 * c->num_sms;
  return xb == 4 ? launch_size<4, 0, false>(a, wide, many, s, pdl) : launch_size<2, 0, false>(a, wide, many, s, pdl);
}

extern "C" int hb_norm(hb_ctx* c, const hb_norm_args* n, void* stream) {
  if (!c || !n || n->n_rows < 0 || n->d < 1 || !(n->eps >= 0.0f)) return HB_ERR_BAD_ARG;
  if (!hb_float_type(n->x_dtype) || (n->residual && !hb_float_type(n->residual_dtype)) || (!hb_float_type(n->y_dtype) && n->y_dtype != HB_DTYPE_E4M3))
    return HB_ERR_BAD_ARG;
  if ((n->sum_out && !n->residual) || (n->y_scale && n->y_dtype != HB_DTYPE_E4M3)) return HB_ERR_BAD_ARG;
  if (n->d > HB_NORM_MAX_D) return HB_ERR_TOO_LARGE;
  if (n->x_stride < n->d || n->y_stride < n->d || (n->residual && n->residual_stride < n->d) || (n->sum_out && n->sum_stride < n->d))
    return HB_ERR_BAD_ARG;
  const int xb = hb_elem_bytes(n->x_dtype), rb = n->residual ? hb_elem_bytes(n->residual_dtype) : 1;
  if (!rows_on(n->x, 0, 1, xb) || !rows_on(n->residual, 0, 1, rb) || !rows_on(n->sum_out, 0, 1, rb) || !rows_on(n->gain, 0, 1, 2) ||
      !rows_on(n->y, 0, 1, hb_elem_bytes(n->y_dtype)) || !rows_on(n->y_scale, 0, 1, 4))
    return HB_ERR_BAD_ARG;
  if (n->n_rows == 0) return HB_OK;
  if (!n->x || !n->y || (n->y_dtype == HB_DTYPE_E4M3 && !n->y_scale)) return HB_ERR_BAD_ARG;
  const int rc = hb_wrong_device(c);
  return rc != HB_OK ? rc : hb_launch_norm(c, *n, static_cast<cudaStream_t>(stream), false);
}

extern "C" int hb_quant_rows(hb_ctx* c, const void* x, int32_t x_dtype, int64_t x_stride, int32_t n_src, const int32_t* index,
                             int32_t n_rows, int32_t d, void* codes, int64_t codes_stride, float* scale, void* stream) {
  if (!c || n_rows < 0 || n_src < 0 || d < 1 || !hb_float_type(x_dtype) || (!index && n_src < n_rows)) return HB_ERR_BAD_ARG;
  if (d > HB_NORM_MAX_D) return HB_ERR_TOO_LARGE;
  if (x_stride < d || codes_stride < d) return HB_ERR_BAD_ARG;
  if (!rows_on(x, 0, 1, hb_elem_bytes(x_dtype)) || !rows_on(index, 0, 1, 4) || !rows_on(scale, 0, 1, 4)) return HB_ERR_BAD_ARG;
  if (n_rows == 0) return HB_OK;
  if ((!x && n_src > 0) || !codes || !scale) return HB_ERR_BAD_ARG;
  const int rc = hb_wrong_device(c);
  return rc != HB_OK ? rc
                     : hb_launch_quant_rows(c, x, x_dtype, x_stride, n_src, index, n_rows, d, codes, codes_stride, scale,
                                            static_cast<cudaStream_t>(stream), false);
}
