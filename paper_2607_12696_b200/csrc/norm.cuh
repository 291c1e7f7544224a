// Residual addition + root-mean-square norm, optionally with the FP8 1x128 quantisation of the result.
//
//   s = x + residual (binary32),  r = 1 / sqrt(mean(s^2) + eps),  y = s * r * w
//   block of 128 columns: scale = act_scale(max |y|), code = e4m3(y / scale)   (common.cuh)
//
// The sum, the norm and the codes are taken from the unrounded binary32 values; what is written in
// bf16 (the sum for the next layer, y) is rounded once, so neither rounding enters the other result.
//
// A CTA works on a row at a time: it is read once, into registers, and everything that follows works on those.
// A thread owns pieces of 8 consecutive columns (one 16-byte access in bf16); 16 neighbouring
// threads own one 128-column block, so its maximum is a butterfly over 16 lanes.  HBM bound for many
// rows; for a few rows the time is one launch, one trip to memory and one block-wide reduction.
#pragma once
#include "common.cuh"

namespace moev {

struct NormArgs {
  const void* x;
  const void* res;
  const void* w;
  void* y;
  void* res_out;
  uint8_t* codes;
  float* scales;
  long long x_stride, res_stride, y_stride, res_out_stride, codes_stride;
  int n, H, quant;
  float eps;
};

template <typename T>
__device__ __forceinline__ float to_float(T v);
template <>
__device__ __forceinline__ float to_float<float>(float v) { return v; }
template <>
__device__ __forceinline__ float to_float<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }

// 8 consecutive values starting at column c; columns from H on read as zero
template <typename T, bool VEC>
__device__ __forceinline__ void norm_load8(const T* row, int c, int H, float (&v)[8]) {
  if constexpr (VEC) {
    if constexpr (sizeof(T) == 2) {
      const uint4 q = *reinterpret_cast<const uint4*>(row + c);
      const uint32_t u[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(u[i] << 16);
        v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
      }
    } else {
      const float4 a = *reinterpret_cast<const float4*>(row + c), b = *reinterpret_cast<const float4*>(row + c + 4);
      v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
      v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = c + i < H ? to_float(row[c + i]) : 0.f;
  }
}
template <typename T, bool VEC>
__device__ __forceinline__ void norm_store8(T* row, int c, int H, const float (&v)[8]) {
  if constexpr (VEC) {
    if constexpr (sizeof(T) == 2) {
      uint32_t u[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 p = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
        u[i] = *reinterpret_cast<const uint32_t*>(&p);
      }
      *reinterpret_cast<uint4*>(row + c) = make_uint4(u[0], u[1], u[2], u[3]);
    } else {
      *reinterpret_cast<float4*>(row + c) = make_float4(v[0], v[1], v[2], v[3]);
      *reinterpret_cast<float4*>(row + c + 4) = make_float4(v[4], v[5], v[6], v[7]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c + i < H) {
        if constexpr (sizeof(T) == 2) row[c + i] = __float2bfloat16_rn(v[i]);
        else row[c + i] = v[i];
      }
  }
}

// 8 values as they are in memory, for rows that are fetched ahead
template <typename T>
struct Raw8 {
  uint4 q[sizeof(T) / 2];
};
template <typename T>
__device__ __forceinline__ Raw8<T> norm_fetch8(const T* row, int c) {
  Raw8<T> r;
#pragma unroll
  for (int i = 0; i < (int)(sizeof(T) / 2); ++i) r.q[i] = reinterpret_cast<const uint4*>(row + c)[i];
  return r;
}
template <typename T>
__device__ __forceinline__ void norm_unpack8(const Raw8<T>& r, float (&v)[8]) {
  if constexpr (sizeof(T) == 2) {
    const uint32_t u[4] = {r.q[0].x, r.q[0].y, r.q[0].z, r.q[0].w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(u[i] << 16);
      v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
    }
  } else {
    const uint32_t u[8] = {r.q[0].x, r.q[0].y, r.q[0].z, r.q[0].w, r.q[1].x, r.q[1].y, r.q[1].z, r.q[1].w};
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(u[i]);
  }
}

// PV pieces of 8 columns per thread (H <= PV * 8 * blockDim.x); VEC: every row of every tensor starts on a
// 16-byte (codes: 8-byte) boundary and H is a multiple of 8.  A CTA takes every gridDim.x-th row.  Where a thread has
// one piece, rows are fetched one ahead, while the CTA waits for the sum of the one before (8192 rows of 7168 with codes:
// a CTA of 448 threads per row 115 us, 896 threads and rows ahead 103 us, and with the warps' sums added across lanes and not
// by every thread 94 us, 5.6 TB/s).
template <typename T, typename TW, int PV, bool VEC>
__global__ void __launch_bounds__(PV == 1 ? 1024 : 512) add_rmsnorm_kernel(NormArgs a) {
  constexpr bool kAhead = VEC && PV == 1;
  __shared__ float part[2][32];
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int tid = threadIdx.x, H = a.H;
  const TW* w = static_cast<const TW*>(a.w);
  Raw8<T> xq[kAhead ? PV : 1], rq[kAhead ? PV : 1];
  Raw8<TW> wq[kAhead ? PV : 1];
  auto fetch = [&](long long row) {
    if constexpr (kAhead) {
#pragma unroll
      for (int p = 0; p < PV; ++p) {
        const int c = (p * blockDim.x + tid) * 8;
        if (c < H) {
          xq[p] = norm_fetch8<T>(static_cast<const T*>(a.x) + row * a.x_stride, c);
          if (a.res) rq[p] = norm_fetch8<T>(static_cast<const T*>(a.res) + row * a.res_stride, c);
        }
      }
    }
  };
  fetch(blockIdx.x);
  if constexpr (kAhead) {
#pragma unroll
    for (int p = 0; p < PV; ++p) {
      const int c = (p * blockDim.x + tid) * 8;
      if (c < H) wq[p] = norm_fetch8<TW>(w, c);
    }
  }
  int turn = 0;
  for (long long row = blockIdx.x; row < a.n; row += gridDim.x, turn ^= 1) {
    float v[PV][8];
    float ss = 0.f;
    const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
    const T* res = a.res ? static_cast<const T*>(a.res) + row * a.res_stride : nullptr;
    T* ro = a.res_out ? static_cast<T*>(a.res_out) + row * a.res_out_stride : nullptr;
#pragma unroll
    for (int p = 0; p < PV; ++p) {
      const int c = (p * blockDim.x + tid) * 8;
      if (c < H) {
        if constexpr (kAhead) norm_unpack8<T>(xq[p], v[p]);
        else norm_load8<T, VEC>(x, c, H, v[p]);
        if (res) {
          float r[8];
          if constexpr (kAhead) norm_unpack8<T>(rq[p], r);
          else norm_load8<T, VEC>(res, c, H, r);
#pragma unroll
          for (int i = 0; i < 8; ++i) v[p][i] += r[i];
        }
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[p][i] = 0.f;
      }
    }
    // this row's inputs are in registers: outputs may take their place
    if (row + gridDim.x < a.n) fetch(row + gridDim.x);
#pragma unroll
    for (int p = 0; p < PV; ++p) {
      const int c = (p * blockDim.x + tid) * 8;
      if (ro && c < H) norm_store8<T, VEC>(ro, c, H, v[p]);
#pragma unroll
      for (int i = 0; i < 8; ++i) ss = fmaf(v[p][i], v[p][i], ss);
    }
    ss = warp_sum(ss);
    if ((tid & 31) == 0) part[turn][tid >> 5] = ss;
    __syncthreads();  // the other half of `part` belongs to the next row
    // the same additions in every warp, with the operands of some exchanged: the same sum everywhere
    const float tot = warp_sum((tid & 31) < (int)(blockDim.x >> 5) ? part[turn][tid & 31] : 0.f);
    const float rs = 1.f / sqrtf(tot / (float)H + a.eps);

    T* y = a.y ? static_cast<T*>(a.y) + row * a.y_stride : nullptr;
#pragma unroll
    for (int p = 0; p < PV; ++p) {
      const int c = (p * blockDim.x + tid) * 8;
      const bool in = c < H;
      if (in) {
        float g[8];
        if constexpr (kAhead) norm_unpack8<TW>(wq[p], g);
        else norm_load8<TW, VEC>(w, c, H, g);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[p][i] = v[p][i] * rs * g[i];
        if (y) norm_store8<T, VEC>(y, c, H, v[p]);
      }
      if (a.quant && (c & ~127) < H) {  // the 16 lanes of a block decide alike
        float m = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) m = fmaxf(m, fabsf(v[p][i]));
        const uint32_t lanes = 0xffffu << (tid & 16);
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(lanes, m, o));
        const float s = act_scale(m, a.quant);
        if (in) {
          float t[8];
          if (a.quant == 2 && s >= 1.17549435e-38f && s <= 8.5070592e37f) {
            // a power of two with a normal reciprocal: the product with that is the quotient, exactly
            const float inv = __uint_as_float(0x7F000000u - __float_as_uint(s));
#pragma unroll
            for (int i = 0; i < 8; ++i) t[i] = v[p][i] * inv;
          } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) t[i] = __fdiv_rn(v[p][i], s);
          }
          uint32_t q[2];
#pragma unroll
          for (int i = 0; i < 2; ++i)
            q[i] = (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(t[4 * i], t[4 * i + 1]), __NV_SATFINITE, __NV_E4M3) |
                   (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(t[4 * i + 2], t[4 * i + 3]), __NV_SATFINITE, __NV_E4M3) << 16;
          uint8_t* cr = a.codes + row * a.codes_stride;
          if constexpr (VEC) *reinterpret_cast<uint2*>(cr + c) = make_uint2(q[0], q[1]);
          else
            for (int i = 0; i < 8; ++i)
              if (c + i < H) cr[c + i] = (uint8_t)(q[i >> 2] >> (8 * (i & 3)));
          if ((c & 127) == 0) a.scales[row * ((H + 127) / 128) + (c >> 7)] = s;
        }
      }
    }
  }
}

}  // namespace moev
