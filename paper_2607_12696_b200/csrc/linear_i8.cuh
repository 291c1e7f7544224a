// y = x W^T + bias with 8-bit integers on both sides: x = code * sx (a scale per token), W = code * sw (a scale per channel).
//
// quant_rows_kernel brings bf16 or binary32 rows to codes: sx = max |x| / 127 (binary32 division; 1 for a row of zeros), code =
// x / sx rounded to the nearest integer, ties to even (127 where a subnormal sx lets it go beyond).  A row with a NaN or an infinity has sx = NaN and codes 0, so all of its y
// is NaN.  One CTA a row, the row in registers between the maximum and the codes.
//
// The product runs on tcgen05.mma kind::i8: exact 32-bit integer sums, so their order does not matter; then
// y = (sum * sx) * sw + bias in binary32 (the sum rounded to binary32 first), rounded to the type of y.
// Rows of 128 codes (one 128-byte swizzle row) come by TMA through a ring; what lies beyond K, N or the tokens is filled with 0.
//
// Many tokens: a tile is 256 tokens x 256 channels of a pair of CTAs, which walk over the tiles, sums of one tile (256 columns of tensor memory)
// are read while the next is computed.
// Few tokens (a draft tree, one token): the weight is the wide operand, 128 channels x up to 128 tokens a tile, and K is shared
// among the CTAs of a cluster, so that all SMs stream the weight; the CTAs add each other's integer sums through distributed
// shared memory, each for its share of the tokens.
//
// Measured, x to codes included: 8001 x 7168 -> 9217 433 to 457 us call after call, 360 on a GPU that has rested for seconds (2.9 POP/s, the tensor pipe
// 88 % busy: the power limit; codes 34 to 45 of it: 5.0 TB/s alone, issue slots next); 1 x 8192 -> 4096 8.5 us (weight 5.1 at the copy rate; a launch, the ring's first fill
// and the cluster's sums are the rest), 1 x 4096 -> 60000 39 us (6.3 TB/s); 50 x 2880 -> 5120 9.4 us.
#pragma once
#include <cuda.h>

#include "attend.cuh"
#include "ptx.cuh"

namespace moev {
namespace i8 {

constexpr int kStep = 128;  // codes of K a stage
constexpr unsigned long long kBudgetNs = kDeviceWaitBudgetNs;

// ---------------------------------------------------------------- x to codes
struct QuantArgs {
  const void* x;
  int8_t* codes;
  float* scales;
  long long x_stride, codes_stride;
  int n, K;
};
// Codes of 8 values, packed.  The product with the reciprocal (unrounded inside the multiply-adds) is off by 127 * 2^-24 at most, so it decides
// except next to a border between two codes; there (rarely) the division does.  Adding 1.5 * 2^23 rounds to the nearest integer, ties to even, and
// leaves it in the low bits.
__device__ __forceinline__ uint2 codes_of(const float (&x)[8], float s, float inv) {
  uint32_t t[8];
  float edge = 0.f;
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    float r0 = x[e], r1 = x[e + 1];
    att::fma2(r0, r1, inv, inv, 12582912.f, 12582912.f);
    t[e] = __float_as_uint(r0);
    t[e + 1] = __float_as_uint(r1);
    att::fma2(r0, r1, -1.f, -1.f, 12582912.f, 12582912.f);
    float q0 = x[e], q1 = x[e + 1];  // what the rounding took away
    att::fma2(q0, q1, inv, inv, r0, r1);
    edge = fmaxf(edge, fmaxf(fabsf(q0), fabsf(q1)));
  }
  if (edge > 0.49998f) {
#pragma unroll
    for (int e = 0; e < 8; ++e) t[e] = (uint32_t)__float2int_rn(__fdiv_rn(x[e], s));
  }
  uint2 u;
  u.x = __byte_perm(__byte_perm(t[0], t[1], 0x0040), __byte_perm(t[2], t[3], 0x0040), 0x5410);
  u.y = __byte_perm(__byte_perm(t[4], t[5], 0x0040), __byte_perm(t[6], t[7], 0x0040), 0x5410);
  return u;
}
// 8 values as they lie in memory: by vectors or one by one, their magnitudes as integers (in that order NaN is beyond infinity), as numbers.
template <typename T>
struct Piece;
template <>
struct Piece<__nv_bfloat16> {
  uint32_t u[4];
  __device__ __forceinline__ void load(const __nv_bfloat16* p) {
    const uint4 w = __ldg(reinterpret_cast<const uint4*>(p));
    u[0] = w.x; u[1] = w.y; u[2] = w.z; u[3] = w.w;
  }
  __device__ __forceinline__ void load(const __nv_bfloat16* p, int n) {
    const uint16_t* q = reinterpret_cast<const uint16_t*>(p);
#pragma unroll
    for (int e = 0; e < 4; ++e) u[e] = (2 * e < n ? q[2 * e] : 0u) | (2 * e + 1 < n ? (uint32_t)q[2 * e + 1] << 16 : 0u);
  }
  __device__ __forceinline__ void clear() { u[0] = u[1] = u[2] = u[3] = 0; }
  __device__ __forceinline__ uint32_t top() const {  // binary32 pattern of the largest magnitude
    uint32_t m = u[0] & 0x7fff7fffu;
#pragma unroll
    for (int e = 1; e < 4; ++e) m = __vmaxu2(m, u[e] & 0x7fff7fffu);
    return max(m & 0xffff0000u, m << 16);
  }
  __device__ __forceinline__ void unpack(float (&v)[8]) const {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[2 * e] = __uint_as_float(u[e] << 16);
      v[2 * e + 1] = __uint_as_float(u[e] & 0xffff0000u);
    }
  }
};
template <>
struct Piece<float> {
  uint32_t u[8];
  __device__ __forceinline__ void load(const float* p) {
    const uint4 a = __ldg(reinterpret_cast<const uint4*>(p)), b = __ldg(reinterpret_cast<const uint4*>(p) + 1);
    u[0] = a.x; u[1] = a.y; u[2] = a.z; u[3] = a.w;
    u[4] = b.x; u[5] = b.y; u[6] = b.z; u[7] = b.w;
  }
  __device__ __forceinline__ void load(const float* p, int n) {
#pragma unroll
    for (int e = 0; e < 8; ++e) u[e] = e < n ? __float_as_uint(p[e]) : 0u;
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int e = 0; e < 8; ++e) u[e] = 0;
  }
  __device__ __forceinline__ uint32_t top() const {
    uint32_t m = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) m = max(m, u[e] & 0x7fffffffu);
    return m;
  }
  __device__ __forceinline__ void unpack(float (&v)[8]) const {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = __uint_as_float(u[e]);
  }
};
// Scale of a row from the pattern of its largest magnitude; NaN where that is not finite.
__device__ __forceinline__ float scale_of(uint32_t top) {
  if (top >= 0x7f800000u) return __int_as_float(0x7fffffff);
  const float s = __fdiv_rn(__uint_as_float(top), 127.f);
  return s == 0.f ? 1.f : s;
}
// Codes of a piece under scale s; inv = reciprocal_of(s).
__device__ __forceinline__ float reciprocal_of(float s) { return s >= 0x1p-120f ? 1.f / s : 0.f; }  // of tiny ones it is no number to multiply by
template <typename T>
__device__ __forceinline__ uint2 encode(const Piece<T>& p, float s, float inv) {
  if (!(s > 0.f)) return make_uint2(0u, 0u);  // NaN
  float f[8];
  p.unpack(f);
  if (inv > 0.f) return codes_of(f, s, inv);
  uint32_t w[2] = {0u, 0u};
#pragma unroll
  for (int e = 0; e < 8; ++e) w[e / 4] |= (uint32_t)(max(-127, min(127, __float2int_rn(__fdiv_rn(f[e], s)))) & 255) << (8 * (e & 3));
  return make_uint2(w[0], w[1]);
}

// PV pieces of 8 columns a thread in registers (0: any width, the row is read twice); VEC: 16-byte loads, 8-byte stores.
template <typename T, int PV, bool VEC, int kThreads>
__global__ void __launch_bounds__(kThreads) quant_rows_kernel(const QuantArgs a) {
  __shared__ uint32_t tops[kThreads / 32];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int tid = threadIdx.x, row = blockIdx.x;
  const T* x = static_cast<const T*>(a.x) + (long long)row * a.x_stride;
  int8_t* codes = a.codes + (long long)row * a.codes_stride;
  constexpr int N = PV > 0 ? PV : 1;
  Piece<T> v[N];
  uint32_t top = 0;
  auto fetch = [&](Piece<T>& p, int at) {
    if (VEC) p.load(x + at);
    else p.load(x + at, a.K - at);
  };
  if (PV > 0) {
#pragma unroll
    for (int p = 0; p < N; ++p) {
      const int at = (p * kThreads + tid) * 8;
      if (at < a.K) fetch(v[p], at);
      else v[p].clear();
    }
#pragma unroll
    for (int p = 0; p < N; ++p) top = max(top, v[p].top());
  } else {
    for (int at = tid * 8; at < a.K; at += 8 * kThreads) {
      fetch(v[0], at);
      top = max(top, v[0].top());
    }
  }
  top = __reduce_max_sync(0xffffffffu, top);
  if ((tid & 31) == 0) tops[tid >> 5] = top;
  __syncthreads();
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
#pragma unroll
  for (int w = 0; w < kThreads / 32; ++w) top = max(top, tops[w]);
  const float s = scale_of(top), inv = reciprocal_of(s);
  if (tid == 0) a.scales[row] = s;
  auto put = [&](int at, const Piece<T>& p) {
    const uint2 u = encode(p, s, inv);
    if (VEC) {
      *reinterpret_cast<uint2*>(codes + at) = u;
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (at + e < a.K) codes[at + e] = (int8_t)((e < 4 ? u.x : u.y) >> (8 * (e & 3)));
    }
  };
  if (PV > 0) {
#pragma unroll
    for (int p = 0; p < N; ++p) {
      const int at = (p * kThreads + tid) * 8;
      if (at < a.K) put(at, v[p]);
    }
  } else {
    for (int at = tid * 8; at < a.K; at += 8 * kThreads) {
      fetch(v[0], at);
      put(at, v[0]);
    }
  }
}

// ---------------------------------------------------------------- product
struct Args {
  const float *sx, *sw, *bias;
  void* y;
  long long y_stride;
  int32_t* status;  // or null
  int n, N, steps;  // tokens, channels, steps of K
  int y_f32;
  int early;        // the kernel in front brings x to codes: the weight can be fetched before it has ended
  int wide_tiles, narrow_tiles;  // tiles of 256 tokens, of 256 channels
  const void* x;                 // rows that few_kernel brings to codes itself
  long long x_stride;
  int K;
};
__device__ __forceinline__ void mma_i8(uint32_t d_tmem, uint32_t a_lo, uint32_t b_lo, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "mov.b64 da, {%1, %5};\n\tmov.b64 db, {%2, %5};\n\t"
      "tcgen05.mma.cta_group::1.kind::i8 [%0], da, db, %3, p;\n\t}" ::"r"(d_tmem),
      "r"(a_lo), "r"(b_lo), "r"(idesc), "r"(accumulate), "r"(ptx::kDescHiSw128)
      : "memory");
}
// signed 8-bit operands (K-major), 32-bit integer sums, M = 128
__device__ __forceinline__ uint32_t idesc_i8(uint32_t n) { return (2u << 4) | (1u << 7) | (1u << 10) | ((n >> 3) << 17) | (8u << 24); }

__device__ __forceinline__ bool wait(uint64_t* bar, uint32_t parity, volatile int* abort_flag, int32_t* status) {
  if (ptx::mbar_try_wait(bar, parity)) return true;
  const uint64_t t0 = ptx::globaltimer_ns();
  for (uint32_t it = 1;; ++it) {
    if (ptx::mbar_try_wait(bar, parity)) return true;
    if ((it & 127u) == 0) {
      if (*abort_flag) return false;
      if (ptx::globaltimer_ns() - t0 > kBudgetNs) {
        *abort_flag = 1;
        kv::report(status, 4);
        return false;
      }
    }
  }
}
__device__ __forceinline__ bool wait_warp(uint64_t* bar, uint32_t parity, volatile int* abort_flag, int32_t* status, int lane) {
  int r = 1;
  if (lane == 0) r = wait(bar, parity, abort_flag, status);
  return __shfl_sync(0xffffffffu, r, 0) != 0;
}
__device__ __forceinline__ void store_y(const Args& a, long long row, int col, float v) {
  if (a.y_f32) static_cast<float*>(a.y)[row * a.y_stride + col] = v;
  else static_cast<__nv_bfloat16*>(a.y)[row * a.y_stride + col] = __float2bfloat16_rn(v);
}

struct Ctl {
  uint64_t full[8], empty[8], done[2], freed[2], drain;
  uint32_t tmem;
  volatile int abort;
  volatile uint32_t loaded;
};

// ---- many tokens
// Two CTAs (a cluster, on neighbouring SMs) compute a tile of 256 tokens x 256 channels together: each holds 128 of the tokens and 128 of the
// channels, the tensor cores read the other's channels too.  One CTA alone would fetch and read 96 KB of shared memory per 512 cycles of MMA,
// more than the 128 bytes a cycle that there are (8001 x 7168 -> 9217: 400 us); a pair needs 64 KB each.
constexpr int kWide = 256, kManyStages = 5, kManyStage = 256 * kStep, kManyThreads = 320;
__device__ __forceinline__ uint32_t in_leader(const void* p) {  // the same place in the cluster's first CTA
  uint32_t r;
  asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(ptx::smem_u32(p)));
  return r;
}
__device__ __forceinline__ void pair_load(void* dst, const void* tmap, uint32_t bar, int c0, int c1) {
  asm volatile(
      "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1, {%3, %4}], [%2], %5;" ::"r"(
          ptx::smem_u32(dst)),
      "l"(tmap), "r"(bar), "r"(c0), "r"(c1), "l"(ptx::kPolicyEvictNormal)
      : "memory");
}
__device__ __forceinline__ void pair_mma(uint32_t d_tmem, uint32_t a_lo, uint32_t b_lo, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "mov.b64 da, {%1, %5};\n\tmov.b64 db, {%2, %5};\n\t"
      "tcgen05.mma.cta_group::2.kind::i8 [%0], da, db, %3, p;\n\t}" ::"r"(d_tmem),
      "r"(a_lo), "r"(b_lo), "r"(idesc), "r"(accumulate), "r"(ptx::kDescHiSw128)
      : "memory");
}
// What was issued so far, when it has ended, arrives on the barrier in both CTAs.
__device__ __forceinline__ void pair_commit(uint64_t* bar) {
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(ptx::smem_u32(bar)), "h"((uint16_t)3)
               : "memory");
}
__device__ __forceinline__ void pair_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
constexpr int kTurn = 32 * 128;  // bytes in which a warp turns 128 bytes of each of its rows of y
constexpr size_t many_smem() { return 1024 + kManyStages * kManyStage + 8 * kTurn + 4 * kWide * 4 + sizeof(Ctl); }
static_assert(many_smem() <= 227 * 1024, "shared memory");

template <bool F32>
__global__ void __launch_bounds__(kManyThreads, 1) many_kernel(const Args a, const __grid_constant__ CUtensorMap tm_x, const __grid_constant__ CUtensorMap tm_w) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  uint8_t* stage_y = smem + kManyStages * kManyStage;
  float* stage_s = reinterpret_cast<float*>(stage_y + 8 * kTurn);  // by tile parity: scales, then biases, of the tile's channels
  Ctl& S = *reinterpret_cast<Ctl*>(stage_s + 4 * kWide);
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  uint32_t rank;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  if (tid == 0) {
    for (int i = 0; i < kManyStages; ++i) {
      ptx::mbar_init(&S.full[i], 1);
      ptx::mbar_init(&S.empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      ptx::mbar_init(&S.done[i], 1);
      ptx::mbar_init(&S.freed[i], 16);  // (the first CTA's) 8 warps of each
    }
    ptx::mbar_init(&S.drain, 1);
    ptx::fence_mbar_init();
    S.abort = 0;
    S.loaded = 0;
  }
  if (warp == 4 && lane == 0) {
    ptx::prefetch_tmap(&tm_x);
    ptx::prefetch_tmap(&tm_w);
  }
  asm volatile("griddepcontrol.wait;" ::: "memory");
  if (warp == 5) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(ptx::smem_u32(&S.tmem)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  ptx::tc_fence_before();
  __syncwarp();
  pair_sync();  // also: the barriers of both are there
  ptx::tc_fence_after();
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const uint32_t tmem = S.tmem;
  const int tiles = a.wide_tiles * a.narrow_tiles;
  // tiles of channels in bands of 8, the tokens' tiles inside: CTAs at work share what they read
  auto tile_at = [&](int i, int& mt, int& nt) {
    const int band = i / (8 * a.wide_tiles), width = min(8, a.narrow_tiles - band * 8), r = i - band * 8 * a.wide_tiles;
    mt = r / width;
    nt = band * 8 + r % width;
  };
  if (warp == 4) {
    if (lane == 0) {
      uint32_t it = 0;
      bool ok = true;
      for (int i = blockIdx.x >> 1; i < tiles && ok; i += gridDim.x >> 1) {
        int mt, nt;
        tile_at(i, mt, nt);
        for (int k = 0; k < a.steps; ++k, ++it) {
          const int st = it % kManyStages;
          if (it >= kManyStages && !wait(&S.empty[st], ((it / kManyStages) & 1) ^ 1, &S.abort, a.status)) {
            ok = false;
            break;
          }
          if (MOEV_TEST_WITHHOLD() && k == a.steps - 1) {
            ok = false;
            break;
          }
          // both CTAs' copies count on the first one's barrier
          if (rank == 0) ptx::mbar_arrive_expect_tx(&S.full[st], 2 * kManyStage);
          S.loaded = it + 1;
          uint8_t* dst = smem + st * kManyStage;
          const uint32_t bar = in_leader(&S.full[st]);
          pair_load(dst, &tm_x, bar, k * kStep, mt * 256 + (int)rank * 128);
          pair_load(dst + 128 * kStep, &tm_w, bar, k * kStep, nt * kWide + (int)rank * 128);
        }
      }
    }
  } else if (warp == 5) {
    if (rank == 0 && ptx::elect_one()) {
      uint32_t it = 0;
      bool ok = true;
      int count = 0;
      const uint32_t lo = ptx::desc_lo_sw128(ptx::smem_u32(smem));
      for (int i = blockIdx.x >> 1; i < tiles && ok; i += gridDim.x >> 1, ++count) {
        const int u = count & 1;
        if (count >= 2) ok = wait(&S.freed[u], ((count >> 1) & 1) ^ 1, &S.abort, a.status);
        for (int k = 0; k < a.steps && ok; ++k, ++it) {
          const int st = it % kManyStages;
          ok = wait(&S.full[st], (it / kManyStages) & 1, &S.abort, a.status);
          if (!ok) break;
          ptx::tc_fence_after();
          const uint32_t base = lo + st * (kManyStage / 16);
#pragma unroll
          for (int e = 0; e < 4; ++e) pair_mma(tmem + u * kWide, base + e * 2, base + 128 * kStep / 16 + e * 2, idesc_i8(kWide) + (8u << 24), k + e > 0);  // M = 256
          pair_commit(&S.empty[st]);
        }
        if (ok) pair_commit(&S.done[u]);
      }
      if (!ok) {  // abort: what was issued must have ended
        pair_commit(&S.drain);
        ptx::drain_wait(&S.drain, 0u, kBudgetNs);
      }
    }
  } else {
    // A thread has a token's row of sums; 128 bytes of y of each row (64 or 32 channels) change places in shared memory so that
    // a row is written by 8 lanes, where its address allows 16 bytes each, or by all.
    int count = 0;
    const int half = warp > 5, quarter = warp & 3, worker = (half ? warp - 2 : warp) * 32 + lane;  // two warps share the columns of 32 rows
    uint8_t* const turn = stage_y + (worker >> 5) * kTurn;
    constexpr int kCols = F32 ? 32 : 64, kSize = F32 ? 4 : 2;
    const bool vec = (reinterpret_cast<uintptr_t>(a.y) & 15) == 0 && a.y_stride * kSize % 16 == 0;
    uint8_t* const y = static_cast<uint8_t*>(a.y);
    for (int i = blockIdx.x >> 1; i < tiles; i += gridDim.x >> 1, ++count) {
      const int u = count & 1;
      int mt, nt;
      tile_at(i, mt, nt);
      float* const sw = stage_s + u * 2 * kWide;  // that of two tiles ago has been read: every warp passed a barrier since
      {
        const int e = worker;
        const int col = nt * kWide + e;
        sw[e] = col < a.N ? a.sw[col] : 0.f;
        sw[kWide + e] = a.bias && col < a.N ? a.bias[col] : 0.f;
      }
      ptx::named_barrier(1, 256);
      wait_warp(&S.done[u], (count >> 1) & 1, &S.abort, a.status, lane);  // one that ran out: on to the end, y is undefined then
      ptx::tc_fence_after();
      const int row0 = mt * 256 + (int)rank * 128 + quarter * 32;
      const float sx = row0 + lane < a.n ? a.sx[row0 + lane] : 0.f;
#pragma unroll 1
      for (int c0 = half * kCols; c0 < kWide && nt * kWide + c0 < a.N; c0 += 2 * kCols) {
#pragma unroll
        for (int h = 0; h < kCols / 32; ++h) {
          uint32_t r[32];
          ptx::tmem_ld32(tmem + ((uint32_t)quarter << 21) + u * kWide + c0 + h * 32, r);
          ptx::tmem_ld_wait();
#pragma unroll
          for (int e = 0; e < 32; e += 16 / kSize) {
            uint32_t w[4];
#pragma unroll
            for (int z = 0; z < 16 / kSize; z += 4) {
              const float4 s4 = *reinterpret_cast<const float4*>(sw + c0 + h * 32 + e + z), b4 = *reinterpret_cast<const float4*>(sw + kWide + c0 + h * 32 + e + z);
              const float v0 = fmaf((float)(int)r[e + z] * sx, s4.x, b4.x), v1 = fmaf((float)(int)r[e + z + 1] * sx, s4.y, b4.y);
              const float v2 = fmaf((float)(int)r[e + z + 2] * sx, s4.z, b4.z), v3 = fmaf((float)(int)r[e + z + 3] * sx, s4.w, b4.w);
              if (F32) {
                w[0] = __float_as_uint(v0); w[1] = __float_as_uint(v1); w[2] = __float_as_uint(v2); w[3] = __float_as_uint(v3);
              } else {
                const __nv_bfloat162 lo = __floats2bfloat162_rn(v0, v1), hi = __floats2bfloat162_rn(v2, v3);
                w[z / 2] = *reinterpret_cast<const uint32_t*>(&lo);
                w[z / 2 + 1] = *reinterpret_cast<const uint32_t*>(&hi);
              }
            }
            const int piece = (h * 32 + e) * kSize / 16;
            *reinterpret_cast<uint4*>(turn + lane * 128 + ((piece ^ (lane & 7)) << 4)) = make_uint4(w[0], w[1], w[2], w[3]);
          }
        }
        __syncwarp();
        const int col0 = nt * kWide + c0, cols = min(kCols, a.N - col0);
        if (vec && cols == kCols) {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int r = e * 4 + (lane >> 3), piece = lane & 7;
            const uint4 w = *reinterpret_cast<const uint4*>(turn + r * 128 + ((piece ^ (r & 7)) << 4));
            if (row0 + r < a.n) *reinterpret_cast<uint4*>(y + ((long long)(row0 + r) * a.y_stride + col0) * kSize + piece * 16) = w;
          }
        } else {
          const int rows = min(32, a.n - row0);
#pragma unroll 1
          for (int r0 = 0; r0 < rows; r0 += 8) {
#pragma unroll
            for (int r = r0; r < r0 + 8; ++r) {  // rows behind the last one are read, not written
              uint8_t* const out = y + ((long long)(row0 + r) * a.y_stride + col0) * kSize;
              auto at = [&](int byte) { return turn + r * 128 + (((byte >> 4) ^ (r & 7)) << 4) + (byte & 15); };
              if (F32) {
                const uint32_t w = *reinterpret_cast<const uint32_t*>(at(lane * 4));
                if (lane < cols && r < rows) *reinterpret_cast<uint32_t*>(out + lane * 4) = w;
              } else {
                // pairs from the first address that is a multiple of 4, what is left at the ends alone
                const int odd = (int)(reinterpret_cast<uintptr_t>(out) >> 1) & 1, c = 2 * lane + odd;
                const uint32_t lo = *reinterpret_cast<const uint16_t*>(at(c * 2)), hi = *reinterpret_cast<const uint16_t*>(at((c * 2 + 2) & 127));
                if (r < rows) {
                  if (c + 1 < cols) *reinterpret_cast<uint32_t*>(out + c * 2) = lo | hi << 16;
                  else if (c < cols) *reinterpret_cast<uint16_t*>(out + c * 2) = (uint16_t)lo;
                  if (odd && lane == 31) *reinterpret_cast<uint16_t*>(out) = (uint16_t)hi;  // the first one: 31 is left with c = 63
                }
              }
            }
          }
        }
        __syncwarp();
      }
      ptx::tc_fence_before();
      __syncwarp();
      if (lane == 0) asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(in_leader(&S.freed[u])) : "memory");
    }
  }
  ptx::tc_fence_before();
  __syncthreads();
  // (the first CTA's barriers count the copies of both; the other one waits for it below)
  if (S.abort && rank == 0 && tid == 128) ptx::drain_ring(S.full, kManyStages, S.loaded, kBudgetNs);
  __syncwarp();
  pair_sync();
  ptx::tc_fence_after();
  if (warp == 5) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
}

// ---- few tokens: NT columns of tokens
template <int NT>
struct Few {
  static constexpr int kStages = NT <= 32 ? 5 : NT <= 64 ? 4 : 3;  // two CTAs fit on an SM
  static constexpr int kStage = (128 + NT) * kStep;
  static constexpr int kTmem = NT < 32 ? 32 : NT;
  static constexpr size_t smem() { return 1024 + (size_t)kStages * kStage + sizeof(Ctl); }
  static_assert(kStages * kStage >= NT * 128 * 4, "the sums take the ring's place");
};

// X: the type of rows that the kernel brings to codes itself (void: they come as codes).  Every CTA reads all of the rows for their maxima, then four
// warps in turn write the codes of a step into the ring beside the weight that TMA puts there.  One launch less, but each CTA's own work grows with the
// rows (us, own | two launches: 1 x 8192 -> 4096 8.9 | 10.5, 1 x 2880 -> 5120 6.5 | 7.3, 2 rows 9.6 | 10.7 and 7.3 | 7.8, 3 rows 10.4 | 10.7 and 7.9 | 7.3;
// 4096 -> 60000, where an SM takes four CTAs in turn, 1 row 39.1 | 40.1, 2 rows 41.7 | 40.0).
constexpr int kOwnRows = 2;
template <int NT, typename X>
__global__ void __launch_bounds__(192) few_kernel(const Args a, const __grid_constant__ CUtensorMap tm_x, const __grid_constant__ CUtensorMap tm_w) {
  using C = Few<NT>;
  constexpr bool kOwn = !std::is_void<X>::value;
  constexpr int kBytes = kOwn ? 128 * kStep : C::kStage;  // of a stage that TMA brings
  __shared__ uint32_t tops[kOwnRows][4];
  __shared__ float scales[kOwnRows];
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  Ctl& S = *reinterpret_cast<Ctl*>(smem + C::kStages * C::kStage);
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  uint32_t rank, ranks;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(ranks));
  const int tile = blockIdx.x / ranks, n0 = blockIdx.y * NT;
  if (tid == 0) {
    for (int i = 0; i < C::kStages; ++i) {
      ptx::mbar_init(&S.full[i], kOwn ? 2 : 1);
      ptx::mbar_init(&S.empty[i], 1);
    }
    ptx::mbar_init(&S.done[0], 1);
    ptx::mbar_init(&S.drain, 1);
    ptx::fence_mbar_init();
    S.abort = 0;
    S.loaded = 0;
  }
  const int first = (int)((long long)a.steps * rank / ranks), last = (int)((long long)a.steps * (rank + 1) / ranks);
  __syncthreads();
  const int fetched = kOwn || a.early ? min(last - first, C::kStages) : 0;
  if (kOwn) asm volatile("griddepcontrol.wait;" ::: "memory");
  if (warp == 4 && lane == 0) {
    if (!kOwn) ptx::prefetch_tmap(&tm_x);
    ptx::prefetch_tmap(&tm_w);
    for (int it = 0; it < fetched; ++it) {
      ptx::mbar_arrive_expect_tx(&S.full[it], kBytes);
      ptx::tma_load_2d(smem + it * C::kStage, &tm_w, &S.full[it], (first + it) * kStep, tile * 128, ptx::kPolicyEvictFirst);
    }
    S.loaded = fetched;
  }
  if (!kOwn) asm volatile("griddepcontrol.wait;" ::: "memory");
  if (warp == 5) {
    ptx::tmem_alloc(&S.tmem, C::kTmem);
    ptx::tmem_relinquish();
  }
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const uint32_t tmem = S.tmem;
  if (warp == 4) {
    if (lane == 0) {
      for (int k = first; k < last; ++k) {
        const int it = k - first, st = it % C::kStages;
        if (it >= C::kStages && !wait(&S.empty[st], ((it / C::kStages) & 1) ^ 1, &S.abort, a.status)) break;
        if (it >= fetched) {
          ptx::mbar_arrive_expect_tx(&S.full[st], kBytes);
          ptx::tma_load_2d(smem + st * C::kStage, &tm_w, &S.full[st], k * kStep, tile * 128, ptx::kPolicyEvictFirst);
        }
        if (!kOwn && MOEV_TEST_WITHHOLD() && k == last - 1) break;
        S.loaded = max(it + 1, fetched);
        if (!kOwn) ptx::tma_load_2d(smem + st * C::kStage + 128 * kStep, &tm_x, &S.full[st], k * kStep, n0, ptx::kPolicyEvictLast);
      }
    }
  } else if (warp == 5) {
    if (ptx::elect_one()) {
      const uint32_t lo = ptx::desc_lo_sw128(ptx::smem_u32(smem));
      bool ok = true;
      for (int k = first; k < last; ++k) {
        const int it = k - first, st = it % C::kStages;
        ok = wait(&S.full[st], (it / C::kStages) & 1, &S.abort, a.status);
        if (!ok) break;
        ptx::tc_fence_after();
        const uint32_t base = lo + st * (C::kStage / 16);
#pragma unroll
        for (int e = 0; e < 4; ++e) mma_i8(tmem, base + e * 2, base + 128 * kStep / 16 + e * 2, idesc_i8(NT), it + e > 0);
        ptx::mma_commit(&S.empty[st]);
      }
      if (ok) ptx::mma_commit(&S.done[0]);
      else ptx::drain_issuer(&S.drain, kBudgetNs);
    }
  } else if constexpr (kOwn) {
    const X* x = static_cast<const X*>(a.x);
    for (int r = 0; r < a.n; ++r) {
      uint32_t top = 0;
      for (int p0 = tid * 8; p0 < a.K; p0 += 8 * 1024) {
        Piece<X> v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          if (p0 + e * 1024 < a.K) v[e].load(x + r * a.x_stride + p0 + e * 1024);
          else v[e].clear();
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) top = max(top, v[e].top());
      }
      top = __reduce_max_sync(0xffffffffu, top);
      if (lane == 0) tops[r][warp] = top;
    }
    asm volatile("bar.sync 1, 128;" ::: "memory");
    // a half of a warp for each row
    const int r = lane >> 4;
    const bool mine = r < a.n;
    const float s = mine ? scale_of(max(max(tops[r][0], tops[r][1]), max(tops[r][2], tops[r][3]))) : 1.f, inv = reciprocal_of(s);
    if (mine && warp == 0 && (lane & 15) == 0) scales[r] = s;
    for (int k = first + warp; k < last; k += 4) {
      const int it = k - first, st = it % C::kStages, at = k * kStep + (lane & 15) * 8;
      Piece<X> v;
      if (mine && at < a.K) v.load(x + r * a.x_stride + at);
      else v.clear();
      if (it >= C::kStages && !wait_warp(&S.empty[st], ((it / C::kStages) & 1) ^ 1, &S.abort, a.status, lane)) break;
      if (MOEV_TEST_WITHHOLD() && k == last - 1) break;
      // rows of 128 bytes with their 16-byte pieces in the order that the swizzle gives; rows behind the last token make sums that nobody reads
      if (mine)
        *reinterpret_cast<uint2*>(smem + st * C::kStage + 128 * kStep + r * kStep + ((((lane & 15) >> 1) ^ r) << 4) + (lane & 1) * 8) = encode(v, s, inv);
      ptx::fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(&S.full[st]);
    }
  }
  // sums of this CTA's part of K: [token][channel], in the ring's place (all of it has been read)
  int* part = reinterpret_cast<int*>(smem);
  const int tokens = min(NT, a.n - n0);
  if (warp < 4) {
    bool ok = first < last;
    if (ok) ok = wait_warp(&S.done[0], 0, &S.abort, a.status, lane);
    ptx::tc_fence_after();
    for (int c0 = 0; c0 < tokens; c0 += 16) {
      uint32_t r[16];
      if (ok) {
        ptx::tmem_ld16(tmem + ((uint32_t)warp << 21) + c0, r);
        ptx::tmem_ld_wait();
      }
#pragma unroll
      for (int e = 0; e < 16; ++e) part[(c0 + e) * 128 + tid] = ok ? (int)r[e] : 0;
    }
  }
  ptx::tc_fence_before();
  __syncwarp();
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
  ptx::tc_fence_after();
  if (warp < 4) {
    // a warp takes a token, a lane 4 channels of it, from all CTAs of the cluster
    const int col = tile * 128 + lane * 4;
    float sw[4], bias[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      sw[e] = col + e < a.N ? a.sw[col + e] : 0.f;
      bias[e] = a.bias && col + e < a.N ? a.bias[col + e] : 0.f;
    }
    const int es = a.y_f32 ? 4 : 2;
    const bool vec = col + 3 < a.N && a.y_stride % 4 == 0 && (reinterpret_cast<uintptr_t>(a.y) & (4 * es - 1)) == 0;
    uint32_t at[8];
#pragma unroll
    for (uint32_t p = 0; p < 8; ++p) {
      at[p] = 0;
      if (p < ranks) asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at[p]) : "r"(ptx::smem_u32(part + lane * 4)), "r"(p));
    }
#pragma unroll 2
    for (int t = warp * ranks + rank; t < tokens; t += 4 * ranks) {
      int4 v[8];
#pragma unroll
      for (uint32_t p = 0; p < 8; ++p)
        if (p < ranks)
          asm volatile("ld.shared::cluster.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v[p].x), "=r"(v[p].y), "=r"(v[p].z), "=r"(v[p].w) : "r"(at[p] + t * 512));
      int4 sum = make_int4(0, 0, 0, 0);
#pragma unroll
      for (uint32_t p = 0; p < 8; ++p)
        if (p < ranks) {
          sum.x += v[p].x;
          sum.y += v[p].y;
          sum.z += v[p].z;
          sum.w += v[p].w;
        }
      const float sx = kOwn ? scales[t] : a.sx[n0 + t];
      const float y[4] = {fmaf((float)sum.x * sx, sw[0], bias[0]), fmaf((float)sum.y * sx, sw[1], bias[1]), fmaf((float)sum.z * sx, sw[2], bias[2]),
                          fmaf((float)sum.w * sx, sw[3], bias[3])};
      const long long out = (long long)(n0 + t) * a.y_stride + col;
      if (vec && a.y_f32) {
        *reinterpret_cast<float4*>(static_cast<float*>(a.y) + out) = make_float4(y[0], y[1], y[2], y[3]);
      } else if (vec) {
        const __nv_bfloat162 lo = __floats2bfloat162_rn(y[0], y[1]), hi = __floats2bfloat162_rn(y[2], y[3]);
        *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(a.y) + out) = make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (col + e < a.N) store_y(a, n0 + t, col + e, y[e]);
      }
    }
  }
  __syncwarp();
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
  if (S.abort && tid == 128) ptx::drain_ring(S.full, C::kStages, S.loaded, kBudgetNs);
  if (warp == 5) ptx::tmem_dealloc(tmem, C::kTmem);
}

}  // namespace i8
}  // namespace moev
