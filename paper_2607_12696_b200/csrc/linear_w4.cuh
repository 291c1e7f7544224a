// y[n, N] = x[n, K] W^T + bias for a few rows of x and 4-bit weights with group scales.
//
//   INT4:  W[o, k] = (q[o, k] - 8) * s[o, k / group]     q in 0..15, s bf16, group 32, 64 or 128
//   MXFP4: W[o, k] = e2m1(q[o, k]) * 2^(s[o, k / 32] - 127)
//
// The codes are exact in bf16, so the products with bf16 activations are exact too; mma.sync adds
// them in binary32 over one group, the group's sum is multiplied by the binary32 scale and added to
// the output's binary32 accumulator: no weight and no partial sum is rounded to fewer bits.
// Bound by the weight stream (N K / 2 bytes + scales): 1.6 FLOP per byte and row of x.
//
// Packed layout (made once per weight, moev_w4_pack).  The weights are the A operand (16 outputs x
// 16 k) and the tokens the B operand (8 columns), since a few tokens fill the narrow side.  A tile of
// 16 outputs and a chunk of 128 k are 1024 consecutive bytes in the order in which the 32 lanes want
// them: half h (64 k), lane 4 g + t, four words {row g, row g + 8} x {32-k block 2 h, 2 h + 1}, each
// word the 8 codes k = 8 t .. 8 t + 7 of its block.  So a warp reads a chunk with two fully used
// 512-byte loads straight into registers, and its B operand for the two MMAs of a block is x[8 t ..
// 8 t + 7]: one 16-byte shared-memory load.  Which k an MMA calls its k-th is free as long as both
// operands agree.  Scales: tile, chunk, row pair g: {row g, row g + 8} x the chunk's 128 / group scales.
#pragma once
#include "common.cuh"

namespace moev {
namespace w4 {

constexpr int kInt4 = 0, kMx = 1;
constexpr int kTileRows = 16, kChunk = 128, kChunkBytes = 1024;
constexpr int kDepth = 4;  // chunks a warp keeps in flight

struct Args {
  const uint8_t* codes;   // packed
  const uint8_t* scales;  // packed
  const __nv_bfloat16* x;
  const float* bias;
  void* y;
  long long x_stride, y_stride;
  int n, N, K, n_chunks;   // n: rows of x in all
  int n_groups;            // row groups of RW tiles
  int kw;                  // warps that share a tile's K
  int phase_chunks;        // chunks of K per staged piece of x (a multiple of kw)
  int x_pitch;             // bytes per staged row
  int n_bufs;              // 1: x is staged whole, 2: piece by piece
  int y_f32, x_vec;
};

// 8 codes of a word -> 4 bf16 pairs, pair p = k 2 p and 2 p + 1.
template <int FMT>
__device__ __forceinline__ void decode(uint32_t w, uint32_t (&r)[4]) {
  if constexpr (FMT == kInt4) {
    // nibble p = k 2 p, nibble p + 4 = k 2 p + 1.  0x4300 | q is 128 + q in bf16; minus 136 is exact.
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      const uint32_t u = ((w >> (4 * p)) & 0x000F000Fu) | 0x43004300u;
      __nv_bfloat162 v = *reinterpret_cast<const __nv_bfloat162*>(&u);
      v = __hsub2(v, __floats2bfloat162_rn(136.f, 136.f));
      r[p] = *reinterpret_cast<uint32_t*>(&v);
    }
  } else {
    // magnitudes in order (nibble i = k i), looked up bytewise: {0, .5, 1, 1.5, 2, 3, 4, 6} as bf16; signs apart:
    // bit 4 p + 3 that of k 2 p, bit 4 p + 19 that of k 2 p + 1.
    const uint32_t s0 = w & 0x77777777u, s1 = s0 >> 16;
    const uint32_t l0 = __byte_perm(0xC0800000u, 0xC0804000u, s0), h0 = __byte_perm(0x3F3F3F00u, 0x40404040u, s0);
    const uint32_t l1 = __byte_perm(0xC0800000u, 0xC0804000u, s1), h1 = __byte_perm(0x3F3F3F00u, 0x40404040u, s1);
    r[0] = __byte_perm(l0, h0, 0x5140) | ((w << 12) & 0x80008000u);
    r[1] = __byte_perm(l0, h0, 0x7362) | ((w << 8) & 0x80008000u);
    r[2] = __byte_perm(l1, h1, 0x5140) | ((w << 4) & 0x80008000u);
    r[3] = __byte_perm(l1, h1, 0x7362) | (w & 0x80008000u);
  }
}

__device__ __forceinline__ void mma_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// GB: 32-k blocks per scale (1, 2, 4); MXFP4 has one byte per block.
template <int FMT, int GB>
struct Scales {
  static constexpr int kPerRow = 4 / GB;                                 // scales per row and chunk
  static constexpr int kBytes = 16 * kPerRow * (FMT == kInt4 ? 2 : 1);  // per tile and chunk
  static constexpr int kLane = kBytes / 8;                               // per row pair: 16, 8, 4 (INT4) or 8 (MXFP4)
  uint32_t u[kLane / 4];
  __device__ __forceinline__ void load(const uint8_t* p) {
    if constexpr (kLane == 16) { const uint4 q = __ldg(reinterpret_cast<const uint4*>(p)); u[0] = q.x; u[1] = q.y; u[2] = q.z; u[3] = q.w; }
    else if constexpr (kLane == 8) { const uint2 q = __ldg(reinterpret_cast<const uint2*>(p)); u[0] = q.x; u[1] = q.y; }
    else u[0] = __ldg(reinterpret_cast<const unsigned int*>(p));
  }
  // scale of row g (half 0) or g + 8 (half 1) for the i-th group of the chunk
  __device__ __forceinline__ float get(int half, int i) const {
    const int at = half * kPerRow + i;
    if constexpr (FMT == kInt4) return bf16_bits_to_float((u[at >> 1] >> (16 * (at & 1))) & 0xffffu);
    else return e8m0_to_float((u[at >> 2] >> (8 * (at & 3))) & 0xffu);
  }
};

// Stage columns [c0, c0 + cols) (cols a multiple of 128, columns from K on as zero) of rows [0, rows) of x.
__device__ __forceinline__ void stage_x(const Args& a, const __nv_bfloat16* x, int rows, uint32_t dst, int c0, int cols) {
  const int per = cols / 8;
  for (int i = threadIdx.x; i < rows * per; i += blockDim.x) {
    const int r = i / per, c = (i - r * per) * 8;
    const uint32_t to = dst + (uint32_t)r * a.x_pitch + c * 2;
    const __nv_bfloat16* from = x + (long long)r * a.x_stride + c0 + c;
    if (c0 + c >= a.K) {  // K is a multiple of 32: a piece of 8 lies inside or outside
      asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(to), "r"(0) : "memory");
    } else if (a.x_vec) {
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
    } else {
      uint32_t u[4];
#pragma unroll
      for (int j = 0; j < 4; ++j)
        u[j] = (uint32_t)__bfloat16_as_ushort(from[2 * j]) | ((uint32_t)__bfloat16_as_ushort(from[2 * j + 1]) << 16);
      asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to), "r"(u[0]), "r"(u[1]), "r"(u[2]), "r"(u[3]) : "memory");
    }
  }
}

// CTA: blockDim / 32 warps = rw x kw; warp (r, k) takes tile r of the row group and every kw-th chunk of
// K, beginning with chunk k.  Row groups go round the grid; the sums of the kw warps meet in shared
// memory, in warp order.  Rows of x beyond 8 NT are the business of other blockIdx.y.
template <int FMT, int GB, int NT>
__global__ void __launch_bounds__(512, 1) linear_w4_kernel(const Args a) {
  extern __shared__ __align__(128) uint8_t smem[];
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int warps = blockDim.x >> 5, kw_n = a.kw, rw_n = warps / kw_n;
  const int wk = warp % kw_n, wr = warp / kw_n;
  const int row0 = blockIdx.y * (8 * NT), rows = min(a.n - row0, 8 * NT);
  const __nv_bfloat16* x = a.x + (long long)row0 * a.x_stride;
  const int n_tiles = (a.N + kTileRows - 1) / kTileRows;
  const int per_group = (a.n_chunks + kw_n - 1) / kw_n;  // chunks per warp and row group
  const int groups = (a.n_groups - (int)blockIdx.x + (int)gridDim.x - 1) / (int)gridDim.x;
  const int total = groups * per_group;
  const uint32_t xs = (uint32_t)__cvta_generic_to_shared(smem);
  const uint32_t buf_bytes = (uint32_t)rows * a.x_pitch;
  float* red = reinterpret_cast<float*>(smem + (size_t)a.n_bufs * min(a.n, 8 * NT) * a.x_pitch);
  using Sc = Scales<FMT, GB>;

  // the i-th chunk of this warp
  uint4 wreg[kDepth][2];
  Sc sreg[kDepth];
  auto fetch = [&](int i, uint4 (&w)[2], Sc& s) {
    const int gi = i / per_group, c = (i - gi * per_group) * kw_n + wk;
    const int tile = ((int)blockIdx.x + gi * (int)gridDim.x) * rw_n + wr;
    if (i < total && c < a.n_chunks && tile < n_tiles) {
      const size_t at = (size_t)tile * a.n_chunks + c;
      const uint4* p = reinterpret_cast<const uint4*>(a.codes + at * kChunkBytes) + lane;
      w[0] = __ldcs(p);
      w[1] = __ldcs(p + 32);
      s.load(a.scales + at * Sc::kBytes + g * Sc::kLane);
    }
  };

  asm volatile("griddepcontrol.wait;" ::: "memory");
#pragma unroll
  for (int d = 0; d < kDepth; ++d) fetch(d, wreg[d], sreg[d]);
  const bool whole = a.n_bufs == 1;
  const int n_phases = (a.n_chunks + a.phase_chunks - 1) / a.phase_chunks;
  const int phase_items = a.phase_chunks / kw_n;
  // piece number q of x (phase q % n_phases of row group q / n_phases) into buffer q & 1
  auto stage = [&](int q) {
    if (q < groups * n_phases) {
      const int c0 = (q % n_phases) * a.phase_chunks;
      const int nc = min(a.phase_chunks, a.n_chunks - c0);
      stage_x(a, x, rows, xs + (whole ? 0u : (uint32_t)(q & 1) * buf_bytes), c0 * kChunk, nc * kChunk);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  stage(0);
  if (whole) {
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    __syncthreads();
  }

  float acc[NT][4] = {};
  int i = 0, j = 0, gi = 0, piece = 0;  // flat item, its place in the row group, row group, piece of x
  const int b_row = min(g, rows - 1);
  while (i < total) {
#pragma unroll
    for (int d = 0; d < kDepth; ++d, ++i) {
      if (i >= total) break;
      if (!whole && j % phase_items == 0) {
        asm volatile("cp.async.wait_group 0;" ::: "memory");
        __syncthreads();  // the piece has landed, and everybody has left the other buffer
        stage(piece + 1);
        ++piece;
      }
      const int c = j * kw_n + wk;
      const int tile = ((int)blockIdx.x + gi * (int)gridDim.x) * rw_n + wr;
      if (c < a.n_chunks && tile < n_tiles) {
        const uint32_t base = xs + (whole ? 0u : (uint32_t)((piece - 1) & 1) * buf_bytes) +
                              (uint32_t)((whole ? c : c % a.phase_chunks) * kChunk * 2 + t * 16);
        const uint32_t word[8] = {wreg[d][0].x, wreg[d][0].y, wreg[d][0].z, wreg[d][0].w,
                                  wreg[d][1].x, wreg[d][1].y, wreg[d][1].z, wreg[d][1].w};
#pragma unroll
        for (int gr = 0; gr < 4 / GB; ++gr) {
          float sum[NT][4] = {};
#pragma unroll
          for (int bb = 0; bb < GB; ++bb) {
            const int b = gr * GB + bb;  // 32-k block of the chunk
            uint32_t lo[4], hi[4];
            decode<FMT>(word[2 * b], lo);
            decode<FMT>(word[2 * b + 1], hi);
#pragma unroll
            for (int q = 0; q < NT; ++q) {
              uint32_t b0, b1, b2, b3;
              const uint32_t at = base + (uint32_t)(NT == 1 ? b_row : min(q * 8 + g, rows - 1)) * a.x_pitch + b * 64;
              asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(b0), "=r"(b1), "=r"(b2), "=r"(b3) : "r"(at));
              mma_bf16(sum[q], lo[0], hi[0], lo[1], hi[1], b0, b1);
              mma_bf16(sum[q], lo[2], hi[2], lo[3], hi[3], b2, b3);
            }
          }
          const float s0 = sreg[d].get(0, gr), s1 = sreg[d].get(1, gr);
#pragma unroll
          for (int q = 0; q < NT; ++q) {
            acc[q][0] = fmaf(s0, sum[q][0], acc[q][0]);
            acc[q][1] = fmaf(s0, sum[q][1], acc[q][1]);
            acc[q][2] = fmaf(s1, sum[q][2], acc[q][2]);
            acc[q][3] = fmaf(s1, sum[q][3], acc[q][3]);
          }
        }
      }
      fetch(i + kDepth, wreg[d], sreg[d]);
      if (++j == per_group) {
        // the row group is done: lane (g, t) holds outputs g and g + 8 of the tile for tokens 2 t and 2 t + 1
        if (kw_n == 1) {
#pragma unroll
          for (int q = 0; q < NT; ++q)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int o = tile * kTileRows + g + 8 * (e >> 1), r = q * 8 + 2 * t + (e & 1);
              if (tile < n_tiles && o < a.N && r < rows) {
                const float v = acc[q][e] + (a.bias ? a.bias[o] : 0.f);
                const long long at = (long long)(row0 + r) * a.y_stride + o;
                if (a.y_f32) static_cast<float*>(a.y)[at] = v;
                else static_cast<__nv_bfloat16*>(a.y)[at] = __float2bfloat16_rn(v);
              }
            }
        } else {
          // [warp][token][output], 17 floats a token
          float* mine = red + warp * (NT * 8 * 17);
#pragma unroll
          for (int q = 0; q < NT; ++q)
#pragma unroll
            for (int e = 0; e < 4; ++e) mine[(q * 8 + 2 * t + (e & 1)) * 17 + g + 8 * (e >> 1)] = acc[q][e];
          __syncthreads();
          const int first = ((int)blockIdx.x + gi * (int)gridDim.x) * rw_n * kTileRows;  // the group's first output
          for (int z = threadIdx.x; z < rw_n * kTileRows * rows; z += blockDim.x) {
            const int r = z / (rw_n * kTileRows), lo = z - r * (rw_n * kTileRows), o = first + lo;
            if (o < a.N) {
              const float* p = red + ((lo >> 4) * kw_n) * (NT * 8 * 17) + r * 17 + (lo & 15);
              float v = 0.f;
              for (int k = 0; k < kw_n; ++k) v += p[k * (NT * 8 * 17)];
              v += a.bias ? a.bias[o] : 0.f;
              const long long at = (long long)(row0 + r) * a.y_stride + o;
              if (a.y_f32) static_cast<float*>(a.y)[at] = v;
              else static_cast<__nv_bfloat16*>(a.y)[at] = __float2bfloat16_rn(v);
            }
          }
          __syncthreads();
        }
#pragma unroll
        for (int q = 0; q < NT; ++q)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[q][e] = 0.f;
        j = 0;
        ++gi;
      }
    }
  }
  asm volatile("cp.async.wait_group 0;" ::: "memory");
}

// One thread per packed word: tile, chunk, half h, lane 4 g + t, word {row g | g + 8} x {block 2 h | 2 h + 1}.
__global__ void pack_codes_kernel(const uint8_t* codes, uint32_t* out, int N, int K, int n_chunks, int fmt, long long words) {
  const long long z = (long long)blockIdx.x * blockDim.x + threadIdx.x;
  if (z >= words) return;
  const int word = (int)(z & 3), lane = (int)((z >> 2) & 31), h = (int)((z >> 7) & 1);
  const long long tc = z >> 8;
  const int chunk = (int)(tc % n_chunks);
  const long long tile = tc / n_chunks;
  const long long row = tile * kTileRows + (lane >> 2) + 8 * (word & 1);
  const int k = chunk * kChunk + (2 * h + (word >> 1)) * 32 + (lane & 3) * 8;
  uint32_t c = fmt == kInt4 ? 0x88888888u : 0u;  // zeros outside the matrix
  if (row < N && k < K) c = *reinterpret_cast<const uint32_t*>(codes + row * (long long)(K / 2) + k / 2);
  uint32_t r = 0;
  if (fmt == kInt4) {  // k 2 p to nibble p, k 2 p + 1 to nibble p + 4
#pragma unroll
    for (int p = 0; p < 4; ++p) r |= ((c >> (8 * p)) & 15u) << (4 * p) | ((c >> (8 * p + 4)) & 15u) << (4 * p + 16);
  } else {
    r = c & 0x77777777u;
#pragma unroll
    for (int p = 0; p < 4; ++p) r |= ((c >> (8 * p + 3)) & 1u) << (4 * p + 3) | ((c >> (8 * p + 7)) & 1u) << (4 * p + 19);
  }
  out[z] = r;
}

// One thread per packed scale: tile, chunk, row pair g, half, group of the chunk.
template <typename S>
__global__ void pack_scales_kernel(const S* scales, S* out, int N, int groups_k, int n_chunks, int per_row, long long count) {
  const long long z = (long long)blockIdx.x * blockDim.x + threadIdx.x;
  if (z >= count) return;
  const int i = (int)(z % per_row), half = (int)((z / per_row) & 1), g = (int)((z / (2 * per_row)) & 7);
  const long long tc = z / (16 * per_row);
  const int chunk = (int)(tc % n_chunks);
  const long long row = tc / n_chunks * kTileRows + g + 8 * half;
  const int gk = chunk * per_row + i;
  out[z] = row < N && gk < groups_k ? scales[row * groups_k + gk] : (S)0;
}

}  // namespace w4
}  // namespace moev
