// y[n, N] = x[n, K] W^T + bias for a few rows of x and 4-bit weights with group scales.
//
//   INT4:  W[o, k] = (q[o, k] - 8) * s[o, k / group]     q in 0..15, s bf16, group 32, 64 or 128
//   MXFP4: W[o, k] = e2m1(q[o, k]) * 2^(s[o, k / 32] - 127)
//
// mma.sync m16n8k16 with binary32 accumulators; products are exact, they are added over one group, multiplied by the
// binary32 scale and added to the output: no weight and no sum is rounded to fewer bits.
//   INT4 in bf16: the codes are exact, x is taken as it is.
//   MXFP4 in f16, where sign and magnitude of an e2m1 code are in place after one shift.  x is brought to f16 by a power of
//   two per row and chunk of 128 k, its largest element to [2^14, 2^15), so that an element keeps all its 8 significant bits
//   down to 2^-28 of the largest (and is off by at most 2^-40 of that below).
// 16 rows, N = 100003, K = 7168, groups of 64: 103 us in a graph, 112 us between other calls, for 387 MB (59 us): 3.5 to 3.8 TB/s, 55 %
// of the issue slots, ALU and tensor pipe 43 % each: no pipe is full; what is left is latency with 16 warps an SM, and a third round
// of tiles that is 64 % full.  1 row, N = 4096, K = 8192: 6.7 us (18 MB, 2.7 us), 8 rows, N = 5120, K = 2880 MXFP4: 7.8 us (8 MB,
// 1.2 us), of which 1 to 2 us are set-up and staging.  More rows: x staged in pieces from about 28 rows of 4096 columns on, and one pass
// over the weight per 32 rows: 5120 x 2880 MXFP4 8 / 16 / 32 / 64 / 128 rows 7.7 / 10.8 / 37 / 71 / 138 us.
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
constexpr int kTailBytes = 4096;  // behind the packed weight: the last warp's ring reads up to three chunks too far
constexpr int kDepth = 4;  // chunks a warp keeps in flight
constexpr int kRedPitch = 20;  // floats per token where the warps' sums meet: lanes (g, t) write to 32 banks

struct Args {
  const uint8_t* codes;   // packed
  const uint8_t* scales;  // packed
  const __nv_bfloat16* x;
  const float* bias;
  void* y;
  long long x_stride, y_stride;
  int n, N, K, n_chunks;   // n: rows of x in all
  int rounds;              // tiles per warp, one after another
  int kw_log2;             // warps that share a tile's K
  int phase_chunks;        // chunks of K per staged piece of x (a multiple of kw)
  int x_pitch;             // bytes per staged row
  int buf_bytes;           // bytes per staged piece of x
  int red_at;              // where the warps' sums meet: 0 = over x, when there is one round
  int n_bufs;              // 1: x is staged whole, 2: piece by piece
  int y_f32, x_vec;
};

// (w & MASK) | bits in one instruction
template <uint32_t MASK>
__device__ __forceinline__ uint32_t and_or(uint32_t w, uint32_t bits) {
  uint32_t r;
  asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(r) : "r"(w), "n"(MASK), "r"(bits));
  return r;
}

// 8 codes of a word -> 4 pairs, pair p = k 2 p and 2 p + 1.  INT4: bf16.  MXFP4: f16, 2^-14 times the value.
template <int FMT>
__device__ __forceinline__ void decode(uint32_t w, uint32_t magic, uint32_t (&r)[4]) {
  if constexpr (FMT == kInt4) {
    // nibble p = k 2 p, nibble p + 4 = k 2 p + 1.  0x4300 | q is 128 + q; minus 136 is exact.
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      const uint32_t u = and_or<0x000F000Fu>(w >> (4 * p), magic);
      const __nv_bfloat162 h = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&u), __floats2bfloat162_rn(136.f, 136.f));
      r[p] = *reinterpret_cast<const uint32_t*>(&h);
    }
  } else {
    // sign | e e m at bits 15 and 11..9 of f16 (subnormals included) is 2^-14 times the e2m1 value.  The packed halves
    // hold pair 0 there, pair 1 three bits lower, the signs of 2 and 3 at 14 and 13, their magnitudes at 5..3 and 2..0.
    r[0] = w & 0x8E008E00u;
    r[1] = (w << 3) & 0x8E008E00u;
    r[2] = and_or<0x0E000E00u>(w << 6, (w << 1) & 0x80008000u);
    r[3] = and_or<0x0E000E00u>(w << 9, (w << 2) & 0x80008000u);
  }
}

template <int FMT>
__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  if constexpr (FMT == kInt4)
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// the same with a zero accumulator
template <int FMT>
__device__ __forceinline__ void mma_first(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  if constexpr (FMT == kInt4)
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}

// GB: 32-k blocks per scale (1, 2, 4); MXFP4 has one byte per block.
template <int FMT, int GB>
struct Scales {
  static constexpr int kPerRow = 4 / GB;                                 // scales per row and chunk
  static constexpr int kBytes = 16 * kPerRow * (FMT == kInt4 ? 2 : 1);  // per tile and chunk
  static constexpr int kLane = kBytes / 8;                               // per row pair: 16, 8, 4 (INT4) or 8 (MXFP4)
  uint32_t u[kLane / 4];
  __device__ __forceinline__ void load(const uint8_t* p) {
    if constexpr (kLane == 16) { const uint4 q = *reinterpret_cast<const uint4*>(p); u[0] = q.x; u[1] = q.y; u[2] = q.z; u[3] = q.w; }
    else if constexpr (kLane == 8) { const uint2 q = *reinterpret_cast<const uint2*>(p); u[0] = q.x; u[1] = q.y; }
    else u[0] = *reinterpret_cast<const uint32_t*>(p);
  }
  // scale of row g (half 0) or g + 8 (half 1) for the i-th group of the chunk
  __device__ __forceinline__ float get(int half, int i) const {
    const int at = half * kPerRow + i;
    if constexpr (FMT == kInt4) return bf16_bits_to_float((u[at >> 1] >> (16 * (at & 1))) & 0xffffu);
    else return e8m0_to_float((u[at >> 2] >> (8 * (at & 3))) & 0xffu) * 16384.f;  // decode() leaves 2^-14
  }
};

// Stage columns [c0, c0 + cols) (cols a multiple of 128, columns from K on as zero) of rows [0, rows) of x as they are.
__device__ __forceinline__ void stage_bf16(const Args& a, const __nv_bfloat16* x, int rows, uint32_t dst, int c0, int cols) {
  const int warps = blockDim.x >> 5, lane = threadIdx.x & 31, per = (cols + 255) >> 8;  // 256 columns a warp and step
  for (int i = threadIdx.x >> 5, r = 0; r < rows; i += warps) {
    while (i >= per) { i -= per; ++r; }
    if (r >= rows) break;
    const int c = i * 256 + lane * 8;
    if (c >= cols) continue;
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

// Stage columns [c0, c0 + cols) (cols a multiple of 128, columns from K on as zero) of rows [0, rows) of x as f16, and
// per chunk and row the power of two that undoes the scaling (bf16).  16 lanes own a row's chunk, 8 columns each.
template <int NT>
__device__ __forceinline__ void stage_x(const Args& a, const __nv_bfloat16* x, int rows, uint8_t* dst, uint16_t* back, int c0, int cols) {
  const int lane = threadIdx.x & 31, half = threadIdx.x >> 4, halves = blockDim.x >> 4;
  const uint32_t lanes = 0xffffu << (lane & 16);
  const int chunks = cols >> 7;
  constexpr int kBatch = 8;  // loads in flight per thread
  int r = 0, ch = half;
  while (ch >= chunks) { ch -= chunks; ++r; }
  while (r < rows) {
    uint32_t u[kBatch][4];
    int rr[kBatch], cc[kBatch];
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      rr[k] = r;
      cc[k] = ch;
      const int c = ch * 128 + (lane & 15) * 8;
      u[k][0] = u[k][1] = u[k][2] = u[k][3] = 0;
      if (r < rows && c0 + c < a.K) {  // K is a multiple of 32: a piece of 8 lies inside or outside
        const __nv_bfloat16* from = x + (long long)r * a.x_stride + c0 + c;
        if (a.x_vec) {
          const uint4 q = *reinterpret_cast<const uint4*>(from);
          u[k][0] = q.x; u[k][1] = q.y; u[k][2] = q.z; u[k][3] = q.w;
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j)
            u[k][j] = (uint32_t)__bfloat16_as_ushort(from[2 * j]) | ((uint32_t)__bfloat16_as_ushort(from[2 * j + 1]) << 16);
        }
      }
      ch += halves;
      while (ch >= chunks) { ch -= chunks; ++r; }
    }
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      if (rr[k] >= rows) break;
      float v[8], m = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        v[2 * j] = __uint_as_float(u[k][j] << 16);
        v[2 * j + 1] = __uint_as_float(u[k][j] & 0xffff0000u);
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) m = fmaxf(m, fabsf(v[j]));
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(lanes, m, o));
      // 2^e <= m < 2^(e + 1): times 2^(14 - e), undone by 2^(e - 14).  Zero and tiny chunks as for e = -111; with an
      // infinity among them the finite values stay finite
      const int e = max((int)(__float_as_uint(m) >> 23) - 127, -111);
      float up = __uint_as_float((uint32_t)(127 + 14 - min(e, 127)) << 23);
      uint32_t down = (uint32_t)(127 + e - 14) << 7;
      if (e > 127) {
        up = 0x1p-113f;
        down = (uint32_t)(127 + 113) << 7;
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const __half2 h = __floats2half2_rn(v[2 * j] * up, v[2 * j + 1] * up);
        u[k][j] = *reinterpret_cast<const uint32_t*>(&h);
      }
      *reinterpret_cast<uint4*>(dst + rr[k] * a.x_pitch + (cc[k] * 128 + (lane & 15) * 8) * 2) = make_uint4(u[k][0], u[k][1], u[k][2], u[k][3]);
      if ((lane & 15) == 0) back[cc[k] * (8 * NT) + rr[k]] = (uint16_t)down;
    }
  }
}

// CTA: 16 warps = rw x kw; the kw warps of a tile take consecutive parts of its K.  Tiles go round all
// CTAs first, then over a CTA's rw rows of warps, so that a last incomplete round leaves every SM the same work.  The
// sums of the kw warps meet in shared memory, in warp order.  Rows of x beyond 8 NT are the business of other blockIdx.y.
//
// A warp walks over segments (one tile and one staged piece of x), each a run of consecutive chunks, in blocks of
// kDepth chunks: the block's code is unrolled, with every address an immediate offset from one register per
// operand, and behind each chunk's use the same registers are loaded with the chunk kDepth further on, across the
// ends of segments.  The last block of a run loads past its end (into another warp's part, or the padding behind the
// weight) and does not use it.
template <int FMT, int GB, int NT, bool WHOLE>
__global__ void __launch_bounds__(512, 1) linear_w4_kernel(const Args a) {
  extern __shared__ __align__(128) uint8_t smem[];
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  using Sc = Scales<FMT, GB>;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int kw_n = 1 << a.kw_log2, rw_log2 = 4 - a.kw_log2, rw_n = 1 << rw_log2;
  const int wk = warp & (kw_n - 1), wr = warp >> a.kw_log2;
  const int row0 = blockIdx.y * (8 * NT), rows = min(a.n - row0, 8 * NT);
  const __nv_bfloat16* x = a.x + (long long)row0 * a.x_stride;
  const int n_tiles = (a.N + kTileRows - 1) / kTileRows;
  const int tile0 = wr * (int)gridDim.x + (int)blockIdx.x, tile_step = rw_n * (int)gridDim.x;
  const int n_phases = WHOLE ? 1 : (a.n_chunks + a.phase_chunks - 1) / a.phase_chunks;
  const int items = a.phase_chunks >> a.kw_log2;           // chunks of a warp per segment, at most
  const int blocks = (items + kDepth - 1) / kDepth;  // the same for every warp and segment
  // a piece of x: rows, then its scales [chunk][8 NT]
  const uint32_t buf_bytes = a.buf_bytes;
  float* red = reinterpret_cast<float*>(smem + a.red_at);

  // chunks of this warp in a phase: the first one, and how many
  auto first_of = [&](int phase) { return phase * a.phase_chunks + wk * items; };
  auto count_of = [&](int phase) { return min(items, min(a.n_chunks, (phase + 1) * a.phase_chunks) - first_of(phase)); };

  // ---- weights: a ring of kDepth chunks in registers
  uint4 wreg[kDepth][2];
  Sc sreg[kDepth];
  int f_round = 0, f_phase = 0, f_block = 0;
  const uint8_t *f_w, *f_s;
  auto f_seek = [&]() {  // to the segment (f_round, f_phase); to the start of the weight where that has no chunk
    const int tile = tile0 + f_round * tile_step;
    const bool on = tile < n_tiles && count_of(f_phase) > 0;
    const size_t at = on ? (size_t)tile * a.n_chunks + first_of(f_phase) : 0;
    f_w = a.codes + at * kChunkBytes + lane * 16;
    f_s = a.scales + at * Sc::kBytes + g * Sc::kLane;
  };
  auto f_next = [&]() {  // one block on
    if (++f_block < blocks) {
      // a run that ends earlier than others' stays in its last blocks' place: nothing of it is used any more
      if (f_block * kDepth < count_of(f_phase)) {
        f_w += kDepth * kChunkBytes;
        f_s += kDepth * Sc::kBytes;
      }
    } else {
      f_block = 0;
      if (++f_phase == n_phases) {
        f_phase = 0;
        ++f_round;
      }
      f_seek();
    }
  };
  auto fetch = [&](int d) {
    const uint4* p = reinterpret_cast<const uint4*>(f_w + d * kChunkBytes);
    wreg[d][0] = __ldcs(p);
    wreg[d][1] = __ldcs(p + 32);
    sreg[d].load(f_s + d * Sc::kBytes);
  };

  asm volatile("griddepcontrol.wait;" ::: "memory");
  f_seek();
#pragma unroll
  for (int d = 0; d < kDepth; ++d) fetch(d);
  f_next();

  // ---- x: whole, or two pieces of K at a time
  int s_phase = 0, s_left = a.rounds * n_phases, s_buf = 0;
  auto stage = [&]() {  // the next piece, into the buffer that is free
    if (s_left > 0) {
      const int c0 = s_phase * a.phase_chunks;
      uint8_t* to = smem + s_buf * buf_bytes;
      if constexpr (FMT == kInt4) stage_bf16(a, x, rows, (uint32_t)__cvta_generic_to_shared(to), c0 * kChunk, min(a.phase_chunks, a.n_chunks - c0) * kChunk);
      else stage_x<NT>(a, x, rows, to, reinterpret_cast<uint16_t*>(to + (size_t)rows * a.x_pitch), c0 * kChunk, min(a.phase_chunks, a.n_chunks - c0) * kChunk);
      --s_left;
      s_phase = s_phase + 1 == n_phases ? 0 : s_phase + 1;
      s_buf ^= 1;
    }
  };
  auto landed = [&] {
    if constexpr (FMT == kInt4) asm volatile("cp.async.wait_all;" ::: "memory");
    __syncthreads();
  };
  stage();
  if (WHOLE) landed();
  // this lane's rows of x (rows that are not there read another one's: their columns of the product are not used) and
  // the scales of tokens 2 t and 2 t + 1
  uint32_t xoff[NT];
#pragma unroll
  for (int q = 0; q < NT; ++q) xoff[q] = (uint32_t)min(q * 8 + g, rows - 1) * a.x_pitch + t * 16;
  const uint32_t boff = (uint32_t)rows * a.x_pitch + t * 4;
  uint32_t magic = 0x43004300u;
  asm volatile("" : "+r"(magic));  // in a register, so that mask and or are one instruction

  int buf = 1;
  for (int round = 0; round < a.rounds; ++round) {
    const int tile = tile0 + round * tile_step;
    float acc[NT][4] = {};
    for (int phase = 0; phase < n_phases; ++phase) {
      if (!WHOLE) {
        landed();  // the piece is there, and everybody has left the other buffer
        stage();
        buf ^= 1;
      }
      int left = tile < n_tiles ? count_of(phase) : 0;
      const uint8_t* piece = smem + (WHOLE ? 0u : buf * buf_bytes);
      const uint8_t *xp[NT], *bp = piece + boff + wk * items * (16 * NT);
#pragma unroll
      for (int q = 0; q < NT; ++q) xp[q] = piece + xoff[q] + wk * items * (kChunk * 2);
      for (int block = 0; block < blocks; ++block) {
#pragma unroll
        for (int d = 0; d < kDepth; ++d) {
          if (d < left) {
            const uint32_t word[8] = {wreg[d][0].x, wreg[d][0].y, wreg[d][0].z, wreg[d][0].w,
                                      wreg[d][1].x, wreg[d][1].y, wreg[d][1].z, wreg[d][1].w};
            float part[NT][4];  // MXFP4: the chunk's sums, in units of its tokens' powers of two
#pragma unroll
            for (int gr = 0; gr < 4 / GB; ++gr) {
              float sum[NT][4];
#pragma unroll
              for (int bb = 0; bb < GB; ++bb) {
                const int b = gr * GB + bb;  // 32-k block of the chunk
                uint32_t lo[4], hi[4];
                decode<FMT>(word[2 * b], magic, lo);
                decode<FMT>(word[2 * b + 1], magic, hi);
#pragma unroll
                for (int q = 0; q < NT; ++q) {
                  const uint4 xb = *reinterpret_cast<const uint4*>(xp[q] + d * (kChunk * 2) + b * 64);
                  if (bb == 0) mma_first<FMT>(sum[q], lo[0], hi[0], lo[1], hi[1], xb.x, xb.y);
                  else mma<FMT>(sum[q], lo[0], hi[0], lo[1], hi[1], xb.x, xb.y);
                  mma<FMT>(sum[q], lo[2], hi[2], lo[3], hi[3], xb.z, xb.w);
                }
              }
              const float s0 = sreg[d].get(0, gr), s1 = sreg[d].get(1, gr);
#pragma unroll
              for (int q = 0; q < NT; ++q)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                  if constexpr (FMT == kInt4) acc[q][e] = fmaf(e < 2 ? s0 : s1, sum[q][e], acc[q][e]);
                  else part[q][e] = gr == 0 ? (e < 2 ? s0 : s1) * sum[q][e] : fmaf(e < 2 ? s0 : s1, sum[q][e], part[q][e]);
            }
#pragma unroll
            for (int q = 0; FMT == kMx && q < NT; ++q) {
              const uint32_t b = *reinterpret_cast<const uint32_t*>(bp + d * (16 * NT) + q * 16);
              const float f0 = __uint_as_float(b << 16), f1 = __uint_as_float(b & 0xffff0000u);
              acc[q][0] = fmaf(f0, part[q][0], acc[q][0]);
              acc[q][1] = fmaf(f1, part[q][1], acc[q][1]);
              acc[q][2] = fmaf(f0, part[q][2], acc[q][2]);
              acc[q][3] = fmaf(f1, part[q][3], acc[q][3]);
            }
          }
          if (d & 1) {
            fetch(d - 1);
            fetch(d);
          }
        }
        f_next();
        left -= kDepth;
        bp += kDepth * 16 * NT;
#pragma unroll
        for (int q = 0; q < NT; ++q) xp[q] += kDepth * kChunk * 2;
      }
    }
    // lane (g, t) holds outputs g and g + 8 of the tile for tokens 2 t and 2 t + 1
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
      // [warp][token][output]
      if (a.red_at == 0) __syncthreads();  // everybody is done with x
      float* mine = red + warp * (NT * 8 * kRedPitch);
#pragma unroll
      for (int q = 0; q < NT; ++q)
#pragma unroll
        for (int e = 0; e < 4; ++e) mine[(q * 8 + 2 * t + (e & 1)) * kRedPitch + g + 8 * (e >> 1)] = acc[q][e];
      __syncthreads();
      for (int z = threadIdx.x; z < rw_n * kTileRows * rows; z += blockDim.x) {
        const int lo = z & 15, rr = z >> 4, w = rr & (rw_n - 1), r = rr >> rw_log2;
        const int o = ((round * rw_n + w) * (int)gridDim.x + (int)blockIdx.x) * kTileRows + lo;
        if (o < a.N) {
          const float* p = red + w * kw_n * (NT * 8 * kRedPitch) + r * kRedPitch + lo;
          float v = 0.f;
          for (int k = 0; k < kw_n; ++k) v += p[k * (NT * 8 * kRedPitch)];
          v += a.bias ? a.bias[o] : 0.f;
          const long long at = (long long)(row0 + r) * a.y_stride + o;
          if (a.y_f32) static_cast<float*>(a.y)[at] = v;
          else static_cast<__nv_bfloat16*>(a.y)[at] = __float2bfloat16_rn(v);
        }
      }
      if (round + 1 < a.rounds) __syncthreads();
    }
  }
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
#pragma unroll
    for (int h = 0; h < 2; ++h) {  // half h: the odd or even k of each pair
      uint32_t q[4];
#pragma unroll
      for (int p = 0; p < 4; ++p) q[p] = (c >> (8 * p + 4 * h)) & 15u;
      const uint32_t v = (q[0] >> 3) << 15 | (q[0] & 7u) << 9 | (q[1] >> 3) << 12 | (q[1] & 7u) << 6 | (q[2] >> 3) << 14 |
                         (q[3] >> 3) << 13 | (q[2] & 7u) << 3 | (q[3] & 7u);
      r |= v << (16 * h);
    }
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
