// Attention of draft tokens over the paged 8-bit cache (kv_cache.cuh).
//
//   score[r, j] = scale * q_r . k_j over the context's keys (the last `window` positions of them) and
//   the draft's own ancestors and itself;  out_r = sum_j p[r, j] v_j,  p = softmax (with an optional
//   sink logit per head in the denominator),  lse_r = log of the denominator + maximum.
//
// Rows of a tile are (draft, query head of one kv head): the heads that share keys share their loads.
// mma.sync m16n8k16 with f16 operands and binary32 accumulators: an e4m3 code is exact in f16, q (bf16)
// is brought to at most 2^14 by a power of two per row, where f16 holds all 8 of its significant bits
// down to 2^-28 of the row's largest element, and the probabilities are rounded once to f16 (2^-11).
// Codes go to the multiplier as they are: the scale of a page's K multiplies the scores, that of its
// V the probabilities.  p * v_scale / u * 2^14, with u the largest V scale seen so far, uses f16's
// range from 2^14 down, so a page whose scale is 2^-20 of the largest still keeps 8 bits or more.
//
// Which key an MMA calls its n-th, and which dimension its k-th, is free as long as both operands agree.
// Lane (g, t) = (lane / 4, lane % 4).  Scores: lane t's 16-byte piece t + 4 i of a key's row holds the
// dimensions of four MMA steps; column n of key tile j is key 16 (n / 2) + 2 j + n % 2, so that lane t
// ends up with the scores of the 16 consecutive keys 16 t .. 16 t + 15 of the 64: one page, one scale.  Second
// product: lane t's 16 bytes of a V row are those 16 keys, four MMA steps of four, and its scores are
// already in the A layout.  Both operands come out of shared memory by full 16-byte loads, no transposition.
//
// Work split: grid = (chunks of the key range, kv head x row tiles, sequence); the WK key groups of a
// CTA take every WK-th tile of 64 keys of the chunk, its WR warps 16 rows each.  Key groups meet in shared
// memory, chunks in a second kernel (attend_combine), both in fixed order.
#pragma once
#include "kv_cache.cuh"

namespace moev {
namespace att {

using kv::Cache;
using kv::Drafts;
using kv::Seq;

constexpr int kTile = 64;

struct Args {
  Drafts d;
  Cache c;
  const __nv_bfloat16* q;
  __nv_bfloat16* out;
  float* lse;          // [n_tokens, n_heads] or null
  const float* sinks;  // [n_heads] or null
  float* part_o;       // [chunks, n_tokens, n_heads, D]
  float2* part_ml;     // [chunks, n_tokens, n_heads]: maximum (base 2), denominator
  long long q_stride, out_stride;
  int n_heads, rep, row_tiles, chunks, chunk_keys, window;
  float scale_log2;
};

__device__ __forceinline__ void mma_f16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// four e4m3 codes -> two f16 pairs
__device__ __forceinline__ void codes_to_f16(uint32_t w, uint32_t& lo, uint32_t& hi) {
  asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}"
      : "=r"(lo), "=r"(hi)
      : "r"(w));
}
__device__ __forceinline__ float exp2_fast(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ uint32_t pack_f16(float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint4 lds128(uint32_t at) {
  uint4 r;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "r"(at));
  return r;
}
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool on) {
  const int n = on ? 16 : 0;  // 0: zeros
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
__device__ __forceinline__ void cp_async4(uint32_t dst, const void* src, bool on) {
  const int n = on ? 4 : 0;
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}

// First key of the range that a sequence's drafts can see (a multiple of 64).
__device__ __forceinline__ int range_start(const Seq& s, int window) {
  return window > 0 ? max(0, s.ctx + 1 - window) & ~(kTile - 1) : 0;
}

template <int D, int WR, int WK, int ST>
struct Cfg {
  static constexpr int kThreads = 32 * WR * WK;
  static constexpr int kStage = 2 * kTile * D + 64;  // K [64][D], V [D][64], 4 + 4 scales, 4 flags: page in the pool
  static constexpr int kRing = WK * ST * kStage;
  static constexpr int kMerge = WK > 1 ? WR * WK * (16 * (D + 4) + 32) * 4 : 0;  // after the loop, over the ring
  static constexpr int kMain = kRing > kMerge ? kRing : kMerge;
  static size_t smem(int words, int tree) {  // + ancestor words, depths and parents of the tile's drafts
    return kMain + (tree ? (size_t)(16 * WR) * (words + 1) * 4 + (size_t)words * 32 * 4 : 0);
  }
};

template <int D, int WR, int WK, int ST>
__global__ void __launch_bounds__(32 * WR * WK, 1) attend_kernel(const Args a) {
  using C = Cfg<D, WR, WK, ST>;
  extern __shared__ __align__(128) uint8_t smem[];
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int page_log2 = a.c.page_log2, page = 1 << page_log2;
  const int b = blockIdx.z, head = blockIdx.y / a.row_tiles, row0 = (blockIdx.y % a.row_tiles) * 16 * WR;
  const Seq s = kv::sequence(a.d, b, page);
  const int R = s.n * a.rep;
  if (row0 >= R) return;
  const int start = range_start(s, a.window);
  const int k_begin = start + blockIdx.x * a.chunk_keys;
  const int k_all = s.ctx + s.n;
  if (k_begin >= k_all) return;
  const bool tree = a.d.parent != nullptr;
  const int i_first = row0 / a.rep, i_last = min(R - 1, row0 + 16 * WR - 1) / a.rep;
  int k_end = min(k_begin + a.chunk_keys, k_all);
  if (!tree) k_end = min(k_end, s.ctx + i_last + 1);  // a chain: nobody here sees later drafts

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
  const int wr = warp % WR, wk = warp / WR;
  const uint32_t ring = (uint32_t)__cvta_generic_to_shared(smem) + wk * (ST * C::kStage);
  const int n_tiles = k_end > k_begin ? (k_end - k_begin + kTile - 1) / kTile : 0;
  const int iters = (n_tiles + WK - 1) / WK;

  // ---- loads: the warps of a key group bring in its tiles
  auto load_tile = [&](int it) {
    const int k0 = k_begin + (it * WK + wk) * kTile;
    const uint32_t dst = ring + (it % ST) * C::kStage;
    if (it < iters && k0 < k_end) {
      // lane's quarter: page of keys 16 (lane & 3) .. of the tile, -1 behind the end
      const int kq = k0 + 16 * t;
      int pid = kq < k_all ? kv::page_of(a.d, a.c, b, kq >> page_log2) : -1;
      const int lt = wr * 32 + lane;
#pragma unroll
      for (int z = 0; z < 4 * D / (32 * WR); ++z) {
        const int p = z * 32 * WR + lt, key = p / (D / 16), c = p % (D / 16);
        const int pg = __shfl_sync(0xffffffffu, pid, key >> 4);
        const uint8_t* src = a.c.k + (((long long)max(pg, 0) * a.c.heads + head) << page_log2) * D + ((k0 + key) & (page - 1)) * D + c * 16;
        const int cs = D == 128 ? c ^ (4 * (key & 1)) : c;  // odd keys swap halves: 8 lanes cover all banks
        cp_async16(dst + key * D + cs * 16, src, pg >= 0);
      }
#pragma unroll
      for (int z = 0; z < 4 * D / (32 * WR); ++z) {
        const int p = z * 32 * WR + lt;
        int dd, quarter;
        if (page_log2 == 4) { dd = p % D; quarter = p / D; }
        else if (page_log2 == 5) { dd = (p >> 1) % D; quarter = (p & 1) + 2 * ((p >> 1) / D); }
        else { dd = p >> 2; quarter = p & 3; }
        const int pg = __shfl_sync(0xffffffffu, pid, quarter);
        const uint8_t* src = a.c.v + (((long long)max(pg, 0) * a.c.heads + head) << page_log2) * D + dd * page + ((k0 + 16 * quarter) & (page - 1));
        cp_async16(dst + kTile * D + dd * kTile + quarter * 16, src, pg >= 0);
      }
      if (wr == 0 && lane < 8) {
        const long long slot = (long long)max(pid, 0) * a.c.heads + head;
        cp_async4(dst + 2 * kTile * D + lane * 4, (lane < 4 ? a.c.ks : a.c.vs) + slot, pid >= 0);
      }
      if (wr == 0 && lane >= 8 && lane < 12)
        asm volatile("st.shared.b32 [%0], %1;" ::"r"(dst + 2 * kTile * D + lane * 4), "r"(pid) : "memory");
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
#pragma unroll
  for (int it = 0; it < ST - 1; ++it) load_tile(it);

  // ---- ancestors of the tile's drafts, as bits over the sequence's drafts, and their depths
  const int words = tree ? (a.d.max_drafts + 31) >> 5 : 0;
  uint32_t* anc = reinterpret_cast<uint32_t*>(smem + C::kMain);  // [16 WR][words]
  int* depth = reinterpret_cast<int*>(anc + 16 * WR * words);   // [16 WR]
  int* par = depth + 16 * WR;                                   // [max_drafts]
  if (tree) {
    for (int i = tid; i < s.n; i += C::kThreads) par[i] = kv::parent_of(a.d.parent + s.lo, i);
    for (int i = tid; i < 16 * WR * words; i += C::kThreads) anc[i] = 0;
    __syncthreads();
    for (int l = tid; l <= i_last - i_first; l += C::kThreads) {
      int n = 0;
      for (int j = i_first + l; j >= 0; j = par[j], ++n)  // parents come earlier: at most s.n steps
        if (a.window <= 0 || n < a.window) anc[l * words + (j >> 5)] |= 1u << (j & 31);
      depth[l] = n - 1;
    }
    __syncthreads();
  }

  // ---- this lane's rows: g and g + 8 of the warp's 16
  uint32_t qf[D / 16][4];
  float rc[2];              // row's factor from raw scores to powers of two
  int low[2], top[2], loc[2];  // context keys > low are seen; a chain sees keys <= top
  bool live[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int r = row0 + wr * 16 + g + 8 * h;
    live[h] = r < R;
    const int rr = live[h] ? r : R - 1, i = rr / a.rep, hq = head * a.rep + rr % a.rep;
    const __nv_bfloat16* src = a.q + (long long)(s.lo + i) * a.q_stride + (long long)hq * D;
    float v[D / 64][16];
    float m = 0.f;
#pragma unroll
    for (int c = 0; c < D / 64; ++c) {
      float x[8], y[8];
      kv::load8(src + (t + 4 * c) * 16, x);
      kv::load8(src + (t + 4 * c) * 16 + 8, y);
#pragma unroll
      for (int e = 0; e < 8; ++e) { v[c][e] = x[e]; v[c][8 + e] = y[e]; m = fmaxf(m, fmaxf(fabsf(x[e]), fabsf(y[e]))); }
    }
    m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 1));
    m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 2));
    // 2^e in [m, 2 m), brought to 2^14; a zero, infinite or NaN row as it is
    const uint32_t e = __float_as_uint(m) >> 23;
    float up = 1.f, back = 1.f;
    if (e >= 30u && e < 255u) {
      const int x = 13 - ((int)e - 127);  // largest element to [2^13, 2^14)
      up = ldexpf(1.f, x);
      back = ldexpf(1.f, -x);
    }
    rc[h] = a.scale_log2 * back;
#pragma unroll
    for (int c = 0; c < D / 64; ++c)
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        qf[4 * c + w][h] = pack_f16(v[c][4 * w] * up, v[c][4 * w + 1] * up);
        qf[4 * c + w][2 + h] = pack_f16(v[c][4 * w + 2] * up, v[c][4 * w + 3] * up);
      }
    loc[h] = i - i_first;
    const int at = s.ctx + (tree ? depth[loc[h]] : i);
    low[h] = a.window > 0 ? at - a.window : -1;
    top[h] = tree ? s.ctx - 1 : at;  // last key of the contiguous part
  }
  const int low_max = a.window > 0 ? s.ctx + s.n - 1 - a.window : -1;  // no row hides a key above this

  float o[D / 8][4] = {};
  float mx[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
  float u = 1.17549435e-38f;

  for (int it = 0; it < iters; ++it) {
    asm volatile("cp.async.wait_group %0;" ::"n"(ST - 2) : "memory");
    if constexpr (WR == 1) __syncwarp();
    else asm volatile("bar.sync %0, %1;" ::"r"(1 + wk), "r"(32 * WR) : "memory");
    load_tile(it + ST - 1);
    const int k0 = k_begin + (it * WK + wk) * kTile;
    if (k0 >= k_end) continue;
    const uint32_t ks = ring + (it % ST) * C::kStage, vs = ks + kTile * D;
    float sc[8][4] = {};
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t row = ks + (16 * (g >> 1) + 2 * j + (g & 1)) * D;
#pragma unroll
      for (int c = 0; c < D / 64; ++c) {
        const uint4 w = lds128(row + (((t + 4 * c) ^ (D == 128 ? 4 * (g & 1) : 0)) * 16));
        const uint32_t ww[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          uint32_t b0, b1;
          codes_to_f16(ww[e], b0, b1);
          mma_f16(sc[j], qf[4 * c + e], b0, b1);
        }
      }
    }
    float k_scale, v_scale;
    asm volatile("ld.shared.f32 %0, [%1];" : "=f"(k_scale) : "r"(vs + kTile * D + 4 * t));
    asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v_scale) : "r"(vs + kTile * D + 16 + 4 * t));
    // lane t's keys: k0 + 16 t + 2 j + e
    const int kq = k0 + 16 * t;
    const bool masked = k0 + kTile > s.ctx || k0 <= low_max;
    uint32_t see[2] = {0xffffu, 0xffffu};
    int pid;  // -1: behind the end, or a page id outside the pool; its keys are not seen
    asm volatile("ld.shared.b32 %0, [%1];" : "=r"(pid) : "r"(vs + kTile * D + 32 + 4 * t));
    if (pid < 0) see[0] = see[1] = 0;
    if (masked) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        // keys low + 1 .. top
        const int from = max(0, low[h] + 1 - kq), to = min(16, top[h] + 1 - kq);
        uint32_t bits = to > from ? (0xffffu >> (16 - to)) & (0xffffu << from) : 0u;
        if (tree && kq + 16 > s.ctx && kq < k_all) {
          const int off = kq - s.ctx;  // draft index of the lane's first key, may be negative
          uint64_t w;
          const uint32_t* an = anc + loc[h] * words;
          if (off < 0) w = (uint64_t)an[0] << (-off);
          else {
            const int wi = off >> 5;
            w = ((uint64_t)an[wi] | (wi + 1 < words ? (uint64_t)an[wi + 1] << 32 : 0ull)) >> (off & 31);
          }
          bits |= (uint32_t)w & 0xffffu;
        }
        see[h] &= bits;
      }
    }
    float mt[2] = {-INFINITY, -INFINITY};
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int h = e >> 1;
        float v = sc[j][e] * k_scale;
        v = (see[h] >> (2 * j + (e & 1))) & 1u ? v : -INFINITY;
        sc[j][e] = v;
        mt[h] = fmaxf(mt[h], v);
      }
    float vm = v_scale;
    vm = fmaxf(vm, __shfl_xor_sync(0xffffffffu, vm, 1));
    vm = fmaxf(vm, __shfl_xor_sync(0xffffffffu, vm, 2));
    const float u_new = fmaxf(u, vm), ur = u / u_new;
    float alpha[2], mr[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      mt[h] = fmaxf(mt[h], __shfl_xor_sync(0xffffffffu, mt[h], 1));
      mt[h] = fmaxf(mt[h], __shfl_xor_sync(0xffffffffu, mt[h], 2));
      const float m_new = fmaxf(mx[h], mt[h]);
      const float m_ref = m_new == -INFINITY ? 0.f : m_new;
      alpha[h] = exp2_fast((mx[h] - m_ref) * rc[h]);
      mr[h] = m_ref * rc[h];
      mx[h] = m_new;
      l[h] *= alpha[h];
      alpha[h] *= ur;
    }
    u = u_new;
    const float f = v_scale / u * 16384.f;
    uint32_t pf[4][4];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float p[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        p[e] = exp2_fast(fmaf(sc[j][e], rc[e >> 1], -mr[e >> 1]));
        l[e >> 1] += p[e];
        p[e] *= f;
      }
      pf[j >> 1][2 * (j & 1)] = pack_f16(p[0], p[1]);
      pf[j >> 1][2 * (j & 1) + 1] = pack_f16(p[2], p[3]);
    }
    if (__any_sync(0xffffffffu, alpha[0] != 1.f || alpha[1] != 1.f)) {
#pragma unroll
      for (int d = 0; d < D / 8; ++d) {
        o[d][0] *= alpha[0];
        o[d][1] *= alpha[0];
        o[d][2] *= alpha[1];
        o[d][3] *= alpha[1];
      }
    }
    uint32_t nan_codes = 0;
#pragma unroll
    for (int d = 0; d < D / 8; ++d) {
      const uint4 w = lds128(vs + (8 * d + g) * kTile + t * 16);
      uint32_t ww[4] = {w.x, w.y, w.z, w.w};
      if (masked) {  // a NaN code must not reach rows that do not see its key: 0 * NaN
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t bad = __vcmpeq4(ww[e] & 0x7f7f7f7fu, 0x7f7f7f7fu);
          nan_codes |= bad;
          ww[e] &= ~bad;
        }
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        uint32_t b0, b1;
        codes_to_f16(ww[e], b0, b1);
        mma_f16(o[d], pf[e], b0, b1);
      }
    }
    if (masked && __any_sync(0xffffffffu, nan_codes != 0)) {
      // rows that do see one: their output is NaN in that dimension (ones in the place of the NaN codes)
#pragma unroll 1
      for (int d = 0; d < D / 8; ++d) {
        const uint4 w = lds128(vs + (8 * d + g) * kTile + t * 16);
        const uint32_t ww[4] = {w.x, w.y, w.z, w.w};
        float hit[4] = {};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          uint32_t b0, b1;
          codes_to_f16(__vcmpeq4(ww[e] & 0x7f7f7f7fu, 0x7f7f7f7fu) & 0x38383838u, b0, b1);
          mma_f16(hit, pf[e], b0, b1);
        }
#pragma unroll
        for (int dd = 0; dd < D / 8; ++dd)
          if (dd == d)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (hit[e] > 0.f) o[dd][e] = __int_as_float(0x7fffffff);
      }
    }
  }
  asm volatile("cp.async.wait_group 0;" ::: "memory");
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    l[h] += __shfl_xor_sync(0xffffffffu, l[h], 1);
    l[h] += __shfl_xor_sync(0xffffffffu, l[h], 2);
    mx[h] *= rc[h];  // to powers of two
  }
  const float back = u * (1.f / 16384.f);
#pragma unroll
  for (int d = 0; d < D / 8; ++d)
#pragma unroll
    for (int e = 0; e < 4; ++e) o[d][e] *= back;

  // one row's result: unnormalised o[c], c = 8 d + 2 t + e
  const bool split = a.chunks > 1;
  auto write2 = [&](int r, int c, float x, float y, float m, float den) {
    const int i = r / a.rep, hq = head * a.rep + r % a.rep;
    const long long token = s.lo + i;
    if (split) {
      const long long at = ((long long)blockIdx.x * a.d.n_tokens + token) * a.n_heads + hq;
      *reinterpret_cast<float2*>(a.part_o + at * D + c) = make_float2(x, y);
      if (c == 0) a.part_ml[at] = make_float2(m, den);
    } else {
      if (a.sinks) {
        const float sk = a.sinks[hq] * 1.4426950408889634f, mm = fmaxf(m, sk);
        const float w = exp2_fast(m - mm);
        den = den * w + exp2_fast(sk - mm);
        x *= w;
        y *= w;
        m = mm;
      }
      const float inv = den > 0.f ? 1.f / den : (den == 0.f ? 0.f : den);
      const __nv_bfloat162 v = __floats2bfloat162_rn(x * inv, y * inv);
      *reinterpret_cast<__nv_bfloat162*>(a.out + token * a.out_stride + (long long)hq * D + c) = v;
      if (c == 0 && a.lse) a.lse[token * a.n_heads + hq] = den == 0.f ? -INFINITY : (m + log2f(den)) * 0.6931471805599453f;
    }
  };
  if constexpr (WK == 1) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
      if (live[h]) {
#pragma unroll
        for (int d = 0; d < D / 8; ++d)
          write2(row0 + wr * 16 + g + 8 * h, 8 * d + 2 * t, o[d][2 * h], o[d][2 * h + 1], mx[h], l[h]);
      }
  } else {
    constexpr int P = D + 4;
    float* om = reinterpret_cast<float*>(smem);       // [WK][16 WR][P]
    float* ml = om + WK * 16 * WR * P;                // [WK][16 WR][2]
    __syncthreads();  // all tiles are used up
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int r = wk * 16 * WR + wr * 16 + g + 8 * h;
#pragma unroll
      for (int d = 0; d < D / 8; ++d) *reinterpret_cast<float2*>(om + r * P + 8 * d + 2 * t) = make_float2(o[d][2 * h], o[d][2 * h + 1]);
      if (t == 0) { ml[2 * r] = mx[h]; ml[2 * r + 1] = l[h]; }
    }
    __syncthreads();
    for (int z = tid; z < 16 * WR * (D / 2); z += C::kThreads) {
      const int r = z / (D / 2), c = (z % (D / 2)) * 2;
      if (row0 + r >= R) continue;
      float m = -INFINITY;
#pragma unroll
      for (int k = 0; k < WK; ++k) m = fmaxf(m, ml[2 * (k * 16 * WR + r)]);
      const float mr = m == -INFINITY ? 0.f : m;
      float den = 0.f, x = 0.f, y = 0.f;
#pragma unroll
      for (int k = 0; k < WK; ++k) {
        const int q = k * 16 * WR + r;
        const float w = exp2_fast(ml[2 * q] - mr);
        const float2 v = *reinterpret_cast<const float2*>(om + q * P + c);
        den = fmaf(w, ml[2 * q + 1], den);
        x = fmaf(w, v.x, x);
        y = fmaf(w, v.y, y);
      }
      write2(row0 + r, c, x, y, m, den);
    }
  }
}

// One warp per (token, head): the chunks' parts, in order, and the sink.
template <int D>
__global__ void __launch_bounds__(128) attend_combine_kernel(const Args a) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int lane = threadIdx.x & 31, b = blockIdx.z, hq = blockIdx.y * 4 + (threadIdx.x >> 5);
  if (hq >= a.n_heads) return;
  const Seq s = kv::sequence(a.d, b, 1 << a.c.page_log2);
  const int i = blockIdx.x;
  if (i >= s.n) return;
  const int span = s.ctx + s.n - range_start(s, a.window);
  const int chunks = (span + a.chunk_keys - 1) / a.chunk_keys;
  const long long token = s.lo + i, step = (long long)a.d.n_tokens * a.n_heads;
  const long long at = token * a.n_heads + hq;
  float m = -INFINITY;
  for (int c = lane; c < chunks; c += 32) m = fmaxf(m, a.part_ml[at + c * step].x);
#pragma unroll
  for (int x = 16; x > 0; x >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, x));
  if (a.sinks) m = fmaxf(m, a.sinks[hq] * 1.4426950408889634f);
  const float mr = m == -INFINITY ? 0.f : m;
  constexpr int V = D / 32;
  float o[V] = {}, den = 0.f;
  for (int c = 0; c < chunks; ++c) {
    const float2 ml = a.part_ml[at + c * step];
    if (ml.y == 0.f) continue;  // nothing seen in this chunk
    const float w = exp2_fast(ml.x - mr);
    den = fmaf(w, ml.y, den);
    const float* p = a.part_o + (at + c * step) * D + lane * V;
    if constexpr (V == 4) {
      const float4 v = *reinterpret_cast<const float4*>(p);
      o[0] = fmaf(w, v.x, o[0]); o[1] = fmaf(w, v.y, o[1]); o[2] = fmaf(w, v.z, o[2]); o[3] = fmaf(w, v.w, o[3]);
    } else {
      const float2 v = *reinterpret_cast<const float2*>(p);
      o[0] = fmaf(w, v.x, o[0]); o[1] = fmaf(w, v.y, o[1]);
    }
  }
  if (a.sinks) den += exp2_fast(a.sinks[hq] * 1.4426950408889634f - mr);
  const float inv = den > 0.f ? 1.f / den : (den == 0.f ? 0.f : den);
  __nv_bfloat16* out = a.out + token * a.out_stride + (long long)hq * D + lane * V;
#pragma unroll
  for (int e = 0; e < V; e += 2) *reinterpret_cast<__nv_bfloat162*>(out + e) = __floats2bfloat162_rn(o[e] * inv, o[e + 1] * inv);
  if (a.lse && lane == 0) a.lse[at] = den == 0.f ? -INFINITY : (m + log2f(den)) * 0.6931471805599453f;
}

}  // namespace att
}  // namespace moev
