// Paged 8-bit key / value cache: the description of a call's drafts, and the kernel that writes them.
//
// A page holds `page` tokens; for every page and kv head the codes of K are [page, D] (a token's row
// contiguous) and those of V are [D, page] (a dimension's tokens contiguous: the order in which the
// second product of attention reads them), e4m3, and K and V have one binary32 scale each, a power of
// two: value = code * scale.  A power of two lets the scale of a page grow when later tokens need
// more range: the tokens that are there are multiplied by 2^-j, which is exact in e4m3 except where
// a code falls below its normal range (then it is rounded once more, by at most half of the smallest
// step of the new scale).
#pragma once
#include "common.cuh"

namespace moev {
namespace kv {

constexpr int kMaxTree = 1024;  // drafts of one sequence when they come with parents

struct Drafts {
  int n_seq, n_tokens, max_drafts, max_len, table_cols;
  const int32_t *cu, *ctx, *table, *parent;
  int32_t* status;
};

struct Cache {
  int n_pages, page_log2, heads;  // page = 1 << page_log2
  uint8_t *k, *v;
  float *ks, *vs;
};

// The largest code of all that is reported stays: a time-out (4) is not hidden by a sequence or page that was left out.
__device__ __forceinline__ void report(int32_t* status, int code) {
  if (status) atomicMax(status, code);
}

struct Seq {
  int lo, n, ctx;  // first token row, drafts, tokens in the cache before them
};

// Sequence b of the call; n = 0 where it has no drafts or where its numbers contradict the call's bounds (reported
// in the status word: nothing outside the caller's buffers is touched whatever the arrays hold).
__device__ __forceinline__ Seq sequence(const Drafts& d, int b, int page) {
  Seq s;
  s.lo = d.cu[b];
  s.n = d.cu[b + 1] - s.lo;
  s.ctx = d.ctx[b];
  const bool ok = s.lo >= 0 && s.n >= 0 && s.n <= d.max_drafts && s.lo <= d.n_tokens - s.n && s.ctx >= 0 &&
                  s.ctx <= d.max_len - s.n && (long long)s.ctx + s.n <= (long long)d.table_cols * page;
  if (!ok) {
    report(d.status, 1);
    s.n = 0;
  }
  return s;
}
__device__ __forceinline__ int page_of(const Drafts& d, const Cache& c, int b, int col) {
  const int p = d.table[(long long)b * d.table_cols + col];
  if (p >= 0 && p < c.n_pages) return p;
  report(d.status, 2);
  return -1;
}
// Parent of draft i, -1 for one that hangs on the context; anything but an earlier draft of the sequence counts as that.
__device__ __forceinline__ int parent_of(const int32_t* parent, int i) {
  const int p = parent[i];
  return p >= 0 && p < i ? p : -1;
}

struct AppendArgs {
  Drafts d;
  Cache c;
  const __nv_bfloat16 *k, *v, *q;
  __nv_bfloat16* q_out;
  long long k_stride, v_stride, q_stride, q_out_stride;
  const float* rope;  // [rope_rows, D]: D / 2 cosines, then D / 2 sines
  int rope_rows, rep, q_parts;  // rep: query heads per kv head, 0 = no q; q_parts: CTAs that share a page's queries
};

__device__ __forceinline__ void load8(const __nv_bfloat16* p, float (&v)[8]) {
  const uint4 q = *reinterpret_cast<const uint4*>(p);
  const uint32_t u[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(u[i] << 16);
    v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, const float (&v)[8]) {
  uint32_t u[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
    u[i] = *reinterpret_cast<const uint32_t*>(&b);
  }
  *reinterpret_cast<uint4*>(p) = make_uint4(u[0], u[1], u[2], u[3]);
}
// columns [c, c + 8) and their partners [c + D / 2, ...) of a row, rotated by the row's angles
template <int D>
__device__ __forceinline__ void load_rotated(const __nv_bfloat16* row, const float* cs, int c, float (&a)[8], float (&b)[8]) {
  load8(row + c, a);
  load8(row + c + D / 2, b);
  if (cs) {
    float co[8], si[8];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const float4 x = *reinterpret_cast<const float4*>(cs + c + 4 * h);
      const float4 y = *reinterpret_cast<const float4*>(cs + D / 2 + c + 4 * h);
      co[4 * h] = x.x; co[4 * h + 1] = x.y; co[4 * h + 2] = x.z; co[4 * h + 3] = x.w;
      si[4 * h] = y.x; si[4 * h + 1] = y.y; si[4 * h + 2] = y.z; si[4 * h + 3] = y.w;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float u = a[i], w = b[i];
      a[i] = u * co[i] - w * si[i];
      b[i] = w * co[i] + u * si[i];
    }
  }
}

// Smallest power of two s with 448 s >= amax, inside the normal range and such that 448 s is finite.
__device__ __forceinline__ float cache_scale(float amax) {
  if (!(amax > 0.f)) return 0.f;
  const float s = act_scale(amax, 2);
  return fminf(fmaxf(s, 1.17549435e-38f), 6.64613998e35f);  // 2^-126 .. 2^119
}
__device__ __forceinline__ uint32_t cache_code(float v, float inv) {
  return (uint32_t)__nv_cvt_float_to_fp8(v * inv, __NV_SATFINITE, __NV_E4M3);
}
// four codes times a power of two
__device__ __forceinline__ uint32_t rescale4(uint32_t w, float f) {
  uint32_t r = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __half_raw h = __nv_cvt_fp8_to_halfraw((__nv_fp8_storage_t)(w >> (8 * i)), __NV_E4M3);
    r |= (uint32_t)__nv_cvt_float_to_fp8(__half2float(*reinterpret_cast<const __half*>(&h)) * f, __NV_SATFINITE, __NV_E4M3) << (8 * i);
  }
  return r;
}

// One CTA per (page that a sequence's drafts touch, kv head, sequence).  The page's new rows are read
// twice, once for the largest magnitude and once to be written, the second time from the caches; the
// codes pass through shared memory, where those of V are turned from token rows into dimension rows.
// Two further CTAs of the page and head rotate the query heads of the group for the page's tokens, two thirds of the
// bytes at 8 query heads a kv head (in the K and V CTA itself: 64 drafts 5.1 us instead of 4.3, 5 500 tokens 44.6 instead
// of 40.1; registers for two rows in flight cost a third of the warps and 10 us of the latter).
// Bound by memory: 2 (Hq + 2 Hkv) D bytes in, 2 Hq D + 2 Hkv D out per token.
template <int D>
__global__ void __launch_bounds__(256) cache_append_kernel(const AppendArgs a) {
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ float red[2][8];
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int page = 1 << a.c.page_log2;
  // roles: K and V of a page and head (part 0), or a share of the queries of its group (parts 1 ..)
  const int b = blockIdx.z, part = blockIdx.y / a.c.heads, head = blockIdx.y - part * a.c.heads, tid = threadIdx.x;
  const Seq s = sequence(a.d, b, page);
  const int col = (s.ctx >> a.c.page_log2) + blockIdx.x;
  const int first = max(s.ctx, col << a.c.page_log2), last = min(s.ctx + s.n, (col + 1) << a.c.page_log2);
  if (s.n == 0 || first >= last) return;
  const int m = last - first, i0 = first - s.ctx, fill = first & (page - 1);  // new tokens, first draft, tokens kept

  int* pos = reinterpret_cast<int*>(smem);             // [page] position of each new token
  int* par = pos + page;                               // [n] parents
  const int n_par = a.d.parent && a.rope ? min(s.n, kMaxTree) : 0;
  uint8_t* kc = smem + (((page + n_par) * 4 + 15) & ~15);  // [page][D] codes
  uint8_t* vc = kc + page * D;                             // [D][page + 4]
  const int v_pitch = page + 4;
  if (a.rope) {
    for (int i = tid; i < n_par; i += blockDim.x) par[i] = parent_of(a.d.parent + s.lo, i);
    __syncthreads();
    for (int r = tid; r < m; r += blockDim.x) {
      int depth = i0 + r;
      if (n_par) {
        depth = 0;
        for (int j = par[i0 + r]; j >= 0; j = par[j]) ++depth;  // parents come earlier: at most n steps
      }
      int p = s.ctx + depth;
      if (p >= a.rope_rows) {
        report(a.d.status, 3);
        p = a.rope_rows - 1;
      }
      pos[r] = p;
    }
    __syncthreads();
  }
  constexpr int kHalf = D / 16;  // pieces of 8 columns in half a row; a thread takes one and its partner
  if (part > 0) {
    const int items = m * a.rep * kHalf, step = a.q_parts * blockDim.x;
    for (int z = (part - 1) * blockDim.x + tid; z < items; z += step) {
      const int rr = z / kHalf, c = (z % kHalf) * 8, r = rr / a.rep, h = head * a.rep + rr - r * a.rep;
      const long long token = s.lo + i0 + r;
      float x[8], y[8];
      load_rotated<D>(a.q + token * a.q_stride + h * D, a.rope ? a.rope + (long long)pos[r] * D : nullptr, c, x, y);
      __nv_bfloat16* o = a.q_out + token * a.q_out_stride + h * D + c;
      store8(o, x);
      store8(o + D / 2, y);
    }
    return;
  }
  const __nv_bfloat16* krow = a.k + (long long)(s.lo + i0) * a.k_stride + head * D;
  const __nv_bfloat16* vrow = a.v + (long long)(s.lo + i0) * a.v_stride + head * D;
  float mk = 0.f, mv = 0.f;
  for (int z = tid; z < m * kHalf; z += blockDim.x) {
    const int r = z / kHalf, c = (z % kHalf) * 8;
    float x[8], y[8];
    load_rotated<D>(krow + (long long)r * a.k_stride, a.rope ? a.rope + (long long)pos[r] * D : nullptr, c, x, y);
#pragma unroll
    for (int i = 0; i < 8; ++i) mk = fmaxf(mk, fmaxf(fabsf(x[i]), fabsf(y[i])));
    load_rotated<D>(vrow + (long long)r * a.v_stride, nullptr, c, x, y);
#pragma unroll
    for (int i = 0; i < 8; ++i) mv = fmaxf(mv, fmaxf(fabsf(x[i]), fabsf(y[i])));
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    mk = fmaxf(mk, __shfl_xor_sync(0xffffffffu, mk, o));
    mv = fmaxf(mv, __shfl_xor_sync(0xffffffffu, mv, o));
  }
  if ((tid & 31) == 0) { red[0][tid >> 5] = mk; red[1][tid >> 5] = mv; }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < 8; ++w) { mk = fmaxf(mk, red[0][w]); mv = fmaxf(mv, red[1][w]); }

  const int pid = page_of(a.d, a.c, b, col);
  if (pid >= 0) {
    const long long slot = (long long)pid * a.c.heads + head;
    const float k_was = a.c.ks[slot], v_was = a.c.vs[slot];
    float k_now = cache_scale(mk), v_now = cache_scale(mv);
    if (fill) { k_now = fmaxf(k_now, k_was); v_now = fmaxf(v_now, v_was); }
    k_now = k_now > 0.f ? k_now : 1.f;
    v_now = v_now > 0.f ? v_now : 1.f;
    __syncthreads();  // everybody has read the old scales
    if (tid == 0) { a.c.ks[slot] = k_now; a.c.vs[slot] = v_now; }
    const float k_inv = 1.f / k_now, v_inv = 1.f / v_now;
    for (int z = tid; z < m * kHalf; z += blockDim.x) {
      const int r = z / kHalf, c = (z % kHalf) * 8;
      float x[8], y[8];
      load_rotated<D>(krow + (long long)r * a.k_stride, a.rope ? a.rope + (long long)pos[r] * D : nullptr, c, x, y);
      uint32_t u[4] = {0, 0, 0, 0};
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        u[i >> 2] |= cache_code(x[i], k_inv) << (8 * (i & 3));
        u[2 + (i >> 2)] |= cache_code(y[i], k_inv) << (8 * (i & 3));
      }
      *reinterpret_cast<uint2*>(kc + r * D + c) = make_uint2(u[0], u[1]);
      *reinterpret_cast<uint2*>(kc + r * D + c + D / 2) = make_uint2(u[2], u[3]);
      load_rotated<D>(vrow + (long long)r * a.v_stride, nullptr, c, x, y);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        vc[(c + i) * v_pitch + fill + r] = (uint8_t)cache_code(x[i], v_inv);
        vc[(c + i + D / 2) * v_pitch + fill + r] = (uint8_t)cache_code(y[i], v_inv);
      }
    }
    __syncthreads();
    // K: the new rows are one contiguous run; the kept rows only where the scale grew
    uint8_t* kp = a.c.k + slot * page * D;
    for (int z = tid; z < m * D / 16; z += blockDim.x)
      reinterpret_cast<uint4*>(kp + fill * D)[z] = reinterpret_cast<const uint4*>(kc)[z];
    if (fill && k_now != k_was) {
      const float f = k_was / k_now;
      for (int z = tid; z < fill * D / 4; z += blockDim.x) {
        uint32_t* p = reinterpret_cast<uint32_t*>(kp) + z;
        *p = rescale4(*p, f);
      }
    }
    // V: words of 4 tokens of one dimension; kept tokens change only where the scale grew, others not at all
    uint8_t* vp = a.c.v + slot * page * D;
    const bool grow = fill && v_now != v_was;
    const float f = grow ? v_was / v_now : 1.f;
    const int w0 = grow ? 0 : fill / 4, nw = (fill + m + 3) / 4 - w0;
    for (int z = tid; z < D * nw; z += blockDim.x) {
      const int d = z / nw, w = w0 + z % nw;
      uint32_t* p = reinterpret_cast<uint32_t*>(vp + d * page) + w;
      const int a0 = fill - 4 * w, a1 = fill + m - 4 * w;  // bytes [a0, a1) of the word are new
      const uint32_t fresh = *reinterpret_cast<const uint32_t*>(vc + d * v_pitch + 4 * w);
      if (a0 <= 0 && a1 >= 4) *p = fresh;
      else {
        const uint32_t low = a0 <= 0 ? 0u : a0 >= 4 ? 0xffffffffu : (1u << (8 * a0)) - 1u;     // kept tokens
        const uint32_t high = a1 >= 4 ? 0u : a1 <= 0 ? 0xffffffffu : 0xffffffffu << (8 * a1);  // not this call's
        const uint32_t was = *p;
        const uint32_t kept = grow ? rescale4(was, f) : was;
        *p = (kept & low) | (was & high) | (fresh & ~(low | high));
      }
    }
  }
}

}  // namespace kv
}  // namespace moev
