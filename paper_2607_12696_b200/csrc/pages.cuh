// What a batch's next call needs, from the lengths of its sequences: offsets of the token rows, pages from a free list for the
// tokens to come, every token's position and cache slot.
//
//   cu[b] = sum of new_len in front of b;  sequence b holds ceil(ctx / page) pages and needs ceil((ctx + new) / page): the ones that
//   are missing are the next of the free list, in the order of the sequences;  token i of b: position ctx + i, slot = page id * page +
//   position % page.
//
// A CTA takes 256 sequences and, of their pages and of groups of 4 tokens, every parts-th block of 256.  It sums the lengths in front of
// its sequences itself (they come from the L2), so there is one launch and nobody waits for anybody.
//
// Measured: 32 sequences of 4 drafts 4.0 us a call (3.6 in a graph), 300 prompts of 450 000 tokens 7.6 (6.7): latency, a chain of lengths, sums, page ids and rows.
#pragma once
#include "kv_cache.cuh"

namespace moev {
namespace pages {

constexpr int kChunk = 256;

struct Args {
  const int32_t *ctx_len, *new_len, *free_pages, *free_first;
  int32_t *table, *cu, *slots, *positions, *taken, *status;
  int n_seq, n_tokens, page_log2, cols, n_free, parts;
  int vec;  // slots and positions on 16-byte boundaries
};
struct Need {
  int ctx, tokens, have, want;  // tokens there and to come, pages there and to come
};
__device__ __forceinline__ Need need_of(const Args& a, int b) {
  Need q{a.ctx_len[b], a.new_len[b], 0, 0};
  const long long room = (long long)a.cols << a.page_log2;
  if (q.ctx < 0 || q.tokens < 0 || (long long)q.ctx + q.tokens > room) {
    kv::report(a.status, 1);
    return Need{0, 0, 0, 0};
  }
  const int up = (1 << a.page_log2) - 1;
  q.have = (int)(((long long)q.ctx + up) >> a.page_log2);
  q.want = (int)(((long long)q.ctx + q.tokens + up) >> a.page_log2) - q.have;
  return q;
}
struct Sums {
  long long tokens, pages;
};
// Inclusive sums over the CTA's threads; `total` gets the last one.
__device__ __forceinline__ Sums scan(Sums v, Sums* warps, Sums& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int o = 1; o < 32; o *= 2) {
    const long long t = __shfl_up_sync(0xffffffffu, v.tokens, o), p = __shfl_up_sync(0xffffffffu, v.pages, o);
    if (lane >= o) {
      v.tokens += t;
      v.pages += p;
    }
  }
  if (lane == 31) warps[warp] = v;
  __syncthreads();
  Sums before{0, 0};
  total = Sums{0, 0};
#pragma unroll
  for (int w = 0; w < kChunk / 32; ++w) {
    if (w == warp) before = total;
    total.tokens += warps[w].tokens;
    total.pages += warps[w].pages;
  }
  __syncthreads();
  return Sums{v.tokens + before.tokens, v.pages + before.pages};
}
// First of the chunk's n entries whose sum is beyond `at`.
__device__ __forceinline__ int find(const long long* ends, int n, long long at) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (ends[mid] > at) hi = mid;
    else lo = mid + 1;
  }
  return lo;
}

__device__ __forceinline__ void put4(int32_t* out, long long r0, const int (&v)[4], bool vec, long long from, long long to) {
  if (vec) {
    *reinterpret_cast<int4*>(out + r0) = make_int4(v[0], v[1], v[2], v[3]);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (r0 + e >= from && r0 + e < to) out[r0 + e] = v[e];
  }
}

__global__ void __launch_bounds__(kChunk) pages_kernel(const Args a) {
  __shared__ Sums warps[kChunk / 32];
  __shared__ long long token_end[kChunk], page_end[kChunk];
  __shared__ Need need[kChunk];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int tid = threadIdx.x, chunk = blockIdx.x / a.parts, part = blockIdx.x % a.parts;
  const int first = chunk * kChunk, n = min(kChunk, a.n_seq - first);
  const int free_first = a.free_first ? *a.free_first : 0;
  const int avail = free_first < 0 || free_first > a.n_free ? 0 : a.n_free - free_first;
  const int32_t* fresh = a.free_pages + (avail ? free_first : 0);
  Need q{0, 0, 0, 0};
  if (tid < n) q = need_of(a, first + tid);
  Sums front{0, 0}, total;
  for (int b = tid; b < first; b += kChunk) {
    const Need other = need_of(a, b);
    front.tokens += other.tokens;
    front.pages += other.want;
  }
  if (first > 0) scan(front, warps, front);
  const Sums end = scan(Sums{q.tokens, q.want}, warps, total);
  need[tid] = q;
  token_end[tid] = end.tokens;
  page_end[tid] = end.pages;
  __syncthreads();
  auto row_of = [](long long t) { return (int32_t)min(t, 0x7fffffffLL); };
  if (part == 0 && tid < n) a.cu[first + tid] = row_of(front.tokens + end.tokens - q.tokens);
  const bool is_last = first + kChunk >= a.n_seq;
  if (part == 0 && is_last && tid == 0) {
    a.cu[a.n_seq] = row_of(front.tokens + total.tokens);
    if (a.taken) *a.taken = (int32_t)min(front.pages + total.pages, (long long)avail);
    if (front.pages + total.pages > avail) kv::report(a.status, 2);
    if ((a.slots || a.positions) && front.tokens + total.tokens > a.n_tokens) kv::report(a.status, 3);
  }
  const long long step = (long long)a.parts * kChunk;
  for (long long i = (long long)part * kChunk + tid; i < total.pages; i += step) {
    const int s = find(page_end, n, i);
    const long long at = front.pages + i;
    a.table[(long long)(first + s) * a.cols + need[s].have + (int)(i - (page_end[s] - need[s].want))] = at < avail ? fresh[at] : -1;
  }
  if (!a.slots && !a.positions) return;
  // A thread takes 4 rows side by side, from a multiple of 4: one search, and 16 bytes written at once where all four are the chunk's.
  const long long end_row = min(front.tokens + total.tokens, (long long)a.n_tokens);
  for (long long r0 = (front.tokens & ~3LL) + 4 * ((long long)part * kChunk + tid); r0 < end_row; r0 += 4 * step) {
    int s = find(token_end, n, max(0LL, r0 - front.tokens)), slot[4], position[4];
    const int32_t* from[4];  // where the page ids stand: looked up side by side (one after the other 32 sequences take 0.5 us more)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const long long i = r0 + e - front.tokens;
      position[e] = -1;
      from[e] = nullptr;
      if (i < 0 || r0 + e >= end_row) continue;
      while (token_end[s] <= i) ++s;
      const Need w = need[s];
      const int pos = w.ctx + (int)(i - (token_end[s] - w.tokens)), col = pos >> a.page_log2;
      const long long at = front.pages + page_end[s] - w.want + (col - w.have);
      position[e] = pos;
      if (col < w.have) from[e] = a.table + (long long)(first + s) * a.cols + col;
      else if (at < avail) from[e] = fresh + at;
    }
    if (a.slots) {
      int id[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) id[e] = from[e] ? *from[e] : -1;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (position[e] >= 0 && (id[e] < 0 || id[e] > 0x7fffffff >> a.page_log2)) {
          kv::report(a.status, 2);
          id[e] = -1;
        }
        slot[e] = id[e] < 0 ? -1 : (id[e] << a.page_log2) + (position[e] & ((1 << a.page_log2) - 1));
      }
    }
    const bool all = r0 >= front.tokens && r0 + 4 <= end_row;
    if (a.positions) put4(a.positions, r0, position, all && a.vec, front.tokens, end_row);
    if (a.slots) put4(a.slots, r0, slot, all && a.vec, front.tokens, end_row);
  }
  if (is_last) {  // rows of no sequence
    for (long long r = front.tokens + total.tokens + (long long)part * kChunk + tid; r < a.n_tokens; r += step) {
      if (a.slots) a.slots[r] = -1;
      if (a.positions) a.positions[r] = -1;
    }
  }
}

}  // namespace pages
}  // namespace moev
