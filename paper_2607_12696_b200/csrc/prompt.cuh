// Causal attention of whole prompts (or of chunks behind keys that are there already) on the fifth-generation tensor cores.
//
//   score[i, j] = scale * q_i . k_j for keys j <= pos(i) = keys - tokens + i of i's own sequence (the last `window` of them),
//   out_i = sum_j p[i, j] v_j,  p = softmax (with an optional sink logit per head in the denominator),  lse_i = log of it + maximum.
//
// A tile is 128 rows (token, query head): the query heads of one kv head lie side by side, 128 / heads tokens of them, so heads
// share the keys they read and a short sequence still fills a tile.  A CTA has two tiles; K and V tiles of 128 keys pass by
// once for both.  Both products are tcgen05.mma kind::f16 in bf16 with binary32 sums:
//   S [128 rows, 128 keys] = Q . K^T  (both from shared memory)       O [128 rows, D] += P . V  (P from tensor memory)
// V stays as it lies in memory ([key][d], its N contiguous).  A softmax thread has half of a row's keys of a tile (with two warps
// for 32 rows there are four on each scheduler to hide their latencies); the halves meet once a tile.  p is rounded once to bf16 (half a
// step 2^-8 relative at most, the type of v and out); maxima, denominators and O are binary32.  The reference of the exponentials is the maximum of the
// first tile that a row sees; it moves (and O is rescaled) only when p has grown beyond 2^8, which is rare and leaves O the range
// of binary32 but for a factor of 2^8: the sum of 2^8 |v| over the keys of a row has to stay below 2^128.
//
// Tensor memory, 512 columns at D = 128: one S (128), P of both tiles (64 each), O of both (128 each).  S is free as soon as it has been
// read into registers: S of the one tile is computed while the other's softmax is under way, the products with V in between, and
// no softmax waits for its own products.
//
// What a mask hides must not count, whatever is there: scores are selected, not added to; in V a masked NaN or infinity would
// survive the product with p = 0, so in tiles that some row does not see whole, values that are not finite become 0 in shared
// memory, and rows that do see them get them back at the end (from memory; such tiles are few and the case is rare).
//
// Roles: one warp loads (TMA ring of K and V tiles), one thread issues the MMAs (elected, so that its operands stay in uniform
// registers: with a test of the lane instead an MMA took 115 cycles to issue, 64 to run), eight warps per tile do its softmax.  Every wait
// is bounded.
//
// Measured (32 query heads, 4 kv heads, D 128): 16 000 tokens 1.58 ms (1.33 PFLOP/s, 0.80 of a large matrix product's rate) on a GPU that has
// rested for seconds, 1.81 to 1.85 ms call after call (the power limit).  What bounds it: two products of 512 cycles each per 128 x 128 scores beside
// 1024 cycles of exponentials (16 a cycle), which two tiles in turn share: tensor pipe and special functions 54 % busy each over a whole call of 4000 tokens,
// issue slots 54 %.
// Other splits that were slower: scores of 64 keys beside P, 870 to 990 TFLOP/s (an MMA that is 64 wide takes 52 cycles, not 32); a quarter of the
// exponentials as polynomials on the FMA pipe, 1082 for 1184 (registers and issue slots); persistent CTAs that draw their tiles (87 KB of code,
// spills: no better in any case but ragged batches, 500 us for 562, which the output's way through shared memory gave as well: 495).  The first loads begin
// before the CTA is set up (window 128: 121 -> 114 us).
#pragma once
#include <cuda.h>

#include "attend.cuh"

namespace moev {
namespace prm {

constexpr int kRows = 128;
constexpr float kSlack = 8.f;  // p may grow to 2^8 before the reference follows
constexpr unsigned long long kBudgetNs = kDeviceWaitBudgetNs;

struct Args {
  const int32_t *cu, *cu_k;
  int32_t* status;
  int n_seq, n_tokens, n_keys, max_tokens;
  const __nv_bfloat16* v;
  __nv_bfloat16* out;
  float* lse;
  const float* sinks;
  long long v_stride, out_stride;
  int n_heads, kv_heads, rep;      // rep: query heads of a kv head
  int tile_heads, groups, tokens;  // query heads of a tile, groups of those per kv head, tokens of a tile
  int window, pairs;               // pairs of tiles that max_tokens make
  float scale_log2;
};

// T = 2: as above.  T = 1: one tile of rows and tiles of 64 keys, small enough for two CTAs on an SM, each of which covers for the other's
// beginning and end: for prompts of few tiles of keys.
template <int D, int T>
struct Cfg {
  static constexpr int kKeys = T == 2 ? 128 : 64;  // of a tile
  static constexpr int kTile = kKeys * D * 2, kHalf = kKeys * 128;  // bytes of a tile of keys, of 64 columns of it
  static constexpr int kQTile = kRows * D * 2, kQHalf = kRows * 128;
  static constexpr int kStages = (D == 128 ? 5 : 10) - (T == 1 ? 1 + 3 * (D == 64) : 0);  // 160 KB, or 64 and 48
  // 8 warps softmax for each tile, 4 more of which one loads and one issues the MMAs.  The registers that a thread is launched with are shared
  // out anew: more for the softmax, fewer for the others
  static constexpr int kSoftmax = 256 * T, kThreads = kSoftmax + 128;
  static constexpr int kRegsLaunch = T == 2 ? 96 : 80, kRegsMore = T == 2 ? 104 : 88, kRegsLess = 64;
  static_assert(kSoftmax * kRegsMore + 128 * kRegsLess <= kThreads * kRegsLaunch && kThreads * kRegsLaunch * (3 - T) <= 65536, "registers");
  static constexpr int kP = kKeys, kO = 128 * T, kTmem = 256 * T;  // columns: S, P of the tiles, O of the tiles; all
  static_assert(kP + T * (kKeys / 2) <= kO && kO + T * D <= kTmem, "tensor memory");
  static constexpr int oQ = 0, oRing = T * kQTile, oCtl = oRing + kStages * kTile;
};
struct Ctl {
  uint64_t full[10], empty[10], q_full, s_full[2], s_free, p_full[2], pv_done[2], drain;
  float swap[2][kRows];  // by tile and row: what the two halves of a row exchange
  uint32_t tmem;
  int bad;  // some V of a masked tile was not finite
  volatile int abort;
  volatile uint32_t loaded;  // tiles the loader armed (read on the abort path)
};
template <int D, int T>
constexpr size_t smem_bytes() {
  return 1024 + Cfg<D, T>::oCtl + sizeof(Ctl);
}
// (an SM has 228 KB, of which each CTA takes one more)
static_assert(smem_bytes<64, 2>() <= 227 * 1024 && smem_bytes<128, 2>() <= 227 * 1024, "shared memory");
static_assert(smem_bytes<64, 1>() <= 113 * 1024 && smem_bytes<128, 1>() <= 113 * 1024, "shared memory of two");

// Place of the tiles of K and V in the order in which they are loaded: K runs one ahead.
__device__ __forceinline__ int k_item(int j) { return max(0, 2 * j - 1); }
__device__ __forceinline__ int v_item(int j, int n) { return min(2 * j + 2, 2 * n - 1); }

// A tile's rows and the keys they see.
struct Span {
  int first, tokens;  // first token of the sequence, number of tokens
  int low, high;      // positions of the first and the last token
  int begin, end;     // keys that some row sees
};
__device__ __forceinline__ Span span_of(const Args& a, int first, int n, int front, int keys) {
  Span s;
  s.first = first;
  s.tokens = max(0, min(a.tokens, n - first));
  s.low = front + first;
  s.high = s.low + s.tokens - 1;
  s.end = s.tokens > 0 ? max(0, min(keys, s.high + 1)) : 0;
  s.begin = a.window > 0 ? max(0, s.low - a.window + 1) : 0;
  s.begin = min(s.begin, s.end);
  return s;
}
// Tiles of keys that every row from position low to high sees whole: those that begin at first .. last.
struct Whole {
  int first, last;
  __device__ __forceinline__ bool at(int k0) const { return k0 >= first && k0 <= last; }
};
template <int KEYS>
__device__ __forceinline__ Whole whole_of(const Args& a, int low, int high) {
  return Whole{a.window > 0 ? high - a.window + 1 : 0, low - KEYS + 1};
}

__device__ __forceinline__ void cluster_sync() {
  __syncwarp();
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// 16 bytes of shared memory that another warp may be replacing by the same values.
__device__ __forceinline__ uint4 load_relaxed(const uint4* p) {
  uint4 w;
  asm volatile("ld.relaxed.cta.shared::cta.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w.x), "=r"(w.y), "=r"(w.z), "=r"(w.w) : "r"(ptx::smem_u32(p)) : "memory");
  return w;
}
__device__ __forceinline__ void store_relaxed(uint4* p, const uint4& w) {
  asm volatile("st.relaxed.cta.shared::cta.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(ptx::smem_u32(p)), "r"(w.x), "r"(w.y), "r"(w.z), "r"(w.w) : "memory");
}

// SPLIT: the CTAs of a cluster share the keys of a tile of rows; each leaves its normalised output and its lse in shared memory, and joins a
// share of the rows from all of them.
template <int D, int T, bool SPLIT>
__global__ void __launch_bounds__(Cfg<D, T>::kThreads, 3 - T) prompt_kernel(const Args a, const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                                                                     const __grid_constant__ CUtensorMap tm_v) {
  using C = Cfg<D, T>;
  constexpr int kKeys = C::kKeys, kLoader = C::kSoftmax / 32, kIssuer = kLoader + 1;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  Ctl& S = *reinterpret_cast<Ctl*>(smem + C::oCtl);
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  if (warp == kLoader && lane == 0) {  // the thread that loads: it begins before the CTA is set up
    for (int i = 0; i < C::kStages; ++i) {
      ptx::mbar_init(&S.full[i], 1);
      ptx::mbar_init(&S.empty[i], 1);
    }
    ptx::mbar_init(&S.q_full, 1);
    for (int i = 0; i < T; ++i) {
      ptx::mbar_init(&S.s_full[i], 1);
      ptx::mbar_init(&S.p_full[i], 8);
      ptx::mbar_init(&S.pv_done[i], 1);
    }
    ptx::mbar_init(&S.s_free, 8);
    ptx::mbar_init(&S.drain, 1);
    ptx::fence_mbar_init();
    ptx::fence_proxy_async_smem();
    S.abort = 0;
    S.bad = 0;
    S.loaded = 0;
    ptx::prefetch_tmap(&tm_q);
    ptx::prefetch_tmap(&tm_k);
    ptx::prefetch_tmap(&tm_v);
  }
  asm volatile("griddepcontrol.wait;" ::: "memory");
  uint32_t rank = 0, ranks = 1;
  if (SPLIT) {
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(ranks));
  }
  // the last pairs of tiles, which see most keys, come first
  const int index = blockIdx.x / ranks, per = a.kv_heads * a.groups * a.n_seq, pair = a.pairs - 1 - index / per;
  const int in_pair = index % per, b = in_pair / (a.kv_heads * a.groups), head_group = in_pair % (a.kv_heads * a.groups);
  const int kv_head = head_group / a.groups, head0 = kv_head * a.rep + head_group % a.groups * a.tile_heads;
  const int lo = a.cu[b], n = a.cu[b + 1] - lo, lo_k = a.cu_k[b], keys = a.cu_k[b + 1] - lo_k;
  if (lo < 0 || n < 0 || n > a.max_tokens || n > a.n_tokens - lo || lo_k < 0 || keys < 0 || keys > a.n_keys - lo_k) {
    if (tid == 0) kv::report(a.status, 1);
    return;
  }
  if (pair * T * a.tokens >= n) return;
  Span sp[2];
#pragma unroll
  for (int t = 0; t < 2; ++t) sp[t] = t < T ? span_of(a, (T * pair + t) * a.tokens, n, keys - n, keys) : Span{0, 0, 0, 0, 0, 0};
  // tiles of keys from the first key that the first tile sees; a tile of rows takes part from .. to
  int k_first = sp[0].begin;
  int from[2], to[2];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    from[t] = max(0, sp[t].begin - k_first) / kKeys;
    to[t] = sp[t].end > sp[t].begin ? (sp[t].end - k_first + kKeys - 1) / kKeys : from[t];
  }
  if (SPLIT) {  // (one tile of rows) this CTA's share of the tiles of keys
    const int all = to[0], at = (int)(all * rank / ranks);
    to[0] = (int)(all * (rank + 1) / ranks) - at;
    k_first += at * kKeys;
  }
  const int n_tiles = max(to[0] > from[0] ? to[0] : 0, to[1] > from[1] ? to[1] : 0);
  // K 0, K 1, V 0, K 2, V 1, .. (k_item, v_item)
  auto load = [&](int i) {
    const int st = i % C::kStages;
    const bool is_v = i == 2 * n_tiles - 1 || (i > 0 && i % 2 == 0);
    const int tile = is_v ? (i == 2 * n_tiles - 1 ? n_tiles - 1 : i / 2 - 1) : (i + 1) / 2;
    ptx::mbar_arrive_expect_tx(&S.full[st], C::kTile);
    S.loaded = i + 1;
    for (int h = 0; h < D / 64; ++h)
      ptx::tma_load_3d(smem + C::oRing + st * C::kTile + h * C::kHalf, is_v ? &tm_v : &tm_k, &S.full[st], h * 64, kv_head, lo_k + k_first + tile * kKeys,
                       ptx::kPolicyEvictLast);
  };
  const int items = 2 * n_tiles - (MOEV_TEST_WITHHOLD() ? 1 : 0), fetched = min(items, C::kStages);
  if (warp == kLoader && lane == 0 && n_tiles > 0) {
    // Q of the tiles that see keys: one that sees none waits for nothing, and its outputs change places where its Q would land
    const uint32_t q_bytes = (uint32_t)a.tile_heads * a.tokens * D * 2;
    ptx::mbar_arrive_expect_tx(&S.q_full, q_bytes * ((to[0] > from[0]) + (to[1] > from[1])));
#pragma unroll
    for (int t = 0; t < 2; ++t)
      for (int h = 0; h < D / 64 && to[t] > from[t]; ++h)
        ptx::tma_load_3d(smem + C::oQ + t * C::kQTile + h * C::kQHalf, &tm_q, &S.q_full, h * 64, head0, lo + sp[t].first, ptx::kPolicyEvictFirst);
#pragma unroll 1
    for (int i = 0; i < fetched; ++i) load(i);
  }
  if (warp == kIssuer) {
    ptx::tmem_alloc(&S.tmem, C::kTmem);
    ptx::tmem_relinquish();
  }
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const uint32_t tmem = S.tmem;

  if (warp >= kLoader) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(C::kRegsLess));
    if (warp == kLoader) {
      // ------------------------------------------------------------ loader
      if (lane == 0) {
        for (int i = fetched; i < items; ++i) {
          if (!att::wait(&S.empty[i % C::kStages], ((i / C::kStages) & 1) ^ 1, &S.abort, a.status)) break;
          load(i);
        }
      }
    } else if (warp == kIssuer) {
      // ------------------------------------------------------------ MMA issuer
      if (n_tiles > 0 && ptx::elect_one()) {
        const uint32_t sdesc = ptx::instr_desc(1, 1, kKeys), odesc = ptx::instr_desc(1, 1, D) | (1u << 16);  // bf16; V with its N contiguous
        const uint32_t q_lo = ptx::desc_lo_sw128(ptx::smem_u32(smem + C::oQ)), k_lo = ptx::desc_lo_sw128(ptx::smem_u32(smem + C::oRing));
        // leading offset of V: from one block of 64 columns to the next
        const uint32_t v_lo = (k_lo & 0xFFFFu) | (uint32_t)(C::kHalf / 16) << 16;
        bool ok = att::wait(&S.q_full, 0, &S.abort, a.status);
        int scores = 0;  // S has been written so many times
        // S(t, j): when what was in S has been read
        auto score = [&](int t, int j) {
          const int item = k_item(j), st = item % C::kStages;
          ok = ok && att::wait(&S.full[st], (item / C::kStages) & 1, &S.abort, a.status);
          ok = ok && (scores == 0 || att::wait(&S.s_free, (scores - 1) & 1, &S.abort, a.status));
          if (!ok) return;
          ++scores;
          ptx::tc_fence_after();
          const uint32_t q_at = q_lo + t * (C::kQTile / 16), k_at = k_lo + st * (C::kTile / 16);
#pragma unroll
          for (int k = 0; k < D / 16; ++k) {
            ptx::mma_f16_lohi(tmem, q_at + (k / 4) * (C::kQHalf / 16) + (k % 4) * 2, k_at + (k / 4) * (C::kHalf / 16) + (k % 4) * 2, ptx::kDescHiSw128, sdesc, k > 0);
          }
          ptx::mma_commit(&S.s_full[t]);
        };
        auto weigh = [&](int t, int j) {
          const int item = v_item(j, n_tiles), st = item % C::kStages, i = j - from[t];
          ok = ok && att::wait(&S.full[st], (item / C::kStages) & 1, &S.abort, a.status);
          ok = ok && att::wait(&S.p_full[t], i & 1, &S.abort, a.status);
          if (!ok) return;
          ptx::tc_fence_after();
          const uint32_t v_at = v_lo + st * (C::kTile / 16);
#pragma unroll
          for (int k = 0; k < kKeys / 16; ++k)
            att::mma_f16_ta(tmem + C::kO + t * D, tmem + C::kP + t * (kKeys / 2) + k * 8, v_at + k * 128, ptx::kDescHiSw128, odesc, i > 0 || k > 0);
          ptx::mma_commit(&S.pv_done[t]);
        };
        // S of the one tile is computed while the other's softmax is under way, the products with V in between
        if (from[0] == 0 && to[0] > 0) score(0, 0);
        for (int j = 0; j <= n_tiles && ok; ++j) {
          if (T == 2 && j >= from[1] && j < to[1]) score(1, j);
          if (ok && j < n_tiles) ptx::mma_commit(&S.empty[k_item(j) % C::kStages]);
          if (j > from[0] && j <= to[0]) weigh(0, j - 1);
          if (j + 1 >= from[0] && j + 1 < to[0]) score(0, j + 1);
          if (T == 2 && j > from[1] && j <= to[1]) weigh(1, j - 1);
          if (ok && j > 0) ptx::mma_commit(&S.empty[v_item(j - 1, n_tiles) % C::kStages]);
        }
        if (!ok) ptx::drain_issuer(&S.drain, kBudgetNs);
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(C::kRegsMore));
    // ------------------------------------------------------------ softmax
    // the warp's quarter of tensor memory, a row a lane; of the row, half of the keys and half of the output's columns
    constexpr int kHalfKeys = kKeys / 2, kChunks = kHalfKeys / 32;
    const int t = T == 2 ? warp >> 3 : 0, half = (warp >> 2) & 1, row = (warp & 3) * 32 + lane, pair = 1 + t * 4 + (warp & 3);
    const Span my = t ? sp[1] : sp[0];
    const int my_from = t ? from[1] : from[0], my_to = t ? to[1] : to[0];
    const int token = row / a.tile_heads, head = row - token * a.tile_heads;
    const bool live = token < my.tokens && head0 + head < (kv_head + 1) * a.rep;
    const int pos = my.low + token;
    const Whole mine = whole_of<kKeys>(a, my.low, my.high), both = whole_of<kKeys>(a, sp[0].low, sp[1].tokens > 0 ? sp[1].high : sp[0].high);
    const int see_to = live ? min(pos, keys - 1) : -1, see_from = a.window > 0 ? pos - a.window + 1 : 0;  // keys see_from .. see_to
    const uint32_t lanes = tmem + ((uint32_t)(warp & 3) << 21), s_at = lanes + half * kHalfKeys, p_at = lanes + C::kP + t * kHalfKeys + half * (kHalfKeys / 2), o_at = lanes + C::kO + t * D + half * (D / 2);
    float* const swap = S.swap[t] + row;
    const float c = a.scale_log2;
    float m = -INFINITY, l = 0.f;  // reference (a score), this half's share of the denominator
    bool ok = true;
    // a wait that ran out ends nothing here: all warps meet at the same barriers to the end, whose outputs are then undefined
    for (int j = my_from; j < my_to; ++j) {
      const int i = j - my_from;
      ok = att::wait_warp(&S.s_full[t], i & 1, &S.abort, a.status, lane) && ok;
      ptx::tc_fence_after();
      uint32_t r[kChunks][32];
#pragma unroll
      for (int q = 0; q < kChunks; ++q) ptx::tmem_ld32(s_at + q * 32, r[q]);
      ptx::tmem_ld_wait();
      ptx::tc_fence_before();
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(&S.s_free);
      const int k0 = k_first + j * kKeys;
      if (!mine.at(k0)) {
        const int first = see_from - k0 - half * kHalfKeys, last = see_to - k0 - half * kHalfKeys;
#pragma unroll
        for (int q = 0; q < kChunks; ++q)
          if (!__all_sync(0xffffffffu, first <= q * 32 && last >= q * 32 + 31)) {
#pragma unroll
            for (int e = 0; e < 32; ++e)
              if (q * 32 + e < first || q * 32 + e > last) r[q][e] = 0xff800000u;
          }
      }
      float tops[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
      for (int q = 0; q < kChunks; ++q)
#pragma unroll
        for (int e = 0; e < 32; e += 2) tops[(e >> 1) & 3] = fmaxf(tops[(e >> 1) & 3], fmaxf(__uint_as_float(r[q][e]), __uint_as_float(r[q][e + 1])));
      float top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
      // both halves of a row have the same reference: they meet here, and where some row's is to move, exchange the maxima
      auto beyond = [&] { return live && top > m && (m == -INFINITY || (top - m) * c > kSlack); };
      if (att::any_of(beyond(), pair, 64)) {
        if (half == 0) *swap = top;
        ptx::named_barrier(pair, 64);
        if (half == 1) *swap = top = fmaxf(top, *swap);
        ptx::named_barrier(pair, 64);
        if (half == 0) top = *swap;
        float f = 1.f;
        if (beyond()) {
          f = m == -INFINITY ? 0.f : att::exp2_fast((m - top) * c);
          m = top;
        }
        l *= f;
        if (i > 0) {  // O is there once the last product has ended
          ok = att::wait_warp(&S.pv_done[t], (i - 1) & 1, &S.abort, a.status, lane) && ok;
          ptx::tc_fence_after();
#pragma unroll 1
          for (int q = 0; q < D / 32; ++q) {
            uint32_t o[16];
            ptx::tmem_ld16(o_at + q * 16, o);
            ptx::tmem_ld_wait();
#pragma unroll
            for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
            att::tmem_st(o_at + q * 16, o);
          }
        }
      }
      const float mc = m == -INFINITY ? 0.f : m * c;
      float sum[4] = {0.f, 0.f, 0.f, 0.f};
      uint32_t p[kHalfKeys / 2];
#pragma unroll
      for (int e = 0; e < kHalfKeys / 2; ++e) {
        float x = __uint_as_float(r[e / 16][2 * (e % 16)]), y = __uint_as_float(r[e / 16][2 * (e % 16) + 1]);
        att::fma2(x, y, c, c, -mc, -mc);
        x = att::exp2_fast(x);
        y = att::exp2_fast(y);
        att::add2(sum[2 * (e & 1)], sum[2 * (e & 1) + 1], x, y);
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(p[e]) : "f"(y), "f"(x));
      }
      // P is read by the product of the tile before
      if (i > 0) ok = att::wait_warp(&S.pv_done[t], (i - 1) & 1, &S.abort, a.status, lane) && ok;
      ptx::tc_fence_after();
      att::tmem_st(p_at, p);
      l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
      if (!both.at(k0)) {
        // what some row does not see must not reach it through p = 0; both tiles' warps see to that, the same values at the same places
        const int iv = v_item(j, n_tiles);
        ok = att::wait_warp(&S.full[iv % C::kStages], (iv / C::kStages) & 1, &S.abort, a.status, lane) && ok;
        uint4* v = reinterpret_cast<uint4*>(smem + C::oRing + (iv % C::kStages) * C::kTile);
        bool bad = false;
#pragma unroll 4
        for (int z = tid & 255; z < C::kTile / 16 && ok; z += 256) {
          const uint4 w = T == 2 ? load_relaxed(v + z) : v[z];
          uint32_t w4[4] = {w.x, w.y, w.z, w.w}, any = 0;
          // an exponent of ones carries into the bit above it
#pragma unroll
          for (int e = 0; e < 4; ++e) any |= ((w4[e] & 0x7f807f80u) >> 1) + 0x00400040u;
          if (any & 0x40004000u) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              if ((w4[e] & 0x7f80u) == 0x7f80u) w4[e] &= 0xffff0000u;
              if ((w4[e] & 0x7f800000u) == 0x7f800000u) w4[e] &= 0xffffu;
            }
            if (k0 + (z & (C::kHalf / 16 - 1)) / 8 < keys) S.bad = 1;  // keys behind the sequence are nobody's
            __threadfence_block();
            const uint4 clean = make_uint4(w4[0], w4[1], w4[2], w4[3]);
            if (T == 2) store_relaxed(v + z, clean);
            else v[z] = clean;
            bad = true;
          }
        }
        if (T == 2 || bad) ptx::fence_proxy_async_smem();  // what it has read may be the other tile's doing, which this tile's product then reads
      }
      att::tmem_st_wait();
      ptx::tc_fence_before();
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(&S.p_full[t]);
    }
    const int n_mine = my_to - my_from;
    if (n_mine > 0) ok = att::wait_warp(&S.pv_done[t], (n_mine - 1) & 1, &S.abort, a.status, lane) && ok;
    if (my.tokens > 0) {
      if (half == 0) *swap = l;
      ptx::named_barrier(9 + t, 256);
      if (half == 1) *swap = l += *swap;
      ptx::named_barrier(9 + t, 256);
      if (half == 0) l = *swap;
      ptx::tc_fence_after();
      const bool fix = *reinterpret_cast<volatile int*>(&S.bad) != 0;
      const float mc = m == -INFINITY ? 0.f : m * c;
      float lse2 = l > 0.f ? mc + att::log2_fast(l) : l == 0.f ? -INFINITY : l;  // NaN stays
      float inv = l > 0.f ? 1.f / l : l == 0.f ? 0.f : l;
      if (!SPLIT && a.sinks && live) {
        const float sink = a.sinks[head0 + head] * 1.4426950408889634f;
        // the larger of the two is the reference of their sum
        const float ref = fmaxf(sink, lse2), all = (sink == ref ? 1.f : att::exp2_fast(sink - ref)) + att::exp2_fast(lse2 - ref);  // (an infinite sink is its own reference)
        if (l != 0.f) {
          inv *= att::exp2_fast(lse2 - ref) / all;
          lse2 = lse2 != lse2 ? lse2 : ref + att::log2_fast(all);
        }
      }
      const int hq = head0 + head;
      const long long out_at = live && ok ? (long long)(lo + my.first + token) * a.out_stride + (long long)hq * D + half * (D / 2) : -1;
      // A row is written by D / 16 lanes, 16 bytes each: they change places where Q was (its last product has ended), a row's pieces swizzled.
      constexpr int kPieces = D / 16, kAtOnce = 32 / kPieces;
      uint8_t* const turn = smem + C::oQ + warp * (32 * D);
#pragma unroll 1
      for (int q = 0; q < D / 64; ++q) {
        uint32_t o[32];
        if (my_to > my_from) {
          ptx::tmem_ld32(o_at + q * 32, o);
          ptx::tmem_ld_wait();
        }
        float x[32];
#pragma unroll
        for (int i = 0; i < 32; ++i) x[i] = l == 0.f ? 0.f : __uint_as_float(o[i]) * inv;
        if (fix && live) {
          for (int j = my_from; j < my_to; ++j) {
            const int k0 = k_first + j * kKeys;
            if (both.at(k0)) continue;
            for (int k = max(k0, see_from); k <= min(k0 + kKeys - 1, see_to); ++k) {
              const __nv_bfloat16* v = a.v + (long long)(lo_k + k) * a.v_stride + (long long)kv_head * D + half * (D / 2) + q * 32;
#pragma unroll
              for (int i = 0; i < 32; ++i) {
                const float y = __bfloat162float(v[i]);
                if (!(fabsf(y) < INFINITY)) x[i] += y;
              }
            }
          }
        }
        if (SPLIT) {
#pragma unroll
          for (int i = 0; i < 32; i += 4)
            *reinterpret_cast<float4*>(smem + row * (4 * D) + (((half * (D / 8) + q * 8 + i / 4) ^ (row & 7)) << 4)) = make_float4(x[i], x[i + 1], x[i + 2], x[i + 3]);
        } else {
#pragma unroll
          for (int i = 0; i < 32; i += 8) {
            uint32_t u[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(u[e]) : "f"(x[i + 2 * e + 1]), "f"(x[i + 2 * e]));
            *reinterpret_cast<uint4*>(turn + lane * D + (((q * 4 + i / 8) ^ (lane & (kPieces - 1))) << 4)) = make_uint4(u[0], u[1], u[2], u[3]);
          }
        }
      }
      if (SPLIT) {
        if (half == 0) S.swap[1][row] = lse2;
      } else {
        __syncwarp();
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
          const int from_row = i * kAtOnce + lane / kPieces, piece = lane % kPieces;
          const long long at = __shfl_sync(0xffffffffu, out_at, from_row);
          const uint4 u = *reinterpret_cast<const uint4*>(turn + from_row * D + ((piece ^ (from_row & (kPieces - 1))) << 4));
          if (at >= 0) *reinterpret_cast<uint4*>(a.out + at + piece * 8) = u;
        }
        if (live && a.lse && half == 0)  // (of a row that sees nothing the sink as it is given)
          a.lse[(long long)(lo + my.first + token) * a.n_heads + hq] = l == 0.f && a.sinks ? a.sinks[hq] : lse2 * 0.6931471805599453f;
      }
    }
  }
  if (SPLIT) {
    cluster_sync();
    if (warp < kLoader) {
      const int rows = kRows / (int)ranks;
      for (int i = tid; i < rows * (D / 4); i += C::kSoftmax) {
        const int row = (int)rank * rows + i / (D / 4), piece = i % (D / 4), token = row / a.tile_heads, head = row - token * a.tile_heads;
        if (token >= sp[0].tokens || head0 + head >= (kv_head + 1) * a.rep) continue;
        float lse2[8];
        float4 x[8];
#pragma unroll
        for (uint32_t p = 0; p < 8; ++p) {
          if (p < ranks) {
            uint32_t at;
            asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(ptx::smem_u32(&S.swap[1][row])), "r"(p));
            asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(lse2[p]) : "r"(at));
            asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(ptx::smem_u32(smem + row * (4 * D) + ((piece ^ (row & 7)) << 4))), "r"(p));
            asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(x[p].x), "=f"(x[p].y), "=f"(x[p].z), "=f"(x[p].w) : "r"(at));
          }
        }
        const float sink_in = a.sinks ? a.sinks[head0 + head] : -INFINITY, sink = sink_in * 1.4426950408889634f;
        float ref = sink, all = 0.f;
#pragma unroll
        for (uint32_t p = 0; p < 8; ++p)
          if (p < ranks) ref = fmaxf(ref, lse2[p]);
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
        if (ref > -INFINITY) {
          all = sink == ref ? 1.f : att::exp2_fast(sink - ref);
#pragma unroll
          for (uint32_t p = 0; p < 8; ++p) {
            if (p < ranks && lse2[p] != -INFINITY) {  // (a part without keys has no output either)
              const float f = att::exp2_fast(lse2[p] - ref);
              all += f;
              o.x = fmaf(f, x[p].x, o.x);
              o.y = fmaf(f, x[p].y, o.y);
              o.z = fmaf(f, x[p].z, o.z);
              o.w = fmaf(f, x[p].w, o.w);
            }
          }
          const float inv = 1.f / all;
          o.x *= inv;
          o.y *= inv;
          o.z *= inv;
          o.w *= inv;
        } else {  // nothing seen, or nothing but NaN
#pragma unroll
          for (uint32_t p = 0; p < 8; ++p)
            if (p < ranks && lse2[p] != lse2[p]) o.x = o.y = o.z = o.w = all = lse2[p];
        }
        const long long at = (long long)(lo + sp[0].first + token);
        const __nv_bfloat162 u = __floats2bfloat162_rn(o.x, o.y), v = __floats2bfloat162_rn(o.z, o.w);
        if (!S.abort)
          *reinterpret_cast<uint2*>(a.out + at * a.out_stride + (long long)(head0 + head) * D + piece * 4) =
              make_uint2(*reinterpret_cast<const uint32_t*>(&u), *reinterpret_cast<const uint32_t*>(&v));
        if (a.lse && piece == 0) {
          bool none = true;  // then the sink as it is given
#pragma unroll
          for (uint32_t p = 0; p < 8; ++p) none = none && (p >= ranks || lse2[p] == -INFINITY);
          a.lse[at * a.n_heads + head0 + head] = none ? sink_in : (ref + att::log2_fast(all)) * 0.6931471805599453f;
        }
      }
    }
    cluster_sync();
  }
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  if (S.abort && warp == kLoader && lane == 0) {  // copies still in flight would land in what the next CTA owns
    ptx::drain_wait(&S.q_full, 0, kBudgetNs);
    ptx::drain_ring(S.full, C::kStages, S.loaded, kBudgetNs);
  }
  if (warp == kIssuer) ptx::tmem_dealloc(tmem, C::kTmem);
}

}  // namespace prm
}  // namespace moev
