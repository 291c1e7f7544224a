// Log probabilities of given tokens under rows of logits, the rows' entropies, and the k most probable tokens.
//
//   l = scale * z,  lse = log sum_v exp(l_v),  logprob_j = l[id_j] - lse,  H = lse - sum_v p_v l_v
//
// One pass over the logits: a thread keeps the maximum x of what it has seen, S = sum 2^d and T = sum d 2^d with d = (z - x) scale
// log2(e); threads, warps and the CTAs of a row (a cluster, where there are few rows) are joined by moving S and T to the larger
// maximum.  Then H = ln(2) (log2 S - T / S): the differences are taken before anything is multiplied, so a row of the type's
// lowest values is as good as any other.  z of -infinity counts nothing; NaN and +infinity make all of a row's numbers NaN.
//
// The k largest come from the threads' maxima: with T the k-th largest of the maxima of groups of 4 threads, k values or more are not
// below T, and they lie in groups whose maximum is not.  Only those groups (hardly more than k of the 128, 64 or 32 that 512, 256 or 128 threads make: with 32 groups and
// k = 32 every one) are read again, a warp a group;
// what is not below T gets its rank by counting.  Where more than fit are equal, the warps keep sorted lists of k
// instead (ties go to the lowest id in either way).
//
// Measured: 4096 x 100003 binary32 240 us without alternatives (6.8 TB/s: memory), 8 of them 295 to 303, 32 376 (the second reading of the groups, rows'
// ends that no other row's loads cover); 64 x 151937 bf16, 5 of them 11.6 us (9 without): 3 us to read, the rest is latency, the joins
// (barriers) and the second reading; one row of 100003, 20 of them 8.7 us on a cluster of 8 (5.1 without).
#pragma once
#include "common.cuh"

namespace moev {
namespace lp {

constexpr int kMaxK = 32, kMaxCand = 256, kMaxRanks = 8;

struct Args {
  const void* logits;
  const int32_t* ids;
  float *logprobs, *entropy, *lse, *top_logprobs;
  int32_t* top_ids;
  long long stride;
  int n, V, m, k;
  float scale;
};
struct Stat {
  float x, s, t;  // maximum (never below the lowest finite number), sum of 2^d, sum of d 2^d
};
constexpr float kLowest = -3.402823466e38f;

__device__ __forceinline__ float ex2(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
// d no lower than -1000, where 2^d is 0 and d 2^d too; a NaN stays
__device__ __forceinline__ float floor_d(float d) {
  float r;
  asm("max.NaN.f32 %0, %1, 0fC47A0000;" : "=f"(r) : "f"(d));
  return r;
}
__device__ __forceinline__ void move_to(Stat& a, float x, float c) {
  const float d = floor_d((a.x - x) * c), f = ex2(d);
  a.t = f * fmaf(d, a.s, a.t);
  a.s *= f;
  a.x = x;
}
__device__ __forceinline__ Stat join(Stat a, Stat b, float c) {
  const float x = fmaxf(a.x, b.x);
  move_to(a, x, c);
  move_to(b, x, c);
  a.s += b.s;
  a.t += b.t;
  return a;
}
// Larger value first, then the lower id; 0 is below every value.  -0 counts as 0.
__device__ __forceinline__ unsigned long long key_of(float z, int id) {
  const uint32_t b = __float_as_uint(z + 0.f);
  return (unsigned long long)(b & 0x80000000u ? ~b : b | 0x80000000u) << 32 | (uint32_t)~id;
}
__device__ __forceinline__ float key_value(unsigned long long key) {
  const uint32_t b = (uint32_t)(key >> 32);
  return __uint_as_float(b & 0x80000000u ? b ^ 0x80000000u : ~b);
}

template <typename T>
struct Vec;
template <>
struct Vec<float> {
  static constexpr int n = 4;
  static __device__ __forceinline__ void unpack(const uint4& w, float (&v)[4]) {
    v[0] = __uint_as_float(w.x); v[1] = __uint_as_float(w.y); v[2] = __uint_as_float(w.z); v[3] = __uint_as_float(w.w);
  }
  static __device__ __forceinline__ float one(const float* p) { return *p; }
};
template <>
struct Vec<__nv_bfloat16> {
  static constexpr int n = 8;
  static __device__ __forceinline__ void unpack(const uint4& w, float (&v)[8]) {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[2 * e] = __uint_as_float(u[e] << 16);
      v[2 * e + 1] = __uint_as_float(u[e] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ float one(const __nv_bfloat16* p) { return __bfloat162float(*p); }
};

template <int N>
__device__ __forceinline__ void take(Stat& a, const float (&v)[N], float c) {
  float top = v[0];
#pragma unroll
  for (int e = 1; e < N; ++e) top = fmaxf(top, v[e]);
  if (top > a.x) move_to(a, top, c);
#pragma unroll
  for (int e = 0; e < N; ++e) {
    const float d = floor_d((v[e] - a.x) * c), p = ex2(d);
    a.s += p;
    a.t = fmaf(d, p, a.t);
  }
}

// Puts a key into a list sorted over the warp's lanes (largest in lane 0).
__device__ __forceinline__ void insert(unsigned long long& mine, unsigned long long key, int lane) {
  const unsigned above = __ballot_sync(0xffffffffu, mine > key);
  const int at = __popc(above);
  const unsigned long long up = __shfl_up_sync(0xffffffffu, mine, 1);
  if (lane == at) mine = key;
  else if (lane > at) mine = up;
}

// kThreads: 128, 256 or 512; 2048 threads per SM whatever they are, so that at 32 registers the loads in flight cover the latency of memory
// (4096 rows of 100003, 8 alternatives, us, with 2048 / 1536 / 1024 threads: fp32 290 / 310 / 293, bf16 184 / 191 / 221).
template <typename T, bool TOP, int kThreads>
__global__ void __launch_bounds__(kThreads, 2048 / kThreads) logprobs_kernel(const Args a) {
  constexpr int N = Vec<T>::n, kWarps = kThreads / 32, kGroups = kThreads / 4, kList = kWarps * kMaxK > kMaxCand ? kWarps * kMaxK : kMaxCand;
  __shared__ Stat stats[kWarps];
  __shared__ Stat cta;                             // of this CTA's part, read by the row's first CTA
  __shared__ alignas(16) float group_top[kGroups];
  __shared__ float limit;
  __shared__ int n_cand, n_groups;
  __shared__ unsigned char group_list[kGroups];
  __shared__ unsigned long long cand[TOP ? kList : 1];
  __shared__ unsigned long long best[TOP ? kMaxK : 1], all_best[TOP ? kMaxRanks * kMaxK : 1];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  uint32_t rank, ranks;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(ranks));
  const int row = blockIdx.x / ranks;
  const float c = a.scale * 1.4426950408889634f;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const T* z = static_cast<const T*>(a.logits) + (long long)row * a.stride;
  // values in front of the first 16-byte boundary, whole vectors, values behind the last
  const int head = min(a.V, (int)((16 - (reinterpret_cast<uintptr_t>(z) & 15)) & 15) / (int)sizeof(T));
  const int vecs = (a.V - head) / N, tail = a.V - head - vecs * N;
  const uint4* zv = reinterpret_cast<const uint4*>(z + head);
  const int first = (int)((long long)vecs * rank / ranks), last = (int)((long long)vecs * (rank + 1) / ranks);
  Stat st{kLowest, 0.f, 0.f};
  int i = first + tid;
  for (; i + 3 * kThreads < last; i += 4 * kThreads) {
    uint4 w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = __ldg(zv + i + e * kThreads);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float v[N];
      Vec<T>::unpack(w[e], v);
      take(st, v, c);
    }
  }
  if (i < last) {  // up to three more, loaded side by side
    uint4 w[3];
#pragma unroll
    for (int e = 0; e < 3; ++e)
      if (i + e * kThreads < last) w[e] = __ldg(zv + i + e * kThreads);
#pragma unroll
    for (int e = 0; e < 3; ++e) {
      if (i + e * kThreads >= last) break;
      float v[N];
      Vec<T>::unpack(w[e], v);
      take(st, v, c);
    }
  }
  // one value more for a few threads of the first CTA
  const int extra = rank != 0 ? -1 : tid < head ? tid : tid >= 8 && tid - 8 < tail ? head + vecs * N + tid - 8 : -1;
  float extra_z = 0.f;
  float seen = st.s > 0.f ? st.x : -INFINITY;  // largest of the vectors
  const bool odd = st.s != st.s;               // some are NaN or +infinity: x may be none of the values
  if (extra >= 0) {
    const float v[1] = {extra_z = Vec<T>::one(z + extra)};
    take(st, v, c);
  }
  // ---- statistics
  Stat w = st;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
    w = join(w, Stat{__shfl_xor_sync(0xffffffffu, w.x, o), __shfl_xor_sync(0xffffffffu, w.s, o), __shfl_xor_sync(0xffffffffu, w.t, o)}, c);
  if (lane == 0) stats[warp] = w;
  if (TOP) {
    // the extra values count for their groups here, and are looked at by their threads below
    float g = extra >= 0 ? fmaxf(seen, extra_z) : seen;
    g = fmaxf(g, __shfl_xor_sync(0xffffffffu, g, 1));
    g = fmaxf(g, __shfl_xor_sync(0xffffffffu, g, 2));
    if ((tid & 3) == 0) group_top[tid >> 2] = g;
    if (tid < kMaxK) best[tid] = 0;
    if (tid == 0) n_cand = n_groups = 0;
  }
  const bool any_odd = TOP ? __syncthreads_or(odd) != 0 : (__syncthreads(), false);
  if (tid < 32) {
    Stat r = stats[lane & (kWarps - 1)];
#pragma unroll
    for (int o = kWarps / 2; o > 0; o >>= 1)
      r = join(r, Stat{__shfl_xor_sync(0xffffffffu, r.x, o), __shfl_xor_sync(0xffffffffu, r.s, o), __shfl_xor_sync(0xffffffffu, r.t, o)}, c);
    if (lane == 0) cta = r;
  }
  if (TOP) {
    {  // rank of every group's maximum among all: a quarter of the comparisons a thread
      const int mine_at = tid >> 2;
      const float mine = group_top[mine_at];
      int above = 0;
#pragma unroll
      for (int g = 0; g < kGroups / 16; ++g) {
        const int at = (g * 4 + (tid & 3)) * 4;
        const float4 o = *reinterpret_cast<const float4*>(group_top + at);
        above += (o.x > mine || (o.x == mine && at < mine_at)) + (o.y > mine || (o.y == mine && at + 1 < mine_at)) + (o.z > mine || (o.z == mine && at + 2 < mine_at)) +
                 (o.w > mine || (o.w == mine && at + 3 < mine_at));
      }
      above += __shfl_xor_sync(0xffffffffu, above, 1);
      above += __shfl_xor_sync(0xffffffffu, above, 2);
      if (above == a.k - 1 && (tid & 3) == 0) limit = mine;
    }
    __syncthreads();
    const float lim = any_odd ? -INFINITY : limit;  // then every group is read again
    if (tid < kGroups && (any_odd || group_top[tid] >= lim)) group_list[atomicAdd(&n_groups, 1)] = (unsigned char)tid;
    __syncthreads();
    const int groups = n_groups, rounds = (last - first + kThreads - 1) / kThreads;
    // every vector of a group: 4 of them side by side, then kThreads further on
    auto for_each = [&](auto&& use) {
      for (int g = warp; g < groups; g += kWarps) {
        const int base = first + 4 * group_list[g];
        for (int r0 = 0; r0 < rounds; r0 += 16) {
          uint4 w[2];
#pragma unroll
          for (int z = 0; z < 2; ++z) {
            const int at = base + (r0 + z * 8 + (lane >> 2)) * kThreads + (lane & 3);
            w[z] = at < last ? __ldg(zv + at) : make_uint4(0u, 0u, 0u, 0u);
          }
#pragma unroll
          for (int z = 0; z < 2; ++z) {
            const int at = base + (r0 + z * 8 + (lane >> 2)) * kThreads + (lane & 3);
            if (r0 + z * 8 >= rounds) break;
            float v[N];
            Vec<T>::unpack(w[z], v);
#pragma unroll
            for (int e = 0; e < N; ++e) use(at < last, v[e], head + at * N + e);
          }
        }
      }
      if (warp == 0) use(extra >= 0, extra_z, extra);  // the threads with an extra value are of the first warp
    };
    for_each([&](bool on, float v, int id) {
      if (on && v >= lim) {
        const int at = atomicAdd(&n_cand, 1);
        if (at < kMaxCand) cand[at] = key_of(v, id);
      }
    });
    __syncthreads();
    int count = n_cand;
    if (count > kMaxCand) {  // many equal values: a sorted list per warp
      __syncthreads();
      unsigned long long mine = 0;
      for_each([&](bool on, float v, int id) {
        const unsigned long long key = on && v >= lim ? key_of(v, id) : 0;
        unsigned todo = __ballot_sync(0xffffffffu, key > __shfl_sync(0xffffffffu, mine, a.k - 1));
        for (; todo; todo &= todo - 1) {
          const unsigned long long k = __shfl_sync(0xffffffffu, key, __ffs(todo) - 1);
          if (k > __shfl_sync(0xffffffffu, mine, a.k - 1)) insert(mine, k, lane);
        }
      });
      cand[warp * kMaxK + lane] = lane < a.k ? mine : 0;
      count = kWarps * kMaxK;  // (never more than the threads)
      __syncthreads();
    }
    for (int i = tid; i < count; i += kThreads) {
      const unsigned long long mine = cand[i];
      int above = 0;
#pragma unroll 4
      for (int g = 0; g < count; ++g) above += cand[g] > mine;
      if (mine && above < a.k) best[above] = mine;
    }
  }
  // ---- the row
  // the first given token of a thread is on its way while the parts wait for each other
  int id = -1;
  float id_z = 0.f;
  if (rank == 0 && tid < a.m) {
    id = a.ids[(long long)row * a.m + tid];
    if (id >= 0 && id < a.V) id_z = Vec<T>::one(z + id);
  }
  if (ranks > 1) {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
  } else {
    __syncthreads();
  }
  if (rank == 0) {
    Stat r = cta;
    unsigned long long key = 0;  // a clustered row has no more keys than threads
    if (ranks > 1) {
      if (TOP && tid < ranks * kMaxK) {
        uint32_t at;
        asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"((uint32_t)__cvta_generic_to_shared(&best[tid % kMaxK])), "r"(tid / kMaxK));
        asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(key) : "r"(at));
      }
      r = Stat{kLowest, 0.f, 0.f};
      if ((lane & 7) < ranks) {  // a lane takes a part, then they join
        uint32_t at;
        asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"((uint32_t)__cvta_generic_to_shared(&cta)), "r"(lane & 7));
        asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(r.x) : "r"(at));
        asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(r.s) : "r"(at + 4));
        asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(r.t) : "r"(at + 8));
      }
#pragma unroll
      for (int o = 4; o > 0; o >>= 1)
        r = join(r, Stat{__shfl_xor_sync(0xffffffffu, r.x, o), __shfl_xor_sync(0xffffffffu, r.s, o), __shfl_xor_sync(0xffffffffu, r.t, o)}, c);
    }
    // nothing but -infinity: no distribution
    const bool none = r.s == 0.f;
    const double log_s = none ? 0.0 : log((double)r.s);
    auto logprob = [&](float v) { return none ? __int_as_float(0x7fffffff) : (float)(((double)v - r.x) * a.scale - log_s); };
    if (tid == 0) {
      if (a.lse) a.lse[row] = none ? -INFINITY : (float)((double)r.x * a.scale + log_s);
      if (a.entropy) a.entropy[row] = none ? __int_as_float(0x7fffffff) : (float)(log_s - 0.6931471805599453 * ((double)r.t / r.s));
    }
    if (a.logprobs) {
      for (int j = tid; j < a.m; j += kThreads) {
        if (j != tid) {
          id = a.ids[(long long)row * a.m + j];
          if (id >= 0 && id < a.V) id_z = Vec<T>::one(z + id);
        }
        a.logprobs[(long long)row * a.m + j] = id < 0 || id >= a.V ? -INFINITY : logprob(id_z);
      }
    }
    if (TOP) {
      auto put = [&](int at, unsigned long long key) {
        a.top_ids[(long long)row * a.k + at] = key ? (int)~(uint32_t)key : -1;
        if (a.top_logprobs) a.top_logprobs[(long long)row * a.k + at] = key ? logprob(key_value(key)) : __int_as_float(0x7fffffff);
      };
      if (ranks == 1) {
        if (tid < a.k) put(tid, best[tid]);
      } else {
        // the parts' lists are sorted: a key's rank is the sum of its places in them
        if (tid < kMaxRanks * kMaxK) all_best[tid] = key;
        const int any = __syncthreads_count(key != 0);  // keys that there are
        if (key) {
          const unsigned long long mine = key;
          int above = 0;
#pragma unroll
          for (uint32_t p = 0; p < kMaxRanks; ++p) {
            if (p >= ranks) break;
            int at = 0;  // keys of the list that are above
#pragma unroll
            for (int step = kMaxK / 2; step > 0; step /= 2)
              if (all_best[p * kMaxK + at + step - 1] > mine) at += step;
            if (all_best[p * kMaxK + at] > mine) ++at;
            above += at;
          }
          if (above < a.k) put(above, mine);
        }
        if (tid < a.k && tid >= any) put(tid, 0);  // fewer than k values that are numbers
      }
    }
  }
  if (ranks > 1) {
    __syncthreads();
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
  }
}

}  // namespace lp
}  // namespace moev
