// Attention of draft tokens over the paged 8-bit cache (kv_cache.cuh), on the fifth-generation tensor cores.
//
//   score[r, j] = scale * q_r . k_j over the context's keys (the last `window` positions of them) and
//   the draft's own ancestors and itself;  out_r = sum_j p[r, j] v_j,  p = softmax (with an optional
//   sink logit per head in the denominator),  lse_r = log of the denominator + maximum.
//
// Rows of a tile are (draft, query head of one kv head): the heads that share keys share their loads.  Both
// products have the cache as the A operand of tcgen05.mma (128 wide whatever the rows) and the rows as the narrow
// one, N = R = 16, 32, 64 or 128:
//   S^T [128 keys, R]  = K tile [128 keys, D] . Q^T          O^T [D, R] += V^T tile [D, 128 keys] . P^T
// K codes go from the cache by TMA to shared memory and from there to the multiplier as they are (a tile is 128 / page
// pages side by side); kind::f8f6f4 wants 8-bit operands on both sides, so q (bf16) is three e4m3 terms of q * 2^e, its
// largest element in [128, 256): each term takes the rest of the one before, what is left is 2^-18 of the row's largest
// element or 2^-12 of the element, whichever is more.  Up to R = 64 the terms stand side by side as 3 R columns, added as
// they are read: an instruction takes about 75 cycles however narrow it is; at R = 128 they add in one accumulator.
// The second product runs in kind::f16: V codes, exact in f16, are widened on their way into tensor memory, which
// holds the A operand (16 KB of codes per tile, whatever R).  In 8 bits p would need two terms and leave the reference below
// 3 bits of room.  The scale of a page's K multiplies its scores, that of its V the probabilities, in binary32, and their
// product is rounded once to f16 (2^-11; 2^-25 in units in which a row's largest is 2^3 or more).
//
// In S^T a thread is a key (one page, one scale) and its registers are rows, so a maximum over keys would go across
// lanes.  It is not taken: the reference m_r of p = 2^(s - m_r) only has to keep p * (V scale) near the top of f16, so it
// follows the largest s + log2(V scale) among the keys that the row sees and whose V is not all zero: a page with a large scale
// that a row does not see, gives no weight or that holds zeros takes no digits from the others.  Only when a product would
// exceed 2^15.9 (in the first tile, then hardly ever) the rows' four warps take the maxima, move m_r and rescale O and the
// denominators.  Those are binary32, of p itself, per thread, summed across lanes once at the end.
//
// Roles: one warp loads (TMA), one thread issues the MMAs, groups of four warps do the softmax of a share of the rows each
// (tensor memory gives a warp a quarter of the lanes) and widen V.  S is double-buffered: S of tile i + 1 is computed
// while the softmax works on tile i, the second product of tile i while it works on tile i + 1.
// Work split: all tiles of the call in one line (sequence, kv head, tile of rows, tile of keys), cut into equal
// runs, one per CTA that the machine holds.  A run may end one (sequence, head, rows) segment, cover others and begin the
// next: every CTA works equally long whatever the lengths, and sets up once or a few times.  A segment that lies in one run is
// finished there; the others' parts meet in a second kernel (attend_combine), in order.  The lengths are device data,
// so every CTA finds its run itself.  Segments of a few tiles (a window) are dealt out whole, without a second kernel.
// Every wait is bounded.
//
// Bound, as measured on B200 (us; bytes at 6.5 TB/s and operations at 1.67 PFLOP/s allow the time in brackets): one draft, 16
// rows, 4096 keys 13 (0.7): two launches, set-up, one tile and the join, each a chain of trips to memory; 64 drafts x 16
// heads over 16 000 keys 130 (20): 28 tiles of 128 x 128 a CTA at 6 300 cycles each (90 us; the softmax warps' instructions, the
// tensor core needs 1 800) and 40 us for the set-up of one or two pieces and the join; 32 ragged sequences up to 24 000 keys,
// 32 rows 206 (121): 81 tiles of 32 KB on either of an SM's two CTAs at 3 250 cycles (134 us, 56 % of the issue slots) and 70 us
// for set-up and join; window of 128, 64 rows, 16 sequences 17 (0.5): three masked tiles a CTA.  The same work on mma.sync
// with the rows as the wide operand took 187 and 333 us for the second and third.
#pragma once
#include <cuda.h>

#include "kv_cache.cuh"
#include "ptx.cuh"

namespace moev {
namespace att {

using kv::Cache;
using kv::Drafts;
using kv::Seq;

constexpr int kKeys = 128;                 // keys of a tile
// Powers of two: what p * (V scale) may reach in f16, and what its largest is brought to when the references move.  V scales are
// relative to a unit, the largest of the first tile, so that p stays in binary32's range: a scale beyond kUnitUp times
// that becomes the new unit, one below 2^kSlight counts as that for the references, and so does a key without values.
constexpr float kLimit = 15.9f, kTop = 3.f, kSlight = -48.f, kUnitUp = 0x1p64f;
constexpr float kUnseen = -3.0e38f;        // reference of a row that has not seen a key yet
constexpr unsigned long long kBudgetNs = kDeviceWaitBudgetNs;  // per wait; test builds can make the last V tile stay out

struct Args {
  Drafts d;
  Cache c;
  const __nv_bfloat16* q;
  __nv_bfloat16* out;
  float* lse;          // [n_tokens, n_heads] or null
  const float* sinks;  // [n_heads] or null
  int2* table;         // [n_seq + 1]: units and segments of the call before a sequence (written by the first CTA)
  float2* part_ml;     // [slots][R]: maximum (base 2), denominator; slot = CTA + segment
  float* part_o;       // [slots][R][D]
  long long q_stride, out_stride;
  int n_heads, rep, window, whole, grid;  // whole: a segment is one unit of work, not split
  float scale_log2;
  int32_t* ctx_status;  // status word of the context that the call belongs to, or null
};

__device__ __forceinline__ float exp2_fast(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float log2_fast(float x) {  // -inf for 0
  float r;
  asm("lg2.approx.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
// Two values as f16, at most the largest finite one (a key whose V is zero may be beyond that).
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.satfinite.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
// Reduces N values (a power of two up to 32) over the warp's lanes: every exchange halves the values a lane holds, N - 1
// shuffles and a few instead of 5 N.  The lane ends up with value `reduced_index`.
template <int N, bool MAX>
__device__ __forceinline__ float warp_reduce(float (&v)[N], int lane) {
  int o = 16;
#pragma unroll
  for (int h = N / 2; h >= 1; h /= 2, o /= 2) {
    const bool up = lane & o;
#pragma unroll
    for (int i = 0; i < h; ++i) {
      const float keep = up ? v[i + h] : v[i], give = up ? v[i] : v[i + h];
      const float got = __shfl_xor_sync(0xffffffffu, give, o);
      v[i] = MAX ? fmaxf(keep, got) : keep + got;
    }
  }
  for (; o >= 1; o /= 2) {
    const float got = __shfl_xor_sync(0xffffffffu, v[0], o);
    v[0] = MAX ? fmaxf(v[0], got) : v[0] + got;
  }
  return v[0];
}
template <int N>
__device__ __forceinline__ int reduced_index(int lane) {
  int r = 0, o = 16;
#pragma unroll
  for (int h = N / 2; h >= 1; h /= 2, o /= 2) r += lane & o ? h : 0;
  return r;
}
__device__ __forceinline__ bool any_of(bool v, int barrier, int threads) {
  int r;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %1, 0;\n\tbar.red.or.pred q, %2, %3, p;\n\tselp.b32 %0, 1, 0, q;\n\t}"
      : "=r"(r)
      : "r"((int)v), "r"(barrier), "r"(threads)
      : "memory");
  return r != 0;
}
// two binary32 operations in one instruction
__device__ __forceinline__ void mul2(float& a, float& b, float c) {
  asm("{\n\t.reg .b64 x, y;\n\tmov.b64 x, {%0, %1};\n\tmov.b64 y, {%2, %2};\n\tmul.rn.f32x2 x, x, y;\n\tmov.b64 {%0, %1}, x;\n\t}"
      : "+f"(a), "+f"(b)
      : "f"(c));
}
__device__ __forceinline__ void fma2(float& a, float& b, float m0, float m1, float c0, float c1) {  // a = a * m0 + c0, b = b * m1 + c1
  asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%0, %1};\n\tmov.b64 y, {%2, %3};\n\tmov.b64 z, {%4, %5};\n\t"
      "fma.rn.f32x2 x, x, y, z;\n\tmov.b64 {%0, %1}, x;\n\t}"
      : "+f"(a), "+f"(b)
      : "f"(m0), "f"(m1), "f"(c0), "f"(c1));
}
__device__ __forceinline__ void add2(float& a, float& b, float c, float d) {
  asm("{\n\t.reg .b64 x, y;\n\tmov.b64 x, {%0, %1};\n\tmov.b64 y, {%2, %3};\n\tadd.rn.f32x2 x, x, y;\n\tmov.b64 {%0, %1}, x;\n\t}"
      : "+f"(a), "+f"(b)
      : "f"(c), "f"(d));
}
__device__ __forceinline__ void tmem_ld8(uint32_t taddr, uint32_t (&r)[8]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "r"(taddr)
               : "memory");
}
__device__ __forceinline__ void tmem_st8(uint32_t taddr, const uint32_t (&r)[8]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%8], {%0,%1,%2,%3,%4,%5,%6,%7};" ::"r"(r[0]), "r"(r[1]), "r"(r[2]),
               "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(taddr)
               : "memory");
}
__device__ __forceinline__ void tmem_st(uint32_t taddr, const uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};" ::"r"(r[0]),
      "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]),
      "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]),
      "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]), "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tmem_st(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};" ::"r"(r[0]),
      "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]),
      "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// D[tmem] (+)= A[tmem] * B[smem desc], f16: a column of A holds two consecutive k of its lane's row
__device__ __forceinline__ void mma_f16_ta(uint32_t d_tmem, uint32_t a_tmem, uint32_t b_lo, uint32_t desc_hi, uint32_t idesc,
                                           uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      ".reg .b64 db;\n\tmov.b64 db, {%2, %5};\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %3, p;\n\t}" ::"r"(d_tmem),
      "r"(a_tmem), "r"(b_lo), "r"(idesc), "r"(accumulate), "r"(desc_hi)
      : "memory");
}
__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(ptx::smem_u32(dst)), "l"(src),
               "r"(bytes), "r"(ptx::smem_u32(bar))
               : "memory");
}
// four e4m3 codes -> two f16 pairs
__device__ __forceinline__ void codes_to_f16(uint32_t w, uint32_t& lo, uint32_t& hi) {
  asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}"
      : "=r"(lo), "=r"(hi)
      : "r"(w));
}

// First key of the range that a sequence's drafts can see (a multiple of 128).
__device__ __forceinline__ int range_start(const Seq& s, int window) {
  return window > 0 ? max(0, s.ctx + 1 - window) & ~(kKeys - 1) : 0;
}

// Byte of 16-byte piece `seg` (16 keys) of dimension d in a V tile: pages side by side, each [D][page] with the swizzle
// of its row length (128, 64 or 32 bytes; none for 16).
template <int D>
__device__ __forceinline__ uint32_t v_piece(int d, int seg, int page_log2) {
  if (page_log2 == 7) return d * 128 + ((seg ^ (d & 7)) << 4);
  if (page_log2 == 6) return (seg >> 2) * (D * 64) + d * 64 + (((seg & 3) ^ ((d >> 1) & 3)) << 4);
  if (page_log2 == 5) return (seg >> 1) * (D * 32) + d * 32 + (((seg & 1) ^ ((d >> 2) & 1)) << 4);
  return seg * (D * 16) + d * 16;
}
// Byte of element (row, d) of a K-major operand with rows of D bytes in the swizzle of that length.
template <int D>
__device__ __forceinline__ uint32_t q_byte(int r, int d) {
  return D == 128 ? r * 128 + (((d >> 4) ^ (r & 7)) << 4) + (d & 15) : r * 64 + (((d >> 4) ^ ((r >> 1) & 3)) << 4) + (d & 15);
}
// Halves of a shared-memory matrix descriptor (K-major, swizzled): address and leading offset | stride between groups of
// 8 rows, version, layout.  A step along K or to another tile is an addition to the lower half.
__device__ __forceinline__ uint32_t desc_lo(uint32_t addr) { return ((addr & 0x3FFFFu) >> 4) | (1u << 16); }
__host__ __device__ constexpr uint32_t desc_hi(uint32_t stride, uint32_t layout) { return (stride >> 4) | (1u << 14) | (layout << 29); }
constexpr uint32_t kSw128 = 2, kSw64 = 4, kSw32 = 6;

// What a sequence brings: tiles of rows and tiles of keys; none without drafts.
struct Extent {
  int row_tiles, key_tiles;
};
__device__ __forceinline__ Extent extent(const Args& a, const Seq& s, int R) {
  Extent e{0, 0};
  if (s.n > 0) {
    e.row_tiles = (s.n * a.rep + R - 1) / R;
    e.key_tiles = (s.ctx + s.n - range_start(s, a.window) + kKeys - 1) / kKeys;
  }
  return e;
}
__device__ __forceinline__ int units_per_cta(int total, int grid) { return max(1, (int)(((unsigned)total + grid - 1) / (unsigned)grid)); }

template <int D, int R>
struct Cfg {
  static constexpr int kCtas = R <= 32 ? 2 : 1;  // per SM
  // groups of 4 softmax warps, each with its share of the rows: 16 or 20 warps per SM, since a warp alone issues an
  // instruction every eight cycles only
  static constexpr int kGroups = R <= 32 ? 2 : 4;
  static constexpr int kThreads = 32 * (4 * kGroups + 2);  // + loader, MMA issuer
  static constexpr int kTile = kKeys * D;        // bytes of a K or V tile
  static constexpr int kKStages = R <= 32 && D == 128 ? 2 : 3, kVStages = 3;
  // scores: columns of a tile, buffers (where two CTAs share the SM, the other one's work covers for the second)
  static constexpr int kSCols = R <= 64 ? 3 * R : R, kSBufs = R <= 32 ? 1 : 2;
  static constexpr int kPBufs = R == 128 ? 2 : 1;
  static constexpr int kChunk = R / kGroups < 16 ? R / kGroups : 16;  // rows that a thread works on at a time
  // P^T is kept [key][row] (rows contiguous: a thread stores its key's rows by 16 bytes): blocks of up to 64 rows, a key's
  // row in the swizzle of its length
  static constexpr int kPRow = R >= 64 ? 128 : 2 * R, kPBlock = kKeys * kPRow, kP = R * kKeys * 2;
  static constexpr int kQ = R * D;
  static constexpr int kO = kSBufs * kSCols, kV16 = kO + R;  // columns: S, O, the widened V tile (64)
  static constexpr int kTmem = R == 16 ? 128 : R == 32 ? 256 : 512;
  static_assert(kV16 + 64 <= kTmem, "tensor memory");
  // byte offsets
  static constexpr int oK = 0, oV = kKStages * kTile, oP = oV + kVStages * kTile, oQ = oP + kPBufs * kP, oCtl = oQ + 3 * kQ;
};

template <int R>
struct Ctl {
  uint64_t k_full[3], k_empty[3], v_full[3], v_empty[3];
  uint64_t s_full[2], s_empty[2], p_full, o_full, q_full, drain;
  alignas(16) float rcm[R / 2][4];  // per two rows: factors from raw scores to powers of two | minus the references m
  float fac_l[R], fac_o[R];     // what moving a reference multiplies; in the end fac_l: the row's accumulators
  float peak[R];                // largest reference so far
  float wmax[4][R], lsum[4][R];
  // by quarter of the dimensions and 32 words per group: byte k of word w is not zero where some V code of key 4 w + k is not.
  // With 128 rows a group's words take the place of its own lsum, which is written after the last tile
  uint32_t valued[R == 128 ? 1 : 4 * 128];
  alignas(16) float ks[3][8], vs[3][8];  // by V stage: scales of a tile's 16-key pieces
  alignas(16) int pid[3][8];             // and their pages
  uint32_t vis[2][R][4];        // by tile parity: draft of the tile sees key (bits)
  uint32_t nan_row[R][4];       // row's output is NaN in these dimensions
  int low[R], top[R];           // by draft of the tile: context keys > low are seen; a chain sees keys <= top
  int2 row[R];                  // token row, query head; -1: no row
  int scan[2][20];              // sums of the warps' sequences: units, segments
  int at_units, at_segs;        // before the sequence in which this CTA's run begins ...
  int at_seq;                   // ... and that sequence
  Seq at;
  float vmax[3];                // by V stage: largest V scale of the tile ...
  int all_there[3];             // ... and whether each of its keys has a page
  int any_nan;                  // some entry of nan_row is not zero
  uint32_t tmem;
  volatile int abort;
  volatile uint32_t k_it, v_it;  // tiles the loader armed (read on the abort path)
};
template <int D, int R>
size_t smem_bytes(int words, bool tree) {  // + ancestor words of the tile's drafts, parents of the sequence
  return 1024 + Cfg<D, R>::oCtl + sizeof(Ctl<R>) + (tree ? (size_t)R * words * 4 + (size_t)words * 128 : 0);
}

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

// The same for a whole warp: one lane looks.
__device__ __forceinline__ bool wait_warp(uint64_t* bar, uint32_t parity, volatile int* abort_flag, int32_t* status, int lane) {
  int r = 1;
  if (lane == 0) r = wait(bar, parity, abort_flag, status);
  return __shfl_sync(0xffffffffu, r, 0) != 0;
}

template <int D, int R>
__global__ void __launch_bounds__(Cfg<D, R>::kThreads, Cfg<D, R>::kCtas) attend_kernel(const Args a, const __grid_constant__ CUtensorMap tm_k,
                                                                            const __grid_constant__ CUtensorMap tm_v) {
  using C = Cfg<D, R>;
  constexpr int KS = C::kKStages, VS = C::kVStages, SB = C::kSBufs, G = C::kGroups, RH = R / G, RC = C::kChunk, NS = 128 * G;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  Ctl<R>& S = *reinterpret_cast<Ctl<R>*>(smem + C::oCtl);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    for (int i = 0; i < KS; ++i) {
      ptx::mbar_init(&S.k_full[i], 1);
      ptx::mbar_init(&S.k_empty[i], 1);
    }
    for (int i = 0; i < VS; ++i) {
      ptx::mbar_init(&S.v_full[i], 1);
      ptx::mbar_init(&S.v_empty[i], 4 * G);
    }
    for (int i = 0; i < 2; ++i) {
      ptx::mbar_init(&S.s_full[i], 1);
      ptx::mbar_init(&S.s_empty[i], 4 * G);
    }
    ptx::mbar_init(&S.p_full, 4 * G);
    ptx::mbar_init(&S.o_full, 1);
    ptx::mbar_init(&S.q_full, 1);
    ptx::mbar_init(&S.drain, 1);
    ptx::fence_mbar_init();
    S.abort = 0;
    S.k_it = S.v_it = 0;
  }
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int page_log2 = a.c.page_log2, page = 1 << page_log2;
  const bool tree = a.d.parent != nullptr;
  // ---- this CTA's run of units
  int run, run_end, seq_units, seq_segs;  // position, end; units and segments before sequence b
  int b;
  Seq s;
  {
    constexpr int kWarps = C::kThreads / 32;
    const bool few = a.d.n_seq <= 32;  // every warp then finds the same for itself, a sequence a lane
    const int each = few ? 1 : (a.d.n_seq + C::kThreads - 1) / C::kThreads, first = few ? lane : tid * each, last = min(a.d.n_seq, first + each);
    auto weigh = [&](const Seq& q, int& units, int& segs) {
      const Extent e = extent(a, q, R);
      segs = e.row_tiles * a.c.heads;
      units = a.whole ? segs : segs * e.key_tiles;
    };
    int un = 0, sg = 0;
    Seq q{0, 0, 0};
    for (int i = first; i < last; ++i) {
      int u, g;
      q = kv::sequence(a.d, i, page);
      weigh(q, u, g);
      un += u;
      sg += g;
    }
    int iu = un, is = sg;  // inclusive sums over the threads
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
      const int u1 = __shfl_up_sync(0xffffffffu, iu, o), s1 = __shfl_up_sync(0xffffffffu, is, o);
      if (lane >= o) { iu += u1; is += s1; }
    }
    int total = 0, segs = 0, eu = iu - un, es = is - sg;  // eu, es: before this thread's sequences
    if (few) {
      total = __shfl_sync(0xffffffffu, iu, 31);
      segs = __shfl_sync(0xffffffffu, is, 31);
    } else {
      if (lane == 31) { S.scan[0][warp] = iu; S.scan[1][warp] = is; }
      __syncthreads();
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        if (w == warp) { eu += total; es += segs; }
        total += S.scan[0][w];
        segs += S.scan[1][w];
      }
    }
    const int per = units_per_cta(total, a.grid);
    run = (int)min((long long)per * blockIdx.x, (long long)total);
    run_end = min(run + per, total);
    const bool tell = blockIdx.x == 0 && !a.whole && (!few || warp == 0), mine = run >= eu && run < eu + un;
    if (tell || mine)
      for (int i = first; i < last; ++i) {
        int u, g;
        if (each > 1) q = kv::sequence(a.d, i, page);
        weigh(q, u, g);
        if (tell) a.table[i] = make_int2(eu, es);
        if (mine && run >= eu && run < eu + u) {
          S.at_units = eu;
          S.at_segs = es;
          S.at_seq = i;
          S.at = q;
        }
        eu += u;
        es += g;
      }
    if (tell && tid == 0) a.table[a.d.n_seq] = make_int2(total, segs);
    if (run >= run_end) return;  // the same for the whole CTA
  }
  // Tensor memory is taken behind the wait and dependents are released behind that: no kernel holds tensor memory while
  // it waits for one that still has to take it.
  if (warp == 4 * G + 1) {
    ptx::tmem_alloc(&S.tmem, C::kTmem);
    ptx::tmem_relinquish();
  }
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const uint32_t tmem = S.tmem;
  b = S.at_seq;
  s = S.at;
  seq_units = S.at_units;
  seq_segs = S.at_segs;

  int gt = 0;  // tiles this CTA has been through: the barriers count on
  for (int piece = 0; run < run_end; ++piece) {
    Extent ext = extent(a, s, R);
    const int in_seq = run - seq_units;
    const int unit_tiles = a.whole ? 1 : ext.key_tiles;
    const int seg_in_seq = in_seq / unit_tiles, first_tile = a.whole ? 0 : in_seq - seg_in_seq * unit_tiles;
    const int head = seg_in_seq / ext.row_tiles, row0 = (seg_in_seq - head * ext.row_tiles) * R;
    const int all_tiles = ext.key_tiles, piece_tiles = a.whole ? all_tiles : min(all_tiles - first_tile, run_end - run);
    const bool split = piece_tiles < all_tiles;
    const int slot = blockIdx.x + seq_segs + seg_in_seq;
    const int n_rows = s.n * a.rep;
    const int k_begin = range_start(s, a.window) + first_tile * kKeys, k_all = s.ctx + s.n;
    const int i_first = row0 / a.rep, i_last = min(n_rows - 1, row0 + R - 1) / a.rep;
    int k_end = min(k_begin + piece_tiles * kKeys, k_all);
    if (!tree) k_end = min(k_end, s.ctx + i_last + 1);  // a chain: nobody here sees later drafts
    const int n_tiles = k_end > k_begin ? (k_end - k_begin + kKeys - 1) / kKeys : 0;
    const int low_max = a.window > 0 ? s.ctx + s.n - 1 - a.window : -1;
    const int words = tree ? (a.d.max_drafts + 31) >> 5 : 0;

    if (warp == 4 * G) {
      // ------------------------------------------------------------ loader
      asm volatile("fence.proxy.async;" ::: "memory");  // the cache was written by ordinary stores of earlier kernels
      if (lane == 0) {
        ptx::prefetch_tmap(&tm_k);
        ptx::prefetch_tmap(&tm_v);
      }
      const int pages = kKeys >> page_log2, seg = lane & 7;
      const int seen_from = a.window > 0 ? s.ctx + 1 - a.window : 0;  // a page that ends before that may be gone: it is not looked up
      auto page_at = [&](int it) {
        const int key = k_begin + it * kKeys + 16 * seg;
        return it < n_tiles && key < k_all && (key | (page - 1)) >= seen_from ? kv::page_of(a.d, a.c, b, key >> page_log2) : -1;
      };
      // page ids two tiles ahead, scales one: each is a trip to memory that the copies do not wait for
      auto scale_at = [&](int p, float& k, float& v) {
        const long long at = (long long)max(p, 0) * a.c.heads + head;
        k = p >= 0 ? a.c.ks[at] : 0.f;
        v = p >= 0 ? a.c.vs[at] : 0.f;
      };
      int pid = page_at(0), pid1 = page_at(1);
      float ks, vs;
      scale_at(pid, ks, vs);
      for (int it = 0; it < n_tiles; ++it) {
        const int ct = gt + it, sk = ct % KS, sv = ct % VS;
        const int pid2 = page_at(it + 2);
        float ks1, vs1;
        scale_at(pid1, ks1, vs1);
        const int mine = __shfl_sync(0xffffffffu, pid, ((lane & 7) << page_log2) >> 4 & 7);  // page `lane` of the tile
        const bool on = lane < pages && mine >= 0;
        const uint32_t bytes = __popc(__ballot_sync(0xffffffffu, on)) * page * D;
        if (ct >= KS && !wait_warp(&S.k_empty[sk], ((ct / KS) & 1) ^ 1, &S.abort, a.d.status, lane)) break;
        uint8_t* dst = smem + C::oK + sk * C::kTile + (lane & 7) * page * D;
        if (lane == 0) {
          ptx::mbar_arrive_expect_tx(&S.k_full[sk], bytes);
          S.k_it = ct + 1;
        }
        __syncwarp();
        if (on) ptx::tma_load_2d(dst, &tm_k, &S.k_full[sk], 0, (mine * a.c.heads + head) << page_log2, ptx::kPolicyEvictNormal);
        if (MOEV_TEST_WITHHOLD() && it == n_tiles - 1) break;
        if (ct >= VS && !wait_warp(&S.v_empty[sv], ((ct / VS) & 1) ^ 1, &S.abort, a.d.status, lane)) break;
        if (lane < 8) {
          S.ks[sv][lane] = ks;
          S.vs[sv][lane] = vs;
          S.pid[sv][lane] = pid;
        }
        float top = vs;  // lanes 0..7 hold the tile's pieces, and the others copies
#pragma unroll
        for (int o = 4; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        const bool there = __all_sync(0xffffffffu, pid >= 0);
        if (lane == 0) {
          S.vmax[sv] = top;
          S.all_there[sv] = there;
        }
        __syncwarp();
        if (lane == 0) {
          ptx::mbar_arrive_expect_tx(&S.v_full[sv], bytes);
          S.v_it = ct + 1;
        }
        __syncwarp();
        dst = smem + C::oV + sv * C::kTile + (lane & 7) * page * D;
        if (on) {
          if (page_log2 == 4) bulk_load(dst, a.c.v + ((long long)mine * a.c.heads + head) * (D * 16), D * 16, &S.v_full[sv]);
          else ptx::tma_load_2d(dst, &tm_v, &S.v_full[sv], 0, (mine * a.c.heads + head) * D, ptx::kPolicyEvictNormal);
        }
        pid = pid1;
        pid1 = pid2;
        ks = ks1;
        vs = vs1;
      }
    } else if (warp == 4 * G + 1) {
      // ------------------------------------------------------------ MMA issuer
      if (lane == 0) {
        const uint32_t sdesc = ptx::instr_desc(0, 0, C::kSCols);        // kind::f8f6f4: e4m3 x e4m3
        const uint32_t pdesc = ptx::instr_desc(0, 0, R) | (1u << 16);  // kind::f16: f16 x f16, B with its rows (N) contiguous
        // leading offset of P: from one block of 64 rows to the next
        const uint32_t kb = desc_lo(ptx::smem_u32(smem + C::oK)), pb = (desc_lo(ptx::smem_u32(smem + C::oP)) & 0xFFFFu) | (uint32_t)(C::kPBlock / 16) << 16, qb = desc_lo(ptx::smem_u32(smem + C::oQ));
        constexpr uint32_t kHi = desc_hi(8 * D, D == 128 ? kSw128 : kSw64), pHi = desc_hi(8 * C::kPRow, C::kPRow == 128 ? kSw128 : C::kPRow == 64 ? kSw64 : kSw32);
        bool ok = true;
        auto scores = [&](int it) {
          const int ct = gt + it, st = ct % KS, u = ct % SB;
          ok = ok && wait(&S.k_full[st], (ct / KS) & 1, &S.abort, a.d.status);
          if (ct >= SB) ok = ok && wait(&S.s_empty[u], ((ct / SB) & 1) ^ 1, &S.abort, a.d.status);
          if (!ok) return;
          ptx::tc_fence_after();
          const uint32_t ka = kb + st * (C::kTile / 16);
#pragma unroll
          for (int term = 0; term < (C::kSCols == R ? 3 : 1); ++term)
#pragma unroll
            for (int k = 0; k < D / 32; ++k)
              ptx::mma_f8f6f4_lohi(tmem + u * C::kSCols, ka + k * 2, qb + (term * C::kQ + k * 32) / 16, kHi, sdesc, term + k > 0);
          ptx::mma_commit(&S.k_empty[st]);
          ptx::mma_commit(&S.s_full[u]);
        };
        {
          ok = wait(&S.q_full, piece & 1, &S.abort, a.d.status);
          if (n_tiles > 0) scores(0);
        }
        for (int it = 0; it < n_tiles && ok; ++it) {
          if (it + 1 < n_tiles) scores(it + 1);
          ok = ok && wait(&S.p_full, (gt + it) & 1, &S.abort, a.d.status);
          if (!ok) break;
          ptx::tc_fence_after();
#pragma unroll
          for (int k = 0; k < kKeys / 16; ++k)
            mma_f16_ta(tmem + C::kO, tmem + C::kV16 + k * 8, pb + ((gt + it) % C::kPBufs) * (C::kP / 16) + k * C::kPRow, pHi, pdesc, it + k > 0);  // 16 keys on
          ptx::mma_commit(&S.o_full);
        }
        if (!ok) {  // abort: what was issued must have ended before tensor memory and shared memory are given back
          ptx::drain_issuer(&S.drain, kBudgetNs);
        }
      }
    } else {
      // ------------------------------------------------------------ softmax
      const int quad = warp & 3, group = warp >> 2, r0 = group * RH, key = quad * 32 + lane;
      uint32_t* anc = reinterpret_cast<uint32_t*>(smem + C::oCtl + sizeof(Ctl<R>));  // [R][words]
      int* par = reinterpret_cast<int*>(anc + R * words);
      if (tree) {
        for (int i = tid; i < s.n; i += NS) par[i] = kv::parent_of(a.d.parent + s.lo, i);
        for (int i = tid; i < R * words; i += NS) anc[i] = 0;
        ptx::named_barrier(2, NS);
      }
      if (tid <= i_last - i_first) {  // one thread per draft of the tile
        const int i = i_first + tid;
        int at = s.ctx + i;
        if (tree) {
          int n = 0;
          for (int j = i; j >= 0; j = par[j], ++n)  // parents come earlier: at most s.n steps
            if (a.window <= 0 || n < a.window) anc[tid * words + (j >> 5)] |= 1u << (j & 31);
          at = s.ctx + n - 1;
        }
        S.low[tid] = a.window > 0 ? at - a.window : -1;
        S.top[tid] = tree ? s.ctx - 1 : at;
      }
      for (int i = tid; i < R * 4; i += NS) (&S.nan_row[0][0])[i] = 0;
      if (tid == 0) S.any_nan = 0;
      // Q: a row's D elements by D / 8 neighbouring lanes, 8 each; all loads first
      constexpr int kPer = D / 8, kItems = R * kPer / NS > 0 ? R * kPer / NS : 1;
      uint4 raw[kItems];
#pragma unroll
      for (int k = 0; k < kItems; ++k) {
        const int z = k * NS + tid, rr = row0 + z / kPer;
        raw[k] = make_uint4(0, 0, 0, 0);
        if (z < R * kPer && rr < n_rows)
          raw[k] = *reinterpret_cast<const uint4*>(a.q + (long long)(s.lo + rr / a.rep) * a.q_stride + (long long)(head * a.rep + rr % a.rep) * D + (z % kPer) * 8);
      }
#pragma unroll
      for (int k = 0; k < kItems; ++k) {
        const int z = k * NS + tid, r = z / kPer, d0 = (z % kPer) * 8, rr = row0 + r;
        if (R * kPer < NS && z >= R * kPer) break;
        const bool live = rr < n_rows;
        const int i = rr / a.rep, hq = head * a.rep + rr % a.rep;
        const uint32_t u4[4] = {raw[k].x, raw[k].y, raw[k].z, raw[k].w};
        float v[8];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          v[2 * e] = __uint_as_float(u4[e] << 16);
          v[2 * e + 1] = __uint_as_float(u4[e] & 0xffff0000u);
        }
        float m = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) m = fmaxf(m, fabsf(v[e]));
        const uint32_t lanes = D == 128 ? 0xffffu << (lane & 16) : 0xffu << (lane & 24);
#pragma unroll
        for (int o = kPer / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(lanes, m, o));
        // 2^e <= m < 2^(e + 1), brought to [128, 256); a zero, infinite or NaN row as it is
        const int ex = (int)(__float_as_uint(m) >> 23) - 127;
        float up = 1.f, back = 1.f;
        if (ex >= -110 && ex < 128) {
          up = __uint_as_float((uint32_t)(127 + 7 - ex) << 23);
          back = __uint_as_float((uint32_t)(127 + ex - 7) << 23);
        }
        if ((z % kPer) == 0) {
          S.rcm[r / 2][r & 1] = a.scale_log2 * back;
          S.rcm[r / 2][2 + (r & 1)] = -kUnseen;
          S.peak[r] = kUnseen;
          S.row[r] = live ? make_int2(s.lo + i, hq) : make_int2(-1, 0);
        }
        if (ex == 128) {  // infinities become NaN: a row with one has NaN scores, as inf * 0 and inf - inf have it
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = fabsf(v[e]) == INFINITY ? __int_as_float(0x7fffffff) : v[e];
        }
        uint32_t code[3][2];
#pragma unroll
        for (int e = 0; e < 8; e += 2) mul2(v[e], v[e + 1], up);
#pragma unroll
        for (int term = 0; term < 3; ++term) {
          uint32_t c[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            c[e] = (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(v[2 * e], v[2 * e + 1]), __NV_SATFINITE, __NV_E4M3);
            const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)c[e], __NV_E4M3);
            const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
            add2(v[2 * e], v[2 * e + 1], -f.x, -f.y);
          }
          code[term][0] = c[0] | c[1] << 16;
          code[term][1] = c[2] | c[3] << 16;
        }
#pragma unroll
        for (int term = 0; term < 3; ++term)
          *reinterpret_cast<uint2*>(smem + C::oQ + term * C::kQ + q_byte<D>(r, d0)) = make_uint2(code[term][0], code[term][1]);
      }
      ptx::fence_proxy_async_smem();
      ptx::named_barrier(2, NS);
      if (tid == 0) ptx::mbar_arrive(&S.q_full);

      float l[RH];
#pragma unroll
      for (int r = 0; r < RH; ++r) l[r] = 0.f;
      float unit_of[RH / RC], inv_of[RH / RC];  // V scale that each part of the rows is in units of, its reciprocal
#pragma unroll
      for (int c = 0; c < RH / RC; ++c) unit_of[c] = inv_of[c] = 0.f;
      const uint32_t lane_base = (uint32_t)(quad * 32) << 16;
      // this key's row of P; 16-byte piece c of it is at c ^ p_xor
      uint8_t* const p_row0 = smem + C::oP + (r0 / 64) * C::kPBlock + key * C::kPRow;
      const int p_xor = C::kPRow == 128 ? key & 7 : C::kPRow == 64 ? (key >> 1) & 3 : (key >> 2) & 1;
      uint32_t(*const valued)[128] = reinterpret_cast<uint32_t(*)[128]>(R == 128 ? reinterpret_cast<uint32_t*>(S.lsum) : S.valued);
      uint32_t v_off[8 / G];
#pragma unroll
      for (int z = 0; z < 8 / G; ++z) v_off[z] = v_piece<D>(quad * 32 + lane, group * (8 / G) + z, page_log2);
      bool ok = true;
      for (int it = 0; it < n_tiles; ++it) {
        const int ct = gt + it, sv = ct % VS, bu = ct & 1;
        const int k0 = k_begin + it * kKeys;
        const bool masked = k0 + kKeys > s.ctx || k0 <= low_max;  // somebody may not see a key of the tile
        if (masked) {
          // what each draft of the tile sees of its keys.  Every group writes all of it (the same words), so that nobody waits
          // for another group here
          for (int z = quad * 32 + lane; z < (i_last - i_first + 1) * 4; z += 128) {
            const int dr = z >> 2, kb = k0 + (z & 3) * 32;
            const int from = max(0, S.low[dr] + 1 - kb), to = min(32, S.top[dr] + 1 - kb);
            uint32_t bits = to > from ? (0xffffffffu >> (32 - to)) & (0xffffffffu << from) : 0u;
            if (tree && kb + 32 > s.ctx && kb < k_all) {
              const int off = kb - s.ctx;  // draft of the word's first key, may be negative
              const uint32_t* an = anc + dr * words;
              if (off < 0) bits |= an[0] << -off;
              else bits |= __funnelshift_r(an[off >> 5], (off >> 5) + 1 < words ? an[(off >> 5) + 1] : 0u, off & 31);
            }
            S.vis[bu][dr][z & 3] = bits;
          }
          ptx::named_barrier(3 + group, 128);
        }
        ok = wait_warp(&S.v_full[sv], (ct / VS) & 1, &S.abort, a.d.status, lane) && ok;
        ok = wait_warp(&S.s_full[ct % SB], (ct / SB) & 1, &S.abort, a.d.status, lane) && ok;
        ptx::tc_fence_after();
        const float k_scale = S.ks[sv][key >> 4], v_scale = S.vs[sv][key >> 4];
        const bool there = S.pid[sv][key >> 4] >= 0;
        const float vm = S.vmax[sv];
        const bool plain = !masked && S.all_there[sv];  // every key is there and every row sees it
        const uint32_t s_at = tmem + lane_base + (ct % SB) * C::kSCols + r0;
        uint8_t* const p_row = p_row0 + (ct % C::kPBufs) * C::kP;
        bool leave = false, looked = false, zeros = false;
#pragma unroll
        for (int rc = 0; rc < RH; rc += RC) {  // RC of this thread's rows at a time
          float v[RC];
          auto load_scores = [&]() {  // times the page's scale; -inf where the row does not see this thread's key
            constexpr int kTerms = C::kSCols / R;
            float w[kTerms][RC];
#pragma unroll
            for (int term = 0; term < kTerms; ++term)
#pragma unroll
              for (int c = 0; c < RC / 8; ++c) tmem_ld8(s_at + term * R + rc + 8 * c, *reinterpret_cast<uint32_t(*)[8]>(&w[term][8 * c]));
            ptx::tmem_ld_wait();
#pragma unroll
            for (int r = 0; r < RC; r += 2) {
              v[r] = w[0][r];
              v[r + 1] = w[0][r + 1];
#pragma unroll
              for (int term = 1; term < kTerms; ++term) add2(v[r], v[r + 1], w[term][r], w[term][r + 1]);
            }
#pragma unroll
            for (int r = 0; r < RC; r += 2) mul2(v[r], v[r + 1], k_scale);
            if (masked) {
              int dr = (row0 + r0 + rc) / a.rep, in = row0 + r0 + rc - dr * a.rep;  // row's draft and its head
              dr -= i_first;
              uint32_t bits = S.vis[bu][min(dr, i_last - i_first)][quad];
#pragma unroll
              for (int r = 0; r < RC; ++r) {
                if (!((bits >> lane) & 1u)) v[r] = -INFINITY;
                if (++in == a.rep) {
                  in = 0;
                  ++dr;
                  bits = S.vis[bu][min(dr, i_last - i_first)][quad];
                }
              }
            }
            if (!there) {
#pragma unroll
              for (int r = 0; r < RC; ++r) v[r] = -INFINITY;
            }
          };
          load_scores();
          float& u = unit_of[rc / RC];
          const bool unit = vm > u * kUnitUp;  // the same in the group's threads
          bool move = it == 0;  // there is no reference yet
          if (it > 0) {
            const float lv = fmaxf(log2_fast(v_scale * inv_of[rc / RC]), kSlight);
            float tmax = ok ? -INFINITY : INFINITY;
#pragma unroll
            for (int r = 0; r < RC; r += 2) {
              const float4 q = *reinterpret_cast<const float4*>(&S.rcm[(r0 + rc + r) / 2][0]);
              fma2(v[r], v[r + 1], q.x, q.y, q.z, q.w);
              tmax = fmaxf(tmax, fmaxf(v[r], v[r + 1]));
            }
            move = any_of(tmax + lv > kLimit || unit, 3 + group, 128);
          }
          if (move) {
            const uint8_t* vt = smem + C::oV + sv * C::kTile;
            bool ask = !ok;
            if (!looked) {  // a key with a value in one of four dimensions is none of the zero ones
              uint32_t some = 0;
#pragma unroll
              for (int e = 0; e < 4; ++e) some |= vt[v_piece<D>(e * (D / 4) + 1, key >> 4, page_log2) + (key & 15)];
              ask = ask || (there && k0 + key < k_all && !(some & 0x7fu));
              looked = true;
            }
            if (any_of(ask, 3 + group, 128)) {
              if (any_of(!ok, 3 + group, 128)) {  // a warp that gave up stays with the others' barriers until here: all of them leave
                leave = true;
                break;
              }
              // which keys have values: a lane has a dimension, the warp's lanes are joined
              zeros = true;
              if (quad * 32 < D) {
                uint32_t mine = 0;
#pragma unroll 1
                for (int seg = 0; seg < 8; ++seg) {
                  const uint4 w = *reinterpret_cast<const uint4*>(vt + v_piece<D>(quad * 32 + lane, seg, page_log2));
                  const uint32_t ww[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                  for (int e = 0; e < 4; ++e) {
                    const uint32_t any = __reduce_or_sync(0xffffffffu, ww[e] & 0x7f7f7f7fu);
                    if (lane == 4 * seg + e) mine = any;
                  }
                }
                valued[quad][group * 32 + lane] = mine;
              }
              ptx::named_barrier(3 + group, 128);
            }
            // move the references to the maxima.  From the scores themselves: relative to the reference of a row that has seen
            // nothing they have lost their digits
            if (it > 0) load_scores();
            const float u_new = unit ? vm : u, inv = u_new > 0.f ? 1.f / u_new : 0.f;
            uint32_t values = zeros ? 0u : 0xffffffffu;
#pragma unroll 1
            for (int z = 0; zeros && z < D / 32; ++z) values |= valued[z][group * 32 + (key >> 2)];
            const float lv = (values >> (8 * (key & 3))) & 0xffu ? fmaxf(log2_fast(v_scale * inv), kSlight) : kSlight;
            float x[RC];
#pragma unroll
            for (int r = 0; r < RC; ++r) {
              v[r] *= S.rcm[(r0 + rc + r) / 2][r & 1];
              x[r] = v[r] + lv;
            }
            const float top = warp_reduce<RC, true>(x, lane);
            S.wmax[quad][r0 + rc + reduced_index<RC>(lane)] = top;
            ptx::named_barrier(3 + group, 128);
            if (quad == 0 && lane < RC) {
              const int r = r0 + rc + lane;
              const float old = -S.rcm[r / 2][2 + (r & 1)], peak = S.peak[r];
              const float turn = u > 0.f && unit ? log2_fast(u) - log2_fast(u_new) : 0.f;  // what is there, in the new unit
              // not far below an earlier one: the denominators stay in range however often the unit grows
              const float least = fmaxf(old + turn, peak + kSlight);
              const float m = fmaxf(least, fmaxf(fmaxf(S.wmax[0][r], S.wmax[1][r]), fmaxf(S.wmax[2][r], S.wmax[3][r])) - kTop);
              S.rcm[r / 2][2 + (r & 1)] = -m;
              S.peak[r] = fmaxf(peak, m);
              S.fac_l[r] = exp2_fast(old - m);
              S.fac_o[r] = exp2_fast(old + turn - m);
            }
            ptx::named_barrier(3 + group, 128);
            u = u_new;
            inv_of[rc / RC] = inv;
#pragma unroll
            for (int r = 0; r < RC; ++r) {
              l[rc + r] *= S.fac_l[r0 + rc + r];
              v[r] += S.rcm[(r0 + rc + r) / 2][2 + (r & 1)];
            }
            if (it > 0) {
              ok = wait_warp(&S.o_full, (ct - 1) & 1, &S.abort, a.d.status, lane) && ok;  // the second product of tile it - 1 has ended
              ptx::tc_fence_after();
              uint32_t o[RC];
              const uint32_t at = tmem + lane_base + C::kO + r0 + rc;
#pragma unroll
              for (int c = 0; c < RC / 8; ++c) tmem_ld8(at + 8 * c, *reinterpret_cast<uint32_t(*)[8]>(o + 8 * c));
              ptx::tmem_ld_wait();
#pragma unroll
              for (int e = 0; e < RC; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * S.fac_o[r0 + rc + e]);
#pragma unroll
              for (int c = 0; c < RC / 8; ++c) tmem_st8(at + 8 * c, *reinterpret_cast<const uint32_t(*)[8]>(o + 8 * c));
              tmem_st_wait();
            }
          }
          if (rc + RC == RH) {  // the scores have been read
            ptx::tc_fence_before();
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(&S.s_empty[ct % SB]);
          }
          const float f = v_scale * inv_of[rc / RC];
          uint32_t p[RC / 2];
#pragma unroll
          for (int r = 0; r < RC; r += 2) {
            float p0 = exp2_fast(v[r]), p1 = exp2_fast(v[r + 1]);
            add2(l[rc + r], l[rc + r + 1], p0, p1);
            mul2(p0, p1, f);
            p[r / 2] = pack_f16(p0, p1);
          }
          // a single P is free once the second product of the tile before has ended
          if (C::kPBufs == 1 && it > 0 && rc == 0) ok = wait_warp(&S.o_full, (ct - 1) & 1, &S.abort, a.d.status, lane) && ok;
#pragma unroll
          for (int c = 0; c < RC / 8; ++c)
            *reinterpret_cast<uint4*>(p_row + ((((r0 + rc) % 64) / 8 + c) ^ p_xor) * 16) = make_uint4(p[4 * c], p[4 * c + 1], p[4 * c + 2], p[4 * c + 3]);
        }
        if (leave) {
          ok = false;
          break;
        }
        if (C::kPBufs == 2 && it > 0) ok = wait_warp(&S.o_full, (ct - 1) & 1, &S.abort, a.d.status, lane) && ok;  // the widened V is free
        // V: this thread's dimension (its lane of tensor memory), its group's share of the keys
        const int d = quad * 32 + lane;
        if (quad * 32 < D) {
          const uint8_t* vt = smem + C::oV + sv * C::kTile;
          uint32_t w16[64 / G];
#pragma unroll
          for (int z = 0; z < 8 / G; ++z) {
            const int seg = group * (8 / G) + z;
            const uint4 w = *reinterpret_cast<const uint4*>(vt + v_off[z]);
            uint32_t ww[4] = {w.x, w.y, w.z, w.w};
            if (!plain) {
              // keys behind the end or without a page count as zero, so that 0 * V is 0; a NaN of a written key goes to the
              // rows that see the key, and to no others
              const int have = S.pid[sv][seg] < 0 ? 0 : min(16, max(0, k_all - (k0 + 16 * seg)));
              if (have < 16) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                  const int keep = min(4, max(0, have - 4 * e));
                  ww[e] &= keep == 0 ? 0u : 0xffffffffu >> (32 - 8 * keep);
                }
              }
              uint32_t any = 0;  // a byte 7f or ff carries into its top bit
#pragma unroll
              for (int e = 0; e < 4; ++e) any |= (ww[e] & 0x7f7f7f7fu) + 0x01010101u;
              if (masked && (any & 0x80808080u)) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                  const uint32_t bad = __vcmpeq4(ww[e] & 0x7f7f7f7fu, 0x7f7f7f7fu);
                  ww[e] &= ~bad;
#pragma unroll 1
                  for (int y = 0; y < 4 && bad; ++y) {
                    if (!((bad >> (8 * y)) & 1u)) continue;
                    const int kk = seg * 16 + 4 * e + y;
                    for (int r = 0; r < R && row0 + r < n_rows; ++r)
                      if ((S.vis[bu][(row0 + r) / a.rep - i_first][kk >> 5] >> (kk & 31)) & 1u) {
                        atomicOr(&S.nan_row[r][d >> 5], 1u << (d & 31));
                        S.any_nan = 1;
                      }
                  }
                }
              }
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) codes_to_f16(ww[e], w16[8 * z + 2 * e], w16[8 * z + 2 * e + 1]);
          }
          tmem_st(tmem + lane_base + C::kV16 + group * (64 / G), w16);
          tmem_st_wait();
        }
        ptx::tc_fence_before();
        ptx::fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) {
          ptx::mbar_arrive(&S.p_full);
          ptx::mbar_arrive(&S.v_empty[sv]);
        }
      }
      // ---- results
      if (ok && n_tiles > 0) ok = wait_warp(&S.o_full, (gt + n_tiles - 1) & 1, &S.abort, a.d.status, lane);
      ptx::tc_fence_after();
      const float sum = warp_reduce<RH, false>(l, lane);
      S.lsum[quad][r0 + reduced_index<RH>(lane)] = sum;
      if (!any_of(!ok, 3 + group, 128)) {
        // one thread per row: its denominator, and what its accumulators are multiplied by
        if (const int r = r0 + quad * 32 + lane; r < r0 + RH) {
          const int2 ro = S.row[r];
          float den = (S.lsum[0][r] + S.lsum[1][r]) + (S.lsum[2][r] + S.lsum[3][r]);
          float m = den == 0.f ? -INFINITY : -S.rcm[r / 2][2 + (r & 1)];
          float fin = RH > RC && r - r0 >= RC ? unit_of[RH / RC - 1] : unit_of[0];
          if (ro.x >= 0) {
            if (split) a.part_ml[(long long)slot * R + r] = make_float2(m, den);
            else {
              if (a.sinks) {
                const float sk = a.sinks[ro.y] * 1.4426950408889634f, mm = fmaxf(m, sk), g = exp2_fast(m - mm);
                den = den * g + exp2_fast(sk - mm);
                fin *= g;
                m = mm;
              }
              fin *= den > 0.f ? 1.f / den : (den == 0.f ? 0.f : den);
              if (a.lse) a.lse[(long long)ro.x * a.n_heads + ro.y] = den == 0.f ? -INFINITY : (m + log2f(den)) * 0.6931471805599453f;
            }
          }
          S.fac_l[r] = fin;
        }
        ptx::named_barrier(3 + group, 128);
        const int d = quad * 32 + lane;
        if (quad * 32 < D) {
          const bool nans = S.any_nan != 0;
          float* part = a.part_o + ((long long)slot * R + r0) * D + d;
#pragma unroll
          for (int c = 0; c < RH; c += 8) {
            uint32_t oh[8] = {0u, 0u, 0u, 0u, 0u, 0u, 0u, 0u};
            if (n_tiles > 0) {
              tmem_ld8(tmem + lane_base + C::kO + r0 + c, oh);
              ptx::tmem_ld_wait();
            }
            float o[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] = __uint_as_float(oh[e]) * S.fac_l[r0 + c + e];
            if (nans) {
#pragma unroll
              for (int e = 0; e < 8; ++e)
                if ((S.nan_row[r0 + c + e][d >> 5] >> (d & 31)) & 1u) o[e] = __int_as_float(0x7fffffff);
            }
            if (split) {
#pragma unroll
              for (int e = 0; e < 8; ++e) part[(c + e) * D] = o[e];  // rows that are not there have room, too
            } else {
#pragma unroll
              for (int e = 0; e < 8; ++e) {
                const int2 ro = S.row[r0 + c + e];
                if (ro.x >= 0) a.out[(long long)ro.x * a.out_stride + (long long)ro.y * D + d] = __float2bfloat16_rn(o[e]);
              }
            }
          }
        }
      }
    }
    // ---- on to the next piece: everybody has left this one
    ptx::tc_fence_before();
    __syncthreads();
    ptx::tc_fence_after();
    if (S.abort) break;
    gt += n_tiles;
    run += a.whole ? 1 : piece_tiles;
    const int seq_all = ext.row_tiles * a.c.heads * (a.whole ? 1 : ext.key_tiles);
    if (run < run_end && run >= seq_units + seq_all) {  // the run goes on in another sequence
      seq_units += seq_all;
      do {
        seq_segs += ext.row_tiles * a.c.heads;
        s = kv::sequence(a.d, ++b, page);
        ext = extent(a, s, R);
      } while (ext.row_tiles == 0);  // units are left: a sequence with drafts follows
    }
  }
  if (S.abort && warp == 4 * G && lane == 0) {  // copies in flight land before the shared memory is given back
    if (a.ctx_status) atomicExch(a.ctx_status, kStatusTimeout);
    ptx::drain_ring(S.k_full, KS, S.k_it, kBudgetNs);
    ptx::drain_ring(S.v_full, VS, S.v_it, kBudgetNs);
  }
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  if (warp == 4 * G + 1) ptx::tmem_dealloc(tmem, C::kTmem);
}

// One warp per (token, head): the parts of its segment, in order, and the sink.  A segment of one part was finished there.
template <int D>
__global__ void __launch_bounds__(128) attend_combine_kernel(const Args a, const int R) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int lane = threadIdx.x & 31, b = blockIdx.z, hq = blockIdx.y * 4 + (threadIdx.x >> 5);
  if (hq >= a.n_heads) return;
  const Seq s = kv::sequence(a.d, b, 1 << a.c.page_log2);
  const int i = blockIdx.x;
  if (i >= s.n) return;
  const Extent ext = extent(a, s, R);
  const int head = hq / a.rep, rr = i * a.rep + hq - head * a.rep;
  const int2 before = a.table[b];
  const int per = units_per_cta(a.table[a.d.n_seq].x, a.grid);
  const int seg = head * ext.row_tiles + rr / R, from = before.x + seg * ext.key_tiles;
  const int c0 = from / per, parts = (from + ext.key_tiles - 1) / per - c0 + 1;
  if (parts == 1) return;
  const long long token = s.lo + i, at = (long long)(c0 + before.y + seg) * R + rr % R;  // row of the first part; R further on that of the next
  float m = -INFINITY;
  for (int c = lane; c < parts; c += 32) m = fmaxf(m, a.part_ml[at + (long long)c * R].x);
#pragma unroll
  for (int x = 16; x > 0; x >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, x));
  if (a.sinks) m = fmaxf(m, a.sinks[hq] * 1.4426950408889634f);
  const float mr = m == -INFINITY ? 0.f : m;
  constexpr int V = D / 32, kBatch = 8;  // parts in flight
  float o[V] = {}, den = 0.f;
  const long long step = (long long)R * D;
  const float* p = a.part_o + at * D + lane * V;
  for (int c0p = 0; c0p < parts; c0p += 32) {  // a lane has a part's weight, all lanes its columns
    const int c = c0p + lane;
    float w = 0.f;
    if (c < parts) {
      const float2 ml = a.part_ml[at + (long long)c * R];
      w = exp2_fast(ml.x - mr);
      den = fmaf(w, ml.y, den);
    }
    const int n = min(32, parts - c0p);
    for (int k = 0; k < n; k += kBatch) {
      float v[kBatch][V];
#pragma unroll
      for (int j = 0; j < kBatch; ++j)
#pragma unroll
        for (int e = 0; e < V; ++e) v[j][e] = 0.f;
#pragma unroll
      for (int j = 0; j < kBatch; ++j)
        if (k + j < n) {
          if constexpr (V == 4) *reinterpret_cast<float4*>(v[j]) = *reinterpret_cast<const float4*>(p + (c0p + k + j) * step);
          else *reinterpret_cast<float2*>(v[j]) = *reinterpret_cast<const float2*>(p + (c0p + k + j) * step);
        }
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        const float wj = __shfl_sync(0xffffffffu, w, (k + j) & 31);
#pragma unroll
        for (int e = 0; e < V; ++e) o[e] = fmaf(wj, v[j][e], o[e]);
      }
    }
  }
#pragma unroll
  for (int x = 16; x > 0; x >>= 1) den += __shfl_xor_sync(0xffffffffu, den, x);
  if (a.sinks) den += exp2_fast(a.sinks[hq] * 1.4426950408889634f - mr);
  const float inv = den > 0.f ? 1.f / den : (den == 0.f ? 0.f : den);
  __nv_bfloat16* out = a.out + token * a.out_stride + (long long)hq * D + lane * V;
#pragma unroll
  for (int e = 0; e < V; e += 2) *reinterpret_cast<__nv_bfloat162*>(out + e) = __floats2bfloat162_rn(o[e] * inv, o[e + 1] * inv);
  if (a.lse && lane == 0) a.lse[token * a.n_heads + hq] = den == 0.f ? -INFINITY : (m + log2f(den)) * 0.6931471805599453f;
}

}  // namespace att
}  // namespace moev
