// Host side of the operators around the MoE layer (the second part of include/moev.h): argument
// checks, launch rules, launches.  Stateless: no context, nothing allocated, nothing kept.
#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstdio>

#include "attend.cuh"
#include "common.cuh"
#include "kv_cache.cuh"
#include "linear_w4.cuh"
#include "norm.cuh"

namespace moev {  // moev_api.cu
const moev_config& ctx_config(const moev_ctx* c);
int32_t* ctx_status_word(const moev_ctx* c);
moev_status ctx_fail(moev_ctx* c, moev_status st, const char* text);
}  // namespace moev

using namespace moev;

namespace {

constexpr int kMaxNorm = 32768;              // columns of a norm
constexpr float kMaxScale = 1e6f;            // of attention scores
constexpr long long kMaxUnits = 0x3fffffff;  // tiles of an attention call

bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

int sm_count() {
  static std::atomic<int> known[64];  // by device; a constant of the hardware, whichever thread finds it
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 148;
  int n = known[dev].load(std::memory_order_relaxed);
  if (n == 0) {
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 148;
    known[dev].store(n, std::memory_order_relaxed);
  }
  return n;
}

// Dependent launch: the kernel may become resident while its predecessor drains; it waits (griddepcontrol.wait) before
// it reads anything.
template <typename... KArgs, typename... Args>
cudaError_t launch(void (*kern)(KArgs...), dim3 grid, dim3 block, size_t smem, cudaStream_t st, Args&&... args) {
  if (smem > 48 * 1024) {
    cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    // without this the driver may leave an SM shared memory for one CTA where two fit
    if (e == cudaSuccess) e = cudaFuncSetAttribute(kern, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared);
    if (e != cudaSuccess) return e;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kern, static_cast<KArgs>(args)...);
}
moev_status done(cudaError_t e) {
  if (e == cudaSuccess) return MOEV_OK;
  cudaGetLastError();
  return MOEV_ECUDA;
}

// ---------------------------------------------------------------- norm
template <typename T, typename TW, bool VEC>
cudaError_t launch_norm(const NormArgs& a, cudaStream_t st) {
  // pieces of 8 columns: one per thread up to 8192 columns, else the fewest of 4, 8 that 512 threads can hold
  const int pieces = (a.H + 7) / 8;
  const int pv = pieces <= 1024 ? 1 : pieces <= 2048 ? 4 : 8;
  int threads = ((pieces + pv - 1) / pv + 31) & ~31;
  // as many CTAs as the machine holds at 64 registers a thread, each with several rows; a row each where none is fetched ahead
  const int resident = sm_count() * std::max(1, std::min(16, 1024 / threads));
  const dim3 grid((unsigned)(VEC && pv == 1 ? std::min(a.n, resident) : a.n));
  switch (pv) {
    case 1: return launch(add_rmsnorm_kernel<T, TW, 1, VEC>, grid, dim3(threads), 0, st, a);
    case 4: return launch(add_rmsnorm_kernel<T, TW, 4, VEC>, grid, dim3(threads), 0, st, a);
    default: return launch(add_rmsnorm_kernel<T, TW, 8, VEC>, grid, dim3(threads), 0, st, a);
  }
}
template <typename T, typename TW>
cudaError_t launch_norm_v(const NormArgs& a, bool vec, cudaStream_t st) {
  return vec ? launch_norm<T, TW, true>(a, st) : launch_norm<T, TW, false>(a, st);
}

// ---------------------------------------------------------------- 4-bit linear
bool linear_ok(const moev_linear* p) {
  if (!p || p->N < 1 || p->N > (1 << 30) || p->K < 32 || p->K % 32 || p->K > (1 << 20)) return false;
  if (p->wfmt == MOEV_W_MXFP4) return p->group == 32;
  return p->wfmt == MOEV_W_INT4 && (p->group == 32 || p->group == 64 || p->group == 128) && p->K % p->group == 0;
}
size_t linear_tiles(const moev_linear* p) { return ((size_t)p->N + 15) / 16; }
int linear_chunks(const moev_linear* p) { return (p->K + w4::kChunk - 1) / w4::kChunk; }
int linear_scale_bytes(const moev_linear* p) {  // per tile and chunk
  return p->wfmt == MOEV_W_MXFP4 ? 64 : 16 * (128 / p->group) * 2;
}

template <int FMT, int GB, int NT>
cudaError_t launch_linear(const w4::Args& a0, cudaStream_t st) {
  w4::Args a = a0;
  const int sms = sm_count();
  const int tiles = (a.N + 15) / 16;
  const int rows = std::min(a.n, 8 * NT), passes = (a.n + 8 * NT - 1) / (8 * NT);
  // All 16 warps of an SM share one copy of x.  kw of them share a tile's K: the fewest with which the tiles occupy
  // most warps (60 %) of the machine, never more than there are chunks.  Measured at 40 / 60 / 80 % (us): 1 row, 8192 -> 4096 9.9 / 6.7 /
  // 6.6; 8 rows, 2880 -> 5120 MXFP4 8.1 / 7.7 / 7.7; 4 rows, 4096 -> 2880 MXFP4 6.4 / 6.4 / 7.0; 16 rows, 4096 -> 20000 25.3 / 23.3 / 23.4;
  // 8 rows, 2880 -> 14000 10.3 / 10.3 / 10.9.
  const int warps = 16;
  int kw = 1;
  while (kw < 16 && 2 * kw <= a.n_chunks && tiles * kw * 10 < sms * warps * 6) kw *= 2;
  // bytes of a piece of x: a row is 256 bytes a chunk + 64 (rows then start in alternating halves of the banks), MXFP4 has scales behind them
  auto piece_bytes = [&](int chunks) { return (size_t)rows * (chunks * 256 + 64) + (FMT == w4::kMx ? (size_t)chunks * 16 * NT : 0); };
  const size_t most = 227 * 1024, red = (size_t)warps * NT * 8 * w4::kRedPitch * 4;
  int grid, piece;
  for (;; kw /= 2) {
    const int rw = warps / kw;
    grid = std::min((tiles + rw - 1) / rw, sms);
    a.rounds = (tiles + rw * grid - 1) / (rw * grid);
    const bool apart = kw > 1 && a.rounds > 1;  // x is needed again after the warps' sums have met
    const size_t budget = most - (apart ? red : 0);
    a.n_bufs = piece_bytes(a.n_chunks) <= budget ? 1 : 2;
    piece = a.n_chunks;
    if (a.n_bufs == 2) {  // two pieces at a time, each of at least one chunk per warp of a tile
      piece = 1;
      while (2 * piece_bytes(piece + 1) <= budget) ++piece;
      if (piece < kw) continue;
      piece = piece / kw * kw;
    }
    a.buf_bytes = (int)piece_bytes(piece);
    a.red_at = apart ? a.n_bufs * a.buf_bytes : 0;
    break;
  }
  a.kw_log2 = 0;
  while ((1 << a.kw_log2) < kw) ++a.kw_log2;
  a.phase_chunks = a.n_bufs == 1 ? (a.n_chunks + kw - 1) / kw * kw : piece;
  a.x_pitch = piece * 256 + 64;
  const size_t smem = std::max((size_t)a.n_bufs * a.buf_bytes, a.red_at + (kw > 1 ? red : 0));
  return a.n_bufs == 1 ? launch(w4::linear_w4_kernel<FMT, GB, NT, true>, dim3(grid, passes), dim3(warps * 32), smem, st, a)
                       : launch(w4::linear_w4_kernel<FMT, GB, NT, false>, dim3(grid, passes), dim3(warps * 32), smem, st, a);
}
template <int FMT, int GB>
cudaError_t launch_linear_n(const w4::Args& a, cudaStream_t st) {
  if (a.n <= 8) return launch_linear<FMT, GB, 1>(a, st);
  if (a.n <= 16) return launch_linear<FMT, GB, 2>(a, st);
  return launch_linear<FMT, GB, 4>(a, st);
}

// ---------------------------------------------------------------- cache
bool batch_ok(const moev_kv_cache* c, const moev_draft_batch* d) {
  if (!c || !d) return false;
  if (c->n_pages < 1 || c->n_kv_heads < 1 || c->n_kv_heads > 1024 || (c->head_dim != 64 && c->head_dim != 128)) return false;
  if (c->page != 16 && c->page != 32 && c->page != 64 && c->page != 128) return false;
  if (!c->k || !c->v || !c->k_scale || !c->v_scale || !aligned(c->k, 16) || !aligned(c->v, 16) || !aligned(c->k_scale, 4) ||
      !aligned(c->v_scale, 4))
    return false;
  if (d->n_seq < 0 || d->n_seq > 65535 || d->n_tokens < 0 || d->max_drafts < 1 || d->max_len < d->max_drafts || d->table_cols < 1) return false;
  if (d->max_len > (1 << 30) || d->max_drafts > (1 << 24)) return false;
  // coordinates of the rows of K and V are 32 bits wide
  if ((long long)c->n_pages * c->n_kv_heads * std::max(c->page, c->head_dim) > 0x7fffffffLL) return false;
  if (d->parent && d->max_drafts > kv::kMaxTree) return false;
  return d->n_seq == 0 || (d->cu && d->ctx_len && d->page_table);
}
// Row stride of a 16-bit tensor of n rows that are read by 16 bytes: of one row it is not looked at.
bool stride_ok(int64_t stride, int64_t width, int n) { return n <= 1 || (stride >= width && stride % 8 == 0); }
kv::Drafts drafts_of(const moev_draft_batch* d) {
  return kv::Drafts{d->n_seq, d->n_tokens, d->max_drafts, d->max_len, d->table_cols, d->cu, d->ctx_len, d->page_table, d->parent, d->status};
}
kv::Cache cache_of(const moev_kv_cache* c) {
  int lg = 4;
  while ((1 << lg) < c->page) ++lg;
  return kv::Cache{c->n_pages, lg, c->n_kv_heads, c->k, c->v, c->k_scale, c->v_scale};
}

struct Plan {
  int rows, grid, whole;  // rows of a tile, CTAs, segments dealt out whole
  long long units;        // tiles of the call, at most
  size_t table, ml, o;    // bytes of the workspace's parts
};
Plan attend_plan(const moev_kv_cache* c, const moev_draft_batch* d, int n_heads, int window) {
  Plan p;
  const int rep = n_heads / c->n_kv_heads;
  const long long rows = (long long)d->max_drafts * rep;
  p.rows = rows <= 16 ? 16 : rows <= 32 ? 32 : rows <= 64 ? 64 : 128;
  // a tile of 128 rows and the ancestors of very large trees do not fit together
  if (p.rows == 128 && att::smem_bytes<128, 128>((d->max_drafts + 31) / 32, d->parent != nullptr) > 227 * 1024) p.rows = 64;
  long long span = d->max_len;
  if (window > 0) span = std::min<long long>(span, (long long)window + d->max_drafts + att::kKeys - 1);
  const long long tiles = (span + att::kKeys - 1) / att::kKeys;  // of keys, at most
  const long long segments = (long long)d->n_seq * c->n_kv_heads * ((rows + p.rows - 1) / p.rows);
  // Whole segments save the second kernel and set up once each, but leave CTAs empty where there are few of them.  Measured at
  // 2 / 4 / 8 / 12 tiles, 8 kv heads, 8 rows each (us, whole | split): 16 sequences 11.5 | 14.7, 14.2 | 16.9, 19.1 | 21.2, 24.5 |
  // 25.2; one sequence 10.9 | 11.6, 13.4 | 11.5, 17.6 | 11.5, 22.2 | 12.2.  Up to 4 tiles neither choice is far off.
  p.whole = tiles <= 4;
  p.units = segments * tiles;
  p.grid = (int)std::min<long long>(sm_count() * (p.rows <= 32 ? 2 : 1), p.whole ? segments : segments * tiles);
  const size_t slots = (size_t)p.grid + (size_t)segments;
  p.table = p.whole ? 0 : (((size_t)d->n_seq + 1) * 8 + 15) & ~(size_t)15;
  p.ml = p.whole ? 0 : slots * p.rows * 8;
  p.o = p.whole ? 0 : slots * p.rows * c->head_dim * 4;
  return p;
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                  const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiledFn encode_tiled_fn() {
  static EncodeTiledFn fn = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    const bool ok = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) == cudaSuccess && q == cudaDriverEntryPointSuccess;
    return ok ? reinterpret_cast<EncodeTiledFn>(p) : nullptr;
  }();
  return fn;
}
// rows of `width` bytes (16 to 128), `box` of them at a time, in the swizzle of that width
bool encode_rows(CUtensorMap* m, const void* ptr, int width, long long rows, int box) {
  EncodeTiledFn fn = encode_tiled_fn();
  if (!fn) return false;
  const cuuint64_t dims[2] = {(cuuint64_t)width, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)width};
  const cuuint32_t b[2] = {(cuuint32_t)width, (cuuint32_t)box}, es[2] = {1, 1};
  const CUtensorMapSwizzle sw = width == 128  ? CU_TENSOR_MAP_SWIZZLE_128B
                                : width == 64 ? CU_TENSOR_MAP_SWIZZLE_64B
                                : width == 32 ? CU_TENSOR_MAP_SWIZZLE_32B
                                              : CU_TENSOR_MAP_SWIZZLE_NONE;
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(ptr), dims, strides, b, es, CU_TENSOR_MAP_INTERLEAVE_NONE, sw,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D, int R>
cudaError_t launch_attend(const att::Args& a, const CUtensorMap& tk, const CUtensorMap& tv, cudaStream_t st) {
  const size_t smem = att::smem_bytes<D, R>((a.d.max_drafts + 31) / 32, a.d.parent != nullptr);
  return launch(att::attend_kernel<D, R>, dim3(a.grid), dim3(att::Cfg<D, R>::kThreads), smem, st, a, tk, tv);
}
template <int D>
cudaError_t launch_attend_d(const att::Args& a, int rows, cudaStream_t st) {
  const int page = 1 << a.c.page_log2;
  const long long blocks = (long long)a.c.n_pages * a.c.heads;
  CUtensorMap tk, tv;
  if (!encode_rows(&tk, a.c.k, D, blocks * page, page) || !encode_rows(&tv, a.c.v, page, blocks * D, D)) return cudaErrorUnknown;
  cudaError_t e;
  if (rows == 16) e = launch_attend<D, 16>(a, tk, tv, st);
  else if (rows == 32) e = launch_attend<D, 32>(a, tk, tv, st);
  else if (rows == 64) e = launch_attend<D, 64>(a, tk, tv, st);
  else e = launch_attend<D, 128>(a, tk, tv, st);
  if (e != cudaSuccess || a.whole) return e;
  return launch(att::attend_combine_kernel<D>, dim3(a.d.max_drafts, (a.n_heads + 3) / 4, a.d.n_seq), dim3(128), 0, st, a, rows);
}

// moev_cache_attend, also for a context whose status word learns of a time-out
moev_status attend(const moev_kv_cache* c, const moev_draft_batch* d, const void* q, int64_t q_stride, int32_t n_heads, float scale,
                   int32_t window, const float* sinks, void* out, int64_t out_stride, float* lse, void* workspace, size_t workspace_bytes,
                   int32_t* ctx_status, void* cuda_stream) {
  if (!batch_ok(c, d) || (d->n_tokens > 0 && (!q || !out)) || n_heads < 1 || n_heads % c->n_kv_heads || window < 0 || !(scale > 0.f) || scale > kMaxScale) return MOEV_EINVAL;
  if (!aligned(q, 16) || !aligned(out, 16) || !aligned(lse, 4) || !aligned(sinks, 4)) return MOEV_EINVAL;
  const int64_t row = (int64_t)n_heads * c->head_dim;
  if (!stride_ok(q_stride, row, d->n_tokens) || !stride_ok(out_stride, row, d->n_tokens)) return MOEV_EINVAL;
  if (d->n_seq == 0 || d->n_tokens == 0) return MOEV_OK;
  const Plan p = attend_plan(c, d, n_heads, window);
  if ((n_heads + 3) / 4 > 65535 || p.units > kMaxUnits) return MOEV_EINVAL;
  const size_t need = p.table + p.ml + p.o;
  if (need && (!workspace || !aligned(workspace, 16) || workspace_bytes < need)) return MOEV_EINVAL;
  att::Args a{};
  a.d = drafts_of(d);
  a.c = cache_of(c);
  a.q = static_cast<const __nv_bfloat16*>(q);
  a.out = static_cast<__nv_bfloat16*>(out);
  a.lse = lse;
  a.sinks = sinks;
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  a.table = reinterpret_cast<int2*>(ws);
  a.part_ml = reinterpret_cast<float2*>(ws + p.table);
  a.part_o = reinterpret_cast<float*>(ws + p.table + p.ml);
  a.q_stride = q_stride;
  a.out_stride = out_stride;
  a.n_heads = n_heads;
  a.rep = n_heads / c->n_kv_heads;
  a.window = window;
  a.whole = p.whole;
  a.grid = p.grid;
  a.scale_log2 = scale * 1.4426950408889634f;
  a.ctx_status = ctx_status;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  return done(c->head_dim == 64 ? launch_attend_d<64>(a, p.rows, st) : launch_attend_d<128>(a, p.rows, st));
}

}  // namespace

extern "C" {

moev_status moev_add_rmsnorm(const moev_norm* p, void* cuda_stream) {
  if (!p || p->n < 0 || p->H < 1 || p->H > kMaxNorm || p->afmt < 0 || p->afmt > MOEV_ACT_BF16 || p->wfmt < 0 || p->wfmt > MOEV_ACT_BF16)
    return MOEV_EINVAL;
  if (p->act_quant < 0 || p->act_quant > MOEV_ACTQ_FP8_B128_POW2 || !(p->eps >= 0.f) || !p->w) return MOEV_EINVAL;
  if (p->n == 0) return MOEV_OK;  // tensors of no rows have no address
  if (!p->x || (!p->y && !p->codes && !p->residual_out) || (p->act_quant != 0) != (p->codes != nullptr) || (p->codes != nullptr) != (p->scales != nullptr))
    return MOEV_EINVAL;
  const int es = p->afmt == MOEV_ACT_BF16 ? 2 : 4, ws = p->wfmt == MOEV_ACT_BF16 ? 2 : 4;
  bool vec = p->H % 8 == 0 && aligned(p->w, 16) && aligned(p->codes, 8) && (!p->codes || p->n == 1 || p->codes_stride % 8 == 0);
  const void* ptr[4] = {p->x, p->residual, p->y, p->residual_out};
  const int64_t stride[4] = {p->x_stride, p->residual_stride, p->y_stride, p->residual_out_stride};
  for (int i = 0; i < 4; ++i) {
    if (!ptr[i]) continue;
    if (!aligned(ptr[i], es) || (p->n > 1 && stride[i] < p->H)) return MOEV_EINVAL;
    vec = vec && aligned(ptr[i], 16) && (p->n == 1 || (stride[i] * es) % 16 == 0);
  }
  if (!aligned(p->w, ws) || !aligned(p->scales, 4) || (p->codes && p->n > 1 && p->codes_stride < p->H)) return MOEV_EINVAL;
  NormArgs a{p->x, p->residual, p->w, p->y, p->residual_out, p->codes, p->scales, p->x_stride, p->residual_stride, p->y_stride,
             p->residual_out_stride, p->codes_stride, p->n, p->H, p->act_quant, p->eps};
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  const bool xb = p->afmt == MOEV_ACT_BF16, wb = p->wfmt == MOEV_ACT_BF16;
  cudaError_t e = xb ? (wb ? launch_norm_v<__nv_bfloat16, __nv_bfloat16>(a, vec, st) : launch_norm_v<__nv_bfloat16, float>(a, vec, st))
                     : (wb ? launch_norm_v<float, __nv_bfloat16>(a, vec, st) : launch_norm_v<float, float>(a, vec, st));
  return done(e);
}

size_t moev_w4_packed_bytes(const moev_linear* p) {
  if (!linear_ok(p)) return 0;
  return linear_tiles(p) * linear_chunks(p) * (size_t)(w4::kChunkBytes + linear_scale_bytes(p)) + w4::kTailBytes;
}

moev_status moev_w4_pack(const moev_linear* p, const void* codes, const void* scales, void* packed, void* cuda_stream) {
  if (!linear_ok(p) || !codes || !scales || !packed || !aligned(codes, 4) || !aligned(packed, 16)) return MOEV_EINVAL;
  if (!aligned(scales, p->wfmt == MOEV_W_INT4 ? 2 : 1)) return MOEV_EINVAL;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  const int chunks = linear_chunks(p);
  const long long units = (long long)linear_tiles(p) * chunks;
  const int fmt = p->wfmt == MOEV_W_INT4 ? w4::kInt4 : w4::kMx;
  const long long words = units * 256;
  uint8_t* sc = static_cast<uint8_t*>(packed) + units * w4::kChunkBytes;
  w4::pack_codes_kernel<<<(unsigned)((words + 255) / 256), 256, 0, st>>>(static_cast<const uint8_t*>(codes), static_cast<uint32_t*>(packed),
                                                                        p->N, p->K, chunks, fmt, words);
  const int per_row = 128 / p->group;
  const long long count = units * 16 * per_row;
  const unsigned blocks = (unsigned)((count + 255) / 256);
  if (fmt == w4::kInt4)
    w4::pack_scales_kernel<uint16_t><<<blocks, 256, 0, st>>>(static_cast<const uint16_t*>(scales), reinterpret_cast<uint16_t*>(sc), p->N,
                                                            p->K / p->group, chunks, per_row, count);
  else
    w4::pack_scales_kernel<uint8_t><<<blocks, 256, 0, st>>>(static_cast<const uint8_t*>(scales), sc, p->N, p->K / p->group, chunks, per_row, count);
  return done(cudaGetLastError());
}

moev_status moev_linear_w4(const moev_linear* p, const void* packed, const float* bias, const void* x, int64_t x_stride, int32_t n, void* y,
                           int64_t y_stride, int32_t yfmt, void* cuda_stream) {
  if (!linear_ok(p) || !packed || (n > 0 && (!x || !y)) || n < 0 || yfmt < 0 || yfmt > MOEV_ACT_BF16) return MOEV_EINVAL;
  if (!aligned(packed, 16) || !aligned(x, 2) || !aligned(y, yfmt == MOEV_ACT_BF16 ? 2 : 4) || !aligned(bias, 4)) return MOEV_EINVAL;
  if (n > 1 && (x_stride < p->K || y_stride < p->N)) return MOEV_EINVAL;
  if (n > 32 * 65535) return MOEV_EINVAL;
  if (n == 0) return MOEV_OK;
  w4::Args a{};
  a.codes = static_cast<const uint8_t*>(packed);
  a.n_chunks = linear_chunks(p);
  a.scales = a.codes + linear_tiles(p) * a.n_chunks * (size_t)w4::kChunkBytes;
  a.x = static_cast<const __nv_bfloat16*>(x);
  a.bias = bias;
  a.y = y;
  a.x_stride = x_stride;
  a.y_stride = y_stride;
  a.n = n;
  a.N = p->N;
  a.K = p->K;
  a.y_f32 = yfmt == MOEV_ACT_FP32;
  a.x_vec = aligned(x, 16) && (n == 1 || x_stride % 8 == 0);
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  if (p->wfmt == MOEV_W_MXFP4) return done(launch_linear_n<w4::kMx, 1>(a, st));
  if (p->group == 32) return done(launch_linear_n<w4::kInt4, 1>(a, st));
  if (p->group == 64) return done(launch_linear_n<w4::kInt4, 2>(a, st));
  return done(launch_linear_n<w4::kInt4, 4>(a, st));
}

moev_status moev_cache_append(const moev_kv_cache* c, const moev_draft_batch* d, const void* k, int64_t k_stride, const void* v,
                              int64_t v_stride, const float* rope, int32_t rope_rows, const void* q, int64_t q_stride, int32_t n_heads,
                              void* q_out, int64_t q_out_stride, void* cuda_stream) {
  if (!batch_ok(c, d) || (d->n_tokens > 0 && (!k || !v)) || !aligned(k, 16) || !aligned(v, 16)) return MOEV_EINVAL;
  const int64_t kv_row = (int64_t)c->n_kv_heads * c->head_dim;
  if (!stride_ok(k_stride, kv_row, d->n_tokens) || !stride_ok(v_stride, kv_row, d->n_tokens)) return MOEV_EINVAL;
  if (rope && (rope_rows < 1 || !aligned(rope, 16))) return MOEV_EINVAL;
  if ((q != nullptr) != (q_out != nullptr)) return MOEV_EINVAL;
  if (q) {
    const int64_t q_row = (int64_t)n_heads * c->head_dim;
    if (n_heads < 1 || n_heads % c->n_kv_heads || !aligned(q, 16) || !aligned(q_out, 16)) return MOEV_EINVAL;
    if (!stride_ok(q_stride, q_row, d->n_tokens) || !stride_ok(q_out_stride, q_row, d->n_tokens)) return MOEV_EINVAL;
  }
  if (d->n_seq == 0 || d->n_tokens == 0) return MOEV_OK;
  kv::AppendArgs a{};
  a.d = drafts_of(d);
  a.c = cache_of(c);
  a.k = static_cast<const __nv_bfloat16*>(k);
  a.v = static_cast<const __nv_bfloat16*>(v);
  a.q = static_cast<const __nv_bfloat16*>(q);
  a.q_out = static_cast<__nv_bfloat16*>(q_out);
  a.k_stride = k_stride; a.v_stride = v_stride; a.q_stride = q_stride; a.q_out_stride = q_out_stride;
  a.rope = rope;
  a.rope_rows = rope_rows;
  a.rep = q ? n_heads / c->n_kv_heads : 0;
  // pages that max_drafts tokens can touch, wherever the first one falls in its page
  const int pages = (d->max_drafts + c->page - 2) / c->page + 1;
  // CTAs for a page's queries: one for up to 2 query heads per kv head, two above.  Measured with 1 / 2 / 3 (us): 2 heads, 4 096 tokens
  // 20.0 / 21.2; 4 heads 25.5 / 24.7 / 25.7; 16 heads 60.8 / 56.2 / 52.5; 64 tokens, 8 heads 9.9 / 7.8 / 7.8.
  a.q_parts = std::min(2, (a.rep + 1) / 2);
  const int n_par = d->parent && rope ? std::min(d->max_drafts, kv::kMaxTree) : 0;
  const size_t smem = (size_t)(((c->page + n_par) * 4 + 15) & ~15) + (size_t)c->page * c->head_dim + (size_t)c->head_dim * (c->page + 4);
  const dim3 grid(pages, c->n_kv_heads * (1 + a.q_parts), d->n_seq);
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  return done(c->head_dim == 64 ? launch(kv::cache_append_kernel<64>, grid, dim3(256), smem, st, a)
                                : launch(kv::cache_append_kernel<128>, grid, dim3(256), smem, st, a));
}

size_t moev_cache_attend_workspace(const moev_kv_cache* c, const moev_draft_batch* d, int32_t n_heads, int32_t window) {
  if (!batch_ok(c, d) || n_heads < 1 || n_heads % c->n_kv_heads) return 0;
  const Plan p = attend_plan(c, d, n_heads, window);
  return p.table + p.ml + p.o;
}

moev_status moev_cache_attend(const moev_kv_cache* c, const moev_draft_batch* d, const void* q, int64_t q_stride, int32_t n_heads, float scale,
                              int32_t window, const float* sinks, void* out, int64_t out_stride, float* lse, void* workspace,
                              size_t workspace_bytes, void* cuda_stream) {
  return attend(c, d, q, q_stride, n_heads, scale, window, sinks, out, out_stride, lse, workspace, workspace_bytes, nullptr, cuda_stream);
}


namespace {
struct BlockBuffers {  // byte offsets in the workspace
  size_t x, qkv, attn, o, attend, total;
};
BlockBuffers block_buffers(const moev_config& g, int n_blocks, const moev_block* blocks, const moev_draft_batch* d, int n_heads) {
  auto up = [](size_t n) { return (n + 255) & ~(size_t)255; };
  size_t qkv = 0, attn = 0, att_ws = 0;
  const size_t T = d->n_tokens;
  for (int l = 0; l < n_blocks; ++l) {
    const moev_kv_cache& c = blocks[l].cache;
    qkv = std::max(qkv, T * (size_t)(n_heads + 2 * c.n_kv_heads) * c.head_dim * 2);
    attn = std::max(attn, T * (size_t)n_heads * c.head_dim * 2);
    att_ws = std::max(att_ws, moev_cache_attend_workspace(&c, d, n_heads, blocks[l].window));
  }
  BlockBuffers b;
  b.x = 0;
  b.qkv = b.x + up(T * g.H * 2);
  b.attn = b.qkv + up(qkv);
  b.o = b.attn + up(attn);
  b.attend = b.o + up(T * g.H * 2);
  b.total = b.attend + up(att_ws);
  return b;
}
// what is wrong with the call, or null
const char* blocks_refuse(const moev_config& g, int n_blocks, const moev_block* blocks, const moev_draft_batch* d, const moev_block_options* o) {
  if (n_blocks < 1 || !blocks || !d || !o) return "no blocks, batch or options";
  if (g.afmt != MOEV_ACT_BF16) return "decoder blocks need a context for bfloat16 activations";
  if (d->n_tokens < 1 || d->n_tokens > g.max_tokens) return "n_tokens must be in 1..max_tokens of the context";
  if (g.H > kMaxNorm) return "rows of more than 32768 columns are not served";
  if (!(o->eps >= 0.f) || !(o->scale >= 0.f) || o->scale > kMaxScale) return "eps must not be negative, scale must be from 0 to 1e6";
  if ((o->final_norm != nullptr) != (o->final_out != nullptr) || !aligned(o->final_norm, 16) || !aligned(o->final_out, 16)) return "final_norm and final_out go together, 16-byte aligned";
  if (o->rope && (o->rope_rows < 1 || !aligned(o->rope, 16))) return "rope needs rows and 16-byte alignment";
  for (int l = 0; l < n_blocks; ++l) {
    const moev_block& b = blocks[l];
    if (!batch_ok(&b.cache, d)) return "a block's cache or the batch is invalid";
    if (o->n_heads < 1 || o->n_heads % b.cache.n_kv_heads) return "n_heads must be a multiple of n_kv_heads";
    const int64_t row = (int64_t)o->n_heads * b.cache.head_dim, all = row + 2 * (int64_t)b.cache.n_kv_heads * b.cache.head_dim;
    if (!linear_ok(&b.qkv) || !linear_ok(&b.o) || b.qkv.K != g.H || b.qkv.N != all || b.o.K != row || b.o.N != g.H)
      return "qkv must be [(n_heads + 2 n_kv_heads) head_dim, H] and o [H, n_heads head_dim]";
    if (!b.attn_norm || !b.ffn_norm || !b.qkv_packed || !b.o_packed || !aligned(b.attn_norm, 16) || !aligned(b.ffn_norm, 16) ||
        !aligned(b.qkv_packed, 16) || !aligned(b.o_packed, 16) || !aligned(b.qkv_bias, 4) || !aligned(b.o_bias, 4) || !aligned(b.sinks, 4))
      return "a block's norm or projection weight is null or misaligned";
    if (b.window < 0) return "window must not be negative";
    if (attend_plan(&b.cache, d, o->n_heads, b.window).units > kMaxUnits) return "the batch's bounds are too large";
  }
  return nullptr;
}
}  // namespace

size_t moev_verify_blocks_workspace(const moev_ctx* ctx, int32_t n_blocks, const moev_block* blocks, const moev_draft_batch* d,
                                    const moev_block_options* o) {
  if (!ctx || blocks_refuse(ctx_config(ctx), n_blocks, blocks, d, o)) return 0;
  return block_buffers(ctx_config(ctx), n_blocks, blocks, d, o->n_heads).total;
}

moev_status moev_verify_blocks(moev_ctx* ctx, int32_t n_blocks, const moev_block* blocks, const moev_draft_batch* d, const moev_block_options* o,
                               void* hidden, const moev_out* outs, void* workspace, size_t workspace_bytes, void* cuda_stream) {
  if (!ctx) return MOEV_EINVAL;
  const moev_config& g = ctx_config(ctx);
  if (const char* why = blocks_refuse(g, n_blocks, blocks, d, o)) return ctx_fail(ctx, MOEV_EINVAL, why);
  if (!hidden || !aligned(hidden, 16) || !outs) return ctx_fail(ctx, MOEV_EINVAL, "hidden or outs is null or misaligned");
  for (int l = 0; l < n_blocks; ++l)
    if (!outs[l].y || !aligned(outs[l].y, 16) || !outs[l].n_active) return ctx_fail(ctx, MOEV_EINVAL, "every block needs outs[l].y (16-byte aligned) and n_active");
  const BlockBuffers w = block_buffers(g, n_blocks, blocks, d, o->n_heads);
  if (!workspace || !aligned(workspace, 16) || workspace_bytes < w.total) return ctx_fail(ctx, MOEV_EINVAL, "workspace too small or misaligned");
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  const int T = d->n_tokens, H = g.H;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  moev_norm n{};
  n.n = T;
  n.H = H;
  n.afmt = n.wfmt = MOEV_ACT_BF16;
  n.eps = o->eps;
  n.x_stride = n.residual_stride = n.residual_out_stride = n.y_stride = H;
#define STEP(call, text)                                    \
  do {                                                      \
    const moev_status r = (call);                           \
    if (r != MOEV_OK) return ctx_fail(ctx, r, text);        \
  } while (0)
  for (int l = 0; l < n_blocks; ++l) {
    const moev_block& b = blocks[l];
    const int D = b.cache.head_dim;
    const int64_t row = (int64_t)o->n_heads * D, kv_row = (int64_t)b.cache.n_kv_heads * D, all = row + 2 * kv_row;
    uint16_t* qkv = reinterpret_cast<uint16_t*>(ws + w.qkv);
    // h += MoE output of the block before, in the norm's pass over it
    n.w = b.attn_norm;
    n.y = ws + w.x;
    n.x = l ? outs[l - 1].y : hidden;
    n.residual = l ? hidden : nullptr;
    n.residual_out = l ? hidden : nullptr;
    STEP(moev_add_rmsnorm(&n, st), "attention norm");
    STEP(moev_linear_w4(&b.qkv, b.qkv_packed, b.qkv_bias, ws + w.x, H, T, qkv, all, MOEV_ACT_BF16, st), "qkv projection");
    STEP(moev_cache_append(&b.cache, d, qkv + row, all, qkv + row + kv_row, all, o->rope, o->rope_rows, qkv, all, o->n_heads, qkv, all, st), "cache append");
    if (cudaMemsetAsync(ws + w.attn, 0, (size_t)T * row * 2, st) != cudaSuccess) return ctx_fail(ctx, MOEV_ECUDA, "memset failed");
    STEP(attend(&b.cache, d, qkv, all, o->n_heads, o->scale > 0.f ? o->scale : (float)(1.0 / std::sqrt((double)D)), b.window, b.sinks,
                ws + w.attn, row, nullptr, ws + w.attend, w.total - w.attend, ctx_status_word(ctx), st),
         "attention");
    STEP(moev_linear_w4(&b.o, b.o_packed, b.o_bias, ws + w.attn, row, T, ws + w.o, H, MOEV_ACT_BF16, st), "output projection");
    n.w = b.ffn_norm;
    n.x = ws + w.o;
    n.residual = n.residual_out = hidden;
    STEP(moev_add_rmsnorm(&n, st), "MoE norm");
    const moev_status r = moev_verify(ctx, &b.moe, ws + w.x, T, &outs[l], st);
    if (r != MOEV_OK) return r;
  }
  n.x = outs[n_blocks - 1].y;
  n.residual = n.residual_out = hidden;
  n.w = o->final_norm ? o->final_norm : blocks[n_blocks - 1].ffn_norm;
  n.y = o->final_out;
  STEP(moev_add_rmsnorm(&n, st), "final norm");
#undef STEP
  return MOEV_OK;
}

#ifdef MOEV_TEST_HOOKS
// Test builds only: while the flag is set, the loader of the attention kernel leaves out the last V tile (see common.cuh).
int32_t moev_test_withhold_attend(int32_t on) {
  const int v = on ? 1 : 0;
  return cudaMemcpyToSymbol(g_test_withhold, &v, sizeof(int)) == cudaSuccess ? 0 : -1;
}
#endif

}  // extern "C"
