// Host side of the operators in front of and behind a verification pass (the third part of include/moev.h): argument checks,
// launch rules, launches.  Stateless: no context, nothing allocated, nothing kept.
#include <algorithm>
#include <climits>

#include "host.cuh"
#include "linear_i8.cuh"
#include "logprobs.cuh"
#include "pages.cuh"
#include "prompt.cuh"

using namespace moev;

namespace {

constexpr int kMaxK8 = 131056;  // of an 8-bit product: 2^14 of each element of K stay below 2^31

// ---------------------------------------------------------------- prompt attention
// [rows][heads][D] bf16, `head_box` heads of `row_box` rows at a time, 64 columns (128 bytes, swizzled)
bool encode_heads(CUtensorMap* m, const void* ptr, int D, int heads, int rows, int64_t stride, int head_box, int row_box) {
  EncodeTiledFn fn = encode_tiled_fn();
  if (!fn) return false;
  if (rows == 1) stride = (int64_t)heads * D;
  const cuuint64_t dims[3] = {(cuuint64_t)D, (cuuint64_t)heads, (cuuint64_t)rows}, strides[2] = {(cuuint64_t)D * 2, (cuuint64_t)stride * 2};
  const cuuint32_t box[3] = {64, (cuuint32_t)head_box, (cuuint32_t)row_box}, es[3] = {1, 1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(ptr), dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D, int T, bool SPLIT = false>
cudaError_t launch_prompt(const prm::Args& a, const moev_prompt* p, int n_keys, unsigned grid, cudaStream_t st, int ranks = 1) {
  using C = prm::Cfg<D, T>;
  // without keys nothing is loaded, but a tensor map needs an address
  const void *k = n_keys > 0 ? p->k : p->q, *v = n_keys > 0 ? p->v : p->q;
  const int keys = std::max(1, n_keys);
  CUtensorMap tq, tk, tv;
  if (!encode_heads(&tq, p->q, D, p->n_heads, a.n_tokens, p->q_stride, a.tile_heads, a.tokens) || !encode_heads(&tk, k, D, p->n_kv_heads, keys, p->k_stride, 1, C::kKeys) ||
      !encode_heads(&tv, v, D, p->n_kv_heads, keys, p->v_stride, 1, C::kKeys))
    return cudaErrorUnknown;
  return launch_clusters(prm::prompt_kernel<D, T, SPLIT>, ranks, dim3(grid * ranks), dim3(C::kThreads), prm::smem_bytes<D, T>(), st, a, tq, tk, tv);
}

// ---------------------------------------------------------------- 8-bit linear
bool linear_i8_ok(const moev_w8* p) {
  return p && p->N >= 1 && p->N <= (1 << 30) && p->K >= 16 && p->K % 16 == 0 && p->K <= kMaxK8 && p->w && p->w_scales && aligned(p->w, 16) &&
         aligned(p->w_scales, 4) && aligned(p->bias, 4) && aligned(p->status, 4);
}
bool encode_codes(CUtensorMap* m, const void* ptr, int K, int rows, int64_t stride, int box_rows) {
  EncodeTiledFn fn = encode_tiled_fn();
  if (!fn) return false;
  if (rows == 1) stride = K;
  const cuuint64_t dims[2] = {(cuuint64_t)K, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)stride};
  const cuuint32_t box[2] = {i8::kStep, (cuuint32_t)box_rows}, es[2] = {1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(ptr), dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
template <typename T, int PV, int THREADS>
cudaError_t launch_quant_v(const i8::QuantArgs& a, bool vec, cudaStream_t st) {
  return vec ? launch(i8::quant_rows_kernel<T, PV, true, THREADS>, dim3(a.n), dim3(THREADS), 0, st, a)
             : launch(i8::quant_rows_kernel<T, PV, false, THREADS>, dim3(a.n), dim3(THREADS), 0, st, a);
}
template <typename T>
cudaError_t launch_quant(const i8::QuantArgs& a, bool vec, cudaStream_t st) {
  // Half as many threads with twice the values each where there are enough rows to fill the SMs all the same: less work around each value.  Us, 128
  // threads | 256: 8001 x 7168 bf16 33.5 | 36.5, 8001 x 2048 11.5 | 14.3, 2000 x 2880 5.4 | 5.6; but 3000 x 8192 16.8 | 16.4, 8 x 8192 3.6 | 2.8.
  if (a.n > 4 * sm_count() && a.K * sizeof(T) < 16384) {
    if (a.K <= 2048) return launch_quant_v<T, 2, 128>(a, vec, st);
    if (a.K <= 4096 || sizeof(T) == 4) return launch_quant_v<T, 4, 128>(a, vec, st);
    return launch_quant_v<T, 8, 128>(a, vec, st);
  }
  if (a.K <= 2048) return launch_quant_v<T, 1, 256>(a, vec, st);
  if (a.K <= 4096) return launch_quant_v<T, 2, 256>(a, vec, st);
  if (a.K <= 8192) return launch_quant_v<T, 4, 256>(a, vec, st);
  return launch_quant_v<T, 0, 256>(a, vec, st);
}
template <int NT, typename X = void>
cudaError_t launch_few(const i8::Args& a, const void* x, int64_t x_stride, const void* w, int K, cudaStream_t st) {
  CUtensorMap tx, tw;
  if (!encode_codes(&tw, w, K, a.N, K, 128)) return cudaErrorUnknown;
  if (!std::is_void<X>::value) tx = tw;
  else if (!encode_codes(&tx, x, K, a.n, x_stride, NT)) return cudaErrorUnknown;
  const int tiles = (a.N + 127) / 128, blocks = (a.n + NT - 1) / NT;
  // CTAs that share a tile's K: up to 1.75 per SM.  (Two fit, but not every SM has a place where a cluster needs it: 1 x 7168 -> 9217 with 292 CTAs
  // 19.9 us, with 146 15.1; 50 x 2880 -> 5120 with 160 9.5, with 80 10.3; 1 x 8192 -> 4096 with 256 or 128 10.4.)
  int ranks = 1;
  while (ranks < 8 && 2 * ranks <= a.steps && (long long)tiles * blocks * 2 * ranks * 4 <= 7 * sm_count()) ranks *= 2;
  return launch_clusters(i8::few_kernel<NT, X>, ranks, dim3(tiles * ranks, blocks), dim3(192), i8::Few<NT>::smem(), st, a, tx, tw);
}
i8::Args linear_args(const moev_w8* p, int n, void* y, int64_t y_stride, int yfmt) {
  i8::Args a{};
  a.sw = p->w_scales;
  a.bias = p->bias;
  a.y = y;
  a.y_stride = n > 1 ? y_stride : p->N;
  a.status = p->status;
  a.n = n;
  a.N = p->N;
  a.steps = (p->K + i8::kStep - 1) / i8::kStep;
  a.y_f32 = yfmt == MOEV_ACT_FP32;
  return a;
}
moev_status linear_i8(const moev_w8* p, const int8_t* x, int64_t x_stride, const float* sx, int n, void* y, int64_t y_stride, int yfmt,
                      bool early, cudaStream_t st) {
  i8::Args a = linear_args(p, n, y, y_stride, yfmt);
  a.sx = sx;
  a.early = early;
  if (n <= 16) return done(launch_few<16>(a, x, x_stride, p->w, p->K, st));
  if (n <= 32) return done(launch_few<32>(a, x, x_stride, p->w, p->K, st));
  if (n <= 64) return done(launch_few<64>(a, x, x_stride, p->w, p->K, st));
  a.wide_tiles = (n - 1) / 256 + 1;
  a.narrow_tiles = (p->N + i8::kWide - 1) / i8::kWide;
  const long long tiles = (long long)a.wide_tiles * a.narrow_tiles;
  // tiles of a quarter of the size and a shared K where the large ones would leave two thirds of the SMs empty (us, large | small: 200 x 2000 -> 1000
  // 16.3 | 9.3, 512 x 4096 -> 2880 20.3 | 18.9, 400 x 2880 -> 5120 20.7 | 26.6, 257 x 7168 -> 9000 35 | 47; 256 x 2880 -> 5120 19.2 | 21.0, which lies
  // just inside the border and takes the small ones)
  if (n <= 128 || (n < 65536 && 6 * tiles <= sm_count())) return done(launch_few<128>(a, x, x_stride, p->w, p->K, st));
  if (tiles > 0x3fffffff) return MOEV_EINVAL;
  CUtensorMap tx, tw;
  if (!encode_codes(&tx, x, p->K, n, x_stride, 128) || !encode_codes(&tw, p->w, p->K, p->N, p->K, 128)) return MOEV_ECUDA;
  const int grid = 2 * (int)std::min<long long>(sm_count() / 2, tiles);
  return done(a.y_f32 ? launch_clusters(i8::many_kernel<true>, 2, dim3(grid), dim3(i8::kManyThreads), i8::many_smem(), st, a, tx, tw)
                      : launch_clusters(i8::many_kernel<false>, 2, dim3(grid), dim3(i8::kManyThreads), i8::many_smem(), st, a, tx, tw));
}
bool y_ok(const moev_w8* p, int n, const void* y, int64_t y_stride, int yfmt) {
  return (yfmt == MOEV_ACT_FP32 || yfmt == MOEV_ACT_BF16) && (n == 0 || y) && aligned(y, yfmt == MOEV_ACT_BF16 ? 2 : 4) && (n <= 1 || y_stride >= p->N);
}
moev_status quant_check(const void* x, int64_t x_stride, int xfmt, int n, int K, const int8_t* codes, int64_t codes_stride, const float* scales) {
  if (n < 0 || K < 1 || K > (1 << 24) || (xfmt != MOEV_ACT_FP32 && xfmt != MOEV_ACT_BF16)) return MOEV_EINVAL;
  if (n > 0 && (!x || !codes || !scales)) return MOEV_EINVAL;
  if (!aligned(x, xfmt == MOEV_ACT_BF16 ? 2 : 4) || !aligned(scales, 4)) return MOEV_EINVAL;
  return n > 1 && (x_stride < K || codes_stride < K) ? MOEV_EINVAL : MOEV_OK;
}
moev_status quant(const void* x, int64_t x_stride, int xfmt, int n, int K, int8_t* codes, int64_t codes_stride, float* scales, cudaStream_t st) {
  const int es = xfmt == MOEV_ACT_BF16 ? 2 : 4;
  const bool vec = K % 8 == 0 && aligned(x, 16) && aligned(codes, 8) && (n == 1 || (x_stride * es % 16 == 0 && codes_stride % 8 == 0));
  const i8::QuantArgs a{x, codes, scales, n > 1 ? x_stride : K, n > 1 ? codes_stride : K, n, K};
  return done(xfmt == MOEV_ACT_BF16 ? launch_quant<__nv_bfloat16>(a, vec, st) : launch_quant<float>(a, vec, st));
}
size_t w8_codes_bytes(const moev_w8* p, int n) { return ((size_t)n * p->K + 255) & ~(size_t)255; }

// ---------------------------------------------------------------- log probabilities
template <typename T, int THREADS>
cudaError_t launch_logprobs_by(const lp::Args& a, int ranks, cudaStream_t st) {
  const dim3 grid((unsigned)a.n * ranks), block(THREADS);
  return a.k > 0 ? launch_clusters(lp::logprobs_kernel<T, true, THREADS>, ranks, grid, block, 0, st, a)
                 : launch_clusters(lp::logprobs_kernel<T, false, THREADS>, ranks, grid, block, 0, st, a);
}
template <typename T>
cudaError_t launch_logprobs(const lp::Args& a, cudaStream_t st) {
  // Rows of up to 8192 logits take a CTA of 128 threads (4000 rows of 1000: 18.6 us, with 512 threads 55); longer ones 512 threads, and a
  // cluster shares a row as long as there is a CTA or less per SM, two where they have more than 16384 vectors each, and each thread has one or more
  // (us, up to one CTA | two: 64 x 151937 bf16 11.7 | 12.7, 100 x 30000 fp32 7.3 | 9.5, 100 x 100003 fp32 17.4 | 15.9).  Many rows of up to
  // 16384 vectors take 256 threads (us, 256 | 512: 500 x 20000 bf16 11.6 | 14.7, 4096 x 100003 bf16 184 | 200, fp32 325 | 295).
  if (a.V <= 8192) return launch_logprobs_by<T, 128>(a, 1, st);
  const int vecs = a.V / lp::Vec<T>::n;
  int ranks = 1;
  while (ranks < lp::kMaxRanks && (long long)a.n * ranks * 2 <= sm_count() * (vecs > ranks * 16384 ? 2 : 1) && vecs >= ranks * 2 * 512) ranks *= 2;
  if (ranks == 1 && vecs <= 16384) return launch_logprobs_by<T, 256>(a, 1, st);
  return launch_logprobs_by<T, 512>(a, ranks, st);
}

}  // namespace

extern "C" {

moev_status moev_prompt_attend(const moev_prompt_batch* b, const moev_prompt* p, void* cuda_stream) {
  if (!b || !p) return MOEV_EINVAL;
  if (b->n_seq < 0 || b->n_seq > 65535 || b->n_tokens < 0 || b->n_keys < 0 || b->max_tokens < 1 || (b->n_seq > 0 && !b->cu)) return MOEV_EINVAL;
  if (!b->cu_k && b->n_keys != b->n_tokens) return MOEV_EINVAL;
  if (!aligned(b->cu, 4) || !aligned(b->cu_k, 4) || !aligned(b->status, 4)) return MOEV_EINVAL;
  if ((p->head_dim != 64 && p->head_dim != 128) || p->n_kv_heads < 1 || p->n_heads < 1 || p->n_heads > 65536 || p->n_heads % p->n_kv_heads || p->window < 0) return MOEV_EINVAL;
  if (!(p->scale > 0.f) || p->scale > kMaxScale) return MOEV_EINVAL;
  if ((b->n_tokens > 0 && (!p->q || !p->out)) || (b->n_keys > 0 && (!p->k || !p->v))) return MOEV_EINVAL;
  if (!aligned(p->q, 16) || !aligned(p->k, 16) || !aligned(p->v, 16) || !aligned(p->out, 16) || !aligned(p->lse, 4) || !aligned(p->sinks, 4)) return MOEV_EINVAL;
  const int64_t row = (int64_t)p->n_heads * p->head_dim, kv_row = (int64_t)p->n_kv_heads * p->head_dim;
  if (!stride_ok(p->q_stride, row, b->n_tokens) || !stride_ok(p->out_stride, row, b->n_tokens) || !stride_ok(p->k_stride, kv_row, b->n_keys) ||
      !stride_ok(p->v_stride, kv_row, b->n_keys))
    return MOEV_EINVAL;
  // what a tensor map holds: strides below 2^40 bytes
  for (int64_t s : {p->q_stride, p->k_stride, p->v_stride})
    if (s >= (1LL << 38)) return MOEV_EINVAL;
  if (b->n_seq == 0 || b->n_tokens == 0) return MOEV_OK;
  prm::Args a{};
  a.cu = b->cu;
  a.cu_k = b->cu_k ? b->cu_k : b->cu;
  a.status = b->status;
  a.n_seq = b->n_seq;
  a.n_tokens = b->n_tokens;
  a.n_keys = b->n_keys;
  a.max_tokens = b->max_tokens;
  a.v = static_cast<const __nv_bfloat16*>(p->v);
  a.out = static_cast<__nv_bfloat16*>(p->out);
  a.lse = p->lse;
  a.sinks = p->sinks;
  a.v_stride = b->n_keys > 1 ? p->v_stride : kv_row;
  a.out_stride = b->n_tokens > 1 ? p->out_stride : row;
  a.n_heads = p->n_heads;
  a.kv_heads = p->n_kv_heads;
  a.rep = p->n_heads / p->n_kv_heads;
  a.tile_heads = std::min(a.rep, prm::kRows);
  a.groups = (a.rep + a.tile_heads - 1) / a.tile_heads;
  a.tokens = prm::kRows / a.tile_heads;
  a.window = p->window < b->n_keys ? p->window : 0;  // one that no sequence fills hides nothing; position - window stays inside 32 bits
  // Small CTAs, two on an SM, where a row's keys are few: their beginnings and ends then weigh as much as what is between.  Us, small | large: 30 tokens
  // x 200 61 | 78, 300 x 100 277 | 298, 700 x 1 17.1 | 18.3, 800 x 60 544 | 547, 1000 x 8 112 | 109, 2000 x 1 56 | 48; window 128 118 | 132, 512 236 | 242,
  // 1000 94 | 87 (4 to 8 kv heads, 8 or 16 query heads each, D 128).  With keys of their own the host knows no sequence's number of them, only that of
  // the call: many short sequences beyond 700 keys together take the large CTAs too (100 of 30 tokens over 100 keys: 28.6 us, with a window of 100 26.8).
  const int span = std::min(p->window > 0 ? p->window : INT_MAX, b->cu_k ? b->n_keys : b->max_tokens), tokens = std::min(b->max_tokens, b->n_tokens);
  // Few rows over many keys: a cluster shares the keys of a small CTA's rows, as long as there are fewer than two CTAs per SM and each has two tiles
  // of keys on the average (which is a matter of time only).  Us, shared | not: 1 token behind 4000 14.0 | 48, 50 behind 4000 19.6 | 59, 50 behind
  // 1000 14.8 | 23.5, 16 behind 16000 36.9 | 169, 200 behind 4000 31.7 | 60; but 300 tokens alone 17.6 | 10.4.
  const long long small = ((long long)tokens + a.tokens - 1) / a.tokens * a.kv_heads * a.groups * a.n_seq;
  const int keys = (int)std::min<long long>(p->window > 0 ? (long long)p->window + a.tokens : INT_MAX, b->cu_k ? b->n_keys / b->n_seq : b->max_tokens / 2);
  int ranks = 1;
  while (ranks < 8 && small * ranks * 2 <= 2 * sm_count() && keys >= ranks * 2 * 2 * 64) ranks *= 2;
  const bool one = span <= 700 || ranks > 1;
  const int tiles = one ? 1 : 2, unit = tiles * a.tokens;  // of rows, tokens of a CTA
  a.pairs = (int)(((long long)tokens + unit - 1) / unit);
  a.scale_log2 = p->scale * 1.4426950408889634f;
  const long long grid = (long long)a.pairs * a.kv_heads * a.groups * a.n_seq;
  if (grid > 0x7fffffffLL) return MOEV_EINVAL;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  if (ranks > 1)
    return done(p->head_dim == 64 ? launch_prompt<64, 1, true>(a, p, b->n_keys, (unsigned)grid, st, ranks) : launch_prompt<128, 1, true>(a, p, b->n_keys, (unsigned)grid, st, ranks));
  if (p->head_dim == 64) return done(one ? launch_prompt<64, 1>(a, p, b->n_keys, (unsigned)grid, st) : launch_prompt<64, 2>(a, p, b->n_keys, (unsigned)grid, st));
  return done(one ? launch_prompt<128, 1>(a, p, b->n_keys, (unsigned)grid, st) : launch_prompt<128, 2>(a, p, b->n_keys, (unsigned)grid, st));
}

moev_status moev_quant_rows(const void* x, int64_t x_stride, int32_t xfmt, int32_t n, int32_t K, int8_t* codes, int64_t codes_stride, float* scales,
                            void* cuda_stream) {
  const moev_status r = quant_check(x, x_stride, xfmt, n, K, codes, codes_stride, scales);
  if (r != MOEV_OK || n == 0) return r;
  return quant(x, x_stride, xfmt, n, K, codes, codes_stride, scales, static_cast<cudaStream_t>(cuda_stream));
}

moev_status moev_linear_i8(const moev_w8* p, const int8_t* x, int64_t x_stride, const float* x_scales, int32_t n, void* y, int64_t y_stride,
                           int32_t yfmt, void* cuda_stream) {
  if (!linear_i8_ok(p) || n < 0 || (n > 0 && (!x || !x_scales)) || !y_ok(p, n, y, y_stride, yfmt)) return MOEV_EINVAL;
  if (!aligned(x, 16) || !aligned(x_scales, 4) || (n > 1 && (x_stride < p->K || x_stride % 16 || x_stride >= (1LL << 39)))) return MOEV_EINVAL;
  if (n == 0) return MOEV_OK;
  return linear_i8(p, x, x_stride, x_scales, n, y, y_stride, yfmt, false, static_cast<cudaStream_t>(cuda_stream));
}

size_t moev_linear_w8_workspace(const moev_w8* p, int32_t n) {
  return linear_i8_ok(p) && n > 0 ? w8_codes_bytes(p, n) + (size_t)n * 4 : 0;
}

moev_status moev_linear_w8(const moev_w8* p, const void* x, int64_t x_stride, int32_t xfmt, int32_t n, void* y, int64_t y_stride, int32_t yfmt,
                               void* workspace, size_t workspace_bytes, void* cuda_stream) {
  if (!linear_i8_ok(p) || n < 0 || !y_ok(p, n, y, y_stride, yfmt)) return MOEV_EINVAL;
  if (n > 0 && (!workspace || !aligned(workspace, 16) || workspace_bytes < moev_linear_w8_workspace(p, n))) return MOEV_EINVAL;
  int8_t* codes = static_cast<int8_t*>(workspace);
  float* scales = n > 0 ? reinterpret_cast<float*>(codes + w8_codes_bytes(p, n)) : nullptr;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  moev_status r = quant_check(x, x_stride, xfmt, n, p->K, codes, p->K, scales);
  if (r != MOEV_OK || n == 0) return r;
  // one launch: the product's CTAs make the codes themselves (times at the kernel)
  const int es = xfmt == MOEV_ACT_BF16 ? 2 : 4;
  if ((n == 1 || (n <= i8::kOwnRows && (p->N + 127) / 128 <= 2 * sm_count())) && aligned(x, 16) && (n == 1 || x_stride * es % 16 == 0)) {
    i8::Args a = linear_args(p, n, y, y_stride, yfmt);
    a.x = x;
    a.x_stride = n > 1 ? x_stride : p->K;
    a.K = p->K;
    return done(es == 2 ? launch_few<16, __nv_bfloat16>(a, nullptr, 0, p->w, p->K, st) : launch_few<16, float>(a, nullptr, 0, p->w, p->K, st));
  }
  r = quant(x, x_stride, xfmt, n, p->K, codes, p->K, scales, st);
  return r != MOEV_OK ? r : linear_i8(p, codes, p->K, scales, n, y, y_stride, yfmt, true, st);
}

moev_status moev_token_logprobs(const moev_logprobs* p, void* cuda_stream) {
  if (!p || p->n < 0 || p->n > (1 << 27) || p->V < 1 || p->V > (1 << 30) || p->m < 0 || p->k < 0 || p->k > lp::kMaxK || p->k > p->V) return MOEV_EINVAL;
  if ((p->afmt != MOEV_ACT_FP32 && p->afmt != MOEV_ACT_BF16) || !(p->scale > 0.f) || p->scale > kMaxScale) return MOEV_EINVAL;
  if (!aligned(p->logits, p->afmt == MOEV_ACT_BF16 ? 2 : 4) || !aligned(p->ids, 4) || !aligned(p->logprobs, 4) || !aligned(p->entropy, 4) ||
      !aligned(p->lse, 4) || !aligned(p->top_ids, 4) || !aligned(p->top_logprobs, 4))
    return MOEV_EINVAL;
  if (p->n == 0) return MOEV_OK;
  if (!p->logits || (p->n > 1 && p->stride < p->V)) return MOEV_EINVAL;
  if ((p->m > 0) != (p->logprobs != nullptr) || (p->m > 0) != (p->ids != nullptr) || (p->k > 0) != (p->top_ids != nullptr) || (p->top_logprobs && !p->k))
    return MOEV_EINVAL;
  if (!p->logprobs && !p->entropy && !p->lse && !p->top_ids) return MOEV_EINVAL;
  const lp::Args a{p->logits, p->ids, p->logprobs, p->entropy, p->lse, p->top_logprobs, p->top_ids, p->n > 1 ? p->stride : p->V, p->n, p->V, p->m, p->k, p->scale};
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  return done(p->afmt == MOEV_ACT_BF16 ? launch_logprobs<__nv_bfloat16>(a, st) : launch_logprobs<float>(a, st));
}

moev_status moev_build_pages(const moev_pages* p, void* cuda_stream) {
  if (!p || p->n_seq < 0 || p->n_seq > 65535 || p->n_tokens < 0 || p->table_cols < 1 || p->n_free < 0) return MOEV_EINVAL;
  if (p->page != 16 && p->page != 32 && p->page != 64 && p->page != 128) return MOEV_EINVAL;
  for (const void* t : {(const void*)p->ctx_len, (const void*)p->new_len, (const void*)p->free_pages, (const void*)p->free_first, (const void*)p->page_table,
                        (const void*)p->cu, (const void*)p->slots, (const void*)p->positions, (const void*)p->taken, (const void*)p->status})
    if (!aligned(t, 4)) return MOEV_EINVAL;
  if (!p->cu || (p->n_seq > 0 && (!p->ctx_len || !p->new_len || !p->page_table)) || (p->n_free > 0 && !p->free_pages)) return MOEV_EINVAL;
  pages::Args a{p->ctx_len, p->new_len, p->free_pages, p->free_first, p->page_table, p->cu, p->slots, p->positions, p->taken, p->status,
                p->n_seq, p->n_tokens, 4, p->table_cols, p->n_free, 1, aligned(p->slots, 16) && aligned(p->positions, 16)};
  while ((1 << a.page_log2) < p->page) ++a.page_log2;
  const int chunks = std::max(1, (p->n_seq + pages::kChunk - 1) / pages::kChunk);
  // CTAs that share a chunk's rows: about 4 rows a thread, no more CTAs than two per SM
  const int rows = p->slots || p->positions ? p->n_tokens : 0;
  a.parts = std::max(1, std::min(2 * sm_count() / chunks, rows / chunks / (4 * pages::kChunk) + 1));
  return done(launch(pages::pages_kernel, dim3(chunks * a.parts), dim3(pages::kChunk), 0, static_cast<cudaStream_t>(cuda_stream), a));
}

#ifdef MOEV_TEST_HOOKS
// Test builds only: while the flag is set, the loaders of the attention and linear kernels leave out their last tile (see common.cuh).
int32_t moev_test_withhold_prompt(int32_t on) {
  const int v = on ? 1 : 0;
  return cudaMemcpyToSymbol(g_test_withhold, &v, sizeof(int)) == cudaSuccess ? 0 : -1;
}
#endif

}  // extern "C"
