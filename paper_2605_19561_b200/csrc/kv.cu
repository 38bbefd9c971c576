// C-ABI entry points of the 4-bit key/value cache (see include/torq.h): argument validation, kernel selection and launch.
#include <cuda_runtime.h>
#include <atomic>
#include <cfloat>
#include <cmath>
#include <type_traits>

#include "../../include/torq.h"
#include "host_launch.cuh"
#include "kv_attention.cuh"
#include "kv_cache.cuh"
#include "kv_evict.cuh"
#include "kv_prefill.cuh"

namespace torq {

static inline bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

// Checks of the cache itself, and the kernels' view of it.
template <int FMT>
static torq_status kv_view(const torq_kv_cache* c, const int32_t* starts, int64_t tokens, KvView* v) {
  if (!c || !c->pages || !c->table || !c->lengths) return TORQ_ERR_NULL;
  if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256) return TORQ_ERR_SHAPE;
  if (c->page_tokens < 16 || c->page_tokens > 1024 || (c->page_tokens & (c->page_tokens - 1))) return TORQ_ERR_SHAPE;
  if (c->kv_heads < 1 || c->kv_heads > 1024 || c->num_pages < 1 || c->num_pages > INT32_MAX || c->batch < 1 || c->batch > (1 << 16) ||
      c->table_width < 1 || c->table_width > (1 << 30) / c->page_tokens)
    return TORQ_ERR_SHAPE;
  if (tokens < 1 || tokens > (1 << 24) || (!starts && tokens != c->batch)) return TORQ_ERR_SHAPE;
  const bool nv = FMT == FMT_NVFP4;
  if (nv && !(c->k_tensor_scale > 0.f && c->k_tensor_scale <= 3.0e38f && c->v_tensor_scale > 0.f && c->v_tensor_scale <= 3.0e38f)) return TORQ_ERR_SHAPE;
  if (!aligned16(c->pages) || !aligned4(c->table) || !aligned4(c->lengths) || !aligned4(starts)) return TORQ_ERR_ALIGN;
  v->pages = static_cast<uint8_t*>(c->pages);
  v->table = c->table;
  v->lengths = c->lengths;
  v->starts = starts;
  v->batch = (int)c->batch;
  v->num_pages = (int)c->num_pages;
  v->width = (int)c->table_width;
  v->page_shift = __builtin_ctzll((unsigned long long)c->page_tokens);
  v->heads = (int)c->kv_heads;
  v->dim = (int)c->head_dim;
  v->tokens = (int)tokens;
  const int codes = v->dim / 2 << v->page_shift, scales = v->dim / kv_block(FMT) << v->page_shift;
  v->k_scales = codes;
  v->v_codes = codes + scales;
  v->v_scales = 2 * codes + scales;
  v->head_bytes = 2 * (codes + scales);
  v->page_bytes = (int64_t)v->heads * v->head_bytes;
  v->k_ts = nv ? c->k_tensor_scale : 1.f;
  v->v_ts = nv ? c->v_tensor_scale : 1.f;
  return TORQ_OK;
}

static torq_status kv_scoring(const torq_kv_scoring* s, KvScoring* a) {
  if (!s) return TORQ_ERR_NULL;
  if (!(s->scale > 0.f && s->scale <= 1e30f) || !(s->softcap >= 0.f && s->softcap <= 1e30f) || s->window < 0) return TORQ_ERR_SHAPE;
  if (!aligned4(s->slopes) || !aligned4(s->prefix) || !aligned4(s->first)) return TORQ_ERR_ALIGN;
  a->scale = s->scale;
  a->softcap = s->softcap * kLog2e;
  a->per_cap = s->softcap > 0.f ? fminf(1.f / a->softcap, FLT_MAX) : 0.f;   // zero times infinity would be no number
  a->slopes = s->slopes;
  a->prefix = s->prefix;
  a->first = s->first;
  a->window = s->window > (1 << 30) ? 1 << 30 : (int)s->window;
  return TORQ_OK;
}

static torq_status kv_queries(const KvView& v, const void* Q, int64_t q_stride, int64_t heads) {
  if (!Q) return TORQ_ERR_NULL;
  if (heads < 1 || heads % v.heads != 0 || heads > (1 << 16) || q_stride < heads * v.dim || (int64_t)v.tokens * heads > INT32_MAX) return TORQ_ERR_SHAPE;
  if (!aligned16(Q) || q_stride % 8 != 0) return TORQ_ERR_ALIGN;
  return TORQ_OK;
}

static inline unsigned grid_of(int64_t threads, int per_cta, int64_t most) {
  const int64_t n = (threads + per_cta - 1) / per_cta;
  return (unsigned)(n < 1 ? 1 : (n > most ? most : n));
}

// Opts a kernel in to `bytes` of dynamic shared memory, once per device (asked every time it costs the host 0.4 us a call).
template <auto KERNEL>
static bool opt_in(int bytes) {
  static std::atomic<uint64_t> done{0};
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev > 63) return false;
  if (done.load(std::memory_order_relaxed) >> dev & 1) return true;
  if (cudaFuncSetAttribute(KERNEL, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) return false;
  done.fetch_or(1ull << dev, std::memory_order_relaxed);
  return true;
}

// A kernel as a type.
template <auto KERNEL>
struct Kernel {
  static constexpr auto value = KERNEL;
};

template <typename F>
static void with_dim(int dim, F f) {
  if (dim == 64) f(std::integral_constant<int, 64>{});
  else if (dim == 128) f(std::integral_constant<int, 128>{});
  else f(std::integral_constant<int, 256>{});
}

// Tokens of a CTA at a time: one while there are few, so that they spread over the SMs, else four.
template <typename F>
static void with_tokens(int tokens, int sms, F f) {
  if (tokens <= 8 * sms) f(std::integral_constant<int, 1>{}, (unsigned)tokens);
  else f(std::integral_constant<int, 4>{}, grid_of(tokens, 4, (int64_t)sms * 64));
}

template <int FMT>
static torq_status append_impl(const torq_kv_cache* cache, const void* K, const void* V, torq_dtype dtype, int64_t k_stride, int64_t v_stride,
                               const int32_t* starts, int64_t tokens, void* stream) {
  if (!K || !V) return TORQ_ERR_NULL;
  KvView v;
  torq_status rc = kv_view<FMT>(cache, starts, tokens, &v);
  if (rc != TORQ_OK) return rc;
  if ((dtype != TORQ_F32 && dtype != TORQ_BF16) || k_stride < (int64_t)v.heads * v.dim || v_stride < (int64_t)v.heads * v.dim) return TORQ_ERR_SHAPE;
  const int64_t threads = (int64_t)v.tokens * v.heads * (v.dim / 4);
  if (threads > INT32_MAX) return TORQ_ERR_SHAPE;
  const int per16 = dtype == TORQ_F32 ? 4 : 8;
  if (!aligned16(K) || !aligned16(V) || k_stride % per16 != 0 || v_stride % per16 != 0) return TORQ_ERR_ALIGN;
  int sms;
  if ((rc = current_device(&sms, &v.err_word)) != TORQ_OK) return rc;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  with_tokens(v.tokens, sms, [&](auto N, unsigned grid) {
    constexpr int TOKENS = decltype(N)::value;
    if (dtype == TORQ_F32)
      launch_tc(kv_append_kernel<FMT, float, TOKENS>, 1, dim3(grid), dim3(256), 0, s, v, static_cast<const float*>(K), static_cast<const float*>(V), k_stride,
                v_stride);
    else
      launch_tc(kv_append_kernel<FMT, __nv_bfloat16, TOKENS>, 1, dim3(grid), dim3(256), 0, s, v, static_cast<const __nv_bfloat16*>(K),
                static_cast<const __nv_bfloat16*>(V), k_stride, v_stride);
  });
  return launch_status();
}

template <int FMT>
static torq_status read_impl(const torq_kv_cache* cache, const int32_t* starts, int64_t tokens, void* K, void* V, torq_dtype dtype, void* stream) {
  if (!K || !V) return TORQ_ERR_NULL;
  KvView v;
  torq_status rc = kv_view<FMT>(cache, starts, tokens, &v);
  if (rc != TORQ_OK) return rc;
  const int64_t threads = (int64_t)v.tokens * v.heads * (v.dim / 4);
  if ((dtype != TORQ_F32 && dtype != TORQ_BF16) || threads > INT32_MAX) return TORQ_ERR_SHAPE;
  if (!aligned16(K) || !aligned16(V)) return TORQ_ERR_ALIGN;
  int sms;
  if ((rc = current_device(&sms, &v.err_word)) != TORQ_OK) return rc;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  with_tokens(v.tokens, sms, [&](auto N, unsigned grid) {
    constexpr int TOKENS = decltype(N)::value;
    if (dtype == TORQ_F32) launch_tc(kv_read_kernel<FMT, float, TOKENS>, 1, dim3(grid), dim3(256), 0, s, v, static_cast<float*>(K), static_cast<float*>(V));
    else launch_tc(kv_read_kernel<FMT, __nv_bfloat16, TOKENS>, 1, dim3(grid), dim3(256), 0, s, v, static_cast<__nv_bfloat16*>(K), static_cast<__nv_bfloat16*>(V));
  });
  return launch_status();
}

// ---- few queries per sequence
// Warps of the streaming kernel at most: the workspace does not depend on the device.
constexpr int max_ranges(int groups) { return groups == 1 ? 2560 : 1280; }
// Rows of a sequence that are worked on at once, in eights.  Heads of 256: always eight rows, since the registers do not hold more.
static int decode_groups(int64_t tokens, int64_t batch, int64_t heads, int64_t kv_heads, int64_t dim) {
  return dim >= 256 || (tokens + batch - 1) / batch * (heads / kv_heads) <= 8 ? 1 : 2;
}
static size_t decode_workspace(int groups, int64_t dim) { return (size_t)max_ranges(groups) * 2 * 8 * groups * (size_t)(dim + 2) * sizeof(float); }

template <int FMT, int D, int NT>
static torq_status decode_launch(const KvView& v, const KvScoring& a, int sms, const void* Q, int64_t q_stride, int heads, void* out, float* lse,
                                 void* workspace, cudaStream_t s) {
  using C = KvDecodeCfg<FMT, D, NT>;
  constexpr auto kernel = kv_decode_kernel<C>;
  if (!opt_in<kernel>(C::SMEM)) return TORQ_ERR_LAUNCH;
  const int most = sms * C::CTAS, ctas = most < max_ranges(NT) / C::WARPS ? most : max_ranges(NT) / C::WARPS, group = heads / v.heads;
  float* partials = static_cast<float*>(workspace);
  __nv_bfloat16* y = static_cast<__nv_bfloat16*>(out);
  launch_tc(kernel, 1, dim3((unsigned)ctas), dim3(C::THREADS), C::SMEM, s, v, a, static_cast<const __nv_bfloat16*>(Q), q_stride, heads, y, lse, partials);
  const torq_status rc = launch_status();
  if (rc != TORQ_OK) return rc;
  // Items at most: every sequence may have a group that is not full.  No more than there are borders can be cut.  Few items: a row to each CTA, with the ranges
  // shared among its warps.
  const int64_t items = ((int64_t)v.tokens * group / C::ROWS + (v.tokens < v.batch ? v.tokens : v.batch)) * v.heads;
  const int ranges = ctas * C::WARPS;
  const bool by_border = items > ranges - 1;
  const unsigned grid = (unsigned)(by_border ? ranges - 1 : items);
  const float* parts = partials;
  if (items <= 64) launch_tc(kv_join_kernel<D, NT, 8>, 1, dim3(grid, C::ROWS), dim3(256), 0, s, v, a, ranges, by_border, heads, parts, y, lse);
  else launch_tc(kv_join_kernel<D, NT, 1>, 1, dim3(grid, NT), dim3(256), 0, s, v, a, ranges, by_border, heads, parts, y, lse);
  return launch_status();
}

// ---- many queries per sequence
constexpr int kMaxPrefill = 160;         // CTAs; as max_ranges
static size_t prefill_workspace(int64_t dim) { return (size_t)kMaxPrefill * 2 * (dim == 256 ? 128 : 256) * (size_t)(dim + 2) * sizeof(float); }
template <int FMT, int D>
static torq_status prefill_launch(const KvView& v, const KvScoring& a, int sms, const void* Q, int64_t q_stride, int heads, void* out, float* lse,
                                  void* workspace, cudaStream_t s) {
  using C = KvPrefillCfg<FMT, D>;
  constexpr auto kernel = kv_prefill_kernel<C>;
  if (!opt_in<kernel>(C::SMEM)) return TORQ_ERR_LAUNCH;
  const int ctas = sms < kMaxPrefill ? sms : kMaxPrefill;
  float* partials = static_cast<float*>(workspace);
  __nv_bfloat16* y = static_cast<__nv_bfloat16*>(out);
  launch_tc(kernel, 1, dim3((unsigned)ctas), dim3(C::THREADS), C::SMEM, s, v, a, static_cast<const __nv_bfloat16*>(Q), q_stride, heads, y, lse, partials);
  const torq_status rc = launch_status();
  if (rc != TORQ_OK || ctas == 1) return rc;
  launch_tc(kv_prefill_join_kernel<C>, 1, dim3((unsigned)ctas - 1, C::ROWS / 32), dim3(256), 0, s, v, a, ctas, heads, static_cast<const float*>(partials), y, lse);
  return launch_status();
}
// Which of the two: the streaming kernel widens the cache anew for every 16 rows of a head (8 of 256 dimensions), the other once for 256 (128), but takes as long for
// one row as for all.  Measured, streaming against the other, us, by rows on average:
//   one sequence of 32768 tokens, 8 heads of 128: 64 rows 62, 65;  96: 87, 69;  512: 380, 126;  of 256: 64 rows 124, 122;  128: 226, 140
//   16 sequences of up to 5000 tokens, 8 heads of 128: about 45 rows 73, 102;  65: 94, 102;  90: 142, 103
//   64 sequences of up to 3000 tokens, 4 heads of 128: about 45 rows 92, 127;  65: 136, 127
// The rule knows the average alone, and these batches are of sequences alike.  Where many decode and one brings a prompt, all of them get one kernel, and the sequences
// that it is not meant for take longer than they would by themselves.
static bool many_rows(int64_t tokens, int64_t batch, int64_t heads, int64_t kv_heads) {
  return tokens / batch * (heads / kv_heads) >= 64;
}

template <int FMT>
static torq_status attention_impl(const torq_kv_cache* cache, const torq_kv_scoring* scoring, const void* Q, int64_t q_stride, int64_t heads,
                                  const int32_t* starts, int64_t tokens, void* out, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  if (!out) return TORQ_ERR_NULL;
  KvView v;
  KvScoring a;
  torq_status rc = kv_view<FMT>(cache, starts, tokens, &v);
  if (rc == TORQ_OK) rc = kv_scoring(scoring, &a);
  if (rc == TORQ_OK) rc = kv_queries(v, Q, q_stride, heads);
  if (rc != TORQ_OK) return rc;
  if (!aligned16(out) || !aligned4(lse)) return TORQ_ERR_ALIGN;
  const size_t need = torq_kv_attention_workspace_bytes(tokens, cache->batch, heads, v.heads, v.dim);
  if (need && (!workspace || workspace_bytes < need)) return TORQ_ERR_WORKSPACE;
  if ((reinterpret_cast<uintptr_t>(workspace) & 255u) != 0) return TORQ_ERR_ALIGN;
  int sms;
  if ((rc = current_device(&sms, &v.err_word)) != TORQ_OK) return rc;
  cudaStream_t stm = static_cast<cudaStream_t>(stream);
  const int groups = decode_groups(tokens, cache->batch, heads, v.heads, v.dim);
  const bool many = many_rows(tokens, cache->batch, heads, v.heads);
  with_dim(v.dim, [&](auto DIM) {
    constexpr int D = decltype(DIM)::value;
    if (many) rc = prefill_launch<FMT, D>(v, a, sms, Q, q_stride, (int)heads, out, lse, workspace, stm);
    else if (groups == 1) rc = decode_launch<FMT, D, 1>(v, a, sms, Q, q_stride, (int)heads, out, lse, workspace, stm);
    else if constexpr (D < 256) rc = decode_launch<FMT, D, 2>(v, a, sms, Q, q_stride, (int)heads, out, lse, workspace, stm);
  });
  return rc;
}

template <int FMT>
static torq_status weights_impl(const torq_kv_cache* cache, const torq_kv_scoring* scoring, const void* Q, int64_t q_stride, int64_t heads,
                                const int32_t* starts, int64_t tokens, const float* lse, const float* weights, float* weights_out, void* stream) {
  if (!lse || !weights || !weights_out) return TORQ_ERR_NULL;
  KvView v;
  KvScoring a;
  torq_status rc = kv_view<FMT>(cache, starts, tokens, &v);
  if (rc == TORQ_OK) rc = kv_scoring(scoring, &a);
  if (rc == TORQ_OK) rc = kv_queries(v, Q, q_stride, heads);
  if (rc != TORQ_OK) return rc;
  if (!aligned4(lse) || !aligned16(weights) || !aligned16(weights_out)) return TORQ_ERR_ALIGN;
  int sms;
  if ((rc = current_device(&sms, &v.err_word)) != TORQ_OK) return rc;
  // By single warps up to one group of eight rows, on average.  Measured, single warps against CTAs, us: 16 sequences of up to 5000 tokens, 8 heads of 128: 8 rows
  // 18.6, 21.6; 12 rows 37.4, 23.1; 64: 91.3, 42.6.  One sequence of 32768 tokens, 8 heads of 256: 8 rows 20.1, 32.1; 12: 55.0, 39.2; 64: 186, 80
  const bool one = (tokens + cache->batch - 1) / cache->batch * (heads / v.heads) <= 8;
  with_dim(v.dim, [&](auto DIM) {
    constexpr int D = decltype(DIM)::value;
    auto run = [&](auto kernel, auto config) {
      using C = decltype(config);
      if (!opt_in<decltype(kernel)::value>(C::SMEM)) {
        rc = TORQ_ERR_LAUNCH;
        return;
      }
      launch_tc(decltype(kernel)::value, 1, dim3((unsigned)(sms * C::CTAS)), dim3(C::THREADS), C::SMEM, static_cast<cudaStream_t>(stream), v, a,
                static_cast<const __nv_bfloat16*>(Q), q_stride, (int)heads, lse, weights, weights_out);
      rc = launch_status();
    };
    using One = KvWeightsCfg<FMT, D>;
    using Rows = KvRowWeightsCfg<FMT, D>;
    if (one) run(Kernel<kv_weights_kernel<One>>{}, One{});
    else run(Kernel<kv_row_weights_kernel<Rows>>{}, Rows{});
  });
  return rc;
}

template <int FMT>
static torq_status evict_impl(const torq_kv_cache* cache, float* weights, const int32_t* new_table, int64_t new_width, int64_t keep, int64_t recent,
                              int32_t* new_lengths, int32_t* kept, void* stream) {
  if (!weights || !new_table || !new_lengths || !kept) return TORQ_ERR_NULL;
  KvView v;
  torq_status rc = kv_view<FMT>(cache, nullptr, cache ? cache->batch : 0, &v);
  if (rc != TORQ_OK) return rc;
  const int64_t room = (int64_t)v.width << v.page_shift;
  if (keep < 1 || keep > (1 << 30) || recent < 0 || recent > keep || new_width < 1 || new_width > (1 << 26) ||
      (new_width << v.page_shift) < (keep < room ? keep : room) || (int64_t)v.batch * v.heads > 65535)
    return TORQ_ERR_SHAPE;
  if (!aligned16(weights) || !aligned4(new_table) || !aligned4(new_lengths) || !aligned4(kept)) return TORQ_ERR_ALIGN;
  int sms;
  if ((rc = current_device(&sms, &v.err_word)) != TORQ_OK) return rc;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const unsigned items = (unsigned)(v.batch * v.heads);
  // CTAs per sequence and head: as many as the SMs have room for, each with 2048 tokens at least
  int cluster = 1;
  while (cluster < 8 && (int64_t)items * cluster * 2 <= sms && room / (cluster * 2) >= 2048) cluster *= 2;
  if (!opt_in<kv_select_kernel>(KvSelectCfg::SMEM)) return TORQ_ERR_LAUNCH;
  launch_tc(kv_select_kernel, cluster, dim3(items * cluster), dim3(KvSelectCfg::THREADS), KvSelectCfg::SMEM, s, v, static_cast<const float*>(weights), (int)keep,
            (int)recent, cluster, new_lengths, kept);
  if ((rc = launch_status()) != TORQ_OK) return rc;
  const int64_t moved = keep < room ? keep : room;
  launch_tc(kv_move_kernel<FMT>, 1, dim3(grid_of(moved * (v.dim / 16), 1024, 4096), items), dim3(256), 0, s, v, weights, new_table, (int)new_width, (int)keep,
            static_cast<const int32_t*>(kept));
  return launch_status();
}

}  // namespace torq

using namespace torq;

extern "C" {

size_t torq_kv_page_bytes(int64_t scale_block, int64_t page_tokens, int64_t head_dim) {
  if ((scale_block != 16 && scale_block != 32) || page_tokens < 1 || head_dim < 1) return 0;
  return (size_t)(2 * page_tokens * (head_dim / 2 + head_dim / scale_block));
}

size_t torq_kv_attention_workspace_bytes(int64_t tokens, int64_t batch, int64_t heads, int64_t kv_heads, int64_t head_dim) {
  if (tokens < 1 || batch < 1 || heads < 1 || kv_heads < 1 || heads % kv_heads != 0 || head_dim < 1) return 0;
  return many_rows(tokens, batch, heads, kv_heads) ? prefill_workspace(head_dim)
                                                   : decode_workspace(decode_groups(tokens, batch, heads, kv_heads, head_dim), head_dim);
}

#define TORQ_KV_ENTRIES(name, FMT)                                                                                                                   \
  torq_status torq_##name##_kv_append(const torq_kv_cache* cache, const void* K, const void* V, torq_dtype dtype, int64_t k_stride, int64_t v_stride, \
                                      const int32_t* starts, int64_t tokens, void* stream) {                                                         \
    return append_impl<FMT>(cache, K, V, dtype, k_stride, v_stride, starts, tokens, stream);                                                         \
  }                                                                                                                                                  \
  torq_status torq_##name##_kv_read(const torq_kv_cache* cache, const int32_t* starts, int64_t tokens, void* K, void* V, torq_dtype dtype,           \
                                    void* stream) {                                                                                                  \
    return read_impl<FMT>(cache, starts, tokens, K, V, dtype, stream);                                                                               \
  }                                                                                                                                                  \
  torq_status torq_##name##_kv_attention(const torq_kv_cache* cache, const torq_kv_scoring* scoring, const void* Q, int64_t q_stride, int64_t heads,  \
                                         const int32_t* starts, int64_t tokens, void* out, float* lse, void* workspace, size_t workspace_bytes,      \
                                         void* stream) {                                                                                             \
    return attention_impl<FMT>(cache, scoring, Q, q_stride, heads, starts, tokens, out, lse, workspace, workspace_bytes, stream);                    \
  }                                                                                                                                                  \
  torq_status torq_##name##_kv_weights(const torq_kv_cache* cache, const torq_kv_scoring* scoring, const void* Q, int64_t q_stride, int64_t heads,    \
                                       const int32_t* starts, int64_t tokens, const float* lse, const float* weights, float* weights_out,            \
                                       void* stream) {                                                                                               \
    return weights_impl<FMT>(cache, scoring, Q, q_stride, heads, starts, tokens, lse, weights, weights_out, stream);                                 \
  }                                                                                                                                                  \
  torq_status torq_##name##_kv_evict(const torq_kv_cache* cache, float* weights, const int32_t* new_table, int64_t new_width, int64_t keep,           \
                                     int64_t recent, int32_t* new_lengths, int32_t* kept, void* stream) {                                            \
    return evict_impl<FMT>(cache, weights, new_table, new_width, keep, recent, new_lengths, kept, stream);                                           \
  }
TORQ_KV_ENTRIES(mxfp4, FMT_MXFP4)
TORQ_KV_ENTRIES(nvfp4, FMT_NVFP4)
TORQ_KV_ENTRIES(mxint4, FMT_MXINT4)

}  // extern "C"
