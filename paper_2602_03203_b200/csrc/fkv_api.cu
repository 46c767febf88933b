// Host side of the C ABI declared in include/fkv.h: argument checks, the
// carve-up of the caller's workspace, a host mirror of the segment lengths
// (lengths evolve deterministically, so no call reads them back), and the
// kernel launches.  No device memory is allocated here.
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>
#include <string.h>

#include <algorithm>
#include <atomic>
#include <cmath>
#include <new>
#include <string>
#include <utility>
#include <vector>

#include "../../include/fkv.h"
#include "fkv_attend.cuh"
#include "fkv_aux.cuh"
#include "fkv_chunk.cuh"
#include "fkv_chunk_features.cuh"
#include "fkv_compact.cuh"
#include "fkv_dev.cuh"
#include "fkv_features.cuh"
#include "fkv_fork.cuh"
#include "fkv_golden.cuh"
#include "fkv_rkv.cuh"
#include "fkv_score.cuh"
#include "fkv_select.cuh"
#include "fkv_tree.cuh"
#include "fkv_tree_attend.cuh"
#include "fkv_verify.cuh"

using namespace fkv;

namespace {

thread_local std::string g_cuda_error;

constexpr int kScorePPS = 8;  // consumer warps of the scorer = pages per tile
constexpr int kAttendMinPages = 4;
constexpr size_t kMaxSmem = 227 * 1024;

inline size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

// The dynamic shared-memory opt-in is a per-device attribute of a kernel: remember, per kernel and per
// device, the largest size already granted, and ask again only for more.
struct SmemOptIn {
  size_t granted[64] = {};
  template <class Kernel>
  cudaError_t ensure(Kernel kernel, size_t bytes) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    size_t &g = granted[dev & 63];
    if (bytes <= g) return cudaSuccess;
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (e == cudaSuccess) g = bytes;
    return e;
  }
};

struct Layout {
  size_t pool, free_stack, ctrl, planhdr, pt, pt_new, len, budget, sp, scores, idx, plan, work, tile1, seq_tickets, seq_fail, att_part, att_tickets, hist_q, hist_mp, hist_n, hist_cnt, chunk_part, chunk_ml, chunk_info, total;
  int cap, max_pages, num_pages, page_bytes, F, att_smax, sp_stride, sp_off_wf, sp_off_b1, sp_off_w2, sp_off_b2;
};

bool valid_config(const fkv_config *c) {
  if (!c) return false;
  if (c->num_layers < 1 || c->num_kv_heads < 1 || c->num_kv_heads > 32 || c->max_batch < 1 || c->max_batch > kMaxBatch)
    return false;
  if (c->group_size < 1 || c->group_size > 8) return false;
  if (c->head_dim != 64 && c->head_dim != 128) return false;
  if (c->page_size != kPage || c->scorer_hidden != kHidden) return false;
  if (c->activation < 0 || c->activation > 3) return false;
  if (c->budget < 1 || c->recent_keep < 0 || c->max_tokens_per_head < 1 || c->num_pages < 0) return false;
  if ((int64_t)c->num_layers * c->max_batch * c->num_kv_heads > (1 << 20)) return false;
  if (c->feature_window < 0 || c->feature_window % 8) return false;
  if (c->feature_window > kFeatMaxQueries) return false;
  return true;
}

Layout make_layout(const fkv_config &c) {
  Layout L{};
  const int D = c.head_dim;
  L.F = 6 * c.group_size;
  L.cap = (int)align_up((size_t)c.max_tokens_per_head, kPage);
  L.max_pages = L.cap / kPage;
  L.page_bytes = 64 * D + 64 * L.F + 64;
  const size_t nseg = (size_t)c.num_layers * c.max_batch * c.num_kv_heads;
  const int bpages = (std::min(c.budget, L.cap) + kPage - 1) / kPage;
  L.num_pages = c.num_pages ? c.num_pages : (int)std::min<size_t>(nseg * ((size_t)L.max_pages + bpages + 1), 0x7fffffff);
  const int KS = 2 * D / 16;
  L.sp_off_wf = 2 * KS * 512;   // fragments of the roundings, then of the remainders
  L.sp_off_b1 = L.sp_off_wf + ScoreSmem::fk(L.F) * 1024;   // feature rows: tf32 fragments, truncations and remainders
  L.sp_off_w2 = L.sp_off_b1 + 64;
  L.sp_off_b2 = L.sp_off_w2 + 64;
  L.sp_stride = (int)align_up((size_t)L.sp_off_b2 + 16, 256);
  size_t off = 0;
  auto take = [&](size_t bytes) { size_t o = off; off = align_up(off + bytes, 256); return o; };
  L.pool = take((size_t)L.num_pages * L.page_bytes);
  L.free_stack = take((size_t)L.num_pages * 4);
  L.ctrl = take(CTRL_WORDS * 4);
  L.planhdr = take(PH_WORDS * 4);
  L.pt = take(nseg * L.max_pages * 4);
  L.pt_new = take(nseg * L.max_pages * 4);
  L.len = take((size_t)c.num_layers * c.max_batch * 4);
  L.budget = take((size_t)c.max_batch * 4);   // (behind the lengths: fkv_sync_lengths reads both at once)
  L.sp = take((size_t)c.num_layers * c.num_kv_heads * L.sp_stride);
  L.scores = take(nseg * L.cap * 4);
  L.idx = take(nseg * L.cap * 4);
  L.plan = take(nseg * sizeof(SegPlan));
  L.work = take(nseg * 4);
  L.tile1 = take((nseg + 1) * 4);
  L.seq_tickets = take((size_t)c.num_layers * c.max_batch * 4);
  L.seq_fail = take((size_t)c.num_layers * c.max_batch * 4);
  // Split-K attention: up to att_smax splits per segment (enough for a few CTAs per SM at this batch size).
  L.att_smax = std::max(1, std::min(kMaxSplits, 512 / (c.max_batch * c.num_kv_heads)));
  L.att_part = take(nseg * L.att_smax * c.group_size * (D + 4) * 4);
  L.att_tickets = take(nseg * 4);
  const size_t ls = (size_t)c.num_layers * c.max_batch, W = (size_t)c.feature_window, Hq = (size_t)c.num_kv_heads * c.group_size;
  const size_t Wp = (W + 15) & ~(size_t)15;   // rows of one query tile
  L.hist_q = take(ls * Wp * Hq * D * 2);
  L.hist_mp = take(ls * Wp * Hq * 4);
  L.hist_n = take(ls * W * 4);
  L.hist_cnt = take(W ? ls * 4 : 0);
  // Attention over chunks: two slots of 2 x 128 query rows per CTA, whatever the shape of the cache.
  L.chunk_part = take((size_t)kChunkCtas * 2 * 256 * D * 4);
  L.chunk_ml = take((size_t)kChunkCtas * 2 * 256 * 8);
  L.chunk_info = take((size_t)kChunkCtas * kChunkInfo * 4);
  L.total = off;
  return L;
}

uint16_t f32_to_bf16_rne(float f) {
  uint32_t u;
  memcpy(&u, &f, 4);
  if ((u & 0x7fffffffu) > 0x7f800000u) return (uint16_t)((u >> 16) | 0x40u);
  u += 0x7fffu + ((u >> 16) & 1u);
  return (uint16_t)(u >> 16);
}

float bf16_to_f32(uint16_t b) {
  const uint32_t u = (uint32_t)b << 16;
  float f;
  memcpy(&f, &u, 4);
  return f;
}

}  // namespace

struct fkv_cache {
  fkv_config cfg;
  Layout lay;
  Ctx ctx;
  std::vector<int> h_len;     // [L][batch] mirror of the device lengths
  std::vector<int> h_budget;  // [batch]
  std::vector<int> mirror;    // lengths and budgets as they lie in the workspace
  std::vector<uint8_t> loaded;  // [L][Hkv] scorer present
  std::vector<uint8_t> staging;
  uint64_t launches = 0;
  int sm_count = 148, device = 0;
  int max_cluster[2] = {0, 0};   // largest attention cluster the device places (found at the first stand-alone launch): plain, windowed
  float feature_scale = 0.f;  // softmax scale of the recorded queries (the last decode call's)
  bool timing = false, timed = false;
  CUtensorMap page_parts;     // ... as [page][64-channel part][row][64 channels]
  CUtensorMap page_rows;      // the page pool's K and V rows as [page][row][64-channel part][64 channels] (tensor copies)
  bool page_rows_ready = false;
  cudaEvent_t ev[7] = {nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr};  // [6]: after the plan
};

namespace fkv {
// For the library's other translation units: record the text of a failed CUDA call for fkv_last_cuda_error.
void note_cuda_error(cudaError_t e) { g_cuda_error = cudaGetErrorString(e); }
}  // namespace fkv

namespace {

int cuda_fail(cudaError_t e) {
  g_cuda_error = cudaGetErrorString(e);
  return FKV_ERR_CUDA;
}
#define FKV_CUDA(x)                           \
  do {                                        \
    cudaError_t e_ = (x);                     \
    if (e_ != cudaSuccess) return cuda_fail(e_); \
  } while (0)
#define FKV_LAUNCHED(c)                       \
  do {                                        \
    ++(c)->launches;                          \
    cudaError_t e_ = cudaGetLastError();      \
    if (e_ != cudaSuccess) return cuda_fail(e_); \
  } while (0)

// The caller's bit array (host, one word per 64 sequences; NULL = every sequence) as the kernels take it.
SeqMask make_mask(const fkv_cache *c, const uint64_t *bits) {
  SeqMask m = {};
  if (bits) {
    m.use = 1;
    for (int i = 0; i < (c->cfg.max_batch + 63) / 64; ++i) m.w[i] = bits[i];
  }
  return m;
}

bool layer_ok(const fkv_cache *c, int layer) { return layer >= 0 && layer < c->cfg.num_layers; }

// Page slots of the scorer's ring: as many as fit the shared memory, a multiple of the number of warps (a slot
// must always come back to the warp that refilled it: its barrier carries one phase bit, and only the warp that
// waited for the slot's previous page knows that phase is over), at most four per warp.
int score_ring_slots(const fkv_cache *c) {
  for (int n = 4 * kScorePPS; n >= kScorePPS; n -= kScorePPS)
    if (ScoreSmem::bytes(c->lay.page_bytes, c->lay.F, kScorePPS, n) <= kMaxSmem) return n;
  return 0;
}

template <int D>
int launch_score(fkv_cache *c, float *out, int seg_base, int tiles_bound, cudaStream_t st) {
  const int nslots = score_ring_slots(c);
  if (nslots == 0) return FKV_ERR_INVALID_ARG;
  const size_t smem = ScoreSmem::bytes(c->lay.page_bytes, c->lay.F, kScorePPS, nslots);
  static SmemOptIn opt_in;
  FKV_CUDA(opt_in.ensure(k_score<D, kScorePPS>, kMaxSmem));
  const int grid = std::max(1, std::min(c->sm_count, tiles_bound));
  k_score<D, kScorePPS><<<grid, kScorePPS * 32, smem, st>>>(c->ctx, out, seg_base, nslots);
  FKV_LAUNCHED(c);
  return FKV_OK;
}

int launch_score_any(fkv_cache *c, float *out, int seg_base, int tiles_bound, cudaStream_t st) {
  return c->cfg.head_dim == 128 ? launch_score<128>(c, out, seg_base, tiles_bound, st)
                                : launch_score<64>(c, out, seg_base, tiles_bound, st);
}

// One selection launch: mode 0 writes kept slot lists, mode 1 keep-priorities of the sampled action.
void launch_select(fkv_cache *c, int mode, int max_old, int nblocks, const float *scores, int32_t *idx,
                   int32_t *kept_count, int seg_base, int fill_pages, float *prio, const float *noise, int noise_stride,
                   int noise_base, cudaStream_t st) {
  // Variant by the longest segment: registers hold a whole segment up to 2048 (256-thread CTAs, many per SM), 8192
  // (two CTAs per SM) or 32768 keys, a pair of CTAs 65536; longer segments stream their rounds from L2.
#define FKV_SEL(S, M, T, P) \
  k_select<S, M, T, P><<<nblocks, T, 0, st>>>(c->ctx, scores, idx, kept_count, seg_base, fill_pages, prio, noise, \
                                             noise_stride, noise_base)
  if (max_old <= kSelTinyThreads * kSelTinyPerThread) {
    if (mode == 0) FKV_SEL(true, 0, kSelTinyThreads, kSelTinyPerThread); else FKV_SEL(true, 1, kSelTinyThreads, kSelTinyPerThread);
  } else if (max_old <= kSelSmallThreads * kSelSmallPerThread) {
    if (mode == 0) FKV_SEL(true, 0, kSelSmallThreads, kSelSmallPerThread); else FKV_SEL(true, 1, kSelSmallThreads, kSelSmallPerThread);
  } else if (max_old <= kSelRound) {
    if (mode == 0) FKV_SEL(true, 0, kSelThreads, 32); else FKV_SEL(true, 1, kSelThreads, 32);
  } else if (max_old <= 2 * kSelRound) {
    // Up to 65536 keys: a pair of CTAs (one cluster) per segment, each with half of the keys in registers.
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(2 * nblocks);
    cfg.blockDim = dim3(kSelThreads);
    cfg.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = 2; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    if (mode == 0)
      (void)cudaLaunchKernelEx(&cfg, k_select<true, 0, kSelThreads, 32, true>, c->ctx, scores, idx, kept_count, seg_base,
                               fill_pages, prio, noise, noise_stride, noise_base);
    else
      (void)cudaLaunchKernelEx(&cfg, k_select<true, 1, kSelThreads, 32, true>, c->ctx, scores, idx, kept_count, seg_base,
                               fill_pages, prio, noise, noise_stride, noise_base);
  } else {
    if (mode == 0) FKV_SEL(false, 0, kSelThreads, 32); else FKV_SEL(false, 1, kSelThreads, 32);
  }
#undef FKV_SEL
}

// Attention features of the segments on the work list (after a k_plan): one persistent CTA per SM, each a
// contiguous range of the plan's 128-pair tiles.
template <int D>
int launch_features_t(fkv_cache *c, int max_old, int nwork_bound, float scale_log2, cudaStream_t st) {
  static_assert(kFeatPages == kScorePPS, "the feature kernel walks the plan's score tiles");
  int na = 0, nq = 0;
  FeatSmem::rings(D, c->cfg.group_size, c->cfg.feature_window, na, nq);
  if (na < 1) return FKV_ERR_INVALID_ARG;
  const size_t smem = FeatSmem::bytes(D, c->cfg.group_size, c->cfg.feature_window, na, nq);
  if (max_old <= 0 || nwork_bound <= 0) return FKV_OK;
  if (FeatSmem::lq(c->cfg.feature_window) <= 128) {   // four accumulators: three reducing warpgroups
    static SmemOptIn opt_in;
    FKV_CUDA(opt_in.ensure(k_features<D, 3>, smem));
    k_features<D, 3><<<c->sm_count, feat_threads(3), smem, st>>>(c->ctx, scale_log2, na, nq);
  } else {                                            // two accumulators, two warpgroups on each
    static SmemOptIn opt_in;
    FKV_CUDA(opt_in.ensure(k_features<D, 4>, smem));
    k_features<D, 4><<<c->sm_count, feat_threads(4), smem, st>>>(c->ctx, scale_log2, na, nq);
  }
  FKV_LAUNCHED(c);
  return FKV_OK;
}
int launch_features(fkv_cache *c, int max_old, int nwork_bound, cudaStream_t st) {
  const float scale_log2 = c->feature_scale * 1.4426950408889634f;
  return c->cfg.head_dim == 128 ? launch_features_t<128>(c, max_old, nwork_bound, scale_log2, st)
                                : launch_features_t<64>(c, max_old, nwork_bound, scale_log2, st);
}

// The driver's tensor-map encoder, reached through the runtime, so the library links no driver stub.
typedef CUresult (*encode_fn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                              const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                              CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
int tensor_map(CUtensorMap *map, void *base, int rank, const cuuint64_t *dims, const cuuint64_t *strides, const cuuint32_t *box,
               CUtensorMapSwizzle swizzle) {
  static std::atomic<void *> known{nullptr};   // (a query's map is encoded at every call)
  void *fn = known.load();
  if (fn == nullptr) {
    cudaDriverEntryPointQueryResult found;
    FKV_CUDA(cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &found));
    if (fn == nullptr || found != cudaDriverEntryPointSuccess) {
      g_cuda_error = "cuTensorMapEncodeTiled is not available from this driver";
      return FKV_ERR_CUDA;
    }
    known.store(fn);
  }
  const cuuint32_t step[5] = {1, 1, 1, 1, 1};
  const CUresult r = reinterpret_cast<encode_fn>(fn)(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, rank, base, dims, strides, box, step,
                                                     CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
                                                     CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (r != CUDA_SUCCESS) {
    g_cuda_error = "cuTensorMapEncodeTiled failed with driver error " + std::to_string((int)r);
    return FKV_ERR_CUDA;
  }
  return FKV_OK;
}

// The tensor map of the page copies: bf16 [num_pages][16 rows][2 D / 64][64 channels] over the page pool (K's 64-channel
// parts, then V's), one box = the 16 rows x 64 channels of one page (2 KB, 16 rows of 128 bytes in shared memory; the
// record's own chunk swizzle stays as it is).
int ensure_page_rows_map(fkv_cache *c) {
  if (c->page_rows_ready) return FKV_OK;
  const int D = c->cfg.head_dim;
  const cuuint64_t dims[4] = {64, (cuuint64_t)(2 * D / 64), (cuuint64_t)kPage, (cuuint64_t)c->ctx.num_pages};
  const cuuint64_t strides[3] = {128, (cuuint64_t)(4 * D), (cuuint64_t)c->ctx.page_bytes};   // bytes, dimensions 1 .. 3
  const cuuint32_t box[4] = {64, 1, (cuuint32_t)kPage, 1};
  if (int e = tensor_map(&c->page_rows, c->ctx.pool, 4, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_NONE)) return e;
  // The same with the rows inside the parts: one box = 16 rows of D channels, 64 channels after another (all of K or V).
  const cuuint64_t dims2[4] = {64, (cuuint64_t)kPage, (cuuint64_t)(2 * D / 64), (cuuint64_t)c->ctx.num_pages};
  const cuuint64_t strides2[3] = {(cuuint64_t)(4 * D), 128, (cuuint64_t)c->ctx.page_bytes};
  const cuuint32_t box2[4] = {64, (cuuint32_t)kPage, (cuuint32_t)(D / 64), 1};
  if (int e = tensor_map(&c->page_parts, c->ctx.pool, 4, dims2, strides2, box2, CU_TENSOR_MAP_SWIZZLE_NONE)) return e;
  c->page_rows_ready = true;
  return FKV_OK;
}

// R-KV baseline scores of the segments on the work list (after a k_plan): the attention term and the reciprocal
// key norms first (the index scratch holds the norms until the selection overwrites it), then the n x n
// contraction.  Work items sit on grid.x (no 65535 limit).
template <int D>
int launch_rkv_t(fkv_cache *c, float *out, int seg_base, int max_old, int nwork_bound, long long tiles, float la, float ls,
                 cudaStream_t st) {
  if (max_old <= 0 || nwork_bound <= 0) return FKV_OK;
  if (int e = ensure_page_rows_map(c)) return e;
  float *rn = reinterpret_cast<float *>(c->ctx.idx);
  k_rkv_prepare<D><<<dim3(nwork_bound, (max_old + 127) / 128), 128, 0, st>>>(c->ctx, out, rn, seg_base,
                                                                             FKV_FEATURE_WINDOW8);
  FKV_LAUNCHED(c);
  if (tiles > 4) {
    // Pairs of CTAs that multiply as one (a unit is up to four tiles).
    const size_t smem = RkvPairSmem::bytes(D);
    static SmemOptIn opt_in;
    FKV_CUDA(opt_in.ensure(k_rkv_score_pair<D>, smem));
    const int npairs = (int)std::max<long long>(1, std::min<long long>(c->sm_count / 2, (tiles + 3) / 4));
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(2 * npairs);
    cfg.blockDim = dim3(kRkvThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = 2; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    FKV_CUDA(cudaLaunchKernelEx(&cfg, k_rkv_score_pair<D>, c->ctx, c->page_rows, out, (const float *)rn, seg_base, la, ls));
  } else {
    const size_t smem = RkvSmem::bytes(D);
    static SmemOptIn opt_in;
    FKV_CUDA(opt_in.ensure(k_rkv_score<D>, smem));
    const int grid = (int)std::max<long long>(1, std::min<long long>(c->sm_count, tiles));
    k_rkv_score<D><<<grid, kRkvThreads, smem, st>>>(c->ctx, c->page_rows, out, rn, seg_base, la, ls);
  }
  FKV_LAUNCHED(c);
  return FKV_OK;
}
int launch_rkv(fkv_cache *c, float *out, int seg_base, int max_old, int nwork_bound, long long tiles, float la, float ls,
               cudaStream_t st) {
  return c->cfg.head_dim == 128 ? launch_rkv_t<128>(c, out, seg_base, max_old, nwork_bound, tiles, la, ls, st)
                                : launch_rkv_t<64>(c, out, seg_base, max_old, nwork_bound, tiles, la, ls, st);
}

int launch_compact(fkv_cache *c, const int32_t *idx, int seg_base, int max_new, int nwork_bound, cudaStream_t st) {
  const int tiles = (max_new + kCompactRows - 1) / kCompactRows;
  const long long ctas = (long long)nwork_bound * tiles;   // one flat grid: no 65535 limit on the work list
  if (ctas == 0) return FKV_OK;
  if (ctas > 0x7fffffffLL) return FKV_ERR_INVALID_ARG;
  if (c->cfg.head_dim == 128) k_compact<128><<<(unsigned)ctas, 256, 0, st>>>(c->ctx, idx, seg_base, tiles);
  else k_compact<64><<<(unsigned)ctas, 256, 0, st>>>(c->ctx, idx, seg_base, tiles);
  FKV_LAUNCHED(c);
  return FKV_OK;
}

// One launch of the attention kernel: `splits` CTAs per segment.  pdl: the launch may run alongside the one
// before it on the stream.  cluster: the splits of a segment are one thread-block cluster (the merge goes through
// distributed shared memory).
template <int D, int NCW, int SLOTS, bool CLUSTER, bool WIN>
int launch_attend_t(fkv_cache *c, const AttendArgs *a, int splits, bool pdl, cudaStream_t st) {
  const size_t smem = AttendSmem::bytes(D, NCW, SLOTS, CLUSTER);
  auto kern = k_attend<D, NCW, SLOTS, CLUSTER, WIN>;
  static SmemOptIn opt_in;
  FKV_CUDA(opt_in.ensure(kern, smem));
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(splits, c->cfg.max_batch * c->cfg.num_kv_heads);
  cfg.blockDim = dim3((NCW + 1) * 32);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute at[2];
  int na = 0;
  if (pdl || a->wait_first) {
    at[na].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[na].val.programmaticStreamSerializationAllowed = 1;
    ++na;
  }
  if (CLUSTER) {
    at[na].id = cudaLaunchAttributeClusterDimension;
    at[na].val.clusterDim.x = splits; at[na].val.clusterDim.y = 1; at[na].val.clusterDim.z = 1;
    ++na;
  }
  cfg.attrs = at;
  cfg.numAttrs = na;
  FKV_CUDA(cudaLaunchKernelEx(&cfg, kern, c->ctx, *a));
  ++c->launches;
  return FKV_OK;
}

// The largest cluster of attention CTAs this device places: 16 (needs the non-portable opt-in), else 8; found once
// per handle.
template <int D, int NCW, int SLOTS, bool WIN>
int attend_max_cluster(fkv_cache *c) {
  auto kern = k_attend<D, NCW, SLOTS, true, WIN>;
  const size_t smem = AttendSmem::bytes(D, NCW, SLOTS, true);
  if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess ||
      cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess) {
    (void)cudaGetLastError();
    return 1;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(kClusterSplits, 1);
  cfg.blockDim = dim3((NCW + 1) * 32);
  cfg.dynamicSmemBytes = smem;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = kClusterSplits; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  int nclusters = 0;
  const bool ok16 = cudaOccupancyMaxActiveClusters(&nclusters, kern, &cfg) == cudaSuccess && nclusters > 0;
  (void)cudaGetLastError();
  return ok16 ? kClusterSplits : 8;
}

template <bool WIN>
int attend_dispatch(fkv_cache *c, const AttendArgs *a, int splits, bool pdl, bool cluster, cudaStream_t st) {
  if (cluster)
    return c->cfg.head_dim == 128 ? launch_attend_t<128, 4, 8, true, WIN>(c, a, splits, pdl, st)
                                  : launch_attend_t<64, 4, 16, true, WIN>(c, a, splits, pdl, st);
  return c->cfg.head_dim == 128 ? launch_attend_t<128, 4, 8, false, WIN>(c, a, splits, pdl, st)
                                : launch_attend_t<64, 4, 16, false, WIN>(c, a, splits, pdl, st);
}

// The windowed form of a decode launch: window == 0 is the plain one.
struct Window {
  int window = 0, sinks = 0;
  const int32_t *q_pos = nullptr;
};

// Attention over `layer`, with the new pair of every participating sequence appended first when k_new is given.
int launch_attend(fkv_cache *c, int layer, const void *q, void *out, float scale, const void *k_new, const void *v_new,
                  const int32_t *pos, const SeqMask &seq_mask, bool pdl, cudaStream_t st, const Window &w = Window()) {
  const int batch = c->cfg.max_batch, Hkv = c->cfg.num_kv_heads, D = c->cfg.head_dim;
  const bool app = k_new != nullptr;
  int maxpages = 0;
  for (int s = 0; s < batch; ++s) {
    const int n = c->h_len[(size_t)layer * batch + s] + ((app && seq_mask.has(s)) ? 1 : 0);
    int pages = (n + kPage - 1) / kPage;
    if (w.window)   // a window of W positions holds at most W pairs, which may begin and end inside a page
      pages = (int)std::min<long long>(pages, ((long long)w.window + kPage - 1) / kPage + 1 + (std::min(w.sinks, n) + kPage - 1) / kPage);
    maxpages = std::max(maxpages, pages);
  }
  // Splits per segment, at least kAttendMinPages pages each.  Consecutive launches of a decode step share the SMs
  // (three CTAs fit on one): CTAs for about three quarters of the SMs per launch.  A launch on its own has the GPU to
  // itself and lasts as long as its longest CTA: CTAs for every slot of every SM - but never more than
  // kSoloMaxSplits per segment, because the merge in a segment's last CTA grows with the splits (8 segments of 8192
  // pairs: 16.9 us per layer launch at 14 splits, 17.6 at 20, 20.4 at 32; 64 segments of 2K - 16K pairs: 96 us at 2
  // splits, which this rule turns into 7).
  constexpr int kSoloMaxSplits = 14;
  const int nseg = batch * Hkv;
  const int want_ctas = pdl ? c->sm_count * 3 / 4 : c->sm_count * 3;
  // (a launch on its own must fit one wave: rounded down, so that no CTA starts after the others have finished)
  int splits = std::min(c->lay.att_smax, std::max(1, pdl ? (want_ctas + nseg / 2) / nseg : want_ctas / nseg));
  if (!pdl) splits = std::min(splits, kSoloMaxSplits);
  splits = std::max(1, std::min(splits, maxpages / kAttendMinPages));
  // A launch on its own over few segments: the splits of a segment as one cluster of 16 (or 8) CTAs, merged through
  // distributed shared memory.  The cluster size is a power of two; with many segments the global-memory merge
  // above, whose split count is free, fills the GPU better.
  bool cluster = false;
  if (!pdl && nseg * kClusterSplits <= c->sm_count * 3 / 2) {
    int &max_cluster = c->max_cluster[w.window ? 1 : 0];
    if (max_cluster == 0) {
      if (w.window)
        max_cluster = c->cfg.head_dim == 128 ? attend_max_cluster<128, 4, 8, true>(c) : attend_max_cluster<64, 4, 16, true>(c);
      else
        max_cluster = c->cfg.head_dim == 128 ? attend_max_cluster<128, 4, 8, false>(c) : attend_max_cluster<64, 4, 16, false>(c);
    }
    int cs = 1;
    while (cs * 2 <= max_cluster && cs * 2 <= kClusterSplits && maxpages / (cs * 2) >= kAttendMinPages) cs *= 2;
    if (cs >= 8) { cluster = true; splits = cs; }
  }
  const int pps = std::max(1, (maxpages + splits - 1) / splits);
  if (scale == 0.f) scale = 1.f / sqrtf((float)D);
  if (app && !w.window) c->feature_scale = scale;
  AttendArgs a;
  a.layer = layer; a.q = (const __nv_bfloat16 *)q; a.out = (__nv_bfloat16 *)out;
  a.scale_log2 = scale * 1.4426950408889634f; a.pps = pps; a.append = app ? 1 : 0;
  a.k_new = (const uint8_t *)k_new; a.v_new = (const uint8_t *)v_new; a.pos_new = pos; a.seq_mask = seq_mask;
  a.window = w.window; a.sinks = w.sinks; a.q_pos = w.q_pos;
  a.wait_first = pdl ? 0 : 1;
  const int rc = w.window ? attend_dispatch<true>(c, &a, splits, pdl, cluster, st) : attend_dispatch<false>(c, &a, splits, pdl, cluster, st);
  if (rc) return rc;
  if (app)
    for (int s = 0; s < batch; ++s)
      if (seq_mask.has(s)) ++c->h_len[(size_t)layer * batch + s];
  return FKV_OK;
}

// ---------------------------------------------------------------- chunks
inline bool aligned(const void *p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }
constexpr int kMaxChunkTokens = 1 << 24;   // of one call, over all sequences

// Prefix sums of the chunk lengths; false if a length is negative or they are too many.
bool make_lens(const fkv_cache *c, const int32_t *chunk_lens, ChunkLens &l) {
  long long t = 0;
  l.tok[0] = 0;
  for (int s = 0; s < kMaxBatch; ++s) {
    if (s < c->cfg.max_batch) {
      if (chunk_lens[s] < 0) return false;
      t += chunk_lens[s];
      if (t > kMaxChunkTokens) return false;
    }
    l.tok[s + 1] = (int)t;
  }
  return true;
}

// A launch with the programmatic attribute whose kernel waits for the launch before it ahead of its first global read.
template <class... P, class... A>
cudaError_t launch_waiting(void (*kern)(P...), dim3 grid, int threads, size_t smem, cudaStream_t st, A &&...args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kern, std::forward<A>(args)...);
}

int check_append_chunk(const fkv_cache *c, int layer, const void *k, const void *v, const int32_t *pos,
                       const int32_t *keep_lens, const int32_t *chunk_lens, ChunkLens &lens) {
  if (!c || !layer_ok(c, layer) || !chunk_lens || !make_lens(c, chunk_lens, lens)) return FKV_ERR_INVALID_ARG;
  const int batch = c->cfg.max_batch;
  if (lens.tok[batch] > 0 && (!k || !v || !aligned(k, 16) || !aligned(v, 16) || !aligned(pos, 4))) return FKV_ERR_INVALID_ARG;
  for (int s = 0; s < batch; ++s) {
    const int n = c->h_len[(size_t)layer * batch + s], keep = keep_lens ? keep_lens[s] : n;
    if (keep < 0 || keep > n) return FKV_ERR_INVALID_ARG;
    if (keep + (long long)chunk_lens[s] > c->lay.cap) return FKV_ERR_CAPACITY;
  }
  return FKV_OK;
}

// masks: of a draft tree, else NULL.
int launch_append_chunk(fkv_cache *c, int layer, const void *k, const void *v, const int32_t *pos, const int32_t *keep_lens,
                        const int32_t *chunk_lens, const ChunkLens &lens, const uint32_t *masks, cudaStream_t st) {
  const int batch = c->cfg.max_batch;
  // (A roll-back to the lengths that the host knows is launched all the same: replayed, it meets others.)
  if (lens.tok[batch] == 0 && !keep_lens) return FKV_OK;
  ChunkKeep keep = {};
  if (keep_lens) {
    keep.use = 1;
    for (int s = 0; s < batch; ++s) keep.keep[s] = keep_lens[s];
  }
  // A warp per pair, up to four CTAs of eight warps on every SM: more pairs than that go round.
  const long long tasks = (long long)lens.tok[batch] * c->cfg.num_kv_heads;
  const int grid = (int)std::max<long long>(1, std::min<long long>((tasks + 7) / 8, 4LL * c->sm_count));
  FKV_CUDA(launch_waiting(masks ? k_append_chunk<true> : k_append_chunk<false>, dim3(grid), 256, 0, st, c->ctx, layer, (const uint8_t *)k,
                          (const uint8_t *)v, pos, lens, keep, masks));
  ++c->launches;
  for (int s = 0; s < batch; ++s) {
    int &n = c->h_len[(size_t)layer * batch + s];
    n = (keep_lens ? keep_lens[s] : n) + chunk_lens[s];
  }
  return FKV_OK;
}

int check_chunk(const fkv_cache *c, int layer, const void *q, const int32_t *chunk_lens, int32_t window, int32_t sinks,
                float scale, ChunkLens &lens) {
  if (!c || !layer_ok(c, layer) || !chunk_lens || !make_lens(c, chunk_lens, lens)) return FKV_ERR_INVALID_ARG;
  if (window < 0 || sinks < 0) return FKV_ERR_INVALID_ARG;
  if (scale != 0.f && !(scale >= 0x1p-100f && scale <= 0x1p100f)) return FKV_ERR_INVALID_ARG;   // (NaN too)
  if (lens.tok[c->cfg.max_batch] > 0 && (!q || !aligned(q, 16))) return FKV_ERR_INVALID_ARG;
  return FKV_OK;
}
// The chunk's own pairs have to be the last ones of their segments (after the append, if the call makes one).
bool chunk_is_stored(const fkv_cache *c, int layer, const int32_t *chunk_lens) {
  for (int s = 0; s < c->cfg.max_batch; ++s)
    if (chunk_lens[s] > c->h_len[(size_t)layer * c->cfg.max_batch + s]) return false;
  return true;
}

// q as [tokens][query heads][D]: one box = 64 channels x `heads` heads x `tokens` tokens, rows of 128 swizzled bytes.
int query_map(const fkv_cache *c, const void *q, int tokens, int box_heads, int box_tokens, CUtensorMap *map) {
  const int D = c->cfg.head_dim, Hq = c->cfg.num_kv_heads * c->cfg.group_size;
  const cuuint64_t dims[3] = {(cuuint64_t)D, (cuuint64_t)Hq, (cuuint64_t)tokens};
  const cuuint64_t strides[2] = {(cuuint64_t)(2 * D), (cuuint64_t)(2 * D * Hq)};
  const cuuint32_t box[3] = {64, (cuuint32_t)box_heads, (cuuint32_t)box_tokens};
  return tensor_map(map, const_cast<void *>(q), 3, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B);
}

template <int D, bool TREE>
int launch_chunk_attend_t(fkv_cache *c, const CUtensorMap &tmq, const ChunkArgs &a, int grid, cudaStream_t st) {
  constexpr size_t smem = ChunkSmem<D>::bytes();
  static_assert(smem <= kMaxSmem, "one CTA's shared memory");
  static SmemOptIn opt_in;
  FKV_CUDA(opt_in.ensure(k_chunk_attend<D, TREE>, smem));
  FKV_CUDA(launch_waiting(k_chunk_attend<D, TREE>, dim3(grid), kChunkThreads, smem, st, c->ctx, c->page_rows, c->page_parts, tmq, a));
  ++c->launches;
  if (grid > 1) {   // (a single CTA cuts nothing)
    // A warp per query row of the largest item, or per 8 rows x 16 channels.
    int longest = 0;
    for (int s = 0; s < c->cfg.max_batch; ++s) longest = std::max(longest, a.lens.tok[s + 1] - a.lens.tok[s]);
    const int G = c->cfg.group_size, tile = kChunkRows / G, rows = std::min(longest, 2 * tile) * G;
    FKV_CUDA(launch_waiting(longest <= tile ? k_chunk_merge<D, true> : k_chunk_merge<D, false>, dim3(grid, (rows + 7) / 8), 256, 0, st, c->ctx, a));
    ++c->launches;
  }
  return FKV_OK;
}

int launch_chunk_attend(fkv_cache *c, int layer, const void *q, const int32_t *chunk_lens, const ChunkLens &lens, int window,
                        int sinks, float scale, void *out, float *lse, const uint32_t *masks, cudaStream_t st) {
  const int batch = c->cfg.max_batch, D = c->cfg.head_dim, G = c->cfg.group_size;
  if (lens.tok[batch] == 0) return FKV_OK;
  if (int e = ensure_page_rows_map(c)) return e;
  ChunkArgs a;
  a.layer = layer; a.window = window; a.sinks = window ? sinks : 0;
  a.scale = scale == 0.f ? 1.f / sqrtf((float)D) : scale;
  a.scale_log2 = a.scale * 1.4426950408889634f;
  a.out = (__nv_bfloat16 *)out; a.lse = lse; a.masks = masks; a.lens = lens;
  CUtensorMap tmq;
  const int tokens_per_tile = kChunkRows / G, block = 2 * tokens_per_tile;
  if (int e = query_map(c, q, lens.tok[batch], G, tokens_per_tile, &tmq)) return e;
  // As many CTAs as there is work for: the pages of all items, by the lengths the host knows (the kernel goes by its own).
  long long pages = 0;
  for (int s = 0; s < batch; ++s) {
    const int T = chunk_lens[s], n = c->h_len[(size_t)layer * batch + s];
    for (int j = 0; j < T && pages < (1LL << 20); j += block) pages += (n - T + std::min(T, j + block) + kPage - 1) / kPage;
  }
  pages *= c->cfg.num_kv_heads;
  const int most = std::min(kChunkCtas, c->sm_count);
  const int grid = (int)std::max<long long>(1, std::min<long long>(most, (pages + kChunkMinPages - 1) / kChunkMinPages));
  if (masks) return D == 128 ? launch_chunk_attend_t<128, true>(c, tmq, a, grid, st) : launch_chunk_attend_t<64, true>(c, tmq, a, grid, st);
  return D == 128 ? launch_chunk_attend_t<128, false>(c, tmq, a, grid, st) : launch_chunk_attend_t<64, false>(c, tmq, a, grid, st);
}

template <int D>
int launch_chunk_features_t(fkv_cache *c, const CUtensorMap &tmq, ChunkFeatArgs &a, int grid, cudaStream_t st) {
  constexpr size_t smem = CfSmem<D>::bytes();
  static_assert(smem <= kMaxSmem, "one CTA's shared memory");
  static SmemOptIn opt_in;
  FKV_CUDA(opt_in.ensure(k_chunk_features<D>, smem));
  int longest = 0;
  for (int s = 0; s < c->cfg.max_batch; ++s) longest = std::max(longest, a.lens.tok[s + 1] - a.lens.tok[s]);
  a.nq = CfSmem<D>::rings(longest, a.nk);
  FKV_CUDA(launch_waiting(k_chunk_features<D>, dim3(grid), kCfThreads, smem, st, c->ctx, c->page_rows, tmq, a));
  ++c->launches;
  return FKV_OK;
}

int launch_chunk_features(fkv_cache *c, int layer, const void *q, const float *lse, const int32_t *chunk_lens, const ChunkLens &lens,
                          int window, int sinks, float scale, bool record_used, cudaStream_t st) {
  const int batch = c->cfg.max_batch, D = c->cfg.head_dim;
  if (lens.tok[batch] == 0) return FKV_OK;
  if (int e = ensure_page_rows_map(c)) return e;
  ChunkFeatArgs a;
  a.record_used = record_used ? 1 : 0;
  a.layer = layer; a.window = window; a.sinks = window ? sinks : 0;
  if (scale == 0.f) scale = 1.f / sqrtf((float)D);
  a.scale_log2 = scale * 1.4426950408889634f;
  a.inv_hi = (float)(1.0 / (double)scale);
  a.inv_lo = (float)(1.0 / (double)scale - (double)a.inv_hi);
  a.lse = lse; a.lens = lens;
  CUtensorMap tmq;
  if (int e = query_map(c, q, lens.tok[batch], 1, kCfQueries, &tmq)) return e;
  long long units = 0;   // (pair of tiles, query head)
  for (int s = 0; s < batch; ++s)
    if (chunk_lens[s] > 0) units += (c->h_len[(size_t)layer * batch + s] + kCfPairs - 1) / kCfPairs;
  units *= c->cfg.num_kv_heads * c->cfg.group_size;
  const int grid = (int)std::max<long long>(1, std::min<long long>(c->sm_count, units));
  return D == 128 ? launch_chunk_features_t<128>(c, tmq, a, grid, st) : launch_chunk_features_t<64>(c, tmq, a, grid, st);
}

// ---------------------------------------------------------------- draft trees
// Lengths of trees: at most kTreeNodes each, and a window (if any) holds every ancestor.
bool trees_ok(const fkv_cache *c, const int32_t *tree_lens, int window) {
  for (int s = 0; s < c->cfg.max_batch; ++s)
    if (tree_lens[s] > kTreeNodes || (window > 0 && tree_lens[s] > window)) return false;
  return true;
}

// Trees whose attention (and store) is one launch of clusters (k_tree_attend).
template <int D, bool WIN, bool HALF>
int tree_attend_config(cudaLaunchConfig_t &cfg, cudaLaunchAttribute (&at)[2], int S, int y, cudaStream_t st) {
  constexpr size_t smem = TaSmem<D>::bytes();
  static_assert(smem <= kMaxSmem, "one CTA's shared memory");
  static SmemOptIn opt_in;
  FKV_CUDA(opt_in.ensure(k_tree_attend<D, WIN, HALF>, smem));
  cfg = cudaLaunchConfig_t{};
  cfg.gridDim = dim3(S, y);
  cfg.blockDim = dim3(kTaThreads<HALF>);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = S; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
  at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = 2;
  return FKV_OK;
}
// How many clusters of S CTAs the device holds at a time (-1: none).
template <int D, bool WIN, bool HALF>
int tree_clusters(int S) {
  cudaLaunchConfig_t cfg;
  cudaLaunchAttribute at[2];
  int n = 0;
  const bool ok = tree_attend_config<D, WIN, HALF>(cfg, at, S, 1, nullptr) == FKV_OK &&
                  cudaFuncSetAttribute(k_tree_attend<D, WIN, HALF>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) == cudaSuccess &&
                  (cfg.numAttrs = 1, cudaOccupancyMaxActiveClusters(&n, k_tree_attend<D, WIN, HALF>, &cfg) == cudaSuccess) && n > 0;
  (void)cudaGetLastError();
  return ok ? n : -1;
}
template <int D, bool WIN, bool HALF>
int launch_tree_attend_t(fkv_cache *c, const CUtensorMap (&in)[3], const TreeArgs &a, int S, int store, cudaStream_t st) {
  cudaLaunchConfig_t cfg;
  cudaLaunchAttribute at[2];
  if (int e = tree_attend_config<D, WIN, HALF>(cfg, at, S, a.rows_y + store, st)) return e;
  FKV_CUDA(cudaLaunchKernelEx(&cfg, k_tree_attend<D, WIN, HALF>, c->ctx, c->page_rows, c->page_parts, in[0], in[1], in[2], a));
  ++c->launches;
  return FKV_OK;
}
// The forms of the kernel by head dimension, window and rows.
#define FKV_TREE_FORM(f, ...)                                                                                                  \
  (c->cfg.head_dim == 128 ? win ? half ? f<128, true, true>(__VA_ARGS__) : f<128, true, false>(__VA_ARGS__)                    \
                                : half ? f<128, false, true>(__VA_ARGS__) : f<128, false, false>(__VA_ARGS__)                  \
                          : win ? half ? f<64, true, true>(__VA_ARGS__) : f<64, true, false>(__VA_ARGS__)                      \
                                : half ? f<64, false, true>(__VA_ARGS__) : f<64, false, false>(__VA_ARGS__))

// How k_tree_attend serves a call: CTAs per block of query rows (0: the general kernel is to serve it), clusters that store, rows twice.
struct TreeShape {
  int S = 0, store = 0;
  bool half = false;
  int block = 0;   // nodes of a block of query rows
};
// ahead: pairs ahead of every tree.
TreeShape tree_shape(fkv_cache *c, const int32_t *tree_lens, const int *ahead, int window, int sinks, bool append) {
  const int batch = c->cfg.max_batch, Hkv = c->cfg.num_kv_heads, G = c->cfg.group_size;
  TreeShape r;
  int longest = 0;
  for (int s = 0; s < batch; ++s) longest = std::max(longest, tree_lens[s]);
  r.half = longest * G <= kChunkRows / 2;
  r.block = (r.half ? kChunkRows / 2 : kChunkRows) / G;
  long long total = 0, segs = 0, tokens = 0;
  int most = 0;
  for (int s = 0; s < batch; ++s) {
    if (tree_lens[s] == 0) continue;
    const int blocks = (tree_lens[s] + r.block - 1) / r.block, all = (ahead[s] + tree_lens[s] + kPage - 1) / kPage + 1;
    // (a window of W positions holds at most W pairs)
    const int pages = window ? (int)std::min<long long>(all, ((long long)window + std::min(sinks, ahead[s]) + tree_lens[s]) / kPage + 3) : all;
    most = std::max(most, pages);
    segs += (long long)blocks * Hkv;
    total += (long long)blocks * Hkv * pages;
    tokens += tree_lens[s];
  }
  if (segs == 0 || segs > std::min(c->sm_count, kTaMaxBlocks)) return r;
  // The largest cluster of which the device holds all at once, one that stores among them, with a few pages at least for every CTA.
  // (asked of the runtime once per device and form: 0 is not asked yet, -1 none)
  static std::atomic<int> clusters[64][2][2][2][kTaMaxCluster + 1] = {};
  const bool win = window > 0, half = r.half;
  int S = (int)std::min<long long>(std::min<long long>(kTaMaxCluster, c->sm_count / segs), std::max(1, most / kAttendMinPages));
  int fit = 0;
  for (; S > 0; --S) {
    std::atomic<int> &known = clusters[c->device & 63][c->cfg.head_dim == 128][win][half][S];
    fit = known.load();
    if (fit == 0) known.store(fit = FKV_TREE_FORM(tree_clusters, S));
    if (fit >= segs + (append ? 1 : 0)) break;
  }
  if (S == 0) return r;
  // The general kernels share the pages evenly over the SMs, but start and join 10 - 30 us later; a page takes a cluster's CTA 0.15 - 0.18 us,
  // and an SM 0.21 where all of them read.  Both timed, D = 128, pages of the longest CTA here : most that the rule lets through: 16 nodes,
  // 8 heads 205 : 210 41.0 us by clusters, 54.4 by the general kernels; 410 : 321 72.4 and 73.5; 820 : 542 138 and 120.  64 nodes 342 : 321
  // 72.8 and 69.2.  Four uneven sequences 342 : 176 60.3 and 48.1; eight 258 : 201 59.1 and 55.6.  The border is off by most where one head
  // is all there is (129 : 113, 27.6 and 53.3; 513 : 155, 84.5 and 60.4) and for 256 nodes over 16384 pairs (521 : 550, 105.7 and 98.9).
  if ((most + S - 1) / S > total / c->sm_count + 100) return r;
  r.S = S;
  const long long warps = (long long)S * ((half ? kTaThreads<true> : kTaThreads<false>) / 32);   // a pair and head each
  if (append) r.store = (int)std::max<long long>(1, std::min<long long>((tokens * Hkv + warps - 1) / warps, fit - segs));
  return r;
}

// k, v: of a tree that is not stored yet, else NULL.
int launch_tree_attend(fkv_cache *c, int layer, const void *k, const void *v, const int32_t *keep_lens, const int32_t *tree_lens,
                       const ChunkLens &lens, const uint32_t *masks, const int32_t *pos, const void *q, int window, int sinks, float scale, void *out,
                       float *lse, const TreeShape &shape, cudaStream_t st) {
  const int batch = c->cfg.max_batch, D = c->cfg.head_dim, Hkv = c->cfg.num_kv_heads;
  if (int e = ensure_page_rows_map(c)) return e;
  TreeArgs a;
  a.layer = layer; a.append = k != nullptr; a.window = window; a.sinks = window ? sinks : 0;
  a.k = (const uint8_t *)k; a.v = (const uint8_t *)v; a.pos = pos;
  a.scale_log2 = (scale == 0.f ? 1.f / sqrtf((float)D) : scale) * 1.4426950408889634f;
  a.out = (__nv_bfloat16 *)out; a.lse = lse; a.masks = masks; a.lens = lens;
  int blocks = 0;
  for (int s = 0; s < batch; ++s)
    for (int b = 0; b * shape.block < tree_lens[s]; ++b, ++blocks) {
      a.seq[blocks] = (uint8_t)s;
      a.block[blocks] = (uint8_t)b;
    }
  a.rows_y = blocks * Hkv;
  a.keep = ChunkKeep{};
  if (keep_lens) {
    a.keep.use = 1;
    for (int s = 0; s < batch; ++s) a.keep.keep[s] = keep_lens[s];
  }
  CUtensorMap in[3];
  if (int e = query_map(c, q, lens.tok[batch], c->cfg.group_size, shape.block, &in[0])) return e;
  in[1] = in[2] = in[0];
  if (k) {   // [tokens][Hkv][D] as (64 channels, tokens, parts of 64 channels, heads): a box = 16 tokens of a head, one part (K) or all (V)
    const cuuint64_t dims[4] = {64, (cuuint64_t)lens.tok[batch], (cuuint64_t)(D / 64), (cuuint64_t)Hkv};
    const cuuint64_t strides[3] = {(cuuint64_t)(2 * D * Hkv), 128, (cuuint64_t)(2 * D)};
    const cuuint32_t box_k[4] = {64, kPage, 1, 1}, box_v[4] = {64, kPage, (cuuint32_t)(D / 64), 1};
    if (int e = tensor_map(&in[1], const_cast<void *>(k), 4, dims, strides, box_k, CU_TENSOR_MAP_SWIZZLE_128B)) return e;
    if (int e = tensor_map(&in[2], const_cast<void *>(v), 4, dims, strides, box_v, CU_TENSOR_MAP_SWIZZLE_128B)) return e;
  }
  const bool win = window > 0, half = shape.half;
  if (int e = FKV_TREE_FORM(launch_tree_attend_t, c, in, a, shape.S, shape.store, st)) return e;
  if (k)
    for (int s = 0; s < batch; ++s) {
      int &n = c->h_len[(size_t)layer * batch + s];
      n = (keep_lens ? keep_lens[s] : n) + tree_lens[s];
    }
  return FKV_OK;
}

// A cluster of CTAs per sequence: eight, or as many as the SMs hold at a time for all that have a tree: a pass is a chain of reads, so a
// large batch too goes by how many pieces are in flight (64 rows of 130001 in 16 bits: 18.1 us with clusters of two).
template <class T, bool Q>
int launch_verify_t(fkv_cache *c, const VerifyArgs &a, cudaStream_t st) {
  int cs = 1, trees = 0;
  for (int s = 0; s < c->cfg.max_batch; ++s) trees += a.lens.tok[s + 1] > a.lens.tok[s];
  while (cs < kVerParts && cs * 2 * trees <= kVerCtasPerSm * c->sm_count) cs *= 2;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(c->cfg.max_batch * cs);
  cfg.blockDim = dim3(kVerThreads);
  cfg.stream = st;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = cs; at[1].val.clusterDim.y = 1; at[1].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = 2;
  FKV_CUDA(cudaLaunchKernelEx(&cfg, k_verify_tree<T, Q>, c->ctx, a));
  ++c->launches;
  return FKV_OK;
}

int check_verify(const fkv_cache *c, const int32_t *tokens, const int32_t *parents, const int32_t *tree_lens, const int32_t *path,
                 const int32_t *path_len, const int32_t *tokens_out, int32_t stride, VerifyArgs &a) {
  if (!c || !tree_lens || !make_lens(c, tree_lens, a.lens) || !trees_ok(c, tree_lens, 0)) return FKV_ERR_INVALID_ARG;
  const int total = a.lens.tok[c->cfg.max_batch];
  if (!path || !path_len || !tokens_out || stride < 1 || !aligned(path, 4) || !aligned(path_len, 4) || !aligned(tokens_out, 4))
    return FKV_ERR_INVALID_ARG;
  if (total > 0 && (!tokens || !parents || !aligned(tokens, 4) || !aligned(parents, 4))) return FKV_ERR_INVALID_ARG;
  for (int s = 0; s < c->cfg.max_batch; ++s)
    if (tree_lens[s] > stride) return FKV_ERR_INVALID_ARG;
  return FKV_OK;
}

// ---------------------------------------------------------------- forks
// What every sequence does, from where each comes; false if nothing changes.
bool make_fork(const fkv_cache *c, const int32_t *from, ForkMap &m, ForkOps &ops) {
  const int batch = c->cfg.max_batch;
  bool any = false;
  for (int s = 0; s < kMaxBatch; ++s) {
    m.from[s] = (short)s;
    m.first[s] = m.next[s] = -1;
    m.what[s] = 0;
    ops.emptied[s] = 0;
  }
  bool moved[kMaxBatch] = {};   // whose pages have been handed over
  for (int s = 0; s < batch; ++s) {
    const int r = from[s];
    m.from[s] = (short)r;
    if (r == s) continue;
    any = true;
    m.what[s] = FORK_CHANGES;
    if (r < 0) {
      ops.emptied[s] = 1;
    } else if (from[r] != r && !moved[r]) {
      moved[r] = true;
      m.what[s] |= FORK_MOVES;
    }
  }
  for (int s = batch - 1; s >= 0; --s) {
    if (!(m.what[s] & FORK_CHANGES)) continue;
    if (!moved[s]) m.what[s] |= FORK_FREED;
    if (m.from[s] >= 0 && !(m.what[s] & FORK_MOVES)) {
      m.next[s] = m.first[m.from[s]];
      m.first[m.from[s]] = (short)s;
    }
  }
  // The record's copies in an order in which no value is overwritten before it is used.
  ops.n = 0;
  int src[kMaxBatch], uses[kForkAside + 1] = {}, ready[kMaxBatch], nready = 0;
  std::fill(src, src + kMaxBatch, -1);
  for (int s = 0; s < batch; ++s)
    if ((m.what[s] & FORK_CHANGES) && m.from[s] >= 0) {
      src[s] = m.from[s];
      ++uses[src[s]];
    }
  auto emit = [&](int d, int s) {
    ops.dst[ops.n] = (short)d;
    ops.src[ops.n] = (short)s;
    ++ops.n;
  };
  auto run_ready = [&]() {
    while (nready > 0) {
      const int d = ready[--nready], s = src[d];
      emit(d, s);
      src[d] = -1;
      if (--uses[s] == 0 && s < batch && src[s] >= 0) ready[nready++] = s;
    }
  };
  for (int s = 0; s < batch; ++s)
    if (src[s] >= 0 && uses[s] == 0) ready[nready++] = s;
  run_ready();
  for (int s = 0; s < batch; ++s) {   // what is left are cycles: one element aside, and the rest follows
    if (src[s] < 0) continue;
    emit(kForkAside, s);
    for (int d = 0; d < batch; ++d)
      if (src[d] == s) src[d] = kForkAside;
    uses[kForkAside] = uses[s];
    uses[s] = 0;
    ready[nready++] = s;
    run_ready();
  }
  return any;
}

}  // namespace

extern "C" {

int fkv_workspace_bytes(const fkv_config *cfg, size_t *bytes) {
  if (!valid_config(cfg) || !bytes) return FKV_ERR_INVALID_ARG;
  *bytes = make_layout(*cfg).total;
  return FKV_OK;
}

int fkv_init_cache(const fkv_config *cfg, void *dev_workspace, size_t bytes, void *stream, fkv_cache **out) {
  if (!valid_config(cfg) || !dev_workspace || !out) return FKV_ERR_INVALID_ARG;
  if (((uintptr_t)dev_workspace & 255u) != 0) return FKV_ERR_INVALID_ARG;
  const Layout L = make_layout(*cfg);
  if (bytes < L.total) return FKV_ERR_WORKSPACE_TOO_SMALL;
  fkv_cache *c = new (std::nothrow) fkv_cache();
  if (!c) return FKV_ERR_INVALID_ARG;
  c->cfg = *cfg;
  c->lay = L;
  uint8_t *ws = (uint8_t *)dev_workspace;
  Ctx &x = c->ctx;
  x.L = cfg->num_layers; x.Hkv = cfg->num_kv_heads; x.G = cfg->group_size; x.D = cfg->head_dim;
  x.batch = cfg->max_batch; x.act = cfg->activation; x.R = cfg->recent_keep; x.F = L.F;
  x.cap = L.cap; x.max_pages = L.max_pages; x.num_pages = L.num_pages;
  x.page_bytes = L.page_bytes; x.off_v = 2 * cfg->head_dim; x.off_f = 64 * cfg->head_dim;
  x.sp_stride = L.sp_stride; x.sp_off_wf = L.sp_off_wf; x.sp_off_b1 = L.sp_off_b1; x.sp_off_w2 = L.sp_off_w2;
  x.sp_off_b2 = L.sp_off_b2;
  x.pool = ws + L.pool; x.free_stack = (int *)(ws + L.free_stack); x.ctrl = (int *)(ws + L.ctrl);
  x.planhdr = (int *)(ws + L.planhdr); x.pt = (int *)(ws + L.pt); x.pt_new = (int *)(ws + L.pt_new);
  x.len = (int *)(ws + L.len); x.budget = (int *)(ws + L.budget); x.sp = ws + L.sp;
  x.scores = (float *)(ws + L.scores); x.idx = (int *)(ws + L.idx); x.plan = (SegPlan *)(ws + L.plan);
  x.work = (int *)(ws + L.work); x.tile1_start = (int *)(ws + L.tile1);
  x.seq_tickets = (int *)(ws + L.seq_tickets);
  x.seq_fail = (int *)(ws + L.seq_fail);
  x.att_part = (float *)(ws + L.att_part); x.att_tickets = (int *)(ws + L.att_tickets); x.att_smax = L.att_smax;
  x.hist_w = cfg->feature_window; x.hist_q = ws + L.hist_q; x.hist_mp = (float *)(ws + L.hist_mp); x.hist_wp = (cfg->feature_window + 15) & ~15;
  x.hist_n = (int *)(ws + L.hist_n); x.hist_cnt = (int *)(ws + L.hist_cnt);
  x.chunk_part = (float *)(ws + L.chunk_part); x.chunk_ml = (float *)(ws + L.chunk_ml); x.chunk_info = (int *)(ws + L.chunk_info);
  c->h_len.assign((size_t)cfg->num_layers * cfg->max_batch, 0);
  c->h_budget.assign(cfg->max_batch, cfg->budget);
  c->mirror.resize((L.budget - L.len) / 4 + cfg->max_batch);
  c->loaded.assign((size_t)cfg->num_layers * cfg->num_kv_heads, 0);
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  c->device = dev;
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&c->sm_count, cudaDevAttrMultiProcessorCount, dev);
  cudaStream_t st = (cudaStream_t)stream;
  // Zero everything: freshly taken pages then hold finite values in the slots not yet written.
  if (e == cudaSuccess) e = cudaMemsetAsync(ws, 0, L.total, st);
  if (e == cudaSuccess)
    e = cudaMemcpyAsync(x.budget, c->h_budget.data(), (size_t)cfg->max_batch * 4, cudaMemcpyHostToDevice, st);
  if (e == cudaSuccess) e = cudaStreamSynchronize(st);
  if (e != cudaSuccess) {
    delete c;
    return cuda_fail(e);
  }
  k_reset<<<256, 256, 0, st>>>(c->ctx);
  ++c->launches;
  e = cudaGetLastError();
  if (e != cudaSuccess) {
    delete c;
    return cuda_fail(e);
  }
  *out = c;
  return FKV_OK;
}

int fkv_destroy(fkv_cache *c) {
  if (c)
    for (cudaEvent_t e : c->ev)
      if (e) cudaEventDestroy(e);
  delete c;
  return FKV_OK;
}

int fkv_reset(fkv_cache *c, void *stream) {
  if (!c) return FKV_ERR_INVALID_ARG;
  k_reset<<<256, 256, 0, (cudaStream_t)stream>>>(c->ctx);
  FKV_LAUNCHED(c);
  std::fill(c->h_len.begin(), c->h_len.end(), 0);
  return FKV_OK;
}

int fkv_load_scorer(fkv_cache *c, int layer, int kv_head, const float *W1, const float *b1, const float *W2, float b2,
                    void *stream) {
  if (!c || !layer_ok(c, layer) || kv_head < 0 || kv_head >= c->cfg.num_kv_heads || !W1 || !b1 || !W2)
    return FKV_ERR_INVALID_ARG;
  const int D = c->cfg.head_dim, F = c->lay.F, H = kHidden, KS = 2 * D / 16;
  c->staging.assign(c->lay.sp_stride, 0);
  uint32_t *wkv = (uint32_t *)c->staging.data();
  auto w1 = [&](int row, int col) { return W1[(size_t)row * H + col]; };
  // Part 0 of a weight is its bf16 rounding, part 1 the bf16 rounding of what that left over.
  auto part = [&](int row, int col, int which) {
    const float w = w1(row, col);
    const uint16_t hi = f32_to_bf16_rne(w);
    if (which == 0) return hi;
    if (!std::isfinite(bf16_to_f32(hi))) return (uint16_t)0;   // inf and NaN carry no remainder
    return f32_to_bf16_rne(w - bf16_to_f32(hi));
  };
  auto pack = [&](int row, int col, int which) {
    return (uint32_t)part(row, col, which) | ((uint32_t)part(row + 1, col, which) << 16);
  };
  // mma B fragments (16 x 8, "col"): lane (gid, tig) holds rows k0 + 2 tig (+1) and k0 + 8 + 2 tig (+1) of
  // column gid; registers 0-1 for hidden units 0-7, 2-3 for hidden units 8-15.  All fragments of the
  // roundings first, then all fragments of the remainders.
  for (int which = 0; which < 2; ++which)
    for (int ks = 0; ks < KS; ++ks)
      for (int lane = 0; lane < 32; ++lane) {
        const int gid = lane >> 2, tig = lane & 3, k0 = ks * 16;
        uint32_t *r = wkv + ((size_t)(which * KS + ks) * 32 + lane) * 4;
        r[0] = pack(k0 + 2 * tig, gid, which);
        r[1] = pack(k0 + 8 + 2 * tig, gid, which);
        r[2] = pack(k0 + 2 * tig, 8 + gid, which);
        r[3] = pack(k0 + 8 + 2 * tig, 8 + gid, which);
      }
  // Per quad lane t the hidden units {2t, 2t+1, 8+2t, 9+2t}: the mma accumulator columns that lane owns.
  auto quad = [&](float *dst, auto get) {
    for (int t = 0; t < 4; ++t) {
      dst[t * 4 + 0] = get(2 * t); dst[t * 4 + 1] = get(2 * t + 1);
      dst[t * 4 + 2] = get(8 + 2 * t); dst[t * 4 + 3] = get(9 + 2 * t);
    }
  };
  // Feature rows of W1 as tf32 mma B fragments (8 x 8, "col"): lane (gid, tig) holds rows k0 + tig and k0 + 4 + tig
  // of column gid.  A weight is its truncation to tf32 (10 mantissa bits) plus the truncated remainder; per k-step
  // and lane eight words: truncations for hidden units 0-7 and 8-15, then the remainders.  Rows past F are zero.
  uint32_t *wf = (uint32_t *)(c->staging.data() + c->lay.sp_off_wf);
  auto tf32_part = [&](int row, int col, int which) -> uint32_t {
    if (row >= F) return 0u;
    const float w = w1(2 * D + row, col);
    uint32_t u;
    memcpy(&u, &w, 4);
    const uint32_t t = u & 0xffffe000u;
    if (which == 0) return t;
    float tf;
    memcpy(&tf, &t, 4);
    if (!std::isfinite(tf)) return 0u;
    const float r = w - tf;
    memcpy(&u, &r, 4);
    return u & 0xffffe000u;
  };
  for (int ks = 0; ks < ScoreSmem::fk(F); ++ks)
    for (int lane = 0; lane < 32; ++lane) {
      const int gid = lane >> 2, tig = lane & 3, k0 = ks * 8;
      uint32_t *r = wf + ((size_t)ks * 32 + lane) * 8;
      for (int which = 0; which < 2; ++which) {
        r[which * 4 + 0] = tf32_part(k0 + tig, gid, which);
        r[which * 4 + 1] = tf32_part(k0 + 4 + tig, gid, which);
        r[which * 4 + 2] = tf32_part(k0 + tig, 8 + gid, which);
        r[which * 4 + 3] = tf32_part(k0 + 4 + tig, 8 + gid, which);
      }
    }
  quad((float *)(c->staging.data() + c->lay.sp_off_b1), [&](int j) { return b1[j]; });
  quad((float *)(c->staging.data() + c->lay.sp_off_w2), [&](int j) { return W2[j]; });
  *(float *)(c->staging.data() + c->lay.sp_off_b2) = b2;
  cudaStream_t st = (cudaStream_t)stream;
  FKV_CUDA(cudaMemcpyAsync(c->ctx.sp + ((size_t)layer * c->cfg.num_kv_heads + kv_head) * c->lay.sp_stride,
                           c->staging.data(), c->lay.sp_stride, cudaMemcpyHostToDevice, st));
  FKV_CUDA(cudaStreamSynchronize(st));
  c->loaded[(size_t)layer * c->cfg.num_kv_heads + kv_head] = 1;
  return FKV_OK;
}

int fkv_set_budget(fkv_cache *c, int seq, int32_t budget, void *stream) {
  if (!c || seq < 0 || seq >= c->cfg.max_batch || budget < 1) return FKV_ERR_INVALID_ARG;
  c->h_budget[seq] = budget;
  cudaStream_t st = (cudaStream_t)stream;
  FKV_CUDA(cudaMemcpyAsync(c->ctx.budget + seq, &c->h_budget[seq], 4, cudaMemcpyHostToDevice, st));
  FKV_CUDA(cudaStreamSynchronize(st));
  return FKV_OK;
}

int fkv_prefill(fkv_cache *c, int layer, int seq, const void *k, const void *v, const float *feat, const int32_t *pos,
                int32_t n, void *stream) {
  if (!c || !layer_ok(c, layer) || seq < 0 || seq >= c->cfg.max_batch || !k || !v || n < 1) return FKV_ERR_INVALID_ARG;
  if (n > c->lay.cap) return FKV_ERR_CAPACITY;
  int &hl = c->h_len[(size_t)layer * c->cfg.max_batch + seq];
  if (hl != 0) return FKV_ERR_INVALID_ARG;
  cudaStream_t st = (cudaStream_t)stream;
  k_prefill_alloc<<<1, 1024, 0, st>>>(c->ctx, layer, seq, n);
  FKV_LAUNCHED(c);
  dim3 grid((n + 7) / 8, c->cfg.num_kv_heads);
  k_prefill_rows<0><<<grid, 256, 0, st>>>(c->ctx, layer, seq, n, (const uint8_t *)k, (const uint8_t *)v, feat, pos);
  FKV_LAUNCHED(c);
  hl = n;
  return FKV_OK;
}

int fkv_set_features(fkv_cache *c, int layer, int seq, const float *feat, void *stream) {
  if (!c || !layer_ok(c, layer) || seq < 0 || seq >= c->cfg.max_batch || !feat) return FKV_ERR_INVALID_ARG;
  const int n = c->h_len[(size_t)layer * c->cfg.max_batch + seq];
  if (n == 0) return FKV_OK;
  dim3 grid((n + 7) / 8, c->cfg.num_kv_heads);
  k_prefill_rows<1><<<grid, 256, 0, (cudaStream_t)stream>>>(c->ctx, layer, seq, n, nullptr, nullptr, feat, nullptr);
  FKV_LAUNCHED(c);
  return FKV_OK;
}

int fkv_append(fkv_cache *c, int layer, const void *k, const void *v, const int32_t *pos, const uint64_t *seq_mask,
               void *stream) {
  if (!c || !layer_ok(c, layer) || !k || !v) return FKV_ERR_INVALID_ARG;
  const int batch = c->cfg.max_batch;
  const SeqMask m = make_mask(c, seq_mask);
  for (int s = 0; s < batch; ++s)
    if (m.has(s) && c->h_len[(size_t)layer * batch + s] >= c->lay.cap) return FKV_ERR_CAPACITY;
  k_append<<<batch, 32 * c->cfg.num_kv_heads, 0, (cudaStream_t)stream>>>(c->ctx, layer, (const uint8_t *)k,
                                                                        (const uint8_t *)v, pos, m);
  FKV_LAUNCHED(c);
  for (int s = 0; s < batch; ++s)
    if (m.has(s)) ++c->h_len[(size_t)layer * batch + s];
  return FKV_OK;
}

// Candidates the sampled action needs noise for in one segment: min(2E, competing pairs).
static int sampled_candidates(int n, int B, int R) {
  if (n <= B) return 0;
  return std::min(2 * (n - B), n - std::min(R, B));
}

// score_kind: -1 the learned scorer, 0..5 a feature column (baseline), kScoreRkv the R-KV baseline with its two weights.
constexpr int kScoreRkv = 100;
static int evict_impl(fkv_cache *c, int layer, const float *noise, int noise_stride, int feature_column, float rkv_a,
                      float rkv_s, void *stream) {
  if (!c || (layer != FKV_ALL_LAYERS && !layer_ok(c, layer))) return FKV_ERR_INVALID_ARG;
  const int l0 = layer == FKV_ALL_LAYERS ? 0 : layer, l1 = layer == FKV_ALL_LAYERS ? c->cfg.num_layers : layer + 1;
  const int batch = c->cfg.max_batch, Hkv = c->cfg.num_kv_heads;
  int nactive = 0, max_new = 0, max_old = 0;
  long long tiles = 0;
  for (int l = l0; l < l1; ++l)
    for (int s = 0; s < batch; ++s) {
      const int n = c->h_len[(size_t)l * batch + s], B = c->h_budget[s];
      if (n > B) {
        for (int h = 0; h < Hkv && feature_column < 0; ++h)
          if (!c->loaded[(size_t)l * Hkv + h]) return FKV_ERR_NOT_READY;
        if (noise && sampled_candidates(n, B, c->cfg.recent_keep) > noise_stride) return FKV_ERR_INVALID_ARG;
        nactive += Hkv;
        max_new = std::max(max_new, B);
        max_old = std::max(max_old, n);
        tiles += (long long)Hkv * ((n + kScorePPS * kPage - 1) / (kScorePPS * kPage));
      }
    }
  if (nactive == 0) return FKV_OK;
  cudaStream_t st = (cudaStream_t)stream;
  const bool tm = c->timing;
  if (tm) FKV_CUDA(cudaEventRecord(c->ev[0], st));
  k_plan<<<1, 1024, 0, st>>>(c->ctx, l0, l1, PLAN_EVICT, kScorePPS * kPage, nullptr, SeqMask{});
  FKV_LAUNCHED(c);
  if (tm) FKV_CUDA(cudaEventRecord(c->ev[6], st));
  if (c->cfg.feature_window > 0 && c->feature_scale > 0.f) {   // refresh a_n from the chunk's recorded queries first
    const int rcf = launch_features(c, max_old, nactive, st);
    if (rcf) return rcf;
  }
  if (tm) FKV_CUDA(cudaEventRecord(c->ev[1], st));
  int rc = FKV_OK;
  if (feature_column < 0) {
    rc = launch_score_any(c, c->ctx.scores, 0, (int)std::min<long long>(tiles, 1 << 30), st);
  } else if (feature_column == kScoreRkv) {
    rc = launch_rkv(c, c->ctx.scores, 0, max_old, nactive, tiles, rkv_a, rkv_s, st);
  } else {   // a baseline: the score is a feature column
    k_score_feature<<<dim3(nactive, (max_old + 127) / 128), 128, 0, st>>>(c->ctx, c->ctx.scores, 0, feature_column);
    FKV_LAUNCHED(c);
  }
  if (rc) return rc;
  if (tm) FKV_CUDA(cudaEventRecord(c->ev[2], st));
  if (noise) {   // sampled action: scores -> keep-priorities (in place), then the same selection over them
    launch_select(c, 1, max_old, nactive, c->ctx.scores, nullptr, nullptr, 0, 0, c->ctx.scores, noise, noise_stride,
                  l0 * batch * Hkv, st);
    FKV_LAUNCHED(c);
  }
  launch_select(c, 0, max_old, nactive, c->ctx.scores, c->ctx.idx, nullptr, 0, 1, nullptr, nullptr, 0, 0, st);
  FKV_LAUNCHED(c);
  if (tm) FKV_CUDA(cudaEventRecord(c->ev[3], st));
  rc = launch_compact(c, c->ctx.idx, 0, max_new, nactive, st);
  if (rc) return rc;
  if (tm) FKV_CUDA(cudaEventRecord(c->ev[4], st));
  k_commit<<<(l1 - l0) * batch * Hkv, 256, 0, st>>>(c->ctx, l0, l1);
  FKV_LAUNCHED(c);
  if (tm) {
    FKV_CUDA(cudaEventRecord(c->ev[5], st));
    c->timed = true;
  }
  for (int l = l0; l < l1; ++l)
    for (int s = 0; s < batch; ++s) {
      int &n = c->h_len[(size_t)l * batch + s];
      n = std::min(n, c->h_budget[s]);
    }
  return FKV_OK;
}

int fkv_evict(fkv_cache *c, int layer, void *stream) { return evict_impl(c, layer, nullptr, 0, -1, 0.f, 0.f, stream); }

int fkv_evict_by_feature(fkv_cache *c, int layer, int32_t column, void *stream) {
  if (column < 0 || column > 5) return FKV_ERR_INVALID_ARG;
  return evict_impl(c, layer, nullptr, 0, column, 0.f, 0.f, stream);
}

int fkv_evict_rkv(fkv_cache *c, int layer, float lambda_attn, float lambda_sim, void *stream) {
  if (!std::isfinite(lambda_attn) || !std::isfinite(lambda_sim)) return FKV_ERR_INVALID_ARG;
  return evict_impl(c, layer, nullptr, 0, kScoreRkv, lambda_attn, lambda_sim, stream);
}

int fkv_score_rkv(fkv_cache *c, int layer, float lambda_attn, float lambda_sim, float *scores_out, void *stream) {
  if (!c || !layer_ok(c, layer) || !scores_out || !std::isfinite(lambda_attn) || !std::isfinite(lambda_sim))
    return FKV_ERR_INVALID_ARG;
  const int batch = c->cfg.max_batch, Hkv = c->cfg.num_kv_heads;
  long long tiles = 0;
  int max_old = 0;
  for (int s = 0; s < batch; ++s) {
    const int n = c->h_len[(size_t)layer * batch + s];
    tiles += (long long)Hkv * ((n + kScorePPS * kPage - 1) / (kScorePPS * kPage));
    max_old = std::max(max_old, n);
  }
  if (tiles == 0) return FKV_OK;
  cudaStream_t st = (cudaStream_t)stream;
  k_plan<<<1, 1024, 0, st>>>(c->ctx, layer, layer + 1, PLAN_SCORE_ALL, kScorePPS * kPage, nullptr, SeqMask{});
  FKV_LAUNCHED(c);
  return launch_rkv(c, scores_out, layer * batch * Hkv, max_old, batch * Hkv, tiles, lambda_attn, lambda_sim, st);
}

int fkv_evict_sampled(fkv_cache *c, int layer, const float *noise, int32_t noise_stride, void *stream) {
  if (!noise || noise_stride < 1) return FKV_ERR_INVALID_ARG;
  return evict_impl(c, layer, noise, noise_stride, -1, 0.f, 0.f, stream);
}

int fkv_decode_attn(fkv_cache *c, int layer, const void *q, void *out, float scale, void *stream) {
  if (!c || !layer_ok(c, layer) || !q || !out) return FKV_ERR_INVALID_ARG;
  return launch_attend(c, layer, q, out, scale, nullptr, nullptr, nullptr, make_mask(c, nullptr), false, (cudaStream_t)stream);
}

int fkv_append_decode_attn(fkv_cache *c, int layer, const void *k, const void *v, const int32_t *pos,
                           const uint64_t *seq_mask, const void *q, void *out, float scale, void *stream) {
  if (!c || !layer_ok(c, layer) || !k || !v || !q || !out) return FKV_ERR_INVALID_ARG;
  const int batch = c->cfg.max_batch;
  const SeqMask m = make_mask(c, seq_mask);
  for (int s = 0; s < batch; ++s)
    if (m.has(s) && c->h_len[(size_t)layer * batch + s] >= c->lay.cap) return FKV_ERR_CAPACITY;
  return launch_attend(c, layer, q, out, scale, k, v, pos, m, false, (cudaStream_t)stream);
}

int fkv_decode_step(fkv_cache *c, const void *k, const void *v, const int32_t *pos, const void *q, void *out,
                    float scale, void *stream) {
  if (!c || !k || !v || !q || !out) return FKV_ERR_INVALID_ARG;
  const int batch = c->cfg.max_batch;
  for (int l = 0; l < c->cfg.num_layers; ++l)
    for (int s = 0; s < batch; ++s)
      if (c->h_len[(size_t)l * batch + s] >= c->lay.cap) return FKV_ERR_CAPACITY;
  const size_t kv_stride = (size_t)batch * c->cfg.num_kv_heads * c->cfg.head_dim * 2;
  const size_t q_stride = kv_stride * c->cfg.group_size;
  const SeqMask all = make_mask(c, nullptr);
  for (int l = 0; l < c->cfg.num_layers; ++l) {
    // Layer l's launch may run alongside layer l - 1's: each touches only its own layer's cache state and
    // tensors.  Layer 0's launch is ordered after everything before it on the stream, as usual.
    const int rc = launch_attend(c, l, (const uint8_t *)q + l * q_stride, (uint8_t *)out + l * q_stride, scale,
                                 (const uint8_t *)k + l * kv_stride, (const uint8_t *)v + l * kv_stride, pos, all, l > 0,
                                 (cudaStream_t)stream);
    if (rc) return rc;
  }
  return FKV_OK;
}

int fkv_append_chunk(fkv_cache *c, int layer, const void *k, const void *v, const int32_t *pos, const int32_t *keep_lens,
                     const int32_t *chunk_lens, void *stream) {
  ChunkLens lens;
  if (int e = check_append_chunk(c, layer, k, v, pos, keep_lens, chunk_lens, lens)) return e;
  return launch_append_chunk(c, layer, k, v, pos, keep_lens, chunk_lens, lens, nullptr, (cudaStream_t)stream);
}

int fkv_chunk_attn(fkv_cache *c, int layer, const void *q, const int32_t *chunk_lens, int32_t window, int32_t sinks, float scale,
                   void *out, float *lse_out, void *stream) {
  ChunkLens lens;
  if (int e = check_chunk(c, layer, q, chunk_lens, window, sinks, scale, lens)) return e;
  if (lens.tok[c->cfg.max_batch] > 0 && (!out || !aligned(out, 16) || !aligned(lse_out, 4))) return FKV_ERR_INVALID_ARG;
  if (!chunk_is_stored(c, layer, chunk_lens)) return FKV_ERR_INVALID_ARG;
  return launch_chunk_attend(c, layer, q, chunk_lens, lens, window, sinks, scale, out, lse_out, nullptr, (cudaStream_t)stream);
}

int fkv_append_chunk_attn(fkv_cache *c, int layer, const void *k, const void *v, const int32_t *pos, const int32_t *keep_lens,
                          const int32_t *chunk_lens, const void *q, int32_t window, int32_t sinks, float scale, void *out,
                          float *lse_out, void *stream) {
  ChunkLens lens;
  if (int e = check_chunk(c, layer, q, chunk_lens, window, sinks, scale, lens)) return e;
  if (int e = check_append_chunk(c, layer, k, v, pos, keep_lens, chunk_lens, lens)) return e;
  if (lens.tok[c->cfg.max_batch] > 0 && (!out || !aligned(out, 16) || !aligned(lse_out, 4))) return FKV_ERR_INVALID_ARG;
  if (int e = ensure_page_rows_map(c)) return e;   // (what can fail does so before anything is stored)
  if (int e = launch_append_chunk(c, layer, k, v, pos, keep_lens, chunk_lens, lens, nullptr, (cudaStream_t)stream)) return e;
  return launch_chunk_attend(c, layer, q, chunk_lens, lens, window, sinks, scale, out, lse_out, nullptr, (cudaStream_t)stream);
}

int fkv_chunk_features(fkv_cache *c, int layer, const void *q, const float *lse, const int32_t *chunk_lens, int32_t window,
                       int32_t sinks, float scale, void *stream) {
  ChunkLens lens;
  if (int e = check_chunk(c, layer, q, chunk_lens, window, sinks, scale, lens)) return e;
  if (lens.tok[c->cfg.max_batch] > 0 && (!lse || !aligned(lse, 4))) return FKV_ERR_INVALID_ARG;
  if (!chunk_is_stored(c, layer, chunk_lens)) return FKV_ERR_INVALID_ARG;
  cudaStream_t st = (cudaStream_t)stream;
  const bool record = lens.tok[c->cfg.max_batch] > 0 && c->cfg.feature_window > 0 && c->feature_scale > 0.f;
  if (record) {
    // Decode queries on record came before the chunk: they move the features on first, and the chunk's kernel then takes
    // them off the record.
    if (int e = ensure_page_rows_map(c)) return e;   // (what can fail does so before anything is changed)
    SeqMask seqs = {};
    seqs.use = 1;
    int max_old = 0;
    for (int s = 0; s < c->cfg.max_batch; ++s)
      if (chunk_lens[s] > 0) {
        seqs.w[s / 64] |= 1ull << (s % 64);
        max_old = std::max(max_old, c->h_len[(size_t)layer * c->cfg.max_batch + s]);
      }
    k_plan<<<1, 1024, 0, st>>>(c->ctx, layer, layer + 1, PLAN_RECORD, kScorePPS * kPage, nullptr, seqs);
    FKV_LAUNCHED(c);
    if (int e = launch_features(c, max_old, c->cfg.max_batch * c->cfg.num_kv_heads, st)) return e;
  }
  return launch_chunk_features(c, layer, q, lse, chunk_lens, lens, window, sinks, scale, record, st);
}

int fkv_tree_masks(fkv_cache *c, const int32_t *parents, const int32_t *tree_lens, uint32_t *masks, void *stream) {
  ChunkLens lens;
  if (!c || !tree_lens || !make_lens(c, tree_lens, lens) || !trees_ok(c, tree_lens, 0)) return FKV_ERR_INVALID_ARG;
  if (lens.tok[c->cfg.max_batch] == 0) return FKV_OK;
  if (!parents || !masks || !aligned(parents, 4) || !aligned(masks, 16)) return FKV_ERR_INVALID_ARG;
  FKV_CUDA(launch_waiting(k_tree_masks, dim3(c->cfg.max_batch), kTreeNodes, 0, (cudaStream_t)stream, c->ctx, lens, parents, masks));
  ++c->launches;
  return FKV_OK;
}

static int check_tree(const fkv_cache *c, const int32_t *tree_lens, const ChunkLens &lens, const uint32_t *masks, int window) {
  if (!trees_ok(c, tree_lens, window)) return FKV_ERR_INVALID_ARG;
  return lens.tok[c->cfg.max_batch] > 0 && (!masks || !aligned(masks, 4)) ? FKV_ERR_INVALID_ARG : FKV_OK;
}

int fkv_append_tree(fkv_cache *c, int layer, const void *k, const void *v, const int32_t *pos, const int32_t *keep_lens,
                    const int32_t *tree_lens, const uint32_t *masks, void *stream) {
  ChunkLens lens;
  if (int e = check_append_chunk(c, layer, k, v, pos, keep_lens, tree_lens, lens)) return e;
  if (int e = check_tree(c, tree_lens, lens, masks, 0)) return e;
  return launch_append_chunk(c, layer, k, v, pos, keep_lens, tree_lens, lens, masks, (cudaStream_t)stream);
}

int fkv_tree_attn(fkv_cache *c, int layer, const void *q, const int32_t *tree_lens, const uint32_t *masks, int32_t window, int32_t sinks,
                  float scale, void *out, float *lse_out, void *stream) {
  ChunkLens lens;
  if (int e = check_chunk(c, layer, q, tree_lens, window, sinks, scale, lens)) return e;
  if (int e = check_tree(c, tree_lens, lens, masks, window)) return e;
  if (lens.tok[c->cfg.max_batch] > 0 && (!out || !aligned(out, 16) || !aligned(lse_out, 4))) return FKV_ERR_INVALID_ARG;
  if (!chunk_is_stored(c, layer, tree_lens)) return FKV_ERR_INVALID_ARG;
  int ahead[kMaxBatch];
  for (int s = 0; s < c->cfg.max_batch; ++s) ahead[s] = c->h_len[(size_t)layer * c->cfg.max_batch + s] - tree_lens[s];
  const TreeShape shape = tree_shape(c, tree_lens, ahead, window, sinks, false);
  if (shape.S)
    return launch_tree_attend(c, layer, nullptr, nullptr, nullptr, tree_lens, lens, masks, nullptr, q, window, sinks, scale, out, lse_out, shape,
                              (cudaStream_t)stream);
  return launch_chunk_attend(c, layer, q, tree_lens, lens, window, sinks, scale, out, lse_out, masks, (cudaStream_t)stream);
}

int fkv_append_tree_attn(fkv_cache *c, int layer, const void *k, const void *v, const int32_t *pos, const int32_t *keep_lens,
                         const int32_t *tree_lens, const uint32_t *masks, const void *q, int32_t window, int32_t sinks, float scale,
                         void *out, float *lse_out, void *stream) {
  ChunkLens lens;
  if (int e = check_chunk(c, layer, q, tree_lens, window, sinks, scale, lens)) return e;
  if (int e = check_append_chunk(c, layer, k, v, pos, keep_lens, tree_lens, lens)) return e;
  if (int e = check_tree(c, tree_lens, lens, masks, window)) return e;
  if (lens.tok[c->cfg.max_batch] > 0 && (!out || !aligned(out, 16) || !aligned(lse_out, 4))) return FKV_ERR_INVALID_ARG;
  int ahead[kMaxBatch];
  for (int s = 0; s < c->cfg.max_batch; ++s) ahead[s] = keep_lens ? keep_lens[s] : c->h_len[(size_t)layer * c->cfg.max_batch + s];
  const TreeShape shape = tree_shape(c, tree_lens, ahead, window, sinks, true);
  if (shape.S)
    return launch_tree_attend(c, layer, k, v, keep_lens, tree_lens, lens, masks, pos, q, window, sinks, scale, out, lse_out, shape,
                              (cudaStream_t)stream);
  if (int e = ensure_page_rows_map(c)) return e;   // (what can fail does so before anything is stored)
  if (int e = launch_append_chunk(c, layer, k, v, pos, keep_lens, tree_lens, lens, masks, (cudaStream_t)stream)) return e;
  return launch_chunk_attend(c, layer, q, tree_lens, lens, window, sinks, scale, out, lse_out, masks, (cudaStream_t)stream);
}

int fkv_verify_tree(fkv_cache *c, const int32_t *tokens, const int32_t *parents, const int32_t *tree_lens, const void *target,
                    int64_t target_stride, const void *draft, int64_t draft_stride, int32_t dtype, int32_t vocab, const float *u_accept,
                    const float *u_sample, int32_t *path, int32_t *path_len, int32_t *tokens_out, int32_t path_stride, void *stream) {
  VerifyArgs a;
  if (int e = check_verify(c, tokens, parents, tree_lens, path, path_len, tokens_out, path_stride, a)) return e;
  if (dtype != FKV_F32 && dtype != FKV_BF16) return FKV_ERR_INVALID_ARG;
  const int size = dtype == FKV_F32 ? 4 : 2;
  if (vocab < 1 || vocab > kVerMaxVocab || target_stride < vocab || (draft && draft_stride < vocab)) return FKV_ERR_INVALID_ARG;
  if (!aligned(target, size) || !aligned(draft, size) || !aligned(u_accept, 4) || !aligned(u_sample, 4)) return FKV_ERR_INVALID_ARG;
  if (a.lens.tok[c->cfg.max_batch] > 0 && (!target || !u_accept || !u_sample)) return FKV_ERR_INVALID_ARG;
  a.target = target; a.draft = draft; a.target_stride = target_stride; a.draft_stride = draft_stride;
  a.tokens = tokens; a.parents = parents; a.u_accept = u_accept; a.u_sample = u_sample;
  a.path = path; a.path_len = path_len; a.out = tokens_out; a.vocab = vocab; a.stride = path_stride;
  cudaStream_t st = (cudaStream_t)stream;
  if (dtype == FKV_F32) return draft ? launch_verify_t<float, true>(c, a, st) : launch_verify_t<float, false>(c, a, st);
  return draft ? launch_verify_t<__nv_bfloat16, true>(c, a, st) : launch_verify_t<__nv_bfloat16, false>(c, a, st);
}

int fkv_verify_tree_greedy(fkv_cache *c, const int32_t *tokens, const int32_t *parents, const int32_t *tree_lens, const int32_t *choice,
                           int32_t *path, int32_t *path_len, int32_t *tokens_out, int32_t path_stride, void *stream) {
  VerifyArgs a = {};
  if (int e = check_verify(c, tokens, parents, tree_lens, path, path_len, tokens_out, path_stride, a)) return e;
  if (a.lens.tok[c->cfg.max_batch] > 0 && (!choice || !aligned(choice, 4))) return FKV_ERR_INVALID_ARG;
  a.tokens = tokens; a.parents = parents; a.path = path; a.path_len = path_len; a.out = tokens_out; a.stride = path_stride;
  FKV_CUDA(launch_waiting(k_verify_greedy, dim3(c->cfg.max_batch), 32, 0, (cudaStream_t)stream, c->ctx, a, choice));
  ++c->launches;
  return FKV_OK;
}

int fkv_commit_tree(fkv_cache *c, int layer, const int32_t *tree_lens, const int32_t *path, const int32_t *path_len, int32_t path_stride,
                    void *stream) {
  ChunkLens lens;
  if (!c || (layer != FKV_ALL_LAYERS && !layer_ok(c, layer)) || !tree_lens || !make_lens(c, tree_lens, lens) || !trees_ok(c, tree_lens, 0))
    return FKV_ERR_INVALID_ARG;
  if (lens.tok[c->cfg.max_batch] == 0) return FKV_OK;
  if (!path || !path_len || path_stride < 1 || !aligned(path, 4) || !aligned(path_len, 4)) return FKV_ERR_INVALID_ARG;
  const int l0 = layer == FKV_ALL_LAYERS ? 0 : layer, nl = layer == FKV_ALL_LAYERS ? c->cfg.num_layers : 1;
  for (int l = l0; l < l0 + nl; ++l)
    if (!chunk_is_stored(c, l, tree_lens)) return FKV_ERR_INVALID_ARG;
  FKV_CUDA(launch_waiting(k_commit_tree, dim3(nl, c->cfg.max_batch), 1024, 0, (cudaStream_t)stream, c->ctx, l0, lens, path, path_len, path_stride));
  ++c->launches;
  return FKV_OK;
}

int fkv_export_chunk(fkv_cache *c, int layer, const int32_t *chunk_lens, void *k, void *v, float *feat, int32_t *pos, void *stream) {
  ChunkLens lens;
  if (!c || !layer_ok(c, layer) || !chunk_lens || !make_lens(c, chunk_lens, lens)) return FKV_ERR_INVALID_ARG;
  if (!chunk_is_stored(c, layer, chunk_lens)) return FKV_ERR_INVALID_ARG;
  if (!aligned(k, 16) || !aligned(v, 16) || !aligned(feat, 8) || !aligned(pos, 4)) return FKV_ERR_INVALID_ARG;
  if (lens.tok[c->cfg.max_batch] == 0 || (!k && !v && !feat && !pos)) return FKV_OK;
  ExportBlocks b;
  b.blk[0] = 0;
  for (int s = 0; s < kMaxBatch; ++s) {
    const int t = lens.tok[s + 1] - lens.tok[s];
    b.blk[s + 1] = b.blk[s] + (t > 0 ? (t + kPage - 1) / kPage + 1 : 0);
  }
  const long long tasks = (long long)b.blk[kMaxBatch] * c->cfg.num_kv_heads;
  const int most = (int)std::min<size_t>(kExportMaxWarps, (kMaxSmem - 2048) / (2 * (size_t)c->ctx.page_bytes));
  const int warps = (int)std::min<long long>(most, (tasks + c->sm_count - 1) / c->sm_count);
  const int grid = (int)std::min<long long>((tasks + warps - 1) / warps, c->sm_count);
  static SmemOptIn opt_in;
  FKV_CUDA(opt_in.ensure(k_export_chunk, kMaxSmem - 2048));
  FKV_CUDA(launch_waiting(k_export_chunk, dim3(grid), warps * 32, (size_t)warps * 2 * c->ctx.page_bytes, (cudaStream_t)stream, c->ctx, layer,
                          lens, b, (uint8_t *)k, (uint8_t *)v, feat, pos));
  ++c->launches;
  return FKV_OK;
}

int fkv_fork(fkv_cache *c, const int32_t *from, void *stream) {
  if (!c || !from) return FKV_ERR_INVALID_ARG;
  const int batch = c->cfg.max_batch, L = c->cfg.num_layers;
  for (int s = 0; s < batch; ++s)
    if (from[s] < -1 || from[s] >= batch) return FKV_ERR_INVALID_ARG;
  ForkMap m;
  ForkOps ops;
  if (!make_fork(c, from, m, ops)) return FKV_OK;
  cudaStream_t st = (cudaStream_t)stream;
  const bool own = L * batch <= kForkOwn;
  if (!own) {
    FKV_CUDA(launch_waiting(k_fork_plan, dim3(1), 1024, 0, st, c->ctx, m));
    ++c->launches;
  }
  constexpr size_t room = kMaxSmem - 1024 - 3 * kForkOwn * 4;
  const int warps = (int)std::min<size_t>(kForkMaxWarps, room / (2 * (size_t)c->ctx.page_bytes));
  const size_t smem = (size_t)warps * 2 * c->ctx.page_bytes;
  static SmemOptIn opt_in[2];
  FKV_CUDA(own ? opt_in[1].ensure(k_fork_copy<true>, room) : opt_in[0].ensure(k_fork_copy<false>, room));
  FKV_CUDA(launch_waiting(own ? k_fork_copy<true> : k_fork_copy<false>, dim3(c->sm_count), warps * 32, smem, st, c->ctx, m));
  ++c->launches;
  FKV_CUDA(launch_waiting(k_fork_commit, dim3(L * batch, c->cfg.num_kv_heads), 256, 0, st, c->ctx, m));
  ++c->launches;
  if (c->cfg.feature_window > 0) {
    const size_t words = (size_t)c->ctx.hist_wp * c->cfg.num_kv_heads * c->cfg.group_size * c->cfg.head_dim / 8;
    FKV_CUDA(launch_waiting(k_fork_record, dim3(L, (unsigned)((words + 255) / 256)), 256, 0, st, c->ctx, ops));
    ++c->launches;
  }
  int old[kMaxBatch];
  for (int l = 0; l < L; ++l) {
    int *h = &c->h_len[(size_t)l * batch];
    std::copy(h, h + batch, old);
    for (int s = 0; s < batch; ++s) h[s] = from[s] < 0 ? 0 : old[from[s]];
  }
  std::copy(c->h_budget.begin(), c->h_budget.end(), old);
  for (int s = 0; s < batch; ++s)
    if (from[s] >= 0) c->h_budget[s] = old[from[s]];
  return FKV_OK;
}

int fkv_decode_attn_window(fkv_cache *c, int layer, const void *q, const int32_t *q_pos, int32_t window, int32_t sinks, void *out,
                           float scale, void *stream) {
  if (!c || !layer_ok(c, layer) || !q || !out || window < 1 || sinks < 0) return FKV_ERR_INVALID_ARG;
  if (!aligned(q, 16) || !aligned(out, 16) || !aligned(q_pos, 4)) return FKV_ERR_INVALID_ARG;
  Window w;
  w.window = window; w.sinks = sinks; w.q_pos = q_pos;
  return launch_attend(c, layer, q, out, scale, nullptr, nullptr, nullptr, make_mask(c, nullptr), false, (cudaStream_t)stream, w);
}

int fkv_append_decode_attn_window(fkv_cache *c, int layer, const void *k, const void *v, const int32_t *pos,
                                  const uint64_t *seq_mask, const void *q, int32_t window, int32_t sinks, void *out, float scale,
                                  void *stream) {
  if (!c || !layer_ok(c, layer) || !k || !v || !q || !out || window < 1 || sinks < 0) return FKV_ERR_INVALID_ARG;
  if (!aligned(k, 16) || !aligned(v, 16) || !aligned(q, 16) || !aligned(out, 16) || !aligned(pos, 4)) return FKV_ERR_INVALID_ARG;
  const int batch = c->cfg.max_batch;
  const SeqMask m = make_mask(c, seq_mask);
  for (int s = 0; s < batch; ++s)
    if (m.has(s) && c->h_len[(size_t)layer * batch + s] >= c->lay.cap) return FKV_ERR_CAPACITY;
  Window w;
  w.window = window; w.sinks = sinks;
  return launch_attend(c, layer, q, out, scale, k, v, pos, m, false, (cudaStream_t)stream, w);
}

int fkv_export_features(fkv_cache *c, int layer, int seq, float *feat, void *stream) {
  if (!c || !layer_ok(c, layer) || seq < 0 || seq >= c->cfg.max_batch) return FKV_ERR_INVALID_ARG;
  const int n = c->h_len[(size_t)layer * c->cfg.max_batch + seq];
  if (n == 0) return FKV_OK;   // (an empty tensor may have no address)
  if (!feat || !aligned(feat, 4)) return FKV_ERR_INVALID_ARG;
  k_export_features<<<dim3((n + 7) / 8, c->cfg.num_kv_heads), 256, 0, (cudaStream_t)stream>>>(c->ctx, layer, seq, n, feat);
  FKV_LAUNCHED(c);
  return FKV_OK;
}

int fkv_update_features(fkv_cache *c, int layer, void *stream) {
  if (!c || !layer_ok(c, layer)) return FKV_ERR_INVALID_ARG;
  if (c->cfg.feature_window == 0) return FKV_ERR_NOT_READY;
  if (c->feature_scale == 0.f) return FKV_OK;   // no query has been recorded yet
  const int batch = c->cfg.max_batch, Hkv = c->cfg.num_kv_heads;
  int max_old = 0;
  for (int s = 0; s < batch; ++s) max_old = std::max(max_old, c->h_len[(size_t)layer * batch + s]);
  if (max_old == 0) return FKV_OK;
  cudaStream_t st = (cudaStream_t)stream;
  k_plan<<<1, 1024, 0, st>>>(c->ctx, layer, layer + 1, PLAN_SCORE_ALL, kScorePPS * kPage, nullptr, SeqMask{});
  FKV_LAUNCHED(c);
  return launch_features(c, max_old, batch * Hkv, st);
}

int fkv_score_stride(const fkv_cache *c, int32_t *cap) {
  if (!c || !cap) return FKV_ERR_INVALID_ARG;
  *cap = c->lay.cap;
  return FKV_OK;
}

int fkv_score(fkv_cache *c, int layer, float *scores_out, void *stream) {
  if (!c || !layer_ok(c, layer) || !scores_out) return FKV_ERR_INVALID_ARG;
  const int batch = c->cfg.max_batch, Hkv = c->cfg.num_kv_heads;
  for (int h = 0; h < Hkv; ++h)
    if (!c->loaded[(size_t)layer * Hkv + h]) return FKV_ERR_NOT_READY;
  long long tiles = 0;
  for (int s = 0; s < batch; ++s)
    tiles += (long long)Hkv * ((c->h_len[(size_t)layer * batch + s] + kScorePPS * kPage - 1) / (kScorePPS * kPage));
  if (tiles == 0) return FKV_OK;
  cudaStream_t st = (cudaStream_t)stream;
  k_plan<<<1, 1024, 0, st>>>(c->ctx, layer, layer + 1, PLAN_SCORE_ALL, kScorePPS * kPage, nullptr, SeqMask{});
  FKV_LAUNCHED(c);
  return launch_score_any(c, scores_out, layer * batch * Hkv, (int)tiles, st);
}

static int select_impl(fkv_cache *c, int layer, const float *scores_in, const float *noise, int noise_stride,
                       int32_t *idx_out, int32_t *kept_count_out, void *stream) {
  if (!c || !layer_ok(c, layer) || !scores_in || !idx_out || !kept_count_out) return FKV_ERR_INVALID_ARG;
  const int batch = c->cfg.max_batch, Hkv = c->cfg.num_kv_heads;
  if (noise)
    for (int s = 0; s < batch; ++s)
      if (sampled_candidates(c->h_len[(size_t)layer * batch + s], c->h_budget[s], c->cfg.recent_keep) > noise_stride)
        return FKV_ERR_INVALID_ARG;
  cudaStream_t st = (cudaStream_t)stream;
  FKV_CUDA(cudaMemsetAsync(kept_count_out, 0, (size_t)batch * Hkv * 4, st));
  k_plan<<<1, 1024, 0, st>>>(c->ctx, layer, layer + 1, PLAN_SELECT, kScorePPS * kPage, nullptr, SeqMask{});
  FKV_LAUNCHED(c);
  int max_old = 0;
  for (int s = 0; s < batch; ++s) max_old = std::max(max_old, c->h_len[(size_t)layer * batch + s]);
  const float *sel_in = scores_in;
  if (noise) {   // keep-priorities go to this layer's part of the workspace scratch
    float *prio = c->ctx.scores + (size_t)layer * batch * Hkv * c->lay.cap;
    launch_select(c, 1, max_old, batch * Hkv, scores_in, nullptr, nullptr, layer * batch * Hkv, 0, prio, noise,
                  noise_stride, layer * batch * Hkv, st);
    FKV_LAUNCHED(c);
    sel_in = prio;
  }
  launch_select(c, 0, max_old, batch * Hkv, sel_in, idx_out, kept_count_out, layer * batch * Hkv, 0, nullptr, nullptr, 0,
                0, st);
  FKV_LAUNCHED(c);
  return FKV_OK;
}

int fkv_select(fkv_cache *c, int layer, const float *scores_in, int32_t *idx_out, int32_t *kept_count_out,
               void *stream) {
  return select_impl(c, layer, scores_in, nullptr, 0, idx_out, kept_count_out, stream);
}

int fkv_select_sampled(fkv_cache *c, int layer, const float *scores_in, const float *noise, int32_t noise_stride,
                       int32_t *idx_out, int32_t *kept_count_out, void *stream) {
  if (!noise || noise_stride < 1) return FKV_ERR_INVALID_ARG;
  return select_impl(c, layer, scores_in, noise, noise_stride, idx_out, kept_count_out, stream);
}

int fkv_compact(fkv_cache *c, int layer, const int32_t *idx, const int32_t *kept_count, void *stream) {
  if (!c || !layer_ok(c, layer) || !idx || !kept_count) return FKV_ERR_INVALID_ARG;
  const int batch = c->cfg.max_batch, Hkv = c->cfg.num_kv_heads;
  int maxn = 0;
  for (int s = 0; s < batch; ++s) maxn = std::max(maxn, c->h_len[(size_t)layer * batch + s]);
  if (maxn == 0) return FKV_OK;
  cudaStream_t st = (cudaStream_t)stream;
  k_plan<<<1, 1024, 0, st>>>(c->ctx, layer, layer + 1, PLAN_COMPACT, kScorePPS * kPage, kept_count, SeqMask{});
  FKV_LAUNCHED(c);
  k_fill_pt_new<<<batch * Hkv, 256, 0, st>>>(c->ctx, layer * batch * Hkv, batch * Hkv);
  FKV_LAUNCHED(c);
  int rc = launch_compact(c, idx, layer * batch * Hkv, maxn, batch * Hkv, st);
  if (rc) return rc;
  k_commit<<<batch * Hkv, 256, 0, st>>>(c->ctx, layer, layer + 1);
  FKV_LAUNCHED(c);
  FKV_CUDA(cudaMemcpyAsync(&c->h_len[(size_t)layer * batch], c->ctx.len + (size_t)layer * batch, (size_t)batch * 4,
                           cudaMemcpyDeviceToHost, st));
  FKV_CUDA(cudaStreamSynchronize(st));
  return FKV_OK;
}

int fkv_export_head(fkv_cache *c, int layer, int seq, int kv_head, void *k, void *v, float *feat, int32_t *pos,
                    void *stream) {
  if (!c || !layer_ok(c, layer) || seq < 0 || seq >= c->cfg.max_batch || kv_head < 0 || kv_head >= c->cfg.num_kv_heads)
    return FKV_ERR_INVALID_ARG;
  const int n = c->h_len[(size_t)layer * c->cfg.max_batch + seq];
  if (n == 0) return FKV_OK;
  k_export_rows<<<(n + 7) / 8, 256, 0, (cudaStream_t)stream>>>(c->ctx, layer, seq, kv_head, (uint8_t *)k, (uint8_t *)v,
                                                               feat, pos);
  FKV_LAUNCHED(c);
  return FKV_OK;
}

int fkv_get_lengths(const fkv_cache *c, int layer, int32_t *host_out) {
  if (!c || !layer_ok(c, layer) || !host_out) return FKV_ERR_INVALID_ARG;
  for (int s = 0; s < c->cfg.max_batch; ++s) host_out[s] = c->h_len[(size_t)layer * c->cfg.max_batch + s];
  return FKV_OK;
}

int fkv_device_status(fkv_cache *c, uint32_t *status_bits, int32_t *free_pages, void *stream) {
  if (!c) return FKV_ERR_INVALID_ARG;
  cudaStream_t st = (cudaStream_t)stream;
  int h[2] = {0, 0};
  FKV_CUDA(cudaMemcpyAsync(h, c->ctx.ctrl, 8, cudaMemcpyDeviceToHost, st));
  FKV_CUDA(cudaStreamSynchronize(st));
  if (h[CTRL_STATUS]) {
    FKV_CUDA(cudaMemsetAsync(c->ctx.ctrl + CTRL_STATUS, 0, 4, st));
    FKV_CUDA(cudaStreamSynchronize(st));
  }
  if (status_bits) *status_bits = (uint32_t)h[CTRL_STATUS];
  if (free_pages) *free_pages = h[CTRL_FREE_TOP];
  return h[CTRL_STATUS] ? FKV_ERR_DEVICE : FKV_OK;
}

int fkv_sync_lengths(fkv_cache *c, void *stream) {
  if (!c) return FKV_ERR_INVALID_ARG;
  cudaStream_t st = (cudaStream_t)stream;
  // Lengths and budgets in one copy (the budgets follow in the workspace): a fork moves both, and when it ran, or whether it found
  // the pages to do anything, the device alone knows.
  FKV_CUDA(cudaMemcpyAsync(c->mirror.data(), c->ctx.len, c->mirror.size() * 4, cudaMemcpyDeviceToHost, st));
  FKV_CUDA(cudaStreamSynchronize(st));
  std::copy_n(c->mirror.begin(), c->h_len.size(), c->h_len.begin());
  std::copy_n(c->mirror.end() - c->cfg.max_batch, c->cfg.max_batch, c->h_budget.begin());
  return FKV_OK;
}

int fkv_set_timing(fkv_cache *c, int on) {
  if (!c) return FKV_ERR_INVALID_ARG;
  if (on)
    for (cudaEvent_t &e : c->ev)
      if (!e) FKV_CUDA(cudaEventCreate(&e));
  c->timing = on != 0;
  c->timed = false;
  return FKV_OK;
}

int fkv_get_evict_timing(fkv_cache *c, float ms_out[6]) {
  if (!c || !ms_out) return FKV_ERR_INVALID_ARG;
  if (!c->timed) return FKV_ERR_NOT_READY;
  FKV_CUDA(cudaEventSynchronize(c->ev[5]));
  for (int i = 0; i < 5; ++i) FKV_CUDA(cudaEventElapsedTime(&ms_out[i], c->ev[i], c->ev[i + 1]));
  FKV_CUDA(cudaEventElapsedTime(&ms_out[5], c->ev[6], c->ev[1]));   // feature refresh: after the plan, before the scorer
  ms_out[0] -= ms_out[5];
  return FKV_OK;
}

int fkv_launch_count(const fkv_cache *c, uint64_t *launches) {
  if (!c || !launches) return FKV_ERR_INVALID_ARG;
  *launches = c->launches;
  return FKV_OK;
}

static int golden_select_launch(const float *alpha, int T, int B, int L, int M, int32_t *kept, cudaStream_t st) {
  if (B > 8192) return FKV_ERR_CAPACITY;   // eight cache entries per thread
  const size_t smem = (size_t)B * 4;
  k_golden_select<<<1, 1024, smem, st>>>(alpha, T, B, L, M, kept);
  FKV_CUDA(cudaGetLastError());
  return FKV_OK;
}

int fkv_golden_steps(int32_t T, int32_t B, int32_t L) {
  if (T < 1 || B < 2 || L < 1 || L >= B) return FKV_ERR_INVALID_ARG;
  const int M = (T - B + L - 1) / L - 1;
  return M < 0 ? 0 : M;
}

int fkv_golden_select(const float *alpha, int32_t T, int32_t B, int32_t L, int32_t M, int32_t *kept_out, void *stream) {
  if (!alpha || !kept_out || M < 1 || fkv_golden_steps(T, B, L) < M) return FKV_ERR_INVALID_ARG;
  return golden_select_launch(alpha, T, B, L, M, kept_out, (cudaStream_t)stream);
}

int fkv_golden_eviction(const float *attn, int32_t g, int32_t T, int32_t B, int32_t L, float *alpha_out,
                        int32_t *kept_out, void *stream) {
  if (!attn || !alpha_out || !kept_out || g < 1) return FKV_ERR_INVALID_ARG;
  const int M = fkv_golden_steps(T, B, L);
  if (M < 0) return M;
  if (M == 0) return FKV_OK;
  if (B > 8192) return FKV_ERR_CAPACITY;
  cudaStream_t st = (cudaStream_t)stream;
  k_golden_pool<<<dim3((T + 255) / 256, M), 256, 0, st>>>(attn, g, T, B, L, alpha_out);
  FKV_CUDA(cudaGetLastError());
  k_golden_suffix_max<<<(T + 255) / 256, 256, 0, st>>>(alpha_out, T, M);
  FKV_CUDA(cudaGetLastError());
  return golden_select_launch(alpha_out, T, B, L, M, kept_out, st);
}

const char *fkv_last_cuda_error(void) { return g_cuda_error.c_str(); }

}  // extern "C"
