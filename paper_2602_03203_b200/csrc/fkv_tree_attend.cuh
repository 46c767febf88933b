// Kernel 10b: attention of draft trees where a launch's fixed cost counts - short caches, few sequences:
//     out_j = sum_i softmax_i(scale <q_j, k_i>) v_i  over the pairs ahead of the tree (window, sinks), j's ancestors and j itself.
// Bound: bytes, 4 D per pair and KV head; for short caches and small trees the latency of one launch and its chain of reads.
// k_chunk_attend computes the same for items of any number that it finds and cuts by itself, behind a store and ahead of a join that are
// launches of their own: 38 us for 16 nodes over 8192 pairs (8 KV heads, g = 4, D = 128), whose bytes take 5.  Here the host says which CTA
// does what, and the call is one launch: 16.9 us.  (256 nodes with a window of 4096: 32.7 us for 75; 33 nodes over 512 pairs, D = 64: 11.6
// for 28.6; all back to back at 1.96 GHz.)
//
// Shape: grid (S, blocks of 128 query rows = (128 / g nodes) x (g heads) of the sequences that have a tree, x KV heads); the S CTAs of a
// block are one cluster, each with a run of its pages.  Inside a CTA everything is as in k_chunk_attend with one tile of query rows (the same tensor
// memory, the same softmax): key tiles go to two streams in turn.
//   warps 0, 2 (and 12, 13)  tensor copies of Q, K and V  warp 1 / 3  tcgen05.mma  S = Q K^T / O += P V          warps 4-11  softmax
// HALF: a launch whose trees all have at most 64 query rows has them twice in the tile, and the second half of the threads takes the
// second half of every key tile's columns: the same products, half the exponentials per thread, four results to join instead of two
// (16 nodes over 8192 pairs: 16.9 us with it, 18.2 without).
// The streams' results meet in shared memory, the CTAs' through distributed shared memory: CTA r of a cluster owns rows r, r + S, ...,
// receives them from all and writes them.
//
// A call that also stores the tree reads its keys and values from the caller's tensors, not from the pages, so no CTA waits for the store:
// some more clusters of the same launch do it (as k_append_chunk does), and of all CTAs the last one to have read the lengths or stored its
// pairs moves the lengths and the free stack.
//
// Where the 17 us go (clocks of one CTA of 10 to a block, cold caches): 0.5 the length, 4 the first scores (page numbers, then pages: two reads of
// memory one after another, descriptors), 1 the first softmax, 0.7 for each of 10 more key tiles (on 80 SMs, 57 GB/s each: a ring of 120 KB at
// the latency of a loaded memory), 0.8 results to shared memory, 1.5 their exchange, 1 the cluster's barrier, 0.9 the join.  Looked at and left out:
// pages asked for into L2 ahead of their copies (the first tile then waits behind them: 18.6 us), one copy for a whole page, K and V in one
// ring (a slot is held from its copy to the product with P: 18.4), V by 16-byte copies of a warp (26.5), products by mma.sync with the pairs on
// the M axis (8 cycles for 16 x 8 x 16: 25 us at 64 rows).
#pragma once
#include "fkv_dev.cuh"
#include "fkv_attend.cuh"
#include "fkv_chunk.cuh"

namespace fkv {

constexpr int kTaMaxCluster = 16;
constexpr int kTaMaxBlocks = 160;     // blocks of a launch, of one KV head (all clusters fit the device at once)
constexpr int kTaRecvRows = 140;      // most of ceil(128 / S) S over S <= 16
template <bool HALF>
constexpr int kTaThreads = kChunkThreads + (HALF ? 64 : 0);   // (a thread with half a tile's columns leaves registers for two more warps)
constexpr int kTaPos = 128;           // positions that are looked at together behind the first window's begin

struct TreeArgs {
  int layer, append;                  // append: the tree is not stored yet
  int window, sinks;
  int rows_y;                         // rows of the grid that attend; those behind store
  float scale_log2;
  const uint8_t *k, *v;               // append: [tokens][Hkv][D] bf16
  const int32_t *pos;                 // append: the nodes' positions or null (one behind the parent's)
  __nv_bfloat16 *out;
  float *lse;
  const uint32_t *masks;
  ChunkLens lens;
  ChunkKeep keep;
  uint8_t seq[kTaMaxBlocks], block[kTaMaxBlocks];   // of every block: its sequence, and which of its blocks
};
static_assert(kMaxBatch <= 256, "a sequence in eight bits");

// What every sequence keeps, takes and returns in a store; worked out by one warp.
struct TreeStore {
  int keep[kMaxBatch], old[kMaxBatch], pop[kMaxBatch], push[kMaxBatch];
  int pops, pushes, top, exhausted;
};
__device__ __forceinline__ void tree_store_plan(const Ctx &c, const TreeArgs &a, TreeStore &ts) {
  const int lane = threadIdx.x & 31;
  int pop[8], push[8], pops = 0, pushes = 0;   // a lane: eight sequences in a row
  const int top = __ldcg(c.ctrl + CTRL_FREE_TOP);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int s = lane * 8 + i;
    pop[i] = push[i] = 0;
    if (s < c.batch) {
      const int nq = __ldcg(c.len + a.layer * c.batch + s), t = a.lens.tok[s + 1] - a.lens.tok[s];
      int kp = a.keep.use ? a.keep.keep[s] : nq;
      if (kp > nq || kp + t > c.cap) kp = -1;
      ts.keep[s] = kp;
      ts.old[s] = nq;
      if (kp >= 0) {
        const int delta = (kp + t + kPage - 1) / kPage - (nq + kPage - 1) / kPage;
        pop[i] = delta > 0 ? delta * c.Hkv : 0;
        push[i] = delta < 0 ? -delta * c.Hkv : 0;
      }
    }
    pops += pop[i];
    pushes += push[i];
  }
  int ip = pops, iq = pushes;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int x = __shfl_up_sync(0xffffffffu, ip, o), y = __shfl_up_sync(0xffffffffu, iq, o);
    if (lane >= o) { ip += x; iq += y; }
  }
  int at = ip - pops, bt = iq - pushes;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int s = lane * 8 + i;
    if (s < c.batch) { ts.pop[s] = at; ts.push[s] = bt; }
    at += pop[i];
    bt += push[i];
  }
  const int all = __shfl_sync(0xffffffffu, ip, 31), back = __shfl_sync(0xffffffffu, iq, 31);
  if (lane == 0) { ts.pops = all; ts.pushes = back; ts.top = top; ts.exhausted = all > top + back; }
  __syncwarp();
}
// The i-th page that sequence q returns: of every head the same number, behind the pages that hold what stays.
__device__ __forceinline__ int tree_store_returned(const Ctx &c, const TreeArgs &a, const TreeStore &ts, int q, int i) {
  const int kept = (ts.keep[q] + a.lens.tok[q + 1] - a.lens.tok[q] + kPage - 1) / kPage, cnt = (ts.old[q] + kPage - 1) / kPage - kept, h = i / cnt;
  return __ldcg(c.pt + (size_t)seg_of(c, a.layer, q, h) * c.max_pages + kept + i - h * cnt);
}
// By the last CTA (one warp of it): returned pages go where the taken ones came from and above, the stack's top and the lengths move,
// decode queries of dropped tokens leave the record (see the end of k_append_chunk).
__device__ __noinline__ void tree_store_finish(const Ctx &c, const TreeArgs &a, TreeStore &ts) {
  const int lane = threadIdx.x & 31;
  __threadfence();
  tree_store_plan(c, a, ts);
  if (lane == 0) {
    c.ctrl[CTRL_CHUNK_TICKET] = 0;
    if (ts.exhausted) set_status(c, kDevPoolExhausted);
  }
  for (int q0 = 0; q0 < c.batch; q0 += 32) {   // a lane per sequence says what there is to do, all lanes do it
    int cnt = 0;
    if (q0 + lane < c.batch) {
      const int s = q0 + lane, kp = ts.keep[s], old = ts.old[s];
      if (kp < 0) set_status(c, a.keep.use && a.keep.keep[s] > old ? kDevBadIndex : kDevCapacity);
      else cnt = ((old + kPage - 1) / kPage - (kp + a.lens.tok[s + 1] - a.lens.tok[s] + kPage - 1) / kPage) * c.Hkv;
    }
    if (ts.exhausted) continue;
    for (unsigned left = __ballot_sync(0xffffffffu, cnt > 0); left; left &= left - 1) {
      const int l = __ffs(left) - 1, q = q0 + l, all = __shfl_sync(0xffffffffu, cnt, l);
      for (int i = lane; i < all; i += 32) {
        const int at = ts.top - ts.pops + ts.push[q] + i;
        if (at >= 0) c.free_stack[at] = tree_store_returned(c, a, ts, q, i);
      }
    }
  }
  __syncwarp();
  if (ts.exhausted) return;
  if (lane == 0) c.ctrl[CTRL_FREE_TOP] = ts.top - ts.pops + ts.pushes;
  for (int s = lane; s < c.batch; s += 32) {
    const int kp = ts.keep[s], ls = a.layer * c.batch + s;
    if (kp < 0) continue;
    c.len[ls] = kp + a.lens.tok[s + 1] - a.lens.tok[s];
    if (c.hist_w && kp < ts.old[s]) {
      const int cnt0 = __ldcg(c.hist_cnt + ls);
      int cnt = cnt0;
      while (cnt > 0 && cnt > cnt0 - c.hist_w && __ldcg(c.hist_n + (size_t)ls * c.hist_w + (cnt - 1) % c.hist_w) > kp) --cnt;
      c.hist_cnt[ls] = (cnt < cnt0 && cnt0 > c.hist_w) ? 0 : cnt;
    }
  }
}
// A CTA's turn in the store's order of arrival, by a whole warp: whether it is the last one.
__device__ __forceinline__ bool tree_store_last(const Ctx &c) {
  int last = 0;
  if ((threadIdx.x & 31) == 0) {
    __threadfence();
    last = atomicAdd(&c.ctrl[CTRL_CHUNK_TICKET], 1) == (int)(gridDim.x * gridDim.y) - 1;
  }
  return __shfl_sync(0xffffffffu, last, 0) != 0;
}
// CTA x of the ones that store: a warp per pair and head.
__device__ __noinline__ void tree_store_cta(const Ctx &c, const TreeArgs &a, TreeStore &ts, int x, int ctas) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, nw = blockDim.x / 32;
  if (warp == 0) tree_store_plan(c, a, ts);
  __syncthreads();
  const int tasks = ts.exhausted ? 0 : a.lens.tok[c.batch] * c.Hkv;
  for (int t = x * nw + warp; t < tasks; t += ctas * nw) {
    const int row = t / c.Hkv, h = t - row * c.Hkv;
    int q = 0, hi = c.batch;   // the sequence of the row: the last one that starts at or before it
    while (hi - q > 1) {
      const int mid = (q + hi) >> 1;
      if (a.lens.tok[mid] <= row) q = mid; else hi = mid;
    }
    const int kp = ts.keep[q];
    if (kp < 0) continue;
    const int j = row - a.lens.tok[q], slot = kp + j, pg = slot / kPage, np_old = (ts.old[q] + kPage - 1) / kPage;
    const int grow = (kp + a.lens.tok[q + 1] - a.lens.tok[q] + kPage - 1) / kPage - np_old;
    int *ptrow = c.pt + (size_t)seg_of(c, a.layer, q, h) * c.max_pages;
    int pid;
    if (pg < np_old) {
      pid = __ldcg(ptrow + pg);
    } else {
      const int y = ts.pop[q] + h * grow + pg - np_old;   // the y-th page that the call takes
      if (y < ts.top) {
        pid = __ldcg(c.free_stack + ts.top - 1 - y);
      } else {
        int r = 0, end = c.batch;   // the sequence that returns page y - top: the last one whose pages begin at or before it
        while (end - r > 1) {
          const int mid = (r + end) >> 1;
          if (ts.push[mid] <= y - ts.top) r = mid; else end = mid;
        }
        pid = tree_store_returned(c, a, ts, r, y - ts.top - ts.push[r]);
      }
      if (lane == 0 && (slot % kPage == 0 || j == 0)) ptrow[pg] = pid;
    }
    int32_t pdef = 0;
    if (!a.pos) {   // one behind the parent's
      pdef = __reduce_add_sync(0xffffffffu, lane < kTreeWords ? tree_before(__ldcg(a.masks + (size_t)row * kTreeWords + lane), lane, j) : 0);
      if (kp > 0) pdef += slot_pos(c, ptrow, kp - 1) + 1;
    }
    const size_t at = ((size_t)row * c.Hkv + h) * c.D * 2;
    move_row<0>(c, c.pool + (size_t)pid * c.page_bytes, slot % kPage, const_cast<uint8_t *>(a.k) + at, const_cast<uint8_t *>(a.v) + at, nullptr,
                a.pos ? const_cast<int32_t *>(a.pos) + row : nullptr, lane, pdef);
  }
  __threadfence();
  __syncthreads();
  if (warp == 0 && tree_store_last(c)) tree_store_finish(c, a, ts);
}

template <int D>
struct TaSmem {
  using CS = ChunkSmem<D>;
  static constexpr int kRow = D + 4;                             // a row of a partial result: O, m, l
  static constexpr size_t kOffK = CS::kTile, kOffV = kOffK + CS::kSlots * CS::kKv, kOffRecv = kOffV + CS::kSlots * CS::kKv;
  static_assert((size_t)2 * kChunkRows * kRow * 4 <= kOffRecv, "the streams' results meet where the operands were");
  static_assert(sizeof(TreeStore) <= (size_t)kTaRecvRows * kRow * 4, "the last CTA's plan, ahead of any row that it receives");
  static constexpr size_t kOffBars = kOffRecv + (size_t)kTaRecvRows * kRow * 4;
  static constexpr size_t kOffWin = kOffBars + 256;              // the search: positions, first slots of the nodes' windows, results
  static constexpr size_t bytes() { return 1024 + kOffWin + (kTaPos + kChunkRows + 4) * 4; }
};

// 16 rows of a head in the caller's keys (64 channels) or values (all): per 64 channels 16 rows of 128 swizzled bytes.
__device__ __forceinline__ void tma_rows(uint32_t dst, const CUtensorMap *tm, int row, int part, int head, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
      ::"r"(dst), "l"(reinterpret_cast<uint64_t>(tm)), "r"(0), "r"(row), "r"(part), "r"(head), "r"(bar)
      : "memory");
}

__device__ __forceinline__ void tmem_ld8_issue(uint32_t taddr, uint32_t (&r)[8]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "r"(taddr)
               : "memory");
}
__device__ __forceinline__ void tmem_ld8_wait(uint32_t (&r)[8]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7])
               :
               : "memory");
}
__device__ __forceinline__ void tmem_st4(uint32_t taddr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x4.b32 [%4], {%0, %1, %2, %3};" ::"r"(a), "r"(b), "r"(c), "r"(d), "r"(taddr) : "memory");
}
// chunk_weights for columns in groups of eight.  P is stored when all of it has been worked out: its columns are free only when the products
// with the tile before are done, and the exponentials run meanwhile.
template <int NG, class Ready>
__device__ __forceinline__ void half_weights(const uint32_t (&v)[NG][8], float scale_log2, float ms, uint32_t tp, Ready ready, float &lt, float &mx) {
  float m2[2] = {-INFINITY, -INFINITY};
  float2 l2[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
  const float2 sc = make_float2(scale_log2, scale_log2), off = make_float2(-ms, -ms);
  uint32_t p[NG][4];
#pragma unroll
  for (int g = 0; g < NG; ++g) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float2 z = make_float2(__uint_as_float(v[g][2 * j]), __uint_as_float(v[g][2 * j + 1]));
      float2 x = __ffma2_rn(z, sc, off);
      x.x = ex2(x.x);
      x.y = ex2(x.y);
      m2[j & 1] = max3(m2[j & 1], z.x, z.y);
      l2[j & 1] = __fadd2_rn(l2[j & 1], x);
      p[g][j] = pack_bf16(x.x, x.y);
    }
  }
  ready();
#pragma unroll
  for (int g = 0; g < NG; ++g) tmem_st4(tp + g * 4, p[g][0], p[g][1], p[g][2], p[g][3]);
  mx = fmaxf(m2[0], m2[1]);
  lt = (l2[0].x + l2[0].y) + (l2[1].x + l2[1].y);
}

template <int D, bool WIN, bool HALF>
__global__ void __launch_bounds__(kTaThreads<HALF>, 1) k_tree_attend(const __grid_constant__ Ctx c, const __grid_constant__ CUtensorMap tmk,
                                                                  const __grid_constant__ CUtensorMap tmv,
                                                                  const __grid_constant__ CUtensorMap tmq,
                                                                  const __grid_constant__ CUtensorMap tki,
                                                                  const __grid_constant__ CUtensorMap tvi,
                                                                  const __grid_constant__ TreeArgs a) {
  using CS = ChunkSmem<D>;
  using SM = TaSmem<D>;
  constexpr int NS = CS::kSlots, NQ = D / 64, TP = CS::kPages, ROW = SM::kRow;
  constexpr uint32_t PAGE_HALF = kPage * 128;
  constexpr int THREADS = kTaThreads<HALF>;
  constexpr int BR = HALF ? kChunkRows / 2 : kChunkRows, HC = CS::kCols / 2;   // query rows of a block; columns of half a key tile
  extern __shared__ uint8_t smem_raw[];
  uint8_t *smem = reinterpret_cast<uint8_t *>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  uint8_t *Qt = smem, *Kt = smem + SM::kOffK, *Vt = smem + SM::kOffV;
  float *recv = reinterpret_cast<float *>(smem + SM::kOffRecv), *mg = reinterpret_cast<float *>(smem);
  uint64_t *bars = reinterpret_cast<uint64_t *>(smem + SM::kOffBars);
  uint64_t *k_full = bars, *k_empty = k_full + NS, *v_full = k_empty + NS, *v_empty = v_full + NS, *q_full = v_empty + NS;
  uint64_t *s_full = q_full + 1, *s_empty = s_full + 2, *p_full = s_empty + 2, *p_empty = p_full + 2, *mma_done = p_empty + 2;
  uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(mma_done + 1);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, G = c.G, TPT = BR / G;
  const int S = gridDim.x, rank = blockIdx.x, head = blockIdx.y % c.Hkv, sb = blockIdx.y / c.Hkv;
  if ((int)blockIdx.y >= a.rows_y) {
    griddep_wait();
    griddep_launch();
    tree_store_cta(c, a, *reinterpret_cast<TreeStore *>(smem), (blockIdx.y - a.rows_y) * S + rank, (gridDim.y - a.rows_y) * S);
    return;
  }
  const int seq = a.seq[sb], row0 = a.lens.tok[seq], T = a.lens.tok[seq + 1] - row0, j0 = a.block[sb] * TPT, j1 = min(T, j0 + TPT);   // nodes [j0, j1)

  if (warp == 3) tmem_alloc(smem_u32(tmem_slot), 512);
  if (threadIdx.x == 0) {
    for (const CUtensorMap *tm : {&tmk, &tmv, &tmq, &tki, &tvi}) asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(tm)) : "memory");
    for (int s = 0; s < NS; ++s) {
      mbar_init(smem_u32(&k_full[s]), 1); mbar_init(smem_u32(&k_empty[s]), 1);
      mbar_init(smem_u32(&v_full[s]), 1); mbar_init(smem_u32(&v_empty[s]), 1);
    }
    mbar_init(smem_u32(q_full), 1);
    for (int t = 0; t < 2; ++t) {
      mbar_init(smem_u32(&s_full[t]), 1); mbar_init(smem_u32(&s_empty[t]), 4);
      mbar_init(smem_u32(&p_full[t]), 4); mbar_init(smem_u32(&p_empty[t]), 1);
    }
    mbar_init(smem_u32(mma_done), 2);
    fence_barrier_init();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  griddep_wait();
  griddep_launch();
  if (warp == 0 && lane == 0) {   // (the queries do not depend on the lengths)
    mbar_arrive_expect_tx(smem_u32(q_full), (uint32_t)(NQ * TPT * G * 128 * (HALF ? 2 : 1)));
    for (int q = 0; q < NQ; ++q)
      for (int h = 0; h < (HALF ? 2 : 1); ++h)
        tma_chunk_q(smem_u32(Qt + (size_t)q * 128 * 128 + (size_t)h * BR * 128), &tmq, q * 64, head * G, row0 + j0, smem_u32(q_full));
  }
  const int ls = a.layer * c.batch + seq;
  const int n_old = __ldcg(c.len + ls);
  __syncthreads();   // every thread has read the length
  if (a.append && warp == 1 && tree_store_last(c)) tree_store_finish(c, a, *reinterpret_cast<TreeStore *>(recv));
  __syncwarp();
  // "I am running, and my place for the rows that I receive is free": waited for ahead of the exchange.
  if (S > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  const int kp = a.append ? (a.keep.use ? a.keep.keep[seq] : n_old) : n_old - T;   // pairs ahead of the tree
  const bool bad = kp < 0 || kp > n_old || kp + T > c.cap;   // (the store says so where there is one)
  if (bad && !a.append && rank == 0 && head == 0 && threadIdx.x == 0) set_status(c, kDevBadIndex);
  const bool active = !bad;
  const int stored = a.append ? kp : kp + T;       // pairs that the pages hold
  const int *ptrow = c.pt + (size_t)(ls * c.Hkv + head) * c.max_pages;
  int *s_pos = reinterpret_cast<int *>(smem + SM::kOffWin), *s_wlo = s_pos + kTaPos, *s_win = s_wlo + kChunkRows;
  // With a window: of the pairs ahead of the tree the block's nodes see slots [0, wa) (sinks) and from s_wlo[node] on, wb the first of these.
  int wa = 0, wb = 0;
  if (WIN) {   // (a window holds all of the tree: it is not shorter than the tree has nodes)
    if (warp == 1 && active) {
      const int W = a.window;
      // The lowest position of the block's nodes: stored ones, given ones, or by the number of nodes on their paths.
      const int lo0 = max(0, kp + 1 - W);
      const int x0 = kp > 0 ? slot_pos(c, ptrow, min(lo0, kp - 1)) : 0;
      const int last = a.append && !a.pos && kp > 0 ? slot_pos(c, ptrow, kp - 1) : -1;
      const int sk = a.sinks ? slot_sinks(c, ptrow, kp, a.sinks) : 0;
      int p[4], low = INT_MAX;   // (a block has at most 128 nodes)
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int j = j0 + lane + 32 * u;
        p[u] = INT_MAX;
        if (j >= j1) continue;
        if (!a.append) {
          p[u] = slot_pos(c, ptrow, kp + j);
        } else if (a.pos) {
          p[u] = __ldcg(a.pos + row0 + j);
        } else {
          const uint32_t *row = a.masks + (size_t)(row0 + j) * kTreeWords;
          p[u] = last + 1;
#pragma unroll
          for (int w = 0; w < kTreeWords; ++w) p[u] += tree_before(__ldcg(row + w), w, j);
        }
        low = min(low, p[u]);
      }
      low = __reduce_min_sync(0xffffffffu, low);
      const int start = window_start(low, W);
      const int f = lo0 >= kp ? kp : x0 >= start ? lo0 : slot_lower_bound_warp(c, ptrow, lo0 + 1, kp, start);
      for (int i = lane; i < kTaPos && f + i < kp; i += 32) s_pos[i] = slot_pos(c, ptrow, f + i);
      __syncwarp();
#pragma unroll
      for (int u = 0; u < 4; ++u) {   // a window that begins d positions later begins at most d slots later
        const int j = j0 + lane + 32 * u;
        if (j >= j1) continue;
        const int from = window_start(p[u], W);
        int lo = f, hi = (int)min((long long)kp, f + (long long)p[u] - low);
        if (hi - f < kTaPos) {
          while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (s_pos[mid - f] < from) lo = mid + 1; else hi = mid;
          }
        } else {
          lo = slot_lower_bound(c, ptrow, lo, hi, from);
        }
        s_wlo[j - j0] = lo;
      }
      if (lane == 0) { s_win[0] = sk; s_win[1] = max(sk, f); }
    }
    __syncthreads();
    if (active) { wa = s_win[0]; wb = s_win[1]; }
  }
  // Units of 16 rows: pages of the sinks, the other pages, then (append) groups of nodes; this CTA's run of them in key tiles of up to TP,
  // the three kinds apart.
  const int np = a.append ? (kp + kPage - 1) / kPage : (kp + j1 + kPage - 1) / kPage;
  const int sp_all = (wa + kPage - 1) / kPage, wp = max(sp_all, wb / kPage), nb = sp_all + max(0, np - wp), nu = nb + (a.append ? (j1 + kPage - 1) / kPage : 0);
  const int per = (nu + S - 1) / S, u0 = min(nu, rank * per), u1 = min(nu, u0 + per);
  const int s0 = min(u0, sp_all), s1 = min(u1, sp_all), shift = wp - sp_all;
  const int pa = min(max(u0, sp_all), nb) + shift, pb = min(max(u1, sp_all), nb) + shift, ga = max(u0, nb) - nb, gb = max(u1, nb) - nb;
  const int ns = (s1 - s0 + TP - 1) / TP, na = ns + (pb - pa + TP - 1) / TP, nt = active ? na + (gb - ga + TP - 1) / TP : 0;
  auto first = [&](int i) { return i < ns ? s0 + TP * i : i < na ? pa + TP * (i - ns) : ga + TP * (i - na); };   // of tile i: its first page, or group
  auto units = [&](int i) { return min(TP, (i < ns ? s1 : i < na ? pb : gb) - first(i)); };

  float m = -INFINITY, l = 0.f;
  if (warp >= 4 && warp < 12) {
    // ---------------- softmax: thread = query row, warpgroup = stream (see k_chunk_attend) ----------------
    const int t = (warp - 4) >> 2, quarter = warp & 3, R = quarter * 32 + lane, tok = R % BR / G, node = j0 + tok;
    const int c0 = HALF ? R / BR * HC : 0;   // this thread's first column of every key tile (the same in a warp)
    const bool live = tok < TPT && node < j1;
    const bool any = __any_sync(0xffffffffu, live);
    const uint32_t ts = tmem_base + ((uint32_t)(quarter * 32) << 16) + t * CS::kStream, tp = ts + CS::kColP, to = ts + CS::kColO;
    const int wlo = WIN && live ? s_wlo[tok] : 0;
    uint32_t sp = 0, pe = 1;
    bool ok = true;
    if (HALF) {   // the other half's weights are zero all along
#pragma unroll
      for (int g = 0; g < HC / 8; ++g) tmem_st4(tp + (HC - c0) / 2 + g * 4, 0u, 0u, 0u, 0u);
      tmem_st_wait();
    }
    for (int i = t; i < nt; i += 2) {
      const int f = first(i), cols = units(i) * kPage;
      // Node of the thread's first column in the tile, and the columns that hold pairs up to the row's own.
      const int at = (i < na ? f * kPage - kp : f * kPage) + c0;
      const int hi = live ? min(cols - c0, min(node + 1 - at, i < na ? stored - f * kPage - c0 : INT_MAX)) : INT_MAX;
      const bool in_tree = at - c0 + cols > 0;
      const int lo = WIN && i < na ? wlo - f * kPage - c0 : 0, sk = WIN ? wa - f * kPage - c0 : 0;   // with a window: columns [0, sk) and from lo on
      constexpr int NCOL = HALF ? HC : CS::kCols;
      if (!mbar_sleep_warp(smem_u32(&s_full[t]), sp)) { set_status(c, kDevWaitTimeout); break; }
      sp ^= 1;
      tc_fence_after();
      bool waited = false;
      auto wait_products = [&]() {   // the products with P of the tile before: P's columns are free, and O may be rescaled
        if (waited) return;
        waited = true;
        if (!mbar_sleep_warp(smem_u32(&p_empty[t]), pe)) { set_status(c, kDevWaitTimeout); ok = false; }
        pe ^= 1;
        tc_fence_after();
      };
      if (any) {
        uint32_t v[HALF ? HC / 8 : TP][HALF ? 8 : 16];
        if constexpr (HALF) {
#pragma unroll
          for (int g = 0; g < HC / 8; ++g) tmem_ld8_issue(ts + c0 + g * 8, v[g]);
#pragma unroll
          for (int g = 0; g < HC / 8; ++g) tmem_ld8_wait(v[g]);
        } else {
#pragma unroll
          for (int q = 0; q < TP; ++q) tmem_ld16_issue(ts + q * 16, v[q]);
#pragma unroll
          for (int q = 0; q < TP; ++q) tmem_ld16_wait(v[q]);
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&s_empty[t]));
        if (!__all_sync(0xffffffffu, hi >= NCOL && (!WIN || lo <= 0 || sk >= NCOL) && !in_tree)) {   // hidden scores become -infinity
          asm volatile("" ::: "memory");
          uint32_t see[3];
          const int k = at >> 5;
          const uint32_t *row = a.masks + (size_t)(row0 + node) * kTreeWords;
          uint32_t w[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) w[j] = !live || k + j < 0 ? ~0u : k + j < kTreeWords ? __ldcg(row + k + j) : 0u;
          auto below = [](int e) { return e <= 0 ? 0u : e >= 32 ? ~0u : (1u << e) - 1u; };   // bits under e
#pragma unroll
          for (int j = 0; j < 3; ++j)
            see[j] = __funnelshift_r(w[j], w[j + 1], at & 31) & below(hi - 32 * j) & (WIN ? below(sk - 32 * j) | ~below(lo - 32 * j) : ~0u);
          constexpr int W = HALF ? 8 : 16;
#pragma unroll
          for (int q = 0; q < NCOL / W; ++q)
#pragma unroll
            for (int j = 0; j < W; ++j)
              if (!((see[(q * W + j) / 32] >> ((q * W + j) % 32)) & 1u)) v[q][j] = 0xff800000u;
        }
        float mx, lt;
        auto weights = [&](float ms) {
          if constexpr (HALF) half_weights<HC / 8>(v, a.scale_log2, ms, tp + c0 / 2, wait_products, lt, mx);
          else chunk_weights<TP>(v, a.scale_log2, ms, tp, wait_products, lt, mx);
        };
        weights(m == -INFINITY ? 0.f : m * a.scale_log2);
        const bool grow = mx > m && (mx - m) * a.scale_log2 > kChunkGrow;
        if (__any_sync(0xffffffffu, grow)) {
          tmem_st_wait();
          const float fa = grow ? ex2((m - mx) * a.scale_log2) : 1.f;
          if (grow) m = mx;
          l *= fa;
          if (i != t) {
#pragma unroll 1
            for (int q = 0; q < D; q += 16) {
              uint32_t o[16];
              tmem_ld16_issue(to + q, o);
              tmem_ld16_wait(o);
#pragma unroll
              for (int j = 0; j < 16; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * fa);
              tmem_st16(to + q, o);
            }
          }
          weights(m == -INFINITY ? 0.f : m * a.scale_log2);
        }
        l += lt;
        tmem_st_wait();
      } else {   // (no row of the warp is in use: only the hand-overs)
        if (lane == 0) mbar_arrive(smem_u32(&s_empty[t]));
        wait_products();
      }
      if (!ok) break;
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&p_full[t]));
    }
  } else if (warp == 0 || warp == 2 || warp >= 12) {
    // ---------------- copies of K / V, a lane per copy ----------------
    // A warp takes 100 - 150 cycles to issue a copy.  For a tile of five pages that is 1450 cycles of K (ten copies) on one warp, more than all
    // the rest of 64 rows takes, so two warps share K and two V there.
    const bool keys = warp == 0 || warp == 12, lead = warp < 12;
    uint64_t *full = keys ? k_full : v_full, *empty = keys ? k_empty : v_empty;
    FeatRing rr{0, 0};
    uint32_t armed = 0, armed_par = 0;    // bit s: slot s has been armed / its last parity
    constexpr int CW = (THREADS - kChunkThreads) / 64 + 1;   // warps for K, and for V
    const int all = keys ? NQ * TP : TP, share = (all + CW - 1) / CW, e = lane + (lead ? 0 : share);   // this lane's copy of a tile: (channels, page) of K
    const bool on = lane < share && e < all;
    const int pg = e % TP, half = e / TP;
    uint8_t *mine = keys ? Kt + (size_t)half * TP * PAGE_HALF + (size_t)pg * PAGE_HALF : Vt + (size_t)pg * NQ * PAGE_HALF;
    auto page_id = [&](int i) { return on && i < nt && i < na && pg < units(i) ? __ldcg(ptrow + first(i) + pg) : 0; };
    int id = page_id(0);
    for (int i = 0; i < nt; ++i) {
      const int idn = page_id(i + 1), n16 = units(i);
      if (!mbar_sleep_warp(smem_u32(&empty[rr.i]), rr.ph ^ 1)) { set_status(c, kDevWaitTimeout); break; }
      const uint32_t bar = smem_u32(&full[rr.i]), dst = smem_u32(mine + rr.i * CS::kKv);
      if (lead && lane == 0) mbar_arrive_expect_tx(bar, (uint32_t)(n16 * NQ) * PAGE_HALF);   // (of both warps)
      armed |= 1u << rr.i;
      armed_par = (armed_par & ~(1u << rr.i)) | ((uint32_t)rr.ph << rr.i);
      __syncwarp();
      if (on && pg < n16) {
        if (i >= na) tma_rows(dst, keys ? &tki : &tvi, row0 + (first(i) + pg) * kPage, keys ? half : 0, head, bar);
        else if (keys) tma_page_k(dst, &tmk, half, id, bar);
        else tma_page_v(dst, &tmv, NQ, id, bar);
      }
      rr.next(NS);
      id = idn;
    }
#pragma unroll
    for (int s = 0; s < NS; ++s)   // no copy may be in flight at the exit
      if (((armed >> s) & 1u) && !mbar_sleep_warp(smem_u32(&full[s]), (armed_par >> s) & 1u)) set_status(c, kDevWaitTimeout);
    if (warp == 0 && !mbar_sleep_warp(smem_u32(q_full), 0)) set_status(c, kDevWaitTimeout);
  } else {
    // ---------------- multiplies: a warp stays together, lane 0 issues ----------------
    const bool scores = warp == 1;
    const uint32_t on = lane == 0, tb = uniform(tmem_base);
    FeatRing r{0, 0};
    uint32_t se = 3, pp = 0;   // bit t: parities of stream t's next s_empty, p_full
    const uint32_t idesc_o = umma_idesc_bf16(kChunkRows, D) | (1u << 16);   // B runs along N
    uint64_t *full = scores ? k_full : v_full, *empty = scores ? k_empty : v_empty;
    bool ok = true;
    if (scores && nt > 0 && !mbar_wait(smem_u32(q_full), 0)) { set_status(c, kDevWaitTimeout); ok = false; }
    for (int i = 0; i < nt && ok; ++i) {
      const int n16 = uniform(units(i)), slot = uniform(r.i), t = i & 1;
      if (!__all_sync(0xffffffffu, mbar_wait(smem_u32(&full[slot]), r.ph))) { set_status(c, kDevWaitTimeout); break; }
      r.next(NS);
      const uint32_t ts = tb + t * CS::kStream;
      if (scores) {
        const uint64_t kd = umma_desc_sw128(smem_u32(Kt + slot * CS::kKv)), qd = umma_desc_sw128(smem_u32(Qt));
        const uint32_t idesc = umma_idesc_bf16(kChunkRows, n16 * kPage);
        if (!__all_sync(0xffffffffu, mbar_wait(smem_u32(&s_empty[t]), (se >> t) & 1))) { set_status(c, kDevWaitTimeout); break; }
        se ^= 1u << t;
        tc_fence_after();
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks)
          umma_bf16_if(on, ts, qd + (uint64_t)(((ks >> 2) * 128 * 128 + (ks & 3) * 32) >> 4),
                       kd + (uint64_t)(((ks >> 2) * TP * (int)PAGE_HALF + (ks & 3) * 32) >> 4), idesc, ks > 0);
        umma_commit_if(on, smem_u32(&s_full[t]));
      } else {
        // Rows that no node of the block sees, behind the last pair or between sinks and windows, are cleared (P is zero there, but
        // zero times an infinity is not).
        const int f16 = first(i) * kPage, end = i < na ? stored : T, gap0 = WIN && i < na ? wa : 0, gap1 = WIN && i < na ? wb : 0;
        if (f16 + n16 * kPage > end || (f16 < gap1 && f16 + n16 * kPage > gap0)) {
          for (int e = lane; e < n16 * kPage * NQ * 8; e += 32) {
            const int row = e / (NQ * 8), ch = e % (NQ * 8), at = f16 + row;
            if (at < end && (at < gap0 || at >= gap1)) continue;
            *reinterpret_cast<uint4 *>(Vt + slot * CS::kKv + (size_t)((row / kPage * NQ + (ch >> 3)) * kPage + row % kPage) * 128 +
                                       (ch & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
          }
          fence_proxy_async();
          __syncwarp();
        }
        const uint64_t vd = umma_desc_mn_sw128(smem_u32(Vt + slot * CS::kKv));
        const uint32_t tp = ts + CS::kColP, to = ts + CS::kColO;
        if (!__all_sync(0xffffffffu, mbar_wait(smem_u32(&p_full[t]), (pp >> t) & 1))) { set_status(c, kDevWaitTimeout); break; }
        pp ^= 1u << t;
        tc_fence_after();
        for (int ks = 0; ks < n16; ++ks) umma_bf16_ta_if(on, to, tp + ks * 8, vd + (uint64_t)((ks * NQ * PAGE_HALF) >> 4), idesc_o, ks > 0 || i >= 2);
        umma_commit_if(on, smem_u32(&p_empty[t]));
      }
      umma_commit_if(on, smem_u32(&empty[slot]));
    }
    umma_commit_if(on, smem_u32(mma_done));
    if (!mbar_wait(smem_u32(mma_done), 0)) set_status(c, kDevWaitTimeout);
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();   // all copies have landed, all products are done: the operands' memory is free
  tc_fence_after();
  if (active) {
    // ---- the streams' results: [stream][row][O, m, l] ----
    if (warp >= 4 && warp < 12) {
      const int t = (warp - 4) >> 2, quarter = warp & 3, R = quarter * 32 + lane;
      const uint32_t to = tmem_base + ((uint32_t)(quarter * 32) << 16) + t * CS::kStream + CS::kColO;
      float *r = mg + (size_t)(t * kChunkRows + R) * ROW;
      if (t < nt)
#pragma unroll 2
        for (int q = 0; q < D; q += 16) {
          uint32_t o[16];
          tmem_ld16_issue(to + q, o);
          tmem_ld16_wait(o);
#pragma unroll
          for (int j = 0; j < 4; ++j)
            *reinterpret_cast<uint4 *>(r + q + 4 * j) = make_uint4(o[4 * j], o[4 * j + 1], o[4 * j + 2], o[4 * j + 3]);
        }
      // (a row whose scores are all NaN has found no maximum, but must not count as one that saw nothing)
      *reinterpret_cast<float2 *>(r + D) = make_float2(l != l ? 0.f : m, l);
      tc_fence_before();
    }
  }
  __syncthreads();
  if (warp == 3) { tc_fence_after(); tmem_dealloc(tmem_base, 512); }
  if (S > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");   // every CTA of the cluster runs
  if (!active) return;   // (of the whole cluster alike)
  const int rows = (j1 - j0) * G;
  // A row's result, four channels per lane.
  auto finish = [&](int r, float4 acc, float M, float L) {
    const float inv = L == 0.f ? 0.f : 1.f / L;   // a row that sees nothing gives zeros
    const size_t orow = ((size_t)(row0 + j0 + r / G) * c.Hkv + head) * G + r % G;
    if (lane * 4 < D) *reinterpret_cast<uint2 *>(a.out + orow * D + lane * 4) = make_uint2(pack_bf16(acc.x * inv, acc.y * inv), pack_bf16(acc.z * inv, acc.w * inv));
    if (a.lse && lane == 0) a.lse[orow] = L == 0.f ? -INFINITY : (M * a.scale_log2 + log2f(L)) * 0.6931471805599453f;
  };
  auto weight = [&](float mi, float M) { return mi == -INFINITY ? 0.f : ex2((mi - M) * a.scale_log2); };
  // ---- a warp per row joins its results (of two streams, and of two halves) and sends it to its owner.  (A short loop: this code runs a
  // few times per launch, and to fetch it costs more than its arithmetic; four rows at a time take 1.5 us longer.) ----
  constexpr int NW = THREADS / 32, NP = HALF ? 4 : 2;
#pragma unroll 1
  for (int r = warp; r < rows; r += NW) {
    const float *p = mg + (size_t)r * ROW;
    float2 x[NP];
    float M = -INFINITY, L = 0.f;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      x[i] = *reinterpret_cast<const float2 *>(p + i * BR * ROW + D);
      M = fmaxf(M, x[i].x);
    }
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const float f = weight(x[i].x, M);
      L = fmaf(f, x[i].y, L);   // (l is 0 where nothing was seen)
      if (lane * 4 < D && f != 0.f) {   // (what was never written is not read)
        const float4 v = *reinterpret_cast<const float4 *>(p + i * BR * ROW + lane * 4);
        acc.x = fmaf(f, v.x, acc.x); acc.y = fmaf(f, v.y, acc.y); acc.z = fmaf(f, v.z, acc.z); acc.w = fmaf(f, v.w, acc.w);
      }
    }
    if (S == 1) {
      finish(r, acc, M, L);
    } else {
      const int block = r / S;
      const uint32_t to = dsmem_addr(smem_u32(recv + (size_t)(block * S + rank) * ROW), r - block * S);
      if (lane * 4 < D) dsmem_st4(to + lane * 16, acc);
      if (lane == 0) dsmem_st2(to + D * 4, M, L);
    }
  }
  if (S == 1) return;
  cluster_sync_all();
  // ---- a warp per own row: lane s has the statistics of part s ----
  for (int r = rank + warp * S; r < rows; r += NW * S) {
    const float *p = recv + (size_t)(r / S * S) * ROW;
    const float2 x = lane < S ? *reinterpret_cast<const float2 *>(p + lane * ROW + D) : make_float2(-INFINITY, 0.f);
    float M = x.x;
#pragma unroll
    for (int sh = 8; sh >= 1; sh >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, sh));
    M = __shfl_sync(0xffffffffu, M, 0);
    const float f = weight(x.x, M);
    float L = f * x.y;
#pragma unroll
    for (int sh = 8; sh >= 1; sh >>= 1) L += __shfl_xor_sync(0xffffffffu, L, sh);
    L = __shfl_sync(0xffffffffu, L, 0);
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int s = 0; s < S; ++s) {
      const float fs = __shfl_sync(0xffffffffu, f, s);
      if (lane * 4 < D) {
        const float4 v = *reinterpret_cast<const float4 *>(p + s * ROW + lane * 4);
        acc.x = fmaf(fs, v.x, acc.x); acc.y = fmaf(fs, v.y, acc.y); acc.z = fmaf(fs, v.z, acc.z); acc.w = fmaf(fs, v.w, acc.w);
      }
    }
    finish(r, acc, M, L);
  }
}

}  // namespace fkv
