// Kernel 10: draft trees around the attention (k_append_chunk<true>, k_chunk_attend<D, true>): masks from parents, the accepted
// path moved together, and the read-out of a chunk.
#pragma once
#include "fkv_dev.cuh"
#include "fkv_attend.cuh"
#include "fkv_chunk.cuh"

namespace fkv {

// ---------------------------------------------------------------- masks
// mask(j) = {j} u mask(parent(j)), by doubling: after round r a node's mask holds its 2^r nearest ancestors and its pointer the next
// one, so the rounds are log2 of the depth.  grid = sequences, a thread per node.  A parent that does not come before its node is an
// error: the node becomes a root.  Bound: latency (a launch, one read, a few rounds in shared memory): 1.7 us for 16 nodes, 3.2 for 256.
__global__ void __launch_bounds__(kTreeNodes) k_tree_masks(Ctx c, const __grid_constant__ ChunkLens lens, const int32_t *parents, uint32_t *masks) {
  __shared__ uint32_t m[2][kTreeWords][kTreeNodes];
  __shared__ short up[2][kTreeNodes];
  griddep_wait();
  griddep_launch();
  const int row0 = lens.tok[blockIdx.x], T = lens.tok[blockIdx.x + 1] - row0, j = threadIdx.x;
  if (T == 0) return;
  int p = -1;
  if (j < T) {
    p = __ldcg(parents + row0 + j);
    if (p < -1 || p >= j) { set_status(c, kDevBadIndex); p = -1; }
  }
  uint32_t own[kTreeWords];
#pragma unroll
  for (int w = 0; w < kTreeWords; ++w) own[w] = w == j / 32 ? 1u << (j & 31) : 0u;
  for (int r = 0; __syncthreads_or(p >= 0); r ^= 1) {   // (the barrier also ends the reads of this half two rounds ago)
#pragma unroll
    for (int w = 0; w < kTreeWords; ++w) m[r][w][j] = own[w];
    up[r][j] = (short)p;
    __syncthreads();
    if (p >= 0) {
#pragma unroll
      for (int w = 0; w < kTreeWords; ++w) own[w] |= m[r][w][p];
      p = up[r][p];
    }
  }
  if (j < T) {
    uint4 *out = reinterpret_cast<uint4 *>(masks + (size_t)(row0 + j) * kTreeWords);
    out[0] = make_uint4(own[0], own[1], own[2], own[3]);
    out[1] = make_uint4(own[4], own[5], own[6], own[7]);
  }
}

// ---------------------------------------------------------------- the accepted path
// grid (layers, sequences), 32 warps: of a sequence's last T pairs, the tree's, those of path[0 .. cnt) (ascending) move to the
// places behind the pairs ahead of the tree; the length follows and the pages behind are returned.
// A pair never moves up (path[i] >= i), and its place may be another's source: 128 / Hkv places of every head are read into
// registers, then written, then the next ones (whose sources lie behind all places written so far).
// Bound: latency (a launch, length and path, page ids, rows); bytes are those of the moved pairs, read and written.  Back to back with
// the store of the tree 6.8 us, of which the store takes 5.0.
__global__ void __launch_bounds__(1024) k_commit_tree(Ctx c, int l0, const __grid_constant__ ChunkLens lens, const int32_t *path,
                                                      const int32_t *path_len, int stride) {
  __shared__ int s_path[kTreeNodes];
  __shared__ int s_push;
  griddep_wait();
  griddep_launch();
  const int seq = blockIdx.y, layer = l0 + blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int T = lens.tok[seq + 1] - lens.tok[seq], ls = layer * c.batch + seq;
  if (T == 0) return;
  const int n = __ldcg(c.len + ls), cnt = __ldcg(path_len + seq), base = n - T;
  bool bad = base < 0 || cnt < 0 || cnt > T || cnt > stride;
  bool moved = false;
  if (!bad && tid < cnt) {
    const int p = __ldcg(path + (size_t)seq * stride + tid), before = tid > 0 ? __ldcg(path + (size_t)seq * stride + tid - 1) : -1;
    bad = p <= before || p >= T;
    moved = p != tid;
    s_path[tid] = p;
  }
  if (__syncthreads_or(bad)) {
    if (tid == 0) set_status(c, kDevBadIndex);
    return;
  }
  const int first = cnt - __syncthreads_count(moved);   // (once a pair moves, so do all behind it)
  const int per = max(1, 128 / c.Hkv), W = c.F + 1;
  for (int i0 = first; i0 < cnt; i0 += per) {
    const int tasks = min(per, cnt - i0) * c.Hkv;
    uint4 kv[4];
    uint32_t meta[4][2];
    auto place = [&](int t, int slot, int &r) {   // page and row of a slot of the task's head
      r = slot % kPage;
      return c.pool + (size_t)__ldcg(c.pt + (size_t)seg_of(c, layer, seq, t % c.Hkv) * c.max_pages + slot / kPage) * c.page_bytes;
    };
    auto chunk = [&](int r) { return lane < c.D / 8 ? kv_chunk_off(r, lane, c.D) : c.off_v + kv_chunk_off(r, lane - c.D / 8, c.D); };
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int t = warp + 32 * u;
      if (t >= tasks) continue;
      int r;
      const uint8_t *page = place(t, base + s_path[i0 + t / c.Hkv], r);
      if (lane < c.D / 4) kv[u] = __ldcg(reinterpret_cast<const uint4 *>(page + chunk(r)));
      const uint32_t *row = reinterpret_cast<const uint32_t *>(meta_row(c, page, r));
      if (lane < W) meta[u][0] = __ldcg(row + lane);
      if (lane + 32 < W) meta[u][1] = __ldcg(row + lane + 32);
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int t = warp + 32 * u;
      if (t >= tasks) continue;
      int r;
      uint8_t *page = place(t, base + i0 + t / c.Hkv, r);
      if (lane < c.D / 4) *reinterpret_cast<uint4 *>(page + chunk(r)) = kv[u];
      uint32_t *row = reinterpret_cast<uint32_t *>(meta_row(c, page, r));
      if (lane < W) row[lane] = meta[u][0];
      if (lane + 32 < W) row[lane + 32] = meta[u][1];
    }
    __syncthreads();
  }
  // Pages behind the path go back to the stack (only pushes happen here; their order does not matter).
  const int kept = (base + cnt + kPage - 1) / kPage, gone = (n + kPage - 1) / kPage - kept;
  if (tid == 0) {
    if (gone > 0) s_push = atomicAdd(&c.ctrl[CTRL_FREE_TOP], gone * c.Hkv);
    c.len[ls] = base + cnt;
    if (c.hist_w) {   // decode queries that saw pairs of the tree leave the record (see k_append_chunk)
      const int cnt0 = c.hist_cnt[ls];
      int q = cnt0;
      while (q > 0 && q > cnt0 - c.hist_w && c.hist_n[(size_t)ls * c.hist_w + (q - 1) % c.hist_w] > base) --q;
      c.hist_cnt[ls] = (q < cnt0 && cnt0 > c.hist_w) ? 0 : q;
    }
  }
  __syncthreads();
  for (int i = tid; i < gone * c.Hkv; i += blockDim.x) {
    const int h = i / gone;
    c.free_stack[s_push + i] = __ldcg(c.pt + (size_t)seg_of(c, layer, seq, h) * c.max_pages + kept + i - h * gone);
  }
}

// ---------------------------------------------------------------- read-out
// The last lens[s] pairs of every sequence, packed: the inverse of k_append_chunk.  A warp per page and head, with two page buffers in
// shared memory: a page is copied in (one bulk copy) while the rows of the one before it go out.  blk: the first of a sequence's pages in
// the list of all (a page more than its pairs fill: they may begin inside one).
// Bound: bytes (read and written).  32768 pairs of 8 heads (160 MB read, as many written) 59.5 us = 5.4 TB/s, 0.94 of a library copy of the same
// size (55.8); a warp per pair took 95, a warp per page with eight rows in registers 70.
struct ExportBlocks {
  int blk[kMaxBatch + 1];
};
constexpr int kExportMaxWarps = 16;
__global__ void __launch_bounds__(kExportMaxWarps * 32) k_export_chunk(Ctx c, int layer, const __grid_constant__ ChunkLens lens,
                                                                       const __grid_constant__ ExportBlocks b, uint8_t *k, uint8_t *v,
                                                                       float *feat, int32_t *pos) {
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ uint64_t bars[kExportMaxWarps][2];
  __shared__ int s_first[kMaxBatch];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, nw = blockDim.x / 32, nch = c.D / 8;
  if (lane == 0) {
    mbar_init(smem_u32(&bars[warp][0]), 1);
    mbar_init(smem_u32(&bars[warp][1]), 1);
    fence_barrier_init();
  }
  griddep_wait();
  griddep_launch();
  for (int s = threadIdx.x; s < c.batch; s += blockDim.x) {
    const int T = lens.tok[s + 1] - lens.tok[s], first = __ldcg(c.len + layer * c.batch + s) - T;
    s_first[s] = first;
    if (first < 0 && blockIdx.x == 0) set_status(c, kDevBadIndex);
  }
  __syncthreads();
  const long long tasks = (long long)b.blk[c.batch] * c.Hkv, step = (long long)gridDim.x * nw;
  const uint32_t bytes = (uint32_t)(feat || pos ? c.page_bytes : 64 * c.D);
  struct Task { int r0, r1, page; size_t at0; };
  auto task = [&](long long t) {
    Task x{0, 0, 0, 0};
    if (t >= tasks) return x;
    const int block = (int)(t / c.Hkv), h = (int)(t - (long long)block * c.Hkv);
    int lo = 0, hi = c.batch;   // the block's sequence: the last one that starts at or before it
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (b.blk[mid] <= block) lo = mid; else hi = mid;
    }
    const int first = s_first[lo], n = first + lens.tok[lo + 1] - lens.tok[lo];
    if (first < 0) return x;
    const int pg = first / kPage + block - b.blk[lo];
    x.r0 = max(first - pg * kPage, 0);
    x.r1 = min(n - pg * kPage, kPage);
    if (x.r0 >= x.r1) return x;
    x.page = __ldcg(c.pt + (size_t)seg_of(c, layer, lo, h) * c.max_pages + pg);
    x.at0 = (size_t)(lens.tok[lo] + pg * kPage - first) * c.Hkv + h;   // row of the page's pair 0, if that is one
    return x;
  };
  uint32_t turn = 0;   // pages copied so far: buffer and parity follow
  uint8_t *buf = smem + (size_t)warp * 2 * c.page_bytes;
  auto copy = [&](const Task &x, uint32_t i) {
    if (x.r0 >= x.r1 || lane != 0) return;
    const uint32_t bar = smem_u32(&bars[warp][i & 1]);
    mbar_arrive_expect_tx(bar, bytes);
    bulk_g2s(smem_u32(buf + (i & 1) * c.page_bytes), c.pool + (size_t)x.page * c.page_bytes, bytes, bar);
  };
  const int half = c.F / 2, inv = 65536 / half + 1;   // (a row's features in pairs; i / half for i < 384)
  long long t = (long long)warp * gridDim.x + blockIdx.x;
  Task x = task(t);
  copy(x, turn);
  while (t < tasks) {
    const Task nx = task(t + step);
    const bool any = x.r0 < x.r1;
    copy(nx, turn + (any ? 1 : 0));
    if (any) {
      if (!__all_sync(0xffffffffu, mbar_wait(smem_u32(&bars[warp][turn & 1]), (turn >> 1) & 1))) {
        set_status(c, kDevWaitTimeout);
        // (no copy may be in flight at the exit: once more for this one, and for the next)
        mbar_wait(smem_u32(&bars[warp][turn & 1]), (turn >> 1) & 1);
        if (nx.r0 < nx.r1) mbar_wait(smem_u32(&bars[warp][(turn + 1) & 1]), ((turn + 1) >> 1) & 1);
        break;
      }
      const uint8_t *page = buf + (turn & 1) * c.page_bytes;
      uint8_t *to = lane < nch ? k : v;
      if (lane < 2 * nch && to)
#pragma unroll 8
        for (int r = x.r0; r < x.r1; ++r)
          __stcs(reinterpret_cast<uint4 *>(to + (x.at0 + (size_t)r * c.Hkv) * c.D * 2 + (lane % nch) * 16),
                 *reinterpret_cast<const uint4 *>(page + (lane < nch ? 0 : c.off_v) + kv_chunk_off(r, lane % nch, c.D)));
      if (feat)
        for (int i = lane; i < (x.r1 - x.r0) * half; i += 32) {
          const int rr = (i * inv) >> 16, r = x.r0 + rr, f = (i - rr * half) * 2;
          const float *row = meta_row(c, page, r) + f;
          __stcs(reinterpret_cast<float2 *>(feat + (x.at0 + (size_t)r * c.Hkv) * c.F + f), make_float2(row[0], row[1]));
        }
      if (pos && x.r0 + lane < x.r1) pos[x.at0 + (size_t)(x.r0 + lane) * c.Hkv] = reinterpret_cast<const int32_t *>(meta_row(c, page, x.r0 + lane))[c.F];
      __syncwarp();   // (the buffer's next copy comes after these reads)
      ++turn;
    }
    x = nx;
    t += step;
  }
}

}  // namespace fkv
