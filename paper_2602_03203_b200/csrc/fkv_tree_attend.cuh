// Kernel 10b: small draft trees, stored and attended in ONE launch - at most 128 query rows per KV head (nodes x g), no window:
//     out_j = sum_i softmax_i(scale <q_j, k_i>) v_i  over the pairs ahead of the tree, j's ancestors and j itself.
// Bound: bytes, 4 D per pair and KV head, once for all rows; for short caches the latency of one launch and its chain of reads.
// k_append_chunk and k_chunk_attend compute the same in three dependent launches made for many rows; a step of one sequence over
// 8192 pairs waits 20 us for them and 5 for its bytes.
//
// Shape: grid (S, sequences x KV heads); the S CTAs of a segment are one cluster, each with a run of its pages.
//   warp 8      copies pages (one bulk copy each: K and V rows as they lie) into a ring;
//   warps 0-7   RW of them share two pages, 16 query rows each; 8 / RW such pairs are worked on at a time.  S^T = K Q^T with the pairs on
//               the M axis (16 of a page, mma m16n8k16 with two column tiles), so that P^T needs only a transpose in registers to
//               become the B operand of O^T = V^T P^T.  Softmax in fp32; P is rounded to bf16 (as V is: half a step, 2^-8, off);
//   warp 9      the store's page arithmetic (as k_append_chunk: prefix sums over the sequences) and the lengths.
// The CTA that has a page of the tree stores the tree's pairs of that page (the page's rows come from L2 by the same bulk copy
// after that, while earlier pages are being worked on).  Partial results meet through distributed shared memory: CTA r of a
// cluster owns rows r, r + S, ..., receives them from all and writes them.
// mma.sync, not tcgen05: with 16 - 128 rows the products take less time than the bytes, and a chain of a page (copy, scores,
// softmax, product) without tensor memory is the shorter one; from 128 rows on the tensor core's kernel is faster.
#pragma once
#include "fkv_dev.cuh"
#include "fkv_attend.cuh"
#include "fkv_chunk.cuh"
#include "fkv_features.cuh"

namespace fkv {

constexpr int kTaWarps = 8, kTaThreads = (kTaWarps + 2) * 32;
constexpr int kTaRows = 128;          // most query rows of a KV head
constexpr int kTaMaxCluster = 16;

struct TreeArgs {
  int layer, append;
  float scale_log2;
  const __nv_bfloat16 *q;
  __nv_bfloat16 *out;
  float *lse;
  const uint32_t *masks;
  const uint8_t *k, *v;
  const int32_t *pos;
  ChunkLens lens;
  ChunkKeep keep;
};

template <int D, int RW>
struct TaSmem {
  static constexpr int kSlots = D == 128 ? 16 : 32, kPageKv = 4 * D * kPage, kGroups = kTaWarps / RW, kR = RW * 16;
  static_assert(kSlots % (2 * kGroups) == 0 && kSlots > 2 * kGroups, "a slot belongs to one group of warps: its barriers carry one parity bit");
  static constexpr size_t kRing = (size_t)kSlots * kPageKv;
  static constexpr int kRow = D + 4;                                       // a row of a partial result: O, m, l
  static_assert((size_t)kTaRows * kRow * 4 <= kRing, "the warps' results meet where the ring was");
  static constexpr size_t kOffRecv = kRing;                                // [row / S][S][kRow]: at most S - 1 rows over
  static constexpr size_t kOffMask = kOffRecv + (size_t)(kR + kTaMaxCluster) * kRow * 4;
  static constexpr size_t kOffBars = kOffMask + (size_t)kTaRows * kTreeWords * 4;
  static constexpr size_t bytes() { return kOffBars + (2 * kSlots + 2) * 8; }
};

// Page arithmetic of a store, by one warp: what every sequence keeps, takes and returns (s_*: per sequence).
struct TreeStore {
  int keep[kMaxBatch], old[kMaxBatch], pop[kMaxBatch], push[kMaxBatch];
  int pops, pushes, top, exhausted, last_pos;
};

template <int D, int RW>
__global__ void __launch_bounds__(kTaThreads, 1) k_tree_attend(Ctx c, const __grid_constant__ TreeArgs a) {
  using SM = TaSmem<D, RW>;
  constexpr int SLOTS = SM::kSlots, KG = SM::kGroups, PAGE_KV = SM::kPageKv, KSQ = D / 16, MT = D / 16, ROW = SM::kRow;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ TreeStore ts;
  float *recv = reinterpret_cast<float *>(smem + SM::kOffRecv);
  uint32_t *s_mask = reinterpret_cast<uint32_t *>(smem + SM::kOffMask);
  uint64_t *full = reinterpret_cast<uint64_t *>(smem + SM::kOffBars), *empty = full + SLOTS, *stored = empty + SLOTS;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, tid = threadIdx.x;
  const int S = gridDim.x, rank = blockIdx.x, seq = blockIdx.y / c.Hkv, head = blockIdx.y % c.Hkv, G = c.G;
  if (warp == kTaWarps && lane == 0) {
    for (int s = 0; s < SLOTS; ++s) {
      mbar_init(smem_u32(&full[s]), 1);
      mbar_init(smem_u32(&empty[s]), RW);
    }
    mbar_init(smem_u32(stored), kTaWarps);
    fence_barrier_init();
  }
  griddep_wait();
  griddep_launch();
  if (S > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");   // "I am running" (waited for ahead of the exchange)
  const int row0 = a.lens.tok[seq], T = a.lens.tok[seq + 1] - row0, rows = T * G;
  const int ls = a.layer * c.batch + seq, seg = ls * c.Hkv + head;
  int *ptrow = c.pt + (size_t)seg * c.max_pages;
  const int n_old = __ldcg(c.len + ls);
  const int kp = a.append ? (a.keep.use ? a.keep.keep[seq] : n_old) : n_old - T;   // pairs ahead of the tree
  const bool bad = kp < 0 || kp > n_old || kp + T > c.cap;
  const bool active = T > 0 && !bad;
  const int n = kp + T, np_all = (n + kPage - 1) / kPage, tp = kp / kPage;   // tp: the first page with a pair of the tree
  const int pps = (np_all + S - 1) / S, pg0 = rank * pps, pg1 = min(np_all, pg0 + pps);
  const bool tail = active && pg1 > pg0 && pg1 > tp;   // this CTA has pages of the tree
  __syncthreads();   // (barriers are set up, and every thread has read the length)

  int npg = active ? max(0, pg1 - pg0) : 0;
  float o[MT][2][4];
  float m_run[2][2], l_run[2][2];
  const int gid = lane >> 2, tig = lane & 3, rw = warp % RW, kg = warp / RW;
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    m_run[t][0] = m_run[t][1] = -INFINITY;
    l_run[t][0] = l_run[t][1] = 0.f;
#pragma unroll
    for (int i = 0; i < MT; ++i) o[i][t][0] = o[i][t][1] = o[i][t][2] = o[i][t][3] = 0.f;
  }
  auto pages_kept = [&](int q) { return (ts.keep[q] + a.lens.tok[q + 1] - a.lens.tok[q] + kPage - 1) / kPage; };
  auto pages_old = [&](int q) { return (ts.old[q] + kPage - 1) / kPage; };
  auto returned = [&](int q, int i) {   // the i-th page that sequence q returns
    const int kept = pages_kept(q), cnt = pages_old(q) - kept, h = i / cnt;
    return __ldcg(c.pt + (size_t)seg_of(c, a.layer, q, h) * c.max_pages + kept + i - h * cnt);
  };

  if (warp == kTaWarps + 1) {
    // ---------------- the store's arithmetic, masks, lengths ----------------
    auto arithmetic = [&]() {   // a lane: eight sequences in a row
      int kpq[8], pop[8], push[8], pops = 0, pushes = 0;
      const int top = __ldcg(c.ctrl + CTRL_FREE_TOP);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int s = lane * 8 + i;
        kpq[i] = -1; pop[i] = push[i] = 0;
        if (s < c.batch) {
          const int nq = __ldcg(c.len + a.layer * c.batch + s), t = a.lens.tok[s + 1] - a.lens.tok[s];
          kpq[i] = a.keep.use ? a.keep.keep[s] : nq;
          if (kpq[i] > nq || kpq[i] + t > c.cap) kpq[i] = -1;
          ts.keep[s] = kpq[i];
          ts.old[s] = nq;
          if (kpq[i] >= 0) {
            const int delta = (kpq[i] + t + kPage - 1) / kPage - (nq + kPage - 1) / kPage;
            pop[i] = delta > 0 ? delta * c.Hkv : 0;
            push[i] = delta < 0 ? -delta * c.Hkv : 0;
          }
        }
        pops += pop[i];
        pushes += push[i];
      }
      int ip = pops, iq = pushes;
#pragma unroll
      for (int o2 = 1; o2 < 32; o2 <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, ip, o2), y = __shfl_up_sync(0xffffffffu, iq, o2);
        if (lane >= o2) { ip += x; iq += y; }
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
    };
    if (tail) {
      if (a.append) {
        int last = -1;
        if (!a.pos && kp > 0) {
          const uint8_t *prev = c.pool + (size_t)__ldcg(ptrow + (kp - 1) / kPage) * c.page_bytes;
          last = __ldcg(reinterpret_cast<const int32_t *>(meta_row(c, prev, (kp - 1) % kPage)) + c.F);
        }
        if (lane == 0) ts.last_pos = last;
        arithmetic();
      } else if (lane == 0) {
        ts.exhausted = 0;
      }
      for (int i = lane; i < T * kTreeWords; i += 32) s_mask[i] = __ldcg(a.masks + (size_t)row0 * kTreeWords + i);
      asm volatile("bar.sync 1, %0;" ::"n"((kTaWarps + 1) * 32) : "memory");
    }
    if (a.append) {
      if (tail && !mbar_wait(smem_u32(stored), 0)) set_status(c, kDevWaitTimeout);
      int last = 0;
      if (lane == 0) {
        __threadfence();   // this CTA's pages and page tables come before its ticket
        last = atomicAdd(&c.ctrl[CTRL_CHUNK_TICKET], 1) == (int)(gridDim.x * gridDim.y) - 1;
      }
      if (__shfl_sync(0xffffffffu, last, 0)) {
        // Every CTA has read the lengths and stored its pairs: pages return, the stack's top and the lengths move (k_append_chunk
        // has the same end, and its comments).
        __threadfence();
        if (!tail) arithmetic();
        if (lane == 0) {
          c.ctrl[CTRL_CHUNK_TICKET] = 0;
          if (ts.exhausted) set_status(c, kDevPoolExhausted);
        }
        const int pops = ts.pops, pushes = ts.pushes, top = ts.top;
        for (int q = 0; q < c.batch; ++q) {
          const int nq = ts.old[q], t = a.lens.tok[q + 1] - a.lens.tok[q];
          if (ts.keep[q] < 0) {
            if (lane == 0) set_status(c, a.keep.use && a.keep.keep[q] > nq ? kDevBadIndex : kDevCapacity);
            continue;
          }
          if (ts.exhausted) continue;
          const int cnt = (pages_old(q) - pages_kept(q)) * c.Hkv;
          for (int i = lane; i < cnt; i += 32) {
            const int at = top - pops + ts.push[q] + i;
            if (at >= 0) c.free_stack[at] = returned(q, i);
          }
          (void)t;
        }
        __syncwarp();
        if (!ts.exhausted) {
          if (lane == 0) c.ctrl[CTRL_FREE_TOP] = top - pops + pushes;
          for (int s = lane; s < c.batch; s += 32) {
            const int kq = ts.keep[s], nq = ts.old[s], lq = a.layer * c.batch + s;
            if (kq < 0) continue;
            c.len[lq] = kq + a.lens.tok[s + 1] - a.lens.tok[s];
            if (c.hist_w && kq < nq) {
              const int cnt0 = c.hist_cnt[lq];
              int cnt = cnt0;
              while (cnt > 0 && cnt > cnt0 - c.hist_w && c.hist_n[(size_t)lq * c.hist_w + (cnt - 1) % c.hist_w] > kq) --cnt;
              c.hist_cnt[lq] = (cnt < cnt0 && cnt0 > c.hist_w) ? 0 : cnt;
            }
          }
        }
      }
    } else if (T > 0 && bad && rank == 0 && head == 0 && lane == 0) {
      set_status(c, kDevBadIndex);
    }
  } else if (warp == kTaWarps) {
    // ---------------- page copies: those ahead of the tree at once, the tree's when its pairs are stored ----------------
    const uint64_t policy = l2_policy_evict_first();
    auto issue = [&](int i, int pid) {
      const uint32_t bar = smem_u32(&full[i % SLOTS]);
      mbar_arrive_expect_tx(bar, PAGE_KV);
      bulk_g2s_hint(smem_u32(smem + (size_t)(i % SLOTS) * PAGE_KV), c.pool + (size_t)pid * c.page_bytes, PAGE_KV, bar, policy);
    };
    bool ok = true;
    auto copy = [&](int i0, int i1) {
      for (int b = i0; b < i1 && ok; b += 32) {
        const int id = b + lane < i1 ? __ldcg(ptrow + pg0 + b + lane) : 0;
        int j = 0;
        if (b < SLOTS) {   // an empty ring: no wait
          j = min(SLOTS, i1) - b;
          if (lane < j) issue(b + lane, id);
        }
        for (; j < min(32, i1 - b); ++j) {
          const int i = b + j, pid = __shfl_sync(0xffffffffu, id, j);
          if (!__all_sync(0xffffffffu, mbar_wait(smem_u32(&empty[i % SLOTS]), ((i / SLOTS) & 1) ^ 1))) {
            if (lane == 0) set_status(c, kDevWaitTimeout);
            ok = false;
            break;
          }
          if (lane == 0) issue(i, pid);
        }
      }
    };
    const int ahead = tail && a.append ? max(0, min(npg, tp - pg0)) : npg;
    copy(0, ahead);
    if (ahead < npg && ok) {
      if (!mbar_wait(smem_u32(stored), 0)) { set_status(c, kDevWaitTimeout); ok = false; }
      __syncwarp();
      if (ts.exhausted) npg = max(ahead, min(npg, (kp + kPage - 1) / kPage - pg0));   // (nothing was stored)
      copy(ahead, npg);
    }
  } else if (active) {
    // ---------------- query rows 16 rw .. of the pages kg, kg + KG, ... ----------------
    // Q^T as B fragments: column gid of column tile t is row 16 rw + 8 t + gid = (node, query head) of the group.
    uint32_t qb[KSQ][2][2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int r = rw * 16 + t * 8 + gid, node = r / G;
      const uint32_t *qr = reinterpret_cast<const uint32_t *>(a.q + (((size_t)(row0 + node) * c.Hkv + head) * G + r - node * G) * D);
#pragma unroll
      for (int ks = 0; ks < KSQ; ++ks) {
        qb[ks][t][0] = r < rows ? __ldcg(qr + ks * 8 + tig) : 0u;
        qb[ks][t][1] = r < rows ? __ldcg(qr + ks * 8 + 4 + tig) : 0u;
      }
    }
    int lim = n;   // slots behind this are not there
    if (tail) {
      asm volatile("bar.sync 1, %0;" ::"n"((kTaWarps + 1) * 32) : "memory");   // the arithmetic and the masks
      if (ts.exhausted) {
        lim = kp;
        npg = max(0, min(npg, (kp + kPage - 1) / kPage - pg0));
      } else if (a.append) {
        // The tree's pairs on this CTA's pages, four at a time.
        const int np_old = (n_old + kPage - 1) / kPage, grow = np_all - np_old, nch = D / 8;
        const int j0 = max(pg0 * kPage, kp) - kp, j1 = min(pg1 * kPage, n) - kp;
        for (int jb = j0 + warp; jb < j1; jb += kTaWarps * 4) {
          uint4 x[4];
          int pid[4], at[4];
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            const int j = jb + u * kTaWarps;
            if (j >= j1) continue;
            const size_t src = ((size_t)(row0 + j) * c.Hkv + head) * D * 2;
            if (lane < 2 * nch) x[u] = __ldcg(reinterpret_cast<const uint4 *>((lane < nch ? a.k : a.v) + src + (lane % nch) * 16));
            const int pg = (kp + j) / kPage;
            if (pg < np_old) {
              pid[u] = __ldcg(ptrow + pg);
            } else {
              const int y = ts.pop[seq] + head * grow + pg - np_old;   // the y-th page that the call takes
              if (y < ts.top) {
                pid[u] = __ldcg(c.free_stack + ts.top - 1 - y);
              } else {
                int q = 0, end = c.batch;
                while (end - q > 1) {
                  const int mid = (q + end) >> 1;
                  if (ts.push[mid] <= y - ts.top) q = mid; else end = mid;
                }
                pid[u] = returned(q, y - ts.top - ts.push[q]);
              }
            }
            if (a.pos) {
              at[u] = __ldcg(a.pos + row0 + j);
            } else {   // one behind the parent's: the last pair's and the number of nodes that this one sees
              at[u] = ts.last_pos + (int)__reduce_add_sync(0xffffffffu, lane < kTreeWords ? __popc(s_mask[j * kTreeWords + lane]) : 0);
            }
          }
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            const int j = jb + u * kTaWarps;
            if (j >= j1) continue;
            const int slot = kp + j, r = slot % kPage;
            uint8_t *page = c.pool + (size_t)pid[u] * c.page_bytes;
            if (lane < 2 * nch) *reinterpret_cast<uint4 *>(page + (lane < nch ? 0 : c.off_v) + kv_chunk_off(r, lane % nch, D)) = x[u];
            float *meta = meta_row(c, page, r);
            for (int f = lane; f < c.F; f += 32) meta[f] = 0.f;
            if (lane == 0) {
              reinterpret_cast<int32_t *>(meta)[c.F] = at[u];
              if (slot / kPage >= np_old && (r == 0 || j == 0)) ptrow[slot / kPage] = pid[u];
            }
          }
        }
        asm volatile("fence.proxy.async;" ::: "memory");   // the copies of these pages come after the stores
      }
      if (a.append) {
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(stored));
      }
    }
    const int krow = ((lane >> 3) & 1) * 8 + (lane & 7), khi = lane >> 4;
    const int vrow = (lane >> 4) * 8 + (lane & 7), vhi = (lane >> 3) & 1;
    const uint32_t rt_zero = gridDim.z - 1;   // 0 at run time, unknown at compile time
    // Two pages at a time: a page's chain (scores, softmax, product) is latency, and two of them fill each other's gaps.
    for (int i = kg * 2; i < npg; i += KG * 2) {
      const bool two = i + 1 < npg;
      const int sl[2] = {i % SLOTS, (i + 1) % SLOTS};
      bool ok = mbar_wait(smem_u32(&full[sl[0]]), (i / SLOTS) & 1);
      if (two) ok = ok && mbar_wait(smem_u32(&full[sl[1]]), ((i + 1) / SLOTS) & 1);
      if (!ok) { set_status(c, kDevWaitTimeout); break; }
      const int slot0 = (pg0 + i) * kPage;
      // (without a second page the first one's rows stand in for it, and none of its pairs is seen)
      const uint32_t kb[2] = {smem_u32(smem + (size_t)sl[0] * PAGE_KV), smem_u32(smem + (size_t)sl[two ? 1 : 0] * PAGE_KV)};
      float s[2][2][4] = {};
#pragma unroll
      for (int ks = 0; ks < KSQ; ++ks) {
        uint32_t x[2][4];
#pragma unroll
        for (int b = 0; b < 2; ++b) ldsm_x4(x[b], kb[b] + kv_chunk_off(krow, ks * 2 + khi, D));
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int t = 0; t < 2; ++t) mma_bf16(s[b][t], x[b][0], x[b][1], x[b][2], x[b][3], qb[ks][t][0], qb[ks][t][1]);
      }
      // This lane: pairs gid and gid + 8 of each page, rows 2 tig and 2 tig + 1 of each column tile.
      const int seen_end = two ? lim : min(lim, slot0 + kPage);
      if (slot0 + 2 * kPage > min(kp, seen_end)) {   // pairs of the tree, or none
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int r = rw * 16 + t * 8 + 2 * tig + e, node = r / G;
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
              for (int u = 0; u < 2; ++u) {
                const int slot = slot0 + b * kPage + gid + u * 8, j = slot - kp;
                const bool sees = slot < seen_end && r < rows && (j < 0 || (j <= node && ((s_mask[node * kTreeWords + (j >> 5)] >> (j & 31)) & 1u)));
                if (!sees) s[b][t][u * 2 + e] = -INFINITY;
              }
          }
      }
      // The reference of a row moves when a score has passed it by more than 2^24 (or there is none yet): until then P is at most
      // 2^24, which bf16 holds as exactly as 1, and nothing is rescaled.
      bool grow = false;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float top = fmaxf(fmaxf(s[0][t][e], s[0][t][2 + e]), fmaxf(s[1][t][e], s[1][t][2 + e]));
          grow = grow || top * a.scale_log2 > m_run[t][e] + kChunkGrow;
        }
      if (__any_sync(0xffffffffu, grow)) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          float f[2];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float top = fmaxf(fmaxf(s[0][t][e], s[0][t][2 + e]), fmaxf(s[1][t][e], s[1][t][2 + e])) * a.scale_log2;
#pragma unroll
            for (int sh = 4; sh < 32; sh <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, sh));
            top = fmaxf(top, m_run[t][e]);
            f[e] = top == -INFINITY ? 1.f : ex2(m_run[t][e] - top);
            m_run[t][e] = top;
            l_run[t][e] *= f[e];
          }
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) {
            o[mt][t][0] *= f[0]; o[mt][t][1] *= f[1]; o[mt][t][2] *= f[0]; o[mt][t][3] *= f[1];
          }
        }
      }
      uint32_t pb[2][2][2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const float z0 = m_run[t][0] == -INFINITY ? 0.f : m_run[t][0], z1 = m_run[t][1] == -INFINITY ? 0.f : m_run[t][1];   // (a row that has seen nothing)
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          const float e0 = ex2(fmaf(s[b][t][0], a.scale_log2, -z0)), e1 = ex2(fmaf(s[b][t][1], a.scale_log2, -z1));
          const float e2 = ex2(fmaf(s[b][t][2], a.scale_log2, -z0)), e3 = ex2(fmaf(s[b][t][3], a.scale_log2, -z1));
          l_run[t][0] += e0 + e2;
          l_run[t][1] += e1 + e3;
          pb[b][t][0] = movmatrix_trans(pack_bf16(e0, e1));
          pb[b][t][1] = movmatrix_trans(pack_bf16(e2, e3));
        }
      }
      // V rows behind the last pair are left out of the product (zero times an infinity is not zero): pairs 2 tig, 2 tig + 1 and
      // those eight further on.
      if (slot0 + 2 * kPage <= seen_end) {
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          uint32_t x[2][4];
#pragma unroll
          for (int b = 0; b < 2; ++b) ldsm_x4_trans(x[b], kb[b] + 2 * D + kv_chunk_off(vrow, mt * 2 + vhi, D));
#pragma unroll
          for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int t = 0; t < 2; ++t) mma_bf16(o[mt][t], x[b][0], x[b][1], x[b][2], x[b][3], pb[b][t][0], pb[b][t][1]);
        }
      } else {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          const int left = seen_end - slot0 - b * kPage;
          auto both = [&](int p) { return (p < left ? 0xffffu : 0u) | (p + 1 < left ? 0xffff0000u : 0u); };
          const uint32_t keep_lo = both(2 * tig), keep_hi = both(2 * tig + 8);
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) {
            uint32_t x[4];
            ldsm_x4_trans(x, kb[b] + 2 * D + kv_chunk_off(vrow, mt * 2 + vhi, D));
            x[0] &= keep_lo; x[1] &= keep_lo; x[2] &= keep_hi; x[3] &= keep_hi;
#pragma unroll
            for (int t = 0; t < 2; ++t) mma_bf16(o[mt][t], x[0], x[1], x[2], x[3], pb[b][t][0], pb[b][t][1]);
          }
        }
      }
      // Every read of the pages has to be complete before the arrivals are seen: their addresses depend on the products' results.
      uint32_t done = 0;
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) done |= __float_as_uint(o[mt][0][0]) | __float_as_uint(o[mt][1][0]);
      __syncwarp();
      if (lane < (two ? 2 : 1)) mbar_arrive(smem_u32(&empty[sl[lane & 1]]) + (done & rt_zero));
    }
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int sh = 4; sh < 32; sh <<= 1) l_run[t][e] += __shfl_xor_sync(0xffffffffu, l_run[t][e], sh);
  }
  __syncthreads();   // all copies have landed and been used: the ring's memory is free
  if (!active) {     // (of the whole cluster alike)
    if (S > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    return;
  }
  // ---- the groups' results: [group][row][O, m, l] ----
  float *mg = reinterpret_cast<float *>(smem);
  if (warp < kTaWarps) {
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float *r = mg + (size_t)(kg * SM::kR + rw * 16 + t * 8 + 2 * tig + e) * ROW;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          r[mt * 16 + gid] = o[mt][t][e];
          r[mt * 16 + 8 + gid] = o[mt][t][2 + e];
        }
        // (a row whose scores are all NaN has found no maximum, but must not count as one that saw nothing)
        if (gid == 0) { r[D] = l_run[t][e] != l_run[t][e] ? 0.f : m_run[t][e]; r[D + 1] = l_run[t][e]; }
      }
  }
  __syncthreads();
  if (S > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");   // every CTA of the cluster runs
  // ---- a warp per row: the groups' sum goes to the row's owner (or is the result) ----
  auto finish = [&](int r, float4 acc, float M, float L) {   // four channels per lane
    const float inv = L == 0.f ? 0.f : 1.f / L;              // a row that sees nothing gives zeros
    const size_t orow = ((size_t)(row0 + r / G) * c.Hkv + head) * G + r % G;
    if (lane * 4 < D) *reinterpret_cast<uint2 *>(a.out + orow * D + lane * 4) = make_uint2(pack_bf16(acc.x * inv, acc.y * inv), pack_bf16(acc.z * inv, acc.w * inv));
    if (a.lse && lane == 0) a.lse[orow] = L == 0.f ? -INFINITY : (M + log2f(L)) * 0.6931471805599453f;
  };
  // Joins `parts` results of a row, `step` floats apart.
  auto join = [&](const float *p, int parts, int step, float4 &acc, float &M, float &L) {
    M = -INFINITY;
    L = 0.f;
    acc = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int g = 0; g < parts; ++g) M = fmaxf(M, p[g * step + D]);
    for (int g = 0; g < parts; ++g) {
      const float mgr = p[g * step + D], f = mgr == -INFINITY ? 0.f : ex2(mgr - M);
      L = f == 0.f ? L : fmaf(f, p[g * step + D + 1], L);
      if (lane * 4 < D && f != 0.f) {
        const float4 x = *reinterpret_cast<const float4 *>(p + g * step + lane * 4);
        acc.x = fmaf(f, x.x, acc.x); acc.y = fmaf(f, x.y, acc.y); acc.z = fmaf(f, x.z, acc.z); acc.w = fmaf(f, x.w, acc.w);
      }
    }
  };
  for (int r = warp; r < rows; r += kTaWarps + 2) {
    float4 acc;
    float M, L;
    join(mg + (size_t)r * ROW, KG, SM::kR * ROW, acc, M, L);
    if (S == 1) {
      finish(r, acc, M, L);
    } else {
      const int owner = r % S;
      const uint32_t to = dsmem_addr(smem_u32(recv + (size_t)(r / S * S + rank) * ROW), owner);
      if (lane * 4 < D) dsmem_st4(to + lane * 16, acc);
      if (lane == 0) dsmem_st2(to + D * 4, M, L);
    }
  }
  if (S == 1) return;
  cluster_sync_all();
  for (int r = rank + warp * S; r < rows; r += (kTaWarps + 2) * S) {
    float4 acc;
    float M, L;
    join(recv + (size_t)(r / S * S) * ROW, S, ROW, acc, M, L);
    finish(r, acc, M, L);
  }
}

}  // namespace fkv
