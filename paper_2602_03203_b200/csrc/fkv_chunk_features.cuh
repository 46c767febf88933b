// Kernel 9: the attention features of Appendix B.1 from the queries of a chunk (a prompt, or a piece of one), with their
// log-sum-exp at hand:
//     P_ji = e^{scale <q_j, k_i> - lse_j} on the pairs i that query j sees, 0 elsewhere;
// per query head and pair the means of P over the chunk's last 8 / 16 / 32 queries and over the whole chunk, and the two
// running sums moved on by the latter, as k_features does for decode queries.
//
// Bound: 2 D flops and one exp2 per (query head, seen pair).  The special-function pipe takes 128 cycles x 8 for a block of
// 128 pairs x 128 queries and the tensor core 512, so the exponentials are what the kernel is built around.
//
// S^T = K Q^T: pairs on the M axis, so a thread owns a pair and adds up along its own row of tensor memory; nothing is
// reduced across threads.  A CTA takes two tiles of 128 pairs at a time and streams the queries of one head past them,
// 128 at a time, newest first (the windows are then prefixes of the walk): a block of queries is read from L2 once for
// 256 pairs.  Persistent CTAs over equal ranges of a line of (pair of tiles, query head), weighed by their query blocks.
//   warp 0      tensor copies: K rows page by page, blocks of queries; the queries' log-sum-exp in units of log2;
//   warp 1      one lane issues tcgen05.mma into one of two accumulators per tile;
//   warp 2      walks the line and looks the positions up;
//   warps 4-11  two warpgroups, one per tile: exp2, sums, and the pair's meta row at the end.
// Every wait is bounded; tensor memory is freed at the common exit.
#pragma once
#include "fkv_chunk.cuh"

namespace fkv {

constexpr int kCfThreads = 384;
constexpr int kCfPairs = 256, kCfQueries = 128;   // pairs of a unit (two tiles), queries of a block
constexpr int kCfItems = 2;

struct ChunkFeatArgs {
  int layer, window, sinks;
  float scale_log2;
  const float *lse;    // [tokens][Hkv * g]
  ChunkLens lens;
};

// Two tiles of one segment and the query heads [j0, j1) of its group.
struct CfItem {
  int kind;            // 0: no more
  int seg, head, pg0;  // first page of the tiles
  int n, T, base;      // pairs, queries, slot of the first query's own pair
  int j0, j1;
  int m0, m1;          // query blocks, counted from the newest: [m0, m1)
  int row0;            // packed index of the chunk's first token
  int p0;              // position of the first query
  int steady;          // the chunk's positions have no gap
  int pad[2];
};

template <int D>
struct CfSmem {
  static constexpr int kQ = D == 128 ? 2 : 4, kL = kQ + 2;   // blocks of queries in flight; their log-sum-exp (see the copies)
  static constexpr size_t kTile = (size_t)(D / 64) * 128 * 128;
  static constexpr size_t kOffQ = 2 * 2 * kTile;  // two pairs of K tiles
  static constexpr size_t kOffL = kOffQ + kQ * kTile;
  static constexpr size_t kOffItems = kOffL + (size_t)kL * kCfQueries * 4;
  static constexpr size_t kOffLen = kOffItems + kCfItems * sizeof(CfItem);
  static constexpr size_t kOffBlk = kOffLen + kMaxBatch * 4;
  static constexpr size_t kOffBars = (kOffBlk + (kMaxBatch + 1) * 4 + 15) & ~(size_t)15;
  static constexpr size_t kNeed = 1024 + kOffBars + 512;
  static constexpr size_t bytes() { return kNeed > 120 * 1024 ? kNeed : 120 * 1024; }   // one CTA per SM (tensor memory)
};

// Query blocks [m0, m1) that may see a pair of the slots [i0, i1), from the lengths alone.
struct CfRange { int m0, m1; };
__device__ __forceinline__ CfRange cf_blocks(int T, int jlo, int jhi) {   // tokens [jlo, jhi)
  CfRange r;
  if (jlo >= jhi) { r.m0 = r.m1 = 0; return r; }
  r.m0 = (T - jhi) / kCfQueries;
  r.m1 = (T - jlo + kCfQueries - 1) / kCfQueries;
  return r;
}
__device__ __forceinline__ CfRange cf_range(int n, int T, int i0, int i1, int W, int S) {
  const int base = n - T, jlo = max(0, i0 - base);
  const int jhi = (!W || i0 < S) ? T : (int)min((long long)T, (long long)i1 - 1 - base + W);
  return cf_blocks(T, jlo, jhi);
}

// 32 queries of one pair, newest first; NEWEST: the chunk's last 32.
template <bool NEWEST, bool MASKED>
__device__ __forceinline__ void cf_chunk(const uint32_t (&r)[32], const float *mp, float scale_log2, int lo, int hi, float &run,
                                         float &w8, float &w16) {
#pragma unroll
  for (int i = 28; i >= 0; i -= 4) {
    const float4 M4 = *reinterpret_cast<const float4 *>(mp + i);
    float p3 = ex2(fmaf(__uint_as_float(r[i + 3]), scale_log2, -M4.w)), p2 = ex2(fmaf(__uint_as_float(r[i + 2]), scale_log2, -M4.z));
    float p1 = ex2(fmaf(__uint_as_float(r[i + 1]), scale_log2, -M4.y)), p0 = ex2(fmaf(__uint_as_float(r[i]), scale_log2, -M4.x));
    if (MASKED) {
      p3 = i + 3 >= lo && i + 3 < hi ? p3 : 0.f; p2 = i + 2 >= lo && i + 2 < hi ? p2 : 0.f;
      p1 = i + 1 >= lo && i + 1 < hi ? p1 : 0.f; p0 = i >= lo && i < hi ? p0 : 0.f;
    }
    run += (p3 + p2) + (p1 + p0);
    if (NEWEST && i == 24) w8 = run;
    if (NEWEST && i == 16) w16 = run;
  }
}

template <int D>
__global__ void __launch_bounds__(kCfThreads, 1) k_chunk_features(Ctx c, const __grid_constant__ CUtensorMap tmkv,
                                                                  const __grid_constant__ CUtensorMap tmq,
                                                                  const __grid_constant__ ChunkFeatArgs a) {
  using SM = CfSmem<D>;
  constexpr int NQ = D / 64, QS = SM::kQ, LS = SM::kL;
  constexpr uint32_t PAGE_HALF = kPage * 128;
  extern __shared__ uint8_t smem_raw[];
  uint8_t *smem = reinterpret_cast<uint8_t *>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  uint8_t *Kt = smem, *Qt = smem + SM::kOffQ;
  float *Lt = reinterpret_cast<float *>(smem + SM::kOffL);
  CfItem *Items = reinterpret_cast<CfItem *>(smem + SM::kOffItems);
  int *Len = reinterpret_cast<int *>(smem + SM::kOffLen), *Blk = reinterpret_cast<int *>(smem + SM::kOffBlk);
  uint64_t *bars = reinterpret_cast<uint64_t *>(smem + SM::kOffBars);
  uint64_t *k_full = bars, *k_empty = k_full + 2, *q_full = k_empty + 2, *q_empty = q_full + QS, *l_full = q_empty + QS;
  uint64_t *acc_full = l_full + LS, *acc_empty = acc_full + 4;   // [tile][buffer]
  uint64_t *it_full = acc_empty + 4, *it_empty = it_full + kCfItems, *mma_done = it_empty + kCfItems;
  uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(mma_done + 1);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, G = c.G, Hq = c.Hkv * c.G;

  if (warp == 3) tmem_alloc(smem_u32(tmem_slot), 512);
  if (threadIdx.x == 0) {
    for (int s = 0; s < 2; ++s) { mbar_init(smem_u32(&k_full[s]), 1); mbar_init(smem_u32(&k_empty[s]), 1); }
    for (int s = 0; s < QS; ++s) { mbar_init(smem_u32(&q_full[s]), 1); mbar_init(smem_u32(&q_empty[s]), 1); }
    for (int s = 0; s < LS; ++s) mbar_init(smem_u32(&l_full[s]), 1);
    for (int s = 0; s < 4; ++s) { mbar_init(smem_u32(&acc_full[s]), 1); mbar_init(smem_u32(&acc_empty[s]), 4); }
    for (int s = 0; s < kCfItems; ++s) { mbar_init(smem_u32(&it_full[s]), 1); mbar_init(smem_u32(&it_empty[s]), 10); }
    mbar_init(smem_u32(mma_done), 1);
    fence_barrier_init();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  griddep_wait();
  griddep_launch();

  if (warp == 2) {
    // ---------------- the walk ----------------
    const int batch = c.batch, W = a.window, S = a.sinks;
    for (int s = lane; s < batch; s += 32) {
      const int n = __ldcg(c.len + a.layer * batch + s);
      Len[s] = n;
      if (blockIdx.x == 0 && n < a.lens.tok[s + 1] - a.lens.tok[s]) set_status(c, kDevBadIndex);
    }
    __syncwarp();
    int NB = 0;   // pairs of tiles of the sequences that take part
    for (int s0 = 0; s0 < batch; s0 += 32) {
      const int s = s0 + lane;
      const int T = s < batch ? a.lens.tok[s + 1] - a.lens.tok[s] : 0;
      const int nb = T > 0 && Len[s] >= T ? (Len[s] + kCfPairs - 1) / kCfPairs : 0;
      int inc = nb;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int t = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += t;
      }
      if (s < batch) Blk[s] = NB + inc - nb;
      NB += __shfl_sync(0xffffffffu, inc, 31);
    }
    if (lane == 0) Blk[batch] = NB;
    __syncwarp();
    struct Block { int s, n, T, i0, i1, cost; };
    auto block = [&](int f) {
      Block b;
      int lo = 0, hi = batch;
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (Blk[mid] <= f) lo = mid; else hi = mid;
      }
      b.s = lo;
      b.T = a.lens.tok[lo + 1] - a.lens.tok[lo];
      b.n = Len[lo];
      b.i0 = (f - Blk[lo]) * kCfPairs;
      b.i1 = min(b.n, b.i0 + kCfPairs);
      const CfRange r = cf_range(b.n, b.T, b.i0, b.i1, W, S);
      b.cost = r.m1 - r.m0 + 1;   // of one head: its query blocks, and about as much as one of them for what frames them
      return b;
    };
    long long P = 0;   // of one KV head
    for (int f0 = 0; f0 < NB; f0 += 32) {
      int u = f0 + lane < NB ? block(f0 + lane).cost * G : 0;
#pragma unroll
      for (int o = 16; o >= 1; o >>= 1) u += __shfl_xor_sync(0xffffffffu, u, o);
      P += u;
    }
    const long long total = P * c.Hkv;
    const long long per = (total + gridDim.x - 1) / gridDim.x;
    const long long u0 = per * blockIdx.x, u1 = min(total, u0 + per);
    long long U = 0;   // where item f of `head` begins on the line
    int head = 0, f = 0, it = 0;
    if (u0 < u1) {
      head = (int)(u0 / P);
      long long rem = u0 - head * P;
      U = head * P;
      for (int f0 = 0; f0 < NB; f0 += 32) {
        const int un = f0 + lane < NB ? block(f0 + lane).cost * G : 0;
        int inc = un;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int t = __shfl_up_sync(0xffffffffu, inc, o);
          if (lane >= o) inc += t;
        }
        const unsigned in = __ballot_sync(0xffffffffu, rem < inc);
        if (in) {
          const int l = __ffs(in) - 1;
          f = f0 + l;
          U += __shfl_sync(0xffffffffu, inc - un, l);
          break;
        }
        const int all = __shfl_sync(0xffffffffu, inc, 31);
        rem -= all;
        U += all;
      }
    }
    for (;;) {
      const int ri = it % kCfItems;
      if (!mbar_wait_warp(smem_u32(&it_empty[ri]), ((it / kCfItems) & 1) ^ 1)) { set_status(c, kDevWaitTimeout); break; }
      CfItem *x = Items + ri;
      if (u0 >= u1 || U >= u1 || head >= c.Hkv) {
        if (lane == 0) { x->kind = 0; mbar_arrive(smem_u32(&it_full[ri])); }
        break;
      }
      const Block b = block(f);
      // The heads whose stretch of the line begins in this CTA's range.
      const int j0 = U >= u0 ? 0 : (int)min((long long)G, (u0 - U + b.cost - 1) / b.cost);
      const int j1 = (int)min((long long)G, (u1 - U + b.cost - 1) / b.cost);
      if (j0 < j1) {
        const int seg = seg_of(c, a.layer, b.s, head), base = b.n - b.T;
        const int *ptrow = c.pt + (size_t)seg * c.max_pages;
        CfRange r = cf_range(b.n, b.T, b.i0, b.i1, W, S);
        int p0 = 0, steady = 1;
        if (W) {   // the blocks that the stored positions leave
          const int x_first = slot_pos(c, ptrow, b.i0), x_last = slot_pos(c, ptrow, b.i1 - 1), p_last = slot_pos(c, ptrow, b.n - 1);
          p0 = slot_pos(c, ptrow, base);
          steady = p_last - p0 == b.T - 1;
          if (x_first >= S && steady) {
            const int jhi = (int)max(0LL, min((long long)b.T, (long long)x_last + W - p0));
            r = cf_blocks(b.T, max(0, b.i0 - base), jhi);
          }
        }
        if (lane == 0) {
          x->kind = 1; x->seg = seg; x->head = head; x->pg0 = b.i0 / kPage;
          x->n = b.n; x->T = b.T; x->base = base;
          x->j0 = j0; x->j1 = j1; x->m0 = r.m0; x->m1 = r.m1;
          x->row0 = a.lens.tok[b.s]; x->p0 = p0; x->steady = steady;
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&it_full[ri]));
        ++it;
      }
      U += (long long)b.cost * G;
      if (++f == NB) { f = 0; ++head; }
    }
  } else if (warp == 0) {
    // ---------------- copies ----------------
    FeatRing kr{0, 0}, qr{0, 0};
    int it = 0, li = 0;
    uint32_t armed = 0, armed_par = 0;   // bit s: K buffer s, bit 8 + s: query stage s
    bool ok = true;
    while (ok) {
      const int ri = it % kCfItems;
      if (!mbar_wait_warp(smem_u32(&it_full[ri]), (it / kCfItems) & 1)) { set_status(c, kDevWaitTimeout); break; }
      const CfItem x = Items[ri];
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&it_empty[ri]));
      ++it;
      if (x.kind == 0) break;
      if (x.m0 >= x.m1) continue;
      {
        // Lane = (channel half, page of the two tiles).
        const int pg = lane & 15, q = lane >> 4, npages = (x.n + kPage - 1) / kPage;
        const bool on = x.pg0 + pg < npages && q < NQ;
        const int pid = on ? __ldcg(c.pt + (size_t)x.seg * c.max_pages + x.pg0 + pg) : 0;
        const int ncopies = __popc(__ballot_sync(0xffffffffu, on));
        if (!mbar_wait_warp(smem_u32(&k_empty[kr.i]), kr.ph ^ 1)) { set_status(c, kDevWaitTimeout); break; }
        if (lane == 0) mbar_arrive_expect_tx(smem_u32(&k_full[kr.i]), (uint32_t)ncopies * PAGE_HALF);
        armed |= 1u << kr.i;
        armed_par = (armed_par & ~(1u << kr.i)) | ((uint32_t)kr.ph << kr.i);
        __syncwarp();
        if (on)
          tma_page_k(smem_u32(Kt + (size_t)(kr.i * 2 + (pg >> 3)) * SM::kTile + (size_t)q * 128 * 128 + (size_t)(pg & 7) * PAGE_HALF),
                     &tmkv, q, pid, smem_u32(&k_full[kr.i]));
        kr.next(2);
      }
      for (int j = x.j0; j < x.j1 && ok; ++j)
        for (int m = x.m0; m < x.m1; ++m) {
          const int t0 = x.T - kCfQueries * (m + 1), hq = x.head * G + j;   // (t0 < 0 in the oldest block)
          float l[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int t = t0 + lane * 4 + i;
            l[i] = t >= 0 ? __ldg(a.lse + (size_t)(x.row0 + t) * Hq + hq) : 0.f;
          }
          if (!mbar_wait_warp(smem_u32(&q_empty[qr.i]), qr.ph ^ 1)) { set_status(c, kDevWaitTimeout); ok = false; break; }
          // No barrier says that the log-sum-exp slot may be overwritten; the depth does: this stage was let go by the
          // products kQ blocks back, which were issued only after the sums of the block two before those were done.
          constexpr float kLog2e = 1.4426950408889634f, kRest = 1.925963033e-8f;   // log2(e) and what fp32 leaves of it
          float4 m4;
          m4.x = fmaf(l[0], kLog2e, l[0] * kRest); m4.y = fmaf(l[1], kLog2e, l[1] * kRest);
          m4.z = fmaf(l[2], kLog2e, l[2] * kRest); m4.w = fmaf(l[3], kLog2e, l[3] * kRest);
          *reinterpret_cast<float4 *>(Lt + li * kCfQueries + lane * 4) = m4;
          __syncwarp();
          if (lane == 0) {
            mbar_arrive(smem_u32(&l_full[li]));
            const uint32_t bar = smem_u32(&q_full[qr.i]);
            mbar_arrive_expect_tx(bar, (uint32_t)SM::kTile);
            for (int q = 0; q < NQ; ++q)
              tma_chunk_q(smem_u32(Qt + (size_t)qr.i * SM::kTile + (size_t)q * 128 * 128), &tmq, q * 64, hq, x.row0 + t0, bar);
          }
          armed |= 1u << (8 + qr.i);
          armed_par = (armed_par & ~(1u << (8 + qr.i))) | ((uint32_t)qr.ph << (8 + qr.i));
          qr.next(QS);
          if (++li == LS) li = 0;
        }
    }
#pragma unroll
    for (int s = 0; s < 2; ++s)
      if (((armed >> s) & 1u) && !mbar_wait_warp(smem_u32(&k_full[s]), (armed_par >> s) & 1u)) set_status(c, kDevWaitTimeout);
#pragma unroll
    for (int s = 0; s < QS; ++s)
      if (((armed >> (8 + s)) & 1u) && !mbar_wait_warp(smem_u32(&q_full[s]), (armed_par >> (8 + s)) & 1u)) set_status(c, kDevWaitTimeout);
  } else if (warp == 1) {
    // ---------------- multiplies ----------------
    FeatRing kr{0, 0}, qr{0, 0};
    int it = 0, blk = 0;
    bool ok = true;
    const uint32_t idesc = umma_idesc_bf16(128, kCfQueries);
    while (ok) {
      const int ri = it % kCfItems;
      if (!mbar_spin(smem_u32(&it_full[ri]), (it / kCfItems) & 1)) { set_status(c, kDevWaitTimeout); break; }
      const CfItem x = Items[ri];
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&it_empty[ri]));
      ++it;
      if (x.kind == 0) break;
      if (x.m0 >= x.m1) continue;
      const int tiles = x.n - x.pg0 * kPage > 128 ? 2 : 1;
      if (!mbar_spin(smem_u32(&k_full[kr.i]), kr.ph)) { set_status(c, kDevWaitTimeout); break; }
      for (int b = 0; b < (x.j1 - x.j0) * (x.m1 - x.m0) && ok; ++b, ++blk) {
        if (!mbar_spin(smem_u32(&q_full[qr.i]), qr.ph)) { set_status(c, kDevWaitTimeout); ok = false; break; }
        for (int t = 0; t < 2; ++t) {   // (an absent second tile is handed over all the same, to keep the phases in step)
          const int acc = t * 2 + (blk & 1);
          if (!mbar_spin(smem_u32(&acc_empty[acc]), ((blk >> 1) & 1) ^ 1)) { set_status(c, kDevWaitTimeout); ok = false; break; }
          tc_fence_after();
          if (lane == 0) {
            if (t < tiles) {
              const uint64_t ad = umma_desc_sw128(smem_u32(Kt + (size_t)(kr.i * 2 + t) * SM::kTile));
              const uint64_t bd = umma_desc_sw128(smem_u32(Qt + (size_t)qr.i * SM::kTile));
#pragma unroll
              for (int ks = 0; ks < D / 16; ++ks) {
                const uint64_t o = (uint64_t)(((ks >> 2) * 128 * 128 + (ks & 3) * 32) >> 4);
                umma_bf16(tmem_base + acc * 128, ad + o, bd + o, idesc, ks > 0);
              }
            }
            umma_commit(smem_u32(&acc_full[acc]));
          }
          __syncwarp();
        }
        if (!ok) break;
        if (lane == 0) umma_commit(smem_u32(&q_empty[qr.i]));
        __syncwarp();
        qr.next(QS);
      }
      if (ok && lane == 0) umma_commit(smem_u32(&k_empty[kr.i]));
      __syncwarp();
      kr.next(2);
    }
    if (lane == 0) umma_commit(smem_u32(mma_done));
    __syncwarp();
    if (!mbar_spin(smem_u32(mma_done), 0)) set_status(c, kDevWaitTimeout);
  } else if (warp >= 4) {
    // ---------------- sums: thread = pair ----------------
    const int t = (warp - 4) >> 2, quarter = warp & 3, R = quarter * 32 + lane;
    const uint32_t trow = tmem_base + ((uint32_t)(quarter * 32) << 16) + t * 256;
    int it = 0, blk = 0;
    FeatRing lr{0, 0};
    bool ok = true;
    while (ok) {
      const int ri = it % kCfItems;
      if (!mbar_wait_warp(smem_u32(&it_full[ri]), (it / kCfItems) & 1)) { set_status(c, kDevWaitTimeout); break; }
      const CfItem x = Items[ri];
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&it_empty[ri]));
      ++it;
      if (x.kind == 0) break;
      const int slot = x.pg0 * kPage + t * 128 + R;
      const bool live = slot < x.n;
      float *frow = nullptr;
      int jlo = INT_MAX, jhi = 0;   // the tokens that see this pair
      if (live) {
        const int *ptrow = c.pt + (size_t)x.seg * c.max_pages;
        frow = meta_row(c, c.pool + (size_t)__ldcg(ptrow + slot / kPage) * c.page_bytes, slot % kPage);
        jlo = max(0, slot - x.base);
        jhi = x.T;
        if (a.window) {
          const int pos = __ldcg(reinterpret_cast<const int32_t *>(frow) + c.F);
          if (pos >= a.sinks) {
            const long long past = (long long)pos + a.window;   // the first position that no longer sees the pair
            if (x.steady) jhi = (int)max(0LL, min((long long)x.T, past - x.p0));
            else jhi = slot_lower_bound(c, ptrow, x.base, x.n, (int)min(past, (long long)INT_MAX)) - x.base;
          }
        }
      }
      const float inv_T = 1.f / (float)x.T;
      const bool any = __any_sync(0xffffffffu, live);
      for (int j = x.j0; j < x.j1 && ok; ++j) {
        float old_sum = 0.f, old_dec = 0.f;
        if (live) { old_sum = __ldcg(frow + j * 6 + 4); old_dec = __ldcg(frow + j * 6 + 5); }
        float run = 0.f, w8 = 0.f, w16 = 0.f, w32 = 0.f;
        for (int m = x.m0; m < x.m1; ++m, ++blk) {
          const int acc = t * 2 + (blk & 1);
          if (!mbar_wait_warp(smem_u32(&l_full[lr.i]), lr.ph) || !mbar_wait_warp(smem_u32(&acc_full[acc]), (blk >> 1) & 1)) {
            set_status(c, kDevWaitTimeout); ok = false; break;
          }
          __syncwarp();
          tc_fence_after();
          if (any) {
            const float *mp = Lt + lr.i * kCfQueries;
            const int t0 = x.T - kCfQueries * (m + 1), lo = jlo - t0, hi = jhi - t0;   // columns [lo, hi) count
            const uint32_t ta = trow + (blk & 1) * 128;
            const bool plain = __all_sync(0xffffffffu, lo <= 0 && hi >= kCfQueries);
#pragma unroll
            for (int q = 3; q >= 0; --q) {
              if (!plain && !__any_sync(0xffffffffu, lo < q * 32 + 32 && hi > q * 32)) {
                if (m == 0 && q == 3) w8 = w16 = w32 = 0.f;
                continue;
              }
              uint32_t v[32];
              tmem_ld32_issue(ta + q * 32, v);
              tmem_ld_wait(v);
              if (q == 3 && m == 0) {
                if (plain) cf_chunk<true, false>(v, mp + q * 32, a.scale_log2, 0, 0, run, w8, w16);
                else cf_chunk<true, true>(v, mp + q * 32, a.scale_log2, lo - q * 32, hi - q * 32, run, w8, w16);
                w32 = run;
              } else {
                float d8, d16;
                if (plain) cf_chunk<false, false>(v, mp + q * 32, a.scale_log2, 0, 0, run, d8, d16);
                else cf_chunk<false, true>(v, mp + q * 32, a.scale_log2, lo - q * 32, hi - q * 32, run, d8, d16);
              }
            }
          }
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_u32(&acc_empty[acc]));
          lr.next(LS);
        }
        if (live && ok) {
          float *f = frow + j * 6;
          const float chunk = run * inv_T;
          f[0] = w8 * (1.f / 8.f); f[1] = w16 * (1.f / 16.f); f[2] = w32 * (1.f / 32.f);
          f[3] = chunk;
          f[4] = old_sum + chunk;
          f[5] = fmaf(kFeatDecay, old_dec, chunk);
        }
      }
    }
  }
  // ---- common exit ----
  tc_fence_before();
  __syncthreads();
  if (warp == 3) tmem_dealloc(tmem_base, 512);
}

}  // namespace fkv
