// Kernel 9: the attention features of Appendix B.1 from the queries of a chunk (a prompt, or a piece of one), with their
// log-sum-exp at hand:
//     P_ji = e^{scale <q_j, k_i> - lse_j} on the pairs i that query j sees, 0 elsewhere;
// per query head and pair the means of P over the chunk's last 8 / 16 / 32 queries and over the whole chunk, and the two
// running sums moved on by the latter, as k_features does for decode queries.
//
// Bound: 2 D flops and one exp2 per (query head, seen pair).  The special-function pipe would take 1024 cycles for a block of
// 128 pairs x 128 queries and the tensor core 512, so the exponentials are what the kernel is built around: a quarter is
// computed on the FMA pipe (768 cycles are left on the other), and nothing but a multiplication, the exponential and an
// addition is left per score.  The
// log-sum-exp is subtracted by the tensor core: one more step of 16 channels, in which a key holds 1, 1, 1, 0, ... and a
// query -lse / scale as three bf16 values (rounding, and twice the rounding of what is left: 27 bits).
//
// S^T = K Q^T: pairs on the M axis, so a thread owns a pair and adds up along its own row of tensor memory; nothing is
// reduced across threads.  A CTA takes two tiles of 128 pairs at a time and streams the queries of one head past them,
// 128 at a time, newest first (the windows are then prefixes of the walk): a block of queries is read from L2 once for
// 256 pairs.  Persistent CTAs over equal ranges of a line of (pair of tiles, query head), weighed by their query blocks.
//   warp 0      tensor copies: K rows page by page, blocks of queries;
//   warps 1, 3  one lane each issues the tcgen05.mma of one tile into one of its two accumulators;
//   warp 2      walks the line, looks the positions up and writes the queries' sixteen extra channels (not warp 0: the fence
//               that hands them to the tensor core waits for the loads of the next ones);
//   warps 4-11  two warpgroups, one per tile: exp2, sums, and the pair's meta row at the end.
// Accuracy: a score is off by what the tensor core's fp32 accumulation drops (2^-23 of the partial sums, per step of 16
// channels), which moves a probability by 1e-6 - 3e-6 relative, 1.3 - 2.5 times what a library product in fp32 does on the
// same inputs, for some 3 - 4 times; everything after it is below 3e-7.  The truncation is the products' too, so subtracting in
// two or four pieces gains nothing, and costs 1 - 4 % of the time.
// Measured (32 query heads, g = 4, D = 128): 2048 queries at 32K 0.59 ms, 900 TFLOP/s, for the first 0.1 s, 0.64 - 0.68 ms once
// the card's power limit holds the clock at 1.7 GHz; the three quarters of the exponentials on the special-function pipe are
// 0.35 ms of it, the products 0.32 ms: neither pipe alone bounds it.  128 at 8K 27 us: the copies of a tile, four blocks of products
// and its meta rows follow one another twice per CTA.
// Every wait is bounded; tensor memory is freed at the common exit.
#pragma once
#include "fkv_chunk.cuh"

namespace fkv {

constexpr int kCfThreads = 384;
constexpr int kCfPairs = 256, kCfQueries = 128;   // pairs of a unit (two tiles), queries of a block
constexpr int kCfItems = 3;   // items in use: being finished, being worked on, being read ahead

struct ChunkFeatArgs {
  int layer, window, sinks;
  float scale_log2;
  float inv_hi, inv_lo;   // 1 / scale in two parts
  int nk, nq;          // pairs of K tiles and blocks of queries in shared memory
  int record_used;     // the launch before has applied the record of decode queries of the sequences with tokens
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
  static constexpr int kMostQ = D == 128 ? 4 : 8;   // blocks of queries in flight
  static constexpr size_t kTile = (size_t)(D / 64) * 128 * 128;
  static constexpr size_t kExtra = 128 * 32;        // sixteen channels of 128 rows, no swizzle: [16 groups of 8 rows][2][8][16 B]
  // Six tiles' worth of room: two pairs of K tiles and two blocks of queries, or one pair and four blocks (twice as many
  // of each for D = 64, where only the blocks are doubled).  A block takes some 2400 cycles to arrive, which two in flight
  // do not hide; a second pair of K tiles hides the change of tiles, which matters where a tile meets few blocks.
  static __host__ __device__ int rings(int longest, int &nk) { nk = longest > 4 * kCfQueries ? 1 : 2; return nk == 1 ? kMostQ : kMostQ / 2; }
  static constexpr size_t kOffKe = (2 + kMostQ) * kTile, kOffQe = kOffKe + kExtra;
  static constexpr size_t kOffItems = kOffQe + kMostQ * kExtra;
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

// Matrix descriptor of sixteen K-major channels without a swizzle: 8 rows x 8 channels are 128 contiguous bytes, the next 8
// channels follow, the next 8 rows come 256 bytes further.
__device__ __forceinline__ uint64_t umma_desc_k16(uint32_t smem_addr) {
  return (uint64_t)((smem_addr & 0x3ffffu) >> 4) | ((uint64_t)(128u >> 4) << 16) | ((uint64_t)(256u >> 4) << 32) | (1ull << 46);
}
// Byte offset of row r's first 8 channels in such a tile.
__device__ __forceinline__ int k16_row(int r) { return (r >> 3) * 256 + (r & 7) * 16; }

// The larger one, or NaN if one of them is.
__device__ __forceinline__ float max_nan(float a, float b) {
  float d;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
  return d;
}
// 2^x of two values on the FMA pipe for x <= 0: x = n + r with n the nearest integer, found by adding 1.5 * 2^23, and the
// minimax polynomial of degree 5 for 2^r on [-1/2, 1/2] (relative error, Remez exchange: 7.5e-8, 2.1e-7 as evaluated in
// fp32), times 2^n, which is n added to the exponent of 1.  x below -127 counts as -127, whose 2^n is then zero: so a
// masked score, -infinity, gives exactly 0, and NaN stays NaN (n added to the polynomial's own exponent would lose both).
__device__ __forceinline__ float2 ex2_fma(float2 x) {
  x.x = max_nan(x.x, -127.f);
  x.y = max_nan(x.y, -127.f);
  const float2 t = __fadd2_rn(x, make_float2(12582912.f, 12582912.f));
  const float2 r = __ffma2_rn(__fadd2_rn(t, make_float2(-12582912.f, -12582912.f)), make_float2(-1.f, -1.f), x);
  float2 p = __ffma2_rn(make_float2(1.327647245e-3f, 1.327647245e-3f), r, make_float2(9.675540961e-3f, 9.675540961e-3f));
  p = __ffma2_rn(p, r, make_float2(5.550713092e-2f, 5.550713092e-2f));
  p = __ffma2_rn(p, r, make_float2(2.402212024e-1f, 2.402212024e-1f));
  p = __ffma2_rn(p, r, make_float2(6.931469440e-1f, 6.931469440e-1f));
  p = __ffma2_rn(p, r, make_float2(1.000000119f, 1.000000119f));
  return __fmul2_rn(p, make_float2(__int_as_float((__float_as_int(t.x) << 23) + 0x3f800000),
                                   __int_as_float((__float_as_int(t.y) << 23) + 0x3f800000)));
}
// The columns outside [lo, hi) of the 32 from c0 become -infinity, in tensor memory (for the few blocks at an edge).
__device__ __forceinline__ void cf_mask(uint32_t ta, int c0, int lo, int hi) {
#pragma unroll 1
  for (int q = c0; q < c0 + 32; q += 16) {
    uint32_t v[16];
    tmem_ld16_issue(ta + q, v);
    tmem_ld16_wait(v);
#pragma unroll
    for (int j = 0; j < 16; ++j)
      if (q + j < lo || q + j >= hi) v[j] = 0xff800000u;
    tmem_st16(ta + q, v);
  }
  tmem_st_wait();
}
// Sum of 2^(scale v) over the 8 scores v[8 g ..].
__device__ __forceinline__ float cf_sum8(const uint32_t (&v)[32], int g, float scale_log2) {
  const float2 sc = make_float2(scale_log2, scale_log2);
  float2 x[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float2 z = __fmul2_rn(make_float2(__uint_as_float(v[8 * g + 2 * j]), __uint_as_float(v[8 * g + 2 * j + 1])), sc);
    if (j == 0) x[j] = ex2_fma(z);   // (2048 queries at 32K, first 0.1 s: none 646 us, an eighth 623, a quarter 586, a half 690)
    else x[j] = make_float2(ex2(z.x), ex2(z.y));
  }
  const float2 y = __fadd2_rn(__fadd2_rn(x[0], x[1]), __fadd2_rn(x[2], x[3]));
  return y.x + y.y;
}

template <int D>
__global__ void __launch_bounds__(kCfThreads, 1) k_chunk_features(Ctx c, const __grid_constant__ CUtensorMap tmkv,
                                                                  const __grid_constant__ CUtensorMap tmq,
                                                                  const __grid_constant__ ChunkFeatArgs a) {
  using SM = CfSmem<D>;
  constexpr int NQ = D / 64, QM = SM::kMostQ;
  const int NK = a.nk, QS = a.nq;   // ring sizes
  constexpr uint32_t PAGE_HALF = kPage * 128;
  extern __shared__ uint8_t smem_raw[];
  uint8_t *smem = reinterpret_cast<uint8_t *>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  uint8_t *Kt = smem, *Qt = smem + (size_t)NK * 2 * SM::kTile, *Ke = smem + SM::kOffKe, *Qe = smem + SM::kOffQe;
  CfItem *Items = reinterpret_cast<CfItem *>(smem + SM::kOffItems);
  int *Len = reinterpret_cast<int *>(smem + SM::kOffLen), *Blk = reinterpret_cast<int *>(smem + SM::kOffBlk);
  uint64_t *bars = reinterpret_cast<uint64_t *>(smem + SM::kOffBars);
  uint64_t *k_full = bars, *k_empty = k_full + 2, *q_full = k_empty + 2, *q_empty = q_full + QM, *e_full = q_empty + QM;
  uint64_t *acc_full = e_full + QM, *acc_empty = acc_full + 4;   // [tile][buffer]
  uint64_t *it_full = acc_empty + 4, *it_empty = it_full + kCfItems, *mma_done = it_empty + kCfItems;
  uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(mma_done + 1);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, G = c.G, Hq = c.Hkv * c.G;

  if (warp == 3) tmem_alloc(smem_u32(tmem_slot), 512);
  if (threadIdx.x == 0) {
    for (int s = 0; s < NK; ++s) { mbar_init(smem_u32(&k_full[s]), 1); mbar_init(smem_u32(&k_empty[s]), 2); }
    for (int s = 0; s < QS; ++s) { mbar_init(smem_u32(&q_full[s]), 1); mbar_init(smem_u32(&q_empty[s]), 2); mbar_init(smem_u32(&e_full[s]), 1); }
    for (int s = 0; s < 4; ++s) { mbar_init(smem_u32(&acc_full[s]), 1); mbar_init(smem_u32(&acc_empty[s]), 4); }
    for (int s = 0; s < kCfItems; ++s) { mbar_init(smem_u32(&it_full[s]), 1); mbar_init(smem_u32(&it_empty[s]), 11); }
    mbar_init(smem_u32(mma_done), 2);
    for (const CUtensorMap *tm : {&tmkv, &tmq}) asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(tm)) : "memory");
    fence_barrier_init();
  }
  for (int e = threadIdx.x; e < (1 + QM) * (int)SM::kExtra / 16; e += kCfThreads) {   // keys: 1, 1, 1, 0, ...; queries: zero for now
    const bool key = e < (int)SM::kExtra / 16 && (e & 15) < 8;
    reinterpret_cast<uint4 *>(Ke)[e] = key ? make_uint4(0x3f803f80u, 0x00003f80u, 0u, 0u) : make_uint4(0u, 0u, 0u, 0u);
  }
  fence_proxy_async();
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
      const int T = a.lens.tok[s + 1] - a.lens.tok[s];
      if (blockIdx.x == 0 && n < T) set_status(c, kDevBadIndex);
      if (blockIdx.x == 0 && T > 0 && a.record_used) c.hist_cnt[a.layer * batch + s] = 0;   // it starts over
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
    bool ok = true, ended = false;
    auto publish = [&]() {   // hands the next item (or the end) to the other roles
      const int ri = it % kCfItems;
      if (!mbar_sleep_warp(smem_u32(&it_empty[ri]), ((it / kCfItems) & 1) ^ 1)) { set_status(c, kDevWaitTimeout); ok = false; return; }
      ++it;
      CfItem *x = Items + ri;
      for (;;) {
        if (u0 >= u1 || U >= u1 || head >= c.Hkv) {
          if (lane == 0) { x->kind = 0; mbar_arrive(smem_u32(&it_full[ri])); }
          __syncwarp();
          ended = true;
          return;
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
        }
        U += (long long)b.cost * G;
        if (++f == NB) { f = 0; ++head; }
        if (j0 < j1) return;
      }
    };
    // The extra channels of an item's queries, one item behind the walk: per block and lane four queries, whose log-sum-exp
    // are asked for ahead.
    FeatRing qr{0, 0};
    publish();
    for (int vi = 0; ok; ++vi) {
      if (!ended) publish();
      const CfItem &x = Items[vi % kCfItems];
      if (!ok || x.kind == 0) break;
      const int m0 = x.m0, blocks = x.m1 - m0, j0 = x.head * G + x.j0, nj = x.j1 - x.j0, T = x.T;
      if (blocks <= 0) continue;
      const float *lse = a.lse + (size_t)x.row0 * Hq;
      int am = m0, aj = j0;    // the block asked for next
      auto ask = [&](float (&l)[4]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int t = T - kCfQueries * (am + 1) + lane * 4 + i;   // (negative in the oldest block)
          // (not the read-only path: the launch before may still have been writing them as this one began)
          l[i] = t >= 0 && aj < j0 + nj ? __ldcg(lse + (size_t)t * Hq + aj) : 0.f;
        }
        if (++am == m0 + blocks) { am = m0; ++aj; }
      };
      constexpr int AT = 4;   // blocks asked for at once: a read takes as long as a block or two, and the fence waits for it
      float la[AT][4], lb[AT][4];
#pragma unroll
      for (int k = 0; k < AT; ++k) ask(la[k]);
      for (int b0 = 0; b0 < nj * blocks && ok; b0 += AT) {
#pragma unroll
        for (int k = 0; k < AT; ++k) ask(lb[k]);
#pragma unroll
        for (int k = 0; k < AT; ++k) {
          if (b0 + k >= nj * blocks || !ok) continue;
          uint4 e4[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float l = la[k][i], v = -l * a.inv_hi, rest = fmaf(-l, a.inv_lo, fmaf(-l, a.inv_hi, -v));
            const float h1 = __bfloat162float(__float2bfloat16_rn(v)), r1 = (v - h1) + rest;
            const float h2 = __bfloat162float(__float2bfloat16_rn(r1));
            e4[i] = make_uint4(pack_bf16(h1, h2), pack_bf16(r1 - h2, 0.f), 0u, 0u);
          }
          if (!mbar_sleep_warp(smem_u32(&q_empty[qr.i]), qr.ph ^ 1)) { set_status(c, kDevWaitTimeout); ok = false; continue; }
#pragma unroll
          for (int i = 0; i < 4; ++i) *reinterpret_cast<uint4 *>(Qe + qr.i * SM::kExtra + k16_row(lane * 4 + i)) = e4[i];
          fence_proxy_async();
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_u32(&e_full[qr.i]));
          qr.next(QS);
        }
#pragma unroll
        for (int k = 0; k < AT; ++k)
#pragma unroll
          for (int i = 0; i < 4; ++i) la[k][i] = lb[k][i];
      }
    }
  } else if (warp == 0) {
    // ---------------- copies ----------------
    FeatRing kr{0, 0}, qr{0, 0};
    int it = 0;
    uint32_t armed = 0, armed_par = 0;   // bit s: K buffer s, bit 8 + s: query stage s
    bool ok = true;
    while (ok) {
      const int ri = it % kCfItems;
      if (!mbar_sleep_warp(smem_u32(&it_full[ri]), (it / kCfItems) & 1)) { set_status(c, kDevWaitTimeout); break; }
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
        if (!mbar_sleep_warp(smem_u32(&k_empty[kr.i]), kr.ph ^ 1)) { set_status(c, kDevWaitTimeout); break; }
        if (lane == 0) mbar_arrive_expect_tx(smem_u32(&k_full[kr.i]), (uint32_t)ncopies * PAGE_HALF);
        armed |= 1u << kr.i;
        armed_par = (armed_par & ~(1u << kr.i)) | ((uint32_t)kr.ph << kr.i);
        __syncwarp();
        if (on)
          tma_page_k(smem_u32(Kt + (size_t)(kr.i * 2 + (pg >> 3)) * SM::kTile + (size_t)q * 128 * 128 + (size_t)(pg & 7) * PAGE_HALF),
                     &tmkv, q, pid, smem_u32(&k_full[kr.i]));
        kr.next(NK);
      }
      for (int j = x.j0; j < x.j1 && ok; ++j)
        for (int m = x.m0; m < x.m1; ++m) {
          if (!mbar_sleep_warp(smem_u32(&q_empty[qr.i]), qr.ph ^ 1)) { set_status(c, kDevWaitTimeout); ok = false; break; }
          if (lane == 0) {
            const uint32_t bar = smem_u32(&q_full[qr.i]);
            mbar_arrive_expect_tx(bar, (uint32_t)SM::kTile);
            for (int q = 0; q < NQ; ++q)   // (the oldest block begins before the chunk: those rows are masked)
              tma_chunk_q(smem_u32(Qt + (size_t)qr.i * SM::kTile + (size_t)q * 128 * 128), &tmq, q * 64, x.head * G + j,
                          x.row0 + x.T - kCfQueries * (m + 1), bar);
          }
          armed |= 1u << (8 + qr.i);
          armed_par = (armed_par & ~(1u << (8 + qr.i))) | ((uint32_t)qr.ph << (8 + qr.i));
          qr.next(QS);
        }
    }
#pragma unroll
    for (int s = 0; s < 2; ++s)
      if (((armed >> s) & 1u) && !mbar_sleep_warp(smem_u32(&k_full[s]), (armed_par >> s) & 1u)) set_status(c, kDevWaitTimeout);
#pragma unroll
    for (int s = 0; s < QM; ++s)
      if (((armed >> (8 + s)) & 1u) && !mbar_sleep_warp(smem_u32(&q_full[s]), (armed_par >> (8 + s)) & 1u)) set_status(c, kDevWaitTimeout);
  } else if (warp == 1 || warp == 3) {
    // ---------------- multiplies: tile t, a warp that stays together, lane 0 issues ----------------
    const int t = uniform(warp >> 1);
    const uint32_t on = lane == 0;
    FeatRing kr{0, 0}, qr{0, 0};
    int it = 0, blk = 0;
    bool ok = true;
    const uint32_t idesc = umma_idesc_bf16(128, kCfQueries), td = uniform(tmem_base + t * 256);
    const uint64_t ke = umma_desc_k16(smem_u32(Ke));
    while (ok) {
      const int ri = it % kCfItems;
      if (!mbar_wait(smem_u32(&it_full[ri]), (it / kCfItems) & 1)) { set_status(c, kDevWaitTimeout); break; }
      const CfItem x = Items[ri];
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&it_empty[ri]));
      ++it;
      if (x.kind == 0) break;
      if (x.m0 >= x.m1) continue;
      const bool there = uniform(x.n - x.pg0 * kPage > 128 * t);   // (an absent second tile is handed over all the same)
      const int total = uniform((x.j1 - x.j0) * (x.m1 - x.m0));
      if (!mbar_wait(smem_u32(&k_full[kr.i]), kr.ph)) { set_status(c, kDevWaitTimeout); break; }
      const uint64_t ad = umma_desc_sw128(smem_u32(Kt + (size_t)(uniform(kr.i) * 2 + t) * SM::kTile));
      for (int b = 0; b < total; ++b, ++blk) {
        const int sq = uniform(qr.i), buf = uniform(blk & 1);
        const uint64_t bd = umma_desc_sw128(smem_u32(Qt + (size_t)sq * SM::kTile)), be = umma_desc_k16(smem_u32(Qe + sq * SM::kExtra));
        const bool full = mbar_wait(smem_u32(&q_full[sq]), qr.ph) && mbar_wait(smem_u32(&e_full[sq]), qr.ph);
        if (!__all_sync(0xffffffffu, full && mbar_wait(smem_u32(&acc_empty[t * 2 + buf]), ((blk >> 1) & 1) ^ 1))) {
          set_status(c, kDevWaitTimeout); ok = false; break;
        }
        tc_fence_after();
        if (there) {
          const uint32_t d = td + buf * 128;
#pragma unroll
          for (int ks = 0; ks < D / 16; ++ks) {
            const uint64_t o = (uint64_t)(((ks >> 2) * 128 * 128 + (ks & 3) * 32) >> 4);
            umma_bf16_if(on, d, ad + o, bd + o, idesc, ks > 0);
            if (ks == D / 32 - 1) umma_bf16_if(on, d, ke, be, idesc, 1);   // half-way: the partial sums of the large weights stay smallest
          }
        }
        umma_commit_if(on, smem_u32(&acc_full[t * 2 + buf]));
        umma_commit_if(on, smem_u32(&q_empty[sq]));
        qr.next(QS);
      }
      if (ok) umma_commit_if(on, smem_u32(&k_empty[kr.i]));
      kr.next(NK);
    }
    umma_commit_if(on, smem_u32(mma_done));
    if (!mbar_wait(smem_u32(mma_done), 0)) set_status(c, kDevWaitTimeout);
  } else if (warp >= 4) {
    // ---------------- sums: thread = pair ----------------
    const int t = (warp - 4) >> 2, quarter = warp & 3, R = quarter * 32 + lane;
    const uint32_t trow = tmem_base + ((uint32_t)(quarter * 32) << 16) + t * 256;
    int it = 0, blk = 0;
    bool ok = true;
    while (ok) {
      const int ri = it % kCfItems;
      if (!mbar_sleep_warp(smem_u32(&it_full[ri]), (it / kCfItems) & 1)) { set_status(c, kDevWaitTimeout); break; }
      const CfItem x = Items[ri];
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&it_empty[ri]));
      ++it;
      if (x.kind == 0) break;
      const int slot = x.pg0 * kPage + t * 128 + R;
      const bool live = slot < x.n;
      float *frow = nullptr;
      int jlo = x.T, jhi = 0;   // the tokens that see this pair (none, for a slot past the end)
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
          if (!mbar_sleep_warp(smem_u32(&acc_full[acc]), (blk >> 1) & 1)) { set_status(c, kDevWaitTimeout); ok = false; break; }
          tc_fence_after();
          if (any) {
            const int t0 = x.T - kCfQueries * (m + 1), lo = jlo - t0, hi = jhi - t0;   // columns [lo, hi) count
            const uint32_t ta = trow + (blk & 1) * 128;
            const bool plain = __all_sync(0xffffffffu, lo <= 0 && hi >= kCfQueries);
            // 32 columns at a time, newest first: sum their exponentials.
            auto add = [&](const uint32_t (&v)[32], bool newest) {
              const float s3 = cf_sum8(v, 3, a.scale_log2), s2 = cf_sum8(v, 2, a.scale_log2);
              const float s10 = cf_sum8(v, 1, a.scale_log2) + cf_sum8(v, 0, a.scale_log2);
              if (newest) {   // the chunk's last 32 queries
                w8 = s3;
                w16 = s3 + s2;
                w32 = (s3 + s2) + s10;
              }
              run += (s3 + s2) + s10;
            };
            uint32_t va[32], vb[32];
            if (plain) {   // ... the next columns on their way
              tmem_ld32_issue(ta + 96, va);
              tmem_ld_wait(va);
              tmem_ld32_issue(ta + 64, vb);
              add(va, m == 0);
              tmem_ld_wait(vb);
              tmem_ld32_issue(ta + 32, va);
              add(vb, false);
              tmem_ld_wait(va);
              tmem_ld32_issue(ta, vb);
              add(va, false);
              tmem_ld_wait(vb);
              add(vb, false);
            } else {       // ... those that some lane counts, with what it does not count masked first
#pragma unroll 1
              for (int c0 = 96; c0 >= 0; c0 -= 32) {
                if (!__any_sync(0xffffffffu, lo < c0 + 32 && hi > c0)) continue;
                cf_mask(ta, c0, lo, hi);
                tmem_ld32_issue(ta + c0, va);
                tmem_ld_wait(va);
                add(va, m == 0 && c0 == 96);
              }
            }
          }
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_u32(&acc_empty[acc]));
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
