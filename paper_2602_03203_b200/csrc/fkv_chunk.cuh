// Kernel 8: a chunk of new tokens per sequence - the pairs are stored behind the ones that stay, and every token of the
// chunk attends over the pairs up to its own:
//     z_ji = scale <q_j, k_i>,   lse_j = ln sum_{i in Seen(j)} e^{z_ji},   o_j = sum_{i in Seen(j)} e^{z_ji - lse_j} v_i,
// Seen(j) = the pairs i at or before query j's own slot with (no window, or p_j - x_i < window, or x_i < sinks): x_i and
// p_j are token positions, so a window means the same before and after an eviction.  Positions grow with the slot: the
// pairs a query sees are slots [0, a) and [w_j, e_j), a and w_j found by searching the stored positions.
//
// Bound: 4 D flops and one exp2 per (query head, seen pair); with few query rows per KV head the bytes of the pairs
// (4 D each, once per group) take longer.
//
// Layout of the contraction.  The g query heads of a group share K and V, so a tile of 128 query rows is (128 / g tokens)
// x (g heads); an item of work is one KV head x two such tiles over the pages their tokens see.  One persistent CTA per
// SM; the pages of all items form one line that is cut into equal ranges, one per CTA, so the split is even whatever the
// batch looks like (one long sequence, many short ones, drafts of a few tokens over long caches).  An item that a cut
// goes through leaves partial results (O, m, l) which k_chunk_merge joins.
//   warp 0      tensor copies (TMA) of the item's query tiles and of K, page by page (one copy = 16 rows x 64 channels; the
//               page record's swizzle is the shared-memory swizzle), into a ring of key tiles of five pages (D = 64: six);
//   warp 1      one lane issues tcgen05.mma S = Q K^T (K-major operands) into tensor memory;
//   warp 3      ... and O += P V with P read from tensor memory and V as an MN-major operand (channels run along its
//               rows: no transpose anywhere);
//   warp 2      walks the items ahead of the others, searches the positions, and copies V (one copy = a page's 16 rows): a
//               warp issues a copy per 80 - 100 cycles, so one for K and V would not keep up;
//   warps 4-11  two warpgroups, each with a stream of its own (S and O accumulators): thread = query row; running
//               maximum, exp2, row sum in fp32, P rounded to bf16 into columns of its own.  O is rescaled only when the
//               maximum has grown by more than 2^24: until then P is at most 2^24, which bf16 holds as exactly as 1.
// Measured (attention and merge, back to back; 32 query heads, g = 4, D = 128): 2048 tokens at 32K 1.00 ms = 1065 TFLOP/s for the
// first 0.1 s, 1.15 - 1.21 ms (880 - 925) once the card's power limit holds the clock at 1.5 GHz; the tensor core and the
// exponentials, 1 : 1 in cycles, hold each other up.  256 tokens at 8K 60 us, 33 of them at that rate and the rest the start, the
// items' ends and the merge; 16 sequences with a few drafts over long caches 88 us = 4.8 TB/s with it all, the pages
// themselves at 6.1 TB/s; 5 drafts at 8K 26 us, latency.
// The streams are the item's two query tiles; an item with one tile gives its key tiles to the streams in turn, and the
// streams' results are joined through shared memory.
// Every wait is bounded; tensor memory is freed at the common exit.
#pragma once
#include <cuda.h>
#include <limits.h>
#include "fkv_dev.cuh"
#include "fkv_attend.cuh"
#include "fkv_features.cuh"
#include "fkv_rkv.cuh"

namespace fkv {

constexpr int kChunkCtas = 148;       // most CTAs of a launch: each has two slots for partial results in the workspace
constexpr int kChunkThreads = 384;
constexpr int kChunkRows = 128;       // query rows of a tile = M of the mma
constexpr int kChunkMinPages = 8;     // least work of a CTA
constexpr int kChunkInfo = 8;         // words that describe a CTA's unfinished item to the merge
constexpr float kChunkGrow = 24.f;    // log2 of the growth of a row's maximum that O is rescaled for
constexpr int kTreeNodes = 256;       // most nodes of a draft tree
constexpr int kTreeWords = kTreeNodes / 32;   // words of a node's mask: bit i says that it sees node i
constexpr int kTreeOne = 2, kTreeTwo = 3;  // what a page counts in an item of a tree with one query tile, and with two
constexpr int kChunkItems = 3;        // items in use: being finished, being worked on, being read ahead

// Prefix sums of the chunk lengths over the sequences, and the pairs that stay (use == 0: all of them).
struct ChunkLens {
  int tok[kMaxBatch + 1];
};
struct ChunkKeep {
  int use;
  int keep[kMaxBatch];
};

// ---------------------------------------------------------------- storing the chunk
// Every CTA works the page arithmetic out for itself (one thread per sequence, two prefix sums): pages to take from the
// free stack where a sequence grows past its last page, pages to return where it shrinks.  Growth that the stack does not
// cover is served from the returned pages, in their order: nothing reads their pairs any more.  A warp stores one pair.  The
// last CTA to finish returns what is left, moves the stack top and the lengths and takes rolled-back queries off the record.
// A sequence that the device finds past its capacity or shorter than `keep` is skipped; without enough pages, free and
// returned together, the whole call is.
// Bound: bytes (8 D a pair and KV head, read and written); back to back 4.7 us for 5 tokens, 5.3 for 256, 12.7 for 2048 on 8 heads
// (a launch and four dependent reads: length, page, last position, free stack).
// TREE: the chunk is a draft tree (kernel 10); a node's position is one behind its parent's, so it follows from the number
// of its ancestors: the nodes ahead of it that its mask names (whatever else a caller's own mask says, it is behind the last pair's).
__device__ __forceinline__ int tree_before(uint32_t word, int w, int j) {   // those in word w of node j's mask
  const int e = j - 32 * w;
  return __popc(word & (e <= 0 ? 0u : e >= 32 ? ~0u : (1u << e) - 1u));
}
template <bool TREE>
__global__ void __launch_bounds__(256) k_append_chunk(Ctx c, int layer, const uint8_t *k, const uint8_t *v, const int32_t *pos,
                                                      const __grid_constant__ ChunkLens lens,
                                                      const __grid_constant__ ChunkKeep keep, const uint32_t *masks) {
  static_assert(kMaxBatch <= 256, "one thread per sequence");
  __shared__ int s_scan[33];
  __shared__ int s_keep[kMaxBatch], s_old[kMaxBatch], s_pop[kMaxBatch], s_push[kMaxBatch];
  __shared__ int s_last;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  griddep_wait();
  griddep_launch();
  const int s = tid;
  int n_old = 0, kp = 0, T = 0, pop = 0, push = 0, bad = 0;
  const int top = __ldcg(c.ctrl + CTRL_FREE_TOP);
  if (s < c.batch) {
    n_old = __ldcg(c.len + layer * c.batch + s);
    T = lens.tok[s + 1] - lens.tok[s];
    kp = keep.use ? keep.keep[s] : n_old;
    if (kp > n_old) { bad = (int)kDevBadIndex; kp = -1; }
    else if (kp + T > c.cap) { bad = (int)kDevCapacity; kp = -1; }
    if (kp >= 0) {
      const int delta = (kp + T + kPage - 1) / kPage - (n_old + kPage - 1) / kPage;
      pop = delta > 0 ? delta * c.Hkv : 0;
      push = delta < 0 ? -delta * c.Hkv : 0;
    }
    s_keep[s] = kp;
    s_old[s] = n_old;
  }
  int pops, pushes;
  const int pop_off = block_excl_scan(pop, s_scan, pops);
  const int push_off = block_excl_scan(push, s_scan, pushes);
  if (s < c.batch) { s_pop[s] = pop_off; s_push[s] = push_off; }
  const bool exhausted = pops > top + pushes;
  if (blockIdx.x == 0) {
    if (bad) set_status(c, (unsigned)bad);
    if (exhausted && tid == 0) set_status(c, kDevPoolExhausted);
  }
  __syncthreads();
  // Pages that sequence q returns: of every head the same number, behind the pages that hold what stays.
  auto pages_kept = [&](int q) { return (s_keep[q] + lens.tok[q + 1] - lens.tok[q] + kPage - 1) / kPage; };
  auto pages_old = [&](int q) { return (s_old[q] + kPage - 1) / kPage; };
  auto returned = [&](int q, int i) {   // the i-th of them
    const int kept = pages_kept(q), cnt = pages_old(q) - kept, h = i / cnt;
    return __ldcg(c.pt + (size_t)seg_of(c, layer, q, h) * c.max_pages + kept + i - h * cnt);
  };
  if (!exhausted) {
    const int tasks = lens.tok[c.batch] * c.Hkv;   // (at most 2^24 x 32)
    for (int t = blockIdx.x * 8 + warp; t < tasks; t += gridDim.x * 8) {
      const int row = t / c.Hkv, h = t - row * c.Hkv;
      int lo = 0, hi = c.batch;   // the sequence of the row: the last one that starts at or before it
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (lens.tok[mid] <= row) lo = mid; else hi = mid;
      }
      const int kp_s = s_keep[lo];
      if (kp_s < 0) continue;
      const int j = row - lens.tok[lo], slot = kp_s + j, pg = slot / kPage;
      const int np_old = (s_old[lo] + kPage - 1) / kPage;
      const int grow = (kp_s + lens.tok[lo + 1] - lens.tok[lo] + kPage - 1) / kPage - np_old;
      int *ptrow = c.pt + (size_t)seg_of(c, layer, lo, h) * c.max_pages;
      int pid;
      if (pg < np_old) {
        pid = __ldcg(ptrow + pg);
      } else {
        const int x = s_pop[lo] + h * grow + pg - np_old;   // the x-th page that the call takes
        if (x < top) {
          pid = __ldcg(c.free_stack + top - 1 - x);
        } else {
          int q = 0, end = c.batch;   // the sequence that returns page x - top: the last one whose pages begin at or before it
          while (end - q > 1) {
            const int mid = (q + end) >> 1;
            if (s_push[mid] <= x - top) q = mid; else end = mid;
          }
          pid = returned(q, x - top - s_push[q]);
        }
        if (lane == 0 && (slot % kPage == 0 || j == 0)) ptrow[pg] = pid;
      }
      int32_t pdef = j;
      if (TREE && !pos) pdef = __reduce_add_sync(0xffffffffu, lane < kTreeWords ? tree_before(__ldcg(masks + (size_t)row * kTreeWords + lane), lane, j) : 0);
      if (!pos && kp_s > 0) {   // the position after the last pair that stays
        const uint8_t *prev = c.pool + (size_t)__ldcg(ptrow + (kp_s - 1) / kPage) * c.page_bytes;
        pdef = __ldcg(reinterpret_cast<const int32_t *>(meta_row(c, prev, (kp_s - 1) % kPage)) + c.F) + 1 + pdef;
      }
      const size_t at = ((size_t)row * c.Hkv + h) * c.D * 2;
      move_row<0>(c, c.pool + (size_t)pid * c.page_bytes, slot % kPage, const_cast<uint8_t *>(k) + at,
                  const_cast<uint8_t *>(v) + at, nullptr, pos ? const_cast<int32_t *>(pos) + row : nullptr, lane, pdef);
    }
  }
  __threadfence();
  __syncthreads();
  if (tid == 0) s_last = atomicAdd(&c.ctrl[CTRL_CHUNK_TICKET], 1) == (int)gridDim.x - 1;
  __syncthreads();
  if (!s_last) return;
  __threadfence();
  if (tid == 0) c.ctrl[CTRL_CHUNK_TICKET] = 0;
  if (exhausted) return;
  // Returned pages go where the taken ones came from and above (every CTA has read those entries by now); the ones that
  // would go below the stack are those that were taken again.
  for (int q = 0; q < c.batch; ++q) {
    if (s_keep[q] < 0) continue;
    const int cnt = (pages_old(q) - pages_kept(q)) * c.Hkv;
    for (int i = tid; i < cnt; i += blockDim.x) {
      const int at = top - pops + s_push[q] + i;
      if (at >= 0) c.free_stack[at] = returned(q, i);
    }
  }
  if (tid == 0) c.ctrl[CTRL_FREE_TOP] = top - pops + pushes;
  if (s < c.batch && kp >= 0) {
    const int ls = layer * c.batch + s;
    c.len[ls] = kp + T;
    if (c.hist_w && kp < n_old) {
      // Queries of rolled-back tokens leave the record (lengths seen grow along it, so they are its newest entries); a
      // record that has wrapped has lost the entries that would take their place and starts over.
      const int cnt0 = c.hist_cnt[ls];
      int cnt = cnt0;
      while (cnt > 0 && cnt > cnt0 - c.hist_w && c.hist_n[(size_t)ls * c.hist_w + (cnt - 1) % c.hist_w] > kp) --cnt;
      c.hist_cnt[ls] = (cnt < cnt0 && cnt0 > c.hist_w) ? 0 : cnt;
    }
  }
}

// ---------------------------------------------------------------- attention over the chunk
struct ChunkArgs {
  int layer, window, sinks;
  float scale, scale_log2;
  __nv_bfloat16 *out;   // [tokens][Hkv * g][D]
  float *lse;           // [tokens][Hkv * g] or null
  const uint32_t *masks;   // TREE: [tokens][kTreeWords]
  ChunkLens lens;
};

// One item as the walk hands it to the other roles: slots and pages are those of the item's segment.
struct ChunkItem {
  int kind;        // 0: no more items, 1: two query tiles, 2: one query tile
  int head, seg;
  int row0;        // packed index of the first token
  int ntok[2];     // tokens of the two tiles
  int e0;          // slots up to and with the first token's own
  int base;        // pairs ahead of the chunk's own
  int a;           // slots [0, a) are sinks
  int pa0, pa1;    // pages of the sinks ...
  int pb0, pb1;    // ... and of the rest that this CTA takes
  int part;        // -1: the whole item is here; 0 / 1: the slot for the partial result
  int w0, e1;      // outside [0, a) and [w0, e1) no token of the item sees a slot
};

// The key tiles of an item: up to TP pages each, those of the sinks first.
template <int TP>
struct ChunkTiles {
  int pa0, pa1, pb0, pb1, na, nt;
  __device__ __forceinline__ explicit ChunkTiles(const ChunkItem &x) : pa0(x.pa0), pa1(x.pa1), pb0(x.pb0), pb1(x.pb1) {
    na = (pa1 - pa0 + TP - 1) / TP;
    nt = na + (pb1 - pb0 + TP - 1) / TP;
  }
  __device__ __forceinline__ int first(int i) const { return i < na ? pa0 + TP * i : pb0 + TP * (i - na); }
  __device__ __forceinline__ int pages(int i) const { return min(TP, (i < na ? pa1 : pb1) - first(i)); }
};

template <int D>
struct ChunkSmem {
  // Tensor memory holds, per stream, S, P and O side by side (a column is 4 bytes of each of 128 rows): with P apart from S
  // the next S is multiplied as soon as the warps have read this one.  That sets the pages of a key tile (N of S, K of O):
  // D = 128 has 256 columns for 80 + 40 + 128; D = 64 would have room for 128 + 64 + 64, but a thread has not for a row's
  // 128 scores and 64 words of P: 96 + 48 + 64.
  static constexpr int kPages = D == 128 ? 5 : 6, kCols = kPages * kPage;
  static constexpr int kColP = kCols, kColO = D == 128 ? 128 : kCols + kCols / 2, kStream = 256;   // S at 0; per stream
  static_assert(kColP + kCols / 2 <= kColO && kColO + D <= kStream, "a stream's columns");
  static constexpr int kSlots = D == 128 ? 3 : 4;                 // key tiles in flight, of K and of V
  static constexpr size_t kTile = (size_t)(D / 64) * 128 * 128;   // a query tile: [D / 64][128 rows][128 B]
  static constexpr size_t kKv = (size_t)kPages * kPage * D * 2;   // a key tile: K [D / 64][rows][128 B], V [page][D / 64][16][128 B]
  static constexpr size_t kMerge = 64 * 128 * 4;
  static constexpr size_t kOffK = 2 * kTile, kOffV = kOffK + kSlots * kKv;
  static constexpr size_t kOffMerge = kOffV + kSlots * kKv;
  static constexpr size_t kOffMl = kOffMerge + kMerge;                 // (m, l) of the second stream's rows
  static constexpr size_t kOffItems = kOffMl + 128 * 8;
  static constexpr size_t kOffWlo = kOffItems + kChunkItems * sizeof(ChunkItem);   // first slot of every token's window
  static constexpr size_t kOffPos = kOffWlo + kChunkItems * 256 * 4;               // positions behind the item's first window
  static constexpr size_t kOffLen = kOffPos + 256 * 4;
  static constexpr size_t kOffBlk = kOffLen + kMaxBatch * 4;
  static constexpr size_t kOffBars = (kOffBlk + (kMaxBatch + 1) * 4 + 15) & ~(size_t)15;
  static constexpr size_t bytes() { return 1024 + kOffBars + 512; }   // (more than half an SM's: one CTA each)
};

// Pages that the tokens [j0, j1) of a chunk of T tokens may see in a segment of n pairs, from the lengths alone (a window
// of W positions holds at most W pairs): sink pages [0, sp) and pages [b0, b1).
struct ChunkRange {
  int sp, b0, b1;
  __device__ __forceinline__ int units() const { return sp + b1 - b0; }
};
__device__ __forceinline__ ChunkRange chunk_range(int n, int T, int j0, int j1, int W, int S) {
  ChunkRange r;
  const int e_first = n - T + j0 + 1, e_last = n - T + j1;
  r.b1 = (e_last + kPage - 1) / kPage;
  r.b0 = W ? max(0, e_first - W) / kPage : 0;
  r.sp = W ? (min(S, e_last) + kPage - 1) / kPage : 0;
  if (r.b0 <= r.sp) r.b0 = r.sp = 0;
  return r;
}

// Matrix descriptor of an operand whose channels run along its 128-byte rows (MN-major, 128-byte swizzle): 64 channels
// to a row, 8-row groups 1024 bytes apart along K, the next 64 channels behind the 16 rows of a page.
__device__ __forceinline__ uint64_t umma_desc_mn_sw128(uint32_t smem_addr) {
  return (uint64_t)((smem_addr & 0x3ffffu) >> 4) | ((uint64_t)(kPage * 128u >> 4) << 16) | ((uint64_t)(1024u >> 4) << 32) |
         (1ull << 46) | (2ull << 61);
}
// The multiplies of a warp that stays together: every lane comes by, the one with on != 0 issues.  (Inside a branch that
// one lane takes, every operand has to be moved to a uniform register for every instruction, and one thread then issues no
// more than a multiply per 100 cycles; guarded instructions in straight code take theirs from where they were worked out.)
__device__ __forceinline__ void umma_bf16_if(uint32_t on, uint32_t tmem_d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(tmem_d), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate), "r"(on)
      : "memory");
}
// D += A B with A (128 rows x 16, bf16, two to a column) in tensor memory.
__device__ __forceinline__ void umma_bf16_ta_if(uint32_t on, uint32_t tmem_d, uint32_t tmem_a, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
      ::"r"(tmem_d), "r"(tmem_a), "l"(bdesc), "r"(idesc), "r"(accumulate), "r"(on)
      : "memory");
}
__device__ __forceinline__ void umma_commit_if(uint32_t on, uint32_t bar) {
  asm volatile(
      "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %1, 0;\n\t"
      "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}"
      ::"r"(bar), "r"(on)
      : "memory");
}
// A value that is the same in all lanes, as the compiler can see.
__device__ __forceinline__ int uniform(int v) { return __shfl_sync(0xffffffffu, v, 0); }

__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// One page's V rows, all channels (from part part0 of the page's row): per 64 channels 16 rows of 128 bytes.
__device__ __forceinline__ void tma_page_v(uint32_t dst, const CUtensorMap *tm, int part0, int page, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
      ::"r"(dst), "l"(reinterpret_cast<uint64_t>(tm)), "r"(0), "r"(0), "r"(part0), "r"(page), "r"(bar)
      : "memory");
}
// 64 channels of the g heads x the tokens of one query tile (rows of 128 bytes, swizzled).
__device__ __forceinline__ void tma_chunk_q(uint32_t dst, const CUtensorMap *tm, int ch, int head, int tok, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
      ::"r"(dst), "l"(reinterpret_cast<uint64_t>(tm)), "r"(ch), "r"(head), "r"(tok), "r"(bar)
      : "memory");
}

// 16 columns (see tmem_ld32_issue).
__device__ __forceinline__ void tmem_ld16_issue(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
               : "r"(taddr)
               : "memory");
}
__device__ __forceinline__ void tmem_ld16_wait(uint32_t (&r)[16]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])
               :
               : "memory");
}

__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};"
               ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]),
               "r"(taddr)
               : "memory");
}
__device__ __forceinline__ void tmem_st8(uint32_t taddr, const uint32_t (&r)[8]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};"
               ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(taddr)
               : "memory");
}

// A row's scores v: P = 2^(scale v - ms) in bf16 to tensor memory at tp (`ready` comes ahead of the first store), its sum
// lt, the scores' maximum mx.
template <int TP, class Ready>
__device__ __forceinline__ void chunk_weights(const uint32_t (&v)[TP][16], float scale_log2, float ms, uint32_t tp, Ready ready, float &lt,
                                              float &mx) {
  float m4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
  float2 l2[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
  const float2 sc = make_float2(scale_log2, scale_log2), off = make_float2(-ms, -ms);
  uint32_t p[2][8];
#pragma unroll
  for (int q = 0; q < TP; ++q) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float2 z = make_float2(__uint_as_float(v[q][2 * j]), __uint_as_float(v[q][2 * j + 1]));
      float2 x = __ffma2_rn(z, sc, off);
      x.x = ex2(x.x);
      x.y = ex2(x.y);
      m4[j & 3] = max3(m4[j & 3], z.x, z.y);
      l2[j & 1] = __fadd2_rn(l2[j & 1], x);
      p[q & 1][j] = pack_bf16(x.x, x.y);
    }
    if (q == 1) {
      ready();
      tmem_st8(tp, p[0]);
    }
    if (q >= 1) tmem_st8(tp + q * 8, p[q & 1]);
  }
  mx = fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3]));
  lt = (l2[0].x + l2[0].y) + (l2[1].x + l2[1].y);
}

// A warp's wait for something that is not urgent: the thread that looks is suspended meanwhile, so that it takes no issue
// slots from the warps that compute.
__device__ __forceinline__ bool mbar_sleep_warp(uint32_t bar, uint32_t parity) {
  bool ok = true;
  if ((threadIdx.x & 31) == 0) ok = mbar_wait(bar, parity);
  return __shfl_sync(0xffffffffu, ok ? 1 : 0, 0) != 0;
}

// TREE: the chunk is a draft tree.  Its nodes see the pairs ahead of it as the tokens of a chunk do; of the tree's own pairs
// a node sees those that its mask names, up to its own.
template <int D, bool TREE>
__global__ void __launch_bounds__(kChunkThreads, 1) k_chunk_attend(Ctx c, const __grid_constant__ CUtensorMap tmk,
                                                                   const __grid_constant__ CUtensorMap tmv,
                                                                   const __grid_constant__ CUtensorMap tmq,
                                                                   const __grid_constant__ ChunkArgs a) {
  using SM = ChunkSmem<D>;
  constexpr int NS = SM::kSlots, NQ = D / 64, TP = SM::kPages;
  constexpr uint32_t PAGE_HALF = kPage * 128;
  extern __shared__ uint8_t smem_raw[];
  uint8_t *smem = reinterpret_cast<uint8_t *>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  uint8_t *Qt = smem, *Kt = smem + SM::kOffK, *Vt = smem + SM::kOffV;
  float *Mg = reinterpret_cast<float *>(smem + SM::kOffMerge);
  float2 *Ml = reinterpret_cast<float2 *>(smem + SM::kOffMl);
  ChunkItem *Items = reinterpret_cast<ChunkItem *>(smem + SM::kOffItems);
  int *Wlo = reinterpret_cast<int *>(smem + SM::kOffWlo), *Pos = reinterpret_cast<int *>(smem + SM::kOffPos);
  int *Len = reinterpret_cast<int *>(smem + SM::kOffLen), *Blk = reinterpret_cast<int *>(smem + SM::kOffBlk);
  uint64_t *bars = reinterpret_cast<uint64_t *>(smem + SM::kOffBars);
  uint64_t *k_full = bars, *k_empty = k_full + NS, *v_full = k_empty + NS, *v_empty = v_full + NS;
  uint64_t *q_full = v_empty + NS, *q_empty = q_full + 2;
  uint64_t *s_full = q_empty + 2, *s_empty = s_full + 2, *p_full = s_empty + 2, *p_empty = p_full + 2;
  uint64_t *o_full = p_empty + 2, *o_empty = o_full + 2;
  uint64_t *it_full = o_empty + 2, *it_empty = it_full + kChunkItems, *j_full = it_empty + kChunkItems, *j_empty = j_full + 1;
  uint64_t *mma_done = j_empty + 1;
  uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(mma_done + 1);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, G = c.G, TPT = kChunkRows / G;

  if (warp == 3) tmem_alloc(smem_u32(tmem_slot), 512);
  if (threadIdx.x == 0) {
    for (const CUtensorMap *tm : {&tmk, &tmv, &tmq}) asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(tm)) : "memory");
    for (int s = 0; s < NS; ++s) {
      mbar_init(smem_u32(&k_full[s]), 1); mbar_init(smem_u32(&k_empty[s]), 1);
      mbar_init(smem_u32(&v_full[s]), 1); mbar_init(smem_u32(&v_empty[s]), 1);
    }
    for (int t = 0; t < 2; ++t) {
      mbar_init(smem_u32(&q_full[t]), 1); mbar_init(smem_u32(&q_empty[t]), 1);
      mbar_init(smem_u32(&s_full[t]), 1); mbar_init(smem_u32(&s_empty[t]), 4);
      mbar_init(smem_u32(&p_full[t]), 4); mbar_init(smem_u32(&p_empty[t]), 1);
      mbar_init(smem_u32(&o_full[t]), 1); mbar_init(smem_u32(&o_empty[t]), 4);
    }
    for (int i = 0; i < kChunkItems; ++i) { mbar_init(smem_u32(&it_full[i]), 1); mbar_init(smem_u32(&it_empty[i]), 11); }
    mbar_init(smem_u32(j_full), 4); mbar_init(smem_u32(j_empty), 4);
    mbar_init(smem_u32(mma_done), 2);
    fence_barrier_init();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  griddep_wait();                          // everything below reads what earlier launches wrote
  griddep_launch();

  if (warp >= 4) {
    // ---------------- softmax: thread = query row of stream t ----------------
    const int t = (warp - 4) >> 2, quarter = warp & 3, R = quarter * 32 + lane;
    const int tok = R / G, hq = R - tok * G;
    const uint32_t trow = tmem_base + ((uint32_t)(quarter * 32) << 16);
    const uint32_t ts = trow + t * SM::kStream, tp = ts + SM::kColP, to = ts + SM::kColO;
    int it = 0;
    uint32_t sp = 0, pe = 1, op = 0, jp = 0;   // parities of s_full, p_empty, o_full and the join's barriers
    bool ok = true;
    while (ok) {
      const int ri = it % kChunkItems;
      if (!mbar_sleep_warp(smem_u32(&it_full[ri]), (it / kChunkItems) & 1)) { set_status(c, kDevWaitTimeout); break; }
      const ChunkItem &x = Items[ri];              // (let go at the item's end: registers are short here)
      const int qt = x.kind == 1 ? t : 0;          // the stream's query tile
      const int tj = qt * TPT + tok;
      const bool live = x.kind != 0 && tok < (qt ? x.ntok[1] : x.ntok[0]);
      const bool any = __any_sync(0xffffffffu, live);   // (a warp without a row in use only keeps the hand-overs going)
      const int e = live ? x.e0 + tj : INT_MAX;    // this row sees slots [0, a) and [wlo, e)
      const int wlo = live && a.window ? Wlo[ri * 256 + tj] : 0;
      ++it;
      if (x.kind == 0) break;
      const ChunkTiles<TP> tl(x);
      const int nt = tl.nt, step = x.kind, i0 = x.kind == 1 ? 0 : t;
      float m = -INFINITY, l = 0.f;
      for (int i = i0; i < nt; i += step) {
        const int p0 = tl.first(i), cols = tl.pages(i) * kPage;
        const int hi = min(cols, e - p0 * kPage), lo = wlo - p0 * kPage, na = x.a - p0 * kPage;
        const bool in_tree = TREE && p0 * kPage + cols > x.base;
        if (!mbar_sleep_warp(smem_u32(&s_full[t]), sp)) { set_status(c, kDevWaitTimeout); ok = false; break; }
        sp ^= 1;
        tc_fence_after();
        bool waited = false;
        // The products with P of the tile before: P's columns are free, and O may be rescaled.
        auto wait_products = [&]() {
          if (waited) return;
          waited = true;
          if (!mbar_sleep_warp(smem_u32(&p_empty[t]), pe)) { set_status(c, kDevWaitTimeout); ok = false; }
          pe ^= 1;
          tc_fence_after();
        };
        if (any) {
          // S into registers; from here on its columns may take the next tile's products.
          uint32_t v[TP][16];
#pragma unroll
          for (int q = 0; q < TP; ++q) tmem_ld16_issue(ts + q * 16, v[q]);
#pragma unroll
          for (int q = 0; q < TP; ++q) tmem_ld16_wait(v[q]);
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_u32(&s_empty[t]));
          if (!__all_sync(0xffffffffu, hi >= SM::kCols && (lo <= 0 || na >= SM::kCols) && !in_tree)) {   // hidden scores become -infinity
            asm volatile("" ::: "memory");   // (a branch: tiles without an edge should not pay for the comparisons)
            if constexpr (TREE) {
              // The row's seen pairs as bits: the tree's mask (ones for pairs ahead of the tree) within the range and the window.
              uint32_t see[3];
              const int at = p0 * kPage - x.base, k = at >> 5;
              const uint32_t *row = a.masks + (size_t)(x.row0 + tj) * kTreeWords;
              uint32_t w[4];
#pragma unroll
              for (int j = 0; j < 4; ++j) w[j] = !live || k + j < 0 ? ~0u : k + j < kTreeWords ? __ldcg(row + k + j) : 0u;
              auto below = [](int e) { return e <= 0 ? 0u : e >= 32 ? ~0u : (1u << e) - 1u; };   // bits under e
#pragma unroll
              for (int j = 0; j < 3; ++j)
                see[j] = __funnelshift_r(w[j], w[j + 1], at & 31) & below(hi - 32 * j) & (below(na - 32 * j) | ~below(lo - 32 * j));
#pragma unroll
              for (int q = 0; q < TP; ++q)
#pragma unroll
                for (int j = 0; j < 16; ++j)
                  if (!((see[q / 2] >> (q % 2 * 16 + j)) & 1u)) v[q][j] = 0xff800000u;
            } else {
#pragma unroll
              for (int q = 0; q < TP; ++q)
#pragma unroll
                for (int j = 0; j < 16; ++j)
                  if (q * 16 + j >= hi || (q * 16 + j < lo && q * 16 + j >= na)) v[q][j] = 0xff800000u;
            }
          }
          // P = 2^(scale s - ms) against the reference m, rounded to bf16 (as V is: at most half a step, 2^-8, off); its sum
          // is not rounded.  The maximum is found on the side: m follows it only when a score has passed m by more than 2^24
          // (or there is no m yet); then O and l are rescaled and P is worked out again.
          float mx, lt;
          chunk_weights<TP>(v, a.scale_log2, m == -INFINITY ? 0.f : m * a.scale_log2, tp, wait_products, lt, mx);
          const bool grow = mx > m && (mx - m) * a.scale_log2 > kChunkGrow;
          if (__any_sync(0xffffffffu, grow)) {
            tmem_st_wait();   // stores to tensor memory are asynchronous: P's first values land before its second ones set out
            const float f = grow ? ex2((m - mx) * a.scale_log2) : 1.f;
            if (grow) m = mx;
            l *= f;
            if (i != i0) {
#pragma unroll 1
              for (int q = 0; q < D; q += 16) {
                uint32_t o[16];
                tmem_ld16_issue(to + q, o);
                tmem_ld16_wait(o);
#pragma unroll
                for (int j = 0; j < 16; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * f);
                tmem_st16(to + q, o);
              }
            }
            chunk_weights<TP>(v, a.scale_log2, m == -INFINITY ? 0.f : m * a.scale_log2, tp, wait_products, lt, mx);
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
      if (!ok) break;
      // ---- the item's end: this stream's O is complete ----
      const bool has = i0 < nt;
      if (has) {
        if (!mbar_sleep_warp(smem_u32(&o_full[t]), op)) { set_status(c, kDevWaitTimeout); ok = false; break; }
        op ^= 1;
        tc_fence_after();
      }
      // Both streams of one query tile: where the item goes on elsewhere the merge takes both results, else they meet here.
      const bool join = x.kind == 2 && nt > 1 && x.part < 0;
      const size_t orow = ((size_t)(x.row0 + tj) * c.Hkv + x.head) * G + hq;
      const int pslot = blockIdx.x * 2 + max(x.part, 0), prow = t * kChunkRows + R;
      float f0 = 1.f, f1 = 0.f;   // weights of the two streams' results
      const bool writes = live && (x.kind == 1 || t == 0 || x.part >= 0);
      __nv_bfloat16 *out = a.out + orow * D;
      // 16 columns at a time: short calls end here, and code that runs for the first time costs more than its arithmetic.
#pragma unroll 1
      for (int q = 0; q < D; q += 16) {
        uint32_t o[16];
        if (has) {
          tmem_ld16_issue(to + q, o);
          tmem_ld16_wait(o);
        }
        if (join) {   // the second stream hands its O over, 64 columns at a time, with m and l ahead of the first
          if (q % 64 == 0) {
            if (!mbar_sleep_warp(smem_u32(t == 1 ? j_empty : j_full), t == 1 ? jp ^ 1 : jp)) { set_status(c, kDevWaitTimeout); ok = false; break; }
            jp ^= 1;
            __syncwarp();
          }
          float *mg = Mg + (q % 64) * 128 + R;
          if (t == 1) {
            if (q == 0) Ml[R] = make_float2(m, l);
#pragma unroll
            for (int j = 0; j < 16; ++j) mg[j * 128] = __uint_as_float(o[j]);
          } else {
            if (q == 0) {
              const float2 other = Ml[R];
              const float M = fmaxf(m, other.x);
              f0 = m == -INFINITY ? 0.f : ex2((m - M) * a.scale_log2);
              f1 = other.x == -INFINITY ? 0.f : ex2((other.x - M) * a.scale_log2);
              m = M;
              l = l * f0 + other.y * f1;
            }
#pragma unroll
            for (int j = 0; j < 16; ++j) o[j] = __float_as_uint(fmaf(mg[j * 128], f1, __uint_as_float(o[j]) * f0));
          }
          if (q % 64 == 48) {
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(t == 1 ? j_full : j_empty));
          }
        }
        if (!writes) continue;
        if (x.part >= 0) {
          if (has) {   // (the two layouts: see k_chunk_merge)
            const int step = x.kind == 1 ? 256 * 4 : 4;
            float *part = c.chunk_part + pslot * (256 * D) + prow * (x.kind == 1 ? 4 : D) + q / 4 * step;
#pragma unroll
            for (int j = 0; j < 4; ++j)
              __stcg(reinterpret_cast<uint4 *>(part + j * step), make_uint4(o[4 * j], o[4 * j + 1], o[4 * j + 2], o[4 * j + 3]));
          }
        } else {
          const float inv = l == 0.f ? 0.f : 1.f / l;   // a row that sees nothing gives zeros
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            uint32_t w[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) w[k] = pack_bf16(__uint_as_float(o[8 * h + 2 * k]) * inv, __uint_as_float(o[8 * h + 2 * k + 1]) * inv);
            *reinterpret_cast<uint4 *>(out + q + 8 * h) = make_uint4(w[0], w[1], w[2], w[3]);
          }
        }
      }
      if (has) {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&o_empty[t]));
      }
      if (!ok) break;
      if (writes) {
        // (a row whose scores are all NaN has found no maximum, but must not count as one that saw nothing)
        if (x.part >= 0)
          __stcg(reinterpret_cast<float2 *>(c.chunk_ml) + pslot * 256 + prow, make_float2(l != l ? 0.f : m, l));
        else if (a.lse)
          a.lse[orow] = l == 0.f ? -INFINITY : fmaf(m, a.scale, logf(l));
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&it_empty[ri]));
    }
  } else {
  if (warp == 2) {
    // ---------------- the walk over this CTA's range of the line of pages ----------------
    const int batch = c.batch, W = a.window, S = a.sinks, TB = 2 * TPT;
    for (int s = lane; s < batch; s += 32) {
      const int n = __ldcg(c.len + a.layer * batch + s);
      Len[s] = n;
      // (the host checks the lengths it knows; a replayed launch is checked here)
      if (blockIdx.x == 0 && n < a.lens.tok[s + 1] - a.lens.tok[s]) set_status(c, kDevBadIndex);
    }
    int NB = 0;   // blocks of two query tiles, over the sequences
    for (int s0 = 0; s0 < batch; s0 += 32) {
      const int s = s0 + lane;
      const int nb = s < batch ? (a.lens.tok[s + 1] - a.lens.tok[s] + TB - 1) / TB : 0;
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
    // What a page counts in the line: in batches of trees items with one query tile and with two come together, and a page takes the
    // latter half as long again (3200 cycles per key tile for 2000: two tiles are bound by products and exponentials, one by the pages'
    // way here).  16 trees of up to 64 nodes, 18 to a tile, over up to 32768 pairs: 199 us where all pages count alike, 179 at 2 : 3 (180 at
    // 5 : 7 and 5 : 8, 182 at 5 : 6, 200 at 1 : 2).  All alike and 2 : 3 on other shapes, attention back to back: 8 heads of 4 317 and 295 us,
    // 4 heads of 8 and of 4 with 64 channels 213 and 190, 138 and 123, window 4096 101 and 93; 40 trees of up to 32 over 8192 pairs 122 and 115;
    // 12 trees of up to 256 158 and 153; 16 of 64 over 8192 pairs 91 and 90.  Batches of other chunks have items with two tiles above all.
    struct Block { int s, j0, j1, n, T; ChunkRange r; int units, weight; };
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
      b.j0 = (f - Blk[lo]) * TB;
      b.j1 = min(b.T, b.j0 + TB);
      b.units = 0;
      b.weight = !TREE ? 1 : b.j1 - b.j0 > TPT ? kTreeTwo : kTreeOne;
      if (b.n >= b.T) {
        b.r = chunk_range(b.n, b.T, TREE ? 0 : b.j0, b.j1, W, S);   // (a node may be near the root whatever its place)
        b.units = b.r.units() * b.weight;
      }
      return b;
    };
    // The pages of one KV head, summed over the blocks 32 at a time; the first 32 stay at hand.
    auto strip = [&](int f0) { return f0 + lane < NB ? block(f0 + lane).units : 0; };
    const int un0 = strip(0);
    long long P = 0;
    for (int f0 = 0; f0 < NB; f0 += 32) P += __reduce_add_sync(0xffffffffu, f0 == 0 ? un0 : strip(f0));
    const long long total = P * c.Hkv;
    // (long divisions take hundreds of cycles, and the first tile waits for these)
    auto quotient = [](long long x, long long y) { return (x | y) >> 32 ? x / y : (long long)((unsigned)x / (unsigned)y); };
    const long long per = max((long long)kChunkMinPages * (TREE ? kTreeOne : 1), quotient(total + gridDim.x - 1, gridDim.x));
    long long u = per * blockIdx.x;
    const long long u_end = min(total, u + per);
    int *info = c.chunk_info + blockIdx.x * kChunkInfo;
    int head = 0, f = 0, off = 0, it = 0;
    bool open = false;   // this CTA begins an item that others go on with
    if (u < u_end) {
      head = (int)quotient(u, P);
      long long rem = u - head * P;
      for (int f0 = 0; f0 < NB; f0 += 32) {   // the block that holds page `rem`
        const int un = f0 == 0 ? un0 : strip(f0);
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
          off = (int)rem - __shfl_sync(0xffffffffu, inc - un, l);
          break;
        }
        rem -= __shfl_sync(0xffffffffu, inc, 31);
      }
    }
    bool ok = true, ended = false;
    // Hands the next item (or the end) to the other roles.
    auto publish = [&]() {
      const int ri = it % kChunkItems;
      if (!mbar_sleep_warp(smem_u32(&it_empty[ri]), ((it / kChunkItems) & 1) ^ 1)) { set_status(c, kDevWaitTimeout); ok = false; return; }
      ++it;
      ChunkItem *x = Items + ri;
      if (u >= u_end) {
        if (lane == 0) { x->kind = 0; mbar_arrive(smem_u32(&it_full[ri])); }
        __syncwarp();
        ended = true;
        return;
      }
      Block b = block(f);
      while (b.units == 0) {
        if (++f == NB) { f = 0; ++head; }
        b = block(f);
      }
      const int take = (int)min((long long)(b.units - off), u_end - u);
      const int ntok = b.j1 - b.j0, nt0 = min(ntok, TPT), seg = seg_of(c, a.layer, b.s, head), e0 = b.n - b.T + b.j0 + 1;
      const int *ptrow = c.pt + (size_t)seg * c.max_pages;
      // This CTA's pages of the item: [pa0, pa1) at the front, [pb0, pb1) behind; with a window, less the pages that the
      // stored positions show to be hidden from every token.
      // (a cut inside a page: the page is the CTA's that has its beginning)
      auto page_at = [&](int o) { return !TREE ? o : (int)((unsigned)(o + b.weight - 1) / (unsigned)b.weight); };
      const int o0 = page_at(off), o1 = page_at(off + take);
      int pa0 = min(o0, b.r.sp), pa1 = min(o1, b.r.sp);
      int pb0 = b.r.b0 + max(o0 - b.r.sp, 0), pb1 = b.r.b0 + max(o1 - b.r.sp, 0);
      int na = 0, first = 0;
      if (TREE && W) {
        const int base = b.n - b.T;
        // A node's window ends with its own pair and holds its ancestors, all of them (W is at least the number of nodes); where
        // it begins ahead of the tree follows from its position: first the lowest one's, then the others' as below.
        na = S ? slot_sinks(c, ptrow, base, S) : 0;
        int low = INT_MAX;
        for (int i = lane; i < ntok; i += 32) low = min(low, slot_pos(c, ptrow, e0 - 1 + i));
        low = __reduce_min_sync(0xffffffffu, low);
        const int lo0 = max(0, base + 1 - W), start = window_start(low, W);
        first = lo0 >= base ? base : slot_pos(c, ptrow, lo0) >= start ? lo0 : slot_lower_bound_warp(c, ptrow, lo0 + 1, base, start);
        __syncwarp();
        for (int i = lane; i < 256 && first + i < base; i += 32) Pos[i] = slot_pos(c, ptrow, first + i);
        __syncwarp();
        for (int i = lane; i < ntok; i += 32) {
          const int p = slot_pos(c, ptrow, e0 - 1 + i), from = window_start(p, W);
          int lo = first, hi = (int)min((long long)base, first + (long long)p - low);
          if (hi - first < 256) {
            while (lo < hi) {
              const int mid = (lo + hi) >> 1;
              if (Pos[mid - first] < from) lo = mid + 1; else hi = mid;
            }
          } else {
            lo = slot_lower_bound(c, ptrow, lo, hi, from);
          }
          Wlo[ri * 256 + i] = lo;
        }
      } else if (W) {
        na = S ? slot_sinks(c, ptrow, b.n, S) : 0;
        // Where the first token's window begins, then the others': a window that begins d positions later begins at most d
        // slots later, so the positions of those slots decide, read together (a search of its own for a token whose
        // window is further off: a chunk with gaps in its positions).
        const int p_first = slot_pos(c, ptrow, e0 - 1), lo0 = max(0, e0 - W), start = window_start(p_first, W);
        first = slot_pos(c, ptrow, lo0) >= start ? lo0 : slot_lower_bound_warp(c, ptrow, lo0 + 1, e0, start);
        __syncwarp();
        for (int i = lane; i < 256 && first + i < b.n; i += 32) Pos[i] = slot_pos(c, ptrow, first + i);
        __syncwarp();
        for (int i = lane; i < ntok; i += 32) {
          const int last = e0 + i - 1, p = slot_pos(c, ptrow, last);
          const long long apart = (long long)p - p_first;   // (>= 0)
          const int from = window_start(p, W);
          int lo = first, hi = (int)min((long long)last, first + apart);
          if (hi - first < 256) {
            while (lo < hi) {
              const int mid = (lo + hi) >> 1;
              if (Pos[mid - first] < from) lo = mid + 1; else hi = mid;
            }
          } else {
            lo = slot_lower_bound(c, ptrow, lo, hi, from);
          }
          Wlo[ri * 256 + i] = lo;
        }
      }
      if (W) {
        const int a16 = (na + kPage - 1) / kPage, w16 = first / kPage;
        if (b.r.sp == 0) {   // one run of pages: split it around the hidden ones
          pa0 = pb0;
          pa1 = max(pa0, min(pb1, a16));
          pb0 = min(pb1, max(pb0, max(a16, w16)));
        } else {
          pa1 = max(pa0, min(pa1, a16));
          pb0 = min(pb1, max(pb0, w16));
        }
      }
      // Whole, or cut by an end of this CTA's range: then its part goes to slot 1 if the item begins here, else to slot 0.
      const bool begins = u - off >= per * blockIdx.x, ends = off + take == b.units;
      const int part = begins ? (ends ? -1 : 1) : 0;
      if (lane == 0) {
        x->kind = ntok > nt0 ? 1 : 2;
        x->head = head; x->seg = seg;
        x->row0 = a.lens.tok[b.s] + b.j0;
        x->ntok[0] = nt0; x->ntok[1] = ntok - nt0;
        x->e0 = e0; x->base = b.n - b.T; x->a = na; x->w0 = first; x->e1 = e0 + ntok - 1;
        x->pa0 = pa0; x->pa1 = pa1; x->pb0 = pb0; x->pb1 = pb1;
        x->part = part;
        if (part == 1) {   // for the merge, with the last CTA that the item reaches
          info[0] = (int)quotient(u - off + b.units - 1, per);
          info[1] = head; info[2] = x->row0; info[3] = nt0; info[4] = ntok - nt0;   // (no second tile: two streams of one)
        }
      }
      if (part == 1) open = true;
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&it_full[ri]));
      u += take;
      off = 0;
      if (++f == NB) { f = 0; ++head; }
    };
    // V of an item, one item behind the walk.
    FeatRing rr{0, 0};
    uint32_t armed = 0, armed_par = 0;    // bit s: slot s has been armed / its last parity
    publish();
    for (int vi = 0; ok; ++vi) {
      if (!ended) publish();
      const ChunkItem &x = Items[vi % kChunkItems];
      if (!ok || x.kind == 0) break;
      const ChunkTiles<TP> tl(x);
      const int *ptrow = c.pt + (size_t)x.seg * c.max_pages;
      auto page_id = [&](int i) { return i < tl.nt && (lane & 7) < tl.pages(i) ? __ldcg(ptrow + tl.first(i) + (lane & 7)) : 0; };
      int id = page_id(0);
      for (int i = 0; i < tl.nt; ++i) {
        const int idn = page_id(i + 1), np = tl.pages(i);
        if (!mbar_sleep_warp(smem_u32(&v_empty[rr.i]), rr.ph ^ 1)) { set_status(c, kDevWaitTimeout); ok = false; break; }
        const uint32_t bar = smem_u32(&v_full[rr.i]);
        if (lane == 0) mbar_arrive_expect_tx(bar, (uint32_t)(np * NQ) * PAGE_HALF);
        armed |= 1u << rr.i;
        armed_par = (armed_par & ~(1u << rr.i)) | ((uint32_t)rr.ph << rr.i);
        __syncwarp();
        if (lane < np) tma_page_v(smem_u32(Vt + rr.i * SM::kKv + (size_t)lane * NQ * PAGE_HALF), &tmv, NQ, id, bar);
        rr.next(NS);
        id = idn;
      }
    }
    if (!open && lane == 0) info[0] = -1;
#pragma unroll
    for (int s = 0; s < NS; ++s)   // no copy may be in flight at the exit
      if (((armed >> s) & 1u) && !mbar_sleep_warp(smem_u32(&v_full[s]), (armed_par >> s) & 1u)) set_status(c, kDevWaitTimeout);
  } else if (warp == 0) {
    // ---------------- copies of the query tiles and of K ----------------
    FeatRing rr{0, 0};
    int it = 0;
    uint32_t qp = 0;                      // bit t: parity of query tile t's next phase
    uint32_t armed = 0, armed_par = 0;    // bit s: ring slot s (bit 16 + t: query tile t) has been armed / its last parity
    bool ok = true;
    const int pg = lane & 7, half = lane >> 3;
    while (ok) {
      const int ri = it % kChunkItems;
      if (!mbar_sleep_warp(smem_u32(&it_full[ri]), (it / kChunkItems) & 1)) { set_status(c, kDevWaitTimeout); break; }
      const ChunkItem x = Items[ri];
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&it_empty[ri]));
      ++it;
      if (x.kind == 0) break;
      const ChunkTiles<TP> tl(x);
      if (tl.nt == 0) continue;
      for (int t = 0; t < (x.kind == 1 ? 2 : 1) && ok; ++t) {
        if (!mbar_sleep_warp(smem_u32(&q_empty[t]), ((qp >> t) & 1) ^ 1)) { set_status(c, kDevWaitTimeout); ok = false; break; }
        if (lane == 0) {
          mbar_arrive_expect_tx(smem_u32(&q_full[t]), (uint32_t)(NQ * TPT * G * 128));
          for (int q = 0; q < NQ; ++q)
            tma_chunk_q(smem_u32(Qt + t * SM::kTile + (size_t)q * 128 * 128), &tmq, q * 64, x.head * G, x.row0 + t * TPT,
                        smem_u32(&q_full[t]));
        }
        armed |= 1u << (16 + t);
        armed_par = (armed_par & ~(1u << (16 + t))) | (((qp >> t) & 1) << (16 + t));
        qp ^= 1u << t;
      }
      if (!ok) break;
      const int *ptrow = c.pt + (size_t)x.seg * c.max_pages;
      auto page_id = [&](int i) { return i < tl.nt && pg < tl.pages(i) ? __ldcg(ptrow + tl.first(i) + pg) : 0; };
      int id = page_id(0);
      for (int i = 0; i < tl.nt; ++i) {   // a lane per copy: page pg, 64 channels
        const int idn = page_id(i + 1), np = tl.pages(i);
        if (!mbar_sleep_warp(smem_u32(&k_empty[rr.i]), rr.ph ^ 1)) { set_status(c, kDevWaitTimeout); ok = false; break; }
        const uint32_t bar = smem_u32(&k_full[rr.i]);
        if (lane == 0) mbar_arrive_expect_tx(bar, (uint32_t)(np * NQ) * PAGE_HALF);
        armed |= 1u << rr.i;
        armed_par = (armed_par & ~(1u << rr.i)) | ((uint32_t)rr.ph << rr.i);
        __syncwarp();
        if (pg < np && half < NQ)
          tma_page_k(smem_u32(Kt + rr.i * SM::kKv + (size_t)half * TP * PAGE_HALF + (size_t)pg * PAGE_HALF), &tmk, half, id, bar);
        rr.next(NS);
        id = idn;
      }
    }
    // No copy may be in flight at the exit.
#pragma unroll
    for (int s = 0; s < NS; ++s)
      if (((armed >> s) & 1u) && !mbar_sleep_warp(smem_u32(&k_full[s]), (armed_par >> s) & 1u)) set_status(c, kDevWaitTimeout);
#pragma unroll
    for (int t = 0; t < 2; ++t)
      if (((armed >> (16 + t)) & 1u) && !mbar_sleep_warp(smem_u32(&q_full[t]), (armed_par >> (16 + t)) & 1u)) set_status(c, kDevWaitTimeout);
  } else if (warp == 1 || warp == 3) {
    // ---------------- multiplies: one warp S = Q K^T, the other O += P V, for both streams; a warp stays together, lane 0
    // issues.  (One warp for both kinds spends longer on its waits and hand-overs than the tensor core on the products.)
    const bool scores = warp == 1;
    const uint32_t on = lane == 0;
    FeatRing r{0, 0};
    int it = 0;
    uint32_t qp = 0, se = 3, pp = 0, op = 3;   // bit t: parities of query tile t's next phase, of stream t's next s_empty, p_full, o_empty
    bool ok = true;
    const uint32_t tb = uniform(tmem_base);
    const uint32_t idesc_o = umma_idesc_bf16(kChunkRows, D) | (1u << 16);   // B runs along N
    uint64_t *full = scores ? k_full : v_full, *empty = scores ? k_empty : v_empty;
    while (ok) {
      const int ri = it % kChunkItems;
      if (!mbar_wait(smem_u32(&it_full[ri]), (it / kChunkItems) & 1)) { set_status(c, kDevWaitTimeout); break; }
      const ChunkItem x = Items[ri];
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&it_empty[ri]));
      ++it;
      if (x.kind == 0) break;
      const ChunkTiles<TP> tl(x);
      const int nt = uniform(tl.nt), step = uniform(x.kind);   // step: key tiles between a stream's tile and its next one
      if (nt == 0) continue;
      if (scores)
        for (int t = 0; t < (step == 1 ? 2 : 1); ++t) {
          if (!mbar_wait(smem_u32(&q_full[t]), (qp >> t) & 1)) { set_status(c, kDevWaitTimeout); ok = false; }
          qp ^= 1u << t;
        }
      for (int i = 0; i < nt && ok; ++i) {
        const int np = uniform(tl.pages(i)), slot = uniform(r.i);
        if (!mbar_wait(smem_u32(&full[slot]), r.ph)) { set_status(c, kDevWaitTimeout); ok = false; break; }
        r.next(NS);
        const int t0 = step == 1 ? 0 : i & 1, t1 = step == 1 ? 2 : t0 + 1;
        if (scores) {
          const uint64_t kd = umma_desc_sw128(smem_u32(Kt + slot * SM::kKv));
          const uint32_t idesc = umma_idesc_bf16(kChunkRows, np * kPage);
          for (int t = t0; t < t1; ++t) {   // as soon as the warps have read the S before
            const uint64_t qd = umma_desc_sw128(smem_u32(Qt + (step == 1 ? t : 0) * SM::kTile));
            const uint32_t ts = tb + t * SM::kStream;
            if (!__all_sync(0xffffffffu, mbar_wait(smem_u32(&s_empty[t]), (se >> t) & 1))) { set_status(c, kDevWaitTimeout); ok = false; break; }
            se ^= 1u << t;
            tc_fence_after();
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks)
              umma_bf16_if(on, ts, qd + (uint64_t)(((ks >> 2) * 128 * 128 + (ks & 3) * 32) >> 4),
                           kd + (uint64_t)(((ks >> 2) * TP * (int)PAGE_HALF + (ks & 3) * 32) >> 4), idesc, ks > 0);
            umma_commit_if(on, smem_u32(&s_full[t]));
          }
        } else {
          // Rows that no token of the item sees (pairs outside every window; past the segment's end whatever the page held
          // before) are cleared: P is zero there, but zero times an infinity is not.
          const int s0 = tl.first(i) * kPage, s1 = s0 + np * kPage;
          if (!((s0 >= x.w0 && s1 <= x.e1) || s1 <= min(x.a, x.e1))) {
            for (int e = lane; e < np * kPage * NQ * 8; e += 32) {
              const int row = e / (NQ * 8), ch = e % (NQ * 8), at = s0 + row;
              if (at < x.e1 && (at < x.a || at >= x.w0)) continue;
              *reinterpret_cast<uint4 *>(Vt + slot * SM::kKv + (size_t)((row / kPage * NQ + (ch >> 3)) * kPage + row % kPage) * 128 +
                                         (ch & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
            }
            fence_proxy_async();
            __syncwarp();
          }
          const uint64_t vd = umma_desc_mn_sw128(smem_u32(Vt + slot * SM::kKv));
          const bool first = i < step;   // the stream's first tile of the item
          for (int t = t0; t < t1; ++t) {
            const uint32_t ts = tb + t * SM::kStream, tp = ts + SM::kColP, to = ts + SM::kColO;
            if (first) {
              if (!mbar_wait(smem_u32(&o_empty[t]), (op >> t) & 1)) { set_status(c, kDevWaitTimeout); ok = false; break; }
              op ^= 1u << t;
            }
            if (!__all_sync(0xffffffffu, mbar_wait(smem_u32(&p_full[t]), (pp >> t) & 1))) { set_status(c, kDevWaitTimeout); ok = false; break; }
            pp ^= 1u << t;
            tc_fence_after();
            umma_bf16_ta_if(on, to, tp, vd, idesc_o, !first);
            if (np == TP) {
#pragma unroll
              for (int ks = 1; ks < TP; ++ks) umma_bf16_ta_if(on, to, tp + ks * 8, vd + (uint64_t)((ks * NQ * PAGE_HALF) >> 4), idesc_o, 1);
            } else {
              for (int ks = 1; ks < np; ++ks) umma_bf16_ta_if(on, to, tp + ks * 8, vd + (uint64_t)((ks * NQ * PAGE_HALF) >> 4), idesc_o, 1);
            }
            umma_commit_if(on, smem_u32(&p_empty[t]));
            if (i + step >= nt) umma_commit_if(on, smem_u32(&o_full[t]));
          }
        }
        if (ok) umma_commit_if(on, smem_u32(&empty[slot]));
      }
      if (scores && ok) {
        umma_commit_if(on, smem_u32(&q_empty[0]));
        if (step == 1) umma_commit_if(on, smem_u32(&q_empty[1]));
      }
    }
    umma_commit_if(on, smem_u32(mma_done));   // nothing may be in flight when tensor memory is freed
    if (!mbar_wait(smem_u32(mma_done), 0)) set_status(c, kDevWaitTimeout);
  }
  }
  // ---- common exit ----
  tc_fence_before();
  __syncthreads();
  if (warp == 3) tmem_dealloc(tmem_base, 512);
}

// Joins the partial results of the items that cuts go through: grid (CTAs of the attention launch, row groups).  CTA x
// looks after the item that CTA x of the attention left open: its own part, and those of the CTAs up to the last one that
// the item reached.  Items come in two forms:
//   two query tiles (more than 128 rows, a few parts).  A thread of the attention has a row, and 32 rows of 512 bytes are 32
//   lines to a store (9000 cycles for an item's end, 4000 like this): a slot holds [D / 4][256 rows][4 channels], and a warp
//   here takes 8 rows x 16 channels.  (256 tokens at 8K: 65 us for both kernels with the form below, 59 with this one.)
//   one query tile (few rows, with drafts over a long cache in many parts; both streams leave one).  A slot holds [256
//   rows][D], and a warp here takes a row.  (5 drafts at 8K: 27 us for both kernels with the form above, 25 with this one.)
// SHORT: a launch whose items all have one tile has no code for the other form (with it, that takes 1.7 us longer).
// A part that saw nothing of a row may not have been written: whatever was read counts for nothing.
template <int D, bool SHORT>
__global__ void __launch_bounds__(256) k_chunk_merge(Ctx c, const __grid_constant__ ChunkArgs a) {
  griddep_wait();
  griddep_launch();
  const int *info = c.chunk_info + blockIdx.x * kChunkInfo;
  const int cl = __ldcg(info);
  if (cl < 0) return;
  const int cf = blockIdx.x, head = __ldcg(info + 1), row0 = __ldcg(info + 2), G = c.G, TPT = kChunkRows / G;
  const int nt0 = __ldcg(info + 3), ntok = nt0 + __ldcg(info + 4), lane = threadIdx.x & 31, warp = threadIdx.x >> 5, rows = ntok * G;
  // Slot 1 of CTA cf, then slots 0 of the CTAs behind it.
  const float *part = c.chunk_part + (size_t)(2 * cf + 1) * 256 * D;
  const float2 *ml = reinterpret_cast<const float2 *>(c.chunk_ml) + (2 * cf + 1) * 256;
  auto slot_of = [](int cta) { return 2 * cta - (cta > 0 ? 1 : 0); };
  if (SHORT || ntok == nt0) {
    const int parts = (cl + 1 - cf) * 2;   // part p: of CTA cf + p / 2 and stream p % 2
    for (int r = blockIdx.y * 8 + warp; r < rows; r += gridDim.y * 8) {
      auto row_of = [&](int p) { return slot_of(p >> 1) * 256 + (p & 1) * kChunkRows + r; };
      // Statistics of 32 parts, one per lane, and the rows of the first eight are asked for together: one round trip to L2 for
      // most items.
      auto row = [&](int p, float (&w)[D / 32]) {
        const float *o = part + row_of(p) * D + lane * (D / 32);
        if (D == 128) {
          const float4 x4 = __ldcg(reinterpret_cast<const float4 *>(o));
          w[0] = x4.x; w[1] = x4.y; w[D / 32 - 2] = x4.z; w[D / 32 - 1] = x4.w;
        } else {
          const float2 x2 = __ldcg(reinterpret_cast<const float2 *>(o));
          w[0] = x2.x; w[1] = x2.y;
        }
      };
      auto stats = [&](int p) { return p < parts ? __ldcg(ml + row_of(p)) : make_float2(-INFINITY, 0.f); };
      float2 x = stats(lane);
      float w[8][D / 32];
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i < parts) row(i, w[i]);
      float M = x.x, L = 0.f;
      for (int p = 32 + lane; p < parts; p += 32) M = fmaxf(M, stats(p).x);
#pragma unroll
      for (int o = 16; o >= 1; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
      float acc[D / 32];
#pragma unroll
      for (int j = 0; j < D / 32; ++j) acc[j] = 0.f;
      for (int p0 = 0; p0 < parts; p0 += 8) {
        if (p0 > 0) {
          if (p0 % 32 == 0) x = stats(p0 + lane);
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (p0 + i < parts) row(p0 + i, w[i]);
        }
        const float f = x.x == -INFINITY ? 0.f : ex2((x.x - M) * a.scale_log2);
        if (p0 % 32 == 0) L += f * x.y;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float fi = __shfl_sync(0xffffffffu, f, (p0 + i) & 31);
          const bool on = p0 + i < parts && fi != 0.f;
#pragma unroll
          for (int j = 0; j < D / 32; ++j) acc[j] = on ? fmaf(fi, w[i][j], acc[j]) : acc[j];
        }
      }
#pragma unroll
      for (int o = 16; o >= 1; o >>= 1) L += __shfl_xor_sync(0xffffffffu, L, o);
      const float inv = L == 0.f ? 0.f : 1.f / L;
      const size_t orow = ((size_t)(row0 + r / G) * c.Hkv + head) * G + r % G;
      uint32_t *dst = reinterpret_cast<uint32_t *>(a.out + orow * D) + lane * (D / 64);
      dst[0] = pack_bf16(acc[0] * inv, acc[1] * inv);
      if (D == 128) dst[1] = pack_bf16(acc[D / 32 - 2] * inv, acc[D / 32 - 1] * inv);
      if (a.lse && lane == 0) a.lse[orow] = L == 0.f ? -INFINITY : fmaf(M, a.scale, logf(L));
    }
    return;
  }
  const int parts = cl + 1 - cf;
  for (int u = blockIdx.y * 8 + warp; u < (rows + 7) / 8 * (D / 16); u += gridDim.y * 8) {
    const int r = u / (D / 16) * 8 + (lane >> 2), ch = u % (D / 16) * 4 + (lane & 3);   // a lane: 4 channels of a row
    const int tj = r / G, hq = r - tj * G;
    const int prow = tj < nt0 ? r : kChunkRows + (tj - TPT) * G + hq;   // row inside a slot
    const float *o = part + (ch * 256 + prow) * 4;
    float M = -INFINITY, L = 0.f, acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
    for (int p0 = 0; p0 < parts; p0 += 8) {   // eight parts are asked for together
      float2 x[8];
      float4 w[8];
      float Mn = M;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[i] = make_float2(-INFINITY, 0.f);
        if (p0 + i < parts && r < rows) {
          x[i] = __ldcg(ml + slot_of(p0 + i) * 256 + prow);
          w[i] = __ldcg(reinterpret_cast<const float4 *>(o + slot_of(p0 + i) * (256 * D)));
        }
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) Mn = fmaxf(Mn, x[i].x);
      const float f0 = M == -INFINITY ? 0.f : ex2((M - Mn) * a.scale_log2);
      M = Mn;
      L *= f0;
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[j] *= f0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (x[i].x == -INFINITY) continue;
        const float f = ex2((x[i].x - M) * a.scale_log2);
        L = fmaf(f, x[i].y, L);
        acc[0] = fmaf(f, w[i].x, acc[0]);
        acc[1] = fmaf(f, w[i].y, acc[1]);
        acc[2] = fmaf(f, w[i].z, acc[2]);
        acc[3] = fmaf(f, w[i].w, acc[3]);
      }
    }
    if (r >= rows) continue;
    const float inv = L == 0.f ? 0.f : 1.f / L;
    const size_t orow = ((size_t)(row0 + tj) * c.Hkv + head) * G + hq;
    *reinterpret_cast<uint2 *>(a.out + orow * D + ch * 4) = make_uint2(pack_bf16(acc[0] * inv, acc[1] * inv), pack_bf16(acc[2] * inv, acc[3] * inv));
    if (a.lse && ch == 0) a.lse[orow] = L == 0.f ? -INFINITY : fmaf(M, a.scale, logf(L));
  }
}

}  // namespace fkv
