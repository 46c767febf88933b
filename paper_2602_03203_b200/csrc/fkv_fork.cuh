// Kernel 12: every sequence becomes what another one was (fkv_fork), in all layers at once.  Pages hold attention features that
// each sequence updates for itself, so two sequences never share one: a copy is a copy of the pages.  A sequence that goes away
// while others become what it was hands its pages to one of them: beams that only change places move page tables.
//   k_fork_plan     the copies' pages, taken from the free stack and, behind those, from the sequences that go away: one CTA, or (up to 512
//                   sequences times layers) at the head of k_fork_copy, where every CTA works it out for itself;
//   k_fork_copy     pages: a warp takes a run of source pages, reads each once and writes up to eight copies (more: it reads again);
//                   new page tables are written aside, since the old ones are being read;
//   k_fork_commit   tables, lengths and budgets; pages of the sequences that went away return to the stack;
//   k_fork_record   the decode queries on record, if there is a record: the host's list of copies, element by element, so that
//                   a cycle needs one register as the place aside.
// Bound: bytes: every source page read once, every copy written once.  8192 pairs of 8 heads in two layers to three copies (80 MB read, 240
// written) 62.9 us back to back = 5.1 TB/s, 8 of them the latency of two dependent launches (what a small fork takes; 11 with a launch for the
// plan); writing 240 MB alone takes 37.  The copy through registers, a warp per page, took 81.
// Pages handed over (every sequence takes another's place): 16 sequences of 4096 pairs, 4 heads 16 us, with 8 heads in 32 layers 43, 4 of 8192 with
// 8 heads in two layers 38: bound by latency, a warp moving the tables of all heads of a (layer, sequence) one after another.
#pragma once
#include "fkv_dev.cuh"
#include "fkv_attend.cuh"

namespace fkv {

enum : unsigned char { FORK_CHANGES = 1, FORK_MOVES = 2, FORK_FREED = 4 };
struct ForkMap {
  short from[kMaxBatch];    // -1: empty
  short first[kMaxBatch];   // the first sequence that gets a copy of this one's pages (-1: none) ...
  short next[kMaxBatch];    // ... and the next one that gets a copy of the same
  unsigned char what[kMaxBatch];
};
// Copies dst <- src in order; kForkAside is a register.
constexpr int kForkAside = kMaxBatch;
struct ForkOps {
  int n;
  short dst[kMaxBatch * 3 / 2], src[kMaxBatch * 3 / 2];
  unsigned char emptied[kMaxBatch];
};
// planhdr: PH_NWORK = source pages to read, PH_NEW_PAGES, PH_OLD_PAGES = pages taken and returned, PH_PUSH_START = the stack's top before, or
// -1 where there are too few pages.  Per (layer, sequence): work = offset of its pages among those taken, tile1_start = among those returned,
// idx[0 ..] = new length, idx[L batch ..] = offset of its pages among the source pages, idx[2 L batch ..] = old length.

struct ForkTotals {
  int units, taken, returned, top;   // top: PH_PUSH_START
};
// By a whole CTA (a multiple of 32 threads, up to 1024).  put(entry, its pages among those taken, among those returned, among the source
// pages, new length, old length).
template <class Put>
__device__ __forceinline__ ForkTotals fork_plan(const Ctx &c, const ForkMap &m, int *s_scan, unsigned long long *s_need, Put put) {
  const int LB = c.L * c.batch, top = __ldcg(c.ctrl + CTRL_FREE_TOP);
  ForkTotals t{0, 0, 0, top};
  if (threadIdx.x == 0) *s_need = 0;
  __syncthreads();
  for (int base = 0; base < LB; base += blockDim.x) {
    const int i = base + threadIdx.x;
    int need = 0, gone = 0, read = 0, len = 0, n = 0;
    if (i < LB) {
      const int s = i % c.batch, l0 = i - s, what = m.what[s], r = m.from[s];
      n = __ldcg(c.len + i);
      len = r < 0 ? 0 : __ldcg(c.len + l0 + r);
      if ((what & FORK_CHANGES) && !(what & FORK_MOVES)) need = (len + kPage - 1) / kPage * c.Hkv;
      if (what & FORK_FREED) gone = (n + kPage - 1) / kPage * c.Hkv;
      if (m.first[s] >= 0) read = (n + kPage - 1) / kPage * c.Hkv;
      if (need) atomicAdd(s_need, (unsigned long long)need);
    }
    int tot;
    const int a = t.taken + block_excl_scan(need, s_scan, tot); t.taken += tot;
    const int b = t.returned + block_excl_scan(gone, s_scan, tot); t.returned += tot;
    const int u = t.units + block_excl_scan(read, s_scan, tot); t.units += tot;
    if (i < LB) put(i, a, b, u, len, n);
  }
  __syncthreads();
  if (*s_need > (unsigned long long)top + t.returned) t.top = -1;   // (the sums above may have wrapped then)
  return t;
}
// One thread writes what the kernels behind go by.
__device__ __forceinline__ void fork_header(const Ctx &c, const ForkTotals &t) {
  if (t.top < 0) set_status(c, kDevPoolExhausted);
  c.planhdr[PH_NWORK] = t.units;
  c.planhdr[PH_NEW_PAGES] = t.taken;
  c.planhdr[PH_OLD_PAGES] = t.returned;
  c.planhdr[PH_PUSH_START] = t.top;
}
__device__ __forceinline__ void fork_put(const Ctx &c, int LB, int i, int a, int b, int u, int len, int n) {
  c.work[i] = a;
  c.tile1_start[i] = b;
  c.idx[i] = len;
  c.idx[LB + i] = u;
  c.idx[2 * LB + i] = n;
}

__global__ void __launch_bounds__(1024) k_fork_plan(Ctx c, const __grid_constant__ ForkMap m) {
  __shared__ int s_scan[33];
  __shared__ unsigned long long s_need;
  griddep_wait();
  griddep_launch();
  const int LB = c.L * c.batch;
  const ForkTotals t = fork_plan(c, m, s_scan, &s_need, [&](int i, int a, int b, int u, int len, int n) { fork_put(c, LB, i, a, b, u, len, n); });
  if (threadIdx.x == 0) fork_header(c, t);
}

// The entry (layer, sequence) whose range of `offsets` holds x: the last one that begins at or before it (by a whole warp).
template <class Offsets>
__device__ __forceinline__ int fork_entry(Offsets offsets, int LB, int x) {
  const int lane = threadIdx.x & 31;
  int lo = 0, hi = LB;   // offsets[lo] <= x, and offsets[hi] > x if hi < LB
  while (hi - lo > 1) {
    const int step = (hi - lo + 31) / 32, at = lo + (lane + 1) * step;
    const int k = __popc(__ballot_sync(0xffffffffu, at < hi && offsets(min(at, hi - 1)) <= x));
    const int l = lo;
    lo = l + k * step;
    hi = min(hi, l + (k + 1) * step);
  }
  return lo;
}

constexpr int kForkMaxWarps = 16, kForkGroup = 8, kForkOwn = 512;

__device__ __forceinline__ void cp_bulk_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
// Shared memory -> global, both 16-byte aligned, size a multiple of 16; completion by the issuing thread's groups.
__device__ __forceinline__ void bulk_s2g_hint(void *dst, uint32_t src, uint32_t bytes, uint64_t pol) {
  asm volatile("cp.async.bulk.global.shared::cta.bulk_group.L2::cache_hint [%0], [%1], %2, %3;" ::"l"(dst), "r"(src), "r"(bytes), "l"(pol) : "memory");
}

// One CTA per SM; a warp has two page buffers in shared memory and moves a run of source pages through them by bulk copies: a page
// is read while the one before it is written, to all its copies (up to eight; it is read again for more).
// OWN: up to kForkOwn entries (layer, sequence) every CTA works the plan out for itself: one launch fewer.
template <bool OWN>
__global__ void __launch_bounds__(kForkMaxWarps * 32) k_fork_copy(Ctx c, const __grid_constant__ ForkMap m) {
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ uint64_t bars[kForkMaxWarps][2];
  __shared__ int s_taken[OWN ? kForkOwn : 1], s_returned[OWN ? kForkOwn : 1], s_units[OWN ? kForkOwn : 1], s_scan[33];
  __shared__ unsigned long long s_need;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, nw = blockDim.x / 32, warps = gridDim.x * nw, w = warp * gridDim.x + blockIdx.x;
  if (lane == 0) {
    mbar_init(smem_u32(&bars[warp][0]), 1);
    mbar_init(smem_u32(&bars[warp][1]), 1);
    fence_barrier_init();
    fence_proxy_async();
  }
  __syncwarp();
  griddep_wait();
  griddep_launch();
  const int LB = c.L * c.batch;
  int top, units;
  if constexpr (OWN) {
    const ForkTotals t = fork_plan(c, m, s_scan, &s_need, [&](int i, int a, int b, int u, int len, int n) {
      s_taken[i] = a;
      s_returned[i] = b;
      s_units[i] = u;
      if (blockIdx.x == 0) fork_put(c, LB, i, a, b, u, len, n);   // (for k_fork_commit)
    });
    if (blockIdx.x == 0 && threadIdx.x == 0) fork_header(c, t);
    top = t.top;
    units = t.units;
  } else {
    top = __ldcg(c.planhdr + PH_PUSH_START);
    units = __ldcg(c.planhdr + PH_NWORK);
  }
  if (top < 0) return;
  const int *at_taken = OWN ? s_taken : c.work, *at_returned = OWN ? s_returned : c.tile1_start, *at_units = OWN ? s_units : c.idx + LB;
  auto entry = [](const int *p) {
    if constexpr (OWN) return *p; else return __ldcg(p);
  };
  auto taken_at = [&](int i) { return entry(at_taken + i); };
  auto returned_at = [&](int i) { return entry(at_returned + i); };
  auto units_at = [&](int i) { return entry(at_units + i); };
  // Page tables that move.
  for (int i = w; i < LB; i += warps) {
    const int s = i % c.batch;
    if (!(m.what[s] & FORK_MOVES)) continue;
    const int src = i - s + m.from[s], pages = (__ldcg(c.len + src) + kPage - 1) / kPage;
    for (int h = 0; h < c.Hkv; ++h)
      for (int j = lane; j < pages; j += 32)
        c.pt_new[((size_t)i * c.Hkv + h) * c.max_pages + j] = __ldcg(c.pt + ((size_t)src * c.Hkv + h) * c.max_pages + j);
  }
  // Copies: this warp's run of source pages.
  int u = (int)((long long)units * w / warps);
  const int u_end = (int)((long long)units * (w + 1) / warps);
  if (u >= u_end) return;
  int e = fork_entry(units_at, LB, u);
  // The x-th page that the call takes: from the stack's top down, then the ones that go away.
  auto page_of = [&](int x) {
    if (x < top) return __ldcg(c.free_stack + top - 1 - x);
    int lo = 0, hi = LB;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (returned_at(mid) <= x - top) lo = mid; else hi = mid;
    }
    const int pages = (__ldcg(c.len + lo) + kPage - 1) / kPage, i = x - top - returned_at(lo), h = i / pages;
    return __ldcg(c.pt + ((size_t)lo * c.Hkv + h) * c.max_pages + i - h * pages);
  };
  const uint32_t buf = smem_u32(smem) + (uint32_t)(warp * 2 * c.page_bytes), bytes = (uint32_t)c.page_bytes;
  const uint64_t policy = l2_policy_evict_first();   // (more than L2 holds passes through: 73 us instead of 77 for 80 MB to three copies)
  uint32_t turn = 0;   // pages read so far: buffer and parity follow
  auto read_page = [&](uint32_t t, int page) {   // (lane 0) once the writes from this buffer have been taken out of it
    asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
    mbar_arrive_expect_tx(smem_u32(&bars[warp][t & 1]), bytes);
    bulk_g2s_hint(buf + (t & 1) * bytes, c.pool + (size_t)page * bytes, bytes, smem_u32(&bars[warp][t & 1]), policy);
  };
  bool ok = true;
  while (u < u_end && ok) {
    // (entries without pages to read begin where the next one does: the last of them is the one that has them)
    while (e + 1 < LB && units_at(e + 1) <= u) ++e;
    const int r = e % c.batch, l0 = e - r, pages = (__ldcg(c.len + e) + kPage - 1) / kPage;
    const int off = u - units_at(e), h = off / pages, j0 = off - h * pages;
    const int take = min(min(32, u_end - u), pages - j0);   // pages j0 .. of one head, a lane each
    const int src = lane < take ? __ldcg(c.pt + ((size_t)e * c.Hkv + h) * c.max_pages + j0 + lane) : 0;
    for (int s = m.first[r]; s >= 0 && ok;) {
      int dst[kForkGroup], nd = 0;
#pragma unroll
      for (int k = 0; k < kForkGroup; ++k) {
        dst[k] = 0;
        if (s < 0) continue;
        if (lane < take) {
          dst[k] = page_of(taken_at(l0 + s) + off + lane);
          c.pt_new[((size_t)(l0 + s) * c.Hkv + h) * c.max_pages + j0 + lane] = dst[k];
        }
        nd = k + 1;
        s = m.next[s];
      }
      if (lane == 0) read_page(turn, src);
      for (int i = 0; i < take && ok; ++i) {
        const int next = __shfl_sync(0xffffffffu, src, (i + 1) & 31);
        if (lane == 0 && i + 1 < take) read_page(turn + 1, next);
        ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&bars[warp][turn & 1]), (turn >> 1) & 1));
        if (!ok) {
          set_status(c, kDevWaitTimeout);
          // (no copy may be in flight at the exit: once more for this one, and for the next)
          mbar_wait(smem_u32(&bars[warp][turn & 1]), (turn >> 1) & 1);
          if (i + 1 < take) mbar_wait(smem_u32(&bars[warp][(turn + 1) & 1]), ((turn + 1) >> 1) & 1);
          break;
        }
#pragma unroll
        for (int k = 0; k < kForkGroup; ++k) {
          const int to = __shfl_sync(0xffffffffu, dst[k], i);
          if (lane == 0 && k < nd) bulk_s2g_hint(c.pool + (size_t)to * bytes, buf + (turn & 1) * bytes, bytes, policy);
        }
        if (lane == 0) cp_bulk_commit();
        ++turn;
      }
    }
    u += take;
  }
  if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");   // all writes are out
}

// grid (layers x sequences, heads).
__global__ void __launch_bounds__(256) k_fork_commit(Ctx c, const __grid_constant__ ForkMap m) {
  __shared__ int s_budget[kMaxBatch];
  griddep_wait();
  griddep_launch();
  const int top = __ldcg(c.planhdr + PH_PUSH_START);
  if (top < 0) return;
  const int i = blockIdx.x, h = blockIdx.y, s = i % c.batch, tid = threadIdx.x, what = m.what[s], LB = c.L * c.batch;
  const int bottom = top - __ldcg(c.planhdr + PH_NEW_PAGES);
  if (i == 0 && h == 0) {   // (the budget goes with the sequence; an emptied place keeps its own)
    if (tid == 0) c.ctrl[CTRL_FREE_TOP] = bottom + c.planhdr[PH_OLD_PAGES];
    static_assert(kMaxBatch <= 256, "one thread per sequence");
    if (tid < c.batch) s_budget[tid] = c.budget[tid];
    __syncthreads();
    if (tid < c.batch && m.from[tid] >= 0) c.budget[tid] = s_budget[m.from[tid]];
  }
  if (!(what & FORK_CHANGES)) return;
  const int n = __ldcg(c.idx + 2 * LB + i), n_new = __ldcg(c.idx + i), cnt_old = (n + kPage - 1) / kPage, cnt_new = (n_new + kPage - 1) / kPage;
  int *ptrow = c.pt + ((size_t)i * c.Hkv + h) * c.max_pages;
  const int *ptnew = c.pt_new + ((size_t)i * c.Hkv + h) * c.max_pages;
  if (what & FORK_FREED) {   // (those that would go below the stack's bottom are the ones that were taken again)
    const int at = bottom + __ldcg(c.tile1_start + i) + h * cnt_old;
    for (int x = tid; x < cnt_old; x += blockDim.x)
      if (at + x >= 0) c.free_stack[at + x] = __ldcg(ptrow + x);
    __syncthreads();
  }
#pragma unroll 4
  for (int x = tid; x < cnt_new; x += blockDim.x) ptrow[x] = __ldcg(ptnew + x);
  if (tid == 0 && h == 0) c.len[i] = n_new;
}

// grid (layers, enough threads for a sequence's record in 16-byte words).  Runs behind k_fork_commit (nothing there reads the record).
__global__ void __launch_bounds__(256) k_fork_record(Ctx c, const __grid_constant__ ForkOps ops) {
  griddep_wait();
  griddep_launch();
  if (__ldcg(c.planhdr + PH_PUSH_START) < 0) return;
  const int layer = blockIdx.x, ls0 = layer * c.batch, heads = c.Hkv * c.G;
  const size_t t = (size_t)blockIdx.y * blockDim.x + threadIdx.x;
  auto run = [&](auto *all, size_t per) {   // the layer's arrays of `per` elements per sequence: element t of each
    if (t >= per) return;
    auto *at = all + (size_t)ls0 * per + t;
    auto aside = at[0];
    for (int i = 0; i < ops.n; ++i) {
      const auto x = ops.src[i] == kForkAside ? aside : at[ops.src[i] * per];
      if (ops.dst[i] == kForkAside) aside = x; else at[ops.dst[i] * per] = x;
    }
  };
  run(reinterpret_cast<uint4 *>(c.hist_q), (size_t)c.hist_wp * heads * c.D / 8);
  run(c.hist_mp, (size_t)c.hist_wp * heads);
  run(c.hist_n, (size_t)c.hist_w);
  run(c.hist_cnt, (size_t)1);
  if (t == 0)
    for (int s = 0; s < c.batch; ++s)
      if (ops.emptied[s]) c.hist_cnt[ls0 + s] = 0;
}

}  // namespace fkv
