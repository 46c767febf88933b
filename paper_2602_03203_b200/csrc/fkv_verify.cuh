// Kernel 11: which drafted tokens stand, and the token after them, from probabilities and given uniform numbers.
//
// The walk starts at the tree's root (a token that stands already).  At node a, with p = the target's and q = the draft model's
// probabilities of the token after it, the children (drawn from q, in the order of their indices) are tried one after another:
// child c with token x is accepted if u_c q(x) < R(x), R = p at first, and a rejection makes R = max(R - q, 0) / sum of that.  The
// walk goes on from an accepted child; where none is left the next token is drawn from R by one uniform number (the first token
// at which the running sum exceeds u times the whole).  Each token that comes out is then distributed as p says.
//
// After k rejections R is max(p - alpha_k q, 0) / S_k with alpha_1 = 1, alpha_{k+1} = alpha_k + S_k and S_k the sum of the
// numerator: max(max(p - a q, 0) / S - q, 0) is max(p - (a + S) q, 0) / S.  So nothing is kept per token but p and q themselves:
// a rejection costs one pass over the two rows, whatever came before it.
// Without draft probabilities a child is a point mass: R loses its token, u_c m < p(x) decides with m = 1 - the mass of the
// rejected ones, and only the last node's row is read.
// Of rows that hold what no probability is, NaN and negative numbers count as 0.  A child whose own q(x) is NaN is rejected whatever its
// number (nothing is known of how it was drawn; R then gives the next token), and q's row at a node is read as a whole only behind a
// rejection there: a draft model has no row for a leaf, and nothing that lies in its place may count.
//
// The walk itself runs in every thread alike, on numbers gathered ahead of it (p and q of every node's own token: one read).
// A pass is cut into pieces of 256 tokens; their sums stay in shared memory, so the piece that holds the drawn token is found
// there and read once more.  Everything is fp64: products of two fp32 numbers are exact, and sums over 10^5 terms that are
// compared with u lose nothing that fp32 inputs hold.  A sequence is a cluster of up to eight CTAs; its pieces are eight parts, summed
// each in the same order whichever CTA has it, and the parts' sums meet through distributed shared memory: results are the same bits
// in all CTAs, in every run and in every batch.
// Bound: bytes of the rows that are read; for few sequences latency (gather, pass, exchange, piece: four dependent reads).  Back to back in
// a graph, vocabulary 130001, 1965 MHz: five drafts of one sequence 8.4 - 9.5 us (six draws), 16 trees of up to 32 nodes with siblings 15.1 -
// 22.5 (by the passes on the longest way; bf16 15.4 - 23.2), 64 sequences without draft probabilities in bf16 14.8 (floor 2.5 us of bytes).
// One tree in a batch of 256 places 8.5, alone 8.2: a cluster without a tree writes its row of -1 and leaves.  Two pieces at a time per
// warp gain nothing (the registers for them spill).
#pragma once
#include "fkv_dev.cuh"
#include "fkv_attend.cuh"
#include "fkv_chunk.cuh"

namespace fkv {

constexpr int kVerThreads = 512, kVerWarps = kVerThreads / 32;
constexpr int kVerPiece = 256;                    // tokens of a piece: eight per lane
constexpr int kVerMaxVocab = 1 << 20;
constexpr int kVerPieces = kVerMaxVocab / kVerPiece;
constexpr int kVerParts = 8;                      // of a row's pieces; CTAs of a cluster: 1, 2, 4 or 8
constexpr int kVerCtasPerSm = 2;                  // that fit at a time

struct VerifyArgs {
  const void *target, *draft;      // rows of a token's successor probabilities, one per node
  long long target_stride, draft_stride;
  const int32_t *tokens, *parents;
  const float *u_accept, *u_sample;
  int32_t *path, *path_len, *out;
  int vocab, stride;
  ChunkLens lens;
};

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ uint32_t cluster_size() {
  uint32_t r;
  asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void dsmem_st_f64(uint32_t addr, double x) {
  asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(addr), "d"(x) : "memory");
}
__device__ __forceinline__ double warp_sum(double x) {
#pragma unroll
  for (int o = 16; o >= 1; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  return x;
}

template <class T, bool Q>
__global__ void __launch_bounds__(kVerThreads, kVerCtasPerSm) k_verify_tree(Ctx c, const __grid_constant__ VerifyArgs a) {
  __shared__ double s_sum[kVerPieces];              // sums of this CTA's pieces
  __shared__ double s_all[2][kVerParts];            // the parts' sums, of this pass and of the last
  __shared__ double s_warp[kVerParts][kVerWarps];
  __shared__ double s_p[kTreeNodes], s_q[kTreeNodes];
  __shared__ float s_u[kTreeNodes];
  __shared__ int s_tok[kTreeNodes];
  __shared__ short s_par[kTreeNodes], s_first[kTreeNodes], s_next[kTreeNodes];
  griddep_wait();
  griddep_launch();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int cs = (int)cluster_size(), rank = (int)cluster_rank(), seq = blockIdx.x / cs;
  const int row0 = a.lens.tok[seq], nodes = a.lens.tok[seq + 1] - row0, V = a.vocab;
  int32_t *path = a.path + (size_t)seq * a.stride, *out = a.out + (size_t)seq * a.stride;
  if (rank == 0)
    for (int i = tid; i < a.stride; i += kVerThreads) path[i] = out[i] = -1;
  if (nodes == 0) {   // (of the whole cluster alike)
    if (rank == 0 && tid == 0) a.path_len[seq] = 0;
    return;
  }
  // "I am running": waited for ahead of the walk, whose passes write into the other CTAs' shared memory (the gather hides the wait).
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  auto row_p = [&](int node) { return reinterpret_cast<const T *>(a.target) + (row0 + node) * a.target_stride; };
  auto row_q = [&](int node) { return reinterpret_cast<const T *>(a.draft) + (row0 + node) * a.draft_stride; };
  if (tid < nodes) {
    const int x = __ldcg(a.tokens + row0 + tid);
    int p = tid > 0 ? __ldcg(a.parents + row0 + tid) : -1;
    if (p >= tid || p < -1) {   // (a node that nothing leads to)
      if (rank == 0) set_status(c, kDevBadIndex);
      p = -1;
    }
    const bool ok = p >= 0 && x >= 0 && x < V;
    s_tok[tid] = ok ? x : -1;
    s_par[tid] = (short)p;
    s_u[tid] = __ldcg(a.u_accept + row0 + tid);
    s_p[tid] = ok ? fmax((double)to_f32(__ldcg(row_p(p) + x)), 0.0) : 0.0;   // (NaN and negative numbers count as 0)
    if (Q) {
      const double q = ok ? (double)to_f32(__ldcg(row_q(p) + x)) : 0.0;
      s_q[tid] = q < 0.0 ? 0.0 : q;   // (NaN stays: no comparison with it holds, so the draft is refused)
    }
  }
  __syncthreads();
  if (tid < nodes) {
    int first = -1, next = -1;
    bool again = false;   // the token of a sibling before: nothing is left of it when this node is tried
    const int par = s_par[tid], x = s_tok[tid];
    for (int i = nodes - 1; i > 0; --i) {
      const int p = s_par[i];
      if (p == tid) first = i;
      if (p == par && i > tid) next = i;
      if (!Q) again = again || (p == par && i < tid && s_tok[i] == x);
    }
    s_first[tid] = (short)first;
    s_next[tid] = (short)next;
    if (again) s_p[tid] = 0.0;
  }
  __syncthreads();
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");   // every CTA of the cluster runs

  const int pieces = (V + kVerPiece - 1) / kVerPiece;
  const int per = kVerParts / cs;   // this CTA's parts are [rank per, (rank + 1) per)
  auto begin = [&](int part) { return (int)((long long)pieces * part / kVerParts); };
  const int c0 = begin(rank * per);
  int turn = 0;
  int cur = 0, len = 0;
  // What R is without its divisor: p - alpha q, or p without the tokens of cur's children.
  auto weight = [&](double p, double q, double alpha) { return Q ? fmax(fma(-alpha, q, p), 0.0) : fmax(p, 0.0); };
  // A lane's eight weights of a piece: tokens lane, lane + 32, ... of it.
  // (The draft's row is read where something was rejected: a leaf's is in general never filled.  R is p elsewhere.)
  auto load = [&](int pc, T (&pv)[8], T (&qv)[8], double alpha) {
    const bool both = Q && alpha != 0.0;
    const T *pr = row_p(cur), *qr = both ? row_q(cur) : nullptr;
    const int x0 = pc * kVerPiece + lane;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const bool in = x0 + 32 * i < V;
      pv[i] = in ? __ldcg(pr + x0 + 32 * i) : T(0.f);
      if (Q) qv[i] = both && in ? __ldcg(qr + x0 + 32 * i) : T(0.f);
    }
  };
  auto weights = [&](int pc, const T (&pv)[8], const T (&qv)[8], double alpha, double (&w)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i)   // (NaN and negative numbers count as 0; in 64 bits the comparison costs a fifth of a pass)
      w[i] = weight((double)to_f32(pv[i]), Q ? (double)fmaxf(to_f32(qv[i]), 0.f) : 0.0, alpha);
    if (!Q)   // without the rejected tokens: those of cur's children, looked for by the whole warp
      for (int j0 = 0; j0 < nodes; j0 += 32) {
        const int j = j0 + lane, x = j < nodes && s_par[j] == cur ? s_tok[j] : -1;
        unsigned in = __ballot_sync(0xffffffffu, x >= 0 && x / kVerPiece == pc);
        for (; in; in &= in - 1) {
          const int at = __shfl_sync(0xffffffffu, x, __ffs(in) - 1) % kVerPiece;
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (at == lane + 32 * i) w[i] = 0.0;
        }
      }
  };
  // The sum over the vocabulary, the same in every CTA; the pieces' sums stay in s_sum, the parts' in s_all[turn ^ 1].
  auto pass = [&](double alpha) {
    for (int part = 0; part < per; ++part) {
      const int b0 = begin(rank * per + part), b1 = begin(rank * per + part + 1);
      double sum = 0.0;
#pragma unroll 1
      for (int pc = b0 + warp; pc < b1; pc += kVerWarps) {
        T pv[8], qv[8];
        load(pc, pv, qv, alpha);
        double w[8];
        weights(pc, pv, qv, alpha, w);
        const double x = warp_sum(((w[0] + w[1]) + (w[2] + w[3])) + ((w[4] + w[5]) + (w[6] + w[7])));
        if (lane == 0) s_sum[pc - c0] = x;
        sum += x;
      }
      if (lane == 0) s_warp[part][warp] = sum;
    }
    __syncthreads();
    for (int e = tid; e < per * cs; e += kVerThreads) {   // (part, CTA that it goes to)
      const int part = e / cs;
      double all = 0.0;
      for (int i = 0; i < kVerWarps; ++i) all += s_warp[part][i];
      dsmem_st_f64(dsmem_addr(smem_u32(&s_all[turn][rank * per + part]), e - part * cs), all);
    }
    cluster_sync_all();   // (a CTA's next pass writes the other half; this one is written again behind the next barrier)
    double all = 0.0;
    for (int i = 0; i < kVerParts; ++i) all += s_all[turn][i];
    turn ^= 1;
    return all;
  };

  double alpha = 0.0, S = 1.0;
  bool summed = false;   // S is the sum over the rows as they stand
  if (rank == 0 && tid == 0) path[0] = 0;
  len = 1;
  for (int ch = s_first[0]; ch >= 0;) {
    if (s_tok[ch] < 0) {   // (a token outside the vocabulary: as if the node were not there)
      ch = s_next[ch];
      continue;
    }
    const double x = s_p[ch], u = (double)s_u[ch];
    const bool ok = Q ? u * s_q[ch] * S < weight(x, s_q[ch], alpha) : u * S < x;
    if (ok) {
      if (rank == 0 && tid == 0) {
        path[len] = ch;
        out[len - 1] = s_tok[ch];
      }
      ++len;
      cur = ch;
      ch = s_first[ch];
      alpha = 0.0;
      S = 1.0;
      summed = false;
      continue;
    }
    if (Q) {
      alpha = summed ? alpha + S : 1.0;   // (never 0)
      S = pass(alpha);
      summed = true;
      if (!(S > 0.0)) {   // nothing is left of p: a rejection that had no probability; p itself serves
        alpha = 0.0;
        S = 1.0;
        summed = false;
      }
    } else {
      S -= x;
    }
    ch = s_next[ch];
  }
  if (!summed) S = pass(Q ? alpha : 0.0);
  if (rank == 0 && tid == 0) a.path_len[seq] = len;
  // The next token: the part, the piece, then the place at which the running sum exceeds u S.
  const double *all = s_all[turn ^ 1];
  const double t = (double)__ldcg(a.u_sample + seq) * S;
  int owner = -1;
  double before = 0.0, run = 0.0;
  for (int i = 0; i < kVerParts; ++i) {
    if (all[i] > 0.0 && (owner < 0 || run <= t)) {   // (the last one that holds anything, where rounding leaves t behind all)
      owner = i;
      before = run;
    }
    run += all[i];
  }
  if (owner < 0 || owner / per != rank || warp != 0) return;   // (owner < 0: no mass at all, and out keeps its -1)
  const int b0 = begin(owner), b1 = begin(owner + 1);
  int at = -1;
  run = before;
  for (int b = b0; b < b1; b += 32) {
    const double x = b + lane < b1 ? s_sum[b + lane - c0] : 0.0;
    double inc = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const double y = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += y;
    }
    const unsigned some = __ballot_sync(0xffffffffu, x > 0.0), past = __ballot_sync(0xffffffffu, x > 0.0 && run + inc > t);
    if (past || some) {
      const int l = past ? __ffs(past) - 1 : 31 - __clz(some);
      at = b + l;
      before = run + __shfl_sync(0xffffffffu, inc - x, l);
      if (past) break;
    }
    run += __shfl_sync(0xffffffffu, inc, 31);
  }
  if (at < 0) return;   // (cannot be: the owner holds something)
  double w[8];
  {
    T pv[8], qv[8];
    load(at, pv, qv, alpha);
    weights(at, pv, qv, alpha, w);
  }
  int found = -1;
  run = before;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    double inc = w[i];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const double y = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += y;
    }
    const unsigned some = __ballot_sync(0xffffffffu, w[i] > 0.0), past = __ballot_sync(0xffffffffu, w[i] > 0.0 && run + inc > t);
    if (past) {
      found = 32 * i + __ffs(past) - 1;
      break;
    }
    if (some) found = 32 * i + 31 - __clz(some);
    run += __shfl_sync(0xffffffffu, inc, 31);
  }
  if (lane == 0) out[len - 1] = at * kVerPiece + found;
}

// Temperature zero: the target's own choice after every node is known, and the walk takes the child that has it (the one with
// the lowest index).  A warp per sequence.  Bound: latency of a launch and two dependent reads: 1.9 us for a tree of 6, 2.5 for 16 of 32,
// 4.9 for 256 trees of 256.
__global__ void __launch_bounds__(32) k_verify_greedy(Ctx c, const __grid_constant__ VerifyArgs a, const int32_t *choice) {
  __shared__ int s_tok[kTreeNodes], s_want[kTreeNodes];
  __shared__ short s_par[kTreeNodes];
  griddep_wait();
  griddep_launch();
  const int seq = blockIdx.x, lane = threadIdx.x, row0 = a.lens.tok[seq], nodes = a.lens.tok[seq + 1] - row0;
  int32_t *path = a.path + (size_t)seq * a.stride, *out = a.out + (size_t)seq * a.stride;
  for (int j = lane; j < nodes; j += 32) {
    int p = j > 0 ? __ldcg(a.parents + row0 + j) : -1;
    if (p >= j || p < -1) {   // (a node that nothing leads to; 16 bits hold what is left)
      set_status(c, kDevBadIndex);
      p = -1;
    }
    s_par[j] = (short)p;
    s_tok[j] = __ldcg(a.tokens + row0 + j);
    s_want[j] = __ldcg(choice + row0 + j);
  }
  __syncwarp();
  int cur = 0, len = 0;
  while (len < nodes) {   // (every turn goes to a later node)
    const int want = s_want[cur];
    if (lane == 0) {
      path[len] = cur;
      out[len] = want;
    }
    ++len;
    int next = -1;
    for (int j0 = cur + 1; j0 < nodes && next < 0; j0 += 32) {
      const unsigned hit = __ballot_sync(0xffffffffu, j0 + lane < nodes && s_par[j0 + lane] == cur && s_tok[j0 + lane] == want);
      if (hit) next = j0 + __ffs(hit) - 1;
    }
    if (next < 0) break;
    cur = next;
  }
  for (int i = len + lane; i < a.stride; i += 32) path[i] = out[i] = -1;
  if (lane == 0) a.path_len[seq] = len;
}

}  // namespace fkv
