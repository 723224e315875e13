// The tree decode step's bookkeeping: the plan of a verify pass over a tree of
// drafted tokens, and the commit of the path that the target's draws lead
// through.  Both are latency: a launch and a few dependent steps over at most
// 256 nodes a sequence.  Measured, calls one after the other: plan of 64 trees of
// 256 nodes 7 to 9 us, commit of 16 sequences x 32 layers (6 MB of rows moved) the
// same: the host's time for a call.
#include "common.cuh"
#include "tree.h"

namespace pard {

// Plan.  One CTA a sequence, a thread a node.  A node's ancestor set is the
// union of its own bit and its parent's set; with links doubled in every round
// (each node takes over the set of the node its link points at, then that
// node's link) a tree of depth d is closed after ceil(log2 d) rounds instead of
// d.  A link of -1 is the top; a node whose parent does not precede it is
// dead (link -2), and so is whatever hangs on it.
__global__ void __launch_bounds__(kTreeMaxNodes) tree_plan_kernel(const TreePlanArgs a) {
  __shared__ uint64_t s_set[kTreeMaxWords][kTreeMaxNodes];
  __shared__ int s_link[kTreeMaxNodes];
  const int b = blockIdx.x, i = threadIdx.x;
  pdl_trigger();
  pdl_wait();
  const int n = min(max(a.n_nodes[b], 0), a.width);
  const int ctx = max(a.ctx_len[b], 0);
  const size_t at = (size_t)b * a.width + i;
  int link = -2;
  if (i < n) {
    const int p = a.parents[at];
    link = p >= -1 && p < i ? p : -2;
  }
  uint64_t set[kTreeMaxWords];
#pragma unroll
  for (int w = 0; w < kTreeMaxWords; ++w) set[w] = i >> 6 == w ? 1ull << (i & 63) : 0ull;
  while (true) {
    s_link[i] = link;
#pragma unroll
    for (int w = 0; w < kTreeMaxWords; ++w)
      if (w < a.words) s_set[w][i] = set[w];
    if (!__syncthreads_or(link >= 0)) break;
    if (link >= 0) {
#pragma unroll
      for (int w = 0; w < kTreeMaxWords; ++w)
        if (w < a.words) set[w] |= s_set[w][link];
      link = s_link[link];
    }
    __syncthreads();
  }
  if (i >= a.width) return;
  const bool live = link == -1;
  int depth = 0;
#pragma unroll
  for (int w = 0; w < kTreeMaxWords; ++w)
    if (w < a.words) {
      if (!live) set[w] = 0;
      depth += __popcll(set[w]);
      a.mask[at * a.words + w] = set[w];
    }
  a.pos[at] = live ? ctx + depth - 1 : 0;
  const int page = live ? page_of(a.page_table + (size_t)b * a.max_pages, ctx + i, a.max_pages, a.n_pages) : -1;
  a.slots[at] = page < 0 ? -1 : (int64_t)page * kPageTok + (ctx + i) % kPageTok;
}

void launch_tree_plan(const TreePlanArgs& a, cudaStream_t s) {
  const int threads = (a.width + 31) / 32 * 32;
  launch_in_turn(tree_plan_kernel, dim3(a.batch), threads, 0, 0, s, a);
}

// Commit.  Every CTA walks its sequence's tree for itself (cheaper than a
// launch of its own) and then moves one layer's keys or values: thread t owns
// 16 bytes of a token's row, all heads in turn, and moves the path's rows in
// ascending order.  Path node j lies at tree index path[j] >= j and moves to
// index j, so a row is overwritten only after it was read: no thread touches
// another's bytes, and a destination j is below every later source.
constexpr int kCommitThreads = 128;
constexpr int kCommitBatch = 8;  // rows a thread has in flight

__global__ void __launch_bounds__(kCommitThreads) tree_commit_kernel(const TreeCommitArgs a) {
  __shared__ int s_next[kTreeMaxNodes], s_said[kTreeMaxNodes];
  __shared__ int16_t s_path[kTreeMaxNodes];
  __shared__ int64_t s_src[kTreeMaxNodes], s_dst[kTreeMaxNodes];
  __shared__ int s_moves, s_count;
  const int b = blockIdx.y, tid = threadIdx.x;
  pdl_trigger();
  pdl_wait();
  const int n = min(max(a.n_nodes[b], 0), a.width);
  const int ctx = max(a.ctx_len[b], 0);
  const size_t at = (size_t)b * a.width;
  for (int i = tid; i < n; i += kCommitThreads) {
    s_next[i] = n;
    s_said[i] = a.sampled[at + i];
  }
  __syncthreads();
  for (int i = tid; i < n; i += kCommitThreads) {
    const int p = a.parents[at + i], t = a.tokens[at + i];
    if (p >= 0 && p < i && t >= 0 && t == s_said[p]) atomicMin(&s_next[p], i);  // the lowest child that matches
  }
  __syncthreads();
  if (tid == 0) {
    int count = 0;
    for (int cur = 0; cur < n; cur = s_next[cur]) s_path[count++] = (int16_t)cur;
    s_count = count;
    s_moves = 0;
  }
  __syncthreads();
  const int count = s_count;
  const int32_t* row = a.page_table + (size_t)b * a.max_pages;
  // nodes before the first gap stay where they are
  for (int j = tid; j < count; j += kCommitThreads) {
    const int from = s_path[j];
    int64_t src = -1, dst = -1;
    if (from != j) {
      const int sp = page_of(row, ctx + from, a.max_pages, a.n_pages), dp = page_of(row, ctx + j, a.max_pages, a.n_pages);
      if (sp >= 0 && dp >= 0) {
        src = sp * a.page_stride + (int64_t)((ctx + from) % kPageTok) * a.head_dim;
        dst = dp * a.page_stride + (int64_t)((ctx + j) % kPageTok) * a.head_dim;
      }
      atomicMax(&s_moves, j + 1);
    }
    s_src[j] = src;
    s_dst[j] = dst;
  }
  if (blockIdx.x == 0) {
    for (int j = tid; j < a.width; j += kCommitThreads) a.emitted[at + j] = j < count ? s_said[s_path[j]] : -1;
    if (tid == 0) {
      a.accept_len[b] = count > 0 ? count - 1 : 0;
      a.new_len[b] = ctx + count;
    }
  }
  __syncthreads();
  const int moves = s_moves;
  if (!moves) return;
  uint16_t* base = a.pool + (int64_t)(blockIdx.x >> 1) * a.layer_stride + (int64_t)(blockIdx.x & 1) * a.kv_stride;
  const int per_head = a.head_dim / 8, pieces = a.n_kv_heads * per_head;
  for (int c = tid; c < pieces; c += kCommitThreads) {
    uint16_t* col = base + (int64_t)(c / per_head) * kPageTok * a.head_dim + (c % per_head) * 8;
    for (int j0 = 0; j0 < moves; j0 += kCommitBatch) {
      uint4 v[kCommitBatch];
#pragma unroll
      for (int e = 0; e < kCommitBatch; ++e)
        if (j0 + e < moves && s_src[j0 + e] >= 0) v[e] = *reinterpret_cast<const uint4*>(col + s_src[j0 + e]);
#pragma unroll
      for (int e = 0; e < kCommitBatch; ++e)
        if (j0 + e < moves && s_src[j0 + e] >= 0) *reinterpret_cast<uint4*>(col + s_dst[j0 + e]) = v[e];
    }
  }
}

void launch_tree_commit(const TreeCommitArgs& a, cudaStream_t s) {
  launch_in_turn(tree_commit_kernel, dim3(2 * a.n_layers, a.batch), kCommitThreads, 0, 0, s, a);
}

}  // namespace pard
