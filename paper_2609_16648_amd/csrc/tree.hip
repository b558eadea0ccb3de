// Draft trees: the masks of a batch of trees, the accept walk, and the commit of the accepted
// path.  A tree has at most 64 nodes: a wave holds one sequence's, a node per lane.
#include <type_traits>

#include "common.h"
#include "tree.h"

namespace gm {

namespace {
__device__ __forceinline__ int nodes_of(const int32_t *n_nodes, int b, int N) {
  if (!n_nodes) return N;
  const int n = n_nodes[b];
  return n < 0 ? 0 : (n > N ? N : n);
}

// The set of a node's ancestors by pointer doubling: after round r the mask holds the 2^r nearest
// (the node itself among them) and `up` is the 2^r-th above it; six rounds cover 64 nodes.
__global__ __launch_bounds__(256) void tree_masks_kernel(int B, int N, const int32_t *__restrict__ parents,
                                                         const int32_t *__restrict__ n_nodes,
                                                         uint64_t *__restrict__ masks, int32_t *__restrict__ depths,
                                                         int32_t *dev_err) {
  const int b = blockIdx.x * 4 + (threadIdx.x >> 6), i = threadIdx.x & 63;
  if (b >= B) return;
  const int n = nodes_of(n_nodes, b, N);
  int up = i < n ? parents[(long)b * N + i] : -1;
  if (up < -1 || up >= i) {
    up = -1;
    raise_dev_err(dev_err, GM_DEVERR_TREE);
  }
  unsigned long long m = i < n ? 1ull << i : 0ull;
#pragma unroll
  for (int r = 0; r < 6; ++r) {
    const int from = up < 0 ? i : up;
    const unsigned long long mu = __shfl(m, from, kWave);
    const int uu = __shfl(up, from, kWave);
    if (up >= 0) {
      m |= mu;
      up = uu;
    }
  }
  if (i < N) {
    masks[(long)b * N + i] = m;
    depths[(long)b * N + i] = i < n ? __popcll(m) - 1 : 0;
  }
}

// The walk, one step per accepted node: the lanes whose parent is the current node and whose token
// is the target's after it; the lowest goes on.
__global__ __launch_bounds__(256) void tree_accept_kernel(int B, int N, const int32_t *__restrict__ parents,
                                                          const int32_t *__restrict__ tokens,
                                                          const int32_t *__restrict__ next_ids,
                                                          const int32_t *__restrict__ n_nodes,
                                                          int32_t *__restrict__ path, int32_t *__restrict__ n_accept,
                                                          int32_t *__restrict__ out_tokens) {
  const int b = blockIdx.x * 4 + (threadIdx.x >> 6), i = threadIdx.x & 63;
  if (b >= B) return;
  const int n = nodes_of(n_nodes, b, N);
  const long at = (long)b * N + i;
  const int par = i > 0 && i < n ? parents[at] : -1;      // (node 0 is nobody's child)
  const int tok = i < n ? tokens[at] : 0, nxt = i < n ? next_ids[at] : 0;
  int cur = 0, steps = 0, my_path = -1, my_out = -1;      // lane j holds entry j
  if (n > 0) {
    if (i == 0) my_path = 0;
    for (;;) {
      const int want = __shfl(nxt, cur, kWave);
      const unsigned long long hit = __ballot(par == cur && i > cur && tok == want);
      if (i == steps) my_out = want;      // the accepted child's token, or the final one
      if (!hit) break;
      cur = __ffsll(hit) - 1;
      ++steps;
      if (i == steps) my_path = cur;
    }
  }
  if (i < N) {
    path[at] = my_path;
    out_tokens[at] = my_out;
  }
  if (i == 0) n_accept[b] = n > 0 ? steps : -1;
}

constexpr int kCommitLayers = 128;   // layers per launch (their pool bases are kernel arguments, 2 KiB of 4)
struct CommitArgs {
  void *pools[kCommitLayers][2];
  const int32_t *path, *n_accept, *block_table, *seq_lens;
  int32_t *dev_err;
  int N, n_kv, page_size, max_pages, num_pages, layers, report;
};

// One workgroup per (sequence, layer, K or V).  A thread owns the same pieces of every token (16 bytes of K, one element
// of V), and moves the path's entries in increasing order, the loads of a batch before its stores.  That order is
// enough: entry i moves from slot path[i] >= i to slot i, so no earlier move has written what it reads, and a later
// one that overwrites slot path[i] comes behind it in the same thread.
// Bound by latency: two dependent loads for the places, then a batch of kBatch entries of kWide pieces each in one
// round trip (a token's K lies in 16-byte pieces and its V in single elements), and then by the lines that those touch.
// 64 sequences, 36 layers of 8 bf16 heads of 128: 37 us in one launch (60 in two, with batches of four elements);
// one sequence 8.
template <typename E, int D>
__global__ __launch_bounds__(256) void tree_commit_kernel(CommitArgs a) {
  __shared__ long src_sh[kMaxNodes], dst_sh[kMaxNodes];    // element offsets of (page, tile) blocks
  __shared__ int ss_sh[kMaxNodes], ds_sh[kMaxNodes];       // token in the tile
  __shared__ int count_sh;
  const int b = blockIdx.x, tid = threadIdx.x;
  if (tid < 64) {
    const int i = tid;
    const int p_any = i < a.N ? a.path[(long)b * a.N + i] : -1;
    const long m = a.seq_lens[b];
    int n = a.n_accept[b];
    n = n < -1 ? -1 : (n >= a.N ? a.N - 1 : n);
    const int p = i <= n ? p_any : -1;
    const int before = __shfl_up(p, 1, kWave);
    const bool bad = i <= n && (p < i || p >= a.N || (i > 0 && p <= before));
    const bool any_bad = __any(bad);
    bool moves = i <= n && !any_bad && p != i;
    if (any_bad && i == 0 && a.report) raise_dev_err(a.dev_err, GM_DEVERR_TREE);
    long src = 0, dst = 0;
    int ss = 0, ds = 0;
    if (moves) {
      // the pages of both places are asked for together
      const long from = m + p, to = m + i, pf = from / a.page_size, pt = to / a.page_size;
      const bool in = m >= 0 && pf < a.max_pages;           // (to < from)
      const int32_t *bt = a.block_table + (long)b * a.max_pages;
      const int gf = in ? bt[pf] : -1, gt = in ? bt[pt] : -1;
      if (gf < 0 || gf >= a.num_pages || gt < 0 || gt >= a.num_pages) {
        moves = false;
        if (a.report) raise_dev_err(a.dev_err, GM_DEVERR_PAGE);
      } else {
        const int of = (int)(from % a.page_size), ot = (int)(to % a.page_size);
        src = (long)gf * a.n_kv * a.page_size * D + (long)(of & ~15) * D;
        dst = (long)gt * a.n_kv * a.page_size * D + (long)(ot & ~15) * D;
        ss = of & 15;
        ds = ot & 15;
      }
    }
    const unsigned long long live = __ballot(moves);
    if (moves) {
      const int at = __popcll(live & ((1ull << i) - 1));
      src_sh[at] = src;
      dst_sh[at] = dst;
      ss_sh[at] = ss;
      ds_sh[at] = ds;
    }
    if (i == 0) count_sh = __popcll(live);
  }
  __syncthreads();
  const int count = count_sh;
  if (count == 0) return;
  // `pieces` of P, kWide per thread at a time; place(piece, token) is a piece's element offset behind its head's tile
  auto move = [&](auto *pool, int pieces, auto wide, auto batch, auto head_of, auto place) {
    constexpr int kWide = decltype(wide)::value, kBatch = decltype(batch)::value;
    using P = typename std::remove_pointer<decltype(pool)>::type;
    for (int x0 = tid; x0 < pieces; x0 += 256 * kWide) {
      for (int i0 = 0; i0 < count; i0 += kBatch) {
        P v[kBatch][kWide];
#pragma unroll
        for (int e = 0; e < kBatch; ++e)
#pragma unroll
          for (int u = 0; u < kWide; ++u) {
            const int x = x0 + 256 * u;
            if (i0 + e < count && x < pieces) v[e][u] = *place(pool, src_sh[i0 + e] + head_of(x), x, ss_sh[i0 + e]);
          }
#pragma unroll
        for (int e = 0; e < kBatch; ++e)
#pragma unroll
          for (int u = 0; u < kWide; ++u) {
            const int x = x0 + 256 * u;
            if (i0 + e < count && x < pieces) *place(pool, dst_sh[i0 + e] + head_of(x), x, ds_sh[i0 + e]) = v[e][u];
          }
      }
    }
  };
  const long head = (long)a.page_size * D;
  if (blockIdx.z == 0) {
    constexpr int kElems = 16 / sizeof(E), kPieces = D / kElems;
    move((uint4 *)a.pools[blockIdx.y][0], a.n_kv * kPieces, std::integral_constant<int, 1>{},
         std::integral_constant<int, 8>{}, [&](int x) { return x / kPieces * head; },
         [&](uint4 *pool, long base, int x, int s) {
           return (uint4 *)((E *)pool + base + k_tile_off(s, x % kPieces * kElems));
         });
  } else {
    move((E *)a.pools[blockIdx.y][1], a.n_kv * D, std::integral_constant<int, 4>{}, std::integral_constant<int, 4>{},
         [&](int x) { return x / D * head; },
         [&](E *pool, long base, int x, int s) { return pool + base + v_tile_off(s, x % D); });
  }
}

// the committed lengths, behind the moves that read them
__global__ __launch_bounds__(256) void tree_lens_kernel(int B, int N, int page_size, int max_pages, int num_pages,
                                                        const int32_t *__restrict__ block_table,
                                                        int32_t *__restrict__ seq_lens,
                                                        const int32_t *__restrict__ n_accept,
                                                        int32_t *__restrict__ slots) {
  const int b = blockIdx.x * 4 + (threadIdx.x >> 6), i = threadIdx.x & 63;
  if (b >= B) return;
  const int m = seq_lens[b];
  int n = n_accept[b];
  n = n < -1 ? -1 : (n >= N ? N - 1 : n);
  if (slots && i < N) {
    int v = -1;
    if (i <= n) {
      const long t = (long)m + i, pi = t / page_size;
      const int page = t >= 0 && pi < max_pages ? block_table[(long)b * max_pages + pi] : -1;
      if (page >= 0 && page < num_pages) v = page * page_size + (int)(t % page_size);
    }
    slots[(long)b * N + i] = v;
  }
  if (i == 0) seq_lens[b] = m + n + 1;
}
}  // namespace

void launch_tree_masks(int B, int N, const int32_t *parents, const int32_t *n_nodes, uint64_t *masks, int32_t *depths,
                       int32_t *dev_err, hipStream_t s) {
  TraceScope ts("tree_masks", s);
  hipLaunchKernelGGL(tree_masks_kernel, dim3((B + 3) / 4), dim3(256), 0, s, B, N, parents, n_nodes, masks, depths,
                     dev_err);
}

void launch_tree_accept(int B, int N, const int32_t *parents, const int32_t *tokens, const int32_t *next_ids,
                        const int32_t *n_nodes, int32_t *path, int32_t *n_accept, int32_t *out_tokens, hipStream_t s) {
  TraceScope ts("tree_accept", s);
  hipLaunchKernelGGL(tree_accept_kernel, dim3((B + 3) / 4), dim3(256), 0, s, B, N, parents, tokens, next_ids, n_nodes,
                     path, n_accept, out_tokens);
}

void launch_tree_commit(const gm_model_config &cfg, const gm_kv_cache &c, int B, int N, const int32_t *path,
                        const int32_t *n_accept, int32_t *slots, int32_t *dev_err, hipStream_t s) {
  for (int l0 = 0; l0 < c.n_layers; l0 += kCommitLayers) {
    CommitArgs a{};
    a.layers = c.n_layers - l0 < kCommitLayers ? c.n_layers - l0 : kCommitLayers;
    for (int l = 0; l < a.layers; ++l) {
      a.pools[l][0] = c.k_pages[l0 + l];
      a.pools[l][1] = c.v_pages[l0 + l];
    }
    a.path = path;
    a.n_accept = n_accept;
    a.block_table = c.block_table;
    a.seq_lens = c.seq_lens;
    a.dev_err = dev_err;
    a.N = N;
    a.n_kv = cfg.n_kv_heads;
    a.page_size = c.page_size;
    a.max_pages = c.max_pages_per_seq;
    a.num_pages = c.num_pages;
    a.report = l0 == 0;
    TraceScope ts("tree_commit", s);
    const dim3 grid(B, a.layers, 2);
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, a); };
    if (cfg.dtype == GM_BF16) launch(tree_commit_kernel<uint16_t, 128>);
    else if (cfg.head_dim == 64) launch(tree_commit_kernel<uint32_t, 64>);
    else launch(tree_commit_kernel<uint32_t, 128>);
  }
  TraceScope ts("tree_lens", s);
  hipLaunchKernelGGL(tree_lens_kernel, dim3((B + 3) / 4), dim3(256), 0, s, B, N, c.page_size, c.max_pages_per_seq,
                     c.num_pages, c.block_table, c.seq_lens, n_accept, slots);
}

}  // namespace gm
