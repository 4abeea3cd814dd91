// arbor_extend, arbor_truncate, arbor_fork: the pages of blocks that grow, shrink
// and are copied (Sec. 3: a block is a token span of the tree; its paged storage
// is this library's).
//
// Each call decides everything in a plan of one workgroup, which checks the whole
// request before it changes anything, and leaves the work that grows with the
// tokens to a launch over the chip:
//   extend    plan: pages of each block by a scan, c_i, n_i, the free-stack top;
//             rows: slot, position and page-table entry of each new token;
//   truncate  plan: the resident tokens each block keeps (a bounded search of
//             its ascending slot positions), freed pages by a scan;
//             clear: slot positions, page-table entries, pushed pages, A;
//   fork      plan: pages by a scan; copy: K/V rows, slot positions, A.
// Pages are popped and pushed in (node, page) order: page j of F popped is stack
// entry top-1-j, and page j of F pushed becomes entry top+F-1-j, so that taking
// tokens back undoes reserving them.
#include "arbor_internal.h"

namespace arbor {

namespace {

constexpr int kPlanThreads = 1024;
constexpr int kTreeLds = 4096;          // blocks of a tree that a plan keeps in LDS

// What the plan leaves for the second launch, one entry per listed block.
struct Grow {
  int32_t *c0, *n0;     // resident and all tokens before the call
  int32_t *first;       // pages of the blocks before it (popped, touched or copied)
  int32_t *start;       // extend: position of the block's first token in its chain;
                        // truncate: resident tokens that stay
  int32_t *meta;        // [0] ready, [1] free-stack top before the call, [2] total of `first`,
                        // [3] truncate: freed pages
  int32_t *freed;       // truncate: freed pages of the blocks before it
  int64_t *rows;        // fork: rows_seen of the source
};

__device__ __forceinline__ int pages_of(int slots, int P) { return (slots + P - 1) / P; }

// Entry of the ascending list that holds x: the last e with first[e] <= x.
template <class T>
__device__ __forceinline__ int last_at_most(const T *first, int n, T x) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (first[mid] <= x) lo = mid;
    else hi = mid;
  }
  return lo;
}

// Tokens that the block x gets in this call (0 unless it is listed).
__device__ __forceinline__ int listed_tokens(const int32_t *nodes, const int32_t *cu, int n,
                                             int x) {
  const int e = last_at_most(nodes, n, x);
  return nodes[e] == x ? cu[e + 1] - cu[e] : 0;
}

// Slot, position and page of the packed tokens t, t + step, ...: the whole work of
// the second launch of extend.
__device__ void extend_rows(const Tree &t, const Pool &pl, const int32_t *__restrict__ nodes,
                            int n_seq, const int32_t *__restrict__ cu, int n_tokens, const Grow &g,
                            int64_t *__restrict__ slots, int32_t *__restrict__ positions,
                            int64_t *__restrict__ tokens, int top, int first, int step,
                            int32_t *status) {
  const int P = pl.P;
  const int live = n_seq > 0 ? cu[n_seq] : 0;
  for (int x = first; x < n_tokens; x += step) {
    if (x >= live) {
      slots[x] = -1;
      positions[x] = 0;
      if (tokens) tokens[x] = -1;
      continue;
    }
    const int e = last_at_most(cu, n_seq, x);
    const int i = nodes[e], j = x - cu[e];
    const int s = g.c0[e] + j, p = g.n0[e] + j, q = s / P;
    const int old = pages_of(g.c0[e], P);
    const int64_t at = t.page_off[i] + q;
    const int page = q < old ? t.page_table[at] : pl.free_stack[top - 1 - (g.first[e] + q - old)];
    if (page < 0 || page >= pl.num_pages) {        // a pool that was not consistent before
      status_error(status, ARBOR_ECORRUPT);
      continue;
    }
    if (q >= old && s % P == 0) t.page_table[at] = page;
    const int64_t slot = (int64_t)page * P + s % P;
    pl.slot_pos[slot] = p;
    slots[x] = slot;
    positions[x] = g.start[e] + p;
    if (tokens) tokens[x] = t.tok_off[i] + p;
  }
}

// Latency: checks 1.3 us, a vote 0.5, walks 1.1, scan 0.8, rows 1.5 (6.9 us for 48 blocks and
// 175 tokens, 7.4 for 16 blocks four levels down and 496 tokens; walks in memory, a dependent
// load a level: 0.5 more).
__global__ __launch_bounds__(kPlanThreads) void extend_plan(
    Tree t, Pool pl, int32_t *n_full, const int32_t *__restrict__ nodes, int n_seq,
    const int32_t *__restrict__ cu, int n_tokens, Grow g, int64_t *__restrict__ slots,
    int32_t *__restrict__ positions, int64_t *__restrict__ tokens, int rows_too, int32_t *status) {
  __shared__ int64_t sm[17];
  // the tree itself, where it is small, so that a walk's steps do not wait for memory
  __shared__ int32_t sh_parent[kTreeLds], sh_full[kTreeLds];
  const bool near = t.V <= kTreeLds;
  if (near)
    for (int i = threadIdx.x; i < t.V; i += blockDim.x) {
      sh_parent[i] = t.parent[i];
      sh_full[i] = t.n_full[i];
    }
  if (status_failed(status)) {
    if (threadIdx.x == 0) g.meta[0] = 0;
    return;
  }
  const int P = pl.P, nt = blockDim.x;
  const int per = (n_seq + nt - 1) / nt;
  const int r0 = min(n_seq, (int)threadIdx.x * per), r1 = min(n_seq, r0 + per);
  int err = 0;
  int64_t need = 0;
  const int top = *pl.free_top, oldest = n_seq > 0 ? nodes[0] : 0;
  if (threadIdx.x == 0 && (cu[0] != 0 || cu[n_seq] > n_tokens || cu[n_seq] < 0)) err = ARBOR_EINVAL;
  if (top < 0 || top > pl.num_pages) err = ARBOR_ECORRUPT;      // (no stack to pop from)
  for (int e = r0; e < r1; ++e) {
    const int i = nodes[e], m = cu[e + 1] - cu[e];
    if (i < 0 || i >= t.V || (e > 0 && nodes[e - 1] >= i) || m < 0 || m > n_tokens) {
      err = ARBOR_EINVAL;
      continue;
    }
    const int c = t.n_kept[i], n = t.n_full[i];
    const int64_t room = t.tok_off[i + 1] - t.tok_off[i];
    const int64_t pages = t.page_off[i + 1] - t.page_off[i];
    if (c < 0 || n < c || (int64_t)n + m > room || ((int64_t)c + m + P - 1) / P > pages) {
      err = ARBOR_EINVAL;
      continue;
    }
    g.c0[e] = c;
    g.n0[e] = n;
    need += pages_of(c + m, P) - pages_of(c, P);
  }
  // (a listed ancestor's tokens are looked up in nodes and cu, which the loop
  // above has checked; so the walks come after the vote)
  if (__syncthreads_or(err)) {
    if (err) status_error(status, err);
    if (threadIdx.x == 0) g.meta[0] = 0;
    return;
  }
  for (int e = r0; e < r1; ++e) {
    int64_t start = 0;
    int depth = 0;
    for (int x = nodes[e];;) {
      const int up = near ? sh_parent[x] : t.parent[x];
      if (up < 0) break;
      if (up >= x) {
        err = ARBOR_EINVAL;
        break;
      }
      if (++depth > ARBOR_MAX_DEPTH) {
        err = ARBOR_EUNSUPPORTED;
        break;
      }
      x = up;
      start += (near ? sh_full[x] : t.n_full[x]) +
               (x < oldest ? 0 : listed_tokens(nodes, cu, n_seq, x));
    }
    g.start[e] = (int32_t)start;
  }
  int64_t total;
  const int64_t base = block_exclusive_scan(need, sm, &total);
  if (total > top) err = err ? err : ARBOR_ENOPAGES;
  if (__syncthreads_or(err)) {
    if (err) status_error(status, err);
    if (threadIdx.x == 0) g.meta[0] = 0;
    return;
  }
  int64_t at = base;
  for (int e = r0; e < r1; ++e) {
    const int i = nodes[e], m = cu[e + 1] - cu[e], c = g.c0[e];
    g.first[e] = (int32_t)at;
    at += pages_of(c + m, P) - pages_of(c, P);
    t.n_kept[i] = c + m;
    n_full[i] = g.n0[e] + m;
  }
  if (threadIdx.x == 0) {
    *pl.free_top = top - (int32_t)total;
    g.meta[0] = 1;
    g.meta[1] = top;
  }
  if (!rows_too) return;
  __syncthreads();
  extend_rows(t, pl, nodes, n_seq, cu, n_tokens, g, slots, positions, tokens, top, threadIdx.x, nt,
              status);
}

__global__ __launch_bounds__(256) void extend_rows_kernel(
    Tree t, Pool pl, const int32_t *__restrict__ nodes, int n_seq, const int32_t *__restrict__ cu,
    int n_tokens, Grow g, int64_t *__restrict__ slots, int32_t *__restrict__ positions,
    int64_t *__restrict__ tokens, int32_t *status) {
  if (status_failed(status) || !g.meta[0]) return;
  extend_rows(t, pl, nodes, n_seq, cu, n_tokens, g, slots, positions, tokens, g.meta[1],
              blockIdx.x * blockDim.x + threadIdx.x, gridDim.x * blockDim.x, status);
}

// Resident tokens of block i at positions below keep.  Positions ascend with the
// slots, at most n - keep of them are dropped, and slot s holds position s or more:
// so the count lies in [c - (n - keep), min(c, keep)].
__device__ int kept_below(const Tree &t, const Pool &pl, int i, int c, int n, int keep) {
  if (keep >= n) return c;
  int lo = max(0, c - (n - keep)), hi = min(c, keep);
  const int64_t po = t.page_off[i];
  bool first = true;
  while (lo < hi) {
    // the newest tokens are mostly resident: try the lower end before halving
    const int mid = first ? lo : (lo + hi) / 2;
    first = false;
    const int page = t.page_table[po + mid / pl.P];
    const int pos = page >= 0 && page < pl.num_pages
                        ? pl.slot_pos[(int64_t)page * pl.P + mid % pl.P] : INT32_MAX;
    if (pos < keep) lo = mid + 1;
    else hi = mid;
  }
  return lo;
}

__global__ __launch_bounds__(kPlanThreads) void truncate_plan(
    Tree t, Pool pl, int32_t *n_full, const int32_t *__restrict__ nodes,
    const int32_t *__restrict__ keep, int n_nodes, Grow g, int scored, int32_t *status) {
  __shared__ int64_t sm[2 * 16];
  if (status_failed(status)) {
    if (threadIdx.x == 0) g.meta[0] = 0;
    return;
  }
  const int P = pl.P, nt = blockDim.x;
  const int per = (n_nodes + nt - 1) / nt;
  const int r0 = min(n_nodes, (int)threadIdx.x * per), r1 = min(n_nodes, r0 + per);
  int err = 0;
  int64_t touched = 0, freed = 0;
  const int top = *pl.free_top;
  for (int e = r0; e < r1; ++e) {
    const int i = nodes[e];
    if (i < 0 || i >= t.V || (e > 0 && nodes[e - 1] >= i) || keep[e] < 0) {
      err = ARBOR_EINVAL;
      continue;
    }
    const int c = t.n_kept[i], n = t.n_full[i];
    if (c < 0 || n < c || pages_of(c, P) > t.page_off[i + 1] - t.page_off[i] ||
        (scored && n > t.tok_off[i + 1] - t.tok_off[i])) {
      err = ARBOR_EINVAL;
      continue;
    }
    const int left = kept_below(t, pl, i, c, n, keep[e]);
    g.c0[e] = c;
    g.n0[e] = n;
    g.start[e] = left;
    touched += pages_of(c, P) - left / P;      // from the page of the first vacated slot
    freed += pages_of(c, P) - pages_of(left, P);
  }
  const int64_t v[2] = {touched, freed};
  int64_t ex[2], tot[2];
  block_exclusive_scan_n<2>(v, ex, tot, sm);
  if (!err && (top < 0 || top + tot[1] > pl.num_pages)) err = ARBOR_ECORRUPT;
  if (__syncthreads_or(err)) {
    if (err) status_error(status, err);
    if (threadIdx.x == 0) g.meta[0] = 0;
    return;
  }
  for (int e = r0; e < r1; ++e) {
    const int i = nodes[e], left = g.start[e];
    g.first[e] = (int32_t)ex[0];
    g.freed[e] = (int32_t)ex[1];
    ex[0] += pages_of(g.c0[e], P) - left / P;
    ex[1] += pages_of(g.c0[e], P) - pages_of(left, P);
    t.n_kept[i] = left;
    n_full[i] = min(g.n0[e], keep[e]);
  }
  if (threadIdx.x == 0) {
    *pl.free_top = top + (int32_t)tot[1];
    g.meta[0] = 1;
    g.meta[1] = top;
    g.meta[2] = (int32_t)tot[0];
    g.meta[3] = (int32_t)tot[1];
  }
}

// (The plan takes 3.5 to 4.7 us, this launch 3.5 to 4.4, mostly their start and the latency of
// five loads; the host does not know how many pages there are, so it is always made.)
// 16 lanes a page: the slots from the first vacated one on, and, where the page is
// freed, its table entry and its place on the stack.  With A, a workgroup a block: the
// attention of the tokens taken back, and the rows that a block has seen once it is empty.
__global__ __launch_bounds__(256) void truncate_clear(Tree t, Pool pl,
                                                      const int32_t *__restrict__ nodes,
                                                      const int32_t *__restrict__ keep,
                                                      int n_nodes, Grow g, float *A,
                                                      int64_t *rows_seen, int32_t *status) {
  __shared__ int32_t sh_first[1024];
  const bool few = n_nodes <= 1024;
  if (few)
    for (int e = threadIdx.x; e < n_nodes; e += 256) sh_first[e] = g.first[e];
  if (status_failed(status) || !g.meta[0]) return;
  const int P = pl.P, lane = threadIdx.x % 16;
  const int top = g.meta[1], total = g.meta[2], freed = g.meta[3];
  __syncthreads();
  for (int x = (blockIdx.x * blockDim.x + threadIdx.x) / 16; x < total;
       x += gridDim.x * blockDim.x / 16) {
    const int e = few ? last_at_most(sh_first, n_nodes, x) : last_at_most(g.first, n_nodes, x);
    const int i = nodes[e], left = g.start[e];
    const int q = left / P + x - g.first[e];
    const int64_t at = t.page_off[i] + q;
    const int page = t.page_table[at];
    if (page < 0 || page >= pl.num_pages) continue;
    for (int r = max(0, left - q * P) + lane; r < P; r += 16)
      pl.slot_pos[(int64_t)page * P + r] = -1;
    if (lane == 0 && q * P >= left) {
      pl.free_stack[top + freed - 1 - (g.freed[e] + q - pages_of(left, P))] = page;
      t.page_table[at] = -1;
    }
  }
  if (!A) return;
  for (int e = blockIdx.x; e < n_nodes; e += gridDim.x) {
    const int i = nodes[e], n0 = g.n0[e], n1 = min(n0, keep[e]);
    float *a = A + t.tok_off[i];
    for (int p = n1 + threadIdx.x; p < n0; p += 256) a[p] = 0.0f;
    if (threadIdx.x == 0 && n1 == 0) rows_seen[i] = 0;
  }
}

__global__ __launch_bounds__(kPlanThreads) void fork_plan(Tree t, Pool pl, int32_t *n_full,
                                                          const int32_t *__restrict__ src,
                                                          const int32_t *__restrict__ dst,
                                                          int n_forks, Grow g, int64_t *rows_seen,
                                                          int32_t *status) {
  __shared__ int64_t sm[17];
  if (status_failed(status)) {
    if (threadIdx.x == 0) g.meta[0] = 0;
    return;
  }
  const int P = pl.P, nt = blockDim.x;
  const int per = (n_forks + nt - 1) / nt;
  const int r0 = min(n_forks, (int)threadIdx.x * per), r1 = min(n_forks, r0 + per);
  int err = 0;
  int64_t need = 0;
  const int top = *pl.free_top;
  for (int e = r0; e < r1; ++e) {
    const int a = src[e], b = dst[e];
    if (top < 0 || top > pl.num_pages) err = ARBOR_ECORRUPT;
    if (a < 0 || a >= t.V || b < 0 || b >= t.V || (e > 0 && dst[e - 1] >= b)) {
      err = ARBOR_EINVAL;
      continue;
    }
    const int c = t.n_kept[a], n = t.n_full[a];
    if (c < 0 || n < c || pages_of(c, P) > t.page_off[a + 1] - t.page_off[a] ||
        n > t.tok_off[a + 1] - t.tok_off[a] || t.n_kept[b] != 0 || t.n_full[b] != 0 ||
        n > t.tok_off[b + 1] - t.tok_off[b] ||
        pages_of(c, P) > t.page_off[b + 1] - t.page_off[b]) {
      err = ARBOR_EINVAL;
      continue;
    }
    g.c0[e] = c;
    g.n0[e] = n;
    if (rows_seen) g.rows[e] = rows_seen[a];
    need += pages_of(c, P);
  }
  int64_t total;
  const int64_t base = block_exclusive_scan(need, sm, &total);
  if (!err && total > top) err = ARBOR_ENOPAGES;
  // (after this barrier every source has been read, one that is a destination too
  // as it was)
  if (__syncthreads_or(err)) {
    if (err) status_error(status, err);
    if (threadIdx.x == 0) g.meta[0] = 0;
    return;
  }
  int64_t at = base;
  for (int e = r0; e < r1; ++e) {
    g.first[e] = (int32_t)at;
    at += pages_of(g.c0[e], P);
    t.n_kept[dst[e]] = g.c0[e];
    n_full[dst[e]] = g.n0[e];
    if (rows_seen) rows_seen[dst[e]] = g.rows[e];
  }
  if (threadIdx.x == 0) {
    *pl.free_top = top - (int32_t)total;
    g.meta[0] = 1;
    g.meta[1] = top;
    g.meta[2] = (int32_t)total;
  }
}

// HBM-bound: every resident row of the sources read once and written once.  A
// workgroup takes one page of one layer at a time, whose K (V) rows of all heads
// lie side by side: [Hkv][P][D].  4 blocks of 32 layers of the 8B shape (268 MB): 47 us,
// 5.7 TB/s, above the rate of a large copy as part of the rows are in the last-level cache;
// 128 ragged blocks of 4 layers (124 MB): 24 us.
__global__ __launch_bounds__(256) void fork_copy(Tree t, Pool pl, const int32_t *__restrict__ src,
                                                 const int32_t *__restrict__ dst, int n_forks,
                                                 Grow g, float *A, int copies, int32_t *status) {
  if (status_failed(status) || !g.meta[0]) return;
  if ((int)blockIdx.x >= copies) {
    for (int e = blockIdx.x - copies; e < n_forks; e += gridDim.x - copies) {
      const float *from = A + t.tok_off[src[e]];
      float *to = A + t.tok_off[dst[e]];
      for (int p = threadIdx.x; p < g.n0[e]; p += 256) to[p] = from[p];
    }
    return;
  }
  const int P = pl.P, top = g.meta[1];
  const int row_vecs = pl.D * pl.esize / 16;
  const int64_t work = (int64_t)g.meta[2] * pl.L;
  const int64_t page_bytes = (int64_t)pl.Hkv * P * pl.D * pl.esize;
  const char *kb = static_cast<const char *>(pl.k), *vb = static_cast<const char *>(pl.v);
  for (int64_t w = blockIdx.x; w < work; w += copies) {
    const int x = (int)(w / pl.L), l = (int)(w % pl.L);
    const int e = last_at_most(g.first, n_forks, x);
    const int q = x - g.first[e];
    const int64_t a = t.page_table[t.page_off[src[e]] + q];
    const int64_t b = pl.free_stack[top - 1 - x];
    if (a < 0 || a >= pl.num_pages || b < 0 || b >= pl.num_pages) {
      if (threadIdx.x == 0) status_error(status, ARBOR_ECORRUPT);
      continue;
    }
    const int rows = min(P, g.c0[e] - q * P);
    if (l == 0) {
      if (threadIdx.x == 0) t.page_table[t.page_off[dst[e]] + q] = (int32_t)b;
      for (int r = threadIdx.x; r < P; r += 256)
        pl.slot_pos[b * P + r] = r < rows ? pl.slot_pos[a * P + r] : -1;
    }
    const int64_t from = ((int64_t)l * pl.num_pages + a) * page_bytes;
    const int64_t to = ((int64_t)l * pl.num_pages + b) * page_bytes;
    const int vecs = rows * row_vecs;               // of each head
    for (int h = 0; h < pl.Hkv; ++h) {
      const int64_t ho = (int64_t)h * P * pl.D * pl.esize;
      for (int y = threadIdx.x; y < vecs; y += 256) {
        const uint4 kv = *reinterpret_cast<const uint4 *>(kb + from + ho + y * 16);
        const uint4 vv = *reinterpret_cast<const uint4 *>(vb + from + ho + y * 16);
        store16_nt(const_cast<char *>(kb) + to + ho + y * 16, kv);
        store16_nt(const_cast<char *>(vb) + to + ho + y * 16, vv);
      }
    }
  }
}

// Threads of the plans of truncate and fork: a fork and a truncate of 4 blocks with 256 and
// 1,024 threads 13.6 and 14.5 us, of 48 15.4 and 16.4, of 256 16.8 and 17.7; of more a thread
// would take several.
inline int plan_threads(int n) { return n <= 256 ? 256 : kPlanThreads; }

bool carve(Grow &g, int n, void *workspace, size_t bytes) {
  Carve cv(workspace, bytes);
  g.c0 = cv.take<int32_t>(n);
  g.n0 = cv.take<int32_t>(n);
  g.first = cv.take<int32_t>(n);
  g.start = cv.take<int32_t>(n);
  g.freed = cv.take<int32_t>(n);
  g.rows = cv.take<int64_t>(n);
  g.meta = cv.take<int32_t>(4);
  return cv.ok;
}

}  // namespace

// (a list of strictly ascending ids has at most num_nodes entries)
size_t pages_workspace(const arbor_sizes_t *sz) { return (size_t)sz->num_nodes * 28 + 4096; }

int launch_extend(const arbor_geom_t *geom, arbor_tree_t *tree, arbor_pool_t *pool, int32_t *n_full,
                  const int32_t *nodes, int32_t n_seq, const int32_t *cu, int32_t n_tokens,
                  int64_t *slots, int32_t *positions, int64_t *tokens, int32_t *status,
                  void *workspace, size_t workspace_bytes, hipStream_t stream) {
  const Tree t = make_tree(tree);
  const Pool pl = make_pool(geom, pool);
  Grow g;
  if (!carve(g, n_seq, workspace, workspace_bytes)) return ARBOR_EWORKSPACE;
  // up to 4,096 tokens the plan's workgroup writes their rows itself
  const int rows_too = n_tokens <= 4 * kPlanThreads;
  // Few waves meet at a barrier sooner, but a thread that has two tokens waits twice: the
  // smallest group with a thread for each token and block.  (A truncate and an extend of 48
  // blocks with 256, 512 and 1,024 threads, us: 200 tokens 13.8, 13.8, 14.1; 288 tokens
  // 15.1, 14.0, 14.3; 640 tokens 16.4, 15.2, 14.6.)
  const int most = n_seq > n_tokens ? n_seq : n_tokens;
  const int threads = most <= 256 ? 256 : most <= 512 ? 512 : kPlanThreads;
  hipLaunchKernelGGL(extend_plan, dim3(1), dim3(threads), 0, stream, t, pl, n_full, nodes,
                     n_seq, cu, n_tokens, g, slots, positions, tokens, rows_too, status);
  if (!rows_too) {
    const int blocks = (n_tokens + 255) / 256 < 2048 ? (n_tokens + 255) / 256 : 2048;
    hipLaunchKernelGGL(extend_rows_kernel, dim3(blocks), dim3(256), 0, stream, t, pl, nodes, n_seq,
                       cu, n_tokens, g, slots, positions, tokens, status);
  }
  return hip_ok(hipGetLastError());
}

int launch_truncate(const arbor_geom_t *geom, arbor_tree_t *tree, arbor_pool_t *pool,
                    int32_t *n_full, const int32_t *nodes, const int32_t *keep, int32_t n_nodes,
                    float *A, int64_t *rows_seen, int32_t *status, void *workspace,
                    size_t workspace_bytes, hipStream_t stream) {
  const Tree t = make_tree(tree);
  const Pool pl = make_pool(geom, pool);
  if (n_nodes == 0) return ARBOR_OK;
  Grow g;
  if (!carve(g, n_nodes, workspace, workspace_bytes)) return ARBOR_EWORKSPACE;
  hipLaunchKernelGGL(truncate_plan, dim3(1), dim3(plan_threads(n_nodes)), 0, stream, t, pl,
                     n_full, nodes, keep, n_nodes, g, A != nullptr, status);
  hipLaunchKernelGGL(truncate_clear, dim3(128), dim3(256), 0, stream, t, pl, nodes, keep, n_nodes,
                     g, A, rows_seen, status);
  return hip_ok(hipGetLastError());
}

int launch_fork(const arbor_geom_t *geom, arbor_tree_t *tree, arbor_pool_t *pool, int32_t *n_full,
                const int32_t *src, const int32_t *dst, int32_t n_forks, float *A,
                int64_t *rows_seen, int32_t *status, void *workspace, size_t workspace_bytes,
                hipStream_t stream) {
  const Tree t = make_tree(tree);
  const Pool pl = make_pool(geom, pool);
  if (n_forks == 0) return ARBOR_OK;
  Grow g;
  if (!carve(g, n_forks, workspace, workspace_bytes)) return ARBOR_EWORKSPACE;
  hipLaunchKernelGGL(fork_plan, dim3(1), dim3(plan_threads(n_forks)), 0, stream, t, pl, n_full,
                     src, dst, n_forks, g, rows_seen, status);
  const int copies = 2048;
  const int marks = A ? (n_forks < 256 ? n_forks : 256) : 0;
  hipLaunchKernelGGL(fork_copy, dim3(copies + marks), dim3(256), 0, stream, t, pl, src, dst,
                     n_forks, g, A, copies, status);
  return hip_ok(hipGetLastError());
}

}  // namespace arbor
