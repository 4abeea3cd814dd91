// arbor_prefill_plan and arbor_tree_prefill_attn: causal attention of the packed new
// tokens of several blocks over their root-to-leaf chains (Sec. 1, Sec. 3).
//
// A tile is up to kRows query rows of one KV head: consecutive packed tokens, of
// one block or of several, times their G query heads.  Its keys are the union of
// its blocks' chains, in 16-slot sub-pages; each chain block carries the set of
// the tile's sequences below it, so that tokens of several blocks share the reads
// of the ancestors they have in common, and a row sees a key when its sequence is
// in the block's set and, in its own block, the slot is not after its own.
//
// The plan (once for all layers; one launch, or three for many tiles): cut the packed
// tokens into tiles; a wave per tile merges its chains; split the tiles whose keys outlast
// the others' into parts, so that a few rows over a long prompt fill the chip.  The
// attention runs one workgroup per (part, KV head) and a second launch joins the parts.
//
// Attention of a tile: a wave holds 32 rows.  S^T = K Q^T with 32x32 MFMA leaves
// each lane one row and half of the keys, so the softmax needs one exchange between
// two lanes only where a row's reference max moves; O^T += V^T P^T takes P as the B
// operand straight from those registers (the order of the keys within a step is the
// one in which S^T leaves them; V^T is read from LDS in the same order, through the
// transposing LDS read for bf16).  Keys and values come by direct loads to LDS
// through a buffer resource over the valid rows of a sub-page, which fills the
// others with zeros; those of the next step are issued before this step's products.
//
// What bounds it: the matrix and vector work of two waves a SIMD, each a chain of logits,
// exponentials and products, which overlap in part.  A step of 64 keys is 1.05 MFLOP of
// products a wave; 8,192 tokens of the 70B shape (1.1 TFLOP) take 1.07 ms, 1.03 PFLOP/s (a
// library's 8,192^3 product: 1.3 to 1.5), of which the matrix units are busy for 50 %; a wave
// waits for its unit in 34 % of its cycles and for data in 25 %.  The same without data
// movement takes 0.88 ms; left out one by one, the loads to LDS are 0.12 ms, the reads of K
// 0.05, of V, which are three products ahead, 0.02.  64 rows a wave halve the reads, but
// leave one wave to a SIMD, which ran 1.55 ms and more; 32 keys a step and three waves 1.77.
// fp32, 4,096 tokens: 132 TFLOP/s in the 70B shape, 115 in the 8B shape, of the 153 of a
// library's product.
#include <type_traits>

#include "arbor_internal.h"
#include "mfma_ops.h"

namespace arbor {

namespace {

constexpr int kRows = 128;              // query rows of a tile: four waves of 32
constexpr int kWaves = kRows / 32;
constexpr int kMaxSeq = 64;             // sequences of a tile: one bit each
constexpr int MAXD = ARBOR_MAX_DEPTH + 1;
constexpr int kEntLds = 128;            // chain blocks of a tile that are kept in LDS (if all)
constexpr int64_t kMagic = 0x61726270726c6601;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
// A row's reference max moves when the terms of some lane add up to more than this:
// until then p = 2^(s - ref) may exceed 1, which costs no precision in fp32 or bf16
// and leaves V 2^100 of headroom, and a step needs neither a max nor a rescale.
constexpr float kMoveAt = 65536.0f;
// Workgroups that the chip holds at a time (two to each of 256 CUs).  Parts for 256 of them
// instead: 64 drafts below 15,000 tokens, two layers, 277 us against 220; 16 ragged blocks
// over a tree, four layers, 240 against 206.
constexpr int kSlots = 512;
// Sub-pages of a step, and steps of the shortest part: a part's fixed work (its way to its
// first key, its sums to memory and back) is worth about two steps.  At 2, 4 and 8 steps
// of 64 keys the 16 blocks above take 206, 206 and 222 us, 16 over a thinned tree 139, 149
// and 149; at one and two steps of 32 keys 48 fp32 tokens over 160 take 26 us, at four 32.
__host__ __device__ constexpr int step_subs(int bytes) { return bytes == 2 ? 4 : 2; }
constexpr int kMinSteps = 2;

struct Header {
  int64_t magic;
  int32_t n_seq, n_tokens, V, G, Hkv, page_size, n_tiles, n_units, n_split;
  int64_t table;                 // entries of the page table
};

struct Tile {
  int32_t t0, nt;       // packed tokens
  int32_t e0, ne;       // sequences that they belong to
  int32_t n_ent;        // chain blocks, at entry kMaxSeq... (see entry_base)
  int32_t n_sub;        // sub-pages of all of them
};

// One chain block of a tile, root first.
struct __attribute__((aligned(16))) Entry {
  int32_t node;
  int32_t limit;        // slots that some row of the tile sees
  int32_t sub0;         // sub-pages of the blocks before it
  int32_t po;           // its first page-table entry
  uint64_t below;       // the tile's sequences whose chain holds it
  uint64_t own;         // those whose own block it is
};

// What a workgroup takes: a part of a tile, and all that it has to know of the tile.
struct __attribute__((aligned(16))) Unit {
  int32_t t0, nt;       // its packed tokens
  int32_t n_ent, part;  // chain blocks; its partial, or -1: the whole tile
  int32_t s0, s1;       // sub-pages [s0, s1)
  int64_t ent;          // first chain block
};

struct PlanPtrs {
  Header *head;
  Tile *tiles;
  Entry *ents;
  Unit *units;
  int4 *split;          // tiles in parts: t0, nt, first partial, parts
  int2 *tok;            // per packed token: own slot, sequence within its tile
  int64_t tiles_cap, units_cap;
};

__host__ __device__ inline int tokens_per_tile(int G) { return kRows / G; }

// Bounds on the tiles and units of a call, known to the host.
inline int64_t tile_bound(int G, int n_seq, int64_t n_tokens) {
  // two neighbouring tiles hold more tokens than one may, or end a run of 64 sequences
  const int64_t b = 2 * (n_tokens / tokens_per_tile(G)) + n_seq / kMaxSeq + 2;
  return b < n_tokens ? b : n_tokens;
}
__host__ __device__ inline int target_parts(int Hkv) {
  const int t = kSlots / Hkv;
  return t > 0 ? t : 1;
}

// Workgroups of the join.  Of one block with twice as many tiles as the chip holds for a KV
// head, none has more than about twice the average's keys, so none is cut, unless most of
// the packed rows are padding, which only the device knows: a few workgroups see to that,
// one item after the other (2 us a layer of 160 where there is none, 4,096 tokens of the 8B
// shape; with as many as elsewhere 6).
inline int64_t join_groups(const arbor_geom_t *g, int n_seq, int n_tokens, int64_t tiles) {
  const int target = target_parts(g->num_kv_heads);
  const int64_t cut = tiles < target / 2 ? tiles : target / 2;     // (two parts or more each)
  const int64_t all = cut * g->num_kv_heads * kWaves;
  const bool whole = n_seq == 1 && n_tokens / tokens_per_tile(g->q_per_kv) >= 2 * target;
  return whole && all > 256 ? 256 : all;
}

PlanPtrs carve_plan(const arbor_geom_t *g, int n_seq, int n_tokens, void *plan, size_t bytes,
                    size_t *need) {
  PlanPtrs p{};
  p.tiles_cap = tile_bound(g->q_per_kv, n_seq, n_tokens);
  p.units_cap = p.tiles_cap + target_parts(g->num_kv_heads) + 1;
  Carve cv(plan, bytes);
  p.head = cv.take<Header>(1);
  p.tiles = cv.take<Tile>(p.tiles_cap + 1);
  p.ents = cv.take<Entry>((size_t)kMaxSeq * ((size_t)n_seq + p.tiles_cap + 1));
  p.units = cv.take<Unit>(p.units_cap);
  p.split = cv.take<int4>(target_parts(g->num_kv_heads) + 1);
  p.tok = cv.take<int2>((size_t)n_tokens + 1);
  if (need) *need = cv.off;
  if (!cv.ok) p.head = nullptr;
  return p;
}

// A tile's region of the entries: a chain has at most MAXD = kMaxSeq blocks, and the
// (tile, sequence) pairs before tile k are at most e0 + k.
static_assert(MAXD == kMaxSeq, "entry regions");
__host__ __device__ inline int64_t entry_base(int tile, int e0) {
  return (int64_t)kMaxSeq * (e0 + tile);
}

// ---- plan ---------------------------------------------------------------------
// Whether the request is sound: ids, cu, and as many resident tokens as are new.  Called
// by a whole workgroup.
// cu_lds, if given, holds cu afterwards.
__device__ bool request_ok(const Tree &t, const int32_t *__restrict__ nodes, int n_seq,
                           const int32_t *__restrict__ cu, int n_tokens, int32_t *cu_lds) {
  int err = threadIdx.x == 0 && (cu[0] != 0 || cu[n_seq] < 0 || cu[n_seq] > n_tokens);
  for (int e = threadIdx.x; e < n_seq; e += blockDim.x) {
    const int i = nodes[e], c0 = cu[e], c1 = cu[e + 1], m = c1 - c0;
    if (cu_lds) {
      cu_lds[e] = c0;
      if (e == n_seq - 1) cu_lds[n_seq] = c1;
    }
    if (i < 0 || i >= t.V || m < 0 || m > n_tokens) err = 1;
    else if (m > t.n_kept[i]) err = 1;
  }
  return !__syncthreads_or(err);
}

// Cuts the packed tokens into tiles; one wave.  A tile takes the next blocks' tokens as
// long as all of a block's fit (two blocks in one tile read the blocks that they share once,
// and nothing twice); a block of more tokens than a tile holds starts its own.  From where a
// tile starts with a block follows where the next one does: lanes find that for 64 blocks at
// a time, and the wave follows these links from the first block on.  Returns how many tiles
// there are.
__device__ int cut_tiles(int G, int n_seq, const int32_t *cu, Tile *tiles, int tiles_cap,
                         int32_t *status) {
  const int lane = lane_id(), TQ = tokens_per_tile(G);
  int k = 0, at = 0;                       // at: the block that the next tile starts with
  for (int e0 = 0; e0 < n_seq; e0 += kWave) {
    const int e = e0 + lane;
    int c0 = 0, full = 0, t = 0, nt = 0, next = e + 1;
    if (e < n_seq) {
      c0 = cu[e];
      const int m = cu[e + 1] - c0;
      full = m / TQ;                       // whole tiles of this block alone
      t = c0 + full * TQ;
      if (m > full * TQ) {                 // the rest of it, and the blocks that fit
        int hi = min(n_seq, e + kMaxSeq);  // last next with cu[next] <= t + TQ
        while (next < hi) {
          const int mid = (next + hi + 1) / 2;
          if (cu[mid] <= t + TQ) next = mid;
          else hi = mid - 1;
        }
        nt = cu[next] - t;
      }
    }
    uint64_t path = 0;
    while (at < min(e0 + kWave, n_seq)) {
      path |= 1ull << (at - e0);
      at = lane_value(next, at - e0);
    }
    const bool on = path >> lane & 1;
    const int mine = on ? full + (nt > 0) : 0;
    const int inc = wave_inclusive_scan(mine), k0 = k + inc - mine;
    constexpr int FEW = 4;                 // tiles that a lane lists by itself
    for (int x = 0; x < FEW; ++x)
      if (on && x < full && k0 + x < tiles_cap) tiles[k0 + x] = Tile{c0 + x * TQ, TQ, e, 1, 0, 0};
    for (uint64_t s = ballot(on && full > FEW); s; s &= s - 1) {
      const int j = __builtin_ctzll(s), c = lane_value(c0, j), f = lane_value(full, j),
                b = lane_value(k0, j);
      for (int x = FEW + lane; x < f; x += kWave)
        if (b + x < tiles_cap) tiles[b + x] = Tile{c + x * TQ, TQ, e0 + j, 1, 0, 0};
    }
    if (on && nt > 0 && k0 + full < tiles_cap) tiles[k0 + full] = Tile{t, nt, e, next - e, 0, 0};
    k += lane_value(inc, kWave - 1);
  }
  if (k > tiles_cap) {                                // (the bound holds)
    if (lane == 0) status_error(status, ARBOR_ECORRUPT);
    k = tiles_cap;
  }
  return k;
}

__device__ void write_header(const PlanPtrs &p, const Tree &t, int G, int Hkv, int P, int n_seq,
                             int n_tokens, int n_tiles) {
  p.head->n_seq = n_seq;
  p.head->n_tokens = n_tokens;
  p.head->V = t.V;
  p.head->table = t.page_off[t.V];
  p.head->G = G;
  p.head->Hkv = Hkv;
  p.head->page_size = P;
  p.head->n_tiles = n_tiles;
}

constexpr int kCol = kWave + 1;          // chains lie side by side, [MAXD][kCol], leaf first

// The chain of the block x (none for x < 0) into column col: its length, or an error code.
template <class C>
__device__ int walk_chain(const int32_t *parent, int x, C *chain, int col) {
  int depth = 0;
  while (x >= 0) {
    if (depth == MAXD) return ARBOR_EUNSUPPORTED;
    chain[depth * kCol + col] = (C)x;
    ++depth;
    const int up = parent[x];
    if (up >= x) return ARBOR_EINVAL;
    x = up;
  }
  return depth;
}

// Tile k's chain blocks, and its tokens' own slots; one wave.  Lane j's sequence has its
// chain, `depth` blocks, in column col.  Blocks come in ascending order of ids, so the next
// one is the smallest id that any lane has next; 64 of them wait in the lanes.
// False if a block has more slots to see than pages: so every entry's slots lie within the
// page table.
template <class C, class O>
__device__ bool merge_chains(const int32_t *n_kept, const O *page_off, int P, const int32_t *cu,
                             const PlanPtrs &p, int k, Tile *tile, const C *chain, int col,
                             int depth) {
  const int lane = lane_id();
  const Tile tl = *tile;
  Entry *ents = p.ents + entry_base(k, tl.e0);
  int lo = 0, hi = 0, leaf = -1, newest = -1;
  if (lane < tl.ne) {
    const int c0 = cu[tl.e0 + lane], c1 = cu[tl.e0 + lane + 1];
    lo = max(c0, tl.t0);
    hi = min(c1, tl.t0 + tl.nt);
    if (hi > lo) {
      leaf = chain[col];
      newest = n_kept[leaf] - (c1 - hi) - 1;    // slot of the sequence's last token here
    }
  }
  int subs = 0, n = 0;
  Entry mine{};
  bool bad = false;
  auto flush = [&](int cnt) {
    int need = 0;
    if (lane < cnt) {
      if (mine.below != mine.own) mine.limit = n_kept[mine.node];
      const int64_t po = page_off[mine.node], end = page_off[mine.node + 1];
      mine.po = (int32_t)po;
      bad = bad || mine.limit < 0 || po < 0 || (end - po) * P < mine.limit;
      need = mine.limit / 16 + (mine.limit % 16 > 0);
    }
    const int inc = wave_inclusive_scan(need);
    mine.sub0 = subs + inc - need;
    if (lane < cnt) ents[(n - 1) / kWave * kWave + lane] = mine;
    subs += lane_value(inc, kWave - 1);
  };
  int at = leaf >= 0 ? depth - 1 : -1;
  if (tl.ne == 1) {                                // one chain: nothing to merge
    n = lane_value(at, 0) + 1;
    if (lane < n) {
      mine.node = chain[(n - 1 - lane) * kCol + lane_value(col, 0)];
      mine.limit = lane_value(newest, 0) + 1;
      mine.below = 1;
      mine.own = lane == n - 1;
    }
    if (n) flush(n);
  } else while (true) {
    const int next = at >= 0 ? (int)chain[at * kCol + col] : INT32_MAX;
    const int mn = wave_allreduce(next, [](int a, int b) { return a < b ? a : b; });
    if (mn == INT32_MAX) break;
    const bool here = next == mn;
    const uint64_t below = ballot(here), own = ballot(here && mn == leaf);
    int last = -1;
    if (own) last = wave_allreduce(here && mn == leaf ? newest : -1,
                                   [](int a, int b) { return a > b ? a : b; });
    if (lane == n % kWave) {
      mine.node = mn;
      mine.limit = last + 1;
      mine.below = below;
      mine.own = own;
    }
    at -= here ? 1 : 0;
    if (++n % kWave == 0) flush(kWave);
  }
  if (tl.ne > 1 && n % kWave) flush(n % kWave);
  if (lane == 0) {
    tile->n_ent = n;
    tile->n_sub = subs;
  }
  // own slot and sequence of each of its tokens
  for (int j = 0; j < tl.ne; ++j) {
    const int l = lane_value(lo, j), h = lane_value(hi, j), last = lane_value(newest, j);
    for (int y = l + lane; y < h; y += kWave) p.tok[y] = int2{last - (h - 1 - y), j};
  }
  return !ballot(bad);
}

// Long tiles are cut into parts, and all parts listed, longest first.  Parts are in
// proportion to a tile's keys, rounded down: all parts together are no more than `target`
// and the uncut tiles, so that they run at once.
struct Cut {
  double per;            // parts per sub-page
  int min_part;
  __device__ Cut(int target, int64_t total, int least)
      : per(total > 0 ? (double)target / (double)total : 0.0), min_part(least) {}
  __device__ int parts(int s) const { return max(1, min((int)(s * per), s / min_part)); }
  __device__ static int length(int s, int np) { return (s + np - 1) / np; }
};

// The np parts of tile k, from unit u and partial part0 on, by a wave.
__device__ void list_parts(const PlanPtrs &p, int k, const Tile &tl, int np, int u, int part0) {
  const int len = tl.n_sub / np, more = tl.n_sub % np;     // the first `more` have one more
  for (int x = lane_id(); x < np; x += kWave)
    if (u + x < p.units_cap)
      p.units[u + x] = Unit{tl.t0, tl.nt, tl.n_ent, part0 + x, len * x + min(x, more),
                            len * (x + 1) + min(x + 1, more), entry_base(k, tl.e0)};
}

__device__ void write_counts(const PlanPtrs &p, int units, int split, int target,
                             int32_t *status) {
  p.head->n_units = units;
  p.head->n_split = split;
  if (units > p.units_cap || split > target) status_error(status, ARBOR_ECORRUPT);
  else p.head->magic = kMagic;
}

// Up to 64 tiles: four waves, one to a SIMD, have them all in their lanes and find their
// order alone, a tile at a time; wave w lists the parts of the tiles 4 x + w.  (One tile in
// three parts takes 2.1 us less than below, which waits at eight barriers.)
__device__ void list_few(const PlanPtrs &p, const Tile *tiles, int n, int target, int min_part,
                         int32_t *status) {
  const int lane = lane_id(), wave = threadIdx.x / kWave, waves = 4;
  if (wave >= waves) return;
  Tile tl{};
  if (lane < n) tl = tiles[lane];
  const Cut cut(target, wave_sum((int64_t)tl.n_sub), min_part);
  const int np = lane < n ? cut.parts(tl.n_sub) : 0;
  const int len = np ? Cut::length(tl.n_sub, np) : 0;
  const int many = np > 1 ? np : 0, part0 = wave_inclusive_scan(many) - many;
  const uint64_t split = ballot(np > 1);
  int u0 = 0, units = 0;
  for (int j = 0; j < n; ++j) {
    const int l = lane_value(len, j), m = lane_value(np, j);
    u0 += l > len || (l == len && j < lane) ? m : 0;
    units += m;
  }
  if (wave == 0) {
    if (np > 1) {
      const int x = popc(split & ((1ull << lane) - 1));
      if (x < target) p.split[x] = int4{tl.t0, tl.nt, part0, np};
    } else if (np == 1 && u0 < p.units_cap) {
      p.units[u0] = Unit{tl.t0, tl.nt, tl.n_ent, -1, 0, tl.n_sub, entry_base(lane, tl.e0)};
    }
    if (lane == 0) write_counts(p, units, popc(split), target, status);
  }
  for (int j = wave; j < n; j += waves)
    if (split >> j & 1) list_parts(p, j, tiles[j], lane_value(np, j), lane_value(u0, j),
                                   lane_value(part0, j));
}

// Any number of tiles; a workgroup of up to 16 waves.
__device__ void list_units(const PlanPtrs &p, const Tile *tiles, int n, int target, int min_part,
                           int32_t *status) {
  constexpr int NB = 256;
  __shared__ int64_t sm[2 * 16];
  __shared__ int32_t bucket[NB + 1], longest;
  // neighbouring tiles go to different waves: each wave has as many to list
  const int nt = blockDim.x, lane = lane_id(), waves = nt / kWave;
  const int tid = threadIdx.x, own = lane * waves + tid / kWave;
  const Tile none{};
  const Tile first = own < n ? tiles[own] : none;
  int64_t subs = 0;
  for (int k = own; k < n; k += nt) subs += k == own ? first.n_sub : tiles[k].n_sub;
  const int64_t total = block_sum(subs, sm);
  for (int b = tid; b <= NB; b += nt) bucket[b] = 0;
  if (tid == 0) longest = 1;
  __syncthreads();
  const Cut cut(target, total, min_part);
  int64_t v[2] = {0, 0}, ex[2], tot[2];        // parts of cut tiles, cut tiles
  int far = 0;
  for (int k = own; k < n; k += nt) {
    const int s = k == own ? first.n_sub : tiles[k].n_sub, np = cut.parts(s);
    far = max(far, Cut::length(s, np));
    v[0] += np > 1 ? np : 0;
    v[1] += np > 1;
  }
  if (far > 1) atomicMax(&longest, far);
  block_exclusive_scan_n<2>(v, ex, tot, sm);
  const float scale = (float)(NB - 1) / (float)longest;
  auto bucket_of = [&](int len) { return NB - 1 - min(NB - 1, (int)((float)len * scale)); };
  for (int k = own; k < n; k += nt) {
    const int s = k == own ? first.n_sub : tiles[k].n_sub, np = cut.parts(s);
    atomicAdd(&bucket[bucket_of(Cut::length(s, np))], np);
  }
  __syncthreads();
  if (tid < kWave) {
    int base = 0;
    for (int b = 0; b < NB; b += kWave) {
      const int c = bucket[b + tid];
      const int inc = wave_inclusive_scan(c);
      bucket[b + tid] = base + inc - c;
      base += lane_value(inc, kWave - 1);
    }
    if (tid == 0) bucket[NB] = base;
  }
  __syncthreads();
  const int units = bucket[NB];
  for (int k0 = own - lane * waves; k0 < n; k0 += nt) {      // a wave's 64 tiles
    const int k = k0 + lane * waves;
    Tile tl = none;
    int np = 0, u0 = 0, part0 = 0;
    if (k < n) {
      tl = k == own ? first : tiles[k];
      np = cut.parts(tl.n_sub);
      u0 = atomicAdd(&bucket[bucket_of(Cut::length(tl.n_sub, np))], np);
      part0 = (int)ex[0];
      if (np > 1) {
        if (ex[1] < target) p.split[ex[1]] = int4{tl.t0, tl.nt, part0, np};
        ++ex[1];
        ex[0] += np;
      } else if (u0 < p.units_cap) {
        p.units[u0] = Unit{tl.t0, tl.nt, tl.n_ent, -1, 0, tl.n_sub, entry_base(k, tl.e0)};
      }
    }
    for (uint64_t m = ballot(np > 1); m; m &= m - 1) {      // a wave lists the parts
      const int j = __builtin_ctzll(m);
      list_parts(p, k0 + j * waves, tiles[k0 + j * waves], lane_value(np, j), lane_value(u0, j),
                 lane_value(part0, j));
    }
  }
  if (tid == 0) write_counts(p, units, (int)tot[1], target, status);
}

// The whole plan of a call with few blocks and tiles, in one launch: a wave walks all
// chains beside one that cuts the tiles, then 16 waves merge them.  What bounds it is the
// latency of one access after the other, so all that it reads twice is in LDS.
// In one launch and in three: 48 tokens 6.7 and 11.9 us, 16 blocks of 128 13.1 and 16.0, 64
// blocks of 8 11.0 and 15.8, one block of 512, 1,024 and 2,048 tokens 7.3 and 13.0, 9.9 and
// 13.4, 12.8 and 12.9.  The last of these may have 130 tiles (it has 64).
constexpr int kSmallTiles = 130, kSmallV = 4096;
__global__ __launch_bounds__(1024) void plan_small(Tree t, int G, int Hkv, int P,
                                                   const int32_t *__restrict__ nodes, int n_seq,
                                                   const int32_t *__restrict__ cu, int n_tokens,
                                                   PlanPtrs p, int target, int min_part,
                                                   int32_t *status) {
  __shared__ int32_t depth[kWave], sh_cu[kWave + 1];
  __shared__ int32_t sh_parent[kSmallV], sh_kept[kSmallV], sh_page_off[kSmallV + 1];
  __shared__ uint16_t chain[MAXD * kCol];
  __shared__ Tile tiles[kSmallTiles];
  __shared__ int n_tiles, bad;
  const int wave = threadIdx.x >> 6, lane = lane_id();
  const int leaf = wave == 1 && lane < n_seq ? nodes[lane] : -1;
  for (int i = threadIdx.x; i <= t.V; i += 1024) {
    const int j = min(i, t.V - 1);                 // (no branch: all loads are in flight together)
    const int up = t.parent[j], kept = t.n_kept[j];
    sh_page_off[i] = (int32_t)t.page_off[i];
    sh_parent[j] = up;
    sh_kept[j] = kept;
  }
  if (threadIdx.x == 0) {
    p.head->magic = 0;
    bad = 0;
  }
  if (status_failed(status)) return;
  if (!request_ok(t, nodes, n_seq, cu, n_tokens, sh_cu)) {
    if (threadIdx.x == 0) status_error(status, ARBOR_EINVAL);
    return;
  }
  int err = 0;
  if (wave == 0) {
    const int n = cut_tiles(G, n_seq, sh_cu, tiles, kSmallTiles, status);
    if (lane == 0) n_tiles = n;
  } else if (wave == 1) {
    const int d = walk_chain(sh_parent, leaf, chain, lane);
    depth[lane] = d;
    err = d < 0 ? d : 0;
  }
  if (__syncthreads_or(err)) {
    if (err) status_error(status, err);
    return;
  }
  for (int k = wave; k < n_tiles; k += 16) {
    const int col = min(tiles[k].e0 + lane, kWave - 1);
    if (!merge_chains(sh_kept, sh_page_off, P, sh_cu, p, k, &tiles[k], chain, col, depth[col]) &&
        lane == 0)
      bad = 1;
  }
  if (threadIdx.x == 0) write_header(p, t, G, Hkv, P, n_seq, n_tokens, n_tiles);
  __syncthreads();
  if (bad) {
    if (threadIdx.x == 0) status_error(status, ARBOR_EINVAL);
    return;
  }
  if (n_tiles <= kWave) list_few(p, tiles, n_tiles, target, min_part, status);
  else list_units(p, tiles, n_tiles, target, min_part, status);
}

// The same in three launches: tiles, a wave for each tile's chains, parts.
constexpr int kCuLds = 4096;
__global__ __launch_bounds__(1024) void plan_tiles(Tree t, int G, int Hkv, int P,
                                                   const int32_t *__restrict__ nodes, int n_seq,
                                                   const int32_t *__restrict__ cu, int n_tokens,
                                                   PlanPtrs p, int32_t *status) {
  __shared__ int32_t sh_cu[kCuLds + 1];
  if (threadIdx.x == 0) p.head->magic = 0;
  if (status_failed(status)) return;
  const bool in_lds = n_seq <= kCuLds;
  if (!request_ok(t, nodes, n_seq, cu, n_tokens, in_lds ? sh_cu : nullptr)) {
    if (threadIdx.x == 0) status_error(status, ARBOR_EINVAL);
    return;
  }
  if (threadIdx.x >= kWave) return;
  const int n = in_lds ? cut_tiles(G, n_seq, sh_cu, p.tiles, (int)p.tiles_cap, status)
                       : cut_tiles(G, n_seq, cu, p.tiles, (int)p.tiles_cap, status);
  if (threadIdx.x == 0) write_header(p, t, G, Hkv, P, n_seq, n_tokens, n);
}
__global__ __launch_bounds__(64) void plan_chains(Tree t, int P,
                                                  const int32_t *__restrict__ nodes,
                                                  const int32_t *__restrict__ cu, PlanPtrs p,
                                                  int32_t *status) {
  __shared__ int32_t chain[MAXD * kCol];
  // (one read for the wave: other tiles may raise an error meanwhile)
  if (__builtin_amdgcn_readfirstlane(status_word(status)) < 0 ||
      (int)blockIdx.x >= p.head->n_tiles)
    return;
  const int lane = lane_id(), e0 = p.tiles[blockIdx.x].e0, ne = p.tiles[blockIdx.x].ne;
  const int d = walk_chain(t.parent, lane < ne ? nodes[e0 + lane] : -1, chain, lane);
  if (d < 0) status_error(status, d);
  if (ballot(d < 0)) return;
  if (!merge_chains(t.n_kept, t.page_off, P, cu, p, blockIdx.x, &p.tiles[blockIdx.x], chain, lane,
                    d) && lane == 0)
    status_error(status, ARBOR_EINVAL);
}
__global__ __launch_bounds__(1024) void plan_units(PlanPtrs p, int target, int min_part,
                                                   int32_t *status) {
  if (status_failed(status)) return;
  list_units(p, p.tiles, p.head->n_tiles, target, min_part, status);
}

// ---- attention -------------------------------------------------------------------
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) void *LdsPtr;

// What the two element types differ in.  KS: MFMA steps over head_dim; a lane's
// operand of step ks are the elements 16-byte piece 2 (ks / SPP) + h of a row, h the
// lane's half of the wave.
template <class T, int D>
struct Cfg {
  static constexpr int ES = (int)sizeof(T);
  static constexpr int ROW = D * ES;                     // bytes of a row
  static constexpr int PIECES = ROW / 16;
  static constexpr int SUBS = step_subs(ES);           // sub-pages of a step
  static constexpr int KEYS = 16 * SUBS;
  static constexpr int NS = KEYS / 32;                   // 32-key tiles of S
  static constexpr int BUF = KEYS * ROW;                 // K (or V) of a step
  static constexpr int LPS = 16 * ROW / 1024;            // 1 KB loads of a sub-page
  static constexpr int DT = D / 32;
  static constexpr int NQ = ROW / 32;                    // 16-byte operand pieces of a lane
  static constexpr int LDS = 4 * BUF;
  static constexpr int PK = ES == 2 ? 16 : 2;            // keys of an MFMA of O
  // How the places of pieces (below) differ, as an exclusive or of byte offsets: of rows
  // 1024 / ROW apart (times c, V's masked), of a lane's K operands 2 pieces apart, and of
  // its V operands 32 columns apart
  static constexpr int FLIP_K = PIECES == 8 ? 64 : 16 * 1024 / ROW;
  static constexpr int FLIP_V = ES == 2 ? 0 : 32 * 1024 / ROW, FLIP_V_MASK = 128;
  static constexpr int STEP_K = 32, STEP_V = ES == 2 ? 64 : 128;
};

// Where piece x of row r of a step's K lies: rows 0..15 (of 16-lane groups that read
// one piece) fall on distinct banks.  The exclusive or lets a lane step through its
// pieces from one address.
template <class T, int D>
__device__ __forceinline__ int k_piece(int r, int x) {
  constexpr int N = Cfg<T, D>::PIECES;
  if constexpr (N == 8) return x ^ ((r >> 1) & 7);
  else return x ^ (r & (N - 1) & 31);
}
// The same of V: the four rows that a transposing read takes 64 bytes of (bf16), or
// the two rows of an fp32 read, fall on distinct banks.
template <class T, int D>
__device__ __forceinline__ int v_piece(int r, int x) {
  constexpr int N = Cfg<T, D>::PIECES;
  if constexpr (sizeof(T) == 4) return x ^ (((r >> 2) & 1) << 3);
  else if constexpr (N == 8) return x ^ (((r >> 1) & 1) << 2);
  else return x ^ ((r & 3) << 2);
}

struct AttnArgs {
  Tree t;
  Pool pl;
  PlanPtrs p;
  int n_seq, n_tokens, layer;
  const void *q;
  void *out;
  float *lse;
  float sl2;            // softmax scale in log2 units
  float *part;          // [parts][Hkv][kWaves][part_floats]
  int64_t part_cap;     // parts that it holds
  int32_t *status;
};

// Floats of a wave's rows in a part: their sums, then their references and sums of terms.
template <int D>
__host__ __device__ constexpr int part_floats() { return 32 * (D + 2); }

// Direct loads to LDS of the rows of one sub-page, `bytes` of which are valid: 16
// bytes a lane, load c from (off ^ (c FLIP & MASK)) + 1024 c to dst + 1024 c.  The buffer
// resource (scalar registers) bounds every access; beyond it zeros are written.
//
// As assembly, which the compiler does not take for a write to LDS: after its builtin it
// waits for all loads in flight before the next read of LDS, whichever buffer that reads,
// so a step's loads had no step to arrive in.  The kernel waits itself, by
// landed_barrier().  The instructions have no result in registers.
// (host-device so the kernel's host-device lambdas can call it; the host pass of the
// compiler never runs it)
template <int N, int FLIP, int MASK>
__host__ __device__ __forceinline__ void load_sub_page(const char *src, int bytes, uint32_t dst,
                                                       int off) {
#if defined(__HIP_DEVICE_COMPILE__)
  const uint64_t base = reinterpret_cast<uint64_t>(src);
  const u32x4 rsrc = {(uint32_t)base, (uint32_t)(base >> 32) & 0xffff, (uint32_t)bytes, 0x00020000};
  // (the instruction's offset, at most 4095, moves both ends)
#define ARBOR_LOAD(C)                                                                           \
  if constexpr (C < N)                                                                          \
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen offset:%c3 lds" \
               :: "s"(dst + C / 4 * 4096), "v"((off ^ (C * FLIP & MASK)) + C / 4 * 4096),       \
               "s"(rsrc), "i"(C % 4 * 1024) : "memory", "m0")
  ARBOR_LOAD(0);
  ARBOR_LOAD(1);
  ARBOR_LOAD(2);
  ARBOR_LOAD(3);
  ARBOR_LOAD(4);
  ARBOR_LOAD(5);
  ARBOR_LOAD(6);
  ARBOR_LOAD(7);
#undef ARBOR_LOAD
#endif
}
// Every direct load of the wave has landed, and every wave of the workgroup is here.
__host__ __device__ __forceinline__ void landed_barrier() {
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
#endif
}

// (the matrix instructions and the transposing read, host-device for the same reason)
__host__ __device__ __forceinline__ f32x16 mfma_bf16(bf16x8 x, bf16x8 y, f32x16 c) {
#if defined(__HIP_DEVICE_COMPILE__)
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, y, c, 0, 0, 0);
#else
  return c;
#endif
}
__host__ __device__ __forceinline__ f32x16 mfma_f32(float x, float y, f32x16 c) {
#if defined(__HIP_DEVICE_COMPILE__)
  return __builtin_amdgcn_mfma_f32_32x32x2f32(x, y, c, 0, 0, 0);
#else
  return c;
#endif
}
// Nothing is scheduled across this place.
__host__ __device__ __forceinline__ void fence_order() {
#if defined(__HIP_DEVICE_COMPILE__)
  __builtin_amdgcn_sched_barrier(0);
#endif
}
// Column of eight keys: four rows from p on and four from `next` bytes further on.
__host__ __device__ __forceinline__ bf16x8 read_transposed(const char *p, int next) {
#if defined(__HIP_DEVICE_COMPILE__)
  typedef short s16x4 __attribute__((ext_vector_type(4)));
  typedef __attribute__((address_space(3))) s16x4 *P4;
  const bf16x4 a = __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((P4)p));
  const bf16x4 b =
      __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((P4)(p + next)));
  return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
#else
  return bf16x8{};
#endif
}

__device__ __forceinline__ float swap_halves_add(float v) {
  float a, b;
  row_swap<true>(v, a, b);
  return a + b;
}
__device__ __forceinline__ float swap_halves_max(float v) {
  float a, b;
  row_swap<true>(v, a, b);
  return fmaxf(a, b);
}

// One sub-page per lane, 64 of them: read by readlane.
struct Window {
  int page;
  int info;      // first row of the page / 16 | valid rows << 8 | flags << 16
  int ent;       // chain block
};
constexpr int kMask = 1 << 16;   // some row of this wave must not see some key of it
constexpr int kNone = 1 << 17;   // no row of this wave sees any

// Whether the plan, whose header is h, is of this call and tree.
__device__ __forceinline__ bool header_ok(const AttnArgs &a, const Header &h, int64_t table) {
  return (h.magic == kMagic) & (h.n_seq == a.n_seq) & (h.n_tokens == a.n_tokens) &
         (h.V == a.t.V) & (h.table == table) & (h.G == a.pl.G) & (h.Hkv == a.pl.Hkv) &
         (h.page_size == a.pl.P);
}

template <class T, int D>
__global__ __launch_bounds__(kRows * 2, 2) void prefill_attn(AttnArgs a) {
  typedef Cfg<T, D> C;
  extern __shared__ __attribute__((aligned(16))) char lds[];
  __shared__ Entry sh_ent[kEntLds];
  __shared__ int32_t sh_status;
  const Pool &pl = a.pl;
  const int g = blockIdx.x % pl.Hkv, u = blockIdx.x / pl.Hkv;
  // (in one round trip: the status, the header, and the unit whether there is one or not)
  const int32_t status = status_word(a.status);
  Header head_of = *a.p.head;
  const int64_t table = a.t.page_off[a.t.V];
  Unit un = a.p.units[u];
  // (no load moves below the branches)
  asm volatile("" : "+s"(head_of.n_units), "+s"(un.t0), "+s"(un.nt), "+s"(un.n_ent), "+s"(un.part),
               "+s"(un.s0), "+s"(un.s1), "+s"(un.ent));
  if (!header_ok(a, head_of, table)) {
    if (blockIdx.x == 0 && threadIdx.x == 0) status_error(a.status, ARBOR_EINVAL);
    return;
  }
  if (u >= head_of.n_units) return;
  // (global and LDS reads of a block stay apart: a pointer that may be either makes flat
  // loads, which wait for both kinds)
  typedef const __attribute__((address_space(1))) Entry *GlobalEnt;
  const GlobalEnt ents = (GlobalEnt)(a.p.ents + un.ent);
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lr = lane & 31, h = lane >> 5;
  const bool ents_lds = un.n_ent <= kEntLds;
  auto planned = [&](int x) __attribute__((always_inline)) -> Entry {
    Entry e;
    e.node = ents[x].node, e.limit = ents[x].limit, e.sub0 = ents[x].sub0, e.po = ents[x].po;
    e.below = ents[x].below, e.own = ents[x].own;
    return e;
  };
  auto entry = [&](int x) __attribute__((always_inline)) -> Entry {
    return ents_lds ? sh_ent[x] : planned(x);
  };
  // the tile's first blocks, this lane's row and its query are loaded together
  const Entry staged = planned(min(tid, un.n_ent - 1));

  // this lane's row
  const int G = pl.G, row = wave * 32 + lr;
  const int tq = row / G;
  const bool live = tq < un.nt;
  const int tok = un.t0 + (live ? tq : 0);
  const int head = g * G + (live ? row - tq * G : 0);
  const int2 info = a.p.tok[tok];
  const int qslot = info.x;
  const int Hq = pl.Hkv * G;
  // Q as the B operand: its row, pieces 2 i + h
  typedef typename std::conditional<sizeof(T) == 2, bf16x8, f32x4>::type qvec;
  typedef typename std::conditional<sizeof(T) == 2, bf16x8, float>::type pvec;
  qvec qf[C::NQ];
  {
    const T *qp = static_cast<const T *>(a.q) + ((int64_t)tok * Hq + head) * D;
#pragma unroll
    for (int i = 0; i < C::NQ; ++i)
      qf[i] = *reinterpret_cast<const qvec *>(qp + (2 * i + h) * (16 / C::ES));
  }
  const uint64_t seq_bit = live ? 1ull << (info.y & 63) : 0;
  const bool any_live = wave * 32 / G < un.nt;
  if (tid < kEntLds) sh_ent[tid] = staged;
  // one read of the status decides for the workgroup: others of this launch may find the
  // plan stale meanwhile
  if (tid == 0) sh_status = status;
  __syncthreads();
  if (sh_status < 0) return;
  // sequences and own slots of the wave's rows
  uint64_t seqs = wave_allreduce(seq_bit, [](uint64_t x, uint64_t y) { return x | y; });
  const int qmin = wave_allreduce(live ? qslot : INT32_MAX,
                                  [](int x, int y) { return x < y ? x : y; });
  const int qmax = wave_allreduce(live ? qslot : -1, [](int x, int y) { return x > y ? x : y; });

  const int n_sub = un.s1 - un.s0;
  const int steps = (n_sub + C::SUBS - 1) / C::SUBS;
  constexpr int WSTEPS = kWave / C::SUBS;         // steps of a window
  // sub-page w0 + lane of the unit
  bool stale = false;
  // (no branch that lanes take differently: the compiler would give the whole loop the
  // control flow, and the copies of O, that such branches need)
  const int ent_bits = 32 - __builtin_clz(un.n_ent);
  auto fill = [&](int w0) __attribute__((always_inline)) -> Window {
    const int sp = un.s0 + w0 + lane;
    const bool in = sp < un.s1;
    // the last block whose sub-pages start at or before this one (a block without a slot
    // to see starts where the next one does)
    int at = 0;
    for (int b = ent_bits - 1; b >= 0; --b) {
      const int up = at + (1 << b);
      const int first = entry(min(up, un.n_ent - 1)).sub0;
      at = up < un.n_ent && first <= sp ? up : at;
    }
    const Entry en = entry(at);
    const int slot = in ? (sp - en.sub0) * 16 : 0;
    const int page = a.t.page_table[(int64_t)en.po + slot / pl.P];
    const bool there = page >= 0 && page < pl.num_pages;
    stale = stale || (in && !there);             // the tree has changed since the plan
    const int valid = in && there ? min(16, en.limit - slot) : 0;
    const uint64_t mine = en.below & seqs, mown = en.own & seqs;
    const bool none = !in || mine == 0 || (mine == mown && slot > qmax);
    const bool mask = mine != seqs || valid < 16 || (mown && slot + 15 > qmin);
    return Window{in && there ? page : 0,
                  slot % pl.P / 16 | valid << 8 | (none ? kNone : mask ? kMask : 0),
                  at};
  };

  // the plane of this layer and head: pages are page_bytes apart
  const int64_t page_bytes = (int64_t)pl.Hkv * pl.P * C::ROW;
  const int64_t plane = (int64_t)a.layer * pl.num_pages * page_bytes + (int64_t)g * pl.P * C::ROW;
  const char *kpool = static_cast<const char *>(pl.k) + plane;
  const char *vpool = static_cast<const char *>(pl.v) + plane;
  // this wave's direct loads of a step: its share of the (sub-page, K or V) pairs
  const int my_sub = C::SUBS == 4 ? wave : wave & 1;
  // 16 bytes a lane: the piece that lies at byte 16 lane of the sub-page in LDS; 1024 c
  // further on it is 1024 / ROW rows later, whose places differ by FLIP_K c, FLIP_V c
  const int lane_row = 16 * lane / C::ROW, lane_x = 16 * lane % C::ROW / 16;
  const int koff = lane_row * C::ROW + 16 * k_piece<T, D>(my_sub * 16 + lane_row, lane_x);
  const int voff = lane_row * C::ROW + 16 * v_piece<T, D>(lane_row, lane_x);

  const uint32_t lds_base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds;
  // K and V of step st, whose sub-pages are in w, into the buffers at byte `at`
  auto issue = [&](const Window &w, int st, int at) __attribute__((always_inline)) {
    const int idx = st % WSTEPS * C::SUBS + my_sub;
    const int page = __builtin_amdgcn_readlane(w.page, idx);
    const int inf = __builtin_amdgcn_readlane(w.info, idx);
    const int64_t off = page * page_bytes + (inf & 255) * (16 * C::ROW);
    const int bytes = (inf >> 8 & 31) * C::ROW;
    const uint32_t dst = lds_base + at + my_sub * 16 * C::ROW;
    // bf16: sub-page `wave` of K and of V; fp32: sub-page wave % 2 of K or V
    if (C::SUBS == 4 || wave < 2)
      load_sub_page<C::LPS, C::FLIP_K, ~0>(kpool + off, bytes, dst, koff);
    if (C::SUBS == 4 || wave >= 2)
      load_sub_page<C::LPS, C::FLIP_V, C::FLIP_V_MASK>(vpool + off, bytes, dst + 2 * C::BUF, voff);
  };

  // this lane's operands in LDS: K row lr, piece 2 i + h at kat ^ (i STEP_K); V^T columns
  // 32 d + .. at vat ^ (d STEP_V)
  const int kat = lr * C::ROW + 16 * k_piece<T, D>(lr, h);
  int vat;
  if constexpr (sizeof(T) == 2) {
    // a transposing read of four keys: lane x of 16 addresses columns 4 (x % 4) .. of
    // key x / 4 and gets column x of the four
    const int x = lane & 15, key = 4 * h + (x >> 2), c = (lane & 16) + 4 * (x & 3);
    vat = key * C::ROW + 16 * v_piece<T, D>(key, c / 8) + c % 8 * 2;
  } else {
    vat = 4 * h * C::ROW + 16 * v_piece<T, D>(4 * h, lr / 4) + lr % 4 * 4;
  }

  f32x16 o[C::DT];
  float ref, l;            // reference max in log2 units (-inf: no key yet), sum of this half
  float base;              // ref, or 0 before the first key
  // (1 or 0, the same in all lanes: kept in scalar registers) every row has a reference;
  // some key was hidden from some row
  int all_set, masked;

  // S^T of 32 keys of the step in the buffer at byte `at`: lane = row, register 4 j + i =
  // key 8 j + 4 h + i
  auto logits = [&](int at, int kt) __attribute__((always_inline)) -> f32x16 {
    f32x16 z;
#pragma unroll
    for (int r = 0; r < 16; ++r) z[r] = 0.0f;
#pragma unroll
    for (int i = 0; i < C::NQ; ++i) {
      const qvec kf = *reinterpret_cast<const qvec *>(lds + ((at + kat) ^ (i * C::STEP_K)) +
                                                      32 * kt * C::ROW);
      if constexpr (sizeof(T) == 2) {
        z = mfma_bf16(kf, qf[i], z);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) z = mfma_f32(kf[e], qf[i][e], z);
      }
    }
    return z;
  };
  // P of 32 keys as the B operand of O^T += V^T P^T (registers 8 ks .. 8 ks + 7 of its
  // 16 keys ks), rounded to V's type; the sum of the lane's unrounded terms, which the LSE
  // needs.  Rounding to bf16 is half a step of each weight: outputs are 0.0022 from the
  // 64-bit values, relative to their norm, 0.0017 of it by their own rounding.  A second
  // bf16 for the rest of each weight and its products would be the decode's precision, and
  // took 1,500 us instead of 1,095 for the long prompt above, 124 instead of 111 for 16 blocks
  // of new thoughts (four layers).
  struct Terms {
    pvec p[32 / C::PK];
    float sum;
  };
  auto terms = [&](const f32x16 &z, float r) __attribute__((always_inline)) -> Terms {
    Terms t;
    float part[4];
#pragma unroll
    for (int x = 0; x < 16; ++x) {
      const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(z[x], a.sl2, -r));
      part[x & 3] = x < 4 ? e : part[x & 3] + e;
      if constexpr (sizeof(T) == 2) t.p[x / 8][x % 8] = (__bf16)e;
      else t.p[x] = e;
    }
    t.sum = (part[0] + part[1]) + (part[2] + part[3]);
    return t;
  };
  // the reference of the rows that move becomes at least the max of these logits, and what
  // has been summed against the old one follows.  (Whether a row moves depends on the row
  // alone, so that other rows of the wave do not change its bits.)
  auto raise = [&](const f32x16 &z, bool moves) __attribute__((always_inline)) {
    float mx = z[0];
#pragma unroll
    for (int x = 1; x < 16; ++x) mx = fmaxf(mx, z[x]);
    mx = swap_halves_max(mx) * a.sl2;
    const float to = moves ? fmaxf(ref, mx) : ref;
    if (ballot(to > ref)) {
      const float by = to == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(ref - to);
      l *= by;
#pragma unroll
      for (int d = 0; d < C::DT; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[d][r] *= by;
      ref = to;
      base = to == -INFINITY ? 0.0f : to;
    }
  };
  Window win = fill(0), nxt = win;
  // V^T operand of 16 keys ks (bf16): keys 4 h + i and 8 + 4 h + i, the order that P has
  auto values = [&](int at, int ks, int d) __attribute__((always_inline)) -> bf16x8 {
    return read_transposed(
        lds + ((at + vat) ^ (d * C::STEP_V)) + (2 * C::BUF + 16 * ks * C::ROW), 8 * C::ROW);
  };
  auto add = [&](const Terms &t, int at, int kt) __attribute__((always_inline)) {
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int ks = 0; ks < 2; ++ks)
#pragma unroll
        for (int d = 0; d < C::DT; ++d)
          o[d] = mfma_bf16(values(at, 2 * kt + ks, d), t.p[ks], o[d]);
    } else {
#pragma unroll
      for (int x = 0; x < 16; ++x)
#pragma unroll
        for (int d = 0; d < C::DT; ++d)
          o[d] = mfma_f32(*reinterpret_cast<const float *>(
                              lds + ((at + vat) ^ (d * C::STEP_V)) +
                              (2 * C::BUF + (8 * (x / 4) + x % 4) * C::ROW)),
                          t.p[x], o[d]);
    }
  };

  // term x of 16, as it goes into the products
  auto weight = [&](const Terms &t, int x) __attribute__((always_inline)) -> float {
    if constexpr (sizeof(T) == 2) return (float)t.p[x / 8][x % 8];
    else return t.p[x];
  };
  // the same with 0 for values that are not finite
  auto add_finite = [&](const Terms &t, int at, int kt) __attribute__((always_inline)) {
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int ks = 0; ks < 2; ++ks)
#pragma unroll
        for (int d = 0; d < C::DT; ++d) {
          u32x4 v = __builtin_bit_cast(u32x4, values(at, 2 * kt + ks, d));
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if ((v[e] & 0x7f80u) == 0x7f80u) v[e] &= 0xffff0000u;
            if ((v[e] & 0x7f800000u) == 0x7f800000u) v[e] &= 0xffffu;
          }
          o[d] = mfma_bf16(__builtin_bit_cast(bf16x8, v), t.p[ks], o[d]);
          fence_order();                         // (one at a time, in few registers)
        }
    } else {
#pragma unroll
      for (int x = 0; x < 16; ++x)
#pragma unroll
        for (int d = 0; d < C::DT; ++d) {
          const float v = *reinterpret_cast<const float *>(
              lds + ((at + vat) ^ (d * C::STEP_V)) +
              (2 * C::BUF + (8 * (x / 4) + x % 4) * C::ROW));
          o[d] = mfma_f32(__builtin_isfinite(v) ? v : 0.0f, t.p[x], o[d]);
          fence_order();
        }
    }
  };

  // hides from each row the keys of half kt of step st that it may not see; the registers
  // hidden, for a careful run
  auto hide = [&](f32x16 &z, const Window &cur, int st, int kt) __attribute__((always_inline)) {
    uint32_t hidden = 0;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int idx = st % WSTEPS * C::SUBS + 2 * kt + half;
      const int valid = __builtin_amdgcn_readlane(cur.info, idx) >> 8 & 31;  // 0: past the end
      const Entry en = entry(__builtin_amdgcn_readlane(cur.ent, idx));
      const int slot = (un.s0 + st * C::SUBS + 2 * kt + half - en.sub0) * 16;
      const int seen = en.own & seq_bit ? qslot + 1 - slot : en.below & seq_bit ? 16 : 0;
      const int lim = live ? min(seen, valid) : valid;
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        const bool out = 8 * (x / 4) + 4 * h + x % 4 >= lim;
        z[8 * half + x] = out ? -INFINITY : z[8 * half + x];
        hidden |= out ? 1u << (8 * half + x) : 0u;
      }
    }
    return hidden;
  };
  // whether some row must not see some key of half kt of step st
  auto hides = [&](const Window &cur, int st, int kt) __attribute__((always_inline)) -> bool {
    const int idx = st % WSTEPS * C::SUBS + 2 * kt;
    return ((__builtin_amdgcn_readlane(cur.info, idx) |
             __builtin_amdgcn_readlane(cur.info, idx + 1)) & (kMask | kNone)) != 0;
  };
  // The new half's terms t of z against the reference, the reference raised where they
  // outgrow it.
  auto check = [&](Terms &t, const f32x16 &z) __attribute__((always_inline)) {
    const uint64_t over = ballot(!(t.sum < kMoveAt));
    if (__builtin_expect(over != 0, 0)) {
      asm volatile("" ::: "memory");             // stays a branch: the rescale is long
      raise(z, (over >> lr | over >> (lr + 32)) & 1);
      t = terms(z, base);
    }
    l += t.sum;
  };
  // Any other step, bit by bit as a common one where a row has a reference.  CAREFUL: see
  // below.
  auto plain_step = [&](const Window &cur, int st, int at, auto careful_c)
                        __attribute__((always_inline)) {
    constexpr bool CAREFUL = decltype(careful_c)::value;
#pragma unroll
    for (int kt = 0; kt < C::NS; ++kt) {
      f32x16 z = logits(at, kt);
      const bool mask = hides(cur, st, kt);
      uint32_t hidden = 0;
      if (mask || !__builtin_amdgcn_readfirstlane(all_set)) {
        if (mask) {
          hidden = hide(z, cur, st, kt);
          masked = __builtin_amdgcn_readfirstlane(1);
        }
        raise(z, ref == -INFINITY);
        all_set = __builtin_amdgcn_readfirstlane(ballot(ref == -INFINITY) == 0);
      }
      Terms t = terms(z, base);
      check(t, z);
      if (!CAREFUL || !mask) {
        add(t, at, kt);
      } else if constexpr (CAREFUL) {
        // The products with every value that is finite, as always: the bits of rows that
        // see no others do not change.  Then the others, for the rows that see them: 16 keys
        // of P at a time go through the buffer that a careful run does not load into; a
        // hidden key is marked by -1
        add_finite(t, at, kt);
        float *scr = reinterpret_cast<float *>(lds + C::BUF) + wave * 512;
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            scr[(8 * (e / 4) + 4 * h + e % 4) * 32 + lr] =
                hidden >> (8 * ks + e) & 1 ? -1.0f : weight(t, 8 * ks + e);
          __builtin_amdgcn_s_waitcnt(0);
          __builtin_amdgcn_wave_barrier();
          for (int key = 0; key < 16; ++key) {
            const float pk = scr[key * 32 + lr];
            const char *vr = lds + at + 2 * C::BUF + (32 * kt + 16 * ks + key) * C::ROW;
#pragma unroll
            for (int d = 0; d < C::DT; ++d)
#pragma unroll
              for (int x = 0; x < 16; ++x) {
                if (x % 4 == 0) fence_order();
                const int c = 32 * d + 8 * (x / 4) + 4 * h + x % 4;
                const float vv = (float)*reinterpret_cast<const T *>(
                    vr + v_piece<T, D>(key, c * C::ES / 16) * 16 + c * C::ES % 16);
                o[d][x] = pk < 0.0f || __builtin_isfinite(vv) ? o[d][x] : o[d][x] + pk * vv;
              }
          }
          __builtin_amdgcn_wave_barrier();
        }
      }
    }
  };
  auto clear = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int d = 0; d < C::DT; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[d][r] = 0.0f;
    ref = -INFINITY;
    base = l = 0.0f;
    all_set = masked = 0;
  };
  // A step in which every row has a reference: the logits of both halves, then the terms and
  // products of one half after the other, V operands read three products ahead.
  auto common_step = [&](int st, int at, bool mask) __attribute__((always_inline)) {
    if constexpr (sizeof(T) == 2) {
      constexpr int NV = 2 * C::DT, AHEAD = 3;           // V operands of a half
      f32x16 z0 = logits(at, 0), z1 = logits(at, 1);
      if (mask) {
        hide(z0, win, st, 0);
        hide(z1, win, st, 1);
        masked = __builtin_amdgcn_readfirstlane(1);
      }
      bf16x8 v[AHEAD + 1];
#pragma unroll
      for (int j = 0; j < AHEAD; ++j) v[j] = values(at, j / C::DT, j % C::DT);
      Terms t = terms(z0, base);
      check(t, z0);
#pragma unroll
      for (int kt = 0; kt < 2; ++kt) {
        Terms u = t;
        if (kt == 0) u = terms(z1, base);
#pragma unroll
        for (int j = kt * NV; j < (kt + 1) * NV; ++j) {
          if (j + AHEAD < 2 * NV)
            v[(j + AHEAD) % (AHEAD + 1)] = values(at, (j + AHEAD) / C::DT, (j + AHEAD) % C::DT);
          o[j % C::DT] = mfma_bf16(v[j % (AHEAD + 1)], t.p[j / C::DT - 2 * kt], o[j % C::DT]);
          fence_order();
        }
        if (kt == 0) check(u, z1);
        t = u;
      }
    } else {
      f32x16 z = logits(at, 0);
      if (mask) {
        hide(z, win, st, 0);
        masked = __builtin_amdgcn_readfirstlane(1);
      }
      Terms t = terms(z, base);
      check(t, z);
      add(t, at, 0);
    }
  };
  clear();
  issue(win, 0, 0);
  int at = 0;
  for (int st = 0; st < steps; ++st) {
    const int ws = st % WSTEPS;
    if (ws == 0 && st + WSTEPS < steps) nxt = fill((st + WSTEPS) * C::SUBS);
    landed_barrier();          // of this step; every wave is done with the other buffer
    if (st + 1 < steps) issue(ws + 1 < WSTEPS ? win : nxt, st + 1, at ^ C::BUF);
    int flags = 0, none = kNone;
#pragma unroll
    for (int sb = 0; sb < C::SUBS; ++sb) {
      const int inf = __builtin_amdgcn_readlane(win.info, ws * C::SUBS + sb);
      flags |= inf;
      none &= inf;
    }
    const bool some = any_live && !none;
    const bool common = some && __builtin_amdgcn_readfirstlane(all_set);
    const bool mask = (flags & (kMask | kNone)) != 0;
    if (some && !common) plain_step(win, st, at, std::false_type{});
    if (common) common_step(st, at, mask);
    if (ws + 1 == WSTEPS) win = nxt;
    at ^= C::BUF;
  }
  // A key that a row may not see has p = 0, but 0 times an infinite or NaN value is not
  // 0.  So a unit that hid keys and whose outputs are not all finite runs once more, its
  // steps with hidden keys without such values but for the rows that see them.
  float odd = 0.0f;                            // NaN if some output is not finite
  if (masked)
#pragma unroll
    for (int d = 0; d < C::DT; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) odd = __builtin_fmaf(o[d][r], 0.0f, odd);
  if (__syncthreads_or(live && odd != 0.0f)) {
    clear();
    for (int st = 0; st < steps; ++st) {
      win = fill(st / WSTEPS * kWave);
      issue(win, st, 0);
      landed_barrier();
      if (any_live) plain_step(win, st, 0, std::true_type{});
      __syncthreads();                         // every wave is done with the buffer
    }
  }
  if (ballot(stale)) {
    if (lane == 0) status_error(a.status, ARBOR_EINVAL);
    return;
  }
  const float lt = swap_halves_add(l);
  if (un.part >= 0) {
    // a part's sums: 1 KB a register quad, rows side by side, and a reference and a sum a row
    if (un.part >= a.part_cap) return;         // (the plan's bound holds)
    float *pp = a.part + (((int64_t)un.part * pl.Hkv + g) * kWaves + wave) * part_floats<D>();
#pragma unroll
    for (int d = 0; d < C::DT; ++d)
#pragma unroll
      for (int r = 0; r < 16; r += 4)
        *reinterpret_cast<f32x4 *>(pp + ((d * 4 + r / 4) * kWave + lane) * 4) =
            f32x4{o[d][r], o[d][r + 1], o[d][r + 2], o[d][r + 3]};
    pp[32 * D + lane] = h ? lt : ref;
    return;
  }
  const float inv = lt == 0.0f ? 0.0f : 1.0f / lt;
  // Rows leave whole, 16 bytes a lane: through the wave's share of LDS, in which a row's
  // 16-byte pieces are turned by its number so that 32 rows' writes spread over the banks
  char *own = lds + wave * (32 * C::ROW);
  constexpr int TURN = C::PIECES < 32 ? C::PIECES - 1 : 31;
  typedef T ovec __attribute__((ext_vector_type(4)));
#pragma unroll
  for (int d = 0; d < C::DT; ++d)
#pragma unroll
    for (int r = 0; r < 16; r += 4) {
      ovec w;
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = (T)(o[d][r + i] * inv);
      const int byte = (32 * d + 2 * r + 4 * h) * C::ES;
      *reinterpret_cast<ovec *>(own + lr * C::ROW +
                                ((byte / 16 ^ (lr & TURN)) * 16 + byte % 16)) = w;
    }
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  constexpr int RPI = kWave / C::PIECES;       // rows that one store covers
#pragma unroll
  for (int x = 0; x < 32 / RPI; ++x) {
    const int r = x * RPI + lane / C::PIECES, c = lane % C::PIECES;
    const u32x4 w = *reinterpret_cast<const u32x4 *>(own + r * C::ROW + ((c ^ (r & TURN)) * 16));
    const int y = wave * 32 + r, yq = y / G;
    if (yq < un.nt)
      *reinterpret_cast<u32x4 *>(static_cast<char *>(a.out) +
                                 (((int64_t)(un.t0 + yq) * Hq + g * G + (y - yq * G)) * C::ROW +
                                  c * 16)) = w;
  }
  if (a.lse && h == 0 && live) {
    const float rf = ref == -INFINITY && lt != 0.0f ? 0.0f : ref;
    a.lse[(int64_t)tok * Hq + head] = (rf + __builtin_amdgcn_logf(lt)) * kLn2;
  }
}

// Joins the parts of the tiles that have several: a workgroup per 32 rows of a tile and KV
// head, whose waves take the register quads that the attention's lanes had, each lane four
// columns of one row at a time, parts in order.  It waits on memory: four parts' sums and
// references are on their way together (60 parts of 8 KV heads, 33 MB, 8.4 us; one part
// after the other, with rows of D + 4 floats, 10.8).
template <class T, int D>
__global__ __launch_bounds__(256) void prefill_join(AttnArgs a) {
  constexpr int U = 4, QUADS = D / 8;
  const Pool &pl = a.pl;
  const int per_tile = kWaves * pl.Hkv;
  const int32_t status = status_word(a.status);
  Header head_of = *a.p.head;
  const int64_t table = a.t.page_off[a.t.V];
  int4 tl = a.p.split[min((int)blockIdx.x / per_tile, target_parts(pl.Hkv) - 1)];
  asm volatile("" : "+s"(head_of.n_split), "+s"(tl.x), "+s"(tl.y), "+s"(tl.z), "+s"(tl.w));
  if (!header_ok(a, head_of, table) | (status < 0)) return;
  for (int x = blockIdx.x; x / per_tile < head_of.n_split; x += gridDim.x) {
    if (x != (int)blockIdx.x) tl = a.p.split[x / per_tile];
    const int rows = x % kWaves;                  // 32 rows: the wave that had them
    const int g = x / kWaves % pl.Hkv;
    const int t0 = tl.x, nt = tl.y, part0 = tl.z, parts = tl.w;
    if (rows * 32 / pl.G >= nt || part0 + parts > a.part_cap) continue;
    const int lane = lane_id(), wave = threadIdx.x / kWave, lr = lane & 31, h = lane >> 5;
    const int64_t stride = (int64_t)pl.Hkv * kWaves * part_floats<D>();
    const float *pp = a.part + (((int64_t)part0 * pl.Hkv + g) * kWaves + rows) * part_floats<D>();
    constexpr int MINE = QUADS / 4;               // quads of a wave
    f32x4 o[MINE], v[U][MINE];
    float ref[U], sum[U];
    auto load = [&](int e0) {
#pragma unroll
      for (int i = 0; i < U; ++i) {
        ref[i] = -INFINITY;
        if (e0 + i >= parts) continue;
        const float *q = pp + (e0 + i) * stride;
        ref[i] = q[32 * D + lr];
        sum[i] = q[32 * D + 32 + lr];
#pragma unroll
        for (int j = 0; j < MINE; ++j)
          v[i][j] = *reinterpret_cast<const f32x4 *>(q + ((wave * MINE + j) * kWave + lane) * 4);
      }
    };
    float m = -INFINITY, l = 0.0f;
#pragma unroll
    for (int j = 0; j < MINE; ++j) o[j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    for (int e0 = 0; e0 < parts; e0 += U) {
      load(e0);
      float to = m;
#pragma unroll
      for (int i = 0; i < U; ++i) to = fmaxf(to, ref[i]);
      const float base = to == -INFINITY ? 0.0f : to;
      const float by = m == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - base);
      l *= by;
#pragma unroll
      for (int j = 0; j < MINE; ++j) o[j] *= by;
      m = to;
#pragma unroll
      for (int i = 0; i < U; ++i)
        if (e0 + i < parts) {
          // a part whose terms have no reference holds sums of 0 (or NaN, which stays)
          const float w = ref[i] == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(ref[i] - base);
          l += w * sum[i];
#pragma unroll
          for (int j = 0; j < MINE; ++j) o[j] += w * v[i][j];
        }
    }
    const int row = rows * 32 + lr, tq = row / pl.G;
    if (tq >= nt) continue;
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    const int Hq = pl.Hkv * pl.G, head = g * pl.G + row - tq * pl.G;
    const int64_t tok = t0 + tq;
    typedef T ovec __attribute__((ext_vector_type(4)));
#pragma unroll
    for (int j = 0; j < MINE; ++j) {
      ovec w;
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = (T)(o[j][i] * inv);
      *reinterpret_cast<ovec *>(static_cast<T *>(a.out) + (tok * Hq + head) * D +
                                (wave * MINE + j) * 8 + 4 * h) = w;
    }
    if (a.lse && wave == 0 && h == 0)
      a.lse[tok * Hq + head] = ((m == -INFINITY && l != 0.0f ? 0.0f : m) +
                                __builtin_amdgcn_logf(l)) * kLn2;
  }
}

inline size_t tile_floats(const arbor_geom_t *g) {      // of a part, all KV heads
  return (size_t)g->num_kv_heads * kRows * (g->head_dim + 2);
}
}  // namespace

size_t prefill_plan_size(const arbor_geom_t *g, int32_t n_seq, int32_t n_tokens) {
  size_t need = 0;
  (void)carve_plan(g, n_seq, n_tokens, nullptr, 0, &need);
  return need + 256;
}

size_t prefill_workspace_size(const arbor_geom_t *g, int32_t n_seq, int32_t n_tokens) {
  if (n_tokens == 0) return 256;
  return (size_t)target_parts(g->num_kv_heads) * tile_floats(g) * 4 + 256;
}

int launch_prefill_plan(const arbor_geom_t *geom, const arbor_tree_t *tree, const int32_t *nodes,
                        int32_t n_seq, const int32_t *cu, int32_t n_tokens, void *plan,
                        size_t plan_bytes, int32_t *status, hipStream_t stream) {
  if (n_tokens == 0 || n_seq == 0) return ARBOR_OK;
  const PlanPtrs p = carve_plan(geom, n_seq, n_tokens, plan, plan_bytes, nullptr);
  if (!p.head) return ARBOR_EWORKSPACE;
  const Tree t = make_tree(tree);
  const int G = geom->q_per_kv, Hkv = geom->num_kv_heads, P = geom->page_size;
  const int target = target_parts(Hkv);
  const int min_part = kMinSteps * step_subs(geom->dtype == ARBOR_BF16 ? 2 : 4);
  if (n_seq <= kMaxSeq && p.tiles_cap <= kSmallTiles && t.V <= kSmallV) {
    hipLaunchKernelGGL(plan_small, dim3(1), dim3(1024), 0, stream, t, G, Hkv, P, nodes, n_seq, cu,
                       n_tokens, p, target, min_part, status);
  } else {
    hipLaunchKernelGGL(plan_tiles, dim3(1), dim3(1024), 0, stream, t, G, Hkv, P, nodes, n_seq, cu,
                       n_tokens, p, status);
    hipLaunchKernelGGL(plan_chains, dim3((unsigned)p.tiles_cap), dim3(64), 0, stream, t, P, nodes,
                       cu, p, status);
    hipLaunchKernelGGL(plan_units, dim3(1), dim3(1024), 0, stream, p, target, min_part,
                       status);
  }
  return hip_ok(hipGetLastError());
}

int launch_prefill(const arbor_geom_t *geom, const arbor_tree_t *tree, const arbor_pool_t *pool,
                   const void *plan, size_t plan_bytes, int32_t n_seq, int32_t n_tokens,
                   int32_t layer, const void *q, void *out, float *lse, float softmax_scale,
                   int32_t *status, void *workspace, size_t workspace_bytes, hipStream_t stream) {
  if (n_tokens == 0 || n_seq == 0) return ARBOR_OK;
  AttnArgs a;
  a.p = carve_plan(geom, n_seq, n_tokens, const_cast<void *>(plan), plan_bytes, nullptr);
  if (!a.p.head) return ARBOR_EWORKSPACE;
  Carve cv(workspace, workspace_bytes);
  a.part_cap = target_parts(geom->num_kv_heads);        // (shares are rounded down)
  a.part = cv.take<float>((size_t)a.part_cap * tile_floats(geom));
  if (!cv.ok) return ARBOR_EWORKSPACE;
  a.t = make_tree(tree);
  a.pl = make_pool(geom, pool);
  a.n_seq = n_seq;
  a.n_tokens = n_tokens;
  a.layer = layer;
  a.q = q;
  a.out = out;
  a.lse = lse;
  a.sl2 = (softmax_scale > 0.0f ? softmax_scale : 1.0f / sqrtf((float)geom->head_dim)) * kLog2e;
  a.status = status;
  const int64_t units = a.p.units_cap * geom->num_kv_heads;
  const int64_t joins = join_groups(geom, n_seq, n_tokens, a.p.tiles_cap);
  if (units > INT32_MAX) return ARBOR_EUNSUPPORTED;
#define ARBOR_PREFILL_LAUNCH(T, D)                                                             \
  do {                                                                                         \
    timing_begin(geom, ARBOR_KERNEL_PREFILL_ATTN, stream);                                     \
    hipLaunchKernelGGL((prefill_attn<T, D>), dim3((unsigned)units), dim3(kRows * 2),           \
                       (Cfg<T, D>::LDS), stream, a);                                           \
    timing_end(geom, ARBOR_KERNEL_PREFILL_ATTN, stream);                                       \
    if (joins > 0)                                                                             \
      hipLaunchKernelGGL((prefill_join<T, D>), dim3((unsigned)joins), dim3(256), 0, stream, a); \
  } while (0)
  if (geom->dtype == ARBOR_BF16) {
    if (geom->head_dim == 128) ARBOR_PREFILL_LAUNCH(__bf16, 128);
    else ARBOR_PREFILL_LAUNCH(__bf16, 64);
  } else {
    if (geom->head_dim == 128) ARBOR_PREFILL_LAUNCH(float, 128);
    else ARBOR_PREFILL_LAUNCH(float, 64);
  }
#undef ARBOR_PREFILL_LAUNCH
  return hip_ok(hipGetLastError());
}

}  // namespace arbor
