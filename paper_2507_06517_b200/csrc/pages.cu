// Page tables of the 8-bit cache: growing and shrinking sequences, making sequences from parents, closing the holes of a pool.
//
// The allocator's whole state is page_ref (0 = free).  Every call has a planning kernel of one block, which decides everything that
// has an order -- who gets which page -- by prefix sums over the sequences and over page_ref, so that the outcome does not depend
// on the order of atomics; reference counts change by atomic integer additions, whose order does not show.  The plan
// (a list of page copies, new entries, a map) lies in the workspace, and a second kernel carries it out over the whole device: the
// copies move four or eight 16-byte pieces per lane at a time and are bound by memory.  The second kernel is launched with
// programmatic stream serialization, so that its blocks are on the device already when the plan is done.
//
// Measured: 32 layers x 32 sequences of 1500 to 4096 tokens forked to a random list of parents 15.7 us (plan 6 to 7, 20 MB of open pages copied); a
// pool of 32 layers x 24 sequences closed up 355 us, of which the copies (1 GB read, 1 GB written) run at 6.07 TB/s and the plan is 15.
#include <algorithm>

#include "paged.cuh"

namespace skv {

constexpr int kPlanThreads = 1024;
constexpr int kCopyThreads = 256;
constexpr int kForkCols = 32;          // table columns of a fork block
constexpr int kForkMaxSeqs = 1024;     // kForkCols entries of every sequence lie in shared memory

// one page copy: the first `blocks` blocks of every head (all of them for a whole page)
struct PageCopy { int32_t src, dst, blocks; };

struct PagesWs {             // the workspace's parts
  int32_t* hdr;              // status block; word 8: number of copies, 9: go (0: the call failed), 10: live pages
  int32_t* old_len;          // [units]
  int32_t* fresh;            // [units] first page taken for a unit
  int32_t* children;         // [n_seqs]
  PageCopy* copies;          // [max(units, n_pages)]
  int32_t* map;              // [n_pages] new number of a page that moves; or the list of pages taken
};
constexpr int kHdrCopies = 8, kHdrGo = 9, kHdrPagesLive = 10;

__device__ __forceinline__ void let_dependents_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_for_plan() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

static size_t pages_ws_layout(int units, int n_seqs, int n_pages, uint8_t* base, PagesWs* w) {
  size_t off = kHeaderBytes;
  auto part = [&](size_t bytes) { const size_t at = off; off = align_up(off + bytes, 256); return base + at; };
  uint8_t* old_len = part((size_t)units * 4);
  uint8_t* fresh = part((size_t)units * 4);
  uint8_t* children = part((size_t)n_seqs * 4);
  uint8_t* copies = part((size_t)std::max(units, n_pages) * sizeof(PageCopy));
  uint8_t* map = part((size_t)n_pages * 4);
  if (w) {
    w->hdr = reinterpret_cast<int32_t*>(base);
    w->old_len = reinterpret_cast<int32_t*>(old_len);
    w->fresh = reinterpret_cast<int32_t*>(fresh);
    w->children = reinterpret_cast<int32_t*>(children);
    w->copies = reinterpret_cast<PageCopy*>(copies);
    w->map = reinterpret_cast<int32_t*>(map);
  }
  return off;
}

size_t pages_workspace_bytes(const spindlekv_page_pool& p, const spindlekv_page_table& t) {
  return pages_ws_layout(t.n_layers * t.n_seqs, t.n_seqs, p.n_pages, nullptr, nullptr);
}

// pages of a length (page sizes are powers of two; lengths stay clear of the top of 32 bits)
__device__ __forceinline__ int pages_of(int len, int ps) { return (len + ps - 1) >> (31 - __clz(ps)); }

// The planning block looks at 32 * per * 32 pages at a time: every warp at 32 * per in order, every lane of it keeps the votes on 32 of
// them, lanes from `per` on none.  `per` is what the pool needs, at most 32.
__device__ __forceinline__ int votes_per_lane(const Pool& pool) { return min((pool.n_pages + kPlanThreads - 1) / kPlanThreads, 32); }
// first page of this thread's 32
__device__ __forceinline__ int first_voted(int base, int per) { return base + ((int)(threadIdx.x >> 5) * per + (int)(threadIdx.x & 31)) * 32; }
// which of them satisfy a test on their reference count (0 in lanes without pages)
template <typename Test>
__device__ __forceinline__ uint32_t vote_pages(const Pool& pool, int base, int per, Test test) {
  const int lane = threadIdx.x & 31, from = base + (int)(threadIdx.x >> 5) * per * 32 + lane;
  uint32_t mine = 0;
#pragma unroll 8
  for (int j = 0; j < per; ++j) {
    const int at = from + 32 * j;
    const uint32_t votes = __ballot_sync(0xffffffffu, at < pool.n_pages && test(pool.ref[at]));
    if (lane == j) mine = votes;
  }
  return mine;
}

struct IsFree {
  __device__ __forceinline__ bool operator()(int32_t r) const { return r == 0; }
};
constexpr IsFree is_free{};

// Lists the lowest `wanted` free pages, ascending, in taken[]; false (for every thread) when there are fewer.  One block.
// `early`: the votes on the first pages, where the caller has them already.
__device__ bool take_free(const Pool& pool, int wanted, int32_t* taken, int* warp_sums, uint32_t early) {
  int have = 0;
  const int per = votes_per_lane(pool);
  for (int base = 0; base < pool.n_pages && have < wanted; base += per * kPlanThreads) {
    const int first = first_voted(base, per);
    uint32_t free = base == 0 ? early : vote_pages(pool, base, per, is_free);
    int total;
    int k = have + block_exclusive_scan(__popc(free), warp_sums, total);
    for (; free && k < wanted; free &= free - 1) taken[k++] = first + __ffs(free) - 1;
    have += total;
  }
  __syncthreads();
  return have >= wanted;
}

__device__ __forceinline__ bool page_ok(const Pool& p, int page) { return page >= 0 && page < p.n_pages; }
__device__ __forceinline__ void add_ref(const Pool& p, int page, int by) {
  if (page_ok(p, page)) atomicAdd(p.ref + page, by);
}

// ---- resize ----------------------------------------------------------------------------------------------------------

struct ResizeParams {
  Pool pool;
  Table table;
  const int32_t* new_lens;
  int add;
  int32_t* start;
  PagesWs ws;
};

// what one unit needs: `grow` pages behind its last, and a copy of the page that writing goes on in if that is shared
struct Need { int len, grow, open; bool copy; };
__device__ __forceinline__ Need need_of(const ResizeParams& p, int u, int old, bool& bad) {
  Need n;
  const long long want = p.new_lens ? (long long)p.new_lens[u] : (long long)p.table.lens[u] + p.add;
  if (want < 0 || want > (long long)p.table.max_pages * p.pool.ps) bad = true;
  n.len = bad ? 0 : (int)want;
  n.grow = min(max(pages_of(n.len, p.pool.ps) - pages_of(old, p.pool.ps), 0), p.pool.n_pages + 1);   // more than there are: no matter how many
  const int upto = min(old, n.len);
  n.open = upto / p.pool.ps;
  n.copy = false;
  if (upto % p.pool.ps) {
    const int page = p.table.pages[(int64_t)u * p.table.max_pages + n.open];
    n.copy = page_ok(p.pool, page) && p.pool.ref[page] > 1;
  }
  return n;
}

__global__ void __launch_bounds__(kPlanThreads) resize_plan_kernel(ResizeParams p) {
  let_dependents_start();
  __shared__ int warp_sums[33];
  const int units = p.table.n_layers * p.table.n_seqs, tid = threadIdx.x;
  const uint32_t early = vote_pages(p.pool, 0, votes_per_lane(p.pool), is_free);
  // 1. how many pages everybody needs, and where each one's run of taken pages begins
  bool bad = false;
  int total_pages = 0, total_copies = 0;
  for (int base = 0; base < units; base += kPlanThreads) {
    const int u = base + tid;
    int pages = 0, copies = 0;
    if (u < units) {
      const int old = unit_len(p.table, p.pool, u);
      bool mine = false;
      const Need n = need_of(p, u, old, mine);
      bad |= mine;
      pages = n.grow + n.copy;
      copies = n.copy;
      p.ws.old_len[u] = old;
    }
    int total;
    const int at = block_exclusive_scan(pages, warp_sums, total);
    if (u < units) p.ws.fresh[u] = total_pages + at;
    total_pages += total;
    (void)block_exclusive_scan(copies, warp_sums, total);
    total_copies += total;
    if (total_pages > p.pool.n_pages) break;   // the same for all threads; the sum stays small
  }
  bad = __syncthreads_or(bad);
  // 2. the pages
  const bool enough = total_pages <= p.pool.n_pages && take_free(p.pool, total_pages, p.ws.map, warp_sums, early);
  const bool go = !bad && enough;
  if (tid == 0) {
    p.ws.hdr[kHdrStatus] = bad ? SPINDLEKV_INVALID_ARG : enough ? SPINDLEKV_OK : SPINDLEKV_CAPACITY;
    p.ws.hdr[kHdrCopies] = go ? total_copies : 0;
  }
  if (!go) {
    for (int u = tid; u < units; u += kPlanThreads) p.start[u] = -1;
    return;
  }
  // 3. the list of copies (every page_ref is still as it was)
  int listed = 0;
  for (int base = 0; base < units && total_copies; base += kPlanThreads) {
    const int u = base + tid;
    Need n{};
    bool mine = false;
    if (u < units) n = need_of(p, u, p.ws.old_len[u], mine);
    int total;
    const int at = listed + block_exclusive_scan(n.copy, warp_sums, total);
    if (n.copy) {
      const int upto = min(p.ws.old_len[u], n.len) % p.pool.ps;
      p.ws.copies[at] = PageCopy{p.table.pages[(int64_t)u * p.table.max_pages + n.open], p.ws.map[p.ws.fresh[u] + n.grow],
                                 (upto + kPagedBlock - 1) / kPagedBlock};
    }
    listed += total;
  }
  __syncthreads();
  // 4. tables, references, lengths: a warp per unit.  Whether a page is copied was decided above on the counts as they were;
  // the entry of the copy tells (its destination is known), so the changing counts are not read again
  const int lane = tid & 31;
  for (int u = tid >> 5; u < units; u += kPlanThreads / 32) {
    const int old = p.ws.old_len[u];
    const long long want = p.new_lens ? (long long)p.new_lens[u] : (long long)p.table.lens[u] + p.add;
    const int len = (int)want, have = pages_of(old, p.pool.ps), keep = pages_of(len, p.pool.ps);
    int32_t* row = p.table.pages + (int64_t)u * p.table.max_pages;
    const int grow = max(keep - have, 0);
    const int next = u + 1 < units ? p.ws.fresh[u + 1] : total_pages;
    const bool copy = next - p.ws.fresh[u] > grow;
    for (int i = lane; i < grow; i += 32) {
      const int page = p.ws.map[p.ws.fresh[u] + i];
      row[have + i] = page;
      p.pool.ref[page] = 1;
    }
    for (int i = keep + lane; i < have; i += 32) add_ref(p.pool, row[i], -1);
    if (copy && lane == 0) {
      const int at = min(old, len) / p.pool.ps, page = p.ws.map[p.ws.fresh[u] + grow];
      add_ref(p.pool, row[at], -1);
      row[at] = page;
      p.pool.ref[page] = 1;
    }
    __syncwarp();
    if (lane == 0) {
      p.table.lens[u] = len;
      p.start[u] = min(old, len);
    }
  }
}

// ---- copies ----------------------------------------------------------------------------------------------------------

// The copies, a warp at a time: all copied blocks of one (copy, head, K or V), which are contiguous, kUnroll 16-byte pieces per lane
// in flight (four for a few blocks of many pages, eight for whole pages); then their scales.  The plan's copies read pages that nobody writes and write pages that were free: no piece is both read
// and written.
template <int D, int kUnroll>
__device__ __forceinline__ void copy_pages(const Pool& pool, const PageCopy* list, int n, int part, int parts) {
  constexpr int kPiece = kPagedBlock * D / 16;        // 16-byte pieces of a block
  constexpr int kWarps = kCopyThreads / 32;
  const int per = pool.per_page(), lane = threadIdx.x & 31;
  const long long items = (long long)n * pool.heads * 2;
  for (long long it = (long long)part * kWarps + (threadIdx.x >> 5); it < items; it += (long long)parts * kWarps) {
    const unsigned ch = (unsigned)(it >> 1);            // at most 2^20 copies of 2^10 heads
    const unsigned which = ch / (unsigned)pool.heads;
    const PageCopy c = list[which];
    const int head = (int)(ch - which * (unsigned)pool.heads);
    const bool v = (it & 1) != 0;
    const int64_t src = ((int64_t)c.src * pool.heads + head) * per, dst = ((int64_t)c.dst * pool.heads + head) * per;
    const uint4* from = reinterpret_cast<const uint4*>((v ? pool.vc : pool.kc) + src * kPagedBlock * D) + lane;
    uint4* to = reinterpret_cast<uint4*>((v ? pool.vc : pool.kc) + dst * kPagedBlock * D) + lane;
    const float* scales = (v ? pool.vs : pool.ks) + src;
    const float scale = lane < c.blocks ? scales[lane] : 0.f;
    const int pieces = c.blocks * kPiece;               // a multiple of 32
    for (int i = 0; i < pieces; i += 32 * kUnroll) {
      uint4 x[kUnroll];
#pragma unroll
      for (int k = 0; k < kUnroll; ++k)
        if (i + 32 * k < pieces) x[k] = __ldcs(from + i + 32 * k);
#pragma unroll
      for (int k = 0; k < kUnroll; ++k)
        if (i + 32 * k < pieces) __stcs(to + i + 32 * k, x[k]);
    }
    if (lane < c.blocks) (v ? pool.vs : pool.ks)[dst + lane] = scale;
  }
}

template <int D>
__global__ void __launch_bounds__(kCopyThreads, 6) copy_kernel(Pool pool, PagesWs ws) {
  wait_for_plan();
  copy_pages<D, 4>(pool, ws.copies, ws.hdr[kHdrCopies], blockIdx.x, gridDim.x);
}

// ---- fork ------------------------------------------------------------------------------------------------------------

struct ForkParams {
  Pool pool;
  Table table;
  const int32_t* parent;
  PagesWs ws;
  int tiles;      // column tiles of a layer
};

__global__ void __launch_bounds__(kPlanThreads) fork_plan_kernel(ForkParams p) {
  let_dependents_start();
  __shared__ int warp_sums[33];
  __shared__ int children[kForkMaxSeqs], first[kForkMaxSeqs];
  const int n = p.table.n_seqs, units = p.table.n_layers * n, tid = threadIdx.x;
  for (int s = tid; s < n; s += kPlanThreads) { children[s] = 0; first[s] = n; }
  const uint32_t early = vote_pages(p.pool, 0, votes_per_lane(p.pool), is_free);
  __syncthreads();
  bool bad = false;
  for (int s = tid; s < n; s += kPlanThreads) {
    const int q = p.parent[s];
    if (q < -1 || q >= n) bad = true;
    else if (q >= 0) { atomicAdd(children + q, 1); atomicMin(first + q, s); }
  }
  bad = __syncthreads_or(bad);
  for (int s = tid; s < n; s += kPlanThreads) p.ws.children[s] = children[s];
  int copies = 0;
  for (int base = 0; base < units && !bad; base += kPlanThreads) {
    const int u = base + tid;
    bool copy = false;
    if (u < units) {
      const int l = u / n, s = u - l * n, q = p.parent[s];
      p.ws.old_len[u] = unit_len(p.table, p.pool, u);
      copy = q >= 0 && first[q] != s && unit_len(p.table, p.pool, l * n + q) % p.pool.ps != 0;
    }
    int total;
    const int at = copies + block_exclusive_scan(copy, warp_sums, total);
    if (u < units) p.ws.fresh[u] = copy ? at : -1;
    copies += total;
  }
  const bool enough = !bad && copies <= p.pool.n_pages && take_free(p.pool, copies, p.ws.map, warp_sums, early);
  if (tid == 0) {
    p.ws.hdr[kHdrStatus] = bad ? SPINDLEKV_INVALID_ARG : enough ? SPINDLEKV_OK : SPINDLEKV_CAPACITY;
    p.ws.hdr[kHdrCopies] = enough ? copies : 0;
    p.ws.hdr[kHdrGo] = enough;
  }
  if (!enough) return;
  __syncthreads();
  for (int u = tid; u < units; u += kPlanThreads) {
    const int l = u / n, s = u - l * n, q = p.parent[s];
    const int len = q >= 0 ? p.ws.old_len[l * n + q] : 0;
    p.table.lens[u] = len;
    const int slot = p.ws.fresh[u];
    if (slot >= 0) {
      const int page = p.ws.map[slot], part = len % p.pool.ps;
      const int src = p.table.pages[(int64_t)(l * n + q) * p.table.max_pages + len / p.pool.ps];
      p.ws.fresh[u] = page;
      p.pool.ref[page] = 1;
      // an entry outside the pool stands for no tokens: nothing to copy, the new page only keeps the place
      p.ws.copies[slot] = PageCopy{page_ok(p.pool, src) ? src : page, page, page_ok(p.pool, src) ? (part + kPagedBlock - 1) / kPagedBlock : 0};
    }
  }
}

// Blocks 0 .. layers*tiles-1 rewrite kForkCols columns of a layer's table in place (all old entries of the columns are in shared
// memory before the first is replaced) and count references; the blocks behind them copy pages.
template <int D>
__global__ void __launch_bounds__(kCopyThreads, 6) fork_kernel(ForkParams p) {
  extern __shared__ __align__(16) int32_t tile[];     // [n_seqs][kForkCols], then four numbers per sequence
  wait_for_plan();
  if (!p.ws.hdr[kHdrGo]) return;
  const int table_blocks = p.table.n_layers * p.tiles;
  if ((int)blockIdx.x >= table_blocks) {
    copy_pages<D, 4>(p.pool, p.ws.copies, p.ws.hdr[kHdrCopies], blockIdx.x - table_blocks, gridDim.x - table_blocks);
    return;
  }
  const int n = p.table.n_seqs, layer = blockIdx.x / p.tiles, c0 = (blockIdx.x - layer * p.tiles) * kForkCols;
  const int ps = p.pool.ps;
  // per sequence: its length before, its children, its parent, its own copy of the parent's open page (or -1)
  int4* seqs = reinterpret_cast<int4*>(tile + n * kForkCols);
  for (int s = threadIdx.x; s < n; s += kCopyThreads)
    seqs[s] = make_int4(p.ws.old_len[layer * n + s], p.ws.children[s], p.parent[s], p.ws.fresh[layer * n + s]);
  __syncthreads();
  int32_t* pages = p.table.pages + (int64_t)layer * n * p.table.max_pages;
#pragma unroll 4
  for (int i = threadIdx.x; i < n * kForkCols; i += kCopyThreads) {
    const int s = i / kForkCols, c = c0 + i % kForkCols;
    const int len = seqs[s].x, kids = seqs[s].y;
    tile[i] = c < pages_of(len, ps) ? pages[(int64_t)s * p.table.max_pages + c] : -1;
    const int by = c == len / ps ? min(kids, 1) - 1 : kids - 1;       // a page that is not full is the first child's alone
    if (by && c < pages_of(len, ps)) add_ref(p.pool, tile[i], by);
  }
  __syncthreads();
#pragma unroll 4
  for (int i = threadIdx.x; i < n * kForkCols; i += kCopyThreads) {
    const int s = i / kForkCols, c = c0 + i % kForkCols, q = seqs[s].z, page = seqs[s].w;
    const int len = q >= 0 ? seqs[q].x : 0;
    if (c < pages_of(len, ps)) pages[(int64_t)s * p.table.max_pages + c] = page >= 0 && c == len / ps ? page : tile[q * kForkCols + i % kForkCols];
  }
}

// ---- compact ---------------------------------------------------------------------------------------------------------

struct PagesCompactParams {
  Pool pool;
  Table table;
  int32_t* n_live;
  PagesWs ws;
};

__global__ void __launch_bounds__(kPlanThreads) compact_plan_kernel(PagesCompactParams p) {
  let_dependents_start();
  __shared__ int warp_sums[33];
  const int n = p.pool.n_pages, tid = threadIdx.x, per = votes_per_lane(p.pool), lane = tid & 31;
  const auto used = [](int32_t r) { return r > 0; };
  // a thread's votes on the first 32768 pages stay in a register; pools beyond that are read twice
  uint32_t kept = 0;
  int mine = 0;
  for (int base = 0; base < n; base += per * kPlanThreads) {
    const uint32_t live = vote_pages(p.pool, base, per, used);
    if (base == 0) kept = live;
    mine += __popc(live);
  }
  int live;
  (void)block_exclusive_scan(mine, warp_sums, live);
  // the r-th free page below `live` takes the r-th live page at or above it: there are equally many
  int holes = 0, moves = 0;
  for (int base = 0; base < n; base += per * kPlanThreads) {
    const int first = first_voted(base, per);
    const uint32_t mask = base == 0 ? kept : vote_pages(p.pool, base, per, used);
    const int below = lane < per ? min(max(live - first, 0), 32) : 0;          // of this thread's pages, those below `live`
    const uint32_t low = below == 32 ? 0xFFFFFFFFu : (1u << below) - 1u;
    uint32_t h = ~mask & low, m = mask & ~low;
    int total_h, total_m;
    int kh = holes + block_exclusive_scan(__popc(h), warp_sums, total_h);
    int km = moves + block_exclusive_scan(__popc(m), warp_sums, total_m);
    for (; h; h &= h - 1) p.ws.copies[kh++].dst = first + __ffs(h) - 1;
    for (; m; m &= m - 1) {
      p.ws.copies[km].src = first + __ffs(m) - 1;
      p.ws.copies[km++].blocks = p.pool.per_page();
    }
    holes += total_h;
    moves += total_m;
  }
  __syncthreads();
  for (int i = tid; i < moves; i += kPlanThreads) {
    const PageCopy c = p.ws.copies[i];
    p.ws.map[c.src] = c.dst;             // of a page below `live` the map says nothing: it stays
    p.pool.ref[c.dst] = p.pool.ref[c.src];
    p.pool.ref[c.src] = 0;
  }
  if (tid == 0) {
    *p.n_live = live;
    p.ws.hdr[kHdrStatus] = SPINDLEKV_OK;
    p.ws.hdr[kHdrCopies] = moves;
    p.ws.hdr[kHdrPagesLive] = live;
  }
}

// Block b maps the entries of unit b, b + gridDim, ...; then all blocks copy.
template <int D>
__global__ void __launch_bounds__(kCopyThreads, 4) compact_kernel(PagesCompactParams p) {
  wait_for_plan();
  const int units = p.table.n_layers * p.table.n_seqs, live = p.ws.hdr[kHdrPagesLive];
  for (int u = blockIdx.x; u < units; u += gridDim.x) {
    const int used = pages_of(unit_len(p.table, p.pool, u), p.pool.ps);
    int32_t* row = p.table.pages + (int64_t)u * p.table.max_pages;
    for (int i = threadIdx.x; i < used; i += kCopyThreads) {
      const int page = row[i];
      if (page >= live && page < p.pool.n_pages && p.ws.hdr[kHdrCopies]) row[i] = p.ws.map[page];
    }
  }
  copy_pages<D, 8>(p.pool, p.ws.copies, p.ws.hdr[kHdrCopies], blockIdx.x, gridDim.x);
}

// ---- launches --------------------------------------------------------------------------------------------------------

// launches `kernel` so that its blocks may start while the plan before it on the stream still runs (they wait for it)
template <typename... Args>
static spindlekv_status launch_behind(void (*kernel)(Args...), unsigned grid, size_t smem, cudaStream_t st, Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(kCopyThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  LaunchScope ls(KC_PAGES, st);
  return cudaLaunchKernelEx(&cfg, kernel, args...) == cudaSuccess ? SPINDLEKV_OK : SPINDLEKV_CUDA;
}

static int sm_count() {
  static int sms[kMaxDevices] = {};
  const int dev = PerDeviceOnce::current();
  if (dev < 0) return 0;
  if (!sms[dev] && cudaDeviceGetAttribute(&sms[dev], cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
  return sms[dev];
}

static spindlekv_status pages_ws(const spindlekv_page_pool& pool, const spindlekv_page_table& table, void* ws, size_t ws_bytes, PagesWs* w) {
  if (ws_bytes < pages_workspace_bytes(pool, table)) return SPINDLEKV_WORKSPACE_TOO_SMALL;
  pages_ws_layout(table.n_layers * table.n_seqs, table.n_seqs, pool.n_pages, static_cast<uint8_t*>(ws), w);
  return SPINDLEKV_OK;
}

spindlekv_status pages_resize_impl(const spindlekv_page_pool& pool, const spindlekv_page_table& table, const int32_t* new_lens, int add,
                                   int32_t* start, void* ws, size_t ws_bytes, cudaStream_t st) {
  ResizeParams p{make_pool(pool), make_table(table), new_lens, add, start, {}};
  const spindlekv_status s = pages_ws(pool, table, ws, ws_bytes, &p.ws);
  if (s != SPINDLEKV_OK) return s;
  const int sms = sm_count();
  if (!sms) return SPINDLEKV_CUDA;
  {
    LaunchScope ls(KC_PAGES, st);
    resize_plan_kernel<<<1, kPlanThreads, 0, st>>>(p);
  }
  if (cudaGetLastError() != cudaSuccess) return SPINDLEKV_CUDA;
  const int units = table.n_layers * table.n_seqs;
  const unsigned grid = (unsigned)std::min<int64_t>(((int64_t)units * pool.n_kv_heads * 2 + kCopyThreads / 32 - 1) / (kCopyThreads / 32), 6 * sms);
  return pool.head_dim == 64 ? launch_behind(copy_kernel<64>, grid, 0, st, p.pool, p.ws) : launch_behind(copy_kernel<128>, grid, 0, st, p.pool, p.ws);
}

spindlekv_status pages_fork_impl(const spindlekv_page_pool& pool, const spindlekv_page_table& table, const int32_t* parent, void* ws,
                                 size_t ws_bytes, cudaStream_t st) {
  if (table.n_seqs > kForkMaxSeqs) return SPINDLEKV_UNSUPPORTED;
  ForkParams p{make_pool(pool), make_table(table), parent, {}, ceil_div(table.max_pages, kForkCols)};
  if ((int64_t)p.tiles * table.n_layers > 0x3FFFFFFF) return SPINDLEKV_UNSUPPORTED;
  const spindlekv_status s = pages_ws(pool, table, ws, ws_bytes, &p.ws);
  if (s != SPINDLEKV_OK) return s;
  const int sms = sm_count();
  if (!sms) return SPINDLEKV_CUDA;
  static PerDeviceOnce once;
  const int dev = PerDeviceOnce::current();
  if (!once.done[dev]) {
    const int most = kForkMaxSeqs * (kForkCols * 4 + 16);
    if (cudaFuncSetAttribute(fork_kernel<64>, cudaFuncAttributeMaxDynamicSharedMemorySize, most) != cudaSuccess ||
        cudaFuncSetAttribute(fork_kernel<128>, cudaFuncAttributeMaxDynamicSharedMemorySize, most) != cudaSuccess)
      return SPINDLEKV_CUDA;
    once.done[dev] = true;
  }
  {
    LaunchScope ls(KC_PAGES, st);
    fork_plan_kernel<<<1, kPlanThreads, 0, st>>>(p);
  }
  if (cudaGetLastError() != cudaSuccess) return SPINDLEKV_CUDA;
  const int64_t units = (int64_t)table.n_layers * table.n_seqs;
  const unsigned grid = (unsigned)(p.tiles * table.n_layers + std::min<int64_t>((units * pool.n_kv_heads * 2 + kCopyThreads / 32 - 1) / (kCopyThreads / 32), 6 * sms));
  const size_t smem = (size_t)table.n_seqs * (kForkCols * 4 + 16);
  return pool.head_dim == 64 ? launch_behind(fork_kernel<64>, grid, smem, st, p) : launch_behind(fork_kernel<128>, grid, smem, st, p);
}

spindlekv_status pages_compact_impl(const spindlekv_page_pool& pool, const spindlekv_page_table& table, int32_t* n_live, void* ws,
                                    size_t ws_bytes, cudaStream_t st) {
  PagesCompactParams p{make_pool(pool), make_table(table), n_live, {}};
  const spindlekv_status s = pages_ws(pool, table, ws, ws_bytes, &p.ws);
  if (s != SPINDLEKV_OK) return s;
  const int sms = sm_count();
  if (!sms) return SPINDLEKV_CUDA;
  {
    LaunchScope ls(KC_PAGES, st);
    compact_plan_kernel<<<1, kPlanThreads, 0, st>>>(p);
  }
  if (cudaGetLastError() != cudaSuccess) return SPINDLEKV_CUDA;
  const unsigned grid = (unsigned)(4 * sms);
  return pool.head_dim == 64 ? launch_behind(compact_kernel<64>, grid, 0, st, p) : launch_behind(compact_kernel<128>, grid, 0, st, p);
}

}  // namespace skv
