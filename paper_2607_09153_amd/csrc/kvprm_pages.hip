// Pages of the cache for gfx950: rows of a page table forked into others with copy-on-write (kvprm_fork_pages), and the
// live pages of a pool moved into its lowest ids (kvprm_compact_pages). Both plan on the device from holders' counts
// and tables and copy the pages of all layers: pools of up to kOnePages pages in one launch whose blocks plan each for
// itself (k_fork_one, k_compact_one), larger ones in a few short launches that share a plan in the workspace.
#include <hip/hip_runtime.h>

#include "kvprm_attn_common.h"
#include "kvprm_internal.h"

namespace kvprm {

// Pages of a scan block: each of its waves takes 64 pages at a time and keeps their flags as one word.
constexpr int kScanPages = 4096, kScanWords = kScanPages / 64;
constexpr int kMaxScanBlocks = 1024;  // blocks of a pool (4 M pages)

// Workspace of both calls. Nothing in it needs to be set on entry.
struct PageScan {
  uint64_t *mask;    // [words] a bit per page: free for fresh pages, or (compact) live
  int32_t *before;   // [words] such pages of the block before the word
  int32_t *total;    // [blocks], then their exclusive sums
  int32_t *count;    // [num_pages] holders besides the old rows; (compact) the pages that move
  int32_t *shared;   // [num_pages] new rows that share the page
  uint64_t *source;  // [words] a bit per page: the source of a copy
  int32_t *row;      // [rows][4] of a fork, see RowPlan
  int32_t *state;    // [8] see State
  size_t bytes;
};
enum State { kBad = 0, kArrived = 1, kTotal = 2, kNeed = 3, kEmpty = 4, kDone = 5 };

// A new row: its tokens, the pages it shares with its parent, the pages it holds, and the source of its copy or -1.
struct RowPlan {
  int len, shared, held, copy;
};

static size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

static PageScan carve_pages(int64_t num_pages, void *base) {
  PageScan w;
  char *p = (char *)base;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    char *r = p + at;
    at += align256(bytes);
    return r;
  };
  const size_t blocks = (size_t)((num_pages + kScanPages - 1) / kScanPages), words = blocks * kScanWords;
  w.mask = (uint64_t *)take(words * 8);
  w.source = (uint64_t *)take(words * 8);
  w.before = (int32_t *)take(words * 4);
  w.total = (int32_t *)take((blocks + 1) * 4);
  w.count = (int32_t *)take((size_t)num_pages * 4);
  w.shared = (int32_t *)take((size_t)num_pages * 4);
  w.row = (int32_t *)take((size_t)kMaxBatch * 16);
  w.state = (int32_t *)take(64);
  w.bytes = at;
  return w;
}

int64_t max_pool_pages() { return (int64_t)kMaxScanBlocks * kScanPages; }
size_t pages_ws_bytes(int64_t num_pages) { return carve_pages(num_pages, nullptr).bytes; }

// Division by a number that a call keeps, without a divide: the quotient by its rounded-down reciprocal is right or one too
// small for x < 2^31.
struct Divisor {
  uint32_t d, inv;
  static Divisor of(uint64_t n) { return {(uint32_t)n, n ? (uint32_t)(0xFFFFFFFFull / n) : 0}; }
  __device__ __forceinline__ uint32_t split(uint32_t x, uint32_t &rest) const {
    uint32_t q = __umulhi(x, inv);
    rest = x - q * d;
    if (rest >= d) ++q, rest -= d;
    return q;
  }
};

struct PageArgs {
  int num_pages, rows, max_pages;
  const int32_t *table, *lengths, *held;
  const int32_t *refs;
  int32_t *new_refs, *result;
  // fork
  int children, to_pages;
  const int32_t *parent, *room;
  int32_t *to_table, *to_lengths, *to_held;
  // compact
  int32_t *moved;
  PageScan w;
  // the pools
  char *pool[2];
  float *scale[2];
  int layers, nkv;
  size_t page_bytes;  // of one page and layer, keys or values
  Divisor by_entries, by_to, by_pieces, by_parts;  // max_pages; to_pages; page_bytes / 16; 2 layers
};

// The k-th page (from 0) whose bit is set: a search among the blocks' sums, one among the block's words, then the
// word's bits.
__device__ __forceinline__ int select_page(const PageScan &w, int blocks, int k) {
  int lo = 0, hi = blocks - 1;  // the last block whose sum is at most k
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (w.total[mid] <= k) lo = mid;
    else hi = mid - 1;
  }
  k -= w.total[lo];
  const int32_t *before = w.before + lo * kScanWords;
  int a = 0, b = kScanWords - 1;
  while (a < b) {
    const int mid = (a + b + 1) / 2;
    if (before[mid] <= k) a = mid;
    else b = mid - 1;
  }
  k -= before[a];
  uint64_t m = w.mask[lo * kScanWords + a];
  int at = 0;
#pragma unroll
  for (int width = 32; width > 0; width >>= 1) {  // the half that holds bit k
    const int low = __popcll(m & ((1ull << width) - 1));
    if (k >= low) k -= low, m >>= width, at += width;
  }
  return (lo * kScanWords + a) * 64 + at;
}
// Set bits among the pages below `page`.
__device__ __forceinline__ int rank_page(const PageScan &w, int page) {
  const int word = page >> 6;
  return w.total[word / kScanWords] + w.before[word] + __popcll(w.mask[word] & ((1ull << (page & 63)) - 1));
}

// A block's flags, counted: words and the block's sum; the last block to arrive turns the sums into exclusive ones.
// 256 threads of blocks 0 .. blocks - 1; flag(page) is called for pages of the pool alone.
template <typename F>
__device__ __forceinline__ void scan_flags(const PageArgs &a, int blocks, F flag) {
  __shared__ int word_s[kScanWords];
  __shared__ int last_s;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int blk = blockIdx.x;
#pragma unroll
  for (int i = 0; i < kScanWords / 4; ++i) {
    const int word = i * 4 + wave, page = blk * kScanPages + word * 64 + lane;
    const uint64_t m = __ballot(page < a.num_pages && flag(page));
    if (lane == 0) {
      word_s[word] = __popcll(m);
      a.w.mask[blk * kScanWords + word] = m;
    }
  }
  __syncthreads();
  if (wave == 0) {
    const int n = word_s[lane], cum = lane_scan(n);
    a.w.before[blk * kScanWords + lane] = cum - n;
    if (lane == 63) {
      __hip_atomic_store(&a.w.total[blk], cum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      __threadfence();
      last_s = __hip_atomic_fetch_add(&a.w.state[kArrived], 1, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == blocks - 1;
    }
  }
  __syncthreads();
  if (!last_s) return;
  __threadfence();
  if (wave == 0) {
    int sum = 0;
    for (int i0 = 0; i0 < blocks; i0 += 64) {
      const int i = i0 + lane;
      const int n = i < blocks ? __hip_atomic_load(&a.w.total[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0;
      const int cum = lane_scan(n);
      if (i < blocks) a.w.total[i] = sum + cum - n;
      sum += __builtin_amdgcn_readlane(cum, 63);
    }
    if (lane == 0) a.w.state[kTotal] = sum;
  }
}

// ------------------------------------------------------------------------------- fork

// Holders before the call, a thread per page; the state.
__global__ __launch_bounds__(256) void k_fork_init(PageArgs a) {
  const int page = blockIdx.x * 256 + threadIdx.x;
  if (page < a.num_pages) a.w.count[page] = a.refs[page], a.w.shared[page] = 0;
  if (page < (a.num_pages + 63) / 64) a.w.source[page] = 0;
  if (blockIdx.x == 0 && threadIdx.x < 8) a.w.state[threadIdx.x] = 0;
}

// What child i takes from its parent (the same in every thread of a block of at least kMaxBatch). False where the
// rows are inconsistent.
__device__ __forceinline__ bool plan_row(const PageArgs &a, int i, RowPlan &r) {
  r = {0, 0, 0, -1};
  const int p = a.parent[i];
  const bool first = !__syncthreads_or((int)threadIdx.x < i && a.parent[threadIdx.x] == p);
  const int64_t room = a.room ? a.room[i] : 0;
  if (p >= a.rows || room < 0) return false;
  if (p >= 0) {
    r.len = a.lengths[p];
    const int held = a.held[p];
    if (r.len < 0 || held < 0 || held > a.max_pages || r.len > (int64_t)held * kPage) return false;
  }
  const int64_t want = (r.len + room + kPage - 1) / kPage;
  if (want > a.to_pages) return false;
  r.held = (int)want;
  r.shared = r.len / kPage;
  if (r.len % kPage == 0) return true;
  const int last = a.table[(size_t)p * a.max_pages + r.shared];
  if (last < 0 || last >= a.num_pages) return false;
  if (first && a.refs[last] == 1) ++r.shared;
  else r.copy = last;
  return true;
}

static_assert(kMaxBatch <= 256, "a block compares a child's parent with every earlier one's");

// Block (row, slice): the entries of one row, old rows first (their holds end), then new ones (those of the pages they
// share begin).
__global__ __launch_bounds__(256) void k_fork_count(PageArgs a) {
  const int row = blockIdx.x;
  const int from = blockIdx.y * 1024, tid = threadIdx.x;
  bool bad = false;
  if (row < a.rows) {
    const int held = a.held[row];
    if (held < 0 || held > a.max_pages) {
      bad = true;
    } else {
      for (int c = from + tid; c < min(held, from + 1024); c += 256) {
        const int id = a.table[(size_t)row * a.max_pages + c];
        if (id < 0 || id >= a.num_pages) bad = true;
        else atomicSub(&a.w.count[id], 1);
      }
    }
  } else {
    const int i = row - a.rows;
    RowPlan r;
    bad = !plan_row(a, i, r);
    if (!bad) {
      const int p = a.parent[i];
      for (int c = from + tid; c < min(r.shared, from + 1024); c += 256) {
        const int id = a.table[(size_t)p * a.max_pages + c];
        if (id < 0 || id >= a.num_pages) bad = true;
        else atomicAdd(&a.w.shared[id], 1);
      }
      if (blockIdx.y == 0 && tid == 0) {
        *(int4 *)(a.w.row + 4 * i) = make_int4(r.len, r.shared, r.held, r.copy);
        if (r.copy >= 0) atomicOr((unsigned long long *)&a.w.source[r.copy >> 6], 1ull << (r.copy & 63));
        atomicAdd(&a.w.state[kNeed], r.held - r.shared);
      }
    }
  }
  if (bad) atomicOr(&a.w.state[kBad], 1);
}

// Pages free for fresh entries, counted: those that nobody holds any more and no copy reads.
__global__ __launch_bounds__(256) void k_fork_scan(PageArgs a) {
  bool bad = false;
  int empty = 0;
  scan_flags(a, gridDim.x, [&](int page) {
    const int others = a.w.count[page], n = others + a.w.shared[page];
    bad = bad || others < 0 || n < 0;
    empty += n == 0;
    return n == 0 && !(a.w.source[page >> 6] >> (page & 63) & 1);
  });
  const int all = lane_scan(empty);
  if ((threadIdx.x & 63) == 63 && all) atomicAdd(&a.w.state[kEmpty], all);
  if (bad) atomicOr(&a.w.state[kBad], 1);
}

// The new rows' tables and the holders of every page.
__global__ __launch_bounds__(256) void k_fork_write(PageArgs a, int scan_blocks) {
  const int need = a.w.state[kNeed], have = a.w.state[kTotal];
  const int status = a.w.state[kBad] ? 2 : need > have ? 1 : 0;
  const int tid = threadIdx.x;
  if (blockIdx.x == 0 && tid == 0) {
    a.result[0] = status;
    a.result[1] = status == 2 ? 0 : need;
    a.result[2] = status == 2 ? 0 : have;
    a.result[3] = status ? 0 : a.w.state[kEmpty] - need;
  }
  if (status) return;
  __shared__ int first_s[kMaxBatch + 1];  // fresh pages of the rows before
  if (tid < 64) {
    int sum = 0;
    for (int i0 = 0; i0 < a.children; i0 += 64) {
      const int i = i0 + tid;
      const int n = i < a.children ? a.w.row[4 * i + 2] - a.w.row[4 * i + 1] : 0;
      const int cum = lane_scan(n);
      if (i < a.children) first_s[i] = sum + cum - n;
      sum += __builtin_amdgcn_readlane(cum, 63);
    }
    if (tid == 0) first_s[a.children] = sum;
  }
  __syncthreads();
  const int64_t threads = (int64_t)gridDim.x * 256, me = (int64_t)blockIdx.x * 256 + tid;
  for (int64_t e = me; e < (int64_t)a.children * a.to_pages; e += threads) {
    const int i = (int)(e / a.to_pages), c = (int)(e - (int64_t)i * a.to_pages);
    const int4 r = *(const int4 *)(a.w.row + 4 * i);
    int id = -1;
    if (c < r.y) id = a.table[(size_t)a.parent[i] * a.max_pages + c];
    else if (c < r.z) id = select_page(a.w, scan_blocks, first_s[i] + c - r.y);
    a.to_table[e] = id;
    if (c == 0) a.to_lengths[i] = r.x, a.to_held[i] = r.z;
  }
  for (int64_t page = me; page < a.num_pages; page += threads) {
    const bool free = a.w.mask[page >> 6] >> (page & 63) & 1;
    a.new_refs[page] = free && rank_page(a.w, (int)page) < need ? 1 : a.w.count[page] + a.w.shared[page];
  }
}

// Pages of every layer, keys and values: blocks take (copy, layer, part) in turn, 16 bytes a thread and load, four in
// flight.
__device__ __forceinline__ void copy_page(const PageArgs &a, int src, int dst, int layer, int part) {
  const size_t base = (size_t)layer * a.num_pages;
  const uint4 *from = (const uint4 *)(a.pool[part] + (base + src) * a.page_bytes);
  uint4 *to = (uint4 *)(a.pool[part] + (base + dst) * a.page_bytes);
  const int n = (int)(a.page_bytes / 16);
  for (int i0 = threadIdx.x; i0 < n; i0 += 1024) {
    uint4 v[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) v[u] = from[min(i0 + 256 * u, n - 1)];
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (i0 + 256 * u < n) to[i0 + 256 * u] = v[u];
  }
  if (a.scale[part])
    for (int i = threadIdx.x; i < a.nkv; i += 256)
      a.scale[part][(base + dst) * a.nkv + i] = a.scale[part][(base + src) * a.nkv + i];
}

__global__ __launch_bounds__(256) void k_fork_copy(PageArgs a) {
  const int i = blockIdx.x;
  const int4 r = *(const int4 *)(a.w.row + 4 * i);
  if (a.result[0] != 0 || r.w < 0) return;
  const int dst = a.to_table[(size_t)i * a.to_pages + r.y];
  for (int k = blockIdx.y; k < 2 * a.layers; k += gridDim.y) copy_page(a, r.w, dst, k >> 1, k & 1);
}

// ------------------------------------------------------------------------------- compact

__global__ __launch_bounds__(64) void k_compact_init(PageArgs a) {
  if (threadIdx.x < 8) a.w.state[threadIdx.x] = 0;
}

// Live pages, counted by the first blocks; the others look whether every entry of the rows names one, 1024 entries
// each.
__global__ __launch_bounds__(256) void k_compact_scan(PageArgs a, int blocks) {
  bool bad = false;
  if ((int)blockIdx.x < blocks) {
    scan_flags(a, blocks, [&](int page) {
      const int n = a.refs[page];
      bad = bad || n < 0;
      return n > 0;
    });
  } else {
    const int per = (a.max_pages + 1023) / 1024, k = blockIdx.x - blocks, row = k / per, from = k % per * 1024;
    const int held = a.held[row];
    bad = held < 0 || held > a.max_pages;
    for (int c = from + threadIdx.x; !bad && c < min(held, from + 1024); c += 256) {
      const int id = a.table[(size_t)row * a.max_pages + c];
      bad = id < 0 || id >= a.num_pages || a.refs[id] <= 0;
    }
  }
  if (bad) atomicOr(&a.w.state[kBad], 1);
}

// The k-th page (from 0) whose bit is not set: a search for it by rank.
__device__ __forceinline__ int select_hole(const PageScan &w, int num_pages, int k) {
  int lo = 0, hi = num_pages - 1;  // the first page with k + 1 holes up to and including it
  while (lo < hi) {
    const int mid = (int)(((int64_t)lo + hi) / 2);
    if (mid + 1 - rank_page(w, mid + 1) >= k + 1) hi = mid;
    else lo = mid + 1;
  }
  return lo;
}

// Where every page goes: the i-th live one past the live pages' number into the i-th hole below it.
__global__ __launch_bounds__(256) void k_compact_plan(PageArgs a) {
  const int live = a.w.state[kTotal];
  const int status = a.w.state[kBad] ? 2 : 0;
  const int page = blockIdx.x * 256 + threadIdx.x;
  const int stay = live < a.num_pages ? rank_page(a.w, live) : live;  // live pages that keep their places
  if (page == 0) {
    a.result[0] = status;
    a.result[1] = status ? 0 : live;
    a.result[2] = status ? 0 : live - stay;
    a.result[3] = status ? 0 : a.num_pages - live;
  }
  if (status || page >= a.num_pages) return;
  const bool alive = a.w.mask[page >> 6] >> (page & 63) & 1;
  int to = -1;
  if (alive) to = page < live ? page : select_hole(a.w, live, rank_page(a.w, page) - stay);
  a.moved[page] = to;
  if (alive) {
    a.new_refs[to] = a.refs[page];
    if (page >= live) {
      a.new_refs[page] = 0;
      a.w.count[rank_page(a.w, page) - stay] = page;  // the list of moves, by rank
    }
  } else if (page >= live) {
    a.new_refs[page] = 0;
  }
}

// The rows' new entries, and the moves: blocks take (move, layer, part) in turn.
__global__ __launch_bounds__(256) void k_compact_move(PageArgs a) {
  if (a.result[0] != 0) return;
  const int moves = a.result[2];
  const int64_t threads = (int64_t)gridDim.x * 256;
  for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < (int64_t)a.rows * a.max_pages; e += threads) {
    const int row = (int)(e / a.max_pages), c = (int)(e - (int64_t)row * a.max_pages);
    a.to_table[e] = c < a.held[row] ? a.moved[a.table[e]] : -1;
  }
  const int per = 2 * a.layers;
  for (int64_t k = blockIdx.x; k < (int64_t)moves * per; k += gridDim.x) {
    const int src = a.w.count[k / per], lp = (int)(k % per);
    copy_page(a, src, a.moved[src], lp >> 1, lp & 1);
  }
}

// ------------------------------------------------------------------------------- one launch

// Pools of up to kOnePages pages: one launch, whose blocks, one to a compute unit, each form the whole plan in LDS from the
// counts and tables (read from the caches, each for itself), then write their share of the results and copy their
// share of the pages. Nothing that a block reads is written by another, so that no block waits for one. Against the
// launches above, whose plan is spread over the blocks (fork / compact, us): a beam of 64 rows of 290 pages in a pool of
// 2270, 31 copies of 917 KB: 24 instead of 41; 4 rows of 10 pages 7 / 7, 20 / 19; 16384 pages, 64 rows of 200 entries
// 19 / 26, 31 / 39. The entries, which every block walks, are limited where forks cross (pages of 2 KB, a copy for every
// second row; one launch / several): 8000 pages, 64 rows of 512 19 / 35, 256 rows of 100, 300 and 512 19 / 41, 35 / 51 and
// 50 / 58; 16384 pages, 64 of 512 23 / 34, 256 of 100, 300, 512 23 / 40, 38 / 48, 52 / 52. Compactions of such small pages
// cross earlier (8000 pages, 256 rows of 300 and 512 30 / 34 and 44 / 33; 16384 pages 37 / 36, 50 / 36) but not those of a
// model's (28 layers, 4 kv-heads of 128 in 4 bits, 243 KB a page: 197 / 267, 202 / 256; 388 / 515, 396 / 506), whose
// copies are the call.
constexpr int kOnePages = 16384, kOneThreads = 1024;
constexpr int64_t kOneEntries = 1 << 17;  // entries of the rows

// Flags of the pool's pages as words in LDS, with the flags before each word, for selecting by rank.
struct WordScan {
  uint64_t *mask;   // [words]
  int32_t *before;  // [words]
  int words;
};
// Exclusive sums of the words' bits; returns their number. Every thread of the block calls it.
__device__ __forceinline__ int scan_words(const WordScan &s) {
  __shared__ int all_s;
  const int tid = threadIdx.x;
  __syncthreads();
  if (tid < 64) {
    int sum = 0;
    for (int i0 = 0; i0 < s.words; i0 += 64) {
      const int i = i0 + tid, n = i < s.words ? __popcll(s.mask[i]) : 0, cum = lane_scan(n);
      if (i < s.words) s.before[i] = sum + cum - n;
      sum += __builtin_amdgcn_readlane(cum, 63);
    }
    if (tid == 0) all_s = sum;
  }
  __syncthreads();
  return all_s;
}
// Bit k of m's set ones.
__device__ __forceinline__ int select_bit(uint64_t m, int k) {
  int at = 0;
#pragma unroll
  for (int width = 32; width > 0; width >>= 1) {  // the half that holds it
    const int low = __popcll(m & ((1ull << width) - 1));
    if (k >= low) k -= low, m >>= width, at += width;
  }
  return at;
}
// The k-th page whose flag is set (NOT: is not set; every word's pages count).
template <bool NOT = false>
__device__ __forceinline__ int select_word(const WordScan &s, int k) {
  int a = 0, b = s.words - 1;  // the last word with at most k before it
  while (a < b) {
    const int mid = (a + b + 1) / 2;
    if ((NOT ? 64 * mid - s.before[mid] : s.before[mid]) <= k) a = mid;
    else b = mid - 1;
  }
  const uint64_t m = NOT ? ~s.mask[a] : s.mask[a];
  return 64 * a + select_bit(m, k - (NOT ? 64 * a - s.before[a] : s.before[a]));
}
__device__ __forceinline__ int rank_word(const WordScan &s, int page) {
  return s.before[page >> 6] + __popcll(s.mask[page >> 6] & ((1ull << (page & 63)) - 1));
}

// The entries of the rows, eight in flight a thread; the first ones are asked for before anything else is known (with rows'
// numbers, lengths and counts asked for then too, and no divides: the beam of 64 rows 25.9 -> 24.2 us, 16 rows of up to
// 144 pages 10.1 -> 9.0).
struct Entries {
  static constexpr int U = 8;
  int id[U];
  __device__ __forceinline__ static uint32_t total(const PageArgs &a) {  // (at most kOneEntries)
    return (uint32_t)(a.rows * a.max_pages);
  }
  __device__ __forceinline__ void load(const PageArgs &a, uint32_t e0) {
    const uint32_t n = total(a);
    if (n == 0) return;
#pragma unroll
    for (int u = 0; u < U; ++u) id[u] = a.table[min(e0 + u * kOneThreads, n - 1)];
  }
  // f(row, entry, id) for every entry that a row holds; held: the rows' counts, in range.
  template <typename F>
  __device__ __forceinline__ void each(const PageArgs &a, const int32_t *held, F f) {
    const uint32_t n = total(a);
    for (uint32_t e0 = threadIdx.x; e0 < n; e0 += U * kOneThreads) {
      int now[U];
#pragma unroll
      for (int u = 0; u < U; ++u) now[u] = id[u];
      if (e0 + U * kOneThreads < n) load(a, e0 + U * kOneThreads);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const uint32_t e = min(e0 + u * kOneThreads, n - 1);
        uint32_t c;
        const int row = (int)a.by_entries.split(e, c);
        if (e0 + u * kOneThreads < n && (int)c < held[row]) f(row, (int)c, now[u]);
      }
    }
  }
};
// Counts of the pages of this wave's first words, asked for early (word wave + 16 k, k < N).
template <int N>
struct Counts {
  int n[N];
  __device__ __forceinline__ void load(const PageArgs &a) {
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
#pragma unroll
    for (int k = 0; k < N; ++k) n[k] = a.refs[min((wave + kOneThreads / 64 * k) * 64 + lane, a.num_pages - 1)];
  }
};

// Pages src[i] -> dst[i] of every layer, keys and values, spread over all threads of the grid in pieces of 16 bytes,
// two of them in flight a thread (I: a type that counts them). Past the caches both ways: 485 pages of 917 KB (890 MB
// moved) 269 us through them, 185 past them; four or eight in flight 189 and 196, each block a range of its own 192.
template <typename I>
__device__ __forceinline__ void copy_pieces(const PageArgs &a, const int32_t *src, const int32_t *dst, I total) {
  constexpr int U = 2;
  const uint32_t per = a.by_pieces.d;
  const I threads = (I)gridDim.x * kOneThreads;
  for (I e0 = (I)blockIdx.x * kOneThreads + threadIdx.x; e0 < total; e0 += U * threads) {
    uint4 v[U];
    uint4 *to[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const I e = min(e0 + u * threads, total - 1);
      uint32_t unit, at, lp;
      if constexpr (sizeof(I) == 4) unit = a.by_pieces.split(e, at);
      else unit = (uint32_t)(e / per), at = (uint32_t)(e - (I)unit * per);
      const uint32_t i = a.by_parts.split(unit, lp);
      char *pool = a.pool[lp & 1];
      const size_t base = (size_t)(lp >> 1) * a.num_pages;
      v[u] = ld_stream((const uint4 *)(pool + (base + src[i]) * a.page_bytes) + at);
      to[u] = (uint4 *)(pool + (base + dst[i]) * a.page_bytes) + at;
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (e0 + u * threads < total)
        __builtin_nontemporal_store(u32x4{v[u].x, v[u].y, v[u].z, v[u].w}, (u32x4 *)to[u]);
  }
}
__device__ __forceinline__ void copy_pages(const PageArgs &a, const int32_t *src, const int32_t *dst, int n) {
  const uint64_t total = (uint64_t)n * 2 * a.layers * (a.page_bytes / 16);
  const int64_t threads = (int64_t)gridDim.x * kOneThreads;
  if (total < 1u << 31) copy_pieces<uint32_t>(a, src, dst, (uint32_t)total);
  else copy_pieces<uint64_t>(a, src, dst, total);
  if (!a.scale[0]) return;
  const int64_t scales = (int64_t)n * 2 * a.layers * a.nkv;
  for (int64_t e = (int64_t)blockIdx.x * kOneThreads + threadIdx.x; e < scales; e += threads) {
    const int unit = (int)(e / a.nkv), h = (int)(e - (int64_t)unit * a.nkv), i = unit / (2 * a.layers), lp = unit - i * 2 * a.layers;
    float *pool = a.scale[lp & 1];
    const size_t base = (size_t)(lp >> 1) * a.num_pages;
    pool[(base + dst[i]) * a.nkv + h] = pool[(base + src[i]) * a.nkv + h];
  }
}

__global__ __launch_bounds__(kOneThreads) void k_fork_one(PageArgs a) {
  extern __shared__ uint64_t lds[];
  const int P = a.num_pages, words = (P + 63) / 64, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  // per page: the rows of `from` that hold it (low half) and those of `to` that share it
  uint64_t *count = lds, *mask = count + P;
  int32_t *before = (int32_t *)(mask + words);
  uint64_t *source = (uint64_t *)(before + ((words + 1) & ~1));
  __shared__ RowPlan row_s[kMaxBatch];
  __shared__ int first_s[kMaxBatch + 1];                    // fresh pages of the rows before
  __shared__ int child_s[kMaxBatch], eldest_s[kMaxBatch];   // of a row of `from`: its children, the first of them
  __shared__ int full_s[kMaxBatch], kept_s[kMaxBatch];      // its full pages; whether a child takes the next one
  __shared__ int src_s[kMaxBatch], dst_s[kMaxBatch];        // the copies; dst_s is the child's number before
  __shared__ int held_s[kMaxBatch], len_s[kMaxBatch];
  __shared__ int bad_s, empty_s, copies_s;
  const int i = tid;
  const int held = tid < a.rows ? a.held[tid] : 0, len = tid < a.rows ? a.lengths[tid] : 0;
  const int p = i < a.children ? a.parent[i] : -1;
  const int64_t room = i < a.children && a.room ? a.room[i] : 0;
  Entries entries;
  entries.load(a, tid);
  Counts<4> counts;
  counts.load(a);
  bool bad = held < 0 || held > a.max_pages;
  if (tid < a.rows) held_s[tid] = bad ? 0 : held, len_s[tid] = len;
  for (int i = tid; i < P; i += kOneThreads) count[i] = 0;
  for (int i = tid; i < words; i += kOneThreads) source[i] = 0;
  if (tid < kMaxBatch) child_s[tid] = kept_s[tid] = full_s[tid] = 0, eldest_s[tid] = kMaxBatch;
  if (tid == 0) bad_s = empty_s = 0;
  __syncthreads();
  bad = bad || p >= a.rows;
  if (p >= 0 && p < a.rows) {
    atomicAdd(&child_s[p], 1);
    atomicMin(&eldest_s[p], i);
  }
  __syncthreads();
  if (i < a.children) {
    RowPlan r = {0, 0, 0, -1};
    bad = bad || room < 0;
    if (p >= 0 && !bad) {
      r.len = len_s[p];
      bad = r.len < 0 || r.len > (int64_t)held_s[p] * kPage;
    }
    const int64_t want = (r.len + room + kPage - 1) / kPage;
    bad = bad || want > a.to_pages;
    if (!bad) {
      r.held = (int)want;
      r.shared = r.len / kPage;
      if (p >= 0) full_s[p] = r.shared;  // (the same for all its children)
      if (r.len % kPage) {
        const int last = a.table[(size_t)p * a.max_pages + r.shared];
        if (last < 0 || last >= P) {
          bad = true;
        } else if (eldest_s[p] == i && a.refs[last] == 1) {
          ++r.shared;
          kept_s[p] = 1;
        } else {
          r.copy = last;
          atomicOr((unsigned long long *)&source[last >> 6], 1ull << (last & 63));
        }
      }
    }
    row_s[i] = r;
  }
  if (bad) bad_s = 1;
  __syncthreads();
  if (bad_s) {
    if (blockIdx.x == 0 && tid < 4) a.result[tid] = tid == 0 ? 2 : 0;
    return;
  }
  entries.each(a, held_s, [&](int row, int c, int id) {
    const uint64_t share = c < full_s[row] ? child_s[row] : c == full_s[row] ? kept_s[row] : 0;
    if (id < 0 || id >= P) bad = true;
    else atomicAdd((unsigned long long *)&count[id], (unsigned long long)(share << 32 | 1));
  });
  __syncthreads();
  int empty = 0;
  auto word_of = [&](int word, int refs) {
    const int page = word * 64 + lane;
    bool free = false;
    if (page < P) {
      const int64_t others = (int64_t)refs - (uint32_t)count[page], n = others + (int64_t)(count[page] >> 32);
      bad = bad || others < 0 || n > INT32_MAX;
      empty += n == 0;
      free = n == 0 && !(source[word] >> lane & 1);
      count[page] = (uint64_t)n;
    }
    const uint64_t m = __ballot(free);
    if (lane == 0) mask[word] = m;
  };
  constexpr int WAVES = kOneThreads / 64;
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (wave + WAVES * k < words) word_of(wave + WAVES * k, counts.n[k]);
  for (int word = wave + 4 * WAVES; word < words; word += WAVES) word_of(word, a.refs[min(word * 64 + lane, P - 1)]);
  empty = lane_scan(empty);
  if (lane == 63 && empty) atomicAdd(&empty_s, empty);
  if (bad) bad_s = 1;
  const WordScan ws = {mask, before, words};
  const int have = scan_words(ws);
  if (tid < 64) {
    // The copies are listed in the order of the children: every block takes its share of the pieces by its own list.
    int sum = 0, copies = 0;
    for (int i0 = 0; i0 < a.children; i0 += 64) {
      const int c = i0 + tid, n = c < a.children ? row_s[c].held - row_s[c].shared : 0, cum = lane_scan(n);
      const int copy = c < a.children ? row_s[c].copy : -1, at = lane_scan(copy >= 0 ? 1 : 0);
      if (c < a.children) first_s[c] = sum + cum - n;
      if (copy >= 0) src_s[copies + at - 1] = copy, dst_s[copies + at - 1] = c;
      sum += __builtin_amdgcn_readlane(cum, 63);
      copies += __builtin_amdgcn_readlane(at, 63);
    }
    if (tid == 0) first_s[a.children] = sum, copies_s = copies;
  }
  __syncthreads();
  const int need = first_s[a.children], status = bad_s ? 2 : need > have ? 1 : 0;
  if (blockIdx.x == 0 && tid == 0) {
    a.result[0] = status;
    a.result[1] = status == 2 ? 0 : need;
    a.result[2] = status == 2 ? 0 : have;
    a.result[3] = status ? 0 : empty_s - need;
  }
  if (status) return;
  if (tid < copies_s) dst_s[tid] = select_word(ws, first_s[dst_s[tid]]);  // (the first fresh page of the row)
  __syncthreads();
  const uint32_t threads = gridDim.x * kOneThreads, me = blockIdx.x * kOneThreads + tid;
  for (uint32_t e = me; e < (uint32_t)(a.children * a.to_pages); e += threads) {  // (at most 2^28)
    uint32_t col;
    const int row = (int)a.by_to.split(e, col), c = (int)col;
    const RowPlan r = row_s[row];
    int id = -1;
    if (c < r.shared) id = a.table[(size_t)a.parent[row] * a.max_pages + c];
    else if (c < r.held) id = select_word(ws, first_s[row] + c - r.shared);
    a.to_table[e] = id;
    if (c == 0) a.to_lengths[row] = r.len, a.to_held[row] = r.held;
  }
  for (uint32_t page = me; page < (uint32_t)P; page += threads) {
    const bool free = mask[page >> 6] >> (page & 63) & 1;
    a.new_refs[page] = free && rank_word(ws, (int)page) < need ? 1 : (int)count[page];
  }
  copy_pages(a, src_s, dst_s, copies_s);
}

__global__ __launch_bounds__(kOneThreads) void k_compact_one(PageArgs a) {
  extern __shared__ uint64_t lds[];
  const int P = a.num_pages, words = (P + 63) / 64, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  uint64_t *mask = lds;
  int32_t *before = (int32_t *)(mask + words), *src = before + words, *dst = src + P / 2;
  __shared__ int held_s[kMaxBatch];
  __shared__ int bad_s;
  const int held = tid < a.rows ? a.held[tid] : 0;
  Counts<4> counts;
  counts.load(a);
  Entries entries;
  entries.load(a, tid);
  if (tid == 0) bad_s = 0;
  bool bad = held < 0 || held > a.max_pages;
  if (tid < a.rows) held_s[tid] = bad ? 0 : held;
  auto word_of = [&](int word, int refs) {
    const int n = word * 64 + lane < P ? refs : 0;
    bad = bad || n < 0;
    const uint64_t m = __ballot(n > 0);
    if (lane == 0) mask[word] = m;
  };
  constexpr int WAVES = kOneThreads / 64;
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (wave + WAVES * k < words) word_of(wave + WAVES * k, counts.n[k]);
  for (int word = wave + 4 * WAVES; word < words; word += WAVES) word_of(word, a.refs[min(word * 64 + lane, P - 1)]);
  const WordScan ws = {mask, before, words};
  const int live = scan_words(ws);
  entries.each(a, held_s, [&](int, int, int id) {
    bad = bad || id < 0 || id >= P || !(mask[id >> 6] >> (id & 63) & 1);
  });
  if (bad) bad_s = 1;
  __syncthreads();
  const int stay = live < P ? rank_word(ws, live) : live;  // live pages that keep their places
  const int moves = live - stay, status = bad_s ? 2 : 0;
  if (blockIdx.x == 0 && tid == 0) {
    a.result[0] = status;
    a.result[1] = status ? 0 : live;
    a.result[2] = status ? 0 : moves;
    a.result[3] = status ? 0 : P - live;
  }
  if (status) return;
  for (int k = tid; k < moves; k += kOneThreads) {  // the i-th live page past the live ones' number, the i-th hole
    src[k] = select_word(ws, stay + k);
    dst[k] = select_word<true>(ws, k);
  }
  __syncthreads();
  // (alive pages only)
  auto goes = [&](int page) { return page < live ? page : dst[rank_word(ws, page) - stay]; };
  const uint32_t threads = gridDim.x * kOneThreads, me = blockIdx.x * kOneThreads + tid;
  for (uint32_t page = me; page < (uint32_t)P; page += threads) {
    const bool alive = mask[page >> 6] >> (page & 63) & 1;
    const int to = alive ? goes((int)page) : -1;
    a.moved[page] = to;
    if (alive) a.new_refs[to] = a.refs[page];
    if ((int)page >= live) a.new_refs[page] = 0;
  }
  for (uint32_t e = me; e < Entries::total(a); e += threads) {
    uint32_t c;
    const int row = (int)a.by_entries.split(e, c);
    a.to_table[e] = (int)c < held_s[row] ? goes(a.table[e]) : -1;
  }
  copy_pages(a, src, dst, moves);
}

// ------------------------------------------------------------------------------- launch

// Blocks of a one-launch call, or 0: the pool or its tables are too large for one.
static int one_launch(const PageArgs &a) {
  return a.num_pages <= kOnePages && (int64_t)a.rows * a.max_pages <= kOneEntries ? 256 : 0;
}
static int fork_lds(int pages) {
  const int words = (pages + 63) / 64;
  return pages * 8 + words * 8 + ((words + 1) & ~1) * 4 + words * 8;
}
static int compact_lds(int pages) {
  const int words = (pages + 63) / 64;
  return words * 12 + pages / 2 * 8;
}

static PageArgs page_args(const Dims &dm, const kvprm_kv_cache &c, const kvprm_page_rows &from, const int32_t *refs,
                          int32_t *new_refs, int32_t *result, void *ws) {
  PageArgs a{};
  a.num_pages = c.num_pages;
  a.rows = from.rows, a.max_pages = from.max_pages;
  a.table = from.page_table, a.lengths = from.lengths, a.held = from.held;
  a.refs = refs, a.new_refs = new_refs, a.result = result;
  a.w = carve_pages(c.num_pages, ws);
  a.pool[0] = (char *)c.k_pages, a.pool[1] = (char *)c.v_pages;
  if (dm.kvdt == 2) a.scale[0] = (float *)c.k_scale, a.scale[1] = (float *)c.v_scale;
  a.layers = dm.layers, a.nkv = dm.nkv;
  a.page_bytes = dm.nkv * tile_bytes(dm.kvdt, dm.d);
  a.by_entries = Divisor::of(a.rows > 0 ? a.max_pages : 0);
  a.by_pieces = Divisor::of(a.page_bytes / 16);
  a.by_parts = Divisor::of(2 * (uint64_t)a.layers);
  return a;
}

hipError_t launch_fork_pages(const Dims &dm, const kvprm_kv_cache &c, const kvprm_page_rows &from,
                             const kvprm_page_rows &to, const int32_t *parent, const int32_t *room, const int32_t *refs,
                             int32_t *new_refs, int32_t *result, void *ws, hipStream_t s) {
  PageArgs a = page_args(dm, c, from, refs, new_refs, result, ws);
  a.children = to.rows, a.to_pages = to.max_pages;
  a.by_to = Divisor::of(a.children > 0 ? a.to_pages : 0);
  a.parent = parent, a.room = room;
  a.to_table = to.page_table, a.to_lengths = to.lengths, a.to_held = to.held;
  if (const int n = one_launch(a)) {
    hipLaunchKernelGGL(k_fork_one, dim3(n), dim3(kOneThreads), fork_lds(a.num_pages), s, a);
    return hipGetLastError();
  }
  const int blocks = (a.num_pages + kScanPages - 1) / kScanPages;
  hipLaunchKernelGGL(k_fork_init, dim3((a.num_pages + 255) / 256), dim3(256), 0, s, a);
  if (a.rows + a.children > 0) {
    const int wide = max(a.rows > 0 ? a.max_pages : 1, 1);
    hipLaunchKernelGGL(k_fork_count, dim3(a.rows + a.children, (wide + 1023) / 1024), dim3(256), 0, s, a);
  }
  hipLaunchKernelGGL(k_fork_scan, dim3(blocks), dim3(256), 0, s, a);
  hipLaunchKernelGGL(k_fork_write, dim3(256), dim3(256), 0, s, a, blocks);
  if (a.children > 0)
    hipLaunchKernelGGL(k_fork_copy, dim3(a.children, min(2 * a.layers, 64)), dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_compact_pages(const Dims &dm, const kvprm_kv_cache &c, const kvprm_page_rows &rows,
                                int32_t *new_table, const int32_t *refs, int32_t *new_refs, int32_t *moved,
                                int32_t *result, void *ws, hipStream_t s) {
  PageArgs a = page_args(dm, c, rows, refs, new_refs, result, ws);
  a.to_table = new_table;
  a.moved = moved;
  if (const int n = one_launch(a)) {
    hipLaunchKernelGGL(k_compact_one, dim3(n), dim3(kOneThreads), compact_lds(a.num_pages), s, a);
    return hipGetLastError();
  }
  const int blocks = (a.num_pages + kScanPages - 1) / kScanPages;
  hipLaunchKernelGGL(k_compact_init, dim3(1), dim3(64), 0, s, a);
  hipLaunchKernelGGL(k_compact_scan, dim3(blocks + a.rows * ((a.max_pages + 1023) / 1024)), dim3(256), 0, s, a, blocks);
  hipLaunchKernelGGL(k_compact_plan, dim3((a.num_pages + 255) / 256), dim3(256), 0, s, a);
  hipLaunchKernelGGL(k_compact_move, dim3(1024), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace kvprm
