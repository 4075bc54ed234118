// A key/value cache in pages: bookkeeping and copies.
//
// Sequence b holds len[b] tokens in pages table[b][0 .. ceil(len / page)); refs[p] counts the table
// entries that hold page p, 0 = free.  A full page may be held by several sequences, the page that a
// sequence writes next never is, so appending needs no copy.
//
// Taking pages is a prefix sum twice over: the pages that each sequence needs, and the free pages in
// ascending order; rank r of the second goes to the sequence whose range of the first holds r.  One
// workgroup does that (a pool's counts are tens of KB; bound by the latency of lengths, counts and
// tables read one after the other: 4 to 5 us a plan), the copies of rows are launches of their own
// over all layers, bound by bandwidth where there are many.  Page ids and lengths come from device memory that the caller writes: every use
// checks or clamps them, so a wrong table gives wrong tokens and no access outside the pool.
#include <algorithm>

#include "device_common.h"
#include "rp_internal.h"

namespace rp {

namespace {

constexpr int kPlanThreads = 1024;
constexpr int kPlanWaves = kPlanThreads / 64;
constexpr int kFreeList = 2048;  // free pages found by the counting pass and kept for the next one

struct PlanShared {
  int32_t cum[kMaxCommit];     // pages needed by sequences 0 .. i
  int32_t free_ids[kFreeList];
  int32_t wave[kPlanWaves];
};

// Inclusive scan of one value a thread over the workgroup; *total: the sum.
__device__ __forceinline__ int block_scan(int v, int32_t* wave, int* total) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  v = wave_scan(v);
  __syncthreads();
  if (lane == 63) wave[w] = v;
  __syncthreads();
  int before = 0, sum = 0;
#pragma unroll
  for (int i = 0; i < kPlanWaves; ++i) {
    const int x = wave[i];
    before += i < w ? x : 0;
    sum += x;
  }
  *total = sum;
  return v + before;
}

__device__ __forceinline__ int seq_len(const PageArgs& a, int seq) {
  return min(max(a.len[seq], 0), a.table_ld << a.lg);
}
__device__ __forceinline__ int pages_of(const PageArgs& a, int tokens) { return (tokens + (1 << a.lg) - 1) >> a.lg; }

// Gives back the pages of sequence `seq` (one wave).
__device__ __forceinline__ void release(const PageArgs& a, int seq, int lane) {
  const int n = pages_of(a, seq_len(a, seq));
  int32_t* row = a.table + (int64_t)seq * a.table_ld;
  for (int j = lane; j < n; j += 64) {
    const int id = row[j];
    if (id >= 0 && id < a.n_pages) atomicSub(a.refs + id, 1);
    row[j] = -1;
  }
  if (lane == 0) a.len[seq] = 0;
}

// Visits the free pages in ascending order until `most` of them were seen: f(rank, id).  Returns how
// many there are, counted up to the end of the block of pages in which `most` was reached.
template <class F>
__device__ __forceinline__ int free_pages(const PageArgs& a, int most, int32_t* wave, F&& f) {
  int found = 0;
  for (int base = 0; base < a.n_pages && found < most; base += 4 * kPlanThreads) {
    const int id0 = base + 4 * (int)threadIdx.x;
    bool is[4];
    int mine = 0, sum;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      is[i] = id0 + i < a.n_pages && a.refs[id0 + i] <= 0;
      mine += is[i];
    }
    int rank = found + block_scan(mine, wave, &sum) - mine;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (is[i]) f(rank++, id0 + i);
    found += sum;
  }
  return found;
}

// Pages for sequences 0 .. n-1: need(i) pages each, the k-th of which goes to put(i, k, page).  A
// sequence that needs pages gets them if the needs up to and with its own are no more than the free
// pages; lack[i] = how many of its pages there were not (0: it has them all, or -1 as need_ok said).
// need(i) < 0: refused before, passed on.
template <class Need, class Put>
__device__ __forceinline__ void take_pages(const PageArgs& a, int n, PlanShared& sh, int32_t* lack, Need&& need, Put&& put) {
  int total = 0;
  for (int base = 0; base < n; base += kPlanThreads) {
    const int i = base + (int)threadIdx.x;
    const int v = i < n ? max(need(i), 0) : 0;
    int sum;
    const int c = total + block_scan(v, sh.wave, &sum);
    if (i < n) sh.cum[i] = c;
    total += sum;
  }
  const int there = free_pages(a, total, sh.wave, [&](int rank, int id) {
    if (rank < kFreeList) sh.free_ids[rank] = id;
  });
  __syncthreads();
  auto give = [&](int rank, int id) {
    if (rank >= total) return;
    int lo = 0, hi = n - 1;  // first sequence whose cum exceeds rank
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (sh.cum[mid] > rank) hi = mid; else lo = mid + 1;
    }
    if (sh.cum[lo] > there) return;
    a.refs[id] = 1;
    put(lo, rank - (lo ? sh.cum[lo - 1] : 0), id);
  };
  const int kept = min(min(there, total), kFreeList);
  for (int r = threadIdx.x; r < kept; r += kPlanThreads) give(r, sh.free_ids[r]);
  if (min(there, total) > kFreeList) {  // the rest by a second search, behind the last page listed
    const int first = sh.free_ids[kFreeList - 1] + 1;
    PageArgs rest = a;
    rest.refs = a.refs + first;
    rest.n_pages = a.n_pages - first;
    free_pages(rest, total - kFreeList, sh.wave, [&](int rank, int id) { give(kFreeList + rank, first + id); });
  }
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += kPlanThreads) {
    const int v = need(i), c = sh.cum[i];
    lack[i] = v < 0 ? -1 : v > 0 && c > there ? min(v, c - there) : 0;
  }
  __syncthreads();
}

}  // namespace

// Room for rows cu[i+1] - cu[i] more tokens of sequences seq[i].
__global__ __launch_bounds__(kPlanThreads) void k_append_plan(PageArgs a, SeqRows q, int32_t* __restrict__ missing) {
  __shared__ PlanShared sh;
  auto need = [&](int i) {
    const int at = seq_len(a, q.seq[i]);
    const int64_t end = (int64_t)at + (q.cu[i + 1] - q.cu[i]);
    if (end > (int64_t)a.table_ld << a.lg) return -1;
    return pages_of(a, (int)end) - pages_of(a, at);
  };
  take_pages(a, q.n, sh, missing, need, [&](int i, int k, int id) {
    a.table[(int64_t)q.seq[i] * a.table_ld + pages_of(a, seq_len(a, q.seq[i])) + k] = id;
  });
  for (int i = threadIdx.x; i < q.n; i += kPlanThreads)
    if (missing[i] == 0) a.len[q.seq[i]] = seq_len(a, q.seq[i]) + (q.cu[i + 1] - q.cu[i]);
}

// The slot (row of a layer) of token `pos` of sequence `seq`; -1 where the table holds none.
__device__ __forceinline__ int64_t slot_of(const PageArgs& a, int seq, int pos) {
  const int id = a.table[(int64_t)seq * a.table_ld + (pos >> a.lg)];
  return id >= 0 && id < a.n_pages ? ((int64_t)id << a.lg) + (pos & ((1 << a.lg) - 1)) : -1;
}

// Copies `bytes` (a multiple of 16) with the threads first, first + step, .. of a group: four loads of each in
// flight, past the caches' keeping (what is copied is not read again soon).  268 MB of pages moved:
// 105 us, 5.1 TB/s read and written; 112 with one plain 16-byte load at a time.
typedef uint32_t words_t __attribute__((ext_vector_type(4)));
__device__ __forceinline__ void copy_bytes(uint8_t* __restrict__ dst, const uint8_t* __restrict__ src, int64_t bytes, int first, int step) {
  words_t* d = reinterpret_cast<words_t*>(dst);
  const words_t* s = reinterpret_cast<const words_t*>(src);
  const int64_t n = bytes / 16;
  int64_t c = first;
  for (; c + 3 * step < n; c += 4 * step) {
    words_t v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = __builtin_nontemporal_load(s + c + i * step);
#pragma unroll
    for (int i = 0; i < 4; ++i) __builtin_nontemporal_store(v[i], d + c + i * step);
  }
  for (; c < n; c += step) __builtin_nontemporal_store(__builtin_nontemporal_load(s + c), d + c);
}

// One row a wave: row r of the packed rows goes to its sequence's token len - rows + (r - cu[i]).
// Four prompts of 4096 tokens, 4 layers (134 MB): 47 us, 5.6 TB/s read and written.
// A launch takes the rows from `first` on (launch_append_rows; a loop over rows in here took those prompts 5 us more).
__global__ __launch_bounds__(256) void k_append_rows(PageArgs a, SeqRows q, const uint8_t* __restrict__ k,
                                                     const uint8_t* __restrict__ v, int64_t layer_bytes,
                                                     const int32_t* __restrict__ missing, int first) {
  const int lane = threadIdx.x & 63;
  const int r = first + __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
  if (r >= q.cu[q.n]) return;
  int lo = 0, hi = q.n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (q.cu[mid] <= r) lo = mid; else hi = mid - 1;
  }
  if (missing[lo] != 0) return;
  const int rows = q.cu[lo + 1] - q.cu[lo];
  const int pos = seq_len(a, q.seq[lo]) - rows + (r - q.cu[lo]);
  const int64_t to = pos >= 0 ? slot_of(a, q.seq[lo], pos) : -1;
  if (to < 0) return;
  const uint8_t* src = (blockIdx.z ? v : k) + blockIdx.y * layer_bytes + (int64_t)r * a.row_bytes;
  uint8_t* dst = (blockIdx.z ? a.v : a.k) + blockIdx.y * a.layer_bytes + to * a.row_bytes;
  for (int c = lane * 16; c < a.row_bytes; c += 1024) *(uint4*)(dst + c) = *(const uint4*)(src + c);
}

__global__ __launch_bounds__(256) void k_pages_free(PageArgs a, SeqRows q) {
  const int i = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (i < q.n) release(a, q.seq[i], threadIdx.x & 63);
}

// dst[i] gives its pages back and gets one of its own for src[i]'s last page, where that is not full.
// 32 children: 5.4 us.
__global__ __launch_bounds__(kPlanThreads) void k_fork_plan(PageArgs a, SeqPairs q, int32_t* __restrict__ missing) {
  __shared__ PlanShared sh;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  for (int i = w; i < q.n; i += kPlanWaves) release(a, q.dst[i], lane);
  __builtin_amdgcn_s_waitcnt(0);  // the counts are down; (a fence of the device's scope took 3 us)
  __syncthreads();
  const int in_page = (1 << a.lg) - 1;
  take_pages(a, q.n, sh, missing, [&](int i) { return (seq_len(a, q.src[i]) & in_page) ? 1 : 0; },
             [&](int i, int, int id) { a.table[(int64_t)q.dst[i] * a.table_ld + (seq_len(a, q.src[i]) >> a.lg)] = id; });
  for (int i = threadIdx.x; i < q.n; i += kPlanThreads)
    if (missing[i] == 0) a.len[q.dst[i]] = seq_len(a, q.src[i]);
}

// The rest of a fork, one workgroup a pair, layer and matrix: the rows of src[i]'s last page, where it is not
// full; the first one also shares the full pages.  32 children, 4 layers: 6.7 us, a chain of loads (shared by
// the plan's workgroup alone, the pages took it 3 us more).
__global__ __launch_bounds__(256) void k_fork_rows(PageArgs a, SeqPairs q, const int32_t* __restrict__ missing) {
  const int i = blockIdx.x;
  if (missing[i] != 0) return;
  const int n = seq_len(a, q.src[i]), rest = n & ((1 << a.lg) - 1);
  if (blockIdx.y == 0 && blockIdx.z == 0) {
    const int32_t* from = a.table + (int64_t)q.src[i] * a.table_ld;
    int32_t* to = a.table + (int64_t)q.dst[i] * a.table_ld;
    for (int j = threadIdx.x; j < n >> a.lg; j += 256) {
      const int id = from[j];
      if (id >= 0 && id < a.n_pages) atomicAdd(a.refs + id, 1);
      to[j] = id;
    }
  }
  if (rest == 0) return;
  const int64_t from = slot_of(a, q.src[i], n - rest), to = slot_of(a, q.dst[i], n - rest);
  if (from < 0 || to < 0) return;
  uint8_t* base = (blockIdx.z ? a.v : a.k) + blockIdx.y * a.layer_bytes;
  const int64_t bytes = (int64_t)rest * a.row_bytes;
  for (int64_t c = threadIdx.x * 16; c < bytes; c += 4096)
    *(uint4*)(base + to * a.row_bytes + c) = *(const uint4*)(base + from * a.row_bytes + c);
}

// Pages in use with ids >= their number n_live change places with the free ones below, both in
// ascending order.  ws: [0] = moves, then map[n_pages] (new id of every page), from[], to[].  2048 pages: 4.8 us
// (a fence of the device's scope between the lists and their use took another 4).
__global__ __launch_bounds__(kPlanThreads) void k_compact_plan(PageArgs a, int32_t* __restrict__ n_live, int32_t* __restrict__ ws) {
  __shared__ int32_t wave[kPlanWaves];
  constexpr int kRound = 4 * kPlanThreads;
  // bits 0..3: which of this thread's four pages of a round are in use; the first round's are kept
  auto in_use = [&](int base) {
    int bits = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int id = base + 4 * (int)threadIdx.x + i;
      bits |= (id < a.n_pages && a.refs[id] > 0) << i;
    }
    return bits;
  };
  const int first = in_use(0);
  int live = 0, sum;
  for (int base = 0; base < a.n_pages; base += kRound) {
    block_scan(__builtin_popcount(base ? in_use(base) : first), wave, &sum);
    live += sum;
  }
  int32_t *map = ws + 1, *from = map + a.n_pages, *to = from + a.n_pages / 2;
  int holes = 0, movers = 0;
  for (int base = 0; base < a.n_pages; base += kRound) {
    const int bits = base ? in_use(base) : first, id0 = base + 4 * (int)threadIdx.x;
    int mine = 0;  // holes, and movers in the upper half (a round has 4096 of both together)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int id = id0 + i;
      if (id < a.n_pages) mine += id < live ? !(bits >> i & 1) : (bits >> i & 1) << 16;
    }
    const int before = block_scan(mine, wave, &sum) - mine;
    int h = holes + (before & 0xffff), m = movers + (before >> 16);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int id = id0 + i;
      if (id >= a.n_pages) continue;
      const bool used = bits >> i & 1;
      map[id] = id;
      if (id < live && !used) to[h++] = id;
      if (id >= live && used) from[m++] = id;
    }
    holes += sum & 0xffff;
    movers += sum >> 16;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < movers; i += kPlanThreads) {
    const int f = from[i], t = to[i];
    map[f] = t;
    a.refs[t] = a.refs[f];
    a.refs[f] = 0;
  }
  if (threadIdx.x == 0) {
    ws[0] = movers;
    if (n_live) *n_live = live;
  }
}

// New ids in the tables (blocks beyond the first `copies`, a wave a sequence and then further ones), and the moved
// pages' contents.
__global__ __launch_bounds__(256) void k_compact_move(PageArgs a, const int32_t* __restrict__ ws, int copies) {
  const int32_t *map = ws + 1, *from = map + a.n_pages, *to = from + a.n_pages / 2;
  if ((int)blockIdx.x >= copies) {
    for (int64_t seq = (blockIdx.x - copies) * 4 + (threadIdx.x >> 6); seq < a.n_seqs; seq += 4 * ((int)gridDim.x - copies)) {
      const int n = pages_of(a, seq_len(a, (int)seq));
      int32_t* row = a.table + seq * a.table_ld;
      for (int j = threadIdx.x & 63; j < n; j += 64) {
        const int id = row[j];
        if (id >= 0 && id < a.n_pages) row[j] = map[id];
      }
    }
    return;
  }
  const int moves = ws[0];
  const int64_t page_bytes = (int64_t)a.row_bytes << a.lg;
  const int64_t items = (int64_t)moves * a.n_layers * 2;
  for (int64_t it = blockIdx.x; it < items; it += copies) {
    const int m = (int)(it / (a.n_layers * 2)), l = (int)(it % (a.n_layers * 2));
    uint8_t* base = (l & 1 ? a.v : a.k) + (l >> 1) * a.layer_bytes;
    const uint8_t* src = base + from[m] * page_bytes;
    uint8_t* dst = base + to[m] * page_bytes;
    copy_bytes(dst, src, page_bytes, threadIdx.x, 256);
  }
}

// The confirmed paths of `count` trees from sequence b0 on, from node 0: the next node is the first child
// whose token is the model's choice at the present one.  Every node offers itself to its parent (the lowest
// wins), then a thread a tree follows the winners.  child: count * N words of LDS.
__device__ __forceinline__ void walk_trees(const TreePick& t, int b0, int count, int32_t* child) {
  const int N = t.N;
  auto nodes = [&](int b) { return t.n_nodes ? min(max(t.n_nodes[b], 0), N) : N; };
  for (int x = threadIdx.x; x < count * N; x += blockDim.x) child[x] = N;
  __syncthreads();
  for (int x = threadIdx.x; x < count * N; x += blockDim.x) {
    const int s = x / N, j = x - s * N;
    const int64_t row = (int64_t)(b0 + s) * N;
    t.accepted[row + j] = -1;
    if (j == 0 || j >= nodes(b0 + s)) continue;
    const int p = t.parents ? t.parents[row + j] : j - 1;
    if (p >= 0 && p < j && t.tokens[row + j] == t.chosen[row + p]) atomicMin(child + s * N + p, j);
  }
  __syncthreads();
  for (int s = threadIdx.x; s < count; s += blockDim.x) {
    const int b = b0 + s;
    int n = 0, last = -1;
    for (int cur = nodes(b) > 0 ? 0 : N; cur < N; cur = child[s * N + cur]) {
      t.accepted[(int64_t)b * N + n++] = cur;
      last = cur;
    }
    t.n_accepted[b] = n;
    t.token_out[b] = last < 0 ? -1 : t.chosen[(int64_t)b * N + last];
  }
  __syncthreads();
}

// Larger batches: a workgroup each kWalkWords words of nodes.
constexpr int kWalkWords = 4096;
__global__ __launch_bounds__(256) void k_tree_walk(TreePick t, int B) {
  __shared__ int32_t child[kWalkWords];
  const int per = kWalkWords / t.N, b0 = blockIdx.x * per;
  walk_trees(t, b0, min(per, B - b0), child);
}

// Room for the confirmed tokens; a sequence without it commits nothing.
// The trees of a small batch (kWalkWords nodes) are walked here, without a launch of their own: 64 trees of 16
// nodes 5.2 us instead of 3.9 + 3.4, 64 of 64 nodes 7.5 instead of 10.0 + 3.6.
template <bool WALK>
__global__ __launch_bounds__(kPlanThreads) void k_commit_plan(PageArgs a, TreePick t, int B, int32_t* __restrict__ missing) {
  __shared__ PlanShared sh;
  __shared__ int32_t child[WALK ? kWalkWords : 1];
  if (WALK) walk_trees(t, 0, B, child);
  auto need = [&](int b) {
    const int at = seq_len(a, b);
    const int64_t end = (int64_t)at + t.n_accepted[b];
    if (end > (int64_t)a.table_ld << a.lg) return -1;
    return pages_of(a, (int)end) - pages_of(a, at);
  };
  take_pages(a, B, sh, missing, need, [&](int b, int k, int id) {
    a.table[(int64_t)b * a.table_ld + pages_of(a, seq_len(a, b)) + k] = id;
  });
  for (int b = threadIdx.x; b < B; b += kPlanThreads) {
    if (missing[b] == 0) {
      a.len[b] = seq_len(a, b) + t.n_accepted[b];
    } else {
      for (int j = 0; j < t.n_accepted[b]; ++j) t.accepted[(int64_t)b * t.N + j] = -1;
      t.n_accepted[b] = 0;
      t.token_out[b] = -1;
    }
  }
}

__global__ __launch_bounds__(256) void k_commit_rows(PageArgs a, int N, const int32_t* __restrict__ accepted,
                                                     const int32_t* __restrict__ n_accepted, const uint8_t* __restrict__ k,
                                                     const uint8_t* __restrict__ v, int64_t layer_bytes) {
  const int b = blockIdx.x, lane = threadIdx.x & 63;
  const int n = n_accepted[b];
  const int first = seq_len(a, b) - n;
  for (int j = threadIdx.x >> 6; j < n; j += 4) {
    const int64_t to = first + j >= 0 ? slot_of(a, b, first + j) : -1;
    if (to < 0) continue;
    const int64_t r = (int64_t)b * N + accepted[(int64_t)b * N + j];
    const uint8_t* src = (blockIdx.z ? v : k) + blockIdx.y * layer_bytes + r * a.row_bytes;
    uint8_t* dst = (blockIdx.z ? a.v : a.k) + blockIdx.y * a.layer_bytes + to * a.row_bytes;
    for (int c = lane * 16; c < a.row_bytes; c += 1024) *(uint4*)(dst + c) = *(const uint4*)(src + c);
  }
}

hipError_t launch_append_plan(hipStream_t s, const PageArgs& a, const SeqRows& q, int32_t* missing) {
  k_append_plan<<<1, kPlanThreads, 0, s>>>(a, q, missing);
  return hipGetLastError();
}
hipError_t launch_append_rows(hipStream_t s, const PageArgs& a, const SeqRows& q, const void* k, const void* v,
                              int64_t layer_bytes, const int32_t* missing) {
  // a launch has fewer than 2^32 threads in x; with more it runs their number modulo 2^32, without an error
  constexpr int kMostRows = 1 << 24;
  const int rows = q.cu[q.n];
  for (int first = 0; first < rows; first += kMostRows) {
    const int groups = (std::min(rows - first, kMostRows) + 3) / 4;
    k_append_rows<<<dim3(groups, a.n_layers, 2), 256, 0, s>>>(a, q, (const uint8_t*)k, (const uint8_t*)v, layer_bytes, missing, first);
  }
  return hipGetLastError();
}
hipError_t launch_pages_free(hipStream_t s, const PageArgs& a, const SeqRows& q) {
  k_pages_free<<<(q.n + 3) / 4, 256, 0, s>>>(a, q);
  return hipGetLastError();
}
hipError_t launch_fork_plan(hipStream_t s, const PageArgs& a, const SeqPairs& q, int32_t* missing) {
  k_fork_plan<<<1, kPlanThreads, 0, s>>>(a, q, missing);
  return hipGetLastError();
}
hipError_t launch_fork_rows(hipStream_t s, const PageArgs& a, const SeqPairs& q, const int32_t* missing) {
  k_fork_rows<<<dim3(q.n, a.n_layers, 2), 256, 0, s>>>(a, q, missing);
  return hipGetLastError();
}
size_t compact_words(int32_t n_pages) { return 1 + 2 * (size_t)n_pages; }
hipError_t launch_compact_plan(hipStream_t s, const PageArgs& a, int32_t* n_live, int32_t* ws) {
  k_compact_plan<<<1, kPlanThreads, 0, s>>>(a, n_live, ws);
  return hipGetLastError();
}
hipError_t launch_compact_move(hipStream_t s, const PageArgs& a, const int32_t* ws) {
  const int copies = (int)std::min<int64_t>(2048, (int64_t)(a.n_pages / 2 + 1) * a.n_layers * 2);
  const int tables = (int)std::min<int64_t>(1 << 16, ((int64_t)a.n_seqs + 3) / 4);  // (2^32 threads run as none)
  k_compact_move<<<copies + tables, 256, 0, s>>>(a, ws, copies);
  return hipGetLastError();
}
bool commit_walks(int32_t B, int32_t N) { return (int64_t)B * N <= kWalkWords; }
hipError_t launch_tree_walk(hipStream_t s, const TreePick& t, int32_t B) {
  const int per = kWalkWords / t.N;
  k_tree_walk<<<(B + per - 1) / per, 256, 0, s>>>(t, B);
  return hipGetLastError();
}
hipError_t launch_commit_plan(hipStream_t s, const PageArgs& a, const TreePick& t, int32_t B, int32_t* missing) {
  if (commit_walks(B, t.N))
    k_commit_plan<true><<<1, kPlanThreads, 0, s>>>(a, t, B, missing);
  else
    k_commit_plan<false><<<1, kPlanThreads, 0, s>>>(a, t, B, missing);
  return hipGetLastError();
}
hipError_t launch_commit_rows(hipStream_t s, const PageArgs& a, int32_t B, int32_t N, const int32_t* accepted,
                              const int32_t* n_accepted, const void* k, const void* v, int64_t layer_bytes) {
  k_commit_rows<<<dim3(B, a.n_layers, 2), 256, 0, s>>>(a, N, accepted, n_accepted, (const uint8_t*)k, (const uint8_t*)v, layer_bytes);
  return hipGetLastError();
}

}  // namespace rp
