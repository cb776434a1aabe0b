// pages.hip -- the pages of a batch's caches: forks, growth with copy on write,
// compaction, the copies that these ask for, and new rows of bf16 caches.
//
// The bookkeeping is whole numbers and every result follows from the arguments
// alone: free pages are dealt in ascending order, sequence after sequence, and the
// only atomics are integer sums.  refs counts the entries that name a page, so a
// page is free where it is not positive.
#include <algorithm>

#include "jl_device.h"
#include "pages.h"

namespace jl {

__device__ inline bool in_pool(int p, int n_pages) { return (unsigned)p < (unsigned)n_pages; }

constexpr int kBookThreads = 1024;  // of the calls that one workgroup makes; small ones take 256
constexpr int kBookWaves = kBookThreads / 64;

// Inclusive sums over the workgroup's threads, in thread order, of one value or a
// pair; s: kBookWaves entries.  Everyone gets the total too.
template <typename T>
__device__ inline T block_scan(T v, T* s, T* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const T incl = wave_scan(v);
  __syncthreads();  // s may still be read from the last scan
  if (lane == 63) s[wave] = incl;
  __syncthreads();
  T before = 0, all = 0;
#pragma unroll
  for (int i = 0; i < kBookWaves; i += 4) {
    if (64 * i >= (int)blockDim.x) break;
#pragma unroll
    for (int j = i; j < i + 4; ++j) {
      const T x = s[j];
      if (j < wave) before += x;
      all += x;
    }
  }
  *total = all;
  return before + incl;
}

// ------------------------------------------------------------------- fork
// Row b becomes what row parent[b] was, or empty where parent[b] names none, all
// rows at once.  A workgroup takes some columns of every row: what the rows get
// goes to LDS before any of them is written.  Rows that stay are not read.
// lens is read and written by the first workgroup alone.  Bound by reads that follow each other
// (parent, the parent's entry, the row's own): 256 rows of 2048 columns of which 64 change 9.4 us,
// 7.8 without the counts' atomics; 32 rows of 64: 3.9, a launch.
struct ForkArgs {
  Pages p;
  const int32_t* parent;
  int cols;  // columns of a workgroup
};

__global__ __launch_bounds__(kBookThreads) void fork_kernel(ForkArgs a) {
  extern __shared__ int32_t s_new[];  // [B][cols]
  const Pages& p = a.p;
  const int c0 = blockIdx.x * a.cols;
  const int n = p.B * a.cols;
  for (int i = threadIdx.x; i < n; i += blockDim.x) {
    const int b = i / a.cols, c = c0 + i - b * a.cols;
    const int from = a.parent[b];
    int page = -1;
    if (from != b && (unsigned)from < (unsigned)p.B && c < p.max_pages)
      page = p.table[(size_t)from * p.max_pages + c];
    s_new[i] = page;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += blockDim.x) {
    const int b = i / a.cols, c = c0 + i - b * a.cols;
    if (a.parent[b] == b || c >= p.max_pages) continue;
    int32_t* at = p.table + (size_t)b * p.max_pages + c;
    const int was = *at, now = s_new[i];
    if (was == now) continue;
    *at = now;
    if (in_pool(was, p.n_pages)) atomicAdd(p.refs + was, -1);
    if (in_pool(now, p.n_pages)) atomicAdd(p.refs + now, 1);
  }
  if (blockIdx.x != 0) return;
  __syncthreads();
  for (int b = threadIdx.x; b < p.B; b += blockDim.x) {
    const int from = a.parent[b];
    s_new[b] = (unsigned)from < (unsigned)p.B ? p.lens[from] : 0;
  }
  __syncthreads();
  for (int b = threadIdx.x; b < p.B; b += blockDim.x) p.lens[b] = s_new[b];
}

// ---------------------------------------------------------------- reserve
// Pages for n_new[b] more rows of every sequence.  One workgroup: the needs of the
// sequences (thread t: a run of them, so that the scan follows their order), how
// many pages are free, then the k-th free page goes to the sequence whose range of
// needs holds k.  A sequence that writes into a partly filled page which others
// name too gets a fresh one for it, but for the last writer of a page that only
// writers name.  If the pages do not suffice nothing is changed.  Before all this, pages that
// a sequence still names behind its last one (its length was lowered) are given up.  Bound by
// latency: length, entries, count, sums and the second read of the counts follow each other (16
// sequences, 512 pages: 11.6 us, 0.4 of them for the entries behind; 12.7 with 1024 threads and
// 64-bit divisions, without those).
struct ReserveArgs {
  Pages p;
  const int32_t* n_new;
  int32_t* starts;
  int32_t* granted;
  int32_t* moves;  // [B][2]: from, to
  int32_t* info;   // moves, pages dealt, pages missing, sequences past max_pages
};

constexpr int kStripPer = 16;  // counts a thread reads at once; a strip: what the workgroup does

// Bits of the free ones among 16 counts from `at` on
__device__ inline uint32_t free_mask(const int32_t* refs, int at, int n_pages) {
  uint32_t m = 0;
  if (at + kStripPer <= n_pages) {
    int4 v[kStripPer / 4];
#pragma unroll
    for (int i = 0; i < kStripPer / 4; ++i) v[i] = ((const int4*)(refs + at))[i];
#pragma unroll
    for (int i = 0; i < kStripPer / 4; ++i)
      m |= (uint32_t)((v[i].x <= 0) | (v[i].y <= 0) << 1 | (v[i].z <= 0) << 2 | (v[i].w <= 0) << 3)
           << (4 * i);
  } else {
    for (int i = 0; i < kStripPer && at + i < n_pages; ++i) m |= (uint32_t)(refs[at + i] <= 0) << i;
  }
  return m;
}

__global__ __launch_bounds__(kBookThreads) void reserve_kernel(ReserveArgs a) {
  extern __shared__ int32_t smem[];
  __shared__ unsigned long long s_scan[kBookWaves];
  __shared__ int s_behind[kBookWaves];
  const Pages& p = a.p;
  int32_t* const s_last = smem;              // the shared page it writes into, else -1 (16-byte aligned)
  int32_t* const s_first = s_last + ((p.B + 3) & ~3);  // needs before sequence b
  int32_t* const s_had = s_first + p.B;      // its pages
  int32_t* const s_move = s_had + p.B;       // its move; -1: no page is replaced, -2: without a copy
  int32_t* const s_len = s_move + p.B;
  const int tid = threadIdx.x, nt = blockDim.x, strip_pages = kStripPer * nt;

  const int n_strips = (p.n_pages + strip_pages - 1) / strip_pages;
  uint32_t mask0;  // the counts of the first strip, on their way while the needs are formed

  const int per = (p.B + nt - 1) >> (31 - __builtin_clz(nt));
  const int b0 = min(tid * per, p.B), b1 = min(b0 + per, p.B);
  for (int turn = 0;; ++turn) {
    mask0 = free_mask(p.refs, min(tid * kStripPer, p.n_pages), p.n_pages);
    bool behind = false;  // one of this thread's names pages behind its last one: the first in s_had
    for (int b = b0; b < b1; ++b) {
      const int len = max(p.lens[b], 0), n = a.n_new[b];
      const int32_t* const row = p.table + (size_t)b * p.max_pages;
      const int slot = (int)((unsigned)len / (unsigned)p.page);
      const int end = slot + (len != slot * p.page);
      const int e = row[min(slot, p.max_pages - 1)], f = row[min(end, p.max_pages - 1)];
      int last = -1, count = 0, next = -1;
      if (end < p.max_pages && in_pool(f, p.n_pages)) {
        next = end;
        behind = true;
      }
      if (n > 0 && end != slot && slot < p.max_pages) {
        last = -2;
        if (in_pool(e, p.n_pages)) {
          count = p.refs[e];
          last = count > 1 ? e : -1;
        }
      }
      s_last[b] = last;
      s_first[b] = count;
      s_len[b] = len;
      s_had[b] = next;
    }
    const unsigned long long some = __ballot(behind);
    if ((tid & 63) == 0) s_behind[tid >> 6] = some != 0;
    __syncthreads();
    bool any = false;
    for (int i = 0; i < nt >> 6; ++i) any |= s_behind[i] != 0;
    if (!any || turn == 1) break;
    for (int b = tid >> 6; b < p.B; b += nt >> 6) {  // a wave for each
      if (s_had[b] < 0) continue;
      int32_t* const row = p.table + (size_t)b * p.max_pages;
      for (unsigned c = s_had[b] + (tid & 63);; c += 64) {
        const int e = c < (unsigned)p.max_pages ? row[c] : -1;
        const unsigned long long none = __ballot(!in_pool(e, p.n_pages));
        if (none == 0 || (tid & 63) < __builtin_ctzll(none)) {
          row[c] = -1;
          atomicAdd(p.refs + e, -1);
        }
        if (none != 0) break;
      }
    }
    __threadfence();  // entries and counts are written
    __syncthreads();
    __threadfence();  // and read anew
  }
  const int cap = p.max_pages * p.page;
  long long need = 0;
  int n_moves = 0, over = 0;
  for (int b = b0; b < b1; ++b) {
    // a length of any kind past the capacity counts as one just past it
    const int len = s_len[b], n = max(a.n_new[b], 0);
    const unsigned end = min((unsigned)len + (unsigned)n, (unsigned)cap + 1u);
    const int has = end == 0 ? 0 : (int)((end - 1) / (unsigned)p.page + 1);
    const int had = min(len == 0 ? 0 : (int)((unsigned)(len - 1) / (unsigned)p.page + 1), has);
    const int last = s_last[b];
    int move = -1;
    if (last == -2) {
      move = -2;
    } else if (last >= 0) {
      int left = s_first[b];  // less the writers before this one
      int e = 0;
      for (; e + 16 <= b; e += 16) {
        int4 x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = ((const int4*)(s_last + e))[i];
#pragma unroll
        for (int i = 0; i < 4; ++i)
          left -= (x[i].x == last) + (x[i].y == last) + (x[i].z == last) + (x[i].w == last);
      }
      for (; e < b; ++e) left -= s_last[e] == last;
      if (left > 1) move = n_moves++;
    }
    over += has > p.max_pages && n > 0;
    s_first[b] = (int)min(need, 0x7fffffffLL);
    s_had[b] = had;
    s_move[b] = move;
    need += (n > 0 ? has - had : 0) + (move != -1);
  }
  // a run's needs may pass 32 bits only where a sequence is past max_pages
  unsigned long long tot, tot2;
  const unsigned long long mine =
      (unsigned long long)min(need, 0x7fffffffLL) | (unsigned long long)n_moves << 44;
  const unsigned long long incl = block_scan(mine, s_scan, &tot);
  const unsigned long long over_free =
      (unsigned long long)over << 40;
  uint32_t n_free = __popc(mask0);
  for (int s = 1; s < n_strips; ++s)
    n_free += __popc(free_mask(p.refs, min(s * strip_pages + tid * kStripPer, p.n_pages), p.n_pages));
  block_scan(over_free + n_free, s_scan, &tot2);
  const long long total = (long long)(tot & ((1ull << 44) - 1));
  const long long all_free = (long long)(tot2 & ((1ull << 40) - 1));
  const int all_over = (int)(tot2 >> 40), all_moves = (int)(tot >> 44);
  const bool fits = all_over == 0 && total <= all_free;
  const unsigned long long before = incl - mine;
  for (int b = b0; b < b1; ++b) {
    s_first[b] += (int)(before & ((1ull << 44) - 1));
    if (s_move[b] >= 0) s_move[b] += (int)(before >> 44);
  }
  __syncthreads();
  if (tid == 0) {
    a.info[0] = fits ? all_moves : 0;
    a.info[1] = fits ? (int)total : 0;
    a.info[2] = (int)min(max(total - all_free, 0LL), 0x7fffffffLL);
    a.info[3] = all_over;
  }
  for (int b = tid; b < p.B; b += nt) {
    const int n = fits ? max(a.n_new[b], 0) : 0;
    const int len = s_len[b];
    a.starts[b] = len;
    a.granted[b] = n;
    if (n > 0) p.lens[b] = len + n;
    if (fits && s_move[b] >= 0) {
      a.moves[2 * s_move[b]] = s_last[b];
      atomicAdd(p.refs + s_last[b], -1);
    }
    if (b >= (fits ? all_moves : 0)) a.moves[2 * b] = a.moves[2 * b + 1] = -1;
  }
  if (!fits || total == 0) return;
  unsigned long long base = 0;
  for (int s = 0; s < n_strips && base < (unsigned long long)total; ++s) {
    const int at = min(s * strip_pages + tid * kStripPer, p.n_pages);
    // pages dealt in an earlier strip are not read again, and the counts lowered
    // above stay positive
    uint32_t m = s == 0 ? mask0 : free_mask(p.refs, at, p.n_pages);
    unsigned long long strip;
    const int cnt = __popc(m);
    long long k = (long long)(base + block_scan((unsigned long long)cnt, s_scan, &strip) - cnt);
    base += strip;
    int b = -1;
    for (; m != 0 && k < total; m &= m - 1, ++k) {
      const int page = at + __builtin_ctz(m);
      if (b < 0 || (b + 1 < p.B && s_first[b + 1] <= k)) {  // the last sequence that begins at or before k
        int lo = 0, hi = p.B - 1;
        while (lo < hi) {
          const int mid = (lo + hi + 1) >> 1;
          if (s_first[mid] <= k) lo = mid; else hi = mid - 1;
        }
        b = lo;
      }
      const int off = (int)(k - s_first[b]), move = s_move[b];
      const int slot = s_had[b] + off - (move != -1);
      p.table[(size_t)b * p.max_pages + slot] = page;
      p.refs[page] = 1;
      if (off == 0 && move >= 0) a.moves[2 * move + 1] = page;
    }
  }
}

// ---------------------------------------------------------------- compact
// With n pages in use, the i-th of those numbered n or more moves to the i-th free
// one below n.  One workgroup lists the moves and where each page went; then the
// tables follow.  Latency: 3.3 us and 2.2 with 512 pages, 5.3 with 4096.
struct CompactArgs {
  Pages p;
  int32_t* moves;  // [n_pages / 2][2]
  int32_t* to;     // [n_pages]: new number of the pages that move
  int32_t* info;   // moves, pages in use, 0, 0
};

__global__ __launch_bounds__(kBookThreads) void compact_kernel(CompactArgs a) {
  __shared__ unsigned long long s_scan[kBookWaves];
  const Pages& p = a.p;
  const int tid = threadIdx.x, nt = blockDim.x, strip_pages = kStripPer * nt;
  const int n_strips = (p.n_pages + strip_pages - 1) / strip_pages;
  uint32_t mask0 = 0;
  unsigned long long used = 0, n_live;
  for (int s = 0; s < n_strips; ++s) {
    const int at = min(s * strip_pages + tid * kStripPer, p.n_pages);
    const uint32_t m = free_mask(p.refs, at, p.n_pages);
    if (s == 0) mask0 = m;
    used += min(kStripPer, p.n_pages - at) - __popc(m);
  }
  block_scan(used, s_scan, &n_live);
  const int live = (int)n_live;
  unsigned long long base = 0;  // free pages below `live` (low half), used ones above it
  for (int s = 0; s < n_strips; ++s) {
    const int at = min(s * strip_pages + tid * kStripPer, p.n_pages);
    const uint32_t m = s == 0 ? mask0 : free_mask(p.refs, at, p.n_pages);
    const int n = min(kStripPer, p.n_pages - at);
    const uint32_t below = live >= at + 16 ? 0xffffu : live <= at ? 0u : (1u << (live - at)) - 1;
    uint32_t holes = m & below, high = ~m & ~below & ((1u << n) - 1);
    unsigned long long strip;
    const unsigned long long cnt =
        (unsigned long long)__popc(holes) | (unsigned long long)__popc(high) << 32;
    const unsigned long long k = base + block_scan(cnt, s_scan, &strip) - cnt;
    base += strip;
    int i = (int)(uint32_t)k, j = (int)(k >> 32);
    for (; holes != 0; holes &= holes - 1) a.moves[2 * i++ + 1] = at + __builtin_ctz(holes);
    for (; high != 0; high &= high - 1) a.moves[2 * j++] = at + __builtin_ctz(high);
  }
  const int n_moves = (int)(uint32_t)base;  // as many free ones below as used ones above
  __syncthreads();
  for (int i = tid; i < p.n_pages / 2; i += nt) {
    if (i < n_moves) {
      const int from = a.moves[2 * i], to = a.moves[2 * i + 1];
      a.to[from] = to;
      p.refs[to] = p.refs[from];
      p.refs[from] = 0;
    } else {
      a.moves[2 * i] = a.moves[2 * i + 1] = -1;
    }
  }
  if (tid == 0) {
    a.info[0] = n_moves;
    a.info[1] = live;
    a.info[2] = a.info[3] = 0;
  }
}

__global__ __launch_bounds__(256) void retable_kernel(CompactArgs a) {
  const Pages& p = a.p;
  const size_t n = (size_t)p.B * p.max_pages;
  const int live = a.info[1];
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (size_t)gridDim.x * 256) {
    const int e = p.table[i];
    if (e >= live && e < p.n_pages) p.table[i] = a.to[e];
  }
}

// ------------------------------------------------------------- page copies
// Moves are cut into units of 16 KB of one pool, dealt to the workgroups in turn.
// Bound by HBM: 8 pools, 1.9 GB read and written in 370 us, 5.1 TB/s; few moves are a launch (4 us).
constexpr int kCopyUnit = 16384;

template <typename V>
__device__ inline void copy_unit(const unsigned char* src, unsigned char* dst, int bytes) {
  constexpr int kPer = 4;
  const int n = bytes / (int)sizeof(V);
  for (int i0 = 0; i0 < n; i0 += 256 * kPer) {
    V v[kPer];
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const int i = i0 + 256 * j + threadIdx.x;
      if (i < n) v[j] = __builtin_nontemporal_load((const V*)src + i);
    }
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const int i = i0 + 256 * j + threadIdx.x;
      if (i < n) __builtin_nontemporal_store(v[j], (V*)dst + i);
    }
  }
}

__global__ __launch_bounds__(256) void copy_pages_kernel(CopyPools a, const int32_t* moves,
                                                         const int32_t* info) {
  const int per = a.first[a.n_pools];
  const long long n = (long long)min(max(info[0], 0), a.max_moves) * per;
  for (long long u = blockIdx.x; u < n; u += gridDim.x) {
    const int mv = (int)(u / per), at = (int)(u - (long long)mv * per);
    const int from = moves[2 * mv], to = moves[2 * mv + 1];
    if (!in_pool(from, a.n_pages) || !in_pool(to, a.n_pages)) continue;
    int i = 0;
    while (at >= a.first[i + 1]) ++i;
    const unsigned long long bytes = a.bytes[i], off = (unsigned long long)(at - a.first[i]) * kCopyUnit;
    const int len = (int)min(bytes - off, (unsigned long long)kCopyUnit);
    const unsigned char* src = a.ptr[i] + (unsigned long long)from * bytes + off;
    unsigned char* dst = a.ptr[i] + (unsigned long long)to * bytes + off;
    if ((((uintptr_t)a.ptr[i] | bytes) & 15) == 0)
      copy_unit<u32x4>(src, dst, len);
    else
      copy_unit<unsigned int>(src, dst, len);
  }
}

// ------------------------------------------------------------------ append
// Rows of bf16 caches: a wave takes one new token (or several in turn), whose K and
// V rows of all heads are contiguous on both sides, 16 bytes a lane.  Bound by HBM: prompts of 266 MB
// read and written in 41 us, 6.5 TB/s; a token of 16 sequences 3.5 us, a launch.
struct RowsArgs {
  const u32x4* k;
  const u32x4* v;
  u32x4* kc;
  u32x4* vc;
  const int32_t* table;  // nullptr: page b is sequence b
  const int32_t* starts;
  const int32_t* n_new;  // nullptr: all
  const int32_t* cu;     // packed rows; nullptr: n rows per sequence
  int B, n, max_pages, n_pages, page, chunks;  // chunks: 16-byte pieces of a token's K
  long long rows, cap;
};

constexpr int kAppendWaves = 4;
// Workgroups at most: a launch counts its threads in 32 bits and drops what lies past them
constexpr int kAppendGrid = 1 << 22;

__global__ __launch_bounds__(64 * kAppendWaves) void append_kernel(RowsArgs a) {
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const long long stride = (long long)gridDim.x * kAppendWaves;
  for (long long t = (long long)blockIdx.x * kAppendWaves + wave; t < a.rows; t += stride) {
    int b, at;
    if (a.cu != nullptr) {  // the last sequence that begins at or before t: cu is not decreasing
      int before = 0;
      for (int c = lane; c - lane < a.B; c += 64)
        before += __popcll(__ballot(c < a.B && a.cu[c + 1] <= t));
      b = __builtin_amdgcn_readfirstlane(before);
      if (b >= a.B) continue;
      const long long o = t - a.cu[b];
      if (o < 0) continue;
      at = (int)o;
    } else {
      b = (int)(t / a.n);
      at = (int)(t - (long long)b * a.n);
    }
    if (a.n_new != nullptr && at >= a.n_new[b]) continue;
    const long long pos = (long long)a.starts[b] + at;
    if (pos < 0 || pos >= a.cap) continue;
    const int slot = (int)(pos / a.page);
    const int page = a.table != nullptr ? a.table[(size_t)b * a.max_pages + slot] : b;
    if (!in_pool(page, a.n_pages)) continue;
    const size_t to = ((size_t)page * a.page + (size_t)(pos - (long long)slot * a.page)) * a.chunks;
    const size_t from = (size_t)t * a.chunks;
    for (int c = lane; c < a.chunks; c += 64) {
      const u32x4 x = a.k[from + c], y = a.v[from + c];
      a.kc[to + c] = x;
      a.vc[to + c] = y;
    }
  }
}

// ---------------------------------------------------------------- launchers
// Barriers of four waves cost less; more counts than four of their strips take the larger one
static int book_threads(const Pages& p) {
  return p.B <= 256 && p.n_pages <= 4 * 256 * kStripPer ? 256 : kBookThreads;
}
static int fork_cols(int B, int max_pages) {
  int c = 32;  // 128 bytes of a row, 64 KB in all; fewer where the grid would not fill the CUs
  while (c > 8 && max_pages / c < 128) c /= 2;
  while (c > 1 && (size_t)c * B * sizeof(int32_t) > (size_t)64 * 1024) c /= 2;
  // more where the launch would pass the threads that 32 bits count
  while (max_pages / c >= 1 << 20 && (size_t)2 * c * B * sizeof(int32_t) <= (size_t)64 * 1024) c *= 2;
  return c;
}

hipError_t launch_pages_fork(const Pages& p, const int32_t* parent, hipStream_t stream) {
  ForkArgs a{p, parent, fork_cols(p.B, p.max_pages)};
  const int grid = (int)(((long long)p.max_pages + a.cols - 1) / a.cols);
  const size_t lds = (size_t)a.cols * p.B * sizeof(int32_t);
  hipLaunchKernelGGL(fork_kernel, dim3(grid), dim3(p.B * a.cols <= 1024 ? 256 : kBookThreads), lds, stream, a);
  return hipGetLastError();
}

hipError_t launch_pages_reserve(const Pages& p, const int32_t* n_new, int32_t* starts,
                                int32_t* granted, int32_t* moves, int32_t* info,
                                hipStream_t stream) {
  ReserveArgs a{p, n_new, starts, granted, moves, info};
  hipLaunchKernelGGL(reserve_kernel, dim3(1), dim3(book_threads(p)), (size_t)(p.B + 3) * 20, stream, a);
  return hipGetLastError();
}

hipError_t launch_pages_compact(const Pages& p, int32_t* moves, int32_t* to, int32_t* info,
                                hipStream_t stream) {
  CompactArgs a{p, moves, to, info};
  hipLaunchKernelGGL(compact_kernel, dim3(1), dim3(book_threads(p)), 0, stream, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const size_t n = (size_t)p.B * p.max_pages;
  hipLaunchKernelGGL(retable_kernel, dim3((unsigned)std::min<size_t>((n + 255) / 256, 2048)),
                     dim3(256), 0, stream, a);
  return hipGetLastError();
}

// Units of one move over these pools; a.first is filled in.
long long copy_units(CopyPools& a) {
  long long at = 0;
  for (int i = 0; i < a.n_pools; ++i) {
    a.first[i] = (int)at;
    at += (long long)((a.bytes[i] + kCopyUnit - 1) / kCopyUnit);
    if (at > 0x7fffffffLL) return -1;
  }
  a.first[a.n_pools] = (int)at;
  return at;
}

hipError_t launch_copy_pages(const CopyPools& a, const int32_t* moves, const int32_t* info,
                             int n_cu, hipStream_t stream) {
  const long long units = (long long)a.first[a.n_pools] * a.max_moves;
  hipLaunchKernelGGL(copy_pages_kernel, dim3((unsigned)std::min<long long>(units, 8LL * n_cu)),
                     dim3(256), 0, stream, a, moves, info);
  return hipGetLastError();
}

hipError_t launch_cache_append(const uint16_t* k, const uint16_t* v, uint16_t* kc, uint16_t* vc,
                               const int32_t* table, int max_pages, int n_pages, int page,
                               const int32_t* starts, const int32_t* n_new, const int32_t* cu,
                               int B, int n, int Hkv, hipStream_t stream) {
  RowsArgs a;
  a.k = (const u32x4*)k;
  a.v = (const u32x4*)v;
  a.kc = (u32x4*)kc;
  a.vc = (u32x4*)vc;
  a.table = table;
  a.starts = starts;
  a.n_new = n_new;
  a.cu = cu;
  a.B = B;
  a.n = n;
  a.max_pages = max_pages;
  a.n_pages = n_pages;
  a.page = page;
  a.chunks = Hkv * (kHeadDim / 8);
  a.rows = cu != nullptr ? n : (long long)B * n;
  a.cap = table != nullptr ? (long long)max_pages * page : page;
  const long long grid = std::min<long long>((a.rows + kAppendWaves - 1) / kAppendWaves, kAppendGrid);
  hipLaunchKernelGGL(append_kernel, dim3((unsigned)grid), dim3(64 * kAppendWaves), 0, stream, a);
  return hipGetLastError();
}

}  // namespace jl
