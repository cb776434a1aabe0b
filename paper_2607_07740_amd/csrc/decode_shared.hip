// decode_shared.hip -- attention of few query rows over long paged bf16 caches: one new
// token of every sequence, where groups of sequences share a prefix whose keys and
// values are read once for all of them, and packed chunks of new tokens behind caches
// of different lengths.
//
// Jet-Long (arXiv 2607.07740): the query of a sequence of L tokens at position q takes a
// key k <= q in the base view where q - k <= w0, else in the remote view of G = max(1,
// ceil(L / w_pretrained)) (Sec. 3, Eqs. (1)-(3)).  The softmax over a row's keys is the
// merge (Eq. (7)) of those over any parts of them, so the keys that n sequences share
// make one attention of n g rows (g query heads of a kv head), matrix shaped, and the
// rest of each sequence one of g rows; n tokens of a chunk make one of n g.
//
// Plan.  A segment is such an attention: up to 256 rows over one range of keys, in
// visits of 32 keys: a visit in the remote view for each tile that holds a remote key and each G >= 2
// that occurs among its rows (one tile's visits follow each other, so that the later ones
// find it in the L2), then one in the base view for each tile that holds a local key.
// All segments' visits are one list, in which a visit counts what it costs; the
// workgroups of a kv head take equal ranges of it, whatever segments these span.  The plan
// follows from the lengths, so that a decoding step makes it once for all layers.
//
// Kernel: a workgroup (8 waves, one CU) streams the tiles of its range through a ring
// in LDS, K, V and the cos/sin rows of the keys' positions, four tiles in flight, and
// rotates tile i + 1 in place while tile i is multiplied.  Rows are the columns of 32 x 32 matrix
// instructions, 32 to a wave.  Up to 128 rows, four waves multiply and the other four copy and
// rotate, so that neither waits for the other (64 chats: 187 -> 134 us when this was
// split off); above, all eight do both.  A wave forms the scores of visit i beside the softmax and
// the value product of visit i - 1.  Each (workgroup, segment) leaves its rows' states (m, l, O)
// in fp32, and the merge kernel joins those of a row; a chunk's block that lies in one range is
// written at once.
//
// What bounds it: HBM where most tiles have one visit (64 chats behind 4 prompts, 536 MB: 118 us
// with 32/8 heads, 4.5 TB/s; the copies alone take 97 to 101), the multiplying waves where tiles
// have several (16 samples of 32K with G = 1 and 2, 222 MB: 89 us, 67 without them; 8 of 128K with
// G = 4 and 5, 544 MB: 220, 179 without), latency where there are few keys (2 sequences of 1.2K: 13).
// Tiles of 32 keys keep four of them in flight beside the two in use, and cut 1000 keys into enough visits
// for 32 workgroups of each of 8 kv heads.
#include <algorithm>
#include <climits>
#include <type_traits>

#include "decode_shared.h"
#include "jl_device.h"
#include "prefill_chunks.h"

namespace jl {

constexpr int kShThreads = 512, kShWaves = 8;
constexpr int kShRows = 32 * kShWaves;  // rows of a segment at most
constexpr int kShSmall = kShRows / 2;   // rows that four waves hold, while the others copy and rotate
constexpr int kShFew = kShRows / 4;     // rows that two waves hold: see state_halves
constexpr int kShTile = 32;             // keys of a tile
constexpr int kShImg = kShTile * kHeadDim * 2;      // K or V of a tile: 8 KB
constexpr int kShBuf = 2 * kShImg + kShTile * 256;  // and its 32 rows of (cos, sin), 16 bits each
constexpr int kShBufs = 6;
constexpr int kShAhead = kShBufs - 2;  // tiles requested before the first is used
constexpr int kShList = 256;           // visits whose addresses are held; refilled by halves
constexpr int kShSegs = 64;            // segments whose records are held
constexpr int kShCopies = 3;           // of a wave per tile

// What a visit costs in the list, and a segment beside its visits.
constexpr int kVisitCost = 4, kSegCost = 16;
__host__ __device__ inline int visit_cost(int rows) {
  return rows <= kShSmall ? kVisitCost : kVisitCost + 2;
}
constexpr int kMaxStep = kVisitCost + 2 + kSegCost;  // most between two visits that follow each other

struct Segment {
  int m0, rows, kend, seq;        // first member, rows, end of its keys, whose table row names its pages
  int k0, n_views, n_rem, loc0;   // first key; remote tiles and views of each; first tile with local keys
  int visits, view0, len, kind;   // view0: its views' place; len: its rows' length for G, 0: each its own
  uint32_t start_lo, start_hi;    // cost before it
  int w_first, n_w;               // workgroups that hold some of its visits
  int row0, q0, pad[2];           // state rows before it; a chunk's first row of q
};
// Whose rows a segment has: several sequences, one, or consecutive tokens of one
enum { kSegShared = 0, kSegOwn = 1, kSegChunk = 2 };
struct View {
  int G;
  uint32_t m, l;  // division by G
  int pad;
};
// A query row per kv head's query head: a sequence of a decode step, a token of a chunk
struct Member {
  int seq;       // row of q and o
  int len;       // its position + 1
  int pre, suf;  // its segments, -1: none
};
// States that a (workgroup, segment) leaves.  Up to 64 rows, two pairs of waves take the visits in
// turn where most tiles have two, their second from the caches (16 samples of 32K, G = 1 and 2: 99 ->
// 89 us, 8 of 128K 266 -> 218); where memory sets the pace the second states cost more (64 chats:
// 121 -> 128).
__host__ __device__ inline int state_halves(const Segment& s) {
  const int tiles = (s.kend - s.k0 + kShTile - 1) / kShTile;
  return s.rows <= kShFew && 2LL * s.visits > 3LL * tiles ? 2 : 1;
}
// Whether a chunk's segment is whole in one range and has one state: then its workgroup writes the
// rows, and the merge passes them over.  Where it has two, no run of it may write them, one in
// bf16 neither: the merge would put the states over them.
__host__ __device__ inline bool written_whole(const Segment& s) {
  return s.len > 0 && s.n_w == 1 && state_halves(s) == 1;
}

struct PlanView {
  int* header;
  int* wg_first;
  Member* members;
  View* views;
  Segment* segs;
};
// members, views, segments of a plan
struct PlanSizes {
  size_t members, views, segs;
};
__host__ __device__ inline PlanSizes decode_sizes(int B, int n_groups, int g) {
  PlanSizes s;
  s.members = (size_t)B;
  s.views = 2 * (size_t)B;
  s.segs = (size_t)n_groups + (size_t)B / (kShRows / g) + 1 + B;
  return s;
}
__host__ __device__ inline PlanSizes chunk_sizes(int B, int T, int g) {
  PlanSizes s;
  s.members = (size_t)T;
  s.segs = (size_t)B + (size_t)T / (kShRows / g) + 1;
  s.views = s.segs;
  return s;
}
constexpr size_t kPlanHead = 128 + 4 * kShMaxWg;
__host__ __device__ inline PlanView plan_view(void* p, const PlanSizes& z) {
  PlanView v;
  char* c = (char*)p;
  v.header = (int*)c;
  v.wg_first = (int*)(c + 128);
  v.members = (Member*)(c + kPlanHead);
  v.views = (View*)(v.members + z.members);
  v.segs = (Segment*)(v.views + z.views);
  return v;
}
static size_t plan_bytes(const PlanSizes& z) {
  return kPlanHead + z.members * sizeof(Member) + z.views * sizeof(View) + z.segs * sizeof(Segment);
}
// Parts of the chunks whose blocks the prefill kernel takes, at most: kPartWaves times the
// workgroups of a kv head and each block rounded up, both twice for the empty ones (a block of a
// whole prompt has half of the longest's visits in the mean).  Of a block that is cut, at
// most 4/3 of its share have states.
constexpr int kPartWaves = 3;
static size_t most_parts(int B, int T, int g, int n_wg) {
  return 2 * (chunk_sizes(B, T, g).segs + (size_t)kPartWaves * n_wg);
}
static size_t most_slots(int n_wg) { return (size_t)kPartWaves * n_wg * 4 / 3 + 2; }
size_t prefill_chunk_state_bytes();
int prefill_chunk_max_pages();
hipError_t launch_prefill_chunks(bool bifocal, const uint16_t* q, const uint16_t* k,
                                 const uint16_t* v, uint16_t* o, float* lse, const float2* table,
                                 const uint32_t* table16, const uint32_t* half, const int32_t* block_table,
                                 int max_pages, int page_shift, int n_pages, int T, int Hq, int Hkv,
                                 int w0, float slack, const ChunkPart* parts, const int* n_parts,
                                 int max_parts, float* states, hipStream_t stream);
size_t shared_plan_bytes(int B, int n_groups, int g) { return plan_bytes(decode_sizes(B, n_groups, g)); }

enum { kHdSegs = 0, kHdWg, kHdTotLo, kHdTotHi, kHdRows, kHdB, kHdG, kHdPage, kHdMaxPages, kHdHkv,
       kHdGroups, kHdBifocal, kHdWPre, kHdW0, kHdParts, kHdMembers };

// State rows of one kv head: every segment's, for each of its halves, and again where a
// workgroup's range ends inside it.
static size_t state_rows(size_t rows, int most, int n_wg) {
  return 2 * rows + (size_t)(n_wg - 1) * std::min<size_t>(kShRows, 2 * (size_t)most);
}
static int head_workgroups(int n_cu, int Hkv) { return std::max(1, std::min(n_cu, kShMaxWg) / Hkv); }
constexpr int kShStateFloats = kHeadDim + 4;  // O, (m, l), and 8 bytes that keep 16-byte alignment
size_t decode_shared_workspace_bytes(int B, int Hq, int Hkv) {
  const int g = Hq / Hkv;
  return (size_t)Hkv * state_rows(2 * (size_t)B * g, B * g, head_workgroups(kShMaxWg, Hkv)) *
         kShStateFloats * sizeof(float);
}
static size_t round256(size_t x) { return (x + 255) / 256 * 256; }

// Whether the blocks of longer chunks go to the prefill kernel, which takes 64 keys of 256 rows in
// the time of 32 here (turns of 512, 600, 1 and 700 rows behind 15000, 34000, 9000 and 0 keys, 32/8
// heads: 754 -> 560 us): where the rows beyond a token per sequence make a few of its blocks, and with what it
// asks of the cache.  A sequence's go there if they are more than 128.
static bool chunk_blocks(int B, int T, int Hkv, int g, int max_pages, int page) {
  // a launch of its parts, 512 threads for each kv head, drops those past 32 bits
  const size_t parts = most_parts(B, T, g, head_workgroups(kShMaxWg, Hkv));
  return kChunkBlockRows % g == 0 && page >= kChunkTile && max_pages <= prefill_chunk_max_pages() &&
         ((long long)T - B) * g >= 4 * kChunkBlockRows && parts * Hkv < ((size_t)1 << 32) / 512;
}

// Scratch of a chunk call: plan, parts, the states of either kernel
struct ChunkScratch {
  size_t parts, states, part_states, end;
};
static ChunkScratch chunk_scratch(int B, int T, int Hq, int Hkv, int max_pages, int page) {
  const int g = Hq / Hkv, n_wg = head_workgroups(kShMaxWg, Hkv);
  const bool blocks = chunk_blocks(B, T, Hkv, g, max_pages, page);
  ChunkScratch c;
  c.parts = round256(plan_bytes(chunk_sizes(B, T, g)));
  c.states = round256(c.parts + (blocks ? most_parts(B, T, g, n_wg) * sizeof(ChunkPart) : 0));
  c.part_states = round256(c.states + (size_t)Hkv * state_rows((size_t)T * g, kShRows, n_wg) *
                                          kShStateFloats * sizeof(float));
  c.end = c.part_states + (blocks ? most_slots(n_wg) * Hkv * prefill_chunk_state_bytes() : 0);
  return c;
}
size_t chunk_scratch_bytes(int B, int T, int Hq, int Hkv, int max_pages, int page) {
  return chunk_scratch(B, T, Hq, Hkv, max_pages, page).end;
}

// ------------------------------------------------------------------- plan
struct SharedPlanArgs {
  const int32_t* kv_lens;
  const int32_t* members;  // nullptr: 0 .. B - 1
  const int32_t* group_starts;
  const int32_t* shared;
  const int32_t* cu;       // chunks: T packed rows
  void* plan;
  int B, n_groups, T, g, Hkv, max_pages, page, n_wg, bifocal, w_pre, w0;
  ChunkPart* parts;        // chunks: of those whose blocks the prefill kernel takes; nullptr: none
  int most_parts;
};

constexpr int kPlThreads = 1024, kPlWaves = kPlThreads / 64;  // at most; few sequences take 256

// Inclusive sums over the workgroup's threads, in thread order; everyone gets the total
template <typename T>
__device__ inline T plan_scan(T v, T* s, T* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const T incl = wave_scan(v);
  __syncthreads();
  if (lane == 63) s[wave] = incl;
  __syncthreads();
  T before = 0, all = 0;
#pragma unroll
  for (int i = 0; i < kPlWaves; i += 4) {
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

// max(1, ceil(len / w_pre)) for len <= 2^23, without a 64-bit division
__device__ inline int rows_group(int len, int bifocal, int w_pre) {
  return !bifocal || len <= w_pre ? 1 : (int)(((uint32_t)len + (uint32_t)w_pre - 1) / (uint32_t)w_pre);
}
__device__ inline int plan_group(const SharedPlanArgs& a, int len) {
  return rows_group(len, a.bifocal, a.w_pre);
}
// The first key that a query at position q takes in the base view (0 where it takes all so)
__device__ inline int first_local(int G, int q, int w0) { return G > 1 ? max(0, q - w0) : 0; }

// make_fastdiv for 2 <= G <= 2^23: its quotient 2^32 (2^l - G) / G, whose numerator a double
// holds, by a division of doubles, one too large at most
__device__ inline View view_of(int G) {
  const uint32_t l = 32 - __builtin_clz((uint32_t)G - 1);
  const uint64_t num = (((uint64_t)1 << l) - (uint32_t)G) << 32;
  uint32_t m = (uint32_t)((double)num / (double)G);
  if ((uint64_t)m * (uint32_t)G > num) --m;
  return View{G, m + 1, l, 0};
}

// Visits of keys [k0, kend) for rows whose first local keys lie between `low` and, among
// those of some G >= 2, `far`, in n_views remote views
__device__ inline void set_visits(Segment& s, int low, int far, int n_views) {
  const int tiles = (s.kend - s.k0 + kShTile - 1) / kShTile;
  s.n_views = max(n_views, 1);
  s.n_rem = n_views > 0 && far > s.k0 ? min(tiles, (far - s.k0 + kShTile - 1) / kShTile) : 0;
  s.loc0 = min(tiles, max(low - s.k0, 0) / kShTile);
  s.visits = s.n_rem * s.n_views + tiles - s.loc0;
}

// Equal ranges of the list for n_wg workgroups: the first r of them one longer
struct Ranges {
  unsigned long long q, r;
  int n_wg;
  __device__ inline unsigned long long begin(int w) const { return q * w + min((unsigned long long)w, r); }
  __device__ inline int owner(unsigned long long x) const {
    const unsigned long long head = r * (q + 1);
    if (((q + 1) * n_wg) >> 32 == 0)
      return (int)(x < head ? (uint32_t)x / (uint32_t)(q + 1)
                            : (uint32_t)r + (uint32_t)(x - head) / (uint32_t)q);
    return (int)(x < head ? x / (q + 1) : r + (x - head) / q);
  }
};
__device__ inline Ranges ranges_of(unsigned long long total, int n_wg) {
  Ranges r;
  r.n_wg = n_wg;
  if (total >> 32 == 0) {
    r.q = (uint32_t)total / (uint32_t)n_wg;
  } else {
    r.q = total / (unsigned)n_wg;
  }
  r.r = total - r.q * n_wg;
  return r;
}

// The end of both plans: costs before each segment, the workgroups' ranges, and the places of
// the states.  s_visits, s_rows, s_states: visits, rows and rows of states of n_segs segments; a
// thread takes a run of them.
__device__ inline void plan_ranges(const SharedPlanArgs& a, const PlanView& v, int n_segs,
                                   const int* s_visits, const short* s_rows, const short* s_states,
                                   unsigned long long* s_scan) {
  const int tid = threadIdx.x;
  const int per = (n_segs + (int)blockDim.x - 1) >> (31 - __builtin_clz(blockDim.x));
  const int i0 = min(tid * per, n_segs), i1 = min(i0 + per, n_segs);
  auto cost = [&](int i) {
    const int n = s_visits[i];
    return n > 0 ? kSegCost + (unsigned long long)n * visit_cost(s_rows[i]) : 0ull;
  };
  unsigned long long mine = 0, total;
  for (int i = i0; i < i1; ++i) mine += cost(i);
  unsigned long long st = plan_scan(mine, s_scan, &total) - mine;
  // ranges that hold a visit wherever they lie inside a segment
  const int n_wg = total == 0 ? 0 : (int)max(1ull, min((unsigned long long)a.n_wg, total / kMaxStep));
  Ranges rg = {};
  if (n_wg > 0) rg = ranges_of(total, n_wg);
  unsigned long long rows = 0;
  const unsigned long long st0 = st;
  __shared__ unsigned long long s_first[kPlThreads];
  const bool one_each = per == 1;
  for (int i = i0; i < i1; ++i) {
    const unsigned long long c = cost(i);
    if (c == 0) continue;
    const int w0 = rg.owner(st + kSegCost), w1 = rg.owner(st + c - visit_cost(s_rows[i]));
    rows += (unsigned long long)(w1 - w0 + 1) * s_states[i];
    if (!one_each) {
      int w = rg.owner(st);  // workgroups whose ranges begin inside this segment
      if (rg.begin(w) < st) ++w;
      for (; w < n_wg && rg.begin(w) < st + c; ++w) v.wg_first[w] = i;
    }
    st += c;
  }
  if (one_each) {  // a thread for each workgroup: the last segment that begins at or before its range
    if (tid < n_segs) s_first[tid] = st0;
    __syncthreads();
    for (int w = tid; w < n_wg; w += (int)blockDim.x) {
      const unsigned long long x = rg.begin(w);
      int lo = 0, hi = n_segs - 1;
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (s_first[mid] <= x) lo = mid; else hi = mid - 1;
      }
      v.wg_first[w] = lo;
    }
  }
  unsigned long long all_rows;
  unsigned long long row = plan_scan(rows, s_scan, &all_rows) - rows;
  st = st0;
  for (int i = i0; i < i1; ++i) {
    const unsigned long long c = cost(i);
    Segment& s = v.segs[i];
    s.start_lo = (uint32_t)st;
    s.start_hi = (uint32_t)(st >> 32);
    if (c == 0) {
      s.w_first = s.n_w = 0;
      s.row0 = 0;
      continue;
    }
    const int w0 = rg.owner(st + kSegCost), w1 = rg.owner(st + c - visit_cost(s_rows[i]));
    s.w_first = w0;
    s.n_w = w1 - w0 + 1;
    s.row0 = (int)row;
    row += (unsigned long long)(w1 - w0 + 1) * s_states[i];
    st += c;
  }
  if (tid == 0) {
    v.header[kHdSegs] = n_segs;
    v.header[kHdWg] = n_wg;
    v.header[kHdTotLo] = (int)(uint32_t)total;
    v.header[kHdTotHi] = (int)(uint32_t)(total >> 32);
    v.header[kHdRows] = (int)all_rows;
    v.header[kHdB] = a.B;
    v.header[kHdG] = a.g;
    v.header[kHdPage] = a.page;
    v.header[kHdMaxPages] = a.max_pages;
    v.header[kHdHkv] = a.Hkv;
    v.header[kHdGroups] = a.n_groups;
    v.header[kHdBifocal] = a.bifocal;
    v.header[kHdWPre] = a.w_pre;
    v.header[kHdW0] = a.w0;
    if (a.cu == nullptr) v.header[kHdMembers] = a.B;
  }
}

// A decode step's plan, by one workgroup: bound by the latency of its dependent reads and scans (7.0 us
// for 2 sequences, 8.0 for 16 with views of two G, 8.6 for 64; 8.5, 11.1 and 11.0 with scans by
// exchanges through LDS and one thread naming a segment's workgroups; 256 threads, not 1024, up to
// 128 sequences: two microseconds).  One plan serves every layer of a step.
__global__ __launch_bounds__(kPlThreads) void shared_plan_kernel(SharedPlanArgs a) {
  extern __shared__ int s_mem[];
  __shared__ unsigned long long s_scan[kPlWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, nt = blockDim.x;
  const PlanSizes z = decode_sizes(a.B, a.n_groups, a.g);
  const PlanView v = plan_view(a.plan, z);
  int* const s_len = s_mem;                    // [B] by member, -1: no such sequence
  int* const s_seq = s_len + a.B;              // [B]
  int* const s_start = s_seq + a.B;            // [n_groups + 1]
  int* const s_pre = s_start + a.n_groups + 1; // [n_groups]: shared keys
  int* const s_blk = s_pre + a.n_groups;       // [n_groups + 1]: prefix blocks before the group
  int* const s_visits = s_blk + a.n_groups + 1;
  short* const s_rows = (short*)(s_visits + z.segs);
  short* const s_states = s_rows + z.segs;
  const int cap = a.max_pages * a.page;
  const int per_block = kShRows / a.g;

  bool bad = false;
  for (int i = tid; i <= a.n_groups; i += nt) {
    const int x = min(max(a.group_starts[i], 0), a.B);
    s_start[i] = x;
    if (i > 0) bad |= min(max(a.group_starts[i - 1], 0), a.B) > x;
  }
  for (int i = tid; i < a.n_groups; i += nt) {
    s_pre[i] = INT_MAX;
    s_blk[i] = a.shared[i];  // until the blocks are counted
  }
  for (int i = tid; i < a.B; i += nt) {
    const int seq = a.members != nullptr ? a.members[i] : i;
    const bool ok = (unsigned)seq < (unsigned)a.B;
    s_seq[i] = ok ? seq : -1;
    s_len[i] = ok ? min(max(a.kv_lens[seq], 0), cap) : -1;
  }
  if (__syncthreads_or(bad)) {  // a start below an earlier one counts as that
    if (tid == 0)
      for (int i = 1; i <= a.n_groups; ++i) s_start[i] = max(s_start[i], s_start[i - 1]);
    __syncthreads();
  }
  // a member's group: the first whose end lies behind it
  auto group_of = [&](int m) {
    int lo = 0, hi = a.n_groups;
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (s_start[mid + 1] > m) hi = mid; else lo = mid + 1;
    }
    return lo < a.n_groups && s_start[lo] <= m ? lo : -1;
  };
  for (int i = tid; i < a.B; i += nt) {
    const int gi = group_of(i);
    if (gi >= 0 && s_len[i] > 0) atomicMin(&s_pre[gi], s_len[i]);
  }
  __syncthreads();
  // the groups' shared keys and their blocks of up to 256 rows
  int n_blocks = 0;
  for (int c0 = 0; c0 < a.n_groups; c0 += nt) {
    const int i = c0 + tid;
    unsigned long long x = 0, tot;
    if (i < a.n_groups) {
      const int n = s_start[i + 1] - s_start[i], low = s_pre[i];
      const int P = n > 1 && low != INT_MAX ? min(max(s_blk[i], 0), low) & -a.page : 0;
      s_pre[i] = P;
      x = P > 0 ? (n + per_block - 1) / per_block : 0;
    }
    const unsigned long long incl = plan_scan(x, s_scan, &tot);
    if (i < a.n_groups) s_blk[i] = n_blocks + (int)(incl - x);
    n_blocks += (int)tot;
  }
  if (tid == 0) s_blk[a.n_groups] = n_blocks;
  __syncthreads();
  // prefix blocks, a wave each, lane -> every 64th of its sequences
  for (int blk = wave; blk < n_blocks; blk += nt >> 6) {
    int gi = 0, hi = a.n_groups - 1;  // the last group that begins at or before it
    while (gi < hi) {
      const int mid = (gi + hi + 1) >> 1;
      if (s_blk[mid] <= blk) gi = mid; else hi = mid - 1;
    }
    const int m0 = s_start[gi] + (blk - s_blk[gi]) * per_block;
    const int n = min(per_block, s_start[gi + 1] - m0);
    int low = INT_MAX, far = 0, from = INT_MAX, G = 1, n_views = 0;
    for (;;) {  // the values of G above 1, ascending
      int next = INT_MAX;
      for (int i = lane; i < n; i += 64) {
        const int len = s_len[m0 + i];
        if (len <= 0) continue;
        const int Gi = plan_group(a, len), lim = first_local(Gi, len - 1, a.w0);
        if (Gi > G) next = min(next, Gi);
        if (G == 1) {
          low = min(low, lim);
          far = max(far, lim);
          from = min(from, i);
        }
      }
      G = wave_min(next);
      if (G == INT_MAX) break;
      if (lane == 0) v.views[m0 + n_views] = view_of(G);
      ++n_views;
    }
    low = wave_min(low);
    far = wave_max(far);
    from = wave_min(from);
    if (lane == 0) {
      Segment s = {};
      s.m0 = m0;
      s.rows = n * a.g;
      s.kend = s_pre[gi];
      s.seq = from == INT_MAX ? 0 : s_seq[m0 + from];
      s.view0 = m0;
      if (from != INT_MAX) set_visits(s, low, far, n_views);
      v.segs[blk] = s;
      s_visits[blk] = s.visits;
      s_rows[blk] = (short)s.rows;
      s_states[blk] = (short)(s.rows * state_halves(s));
    }
  }
  // the members' own keys
  for (int i = tid; i < a.B; i += nt) {
    const int gi = group_of(i), len = s_len[i], seg = n_blocks + i;
    Segment s = {};
    Member m = {gi >= 0 && len >= 0 ? s_seq[i] : -1, max(len, 0), -1, -1};
    if (gi >= 0 && len > 0) {
      const int P = s_pre[gi], G = plan_group(a, len), lim = first_local(G, len - 1, a.w0);
      s.m0 = i;
      s.kind = kSegOwn;
      s.rows = a.g;
      s.k0 = P;
      s.kend = len;
      s.seq = m.seq;
      s.view0 = a.B + i;
      set_visits(s, lim, lim, G > 1 ? 1 : 0);
      if (G > 1) v.views[a.B + i] = view_of(G);
      if (P > 0) m.pre = s_blk[gi] + (i - s_start[gi]) / per_block;
      if (s.visits > 0) m.suf = seg;
    }
    v.members[i] = m;
    v.segs[seg] = s;
    s_visits[seg] = s.visits;
    s_rows[seg] = (short)s.rows;
    s_states[seg] = (short)(s.rows * state_halves(s));
  }
  __syncthreads();
  plan_ranges(a, v, n_blocks + a.B, s_visits, s_rows, s_states, s_scan);
}

// The plan of packed chunks: sequence b's rows are cu[b] .. cu[b + 1] - 1 of the packed ones,
// the last kv_lens[b] - n .. kv_lens[b] - 1 of its positions (rows that would lie before
// position 0 are left out).  Blocks of up to 256 / g tokens, the last of a sequence shorter,
// are segments, or parts for the prefill kernel; the members are the tokens of segments.
__global__ __launch_bounds__(kPlThreads) void chunk_plan_kernel(SharedPlanArgs a) {
  extern __shared__ int s_mem[];
  __shared__ unsigned long long s_scan[kPlWaves];
  const int tid = threadIdx.x, nt = blockDim.x;
  const int log_nt = 31 - __builtin_clz(nt);
  const PlanSizes z = chunk_sizes(a.B, a.T, a.g);
  const PlanView v = plan_view(a.plan, z);
  int* const s_start = s_mem;               // [B + 1]
  int* const s_len = s_start + a.B + 1;     // [B]
  int* const s_blk = s_len + a.B;           // [B + 1]: segments before the sequence
  int* const s_big = s_blk + a.B + 1;       // [B + 1]: the prefill kernel's blocks before it
  int* const s_tok = s_big + a.B + 1;       // [B + 1]: members before it; then parts
  int* const s_visits = s_tok + a.B + 1;
  int* const s_slot = s_visits + z.segs;    // states before a block of the prefill kernel
  short* const s_rows = (short*)(s_slot + z.segs);
  short* const s_states = s_rows + z.segs;
  const int cap = a.max_pages * a.page;
  const int per_block = kShRows / a.g;
  bool bad = false;
  for (int i = tid; i <= a.B; i += nt) {
    const int x = min(max(a.cu[i], 0), a.T);
    s_start[i] = x;
    if (i > 0) bad |= min(max(a.cu[i - 1], 0), a.T) > x;
    if (i < a.B) s_len[i] = min(max(a.kv_lens[i], 0), cap);
  }
  if (__syncthreads_or(bad)) {  // a start below an earlier one counts as that
    if (tid == 0)
      for (int i = 1; i <= a.B; ++i) s_start[i] = max(s_start[i], s_start[i - 1]);
    __syncthreads();
  }
  auto is_big = [&](int b) {
    const int n = s_start[b + 1] - s_start[b];
    return a.parts != nullptr && n * a.g > kShSmall && s_len[b] >= n;
  };
  // the last b whose entry of `list` is at or below x
  auto find = [&](const int* list, int x) {
    int b = 0, hi = a.B - 1;
    while (b < hi) {
      const int mid = (b + hi + 1) >> 1;
      if (list[mid] <= x) b = mid; else hi = mid - 1;
    }
    return b;
  };
  int n_segs = 0, n_big = 0, n_tok = 0;
  for (int c0 = 0; c0 < a.B; c0 += nt) {
    const int i = c0 + tid;
    unsigned long long x = 0, tot;  // members, segments, blocks: 24, 20 and 20 bits
    if (i < a.B) {
      const int n = s_start[i + 1] - s_start[i];
      const unsigned long long blocks = (unsigned)(n + per_block - 1) / (unsigned)per_block;
      x = is_big(i) ? blocks << 44 : blocks << 24 | (unsigned)n;
    }
    const unsigned long long incl = plan_scan(x, s_scan, &tot);
    const unsigned long long before = incl - x;
    if (i < a.B) {
      s_tok[i] = n_tok + (int)(before & 0xffffff);
      s_blk[i] = n_segs + (int)(before >> 24 & 0xfffff);
      s_big[i] = n_big + (int)(before >> 44);
    }
    n_tok += (int)(tot & 0xffffff);
    n_segs += (int)(tot >> 24 & 0xfffff);
    n_big += (int)(tot >> 44);
  }
  if (tid == 0) {
    s_tok[a.B] = n_tok;
    s_blk[a.B] = n_segs;
    s_big[a.B] = n_big;
  }
  __syncthreads();
  for (int seg = tid; seg < n_segs; seg += nt) {
    const int b = find(s_blk, seg);
    const int n = s_start[b + 1] - s_start[b], t0 = (seg - s_blk[b]) * per_block;
    const int cnt = min(per_block, n - t0), len = s_len[b];
    const int p0 = len - n + t0, p1 = p0 + cnt - 1;  // positions of its first and last token
    const int G = plan_group(a, len);
    Segment s = {};
    s.m0 = s_tok[b] + t0;
    s.rows = cnt * a.g;
    s.kend = max(p1 + 1, 0);
    s.seq = b;
    s.view0 = seg;
    s.len = max(len, 1);
    s.kind = kSegChunk;
    s.q0 = s_start[b] + t0;
    set_visits(s, first_local(G, p0, a.w0), first_local(G, p1, a.w0), G > 1 ? 1 : 0);
    if (G > 1) v.views[seg] = view_of(G);
    v.segs[seg] = s;
    s_visits[seg] = s.visits;
    s_rows[seg] = (short)s.rows;
    s_states[seg] = (short)(s.rows * state_halves(s));
  }
  for (int t = tid; t < n_tok; t += nt) {
    const int b = find(s_tok, t), i = t - s_tok[b];
    const int pos = s_len[b] - (s_start[b + 1] - s_start[b]) + i;
    v.members[t] = pos >= 0 ? Member{s_start[b] + i, pos + 1, s_blk[b] + i / per_block, -1}
                            : Member{-1, 0, -1, -1};
  }
  __syncthreads();
  // The prefill kernel's blocks, cut into parts of about the same visits: for every workgroup of a
  // kv head as many as there are blocks for it, rounded up, at most kPartWaves (29 blocks for 32
  // workgroups, the turns above: one 550 us, three 590; 88 blocks: one 1440, three 1170).  A sequence's parts are listed part after part, so that the
  // blocks that run beside each other read the same keys; blocks of fewer parts leave empty ones.
  int n_parts = 0;
  if (n_big > 0) {
    auto visits_of = [&](int b, int block) {
      const int len = s_len[b], n = s_start[b + 1] - s_start[b];
      const int q0 = len - n + block * per_block, q1 = min(q0 + per_block, len) - 1;
      const VisitRanges vr = visit_ranges(q0, q1, plan_group(a, len) > 1 ? a.w0 : INT_MAX, kChunkTile);
      return vr.n_r + vr.n_kt - vr.kt_l;
    };
    const int per = (n_big + nt - 1) >> log_nt;
    const int j0 = min(tid * per, n_big), j1 = min(j0 + per, n_big);
    unsigned long long mine = 0, all, tot;
    for (int j = j0; j < j1; ++j) {
      const int b = find(s_big, j);
      mine += (unsigned long long)visits_of(b, j - s_big[b]);
    }
    plan_scan(mine, s_scan, &all);
    const unsigned shares =
        (unsigned)min(kPartWaves, (n_big + a.n_wg - 1) / a.n_wg) * (unsigned)a.n_wg;
    const unsigned long long even = all >> 32 == 0 ? ((unsigned)all + shares - 1) / shares : all / shares + 1;
    int target = (int)min(max(even, (unsigned long long)kChunkMinPart), 0x1fffffffull);
    auto parts_of = [&](int visits) { return max(1, min(16, (visits + target / 2) / target)); };
    // entries of each sequence: its blocks times the parts of its last block, the longest
    for (;; target *= 2) {  // longer parts where the list could not hold them
      n_parts = 0;
      for (int c0 = 0; c0 < a.B; c0 += nt) {
        const int b = c0 + tid;
        unsigned long long x = 0;
        if (b < a.B && s_big[b + 1] > s_big[b]) {
          const int blocks = s_big[b + 1] - s_big[b];
          x = (unsigned long long)(blocks * parts_of(visits_of(b, blocks - 1)));
        }
        const unsigned long long incl = plan_scan(x, s_scan, &tot);
        if (b < a.B) s_tok[b] = n_parts + (int)(incl - x);
        n_parts += (int)tot;
      }
      if (n_parts <= a.most_parts || target > 0x1fffffff) break;
    }
    mine = 0;  // parts of blocks that are cut
    for (int j = j0; j < j1; ++j) {
      const int b = find(s_big, j), c = parts_of(visits_of(b, j - s_big[b]));
      s_slot[j] = (int)mine;
      mine += c > 1 ? c : 0;
    }
    const int slot0 = (int)(plan_scan(mine, s_scan, &tot) - mine);
    for (int j = j0; j < j1; ++j) s_slot[j] += slot0;
    __syncthreads();
    for (int e = tid; e < n_parts; e += nt) {
      const int b = find(s_tok, e), blocks = s_big[b + 1] - s_big[b], r = e - s_tok[b];
      ChunkPart p = {};
      p.part = r / blocks;
      p.block = r - p.part * blocks;
      p.seq = b;
      p.row0 = s_start[b];
      p.n = s_start[b + 1] - s_start[b];
      p.L = s_len[b];
      p.G = plan_group(a, p.L);
      p.parts = parts_of(visits_of(b, p.block));
      p.slot = s_slot[s_big[b] + p.block];
      if (p.part >= p.parts) p.parts = 0;
      a.parts[e] = p;
    }
  }
  if (tid == 0) {
    v.header[kHdParts] = n_parts;
    v.header[kHdMembers] = n_tok;
  }
  plan_ranges(a, v, n_segs, s_visits, s_rows, s_states, s_scan);
}

// --------------------------------------------------------------- attention
struct SharedArgs {
  const uint16_t* q;
  const uint16_t* k;
  const uint16_t* v;
  const int32_t* table;
  uint16_t* o;
  float* lse;  // [Hq][T] of a chunk, or nullptr
  const float2* rope;
  const uint32_t* half;    // the same in fp16, one word a pair
  const uint32_t* rope16;  // and in bf16
  void* plan;
  float* states;
  int B, n_groups, T, Hq, Hkv, g, max_pages, n_pages, page, page_shift, n_wg;
  int chunk, bifocal, w_pre, w0;
  float q_scale;
  int g_inv;  // floor(2^16 / g) + 1
};

__device__ inline PlanView plan_of(const SharedArgs& a) {
  return plan_view(a.plan, a.chunk ? chunk_sizes(a.B, a.T, a.g) : decode_sizes(a.B, a.n_groups, a.g));
}
// Whether the plan is one for this call: else nothing is computed.
__device__ inline bool plan_fits(const SharedArgs& a, const int* h) {
  return h[kHdB] == a.B && h[kHdG] == a.g && h[kHdPage] == a.page && h[kHdMaxPages] == a.max_pages &&
         h[kHdHkv] == a.Hkv && h[kHdGroups] == a.n_groups && h[kHdBifocal] == a.bifocal &&
         h[kHdWPre] == a.w_pre && h[kHdW0] == a.w0 && h[kHdWg] <= a.n_wg;
}

// LDS layouts: K key r at r * 256, its 16-byte chunk c in slot c ^ sh_kswz(r) (16 keys read
// at one chunk, and a key's halves, hit distinct banks); V key r in slot c ^ sh_vswz(r) (so do
// the transposing reads of 8 keys x 32 B and of 4 keys x 64 B); cos/sin row of key r at r * 256.
__device__ inline int sh_kswz(int r) { return ((r & 15) >> 1) | ((r & 1) << 3); }
__device__ inline int sh_vswz(int r) { return 4 * (r & 3) | 2 * ((r >> 2) & 1); }
__device__ inline int sh_koff(int r, int c) { return r * 256 + 16 * (c ^ sh_kswz(r)); }
__device__ inline int sh_voff(int r, int c) { return r * 256 + 16 * (c ^ sh_vswz(r)); }

// A visit of the list
struct Tile {
  int row0, row1;  // pool rows of its first and its 17th key
  int k0;
  int flags;       // bits 0..4: last valid key of the tile; kTfLast; the held segment from bit 9 on
  int f0, km;      // remote view: f(k0) and k0 - G f(k0)
  uint32_t m, lG;  // its view: l and, from bit 6 on, G (0: the base view)
};
constexpr int kTfLast = 32, kTfSeg = 9;

typedef __bf16 sh_bf16x2 __attribute__((ext_vector_type(2)));
typedef unsigned sh_u32x2 __attribute__((ext_vector_type(2)));

// Keys and queries are multiplied in fp16, whose 11 bits hold the rotated values eight times as
// well as bf16 would: at 16 samples of 32K the output's distance from 64 bits falls from 0.0047
// of its size to 0.0024 (0.0017 is the output's own rounding).  A range that meets a row whose
// largest channel fp16 holds less well, outside [2^-8, 2^15), is done again in bf16.
constexpr float kShLow = 1.f / 256.f, kShHigh = 32768.f;
__device__ inline bool sh_outside(float amax) {  // of a whole row; nor does bf16 help inf and NaN
  return (amax > 0.f && amax < kShLow) || (amax >= kShHigh && amax < INFINITY);
}

__device__ inline float sh_max32(float x) {  // over lanes l and l ^ 32
  const sh_u32x2 r =
      __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
// Channels d .. d + 7 and d + 64 .. d + 71 of a query row, rotated to position pos and scaled, as
// operands; amax: the largest of them
template <typename Op>
__device__ inline void sh_rotate_q(const uint16_t* qrow, int d, const float2* table, int pos,
                                   float scale, Op& olo, Op& ohi, float& amax) {
  float lo[8], hi[8], ylo[8], yhi[8];
  unpack8(load16(qrow + d), lo);
  unpack8(load16(qrow + d + kHalf), hi);
  const float4* c4 = (const float4*)(table + (size_t)pos * kHalf + d);
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    const float4 w = c4[t];
    const int j = 2 * t;
    ylo[j] = (lo[j] * w.x - hi[j] * w.y) * scale;
    yhi[j] = (hi[j] * w.x + lo[j] * w.y) * scale;
    ylo[j + 1] = (lo[j + 1] * w.z - hi[j + 1] * w.w) * scale;
    yhi[j + 1] = (hi[j + 1] * w.z + lo[j + 1] * w.w) * scale;
  }
  if constexpr (std::is_same_v<Op, bf16x8>) {
    olo = pack8(ylo);
    ohi = pack8(yhi);
  } else {
#pragma unroll
    for (int t = 0; t < 8; ++t) {
      olo[t] = (_Float16)ylo[t];
      ohi[t] = (_Float16)yhi[t];
      amax = fmaxf(amax, fmaxf(fabsf(ylo[t]), fabsf(yhi[t])));
    }
  }
}

// A tile's weights of a row may add up to this before the row's reference moves: far inside
// fp32 and bf16.
constexpr float kShMaxSum = 65536.f;

__global__ __launch_bounds__(kShThreads, 2) void shared_rows_kernel(SharedArgs a) {
  __shared__ __attribute__((aligned(1024))) unsigned char smem[kShBufs * kShBuf];
  __shared__ __attribute__((aligned(16))) Tile s_tiles[kShList];
  __shared__ __attribute__((aligned(16))) Segment s_segs[kShSegs];
  __shared__ int s_from[kShSegs], s_before[kShSegs];  // first visit here, visits of earlier ones
  __shared__ int s_again;                             // rows that fp16 does not hold were met
  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // The kv heads of one range run on one XCD (blocks go to the 8 of them in turn): they read
  // neighbouring pieces of the same pool rows, and the same cos/sin rows.
  int h, w;
  if ((a.n_wg & 7) == 0) {
    const int t = blockIdx.x >> 3, u = t / a.Hkv;
    h = t - u * a.Hkv;
    w = 8 * u + (blockIdx.x & 7);
  } else {
    w = blockIdx.x / a.Hkv;
    h = blockIdx.x - w * a.Hkv;
  }
  const PlanView pv = plan_of(a);
  if (!plan_fits(a, pv.header) || w >= pv.header[kHdWg]) return;
  auto uni = [](int x) { return __builtin_amdgcn_readfirstlane(x); };
  const int n_segs = uni(pv.header[kHdSegs]), all_rows = uni(pv.header[kHdRows]);
  unsigned long long x0, x1;
  {
    const unsigned long long total =
        (uint32_t)pv.header[kHdTotLo] | (unsigned long long)(uint32_t)pv.header[kHdTotHi] << 32;
    const Ranges rg = ranges_of(total, pv.header[kHdWg]);
    auto uni64 = [&](unsigned long long x) {
      return (uint32_t)uni((int)(uint32_t)x) | (unsigned long long)(uint32_t)uni((int)(x >> 32)) << 32;
    };
    x0 = uni64(rg.begin(w));
    x1 = uni64(rg.begin(w + 1));
  }
  const uint32_t smem_base = lds_addr(smem);
  const uint32_t kv_row_bytes = (uint32_t)a.Hkv * (kHeadDim * 2);
  const unsigned char* kbase = (const unsigned char*)(a.k + (size_t)h * kHeadDim);
  const unsigned char* vbase = (const unsigned char*)(a.v + (size_t)h * kHeadDim);

  // ---- what a wave does of a tile's copies and rotation: with ALL keys 4 wave .. + 3, else
  // the last four waves take 8 each
  // Per lane and copy of 4 keys: byte offsets of its piece of K, V and the cos/sin rows inside a
  // whole tile
  struct Piece {
    uint32_t k, v, cs;
  };
  auto piece_of = [&](int ln, int key0) {
    const int slot = ln & 15, key = key0 + (ln >> 4);
    const uint32_t ro = (uint32_t)(key & 15) * kv_row_bytes;
    return Piece{ro + 16 * (slot ^ sh_kswz(key)), ro + 16 * (slot ^ sh_vswz(key)),
                 (uint32_t)(256 * key + 16 * slot)};
  };
  // requests keys key0 .. key0 + 3 of K and V, and their cos/sin rows
  auto copy4 = [&](auto all, auto half, const Tile& t, int ln, int key0, const Piece& pc, uint32_t buf) __attribute__((always_inline)) {
    const int klim = t.flags & 31;
    const uint32_t dst = buf + 256 * key0;
    uint32_t ko = pc.k, vo = pc.v, co = pc.cs;
    int row = key0 < 16 ? t.row0 : t.row1;
    int key = key0 + (ln >> 4);
    if (klim != kShTile - 1) {  // keys behind the last one repeat it
      const int slot = ln & 15, mine = key;
      row = min(key0, klim) < 16 ? t.row0 : t.row1;
      key = min(key, klim);
      const uint32_t ro = (uint32_t)(key & 15) * kv_row_bytes;
      ko = ro + 16 * (slot ^ sh_kswz(mine));
      vo = ro + 16 * (slot ^ sh_vswz(mine));
      co = 256 * key + 16 * slot;
    }
    const size_t off = (size_t)(uint32_t)row * kv_row_bytes;
    // few rows: their keys are theirs alone, and not kept in the caches (passes over new inputs: 64
    // chats 133 -> 126 us, drafts 111 -> 107, 8 samples of 128K 230 -> 228, though their tiles' next
    // views then miss the L2: 774 MB fetched for 569); blocks of many rows mostly share theirs
    if constexpr (decltype(all)::value) {
      dma16_s(kbase + off, ko, dst);
      dma16_s(vbase + off, vo, dst + kShImg);
    } else {
      dma16_s_nt(kbase + off, ko, dst);
      dma16_s_nt(vbase + off, vo, dst + kShImg);
    }
    if (t.lG != 0) {
      const FastDiv f = {t.m, t.lG & 63, 2};
      co = fastdiv_ge2((uint32_t)(t.km + key), f) * 256 + 16 * (ln & 15);
    }
    const uint32_t* const cs = decltype(half)::value ? a.half : a.rope16;
    dma16_s(cs + (size_t)(t.lG != 0 ? t.f0 : t.k0) * 64, co, dst + 2 * kShImg);
  };
  // The copies of a wave, in the order of the list; a visit's description is read one ahead
  struct Copier {
    Piece pc[2];
    Tile nx;
  };
  auto peek = [&](Copier& c, int j) __attribute__((always_inline)) { c.nx = s_tiles[j & (kShList - 1)]; };
  auto copier = [&](auto all, int ln) __attribute__((always_inline)) {
    Copier c;
    c.pc[0] = piece_of(ln, decltype(all)::value ? 4 * wave : 8 * (wave - 4));
    c.pc[1] = piece_of(ln, decltype(all)::value ? 4 * wave : 8 * (wave - 4) + 4);
    peek(c, 0);
    return c;
  };
  auto issue = [&](auto all, auto half, Copier& c, int ln, int j) __attribute__((always_inline)) {
    const Tile t = {uni(c.nx.row0), uni(c.nx.row1), uni(c.nx.k0), uni(c.nx.flags), uni(c.nx.f0),
                    uni(c.nx.km), (uint32_t)uni((int)c.nx.m), (uint32_t)uni((int)c.nx.lG)};
    peek(c, j + 1);
    const uint32_t buf = smem_base + (uint32_t)(j % kShBufs) * kShBuf;
    if constexpr (decltype(all)::value) {
      copy4(all, half, t, ln, 4 * wave, c.pc[0], buf);
    } else {
      copy4(all, half, t, ln, 8 * (wave - 4), c.pc[0], buf);
      copy4(all, half, t, ln, 8 * (wave - 4) + 4, c.pc[1], buf);
    }
  };
  // Whether fp16 holds the keys of a wave, each spread over some lanes
  auto check = [&](float amax, int lanes) __attribute__((always_inline)) {
    if (__ballot(!(amax >= kShLow && amax < kShHigh)) == 0) return;
    for (int d = 1; d < lanes; d <<= 1) amax = fmaxf(amax, __shfl_xor(amax, d));
    if (sh_outside(amax)) s_again = 1;
  };
  // Rotation in place.  4 keys: lane -> key, half of a chunk pair; 8 keys: lane -> key, chunk pair
  auto rotate = [&](auto all, auto half, int ln, int j) __attribute__((always_inline)) {
    unsigned char* b = smem + (j % kShBufs) * kShBuf;
    if constexpr (decltype(all)::value) {
      const int r4_key = 4 * wave + (ln >> 4), r4_c = (ln >> 1) & 7, r4_h = ln & 1;
      const int r4_lo = sh_koff(r4_key, r4_c) + 8 * r4_h, r4_hi = sh_koff(r4_key, r4_c + 8) + 8 * r4_h;
      const int r4_cs = 2 * kShImg + r4_key * 256 + 32 * r4_c + 16 * r4_h;
      const sh_u32x2 xl = *(const sh_u32x2*)(b + r4_lo), xh = *(const sh_u32x2*)(b + r4_hi);
      const u32x4 cs = *(const u32x4*)(b + r4_cs);
      if constexpr (decltype(half)::value) {
        float v[8], amax = 0.f;
        rot_pairs_f16(xl[0], xh[0], cs[0], cs[1], v, amax);
        rot_pairs_f16(xl[1], xh[1], cs[2], cs[3], v + 4, amax);
        *(sh_u32x2*)(b + r4_lo) = sh_u32x2{pack_f16(v[0], v[1]), pack_f16(v[4], v[5])};
        *(sh_u32x2*)(b + r4_hi) = sh_u32x2{pack_f16(v[2], v[3]), pack_f16(v[6], v[7])};
        check(amax, 16);
        return;
      }
      uint32_t l0, h0, l1, h1;
      rot_word_dot2(xl[0], xh[0], cs[0], cs[1], l0, h0);
      rot_word_dot2(xl[1], xh[1], cs[2], cs[3], l1, h1);
      *(sh_u32x2*)(b + r4_lo) = sh_u32x2{l0, l1};
      *(sh_u32x2*)(b + r4_hi) = sh_u32x2{h0, h1};
    } else {
      const int r8_key = 8 * (wave - 4) + (ln >> 3), r8_c = ln & 7;
      const int r8_lo = sh_koff(r8_key, r8_c), r8_hi = sh_koff(r8_key, r8_c + 8);
      const int r8_cs = 2 * kShImg + r8_key * 256 + 32 * r8_c;
      const u32x4 xl = *(const u32x4*)(b + r8_lo), xh = *(const u32x4*)(b + r8_hi);
      const u32x4 ca = *(const u32x4*)(b + r8_cs), cb = *(const u32x4*)(b + r8_cs + 16);
      u32x4 lo, hi;
      if constexpr (decltype(half)::value) {
        float amax = 0.f;
#pragma unroll
        for (int w2 = 0; w2 < 4; ++w2) {
          float v[4];
          rot_pairs_f16(xl[w2], xh[w2], w2 < 2 ? ca[2 * w2] : cb[2 * w2 - 4],
                        w2 < 2 ? ca[2 * w2 + 1] : cb[2 * w2 - 3], v, amax);
          lo[w2] = pack_f16(v[0], v[1]);
          hi[w2] = pack_f16(v[2], v[3]);
        }
        *(u32x4*)(b + r8_lo) = lo;
        *(u32x4*)(b + r8_hi) = hi;
        check(amax, 8);
        return;
      }
#pragma unroll
      for (int w2 = 0; w2 < 4; ++w2) {
        uint32_t l, hh;
        rot_word_dot2(xl[w2], xh[w2], w2 < 2 ? ca[2 * w2] : cb[2 * w2 - 4],
                      w2 < 2 ? ca[2 * w2 + 1] : cb[2 * w2 - 3], l, hh);
        lo[w2] = l;
        hi[w2] = hh;
      }
      *(u32x4*)(b + r8_lo) = lo;
      *(u32x4*)(b + r8_hi) = hi;
    }
  };

  int n = 0;  // visits of the held segments
  // Addresses of visits j0 .. j0 + count - 1, a thread each: the last waves
  auto fill = [&](int j0, int count) __attribute__((always_inline)) {
    int me = tid;
    asm volatile("" : "+v"(me));  // as above: nothing of this is held in between
    const int at = me - (kShThreads - count), j = j0 + at;
    if (at < 0 || j >= n) return;
    int i = 0;  // the held segment: the last that begins at or before the visit
#pragma unroll
    for (int d = kShSegs / 2; d > 0; d >>= 1)
      if (s_before[i + d] <= j) i += d;
    const Segment& sg = s_segs[i];
    const int vis = s_from[i] + j - s_before[i];
    const int rem = sg.n_rem * sg.n_views;
    Tile s = {};
    int t = sg.loc0 + vis - rem;
    View vw = {};
    if (vis < rem) {
      t = sg.n_views == 1 ? vis : vis / sg.n_views;
      vw = pv.views[sg.view0 + vis - t * sg.n_views];
    }
    s.k0 = sg.k0 + t * kShTile;
    const int klim = min(kShTile - 1, sg.kend - 1 - s.k0);
    const int32_t* bt = a.table + (size_t)sg.seq * a.max_pages;
    auto pool_row = [&](int k) {
      const int pg = min(max(bt[k >> a.page_shift], 0), a.n_pages - 1);
      return (pg << a.page_shift) + (k & (a.page - 1));
    };
    s.row0 = pool_row(s.k0);
    s.row1 = klim < 16 ? s.row0 : a.page >= kShTile && (s.k0 & (a.page - 1)) + 16 < a.page
                                      ? s.row0 + 16
                                      : pool_row(s.k0 + 16);
    const bool last = j + 1 == n || (i + 1 < kShSegs && s_before[i + 1] == j + 1);
    s.flags = klim | (last ? kTfLast : 0) | i << kTfSeg;
    if (vis < rem) {
      const FastDiv f = {vw.m, vw.l, (uint32_t)vw.G};
      s.f0 = (int)fastdiv_ge2((uint32_t)s.k0, f);
      s.km = s.k0 - vw.G * s.f0;
      s.m = vw.m;
      s.lG = vw.l | (uint32_t)vw.G << 6;
    }
    s_tiles[j & (kShList - 1)] = s;
  };

  // A wave's copies of tile i + 1 have landed; those of the next two may fly
  auto landed = [&](auto all, int i) __attribute__((always_inline)) {
    constexpr int k = decltype(all)::value ? kShCopies : 2 * kShCopies;
    if (i + 3 < n)
      wait_vmem_n<2 * k>();
    else if (i + 2 < n)
      wait_vmem_n<k>();
    else
      wait_vmem();
  };
  // Beside visit i: the request of the tile that takes visit i - 2's buffer, the next one's
  // rotation
  auto produce = [&](auto all, auto half, Copier& cp, int ln, int i) __attribute__((always_inline)) {
    if (i + kShAhead < n) issue(all, half, cp, ln, i + kShAhead);
    if (i + 1 < n) rotate(all, half, ln, i + 1);
  };
  auto refill = [&](int i) __attribute__((always_inline)) {
    if ((i & (kShList / 2 - 1)) == 0 && i > 0 && i + kShList / 2 < n) fill(i + kShList / 2, kShList / 2);
  };
  auto start = [&](auto all, auto half, Copier& cp, int ln) __attribute__((always_inline)) {
    constexpr int k = decltype(all)::value ? kShCopies : 2 * kShCopies;
    const int first = min(n, kShAhead);
    for (int j = 0; j < first; ++j) issue(all, half, cp, ln, j);
    if (first == kShAhead)
      wait_vmem_n<(kShAhead - 1) * k>();
    else
      wait_vmem();
    rotate(all, half, ln, 0);
  };

  // Row of a segment (up to 256) over the query heads of a kv head: the inverse is less than
  // 2^-16 too large, so the quotient of 256 less than 1 / g
  auto by_g = [&](int r) { return (int)((uint32_t)r * (uint32_t)a.g_inv >> 16); };
  // The row that a lane serves: its query, position, G and first local key
  struct Row {
    const uint16_t* q;
    int pos, G, lim;
  };
  auto row_of = [&](const Segment& sg, int r) {
    Row x;
    r = min(r, sg.rows - 1);
    const int t = by_g(r);
    int seq, len;
    if (sg.kind == kSegShared) {
      const Member mb = pv.members[sg.m0 + t];
      seq = mb.seq;
      len = mb.len;
    } else if (sg.kind == kSegOwn) {
      seq = sg.seq;
      len = sg.kend;
    } else {  // the last row's position is kend - 1
      seq = sg.q0 + t;
      len = sg.kend - (by_g(sg.rows) - 1 - t);
    }
    x.pos = max(len - 1, 0);
    x.G = rows_group(sg.len > 0 ? sg.len : len, a.bifocal, a.w_pre);
    x.lim = first_local(x.G, x.pos, a.w0);
    x.q = a.q + ((size_t)max(seq, 0) * a.Hq + h * a.g + r - t * a.g) * kHeadDim;
    return x;
  };
  // Keys [lo, hi) of the tile that a row keeps: in the remote view those before its first
  // local key, if its G is the view's, else those from it on; none behind itself
  auto keep = [&](const Row& x, int view_G, int k0, int kend, int* lo, int* hi) __attribute__((always_inline)) {
    *hi = min(kend, x.pos + 1) - k0;
    *lo = 0;
    if (view_G > 0)
      *hi = x.G == view_G ? min(*hi, x.lim - k0) : 0;
    else
      *lo = x.lim - k0;
  };
  auto state_at = [&](const Segment& sg, int half) {
    const int rows = uni(sg.rows), halves = uni(state_halves(sg));
    return a.states + ((size_t)h * all_rows + uni(sg.row0) +
                       (size_t)((w - uni(sg.w_first)) * halves + half) * rows) * kShStateFloats;
  };

  // ---- the visits of a segment from i on, by the waves that hold its rows: 32 of them and all
  // keys of a tile each.  The scores of visit i are formed beside the softmax and the value
  // product of visit i - 1, whose tile stays in its buffer until then.
  auto consume = [&](auto all, auto few, auto half, Copier& cp, int i) __attribute__((always_inline)) {
    int ln = lane;  // what follows from it is formed here: held across all loops it would spill
    asm volatile("" : "+v"(ln));
    const Segment& sg = s_segs[uni(s_tiles[i & (kShList - 1)].flags) >> kTfSeg];
    const int rows = uni(sg.rows), kend = uni(sg.kend);
    const int hl32 = ln >> 5, kr_lane = ln & 31;
    const int vk_lane = 4 * hl32 + ((ln & 15) >> 2);
    const int vc_lane = 2 * ((ln >> 4) & 1) + ((ln & 3) >> 1);
    constexpr bool FEW = decltype(few)::value;
    using Op = std::conditional_t<decltype(half)::value, f16x8, bf16x8>;
    const int rw = FEW ? wave & 1 : wave, set = wave >> 1;
    const int row = 32 * rw + kr_lane;
    const bool on = 32 * rw < rows;
    const Row x = row_of(sg, row);
    Op qop[8];
    f32x16 acc[4], nx_sc = f32x16{}, neg_m = f32x16{};
    float m_ref = 0.f, l_run = 0.f;
#pragma unroll
    for (int d = 0; d < 4; ++d) acc[d] = f32x16{};
#pragma unroll
    for (int s = 0; s < 8; ++s) qop[s] = Op{};
    int q_view = -1;

    // the visit's scalars, read a visit ahead
    int nx_flags = s_tiles[i & (kShList - 1)].flags, nx_k0 = s_tiles[i & (kShList - 1)].k0;
    uint32_t nx_lG = s_tiles[i & (kShList - 1)].lG;
    int flags, k0, view_G;
    auto enter = [&]() __attribute__((always_inline)) {
      if constexpr (decltype(all)::value) landed(all, i);
      flags = uni(nx_flags);
      k0 = uni(nx_k0);
      view_G = uni((int)nx_lG) >> 6;
      __syncthreads();  // tile i is rotated, tile i - 2 used by all
      const Tile& t = s_tiles[(i + 1) & (kShList - 1)];
      nx_flags = t.flags;
      nx_k0 = t.k0;
      nx_lG = t.lG;
      if constexpr (decltype(all)::value) {
        produce(all, half, cp, ln, i);
        refill(i);
      }
      if (on && (view_G > 0) != q_view && (!FEW || (i & 1) == set)) {
        q_view = view_G > 0;
        const int pos = view_G > 0 ? x.pos / x.G : x.pos;
        float amax = 0.f;
#pragma unroll
        for (int s = 0; s < 4; ++s)
          sh_rotate_q(x.q, 16 * s + 8 * hl32, a.rope, pos, a.q_scale, qop[s], qop[s + 4], amax);
        if constexpr (decltype(half)::value) {
          if (sh_outside(sh_max32(amax))) s_again = 1;
        }
      }
    };
    // S^T = K Q^T - m of visit i: its key operands are requested ahead, then multiplied
    constexpr int kKr = FEW ? 8 : 4;
    Op kr[kKr];
    auto kop = [&](int s) __attribute__((always_inline)) {
      return *(const Op*)(smem + (i % kShBufs) * kShBuf + sh_koff(kr_lane, 2 * s + hl32));
    };
    auto keys = [&]() __attribute__((always_inline)) {
#pragma unroll
      for (int s = 0; s < kKr; ++s) kr[s] = kop(s);
    };
    auto scores = [&]() __attribute__((always_inline)) {
      if constexpr (!FEW) {  // -m takes no registers between visits
#pragma unroll
        for (int e = 0; e < 16; ++e) nx_sc[e] = -m_ref;
      } else {
        nx_sc = neg_m;
      }
#pragma unroll
      for (int s = 0; s < 8; ++s) {
        nx_sc = mfma32(kr[s & (kKr - 1)], qop[s], nx_sc);
        if (s + kKr < 8) kr[s & (kKr - 1)] = kop(s + kKr);
      }
    };
    // Scores of a visit at key c0 in view cG, masked
    bool has = false;  // whether the row has a key in that tile
    auto mask = [&](f32x16& sc, int c0, int cG) __attribute__((always_inline)) {
      int lo, hi;
      keep(x, cG, c0, kend, &lo, &hi);
      has = lo < min(hi, kShTile);
      if (__ballot(lo > 0 || hi < kShTile) != 0) {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int t = 8 * (e >> 2) + (e & 3) + 4 * hl32;
          sc[e] = t >= lo && t < hi ? sc[e] : -INFINITY;
        }
      }
    };
    bf16x8 pb[2];
    // The weights and their sum over both lanes of a row
    auto weights = [&](const f32x16& sc) __attribute__((always_inline)) {
      float ps0 = 0.f, ps1 = 0.f;
      const sh_bf16x2 one = {(__bf16)1.0f, (__bf16)1.0f};
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        float p[8];
#pragma unroll
        for (int t = 0; t < 8; ++t) p[t] = fast_exp2(sc[8 * q + t]);
        pb[q] = pack8(p);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const sh_bf16x2 pr = {pb[q][2 * u], pb[q][2 * u + 1]};
          if (u & 1)
            ps1 = __builtin_amdgcn_fdot2_f32_bf16(pr, one, ps1, false);
          else
            ps0 = __builtin_amdgcn_fdot2_f32_bf16(pr, one, ps0, false);
        }
      }
      const float ps = ps0 + ps1;
      const sh_u32x2 both =
          __builtin_amdgcn_permlane32_swap(__float_as_uint(ps), __float_as_uint(ps), false, false);
      return __uint_as_float(both[0]) + __uint_as_float(both[1]);
    };
    // The row's reference follows its first keys, and scores far above it: noticed by the sum of the
    // weights, which are then formed again (and the next visit's scores, which were taken
    // against the old reference, moved)
    auto settle = [&](f32x16& sc, float ps, bool next) __attribute__((always_inline)) {
      const bool bad = !(ps <= kShMaxSum) || (l_run == 0.f && has && ps < 1.f);
      if (__ballot(bad) != 0) {
        float mt = fmaxf(sc[0], sc[1]);
#pragma unroll
        for (int e = 2; e < 16; e += 2) mt = fmaxf(mt, fmaxf(sc[e], sc[e + 1]));
        mt = sh_max32(mt);
        const float shift = bad && mt != -INFINITY ? mt : 0.f;
        const float alpha = l_run == 0.f ? 1.f : fast_exp2(-shift);
#pragma unroll
        for (int e = 0; e < 16; ++e) sc[e] -= shift;
        if (next) {
#pragma unroll
          for (int e = 0; e < 16; ++e) nx_sc[e] -= shift;
        }
#pragma unroll
        for (int d = 0; d < 4; ++d) acc[d] *= alpha;
        l_run *= alpha;
        m_ref += shift;
        if constexpr (FEW) {
#pragma unroll
          for (int e = 0; e < 16; ++e) neg_m[e] = -m_ref;
        }
        ps = weights(sc);
      }
      l_run += ps;
    };
    // Value operand m of visit j, and the product: the first of them requested ahead
    constexpr int kVr = FEW ? 8 : 4;
    bf16x8 vr[kVr];
    auto vop = [&](int j, int m) __attribute__((always_inline)) {
      const unsigned char* p = smem + (j % kShBufs) * kShBuf + kShImg + 4096 * (m >> 2) +
                               sh_voff(vk_lane, 4 * (m & 3) + vc_lane) + 8 * (ln & 1);
      return concat_tr(lds_read_tr4(p), lds_read_tr4(p + 2048));
    };
    auto tile_values = [&](int j) __attribute__((always_inline)) {
#pragma unroll
      for (int m = 0; m < kVr; ++m) vr[m] = vop(j, m);
    };
    auto values = [&](int j) __attribute__((always_inline)) {
#pragma unroll
      for (int m = 0; m < 8; ++m) {
        acc[m & 3] = mfma32(vr[m & (kVr - 1)], pb[m >> 2], acc[m & 3]);
        if (m + kVr < 8) vr[m & (kVr - 1)] = vop(j, m + kVr);
      }
    };
    auto fence = []() __attribute__((always_inline)) { __builtin_amdgcn_sched_barrier(0); };

    if constexpr (FEW) {
      // A pair's visit takes two barriers' time: its scores, then the softmax and the value product
      bool last = false;
      if ((i & 1) != set) {  // begins with the other pair's
        enter();
        last = (flags & kTfLast) != 0;
        if (!last) ++i;
      }
      while (!last) {
        enter();
        last = (flags & kTfLast) != 0;
        const int own_i = i, own_k0 = k0, own_G = view_G;
        if (on) {
          keys();
          fence();
          scores();
        }
        if (!last) {
          ++i;
          enter();
          last = (flags & kTfLast) != 0;
          if (!last) ++i;
        }
        if (on) {
          tile_values(own_i);
          fence();
          mask(nx_sc, own_k0, own_G);
          const float ps = weights(nx_sc);
          settle(nx_sc, ps, false);
          values(own_i);
        }
      }
    } else {
      enter();
      if (on) {
        keys();
        fence();
        scores();
      }
      while ((flags & kTfLast) == 0) {
        const int c0 = k0, cG = view_G;
        ++i;
        enter();
        if (on) {
          keys();
          f32x16 sc = nx_sc;
          mask(sc, c0, cG);
          scores();
          const float ps = weights(sc);
          settle(sc, ps, true);
          tile_values(i - 1);
          values(i - 1);
        }
      }
      if (on) {
        tile_values(i);
        fence();
        mask(nx_sc, k0, view_G);
        const float ps = weights(nx_sc);
        settle(nx_sc, ps, false);
        values(i);
      }
    }
    if (row < rows) {
      if (!FEW && written_whole(sg)) {
        const int t = by_g(row);
        const Member mb = pv.members[sg.m0 + t];
        if (mb.seq >= 0) {
          const float inv = 1.f / l_run;
          const int hd = h * a.g + row - t * a.g;
          uint16_t* o = a.o + ((size_t)mb.seq * a.Hq + hd) * kHeadDim;
          if (a.lse != nullptr && hl32 == 0)
            a.lse[(size_t)hd * a.T + mb.seq] = (m_ref + log2f(l_run)) * 0.69314718055994531f;
#pragma unroll
          for (int db = 0; db < 4; ++db) {
#pragma unroll
            for (int q4 = 0; q4 < 4; ++q4) {
              f32x4 y;
#pragma unroll
              for (int jj = 0; jj < 4; ++jj) y[jj] = acc[db][4 * q4 + jj] * inv;
              *(bf16x4*)(o + 32 * db + 8 * q4 + 4 * hl32) = __builtin_convertvector(y, bf16x4);
            }
          }
        }
      } else {
        float* st = state_at(sg, FEW ? set : 0);
#pragma unroll
        for (int db = 0; db < 4; ++db) {
#pragma unroll
          for (int q4 = 0; q4 < 4; ++q4) {
            f32x4 t;
#pragma unroll
            for (int jj = 0; jj < 4; ++jj) t[jj] = acc[db][4 * q4 + jj];
            *(f32x4*)(st + ((size_t)(8 * db + 2 * q4 + hl32) * rows + row) * 4) = t;
          }
        }
        if (hl32 == 0)
          *(float2*)(st + (size_t)rows * kHeadDim + 2 * row) =
              make_float2(l_run == 0.f ? -INFINITY : m_ref, l_run);
        if constexpr (!decltype(half)::value) {  // all by one wave here: the second state is empty
          if (hl32 == 0 && uni(state_halves(sg)) == 2)
            *(float2*)(state_at(sg, 1) + (size_t)rows * kHeadDim + 2 * row) = make_float2(-INFINITY, 0.f);
        }
      }
    }
    return i + 1;
  };

  // ---- the segments of the range, up to 64 of one kind at a time
  for (int s0 = uni(pv.wg_first[w]); s0 < n_segs;) {
    if (wave == 0) {
      int ln = lane;
      asm volatile("" : "+v"(ln));
      const int i = s0 + ln;
      int va = 0, vb = 0;
      bool past = true, large = false;
      if (i < n_segs) {
        const Segment sg = pv.segs[i];
        s_segs[ln] = sg;
        const unsigned long long st = sg.start_lo | (unsigned long long)sg.start_hi << 32;
        const uint32_t c = (uint32_t)visit_cost(sg.rows);
        auto below = [&](unsigned long long x) {  // its visits that begin before x
          if (x <= st + kSegCost) return 0;
          const unsigned long long d = x - st - kSegCost;
          return d >= (unsigned long long)sg.visits * c ? sg.visits
                                                        : (int)(((uint32_t)d + c - 1) / c);
        };
        va = below(x0);
        vb = below(x1);
        past = st >= x1;
        large = sg.rows > kShSmall;
      }
      // those before the first of the other kind
      const unsigned long long some = __ballot(vb > va), big = __ballot(vb > va && large);
      const bool kind = some != 0 && (big >> __builtin_ctzll(some) & 1) != 0;
      const unsigned long long other = some & (kind ? ~big : big);
      const int stop = other != 0 ? __builtin_ctzll(other) : kShSegs;
      if (ln >= stop) vb = va;
      const int incl = wave_scan(vb - va);
      s_from[ln] = va;
      s_before[ln] = incl - (vb - va);
      if (ln == 63) s_tiles[0].k0 = incl;
      if (__ballot(past && ln < stop) == 0 || stop < kShSegs) {
        if (ln == 0) s_tiles[0].row0 = s0 + stop;
      } else if (ln == 0) {
        s_tiles[0].row0 = n_segs;
      }
      if (ln == 0) s_tiles[0].row1 = kind;
    }
    __syncthreads();
    n = uni(s_tiles[0].k0);
    const int next = uni(s_tiles[0].row0), kind = uni(s_tiles[0].row1);
    __syncthreads();
    auto run = [&](auto half) __attribute__((always_inline)) {
      if (tid == 0) s_again = 0;
      fill(0, kShList);
      __syncthreads();
      if (kind) {
        int ln = lane;
        asm volatile("" : "+v"(ln));
        Copier cp = copier(std::true_type{}, ln);
        start(std::true_type{}, half, cp, ln);
        for (int i = 0; i < n;) i = consume(std::true_type{}, std::false_type{}, half, cp, i);
      } else if (wave < 4) {
        Copier none;
        for (int i = 0; i < n;) {
          const Segment& sg = s_segs[uni(s_tiles[i & (kShList - 1)].flags) >> kTfSeg];
          i = decltype(half)::value && uni(state_halves(sg)) == 2
                  ? consume(std::false_type{}, std::true_type{}, half, none, i)
                  : consume(std::false_type{}, std::false_type{}, half, none, i);
        }
      } else {
        int ln = lane;
        asm volatile("" : "+v"(ln));
        Copier cp = copier(std::false_type{}, ln);
        start(std::false_type{}, half, cp, ln);
        for (int i = 0; i < n; ++i) {
          landed(std::false_type{}, i);
          __syncthreads();
          produce(std::false_type{}, half, cp, ln, i);
          refill(i);
        }
      }
    };
    if (n > 0) {
      run(std::true_type{});
      __syncthreads();
      if (uni(s_again) != 0) {
        __syncthreads();
        run(std::false_type{});
      }
    }
    s0 = next;
    if (s0 < n_segs) __syncthreads();  // the lists and the buffers are free
  }
}

// The states of a row, joined: O = sum 2^(m - M) O~ / sum 2^(m - M) l.  Workgroup: 8
// rows of one kv head in member order; thread -> row, 4 channels, every other state, four of
// them requested at once.  4.6 us for 2 sequences, 8.8 for the 64 states of a row that
// all workgroups of a kv head leave: latency.
constexpr int kMgRows = 8;
__global__ __launch_bounds__(512) void merge_shared_kernel(SharedArgs a) {
  __shared__ f32x4 s_o[32][kMgRows];
  __shared__ float2 s_ml[32][kMgRows];
  const PlanView pv = plan_of(a);
  if (!plan_fits(a, pv.header)) return;
  const int h = blockIdx.y;
  const int rl = threadIdx.x & (kMgRows - 1), c = (threadIdx.x / kMgRows) & 31, half = threadIdx.x >> 8;
  const int n_rows = pv.header[kHdMembers] * a.g;
  for (int r0 = blockIdx.x * kMgRows; r0 < n_rows; r0 += gridDim.x * kMgRows) {
    const int r = r0 + rl;
    const Member mb = pv.members[min(r, n_rows - 1) / a.g];
    bool on = r < n_rows && mb.seq >= 0;
    float M = -INFINITY, den = 0.f;
    f32x4 acc = f32x4{};
    const float* base = a.states + (size_t)h * pv.header[kHdRows] * kShStateFloats;
    auto join = [&](int seg, bool block) {
      if (seg < 0) return;
      const Segment sg = pv.segs[seg];
      const int n = sg.n_w * state_halves(sg);
      if (written_whole(sg)) {
        on = false;
        return;
      }
      const int at = block ? r - sg.m0 * a.g : r % a.g;
      constexpr int kAtOnce = 4;
      for (int i0 = half; i0 < n; i0 += 2 * kAtOnce) {
        float2 ml[kAtOnce];
        f32x4 x[kAtOnce];
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
          const float* st = base + (size_t)(sg.row0 + min(i0 + 2 * j, n - 1) * sg.rows) * kShStateFloats;
          ml[j] = *(const float2*)(st + (size_t)sg.rows * kHeadDim + 2 * at);
          x[j] = *(const f32x4*)(st + ((size_t)c * sg.rows + at) * 4);
          if (i0 + 2 * j >= n) ml[j] = make_float2(-INFINITY, 0.f);
        }
        float top = M;
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
          if (ml[j].y == 0.f) ml[j].x = -INFINITY;  // no key of this row
          top = fmaxf(top, ml[j].x);
        }
        const float wa = M == -INFINITY ? 0.f : fast_exp2(M - top);
        den *= wa;
        acc *= wa;
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
          if (ml[j].y == 0.f) continue;
          const float wb = fast_exp2(ml[j].x - top);
          den += wb * ml[j].y;
          acc += wb * x[j];
        }
        M = top;
      }
    };
    if (on) {
      join(mb.pre, true);
      join(mb.suf, false);
    }
    if (half == 1) {
      s_o[c][rl] = acc;
      s_ml[c][rl] = make_float2(M, den);
    }
    __syncthreads();
    if (half == 0 && on) {
      const float2 ml = s_ml[c][rl];
      const float top = fmaxf(M, ml.x);
      f32x4 out = f32x4{};
      float lse = -INFINITY;
      if (den != 0.f || ml.y != 0.f) {
        const float wa = den == 0.f ? 0.f : fast_exp2(M - top);
        const float wb = ml.y == 0.f ? 0.f : fast_exp2(ml.x - top);
        f32x4 sum = f32x4{};
        if (den != 0.f) sum += wa * acc;
        if (ml.y != 0.f) sum += wb * s_o[c][rl];
        const float all = wa * den + wb * ml.y;
        out = sum * (1.f / all);
        lse = (top + log2f(all)) * 0.69314718055994531f;
      }
      const int hd = h * a.g + r % a.g;
      *(bf16x4*)(a.o + ((size_t)mb.seq * a.Hq + hd) * kHeadDim + 4 * c) =
          __builtin_convertvector(out, bf16x4);
      if (a.lse != nullptr && c == 0) a.lse[(size_t)hd * a.T + mb.seq] = lse;
    }
    __syncthreads();  // s_o and s_ml are read
  }
}

// ---------------------------------------------------------------- launchers
static size_t chunk_plan_lds(int B, int T, int g) {
  return (5 * (size_t)B + 4) * sizeof(int) + chunk_sizes(B, T, g).segs * 12 + 8;
}
// 60 KB for the segments that the rows fill, beside 32 bytes for each of up to 2048 sequences
bool chunk_rows_fit(int T, int g) { return chunk_plan_lds(0, T, g) <= 60 * 1024; }

static hipError_t launch_plan(bool chunk, SharedPlanArgs& a, hipStream_t stream) {
  if (chunk) {
    const bool few = a.B <= 256 && a.T <= 4096;
    hipLaunchKernelGGL(chunk_plan_kernel, dim3(1), dim3(few ? 256 : kPlThreads),
                       chunk_plan_lds(a.B, a.T, a.g), stream, a);
  } else {
    const PlanSizes z = decode_sizes(a.B, a.n_groups, a.g);
    const size_t lists = z.segs * 8 + 8;
    const size_t lds = (2 * (size_t)a.B + 3 * (size_t)a.n_groups + 2) * sizeof(int) + lists;
    const bool few = a.B <= 128 && a.n_groups <= 128;
    hipLaunchKernelGGL(shared_plan_kernel, dim3(1), dim3(few ? 256 : kPlThreads), lds, stream, a);
  }
  return hipGetLastError();
}

hipError_t launch_shared_plan(bool bifocal, const int32_t* kv_lens, const int32_t* members,
                              const int32_t* group_starts, const int32_t* shared, int B,
                              int n_groups, int Hq, int Hkv, int max_pages, int page, int w_pre,
                              int w0, int n_cu, void* plan, hipStream_t stream) {
  SharedPlanArgs a{kv_lens, members, group_starts, shared, nullptr, plan, B, n_groups, 0, Hq / Hkv,
                   Hkv, max_pages, page, head_workgroups(n_cu, Hkv), bifocal ? 1 : 0, w_pre, w0,
                   nullptr, 0};
  return launch_plan(false, a, stream);
}

static hipError_t launch_rows(SharedArgs& a, hipStream_t stream, hipEvent_t ev0, hipEvent_t ev1) {
  // a chunk's tokens may all be the prefill kernel's
  const long long rows = (long long)(a.chunk ? a.T : a.B) * a.g;
  long long merges = (rows + kMgRows - 1) / kMgRows;
  if (a.chunk) merges = std::min<long long>(merges, std::max(1, 512 / a.Hkv));
  hipError_t e = hipSuccess;
  if (ev0 != nullptr && (e = hipEventRecord(ev0, stream)) != hipSuccess) return e;
  hipLaunchKernelGGL(shared_rows_kernel, dim3((unsigned)a.n_wg * a.Hkv), dim3(kShThreads), 0, stream, a);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  if (ev1 != nullptr && (e = hipEventRecord(ev1, stream)) != hipSuccess) return e;
  hipLaunchKernelGGL(merge_shared_kernel, dim3((unsigned)merges, (unsigned)a.Hkv),
                     dim3(512), 0, stream, a);
  return hipGetLastError();
}

static SharedArgs rows_args(bool bifocal, const uint16_t* q, const uint16_t* k, const uint16_t* v,
                            const int32_t* table, int max_pages, int n_pages, int page_shift,
                            void* plan, void* states, uint16_t* o, const float2* rope,
                            const uint32_t* half, const uint32_t* rope16, int B, int Hq, int Hkv, int w_pre, int w0,
                            int n_cu) {
  SharedArgs a = {};
  a.q = q;
  a.k = k;
  a.v = v;
  a.table = table;
  a.o = o;
  a.rope = rope;
  a.half = half;
  a.rope16 = rope16;
  a.plan = plan;
  a.states = (float*)states;
  a.B = B;
  a.Hq = Hq;
  a.Hkv = Hkv;
  a.g = Hq / Hkv;
  a.g_inv = 65536 / a.g + 1;
  a.max_pages = max_pages;
  a.n_pages = n_pages;
  a.page = 1 << page_shift;
  a.page_shift = page_shift;
  a.n_wg = head_workgroups(n_cu, Hkv);
  a.bifocal = bifocal ? 1 : 0;
  a.w_pre = w_pre;
  a.w0 = w0;
  a.q_scale = 1.4426950408889634f / sqrtf((float)kHeadDim);
  return a;
}

hipError_t launch_decode_shared(bool bifocal, const uint16_t* q, const uint16_t* k,
                                const uint16_t* v, const int32_t* table, int max_pages,
                                int n_pages, int page_shift, void* plan, uint16_t* o,
                                const float2* rope, const uint32_t* half, const uint32_t* rope16,
                                int B, int n_groups,
                                int Hq, int Hkv, int w_pre, int w0, int n_cu, void* ws,
                                hipStream_t stream, hipEvent_t ev0, hipEvent_t ev1) {
  SharedArgs a = rows_args(bifocal, q, k, v, table, max_pages, n_pages, page_shift, plan, ws, o, rope,
                           half, rope16, B, Hq, Hkv, w_pre, w0, n_cu);
  a.n_groups = n_groups;
  return launch_rows(a, stream, ev0, ev1);
}

// scratch: chunk_scratch_bytes
hipError_t launch_chunk_rows(bool bifocal, const uint16_t* q, const uint16_t* k, const uint16_t* v,
                             const int32_t* table, int max_pages, int n_pages, int page_shift,
                             const int32_t* cu, const int32_t* kv_lens, uint16_t* o, float* lse,
                             const float2* rope, const uint32_t* half, const uint32_t* rope16,
                             int B, int T, int Hq, int Hkv, int w_pre, int w0, float slack, int n_cu, void* scratch,
                             hipStream_t stream, hipEvent_t ev0, hipEvent_t ev1) {
  const int g = Hq / Hkv, page = 1 << page_shift;
  const ChunkScratch at = chunk_scratch(B, T, Hq, Hkv, max_pages, page);
  char* const mem = (char*)scratch;
  const bool blocks = chunk_blocks(B, T, Hkv, g, max_pages, page);
  SharedPlanArgs p{kv_lens, nullptr, nullptr, nullptr, cu, scratch, B, 0, T, g, Hkv, max_pages,
                   page, head_workgroups(n_cu, Hkv), bifocal ? 1 : 0, w_pre, w0,
                   blocks ? (ChunkPart*)(mem + at.parts) : nullptr,
                   (int)most_parts(B, T, g, head_workgroups(kShMaxWg, Hkv))};
  hipError_t e = launch_plan(true, p, stream);
  if (e != hipSuccess) return e;
  if (ev0 != nullptr && (e = hipEventRecord(ev0, stream)) != hipSuccess) return e;
  if (blocks) {
    // no sequence past the window: G = 1 for all, and the vanilla kernel does
    const bool fused = bifocal && (long long)max_pages * page > w_pre;
    e = launch_prefill_chunks(fused, q, k, v, o, lse, rope, rope16, half, table, max_pages, page_shift,
                              n_pages, T, Hq, Hkv, w0, slack, p.parts, (int*)scratch + kHdParts,
                              p.most_parts, (float*)(mem + at.part_states), stream);
    if (e != hipSuccess) return e;
  }
  SharedArgs a = rows_args(bifocal, q, k, v, table, max_pages, n_pages, page_shift, scratch,
                           mem + at.states, o, rope, half, rope16, B, Hq, Hkv, w_pre, w0, n_cu);
  a.chunk = 1;
  a.T = T;
  a.lse = lse;
  return launch_rows(a, stream, nullptr, ev1);
}

}  // namespace jl
