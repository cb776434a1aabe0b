// decode_shared.hip -- one new token of every sequence over a paged bf16 cache in
// which sequences share a prefix: its keys and values are read once for all of them.
//
// Jet-Long (arXiv 2607.07740): the query of sequence b sits at q = L - 1, L its length,
// and takes a key k in the base view where q - k <= w0, else in the remote view of its
// own G = max(1, ceil(L / w_pretrained)) (Sec. 3, Eqs. (1)-(3)).  The softmax over a
// sequence's keys is the merge (Eq. (7)) of those over any parts of them, so the keys
// that n sequences share make one attention of n g rows (g query heads of a kv head),
// matrix shaped, and the rest of each sequence one of g rows.
//
// Plan (once per step, for every layer).  A segment is such an attention: up to 256
// rows, i.e. up to 256 / g sequences of a group, over the group's prefix, or one
// sequence over what lies behind it.  Its visits are grouped by the view that the
// keys are rotated to: one phase for each G >= 2 that occurs among its sequences, over
// the tiles that hold a remote key for one of these, and one in the base view.  The phases of
// all segments are one list, in which a tile of 32 keys counts what it costs; the
// workgroups of a kv head take equal ranges of it, whatever segments these span.
//
// Kernel: a workgroup (8 waves, one CU) streams the tiles of its range through a ring
// in LDS, K, V and the cos/sin rows of the keys' positions, four tiles in flight.  While
// tile i is multiplied, tile i + 1 is rotated in place, four keys a wave.  A wave owns
// 32 rows: S^T = K Q^T, online softmax of a row per lane pair, O^T += V^T P^T, as the
// prefill kernel.  Each (workgroup, segment) leaves its rows' states (m, l, O) in fp32,
// and the merge kernel joins those of a row.
#include <algorithm>
#include <climits>

#include "decode_shared.h"
#include "jl_device.h"

namespace jl {

constexpr int kShThreads = 512, kShWaves = 8;
constexpr int kShRows = 32 * kShWaves;  // rows of a segment at most
constexpr int kShTile = 32;             // keys of a tile
constexpr int kShImg = kShTile * kHeadDim * 2;       // K or V of a tile: 8 KB
constexpr int kShBuf = 2 * kShImg + kShTile * 256;   // and its 32 rows of bf16 (cos, sin)
constexpr int kShBufs = 6;
constexpr int kShAhead = kShBufs - 1;  // tiles requested before the first is used
constexpr int kShList = 256;           // tiles whose addresses are formed at once
constexpr int kShCopies = 3;           // of a wave per tile

// What a tile costs in the list, and a phase beside its tiles.
constexpr int kTileCost = 4, kPhaseCost = 16;
__host__ __device__ inline int tile_cost(int rows) { return rows <= 128 ? kTileCost : kTileCost + 2; }
constexpr int kMaxStep = kTileCost + 2 + kPhaseCost;  // most between two tiles that follow each other

struct Phase {
  int seg, G;      // G: the remote view of this G (>= 2), 0: the base view
  int k0, n;       // first key, tiles
  uint32_t start_lo, start_hi;  // cost before the phase
  int cost, kend;  // of a tile; end of the segment's keys
  uint32_t m, l;   // division by G
  int pad[2];
};
struct Segment {
  int m0, rows, g_seqs, kend;  // first member, rows, sequences, end of its keys
  int w_first, n_w;            // workgroups that hold some of its tiles
  int row0;                    // state rows before it
  int seq;                     // whose table row names its pages
};
struct Member {
  int seq, len;
  int pre, suf;  // its segments, -1: none
};

struct PlanView {
  int* header;
  int* wg_first;
  Member* members;
  Segment* segs;
  Phase* phases;
};

__host__ __device__ inline size_t plan_blocks(int B, int n_groups, int g) {
  return (size_t)n_groups + (size_t)B / (kShRows / g) + 1;
}
__host__ __device__ inline PlanView plan_view(void* p, int B, int n_groups, int g) {
  PlanView v;
  char* c = (char*)p;
  v.header = (int*)c;
  v.wg_first = (int*)(c + 128);
  v.members = (Member*)(c + 128 + 4 * kShMaxWg);
  v.segs = (Segment*)(v.members + B);
  v.phases = (Phase*)(v.segs + plan_blocks(B, n_groups, g) + B);
  return v;
}
enum { kHdPhases = 0, kHdWg, kHdTotLo, kHdTotHi, kHdRows, kHdB, kHdG, kHdPage, kHdMaxPages,
       kHdHkv, kHdGroups, kHdBifocal, kHdWPre, kHdW0 };

size_t shared_plan_bytes(int B, int n_groups, int g) {
  const size_t blocks = plan_blocks(B, n_groups, g);
  return 128 + 4 * kShMaxWg + (size_t)B * sizeof(Member) + (blocks + B) * sizeof(Segment) +
         (blocks + 3 * (size_t)B) * sizeof(Phase);
}
// State rows of one kv head: every segment's once, and a segment's again where a
// workgroup's range ends inside it.
static size_t state_rows(int B, int g, int n_wg) {
  return 2 * (size_t)B * g + (size_t)(n_wg - 1) * std::min<size_t>(kShRows, (size_t)B * g);
}
static int head_workgroups(int n_cu, int Hkv) { return std::max(1, std::min(n_cu, kShMaxWg) / Hkv); }
constexpr int kShStateFloats = kHeadDim + 4;  // O, (m, l), and 8 bytes that keep 16-byte alignment
size_t decode_shared_workspace_bytes(int B, int Hq, int Hkv) {
  return (size_t)Hkv * state_rows(B, Hq / Hkv, head_workgroups(kShMaxWg, Hkv)) * kShStateFloats *
         sizeof(float);
}

// ------------------------------------------------------------------- plan
struct SharedPlanArgs {
  const int32_t* kv_lens;
  const int32_t* members;  // nullptr: 0 .. B - 1
  const int32_t* group_starts;
  const int32_t* shared;
  void* plan;
  int B, n_groups, g, Hkv, max_pages, page, n_wg, bifocal, w_pre, w0;
};

constexpr int kPlThreads = 1024, kPlWaves = kPlThreads / 64;

template <typename T>
__device__ inline T plan_scan(T v, T* s, T* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  T incl = v;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const T x = __shfl_up(incl, d);
    if (lane >= d) incl += x;
  }
  __syncthreads();
  if (lane == 63) s[wave] = incl;
  __syncthreads();
  T before = 0, all = 0;
#pragma unroll
  for (int i = 0; i < kPlWaves; ++i) {
    const T x = s[i];
    if (i < wave) before += x;
    all += x;
  }
  *total = all;
  return before + incl;
}

__device__ inline int wave_min(int v) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) v = min(v, __shfl_xor(v, d));
  return v;
}
__device__ inline int wave_max(int v) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) v = max(v, __shfl_xor(v, d));
  return v;
}

// A row's views: G, and its first key in the base view (0 where all are)
__device__ inline int plan_group(const SharedPlanArgs& a, int len) {
  return a.bifocal ? group_size(len, a.w_pre) : 1;
}
__device__ inline int first_local(int G, int len, int w0) {
  return G > 1 ? max(0, len - 1 - w0) : 0;
}

__device__ inline void put_phase(Phase* p, int seg, int G, int k0, int n, int rows, int kend) {
  const FastDiv f = make_fastdiv((uint32_t)max(G, 1));
  Phase x;
  x.seg = seg;
  x.G = G;
  x.k0 = k0;
  x.n = n;
  x.start_lo = x.start_hi = 0;
  x.cost = tile_cost(rows);
  x.kend = kend;
  x.m = f.m;
  x.l = f.l;
  x.pad[0] = x.pad[1] = 0;
  *p = x;
}

// The phases of a prefix block, by one wave (lane -> every 64th of its sequences):
// counts them, or writes them where `out` is given.
__device__ inline int block_phases(const SharedPlanArgs& a, const int* s_len, int m0, int n, int P,
                                   int seg, Phase* out) {
  const int lane = threadIdx.x & 63;
  const int tiles = (P + kShTile - 1) / kShTile;
  int count = 0, low = INT_MAX, G = 1;
  for (;;) {
    int next = INT_MAX, far = 0;  // the smallest G above the last, its furthest first local key
    for (int i = lane; i < n; i += 64) {
      const int len = s_len[m0 + i];
      if (len <= 0) continue;
      const int Gi = plan_group(a, len), lim = first_local(Gi, len, a.w0);
      if (G == 1) low = min(low, lim);
      if (Gi > G && Gi < next) {
        next = Gi;
        far = lim;
      } else if (Gi == next) {
        far = max(far, lim);
      }
    }
    const int nx = wave_min(next);
    far = wave_max(next == nx ? far : 0);
    if (G == 1) low = wave_min(low);
    if (nx == INT_MAX) break;
    G = nx;
    const int t = min(tiles, (far + kShTile - 1) / kShTile);
    if (t > 0) {
      if (out != nullptr && lane == 0) put_phase(out + count, seg, G, 0, t, n * a.g, P);
      ++count;
    }
  }
  const int t0 = low / kShTile;
  if (t0 < tiles) {
    if (out != nullptr && lane == 0)
      put_phase(out + count, seg, 0, t0 * kShTile, tiles - t0, n * a.g, P);
    ++count;
  }
  return count;
}

// One workgroup.  LDS: the members' lengths and groups' bounds.
__global__ __launch_bounds__(kPlThreads) void shared_plan_kernel(SharedPlanArgs a) {
  extern __shared__ int s_mem[];
  __shared__ unsigned long long s_scan[kPlWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const PlanView v = plan_view(a.plan, a.B, a.n_groups, a.g);
  int* const s_len = s_mem;                    // [B] by member, -1: no such sequence
  int* const s_start = s_len + a.B;            // [n_groups + 1]
  int* const s_pre = s_start + a.n_groups + 1; // [n_groups]: shared keys
  int* const s_blk = s_pre + a.n_groups;       // [n_groups + 1]: prefix blocks before the group
  int* const s_cnt = s_blk + a.n_groups + 1;   // [blocks + 1]: phases of a prefix block
  const int cap = (int)min((long long)a.max_pages * a.page, (long long)INT_MAX);
  const int per_block = kShRows / a.g;

  for (int i = tid; i <= a.n_groups; i += kPlThreads)
    s_blk[i] = min(max(a.group_starts[i], 0), a.B);
  for (int i = tid; i < a.B; i += kPlThreads) {
    const int seq = a.members != nullptr ? a.members[i] : i;
    const bool ok = (unsigned)seq < (unsigned)a.B;
    s_len[i] = ok ? min(max(a.kv_lens[seq], 0), cap) : -1;
  }
  __syncthreads();
  for (int i = tid; i <= a.n_groups; i += kPlThreads) {  // a start below an earlier one counts as that
    int top = 0;
    for (int j = 0; j <= i; ++j) top = max(top, s_blk[j]);
    s_start[i] = top;
    if (i < a.n_groups) s_pre[i] = INT_MAX;
  }
  __syncthreads();
  // a member's group: the first whose end lies behind it
  auto group_of = [&](int m) {
    int lo = 0, hi = a.n_groups;
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (s_start[mid + 1] > m) hi = mid; else lo = mid + 1;
    }
    return lo < a.n_groups && s_start[lo] <= m ? lo : -1;
  };
  for (int i = tid; i < a.B; i += kPlThreads) {
    const int gi = group_of(i);
    if (gi >= 0 && s_len[i] > 0) atomicMin(&s_pre[gi], s_len[i]);
  }
  __syncthreads();
  for (int i = tid; i < a.n_groups; i += kPlThreads) {
    const int n = s_start[i + 1] - s_start[i];
    s_pre[i] = n > 1 && s_pre[i] != INT_MAX ? min(max(a.shared[i], 0), s_pre[i]) / a.page * a.page : 0;
    s_blk[i] = n > 1 && s_pre[i] > 0 ? (n + per_block - 1) / per_block : 0;
  }
  __syncthreads();
  // prefix blocks before each group
  int n_blocks = 0;
  for (int c0 = 0; c0 < a.n_groups; c0 += kPlThreads) {
    const int i = c0 + tid;
    const unsigned long long x = i < a.n_groups ? (unsigned long long)s_blk[i] : 0ull;
    unsigned long long tot;
    const unsigned long long incl = plan_scan(x, s_scan, &tot);
    if (i < a.n_groups) s_blk[i] = n_blocks + (int)(incl - x);
    n_blocks += (int)tot;
  }
  if (tid == 0) s_blk[a.n_groups] = n_blocks;
  __syncthreads();
  auto block_of = [&](int blk, int* m0, int* n, int* P) {  // the last group that begins at or before it
    int lo = 0, hi = a.n_groups - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (s_blk[mid] <= blk) lo = mid; else hi = mid - 1;
    }
    *m0 = s_start[lo] + (blk - s_blk[lo]) * per_block;
    *n = min(per_block, s_start[lo + 1] - *m0);
    *P = s_pre[lo];
  };
  for (int blk = wave; blk < n_blocks; blk += kPlWaves) {
    int m0, n, P;
    block_of(blk, &m0, &n, &P);
    const int c = block_phases(a, s_len, m0, n, P, blk, nullptr);
    if (lane == 0) s_cnt[blk] = c;
  }
  __syncthreads();
  int at = 0;  // phases of the blocks
  for (int c0 = 0; c0 < n_blocks; c0 += kPlThreads) {
    const int i = c0 + tid;
    const unsigned long long x = i < n_blocks ? (unsigned long long)s_cnt[i] : 0ull;
    unsigned long long tot;
    const unsigned long long incl = plan_scan(x, s_scan, &tot);
    if (i < n_blocks) s_cnt[i] = at + (int)(incl - x);
    at += (int)tot;
  }
  __syncthreads();
  for (int blk = wave; blk < n_blocks; blk += kPlWaves) {
    int m0, n, P;
    block_of(blk, &m0, &n, &P);
    block_phases(a, s_len, m0, n, P, blk, v.phases + s_cnt[blk]);
    int from = INT_MAX;  // any sequence of the block that has keys
    for (int i = lane; i < n; i += 64)
      if (s_len[m0 + i] > 0) from = min(from, m0 + i);
    from = wave_min(from);
    if (lane == 0) {
      const int seq = from == INT_MAX ? 0 : a.members != nullptr ? a.members[from] : from;
      v.segs[blk] = Segment{m0, n * a.g, n, P, 0, 0, 0, seq};
    }
  }
  // the members' own keys
  for (int c0 = 0; c0 < a.B; c0 += kPlThreads) {
    const int i = c0 + tid;
    int gi = -1, len = -1, P = 0, near = 0, G = 1, n_rem = 0, t0 = 0, tiles = 0;
    unsigned long long cnt = 0;
    if (i < a.B) {
      gi = group_of(i);
      len = s_len[i];
      if (gi >= 0 && len > 0) {
        P = s_pre[gi];
        G = plan_group(a, len);
        near = first_local(G, len, a.w0);
        tiles = (len - P + kShTile - 1) / kShTile;
        n_rem = near > P ? (near - P + kShTile - 1) / kShTile : 0;
        t0 = max(near - P, 0) / kShTile;
        cnt = (n_rem > 0) + (t0 < tiles);
      }
    }
    unsigned long long tot;
    const unsigned long long incl = plan_scan(cnt, s_scan, &tot);
    if (i < a.B) {
      const int seg = n_blocks + i;
      Phase* p = v.phases + at + (int)(incl - cnt);
      if (cnt > 0) {
        if (n_rem > 0) put_phase(p++, seg, G, P, n_rem, a.g, len);
        if (t0 < tiles) put_phase(p, seg, 0, P + t0 * kShTile, tiles - t0, a.g, len);
      }
      Member m;
      m.seq = gi >= 0 && len >= 0 ? (a.members != nullptr ? a.members[i] : i) : -1;
      m.len = max(len, 0);
      v.segs[seg] = Segment{i, cnt > 0 ? a.g : 0, 1, len, 0, 0, 0, m.seq};
      m.pre = P > 0 ? s_blk[gi] + (i - s_start[gi]) / per_block : -1;
      m.suf = cnt > 0 ? seg : -1;
      v.members[i] = m;
    }
    at += (int)tot;
  }
  const int n_phases = at;
  __syncthreads();
  // costs before each phase
  unsigned long long total = 0;
  for (int c0 = 0; c0 < n_phases; c0 += kPlThreads) {
    const int i = c0 + tid;
    unsigned long long x = 0;
    if (i < n_phases) x = kPhaseCost + (unsigned long long)v.phases[i].n * v.phases[i].cost;
    unsigned long long tot;
    const unsigned long long incl = plan_scan(x, s_scan, &tot);
    if (i < n_phases) {
      const unsigned long long st = total + incl - x;
      v.phases[i].start_lo = (uint32_t)st;
      v.phases[i].start_hi = (uint32_t)(st >> 32);
    }
    total += tot;
  }
  // ranges that hold a tile wherever they lie inside a segment
  const unsigned long long most = total / kMaxStep;
  const int n_wg = total == 0 ? 0 : (int)max(1ull, min((unsigned long long)a.n_wg, most));
  __syncthreads();
  auto owner = [&](unsigned long long x) {  // the workgroup whose range holds x
    int w = (int)min((unsigned long long)(n_wg - 1), (unsigned long long)((double)x * n_wg / (double)total));
    while (w > 0 && total * w / n_wg > x) --w;
    while (w + 1 < n_wg && total * (w + 1) / n_wg <= x) ++w;
    return w;
  };
  for (int i = tid; i < n_phases; i += kPlThreads) {
    const Phase p = v.phases[i];
    const unsigned long long st = p.start_lo | (unsigned long long)p.start_hi << 32;
    const unsigned long long end = st + kPhaseCost + (unsigned long long)p.n * p.cost;
    // the workgroups whose ranges begin inside this phase
    int w = owner(st);
    if (total * w / n_wg < st) ++w;
    for (; w < n_wg && total * w / n_wg < end; ++w) v.wg_first[w] = i;
    if (i == 0 || v.phases[i - 1].seg != p.seg) v.segs[p.seg].w_first = owner(st + kPhaseCost);
    if (i == n_phases - 1 || v.phases[i + 1].seg != p.seg) v.segs[p.seg].n_w = owner(end - p.cost);
  }
  __syncthreads();
  int rows = 0;
  for (int c0 = 0; c0 < n_blocks + a.B; c0 += kPlThreads) {
    const int i = c0 + tid;
    unsigned long long x = 0;
    int n_w = 0;
    if (i < n_blocks + a.B && v.segs[i].rows > 0) {
      n_w = v.segs[i].n_w - v.segs[i].w_first + 1;
      x = (unsigned long long)n_w * v.segs[i].rows;
    }
    unsigned long long tot;
    const unsigned long long incl = plan_scan(x, s_scan, &tot);
    if (i < n_blocks + a.B) {
      v.segs[i].n_w = n_w;
      v.segs[i].row0 = rows + (int)(incl - x);
    }
    rows += (int)tot;
  }
  if (tid == 0) {
    v.header[kHdPhases] = n_phases;
    v.header[kHdWg] = n_wg;
    v.header[kHdTotLo] = (int)(uint32_t)total;
    v.header[kHdTotHi] = (int)(uint32_t)(total >> 32);
    v.header[kHdRows] = rows;
    v.header[kHdB] = a.B;
    v.header[kHdG] = a.g;
    v.header[kHdPage] = a.page;
    v.header[kHdMaxPages] = a.max_pages;
    v.header[kHdHkv] = a.Hkv;
    v.header[kHdGroups] = a.n_groups;
    v.header[kHdBifocal] = a.bifocal;
    v.header[kHdWPre] = a.w_pre;
    v.header[kHdW0] = a.w0;
  }
}

// ------------------------------------------------------------------ decode
struct SharedArgs {
  const uint16_t* q;
  const uint16_t* k;
  const uint16_t* v;
  const int32_t* table;
  uint16_t* o;
  const float2* rope;
  const uint32_t* rope16;
  void* plan;
  float* states;
  int B, n_groups, Hq, Hkv, g, max_pages, n_pages, page, page_shift, n_wg;
  int bifocal, w_pre, w0;
  float q_scale;
};

// Whether the plan is one for this call: else nothing is computed.
__device__ inline bool plan_fits(const SharedArgs& a, const int* h) {
  return h[kHdB] == a.B && h[kHdG] == a.g && h[kHdPage] == a.page && h[kHdMaxPages] == a.max_pages &&
         h[kHdHkv] == a.Hkv && h[kHdGroups] == a.n_groups && h[kHdBifocal] == a.bifocal &&
         h[kHdWPre] == a.w_pre && h[kHdW0] == a.w0 && h[kHdWg] <= a.n_wg;
}

// LDS layouts: K key r at r * 256, its 16-byte chunk c in slot c ^ sh_kswz(r); V as
// the prefill kernel's tiles; cos/sin row of key r at r * 256.
__device__ inline int sh_kswz(int r) { return ((r & 15) >> 1) | ((r & 1) << 3); }
__device__ inline int sh_koff(int r, int c) { return r * 256 + 16 * (c ^ sh_kswz(r)); }
__device__ inline int sh_voff(int r, int c) { return r * 256 + 16 * (c ^ (4 * (r & 3))); }

// A tile of the list
struct Tile {
  int row0, row1;  // pool rows of its first and its 17th key
  int k0;
  int flags;  // bits 0..4: last valid key of the tile; kTf*; the phase from bit 9 on
  int f0, km;      // remote view: f(k0) and k0 - G f(k0)
  uint32_t m, l;
};
constexpr int kTfRemote = 32, kTfView = 64, kTfSeg = 128, kTfLast = 256, kTfPhase = 9;

// The slice of fp32 head row `row` that a lane feeds as B operand: as the prefill's.
__device__ inline void sh_load_q(const uint16_t* qrow, int half, const float2* table, int pos,
                                 float scale, bf16x8* out) {
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    const int d = 16 * s + 8 * half;
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
    out[s] = pack8(ylo);
    out[s + 4] = pack8(yhi);
  }
}

typedef __bf16 sh_bf16x2 __attribute__((ext_vector_type(2)));

// Scores may exceed the row's reference by this (log2 units) before it moves: weights
// stay below 2^16, far inside fp32 and bf16.
constexpr float kShSlack = 16.f;

__global__ __launch_bounds__(kShThreads, 2) void decode_shared_kernel(SharedArgs a) {
  __shared__ __attribute__((aligned(1024))) unsigned char smem[kShBufs * kShBuf];
  __shared__ __attribute__((aligned(16))) Tile s_tiles[kShList];
  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int hl32 = lane >> 5;
  const int h = blockIdx.x % a.Hkv;
  const int w = blockIdx.x / a.Hkv;
  const PlanView pv = plan_view(a.plan, a.B, a.n_groups, a.g);
  if (!plan_fits(a, pv.header) || w >= pv.header[kHdWg]) return;
  const int n_phases = pv.header[kHdPhases], n_wg = pv.header[kHdWg];
  const unsigned long long total =
      (uint32_t)pv.header[kHdTotLo] | (unsigned long long)(uint32_t)pv.header[kHdTotHi] << 32;
  const unsigned long long x0 = total * w / n_wg, x1 = total * (w + 1) / n_wg;
  const uint32_t smem_base = lds_addr(smem);
  const uint32_t kv_row_bytes = (uint32_t)a.Hkv * (kHeadDim * 2);
  const unsigned char* kbase = (const unsigned char*)(a.k + (size_t)h * kHeadDim);
  const unsigned char* vbase = (const unsigned char*)(a.v + (size_t)h * kHeadDim);

  // tiles [ta, tb) of a phase that this workgroup holds
  auto tiles_of = [&](const Phase& p, int* ta, int* tb) {
    const unsigned long long st = (p.start_lo | (unsigned long long)p.start_hi << 32) + kPhaseCost;
    auto below = [&](unsigned long long x) {
      return x <= st ? 0 : (int)min((unsigned long long)p.n, (x - st + p.cost - 1) / p.cost);
    };
    *ta = below(x0);
    *tb = below(x1);
  };

  // ---- copies of a tile: keys 4 wave .. + 3 of K, V and their cos/sin rows
  const int cp_key = 4 * wave + (lane >> 4), cp_slot = lane & 15;
  const uint32_t cp_k = 16 * (cp_slot ^ sh_kswz(cp_key));
  const uint32_t cp_v = 16 * (cp_slot ^ (4 * (cp_key & 3)));
  auto uni = [](int x) { return __builtin_amdgcn_readfirstlane(x); };
  auto issue = [&](int j) __attribute__((always_inline)) {
    const Tile& s = s_tiles[j];
    const int flags = uni(s.flags), klim = flags & 31, k0 = uni(s.k0);
    const int row = min(4 * wave, klim) < 16 ? uni(s.row0) : uni(s.row1);
    const int key = min(cp_key, klim);
    const size_t off = (size_t)(uint32_t)row * kv_row_bytes;
    const uint32_t buf = smem_base + (uint32_t)(j % kShBufs) * kShBuf + 1024 * wave;
    const uint32_t ro = (uint32_t)(key & 15) * kv_row_bytes;
    dma16_s_nt(kbase + off, ro + cp_k, buf);
    dma16_s_nt(vbase + off, ro + cp_v, buf + kShImg);
    int pos = k0 + key;
    if (flags & kTfRemote) {
      const FastDiv f = {(uint32_t)uni((int)s.m), (uint32_t)uni((int)s.l), 2};
      pos = uni(s.f0) + (int)fastdiv_ge2((uint32_t)(uni(s.km) + key), f);
    }
    dma16_s(a.rope16, (uint32_t)pos * 256 + 16 * cp_slot, buf + 2 * kShImg);
  };
  // Rotation of this wave's four keys, in place: lane -> key, a chunk pair's half
  const int rt_key = 4 * wave + (lane >> 4), rt_c = (lane >> 1) & 7, rt_h = lane & 1;
  const int rt_lo = sh_koff(rt_key, rt_c) + 8 * rt_h, rt_hi = sh_koff(rt_key, rt_c + 8) + 8 * rt_h;
  const int rt_cs = 2 * kShImg + rt_key * 256 + 32 * rt_c + 16 * rt_h;
  auto rotate = [&](int j) __attribute__((always_inline)) {
    unsigned char* b = smem + (j % kShBufs) * kShBuf;
    typedef unsigned u32x2v __attribute__((ext_vector_type(2)));
    const u32x2v xl = *(const u32x2v*)(b + rt_lo), xh = *(const u32x2v*)(b + rt_hi);
    const u32x4 cs = *(const u32x4*)(b + rt_cs);
    uint32_t l0, h0, l1, h1;
    rot_word_dot2(xl[0], xh[0], cs[0], cs[1], l0, h0);
    rot_word_dot2(xl[1], xh[1], cs[2], cs[3], l1, h1);
    *(u32x2v*)(b + rt_lo) = u32x2v{l0, l1};
    *(u32x2v*)(b + rt_hi) = u32x2v{h0, h1};
  };

  // ---- state of this lane's row
  bf16x8 qop[8];
  f32x16 acc_o[4];
  f32x16 neg_m = f32x16{};
  float m_ref = 0.f, l_run = 0.f;
  int rows = 0, kend = 0;              // of the segment
  int lim = 0, row_G = 1, qpos = 0;    // of the row: first key in its base view, G, position
  const uint16_t* qrow = a.q;
  int ph_G = 0;                        // the phase's view
#pragma unroll
  for (int i = 0; i < 4; ++i) acc_o[i] = f32x16{};
#pragma unroll
  for (int s = 0; s < 8; ++s) qop[s] = bf16x8{};
  const int row = 32 * wave + (lane & 31);
  const int kr_lane = lane & 31;
  const int vk_lane = 4 * hl32 + ((lane & 15) >> 2);
  const int vc_lane = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);

  int ph = pv.wg_first[w];  // next phase of the list, and its first tile that is not listed yet
  int ph_t = -1;
  int seg_now = -1;         // the segment of the last listed tile
  while (ph < n_phases) {
    // ---- list the next tiles of the range
    int n = 0;
    while (ph < n_phases && n < kShList) {
      const Phase p = pv.phases[ph];
      int ta, tb;
      tiles_of(p, &ta, &tb);
      if ((p.start_lo | (unsigned long long)p.start_hi << 32) >= x1) {
        ph = n_phases;
        break;
      }
      const bool first = ph_t < 0;  // of the phase, here
      const int t0 = first ? ta : ph_t;
      const int cnt = min(tb - t0, kShList - n);
      if (cnt > 0) {
        const int32_t* bt = a.table + (size_t)pv.segs[p.seg].seq * a.max_pages;
        const FastDiv f = {p.m, p.l, (uint32_t)p.G};
        for (int i = tid; i < cnt; i += kShThreads) {
          Tile s;
          s.k0 = p.k0 + (t0 + i) * kShTile;
          const int klim = min(kShTile - 1, p.kend - 1 - s.k0);
          auto pool_row = [&](int k) {
            const int pg = min(max(bt[k >> a.page_shift], 0), a.n_pages - 1);
            return (pg << a.page_shift) + (k & (a.page - 1));
          };
          s.row0 = pool_row(s.k0);
          s.row1 = klim >= 16 ? pool_row(s.k0 + 16) : s.row0;
          const bool fl = first && i == 0;  // the phase's first tile of this workgroup
          s.flags = klim | (p.G > 0 ? kTfRemote : 0) | (fl ? kTfView : 0) |
                    (fl && p.seg != seg_now ? kTfSeg : 0) | ph << kTfPhase;
          s.f0 = p.G > 0 ? (int)fastdiv((uint32_t)s.k0, f) : 0;
          s.km = p.G > 0 ? s.k0 - p.G * s.f0 : 0;
          s.m = p.m;
          s.l = p.l;
          // the last tile here of its segment: the next phase is another segment's, or lies
          // behind the range
          if (t0 + i == tb - 1) {
            bool last = true;
            if (tb == p.n && ph + 1 < n_phases) {
              const Phase nx = pv.phases[ph + 1];
              int na, nb;
              tiles_of(nx, &na, &nb);
              last = nx.seg != p.seg || nb <= na;
            }
            if (last) s.flags |= kTfLast;
          }
          s_tiles[n + i] = s;
        }
        seg_now = p.seg;
        n += cnt;
      }
      if (t0 + cnt < tb) {
        ph_t = t0 + cnt;
      } else {
        ph_t = -1;
        ++ph;
      }
    }
    __syncthreads();
    if (n == 0) break;

    // ---- stream them
    const int n_first = min(n, kShAhead);
    for (int j = 0; j < n_first; ++j) issue(j);
    if (n_first >= 5)
      wait_vmem_n<4 * kShCopies>();
    else
      wait_vmem();
    rotate(0);
    for (int i = 0; i < n; ++i) {
      // this wave's copies of tile i + 1 have landed; the next three may fly
      if (i + 4 < n)
        wait_vmem_n<3 * kShCopies>();
      else if (i + 3 < n)
        wait_vmem_n<2 * kShCopies>();
      else if (i + 2 < n)
        wait_vmem_n<kShCopies>();
      else
        wait_vmem();
      __syncthreads();  // tile i is rotated everywhere, tile i - 1 used by all
      if (i + kShAhead < n) issue(i + kShAhead);
      if (i + 1 < n) rotate(i + 1);
      const int flags = uni(s_tiles[i].flags), k0 = uni(s_tiles[i].k0);
      if (flags & kTfView) {
        const Phase p = pv.phases[flags >> kTfPhase];
        ph_G = p.G;
        if (flags & kTfSeg) {
          const Segment sg = pv.segs[p.seg];
          rows = sg.rows;
          kend = sg.kend;
          const int r = min(row, rows - 1);
          const Member mb = pv.members[sg.m0 + r / a.g];
          qpos = max(mb.len - 1, 0);
          row_G = a.bifocal ? group_size(mb.len, a.w_pre) : 1;
          lim = first_local(row_G, mb.len, a.w0);
          qrow = a.q + ((size_t)max(mb.seq, 0) * a.Hq + h * a.g + r % a.g) * kHeadDim;
#pragma unroll
          for (int d = 0; d < 4; ++d) acc_o[d] = f32x16{};
          neg_m = f32x16{};
          m_ref = 0.f;
          l_run = 0.f;
        }
        if (32 * wave < rows)
          sh_load_q(qrow, hl32, a.rope, ph_G > 0 ? qpos / row_G : qpos, a.q_scale, qop);
      }
      if (32 * wave >= rows) continue;
      const unsigned char* kb = smem + (i % kShBufs) * kShBuf;
      const unsigned char* vb = kb + kShImg;
      // S^T = K Q^T - m
      f32x16 sc;
      {
        bf16x8 ring[4];
#pragma unroll
        for (int s = 0; s < 4; ++s) ring[s] = *(const bf16x8*)(kb + sh_koff(kr_lane, 2 * s + hl32));
        sc = neg_m;
#pragma unroll
        for (int s = 0; s < 8; ++s) {
          sc = mfma32(ring[s & 3], qop[s], sc);
          if (s + 4 < 8) ring[s & 3] = *(const bf16x8*)(kb + sh_koff(kr_lane, 2 * (s + 4) + hl32));
        }
      }
      auto vop = [&](int m) __attribute__((always_inline)) {
        const unsigned char* p = vb + 4096 * (m >> 2) + sh_voff(vk_lane, 4 * (m & 3) + vc_lane) + 8 * (lane & 1);
        return concat_tr(lds_read_tr4(p), lds_read_tr4(p + 2048));
      };
      bf16x8 vr[4];
#pragma unroll
      for (int m = 0; m < 4; ++m) vr[m] = vop(m);
      // keep the keys [lo, hi) of the tile: in the remote view those before the row's
      // first local key, where its G is the phase's, else those from it on
      int lo = 0, hi = kend - k0;
      if (ph_G > 0)
        hi = row_G == ph_G ? min(hi, lim - k0) : 0;
      else
        lo = lim - k0;
      if (__ballot(lo > 0 || hi < kShTile) != 0) {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int t = 8 * (e >> 2) + (e & 3) + 4 * hl32;
          sc[e] = t >= lo && t < hi ? sc[e] : -INFINITY;
        }
      }
      float mt = fmaxf(sc[0], sc[1]);
#pragma unroll
      for (int e = 2; e < 16; e += 2) mt = fmaxf(mt, fmaxf(sc[e], sc[e + 1]));
      {
        typedef unsigned u32x2v __attribute__((ext_vector_type(2)));
        const u32x2v r =
            __builtin_amdgcn_permlane32_swap(__float_as_uint(mt), __float_as_uint(mt), false, false);
        mt = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
      }
      // the reference follows the first keys of a row, and scores far above it
      const float l_both = l_run;  // zero in both lanes of the row or in neither, see below
      const bool upd = mt != -INFINITY && (mt > kShSlack || l_both == 0.f);
      if (__ballot(upd) != 0) {
        const float shift = upd ? mt : 0.f;
        const float alpha = l_both == 0.f ? 1.f : fast_exp2(-shift);
#pragma unroll
        for (int e = 0; e < 16; ++e) sc[e] -= shift;
#pragma unroll
        for (int d = 0; d < 4; ++d) acc_o[d] *= alpha;
        l_run *= alpha;
        m_ref += shift;
#pragma unroll
        for (int e = 0; e < 16; ++e) neg_m[e] = -m_ref;
      }
      bf16x8 pb[2];
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
      // both lanes of a row add the row's whole sum, so that l_run says in either
      // whether the row has a key
      float ps = ps0 + ps1;
      {
        typedef unsigned u32x2v __attribute__((ext_vector_type(2)));
        const u32x2v r =
            __builtin_amdgcn_permlane32_swap(__float_as_uint(ps), __float_as_uint(ps), false, false);
        ps = __uint_as_float(r[0]) + __uint_as_float(r[1]);
      }
      l_run += ps;
#pragma unroll
      for (int m = 0; m < 8; ++m) {
        acc_o[m & 3] = mfma32(vr[m & 3], pb[m >> 2], acc_o[m & 3]);
        if (m + 4 < 8) vr[m & 3] = vop(m + 4);
      }
      if ((flags & kTfLast) && row < rows) {
        const Phase p = pv.phases[flags >> kTfPhase];
        const Segment sg = pv.segs[p.seg];
        float* st = a.states + ((size_t)h * pv.header[kHdRows] + sg.row0 + (size_t)(w - sg.w_first) * rows) *
                                   kShStateFloats;
#pragma unroll
        for (int db = 0; db < 4; ++db) {
#pragma unroll
          for (int q4 = 0; q4 < 4; ++q4) {
            f32x4 t;
#pragma unroll
            for (int jj = 0; jj < 4; ++jj) t[jj] = acc_o[db][4 * q4 + jj];
            *(f32x4*)(st + ((size_t)(8 * db + 2 * q4 + hl32) * rows + row) * 4) = t;
          }
        }
        if (hl32 == 0) *(float2*)(st + (size_t)rows * kHeadDim + 2 * row) = make_float2(m_ref, l_run);
      }
    }
    __syncthreads();  // the list and the buffers are free
  }
}

// The states of a row, joined: O = sum 2^(m - M) O~ / sum 2^(m - M) l.  Workgroup: 8
// rows of one kv head in member order; thread -> row, 4 channels, every other state.
constexpr int kMgRows = 8;
__global__ __launch_bounds__(512) void merge_shared_kernel(SharedArgs a) {
  __shared__ f32x4 s_o[32][kMgRows];
  __shared__ float2 s_ml[32][kMgRows];
  const PlanView pv = plan_view(a.plan, a.B, a.n_groups, a.g);
  if (!plan_fits(a, pv.header)) return;
  const int h = blockIdx.y;
  const int rl = threadIdx.x & (kMgRows - 1), c = (threadIdx.x / kMgRows) & 31, half = threadIdx.x >> 8;
  const int r = blockIdx.x * kMgRows + rl;
  const int mi = min(r / a.g, a.B - 1);
  const Member mb = pv.members[mi];
  const bool on = r < a.B * a.g && mb.seq >= 0;
  float M = -INFINITY, den = 0.f;
  f32x4 acc = f32x4{};
  const float* base = a.states + (size_t)h * pv.header[kHdRows] * kShStateFloats;
  auto join = [&](int seg, bool prefix) {
    if (seg < 0) return;
    const Segment sg = pv.segs[seg];
    const int at = prefix ? r - sg.m0 * a.g : r % a.g;
    for (int i = half; i < sg.n_w; i += 2) {
      const float* st = base + (size_t)(sg.row0 + i * sg.rows) * kShStateFloats;
      const float2 ml = *(const float2*)(st + (size_t)sg.rows * kHeadDim + 2 * at);
      const f32x4 x = *(const f32x4*)(st + ((size_t)c * sg.rows + at) * 4);
      if (ml.y == 0.f) continue;  // no key of this row
      const float m = fmaxf(M, ml.x);
      const float wa = M == -INFINITY ? 0.f : fast_exp2(M - m), wb = fast_exp2(ml.x - m);
      den = wa * den + wb * ml.y;
      acc = wa * acc + wb * x;
      M = m;
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
  if (half == 1 || !on) return;
  const float2 ml = s_ml[c][rl];
  const float top = fmaxf(M, ml.x);
  f32x4 out = f32x4{};
  if (top != -INFINITY) {
    const float wa = M == -INFINITY ? 0.f : fast_exp2(M - top);
    const float wb = ml.x == -INFINITY ? 0.f : fast_exp2(ml.x - top);
    out = (wa * acc + wb * s_o[c][rl]) * (1.f / (wa * den + wb * ml.y));
  }
  *(bf16x4*)(a.o + ((size_t)mb.seq * a.Hq + h * a.g + r % a.g) * kHeadDim + 4 * c) =
      __builtin_convertvector(out, bf16x4);
}

// ---------------------------------------------------------------- launchers
hipError_t launch_shared_plan(bool bifocal, const int32_t* kv_lens, const int32_t* members,
                              const int32_t* group_starts, const int32_t* shared, int B,
                              int n_groups, int Hq, int Hkv, int max_pages, int page, int w_pre,
                              int w0, int n_cu, void* plan, hipStream_t stream) {
  SharedPlanArgs a{kv_lens, members, group_starts, shared, plan, B, n_groups, Hq / Hkv, Hkv,
                   max_pages, page, head_workgroups(n_cu, Hkv), bifocal ? 1 : 0, w_pre, w0};
  const size_t lds = ((size_t)B + 3 * n_groups + 2 + plan_blocks(B, n_groups, a.g) + 1) * sizeof(int);
  hipLaunchKernelGGL(shared_plan_kernel, dim3(1), dim3(kPlThreads), lds, stream, a);
  return hipGetLastError();
}

hipError_t launch_decode_shared(bool bifocal, const uint16_t* q, const uint16_t* k,
                                const uint16_t* v, const int32_t* table, int max_pages,
                                int n_pages, int page_shift, void* plan, uint16_t* o,
                                const float2* rope, const uint32_t* rope16, int B, int n_groups,
                                int Hq, int Hkv, int w_pre, int w0, int n_cu, void* ws,
                                hipStream_t stream, hipEvent_t ev0, hipEvent_t ev1) {
  SharedArgs a;
  a.q = q;
  a.k = k;
  a.v = v;
  a.table = table;
  a.o = o;
  a.rope = rope;
  a.rope16 = rope16;
  a.plan = plan;
  a.states = (float*)ws;
  a.B = B;
  a.n_groups = n_groups;
  a.Hq = Hq;
  a.Hkv = Hkv;
  a.g = Hq / Hkv;
  a.max_pages = max_pages;
  a.n_pages = n_pages;
  a.page = 1 << page_shift;
  a.page_shift = page_shift;
  a.n_wg = head_workgroups(n_cu, Hkv);
  a.bifocal = bifocal ? 1 : 0;
  a.w_pre = w_pre;
  a.w0 = w0;
  a.q_scale = 1.4426950408889634f / sqrtf((float)kHeadDim);
  hipError_t e = hipSuccess;
  if (ev0 != nullptr && (e = hipEventRecord(ev0, stream)) != hipSuccess) return e;
  hipLaunchKernelGGL(decode_shared_kernel, dim3((unsigned)a.n_wg * Hkv), dim3(kShThreads), 0, stream, a);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  if (ev1 != nullptr && (e = hipEventRecord(ev1, stream)) != hipSuccess) return e;
  hipLaunchKernelGGL(merge_shared_kernel,
                     dim3((unsigned)((B * a.g + kMgRows - 1) / kMgRows), (unsigned)Hkv), dim3(512), 0,
                     stream, a);
  return hipGetLastError();
}

}  // namespace jl
