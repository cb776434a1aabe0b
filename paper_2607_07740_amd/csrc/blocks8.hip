// blocks8.hip -- which blocks of an 8-bit cache a query attends to: a score per
// block from its mean key, and the choice of the largest.
#include <algorithm>
#include <type_traits>

#include "cache8.h"

namespace jl {

struct ScoresArgs {
  Cache8 c;
  const uint16_t* q;
  const int32_t* kv_lens;
  float* scores;  // [B][Hkv][n_blocks]
  const float2* table;
  int B, Hq, g;
  int n_tiles, n_runs, n_hgroups;  // tiles of 16 blocks, waves that share them, groups of 4 heads
  int w_pre;
  float q_scale;
};

constexpr int kScoreHeads = 4;  // kv heads of a workgroup: one wave each, on the same blocks

// The 16 pairs (x_f, x_{f+64}) of lane group g4: f = 8 g4 + j and 32 + 8 g4 + j, j < 8.
struct Pairs {
  float lo[16], hi[16];
};
__device__ inline void load_pairs(const uint16_t* row, int g4, u32x4* raw) {
#pragma unroll
  for (int i = 0; i < 4; ++i) raw[i] = load16(row + 32 * i + 8 * g4);
}
// ... rotated by the row's cos/sin pairs, in fp32
__device__ inline void rotate_pairs(const u32x4* raw, const float2* cs_row, int g4, Pairs& y) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    float lo[8], hi[8];
    unpack8(raw[i], lo);
    unpack8(raw[2 + i], hi);
    const float4* cs = (const float4*)(cs_row + 32 * i + 8 * g4);
#pragma unroll
    for (int j = 0; j < 8; j += 2) {
      const float4 c = cs[j / 2];
      y.lo[8 * i + j] = lo[j] * c.x - hi[j] * c.y;
      y.hi[8 * i + j] = hi[j] * c.x + lo[j] * c.y;
      y.lo[8 * i + j + 1] = lo[j + 1] * c.z - hi[j + 1] * c.w;
      y.hi[8 * i + j + 1] = hi[j + 1] * c.z + lo[j + 1] * c.w;
    }
  }
}

// NaN above all.
__device__ inline float max_nan(float a, float b) {
  return a != a || b != b ? NAN : fmaxf(a, b);
}
// Four values of each lane, summed over the lanes l, l ^ 16, l ^ 32, l ^ 48: lane group g4 gets
// the g4-th sum.
__device__ inline float sum_of_groups(f32x4 x) {
  auto add = [](u32x2 r) { return __uint_as_float(r[0]) + __uint_as_float(r[1]); };
  auto u = [](float f) { return __float_as_uint(f); };
  const float lo = add(__builtin_amdgcn_permlane32_swap(u(x[0]), u(x[2]), false, false));
  const float hi = add(__builtin_amdgcn_permlane32_swap(u(x[1]), u(x[3]), false, false));
  return add(__builtin_amdgcn_permlane16_swap(u(lo), u(hi), false, false));
}
__device__ inline float max_of_groups(float x) {
  auto most = [](u32x2 r) { return max_nan(__uint_as_float(r[0]), __uint_as_float(r[1])); };
  x = most(__builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false));
  return most(__builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false));
}
// acc += q value n of 32 (n = 4 c + x: of register c, from the lanes with l / 4 % 4 = x) times
// the lane's own m, for the four heads of l % 4.
template <int X>
__device__ inline f32x4 mfma4(float q, float m, f32x4 acc) {
  return __builtin_amdgcn_mfma_f32_4x4x1f32(q, m, acc, 2, X, 0);
}

// score[b][h][j] = max over the group's heads of <R(f(q)) x_q, R(f(64 j + 31)) mean_j>
// / sqrt(d): what the block's middle key would score in the remote view if it were the
// mean.  Blocks past the sequence get -inf.
//
// A wave takes 16 blocks of one kv head at a time: means and queries are rotated in
// fp32 and meet in the fp32 matrix instruction of sixteen 4 x 4 products, so nothing is
// rounded to fewer bits: four blocks and four heads each, and in each lane group another
// quarter of the channels, which are summed at the end.  (The 16 x 16 product leaves half of
// its columns or more without a head.)  The four waves of a workgroup, of four heads, share
// the blocks' cos/sin rows, 512 bytes a block beside its mean's 256, through LDS; means and
// rows are requested one tile ahead, page indices two.  Bound by the chain length -> page ->
// mean at one sequence (131072 tokens, 32/8 heads: 3.9 us, 2.4 of them an empty launch; 4.3
// with 16 x 16 products) and at many by that and a tile's 300 vector instructions (8 of 32K
// to 128K, 64/8 heads: 9.7 to 10.4 us for 21 MB of means; 12.4 with 16 x 16 products, 17 with
// rows through each wave's own loads).  These are times in a captured graph; a trace of single
// kernels shows 4.3 and 10.7.
constexpr int kScoreRow = kHalf + 2;  // float2s of a row in LDS: rows start 4 banks apart
template <bool BIFOCAL, int SETS>  // SETS: of four heads
__global__ __launch_bounds__(64 * kScoreHeads) void block_scores_kernel(ScoresArgs a) {
  __shared__ __attribute__((aligned(16))) float2 rows[2][16][kScoreRow];
  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int i16 = lane & 15, g4 = lane >> 4;
  int w = blockIdx.x;
  const int run = w % a.n_runs;
  w /= a.n_runs;
  const int hg = w % a.n_hgroups, b = w / a.n_hgroups;
  const bool on = hg * kScoreHeads + wave < a.c.Hkv;
  const int h = min(hg * kScoreHeads + wave, a.c.Hkv - 1);
  const int kv_len = min(max(a.kv_lens[b], 0), a.c.n_blocks * kBlk);
  const int n_live = (kv_len + kBlk - 1) / kBlk;
  const int qpos = max(kv_len - 1, 0);
  const uint32_t G = BIFOCAL ? max(1u, (uint32_t)qpos / (uint32_t)a.w_pre + 1) : 1u;
  float* out = a.scores + ((size_t)b * a.c.Hkv + h) * a.c.n_blocks;

  auto block_of = [&](int t, int i) { return min(16 * t + i, max(n_live - 1, 0)); };
  // this thread's half of the cos/sin row of block tid / 16 of a tile
  u32x4 cs0, cs1;
  auto request_rows = [&](int t) __attribute__((always_inline)) {
    const uint32_t mid = (uint32_t)(block_of(t, tid >> 4) * kBlk + kBlk / 2 - 1);
    const u32x4* row = (const u32x4*)(a.table + (size_t)(BIFOCAL ? mid / G : mid) * kHalf);
    cs0 = row[tid & 15];
    cs1 = row[16 + (tid & 15)];
  };
  u32x4 raw[4];
  auto request_mean = [&](int t, int page) __attribute__((always_inline)) {
    const int blk = block_of(t, i16);
    page = min(max(page, 0), a.c.n_pages - 1);
    load_pairs(a.c.k_mean + (size_t)pool_block(a.c, page, h, in_page(a.c, blk)) * kHeadDim, g4, raw);
  };
  int t = run;
  int page = page_of(a.c, b, block_of(t, i16));
  request_rows(t);
  int page_next = page_of(a.c, b, block_of(t + a.n_runs, i16));
  // this lane's share of the queries: value 4 c + x of the 32 of its lane group, of head
  // l % 4 of each set; lanes past the group of heads repeat its last
  float q[SETS][8];
  {
    const int x = (lane >> 2) & 3;
    const float2* cs = a.table + (size_t)(BIFOCAL ? (uint32_t)qpos / G : (uint32_t)qpos) * kHalf;
    uint16_t raw_lo[SETS][4], raw_hi[SETS][4];
    float2 r[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const int f = 32 * (c >> 1) + 8 * g4 + 4 * (c & 1) + x;
      r[c] = cs[f];
#pragma unroll
      for (int s = 0; s < SETS; ++s) {
        const uint16_t* row =
            a.q + ((size_t)b * a.Hq + h * a.g + min(4 * s + (lane & 3), a.g - 1)) * kHeadDim;
        raw_lo[s][c] = row[f];
        raw_hi[s][c] = row[f + kHalf];
      }
    }
    request_mean(t, page);
#pragma unroll
    for (int s = 0; s < SETS; ++s)
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const float lo = bf16_lo(raw_lo[s][c]), hi = bf16_lo(raw_hi[s][c]);
        q[s][c] = lo * r[c].x - hi * r[c].y;
        q[s][4 + c] = hi * r[c].x + lo * r[c].y;
      }
  }
  // the same turns for the whole workgroup
  for (int n = 0; 16 * t < n_live; t += a.n_runs, ++n) {
    u32x4* dst = (u32x4*)rows[n & 1][tid >> 4];
    dst[tid & 15] = cs0;
    dst[16 + (tid & 15)] = cs1;
    __syncthreads();  // one is enough: the other buffer was read in front of it
    Pairs m;
    rotate_pairs(raw, rows[n & 1][i16], g4, m);
    // the rotated means stand here, so that the next tile's loads take the registers of these:
    // in others they would be copied at the loop's end, and waited for there (11.0 -> 10.4 us)
#pragma unroll
    for (int i = 0; i < 16; ++i) asm volatile("" : "+v"(m.lo[i]), "+v"(m.hi[i]));
    request_rows(t + a.n_runs);  // past the end: the last block's again
    request_mean(t + a.n_runs, page_next);
    page_next = page_of(a.c, b, block_of(t + 2 * a.n_runs, i16));
    // four chains of products in turn, each waits for its own last one
    constexpr int kChains = 4 / SETS;  // of a set
    f32x4 acc[SETS][kChains];
#pragma unroll
    for (int s = 0; s < SETS; ++s)
#pragma unroll
      for (int i = 0; i < kChains; ++i) acc[s][i] = f32x4{};
#pragma unroll
    for (int c = 0; c < 8; c += kChains) {
      auto four = [&](auto x) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < kChains; ++i) {
          const int n = 4 * (c + i) + x.value;
          const float mean = n < 16 ? m.lo[n & 15] : m.hi[n & 15];
#pragma unroll
          for (int s = 0; s < SETS; ++s)
            acc[s][i] = mfma4<x.value>(q[s][c + i], mean, acc[s][i]);
        }
      };
      four(std::integral_constant<int, 0>{});
      four(std::integral_constant<int, 1>{});
      four(std::integral_constant<int, 2>{});
      four(std::integral_constant<int, 3>{});
    }
    auto total = [&](int s) {
      f32x4 x = acc[s][0];
#pragma unroll
      for (int i = 1; i < kChains; ++i) x += acc[s][i];
      return sum_of_groups(x);
    };
    // lane: block i16; the lane group's channels, heads 0 .. 3 of a set
    float best = total(0);
    if (SETS > 1) best = max_nan(best, total(SETS - 1));
    best = max_of_groups(best * a.q_scale);
    const int blk = 16 * t + i16;
    if (on && g4 == 0 && blk < a.c.n_blocks) out[blk] = blk < n_live ? best : -INFINITY;
  }
  for (; t < a.n_tiles; t += a.n_runs) {
    const int blk = 16 * t + i16;
    if (on && g4 == 0 && blk < a.c.n_blocks) out[blk] = -INFINITY;
  }
}

// ------------------------------------------------------------------ choice
struct SelectArgs {
  const float* scores;  // [B][Hkv][n_blocks]
  const int32_t* kv_lens;
  int32_t* blocks;  // [B][Hkv][n_select]
  int Hkv, n_blocks, n_select, w0, n_first;
};

typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));  // rows start anywhere

// A score as an unsigned number of the same order: NaN above everything, both zeros equal.
__device__ inline uint32_t order_of(float x) {
  if (x != x) return 0xfffffffeu;
  const uint32_t b = __float_as_uint(x + 0.f);
  return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}

// Most scores share a few values of the first digit: its counts are held four times, the copies
// of a count in different banks (2048 scores: 6.3 -> 5.8 us).
constexpr int kSelCopies = 4, kSelCopy = 256 + 16;

// Workgroup = one row.  The blocks that are always chosen count as the largest number.
// The want-th largest number is found eight bits at a time from counts of that digit
// among the numbers that share the digits so far; then one scan in index order gives
// every chosen block its place, the numbers equal to the last one in turn until the
// list is full.  Every wave reads the counts for itself: one barrier a digit.
// T threads hold R numbers each, side by side; a longer row is read anew for each digit.
// Bound by latency, 2.4 us of it an empty launch: 5.8 to 6.1 us for 2048 scores, one row or 64,
// 9.9 for 8192, 14.6 for 16384 (a million tokens), 120 for 131072.
// The band goes by the length as it is given, even past the row's end.
template <int T, int R>
__global__ __launch_bounds__(T) void select_blocks_kernel(SelectArgs a) {
  __shared__ __attribute__((aligned(16))) int first[kSelCopies * kSelCopy];
  __shared__ __attribute__((aligned(16))) int hist[3][256];
  __shared__ unsigned long long s_sum[T / 64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int b = blockIdx.x / a.Hkv;
  const int kv_len = max(a.kv_lens[b], 0);
  const int nb = (int)min((long long)a.n_blocks, ((long long)kv_len + kBlk - 1) / kBlk);
  const float* row = a.scores + (size_t)blockIdx.x * a.n_blocks;
  int32_t* out = a.blocks + (size_t)blockIdx.x * a.n_select;
  const int want = min(a.n_select, nb);
  for (int i = want + tid; i < a.n_select; i += T) out[i] = -1;
  if (nb <= a.n_select) {
    for (int i = tid; i < nb; i += T) out[i] = i;
    return;
  }
  // the first block that holds a key of the band
  const long long first_key = (long long)kv_len - 1 - a.w0;
  const int band = (int)min((long long)nb, first_key > 0 ? first_key / kBlk : 0LL);
  uint32_t x[R];
  auto load = [&](int j0) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < R; i += 4) {
      const int j = j0 + tid * R + i;
      float s[4];
      if (j + 3 < nb) {
        const f32x4_any v = *(const f32x4_any*)(row + j);
#pragma unroll
        for (int n = 0; n < 4; ++n) s[n] = v[n];
      } else {
#pragma unroll
        for (int n = 0; n < 4; ++n) s[n] = row[min(j + n, nb - 1)];
      }
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        x[i + n] = j + n < a.n_first || j + n >= band ? 0xffffffffu : order_of(s[n]);
        if (j + n >= nb) x[i + n] = 0;  // below every score
      }
    }
  };
  const int tile = T * R;
  load(0);
  for (int i = tid; i < kSelCopies * kSelCopy; i += T) first[i] = 0;
  for (int i = tid; i < 3 * 256; i += T) (&hist[0][0])[i] = 0;
  __syncthreads();
  uint32_t cut = 0;  // the digits of the want-th largest number so far
  int left = want;   // its place among the numbers that share them
#pragma unroll
  for (int d = 0; d < 4; ++d) {
    const int shift = 24 - 8 * d;
    for (int j0 = 0; j0 < nb; j0 += tile) {
      if (nb > tile) load(j0);
#pragma unroll
      for (int i = 0; i < R; ++i)
        if (j0 + tid * R + i < nb && (d == 0 || (x[i] ^ cut) >> (shift + 8 * (d > 0)) == 0))
          atomicAdd(d == 0 ? &first[tid % kSelCopies * kSelCopy + (x[i] >> 24)]
                           : &hist[max(d - 1, 0)][(x[i] >> shift) & 255], 1);
    }
    __syncthreads();
    // counts of this lane's four digits, and how many numbers have a larger one
    int4 n;
    if (d == 0) {
      n = make_int4(0, 0, 0, 0);
#pragma unroll
      for (int c = 0; c < kSelCopies; ++c) {
        const int4 f = *(const int4*)&first[c * kSelCopy + 4 * lane];
        n.x += f.x;
        n.y += f.y;
        n.z += f.z;
        n.w += f.w;
      }
    } else {
      n = *(const int4*)&hist[max(d - 1, 0)][4 * lane];
    }
    int above = n.x + n.y + n.z + n.w;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int y = __shfl_down(above, o);
      if (lane + o < 64) above += y;
    }
    above -= n.x + n.y + n.z + n.w;
    const int c3 = above + n.w, c2 = c3 + n.z, c1 = c2 + n.y, c0 = c1 + n.x;
    const bool mine = above < left && left <= c0;
    const int digit = left <= c3 ? 3 : left <= c2 ? 2 : left <= c1 ? 1 : 0;
    const int over = digit == 3 ? above : digit == 2 ? c3 : digit == 1 ? c2 : c1;
    const int at = __ffsll(__ballot(mine)) - 1;
    cut |= (uint32_t)__shfl(4 * lane + digit, at) << shift;
    left -= __shfl(over, at);
  }
  // ---- places: `left` numbers equal to cut are taken, in index order
  unsigned long long before = 0;  // taken so far and, in the upper word, equal ones so far
  for (int j0 = 0; j0 < nb; j0 += tile) {
    if (nb > tile) load(j0);
    uint32_t n_more = 0, n_same = 0;
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const bool in = j0 + tid * R + i < nb;
      n_more += in && x[i] > cut;
      n_same += in && x[i] == cut;
    }
    unsigned long long sum = (unsigned long long)n_same << 32 | n_more;
    const unsigned long long own = sum;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const unsigned long long y = __shfl_up(sum, o);
      if (lane >= o) sum += y;
    }
    __syncthreads();
    if (lane == 63) s_sum[wave] = sum;
    __syncthreads();
    unsigned long long at = before + sum - own;
#pragma unroll
    for (int i = 0; i < T / 64; ++i) {
      if (i < wave) at += s_sum[i];
      before += s_sum[i];
    }
    int more = (int)(uint32_t)at, same = (int)(at >> 32);
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int j = j0 + tid * R + i;
      if (j >= nb) continue;
      if (x[i] > cut) out[more++ + min(same, left)] = j;
      if (x[i] == cut && same++ < left) out[more + same - 1] = j;
    }
  }
}

// ---------------------------------------------------------------- launchers
int cu_count();

hipError_t launch_block_scores8(bool bifocal, const Cache8& c, const uint16_t* q,
                                const int32_t* kv_lens, float* scores, const float2* table, int B,
                                int Hq, int w_pre, hipStream_t stream) {
  ScoresArgs a{c, q, kv_lens, scores, table, B, Hq, Hq / c.Hkv, 0, 0, 0, w_pre,
               1.f / sqrtf((float)kHeadDim)};
  a.n_tiles = (c.n_blocks + 15) / 16;
  a.n_hgroups = (c.Hkv + kScoreHeads - 1) / kScoreHeads;
  // about two workgroups per CU; a wave rotates its query once for all of its tiles
  const long long rows = (long long)B * a.n_hgroups;
  a.n_runs = (int)std::max(1LL, std::min<long long>(a.n_tiles, (2LL * cu_count() + rows - 1) / rows));
  const long long wgs = rows * a.n_runs;
  if (wgs > 0x7fffffffLL) return hipErrorInvalidConfiguration;
  const dim3 grid((unsigned)wgs), block(64 * kScoreHeads);
#define JL_SCORES(bif, sets) \
  hipLaunchKernelGGL((block_scores_kernel<bif, sets>), grid, block, 0, stream, a)
  if (a.g <= 4) {
    if (bifocal) JL_SCORES(true, 1);
    else JL_SCORES(false, 1);
  } else {
    if (bifocal) JL_SCORES(true, 2);
    else JL_SCORES(false, 2);
  }
#undef JL_SCORES
  return hipGetLastError();
}

hipError_t launch_select_blocks(const float* scores, const int32_t* kv_lens, int32_t* blocks,
                                int B, int Hkv, int n_blocks, int n_select, int w0, int n_first,
                                hipStream_t stream) {
  SelectArgs a{scores, kv_lens, blocks, Hkv, n_blocks, n_select, w0, n_first};
  const dim3 grid((unsigned)(B * Hkv));
#define JL_SELECT(t, r) \
  hipLaunchKernelGGL((select_blocks_kernel<t, r>), grid, dim3(t), 0, stream, a)
  // The smallest that holds a row: 2048 scores 5.8 us with (512, 4), 6.6 with (256, 8); 4096 7.0
  // with (512, 8), 7.7 with (1024, 4), 9.0 with (1024, 8); 8192 9.9 with (1024, 8), 10.3 with
  // (512, 16); 16384 14.5 with (1024, 16), 16.6 with (512, 32), 20.4 with (1024, 8).
  if (n_blocks <= 512 * 4) JL_SELECT(512, 4);
  else if (n_blocks <= 512 * 8) JL_SELECT(512, 8);
  else if (n_blocks <= 1024 * 8) JL_SELECT(1024, 8);
  else JL_SELECT(1024, 16);
#undef JL_SELECT
  return hipGetLastError();
}

}  // namespace jl
