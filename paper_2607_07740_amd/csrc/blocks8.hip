// blocks8.hip -- which blocks of an 8-bit cache a query attends to: a score per
// block from its mean key, and the choice of the largest.
#include "cache8.h"

namespace jl {

struct ScoresArgs {
  Cache8 c;
  const uint16_t* q;
  const int32_t* kv_lens;
  float* scores;  // [B][Hkv][n_blocks]
  const float2* table;
  int B, Hq, g;
  int w_pre;
  float q_scale;
};

// score[b][h][j] = max over the group's heads of <R(f(q)) x_q, R(f(64 j + 31)) mean_j>
// / sqrt(d): what the block's middle key would score in the remote view if it were the
// mean.  Blocks past the sequence get -inf.
template <bool BIFOCAL>
__global__ __launch_bounds__(256) void block_scores_kernel(ScoresArgs a) {
  __shared__ float sq[8][kHeadDim];
  const int tid = threadIdx.x;
  const int n_wg = (a.c.n_blocks + 255) / 256;
  const int bh = blockIdx.x / n_wg, part = blockIdx.x - bh * n_wg;
  const int b = bh / a.c.Hkv, h = bh - b * a.c.Hkv;
  const int kv_len = min(max(a.kv_lens[b], 0), a.c.n_blocks * kBlk);
  const int qpos = max(kv_len - 1, 0);
  const FastDiv gdiv = make_fastdiv(BIFOCAL ? group_size(max(kv_len, 1), a.w_pre) : 1);
  for (int i = tid; i < a.g * kHalf; i += 256) {
    const int j = i >> 6, f = i & 63;
    const uint16_t* q = a.q + ((size_t)b * a.Hq + h * a.g + j) * kHeadDim;
    const float lo = __uint_as_float((uint32_t)q[f] << 16) * a.q_scale;
    const float hi = __uint_as_float((uint32_t)q[f + 64] << 16) * a.q_scale;
    const float2 cs = a.table[(size_t)remote_pos(qpos, gdiv) * kHalf + f];
    sq[j][f] = lo * cs.x - hi * cs.y;
    sq[j][f + 64] = hi * cs.x + lo * cs.y;
  }
  __syncthreads();
  const int blk = part * 256 + tid;
  if (blk >= a.c.n_blocks) return;
  float best = -INFINITY;
  if (blk * kBlk < kv_len) {
    const int page = min(max(page_of(a.c, b, blk), 0), a.c.n_pages - 1);
    const uint16_t* mean =
        a.c.k_mean + (size_t)pool_block(a.c, page, h, in_page(a.c, blk)) * kHeadDim;
    const int mid = remote_pos(blk * kBlk + kBlk / 2 - 1, gdiv);
    float sc[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) sc[j] = 0.f;
    for (int f = 0; f < kHalf; ++f) {
      const float x = __uint_as_float((uint32_t)mean[f] << 16);
      const float y = __uint_as_float((uint32_t)mean[f + 64] << 16);
      const float2 cs = a.table[(size_t)mid * kHalf + f];
      const float lo = x * cs.x - y * cs.y, hi = y * cs.x + x * cs.y;
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (j < a.g) sc[j] += lo * sq[j][f] + hi * sq[j][f + 64];
    }
    bool nan = false;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (j >= a.g) continue;
      best = fmaxf(best, sc[j]);
      nan |= sc[j] != sc[j];
    }
    if (nan) best = NAN;
  }
  a.scores[(size_t)bh * a.c.n_blocks + blk] = best;
}

struct SelectArgs {
  const float* scores;  // [B][Hkv][n_blocks]
  const int32_t* kv_lens;
  int32_t* blocks;  // [B][Hkv][n_select]
  int Hkv, n_blocks, n_select, w0, n_first;
};

// A score as an unsigned number of the same order: NaN above everything, both zeros equal.
__device__ inline uint32_t order_of(float x) {
  if (x != x) return 0xfffffffeu;
  const uint32_t b = __float_as_uint(x + 0.f);
  return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}

// Workgroup = one row.  The blocks that are always chosen count as the largest
// number; the n-th largest number is found bit by bit.
__global__ __launch_bounds__(256) void select_blocks_kernel(SelectArgs a) {
  __shared__ int s_n[4];
  const int tid = threadIdx.x, wave = tid >> 6;
  const int b = blockIdx.x / a.Hkv;
  const int kv_len = max(a.kv_lens[b], 0);
  const int nb = (int)min((long long)a.n_blocks, ((long long)kv_len + kBlk - 1) / kBlk);
  const float* row = a.scores + (size_t)blockIdx.x * a.n_blocks;
  int32_t* out = a.blocks + (size_t)blockIdx.x * a.n_select;
  auto value = [&](int j) {
    const bool always = j < a.n_first || (long long)j * kBlk + kBlk - 1 >= (long long)kv_len - 1 - a.w0;
    return always ? 0xffffffffu : order_of(row[j]);
  };
  auto total = [&](int n) {
    for (int o = 1; o < 64; o <<= 1) n += __shfl_xor(n, o);
    __syncthreads();
    if ((tid & 63) == 0) s_n[wave] = n;
    __syncthreads();
    return s_n[0] + s_n[1] + s_n[2] + s_n[3];
  };
  const int want = min(a.n_select, nb);
  uint32_t cut = 0;  // the largest number that at least `want` blocks reach
  for (int bit = 31; bit >= 0; --bit) {
    const uint32_t t = cut | (1u << bit);
    int n = 0;
    for (int j = tid; j < nb; j += 256) n += value(j) >= t ? 1 : 0;
    if (total(n) >= want) cut = t;
  }
  int above = 0;
  for (int j = tid; j < nb; j += 256) above += value(j) > cut ? 1 : 0;
  above = total(above);
  if (tid < 64) {  // one wave writes the list in order
    int n = 0, ties = want - above;
    for (int j0 = 0; j0 < nb; j0 += 64) {
      const int j = j0 + tid;
      const uint32_t x = j < nb ? value(j) : 0;
      const bool tie = j < nb && x == cut;
      const unsigned long long below = (1ull << tid) - 1;
      const unsigned long long mt = __ballot(tie);
      const bool take = j < nb && (x > cut || (tie && __popcll(mt & below) < ties));
      const unsigned long long mk = __ballot(take);
      if (take) out[n + __popcll(mk & below)] = j;
      n += __popcll(mk);
      ties -= min(ties, (int)__popcll(mt));
    }
    for (int i = n + tid; i < a.n_select; i += 64) out[i] = -1;
  }
}

// ---------------------------------------------------------------- launchers
hipError_t launch_block_scores8(bool bifocal, const Cache8& c, const uint16_t* q,
                                const int32_t* kv_lens, float* scores, const float2* table, int B,
                                int Hq, int w_pre, hipStream_t stream) {
  ScoresArgs a{c, q, kv_lens, scores, table, B, Hq, Hq / c.Hkv, w_pre,
               1.f / sqrtf((float)kHeadDim)};
  const long long wgs = (long long)B * c.Hkv * ((c.n_blocks + 255) / 256);
  if (wgs > 0x7fffffffLL) return hipErrorInvalidConfiguration;
  if (bifocal)
    hipLaunchKernelGGL(block_scores_kernel<true>, dim3((unsigned)wgs), dim3(256), 0, stream, a);
  else
    hipLaunchKernelGGL(block_scores_kernel<false>, dim3((unsigned)wgs), dim3(256), 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_select_blocks(const float* scores, const int32_t* kv_lens, int32_t* blocks,
                                int B, int Hkv, int n_blocks, int n_select, int w0, int n_first,
                                hipStream_t stream) {
  SelectArgs a{scores, kv_lens, blocks, Hkv, n_blocks, n_select, w0, n_first};
  hipLaunchKernelGGL(select_blocks_kernel, dim3((unsigned)B * Hkv), dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace jl
