// cache8.h -- the 8-bit cache: blocks of 64 tokens of one kv head, e4m3 values
// with one power-of-two scale, in the order the decode kernel's matrix
// instructions take them.
//
//   K image of a block: key 32 a + 16 t + r, channel 64 p + 32 u + 8 g + j at
//     [a 2][t 2][u 2][g 4][r 16][j 8][p 2]: 16 bytes are 8 rotate-half pairs of
//     one key, and 64 lanes (r, g) read 1 KB of a 16-key operand in one go.
//   V image: key 32 a + 16 t + 4 g + i, channel 32 c + 16 e + m at
//     [a 2][c 4][g 4][m 16][e 2][t 2][i 4]: 16 bytes are 8 keys at two channels,
//     the keys whose probabilities lane group g holds after a 16 x 16 score tile.
// So a wave loads either one straight into its registers, 16 bytes a lane, and
// no byte passes through LDS.
#pragma once

#include "jl_device.h"

namespace jl {

typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));

constexpr int kBlk = 64;                    // tokens of a block
constexpr int kBlkBytes = kBlk * kHeadDim;  // one image: 8 KB
constexpr int kScaleExpMin = -117, kScaleExpMax = 119;

// Pools [n_pages][Hkv][page_size / 64] of images, scales and mean keys.  Block j
// of sequence b lies in page table[b][j / per], or in page b where table is null.
struct Cache8 {
  unsigned char* k;
  unsigned char* v;
  float* k_scale;
  float* v_scale;
  uint16_t* k_mean;
  const int32_t* table;
  int n_pages, per, Hkv;   // per: blocks of a page
  int max_pages, n_blocks;  // of a sequence: pages and blocks it can hold
  FastDiv by_per;
};

// Index of a (page, head, block of the page) in the pools; pools hold < 2^31 blocks.
__device__ inline int pool_block(const Cache8& c, int page, int h, int in_page) {
  return (page * c.Hkv + h) * c.per + in_page;
}

// Without a table a sequence is one page of n_blocks = per blocks.
__device__ inline int page_index(const Cache8& c, int blk) {
  const int p = (int)fastdiv_ge2((uint32_t)blk, c.by_per);
  return c.per > 1 ? p : blk;
}
__device__ inline int page_of(const Cache8& c, int b, int blk) {
  return c.table != nullptr ? c.table[(size_t)b * c.max_pages + page_index(c, blk)] : b;
}
__device__ inline int in_page(const Cache8& c, int blk) { return blk - page_index(c, blk) * c.per; }

__host__ __device__ inline int k_offset(int key, int d) {
  const int a = key >> 5, t = (key >> 4) & 1, r = key & 15;
  const int p = d >> 6, u = (d >> 5) & 1, g = (d >> 3) & 3, j = d & 7;
  return ((((a * 2 + t) * 2 + u) * 4 + g) * 16 + r) * 16 + 2 * j + p;
}
__host__ __device__ inline int v_offset(int key, int d) {
  const int a = key >> 5, t = (key >> 4) & 1, g = (key >> 2) & 3, i = key & 3;
  const int c = d >> 5, e = (d >> 4) & 1, m = d & 15;
  return (((a * 4 + c) * 4 + g) * 16 + m) * 16 + 8 * e + 4 * t + i;
}

// Two e4m3 values of a word (its low or its high half) as fp32.
template <bool HIGH>
__device__ inline float2 e4m3_pair(uint32_t w) {
  const f32x2 f = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, HIGH);
  return make_float2(f[0], f[1]);
}
// 16 bytes of e4m3 as fp32.
__device__ inline void e4m3_16(const u32x4 w, float* f) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 a = e4m3_pair<false>(w[i]), b = e4m3_pair<true>(w[i]);
    f[4 * i] = a.x;
    f[4 * i + 1] = a.y;
    f[4 * i + 2] = b.x;
    f[4 * i + 3] = b.y;
  }
}

// fp32 to e4m3, round to nearest even, the finite values beyond +-448 (and the
// infinities) to +-448; NaN stays NaN.
__device__ inline float e4m3_clamp(float x) {
  return x != x ? x : __builtin_amdgcn_fmed3f(x, -448.f, 448.f);
}
__device__ inline uint32_t e4m3_word(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(e4m3_clamp(a), e4m3_clamp(b), 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(e4m3_clamp(c), e4m3_clamp(d), w, true);
}

__device__ inline float pow2f(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// The smallest e in [kScaleExpMin, kScaleExpMax] with top <= 448 * 2^e, for a
// magnitude of bf16's range (beyond the last e the largest values saturate:
// 448 * 2^119 is the largest such product that fp32 and bf16 hold).
__device__ inline int scale_exponent(float top) {
  const uint32_t b = __float_as_uint(top);
  const int e = (int)(b >> 23) - 127 - 8 + ((b & 0x7fffffu) > 0x600000u ? 1 : 0);
  return max(kScaleExpMin, min(kScaleExpMax, e));
}

}  // namespace jl
