// cache8.hip -- rows into and out of the 8-bit cache (layout: cache8.h).
#include "cache8.h"

namespace jl {

struct AppendArgs {
  Cache8 c;
  const uint16_t* k;  // [B][n][Hkv][128] bf16
  const uint16_t* v;
  const int32_t* starts;
  const int32_t* n_new;  // or nullptr: n rows of every sequence
  int n, nb;             // nb: blocks a sequence's new rows can touch
};

// The sum over 16 lanes (a row) of 16 values each: lane i gets that of value i.  Each step
// halves the values: a lane keeps one half and adds its partner's.
__device__ inline float sum_rows16(float (&v)[16], int lane) {
  const bool b3 = lane & 8, b2 = lane & 4, b1 = lane & 2, b0 = lane & 1;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float keep = b3 ? v[8 + i] : v[i], give = b3 ? v[i] : v[8 + i];
    v[i] = keep + __shfl_xor(give, 8);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float keep = b2 ? v[4 + i] : v[i], give = b2 ? v[i] : v[4 + i];
    v[i] = keep + __shfl_xor(give, 4);
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const float keep = b1 ? v[2 + i] : v[i], give = b1 ? v[i] : v[2 + i];
    v[i] = keep + __shfl_xor(give, 2);
  }
  const float keep = b0 ? v[1] : v[0], give = b0 ? v[0] : v[1];
  return keep + __shfl_xor(give, 1);
}

// Workgroup = one block of one kv head that takes new rows.  Its rows are read
// once into registers, their largest magnitude gives the block's scale, and the
// images are put together in LDS and written whole.  Rows the block held before
// are kept; where the scale grows they are rounded again to the new one (a power
// of two further, so only values that fall among the subnormals move).  What a
// block held is requested with its new rows, and written back only where it changed:
// a token of decode writes 72 of the 1024 16-byte units.  The mean key
// sums e4m3 values, multiples of 2^-9 below 2^15 in all: exactly, in any order.
//
// Bound by memory for a prompt: 30001 rows of 8 heads 31 us over the same pool, 40 over three in
// turn (123 MB read and 62 written, as few as there are: 4.6 to 5.9 TB/s; one after another with
// the reading of 32768 such rows, 73 us in all).  A row each of 16 sequences takes 6.0 us, 2.4 of them
// an empty launch, the rest the chain length -> page -> block -> scale.  A run of units
// on each die, whose L2 then has all heads of a row: 39.3 for 37.9 us, 7.7 for 7.7 with 64
// sequences of one row.
__global__ __launch_bounds__(256) void append8_kernel(AppendArgs a) {
  __shared__ __attribute__((aligned(16))) unsigned char img[2][kBlkBytes];
  __shared__ float s_top[2][4];
  __shared__ float s_sum[2][kHeadDim];
  const int tid = threadIdx.x;
  const int h = blockIdx.x % a.c.Hkv;
  const int bi = blockIdx.x / a.c.Hkv;
  const int b = bi / a.nb;
  const long long start = a.starts[b];
  const long long cap = (long long)a.c.n_blocks * kBlk;
  const int n = a.n_new != nullptr ? min(max(a.n_new[b], 0), a.n) : a.n;
  const long long lo = max(start, 0LL), hi = min(start + n, cap);
  const long long base = (lo / kBlk + (bi - b * a.nb)) * kBlk;  // the block's first position
  if (base >= hi || lo >= hi) return;
  const int blk = (int)(base / kBlk);
  const int page = page_of(a.c, b, blk);
  const int r0 = (int)max(start - base, 0LL);               // rows held before
  const int r1 = (int)min(hi - base, (long long)kBlk);      // rows held after

  // ---- new rows: K as (row, 16 rotate-half pairs), V as (8 keys of a lane group, 4 channels)
  const size_t row = (size_t)a.c.Hkv * kHeadDim;
  const uint16_t* ksrc = a.k + ((size_t)b * a.n * a.c.Hkv + h) * kHeadDim;
  const uint16_t* vsrc = a.v + ((size_t)b * a.n * a.c.Hkv + h) * kHeadDim;
  const int kr = tid >> 2, kc = tid & 3;
  u32x4 kw[4] = {u32x4{}, u32x4{}, u32x4{}, u32x4{}};
  if (kr >= r0 && kr < r1) {
    const uint16_t* src = ksrc + (size_t)(base + kr - start) * row;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      kw[i] = load16(src + 32 * i + 8 * kc);
      kw[2 + i] = load16(src + 64 + 32 * i + 8 * kc);
    }
  }
  const int va = tid >> 7, vg = (tid >> 5) & 3, vd = 4 * (tid & 31);
  uint2 vw[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int key = 32 * va + 16 * (i >> 2) + 4 * vg + (i & 3);
    vw[i] = make_uint2(0, 0);
    if (key >= r0 && key < r1) vw[i] = *(const uint2*)(vsrc + (size_t)(base + key - start) * row + vd);
  }

  // ---- what the block holds: 16-byte units tid and tid + 256 of each image
  if (page < 0 || page >= a.c.n_pages) return;  // a page outside the pool is never written
  const size_t at = (size_t)pool_block(a.c, page, h, in_page(a.c, blk));
  unsigned char* const pool[2] = {a.c.k + at * kBlkBytes + 16 * tid, a.c.v + at * kBlkBytes + 16 * tid};
  u32x4 was[4] = {u32x4{}, u32x4{}, u32x4{}, u32x4{}};
  float old[2] = {0.f, 0.f};
  if (r0 > 0) {
#pragma unroll
    for (int i = 0; i < 4; ++i) was[i] = load16(pool[i >> 1] + 4096 * (i & 1));
    old[0] = a.c.k_scale[at];
    old[1] = a.c.v_scale[at];
  }

  // ---- scales: fmaxf passes NaN over; an infinity counts as the largest finite value
  float kf[32], vf[8][4];
#pragma unroll
  for (int i = 0; i < 4; ++i) unpack8(kw[i], kf + 8 * i);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    vf[i][0] = bf16_lo(vw[i].x);
    vf[i][1] = bf16_hi(vw[i].x);
    vf[i][2] = bf16_lo(vw[i].y);
    vf[i][3] = bf16_hi(vw[i].y);
  }
  float ktop = 0.f, vtop = 0.f;
#pragma unroll
  for (int i = 0; i < 32; ++i) ktop = fmaxf(ktop, fabsf(kf[i]));
#pragma unroll
  for (int i = 0; i < 32; ++i) vtop = fmaxf(vtop, fabsf(vf[i >> 2][i & 3]));
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    ktop = fmaxf(ktop, __shfl_xor(ktop, o));
    vtop = fmaxf(vtop, __shfl_xor(vtop, o));
  }
  if ((tid & 63) == 0) {
    s_top[0][tid >> 6] = ktop;
    s_top[1][tid >> 6] = vtop;
  }
  __syncthreads();
  float scale[2], back[2];  // the new scale, and old / new
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const float top = fmaxf(fmaxf(s_top[i][0], s_top[i][1]), fmaxf(s_top[i][2], s_top[i][3]));
    scale[i] = fmaxf(pow2f(scale_exponent(top)), old[i]);
    back[i] = old[i] / scale[i];
  }
  {
    const float inv = 1.f / scale[0];
    const int aa = kr >> 5, t = (kr >> 4) & 1, r = kr & 15;
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      u32x4 w;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float* x = kf + 8 * q + 2 * i;
        w[i] = e4m3_word(x[0] * inv, x[16] * inv, x[1] * inv, x[17] * inv);
      }
      *(u32x4*)&img[0][((((aa * 2 + t) * 2 + q) * 4 + kc) * 16 + r) * 16] = w;
    }
  }
  {
    const float inv = 1.f / scale[1];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint2 w = make_uint2(
          e4m3_word(vf[0][j] * inv, vf[1][j] * inv, vf[2][j] * inv, vf[3][j] * inv),
          e4m3_word(vf[4][j] * inv, vf[5][j] * inv, vf[6][j] * inv, vf[7][j] * inv));
      *(uint2*)&img[1][v_offset(32 * va + 4 * vg, vd + j)] = w;
    }
  }
  __syncthreads();

  // ---- earlier rows back in, and the images out
  float sum[16];  // of this thread's two keys of K, 32 apart: 8 pairs
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int which = i >> 1;
    const int unit = tid + 256 * (i & 1);
    u32x4 w = *(const u32x4*)&img[which][16 * unit];
    bool write = true;
    if (r0 > 0) {
      float f[16];
      e4m3_16(was[i], f);
      const int key0 = which == 0 ? 32 * (unit >> 8) + 16 * ((unit >> 7) & 1) + (unit & 15)
                                  : 32 * (unit >> 8) + 4 * ((unit >> 4) & 3);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        uint32_t again = was[i][j];
        if (back[which] != 1.f)
          again = e4m3_word(f[4 * j] * back[which], f[4 * j + 1] * back[which],
                            f[4 * j + 2] * back[which], f[4 * j + 3] * back[which]);
        uint32_t keep = 0;  // bytes of earlier rows
        if (which == 0) {
          keep = key0 < r0 ? ~0u : 0u;
        } else {
          const int left = r0 - (key0 + 16 * (j & 1));  // keys of this word (i = 0..3) below r0
          keep = left >= 4 ? ~0u : left > 0 ? (1u << (8 * left)) - 1 : 0u;
        }
        w[j] = (again & keep) | (w[j] & ~keep);
      }
      write = ((w[0] ^ was[i][0]) | (w[1] ^ was[i][1]) | (w[2] ^ was[i][2]) | (w[3] ^ was[i][3])) != 0;
    }
    if (write) *(u32x4*)(pool[which] + 4096 * (i & 1)) = w;
    if (which == 0) {
      float f[16];
      e4m3_16(w, f);
#pragma unroll
      for (int j = 0; j < 16; ++j) sum[j] = i == 0 ? f[j] : sum[j] + f[j];
    }
  }
  if (tid == 0) {
    a.c.k_scale[at] = scale[0];
    a.c.v_scale[at] = scale[1];
  }

  // ---- mean key: lane i of 16 has value i of their unit column (u, g): pair i / 2
  const float column = sum_rows16(sum, tid & 15);
  const int d = 64 * (tid & 1) + 32 * ((tid >> 6) & 1) + 8 * ((tid >> 4) & 3) + ((tid & 15) >> 1);
  s_sum[tid >> 7][d] = column;
  __syncthreads();
  if (tid < kHeadDim) {
    const __bf16 m = (__bf16)((s_sum[0][tid] + s_sum[1][tid]) / (float)r1 * scale[0]);
    a.c.k_mean[at * kHeadDim + tid] = __builtin_bit_cast(uint16_t, m);
  }
}

struct ReadArgs {
  Cache8 c;
  uint16_t* k;  // [B][n][Hkv][128] bf16
  uint16_t* v;
  int start, n, blk0, nb;
};

__device__ inline uint32_t bf16_pair(float a, float b) {
  f32x2 t = {a, b};
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(t, bf16x2));
}

// Workgroup = one block of one kv head.  A value has 4 significant bits and a
// magnitude of at least 2^-126 or zero, so bf16 holds it exactly.  Bound by memory:
// 32768 rows of 8 heads 31 to 36 us, 67 MB read and 134 written.
__global__ __launch_bounds__(256) void read8_kernel(ReadArgs a) {
  const int tid = threadIdx.x;
  const int h = blockIdx.x % a.c.Hkv;
  const int bi = blockIdx.x / a.c.Hkv;
  const int b = bi / a.nb;
  const int blk = a.blk0 + bi - b * a.nb;
  const int page = min(max(page_of(a.c, b, blk), 0), a.c.n_pages - 1);
  const size_t at = (size_t)pool_block(a.c, page, h, in_page(a.c, blk));
  const size_t row = (size_t)a.c.Hkv * kHeadDim;
  const size_t out0 = ((size_t)b * a.n * a.c.Hkv + h) * kHeadDim;
  const int pos0 = blk * kBlk - a.start;  // output row of the block's first key
  const float ks = a.c.k_scale[at], vs = a.c.v_scale[at];
  // Eight threads a key: a store instruction writes whole 128-byte lines and no cache need keep
  // them (those 32768 rows: 51 us with pieces of 32 bytes, which wrote 174 MB; 45 with whole
  // lines; 35 with the nontemporal hint on K and V too).
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int key = 32 * i + (tid >> 3), d = 8 * (tid & 7);
    const int o = pos0 + key;
    if (o < 0 || o >= a.n) continue;
    float f[16];
    e4m3_16(load16(a.c.k + at * kBlkBytes + k_offset(key, d)), f);
    u32x4 lo, hi;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      lo[j] = bf16_pair(f[4 * j] * ks, f[4 * j + 2] * ks);
      hi[j] = bf16_pair(f[4 * j + 1] * ks, f[4 * j + 3] * ks);
    }
    uint16_t* dst = a.k + out0 + (size_t)o * row + d;
    __builtin_nontemporal_store(lo, (u32x4*)dst);
    __builtin_nontemporal_store(hi, (u32x4*)(dst + kHalf));
  }
  {
    const int va = tid >> 7, vg = (tid >> 5) & 3, vd = 4 * (tid & 31);
    const unsigned char* src = a.c.v + at * kBlkBytes;
    float f[4][8];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint2 w = *(const uint2*)(src + v_offset(32 * va + 4 * vg, vd + j));
      const float2 x0 = e4m3_pair<false>(w.x), x1 = e4m3_pair<true>(w.x);
      const float2 x2 = e4m3_pair<false>(w.y), x3 = e4m3_pair<true>(w.y);
      f[j][0] = x0.x; f[j][1] = x0.y; f[j][2] = x1.x; f[j][3] = x1.y;
      f[j][4] = x2.x; f[j][5] = x2.y; f[j][6] = x3.x; f[j][7] = x3.y;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int o = pos0 + 32 * va + 16 * (i >> 2) + 4 * vg + (i & 3);
      if (o < 0 || o >= a.n) continue;
      const u32x2 w = {bf16_pair(f[0][i] * vs, f[1][i] * vs), bf16_pair(f[2][i] * vs, f[3][i] * vs)};
      __builtin_nontemporal_store(w, (u32x2*)(a.v + out0 + (size_t)o * row + vd));
    }
  }
}

// ---------------------------------------------------------------- launchers
hipError_t launch_append8(const Cache8& c, const uint16_t* k, const uint16_t* v,
                          const int32_t* starts, const int32_t* n_new, int B, int n,
                          hipStream_t stream) {
  AppendArgs a{c, k, v, starts, n_new, n, (int)((n + kBlk - 2LL) / kBlk + 1)};
  const long long wgs = (long long)B * a.nb * c.Hkv;
  if (wgs > 0x7fffffffLL) return hipErrorInvalidConfiguration;
  hipLaunchKernelGGL(append8_kernel, dim3((unsigned)wgs), dim3(256), 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_read8(const Cache8& c, uint16_t* k, uint16_t* v, int B, int start, int n,
                        hipStream_t stream) {
  ReadArgs a{c, k, v, start, n, start / kBlk, 0};
  a.nb = (start + n - 1) / kBlk - a.blk0 + 1;
  const long long wgs = (long long)B * a.nb * c.Hkv;
  if (wgs > 0x7fffffffLL) return hipErrorInvalidConfiguration;
  hipLaunchKernelGGL(read8_kernel, dim3((unsigned)wgs), dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace jl
