// decode8.hip -- single-query bifocal-RoPE decode over the 8-bit cache (cache8.h),
// over all keys of a sequence or over a list of its blocks.
//
// The method is decode.hip's (Jet-Long, arXiv 2607.07740, Sec. 3.2): the query of
// sequence b sits at kv_len[b] - 1, G follows from kv_len[b], a key is rotated to
// the view its distance selects (Eq. (1)).  A sequence without keys, or whose list
// names none, gets zeros.
#include "cache8.h"

namespace jl {

struct Decode8Args {
  Cache8 c;
  const uint16_t* q;
  const int32_t* kv_lens;
  const int32_t* blocks;  // [B][Hkv][n_select], or nullptr: every block
  uint16_t* o;
  const float2* table;
  int B, Hq, g, n_select;
  int w_pre, w0;
  float q_scale;
};

// Workgroup = (sequence, kv head), fp32 throughout: scores of 64 keys, softmax
// step, values.
template <bool BIFOCAL>
__global__ __launch_bounds__(256) void decode8_kernel(Decode8Args a) {
  __shared__ float sq[2][8][kHeadDim];  // the rotated queries of both views
  __shared__ float sp[8][kBlk];
  __shared__ float so[8][kHeadDim];
  const int tid = threadIdx.x;
  const int b = blockIdx.x / a.c.Hkv, h = blockIdx.x - b * a.c.Hkv;
  const int kv_len = min(max(a.kv_lens[b], 0), a.c.n_blocks * kBlk);
  const int qpos = kv_len - 1;
  const FastDiv gdiv = make_fastdiv(BIFOCAL ? group_size(max(kv_len, 1), a.w_pre) : 1);
  for (int i = tid; i < a.g * kHalf; i += 256) {
    const int j = i >> 6, f = i & 63;
    const uint16_t* q = a.q + ((size_t)b * a.Hq + h * a.g + j) * kHeadDim;
    const float lo = __uint_as_float((uint32_t)q[f] << 16) * a.q_scale;
    const float hi = __uint_as_float((uint32_t)q[f + 64] << 16) * a.q_scale;
    for (int view = 0; view < 2; ++view) {
      const int pos = max(view == 0 ? qpos : remote_pos(max(qpos, 0), gdiv), 0);
      const float2 cs = a.table[(size_t)pos * kHalf + f];
      sq[view][j][f] = lo * cs.x - hi * cs.y;
      sq[view][j][f + 64] = hi * cs.x + lo * cs.y;
    }
  }
  __syncthreads();
  const int key = tid >> 2, part = tid & 3;
  const int d = tid & 127, half = tid >> 7;
  float m[8], l[8], acc[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    m[j] = -INFINITY;
    l[j] = acc[j] = 0.f;
  }
  const int n_steps = a.blocks != nullptr ? a.n_select : (kv_len + kBlk - 1) / kBlk;
  for (int s = 0; s < n_steps; ++s) {
    const int blk =
        a.blocks != nullptr ? a.blocks[((size_t)b * a.c.Hkv + h) * a.n_select + s] : s;
    if (blk < 0 || blk >= a.c.n_blocks || blk * kBlk >= kv_len) continue;
    const int page = min(max(page_of(a.c, b, blk), 0), a.c.n_pages - 1);
    const size_t at = (size_t)pool_block(a.c, page, h, in_page(a.c, blk));
    const unsigned char* kb = a.c.k + at * kBlkBytes;
    const unsigned char* vb = a.c.v + at * kBlkBytes;
    const int pos = blk * kBlk + key;
    const int view = BIFOCAL && qpos - pos > a.w0 ? 1 : 0;
    const int rp = view == 1 ? remote_pos(pos, gdiv) : pos;
    float sc[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) sc[j] = 0.f;
    for (int i = 0; i < 16; ++i) {
      const int f = 16 * part + i;
      const uint32_t w = *(const uint16_t*)(kb + k_offset(key, f));
      const float2 x = e4m3_pair<false>(w);
      const float2 cs = a.table[(size_t)rp * kHalf + f];
      const float lo = x.x * cs.x - x.y * cs.y, hi = x.y * cs.x + x.x * cs.y;
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (j < a.g) sc[j] += lo * sq[view][j][f] + hi * sq[view][j][f + 64];
    }
    const float ks = a.c.k_scale[at], vs = a.c.v_scale[at];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      sc[j] += __shfl_xor(sc[j], 1);
      sc[j] += __shfl_xor(sc[j], 2);
      if (part == 0 && j < a.g) sp[j][key] = pos < kv_len ? sc[j] * ks : -INFINITY;
    }
    __syncthreads();
    for (int j = 0; j < a.g; ++j) {
      float mx = m[j];
      for (int i = 0; i < kBlk; ++i) mx = fmaxf(mx, sp[j][i]);
      const float use = mx == -INFINITY ? 0.f : mx;
      const float alpha = fast_exp2(m[j] - use);
      m[j] = mx;
      float sum = 0.f, o = 0.f;
      for (int i = 0; i < 32; ++i) {
        const int k2 = 32 * half + i;
        const float p = fast_exp2(sp[j][k2] - use);
        const float v = e4m3_pair<false>(vb[v_offset(k2, d)]).x;
        sum += p;
        if (blk * kBlk + k2 < kv_len) o += p * v;
      }
      l[j] = l[j] * alpha + sum;
      acc[j] = acc[j] * alpha + o * vs;
    }
    __syncthreads();
  }
  for (int j = 0; j < a.g; ++j) {
    if (half == 1) {
      so[j][d] = acc[j];
      if (d == 0) sp[j][0] = l[j];
    }
  }
  __syncthreads();
  if (half == 0) {
    for (int j = 0; j < a.g; ++j) {
      const float den = l[j] + sp[j][0];
      const __bf16 r = (__bf16)(den == 0.f ? 0.f : (acc[j] + so[j][d]) / den);
      a.o[((size_t)b * a.Hq + h * a.g + j) * kHeadDim + d] = __builtin_bit_cast(uint16_t, r);
    }
  }
}

// ---------------------------------------------------------------- launcher
size_t decode8_workspace_bytes(int g) { return 4096 + (size_t)1024 * g * 528; }

hipError_t launch_decode8(bool bifocal, const Cache8& c, const uint16_t* q, const int32_t* kv_lens,
                          const int32_t* blocks, int n_select, uint16_t* o, const float2* table,
                          int B, int Hq, int w_pre, int w0, void* /*ws*/, hipStream_t stream) {
  Decode8Args a{c, q, kv_lens, blocks, o, table, B, Hq, Hq / c.Hkv, n_select, w_pre, w0,
                1.4426950408889634f / sqrtf((float)kHeadDim)};
  const long long wgs = (long long)B * c.Hkv;
  if (wgs > 0x7fffffffLL) return hipErrorInvalidConfiguration;
  if (bifocal)
    hipLaunchKernelGGL(decode8_kernel<true>, dim3((unsigned)wgs), dim3(256), 0, stream, a);
  else
    hipLaunchKernelGGL(decode8_kernel<false>, dim3((unsigned)wgs), dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace jl
