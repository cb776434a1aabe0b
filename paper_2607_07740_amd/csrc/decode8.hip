// decode8.hip -- single-query bifocal-RoPE decode over the 8-bit cache (cache8.h),
// over all keys of a sequence or over a list of its blocks.
//
// The method is decode.hip's (Jet-Long, arXiv 2607.07740, Sec. 3.2): the query of
// sequence b sits at kv_len[b] - 1, G follows from kv_len[b], a key is rotated to
// the view its distance selects (Eq. (1)), and the 16 columns of a matrix
// instruction are the group's heads in the base (0..7) and the remote view (8..15);
// a column keeps the keys of its own view, so that each is a partial softmax state,
// and the states merge by Eq. (7).  A sequence without keys, or whose list names
// none, gets zeros.
#include <algorithm>
#include <climits>

#include "cache8.h"

namespace jl {

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

constexpr int kD8MaxWg = 512;    // workgroups of a call: workspaces are sized for as many
constexpr int kD8SegCost = 6;    // what a workgroup pays for a further segment, in steps
constexpr int kD8State = 132;    // floats of a state: m, l, pad, pad, O[128]
constexpr float kD8Up = 15.f, kD8Down = 0x1p-15f;  // weights in fp16 are times 2^15
constexpr int kD8Counters = 1024;  // at the front of the workspace (4096 bytes)

struct Decode8Args {
  Cache8 c;
  const uint16_t* q;
  const int32_t* kv_lens;
  const int32_t* blocks;  // [B][Hkv][n_select], or nullptr: every block
  uint16_t* o;
  const float2* table;
  const unsigned char* offsets;  // kD8TabBytes: see offset_rows_kernel
  int* counters;
  float* states;  // [2 n_wg][g][kD8State]
  int B, Hq, g, n_select;
  int n_wg, w_pre, w0;
  bool even;            // lists: each gets the same number of workgroups, none works on two
  int n_sets, n_merge;  // of a merge: sets of threads, and states that one workgroup takes
  float q_scale;
};

// The (sequence, kv head) pairs are segments of a list, each as long as its steps of
// 64 keys and kD8SegCost empty ones, and workgroup w takes the w-th of n equal
// ranges.  Workgroups that share a segment meet in its counter: the first's
// index names it, since only a range's last segment goes on in the next range.
// Where they merge in two steps, that is the first group's; the others' are in a
// second row of counters, where one workgroup is a further one of one segment at
// most, and the groups meet in the second workgroup's, whom no group begins with.
struct Segments {
  uint32_t q, r;  // entries per range, and ranges (the first ones) with one more
  int n;             // ranges
};

__device__ inline void make_ranges(Segments& s, int n_wg, int waves, uint32_t V) {
  // as many ranges as hold about one step per wave and the cost of a segment each: where that does
  // not come out even they are shorter, none below half of that
  const uint32_t least = (uint32_t)(waves + kD8SegCost);
  s.n = (int)min((uint32_t)n_wg, (V + least - 1) / least);
  s.q = V / (uint32_t)s.n;
  s.r = V - s.q * (uint32_t)s.n;
}
__device__ inline uint32_t range_start(const Segments& s, uint32_t w) {
  return s.q * w + min(w, s.r);
}
__device__ inline int range_at(const Segments& s, uint32_t x) {
  const uint32_t head = s.r * (s.q + 1);
  return (int)(x < head ? x / (s.q + 1) : s.r + (x - head) / s.q);
}

// floor(x / d) for a run-time d < 2^24 (make_fastdiv, whose 64-bit division is slow here,
// by way of a double quotient that is corrected in integers).
__device__ inline FastDiv make_fastdiv24(uint32_t d) {
  FastDiv f;
  f.d = d;
  f.m = f.l = 0;
  if (d <= 1) return f;
  f.l = 32 - __builtin_clz(d - 1);
  const uint32_t num = (1u << f.l) - d;
  uint32_t m = (uint32_t)(4294967296.0 * (double)num / (double)d);
  long long rem = ((long long)num << 32) - (long long)((unsigned long long)m * d);
  if (rem < 0) {
    --m;
    rem += d;
  }
  if (rem >= (long long)d) ++m;
  f.m = m + 1;
  return f;
}

__device__ inline int len8(const Decode8Args& a, int b) {
  return min(max(a.kv_lens[b], 0), a.c.n_blocks * kBlk);
}
// list entries of a segment of sequence b
__device__ inline int entries8(const Decode8Args& a, int b) {
  return (len8(a, b) + kBlk - 1) / kBlk + kD8SegCost;
}

// States pass between workgroups, and so between dies whose L2s know nothing of each
// other: they are written through and read past the L2 (device scope, the sc1 bit),
// with the writer's own wait before its arrival is counted.  A device-scope fence
// instead writes the whole L2 back and empties it, in every workgroup: 145 us in place
// of 57 for 131072 keys, 32/8 heads.
typedef __amdgpu_buffer_rsrc_t buffer_t;
constexpr int kDeviceScope = 16;  // sc1
__device__ inline buffer_t make_buffer(const void* p, size_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc((void*)p, 0, (int)bytes, 0x00027000);
}
__device__ inline void put4(buffer_t r, uint32_t at, f32x4 x) {
  __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, x), r, at, 0, kDeviceScope);
}
__device__ inline f32x4 get4(buffer_t r, uint32_t at) {
  return __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(r, at, 0, kDeviceScope));
}
__device__ inline float2 get2(buffer_t r, uint32_t at) {
  const u32x2 x = __builtin_amdgcn_raw_buffer_load_b64(r, at, 0, kDeviceScope);
  return make_float2(__uint_as_float(x[0]), __uint_as_float(x[1]));
}
// Byte offset of a state: a workgroup has one slot for the segment that came to it and one
// for the segment that begins in it.
__device__ inline uint32_t state_at(const Decode8Args& a, int w, bool begins, int head) {
  return (uint32_t)((2 * w + (begins ? 1 : 0)) * a.g + head) * (kD8State * 4);
}

// Maximum over the lanes l, l ^ 16, l ^ 32, l ^ 48, by lane swaps in registers.
__device__ inline float max_over_groups(float x) {
  u32x2 r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
  r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

__device__ inline f32x4 mfma16h(f16x8 a, f16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

// Two e4m3 numbers of a word's low or high half as fp16 (exact).
template <bool HIGH>
__device__ inline f16x2 e4m3_f16(uint32_t w) {
  return __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, HIGH);
}
// The pair (x_i, x_{i+64}) rotated by cs = (cos, sin): two packed fp16 instructions.
__device__ inline f16x2 rotate_pair(f16x2 x, f16x2 cs) {
  const f16x2 c = __builtin_shufflevector(cs, cs, 0, 0);
  const f16x2 s = {-cs[1], cs[1]};
  const f16x2 sw = __builtin_shufflevector(x, x, 1, 0);
  return __builtin_elementwise_fma(x, c, sw * s);
}

constexpr int kD8TabRow = kHalf * 4 + 16;  // 64 fp16 (cos, sin) and 16 bytes, so that rows start 4 banks apart
constexpr int kD8TabBytes = kBlk * kD8TabRow;
static_assert(kD8TabBytes % 1024 == 0, "copied in pieces of 1 KB");
constexpr int kD8Row = kHeadDim + 4;       // floats of a merge row

// The first 64 rows of a cos/sin table in fp16, as the decode kernel keeps them in LDS.
__global__ void offset_rows_kernel(const float2* table, unsigned char* out) {
  const int i = blockIdx.x * blockDim.x + threadIdx.x;
  if (i >= kD8TabBytes / 4) return;
  const int r = i / (kD8TabRow / 4), f = i - r * (kD8TabRow / 4);
  f16x2 h = {(_Float16)0.f, (_Float16)0.f};
  if (f < kHalf) {
    const float2 cs = table[r * kHalf + f];
    h = f16x2{(_Float16)cs.x, (_Float16)cs.y};
  }
  ((f16x2*)out)[i] = h;
}

// What a call's workgroups share out: the steps of a batch's sequences, those of one
// sequence, or lists of blocks.
enum Decode8Mode : int { kBatch8 = 0, kOne8 = 1, kListed8 = 2, kWideList8 = 3 };
// Waves of a workgroup.  One sequence: eight and a workgroup per CU leave half the states
// to merge, which one workgroup per kv head reads at a CU's own rate (131072 keys, 32/8
// heads: 54.6 -> 51.3 us; 32768 21.6 -> 19.4; 1999 keys, 16/8 heads 11.6 -> 11.8).
// Otherwise four, two workgroups per CU, one of which streams while the other merges
// (256 sequences of 0.2K to 2K: 124 -> 111 us; 128 listed blocks 14.6 -> 14.2).
__host__ __device__ constexpr int decode8_waves(int mode) {
  return mode == kOne8 || mode == kWideList8 ? 8 : 4;
}

template <int kD8Waves>
struct __attribute__((aligned(1024))) Decode8Smem {
  unsigned char tab[kD8TabBytes];           // (cos, sin)(t omega_i), t < 64
  float2 rows[kD8Waves][2][kHalf];          // a step's (cos, sin) rows that rotate its query
  union {
    float o[kD8Waves][16][kD8Row];          // the waves' states
    float set_o[2 * kD8Waves][kD8Row];                 // the sums of the last workgroup's sets of threads
  };
  float m[kD8Waves][16], l[kD8Waves][16];
  float set_m[2 * kD8Waves], set_l[2 * kD8Waves];
  struct {
    size_t o;   // where its output goes
    int wf, n;  // its first workgroup, how many (0: no such segment)
  } due[2];
  int last[2];
};

// Workgroup w: its range's segments one after another; each of its waves takes every
// fourth (eighth) step of 64 keys and keeps the 16 columns' states in registers.
//
// A step is 16 KB, K and V, that go from memory into registers, 16 bytes a lane and
// 1 KB an instruction; the layout is the matrix operands' own.  K is requested one step
// ahead.  V is written so too, but the compiler joins those requests with the first
// step's at the head of the loop: a step's V is on its way during its own scores.
// Rotation by offset in the block: with k0 the block's first position, a key is
// rotated by t = k - k0 (base) or f(k) - f(k0) (remote), from 64 rows of fp16
// (cos, sin) in LDS, and the query's columns by q - k0 or f(q) - f(k0) in fp32:
// only relative positions matter (Sec. 3.2, Eq. (6)).  A rotated pair costs a
// conversion and two packed fp16 instructions (cos and sin, the product with sin and the
// sum each round to fp16) and goes to the matrix cores as
// it is: e4m3 numbers are exact in fp16, and with |x| <= 448 none overflows.  The
// block's scale of K multiplies the scores, that of V the step's product.
// The query is brought to fp16's upper range by a power of two first, its own range aside.
//
// Bound by memory where keys are many: 8 sequences of 32K to 128K, 32/8 heads 208 to 219 us,
// 1.34 GB at 6.1 to 6.4 TB/s (the loads alone 6.4 to 6.9); one of 1048576 318 to 334 us, 6.4 to
// 6.8; of 131072 49 us, 5.5; 32 of 0.5K to 16K on pages of 64 tokens 67 to 71 us, 5.0 to 5.3.  A
// step's 680 VALU instructions fit beside its loads: one without the masks of steps in one view
// took as long.  Bound by a chain
// of latencies where they are few (1999 keys, 16/8 heads: 10.6 to 11.3 us; 192 keys 6.4): an empty
// launch 2.4 us, length, page and step about 0.8 each from a request to the data, a step's work
// 2, the waves' merge 0.9, a state's way to another workgroup and the merge there 2.6.
template <bool BIFOCAL, int MODE>
__global__ __launch_bounds__(64 * decode8_waves(MODE), 2) void decode8_kernel(Decode8Args a) {
  constexpr int kD8Waves = decode8_waves(MODE);
  constexpr int kD8Threads = 64 * kD8Waves;
  constexpr bool LISTED = MODE == kListed8 || MODE == kWideList8;
  __shared__ Decode8Smem<kD8Waves> sm;
  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int i16 = lane & 15, g4 = lane >> 4;
  const int w = blockIdx.x;

  // ---- offset rows, straight into LDS (a workgroup without work waits for them too, while it
  // holds the LDS they go to)
  for (int n = wave; n < kD8TabBytes / 1024; n += kD8Waves)
    dma16_s(a.offsets, 1024 * n + 16 * lane, lds_addr(sm.tab) + 1024 * n);

  // ---- this workgroup's range, and the sequence and head it begins in
  Segments sg = {};
  uint32_t pos = 0;  // list entry of the current segment's first step
  uint32_t x0, x1;
  int b, h;
  // Segments of one length, no more than workgroups: each may get the same number of them, and
  // no workgroup works on two.
  const int segs = a.B * a.c.Hkv;
  const bool even = MODE == kOne8 || MODE == kWideList8 || (LISTED && a.even);
  int first_wg = 0, parts = 0;
  if (even) {
    const int per = a.n_wg / segs;
    const int seg = w / per;
    if (seg >= segs) return wait_vmem();
    b = seg / a.c.Hkv;
    h = seg - b * a.c.Hkv;
    const int n = LISTED ? a.n_select : (len8(a, 0) + kBlk - 1) / kBlk;
    first_wg = seg * per;
    parts = __builtin_amdgcn_readfirstlane(max(1, min(per, (n + kD8Waves - 1) / kD8Waves)));
    x0 = (uint32_t)(w - first_wg);
    if ((int)x0 >= parts) return wait_vmem();
    x1 = UINT_MAX;
  } else if (LISTED) {
    const uint32_t e = (uint32_t)(a.n_select + kD8SegCost);
    make_ranges(sg, a.n_wg, kD8Waves, e * (uint32_t)segs);
    if (w >= sg.n) return wait_vmem();
    x0 = range_start(sg, w);
    const uint32_t seg = x0 / e;
    b = (int)(seg / (uint32_t)a.c.Hkv);
    h = (int)(seg - (uint32_t)b * a.c.Hkv);
    pos = seg * e;
    x1 = range_start(sg, (uint32_t)w + 1);
  } else {
    // all lengths, 64 at a time; every wave for itself
    uint32_t V = 0, v = 0;
    for (int b0 = 0; b0 < a.B; b0 += 64) {
      v = b0 + lane < a.B ? (uint32_t)entries8(a, b0 + lane) * a.c.Hkv : 0;
      uint32_t t = v;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) t += __shfl_xor(t, o);
      V += t;
    }
    make_ranges(sg, a.n_wg, kD8Waves, __builtin_amdgcn_readfirstlane(V));
    if (w >= sg.n) return wait_vmem();
    x0 = range_start(sg, w);
    uint32_t before = 0;
    b = 0;
    for (int b0 = 0; b0 < a.B; b0 += 64) {
      if (a.B > 64) v = b0 + lane < a.B ? (uint32_t)entries8(a, b0 + lane) * a.c.Hkv : 0;
      uint32_t incl = v;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const uint32_t t = __shfl_up(incl, o);
        if (lane >= o) incl += t;
      }
      const uint32_t all = __builtin_amdgcn_readlane(incl, 63);
      if (x0 < before + all) {
        const int i = (int)__popcll(__ballot(before + incl <= x0));
        b = b0 + i;
        pos = before + __builtin_amdgcn_readlane(incl - v, i);
        break;
      }
      before += all;
    }
    b = __builtin_amdgcn_readfirstlane(b);
    pos = __builtin_amdgcn_readfirstlane(pos);
    const uint32_t e = (uint32_t)entries8(a, b);
    h = (int)((x0 - pos) / e);
    pos += (uint32_t)h * e;
    x1 = range_start(sg, (uint32_t)w + 1);
  }
  h = __builtin_amdgcn_readfirstlane(h);
  pos = __builtin_amdgcn_readfirstlane(pos);

  // query columns: col = (view, head); the distances q - k that a column keeps are
  // [keep_lo, keep_lo + keep_n) as one unsigned compare (none for unused columns)
  const int view = i16 >> 3, hj = i16 & 7;
  const bool col_on = hj < a.g && (BIFOCAL || view == 0);

  const buffer_t states =
      make_buffer(a.states, (size_t)2 * kD8MaxWg * a.g * kD8State * sizeof(float));
  bool shared = false;  // some segment is shared with other workgroups
  if (tid < 2) sm.due[tid].n = 0;
  wait_vmem();  // the offset rows have landed, in every wave
  __syncthreads();

  for (; pos < x1 && b < a.B;) {
    const int kv_len = __builtin_amdgcn_readfirstlane(len8(a, b));
    const int n_real = LISTED ? a.n_select : (kv_len + kBlk - 1) / kBlk;
    // this workgroup's steps of the segment
    const uint32_t end = pos + (uint32_t)n_real;
    int off, n_steps;
    if (even) {
      const int q = n_real / parts, r = n_real - q * parts;
      off = q * (int)x0 + min((int)x0, r);
      n_steps = q + ((int)x0 < r ? 1 : 0);
    } else {
      const uint32_t from = max(x0, pos);
      off = (int)(from - pos);
      n_steps = (int)min(x1, end) - (int)from;
    }
    const size_t o_at = ((size_t)b * a.Hq + h * a.g) * kHeadDim;
    if (n_real == 0 && (even || pos >= x0)) {  // a sequence without keys
      for (int i = tid; i < a.g * kHeadDim / 8; i += kD8Threads) ((u32x4*)(a.o + o_at))[i] = u32x4{};
    }
    if (n_steps > 0) {
      u32x4 qraw[4];
      {
        const uint16_t* qrow = a.q + o_at + (size_t)min(hj, a.g - 1) * kHeadDim + 8 * g4;
#pragma unroll
        for (int u = 0; u < 4; ++u) qraw[u] = load16(qrow + 32 * u);
      }
      const int G = BIFOCAL ? (int)((uint32_t)max(kv_len - 1, 0) / (uint32_t)a.w_pre) + 1 : 1;
      const FastDiv gdiv = make_fastdiv24((uint32_t)G);
      const int w0 = G > 1 ? a.w0 : INT_MAX;  // one view only where f is the identity
      const int qpos = max(kv_len - 1, 0);
      const int fq = (int)fastdiv((uint32_t)qpos, gdiv);
      const int keep_lo = BIFOCAL && view == 1 ? (int)min((uint32_t)w0 + 1u, (uint32_t)INT_MAX) : 0;
      const uint32_t keep = !col_on ? 0u
                            : view == 0 ? (uint32_t)w0 + 1u
                                        : (uint32_t)INT_MAX - (uint32_t)w0;

      f32x4 acc[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) acc[i] = f32x4{};
      float m_run = -INFINITY, l_run = 0.f;

      // the column's query in fp32, pairs 32 u + 8 g4 + j, scaled by log2(e) / sqrt(d) and by
      // the power of two that brings its largest value to [2^16, 2^17): rotated, it is at most
      // 0.1276 sqrt(2) 2^17 = 23700, which fp16 holds, and so it does the values down to 2^-27 of
      // the largest to 11 bits and to 2^-37 at all
      float qlo[16], qhi[16];
      float q_back;  // what undoes the latter

      // the step in hand; each of K's registers takes the next step's piece as soon as its own is
      // used
      u32x4 kx[8], vx[8], row;
      float ks, vs;
      int k0;         // first position of the step's block
      bool on;        // there is one (a list may name none)
      int k0n, phys;  // of the step that is loaded
      // Lane l holds this wave's l-th step of 64: its position (-1 where there is nothing to do)
      // and its block of the pools.
      int at_k0, at_phys;
      auto look_up = [&](int first) __attribute__((always_inline)) {
        const int i = first + kD8Waves * lane;
        at_k0 = -1;
        at_phys = 0;
        if (i < n_steps) {
          int blk = off + i;
          if (LISTED) blk = a.blocks[((size_t)b * a.c.Hkv + h) * a.n_select + blk];
          if (blk >= 0 && blk < a.c.n_blocks && blk * kBlk < kv_len) {
            const int page = min(max(page_of(a.c, b, blk), 0), a.c.n_pages - 1);
            at_k0 = blk * kBlk;
            at_phys = pool_block(a.c, page, h, in_page(a.c, blk));
          }
        }
      };
      // Where the loaded step's pieces come from.  Behind the last step, and where a list names no
      // block, that is one piece of the table: every turn of the loop has the same loads in
      // flight.  (Where they may or may not be, each wait is for the path with fewer, which
      // drains the pipeline.)
      const unsigned char *kp, *vp;
      int piece;
      const unsigned char* rp;
      auto set_step = [&](int l) __attribute__((always_inline)) {
        k0n = __builtin_amdgcn_readlane(at_k0, l);
        phys = __builtin_amdgcn_readlane(at_phys, l);
        kp = k0n >= 0 ? a.c.k + (size_t)phys * kBlkBytes : (const unsigned char*)a.table;
        vp = k0n >= 0 ? a.c.v + (size_t)phys * kBlkBytes : (const unsigned char*)a.table;
        piece = k0n >= 0 ? 16 * lane : 0;
        const int kk = max(k0n, 0);
        int r = qpos - kk;
        if (BIFOCAL && lane >= 32) r = fq - (int)fastdiv((uint32_t)kk, gdiv);
        rp = (const unsigned char*)a.table + (size_t)(uint32_t)max(r, 0) * (kHalf * 8) + 16 * (lane & 31);
      };
      auto load_k = [&](int n) __attribute__((always_inline)) {
        kx[n] = __builtin_nontemporal_load((const u32x4*)(kp + 1024 * n + piece));
      };
      auto load_v = [&](int n) __attribute__((always_inline)) {
        vx[n] = __builtin_nontemporal_load((const u32x4*)(vp + 1024 * n + piece));
      };

      // sc: the scores of four tiles of 16 keys, in units of the block's scale
      f32x4 sc[4];
      auto scores = [&]() __attribute__((always_inline)) {
        // ---- the query rotated by q - k0 (base columns) or f(q) - f(k0) (remote)
        f16x8 qop[4];
        {
          float2* rows = &sm.rows[wave][0][0];
          ((u32x4*)rows)[lane] = row;
          row = *(const u32x4*)rp;
          __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
          __builtin_amdgcn_wave_barrier();
          const float4* cs = (const float4*)(rows + (BIFOCAL ? view * kHalf : 0));
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int j = 0; j < 8; j += 2) {
              const float4 c = cs[16 * u + 4 * g4 + j / 2];
              const int n = 8 * u + j;
              f16x8& o = qop[2 * u + j / 4];
              const int at = 2 * (j & 3);
              o[at] = (_Float16)(qlo[n] * c.x - qhi[n] * c.y);
              o[at + 1] = (_Float16)(qhi[n] * c.x + qlo[n] * c.y);
              o[at + 2] = (_Float16)(qlo[n + 1] * c.z - qhi[n + 1] * c.w);
              o[at + 3] = (_Float16)(qhi[n + 1] * c.z + qlo[n + 1] * c.w);
            }
          __builtin_amdgcn_wave_barrier();
        }

        const int fk0 = BIFOCAL ? (int)fastdiv_ge2((uint32_t)k0, gdiv) : 0;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const int off = 16 * t + i16;  // of this lane's key in the block
          int r = off;
          if (BIFOCAL && qpos - (k0 + off) > w0)
            r = (int)fastdiv_ge2((uint32_t)(k0 + off), gdiv) - fk0;
          const unsigned char* row = sm.tab + r * kD8TabRow + 32 * g4;
          sc[t] = f32x4{};
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const f16x8 c0 = *(const f16x8*)(row + 128 * u), c1 = *(const f16x8*)(row + 128 * u + 16);
            const u32x4 x = kx[2 * t + u];
            load_k(2 * t + u);
            f16x8 y0, y1;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const f16x8& c = i < 2 ? c0 : c1;
              f16x8& y = i < 2 ? y0 : y1;
              const int p = 4 * (i & 1);
              const f16x2 ya = rotate_pair(e4m3_f16<false>(x[i]), f16x2{c[p], c[p + 1]});
              const f16x2 yb = rotate_pair(e4m3_f16<true>(x[i]), f16x2{c[p + 2], c[p + 3]});
              y[p] = ya[0];
              y[p + 1] = ya[1];
              y[p + 2] = yb[0];
              y[p + 3] = yb[1];
            }
            sc[t] = mfma16h(y0, qop[2 * u], sc[t]);
            sc[t] = mfma16h(y1, qop[2 * u + 1], sc[t]);
          }
        }

      };

      f16x8 p[2];
      float weight;  // of the step's sums in the column's
      auto softmax = [&](float ks) __attribute__((always_inline)) {
        // ---- each column keeps the keys of its own view; lane: keys 16 t + 4 g4 + i
        const uint32_t dist = (uint32_t)(qpos - k0 - 4 * g4) - (uint32_t)keep_lo;
        const uint32_t keep_n = LISTED && !on ? 0u : keep;
        float mt = -INFINITY;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            sc[t][i] = dist - (uint32_t)(16 * t + i) < keep_n ? sc[t][i] : -INFINITY;
            mt = fmaxf(mt, sc[t][i]);
          }
        // a power of two, so f times a score is exact; positive and finite, so that a masked
        // score stays -inf
        const float f = __builtin_amdgcn_fmed3f(ks * q_back, 0x1p-126f, 0x1p126f);
        mt = max_over_groups(mt) * f;
        // A step's weights are taken against a reference of its own, kD8Up below its maximum: they
        // are at most 2^15, and fp16 holds 2^-29 .. 1 of the step's largest to 11 bits and 2^-39
        // of it at all.  (A maximum whose last bit is above 1 is the reference itself: 2^-14 and
        // 2^-24 of it.)  Against the column's maximum so far, whole blocks of small weights would
        // be lost beside one large, and their values may be as much larger; the step's sums enter
        // the column's in fp32, by `weight`.  The sum is that of the rounded weights.
        mt = fabsf(mt) < 0x1p22f ? mt - kD8Up : mt;
        const float m_new = fmaxf(m_run, mt);
        const float m_use = m_new == -INFINITY ? 0.f : m_new;
        const float m_step = mt == -INFINITY ? 0.f : mt;
        const float alpha = m_new == m_run ? 1.f : fast_exp2(m_run - m_use);
        weight = m_new == mt ? 1.f : fast_exp2(mt - m_use);
        float l = 0.f;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const f16x2 one = {(_Float16)1.f, (_Float16)1.f};
#pragma unroll
          for (int i = 0; i < 4; i += 2) {
            const f16x2 pp = {(_Float16)fast_exp2(__builtin_fmaf(sc[t][i], f, -m_step)),
                              (_Float16)fast_exp2(__builtin_fmaf(sc[t][i + 1], f, -m_step))};
            l = __builtin_amdgcn_fdot2(pp, one, l, false);
            p[t >> 1][4 * (t & 1) + i] = pp[0];
            p[t >> 1][4 * (t & 1) + i + 1] = pp[1];
          }
        }
        l_run = l_run * alpha + l * weight;
        m_run = m_new;
        if (__ballot(alpha != 1.f) != 0) {  // most steps leave every maximum alone
#pragma unroll
          for (int i = 0; i < 8; ++i) acc[i] *= alpha;
        }
      };

      auto values = [&]() __attribute__((always_inline)) {
        // ---- O += scale V^T P^T; where the sequence ends inside the block the values behind
        // its end are zeroed, since 0 times what lies there may be NaN
        const int len = LISTED && !on ? 0 : kv_len;
        if (k0 + kBlk > len) {
#pragma unroll
          for (int hf = 0; hf < 2; ++hf)
#pragma unroll
            for (int t = 0; t < 2; ++t) {
              const int left = len - (k0 + 32 * hf + 16 * t + 4 * g4);
              const uint32_t keep = left >= 4 ? ~0u : left > 0 ? (1u << (8 * left)) - 1 : 0u;
#pragma unroll
              for (int c = 0; c < 4; ++c) {
                vx[4 * hf + c][t] &= keep;
                vx[4 * hf + c][2 + t] &= keep;
              }
            }
        }
        // a step without a block holds some other block's scale, perhaps no number
        const float up = LISTED && !on ? 0.f : vs * kD8Down * weight;
        vs = a.c.v_scale[phys];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const u32x4 x[2] = {vx[c], vx[4 + c]};
          load_v(c);
          load_v(4 + c);
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            f32x4 d = f32x4{};
#pragma unroll
            for (int hf = 0; hf < 2; ++hf) {
              const f16x2 v0 = e4m3_f16<false>(x[hf][2 * e]), v1 = e4m3_f16<true>(x[hf][2 * e]);
              const f16x2 v2 = e4m3_f16<false>(x[hf][2 * e + 1]), v3 = e4m3_f16<true>(x[hf][2 * e + 1]);
              const f16x8 v = {v0[0], v0[1], v1[0], v1[1], v2[0], v2[1], v3[0], v3[1]};
              d = mfma16h(v, p[hf], d);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
              acc[2 * c + e][i] = __builtin_fmaf(d[i], up, acc[2 * c + e][i]);
          }
        }
      };

      const int mine = (n_steps - wave + kD8Waves - 1) / kD8Waves;  // this wave's steps
      look_up(wave);
      set_step(0);
      ks = a.c.k_scale[phys];
      row = *(const u32x4*)rp;
#pragma unroll
      for (int n = 0; n < 8; ++n) load_k(n);
      vs = a.c.v_scale[phys];
#pragma unroll
      for (int n = 0; n < 8; ++n) load_v(n);

#pragma unroll
      for (int u = 0; u < 2; ++u) {
        unpack8(qraw[u], qlo + 8 * u);
        unpack8(qraw[2 + u], qhi + 8 * u);
      }
      {
        float top = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) top = fmaxf(top, fmaxf(fabsf(qlo[i]), fabsf(qhi[i])));
        top = max_over_groups(top);
        const int e = max((int)(__float_as_uint(top) >> 23) - 127 - 16, -126);
        const float down = pow2f(-e);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          qlo[i] = qlo[i] * down * a.q_scale;
          qhi[i] = qhi[i] * down * a.q_scale;
        }
        q_back = pow2f(e);
      }
      for (int i = 0; i < mine; ++i) {
        on = k0n >= 0;
        k0 = max(k0n, 0);
        if (((i + 1) & 63) == 0) look_up(wave + kD8Waves * (i + 1));
        set_step((i + 1) & 63);
        const float ks_now = ks;
        ks = a.c.k_scale[phys];
        scores();
        softmax(ks_now);
        values();
      }

      // ---- the waves' states, and the two views of a head, into one (max-shifted)
      l_run += __shfl_xor(l_run, 16);
      l_run += __shfl_xor(l_run, 32);
#pragma unroll
      for (int db = 0; db < 8; ++db) *(f32x4*)&sm.o[wave][i16][16 * db + 4 * g4] = acc[db];
      if (g4 == 0) {
        sm.m[wave][i16] = m_run;
        sm.l[wave][i16] = l_run * kD8Down;
      }
      __syncthreads();
      const int wf = even ? first_wg : range_at(sg, pos);
      const int n_parts = even ? parts : range_at(sg, end - 1) - wf + 1;
      const int j = tid >> 5, c4 = 4 * (tid & 31);  // head and channels of this thread
      if (j < a.g) {
        float M = -INFINITY;
#pragma unroll
        for (int x = 0; x < 2 * kD8Waves; ++x) M = fmaxf(M, sm.m[x >> 1][(x & 1) * 8 + j]);
        float den = 0.f;
        f32x4 num = f32x4{};
#pragma unroll
        for (int x = 0; x < 2 * kD8Waves; ++x) {
          const int col = (x & 1) * 8 + j;
          const float mx = sm.m[x >> 1][col];
          const float wt = mx == M ? 1.f : fast_exp2(mx - M);
          den += wt * sm.l[x >> 1][col];
          num += wt * *(const f32x4*)&sm.o[x >> 1][col][c4];
        }
        if (n_parts == 1) {
          bf16x4 r;
#pragma unroll
          for (int i = 0; i < 4; ++i) r[i] = (__bf16)(den == 0.f ? 0.f : num[i] / den);
          *(bf16x4*)(a.o + o_at + (size_t)j * kHeadDim + c4) = r;
        } else {
          const uint32_t at = state_at(a, w, w == wf, j);
          put4(states, at + 16 + 4 * c4, num);
          if (c4 == 0) put4(states, at, f32x4{M, den, 0.f, 0.f});
        }
      }
      if (n_parts > 1) {
        shared = true;
        if (tid == 0) sm.due[w == wf ? 1 : 0] = {o_at, wf, n_parts};
      }
      __syncthreads();  // the merge area and the list are free again
    }
    if (even) break;
    // ---- the next segment
    pos = end + kD8SegCost;
    if (++h == a.c.Hkv) {
      h = 0;
      ++b;
    }
  }

  // ---- segments that this workgroup shares with others, two at most: the last of a
  // segment's workgroups merges the states, in list order.  One workgroup reads them at a CU's
  // own rate, 0.1 us for those of 8 heads, so more than n_merge go in two steps: the last of a
  // group of sqrt(n) of them puts its sum in place of the group's first, and the last group's
  // merges the sums (131072 keys, 8 heads: 1 kv head 29.3 -> 17.1 us, 2 of 8 25.4 -> 21.9,
  // two sequences 44.4 -> 27.0; but 32 states of 8 heads 50.5 -> 53.2, 21 of them in four waves
  // 27.0 -> 28.6).
  if (!shared) return;
  auto group_of = [&](int n) { return (int)ceilf(sqrtf((float)n)); };
  auto arrive = [&](int i, int n) {
    const bool last = __hip_atomic_fetch_add(a.counters + i, 1, __ATOMIC_RELAXED,
                                             __HIP_MEMORY_SCOPE_AGENT) == n - 1;
    if (last) a.counters[i] = 0;  // as the next call expects it
    return last;
  };
  wait_vmem();  // this wave's states have arrived
  __syncthreads();
  if (tid < 2) {
    const int n = sm.due[tid].n, wf = sm.due[tid].wf;
    bool last = false;
    if (n > 0) {
      if (n <= a.n_merge) {
        last = arrive(wf, n);
      } else {
        const int gs = group_of(n), first = (w - wf) / gs * gs;
        last = arrive(first == 0 ? wf : kD8MaxWg + wf + first, min(gs, n - first));
      }
    }
    sm.last[tid] = last;
  }
  __syncthreads();
  const int j = tid >> 5, l32 = tid & 31, c4 = 4 * l32;
  // sets of 32 g threads: a thread has four channels of a head, a set every n_sets-th part
  const int n_sets = a.n_sets;
  const int set = j / a.g, head = j - set * a.g;
  for (int slot = 0; slot < 2; ++slot) {
    if (!sm.last[slot]) continue;
    const int n_all = __builtin_amdgcn_readfirstlane(sm.due[slot].n);
    const int wf = __builtin_amdgcn_readfirstlane(sm.due[slot].wf);
    // the states of parts first + step p, p < n, as the sums of the sets in LDS ...
    auto merge = [&](int first, int step, int n) __attribute__((always_inline)) {
      const uint32_t at0 = state_at(a, wf + first, false, head), more = state_at(a, step, false, 0);
      const uint32_t begins = first == 0 ? state_at(a, 0, true, 0) : 0;
      auto state = [&](int p) { return at0 + (uint32_t)p * more + (p == 0 ? begins : 0); };
      if (set < n_sets) {
        f32x4 num = f32x4{};
        float M = -INFINITY, den = 0.f;
        constexpr int kBatch = 8;
        for (int p0 = set; p0 < n; p0 += kBatch * n_sets) {
          f32x4 x[kBatch];
          float2 ml[kBatch];
#pragma unroll
          for (int i = 0; i < kBatch; ++i) {
            const uint32_t at = state(min(p0 + i * n_sets, n - 1));
            ml[i] = get2(states, at);
            x[i] = get4(states, at + 16 + 4 * c4);
          }
          float top = M;
#pragma unroll
          for (int i = 0; i < kBatch; ++i) {
            if (p0 + i * n_sets >= n) ml[i] = make_float2(-INFINITY, 0.f);
            top = fmaxf(top, ml[i].x);
          }
          const float use = top == -INFINITY ? 0.f : top;
          const float old = M == top ? 1.f : fast_exp2(M - use);
          den *= old;
          num *= old;
#pragma unroll
          for (int i = 0; i < kBatch; ++i) {
            const float wt = ml[i].x == top && top != -INFINITY ? 1.f : fast_exp2(ml[i].x - use);
            den += wt * ml[i].y;
            num += wt * x[i];
          }
          M = top;
        }
        *(f32x4*)&sm.set_o[j][c4] = num;
        if (l32 == 0) {
          sm.set_m[j] = M;
          sm.set_l[j] = den;
        }
      }
      __syncthreads();
    };
    // ... and the sets' as one, of head j
    auto sum = [&](float& M, float& den, f32x4& num) __attribute__((always_inline)) {
      M = -INFINITY;
      for (int t = 0; t < n_sets; ++t) M = fmaxf(M, sm.set_m[j + t * a.g]);
      den = 0.f;
      num = f32x4{};
      for (int t = 0; t < n_sets; ++t) {
        const float mx = sm.set_m[j + t * a.g];
        const float wt = mx == M ? 1.f : fast_exp2(mx - M);
        den += wt * sm.set_l[j + t * a.g];
        num += wt * *(const f32x4*)&sm.set_o[j + t * a.g][c4];
      }
    };
    auto finish = [&]() __attribute__((always_inline)) {
      if (j < a.g) {
        float M, den;
        f32x4 num;
        sum(M, den, num);
        bf16x4 r;
#pragma unroll
        for (int i = 0; i < 4; ++i) r[i] = (__bf16)(den == 0.f ? 0.f : num[i] / den);
        *(bf16x4*)(a.o + sm.due[slot].o + (size_t)j * kHeadDim + c4) = r;
      }
    };
    if (n_all <= a.n_merge) {
      merge(0, 1, n_all);
      finish();
    } else {
      const int gs = __builtin_amdgcn_readfirstlane(group_of(n_all));
      const int first = (w - wf) / gs * gs, groups = (n_all + gs - 1) / gs;
      merge(first, 1, min(gs, n_all - first));
      if (j < a.g) {
        float M, den;
        f32x4 num;
        sum(M, den, num);
        const uint32_t at = state_at(a, wf + first, first == 0, j);
        put4(states, at + 16 + 4 * c4, num);
        if (c4 == 0) put4(states, at, f32x4{M, den, 0.f, 0.f});
      }
      wait_vmem();
      __syncthreads();
      if (tid == 0) sm.last[slot] = arrive(kD8MaxWg + wf + 1, groups);  // no group begins there
      __syncthreads();
      if (sm.last[slot]) {
        merge(0, gs, groups);
        finish();
      }
    }
    __syncthreads();  // the sums are read
  }
}

// ---------------------------------------------------------------- launcher
int cu_count();

size_t offset_rows_bytes() { return kD8TabBytes; }
hipError_t launch_offset_rows(const float2* table, void* out, hipStream_t stream) {
  hipLaunchKernelGGL(offset_rows_kernel, dim3((kD8TabBytes / 4 + 255) / 256), dim3(256), 0, stream,
                     table, (unsigned char*)out);
  return hipGetLastError();
}

size_t decode8_workspace_bytes(int g) {
  return kD8Counters * sizeof(int) + (size_t)2 * kD8MaxWg * g * kD8State * sizeof(float);
}

// list entries of a segment of n steps: those of a call must stay below 2^31
long long decode8_entries(int n) { return (long long)n + kD8SegCost; }

hipError_t launch_decode8(bool bifocal, const Cache8& c, const uint16_t* q, const int32_t* kv_lens,
                          const int32_t* blocks, int n_select, uint16_t* o, const float2* table,
                          const void* offsets, int B, int Hq, int w_pre, int w0, void* ws,
                          hipStream_t stream, hipEvent_t ev0, hipEvent_t ev1) {
  static_assert(2 * kD8MaxWg <= kD8Counters, "two counters per workgroup");
  // One sequence: at least four workgroups for each of its heads.
  // Lists, where there is one for each of most CUs: a workgroup of eight waves for each, and no
  // state to merge (256 lists of 32 blocks 31.6 us in four waves and two workgroups a list, 27.5;
  // 200 of 128 76.5, 68.1; but 512 of 32 48.8, 53.3).  The other CUs have no work then, so long
  // lists get three workgroups of four waves each where as many fit (136 of 512 204 -> 184 us, of
  // 200 85.0 -> 80.3; 160 of 512 214 -> 205; 176 of 512, where two fit, would take 225 -> 255).
  // Up to two lists a CU: a workgroup of four waves for each, none to merge, but some CUs have one
  // and some two, so up to one and a half a CU long lists are cut into equal ranges (264 lists of
  // 128 127 -> 98.6 us, of 512 477 -> 334; 320 of 512 490 -> 403; 360 of 180 183 -> 175; but 320
  // of 32 39.5 -> 40.5, 440 of 512 541 -> 551).
  // Long are lists of which idle CUs could take more than 80 steps each: the crossings lie
  // between 45 (136 lists) and 75 (160), and between 20 (264) and 75 (360).
  const int cus = std::min(cu_count(), kD8MaxWg / 2);
  const long long segs = (long long)B * c.Hkv;
  auto is_long = [&](long long slots) { return n_select * (slots - segs) > 80LL * cus; };
  const bool wide = 2 * segs > cus && segs <= cus && (3 * segs > 2 * cus || !is_long(cus));
  const bool cut = segs > 2 * cus || (segs > cus && 2 * segs <= 3 * cus && is_long(2 * cus));
  const int mode = blocks == nullptr ? (B == 1 && c.Hkv <= 64 ? kOne8 : kBatch8)
                                     : (wide ? kWideList8 : kListed8);
  const int waves = decode8_waves(mode);
  const int per_cu = 8 / waves;  // registers for two waves per SIMD
  Decode8Args a{c, q, kv_lens, blocks, o, table, (const unsigned char*)offsets, (int*)ws,
                (float*)ws + kD8Counters, B, Hq, Hq / c.Hkv, n_select,
                std::max(per_cu * cus, mode == kOne8 ? c.Hkv : 1),
                w_pre, w0, !cut,
                2 * waves / (Hq / c.Hkv), 256 / (Hq / c.Hkv),
                1.4426950408889634f / sqrtf((float)kHeadDim)};
  const dim3 grid(a.n_wg), block(64 * waves);
  // ev0 / ev1 (optional) are recorded on the stream around the kernel
  hipError_t e;
  if (ev0 != nullptr && (e = hipEventRecord(ev0, stream)) != hipSuccess) return e;
#define JL_DECODE8(bif, m) hipLaunchKernelGGL((decode8_kernel<bif, m>), grid, block, 0, stream, a)
  if (bifocal) {
    if (mode == kListed8) JL_DECODE8(true, kListed8);
    else if (mode == kWideList8) JL_DECODE8(true, kWideList8);
    else if (mode == kOne8) JL_DECODE8(true, kOne8);
    else JL_DECODE8(true, kBatch8);
  } else {
    if (mode == kListed8) JL_DECODE8(false, kListed8);
    else if (mode == kWideList8) JL_DECODE8(false, kWideList8);
    else if (mode == kOne8) JL_DECODE8(false, kOne8);
    else JL_DECODE8(false, kBatch8);
  }
#undef JL_DECODE8
  e = hipGetLastError();
  if (e == hipSuccess && ev1 != nullptr) e = hipEventRecord(ev1, stream);
  return e;
}

}  // namespace jl
