// pages.h -- what the page kernels and the host layer share: the tables of a
// batch of sequences over one pool of pages, and the pools that moves copy.
#pragma once

#include <stddef.h>
#include <stdint.h>

namespace jl {

// table [B][max_pages], lens [B], refs [n_pages].  A sequence of lens[b] tokens
// names its pages in the first ceil(lens[b] / page) entries of its row, the others
// are -1; refs[p] is how many entries name page p.
struct Pages {
  int32_t* table;
  int32_t* lens;
  int32_t* refs;
  int B, max_pages, n_pages, page;
};

constexpr int kPagesMaxSeqs = 2048;   // rows of one call: their bookkeeping lies in LDS
constexpr int kPagesMaxPages = 1 << 30;

// Pools whose pages one copy launch moves: page p of pool i is `bytes[i]` bytes at
// ptr[i] + p * bytes[i].
constexpr int kCopyPools = 64;
struct CopyPools {
  unsigned char* ptr[kCopyPools];
  unsigned long long bytes[kCopyPools];
  int first[kCopyPools + 1];  // units of a move before pool i
  int n_pools, n_pages, max_moves;
};

}  // namespace jl
