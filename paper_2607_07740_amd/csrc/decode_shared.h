// decode_shared.h -- limits of the rows over paged caches (shared prefixes, packed chunks), as
// the host layer checks them.
#pragma once

namespace jl {
constexpr int kShMaxWg = 256;     // workgroups in all: one per CU
constexpr int kShMaxSeqs = 2048;  // sequences and groups of a plan: its lists lie in LDS
constexpr int kShMaxGroup = 256;  // query heads of a kv head: a token's rows fit one segment
}  // namespace jl
