// decode_shared.h -- limits of the decode over shared prefixes, as the host layer checks them.
#pragma once

namespace jl {
constexpr int kShMaxWg = 256;     // workgroups in all: one per CU
constexpr int kShMaxSeqs = 2048;  // sequences and groups of a plan: its lists lie in LDS
}  // namespace jl
