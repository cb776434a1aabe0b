// prefill_chunks.h -- what the planning kernel of packed chunks (decode_shared.hip) hands to the
// prefill kernel: parts of query blocks.
#pragma once

namespace jl {

constexpr int kChunkBlockRows = 256;  // rows of a block: (query head of a kv head, token)
constexpr int kChunkTile = 64;        // keys of a visit
constexpr int kChunkMinPart = 16;     // visits of a part at least

struct ChunkPart {
  int seq, row0, n, L;           // sequence, its first packed row, its rows, its keys
  int block, part, parts, slot;  // block of its rows; part of how many, whose states begin at slot
  int G, pad[3];
};

}  // namespace jl
