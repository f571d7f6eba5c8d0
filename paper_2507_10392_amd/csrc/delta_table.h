// Where the chunks of a document stand in the table of a microbatch's chunks (delta_chunks_kernel), in the host's and the device's arithmetic.
//
// Offsets that fall make documents overlap: documents of T = 2^26 tokens each are 2^20 chunks each, and 2^18 such documents 2^38 together, beyond 32 bits
// and beyond the table.  So chunks are counted within a turn of DELTA_TURN documents, where there are 2^30 of them at most, and what a turn ends with is cut
// to the chunks that the table has room for (2^20 + 2^18 at most), behind which every document is empty.  Offsets that rise never reach either.
#pragma once

namespace zs {

constexpr int DELTA_MAX_TOKENS = 1 << 26, DELTA_MAX_DOCS = 1 << 18;
constexpr int DELTA_CHUNK = 64;    // tokens of a document that are worked on together
constexpr int DELTA_TURN = 1024;   // documents that the table's kernel takes at a time
static_assert((long long)DELTA_TURN * (DELTA_MAX_TOKENS / DELTA_CHUNK) + DELTA_MAX_TOKENS / DELTA_CHUNK + DELTA_MAX_DOCS < 1ll << 31, "");
static_assert(DELTA_MAX_TOKENS + (long long)DELTA_CHUNK * DELTA_MAX_DOCS < 1ll << 31, "");

__host__ __device__ inline int delta_chunks_of(int tokens) { return (tokens + DELTA_CHUNK - 1) / DELTA_CHUNK; }
// Chunks of all turns up to one that has `turn` of them behind `before`.
__host__ __device__ inline int delta_turn_end(int before, int turn, int nchunks) { return before + turn < nchunks ? before + turn : nchunks; }
// A document's first chunk, with `in_turn` chunks of its turn in front of it, and those of its tokens that the table has room for.
struct DeltaPlace { int chunk0, tokens; };
__host__ __device__ inline DeltaPlace delta_place(int before, int in_turn, int tokens, int nchunks) {
  const int chunk0 = delta_turn_end(before, in_turn, nchunks), room = (nchunks - chunk0) * DELTA_CHUNK;
  return DeltaPlace{chunk0, tokens < room ? tokens : room};
}

}  // namespace zs
