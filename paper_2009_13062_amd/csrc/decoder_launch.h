// Launches of the decoders' tiled kernels, defined in the translation units that instantiate them.
#pragma once
#include "decoder.h"

namespace nf {

// Keys of a cache that one workgroup takes: by the rows that read it alone, so that a sequence's bits do not depend on what is merged with it or
// on the capacity.  Partial sums cost 8 bytes per row and feature and chunk, the cache 4 (bfloat16) per key and feature: with 16 keys per row they stay below an
// eighth of it; below 512 keys a chunk is not worth its own start.
inline int tree_chunk(int rows) {
  int chunk = 512;
  while (chunk < 16LL * rows && chunk < 1024) chunk *= 2;
  return chunk;
}
inline int tree_features(int d) { return d <= 64 ? 64 : d <= 128 ? 128 : 256; }

struct WeighArgs;
// decoder_tiles.h: bfloat16
nf_status launch_prompt_tiles(const DecArgs& a, hipStream_t s);
nf_status launch_tree_tiles(const DecArgs& a, int chunk, int splits, hipStream_t s);
// decoder_stream.h: float32 prompts, trees of either type
nf_status launch_prompt_stream(const DecArgs& a, hipStream_t s);
nf_status launch_tree_stream(const DecArgs& a, int chunk, int splits, nf_dtype dt, hipStream_t s);
nf_status launch_tree_join(const DecArgs& a, int chunk, int splits, nf_dtype dt, hipStream_t s);
nf_status launch_weigh_tiles(const WeighArgs& a, nf_dtype dt, hipStream_t s);

}  // namespace nf
