// Launches of the decoders' tiled kernels, defined in the translation units that instantiate them.
#pragma once
#include "decoder.h"

namespace nf {

// Keys of a cache that one workgroup takes: by type and by the rows that read it alone, so that a sequence's bits do not depend on what is merged with it or
// on the capacity.  512 where few rows read it (8 key heads, one token of a group of 4, us, 256 / 512 / 1024 / 2048 keys: bfloat16, 32 models of 4 caches of 1024 entries
// 79 / 69 / 64 / 65 at 64 features; float32, one cache of 4096 16 / 18 / 24 / 37, 8 of them 44 / 40 / 44 / 44).  Partial sums cost 8 bytes per row and
// feature and chunk, the cache 4 (bfloat16) or 8 per key and feature: from 33 rows (65 in float32) on 1024 (512 / 1024 / 2048: bfloat16 of 128 features, 26 tokens, 16 caches of 4096
// 103 / 83 / 104, 64 tokens over one of 8192 36 / 49 / 81, 16 tokens over 32 of 8192 370 / 292; float32, 12 tokens over 16 of 4096, 2 heads 59 / 101, 8 heads 201 / 198,
// 64 tokens 754 / 702).
inline int tree_chunk(int rows, nf_dtype dt) { return rows > (dt == NF_F32 ? 64 : 32) ? 1024 : 512; }
inline int tree_features(int d) { return d <= 64 ? 64 : d <= 128 ? 128 : 256; }

// Of a cache of 4 bits, whose chunks are shorter in bytes: one length for any rows and either type, between what few caches and what many would have (8 key heads of 128, groups of 4, caches of 4096
// unless said, us, 512 / 1024 / 2048 keys.  bfloat16, one token over 1 cache 11.6 / 13.6 / 18.2, over 32 40 / 34 / 30, over two of 100000 54 / 48 / 47; 5 tokens over 8 22.8 / 23.3 / 35, over 32
// 66 / 58 / 55; 9 over 16 57 / 49 / 71; 26 over 1 28 / 42 / 71, over 8 39 / 46 / 74, over 32 132 / 108 / 103; 64 over 32 267 / 215 / 195.  float32, one token over 1 14 / 18 / 24, over 32
// 53 / 43 / 40; 5 over 1 20 / 28 / 43, over 8 30 / 30 / 48, over 32 88 / 77 / 76; 26 over 1 30 / 45 / 76, over 8 87 / 79 / 87, over 32 301 / 268 / 250).  The caches that are merged may not choose
// it, as a sequence's bits would follow from them.
constexpr int kTreeFp4Chunk = 1024;
// Rows of bfloat16 up to which it is streamed; more go through LDS, as with caches of bfloat16, but from 65 up where heads are large (36 rows of 256 features over 8 caches of 4096, us, registers /
// LDS 64 / 79, 104 rows - / 88; of 128, 36 rows over 16 51 / 48, 32 over 32 84 / 115; of 64, 20 rows over 16 32.7 / 31.5).
constexpr int tree_fp4_streamed(int d) { return d <= 64 ? 16 : d <= 128 ? 32 : 64; }
nf_status launch_tree_fp4_tiles(const DecArgs& a, int chunk, int splits, hipStream_t s);        // bfloat16
nf_status launch_tree_fp4_stream(const DecArgs& a, int chunk, int splits, nf_dtype dt, hipStream_t s);

struct WeighArgs;
// decoder_tiles.h: bfloat16
nf_status launch_prompt_tiles(const DecArgs& a, hipStream_t s);
nf_status launch_tree_tiles(const DecArgs& a, int chunk, int splits, hipStream_t s);
// decoder_stream.h: float32 prompts, trees of either type
nf_status launch_prompt_stream(const DecArgs& a, hipStream_t s);
nf_status launch_tree_stream(const DecArgs& a, int chunk, int splits, nf_dtype dt, hipStream_t s);
long long tree_join_blocks(const DecArgs& a, int splits);       // workgroups of 256
nf_status launch_tree_join(const DecArgs& a, int chunk, int splits, nf_dtype dt, hipStream_t s);
nf_status launch_weigh_tiles(const WeighArgs& a, nf_dtype dt, hipStream_t s);

}  // namespace nf
