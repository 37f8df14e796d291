// Shared declarations of what several continuations of a prompt need: pages that are shared (pages.hip), the selection over beams and
// vocabulary (beam.hip), and the attention of rows with common leading blocks (shared_attention.hip).
#pragma once

#include "ee_common.h"

namespace ee {

// ---- pages.hip ---------------------------------------------------------------------------------------------------
struct PageRows {
  int32_t* tables;   // [rows][max_blocks]
  int32_t* lens;     // [rows]
  int rows, max_blocks;
};
constexpr int kPageChunk = 1024;   // block ids of a chunk: a bit each in 16 words, and their number

// What the calls keep between their launches.
struct PageWork {
  uint64_t* taken;     // [chunks][16]: a bit for each block that has references
  int32_t* counts;     // [chunks]: their number
  int32_t* claims;     // [num_blocks]: rows of a call that write the block
  int32_t* latest;     // [num_blocks]: the last of these rows
  int32_t* row_first;  // [rows + 1]: blocks that the rows before want
  int32_t* replaces;   // [rows]: whether the row's last block is replaced
};
inline int page_chunks(int num_blocks) { return (num_blocks + kPageChunk - 1) / kPageChunk; }

void launch_pages_fork(int32_t* refs, int num_blocks, const PageRows& src, const int32_t* parents, const PageRows& dst, hipStream_t st);
void launch_pages_release(int32_t* refs, int num_blocks, const PageRows& r, hipStream_t st);
void launch_pages_grow(int32_t* refs, int num_blocks, const PageRows& r, const int32_t* new_lens, int32_t* moves, int32_t* missing, const PageWork& w,
                       hipStream_t st);
void launch_pages_compact(int32_t* refs, int num_blocks, const PageRows& r, int32_t* remap, int32_t* moves, int32_t* n_moves, const PageWork& w, hipStream_t st);
void launch_pages_shared(const PageRows& r, const int32_t* first_row, int n_groups, int32_t* shared, hipStream_t st);

// Pools of a cache whose blocks are copied: `planes` of [num_blocks] blocks each (layers one after the other).
struct PagePlane {
  char* base;
  size_t block_bytes;   // a multiple of 8, of 16 where `base` starts on 16
  int planes;
  int pieces, wide;     // set by the launch: pieces of one block in all planes; whether they are copied in 16 bytes
};
struct PageCopyArgs {
  PagePlane pool[3];
  int n_pools, num_blocks, pieces;
  const int32_t* moves;   // [n][2]
  const int32_t* count;   // nullptr, or how many of them there are
  int n;
};
void launch_pages_copy(PageCopyArgs a, hipStream_t st);

// ---- beam.hip ------------------------------------------------------------------------------------------------------
constexpr int kBeamMost = 128;     // beams of a group, and candidates that come back of one
constexpr int kBeamFewOut = 32;    // up to so many of a group, the scan's chunks are the smaller ones
constexpr int kBeamWgs = 1536;     // workgroups of the scan that run at once
struct BeamArgs {
  const void* logits;        // [rows][stride]
  int64_t stride;
  const float* scores;       // [rows]
  const int32_t* finished;   // nullptr, or [rows]
  int groups, beams, vocab, n_out, end_token;
  int32_t *tokens, *parents, *finished_out;   // [groups * n_out]; finished_out may be nullptr
  float* scores_out;
  int chunks;                // of a row
  int threads, each;         // workgroup of the scan, and values of a thread
  double2* stats;            // [rows][chunks]: maximum and sum of exponentials relative to it
  uint64_t* found;           // [groups][n_out][beams][chunks]: key of the logit and complement of its token, falling along n_out; 0: none
};
void beam_plan(BeamArgs& a);   // chunks, threads, each
int64_t beam_most_chunks(int64_t rows, int vocab, bool few);   // of all rows of a call up to these sizes; few: up to kBeamFewOut come back
void launch_beam_select(const BeamArgs& a, int dtype, hipStream_t st);
struct RowCopyArgs {
  const char* in;
  char* out;
  int64_t in_stride, out_stride, row_bytes;
  const int32_t* parents;
  int in_rows, rows;
};
void launch_reorder_rows(const RowCopyArgs& a, hipStream_t st);

// ---- shared_attention.hip --------------------------------------------------------------------------------------------
struct SharedAttnArgs {
  const float* q;
  float* out;
  const void *k, *v;           // layer base [num_blocks][kv_heads][16][dh]
  const int32_t *context_lens, *block_tables, *row_table;
  int max_blocks, rows, kv_heads, group, dh, num_blocks;
  const int32_t *first_row, *shared_blocks;
  int n_groups, max_shared, max_context;
  // Set by shared_attn_plan: columns (a row and one of its query heads) of a tile, tiles, and workgroups of a K/V head that are dealt out to the tiles (0: one a tile).
  int columns, rows_per_tile, head_chunks, tiles, dealt;
  int4* tile_of;               // dealt: [tiles]: first row, rows, first workgroup and how many
  float* records;              // dealt: [head chunks][kv heads][workgroup][columns][dh + 4]: maximum, sum, -, -, sums of V
};
void shared_attn_plan(SharedAttnArgs& a, int dtype);
size_t shared_attn_record_floats(const SharedAttnArgs& a);
// The most that calls of up to a's rows, groups and context need: floats of records, and tiles.
size_t shared_attn_most_floats(SharedAttnArgs& a, int dtype, size_t* tiles);
void launch_shared_attention(const SharedAttnArgs& a, int dtype, hipStream_t st);

}  // namespace ee
