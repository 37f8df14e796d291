// Shared declarations of the 8-bit cache and of the rotary embedding on its own (rotary.hip, quant_cache.hip,
// quant_attention.hip): launch interfaces, and what a byte of the cache stands for.
#pragma once

#include <type_traits>

#include "ee_common.h"

namespace ee {

typedef _Float16 half_t;
typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
typedef _Float16 half8_t __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef bf16_t bf16x2 __attribute__((ext_vector_type(2)));

constexpr float kQuantScaleFloor = 1.17549435e-38f;   // 2^-126: a block of zeros; its reciprocal is finite
constexpr int kQuantMaxHeadDim = 256;

// rotary.hip
struct RotaryRows {
  const void* in;
  void* out;
  int64_t in_stride, out_stride;   // elements
  int n_heads;
};
struct RotaryArgs {
  const double* freqs;
  const int32_t* positions;
  RotaryRows q, k;   // n_heads == 0: none
  int rows, head_dim, rotary_dim;
  float amplitude;
  float sign;        // +1, or -1 for the transposed rotation
};
void launch_rotary_frequencies(const ee_rotary_desc& d, double* freqs, hipStream_t st);
void launch_rotary(const RotaryArgs& a, int dtype, int layout, hipStream_t st);

// One layer of an 8-bit cache.
struct QuantCache {
  int8_t* k;       // [num_blocks][heads][16][dh]
  int8_t* v;       // [num_blocks][heads][dh][16]
  float* scales;   // [num_blocks][heads][2]
  int num_blocks, heads, dh, format;
};
// Rows of a call and where their positions live.
struct QuantRows {
  const int32_t* context_lens;
  const int32_t* block_tables;
  const int32_t* row_table;   // nullptr: row m is sequence m
  int rows, max_blocks;
};

// quant_cache.hip
struct QuantAppendArgs {
  QuantCache c;
  QuantRows r;
  const void *k, *v;
  int64_t k_stride, v_stride;
};
void launch_quant_append(const QuantAppendArgs& a, int dtype, hipStream_t st);
struct QuantReadArgs {
  QuantCache c;
  QuantRows r;
  void *k, *v;
};
void launch_quant_read(const QuantReadArgs& a, int dtype, hipStream_t st);
struct QuantEvictArgs {
  QuantCache c;
  QuantRows r;
  const int32_t* dst_tables;   // nullptr: in place, by way of `images`
  int dst_max_blocks;
  const float* weights_in;
  float* weights_out;
  int pitch_in, pitch_out;
  int max_context, keep, recent;
  int32_t* kept;
  int32_t* out_lens;
  int8_t* images;              // [B][heads][blocks of keep][2][16 * dh]
  float* image_scales;         // [B][heads][blocks of keep][2]
};
void launch_quant_evict(const QuantEvictArgs& a, hipStream_t st);

// quant_attention.hip
struct QuantAttnArgs {
  QuantCache c;
  QuantRows r;
  int n_heads, max_context;
  const float* q;
  float* out;
  const float* weights_in;
  float* weights_out;          // nullptr: none
  int weights_pitch;
  // A context's parts leave records of head_dim + 4 floats: running maximum's reference, sum, -, -, the part's own result.
  //   row_table: [rows][n_heads][n_parts], n_parts > 1;   else [kv heads][slots][columns of a tile] (see quant_attn_plan).
  float* parts;                // nullptr: none
  int2* spans;                 // dealt: [rows * tiles] first workgroup and number of workgroups that have a unit's steps
  float* scores;               // weights: [rows][n_heads][quant_score_pitch(max_context)], in units of log 2
  int n_parts, part_steps;     // row_table: parts of a context, and 64-position steps of a part
  bool whole;                  // else: whether there is a launch in which contexts are whole pieces
  int dealt;                   // 0, or workgroups of a K/V head that all rows' steps are dealt out to
  int long_steps;              // with both: contexts of more steps than this are dealt out (0: all)
  int slots;
};
__host__ __device__ inline size_t quant_score_pitch(int max_context) { return (size_t)((max_context + 63) / 64) * 64; }
// How a call's work is divided (sets n_parts, part_steps, whole, dealt, long_steps), and the floats of `parts` that it needs, and entries of `spans`; the former for
// all calls of up to so many rows and positions.
size_t quant_attn_plan(QuantAttnArgs& a, size_t* spans);
size_t quant_attn_part_floats(const QuantCache& c, int n_heads, int max_rows, int max_context, bool weights);
constexpr int kQuantMostSpans = 1024;
// Tiles of a K/V head: of up to 16 heads of one row, or of 32 (row, head) pairs with row_table.
int64_t quant_attn_tiles(int rows, int group, bool row_table);
void launch_quant_attention(const QuantAttnArgs& a, hipStream_t st);

#ifdef __HIPCC__
// The maximum of a wavefront's 64 values (of magnitudes' bits, which are ordered like integers), on the cross-lane network.
__device__ inline uint32_t wave_max(uint32_t v) {
  auto with = [&](auto ctrl, auto rows) { v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, decltype(ctrl)::value, decltype(rows)::value, 0xf, false)); };
  with(std::integral_constant<int, 0x111>{}, std::integral_constant<int, 0xf>{});   // row_shr 1, 2, 4, 8: lane 15 of each 16 has theirs
  with(std::integral_constant<int, 0x112>{}, std::integral_constant<int, 0xf>{});
  with(std::integral_constant<int, 0x114>{}, std::integral_constant<int, 0xf>{});
  with(std::integral_constant<int, 0x118>{}, std::integral_constant<int, 0xf>{});
  with(std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xa>{});   // row_bcast 15, 31: lane 63 has all
  with(std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xc>{});
  return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}
__device__ inline int lane_value(int v, int lane) { return __builtin_amdgcn_readlane(v, lane); }
__device__ inline float lane_value(float v, int lane) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane)); }

__device__ inline int quant_seq(const QuantRows& r, int m) { return r.row_table ? safe_row(r.row_table[m], r.rows) : m; }
#endif

}  // namespace ee
