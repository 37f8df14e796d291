// Attention over the 8-bit cache, on the matrix cores.
//
// A workgroup has up to 16 or 32 columns, (row, query head) pairs that read the same K/V head: the grouped heads of one row, or of prompt rows.
// A wavefront takes 64 positions (four blocks T_0..T_3) a step and multiplies
//   S = K Q^T:  16 positions x 32 channels x 16 columns an instruction, the positions of instruction i being 4i..4i+3 of each block, so that
//               lane (column n, group g) ends up with the scores of all 16 positions of block T_g;
//   O += V^T P: 16 channels x 32 positions x 16 columns, contracted over positions 8h..8h+7 of each block: lane (n, g) has those
//               eight probabilities already, and the bytes of a channel's 16 positions are consecutive in V's blocks.
// No value crosses lanes but the running maxima, and every load is 16 bytes a lane.  Bytes become fp16 without error.  q (scaled by a power of two
// to 2^13..2^14) and the probabilities (times the block's scale of V, in units of their own) are split into an fp16 head and remainder: 22 bits
// together, as far as the remainder's last place, 2^-24, allows.  A channel of q is off by 2^-38 of its row's largest at least, a weighted probability by 2^-37
// of the largest probability times scale that its row has had.
// Softmax statistics and results are float, running over a wavefront's steps; the wavefronts of a unit, and the parts of a context that
// several workgroups have, are joined in a fixed order.
// A column has two references, both whole powers of two, so that changing them rounds nothing:
//   2^m for the sum: m is 32 below the largest score so far (in units of log 2, rounded up).  A probability is then a float, not 0, down to 2^-158 of
//       the largest, and a block's scale times 2^(m - ..) stays a float where one with a small scale has the largest score;
//   2^(m + r - 15) for the result: r follows the blocks' largest scores and scales together, over the positions that the column attends.  With the
//       largest scale alone, a block that hardly counts (or another sequence's in the tile, or a later one's) would push all others into fp16's last places.
//
// Single rows are bound by the cache's bytes (head_dim 128, shuffled blocks; a plain read of this card makes 6.3 to 6.8 TB/s): one sequence of 131000 positions,
// 8 K/V heads, 268 MB: 48 us (5.6 TB/s) and 5 to join 64 parts; 64 of 2000 to 6000: 96 us (5.4 TB/s) + 6; 32 of 576, 32 heads: 30 us (5.1).
// Without products, or without softmax, these times hardly change; two workgroups a compute unit with a step's 16 KB a wavefront in flight are
// enough, three were no faster.  What is left is the beginning and end of a workgroup, about 2 us each.  512 prompt rows of four prompts up to
// 3100 positions, 4 heads to a K/V head: 46 us, 25 GFLOP (12.6 in two pieces each).  All tiles are resident at once, and a K/V head's 64 have 1 to 49 steps (mean 25): the
// call takes as long as the longest and what shares its compute unit.  Within a step it is the issue of instructions (about 600 vector and 128 matrix ones): prompts of
// 12000 positions, tiles of one length, make 860 TFLOP/s, three quarters of a large matrix product's.  Weights cost 27 us of the 64 sequences' call: 33 MB of scores written among 524 MB of reads (24 us;
// with stores that are dropped the launch takes 98), and 9 to read them.
#include "quant.h"

namespace ee {

namespace {

constexpr int kWaves = 4, kThreads = 64 * kWaves;
constexpr int kTableSteps = 256;     // steps whose block ids and scales are in LDS at a time
constexpr int kDealtRows = kQuantMostSpans;   // rows (tiles of them) whose steps are dealt out evenly, at most: every workgroup adds up their lengths
constexpr int kResident = 512;       // workgroups at once: two a compute unit
constexpr float kLog2e = 1.4426950408889634f;
// Scores beyond this are rounded before the reference is taken off, as the largest one was; a fused subtraction would leave what that rounding took, a large number.
constexpr float kLargeScore = 1048576.0f;
constexpr float kBelow = 32.0f;      // how far a column's reference is below its largest score

// Eight bytes -> eight fp16.
template <int FMT>
__device__ inline half8_t widen(uint32_t a, uint32_t b) {
  half2_t h[4];
  if constexpr (FMT == EE_QUANT_INT8) {
    // byte + 128 below the exponent of 1024 is the number 1024 + byte + 128
    a ^= 0x80808080u;
    b ^= 0x80808080u;
    const half2_t off = {(half_t)1152.0f, (half_t)1152.0f};
    h[0] = __builtin_bit_cast(half2_t, __builtin_amdgcn_perm(0x64646464u, a, 0x04010400u)) - off;
    h[1] = __builtin_bit_cast(half2_t, __builtin_amdgcn_perm(0x64646464u, a, 0x04030402u)) - off;
    h[2] = __builtin_bit_cast(half2_t, __builtin_amdgcn_perm(0x64646464u, b, 0x04010400u)) - off;
    h[3] = __builtin_bit_cast(half2_t, __builtin_amdgcn_perm(0x64646464u, b, 0x04030402u)) - off;
  } else {
    h[0] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.0f, false);
    h[1] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.0f, true);
    h[2] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.0f, false);
    h[3] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.0f, true);
  }
  return half8_t{h[0][0], h[0][1], h[1][0], h[1][1], h[2][0], h[2][1], h[3][0], h[3][1]};
}

__device__ inline f32x4 mma(half8_t a, half8_t b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

// Two floats as an fp16 head and remainder.
__device__ inline void split(f32x2 x, half2_t& hi, half2_t& lo) {
  hi = __builtin_convertvector(x, half2_t);
  lo = __builtin_convertvector(f32x2{x[0] - (float)hi[0], x[1] - (float)hi[1]}, half2_t);
}

__device__ inline float largest(const f32x4 (&x)[4]) {
  float v = x[0][0];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) v = fmaxf(v, x[i][e]);
  return v;
}

// The maximum over the four lanes that share a column.
__device__ inline float max_over_groups(float v) {
  v = fmaxf(v, __shfl_xor(v, 16));
  return fmaxf(v, __shfl_xor(v, 32));
}

template <bool STREAM>
__device__ inline u32x4 load16(const int8_t* p) {
  if constexpr (STREAM)
    return __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p));
  else
    return *reinterpret_cast<const u32x4*>(p);
}

// The last position that a row with this context length attends: -1 for none.
__device__ inline int last_position(const QuantAttnArgs& a, int context_len) {
  return max(-1, min(context_len, min(a.max_context, a.r.max_blocks * 16) - 1));
}
__device__ inline int steps_to(int last) { return (last >> 6) + 1; }   // (-1: 0)
// Whether a row of so many steps is this launch's: where long contexts are dealt out and the others are not, that is two launches.
__device__ inline bool takes(const QuantAttnArgs& a, int steps) { return !a.long_steps || (steps > a.long_steps) == (a.dealt != 0); }

// Rows without row_table are cut into tiles of up to 16 of a K/V head's query heads ("units": row * tiles + tile).
__host__ __device__ inline int unit_tiles(int group) { return (group + 15) / 16; }
__host__ __device__ inline int unit_columns(int group) { return group < 16 ? group : 16; }

// The steps of all units behind each other, dealt out to `a.dealt` workgroups a K/V head: start[u] = steps of the units in front of u, and
// workgroup w has steps bound(w) .. bound(w + 1) - 1.
struct Deal {
  int total, workgroups;
  __device__ int bound(int w) const { return (int)((int64_t)w * total / workgroups); }
  __device__ int owner(int step) const { return (int)((((int64_t)step + 1) * workgroups + total - 1) / total) - 1; }
};
__device__ inline Deal deal_out(const QuantAttnArgs& a, int tiles, int* start /* LDS [kDealtRows + 1] */, int* scratch /* LDS [kWaves] */) {
  const int units = a.r.rows * tiles, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int n[4], sum = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int u = 4 * tid + e;
    n[e] = u < units ? steps_to(last_position(a, a.r.context_lens[u / tiles])) : 0;
    if (!takes(a, n[e])) n[e] = 0;
    sum += n[e];
  }
  int upto = sum;
#pragma unroll
  for (int x = 1; x < 64; x <<= 1) {
    const int o = __shfl_up(upto, x);
    if (lane >= x) upto += o;
  }
  if (lane == 63) scratch[wave] = upto;
  __syncthreads();
  int before = upto - sum, total = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    if (w < wave) before += scratch[w];
    total += scratch[w];
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if (4 * tid + e <= units) start[4 * tid + e] = before;
    before += n[e];
  }
  if (tid == kThreads - 1 && units == kDealtRows) start[units] = before;
  __syncthreads();
  // (a workgroup has two steps a wavefront at least: more parts take longer to join)
  return Deal{__builtin_amdgcn_readfirstlane(total), __builtin_amdgcn_readfirstlane(max(1, min(a.dealt, total / (2 * kWaves))))};
}

// The attention that positions j .. j + 3 got from the G heads whose maximum and 1 / sum are in head_stat.
__device__ inline void add_weights(const QuantAttnArgs& a, const f32x2* head_stat, int m, int hk, int G, int last, int j) {
  const size_t sp = quant_score_pitch(a.max_context);
  const float* s = a.scores + ((size_t)m * a.n_heads + hk * G) * sp + j;   // (rows are of whole 64 positions: four are there)
  const size_t at = ((size_t)m * a.c.heads + hk) * a.weights_pitch + j;
  f32x4 w = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
  for (int h = 0; h < G; ++h) {
    const f32x4 x = *reinterpret_cast<const f32x4*>(s + h * sp);
    const f32x2 st = head_stat[h];
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] += __builtin_amdgcn_exp2f(x[e] - st[0]) * st[1];
  }
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (j + e <= last) a.weights_out[at + e] = a.weights_in && j + e < last ? a.weights_in[at + e] + w[e] : w[e];
}

// DH: the head's channels, or 0 for a.c.dh; NL: loads of 16 bytes a lane and position (64 channels each).  SHARED: rows that may share a sequence,
// 32 columns; else units, 16 columns.
constexpr int quant_tiles(bool shared) { return shared ? 2 : 1; }
// KW: wavefronts of a unit.  With 2 a workgroup has two K/V heads of one row (the same blocks, so the loops stay in step).
template <int FMT, int DH, int NL, bool SHARED, bool WEIGHTS, int KW>
__global__ __launch_bounds__(kThreads, NL <= 2 ? 2 : 1) void quant_attn_kernel(QuantAttnArgs a) {
  constexpr int UNITS = kWaves / KW;
  constexpr int NT = quant_tiles(SHARED), C = 16 * NT, CT = 4 * NL;
  constexpr bool QREG = !SHARED;        // q's fragments in registers, or in LDS
  __shared__ half8_t q_lds[QREG ? 1 : NT * NL * 2 * 2 * 64];
  __shared__ float stat[2][kWaves][C];
  __shared__ f32x4 meet[kWaves][4][NT][64];
  __shared__ int block_id[kTableSteps * 4];      // blocks of the steps at hand, and their scales of K and V
  __shared__ f32x2 block_scale[kTableSteps * 4];
  __shared__ int start[SHARED ? 1 : kDealtRows + 1], scratch[kWaves];
  __shared__ f32x2 head_stat[UNITS][C];          // maximum, 1 / sum
  const int tid = threadIdx.x, lane = tid & 63, col = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), mine = UNITS > 1 ? wave / KW : 0, turn = wave - mine * KW;   // the unit, the wavefront's place in it
  const int dh = DH ? DH : a.c.dh, G = __builtin_amdgcn_readfirstlane(a.n_heads / a.c.heads), hk = blockIdx.x * UNITS + mine, last_entry = a.r.max_blocks - 1;
  const int tiles = SHARED ? 1 : unit_tiles(G);
  const size_t block_bytes = (size_t)16 * dh, block_pitch = block_bytes * a.c.heads;
  const int8_t* k_base = a.c.k + hk * block_bytes;
  const int8_t* v_base = a.c.v + hk * block_bytes;

  int unit = blockIdx.y, worker = blockIdx.y, at = 0, stop = 0, early = 0;
  Deal deal{};
  const bool dealt = !SHARED && UNITS == 1 && a.dealt;
  if (!SHARED && tiles > 1) {
    // the tiles of a row read the same bytes: workgroups whose ids differ by eight share a chiplet and its L2
    if (dealt) {
      if (a.dealt % 8 == 0) worker = (blockIdx.y % 8) * (a.dealt / 8) + blockIdx.y / 8;
    } else {
      const int whole = a.r.rows / 8 * 8, y = blockIdx.y, rest = y - whole * tiles;
      const int row = rest < 0 ? y / (8 * tiles) * 8 + y % 8 : whole + rest % (a.r.rows - whole);
      unit = __builtin_amdgcn_readfirstlane(row * tiles + (rest < 0 ? y / 8 % tiles : rest / (a.r.rows - whole)));
    }
  }
  if (dealt) {
    deal = deal_out(a, tiles, start, scratch);
    if (worker >= deal.workgroups) return;
    if (blockIdx.x == 0 && worker == 0)          // for the launch that joins the parts
      for (int u = tid; u < a.r.rows * tiles; u += kThreads) {
        const int first = start[u + 1] > start[u] ? deal.owner(start[u]) : 0;
        a.spans[u] = make_int2(first, start[u + 1] > start[u] ? deal.owner(start[u + 1] - 1) - first + 1 : 0);
      }
    if (deal.total == 0) return;
    at = deal.bound(worker);
    stop = deal.bound(worker + 1);
    int lower = 0;                               // the unit that step `at` belongs to: units that end in front of it
    for (int u = tid; u < a.r.rows * tiles; u += kThreads) lower += start[u + 1] <= at;
    for (int x = 1; x < 64; x <<= 1) lower += __shfl_xor(lower, x);
    if (lane == 0) scratch[wave] = lower;
    __syncthreads();
    unit = __builtin_amdgcn_readfirstlane(scratch[0] + scratch[1] + scratch[2] + scratch[3]);
  } else if (!SHARED) {
    // block ids are asked for beside the row's length (entries behind it may be anything, see below)
    early = a.r.block_tables[(size_t)(unit / tiles) * a.r.max_blocks + min(tid, last_entry)];
  }
  do {
    // ---- a piece: columns f0 .. f1 - 1, steps s0 .. s1 - 1 ----
    int f0, f1, s0 = 0, s1 = 0, unit_steps = 0;
    if constexpr (SHARED) {
      f0 = blockIdx.y * C;
      f1 = min(f0 + C, a.r.rows * G);
      s0 = blockIdx.z * a.part_steps;
    } else {
      const int m = __builtin_amdgcn_readfirstlane(unit / tiles);
      f0 = m * G + (unit - m * tiles) * C;
      f1 = min(f0 + C, (m + 1) * G);
    }
    const int r0 = __builtin_amdgcn_readfirstlane(f0 / G), n_rows = __builtin_amdgcn_readfirstlane((f1 - 1) / G) - r0 + 1;
    const int m_lane = r0 + min(lane, n_rows - 1);   // the piece's rows, one a lane
    const int ctx = a.r.context_lens[m_lane], row_seq = quant_seq(a.r, m_lane);
    if constexpr (SHARED) early = a.r.block_tables[(size_t)__builtin_amdgcn_readfirstlane(row_seq) * a.r.max_blocks + min(s0 * 4 + tid, last_entry)];
    // q: a wavefront's own in registers, or for LDS a quarter of the workgroup's (of one column tile, half of the channels): a load takes 16 bytes from
    // each of up to 64 lines, so four times the loads are four times the time.
    constexpr int QF = QREG ? 2 * NL : NL;         // fragments of 8 channels a lane
    const int q_tile = QREG ? 0 : wave % NT, q_first = QREG ? 0 : wave / NT * QF, q_col = f0 + q_tile * 16 + col;
    f32x4 qx[QF][2];
    {
      const int f = min(q_col, f1 - 1), m = f / G;
      const float* q = a.q + ((size_t)m * a.n_heads + hk * G + (f - m * G)) * dh;
#pragma unroll
      for (int k = 0; k < QF; ++k) {
        const int c = ((q_first + k) >> 1) * 64 + g * 16 + ((q_first + k) & 1) * 8;
#pragma unroll
        for (int e = 0; e < 2; ++e) qx[k][e] = *reinterpret_cast<const f32x4*>(q + (c < dh ? c : 0) + 4 * e);
      }
    }
    const int row_pos = last_position(a, ctx);
    if constexpr (SHARED) {
      if (blockIdx.z > 0 && !__any((row_pos >> 6) >= s0)) return;
    } else {
      unit_steps = __builtin_amdgcn_readfirstlane(steps_to(row_pos));
      s1 = unit_steps;
      if (!dealt && !takes(a, unit_steps)) return;
      if (dealt) {
        const int begin = __builtin_amdgcn_readfirstlane(start[unit]);
        unit_steps = __builtin_amdgcn_readfirstlane(start[unit + 1]) - begin;
        s0 = at - begin;
        s1 = min(stop - begin, unit_steps);
        at = begin + s1;
      }
    }

    // q, split; the factor that turns a product back into a score in units of log 2
    half8_t qf[QREG ? 2 * NL : 1][2];
    float to_score[NT], m_run[NT], l_run[NT], r_run[NT];
    int col_row[NT], col_pos[NT];
    float most = 0.0f;
#pragma unroll
    for (int k = 0; k < QF; ++k)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        if (q_col >= f1 || ((q_first + k) >> 1) * 64 + g * 16 >= dh) qx[k][e] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int j = 0; j < 4; ++j) most = fmaxf(most, fabsf(qx[k][e][j]));
      }
    most = max_over_groups(most);
    if constexpr (!QREG) {
      if (g == 0) stat[0][wave][col] = most;
      __syncthreads();
    }
    float up = 0.0f;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int f = f0 + nt * 16 + col;
      const bool valid = f < f1;
      col_row[nt] = (valid ? f / G : r0) - r0;
      col_pos[nt] = __shfl(row_pos, col_row[nt]);
      if (!valid) col_pos[nt] = -1;
      if constexpr (!QREG) most = fmaxf(stat[0][nt][col], stat[0][NT + nt][col]);
      int ex = 14;
      if (most < INFINITY && most > 0.0f) (void)frexpf(most, &ex);
      ex = max(ex, -100);
      if (nt == q_tile) up = ldexpf(1.0f, 14 - ex);
      to_score[nt] = ldexpf(1.0f, ex - 14) * (kLog2e / sqrtf((float)dh));
      m_run[nt] = r_run[nt] = -INFINITY;
      l_run[nt] = 0.0f;
    }
#pragma unroll
    for (int k = 0; k < QF; ++k) {
      half8_t hi, lo;
#pragma unroll
      for (int j = 0; j < 8; j += 2) {
        half2_t h, l;
        split(f32x2{qx[k][j >> 2][j & 3] * up, qx[k][j >> 2][(j & 3) + 1] * up}, h, l);
        hi[j] = h[0], hi[j + 1] = h[1];
        lo[j] = l[0], lo[j + 1] = l[1];
      }
      if constexpr (QREG) {
        qf[k][0] = hi;
        qf[k][1] = lo;
      } else {
        q_lds[((q_tile * 2 * NL + q_first + k) * 2 + 0) * 64 + lane] = hi;
        q_lds[((q_tile * 2 * NL + q_first + k) * 2 + 1) * 64 + lane] = lo;
      }
    }
    if constexpr (!QREG) __syncthreads();

    f32x4 o[CT][NT];
#pragma unroll
    for (int ct = 0; ct < CT; ++ct)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) o[ct][nt] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    // The scores' rows of the piece's columns.  A wavefront collects 16 rows of 64 in LDS before it stores them: stores are counted in line with loads,
    // and one in every step holds up the bytes behind it.
    const size_t score_pitch = quant_score_pitch(a.max_context) * sizeof(float);
    const auto score_rows = __builtin_amdgcn_make_buffer_rsrc(
        reinterpret_cast<char*>(a.scores) + ((size_t)r0 * a.n_heads + hk * G + (f0 - r0 * G)) * score_pitch, 0, (int)((f1 - f0) * score_pitch), 0x00020000);
    f32x4* const collected = meet[wave][0][0];
    const int held_shift = 31 - __builtin_clz(max(1, 16 / (f1 - f0)));   // row of column c, step k: (c << held_shift) + k
    int held = 0;

    // runs of rows that share a sequence, one after the other
    for (int r = 0; r < n_rows;) {
      const bool first = r == 0;          // (block ids of the piece's first row are there)
      int seq = r0, longest = __builtin_amdgcn_readfirstlane(row_pos), shortest = longest;
      int limit[NT];
      if constexpr (!SHARED) {
        r = n_rows;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) limit[nt] = col_pos[nt];
      } else {
        seq = lane_value(row_seq, r);
        const uint64_t other = ~__ballot(row_seq == seq && lane < n_rows) >> r;
        const int r_end = min(n_rows, r + (other ? __ffsll((unsigned long long)other) - 1 : 64));
        longest = (int)wave_max((uint32_t)((lane >= r && lane < r_end ? row_pos : -1) + 1)) - 1;
        // (columns of other runs have no position in this one)
        shortest = r_end - r < n_rows ? -1 : -(int)wave_max((uint32_t)(lane < n_rows ? 0x40000000 - row_pos : 0)) + 0x40000000;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) limit[nt] = col_row[nt] >= r && col_row[nt] < r_end ? col_pos[nt] : -1;
        r = r_end;
        s1 = min(s0 + a.part_steps, steps_to(longest));
      }
      const int32_t* table = a.r.block_tables + (size_t)seq * a.r.max_blocks;
      for (int c0 = s0; c0 < s1; c0 += kTableSteps / UNITS) {
        // Block ids, then their scales, go to LDS: a step's loads from memory are then its bytes alone.  (Loads return in the order they were
        // asked for: waiting for an id behind a step's bytes would be waiting for the bytes.)
        // Blocks behind the sequence's last one may be any of the pool's: none of their positions passes a limit; they get scales of 1
        // and 0.
        const int steps = min(kTableSteps / UNITS, s1 - c0);
        f32x2* const scales = block_scale + mine * (kTableSteps / UNITS * 4);
        if (!(SHARED ? first : !dealt) || c0 > s0) __syncthreads();   // (the tables in front have been read)
        for (int i = tid; i < steps * 4; i += kThreads) {
          const int blk = !(SHARED ? first : !dealt) || c0 > s0 || i >= kThreads ? table[min(c0 * 4 + i, last_entry)] : early;
          block_id[i] = safe_block(blk, a.c.num_blocks);
        }
        __syncthreads();
        // (a unit's scales are its own wavefronts' to fetch)
        const int place = tid - mine * (64 * KW);
        auto scales_of = [&](int i) {
          const f32x2 sc = *reinterpret_cast<const f32x2*>(a.c.scales + ((size_t)block_id[min(i, steps * 4 - 1)] * a.c.heads + hk) * 2);
          return (c0 * 4 + i) * 16 > longest ? f32x2{1.0f, 0.0f} : sc;
        };
        const f32x2 own_scale = scales_of(place);
        u32x4 kr[4][NL], vr[CT];
        // (channels and channel tiles from dh on are read as the first ones: the former meet zeros of q, the latter's results are dropped.
        // Every load is made, behind the last step from one place, so that what is in flight is known when the program is compiled.)
        auto load_k = [&](int blk, bool there) {
          const int8_t* p = there ? k_base + (size_t)blk * block_pitch + (col & 3) * dh : k_base;
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int l = 0; l < NL; ++l) {
              const int c = l * 64 + g * 16;
              kr[i][l] = load16<!SHARED>(p + 4 * i * dh + (DH || c < dh ? c : 0));
            }
        };
        auto load_v = [&](int blk, bool there) {
          const int8_t* p = there ? v_base + (size_t)blk * block_pitch + col * 16 : v_base;
#pragma unroll
          for (int ct = 0; ct < CT; ++ct) vr[ct] = load16<!SHARED>(p + (DH || ct * 16 < dh ? ct * 256 : 0));
        };
        load_k(block_id[min(turn, steps - 1) * 4 + (col >> 2)], turn < steps);
        load_v(block_id[min(turn, steps - 1) * 4 + g], turn < steps);
        if (place < steps * 4) scales[place] = own_scale;
        for (int i = place + 64 * KW; i < steps * 4; i += 64 * KW) scales[i] = scales_of(i);
        __syncthreads();
        // a step asks for the next one's bytes as soon as its own have been used
        for (int s = turn; s < steps; s += KW) {
          const bool more = s + KW < steps;
          const int ahead = min(s + KW, steps - 1) * 4;
          const int pos0 = ((c0 + s) * 4 + g) * 16;
          const f32x2 sc = scales[s * 4 + g];
          const int k_blk = block_id[ahead + (col >> 2)], v_blk = block_id[ahead + g];
          // S = K Q^T
          f32x4 sd[NT][4];
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < 4; ++i) sd[nt][i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
          for (int l = 0; l < NL; ++l)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              half8_t kh[4];
#pragma unroll
              for (int i = 0; i < 4; ++i) kh[i] = widen<FMT>(kr[i][l][2 * h], kr[i][l][2 * h + 1]);
#pragma unroll
              for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                  half8_t qv;
                  if constexpr (QREG)
                    qv = qf[2 * l + h][e];
                  else
                    qv = q_lds[((nt * 2 * NL + 2 * l + h) * 2 + e) * 64 + lane];
#pragma unroll
                  for (int i = 0; i < 4; ++i) sd[nt][i] = mma(kh[i], qv, sd[nt][i]);
                }
              __builtin_amdgcn_sched_barrier(0);   // (else every byte is widened first, and there are not as many registers)
            }
          load_k(k_blk, more);
          __builtin_amdgcn_sched_barrier(0);
          const bool ragged = (c0 + s) * 64 + 63 > shortest;   // some positions are behind some column's last one
          // sc[1] is below 2 to v_exponent, and times 2 to v_most still a float
          const float v_exponent = (float)__builtin_amdgcn_frexp_expf(sc[1]), v_most = 127.0f - v_exponent;
          half8_t ph[NT][2], pl[NT][2];
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            // scales are positive: the largest product gives the largest score.  A block without a position for a column has
            // none of its scales in the column's result.
            float f = sc[0] * to_score[nt], v_scale = sc[1];
            if (ragged) {
              if (pos0 > limit[nt]) f = 1.0f, v_scale = 0.0f;
              if (f == 0.0f) f = kQuantScaleFloor;   // (times minus infinity)
#pragma unroll
              for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                  if (pos0 + 4 * i + e > limit[nt]) sd[nt][i][e] = -INFINITY;
            }
            const float mx = largest(sd[nt]);
            if constexpr (WEIGHTS) {
              if (f0 + col < f1) {
#pragma unroll
                for (int i = 0; i < 4; ++i) collected[((col << held_shift) + held) * 16 + ((g * 4 + i) ^ col)] = sd[nt][i] * f;
              }
            }
            const float m_new = fmaxf(m_run[nt], ceilf(max_over_groups(mx * f)) - kBelow);
            const float base = m_new == -INFINITY ? 0.0f : m_new;
            const float less = m_run[nt] - base, alpha = __builtin_amdgcn_exp2f(less);
            m_run[nt] = m_new;
            r_run[nt] += less;
            // What the block adds to the result is below 2^adds times its bytes.  The unit is kept until that is past twice the unit; then a column that needs it
            // takes another one.
            float adds = fmaf(mx, f, -base) + v_exponent;
            if (__any(adds > r_run[nt] || fabsf(base) > kLargeScore)) {
              if (__any(fabsf(base) > kLargeScore)) {
#pragma unroll
                for (int i = 0; i < 4; ++i) sd[nt][i] *= f;
                f = 1.0f;
                adds = largest(sd[nt]) - base + v_exponent;
              }
              const float reach = ceilf(max_over_groups(adds)) + 1.0f;
              const float r_new = reach > r_run[nt] + 1.0f ? reach : r_run[nt];
              const float beta = __builtin_amdgcn_exp2f(r_run[nt] - (r_new == -INFINITY ? 0.0f : r_new));
#pragma unroll
              for (int ct = 0; ct < CT; ++ct) o[ct][nt] *= beta;
              r_run[nt] = r_new;
            }
            // (bounded where the probabilities are 0, which have to stay so)
            const float v_factor = __builtin_ldexpf(v_scale, (int)fminf(15.0f - r_run[nt], v_most));
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
              for (int e = 0; e < 4; e += 2) {
                const float p0 = __builtin_amdgcn_exp2f(fmaf(sd[nt][i][e], f, -base)), p1 = __builtin_amdgcn_exp2f(fmaf(sd[nt][i][e + 1], f, -base));
                sum += p0;
                sum += p1;
                half2_t hi, lo;
                split(f32x2{p0 * v_factor, p1 * v_factor}, hi, lo);
                ph[nt][i >> 1][(i & 1) * 4 + e] = hi[0], ph[nt][i >> 1][(i & 1) * 4 + e + 1] = hi[1];
                pl[nt][i >> 1][(i & 1) * 4 + e] = lo[0], pl[nt][i >> 1][(i & 1) * 4 + e + 1] = lo[1];
              }
            l_run[nt] = l_run[nt] * alpha + sum;
          }
          __builtin_amdgcn_sched_barrier(0);
          // O += V^T P
          if constexpr (FMT == EE_QUANT_E4M3) {
            if ((c0 + s) * 64 + 63 > longest) {    // bytes that hold no position may be NaN, which zero weights do not cover
#pragma unroll
              for (int wd = 0; wd < 4; ++wd) {
                const int n = longest + 1 - pos0 - 4 * wd;
                const uint32_t keep = n >= 4 ? 0xffffffffu : n <= 0 ? 0u : (1u << (8 * n)) - 1;
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) vr[ct][wd] &= keep;
              }
            }
          }
#pragma unroll
          for (int ct = 0; ct < CT; ++ct)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const half8_t vh = widen<FMT>(vr[ct][2 * h], vr[ct][2 * h + 1]);
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) {
                o[ct][nt] = mma(vh, ph[nt][h], o[ct][nt]);
                o[ct][nt] = mma(vh, pl[nt][h], o[ct][nt]);
              }
              if (h == 1 && (ct & 1)) __builtin_amdgcn_sched_barrier(0);
            }
          load_v(v_blk, more);
          if constexpr (WEIGHTS) {
            __builtin_amdgcn_sched_barrier(0);
            if (++held >> held_shift || !more) {
              int again = lane;                      // (else the addresses are computed in front of the loop, and there are not as many registers)
              asm("" : "+v"(again));
              const int piece = again & 15;
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                const int row = 4 * j + (again >> 4), step = row & ((1 << held_shift) - 1), c = row >> held_shift;
                const uint32_t to = (uint32_t)c * (uint32_t)score_pitch + (uint32_t)((c0 + s - (held - 1 - step) * KW) * 64 + 4 * piece) * 4;
                // (rows of no column or step are out of the buffer's range: not stored)
                __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, collected[row * 16 + (piece ^ c)]), score_rows,
                                                       step < held && c < f1 - f0 ? to : 0x80000000u, 0, 0);
              }
              held = 0;
            }
          }
        }
      }
    }

    // ---- the wavefronts' results, joined in their order ----
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      l_run[nt] += __shfl_xor(l_run[nt], 16);
      l_run[nt] += __shfl_xor(l_run[nt], 32);
      if (g == 0) {
        stat[0][wave][nt * 16 + col] = m_run[nt];
        stat[1][wave][nt * 16 + col] = l_run[nt];
      }
    }
    __syncthreads();
    float m_all[NT], l_all[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      float mm = -INFINITY, ll = 0.0f;
#pragma unroll
      for (int w = 0; w < KW; ++w) mm = fmaxf(mm, stat[0][mine * KW + w][nt * 16 + col]);
      const float base = mm == -INFINITY ? 0.0f : mm;
#pragma unroll
      for (int w = 0; w < KW; ++w) ll += stat[1][mine * KW + w][nt * 16 + col] * __builtin_amdgcn_exp2f(stat[0][mine * KW + w][nt * 16 + col] - base);
      m_all[nt] = mm;
      l_all[nt] = ll;
      // divided by the sum first (the largest values' sums would be no floats), then in units of 1
      const float inv = ll == 0.0f ? 0.0f : 1.0f / ll;
      const int unit = (int)fmaxf(m_run[nt] - base + r_run[nt], -1000.0f) - 15;
#pragma unroll
      for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[ct][nt][e] = __builtin_ldexpf(o[ct][nt][e] * inv, unit);
    }
    const bool whole = SHARED ? a.parts == nullptr : s0 == 0 && s1 == unit_steps;
    const bool leaves_part = SHARED ? !whole : !whole || (WEIGHTS && (dealt || tiles > 1));
#pragma unroll
    for (int c0 = 0; c0 < CT; c0 += 4) {
      if (c0) __syncthreads();
#pragma unroll
      for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) meet[wave][c][nt][lane] = o[c0 + c][nt];
      __syncthreads();
#pragma unroll
      for (int c = turn * UNITS; c < (turn + 1) * UNITS; ++c) {   // (a unit's wavefronts share its channels)
        const int ch = (c0 + c) * 16 + g * 4;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          const int f = f0 + nt * 16 + col;
          f32x4 sum = meet[mine * KW][c][nt][lane];
#pragma unroll
          for (int w = 1; w < KW; ++w) sum += meet[mine * KW + w][c][nt][lane];
          if (f >= f1 || ch >= dh) continue;
          const int m = f / G;
          const size_t row = (size_t)m * a.n_heads + hk * G + (f - m * G);
          if (whole) *reinterpret_cast<f32x4*>(a.out + row * dh + ch) = sum;
          if (leaves_part) {
            const size_t slot = SHARED ? row * a.n_parts + blockIdx.z
                                       : ((size_t)hk * a.slots + unit + (dealt ? worker : 0)) * unit_columns(G) + col;
            float* p = a.parts + slot * (dh + 4);
            if (ch == 0) *reinterpret_cast<f32x2*>(p) = f32x2{m_all[nt], l_all[nt]};
            if (!whole) *reinterpret_cast<f32x4*>(p + 4 + ch) = sum;
          }
        }
      }
    }
    if constexpr (WEIGHTS) {
      if (turn == 0 && g == 0) head_stat[mine][col] = f32x2{m_all[0] == -INFINITY ? 0.0f : m_all[0], 1.0f / l_all[0]};
    }
    if (!dealt) break;
    do ++unit;
    while (at < stop && __builtin_amdgcn_readfirstlane(start[unit + 1]) <= at);
  } while (at < stop);
  if constexpr (WEIGHTS) {
    // a context that one workgroup has whole, with all heads that share it
    if (!dealt && tiles == 1) {
      __syncthreads();                               // (scores and statistics that the other wavefronts have written)
      const int m = blockIdx.y, last = last_position(a, a.r.context_lens[m]);
      for (int j = 4 * (tid - mine * (64 * KW)); j <= last; j += 4 * 64 * KW) add_weights(a, head_stat[mine], m, hk, G, last, j);
    }
  }
}

// The parts of contexts joined in their order, a (row, head) a workgroup: each of its WAVES wavefronts adds every WAVES-th part's result, their sums
// meet in LDS.  In workgroups behind those: the attention every position got, four positions a thread, 2048 a workgroup.
// Eight wavefronts where there are few (row, head) pairs (one row of 8 heads in 256 parts: 8 us instead of 11), else four (64 rows of 32 heads in two or
// three parts: 6 us instead of 9).
constexpr int kWeightPositions = 2048, kMostParts = kResident;
template <bool SHARED, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void quant_join_kernel(QuantAttnArgs a) {
  extern __shared__ f32x2 head_stat[];   // [G] maximum, 1 / sum
  __shared__ f32x4 meet[WAVES][64];
  __shared__ float shares[kMostParts];
  const int m = blockIdx.y, G = a.n_heads / a.c.heads, dh = a.c.dh, tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int tiles = SHARED ? 1 : unit_tiles(G);
  const int last = last_position(a, a.r.context_lens[m]);
  if (!SHARED && !takes(a, steps_to(last))) return;
  const int joined = SHARED || a.dealt ? a.n_heads : 0;
  const bool joins = (int)blockIdx.x < joined;
  const int chunks = (a.max_context + kWeightPositions - 1) / kWeightPositions;
  const int job = blockIdx.x - joined, j0 = joins ? 0 : (job % chunks) * kWeightPositions;
  if (!joins && j0 > last) return;
  // a head's parts: n records, `pitch` floats apart
  const size_t pitch = (size_t)(dh + 4) * (SHARED ? 1 : unit_columns(G));
  auto parts_of = [&](int head, int* n) {
    if constexpr (SHARED) {
      *n = last < 0 ? 0 : (last >> 6) / a.part_steps + 1;
      return a.parts + ((size_t)m * a.n_heads + head) * a.n_parts * pitch;
    } else {
      const int hk = head / G, h = head - hk * G, u = m * tiles + h / 16;
      const int2 span = a.dealt ? a.spans[u] : make_int2(0, last >= 0);
      const int slot = u + span.x;
      *n = span.y;
      return a.parts + (((size_t)hk * a.slots + slot) * unit_columns(G) + h % 16) * (dh + 4);
    }
  };
  // maximum and sum over a head's parts, and the parts' shares of the sum (before the division by it)
  auto statistics = [&](const float* p, int n, bool keep) {
    float mm = -INFINITY, sum = 0.0f;
    for (int z = lane; z < n; z += 64) mm = fmaxf(mm, p[z * pitch]);
#pragma unroll
    for (int x = 1; x < 64; x <<= 1) mm = fmaxf(mm, __shfl_xor(mm, x));
    const float base = mm == -INFINITY ? 0.0f : mm;
    for (int z = lane; z < n; z += 64) {
      const f32x2 st = *reinterpret_cast<const f32x2*>(p + z * pitch);
      const float share = st[1] * __builtin_amdgcn_exp2f(st[0] - base);
      sum += share;
      if (keep) shares[z] = share;
    }
#pragma unroll
    for (int x = 1; x < 64; x <<= 1) sum += __shfl_xor(sum, x);
    return f32x2{base, sum};
  };
  if (joins) {
    const int head = blockIdx.x, c = min(lane * 4, dh - 4);
    int n;
    const float* p = parts_of(head, &n);
    float* out = a.out + ((size_t)m * a.n_heads + head) * dh;
    if (n == 0 && wave == 0 && lane * 4 < dh) *reinterpret_cast<f32x4*>(out + c) = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    if (n == 0 || (!SHARED && n == 1)) return;   // (whole contexts have their results)
    const f32x2 st = statistics(p, n, wave == 0);
    __syncthreads();
    const float inv = st[1] == 0.0f ? 0.0f : 1.0f / st[1];
    f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int z0 = wave; z0 < n; z0 += 4 * WAVES) {   // four parts in flight (behind the last: that one again, times 0)
      f32x4 x[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = *reinterpret_cast<const f32x4*>(p + min(z0 + e * WAVES, n - 1) * pitch + 4 + c);
#pragma unroll
      for (int e = 0; e < 4; ++e) o += x[e] * (z0 + e * WAVES < n ? shares[z0 + e * WAVES] * inv : 0.0f);
    }
    meet[wave][lane] = o;
    __syncthreads();
    if (wave || lane * 4 >= dh) return;
#pragma unroll
    for (int w = 1; w < WAVES; ++w) o += meet[w][lane];
    *reinterpret_cast<f32x4*>(out + c) = o;
    return;
  }
  const int hk = job / chunks;
  if constexpr (!SHARED) {
    // (contexts that one workgroup had whole are done)
    if (tiles == 1 && !a.dealt) return;
  }
  for (int h = wave; h < G; h += WAVES) {
    int n;
    const float* p = parts_of(hk * G + h, &n);
    const f32x2 st = statistics(p, n, false);
    if (lane == 0) head_stat[h] = f32x2{st[0], 1.0f / st[1]};
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kWeightPositions / (256 * WAVES); ++i) {
    const int j = j0 + 4 * (tid + i * 64 * WAVES);
    if (j <= last) add_weights(a, head_stat, m, hk, G, last, j);
  }
}

// Whether two K/V heads share a workgroup: where half as many workgroups still are as many as there can be at once.  Each has twice the steps then, and
// its beginning and end take the same time.
bool pairs_heads(const QuantAttnArgs& a) {
  return !a.r.row_table && !a.dealt && a.c.heads % 2 == 0 && (int64_t)a.slots * a.c.heads >= 2 * kResident;
}
template <int FMT, int DH, int NL, bool WEIGHTS>
void launch_units(const QuantAttnArgs& a, dim3 grid, hipStream_t st) {
  if (pairs_heads(a))
    quant_attn_kernel<FMT, DH, NL, false, WEIGHTS, 2><<<dim3(grid.x / 2, grid.y), kThreads, 0, st>>>(a);
  else
    quant_attn_kernel<FMT, DH, NL, false, WEIGHTS, 4><<<grid, kThreads, 0, st>>>(a);
}
template <int FMT, int DH, int NL>
void launch_rows(const QuantAttnArgs& a, dim3 grid, hipStream_t st) {
  if (a.r.row_table)
    quant_attn_kernel<FMT, DH, NL, true, false, 4><<<grid, kThreads, 0, st>>>(a);
  else if (a.scores)
    launch_units<FMT, DH, NL, true>(a, grid, st);
  else
    launch_units<FMT, DH, NL, false>(a, grid, st);
}
// Heads of 64 and 128 channels have kernels of their own: offsets within a block are then part of the load instructions.
template <int FMT>
void launch_format(const QuantAttnArgs& a, dim3 grid, hipStream_t st) {
  const int dh = a.c.dh;
  if (dh == 64)
    launch_rows<FMT, 64, 1>(a, grid, st);
  else if (dh == 128)
    launch_rows<FMT, 128, 2>(a, grid, st);
  else if (dh < 64)
    launch_rows<FMT, 0, 1>(a, grid, st);
  else if (dh < 128)
    launch_rows<FMT, 0, 2>(a, grid, st);
  else if (dh <= 192)
    launch_rows<FMT, 0, 3>(a, grid, st);
  else
    launch_rows<FMT, 0, 4>(a, grid, st);
}

constexpr int kSharedParts = 64;

int deal_workgroups(int kv) { return kResident / kv > 1 ? kResident / kv : 1; }
// Contexts of up to 16 steps are whole pieces: a workgroup's four wavefronts have four steps each, which takes no longer than a second launch
// would.  With four times the resident workgroups in whole contexts, the order in which they end evens them out, as far as no context is much of the work.
// Lengths are the device's; all the host knows is how long a context may be.  If that is more than kLongSteps (8192 positions), two further launches deal
// out the contexts that are.  256 rows over 8 K/V heads, one of 131000 positions among 500 each: 109 us instead of 1790; one of 20000: 76 instead of 302; 1000 to 16000: 809
// instead of 929.  The price: 110 instead of 105 where the longest is 1500, 1009 instead of 972 where all are 12000.  (All of them dealt out: 129, 90, - and 122.)
constexpr int kLongSteps = 128;
// Rows that are dealt out in one launch.
int deal_rows(int rows, int group) {
  const int most = kDealtRows / unit_tiles(group);
  return rows < most ? rows : most;
}
int shared_parts(int rows, int group, int kv, int steps) {
  const int64_t units = quant_attn_tiles(rows, group, true) * kv, want = kResident / units, most = steps / kWaves;
  const int64_t parts = want < most ? want : most;
  return (int)(parts < 1 ? 1 : parts > kSharedParts ? kSharedParts : parts);
}

}  // namespace

int64_t quant_attn_tiles(int rows, int group, bool row_table) { return row_table ? ((int64_t)rows * group + 31) / 32 : (int64_t)rows * unit_tiles(group); }

size_t quant_attn_plan(QuantAttnArgs& a, size_t* spans) {
  *spans = 0;
  const int steps = (a.max_context + 63) / 64, rows = a.r.rows, G = a.n_heads / a.c.heads, kv = a.c.heads;
  const size_t record = a.c.dh + 4;
  a.n_parts = 1;
  a.part_steps = steps;
  a.whole = false;
  a.dealt = a.slots = a.long_steps = 0;
  if (a.r.row_table) {
    const int parts = shared_parts(rows, G, kv, steps);
    a.part_steps = (steps + parts - 1) / parts;
    a.n_parts = (steps + a.part_steps - 1) / a.part_steps;
    return a.n_parts > 1 ? (size_t)rows * a.n_heads * a.n_parts * record : 0;
  }
  const int tiles = unit_tiles(G);
  const bool many = quant_attn_tiles(rows, G, false) > kDealtRows || quant_attn_tiles(rows, G, false) * kv >= 4 * kResident;
  a.whole = many || steps <= 16;
  if (!a.whole || steps > kLongSteps) {
    a.dealt = deal_workgroups(kv);
    *spans = (size_t)deal_rows(rows, G) * tiles;
  }
  if (a.whole && a.dealt) a.long_steps = kLongSteps;
  const size_t whole_slots = a.whole && a.weights_out && tiles > 1 ? (size_t)rows * tiles : 0, deal_slots = a.dealt ? *spans + a.dealt : 0;
  return (size_t)kv * (whole_slots > deal_slots ? whole_slots : deal_slots) * unit_columns(G) * record;
}

// An upper bound that grows with its arguments: a call of fewer rows may be split where one of more is not.
size_t quant_attn_part_floats(const QuantCache& c, int n_heads, int max_rows, int max_context, bool weights) {
  const int steps = (max_context + 63) / 64, G = n_heads / c.heads, kv = c.heads;
  const size_t record = c.dh + 4, columns = (size_t)kv * unit_columns(G);
  const int64_t units = quant_attn_tiles(max_rows, G, false);
  size_t most = weights ? (size_t)units * columns * record : 0;
  if (steps > 16) {
    // dealt out: units in front of the bounds of `deals`
    int64_t u = units < kDealtRows ? units : kDealtRows;
    const int64_t cap = (4 * kResident + kv - 1) / kv;
    if (u > cap && steps <= kLongSteps) u = cap;
    const size_t dealt = (size_t)(u + deal_workgroups(kv)) * columns * record;
    if (dealt > most) most = dealt;
  }
  // row_table: rows * heads * parts <= 32 columns a workgroup x the workgroups aimed at, and <= rows * heads * parts by steps
  if (steps / kWaves > 1) {
    const size_t by_steps = (size_t)max_rows * n_heads * (steps / kWaves < kSharedParts ? steps / kWaves : kSharedParts), aim = (size_t)32 * kResident;
    const size_t shared = (by_steps < aim ? by_steps : aim) * record;
    if (shared > most) most = shared;
  }
  return most;
}

namespace {

void launch_part(const QuantAttnArgs& a, hipStream_t st) {
  const int G = a.n_heads / a.c.heads;
  const int y = a.dealt ? a.dealt : (int)quant_attn_tiles(a.r.rows, G, a.r.row_table != nullptr);
  const dim3 grid(a.c.heads, y, a.n_parts);
  a.c.format == EE_QUANT_INT8 ? launch_format<EE_QUANT_INT8>(a, grid, st) : launch_format<EE_QUANT_E4M3>(a, grid, st);
  if (!a.parts) return;
  const bool few = (int64_t)a.r.rows * a.n_heads <= kResident;
  if (a.r.row_table) {
    const dim3 heads(a.n_heads, a.r.rows);
    few ? quant_join_kernel<true, 8><<<heads, 512, 0, st>>>(a) : quant_join_kernel<true, 4><<<heads, 256, 0, st>>>(a);
  } else {
    const int chunks = a.weights_out ? (a.max_context + kWeightPositions - 1) / kWeightPositions : 0;
    const dim3 jobs((a.dealt ? a.n_heads : 0) + a.c.heads * chunks, a.r.rows);
    const size_t lds = (size_t)G * sizeof(f32x2);
    few ? quant_join_kernel<false, 8><<<jobs, 512, lds, st>>>(a) : quant_join_kernel<false, 4><<<jobs, 256, lds, st>>>(a);
  }
}

}  // namespace

void launch_quant_attention(const QuantAttnArgs& a, hipStream_t st) {
  if (a.r.row_table) return launch_part(a, st);
  const int G = a.n_heads / a.c.heads, tiles = unit_tiles(G);
  if (a.whole) {
    QuantAttnArgs part = a;
    part.dealt = 0;
    part.slots = a.r.rows * tiles;
    if (!a.weights_out || tiles == 1) part.parts = nullptr;
    launch_part(part, st);
  }
  const int each = deal_rows(a.r.rows, G);
  for (int r = 0; a.dealt && r < a.r.rows; r += each) {   // (the workspace serves one after the other)
    QuantAttnArgs part = a;
    part.r.rows = each < a.r.rows - r ? each : a.r.rows - r;
    part.r.context_lens += r;
    part.r.block_tables += (size_t)r * a.r.max_blocks;
    part.q += (size_t)r * a.n_heads * a.c.dh;
    part.out += (size_t)r * a.n_heads * a.c.dh;
    const size_t weights = (size_t)r * a.c.heads * a.weights_pitch;
    if (a.weights_in) part.weights_in += weights;
    if (a.weights_out) part.weights_out += weights;
    part.slots = part.r.rows * tiles + a.dealt;           // (unit u's part in workgroup w is in slot u + w: either grows from one piece to the next)
    launch_part(part, st);
  }
}

}  // namespace ee
