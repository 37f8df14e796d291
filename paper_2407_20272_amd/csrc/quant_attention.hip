// Attention over the 8-bit cache, on the matrix cores.
//
// A workgroup has up to 16 * NT columns, (row, query head) pairs that read the same K/V head: the grouped heads of one row, or of a run of
// prompt rows.  A wavefront takes 64 positions (four blocks T_0..T_3) a step and multiplies
//   S = K Q^T:  16 positions x 32 channels x 16 columns an instruction, the positions of instruction i being 4i..4i+3 of each block, so that
//               lane (column n, group g) ends up with the scores of all 16 positions of block T_g;
//   O += V^T P: 16 channels x 32 positions x 16 columns, contracted over positions 8h..8h+7 of each block: lane (n, g) has those
//               eight probabilities already, and the bytes of a channel's 16 positions are consecutive in V's blocks.
// No value crosses lanes but the running maxima, and every load is 16 bytes a lane.  Bytes become fp16 without error.  q (scaled by a power of two
// to 2^13..2^14) and the probabilities (times the block's scale, relative to the largest scale so far) are split into an fp16 head and
// remainder, 22 bits together: the products are float in effect, as in the float cache's attention.
// Softmax statistics and results are float, running over a wavefront's steps; the four wavefronts and the parts of a long context are
// joined in a fixed order.
#include "quant.h"

namespace ee {

namespace {

constexpr int kWaves = 4;
constexpr int kMinPart = 4, kMaxPart = 256;   // 64-position steps of a part of a context: one a wavefront, and what the tables in LDS hold
constexpr float kLog2e = 1.4426950408889634f;

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

// The last position row m attends: -1 for none.
__device__ inline int last_position(const QuantAttnArgs& a, int m) {
  return max(-1, min(a.r.context_lens[m], min(a.max_context, a.r.max_blocks * 16) - 1));
}

// DH: the head's channels, or 0 for a.c.dh; NL: loads of 16 bytes a lane and position (64 channels each).  SHARED: rows that may share a sequence,
// 32 columns; else the grouped heads of one row, 16 columns.
constexpr int quant_tiles(bool shared) { return shared ? 2 : 1; }
template <int FMT, int DH, int NL, bool SHARED, bool WEIGHTS>
__global__ __launch_bounds__(64 * kWaves, NL * quant_tiles(SHARED) <= 2 ? 2 : 1) void quant_attn_kernel(QuantAttnArgs a) {
  constexpr int NT = quant_tiles(SHARED), C = 16 * NT, CT = 4 * NL;
  constexpr bool QREG = NT == 1;        // q's fragments in registers, or in LDS
  __shared__ half8_t q_lds[QREG ? 1 : NT * NL * 2 * 2 * 64];
  __shared__ float stat[2][kWaves][C];
  __shared__ f32x4 meet[kWaves][4][NT][64];
  __shared__ int block_id[kMaxPart * 4];         // the part's blocks, and their scales of K and V
  __shared__ f32x2 block_scale[kMaxPart * 4];
  const int lane = threadIdx.x & 63, col = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int dh = DH ? DH : a.c.dh, G = a.n_heads / a.c.heads, hk = blockIdx.x, part = blockIdx.z;
  int f0, f1;
  if constexpr (SHARED) {
    f0 = blockIdx.y * C;
    f1 = min(f0 + C, a.r.rows * G);
  } else {
    const int per_row = (G + C - 1) / C, m = blockIdx.y / per_row;
    f0 = m * G + (blockIdx.y - m * per_row) * C;
    f1 = min(f0 + C, (m + 1) * G);
  }
  // The tile's rows, one a lane.  What a wavefront needs before its first bytes (positions, block ids, q) is asked for at once: the ids of a
  // row of its own without waiting for its length (entries behind it may be anything, see block_of).
  const int r0 = f0 / G, n_rows = (f1 - 1) / G - r0 + 1;
  const int m_lane = r0 + min(lane, n_rows - 1);
  const int ctx = a.r.context_lens[m_lane];
  const int first = part * a.part_steps, last_entry = a.r.max_blocks - 1;
  int own_block = 0;
  if constexpr (!SHARED) own_block = a.r.block_tables[(size_t)r0 * a.r.max_blocks + min(first * 4 + (int)threadIdx.x, last_entry)];
  f32x4 qx[NT][2 * NL][2];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int f = min(f0 + nt * 16 + col, f1 - 1), m = f / G;
    const float* q = a.q + ((size_t)m * a.n_heads + hk * G + (f - m * G)) * dh;
#pragma unroll
    for (int k = 0; k < 2 * NL; ++k) {
      const int c = (k >> 1) * 64 + g * 16 + (k & 1) * 8;
#pragma unroll
      for (int e = 0; e < 2; ++e) qx[nt][k][e] = *reinterpret_cast<const f32x4*>(q + (c < dh ? c : 0) + 4 * e);
    }
  }
  const int row_seq = quant_seq(a.r, m_lane), row_pos = max(-1, min(ctx, min(a.max_context, a.r.max_blocks * 16) - 1));
  if (part > 0 && !__any((row_pos >> 6) >= part * a.part_steps)) return;

  // q, split; the factor that turns a product back into a score in units of log 2
  half8_t qf[QREG ? 2 * NL : 1][2];
  float to_score[NT], m_run[NT], l_run[NT];
  int col_row[NT], col_pos[NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int f = f0 + nt * 16 + col;
    const bool valid = f < f1;
    col_row[nt] = (valid ? f / G : r0) - r0;
    col_pos[nt] = __shfl(row_pos, col_row[nt]);
    if (!valid) col_pos[nt] = -1;
    float most = 0.0f;
#pragma unroll
    for (int k = 0; k < 2 * NL; ++k)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        if (!valid || (k >> 1) * 64 + g * 16 >= dh) qx[nt][k][e] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int j = 0; j < 4; ++j) most = fmaxf(most, fabsf(qx[nt][k][e][j]));
      }
    most = max_over_groups(most);
    int ex = 14;
    if (most < INFINITY && most > 0.0f) (void)frexpf(most, &ex);
    ex = max(ex, -100);
    const float up = ldexpf(1.0f, 14 - ex);
    to_score[nt] = ldexpf(1.0f, ex - 14) * (kLog2e / sqrtf((float)dh));
    m_run[nt] = -INFINITY;
    l_run[nt] = 0.0f;
#pragma unroll
    for (int k = 0; k < 2 * NL; ++k) {
      half8_t hi, lo;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float y = qx[nt][k][j >> 2][j & 3] * up;
        hi[j] = (half_t)y;
        lo[j] = (half_t)(y - (float)hi[j]);
      }
      if constexpr (QREG) {
        qf[k][0] = hi;
        qf[k][1] = lo;
      } else if (wave == nt) {
        q_lds[((nt * 2 * NL + k) * 2 + 0) * 64 + lane] = hi;
        q_lds[((nt * 2 * NL + k) * 2 + 1) * 64 + lane] = lo;
      }
    }
  }
  if constexpr (!QREG) __syncthreads();

  f32x4 o[CT][NT];
#pragma unroll
  for (int ct = 0; ct < CT; ++ct)
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) o[ct][nt] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  float v_ref = 0.0f, v_up = 0.0f;      // the power of two that is at least every scale of V so far; 2^14 / v_ref

  const size_t block_bytes = (size_t)16 * dh, block_pitch = block_bytes * a.c.heads;
  const int8_t* k_base = a.c.k + hk * block_bytes;
  const int8_t* v_base = a.c.v + hk * block_bytes;

  // the scores' rows of the tile's columns
  const size_t score_pitch = quant_score_pitch(a.max_context) * sizeof(float);
  const auto score_rows = __builtin_amdgcn_make_buffer_rsrc(
      reinterpret_cast<char*>(a.scores) + ((size_t)r0 * a.n_heads + hk * G + (f0 - r0 * G)) * score_pitch, 0, (int)((f1 - f0) * score_pitch), 0x00020000);
  const uint32_t score_at = f0 + col < f1 ? (uint32_t)(col * score_pitch) : 0x80000000u;

  // runs of rows that share a sequence, one after the other
  for (int r = 0; r < n_rows;) {
    int seq = r0, longest = __builtin_amdgcn_readfirstlane(row_pos);
    int limit[NT];
    if constexpr (!SHARED) {
      r = n_rows;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) limit[nt] = col_pos[nt];
    } else {
      seq = __shfl(row_seq, r);
      const uint64_t other = ~__ballot(row_seq == seq && lane < n_rows) >> r;
      const int r_end = min(n_rows, r + (other ? __ffsll((unsigned long long)other) - 1 : 64));
      longest = lane >= r && lane < r_end ? row_pos : -1;
#pragma unroll
      for (int x = 1; x < 64; x <<= 1) longest = max(longest, __shfl_xor(longest, x));
      longest = __builtin_amdgcn_readfirstlane(longest);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) limit[nt] = col_row[nt] >= r && col_row[nt] < r_end ? col_pos[nt] : -1;
      r = r_end;
    }
    const int steps = min(a.part_steps, (longest >> 6) + 1 - first);      // (longest = -1: none)
    if (steps <= 0) continue;

    // The part's block ids, then their scales, go to LDS: a step's loads from memory are then its bytes alone.  (Loads return in the order they were
    // asked for: waiting for an id behind a step's bytes would be waiting for the bytes.)
    // Blocks behind the sequence's last one may be any of the pool's: none of their positions passes a limit, their scales and V's bytes are
    // replaced by zeros.
    const int32_t* table = a.r.block_tables + (size_t)seq * a.r.max_blocks + first * 4;
    if constexpr (SHARED) __syncthreads();     // (the run in front has been read)
    for (int i = threadIdx.x; i < steps * 4; i += 64 * kWaves) {
      if (SHARED || i >= 64 * kWaves) own_block = table[min(i, last_entry - first * 4)];
      block_id[i] = safe_block(own_block, a.c.num_blocks);
    }
    __syncthreads();
    auto scales_of = [&](int i) {
      const f32x2 sc = *reinterpret_cast<const f32x2*>(a.c.scales + ((size_t)block_id[min(i, steps * 4 - 1)] * a.c.heads + hk) * 2);
      return (first * 4 + i) * 16 > longest ? f32x2{0.0f, 0.0f} : sc;
    };
    const f32x2 own_scale = scales_of(threadIdx.x);
    u32x4 kr[4][NL], vr[CT];
    // (channels and channel tiles from dh on are read as the first ones: the former meet zeros of q, the latter's results are dropped.  Every
    // load is made, behind the last step from one place, so that what is in flight is known when the program is compiled.)
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

    load_k(block_id[min(wave, steps - 1) * 4 + (col >> 2)], wave < steps);
    load_v(block_id[min(wave, steps - 1) * 4 + g], wave < steps);
    if ((int)threadIdx.x < steps * 4) block_scale[threadIdx.x] = own_scale;
    for (int i = threadIdx.x + 64 * kWaves; i < steps * 4; i += 64 * kWaves) block_scale[i] = scales_of(i);
    __syncthreads();
    // results are kept relative to the largest scale of V so far
    float most_v = 0.0f;
    for (int i = lane; i < steps * 4; i += 64) most_v = fmaxf(most_v, block_scale[i][1]);
    most_v = __builtin_bit_cast(float, wave_max(__builtin_bit_cast(uint32_t, most_v)));
    if (most_v > v_ref) {
      int e;
      (void)frexpf(most_v, &e);
      const float next = ldexpf(1.0f, max(-100, min(e, 127)));
      const float f = v_ref / next;
      v_ref = next;
      v_up = 16384.0f / next;
#pragma unroll
      for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) o[ct][nt] *= f;
    }
    // a step asks for the next one's bytes as soon as its own have been used
    for (int s = wave; s < steps; s += kWaves) {
      const bool more = s + kWaves < steps;
      const int ahead = min(s + kWaves, steps - 1) * 4;
      const int pos0 = ((first + s) * 4 + g) * 16;
      const f32x2 sc = block_scale[s * 4 + g];
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
      const float v_factor = sc[1] * v_up;
      half8_t ph[NT][2], pl[NT][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const float f = sc[0] * to_score[nt];
        float mx = -INFINITY;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float t = pos0 + 4 * i + e <= limit[nt] ? sd[nt][i][e] * f : -INFINITY;
            sd[nt][i][e] = t;
            mx = fmaxf(mx, t);
          }
        if constexpr (WEIGHTS) {   // lanes of no column are out of the buffer's range: their stores are dropped, and every store is made
#pragma unroll
          for (int i = 0; i < 4; ++i)
            __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, sd[nt][i]), score_rows, score_at + (uint32_t)(pos0 + 4 * i) * 4, 0, 0);
        }
        const float m_new = fmaxf(m_run[nt], max_over_groups(mx));
        const float base = m_new == -INFINITY ? 0.0f : m_new;
        const float alpha = __builtin_amdgcn_exp2f(m_run[nt] - base);
        if (__any(m_new != m_run[nt])) {
#pragma unroll
          for (int ct = 0; ct < CT; ++ct) o[ct][nt] *= alpha;
        }
        m_run[nt] = m_new;
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float p = __builtin_amdgcn_exp2f(sd[nt][i][e] - base);
            sum += p;
            const float w = p == 0.0f ? 0.0f : p * v_factor;   // (a masked position's scale may be anything)
            const half_t hi = (half_t)w;
            ph[nt][i >> 1][(i & 1) * 4 + e] = hi;
            pl[nt][i >> 1][(i & 1) * 4 + e] = (half_t)(w - (float)hi);
          }
        l_run[nt] = l_run[nt] * alpha + sum;
      }
      __builtin_amdgcn_sched_barrier(0);
      // O += V^T P
      if constexpr (FMT == EE_QUANT_E4M3) {
        if ((first + s) * 64 + 63 > longest) {    // bytes that hold no position may be NaN, which zero weights do not cover
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
    }
  }

  // the wavefronts' results, joined in their order
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
    for (int w = 0; w < kWaves; ++w) mm = fmaxf(mm, stat[0][w][nt * 16 + col]);
    const float base = mm == -INFINITY ? 0.0f : mm;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) ll += stat[1][w][nt * 16 + col] * __builtin_amdgcn_exp2f(stat[0][w][nt * 16 + col] - base);
    m_all[nt] = mm;
    l_all[nt] = ll;
    const float f = __builtin_amdgcn_exp2f(m_run[nt] - base) * v_ref * (1.0f / 16384.0f);
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) o[ct][nt] *= f;
  }
  const bool direct = a.parts == nullptr;
#pragma unroll
  for (int c0 = 0; c0 < CT; c0 += 4) {
    if (c0) __syncthreads();
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) meet[wave][c][nt][lane] = o[c0 + c][nt];
    __syncthreads();
    const int ch = (c0 + wave) * 16 + g * 4;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int f = f0 + nt * 16 + col;
      f32x4 sum = meet[0][wave][nt][lane];
#pragma unroll
      for (int w = 1; w < kWaves; ++w) sum += meet[w][wave][nt][lane];
      if (f >= f1 || ch >= dh) continue;
      const int m = f / G;
      const size_t at = (size_t)m * a.n_heads + hk * G + (f - m * G);
      if (direct) {
        const float inv = l_all[nt] == 0.0f ? 0.0f : 1.0f / l_all[nt];
        *reinterpret_cast<f32x4*>(a.out + at * dh + ch) = sum * inv;
      } else {
        float* p = a.parts + (at * a.n_parts + part) * (dh + 4);
        if (ch == 0) *reinterpret_cast<f32x2*>(p) = f32x2{m_all[nt], l_all[nt]};
        *reinterpret_cast<f32x4*>(p + 4 + ch) = sum;
      }
    }
  }
}

// The parts of a context joined in their order, a (row, head) a workgroup: a lane has the statistics of a part, each wavefront adds every fourth
// part's result, the four sums meet in LDS.  In workgroups behind those: the attention every position got, four positions a thread.
constexpr int kWeightPositions = 1024;
__global__ __launch_bounds__(256) void quant_join_kernel(QuantAttnArgs a) {
  extern __shared__ f32x2 head_stat[];   // [G] maximum, 1 / sum
  __shared__ f32x4 meet[kWaves][64];
  const int m = blockIdx.y, G = a.n_heads / a.c.heads, dh = a.c.dh, tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int last = last_position(a, m);
  const int n = last < 0 ? 0 : (last >> 6) / a.part_steps + 1;
  const size_t pitch = dh + 4;
  // the factor of each lane's part, relative to the maximum over the parts, and the sum of all of them
  auto factor = [&](int head, float* base, float* sum) {
    const float* p = a.parts + (((size_t)m * a.n_heads + head) * a.n_parts + min(lane, a.n_parts - 1)) * pitch;
    const f32x2 stat = *reinterpret_cast<const f32x2*>(p);
    float mm = lane < n ? stat[0] : -INFINITY;
#pragma unroll
    for (int x = 1; x < 64; x <<= 1) mm = fmaxf(mm, __shfl_xor(mm, x));
    *base = mm == -INFINITY ? 0.0f : mm;
    const float f = lane < n ? __builtin_amdgcn_exp2f(stat[0] - *base) : 0.0f;
    float s = lane < n ? stat[1] * f : 0.0f;
#pragma unroll
    for (int x = 1; x < 64; x <<= 1) s += __shfl_xor(s, x);
    *sum = s;
    return f;
  };
  if ((int)blockIdx.x < a.n_heads) {
    const int head = blockIdx.x, c = min(lane * 4, dh - 4);
    const float* p = a.parts + ((size_t)m * a.n_heads + head) * a.n_parts * pitch + 4 + c;
    float base, sum;
    const float f = factor(head, &base, &sum);
    f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int z = wave; z < n; z += kWaves) o += *reinterpret_cast<const f32x4*>(p + z * pitch) * __shfl(f, z);
    meet[wave][lane] = o;
    __syncthreads();
    if (wave || lane * 4 >= dh) return;
#pragma unroll
    for (int w = 1; w < kWaves; ++w) o += meet[w][lane];
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    *reinterpret_cast<f32x4*>(a.out + ((size_t)m * a.n_heads + head) * dh + c) = o * inv;
    return;
  }
  const int chunks = (a.max_context + kWeightPositions - 1) / kWeightPositions;
  const int job = blockIdx.x - a.n_heads, hk = job / chunks, j = (job - hk * chunks) * kWeightPositions + 4 * tid;
  if (j - 4 * tid > last) return;
  for (int h = wave; h < G; h += kWaves) {
    float base, sum;
    (void)factor(hk * G + h, &base, &sum);
    if (lane == 0) head_stat[h] = f32x2{base, 1.0f / sum};
  }
  __syncthreads();
  if (j > last) return;
  const size_t sp = quant_score_pitch(a.max_context);
  const float* s = a.scores + ((size_t)m * a.n_heads + hk * G) * sp + j;   // (rows of 64 positions: four are there)
  const size_t row = ((size_t)m * a.c.heads + hk) * a.weights_pitch + j;
  f32x4 w = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
  for (int h = 0; h < G; ++h) {
    const f32x4 x = *reinterpret_cast<const f32x4*>(s + h * sp);
    const f32x2 stat = head_stat[h];
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] += __builtin_amdgcn_exp2f(x[e] - stat[0]) * stat[1];
  }
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (j + e <= last) a.weights_out[row + e] = a.weights_in && j + e < last ? a.weights_in[row + e] + w[e] : w[e];
}

template <int FMT, int DH, int NL>
void launch_rows(const QuantAttnArgs& a, dim3 grid, hipStream_t st) {
  if (a.r.row_table)
    quant_attn_kernel<FMT, DH, NL, true, false><<<grid, 64 * kWaves, 0, st>>>(a);
  else if (a.scores)
    quant_attn_kernel<FMT, DH, NL, false, true><<<grid, 64 * kWaves, 0, st>>>(a);
  else
    quant_attn_kernel<FMT, DH, NL, false, false><<<grid, 64 * kWaves, 0, st>>>(a);
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

constexpr int kTarget = 512;             // workgroups to aim at by splitting contexts: two a compute unit
constexpr int kMostParts = 64;           // (a lane each where they are joined)

// Workgroups of an unsplit call.
int64_t plan_units(int rows, int G, int kv, bool shared) {
  const int64_t C = 16 * quant_tiles(shared);
  return (shared ? ((int64_t)rows * G + C - 1) / C : rows * ((G + C - 1) / C)) * kv;
}
int plan_parts(int64_t units, int steps) {
  const int64_t most = steps / kMinPart, want = kTarget / units, least = (steps + kMaxPart - 1) / kMaxPart;
  int64_t parts = want < 1 || most < 1 ? 1 : want < most ? want : most;
  if (parts > kMostParts) parts = kMostParts;
  return (int)(parts > least ? parts : least);
}

}  // namespace

void quant_attn_plan(QuantAttnArgs& a) {
  const int steps = (a.max_context + 63) / 64;
  const int64_t units = plan_units(a.r.rows, a.n_heads / a.c.heads, a.c.heads, a.r.row_table != nullptr);
  const int parts = plan_parts(units, steps);
  a.part_steps = ((steps + parts - 1) / parts + kMinPart - 1) / kMinPart * kMinPart;
  a.n_parts = (steps + a.part_steps - 1) / a.part_steps;
}

// A call of fewer rows may be split into more parts: what all of them together take is bounded by the workgroups aimed at.
size_t quant_attn_part_floats(const QuantCache& c, int n_heads, int max_rows, int max_context, bool weights) {
  const int steps = (max_context + 63) / 64;
  const size_t pitch = c.dh + 4, columns = (size_t)max_rows * n_heads;
  if (plan_parts(1, steps) == 1) return weights ? columns * pitch : 0;
  // at most 32 columns a workgroup
  const size_t split = columns * (size_t)(steps / kMinPart), aim = (size_t)kTarget * 32;
  const size_t least = columns * (size_t)((steps + kMaxPart - 1) / kMaxPart);
  return (split < aim ? split : least > aim ? least : aim) * pitch;
}

void launch_quant_attention(const QuantAttnArgs& a, hipStream_t st) {
  const int G = a.n_heads / a.c.heads, C = 16 * quant_tiles(a.r.row_table != nullptr);
  const int y = a.r.row_table ? (int)(((int64_t)a.r.rows * G + C - 1) / C) : a.r.rows * ((G + C - 1) / C);
  const dim3 grid(a.c.heads, y, a.n_parts);
  a.c.format == EE_QUANT_INT8 ? launch_format<EE_QUANT_INT8>(a, grid, st) : launch_format<EE_QUANT_E4M3>(a, grid, st);
  if (!a.parts) return;
  const int chunks = a.weights_out ? (a.max_context + kWeightPositions - 1) / kWeightPositions : 0;
  quant_join_kernel<<<dim3(a.n_heads + a.c.heads * chunks, a.r.rows), 256, (size_t)G * sizeof(f32x2), st>>>(a);
}

}  // namespace ee
