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

// NL: loads of 16 bytes a lane and position (64 channels each); NT: tiles of 16 columns.
template <int FMT, int NL, int NT>
__global__ __launch_bounds__(64 * kWaves, NL * NT <= 2 ? 2 : 1) void quant_attn_kernel(QuantAttnArgs a) {
  constexpr int C = 16 * NT, CT = 4 * NL;
  constexpr bool QREG = NT == 1;        // q's fragments in registers, or in LDS
  __shared__ half8_t q_lds[QREG ? 1 : NT * NL * 2 * 2 * 64];
  __shared__ float stat[2][kWaves][C];
  __shared__ f32x4 meet[kWaves][4][NT][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, g = lane >> 4;
  const int dh = a.c.dh, G = a.n_heads / a.c.heads, hk = blockIdx.x, part = blockIdx.z;
  int f0, f1;
  if (a.r.row_table) {
    f0 = blockIdx.y * C;
    f1 = min(f0 + C, a.r.rows * G);
  } else {
    const int per_row = (G + C - 1) / C, m = blockIdx.y / per_row;
    f0 = m * G + (blockIdx.y - m * per_row) * C;
    f1 = min(f0 + C, (m + 1) * G);
  }
  // the tile's rows, one a lane
  const int r0 = f0 / G, n_rows = (f1 - 1) / G - r0 + 1;
  int row_seq = -1, row_pos = -1;
  if (lane < n_rows) {
    row_seq = quant_seq(a.r, r0 + lane);
    row_pos = last_position(a, r0 + lane);
  }
  if (part > 0 && !__any((row_pos >> 6) >= part * a.part_steps)) return;

  // q, split; the factor that turns a product back into a score in units of log 2
  half8_t qf[QREG ? 2 * NL : 1][2];
  float to_score[NT], m_run[NT], l_run[NT];
  int col_row[NT], col_pos[NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int f = f0 + nt * 16 + col;
    const bool valid = f < f1;
    const int m = valid ? f / G : r0;
    col_row[nt] = m - r0;
    col_pos[nt] = __shfl(row_pos, m - r0);
    if (!valid) col_pos[nt] = -1;
    const float* q = a.q + ((size_t)m * a.n_heads + hk * G + (valid ? f - m * G : 0)) * dh;
    f32x4 x[2 * NL][2];
    float most = 0.0f;
#pragma unroll
    for (int k = 0; k < 2 * NL; ++k) {
      const int c = (k >> 1) * 64 + g * 16 + (k & 1) * 8;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        x[k][e] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        if (valid && c < dh) x[k][e] = *reinterpret_cast<const f32x4*>(q + c + 4 * e);
#pragma unroll
        for (int j = 0; j < 4; ++j) most = fmaxf(most, fabsf(x[k][e][j]));
      }
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
        const float y = x[k][j >> 2][j & 3] * up;
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

  // runs of rows that share a sequence, one after the other
  for (int r = 0; r < n_rows;) {
    const int seq = __shfl(row_seq, r);
    const uint64_t other = ~__ballot(row_seq == seq && lane < n_rows) >> r;
    const int r_end = min(n_rows, r + (other ? __ffsll((unsigned long long)other) - 1 : 64));
    int longest = lane >= r && lane < r_end ? row_pos : -1;
#pragma unroll
    for (int x = 1; x < 64; x <<= 1) longest = max(longest, __shfl_xor(longest, x));
    longest = __builtin_amdgcn_readfirstlane(longest);
    int limit[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) limit[nt] = col_row[nt] >= r && col_row[nt] < r_end ? col_pos[nt] : -1;
    r = r_end;
    const int end = min((part + 1) * a.part_steps, (longest >> 6) + 1);   // (longest = -1: 0)
    int s = part * a.part_steps + wave;
    if (s >= end) continue;

    const int32_t* table = a.r.block_tables + (size_t)seq * a.r.max_blocks;
    const int last_block = longest >> 4;
    // (blocks behind the last one are read as the last one; none of their positions passes a limit)
    auto block_of = [&](int logical) { return safe_block(table[min(logical, last_block)], a.c.num_blocks); };
    u32x4 kr[4][NL], vr[CT];
    f32x2 sc;
    auto load_k = [&](int blk) {
      const int8_t* p = k_base + (size_t)blk * block_pitch + (col & 3) * dh;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int l = 0; l < NL; ++l) {
          const int c = l * 64 + g * 16;
          kr[i][l] = load16<NT == 1>(p + 4 * i * dh + (c < dh ? c : 0));   // (channels from dh on meet zeros of q)
        }
    };
    auto load_v = [&](int blk) {
      const int8_t* p = v_base + (size_t)blk * block_pitch + col * 16;
#pragma unroll
      for (int ct = 0; ct < CT; ++ct)
        if (ct * 16 < dh) vr[ct] = load16<NT == 1>(p + ct * 256);
    };
    auto load_scales = [&](int blk) { return *reinterpret_cast<const f32x2*>(a.c.scales + ((size_t)blk * a.c.heads + hk) * 2); };

    int k_blk = block_of(s * 4 + (col >> 2)), v_blk = block_of(s * 4 + g);
    load_k(k_blk);
    sc = load_scales(v_blk);
    load_v(v_blk);
    k_blk = block_of((s + kWaves) * 4 + (col >> 2));
    v_blk = block_of((s + kWaves) * 4 + g);
    for (; s < end; s += kWaves) {
      const bool more = s + kWaves < end;
      const int pos0 = (s * 4 + g) * 16;
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
        }
      const f32x2 sc_now = sc;
      const int v_next = v_blk;
      if (more) {
        load_k(k_blk);
        sc = load_scales(v_blk);
      }
      // the scales of V: results are kept relative to the largest so far
      const float vs = pos0 <= longest ? sc_now[1] : 0.0f;
      const float vm = max_over_groups(vs);
      if (vm > v_ref) {
        int e;
        (void)frexpf(vm, &e);
        const float next = ldexpf(1.0f, max(-100, min(e, 127)));
        const float f = v_ref / next;
        v_ref = next;
        v_up = 16384.0f / next;
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) o[ct][nt] *= f;
      }
      const float v_factor = vs * v_up;
      half8_t ph[NT][2], pl[NT][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const float f = sc_now[0] * to_score[nt];
        float mx = -INFINITY;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float t = pos0 + 4 * i + e <= limit[nt] ? sd[nt][i][e] * f : -INFINITY;
            sd[nt][i][e] = t;
            mx = fmaxf(mx, t);
          }
        if (a.scores && f0 + nt * 16 + col < f1) {
          const int fc = f0 + nt * 16 + col, m = fc / G;
          float* p = a.scores + ((size_t)m * a.n_heads + hk * G + (fc - m * G)) * quant_score_pitch(a.max_context) + pos0;
#pragma unroll
          for (int i = 0; i < 4; ++i) *reinterpret_cast<f32x4*>(p + 4 * i) = sd[nt][i];
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
      // O += V^T P
      if constexpr (FMT == EE_QUANT_E4M3) {
        if (s * 64 + 63 > longest) {    // bytes that hold no position may be NaN, which zero weights do not cover
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
        if (ct * 16 < dh) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const half8_t vh = widen<FMT>(vr[ct][2 * h], vr[ct][2 * h + 1]);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              o[ct][nt] = mma(vh, ph[nt][h], o[ct][nt]);
              o[ct][nt] = mma(vh, pl[nt][h], o[ct][nt]);
            }
          }
        }
      if (more) {
        load_v(v_next);
        k_blk = block_of((s + 2 * kWaves) * 4 + (col >> 2));
        v_blk = block_of((s + 2 * kWaves) * 4 + g);
      }
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

// The parts of a context joined in their order; in workgroups behind those of the results, the attention every position got.
constexpr int kWeightPositions = 1024;
__global__ __launch_bounds__(256) void quant_join_kernel(QuantAttnArgs a) {
  extern __shared__ f32x2 head_stat[];   // [G] maximum, 1 / sum
  const int m = blockIdx.y, G = a.n_heads / a.c.heads, dh = a.c.dh, tid = threadIdx.x, lane = tid & 63;
  const int last = last_position(a, m);
  const int n = last < 0 ? 0 : (last >> 6) / a.part_steps + 1;
  const size_t pitch = dh + 4;
  auto part_of = [&](int head, int z) { return a.parts + (((size_t)m * a.n_heads + head) * a.n_parts + z) * pitch; };
  const int merges = (a.n_heads + 3) / 4;
  if ((int)blockIdx.x < merges) {        // a head a wavefront
    const int head = blockIdx.x * 4 + (tid >> 6);
    if (head >= a.n_heads) return;
    float mm = -INFINITY;
    for (int z = lane; z < n; z += 64) mm = fmaxf(mm, part_of(head, z)[0]);
#pragma unroll
    for (int x = 1; x < 64; x <<= 1) mm = fmaxf(mm, __shfl_xor(mm, x));
    const float base = mm == -INFINITY ? 0.0f : mm;
    float ll = 0.0f;
    f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
    const int c = lane * 4;
    for (int z = 0; z < n; ++z) {
      const float* p = part_of(head, z);
      const float f = __builtin_amdgcn_exp2f(p[0] - base);
      ll += p[1] * f;
      if (c < dh) o += *reinterpret_cast<const f32x4*>(p + 4 + c) * f;
    }
    const float inv = ll == 0.0f ? 0.0f : 1.0f / ll;
    if (c < dh) *reinterpret_cast<f32x4*>(a.out + ((size_t)m * a.n_heads + head) * dh + c) = o * inv;
    return;
  }
  const int chunks = (a.max_context + kWeightPositions - 1) / kWeightPositions;
  const int job = blockIdx.x - merges, hk = job / chunks, j0 = (job - hk * chunks) * kWeightPositions;
  if (j0 > last) return;
  for (int h = tid; h < G; h += 256) {
    float mm = -INFINITY, ll = 0.0f;
    for (int z = 0; z < n; ++z) mm = fmaxf(mm, part_of(hk * G + h, z)[0]);
    const float base = mm == -INFINITY ? 0.0f : mm;
    for (int z = 0; z < n; ++z) ll += part_of(hk * G + h, z)[1] * __builtin_amdgcn_exp2f(part_of(hk * G + h, z)[0] - base);
    head_stat[h] = f32x2{base, 1.0f / ll};
  }
  __syncthreads();
  const size_t sp = quant_score_pitch(a.max_context);
  const float* s = a.scores + ((size_t)m * a.n_heads + hk * G) * sp;
  const size_t row = ((size_t)m * a.c.heads + hk) * a.weights_pitch;
  for (int j = j0 + tid; j < j0 + kWeightPositions && j <= last; j += 256) {
    float w = 0.0f;
    for (int h = 0; h < G; ++h) w += __builtin_amdgcn_exp2f(s[h * sp + j] - head_stat[h][0]) * head_stat[h][1];
    a.weights_out[row + j] = a.weights_in && j < last ? a.weights_in[row + j] + w : w;
  }
}

template <int FMT, int NL>
void launch_tiles(const QuantAttnArgs& a, dim3 grid, hipStream_t st) {
  if (a.tiles == 1)
    quant_attn_kernel<FMT, NL, 1><<<grid, 64 * kWaves, 0, st>>>(a);
  else
    quant_attn_kernel<FMT, NL, 2><<<grid, 64 * kWaves, 0, st>>>(a);
}
template <int FMT>
void launch_format(const QuantAttnArgs& a, dim3 grid, hipStream_t st) {
  if (a.c.dh <= 64)
    launch_tiles<FMT, 1>(a, grid, st);
  else if (a.c.dh <= 128)
    launch_tiles<FMT, 2>(a, grid, st);
  else if (a.c.dh <= 192)
    launch_tiles<FMT, 3>(a, grid, st);
  else
    launch_tiles<FMT, 4>(a, grid, st);
}

constexpr int kMinPart = 4;              // steps of a part: one a wavefront
constexpr int kTarget = 2048;            // workgroups to aim at by splitting contexts

// Workgroups of an unsplit call.
int64_t plan_units(int rows, int G, int kv, bool shared, int* tiles) {
  *tiles = (shared ? (int64_t)rows * G : G) > 16 ? 2 : 1;
  const int64_t C = 16 * *tiles;
  return (shared ? ((int64_t)rows * G + C - 1) / C : rows * ((G + C - 1) / C)) * kv;
}
int plan_parts(int64_t units, int steps) {
  const int64_t most = steps / kMinPart, want = kTarget / units;
  return (int)(want < 1 || most < 1 ? 1 : want < most ? want : most);
}

}  // namespace

void quant_attn_plan(QuantAttnArgs& a) {
  const int steps = (a.max_context + 63) / 64;
  const int64_t units = plan_units(a.r.rows, a.n_heads / a.c.heads, a.c.heads, a.r.row_table != nullptr, &a.tiles);
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
  return (split < aim ? split : columns > aim ? columns : aim) * pitch;
}

void launch_quant_attention(const QuantAttnArgs& a, hipStream_t st) {
  const int G = a.n_heads / a.c.heads, C = 16 * a.tiles;
  const int y = a.r.row_table ? (int)(((int64_t)a.r.rows * G + C - 1) / C) : a.r.rows * ((G + C - 1) / C);
  const dim3 grid(a.c.heads, y, a.n_parts);
  a.c.format == EE_QUANT_INT8 ? launch_format<EE_QUANT_INT8>(a, grid, st) : launch_format<EE_QUANT_E4M3>(a, grid, st);
  if (!a.parts) return;
  const int chunks = a.weights_out ? (a.max_context + kWeightPositions - 1) / kWeightPositions : 0;
  quant_join_kernel<<<dim3((a.n_heads + 3) / 4 + a.c.heads * chunks, a.r.rows), 256, (size_t)G * sizeof(f32x2), st>>>(a);
}

}  // namespace ee
