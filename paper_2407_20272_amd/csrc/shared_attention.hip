// Attention of single positions whose sequences begin with the same blocks (beams of one prompt, questions about one document): those blocks are read
// once for all rows of a group, not once a row.
//
//   out[m][h] = softmax_j(q[m][h] . K[j][h / g] / sqrt(dh)) . V[j][h / g],   j = 0..context_lens[m]
//
// A column is a row and one of the g query heads that share a K/V head.  A tile is up to 16 * NT columns of one group.  Its walk is one list of steps
// of 32 positions: first the shared blocks, multiplied with every column, then each row's own positions, which count for that row's columns alone.  The list
// is divided into equal parts (a workgroup each), a part's steps go round its wavefronts, and where there is more than one part a second launch joins them.
//
// Both products are transposed, so that no value changes lanes between them:
//   scores^T [position][column] = K [position][dh] . q^T,      out^T [dh][column] += V^T [dh][position] . p^T
// A lane ends the first with positions 4j..4j+3 of two blocks (j = lane / 16) of one column, and these are the positions that it contracts over in the second:
// V's lanes load the same ones, a row's 16 bytes each, and turn eight rows of eight channels around in registers.  Nothing passes through LDS.
// bf16: q and the probabilities are split into three bf16 parts, 24 bits, multiplied one after the other: float in effect, with a float's range.  fp32: the float matrix instructions.
#include "beams.h"

namespace ee {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int kWaves = 4;
constexpr int kThreads = kWaves * 64;
constexpr float kNegBig = -1.0e30f;
constexpr int kMostRows = 64;   // of a tile

// The upper halves of two words (two floats truncated to bf16), the first in the low half.
__device__ inline uint32_t high_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }
__device__ inline uint32_t low_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }

// Eight floats as three bf16 parts, whose sum is the float (truncated parts: 8 + 8 + 8 bits; what is infinite or NaN becomes NaN).
__device__ inline void split3(const float (&x)[8], u32x4 (&part)[3]) {
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    float a = x[2 * w], b = x[2 * w + 1];
#pragma unroll
    for (int p = 0; p < 3; ++p) {
      const uint32_t ua = __float_as_uint(a), ub = __float_as_uint(b);
      part[p][w] = high_halves(ua, ub);
      a -= __uint_as_float(ua & 0xffff0000u);
      b -= __uint_as_float(ub & 0xffff0000u);
    }
  }
}

// The tile's rows: found by the sums of the groups' tiles.  s_tile: first row, rows (0: there is no such tile), group.
__device__ inline void find_tile(const SharedAttnArgs& a, int tile, int* s_tile) {
  __shared__ int s_wave[kWaves];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  if (threadIdx.x == 0) s_tile[1] = 0;
  int sum = 0;
  for (int g0 = 0; g0 < a.n_groups; g0 += kThreads) {
    const int g = g0 + threadIdx.x;
    int first = 0, rows = 0;
    if (g < a.n_groups) {
      first = min(max(a.first_row[g], 0), a.rows);
      rows = min(max(a.first_row[g + 1], first), a.rows) - first;
    }
    const int tiles = (rows + a.rows_per_tile - 1) / a.rows_per_tile;
    int upto = tiles;
#pragma unroll
    for (int x = 1; x < 64; x <<= 1) {
      const int o = __shfl_up(upto, x);
      if (lane >= x) upto += o;
    }
    __syncthreads();
    if (lane == 63) s_wave[wave] = upto;
    __syncthreads();
    int before = sum + upto - tiles;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) {
      if (i < wave) before += s_wave[i];
      sum += s_wave[i];
    }
    if (tile >= before && tile < before + tiles) {
      const int r0 = (tile - before) * a.rows_per_tile;
      s_tile[0] = first + r0;
      s_tile[1] = min(a.rows_per_tile, rows - r0);
      s_tile[2] = g;
    }
  }
  __syncthreads();
}

// Fragments of a step's two blocks.
template <class T, int DH>
struct Frags;
template <int DH>
struct Frags<bf16_t, DH> {
  static constexpr int KS = DH / 32, CT = DH / 16;   // contraction steps of q . K; tiles of 16 channels: channel m * CT + t is row m of tile t
  u32x4 k[2][KS];
  typedef uint32_t row_t __attribute__((ext_vector_type(CT / 2)));
  row_t v[2][4];
};
template <int DH>
struct Frags<float, DH> {
  static constexpr int KS = DH / 16, CT = DH / 16;
  f32x4 k[2][KS];
  f32x4 v[2][4][CT / 4];
};

template <class T, int DH>
__global__ __launch_bounds__(kThreads) void shared_attn_kernel(SharedAttnArgs a) {
  constexpr bool BF16 = sizeof(T) == 2;
  typedef Frags<T, DH> F;
  constexpr int KS = F::KS, CT = F::CT;
  __shared__ int s_tile[3];
  __shared__ int s_first[kMostRows + 2];                 // of every run (the shared blocks, then the rows' own positions): steps before it
  __shared__ int s_from[kMostRows + 1], s_end[kMostRows + 1], s_row[kMostRows + 1];   // its positions, and the row whose table it walks (of the tile's)
  __shared__ int s_with[kMostRows];                      // whether a row attends all shared blocks with the others
  __shared__ float s_m[kWaves][16], s_l[kWaves][16];
  __shared__ __align__(16) float s_o[kWaves][16][DH];

  const int kvh = blockIdx.x % a.kv_heads, hc = blockIdx.x / a.kv_heads;
  const int tile = blockIdx.y, part = blockIdx.z;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l16 = lane & 15, j = lane >> 4;
  find_tile(a, tile, s_tile);
  const int row0 = __builtin_amdgcn_readfirstlane(s_tile[0]), n_rows = __builtin_amdgcn_readfirstlane(s_tile[1]);
  const bool writes_tile = a.parts > 1 && part == 0 && blockIdx.x == 0 && threadIdx.x == 0;
  if (n_rows == 0) {
    if (writes_tile) a.tile_of[tile] = make_int4(0, 0, 0, 0);
    return;
  }
  auto seq_of = [&](int m) { return a.row_table ? safe_row(a.row_table[m], a.rows) : m; };
  // The runs, by the first wavefront: lane r has row r.
  if (wave == 0) {
    const int shared = min(min(max(a.shared_blocks[s_tile[2]], 0), a.max_shared), a.max_blocks) * 16;
    const int npos = lane < n_rows ? min(max(a.context_lens[row0 + lane], -1), a.max_blocks * 16 - 1) + 1 : 0;
    const bool with = lane < n_rows && shared > 0 && npos >= shared;
    const int prefix_steps = __any(with) ? (shared + 31) >> 5 : 0;
    const int from = with ? shared : 0, steps = lane < n_rows ? (npos - from + 31) >> 5 : 0;
    int upto = steps;
#pragma unroll
    for (int x = 1; x < 64; x <<= 1) {
      const int o = __shfl_up(upto, x);
      if (lane >= x) upto += o;
    }
    const unsigned long long who = __ballot(with);
    if (lane < n_rows) {
      s_first[lane + 1] = prefix_steps + upto - steps;
      s_from[lane + 1] = from;
      s_end[lane + 1] = npos;
      s_row[lane + 1] = lane;
      s_with[lane] = with;
    }
    if (lane == n_rows - 1) s_first[n_rows + 1] = prefix_steps + upto;
    if (lane == 0) {
      s_first[0] = 0;
      s_from[0] = 0;
      s_end[0] = shared;
      s_row[0] = who ? __builtin_ctzll(who) : 0;
    }
  }
  __syncthreads();
  const int total = __builtin_amdgcn_readfirstlane(s_first[n_rows + 1]);
  const int per = max((total + a.parts - 1) / a.parts, 2 * kWaves);
  const int live = max(1, (total + per - 1) / per);
  if (writes_tile) a.tile_of[tile] = make_int4(row0, n_rows, live, 0);
  if (part >= live) return;
  const int lo = part * per, hi = min(total, lo + per);

  // this lane's column
  const int gc = min(a.group - hc * a.columns, a.columns);              // query heads of a row in the tile
  const int col_row = l16 / gc, col_head = kvh * a.group + hc * a.columns + l16 % gc;
  const bool col_ok = col_row < n_rows;
  const int heads = a.kv_heads * a.group;
  const bool col_with = col_ok && s_with[col_ok ? col_row : 0];
  const bool all_with = __all(!col_ok || col_with);
  const float* qp = a.q + ((size_t)(row0 + (col_ok ? col_row : 0)) * heads + col_head) * DH;
  const float scale = col_ok ? 1.4426950408889634f / sqrtf((float)DH) : 0.0f;
  u32x4 qb[BF16 ? KS : 1][3];
  f32x4 qf[BF16 ? 1 : KS];
  if constexpr (BF16) {
#pragma unroll
    for (int c = 0; c < KS; ++c) {
      const f32x4 x = *reinterpret_cast<const f32x4*>(qp + c * 32 + j * 8), y = *reinterpret_cast<const f32x4*>(qp + c * 32 + j * 8 + 4);
      const float v[8] = {x[0] * scale, x[1] * scale, x[2] * scale, x[3] * scale, y[0] * scale, y[1] * scale, y[2] * scale, y[3] * scale};
      split3(v, qb[c]);
    }
  } else {
#pragma unroll
    for (int c = 0; c < KS; ++c) qf[c] = *reinterpret_cast<const f32x4*>(qp + c * 16 + j * 4) * scale;
  }

  const size_t block_elems = (size_t)a.kv_heads * 16 * DH;
  const T* kpool = reinterpret_cast<const T*>(a.k) + (size_t)kvh * 16 * DH;
  const T* vpool = reinterpret_cast<const T*>(a.v) + (size_t)kvh * 16 * DH;
  // lane offsets within a block
  const int k_at = l16 * DH + j * (BF16 ? 8 : 4);     // position l16, channels + c * 32 (16)
  const int v_at = j * 4 * DH + l16 * CT;             // positions 4j + i, channels l16 * CT ..

  float m_run = kNegBig, l_run = 0.0f;
  f32x4 o[CT];
#pragma unroll
  for (int t = 0; t < CT; ++t) o[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

  int run = 0;
  for (int s = lo + wave; s < hi; s += kWaves) {
    while (s >= __builtin_amdgcn_readfirstlane(s_first[run + 1])) ++run;
    const int first = __builtin_amdgcn_readfirstlane(s_first[run]);
    const int tok0 = __builtin_amdgcn_readfirstlane(s_from[run]) + (s - first) * 32, end = __builtin_amdgcn_readfirstlane(s_end[run]);
    const int32_t* table = a.block_tables + (size_t)seq_of(row0 + __builtin_amdgcn_readfirstlane(s_row[run])) * a.max_blocks;
    const int b0 = tok0 >> 4, b1 = min(b0 + 1, (end - 1) >> 4);     // (a step's second block may not be there: the first again, masked)
    const size_t at0 = (size_t)safe_block(table[b0], a.num_blocks) * block_elems, at1 = (size_t)safe_block(table[b1], a.num_blocks) * block_elems;
    F f;
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const T* kb = kpool + (b ? at1 : at0) + k_at;
#pragma unroll
      for (int c = 0; c < KS; ++c) {
        if constexpr (BF16) f.k[b][c] = *reinterpret_cast<const u32x4*>(kb + c * 32);
        else f.k[b][c] = *reinterpret_cast<const f32x4*>(kb + c * 16);
      }
    }
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const T* vb = vpool + (b ? at1 : at0) + v_at;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (BF16) {
          f.v[b][i] = *reinterpret_cast<const typename F::row_t*>(vb + i * DH);
        } else {
#pragma unroll
          for (int u = 0; u < CT / 4; ++u) f.v[b][i][u] = *reinterpret_cast<const f32x4*>(vb + i * DH + u * 4);
        }
      }
    }
    f32x4 st[2];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      st[b] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int c = 0; c < KS; ++c) {
        if constexpr (BF16) {
#pragma unroll
          for (int p = 2; p >= 0; --p)
            st[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, f.k[b][c]), __builtin_bit_cast(bf16x8, qb[c][p]), st[b], 0, 0, 0);
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) st[b] = __builtin_amdgcn_mfma_f32_16x16x4f32(f.k[b][c][e], qf[c][e], st[b], 0, 0, 0);
        }
      }
    }
    const bool mine = run == 0 ? col_with : col_ok && col_row == run - 1;
    const bool all_mine = run == 0 && all_with;          // (columns that are none have q = 0 and are not written)
    const bool whole = tok0 + 32 <= end;
    if (!whole || !all_mine) {
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i) st[b][i] = mine && tok0 + b * 16 + j * 4 + i < end ? st[b][i] : kNegBig;
    }
    float mx = m_run;
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int i = 0; i < 4; ++i) mx = fmaxf(mx, st[b][i]);
    mx = fmaxf(mx, __shfl_xor(mx, 16));
    mx = fmaxf(mx, __shfl_xor(mx, 32));
    // (the sums are relative to a maximum that follows only where it has grown by a factor of sqrt(2): they are rescaled less often)
    if (__any(mx > m_run + 0.5f)) {
      const float alpha = __builtin_amdgcn_exp2f(m_run - mx);
      m_run = mx;
      l_run *= alpha;
#pragma unroll
      for (int t = 0; t < CT; ++t) o[t] *= alpha;
    }
    float p[8];
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int i = 0; i < 4; ++i) p[b * 4 + i] = __builtin_amdgcn_exp2f(st[b][i] - m_run);
    if (!whole || !all_mine) {
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i) p[b * 4 + i] = mine && tok0 + b * 16 + j * 4 + i < end ? p[b * 4 + i] : 0.0f;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) l_run += p[i];
    if (!whole) {   // what nobody has cached may be anything: 0 times it has to be 0
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const bool there = tok0 + b * 16 + j * 4 + i < end;
          if constexpr (BF16) {
#pragma unroll
            for (int u = 0; u < CT / 2; ++u) f.v[b][i][u] = there ? f.v[b][i][u] : 0u;
          } else {
#pragma unroll
            for (int u = 0; u < CT / 4; ++u)
#pragma unroll
              for (int e = 0; e < 4; ++e) f.v[b][i][u][e] = there ? f.v[b][i][u][e] : 0.0f;
          }
        }
    }
    u32x4 pp[3];
    if constexpr (BF16) split3(p, pp);
#pragma unroll
    for (int t = 0; t < CT; ++t) {
      f32x4 n = o[t];
      if constexpr (BF16) {
        u32x4 vt;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const uint32_t x = f.v[w >> 1][2 * (w & 1)][t / 2], y = f.v[w >> 1][2 * (w & 1) + 1][t / 2];
          vt[w] = t & 1 ? high_halves(x, y) : low_halves(x, y);
        }
#pragma unroll
        for (int q = 2; q >= 0; --q) n = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vt), __builtin_bit_cast(bf16x8, pp[q]), n, 0, 0, 0);
      } else {
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int i = 0; i < 4; ++i) n = __builtin_amdgcn_mfma_f32_16x16x4f32(f.v[b][i][t / 4][t % 4], p[b * 4 + i], n, 0, 0, 0);
      }
      // (0 times an Inf that another row has cached is NaN: only the columns the step is for take it)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[t][e] = all_mine || mine ? n[e] : o[t][e];
    }
  }

  // the four lanes of a column have sums over positions of their own; then the wavefronts, in order
  l_run += __shfl_xor(l_run, 16);
  l_run += __shfl_xor(l_run, 32);
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int t = 0; t < CT; t += 4)
      *reinterpret_cast<f32x4*>(&s_o[wave][l16][(j * 4 + i) * CT + t]) = f32x4{o[t][i], o[t + 1][i], o[t + 2][i], o[t + 3][i]};
  if (j == 0) {
    s_m[wave][l16] = m_run;
    s_l[wave][l16] = l_run;
  }
  __syncthreads();
  for (int u = threadIdx.x; u < 16 * (DH / 4); u += kThreads) {
    const int c = u / (DH / 4), ch = u % (DH / 4) * 4;
    const int r = c / gc;
    if (r >= n_rows) continue;
    float M = kNegBig, L = 0.0f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) M = fmaxf(M, s_m[w][c]);
    f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float wgt = __builtin_amdgcn_exp2f(s_m[w][c] - M);
      L += s_l[w][c] * wgt;
      acc += *reinterpret_cast<const f32x4*>(&s_o[w][c][ch]) * wgt;
    }
    if (live == 1) {
      const int head = kvh * a.group + hc * a.columns + c % gc;
      const float inv = s_end[r + 1] > 0 ? 1.0f / L : 0.0f;      // a row without a position: 0
      *reinterpret_cast<f32x4*>(a.out + ((size_t)(row0 + r) * heads + head) * DH + ch) = acc * inv;
    } else {
      float* rec = a.records + ((((size_t)tile * a.head_chunks + hc) * a.kv_heads + kvh) * a.parts + part) * a.columns * (DH + 4) + (size_t)c * (DH + 4);
      if (ch == 0) *reinterpret_cast<f32x4*>(rec) = f32x4{M, L, 0.0f, 0.0f};
      *reinterpret_cast<f32x4*>(rec + 4 + ch) = acc;
    }
  }
}

// Adds the parts of a tile's columns in their order: a workgroup has 8 columns, 32 threads each.
template <int DH>
__global__ __launch_bounds__(kThreads) void shared_join_kernel(SharedAttnArgs a) {
  const int kvh = blockIdx.x % a.kv_heads, hc = blockIdx.x / a.kv_heads, tile = blockIdx.y;
  const int4 td = a.tile_of[tile];
  if (td.y == 0 || td.z < 2) return;
  const int gc = min(a.group - hc * a.columns, a.columns);
  const int c = blockIdx.z * 8 + (threadIdx.x >> 5), r = c / gc;
  if (c >= a.columns || r >= td.y) return;
  const float* rec = a.records + (((size_t)tile * a.head_chunks + hc) * a.kv_heads + kvh) * a.parts * a.columns * (DH + 4) + (size_t)c * (DH + 4);
  const size_t pitch = (size_t)a.columns * (DH + 4);
  float M = kNegBig, L = 0.0f;
  for (int p = 0; p < td.z; ++p) M = fmaxf(M, rec[p * pitch]);
  constexpr int PER = DH / 32;
  float acc[PER] = {};
  const int ch = (threadIdx.x & 31) * PER;
  for (int p = 0; p < td.z; ++p) {
    const float wgt = __builtin_amdgcn_exp2f(rec[p * pitch] - M);
    L += rec[p * pitch + 1] * wgt;
#pragma unroll
    for (int e = 0; e < PER; ++e) acc[e] += rec[p * pitch + 4 + ch + e] * wgt;
  }
  const int head = kvh * a.group + hc * a.columns + c % gc;
  const bool some = a.context_lens[td.x + r] >= 0;
  const float inv = some ? 1.0f / L : 0.0f;
#pragma unroll
  for (int e = 0; e < PER; ++e) a.out[((size_t)(td.x + r) * a.kv_heads * a.group + head) * DH + ch + e] = acc[e] * inv;
}

template <class T, int DH>
void launch(const SharedAttnArgs& a, hipStream_t st) {
  shared_attn_kernel<T, DH><<<dim3(a.kv_heads * a.head_chunks, a.tiles, a.parts), kThreads, 0, st>>>(a);
  if (a.parts > 1) shared_join_kernel<DH><<<dim3(a.kv_heads * a.head_chunks, a.tiles, (a.columns + 7) / 8), kThreads, 0, st>>>(a);
}

}  // namespace

void shared_attn_plan(SharedAttnArgs& a, int dtype) {
  a.columns = 16;
  a.rows_per_tile = a.group < a.columns ? a.columns / a.group : 1;
  a.head_chunks = (a.group + a.columns - 1) / a.columns;
  a.tiles = a.rows / a.rows_per_tile + a.n_groups;   // (a group's last tile may have fewer rows)
  const int64_t wgs = (int64_t)a.tiles * a.kv_heads * a.head_chunks;
  const int64_t steps = (a.max_context + 31) / 32;
  int64_t parts = (1024 + wgs - 1) / wgs;
  if (parts > steps / 8) parts = steps / 8;
  if (parts > 64) parts = 64;
  a.parts = parts < 2 ? 1 : (int)parts;
}

size_t shared_attn_record_floats(const SharedAttnArgs& a) {
  return a.parts > 1 ? (size_t)a.tiles * a.kv_heads * a.head_chunks * a.parts * a.columns * (a.dh + 4) : 0;
}

// (wgs * parts is at most wgs + 1023, and no more than 64 or steps / 8 times wgs: each grows with rows, groups and context)
size_t shared_attn_most_floats(SharedAttnArgs& a, int dtype, size_t* tiles) {
  shared_attn_plan(a, dtype);
  const size_t wgs = (size_t)a.tiles * a.kv_heads * a.head_chunks, steps = (size_t)(a.max_context + 31) / 32;
  size_t units = wgs + 1023;
  if (units > wgs * 64) units = wgs * 64;
  if (units > wgs * (steps / 8)) units = wgs * (steps / 8);
  *tiles = steps / 8 >= 2 ? a.tiles : 0;
  return steps / 8 >= 2 ? units * a.columns * (a.dh + 4) : 0;
}

void launch_shared_attention(const SharedAttnArgs& a, int dtype, hipStream_t st) {
  if (dtype == EE_BF16) a.dh == 64 ? launch<bf16_t, 64>(a, st) : launch<bf16_t, 128>(a, st);
  else a.dh == 64 ? launch<float, 64>(a, st) : launch<float, 128>(a, st);
}

}  // namespace ee
