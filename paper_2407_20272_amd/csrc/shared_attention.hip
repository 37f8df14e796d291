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
#include <type_traits>

#include "beams.h"

namespace ee {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int kWaves = 8;
constexpr int kThreads = kWaves * 64;
constexpr float kNegBig = -1.0e30f;
constexpr int kMostColumns = 48;    // of a tile (64 columns' sums and what is multiplied with them are more than 256 registers)
constexpr int kMostRows = kMostColumns;
constexpr int kMostWgs = 256, kMostParts = 256, kFewSteps = 16;   // workgroups that run at once; parts of a tile; steps that are worth a part
constexpr int kEarlyRows = 1024;    // up to so many rows' lengths are asked for together with the groups

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

// The tile's rows: found by the sums of the groups' tiles.  s_tile: first row, rows (0: there is no such tile), shared blocks.  The rows' lengths come along.
__device__ inline void find_tile(const SharedAttnArgs& a, int tile, int* s_tile, int* s_lens) {
  __shared__ int s_wave[kWaves];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  if (threadIdx.x == 0) s_tile[1] = 0;
  if (a.rows <= kEarlyRows)
    for (int m = threadIdx.x; m < a.rows; m += kThreads) s_lens[m] = a.context_lens[m];
  int sum = 0;
  for (int g0 = 0; g0 < a.n_groups; g0 += kThreads) {
    const int g = g0 + threadIdx.x;
    int first = 0, rows = 0, shared = 0;
    if (g < a.n_groups) {
      shared = a.shared_blocks[g];
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
    if (g0) __syncthreads();
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
      s_tile[2] = min(min(max(shared, 0), a.max_shared), a.max_blocks);
    }
  }
  __syncthreads();
}

// The maximum over the four lanes of a column.
__device__ inline float column_max(float x) {
  typedef uint32_t pair __attribute__((ext_vector_type(2)));
  const pair a = __builtin_bit_cast(pair, __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false));
  x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const pair b = __builtin_bit_cast(pair, __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false));
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// A lane's share of K and V in a step's two blocks, and of q.
template <class T, int DH>
struct Frags;
template <int DH>
struct Frags<bf16_t, DH> {
  static constexpr int KS = DH / 32, CT = DH / 16;   // contraction steps of q . K; tiles of 16 channels: channel m * CT + t is row m of tile t
  static constexpr int QP = 3;                       // 16-byte pieces of q a contraction step
  typedef uint32_t row_t __attribute__((ext_vector_type(CT / 2)));
  u32x4 k[2][KS];
  row_t v[2][4];
};
template <int DH>
struct Frags<float, DH> {
  static constexpr int KS = DH / 16, CT = DH / 16;
  static constexpr int QP = 1;
  f32x4 k[2][KS];
  f32x4 v[2][4][CT / 4];
};

template <class T, int DH, int NT>
__global__ __launch_bounds__(kThreads) void shared_attn_kernel(SharedAttnArgs a) {
  constexpr bool BF16 = sizeof(T) == 2;
  typedef Frags<T, DH> F;
  constexpr int KS = F::KS, CT = F::CT, QP = F::QP;
  constexpr int PITCH = DH + 4;                          // (of a column's sums in LDS: 16 columns' rows begin in 16 different groups of banks)
  constexpr size_t Q_BYTES = NT > 1 ? (size_t)NT * KS * QP * 1024 : 0, O_BYTES = (size_t)kWaves * 16 * PITCH * 4;
  __shared__ __align__(16) char s_space[Q_BYTES > O_BYTES ? Q_BYTES : O_BYTES];   // q [NT][KS][QP][64 lanes] of 16 bytes, then the wavefronts' sums
  __shared__ int s_tile[3];
  __shared__ int s_lens[kEarlyRows];
  __shared__ int s_first[kMostRows + 2];                 // of every run (the shared blocks, then the rows' own positions): steps before it
  __shared__ int s_from[kMostRows + 1], s_end[kMostRows + 1], s_seq[kMostRows + 1];   // its positions, and the block table that it walks
  __shared__ int s_with[kMostRows];                      // whether a row attends all shared blocks with the others
  __shared__ float s_m[kWaves][16], s_l[kWaves][16];

  const int kvh = blockIdx.x % a.kv_heads, hc = blockIdx.x / a.kv_heads;
  const int part = blockIdx.y, tile = blockIdx.z;   // (tiles that there are not come last)
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l16 = lane & 15, j = lane >> 4;
  find_tile(a, tile, s_tile, s_lens);
  const int row0 = __builtin_amdgcn_readfirstlane(s_tile[0]), n_rows = __builtin_amdgcn_readfirstlane(s_tile[1]);
  const bool writes_tile = a.parts > 1 && part == 0 && blockIdx.x == 0 && threadIdx.x == 0;
  if (n_rows == 0) {
    if (writes_tile) a.tile_of[tile] = make_int4(0, 0, 0, 0);
    return;
  }
  // The runs, by the first wavefront: lane r has row r.
  if (wave == 0) {
    const int m = row0 + min(lane, n_rows - 1);
    const int seq = a.row_table ? safe_row(a.row_table[m], a.rows) : m;
    const int len = a.rows <= kEarlyRows ? s_lens[m] : a.context_lens[m];
    const int shared = s_tile[2] * 16;
    const int npos = lane < n_rows ? min(max(len, -1), a.max_blocks * 16 - 1) + 1 : 0;
    const bool with = lane < n_rows && shared > 0 && npos >= shared;
    const unsigned long long who = __ballot(with);
    const int prefix_steps = who ? (shared + 31) >> 5 : 0;
    const int from = with ? shared : 0, steps = (npos - from + 31) >> 5;
    int upto = lane < n_rows ? steps : 0;
#pragma unroll
    for (int x = 1; x < 64; x <<= 1) {
      const int o = __shfl_up(upto, x);
      if (lane >= x) upto += o;
    }
    if (lane < n_rows) {
      s_first[lane + 1] = prefix_steps + upto - steps;
      s_from[lane + 1] = from;
      s_end[lane + 1] = npos;
      s_seq[lane + 1] = seq;
      s_with[lane] = with;
    }
    if (lane == n_rows - 1) s_first[n_rows + 1] = prefix_steps + upto;
    if (lane == (who ? __builtin_ctzll(who) : 0)) s_seq[0] = seq;
    if (lane == 0) {
      s_first[0] = 0;
      s_from[0] = 0;
      s_end[0] = shared;
    }
  }
  __syncthreads();
  const int total = __builtin_amdgcn_readfirstlane(s_first[n_rows + 1]);
  const int per = max((total + a.parts - 1) / a.parts, kWaves);
  const int live = max(1, (total + per - 1) / per);
  if (writes_tile) a.tile_of[tile] = make_int4(row0, n_rows, live, 0);
  if (part >= live) return;
  const int lo = part * per, hi = min(total, lo + per);
  const int nk = hi - lo > wave ? (hi - lo - wave + kWaves - 1) / kWaves : 0;   // steps of this wavefront: lo + wave + k * kWaves

  const size_t block_elems = (size_t)a.kv_heads * 16 * DH;
  const T* kpool = reinterpret_cast<const T*>(a.k) + (size_t)kvh * 16 * DH;
  const T* vpool = reinterpret_cast<const T*>(a.v) + (size_t)kvh * 16 * DH;
  // lane offsets within a block
  const int k_at = l16 * DH + j * (BF16 ? 8 : 4);     // position l16, channels + c * 32 (16)
  const int v_at = j * 4 * DH + l16 * CT;             // positions 4j + i, channels l16 * CT ..

  // The blocks of the wavefront's next 32 steps, two lanes a step (a step's second block may not be there: the first again, masked).
  int off_lo = 0, off_hi = 0;
  auto load_ids = [&](int k0) {
    const int s = min(lo + wave + (k0 + (lane >> 1)) * kWaves, hi - 1);
    int r = 0, z = n_rows;           // the last run that begins at or before s (runs without steps lie in front of the next)
    while (r < z) {
      const int mid = (r + z + 1) >> 1;
      if (s_first[mid] <= s) r = mid;
      else z = mid - 1;
    }
    const int at = s_from[r] + (s - s_first[r]) * 32 + (lane & 1) * 16;
    const int b = min(at, s_end[r] - 1) >> 4;
    const size_t off = (size_t)safe_block(a.block_tables[(size_t)s_seq[r] * a.max_blocks + b], a.num_blocks) * block_elems * sizeof(T);
    off_lo = (int)(uint32_t)off;
    off_hi = (int)(uint32_t)(off >> 32);
  };
  auto block_at = [&](const T* pool, int k, int b) {
    const int i = (2 * k + b) & 63;
    const uint32_t l = __builtin_amdgcn_readlane(off_lo, i), h = __builtin_amdgcn_readlane(off_hi, i);
    return reinterpret_cast<const T*>(reinterpret_cast<const char*>(pool) + ((size_t)h << 32 | l));
  };
  F f;
  auto load_k = [&](int k) {
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const T* kb = block_at(kpool, k, b) + k_at;
#pragma unroll
      for (int c = 0; c < KS; ++c) {
        if constexpr (BF16) f.k[b][c] = *reinterpret_cast<const u32x4*>(kb + c * 32);
        else f.k[b][c] = *reinterpret_cast<const f32x4*>(kb + c * 16);
      }
    }
  };
  auto load_v = [&](int k) {
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const T* vb = block_at(vpool, k, b) + v_at;
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
  };
  if (nk > 0) {
    load_ids(0);
    load_k(0);
    load_v(0);
  }

  // this lane's columns: l16 of every tile of 16
  const int gc = min(a.group - hc * a.columns, a.columns);              // query heads of a row in the tile
  const int n_columns = n_rows * gc, heads = a.kv_heads * a.group, head0 = kvh * a.group + hc * a.columns;
  const float scale = 1.4426950408889634f / sqrtf((float)DH);
  auto q_piece = [&](int column, int c, int jj, u32x4 (&piece)[QP]) {   // channels of contraction step c and lane group jj
    const bool ok = column < n_columns;
    const int r = ok ? column / gc : 0, h = ok ? column - r * gc : 0;
    const float* qp = a.q + ((size_t)(row0 + r) * heads + head0 + h) * DH;
    const float sc = ok ? scale : 0.0f;
    if constexpr (BF16) {
      const f32x4 x = *reinterpret_cast<const f32x4*>(qp + c * 32 + jj * 8), y = *reinterpret_cast<const f32x4*>(qp + c * 32 + jj * 8 + 4);
      const float v[8] = {x[0] * sc, x[1] * sc, x[2] * sc, x[3] * sc, y[0] * sc, y[1] * sc, y[2] * sc, y[3] * sc};
      split3(v, piece);
    } else {
      piece[0] = __builtin_bit_cast(u32x4, *reinterpret_cast<const f32x4*>(qp + c * 16 + jj * 4) * sc);
    }
  };
  u32x4 q1[NT == 1 ? KS : 1][QP];
  u32x4* q_lds = reinterpret_cast<u32x4*>(s_space);
  if constexpr (NT == 1) {
#pragma unroll
    for (int c = 0; c < KS; ++c) q_piece(l16, c, j, q1[c]);
  } else {
    for (int i = threadIdx.x; i < NT * KS * 64; i += kThreads) {
      const int ln = i & 63, c = (i >> 6) % KS, t = (i >> 6) / KS;
      u32x4 piece[QP];
      q_piece(t * 16 + (ln & 15), c, ln >> 4, piece);
#pragma unroll
      for (int p = 0; p < QP; ++p) q_lds[((t * KS + c) * QP + p) * 64 + ln] = piece[p];
    }
    __syncthreads();
  }
  int col_row[NT];
  bool col_with[NT];
  bool all_with = true;
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int column = t * 16 + l16;
    const bool ok = column < n_columns;
    col_row[t] = ok ? column / gc : -1;
    col_with[t] = ok && s_with[ok ? col_row[t] : 0];
    all_with = all_with && __all(!ok || col_with[t]);
  }

  float m_run[NT], l_run[NT];
  f32x4 o[NT][CT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    m_run[t] = kNegBig;
    l_run[t] = 0.0f;
#pragma unroll
    for (int u = 0; u < CT; ++u) o[t][u] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  }

  // A step whose positions all columns attend needs no masks (columns that are none have q = 0 and are not written): the first ones, in a loop of their own.
  auto step = [&](auto plain_c, int k, int run, int tok0, int end) {
    constexpr bool PLAIN = decltype(plain_c)::value;
    // the tiles of 16 columns that the step is for
    const int t_lo = run == 0 ? 0 : (run - 1) * gc >> 4, t_hi = run == 0 ? (n_columns - 1) >> 4 : (run * gc - 1) >> 4;
    auto scores = [&](int t, f32x4 (&st)[2]) {
      st[0] = st[1] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int c = 0; c < KS; ++c) {
        u32x4 qq[QP];
#pragma unroll
        for (int p = 0; p < QP; ++p) {
          if constexpr (NT == 1) qq[p] = q1[c][p];
          else qq[p] = q_lds[((t * KS + c) * QP + p) * 64 + lane];
        }
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          if constexpr (BF16) {
#pragma unroll
            for (int p = QP - 1; p >= 0; --p)
              st[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, f.k[b][c]), __builtin_bit_cast(bf16x8, qq[p]), st[b], 0, 0, 0);
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) st[b] = __builtin_amdgcn_mfma_f32_16x16x4f32(f.k[b][c][e], __uint_as_float(qq[0][e]), st[b], 0, 0, 0);
          }
        }
      }
    };
    auto next_k = [&] {
      if (k + 1 < nk) {
        if (((k + 1) & 31) == 0) load_ids(k + 1);   // (V of this step has been asked for: its blocks' ids are no longer needed)
        load_k(k + 1);
      }
    };
    constexpr bool EARLY = NT < 3;   // all scores first, so that the next K comes while the rest of the step is done; three tiles' do not fit beside it
    f32x4 st[EARLY ? NT : 1][2];
    if constexpr (EARLY) {
#pragma unroll
      for (int t = 0; t < NT; ++t)
        if (NT == 1 || (t <= t_hi && (PLAIN || t >= t_lo))) scores(t, st[t]);
      next_k();
    }
    if (!PLAIN && tok0 + 32 > end) {   // what nobody has cached may be anything: 0 times it has to be 0
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
    u32x4 vt[BF16 ? CT : 1];   // V^T: positions along a register, channels along the lanes
    if constexpr (BF16) {
#pragma unroll
      for (int u = 0; u < CT; ++u)
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const uint32_t x = f.v[w >> 1][2 * (w & 1)][u / 2], y = f.v[w >> 1][2 * (w & 1) + 1][u / 2];
          vt[u][w] = u & 1 ? high_halves(x, y) : low_halves(x, y);
        }
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      if (NT > 1 && (t > t_hi || (!PLAIN && t < t_lo))) continue;
      const bool mine = run == 0 ? col_with[t] : col_row[t] == run - 1;
      if constexpr (!EARLY) {
        scores(t, st[0]);
        if (t == t_hi) next_k();
      }
      float p[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) p[i] = st[EARLY ? t : 0][i >> 2][i & 3];
      if constexpr (!PLAIN) {
#pragma unroll
        for (int i = 0; i < 8; ++i) p[i] = mine && tok0 + (i >> 2) * 16 + j * 4 + (i & 3) < end ? p[i] : kNegBig;
      }
      float mx = m_run[t];
#pragma unroll
      for (int i = 0; i < 8; ++i) mx = fmaxf(mx, p[i]);
      mx = column_max(mx);
      // (the sums are relative to a maximum that follows only where it has grown by a factor of sqrt(2): they are rescaled less often)
      if (__any(mx > m_run[t] + 0.5f)) {
        const float alpha = __builtin_amdgcn_exp2f(m_run[t] - mx);
        m_run[t] = mx;
        l_run[t] *= alpha;
#pragma unroll
        for (int u = 0; u < CT; ++u) o[t][u] *= alpha;
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) p[i] = __builtin_amdgcn_exp2f(p[i] - m_run[t]);
      if constexpr (!PLAIN) {
#pragma unroll
        for (int i = 0; i < 8; ++i) p[i] = mine && tok0 + (i >> 2) * 16 + j * 4 + (i & 3) < end ? p[i] : 0.0f;
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) l_run[t] += p[i];
      u32x4 pp[3];
      if constexpr (BF16) split3(p, pp);
#pragma unroll
      for (int u = 0; u < CT; ++u) {
        f32x4 n = o[t][u];
        if constexpr (BF16) {
#pragma unroll
          for (int q = 2; q >= 0; --q) n = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vt[u]), __builtin_bit_cast(bf16x8, pp[q]), n, 0, 0, 0);
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) n = __builtin_amdgcn_mfma_f32_16x16x4f32(f.v[i >> 2][i & 3][u / 4][u % 4], p[i], n, 0, 0, 0);
        }
        // (0 times an Inf that another row has cached is NaN: only the columns the step is for take it)
        if constexpr (PLAIN) {
          o[t][u] = n;
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) o[t][u][e] = mine ? n[e] : o[t][u][e];
        }
      }
    }
    if (k + 1 < nk) load_v(k + 1);
  };
  const int plain_steps = all_with ? __builtin_amdgcn_readfirstlane(s_end[0]) >> 5 : 0;
  int k = 0;
  for (; k < nk && lo + wave + k * kWaves < plain_steps; ++k) step(std::true_type{}, k, 0, 0, 0);
  for (int run = 0; k < nk; ++k) {
    const int at = lo + wave + k * kWaves;
    while (at >= __builtin_amdgcn_readfirstlane(s_first[run + 1])) ++run;
    const int tok0 = __builtin_amdgcn_readfirstlane(s_from[run]) + (at - __builtin_amdgcn_readfirstlane(s_first[run])) * 32;
    step(std::false_type{}, k, run, tok0, __builtin_amdgcn_readfirstlane(s_end[run]));
  }

  // the four lanes of a column have sums over positions of their own; then the wavefronts, in order, 16 columns at a time
  typedef float sums_t[16][PITCH];
  sums_t* s_o = reinterpret_cast<sums_t*>(s_space);
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    if (t * 16 >= n_columns) break;
    if (t || NT > 1) __syncthreads();   // q, or the columns before, have been read
    float l = l_run[t];
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int u = 0; u < CT; u += 4)
        *reinterpret_cast<f32x4*>(&s_o[wave][l16][(j * 4 + i) * CT + u]) = f32x4{o[t][u][i], o[t][u + 1][i], o[t][u + 2][i], o[t][u + 3][i]};
    if (j == 0) {
      s_m[wave][l16] = m_run[t];
      s_l[wave][l16] = l;
    }
    __syncthreads();
    for (int x = threadIdx.x; x < 16 * (DH / 4); x += kThreads) {
      const int c = x / (DH / 4), ch = x % (DH / 4) * 4, column = t * 16 + c;
      if (column >= n_columns) continue;
      const int r = column / gc;
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
        const float inv = s_end[r + 1] > 0 ? 1.0f / L : 0.0f;      // a row without a position: 0
        *reinterpret_cast<f32x4*>(a.out + ((size_t)(row0 + r) * heads + head0 + column - r * gc) * DH + ch) = acc * inv;
      } else {
        float* rec = a.records + ((((size_t)tile * a.head_chunks + hc) * a.kv_heads + kvh) * a.parts + part) * a.columns * PITCH + (size_t)column * PITCH;
        if (ch == 0) *reinterpret_cast<f32x4*>(rec) = f32x4{M, L, 0.0f, 0.0f};
        *reinterpret_cast<f32x4*>(rec + 4 + ch) = acc;
      }
    }
  }
}

// Adds the parts of a tile's columns: a workgroup has one column, DH / 4 threads to every eighth (sixteenth) part; then these, in order.
template <int DH>
__global__ __launch_bounds__(256) void shared_join_kernel(SharedAttnArgs a) {
  constexpr int TH = DH / 4, G = 256 / TH, PITCH = DH + 4;
  __shared__ __align__(16) float s_acc[G][DH];
  __shared__ float s_m[G], s_l[G];
  const int kvh = blockIdx.x % a.kv_heads, hc = blockIdx.x / a.kv_heads, tile = blockIdx.y, c = blockIdx.z;
  const int4 td = a.tile_of[tile];
  const int gc = min(a.group - hc * a.columns, a.columns);
  if (td.z < 2 || c >= td.y * gc) return;
  const int g = threadIdx.x / TH, ch = threadIdx.x % TH * 4, r = c / gc;
  const float* rec = a.records + (((size_t)tile * a.head_chunks + hc) * a.kv_heads + kvh) * a.parts * a.columns * PITCH + (size_t)c * PITCH;
  const size_t pitch = (size_t)a.columns * PITCH;
  float M = kNegBig, L = 0.0f;
  f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int p = g; p < td.z; p += G) {
    const float m = rec[p * pitch], l = rec[p * pitch + 1];
    const f32x4 x = *reinterpret_cast<const f32x4*>(rec + p * pitch + 4 + ch);
    const float to = fmaxf(M, m), was = __builtin_amdgcn_exp2f(M - to), now = __builtin_amdgcn_exp2f(m - to);
    L = L * was + l * now;
    acc = acc * was + x * now;
    M = to;
  }
  *reinterpret_cast<f32x4*>(&s_acc[g][ch]) = acc;
  if (ch == 0) {
    s_m[g] = M;
    s_l[g] = L;
  }
  __syncthreads();
  if (g) return;
  M = kNegBig;
#pragma unroll
  for (int i = 0; i < G; ++i) M = fmaxf(M, s_m[i]);
  L = 0.0f;
  acc = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int i = 0; i < G; ++i) {
    const float w = __builtin_amdgcn_exp2f(s_m[i] - M);
    L += s_l[i] * w;
    acc += *reinterpret_cast<const f32x4*>(&s_acc[i][ch]) * w;
  }
  const float inv = a.context_lens[td.x + r] >= 0 ? 1.0f / L : 0.0f;
  const int head = kvh * a.group + hc * a.columns + c - r * gc;
  *reinterpret_cast<f32x4*>(a.out + ((size_t)(td.x + r) * a.kv_heads * a.group + head) * DH + ch) = acc * inv;
}

template <class T, int DH, int NT>
void launch_tiles(const SharedAttnArgs& a, hipStream_t st) {
  shared_attn_kernel<T, DH, NT><<<dim3(a.kv_heads * a.head_chunks, a.parts, a.tiles), kThreads, 0, st>>>(a);
  if (a.parts > 1) shared_join_kernel<DH><<<dim3(a.kv_heads * a.head_chunks, a.tiles, a.columns), 256, 0, st>>>(a);
}

template <class T, int DH>
void launch(const SharedAttnArgs& a, hipStream_t st) {
  if (a.columns == 16) launch_tiles<T, DH, 1>(a, st);
  else if (a.columns == 32) launch_tiles<T, DH, 2>(a, st);
  else if constexpr (sizeof(T) == 2) launch_tiles<T, DH, 3>(a, st);
}

}  // namespace

// A tile's width, and what goes with it.
static void tile_widths(SharedAttnArgs& a, int columns, int most) {
  a.head_chunks = (a.group + most - 1) / most;
  if (a.head_chunks > 1) columns = ((a.group + a.head_chunks - 1) / a.head_chunks + 15) / 16 * 16;
  a.columns = columns < 16 ? 16 : columns;
  if (a.group > a.columns && a.head_chunks == 1) a.columns = (a.group + 15) / 16 * 16;
  a.rows_per_tile = a.group < a.columns ? a.columns / a.group : 1;
  while (a.columns > 16 && a.rows_per_tile * a.group <= a.columns - 16 && a.head_chunks == 1) a.columns -= 16;   // (no more columns than rows fill)
}

// Tiles that all groups together have at most: a group's last one may have fewer rows.
static int most_tiles(const SharedAttnArgs& a) { return (int)(((int64_t)a.rows + (int64_t)a.n_groups * (a.rows_per_tile - 1)) / a.rows_per_tile); }

void shared_attn_plan(SharedAttnArgs& a, int dtype) {
  // As many columns as a group has on average: a tile's shared blocks are read once.
  const int most = dtype == EE_FP32 ? 32 : kMostColumns;
  const int64_t columns = ((int64_t)a.rows * a.group + a.n_groups - 1) / a.n_groups;
  tile_widths(a, columns > most ? most : (int)(columns + 15) / 16 * 16, most);
  a.tiles = most_tiles(a);
  const int64_t wgs = (int64_t)a.tiles * a.kv_heads * a.head_chunks;
  const int64_t steps = (a.max_context + 31) / 32;
  int64_t parts = kMostWgs / wgs;
  if (parts > steps / kFewSteps) parts = steps / kFewSteps;
  if (parts > kMostParts) parts = kMostParts;
  a.parts = parts < 2 ? 1 : (int)parts;
}

size_t shared_attn_record_floats(const SharedAttnArgs& a) {
  return a.parts > 1 ? (size_t)a.tiles * a.kv_heads * a.head_chunks * a.parts * a.columns * (a.dh + 4) : 0;
}

// For calls of fewer rows, groups and positions, which may have narrower tiles.  Of each width the tiles grow with rows and groups; the parts of all of them together
// are at most kMostWgs where there are any.
size_t shared_attn_most_floats(SharedAttnArgs& a, int dtype, size_t* tiles) {
  size_t most = 0;
  const int64_t steps = (a.max_context + 31) / 32, apart = steps / kFewSteps;
  const int widest = dtype == EE_FP32 ? 32 : kMostColumns;
  *tiles = 0;
  for (int columns = 16; columns <= widest; columns += 16) {
    tile_widths(a, columns, widest);
    a.tiles = most_tiles(a);
    if (*tiles < (size_t)a.tiles) *tiles = a.tiles;
    const size_t floats = (size_t)kMostWgs * a.columns * (a.dh + 4);
    if (most < floats) most = floats;
  }
  if (apart < 2) most = *tiles = 0;
  if (*tiles > kMostWgs) *tiles = kMostWgs;   // (more of them have one part each)
  shared_attn_plan(a, dtype);
  return most;
}

void launch_shared_attention(const SharedAttnArgs& a, int dtype, hipStream_t st) {
  if (dtype == EE_BF16) a.dh == 64 ? launch<bf16_t, 64>(a, st) : launch<bf16_t, 128>(a, st);
  else a.dh == 64 ? launch<float, 64>(a, st) : launch<float, 128>(a, st);
}

}  // namespace ee
