// Attention of single positions whose sequences begin with the same blocks (beams of one prompt, questions about one document): those blocks are read
// once for all rows of a group, not once a row.
//
//   out[m][h] = softmax_j(q[m][h] . K[j][h / g] / sqrt(dh)) . V[j][h / g],   j = 0..context_lens[m]
//
// A column is a row and one of the g query heads that share a K/V head.  A tile is 16, 32 or 48 columns of one group, the next that hold a group on average: its walk is one list of
// steps of 32 positions, first the shared blocks, multiplied with every column, then each row's own positions, which count for that row's columns alone.  A workgroup of eight
// wavefronts, which take the steps in turn, has a tile, or one of the equal parts of it that its share of all steps is worth (`dealt`: a second launch joins them, by maximum and sum).
//
// Both products are transposed, so that no value changes lanes between them:
//   scores^T [position][column] = K [position][dh] . q^T,      out^T [dh][column] += V^T [dh][position] . p^T
// A lane ends the first with positions 4j..4j+3 of two blocks (j = lane / 16) of one column, and these are the positions that it contracts over in the second:
// V's lanes load the same ones, a row's 16 bytes each, and turn eight rows of eight channels around in registers.  K and V never pass through LDS; q does where there is more than one
// tile of 16 columns.  bf16: q and the probabilities are split into three bf16 parts, 24 bits, multiplied one after the other: float in effect, with a float's range (relative error
// 3.1e-7 on 4 rows behind 96 positions; with the probabilities in two parts 5.1e-6, and the long cases below 4 % faster).  fp32: the float matrix instructions.
//
// Bound by what a compute unit takes in (26 GB/s of memory, 28 to 30 with what comes from cache), and for short contexts by the chain in front of it: groups and lengths, block ids, K and V (4 us),
// and the meeting of the wavefronts (1.5 us).  Kernel times, bf16, dh 128, 32 query heads:
//   4 rows behind 96 positions, heads of their own: 7.4 to 8.2 us.    8 x 4 rows behind 512 (85 MB): 17.8 us, 12.5 at 6.8 TB/s.
//   64 rows behind 2000, 100 to 900 of their own, over 8 heads (141 MB): 35.2 + 4.7 us, 20.8 at 6.8 TB/s (tiles of 16 columns 50, of 32 37; whole tiles a workgroup 50 in tiles of 16).
//   48 rows behind 100000, heads of their own (1.7 GB, 52 steps a wavefront): 336 us in all, 5.1 TB/s.
//   12 rows behind 100000 over 8 heads (410 MB): 82 to 85 + 4.8 us, 60 at 6.8 TB/s (16 columns 130, 32 124; whole tiles 932).  The counters show no byte read twice.  K through LDS, in whole kilobytes and a step ahead: 39 and 94 us.
//   Four wavefronts a workgroup were 62 and 220 us where eight were 43 and 156; with tiles that begin in the middle of a workgroup's share of steps the 64 rows took 40.
#include <type_traits>

#include "beams.h"

namespace ee {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int kWaves = 8;
constexpr int kThreads = kWaves * 64;
constexpr float kNegBig = -3.4028235e38f;   // the lowest float: no score that is one is below it
constexpr int kMostColumns = 48;    // of a tile (64 columns' sums and what is multiplied with them are more than 256 registers)
constexpr int kMostRows = kMostColumns;
constexpr int kMostWgs = 256;   // workgroups that run at once
// Steps of a tile of up to 16 KB (half as many of 32) from which its parts are worth the second launch (5 us and a gap): 39 steps of 35 float rows in 7 groups took 11 to 13 us as whole tiles,
// 13.3 + 4 dealt out; 31 steps of 32 KB, 45 rows in 15 groups, 28 us whole and 22 dealt out.
constexpr int kWorthDealing = 64;
constexpr int kDealRows = 1024, kDealGroups = 512, kDealTiles = 512;   // up to so many are dealt out

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

// Sums over the lanes up to each one, on the cross-lane network.
__device__ inline int wave_sums(int v) {
  auto add = [&](auto ctrl, auto rows) { v += __builtin_amdgcn_update_dpp(0, v, decltype(ctrl)::value, decltype(rows)::value, 0xf, false); };
  add(std::integral_constant<int, 0x111>{}, std::integral_constant<int, 0xf>{});   // row_shr 1, 2, 4, 8
  add(std::integral_constant<int, 0x112>{}, std::integral_constant<int, 0xf>{});
  add(std::integral_constant<int, 0x114>{}, std::integral_constant<int, 0xf>{});
  add(std::integral_constant<int, 0x118>{}, std::integral_constant<int, 0xf>{});
  add(std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xa>{});   // row_bcast 15, 31
  add(std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xc>{});
  return v;
}

// The sum of the values of the threads before each, over the workgroup, and of all.
__device__ inline int block_sums(int v, int* s_wave, int& all) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int upto = wave_sums(v);
  __syncthreads();
  if (lane == 63) s_wave[wave] = upto;
  __syncthreads();
  int before = upto - v;
  all = 0;
#pragma unroll
  for (int i = 0; i < kWaves; ++i) {
    if (i < wave) before += s_wave[i];
    all += s_wave[i];
  }
  return before;
}

// The last of n ascending numbers that is at most x (the first where none is).
__device__ inline int last_within(const int* s, int n, int x) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (s[mid] <= x) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

struct Group {
  int first, rows, shared;   // shared: blocks
};
__device__ inline Group group_of(const SharedAttnArgs& a, int g) {
  Group r{0, 0, 0};
  if (g < a.n_groups) {
    const int first = a.first_row[g], next = a.first_row[g + 1], shared = a.shared_blocks[g];
    r.first = min(max(first, 0), a.rows);
    r.rows = min(max(next, r.first), a.rows) - r.first;
    r.shared = min(min(max(shared, 0), a.max_shared), a.max_blocks);
  }
  return r;
}
// Rows from .. to of a group, and its shared blocks; no rows: there is no such tile.
struct Tile {
  int row0, rows, shared;
};
__device__ inline int positions_of(const SharedAttnArgs& a, int len) { return min(max(len, -1), a.max_blocks * 16 - 1) + 1; }

// A tile by its number.  Up to 64 groups every wavefront looks for itself, by registers; else they meet in LDS.
__device__ inline Tile find_tile(const SharedAttnArgs& a, int tile, int* s_wave, int* s_tile) {
  const int lane = threadIdx.x & 63;
  if (a.n_groups <= 64) {
    const Group g = group_of(a, lane);
    const int tiles = (g.rows + a.rows_per_tile - 1) / a.rows_per_tile, upto = wave_sums(tiles);
    const unsigned long long here = __ballot(tile >= upto - tiles && tile < upto);
    if (!here) return Tile{0, 0, 0};
    const int at = __builtin_ctzll(here), r0 = (tile - (upto - tiles)) * a.rows_per_tile;
    return Tile{__builtin_amdgcn_readlane(g.first + r0, at), __builtin_amdgcn_readlane(min(a.rows_per_tile, g.rows - r0), at), __builtin_amdgcn_readlane(g.shared, at)};
  }
  if (threadIdx.x == 0) s_tile[1] = 0;
  int sum = 0;
  for (int g0 = 0; g0 < a.n_groups; g0 += kThreads) {
    const Group g = group_of(a, g0 + threadIdx.x);
    const int tiles = (g.rows + a.rows_per_tile - 1) / a.rows_per_tile;
    int all;
    const int before = sum + block_sums(tiles, s_wave, all);
    sum += all;
    if (tile >= before && tile < before + tiles) {
      const int r0 = (tile - before) * a.rows_per_tile;
      s_tile[0] = g.first + r0;
      s_tile[1] = min(a.rows_per_tile, g.rows - r0);
      s_tile[2] = g.shared;
    }
  }
  __syncthreads();
  return Tile{__builtin_amdgcn_readfirstlane(s_tile[0]), __builtin_amdgcn_readfirstlane(s_tile[1]), __builtin_amdgcn_readfirstlane(s_tile[2])};
}

// All tiles of a call, and how many workgroups each gets: about as many as its share of the steps, in every workgroup's LDS.
struct Deal {
  int group_first[kDealGroups], group_tile[kDealGroups], group_rows[kDealGroups], group_shared[kDealGroups];   // of each group: first row, tiles before it, ..
  int steps[kDealTiles], with[kDealTiles], first[kDealTiles], parts[kDealTiles];   // of each tile: steps, whether rows attend the shared blocks together, workgroups before it, its own
};
__device__ inline Tile dealt_tile(const SharedAttnArgs& a, const Deal& d, int tile) {
  const int g = last_within(d.group_tile, a.n_groups, tile), r0 = (tile - d.group_tile[g]) * a.rows_per_tile;
  return Tile{d.group_first[g] + r0, min(a.rows_per_tile, d.group_rows[g] - r0), d.group_shared[g]};
}
// Tiles; `all`: workgroups that have something to do.
__device__ inline int deal_tiles(const SharedAttnArgs& a, Deal& d, int* s_wave, int& all) {
  const int t = threadIdx.x;
  const Group g = group_of(a, t);
  constexpr int EACH = kDealRows / kThreads;
  int lens[EACH];
#pragma unroll
  for (int i = 0; i < EACH; ++i) lens[i] = t + i * kThreads < a.rows ? a.context_lens[t + i * kThreads] : 0;
  for (int i = t; i < a.tiles; i += kThreads) d.steps[i] = d.with[i] = 0;
  int tiles;
  const int before = block_sums((g.rows + a.rows_per_tile - 1) / a.rows_per_tile, s_wave, tiles);
  if (t < a.n_groups) {
    d.group_first[t] = g.first;
    d.group_tile[t] = before;
    d.group_rows[t] = g.rows;
    d.group_shared[t] = g.shared;
  }
  tiles = min(tiles, a.tiles);
  __syncthreads();
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    const int m = t + i * kThreads;
    if (m >= a.rows) break;
    const int of = last_within(d.group_first, a.n_groups, m), r = m - d.group_first[of], tile = d.group_tile[of] + r / a.rows_per_tile;
    if (r < 0 || r >= d.group_rows[of] || tile >= tiles) continue;   // a row of no group
    const int npos = positions_of(a, lens[i]), shared = d.group_shared[of] * 16;
    const bool with = shared > 0 && npos >= shared;
    atomicAdd(&d.steps[tile], (npos - (with ? shared : 0) + 31) >> 5);
    if (with) d.with[tile] = 1;
  }
  __syncthreads();
  static_assert(kDealTiles <= kThreads && kDealGroups <= kThreads, "a thread a tile");
  int steps = 0, sum;
  if (t < tiles) steps = d.steps[t] + (d.with[t] ? (dealt_tile(a, d, t).shared * 16 + 31) >> 5 : 0);
  block_sums(steps, s_wave, sum);
  const int most = max(1, steps / kWaves);   // (a step a wavefront at least)
  const int parts = t < tiles ? min(most, max(1, (int)((int64_t)a.dealt * steps / max(sum, 1)))) : 0;
  const int first = block_sums(parts, s_wave, all);
  if (t < tiles) {
    d.first[t] = first;
    d.parts[t] = parts;
  }
  __syncthreads();
  return tiles;
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
  // Of every run (the shared blocks, then the rows' own positions), each wavefront for itself: steps before it, its positions from .. to, the block table that it walks.
  __shared__ int4 s_runs[kWaves][kMostRows + 2];
  __shared__ float s_m[kWaves][16], s_l[kWaves][16];
  __shared__ int s_wave[kWaves], s_tile[3];
  __shared__ Deal s_deal;

  const int kvh = blockIdx.x % a.kv_heads, hc = blockIdx.x / a.kv_heads, wg = blockIdx.y;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l16 = lane & 15, j = lane >> 4;
  int4* runs = s_runs[wave];
  // What this workgroup does: tile number wg, or part `part` of `parts` of a tile.
  const int early_len = a.rows <= 64 ? a.context_lens[min(lane, a.rows - 1)] : 0;   // (asked for together with the groups)
  int tile = wg, part = 0, parts = 1;
  Tile here;
  if (a.dealt) {
    int all;
    const int n_tiles = deal_tiles(a, s_deal, s_wave, all);
    if (wg == 0 && blockIdx.x == 0 && threadIdx.x < a.tiles) {
      const int t = threadIdx.x;
      const Tile x = t < n_tiles ? dealt_tile(a, s_deal, t) : Tile{0, 0, 0};
      a.tile_of[t] = t < n_tiles ? make_int4(x.row0, x.rows, s_deal.first[t], s_deal.parts[t]) : make_int4(0, 0, 0, 0);
    }
    if (wg >= all) return;
    tile = __builtin_amdgcn_readfirstlane(last_within(s_deal.first, n_tiles, wg));
    part = wg - __builtin_amdgcn_readfirstlane(s_deal.first[tile]);
    parts = __builtin_amdgcn_readfirstlane(s_deal.parts[tile]);
    const Tile x = dealt_tile(a, s_deal, tile);
    here = Tile{__builtin_amdgcn_readfirstlane(x.row0), __builtin_amdgcn_readfirstlane(x.rows), __builtin_amdgcn_readfirstlane(x.shared)};
  } else {
    here = find_tile(a, tile, s_wave, s_tile);
    if (here.rows == 0) return;
  }

  const size_t block_elems = (size_t)a.kv_heads * 16 * DH;
  const T* kpool = reinterpret_cast<const T*>(a.k) + (size_t)kvh * 16 * DH;
  const T* vpool = reinterpret_cast<const T*>(a.v) + (size_t)kvh * 16 * DH;
  // lane offsets within a block
  const int k_at = l16 * DH + j * (BF16 ? 8 : 4);     // position l16, channels + c * 32 (16)
  const int v_at = j * 4 * DH + l16 * CT;             // positions 4j + i, channels l16 * CT ..

  int total;
  const int row0 = here.row0, n_rows = here.rows;
  {   // the runs: lane r has row r
    const int m = row0 + min(lane, n_rows - 1);
    const int seq = a.row_table ? safe_row(a.row_table[m], a.rows) : m;
    const int len = a.rows <= 64 ? __shfl(early_len, m) : a.context_lens[m];
    const int shared = here.shared * 16, npos = positions_of(a, len);
    const bool with = lane < n_rows && shared > 0 && npos >= shared;
    const unsigned long long who = __ballot(with);
    const int prefix_steps = who ? (shared + 31) >> 5 : 0;
    const int from = with ? shared : 0, steps = lane < n_rows ? (npos - from + 31) >> 5 : 0;
    const int upto = wave_sums(steps);
    total = prefix_steps + __builtin_amdgcn_readlane(upto, 63);
    if (lane < n_rows) runs[lane + 1] = make_int4(prefix_steps + upto - steps, from, npos, seq);
    if (lane == (who ? __builtin_ctzll(who) : 0)) runs[0] = make_int4(0, 0, shared, seq);
    if (lane == 0) runs[n_rows + 1] = make_int4(total, 0, 0, 0);
  }
  const int per = (total + parts - 1) / parts, lo = min(part * per, total), hi = min(total, lo + per);
  const bool alone = parts == 1;   // the tile's result is this workgroup's
  const int nk = hi - lo > wave ? (hi - lo - wave + kWaves - 1) / kWaves : 0;   // steps of this wavefront: lo + wave + k * kWaves

  // The blocks of the wavefront's next 32 steps, two lanes a step (a step's second block may not be there: the first again, masked).
  int off_lo = 0, off_hi = 0;
  auto load_ids = [&](int k0) {
    const int s = min(lo + wave + (k0 + (lane >> 1)) * kWaves, hi - 1);
    int r = 0, z = n_rows;           // the last run that begins at or before s (runs without steps lie in front of the next)
    while (r < z) {
      const int mid = (r + z + 1) >> 1;
      if (runs[mid].x <= s) r = mid;
      else z = mid - 1;
    }
    const int4 of = runs[r];
    const int b = min(of.y + (s - of.x) * 32 + (lane & 1) * 16, of.z - 1) >> 4;
    const size_t off = (size_t)safe_block(a.block_tables[(size_t)of.w * a.max_blocks + b], a.num_blocks) * block_elems * sizeof(T);
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
  // This lane's columns are l16 of every tile of 16.  q is asked for before K and V, and split while they are on their way.
  const int gc = min(a.group - hc * a.columns, a.columns);              // query heads of a row in the tile
  const int n_columns = n_rows * gc, heads = a.kv_heads * a.group, head0 = kvh * a.group + hc * a.columns;
  const float scale = 1.4426950408889634f / sqrtf((float)DH);
  constexpr int Q_MINE = NT == 1 ? KS : (NT * KS * 64 + kThreads - 1) / kThreads, Q_VECS = BF16 ? 2 : 1;   // of a thread: contraction steps, or pieces for LDS
  f32x4 q_raw[Q_MINE][Q_VECS];
  auto q_place = [&](int i, int& column, int& c, int& jj) {   // of piece i of this thread
    const int at = threadIdx.x + i * kThreads;
    column = NT == 1 ? l16 : (at >> 6) / KS * 16 + (at & 15);
    c = NT == 1 ? i : (at >> 6) % KS;
    jj = NT == 1 ? j : (at & 63) >> 4;
  };
#pragma unroll
  for (int i = 0; i < Q_MINE; ++i) {
    int column, c, jj;
    q_place(i, column, c, jj);
    const bool ok = column < n_columns;
    const int r = ok ? column / gc : 0, h = ok ? column - r * gc : 0;
    const float* qp = a.q + ((size_t)(row0 + r) * heads + head0 + h) * DH + (BF16 ? c * 32 + jj * 8 : c * 16 + jj * 4);
#pragma unroll
    for (int u = 0; u < Q_VECS; ++u) q_raw[i][u] = *reinterpret_cast<const f32x4*>(qp + u * 4) * (ok ? scale : 0.0f);
  }
  if (nk > 0) {
    load_ids(0);
    load_k(0);
    load_v(0);
  }
  auto q_parts = [&](int i, u32x4 (&piece)[QP]) {
    if constexpr (BF16) {
      const f32x4 x = q_raw[i][0], y = q_raw[i][Q_VECS - 1];
      const float v[8] = {x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
      split3(v, piece);
    } else {
      piece[0] = __builtin_bit_cast(u32x4, q_raw[i][0]);
    }
  };
  u32x4 q1[NT == 1 ? KS : 1][QP];
  u32x4* q_lds = reinterpret_cast<u32x4*>(s_space);
  if constexpr (NT == 1) {
#pragma unroll
    for (int c = 0; c < KS; ++c) q_parts(c, q1[c]);
  } else {
#pragma unroll
    for (int i = 0; i < Q_MINE; ++i) {
      const int at = threadIdx.x + i * kThreads;
      u32x4 piece[QP];
      q_parts(i, piece);
      if (at < NT * KS * 64) {
#pragma unroll
        for (int p = 0; p < QP; ++p) q_lds[((at >> 6) * QP + p) * 64 + (at & 63)] = piece[p];
      }
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
    col_with[t] = ok && runs[(ok ? col_row[t] : 0) + 1].y > 0;
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
    constexpr bool EARLY = NT < 3;   // all scores first, so that the next K comes while the rest of the step is done; three tiles' do not fit beside it
    constexpr bool EARLY_V = BF16 && NT == 3;   // the next V as soon as this one is turned: 87 -> 83 us for the 100000 positions above, but 17.6 -> 18.2 for tiles of 16 columns
    auto next_ids = [&] {   // in front of whichever of the next step's K and V is asked for first (both of this step's have been)
      if (((k + 1) & 31) == 0) load_ids(k + 1);
    };
    auto next_k = [&] {
      if (k + 1 < nk) {
        if constexpr (!EARLY_V) next_ids();
        load_k(k + 1);
      }
    };
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
      if constexpr (EARLY_V) {   // (the registers of V are free)
        if (k + 1 < nk) {
          next_ids();
          load_v(k + 1);
        }
        __builtin_amdgcn_sched_barrier(0);
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
    if constexpr (!EARLY_V)
      if (k + 1 < nk) load_v(k + 1);
  };
  const int plain_steps = all_with ? __builtin_amdgcn_readfirstlane(runs[0].z) >> 5 : 0;
  int k = 0;
  for (; k < nk && lo + wave + k * kWaves < plain_steps; ++k) step(std::true_type{}, k, 0, 0, 0);
  for (int run = 0; k < nk; ++k) {
    const int at = lo + wave + k * kWaves;
    while (at >= __builtin_amdgcn_readfirstlane(runs[run + 1].x)) ++run;
    const int4 of = runs[run];
    const int tok0 = __builtin_amdgcn_readfirstlane(of.y + (at - of.x) * 32);
    step(std::false_type{}, k, run, tok0, __builtin_amdgcn_readfirstlane(of.z));
  }

  // the four lanes of a column have sums over positions of their own; then the wavefronts, in order, 16 columns at a time (one that had no step has sums of 0)
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
      float m[kWaves], M = kNegBig, L = 0.0f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        m[w] = s_m[w][c];
        M = fmaxf(M, m[w]);
      }
      f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float wgt = __builtin_amdgcn_exp2f(m[w] - M);
        L += s_l[w][c] * wgt;
        acc += *reinterpret_cast<const f32x4*>(&s_o[w][c][ch]) * wgt;
      }
      if (alone) {
        const float inv = runs[r + 1].z > 0 ? 1.0f / L : 0.0f;      // a row without a position: 0
        *reinterpret_cast<f32x4*>(a.out + ((size_t)(row0 + r) * heads + head0 + column - r * gc) * DH + ch) = acc * inv;
      } else {
        float* rec = a.records + (((size_t)hc * a.kv_heads + kvh) * (a.dealt + a.tiles) + wg) * a.columns * PITCH + (size_t)column * PITCH;
        if (ch == 0) *reinterpret_cast<f32x4*>(rec) = f32x4{M, L, 0.0f, 0.0f};
        *reinterpret_cast<f32x4*>(rec + 4 + ch) = acc;
      }
    }
  }
}

// Adds the parts of the tiles that several workgroups had: a workgroup a column, DH / 4 threads to every eighth (sixteenth) part; then these, in order.
template <int DH>
__global__ __launch_bounds__(256) void shared_join_kernel(SharedAttnArgs a) {
  constexpr int TH = DH / 4, G = 256 / TH, PITCH = DH + 4;
  __shared__ __align__(16) float s_acc[G][DH];
  __shared__ float s_m[G], s_l[G];
  const int kvh = blockIdx.x % a.kv_heads, hc = blockIdx.x / a.kv_heads, tile = blockIdx.y, c = blockIdx.z;
  const int4 td = a.tile_of[tile];
  const int gc = min(a.group - hc * a.columns, a.columns);
  const int parts = td.w;
  if (parts < 2 || c >= td.y * gc) return;
  const int g = threadIdx.x / TH, ch = threadIdx.x % TH * 4, r = c / gc;
  const float* rec = a.records + (((size_t)hc * a.kv_heads + kvh) * (a.dealt + a.tiles) + td.z) * a.columns * PITCH + (size_t)c * PITCH;
  const size_t pitch = (size_t)a.columns * PITCH;
  float M = kNegBig, L = 0.0f;
  f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int p = g; p < parts; p += G) {
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
  shared_attn_kernel<T, DH, NT><<<dim3(a.kv_heads * a.head_chunks, a.dealt ? a.dealt + a.tiles : a.tiles), kThreads, 0, st>>>(a);
  if (a.dealt) shared_join_kernel<DH><<<dim3(a.kv_heads * a.head_chunks, a.tiles, a.columns), 256, 0, st>>>(a);
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
  // Whole tiles a workgroup, or all tiles' steps dealt out evenly: where there are fewer tiles than run at once and they are long, and where they are few enough
  // for a long one to be waited for.  (Lengths are the device's: these are bounds.)
  const int64_t heads = (int64_t)a.kv_heads * a.head_chunks, wgs = a.tiles * heads;
  const int64_t shared = a.max_shared < a.max_context / 16 ? a.max_shared : a.max_context / 16, own = a.max_context - shared * 16;
  const int64_t steps = (shared * 16 + 31) / 32 + (int64_t)(a.rows < a.rows_per_tile ? a.rows : a.rows_per_tile) * ((own + 31) / 32);
  const bool deal = wgs < kMostWgs ? steps * (dtype == EE_FP32 && a.dh == 128 ? 2 : 1) >= kWorthDealing : wgs < 8 * kMostWgs && wgs * steps >= 8 * kWaves * kMostWgs;
  const bool can = a.rows <= kDealRows && a.n_groups <= kDealGroups && a.tiles <= kDealTiles;
  a.dealt = deal && can ? (heads < kMostWgs ? (int)(kMostWgs / heads) : 1) : 0;
  // Few tiles, each of more steps than wavefronts: fewer rows in each, whose own positions then go side by side (the shared ones are read more often, from cache).  35 float
  // rows in 7 groups, 12 heads over 4: 15.5 -> 11 us.
  for (int64_t n = steps; !a.dealt && a.head_chunks == 1 && a.rows_per_tile > 1 && n > kWaves && 2 * a.tiles * heads <= kMostWgs;) {
    const int rows = (a.rows_per_tile + 1) / 2;
    n -= (a.rows_per_tile - rows) * ((own + 31) / 32);
    a.rows_per_tile = rows;
    a.columns = (rows * a.group + 15) / 16 * 16;
    a.tiles = most_tiles(a);
  }
}

size_t shared_attn_record_floats(const SharedAttnArgs& a) {
  return a.dealt ? (size_t)a.kv_heads * a.head_chunks * (a.dealt + a.tiles) * a.columns * (a.dh + 4) : 0;
}

// For calls of fewer rows, groups and positions, which may have narrower tiles: of each width the tiles grow with rows and groups.
size_t shared_attn_most_floats(SharedAttnArgs& a, int dtype, size_t* tiles) {
  size_t most = 0;
  const int widest = dtype == EE_FP32 ? 32 : kMostColumns;
  *tiles = 0;
  for (int columns = 16; columns <= widest; columns += 16) {
    tile_widths(a, columns, widest);
    const int64_t heads = (int64_t)a.kv_heads * a.head_chunks;
    int64_t t = most_tiles(a);
    if (t > kDealTiles) t = kDealTiles;
    if (t * heads > 8 * kMostWgs) t = (8 * kMostWgs + heads - 1) / heads;
    const size_t floats = (size_t)(kMostWgs + heads + t * heads) * a.columns * (a.dh + 4);
    if (*tiles < (size_t)t) *tiles = t;
    if (most < floats) most = floats;
  }
  shared_attn_plan(a, dtype);
  return most;
}

void launch_shared_attention(const SharedAttnArgs& a, int dtype, hipStream_t st) {
  if (dtype == EE_BF16) a.dh == 64 ? launch<bf16_t, 64>(a, st) : launch<bf16_t, 128>(a, st);
  else a.dh == 64 ? launch<float, 64>(a, st) : launch<float, 128>(a, st);
}

}  // namespace ee
