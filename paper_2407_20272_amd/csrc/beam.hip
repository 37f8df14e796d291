// One step of beam search: the best continuations of every group over its beams and the whole vocabulary, and rows of states in their new order.
//
//   score(b, t) = scores[b] + (z[b][t] - log sum_t' exp z[b][t'])
//
// Two launches.  The scan reads the logits once: a workgroup takes a chunk of a row, keeps its values in registers, and leaves the chunk's maximum, its
// sum of exponentials and its n best, in order (within a beam the order of the scores is that of the logits, so this needs no sum of the whole row).
// The join forms the rows' sums from the chunks', the scores of what was found, and the n best of these.
// What is compared are scores in double: rounded to float many candidates of a beam would be equal, and beams' sums meet there.  (Where even these are equal, within a beam by logits: it is these that its lists are of.)  Exponentials are floats, a thread's sixteen or 32 are added
// in float and everything behind that in double.
//
// Scan + join, kernel times: 4 rows of 2048 floats 4.5 + 3.7 us; 128 rows of 32000 bf16, 8 of 4 back: 7.1 + 7.1; 128 rows of 100003 floats (51 MB, 41 of them read: a fifth is finished), 16 of 8 back: 13.7 + 8.5;
// 64 rows of 32000 floats, 128 of 64 back: 9.4 + 11.4.  The scan of many rows is bound by memory and by the latency of one chunk (values, maximum, sum, bound, list: 6 us), the join by the latency of its
// dozen barriers.  Values in chunks of 4096 where all workgroups run at once, else of 8192: the 128 rows of 100003 took 19 us in 4096, more than one round, also with the next chunk's
// values on their way.
#include <type_traits>

#include "beams.h"

namespace ee {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Floats in the order of unsigned integers; 0 is below all of them (what is NaN or -inf is no candidate).
__device__ inline uint32_t key_of(float z) {
  if (!(z > -INFINITY)) return 0;
  const uint32_t u = __float_as_uint(z + 0.0f);   // (-0 is 0)
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
constexpr uint32_t kLowestKey = 0x00800000u;   // of the lowest float
__device__ inline float float_of(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key); }
__device__ inline uint64_t key_of(double s) {
  const uint64_t u = (uint64_t)__double_as_longlong(s + 0.0);
  return u >> 63 ? ~u : u | 1ull << 63;
}
__device__ inline double double_of(uint64_t key) { return __longlong_as_double((long long)(key >> 63 ? key & ~(1ull << 63) : ~key)); }

// The largest bound of which at least n of the keys are not below (each lane has K of them; the wavefront's together), to its upper 2 * PAIRS bits; at least 1.
// (Two bits at a time: what a step takes is its chain of scalar instructions, and three counts go through it side by side.)
template <int K, int PAIRS>
__device__ inline uint32_t wave_bound(const uint32_t (&key)[K], int n) {
  uint32_t bound = 0;
  for (int bit = 30; bit >= 32 - 2 * PAIRS; bit -= 2) {
    int count[3] = {0, 0, 0};
#pragma unroll
    for (int i = 0; i < K; ++i)
#pragma unroll
      for (int q = 0; q < 3; ++q) count[q] += __popcll(__ballot(key[i] >= (bound | (uint32_t)(q + 1) << bit)));
    bound |= (uint32_t)((count[0] >= n) + (count[1] >= n) + (count[2] >= n)) << bit;
  }
  return bound ? bound : 1u;
}

// The largest of a wavefront's values, and the sums of its numbers (in a fixed order), on the cross-lane network: every lane has them.
__device__ inline uint32_t wave_largest(uint32_t v) {
  auto with = [&](auto ctrl, auto rows) { v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, decltype(ctrl)::value, decltype(rows)::value, 0xf, false)); };
  with(std::integral_constant<int, 0x111>{}, std::integral_constant<int, 0xf>{});   // row_shr 1, 2, 4, 8
  with(std::integral_constant<int, 0x112>{}, std::integral_constant<int, 0xf>{});
  with(std::integral_constant<int, 0x114>{}, std::integral_constant<int, 0xf>{});
  with(std::integral_constant<int, 0x118>{}, std::integral_constant<int, 0xf>{});
  with(std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xa>{});   // row_bcast 15, 31
  with(std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xc>{});
  return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}
__device__ inline int wave_upto(int v) {   // over the lanes up to each
  auto add = [&](auto ctrl, auto rows) { v += __builtin_amdgcn_update_dpp(0, v, decltype(ctrl)::value, decltype(rows)::value, 0xf, false); };
  add(std::integral_constant<int, 0x111>{}, std::integral_constant<int, 0xf>{});
  add(std::integral_constant<int, 0x112>{}, std::integral_constant<int, 0xf>{});
  add(std::integral_constant<int, 0x114>{}, std::integral_constant<int, 0xf>{});
  add(std::integral_constant<int, 0x118>{}, std::integral_constant<int, 0xf>{});
  add(std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xa>{});
  add(std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xc>{});
  return v;
}
__device__ inline int wave_total(int v) { return __builtin_amdgcn_readlane(wave_upto(v), 63); }
// The sum over eight neighbouring lanes: all of them have it.
__device__ inline int sum_of_8(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0xB1, 0xf, 0xf, true);    // quad_perm [1,0,3,2], [2,3,0,1], row_half_mirror
  v += __builtin_amdgcn_update_dpp(0, v, 0x4E, 0xf, 0xf, true);
  return v + __builtin_amdgcn_update_dpp(0, v, 0x141, 0xf, 0xf, true);
}
__device__ inline double wave_sum(double v) {
  auto add = [&](auto ctrl, auto rows) {
    const uint64_t u = (uint64_t)__double_as_longlong(v);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)u, decltype(ctrl)::value, decltype(rows)::value, 0xf, false);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(u >> 32), decltype(ctrl)::value, decltype(rows)::value, 0xf, false);
    v += __longlong_as_double((long long)((uint64_t)hi << 32 | lo));
  };
  add(std::integral_constant<int, 0x111>{}, std::integral_constant<int, 0xf>{});
  add(std::integral_constant<int, 0x112>{}, std::integral_constant<int, 0xf>{});
  add(std::integral_constant<int, 0x114>{}, std::integral_constant<int, 0xf>{});
  add(std::integral_constant<int, 0x118>{}, std::integral_constant<int, 0xf>{});
  add(std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xa>{});
  add(std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xc>{});
  const uint64_t u = (uint64_t)__double_as_longlong(v);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)u, 63), hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(u >> 32), 63);
  return __longlong_as_double((long long)((uint64_t)hi << 32 | lo));
}

constexpr int kScanList = 512;   // candidates of a chunk that are put in order

// A chunk of THREADS * EACH values.  What falls behind the n-th largest of 256 parts' maxima is none of the n best; the others (n and a few) are
// gathered and put in order by counting, for each, those in front of it.  Where they are too many (many equal values), the n-th of all is found bit by bit first.
template <class T, int THREADS, int EACH>
__global__ __launch_bounds__(THREADS, EACH > 16 ? 6 : 4) void beam_scan_kernel(BeamArgs a) {
  constexpr int VEC = 16 / sizeof(T), LOADS = EACH / VEC, WAVES = THREADS / 64;
  __shared__ __align__(16) uint64_t s_list[kScanList];
  __shared__ uint32_t s_most[256];
  __shared__ double s_sum[WAVES];
  __shared__ uint32_t s_top[WAVES];
  __shared__ uint32_t s_bound;
  __shared__ int s_count, s_below[WAVES];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int chunk = blockIdx.x, row = blockIdx.y, base = chunk * THREADS * EACH, n = a.n_out, lists = a.beams * a.chunks;
  if (a.finished && a.finished[row]) return;   // (before any value is asked for: the row's logits may be nowhere)
  const char* z = reinterpret_cast<const char*>(a.logits) + (size_t)row * a.stride * sizeof(T);
  // Values `at(l) + e` for part l; the same places whether the row starts on 16 bytes or not, so that equal rows have equal sums.
  auto at = [&](int l) { return base + (l * THREADS + (int)threadIdx.x) * VEC; };
  float x[EACH];
  constexpr uint32_t NONE = sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;   // -inf
  if ((reinterpret_cast<uintptr_t>(z) & 15) == 0 && (base + THREADS * EACH <= a.vocab || a.vocab % VEC == 0)) {
    u32x4 raw[LOADS];
#pragma unroll
    for (int l = 0; l < LOADS; ++l) {
      raw[l] = u32x4{NONE, NONE, NONE, NONE};
      if (at(l) < a.vocab) raw[l] = *reinterpret_cast<const u32x4*>(z + (uint32_t)at(l) * (uint32_t)sizeof(T));
    }
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      if constexpr (sizeof(T) == 4) x[i] = __uint_as_float(raw[i / 4][i % 4]);
      else x[i] = __uint_as_float(i & 1 ? raw[i / 8][i % 8 / 2] & 0xffff0000u : raw[i / 8][i % 8 / 2] << 16);
    }
  } else {
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      const int t = at(i / VEC) + i % VEC;
      x[i] = t < a.vocab ? (float)*reinterpret_cast<const T*>(z + (uint32_t)t * (uint32_t)sizeof(T)) : -INFINITY;
    }
  }

  float most = -INFINITY;
#pragma unroll
  for (int i = 0; i < EACH; ++i) most = fmaxf(most, x[i]);
  const uint32_t most_key = key_of(most);
  if constexpr (THREADS == 256) {
    s_most[threadIdx.x] = most_key;
  } else {   // four threads' together: quad_perm [1,0,3,2], [2,3,0,1]
    uint32_t four = max(most_key, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)most_key, 0xB1, 0xf, 0xf, true));
    four = max(four, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)four, 0x4E, 0xf, 0xf, true));
    if ((threadIdx.x & 3) == 0) s_most[threadIdx.x / 4] = four;
  }
  uint32_t top_key = wave_largest(most_key);
  if (lane == 0) s_top[wave] = top_key;
  if (threadIdx.x == 0) s_count = 0;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < WAVES; ++i) top_key = max(top_key, s_top[i]);
  const float top = top_key ? float_of(top_key) : -INFINITY;
  // (a chunk without a value has a sum of 0, one with a NaN or +inf a sum that is NaN: so has its row)
  const float ref = top == -INFINITY ? 0.0f : top;
  float part = 0.0f;
#pragma unroll
  for (int i = 0; i < EACH; ++i) part += __expf(x[i] - ref);
  const double sum = wave_sum(part);
  if (lane == 0) s_sum[wave] = sum;

  // the n-th largest of the 256 maxima: below it is none of the n best
  if (wave == 0) {
    uint32_t key[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) key[i] = s_most[i * 64 + lane];
    const uint32_t bound = wave_bound<4, 9>(key, n);
    if (lane == 0) s_bound = bound;
  }
  __syncthreads();
  const float bound = s_bound < kLowestKey ? -3.4028235e38f : float_of(s_bound);
  auto composite = [&](int i) { return (uint64_t)key_of(x[i]) << 32 | (0xffffffffu - (uint32_t)(at(i / VEC) + i % VEC)); };
  auto take = [&](int i) {
    const int k = atomicAdd(&s_count, 1);
    if (k < kScanList) s_list[k] = composite(i);
  };
#pragma unroll
  for (int i = 0; i < EACH; ++i)
    if (x[i] >= bound) take(i);
  __syncthreads();
  int count = s_count;
  if (count > kScanList) {
    uint64_t from = 0;
    for (int bit = 63; bit >= 0; --bit) {
      const uint64_t c = from | 1ull << bit;
      int mine = 0;
#pragma unroll
      for (int i = 0; i < EACH; ++i) mine += composite(i) >= c;
      mine = wave_total(mine);
      __syncthreads();
      if (lane == 0) s_below[wave] = mine;
      __syncthreads();
      int all = 0;
#pragma unroll
      for (int i = 0; i < WAVES; ++i) all += s_below[i];
      if (all >= n) from = c;
    }
    if (threadIdx.x == 0) s_count = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < EACH; ++i)
      if (composite(i) >= from) take(i);   // (composites differ: n of them)
    __syncthreads();
    count = min(s_count, kScanList);
  }
  if (threadIdx.x == 0) {
    double total = 0.0;
    for (int i = 0; i < WAVES; ++i) total += s_sum[i];
    a.stats[(size_t)row * a.chunks + chunk] = make_double2(top, total);
  }
  // place k of this list among the group's: [k][beam][chunk]
  uint64_t* found = a.found + (size_t)(row / a.beams) * n * lists + (size_t)(row % a.beams) * a.chunks + chunk;
  for (int i0 = 0; i0 < count; i0 += THREADS / 8) {   // eight threads a candidate, each against every eighth
    const int i = i0 + (int)threadIdx.x / 8;
    const uint64_t c = i < count ? s_list[i] : 0;
    int rank = 0;
#pragma unroll 4
    for (int j = threadIdx.x & 7; j < count; j += 8) rank += s_list[j] > c;
    rank = sum_of_8(rank);
    if (i < count && rank < n && (threadIdx.x & 7) == 0) found[(size_t)rank * lists] = c;
  }
  for (int i = count + (int)threadIdx.x; i < n; i += THREADS) found[(size_t)i * lists] = 0;
}

constexpr int kJoinThreads = 1024;
constexpr int kJoinList = 1024;
constexpr int kJoinKept = 4096;   // candidates that are looked at first
constexpr int kJoinDeep = 12288;  // and behind these, of the lists that may have more; rough scores of both stay in LDS
constexpr int kJoinFew = 128;    // so many are put in order without a look at which may count

// A workgroup a group.  The n best of its beams' chunks' are found as in the scan, by the n-th largest of 256 maxima; where this lets many more through than n, the bound is moved up by counts
// of 256 parts until few are left.  The lists' first places are looked at, and more of a list only where its last of these is not below the bound (64 rows, 128 back: 16384 candidates looked at 19.5 us,
// 4096 and some 11; both launches, one beam with all the best of 128 over 128256 tokens: 169 and 40; 64 beams of 32000 tokens, all but one at -1e9: 36).  Then by counting what is in front.
__global__ __launch_bounds__(kJoinThreads) void beam_join_kernel(BeamArgs a, int is_bf16) {
  constexpr int WAVES = kJoinThreads / 64;
  struct Candidate {
    uint64_t key, index;   // of the score in double, 0: none; among equal scores the beam of the group (8 bits), what its logit is below the highest (32), the token (24)
  };
  __shared__ double s_off[kBeamMost], s_base[kBeamMost];   // of a beam: the logarithm of its sum; its score
  __shared__ int s_done[kBeamMost];
  __shared__ float s_rough_off[kBeamMost], s_best[kBeamMost];   // half of what is added to its logits (the whole may be twice the largest float), and its best score, as floats
  __shared__ uint32_t s_most[kJoinThreads / 4];
  __shared__ uint64_t s_key[kJoinList], s_index[kJoinList];
  __shared__ uint32_t s_rough[kJoinKept + kJoinDeep];
  __shared__ uint64_t s_found[kJoinKept];
  __shared__ uint32_t s_bound;
  __shared__ uint16_t s_deep[kJoinKept];
  __shared__ int s_count, s_n_deep, s_below[WAVES], s_digits[16];
  __shared__ __align__(16) int s_bins[2][256];
  __shared__ unsigned long long s_span[2];
  const int g = blockIdx.x, n = a.n_out, W = a.beams, row0 = g * W;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int lists = W * a.chunks, all = lists * n;
  const uint64_t* found = a.found + (size_t)g * all;   // the lists' first ones, then the second ones, ..
  if (threadIdx.x == 0) s_count = s_n_deep = 0;
  const int places = min(n, kJoinKept / lists), kept = places ? places * lists : kJoinKept;   // (without whole places the first ones give a bound, and are looked at again)
  uint64_t first[kJoinKept / kJoinThreads];   // (on their way while the sums are formed)
#pragma unroll
  for (int u = 0; u < kJoinKept / kJoinThreads; ++u) first[u] = (int)threadIdx.x + u * kJoinThreads < kept ? found[threadIdx.x + u * kJoinThreads] : 0;
  // The rows' sums: 2^p lanes a row, as many as it has chunks (in a fixed order of additions).
  {
    int p = 0;
    while (p < 6 && 1 << p < a.chunks) ++p;
    const int c0 = lane & ((1 << p) - 1);
    for (int b0 = wave << (6 - p); b0 < W; b0 += WAVES << (6 - p)) {
      const int b = b0 + (lane >> p), row = row0 + min(b, W - 1);
      const int done = a.finished ? a.finished[row] : 0;
      const float base = a.scores[row];
      const double2* stats = a.stats + (size_t)row * a.chunks;
      double2 own = stats[min(c0, a.chunks - 1)];
      if (c0 >= a.chunks || done) own = make_double2(-INFINITY, 0.0);
      float m = (float)own.x;   // (maxima are floats)
      if (!done)
        for (int k = c0 + 64; k < a.chunks; k += 64) m = fmaxf(m, (float)stats[k].x);
      for (int o = 1; o < 1 << p; o <<= 1) m = fmaxf(m, __shfl_xor(m, o));
      double sum = own.y != 0.0 ? own.y * exp(own.x - m) : 0.0;   // (NaN stays)
      if (!done)
        for (int k = c0 + 64; k < a.chunks; k += 64) {
          const double2 s = stats[k];
          if (s.y != 0.0) sum += s.y * exp(s.x - m);
        }
      for (int o = 1; o < 1 << p; o <<= 1) sum += __shfl_xor(sum, o);
      if (c0 == 0 && b < W) {
        const double off = done ? 0.0 : m + log(sum), to = base - off;
        s_off[b] = off;
        s_base[b] = base;
        s_done[b] = done != 0;
        // what is not finite stands for rows that have no candidates; a score that no float is for the lowest
        s_rough_off[b] = to - to == 0.0 ? (float)(0.5 * to) : NAN;
        s_best[b] = done ? (to - to == 0.0 ? base : NAN) : fminf(fmaxf((float)(to + m), -3.4028235e38f), 3.4028235e38f);
      }
    }
  }
  __syncthreads();
  float far = 0.0f;   // the largest magnitude of half of what is added to logits
  {
    uint32_t most_far = 0;
    for (int b = lane; b < W; b += 64) most_far = max(most_far, __float_as_uint(fmaxf(fabsf(s_rough_off[b]), 0.0f)));   // (a NaN is 0)
    far = __uint_as_float(wave_largest(most_far));
  }
  // A thread's candidates are 1024 apart: the list goes round, the beam is a quotient by a product of 32 bits (exact: lists * chunks is below 2^32).
  const uint32_t by_chunks = a.chunks > 1 ? 0xffffffffu / (uint32_t)a.chunks + 1 : 0;
  auto beam_of = [&](int list) { return a.chunks > 1 ? (int)__umulhi((uint32_t)list, by_chunks) : list; };
  const int list0 = (int)threadIdx.x % lists, turn_by = kJoinThreads % lists;
  auto next_list = [&](int list) {
    list += turn_by;
    return list >= lists ? list - lists : list;
  };
  auto candidate = [&](int list, uint64_t cc, bool first) {   // of this list, the first one or not; its logit and token are cc
    const int b = beam_of(list);
    double s;
    Candidate r;
    if (s_done[b]) {
      s = first && list == b * a.chunks ? s_base[b] : -INFINITY;
      r.index = (uint64_t)b << 56 | (uint32_t)a.end_token;
    } else {
      s = cc >> 32 ? s_base[b] + ((double)float_of((uint32_t)(cc >> 32)) - s_off[b]) : -INFINITY;
      r.index = (uint64_t)b << 56 | (~cc >> 32) << 24 | (0xffffffffu - (uint32_t)cc);
    }
    r.key = s - s == 0.0 ? key_of(s) : 0;   // what is not finite is none
    return r;
  };
  // The order of a float near the score, for the first look: the row's part is rounded, and the sum (to less than 2^-22 of the row's part and the score together).  0 for none.
  auto rough = [&](int list, uint64_t cc, bool first) {
    const int b = beam_of(list);
    float f;
    if (s_done[b]) f = first && list == b * a.chunks ? s_best[b] : NAN;
    else f = cc >> 32 ? 2.0f * fmaf(0.5f, float_of((uint32_t)(cc >> 32)), s_rough_off[b]) : NAN;
    return f == f ? key_of(fminf(fmaxf(f, -3.4028235e38f), 3.4028235e38f)) : 0u;
  };
  // Of the lists' first places, as many as fit, the scores give a bound for all.  Behind them (the lists fall) are candidates only where a list's last place is not below it.
  uint32_t most = 0;
  int list_of = list0;
#pragma unroll
  for (int u = 0; u < kJoinKept / kJoinThreads; ++u)
    if (const int i = (int)threadIdx.x + u * kJoinThreads; i < kept) {
      const uint32_t k = rough(list_of, first[u], i < lists);
      s_rough[i] = k;
      s_found[i] = first[u];
      most = max(most, k);
      list_of = next_list(list_of);
    }
  uint32_t bound = 1, above = 0;
  // The bound moved up until few of these are at it or above (n at least are, or it stays; fewer than n from `above` on): counted, then 256 parts of what is between bound and `above` at a time.
  auto move_up = [&](int from, int to, uint32_t above) {
    int mine = 0;
#pragma unroll 4
    for (int i = from + (int)threadIdx.x; i < to; i += kJoinThreads) mine += s_rough[i] >= bound;
    mine = wave_total(mine);
    if (lane == 0) s_below[wave] = mine;
    if (threadIdx.x < 512) (&s_bins[0][0])[threadIdx.x] = 0;
    __syncthreads();
    int there = 0;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) there += s_below[i];
    for (int turn = 0; there > max(2 * n, 64) && above - bound > 1; ++turn) {
      const int shift = max(0, 24 - __builtin_clz(above - 1 - bound));
      int* bins = s_bins[turn & 1];
      // (the highest part first, with those that a turn before has left at `above` or over it; those in the lowest are not counted: n are there or above)
#pragma unroll 4
      for (int i = from + (int)threadIdx.x; i < to; i += kJoinThreads) {
        const uint32_t k = s_rough[i];
        if (k > bound && (k - bound) >> shift) atomicAdd(&bins[255 - min((k - bound) >> shift, 255u)], 1);
      }
      __syncthreads();
      const int4 four = *reinterpret_cast<const int4*>(&bins[lane * 4]);
      const int upto = wave_upto(four.x + four.y + four.z + four.w);
      const unsigned long long enough = __ballot(upto >= n);
      uint32_t part = 0;
      if (enough) {
        const int at = __builtin_ctzll(enough);
        int sum = __builtin_amdgcn_readlane(upto - four.x - four.y - four.z - four.w, at), e = 0;
        for (; e < 4; ++e) {
          sum += e == 0 ? __builtin_amdgcn_readlane(four.x, at) : e == 1 ? __builtin_amdgcn_readlane(four.y, at) : e == 2 ? __builtin_amdgcn_readlane(four.z, at) : __builtin_amdgcn_readlane(four.w, at);
          if (sum >= n) break;
        }
        part = 255 - (at * 4 + e);
        there = sum;
      }
      bound += part << shift;
      if (above - bound > 1u << shift) above = bound + (1u << shift);   // (fewer than n are there)
      if (threadIdx.x < 256) s_bins[(turn + 1) & 1][threadIdx.x] = 0;   // (read a turn ago)
      __syncthreads();
    }
  };
  if (all > kJoinFew) {
    // four threads' together: quad_perm [1,0,3,2], [2,3,0,1]
    most = max(most, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)most, 0xB1, 0xf, 0xf, true));
    most = max(most, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)most, 0x4E, 0xf, 0xf, true));
    if ((threadIdx.x & 3) == 0) s_most[threadIdx.x / 4] = most;
    __syncthreads();
    uint32_t key[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) key[i] = s_most[i * 64 + lane];
    if (wave == 0) {
      const uint32_t b = wave_bound<4, 9>(key, n);
      if (lane == 0) s_bound = b;
    }
    above = wave_largest(max(max(key[0], key[1]), max(key[2], key[3]))) + 1;   // nothing is here or above
    __syncthreads();
    bound = s_bound;
    move_up(0, kept, above);
  }
  // Whose score may be at the bound's: rough scores are off by less than 2^-22 of themselves and of what was added to the logits.  Where that is much, it is looked at of which beams: a search begins
  // with scores like -1e9 for all beams but one, and a margin for these would let all of the one's candidates through.
  auto lowered = [&](uint32_t at) -> uint32_t {
    if (at <= 1) return 1;
    const float f = float_of(at);
    auto margin = [&](float off) { return fabsf(f) * 0x1p-20f + off * 0x1p-18f + 0x1p-140f; };   // (the last of these: halves of the smallest floats)
    float least = far > 256.0f ? f : f - margin(far);
    for (int turn = 0; far > 256.0f && turn < 2; ++turn) {   // beams that reach the bound; then those that reach what these leave of it
      uint32_t most_far = 0;
      for (int b = lane; b < W; b += 64) {
        const float off = fabsf(s_rough_off[b]);
        if (s_best[b] + margin(off) >= least) most_far = max(most_far, __float_as_uint(off));
      }
      least = f - margin(__uint_as_float(wave_largest(most_far)));
    }
    return least > -3.4028235e38f ? key_of(least) : 1;
  };
  // Deeper: first the lists whose last place is above the bound, as many of their next places as fit, all lists' one after the other.  Their candidates count for the bound as well; then
  // the lists that it leaves (those whose last place is like the first bound: of beams far below, floats are alike).
  const int per = n - places;   // candidates of a list behind those kept
  int deep = 0, held = 0, late = 0;
  if (per > 0) {
    auto gather = [&](auto&& test) {
      for (int l = threadIdx.x; l < lists; l += kJoinThreads)
        if (test(s_rough[(places - 1) * lists + l])) s_deep[atomicAdd(&s_n_deep, 1)] = (uint16_t)l;
      __syncthreads();
      const int there = s_n_deep;
      __syncthreads();   // (it has been read)
      return there;
    };
    const uint32_t first_bound = bound;
    deep = places ? gather([&](uint32_t k) { return k > first_bound; }) : lists;
    if (deep) {
      held = min(per, kJoinDeep / deep) * deep;
#pragma unroll 4
      for (int q = threadIdx.x; q < held; q += kJoinThreads) {
        const int to = q / deep, d = q - to * deep, l = places ? s_deep[d] : d;
        s_rough[kept + q] = rough(l, found[(size_t)(places + to) * lists + l], places + to == 0);
      }
      __syncthreads();
      move_up(places ? 0 : kept, kept + held, places ? above : ~(kLowestKey - 1));   // (of the highest float, and one)
    }
    bound = lowered(bound);
    if (places) late = gather([&](uint32_t k) { return k <= first_bound && k >= bound; }) - deep;
  } else {
    bound = lowered(bound);
  }
  const int from_kept = places * lists, from_deep = from_kept + deep * per;
  // use(candidate) of all that may count (one loop: its code is what has to be fetched)
  auto each = [&](auto&& use) {
    int list = list0;
#pragma unroll 1
    for (int i = threadIdx.x; i < from_deep + late * per; i += kJoinThreads) {
      uint32_t k = 0;
      uint64_t c = 0;
      int l = list;
      bool its_first = i < lists;
      if (i < from_kept) {
        k = s_rough[i];
        c = s_found[i];
      } else {
        const bool of_deep = i < from_deep;
        const int q = of_deep ? i - from_kept : i - from_deep, many = of_deep ? deep : late, to = q / many, d = q - to * many;
        l = places ? s_deep[of_deep ? d : deep + d] : d;
        its_first = places + to == 0;
        const bool kept_here = of_deep && q < held;
        if (kept_here) k = s_rough[kept + q];
        if (kept_here ? k >= bound : !of_deep || held == 0 || s_rough[kept + held - deep + d] >= bound) c = found[(size_t)(places + to) * lists + l];
        if (!kept_here) k = rough(l, c, its_first);
      }
      if (k >= bound) use(candidate(l, c, its_first));   // (k of none is 0)
      list = next_list(list);
    }
  };
  auto put_by = [&](const Candidate& x) {
    if (!x.key) return;
    const int at = atomicAdd(&s_count, 1);
    if (at < kJoinList) {
      s_key[at] = x.key;
      s_index[at] = x.index;
    }
  };
  each(put_by);
  __syncthreads();
  int count = s_count;
  if (count > kJoinList) {   // so many (nearly) equal scores: the n-th four bits at a time, then of those like it the last that is needed
    int need = n;
    auto nth = [&](auto&& part, bool down) {   // of the part(x, bits) that are asked for, from above or below; what all have in common is seen at once
      if (threadIdx.x == 0) {
        s_span[0] = ~0ull;
        s_span[1] = 0;
      }
      __syncthreads();
      uint64_t lo = ~0ull, hi = 0;
      each([&](const Candidate& x) {
        uint64_t bits;
        if (!x.key || !part(x, bits)) return;
        lo = min(lo, bits);
        hi = max(hi, bits);
      });
      atomicMin(&s_span[0], (unsigned long long)lo);
      atomicMax(&s_span[1], (unsigned long long)hi);
      __syncthreads();
      lo = s_span[0];
      hi = s_span[1];
      int shift = lo == hi ? -4 : (63 - __builtin_clzll(lo ^ hi)) & ~3;
      uint64_t at = lo == hi ? hi : hi & ~(((1ull << shift) << 4) - 1);
      for (; shift >= 0; shift -= 4) {
        if (threadIdx.x < 16) s_digits[threadIdx.x] = 0;
        __syncthreads();
        int mine[16];
#pragma unroll
        for (int d = 0; d < 16; ++d) mine[d] = 0;
        each([&](const Candidate& x) {
          uint64_t bits;
          const bool counts = x.key && part(x, bits) && bits >> shift >> 4 == at >> shift >> 4;
#pragma unroll
          for (int d = 0; d < 16; ++d) mine[d] += counts && (int)(bits >> shift & 15) == d;
        });
#pragma unroll
        for (int d = 0; d < 16; ++d) {
          const int sum = wave_total(mine[d]);
          if (lane == 0 && sum) atomicAdd(&s_digits[d], sum);
        }
        __syncthreads();
        int digit = down ? 15 : 0;
        for (int there; need > (there = s_digits[digit]) && digit != (down ? 0 : 15); digit += down ? -1 : 1) need -= there;
        at |= (uint64_t)digit << shift;
        __syncthreads();   // (they have been read)
      }
      __syncthreads();
      return at;
    };
    const uint64_t from = nth([&](const Candidate& x, uint64_t& bits) { bits = x.key; return true; }, true);
    const uint64_t up_to = nth([&](const Candidate& x, uint64_t& bits) { bits = x.index; return x.key == from; }, false);
    if (threadIdx.x == 0) s_count = 0;
    __syncthreads();
    each([&](const Candidate& x) {
      if (x.key > from || (x.key == from && x.index <= up_to)) put_by(x);
    });
    __syncthreads();
    count = min(s_count, kJoinList);
  }
  auto put = [&](int rank, double s, int b, int t) {
    const size_t at = (size_t)g * n + rank;
    a.scores_out[at] = (float)s;
    a.tokens[at] = t;
    a.parents[at] = row0 + b;
    if (a.finished_out) a.finished_out[at] = s_done[b] || t == a.end_token;
  };
  // in front: a larger score, or an equal one and the lower index (eight threads a candidate, each against every eighth; the indices are looked at only where scores are equal)
  for (int i0 = 0; i0 < count; i0 += kJoinThreads / 8) {
    const int i = i0 + (int)threadIdx.x / 8;
    const uint64_t key = s_key[min(i, count - 1)], index = s_index[min(i, count - 1)];
    int rank = 0, like = 0;
#pragma unroll 4
    for (int k = threadIdx.x & 7; k < count; k += 8) {
      const uint64_t other = s_key[k];
      rank += other > key;
      like += other == key;
    }
    if (__any(sum_of_8(like) > 1))
      for (int k = threadIdx.x & 7; k < count; k += 8) rank += (int)(s_key[k] == key) & (int)(s_index[k] < index);
    rank = sum_of_8(rank);
    if (i < count && rank < n && (threadIdx.x & 7) == 0) put(rank, double_of(key), (int)(index >> 56), (int)(index & 0xffffff));
  }
  if (count >= n) return;
  // Fewer candidates than asked for: the rest are the lowest indices whose score is -inf, found by looking (one wavefront, 64 indices at a time).
  if (wave) return;
  int rank = count;
  for (uint64_t i0 = 0; rank < n && i0 < (uint64_t)W * a.vocab; i0 += 64) {
    const uint64_t index = i0 + lane;
    const int b = (int)(index / a.vocab), t = (int)(index - (uint64_t)b * a.vocab);
    bool none = b < W;
    if (none) {
      if (s_done[b]) {
        none = t != a.end_token || !(s_base[b] - s_base[b] == 0.0);
      } else {
        const size_t at = (size_t)(row0 + b) * a.stride + t;
        const float z = is_bf16 ? (float)reinterpret_cast<const bf16_t*>(a.logits)[at] : reinterpret_cast<const float*>(a.logits)[at];
        const double s = s_base[b] + ((double)z - s_off[b]);
        none = !(s - s == 0.0);
      }
    }
    const uint64_t bal = __ballot(none);
    const int mine = rank + __popcll(bal & ((1ull << lane) - 1));
    if (none && mine < n) put(mine, -INFINITY, b, t);
    rank += __popcll(bal);
  }
}

// A workgroup copies up to 16 KiB of a row, in the widest pieces that addresses, strides and the row allow.
constexpr int kRowPiece = 16384;
template <class V>   // (a vector type of the compiler's: an array of structures would pass through LDS)
__global__ __launch_bounds__(256) void reorder_rows_kernel(RowCopyArgs a, int pieces) {
  const int row = blockIdx.x / pieces, piece = blockIdx.x - row * pieces;
  const int p = a.parents[row];
  if ((unsigned)p >= (unsigned)a.in_rows) return;
  const int64_t from = (int64_t)piece * kRowPiece, bytes = min((int64_t)kRowPiece, a.row_bytes - from);
  const V* in = reinterpret_cast<const V*>(a.in + p * a.in_stride + from);
  V* out = reinterpret_cast<V*>(a.out + row * a.out_stride + from);
  constexpr int U = 4;
  const int n = (int)(bytes / sizeof(V));
  for (int i0 = threadIdx.x; i0 < n; i0 += 256 * U) {
    V v[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (i0 + u * 256 < n) v[u] = in[i0 + u * 256];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (i0 + u * 256 < n) out[i0 + u * 256] = v[u];
  }
}

template <class T>
void launch_scan(const BeamArgs& a, hipStream_t st) {
  const dim3 grid(a.chunks, a.groups * a.beams);
  if (a.threads == 256 && a.each == 16) beam_scan_kernel<T, 256, 16><<<grid, 256, 0, st>>>(a);
  else if (a.threads == 256) beam_scan_kernel<T, 256, 32><<<grid, 256, 0, st>>>(a);
  else beam_scan_kernel<T, 1024, 16><<<grid, 1024, 0, st>>>(a);
}

}  // namespace

void beam_plan(BeamArgs& a) {
  a.threads = a.n_out > kBeamFewOut ? 1024 : 256;
  // (chunks of twice the size where the others would not run at once)
  a.each = a.threads == 256 && (int64_t)a.groups * a.beams * ((a.vocab + 4095) / 4096) > kBeamWgs ? 32 : 16;
  a.chunks = (a.vocab + a.threads * a.each - 1) / (a.threads * a.each);
}

// Fewer rows or tokens may have the smaller chunks: as many of these as run at once.
int64_t beam_most_chunks(int64_t rows, int vocab, bool few) {
  auto chunks = [&](int size) { return rows * ((vocab + size - 1) / size); };
  if (!few) return chunks(16384);
  const int64_t small = chunks(4096), large = chunks(8192);
  return small <= kBeamWgs ? small : large > kBeamWgs ? large : kBeamWgs;
}

void launch_beam_select(const BeamArgs& a, int dtype, hipStream_t st) {
  if (dtype == EE_BF16) launch_scan<bf16_t>(a, st);
  else launch_scan<float>(a, st);
  beam_join_kernel<<<a.groups, kJoinThreads, 0, st>>>(a, dtype == EE_BF16);
}

void launch_reorder_rows(const RowCopyArgs& a, hipStream_t st) {
  const uint64_t all = reinterpret_cast<uintptr_t>(a.in) | reinterpret_cast<uintptr_t>(a.out) | a.in_stride | a.out_stride | a.row_bytes;
  const int pieces = (int)((a.row_bytes + kRowPiece - 1) / kRowPiece);
  const unsigned grid = (unsigned)((int64_t)a.rows * pieces);
  if (all % 16 == 0) reorder_rows_kernel<u32x4><<<grid, 256, 0, st>>>(a, pieces);
  else if (all % 4 == 0) reorder_rows_kernel<uint32_t><<<grid, 256, 0, st>>>(a, pieces);
  else reorder_rows_kernel<uint8_t><<<grid, 256, 0, st>>>(a, pieces);
}

}  // namespace ee
