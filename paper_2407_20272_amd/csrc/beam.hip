// One step of beam search: the best continuations of every group over its beams and the whole vocabulary, and rows of states in their new order.
//
//   score(b, t) = scores[b] + (z[b][t] - log sum_t' exp z[b][t'])
//
// Two launches.  The scan reads the logits once: a workgroup takes a chunk of a row, keeps its values in registers, and leaves the chunk's maximum, its
// sum of exponentials and its n best, in order (within a beam the order of the scores is that of the logits, so this needs no sum of the whole row).
// The join forms the rows' sums from the chunks', the scores of what was found, and the n best of these.
// What is compared are scores in double: rounded to float many candidates of a beam would be equal, and beams' sums meet there.
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
__device__ inline float float_of(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key); }
__device__ inline uint64_t key_of(double s) {
  const uint64_t u = (uint64_t)__double_as_longlong(s + 0.0);
  return u >> 63 ? ~u : u | 1ull << 63;
}
__device__ inline double double_of(uint64_t key) { return __longlong_as_double((long long)(key >> 63 ? key & ~(1ull << 63) : ~key)); }

// The largest bound of which at least n of the keys are not below (each lane has K of them; the wavefront's together), to its upper `BITS` bits; at least 1.
template <int K, int BITS>
__device__ inline uint32_t wave_bound(const uint32_t (&key)[K], int n) {
  uint32_t bound = 0;
  for (int bit = 31; bit >= 32 - BITS; --bit) {
    const uint32_t c = bound | 1u << bit;
    int count = 0;
#pragma unroll
    for (int i = 0; i < K; ++i) count += __popcll(__ballot(key[i] >= c));
    if (count >= n) bound = c;
  }
  return bound ? bound : 1u;
}

constexpr int kScanList = 512;   // candidates of a chunk that are put in order

// A chunk of THREADS * EACH values.  What falls behind the n-th largest of the threads' maxima is none of the n best; the others (n and a few) are
// gathered and put in order by counting, for each, those in front of it.  Where they are too many (many equal values), the n-th of all is found bit by bit first.
template <class T, int THREADS, int EACH>
__global__ __launch_bounds__(THREADS) void beam_scan_kernel(BeamArgs a) {
  constexpr int VEC = 16 / sizeof(T), LOADS = EACH / VEC, WAVES = THREADS / 64;
  __shared__ uint64_t s_list[kScanList];
  __shared__ uint32_t s_most[THREADS];
  __shared__ double s_sum[WAVES];
  __shared__ float s_max[WAVES];
  __shared__ int s_count, s_below[WAVES];
  const int row = blockIdx.y, chunk = blockIdx.x;
  if (a.finished && a.finished[row]) return;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int base = chunk * THREADS * EACH;
  const T* z = reinterpret_cast<const T*>(a.logits) + (size_t)row * a.stride;
  if (threadIdx.x == 0) s_count = 0;

  // Values `at(l) + e` for piece l; the same places whether the row starts on 16 bytes or not, so that equal rows have equal sums.
  auto at = [&](int l) { return base + (l * THREADS + (int)threadIdx.x) * VEC; };
  float x[EACH];
  const bool aligned = ((reinterpret_cast<uintptr_t>(a.logits) | (a.stride * sizeof(T))) & 15) == 0;
  if (aligned) {
    u32x4 raw[LOADS];
#pragma unroll
    for (int l = 0; l < LOADS; ++l)
      if (at(l) + VEC <= a.vocab) raw[l] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(z + at(l)));
#pragma unroll
    for (int l = 0; l < LOADS; ++l) {
      if (at(l) + VEC <= a.vocab) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          if constexpr (sizeof(T) == 4) x[l * VEC + e] = __uint_as_float(raw[l][e]);
          else x[l * VEC + e] = __uint_as_float(e & 1 ? raw[l][e / 2] & 0xffff0000u : raw[l][e / 2] << 16);
        }
      } else {
#pragma unroll
        for (int e = 0; e < VEC; ++e) x[l * VEC + e] = at(l) + e < a.vocab ? (float)z[at(l) + e] : -INFINITY;
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      const int t = at(i / VEC) + i % VEC;
      x[i] = t < a.vocab ? (float)z[t] : -INFINITY;
    }
  }

  float most = -INFINITY;
#pragma unroll
  for (int i = 0; i < EACH; ++i) most = fmaxf(most, x[i]);
  s_most[threadIdx.x] = key_of(most);
  float top = most;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) top = fmaxf(top, __shfl_xor(top, o));
  if (lane == 0) s_max[wave] = top;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < WAVES; ++i) top = fmaxf(top, s_max[i]);
  // (a chunk without a value has a sum of 0, one with a NaN or +inf a sum that is NaN: so has its row)
  const float ref = top == -INFINITY ? 0.0f : top;
  float part = 0.0f;
#pragma unroll
  for (int i = 0; i < EACH; ++i) part += __expf(x[i] - ref);
  double sum = part;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) sum += __shfl_xor(sum, o);
  if (lane == 0) s_sum[wave] = sum;

  // the n-th largest of the threads' maxima, found by every wavefront for itself
  const int n = a.n_out;
  uint32_t bound;
  {
    uint32_t key[WAVES];
#pragma unroll
    for (int i = 0; i < WAVES; ++i) key[i] = s_most[i * 64 + lane];
    bound = wave_bound<WAVES, 20>(key, n);
  }
  auto composite = [&](int i) { return (uint64_t)key_of(x[i]) << 32 | (0xffffffffu - (uint32_t)(at(i / VEC) + i % VEC)); };
  auto gather = [&](uint64_t from) {
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      const uint64_t c = composite(i);
      if (c >= from) {
        const int k = atomicAdd(&s_count, 1);
        if (k < kScanList) s_list[k] = c;
      }
    }
  };
  gather((uint64_t)bound << 32);
  __syncthreads();
  int count = s_count;
  if (count > kScanList) {
    uint64_t from = 0;
    for (int bit = 63; bit >= 0; --bit) {
      const uint64_t c = from | 1ull << bit;
      int mine = 0;
#pragma unroll
      for (int i = 0; i < EACH; ++i) mine += composite(i) >= c;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) mine += __shfl_xor(mine, o);
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
    gather(from);   // (composites differ: n of them)
    __syncthreads();
    count = min(s_count, kScanList);
  }
  const size_t piece = (size_t)row * a.chunks + chunk;
  if (threadIdx.x == 0) {
    double total = 0.0;
    for (int i = 0; i < WAVES; ++i) total += s_sum[i];
    a.stats[piece] = make_double2(top, total);
  }
  uint64_t* found = a.found + piece * n;
  for (int i = threadIdx.x; i < count; i += THREADS) {
    const uint64_t c = s_list[i];
    int rank = 0;
    for (int j = 0; j < count; ++j) rank += s_list[j] > c;
    if (rank < n) found[rank] = c;
  }
  for (int i = count + (int)threadIdx.x; i < n; i += THREADS) found[i] = 0;
}

constexpr int kJoinThreads = 1024;
constexpr int kJoinList = 1024;

// A workgroup a group.
__global__ __launch_bounds__(kJoinThreads) void beam_join_kernel(BeamArgs a, int is_bf16) {
  constexpr int WAVES = kJoinThreads / 64;
  __shared__ double s_lse[kBeamMost], s_base[kBeamMost];
  __shared__ int s_done[kBeamMost];
  __shared__ uint32_t s_most[kJoinThreads];
  __shared__ uint64_t s_key[kJoinList];
  __shared__ uint64_t s_cand[kJoinList]; // index: beam * vocab + token
  __shared__ int s_count, s_below[WAVES];
  const int g = blockIdx.x, n = a.n_out, W = a.beams, row0 = g * W;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  if (threadIdx.x == 0) s_count = 0;
  // the rows' sums, a wavefront a row (a fixed order of additions)
  for (int b = wave; b < W; b += WAVES) {
    const int row = row0 + b;
    const bool done = a.finished && a.finished[row];
    double m = -INFINITY, sum = 0.0;
    if (!done) {
      for (int c = lane; c < a.chunks; c += 64) m = fmax(m, a.stats[(size_t)row * a.chunks + c].x);
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) m = fmax(m, __shfl_xor(m, o));
      for (int c = lane; c < a.chunks; c += 64) {
        const double2 s = a.stats[(size_t)row * a.chunks + c];
        if (s.y != 0.0) sum += s.y * exp(s.x - m);   // (NaN stays)
      }
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) sum += __shfl_xor(sum, o);
    }
    if (lane == 0) {
      s_lse[b] = m + log(sum);
      s_base[b] = a.scores[row];
      s_done[b] = done;
    }
  }
  __syncthreads();
  const int per_beam = a.chunks * n;
  const int all = W * per_beam;
  // key of candidate i (0: none), and its index
  auto candidate = [&](int i, uint64_t& index) -> uint64_t {
    const int b = i / per_beam, j = i - b * per_beam;
    double s;
    if (s_done[b]) {
      if (j) return 0;
      s = s_base[b];
      index = (uint64_t)b * a.vocab + a.end_token;
    } else {
      const uint64_t c = a.found[(size_t)(row0 + b) * per_beam + j];
      if (!(c >> 32)) return 0;
      s = s_base[b] + ((double)float_of((uint32_t)(c >> 32)) - s_lse[b]);
      index = (uint64_t)b * a.vocab + (0xffffffffu - (uint32_t)c);
    }
    return s - s == 0.0 ? key_of(s) : 0;   // what is not finite is none
  };
  uint32_t most = 0;
  for (int i = threadIdx.x; i < all; i += kJoinThreads) {
    uint64_t index;
    most = max(most, (uint32_t)(candidate(i, index) >> 32));
  }
  s_most[threadIdx.x] = most;
  __syncthreads();
  uint32_t bound;
  {
    uint32_t key[WAVES];
#pragma unroll
    for (int i = 0; i < WAVES; ++i) key[i] = s_most[i * 64 + lane];
    bound = wave_bound<WAVES, 32>(key, n);
  }
  // in front: larger score, or an equal one and the lower index
  auto gather = [&](uint64_t from, uint64_t up_to) {
    for (int i = threadIdx.x; i < all; i += kJoinThreads) {
      uint64_t index;
      const uint64_t k = candidate(i, index);
      if (k > from || (k == from && index <= up_to)) {
        const int at = atomicAdd(&s_count, 1);
        if (at < kJoinList) {
          s_key[at] = k;
          s_cand[at] = index;
        }
      }
    }
  };
  auto block_count = [&](auto&& test) {
    int mine = 0;
    for (int i = threadIdx.x; i < all; i += kJoinThreads) {
      uint64_t index;
      const uint64_t k = candidate(i, index);
      mine += k != 0 && test(k, index);
    }
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) mine += __shfl_xor(mine, o);
    __syncthreads();
    if (lane == 0) s_below[wave] = mine;
    __syncthreads();
    int sum = 0;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) sum += s_below[i];
    return sum;
  };
  gather((uint64_t)bound << 32, ~0ull);
  __syncthreads();
  int count = s_count;
  if (count > kJoinList) {   // many equal scores: the n-th bit by bit, then its index
    uint64_t from = 0;
    for (int bit = 63; bit >= 0; --bit) {
      const uint64_t c = from | 1ull << bit;
      if (block_count([&](uint64_t k, uint64_t) { return k >= c; }) >= n) from = c;
    }
    uint64_t up_to = 0;   // the least index with which n are in front of or at (from, index)
    for (int bit = 39; bit >= 0; --bit) {
      const uint64_t c = up_to | 1ull << bit;
      if (block_count([&](uint64_t k, uint64_t index) { return k > from || (k == from && index < c); }) < n) up_to = c;
    }
    if (threadIdx.x == 0) s_count = 0;
    __syncthreads();
    gather(from, up_to);
    __syncthreads();
    count = min(s_count, kJoinList);
  }
  auto put = [&](int rank, double s, uint64_t index) {
    const int b = (int)(index / a.vocab), t = (int)(index - (uint64_t)b * a.vocab);
    const size_t at = (size_t)g * n + rank;
    a.scores_out[at] = (float)s;
    a.tokens[at] = t;
    a.parents[at] = row0 + b;
    if (a.finished_out) a.finished_out[at] = s_done[b] || t == a.end_token;
  };
  for (int i = threadIdx.x; i < count; i += kJoinThreads) {
    const uint64_t k = s_key[i], index = s_cand[i];
    int rank = 0;
    for (int j = 0; j < count; ++j) rank += s_key[j] > k || (s_key[j] == k && s_cand[j] < index);
    if (rank < n) put(rank, double_of(k), index);
  }
  if (count >= n) return;
  // Fewer candidates than asked for: the rest are the lowest indices whose score is -inf, found by looking (one wavefront, 64 indices at a time).
  if (wave) return;
  int rank = count;
  for (uint64_t i0 = 0; rank < n && i0 < (uint64_t)W * a.vocab; i0 += 64) {
    const uint64_t index = i0 + lane;
    bool none = index < (uint64_t)W * a.vocab;
    if (none) {
      const int b = (int)(index / a.vocab), t = (int)(index - (uint64_t)b * a.vocab);
      if (s_done[b]) {
        none = t != a.end_token || !(s_base[b] - s_base[b] == 0.0);
      } else {
        const size_t at = (size_t)(row0 + b) * a.stride + t;
        const float z = is_bf16 ? (float)reinterpret_cast<const bf16_t*>(a.logits)[at] : reinterpret_cast<const float*>(a.logits)[at];
        const double s = s_base[b] + ((double)z - s_lse[b]);
        none = !(s - s == 0.0);
      }
    }
    const uint64_t bal = __ballot(none);
    const int mine = rank + __popcll(bal & ((1ull << lane) - 1));
    if (none && mine < n) put(mine, -INFINITY, index);
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
  if (a.threads == 256) beam_scan_kernel<T, 256, 16><<<grid, 256, 0, st>>>(a);
  else beam_scan_kernel<T, 1024, 16><<<grid, 1024, 0, st>>>(a);
}

}  // namespace

void beam_plan(BeamArgs& a) {
  a.threads = a.n_out > kBeamFewOut ? 1024 : 256;
  a.each = 16;
  a.chunks = (a.vocab + a.threads * a.each - 1) / (a.threads * a.each);
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
