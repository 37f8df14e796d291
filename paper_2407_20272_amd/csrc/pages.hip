// Pages of a cache that several sequences may share: tables are forked, grown with copy on write, released and packed on the device, by
// counts of the references to every block.  Nothing here waits for the host.
//
// All but the copies are bound by latency: a launch and three or four loads that wait for each other.  Kernel times: 4 beams of one prompt forked 2.2 us, grown 5.5, their last blocks copied 4.2,
// shared blocks found 3.9, released 2.1; 32 beams of 8 prompts 3.4, 7.1, 15 (28 blocks of 2.1 MB, 117 MB read
// and written, in part from the last-level cache), 5.6, 2.5; a pool of 2700 blocks packed 9.2, and 650 blocks of 0.26 MB copied 70 to 75
// (341 MB, 4.6 to 4.9 TB/s; a large copy makes 4.75).  Growing and packing look through small pools in one workgroup (4 rows grown: 5.5 us, in two launches 5.6 + 3.9).
#include "beams.h"

namespace ee {

namespace {

constexpr int kThreads = 256;
constexpr int kCopyWgs = 2048;   // workgroups of a copy that run at once

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__device__ inline int blocks_of(int len, int max_blocks) { return (min(max(len, 0), max_blocks * 16) + 15) >> 4; }

// A workgroup a row.  Rows of one parent count up the same blocks: integer additions, whose order does not show.
__global__ __launch_bounds__(kThreads) void pages_fork_kernel(int32_t* refs, int num_blocks, PageRows src, const int32_t* parents, PageRows dst) {
  const int row = blockIdx.x, p = parents[row];
  const bool some = (unsigned)p < (unsigned)src.rows;
  const int len = some ? min(max(src.lens[p], 0), src.max_blocks * 16) : 0;
  const int n = blocks_of(len, src.max_blocks);
  for (int e = threadIdx.x; e < n; e += kThreads) {
    const int b = src.tables[(size_t)p * src.max_blocks + e];
    dst.tables[(size_t)row * dst.max_blocks + e] = b;
    if ((unsigned)b < (unsigned)num_blocks) atomicAdd(&refs[b], 1);
  }
  if (threadIdx.x == 0) dst.lens[row] = len;
}

__global__ __launch_bounds__(kThreads) void pages_release_kernel(int32_t* refs, int num_blocks, PageRows r) {
  const int row = blockIdx.x;
  const int n = blocks_of(r.lens[row], r.max_blocks);
  for (int e = threadIdx.x; e < n; e += kThreads) {
    const int b = r.tables[(size_t)row * r.max_blocks + e];
    if ((unsigned)b < (unsigned)num_blocks) atomicSub(&refs[b], 1);
  }
  __syncthreads();   // every thread has read the length
  if (threadIdx.x == 0) r.lens[row] = 0;
}

// Which blocks of a chunk of 1024 have references: a bit each, and their number.
__device__ inline void taken_chunk(const int32_t* refs, int num_blocks, int chunk, const PageWork& w) {
  __shared__ int s_count[4];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  int count = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int word = wave * 4 + i, b = chunk * kPageChunk + word * 64 + lane;
    const uint64_t bits = __ballot(b < num_blocks && refs[b] > 0);
    count += __popcll(bits);
    if (lane == 0) w.taken[chunk * 16 + word] = bits;
  }
  if (lane == 0) s_count[wave] = count;
  __syncthreads();
  if (threadIdx.x == 0) w.counts[chunk] = s_count[0] + s_count[1] + s_count[2] + s_count[3];
}

// Sums of the values before each thread's, over the workgroup; `total` gets the sum of all.
__device__ inline int scan_before(int v, int& total) {
  __shared__ int s_wave[kThreads / 64];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  int upto = v;
#pragma unroll
  for (int x = 1; x < 64; x <<= 1) {
    const int o = __shfl_up(upto, x);
    if (lane >= x) upto += o;
  }
  __syncthreads();
  if (lane == 63) s_wave[wave] = upto;
  __syncthreads();
  int before = upto - v;
  total = 0;
#pragma unroll
  for (int i = 0; i < kThreads / 64; ++i) {
    if (i < wave) before += s_wave[i];
    total += s_wave[i];
  }
  return before;
}

// What the rows of a call want.  The last workgroup looks at the rows (a row whose partial last block others refer to wants a block in its place,
// but for the last of the call's rows where nobody else refers to it), the others at the pool.
__global__ __launch_bounds__(kThreads) void pages_want_kernel(const int32_t* refs, int num_blocks, int chunks, PageRows r, const int32_t* new_lens, PageWork w) {
  if ((int)blockIdx.x < chunks) {
    taken_chunk(refs, num_blocks, blockIdx.x, w);
    return;
  }
  const int cap = r.max_blocks * 16;
  auto written = [&](int m) {   // the partial block that row m goes on writing, or -1
    const int len = min(max(r.lens[m], 0), cap), to = min(new_lens[m], cap);
    if (to <= len || !(len & 15)) return -1;
    const int b = r.tables[(size_t)m * r.max_blocks + (len >> 4)];
    return (unsigned)b < (unsigned)num_blocks && refs[b] > 1 ? b : -1;
  };
  // (atomics throughout: these words pass from thread to thread)
  for (int m = threadIdx.x; m < r.rows; m += kThreads) {
    const int b = written(m);
    if (b >= 0) {
      atomicExch(&w.claims[b], 0);
      atomicExch(&w.latest[b], -1);
    }
  }
  __threadfence();
  __syncthreads();
  for (int m = threadIdx.x; m < r.rows; m += kThreads) {
    const int b = written(m);
    if (b >= 0) {
      atomicAdd(&w.claims[b], 1);
      atomicMax(&w.latest[b], m);
    }
  }
  __threadfence();
  __syncthreads();
  int sum = 0;
  for (int m0 = 0; m0 < r.rows; m0 += kThreads) {
    const int m = m0 + threadIdx.x;
    int want = 0;
    if (m < r.rows) {
      const int b = written(m);
      bool replace = b >= 0;
      if (replace) {
        const int claims = __hip_atomic_load(&w.claims[b], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        const int latest = __hip_atomic_load(&w.latest[b], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        replace = !(claims == refs[b] && latest == m);
      }
      w.replaces[m] = replace;
      want = replace + max(0, blocks_of(new_lens[m], r.max_blocks) - blocks_of(r.lens[m], r.max_blocks));
    }
    int total;
    const int before = scan_before(want, total);
    if (m < r.rows) w.row_first[m] = sum + before;
    sum += total;
  }
  if (threadIdx.x == 0) w.row_first[r.rows] = sum;
}

// The k-th bit that is not set of a word (k below their number).
__device__ inline int free_bit(uint64_t taken, int k) {
  uint64_t f = ~taken;
  int at = 0;
#pragma unroll
  for (int half = 32; half > 0; half >>= 1) {
    const int n = __popcll(f & ((1ull << half) - 1));
    if (k >= n) {
      k -= n;
      f >>= half;
      at += half;
    }
  }
  return at;
}

// The k-th free block (k below their number), by the chunks' free blocks before them.
__device__ inline int free_block(const PageWork& w, const int32_t* free_before, int chunks, int k) {
  int lo = 0, hi = chunks - 1;
  while (lo < hi) {   // the last chunk with free_before <= k
    const int mid = (lo + hi + 1) >> 1;
    if (free_before[mid] <= k) lo = mid;
    else hi = mid - 1;
  }
  k -= free_before[lo];
  for (int i = 0;; ++i) {
    const uint64_t t = w.taken[lo * 16 + i];
    const int n = 64 - __popcll(t);
    if (k < n || i == 15) return lo * kPageChunk + i * 64 + free_bit(t, k);
    k -= n;
  }
}

// free_before[c] of every chunk (in LDS), and the free blocks of the pool.
__device__ inline int count_free(const PageWork& w, int num_blocks, int chunks, int32_t* free_before) {
  int sum = 0;
  for (int c0 = 0; c0 < chunks; c0 += kThreads) {
    const int c = c0 + threadIdx.x;
    int total;
    const int before = scan_before(c < chunks ? min(kPageChunk, num_blocks - c * kPageChunk) - w.counts[c] : 0, total);
    if (c < chunks) free_before[c] = sum + before;
    sum += total;
  }
  __syncthreads();
  return sum;
}

// Hands the lowest free blocks to the rows, in the order of rows and entries: wanted block k is the k-th free one.  All rows or none.
__global__ __launch_bounds__(kThreads) void pages_give_kernel(int32_t* refs, int num_blocks, int chunks, PageRows r, const int32_t* new_lens, int32_t* moves,
                                                              int32_t* missing, PageWork w) {
  extern __shared__ int32_t free_before[];
  const int have = count_free(w, num_blocks, chunks, free_before);
  const int wanted = w.row_first[r.rows];
  const bool enough = wanted <= have;
  const int step = gridDim.x * kThreads, first = blockIdx.x * kThreads + threadIdx.x;
  if (first == 0) *missing = enough ? 0 : wanted - have;
  for (int m = first; m < r.rows; m += step) {
    if (!enough || !w.replaces[m]) {
      moves[2 * m] = -1;
      moves[2 * m + 1] = -1;
    }
  }
  if (!enough) return;
  for (int k = first; k < wanted; k += step) {
    int lo = 0, hi = r.rows - 1;   // the row whose blocks k is among: the last with row_first <= k
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (w.row_first[mid] <= k) lo = mid;
      else hi = mid - 1;
    }
    const int m = lo, i = k - w.row_first[m], replace = w.replaces[m];
    const int len = min(max(r.lens[m], 0), r.max_blocks * 16);
    const int block = free_block(w, free_before, chunks, k);
    int32_t* row = r.tables + (size_t)m * r.max_blocks;
    refs[block] = 1;
    if (replace && i == 0) {
      const int old = row[len >> 4];
      row[len >> 4] = block;
      atomicSub(&refs[old], 1);
      moves[2 * m] = old;
      moves[2 * m + 1] = block;
    } else {
      row[((len + 15) >> 4) + i - replace] = block;
    }
  }
}

// Both of these for rows and pools that one workgroup looks through: a launch and its waits less.  A thread has a row, a wavefront sixteen times 64 blocks; what it finds
// free it writes where the blocks before leave it in the list of free ones.
constexpr int kSmallRows = 1024, kSmallBlocks = 16384;
__global__ __launch_bounds__(1024) void pages_grow_kernel(int32_t* refs, int num_blocks, PageRows r, const int32_t* new_lens, int32_t* moves, int32_t* missing) {
  __shared__ int s_free[kSmallBlocks];
  __shared__ __align__(16) int s_written[kSmallRows];
  __shared__ int s_first[kSmallRows + 1];
  __shared__ int s_wave[2][16];
  const int t = threadIdx.x, wave = t >> 6, lane = t & 63, cap = r.max_blocks * 16;
  // the wavefront's blocks
  uint64_t free_bits[16];
  int n_free = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int b = wave * 1024 + i * 64 + lane;
    free_bits[i] = __ballot(b < num_blocks && refs[min(b, num_blocks - 1)] <= 0);
    n_free += __popcll(free_bits[i]);
  }
  // this thread's row: the block that it goes on writing, if others refer to it too
  int len = 0, to = 0, last = -1, count = 0;
  if (t < r.rows) {
    len = min(max(r.lens[t], 0), cap);
    to = max(len, min(new_lens[t], cap));
    if (to > len && (len & 15)) {
      last = r.tables[(size_t)t * r.max_blocks + (len >> 4)];
      if ((unsigned)last >= (unsigned)num_blocks) last = -1;
      else if ((count = refs[last]) <= 1) last = -1;
    }
  }
  s_written[t] = last;
  __syncthreads();
  bool replace = false;
  if (last >= 0) {   // all of its references are rows of this call, and this is the last of them: it keeps the block
    int claims = 0, later = 0;
    for (int m = 0; m < r.rows; m += 4) {
      const int4 w = *reinterpret_cast<const int4*>(&s_written[m]);   // (rows that there are not: -1)
      const int same = (w.x == last) + (w.y == last) + (w.z == last) + (w.w == last);
      claims += same;
      later |= (w.x == last && m > t) | (w.y == last && m + 1 > t) | (w.z == last && m + 2 > t) | (w.w == last && m + 3 > t);
    }
    replace = claims != count || later;
  }
  const int want = replace + ((to + 15) >> 4) - ((len + 15) >> 4);   // (0 of threads without a row)
  // sums of what is wanted before each thread, and of what is free before each wavefront
  int upto = want;
#pragma unroll
  for (int x = 1; x < 64; x <<= 1) {
    const int o = __shfl_up(upto, x);
    if (lane >= x) upto += o;
  }
  if (lane == 63) {
    s_wave[0][wave] = upto;
    s_wave[1][wave] = n_free;
  }
  __syncthreads();
  int first = upto - want, at = 0, wanted = 0, have = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    if (i < wave) {
      first += s_wave[0][i];
      at += s_wave[1][i];
    }
    wanted += s_wave[0][i];
    have += s_wave[1][i];
  }
  const bool enough = wanted <= have;
  if (t == 0) *missing = enough ? 0 : wanted - have;
  s_first[t] = first;
  if (t == 0) s_first[kSmallRows] = wanted;
  if (enough) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int k = at + __popcll(free_bits[i] & ((1ull << lane) - 1));
      if ((free_bits[i] >> lane & 1) && k < wanted) s_free[k] = wave * 1024 + i * 64 + lane;
      at += __popcll(free_bits[i]);
    }
  }
  __syncthreads();
  if (t < r.rows) {
    const int block = enough && replace ? s_free[first] : -1;
    moves[2 * t] = block >= 0 ? last : -1;
    moves[2 * t + 1] = block;
    if (block >= 0) {
      refs[block] = 1;
      r.tables[(size_t)t * r.max_blocks + (len >> 4)] = block;
      atomicSub(&refs[last], 1);
    }
    s_written[t] = replace ? ~((len + 15) >> 4) : (len + 15) >> 4;   // where its other blocks go (as the complement: the first has gone)
  }
  __syncthreads();
  if (!enough) return;
  for (int k = t; k < wanted; k += 1024) {
    int lo = 0, hi = r.rows - 1;   // the row whose blocks k is among: the last with s_first <= k
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (s_first[mid] <= k) lo = mid;
      else hi = mid - 1;
    }
    const int i = k - s_first[lo], behind = s_written[lo], replaced = behind < 0;
    if (i < replaced) continue;
    const int block = s_free[k];
    refs[block] = 1;
    r.tables[(size_t)lo * r.max_blocks + (replaced ? ~behind : behind) + i - replaced] = block;
  }
}

__global__ __launch_bounds__(kThreads) void pages_taken_kernel(const int32_t* refs, int num_blocks, PageWork w) { taken_chunk(refs, num_blocks, blockIdx.x, w); }

// Packing: with n blocks in use, the i-th of them behind the first n places goes to the i-th free place among these.  Every block finds its place by the
// counts alone, so one launch moves them all; what it reads of `refs` is only its own blocks' entries that move, which nobody writes.
__global__ __launch_bounds__(kThreads) void pages_pack_kernel(int32_t* refs, int num_blocks, int chunks, int32_t* remap, int32_t* moves, int32_t* n_moves, PageWork w) {
  extern __shared__ int32_t free_before[];
  const int n_free = count_free(w, num_blocks, chunks, free_before), n = num_blocks - n_free;
  auto before = [&](int b) {   // free blocks before block b (b < num_blocks)
    const int c = b / kPageChunk, word = (b % kPageChunk) >> 6;
    int k = free_before[c];
    for (int i = 0; i < word; ++i) k += 64 - __popcll(w.taken[c * 16 + i]);
    return k + __popcll(~w.taken[c * 16 + word] & ((1ull << (b & 63)) - 1));
  };
  const int n_go = n < num_blocks ? before(n) : n_free;   // free places among the first n: as many blocks lie behind
  if (blockIdx.x == 0 && threadIdx.x == 0) *n_moves = n_go;
  for (int b = blockIdx.x * kThreads + threadIdx.x; b < num_blocks; b += gridDim.x * kThreads) {
    const bool taken = w.taken[b / 64] >> (b & 63) & 1;
    if (b >= n_go) {
      moves[2 * b] = -1;
      moves[2 * b + 1] = -1;
    }
    if (!taken) {
      remap[b] = -1;
    } else if (b < n) {
      remap[b] = b;
    } else {
      const int rank = (b - before(b)) - (n - n_go);   // blocks in use before b, less those among the first n
      const int to = free_block(w, free_before, chunks, rank);
      remap[b] = to;
      moves[2 * rank] = b;
      moves[2 * rank + 1] = to;
      refs[to] = refs[b];
      refs[b] = 0;
    }
  }
}

// The same for pools that one workgroup looks through: the free places among the first n stand in a list.  `r` has rows where their tables are few enough to follow here.
constexpr int kSmallEntries = 16384;
__global__ __launch_bounds__(1024) void pages_pack_small_kernel(int32_t* refs, int num_blocks, PageRows r, int32_t* remap, int32_t* moves, int32_t* n_moves) {
  __shared__ int s_free[kSmallBlocks];
  __shared__ int s_wave[16];
  const int t = threadIdx.x, wave = t >> 6, lane = t & 63;
  uint64_t free_bits[16];
  int own[16], n_free = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int b = wave * 1024 + i * 64 + lane;
    own[i] = refs[min(b, num_blocks - 1)];
    free_bits[i] = __ballot(b < num_blocks && own[i] <= 0);
    n_free += __popcll(free_bits[i]);
  }
  if (lane == 0) s_wave[wave] = n_free;
  __syncthreads();
  int before = 0, all = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    if (i < wave) before += s_wave[i];
    all += s_wave[i];
  }
  const int n = num_blocks - all;
  // free blocks in front of each block; the last one among the first n leaves how many there are
  int at = before;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int b = wave * 1024 + i * 64 + lane, k = at + __popcll(free_bits[i] & ((1ull << lane) - 1));
    if (free_bits[i] >> lane & 1) s_free[k] = b;
    at += __popcll(free_bits[i]);
  }
  __syncthreads();
  int lo = 0, hi = all;            // free places among the first n: those of the list (ascending) below n
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (s_free[mid] < n) lo = mid + 1;
    else hi = mid;
  }
  const int n_go = lo;
  if (t == 0) *n_moves = n_go;
  at = before;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int b = wave * 1024 + i * 64 + lane, k = at + __popcll(free_bits[i] & ((1ull << lane) - 1));
    at += __popcll(free_bits[i]);
    if (b >= num_blocks) continue;
    if (b >= n_go) {
      moves[2 * b] = -1;
      moves[2 * b + 1] = -1;
    }
    if (own[i] <= 0) {
      remap[b] = -1;
    } else if (b < n) {
      remap[b] = b;
    } else {
      const int rank = (b - k) - (n - n_go), to = s_free[rank];
      remap[b] = to;
      moves[2 * rank] = b;
      moves[2 * rank + 1] = to;
      refs[to] = own[i];
      refs[b] = 0;
    }
  }
  __syncthreads();   // (what the workgroup has written it may read)
  for (int i = t; i < r.rows * r.max_blocks; i += 1024) {
    const int row = i / r.max_blocks, e = i - row * r.max_blocks, b = r.tables[i];
    if (e < blocks_of(r.lens[row], r.max_blocks) && (unsigned)b < (unsigned)num_blocks) r.tables[i] = remap[b];
  }
}

__global__ __launch_bounds__(kThreads) void pages_remap_kernel(const int32_t* remap, int num_blocks, PageRows r) {
  const int row = blockIdx.x, n = blocks_of(r.lens[row], r.max_blocks);
  for (int e = threadIdx.x; e < n; e += kThreads) {
    int32_t* at = r.tables + (size_t)row * r.max_blocks + e;
    const int b = *at;
    if ((unsigned)b < (unsigned)num_blocks) *at = remap[b];
  }
}

// A workgroup a group: the first entry that one of its rows has otherwise than the first row, or that one of them has not filled.
__global__ __launch_bounds__(kThreads) void pages_shared_kernel(PageRows r, const int32_t* first_row, int32_t* shared) {
  __shared__ int s_least;
  const int g = blockIdx.x;
  const int a = min(max(first_row[g], 0), r.rows), z = min(max(first_row[g + 1], a), r.rows);
  if (threadIdx.x == 0) s_least = r.max_blocks;
  __syncthreads();
  for (int m = a + threadIdx.x; m < z; m += kThreads) atomicMin(&s_least, min(max(r.lens[m], 0), r.max_blocks * 16) >> 4);
  __syncthreads();
  const int full = a < z ? s_least : 0;
  int same = full;
  for (int e0 = 0; e0 < full; e0 += kThreads) {
    const int e = e0 + threadIdx.x;
    if (e < full) {
      const int b = r.tables[(size_t)a * r.max_blocks + e];
      bool differs = false;
#pragma unroll 8
      for (int m = a + 1; m < z; ++m) differs |= r.tables[(size_t)m * r.max_blocks + e] != b;
      if (differs) same = min(same, e);
    }
    if (__syncthreads_or(same < full)) break;
  }
  atomicMin(&s_least, same);
  __syncthreads();
  if (threadIdx.x == 0) shared[g] = a < z ? s_least : 0;
}

// Copies blocks of every pool, in pieces of 16 KiB: a workgroup takes its pieces of the moves that are its own in turn.  Bound by memory.
constexpr int kCopyMoves = 1024;
constexpr int kCopyPiece = 16384;

__device__ inline void copy_piece(const PageCopyArgs& a, int2 move, int piece) {
  int p = 0;
  while (p + 1 < a.n_pools && piece >= a.pool[p].pieces) piece -= a.pool[p++].pieces;
  const PagePlane& pool = a.pool[p];
  const int each = (int)((pool.block_bytes + kCopyPiece - 1) / kCopyPiece), plane = piece / each, at0 = piece - plane * each;
  char* base = pool.base + (size_t)plane * a.num_blocks * pool.block_bytes + (size_t)at0 * kCopyPiece;
  const char* src = base + (size_t)move.x * pool.block_bytes;
  char* dst = base + (size_t)move.y * pool.block_bytes;
  const int bytes = (int)min((size_t)kCopyPiece, pool.block_bytes - (size_t)at0 * kCopyPiece);
  if (pool.wide) {
    u32x4 v[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int at = (u * kThreads + threadIdx.x) * 16;
      v[u] = u32x4{};
      if (at < bytes) v[u] = *reinterpret_cast<const u32x4*>(src + at);
    }
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (const int at = (u * kThreads + threadIdx.x) * 16; at < bytes) *reinterpret_cast<u32x4*>(dst + at) = v[u];
  } else {
    for (int at = threadIdx.x * 8; at < bytes; at += kThreads * 8) *reinterpret_cast<u32x2*>(dst + at) = *reinterpret_cast<const u32x2*>(src + at);
  }
}

__device__ inline bool is_move(const PageCopyArgs& a, int2 m) {
  return (unsigned)m.x < (unsigned)a.num_blocks && (unsigned)m.y < (unsigned)a.num_blocks && m.x != m.y;
}

// The list has `count` moves, one behind the other (any of them may be none).
__global__ __launch_bounds__(kThreads) void pages_copy_kernel(PageCopyArgs a) {
  const int n = min(max(*a.count, 0), a.n);
  for (int m = blockIdx.y; m < n; m += gridDim.y) {
    const int2 move = make_int2(a.moves[2 * m], a.moves[2 * m + 1]);
    if (!is_move(a, move)) continue;
    for (int piece = blockIdx.x; piece < a.pieces; piece += gridDim.x) copy_piece(a, move, piece);
  }
}

// Moves anywhere in the list: those there are of 1024 entries at a time are gathered in LDS, in their order.
__global__ __launch_bounds__(kThreads) void pages_copy_sparse_kernel(PageCopyArgs a) {
  __shared__ int2 s_move[kCopyMoves];
  for (int m0 = 0; m0 < a.n; m0 += kCopyMoves) {
    int there = 0;
    __syncthreads();
    for (int m1 = m0; m1 < min(a.n, m0 + kCopyMoves); m1 += kThreads) {
      const int m = m1 + threadIdx.x;
      const int2 move = m < a.n ? make_int2(a.moves[2 * m], a.moves[2 * m + 1]) : make_int2(-1, -1);
      const bool goes = is_move(a, move);
      int total;
      const int before = scan_before(goes, total);
      if (goes) s_move[there + before] = move;
      there += total;
    }
    __syncthreads();
    for (int m = blockIdx.y; m < there; m += gridDim.y)
      for (int piece = blockIdx.x; piece < a.pieces; piece += gridDim.x) copy_piece(a, s_move[m], piece);
  }
}

}  // namespace

void launch_pages_fork(int32_t* refs, int num_blocks, const PageRows& src, const int32_t* parents, const PageRows& dst, hipStream_t st) {
  pages_fork_kernel<<<dst.rows, kThreads, 0, st>>>(refs, num_blocks, src, parents, dst);
}

void launch_pages_release(int32_t* refs, int num_blocks, const PageRows& r, hipStream_t st) { pages_release_kernel<<<r.rows, kThreads, 0, st>>>(refs, num_blocks, r); }

void launch_pages_grow(int32_t* refs, int num_blocks, const PageRows& r, const int32_t* new_lens, int32_t* moves, int32_t* missing, const PageWork& w,
                       hipStream_t st) {
  if (r.rows <= kSmallRows && num_blocks <= kSmallBlocks) {
    pages_grow_kernel<<<1, 1024, 0, st>>>(refs, num_blocks, r, new_lens, moves, missing);
    return;
  }
  const int chunks = page_chunks(num_blocks);
  pages_want_kernel<<<chunks + 1, kThreads, 0, st>>>(refs, num_blocks, chunks, r, new_lens, w);
  const int wgs = r.rows < 4096 ? 8 : 64;   // (rows want about one block each; a prompt's thousand are four blocks a thread)
  pages_give_kernel<<<wgs, kThreads, chunks * sizeof(int32_t), st>>>(refs, num_blocks, chunks, r, new_lens, moves, missing, w);
}

void launch_pages_compact(int32_t* refs, int num_blocks, const PageRows& r, int32_t* remap, int32_t* moves, int32_t* n_moves, const PageWork& w, hipStream_t st) {
  if (num_blocks <= kSmallBlocks) {
    const bool follow = (int64_t)r.rows * r.max_blocks <= kSmallEntries;
    pages_pack_small_kernel<<<1, 1024, 0, st>>>(refs, num_blocks, follow ? r : PageRows{}, remap, moves, n_moves);
    if (follow) return;
  } else {
    const int chunks = page_chunks(num_blocks);
    pages_taken_kernel<<<chunks, kThreads, 0, st>>>(refs, num_blocks, w);
    pages_pack_kernel<<<(num_blocks + kThreads - 1) / kThreads, kThreads, chunks * sizeof(int32_t), st>>>(refs, num_blocks, chunks, remap, moves, n_moves, w);
  }
  if (r.rows > 0) pages_remap_kernel<<<r.rows, kThreads, 0, st>>>(remap, num_blocks, r);
}

void launch_pages_shared(const PageRows& r, const int32_t* first_row, int n_groups, int32_t* shared, hipStream_t st) {
  pages_shared_kernel<<<n_groups, kThreads, 0, st>>>(r, first_row, shared);
}

void launch_pages_copy(PageCopyArgs a, hipStream_t st) {
  a.pieces = 0;
  for (int p = 0; p < a.n_pools; ++p) {
    PagePlane& pool = a.pool[p];
    pool.pieces = pool.planes * (int)((pool.block_bytes + kCopyPiece - 1) / kCopyPiece);
    pool.wide = ((pool.block_bytes | reinterpret_cast<uintptr_t>(pool.base)) & 15) == 0;
    a.pieces += pool.pieces;
  }
  // As many workgroups as run at once, or as the moves have pieces.
  const int across = a.pieces < kCopyWgs ? a.pieces : kCopyWgs;
  int down = (kCopyWgs + across - 1) / across;
  if (down > a.n) down = a.n;
  if (a.count) pages_copy_kernel<<<dim3(across, down), kThreads, 0, st>>>(a);
  else pages_copy_sparse_kernel<<<dim3(across, down), kThreads, 0, st>>>(a);
}

}  // namespace ee
