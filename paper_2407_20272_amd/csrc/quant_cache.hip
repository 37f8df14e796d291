// The 8-bit cache: appending, reading back, eviction.
//
// A wavefront works on one (block, head) of K or of V.  Lane l holds the channels (2l, 2l + 1) (and 128 further on for heads of more than 128
// channels) of up to 16 positions, so a position's row is one load of consecutive bytes, the largest magnitude is one reduction over the wavefront, and V,
// whose block is [head_dim][16], is 16 consecutive bytes a channel.
#include "quant.h"

namespace ee {

namespace {

constexpr int kThreads = 256;

// The float that a byte of value v stands for.
template <int FMT>
__device__ inline f32x2 byte_pair(uint32_t two) {   // bytes 0 and 1
  if constexpr (FMT == EE_QUANT_INT8) {
    return f32x2{(float)(int8_t)(two & 0xff), (float)(int8_t)((two >> 8) & 0xff)};
  } else {
    return __builtin_amdgcn_cvt_pk_f32_fp8(two, false);
  }
}

// The largest scales: 127 times this one is still a float; with the other a byte may be 240 at most (256 times it is none, the largest float divided by it is
// next to 256).
constexpr float kInt8ScaleMost = 0x1.020406p+121f, kE4m3ScaleMost = 0x1p120f;

// The smallest scale with which `largest` fits; NaN for an infinity or NaN (a magnitude's bits are ordered as integers).
template <int FMT>
__device__ inline float scale_for(float largest) {
  if (!(largest < INFINITY)) return __builtin_nanf("");
  if constexpr (FMT == EE_QUANT_INT8) {
    return fminf(fmaxf(largest / 127.0f, kQuantScaleFloor), kInt8ScaleMost);
  } else {
    int e;
    const float m = frexpf(largest, &e);             // 448 = 0.875 * 2^9
    return largest > 0.0f ? ldexpf(1.0f, max(e - 9 + (m > 0.875f), -126)) : kQuantScaleFloor;
  }
}

// The bytes nearest to x / s, ties to even, of a number of pairs (inv = 1 / s).
// E4M3: s is a power of two, so the product with inv is exact and the conversion rounds once.
// INT8: adding 1.5 * 2^23 to the product leaves its nearest integer in the sum's low byte.  The product is up to 2.3e-5 away from x / s, which
// matters where it lies that near to the middle between two integers (one wavefront in eight): there the exact remainder x - q s decides (one fma:
// |remainder| <= s and a multiple of the smaller operand's last place, so it has 24 bits).
template <int FMT, int N, class F>
__device__ inline void quantise(F&& value, uint32_t (&out)[N], float s, float inv) {
  if (s != s) {
#pragma unroll
    for (int i = 0; i < N; ++i) out[i] = 0;
    return;
  }
  if constexpr (FMT == EE_QUANT_E4M3) {
    if (s >= kE4m3ScaleMost) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const f32x2 x = value(i);
        out[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(fminf(fmaxf(x[0] * inv, -240.0f), 240.0f), fminf(fmaxf(x[1] * inv, -240.0f), 240.0f), 0, false) & 0xffff;
      }
      return;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const f32x2 x = value(i);
      out[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[0] * inv, x[1] * inv, 0, false) & 0xffff;
    }
  } else {
    constexpr float kInteger = 12582912.0f;
    float off = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const f32x2 x = value(i);
      const float y0 = fmaf(x[0], inv, kInteger), y1 = fmaf(x[1], inv, kInteger);
      off = fmaxf(off, fmaxf(fabsf(fmaf(x[0], inv, kInteger - y0)), fabsf(fmaf(x[1], inv, kInteger - y1))));
      out[i] = __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, y1), __builtin_bit_cast(uint32_t, y0), 0x0c0c0400u);
    }
    if (__any(off > 0.49997f)) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const f32x2 x = value(i);
        uint32_t r = 0;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float q = rintf(x[e] * inv);
          const float rem = fmaf(-q, s, x[e]), twice = 2.0f * fabsf(rem);
          if (twice > s || (twice == s && ((int)q & 1))) q += copysignf(1.0f, rem);
          r |= (uint32_t)((int)q & 0xff) << (8 * e);
        }
        out[i] = r;
      }
    }
  }
}

// The larger of two scales; NaN if either is.
__device__ inline float scale_max(float a, float b) { return a != a || b != b ? __builtin_nanf("") : fmaxf(a, b); }

// Rows that go into (or come from) one block are taken together: a run is rows at consecutive positions of one block.  A workgroup has kGroup
// rows (one, where every row is a sequence of its own) of two heads and takes the runs that begin among them, one after the other;
// a wavefront for K and V of either head.  (Groups of 8: a chunk's runs of 16 leave every second workgroup empty, rows of many sequences take eight turns.
// With a wavefront a row, 15 of 16 of them empty, 2103 rows took 43 us instead of 17.  Groups of 4, 8, 16, E4M3: 2103 rows of three sequences 17.4, 14.3, 14.6 us where
// no scale grows and 18.5, 18.1, 20.1 where those of the first blocks do; 300 rows of 100 sequences 6.2, 6.6, 11.4 and 14.2, 16.2, 25.8; 1000 rows of 500 sequences
// 10.2, 11.7, 15.2 and 26, 32, 37.  INT8: 24, 20, 21 and 26, 23, 26; 7.0, 9.0, 14.0 and 14.9, 17.5, 29; 10.5, 12.6, 18.3 and 27, 33, 39.)
constexpr int kGroup = 8;
struct Run {
  int m, n, off, seq, logical;   // first row, rows, the first one's place in its block
};
struct Runs {
  int base, pos, seq;            // lane i stands for row base - 1 + i
  uint64_t goes_on, first;       // the lanes whose row goes on with the run of the row in front; that begin a run of this workgroup

  __device__ Runs(const QuantRows& r, int base_, int group) : base(base_) {
    const int lane = threadIdx.x & 63, at = base - 1 + lane;
    const bool there = lane <= group + 15 && at >= 0 && at < r.rows;
    pos = there ? r.context_lens[at] : -1;
    seq = there && r.row_table ? r.row_table[at] : at;
    if ((unsigned)seq >= (unsigned)r.rows) pos = -1; // (a row of no sequence is written nowhere)
    const int pos_before = __shfl_up(pos, 1), seq_before = __shfl_up(seq, 1);
    const bool on = lane > 0 && pos > 0 && pos_before == pos - 1 && seq_before == seq && (pos & 15) != 0;
    goes_on = __ballot(on);
    first = __ballot(lane > 0 && lane <= group && pos >= 0 && !on);
  }
  __device__ Run of(int lane) const {
    const uint64_t stop = ~(goes_on >> (lane + 1));            // (lanes behind group + 15 never go on)
    const int p = lane_value(pos, lane);
    return Run{base - 1 + lane, __ffsll((unsigned long long)stop), p & 15, lane_value(seq, lane), p >> 4};
  }
};

template <class T>
__device__ inline f32x2 load_pair(const T* p);
template <>
__device__ inline f32x2 load_pair<float>(const float* p) { return *reinterpret_cast<const f32x2*>(p); }
template <>
__device__ inline f32x2 load_pair<bf16_t>(const bf16_t* p) {
  const uint32_t u = *reinterpret_cast<const uint32_t*>(p);
  return f32x2{__builtin_bit_cast(float, u << 16), __builtin_bit_cast(float, u & 0xffff0000u)};
}

__device__ inline uint32_t magnitude(float x) { return __builtin_bit_cast(uint32_t, x) & 0x7fffffffu; }

// What a run's rows are to become: where they are, their block, its scale in front.
template <class T>
struct AppendTo {
  const T* src;
  int64_t stride;
  int8_t* block;
  float* scale;
  bool there;
  __device__ AppendTo(const QuantAppendArgs& a, const Run& run, int head, int which) {
    src = reinterpret_cast<const T*>(which ? a.v : a.k) + (size_t)run.m * (which ? a.v_stride : a.k_stride) + (size_t)head * a.c.dh;
    stride = which ? a.v_stride : a.k_stride;
    const int blk = run.logical < a.r.max_blocks ? a.r.block_tables[(size_t)run.seq * a.r.max_blocks + run.logical] : -1;
    there = (unsigned)blk < (unsigned)a.c.num_blocks;
    const size_t unit = (size_t)(there ? blk : 0) * a.c.heads + head;
    block = (which ? a.c.v : a.c.k) + unit * 16 * a.c.dh;
    scale = a.c.scales + unit * 2 + which;
  }
};
template <class T>
struct RawPair;
template <>
struct RawPair<float> {
  typedef f32x2 type;
  static __device__ f32x2 value(f32x2 r) { return r; }
};
template <>
struct RawPair<bf16_t> {
  typedef uint32_t type;
  static __device__ f32x2 value(uint32_t u) { return f32x2{__builtin_bit_cast(float, u << 16), __builtin_bit_cast(float, u & 0xffff0000u)}; }
};

// Four positions' bytes of channels c and c + 1 -> the two channels' words.
__device__ inline void words_of(uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t& lo, uint32_t& hi) {
  const uint32_t first = a0 | a1 << 16, second = a2 | a3 << 16;
  lo = __builtin_amdgcn_perm(second, first, 0x06040200u);
  hi = __builtin_amdgcn_perm(second, first, 0x07050301u);
}

// A whole block.
template <int FMT, class T, int CP>
__device__ inline void append_block(const QuantAppendArgs& a, const Run& run, int head, int which) {
  typedef typename RawPair<T>::type raw_t;
  const int lane = threadIdx.x & 63, dh = a.c.dh;
  const AppendTo<T> to(a, run, head, which);
  raw_t x[16 * CP];
  uint32_t most = 0;
#pragma unroll
  for (int t = 0; t < 16; ++t)
#pragma unroll
    for (int i = 0; i < CP; ++i) {
      const int c = 2 * lane + 128 * i;
      x[t * CP + i] = raw_t{};
      if (c < dh) x[t * CP + i] = *reinterpret_cast<const raw_t*>(to.src + t * to.stride + c);
    }
  if (!to.there) return;
#pragma unroll
  for (int i = 0; i < 16 * CP; ++i) {
    const f32x2 y = RawPair<T>::value(x[i]);
    most = max(most, max(magnitude(y[0]), magnitude(y[1])));
  }
  const float s = scale_for<FMT>(__builtin_bit_cast(float, wave_max(most)));
  if (lane == 0) *to.scale = s;
  uint32_t two[16 * CP];
  quantise<FMT>([&](int i) { return RawPair<T>::value(x[i]); }, two, s, 1.0f / s);
#pragma unroll
  for (int i = 0; i < CP; ++i) {
    const int c = 2 * lane + 128 * i;
    if (c >= dh) continue;
    if (which == 0) {
#pragma unroll
      for (int t = 0; t < 16; ++t) *reinterpret_cast<uint16_t*>(to.block + t * dh + c) = (uint16_t)two[t * CP + i];
    } else {
      u32x4 lo, hi;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        uint32_t l, h;
        words_of(two[(4 * w) * CP + i], two[(4 * w + 1) * CP + i], two[(4 * w + 2) * CP + i], two[(4 * w + 3) * CP + i], l, h);
        lo[w] = l;
        hi[w] = h;
      }
      *reinterpret_cast<u32x4*>(to.block + (size_t)c * 16) = lo;
      *reinterpret_cast<u32x4*>(to.block + (size_t)c * 16 + 16) = hi;
    }
  }
}

// Part of a block, position by position.  What stood in front of the call's positions rounds again where the scale grew; what stands behind them stays
// as it is.
template <int FMT, class T, int CP>
__device__ inline void append_positions(const QuantAppendArgs& a, const Run& run, int head, int which) {
  const int lane = threadIdx.x & 63, dh = a.c.dh;
  const AppendTo<T> to(a, run, head, which);
  if (!to.there) return;
  const float was = run.off ? *to.scale : kQuantScaleFloor;
  // (lanes without channels read the last two)
  auto channel = [&](int i) { return min(2 * lane + 128 * i, dh - 2); };
  uint32_t most = 0;
  for (int t0 = 0; t0 < run.n; t0 += 4) {            // (four positions in flight; behind the last: that one again)
    f32x2 y[4][CP];
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int i = 0; i < CP; ++i) y[e][i] = load_pair<T>(to.src + min(t0 + e, run.n - 1) * to.stride + channel(i));
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int i = 0; i < CP; ++i) most = max(most, max(magnitude(y[e][i][0]), magnitude(y[e][i][1])));
  }
  const float need = scale_for<FMT>(__builtin_bit_cast(float, wave_max(most)));
  const float s = run.off ? scale_max(was, need) : need, inv = 1.0f / s;
  if (lane == 0) *to.scale = s;
  // bytes of channels c, c + 1 of a position are `apart` from those of the next, and `beside` from each other
  const int apart = which ? 1 : dh, beside = which ? 16 : 1;
  const int from = run.off && !(s == was) ? 0 : run.off;
  const int end = run.off + run.n;
  for (int t0 = from; t0 < end; t0 += 4) {
    f32x2 y[4 * CP];
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int i = 0; i < CP; ++i) {
        const int t = min(t0 + e, end - 1);
        if (t < run.off) {
          const uint8_t* p = reinterpret_cast<const uint8_t*>(to.block) + t * apart + channel(i) * (which ? 16 : 1);
          const f32x2 o = byte_pair<FMT>(p[0] | (uint32_t)p[beside] << 8);
          y[e * CP + i] = f32x2{o[0] * was, o[1] * was};
        } else {
          y[e * CP + i] = load_pair<T>(to.src + (t - run.off) * to.stride + channel(i));
        }
      }
    uint32_t two[4 * CP];
    quantise<FMT>([&](int k) { return y[k]; }, two, s, inv);
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int i = 0; i < CP; ++i) {
        const int t = t0 + e, c = 2 * lane + 128 * i;
        uint8_t* p = reinterpret_cast<uint8_t*>(to.block) + t * apart + c * (which ? 16 : 1);
        if (t < end && c < dh) {
          p[0] = (uint8_t)(two[e * CP + i] & 0xff);
          p[beside] = (uint8_t)(two[e * CP + i] >> 8);
        }
      }
  }
}

// 2103 bf16 rows of 32 heads of 128 channels, E4M3: 17 us, 52 MB (3 TB/s; INT8 22).  256 rows of 256 sequences, 8 heads: 6 to 7 us where no scale grows, of which an
// empty launch takes 2 and three dependent loads most of the rest.  Where one does, what stands in front is rounded again, four positions at a time, each four
// behind the stores of those before: with 1, 4, 8, 12, 15 positions in front 7, 10, 14, 18, 20 us (INT8; E4M3, whose scales grow in steps of two, 6 to 18).  In a decode some
// wavefront of a large batch has a growing scale in nearly every call.
template <int FMT, class T, int CP>
__global__ __launch_bounds__(kThreads) void quant_append_kernel(QuantAppendArgs a, int group, int first) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Runs runs(a.r, (first + blockIdx.x) * group, group);
  const int head = blockIdx.y * 2 + (wave >> 1);
  if (head >= a.c.heads) return;
  for (uint64_t left = runs.first; left; left &= left - 1) {
    const Run run = runs.of(__ffsll((unsigned long long)left) - 1);
    if (run.n == 16)
      append_block<FMT, T, CP>(a, run, head, wave & 1);
    else
      append_positions<FMT, T, CP>(a, run, head, wave & 1);
  }
}

template <class T>
__device__ inline void store_pair(T* p, f32x2 x);
template <>
__device__ inline void store_pair<float>(float* p, f32x2 x) { *reinterpret_cast<f32x2*>(p) = x; }
template <>
__device__ inline void store_pair<bf16_t>(bf16_t* p, f32x2 x) { *reinterpret_cast<bf16x2*>(p) = bf16x2{(bf16_t)x[0], (bf16_t)x[1]}; }

template <int FMT, class T, int CP>
__device__ inline void read_run(const QuantReadArgs& a, const Run& run, int head, int which) {
  const int lane = threadIdx.x & 63;
  const int dh = a.c.dh;
  T* dst = reinterpret_cast<T*>(which ? a.v : a.k) + ((size_t)run.m * a.c.heads + head) * dh;
  const size_t stride = (size_t)a.c.heads * dh;
  const int logical = min(run.logical, a.r.max_blocks - 1);
  const int blk = safe_block(a.r.block_tables[(size_t)run.seq * a.r.max_blocks + logical], a.c.num_blocks);
  const size_t unit = (size_t)blk * a.c.heads + head;
  const float s = a.c.scales[unit * 2 + which];
  const int8_t* p = (which ? a.c.v : a.c.k) + unit * 16 * dh;
#pragma unroll
  for (int i = 0; i < CP; ++i) {
    const int c = 2 * lane + 128 * i;
    if (c >= dh) continue;
    if (which == 0) {
      uint32_t two[16];
#pragma unroll
      for (int t = 0; t < 16; ++t) two[t] = t < run.n ? *reinterpret_cast<const uint16_t*>(p + (run.off + t) * dh + c) : 0;
#pragma unroll
      for (int t = 0; t < 16; ++t)
        if (t < run.n) {
          const f32x2 q = byte_pair<FMT>(two[t]);
          store_pair<T>(dst + t * stride + c, f32x2{q[0] * s, q[1] * s});
        }
    } else {
      const u32x4 lo = *reinterpret_cast<const u32x4*>(p + (size_t)c * 16);
      const u32x4 hi = *reinterpret_cast<const u32x4*>(p + (size_t)c * 16 + 16);
#pragma unroll
      for (int t = 0; t < 16; ++t)
        if (t >= run.off && t < run.off + run.n) {
          const int sh = 8 * (t & 3);
          const f32x2 q = byte_pair<FMT>(((lo[t >> 2] >> sh) & 0xff) | (((hi[t >> 2] >> sh) & 0xff) << 8));
          store_pair<T>(dst + (t - run.off) * stride + c, f32x2{q[0] * s, q[1] * s});
        }
    }
  }
}

// Bound by what it writes: the same 2103 rows and what stands in their blocks as floats, 17 MB read and 70 MB written, 17 us.
template <int FMT, class T, int CP>
__global__ __launch_bounds__(kThreads) void quant_read_kernel(QuantReadArgs a, int group, int first) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Runs runs(a.r, (first + blockIdx.x) * group, group);
  const int head = blockIdx.y * 2 + (wave >> 1);
  if (head >= a.c.heads) return;
  for (uint64_t left = runs.first; left; left &= left - 1) read_run<FMT, T, CP>(a, runs.of(__ffsll((unsigned long long)left) - 1), head, wave & 1);
  // rows that read nothing
  for (uint64_t left = __ballot(lane > 0 && lane <= group && runs.base - 1 + lane < a.r.rows && runs.pos < 0); left; left &= left - 1) {
    const size_t m = runs.base + __ffsll((unsigned long long)left) - 2;
    T* dst = reinterpret_cast<T*>(wave & 1 ? a.v : a.k) + (m * a.c.heads + head) * a.c.dh;
    for (int c = 2 * lane; c < a.c.dh; c += 128) store_pair<T>(dst + c, f32x2{0.0f, 0.0f});
  }
}

// ---- eviction ----------------------------------------------------------------------------------------------------
constexpr int kSelThreads = 1024;

// A weight's place in the order: larger weights have larger keys, -0 and 0 the same one, NaN the largest.
__device__ inline uint32_t order_key(float w) {
  if (w != w) return 0xffffffffu;
  const uint32_t u = __builtin_bit_cast(uint32_t, w + 0.0f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Which positions of one (sequence, head) stay.  The key of the last one that stays for its weight is found eight bits at a time (a histogram in
// LDS over the keys that agree so far); another walk numbers what stays in ascending order.  The first kSelKeys keys are held in LDS.  Bound by
// latency: a dozen barriers and what stands between them.  300 positions 9 us, 6000 15 us (four wavefronts instead of sixteen: 8.5 at 300,
// 13 instead of 11 at 2000).
constexpr int kEach = 12, kSelKeys = kEach * kSelThreads;
__global__ __launch_bounds__(kSelThreads) void quant_select_kernel(QuantEvictArgs a) {
  __shared__ uint32_t keys[kSelKeys];
  __shared__ uint32_t hist[256];
  __shared__ uint32_t wave_n[kSelThreads / 64];
  __shared__ uint32_t chosen;
  __shared__ int above;
  const int b = blockIdx.y, head = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int n = max(0, min(a.r.context_lens[b], min(a.max_context, a.r.max_blocks * 16)));
  const size_t row = (size_t)b * a.c.heads + head;
  const float* w = a.weights_in + row * a.pitch_in;
  float* w_out = a.weights_out ? a.weights_out + row * a.pitch_out : nullptr;
  int32_t* kept = a.kept + row * a.keep;
  if (head == 0 && tid == 0) a.out_lens[b] = min(n, a.keep);
  const int old = n > a.keep ? n - a.recent : n;     // positions that are chosen from; the others stay
  int want = n > a.keep ? a.keep - a.recent : n;     // how many of them stay
  uint32_t prefix = 0;
  auto key_of = [&](int i) { return i < kSelKeys ? keys[i] : order_key(w[i]); };
  if (want < old && want > 0) {
#pragma unroll 4
    for (int i = tid; i < min(n, kSelKeys); i += kSelThreads) keys[i] = order_key(w[i]);
    for (int shift = 24; shift >= 0; shift -= 8) {
      for (int i = tid; i < 256; i += kSelThreads) hist[i] = 0;
      __syncthreads();
      for (int i = tid; i < old; i += kSelThreads) {
        const uint32_t k = key_of(i);
        if (shift == 24 || (k >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&hist[(k >> shift) & 255], 1u);
      }
      __syncthreads();
      if (tid < 64) {                                // four bins a lane, the largest first
        uint32_t c[4], sum = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) c[e] = hist[255 - (4 * lane + e)], sum += c[e];
        uint32_t upto = sum;
#pragma unroll
        for (int x = 1; x < 64; x <<= 1) {
          const uint32_t o = __shfl_up(upto, x);
          if (lane >= x) upto += o;
        }
        uint32_t before = upto - sum;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (before < (uint32_t)want && before + c[e] >= (uint32_t)want) {
            chosen = 255 - (4 * lane + e);
            above = (int)before;
          }
          before += c[e];
        }
      }
      __syncthreads();
      prefix |= chosen << shift;
      want -= above;                                 // those with a larger key all stay
    }
  }
  // `want` positions whose key is `prefix` stay, the lowest ones.  A thread numbers kEach neighbours at a time: of those in front, the ones that stay for
  // certain, and of the ties as many as may.
  const bool all = want >= old, none = n > a.keep && a.keep == a.recent;
  int sures = 0, ties = 0;
  for (int i0 = 0; i0 < n; i0 += kSelKeys) {
    const int each = (min(n - i0, kSelKeys) + kSelThreads - 1) / kSelThreads, begin = i0 + tid * each;
    uint32_t mine = 0, held = 0;                     // counts: certain in the low half, ties in the high half; the kinds of this thread's positions
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const int i = begin + e;
      if (e >= each || i >= n) continue;
      uint32_t kind = 1;
      if (!all && i < old) {
        const uint32_t k = none ? 0 : key_of(i);
        kind = none || k < prefix ? 0 : k == prefix ? 0x10000u : 1;
      }
      mine += kind;
      held |= (kind == 1 ? 1u : kind ? 2u : 0u) << (2 * e);
    }
    uint32_t upto = mine;
#pragma unroll
    for (int x = 1; x < 64; x <<= 1) {
      const uint32_t o = __shfl_up(upto, x);
      if (lane >= x) upto += o;
    }
    if (lane == 63) wave_n[wave] = upto;
    __syncthreads();
    uint32_t before = upto - mine, total = 0;
#pragma unroll
    for (int v = 0; v < kSelThreads / 64; ++v) {
      if (v < wave) before += wave_n[v];
      total += wave_n[v];
    }
    int sure_at = sures + (int)(before & 0xffff), tie_at = ties + (int)(before >> 16);
    float x[kEach];
    int to[kEach];
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const uint32_t kind = (held >> (2 * e)) & 3;
      to[e] = kind == 1 || (kind == 2 && tie_at < want) ? sure_at + min(tie_at, all ? 0 : want) : -1;
      sure_at += kind == 1;
      tie_at += kind == 2;
      x[e] = to[e] >= 0 && w_out ? w[begin + e] : 0.0f;
    }
    __syncthreads();                                 // (w_out may be w: everything up to here has been read, and no place is behind its position)
#pragma unroll
    for (int e = 0; e < kEach; ++e)
      if (to[e] >= 0) {
        kept[to[e]] = begin + e;
        if (w_out) w_out[to[e]] = x[e];
      }
    sures += (int)(total & 0xffff);
    ties += (int)(total >> 16);
  }
  for (int i = min(n, a.keep) + tid; i < a.keep; i += kSelThreads) kept[i] = -1;
}

// One block of what stays: 16 positions from up to 16 blocks.  A value needs the scale with which it fits; an INT8 byte that fills its block's range
// needs that block's scale itself, so a block that stays whole keeps its bytes.
// Bound by a chain of loads (kept positions, block ids, scales, bytes) at six wavefronts a SIMD, and by V: a channel's 16 positions share a line, so
// every block that anything stays of is read whole.  16 sequences of 700 to 6000 positions cut to 1000, 8 heads of 128: 33 us for 33 MB kept
// (INT8 40; V byte by byte: 50; with the values as floats in registers, three wavefronts a SIMD: 54; a maximum of each position instead of all: 37).
template <int FMT, int CP>
__global__ __launch_bounds__(kThreads, CP == 1 ? 6 : 3) void quant_build_kernel(QuantEvictArgs a, int slots) {
  const int lane = threadIdx.x & 63;
  const int task = blockIdx.x * (kThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int b = blockIdx.y;
  if (task >= slots * 2 * a.c.heads) return;
  const int which = task & 1, head = (task >> 1) % a.c.heads, slot = (task >> 1) / a.c.heads;
  const int dh = a.c.dh;
  const size_t row = (size_t)b * a.c.heads + head;
  const int mine = slot * 16 + (lane & 15);
  const int n = a.r.context_lens[b];
  const int pos = mine < a.keep ? a.kept[row * a.keep + mine] : -1;   // (-1 behind what stays)
  if (lane_value(pos, 0) < 0 || (!a.dst_tables && n <= a.keep)) return;
  int blk = 0;
  float was = kQuantScaleFloor;
  if (pos >= 0) {
    blk = safe_block(a.r.block_tables[(size_t)b * a.r.max_blocks + (pos >> 4)], a.c.num_blocks);
    was = a.c.scales[((size_t)blk * a.c.heads + head) * 2 + which];
  }
  uint32_t two[16][CP];                              // a position's bytes of channels c and c + 1
  if (which == 0) {
#pragma unroll
    for (int t = 0; t < 16; ++t) {
      const int pt = lane_value(pos, t);
      const int8_t* p = a.c.k + ((size_t)lane_value(blk, t) * a.c.heads + head) * 16 * dh + (pt & 15) * dh;
#pragma unroll
      for (int i = 0; i < CP; ++i) {
        const int c = 2 * lane + 128 * i;
        two[t][i] = pt >= 0 && c < dh ? *reinterpret_cast<const uint16_t*>(p + c) : 0;
      }
    }
  } else {
    // a channel's 16 positions are one load: a block that several of ours come from is read once, the next one while this one is taken apart
    const int before = __shfl_up(pos, 1);
    const uint32_t begins = (uint32_t)__ballot(lane < 16 && pos >= 0 && (lane == 0 || (pos >> 4) != (before >> 4)));
    u32x4 now[CP][2], next[CP][2];
    auto load = [&](uint32_t left, u32x4 (&to)[CP][2]) {
      const int8_t* p = a.c.v + ((size_t)lane_value(blk, left ? __ffs(left) - 1 : 0) * a.c.heads + head) * 16 * dh;
#pragma unroll
      for (int i = 0; i < CP; ++i) {
        const int c = 2 * lane + 128 * i;
#pragma unroll
        for (int e = 0; e < 2; ++e) to[i][e] = *reinterpret_cast<const u32x4*>(p + (size_t)(c < dh ? c + e : 0) * 16);
      }
    };
    load(begins, next);
#pragma unroll
    for (int t = 0; t < 16; ++t) {
      if (begins >> t & 1) {
#pragma unroll
        for (int i = 0; i < CP; ++i) now[i][0] = next[i][0], now[i][1] = next[i][1];
        load(begins >> (t + 1) << (t + 1), next);
      }
      const int pt = lane_value(pos, t), word = (pt >> 2) & 3, sh = 8 * (pt & 3);
#pragma unroll
      for (int i = 0; i < CP; ++i) {
        uint32_t lo = now[i][0][0], hi = now[i][1][0];
#pragma unroll
        for (int w = 1; w < 4; ++w)
          if (word == w) lo = now[i][0][w], hi = now[i][1][w];
        two[t][i] = pt >= 0 && 2 * lane + 128 * i < dh ? ((lo >> sh) & 0xff) | (((hi >> sh) & 0xff) << 8) : 0;
      }
    }
  }
  // The largest value decides: scales grow with it.  (Magnitudes' bits are ordered as integers, NaN behind all of them.)
  uint32_t most = 0, filled = 0;
#pragma unroll
  for (int t = 0; t < 16; ++t) {
    const float wt = lane_value(was, t);
#pragma unroll
    for (int i = 0; i < CP; ++i) {
      const f32x2 q = byte_pair<FMT>(two[t][i]);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const uint32_t value = magnitude(q[e] * wt);
        const bool fills = FMT == EE_QUANT_INT8 && fabsf(q[e]) >= 127.0f;
        most = max(most, fills ? 0u : value);
        if (FMT == EE_QUANT_INT8) filled = max(filled, fills ? magnitude(wt) : 0u);
      }
    }
  }
  float need = scale_for<FMT>(__builtin_bit_cast(float, wave_max(most)));
  if constexpr (FMT == EE_QUANT_INT8) need = scale_max(need, __builtin_bit_cast(float, wave_max(filled)));
  const float s = need, inv = 1.0f / s;
  int8_t* out;
  float* sp;
  if (a.dst_tables) {
    const int to = a.dst_tables[(size_t)b * a.dst_max_blocks + slot];
    if ((unsigned)to >= (unsigned)a.c.num_blocks) return;
    const size_t unit = (size_t)to * a.c.heads + head;
    out = (which ? a.c.v : a.c.k) + unit * 16 * dh;
    sp = a.c.scales + unit * 2 + which;
  } else {
    const size_t unit = (row * slots + slot) * 2 + which;
    out = a.images + unit * 16 * dh;
    sp = a.image_scales + unit;
  }
  if (lane == 0) *sp = s;
  uint32_t again[16 * CP];
  quantise<FMT>([&](int k) {
    const f32x2 q = byte_pair<FMT>(two[k / CP][k % CP]);
    const float wt = lane_value(was, k / CP);
    return f32x2{q[0] * wt, q[1] * wt};
  }, again, s, inv);
#pragma unroll
  for (int i = 0; i < CP; ++i) {
    const int c = 2 * lane + 128 * i;
    if (c >= dh) continue;
    if (which == 0) {
#pragma unroll
      for (int t = 0; t < 16; ++t) *reinterpret_cast<uint16_t*>(out + t * dh + c) = (uint16_t)again[t * CP + i];
    } else {
      u32x4 lo, hi;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        uint32_t l, h;
        words_of(again[(4 * w) * CP + i], again[(4 * w + 1) * CP + i], again[(4 * w + 2) * CP + i], again[(4 * w + 3) * CP + i], l, h);
        lo[w] = l;
        hi[w] = h;
      }
      *reinterpret_cast<u32x4*>(out + (size_t)c * 16) = lo;
      *reinterpret_cast<u32x4*>(out + (size_t)c * 16 + 16) = hi;
    }
  }
}

// In place: the finished blocks go where the sequence's first blocks are.
__global__ __launch_bounds__(kThreads) void quant_place_kernel(QuantEvictArgs a, int slots) {
  const int lane = threadIdx.x & 63;
  const int task = blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6);
  const int b = blockIdx.y;
  if (task >= slots * 2 * a.c.heads) return;
  const int which = task & 1, head = (task >> 1) % a.c.heads, slot = (task >> 1) / a.c.heads;
  const int n = max(0, min(a.r.context_lens[b], min(a.max_context, a.r.max_blocks * 16)));
  if (n <= a.keep || slot * 16 >= a.keep) return;
  const int to = a.r.block_tables[(size_t)b * a.r.max_blocks + slot];
  if ((unsigned)to >= (unsigned)a.c.num_blocks) return;
  const size_t from = (((size_t)b * a.c.heads + head) * slots + slot) * 2 + which, unit = (size_t)to * a.c.heads + head;
  const int dh = a.c.dh;
  const u32x4* src = reinterpret_cast<const u32x4*>(a.images + from * 16 * dh);
  u32x4* dst = reinterpret_cast<u32x4*>((which ? a.c.v : a.c.k) + unit * 16 * dh);
  for (int i = lane; i < dh; i += 64) dst[i] = src[i];
  if (lane == 0) a.c.scales[unit * 2 + which] = a.image_scales[from];
}

// A launch has fewer than 2^32 threads a dimension.
constexpr int kLaunchGroups = (1 << 24) - 1;
template <class F>
void for_groups(const QuantRows& r, int heads, F&& launch) {
  const int group = r.row_table ? kGroup : 1, all = (int)(((int64_t)r.rows + group - 1) / group);
  for (int first = 0; first < all; first += kLaunchGroups) launch(dim3(min(all - first, kLaunchGroups), (heads + 1) / 2), group, first);
}

int groups(int64_t tasks) { return (int)((tasks + kThreads / 64 - 1) / (kThreads / 64)); }

}  // namespace

template <int FMT, class T>
static void append_as(const QuantAppendArgs& a, hipStream_t st) {
  if (a.c.dh <= 128)
    for_groups(a.r, a.c.heads, [&](dim3 grid, int group, int first) { quant_append_kernel<FMT, T, 1><<<grid, kThreads, 0, st>>>(a, group, first); });
  else
    for_groups(a.r, a.c.heads, [&](dim3 grid, int group, int first) { quant_append_kernel<FMT, T, 2><<<grid, kThreads, 0, st>>>(a, group, first); });
}
void launch_quant_append(const QuantAppendArgs& a, int dtype, hipStream_t st) {
  if (a.c.format == EE_QUANT_INT8)
    dtype == EE_BF16 ? append_as<EE_QUANT_INT8, bf16_t>(a, st) : append_as<EE_QUANT_INT8, float>(a, st);
  else
    dtype == EE_BF16 ? append_as<EE_QUANT_E4M3, bf16_t>(a, st) : append_as<EE_QUANT_E4M3, float>(a, st);
}

template <int FMT, class T>
static void read_as(const QuantReadArgs& a, hipStream_t st) {
  if (a.c.dh <= 128)
    for_groups(a.r, a.c.heads, [&](dim3 grid, int group, int first) { quant_read_kernel<FMT, T, 1><<<grid, kThreads, 0, st>>>(a, group, first); });
  else
    for_groups(a.r, a.c.heads, [&](dim3 grid, int group, int first) { quant_read_kernel<FMT, T, 2><<<grid, kThreads, 0, st>>>(a, group, first); });
}
void launch_quant_read(const QuantReadArgs& a, int dtype, hipStream_t st) {
  if (a.c.format == EE_QUANT_INT8)
    dtype == EE_BF16 ? read_as<EE_QUANT_INT8, bf16_t>(a, st) : read_as<EE_QUANT_INT8, float>(a, st);
  else
    dtype == EE_BF16 ? read_as<EE_QUANT_E4M3, bf16_t>(a, st) : read_as<EE_QUANT_E4M3, float>(a, st);
}

template <int FMT>
static void build_as(const QuantEvictArgs& a, int slots, dim3 grid, hipStream_t st) {
  if (a.c.dh <= 128)
    quant_build_kernel<FMT, 1><<<grid, kThreads, 0, st>>>(a, slots);
  else
    quant_build_kernel<FMT, 2><<<grid, kThreads, 0, st>>>(a, slots);
}
void launch_quant_evict(const QuantEvictArgs& a, hipStream_t st) {
  quant_select_kernel<<<dim3(a.c.heads, a.r.rows), kSelThreads, 0, st>>>(a);
  const int slots = (min(a.keep, a.max_context) + 15) / 16;
  const dim3 grid(groups((int64_t)slots * a.c.heads * 2), a.r.rows);
  a.c.format == EE_QUANT_INT8 ? build_as<EE_QUANT_INT8>(a, slots, grid, st) : build_as<EE_QUANT_E4M3>(a, slots, grid, st);
  if (!a.dst_tables) quant_place_kernel<<<grid, kThreads, 0, st>>>(a, slots);
}

}  // namespace ee
