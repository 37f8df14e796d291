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

// The smallest scale with which `largest` fits; NaN for an infinity or NaN (a magnitude's bits are ordered as integers).
template <int FMT>
__device__ inline float scale_for(float largest) {
  if (!(largest < INFINITY)) return __builtin_nanf("");
  if constexpr (FMT == EE_QUANT_INT8) {
    return fmaxf(largest / 127.0f, kQuantScaleFloor);
  } else {
    int e;
    const float m = frexpf(largest, &e);             // 448 = 0.875 * 2^9
    return largest > 0.0f ? ldexpf(1.0f, max(e - 9 + (m > 0.875f), -126)) : kQuantScaleFloor;
  }
}

// The bytes nearest to x / s, ties to even.  INT8: x / s is estimated by a product with 1/s and then set right by the exact remainder x - q s
// (one fma: |remainder| <= s and a multiple of the smaller operand's last place, so it has 24 bits), because the quotient
// rounded to float may land on a tie that x / s is not on.  E4M3: s is a power of two, the product is exact and the conversion rounds once.
template <int FMT>
__device__ inline uint32_t quantise_pair(f32x2 x, float s, float inv) {
  if (s != s) return 0;
  if constexpr (FMT == EE_QUANT_INT8) {
    uint32_t r = 0;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      float q = rintf(x[e] * inv);
      const float rem = fmaf(-q, s, x[e]), twice = 2.0f * fabsf(rem);
      if (twice > s || (twice == s && ((int)q & 1))) q += copysignf(1.0f, rem);
      r |= (uint32_t)((int)fminf(fmaxf(q, -127.0f), 127.0f) & 0xff) << (8 * e);
    }
    return r;
  } else {
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[0] * inv, x[1] * inv, 0, false) & 0xffff;
  }
}

// The larger of two scales; NaN if either is.
__device__ inline float scale_max(float a, float b) { return a != a || b != b ? __builtin_nanf("") : fmaxf(a, b); }

// Rows that go into (or come from) one block are taken together: a run is rows at consecutive positions of one block.  A workgroup has kGroup
// rows (where every row is a sequence of its own, two) of one head and takes the runs that begin among them; wavefronts 0 and 2 K's, 1 and 3 V's.
constexpr int kGroup = 8, kApart = 2;
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
    seq = there ? quant_seq(r, at) : -1;
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

template <int FMT, class T, int CP>
__device__ inline void append_run(const QuantAppendArgs& a, const Run& run, int head, int which) {
  const int lane = threadIdx.x & 63;
  if (run.logical >= a.r.max_blocks) return;
  const int blk = a.r.block_tables[(size_t)run.seq * a.r.max_blocks + run.logical];
  if ((unsigned)blk >= (unsigned)a.c.num_blocks) return;
  const int dh = a.c.dh;
  const T* src = reinterpret_cast<const T*>(which ? a.v : a.k) + (size_t)run.m * (which ? a.v_stride : a.k_stride) + (size_t)head * dh;
  const int64_t stride = which ? a.v_stride : a.k_stride;
  const size_t unit = (size_t)blk * a.c.heads + head;
  float* sp = a.c.scales + unit * 2 + which;
  const float was = run.off ? *sp : kQuantScaleFloor;

  const int end = run.off + run.n;
  f32x2 x[16][CP];                                   // by place in the block
  uint32_t most = 0;
#pragma unroll
  for (int t = 0; t < 16; ++t)
#pragma unroll
    for (int i = 0; i < CP; ++i) {
      const int c = 2 * lane + 128 * i;
      x[t][i] = f32x2{0.0f, 0.0f};
      if (t >= run.off && t < end && c < dh) x[t][i] = load_pair<T>(src + (t - run.off) * stride + c);
    }
#pragma unroll
  for (int t = 0; t < 16; ++t)
#pragma unroll
    for (int i = 0; i < CP; ++i) most = max(most, max(magnitude(x[t][i][0]), magnitude(x[t][i][1])));
  const float need = scale_for<FMT>(__builtin_bit_cast(float, wave_max(most)));
  const float s = run.off ? scale_max(was, need) : need, inv = 1.0f / s;
  const bool grew = run.off && !(s == was);
  if (lane == 0) *sp = s;

  // what stood in front of the call's positions rounds again where the scale grew
  if (which == 0) {
    int8_t* kp = a.c.k + unit * 16 * dh;
#pragma unroll
    for (int t = 0; t < 16; ++t)
#pragma unroll
      for (int i = 0; i < CP; ++i) {
        const int c = 2 * lane + 128 * i;
        uint16_t* p = reinterpret_cast<uint16_t*>(kp + t * dh + c);
        f32x2 y = x[t][i];
        if (c >= dh || t >= end || (t < run.off && !grew)) continue;
        if (t < run.off) {
          y = byte_pair<FMT>(*p);
          y = f32x2{y[0] * was, y[1] * was};
        }
        *p = (uint16_t)quantise_pair<FMT>(y, s, inv);
      }
    return;
  }
  int8_t* vp = a.c.v + unit * 16 * dh;
#pragma unroll
  for (int i = 0; i < CP; ++i) {
    const int c = 2 * lane + 128 * i;
    if (c >= dh) continue;
    int8_t* line = vp + (size_t)c * 16;              // channels c and c + 1: 32 bytes
    u32x4 lo{}, hi{};
    if (run.n < 16) {                                // (what stands behind the call's positions stays as it is)
      lo = *reinterpret_cast<const u32x4*>(line);
      hi = *reinterpret_cast<const u32x4*>(line + 16);
    }
#pragma unroll
    for (int t = 0; t < 16; ++t) {
      const int sh = 8 * (t & 3);
      f32x2 y = x[t][i];
      if (t >= end || (t < run.off && !grew)) continue;
      if (t < run.off) {
        y = byte_pair<FMT>(((lo[t >> 2] >> sh) & 0xff) | (((hi[t >> 2] >> sh) & 0xff) << 8));
        y = f32x2{y[0] * was, y[1] * was};
      }
      const uint32_t q = quantise_pair<FMT>(y, s, inv);
      lo[t >> 2] = (lo[t >> 2] & ~(0xffu << sh)) | ((q & 0xff) << sh);
      hi[t >> 2] = (hi[t >> 2] & ~(0xffu << sh)) | ((q >> 8) << sh);
    }
    *reinterpret_cast<u32x4*>(line) = lo;
    *reinterpret_cast<u32x4*>(line + 16) = hi;
  }
}

template <int FMT, class T, int CP>
__global__ __launch_bounds__(kThreads) void quant_append_kernel(QuantAppendArgs a, int group) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Runs runs(a.r, blockIdx.x * group, group);
  int i = 0;
  for (uint64_t left = runs.first; left; left &= left - 1, ++i)
    if ((i & 1) == (wave >> 1)) append_run<FMT, T, CP>(a, runs.of(__ffsll((unsigned long long)left) - 1), blockIdx.y, wave & 1);
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

template <int FMT, class T, int CP>
__global__ __launch_bounds__(kThreads) void quant_read_kernel(QuantReadArgs a, int group) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Runs runs(a.r, blockIdx.x * group, group);
  int i = 0;
  for (uint64_t left = runs.first; left; left &= left - 1, ++i)
    if ((i & 1) == (wave >> 1)) read_run<FMT, T, CP>(a, runs.of(__ffsll((unsigned long long)left) - 1), blockIdx.y, wave & 1);
  // rows that read nothing
  for (uint64_t left = __ballot(lane > 0 && lane <= group && runs.base - 1 + lane < a.r.rows && runs.pos < 0); left; left &= left - 1) {
    const size_t m = runs.base + __ffsll((unsigned long long)left) - 2;
    T* dst = reinterpret_cast<T*>(wave & 1 ? a.v : a.k) + (m * a.c.heads + blockIdx.y) * a.c.dh;
    for (int c = 2 * lane; c < a.c.dh && wave < 2; c += 128) store_pair<T>(dst + c, f32x2{0.0f, 0.0f});
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
// LDS over the keys that agree so far); a second walk numbers what stays in ascending order.
__global__ __launch_bounds__(kSelThreads) void quant_select_kernel(QuantEvictArgs a) {
  __shared__ uint32_t hist[256];
  __shared__ int wave_n[2][kSelThreads / 64];
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
  if (want < old && want > 0) {
    for (int shift = 24; shift >= 0; shift -= 8) {
      for (int i = tid; i < 256; i += kSelThreads) hist[i] = 0;
      __syncthreads();
      for (int i = tid; i < old; i += kSelThreads) {
        const uint32_t k = order_key(w[i]);
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
  // `want` positions whose key is `prefix` stay, the lowest ones
  const bool all = want >= old, none = n > a.keep && a.keep == a.recent;
  int at = 0, ties = 0;
  for (int i0 = 0; i0 < n; i0 += kSelThreads) {
    const int i = i0 + tid;
    const float x = i < n ? w[i] : 0.0f;
    const uint32_t k = order_key(x);
    const bool sure = i < n && (all || i >= old || (!none && k > prefix));
    const bool tie = i < old && !all && !none && k == prefix;
    const uint64_t mine = (1ull << lane) - 1;
    const uint64_t t = __ballot(tie);
    if (lane == 0) wave_n[0][wave] = __popcll(t);
    __syncthreads();
    int t0 = ties, t_all = ties;
    for (int v = 0; v < kSelThreads / 64; ++v) {
      if (v < wave) t0 += wave_n[0][v];
      t_all += wave_n[0][v];
    }
    const bool stays = sure || (tie && t0 + __popcll(t & mine) < want);
    const uint64_t s = __ballot(stays);
    if (lane == 0) wave_n[1][wave] = __popcll(s);
    __syncthreads();
    int s0 = at, s_all = at;
    for (int v = 0; v < kSelThreads / 64; ++v) {
      if (v < wave) s0 += wave_n[1][v];
      s_all += wave_n[1][v];
    }
    if (stays) {
      const int to = s0 + __popcll(s & mine);        // <= i, and everything up to i0 + 1023 has been read
      kept[to] = i;
      if (w_out) w_out[to] = x;
    }
    at = s_all;
    ties = t_all;
  }
  for (int i = at + tid; i < a.keep; i += kSelThreads) kept[i] = -1;
}

// One block of what stays: 16 positions from up to 16 blocks.  A position needs the scale with which its largest byte fits; one that fills its
// block's range needs that block's scale itself, so a block that stays whole keeps its bytes.
template <int FMT, int CP>
__global__ __launch_bounds__(kThreads) void quant_build_kernel(QuantEvictArgs a, int slots) {
  const int lane = threadIdx.x & 63;
  const int task = blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6);
  const int b = blockIdx.y;
  if (task >= slots * 2 * a.c.heads) return;
  const int which = task & 1, head = (task >> 1) % a.c.heads, slot = (task >> 1) / a.c.heads;
  const int dh = a.c.dh;
  const int n = max(0, min(a.r.context_lens[b], min(a.max_context, a.r.max_blocks * 16)));
  const int stay = min(n, a.keep);
  if (slot * 16 >= stay || (!a.dst_tables && n <= a.keep)) return;
  const size_t row = (size_t)b * a.c.heads + head;
  const int mine = slot * 16 + (lane & 15);
  const int pos = mine < stay ? a.kept[row * a.keep + mine] : -1;
  int blk = -1;
  float was = kQuantScaleFloor;
  if (pos >= 0) {
    blk = safe_block(a.r.block_tables[(size_t)b * a.r.max_blocks + (pos >> 4)], a.c.num_blocks);
    was = a.c.scales[((size_t)blk * a.c.heads + head) * 2 + which];
  }
  f32x2 x[16][CP];
  float need = kQuantScaleFloor;
#pragma unroll
  for (int t = 0; t < 16; ++t) {
    const int pt = lane_value(pos, t), bt = lane_value(blk, t);
    const int8_t* p = (which ? a.c.v : a.c.k) + ((size_t)max(bt, 0) * a.c.heads + head) * 16 * dh;
#pragma unroll
    for (int i = 0; i < CP; ++i) {
      const int c = 2 * lane + 128 * i;
      uint32_t two = 0;
      if (pt >= 0 && c < dh) {
        if (which == 0) {
          two = *reinterpret_cast<const uint16_t*>(p + (pt & 15) * dh + c);
        } else {
          const uint8_t* line = reinterpret_cast<const uint8_t*>(p) + (size_t)c * 16 + (pt & 15);
          two = line[0] | ((uint32_t)line[16] << 8);
        }
      }
      x[t][i] = byte_pair<FMT>(two);
    }
  }
#pragma unroll
  for (int t = 0; t < 16; ++t) {
    const float wt = lane_value(was, t);
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < CP; ++i) {
      most = max(most, max(magnitude(x[t][i][0]), magnitude(x[t][i][1])));
      x[t][i] = f32x2{x[t][i][0] * wt, x[t][i][1] * wt};
    }
    const float top = __builtin_bit_cast(float, wave_max(most));
    float nt = scale_for<FMT>(top * wt);
    if (FMT == EE_QUANT_INT8 && top >= 127.0f) nt = wt;
    if (lane_value(pos, t) >= 0) need = scale_max(need, nt);
  }
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
#pragma unroll
  for (int i = 0; i < CP; ++i) {
    const int c = 2 * lane + 128 * i;
    if (c >= dh) continue;
    if (which == 0) {
#pragma unroll
      for (int t = 0; t < 16; ++t) *reinterpret_cast<uint16_t*>(out + t * dh + c) = (uint16_t)quantise_pair<FMT>(x[t][i], s, inv);
    } else {
      u32x4 lo{}, hi{};
#pragma unroll
      for (int t = 0; t < 16; ++t) {
        const uint32_t q = quantise_pair<FMT>(x[t][i], s, inv);
        lo[t >> 2] |= (q & 0xff) << (8 * (t & 3));
        hi[t >> 2] |= (q >> 8) << (8 * (t & 3));
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

int groups(int64_t tasks) { return (int)((tasks + kThreads / 64 - 1) / (kThreads / 64)); }

}  // namespace

template <int FMT, class T>
static void append_as(const QuantAppendArgs& a, hipStream_t st) {
  const int group = a.r.row_table ? kGroup : kApart;
  const dim3 grid((a.r.rows + group - 1) / group, a.c.heads);
  if (a.c.dh <= 128)
    quant_append_kernel<FMT, T, 1><<<grid, kThreads, 0, st>>>(a, group);
  else
    quant_append_kernel<FMT, T, 2><<<grid, kThreads, 0, st>>>(a, group);
}
void launch_quant_append(const QuantAppendArgs& a, int dtype, hipStream_t st) {
  if (a.c.format == EE_QUANT_INT8)
    dtype == EE_BF16 ? append_as<EE_QUANT_INT8, bf16_t>(a, st) : append_as<EE_QUANT_INT8, float>(a, st);
  else
    dtype == EE_BF16 ? append_as<EE_QUANT_E4M3, bf16_t>(a, st) : append_as<EE_QUANT_E4M3, float>(a, st);
}

template <int FMT, class T>
static void read_as(const QuantReadArgs& a, hipStream_t st) {
  const int group = a.r.row_table ? kGroup : kApart;
  const dim3 grid((a.r.rows + group - 1) / group, a.c.heads);
  if (a.c.dh <= 128)
    quant_read_kernel<FMT, T, 1><<<grid, kThreads, 0, st>>>(a, group);
  else
    quant_read_kernel<FMT, T, 2><<<grid, kThreads, 0, st>>>(a, group);
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
