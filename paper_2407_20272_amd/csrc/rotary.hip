// Rotary embedding on its own: query and key rows of any stride, either pair layout, part of a head, frequencies the caller hands over.
#include "quant.h"

namespace ee {

namespace {

constexpr int kThreads = 256;
constexpr int kTasks = 1024;   // pieces of a workgroup
constexpr int kMaxRows = 8;    // rows of a workgroup

__global__ void rotary_frequencies_kernel(ee_rotary_desc d, double* freqs) {
  const int j = blockIdx.x * blockDim.x + threadIdx.x;
  if (j >= d.rotary_dim / 2) return;
  double f = pow(d.theta, -2.0 * j / d.rotary_dim);
  if (d.scaling == EE_ROTARY_LINEAR) f /= d.factor;
  if (d.scaling == EE_ROTARY_TURNS) {
    const double turns = d.original_context * f / (2.0 * M_PI);
    const double w = fmin(1.0, fmax(0.0, (turns - d.turns_low) / (d.turns_high - d.turns_low)));
    f *= w + (1.0 - w) / d.factor;
  }
  freqs[j] = f;
}

__device__ inline float to_float(float x) { return x; }
__device__ inline float to_float(bf16_t x) { return (float)x; }

// One product rounded, one fused: the same bits in every variant.
__device__ inline float turned_a(float a, float b, float2 w) { return fmaf(a, w.x, -(b * w.y)); }
__device__ inline float turned_b(float a, float b, float2 w) { return fmaf(a, w.y, b * w.x); }

template <class T, int N>
struct alignas(sizeof(T) * N) Piece {
  T v[N];
};

// A head is rotated in pieces of VEC elements (16 bytes, or single elements where sizes, strides or addresses do not allow more): with HALF a
// piece and its partner rotary_dim/2 further on, else a piece of VEC/2 neighbouring pairs (one pair where VEC is 1).
// The workgroup's rows share the tables of (cos, sin): their double products, reductions and sincospi are done once a row and pair, not once a
// head.  Bound by memory: it reads and writes every element once.  4096 rows of 40 heads of 128 bf16 channels, 84 MB: 15 us, 5.6 TB/s (a large copy
// makes 5.1; the 84 MB stay in the last-level cache between calls); one row of 64 heads 2.9 us, an empty launch 2.  1001 float rows with 48 of 80 channels interleaved, 16 MB:
// 6.9 us, twice what memory takes: a thread's loads wait for the stores of its piece before (in and out may be one buffer).  Where halves are no whole number of 16 bytes
// everything goes element by element.
template <class T, int LAYOUT, int VEC>
__global__ __launch_bounds__(kThreads) void rotary_kernel(RotaryArgs a, int rows_per_wg, int tasks_per_row, int tasks_per_wg) {
  extern __shared__ float2 turn[];   // [rows_per_wg][rotary_dim / 2]
  const int pairs = a.rotary_dim / 2;
  const int m0 = blockIdx.x * rows_per_wg;
  const int n_rows = min(rows_per_wg, a.rows - m0);
  for (int i = threadIdx.x; i < n_rows * pairs; i += kThreads) {
    const int m = i / pairs, j = i - m * pairs;
    // whole turns go before the angle leaves double: at position 10^5 a float angle has no fraction of a degree left
    double t = (double)a.positions[m0 + m] * a.freqs[j] * 0.15915494309189534;
    t -= rint(t);
    float s, c;
    sincospif(2.0f * (float)t, &s, &c);
    turn[i] = make_float2(a.amplitude * c, a.sign * a.amplitude * s);
  }
  __syncthreads();
  constexpr int STEP = LAYOUT == EE_ROTARY_HALF ? VEC : (VEC == 1 ? 2 : VEC);   // channels (of a half) that a rotated piece covers
  const int span = LAYOUT == EE_ROTARY_HALF ? pairs : a.rotary_dim;
  const int turned = span / STEP, pieces = turned + (a.head_dim - a.rotary_dim) / VEC;
  const int first = blockIdx.y * tasks_per_wg, last = min(first + tasks_per_wg, tasks_per_row);
  const int n = last - first;
  for (int i = threadIdx.x; i < n * n_rows; i += kThreads) {
    const int m = i / n, task = first + (i - m * n);
    const int head = task / pieces, p = task - head * pieces;
    const bool is_q = head < a.q.n_heads;
    const RotaryRows& r = is_q ? a.q : a.k;
    const size_t at = (size_t)(is_q ? head : head - a.q.n_heads) * a.head_dim;
    const T* in = reinterpret_cast<const T*>(r.in) + (size_t)(m0 + m) * r.in_stride + at;
    T* out = reinterpret_cast<T*>(r.out) + (size_t)(m0 + m) * r.out_stride + at;
    const float2* cs = turn + m * pairs;
    typedef Piece<T, VEC> P;
    if (p >= turned) {
      const int c = a.rotary_dim + (p - turned) * VEC;
      if (in != out) *reinterpret_cast<P*>(out + c) = *reinterpret_cast<const P*>(in + c);
    } else if constexpr (LAYOUT == EE_ROTARY_HALF) {
      const int c = p * VEC;
      P x = *reinterpret_cast<const P*>(in + c), y = *reinterpret_cast<const P*>(in + c + pairs);
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const float2 w = cs[c + e];
        const float u = to_float(x.v[e]), v = to_float(y.v[e]);
        x.v[e] = (T)turned_a(u, v, w);
        y.v[e] = (T)turned_b(u, v, w);
      }
      *reinterpret_cast<P*>(out + c) = x;
      *reinterpret_cast<P*>(out + c + pairs) = y;
    } else if constexpr (VEC == 1) {
      const float2 w = cs[p];
      const float u = to_float(in[2 * p]), v = to_float(in[2 * p + 1]);
      out[2 * p] = (T)turned_a(u, v, w);
      out[2 * p + 1] = (T)turned_b(u, v, w);
    } else {
      const int c = p * VEC;
      P x = *reinterpret_cast<const P*>(in + c);
#pragma unroll
      for (int e = 0; e < VEC; e += 2) {
        const float2 w = cs[(c + e) / 2];
        const float u = to_float(x.v[e]), v = to_float(x.v[e + 1]);
        x.v[e] = (T)turned_a(u, v, w);
        x.v[e + 1] = (T)turned_b(u, v, w);
      }
      *reinterpret_cast<P*>(out + c) = x;
    }
  }
}

template <class T, int LAYOUT, int VEC>
void launch(const RotaryArgs& a, hipStream_t st) {
  const int span = LAYOUT == EE_ROTARY_HALF ? a.rotary_dim / 2 : a.rotary_dim;
  const int step = LAYOUT == EE_ROTARY_HALF ? VEC : (VEC == 1 ? 2 : VEC);
  const int tasks = (a.q.n_heads + a.k.n_heads) * (span / step + (a.head_dim - a.rotary_dim) / VEC);
  int rows = kTasks / tasks;   // rows of few pieces share a workgroup
  rows = rows < 1 ? 1 : rows > kMaxRows ? kMaxRows : rows;
  // A launch has at most 65535 workgroups in the second dimension, and fewer than 2^32 threads in the first.
  const int each = tasks > kTasks * 65535 ? (tasks + 65534) / 65535 : kTasks;
  const int64_t slice = (int64_t)((1 << 24) - 1) * rows;
  for (int64_t m = 0; m < a.rows; m += slice) {
    RotaryArgs part = a;
    part.positions += m;
    part.rows = (int)(a.rows - m < slice ? a.rows - m : slice);
    for (RotaryRows* r : {&part.q, &part.k}) {
      r->in = reinterpret_cast<const T*>(r->in) + m * r->in_stride;
      r->out = reinterpret_cast<T*>(r->out) + m * r->out_stride;
    }
    const dim3 grid((int)(((int64_t)part.rows + rows - 1) / rows), (tasks + each - 1) / each);
    rotary_kernel<T, LAYOUT, VEC><<<grid, kThreads, (size_t)rows * (a.rotary_dim / 2) * sizeof(float2), st>>>(part, rows, tasks, each);
  }
}

bool aligned(const RotaryRows& r, int size, int vec) {
  if (!r.n_heads) return true;
  const uintptr_t addr = reinterpret_cast<uintptr_t>(r.in) | reinterpret_cast<uintptr_t>(r.out);
  return (addr & 15) == 0 && r.in_stride % vec == 0 && r.out_stride % vec == 0 && size * vec == 16;
}

template <class T, int LAYOUT>
void pick(const RotaryArgs& a, hipStream_t st) {
  constexpr int VEC = 16 / sizeof(T);
  const int span = LAYOUT == EE_ROTARY_HALF ? a.rotary_dim / 2 : a.rotary_dim;
  if (a.head_dim % VEC == 0 && span % VEC == 0 && a.rotary_dim % VEC == 0 && aligned(a.q, sizeof(T), VEC) && aligned(a.k, sizeof(T), VEC))
    launch<T, LAYOUT, VEC>(a, st);
  else
    launch<T, LAYOUT, 1>(a, st);
}

}  // namespace

void launch_rotary_frequencies(const ee_rotary_desc& d, double* freqs, hipStream_t st) {
  rotary_frequencies_kernel<<<(d.rotary_dim / 2 + 63) / 64, 64, 0, st>>>(d, freqs);
}

void launch_rotary(const RotaryArgs& a, int dtype, int layout, hipStream_t st) {
  if (dtype == EE_BF16)
    layout == EE_ROTARY_HALF ? pick<bf16_t, EE_ROTARY_HALF>(a, st) : pick<bf16_t, EE_ROTARY_INTERLEAVED>(a, st);
  else
    layout == EE_ROTARY_HALF ? pick<float, EE_ROTARY_HALF>(a, st) : pick<float, EE_ROTARY_INTERLEAVED>(a, st);
}

}  // namespace ee
