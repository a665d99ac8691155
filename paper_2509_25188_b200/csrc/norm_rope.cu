// Norms of queries and keys for each head, with the rotation by position in the same pass:
//     y = x g / sqrt(mean(x^2) + eps)        over the dh values of a (row, head)
//     (y_i, y_{i + dh/2}) turned by the angle position * theta^(-2i/dh)
// in fp32 between the load and the one rounding at the store; the angle is reduced in 64 bits, so that far positions keep their phase.
//
// Bound by memory: every value is read and written once.  A block takes R rows: their sines and cosines (R dh/2 of them, for all
// heads) go to shared memory while the first rows are on their way.  A thread holds eight values of a head's first half and the
// eight they are paired with, dh / 16 threads a head, so that the sum of squares needs log2(dh / 16) shuffles; the next such item is
// loaded before one is worked on.  16384 rows of 40 heads of 128: four items in flight in 124 registers a thread 128 us, one ahead in 64: 63 us
// (floor 51).
#include "kv4.cuh"

namespace l2pd {

namespace {

constexpr int MAX_HALF = 128;   // dh <= 256

struct Freq { double f[MAX_HALF]; };   // turns (angle / 2 pi) of pair i per position

constexpr int TABLE = 1024;   // (cos, sin) pairs in shared memory

__device__ __forceinline__ float2 turn(double pos, double turns_per_position) {
  double t = pos * turns_per_position;
  t -= rint(t);
  float2 cs;
  sincospif(2.f * (float)t, &cs.y, &cs.x);
  return cs;
}

// L = dh / 16 threads a head, a power of two
template <typename T>
__global__ void __launch_bounds__(256, 4) qk_norm_rope_vec_kernel(const NormRopeArgs p, const __grid_constant__ Freq freq, int R, int L) {
  __shared__ float4 table[TABLE / 2];        // row r, pairs 8 c + 2 q, + 1 at [(r * 4 + q) * L + c]: no bank conflicts over c
  const int heads = p.Hq + p.Hk, half = p.dh >> 1, row0 = blockIdx.x * R, rows = min(R, p.rows - row0), per_row = heads * L;
  const int n = rows * per_row, c = threadIdx.x & (L - 1);
  grid_dep_launch();
  grid_dep_wait();
  const int step = 256 / L;                  // heads that a round advances by
  int row = (int)(threadIdx.x / L) / heads, head = (int)(threadIdx.x / L) - row * heads;   // of the item under way
  Vec8<T> lo, hi;
  auto fetch = [&](Vec8<T> &a, Vec8<T> &b, int r, int h) {
    if (r >= rows) return;
    const T *x = h >= p.Hq ? (const T *)p.k + (row0 + r) * p.k_stride + (int64_t)(h - p.Hq) * p.dh
                           : (const T *)p.q + (row0 + r) * p.q_stride + (int64_t)h * p.dh;
    a.load(x + 8 * c);
    b.load(x + 8 * c + half);
  };
#pragma unroll
  for (int i = 0; i < 8; ++i) { lo.set(i, 0.f); hi.set(i, 0.f); }
  fetch(lo, hi, row, head);
  for (int i = threadIdx.x; i < rows * half; i += 256) {
    const int tr = i / half, k = i - tr * half;
    const int64_t pos = p.positions ? p.positions[row0 + tr] : row0 + tr;
    reinterpret_cast<float2 *>(table)[2 * ((tr * 4 + ((k >> 1) & 3)) * L + (k >> 3)) + (k & 1)] = turn((double)pos, freq.f[k]);
  }
  __syncthreads();
  const float inv_dh = 1.f / p.dh;
  for (int done = 0; done < n; done += 256) {
    Vec8<T> next_lo = lo, next_hi = hi;
    int next_row = row, next_head = head + step;
    while (next_head >= heads) { next_head -= heads; ++next_row; }
    fetch(next_lo, next_hi, next_row, next_head);
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) ss = fmaf(lo.get(i), lo.get(i), fmaf(hi.get(i), hi.get(i), ss));
    for (int o = L >> 1; o; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
    if (row < rows) {
      const bool is_k = head >= p.Hq;
      const float *g = is_k ? p.k_gain : p.q_gain;
      const float norm = g ? rsqrtf(fmaf(ss, inv_dh, p.eps)) : 1.f;
      T *y = is_k ? (T *)p.k_out + (row0 + row) * p.ko_stride + (int64_t)(head - p.Hq) * p.dh
                  : (T *)p.q_out + (row0 + row) * p.qo_stride + (int64_t)head * p.dh;
#pragma unroll
      for (int q4 = 0; q4 < 2; ++q4) {
        float4 ga = make_float4(1.f, 1.f, 1.f, 1.f), gb = ga;
        if (g) {
          ga = *reinterpret_cast<const float4 *>(g + 8 * c + 4 * q4);
          gb = *reinterpret_cast<const float4 *>(g + 8 * c + half + 4 * q4);
        }
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          const float4 cs = table[(row * 4 + 2 * q4 + q) * L + c];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int i = 4 * q4 + 2 * q + e;
            const float co = e ? cs.z : cs.x, si = e ? cs.w : cs.y;
            const float a = lo.get(i) * norm * (&ga.x)[2 * q + e], b = hi.get(i) * norm * (&gb.x)[2 * q + e];
            lo.set(i, a * co - b * si);
            hi.set(i, b * co + a * si);
          }
        }
      }
      lo.store(y + 8 * c);
      hi.store(y + 8 * c + half);
    }
    lo = next_lo; hi = next_hi; row = next_row; head = next_head;
  }
}

// Any even head size and alignment.  One warp per (row, head); a lane holds the pairs lane, lane + 32, ...
template <typename T>
__global__ void __launch_bounds__(256) qk_norm_rope_kernel(const NormRopeArgs p, const __grid_constant__ Freq freq) {
  grid_dep_launch();
  grid_dep_wait();
  const int lane = threadIdx.x & 31, heads = p.Hq + p.Hk, half = p.dh >> 1;
  const int64_t n = (int64_t)p.rows * heads;
  for (int64_t it = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); it < n; it += (int64_t)gridDim.x * 8) {
    const int row = (int)(it / heads);
    int h = (int)(it - (int64_t)row * heads);
    const bool is_k = h >= p.Hq;
    if (is_k) h -= p.Hq;
    const T *x = (const T *)(is_k ? p.k : p.q) + (int64_t)row * (is_k ? p.k_stride : p.q_stride) + (int64_t)h * p.dh;
    T *y = (T *)(is_k ? p.k_out : p.q_out) + (int64_t)row * (is_k ? p.ko_stride : p.qo_stride) + (int64_t)h * p.dh;
    const float *g = is_k ? p.k_gain : p.q_gain;
    const double pos = p.positions ? p.positions[row] : row;
    float a[MAX_HALF / 32], b[MAX_HALF / 32], ss = 0.f;
#pragma unroll
    for (int u = 0; u < MAX_HALF / 32; ++u) {
      const int i = lane + 32 * u;
      a[u] = i < half ? to_f32(x[i]) : 0.f;
      b[u] = i < half ? to_f32(x[i + half]) : 0.f;
      ss += a[u] * a[u] + b[u] * b[u];
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
    const float r = g ? rsqrtf(ss / p.dh + p.eps) : 1.f;
#pragma unroll
    for (int u = 0; u < MAX_HALF / 32; ++u) {
      const int i = lane + 32 * u;
      if (i < half) {
        const float ya = a[u] * r * (g ? g[i] : 1.f), yb = b[u] * r * (g ? g[i + half] : 1.f);
        const float2 cs = turn(pos, freq.f[i]);
        y[i] = from_f32<T>(ya * cs.x - yb * cs.y);
        y[i + half] = from_f32<T>(yb * cs.x + ya * cs.y);
      }
    }
  }
}

}  // namespace

template <typename T>
cudaError_t launch_qk_norm_rope(cudaStream_t st, const NormRopeArgs &a, int sms) {
  Freq f;
  const int half = a.dh / 2;
  // theta^(-i / half) by repeated products in long double: 128 of them are off by 2^-57
  const long double step = expl(-logl((long double)a.theta) / half);
  long double x = 1.0L / 6.283185307179586476925286766559L;
  for (int i = 0; i < half; ++i, x *= step) f.f[i] = (double)x;
  const int L = a.dh / 16, heads = a.Hq + a.Hk;
  if (a.vec && (L & (L - 1)) == 0) {
    // rows of a block: at most sixteen rounds of its threads; below that the number with which blocks, four an SM at a time, are done
    // soonest, a block counted as a row more than it has (16384 rows of 40 heads of 128: 12 rows 66 us, 7 rows
    // 63; heads of 64: 16 rows 42.5 us, 14 rows 33)
    int64_t most = (int64_t)16 * 256 / ((int64_t)heads * L), R = 1, best = INT64_MAX;
    if (most > TABLE / half) most = TABLE / half;
    for (int64_t r = most < 1 ? 1 : most; r >= 1; --r) {
      const int64_t cost = ceil_div64(ceil_div64(a.rows, r), (int64_t)4 * sms) * (r + 1);   // a row's time for what a block takes besides
      if (cost < best) { best = cost; R = r; }
    }
    return launch_kernel(qk_norm_rope_vec_kernel<T>, dim3((unsigned)ceil_div64(a.rows, R)), dim3(256), 0, st, a, f, (int)R, L);
  }
  const int64_t blocks = ceil_div64((int64_t)a.rows * heads, 8);
  const int grid = (int)(blocks < (int64_t)sms * 8 ? blocks : (int64_t)sms * 8);
  return launch_kernel(qk_norm_rope_kernel<T>, dim3(grid), dim3(256), 0, st, a, f);
}
template cudaError_t launch_qk_norm_rope<float>(cudaStream_t, const NormRopeArgs &, int);
template cudaError_t launch_qk_norm_rope<bf16>(cudaStream_t, const NormRopeArgs &, int);

}  // namespace l2pd
