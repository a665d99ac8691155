// Norms of queries and keys for each head, with the rotation by position in the same pass:
//     y = x g / sqrt(mean(x^2) + eps)        over the dh values of a (row, head)
//     (y_i, y_{i + dh/2}) turned by the angle position * theta^(-2i/dh)
// in fp32 between the load and the one rounding at the store.
#include "kv4.cuh"

namespace l2pd {

namespace {

constexpr int MAX_HALF = 128;   // dh <= 256

struct Freq { double f[MAX_HALF]; };   // turns (angle / 2 pi) of pair i per position

// One warp per (row, head); a lane holds the pairs lane, lane + 32, ...
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
        double turns = pos * freq.f[i];
        turns -= rint(turns);
        float s, c;
        sincospif(2.f * (float)turns, &s, &c);
        y[i] = from_f32<T>(ya * c - yb * s);
        y[i + half] = from_f32<T>(yb * c + ya * s);
      }
    }
  }
}

}  // namespace

template <typename T>
cudaError_t launch_qk_norm_rope(cudaStream_t st, const NormRopeArgs &a, int sms) {
  Freq f;
  const int half = a.dh / 2;
  for (int i = 0; i < half; ++i) f.f[i] = exp(-log((double)a.theta) * i / half) / 6.283185307179586476925286766559;
  const int64_t blocks = ceil_div64((int64_t)a.rows * (a.Hq + a.Hk), 8);
  const int grid = (int)(blocks < (int64_t)sms * 8 ? blocks : (int64_t)sms * 8);
  return launch_kernel(qk_norm_rope_kernel<T>, dim3(grid), dim3(256), 0, st, a, f);
}
template cudaError_t launch_qk_norm_rope<float>(cudaStream_t, const NormRopeArgs &, int);
template cudaError_t launch_qk_norm_rope<bf16>(cudaStream_t, const NormRopeArgs &, int);

}  // namespace l2pd
