// Attention over a key/value cache in 4 bits, and the sum of the weights each key receives.
//
// The columns of a (sequence, key head) are its query rows times the query heads that share the key head.  Scores are computed as
// S^T = K Q^T, keys on the M side of mma.sync.m16n8k16, so that one query row pads to 8 columns instead of 16 rows, and the
// output as O^T = V^T P^T.  A code c in the low four bits of an fp16 is the subnormal number c 2^-24, exactly: the codes go to the
// product as they lie, by a mask (those in bits 4..7 as 16 c 2^-24, against queries divided by 16).  With q' = q scaled by a power
// of two of its own into fp16's range (8 significant bits of 11), and cf what undoes it:
//     t_j = log2 of exp(scale q . k_j) + e_j - E = cf (s_j sum(c q') + m_j sum(q')) + e_j - E
// 2^e_j bounds the value row's s_j and |m_j| / 16, E is above all e_j so far.  Probabilities are taken as p'_j = 2^(t_j - M), M a reference
// 2^9 to 2^15 below the running maximum of t, so that p'_j s_j 2^-e_j, what multiplies the codes of V, stays within fp16 whatever the
// values' magnitude (attention_kv4.cuh has what becomes of M and the sums where E rises).  Rounding that to fp16 is the only step to less than 32
// bits between the queries and the output.
//
// Work: the key tiles of all (sequence, head, chunk of columns) stand in one line and every CTA takes an equal run of it; a run
// that starts or ends inside an item leaves a partial result, joined in the order of the tiles by a second kernel.  A warp takes
// every fourth tile of its CTA's run, through a ring of its own.  Two to four CTAs an SM: one computes while another fetches
// queries or brings its warps' sums together.
//
// What bounds it.  One row of 32/8 heads on 4000 keys: the latency of a few dependent steps and of two launches, 11 us.  Up to 8
// columns on many keys: memory (64 rows of 32/8 heads on 8192 keys each: 103 us, 5.5 TB/s).  32 columns (8 x 32 rows of 32 heads of
// 128 on 2048 keys, 43 us; 255 registers, 36 bytes spilled): products 512 cycles of a scheduler and 453 instructions for 16 keys, which take 1250; registers leave two
// warps a scheduler, and each goes through products, exponentials and products in turn.
#include <cuda_fp16.h>
#include <math.h>

#include "attention_kv4.cuh"

namespace l2pd {

namespace {

using namespace kv4;
using ptx::F2;

constexpr int WARPS = 4;

// The four registers of two MMA steps in a word of eight codes: codes 0 and 4, 1 and 5 (times 16), 2 and 6, 3 and 7 (times 16).
__device__ __forceinline__ void spread(uint32_t w, uint32_t *r) {
  r[0] = w & 0x000f000fu; r[1] = w & 0x00f000f0u;
  w >>= 8;
  r[2] = w & 0x000f000fu; r[3] = w & 0x00f000f0u;
}

// tile row of MMA row k (0..7): in every other pair the two change places, so that the four keys whose V rows a warp reads at
// once lie in different banks
__device__ __forceinline__ int tile_row(int k) { return k ^ ((k >> 1) & 1); }

// ---- queries as B fragments --------------------------------------------------------------------------------------------
// Eight columns: lane (g, t) holds of column g the dimensions [t dh/4, (t + 1) dh/4).
template <int DH> struct Queries {
  uint32_t raw[DH / 8];
  uint32_t top;                                    // the column's largest magnitude, as bits; non-finite ones above all
  __device__ __forceinline__ void load(const bf16 *q, bool there) {
#pragma unroll
    for (int j = 0; j < DH / 32; ++j) {
      const uint4 x = there ? *reinterpret_cast<const uint4 *>(q + 8 * j) : make_uint4(0, 0, 0, 0);
      raw[4 * j] = x.x; raw[4 * j + 1] = x.y; raw[4 * j + 2] = x.z; raw[4 * j + 3] = x.w;
    }
    top = 0;
#pragma unroll
    for (int i = 0; i < DH / 8; ++i) top = max(top, max(raw[i] << 16 & 0x7fffffffu, raw[i] & 0x7fff0000u));
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
  }
  __device__ __forceinline__ bool finite() const { return top < 0x7f800000u; }
  // Power of two that takes the column's largest to 2^14 .. 2^15: what is less than 2^-35 of it is lost (odd dimensions go in divided by 16).
  // Columns have powers of their own: rows of a block may differ without limit.
  __device__ __forceinline__ int exponent() const { return finite() ? min(14 - ((int)(top >> 23) - 127), 126) : 0; }
  // Scaled by 2^u to fp16.  Returns the column's sum in the scale of the products with codes; NaN: a column that holds an
  // infinity or NaN, whose scores are all NaN.
  __device__ __forceinline__ float convert(int u, uint32_t (&f)[DH / 8]) const {
    const float up = __uint_as_float((uint32_t)(127 + u) << 23);
    float sum = 0.f;
#pragma unroll
    for (int j = 0; j < DH / 32; ++j) {
      float y[8];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t w = finite() ? raw[4 * j + i] : 0u;
        y[2 * i] = __uint_as_float(w << 16) * up; y[2 * i + 1] = __uint_as_float(w & 0xffff0000u) * up;
        sum += y[2 * i] + y[2 * i + 1];
      }
      auto pair = [](float a, float b) { __half2 h = __floats2half2_rn(a, b); return *reinterpret_cast<uint32_t *>(&h); };
      f[4 * j] = pair(y[0], y[4]); f[4 * j + 1] = pair(y[1] * 0.0625f, y[5] * 0.0625f);
      f[4 * j + 2] = pair(y[2], y[6]); f[4 * j + 3] = pair(y[3] * 0.0625f, y[7] * 0.0625f);
    }
    sum += __shfl_xor_sync(0xffffffffu, sum, 1);
    sum += __shfl_xor_sync(0xffffffffu, sum, 2);
    return finite() ? sum * __uint_as_float((127 - 24) << 23) : __uint_as_float(0x7fc00000u);
  }
};
// What turns a column's products, with K's s and m times 2^12, into log2 scores: scale 2^(12 - u).  (2^24 in one place would pass fp32 for
// queries near 2^127.)
constexpr float K_UNIT = 4096.f;
__device__ __forceinline__ float query_factor(float scale_log2, int u) { return scale_log2 * __uint_as_float((uint32_t)(127 + 12 - u) << 23); }

template <int DH, int NT> struct AttnShape {
  static constexpr int CH = 8 * NT, TILE = KV4_TILE * (DH + 8), STAGES = NT == 4 ? 4 : 3, RING = STAGES * TILE;
  static constexpr int CTAS = NT == 1 && DH == 64 ? 4 : NT <= 2 ? 3 : 2;   // an SM's, as registers and shared memory allow
  static constexpr bool Q_REGS = NT < 4;           // queries in registers; with 32 columns they are read from shared memory where they are used
  static constexpr int META = KV4_TILE * 24, QBYTES = NT * DH * 16;
  static constexpr int OFF_META = WARPS * RING, OFF_Q = OFF_META + WARPS * META, SMEM = OFF_Q + QBYTES;
  static_assert(CTAS * (SMEM + 1536 + 1024) <= 228 * 1024, "with what the kernel declares itself (1536 at most) and what a CTA costs besides");
};

template <int DH, int NT>
__global__ void __launch_bounds__(WARPS * 32, AttnShape<DH, NT>::CTAS) attention_kv4_kernel(const AttnParams p) {
  using Sh = AttnShape<DH, NT>;
  constexpr int W = DH / 32, MT = DH / 16, CH = Sh::CH, MS = NT == 2 ? 1 : 2;   // MS: groups of 16 keys taken together
  constexpr int TILE = Sh::TILE, RING = Sh::RING, STAGES = Sh::STAGES, LDO = DH + 4;
  static_assert(KV4_TILE == 32 && CH * LDO * 4 <= RING, "a warp's output goes to its ring");
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ __align__(8) uint64_t bars[WARPS * STAGES];
  __shared__ float fin[WARPS][2][CH];              // reference and sum of weights
  __shared__ float4 qcol[CH / 2];                  // of two columns: sums of q' times cf, and cf
  __shared__ int abort_flag;
  const int warp = ptx::warp_index(), lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const uint32_t bar0 = ptx::smem_u32(&bars[warp * STAGES]);
  uint8_t *const ring = smem + warp * RING;
  const uint32_t ring_u = ptx::smem_u32(ring);
  float4 *const meta_a = reinterpret_cast<float4 *>(smem + Sh::OFF_META + warp * Sh::META);   // by key: s, m of K, e - E, 2^(E - e - LOG_L)
  float2 *const meta_b = reinterpret_cast<float2 *>(meta_a + KV4_TILE);                        // s 2^-e, m 2^-e of V
  uint4 *const qs = reinterpret_cast<uint4 *>(smem + Sh::OFF_Q);
  if (lane == 0) {
    for (int i = 0; i < STAGES; ++i) ptx::mbar_init(bar0 + 8 * i, 1);
    ptx::fence_barrier_init();
    ptx::fence_proxy_async();
  }
  if (threadIdx.x == 0) abort_flag = 0;
  __syncthreads();
  grid_dep_wait();
  grid_dep_launch();                               // behind the wait: see the joining kernel

  const Line &ln = p.line;
  const Seq own = ln.seq(lane);
  uint32_t share;
  const uint32_t total = ln.survey(own, gridDim.x, 0, &share, nullptr);
  uint32_t pos = min((uint64_t)share * blockIdx.x, (uint64_t)total);
  const uint32_t end = min(total, pos + share);
  uint32_t used = 0;                               // tiles this warp has taken: stage and parity
  while (pos < end) {
    uint32_t before;
    const Seq sq = ln.find(own, pos, &before);
    const int nt = sq.tiles, item = (int)((pos - before) / nt), t0 = (int)(pos - before) - item * nt, t1 = (int)min((uint32_t)nt, t0 + (end - pos));
    const int h = item / sq.chunks, c0 = (item - h * sq.chunks) * CH, cols = min(CH, sq.rows * ln.group - c0);
    const int n_keys = sq.keys, row0 = sq.row0;
    const uint8_t *src = p.c.tile(sq.slot, h, 0);
    pos += t1 - t0;

    // this warp's tiles: t0 + warp, + WARPS, ...
    const int mine = (t1 - t0 - warp + WARPS - 1) / WARPS;
    auto request = [&](int i) {
      if (i < mine && ptx::elect_one()) {
        const uint32_t s = (used + i) % STAGES;
        ptx::mbar_arrive_expect_tx(bar0 + 8 * s, TILE);
        ptx::bulk_load(ring_u + s * TILE, src + (int64_t)(t0 + warp + i * WARPS) * TILE, TILE, bar0 + 8 * s);
      }
    };
    for (int i = 0; i < STAGES; ++i) request(i);

    // queries: warp n converts the columns 8 n .. 8 n + 7 for all
    if (warp < NT) {
      const int col = c0 + 8 * warp + g, r = col / ln.group;
      Queries<DH> qn;
      qn.load(p.q + (int64_t)(row0 + r) * p.q_stride + (int64_t)(h * ln.group + col - r * ln.group) * DH + t * (DH / 4), 8 * warp + g < cols);
      uint32_t f[DH / 8];
      const int u = qn.exponent();
      const float sum = qn.convert(u, f), cf = query_factor(p.scale_log2, u);
      if (t == 0) {
        float *of = reinterpret_cast<float *>(&qcol[4 * warp + (g >> 1)]) + (g & 1);
        of[0] = sum * cf; of[2] = cf;
      }
#pragma unroll
      for (int j = 0; j < W; ++j) qs[(warp * W + j) * 32 + lane] = make_uint4(f[4 * j], f[4 * j + 1], f[4 * j + 2], f[4 * j + 3]);
    }
    __syncthreads();
    uint32_t qf[Sh::Q_REGS ? NT : 1][DH / 8];
    F2 cs[Sh::Q_REGS ? NT : 1], cf[Sh::Q_REGS ? NT : 1];   // columns 2t and 2t + 1 of each eight
    auto column_factors = [&](int n, F2 &sum, F2 &factor) {
      const float4 x = qcol[4 * n + t];
      sum = ptx::f2(x.x, x.y); factor = ptx::f2(x.z, x.w);
    };
    F2 neg_m[NT], l[NT], wm[NT];                   // minus the reference, sum of probabilities, sum of probability times m
    float o[MT][NT][4];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
      for (int j = 0; Sh::Q_REGS && j < W; ++j) *reinterpret_cast<uint4 *>(&qf[Sh::Q_REGS ? n : 0][4 * j]) = qs[(n * W + j) * 32 + lane];
      if (Sh::Q_REGS) column_factors(n, cs[Sh::Q_REGS ? n : 0], cf[Sh::Q_REGS ? n : 0]);
      neg_m[n] = l[n] = wm[n] = ptx::f2(0.f, 0.f);
#pragma unroll
      for (int m = 0; m < MT; ++m) o[m][n][0] = o[m][n][1] = o[m][n][2] = o[m][n][3] = 0.f;
    }
    int e0 = -1000;                                // E
    bool ok = true, first = true;
    for (int i = 0; i < mine; ++i) {
      const uint32_t s = (used + i) % STAGES;
      ok = ptx::mbar_wait_warp(bar0 + 8 * s, ((used + i) / STAGES) & 1u);
      if (!ok) break;
      const uint8_t *tile = ring + s * TILE;
      const int left = n_keys - (t0 + warp + i * WARPS) * KV4_TILE;    // keys of this tile, or more
      // what belongs to a key, once for all columns; keys behind the end get weight 0
      {
        const bool real = lane < left;
        const uint32_t km = real ? *reinterpret_cast<const uint32_t *>(tile + kv4_off_kmeta(DH) + 4 * lane) : 0u;
        const uint32_t vm = real ? *reinterpret_cast<const uint32_t *>(tile + kv4_off_vmeta(DH) + 4 * lane) : 0u;
        const int ex = min(max((int)((vm >> 7) & 255u), (int)((vm >> 23) & 255u) - 4) - 126, 125);   // NaN: 125
        const int ex_top = __reduce_max_sync(0xffffffffu, ex);
        if (ex_top > e0) {                         // rare
          const float d = e0 == -1000 ? 0.f : (float)(max(ex_top, -100) + 2 - e0);
          e0 = max(ex_top, -100) + 2;
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            const F2 was = neg_m[n];
            neg_m[n] = ptx::add2(was, ptx::f2(d, d));
            const float da = ptx::f2_lo(neg_m[n]) - ptx::f2_lo(was), db = ptx::f2_hi(neg_m[n]) - ptx::f2_hi(was);
            l[n] = ptx::f2(ex2_scaled(ptx::f2_lo(l[n]), da), ex2_scaled(ptx::f2_hi(l[n]), db));
            if (__any_sync(0xffffffffu, da != d || db != d)) {   // references beyond 2^24 do not move by d exactly
              const float fa = ptx::ex2(da - d), fb = ptx::ex2(db - d);
              wm[n] = ptx::mul2(wm[n], ptx::f2(fa, fb));
#pragma unroll
              for (int m = 0; m < MT; ++m) { o[m][n][0] *= fa; o[m][n][2] *= fa; o[m][n][1] *= fb; o[m][n][3] *= fb; }
            }
          }
        }
        const int e = max(ex, e0 + (int)FLOOR);
        const float w = __uint_as_float((uint32_t)(127 - e) << 23);
        meta_a[lane] = make_float4(kv4_scale(km) * K_UNIT, kv4_min(km) * K_UNIT, real ? (float)(e - e0) : -INFINITY,
                                   pow2(e0 - e - LOG_L));
        meta_b[lane] = make_float2(kv4_scale(vm) * w, kv4_min(vm) * w);
        __syncwarp();
      }
#pragma unroll 1
      for (int s0 = 0; s0 < KV4_TILE / 16; s0 += MS) {
        float acc[MS][NT][4];
        const int kr = 16 * s0 + tile_row(g);
        uint32_t ka[MS][W], kb[MS][W];
#pragma unroll
        for (int u = 0; u < MS; ++u) {
          const uint8_t *a = tile + (kr + 16 * u) * (DH / 2) + t * (DH / 8), *c = a + 8 * (DH / 2);
          if (DH == 128) {
            *reinterpret_cast<uint4 *>(ka[u]) = *reinterpret_cast<const uint4 *>(a);
            *reinterpret_cast<uint4 *>(kb[u]) = *reinterpret_cast<const uint4 *>(c);
          } else {
            *reinterpret_cast<uint2 *>(ka[u]) = *reinterpret_cast<const uint2 *>(a);
            *reinterpret_cast<uint2 *>(kb[u]) = *reinterpret_cast<const uint2 *>(c);
          }
        }
#pragma unroll
        for (int j = 0; j < W; ++j) {
          uint32_t x[MS][4], y[MS][4];
#pragma unroll
          for (int u = 0; u < MS; ++u) { spread(ka[u][j], x[u]); spread(kb[u][j], y[u]); }
          uint4 q4[NT];
#pragma unroll
          for (int n = 0; n < NT; ++n)
            q4[n] = Sh::Q_REGS ? make_uint4(qf[Sh::Q_REGS ? n : 0][4 * j], qf[Sh::Q_REGS ? n : 0][4 * j + 1], qf[Sh::Q_REGS ? n : 0][4 * j + 2], qf[Sh::Q_REGS ? n : 0][4 * j + 3])
                               : qs[(n * W + j) * 32 + lane];
          // one step of all sums, then the next: a sum's steps depend on one another
#pragma unroll
          for (int u = 0; u < MS; ++u)
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              if (j == 0) ptx::mma_f16_16x8x16_first(acc[u][n], x[u][0], y[u][0], x[u][1], y[u][1], q4[n].x, q4[n].y);
              else ptx::mma_f16_16x8x16(acc[u][n], x[u][0], y[u][0], x[u][1], y[u][1], q4[n].x, q4[n].y);
            }
#pragma unroll
          for (int u = 0; u < MS; ++u)
#pragma unroll
            for (int n = 0; n < NT; ++n)
              ptx::mma_f16_16x8x16(acc[u][n], x[u][2], y[u][2], x[u][3], y[u][3], q4[n].z, q4[n].w);
        }
        // scores against the reference
        float top = -INFINITY;
#pragma unroll
        for (int u = 0; u < MS; ++u)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float4 k = meta_a[kr + 16 * u + 8 * e];
            const F2 ks = ptx::f2(k.x, k.x), km = ptx::f2(k.y, k.y), bias = ptx::f2(k.z, k.z);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              float *x = &acc[u][n][2 * e];
              F2 sum = cs[Sh::Q_REGS ? n : 0], factor = cf[Sh::Q_REGS ? n : 0];
              if (!Sh::Q_REGS) column_factors(n, sum, factor);
              const F2 y = ptx::fma2(ptx::mul2(ptx::f2(x[0], x[1]), factor), ks, ptx::fma2(km, sum, ptx::add2(bias, neg_m[n])));   // exponents first: they cancel
              x[0] = ptx::f2_lo(y); x[1] = ptx::f2_hi(y);
              top = fmaxf(top, fmaxf(x[0], x[1]));
            }
          }
        // a new reference where the maximum has passed the old one by LAZY, and at the start
        if (__any_sync(0xffffffffu, first || top > LAZY)) {
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            float xa = -INFINITY, xb = -INFINITY;
#pragma unroll
            for (int u = 0; u < MS; ++u) {
              xa = fmaxf(xa, fmaxf(acc[u][n][0], acc[u][n][2]));
              xb = fmaxf(xb, fmaxf(acc[u][n][1], acc[u][n][3]));
            }
#pragma unroll
            for (int x = 4; x < 32; x <<= 1) {
              xa = fmaxf(xa, __shfl_xor_sync(0xffffffffu, xa, x));
              xb = fmaxf(xb, __shfl_xor_sync(0xffffffffu, xb, x));
            }
            const float least = first ? -3e38f : 0.f;        // afterwards references rise only
            const float da = xa == -INFINITY ? 0.f : fmaxf(xa - BELOW, least), db = xb == -INFINITY ? 0.f : fmaxf(xb - BELOW, least);
            const float sa = first ? 0.f : ptx::ex2(-da), sb = first ? 0.f : ptx::ex2(-db);
            const F2 d = ptx::f2(-da, -db), sc = ptx::f2(sa, sb);
            neg_m[n] = ptx::add2(neg_m[n], d);
            l[n] = ptx::f2(ex2_scaled(ptx::f2_lo(l[n]), -da), ex2_scaled(ptx::f2_hi(l[n]), -db));
            wm[n] = ptx::mul2(wm[n], sc);
#pragma unroll
            for (int m = 0; m < MT; ++m) { o[m][n][0] *= sa; o[m][n][2] *= sa; o[m][n][1] *= sb; o[m][n][3] *= sb; }
#pragma unroll
            for (int u = 0; u < MS; ++u) { acc[u][n][0] -= da; acc[u][n][2] -= da; acc[u][n][1] -= db; acc[u][n][3] -= db; }
          }
          first = false;
        }
#pragma unroll
        for (int u = 0; u < MS; ++u) {
          uint32_t pf[NT][2];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float w = meta_a[kr + 16 * u + 8 * e].w;
            const float2 v = meta_b[kr + 16 * u + 8 * e];
            const F2 vw = ptx::f2(w, w), vs = ptx::f2(v.x, v.x), vm = ptx::f2(v.y, v.y);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              const F2 pr = ptx::f2(ptx::ex2(acc[u][n][2 * e]), ptx::ex2(acc[u][n][2 * e + 1]));
              l[n] = ptx::fma2(pr, vw, l[n]);
              wm[n] = ptx::fma2(pr, vm, wm[n]);
              const F2 ps = ptx::mul2(pr, vs);
              __half2 hp = __floats2half2_rn(ptx::f2_lo(ps), ptx::f2_hi(ps));
              pf[n][e] = ptx::transpose_8x8(*reinterpret_cast<uint32_t *>(&hp));
            }
          }
          // values: lane (g, t) holds dimensions [g dh/8, (g + 1) dh/8) of the keys of MMA columns 2t, 2t + 1, 2t + 8, 2t + 9
          constexpr int VW = DH / 64;
          uint32_t va[4][VW];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int r = 16 * (s0 + u) + tile_row(2 * t + (e & 1)) + 8 * (e >> 1);
            const uint8_t *a = tile + kv4_off_v(DH) + r * (DH / 2) + ((g * (DH / 16)) ^ kv4_v_swizzle(r, DH));
            if (DH == 128) *reinterpret_cast<uint2 *>(va[e]) = *reinterpret_cast<const uint2 *>(a);
            else va[e][0] = *reinterpret_cast<const uint32_t *>(a);
          }
#pragma unroll
          for (int w = 0; w < VW; ++w)
#pragma unroll
            for (int hw = 0; hw < 2; ++hw) {
              uint32_t x[4], y[4];
              spread(__byte_perm(va[0][w], va[1][w], hw ? 0x7632 : 0x5410), x);
              spread(__byte_perm(va[2][w], va[3][w], hw ? 0x7632 : 0x5410), y);
              const int m = 4 * w + 2 * hw;
#pragma unroll
              for (int n = 0; n < NT; ++n) {
                ptx::mma_f16_16x8x16(o[m][n], x[0], x[1], y[0], y[1], pf[n][0], pf[n][1]);
                ptx::mma_f16_16x8x16(o[m + 1][n], x[2], x[3], y[2], y[3], pf[n][0], pf[n][1]);
              }
            }
        }
      }
      ptx::fence_proxy_async();                    // the next copy overwrites what was read: no read is put off behind it
      __syncwarp();
      request(i + STAGES);
    }
    if (!ok) { fail(p.status, DEV_TIMEOUT_EPILOGUE); abort_flag = 1; }
    used += max(mine, 0);

    // the warps meet: every warp's sums and outputs go to shared memory, each against its own reference
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      float la = ptx::f2_lo(l[n]), lb = ptx::f2_hi(l[n]), wa = ptx::f2_lo(wm[n]), wb = ptx::f2_hi(wm[n]);
#pragma unroll
      for (int x = 4; x < 32; x <<= 1) {
        la += __shfl_xor_sync(0xffffffffu, la, x); lb += __shfl_xor_sync(0xffffffffu, lb, x);
        wa += __shfl_xor_sync(0xffffffffu, wa, x); wb += __shfl_xor_sync(0xffffffffu, wb, x);
      }
      const Normal na = normalised(la, -ptx::f2_lo(neg_m[n]), max(e0, -100)), nb = normalised(lb, -ptx::f2_hi(neg_m[n]), max(e0, -100));
      if (g == 0) {
        fin[warp][0][8 * n + 2 * t] = na.ref; fin[warp][0][8 * n + 2 * t + 1] = nb.ref;      // no tiles: -inf
        fin[warp][1][8 * n + 2 * t] = na.x; fin[warp][1][8 * n + 2 * t + 1] = nb.x;
      }
      float *oa = reinterpret_cast<float *>(ring) + (8 * n + 2 * t) * LDO + g * (DH / 8), *ob = oa + LDO;
      constexpr float EVEN = 16777216.f, ODD = 1048576.f;             // the codes' 2^24, and 2^20 where they came 16 times
      auto in_unit = [](float x, float unit, float w, const Normal &f) { return fmaf(x, unit, w) * f.up_a * f.up_b; };
#pragma unroll
      for (int m = 0; m < MT; m += 2) {
        *reinterpret_cast<float4 *>(oa + 2 * m) = make_float4(in_unit(o[m][n][0], EVEN, wa, na), in_unit(o[m][n][2], ODD, wa, na),
                                                              in_unit(o[m + 1][n][0], EVEN, wa, na), in_unit(o[m + 1][n][2], ODD, wa, na));
        *reinterpret_cast<float4 *>(ob + 2 * m) = make_float4(in_unit(o[m][n][1], EVEN, wb, nb), in_unit(o[m][n][3], ODD, wb, nb),
                                                              in_unit(o[m + 1][n][1], EVEN, wb, nb), in_unit(o[m + 1][n][3], ODD, wb, nb));
      }
    }
    __syncthreads();
    if (abort_flag) break;
    const bool whole = t0 == 0 && t1 == nt;
    float *part = p.part + (int64_t)(2 * blockIdx.x + (t0 == 0 ? 1 : 0)) * part_floats(CH, DH);
    for (int x = threadIdx.x; x < cols * (DH / 4); x += WARPS * 32) {
      const int c = x / (DH / 4), d = x % (DH / 4) * 4;
      float m = -INFINITY;
#pragma unroll
      for (int w = 0; w < WARPS; ++w) m = fmaxf(m, fin[w][0][c]);
      float sum = 0.f;
      float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < WARPS; ++w) {
        const float mw = fin[w][0][c], f = mw == -INFINITY ? 0.f : ptx::ex2(mw - m);
        const float4 z = *reinterpret_cast<const float4 *>(smem + w * RING + (c * LDO + d) * 4);
        sum = fmaf(fin[w][1][c], f, sum);
        y.x = fmaf(z.x, f, y.x); y.y = fmaf(z.y, f, y.y); y.z = fmaf(z.z, f, y.z); y.w = fmaf(z.w, f, y.w);
      }
      if (whole) {
        const int col = c0 + c, r = col / ln.group, hq = h * ln.group + col - r * ln.group;
        const float inv = 1.f / sum;
        __nv_bfloat162 y0 = __floats2bfloat162_rn(y.x * inv, y.y * inv), y1 = __floats2bfloat162_rn(y.z * inv, y.w * inv);
        *reinterpret_cast<uint2 *>(p.out + (int64_t)(row0 + r) * p.out_stride + (int64_t)hq * DH + d) =
            make_uint2(*reinterpret_cast<uint32_t *>(&y0), *reinterpret_cast<uint32_t *>(&y1));
        if (d == 0 && p.lse) p.lse[(int64_t)(row0 + r) * p.Hq + hq] = (m + log2f(sum)) * 0.6931471805599453f;
      } else {
        *reinterpret_cast<float4 *>(part + c * LDO + d) = y;
        if (d == 0) { part[c * LDO + DH] = m; part[c * LDO + DH + 1] = sum; }
      }
    }
    ptx::fence_proxy_async();                      // the ring was written by the threads: the next copies come after
    __syncthreads();
  }
  if (abort_flag) {                                // a wait ran out: copies in flight land before shared memory goes away
    const uint64_t start = ptx::globaltimer();
    while (ptx::globaltimer() - start < 200000ull) __nanosleep(1000);
  }
}

// Joins the partial results of an item, in the order of its tiles.  WPC warps have a column (4: few columns of many pieces);
// a block of four warps, 4 / WPC columns.  Sequences without keys: output 0, log-sum -inf.
// The attention kernel lets it start only behind its own wait for what came before: the batch's arrays are then final, and the
// survey runs beside the attention's end (one row on 4000 keys 13.3 -> 11.1 us, 3 x 27 rows 18.3 -> 15.2).
template <int DH, int WPC>
__global__ void __launch_bounds__(128) kv4_join_kernel(const AttnParams p, int n_ctas) {
  constexpr int LDO = DH + 4;
  __shared__ float sm_m[4], sm_l[4];
  __shared__ float4 sm_o[4][32];
  const Line &ln = p.line;
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, b = blockIdx.y, h = blockIdx.z, col = blockIdx.x * (4 / WPC) + w / WPC;
  const Seq own = ln.seq(lane), sq = ln.seq(b);
  uint32_t share = 1, before = 0;
  if (sq.tiles) ln.survey(own, n_ctas, b, &share, &before);
  grid_dep_launch();
  grid_dep_wait();
  if (col >= sq.rows * ln.group) return;           // WPC 4: the whole block
  const int nt = sq.tiles, r = col / ln.group, hq = h * ln.group + col - r * ln.group;
  const int64_t row = (int64_t)sq.row0 + r;
  bf16 *out = p.out + row * p.out_stride + (int64_t)hq * DH + 4 * lane;
  float *lse = p.lse ? p.lse + row * p.Hq + hq : nullptr;
  const bool mine = 4 * lane < DH, lead = w % WPC == 0;
  if (nt == 0) {
    if (lead && mine) *reinterpret_cast<uint2 *>(out) = make_uint2(0u, 0u);
    if (lead && lane == 0 && lse) *lse = -INFINITY;
    return;
  }
  const uint32_t start = before + ((uint32_t)h * sq.chunks + col / ln.chunk) * nt;
  const int i0 = (int)(start / share), i1 = (int)((start + nt - 1) / share);
  if (i0 == i1) return;                            // stored by its CTA
  const int c = col % ln.chunk;
  float m = -INFINITY, l = 0.f;
  float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
  for (int i = i0 + w % WPC; i <= i1; i += WPC) {
    const float *part = p.part + (int64_t)(2 * i + (i == i0 ? 1 : 0)) * part_floats(ln.chunk, DH) + c * LDO;
    const float2 ml = *reinterpret_cast<const float2 *>(part + DH);
    const float4 z = mine ? *reinterpret_cast<const float4 *>(part + 4 * lane) : make_float4(0.f, 0.f, 0.f, 0.f);
    const float mn = fmaxf(m, ml.x), f = m == -INFINITY ? 0.f : ptx::ex2(m - mn), fp = ml.x == -INFINITY ? 0.f : ptx::ex2(ml.x - mn);
    l = l * f + ml.y * fp;
    y.x = y.x * f + z.x * fp; y.y = y.y * f + z.y * fp; y.z = y.z * f + z.z * fp; y.w = y.w * f + z.w * fp;
    m = mn;
  }
  if (WPC == 4) {
    if (lane == 0) { sm_m[w] = m; sm_l[w] = l; }
    sm_o[w][lane] = y;
    __syncthreads();
    if (w) return;
    m = fmaxf(fmaxf(sm_m[0], sm_m[1]), fmaxf(sm_m[2], sm_m[3]));
    l = 0.f; y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float f = sm_m[i] == -INFINITY ? 0.f : ptx::ex2(sm_m[i] - m);
      const float4 z = sm_o[i][lane];
      l = fmaf(sm_l[i], f, l);
      y.x = fmaf(z.x, f, y.x); y.y = fmaf(z.y, f, y.y); y.z = fmaf(z.z, f, y.z); y.w = fmaf(z.w, f, y.w);
    }
  }
  const float inv = 1.f / l;
  if (mine) {
    __nv_bfloat162 y0 = __floats2bfloat162_rn(y.x * inv, y.y * inv), y1 = __floats2bfloat162_rn(y.z * inv, y.w * inv);
    *reinterpret_cast<uint2 *>(out) = make_uint2(*reinterpret_cast<uint32_t *>(&y0), *reinterpret_cast<uint32_t *>(&y1));
  }
  if (lane == 0 && lse) *lse = (m + log2f(l)) * 0.6931471805599453f;
}

// Up to 32 columns: the warp-level kernel, whose codes and probabilities never leave registers (queries of 32 columns do).  More: tcgen05
// with 64 or 128 lanes.  (8 sequences of 32 heads, us at 128 / 2048 / 8192 keys: 16 columns 10 / 32 / 80 against 20 / 52 / 145 on tcgen05,
// 32 columns 15 / 43 / 125 against 21 / 53 / 148; heads of 64: 7 / 32 / 57 against 17 / 42 / 116, 12 / 29 / 83 against 18 / 43 / 117.)
struct AttnPlan { int chunk, ctas, tc; };

AttnPlan plan_attention(const Kv4View &c, int B, int rows, int Hq, int max_len, int sms) {
  AttnPlan pl;
  const int heads = c.heads;
  if (max_len > c.cap) max_len = c.cap;            // a max_len of 2^31 - 1 says no more
  const int cols = rows * (Hq / heads);
  pl.tc = cols > 32;
  pl.chunk = cols <= 8 ? 8 : cols <= 16 ? 16 : cols <= 32 ? 32 : cols <= 64 ? 64 : 128;
  // no more CTAs than there are tiles for each, or for each warp of them
  const int64_t items = (int64_t)B * heads * ceil_div(cols, pl.chunk);
  const int64_t want = pl.tc ? items * ceil_div(max_len, TC_TILE) : ceil_div64(items * ceil_div(max_len, KV4_TILE), WARPS);
  const int most = pl.tc ? sms : sms * (pl.chunk == 32 ? 2 : pl.chunk == 8 && c.dh == 64 ? AttnShape<64, 1>::CTAS : AttnShape<128, 1>::CTAS);
  pl.ctas = (int)(want < 1 ? 1 : want < most ? want : most);
  return pl;
}

}  // namespace

bool attention_kv4_fits(const Kv4View &c, int B, int rows, int Hq, int max_len) {
  const double len = max_len < c.cap ? max_len : c.cap;
  return (double)B * c.heads * ((double)rows * (Hq / c.heads) / 8 + 1) * (len / KV4_TILE + 1) < 2147483648.0;
}

int64_t attention_kv4_scratch_floats(const Kv4View &c, int B, int rows, int Hq, int max_len, int sms) {
  const AttnPlan pl = plan_attention(c, B, rows, Hq, max_len, sms);
  return (int64_t)2 * pl.ctas * part_floats(pl.chunk, c.dh);
}

template <int DH, int NT>
static cudaError_t launch_attn(cudaStream_t st, const AttnParams &p, int ctas) {
  constexpr int smem = AttnShape<DH, NT>::SMEM;
  static std::atomic<uint64_t> done{0};
  const cudaError_t e = allow_shared((const void *)attention_kv4_kernel<DH, NT>, smem, done);
  if (e != cudaSuccess) return e;
  return launch_kernel(attention_kv4_kernel<DH, NT>, dim3(ctas), dim3(WARPS * 32), (size_t)smem, st, p);
}

template <int DH>
static cudaError_t launch_join(cudaStream_t st, const AttnParams &p, int ctas, int cols) {
  const int64_t all = (int64_t)cols * p.line.B * p.line.H;
  if (all <= 2048) return launch_kernel(kv4_join_kernel<DH, 4>, dim3(cols, p.line.B, p.line.H), dim3(128), 0, st, p, ctas);
  return launch_kernel(kv4_join_kernel<DH, 1>, dim3(ceil_div(cols, 4), p.line.B, p.line.H), dim3(128), 0, st, p, ctas);
}

cudaError_t launch_attention_kv4(cudaStream_t st, const Kv4AttnArgs &a, int sms) {
  const AttnPlan pl = plan_attention(a.c, a.b.B, a.b.rows, a.Hq, a.max_len, sms);
  AttnParams p;
  p.c = a.c; p.Hq = a.Hq; p.q = a.q; p.out = a.out; p.lse = a.lse; p.q_stride = a.q_stride; p.out_stride = a.out_stride;
  p.scale_log2 = a.scale * 1.4426950408889634f; p.part = a.scratch; p.status = a.status;
  Line &ln = p.line;
  ln.B = a.b.B; ln.H = a.c.heads; ln.chunk = pl.chunk; ln.group = a.Hq / a.c.heads; ln.slots = a.c.slots;
  ln.max_keys = a.max_len < a.c.cap ? a.max_len : a.c.cap; ln.tile_keys = pl.tc ? TC_TILE : KV4_TILE; ln.min_chunks = 0; ln.b = a.b;
  ln.sms = sms; ln.piece = pl.tc ? 10 : pl.chunk == 8 ? 64 : pl.chunk == 16 ? 32 : 24;
  const int cols = a.b.rows * ln.group;
  cudaError_t e;
  if (pl.tc) e = launch_attention_kv4_tc(st, p, a.c.dh, pl.ctas);
  else if (a.c.dh == 128) e = pl.chunk == 8 ? launch_attn<128, 1>(st, p, pl.ctas) : pl.chunk == 16 ? launch_attn<128, 2>(st, p, pl.ctas) : launch_attn<128, 4>(st, p, pl.ctas);
  else e = pl.chunk == 8 ? launch_attn<64, 1>(st, p, pl.ctas) : pl.chunk == 16 ? launch_attn<64, 2>(st, p, pl.ctas) : launch_attn<64, 4>(st, p, pl.ctas);
  if (e != cudaSuccess) return e;
  return a.c.dh == 128 ? launch_join<128>(st, p, pl.ctas, cols) : launch_join<64>(st, p, pl.ctas, cols);
}

// ---- weights -----------------------------------------------------------------------------------------------------------
// w_out = w_in + the probabilities exp(scale q . k - lse) of a key, summed over the columns of its head.  The scores alone: the first half
// of a cache tile, codes and (s, m) of K.  A warp keeps 32 keys as A fragments in registers and passes the columns by them, whose B
// fragments lie in shared memory for all warps of the CTA; more than 64 columns in several passes over the CTA's run.
//
// Few columns: bound by memory (16 x 1 token of 32/8 heads on 30000 keys: 64 us, 4.6 TB/s with the sums).  Many: by the products, 16
// MMAs of 8 cycles for 32 keys and 8 columns (8 x 32 rows of 32 heads on 2048 keys: 21 us, the products alone 7.8), and by the
// launch, the queries' conversion in every CTA and the exponentials beside them.
namespace {

struct WeighParams {
  Kv4View c;
  Line line;
  int Hq;
  const bf16 *q; const float *lse;
  int64_t q_stride;
  float scale_log2;
  const float *w_in; float *w_out;
  int32_t *status;
};

constexpr int WEIGH_COLS = 64;       // columns of a pass

template <int DH> struct WeighShape {
  static constexpr int PART = KV4_TILE * (DH / 2 + 4), STAGES = 4, RING = STAGES * PART;   // codes and (s, m) of K
  static constexpr int OFF_Q = WARPS * RING, SMEM = OFF_Q + WEIGH_COLS * DH * 2;
};

template <int DH>
__global__ void __launch_bounds__(WARPS * 32, 4) kv4_weights_kernel(const WeighParams p) {
  using Sh = WeighShape<DH>;
  constexpr int W = DH / 32, STAGES = Sh::STAGES;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ __align__(8) uint64_t bars[WARPS * STAGES];
  __shared__ __align__(16) float2 of_col[WEIGH_COLS];            // sum of the scaled queries times cf, minus the log-sum
  __shared__ __align__(16) float cf_col[WEIGH_COLS];             // cf
  __shared__ int abort_flag;
  const int warp = ptx::warp_index(), lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const uint32_t bar0 = ptx::smem_u32(&bars[warp * STAGES]);
  uint8_t *const ring = smem + warp * Sh::RING;
  const uint32_t ring_u = ptx::smem_u32(ring);
  uint4 *const qs = reinterpret_cast<uint4 *>(smem + Sh::OFF_Q);
  if (lane == 0) {
    for (int i = 0; i < STAGES; ++i) ptx::mbar_init(bar0 + 8 * i, 1);
    ptx::fence_barrier_init();
    ptx::fence_proxy_async();
  }
  if (threadIdx.x == 0) abort_flag = 0;
  __syncthreads();
  grid_dep_launch();
  grid_dep_wait();

  const Line &ln = p.line;
  const Seq own = ln.seq(lane);
  uint32_t share;
  const uint32_t total = ln.survey(own, gridDim.x, 0, &share, nullptr);
  uint32_t pos = (uint32_t)min((uint64_t)share * blockIdx.x, (uint64_t)total);
  const uint32_t end = min(total, pos + share);
  uint32_t used = 0;
  while (pos < end) {
    uint32_t before;
    const Seq sq = ln.find(own, pos, &before);
    const int nt = sq.tiles, h = (int)((pos - before) / nt), t0 = (int)(pos - before) - h * nt, t1 = (int)min((uint32_t)nt, t0 + (end - pos));
    const int cols = sq.rows * ln.group;
    const uint8_t *src = p.c.tile(sq.slot, h, 0);
    const int64_t w_at = ((int64_t)sq.slot * p.c.heads + h) * p.c.cap;
    pos += t1 - t0;
    const int mine = (t1 - t0 - warp + WARPS - 1) / WARPS;   // this warp's tiles: t0 + warp, + WARPS, ...
    for (int c0 = 0; c0 == 0 || c0 < cols; c0 += WEIGH_COLS) {
      const int here = min(WEIGH_COLS, cols - c0), nts = (here + 7) / 8;
      auto request = [&](int i) {
        if (i < mine && ptx::elect_one()) {
          const uint32_t s = (used + i) % STAGES;
          ptx::mbar_arrive_expect_tx(bar0 + 8 * s, Sh::PART);
          ptx::bulk_load(ring_u + s * Sh::PART, src + (int64_t)(t0 + warp + i * WARPS) * kv4_tile_bytes(DH), Sh::PART, bar0 + 8 * s);
        }
      };
      for (int i = 0; i < STAGES; ++i) request(i);
      // queries: each warp converts every fourth eight of columns
      for (int n = warp; n < nts; n += WARPS) {
        const int col = c0 + 8 * n + g, r = col / ln.group, row = sq.row0 + r, head = h * ln.group + col - r * ln.group;
        const bool there = 8 * n + g < here;
        Queries<DH> qn;
        qn.load(p.q + (int64_t)row * p.q_stride + (int64_t)head * DH + t * (DH / 4), there);
        uint32_t f[DH / 8];
        const int u = qn.exponent();
        const float sum = qn.convert(u, f), cf = query_factor(p.scale_log2, u);
        if (t == 0) {
          float l = there ? p.lse[(int64_t)row * p.Hq + head] * 1.4426950408889634f : INFINITY;
          if (l == -INFINITY) l = INFINITY;        // a row without keys gives no weight
          of_col[8 * n + g] = make_float2(sum * cf, -l);
          cf_col[8 * n + g] = cf;
        }
#pragma unroll
        for (int j = 0; j < W; ++j) qs[(n * W + j) * 32 + lane] = make_uint4(f[4 * j], f[4 * j + 1], f[4 * j + 2], f[4 * j + 3]);
      }
      __syncthreads();
      bool ok = true;
      for (int i = 0; i < mine; ++i) {
        const uint32_t s = (used + i) % STAGES;
        const int key0 = (t0 + warp + i * WARPS) * KV4_TILE, key = key0 + g + 8 * t;   // the key whose weight this lane writes
        const bool real = key < sq.keys;
        const float was = !real ? 0.f : c0 ? p.w_out[w_at + key] : p.w_in[w_at + key];
        ok = ptx::mbar_wait_warp(bar0 + 8 * s, ((used + i) / STAGES) & 1u);
        if (!ok) break;
        const uint8_t *tile = ring + s * Sh::PART;
        uint32_t k[4][W];                          // rows g, g + 8, g + 16, g + 24
        float ks[4], km[4], w[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint8_t *a = tile + (g + 8 * e) * (DH / 2) + t * (DH / 8);
          if (DH == 128) *reinterpret_cast<uint4 *>(k[e]) = *reinterpret_cast<const uint4 *>(a);
          else *reinterpret_cast<uint2 *>(k[e]) = *reinterpret_cast<const uint2 *>(a);
          const uint32_t m = *reinterpret_cast<const uint32_t *>(tile + kv4_off_kmeta(DH) + 4 * (g + 8 * e));
          ks[e] = kv4_scale(m) * K_UNIT; km[e] = kv4_min(m) * K_UNIT;
        }
        ptx::fence_proxy_async();                  // the next copy overwrites what was read: no read is put off behind it
        __syncwarp();
        request(i + STAGES);
        uint32_t x[4][4 * W];
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int j = 0; j < W; ++j) spread(k[e][j], &x[e][4 * j]);
#pragma unroll 2                                     // four sums under way: heads of 64 18.0 -> 15.6 us, of 128 22.7 -> 22.3
        for (int n = 0; n < nts; ++n) {
          float acc[2][4];
#pragma unroll
          for (int j = 0; j < W; ++j) {
            const uint4 f = qs[(n * W + j) * 32 + lane];
#pragma unroll
            for (int m = 0; m < 2; ++m) {
              if (j == 0) ptx::mma_f16_16x8x16_first(acc[m], x[2 * m][0], x[2 * m + 1][0], x[2 * m][1], x[2 * m + 1][1], f.x, f.y);
              else ptx::mma_f16_16x8x16(acc[m], x[2 * m][4 * j], x[2 * m + 1][4 * j], x[2 * m][4 * j + 1], x[2 * m + 1][4 * j + 1], f.x, f.y);
            }
#pragma unroll
            for (int m = 0; m < 2; ++m)
              ptx::mma_f16_16x8x16(acc[m], x[2 * m][4 * j + 2], x[2 * m + 1][4 * j + 2], x[2 * m][4 * j + 3], x[2 * m + 1][4 * j + 3], f.z, f.w);
          }
          const float4 of = *reinterpret_cast<const float4 *>(&of_col[8 * n + 2 * t]);   // columns 2t and 2t + 1
          const float2 cf2 = *reinterpret_cast<const float2 *>(&cf_col[8 * n + 2 * t]);
          const F2 cf = ptx::f2(cf2.x, cf2.y);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float *a = &acc[e >> 1][2 * (e & 1)];
            const F2 x = ptx::mul2(ptx::f2(a[0], a[1]), cf);
            w[e] += ptx::ex2(fmaf(ptx::f2_lo(x), ks[e], fmaf(km[e], of.x, of.y))) + ptx::ex2(fmaf(ptx::f2_hi(x), ks[e], fmaf(km[e], of.z, of.w)));
          }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          w[e] += __shfl_xor_sync(0xffffffffu, w[e], 1);
          w[e] += __shfl_xor_sync(0xffffffffu, w[e], 2);
        }
        const float sum = t == 0 ? w[0] : t == 1 ? w[1] : t == 2 ? w[2] : w[3];
        if (real) p.w_out[w_at + key] = was + sum;
      }
      if (!ok) { fail(p.status, DEV_TIMEOUT_EPILOGUE); abort_flag = 1; }
      used += max(mine, 0);
      __syncthreads();                             // the queries may be overwritten
      if (abort_flag) break;
    }
    if (abort_flag) break;
  }
  if (abort_flag) {                                // a wait ran out: copies in flight land before shared memory goes away
    const uint64_t start = ptx::globaltimer();
    while (ptx::globaltimer() - start < 200000ull) __nanosleep(1000);
  }
}

template <int DH> cudaError_t launch_weigh(cudaStream_t st, const WeighParams &p, int ctas) {
  constexpr int smem = WeighShape<DH>::SMEM;
  static std::atomic<uint64_t> done{0};
  const cudaError_t e = allow_shared((const void *)kv4_weights_kernel<DH>, smem, done);
  if (e != cudaSuccess) return e;
  return launch_kernel(kv4_weights_kernel<DH>, dim3(ctas), dim3(WARPS * 32), (size_t)smem, st, p);
}

}  // namespace

cudaError_t launch_kv4_weights(cudaStream_t st, const Kv4WeighArgs &a, int sms) {
  WeighParams p;
  p.c = a.c; p.Hq = a.Hq; p.q = a.q; p.lse = a.lse; p.q_stride = a.q_stride; p.scale_log2 = a.scale * 1.4426950408889634f;
  p.w_in = a.w_in; p.w_out = a.w_out; p.status = a.status;
  Line &ln = p.line;
  // one item a head, whatever its columns: a key's weight is written by one thread.  Sequences without rows too: their weights are copied
  ln.B = a.b.B; ln.H = a.c.heads; ln.chunk = 0x7fffffff; ln.min_chunks = 1; ln.group = a.Hq / a.c.heads; ln.slots = a.c.slots;
  ln.max_keys = a.max_len < a.c.cap ? a.max_len : a.c.cap; ln.tile_keys = KV4_TILE; ln.b = a.b; ln.sms = sms; ln.piece = 32;
  const int64_t want = ceil_div64((int64_t)a.b.B * a.c.heads * ceil_div(ln.max_keys, KV4_TILE), WARPS);
  const int ctas = (int)(want < 1 ? 1 : want < sms * 4 ? want : sms * 4);
  return a.c.dh == 128 ? launch_weigh<128>(st, p, ctas) : launch_weigh<64>(st, p, ctas);
}

}  // namespace l2pd
