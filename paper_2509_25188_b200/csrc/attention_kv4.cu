// Attention over a key/value cache in 4 bits, and the sum of the weights each key receives.
//
// The columns of a (sequence, key head) are its query rows times the query heads that share the key head.  Scores are computed as
// S^T = K Q^T, keys on the M side of mma.sync.m16n8k16, so that one query row pads to 8 columns instead of 16 rows, and the
// output as O^T = V^T P^T.  A code c in the low four bits of an fp16 is the subnormal number c 2^-24, exactly: the codes go to the
// product as they lie, by a mask (those in bits 4..7 as 16 c 2^-24, against queries divided by 16).  With q' = q scaled by a power
// of two into fp16's range (8 significant bits of 11):
//     t_j = log2 of exp(scale q . k_j) + e_j = cf (s_j sum(c q') + m_j sum(q')) + e_j - E
// 2^e_j bounds the value row's s_j and |m_j| / 16, E the largest e_j.  Probabilities are taken as p'_j = 2^(t_j - M), M a reference at
// most 2^6 below the running maximum of t, so that p'_j s_j 2^-e_j, what multiplies the codes of V, stays within fp16 whatever the
// values' magnitude.  (e_j is at least E - 60, so that a row of zeros keeps its part of the sum of probabilities p'_j 2^(E - e_j).)
// Rounding it to fp16 is the only step to less than 32 bits between the queries and the output.
//
// Work: the key tiles of all (sequence, head, chunk of columns) stand in one line and every CTA takes an equal run of it; a run
// that starts or ends inside an item leaves a partial result, joined in the order of the tiles by a second kernel.  A warp takes
// every eighth tile of its CTA's run, through a ring of its own.
#include <cuda_fp16.h>
#include <math.h>

#include "kv4.cuh"
#include "ptx.cuh"

namespace l2pd {

namespace {

constexpr int WARPS = 8, STAGES = 3;
constexpr float LAZY = 6.0f;         // log2 units the running maximum may pass the reference

// ---- the line of work --------------------------------------------------------------------------------------------------
// Items: for sequence b, key heads times chunks of CH columns (those that have rows), tiles_b key tiles each.
struct Line {
  int B, H, chunk, group, slots, max_keys;
  Kv4Batch b;
  __device__ __forceinline__ int keys(int s) const { return b.slot(s, slots) < 0 ? 0 : max(0, min(b.keys[s], max_keys)); }
  __device__ __forceinline__ int chunks(int s) const { return (b.n_rows(s) * group + chunk - 1) / chunk; }
  __device__ __forceinline__ int tiles(int s) const { return (keys(s) + KV4_TILE - 1) / KV4_TILE; }
  __device__ __forceinline__ int64_t all_tiles(int s) const { return (int64_t)H * chunks(s) * tiles(s); }
  // tiles of the sequences [0, s), every lane of the warp receives it (whole warp)
  __device__ int64_t before(int s) const {
    int64_t x = 0;
    for (int i = threadIdx.x & 31; i < s; i += 32) x += all_tiles(i);
#pragma unroll
    for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
  }
};

struct AttnParams {
  Kv4View c;
  Line line;
  int Hq;
  const bf16 *q; bf16 *out; float *lse;
  int64_t q_stride, out_stride;
  float scale_log2;
  float *part;             // [2 * CTAs][chunk][dh + 4]: O, M, L of a partial item
  int32_t *status;
};

__host__ __device__ constexpr int part_floats(int chunk, int dh) { return chunk * (dh + 4); }

__device__ __forceinline__ void fail(int32_t *status, int code) { if (status) atomicCAS(status, 0, code); }

// The four registers of two MMA steps in a word of eight codes: codes 0 and 4, 1 and 5 (times 16), 2 and 6, 3 and 7 (times 16).
__device__ __forceinline__ void spread(uint32_t w, uint32_t *r) {
  r[0] = w & 0x000f000fu; r[1] = w & 0x00f000f0u;
  w >>= 8;
  r[2] = w & 0x000f000fu; r[3] = w & 0x00f000f0u;
}

// tile row of MMA row k (0..7): odd and even rows change places in every other pair, see kv4.cuh on banks
__device__ __forceinline__ int tile_row(int k) { return k ^ ((k >> 1) & 1); }

// Queries of eight columns as B fragments: lane (g, t) holds of column g the dimensions [t dh/4, (t + 1) dh/4).
// csum: sum of the column's scaled queries in the scale of the codes' products, cf: what turns those into log2 scores.
template <int DH>
__device__ __forceinline__ void load_queries(const bf16 *q, bool there, float scale_log2, uint32_t (&f)[DH / 8], float &cf, float &csum) {
  constexpr int W = DH / 32;                       // words of codes a lane holds: 8 dimensions each
  uint32_t raw[DH / 8];
#pragma unroll
  for (int j = 0; j < W; ++j) {
    const uint4 x = there ? *reinterpret_cast<const uint4 *>(q + 8 * j) : make_uint4(0, 0, 0, 0);
    raw[4 * j] = x.x; raw[4 * j + 1] = x.y; raw[4 * j + 2] = x.z; raw[4 * j + 3] = x.w;
  }
  uint32_t top = 0;                                // largest magnitude, as bits: infinities and NaN above all
  float x[DH / 4];
#pragma unroll
  for (int i = 0; i < DH / 8; ++i) {
    x[2 * i] = __uint_as_float(raw[i] << 16); x[2 * i + 1] = __uint_as_float(raw[i] & 0xffff0000u);
    top = max(top, max(__float_as_uint(x[2 * i]) & 0x7fffffffu, __float_as_uint(x[2 * i + 1]) & 0x7fffffffu));
  }
  top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
  top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
  // the largest becomes 2^14 .. 2^15
  const int e = (int)(top >> 23) - 127;
  const float up = __uint_as_float((uint32_t)(127 + min(14 - e, 126)) << 23);
  cf = scale_log2 * 1024.f * __uint_as_float((uint32_t)(127 - min(14 - e, 126) + 14) << 23);   // 2^24 / up
  if (e == 128) cf = __uint_as_float(0x7fc00000u);   // infinity or NaN among the queries: the column is NaN
  csum = 0.f;
#pragma unroll
  for (int i = 0; i < DH / 4; ++i) {
    x[i] = e == 128 ? 0.f : x[i] * up;
    csum += x[i];
  }
  csum += __shfl_xor_sync(0xffffffffu, csum, 1);
  csum += __shfl_xor_sync(0xffffffffu, csum, 2);
  csum *= __uint_as_float((127 - 24) << 23);
#pragma unroll
  for (int j = 0; j < W; ++j) {
    const float *y = x + 8 * j;
    auto pair = [](float a, float b) { __half2 h = __floats2half2_rn(a, b); return *reinterpret_cast<uint32_t *>(&h); };
    f[4 * j] = pair(y[0], y[4]); f[4 * j + 1] = pair(y[1] * 0.0625f, y[5] * 0.0625f);
    f[4 * j + 2] = pair(y[2], y[6]); f[4 * j + 3] = pair(y[3] * 0.0625f, y[7] * 0.0625f);
  }
}

template <int DH, int NT>
__global__ void __launch_bounds__(WARPS * 32, 1) attention_kv4_kernel(const AttnParams p) {
  constexpr int W = DH / 32, MT = DH / 16, CH = 8 * NT, MS = 4 / NT;   // MS: groups of 16 keys taken together
  constexpr int TILE = KV4_TILE * (DH + 8), RING = STAGES * TILE, LDO = DH + 4;
  static_assert(CH * LDO * 4 <= RING, "a warp's output goes to its ring");
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ __align__(8) uint64_t bars[WARPS * STAGES];
  __shared__ float fin[WARPS][3][CH];              // reference, sum of probabilities, sum of probability times m
  __shared__ int abort_flag;
  const int warp = ptx::warp_index(), lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const uint32_t bar0 = ptx::smem_u32(&bars[warp * STAGES]);
  uint8_t *const ring = smem + warp * RING;
  const uint32_t ring_u = ptx::smem_u32(ring);
  if (lane == 0)
    for (int i = 0; i < STAGES; ++i) ptx::mbar_init(bar0 + 8 * i, 1);
  if (threadIdx.x == 0) abort_flag = 0;
  if (lane == 0) { ptx::fence_barrier_init(); ptx::fence_proxy_async(); }
  __syncthreads();
  grid_dep_launch();
  grid_dep_wait();

  const Line &ln = p.line;
  const int64_t total = ln.before(ln.B), share = (total + gridDim.x - 1) / gridDim.x;
  int64_t pos = share * blockIdx.x;
  const int64_t end = min(total, pos + share);
  uint32_t used = 0;                               // tiles this warp has taken: stage and parity
  int b = -1;
  int64_t b_start = 0, b_tiles = 0;
  while (pos < end) {
    while (b < 0 || pos >= b_start + b_tiles) { b_start += b_tiles; ++b; b_tiles = ln.all_tiles(b); }
    const int n_keys = ln.keys(b), nt = ln.tiles(b), nc = ln.chunks(b), rows = ln.b.n_rows(b), row0 = ln.b.row0(b);
    const int64_t in_b = pos - b_start;
    const int item = (int)(in_b / nt), t0 = (int)(in_b - (int64_t)item * nt), t1 = (int)min((int64_t)nt, t0 + (end - pos));
    const int h = item / nc, c0 = (item - h * nc) * CH, cols = min(CH, rows * ln.group - c0);
    const uint8_t *src = p.c.tile(ln.b.slot(b, ln.slots), h, 0);
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

    uint32_t qf[NT][DH / 8];
    float cfa[NT], cfb[NT], za[NT], zb[NT];        // of the columns 2t and 2t + 1 of each eight
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int col = c0 + 8 * n + g, r = col / ln.group;
      const bool there = 8 * n + g < cols;
      float cf, cs;
      load_queries<DH>(p.q + (int64_t)(row0 + r) * p.q_stride + (int64_t)(h * ln.group + col - r * ln.group) * DH + t * (DH / 4), there,
                       p.scale_log2, qf[n], cf, cs);
      cs *= cf;
      cfa[n] = __shfl_sync(0xffffffffu, cf, 8 * t); cfb[n] = __shfl_sync(0xffffffffu, cf, 8 * t + 4);
      za[n] = __shfl_sync(0xffffffffu, cs, 8 * t); zb[n] = __shfl_sync(0xffffffffu, cs, 8 * t + 4);
    }
    float o[MT][NT][4], la[NT], lb[NT], wa[NT], wb[NT], ma[NT], mb[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      la[n] = lb[n] = wa[n] = wb[n] = 0.f; ma[n] = mb[n] = -INFINITY;
#pragma unroll
      for (int m = 0; m < MT; ++m) o[m][n][0] = o[m][n][1] = o[m][n][2] = o[m][n][3] = 0.f;
    }
    int e0 = -1000;                                // E
    bool ok = true;
    for (int i = 0; i < mine; ++i) {
      const uint32_t s = (used + i) % STAGES;
      ok = ptx::mbar_wait_warp(bar0 + 8 * s, ((used + i) / STAGES) & 1u);
      if (!ok) break;
      const uint8_t *tile = ring + s * TILE;
      const int left = n_keys - (t0 + warp + i * WARPS) * KV4_TILE;    // keys of this tile, or more
#pragma unroll 1
      for (int s0 = 0; s0 < 4; s0 += MS) {
        float acc[MS][NT][4];
#pragma unroll
        for (int u = 0; u < MS; ++u)
#pragma unroll
          for (int n = 0; n < NT; ++n) acc[u][n][0] = acc[u][n][1] = acc[u][n][2] = acc[u][n][3] = 0.f;
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
        for (int j = 0; j < W; ++j)
#pragma unroll
          for (int u = 0; u < MS; ++u) {
            uint32_t x[4], y[4];
            spread(ka[u][j], x); spread(kb[u][j], y);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              ptx::mma_f16_16x8x16(acc[u][n], x[0], y[0], x[1], y[1], qf[n][4 * j], qf[n][4 * j + 1]);
              ptx::mma_f16_16x8x16(acc[u][n], x[2], y[2], x[3], y[3], qf[n][4 * j + 2], qf[n][4 * j + 3]);
            }
          }
        // what belongs to a key: s and m of K; of V the exponent e, 2^-e, s 2^-e and m 2^-e
        float vs[MS][2], vm[MS][2], vw[MS][2];
        uint32_t vmeta[MS][2];
        int ex[MS][2], ex_top = -126;
#pragma unroll
        for (int u = 0; u < MS; ++u)
#pragma unroll
          for (int e2 = 0; e2 < 2; ++e2) {
            const int k = kr + 16 * u + 8 * e2;
            vmeta[u][e2] = k < left ? *reinterpret_cast<const uint32_t *>(tile + kv4_off_vmeta(DH) + 4 * k) : 0u;
            ex[u][e2] = min(max((int)((vmeta[u][e2] >> 7) & 255u), (int)((vmeta[u][e2] >> 23) & 255u) - 4) - 126, 100);
            ex_top = max(ex_top, ex[u][e2]);
          }
        ex_top = __reduce_max_sync(0xffffffffu, ex_top);
        if (ex_top > e0) {                         // rare: what came before is in units of 2^e0
          const int up = e0;
          e0 = max(ex_top, -100) + 2;
          const float f = __uint_as_float((uint32_t)max(127 - (e0 - up), 0) << 23);
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            wa[n] *= f; wb[n] *= f;
#pragma unroll
            for (int m = 0; m < MT; ++m) { o[m][n][0] *= f; o[m][n][1] *= f; o[m][n][2] *= f; o[m][n][3] *= f; }
          }
        }
#pragma unroll
        for (int u = 0; u < MS; ++u)
#pragma unroll
          for (int e2 = 0; e2 < 2; ++e2) {
            const int k = kr + 16 * u + 8 * e2;
            const bool real = k < left;
            const uint32_t km = real ? *reinterpret_cast<const uint32_t *>(tile + kv4_off_kmeta(DH) + 4 * k) : 0u;
            const int e = max(ex[u][e2], e0 - 60);
            const float w = __uint_as_float((uint32_t)(127 - e) << 23), bias = real ? (float)(e - e0) : -INFINITY;
            vw[u][e2] = __uint_as_float((uint32_t)(127 - e + e0) << 23); vs[u][e2] = kv4_scale(vmeta[u][e2]) * w; vm[u][e2] = kv4_min(vmeta[u][e2]) * w;
            const float ks = kv4_scale(km), kmin = kv4_min(km);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              float &ta = acc[u][n][2 * e2], &tb = acc[u][n][2 * e2 + 1];
              ta = fmaf(ta * cfa[n], ks, fmaf(kmin, za[n], bias)) - (ma[n] == -INFINITY ? 0.f : ma[n]);
              tb = fmaf(tb * cfb[n], ks, fmaf(kmin, zb[n], bias)) - (mb[n] == -INFINITY ? 0.f : mb[n]);
            }
          }
        // a new reference where the maximum has passed the old one by LAZY (or there was none)
        bool grow = false;
        float xa[NT], xb[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          xa[n] = xb[n] = -INFINITY;
#pragma unroll
          for (int u = 0; u < MS; ++u) {
            xa[n] = fmaxf(xa[n], fmaxf(acc[u][n][0], acc[u][n][2]));
            xb[n] = fmaxf(xb[n], fmaxf(acc[u][n][1], acc[u][n][3]));
          }
          grow = grow || xa[n] > LAZY || xb[n] > LAZY || (ma[n] == -INFINITY && xa[n] > -INFINITY) || (mb[n] == -INFINITY && xb[n] > -INFINITY);
        }
        if (__any_sync(0xffffffffu, grow)) {
#pragma unroll
          for (int n = 0; n < NT; ++n) {
#pragma unroll
            for (int x = 4; x < 32; x <<= 1) {
              xa[n] = fmaxf(xa[n], __shfl_xor_sync(0xffffffffu, xa[n], x));
              xb[n] = fmaxf(xb[n], __shfl_xor_sync(0xffffffffu, xb[n], x));
            }
            const bool fa = ma[n] == -INFINITY, fb = mb[n] == -INFINITY;   // no key yet
            const float da = fa ? (xa[n] == -INFINITY ? 0.f : xa[n]) : fmaxf(xa[n], 0.f), db = fb ? (xb[n] == -INFINITY ? 0.f : xb[n]) : fmaxf(xb[n], 0.f);
            const float sa = fa ? 0.f : ptx::ex2(-da), sb = fb ? 0.f : ptx::ex2(-db);
            ma[n] = fa ? (xa[n] == -INFINITY ? -INFINITY : xa[n]) : ma[n] + da;
            mb[n] = fb ? (xb[n] == -INFINITY ? -INFINITY : xb[n]) : mb[n] + db;
            la[n] *= sa; lb[n] *= sb; wa[n] *= sa; wb[n] *= sb;
#pragma unroll
            for (int m = 0; m < MT; ++m) { o[m][n][0] *= sa; o[m][n][2] *= sa; o[m][n][1] *= sb; o[m][n][3] *= sb; }
#pragma unroll
            for (int u = 0; u < MS; ++u) { acc[u][n][0] -= da; acc[u][n][2] -= da; acc[u][n][1] -= db; acc[u][n][3] -= db; }
          }
        }
#pragma unroll
        for (int u = 0; u < MS; ++u) {
          uint32_t pf[NT][2];
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e2 = 0; e2 < 2; ++e2) {
              const float pa = ptx::ex2(acc[u][n][2 * e2]), pb = ptx::ex2(acc[u][n][2 * e2 + 1]);
              la[n] = fmaf(pa, vw[u][e2], la[n]); lb[n] = fmaf(pb, vw[u][e2], lb[n]);
              wa[n] = fmaf(pa, vm[u][e2], wa[n]); wb[n] = fmaf(pb, vm[u][e2], wb[n]);
              __half2 hp = __floats2half2_rn(pa * vs[u][e2], pb * vs[u][e2]);
              pf[n][e2] = ptx::transpose_8x8(*reinterpret_cast<uint32_t *>(&hp));
            }
          // values: lane (g, t) holds dimensions [g dh/8, (g + 1) dh/8) of the keys of MMA columns 2t, 2t + 1, 2t + 8, 2t + 9
          constexpr int VW = DH / 64;
          uint32_t va[4][VW];
          const int vr = 16 * (s0 + u) + tile_row(2 * t), vr1 = 16 * (s0 + u) + tile_row(2 * t + 1);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int r = (e & 1 ? vr1 : vr) + 8 * (e >> 1);
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
      __syncwarp();
      request(i + STAGES);
    }
    if (!ok) { fail(p.status, DEV_TIMEOUT_EPILOGUE); abort_flag = 1; }
    used += max(mine, 0);

    // the warps meet: every warp's sums and outputs go to shared memory, each against its own reference
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
      for (int x = 4; x < 32; x <<= 1) {
        la[n] += __shfl_xor_sync(0xffffffffu, la[n], x); lb[n] += __shfl_xor_sync(0xffffffffu, lb[n], x);
        wa[n] += __shfl_xor_sync(0xffffffffu, wa[n], x); wb[n] += __shfl_xor_sync(0xffffffffu, wb[n], x);
      }
      if (g == 0) {
        fin[warp][0][8 * n + 2 * t] = ma[n]; fin[warp][0][8 * n + 2 * t + 1] = mb[n];
        fin[warp][1][8 * n + 2 * t] = la[n]; fin[warp][1][8 * n + 2 * t + 1] = lb[n];
      }
      float *oa = reinterpret_cast<float *>(ring) + (8 * n + 2 * t) * LDO + g * (DH / 8), *ob = oa + LDO;
      constexpr float EVEN = 16777216.f, ODD = 1048576.f;             // the codes' 2^24, and 2^20 where they came 16 times
      const float unit = __uint_as_float((uint32_t)(127 + max(e0, -126)) << 23);
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        *reinterpret_cast<float2 *>(oa + 2 * m) = make_float2(fmaf(o[m][n][0], EVEN, wa[n]) * unit, fmaf(o[m][n][2], ODD, wa[n]) * unit);
        *reinterpret_cast<float2 *>(ob + 2 * m) = make_float2(fmaf(o[m][n][1], EVEN, wb[n]) * unit, fmaf(o[m][n][3], ODD, wb[n]) * unit);
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
      float l = 0.f;
      float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < WARPS; ++w) {
        const float mw = fin[w][0][c], f = mw == -INFINITY ? 0.f : ptx::ex2(mw - m);
        const float4 z = *reinterpret_cast<const float4 *>(smem + w * RING + (c * LDO + d) * 4);
        l = fmaf(fin[w][1][c], f, l);
        y.x = fmaf(z.x, f, y.x); y.y = fmaf(z.y, f, y.y); y.z = fmaf(z.z, f, y.z); y.w = fmaf(z.w, f, y.w);
      }
      if (whole) {
        const int col = c0 + c, r = col / ln.group, hq = h * ln.group + col - r * ln.group;
        const float inv = 1.f / l;
        __nv_bfloat162 y0 = __floats2bfloat162_rn(y.x * inv, y.y * inv), y1 = __floats2bfloat162_rn(y.z * inv, y.w * inv);
        uint2 pk = make_uint2(*reinterpret_cast<uint32_t *>(&y0), *reinterpret_cast<uint32_t *>(&y1));
        *reinterpret_cast<uint2 *>(p.out + (int64_t)(row0 + r) * p.out_stride + (int64_t)hq * DH + d) = pk;
        if (d == 0 && p.lse) p.lse[(int64_t)(row0 + r) * p.Hq + hq] = (m + log2f(l)) * 0.6931471805599453f;
      } else {
        *reinterpret_cast<float4 *>(part + c * LDO + d) = y;
        if (d == 0) { part[c * LDO + DH] = m; part[c * LDO + DH + 1] = l; }
      }
    }
    ptx::fence_proxy_async();                      // the ring was written by the threads: the next copies come after
    __syncthreads();
  }
  if (abort_flag) {                                // a wait ran out: copies in flight land before shared memory goes away
    const uint64_t t0 = ptx::globaltimer();
    while (ptx::globaltimer() - t0 < 200000ull) __nanosleep(1000);
  }
}

// Joins the partial results of an item, in the order of its tiles; a block has one column of it.  Sequences without keys: output
// 0, log-sum -inf.
template <int DH>
__global__ void __launch_bounds__(128) kv4_join_kernel(const AttnParams p, int n_ctas) {
  constexpr int LDO = DH + 4;
  __shared__ float sm_m[4], sm_l[4];
  __shared__ float4 sm_o[4][32];
  grid_dep_launch();
  const Line &ln = p.line;
  const int b = blockIdx.y, h = blockIdx.z, col = blockIdx.x, lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  grid_dep_wait();
  if (col >= ln.b.n_rows(b) * ln.group) return;
  const int nt = ln.tiles(b), nc = ln.chunks(b), r = col / ln.group, hq = h * ln.group + col - r * ln.group;
  const int64_t row = ln.b.row0(b) + r;
  bf16 *out = p.out + row * p.out_stride + (int64_t)hq * DH + 4 * lane;
  float *lse = p.lse ? p.lse + row * p.Hq + hq : nullptr;
  const bool mine = 4 * lane < DH;
  if (nt == 0) {
    if (w == 0 && mine) *reinterpret_cast<uint2 *>(out) = make_uint2(0u, 0u);
    if (threadIdx.x == 0 && lse) *lse = -INFINITY;
    return;
  }
  const int64_t total = ln.before(ln.B), share = (total + n_ctas - 1) / n_ctas;
  const int64_t start = ln.before(b) + ((int64_t)h * nc + col / ln.chunk) * nt;
  const int i0 = (int)(start / share), i1 = (int)((start + nt - 1) / share);
  if (i0 == i1) return;                            // stored by its CTA
  const int c = col % ln.chunk;
  float m = -INFINITY, l = 0.f;
  float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int i = i0 + w; i <= i1; i += 4) {
    const float *part = p.part + (int64_t)(2 * i + (i == i0 ? 1 : 0)) * part_floats(ln.chunk, DH) + c * LDO;
    const float pm = part[DH], pl = part[DH + 1];
    const float4 z = mine ? *reinterpret_cast<const float4 *>(part + 4 * lane) : make_float4(0.f, 0.f, 0.f, 0.f);
    const float mn = fmaxf(m, pm), f = m == -INFINITY ? 0.f : ptx::ex2(m - mn), fp = pm == -INFINITY ? 0.f : ptx::ex2(pm - mn);
    l = l * f + pl * fp;
    y.x = y.x * f + z.x * fp; y.y = y.y * f + z.y * fp; y.z = y.z * f + z.z * fp; y.w = y.w * f + z.w * fp;
    m = mn;
  }
  if (lane == 0) { sm_m[w] = m; sm_l[w] = l; }
  sm_o[w][lane] = y;
  __syncthreads();
  if (w) return;
  float mx = fmaxf(fmaxf(sm_m[0], sm_m[1]), fmaxf(sm_m[2], sm_m[3]));
  l = 0.f; y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float f = sm_m[i] == -INFINITY ? 0.f : ptx::ex2(sm_m[i] - mx);
    const float4 z = sm_o[i][lane];
    l = fmaf(sm_l[i], f, l);
    y.x = fmaf(z.x, f, y.x); y.y = fmaf(z.y, f, y.y); y.z = fmaf(z.z, f, y.z); y.w = fmaf(z.w, f, y.w);
  }
  const float inv = 1.f / l;
  if (mine) {
    __nv_bfloat162 y0 = __floats2bfloat162_rn(y.x * inv, y.y * inv), y1 = __floats2bfloat162_rn(y.z * inv, y.w * inv);
    *reinterpret_cast<uint2 *>(out) = make_uint2(*reinterpret_cast<uint32_t *>(&y0), *reinterpret_cast<uint32_t *>(&y1));
  }
  if (lane == 0 && lse) *lse = (mx + log2f(l)) * 0.6931471805599453f;
}

struct AttnPlan { int chunk, ctas; };

AttnPlan plan_attention(int heads, int B, int rows, int Hq, int max_len, int sms) {
  AttnPlan pl;
  const int cols = rows * (Hq / heads);
  pl.chunk = cols <= 8 ? 8 : cols <= 16 ? 16 : 32;
  // no more CTAs than give each warp of them a tile
  const int64_t tiles = (int64_t)B * heads * ceil_div(cols, pl.chunk) * ceil_div(max_len, KV4_TILE), want = ceil_div64(tiles, WARPS);
  pl.ctas = (int)(want < 1 ? 1 : want < sms ? want : sms);
  return pl;
}

}  // namespace

int64_t attention_kv4_scratch_floats(const Kv4View &c, int B, int rows, int Hq, int max_len, int sms) {
  const AttnPlan pl = plan_attention(c.heads, B, rows, Hq, max_len, sms);
  return (int64_t)2 * pl.ctas * part_floats(pl.chunk, c.dh);
}

template <int DH, int NT>
static cudaError_t launch_attn(cudaStream_t st, const AttnParams &p, int ctas) {
  constexpr size_t smem = (size_t)WARPS * STAGES * KV4_TILE * (DH + 8);
  cudaError_t e = cudaFuncSetAttribute(attention_kv4_kernel<DH, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e != cudaSuccess) return e;
  return launch_kernel(attention_kv4_kernel<DH, NT>, dim3(ctas), dim3(WARPS * 32), smem, st, p);
}

cudaError_t launch_attention_kv4(cudaStream_t st, const Kv4AttnArgs &a, int sms) {
  const AttnPlan pl = plan_attention(a.c.heads, a.b.B, a.b.rows, a.Hq, a.max_len, sms);
  AttnParams p;
  p.c = a.c; p.Hq = a.Hq; p.q = a.q; p.out = a.out; p.lse = a.lse; p.q_stride = a.q_stride; p.out_stride = a.out_stride;
  p.scale_log2 = a.scale * 1.4426950408889634f; p.part = a.scratch; p.status = a.status;
  Line &ln = p.line;
  ln.B = a.b.B; ln.H = a.c.heads; ln.chunk = pl.chunk; ln.group = a.Hq / a.c.heads; ln.slots = a.c.slots;
  ln.max_keys = a.max_len < a.c.cap ? a.max_len : a.c.cap; ln.b = a.b;
  const int nt = pl.chunk / 8;
  cudaError_t e;
  if (a.c.dh == 128) e = nt == 1 ? launch_attn<128, 1>(st, p, pl.ctas) : nt == 2 ? launch_attn<128, 2>(st, p, pl.ctas) : launch_attn<128, 4>(st, p, pl.ctas);
  else e = nt == 1 ? launch_attn<64, 1>(st, p, pl.ctas) : nt == 2 ? launch_attn<64, 2>(st, p, pl.ctas) : launch_attn<64, 4>(st, p, pl.ctas);
  if (e != cudaSuccess) return e;
  const dim3 grid((unsigned)(a.b.rows * ln.group), a.b.B, a.c.heads);
  if (a.c.dh == 128) return launch_kernel(kv4_join_kernel<128>, grid, dim3(128), 0, st, p, pl.ctas);
  return launch_kernel(kv4_join_kernel<64>, grid, dim3(128), 0, st, p, pl.ctas);
}

// ---- weights -----------------------------------------------------------------------------------------------------------
namespace {

struct WeighParams {
  Kv4View c;
  Line line;
  int Hq;
  const bf16 *q; const float *lse;
  int64_t q_stride;
  float scale_log2;
  const float *w_in; float *w_out;
};

// A warp takes 16 keys at a time and all columns of their head.
template <int DH>
__global__ void __launch_bounds__(256) kv4_weights_kernel(const WeighParams p) {
  constexpr int W = DH / 32;
  grid_dep_launch();
  grid_dep_wait();
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const Line &ln = p.line;
  const int b = blockIdx.y, h = blockIdx.z, key0 = blockIdx.x * 128 + (threadIdx.x >> 5) * 16;
  const int n_keys = ln.keys(b);
  if (key0 >= n_keys) return;
  const int slot = ln.b.slot(b, ln.slots), cols = ln.b.n_rows(b) * ln.group, row0 = ln.b.row0(b);
  const uint8_t *tile = p.c.tile(slot, h, key0 / KV4_TILE);
  const int kr = key0 % KV4_TILE + g;
  uint32_t ka[W], kb[W];
#pragma unroll
  for (int j = 0; j < W; ++j) {
    ka[j] = *reinterpret_cast<const uint32_t *>(tile + kr * (DH / 2) + t * (DH / 8) + 4 * j);
    kb[j] = *reinterpret_cast<const uint32_t *>(tile + (kr + 8) * (DH / 2) + t * (DH / 8) + 4 * j);
  }
  const uint32_t m0 = *reinterpret_cast<const uint32_t *>(tile + kv4_off_kmeta(DH) + 4 * kr);
  const uint32_t m1 = *reinterpret_cast<const uint32_t *>(tile + kv4_off_kmeta(DH) + 4 * kr + 32);
  float w0 = 0.f, w1 = 0.f;
  for (int n = 0; n < cols; n += 8) {
    const int col = n + g, r = col / ln.group, hq = h * ln.group + col - r * ln.group;
    const bool there = col < cols;
    uint32_t qf[DH / 8];
    float cf, cs;
    load_queries<DH>(p.q + (int64_t)(row0 + r) * p.q_stride + (int64_t)hq * DH + t * (DH / 4), there, p.scale_log2, qf, cf, cs);
    float lse = there ? p.lse[(int64_t)(row0 + r) * p.Hq + hq] * 1.4426950408889634f : INFINITY;
    if (lse == -INFINITY) lse = INFINITY;          // a row without keys gives no weight
    float acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < W; ++j) {
      uint32_t x[4], y[4];
      spread(ka[j], x); spread(kb[j], y);
      ptx::mma_f16_16x8x16(acc, x[0], y[0], x[1], y[1], qf[4 * j], qf[4 * j + 1]);
      ptx::mma_f16_16x8x16(acc, x[2], y[2], x[3], y[3], qf[4 * j + 2], qf[4 * j + 3]);
    }
    cs *= cf;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const float f = __shfl_sync(0xffffffffu, cf, 8 * t + 4 * e), z = __shfl_sync(0xffffffffu, cs, 8 * t + 4 * e);
      const float l = __shfl_sync(0xffffffffu, lse, 8 * t + 4 * e);
      w0 += ptx::ex2(fmaf(acc[e] * f, kv4_scale(m0), fmaf(kv4_min(m0), z, -l)));
      w1 += ptx::ex2(fmaf(acc[2 + e] * f, kv4_scale(m1), fmaf(kv4_min(m1), z, -l)));
    }
  }
#pragma unroll
  for (int x = 1; x < 4; x <<= 1) { w0 += __shfl_xor_sync(0xffffffffu, w0, x); w1 += __shfl_xor_sync(0xffffffffu, w1, x); }
  if (t == 0) {
    const int64_t at = ((int64_t)slot * p.c.heads + h) * p.c.cap + key0 + g;
    if (key0 + g < n_keys) p.w_out[at] = p.w_in[at] + w0;
    if (key0 + g + 8 < n_keys) p.w_out[at + 8] = p.w_in[at + 8] + w1;
  }
}

}  // namespace

cudaError_t launch_kv4_weights(cudaStream_t st, const Kv4WeighArgs &a, int sms) {
  WeighParams p;
  p.c = a.c; p.Hq = a.Hq; p.q = a.q; p.lse = a.lse; p.q_stride = a.q_stride; p.scale_log2 = a.scale * 1.4426950408889634f;
  p.w_in = a.w_in; p.w_out = a.w_out;
  Line &ln = p.line;
  ln.B = a.b.B; ln.H = a.c.heads; ln.chunk = 8; ln.group = a.Hq / a.c.heads; ln.slots = a.c.slots;
  ln.max_keys = a.max_len < a.c.cap ? a.max_len : a.c.cap; ln.b = a.b;
  const dim3 grid((unsigned)ceil_div(a.max_len, 128), a.b.B, a.c.heads);
  if (a.c.dh == 128) return launch_kernel(kv4_weights_kernel<128>, grid, dim3(256), 0, st, p);
  return launch_kernel(kv4_weights_kernel<64>, grid, dim3(256), 0, st, p);
}

}  // namespace l2pd
