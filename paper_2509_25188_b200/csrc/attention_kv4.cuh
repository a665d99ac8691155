// What the two attention kernels over the 4-bit cache share (internal): the line of work, parameters, partial results.
#pragma once
#include "kv4.cuh"
#include "ptx.cuh"

namespace l2pd {
namespace kv4 {

// Log2 units by which a reference is set below the largest, and by which the largest may pass it before it is moved.  A probability is below
// 2^15 then, within fp16, and vanishes 2^34 below the largest (without the first, a million keys 2^25 below one would, with 3 % of the output).
constexpr float BELOW = 9.0f, LAZY = 15.0f;

// ---- one unit for values of any size -----------------------------------------------------------------------------------
// A key's probability goes to the product as p' = 2^(log2 w - M + b), w its weight, b = the exponent of its values - E, E one that no value
// has passed so far.  Two sums then stand for the output: O = sum p' v 2^-(E + b) = sum w v 2^(-E - M), and l = sum p' 2^-b = sum w 2^-M.
// Where E rises by d, M is lowered by d: what is in O stays, the keys to come keep their bits whatever the size of the row that raised E
// (which may have no weight at all), and l alone grows by 2^d.  l is at least 1, and as large as the values that have the weight are
// smaller than E: it is kept as l 2^-LOG_L, which bears 2^180.  FLOOR: the least b, so that p' is no zero where w counts; values 2^100
// below the largest so far lose their size, rows of zeros take it.
constexpr int LOG_L = 80;
constexpr float FLOOR = -100.f;

__device__ __forceinline__ float pow2(int n) { return __uint_as_float((uint32_t)(127 + n) << 23); }   // -126 <= n <= 127
// x 2^d for d beyond one exponent's range
__device__ __forceinline__ float ex2_scaled(float x, float d) { const float h = ptx::ex2(0.5f * d); return x * h * h; }
// A sum l 2^-LOG_L against the reference M, as x 2^ref with x in [1, 2): sums against references far apart can then be added, and so can the
// outputs that stand in the unit x 2^ref.  They come from O in the unit 2^unit by the two powers.  0: a sum of nothing; NaN stays.
struct Normal { float x, ref, up_a, up_b; };
__device__ __forceinline__ Normal normalised(float l, float m, int unit) {
  const uint32_t u = __float_as_uint(l) & 0x7fffffffu;
  const int e = (int)(u >> 23), k = e - 127 + LOG_L, n = max(unit - k, -250), h = n >> 1;
  Normal r;
  r.x = e == 255 ? l : e ? __uint_as_float((u & 0x7fffffu) | 0x3f800000u) : 0.f;
  r.ref = e ? m + (float)k : -INFINITY;
  r.up_a = e ? pow2(h) : 0.f; r.up_b = pow2(n - h);
  return r;
}

// ---- the line of work --------------------------------------------------------------------------------------------------
// Items: for sequence b, key heads times chunks of `chunk` columns (those that have rows), tiles_b key tiles each.  Fewer than 2^31
// tiles in all (the host sees to it).  Every warp surveys the line for itself, a lane a sequence: the lengths and rows of 32
// sequences are one round of loads.
struct Seq { int keys, rows, row0, slot, tiles, chunks; uint32_t count; };
struct Line {
  int B, H, chunk, group, slots, max_keys, tile_keys, min_chunks, sms, piece;   // piece: see survey
  Kv4Batch b;
  __device__ __forceinline__ Seq seq(int s) const {
    Seq q = {0, 0, 0, -1, 0, 0, 0u};
    if (s >= B) return q;
    const int len = b.keys[s];
    q.rows = b.n_rows(s); q.row0 = b.row0(s); q.slot = b.slot(s, slots);
    q.keys = q.slot < 0 ? 0 : max(0, min(len, max_keys));
    q.tiles = (q.keys + tile_keys - 1) / tile_keys;
    q.chunks = max(min_chunks, (int)(((uint32_t)(q.rows * group) + (uint32_t)chunk - 1u) / (uint32_t)chunk));
    q.count = (uint32_t)H * q.chunks * q.tiles;
    return q;
  }
  // Tiles of the line and of a CTA's run; *before: tiles of the sequences ahead of `upto`.  `own` is seq(lane).  (Whole warp.)
  // Equal runs split items, and every piece of one costs a CTA its queries, its output and, split, a way through memory: about what
  // an SM takes for `piece` tiles (measured, as is 1.15).  Sequences of one length: whole items where the SM with most of them is done sooner
  // (8 x 16 rows of 32 heads on 512 keys: 19 us split, 16 whole; on 8192 keys 79 split; 8 x 32 rows on 2048 keys 43.8 split, 43.2 whole).
  // An SM with fewer CTAs than fit takes longer for a tile.
  __device__ uint32_t survey(const Seq &own, uint32_t ctas, int upto, uint32_t *share, uint32_t *before) const {
    const int lane = threadIdx.x & 31;
    uint32_t total = 0, ahead = 0, lo = 0xffffffffu, hi = 0;
    Seq q = own;
    for (int s0 = 0;;) {
      total += __reduce_add_sync(0xffffffffu, q.count);
      ahead += __reduce_add_sync(0xffffffffu, s0 + lane < upto ? q.count : 0u);
      lo = min(lo, __reduce_min_sync(0xffffffffu, q.chunks ? (uint32_t)q.tiles : 0xffffffffu));
      hi = max(hi, __reduce_max_sync(0xffffffffu, q.chunks ? (uint32_t)q.tiles : 0u));
      if ((s0 += 32) >= B) break;
      q = seq(s0 + lane);
    }
    uint32_t even = (total + ctas - 1) / ctas;
    if (lo == hi && hi) {
      const uint32_t items = total / hi, rounds = (items + ctas - 1) / ctas;
      const uint32_t per_sm = (items + sms - 1) / sms;
      const float most = items <= ctas ? (per_sm * sms < ctas ? 1.15f : 1.f) * per_sm * hi : (float)rounds * hi * ctas / sms;
      if (most + (float)piece * rounds <= (float)total / sms + (float)piece * (1.f + (float)even / hi)) even = rounds * hi;
    }
    *share = even;
    if (before) *before = ahead;
    return total;
  }
  // The sequence that tile `pos` of the line belongs to, and the tiles before it.  (Whole warp, pos below the line's end.)
  __device__ Seq find(const Seq &own, uint32_t pos, uint32_t *start) const {
    const int lane = threadIdx.x & 31;
    uint32_t run = 0;
    Seq q = own;
    for (int s0 = 0;;) {
      uint32_t x = q.count;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
      }
      const unsigned here = __ballot_sync(0xffffffffu, pos < run + x);
      if (here || s0 + 32 >= B) {
        const int l = here ? __ffs(here) - 1 : 31;
        *start = run + __shfl_sync(0xffffffffu, x - q.count, l);
        Seq r;
        r.keys = __shfl_sync(0xffffffffu, q.keys, l); r.rows = __shfl_sync(0xffffffffu, q.rows, l);
        r.row0 = __shfl_sync(0xffffffffu, q.row0, l); r.slot = __shfl_sync(0xffffffffu, q.slot, l);
        r.tiles = __shfl_sync(0xffffffffu, q.tiles, l); r.chunks = __shfl_sync(0xffffffffu, q.chunks, l);
        r.count = 0;
        return r;
      }
      run += __shfl_sync(0xffffffffu, x, 31);
      q = seq((s0 += 32) + lane);
    }
  }
};

struct AttnParams {
  Kv4View c;
  Line line;
  int Hq;
  const bf16 *q; bf16 *out; float *lse;
  int64_t q_stride, out_stride;
  float scale_log2;
  float *part;             // [2 * CTAs][chunk][dh + 4]: of a partial item O, reference, sum of weights
  int32_t *status;
};

__host__ __device__ constexpr int part_floats(int chunk, int dh) { return chunk * (dh + 4); }

__device__ __forceinline__ void fail(int32_t *status, int code) { if (status) atomicCAS(status, 0, code); }

// attention_kv4_tc.cu: chunks of 64 or 128 columns on tcgen05 (chunk: line.chunk; ctas: at most an SM each)
cudaError_t launch_attention_kv4_tc(cudaStream_t st, const AttnParams &p, int dh, int ctas);
constexpr int TC_TILE = 128;         // its key tiles

}  // namespace kv4
}  // namespace l2pd
