// A key/value cache in 4 bits: rows written into it, read back as values, and evicted from it.
#include "kv4.cuh"
#include "ptx.cuh"

namespace l2pd {

namespace {

// ---- store -------------------------------------------------------------------------------------------------------------
// A thread holds 32 values, in four pieces.  The codes are those of the exact quotient (x - m) / s, half to even; quotients of
// bf16 numbers lie on a border once in a hundred values, so borders are no rare case.  1 / s is taken a little too small, by 2^-21: the
// fp32 quotient is below the exact one, by less than 1e-5, and its rounding c too small by one where the rest e = (x - m) - c s says so:
// e > s / 2, or e = s / 2 and c odd.  e is exact if x - m is, which holds where the row's exponents lie within 15 of each other; in other
// rows (WIDE) what x - m lost decides at a border.  Steps s so small that they lack bits: in 64 bits.
// Many rows: bound by the instructions a value takes, then by memory.  Two values an instruction for the least and the largest, the
// rounding by an addition of 1.5 2^23, whose sum ends in the code's bits; 32 values a thread, so that what a row takes counts little
// (8 x 2048 rows of 32 heads: 8 a thread 34 instructions a value and 183 us, 32 a thread 97; floor 52).
template <bool WIDE>
__device__ __forceinline__ uint32_t kv4_codes(const uint32_t *raw, float m, float s, float inv) {
  constexpr float MAGIC = 12582912.f;
  const float half = 0.5f * s;
  const uint32_t up = __float_as_uint(half) + 1u;           // the next number, for even codes
  uint32_t w = 0;
  const ptx::F2 less = ptx::f2(-m, -m), inv2 = ptx::f2(inv, inv), magic = ptx::f2(MAGIC, MAGIC), back = ptx::f2(-MAGIC, -MAGIC), step = ptx::f2(-s, -s);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const ptx::F2 x2 = ptx::f2(__uint_as_float(raw[i] << 16), __uint_as_float(raw[i] & 0xffff0000u));
    const ptx::F2 d2 = ptx::add2(x2, less), c2 = ptx::fma2(d2, inv2, magic), e2 = ptx::fma2(step, ptx::add2(c2, back), d2);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      float c = j ? ptx::f2_hi(c2) : ptx::f2_lo(c2);
      const float e = j ? ptx::f2_hi(e2) : ptx::f2_lo(e2);
      bool fix = e >= __uint_as_float(up - (__float_as_uint(c) & 1u));
      if (WIDE) {
        const float x = j ? ptx::f2_hi(x2) : ptx::f2_lo(x2), d = j ? ptx::f2_hi(d2) : ptx::f2_lo(d2);
        const float t = d - x, lost = (x - (d - t)) + (-m - t);
        if (e == half && lost != 0.f) fix = lost > 0.f;
      }
      if (fix) c += 1.f;
      w += __float_as_uint(c) << (4 * (2 * i + j));
    }
  }
  return w - 0x4b400000u * 0x11111111u;                     // the sums' upper bits, shifted and added
}
__device__ __noinline__ uint32_t kv4_codes_64(uint4 raw4, float m, float s) {
  const uint32_t raw[4] = {raw4.x, raw4.y, raw4.z, raw4.w};
  uint32_t w = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const double x = __uint_as_float(i & 1 ? raw[i >> 1] & 0xffff0000u : raw[i >> 1] << 16);
    const double c = rint((x - (double)m) / (double)s);
    w |= (uint32_t)(c < 15.0 ? c : 15.0) << (4 * i);
  }
  return w;
}
// Larger of two signed 16-bit numbers, twice
__device__ __forceinline__ uint32_t max_s2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("max.s16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
// x / 15, correctly rounded: the reciprocal's product and one correction by the rest (P. W. Markstein, IBM J. Res. Dev. 34, 1990; the tests go
// through every mantissa); for tiny x, whose rest would lose bits, a division.
__device__ __forceinline__ float fifteenth(float x) {
  constexpr float R = 1.f / 15.f;
  const float q = x * R;
  return x > 1e-30f ? fmaf(fmaf(-15.f, q, x), R, q) : __fdiv_rn(x, 15.f);
}
// Least and largest of two bf16 at a time; NaN wins.
__device__ __forceinline__ uint32_t min2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("min.NaN.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
__device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}

template <int DH>
__global__ void __launch_bounds__(256, 5) kv4_store_kernel(const Kv4View c, const bf16 *k, const bf16 *v, const Kv4Batch b, int64_t k_stride,
                                                        int64_t v_stride) {
  constexpr int G = DH / 32, ROWS = 256 / G;           // threads of a row, rows of a block
  grid_dep_launch();
  grid_dep_wait();
  const int seq = blockIdx.y, h = blockIdx.x % c.heads, first = blockIdx.x / c.heads * ROWS, r = first + threadIdx.x / G;
  const int n = b.n_rows(seq), slot = b.slot(seq, c.slots);
  if (slot < 0 || first >= n) return;
  const bool is_v = blockIdx.z;
  const int64_t stride = is_v ? v_stride : k_stride;
  const int part = threadIdx.x % G, start = b.keys ? b.keys[seq] : 0;
  const bf16 *src = (is_v ? v : k) + (b.row0(seq) + (int64_t)min(r, n - 1)) * stride + (int64_t)h * DH + 32 * part;
  uint4 raw[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) raw[i] = reinterpret_cast<const uint4 *>(src)[i];
  const uint32_t *wv = &raw[0].x;
  // the least magnitude that is not 0, as 0x8000 minus its bits: a 0 becomes the smallest signed number
  uint32_t lo = wv[0], hi = wv[0], near = 0x80008000u;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    lo = min2(lo, wv[i]); hi = max2(hi, wv[i]);
    near = max_s2(near, 0x80008000u - (wv[i] & 0x7fff7fffu));
  }
#pragma unroll
  for (int o = G / 2; o; o >>= 1) {
    lo = min2(lo, __shfl_xor_sync(0xffffffffu, lo, o));
    hi = max2(hi, __shfl_xor_sync(0xffffffffu, hi, o));
    near = max_s2(near, __shfl_xor_sync(0xffffffffu, near, o));
  }
  lo = min2(lo, lo >> 16); hi = max2(hi, hi >> 16); near = max_s2(near, near >> 16);   // the lower halves
  const int least = (int)((0x8000u - (near & 0xffffu)) & 0x7fffu) >> 7, most = (int)max(lo & 0x7fffu, hi & 0x7fffu) >> 7;   // exponents
  const float mn = __uint_as_float(lo << 16), range = __uint_as_float(hi << 16) - mn;
  const bool fine = range < INFINITY;                  // no infinity, no NaN, no range beyond fp32
  const float s = fine ? __bfloat162float(__float2bfloat16_rn(fifteenth(range))) : __uint_as_float(0x7fc00000u);
  uint4 codes = make_uint4(0u, 0u, 0u, 0u);
  if (fine && s > 1e-36f) {
    float inv;
    asm("rcp.approx.f32 %0, %1;" : "=f"(inv) : "f"(s));
    inv = fmaf(inv, -4.76837158203125e-7f, inv);
    // a subnormal has the exponent field 0, as no value at all has: `near` tells them apart
    if ((near & 0xffffu) != 0x8000u && most - least > 15)
      codes = make_uint4(kv4_codes<true>(wv, mn, s, inv), kv4_codes<true>(wv + 4, mn, s, inv), kv4_codes<true>(wv + 8, mn, s, inv), kv4_codes<true>(wv + 12, mn, s, inv));
    else
      codes = make_uint4(kv4_codes<false>(wv, mn, s, inv), kv4_codes<false>(wv + 4, mn, s, inv), kv4_codes<false>(wv + 8, mn, s, inv), kv4_codes<false>(wv + 12, mn, s, inv));
  } else if (fine && s > 0.f) {
    codes = make_uint4(kv4_codes_64(raw[0], mn, s), kv4_codes_64(raw[1], mn, s), kv4_codes_64(raw[2], mn, s), kv4_codes_64(raw[3], mn, s));
  }
  const int64_t key = (int64_t)start + r;
  if (r >= n || key < 0 || key >= c.cap) return;
  uint8_t *t = c.tile(slot, h, (int)(key / KV4_TILE));
  const int kr = (int)(key % KV4_TILE);
  const int off = is_v ? kv4_off_v(DH) + kr * (DH / 2) + ((16 * part) ^ kv4_v_swizzle(kr, DH)) : kr * (DH / 2) + 16 * part;
  *reinterpret_cast<uint4 *>(t + off) = codes;
  if (part == 0) {
    const uint32_t meta = (__float_as_uint(s) >> 16) | (fine ? __float_as_uint(mn) & 0xffff0000u : 0x7fc00000u);
    *reinterpret_cast<uint32_t *>(t + (is_v ? kv4_off_vmeta(DH) : kv4_off_kmeta(DH)) + 4 * kr) = meta;
  }
}

// ---- load --------------------------------------------------------------------------------------------------------------
// As store, backwards, with dh / 8 threads a row: a warp then writes whole lines.  Rows whose key or slot does not exist read as 0.
// A block takes rows of one head; a thread has four of them in flight.
template <int DH> constexpr int LOAD_ROWS = 4 * 256 / (DH / 8);

template <int DH, typename T>
__global__ void __launch_bounds__(256) kv4_load_kernel(const Kv4View c, T *k, T *v, const Kv4Batch b, int64_t k_stride, int64_t v_stride) {
  constexpr int G = DH / 8, STEP = 256 / G;
  grid_dep_launch();
  grid_dep_wait();
  const int seq = blockIdx.y, h = blockIdx.x % c.heads, r0 = blockIdx.x / c.heads * LOAD_ROWS<DH> + threadIdx.x / G;
  const int n = b.n_rows(seq), slot = b.slot(seq, c.slots);
  if (r0 >= n) return;
  const bool is_v = blockIdx.z;
  const int64_t stride = is_v ? v_stride : k_stride;
  const int li = threadIdx.x % G, start = b.keys ? b.keys[seq] : 0;
  T *dst = (is_v ? v : k) + b.row0(seq) * stride + (int64_t)h * DH + 8 * li;
  uint32_t codes[4], meta[4];
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const int64_t key = (int64_t)start + r0 + u * STEP;
    codes[u] = meta[u] = 0;
    if (slot >= 0 && r0 + u * STEP < n && key >= 0 && key < c.cap) {
      const uint8_t *t = c.tile(slot, h, (int)(key / KV4_TILE));
      const int kr = (int)(key % KV4_TILE);
      const int off = is_v ? kv4_off_v(DH) + kr * (DH / 2) + ((4 * li) ^ kv4_v_swizzle(kr, DH)) : kr * (DH / 2) + 4 * li;
      codes[u] = *reinterpret_cast<const uint32_t *>(t + off);
      meta[u] = *reinterpret_cast<const uint32_t *>(t + (is_v ? kv4_off_vmeta(DH) : kv4_off_kmeta(DH)) + 4 * kr);
    }
  }
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    if (r0 + u * STEP >= n) break;
    const float s = kv4_scale(meta[u]), m = kv4_min(meta[u]);
    Vec8<T> y;
#pragma unroll
    for (int i = 0; i < 8; ++i) y.set(i, fmaf((float)((codes[u] >> (4 * i)) & 15u), s, m));   // c s is exact
    y.store(dst + (r0 + u * STEP) * stride);
  }
}

// ---- eviction ----------------------------------------------------------------------------------------------------------
// Rank of a weight as an unsigned number: the order of the floats, both zeros alike, NaN below all, protected keys above all.
__device__ __forceinline__ uint32_t weight_rank(float w, bool is_protected) {
  if (is_protected) return 0xffffffffu;
  if (!(w == w)) return 0u;
  const uint32_t u = w == 0.f ? 0u : __float_as_uint(w);
  return u >> 31 ? ~u : u | 0x80000000u;
}

constexpr int SELECT_THREADS = 512;
constexpr int SELECT_CACHE = 32768;   // ranks of a CTA's slice that fit its shared memory

// Exclusive sum over the block of one value a thread; *total receives the sum.
__device__ __forceinline__ int block_scan(int x, int *warp_sums, int *total) {
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  int s = x;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, s, o);
    if (lane >= o) s += y;
  }
  __syncthreads();
  if (lane == 31) warp_sums[w] = s;
  __syncthreads();
  if (w == 0) {
    int y = lane < (int)(blockDim.x >> 5) ? warp_sums[lane] : 0;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int z = __shfl_up_sync(0xffffffffu, y, o);
      if (lane >= o) y += z;
    }
    warp_sums[lane] = y;
  }
  __syncthreads();
  *total = warp_sums[(blockDim.x >> 5) - 1];
  return s - x + (w ? warp_sums[w - 1] : 0);
}

// One cluster of CTAs per (head, sequence), each with a slice of the keys.  The rank of the last kept key is found digit by digit (four
// histograms of 256, added over the cluster); a bitmap of the kept keys with the running count before each word then answers both "how many
// free places before j" and "which is the i-th kept key", in the slice of any CTA, so that no list is built.
// Bound by the latency of its steps.  8 heads x 4 sequences of 65000 keys down to 8000: one CTA each 141 us, eight that deal the
// places out 34, all of a slice's weights in flight and four words of the search a step 29 (the records' move behind it 19).
__device__ __forceinline__ uint32_t ld_cluster(const void *p, uint32_t rank) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(ptx::mapa(ptx::smem_u32(p), rank)));
  return v;
}

__global__ void __launch_bounds__(SELECT_THREADS) kv4_select_kernel(const Kv4EvictArgs a, int cluster, int slice) {
  extern __shared__ uint32_t sm[];
  __shared__ int hist[4][256], sums[256], warp_sums[32], pick[2];
  __shared__ int counts[3];                       // of the slice: ties, kept keys, kept keys below the new length
  grid_dep_launch();
  grid_dep_wait();
  const int me = blockIdx.x % cluster, h = blockIdx.x / cluster, seq = blockIdx.y, H = a.src.heads, tid = threadIdx.x;
  const int slot = a.b.slot(seq, min(a.src.slots, a.dst.slots));
  const int n = slot < 0 ? 0 : max(0, min(min(a.b.keys[seq], a.max_len), a.src.cap)), m = min(n, a.keep);
  int32_t *kept = a.kept + ((int64_t)seq * H + h) * a.keep;
  if (blockIdx.x == 0 && tid == 0) a.lens_out[seq] = m;
  for (uint32_t j = m + me * SELECT_THREADS + tid; j < (uint32_t)a.keep; j += cluster * SELECT_THREADS) kept[j] = -1;   // keep may end at 2^31 - 1
  if (n <= a.keep) {                              // the whole cluster
    for (int j = me * SELECT_THREADS + tid; j < n; j += cluster * SELECT_THREADS) kept[j] = j;
    return;
  }
  const int lo = min(me * slice, n), count = min(slice, n - lo), words = (count + 31) >> 5;   // slice: a multiple of 32
  uint32_t *bits = sm;
  int *before = reinterpret_cast<int *>(sm) + slice / 32;
  uint32_t *cache = sm + slice / 16;
  const bool cached = slice <= SELECT_CACHE;
  const int64_t base = ((int64_t)slot * H + h) * a.src.cap + lo;
  const int from = a.protect_from ? a.protect_from[seq] : 0x7fffffff;
  auto rank_of = [&](int j) {
    const int pos = a.positions ? a.positions[base + j] : lo + j;
    return weight_rank(a.weights[base + j], pos < a.first || pos >= from);
  };
  auto rank = [&](int j) { return cached ? cache[j] : rank_of(j); };
  for (int i = tid; i < 1024; i += SELECT_THREADS) hist[i >> 8][i & 255] = 0;
  if (tid < 3) counts[tid] = 0;
  if (cached) {
    // sixteen keys a thread at once: a slice of 8192 is one round of loads
    for (int j0 = tid; j0 < count; j0 += 16 * SELECT_THREADS) {
      float w[16];
      int pos[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int j = min(j0 + i * SELECT_THREADS, count - 1);
        w[i] = a.weights[base + j];
        pos[i] = a.positions ? a.positions[base + j] : lo + j;
      }
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (j0 + i * SELECT_THREADS < count) cache[j0 + i * SELECT_THREADS] = weight_rank(w[i], pos[i] < a.first || pos[i] >= from);
    }
  }
  __syncthreads();
  uint32_t prefix = 0, mask = 0;
  int need = m;                                   // of the keys whose leading digits equal the prefix, this many are kept
  for (int pass = 0; pass < 4; ++pass) {
    const int shift = 24 - 8 * pass;
#pragma unroll 8
    for (int j = tid; j < count; j += SELECT_THREADS) {
      const uint32_t r = rank(j);
      if ((r & mask) == prefix) atomicAdd(&hist[pass][(r >> shift) & 255u], 1);
    }
    if (cluster == 1) __syncthreads();
    else {
      ptx::cluster_sync();
      if (tid < 256) {
        int x[8], y = 0;
#pragma unroll
        for (int c = 0; c < 8; ++c) x[c] = c < cluster ? (int)ld_cluster(&hist[pass][tid], c) : 0;
#pragma unroll
        for (int c = 0; c < 8; ++c) y += x[c];
        sums[tid] = y;
      }
      __syncthreads();
    }
    if (tid < 32) {                               // keys in higher digits, counted from the top: lane l has the digits 255 - 8 l and below
      const int *of = (cluster == 1 ? hist[pass] : sums) + 248 - 8 * tid;
      int x[8], own = 0, digit = -1;
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = of[i];
#pragma unroll
      for (int i = 0; i < 8; ++i) own += x[i];
      int above = own;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, above, o);
        if (tid >= o) above += y;
      }
      above -= own;
#pragma unroll
      for (int i = 7; i >= 0; --i) {              // the digit that the need-th key falls into
        if (above < need && above + x[i] >= need) { digit = 248 - 8 * tid + i; own = above; }
        above += x[i];
      }
      if (digit >= 0) { pick[0] = digit; pick[1] = own; }
    }
    __syncthreads();
    prefix |= (uint32_t)pick[0] << shift;
    mask |= 255u << shift;
    need -= pick[1];
    __syncthreads();
  }
  // bitmap: all above the last kept rank, and of the equal ones the first `need`
  const int lane = tid & 31;
  int eqs = 0;
  for (int w = tid >> 5; w < words; w += SELECT_THREADS / 32) {
    const int j = w * 32 + lane;
    const uint32_t r = j < count ? rank(j) : 0u;
    const uint32_t up = __ballot_sync(0xffffffffu, j < count && r > prefix), eq = __ballot_sync(0xffffffffu, j < count && r == prefix);
    if (lane == 0) { bits[w] = up; before[w] = (int)eq; eqs += __popc(eq); }
  }
  if (lane == 0 && eqs) atomicAdd(&counts[0], eqs);
  ptx::cluster_sync();
  int ties = 0;                                   // in the slices before this one
  for (int c = 0; c < me; ++c) ties += (int)ld_cluster(&counts[0], c);
  int sum = 0, low = 0;
  for (int w0 = 0; w0 < words; w0 += SELECT_THREADS) {
    const int w = w0 + tid;
    uint32_t eq = w < words ? (uint32_t)before[w] : 0u;
    uint32_t up = w < words ? bits[w] : 0u;
    int total;
    int room = need - ties - block_scan(__popc(eq), warp_sums, &total);
    ties += total;
    for (; eq && room > 0; --room) { up |= eq & (0u - eq); eq &= eq - 1; }
    const int e = block_scan(__popc(up), warp_sums, &total);
    if (w < words) {
      bits[w] = up;
      before[w] = sum + e;
      const int k = m - lo - w * 32;              // keys of this word below the new length
      low += k >= 32 ? __popc(up) : k > 0 ? __popc(up & ((1u << k) - 1u)) : 0;
    }
    sum += total;
  }
  if (low) atomicAdd(&counts[2], low);
  if (tid == 0) counts[1] = sum;
  ptx::cluster_sync();
  int held[8], front = 0;                         // kept keys of each slice; kept keys that stay where they are
#pragma unroll
  for (int c = 0; c < 8; ++c) {
    held[c] = c < cluster ? (int)ld_cluster(&counts[1], c) : 0;
    if (c < cluster) front += (int)ld_cluster(&counts[2], c);
  }
  auto peek = [&](const void *p, int c) { return cluster == 1 ? *reinterpret_cast<const uint32_t *>(p) : ld_cluster(p, c); };
  // the places, dealt out to all threads of the cluster
  for (int j = me * SELECT_THREADS + tid; j < m; j += cluster * SELECT_THREADS) {
    const int owner = j / slice, at = (j - owner * slice) >> 5;
    const uint32_t word = peek(&bits[at], owner), bit = 1u << (j & 31);
    int src = j;
    if (!(word & bit)) {
      // the kept key with `want` of them before it: as many as there are free places before this one, behind the front
      int want = front + j - (int)peek(&before[at], owner) - __popc(word & (bit - 1u)), c = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) if (i < owner) want -= held[i];
#pragma unroll
      for (int i = 0; i < 7; ++i)
        if (c == i && i < cluster - 1 && want >= held[i]) { want -= held[i]; ++c; }
      int x = 0, y = (min(slice, n - c * slice) + 31) / 32 - 1;   // its word: the last whose count does not pass `want`
      while (x < y) {                               // a quarter of the words a step
        const int step = (y - x + 4) >> 2, p1 = min(x + step, y), p2 = min(x + 2 * step, y), p3 = min(x + 3 * step, y);
        const int b1 = (int)peek(&before[p1], c), b2 = (int)peek(&before[p2], c), b3 = (int)peek(&before[p3], c);
        if (b3 <= want) x = p3;
        else if (b2 <= want) { x = p2; y = p3 - 1; }
        else if (b1 <= want) { x = p1; y = p2 - 1; }
        else y = p1 - 1;
      }
      uint32_t u = peek(&bits[x], c);
      want -= (int)peek(&before[x], c);             // the bit with `want` set ones below it, halving
      int bit_at = 0;
#pragma unroll
      for (int half = 16; half; half >>= 1) {
        const int below = __popc(u & ((1u << half) - 1u));
        if (want >= below) { want -= below; bit_at += half; u >>= half; }
      }
      src = c * slice + x * 32 + bit_at;
    }
    kept[j] = src;
  }
  ptx::cluster_sync();                            // others may still read this CTA's bitmap
}

// Moves the records: a block takes 128 places, four threads a place, two places a thread at once.  In place only the filled holes move;
// their sources lie at or behind the new end, all destinations before it.
constexpr int MOVE_PLACES = 128;

__global__ void __launch_bounds__(256) kv4_move_kernel(const Kv4EvictArgs a) {
  grid_dep_launch();
  grid_dep_wait();
  const int seq = blockIdx.y, H = a.src.heads, h = blockIdx.x % H, part = threadIdx.x & 3;
  const int slot = a.b.slot(seq, min(a.src.slots, a.dst.slots));
  if (slot < 0) return;
  const int dh = a.src.dh, row = dh / 2, meta = part ? kv4_off_vmeta(dh) : kv4_off_kmeta(dh);
  const int64_t head = (int64_t)slot * H + h;
  int j[2], s[2];
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    j[u] = blockIdx.x / H * MOVE_PLACES + 64 * u + (threadIdx.x >> 2);
    s[u] = j[u] < a.keep ? a.kept[((int64_t)seq * H + h) * a.keep + j[u]] : -1;
  }
  uint4 k[2], v[2];
  uint32_t m[2], x[2];
  bool rec[2], val[2];                             // the record moves; the weight or position does
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    rec[u] = s[u] >= 0 && !(a.src.data == a.dst.data && s[u] == j[u]);
    const int64_t from = head * a.src.cap + s[u], to = head * a.dst.cap + j[u];
    val[u] = s[u] >= 0 && (part == 2 ? a.weights_dst && a.weights + from != a.weights_dst + to
                           : part == 3 && a.positions_dst && !(a.positions && a.positions + from == a.positions_dst + to));
    if (val[u]) x[u] = part == 2 ? __float_as_uint(a.weights[from]) : a.positions ? (uint32_t)a.positions[from] : (uint32_t)s[u];
    if (rec[u]) {
      const uint8_t *t = a.src.tile(slot, h, s[u] / KV4_TILE);
      const int r = s[u] % KV4_TILE;
      if (part * 16 < row) {
        k[u] = *reinterpret_cast<const uint4 *>(t + r * row + part * 16);
        v[u] = *reinterpret_cast<const uint4 *>(t + kv4_off_v(dh) + r * row + ((part * 16) ^ kv4_v_swizzle(r, dh)));
      }
      if (part < 2) m[u] = *reinterpret_cast<const uint32_t *>(t + meta + 4 * r);
    }
  }
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int64_t to = head * a.dst.cap + j[u];
    if (val[u]) { if (part == 2) a.weights_dst[to] = __uint_as_float(x[u]); else a.positions_dst[to] = (int32_t)x[u]; }
    if (rec[u]) {
      uint8_t *t = a.dst.tile(slot, h, j[u] / KV4_TILE);
      const int r = j[u] % KV4_TILE;
      if (part * 16 < row) {
        *reinterpret_cast<uint4 *>(t + r * row + part * 16) = k[u];
        *reinterpret_cast<uint4 *>(t + kv4_off_v(dh) + r * row + ((part * 16) ^ kv4_v_swizzle(r, dh))) = v[u];
      }
      if (part < 2) *reinterpret_cast<uint32_t *>(t + meta + 4 * r) = m[u];
    }
  }
}

}  // namespace

cudaError_t launch_kv4_store(cudaStream_t st, const Kv4View &c, const bf16 *k, const bf16 *v, const Kv4Batch &b, int64_t k_stride,
                             int64_t v_stride) {
  const dim3 grid((unsigned)(ceil_div(b.rows, 256 / (c.dh / 32)) * c.heads), b.B, 2);
  if (c.dh == 128) return launch_kernel(kv4_store_kernel<128>, grid, dim3(256), 0, st, c, k, v, b, k_stride, v_stride);
  return launch_kernel(kv4_store_kernel<64>, grid, dim3(256), 0, st, c, k, v, b, k_stride, v_stride);
}

cudaError_t launch_kv4_load(cudaStream_t st, const Kv4View &c, int dtype, void *k, void *v, const Kv4Batch &b, int64_t k_stride,
                            int64_t v_stride) {
  const dim3 grid((unsigned)(ceil_div(b.rows, c.dh == 128 ? LOAD_ROWS<128> : LOAD_ROWS<64>) * c.heads), b.B, 2);
  if (dtype == L2PD_BF16) {
    auto fn = c.dh == 128 ? kv4_load_kernel<128, bf16> : kv4_load_kernel<64, bf16>;
    return launch_kernel(fn, grid, dim3(256), 0, st, c, (bf16 *)k, (bf16 *)v, b, k_stride, v_stride);
  }
  auto fn = c.dh == 128 ? kv4_load_kernel<128, float> : kv4_load_kernel<64, float>;
  return launch_kernel(fn, grid, dim3(256), 0, st, c, (float *)k, (float *)v, b, k_stride, v_stride);
}

cudaError_t launch_kv4_evict(cudaStream_t st, const Kv4EvictArgs &a) {
  // CTAs of a cluster: a slice of 4096 keys each, eight at most (1 x 8 heads on 4000 keys in four: 14.1 us instead of 15.8, on 1500 in
  // two: 12.7 instead of 11.7)
  int cluster = 1;
  while (cluster < 8 && a.max_len > 4096 * cluster) cluster *= 2;
  const int slice = ceil_div(ceil_div(a.max_len > 1 ? a.max_len : 1, cluster), 32) * 32;
  const size_t smem = (size_t)slice / 32 * 8 + (slice <= SELECT_CACHE ? (size_t)slice * 4 : 0);
  cudaError_t e = cudaSuccess;
  static std::atomic<uint64_t> done{0};
  if (smem > 32 * 1024) e = allow_shared((const void *)kv4_select_kernel, SELECT_CACHE * 4 + KV4_MAX_EVICT / 8 / 4, done);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(a.src.heads * cluster, a.b.B); cfg.blockDim = dim3(SELECT_THREADS); cfg.dynamicSmemBytes = smem; cfg.stream = st;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = cluster; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
  at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at; cfg.numAttrs = pdl_enabled() ? 2 : 1;
  e = cudaLaunchKernelEx(&cfg, kv4_select_kernel, a, cluster, slice);
  if (e != cudaSuccess) return e;
  const int places = a.keep < a.max_len ? a.keep : a.max_len;   // no place behind them is filled, whatever `keep` allows
  if (places == 0) return cudaSuccess;
  return launch_kernel(kv4_move_kernel, dim3((unsigned)(ceil_div(places, MOVE_PLACES) * a.src.heads), a.b.B), dim3(256), 0, st, a);
}

}  // namespace l2pd
