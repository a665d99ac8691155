// Attention over a key/value cache in 4 bits on the 5th-generation tensor cores, for 9 to 128 columns (query rows times query heads
// that share a key head) of a sequence and key head at once.
//
// S = Q K^T and O += P V, the columns on the M side (128 lanes of tensor memory), tiles of 64 keys.  Eight warps turn codes into
// fp16 operands in shared memory, in the 128-byte swizzle:
//     K: (c - 8) s 2^-E    exact: c - 8 has three significant bits (or is 8), s has eight.  The rest of the value, a = m + 8 s, reaches the scores
//        through sixteen further products of depth: (a_hi, a_hi, a_lo) against (sum q_hi, sum q_lo, sum q_hi): no number of a key's
//        own is left for the softmax
//     V: c s 2^-E + m 2^-E in one fused operation, rounded once (2^-11 relative)
// E belongs to 32 keys (a warp).  A code reaches fp16 as it lies, as the subnormal c 2^-24 (or 16 c 2^-24 from bits 4..7), and the
// multiplication by s 2^24 (2^20) lifts it.  Eight codes of a word come out in the order 0 4 1 5 2 6 3 7: queries are written in that order, and
// outputs read in it.
// Two groups of four softmax warps take the tiles alternately, each with sums, reference and O of its own, so that one is at its
// exponentials while the other waits for the tensor pipe; they are added at the end of an item.  A thread owns a lane:
// t = cf 2^E acc + (E_V - E0) - M, P = 2^t as fp16 over the scores, as the A operand of the second product.  M is a reference that follows
// the running maximum lazily, E0 the largest E_V so far; O is rescaled when one moves.
//
// Fewer columns than lanes: chunks of 32 (64) columns stand four times (twice) in the lanes, and each copy takes its quarter (half) of a
// tile's keys, its probabilities of the others being 0.  The tensor pipe and shared memory do the same work as for 128 columns, but the
// exponentials are spread over all warps; the copies are added at the end.
//
// What bounds it: shared memory.  128 keys of 128: 17 KB of codes in and out, 64 KB of operands out and in: 1300 cycles at 128 bytes; the
// products 1090, the exponentials (128 columns) 1024.
//
// Warp roles (576 threads): 0-3 and 4-7 softmax and output, 8-11 and 12-15 operands (two warps K, two V), 16 copies of codes, 17 MMA
// issuer (owns tensor memory).  Tensor memory: S at 0 and 64, O at 128 and 256, Q at 384.
#include <cuda_fp16.h>
#include <math.h>

#include "attention_kv4.cuh"

namespace l2pd {
namespace kv4 {

namespace {

constexpr int RING = 5, NB = 4;                    // tiles of codes on their way; operand buffers
constexpr uint32_t ATOM = TC_TILE * 128;           // 64 rows x 64 fp16
constexpr int NONE = -1000;                        // no exponent
constexpr int LDS_O = 20;                          // floats of a staged row of 16
constexpr int SOFTMAX = 256, THREADS = 576;

template <int DH> struct Tc {
  static constexpr int ATOMS = DH / 64, TILE32 = KV4_TILE * (DH + 8), STAGE = 2 * TILE32;
  static constexpr uint32_t K = 0, AUG = NB * ATOMS * ATOM, V = AUG + ATOM, CODES = V + NB * ATOMS * ATOM,
                            STAGING = CODES + RING * STAGE, BYTES = STAGING + 2 * 128 * LDS_O * 4;
};

enum { B_FULL = 0, B_EMPTY = B_FULL + RING, B_KRDY = B_EMPTY + RING, B_KFREE = B_KRDY + NB, B_VRDY = B_KFREE + NB, B_VFREE = B_VRDY + NB,
       B_SFULL = B_VFREE + NB, B_PRDY = B_SFULL + 2, B_QRDY = B_PRDY + 2, B_OFREE = B_QRDY + 1, B_COUNT = B_OFREE + 1 };

__device__ __forceinline__ float pow2(int n) { return __uint_as_float((uint32_t)(127 + n) << 23); }   // -126 <= n <= 127
// x 2^n for n beyond one exponent's range
__device__ __forceinline__ float scaled(float x, int n) { const int h = n >> 1; return x * pow2(h) * pow2(n - h); }
__device__ __forceinline__ uint32_t dup(float x) { __half2 h = __float2half2_rn(x); return *reinterpret_cast<uint32_t *>(&h); }
__device__ __forceinline__ uint32_t pair(float a, float b) { __half2 h = __floats2half2_rn(a, b); return *reinterpret_cast<uint32_t *>(&h); }
__device__ __forceinline__ uint32_t hfma2(uint32_t a, uint32_t b, uint32_t c) {
  uint32_t d;
  asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
  return d;
}
__device__ __forceinline__ void softmax_sync() { asm volatile("bar.sync 1, 256;" ::: "memory"); }

// One row of codes to its fp16 row: value = c s + o, s and o given times the powers of two above.  `row` and `out`: shared
// addresses of the codes and of the row in its first atom, r: the tile row.  The quarters of a row are read in an order that
// differs from row to row, so that eight lanes touch all banks, reading and writing.
template <int DH>
__device__ __forceinline__ void unpack_row(uint32_t row, uint32_t out, int r, uint32_t s, uint32_t s16, uint32_t o, uint32_t swz) {
  constexpr int PARTS = DH / 32;
#pragma unroll
  for (int i = 0; i < PARTS; ++i) {
    const int c = (i + (r >> 1)) & (PARTS - 1);
    const uint4 w4 = ptx::ld_shared_v4(row + ((16 * c) ^ swz));
    const uint32_t w[4] = {w4.x, w4.y, w4.z, w4.w};
    const uint32_t at = out + (c >> 1) * ATOM + (((4 * (c & 1)) ^ (r & 7)) << 4);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t hi = w[j] >> 8;
      ptx::st_shared_v4(at ^ (j << 4), make_uint4(hfma2(w[j] & 0x000f000fu, s, o), hfma2(w[j] & 0x00f000f0u, s16, o),
                                                  hfma2(hi & 0x000f000fu, s, o), hfma2(hi & 0x00f000f0u, s16, o)));
    }
  }
}

template <int DH, int COPIES>
__global__ void __launch_bounds__(THREADS, 1) attention_kv4_tc_kernel(const AttnParams p) {
  using T = Tc<DH>;
  constexpr int CHUNK = 128 / COPIES, NK = TC_TILE / COPIES;   // columns; keys of a tile that a copy takes
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t bars[B_COUNT];
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_flag;
  // exponents of a tile's two groups of 32 keys.  K runs ahead of the softmax: its buffer is free once the scores are there
  __shared__ int expo_k[2 * NB][2], expo_v[NB][2];
  __shared__ int lost;                             // a softmax warp's wait ran out
  __shared__ float2 ml[2][128];                    // a lane's reference and sum
  __shared__ float q_factor[128];
  const int warp = ptx::warp_index(), lane = threadIdx.x & 31;
  const uint32_t base = (ptx::smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t bar0 = ptx::smem_u32(bars);
  auto bar = [&](int i) { return bar0 + 8u * i; };
  if (threadIdx.x == 0) {
    for (int i = 0; i < RING; ++i) { ptx::mbar_init(bar(B_FULL + i), 1); ptx::mbar_init(bar(B_EMPTY + i), 4); }
    for (int i = 0; i < NB; ++i) {
      ptx::mbar_init(bar(B_KRDY + i), 2); ptx::mbar_init(bar(B_KFREE + i), 1);
      ptx::mbar_init(bar(B_VRDY + i), 2); ptx::mbar_init(bar(B_VFREE + i), 1);
    }
    for (int i = 0; i < 2; ++i) { ptx::mbar_init(bar(B_SFULL + i), 2); ptx::mbar_init(bar(B_PRDY + i), 4); }
    ptx::mbar_init(bar(B_QRDY), 4); ptx::mbar_init(bar(B_OFREE), 8);
    abort_flag = 0; lost = 0;
    ptx::fence_barrier_init();
    ptx::fence_proxy_async();
  }
  if (warp == 17) { ptx::tmem_alloc(ptx::smem_u32(&tmem_slot), 512); ptx::tmem_relinquish(); }
  ptx::tc_fence_before_sync();
  __syncthreads();
  ptx::tc_fence_after_sync();
  const uint32_t tS = tmem_slot, tO = tS + 128, tQ = tS + 384;
  int32_t *const status = p.status;
  grid_dep_launch();
  grid_dep_wait();

  // the run of tiles, the same in every warp
  const Line &ln = p.line;
  const Seq own = ln.seq(lane);
  uint32_t share;
  const uint32_t total = ln.survey(own, gridDim.x, 0, &share, nullptr);
  const uint32_t begin = (uint32_t)min((uint64_t)share * blockIdx.x, (uint64_t)total), end = min(total, begin + share);
  struct Piece { int t0, t1, nt, h, c0, cols, keys, row0, slot; };
  auto piece_at = [&](uint32_t pos) {
    uint32_t before;
    const Seq sq = ln.find(own, pos, &before);
    Piece w;
    const int item = (int)((pos - before) / sq.tiles);
    w.nt = sq.tiles; w.t0 = (int)(pos - before) - item * sq.tiles;
    w.t1 = (int)min((uint32_t)sq.tiles, w.t0 + (end - pos));
    w.h = item / sq.chunks; w.c0 = (item - w.h * sq.chunks) * CHUNK; w.cols = min(CHUNK, sq.rows * ln.group - w.c0);
    w.keys = sq.keys; w.row0 = sq.row0; w.slot = sq.slot;
    return w;
  };

  if (warp == 16) {
    // ------------------------------------------------------------------ codes: one or two tiles of the cache, one contiguous piece
    int slot = 0;
    uint32_t par = 1;
    for (uint32_t pos = begin; pos < end;) {
      const Piece w = piece_at(pos);
      const uint8_t *src = p.c.tile(w.slot, w.h, 0);
      for (int t = w.t0; t < w.t1; ++t) {
        const bool ok = ptx::mbar_wait_or_abort(bar(B_EMPTY + slot), par, &abort_flag, status, DEV_TIMEOUT_PRODUCER);
        const uint32_t bytes = min(2, (w.keys - t * TC_TILE + KV4_TILE - 1) / KV4_TILE) * T::TILE32;
        if (ptx::elect_one() && ok) {
          ptx::mbar_arrive_expect_tx(bar(B_FULL + slot), bytes);
          ptx::bulk_load(base + T::CODES + slot * T::STAGE, src + (int64_t)t * T::STAGE, bytes, bar(B_FULL + slot));
        }
        if (++slot == RING) { slot = 0; par ^= 1u; }
      }
      pos += w.t1 - w.t0;
    }
  } else if (warp == 17) {
    // ------------------------------------------------------------------ MMA issuer: S(0) S(1) PV(0) S(2) PV(1) S(3) ...
    constexpr uint32_t F32 = 1u << 4, M128 = (128u >> 4) << 24;
    const uint32_t idesc_s = F32 | M128 | ((TC_TILE >> 3) << 17), idesc_o = F32 | M128 | ((DH >> 3) << 17) | (1u << 16);
    uint32_t ts = 0, tp = 0, qpar = 0, opar = 1;     // tiles whose S, whose PV was issued
    auto scores = [&]() {
      const uint32_t b = ts % NB, g = ts & 1u;
      const bool ok = ptx::mbar_wait_or_abort(bar(B_KRDY + b), (ts / NB) & 1u, &abort_flag, status, DEV_TIMEOUT_MMA);
      ptx::tc_fence_after_sync();
      const uint64_t kd = ptx::smem_desc_sw128(base + T::K + b * T::ATOMS * ATOM), ad = ptx::smem_desc_sw128(base + T::AUG) + 2u * b;
      if (ptx::elect_one() && ok) {
#pragma unroll
        for (int k = 0; k < DH / 16; ++k)
          ptx::mma_bf16_ts(tS + g * TC_TILE, tQ + 8 * k, kd + (k >> 2) * (ATOM >> 4) + 2u * (k & 3), idesc_s, k ? 1u : 0u);
        ptx::mma_bf16_ts(tS + g * TC_TILE, tQ + DH / 2, ad, idesc_s, 1u);
        ptx::mma_commit(bar(B_KFREE + b));
        ptx::mma_commit(bar(B_SFULL + g));
        ptx::mbar_arrive(bar(B_SFULL + g));          // passes on what the K warps wrote besides
      }
      ++ts;
    };
    auto output = [&](bool first, bool wait_o) {
      const uint32_t b = tp % NB, g = tp & 1u;
      bool ok = ptx::mbar_wait_or_abort(bar(B_VRDY + b), (tp / NB) & 1u, &abort_flag, status, DEV_TIMEOUT_MMA);
      if (wait_o) {                                  // the piece before has been read out of O
        ok = ptx::mbar_wait_or_abort(bar(B_OFREE), opar, &abort_flag, status, DEV_TIMEOUT_MMA) && ok;
        opar ^= 1u;
      }
      ok = ptx::mbar_wait_or_abort(bar(B_PRDY + g), (tp >> 1) & 1u, &abort_flag, status, DEV_TIMEOUT_MMA) && ok;
      ptx::tc_fence_after_sync();
      const uint64_t vd = ptx::smem_desc_sw128_mn(base + T::V + b * T::ATOMS * ATOM, ATOM);
      if (ptx::elect_one() && ok) {
#pragma unroll
        for (int k = 0; k < TC_TILE / 16; ++k)
          ptx::mma_bf16_ts(tO + g * 128, tS + g * TC_TILE + 8 * k, vd + k * (2048u >> 4), idesc_o, k ? 1u : first ? 0u : 1u);
        ptx::mma_commit(bar(B_VFREE + b));
      }
      ++tp;
    };
    for (uint32_t pos = begin; pos < end;) {
      const Piece w = piece_at(pos);
      const int n = w.t1 - w.t0;
      ptx::mbar_wait_or_abort(bar(B_QRDY), qpar, &abort_flag, status, DEV_TIMEOUT_MMA);
      qpar ^= 1u;
      scores();
      if (n > 1) scores();
      for (int i = 0; i < n; ++i) {
        output(i < 2, i == 0);
        if (i + 2 < n) scores();
      }
      pos += n;
    }
  } else if (warp >= 8) {
    // ------------------------------------------------------------------ codes to operands: every other tile
    const bool is_v = warp & 2;
    const int grp = warp & 1, r = 32 * grp + lane, swz = is_v ? kv4_v_swizzle(lane, DH) : 0;
    const uint32_t out = base + (is_v ? T::V : T::K) + r * 128, aug = base + T::AUG + r * 128;
    const uint32_t row_off = grp * T::TILE32 + (is_v ? kv4_off_v(DH) : 0) + lane * (DH / 2);
    const uint32_t meta_off = grp * T::TILE32 + (is_v ? kv4_off_vmeta(DH) : kv4_off_kmeta(DH)) + 4 * lane;
    uint32_t tile = 0;
    bool ok = true;
    for (uint32_t pos = begin; pos < end && ok;) {
      const Piece w = piece_at(pos);
      for (int t = w.t0; t < w.t1 && ok; ++t, ++tile) {
        if ((tile & 1u) != (uint32_t)(warp >= 12)) continue;
        const uint32_t b = tile % NB, slot = tile % RING;
        ok = ptx::mbar_wait_warp(bar(B_FULL + slot), (tile / RING) & 1u);
        ok = ok && ptx::mbar_wait_warp(bar((is_v ? B_VFREE : B_KFREE) + b), ((tile / NB) & 1u) ^ 1u);
        if (!ok) break;
        const uint32_t stage = base + T::CODES + slot * T::STAGE;
        uint32_t meta = 0;
        if (t * TC_TILE + r < w.keys) asm volatile("ld.shared.b32 %0, [%1];" : "=r"(meta) : "r"(stage + meta_off) : "memory");
        const float s = kv4_scale(meta), m = kv4_min(meta);
        // the group's exponent; keys that are not finite stay outside it
        const int es = (int)((meta >> 7) & 255u), em = (int)((meta >> 23) & 255u);
        int e = es == 255 || em == 255 ? 0 : is_v ? max(es + 4, em) : max(es, em - 11);
        const bool none = is_v && __all_sync(0xffffffffu, (meta & 0x7fff7fffu) == 0u);   // values that are all 0 have no exponent
        e = max((int)__reduce_max_sync(0xffffffffu, (uint32_t)max(e, 0)) - 126, -100);
        if (is_v) {
          e += 1;                                    // |value| < 2^e; as fp16 times 2^-(e + 5)
          const float s1 = scaled(s, -(e + 5)), m1 = scaled(m, -(e + 5));
          unpack_row<DH>(stage + row_off, out + b * T::ATOMS * ATOM, r, dup(s1 * 16777216.f), dup(s1 * 1048576.f), dup(m1), swz);
        } else {
          const float s1 = scaled(s, -(e + 9)), a = scaled(m, -(e + 9)) + 8.f * s1;
          unpack_row<DH>(stage + row_off, out + b * T::ATOMS * ATOM, r, dup(s1 * 16777216.f), dup(s1 * 1048576.f), dup(-8.f * s1), swz);
          const float hi = __half2float(__float2half_rn(a));
          const uint32_t at = aug + (((2 * b) ^ (r & 7)) << 4);
          ptx::st_shared_v4(at, make_uint4(pair(hi, hi), pair((a - hi) * 2048.f, 0.f), 0u, 0u));
          ptx::st_shared_v4(at ^ 16u, make_uint4(0u, 0u, 0u, 0u));
        }
        if (lane == 0) {
          if (is_v) expo_v[b][grp] = none ? NONE : e; else expo_k[tile % (2 * NB)][grp] = e;
        }
        ptx::fence_proxy_async();
        __syncwarp();
        if (lane == 0) {
          ptx::mbar_arrive(bar((is_v ? B_VRDY : B_KRDY) + b));
          ptx::mbar_arrive(bar(B_EMPTY + slot));
        }
      }
      pos += w.t1 - w.t0;
    }
    if (!ok) { fail(status, DEV_TIMEOUT_PRODUCER); abort_flag = 1; }
  } else {
    // ------------------------------------------------------------------ queries, softmax, output
    const int g = warp >> 2, q = warp & 3, row = 32 * q + lane;
    const int col = row & (CHUNK - 1);               // this lane's column of the chunk
    const int k0 = q / (4 / COPIES) * NK;            // first key of a tile that it takes
    constexpr int NG = NK > 32 ? NK / 32 : 1, GK = NK / NG;   // its groups of one exponent, their keys
    const uint32_t lane_base = (uint32_t)(32 * q) << 16, tSg = tS + lane_base + g * TC_TILE, tOg = tO + lane_base + g * 128;
    uint32_t tile = 0;
    bool ok = true;
    for (uint32_t pos = begin; pos < end;) {
      const Piece w = piece_at(pos);
      if (g == 0) {
        // queries to tensor memory: the largest of a row becomes 2^7 .. 2^8
        const int c = w.c0 + col, rr = c / ln.group;
        const bool there = col < w.cols;
        const bf16 *src = p.q + (int64_t)(w.row0 + rr) * p.q_stride + (int64_t)(w.h * ln.group + c - rr * ln.group) * DH;
        uint32_t raw[DH / 2], top = 0;
#pragma unroll
        for (int j = 0; j < DH / 8; ++j) {
          const uint4 x = there ? *reinterpret_cast<const uint4 *>(src + 8 * j) : make_uint4(0, 0, 0, 0);
          raw[4 * j] = x.x; raw[4 * j + 1] = x.y; raw[4 * j + 2] = x.z; raw[4 * j + 3] = x.w;
        }
#pragma unroll
        for (int j = 0; j < DH / 2; ++j) top = max(top, max((raw[j] << 16) & 0x7fffffffu, raw[j] & 0x7fff0000u));
        const bool finite = top < 0x7f800000u;
        const int u = finite ? min(7 - ((int)(top >> 23) - 127), 126) : 0;
        const float up = pow2(u);
        q_factor[row] = p.scale_log2 * pow2(-u);
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < DH / 8; ++j) {
          float y[8];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t x = finite ? raw[4 * j + i] : 0u;
            y[2 * i] = __uint_as_float(x << 16) * up; y[2 * i + 1] = __uint_as_float(x & 0xffff0000u) * up;
            sum += y[2 * i] + y[2 * i + 1];
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) raw[4 * j + i] = pair(y[i], y[i + 4]);
        }
#pragma unroll
        for (int j = 0; j < DH / 2; j += 32) ptx::tmem_st_x32(tQ + lane_base + j, raw + j);
        const float hi = __half2float(__float2half_rn(sum));
        raw[0] = finite ? pair(hi, sum - hi) : 0x7fff7fffu;          // a NaN here makes every score of the row NaN
        raw[1] = pair(hi * (1.f / 2048.f), 0.f);
#pragma unroll
        for (int i = 2; i < 32; ++i) raw[i] = 0u;
        ptx::tmem_st_x32(tQ + lane_base + DH / 2, raw);
        ptx::tmem_st_wait();
        ptx::tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(bar(B_QRDY));
      }
      softmax_sync();
      const float cf = q_factor[row];
      float m_ref = 0.f, l = 0.f;
      int e0 = NONE;
      uint32_t last_v = 0;                           // this group's tile before, plus one
      bool first = true;
      for (int t = w.t0; t < w.t1 && ok; ++t, ++tile) {
        if ((tile & 1u) != (uint32_t)g) continue;
        // the exponents of V come with its operands
        ok = ptx::mbar_wait_warp(bar(B_VRDY + tile % NB), (tile / NB) & 1u);
        ok = ok && ptx::mbar_wait_warp(bar(B_SFULL + g), (tile >> 1) & 1u);
        if (!ok) break;
        ptx::tc_fence_after_sync();
        uint32_t s[NK];
        if (NK == 16) ptx::tmem_ld_x16(tSg + k0, s);
        else {
#pragma unroll
          for (int i = 0; i < NK; i += 32) ptx::tmem_ld_x32(tSg + k0 + i, s + i);
        }
        float k[NG], o[NG], w_of[NG], fac = 1.f;
        {
          int ek[NG], ev[NG], e_top = NONE;
#pragma unroll
          for (int i = 0; i < NG; ++i) {
            ek[i] = expo_k[tile % (2 * NB)][(k0 >> 5) + i];
            ev[i] = expo_v[tile % NB][(k0 >> 5) + i];
            e_top = max(e_top, ev[i]);
          }
          if (e_top > e0) {                          // warp-uniform
            fac = first ? 0.f : pow2(max(e0 - (e_top + 2), -126));
            e0 = e_top + 2;
          }
#pragma unroll
          for (int i = 0; i < NG; ++i) {
            const int e = ev[i] == NONE ? 0 : max(ev[i] - e0, -120);
            k[i] = scaled(cf, ek[i] + 9); o[i] = (float)e - m_ref; w_of[i] = pow2(-e);
          }
        }
        const int left = w.keys - t * TC_TILE - k0;
        ptx::tmem_ld_wait();
#pragma unroll
        for (int j = 0; j < NK; ++j) s[j] = __float_as_uint(fmaf(__uint_as_float(s[j]), k[j / GK], o[j / GK]));
        if (left < NK) {
#pragma unroll
          for (int j = 0; j < NK; ++j) if (j >= left) s[j] = 0xff800000u;
        }
        float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
        for (int j = 0; j < NK; j += 4)
#pragma unroll
          for (int e = 0; e < 4; ++e) mx[e] = fmaxf(mx[e], __uint_as_float(s[j + e]));
        const float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
        // a copy whose keys all lie behind the end keeps an open reference
        const bool grow = first ? top > -INFINITY : top > LAZY;
        if (__any_sync(0xffffffffu, grow)) {
          const float d = grow ? top : 0.f;
          m_ref += d;
          const float x = first ? 0.f : ptx::ex2(-d);
          fac *= x; l *= x;
#pragma unroll
          for (int j = 0; j < NK; ++j) s[j] = __float_as_uint(__uint_as_float(s[j]) - d);
        }
        first = first && !(top > -INFINITY);
        // probabilities
        float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < NK; j += 2) {
          const float p0 = ptx::ex2(__uint_as_float(s[j])), p1 = ptx::ex2(__uint_as_float(s[j + 1]));
          float &acc = sum[NG == 2 ? 2 * (j / GK) + ((j >> 1) & 1) : (j >> 1) & 3];
          acc += p0 + p1;
          s[j >> 1] = pair(p0, p1);
        }
        if (NG == 2) l = fmaf(sum[2] + sum[3], w_of[NG - 1], fmaf(sum[0] + sum[1], w_of[0], l));
        else l = fmaf((sum[0] + sum[1]) + (sum[2] + sum[3]), w_of[0], l);
        if (COPIES == 1) ptx::tmem_st_x32(tSg, s);
        else {
          // zeros where the other copies' keys are
          constexpr int OWN = NK / 2;
          uint32_t z[32];
#pragma unroll
          for (int j = 0; j < 32; ++j) z[j] = j / OWN == k0 / NK ? s[j % OWN] : 0u;
          ptx::tmem_st_x32(tSg, z);
        }
        const bool rescale = last_v && fac != 1.f;
        if (__any_sync(0xffffffffu, rescale)) {
          ok = ptx::mbar_wait_warp(bar(B_VFREE + (last_v - 1) % NB), ((last_v - 1) / NB) & 1u);
          ptx::tc_fence_after_sync();
#pragma unroll
          for (int i = 0; i < DH; i += 16) {
            uint32_t v[16];
            ptx::tmem_ld_x16(tOg + i, v);
            ptx::tmem_ld_wait();
#pragma unroll
            for (int j = 0; j < 16; ++j) v[j] = __float_as_uint(__uint_as_float(v[j]) * (rescale ? fac : 1.f));
            ptx::tmem_st_x16(tOg + i, v);
          }
        }
        last_v = tile + 1;
        ptx::tmem_st_wait();
        ptx::tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(bar(B_PRDY + g));
      }
      // ---------------------------------------------------------------- groups and copies of a column meet; 16 dimensions at a time
      ml[g][row] = make_float2(first ? -INFINITY : m_ref, l);
      if (last_v && ok) ok = ptx::mbar_wait_warp(bar(B_VFREE + (last_v - 1) % NB), ((last_v - 1) / NB) & 1u);
      if (!ok) lost = 1;
      softmax_sync();
      if (lost) break;                               // all eight warps or none: they meet at barriers
      float m = -INFINITY, sum = 0.f;
#pragma unroll
      for (int i = 0; i < 2 * COPIES; ++i) m = fmaxf(m, ml[i & 1][col + (i >> 1) * CHUNK].x);
#pragma unroll
      for (int i = 0; i < 2 * COPIES; ++i) {
        const float2 x = ml[i & 1][col + (i >> 1) * CHUNK];
        sum = fmaf(x.y, x.x == -INFINITY ? 0.f : ptx::ex2(x.x - m), sum);
      }
      const bool whole = w.t0 == 0 && w.t1 == w.nt;
      // the lane's own factor: to the common reference, and the quotient where the item is whole
      const float own_f = (first ? 0.f : ptx::ex2(m_ref - m)) * (whole ? 1.f / sum : 1.f);
      float *part = p.part + (int64_t)(2 * blockIdx.x + (w.t0 == 0 ? 1 : 0)) * part_floats(CHUNK, DH);
      if (g == 0 && row < w.cols) {                  // of the first copy
        const int c = w.c0 + row, rr = c / ln.group;
        if (!whole) { part[row * (DH + 4) + DH] = m; part[row * (DH + 4) + DH + 1] = sum; }
        else if (p.lse) p.lse[(int64_t)(w.row0 + rr) * p.Hq + w.h * ln.group + c - rr * ln.group] = (m + log2f(sum)) * 0.6931471805599453f;
      }
      ptx::tc_fence_after_sync();
      const uint32_t staging = base + T::STAGING;
      for (int i = 0; i < DH; i += 16) {
        uint32_t v[16];
        if (last_v) {
          ptx::tmem_ld_x16(tOg + i, v);
          ptx::tmem_ld_wait();
        } else {                                     // no tile of this piece was the group's
#pragma unroll
          for (int j = 0; j < 16; ++j) v[j] = 0u;
        }
        if (i + 16 == DH) {
          ptx::tc_fence_before_sync();
          __syncwarp();
          if (lane == 0) ptx::mbar_arrive(bar(B_OFREE));
        }
#pragma unroll
        for (int j = 0; j < 16; j += 4) {
          uint4 x;
          uint32_t *xw = &x.x;
#pragma unroll
          for (int e = 0; e < 4; ++e) xw[e] = __float_as_uint(scaled(__uint_as_float(v[j + e]), max(e0, -200) + 5) * own_f);
          ptx::st_shared_v4(staging + (g * 128 + row) * (LDS_O * 4) + j * 4, x);
        }
        softmax_sync();
        // eight dimensions of a column a thread: they lie in the order 0 4 1 5 2 6 3 7
        for (int x = threadIdx.x; x < w.cols * 2; x += SOFTMAX) {
          const int c = x >> 1, d = (x & 1) * 8;
          float y[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int e = 0; e < 2 * COPIES; ++e) {
            const uint32_t at = staging + ((e & 1) * 128 + c + (e >> 1) * CHUNK) * (LDS_O * 4) + d * 4;
            const uint4 lo = ptx::ld_shared_v4(at), hi = ptx::ld_shared_v4(at + 16);
            y[0] += __uint_as_float(lo.x); y[4] += __uint_as_float(lo.y); y[1] += __uint_as_float(lo.z); y[5] += __uint_as_float(lo.w);
            y[2] += __uint_as_float(hi.x); y[6] += __uint_as_float(hi.y); y[3] += __uint_as_float(hi.z); y[7] += __uint_as_float(hi.w);
          }
          if (whole) {
            const int cc = w.c0 + c, rr = cc / ln.group;
            Vec8<bf16> ov;
#pragma unroll
            for (int e = 0; e < 8; ++e) ov.set(e, y[e]);
            ov.store(p.out + (int64_t)(w.row0 + rr) * p.out_stride + (int64_t)(w.h * ln.group + cc - rr * ln.group) * DH + i + d);
          } else {
            float4 *dst = reinterpret_cast<float4 *>(part + c * (DH + 4) + i + d);
            dst[0] = make_float4(y[0], y[1], y[2], y[3]); dst[1] = make_float4(y[4], y[5], y[6], y[7]);
          }
        }
        softmax_sync();
      }
      pos += w.t1 - w.t0;
    }
    if (lost) { fail(status, DEV_TIMEOUT_EPILOGUE); abort_flag = 1; }
  }

  // ---------------------------------------------------------------------- teardown
  __syncwarp();
  ptx::tc_fence_before_sync();
  __syncthreads();
  if (abort_flag) {                                  // a wait ran out: copies in flight land before shared memory goes away
    const uint64_t t0 = ptx::globaltimer();
    while (ptx::globaltimer() - t0 < 200000ull) __nanosleep(1000);
    __syncthreads();
  }
  if (warp == 17) {
    ptx::tc_fence_after_sync();
    ptx::tmem_dealloc(tS, 512);
  }
}

template <int DH, int COPIES> cudaError_t launch(cudaStream_t st, const AttnParams &p, int ctas) {
  constexpr int smem = Tc<DH>::BYTES + 1024;
  cudaError_t e = cudaFuncSetAttribute(attention_kv4_tc_kernel<DH, COPIES>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  return launch_kernel(attention_kv4_tc_kernel<DH, COPIES>, dim3(ctas), dim3(THREADS), (size_t)smem, st, p);
}

template <int DH> cudaError_t launch_chunk(cudaStream_t st, const AttnParams &p, int ctas) {
  switch (p.line.chunk) {
    case 32: return launch<DH, 4>(st, p, ctas);
    case 64: return launch<DH, 2>(st, p, ctas);
    default: return launch<DH, 1>(st, p, ctas);
  }
}

}  // namespace

cudaError_t launch_attention_kv4_tc(cudaStream_t st, const AttnParams &p, int dh, int ctas) {
  return dh == 128 ? launch_chunk<128>(st, p, ctas) : launch_chunk<64>(st, p, ctas);
}

}  // namespace kv4
}  // namespace l2pd
