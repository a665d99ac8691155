// Attention over a key/value cache in 4 bits on the 5th-generation tensor cores, for 33 to 128 columns (query rows times query heads
// that share a key head) of a sequence and key head at once.
//
// S = Q K^T and O += P V, the columns on the M side (128 lanes of tensor memory), tiles of 128 keys.  Eight warps turn codes into
// fp16 operands in shared memory, in the 128-byte swizzle:
//     K: (c - 8) s 2^-E    exact: c - 8 has three significant bits (or is 8), s has eight.  The rest of the value, a = m + 8 s,
//        reaches the scores through sixteen further products of depth, (a_hi, a_hi, a_lo) against (sum q_hi, sum q_lo, sum q_hi):
//        no number of a key's own is left for the softmax
//     V: c s 2^-E + m 2^-E in one fused operation, rounded once (2^-12 relative, or 2^-20 of 2^E)
// E belongs to 32 keys (a warp), unless one of them is 2^8 and more below the largest: then each has its own, and the softmax takes the
// tile key by key (below; likewise where scores are millions), so that a key's bits do not hang on its neighbours' size.  A code reaches fp16 as it lies, as the subnormal
// c 2^-24 (or 16 c 2^-24 from bits 4..7), and the multiplication by s 2^24 (2^20) lifts it.  Eight codes of a word come out in the order
// 0 4 1 5 2 6 3 7: queries are written in that order, and outputs read in it.
// Two groups of four softmax warps take the tiles alternately, a thread a lane: t = cf 2^E acc + (E_V - E0) - M, P = 2^t as fp16,
// the A operand of the second product.  M is a reference that follows the running maximum lazily, E0 above the largest E_V so far
// (attention_kv4.cuh has what becomes of M and the sums where it rises); O is rescaled when M moves against the scores.  The thread that has
// fixed them for a tile hands them to the other group's thread of its lane before its
// exponentials.  128 keys of a lane are read twice, 64 at a time (registers): the maximum first, then the second half, at hand
// still, then the first.  From that last read on S belongs to the tile after next, whose product runs under the exponentials (P
// over S instead: 64 numbers a head 14 % slower, 128 numbers 1 % faster).
//
// 33 to 64 columns stand twice in the lanes, and each copy takes its half of a tile's keys, its probabilities of the others being
// 0: the products are those of 128 columns, but the exponentials are spread over all warps; the copies are added at the end.
//
// What bounds it.  A tile of 128 keys of 128 numbers needs, in cycles: shared memory 1300 (17 KB of codes in and out, 64 KB of
// operands out and in, at 128 bytes), products 1090, exponentials of 128 columns 1024, issue slots 1400 of each scheduler.  It
// takes 2370 with 64 columns and 3090 with 128, no unit more than half busy: with five warps a scheduler, dependent instructions,
// instruction fetches and waits on barriers (100 each, ready or not) add up.  With exponentials, operand stores and products all
// left out the rest alone took 70 % of the time.  8 x 64 rows of 32/32 heads of 128 on 8192 keys: 154 us; 4 x 32 rows of 32/8 heads
// on 65000 keys: 186 us of 128 numbers a head, 155 of 64 (146, 170 and 140 without the look for rows apart from their neighbours and the
// code that takes them; 48 to 64 bytes of a thread's registers are spilled).  No gain: a second issuing warp, P V in two halves,
// waits that read no clock, packed f32x2 arithmetic, other register splits, all probabilities ahead of the wait for the product before.
//
// Warp roles (640 threads): 0-3 and 4-7 softmax and output, 4-7 the next piece's queries before that, 8-11 K, 12-15 V, 16 copies of
// codes, 17 MMA issuer (owns tensor memory), 18 and 19 bring the next piece's queries near.  Tensor memory: S at 0 and 128, O at
// 256, Q at 384, P at 448.
#include <cuda_fp16.h>
#include <math.h>

#include "attention_kv4.cuh"

namespace l2pd {
namespace kv4 {

namespace {

constexpr int RING = 3, NB = 2;                    // tiles of codes on their way; operand buffers
constexpr uint32_t ATOM = TC_TILE * 128;           // 128 rows x 64 fp16
constexpr float NONE = -1000.f;                    // no exponent
constexpr float FAR = 1048576.f;                   // log2 scores beyond: M, which is rounded, would take the last bits of t in one step
constexpr int SPREAD = 8;                          // 2^8 below the largest of 32, (c - 8) s is still exact and values are within 2^-11 of their row's largest
constexpr int LDS_O = 20;                          // floats of a staged row of 16
constexpr int THREADS = 640;
constexpr int REGS_SOFTMAX = 120, REGS_CODES = 88, REGS_LEAN = 56;   // 256 x 120 + 256 x 88 + 128 x 56 of 640 x 96

template <int DH> struct Tc {
  static constexpr int ATOMS = DH / 64, TILE32 = KV4_TILE * (DH + 8), STAGE = 4 * TILE32;
  // AUG: in one atom the further depth of both K buffers (32 bytes of a row each) and, at byte 64, that of the queries
  static constexpr uint32_t K = 0, AUG = NB * ATOMS * ATOM, V = AUG + ATOM, CODES = V + NB * ATOMS * ATOM,
                            STAGING = CODES + RING * STAGE, BYTES = STAGING + 2 * 128 * LDS_O * 4;
};

enum { B_FULL = 0, B_EMPTY = B_FULL + RING, B_KRDY = B_EMPTY + RING, B_KFREE = B_KRDY + NB, B_VRDY = B_KFREE + NB, B_VFREE = B_VRDY + NB,
       B_SFULL = B_VFREE + NB, B_PRDY = B_SFULL + 2, B_QRDY = B_PRDY + 2, B_OFREE = B_QRDY + 1, B_HAND = B_OFREE + 1, B_EXPO = B_HAND + 8, B_SREAD = B_EXPO + 4, B_COUNT = B_SREAD + 2 };

// x 2^n for n beyond one exponent's range
__device__ __forceinline__ float scaled(float x, int n) { const int h = n >> 1; return x * pow2(h) * pow2(n - h); }
__device__ __forceinline__ uint32_t dup(float x) { __half2 h = __float2half2_rn(x); return *reinterpret_cast<uint32_t *>(&h); }
__device__ __forceinline__ uint32_t pair(float a, float b) { __half2 h = __floats2half2_rn(a, b); return *reinterpret_cast<uint32_t *>(&h); }
__device__ __forceinline__ uint32_t hfma2(uint32_t a, uint32_t b, uint32_t c) {
  uint32_t d;
  asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
  return d;
}
__device__ __forceinline__ float key_factor(float cf, float expo_k) { return fmaxf(cf * expo_k * 4294967296.f, 1.2e-38f); }   // never 0: -inf times it stays -inf
__device__ __forceinline__ void softmax_sync() { asm volatile("bar.sync 1, 256;" ::: "memory"); }
__device__ __forceinline__ void output_sync(int g) { asm volatile("bar.sync %0, 128;" ::"r"(2 + g) : "memory"); }   // one group
// A row of codes, its quarters in an order that differs from row to row: eight lanes touch all banks, reading and writing.
template <int DH> struct Row {
  uint4 w[DH / 32];
  __device__ __forceinline__ void load(uint32_t row, int r, uint32_t swz) {
#pragma unroll
    for (int i = 0; i < DH / 32; ++i) w[i] = ptx::ld_shared_v4(row + ((16 * ((i + (r >> 1)) & (DH / 32 - 1))) ^ swz));
  }
  // To fp16: value = c s + o, s and o given times the powers of two above.  `out`: shared address of the row in the first atom.
  __device__ __forceinline__ void store(uint32_t out, int r, uint32_t s, uint32_t s16, uint32_t o) const {
#pragma unroll
    for (int i = 0; i < DH / 32; ++i) {
      const int c = (i + (r >> 1)) & (DH / 32 - 1);
      const uint32_t v[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
      const uint32_t at = out + (c >> 1) * ATOM + (((4 * (c & 1)) ^ (r & 7)) << 4);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t hi = v[j] >> 8;
        ptx::st_shared_v4(at ^ (j << 4), make_uint4(hfma2(v[j] & 0x000f000fu, s, o), hfma2(v[j] & 0x00f000f0u, s16, o),
                                                    hfma2(hi & 0x000f000fu, s, o), hfma2(hi & 0x00f000f0u, s16, o)));
      }
    }
  }
};

// Exponents of a tile, by group of 32 keys; those of V are told ahead of the operands, those of K come with the scores
struct Exponents {
  float k[4], v[4];                                // negative, and larger by APART: the group's keys have exponents of their own,
  int16_t below_k[TC_TILE], below_v[TC_TILE];      // that lie below it by this
};
constexpr int APART = 1024;

template <int DH, int COPIES>
__global__ void __launch_bounds__(THREADS, 1) attention_kv4_tc_kernel(const AttnParams p) {
  using T = Tc<DH>;
  constexpr int CHUNK = 128 / COPIES, KEYS = TC_TILE / COPIES;   // columns; keys of a tile that a copy takes
  // Halves of a copy's keys whose exponentials are written out: the code of the tile loop is fetched again and again by eight warps at
  // different places in it (128 columns, 65000 keys, us, one / two: heads of 64 154 / 157, of 128 189 / 185)
  constexpr int TURNS = DH == 64 ? 1 : 2;
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t bars[B_COUNT];
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_flag;
  __shared__ __align__(16) Exponents expo[4];      // of tile % 4
  __shared__ int lost;                             // a softmax warp's wait ran out
  __shared__ float2 hand[2][128];                  // [group][lane]: reference and E0 of the group's last tile
  __shared__ float2 sums[2][128];                  // [group][lane]: the reference its sum is against, the sum
  __shared__ float2 ml[2][128];                    // [group][lane]: a lane's reference and sum
  __shared__ float q_factor[2][128];
  const int warp = ptx::warp_index(), lane = threadIdx.x & 31;
  const uint32_t base = (ptx::smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t bar0 = ptx::smem_u32(bars);
  auto bar = [&](int i) { return bar0 + 8u * i; };
  if (threadIdx.x == 0) {
    for (int i = 0; i < RING; ++i) { ptx::mbar_init(bar(B_FULL + i), 1); ptx::mbar_init(bar(B_EMPTY + i), 8); }
    for (int i = 0; i < NB; ++i) {
      ptx::mbar_init(bar(B_KRDY + i), 4); ptx::mbar_init(bar(B_KFREE + i), 1);
      ptx::mbar_init(bar(B_VRDY + i), 4); ptx::mbar_init(bar(B_VFREE + i), 1);
    }
    for (int i = 0; i < 2; ++i) { ptx::mbar_init(bar(B_SFULL + i), 2); ptx::mbar_init(bar(B_SREAD + i), 4); ptx::mbar_init(bar(B_PRDY + i), 4); }
    ptx::mbar_init(bar(B_QRDY), 4); ptx::mbar_init(bar(B_OFREE), 8);
    for (int i = 0; i < 8; ++i) ptx::mbar_init(bar(B_HAND + i), 1);
    for (int i = 0; i < 4; ++i) ptx::mbar_init(bar(B_EXPO + i), 4);
    abort_flag = 0; lost = 0;
    ptx::fence_barrier_init();
    ptx::fence_proxy_async();
  }
  if (warp == 17) { ptx::tmem_alloc(ptx::smem_u32(&tmem_slot), 512); ptx::tmem_relinquish(); }
  ptx::tc_fence_before_sync();
  __syncthreads();
  ptx::tc_fence_after_sync();
  const uint32_t tS = tmem_slot, tO = tS + 256, tQ = tS + 384, tP = tS + 448;
  int32_t *const status = p.status;
  grid_dep_wait();
  grid_dep_launch();                               // behind the wait: see the joining kernel

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

  if (warp >= 16) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(REGS_LEAN));
  if (warp == 16) {
    // ------------------------------------------------------------------ codes: up to four tiles of the cache, one contiguous piece
    int slot = 0;
    uint32_t par = 1;
    for (uint32_t pos = begin; pos < end;) {
      const Piece w = piece_at(pos);
      const uint8_t *src = p.c.tile(w.slot, w.h, 0);
      for (int t = w.t0; t < w.t1; ++t) {
        const bool ok = ptx::mbar_wait_or_abort(bar(B_EMPTY + slot), par, &abort_flag, status, DEV_TIMEOUT_PRODUCER);
        const uint32_t bytes = min(4, (w.keys - t * TC_TILE + KV4_TILE - 1) / KV4_TILE) * T::TILE32;
        if (ptx::elect_one() && ok) {
          ptx::mbar_arrive_expect_tx(bar(B_FULL + slot), bytes);
          ptx::bulk_load(base + T::CODES + slot * T::STAGE, src + (int64_t)t * T::STAGE, bytes, bar(B_FULL + slot));
        }
        if (++slot == RING) { slot = 0; par ^= 1u; }
      }
      pos += w.t1 - w.t0;
    }
  } else if (warp == 17) {
    // ------------------------------------------------------------------ MMA issuer: S(0) S(1) S(2) PV(0) S(3) PV(1) ...
    constexpr uint32_t F32 = 1u << 4, M128 = (128u >> 4) << 24;
    const uint32_t idesc_s = F32 | M128 | ((TC_TILE >> 3) << 17), idesc_o = F32 | M128 | ((DH >> 3) << 17) | (1u << 16);
    uint32_t ts = 0, tp = 0, qpar = 0, opar = 1;     // tiles whose S, whose PV was issued
    auto scores = [&]() {
      const uint32_t b = ts & 1u;
      bool ok = ptx::mbar_wait_or_abort(bar(B_KRDY + b), (ts >> 1) & 1u, &abort_flag, status, DEV_TIMEOUT_MMA);
      ok = ptx::mbar_wait_or_abort(bar(B_SREAD + b), ((ts >> 1) & 1u) ^ 1u, &abort_flag, status, DEV_TIMEOUT_MMA) && ok;
      ptx::tc_fence_after_sync();
      const uint64_t kd = ptx::smem_desc_sw128(base + T::K + b * T::ATOMS * ATOM), ad = ptx::smem_desc_sw128(base + T::AUG);
      if (ptx::elect_one() && ok) {
#pragma unroll
        for (int k = 0; k < DH / 16; ++k)
          ptx::mma_bf16_ts(tS + b * TC_TILE, tQ + 8 * k, kd + (k >> 2) * (ATOM >> 4) + 2u * (k & 3), idesc_s, k ? 1u : 0u);
        ptx::mma_bf16_ss(tS + b * TC_TILE, ad + 4u, ad + 2u * b, idesc_s, 1u);
        ptx::mma_commit(bar(B_KFREE + b));
        ptx::mma_commit(bar(B_SFULL + b));
        ptx::mbar_arrive(bar(B_SFULL + b));          // passes on what the K and the query warps wrote besides
      }
      ++ts;
    };
    auto output = [&](bool first) {
      const uint32_t b = tp & 1u, par = (tp >> 1) & 1u;
      bool ok = ptx::mbar_wait_or_abort(bar(B_VRDY + b), par, &abort_flag, status, DEV_TIMEOUT_MMA);
      if (first) {                                   // the piece before has been read out of O
        ok = ptx::mbar_wait_or_abort(bar(B_OFREE), opar, &abort_flag, status, DEV_TIMEOUT_MMA) && ok;
        opar ^= 1u;
      }
      ok = ptx::mbar_wait_or_abort(bar(B_PRDY + b), par, &abort_flag, status, DEV_TIMEOUT_MMA) && ok;
      ptx::tc_fence_after_sync();
      const uint64_t vd = ptx::smem_desc_sw128_mn(base + T::V + b * T::ATOMS * ATOM, ATOM);
      if (ptx::elect_one() && ok) {
#pragma unroll
        for (int k = 0; k < TC_TILE / 16; ++k)
          ptx::mma_bf16_ts(tO, tP + 8 * k, vd + k * (2048u >> 4), idesc_o, k ? 1u : first ? 0u : 1u);
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
        if (i + 2 < n) scores();
        output(i == 0);
      }
      pos += n;
    }
  } else if (warp >= 18) {
    // ------------------------------------------------------------------ the next piece's query rows to this SM's cache
    for (uint32_t pos = begin; pos < end;) {
      const Piece w = piece_at(pos);
      const int c = w.c0 + (warp - 18) * 32 + lane;
      for (int x = c; x < w.c0 + w.cols; x += 64) {
        const int rr = x / ln.group;
        const bf16 *src = p.q + (int64_t)(w.row0 + rr) * p.q_stride + (int64_t)(w.h * ln.group + x - rr * ln.group) * DH;
#pragma unroll
        for (int i = 0; i < DH; i += 64) asm volatile("{\n\t.reg .b32 t;\n\tld.global.ca.b32 t, [%0];\n\t}" ::"l"(src + i) : "memory");
      }
      pos += w.t1 - w.t0;
    }
  } else if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(REGS_CODES));
    // ------------------------------------------------------------------ codes to operands
    const bool is_v = warp >= 12;
    const int grp = warp & 3, r = 32 * grp + lane;
    const uint32_t swz = is_v ? kv4_v_swizzle(lane, DH) : 0;
    const uint32_t out = base + (is_v ? T::V : T::K) + r * 128, aug = base + T::AUG + r * 128;
    const uint32_t row_off = grp * T::TILE32 + (is_v ? kv4_off_v(DH) : 0) + lane * (DH / 2);
    const uint32_t meta_off = grp * T::TILE32 + (is_v ? kv4_off_vmeta(DH) : kv4_off_kmeta(DH)) + 4 * lane;
    int slot = 0;
    uint32_t par = 0, tile = 0;
    bool ok = true;
    for (uint32_t pos = begin; pos < end && ok;) {
      const Piece w = piece_at(pos);
      for (int t = w.t0; t < w.t1 && ok; ++t, ++tile) {
        const uint32_t b = tile & 1u, stage = base + T::CODES + slot * T::STAGE;
        ok = ptx::mbar_wait_warp(bar(B_FULL + slot), par);
        if (!ok) break;
        Row<DH> row;
        row.load(stage + row_off, r, swz);
        uint32_t meta = 0;
        if (t * TC_TILE + r < w.keys) asm volatile("ld.shared.b32 %0, [%1];" : "=r"(meta) : "r"(stage + meta_off) : "memory");
        const float s = kv4_scale(meta), m = kv4_min(meta);
        // the group's exponent; keys that are not finite stay outside it
        const int es = (int)((meta >> 7) & 255u), em = (int)((meta >> 23) & 255u);
        int e = es == 255 || em == 255 ? 0 : is_v ? max(es + 4, em) : max(es, em - 11);
        const bool zero = (meta & 0x7fff7fffu) == 0u, none = is_v && __all_sync(0xffffffffu, zero);   // values that are all 0 have no exponent
        const bool real = !zero && es != 255 && em != 255;
        e = max(e, 0);
        const int most = max((int)__reduce_max_sync(0xffffffffu, (uint32_t)e), 26), least = max((int)__reduce_min_sync(0xffffffffu, real ? (uint32_t)e : 255u), 26);
        const int group_e = most - 126 + (is_v ? 1 : 0);
        // V: |value| < 2^e, as fp16 times 2^-(e + 5); K: s < 2^e, times 2^-(e + 9)
        const int down = -(group_e + (is_v ? 5 : 9));
        float s1 = scaled(s, down), m1 = scaled(m, down);
        int below_k = 0;
        const bool apart = most - least > SPREAD;
        if (apart) {
          // rows further below the group's largest than fp16 bears keep exponents of their own; rows of zeros go with the smallest
          const int below = real ? max(e, 26) - most : zero ? least - most : 0;
          if (is_v) expo[tile & 3u].below_v[r] = (int16_t)below;
          else below_k = below;
          s1 = scaled(s, down - below); m1 = scaled(m, down - below);
        }
        if (is_v && lane == 0) expo[tile & 3u].v[grp] = none ? NONE : (float)(apart ? group_e + APART : group_e);
        const float o = is_v ? m1 : -8.f * s1, a = m1 + 8.f * s1;
        // the next copy overwrites what was read: reads come before it only by a fence between the two ways to shared memory (without one
        // the compiler may put them off to where the values are used, behind the wait below)
        ptx::fence_proxy_async();
        __syncwarp();
        if (lane == 0) {
          ptx::mbar_arrive(bar(B_EMPTY + slot));
          if (is_v) ptx::mbar_arrive(bar(B_EXPO + (tile & 3u)));
        }
        ok = ptx::mbar_wait_warp(bar((is_v ? B_VFREE : B_KFREE) + b), ((tile >> 1) & 1u) ^ 1u);
        if (!ok) break;
        row.store(out + b * T::ATOMS * ATOM, r, dup(s1 * 16777216.f), dup(s1 * 1048576.f), dup(o));
        if (!is_v) {
          const float hi = __half2float(__float2half_rn(a));
          const uint32_t at = aug + (((2 * b) ^ (r & 7)) << 4);
          ptx::st_shared_v4(at, make_uint4(pair(hi, hi), pair((a - hi) * 2048.f, 0.f), 0u, 0u));
          ptx::st_shared_v4(at ^ 16u, make_uint4(0u, 0u, 0u, 0u));
        }
        if (!is_v && apart) expo[tile & 3u].below_k[r] = (int16_t)below_k;
        if (!is_v && lane == 0) expo[tile & 3u].k[grp] = apart ? -pow2(group_e + 9 - 32) : pow2(group_e + 9 - 32);   // group_e reaches 128
        ptx::fence_proxy_async();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(bar((is_v ? B_VRDY : B_KRDY) + b));
        if (++slot == RING) { slot = 0; par ^= 1u; }
      }
      pos += w.t1 - w.t0;
    }
    if (!ok) { fail(status, DEV_TIMEOUT_PRODUCER); abort_flag = 1; }
  } else {
    // ------------------------------------------------------------------ queries, softmax, output
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(REGS_SOFTMAX));
    const int g = warp >> 2, q = warp & 3, row = 32 * q + lane;
    const int col = row & (CHUNK - 1);               // this lane's column of the chunk
    const int copy = q / (4 / COPIES);               // its first key of a tile: copy * KEYS
    constexpr int NG = KEYS / 32, HALF = 64, HG = HALF / 32;      // exponents of a copy's keys; keys taken at once
    const uint32_t mine = bar(B_HAND + 4 * g + q), theirs = bar(B_HAND + 4 * (g ^ 1) + q);
    const uint32_t lane_base = (uint32_t)(32 * q) << 16, tOr = tO + lane_base, tPr = tP + lane_base;
    if (COPIES > 1 && g == 0) {                      // zeros where the other copy's keys are
      uint32_t z[32];
#pragma unroll
      for (int j = 0; j < 32; ++j) z[j] = 0u;
      ptx::tmem_st_x32(tPr + 32 * (copy ^ 1), z);
      ptx::tmem_st_wait();
    }
    uint32_t tile = 0, piece = 0;
    bool ok = true;
    // Queries of a piece to tensor memory and AUG (group 1): the largest of a row becomes 2^7 .. 2^8
    auto queries = [&](const Piece &w, uint32_t parity) {
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
      // the scale's sign goes with the queries: the largest product is then the largest score
      const float up = p.scale_log2 < 0.f ? -pow2(u) : pow2(u);
      q_factor[parity][row] = fabsf(p.scale_log2) * pow2(-u);
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
      const uint32_t at = base + T::AUG + row * 128 + ((4 ^ (row & 7)) << 4);
      // a NaN here makes every score of the row NaN
      ptx::st_shared_v4(at, make_uint4(finite ? pair(hi, sum - hi) : 0x7fff7fffu, pair(hi * (1.f / 2048.f), 0.f), 0u, 0u));
      ptx::st_shared_v4(at ^ 16u, make_uint4(0u, 0u, 0u, 0u));
      ptx::fence_proxy_async();
      ptx::tmem_st_wait();
      ptx::tc_fence_before_sync();
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(bar(B_QRDY));
    };
    // Queries of a piece, then the output of the one before, then the piece's tiles
    Piece w = {}, old = {};
    float2 last = {}, x0 = {}, x1 = {};              // of the piece before: reference, the groups' sums
    for (uint32_t pos = begin; begin < end; ++piece) {
      const bool more = pos < end;
      if (more) {
        w = piece_at(pos);
        if (g == 1) queries(w, piece & 1u);
      }
      if (piece > 0) {
        // the copies of a column meet.  Each group brings half of the dimensions, 16 at a time
        const float m_ref = last.x;
        // without a reference: no keys, or NaN alone
        auto against = [&](float2 x) { return x.x == -INFINITY ? 0.f * x.y : ex2_scaled(x.y, x.x - m_ref); };
        const Normal own = normalised(against(x0) + against(x1), m_ref, (int)fmaxf(last.y, -100.f) + 5);   // values in the unit 2^(E0 + 5)
        ml[g][row] = make_float2(own.ref, own.x);
        ok = ok && ptx::mbar_wait_warp(bar(B_VFREE + ((tile - 1) & 1u)), ((tile - 1) >> 1) & 1u);
        output_sync(g);
        float m = -INFINITY, sum = 0.f;
#pragma unroll
        for (int i = 0; i < COPIES; ++i) m = fmaxf(m, ml[g][col + i * CHUNK].x);
#pragma unroll
        for (int i = 0; i < COPIES; ++i) {
          const float2 x = ml[g][col + i * CHUNK];
          sum = fmaf(x.y, x.x == -INFINITY ? 0.f : ptx::ex2(x.x - m), sum);
        }
        const bool whole = old.t0 == 0 && old.t1 == old.nt;
        // the lane's own factor: to the common reference, and the quotient where the item is whole
        const float f_a = (own.ref == -INFINITY ? 0.f : ptx::ex2(own.ref - m)) * (whole ? 1.f / sum : 1.f) * own.up_a, f_b = own.up_b;
        float *part = p.part + (int64_t)(2 * blockIdx.x + (old.t0 == 0 ? 1 : 0)) * part_floats(CHUNK, DH);
        if (g == 0 && row < old.cols) {                  // of the first copy
          const int c = old.c0 + row, rr = c / ln.group;
          if (!whole) { part[row * (DH + 4) + DH] = m; part[row * (DH + 4) + DH + 1] = sum; }
          else if (p.lse) p.lse[(int64_t)(old.row0 + rr) * p.Hq + old.h * ln.group + c - rr * ln.group] = (m + log2f(sum)) * 0.6931471805599453f;
        }
        ptx::tc_fence_after_sync();
        const uint32_t staging = base + T::STAGING + g * (128 * LDS_O * 4);
#pragma unroll 1
        for (int i = g * (DH / 2); i < (g + 1) * (DH / 2); i += 16) {
          uint32_t v[16];
          ptx::tmem_ld_x16(tOr + i, v);
          ptx::tmem_ld_wait();
          if (i + 16 == (g + 1) * (DH / 2)) {
            ptx::tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(bar(B_OFREE));
          }
#pragma unroll
          for (int j = 0; j < 16; j += 4) {
            uint4 x;
            uint32_t *xw = &x.x;
#pragma unroll
            for (int e = 0; e < 4; ++e) xw[e] = __float_as_uint(__uint_as_float(v[j + e]) * f_a * f_b);
            ptx::st_shared_v4(staging + row * (LDS_O * 4) + j * 4, x);
          }
          output_sync(g);
          // eight dimensions of a column a thread: they lie in the order 0 4 1 5 2 6 3 7
          for (int x = threadIdx.x & 127; x < old.cols * 2; x += 128) {
            const int c = x >> 1, d = (x & 1) * 8;
            float y[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int e = 0; e < COPIES; ++e) {
              const uint32_t at = staging + (c + e * CHUNK) * (LDS_O * 4) + d * 4;
              const uint4 lo = ptx::ld_shared_v4(at), hi = ptx::ld_shared_v4(at + 16);
              y[0] += __uint_as_float(lo.x); y[4] += __uint_as_float(lo.y); y[1] += __uint_as_float(lo.z); y[5] += __uint_as_float(lo.w);
              y[2] += __uint_as_float(hi.x); y[6] += __uint_as_float(hi.y); y[3] += __uint_as_float(hi.z); y[7] += __uint_as_float(hi.w);
            }
            if (whole) {
              const int cc = old.c0 + c, rr = cc / ln.group;
              Vec8<bf16> ov;
#pragma unroll
              for (int e = 0; e < 8; ++e) ov.set(e, y[e]);
              ov.store(p.out + (int64_t)(old.row0 + rr) * p.out_stride + (int64_t)(old.h * ln.group + cc - rr * ln.group) * DH + i + d);
            } else {
              float4 *dst = reinterpret_cast<float4 *>(part + c * (DH + 4) + i + d);
              dst[0] = make_float4(y[0], y[1], y[2], y[3]); dst[1] = make_float4(y[4], y[5], y[6], y[7]);
            }
          }
          output_sync(g);
        }
      }
      if (!more) break;
      float m_own = -INFINITY, l = 0.f, cf = 0.f;    // the reference l is against
      for (int t = w.t0; t < w.t1; ++t, ++tile) {
        if ((tile & 1u) != (uint32_t)g) continue;
        const uint32_t b = (uint32_t)g, par = (tile >> 1) & 1u;
        ok = ok && ptx::mbar_wait_warp(bar(B_EXPO + (tile & 3u)), (tile >> 2) & 1u);
        ok = ok && ptx::mbar_wait_warp(bar(B_SFULL + b), par);
        if (!ok) break;
        ptx::tc_fence_after_sync();
        if (m_own == -INFINITY) cf = q_factor[piece & 1u][row];
        const uint32_t tSr = tS + lane_base + b * TC_TILE, tSk = tSr + copy * KEYS;
        const Exponents &ex = expo[tile & 3u];
        float k[NG], ev[NG], e_top = NONE, k_least = 0.f;
#pragma unroll
        for (int i = 0; i < NG; ++i) {
          ev[i] = ex.v[copy * NG + i];
          k[i] = key_factor(cf, ex.k[copy * NG + i]);
          e_top = fmaxf(e_top, ev[i]);
          k_least = fminf(k_least, ex.k[copy * NG + i]);
        }
        const int left = w.keys - t * TC_TILE - copy * KEYS;
        uint32_t s[HALF];
        auto load = [&](int from) {
#pragma unroll
          for (int i = 0; i < HALF; i += 32) ptx::tmem_ld_x32(tSk + from + i, s + i);
          ptx::tmem_ld_wait();
        };
        // Scores behind the end.  In tensor memory and 16 at a time, as all that is rare here: the code of the tile loop is read again and again
        // by eight warps at different places, and each KB of it beside the exponentials costs every tile
        if (left < KEYS) {
#pragma unroll 1
          for (int c = max(left, 0) & ~15; c < KEYS; c += 16) {
            uint32_t x[16];
            ptx::tmem_ld_x16(tSk + c, x);
            ptx::tmem_ld_wait();
#pragma unroll
            for (int j = 0; j < 16; ++j) if (c + j >= left) x[j] = 0xff800000u;
            ptx::tmem_st_x16(tSk + c, x);
          }
          ptx::tmem_st_wait();
        }
        auto release = [&]() {                       // these scores were read for the last time
          ptx::tc_fence_before_sync();
          __syncwarp();
          if (lane == 0) ptx::mbar_arrive(bar(B_SREAD + b));
        };
        float top[NG], hi = -INFINITY;               // largest scores of the groups, of all
#pragma unroll 1
        for (int from = 0; from < KEYS; from += HALF) {
          load(from);
#pragma unroll
          for (int i = 0; i < HG; ++i) {
            float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
            for (int j = 0; j < 32; ++j) mx[j & 3] = fmaxf(mx[j & 3], __uint_as_float(s[32 * i + j]));
            top[NG - HG + i] = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
            if (KEYS > HALF && from == 0) top[i] = top[NG - HG + i];
          }
        }
#pragma unroll
        for (int i = 0; i < NG; ++i) {
          top[i] *= k[i];
          hi = fmaxf(hi, top[i]);
        }
        const bool by_key = __any_sync(0xffffffffu, k_least < 0.f || e_top > APART / 2 || (fabsf(hi) > FAR && hi > -INFINITY));
        float m_was = -INFINITY, e_was = NONE;       // the reference of the tile before
        auto received = [&]() {
          if (t == w.t0) return;
          ok = ptx::mbar_wait_warp(theirs, ((tile - 1) >> 1) & 1u);
          const float2 x = hand[g ^ 1][row];
          m_was = x.x; e_was = x.y;
        };
        auto hand_over = [&](float m, float e) {
          hand[g][row] = make_float2(m, e);
          __syncwarp();
          if (lane == 0) ptx::mbar_arrive(mine);
          if (m_own != m) l = m_own == -INFINITY ? 0.f * l : ex2_scaled(l, m_own - m);
          m_own = m;
        };
        auto product_done = [&]() {                  // that of the tile before: its probabilities may be written over
          if (t == w.t0) return;
          ok = ptx::mbar_wait_warp(bar(B_VFREE + (b ^ 1u)), ((tile - 1) >> 1) & 1u);
          ptx::tc_fence_after_sync();
        };
        bool moved;
        float fac;                                   // of O
        if (!by_key) {
          if (KEYS == HALF) release();
          received();
          if (!ok) break;
          // E0 rises to a new largest exponent, M falls with it and moves where need be
          const float e0 = e_top > e_was ? e_top + 2.f : e_was, d = e_was == NONE ? 0.f : e0 - e_was, m_low = m_was - d;
          float rise = -INFINITY, o[NG];
#pragma unroll
          for (int i = 0; i < NG; ++i) {             // keys whose values are all 0 have no exponent
            o[i] = ev[i] == NONE ? FLOOR : fmaxf(ev[i] - e0, FLOOR);
            rise = fmaxf(rise, top[i] + o[i]);
          }
          // a copy whose keys all lie behind the end keeps an open reference
          const bool open = m_was == -INFINITY;
          const float m_ref = open || rise - m_low > LAZY ? rise - BELOW : m_low;
          hand_over(m_ref, e0);
          moved = t > w.t0 && m_was - m_ref != d;    // NaN where both are open; not m_low: beyond 2^24 it is no exact difference
          fac = open ? 0.f : ptx::ex2(m_was - m_ref - d);
          const float m_use = m_ref == -INFINITY ? 0.f : m_ref;
          // probabilities, the second half first
#pragma unroll TURNS
          for (int from = KEYS - HALF; from >= 0; from -= HALF) {
            if (from != KEYS - HALF) {
              load(from);
              release();
            }
#pragma unroll
            for (int i = 0; i < HG; ++i) {
              const float kk = from ? k[NG - HG + i] : k[i], oi = from ? o[NG - HG + i] : o[i], oo = oi - m_use;
              float sum[2] = {0.f, 0.f};
#pragma unroll
              for (int j = 0; j < 32; j += 2) {
                const float p0 = ptx::ex2(fmaf(__uint_as_float(s[32 * i + j]), kk, oo)), p1 = ptx::ex2(fmaf(__uint_as_float(s[32 * i + j + 1]), kk, oo));
                sum[(j >> 1) & 1] += p0 + p1;
                s[16 * i + (j >> 1)] = pair(p0, p1);
              }
              l = fmaf(sum[0] + sum[1], ptx::ex2(-oi - LOG_L), l);
            }
            if (from == KEYS - HALF) product_done();
            ptx::tmem_st_x32(tPr + (copy * KEYS + from) / 2, s);
          }
        } else {
          // Key by key, 16 at a time, the parts of t apart.  (M, E0) become score and exponent of the key with the largest sum of both
          float m_top = -INFINITY, e_best = NONE;
          auto each_key = [&](auto &&use) {
#pragma unroll 1
            for (int c = 0; c < KEYS; c += 16) {
              uint32_t v[16];
              ptx::tmem_ld_x16(tSk + c, v);
              const int grp = copy * NG + c / 32;
              const bool own_k = ex.k[grp] < 0.f, own_v = ex.v[grp] > APART / 2;
              const float kk = key_factor(cf, fabsf(ex.k[grp])), e = own_v ? ex.v[grp] - APART : ex.v[grp];
              ptx::tmem_ld_wait();
#pragma unroll
              for (int j = 0; j < 16; ++j)
                use(c, j, __fmul_rn(__uint_as_float(v[j]), own_k ? kk * pow2(max((int)ex.below_k[copy * KEYS + c + j], -126)) : kk),
                    own_v ? e + (float)ex.below_v[copy * KEYS + c + j] : e);
            }
          };
          each_key([&](int, int, float x, float e) {
            if (m_top == -INFINITY || x - m_top + (e - e_best) > 0.f) { m_top = x; e_best = e; }
          });
          received();
          if (!ok) break;
          const bool open = m_was == -INFINITY, move = open || m_top - m_was + (e_best - e_was) > LAZY;
          const float m_ref = move ? m_top - BELOW : m_was, e_ref = move ? e_best : e_was, m_use = m_ref == -INFINITY ? 0.f : m_ref;
          hand_over(m_ref, e_ref);
          moved = t > w.t0 && move;
          fac = open ? 0.f : ptx::ex2(m_was - m_ref + (e_was - e_ref));
          product_done();
          float sum = 0.f;
          uint32_t packed[8];
          float even = 0.f;
          each_key([&](int c, int j, float x, float e) {
            const float y = ptx::ex2(x - m_use + (e - e_ref));
            sum += ptx::ex2(x - m_use - LOG_L);
            if (j & 1) packed[j >> 1] = pair(even, y); else even = y;
            if (j == 15) ptx::tmem_st_x8(tPr + (copy * KEYS + c) / 2, packed);
          });
          l += sum;
          release();
        }
        if (!ok) break;
        if (__any_sync(0xffffffffu, moved)) {
#pragma unroll 1
          for (int i = 0; i < DH; i += 32) {
            uint32_t v[32];
            ptx::tmem_ld_x32(tOr + i, v);
            ptx::tmem_ld_wait();
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] = __float_as_uint(__uint_as_float(v[j]) * fac);
            ptx::tmem_st_x32(tOr + i, v);
          }
        }
        ptx::tmem_st_wait();
        ptx::tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(bar(B_PRDY + b));
      }
      // ---------------------------------------------------------------- the end of a piece
      pos += w.t1 - w.t0;
      sums[g][row] = make_float2(m_own, l);
      if (!ok) lost = 1;
      softmax_sync();
      if (lost) break;                               // all eight warps or none: they meet at barriers
      last = hand[(tile - 1) & 1u][row]; x0 = sums[0][row]; x1 = sums[1][row];
      old = w;
      softmax_sync();                                // the next piece may write them again
    }
    if (!ok || lost) { fail(status, DEV_TIMEOUT_EPILOGUE); abort_flag = 1; }
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
  static_assert(smem + 9888 <= 227 * 1024, "with what the kernel declares itself");
  static std::atomic<uint64_t> done{0};
  const cudaError_t e = allow_shared((const void *)attention_kv4_tc_kernel<DH, COPIES>, smem, done);
  if (e != cudaSuccess) return e;
  return launch_kernel(attention_kv4_tc_kernel<DH, COPIES>, dim3(ctas), dim3(THREADS), (size_t)smem, st, p);
}

template <int DH> cudaError_t launch_chunk(cudaStream_t st, const AttnParams &p, int ctas) {
  switch (p.line.chunk) {
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
