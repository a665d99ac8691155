// Layout of a key/value cache in 4 bits (internal).
//
// A row x of dh values (a key's, or a value's, of one head) is kept as dh codes c of 4 bits and two bf16 numbers:
//     m = min x,  s = (max x - m) / 15,  c = round((x - m) / s),  x ~ c s + m
// Products with a row then need no values, only codes: q . x = s (q . c) + m sum(q), and sum_j p_j x_j = sum_j (p_j s_j) c_j +
// sum_j p_j m_j: s and m meet the scores and the probabilities, one number a key instead of one a value.
//
// A (slot, head) is a run of tiles of 32 keys; a tile is one contiguous piece, which one bulk copy brings to shared memory:
//     [32][dh/2] codes of K | [32] (s, m) of K | [32] (s, m) of V | [32][dh/2] codes of V        32 (dh + 8) bytes
// so that the scores alone read its first half.  A row's codes are in the order of the dimensions, the even one in a byte's low
// half.  Head size 128: in V rows of keys 4..7 of every eight, the two halves of a row change places, so that the four keys whose
// rows a warp reads at once (4 keys x 32 bytes) lie in different banks.
#pragma once
#include <atomic>

#include "common.cuh"

namespace l2pd {

constexpr int KV4_TILE = 32;
constexpr int KV4_MAX_EVICT = 1 << 19;   // longest sequence an eviction takes: its bitmap lies in shared memory

__host__ __device__ __forceinline__ int kv4_tile_bytes(int dh) { return KV4_TILE * (dh + 8); }
__host__ __device__ __forceinline__ int kv4_off_kmeta(int dh) { return KV4_TILE * dh / 2; }
__host__ __device__ __forceinline__ int kv4_off_vmeta(int dh) { return KV4_TILE * dh / 2 + KV4_TILE * 4; }
__host__ __device__ __forceinline__ int kv4_off_v(int dh) { return KV4_TILE * dh / 2 + KV4_TILE * 8; }
// byte b of the V row of tile row r lies at byte b ^ kv4_v_swizzle
__host__ __device__ __forceinline__ int kv4_v_swizzle(int r, int dh) { return dh == 128 ? ((r >> 2) & 1) << 5 : 0; }

// Raises a kernel's shared-memory limit once a device; `done` has a bit a device.
inline cudaError_t allow_shared(const void *kernel, int bytes, std::atomic<uint64_t> &done) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess || (dev < 64 && (done.load(std::memory_order_relaxed) >> dev & 1u))) return e;
  e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == cudaSuccess && dev < 64) done.fetch_or(1ull << dev, std::memory_order_relaxed);
  return e;
}

struct Kv4View {
  uint8_t *data;
  int slots, heads, dh, cap;          // cap: keys the caller may address
  int64_t head_bytes, slot_bytes;
  __host__ __device__ __forceinline__ uint8_t *tile(int64_t slot, int head, int t) const {
    return data + slot * slot_bytes + head * head_bytes + (int64_t)t * kv4_tile_bytes(dh);
  }
};

// Which rows of a packed batch belong to which sequence, and where its keys lie (device arrays, each may be null)
struct Kv4Batch {
  int B, rows;                        // sequences; most rows of one
  const int32_t *row_start;           // [B + 1]; null: sequence b has the rows [b rows, (b + 1) rows)
  const int32_t *slots;               // [B]; null: sequence b lies in slot b
  const int32_t *keys;                // [B]; keys of a sequence, or its first key
  __device__ __forceinline__ int row0(int b) const { return row_start ? row_start[b] : b * rows; }
  // rows of sequence b; what the arrays cannot mean counts as none
  __device__ __forceinline__ int n_rows(int b) const {
    if (!row_start) return rows;
    const int lo = row_start[b], n = row_start[b + 1] - lo;
    return lo < 0 || n < 0 ? 0 : min(n, rows);
  }
  __device__ __forceinline__ int slot(int b, int n_slots) const {   // -1: no such slot
    const int s = slots ? slots[b] : b;
    return s >= 0 && s < n_slots ? s : -1;
  }
};

__device__ __forceinline__ float kv4_scale(uint32_t meta) { return __uint_as_float(meta << 16); }
__device__ __forceinline__ float kv4_min(uint32_t meta) { return __uint_as_float(meta & 0xffff0000u); }

// kv4.cu
cudaError_t launch_kv4_store(cudaStream_t st, const Kv4View &c, const bf16 *k, const bf16 *v, const Kv4Batch &b, int64_t k_stride, int64_t v_stride);
cudaError_t launch_kv4_load(cudaStream_t st, const Kv4View &c, int dtype, void *k, void *v, const Kv4Batch &b, int64_t k_stride, int64_t v_stride);
struct Kv4EvictArgs {
  Kv4View src, dst;
  Kv4Batch b;                         // keys: lengths
  int max_len, keep, first;
  const float *weights; float *weights_dst;            // [slots][heads][cap] of the cache they belong to; null
  const int32_t *positions; int32_t *positions_dst;
  const int32_t *protect_from;        // [B] or null
  int32_t *kept, *lens_out;           // [B][heads][keep], [B]
};
cudaError_t launch_kv4_evict(cudaStream_t st, const Kv4EvictArgs &a);

// attention_kv4.cu
struct Kv4AttnArgs {
  Kv4View c;
  Kv4Batch b;                         // keys: lengths
  int max_len, Hq;
  const bf16 *q; bf16 *out; float *lse;
  int64_t q_stride, out_stride;
  float scale;
  float *scratch;
  int32_t *status;
};
bool attention_kv4_fits(const Kv4View &c, int B, int rows, int Hq, int max_len);   // fewer than 2^31 tiles of work
int64_t attention_kv4_scratch_floats(const Kv4View &c, int B, int rows, int Hq, int max_len, int sms);
cudaError_t launch_attention_kv4(cudaStream_t st, const Kv4AttnArgs &a, int sms);
struct Kv4WeighArgs {
  Kv4View c;
  Kv4Batch b;
  int max_len, Hq;
  const bf16 *q; const float *lse;
  int64_t q_stride;
  float scale;
  const float *w_in; float *w_out;    // [slots][heads][cap]
  int32_t *status;
};
cudaError_t launch_kv4_weights(cudaStream_t st, const Kv4WeighArgs &a, int sms);

// norm_rope.cu
struct NormRopeArgs {
  const void *q, *k; void *q_out, *k_out;
  const float *q_gain, *k_gain;       // null: no norm
  const int32_t *positions;           // null: the row's number
  int rows, Hq, Hk, dh;
  int64_t q_stride, k_stride, qo_stride, ko_stride;
  float eps, theta;
  int vec;                            // 16-byte accesses allowed
};
template <typename T> cudaError_t launch_qk_norm_rope(cudaStream_t st, const NormRopeArgs &a, int sms);

}  // namespace l2pd
