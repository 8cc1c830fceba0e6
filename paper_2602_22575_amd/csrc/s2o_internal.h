// Internal declarations shared by the host API and the gfx950 kernels of the S2O library.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <mutex>

namespace s2o {

// Packed start of prefix row n (n >= 1) inside one head's KV_perm / s_K array.
__host__ __device__ inline int64_t kv_row_offset(int64_t n, int64_t S) { return S * n * (n - 1) / 2; }

// Rows of KV_perm / s_K for one head.  Causal (the paper's setting): row n ranks the n*S
// tokens before segment n and the rows are packed.  Without causality (params.non_causal,
// the setting of the paper's non-causal decomposition and top-k comparisons) every row
// ranks all L tokens.
__host__ __device__ inline int64_t kv_row_len(int64_t n, int64_t S, int64_t L, int nc) { return nc ? L : n * S; }
__host__ __device__ inline int64_t kv_row_start(int64_t n, int64_t S, int64_t L, int nc) {
  return nc ? n * L : kv_row_offset(n, S);
}
__host__ __device__ inline int64_t kv_rows_total(int64_t N, int64_t S, int64_t L, int nc) {
  return nc ? N * L : kv_row_offset(N, S);
}

// Runs `setup` (kernel attributes such as the dynamic LDS limit are per device) once per
// device, before the first launch there; other host threads wait until it is done.  A failed
// setup is retried by the next call.
template <class F>
inline hipError_t once_per_device(std::mutex& mu, uint64_t& done, F setup) {
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  const uint64_t bit = 1ull << (dev & 63);
  std::lock_guard<std::mutex> lock(mu);
  if (done & bit) return hipSuccess;
  e = setup();
  if (e == hipSuccess) done |= bit;
  return e;
}

struct AttnArgs {
  const uint16_t* Q;
  const uint16_t* K;
  const uint16_t* V;
  uint16_t* O;
  const int32_t* q_perm;
  const int32_t* kv_perm;
  int32_t* computed;
  int32_t* skipped;
  int passes;     // 0: one fused launch; bit 0: Alg. 2 into the state buffers; bit 1: Alg. 3 from them
  float* st_acc;  // state buffers: acc [Z*H*L][128] (four 128-byte lines per row, see attn_tile.h), then l and m [Z*H*L]
  float* st_l;
  float* st_m;
  int Z, H, Hkv, L, S, N;
  int BM;  // query tile rows (64 or 128); the key tile is 64 tokens
  int use_q_perm, stop_mode;
  int non_causal; // every query attends every key: no own-segment pass, rows of L ranked keys
  int max_tiles;  // > 0: a query tile visits at most this many prefix tiles
  float tau;
  float scale_log2e;  // softmax_scale * log2(e): logits are kept in base-2 units
  int64_t qs[3], ks[3], vs[3], os[3];
};

struct PlanArgs {
  const uint16_t* Q;
  const uint16_t* K;
  int32_t* q_perm;
  int32_t* kv_perm;
  float* s_q;
  float* s_k;
  float* q_mean;
  float* k_guide;
  int32_t* status;   // optional: receives the S2O_PLAN_* bits (0 = every invariant held)
  int Z, H, Hkv, L, S, N;
  int non_causal;
  int64_t qs[3], ks[3];
  void* scratch;
  size_t scratch_bytes;
};

size_t plan_scratch_bytes(int Z, int H, int Hkv, int L, int S, int non_causal);
// Size of the library's built-in plan scratch (S2O_STATIC_SCRATCH_BYTES of the C header) and its
// device address on the current GPU.
constexpr size_t kStaticPlanScratchBytes = (size_t)32 << 20;
hipError_t static_plan_scratch(void** ptr);
size_t attention_state_bytes(int Z, int H, int L);
hipError_t launch_plan(const PlanArgs& a, hipStream_t stream);
hipError_t launch_attention(const AttnArgs& a, hipStream_t stream);
// Debug check of q_perm / kv_perm ranges (allocates, synchronises `stream`); bits: 1 = Q_perm, 2 = KV_perm
hipError_t validate_maps(const AttnArgs& a, hipStream_t stream, int* bits);
// Alg. 2 alone (local.hip): own-segment pass in original query order into the state buffers
hipError_t launch_local(const AttnArgs& a, hipStream_t stream);
// Alg. 3 alone (prefix.hip): prefix walk in permuted query order from the state buffers
hipError_t launch_prefix(const AttnArgs& a, hipStream_t stream);

// Notes a failed HIP call for s2o_last_hip_error; S2O_EHIP.
int hip_fail(hipError_t e);

// A launch counts its threads in 32 bits.  (The cache's launches return hipErrorNotSupported, before the first one, where that is too few.)
inline bool fits_launch(int64_t blocks, int threads) { return blocks > 0 && blocks <= (int64_t)0xffffffff / threads; }

// Quotient and rest of non-negative numbers below 2^31 by d = 1 .. 2^31 - 1 that the host has prepared: a product's upper half instead of the
// forty instructions of a division.  mul = ceil(2^(31 + s) / d), 2^(s-1) < d <= 2^s: n * mul / 2^(31 + s) is off by less than 1/d above.
// Laid out to be loaded in one piece.
struct alignas(16) Divisor {
  uint32_t mul, shift, d, whole;   // whole: all bits set where d = 1, whose mul has no room
  Divisor() = default;
  __host__ explicit Divisor(uint32_t d_) : mul(0), shift(0), d(d_), whole(~0u) {
    if (d <= 1) return;
    uint32_t s = 0;
    while ((1ull << s) < d) ++s;
    mul = (uint32_t)(((1ull << (31 + s)) + d - 1) / d);
    shift = s - 1;
    whole = 0;
  }
  __device__ __forceinline__ int by(int n, int& rest) const {
    const uint32_t q = (__umulhi((uint32_t)n, mul) + ((uint32_t)n & whole)) >> shift;
    rest = n - (int)(q * d);
    return (int)q;
  }
};

// s2o_decode (decode.hip).  qs, oks, ovs, os: strides for (z, b, head, row); ks, vs: (z, head, row).
struct DecodeArgs {
  const void *Q, *K, *V, *oK, *oV;
  const int32_t *lens, *own_lens;
  void* O;
  float* lse;
  int Z, B, H, Hkv, G, D, T, L, Lo, f16;
  float c2;              // softmax_scale * log2(e)
  int64_t qs[4], ks[3], vs[3], oks[4], ovs[4], os[4];
  // set by the launch: states of the parts [part][row][D], {reference, sum} [part][row]; row blocks and parts of either kind
  float* part_acc;
  float2* part_ml;
  int blocks_s, splits_s, blocks_o, splits_o, direct;
  int64_t rows;                  // Z * B * H * T
  int units_s, units_o, ids_s;   // (cache, KV head, part) and (.., sequence, part); block ids of shared row blocks
  Divisor by_blocks_s, by_blocks_o, by_splits_s, by_splits_o, by_Z, by_B, by_H, by_Hkv, by_G, by_BG, by_T;   // (by_blocks: eight units' blocks)
};
size_t decode_scratch_bytes(const DecodeArgs& a);
hipError_t launch_decode(DecodeArgs a, void* scratch, hipStream_t stream);

// s2o_key_weights (weights.hip)
struct WeightsArgs {
  const void *Q, *K;
  const float *lse, *prev;
  const int32_t* lens;
  float* out;
  int Z, B, H, Hkv, G, D, T, L, f16, causal;
  float c2;              // softmax_scale * log2(e), and c2 / softmax_scale in two parts: what turns an lse into the scores' unit
  float l2e_hi, l2e_lo;
  int64_t qs[4], ks[3];
  // set by the launch
  float2* stats;         // [key part][cache, KV head][row]: {reference, sum}, joined: {reference, 1 / sum}
  float* sums;           // [row part][cache, KV head][key]
  int row_blocks, key_parts, ranges, range_tiles, row_parts;
  Divisor by_Z, by_Hkv, by_G, by_BG, by_key_parts, by_row_parts;
};
size_t weights_scratch_bytes(WeightsArgs a, bool given);
hipError_t launch_weights(WeightsArgs a, void* scratch, hipStream_t stream);

// s2o_evict (evict.hip)
struct EvictArgs {
  const void *K, *V;
  const float* weights;
  const int32_t* lens;
  void *K_out, *V_out;
  float* weights_out;
  int32_t *kept, *lens_out;
  int Z, Hkv, D, L, keep, sink, recent;
  int64_t ks[3], vs[3], kos[3], vos[3];
  uint32_t* scratch;     // set by the launch
};
size_t evict_scratch_bytes(const EvictArgs& a);
hipError_t launch_evict(EvictArgs a, void* scratch, hipStream_t stream);

}  // namespace s2o
