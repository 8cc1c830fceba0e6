// Eviction from a cache by accumulated attention weight, for gfx950: of n rows the first `sink`, the last `recent` and, of those
// between, the ones of the largest weights stay (ties: the lowest index), in their order, moved together.
//
// Weights are ranked by an unsigned key that orders like the float (-0 as +0, NaN as -inf).  select_kernel finds, a
// workgroup per (cache, KV head), the key of the last row that stays and how many rows of just that key do, by four rounds
// of 8 bits; its wavefronts then count and list the rows of their own stretch of the cache.  gather_kernel copies the listed
// rows of K and V.  Bound: HBM bandwidth of the copy; the selection reads the weights from L2 after the first round.
#include "cache_tile.h"
#include "s2o_internal.h"

namespace s2o {

namespace {

using namespace cache;

constexpr int kSelectThreads = 1024, kSelectWaves = kSelectThreads / 64;

// larger key = stays longer
__device__ __forceinline__ uint32_t rank_key(float w) {
  if (w != w) w = -INFINITY;
  const uint32_t b = __float_as_uint(w + 0.0f);          // -0 + 0 = +0
  return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}

__global__ __launch_bounds__(kSelectThreads) void select_kernel(const EvictArgs a) {
  __shared__ uint32_t hist[256];
  __shared__ uint32_t found[2];                          // digit, rows above it
  __shared__ int counts[kSelectWaves][2];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t head = blockIdx.x;
  const int z = (int)(head / a.Hkv);
  const int n = filled(a.lens, z, a.L), stay = min(n, a.keep);
  const float* w = a.weights + head * a.L;
  if (a.lens_out && head % a.Hkv == 0 && tid == 0) a.lens_out[z] = stay;

  // rows lo .. hi - 1 compete for `want` places
  const int lo = min(a.sink, n), hi = max(lo, n - a.recent);
  const int want = stay - (n - (hi - lo));
  uint32_t key = 0;                                      // the last one's, found from the top digit down
  int above = 0;                                         // rows with a larger key
  if (want > 0 && want < hi - lo) {
    for (int shift = 24; shift >= 0; shift -= 8) {
      if (tid < 256) hist[tid] = 0;
      __syncthreads();
      for (int i = lo + tid; i < hi; i += kSelectThreads) {
        const uint32_t k = rank_key(w[i]);
        if (shift == 24 || (k >> (shift + 8)) == (key >> (shift + 8))) atomicAdd(&hist[(k >> shift) & 255], 1u);
      }
      __syncthreads();
      if (wave == 0) {                                   // suffix sums of 256 counts, 4 a lane, the largest digit first
        uint32_t c[4], own = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) { c[j] = hist[255 - (4 * lane + j)]; own += c[j]; }
        uint32_t sum = own;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
          const uint32_t o = __shfl_up(sum, d);
          if (lane >= d) sum += o;
        }
        uint32_t before = above + sum - own;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if (before < (uint32_t)want && before + c[j] >= (uint32_t)want) {
            found[0] = 255 - (4 * lane + j);
            found[1] = before;
          }
          before += c[j];
        }
      }
      __syncthreads();
      key |= found[0] << shift;
      above = (int)found[1];
      __syncthreads();
    }
  }
  const bool all = want >= hi - lo;                      // every competing row stays
  const int ties = want - above;                         // rows of exactly `key` that stay

  // every wavefront lists its own stretch; what stands in front of it is counted first
  const int per = ((n + kSelectWaves - 1) / kSelectWaves + 63) / 64 * 64;
  const int from = min(wave * per, n), to = min(from + per, n);
  auto classify = [&](int i, bool& sure, bool& tie) {
    sure = tie = false;
    if (i >= to) return;
    if (i < lo || i >= hi || all) { sure = true; return; }
    if (want <= 0) return;
    const uint32_t k = rank_key(w[i]);
    sure = k > key;
    tie = k == key;
  };
  int sures = 0, tied = 0;
  for (int i = from + lane; i - lane < to; i += 64) {
    bool sure, tie;
    classify(i, sure, tie);
    sures += __popcll(__ballot(sure));
    tied += __popcll(__ballot(tie));
  }
  if (lane == 0) { counts[wave][0] = sures; counts[wave][1] = tied; }
  __syncthreads();
  int sure_before = 0, tie_before = 0;
  for (int v = 0; v < wave; ++v) { sure_before += counts[v][0]; tie_before += counts[v][1]; }
  const uint64_t below = (1ull << lane) - 1;
  for (int i = from + lane; i - lane < to; i += 64) {
    bool sure, tie;
    classify(i, sure, tie);
    const uint64_t sm = __ballot(sure), tm = __ballot(tie);
    const int my_tie = tie_before + __popcll(tm & below), my_sure = sure_before + __popcll(sm & below);
    if (sure || (tie && my_tie < ties)) {
      const int64_t at = head * a.keep + my_sure + min(my_tie, ties);
      a.kept[at] = i;
      if (a.weights_out) a.weights_out[at] = w[i];
    }
    sure_before += __popcll(sm);
    tie_before += __popcll(tm);
  }
}

// Rows of 2 * D bytes, D / 8 lanes a row; blockIdx.y: K or V.
__global__ __launch_bounds__(256) void gather_kernel(const EvictArgs a, int lanes, int rows_block, int chunks) {
  const int64_t head = blockIdx.x / chunks;
  const int z = (int)(head / a.Hkv), hk = (int)(head % a.Hkv);
  const int stay = min(filled(a.lens, z, a.L), a.keep);
  const int row0 = (int)(blockIdx.x % chunks) * rows_block;
  const int end = min(row0 + rows_block, stay);
  const uint16_t* src = static_cast<const uint16_t*>(blockIdx.y ? a.V : a.K);
  uint16_t* dst = static_cast<uint16_t*>(blockIdx.y ? a.V_out : a.K_out);
  if (!src) return;
  const int64_t* ss = blockIdx.y ? a.vs : a.ks;
  const int64_t* ds = blockIdx.y ? a.vos : a.kos;
  src += z * ss[0] + hk * ss[1] + 8 * (threadIdx.x % lanes);
  dst += z * ds[0] + hk * ds[1] + 8 * (threadIdx.x % lanes);
#pragma unroll 4
  for (int r = row0 + threadIdx.x / lanes; r < end; r += 256 / lanes) {
    const int from = a.kept[head * a.keep + r];
    *reinterpret_cast<u32x4*>(dst + r * ds[2]) = *reinterpret_cast<const u32x4*>(src + from * ss[2]);
  }
}

}  // namespace

size_t evict_scratch_bytes(const EvictArgs&) { return 0; }

hipError_t launch_evict(const EvictArgs& a, void*, hipStream_t stream) {
  const int64_t heads = (int64_t)a.Z * a.Hkv;
  if (heads > 0x7fffffff) return hipErrorInvalidValue;
  hipLaunchKernelGGL(select_kernel, dim3((unsigned)heads), dim3(kSelectThreads), 0, stream, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || (!a.K && !a.V)) return e;
  const int lanes = a.D / 8, rows_block = 4 * (256 / lanes), chunks = (a.keep + rows_block - 1) / rows_block;
  if (heads * chunks > 0x7fffffff) return hipErrorInvalidValue;
  hipLaunchKernelGGL(gather_kernel, dim3((unsigned)(heads * chunks), 2), dim3(256), 0, stream, a, lanes, rows_block, chunks);
  return hipGetLastError();
}

}  // namespace s2o
