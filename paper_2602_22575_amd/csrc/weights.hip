// What every key of a cache was worth to a set of queries, for gfx950: softmax weights added up over the query rows.
//
//   w[j] = prev[j] + sum_r exp(x_rj - lse_r),   x_rj = scale <q_r, k_j>,   r over the B*T*G rows of a (cache, KV head) that see j
//
// With the rows' lse given (of a softmax over more than these keys) one pass over the scores is enough; without it the
// rows' softmax over the keys they see comes first, in a pass of its own.  Both passes form scores with MFMAs and keep one side of the product in
// registers while 64-row tiles of the other stream through LDS, shared by the workgroup's four wavefronts:
//   stats_kernel   64 query rows a wavefront as columns, key tiles stream: a lane keeps its own maximum and sum of its columns
//                  over the keys it meets, lanes are joined once at the end;
//   sum_kernel     64 keys a wavefront as columns, query tiles stream: a lane keeps one sum per key and nothing is
//                  exchanged until the end.  A key's sum is made in one order by one workgroup: no atomics, the same bits every time.
// Rows are counted r = (t * B + b) * G + g, so that what a key is seen by is one range of rows.
//
// Statistics are kept as a base-2 reference m and 1/l instead of one lse: rounding m + log2 l would cost the weights
// 2^-20 of their value.  An lse that is given is turned into the same pair, its base-2 form rounded and the rest in the factor.
#include "cache_tile.h"
#include "s2o_internal.h"

namespace s2o {

namespace {

using namespace cache;

constexpr int kWaves = 4, kThreads = 64 * kWaves, kTileRows = 64;
constexpr int kCols = 64;                          // columns of a wavefront: four blocks of 16
constexpr int kColsWg = kCols * kWaves;

struct RowOf {
  int t, b, g;
  __device__ __forceinline__ void set(const WeightsArgs& a, int r) {
    const int per_t = a.B * a.G, rest = r % per_t;
    t = r / per_t;
    b = rest / a.G;
    g = rest % a.G;
  }
};

// A tile of 64 rows on its way to LDS: D/32 pieces of 16 bytes a thread, row (D/8 lanes each) tid / (D/8) + i * rows a pass.
template <int D>
struct Staged {
  static constexpr int kLanes = D / 8, kPerPass = kThreads / kLanes, kPasses = kTileRows / kPerPass;
  u32x4 x[kPasses];
  __device__ __forceinline__ void store(unsigned char* tile, int tid) const {
#pragma unroll
    for (int i = 0; i < kPasses; ++i) *reinterpret_cast<u32x4*>(tile + at<D>(kPerPass * i + tid / kLanes, tid % kLanes)) = x[i];
  }
};

// ---- rows' softmax statistics over the keys they see
template <class E, int D>
__global__ __launch_bounds__(kThreads, 2) void stats_kernel(const WeightsArgs a) {
  typedef typename Vec<E>::x8 x8;
  constexpr int kTile = kTileRows * D * 2;
  __shared__ __attribute__((aligned(256))) unsigned char smem[2 * kTile];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int mm = lane & 15, g = lane >> 4;
  int id = blockIdx.x;
  const int rb = id % a.row_blocks;
  id /= a.row_blocks;
  const int hk = id % a.Hkv;
  id /= a.Hkv;
  const int z = id % a.Z, part = id / a.Z;
  const int R = a.B * a.T * a.G, len = filled(a.lens, z, a.L);
  const E* Q = static_cast<const E*>(a.Q) + z * a.qs[0];
  const E* K = static_cast<const E*>(a.K) + z * a.ks[0] + hk * a.ks[1];

  x8 q[4][D / 32];
  int lim[4];
  float m[4], l[4];
#pragma unroll
  for (int cb = 0; cb < 4; ++cb) {
    RowOf row;
    row.set(a, min(rb * kColsWg + wave * kCols + 16 * cb + mm, R - 1));
    const E* p = Q + row.b * a.qs[1] + (hk * a.G + row.g) * a.qs[2] + row.t * a.qs[3];
#pragma unroll
    for (int kk = 0; kk < D / 32; ++kk) q[cb][kk] = *reinterpret_cast<const x8*>(p + 32 * kk + 8 * g);
    lim[cb] = a.causal ? min(max(len - a.T + row.t + 1, 0), len) : len;
    m[cb] = -INFINITY;
    l[cb] = 0.f;
  }
  // keys that the workgroup's last row sees
  RowOf last;
  last.set(a, min((rb + 1) * kColsWg, R) - 1);
  const int seen = a.causal ? min(max(len - a.T + last.t + 1, 0), len) : len;
  const int tiles = (seen + kTileRows - 1) / kTileRows;
  const int from = (int)((int64_t)tiles * part / a.key_parts), to = (int)((int64_t)tiles * (part + 1) / a.key_parts);

  Staged<D> st;
  const uint32_t krow = (uint32_t)(a.ks[2] * 2);
  auto load = [&](int t) {
    const char* base = reinterpret_cast<const char*>(K + (int64_t)t * kTileRows * a.ks[2]);
    const int most = len - 1 - t * kTileRows;
#pragma unroll
    for (int i = 0; i < st.kPasses; ++i) {
      const uint32_t off = (uint32_t)min(st.kPerPass * i + tid / st.kLanes, most) * krow + 16 * (tid % st.kLanes);
      st.x[i] = *reinterpret_cast<const u32x4*>(base + off);
    }
  };
  if (from < to) load(from);
  for (int t = from; t < to; ++t) {
    unsigned char* tile = smem + ((t - from) & 1) * kTile;
    st.store(tile, tid);
    __syncthreads();
    if (t + 1 < to) load(t + 1);
    f32x4 s[4][4];                                 // [16-key block][column block]
#pragma unroll
    for (int kb = 0; kb < 4; ++kb) {
      x8 k[D / 32];
#pragma unroll
      for (int kk = 0; kk < D / 32; ++kk) k[kk] = *reinterpret_cast<const x8*>(tile + at<D>(16 * kb + mm, 4 * kk + g));
#pragma unroll
      for (int cb = 0; cb < 4; ++cb) {
        s[kb][cb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kk = 0; kk < D / 32; ++kk) s[kb][cb] = mfma(k[kk], q[cb][kk], s[kb][cb]);
      }
    }
    const int key0 = t * kTileRows;
    bool hidden = false;
#pragma unroll
    for (int cb = 0; cb < 4; ++cb) hidden |= lim[cb] < key0 + kTileRows;
    if (__builtin_amdgcn_ballot_w64(hidden) != 0) {
#pragma unroll
      for (int kb = 0; kb < 4; ++kb)
#pragma unroll
        for (int cb = 0; cb < 4; ++cb)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (key0 + 16 * kb + 4 * g + i >= lim[cb]) s[kb][cb][i] = -INFINITY;
    }
#pragma unroll
    for (int cb = 0; cb < 4; ++cb) {
      float top = -INFINITY;
#pragma unroll
      for (int kb = 0; kb < 4; ++kb)
#pragma unroll
        for (int i = 0; i < 4; ++i) top = fmaxf(top, s[kb][cb][i]);
      const float m_new = fmaxf(m[cb], top * a.c2), ref = m_new == -INFINITY ? 0.f : m_new;
      float sum = 0.f;
#pragma unroll
      for (int kb = 0; kb < 4; ++kb)
#pragma unroll
        for (int i = 0; i < 4; ++i) sum += exp2_(fmaf(s[kb][cb][i], a.c2, -ref));
      l[cb] = fmaf(l[cb], exp2_(m[cb] - ref), sum);
      m[cb] = m_new;
    }
  }
  // join the four lanes of a column
  const int64_t rows = (int64_t)a.Z * a.Hkv * R;
#pragma unroll
  for (int cb = 0; cb < 4; ++cb) {
    const float top = column_max(m[cb]), ref = top == -INFINITY ? 0.f : top;
    const float sum = column_sum(l[cb] * exp2_(m[cb] - ref));
    const int r = rb * kColsWg + wave * kCols + 16 * cb + mm;
    if (g == 0 && r < R) {
      const int64_t i = ((int64_t)z * a.Hkv + hk) * R + r;
      // (nothing seen: a reference and factor that make every weight zero)
      a.stats[part * rows + i] = a.key_parts > 1 ? float2{top, sum} : sum == 0.f ? float2{INFINITY, 0.f} : float2{ref, 1.0f / sum};
    }
  }
}

__global__ __launch_bounds__(256) void stats_join_kernel(float2* stats, int64_t rows, int parts) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= rows) return;
  float top = -INFINITY, sum = 0.f;
  for (int p = 0; p < parts; ++p) top = fmaxf(top, stats[p * rows + i].x);
  const float ref = top == -INFINITY ? 0.f : top;
  for (int p = 0; p < parts; ++p) {
    const float2 s = stats[p * rows + i];
    sum = fmaf(exp2_(s.x - ref), s.y, sum);
  }
  stats[i] = sum == 0.f ? float2{INFINITY, 0.f} : float2{ref, 1.0f / sum};
}

// ---- the weights
template <class E, int D, bool kGiven>
__global__ __launch_bounds__(kThreads, 2) void sum_kernel(const WeightsArgs a) {
  typedef typename Vec<E>::x8 x8;
  constexpr int kTile = kTileRows * D * 2;
  __shared__ __attribute__((aligned(256))) unsigned char smem[2 * kTile];
  __shared__ __attribute__((aligned(16))) float ref_s[2][kTileRows], inv_s[2][kTileRows];
  __shared__ __attribute__((aligned(16))) int lim_s[2][kTileRows];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int mm = lane & 15, g = lane >> 4;
  int id = blockIdx.x;
  const int hk = id % a.Hkv;
  id /= a.Hkv;
  const int z = id % a.Z;
  id /= a.Z;
  const int part = id % a.row_parts, kblock = id / a.row_parts;
  const int R = a.B * a.T * a.G, len = filled(a.lens, z, a.L);
  const int key0 = kblock * kColsWg;
  if (key0 >= len) return;                         // (uniform: rows behind the cache's end stay as they are)
  const E* Q = static_cast<const E*>(a.Q) + z * a.qs[0];
  const E* K = static_cast<const E*>(a.K) + z * a.ks[0] + hk * a.ks[1];
  const int64_t head = (int64_t)z * a.Hkv + hk;

  x8 k[4][D / 32];
  float acc[4] = {0.f, 0.f, 0.f, 0.f};
  const int wkey0 = key0 + wave * kCols;
#pragma unroll
  for (int cb = 0; cb < 4; ++cb) {
    const E* p = K + (int64_t)min(wkey0 + 16 * cb + mm, len - 1) * a.ks[2];
#pragma unroll
    for (int kk = 0; kk < D / 32; ++kk) k[cb][kk] = *reinterpret_cast<const x8*>(p + 32 * kk + 8 * g);
  }
  // rows that see the first of the keys, and of these the part's share
  const int first_t = a.causal ? max(key0 - (len - a.T), 0) : 0;
  const int r_first = min((int64_t)first_t * a.B * a.G, (int64_t)R) & ~(kTileRows - 1);
  const int tiles = (R - r_first + kTileRows - 1) / kTileRows;
  const int from = (int)((int64_t)tiles * part / a.row_parts), to = (int)((int64_t)tiles * (part + 1) / a.row_parts);

  Staged<D> st;
  float my_ref = 0.f, my_inv = 0.f;
  int my_lim = 0;
  auto load = [&](int t) {
    const int r0 = r_first + t * kTileRows;
#pragma unroll
    for (int i = 0; i < st.kPasses; ++i) {
      RowOf row;
      row.set(a, min(r0 + st.kPerPass * i + tid / st.kLanes, R - 1));
      const E* p = Q + row.b * a.qs[1] + (hk * a.G + row.g) * a.qs[2] + row.t * a.qs[3];
      st.x[i] = *reinterpret_cast<const u32x4*>(p + 8 * (tid % st.kLanes));
    }
    if (tid < kTileRows) {
      const int r = r0 + tid;
      my_lim = 0; my_ref = INFINITY; my_inv = 0.f;
      if (r < R) {
        RowOf row;
        row.set(a, r);
        my_lim = a.causal ? min(max(len - a.T + row.t + 1, 0), len) : len;
        if (kGiven) {
          const float x = a.lse[(((int64_t)z * a.B + row.b) * a.H + hk * a.G + row.g) * a.T + row.t];
          if (isinf(x)) {                          // -inf: a row that saw nothing; +inf: exp(x - inf)
            my_lim = 0;
          } else {
            my_ref = x * a.l2e_hi;
            my_inv = exp2_(-(fmaf(x, a.l2e_hi, -my_ref) + x * a.l2e_lo));
          }
        } else {
          const float2 s = a.stats[head * R + r];
          my_ref = s.x;
          my_inv = s.y;
        }
      }
    }
  };
  if (from < to) load(from);
  for (int t = from; t < to; ++t) {
    const int buf = (t - from) & 1, r0 = r_first + t * kTileRows;
    unsigned char* tile = smem + buf * kTile;
    st.store(tile, tid);
    if (tid < kTileRows) {
      ref_s[buf][tid] = my_ref;
      inv_s[buf][tid] = my_inv;
      lim_s[buf][tid] = my_lim;
    }
    __syncthreads();
    if (t + 1 < to) load(t + 1);
    const int blocks = min(R - r0 + 15, kTileRows) >> 4;
    // some row of the tile does not see all of the wavefront's keys, or is none
    const bool edge = __builtin_amdgcn_ballot_w64(lim_s[buf][lane] < wkey0 + kCols) != 0;
    for (int qb = 0; qb < blocks; ++qb) {
      x8 q[D / 32];
#pragma unroll
      for (int kk = 0; kk < D / 32; ++kk) q[kk] = *reinterpret_cast<const x8*>(tile + at<D>(16 * qb + mm, 4 * kk + g));
      const f32x4 ref = *reinterpret_cast<const f32x4*>(&ref_s[buf][16 * qb + 4 * g]);
      const f32x4 inv = *reinterpret_cast<const f32x4*>(&inv_s[buf][16 * qb + 4 * g]);
      f32x4 s[4];
#pragma unroll
      for (int cb = 0; cb < 4; ++cb) {
        s[cb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kk = 0; kk < D / 32; ++kk) s[cb] = mfma(q[kk], k[cb][kk], s[cb]);
      }
      if (edge) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int lim = lim_s[buf][16 * qb + 4 * g + i];
#pragma unroll
          for (int cb = 0; cb < 4; ++cb) {
            const float p = exp2_(fmaf(s[cb][i], a.c2, -ref[i]));
            if (wkey0 + 16 * cb + mm < lim) acc[cb] = fmaf(p, inv[i], acc[cb]);
          }
        }
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int cb = 0; cb < 4; ++cb) acc[cb] = fmaf(exp2_(fmaf(s[cb][i], a.c2, -ref[i])), inv[i], acc[cb]);
      }
    }
  }
#pragma unroll
  for (int cb = 0; cb < 4; ++cb) acc[cb] = column_sum(acc[cb]);
  const float mine = g == 0 ? acc[0] : g == 1 ? acc[1] : g == 2 ? acc[2] : acc[3];
  const int key = wkey0 + lane;
  if (key >= len) return;
  if (a.row_parts > 1) a.sums[((int64_t)part * a.Z * a.Hkv + head) * a.L + key] = mine;
  else a.out[head * a.L + key] = a.prev ? a.prev[head * a.L + key] + mine : mine;
}

__global__ __launch_bounds__(256) void sum_join_kernel(const WeightsArgs a) {
  const int64_t heads = (int64_t)a.Z * a.Hkv;
  const int key = blockIdx.x * 256 + threadIdx.x;
  for (int64_t head = blockIdx.y; head < heads; head += gridDim.y) {
    if (key >= filled(a.lens, (int)(head / a.Hkv), a.L)) continue;
    float w = 0.f;
    for (int p = 0; p < a.row_parts; ++p) w += a.sums[(p * heads + head) * a.L + key];
    a.out[head * a.L + key] = a.prev ? a.prev[head * a.L + key] + w : w;
  }
}

constexpr int kWorkgroups = 768;   // that the splits aim at: three on each of 256 CUs

void shape_of(WeightsArgs& a, bool given) {
  const int64_t R = (int64_t)a.B * a.T * a.G, heads = (int64_t)a.Z * a.Hkv;
  auto parts = [](int64_t units, int64_t tiles) {
    const int64_t want = (kWorkgroups + units - 1) / units;
    return (int)(want < tiles ? want : tiles);
  };
  a.row_blocks = (int)((R + kColsWg - 1) / kColsWg);
  a.key_blocks = (a.L + kColsWg - 1) / kColsWg;
  // a part has four tiles at least
  a.key_parts = given ? 0 : parts(heads * a.row_blocks, (a.L + 4 * kTileRows - 1) / (4 * kTileRows));
  a.row_parts = parts(heads * a.key_blocks, (R + 4 * kTileRows - 1) / (4 * kTileRows));
}

size_t stats_bytes(const WeightsArgs& a) {
  return ((size_t)a.key_parts * a.Z * a.Hkv * a.B * a.T * a.G * 8 + 255) / 256 * 256;
}

template <class E, int D>
hipError_t launch(const WeightsArgs& a, hipStream_t stream) {
  const int64_t heads = (int64_t)a.Z * a.Hkv, rows = heads * a.B * a.T * a.G;
  const int64_t sum_blocks = heads * a.row_parts * a.key_blocks;
  if (sum_blocks > 0x7fffffff) return hipErrorInvalidValue;
  if (a.lse) {
    hipLaunchKernelGGL((sum_kernel<E, D, true>), dim3((unsigned)sum_blocks), dim3(kThreads), 0, stream, a);
  } else {
    const int64_t blocks = heads * a.row_blocks * a.key_parts;
    if (blocks > 0x7fffffff) return hipErrorInvalidValue;
    hipLaunchKernelGGL((stats_kernel<E, D>), dim3((unsigned)blocks), dim3(kThreads), 0, stream, a);
    if (a.key_parts > 1)
      hipLaunchKernelGGL(stats_join_kernel, dim3((unsigned)((rows + 255) / 256)), dim3(256), 0, stream, a.stats, rows, a.key_parts);
    hipLaunchKernelGGL((sum_kernel<E, D, false>), dim3((unsigned)sum_blocks), dim3(kThreads), 0, stream, a);
  }
  if (a.row_parts > 1)
    hipLaunchKernelGGL(sum_join_kernel, dim3((unsigned)((a.L + 255) / 256), (unsigned)(heads < 65535 ? heads : 65535)), dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

size_t weights_scratch_bytes(WeightsArgs a, bool given) {
  shape_of(a, given);
  const size_t sums = a.row_parts > 1 ? (size_t)a.row_parts * a.Z * a.Hkv * a.L * 4 : 0;
  return (given ? 0 : stats_bytes(a)) + sums;
}

hipError_t launch_weights(WeightsArgs a, void* scratch, hipStream_t stream) {
  shape_of(a, a.lse != nullptr);
  a.stats = static_cast<float2*>(scratch);
  a.sums = reinterpret_cast<float*>(static_cast<char*>(scratch) + (a.lse ? 0 : stats_bytes(a)));
  if (a.f16) return a.D == 128 ? launch<_Float16, 128>(a, stream) : launch<_Float16, 64>(a, stream);
  return a.D == 128 ? launch<__bf16, 128>(a, stream) : launch<__bf16, 64>(a, stream);
}

}  // namespace s2o
