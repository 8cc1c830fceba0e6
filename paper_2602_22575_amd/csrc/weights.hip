// What every key of a cache was worth to a set of queries, for gfx950: softmax weights added up over the query rows.
//
//   w[j] = prev[j] + sum_r exp(x_rj - lse_r),   x_rj = scale <q_r, k_j>,   r over the B*T*G rows of a (cache, KV head) that see j
//
// With the rows' lse given (of a softmax over more than these keys) one pass over the scores is enough; without it the
// rows' softmax over the keys they see comes first, in a pass of its own.  Both passes form scores with MFMAs, hold 64 query rows a wavefront in
// registers and stream tiles of 64 keys through LDS, shared by the workgroup's four wavefronts:
//   stats_kernel   query rows are the columns: a lane keeps its own maximum and sum of its rows over the keys it meets, lanes are
//                  joined once at the end;
//   sum_kernel     keys are the columns: a lane adds up a key's terms over the rows in its registers.  Every sum is made in one order: no
//                  atomics, the same bits every time.
// Rows are counted r = (t * B + b) * G + g, so that what a key is seen by is one range of rows.
//
// Bound: a score costs 2 D FLOP on the matrix cores and an exponential, a multiply-add and an addition on the vector units, which take about as
// long (17.2 and 16.6 clocks for 64 lanes' worth of one product) and overlap by half (25.5 together).  64 queries of 32 heads on 128K keys of 8
// (69 GFLOP a pass): statistics 72 to 81 us, sums 80 to 92, by the clock that the power limit leaves: 0.75 to 0.96 PFLOP/s.  All 8192 queries of a
// prompt (275 GFLOP a pass): 260 and 340.
//
// Statistics are kept as a base-2 reference m and 1/l instead of one lse: rounding m + log2 l would cost the weights
// 2^-20 of their value.  An lse that is given is turned into the same pair, its base-2 form rounded and the rest in the factor.
#include "cache_tile.h"
#include "s2o_internal.h"

namespace s2o {

namespace {

using namespace cache;

constexpr int kWaves = 4, kThreads = 64 * kWaves, kTileRows = 64;
// CB: blocks of 16 query rows of a wavefront, 4 where there are more than 128 rows, so that tiles are read as rarely as possible; with
// fewer rows 2 or 1, so that all four wavefronts have some (32K keys of 8 heads, lse given: 128 rows 18 us, with 1 and 4 blocks 26 and 22;
// 48 rows 15 us, with 2 blocks 18).
template <int CB>
constexpr int kRowsWg = 16 * CB * kWaves;
// Parts of a row's statistics that its readers join themselves: a launch less (4 queries of 32 heads on 2000 keys 11 us, else 15).
constexpr int kFewParts = 8;
constexpr int kRange = 32;                         // tiles of keys of a workgroup of sum_kernel at most

struct RowOf {
  int t, b, g;
  __device__ __forceinline__ void set(const WeightsArgs& a, int r) {
    int rest;
    t = a.by_BG.by(r, rest);
    b = a.by_G.by(rest, g);
  }
};

// Of `all` things in parts (by_parts), those of one part: as many for each, or one more in the first parts.
__device__ __forceinline__ void share(const Divisor& by_parts, int all, int part, int& from, int& to) {
  int more;
  const int each = by_parts.by(all, more);
  from = part * each + min(part, more);
  to = from + each + (part < more);
}

// Keys that query token t sees.
__device__ __forceinline__ int row_limit(const WeightsArgs& a, int len, int t) { return a.causal ? min(max(len - a.T + t + 1, 0), len) : len; }

// A tile of 64 keys in this order of instructions: the products of a block of 16 keys one by one, behind each its share of the values (scores)
// of the block before; keys are read a block ahead.  Every product, and what stands behind it, is a scheduling region of its
// own.  (Left to itself the compiler waits for one block's results and then works on them.)  product(k, kk, cb, s): s plus the product of 32
// dims; value(kb, x, s): works on score 4 * column block + i of 4 * CB in a lane.
template <class E, int D, int CB, class P, class V>
__device__ __forceinline__ void tile_in_order(const unsigned char* tile, int mm, int g, P product, V value) {
  typedef typename Vec<E>::x8 x8;
  constexpr int kReads = D / 32, kEach = 4 / kReads;
  x8 k[2][kReads];
  f32x4 s[2][CB];
  auto read = [&](int kb, int kk) { k[kb & 1][kk] = *reinterpret_cast<const x8*>(tile + 16 * kb * 2 * D + (at<D>(mm, g) ^ (kk << 6))); };
#pragma unroll
  for (int kk = 0; kk < kReads; ++kk) read(0, kk);
#pragma unroll
  for (int kb = 0; kb < 4; ++kb)
#pragma unroll
    for (int kk = 0; kk < kReads; ++kk) {
      if (kb < 3) read(kb + 1, kk);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int cb = 0; cb < CB; ++cb) {
        f32x4& x = s[kb & 1][cb];
        x = product(k[kb & 1][kk], kk, cb, kk == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : x);
        if (kb > 0) {
#pragma unroll
          for (int e = 0; e < kEach; ++e) value(kb - 1, (kk * CB + cb) * kEach + e, s[(kb - 1) & 1]);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
#pragma unroll
  for (int x = 0; x < 4 * CB; ++x) value(3, x, s[1]);
}

// Streams tiles from .. to - 1 of 64 keys through three LDS buffers, two tiles ahead of the one that is worked on: two workgroups a CU
// then have 64 KB on their way (with one tile ahead the kernels waited for memory).  All threads of the workgroup; fast(t, tile) or, where it returns false, any(t, tile) works on tile t; the buffers are separate arrays, so
// that the compiler sees that reads of one need not wait for the loads that fill another.
template <class E, int D, class F, class G>
__device__ __forceinline__ void stream_keys(const E* K, int64_t stride, int len, int from, int to, unsigned char* b0, unsigned char* b1,
                                            unsigned char* b2, int tid, F fast, G any) {
  constexpr int kLanes = D / 8, kRowsPerLoad = 64 / kLanes, kLoads = 16 / kRowsPerLoad;   // a wavefront loads 16 rows
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lr = lane / kLanes;
  // LDS takes a load's lanes in order: each fetches the chunk that belongs at its slot
  const uint32_t chunk = 16 * ((lane % kLanes) ^ swz<D>(lr)), row = (uint32_t)(stride * 2), off = (uint32_t)lr * row;
  auto issue = [&](int t, unsigned char* tile) {
    const auto keys = rows_buffer(K, stride * 2, t * kTileRows, len, kTileRows, 2 * D);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int r = 16 * wave + kRowsPerLoad * i;
      buffer_load_to_lds(keys, off + r * row + (chunk ^ (swz<D>(kRowsPerLoad * i) << 4)), tile + r * 2 * D);
    }
  };
  if (from >= to) return;
  issue(from, b0);
  if (from + 1 < to) issue(from + 1, b1);
  auto step = [&](int t, unsigned char* tile, unsigned char* ahead) {
    // what this wavefront fetched of tile t has landed (loads complete in order), and what it read of tile t - 1 is in its registers
    asm volatile("" ::: "memory");
    if (t + 1 < to) __builtin_amdgcn_s_waitcnt(0x0070 | kLoads);   // vmcnt(kLoads) lgkmcnt(0)
    else __builtin_amdgcn_s_waitcnt(0x0070);
    asm volatile("s_barrier" ::: "memory");
    if (t + 2 < to) issue(t + 2, ahead);
    if (!fast(t, tile)) any(t, tile);
  };
  for (int t = from;;) {
    step(t, b0, b2);
    if (++t >= to) break;
    step(t, b1, b0);
    if (++t >= to) break;
    step(t, b2, b1);
    if (++t >= to) break;
  }
}

// ---- rows' softmax statistics over the keys they see
//
// A column's reference is the largest of the first scores that the lane meets: never above the true maximum, so that nothing
// is lost below it, and 32-bit sums have room for 2^90 times as much above it.  So only a tile with hidden keys, the first one, and one after
// which a sum has outgrown that look for the maximum; the others are products, exponentials and additions.
constexpr float kRoomAbove = 0x1p90f;

template <class E, int D, int CB>
struct Stats {
  typedef typename Vec<E>::x8 x8;
  x8 q[CB][D / 32];
  int lim[CB];
  float m[CB], l[CB];              // reference (base 2), the lane's part of the sum

  __device__ __forceinline__ void scores(const unsigned char* tile, int kb, f32x4 (&s)[CB], int mm, int g) const {
    x8 k[D / 32];
#pragma unroll
    for (int kk = 0; kk < D / 32; ++kk) k[kk] = *reinterpret_cast<const x8*>(tile + 16 * kb * 2 * D + (at<D>(mm, g) ^ (kk << 6)));
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) s[cb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int kk = 0; kk < D / 32; ++kk)
#pragma unroll
      for (int cb = 0; cb < CB; ++cb) s[cb] = mfma(k[kk], q[cb][kk], s[cb]);
  }
  // All 64 keys seen, against the references as they are.
  __device__ __forceinline__ bool tile_fast(const unsigned char* tile, float c2, int mm, int g) {
    float sum[CB] = {}, last = 0.f;                // a numerator is added behind the next one's exponential, which it would wait for
    tile_in_order<E, D, CB>(
        tile, mm, g, [&](const x8& k, int kk, int cb, const f32x4& s) { return mfma(k, q[cb][kk], s); },
        [&](int, int x, const f32x4 (&s)[CB]) {
          const float p = exp2_(fmaf(s[x >> 2][x & 3], c2, -m[x >> 2]));
          sum[(x + 4 * CB - 1) / 4 % CB] += last;  // (of the value before this one)
          last = p;
        });
    sum[CB - 1] += last;
    bool fits = true;
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) fits &= l[cb] + sum[cb] <= kRoomAbove;    // (false for NaN)
    if (__builtin_amdgcn_ballot_w64(!fits) != 0) return false;
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) l[cb] += sum[cb];
    return true;
  }
  __device__ __forceinline__ void tile_any(const unsigned char* tile, int key0, float c2, int mm, int g) {
#pragma unroll 1
    for (int kb = 0; kb < 4; ++kb) {
      f32x4 s[CB];
      scores(tile, kb, s, mm, g);
#pragma unroll
      for (int cb = 0; cb < CB; ++cb) {
        float top = -INFINITY;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (key0 + 16 * kb + 4 * g + i >= lim[cb]) s[cb][i] = -INFINITY;
          top = fmaxf(top, s[cb][i]);
        }
        const float m_new = fmaxf(m[cb], top * c2), ref = m_new == -INFINITY ? 0.f : m_new;
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) sum += exp2_(fmaf(s[cb][i], c2, -ref));
        l[cb] = fmaf(l[cb], exp2_(m[cb] - ref), sum);
        m[cb] = m_new;
      }
    }
  }
};

// (Nothing seen: a reference and factor that make every weight zero.)
__device__ __forceinline__ float2 joined(float top, float sum) {
  return sum == 0.f ? float2{INFINITY, 0.f} : float2{top == -INFINITY ? 0.f : top, 1.0f / sum};
}

template <class E, int D, int CB>
__global__ __launch_bounds__(kThreads, 3) void stats_kernel(const WeightsArgs a) {
  constexpr int kTile = kTileRows * D * 2;
  __shared__ __attribute__((aligned(256))) unsigned char b0[kTile], b1[kTile], b2[kTile];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int mm = lane & 15, g = lane >> 4;
  // the row blocks that see the most keys first
  touch_args<WeightsArgs>();
  int hk, z, part;
  const int rb = a.row_blocks - 1 - a.by_key_parts.by(a.by_Z.by(a.by_Hkv.by(blockIdx.x, hk), z), part);
  const int R = a.B * a.T * a.G, len = filled(a.lens, z, a.L);
  const E* Q = static_cast<const E*>(a.Q) + z * a.qs[0];
  const E* K = static_cast<const E*>(a.K) + z * a.ks[0] + hk * a.ks[1];

  Stats<E, D, CB> w;
#pragma unroll
  for (int cb = 0; cb < CB; ++cb) {
    RowOf row;
    row.set(a, min(rb * kRowsWg<CB> + wave * 16 * CB + 16 * cb + mm, R - 1));
    const E* p = Q + row.b * a.qs[1] + (hk * a.G + row.g) * a.qs[2] + row.t * a.qs[3];
#pragma unroll
    for (int kk = 0; kk < D / 32; ++kk) w.q[cb][kk] = *reinterpret_cast<const typename Vec<E>::x8*>(p + 32 * kk + 8 * g);
    w.lim[cb] = row_limit(a, len, row.t);
    w.m[cb] = -INFINITY;
    w.l[cb] = 0.f;
  }
  // keys that the workgroup's first and last row see
  RowOf row;
  row.set(a, rb * kRowsWg<CB>);
  const int full = row_limit(a, len, row.t) / kTileRows;
  row.set(a, min((rb + 1) * kRowsWg<CB>, R) - 1);
  const int tiles = (row_limit(a, len, row.t) + kTileRows - 1) / kTileRows;
  int from, to;
  share(a.by_key_parts, tiles, part, from, to);
  const bool active = rb * kRowsWg<CB> + wave * 16 * CB < R;     // the wavefront has rows at all

  stream_keys<E, D>(K, a.ks[2], len, from, to, b0, b1, b2, tid,
                    [&](int t, const unsigned char* tile) { return !active || (t > from && t < full && w.tile_fast(tile, a.c2, mm, g)); },
                    [&](int t, const unsigned char* tile) { w.tile_any(tile, t * kTileRows, a.c2, mm, g); });
  // join the four lanes of a column
  const int64_t rows = (int64_t)a.Z * a.Hkv * R;
#pragma unroll
  for (int cb = 0; cb < CB; ++cb) {
    const float top = column_max(w.m[cb]);
    const float sum = column_sum(w.l[cb] * exp2_(w.m[cb] - (top == -INFINITY ? 0.f : top)));
    const int r = rb * kRowsWg<CB> + wave * 16 * CB + 16 * cb + mm;
    if (g == 0 && r < R) {
      const int64_t i = ((int64_t)z * a.Hkv + hk) * R + r;
      a.stats[part * rows + i] = a.key_parts > 1 ? float2{top, sum} : joined(top, sum);
    }
  }
}

// Joins the statistics of a row's parts where they are more than kFewParts: sixteen rows a workgroup, sixteen lanes a row.
__global__ __launch_bounds__(256) void stats_join_kernel(float2* stats, int64_t rows, int parts) {
  const int64_t i = (int64_t)blockIdx.x * 16 + threadIdx.x / 16;
  const int lane = threadIdx.x % 16;
  float top = -INFINITY, sum = 0.f;
  if (i < rows) {
#pragma unroll 4
    for (int p = lane; p < parts; p += 16) {
      const float2 s = stats[p * rows + i];
      const float next = fmaxf(top, s.x), ref = next == -INFINITY ? 0.f : next;
      sum = fmaf(sum, exp2_(top - ref), s.y * exp2_(s.x - ref));
      top = next;
    }
  }
  float all = top;
#pragma unroll
  for (int d = 1; d < 16; d *= 2) all = fmaxf(all, __shfl_xor(all, d));
  const float ref = all == -INFINITY ? 0.f : all;
  sum *= exp2_(top - ref);
#pragma unroll
  for (int d = 1; d < 16; d *= 2) sum += __shfl_xor(sum, d);
  if (i < rows && lane == 0) stats[i] = joined(all, sum);
}

// ---- the weights
//
// A workgroup has a range of up to kRange tiles of keys and some of the row blocks.  Per row block its wavefronts hold 64 rows each, this time as the
// A side, so that a lane of an accumulator block is a key and its registers are rows: a key's terms are added up inside the lane.  A tile's sums of the four
// wavefronts meet in LDS and add to the range's.
template <class E, int D, int CB, bool kGiven>
__global__ __launch_bounds__(kThreads, 2) void sum_kernel(const WeightsArgs) {
  const WeightsArgs& a = kernel_args<WeightsArgs>();
  typedef typename Vec<E>::x8 x8;
  constexpr int kTile = kTileRows * D * 2;
  __shared__ __attribute__((aligned(256))) unsigned char b0[kTile], b1[kTile], b2[kTile];
  __shared__ float range_s[kRange * kTileRows], tile_s[2][kWaves][kTileRows];
  __shared__ __attribute__((aligned(16))) float ref_s[kWaves][16 * CB], inv_s[kWaves][16 * CB];
  __shared__ __attribute__((aligned(16))) int lim_s[kWaves][16 * CB];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int mm = lane & 15, g = lane >> 4;
  // the ranges and the row blocks with the most work first: the first keys, the last rows
  touch_args<WeightsArgs>();
  int hk, z, part;
  const int range = a.by_row_parts.by(a.by_Z.by(a.by_Hkv.by(blockIdx.x, hk), z), part);
  part = a.row_parts - 1 - part;
  const int R = a.B * a.T * a.G, len = filled(a.lens, z, a.L);
  const int t0 = range * a.range_tiles, t1 = min(t0 + a.range_tiles, (len + kTileRows - 1) / kTileRows);
  if (t0 >= t1) return;                            // (uniform: entries behind the cache's end stay as they are)
  const E* Q = static_cast<const E*>(a.Q) + z * a.qs[0];
  const E* K = static_cast<const E*>(a.K) + z * a.ks[0] + hk * a.ks[1];
  const int64_t head = (int64_t)z * a.Hkv + hk;
  for (int i = tid; i < (t1 - t0) * kTileRows; i += kThreads) range_s[i] = 0.f;

  // adds a tile's sums, whose barrier has passed, to the range's
  auto collect = [&](int t) {
    if (wave == (t & (kWaves - 1))) {
      float x = 0.f;
#pragma unroll
      for (int v = 0; v < kWaves; ++v) x += tile_s[t & 1][v][lane];
      range_s[(t - t0) * kTileRows + lane] += x;
    }
  };
  int rb0, rb1;
  share(a.by_row_parts, a.row_blocks, part, rb0, rb1);
  for (int rb = rb0; rb < rb1; ++rb) {
    const WeightsArgs& a = kernel_args<WeightsArgs>();
    RowOf row;
    row.set(a, min((rb + 1) * kRowsWg<CB>, R) - 1);
    const int end = min(t1, (row_limit(a, len, row.t) + kTileRows - 1) / kTileRows);   // tiles that the block's last row sees
    if (end <= t0) continue;
    // this wavefront's rows: operands, and what is known of a row at its lane
    const int r0 = rb * kRowsWg<CB> + wave * 16 * CB;
    const bool active = r0 < R;
    x8 q[CB][D / 32];
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
      row.set(a, min(r0 + 16 * cb + mm, R - 1));
      const E* p = Q + row.b * a.qs[1] + (hk * a.G + row.g) * a.qs[2] + row.t * a.qs[3];
#pragma unroll
      for (int kk = 0; kk < D / 32; ++kk) q[cb][kk] = *reinterpret_cast<const x8*>(p + 32 * kk + 8 * g);
    }
    float my_ref = INFINITY, my_inv = 0.f;
    int my_lim = 0;                                // (of a row that is none: no key is seen)
    if (lane < 16 * CB && r0 + lane < R) {
      row.set(a, r0 + lane);
      my_lim = row_limit(a, len, row.t);
      if (kGiven) {
        const float x = a.lse[(((int64_t)z * a.B + row.b) * a.H + hk * a.G + row.g) * a.T + row.t];
        if (isinf(x)) {                            // -inf: a row that saw nothing; +inf: exp(x - inf)
          my_lim = 0;
        } else {
          my_ref = x * a.l2e_hi;
          my_inv = exp2_(-(fmaf(x, a.l2e_hi, -my_ref) + x * a.l2e_lo));
        }
      } else {
        const int64_t rows = (int64_t)a.Z * a.Hkv * R, i = head * R + r0 + lane;
        const bool one = a.key_parts == 1 || a.key_parts > kFewParts;      // what the launches before have made of them
        float2 s[kFewParts];
#pragma unroll
        for (int p = 0; p < kFewParts; ++p) s[p] = a.stats[(one ? 0 : min(p, a.key_parts - 1)) * rows + i];
        if (!one) {
          float top = -INFINITY, l = 0.f;
#pragma unroll
          for (int p = 0; p < kFewParts; ++p) top = fmaxf(top, s[p].x);
#pragma unroll
          for (int p = 0; p < kFewParts; ++p)
            if (p < a.key_parts) l = fmaf(s[p].y, exp2_(s[p].x - (top == -INFINITY ? 0.f : top)), l);
          s[0] = joined(top, l);
        }
        my_ref = s[0].x;
        my_inv = s[0].y;
      }
    }
    wave_fence();
    if (lane < 16 * CB) {
      ref_s[wave][lane] = my_ref;
      inv_s[wave][lane] = my_inv;
      lim_s[wave][lane] = my_lim;
    }
    wave_fence();
    f32x4 ref[CB], inv[CB];
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
      ref[cb] = *reinterpret_cast<const f32x4*>(&ref_s[wave][16 * cb + 4 * g]);
      inv[cb] = *reinterpret_cast<const f32x4*>(&inv_s[wave][16 * cb + 4 * g]);
    }

    auto scores = [&](const unsigned char* tile, int kb, f32x4 (&s)[CB]) {
      x8 k[D / 32];
#pragma unroll
      for (int kk = 0; kk < D / 32; ++kk) k[kk] = *reinterpret_cast<const x8*>(tile + 16 * kb * 2 * D + (at<D>(mm, g) ^ (kk << 6)));
#pragma unroll
      for (int cb = 0; cb < CB; ++cb) s[cb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int kk = 0; kk < D / 32; ++kk)
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) s[cb] = mfma(q[cb][kk], k[kk], s[cb]);
    };
    // of the keys of a tile, 16 * g + mm is the lane's
    stream_keys<E, D>(
        K, a.ks[2], len, t0, end, b0, b1, b2, tid,
        [&](int t, const unsigned char* tile) {
          if (t > t0) collect(t - 1);
          float sum[4] = {0.f, 0.f, 0.f, 0.f};
          if (active) {
            // some row does not see all of the keys, or is none
            if (__builtin_amdgcn_ballot_w64(lane < 16 * CB && my_lim < (t + 1) * kTileRows) != 0) return false;
            float last = 0.f;                      // (added behind the next one's exponential, as in Stats)
            tile_in_order<E, D, CB>(
                tile, mm, g, [&](const x8& k, int kk, int cb, const f32x4& s) { return mfma(q[cb][kk], k, s); },
                [&](int kb, int x, const f32x4 (&s)[CB]) {
                  const float p = exp2_(fmaf(s[x >> 2][x & 3], a.c2, -ref[x >> 2][x & 3]));
                  const int y = (x + 4 * CB - 1) % (4 * CB);
                  float& of = sum[x > 0 ? kb : kb > 0 ? kb - 1 : 0];
                  of = fmaf(last, inv[y >> 2][y & 3], of);
                  last = p;
                });
            sum[3] = fmaf(last, inv[CB - 1][3], sum[3]);
          }
#pragma unroll
          for (int kb = 0; kb < 4; ++kb) sum[kb] = column_sum(sum[kb]);
          tile_s[t & 1][wave][lane] = g == 0 ? sum[0] : g == 1 ? sum[1] : g == 2 ? sum[2] : sum[3];
          return true;
        },
        [&](int t, const unsigned char* tile) {
          float mine = 0.f;
#pragma unroll 1
          for (int kb = 0; kb < 4; ++kb) {
            f32x4 s[CB];
            scores(tile, kb, s);
            float sum = 0.f;
#pragma unroll
            for (int cb = 0; cb < CB; ++cb)
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const float p = exp2_(fmaf(s[cb][i], a.c2, -ref[cb][i])) * inv[cb][i];
                sum += t * kTileRows + 16 * kb + mm < lim_s[wave][16 * cb + 4 * g + i] ? p : 0.f;
              }
            sum = column_sum(sum);
            mine = g == kb ? sum : mine;
          }
          tile_s[t & 1][wave][lane] = mine;
        });
    __syncthreads();
    collect(end - 1);
    __syncthreads();                               // (tile and sums' buffers are free again)
  }
  __syncthreads();
  const WeightsArgs& e = kernel_args<WeightsArgs>();
  const int key = t0 * kTileRows;
  for (int i = tid; i < min((t1 - t0) * kTileRows, len - key); i += kThreads) {
    if (e.row_parts > 1) e.sums[((int64_t)part * e.Z * e.Hkv + head) * e.L + key + i] = range_s[i];
    else e.out[head * e.L + key + i] = e.prev ? e.prev[head * e.L + key + i] + range_s[i] : range_s[i];
  }
}

__global__ __launch_bounds__(256) void sum_join_kernel(const WeightsArgs a) {
  const int64_t heads = (int64_t)a.Z * a.Hkv;
  const int key = blockIdx.x * 256 + threadIdx.x;
  for (int64_t head = blockIdx.y; head < heads; head += gridDim.y) {
    if (key >= filled(a.lens, (int)(head / a.Hkv), a.L)) continue;
    float w = 0.f;
#pragma unroll 8
    for (int p = 0; p < a.row_parts; ++p) w += a.sums[(p * heads + head) * a.L + key];
    a.out[head * a.L + key] = a.prev ? a.prev[head * a.L + key] + w : w;
  }
}

constexpr int kStatsSlots = 3 * 256, kSumSlots = 2 * 256;   // workgroups that are in flight together

int row_blocks_wave(const WeightsArgs& a) {
  const int64_t R = (int64_t)a.B * a.T * a.G;
  return R <= 64 ? 1 : R <= 128 ? 2 : 4;
}

void shape_of(WeightsArgs& a, bool given) {
  const int64_t R = (int64_t)a.B * a.T * a.G, heads = (int64_t)a.Z * a.Hkv;
  // `slots` workgroups, as far as every part still has four tiles
  auto parts = [](int64_t units, int64_t slots, int64_t tiles) {
    const int64_t want = slots / units > 1 ? slots / units : 1, most = (tiles + 3) / 4;
    return (int)(want < most ? want : most);
  };
  const int64_t tiles = (a.L + kTileRows - 1) / kTileRows;
  const int rows_wg = 64 * row_blocks_wave(a);
  a.row_blocks = (int)((R + rows_wg - 1) / rows_wg);
  a.key_parts = given ? 0 : parts(heads * a.row_blocks, kStatsSlots, tiles);
  // one round of ranges where there is one row block, longer ranges where there are many (a prompt of 8K 580 us; with no more ranges than for
  // one block 726)
  const int64_t ranges = parts(heads * ((a.row_blocks + 3) / 4), kSumSlots, tiles);
  a.range_tiles = (int)((tiles + ranges - 1) / ranges < kRange ? (tiles + ranges - 1) / ranges : kRange);
  a.ranges = (int)((tiles + a.range_tiles - 1) / a.range_tiles);
  // several rounds where there are row blocks enough, since some are shorter than others (the same prompt in one round 760 us)
  a.row_parts = parts(heads * a.ranges, 4 * kSumSlots, 4 * a.row_blocks);
}

size_t stats_bytes(const WeightsArgs& a) {
  return ((size_t)a.key_parts * a.Z * a.Hkv * a.B * a.T * a.G * 8 + 255) / 256 * 256;
}

template <class E, int D, int CB>
hipError_t launch(WeightsArgs a, hipStream_t stream) {
  a.by_Z = Divisor(a.Z); a.by_Hkv = Divisor(a.Hkv); a.by_G = Divisor(a.G); a.by_BG = Divisor(a.B * a.G);
  a.by_key_parts = Divisor(a.key_parts); a.by_row_parts = Divisor(a.row_parts);
  const int64_t heads = (int64_t)a.Z * a.Hkv, rows = heads * a.B * a.T * a.G;
  const int64_t sum_blocks = heads * a.row_parts * a.ranges, blocks = heads * a.row_blocks * a.key_parts, joins = (rows + 15) / 16;
  if (!fits_launch(sum_blocks, kThreads)) return hipErrorNotSupported;
  if (!a.lse && (!fits_launch(blocks, kThreads) || (a.key_parts > kFewParts && !fits_launch(joins, 256)))) return hipErrorNotSupported;
  if (a.lse) {
    hipLaunchKernelGGL((sum_kernel<E, D, CB, true>), dim3((unsigned)sum_blocks), dim3(kThreads), 0, stream, a);
  } else {
    hipLaunchKernelGGL((stats_kernel<E, D, CB>), dim3((unsigned)blocks), dim3(kThreads), 0, stream, a);
    if (a.key_parts > kFewParts)
      hipLaunchKernelGGL(stats_join_kernel, dim3((unsigned)joins), dim3(256), 0, stream, a.stats, rows, a.key_parts);
    hipLaunchKernelGGL((sum_kernel<E, D, CB, false>), dim3((unsigned)sum_blocks), dim3(kThreads), 0, stream, a);
  }
  if (a.row_parts > 1)
    hipLaunchKernelGGL(sum_join_kernel, dim3((unsigned)((a.L + 255) / 256), (unsigned)(heads < 65535 ? heads : 65535)), dim3(256), 0, stream, a);
  return hipGetLastError();
}

template <class E, int D>
hipError_t launch_rows(const WeightsArgs& a, hipStream_t stream) {
  const int cb = row_blocks_wave(a);
  return cb == 1 ? launch<E, D, 1>(a, stream) : cb == 2 ? launch<E, D, 2>(a, stream) : launch<E, D, 4>(a, stream);
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
  if (a.f16) return a.D == 128 ? launch_rows<_Float16, 128>(a, stream) : launch_rows<_Float16, 64>(a, stream);
  return a.D == 128 ? launch_rows<__bf16, 128>(a, stream) : launch_rows<__bf16, 64>(a, stream);
}

}  // namespace s2o
