// Decoding against a shared cache for gfx950: B sequences attend the cache of their common prefix, read once for all of
// them, and each its own rows behind it.
//
//   x_j = scale <q, k_j>,  lse = log sum_j exp(x_j),  O = sum_j exp(x_j - lse) v_j
//
// over the rows j that a query sees: all of the shared cache, and of its sequence's own p rows the first p - T + t + 1 for
// query token t of T.  The B*T*G query rows of one (cache, KV head) are the columns of one matrix product with the
// shared rows; the T*G rows of a sequence are the columns of a product with its own.
//
// One launch covers both kinds of row blocks, each split over its keys (a part is one workgroup's share of keys), and leaves an
// un-normalised softmax state (accumulator, maximum, sum) per query row and part; a second launch joins the parts.  Where
// all keys are few, a workgroup walks a sequence's shared and own rows in turn and writes the result itself.
//
// A wavefront walks tiles of 32 keys of its own, without barriers: K operands come straight from global memory (16 rows x 64
// bytes an instruction), V passes through a wavefront's private 32 x D of LDS for the transposing read.  The next
// tile's loads are issued as soon as the score products have consumed the current ones.  Bound: HBM bandwidth.
#include "cache_tile.h"
#include "s2o_internal.h"

namespace s2o {

namespace {

using namespace cache;

constexpr int kWaves = 4, kThreads = 64 * kWaves, kKeys = 32;
constexpr float kLazy = 8.0f;    // the softmax reference follows the maximum in steps of 2^8 at least (attn_tile.h)

// Query rows of a workgroup: those of one sequence (b >= 0) or of all that read the cache, with t the slowest index.
struct Rows {
  int z, b, g, count;
  __device__ __forceinline__ void find(const DecodeArgs& a, int r, int& bb, int& h, int& t) const {
    const int per_t = b < 0 ? a.B * a.G : a.G, rest = r % per_t;
    t = r / per_t;
    bb = b < 0 ? rest / a.G : b;
    h = g * a.G + rest % a.G;
  }
};

template <class E, int D, int CB>
struct Walk {
  typedef typename Vec<E>::x8 x8;
  x8 q[CB][D / 32];
  f32x4 o[CB][D / 16];
  float m[CB], l[CB];            // reference (base 2) and the lane's part of the sum

  __device__ __forceinline__ void start() {
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
      m[cb] = -INFINITY;
      l[cb] = 0.f;
#pragma unroll
      for (int db = 0; db < D / 16; ++db) o[cb][db] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
  }

  // Tiles first, first + step, .. < end of a cache of `len` rows; the lane's column cb sees the first lim[cb] of them.
  // vt: the wavefront's 32 x D elements of LDS.
  __device__ __forceinline__ void tiles(const E* K, const E* V, int64_t kstride, int64_t vstride, int len, const int (&lim)[CB],
                                        int first, int end, int step, float c2, unsigned char* vt, int lane) {
    constexpr int kRowLanes = D / 8, kLoads = D / 16;      // 16-byte pieces a row; V loads a lane
    constexpr int kRowsPerLoad = 64 / kRowLanes;
    const int mm = lane & 15, g = lane >> 4;
    u32x4 kr[2][D / 32], vr[kLoads];
    const uint32_t krow = (uint32_t)(kstride * 2), vrow = (uint32_t)(vstride * 2);
    auto load = [&](int t) {
      const char* kt = reinterpret_cast<const char*>(K + (int64_t)t * kKeys * kstride);
      const char* vtile = reinterpret_cast<const char*>(V + (int64_t)t * kKeys * vstride);
      const int last = len - 1 - t * kKeys;                // rows behind the cache's end are not read: the last one instead
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        const uint32_t off = (uint32_t)min(16 * kb + mm, last) * krow + 16 * g;
#pragma unroll
        for (int kk = 0; kk < D / 32; ++kk) kr[kb][kk] = *reinterpret_cast<const u32x4*>(kt + off + 64 * kk);
      }
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const uint32_t off = (uint32_t)min(kRowsPerLoad * i + lane / kRowLanes, last) * vrow + 16 * (lane % kRowLanes);
        vr[i] = *reinterpret_cast<const u32x4*>(vtile + off);
      }
    };
    if (first < end) load(first);
    for (int t = first; t < end; t += step) {
      const int key0 = t * kKeys;
      bool hidden = false;                                 // some row of this tile is not seen by some column
#pragma unroll
      for (int cb = 0; cb < CB; ++cb) hidden |= lim[cb] < key0 + kKeys;
      hidden = __builtin_amdgcn_ballot_w64(hidden) != 0;
      bool odd_values = false;
      wave_fence();                                        // the last tile's reads are through
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int r = kRowsPerLoad * i + lane / kRowLanes;
        u32x4 v = vr[i];
        if (hidden) {
          if (key0 + r >= len) v = u32x4{0, 0, 0, 0};
          odd_values |= not_finite<E>(v);
        }
        *reinterpret_cast<u32x4*>(vt + at<D>(r, lane % kRowLanes)) = v;
      }
      wave_fence();
      f32x4 s[2][CB];
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) {
          s[kb][cb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int kk = 0; kk < D / 32; ++kk) s[kb][cb] = mfma(__builtin_bit_cast(x8, kr[kb][kk]), q[cb][kk], s[kb][cb]);
        }
      if (t + step < end) load(t + step);
      if (hidden) {
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int cb = 0; cb < CB; ++cb)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (key0 + 16 * kb + 4 * g + i >= lim[cb]) s[kb][cb][i] = -INFINITY;
      }
      // softmax numerators against a lazily moving reference; the sums stay per lane until the end
      x8 pb[CB];
#pragma unroll
      for (int cb = 0; cb < CB; ++cb) {
        float top = fmaxf(fmaxf(fmaxf(s[0][cb][0], s[0][cb][1]), fmaxf(s[0][cb][2], s[0][cb][3])),
                          fmaxf(fmaxf(s[1][cb][0], s[1][cb][1]), fmaxf(s[1][cb][2], s[1][cb][3])));
        top = column_max(top) * c2;
        const bool grow = top > m[cb] + kLazy;
        if (__builtin_amdgcn_ballot_w64(grow) != 0) {
          const float m_new = grow ? top : m[cb];
          const float alpha = grow ? exp2_(m[cb] - m_new) : 1.0f;
          m[cb] = m_new;
          l[cb] *= alpha;
#pragma unroll
          for (int db = 0; db < D / 16; ++db)
#pragma unroll
            for (int i = 0; i < 4; ++i) o[cb][db][i] *= alpha;
        }
        const float ref = m[cb] == -INFINITY ? 0.f : m[cb];
        float sum = 0.f;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float p = exp2_(fmaf(s[kb][cb][i], c2, -ref));
            s[kb][cb][i] = p;
            sum += p;
          }
        l[cb] += sum;
        // rounded for the second product (half a step of the cache's own type); the sum is of the unrounded ones
        u32x4 w;
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = pack2<E>(s[j >> 1][cb][2 * (j & 1)], s[j >> 1][cb][2 * (j & 1) + 1]);
        pb[cb] = __builtin_bit_cast(x8, w);
      }
      if (hidden && __builtin_amdgcn_ballot_w64(odd_values) != 0) {
        // An infinity or NaN in a row that some column does not see must not reach it as 0 * inf: key by key, hidden
        // ones left out.
#pragma unroll 1
        for (int r = 0; r < kKeys; ++r) {
#pragma unroll
            for (int cb = 0; cb < CB; ++cb) {
              const f32x4 sv = r >= 16 ? s[1][cb] : s[0][cb];
              const float mine = (r & 3) == 0 ? sv[0] : (r & 3) == 1 ? sv[1] : (r & 3) == 2 ? sv[2] : sv[3];
              const float p = __shfl(mine, 16 * ((r & 15) >> 2) + mm);
              if (key0 + r < lim[cb])
#pragma unroll
                for (int db = 0; db < D / 16; ++db) {
                  const E* v = reinterpret_cast<const E*>(vt + at<D>(r, 2 * db + (g >> 1)) + 8 * (g & 1));
#pragma unroll
                  for (int i = 0; i < 4; ++i) o[cb][db][i] = fmaf(p, (float)v[i], o[cb][db][i]);
                }
            }
          }
      } else {
        const int rl = 4 * g + (mm >> 2);
#pragma unroll
        for (int db = 0; db < D / 16; ++db) {
          typedef __attribute__((address_space(3))) i16x4 lds_i16x4;
          const int c = 2 * db + ((mm & 3) >> 1), in = 8 * (mm & 1);
          const i16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(vt + at<D>(rl, c) + in));
          const i16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(vt + at<D>(16 + rl, c) + in));
          const u32x2 w0 = __builtin_bit_cast(u32x2, v0), w1 = __builtin_bit_cast(u32x2, v1);
          const x8 vf = __builtin_bit_cast(x8, u32x4{w0.x, w0.y, w1.x, w1.y});
#pragma unroll
          for (int cb = 0; cb < CB; ++cb) o[cb][db] = mfma(vf, pb[cb], o[cb][db]);
        }
      }
    }
  }
};

// Joins softmax states: weights of the parts relative to their common reference.
__device__ __forceinline__ float part_weight(float m, float top) { return exp2_(m - (top == -INFINITY ? 0.f : top)); }
__device__ __forceinline__ float natural_lse(float top, float sum) {
  // sum == 0: nothing was seen (a NaN sum goes on as NaN)
  return sum == 0.f ? -INFINITY : ((top == -INFINITY ? 0.f : top) + __builtin_amdgcn_logf(sum)) * kLn2;
}

template <class E, int D, int CB>
__global__ __launch_bounds__(kThreads, 2) void decode_kernel(const DecodeArgs a) {
  constexpr int kPad = D + 4;
  constexpr int kTile = kKeys * D * 2;
  constexpr int kJoin = kWaves * 16 * kPad * 4;
  __shared__ __attribute__((aligned(256))) unsigned char smem[kWaves * kTile > kJoin ? kWaves * kTile : kJoin];
  __shared__ float2 ml[kWaves][16];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int mm = lane & 15, g = lane >> 4;

  // block id -> shared units (cache, KV head, row block) x parts, then own units (.., sequence, ..) x parts
  const int units_s = a.Z * a.Hkv * a.blocks_s;
  int id = blockIdx.x, part;
  Rows rows;
  int rb;
  bool shared = !a.direct && id < units_s * a.splits_s;
  if (shared) {
    part = id / units_s;
    id -= part * units_s;
    rb = id % a.blocks_s;
    id /= a.blocks_s;
    rows.g = id % a.Hkv;
    rows.z = id / a.Hkv;
    rows.b = -1;
    rows.count = a.B * a.T * a.G;
  } else {
    if (!a.direct) id -= units_s * a.splits_s;
    const int units_o = a.Z * a.B * a.Hkv * a.blocks_o;
    part = id / units_o;
    id -= part * units_o;
    rb = id % a.blocks_o;
    id /= a.blocks_o;
    rows.g = id % a.Hkv;
    id /= a.Hkv;
    rows.b = id % a.B;
    rows.z = id / a.B;
    rows.count = a.T * a.G;
  }
  const int z = rows.z, hk = rows.g;

  Walk<E, D, CB> w;
  w.start();
  int t_of[CB];
  const E* Q = static_cast<const E*>(a.Q);
#pragma unroll
  for (int cb = 0; cb < CB; ++cb) {
    int b, h;
    rows.find(a, min(16 * (rb * CB + cb) + mm, rows.count - 1), b, h, t_of[cb]);
    const E* q = Q + z * a.qs[0] + b * a.qs[1] + h * a.qs[2] + t_of[cb] * a.qs[3];
#pragma unroll
    for (int kk = 0; kk < D / 32; ++kk) w.q[cb][kk] = *reinterpret_cast<const typename Vec<E>::x8*>(q + 32 * kk + 8 * g);
  }
  unsigned char* vt = smem + wave * kTile;
  // the shared rows, the sequence's own, or both
#pragma unroll 1
  for (int own = shared || a.direct ? 0 : 1; own < (shared ? 1 : 2); ++own) {
    const E *K, *V;
    int64_t kst, vst;
    int len, splits = 1, lim[CB];
    if (own) {
      K = static_cast<const E*>(a.oK) + z * a.oks[0] + rows.b * a.oks[1] + hk * a.oks[2];
      V = static_cast<const E*>(a.oV) + z * a.ovs[0] + rows.b * a.ovs[1] + hk * a.ovs[2];
      kst = a.oks[3]; vst = a.ovs[3];
      len = filled(a.own_lens, z * a.B + rows.b, a.Lo);
      if (!a.direct) splits = a.splits_o;
    } else {
      K = static_cast<const E*>(a.K) + z * a.ks[0] + hk * a.ks[1];
      V = static_cast<const E*>(a.V) + z * a.vs[0] + hk * a.vs[1];
      kst = a.ks[2]; vst = a.vs[2];
      len = filled(a.lens, z, a.L);
      if (!a.direct) splits = a.splits_s;
    }
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) lim[cb] = own ? min(max(len - a.T + t_of[cb] + 1, 0), len) : len;
    const int tiles = (len + kKeys - 1) / kKeys;
    const int from = (int)((int64_t)tiles * part / splits), to = (int)((int64_t)tiles * (part + 1) / splits);
    w.tiles(K, V, kst, vst, len, lim, from + wave, to, kWaves, a.c2, vt, lane);
  }

  // join the wavefronts, 16 rows at a time
  const int64_t all_rows = (int64_t)a.Z * a.B * a.H * a.T;
  const int slot = shared ? part : a.splits_s + part;
#pragma unroll
  for (int cb = 0; cb < CB; ++cb) {
    __syncthreads();
    float* ob = reinterpret_cast<float*>(smem);
    const float l = column_sum(w.l[cb]);
#pragma unroll
    for (int db = 0; db < D / 16; ++db) *reinterpret_cast<f32x4*>(ob + (wave * 16 + mm) * kPad + 16 * db + 4 * g) = w.o[cb][db];
    if (g == 0) ml[wave][mm] = float2{w.m[cb], l};
    __syncthreads();
    const int i = tid >> 4, r = 16 * (rb * CB + cb) + i, d0 = (tid & 15) * (D / 16);
    if (r < rows.count) {
      float top = -INFINITY, sum = 0.f;
#pragma unroll
      for (int v = 0; v < kWaves; ++v) top = fmaxf(top, ml[v][i].x);
      float acc[D / 16];
#pragma unroll
      for (int d = 0; d < D / 16; ++d) acc[d] = 0.f;
#pragma unroll
      for (int v = 0; v < kWaves; ++v) {
        const float f = part_weight(ml[v][i].x, top);
        sum = fmaf(f, ml[v][i].y, sum);
#pragma unroll
        for (int d = 0; d < D / 16; ++d) acc[d] = fmaf(f, ob[(v * 16 + i) * kPad + d0 + d], acc[d]);
      }
      int b, h, t;
      rows.find(a, r, b, h, t);
      const int64_t row = (((int64_t)z * a.B + b) * a.H + h) * a.T + t;
      if (a.part_acc) {
        float* p = a.part_acc + (slot * all_rows + row) * D + d0;
#pragma unroll
        for (int d = 0; d < D / 16; d += 4) *reinterpret_cast<f32x4*>(p + d) = f32x4{acc[d], acc[d + 1], acc[d + 2], acc[d + 3]};
        if ((tid & 15) == 0) a.part_ml[slot * all_rows + row] = float2{top, sum};
      } else {
        const float inv = sum == 0.f ? 0.f : 1.0f / sum;
        uint32_t* o = reinterpret_cast<uint32_t*>(static_cast<E*>(a.O) + z * a.os[0] + b * a.os[1] + h * a.os[2] + t * a.os[3] + d0);
#pragma unroll
        for (int d = 0; d < D / 16; d += 2) o[d / 2] = pack2<E>(acc[d] * inv, acc[d + 1] * inv);
        if (a.lse && (tid & 15) == 0) a.lse[row] = natural_lse(top, sum);
      }
    }
  }
}

// Joins the parts of a row: D/4 threads x `lanes` part lanes a row.
template <class E, int D>
__global__ __launch_bounds__(256) void decode_join_kernel(const DecodeArgs a, int parts, int lanes) {
  constexpr int kQuads = D / 4;
  __shared__ f32x4 acc_s[256];
  __shared__ float sum_s[256];
  const int64_t all_rows = (int64_t)a.Z * a.B * a.H * a.T;
  const int per_row = kQuads * lanes, tid = threadIdx.x;
  const int64_t row = (int64_t)blockIdx.x * (256 / per_row) + tid / per_row;
  const int pl = tid % per_row / kQuads, quad = tid % kQuads;
  const bool live = row < all_rows;
  float top = -INFINITY, sum = 0.f;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  if (live) {
    for (int p = 0; p < parts; ++p) top = fmaxf(top, a.part_ml[p * all_rows + row].x);
#pragma unroll 4
    for (int p = pl; p < parts; p += lanes) {
      const float2 s = a.part_ml[p * all_rows + row];
      const f32x4 v = *reinterpret_cast<const f32x4*>(a.part_acc + (p * all_rows + row) * D + 4 * quad);
      const float f = part_weight(s.x, top);
      sum = fmaf(f, s.y, sum);
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[i] = fmaf(f, v[i], acc[i]);
    }
  }
  if (lanes > 1) {
    acc_s[tid] = acc;
    sum_s[tid] = sum;
    __syncthreads();
    if (pl != 0) return;
    for (int p = 1; p < lanes; ++p) {
      sum += sum_s[tid + p * kQuads];
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[i] += acc_s[tid + p * kQuads][i];
    }
  }
  if (!live) return;
  const int t = (int)(row % a.T);
  int64_t i = row / a.T;
  const int h = (int)(i % a.H);
  i /= a.H;
  const int b = (int)(i % a.B), z = (int)(i / a.B);
  const float inv = sum == 0.f ? 0.f : 1.0f / sum;
  E* o = static_cast<E*>(a.O) + z * a.os[0] + b * a.os[1] + h * a.os[2] + t * a.os[3] + 4 * quad;
  *reinterpret_cast<u32x2*>(o) = u32x2{pack2<E>(acc[0] * inv, acc[1] * inv), pack2<E>(acc[2] * inv, acc[3] * inv)};
  if (a.lse && quad == 0) a.lse[row] = natural_lse(top, sum);
}

constexpr int kWorkgroups = 768;   // that the split aims at: three on each of 256 CUs

struct Shape {
  int cb_s, blocks_s, splits_s, blocks_o, splits_o, direct;
  int parts() const { return splits_s + splits_o; }
};

// How the call's keys are dealt out.  (Host; a rule on the sizes the memory was laid out for, since the lengths may live on the device.)
Shape shape_of(const DecodeArgs& a) {
  Shape s{};
  const int64_t rows_s = (int64_t)a.B * a.T * a.G, rows_o = (int64_t)a.T * a.G;
  const int64_t units = (int64_t)a.Z * a.Hkv;
  s.blocks_s = (int)((rows_s + 15) / 16);
  s.blocks_o = (int)((rows_o + 15) / 16);
  const int64_t units_s = units * s.blocks_s, units_o = units * a.B * s.blocks_o;
  s.direct = a.L + a.Lo <= 512 || (a.L == 0 && units_o >= kWorkgroups);
  if (s.direct) {
    s.splits_s = 0;
    s.splits_o = 1;
    return s;
  }
  auto split = [](int64_t units, int64_t keys) {
    const int64_t want = (kWorkgroups + units - 1) / units, most = (keys + 255) / 256;
    return (int)(want < most ? want : most);
  };
  s.splits_s = a.L ? split(units_s, a.L) : 0;
  s.splits_o = a.Lo ? split(units_o, a.Lo) : 0;
  return s;
}

template <class E, int D>
hipError_t launch(DecodeArgs a, const Shape& s, hipStream_t stream) {
  const int64_t all_rows = (int64_t)a.Z * a.B * a.H * a.T;
  const int64_t units_s = (int64_t)a.Z * a.Hkv * s.blocks_s, units_o = (int64_t)a.Z * a.Hkv * a.B * s.blocks_o;
  const int64_t blocks = units_s * s.splits_s + units_o * s.splits_o;
  if (blocks <= 0 || blocks > 0x7fffffff) return hipErrorInvalidValue;
  if (s.direct) a.part_acc = nullptr;
  hipLaunchKernelGGL((decode_kernel<E, D, 1>), dim3((unsigned)blocks), dim3(kThreads), 0, stream, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || s.direct) return e;
  int lanes = 1;
  while (lanes < 1024 / D && lanes * 2 <= s.parts()) lanes *= 2;
  const int64_t per = 256 / (D / 4 * lanes);
  hipLaunchKernelGGL((decode_join_kernel<E, D>), dim3((unsigned)((all_rows + per - 1) / per)), dim3(256), 0, stream, a, s.parts(), lanes);
  return hipGetLastError();
}

}  // namespace

size_t decode_scratch_bytes(const DecodeArgs& a) {
  const Shape s = shape_of(a);
  if (s.direct) return 0;
  const size_t rows = (size_t)a.Z * a.B * a.H * a.T;
  return (size_t)s.parts() * rows * (a.D * 4 + 8);
}

hipError_t launch_decode(DecodeArgs a, void* scratch, hipStream_t stream) {
  const Shape s = shape_of(a);
  a.blocks_s = s.blocks_s; a.splits_s = s.splits_s; a.blocks_o = s.blocks_o; a.splits_o = s.splits_o; a.direct = s.direct;
  const size_t rows = (size_t)a.Z * a.B * a.H * a.T;
  a.part_acc = static_cast<float*>(scratch);
  a.part_ml = reinterpret_cast<float2*>(a.part_acc + (size_t)s.parts() * rows * a.D);
  if (a.f16) return a.D == 128 ? launch<_Float16, 128>(a, s, stream) : launch<_Float16, 64>(a, s, stream);
  return a.D == 128 ? launch<__bf16, 128>(a, s, stream) : launch<__bf16, 64>(a, s, stream);
}

}  // namespace s2o
