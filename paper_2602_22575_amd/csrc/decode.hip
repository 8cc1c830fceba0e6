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
// A row block of up to 16 rows is walked by wavefronts on their own (Walk::narrow): each takes tiles of 32 keys in turn, without
// barriers; K operands come straight from global memory (16 rows x 64 bytes an instruction), V passes through a wavefront's
// private 32 x D of LDS for the transposing read.  The next tile's loads are issued as soon as the score products have consumed the
// current ones.  Bound: HBM bandwidth.
// Blocks of 128 rows share tiles of 64 keys between four wavefronts of 32 rows each (Walk::wide): global memory goes
// straight to LDS, one tile ahead (one and a half ahead, with a second barrier a tile, was 2 to 4 % slower).  Bound: HBM bandwidth up to
// about 256 rows a KV head, the matrix cores beyond.
//
// Measured, bf16, D 128, 32 query heads on 8: one sequence on 32K keys 26 us and 4 for the join, 5.2 TB/s; 32 sequences on 32K keys and up to
// 512 of their own each 38 and 6; 64 on 128K and up to 1024 of their own 143 to 170, by the clock that the power limit leaves, and 8: 0.76 to
// 0.9 PFLOP/s.  Of a launch 3 us pass until the first keys are asked for (arguments, indices, the first pass through the code) and 3 while
// the parts' states are written.
#include <type_traits>

#include "cache_tile.h"
#include "s2o_internal.h"

namespace s2o {

namespace {

using namespace cache;

constexpr int kWaves = 4, kThreads = 64 * kWaves;
constexpr int kCus = 256;
constexpr int kSplitWaves = 8;                  // of a workgroup without wide blocks, where the keys are split
constexpr int kKeys = 32, kWideKeys = 64;       // tiles of the two walks
constexpr int kNarrowRows = 16, kWideRows = 32 * kWaves;   // query rows of a workgroup
constexpr float kLazy = 8.0f;    // the softmax reference follows the maximum in steps of 2^8 at least (attn_tile.h)

// Query rows of a workgroup: those of one sequence (b >= 0) or of all that read the cache, with t the slowest index.
struct Rows {
  int z, b, g, count;
  __device__ __forceinline__ void find(const DecodeArgs& a, int r, int& bb, int& h, int& t) const {
    int rest, in_group;
    t = (b < 0 ? a.by_BG : a.by_G).by(r, rest);
    const int sequence = a.by_G.by(rest, in_group);
    bb = b < 0 ? sequence : b;
    h = g * a.G + in_group;
  }
};

// The softmax state of 16 * CB query rows in a wavefront (column cb of lane l: row 16 * cb + l % 16).
template <class E, int D, int CB>
struct Walk {
  typedef typename Vec<E>::x8 x8;
  x8 q[CB][D / 32];
  f32x4 o[CB][D / 16];
  float m[CB], l[CB];            // reference (base 2) and the lane's part of the sum

  // keep: the references stay
  __device__ __forceinline__ void start(bool keep = false) {
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
      if (!keep) m[cb] = -INFINITY;
      l[cb] = 0.f;
#pragma unroll
      for (int db = 0; db < D / 16; ++db) o[cb][db] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
  }

  // Scores of KB blocks of 16 keys -> softmax numerators (in s, fp32) and their rounding for the second product (half a step of the cache's
  // own type; the sums are of the unrounded ones).  The reference follows the maximum lazily; sums stay per lane until the end.
  template <int KB, bool kHidden>
  __device__ __forceinline__ void softmax(f32x4 (&s)[KB][CB], x8 (&pb)[KB / 2][CB], int key0, const int (&lim)[CB], float c2, int g) {
    if constexpr (kHidden) {
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int cb = 0; cb < CB; ++cb)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (key0 + 16 * kb + 4 * g + i >= lim[cb]) s[kb][cb][i] = -INFINITY;
    }
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
      float top = -INFINITY;
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int i = 0; i < 4; ++i) top = fmaxf(top, s[kb][cb][i]);
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
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float p = exp2_(fmaf(s[kb][cb][i], c2, -ref));
          s[kb][cb][i] = p;
          sum += p;
        }
      l[cb] += sum;
#pragma unroll
      for (int st = 0; st < KB / 2; ++st) {
        u32x4 w;
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = pack2<E>(s[2 * st + (j >> 1)][cb][2 * (j & 1)], s[2 * st + (j >> 1)][cb][2 * (j & 1) + 1]);
        pb[st][cb] = __builtin_bit_cast(x8, w);
      }
    }
  }

  // The V^T operand of 16 dims and 32 keys whose rows start at `vt` in LDS: keys 4 * g + (0..3) and 16 + 4 * g + (0..3).
  // kMade: the place of the upper dims is made from that of the lower ones each time, not kept in a register.
  template <bool kMade = false>
  static __device__ __forceinline__ u32x4 value_operand(const unsigned char* vt, int db, int mm, int g) {
    typedef __attribute__((address_space(3))) i16x4 lds_i16x4;
    uint32_t place = (at<D>(4 * g + (mm >> 2), (mm & 3) >> 1) + 8 * (mm & 1)) ^ ((kMade ? db & 3 : db) << 5);
    if (kMade && db >= 4) asm volatile("v_xor_b32 %0, 0x80, %1" : "=v"(place) : "v"(place));
    const unsigned char* p = vt + place;
    const i16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)p);
    const i16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(p + 16 * 2 * D));
    const u32x2 w0 = __builtin_bit_cast(u32x2, v0), w1 = __builtin_bit_cast(u32x2, v1);
    return u32x4{w0.x, w0.y, w1.x, w1.y};
  }
  // O^T += V^T P^T for 32 * ST keys
  template <int ST>
  __device__ __forceinline__ void values(const unsigned char* vt, const x8 (&pb)[ST][CB], int mm, int g) {
#pragma unroll
    for (int st = 0; st < ST; ++st)
#pragma unroll
      for (int db = 0; db < D / 16; ++db) {
        const x8 vf = __builtin_bit_cast(x8, value_operand(vt + st * 64 * D, db, mm, g));
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) o[cb][db] = mfma(vf, pb[st][cb], o[cb][db]);
      }
  }
  // The same where some column does not see all of the keys.  A row that a column does not see has p = 0 there, but may hold an infinity or
  // NaN: per limit that occurs (one, but for the last tokens of several) a product with the rows behind it as zeros, added to
  // the columns of that limit.
  template <int ST>
  __device__ __forceinline__ void values_hidden(const unsigned char* vt, const x8 (&pb)[ST][CB], int key0, const int (&lim)[CB], int mm, int g) {
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
      uint64_t todo = ~0ull;
      while (todo) {
        const int u = __builtin_amdgcn_readlane(lim[cb], __builtin_ctzll(todo));
        const bool mine = lim[cb] == u;
        todo &= ~__builtin_amdgcn_ballot_w64(mine);
#pragma unroll
        for (int st = 0; st < ST; ++st)
#pragma unroll
          for (int db = 0; db < D / 16; ++db) {
            u32x4 v = value_operand(vt + st * 64 * D, db, mm, g);
            const int left = u - key0 - 32 * st - 4 * g;             // of the operand's keys 0..3, 16..19
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const int key = 16 * (j >> 1) + 2 * (j & 1);
              v[j] = key + 1 < left ? v[j] : key < left ? v[j] & 0xffffu : 0u;
            }
            const f32x4 sum = mfma(__builtin_bit_cast(x8, v), pb[st][cb], f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
            for (int i = 0; i < 4; ++i) o[cb][db][i] += mine ? sum[i] : 0.f;
          }
      }
    }
  }

  // Tiles first, first + step, .. < end of a cache of `len` rows.  `rows` loads the queries, behind the first keys, and tells what they see: the
  // lane's column cb the first lim[cb] rows, every column the first lim_all.  vt: the wavefront's 32 x D elements of LDS.
  // (The tiles that some column does not see all of, the last ones, have a loop of their own here and in `wide`: what they need
  // beside the products would cost every tile registers.)
  template <class F>
  __device__ __forceinline__ void narrow(const E* K, const E* V, int64_t kstride, int64_t vstride, int len, int first, int end, int step,
                                         float c2, unsigned char* vt, int lane, F rows) {
    if (first >= end) return;
    constexpr int kRowLanes = D / 8, kLoads = D / 16;      // 16-byte pieces a row; V loads a lane
    constexpr int kRowsPerLoad = 64 / kRowLanes;
    const int mm = lane & 15, g = lane >> 4, lr = lane / kRowLanes;
    u32x4 kr[2][D / 32], vr[kLoads];
    const uint32_t koff = (uint32_t)mm * (uint32_t)(kstride * 2) + 16 * g, voff = (uint32_t)lr * (uint32_t)(vstride * 2) + 16 * (lane % kRowLanes);
    const int vst = at<D>(lr, lane % kRowLanes);
    auto load = [&](int t) {
      const auto kt = rows_buffer(K, kstride * 2, t * kKeys, len, kKeys, 2 * D), vtile = rows_buffer(V, vstride * 2, t * kKeys, len, kKeys, 2 * D);
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int kk = 0; kk < D / 32; ++kk) kr[kb][kk] = buffer_load(kt, koff + 16 * kb * (uint32_t)(kstride * 2) + 64 * kk);
#pragma unroll
      for (int i = 0; i < kLoads; ++i) vr[i] = buffer_load(vtile, voff + kRowsPerLoad * i * (uint32_t)(vstride * 2));
    };
    int lim[CB], lim_all;
    auto tile = [&](int t, auto hidden_) {
      constexpr bool kHidden = decltype(hidden_)::value;
      const int key0 = t * kKeys;
      wave_fence();                                        // the last tile's reads are through
#pragma unroll
      for (int i = 0; i < kLoads; ++i)
        *reinterpret_cast<u32x4*>(vt + kRowsPerLoad * i * 2 * D + (vst ^ (swz<D>(kRowsPerLoad * i) << 4))) = vr[i];
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
      __builtin_amdgcn_sched_barrier(0);                   // (the loads take over the products' operand registers)
      if (t + step < end) load(t + step);
      x8 pb[1][CB];
      softmax<2, kHidden>(s, pb, key0, lim, c2, g);
      if constexpr (kHidden) values_hidden<1>(vt, pb, key0, lim, mm, g);
      else values<1>(vt, pb, mm, g);
    };
    load(first);
    rows(lim, lim_all);
    int t = first;
    for (; t < end && (t + 1) * kKeys <= lim_all; t += step) tile(t, std::false_type{});
    for (; t < end; t += step) tile(t, std::true_type{});
  }

  // Tiles from .. to - 1 of 64 keys, by all four wavefronts together; `rows` as above.  ka, kb_, va, vb: K and V tile of even and odd steps (separate
  // arrays, so that the compiler sees that reads of one need not wait for the loads that fill another).
  //
  // The first keys find the references that there are not yet (16 of them; 64 for fp16, whose numerators have room for 2^15), the last tiles may have
  // hidden keys.  For the others, if `fast`, a tile's products and exponentials are one straight run of instructions, its second half's
  // exponentials behind its first half's products: numerators are formed against the references as they are, and a reference moves
  // afterwards, where two tiles' sum has outgrown 2^10.  Returns false where a numerator or an accumulator may have outgrown its type on the
  // way: all of it is to be done again, with the references that are known by then.
  template <class F>
  __device__ __forceinline__ bool wide(const E* K, const E* V, int64_t kstride, int64_t vstride, int len, int from, int to, float c2,
                                       unsigned char* ka, unsigned char* kb_, unsigned char* va, unsigned char* vb, int wave, int lane,
                                       bool fast, F rows) {
    if (from >= to) return true;
    int lim[CB], lim_all;
    constexpr int kRowLanes = D / 8, kRowsPerLoad = 64 / kRowLanes, kLoads = 16 / kRowsPerLoad;   // a wavefront loads 16 rows of each
    constexpr float kMove = 0x1p10f, kMost = __is_same(E, __bf16) ? 0x1p60f : 0x1p15f;
    const int mm = lane & 15, g = lane >> 4;
    // LDS takes a load's lanes in order: each fetches the chunk that belongs at its slot.  (Offsets are made for every tile: kept, they would
    // be put aside in memory.)
    const uint32_t krow = (uint32_t)(kstride * 2), vrow = (uint32_t)(vstride * 2);
    auto fetch = [&](int t, unsigned char* kt, unsigned char* vt) {
      const auto kg = rows_buffer(K, kstride * 2, t * kWideKeys, len, kWideKeys, 2 * D), vg = rows_buffer(V, vstride * 2, t * kWideKeys, len, kWideKeys, 2 * D);
      const int ln = lane_id(), lr = ln / kRowLanes;
      const uint32_t ko = (uint32_t)lr * krow, vo = (uint32_t)lr * vrow, ch = 16 * ((ln % kRowLanes) ^ swz<D>(lr));
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int r = 16 * wave + kRowsPerLoad * i;
        const uint32_t c = ch ^ (swz<D>(kRowsPerLoad * i) << 4);
        buffer_load_to_lds(kg, ko + r * krow + c, kt + r * 2 * D);
        buffer_load_to_lds(vg, vo + r * vrow + c, vt + r * 2 * D);
      }
    };
    // what this wavefront fetched has landed and what it read is in its registers; then everybody's
    auto meet = [] {
      asm volatile("" ::: "memory");
      __builtin_amdgcn_s_waitcnt(0x0070);                  // vmcnt(0) lgkmcnt(0)
      asm volatile("s_barrier" ::: "memory");
    };
    auto scores = [&](const unsigned char* kt, f32x4 (&s)[4][CB]) {
#pragma unroll
      for (int kb = 0; kb < 4; ++kb) {
        x8 k[D / 32];
#pragma unroll
        for (int kk = 0; kk < D / 32; ++kk) k[kk] = *reinterpret_cast<const x8*>(kt + 16 * kb * 2 * D + (at<D>(mm, g) ^ (kk << 6)));
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) s[kb][cb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kk = 0; kk < D / 32; ++kk)
#pragma unroll
          for (int cb = 0; cb < CB; ++cb) s[kb][cb] = mfma(k[kk], q[cb][kk], s[kb][cb]);
      }
    };
    auto any_tile = [&](int t, unsigned char* kt, unsigned char* vt, unsigned char* knext, unsigned char* vnext) {
      if (t + 1 < to) fetch(t + 1, knext, vnext);
      const int key0 = t * kWideKeys;
      f32x4 s[4][CB];
      scores(kt, s);
      x8 pb[2][CB];
      softmax<4, true>(s, pb, key0, lim, c2, g);
      values_hidden<2>(vt, pb, key0, lim, mm, g);
      meet();
    };
    bool fits = true;
    auto fast_tile = [&](int t, unsigned char* kt, unsigned char* vt, unsigned char* knext, unsigned char* vnext, float (&sum)[CB]) {
      if (t + 1 < to) fetch(t + 1, knext, vnext);
      // K operands in pairs p = (32-key half, 32 dims), two pairs ahead of their products; V operands behind them, four ahead.  Every
      // product, and what stands behind it, is a scheduling region of its own.
      constexpr int kDims = D / 32, kPairs = 2 * kDims, kBlocks = D / 16, kAhead = 4;
      constexpr int kEach = 16 / (2 * kDims * CB);         // scores a lane that are worked on behind a product: 16 a half
      static_assert(CB == 2 && kEach * 2 * kDims * CB == 16 && kBlocks == 2 * kDims);
      f32x4 s[4][CB];
      x8 kf[kPairs][2], vf[2 * kBlocks], pb[2][CB];
      float p[2][16];
      auto read_keys = [&](int pair) {
#pragma unroll
        for (int e = 0; e < 2; ++e)
          kf[pair][e] = *reinterpret_cast<const x8*>(kt + 16 * (2 * (pair / kDims) + e) * 2 * D + (at<D>(mm, g) ^ ((pair % kDims) << 6)));
      };
      auto read_values = [&](int f) { vf[f] = __builtin_bit_cast(x8, value_operand<true>(vt + (f / kBlocks) * 64 * D, f % kBlocks, mm, g)); };
      auto numerators = [&](int half, int first) {         // of the half's scores first .. first + kEach - 1: 8 * column block + key
#pragma unroll
        for (int x = first; x < first + kEach; ++x) {
          const int cb = x >> 3, j = x & 7;
          p[half][x] = exp2_(fmaf(s[2 * half + (j >> 2)][cb][j & 3], c2, -m[cb]));
          sum[cb] += p[half][x];
        }
      };
      auto pack = [&](int half) {
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) {
          u32x4 w;
#pragma unroll
          for (int j = 0; j < 4; ++j) w[j] = pack2<E>(p[half][8 * cb + 2 * j], p[half][8 * cb + 2 * j + 1]);
          pb[half][cb] = __builtin_bit_cast(x8, w);
        }
      };
      read_keys(0);
      read_keys(1);
#pragma unroll
      for (int pair = 0; pair < kPairs; ++pair) {
        const int half = pair / kDims, kk = pair % kDims;
        if (pair + 2 < kPairs) read_keys(pair + 2);
        else { read_values(2 * (pair + 2 - kPairs)); read_values(2 * (pair + 2 - kPairs) + 1); }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
          for (int cb = 0; cb < CB; ++cb) {
            f32x4& x = s[2 * half + e][cb];
            x = mfma(kf[pair][e], q[cb][kk], kk == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : x);
            if (half == 1) numerators(0, kEach * (4 * kk + 2 * e + cb));
            __builtin_amdgcn_sched_barrier(0);
          }
      }
      pack(0);
#pragma unroll
      for (int f = 0; f < 2 * kBlocks; ++f) {
        const int half = f / kBlocks, db = f % kBlocks;
        if (f == kBlocks) pack(1);
        if (f + kAhead < 2 * kBlocks) read_values(f + kAhead);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) {
          o[cb][db] = mfma(vf[f], pb[half][cb], o[cb][db]);
          if (half == 0) numerators(1, kEach * (2 * db + cb));
          __builtin_amdgcn_sched_barrier(0);
        }
      }
#pragma unroll
      for (int cb = 0; cb < CB; ++cb) asm volatile("" : "+v"(sum[cb]));      // (added up where the numerators are made)
      meet();
    };
    // Behind a run of fast tiles with these sums: references that have to move do.
    auto settle = [&](const float (&sum)[CB]) {
      bool moves = false;
#pragma unroll
      for (int cb = 0; cb < CB; ++cb) {
        l[cb] += sum[cb];
        moves |= !(sum[cb] <= kMove);
      }
      if (__builtin_amdgcn_ballot_w64(moves) == 0) return;
#pragma unroll
      for (int cb = 0; cb < CB; ++cb) {
        const float most = column_max(sum[cb]);
        fits &= !(__builtin_amdgcn_ballot_w64(!(sum[cb] <= kMost)) != 0);
        const int up = most > kMove && most < INFINITY ? __builtin_amdgcn_frexp_expf(most) : 0;
        const float alpha = __builtin_amdgcn_ldexpf(1.0f, -up);
        m[cb] += (float)up;
        l[cb] *= alpha;
#pragma unroll
        for (int db = 0; db < D / 16; ++db)
#pragma unroll
          for (int i = 0; i < 4; ++i) o[cb][db][i] *= alpha;
      }
    };
    fetch(from, ka, va);
    rows(lim, lim_all);
    meet();
    const int full = fast ? min(to, lim_all / kWideKeys) : from;
    int t = from;
    if (t < full) {
#pragma unroll
      for (int cb = 0; cb < CB; ++cb) {
        float top = -INFINITY;
#pragma unroll
        for (int kb = 0; kb < (__is_same(E, __bf16) ? 1 : 4); ++kb) {
          f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int kk = 0; kk < D / 32; ++kk) s = mfma(*reinterpret_cast<const x8*>(ka + 16 * kb * 2 * D + (at<D>(mm, g) ^ (kk << 6))), q[cb][kk], s);
          top = fmaxf(top, fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3])));
        }
        top = column_max(top) * c2;
        const float first = m[cb] == -INFINITY ? top : m[cb];   // (a second cache goes on with the first one's, a second attempt with those that the first found)
        m[cb] = first;
        fits &= __builtin_amdgcn_ballot_w64(!(fabsf(first) < INFINITY)) == 0;
      }
    }
    for (; t + 1 < full; t += 2) {                         // (one place for moving: two made the compiler copy all accumulators once a tile)
      float sum[CB] = {};
      fast_tile(t, ka, va, kb_, vb, sum);
      fast_tile(t + 1, kb_, vb, ka, va, sum);
      settle(sum);
    }
    if (t < full) {
      float sum[CB] = {};
      fast_tile(t, ka, va, kb_, vb, sum);
      settle(sum);
    }
    for (t = max(from, full); t < to; ++t) {
      const bool odd = (t - from) & 1;
      any_tile(t, odd ? kb_ : ka, odd ? vb : va, odd ? ka : kb_, odd ? va : vb);
    }
    // (values near the end of the 32-bit range, times numerators far above 1)
    float rest = 0.f;
#pragma unroll
    for (int cb = 0; cb < CB; ++cb)
#pragma unroll
      for (int db = 0; db < D / 16; ++db)
#pragma unroll
        for (int i = 0; i < 4; ++i) rest = fmaf(o[cb][db][i], 0.f, rest);
    return fits && __builtin_amdgcn_ballot_w64(!(rest == 0.f)) == 0;
  }
};

// Joins softmax states: weights of the parts relative to their common reference.
__device__ __forceinline__ float part_weight(float m, float top) { return exp2_(m - (top == -INFINITY ? 0.f : top)); }
__device__ __forceinline__ float natural_lse(float top, float sum) {
  // sum == 0: nothing was seen (a NaN sum goes on as NaN)
  return sum == 0.f ? -INFINITY : ((top == -INFINITY ? 0.f : top) + __builtin_amdgcn_logf(sum)) * kLn2;
}

// kWideS, kWideO: shared / own row blocks are walked 128 rows at a time, else 16.  Both kinds of block in one launch: the long
// shared ones first.
template <class E, int D>
struct Block {
  Rows rows;
  int rb, part;
  bool shared;

  float* acc;                      // the part's states of the block's rows (null: nothing is joined, results are written)
  float2* ml;

  // [part][cache, KV head][row], behind them [part][cache, sequence, KV head][row].
  __device__ __forceinline__ void find_states(const DecodeArgs& a, int rows_block) {
    const int64_t unit = shared ? (int64_t)rows.z * a.Hkv + rows.g : ((int64_t)rows.z * a.B + rows.b) * a.Hkv + rows.g;
    const int64_t i = (shared ? part : a.splits_s + part) * a.rows + unit * rows.count + rows_block * rb;
    acc = a.part_acc ? a.part_acc + i * D : nullptr;
    ml = a.part_ml + i;
  }
  // Part or result of the narrow block's row i, of which the thread holds D / 16 dims.
  __device__ __forceinline__ void write(int i, int d0, const float (&x)[D / 16], float top, float sum, bool first) const {
    if (acc) {
      float* p = acc + i * D + d0;
#pragma unroll
      for (int d = 0; d < D / 16; d += 4) *reinterpret_cast<f32x4*>(p + d) = f32x4{x[d], x[d + 1], x[d + 2], x[d + 3]};
      if (first) ml[i] = float2{top, sum};
    } else {
      const DecodeArgs& a = kernel_args<DecodeArgs>();
      int b, h, t;
      rows.find(a, kNarrowRows * rb + i, b, h, t);
      const int z = rows.z;
      const float inv = sum == 0.f ? 0.f : 1.0f / sum;
      uint32_t* o = reinterpret_cast<uint32_t*>(static_cast<E*>(a.O) + z * a.os[0] + b * a.os[1] + h * a.os[2] + t * a.os[3] + d0);
#pragma unroll
      for (int d = 0; d < D / 16; d += 2) o[d / 2] = pack2<E>(x[d] * inv, x[d + 1] * inv);
      if (a.lse && first) a.lse[(((int64_t)z * a.B + b) * a.H + h) * a.T + t] = natural_lse(top, sum);
    }
  }

  // Loads the query rows from r0 on into the columns of `w`; tokens of the rows.
  template <int CB>
  __device__ __forceinline__ void load(Walk<E, D, CB>& w, int r0, int (&t_of)[CB], int lane) const {
    const DecodeArgs& a = kernel_args<DecodeArgs>();
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
      int b, h;
      rows.find(a, min(r0 + 16 * cb + (lane & 15), rows.count - 1), b, h, t_of[cb]);
      const E* q = static_cast<const E*>(a.Q) + rows.z * a.qs[0] + b * a.qs[1] + h * a.qs[2] + t_of[cb] * a.qs[3];
#pragma unroll
      for (int kk = 0; kk < D / 32; ++kk) w.q[cb][kk] = *reinterpret_cast<const typename Vec<E>::x8*>(q + 32 * kk + 8 * (lane >> 4));
    }
  }

  __device__ __forceinline__ int first_cache() const { return shared || kernel_args<DecodeArgs>().direct ? 0 : 1; }
  // The cache that the block walks (own: its sequence's), and this part's tiles of `keys` rows.
  struct Cache {
    const E *K, *V;
    int64_t kst, vst;
    int len, from, to;
    float c2;
  };
  __device__ __forceinline__ Cache cache(bool own, int keys) const {
    const DecodeArgs& a = kernel_args<DecodeArgs>();
    const int z = rows.z, hk = rows.g, b = rows.b;
    Cache c;
    c.c2 = a.c2;
    if (own) {
      c.K = static_cast<const E*>(a.oK) + z * a.oks[0] + b * a.oks[1] + hk * a.oks[2];
      c.V = static_cast<const E*>(a.oV) + z * a.ovs[0] + b * a.ovs[1] + hk * a.ovs[2];
      c.kst = a.oks[3]; c.vst = a.ovs[3];
      c.len = filled(a.own_lens, z * a.B + b, a.Lo);
    } else {
      c.K = static_cast<const E*>(a.K) + z * a.ks[0] + hk * a.ks[1];
      c.V = static_cast<const E*>(a.V) + z * a.vs[0] + hk * a.vs[1];
      c.kst = a.ks[2]; c.vst = a.vs[2];
      c.len = filled(a.lens, z, a.L);
    }
    // as many tiles a part, or one more in the first ones
    int more, tiles = (c.len + keys - 1) / keys;
    if (a.direct) {
      c.from = 0;
    } else {
      tiles = (own ? a.by_splits_o : a.by_splits_s).by(tiles, more);
      c.from = part * tiles + min(part, more);
      tiles += part < more;
    }
    c.to = c.from + tiles;
    return c;
  }
  // Rows that query token t_of[cb] sees, and those that all of the block's rows do: its first one's.
  template <int CB>
  __device__ __forceinline__ void limits(const Cache& c, bool own, int rows_block, const int (&t_of)[CB], int (&lim)[CB], int& lim_all) const {
    lim_all = c.len;
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) lim[cb] = c.len;
    if (!own) return;
    const DecodeArgs& a = kernel_args<DecodeArgs>();
    int rest;
    const int T = a.T, t = a.by_G.by(rows_block * rb, rest);
    lim_all = min(max(c.len - T + t + 1, 0), c.len);
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) lim[cb] = min(max(c.len - T + t_of[cb] + 1, 0), c.len);
  }
};

// `area(v)`: 32 x D elements of LDS for wavefront v.
template <class E, int D, int NW, class F>
__device__ __forceinline__ void narrow_block(const Block<E, D>& k, F area, float2 (*ml)[16], int tid) {
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), mm = lane & 15, g = lane >> 4;
  Walk<E, D, 1> w;
  w.start();
  int t_of[1];
  bool loaded = false;
  // the shared rows, the sequence's own, or both
#pragma unroll 1
  for (int own = k.first_cache(); own < (k.shared ? 1 : 2); ++own) {
    const auto c = k.cache(own, kKeys);
    w.narrow(c.K, c.V, c.kst, c.vst, c.len, c.from + wave, c.to, NW, c.c2, area(wave), lane, [&](int (&lim)[1], int& lim_all) {
      if (!loaded) k.load(w, kNarrowRows * k.rb, t_of, lane);
      loaded = true;
      k.limits(c, own, kNarrowRows, t_of, lim, lim_all);
    });
  }
  // join the wavefronts: 16 rows x D in 32 bits fill a wavefront's area; the 16-byte pieces of row r sit at piece ^ r
  __syncthreads();
  const float l = column_sum(w.l[0]);
#pragma unroll
  for (int db = 0; db < D / 16; ++db) *reinterpret_cast<f32x4*>(area(wave) + mm * (4 * D) + (((4 * db + g) ^ mm) << 4)) = w.o[0][db];
  if (g == 0) ml[wave][mm] = float2{w.m[0], l};
  __syncthreads();
  const int i = tid >> 4, d0 = (tid & 15) * (D / 16);
  if (i >= min(kNarrowRows, k.rows.count - kNarrowRows * k.rb)) return;
  float top = -INFINITY, sum = 0.f, acc[D / 16];
#pragma unroll
  for (int v = 0; v < NW; ++v) top = fmaxf(top, ml[v][i].x);
#pragma unroll
  for (int d = 0; d < D / 16; ++d) acc[d] = 0.f;
#pragma unroll
  for (int v = 0; v < NW; ++v) {
    const float f = part_weight(ml[v][i].x, top);
    sum = fmaf(f, ml[v][i].y, sum);
#pragma unroll
    for (int d = 0; d < D / 16; d += 4) {
      const f32x4 x = *reinterpret_cast<const f32x4*>(area(v) + i * (4 * D) + ((((d0 + d) / 4) ^ i) << 4));
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[d + j] = fmaf(f, x[j], acc[d + j]);
    }
  }
  k.write(i, d0, acc, top, sum, (tid & 15) == 0);
}

template <class E, int D>
__device__ __forceinline__ void wide_block(const Block<E, D>& k, unsigned char* ka, unsigned char* kb, unsigned char* va, unsigned char* vb, int tid) {
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), mm = lane & 15, g = lane >> 4;
  const int r0 = kWideRows * k.rb + 32 * wave;
  Walk<E, D, 2> w;
  int t_of[2];
  bool loaded = false;
#pragma unroll 1
  for (int attempt = 0;; ++attempt) {                      // fast, fast with the references that the first attempt found, not fast
    w.start(attempt == 1);
    bool fits = true;
#pragma unroll 1
    for (int own = k.first_cache(); own < (k.shared ? 1 : 2); ++own) {
      const auto c = k.cache(own, kWideKeys);
      fits &= w.wide(c.K, c.V, c.kst, c.vst, c.len, c.from, c.to, c.c2, ka, kb, va, vb, wave, lane, attempt < 2, [&](int (&lim)[2], int& lim_all) {
        if (!loaded) k.load(w, r0, t_of, lane);
        loaded = true;
        k.limits(c, own, kWideRows, t_of, lim, lim_all);
      });
    }
    if (attempt == 2 || !__syncthreads_or(!fits)) break;
  }
  // O^T to rows: lane l's piece of row l % 16 is dims 16 * db + 4 * g .. + 3
#pragma unroll
  for (int cb = 0; cb < 2; ++cb) {
    const float sum = column_sum(w.l[cb]);
    const int r = r0 + 16 * cb + mm;
    if (r >= k.rows.count) continue;
    if (k.acc) {
      const uint32_t i = 32 * wave + 16 * cb + mm;
      float* p = k.acc + (i * D + 4 * g);
#pragma unroll
      for (int db = 0; db < D / 16; ++db) *reinterpret_cast<f32x4*>(p + 16 * db) = w.o[cb][db];
      if (g == 0) k.ml[i] = float2{w.m[cb], sum};
    } else {
      const DecodeArgs& a = kernel_args<DecodeArgs>();
      int b, h, t;
      k.rows.find(a, r, b, h, t);
      const int z = k.rows.z;
      const float inv = sum == 0.f ? 0.f : 1.0f / sum;
      E* o = static_cast<E*>(a.O) + z * a.os[0] + b * a.os[1] + h * a.os[2] + t * a.os[3] + 4 * g;
#pragma unroll
      for (int db = 0; db < D / 16; ++db) {
        const f32x4 x = w.o[cb][db];
        *reinterpret_cast<u32x2*>(o + 16 * db) = u32x2{pack2<E>(x[0] * inv, x[1] * inv), pack2<E>(x[2] * inv, x[3] * inv)};
      }
      if (a.lse && g == 0) a.lse[(((int64_t)z * a.B + b) * a.H + h) * a.T + t] = natural_lse(w.m[cb], sum);
    }
  }
}

// kNW: wavefronts of a workgroup (kWaves with wide blocks).
template <class E, int D, bool kWideS, bool kWideO, int kNW>
__global__ __launch_bounds__(64 * kNW, kWideS ? 2 : 1) void decode_kernel(const DecodeArgs) {
  static_assert(kNW == kWaves || !kWideS);
  touch_args<DecodeArgs>();
  const DecodeArgs& a = kernel_args<DecodeArgs>();
  const int tid = threadIdx.x;
  // block id -> shared units (cache, KV head, part) x row blocks, then own units (.., sequence, part) x row blocks.  Row blocks of a unit
  // read the same keys: they are given ids 8 apart, which land on one XCD at about the same time.
  int id = blockIdx.x, in_turn;
  Block<E, D> k;
  k.shared = id < a.ids_s;
  if (!k.shared) id -= a.ids_s;
  const int turn = (k.shared ? a.by_blocks_s : a.by_blocks_o).by(id, in_turn);
  k.rb = in_turn / 8;
  int unit = turn * 8 + in_turn % 8;
  if (unit >= (k.shared ? a.units_s : a.units_o)) return;  // an id that only rounds the grid up
  unit = a.by_Hkv.by(unit, k.rows.g);
  k.rows.b = -1;
  if (!k.shared) unit = a.by_B.by(unit, k.rows.b);
  k.part = a.by_Z.by(unit, k.rows.z);
  k.rows.count = (k.shared ? a.B : 1) * a.T * a.G;
  k.find_states(a, (k.shared ? kWideS : kWideO) ? kWideRows : kNarrowRows);

  constexpr int kTile = kKeys * D * 2, kWideTile = kWideKeys * D * 2;
  __shared__ float2 ml[kNW][16];
  if constexpr (!kWideS && !kWideO) {
    __shared__ __attribute__((aligned(256))) unsigned char smem[kNW * kTile];
    narrow_block<E, D, kNW>(k, [&](int v) { return smem + v * kTile; }, ml, tid);
  } else {
    __shared__ __attribute__((aligned(256))) unsigned char ka[kWideTile], kb[kWideTile], va[kWideTile], vb[kWideTile];
    if (kWideO || k.shared) wide_block(k, ka, kb, va, vb, tid);
    else narrow_block<E, D, kNW>(k, [&](int v) { return (v < 2 ? ka : kb) + (v & 1) * kTile; }, ml, tid);
  }
}

// Joins the parts of a row: D/4 threads x `lanes` part lanes a row.
template <class E, int D>
__global__ __launch_bounds__(256) void decode_join_kernel(const DecodeArgs a, int parts, int lanes) {
  constexpr int kQuads = D / 4, kBatch = 4;
  __shared__ f32x4 acc_s[256];
  __shared__ float2 ml_s[256];
  const int64_t all_rows = (int64_t)a.Z * a.B * a.H * a.T;
  const int per_row = kQuads * lanes, tid = threadIdx.x;
  const int64_t row = (int64_t)blockIdx.x * (256 / per_row) + tid / per_row;
  const int pl = tid % per_row / kQuads, quad = tid % kQuads;
  const bool live = row < all_rows;
  int t, h, b, in_group;
  const int z = a.by_B.by(a.by_H.by(a.by_T.by((int)row, t), h), b), hk = a.by_G.by(h, in_group);
  // the row in a shared part, and in one of its sequence's (Block::find_states)
  const int64_t row_s = ((int64_t)z * a.Hkv + hk) * (a.B * a.T * a.G) + (t * a.B + b) * a.G + in_group;
  const int64_t row_o = (((int64_t)z * a.B + b) * a.Hkv + hk) * (a.T * a.G) + t * a.G + in_group;
  float top = -INFINITY, sum = 0.f;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  if (live) {
#pragma unroll 1
    for (int p0 = pl; p0 < parts; p0 += kBatch * lanes) {  // their loads in flight together
      float2 s[kBatch];
      f32x4 v[kBatch];
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        const int p = min(p0 + j * lanes, parts - 1);
        const int64_t i = p * all_rows + (p < a.splits_s ? row_s : row_o);
        s[j] = a.part_ml[i];
        v[j] = *reinterpret_cast<const f32x4*>(a.part_acc + i * D + 4 * quad);
      }
      float next = top;
#pragma unroll
      for (int j = 0; j < kBatch; ++j) next = fmaxf(next, s[j].x);
      const float f0 = part_weight(top, next);
      top = next;
      sum *= f0;
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[i] *= f0;
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        if (p0 + j * lanes < parts) {
          const float f = part_weight(s[j].x, top);
          sum = fmaf(f, s[j].y, sum);
#pragma unroll
          for (int i = 0; i < 4; ++i) acc[i] = fmaf(f, v[j][i], acc[i]);
        }
      }
    }
  }
  if (lanes > 1) {
    acc_s[tid] = acc;
    ml_s[tid] = float2{top, sum};
    __syncthreads();
    if (pl != 0) return;
#pragma unroll 1
    for (int p = 1; p < lanes; ++p) top = fmaxf(top, ml_s[tid + p * kQuads].x);
    sum = 0.f;
    acc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
    for (int p = 0; p < lanes; ++p) {
      const float f = part_weight(ml_s[tid + p * kQuads].x, top);
      sum = fmaf(f, ml_s[tid + p * kQuads].y, sum);
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[i] = fmaf(f, acc_s[tid + p * kQuads][i], acc[i]);
    }
  }
  if (!live) return;
  const float inv = sum == 0.f ? 0.f : 1.0f / sum;
  E* o = static_cast<E*>(a.O) + z * a.os[0] + b * a.os[1] + h * a.os[2] + t * a.os[3] + 4 * quad;
  *reinterpret_cast<u32x2*>(o) = u32x2{pack2<E>(acc[0] * inv, acc[1] * inv), pack2<E>(acc[2] * inv, acc[3] * inv)};
  if (a.lse && quad == 0) a.lse[row] = natural_lse(top, sum);
}

struct Shape {
  bool wide_s, wide_o, direct;
  int blocks_s, splits_s, blocks_o, splits_o;
  int parts() const { return splits_s + splits_o; }
};

// How the call's keys are dealt out.  (Host; a rule on the sizes the memory was laid out for, since the lengths may live on the device.)
Shape shape_of(const DecodeArgs& a) {
  Shape s{};
  const int64_t rows_o = (int64_t)a.T * a.G, rows_s = a.B * rows_o, heads = (int64_t)a.Z * a.Hkv;
  // Few keys: a workgroup takes a sequence through both caches and nothing has to be joined.  Not where many sequences, more than there is room
  // for at once, would read the same keys (35 sequences on each of 5 caches of 444 keys 55 us, so 79; 64 caches of 4 sequences 58 and 47).
  const bool many = heads * a.B > 2 * kCus && rows_s > 2 * kNarrowRows && a.L > 64;
  s.direct = a.L == 0 || (a.L + a.Lo <= 512 && !many);
  // A sequence's rows are up to three narrow blocks (20 rows on 976 + 13 keys of 45 x 5 sequences 75 us, a wide block 93; 35 on 602 + 43 of 55 x 3 82 and
  // 105; 64 on 4096 46 and 43), two where nothing is joined (35 on 235 keys 81 and 67).
  s.wide_o = rows_o > (s.direct ? 2 : 3) * kNarrowRows;
  // Up to 32 shared rows are two narrow blocks: on 32K keys of 8 heads 36 us, a wide one 40, of whose wavefronts one has rows (64 rows: 52 and 43).
  s.wide_s = s.wide_o || (rows_s > 2 * kNarrowRows && !s.direct);
  const int rows_wg_s = s.wide_s ? kWideRows : kNarrowRows, rows_wg_o = s.wide_o ? kWideRows : kNarrowRows;
  s.blocks_s = (int)((rows_s + rows_wg_s - 1) / rows_wg_s);
  s.blocks_o = (int)((rows_o + rows_wg_o - 1) / rows_wg_o);
  const int64_t units_s = heads * s.blocks_s, units_o = heads * a.B * s.blocks_o;
  if (s.direct && (a.L > 0 || units_o >= kCus || a.Lo <= 512)) {
    s.splits_s = 0;
    s.splits_o = 1;
    return s;
  }
  s.direct = false;
  // One round of workgroups with the same number of keys each, 128 at least: every part more has to be written and joined.
  const int64_t keys_s = units_s * a.L, keys_o = units_o * a.Lo;
  auto split = [](int64_t len, int64_t keys) { return (int)(len == 0 ? 0 : len / (keys > 128 ? keys : 128) > 1 ? len / (keys > 128 ? keys : 128) : 1); };
  if (!s.wide_s) {
    // One of eight wavefronts a CU: 128 KB on their way are enough (one sequence on 32K keys 30.5 us, two such workgroups a CU 34.4, three of
    // four wavefronts 33.1).
    s.splits_s = split(a.L, (keys_s + keys_o) / kCus);
    s.splits_o = split(a.Lo, (keys_s + keys_o) / kCus);
    return s;
  }
  // Wide blocks: one a CU, and two only where several row blocks share keys, so that the matrix cores are what they wait for, and there are
  // many of them (32 sequences on 16K keys 24 us, with two 33; 64 on 16K 32 and 38, on 128K 183 and 164).
  const int64_t keys_w = keys_s + (s.wide_o ? keys_o : 0);
  const bool two = (a.L ? s.blocks_s : s.blocks_o) > 1 && keys_w > kCus * 1536;
  // Narrow own blocks beside them wait for memory alone: they take the room that is left beside one, and beside two count half (64 sequences
  // on 128K keys and up to 1024 of their own 171 us, else 177; 200 on 16K and 800 116 and 137).
  const int64_t beside = s.wide_o ? 0 : keys_o;
  const int64_t keys = two ? (keys_w + beside / 2) / (2 * kCus) : keys_w / kCus;
  s.splits_s = split(a.L, keys);
  s.splits_o = split(a.Lo, two || s.wide_o ? keys : (keys_w + beside) / (2 * kCus));
  return s;
}

template <class E, int D>
hipError_t launch(DecodeArgs a, const Shape& s, hipStream_t stream) {
  const int64_t all_rows = (int64_t)a.Z * a.B * a.H * a.T;
  const int64_t units_s = (int64_t)a.Z * a.Hkv * s.splits_s, units_o = (int64_t)a.Z * a.Hkv * a.B * s.splits_o;
  const int64_t ids_s = (units_s + 7) / 8 * 8 * s.blocks_s, ids_o = (units_o + 7) / 8 * 8 * s.blocks_o;
  int lanes = 1;
  while (lanes < 1024 / D && lanes * 2 <= s.parts()) lanes *= 2;
  const int64_t per = 256 / (D / 4 * lanes), joins = (all_rows + per - 1) / per;
  if (!fits_launch(ids_s + ids_o, 64 * kSplitWaves) || (s.parts() > 1 && !fits_launch(joins, 256))) return hipErrorNotSupported;
  a.rows = all_rows;
  a.units_s = (int)units_s; a.units_o = (int)units_o; a.ids_s = (int)ids_s;
  a.by_blocks_s = Divisor(8 * s.blocks_s); a.by_blocks_o = Divisor(8 * s.blocks_o);
  a.by_splits_s = Divisor(s.splits_s); a.by_splits_o = Divisor(s.splits_o);
  a.by_Z = Divisor(a.Z); a.by_B = Divisor(a.B); a.by_H = Divisor(a.H); a.by_Hkv = Divisor(a.Hkv);
  a.by_G = Divisor(a.G); a.by_BG = Divisor(a.B * a.G); a.by_T = Divisor(a.T);
  if (s.parts() == 1) a.part_acc = nullptr;                // nothing to join
  const dim3 grid((unsigned)(ids_s + ids_o)), threads(kThreads);
  if (s.wide_o) hipLaunchKernelGGL((decode_kernel<E, D, true, true, kWaves>), grid, threads, 0, stream, a);
  else if (s.wide_s) hipLaunchKernelGGL((decode_kernel<E, D, true, false, kWaves>), grid, threads, 0, stream, a);
  else if (s.direct) hipLaunchKernelGGL((decode_kernel<E, D, false, false, kWaves>), grid, threads, 0, stream, a);
  else hipLaunchKernelGGL((decode_kernel<E, D, false, false, kSplitWaves>), grid, dim3(64 * kSplitWaves), 0, stream, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !a.part_acc) return e;
  hipLaunchKernelGGL((decode_join_kernel<E, D>), dim3((unsigned)joins), dim3(256), 0, stream, a, s.parts(), lanes);
  return hipGetLastError();
}

}  // namespace

size_t decode_scratch_bytes(const DecodeArgs& a) {
  const Shape s = shape_of(a);
  if (s.parts() == 1) return 0;
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
