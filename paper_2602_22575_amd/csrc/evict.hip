// Eviction from a cache by accumulated attention weight, for gfx950: of n rows the first `sink`, the last `recent` and, of those
// between, the ones of the largest weights stay (ties: the lowest index), in their order, moved together.
//
// Weights are ranked by an unsigned key that orders like the float (-0 as +0, NaN as -inf).  What stays is the rows above the key of the
// last one, and of those that share it the first few.
//   select_kernel  up to 20K rows, a workgroup per (cache, KV head): all keys, and counts of 11, 11 and 10 of their bits, in LDS
//   count_kernel, collect_kernel, list_kernel    more rows, a workgroup per stretch of 4096 or more: count the keys' upper 11 bits; collect
//                  the other 21 bits of the rows that share the last one's; settle them (every workgroup for itself, from LDS where they
//                  fit) and list.  Nothing is added up by atomics in memory, so that nothing has to be cleared.  Three passes over the weights by
//                  all of the chip, 4, 7 and 10 us for 8 heads of 128K rows (one workgroup a head: 102, the instructions of one CU).
// gather_kernel copies the listed rows of K and V and their weights.  Bound: HBM bandwidth of the copy, 26 to 29 us for 134 MB, 4.6 to 5.1 TB/s.
// select_kernel is bound by one CU's dependent passes: 17 us for 20K rows, of which reading and the first count take 4, the two other
// counts 5, listing 3.
#include "cache_tile.h"
#include "s2o_internal.h"

namespace s2o {

namespace {

using namespace cache;

// larger key = stays longer
__device__ __forceinline__ uint32_t rank_key(float w) {
  if (w != w) w = -INFINITY;
  const uint32_t b = __float_as_uint(w + 0.0f);          // -0 + 0 = +0
  return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}

// The rows lo .. hi - 1 of n compete for `want` places, the others stay; `stay` in all.
struct Places {
  int n, stay, lo, hi, want;
  __device__ __forceinline__ Places(const EvictArgs& a, int z) {
    n = filled(a.lens, z, a.L);
    stay = min(n, a.keep);
    lo = min(a.sink, n);
    hi = max(lo, n - a.recent);
    want = stay - (n - (hi - lo));
  }
  __device__ __forceinline__ bool choose() const { return want > 0 && want < hi - lo; }   // else none of them stays, or all do
};

constexpr int kT = 1024, kWaves = kT / 64;
constexpr int kOneGroup = 20 * kT;  // rows that select_kernel takes (8 heads of 16K rows 22 us, of 24K 29; by stretches 24 and 27)
constexpr int kBlock = 4 * kT;      // rows that a workgroup looks at at once, four in a row a thread
constexpr int kStretches = 64;      // a head's rows are cut into, as far as a stretch has no more than kMostBlocks blocks
constexpr int kMostBlocks = 15;     // (its counts have 16 bits)
constexpr int kBins = 2048;
constexpr int kRoom = 16384;        // entries that list_kernel keeps in LDS

// Sums over the lanes up to and with this one: 16 lanes by shifts, then the rows' last lanes passed on.
__device__ __forceinline__ int wave_scan(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);   // row_shr:1, 2, 4, 8
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);   // row_bcast:15 into rows 1 and 3
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);   // row_bcast:31 into rows 2 and 3
  return x;
}

// Sums over the threads in front of this one, and over all, of two numbers.  `part`: a pair a wavefront.  (A barrier in front: `part` may be
// in use.)
struct Sums { int a, b, all_a, all_b; };
__device__ __forceinline__ Sums block_scan(int a, int b, int2* part, int tid) {
  const int sa = wave_scan(a), sb = wave_scan(b);
  __syncthreads();
  if ((tid & 63) == 63) part[tid >> 6] = int2{sa, sb};
  __syncthreads();
  Sums s{sa - a, sb - b, 0, 0};
#pragma unroll
  for (int v = 0; v < kWaves; ++v) {
    const int2 x = part[v];
    if (v < tid >> 6) { s.a += x.x; s.b += x.y; }
    s.all_a += x.x;
    s.all_b += x.y;
  }
  return s;
}

// The bin of the want-th largest (1 <= want <= the counts' sum), how many it holds, and how many lie in larger bins.  Bins are dealt out from
// the largest down, two a thread: c, with `tag` to be had back of the bin that is found.
constexpr int bins_of(int tid) { return kBins - 2 - 2 * tid; }
struct Bin { int bin, holds, above, tag; };
__device__ __forceinline__ Bin find_bin(uint2 c, uint2 tag, int2* part, Bin* found, int want, int tid) {
  static_assert(kBins == 2 * kT, "two bins a thread");
  const int b = bins_of(tid);
  const int own = (int)(c.x + c.y), before = block_scan(own, 0, part, tid).a;
  if (before < want && before + own >= want) {
    const bool upper = before + (int)c.y >= want;
    *found = upper ? Bin{b + 1, (int)c.y, before, (int)tag.y} : Bin{b, (int)c.x, before + (int)c.y, (int)tag.x};
  }
  __syncthreads();
  return *found;
}
__device__ __forceinline__ Bin find_bin(const uint32_t* counts, int2* part, Bin* found, int want, int tid) {
  return find_bin(*reinterpret_cast<const uint2*>(counts + bins_of(tid)), uint2{0, 0}, part, found, want, tid);
}

__host__ __device__ inline int stretch_rows(int L) {
  const int64_t blocks = ((int64_t)L + (int64_t)kStretches * kBlock - 1) / ((int64_t)kStretches * kBlock);
  return kBlock * (int)(blocks < kMostBlocks ? blocks : kMostBlocks);
}
__host__ __device__ inline int stretches(int L) { return (L + stretch_rows(L) - 1) / stretch_rows(L); }

// The scratch words of a head: counts of its stretches, then what the kernels hand on, then entries.
struct Scratch {
  uint32_t* counts;    // [stretches][kBins / 2]: pairs of counts of the keys' upper 11 bits
  uint32_t* known;     // [0]: those of the last row that stays, [1]: places for the rows that share them, [2]: how many do
  uint32_t* above;     // [stretches] rows of larger upper bits
  uint32_t* first;     // [stretches] rows in front of the stretch that share them
  uint32_t* entries;   // the other 21 bits of those that do, stretch after stretch
  static __host__ __device__ size_t list_words(int L) { return (size_t)(stretches(L) + 63) / 64 * 64; }
  static __host__ __device__ size_t words(int L) { return (size_t)stretches(L) * (kBins / 2) + 64 + 2 * list_words(L) + ((size_t)L + 63) / 64 * 64; }
  __device__ __forceinline__ Scratch(const EvictArgs& a, int64_t head) {
    counts = a.scratch + head * (int64_t)words(a.L);
    known = counts + (size_t)stretches(a.L) * (kBins / 2);
    above = known + 64;
    first = above + list_words(a.L);
    entries = first + list_words(a.L);
  }
};

// Keys of four rows i, i + step, .. (behind the end: the last row's).  n > 0.  (Four loads without a branch rather than one with: several
// calls' are in flight together.)  Steps of 1 only where a thread needs rows in a row: it reads sixteen lines an instruction, not four.
template <int kStep>
__device__ __forceinline__ void four(const float* w, int i, int n, uint32_t (&k)[4]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) k[e] = rank_key(w[min(i + kStep * e, n - 1)]);
}

// Lists rows of a thread: from + j for the bits j of `sure`, and of `tie` those that find a place.  s, t: such rows in front of the thread's.
__device__ __forceinline__ void list_rows(int32_t* list, int from, uint64_t sure, uint64_t tie, int s, int t, int ties) {
  uint64_t left = sure | tie;
  while (left) {
    const int j = __builtin_ctzll(left);
    const int is_tie = (int)(tie >> j) & 1;
    left &= left - 1;
    if (!is_tie || t < ties) list[s + min(t, ties)] = from + j;
    s += 1 - is_tie;
    t += is_tie;
  }
}

__global__ __launch_bounds__(kT) void count_kernel(const EvictArgs a) {
  touch_args<EvictArgs>();
  __shared__ uint32_t counts[kBins];
  const int tid = threadIdx.x;
  const int stretch = (int)(blockIdx.x % stretches(a.L));
  const int64_t head = blockIdx.x / stretches(a.L);
  const Places p(a, (int)(head / a.Hkv));
  const int per = stretch_rows(a.L), from = stretch * per, to = min(p.hi, from + per);
  if (!p.choose() || from >= to) return;
  for (int i = tid; i < kBins; i += kT) counts[i] = 0;
  __syncthreads();
  const float* w = a.weights + head * a.L;
  for (int i = from + tid; i < to; i += kBlock) {
    uint32_t k[4];
    four<kT>(w, i, p.n, k);
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (i + kT * e >= p.lo && i + kT * e < to) atomicAdd(&counts[k[e] >> 21], 1u);
  }
  __syncthreads();
  const uint2 c = *reinterpret_cast<const uint2*>(counts + 2 * tid);
  Scratch(a, head).counts[(int64_t)stretch * (kBins / 2) + tid] = c.x | c.y << 16;
}

__global__ __launch_bounds__(kT) void collect_kernel(const EvictArgs a) {
  touch_args<EvictArgs>();
  __shared__ int2 part[kWaves];
  __shared__ Bin found;
  const int tid = threadIdx.x;
  const int stretch = (int)(blockIdx.x % stretches(a.L));
  const int64_t head = blockIdx.x / stretches(a.L);
  const Places p(a, (int)(head / a.Hkv));
  const int per = stretch_rows(a.L), from = stretch * per, to = min(p.hi, from + per);
  if (!p.choose() || from >= p.n) return;
  const Scratch s(a, head);
  const float* w = a.weights + head * a.L;
  uint32_t next[4];                                        // keys of the first block, on their way meanwhile
  four<kT>(w, from + tid, p.n, next);
  uint2 all = {0, 0}, front = {0, 0};                      // counts of all stretches, and of those in front
  const int counted = (p.hi + per - 1) / per;
#pragma unroll 16
  for (int i = 0; i < counted; ++i) {
    const uint32_t c = s.counts[(int64_t)i * (kBins / 2) + bins_of(tid) / 2];
    all.x += c & 0xffffu;
    all.y += c >> 16;
    front.x += i < stretch ? c & 0xffffu : 0u;
    front.y += i < stretch ? c >> 16 : 0u;
  }
  const Bin last = find_bin(all, front, part, &found, p.want, tid);
  if (stretch == 0 && tid == 0) {
    s.known[0] = (uint32_t)last.bin;
    s.known[1] = (uint32_t)(p.want - last.above);
    s.known[2] = (uint32_t)last.holds;
  }
  int above = 0, base = last.tag;
  for (int i0 = from; i0 < to; i0 += kBlock) {
    const int i = i0 + tid;
    uint32_t k[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) k[e] = next[e];
    if (i0 + kBlock < to) four<kT>(w, i + kBlock, p.n, next);
    int mine = 0, larger = 0;
    bool same[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const bool in = i + kT * e >= p.lo && i + kT * e < to;
      larger += in && (int)(k[e] >> 21) > last.bin;
      same[e] = in && (int)(k[e] >> 21) == last.bin;
      mine += same[e];
    }
    const Sums sums = block_scan(mine, larger, part, tid);
    above += sums.all_b;
    int at = base + sums.a;
    base += sums.all_a;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (same[e]) s.entries[at++] = k[e] & 0x1fffffu;
  }
  if (tid == 0) {
    s.above[stretch] = (uint32_t)above;
    s.first[stretch] = (uint32_t)last.tag;
  }
}

__global__ __launch_bounds__(kT) void list_kernel(const EvictArgs a) {
  touch_args<EvictArgs>();
  __shared__ uint32_t counts[kBins], room[kRoom];
  __shared__ int2 part[kWaves];
  __shared__ Bin found;
  const int tid = threadIdx.x;
  const int stretch = (int)(blockIdx.x % stretches(a.L));
  const int64_t head = blockIdx.x / stretches(a.L);
  const Places p(a, (int)(head / a.Hkv));
  const int per = stretch_rows(a.L), from = stretch * per, to = min(p.n, from + per);
  if (a.lens_out && stretch == 0 && head % a.Hkv == 0 && tid == 0) a.lens_out[head / a.Hkv] = p.stay;
  if (from >= to) return;
  const Scratch s(a, head);
  const bool choose = p.choose(), all = !choose && p.want > 0;
  const float* w = a.weights + head * a.L;
  uint32_t next[4];
  four<1>(w, from + 4 * tid, p.n, next);
  uint32_t key = 0;
  int ties = 0, kept_before = all ? from : min(p.lo, from) + max(0, from - p.hi), tied_before = 0;
  if (choose) {
    const int used = (int)s.known[2], here = min(used, kRoom), first = (int)s.first[stretch];
    key = s.known[0] << 21;
    ties = (int)s.known[1];
    int kept = 0, tied = 0;
    for (int i = tid; i < stretch; i += kT) kept += (int)s.above[i];
#pragma unroll 4
    for (int i = tid; i < here; i += kT) room[i] = s.entries[i];
    auto each = [&](auto f) {
#pragma unroll 1
      for (int i = tid; i < here; i += kT) f(room[i], i);
#pragma unroll 1
      for (int i = kRoom + tid; i < used; i += kT) f(s.entries[i], i);
    };
    // 11 and 10 bits more
#pragma unroll 1
    for (int shift = 10; shift >= 0; shift -= 10) {
      const uint32_t known = shift == 10 ? 21 : 10, mask = shift == 10 ? 2047 : 1023;
      __syncthreads();
      for (int i = tid; i < kBins; i += kT) counts[i] = 0;
      __syncthreads();
      each([&](uint32_t k, int) {
        if ((k >> known) == ((key & 0x1fffffu) >> known)) atomicAdd(&counts[(k >> shift) & mask], 1u);
      });
      __syncthreads();
      const Bin last = find_bin(counts, part, &found, ties, tid);
      key |= (uint32_t)last.bin << shift;
      ties -= last.above;
    }
    // what stays in front of this stretch, for certain and if there are places
    each([&](uint32_t k, int i) {
      const uint32_t last = key & 0x1fffffu;
      kept += i < first && k > last;
      tied += i < first && k == last;
    });
    const Sums sums = block_scan(kept, tied, part, tid);
    kept_before += sums.all_a;
    tied_before = sums.all_b;
  }
  for (int i0 = from; i0 < to; i0 += kBlock) {
    const int i = i0 + 4 * tid;
    uint32_t k[4], sure = 0, tie = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) k[e] = next[e];
    if (i0 + kBlock < to) four<1>(w, i + kBlock, p.n, next);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const bool competes = i + e >= p.lo && i + e < p.hi;
      if (i + e < to && (!competes || all || (choose && k[e] > key))) sure |= 1u << e;
      if (i + e < to && competes && choose && k[e] == key) tie |= 1u << e;
    }
    const Sums sums = block_scan(__popc(sure), __popc(tie), part, tid);
    list_rows(a.kept + head * a.keep, i, sure, tie, kept_before + sums.a, tied_before + sums.b, ties);
    kept_before += sums.all_a;
    tied_before += sums.all_b;
  }
}

// kRows: of a head at most; a thread holds its share of them in registers (8 heads of 12K rows 18 us, in the form for 20K 20).
template <int kRows>
__global__ __launch_bounds__(kT) void select_kernel(const EvictArgs a) {
  touch_args<EvictArgs>();
  __shared__ __attribute__((aligned(16))) uint32_t keys[kRows];   // 0: a row that does not compete (the least key is 0x7fffff)
  __shared__ uint32_t counts[kBins];
  __shared__ int2 part[kWaves];
  __shared__ Bin found;
  const int tid = threadIdx.x;
  const int64_t head = blockIdx.x;
  const Places p(a, (int)(head / a.Hkv));
  if (a.lens_out && head % a.Hkv == 0 && tid == 0) a.lens_out[head / a.Hkv] = p.stay;
  if (p.n == 0) return;
  const float* w = a.weights + head * a.L;
  const bool choose = p.choose(), all = !choose && p.want > 0;
  for (int i = tid; i < kBins; i += kT) counts[i] = 0;
  __syncthreads();
  constexpr int kFours = 2;                                // in flight together
  for (int i = tid; i < p.n; i += kFours * kBlock) {
    uint32_t k[kFours][4];
#pragma unroll
    for (int j = 0; j < kFours; ++j) four<kT>(w, i + j * kBlock, p.n, k[j]);
#pragma unroll
    for (int j = 0; j < kFours; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int at = i + j * kBlock + kT * e;
        if (at < p.lo || at >= p.hi) k[j][e] = 0;
        if (k[j][e] && choose) atomicAdd(&counts[k[j][e] >> 21], 1u);
        if (at < p.n) keys[at] = k[j][e];
      }
  }
  __syncthreads();
  // From here on a thread has a stretch of its own, in registers: an odd number of pieces of four rows, so that a wavefront's reads meet different banks.
  constexpr int kPieces = (kRows / kBlock) | 1;
  const int per = 4 * (((p.n + kBlock - 1) / kBlock) | 1), from = min(tid * per, p.n), to = min(from + per, p.n);
  u32x4 mine[kPieces];
#pragma unroll
  for (int j = 0; j < kPieces; ++j) {
    mine[j] = *reinterpret_cast<const u32x4*>(keys + min(tid * per + 4 * j, kRows - 4));
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (from + 4 * j + e >= to) mine[j][e] = 0;
  }
  uint32_t key = 0, known = 0;                             // what is known of the last row's key, from the top down
  int ties = p.want;                                       // places for the rows that share it
  if (choose) {
#pragma unroll 1
    for (int shift = 21; ; shift = shift == 21 ? 10 : 0) {
      const uint32_t mask = shift == 0 ? 1023 : 2047;
      if (shift != 21) {
        for (int i = tid; i < kBins; i += kT) counts[i] = 0;
        __syncthreads();
#pragma unroll
        for (int j = 0; j < kPieces; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (mine[j][e] && (mine[j][e] & known) == key) atomicAdd(&counts[(mine[j][e] >> shift) & mask], 1u);
        __syncthreads();
      }
      const Bin last = find_bin(counts, part, &found, ties, tid);
      key |= (uint32_t)last.bin << shift;
      known |= mask << shift;
      ties -= last.above;
      if (last.holds == ties || shift == 0) break;         // (all that share it stay)
      __syncthreads();
    }
  }
  static_assert(4 * kPieces <= 64, "a thread's rows are the bits of a word");
  uint64_t sure = 0, tie = 0;
#pragma unroll
  for (int j = 0; j < kPieces; ++j)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t k = mine[j][e];
      sure |= (uint64_t)(k == 0 || all || (choose && (k & known) > key)) << (4 * j + e);
      tie |= (uint64_t)(k != 0 && choose && (k & known) == key) << (4 * j + e);
    }
  sure &= to - from < 64 ? (1ull << (to - from)) - 1 : ~0ull;
  const Sums sums = block_scan(__popcll(sure), __popcll(tie), part, tid);
  list_rows(a.kept + head * a.keep, from, sure, tie, sums.a, sums.b, ties);
}

// Rows of 2 * D bytes, D / 8 lanes a row, kEach of them a thread; blockIdx.y: K and the weights, or V.
template <int D, int kEach>
__global__ __launch_bounds__(256) void gather_kernel(const EvictArgs a, int chunks) {
  touch_args<EvictArgs>();
  constexpr int kLanes = D / 8, kStep = 256 / kLanes;
  const int64_t head = blockIdx.x / chunks;
  const int z = (int)(head / a.Hkv), hk = (int)(head % a.Hkv), lane = threadIdx.x % kLanes;
  const int stay = min(filled(a.lens, z, a.L), a.keep);
  const int r0 = (int)(blockIdx.x % chunks) * (kStep * kEach) + threadIdx.x / kLanes;
  if (r0 >= stay) return;
  int from[kEach];
#pragma unroll
  for (int j = 0; j < kEach; ++j) from[j] = a.kept[head * a.keep + min(r0 + kStep * j, stay - 1)];
  const uint16_t* src = static_cast<const uint16_t*>(blockIdx.y ? a.V : a.K);
  if (src) {
    uint16_t* dst = static_cast<uint16_t*>(blockIdx.y ? a.V_out : a.K_out);
    const int64_t* ss = blockIdx.y ? a.vs : a.ks;
    const int64_t* ds = blockIdx.y ? a.vos : a.kos;
    src += z * ss[0] + hk * ss[1] + 8 * lane;
    dst += z * ds[0] + hk * ds[1] + 8 * lane;
    u32x4 x[kEach];
#pragma unroll
    for (int j = 0; j < kEach; ++j) x[j] = *reinterpret_cast<const u32x4*>(src + from[j] * ss[2]);
#pragma unroll
    for (int j = 0; j < kEach; ++j)
      if (r0 + kStep * j < stay) *reinterpret_cast<u32x4*>(dst + (r0 + kStep * j) * ds[2]) = x[j];
  }
  if (blockIdx.y == 0 && a.weights_out && lane < kEach) {
    int mine = from[0];
#pragma unroll
    for (int j = 1; j < kEach; ++j) mine = lane == j ? from[j] : mine;
    if (r0 + kStep * lane < stay) a.weights_out[head * a.keep + r0 + kStep * lane] = a.weights[head * a.L + mine];
  }
}

}  // namespace

size_t evict_scratch_bytes(const EvictArgs& a) {
  return a.L <= kOneGroup ? 0 : (size_t)a.Z * a.Hkv * Scratch::words(a.L) * 4;
}

hipError_t launch_evict(EvictArgs a, void* scratch, hipStream_t stream) {
  const int64_t heads = (int64_t)a.Z * a.Hkv, blocks = a.L <= kOneGroup ? heads : heads * stretches(a.L);
  constexpr int kEach = 4;
  const int rows = 2048 / a.D * kEach, chunks = (a.keep + rows - 1) / rows;
  const bool moves = a.K || a.V || a.weights_out;
  if (!fits_launch(blocks, kT) || (moves && !fits_launch(heads * chunks, 256))) return hipErrorNotSupported;
  const dim3 grid((unsigned)blocks);
  if (a.L <= 4 * kT) {
    hipLaunchKernelGGL(select_kernel<4 * kT>, grid, dim3(kT), 0, stream, a);
  } else if (a.L <= 12 * kT) {
    hipLaunchKernelGGL(select_kernel<12 * kT>, grid, dim3(kT), 0, stream, a);
  } else if (a.L <= kOneGroup) {
    hipLaunchKernelGGL(select_kernel<kOneGroup>, grid, dim3(kT), 0, stream, a);
  } else {
    a.scratch = static_cast<uint32_t*>(scratch);
    hipLaunchKernelGGL(count_kernel, grid, dim3(kT), 0, stream, a);
    hipLaunchKernelGGL(collect_kernel, grid, dim3(kT), 0, stream, a);
    hipLaunchKernelGGL(list_kernel, grid, dim3(kT), 0, stream, a);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !moves) return e;
  const dim3 gather((unsigned)(heads * chunks), a.V ? 2 : 1);
  if (a.D == 128) hipLaunchKernelGGL((gather_kernel<128, kEach>), gather, dim3(256), 0, stream, a, chunks);
  else hipLaunchKernelGGL((gather_kernel<64, kEach>), gather, dim3(256), 0, stream, a, chunks);
  return hipGetLastError();
}

}  // namespace s2o
