// Building blocks of the kernels that work on a key/value cache (decode.hip, weights.hip) for gfx950, for
// bf16 and fp16 elements and head dimensions 64 and 128.
//
// Products are v_mfma_f32_16x16x32 in the transposed form of attn_tile.h: lane l = (m = l % 16, g = l / 16) of an accumulator block
// holds in register i the element [row 4*g + i of the A side][row m of the B side]; an operand is 8 consecutive elements
// 32*kk + 8*g .. +7 of row m.  For O^T = V^T P^T the A side is read with the transposing LDS load: lane r of group g
// points at (key 4*g + r/4, dims 4*(r%4) .. +3) and gets keys 4*g .. 4*g+3 at dim r.
//
// Rows in LDS are unpadded; the 16-byte chunk c of row r sits at slot c ^ swz(r), so that the 16 rows of an operand read, and
// the 8 rows x 32 bytes that half a wavefront touches in a transposing read, land on different banks.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace s2o {
namespace cache {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef short i16x4 __attribute__((ext_vector_type(4)));

template <class E>
struct Vec {
  typedef E x8 __attribute__((ext_vector_type(8)));
  typedef E x2 __attribute__((ext_vector_type(2)));
};

__device__ __forceinline__ f32x4 mfma(const Vec<__bf16>::x8& a, const Vec<__bf16>::x8& b, const f32x4& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mfma(const Vec<_Float16>::x8& a, const Vec<_Float16>::x8& b, const f32x4& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

template <int D>
__device__ __forceinline__ int swz(int r) {
  if constexpr (D == 128) return ((r & 3) << 2) | ((((r >> 2) ^ (r >> 3)) & 1) << 1) | ((r >> 3) & 1);
  else return (((r >> 1) & 3) << 1) | ((r >> 3) & 1);
}
// Byte address of chunk c of row r in a tile of rows of D elements.  swz(r + r') = swz(r) ^ swz(r') where r and r' share no bits, so
// that addresses of one lane follow from a first one by an XOR with a constant.
template <int D>
__device__ __forceinline__ int at(int r, int c) { return r * (2 * D) + ((c ^ swz<D>(r)) << 4); }

// Rows row0 .. row0 + most - 1 of a cache of `len` rows as a buffer: loads of rows behind the cache's end give zeros and touch no
// memory.  Uniform arguments, row0 < len; `stride` in bytes, less than 2^24.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_buffer(const void* cache, int64_t stride, int row0, int len, int most, int row_bytes) {
  const char* p = static_cast<const char*>(cache) + row0 * stride;
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(p), 0, (uint32_t)(min(len - row0, most) - 1) * (uint32_t)stride + row_bytes, 0x00027000);
}
__device__ __forceinline__ u32x4 buffer_load(__amdgpu_buffer_rsrc_t b, uint32_t offset) {
  return __builtin_amdgcn_raw_buffer_load_b128(b, offset, 0, 0);
}
__device__ __forceinline__ void buffer_load_to_lds(__amdgpu_buffer_rsrc_t b, uint32_t offset, unsigned char* lds) {
  typedef __attribute__((address_space(3))) void lvoid;
  __builtin_amdgcn_raw_ptr_buffer_load_lds(b, (lvoid*)lds, 16, offset, 0, 0, 0);
}

template <class E>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  typename Vec<E>::x2 t = {(E)lo, (E)hi};
  return __builtin_bit_cast(uint32_t, t);
}

// Over the four lanes l % 16 + 16 * {0..3} that share a column of an accumulator block.
__device__ __forceinline__ float column_max(float x) {
  const u32x2 r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(r.x), __uint_as_float(r.y));
  const u32x2 q = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(q.x), __uint_as_float(q.y));
}
__device__ __forceinline__ float column_sum(float x) {
  const u32x2 r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(r.x) + __uint_as_float(r.y);
  const u32x2 q = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(q.x) + __uint_as_float(q.y);
}

// Asks for every 64-byte line of the kernel's arguments at once.
template <class A>
__device__ __forceinline__ void touch_args() {
  typedef const __attribute__((address_space(4))) volatile uint32_t* Words;
  const Words p = (Words)__builtin_amdgcn_kernarg_segment_ptr();
  uint32_t x = 0;
#pragma unroll
  for (size_t i = 0; i < sizeof(A) / 4; i += 16) x |= p[i];
  asm volatile("" ::"s"(x));
}

// The lane's number, made anew where it is asked for.
__device__ __forceinline__ int lane_id() {
  int n = __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u));
  asm volatile("" : "+v"(n));
  return n;
}

// A wavefront's own LDS writes stand before its own LDS reads: the hardware keeps their order, this keeps the compiler's.
__device__ __forceinline__ void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

// The arguments of a kernel whose one parameter is an A, to be read from here on: what a stretch of code needs of them is loaded there, and does
// not stay in scalar registers from the first stretch to the last (where they do not all fit).
template <class A>
__device__ __forceinline__ const A& kernel_args() {
  typedef const __attribute__((address_space(4))) A* Pointer;
  Pointer p = (Pointer)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  return *(const A*)p;
}

constexpr float kLn2 = 0.6931471805599453f;

// rows in a cache: what the caller says, kept inside the memory it has
__device__ __forceinline__ int filled(const int32_t* lens, int i, int most) {
  return lens ? min(max(lens[i], 0), most) : most;
}

}  // namespace cache
}  // namespace s2o
