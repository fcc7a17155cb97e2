// Device helpers shared by the attention kernels: operand types, exchanges between the lanes that share a row, conversions.
#pragma once

#include <hip/hip_runtime.h>

namespace cronus {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));

typedef __attribute__((address_space(3))) unsigned char lds_byte;

constexpr float kLazyLog2 = 8.0f;  // slack of the running reference of the online softmax, in bits
constexpr float kNeg = -1.0e30f;  // initial running maximum: finite, so that differences of maxima stay finite

// Row r of a 32-row S^T tile of v_mfma_f32_32x32x16_bf16 holds key perm32(r) of the 32-key sub-tile (bits 2 and 3
// swapped): the accumulators that a lane holds are then, in order, the 8-key chunks that the P^T operand needs.
__device__ __forceinline__ int perm32(int r) { return (r & ~12) | ((r & 4) << 1) | ((r & 8) >> 1); }

// Combine a value with the one held by lane^32 (rows of 32 lanes swapped).
__device__ __forceinline__ float pair_max(float x) {
  auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float pair_sum(float x) {
  auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

__device__ __forceinline__ bf16x8 as_bf16x8(u32x4 v) { return __builtin_bit_cast(bf16x8, v); }

__device__ __forceinline__ unsigned int pack_bf16(float a, float b) {
  f32x2 f = {a, b};
  return __builtin_bit_cast(unsigned int, __builtin_convertvector(f, bf16x2));
}

// 8 e4m3 codes -> 8 bf16 (exact: every e4m3 value is a bf16 value).
__device__ __forceinline__ u32x4 fp8x8_to_bf16x8(u32x2 c) {
  u32x4 r;
  r[0] = __builtin_bit_cast(unsigned int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[0], 1.0f, false));
  r[1] = __builtin_bit_cast(unsigned int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[0], 1.0f, true));
  r[2] = __builtin_bit_cast(unsigned int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[1], 1.0f, false));
  r[3] = __builtin_bit_cast(unsigned int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[1], 1.0f, true));
  return r;
}

// Zero the elements e of a V chunk (8 consecutive keys kv0+e) whose key is >= kv_len:
// slots past the sequence's length hold arbitrary bits and P = 0 there must give 0.
__device__ __forceinline__ u32x4 zero_tail(u32x4 v, int kv0, int kv_len) {
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    unsigned int m = 0;
    if (kv0 + 2 * w < kv_len) m |= 0x0000ffffu;
    if (kv0 + 2 * w + 1 < kv_len) m |= 0xffff0000u;
    v[w] &= m;
  }
  return v;
}

// Numerators 2^(c (s - m)) as bf16 P^T operands, and this lane's sum of them.  The sum
// adds the ROUNDED numerators (one dot product with (1, 1) per packed pair), so l
// normalises exactly the weights that multiply V.
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
__device__ __forceinline__ float softmax_exp_part(const f32x16& s, float c, float m, u32x4 (&p)[2]) {
  const float mc = m * c;
  const bf16x2_t ones = __builtin_bit_cast(bf16x2_t, 0x3f803f80u);
  float sum = 0.f;
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float e0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[8 * t + 2 * w], c, -mc));
      const float e1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[8 * t + 2 * w + 1], c, -mc));
      const f32x2 e = {e0, e1};
      const bf16x2_t pk = __builtin_convertvector(e, bf16x2_t);
      p[t][w] = __builtin_bit_cast(unsigned int, pk);
      sum = __builtin_amdgcn_fdot2_f32_bf16(pk, ones, sum, false);
    }
  return sum;
}

template <int N>
__device__ __forceinline__ void wait_vmcnt() {
  static_assert(N >= 0 && N < 64, "vmcnt is a 6-bit counter");
  asm volatile("s_waitcnt vmcnt(%0)" ::"i"(N) : "memory");
}

// LDS reads of data that arrived by global_load_lds are written as asm, so that the
// waits on those loads are the explicit vmcnt waits of the pipelines and nothing coarser
// (the compiler would wait for every DMA in flight before any LDS read).  The reads and
// the wait for them form ONE asm statement: its outputs are valid when it ends, so no
// register copy the compiler may insert afterwards can see a value that has not arrived.
template <int O0, int O1, int O2, int O3>
__device__ __forceinline__ void lds_read4(u32x4& x0, u32x4& x1, u32x4& x2, u32x4& x3, unsigned addr) {
  asm volatile(
      "ds_read_b128 %0, %4 offset:%5\n\tds_read_b128 %1, %4 offset:%6\n\t"
      "ds_read_b128 %2, %4 offset:%7\n\tds_read_b128 %3, %4 offset:%8\n\ts_waitcnt lgkmcnt(0)"
      : "=&v"(x0), "=&v"(x1), "=&v"(x2), "=&v"(x3)
      : "v"(addr), "i"(O0), "i"(O1), "i"(O2), "i"(O3)
      : "memory");
}
template <int O0, int O1, int O2, int O3, int O4, int O5, int O6, int O7>
__device__ __forceinline__ void lds_read8(u32x4 (&x)[8], unsigned addr) {
  asm volatile(
      "ds_read_b128 %0, %8 offset:%9\n\tds_read_b128 %1, %8 offset:%10\n\t"
      "ds_read_b128 %2, %8 offset:%11\n\tds_read_b128 %3, %8 offset:%12\n\t"
      "ds_read_b128 %4, %8 offset:%13\n\tds_read_b128 %5, %8 offset:%14\n\t"
      "ds_read_b128 %6, %8 offset:%15\n\tds_read_b128 %7, %8 offset:%16\n\ts_waitcnt lgkmcnt(0)"
      : "=&v"(x[0]), "=&v"(x[1]), "=&v"(x[2]), "=&v"(x[3]), "=&v"(x[4]), "=&v"(x[5]), "=&v"(x[6]), "=&v"(x[7])
      : "v"(addr), "i"(O0), "i"(O1), "i"(O2), "i"(O3), "i"(O4), "i"(O5), "i"(O6), "i"(O7)
      : "memory");
}

// Read the NOPS 1-KiB operand planes of this lane (plane n at addr + 1024 n).
template <int NOPS>
__device__ __forceinline__ void lds_read_planes(u32x4 (&x)[NOPS], unsigned addr) {
  static_assert(NOPS == 4 || NOPS == 8, "D = 64 or 128");
  if constexpr (NOPS == 8) lds_read8<0, 1024, 2048, 3072, 4096, 5120, 6144, 7168>(x, addr);
  else lds_read4<0, 1024, 2048, 3072>(x[0], x[1], x[2], x[3], addr);
}

// Operand chunks of 8 bytes picked out of a block image in LDS (fp8 codes).
template <int O0, int O1, int O2, int O3, int O4, int O5, int O6, int O7>
__device__ __forceinline__ void lds_read8_b64(u32x2 (&x)[8], unsigned addr) {
  asm volatile(
      "ds_read_b64 %0, %8 offset:%9\n\tds_read_b64 %1, %8 offset:%10\n\t"
      "ds_read_b64 %2, %8 offset:%11\n\tds_read_b64 %3, %8 offset:%12\n\t"
      "ds_read_b64 %4, %8 offset:%13\n\tds_read_b64 %5, %8 offset:%14\n\t"
      "ds_read_b64 %6, %8 offset:%15\n\tds_read_b64 %7, %8 offset:%16\n\ts_waitcnt lgkmcnt(0)"
      : "=&v"(x[0]), "=&v"(x[1]), "=&v"(x[2]), "=&v"(x[3]), "=&v"(x[4]), "=&v"(x[5]), "=&v"(x[6]), "=&v"(x[7])
      : "v"(addr), "i"(O0), "i"(O1), "i"(O2), "i"(O3), "i"(O4), "i"(O5), "i"(O6), "i"(O7)
      : "memory");
}
template <int O0, int O1, int O2, int O3>
__device__ __forceinline__ void lds_read4_b64(u32x2 (&x)[4], unsigned addr) {
  asm volatile(
      "ds_read_b64 %0, %4 offset:%5\n\tds_read_b64 %1, %4 offset:%6\n\t"
      "ds_read_b64 %2, %4 offset:%7\n\tds_read_b64 %3, %4 offset:%8\n\ts_waitcnt lgkmcnt(0)"
      : "=&v"(x[0]), "=&v"(x[1]), "=&v"(x[2]), "=&v"(x[3])
      : "v"(addr), "i"(O0), "i"(O1), "i"(O2), "i"(O3)
      : "memory");
}

}  // namespace cronus
