// The 8-bit activation record and the vector loads and stores that the kernels on activations share.
//
// A record of x [T, H] holds one byte per value and one power of two per 32 consecutive values of a row:
//   x[t, h] ~ code[t, h] * 2^e[t, h / 32],   code = int8 (-127 .. 127) or e4m3 (|code| <= 448)
//   e = the smallest integer with max |x| <= Q 2^e over the 32 values, Q = 127 or 448, at least kActMinExp
//   code = x 2^-e rounded to nearest even (exact scaling: nothing saturates); stored scale byte = e + 127
//   (where rounding up would pass the largest finite fp32 number, the code below it is taken: 63 2^122 or 240 2^120)
// A group that holds an infinity or a NaN stores byte 255 and reads back as NaN in all its 32 places.
// Why a power of two per 32 and not one fp32 factor per row or per 128: 7 or 4 significant bits times a power of two
// are exact in bf16 (down to its last subnormal, 2^-133: e4m3 codes at e = -126 go on to 2^-135), so a record is a bf16
// operand of the tensor cores without a second rounding, and scaling by it is exact everywhere. What the coarser factor
// loses (a factor of at most 2 in the int8 step) the shorter group gains back: the largest of 32 normal values is about
// 2.1 deviations, of 128 about 2.8.
//
// Layout in one buffer: codes [T, Hp] with Hp = H rounded up to 32 (padding codes are 0), then at the next multiple of
// 256 bytes the scale bytes [T, Sp] with Sp = Hp / 32 rounded up to 16: both are tensor-map pitches.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "sm100_prims.cuh"

namespace kdkl {

constexpr int kActGroup = 32;
constexpr int kActMinExp = -126;        // 2^e and 2^-e are then normal fp32 numbers
constexpr int kFmtInt8 = 0, kFmtE4M3 = 1;

struct ActRecord {                      // a record in device memory
  uint8_t* codes;
  uint8_t* scales;
};
__host__ __device__ inline long long act_codes_pitch(long long H) { return (H + 31) / 32 * 32; }
__host__ __device__ inline long long act_scale_pitch(long long H) { return (act_codes_pitch(H) / 32 + 15) / 16 * 16; }
__host__ __device__ inline long long act_scales_at(long long T, long long H) {
  return (T * act_codes_pitch(H) + 255) / 256 * 256;
}

// ------------------------------------------------------------------ two fp32 values an instruction
__device__ __forceinline__ uint64_t f2_bits(float2 a) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a.x), "f"(a.y));
  return r;
}
__device__ __forceinline__ float2 f2_of(uint64_t r) {
  float2 a;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(a.x), "=f"(a.y) : "l"(r));
  return a;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(f2_bits(a)), "l"(f2_bits(b)), "l"(f2_bits(c)));
  return f2_of(r);
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(f2_bits(a)), "l"(f2_bits(b)));
  return f2_of(r);
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(f2_bits(a)), "l"(f2_bits(b)));
  return f2_of(r);
}
__device__ __forceinline__ float2 both(float x) { return make_float2(x, x); }

// ------------------------------------------------------------------ eight values of a row
// Which eight columns a thread has depends on the rows. VEC: they start on 16 bytes (fp32: 32) and H % 8 == 0, so that a
// thread's columns c .. c + 7 are one aligned word of 16 or 32 bytes and four lanes share a group of a record.
// Otherwise a warp's lanes take neighbouring columns and a thread every 32nd, c, c + 32, .., c + 224: element by element,
// but still whole lines a warp, and a group of a record is a warp's. What lies past the row's end reads as 0 and is not
// written. first_column gives c of the v-th thread of a row (whole warps).
template <bool VEC> __device__ __forceinline__ int first_column(int v) { return VEC ? 8 * v : (v & ~31) * 8 + (v & 31); }
template <bool VEC> __device__ __forceinline__ int column(int c, int i) { return VEC ? c + i : c + 32 * i; }
__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_f32(__half x) { return __half2float(x); }
template <typename T> __device__ __forceinline__ T from_f32(float x);
template <> __device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half from_f32<__half>(float x) { return __float2half_rn(x); }

template <typename T> struct Raw8 { uint4 v; };            // eight 16-bit values as they were loaded
template <> struct Raw8<float> { uint4 v, w; };

__device__ __forceinline__ void words_to_f32(const uint4& v, float (&f)[8], __nv_bfloat16) {
  const __nv_bfloat162* p = reinterpret_cast<const __nv_bfloat162*>(&v);
#pragma unroll
  for (int i = 0; i < 4; ++i) { const float2 x = __bfloat1622float2(p[i]); f[2 * i] = x.x; f[2 * i + 1] = x.y; }
}
__device__ __forceinline__ void words_to_f32(const uint4& v, float (&f)[8], __half) {
  const __half2* p = reinterpret_cast<const __half2*>(&v);
#pragma unroll
  for (int i = 0; i < 4; ++i) { const float2 x = __half22float2(p[i]); f[2 * i] = x.x; f[2 * i + 1] = x.y; }
}
template <typename T> __device__ __forceinline__ void raw_to_f32(const Raw8<T>& r, float (&f)[8]) {
  words_to_f32(r.v, f, T());
}
template <> __device__ __forceinline__ void raw_to_f32<float>(const Raw8<float>& r, float (&f)[8]) {
  f[0] = __uint_as_float(r.v.x); f[1] = __uint_as_float(r.v.y); f[2] = __uint_as_float(r.v.z); f[3] = __uint_as_float(r.v.w);
  f[4] = __uint_as_float(r.w.x); f[5] = __uint_as_float(r.w.y); f[6] = __uint_as_float(r.w.z); f[7] = __uint_as_float(r.w.w);
}
__device__ __forceinline__ void f32_to_words(const float (&f)[8], uint4& v, __nv_bfloat16) {
  __nv_bfloat162* p = reinterpret_cast<__nv_bfloat162*>(&v);
#pragma unroll
  for (int i = 0; i < 4; ++i) p[i] = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
}
__device__ __forceinline__ void f32_to_words(const float (&f)[8], uint4& v, __half) {
  __half2* p = reinterpret_cast<__half2*>(&v);
#pragma unroll
  for (int i = 0; i < 4; ++i) p[i] = __floats2half2_rn(f[2 * i], f[2 * i + 1]);
}
template <typename T> __device__ __forceinline__ Raw8<T> f32_to_raw(const float (&f)[8]) {
  Raw8<T> r;
  f32_to_words(f, r.v, T());
  return r;
}
template <> __device__ __forceinline__ Raw8<float> f32_to_raw<float>(const float (&f)[8]) {
  Raw8<float> r;
  r.v = make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
  r.w = make_uint4(__float_as_uint(f[4]), __float_as_uint(f[5]), __float_as_uint(f[6]), __float_as_uint(f[7]));
  return r;
}

// Loads here are coherent ones, never ld.global.nc (nor const __restrict__, which lets the compiler choose it): a kernel
// that may start while the one before it drains (grid_dependency_wait) reads what is written during its own lifetime, and
// the non-coherent path is defined only for memory that nobody writes in that time.
// (Bytes by an instruction of their own: from plain C++ loads the compiler takes 5 to 13 registers more in the element-wise
// kernels, a block less an SM. Gated backward 16384 x 7167, int8: 851 against 1380 us.)
__device__ __forceinline__ uint32_t ld_global_u8(const uint8_t* p) {
  uint32_t v;
  asm volatile("ld.global.u8 %0, [%1];" : "=r"(v) : "l"(p));
  return v;
}
// A thread's eight columns of a row of `width` values:
template <typename T, bool VEC>
__device__ __forceinline__ Raw8<T> load_raw8(const T* row, int c, int width) {
  Raw8<T> r;
  if (VEC) {
    if (c < width) {
      if constexpr (sizeof(T) == 4) {
        asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                     : "=r"(r.v.x), "=r"(r.v.y), "=r"(r.v.z), "=r"(r.v.w), "=r"(r.w.x), "=r"(r.w.y), "=r"(r.w.z), "=r"(r.w.w)
                     : "l"(row + c));
      } else {
        r.v = *reinterpret_cast<const uint4*>(row + c);
      }
    } else {
      r.v = make_uint4(0u, 0u, 0u, 0u);
      if constexpr (sizeof(T) == 4) r.w = r.v;
    }
  } else {
    float f[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = column<VEC>(c, i) < width ? to_f32(row[column<VEC>(c, i)]) : 0.f;
    r = f32_to_raw<T>(f);                 // back to the type it came from: exact
  }
  return r;
}
template <typename T, bool VEC>
__device__ __forceinline__ void load8(const T* row, int c, int width, float (&f)[8]) {
  raw_to_f32(load_raw8<T, VEC>(row, c, width), f);
}
template <typename T, bool VEC>
__device__ __forceinline__ void store_raw8(T* row, int c, int width, const Raw8<T>& r) {
  if (VEC) {
    if (c < width) {
      if constexpr (sizeof(T) == 4) {
        asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(row + c), "r"(r.v.x), "r"(r.v.y),
                     "r"(r.v.z), "r"(r.v.w), "r"(r.w.x), "r"(r.w.y), "r"(r.w.z), "r"(r.w.w) : "memory");
      } else {
        *reinterpret_cast<uint4*>(row + c) = r.v;
      }
    }
  } else {
    float f[8];
    raw_to_f32(r, f);
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (column<VEC>(c, i) < width) row[column<VEC>(c, i)] = from_f32<T>(f[i]);
  }
}

// ------------------------------------------------------------------ codes
// Scale byte of a group from the largest |x| of it, taken as an unsigned integer of the fp32 bits (which orders
// magnitudes, infinities above all numbers and NaNs above those).
template <int FMT>
__device__ __forceinline__ uint32_t act_scale_byte(uint32_t amax_bits) {
  // max|x| = (1 + m / 2^23) 2^(E - 127); Q = 1.984375 * 2^6 or 1.75 * 2^8: adding what carries into E where m is beyond
  // Q's fraction gives E rounded up as needed
  constexpr uint32_t kCarry = 0x7fffffu - (FMT == kFmtInt8 ? 0x7e0000u : 0x600000u);
  constexpr int kShift = FMT == kFmtInt8 ? 6 : 8;
  const int byte = max((int)((amax_bits + kCarry) >> 23) - kShift, kActMinExp + 127);    // zeros and subnormal maxima too
  return amax_bits >= 0x7f800000u ? 255u : (uint32_t)byte;
}
__device__ __forceinline__ float act_scale(uint32_t byte) {          // 2^e, NaN for byte 255
  return byte == 255u ? __uint_as_float(0x7fffffffu) : __uint_as_float(byte << 23);
}
__device__ __forceinline__ float act_inverse(uint32_t byte) {        // 2^-e; 0 for byte 255 (codes 0)
  return byte == 255u ? 0.f : __uint_as_float((254u - byte) << 23);
}
// the largest |x| of eight as fp32 bits; NaN where there is one
__device__ __forceinline__ float max3_abs(float a, float b, float c) {
  float r;
  asm("{\n\t.reg .f32 x, y, z;\n\tabs.f32 x, %1;\n\tabs.f32 y, %2;\n\tabs.f32 z, %3;\n\tmax.NaN.f32 %0, x, y, z;\n\t}"
      : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
__device__ __forceinline__ uint32_t abs_max_bits(const float (&f)[8]) {
  const float m = max3_abs(max3_abs(f[0], f[1], f[2]), f[3], f[4]);
  return __float_as_uint(max3_abs(max3_abs(m, f[5], f[6]), f[7], f[7]));
}
// the largest of the four neighbouring lanes that share a group (all four take part)
__device__ __forceinline__ uint32_t group_max(uint32_t m) {
  m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
  return max(m, __shfl_xor_sync(0xffffffffu, m, 2));
}
// (the whole warp calls)
template <int FMT>
__device__ __forceinline__ uint2 act_codes(const float (&x)[8], uint32_t byte) {
  const float inv = act_inverse(byte);
  const bool bad = byte == 255u;
  float f[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = x[i];
  // the one exponent at which a code rounded up would stand for 2^128
  constexpr uint32_t kTopByte = FMT == kFmtInt8 ? 122 + 127 : 120 + 127;
  constexpr float kTopCode = FMT == kFmtInt8 ? 63.f : 240.f;
  if (__any_sync(0xffffffffu, byte == kTopByte)) {
    const float lim = byte == kTopByte ? kTopCode * act_scale(byte) : __uint_as_float(0x7f7fffffu);
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = fminf(fmaxf(f[i], -lim), lim);
  }
  uint32_t w[2];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    if (FMT == kFmtInt8) {
      // 1.5 * 2^23 + code: rounded to nearest even by the addition, the code in the low byte in two's complement
      const float2 magic = both(12582912.f);
      const float2 u = fma2(make_float2(f[4 * k], f[4 * k + 1]), both(inv), magic);
      const float2 v = fma2(make_float2(f[4 * k + 2], f[4 * k + 3]), both(inv), magic);
      const uint32_t c = __byte_perm(__byte_perm(__float_as_uint(u.x), __float_as_uint(u.y), 0x0040),
                                     __byte_perm(__float_as_uint(v.x), __float_as_uint(v.y), 0x0040), 0x5410);
      w[k] = bad ? 0u : c;
    } else {
      const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(f[4 * k] * inv, f[4 * k + 1] * inv), __NV_SATFINITE, __NV_E4M3);
      const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(f[4 * k + 2] * inv, f[4 * k + 3] * inv), __NV_SATFINITE, __NV_E4M3);
      w[k] = bad ? 0u : (lo & 0xffffu) | (hi << 16);
    }
  }
  return make_uint2(w[0], w[1]);
}
template <int FMT>
__device__ __forceinline__ void act_values(const uint2& codes, uint32_t byte, float (&f)[8]) {
  const float s = act_scale(byte);
  const uint32_t w[2] = {codes.x, codes.y};
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    if (FMT == kFmtInt8) {
      // 2^23 + (code + 128) as bits, minus 2^23 + 128, times 2^e: every step is exact
      const uint32_t u = w[k] ^ 0x80808080u;
      const float2 off = make_float2(-8388736.f, -8388736.f), s2 = make_float2(s, s);
      const float2 a = mul2(add2(make_float2(__uint_as_float(__byte_perm(u, 0x4b000000u, 0x7540)),
                                             __uint_as_float(__byte_perm(u, 0x4b000000u, 0x7541))), off), s2);
      const float2 b = mul2(add2(make_float2(__uint_as_float(__byte_perm(u, 0x4b000000u, 0x7542)),
                                             __uint_as_float(__byte_perm(u, 0x4b000000u, 0x7543))), off), s2);
      f[4 * k] = a.x; f[4 * k + 1] = a.y; f[4 * k + 2] = b.x; f[4 * k + 3] = b.y;
    } else {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w[k] >> (16 * i)), __NV_E4M3);
        const float2 v = __half22float2(__half2(h));
        f[4 * k + 2 * i] = v.x * s;
        f[4 * k + 2 * i + 1] = v.y * s;
      }
    }
  }
}

// One code and what it stands for.
template <int FMT> __device__ __forceinline__ uint32_t act_code(float x, uint32_t byte) {
  float f[8] = {x, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  return act_codes<FMT>(f, byte).x & 0xffu;
}
template <int FMT> __device__ __forceinline__ float act_value(uint32_t code, uint32_t byte) {
  float f[8];
  act_values<FMT>(make_uint2(code, 0u), byte, f);
  return f[0];
}

// Write a thread's eight values of row t into a record; the whole warp calls. Values past the row's end are 0.
template <int FMT, bool VEC>
__device__ __forceinline__ void record_write8(const ActRecord& r, long long t, long long cpitch, long long spitch, int c,
                                              const float (&f)[8]) {
  uint8_t* codes = r.codes + t * cpitch;
  uint8_t* scales = r.scales + t * spitch;
  if (VEC) {
    const uint32_t byte = act_scale_byte<FMT>(group_max(abs_max_bits(f)));
    const uint2 v = act_codes<FMT>(f, byte);
    if (c < cpitch) *reinterpret_cast<uint2*>(codes + c) = v;
    if (c < cpitch && (c & 31) == 0) scales[c >> 5] = (uint8_t)byte;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int col = column<VEC>(c, i);
      const uint32_t byte = act_scale_byte<FMT>(__reduce_max_sync(0xffffffffu, __float_as_uint(f[i]) & 0x7fffffffu));
      const uint32_t code = act_code<FMT>(f[i], byte);
      if (col < cpitch) codes[col] = (uint8_t)code;
      if (col < cpitch && (col & 31) == 0) scales[col >> 5] = (uint8_t)byte;
    }
  }
}
// eight neighbouring codes and their scale byte, for act_values
__device__ __forceinline__ void record_fetch8(const ActRecord& r, long long t, long long cpitch, long long spitch, int c,
                                              uint2& codes, uint32_t& byte) {
  codes = *reinterpret_cast<const uint2*>(r.codes + t * cpitch + c);
  byte = ld_global_u8(r.scales + t * spitch + (c >> 5));
}
// a thread's eight values; 0 past the end
template <int FMT, bool VEC>
__device__ __forceinline__ void record_read8(const ActRecord& r, long long t, long long cpitch, long long spitch, int c,
                                             float (&f)[8]) {
  if (VEC) {
    uint2 codes = make_uint2(0u, 0u);
    uint32_t byte = 1u;
    if (c < cpitch) record_fetch8(r, t, cpitch, spitch, c, codes, byte);
    act_values<FMT>(codes, byte, f);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int col = column<VEC>(c, i);
      f[i] = col < cpitch ? act_value<FMT>(ld_global_u8(r.codes + t * cpitch + col), ld_global_u8(r.scales + t * spitch + (col >> 5))) : 0.f;
    }
  }
}
// The same with a format that is known at run time, uniform over a launch.
template <bool VEC>
__device__ __forceinline__ void record_write8(int fmt, const ActRecord& r, long long t, long long cpitch, long long spitch,
                                              int c, const float (&f)[8]) {
  if (fmt == kFmtInt8) record_write8<kFmtInt8, VEC>(r, t, cpitch, spitch, c, f);
  else record_write8<kFmtE4M3, VEC>(r, t, cpitch, spitch, c, f);
}
template <bool VEC>
__device__ __forceinline__ void record_read8(int fmt, const ActRecord& r, long long t, long long cpitch, long long spitch,
                                             int c, float (&f)[8]) {
  if (fmt == kFmtInt8) record_read8<kFmtInt8, VEC>(r, t, cpitch, spitch, c, f);
  else record_read8<kFmtE4M3, VEC>(r, t, cpitch, spitch, c, f);
}

// ------------------------------------------------------------------ store and load
// One thread per eight values; a block covers an even share of the columns, at most 2048, of the rows blockIdx.y, blockIdx.y + gridDim.y, ... Bound by
// memory. Many short blocks keep more loads in flight than few long ones (128 or 64 an SM against 16: 5 to 10 %); two
// rows asked for at once pay only where little is done with a row, in load.
// 32768 x 4096 bf16, one B200: store 70 us (5.8 TB/s), load 64 us (6.4 TB/s, 0.99 of a copy).
// Element by element at most 40 registers, for a sixth block an SM: 16384 x 4095 bf16, e4m3: 139 against 161 us.
template <typename T, int FMT, bool VEC>
__global__ void __launch_bounds__(256, VEC ? 0 : 6)
act8_store_kernel(const T* x, long long ld, long long rows, int H, ActRecord rec) {
  const long long cpitch = act_codes_pitch(H), spitch = act_scale_pitch(H);
  const int c = first_column<VEC>(blockIdx.x * blockDim.x + threadIdx.x);
  grid_dependents_launch();
  grid_dependency_wait();
  for (long long t = blockIdx.y; t < rows; t += gridDim.y) {
    float f[8];
    load8<T, VEC>(x + t * ld, c, H, f);
    record_write8<FMT, VEC>(rec, t, cpitch, spitch, c, f);
  }
}
template <typename T, int FMT, bool VEC>
__global__ void __launch_bounds__(256)
act8_load_kernel(ActRecord rec, long long rows, int H, T* __restrict__ out, long long ld) {
  const long long cpitch = act_codes_pitch(H), spitch = act_scale_pitch(H);
  const int c = first_column<VEC>(blockIdx.x * blockDim.x + threadIdx.x);
  grid_dependents_launch();
  grid_dependency_wait();
  if (c >= H) return;
  auto put = [&](float (&f)[8], long long t) {
    if constexpr (std::is_same<T, __half>::value) {       // a code rounded up past the largest fp16 value
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = f[i] > 65504.f ? 65504.f : f[i] < -65504.f ? -65504.f : f[i];
    }
    store_raw8<T, VEC>(out + t * ld, c, H, f32_to_raw<T>(f));
  };
  constexpr int U = VEC ? 2 : 1;
  for (long long t0 = blockIdx.y; t0 < rows; t0 += (long long)U * gridDim.y) {
    float f[8];
    if constexpr (VEC) {
      uint2 codes[U];
      uint32_t bytes[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const long long t = t0 + (long long)u * gridDim.y;
        if (t < rows) record_fetch8(rec, t, cpitch, spitch, c, codes[u], bytes[u]);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const long long t = t0 + (long long)u * gridDim.y;
        if (t >= rows) break;
        act_values<FMT>(codes[u], bytes[u], f);
        put(f, t);
      }
    } else {
      record_read8<FMT, VEC>(rec, t0, cpitch, spitch, c, f);
      put(f, t0);
    }
  }
}

}  // namespace kdkl
