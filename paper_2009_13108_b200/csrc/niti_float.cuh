// Floating-point tensors at the boundary of the integer format: types, vector accesses, and the rounding of a float to an
// int8 payload with a power-of-two exponent (value = payload * 2^s).
#pragma once
#include "niti_common.cuh"
#include <cuda_bf16.h>
#include <cuda_fp16.h>

template <int T> struct FloatOf;
template <> struct FloatOf<NITI_F32> { typedef float type; };
template <> struct FloatOf<NITI_BF16> { typedef __nv_bfloat16 type; };
template <> struct FloatOf<NITI_F16> { typedef __half type; };
static inline int niti_type_size(int type) { return type == NITI_F32 ? 4 : 2; }
static inline bool niti_type_ok(int type) { return type == NITI_F32 || type == NITI_BF16 || type == NITI_F16; }

// VEC consecutive elements as the words that one access moves: 16 bytes, or a single element.
template <int T, int VEC>
struct Pack {
  static constexpr int BYTES = VEC * (int)sizeof(typename FloatOf<T>::type);
  static_assert(BYTES == 16 || VEC == 1, "16-byte vectors or single elements");
  static constexpr int WORDS = (BYTES + 3) / 4;
  unsigned w[WORDS];

  // KEEP: the next launch reads it again (else marked as the first to leave L2)
  template <bool KEEP = false>
  __device__ __forceinline__ void load(const void *p, long long i) {
    const char *q = reinterpret_cast<const char *>(p) + i * (long long)sizeof(typename FloatOf<T>::type);
    if constexpr (BYTES == 16) {
      const uint4 v = KEEP ? __ldcg(reinterpret_cast<const uint4 *>(q)) : __ldcs(reinterpret_cast<const uint4 *>(q));
      w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
    } else if constexpr (BYTES == 4) {
      w[0] = *reinterpret_cast<const unsigned *>(q);
    } else {
      w[0] = *reinterpret_cast<const unsigned short *>(q);
    }
  }
  __device__ __forceinline__ void store(void *p, long long i) const {
    char *q = reinterpret_cast<char *>(p) + i * (long long)sizeof(typename FloatOf<T>::type);
    if constexpr (BYTES == 16) *reinterpret_cast<uint4 *>(q) = make_uint4(w[0], w[1], w[2], w[3]);
    else if constexpr (BYTES == 4) *reinterpret_cast<unsigned *>(q) = w[0];
    else *reinterpret_cast<unsigned short *>(q) = (unsigned short)w[0];
  }
  // this + b, rounded to the type once
  __device__ __forceinline__ void add(const Pack &b) {
#pragma unroll
    for (int i = 0; i < WORDS; ++i) {
      if constexpr (T == NITI_F32) {
        w[i] = __float_as_uint(__uint_as_float(w[i]) + __uint_as_float(b.w[i]));
      } else if constexpr (T == NITI_BF16) {
        const __nv_bfloat162 s = __hadd2(*reinterpret_cast<const __nv_bfloat162 *>(&w[i]), *reinterpret_cast<const __nv_bfloat162 *>(&b.w[i]));
        w[i] = *reinterpret_cast<const unsigned *>(&s);
      } else {
        const __half2 s = __hadd2(*reinterpret_cast<const __half2 *>(&w[i]), *reinterpret_cast<const __half2 *>(&b.w[i]));
        w[i] = *reinterpret_cast<const unsigned *>(&s);
      }
    }
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < WORDS; ++i) w[i] = 0u;
  }
  __device__ __forceinline__ float get(int j) const {
    if constexpr (T == NITI_F32) return __uint_as_float(w[j]);
    else if constexpr (T == NITI_BF16) return __uint_as_float((j & 1) ? w[j >> 1] & 0xffff0000u : w[j >> 1] << 16);
    else return __half2float(__ushort_as_half((unsigned short)((j & 1) ? w[j >> 1] >> 16 : w[j >> 1])));
  }
  // rounded to the type (to nearest even)
  __device__ __forceinline__ void set(const float (&v)[VEC]) {
    if constexpr (T == NITI_F32) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) w[j] = __float_as_uint(v[j]);
    } else if constexpr (VEC == 1) {
      if constexpr (T == NITI_BF16) w[0] = __bfloat16_as_ushort(__float2bfloat16_rn(v[0]));
      else w[0] = __half_as_ushort(__float2half_rn(v[0]));
    } else {
#pragma unroll
      for (int j = 0; j < WORDS; ++j) {
        if constexpr (T == NITI_BF16) {
          const __nv_bfloat162 p = __floats2bfloat162_rn(v[2 * j], v[2 * j + 1]);
          w[j] = *reinterpret_cast<const unsigned *>(&p);
        } else {
          const __half2 p = __floats2half2_rn(v[2 * j], v[2 * j + 1]);
          w[j] = *reinterpret_cast<const unsigned *>(&p);
        }
      }
    }
  }
};

// Two float32 values for the packed instructions (each a multiply-add, multiplication or addition of both).
struct F2 {
  unsigned long long v;
  __device__ __forceinline__ F2(float a, float b) { asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(a), "f"(b)); }
  __device__ __forceinline__ explicit F2(float a) : F2(a, a) {}
  __device__ __forceinline__ void get(float &a, float &b) const { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
};
__device__ __forceinline__ F2 fma2(F2 a, F2 b, F2 c) {
  F2 r = c;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
  return r;
}
__device__ __forceinline__ F2 mul2(F2 a, F2 b) {
  F2 r = a;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}
__device__ __forceinline__ F2 add2(F2 a, F2 b) {
  F2 r = a;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}

// 32 bytes, a whole sector (pointers 32-byte aligned)
__device__ __forceinline__ void load32(const void *src, unsigned (&w)[8]) {
  asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
               : "l"(src)
               : "memory");
}
__device__ __forceinline__ void store32(void *dst, const unsigned (&w)[8]) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
               ::"l"(dst), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
               : "memory");
}
// 32 bytes of a type from (and to) 32 / size floats
template <int T, int N>
__device__ __forceinline__ void pack32(const float *v, unsigned (&w)[8]) {
  static_assert(N == 32 / (int)sizeof(typename FloatOf<T>::type), "");
  constexpr int V = N / 2;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    float part[V];
#pragma unroll
    for (int j = 0; j < V; ++j) part[j] = v[V * h + j];
    Pack<T, V> k;
    k.set(part);
#pragma unroll
    for (int j = 0; j < 4; ++j) w[4 * h + j] = k.w[j];
  }
}
template <int T, int N>
__device__ __forceinline__ float get32(const unsigned (&w)[8], int j) {
  constexpr int V = N / 2;
  Pack<T, V> k;
#pragma unroll
  for (int i = 0; i < 4; ++i) k.w[i] = w[4 * (j / V) + i];
  return k.get(j % V);
}

// ---- rounding to payloads -------------------------------------------------------------------
// Exponent of a tensor (or row) whose largest magnitude has these bits: the one that leaves seven integer bits, so that
// payload magnitudes reach 64 .. 127 (the effective bit-width rule of Section 3.2 on floats).  Not below NITI_EXP_LOWEST
// (2^-s stays a normal float); 0 for a tensor of zeros; that of the largest finite magnitude where one is not finite.
#define NITI_EXP_LOWEST (-100)
__device__ __forceinline__ int niti_exponent_of(unsigned max_bits, int integer_bits = 7) {
  if (max_bits == 0u) return 0;
  const int e = (int)(max_bits >> 23);
  const int s = (e > 254 ? 254 : e) - 126 - integer_bits;
  return s < NITI_EXP_LOWEST ? NITI_EXP_LOWEST : s;
}
// 2^e for e in [-126, 127]
__device__ __forceinline__ float niti_pow2(int e) { return __int_as_float((e + 127) << 23); }

// The larger magnitude of two, NaN if either is.
__device__ __forceinline__ float niti_absmax(float m, float x) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(m), "f"(fabsf(x)));
  return r;
}

// Magnitudes in units of the result to whole numbers, at most 127.  Pseudo-stochastic: the 16 fraction bits are split into
// halves, rounded up where the top half is larger than the bottom half (Algorithm 3 with bp = 16; the sum carries into bit
// 16 exactly then).  To nearest: half up, as everywhere in the library.
// `scale` is that of niti_payload_scale(): in the first case results come in bits 16 .. 22, so that the multiplication
// that scales also makes room for the fraction.  The whole part comes out of an addition of 2^23 that rounds towards zero (a
// conversion instruction takes a slot of the pipe of exponentials and reciprocals, a quarter as wide); the exponent that it
// leaves in the word does not reach bit 23.  NaN becomes 127.
__device__ __forceinline__ float niti_payload_scale(float units, int round_mode) {
  return round_mode == NITI_ROUND_PSR ? units * 65536.0f : units;
}
template <bool PSR>
__device__ __forceinline__ unsigned niti_unit_mag(float x, float scale) {
  if constexpr (PSR) {
    const unsigned v = __float_as_uint(__fadd_rz(fminf(fabsf(x) * scale, 127.0f * 65536.0f), 8388608.0f));
    return v + (~v & 255u) * 256u;
  } else {
    // (plus the float below 1/2, 1/2 - 2^-25: 1/2 itself would lift a magnitude of 1/2 - 2^-25 to 1 by the sum's rounding, and
    // what is missing from k + 1/2 to k + 1 the rounding adds, half a step below 1 and less below the others)
    return __float_as_uint(__fadd_rz(fminf(fmaf(fabsf(x), scale, 0.49999997f), 127.0f), 8388608.0f));
  }
}
// (of 127 << 16 the sum is 127 << 16 | 0xff00: the same byte)
template <bool PSR>
__device__ __forceinline__ int niti_payload(float x, float scale) {
  const int q = (int)((PSR ? niti_unit_mag<PSR>(x, scale) >> 16 : niti_unit_mag<PSR>(x, scale)) & 127u);
  return x < 0.0f ? -q : q;
}
// Four payloads in a word: magnitudes gathered by byte permutes, signs as bytes of zeros or ones (a permute with sign
// replication), and two's complement of four bytes at once: the low seven bits plus one where negative do not reach the next
// byte, and their carry into bit 7 turns the sign off again for a magnitude of zero.  7.5 instructions a value, 13 one by one.
template <bool PSR>
__device__ __forceinline__ unsigned niti_payload4(float x0, float x1, float x2, float x3, float scale) {
  const unsigned a = niti_unit_mag<PSR>(x0, scale), b = niti_unit_mag<PSR>(x1, scale), c = niti_unit_mag<PSR>(x2, scale), d = niti_unit_mag<PSR>(x3, scale);
  constexpr unsigned PAIR = PSR ? 0x0062u : 0x0040u;                       // byte 2 (0) of both
  const unsigned m = __byte_perm(__byte_perm(a, b, PAIR), __byte_perm(c, d, PAIR), 0x5410);
  unsigned s01, s23, s;
  asm("prmt.b32 %0, %1, %2, 0x00fb;" : "=r"(s01) : "r"(__float_as_uint(x0)), "r"(__float_as_uint(x1)));    // sign bytes of both
  asm("prmt.b32 %0, %1, %2, 0x00fb;" : "=r"(s23) : "r"(__float_as_uint(x2)), "r"(__float_as_uint(x3)));
  s = __byte_perm(s01, s23, 0x5410);
  return (((m ^ s) & 0x7f7f7f7fu) + (s & 0x01010101u)) ^ (s & 0x80808080u);
}
// VEC payload bytes at p + i
template <int VEC, bool PSR>
__device__ __forceinline__ void niti_store_payload(int8_t *p, long long i, const float (&x)[VEC], float scale) {
  if constexpr (VEC == 1) {
    p[i] = (int8_t)niti_payload<PSR>(x[0], scale);
  } else {
    const unsigned w0 = niti_payload4<PSR>(x[0], x[1], x[2], x[3], scale);
    if constexpr (VEC == 8) *reinterpret_cast<uint2 *>(p + i) = make_uint2(w0, niti_payload4<PSR>(x[4], x[5], x[6], x[7], scale));
    else *reinterpret_cast<unsigned *>(p + i) = w0;
  }
}
