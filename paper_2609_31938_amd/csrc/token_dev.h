// Device helpers of the token operators' kernels: element types, 16-byte
// access at any alignment, reductions over a wave.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace c3c {

typedef float tok_f32x4 __attribute__((ext_vector_type(4)));
typedef float tok_f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t tok_u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t tok_u32x2 __attribute__((ext_vector_type(2)));
typedef int32_t tok_i32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 tok_bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 tok_bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 tok_f16x2 __attribute__((ext_vector_type(2)));

// element types by their storage: widen() is exact, narrow() rounds to
// nearest even
struct ElemBf16 {
  typedef uint16_t store;
  static constexpr int VEC = 8;  // elements of a 16-byte access
  __device__ static float widen(store v) { return __uint_as_float(static_cast<uint32_t>(v) << 16); }
  __device__ static store narrow(float f) {
    return static_cast<store>(
        __builtin_bit_cast(uint32_t, __builtin_convertvector((tok_f32x2{f, 0.f}), tok_bf16x2)));
  }
};
struct ElemF16 {
  typedef uint16_t store;
  static constexpr int VEC = 8;
  __device__ static float widen(store v) { return static_cast<float>(__builtin_bit_cast(_Float16, v)); }
  __device__ static store narrow(float f) { return __builtin_bit_cast(store, static_cast<_Float16>(f)); }
};
struct ElemF32 {
  typedef float store;
  static constexpr int VEC = 4;
  __device__ static float widen(store v) { return v; }
  __device__ static store narrow(float f) { return f; }
};

// VEC elements as they are stored
template <class E>
struct Raw {
  typename E::store v[E::VEC];
  __device__ void widen(float (&f)[E::VEC]) const {
#pragma unroll
    for (int e = 0; e < E::VEC; ++e) f[e] = E::widen(v[e]);
  }
};

// VEC elements from p (any alignment of the element's size), of which the
// first m exist; the others are 0
template <class E>
__device__ inline void load_raw(const typename E::store* p, int m, Raw<E>& r) {
  if (m >= E::VEC) {
    __builtin_memcpy(r.v, p, 16);
  } else {
#pragma unroll
    for (int e = 0; e < E::VEC; ++e) r.v[e] = e < m ? p[e] : typename E::store(0);
  }
}
template <class E>
__device__ inline void load_vec(const typename E::store* p, int m, float (&f)[E::VEC]) {
  Raw<E> r;
  load_raw<E>(p, m, r);
  r.widen(f);
}

// stream: past the caches' memory of what was used last
template <class E>
__device__ inline void store_vec(typename E::store* p, int m, const float (&f)[E::VEC], bool stream = false) {
  typename E::store v[E::VEC];
#pragma unroll
  for (int e = 0; e < E::VEC; ++e) v[e] = E::narrow(f[e]);
  if (m >= E::VEC) {
    if (stream) {
      typedef tok_u32x4 __attribute__((aligned(2))) any;
      tok_u32x4 w;
      __builtin_memcpy(&w, v, 16);
      __builtin_nontemporal_store(w, reinterpret_cast<any*>(p));
    } else {
      __builtin_memcpy(p, v, 16);
    }
  } else {
#pragma unroll
    for (int e = 0; e < E::VEC - 1; ++e)
      if (e < m) p[e] = v[e];
  }
}

__device__ inline float wave_sum(float v) {
#pragma unroll
  for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
  return v;
}

__device__ inline float wave_max(float v) {
#pragma unroll
  for (int o = 32; o; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
  return v;
}

// ---- 8-bit rows: q = x / s to the nearest integer, s = max|x| / 127

// |v|, infinite for a NaN too: a maximum of these says whether all are finite
__device__ inline float magnitude(float v) {
  const float a = fabsf(v);
  return a < __builtin_inff() ? a : __builtin_inff();
}

// the scale of an 8-bit row, and one code of it (IEEE division: the codes are
// those of the definition)
__device__ inline float row_scale(float amax) { return amax < __builtin_inff() ? amax / 127.f : __builtin_nanf(""); }
__device__ inline int code(float v, float s) {
  const float q = rintf(v / s);
  // s rounds amax / 127, so |v| / s may round past 127 for a tiny s
  return s > 0.f ? static_cast<int>(fminf(fmaxf(q, -127.f), 127.f)) : 0;
}

// The integer nearest to 127 v / top itself (top: the row's largest magnitude), not
// to v / s with its rounded scale.  The two differ only where a code is doubtful:
// next to a half (v / s errs by less than 2^-16), or anywhere under a subnormal
// scale, which has few bits.
__device__ inline bool doubtful(float v, float s) {
  const float t = v / s;
  return s < 0x1p-126f || fabsf(fabsf(t - rintf(t)) - 0.5f) < 0x1p-15f;
}
__device__ inline int true_code(float v, float s, float top) {
  return s > 0.f ? static_cast<int>(rint(static_cast<double>(v) * 127.0 / static_cast<double>(top))) : 0;
}

// top: 0, or the row's largest magnitude for codes by true_code
template <int N>
__device__ inline void store_codes(int8_t* p, int m, const float (&v)[N], float s, float top = 0.f) {
  uint32_t w[(N + 3) / 4];
#pragma unroll
  for (int i = 0; i < (N + 3) / 4; ++i) w[i] = 0;
#pragma unroll
  for (int e = 0; e < N; ++e) w[e >> 2] |= (static_cast<uint32_t>(code(v[e], s)) & 255u) << (8 * (e & 3));
  if (top > 0.f) {
    bool any = false;
#pragma unroll
    for (int e = 0; e < N; ++e) any |= doubtful(v[e], s);
    if (__builtin_expect(any, 0)) {
#pragma unroll
      for (int i = 0; i < (N + 3) / 4; ++i) w[i] = 0;
#pragma unroll
      for (int e = 0; e < N; ++e) w[e >> 2] |= (static_cast<uint32_t>(true_code(v[e], s, top)) & 255u) << (8 * (e & 3));
    }
  }
  if (m >= N) {
    __builtin_memcpy(p, w, N);
  } else {
#pragma unroll
    for (int e = 0; e < N - 1; ++e)
      if (e < m) p[e] = static_cast<int8_t>(w[e >> 2] >> (8 * (e & 3)));
  }
}

}  // namespace c3c
