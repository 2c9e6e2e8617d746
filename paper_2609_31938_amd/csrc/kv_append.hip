// Rotation of queries and keys, and keys and values into the paged 8-bit cache.
//
//   pair (a, b), angle (c, s):  (a c - b s, b c + a s)
//   block of 16 tokens and head: scale 2^e, e least with max|x| <= 448 2^e;
//   codes e4m3(x 2^-e)
//
// One wave owns one block of 16 tokens of one head (of k, v or q): it holds
// the block's new values in registers, a pair of channels a lane and token,
// so the block's maximum is one reduction over the wave and every element is
// read once and written once.  Nobody else writes the block, so the scale
// needs no atomics, and an append of many tokens and many appends of one give
// the same scales.  Bound by memory traffic for frames of tokens and by
// latency for single ones.
//
// The products and sums of a rotation are rounded one by one (no fused
// multiply-add), so that a code is decided by the formula's own fp32 value.
#include "token_dev.h"
#include "tokens_internal.h"

#pragma clang fp contract(off)

namespace c3c {
namespace {

constexpr float kInf = __builtin_inff();

// least e >= -126 with amax <= 448 * 2^e (448 = 1.75 * 2^8)
__device__ inline int exponent_for(float amax) {
  const uint32_t b = __float_as_uint(amax);
  const int e = static_cast<int>(b >> 23) - 135 + ((b & 0x7fffffu) > 0x600000u ? 1 : 0);
  return e > -126 ? e : -126;
}
__device__ inline float pow2(int e) { return __uint_as_float(static_cast<uint32_t>(e + 127) << 23); }  // -126 .. 127

// e4m3 codes of two values (finite ones at most 448; others become NaN), in
// the low 16 bits
__device__ inline uint32_t codes2(float a, float b) {
  uint32_t r = static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false)) & 0xffffu;
  if (!(fabsf(a) < kInf)) r = (r & 0xff00u) | 0x7fu;
  if (!(fabsf(b) < kInf)) r = (r & 0x00ffu) | 0x7f00u;
  return r;
}

// Two elements of a row at channel c (even).
template <class E, bool AL>
__device__ inline void load2(const typename E::store* p, float& a, float& b) {
  typename E::store v[2];
  if (AL) {
    __builtin_memcpy(v, __builtin_assume_aligned(p, 2 * sizeof(v[0])), sizeof v);
  } else {
    v[0] = p[0];
    v[1] = p[1];
  }
  a = E::widen(v[0]);
  b = E::widen(v[1]);
}

// NP pairs of channels a lane: lane l holds channels 2 (l + 64 i) and the next.
template <class E, int NP, bool AL>
__global__ __launch_bounds__(256) void kv_append_k(AppendArgs a) {
  typedef typename E::store S;
  const int lane = threadIdx.x & 63;
  const int64_t b = blockIdx.z;
  const int heads = static_cast<int>(a.c.heads), D = static_cast<int>(a.c.dim);
  // one wave a head: keys, values, then queries
  int unit = __builtin_amdgcn_readfirstlane(static_cast<int>(blockIdx.y) * 4 + (threadIdx.x >> 6));
  if (unit >= 2 * heads + static_cast<int>(a.q_out ? a.q_heads : 0)) return;
  const int what = unit < heads ? 0 : unit < 2 * heads ? 1 : 2;
  const int head = unit - what * heads;

  // this sequence's rows and places
  int64_t row0 = a.b.cu[b], row1 = a.b.cu[b + 1];
  row0 = row0 < 0 ? 0 : row0;
  row1 = row1 > a.b.T ? a.b.T : row1;
  const int64_t n = row1 - row0;
  if (n <= 0) return;
  const int64_t len = a.b.len[b];
  const int64_t start = len - n;  // place of the first new token; negative if len is too short
  const int64_t first = start >= 0 ? start / 16 : -((15 - start) / 16);
  const int64_t last = (len - 1 >= 0) ? (len - 1) / 16 : -((16 - len) / 16);

  const S* src = static_cast<const S*>(what == 0 ? a.k : what == 1 ? a.v : a.q) + static_cast<int64_t>(head) * D;
  const int64_t ld = what == 0 ? a.ld_k : what == 1 ? a.ld_v : a.ld_q;
  const int rot = (what != 1 && a.r.cos) ? static_cast<int>(a.r.rot) : 0;

  for (int64_t blk = first + blockIdx.x; blk <= last; blk += gridDim.x) {
    const int64_t p0 = blk * 16;
    const int lo = start > p0 ? static_cast<int>(start - p0) : 0;
    const int hi = len - p0 < 16 ? static_cast<int>(len - p0) : 16;
    const int64_t r0 = row0 + (p0 - start);  // row of place 0 of the block (valid from lo to hi)
    float x[16][NP][2];
#pragma unroll
    for (int t = 0; t < 16; ++t)
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        const int c = 2 * (lane + 64 * i);
        x[t][i][0] = x[t][i][1] = 0.f;
        if (t >= lo && t < hi && c < D) load2<E, AL>(src + (r0 + t) * ld + c, x[t][i][0], x[t][i][1]);
      }
    if (rot) {
      const int half = rot >> 1;
#pragma unroll
      for (int t = 0; t < 16; ++t) {
        if (t < lo || t >= hi) continue;
        const int64_t at = a.r.pos ? a.r.pos[r0 + t] : p0 + t;
        const bool ok = at >= 0 && at < a.r.rows;
        const float* cs = a.r.cos + (ok ? at : 0) * half;
        const float* sn = a.r.sin + (ok ? at : 0) * half;
#pragma unroll
        for (int i = 0; i < NP; ++i) {
          const int c = 2 * (lane + 64 * i);
          if (a.r.pairs) {
            if (c < rot) {
              const float co = cs[c >> 1], si = sn[c >> 1], u = x[t][i][0], v = x[t][i][1];
              x[t][i][0] = u * co - v * si;
              x[t][i][1] = v * co + u * si;
            }
          } else {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const int ch = c + e;
              if (ch < rot) {
                const bool low = ch < half;
                const int j = low ? ch : ch - half;
                const float other = E::widen(src[(r0 + t) * ld + (low ? ch + half : j)]);
                const float co = cs[j], si = sn[j], u = x[t][i][e];
                x[t][i][e] = low ? u * co - other * si : u * co + other * si;
              }
            }
          }
          if (!ok) x[t][i][0] = x[t][i][1] = __builtin_nanf("");
        }
      }
    }
    if (what == 2) {
      S* out = static_cast<S*>(a.q_out) + static_cast<int64_t>(head) * D;
#pragma unroll
      for (int t = 0; t < 16; ++t) {
        if (t < lo || t >= hi) continue;
#pragma unroll
        for (int i = 0; i < NP; ++i) {
          const int c = 2 * (lane + 64 * i);
          if (c >= D) continue;
          S* o = out + (r0 + t) * (a.q_heads * D) + c;
          S v[2] = {E::narrow(x[t][i][0]), E::narrow(x[t][i][1])};
          if (AL) {
            __builtin_memcpy(__builtin_assume_aligned(o, 2 * sizeof(S)), v, sizeof v);
          } else {
            o[0] = v[0];
            o[1] = v[1];
          }
        }
      }
      continue;
    }
    // the block's page; tokens without a valid one are not stored
    if (p0 + 16 <= 0 || blk < 0) continue;
    const int64_t col = p0 / a.c.page;
    if (col >= a.b.cols) continue;
    const int64_t page = a.b.table[b * a.b.cols + col];
    if (page < 0 || page >= a.c.pages) continue;
    const int64_t nb = a.c.page / 16, pb = blk - col * nb;  // block of the page
    float* scale = (what == 0 ? a.c.k_scale : a.c.v_scale) + (page * heads + head) * nb + pb;

    float top = 0.f;
#pragma unroll
    for (int t = 0; t < 16; ++t)
#pragma unroll
      for (int i = 0; i < NP; ++i)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float m = fabsf(x[t][i][e]);
          top = fmaxf(top, m < kInf ? m : 0.f);
        }
    int ex = exponent_for(wave_max(top));
    int shrink = 0;  // earlier codes are multiplied by 2^-shrink
    if (lo > 0) {
      int old = static_cast<int>((__float_as_uint(*scale) >> 23) & 255u) - 127;
      old = old < -126 ? -126 : old > 127 ? 127 : old;
      ex = ex > old ? ex : old;
      shrink = ex - old;
    }
    const float inv = pow2(-ex < -126 ? -126 : -ex);
    const float fix = ex > 126 ? 0.5f : 1.f;  // 2^-127 is no normal number
    const float less = shrink > 126 ? 0.f : pow2(-shrink);
    if (lane == 0) *scale = pow2(ex);

    if (what == 0) {
      uint8_t* k = static_cast<uint8_t*>(a.c.k) + ((page * heads + head) * a.c.page + pb * 16) * D;
#pragma unroll
      for (int t = 0; t < 16; ++t)
#pragma unroll
        for (int i = 0; i < NP; ++i) {
          const int c = 2 * (lane + 64 * i);
          if (c >= D || t >= hi) continue;
          uint16_t* p = reinterpret_cast<uint16_t*>(k + static_cast<int64_t>(t) * D + c);
          if (t >= lo) {
            *p = static_cast<uint16_t>(codes2(x[t][i][0] * inv * fix, x[t][i][1] * inv * fix));
          } else if (shrink) {
            const tok_f32x2 f = __builtin_amdgcn_cvt_pk_f32_fp8(*p, false);
            *p = static_cast<uint16_t>(codes2(f[0] * less, f[1] * less));
          }
        }
    } else {
      uint8_t* v = static_cast<uint8_t*>(a.c.v) + ((page * heads + head) * nb + pb) * D * 16;
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        const int c = 2 * (lane + 64 * i);
        if (c >= D) continue;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          tok_u32x4* p = reinterpret_cast<tok_u32x4*>(v + (c + e) * 16);
          tok_u32x4 w = {0, 0, 0, 0};
          if (lo > 0 || hi < 16) w = *p;
#pragma unroll
          for (int t = 0; t < 16; t += 2) {
            const int sh = 8 * (t & 3);
            uint32_t old = (w[t >> 2] >> sh) & 0xffffu;
            if (shrink && t < lo) {
              const tok_f32x2 f = __builtin_amdgcn_cvt_pk_f32_fp8(old, false);
              old = codes2(f[0] * less, f[1] * less);
            }
            const uint32_t now = codes2(x[t][i][e] * inv * fix, x[t + 1][i][e] * inv * fix);
            const uint32_t keep = (t >= lo && t < hi ? 0u : 0xffu) | (t + 1 >= lo && t + 1 < hi ? 0u : 0xff00u);
            w[t >> 2] = (w[t >> 2] & ~(0xffffu << sh)) | (((old & keep) | (now & ~keep)) << sh);
          }
          *p = w;
        }
      }
    }
  }
}

template <class E, bool AL>
hipError_t run(const AppendArgs& a, dim3 grid, hipStream_t s) {
  auto k = a.c.dim <= 128 ? kv_append_k<E, 1, AL> : kv_append_k<E, 2, AL>;
  hipLaunchKernelGGL(k, grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

template <class E>
hipError_t typed(const AppendArgs& a, dim3 grid, hipStream_t s) {
  const int64_t two = 2 * static_cast<int64_t>(sizeof(typename E::store));
  auto even = [&](const void* p, int64_t ld) {
    return reinterpret_cast<uintptr_t>(p) % two == 0 && ld % 2 == 0;
  };
  const bool al = even(a.k, a.ld_k) && even(a.v, a.ld_v) && (!a.q_out || (even(a.q, a.ld_q) && even(a.q_out, 0)));
  return al ? run<E, true>(a, grid, s) : run<E, false>(a, grid, s);
}

}  // namespace

hipError_t launch_kv_append(const AppendArgs& a, int dtype, hipStream_t s) {
  if (a.b.B == 0 || a.b.T == 0 || a.b.max_new == 0) return hipSuccess;
  // n new tokens touch at most (n + 14) / 16 + 1 blocks
  int64_t bx = (a.b.max_new + 14) / 16 + 1;
  const int64_t units = 2 * a.c.heads + (a.q_out ? a.q_heads : 0), by = (units + 3) / 4;
  if (a.b.B > 65535 || by > 65535 || bx > 0x7fffffff) return hipErrorInvalidConfiguration;
  const dim3 grid(static_cast<unsigned>(bx), static_cast<unsigned>(by), static_cast<unsigned>(a.b.B));
  return dtype == C3C_DTYPE_BF16  ? typed<ElemBf16>(a, grid, s)
         : dtype == C3C_DTYPE_F16 ? typed<ElemF16>(a, grid, s)
                                  : typed<ElemF32>(a, grid, s);
}

}  // namespace c3c
