// Rotation of queries and keys, and keys and values into the paged 8-bit cache.
//
//   pair (a, b), angle (c, s):  (a c - b s, b c + a s)
//   block of 16 tokens and head: scale 2^e, e least with max|x| <= 448 2^e;
//   codes e4m3(x 2^-e)
//
// One wave owns one block of 16 tokens of one head (of k, v or q): lane l holds
// 8 channels from 8 (l % 16) on (and the same past 128) of the 4 tokens from
// 4 (l / 16) on, 16 bytes a load.  So the block's maximum is one reduction over
// the wave and every element is read once and written once.  Nobody else
// writes the block, so the scale needs no atomics, and an append of many tokens
// and many appends of one give the same scales.  V's 4 x 4 (lane groups x
// pairs of channels) dwords of 4 tokens are transposed between the lane groups,
// so that a lane stores whole 16-byte rows.  The page, a lane's
// four tokens, the block's old scale and the tokens' angles are read one after
// another: each load stands behind a condition and is waited for there.  A
// single token's time is that chain of memory latencies (64 tokens of 64
// sequences, 32 + 8 + 8 heads of 128: 7 us); frames move 3.8 TB/s (4 x 1560
// tokens, 3 x 12 heads of 128 in bf16: 26 us).
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

// 8 elements of a row, at any alignment
template <class E>
__device__ inline void load8(const typename E::store* p, float (&f)[8]) {
  typename E::store v[8];
  __builtin_memcpy(v, p, sizeof v);
#pragma unroll
  for (int e = 0; e < 8; ++e) f[e] = E::widen(v[e]);
}
template <int N>
__device__ inline void load_f(const float* p, float (&f)[N]) {
  __builtin_memcpy(f, p, 4 * N);
}

// How the pairs of a rotation lie among a lane's 8 channels: all its pairs are
// its own (NEXT), the other halves are 8 channels elsewhere (HALF), or anything.
enum Turn { NONE, NEXT, HALF, ANY };

// Rotates 8 channels from c on; src: the row (for the other half of a pair),
// cs and sn: the angle's rows.
template <class E, Turn TURN>
__device__ inline void rotate(const typename E::store* src, const float* cs, const float* sn, int c, int rot, int pairs,
                              float (&x)[8]) {
  const int half = rot >> 1;
  if (c >= rot) return;
  if (TURN == NEXT) {
    float co[4], si[4];
    load_f(cs + (c >> 1), co);
    load_f(sn + (c >> 1), si);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float u = x[2 * e], v = x[2 * e + 1];
      x[2 * e] = u * co[e] - v * si[e];
      x[2 * e + 1] = v * co[e] + u * si[e];
    }
  } else if (TURN == HALF) {
    const bool low = c < half;
    const int j = low ? c : c - half;
    float o[8], co[8], si[8];
    load8<E>(src + (low ? c + half : j), o);
    load_f(cs + j, co);
    load_f(sn + j, si);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float a = x[e] * co[e], b = o[e] * si[e];
      x[e] = low ? a - b : a + b;
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int ch = c + e;
      if (ch < rot) {
        // the first of a pair is turned with its second, the second with the first
        const bool first = pairs ? (ch & 1) == 0 : ch < half;
        const int j = pairs ? ch >> 1 : first ? ch : ch - half, other = pairs ? ch ^ 1 : first ? ch + half : j;
        const float a = x[e] * cs[j], b = E::widen(src[other]) * sn[j];
        x[e] = first ? a - b : a + b;
      }
    }
  }
}

// d[j] of lane group g: 4 tokens (from 4 g on) of channel j.  Afterwards
// d[4 * i + t] of lane group g: tokens 4 t .. of channel 2 g + i.
__device__ inline void transpose(uint32_t (&d)[8]) {
  uint32_t e[8];
#pragma unroll
  for (int j = 0; j < 4; ++j) {  // lanes below 32 keep channels 0-3, the others 4-7
    const auto p = __builtin_amdgcn_permlane32_swap(d[j], d[j + 4], false, false);
    e[j] = p[0];      // of groups 0 and 1 (this lane's g % 2)
    e[4 + j] = p[1];  // of groups 2 and 3
  }
#pragma unroll
  for (int h = 0; h < 2; ++h)    // token groups 2 h, 2 h + 1
#pragma unroll
    for (int i = 0; i < 2; ++i) {  // even groups keep channels 0, 1, odd ones 2, 3
      const auto p = __builtin_amdgcn_permlane16_swap(e[4 * h + i], e[4 * h + i + 2], false, false);
      d[4 * i + 2 * h] = p[0];
      d[4 * i + 2 * h + 1] = p[1];
    }
}

// four codes, as many multiplied by 2^-shrink
__device__ inline uint32_t shrunk(uint32_t w, float less) {
  const tok_f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
  return codes2(a[0] * less, a[1] * less) | codes2(b[0] * less, b[1] * less) << 16;
}

template <class E, int NP, Turn TURN>  // NP: 1, or 2 beyond 128 channels
__global__ __launch_bounds__(256, NP == 1 && TURN != ANY ? 4 : 2) void kv_append_k(AppendArgs a) {
  typedef typename E::store S;
  const int lane = threadIdx.x & 63, g = lane >> 4, c0 = (lane & 15) * 8;
  const int64_t b = blockIdx.z;
  const int heads = static_cast<int>(a.c.heads), D = static_cast<int>(a.c.dim);
  // one wave a head: keys, values, then queries
  const int unit = __builtin_amdgcn_readfirstlane(static_cast<int>(blockIdx.y) * 4 + (threadIdx.x >> 6));
  if (unit >= 2 * heads + static_cast<int>(a.q_out ? a.q_heads : 0)) return;
  const int what = unit < heads ? 0 : unit < 2 * heads ? 1 : 2;
  const int head = unit - what * heads;

  // this sequence's rows and places
  int64_t row0 = a.b.cu[b], row1 = a.b.cu[b + 1];
  const int64_t len = a.b.len[b];
  row0 = row0 < 0 ? 0 : row0;
  row1 = row1 > a.b.T ? a.b.T : row1;
  const int64_t n = row1 - row0;
  if (n <= 0) return;
  const int64_t start = len - n;  // place of the first new token; negative if len is too short
  // floor of the first and last place over 16
  const int64_t first = start >> 4, last = (len - 1) >> 4;

  const S* src = static_cast<const S*>(what == 0 ? a.k : what == 1 ? a.v : a.q) + static_cast<int64_t>(head) * D;
  const int64_t ld = what == 0 ? a.ld_k : what == 1 ? a.ld_v : a.ld_q;
  const int rot = (what != 1 && TURN != NONE) ? static_cast<int>(a.r.rot) : 0;
  const int nb = static_cast<int>(a.c.page) >> 4;

  for (int64_t blk = first + blockIdx.x; blk <= last; blk += gridDim.x) {
    const int64_t p0 = blk * 16;
    const int lo = start > p0 ? static_cast<int>(start - p0) : 0;
    const int hi = len - p0 < 16 ? static_cast<int>(len - p0) : 16;
    const int64_t r0 = row0 + (p0 - start);  // row of place 0 of the block (valid from lo to hi)
    // the block's page; tokens without a valid one are not stored
    int64_t at = -1;  // of the block among the cache's
    if (what < 2 && blk >= 0) {
      const int64_t col = blk / nb;
      if (col < a.b.cols) {
        const int64_t page = a.b.table[b * a.b.cols + col];
        if (page >= 0 && page < a.c.pages) at = (page * heads + head) * nb + (blk - col * nb);
      }
    }
    float x[4][NP][8];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const int place = 4 * g + t;
      const bool in = place >= lo && place < hi;
#pragma unroll
      for (int i = 0; i < NP; ++i) {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[t][i][e] = 0.f;
        if (in && c0 + 128 * i < D) load8<E>(src + (r0 + place) * ld + c0 + 128 * i, x[t][i]);
      }
    }
    float* scale = nullptr;
    uint8_t* codes = nullptr;
    int old = -126;
    tok_u32x4 was[NP][2];  // v: this lane's two rows of earlier and later tokens
    if (at >= 0) {
      scale = (what == 0 ? a.c.k_scale : a.c.v_scale) + at;
      codes = static_cast<uint8_t*>(what == 0 ? a.c.k : a.c.v) + at * D * 16;
      if (lo > 0) old = static_cast<int>((__float_as_uint(*scale) >> 23) & 255u) - 127;
      if (what == 1 && (lo > 0 || hi < 16)) {
#pragma unroll
        for (int i = 0; i < NP; ++i)
#pragma unroll
          for (int e = 0; e < 2; ++e)
            if (c0 + 128 * i < D) was[i][e] = *reinterpret_cast<const tok_u32x4*>(codes + (c0 + 128 * i + 2 * g + e) * 16);
      }
    }
    if (TURN != NONE && rot) {
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        // two tokens' angles at a time: registers for four waves a SIMD
        if (t & 1) __builtin_amdgcn_sched_barrier(0);
        const int place = 4 * g + t;
        if (place < lo || place >= hi) continue;
        const int64_t row = a.r.pos ? a.r.pos[r0 + place] : p0 + place;
        const bool ok = row >= 0 && row < a.r.rows;
        const float* cs = a.r.cos + (ok ? row : 0) * (rot >> 1);
        const float* sn = a.r.sin + (ok ? row : 0) * (rot >> 1);
#pragma unroll
        for (int i = 0; i < NP; ++i) {
          if (c0 + 128 * i < D) rotate<E, TURN>(src + (r0 + place) * ld, cs, sn, c0 + 128 * i, rot, a.r.pairs, x[t][i]);
          if (!ok) {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[t][i][e] = __builtin_nanf("");
          }
        }
      }
    }
    if (what == 2) {
      S* out = static_cast<S*>(a.q_out) + static_cast<int64_t>(head) * D;
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const int place = 4 * g + t;
#pragma unroll
        for (int i = 0; i < NP; ++i) {
          const int c = c0 + 128 * i;
          if (place < lo || place >= hi || c >= D) continue;
          S v[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = E::narrow(x[t][i][e]);
          __builtin_memcpy(out + (r0 + place) * (a.q_heads * D) + c, v, sizeof v);
        }
      }
      continue;
    }
    if (at < 0) continue;

    float top = 0.f;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int i = 0; i < NP; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float m = fabsf(x[t][i][e]);
          top = fmaxf(top, m < kInf ? m : 0.f);
        }
    int ex = exponent_for(wave_max(top));
    old = old < -126 ? -126 : old > 127 ? 127 : old;
    ex = ex > old ? ex : old;
    const int shrink = lo > 0 ? ex - old : 0;  // earlier codes are multiplied by 2^-shrink
    // 2^-ex as two factors: 2^-127 is no normal number
    const float inv = pow2(-ex < -126 ? -126 : -ex), fix = ex > 126 ? 0.5f : 1.f;
    const float less = shrink > 126 ? 0.f : pow2(-shrink);
    if (lane == 0) *scale = pow2(ex);

    if (what == 0) {
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const int place = 4 * g + t;
#pragma unroll
        for (int i = 0; i < NP; ++i) {
          const int c = c0 + 128 * i;
          if (c >= D || place >= hi) continue;
          tok_u32x2* p = reinterpret_cast<tok_u32x2*>(codes + static_cast<int64_t>(place) * D + c);
          if (place >= lo) {
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = x[t][i][e] * inv * fix;
            *p = tok_u32x2{codes2(v[0], v[1]) | codes2(v[2], v[3]) << 16, codes2(v[4], v[5]) | codes2(v[6], v[7]) << 16};
          } else if (shrink) {
            const tok_u32x2 w = *p;
            *p = tok_u32x2{shrunk(w[0], less), shrunk(w[1], less)};
          }
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        uint32_t d[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          float v[4];
#pragma unroll
          for (int t = 0; t < 4; ++t) v[t] = x[t][i][e] * inv * fix;
          d[e] = codes2(v[0], v[1]) | codes2(v[2], v[3]) << 16;
        }
        transpose(d);
        if (c0 + 128 * i >= D) continue;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          tok_u32x4 w;
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            w[q] = d[4 * e + q];
            if (lo > 0 || hi < 16) {
              uint32_t before = 0, now = 0;  // bytes of earlier and of new tokens
#pragma unroll
              for (int t = 0; t < 4; ++t) {
                if (4 * q + t < lo) before |= 255u << (8 * t);
                if (4 * q + t >= lo && 4 * q + t < hi) now |= 255u << (8 * t);
              }
              uint32_t o = was[i][e][q];
              if (shrink) o = (o & ~before) | (shrunk(o, less) & before);
              w[q] = (w[q] & now) | (o & ~now);
            }
          }
          *reinterpret_cast<tok_u32x4*>(codes + (c0 + 128 * i + 2 * g + e) * 16) = w;
        }
      }
    }
  }
}

template <class E, int NP>
hipError_t typed(const AppendArgs& a, dim3 grid, hipStream_t s) {
  auto k = !a.r.cos                                ? kv_append_k<E, NP, NONE>
           : a.r.pairs && a.r.rot % 8 == 0         ? kv_append_k<E, NP, NEXT>
           : !a.r.pairs && a.r.rot % 16 == 0       ? kv_append_k<E, NP, HALF>
                                                   : kv_append_k<E, NP, ANY>;
  hipLaunchKernelGGL(k, grid, dim3(256), 0, s, a);
  return hipGetLastError();
}
template <class E>
hipError_t typed(const AppendArgs& a, dim3 grid, hipStream_t s) {
  return a.c.dim <= 128 ? typed<E, 1>(a, grid, s) : typed<E, 2>(a, grid, s);
}

}  // namespace

hipError_t launch_kv_append(const AppendArgs& a, int dtype, hipStream_t s) {
  if (a.b.B == 0 || a.b.T == 0 || a.b.max_new == 0) return hipSuccess;
  // n new tokens touch at most (n + 14) / 16 + 1 blocks; no sequence has more
  // than T, and blocks past the 2^23 of a launch's threads are taken in turn
  const int64_t n = a.b.max_new < a.b.T ? a.b.max_new : a.b.T, most = int64_t(1) << 23;
  const int64_t bx = (n + 14) / 16 + 1 < most ? (n + 14) / 16 + 1 : most;
  const int64_t units = 2 * a.c.heads + (a.q_out ? a.q_heads : 0), by = (units + 3) / 4;
  if (a.b.B > 65535 || by > 65535) return hipErrorInvalidConfiguration;
  const dim3 grid(static_cast<unsigned>(bx), static_cast<unsigned>(by), static_cast<unsigned>(a.b.B));
  return dtype == C3C_DTYPE_BF16  ? typed<ElemBf16>(a, grid, s)
         : dtype == C3C_DTYPE_F16 ? typed<ElemF16>(a, grid, s)
                                  : typed<ElemF32>(a, grid, s);
}

}  // namespace c3c
