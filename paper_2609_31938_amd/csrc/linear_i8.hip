// Matrix product in 8-bit integers:
//   y[m][n] = (sum_k x[m][k] w[n][k]) * x_scale[m] * w_scale[n] + bias[n]
// with x int8 [M][ldx], w int8 [N][K] (both K-contiguous) and an exact int32
// sum on v_mfma_i32_16x16x64_i8: the weights are the A operand (rows n), the
// tokens B (columns m), so that a lane's four results are four consecutive n
// of one token and are stored together.
//
// What happens to a result before its rounding is compiled in (EPI): nothing;
// an activation, a gate and a residual; or, with weights of 2 N rows, the
// product of an activation of one half and the other (gated).  A gated tile takes
// its rows half from each half of the weights, so that both results of a
// channel meet in one lane.
//
// skinny: at most 32 tokens.  The weights are read once, straight into
//   registers (no tile of them is used twice), by 4 waves that share 16 rows
//   and take every fourth 128-byte piece of K, 8 of them in flight; their sums
//   meet in LDS.  Up to 4 tokens of floats are quantised in the same kernel, by
//   every workgroup for itself, which saves a launch and its wait.  The first
//   weights are asked for before the tokens; loads return in order, so the
//   quantisation waits for them.
// tiled: BM x BN tiles, stages of 64 or 128 bytes of K in an LDS ring, the
//   fragments of the next 64 bytes read between the products of these.  The
//   largest tile takes two stages of 128 bytes (whole cache lines; 790 us for
//   32760 x 5120 x 5120 quantised normal values, 2.17 POP/s) over four of 64
//   (865 us).  What bounds it is the way to LDS: the loads alone take 710 us,
//   the products alone 620 (at the clock that power leaves them; 3.5 PFLOP/s
//   with random operands in registers).  With 16-byte rows the stages are loaded
//   straight into LDS (the buffer's bounds make rows past M or N and pieces
//   past K zero); rows of any other length are copied to such rows first where
//   there is workspace for them (linear_pads), else they go through registers
//   (4096 x 4095, 8192 tokens: 292 us).
#include "token_dev.h"
#include "tokens_internal.h"

namespace c3c {
namespace {

typedef __attribute__((address_space(3))) void lds_void;

struct Codes {};  // int8 activations, where float ones name their type
template <class E>
struct is_codes {
  static constexpr bool value = false;
};
template <>
struct is_codes<Codes> {
  static constexpr bool value = true;
};

enum { PLAIN = LinearEpilogue::kPlain, EPILOGUE = LinearEpilogue::kEpilogue, GATED = LinearEpilogue::kGated };

struct LinArgs {
  const int8_t *x, *w;  // x: also the address of float tokens (linear_skinny)
  const float *x_scale, *w_scale, *bias;
  void* y;
  int32_t* part;  // [splits][M][N] (gated: 2 N), or NULL: y is written
  int64_t M, N, K, ldx;
  int tiles_m, tiles_n;
  int splits;     // along K, in stages
  int y_dtype;
  int64_t first;  // workgroup of this launch
  LinearEpilogue e;
};

// w_scale and bias of four consecutive channels (the last one's past N), gated
// also of those N further on
template <int EPI>
struct Channels {
  static constexpr int H = EPI == GATED ? 2 : 1;
  float s[H][4], b[H][4];
};
template <int EPI>
__device__ inline Channels<EPI> channels(const LinArgs& a, int64_t n) {
  Channels<EPI> c;
#pragma unroll
  for (int h = 0; h < c.H; ++h) {
    const float *ws = a.w_scale + h * a.N, *bias = a.bias ? a.bias + h * a.N : nullptr;
    if (n + 4 <= a.N) {
      __builtin_memcpy(c.s[h], ws + n, 16);
      if (bias) __builtin_memcpy(c.b[h], bias + n, 16);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int64_t at = n + i < a.N ? n + i : a.N - 1;
        c.s[h][i] = ws[at];
        if (bias) c.b[h][i] = bias[at];
      }
    }
  }
  return c;
}

// z Phi(z), Phi the normal distribution: Phi(-a) = exp(-a^2 / 2) R(a) for a >= 0,
// and 1 - that for a > 0 (z/2 (1 + erf) would cancel where z < 0: at -5 to 4% of the
// result).  R, between 1/2 and 1 / (a sqrt(2 pi)), is t times a polynomial in t = 1 /
// (1 + 0.35 a): the best one of degree 8, fitted to erfc in 64 bits (relative
// error 2^-25 up to a = 15, where exp(-a^2 / 2) is 0).  Roundings leave 2^-21 for
// |z| < 1 and 1.3 z^2 2^-24 of the exponent.  The library's erfc is as good and
// longer: with it 8192 tokens x 8192 channels of 4096 take 353 us, so 309.
__device__ inline float gelu(float z) {
  const float a = fabsf(z), t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.35f, a, 1.f));
  constexpr float c[9] = {0.139621258f, 0.13986434f, 0.119815491f, 0.105574816f, -0.023263881f,
                          0.159392983f, -0.255901933f, 0.144060835f, -0.0291639324f};
  float r = c[8];
#pragma unroll
  for (int i = 7; i >= 0; --i) r = __builtin_fmaf(r, t, c[i]);
  const float below = __builtin_amdgcn_exp2f(-0.721347520f * (a * a)) * (r * t);
  return z * (z < 0.f ? below : 1.f - below);
}

__device__ inline float activate(int act, float z) {
  if (act == C3C_ACT_NONE) return z;
  if (act == C3C_ACT_GELU) return gelu(z);
  // z / (1 + exp(-u)); u = z, or 2 sqrt(2 / pi) (z + 0.044715 z^3), since
  // (1 + tanh v) / 2 = 1 / (1 + exp(-2 v))
  const float u = act == C3C_ACT_SILU ? z : 1.59576912f * (z + 0.044715f * z * z * z);
  return z * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.44269504f * u));
}

// four values of a row from p, those past N being 0
__device__ inline void get4(int dtype, const void* p, int64_t at, int64_t left, float (&f)[4]) {
  if (dtype == C3C_DTYPE_F32) {
    const float* q = static_cast<const float*>(p) + at;
    if (left >= 4) {
      __builtin_memcpy(f, q, 16);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) f[i] = i < left ? q[i] : 0.f;
    }
  } else {
    const uint16_t* q = static_cast<const uint16_t*>(p) + at;
    uint16_t h[4];
    if (left >= 4) {
      __builtin_memcpy(h, q, 8);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) h[i] = i < left ? q[i] : uint16_t(0);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = dtype == C3C_DTYPE_BF16 ? ElemBf16::widen(h[i]) : ElemF16::widen(h[i]);
  }
}

// eight values of a row as they are stored, those past N being 0
struct Stored8 {
  tok_u32x4 a, b;  // 16-bit types: a alone
};
__device__ inline Stored8 stored8(int dtype, const void* p, int64_t at, int64_t left) {
  Stored8 x = {{0u, 0u, 0u, 0u}, {0u, 0u, 0u, 0u}};
  if (dtype == C3C_DTYPE_F32) {
    const float* q = static_cast<const float*>(p) + at;
    if (left >= 8) {
      __builtin_memcpy(&x.a, q, 16);
      __builtin_memcpy(&x.b, q + 4, 16);
    } else {
#pragma unroll
      for (int i = 0; i < 7; ++i)
        if (i < left) (i < 4 ? x.a : x.b)[i & 3] = __float_as_uint(q[i]);
    }
  } else {
    const uint16_t* q = static_cast<const uint16_t*>(p) + at;
    if (left >= 8) {
      __builtin_memcpy(&x.a, q, 16);
    } else {
#pragma unroll
      for (int i = 0; i < 7; ++i)
        if (i < left) x.a[i >> 1] |= static_cast<uint32_t>(q[i]) << (16 * (i & 1));
    }
  }
  return x;
}
// the same of U rows; whole: they all have eight (loads behind conditions of
// single lanes are waited for one by one)
template <int U>
__device__ inline void stored_rows(int dtype, const void* p, const int64_t (&at)[U], int64_t left, bool whole, Stored8 (&x)[U]) {
  if (whole && dtype == C3C_DTYPE_F32) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      __builtin_memcpy(&x[u].a, static_cast<const float*>(p) + at[u], 16);
      __builtin_memcpy(&x[u].b, static_cast<const float*>(p) + at[u] + 4, 16);
    }
  } else if (whole) {
#pragma unroll
    for (int u = 0; u < U; ++u) __builtin_memcpy(&x[u].a, static_cast<const uint16_t*>(p) + at[u], 16);
  } else {
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (left > 0) x[u] = stored8(dtype, p, at[u], left);
  }
}
__device__ inline float value(int dtype, const Stored8& x, int i) {
  if (dtype == C3C_DTYPE_F32) return __uint_as_float((i < 4 ? x.a : x.b)[i & 3]);
  const uint16_t h = static_cast<uint16_t>(x.a[i >> 1] >> (16 * (i & 1)));
  return dtype == C3C_DTYPE_BF16 ? ElemBf16::widen(h) : ElemF16::widen(h);
}

// What four results meet: the residual and the gates (EPILOGUE).
struct Beside {
  float residual[4], gate[4];
};
template <int EPI>
__device__ inline Beside beside(const LinArgs& a, int64_t m, int64_t n) {
  Beside x;
  if constexpr (EPI == EPILOGUE) {
    if (a.e.residual) get4(a.y_dtype, a.e.residual, m * a.N + n, a.N - n, x.residual);
    if (a.e.gate) get4(a.y_dtype, a.e.gate, static_cast<int64_t>(static_cast<uint32_t>(m) / a.e.rows_per_gate) * a.N + n, a.N - n, x.gate);
  }
  return x;
}

// four results of token m, of which those below N are stored; gated: v[0] those
// of the first half of the weights, v[1] of the second
template <int EPI>
__device__ inline void put4(const LinArgs& a, int64_t m, int64_t n, const tok_i32x4 (&v)[Channels<EPI>::H], float s,
                            const Channels<EPI>& c, const Beside& x) {
  float f[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float z[Channels<EPI>::H];
#pragma unroll
    for (int h = 0; h < Channels<EPI>::H; ++h) {
      z[h] = static_cast<float>(v[h][i]) * s * c.s[h][i];
      if (a.bias) z[h] += c.b[h][i];
    }
    f[i] = EPI == PLAIN ? z[0] : activate(a.e.act, z[0]);
    if constexpr (EPI == GATED) f[i] *= z[1];
    if constexpr (EPI == EPILOGUE) {
      if (a.e.gate) f[i] *= x.gate[i];
      if (a.e.residual) f[i] = __builtin_fmaf(a.e.alpha, x.residual[i], f[i]);
    }
  }
  const int64_t at = m * a.N + n;
  if (a.y_dtype == C3C_DTYPE_F32) {
    float* p = static_cast<float*>(a.y) + at;
    if (n + 4 <= a.N) {
      __builtin_memcpy(p, f, 16);
    } else {
      for (int i = 0; i < 3; ++i)
        if (n + i < a.N) p[i] = f[i];
    }
  } else {
    uint16_t h[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) h[i] = a.y_dtype == C3C_DTYPE_BF16 ? ElemBf16::narrow(f[i]) : ElemF16::narrow(f[i]);
    uint16_t* p = static_cast<uint16_t*>(a.y) + at;
    if (n + 4 <= a.N) {
      __builtin_memcpy(p, h, 8);
    } else {
      for (int i = 0; i < 3; ++i)
        if (n + i < a.N) p[i] = h[i];
    }
  }
}

// 16 bytes of a row from p, of which the first m exist (AL: 0 or 16 of them,
// aligned); the others are 0
template <bool AL>
__device__ inline tok_i32x4 piece(const int8_t* p, int64_t m) {
  tok_i32x4 v = {0, 0, 0, 0};
  if (AL) {
    if (m > 0) v = *reinterpret_cast<const tok_i32x4*>(p);
  } else if (m >= 16) {
    __builtin_memcpy(&v, p, 16);
  } else if (m > 0) {  // rows past the last would take all the branches in vain
#pragma unroll
    for (int e = 0; e < 15; ++e)
      if (e < m) v[e >> 2] |= (static_cast<int32_t>(p[e]) & 255) << (8 * (e & 3));
  }
  return v;
}

constexpr int kFusedBytes = 32768;  // of quantised rows in LDS

// MT tiles of 16 tokens.  E: int8 for codes, or the type of float tokens that
// the kernel quantises (MT = 1, at most kFusedBytes of codes).
// Three workgroups a compute unit: gated, of floats, it would have registers for
// two (1 token, 2 x 10240 channels of 4096: 24.0 us, so 20.6).
template <class E, int MT, bool AL, int EPI>
__global__ __launch_bounds__(256, (AL && EPI == GATED && MT == 1 ? 3 : 1)) void linear_skinny(LinArgs a) {
  constexpr bool FUSE = !is_codes<E>::value;
  constexpr int H = Channels<EPI>::H;
  __shared__ tok_i32x4 sums[3][MT][H][64];
  __shared__ __align__(16) int8_t rows[FUSE ? kFusedBytes : 16];
  __shared__ float tops[4][16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int r = lane & 15, g = lane >> 4;
  const int64_t n0 = (a.first + blockIdx.x) * 16;
  const int64_t nr = n0 + r < a.N ? n0 + r : a.N - 1;
  const int8_t* wp = a.w + nr * a.K;
  constexpr int U = H == 2 || 8 / MT < 4 ? 4 : 8 / MT;  // stages in flight
  tok_i32x4 wv[U][2][H];
  auto fetch = [&](int64_t k0) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int64_t k = k0 + 512 * u + 64 * j + 16 * g;
#pragma unroll
        for (int h = 0; h < H; ++h) wv[u][j][h] = piece<AL>(wp + h * a.N * a.K + k, a.K - k);
      }
  };
  fetch(wave * 128);
  const int pitch = static_cast<int>((a.K + 15) / 16 * 16);
  if constexpr (FUSE) {
    typedef typename E::store S;
    const S* x = reinterpret_cast<const S*>(a.x);
    const int M = static_cast<int>(a.M), K = static_cast<int>(a.K);
    for (int m = 0; m < M; ++m) {
      float top = 0.f;
      for (int k = threadIdx.x * E::VEC; k < K; k += 256 * E::VEC) {
        float f[E::VEC];
        load_vec<E>(x + m * a.ldx + k, K - k, f);
#pragma unroll
        for (int e = 0; e < E::VEC; ++e) top = fmaxf(top, magnitude(f[e]));
      }
      top = wave_max(top);
      if (lane == 0) tops[wave][m] = top;
    }
    __syncthreads();
    for (int m = 0; m < M; ++m) {
      const float top = fmaxf(fmaxf(tops[0][m], tops[1][m]), fmaxf(tops[2][m], tops[3][m])), s = row_scale(top);
      for (int k = threadIdx.x * E::VEC; k < pitch; k += 256 * E::VEC) {
        float f[E::VEC];
        load_vec<E>(x + m * a.ldx + k, K - k, f);
        store_codes<E::VEC>(rows + m * pitch + k, E::VEC, f, s, EPI == PLAIN ? 0.f : top);
      }
    }
    __syncthreads();
  }
  const int8_t* xp[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    const int64_t m = t * 16 + r < a.M ? t * 16 + r : a.M - 1;
    xp[t] = FUSE ? rows + m * pitch : a.x + m * a.ldx;
  }
  tok_i32x4 acc[MT][H];
#pragma unroll
  for (int t = 0; t < MT; ++t)
#pragma unroll
    for (int h = 0; h < H; ++h) acc[t][h] = tok_i32x4{0, 0, 0, 0};
  for (int64_t k0 = wave * 128; k0 < a.K; k0 += 512 * U) {
    tok_i32x4 now[U][2][H];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int h = 0; h < H; ++h) now[u][j][h] = wv[u][j][h];
    if (k0 + 512 * U < a.K) fetch(k0 + 512 * U);
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int64_t k = k0 + 512 * u + 64 * j + 16 * g;
#pragma unroll
        for (int t = 0; t < MT; ++t) {
          const tok_i32x4 xv = FUSE ? piece<true>(xp[t] + k, a.K - k) : piece<AL>(xp[t] + k, a.K - k);
#pragma unroll
          for (int h = 0; h < H; ++h) acc[t][h] = __builtin_amdgcn_mfma_i32_16x16x64_i8(now[u][j][h], xv, acc[t][h], 0, 0, 0);
        }
      }
  }
  if (wave > 0) {
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
      for (int h = 0; h < H; ++h) sums[wave - 1][t][h][lane] = acc[t][h];
  }
  __syncthreads();
  if (wave > 0) return;
#pragma unroll
  for (int t = 0; t < MT; ++t) {
#pragma unroll
    for (int w = 0; w < 3; ++w)
#pragma unroll
      for (int h = 0; h < H; ++h) acc[t][h] += sums[w][t][h][lane];
    const int64_t m = t * 16 + r, n = n0 + g * 4;
    if (m >= a.M || n >= a.N) continue;
    const float s = FUSE ? row_scale(fmaxf(fmaxf(tops[0][m], tops[1][m]), fmaxf(tops[2][m], tops[3][m]))) : a.x_scale[m];
    put4<EPI>(a, m, n, acc[t], s, channels<EPI>(a, n), beside<EPI>(a, m, n));
  }
}

// Place of piece c of row r in its LDS row: the pieces of one column spread
// over all banks.
template <int BK>
__device__ inline int spread(int r, int c) {
  return BK == 128 ? c ^ (r & 7) : c ^ (r >> 2 & 3);
}

// vmcnt(n), with the other counters left alone
#define C3C_VMCNT(n) __builtin_amdgcn_s_waitcnt(((n) & 15) | (((n) >> 4) << 14) | (7 << 4) | (15 << 8))

// (BM / WM) * (BN / WN) waves, each with a WM x WN part of the tile.
// Gated, the rows of w in a wave's part are half of one half, half of the other.
template <int BM, int BN, int WM, int WN, int BK, int NS, bool AL, int EPI>
__global__ __launch_bounds__((BM / WM) * (BN / WN) * 64) void linear_tiled(LinArgs a) {
  constexpr int H = Channels<EPI>::H, ON = BN / H;  // channels of y
  constexpr int NW = (BM / WM) * (BN / WN);
  constexpr int MT = WM / 16, NT = WN / 16;
  constexpr int ROWS = BM + BN;              // rows of w, then rows of x
  constexpr int KS = BK / 64;                // matrix-core steps a stage
  constexpr int LR = 1024 / BK;              // rows of a 1024-byte load
  constexpr int LOADS = ROWS / LR / NW;      // loads a wave and stage
  static_assert(ROWS % (LR * NW) == 0 && BN % LR == 0, "whole loads");
  __shared__ __align__(16) int8_t lds[NS * ROWS * BK];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r = lane & 15, g = lane >> 4;

  // tiles in an order that keeps each of the 8 L2 caches on neighbouring
  // ones: workgroup b runs on cache b % 8, which gets a run of consecutive
  // tiles, walked in columns of 6 tiles of tokens (32760 x 5120 x 5120, in
  // one sitting: 794 us, columns of 4 809, of 8 857; other shapes not tried)
  const int total = a.tiles_m * a.tiles_n;
  int b = static_cast<int>(a.first) + blockIdx.x;
  const int split = b / total;
  b -= split * total;
  {
    const int each = total / 8, rest = total % 8, c = b % 8, i = b / 8;
    b = c * each + (c < rest ? c : rest) + i;
  }
  constexpr int COL = 6;
  const int colg = b / (COL * a.tiles_n), in = b - colg * COL * a.tiles_n;
  const int high = a.tiles_m - colg * COL < COL ? a.tiles_m - colg * COL : COL;
  const int tm = colg * COL + in % high, tn = in / high;
  const int64_t m0 = static_cast<int64_t>(tm) * BM, n0 = static_cast<int64_t>(tn) * ON;

  const int stages = static_cast<int>((a.K + BK - 1) / BK);
  const int s0 = static_cast<int>(static_cast<int64_t>(stages) * split / a.splits);
  const int count = static_cast<int>(static_cast<int64_t>(stages) * (split + 1) / a.splits) - s0;

  const int64_t nrows = a.N - n0 < ON ? a.N - n0 : ON, mrows = a.M - m0 < BM ? a.M - m0 : BM;
  const int8_t* wb = a.w + n0 * a.K;
  const int8_t* xb = a.x + m0 * a.ldx;
  // the part of a load that this lane brings: row and piece
  const int lrow = lane / (BK / 16), lpiece = spread<BK>(lrow, lane % (BK / 16));
  const __amdgpu_buffer_rsrc_t wrs = __builtin_amdgcn_make_buffer_rsrc(
      const_cast<int8_t*>(wb), 0, static_cast<int>(nrows * a.K), 0x00020000);
  const int64_t half = EPI == GATED ? a.N * a.K : 0;  // to the rows of the second half
  const __amdgpu_buffer_rsrc_t xrs = __builtin_amdgcn_make_buffer_rsrc(
      const_cast<int8_t*>(xb), 0, static_cast<int>((mrows - 1) * a.ldx + a.K), 0x00020000);
  tok_i32x4 staged[LOADS];  // !AL
  // load i of stage st of this split
  auto load = [&](int st, int i) __attribute__((always_inline)) {
    const int k = (s0 + st) * BK + lpiece * 16, buf = st % NS;
    const int row = (i * NW + wave) * LR;  // of ROWS, uniform; whole loads are of w or of x
    const bool isw = row < BN;
    // of w: the row within its half, and which half (whole loads are of one half)
    const bool second = EPI == GATED && row / (WN / 2) % 2 == 1;
    const int wrow = EPI == GATED ? row / WN * (WN / 2) + row % (WN / 2) : row;
    const int rr = (isw ? wrow : row - BN) + lrow;
    if (AL) {
      const int ld = static_cast<int>(isw ? a.K : a.ldx);
      // past K: a sign bit takes the offset out of every buffer
      const int off = (rr * ld + k) | ((static_cast<int>(a.K) - 1 - k) & static_cast<int>(0x80000000u));
      lds_void* to = (lds_void*)(lds + buf * ROWS * BK + row * BK);
      if constexpr (EPI == GATED) {
        // (a choice among three variables is compiled into scratch memory)
        const int8_t* base = isw ? wb + (second ? half : 0) : xb + 0;
        const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(
            const_cast<int8_t*>(base), 0, static_cast<int>(isw ? nrows * a.K : (mrows - 1) * a.ldx + a.K), 0x00020000);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, to, 16, off, 0, 0, 0);
      } else {
        __builtin_amdgcn_raw_ptr_buffer_load_lds(isw ? wrs : xrs, to, 16, off, 0, 0, 0);
      }
    } else {
      const int64_t ld = isw ? a.K : a.ldx;
      const bool ok = rr < (isw ? nrows : mrows);
      const int8_t* base = isw ? wb + (second ? half : 0) : xb + 0;
      staged[i] = piece<false>(base + (ok ? rr * ld + k : 0), ok ? a.K - k : 0);
    }
  };
  auto settle = [&](int st) __attribute__((always_inline)) {  // !AL
#pragma unroll
    for (int i = 0; i < LOADS; ++i)
      *reinterpret_cast<tok_i32x4*>(lds + (st % NS) * ROWS * BK + (i * NW + wave) * LR * BK + lane * 16) = staged[i];
  };

  const int wm = wave % (BM / WM) * WM, wn = wave / (BM / WM) * WN;
  struct Frags {
    tok_i32x4 w[NT], x[MT];
  };
  // fragment n of NT + MT of step ks of a stage; every fragment row is
  // congruent to r modulo 16
  auto read = [&](int st, int ks, int n, Frags& f) __attribute__((always_inline)) {
    const int8_t* base = lds + (st % NS) * ROWS * BK + r * BK + spread<BK>(r, ks * 4 + g) * 16;
    if (n < NT)
      f.w[n] = *reinterpret_cast<const tok_i32x4*>(base + (wn + n * 16) * BK);
    else
      f.x[n - NT] = *reinterpret_cast<const tok_i32x4*>(base + (BN + wm + (n - NT) * 16) * BK);
  };
  tok_i32x4 acc[NT][MT];
#pragma unroll
  for (int i = 0; i < NT; ++i)
#pragma unroll
    for (int j = 0; j < MT; ++j) acc[i][j] = tok_i32x4{0, 0, 0, 0};

  // One step: its products, the next step's fragments.  The last step of a
  // stage waits for stage st + 1 and, once every wave has read the last of
  // stage st, loads stage st + NS into its place.  Reads and products take
  // turns: reads all at once would keep LDS and the matrix cores busy one after
  // the other.  What is read and loaded past the last stage is never used.
  auto step = [&](int st, int ks, const Frags& cur, Frags& nxt) __attribute__((always_inline)) {
    const bool end = ks == KS - 1;
    if (end) {
      if (AL) C3C_VMCNT((NS - 2) * LOADS);  // stage st + 1 has landed: the loads behind it may be on their way
      asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    }
    constexpr int STEPS = NT + MT;
#pragma unroll
    for (int n = 0; n < STEPS; ++n) {
      __builtin_amdgcn_sched_barrier(0);
      read(end ? st + 1 : st, end ? 0 : ks + 1, n, nxt);
      if (end) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i)
          if (i * STEPS / LOADS == n) load(st + (AL ? NS : 2), i);
      }
#pragma unroll
      for (int e = n * NT * MT / STEPS; e < (n + 1) * NT * MT / STEPS; ++e)
        acc[e / MT][e % MT] = __builtin_amdgcn_mfma_i32_16x16x64_i8(cur.w[e / MT], cur.x[e % MT], acc[e / MT][e % MT], 0, 0, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
    if (end && !AL) settle(st + 2);
  };
  Frags fa, fb;
#pragma unroll
  for (int s = 0; s < (AL ? NS : 2); ++s) {
#pragma unroll
    for (int i = 0; i < LOADS; ++i) load(s, i);
    if (!AL) settle(s);
  }
  if (AL) C3C_VMCNT((NS - 1) * LOADS);
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
#pragma unroll
  for (int n = 0; n < NT + MT; ++n) read(0, 0, n, fa);
  if (KS == 2) {
    for (int st = 0; st < count; ++st) {
      step(st, 0, fa, fb);
      step(st, 1, fb, fa);
    }
  } else {
    for (int st = 0; st < count; st += 2) {
      step(st, 0, fa, fb);
      if (st + 1 < count) step(st + 1, 0, fb, fa);
    }
  }
  C3C_VMCNT(0);  // nothing is on its way into LDS when the workgroup ends

  float xs[MT];
  if (EPI == PLAIN && !a.part) {
#pragma unroll
    for (int j = 0; j < MT; ++j) {
      const int64_t m = m0 + wm + j * 16 + r;
      xs[j] = a.x_scale[m < a.M ? m : a.M - 1];
    }
  }
  constexpr int OT = NT / H;  // tiles of 16 channels of y
#pragma unroll
  for (int i = 0; i < OT; ++i) {
    const int64_t n = n0 + wn / H + i * 16 + g * 4;
    if (n >= a.N || (EPI != PLAIN && !a.part)) continue;
    Channels<EPI> c;
    if (!a.part) c = channels<EPI>(a, n);
#pragma unroll
    for (int j = 0; j < MT; ++j) {
      const int64_t m = m0 + wm + j * 16 + r;
      if (m >= a.M) continue;
      if (a.part) {
#pragma unroll
        for (int h = 0; h < H; ++h) {
          int32_t* p = a.part + ((split * a.M + m) * H + h) * a.N + n;
          if (n + 4 <= a.N) {
            __builtin_memcpy(p, &acc[i + h * OT][j], 16);
          } else {
            for (int e = 0; e < 3; ++e)
              if (n + e < a.N) p[e] = acc[i + h * OT][j][e];
          }
        }
      } else if constexpr (EPI == PLAIN) {
        const tok_i32x4 v[1] = {acc[i][j]};
        put4<EPI>(a, m, n, v, xs[j], c, Beside());
      }
    }
  }
  if constexpr (EPI == EPILOGUE) {
    // Onto a residual without an activation (of 16 bits, a whole tile, its tokens
    // under one row of gates): everything is read before anything is stored, since
    // a load is waited for with every store before it, and all workgroups are
    // here at once (32760 x 5120 x 5120: 900 us, through LDS 1017, without a residual
    // 790; loads past the caches 926).  The residual's 64 registers beside 128 sums
    // leave 136 bytes a lane in scratch memory, and a wave's loads take a quarter of
    // a line at a time: 3.7 GB are read, of which the residual is 0.3.
    const uint32_t group = static_cast<uint32_t>(m0) / a.e.rows_per_gate;
    if (!a.part && a.e.act == C3C_ACT_NONE && a.e.residual && a.y_dtype != C3C_DTYPE_F32 && n0 + BN <= a.N &&
        static_cast<uint32_t>(m0 + mrows - 1) / a.e.rows_per_gate == group) {
      const uint16_t* from = static_cast<const uint16_t*>(a.e.residual) + m0 * a.N + n0 + wn + g * 4;
      tok_u32x2 res[NT][MT];
#pragma unroll
      for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int j = 0; j < MT; ++j) {
          const int64_t row = wm + j * 16 + r < mrows ? wm + j * 16 + r : mrows - 1;
          __builtin_memcpy(&res[i][j], from + row * a.N + i * 16, 8);
        }
#pragma unroll
      for (int j = 0; j < MT; ++j) xs[j] = a.x_scale[m0 + (wm + j * 16 + r < mrows ? wm + j * 16 + r : mrows - 1)];
#pragma unroll
      for (int i = 0; i < NT; ++i) {
        const int64_t n = n0 + wn + i * 16 + g * 4;
        const Channels<EPI> c = channels<EPI>(a, n);
        float gate[4];
        if (a.e.gate) get4(a.y_dtype, a.e.gate, group * a.N + n, 4, gate);
#pragma unroll
        for (int j = 0; j < MT; ++j) {
          uint16_t h[4];
          __builtin_memcpy(h, &res[i][j], 8);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float z = static_cast<float>(acc[i][j][e]) * xs[j] * c.s[0][e];
            if (a.bias) z += c.b[0][e];
            if (a.e.gate) z *= gate[e];
            const float f = a.y_dtype == C3C_DTYPE_BF16 ? ElemBf16::widen(h[e]) : ElemF16::widen(h[e]);
            z = __builtin_fmaf(a.e.alpha, f, z);
            h[e] = a.y_dtype == C3C_DTYPE_BF16 ? ElemBf16::narrow(z) : ElemF16::narrow(z);
          }
          __builtin_memcpy(&res[i][j], h, 8);
        }
      }
      uint16_t* to = static_cast<uint16_t*>(a.y) + m0 * a.N + n0 + wn + g * 4;
#pragma unroll
      for (int j = 0; j < MT; ++j)
        if (wm + j * 16 + r < mrows) {
#pragma unroll
          for (int i = 0; i < NT; ++i) __builtin_memcpy(to + (wm + j * 16 + r) * a.N + i * 16, &res[i][j], 8);
        }
      return;
    }
  }
  if constexpr (EPI != PLAIN) {
    if (a.part) return;
    // The sums change places in LDS, where a wave now has room for 64 tokens of
    // its part: a lane takes 8 channels of one token after another, whose
    // residual, gates and results are whole 16-byte pieces.  In place, four
    // channels of many tokens a lane, the functions are unrolled 128 times and
    // the sums end in scratch memory (32760 x 5120 x 5120 onto a residual: 1564 us).
    constexpr int ROOM = WM < 64 ? WM : 64, OC = WN / H, LPR = OC / 8, RPI = 64 / LPR;
    constexpr int U = ROOM / RPI < 2 ? ROOM / RPI : 2;  // tokens of a lane at once
    static_assert(NW * ROOM * WN * 4 <= static_cast<int>(sizeof(lds)) && ROOM % (RPI * U) == 0, "room, whole rounds");
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");  // no wave reads a stage any more
    int8_t* const mine = lds + wave * ROOM * WN * 4;
    const int c8 = lane % LPR;
    const int64_t n = n0 + wn / H + c8 * 8;
    const bool whole = n0 + ON <= a.N;
    Channels<EPI> c[2] = {channels<EPI>(a, n < a.N ? n : 0), channels<EPI>(a, n + 4 < a.N ? n + 4 : 0)};
#pragma unroll
    for (int first = 0; first < MT; first += ROOM / 16) {
#pragma unroll
      for (int j = 0; j < ROOM / 16; ++j)
#pragma unroll
        for (int i = 0; i < NT; ++i)
          *reinterpret_cast<tok_i32x4*>(mine + (j * 16 + r) * WN * 4 + ((i * 4 + g) ^ (r & 7)) * 16) = acc[i][first + j];
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll 1
      for (int it = 0; it < ROOM / RPI; it += U) {
        // asked for together, as they are stored: y may be the residual
        Stored8 res[U], gate[U];
        int64_t m[U];
        int64_t at[U], gate_at[U];  // of rows that exist
#pragma unroll
        for (int u = 0; u < U; ++u) {
          m[u] = m0 + wm + first * 16 + (it + u) * RPI + lane / LPR;
          const int64_t row = m[u] < a.M ? m[u] : a.M - 1;
          at[u] = row * a.N + n;
          if constexpr (EPI == EPILOGUE) gate_at[u] = static_cast<int64_t>(static_cast<uint32_t>(row) / a.e.rows_per_gate) * a.N + n;
        }
        if constexpr (EPI == EPILOGUE) {
          if (a.e.residual) stored_rows(a.y_dtype, a.e.residual, at, a.N - n, whole, res);
          if (a.e.gate) stored_rows(a.y_dtype, a.e.gate, gate_at, a.N - n, whole, gate);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
          if (m[u] >= a.M) continue;
          const float s = a.x_scale[m[u]];
          const int row = (it + u) * RPI + lane / LPR;
#pragma unroll
          for (int p = 0; p < 2; ++p) {
            tok_i32x4 v[H];
#pragma unroll
            for (int h = 0; h < H; ++h)
              v[h] = *reinterpret_cast<const tok_i32x4*>(mine + row * WN * 4 + ((h * OC / 4 + c8 * 2 + p) ^ (row & 7)) * 16);
            Beside x;
            if constexpr (EPI == EPILOGUE) {
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                if (a.e.residual) x.residual[i] = value(a.y_dtype, res[u], 4 * p + i);
                if (a.e.gate) x.gate[i] = value(a.y_dtype, gate[u], 4 * p + i);
              }
            }
            if (n + 4 * p < a.N) put4<EPI>(a, m[u], n + 4 * p, v, s, c[p], x);
          }
        }
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
  }
}

// y from the partial sums of a split call: four results a thread.
template <int EPI>
__global__ __launch_bounds__(256) void linear_join(LinArgs a) {
  constexpr int H = Channels<EPI>::H;
  const int64_t quads = (a.N + 3) / 4;
  const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (i >= a.M * quads) return;
  const int64_t m = i / quads, n = i % quads * 4;
  const Beside x = beside<EPI>(a, m, n);
  tok_i32x4 v[H];
#pragma unroll
  for (int h = 0; h < H; ++h) v[h] = tok_i32x4{0, 0, 0, 0};
  for (int s = 0; s < a.splits; ++s) {
#pragma unroll
    for (int h = 0; h < H; ++h) {
      const int32_t* p = a.part + ((s * a.M + m) * H + h) * a.N + n;
      if (n + 4 <= a.N) {
        tok_i32x4 t;
        __builtin_memcpy(&t, p, 16);
        v[h] += t;
      } else {
        for (int e = 0; e < 3; ++e)
          if (n + e < a.N) v[h][e] += p[e];
      }
    }
  }
  put4<EPI>(a, m, n, v, a.x_scale[m], channels<EPI>(a, n), x);
}

// Rows of n bytes, ld apart, to rows of ldd (a multiple of 16), zero past n: 16
// bytes a thread.
__global__ __launch_bounds__(256) void pad_rows(const int8_t* src, int64_t rows, int64_t n, int64_t ld, int8_t* dst, int64_t ldd,
                                               int64_t first) {
  const int64_t per = ldd / 16, i = (first + blockIdx.x) * 256 + threadIdx.x;
  if (i >= rows * per) return;
  const int64_t r = i / per, c = i % per * 16;
  *reinterpret_cast<tok_i32x4*>(dst + r * ldd + c) = piece<false>(src + r * ld + c, n - c);
}

int64_t up(int64_t a, int64_t b) { return (a + b - 1) / b; }

// The tile of a call: the largest whose tiles fill the device, for it moves
// the fewest bytes through LDS for a product.
struct Tile {
  int bm, bn;
};
Tile tile_of(int64_t M, int64_t N) {
  const int64_t cus = device_compute_units();
  if (up(M, 256) * up(N, 256) >= cus) return {256, 256};
  if (up(M, 128) * up(N, 128) >= cus) return {128, 128};
  return {64, 64};
}

template <int BM, int BN, int WM, int WN, int BK, int NS, bool AL, int EPI>
hipError_t run_tiled(LinArgs a, hipStream_t s) {
  constexpr int threads = (BM / WM) * (BN / WN) * 64;
  auto k = linear_tiled<BM, BN, WM, WN, BK, NS, AL, EPI>;
  a.tiles_m = static_cast<int>(up(a.M, BM));
  a.tiles_n = static_cast<int>(up(a.N, BN / Channels<EPI>::H));
  const int64_t blocks = static_cast<int64_t>(a.tiles_m) * a.tiles_n * a.splits;
  if (blocks > 0x7fffffff) return hipErrorInvalidConfiguration;
  return in_launches(blocks, threads, [&](int64_t first, unsigned count) {
    a.first = first;
    hipLaunchKernelGGL(k, dim3(count), dim3(threads), 0, s, a);
  });
}

hipError_t run_skinny(void (*k)(LinArgs), LinArgs a, hipStream_t s) {
  return in_launches(up(a.N, 16), 256, [&](int64_t first, unsigned count) {
    a.first = first;
    hipLaunchKernelGGL(k, dim3(count), dim3(256), 0, s, a);
  });
}

// tokens of the skinny kernel (4096 x 4096: 32 tokens 13.4 us, 65 in tiles 12.2;
// 48 tokens took 18.7 in it)
constexpr int64_t kSkinny = 32;

}  // namespace

LinearPlan plan_linear_i8(int64_t M, int64_t N, int64_t K) {
  LinearPlan p;
  if (M <= kSkinny) return p;
  const Tile t = tile_of(M, N);
  const int64_t tiles = up(M, t.bm) * up(N, t.bn), stages = up(K, 64), cus = device_compute_units();
  // Split while the device has idle compute units and it pays: a stage of 64
  // bytes takes about 0.5 us where few workgroups run (it is latency), joining
  // 4 us and the traffic of the partial sums.
  int64_t s = 1;
  double best = 0;
  for (int64_t n = 1; n <= stages / 4 && (n == 1 || tiles * n <= 2 * cus); ++n) {
    const double us = 0.5 * up(stages, n) * up(tiles * n, cus) + (n > 1 ? 4 + 8e-6 / 4 * n * M * N : 0);
    if (n == 1 || us < best) {
      best = us;
      s = n;
    }
  }
  if (s > 1) {
    p.splits = static_cast<int>(s);
    p.part_bytes = s * M * N * 4;
  }
  return p;
}

namespace {

template <int EPI>
hipError_t run_linear(LinArgs a, hipStream_t s) {
  // 16-byte pieces, and a tile's rows within the 31-bit offsets of a buffer
  const bool al = a.K % 16 == 0 && a.ldx % 16 == 0 && a.ldx < (1 << 22) && reinterpret_cast<uintptr_t>(a.x) % 16 == 0 &&
                  reinterpret_cast<uintptr_t>(a.w) % 16 == 0;
  if (a.M <= kSkinny) {
    auto k = a.M <= 16   ? (al ? linear_skinny<Codes, 1, true, EPI> : linear_skinny<Codes, 1, false, EPI>)
                         : (al ? linear_skinny<Codes, 2, true, EPI> : linear_skinny<Codes, 2, false, EPI>);
    return run_skinny(k, a, s);
  }
  const Tile t = tile_of(a.M, a.N * Channels<EPI>::H);
  hipError_t e = t.bm == 256   ? (al ? run_tiled<256, 256, 128, 64, 128, 2, true, EPI>(a, s) : run_tiled<256, 256, 128, 64, 64, 4, false, EPI>(a, s))
                 : t.bm == 128 ? (al ? run_tiled<128, 128, 64, 64, 64, 4, true, EPI>(a, s) : run_tiled<128, 128, 64, 64, 64, 4, false, EPI>(a, s))
                               : (al ? run_tiled<64, 64, 32, 32, 64, 4, true, EPI>(a, s) : run_tiled<64, 64, 32, 32, 64, 4, false, EPI>(a, s));
  if (e == hipSuccess && a.part) {
    const int64_t blocks = up(a.M * up(a.N, 4), 256);  // few: a call of many tiles is not split
    hipLaunchKernelGGL(linear_join<EPI>, dim3(static_cast<unsigned>(blocks)), dim3(256), 0, s, a);
    e = hipGetLastError();
  }
  return e;
}

template <int EPI>
hipError_t run_float(const LinArgs& a, int x_dtype, hipStream_t s) {
  const bool al = a.K % 16 == 0 && reinterpret_cast<uintptr_t>(a.w) % 16 == 0;
  auto k = x_dtype == C3C_DTYPE_BF16  ? (al ? linear_skinny<ElemBf16, 1, true, EPI> : linear_skinny<ElemBf16, 1, false, EPI>)
           : x_dtype == C3C_DTYPE_F16 ? (al ? linear_skinny<ElemF16, 1, true, EPI> : linear_skinny<ElemF16, 1, false, EPI>)
                                      : (al ? linear_skinny<ElemF32, 1, true, EPI> : linear_skinny<ElemF32, 1, false, EPI>);
  return run_skinny(k, a, s);
}

}  // namespace

hipError_t launch_linear_i8(int64_t M, int64_t N, int64_t K, const int8_t* x, int64_t ldx,
                            const float* x_scale, const int8_t* w, const float* w_scale,
                            const float* bias, void* y, int y_dtype, const LinearEpilogue& e,
                            const LinearPlan& plan, int32_t* part, hipStream_t s) {
  if (M == 0) return hipSuccess;
  LinArgs a{x, w, x_scale, w_scale, bias, y, part, M, N, K, ldx, 0, 0, part ? plan.splits : 1, y_dtype, 0, e};
  return e.kind == EPILOGUE ? run_linear<EPILOGUE>(a, s) : e.kind == GATED ? run_linear<GATED>(a, s) : run_linear<PLAIN>(a, s);
}

// The copy costs its traffic and a launch, and up to halves the products: it pays
// from some hundred tokens on where these are large (channels of 4095, 4096 of
// them: 400 tokens 35 us, through registers 48; 8000 tokens 148, 292), and costs
// small ones a launch (777 of 333, 400 tokens: 12.4, 9.1).
bool linear_pads(int64_t M, int64_t K, int64_t ld) { return M > 64 && (K % 16 != 0 || ld % 16 != 0); }

hipError_t launch_pad_rows(const int8_t* src, int64_t rows, int64_t n, int64_t ld, int8_t* dst, int64_t ldd, hipStream_t s) {
  return in_launches(up(rows * (ldd / 16), 256), 256, [&](int64_t first, unsigned count) {
    hipLaunchKernelGGL(pad_rows, dim3(count), dim3(256), 0, s, src, rows, n, ld, dst, ldd, first);
  });
}

bool linear_quantises(int64_t M, int64_t K) { return M <= 4 && M * ((K + 15) / 16 * 16) <= kFusedBytes; }

hipError_t launch_linear_float(int64_t M, int64_t N, int64_t K, const void* x, int64_t ldx, int x_dtype,
                               const int8_t* w, const float* w_scale, const float* bias, void* y, int y_dtype,
                               const LinearEpilogue& e, hipStream_t s) {
  if (M == 0) return hipSuccess;
  LinArgs a{static_cast<const int8_t*>(x), w, nullptr, w_scale, bias, y, nullptr, M, N, K, ldx, 0, 0, 1, y_dtype, 0, e};
  return e.kind == EPILOGUE ? run_float<EPILOGUE>(a, x_dtype, s) : e.kind == GATED ? run_float<GATED>(a, x_dtype, s) : run_float<PLAIN>(a, x_dtype, s);
}

}  // namespace c3c
