// Matrix product in 8-bit integers:
//   y[m][n] = (sum_k x[m][k] w[n][k]) * x_scale[m] * w_scale[n] + bias[n]
// with x int8 [M][ldx], w int8 [N][K] (both K-contiguous) and an exact int32
// sum on v_mfma_i32_16x16x64_i8: the weights are the A operand (rows n), the
// tokens B (columns m), so that a lane's four results are four consecutive n
// of one token and are stored together.
//
// skinny: at most 64 tokens.  The weights are read once, straight into
//   registers (no tile of them is used twice), by 4 waves that share 16 rows
//   and take every fourth 128-byte piece of K; their sums meet in LDS.
// tiled: BM x BN tiles, 128 bytes of K a stage, two stages in LDS.  With
//   16-byte rows the stages are loaded straight into LDS (the buffer's bounds
//   make rows past M or N and pieces past K zero); rows of any other length go
//   through registers.  A 16-byte piece c of row r lies at place c ^ (r & 7):
//   the 16 rows that a fragment read touches then spread over all banks.
#include "token_dev.h"
#include "tokens_internal.h"

namespace c3c {
namespace {

typedef __attribute__((address_space(3))) void lds_void;

struct LinArgs {
  const int8_t *x, *w;
  const float *x_scale, *w_scale, *bias;
  void* y;
  int32_t* part;  // [splits][M][N], or NULL: y is written
  int64_t M, N, K, ldx;
  int tiles_m, tiles_n;
  int splits;     // along K, in stages
  int y_dtype;
};

__device__ inline void put4(const LinArgs& a, int64_t m, int64_t n, tok_i32x4 v) {
  const float s = a.x_scale[m];
  float f[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t nn = n + i < a.N ? n + i : a.N - 1;
    f[i] = static_cast<float>(v[i]) * s * a.w_scale[nn];
    if (a.bias) f[i] += a.bias[nn];
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
  } else {
#pragma unroll
    for (int e = 0; e < 15; ++e)
      if (e < m) v[e >> 2] |= (static_cast<int32_t>(p[e]) & 255) << (8 * (e & 3));
  }
  return v;
}

// MT tiles of 16 tokens.
template <int MT, bool AL>
__global__ __launch_bounds__(256) void linear_skinny(LinArgs a) {
  __shared__ tok_i32x4 sums[3][MT][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int r = lane & 15, g = lane >> 4;
  const int64_t n0 = static_cast<int64_t>(blockIdx.x) * 16;
  const int64_t nr = n0 + r < a.N ? n0 + r : a.N - 1;
  const int8_t* wp = a.w + nr * a.K;
  const int8_t* xp[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    const int64_t m = t * 16 + r;
    xp[t] = a.x + (m < a.M ? m : a.M - 1) * a.ldx;
  }
  tok_i32x4 acc[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) acc[t] = tok_i32x4{0, 0, 0, 0};
  constexpr int U = 4;  // stages in flight
  for (int64_t k0 = wave * 128; k0 < a.K; k0 += 512 * U) {
    tok_i32x4 wv[U][2];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int64_t k = k0 + 512 * u + 64 * j + 16 * g;
        wv[u][j] = piece<AL>(wp + k, a.K - k);
      }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int64_t k = k0 + 512 * u + 64 * j + 16 * g;
#pragma unroll
        for (int t = 0; t < MT; ++t)
          acc[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wv[u][j], piece<AL>(xp[t] + k, a.K - k), acc[t], 0, 0, 0);
      }
  }
  if (wave > 0) {
#pragma unroll
    for (int t = 0; t < MT; ++t) sums[wave - 1][t][lane] = acc[t];
  }
  __syncthreads();
  if (wave > 0) return;
#pragma unroll
  for (int t = 0; t < MT; ++t) {
#pragma unroll
    for (int w = 0; w < 3; ++w) acc[t] += sums[w][t][lane];
    const int64_t m = t * 16 + r, n = n0 + g * 4;
    if (m < a.M && n < a.N) put4(a, m, n, acc[t]);
  }
}

constexpr int BK = 128;  // bytes of K a stage

// NW waves, each with a WM x WN part of the tile.
template <int BM, int BN, int WM, int WN, bool AL>
__global__ __launch_bounds__((BM / WM) * (BN / WN) * 64) void linear_tiled(LinArgs a) {
  constexpr int NW = (BM / WM) * (BN / WN);
  constexpr int MT = WM / 16, NT = WN / 16;
  constexpr int ROWS = BM + BN;              // rows of w, then rows of x
  constexpr int LOADS = ROWS / 8 / NW;       // 1024-byte loads a wave and stage
  static_assert(ROWS % (8 * NW) == 0 && BN % 8 == 0, "whole loads");
  __shared__ __align__(16) int8_t lds[2 * ROWS * BK];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r = lane & 15, g = lane >> 4;

  // tiles in an order that keeps each of the 8 L2 caches on neighbouring
  // ones: workgroup b runs on cache b % 8, which gets a run of consecutive
  // tiles, walked in columns of 8 tiles of tokens
  const int total = a.tiles_m * a.tiles_n;
  int b = blockIdx.x;
  const int split = b / total;
  b -= split * total;
  {
    const int each = total / 8, rest = total % 8, c = b % 8, i = b / 8;
    b = c * each + (c < rest ? c : rest) + i;
  }
  constexpr int COL = 8;
  const int colg = b / (COL * a.tiles_n), in = b - colg * COL * a.tiles_n;
  const int high = a.tiles_m - colg * COL < COL ? a.tiles_m - colg * COL : COL;
  const int tm = colg * COL + in % high, tn = in / high;
  const int64_t m0 = static_cast<int64_t>(tm) * BM, n0 = static_cast<int64_t>(tn) * BN;

  const int stages = static_cast<int>((a.K + BK - 1) / BK);
  const int s0 = static_cast<int>(static_cast<int64_t>(stages) * split / a.splits);
  const int s1 = static_cast<int>(static_cast<int64_t>(stages) * (split + 1) / a.splits);

  const int64_t nrows = a.N - n0 < BN ? a.N - n0 : BN, mrows = a.M - m0 < BM ? a.M - m0 : BM;
  const int8_t* wb = a.w + n0 * a.K;
  const int8_t* xb = a.x + m0 * a.ldx;
  // the part of a 1024-byte load (8 rows) that this lane brings: row lane / 8,
  // place lane % 8, hence piece (lane % 8) ^ (lane / 8)
  const int lrow = lane >> 3, lpiece = (lane & 7) ^ lrow;
  tok_i32x4 staged[LOADS];  // !AL
  const __amdgpu_buffer_rsrc_t wrs = __builtin_amdgcn_make_buffer_rsrc(
      const_cast<int8_t*>(wb), 0, static_cast<int>(nrows * a.K), 0x00020000);
  const __amdgpu_buffer_rsrc_t xrs = __builtin_amdgcn_make_buffer_rsrc(
      const_cast<int8_t*>(xb), 0, static_cast<int>((mrows - 1) * a.ldx + a.K), 0x00020000);
  auto load = [&](int st, int buf) __attribute__((always_inline)) {
    const int k = st * BK + lpiece * 16;
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int row = (i * NW + wave) * 8;  // of ROWS, uniform; whole loads are of w or of x
      const bool isw = row < BN;
      const int rr = (isw ? row : row - BN) + lrow;
      if (AL) {
        const int ld = static_cast<int>(isw ? a.K : a.ldx);
        const int off = k < a.K ? rr * ld + k : 0x7fffffff;
        lds_void* to = (lds_void*)(lds + buf * ROWS * BK + row * BK);
        if (isw)
          __builtin_amdgcn_raw_ptr_buffer_load_lds(wrs, to, 16, off, 0, 0, 0);
        else
          __builtin_amdgcn_raw_ptr_buffer_load_lds(xrs, to, 16, off, 0, 0, 0);
      } else {
        const int64_t ld = isw ? a.K : a.ldx;
        const bool ok = rr < (isw ? nrows : mrows);
        staged[i] = piece<false>((isw ? wb : xb) + (ok ? rr * ld + k : 0), ok ? a.K - k : 0);
      }
    }
  };
  auto settle = [&](int buf) __attribute__((always_inline)) {
    if (!AL) {
#pragma unroll
      for (int i = 0; i < LOADS; ++i)
        *reinterpret_cast<tok_i32x4*>(lds + buf * ROWS * BK + (i * NW + wave) * 8 * BK + lane * 16) = staged[i];
    }
  };

  const int wm = wave % (BM / WM) * WM, wn = wave / (BM / WM) * WN;
  tok_i32x4 acc[NT][MT];
#pragma unroll
  for (int i = 0; i < NT; ++i)
#pragma unroll
    for (int j = 0; j < MT; ++j) acc[i][j] = tok_i32x4{0, 0, 0, 0};

  if (s0 < s1) {
    load(s0, 0);
    settle(0);
  }
  __syncthreads();
  for (int st = s0; st < s1; ++st) {
    const int cur = (st - s0) & 1;
    if (st + 1 < s1) load(st + 1, cur ^ 1);
    const int8_t* base = lds + cur * ROWS * BK;
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      // every fragment row is congruent to r modulo 8
      const int place = ((ks * 4 + g) ^ (r & 7)) * 16;
      tok_i32x4 av[NT], bv[MT];
#pragma unroll
      for (int i = 0; i < NT; ++i)
        av[i] = *reinterpret_cast<const tok_i32x4*>(base + (wn + i * 16 + r) * BK + place);
#pragma unroll
      for (int j = 0; j < MT; ++j)
        bv[j] = *reinterpret_cast<const tok_i32x4*>(base + (BN + wm + j * 16 + r) * BK + place);
#pragma unroll
      for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int j = 0; j < MT; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(av[i], bv[j], acc[i][j], 0, 0, 0);
    }
    if (st + 1 < s1) settle(cur ^ 1);
    __syncthreads();
  }

#pragma unroll
  for (int j = 0; j < MT; ++j) {
    const int64_t m = m0 + wm + j * 16 + r;
    if (m >= a.M) continue;
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      const int64_t n = n0 + wn + i * 16 + g * 4;
      if (n >= a.N) continue;
      if (a.part) {
        int32_t* p = a.part + (split * a.M + m) * a.N + n;
        if (n + 4 <= a.N) {
          __builtin_memcpy(p, &acc[i][j], 16);
        } else {
          for (int e = 0; e < 3; ++e)
            if (n + e < a.N) p[e] = acc[i][j][e];
        }
      } else {
        put4(a, m, n, acc[i][j]);
      }
    }
  }
}

// y from the partial sums of a split call: four results a thread.
__global__ __launch_bounds__(256) void linear_join(LinArgs a) {
  const int64_t quads = (a.N + 3) / 4;
  const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (i >= a.M * quads) return;
  const int64_t m = i / quads, n = i % quads * 4;
  tok_i32x4 v = {0, 0, 0, 0};
  for (int s = 0; s < a.splits; ++s) {
    const int32_t* p = a.part + (s * a.M + m) * a.N + n;
    if (n + 4 <= a.N) {
      tok_i32x4 t;
      __builtin_memcpy(&t, p, 16);
      v += t;
    } else {
      for (int e = 0; e < 3; ++e)
        if (n + e < a.N) v[e] += p[e];
    }
  }
  put4(a, m, n, v);
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

template <int BM, int BN, int WM, int WN, bool AL>
hipError_t run_tiled(LinArgs a, hipStream_t s) {
  constexpr int threads = (BM / WM) * (BN / WN) * 64;
  auto k = linear_tiled<BM, BN, WM, WN, AL>;
  a.tiles_m = static_cast<int>(up(a.M, BM));
  a.tiles_n = static_cast<int>(up(a.N, BN));
  const int64_t blocks = static_cast<int64_t>(a.tiles_m) * a.tiles_n * a.splits;
  if (blocks > 0x7fffffff) return hipErrorInvalidConfiguration;
  hipLaunchKernelGGL(k, dim3(static_cast<unsigned>(blocks)), dim3(threads), 0, s, a);
  return hipGetLastError();
}

constexpr int64_t kSkinny = 64;  // tokens

}  // namespace

LinearPlan plan_linear_i8(int64_t M, int64_t N, int64_t K) {
  LinearPlan p;
  if (M <= kSkinny) return p;
  const Tile t = tile_of(M, N);
  const int64_t tiles = up(M, t.bm) * up(N, t.bn), stages = up(K, BK), cus = device_compute_units();
  // at least 8 stages a split: fewer cost more in partial sums than they save
  const int64_t s = cus / tiles < stages / 8 ? cus / tiles : stages / 8;
  if (s > 1) {
    p.splits = static_cast<int>(s);
    p.part_bytes = s * M * N * 4;
  }
  return p;
}

hipError_t launch_linear_i8(int64_t M, int64_t N, int64_t K, const int8_t* x, int64_t ldx,
                            const float* x_scale, const int8_t* w, const float* w_scale,
                            const float* bias, void* y, int y_dtype, const LinearPlan& plan,
                            int32_t* part, hipStream_t s) {
  if (M == 0) return hipSuccess;
  LinArgs a{x, w, x_scale, w_scale, bias, y, part, M, N, K, ldx, 0, 0, part ? plan.splits : 1, y_dtype};
  // 16-byte pieces, and a tile's rows within the 31-bit offsets of a buffer
  const bool al = K % 16 == 0 && ldx % 16 == 0 && ldx < (1 << 22) && reinterpret_cast<uintptr_t>(x) % 16 == 0 &&
                  reinterpret_cast<uintptr_t>(w) % 16 == 0;
  if (M <= kSkinny) {
    const int64_t blocks = up(N, 16);
    auto k = M <= 16   ? (al ? linear_skinny<1, true> : linear_skinny<1, false>)
             : M <= 32 ? (al ? linear_skinny<2, true> : linear_skinny<2, false>)
                       : (al ? linear_skinny<4, true> : linear_skinny<4, false>);
    hipLaunchKernelGGL(k, dim3(static_cast<unsigned>(blocks)), dim3(256), 0, s, a);
    return hipGetLastError();
  }
  const Tile t = tile_of(M, N);
  hipError_t e = t.bm == 256   ? (al ? run_tiled<256, 256, 128, 64, true>(a, s) : run_tiled<256, 256, 128, 64, false>(a, s))
                 : t.bm == 128 ? (al ? run_tiled<128, 128, 64, 64, true>(a, s) : run_tiled<128, 128, 64, 64, false>(a, s))
                               : (al ? run_tiled<64, 64, 32, 32, true>(a, s) : run_tiled<64, 64, 32, 32, false>(a, s));
  if (e == hipSuccess && part) {
    const int64_t blocks = up(M * up(N, 4), 256);
    if (blocks > 0x7fffffff) return hipErrorInvalidConfiguration;
    hipLaunchKernelGGL(linear_join, dim3(static_cast<unsigned>(blocks)), dim3(256), 0, s, a);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace c3c
