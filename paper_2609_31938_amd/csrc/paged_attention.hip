// Attention over the paged 8-bit cache:
//   s_ij = scale q_i . k_j over the tokens j that query i sees,
//   o_i = sum_j 2^(c s_ij - m_i) v_j / sum_j 2^(c s_ij - m_i)
// (c = log2 e; the running maximum m and sum of a one-pass softmax), on
// v_mfma_f32_16x16x32_{bf16,f16} with fp32 sums.
//
// Both products are taken transposed, so that nothing moves between lanes:
//   S^T = K Q^T   A: 16 tokens x 32 channels of K, B: 32 channels x 16 queries
//   O^T = V^T P^T A: 16 channels x 32 tokens of V, B: 32 tokens x 16 queries
// A wave works on 64 tokens, four 16-token blocks of the cache.  Row m of the
// t-th S tile is token 16 (m / 4) + 4 t + m % 4 of the 64: with the C layout's
// four rows a lane (group g = lane / 16 holds rows 4 g ..), a lane ends up with
// the 16 scores of block g for one query, which are the B operand of the second
// product as they stand, and V's 16 codes of block g for one channel, 16 bytes
// side by side in the cache, are its A operand.  So a block's scales are one
// value a lane.
//
// K: e4m3 codes are exact in bf16 and f16; the scale joins c.
// Q: in its own type, f32 as the sum of three bf16 terms.
// P: 2^15 p as a sum of f16 terms (1 for bf16 calls, 2 for f16, 3 for f32):
//   11 bits each, where a bf16 term would have 8 and its rounding would be
//   seen in a bf16 output.
// V: codes in f16 times 2^k.  The accumulator is kept in units of 2^E, E the
//   largest exponent of a value scale so far; k = e - E while that is -15 or
//   more (codes then stay exact), and what is left of e - E goes to P.  Values
//   lose precision from 2^30 below the largest value scale seen on.
#include <math.h>

#include "token_dev.h"
#include "tokens_internal.h"

namespace c3c {
namespace {

constexpr float kInf = __builtin_inff();
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// 8 codes (two dwords) as bf16 (exact) or as f16 times a power of two, in a
// fragment's four dwords
__device__ inline tok_u32x4 codes_bf16(uint32_t lo, uint32_t hi) {
  return tok_u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, false)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, true)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, false)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, true))};
}
__device__ inline tok_u32x4 codes_f16(uint32_t lo, uint32_t hi, float scale) {
  return tok_u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, scale, false)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, scale, true)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, scale, false)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, scale, true))};
}

typedef _Float16 tok_f16x8 __attribute__((ext_vector_type(8)));
__device__ inline tok_f32x4 mfma_f16(tok_u32x4 a, tok_u32x4 b, tok_f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(tok_f16x8, a), __builtin_bit_cast(tok_f16x8, b), c, 0, 0, 0);
}
__device__ inline tok_f32x4 mfma_bf16(tok_u32x4 a, tok_u32x4 b, tok_f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(tok_bf16x8, a), __builtin_bit_cast(tok_bf16x8, b), c, 0, 0, 0);
}

// 8 fp32 values as N vectors of a 16-bit type V2 (two at a time) that sum to them
template <class V2, int N>
__device__ inline void to_terms(const float (&f)[8], tok_u32x4 (&t)[N]) {
  float rest[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) rest[e] = f[e];
#pragma unroll
  for (int n = 0; n < N; ++n)
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
      const V2 v = __builtin_convertvector((tok_f32x2{rest[e], rest[e + 1]}), V2);
      t[n][e >> 1] = __builtin_bit_cast(uint32_t, v);
      if (n + 1 < N) {
        rest[e] -= static_cast<float>(v[0]);
        rest[e + 1] -= static_cast<float>(v[1]);
      }
    }
}

// How a call's type enters: terms of a query and of a probability, and the
// first product.
template <class E>
struct Form;
template <>
struct Form<ElemBf16> {
  static constexpr int NQ = 1, NP = 1;
  typedef tok_bf16x2 Q2;
  __device__ static tok_u32x4 k(uint32_t lo, uint32_t hi) { return codes_bf16(lo, hi); }
  __device__ static tok_f32x4 mfma(tok_u32x4 a, tok_u32x4 b, tok_f32x4 c) { return mfma_bf16(a, b, c); }
};
template <>
struct Form<ElemF16> {
  static constexpr int NQ = 1, NP = 2;
  typedef tok_f16x2 Q2;
  __device__ static tok_u32x4 k(uint32_t lo, uint32_t hi) { return codes_f16(lo, hi, 1.f); }
  __device__ static tok_f32x4 mfma(tok_u32x4 a, tok_u32x4 b, tok_f32x4 c) { return mfma_f16(a, b, c); }
};
template <>
struct Form<ElemF32> : Form<ElemBf16> {
  static constexpr int NQ = 3, NP = 3;
};

// fp32 2^e for any int e the kernels form (0 below the normal range)
__device__ inline float pow2(int e) { return e < -126 ? 0.f : __uint_as_float(static_cast<uint32_t>((e < 127 ? e : 127) + 127) << 23); }
__device__ inline int exponent_of(float scale) { return static_cast<int>((__float_as_uint(scale) >> 23) & 255u) - 127; }

constexpr int kLift = 15;  // P is 2^15 p: at most 2^15, and p keeps its bits down to 2^-29
constexpr int kDeep = -15; // least k: codes down to 2^-9 stay multiples of 2^-24

// whether a dword holds the code of a NaN
__device__ inline bool nan_code(uint32_t w) { return (((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) != 0; }
// NaN codes replaced by 0
__device__ inline uint32_t no_nan(uint32_t w) {
  const uint32_t at = (((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) >> 7;
  return w & ~(at * 255u);
}

// What a column (a query) sees: tokens [begin, end) of its sequence.
struct Sight {
  int begin, end;
};
__device__ inline Sight sight(const AttendArgs& a, int len, int p) {
  Sight s{0, len};
  if (a.causal && p + 1 < s.end) s.end = p + 1;
  if (a.window > 0 && p - a.window + 1 > s.begin) s.begin = static_cast<int>(p - a.window + 1);
  return s;
}

// The sequence b as the kernels read it from the device: nothing of it is
// trusted.
struct Seq {
  int64_t row0;
  int n, len, start;  // new tokens, all tokens that the table can hold, place of the first new one
};
__device__ inline Seq sequence(const AttendArgs& a, int64_t b) {
  int64_t r0 = a.b.cu[b], r1 = a.b.cu[b + 1];
  r0 = r0 < 0 ? 0 : r0;
  r1 = r1 > a.b.T ? a.b.T : r1;
  const int64_t all = a.b.cols * a.c.page, cap = all < 0x7fffff00 ? all : 0x7fffff00;
  const int64_t len = a.b.len[b], n = r1 - r0;
  return {r0, static_cast<int>(n > 0 ? n : 0), static_cast<int>(len < cap ? len : cap), static_cast<int>(len - n)};
}

// One workgroup: 16 columns (queries and heads that read one key/value head)
// of one sequence and one split of its tokens; its 4 waves take every fourth
// 64-token tile of the split and join their results in LDS.  Columns are
// numbered token by token, the G heads of a token side by side.
template <class E, int DP>  // DP: channels padded to 64
__global__ __launch_bounds__(256) void attend_few(AttendArgs a, int splits, int split_tiles, int coltiles) {
  typedef Form<E> F;
  constexpr int KS = DP / 32, DT = DP / 16, NQ = F::NQ, NP = F::NP;
  typedef typename E::store S;
  __shared__ float sm[4][16], sl[4][16];
  __shared__ __align__(16) float so[4][16][DP + 4];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 15, g = lane >> 4;
  const int split = blockIdx.x % splits;
  const int64_t b = blockIdx.z;
  const int hk = blockIdx.y, heads = static_cast<int>(a.c.heads), D = static_cast<int>(a.c.dim);
  const int G = static_cast<int>(a.q_heads) / heads;
  const Seq q = sequence(a, b);
  const int64_t columns = static_cast<int64_t>(q.n) * G;
  const int nb = static_cast<int>(a.c.page) / 16;
  const int pow = (nb & (nb - 1)) == 0 ? __builtin_ctz(nb) : -1;
  const int32_t* table = a.b.table + b * a.b.cols;
  const float c = a.scale * kLog2e;

  for (int64_t col0 = static_cast<int64_t>(blockIdx.x / splits) * 16; col0 < columns; col0 += static_cast<int64_t>(coltiles) * 16) {
    const int64_t col = col0 + r < columns ? col0 + r : columns - 1;
    const int qi = static_cast<int>(col / G), qh = hk * G + static_cast<int>(col % G);
    const Sight mine = sight(a, q.len, q.start + qi);
    // what all columns see together, and what each of them sees
    const int i0 = static_cast<int>(col0 / G);
    const int64_t lastcol = col0 + 15 < columns ? col0 + 15 : columns - 1;
    const int i1 = static_cast<int>(lastcol / G);
    const Sight lowest = sight(a, q.len, q.start + i0), highest = sight(a, q.len, q.start + i1);
    const int ub = lowest.begin, ue = highest.end, cb = highest.begin, ce = lowest.end;
    const int t0 = ub / 64 + split * split_tiles;
    int t1 = (ue + 63) / 64;
    // the last split takes what is left
    if (split + 1 < splits && t0 + split_tiles < t1) t1 = t0 + split_tiles;

    tok_u32x4 qf[KS][NQ];
    {
      const S* qp = static_cast<const S*>(a.q) + (q.row0 + qi) * a.ld_q + static_cast<int64_t>(qh) * D;
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        float f[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int d = (k >> 1) * 64 + g * 16 + (k & 1) * 8 + e;
          f[e] = d < D ? E::widen(qp[d]) : 0.f;
        }
        to_terms<typename F::Q2, NQ>(f, qf[k]);
      }
    }
    tok_f32x4 acc[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d) acc[d] = tok_f32x4{0.f, 0.f, 0.f, 0.f};
    float m = -kInf, l = 0.f;  // l: this lane's part of 2^15 times the sum
    int unit = -126;           // E

    for (int tile = t0 + wave; tile < t1; tile += 4) {
      const int blk0 = tile * 4, tok0 = tile * 64;
      auto find = [&](int blk) __attribute__((always_inline)) {  // block index among the cache's, or -1
        const int colp = pow >= 0 ? blk >> pow : blk / nb;
        if (blk * 16 >= ue || colp >= a.b.cols) return static_cast<int64_t>(-1);
        const int64_t page = table[colp];
        if (page < 0 || page >= a.c.pages) return static_cast<int64_t>(-1);
        return (page * heads + hk) * nb + (blk - colp * nb);
      };
      const int64_t kb = find(blk0 + (r >> 2)), vb = find(blk0 + g);
      const uint8_t* kp = static_cast<const uint8_t*>(a.c.k) + (kb * 16 + (r & 3)) * D + g * 16;
      const uint8_t* vp = static_cast<const uint8_t*>(a.c.v) + (vb * D + r) * 16;
      // scales of block g; c times the key's, 0 kept off so that -inf stays -inf
      const float cg = vb >= 0 ? fmaxf(c * a.c.k_scale[vb], 0x1p-126f) : 1.f;
      const int ve = vb >= 0 ? exponent_of(a.c.v_scale[vb]) : -126;
      tok_u32x4 kv[4][DP / 64], vv[DT];
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int j = 0; j < DP / 64; ++j) {
          kv[t][j] = tok_u32x4{0, 0, 0, 0};
          if (kb >= 0 && j * 64 + g * 16 < D) kv[t][j] = *reinterpret_cast<const tok_u32x4*>(kp + 4 * t * D + j * 64);
        }
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        vv[d] = tok_u32x4{0, 0, 0, 0};
        if (vb >= 0 && d * 16 < D) vv[d] = *reinterpret_cast<const tok_u32x4*>(vp + d * 256);
      }
      tok_f32x4 s[4];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        s[t] = tok_f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < KS; ++k) {
          const tok_u32x4 kf = F::k(kv[t][k >> 1][(k & 1) * 2], kv[t][k >> 1][(k & 1) * 2 + 1]);
#pragma unroll
          for (int n = 0; n < NQ; ++n) s[t] = F::mfma(kf, qf[k][n], s[t]);
        }
      }
      // a tile that some column sees in part only, or with a page missing
      const bool edge = tok0 < cb || tok0 + 64 > ce || __ballot(vb < 0) != 0;
      bool bad = false;
      if (edge) {
        const int base = tok0 + 16 * g;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int tok = base + 4 * t + i;
            if (tok < mine.begin || tok >= mine.end || vb < 0) s[t][i] = -kInf;
          }
        // values that no column sees become 0; NaN among the others are
        // taken out of the product and put back where they are seen
        uint32_t keep[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          keep[t] = 0;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int tok = base + 4 * t + i;
            if (tok >= ub && tok < ue) keep[t] |= 255u << (8 * i);
          }
        }
        bool any = false;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
          for (int t = 0; t < 4; ++t) {
            vv[d][t] &= keep[t];
            any |= nan_code(vv[d][t]);
          }
        bad = __ballot(any) != 0;
        if (bad) {
#pragma unroll
          for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int t = 0; t < 4; ++t) vv[d][t] = no_nan(vv[d][t]);
        }
      }
      float top = -kInf;
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) top = fmaxf(top, s[t][i]);
      top *= cg;
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      int ve4 = ve;
      ve4 = max(ve4, __shfl_xor(ve4, 16));
      ve4 = max(ve4, __shfl_xor(ve4, 32));
      const float next = fmaxf(m, top);
      const float ref = next == -kInf ? 0.f : next;
      if (__ballot(next > m || ve4 > unit)) {
        const float down = __builtin_amdgcn_exp2f(m - ref);
        const int grown = max(ve4, unit);
        l *= down;
        const float all = down * pow2(unit - grown);
#pragma unroll
        for (int d = 0; d < DT; ++d) acc[d] *= all;
        m = next;
        unit = grown;
      }
      const int k = max(ve - unit, kDeep), f = ve - unit - k;
      const float vk = pow2(k), lift = kLift - ref;
      const bool low = __ballot(f < 0) != 0;
      tok_u32x4 pf[2][NP];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        float p[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          p[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[2 * u + (e >> 2)][e & 3], cg, lift));
          l += p[e];
        }
        if (low) {
#pragma unroll
          for (int e = 0; e < 8; ++e) p[e] *= pow2(f);
        }
        to_terms<tok_f16x2, NP>(p, pf[u]);
      }
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const tok_u32x4 vf = codes_f16(vv[d][2 * u], vv[d][2 * u + 1], vk);
#pragma unroll
          for (int n = 0; n < NP; ++n) acc[d] = mfma_f16(vf, pf[u][n], acc[d]);
        }
      if (bad) {
        for (int o = 0; o < 4; ++o) {
          const int64_t ob = __shfl(vb, 16 * o);
          if (ob < 0) continue;
          for (int t = 0; t < 16; ++t) {
            const int tok = tok0 + 16 * o + t;
            if (tok < mine.begin || tok >= mine.end) continue;
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const int ch = d * 16 + g * 4 + i;
                if (ch < D && (static_cast<const uint8_t*>(a.c.v)[(ob * D + ch) * 16 + t] & 127) == 127)
                  acc[d][i] = __builtin_nanf("");
              }
          }
        }
      }
    }
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    l *= pow2(-kLift);
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[d][i] = ldexpf(acc[d][i], unit - kLift);

    // join the waves: the weights of their results, then 4 rows of sums
    if (g == 0) {
      sm[wave][r] = m;
      sl[wave][r] = l;
    }
#pragma unroll
    for (int d = 0; d < DT; ++d) *reinterpret_cast<tok_f32x4*>(&so[wave][r][d * 16 + g * 4]) = acc[d];
    __syncthreads();
    // 16 threads a column
    const int oc = threadIdx.x >> 4, ol = threadIdx.x & 15;
    float all = fmaxf(fmaxf(sm[0][oc], sm[1][oc]), fmaxf(sm[2][oc], sm[3][oc])), w[4], sum = 0.f;
    const float ref = all == -kInf ? 0.f : all;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      w[i] = __builtin_amdgcn_exp2f(sm[i][oc] - ref);
      sum += w[i] * sl[i][oc];
    }
    if (col0 + oc < columns) {
      const int64_t oi = (col0 + oc) / G, oh = hk * G + (col0 + oc) % G;
      const int64_t row = (q.row0 + oi) * a.q_heads + oh;
      float* part = splits > 1 ? a.part + (static_cast<int64_t>(split) * a.b.T * a.q_heads + row) * (D + 2) : nullptr;
      const float inv = sum == 0.f ? 0.f : 1.f / sum;
      for (int d = ol; d < D; d += 16) {
        float o = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) o += w[i] * so[i][oc][d];
        if (part)
          part[2 + d] = o;
        else
          static_cast<S*>(a.out)[row * D + d] = E::narrow(o * inv);
      }
      if (ol == 0) {
        if (part) {
          part[0] = all;
          part[1] = sum;
        } else if (a.lse) {
          a.lse[row] = sum == 0.f ? -kInf : all * kLn2 + logf(sum);
        }
      }
    }
    __syncthreads();
  }
}

// out and lse from the partial results of a split call: one wave a row.
template <class E>
__global__ __launch_bounds__(256) void attend_join(AttendArgs a, int splits) {
  const int64_t row = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6), rows = a.b.T * a.q_heads;
  if (row >= rows) return;
  const int lane = threadIdx.x & 63, D = static_cast<int>(a.c.dim);
  const float* part = a.part + row * (D + 2);
  const int64_t step = rows * (D + 2);
  float m = -kInf;
  for (int s = 0; s < splits; ++s) m = fmaxf(m, part[s * step]);
  const float ref = m == -kInf ? 0.f : m;
  float l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
  for (int s = 0; s < splits; ++s) {
    const float part_l = part[s * step + 1];
    if (part_l == 0.f) continue;  // nothing seen
    const float w = __builtin_amdgcn_exp2f(part[s * step] - ref);
    l += w * part_l;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (lane + 64 * i < D) o[i] += w * part[s * step + 2 + lane + 64 * i];
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (lane + 64 * i < D) static_cast<typename E::store*>(a.out)[row * D + lane + 64 * i] = E::narrow(o[i] * inv);
  if (a.lse && lane == 0) a.lse[row] = l == 0.f ? -kInf : m * kLn2 + logf(l);
}

int64_t up(int64_t a, int64_t b) { return (a + b - 1) / b; }

// 64-token tiles that one column tile sees at most
int64_t tiles_seen(const c3c_kv_batch& b, int64_t page, int64_t window) {
  int64_t tokens = b.max_len < b.cols * page ? b.max_len : b.cols * page;
  if (window > 0 && window + b.max_new < tokens) tokens = window + b.max_new + 64;
  return up(tokens, 64);
}

template <class E>
hipError_t run(const AttendArgs& a, const AttendPlan& p, hipStream_t s) {
  const int64_t G = a.q_heads / a.c.heads, coltiles = up(a.b.max_new * G, 16);
  const int64_t tiles = tiles_seen(a.b, a.c.page, a.window);
  const int64_t blocks = coltiles * p.splits;
  if (a.b.B > 65535 || a.c.heads > 65535 || blocks > 0x7fffffff) return hipErrorInvalidConfiguration;
  auto k = a.c.dim <= 64    ? attend_few<E, 64>
           : a.c.dim <= 128 ? attend_few<E, 128>
           : a.c.dim <= 192 ? attend_few<E, 192>
                            : attend_few<E, 256>;
  hipLaunchKernelGGL(k, dim3(static_cast<unsigned>(blocks), static_cast<unsigned>(a.c.heads), static_cast<unsigned>(a.b.B)),
                     dim3(256), 0, s, a, p.splits, static_cast<int>(up(tiles, p.splits)), static_cast<int>(coltiles));
  hipError_t e = hipGetLastError();
  if (e == hipSuccess && p.splits > 1) {
    const int64_t jb = up(a.b.T * a.q_heads, 4);
    if (jb > 0x7fffffff) return hipErrorInvalidConfiguration;
    hipLaunchKernelGGL(attend_join<E>, dim3(static_cast<unsigned>(jb)), dim3(256), 0, s, a, p.splits);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace

AttendPlan plan_attend(const c3c_kv_cache& c, const c3c_kv_batch& b, int dtype, int64_t q_heads,
                       int causal, int64_t window) {
  AttendPlan p;
  const int64_t base = up(b.max_new * (q_heads / c.heads), 16) * c.heads * b.B;
  const int64_t tiles = tiles_seen(b, c.page, window);
  if (base == 0) return p;
  // enough workgroups to fill the device several times (sequences are
  // ragged), of at least one tile a wave
  const int64_t want = up(8 * device_compute_units(), base), most = up(tiles, 4);
  const int64_t s = want < most ? want : most;
  if (s > 1) {
    p.splits = static_cast<int>(s);
    p.part_bytes = s * b.T * q_heads * (c.dim + 2) * 4;
  }
  return p;
}

hipError_t launch_attend(const AttendArgs& a, int dtype, const AttendPlan& plan, hipStream_t s) {
  if (a.b.B == 0 || a.b.T == 0 || a.b.max_new == 0) return hipSuccess;
  return dtype == C3C_DTYPE_BF16  ? run<ElemBf16>(a, plan, s)
         : dtype == C3C_DTYPE_F16 ? run<ElemF16>(a, plan, s)
                                  : run<ElemF32>(a, plan, s);
}

}  // namespace c3c
