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
// P: 2^7 p as a sum of f16 terms (1 for bf16 calls, 2 for f16, 3 for f32):
//   11 bits each, where a bf16 term would have 8 and its rounding would be
//   seen in a bf16 output.
// V: codes in f16 times 2^k.  The accumulator is kept in units of 2^E, E the
//   largest exponent of a value scale so far; k = e - E while that is -15 or
//   more (codes then stay exact), and what is left of e - E goes to P.  P's terms
//   are spaced by 2^-24 at least: p is held to 2^-25 / 2^7 = 2^-32 beside its
//   relative 11 bits a term, and to 2^(d - 47) where e is d > 15 below E.
// attend_few: few queries (single tokens): the cache is read once, from HBM
// straight into registers, and its traffic is the bound: 64 sequences of 1000
// to 32768 tokens, 32 query and 8 key/value heads of 128, 483 us, 4.6 TB/s.
// attend_many: chunks of queries share tiles in LDS; exponentials, conversions
// and products of two waves a SIMD are the bound: 8192 causal queries of the
// same heads 599 us, 918 TFLOP/s.
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

// P is 2^7 p.  The maximum that p is taken against may stay up to 2^8 behind
// the true one, so P is at most 2^15, and p keeps its bits down to 2^-21.
constexpr int kLift = 7;
constexpr float kSlack = 8.f;
constexpr int kDeep = -15; // least k: codes down to 2^-9 stay multiples of 2^-24

// whether a dword holds the code of a NaN
__device__ inline bool nan_code(uint32_t w) { return (((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) != 0; }
// NaN codes replaced by 0
__device__ inline uint32_t no_nan(uint32_t w) {
  const uint32_t at = (((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) >> 7;
  return w & ~(at * 255u);
}

// The kernels' arguments: scalar registers are short beside two products and
// a softmax, so sizes are 32 bits and what the host can work out is.
struct Dev {
  const uint8_t *k, *v;
  const float *ks, *vs;
  const int32_t *table, *cu, *len;
  const void* q;
  void* out;
  float *lse, *part;
  int64_t ld_q;
  int T, q_heads, heads, G, D;
  int pages, nb, pow, cols, cap;  // blocks of a page, their log2 or -1; tokens of a table row
  int causal, window;
  float c;                        // scale * log2 e
  int splits, split_tiles, coltiles;
  uint32_t total;  // workgroups of attend_many
  int64_t first;   // workgroup of this launch (attend_many, attend_join)
};

// What a column (a query) sees: tokens [begin, end) of its sequence.
struct Sight {
  int begin, end;
};
__device__ inline Sight sight(const Dev& a, int len, int p) {
  Sight s{0, len};
  if (a.causal && p + 1 < s.end) s.end = p + 1;
  if (a.window > 0 && p >= a.window) s.begin = p - a.window + 1;
  return s;
}

// The sequence b as the kernels read it from the device: nothing of it is
// trusted.
struct Seq {
  int row0, n, len, start;  // new tokens, all tokens that the table can hold, place of the first new one
};
__device__ inline Seq sequence(const Dev& a, int b) {
  int r0 = a.cu[b], r1 = a.cu[b + 1];
  r0 = r0 < 0 ? 0 : r0;
  r1 = r1 > a.T ? a.T : r1;
  const int len = a.len[b], n = r1 > r0 ? r1 - r0 : 0;
  // a negative length is one of nothing: its queries see nothing either way
  return {r0, n, len < a.cap ? len : a.cap, (len < 0 ? 0 : len) - n};
}

// Blocks of a sequence are found in two steps, so that nothing waits for the
// page table: peek reads the page of block blk (none where no token of it lies
// in [begin, end)), settle makes it the block's index among the cache's (of
// head hk), or kNone.  A block that no query sees may hold anything, its scales
// included: it is not read.
constexpr uint32_t kNone = 0xffffffffu;
__device__ inline int column_of(const Dev& a, int blk) { return a.pow >= 0 ? blk >> a.pow : blk / a.nb; }
__device__ inline uint32_t peek(const Dev& a, const int32_t* row, int blk, int begin, int end) {
  const int col = column_of(a, blk);
  return blk * 16 + 15 >= begin && blk * 16 < end && col < a.cols ? static_cast<uint32_t>(row[col]) : kNone;
}
__device__ inline uint32_t settle(const Dev& a, int hk, int blk, uint32_t page) {
  return page < static_cast<uint32_t>(a.pages) ? (page * a.heads + hk) * a.nb + (blk - column_of(a, blk) * a.nb) : kNone;
}

// v, as a value that the compiler cannot compute with ahead of time: keeps
// what rare or early code derives from it out of the main loop's registers
__device__ inline int apart(int v) {
  asm volatile("" : "+s"(v));
  return v;
}

// v, known here: sums that are due beside products are not put off until the
// round's end, where their chain has nothing beside it
__device__ inline void settled(float& v) { asm volatile("" : "+v"(v)); }

// The query of column (qi, qh), as terms, in the order of K's fragments:
// element e of step k is channel 64 (k / 2) + 16 g + 8 (k % 2) + e.
template <class E, int KS>
__device__ inline void load_query(const Dev& a, int64_t row, int qh, int g, tok_u32x4 (&qf)[KS][Form<E>::NQ]) {
  typedef typename E::store S;
  const int D = apart(a.D);
  const S* qp = static_cast<const S*>(a.q) + row * a.ld_q + static_cast<int64_t>(qh) * D + g * 16;
#pragma unroll
  for (int k = 0; k < KS; ++k) {
    S v[8] = {};
    if ((k >> 1) * 64 + g * 16 < D) __builtin_memcpy(v, qp + (k >> 1) * 64 + (k & 1) * 8, sizeof v);
    float f[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = E::widen(v[e]);
    to_terms<typename Form<E>::Q2, Form<E>::NQ>(f, qf[k]);
  }
}

// An edge tile's scores: what a column does not see becomes -inf.  base: the
// first token of this lane's block.
__device__ inline void hide(tok_f32x4 (&s)[4], int base, const Sight& mine, bool page) {
#pragma unroll
  for (int t = 0; t < 4; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int tok = base + 4 * t + i;
      if (tok < mine.begin || tok >= mine.end || !page) s[t][i] = -kInf;
    }
}
// mask of dword t of a value fragment: the bytes of tokens in [ub, ue)
__device__ inline uint32_t kept(int base, int t, int ub, int ue) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (base + 4 * t + i >= ub && base + 4 * t + i < ue) m |= 255u << (8 * i);
  return m;
}
// NaN that were taken out of an edge tile's values come back to the channels
// of the columns that see them.  vb: this lane's block.
template <int DT>
__device__ inline void put_nan(const Dev& a, uint32_t vb, int tok0, int g, const Sight& mine, tok_f32x4 (&acc)[DT]) {
  const int D = apart(a.D);
  for (int o = 0; o < 4; ++o) {
    const uint32_t ob = __shfl(vb, 16 * o);
    if (ob == kNone) continue;
    for (int t = 0; t < 16; ++t) {
      const int tok = tok0 + 16 * o + t;
      if (tok < mine.begin || tok >= mine.end) continue;
      const uint8_t* v = a.v + (static_cast<int64_t>(ob) * D + g * 4) * 16 + t;
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        if (d * 16 >= D) break;
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if ((v[(d * 16 + i) * 16] & 127) == 127) acc[d][i] = __builtin_nanf("");
      }
    }
  }
}

// A maximum over the four lane groups
__device__ inline float over_groups(float v) {
  auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
  p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
}
__device__ inline int over_groups(int v) {
  auto p = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  v = max(static_cast<int>(p[0]), static_cast<int>(p[1]));
  p = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return max(static_cast<int>(p[0]), static_cast<int>(p[1]));
}

// The running softmax of one column tile over one 64-token tile, in two
// steps.  First the maximum m and the accumulators in its units (cg: c times
// the key scale of this lane's block; shrink: 2^(E before - E now)).  The
// maximum moves only when a score passes it by more than kSlack: the
// exponentials' range allows it, and it then seldom costs a reduction over
// lanes and a pass over the accumulators.
template <int DT>
__device__ inline void rescale(const tok_f32x4 (&s)[4], float cg, float shrink, float& m, float& l, tok_f32x4 (&acc)[DT]) {
  float top = -kInf;
#pragma unroll
  for (int t = 0; t < 4; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) top = fmaxf(top, s[t][i]);
  top *= cg;
  if (__ballot(top > m + kSlack) || shrink != 1.f) {
    top = over_groups(top);
    const float next = top > m + kSlack ? top : m;
    const float down = __builtin_amdgcn_exp2f(m - (next == -kInf ? 0.f : next));
    l *= down;
    const float all = down * shrink;
#pragma unroll
    for (int d = 0; d < DT; ++d) acc[d] *= all;
    m = next;
  }
}

// Then the probabilities as terms, 2^f P, and this lane's part l of their sum
// (before their rounding to terms, for lse is held to fp32).  f: what of the
// block's value exponent goes to P; below 2^-60 nothing is left of it.
constexpr int kLeast = -60;
template <int NP>
__device__ inline void weigh(const tok_f32x4 (&s)[4], float cg, int f, float m, float& l, tok_u32x4 (&pf)[2][NP]) {
  const float lift = kLift + f - (m == -kInf ? 0.f : m);
  float sum = 0.f;
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    float p[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      p[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[2 * u + (e >> 2)][e & 3], cg, lift));
      sum += p[e];
    }
    to_terms<tok_f16x2, NP>(p, pf[u]);
  }
  l = __builtin_fmaf(sum, pow2(-f), l);
}

// One workgroup: 16 columns (queries and heads that read one key/value head)
// of one sequence and one split of its tokens; its 4 waves take every fourth
// 64-token tile of the split and join their results in LDS.  Columns are
// numbered token by token, the G heads of a token side by side.
template <class E, int DP>  // DP: channels padded to 64
__global__ __launch_bounds__(256, DP <= 128 ? 2 : 1) void attend_few(Dev a) {
  typedef Form<E> F;
  constexpr int KS = DP / 32, DT = DP / 16, NQ = F::NQ, NP = F::NP;
  typedef typename E::store S;
  __shared__ float sm[4][16], sl[4][16];
  __shared__ __align__(16) float so[4][16][DP + 4];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 15, g = lane >> 4;
  const int split = blockIdx.x, hk = blockIdx.y, b = blockIdx.z;
  const int D = a.D, G = a.G;
  const Seq q = sequence(a, b);
  const int columns = q.n * G < 16 ? q.n * G : 16;
  if (columns == 0) return;
  const int col = r < columns ? r : columns - 1;
  const int qi = col / G, qh = hk * G + col % G;
  const Sight mine = sight(a, q.len, q.start + qi);
  // what all columns see together, and what each of them sees
  const Sight lowest = sight(a, q.len, q.start), highest = sight(a, q.len, q.start + (columns - 1) / G);
  const int ub = lowest.begin, ue = highest.end, cb = highest.begin, ce = lowest.end;
  const int t0 = ub / 64 + split * a.split_tiles;
  int t1 = (ue + 63) / 64;
  // the last split takes what is left
  if (split + 1 < a.splits && t0 + a.split_tiles < t1) t1 = t0 + a.split_tiles;

  tok_u32x4 qf[KS][NQ];
  load_query<E, KS>(a, q.row0 + qi, qh, g, qf);
  tok_f32x4 acc[DT];
#pragma unroll
  for (int d = 0; d < DT; ++d) acc[d] = tok_f32x4{0.f, 0.f, 0.f, 0.f};
  float m = -kInf, l = 0.f;  // l: this lane's part of 2^kLift times the sum
  int unit = -126;           // E

  const int32_t* pages = a.table + static_cast<int64_t>(b) * a.cols;
  // A tile's codes and scales are asked for before the tile before is worked on,
  // where the registers hold both.  (The page read behind them, under a condition,
  // waits for them: what overlaps is the work of the compute unit's other waves.)
  constexpr bool AHEAD = DP <= 128;
  struct Tile {
    uint32_t vb;  // block g, or kNone
    float ks, vs;
    tok_u32x4 kv[4][DP / 64], vv[DT];
  };
  auto load = [&](int tile, uint32_t page, Tile& x) __attribute__((always_inline)) {
    x.vb = settle(a, hk, tile * 4 + g, page);
    const uint32_t kb = __shfl(x.vb, (r >> 2) * 16);
    const bool kok = kb != kNone, vok = x.vb != kNone;
    const uint8_t* kp = a.k + (static_cast<int64_t>(kb) * 16 + (r & 3)) * D + g * 16;
    const uint8_t* vp = a.v + (static_cast<int64_t>(x.vb) * D + r) * 16;
    x.ks = vok ? a.ks[x.vb] : 1.f;
    x.vs = vok ? a.vs[x.vb] : 0x1p-126f;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int j = 0; j < DP / 64; ++j) {
        x.kv[t][j] = tok_u32x4{0, 0, 0, 0};
        if (kok && j * 64 + g * 16 < D) x.kv[t][j] = *reinterpret_cast<const tok_u32x4*>(kp + 4 * t * D + j * 64);
      }
#pragma unroll
    for (int d = 0; d < DT; ++d) {
      x.vv[d] = tok_u32x4{0, 0, 0, 0};
      if (vok && d * 16 < D) x.vv[d] = *reinterpret_cast<const tok_u32x4*>(vp + d * 256);
    }
  };
  Tile next;
  uint32_t page = peek(a, pages, (t0 + wave) * 4 + g, ub, ue);
  if (AHEAD && t0 + wave < t1) load(t0 + wave, page, next);
  page = peek(a, pages, (t0 + wave + (AHEAD ? 4 : 0)) * 4 + g, ub, ue);
  for (int tile = t0 + wave; tile < t1; tile += 4) {
    const int tok0 = tile * 64;
    Tile now;
    if (AHEAD) {
      now = next;
      if (tile + 4 < t1) load(tile + 4, page, next);
      page = peek(a, pages, (tile + 8) * 4 + g, ub, ue);
    } else {
      load(tile, page, now);
      page = peek(a, pages, (tile + 4) * 4 + g, ub, ue);
    }
    const uint32_t vb = now.vb;
    const bool vok = vb != kNone;
    auto& kv = now.kv;
    auto& vv = now.vv;
    // c times the key scale of block g; 0 kept off so that -inf stays -inf
    const float cg = fmaxf(a.c * now.ks, 0x1p-126f);
    const int ve = exponent_of(now.vs);
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
    const bool edge = tok0 < cb || tok0 + 64 > ce || __ballot(!vok) != 0;
    bool bad = false;
    if (edge) {
      const int base = tok0 + 16 * g;
      hide(s, base, mine, vok);
      // values that no column sees become 0; NaN among the others are
      // taken out of the product and put back where they are seen
      uint32_t keep[4];
#pragma unroll
      for (int t = 0; t < 4; ++t) keep[t] = kept(base, t, ub, ue);
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
    const int grown = max(unit, over_groups(ve));
    const int k = max(ve - grown, kDeep), f = max(ve - grown - k, kLeast);
    const float vk = pow2(k);
    tok_u32x4 pf[2][NP];
    rescale<DT>(s, cg, pow2(unit - grown), m, l, acc);
    weigh<NP>(s, cg, f, m, l, pf);
    unit = grown;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const tok_u32x4 vf = codes_f16(vv[d][2 * u], vv[d][2 * u + 1], vk);
#pragma unroll
        for (int n = 0; n < NP; ++n) acc[d] = mfma_f16(vf, pf[u][n], acc[d]);
      }
    if (bad) put_nan<DT>(a, vb, tok0, g, mine, acc);
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
  if (oc >= columns) return;
  const int64_t row = static_cast<int64_t>(q.row0 + oc / G) * a.q_heads + hk * G + oc % G;
  float* part = a.splits > 1 ? a.part + (static_cast<int64_t>(split) * a.T * a.q_heads + row) * (D + 2) : nullptr;
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

__device__ const uint32_t kZeros[4] = {0, 0, 0, 0};
typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(1))) const void global_void;

// Workgroup barrier behind which every wave sees what the others stored in LDS
// and loaded into it.  The waits are written out: __syncthreads() asks for none
// for a wave's loads into LDS, and at the head of a loop this compiler drops the
// one for the stores of the loop's end.
__device__ inline void lds_barrier() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// One workgroup: 4 waves of CT column tiles each, one sequence, one key/value
// head, one split of the tokens.  K's codes of a 64-token tile come straight
// into LDS, fragment by fragment (1 KB each: a lane's 16 bytes side by side, so
// reads have no bank conflicts), and every wave converts the fragments that
// it multiplies.  V's go through registers: each wave converts a quarter of
// them to f16 for all.  Two tiles in turn.  What bounds it is the vector
// units: conversions and exponentials beside the products; that is why V is
// converted once (K too would make LDS reads the bound).
// WHOLE: pages are multiples of 64 tokens, so that a tile lies in one page and
// its addresses are scalars; otherwise the vector units find blocks of 16
// tokens.  FULL: and no channel is padding, so that no load has a condition
// (32 query heads of 128, 8192 causal tokens: a tenth more time without FULL).
template <class E, int DP, int CT, bool WHOLE, bool FULL>
__global__ __launch_bounds__(256, DP <= 128 ? 2 : 1) void attend_many(Dev a) {
  typedef Form<E> F;
  typedef typename E::store S;
  constexpr int KS = DP / 32, DT = DP / 16, NJ = DP / 64, NQ = F::NQ, NP = F::NP;
  constexpr int VW = DT / 4;  // V fragments that a wave converts
  __shared__ __align__(16) uint8_t kbuf[2][4 * NJ * 1024];
  __shared__ __align__(16) uint8_t vbuf[2][DT * 2048];
  __shared__ int nan_seen[2][4];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 15, g = lane >> 4;
  // workgroup i runs on L2 cache i % 8: each cache gets a run of consecutive
  // units, so that one cache reads a head's codes; the last columns, which see
  // most in a causal call, come first
  const int D = FULL ? DP : a.D, G = a.G;
  uint32_t id = static_cast<uint32_t>(a.first) + blockIdx.x;
  {
    const uint32_t total = a.total, each = total / 8, rest = total % 8, c = id % 8;
    id = c * each + (c < rest ? c : rest) + id / 8;
  }
  const int ct = a.coltiles - 1 - static_cast<int>(id % a.coltiles);
  id /= a.coltiles;
  const int split = static_cast<int>(id % a.splits);
  id /= a.splits;
  const int hk = static_cast<int>(id % a.heads), b = static_cast<int>(id / a.heads);
  const Seq q = sequence(a, b);
  constexpr int WG = 64 * CT;  // columns
  const int columns = q.n * G, wg0 = ct * WG;
  if (wg0 >= columns) return;
  // what the workgroup's columns see together, and what this wave's do
  auto sight_of = [&](int col) { return sight(a, q.len, q.start + (col < columns ? col : columns - 1) / G); };
  const Sight lo = sight_of(wg0), hi = sight_of(wg0 + WG - 1);
  const int ub = lo.begin, ue = hi.end;
  const int col0 = wg0 + wave * 16 * CT;
  const Sight wlo = sight_of(col0), whi = sight_of(col0 + 16 * CT - 1);
  const int t0 = ub / 64 + split * a.split_tiles;
  int t1 = (ue + 63) / 64;
  if (split + 1 < a.splits && t0 + a.split_tiles < t1) t1 = t0 + a.split_tiles;

  tok_u32x4 qf[CT][KS][NQ];
  Sight mine[CT];
  tok_f32x4 acc[CT][DT];
  float m[CT], l[CT];
#pragma unroll
  for (int x = 0; x < CT; ++x) {
    const int col = col0 + 16 * x + r < columns ? col0 + 16 * x + r : columns - 1;
    const int qi = col / G, qh = hk * G + col % G;
    mine[x] = sight(a, q.len, q.start + qi);
    load_query<E, KS>(a, q.row0 + qi, qh, g, qf[x]);
    m[x] = -kInf;
    l[x] = 0.f;
#pragma unroll
    for (int d = 0; d < DT; ++d) acc[x][d] = tok_f32x4{0.f, 0.f, 0.f, 0.f};
  }
  // Tiles on their way: block g of the tile of this lane, its scales, K in
  // LDS, this wave's part of V in registers.
  const int32_t* pages = a.table + static_cast<int64_t>(b) * a.cols;
  // Tiles are asked for in turn: page_of a round before block.  The block is
  // this lane's; WHOLE: the first of the tile, a scalar, the page's column and
  // the tile's place in it counted rather than divided for.
  int column = WHOLE ? column_of(a, t0 * 4) : 0, place = WHOLE ? t0 * 4 - column * a.nb : 0, was = 0;
  auto page_of = [&](int tile) __attribute__((always_inline)) {
    if constexpr (WHOLE) {
      const uint32_t page = tile < t1 ? static_cast<uint32_t>(pages[column]) : kNone;
      was = place;
      place += 4;
      if (place == a.nb) {
        place = 0;
        ++column;
      }
      return page;
    } else {
      return peek(a, pages, tile * 4 + g, ub, ue);
    }
  };
  auto block = [&](int tile, uint32_t page) __attribute__((always_inline)) {
    if constexpr (WHOLE) {
      page = __builtin_amdgcn_readfirstlane(page);
      return page < static_cast<uint32_t>(a.pages) ? (page * a.heads + hk) * a.nb + was : kNone;
    } else
      return settle(a, hk, tile * 4 + g, page);
  };
  auto mine_of = [&](uint32_t vb) { return WHOLE && vb != kNone ? vb + g : vb; };
  tok_u32x4 vr[VW];
  typedef __attribute__((address_space(1))) const uint8_t global_u8;
  global_u8* zeros = (global_u8*)kZeros;
  constexpr bool EVEN = 4 % NJ == 0;  // every fourth fragment is 4 / NJ row tiles on
  const int klane = ((r >> 2) * 16 + (r & 3) + (EVEN ? wave / NJ * 4 : 0)) * D + (EVEN ? wave % NJ * 64 : 0) + g * 16;
  const int vlane = (g * D + r) * 16;
  auto fetch_k = [&](uint32_t vb, int buf) __attribute__((always_inline)) {
    global_u8* kp;
    if constexpr (WHOLE) {
      if (vb == kNone) return;  // whatever is there is hidden
      kp = (global_u8*)a.k + static_cast<int64_t>(vb) * 16 * D + klane;
    } else {
      vb = __shfl(vb, (r >> 2) * 16);
      kp = (global_u8*)a.k + (static_cast<int64_t>(vb) * 16 + (r & 3)) * D + g * 16;
    }
#pragma unroll
    for (int n = 0; n < NJ; ++n) {
      const int f = n * 4 + wave, t = f / NJ, j = f - t * NJ;
      global_u8* p = kp + (WHOLE && EVEN ? 16 / NJ * n * D : 4 * t * D + j * 64);
      if (WHOLE ? !FULL && j * 64 + g * 16 >= D : vb == kNone || j * 64 + g * 16 >= D) p = zeros;
      __builtin_amdgcn_global_load_lds((global_void*)p, (lds_void*)(&kbuf[buf][f * 1024]), 16, 0, 0);
    }
  };
  auto fetch_v = [&](uint32_t vb) __attribute__((always_inline)) {
    if (WHOLE && vb == kNone) {
#pragma unroll
      for (int n = 0; n < VW; ++n) vr[n] = tok_u32x4{0, 0, 0, 0};
      return;
    }
    global_u8* vp = WHOLE ? (global_u8*)a.v + static_cast<int64_t>(vb) * 16 * D + vlane
                          : (global_u8*)a.v + (static_cast<int64_t>(vb) * D + r) * 16;
#pragma unroll
    for (int n = 0; n < VW; ++n) {
      const int d = n * 4 + wave;
      global_u8* p = vp + d * 256;
      if (WHOLE ? !FULL && d * 16 >= D : vb == kNone || d * 16 >= D) p = zeros;
      vr[n] = *(__attribute__((address_space(1))) const tok_u32x4*)p;
    }
  };
  // a tile that some column of the workgroup does not see whole
  auto lost = [&](uint32_t vb) { return WHOLE ? vb == kNone : __ballot(vb == kNone) != 0; };
  auto partial = [&](int tok0, uint32_t vb) { return tok0 < hi.begin || tok0 + 64 > lo.end || lost(vb); };
  int unit = -126, grown = -126, rest = 0;  // E, E after the next tile, what of its exponents goes to P
  auto convert = [&](int tile, uint32_t vb, float vs, int buf) __attribute__((always_inline)) {
    settled(vs);  // its exponent, taken where it is loaded, would wait for that load
    int ve = exponent_of(vs);
    if (partial(tile * 64, vb)) {
      // values that no column sees become 0; NaN among the others are taken
      // out of the product and put back where they are seen
      bool any = false;
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const uint32_t keep = kept(tile * 64 + 16 * g, t, ub, ue);
#pragma unroll
        for (int n = 0; n < VW; ++n) {
          vr[n][t] &= keep;
          any |= nan_code(vr[n][t]);
          vr[n][t] = no_nan(vr[n][t]);
        }
      }
      // nor do the scales of whole tiles' unseen blocks count, which may be
      // anything (key scales do no harm: scores of -inf stay so).  Outside this
      // branch the test costs 10 us of the 596 of 8192 causal tokens.
      if (WHOLE && (tile * 64 + 16 * g + 15 < ub || tile * 64 + 16 * g >= ue)) ve = -126;
      const bool seen = __ballot(any) != 0;
      if (lane == 0) nan_seen[buf][wave] = seen;
    }
    grown = max(unit, over_groups(ve));
    const int k = max(ve - grown, kDeep);
    rest = max(ve - grown - k, kLeast);
    const float vk = pow2(k);
#pragma unroll
    for (int n = 0; n < VW; ++n)
#pragma unroll
      for (int u = 0; u < 2; ++u)
        *reinterpret_cast<tok_u32x4*>(&vbuf[buf][((n * 4 + wave) * 2 + u) * 1024 + lane * 16]) =
            codes_f16(vr[n][2 * u], vr[n][2 * u + 1], vk);
  };
  auto scales = [&](uint32_t vb, float& k, float& v) {
    vb = mine_of(vb);
    k = vb != kNone ? a.ks[vb] : 1.f;
    v = vb != kNone ? a.vs[vb] : 0x1p-126f;
  };

  tok_f32x4 s[CT][4];
  auto first = [&](int buf, tok_f32x4 (&s)[CT][4]) __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int x = 0; x < CT; ++x) s[x][t] = tok_f32x4{0.f, 0.f, 0.f, 0.f};
    // the four row tiles in turn: a product waits for none of its neighbours
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      tok_u32x4 kv[4];
#pragma unroll
      for (int t = 0; t < 4; ++t) kv[t] = *reinterpret_cast<const tok_u32x4*>(&kbuf[buf][(t * NJ + j) * 1024 + lane * 16]);
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const tok_u32x4 kf = F::k(kv[t][2 * h], kv[t][2 * h + 1]);
#pragma unroll
          for (int x = 0; x < CT; ++x)
#pragma unroll
            for (int n = 0; n < NQ; ++n) s[x][t] = F::mfma(kf, qf[x][2 * j + h][n], s[x][t]);
        }
    }
  };

  // A round works on tile t's softmax and second product and on tile t + 1's
  // first, which has nothing to wait for while the exponentials run.  K is
  // fetched two tiles ahead, V one.
  uint32_t cur = kNone, nxt = kNone;  // blocks of tiles t, t + 1
  uint32_t page = kNone;              // page of tile t + 2
  float ks = 1.f;
  if (t0 < t1) {
    float vs;
    cur = block(t0, page_of(t0));
    fetch_k(cur, t0 & 1);
    fetch_v(cur);
    scales(cur, ks, vs);
    if (t0 + 1 < t1) {
      nxt = block(t0 + 1, page_of(t0 + 1));
      fetch_k(nxt, (t0 + 1) & 1);
    }
    page = page_of(t0 + 2);
    convert(t0, cur, vs, t0 & 1);
    lds_barrier();
    first(t0 & 1, s);
  }
  for (int tile = t0; tile < t1; ++tile) {
    const int buf = tile & 1, tok0 = tile * 64;
    lds_barrier();  // what this round reads is in LDS, and nobody reads what it writes
    float ks1 = 1.f, vs1 = 1.f;
    const uint32_t far = block(tile + 2, page);
    if (tile + 1 < t1) {
      fetch_v(nxt);
      scales(nxt, ks1, vs1);
      if (tile + 2 < t1) fetch_k(far, buf);
      page = page_of(tile + 3);
    }
    const float cg = fmaxf(a.c * ks, 0x1p-126f), shrink = pow2(unit - grown);
    const int f = rest;
    unit = grown;
    if (tok0 < whi.begin || tok0 + 64 > wlo.end || lost(cur)) {
#pragma unroll
      for (int x = 0; x < CT; ++x) hide(s[x], tok0 + 16 * g, mine[x], cur != kNone);
    }
#pragma unroll
    for (int x = 0; x < CT; ++x) rescale<DT>(s[x], cg, shrink, m[x], l[x], acc[x]);
    // Tile t + 1's first product (past the last tile: of stale codes, and never
    // used) and this tile's probabilities, one group of products and its share
    // of exponentials at a time: left to itself the compiler puts all of one
    // before the other.
    tok_f32x4 s1[CT][4];
    tok_u32x4 pf[CT][2][NP];
    {
      float lift[CT], sum[CT], p[CT][8];
      tok_u32x4 kv[2][4];
      auto read_k = [&](int j) __attribute__((always_inline)) {
#pragma unroll
        for (int t = 0; t < 4; ++t)
          kv[j & 1][t] = *reinterpret_cast<const tok_u32x4*>(&kbuf[buf ^ 1][(t * NJ + j) * 1024 + lane * 16]);
      };
      read_k(0);
#pragma unroll
      for (int x = 0; x < CT; ++x) {
        lift[x] = kLift + f - (m[x] == -kInf ? 0.f : m[x]);
        sum[x] = 0.f;
#pragma unroll
        for (int t = 0; t < 4; ++t) s1[x][t] = tok_f32x4{0.f, 0.f, 0.f, 0.f};
      }
      constexpr int GROUPS = 8 * NJ;
#pragma unroll
      for (int n = 0; n < GROUPS; ++n) {
        const int j = n / 8, h = n / 4 % 2, t = n % 4;
        __builtin_amdgcn_sched_barrier(0);
        if (n % 8 == 0 && j + 1 < NJ) read_k(j + 1);
        const tok_u32x4 kf = F::k(kv[j & 1][t][2 * h], kv[j & 1][t][2 * h + 1]);
#pragma unroll
        for (int x = 0; x < CT; ++x)
#pragma unroll
          for (int q = 0; q < NQ; ++q) s1[x][t] = F::mfma(kf, qf[x][2 * j + h][q], s1[x][t]);
#pragma unroll
        for (int e = n * 16 / GROUPS; e < (n + 1) * 16 / GROUPS; ++e)
#pragma unroll
          for (int x = 0; x < CT; ++x) {
            p[x][e & 7] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[x][e >> 2][e & 3], cg, lift[x]));
            sum[x] += p[x][e & 7];
            settled(sum[x]);
            if ((e & 7) == 7) to_terms<tok_f16x2, NP>(p[x], pf[x][e >> 3]);
          }
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int x = 0; x < CT; ++x) {
        l[x] = __builtin_fmaf(sum[x], pow2(-f), l[x]);
        settled(l[x]);
      }
    }
    // the second product, each 16 channels' fragments read while the ones
    // before are multiplied
    tok_u32x4 vf[2][2];
    auto read_v = [&](int d) __attribute__((always_inline)) {
#pragma unroll
      for (int u = 0; u < 2; ++u)
        vf[d & 1][u] = *reinterpret_cast<const tok_u32x4*>(&vbuf[buf][(d * 2 + u) * 1024 + lane * 16]);
    };
    read_v(0);
#pragma unroll
    for (int d = 0; d < DT; ++d) {
      __builtin_amdgcn_sched_barrier(0);
      if (d + 1 < DT) read_v(d + 1);
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int x = 0; x < CT; ++x)
#pragma unroll
          for (int n = 0; n < NP; ++n) acc[x][d] = mfma_f16(vf[d & 1][u], pf[x][u][n], acc[x][d]);
    }
    __builtin_amdgcn_sched_barrier(0);
    if (partial(tok0, cur) && (nan_seen[buf][0] | nan_seen[buf][1] | nan_seen[buf][2] | nan_seen[buf][3])) {
#pragma unroll
      for (int x = 0; x < CT; ++x) put_nan<DT>(a, mine_of(cur), tok0, g, mine[x], acc[x]);
    }
    if (tile + 1 < t1) convert(tile + 1, nxt, vs1, buf ^ 1);
    cur = nxt;
    nxt = far;
    ks = ks1;
#pragma unroll
    for (int x = 0; x < CT; ++x)
#pragma unroll
      for (int t = 0; t < 4; ++t) s[x][t] = s1[x][t];
  }

#pragma unroll
  for (int x = 0; x < CT; ++x) {
    float sum = l[x];
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
    sum *= pow2(-kLift);
    const int col = col0 + 16 * x + r;
    if (col >= columns) continue;
    const int64_t row = static_cast<int64_t>(q.row0 + col / G) * a.q_heads + hk * G + col % G;
    float* part = a.splits > 1 ? a.part + (static_cast<int64_t>(split) * a.T * a.q_heads + row) * (D + 2) : nullptr;
    const float inv = part ? 1.f : sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
    for (int d = 0; d < DT; ++d) {
      if (d * 16 >= D) continue;
      float o[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] = ldexpf(acc[x][d][i], unit - kLift) * inv;
      if (part) {
        __builtin_memcpy(part + 2 + d * 16 + g * 4, o, 16);
      } else {
        S v[4] = {E::narrow(o[0]), E::narrow(o[1]), E::narrow(o[2]), E::narrow(o[3])};
        __builtin_memcpy(static_cast<S*>(a.out) + row * D + d * 16 + g * 4, v, sizeof v);
      }
    }
    if (g == 0) {
      if (part) {
        part[0] = m[x];
        part[1] = sum;
      } else if (a.lse) {
        a.lse[row] = sum == 0.f ? -kInf : m[x] * kLn2 + logf(sum);
      }
    }
  }
}

// out and lse from the partial results of a split call: one wave a row.
// Everything of U splits is read at once: a chain of reads was most of a single
// token's time.
template <class E, int NV>  // NV: channels a lane
__global__ __launch_bounds__(256) void attend_join(Dev a) {
  constexpr int U = 8;
  const int64_t row = (a.first + blockIdx.x) * 4 + (threadIdx.x >> 6), rows = static_cast<int64_t>(a.T) * a.q_heads;
  if (row >= rows) return;
  const int lane = threadIdx.x & 63, D = a.D;
  const float* part = a.part + row * (D + 2);
  const int64_t step = rows * (D + 2);
  int ch[NV];  // lanes past the last channel work on it again and store nothing
#pragma unroll
  for (int i = 0; i < NV; ++i) ch[i] = lane + 64 * i < D ? lane + 64 * i : D - 1;
  float m = -kInf, l = 0.f, o[NV] = {};
  for (int s0 = 0; s0 < a.splits; s0 += U) {
    const int n = a.splits - s0 < U ? a.splits - s0 : U;
    const float* p = part + (s0 + (lane < n ? lane : n - 1)) * step;
    const float pm = p[0], pl = p[1];
    float v[U][NV];
#pragma unroll
    for (int s = 0; s < U; ++s)
#pragma unroll
      for (int i = 0; i < NV; ++i) v[s][i] = part[(s0 + (s < n ? s : n - 1)) * step + 2 + ch[i]];
    const float next = fmaxf(m, wave_max(pm)), ref = next == -kInf ? 0.f : next;
    const float down = __builtin_amdgcn_exp2f(m - ref);
    const float w = lane < n && pl != 0.f ? __builtin_amdgcn_exp2f(pm - ref) : 0.f;  // 0: nothing seen
    m = next;
    l = l * down + (lane < n ? w * pl : 0.f);
#pragma unroll
    for (int i = 0; i < NV; ++i) o[i] *= down;
#pragma unroll
    for (int s = 0; s < U; ++s) {
      const float ws = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(w), s));
#pragma unroll
      for (int i = 0; i < NV; ++i) o[i] += s < n ? ws * v[s][i] : 0.f;
    }
  }
  l = wave_sum(l);
  const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
  for (int i = 0; i < NV; ++i)
    if (lane + 64 * i < D) static_cast<typename E::store*>(a.out)[row * D + lane + 64 * i] = E::narrow(o[i] * inv);
  if (a.lse && lane == 0) a.lse[row] = l == 0.f ? -kInf : m * kLn2 + logf(l);
}

int64_t up(int64_t a, int64_t b) { return (a + b - 1) / b; }

// New tokens of a sequence: max_new is a bound, which may be a loose one.
int64_t most_new(const c3c_kv_batch& b) { return b.max_new < b.T ? b.max_new : b.T; }

// 64-token tiles that one column tile sees at most
int64_t tiles_seen(const c3c_kv_batch& b, int64_t page, int64_t window) {
  int64_t tokens = b.max_len < b.cols * page ? b.max_len : b.cols * page;
  if (window > 0 && window + most_new(b) < tokens) tokens = window + most_new(b) + 64;
  return up(tokens, 64);
}

// Column tiles a wave: two keep two waves on a SIMD, whose exponentials and
// matrix products overlap; f32's three terms leave room for one.
constexpr int column_tiles(int dp, int terms) { return dp > 192 || terms > 1 ? 1 : 2; }
int64_t workgroup_columns(int64_t dim, int dtype) {
  return 64 * column_tiles(static_cast<int>(dim), dtype == C3C_DTYPE_F32 ? 3 : 1);
}

// Calls of at most 16 columns a sequence and head take attend_few.
bool few(int64_t columns) { return columns <= 16; }

template <class E, int NQ, bool WHOLE, bool FULL>
auto pick_many(int dim) {
  return dim <= 64    ? attend_many<E, 64, column_tiles(64, NQ), WHOLE, FULL>
         : dim <= 128 ? attend_many<E, 128, column_tiles(128, NQ), WHOLE, FULL>
         : dim <= 192 ? attend_many<E, 192, column_tiles(192, NQ), WHOLE, FULL>
                      : attend_many<E, 256, column_tiles(256, NQ), WHOLE, FULL>;
}

template <class E>
hipError_t run(const AttendArgs& h, const AttendPlan& p, int dtype, hipStream_t s) {
  const int64_t G = h.q_heads / h.c.heads, columns = most_new(h.b) * G, nb = h.c.page / 16;
  const int64_t cap = h.b.cols * h.c.page, coltiles = up(columns, workgroup_columns(h.c.dim, dtype));
  const int64_t blocks = coltiles * p.splits * h.c.heads * h.b.B, joins = up(h.b.T * h.q_heads, 4);
  // 32-bit numbering of columns, blocks and workgroups
  if (up(h.b.T * G, 16) * 16 + 1024 > 0x7fffffff ||
      h.c.pages * h.c.heads * nb >= 0xffffffffll || (few(columns) ? h.b.B > 65535 || h.c.heads > 65535 : blocks > 0x7fffffff))
    return hipErrorInvalidConfiguration;
  Dev a{static_cast<const uint8_t*>(h.c.k), static_cast<const uint8_t*>(h.c.v), h.c.k_scale, h.c.v_scale,
              h.b.table, h.b.cu, h.b.len, h.q, h.out, h.lse, h.part, h.ld_q,
              static_cast<int>(h.b.T), static_cast<int>(h.q_heads), static_cast<int>(h.c.heads), static_cast<int>(G),
              static_cast<int>(h.c.dim), static_cast<int>(h.c.pages), static_cast<int>(nb),
              (nb & (nb - 1)) == 0 ? __builtin_ctzll(nb) : -1, static_cast<int>(h.b.cols),
              // room for the tile arithmetic past the last token
              static_cast<int>(cap < 0x7fff0000 ? cap : 0x7fff0000), h.causal, static_cast<int>(h.window),
              h.scale * kLog2e, p.splits, static_cast<int>(up(tiles_seen(h.b, h.c.page, h.window), p.splits)),
              static_cast<int>(coltiles), static_cast<uint32_t>(few(columns) ? 0 : blocks), 0};
  hipError_t e;
  if (few(columns)) {
    auto k = a.D <= 64 ? attend_few<E, 64> : a.D <= 128 ? attend_few<E, 128> : a.D <= 192 ? attend_few<E, 192> : attend_few<E, 256>;
    hipLaunchKernelGGL(k, dim3(p.splits, a.heads, static_cast<unsigned>(h.b.B)), dim3(256), 0, s, a);
    e = hipGetLastError();
  } else {
    constexpr int NQ = Form<E>::NQ;
    auto k = nb % 4 != 0 ? pick_many<E, NQ, false, false>(a.D) : a.D % 64 != 0 ? pick_many<E, NQ, true, false>(a.D) : pick_many<E, NQ, true, true>(a.D);
    e = in_launches(blocks, 256, [&](int64_t first, unsigned count) {
      a.first = first;
      hipLaunchKernelGGL(k, dim3(count), dim3(256), 0, s, a);
    });
  }
  if (e == hipSuccess && p.splits > 1) {
    auto join = a.D <= 64 ? attend_join<E, 1> : a.D <= 128 ? attend_join<E, 2> : attend_join<E, 4>;
    e = in_launches(joins, 256, [&](int64_t first, unsigned count) {
      a.first = first;
      hipLaunchKernelGGL(join, dim3(count), dim3(256), 0, s, a);
    });
  }
  return e;
}

}  // namespace

AttendPlan plan_attend(const c3c_kv_cache& c, const c3c_kv_batch& b, int dtype, int64_t q_heads,
                       int causal, int64_t window) {
  AttendPlan p;
  const int64_t columns = most_new(b) * (q_heads / c.heads), tiles = tiles_seen(b, c.page, window);
  const int64_t base = up(columns, few(columns) ? 16 : workgroup_columns(c.dim, dtype)) * c.heads * b.B;
  if (base == 0) return p;
  const int64_t cus = device_compute_units(), most = up(tiles, 4);
  int64_t s = 1;
  if (few(columns)) {
    // two workgroups a compute unit, of at least one tile a wave and at most
    // 256 tiles: a split more costs its start (64 sequences of 1000 to 32768
    // tokens, 8 heads of 128: one split 452 us, four 494), but a sequence far
    // longer than the others would be waited for
    s = up(2 * cus, base);
    if (s < up(tiles, 256)) s = up(tiles, 256);
    if (s > most) s = most;
  } else {
    // the fewest rounds of workgroups, counted in tiles: each round costs its
    // tiles and about 3 more to begin and end, the join its launch and its
    // traffic (a tile takes about 2.8 us at 128 channels, 1 us reads and writes
    // 4 MB).  Two bf16 sequences of 1560 queries, 12 heads and 9400 tokens: 312
    // workgroups for 512 places; three splits 318 us, one 423.
    const int64_t places = cus * (c.dim <= 128 ? 2 : 1);
    const double bytes = 8.0 * b.T * q_heads * (c.dim + 2), tile_us = 2.8 * c.dim / 128;
    double best = 0;
    for (int64_t n = 1; n <= most && n <= 32; ++n) {
      const double t = up(base * n, places) * (static_cast<double>(up(tiles, n)) + 3) +
                       (n > 1 ? (5 + n * bytes / 4e6) / tile_us : 0);
      if (n == 1 || t < best) {
        best = t;
        s = n;
      }
    }
  }
  if (s > 1) {
    p.splits = static_cast<int>(s);
    p.part_bytes = s * b.T * q_heads * (c.dim + 2) * 4;
  }
  return p;
}

hipError_t launch_attend(const AttendArgs& a, int dtype, const AttendPlan& plan, hipStream_t s) {
  if (a.b.B == 0 || a.b.T == 0 || a.b.max_new == 0) return hipSuccess;
  return dtype == C3C_DTYPE_BF16  ? run<ElemBf16>(a, plan, dtype, s)
         : dtype == C3C_DTYPE_F16 ? run<ElemF16>(a, plan, dtype, s)
                                  : run<ElemF32>(a, plan, dtype, s);
}

}  // namespace c3c
