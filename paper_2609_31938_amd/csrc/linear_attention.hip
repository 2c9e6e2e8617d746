// Linear attention with a decay for each head:
//   S <- exp(g_t) S + k_t v_t^T,   out_t = scale q_t S        (S: dim_k x dim_v)
//
// By chunks of C tokens, with G_i the sum of g over the chunk's tokens up to i:
//   out_i = scale (exp(G_i) q_i S + sum_{j <= i} exp(G_i - G_j) (q_i . k_j) v_j)
//   S    <- exp(G_C) S + sum_j k_j (exp(G_C - G_j) v_j)^T
// Four products for the matrix cores.  Every weight is the exponential of a
// difference that is at most 0 for decays, so nothing overflows however fast a
// head forgets; the sums G are formed in 64 bits and kept as two floats, since
// they may be large (a token that resets the state) next to their differences.
//
// Precision: an operand of the matrix cores is a sum of bf16 terms.  Inputs are
// exact in 1 (bf16), 2 (f16) or 3 (f32) of them; S and the weighted products P of
// queries and keys, which meet outputs of 16 bits, take 2 (2^-18 of a value; one
// would add an error as large as the output's own rounding), for f32 3; weighted
// values, which end in the fp32 states, take 3.
//
// chunks: a workgroup takes one head and up to 128 columns of S, of which a wave
//   holds 16 or 32 in the matrix cores' accumulators, all dim_k rows of them: the
//   layout of an accumulator is that of an operand whose rows are taken in
//   another order, so S goes into the first product without passing through LDS,
//   and no two waves share a column of out.  What the waves share is q, k and P,
//   in LDS.  A clip of 32760 tokens x 32 heads of 128 (bf16) takes 304 to 313
//   us, at the clock that a card keeps over many of them; 350 in the short runs that
//   the other figures of this paragraph are from.  Its loads and stores alone take
//   211; two waves a SIMD (of 247 registers) wait for LDS, products and barriers in
//   turn: without loads and stores it takes 291, without any one of the products 300
//   to 350.  Tried, and slower or no faster there: 16 columns a wave with four
//   waves a SIMD (registers in scratch memory, 410), chunks of 64 tokens (340 to
//   400; a frame of 1560 tokens 31 us, 23 so), one term in place of two or three
//   (370), S scaled only where it has to be.
// parts: few heads and sequences leave compute units idle.  Their sequences
//   are split into parts of whole chunks: one launch forms each part's own
//   state (143 us there, 160 in the short runs; it reads k and v once more, whose
//   loads alone take 110 in these), one joins them in order (13 us), one forms the
//   outputs of all parts.
// tokens: few new tokens (single ones, drafted ones) take the recurrence as it
//   stands, S in registers: it is bound by reading and writing S (64 sequences x
//   32 heads of 128: 268 MB in 42 to 56 us by what the caches hold).
#include "token_dev.h"
#include "tokens_internal.h"

namespace c3c {
namespace {

typedef short tok_i16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) tok_i16x4 lds_i16x4;

constexpr int C = 32;  // tokens of a chunk: a step of the matrix cores
constexpr double kLog2e = 1.4426950408889634;
constexpr float kForget = -110.f;  // exp of it is 0 in fp32

struct Args {
  float* state;
  const int32_t *cu, *len, *slot;
  const void *q, *k, *v;
  const float* decay;
  void* out;
  float* part;    // [B][parts][heads][dim_k][dim_v], then a factor for each
  float* factor;  // [B][parts][heads]
  int64_t slots, B, T, ld_q, ld_k, ld_v, ld_decay;
  int64_t part_tokens;  // of every part but the last
  int64_t first;        // workgroup of this launch
  int64_t groups;       // workgroups of the call
  int heads, qk_heads, dim_k, dim_v, parts, slices;
  float scale;
};

// The new tokens of a sequence.
struct Seq {
  int64_t first, n;
  int64_t slot;  // -1: none
  bool fresh;    // begins at zero
};
__device__ inline Seq sequence(const Args& a, int64_t b) {
  Seq s;
  const int64_t c0 = a.cu[b], c1 = a.cu[b + 1];
  s.first = c0 < 0 ? 0 : c0 < a.T ? c0 : a.T;
  const int64_t end = c1 < s.first ? s.first : c1 < a.T ? c1 : a.T;
  s.n = end - s.first;
  const int64_t slot = a.slot ? a.slot[b] : b;
  s.slot = slot >= 0 && slot < a.slots ? slot : -1;
  s.fresh = s.slot < 0 || a.len[b] <= c1 - c0;
  return s;
}
// parts of it that hold tokens
__device__ inline int live_parts(const Args& a, int64_t n) {
  const int64_t p = (n + a.part_tokens - 1) / a.part_tokens;
  return static_cast<int>(p < 1 ? 1 : p < a.parts ? p : a.parts);
}

__device__ inline float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

template <class E>
struct Terms;  // bf16 terms that hold an input exactly
template <>
struct Terms<ElemBf16> {
  static constexpr int IN = 1, OUT = 2;
};
template <>
struct Terms<ElemF16> {
  static constexpr int IN = 2, OUT = 2;
};
template <>
struct Terms<ElemF32> {
  static constexpr int IN = 3, OUT = 3;
};
constexpr int kStateTerms = 3;  // of a weighted value: the state is an output in fp32

// Two values as NT terms of bf16 each, the next the rounding error of those
// before it: 2 terms hold 2^-18 of a value, 3 all of a float.
template <int NT>
__device__ inline void split2(float x, float y, uint32_t (&w)[NT]) {
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    w[t] = __builtin_bit_cast(uint32_t, __builtin_convertvector((tok_f32x2{x, y}), tok_bf16x2));
    if (t + 1 < NT) {
      x -= __uint_as_float(w[t] << 16);
      y -= __uint_as_float(w[t] & 0xffff0000u);
    }
  }
}

template <int NT>
__device__ inline void split8(const float (&f)[8], tok_bf16x8 (&o)[NT]) {
  tok_u32x4 w[NT];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t p[NT];
    split2<NT>(f[2 * i], f[2 * i + 1], p);
#pragma unroll
    for (int t = 0; t < NT; ++t) w[t][i] = p[t];
  }
#pragma unroll
  for (int t = 0; t < NT; ++t) o[t] = __builtin_bit_cast(tok_bf16x8, w[t]);
}

// acc += a b over the pairs of terms whose product exceeds 2^-9(LAST + 1)
template <int LAST, int NA, int NB>
__device__ inline void mfma_terms(const tok_bf16x8 (&a)[NA], const tok_bf16x8 (&b)[NB], tok_f32x4& acc) {
#pragma unroll
  for (int i = 0; i < NA; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j)
      if (i + j <= LAST) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[i], b[j], acc, 0, 0, 0);
}

// Everything that this wave has stored to LDS has landed before the others
// pass.  (A __syncthreads() at a loop's head has been compiled without the wait
// for the stores at the loop's end.)
__device__ inline void meet() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// v, of which the compiler knows nothing: what is computed from it in a loop
// stays there.  (Left to itself it forms all addresses of a chunk before the loop,
// and keeps them in scratch memory.)
__device__ inline int unknown(int v) {
  asm volatile("" : "+v"(v));
  return v;
}

// Operands of the matrix cores hold 8 of 32 rows a lane, in any order that both
// share: here rows 4 g .. 4 g + 3 and those 16 further on, g = lane / 16, as an
// accumulator's two tiles lie.  By columns (a row is a token, the lane's column
// its lane % 16): ds_read_b64_tr_b16 gives lane i of 16 element i % 4 of what
// lanes 4 e + i / 4 address, e = 0 .. 3.  at: where this lane reads, in the first
// row's place.
__device__ inline tok_bf16x8 column8(const unsigned char* at, int pitch) {
  const tok_i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)at);
  const tok_i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(at + 16 * pitch));
  return __builtin_bit_cast(tok_bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}
// By rows (the row of this lane, 8 of 32 channels from at on) ...
__device__ inline tok_bf16x8 row8(const unsigned char* at) {
  const tok_i16x4 lo = *reinterpret_cast<const tok_i16x4*>(at), hi = *reinterpret_cast<const tok_i16x4*>(at + 32);
  return __builtin_bit_cast(tok_bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}
// ... or where a row keeps these 8 side by side (q, P): 16-byte pieces, whose
// places change from row to row so that neither 16 rows of one piece nor a mixture
// of two pieces, as the lanes of a 16-byte read are served, meet in a bank.
// Place of piece g of the first 32 channels in a row; that of the s-th is the same
// ^ 64 s.
template <int PITCH>
__device__ inline int piece_at(int row, int g) {
  const int h = PITCH >= 256 ? row & 15 : PITCH == 128 ? row >> 1 & 7 : -(row >> 2) & 3;
  return row * PITCH + ((h >> 2) << 6) + ((g ^ (h & 3)) << 4);
}
// Place of the four channels that are the c-th in order.
template <int PITCH>
__device__ inline int four_at(int row, int c) {
  return (piece_at<PITCH>(row, c & 3) ^ ((c >> 3) << 6)) + (c >> 2 & 1) * 8;
}

// E: input type.  DK: rows of S (dim_k, filled up with zeros).  DVS: columns of
// this workgroup, CT tiles of 16 a wave.  C: tokens of a chunk.  STATES: only the state of a
// part.
template <class E, int DK, int DVS, int CT, bool STATES>
struct Chunk {
  static constexpr int NI = Terms<E>::IN, NO = Terms<E>::OUT;
  static constexpr int THREADS = DVS * 4 / CT;
  // Bytes between rows.  Of k and v, read by columns, 8 rows of 32 bytes meet in
  // no bank: an odd number of 32 bytes; their second 8 of 16 rows begin 16 bytes
  // further on, so that 16 rows of 8 or 16 bytes don't either.
  static constexpr int Q_PITCH = DK * 2, K_PITCH = DK * 2 + 32, V_PITCH = DVS * 2 + 32, P_PITCH = C * 2;
  static constexpr int Q_BYTES = STATES ? 0 : NI * C * Q_PITCH, K_BYTES = NI * C * K_PITCH, V_BYTES = NI * C * V_PITCH;
  static constexpr int P_BYTES = STATES ? 0 : NO * C * P_PITCH;
  static constexpr int K_AT = Q_BYTES, V_AT = K_AT + K_BYTES;
  static constexpr int W_AT = V_AT + V_BYTES;  // weights: 4 floats a token, and the chunk's
  static constexpr int BUFFER = (W_AT + 4 * C * 4 + 4 + 255) / 256 * 256;
  // Eight waves a compute unit, in one workgroup or two.  Two buffers where they
  // fit: the products of a chunk's queries and keys are then formed beside the
  // chunk before.
  static constexpr int LDS = 160 * 1024 / (512 / THREADS);  // of a workgroup
  static constexpr int BUFS = STATES || 2 * (BUFFER + P_BYTES) > LDS ? 1 : 2;
  static constexpr int P_AT = BUFS * BUFFER, BYTES = P_AT + BUFS * P_BYTES;
  // 16-byte pieces of q or k, of v, and how many a thread takes
  static constexpr int K_ALL = C * DK / E::VEC, V_ALL = C * DVS / E::VEC;
  static constexpr int KP = (K_ALL + THREADS - 1) / THREADS, VP = (V_ALL + THREADS - 1) / THREADS;
  // waves of a SIMD: two (256 registers), for a part's state alone four (128)
  static constexpr int MOST = STATES ? 4 : 2, FIT = 160 * 1024 / BYTES * THREADS / 256;
  static constexpr int WAVES = FIT < MOST ? FIT : MOST;
};

template <class E, int DK, int DVS, int CT, bool STATES>
__global__ __launch_bounds__((Chunk<E, DK, DVS, CT, STATES>::THREADS), (Chunk<E, DK, DVS, CT, STATES>::WAVES)) void chunks(Args a) {
  typedef Chunk<E, DK, DVS, CT, STATES> K;
  typedef typename E::store store;
  constexpr int NI = K::NI, NO = K::NO, VEC = E::VEC, THREADS = K::THREADS, NW = THREADS / 64;
  constexpr int LAST = NO - 1;
  constexpr int KS = DK / 32, RT = C / 16;
  __shared__ __align__(16) unsigned char lds[K::BYTES];
  int tid = threadIdx.x;
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r = lane & 15, g = lane >> 4;

  // workgroup -> (sequence, part, head) and slice: the slices of a head, which
  // read the same q and k, run on the same one of the 8 L2 caches
  const int64_t id = a.first + blockIdx.x;
  const int64_t unit = id / (8 * a.slices) * 8 + id % 8;
  const int slice = static_cast<int>(id / 8 % a.slices);
  if (unit >= a.groups) return;
  const int h = static_cast<int>(unit % a.heads);
  const int runs = STATES ? a.parts - 1 : a.parts;
  const int part = static_cast<int>(unit / a.heads % runs);
  const int64_t b = unit / a.heads / runs;
  const Seq seq = sequence(a, b);
  const int live = live_parts(a, seq.n);
  if (seq.n == 0 || part >= (STATES ? live - 1 : live)) return;
  const int64_t t0 = seq.first + part * a.part_tokens;
  const int64_t end = part + 1 < live ? t0 + a.part_tokens : seq.first + seq.n;
  const int hk = h / (a.heads / a.qk_heads);
  const int c0 = slice * DVS;  // first column
  const store* qp = static_cast<const store*>(a.q) + static_cast<int64_t>(hk) * a.dim_k;
  const store* kp = static_cast<const store*>(a.k) + static_cast<int64_t>(hk) * a.dim_k;
  const store* vp = static_cast<const store*>(a.v) + static_cast<int64_t>(h) * a.dim_v + c0;
  const int cols = a.dim_v - c0 < DVS ? a.dim_v - c0 : DVS;

  // ---- a chunk's inputs: asked for one chunk ahead, in registers until their place in LDS is free
  tok_u32x4 rq[STATES ? 1 : K::KP], rk[K::KP], rv[K::VP];
  float rg = 0.f;
  // Rows past the last one and columns past the width are read from others, and
  // made zero when they are placed: a load behind a condition is waited for
  // before the next.  The offsets in a chunk are 32 bits.
  auto row_of = [&](int i, int per) __attribute__((always_inline)) { return (i * THREADS + tid) / per % C; };
  auto col_of = [&](int per) __attribute__((always_inline)) { return tid % per * VEC; };
  static_assert(THREADS % (DK / VEC) == 0 && THREADS % (DVS / VEC) == 0, "a thread's pieces lie in one column");
  auto get = [&](const store* p, int64_t ld, int rows, int i, int per, int width) __attribute__((always_inline)) {
    const int row = row_of(i, per), col = col_of(per);
    const uint32_t off = static_cast<uint32_t>(row < rows ? row : rows - 1) * (static_cast<uint32_t>(ld) * sizeof(store)) +
                         (col < width ? col : 0) * sizeof(store);
    tok_u32x4 x;
    __builtin_memcpy(&x, reinterpret_cast<const char*>(p) + off, 16);
    return x;
  };
  auto ask = [&](int64_t t) __attribute__((always_inline)) {
    const int rows = end - t < C ? static_cast<int>(end - t) : C;
    if constexpr (!STATES) {
#pragma unroll
      for (int i = 0; i < K::KP; ++i) rq[i] = get(qp + t * a.ld_q, a.ld_q, rows, i, DK / VEC, a.dim_k);
    }
#pragma unroll
    for (int i = 0; i < K::KP; ++i) rk[i] = get(kp + t * a.ld_k, a.ld_k, rows, i, DK / VEC, a.dim_k);
#pragma unroll
    for (int i = 0; i < K::VP; ++i) rv[i] = get(vp + t * a.ld_v, a.ld_v, rows, i, DVS / VEC, cols);
    if (wave == 0) rg = a.decay[(t + (lane < rows ? lane : rows - 1)) * a.ld_decay + h];
  };
  auto put = [&](tok_u32x4 x, unsigned char* at, int plane, int pitch, int i, int per, int all, bool q) __attribute__((always_inline)) {
    if (all % THREADS != 0 && i * THREADS + tid >= all) return;
    const int row = row_of(i, per), col = col_of(per);
    unsigned char* to = at + (q ? four_at<K::Q_PITCH>(row, col / 4) : row * pitch + (row & 8) * 2 + col * 2);
    unsigned char* to2 = at + (q ? four_at<K::Q_PITCH>(row, col / 4 + 1) : 0);
    if constexpr (NI == 1) {
      if (q) {
        *reinterpret_cast<tok_u32x2*>(to) = tok_u32x2{x[0], x[1]};
        *reinterpret_cast<tok_u32x2*>(to2) = tok_u32x2{x[2], x[3]};
      } else {
        *reinterpret_cast<tok_u32x4*>(to) = x;
      }
    } else {
      store v[VEC];
      __builtin_memcpy(v, &x, 16);
      uint32_t w[NI][VEC / 2];
#pragma unroll
      for (int e = 0; e < VEC; e += 2) {
        uint32_t t[NI];
        split2<NI>(E::widen(v[e]), E::widen(v[e + 1]), t);
#pragma unroll
        for (int n = 0; n < NI; ++n) w[n][e / 2] = t[n];
      }
#pragma unroll
      for (int n = 0; n < NI; ++n) {
        if (VEC == 8 && q) {
          __builtin_memcpy(__builtin_assume_aligned(to + n * plane, 8), w[n], 8);
          __builtin_memcpy(__builtin_assume_aligned(to2 + n * plane, 8), w[n] + 2, 8);
        } else {
          __builtin_memcpy(__builtin_assume_aligned(to + n * plane, VEC * 2), w[n], VEC * 2);
        }
      }
    }
  };
  auto place = [&](unsigned char* buf, int64_t t) __attribute__((always_inline)) {
    const int rows = end - t < C ? static_cast<int>(end - t) : C;
    if (rows < C || a.dim_k < DK || cols < DVS) {
      const tok_u32x4 none = {0u, 0u, 0u, 0u};
#pragma unroll
      for (int i = 0; i < K::KP; ++i) {
        const bool ok = row_of(i, DK / VEC) < rows && col_of(DK / VEC) < a.dim_k;
        if constexpr (!STATES) rq[i] = ok ? rq[i] : none;
        rk[i] = ok ? rk[i] : none;
      }
#pragma unroll
      for (int i = 0; i < K::VP; ++i) rv[i] = row_of(i, DVS / VEC) < rows && col_of(DVS / VEC) < cols ? rv[i] : none;
      rg = lane < rows ? rg : 0.f;
    }
    if constexpr (!STATES) {
#pragma unroll
      for (int i = 0; i < K::KP; ++i) put(rq[i], buf, C * K::Q_PITCH, K::Q_PITCH, i, DK / VEC, K::K_ALL, true);
    }
#pragma unroll
    for (int i = 0; i < K::KP; ++i) put(rk[i], buf + K::K_AT, C * K::K_PITCH, K::K_PITCH, i, DK / VEC, K::K_ALL, false);
#pragma unroll
    for (int i = 0; i < K::VP; ++i) put(rv[i], buf + K::V_AT, C * K::V_PITCH, K::V_PITCH, i, DVS / VEC, K::V_ALL, false);
    if (wave == 0) {
      double s = static_cast<double>(rg < kForget ? kForget : rg) * kLog2e;
#pragma unroll
      for (int o = 1; o < C; o <<= 1) {
        const double up = __shfl_up(s, o);
        if (lane >= o) s += up;
      }
      const double all = __shfl(s, C - 1);
      if (lane < C) {
        // for each token G in units of log 2 (its float and the rest), scale
        // exp(G_i), exp(G_C - G_i); exp(G_C)
        float* const w = reinterpret_cast<float*>(buf + K::W_AT) + lane;
        const float hi = static_cast<float>(s);
        w[0] = hi;
        // a sum that is infinite or NaN has no rest
        w[C] = fabsf(hi) < __builtin_inff() ? static_cast<float>(s - static_cast<double>(hi)) : 0.f;
        w[2 * C] = a.scale * exp2_of(hi);
        w[3 * C] = exp2_of(static_cast<float>(all - s));
        if (lane == 0) w[4 * C] = exp2_of(static_cast<float>(all));
      }
    }
  };

  // ---- S: tile [s][t] holds rows 32 s + 16 t + 4 g + e of this wave's column
  // 16 c + r
  const int wc = wave * 16 * CT, col = c0 + wc + r;
  tok_f32x4 S[CT][KS][2];
  float factor = 1.f;
  const int64_t head_size = static_cast<int64_t>(a.dim_k) * a.dim_v;
  const float* from = STATES                ? nullptr
                      : a.parts > 1         ? a.part + ((b * a.parts + part) * a.heads + h) * head_size
                      : seq.fresh           ? nullptr
                                            : a.state + (seq.slot * a.heads + h) * head_size;
#pragma unroll
  for (int s = 0; s < KS; ++s)
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int row = 32 * s + 16 * t + 4 * g + e;
#pragma unroll
        for (int c = 0; c < CT; ++c)
          S[c][s][t][e] = from && row < a.dim_k && col + 16 * c < a.dim_v ? from[static_cast<int64_t>(row) * a.dim_v + col + 16 * c] : 0.f;
      }
  const int64_t lane_out = static_cast<int64_t>(r) * a.heads * a.dim_v + wc + 4 * g;

  // P of a chunk: tiles of 16 keys x 16 queries on and below the diagonal, in turn
  auto weigh = [&](const unsigned char* buf, unsigned char* P) __attribute__((always_inline)) {
    constexpr int JOBS = 3;
    const int r = tid & 15, g = tid >> 4 & 3, q_at = piece_at<K::Q_PITCH>(r, g);
    const float *g_hi = reinterpret_cast<const float*>(buf + K::W_AT), *g_lo = g_hi + C;
    static_assert(NW >= JOBS && RT == 2, "a tile a wave");
    const int j = wave;
    if (j >= JOBS) return;
    const int qt = j > 0, kt = j > 1;
    tok_f32x4 p = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      tok_bf16x8 fq[NI], fk[NI];
#pragma unroll
      for (int n = 0; n < NI; ++n) {
        fq[n] = *reinterpret_cast<const tok_bf16x8*>(buf + (n * C + qt * 16) * K::Q_PITCH + (q_at ^ s * 64));
        fk[n] = row8(buf + K::K_AT + (n * C + kt * 16 + r) * K::K_PITCH + (r & 8) * 2 + s * 64 + g * 8);
      }
      mfma_terms<LAST, NI, NI>(fk, fq, p);
    }
    const int i = qt * 16 + r, key = kt * 16 + 4 * g;
    const tok_f32x4 hi = *reinterpret_cast<const tok_f32x4*>(g_hi + key), lo = *reinterpret_cast<const tok_f32x4*>(g_lo + key);
    const float ih = g_hi[i], il = g_lo[i];
#pragma unroll
    for (int e = 0; e < 4; ++e) p[e] = key + e <= i ? p[e] * a.scale * exp2_of((ih - hi[e]) + (il - lo[e])) : 0.f;
    uint32_t w0[NO], w1[NO];
    split2<NO>(p[0], p[1], w0);
    split2<NO>(p[2], p[3], w1);
#pragma unroll
    for (int n = 0; n < NO; ++n)
      *reinterpret_cast<tok_u32x2*>(P + n * C * K::P_PITCH + four_at<K::P_PITCH>(i, kt * 4 + g)) = tok_u32x2{w0[n], w1[n]};
  };

  // out of a chunk, and S after it
  tok_f32x4 O[CT][STATES ? 1 : RT];  // of token 16 i + r: columns wc + 16 c + 4 g + e
  auto chunk = [&](const unsigned char* buf, const unsigned char* P) __attribute__((always_inline)) {
    const int r = tid & 15, g = tid >> 4 & 3, q_at = piece_at<K::Q_PITCH>(r, g), p_at = piece_at<K::P_PITCH>(r, g);
    const float *w_q = reinterpret_cast<const float*>(buf + K::W_AT) + 2 * C, *w_k = w_q + C;
    if constexpr (!STATES) {
      // exp(G_i) q_i S
#pragma unroll
      for (int c = 0; c < CT; ++c)
#pragma unroll
        for (int i = 0; i < RT; ++i) O[c][i] = tok_f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        __builtin_amdgcn_sched_barrier(0);
        tok_bf16x8 fs[CT][NO], fq[RT][NI];
#pragma unroll
        for (int i = 0; i < RT; ++i)
#pragma unroll
          for (int n = 0; n < NI; ++n)
            fq[i][n] = *reinterpret_cast<const tok_bf16x8*>(buf + (n * C + i * 16) * K::Q_PITCH + (q_at ^ s * 64));
#pragma unroll
        for (int c = 0; c < CT; ++c) {
          float f[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) f[e] = S[c][s][e >> 2][e & 3];
          split8<NO>(f, fs[c]);
        }
#pragma unroll
        for (int x = 0; x < NO; ++x)
#pragma unroll
          for (int y = 0; y < NI; ++y)
#pragma unroll
            for (int c = 0; c < CT; ++c)
#pragma unroll
              for (int i = 0; i < RT; ++i)
                if (x + y <= LAST) O[c][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fs[c][x], fq[i][y], O[c][i], 0, 0, 0);
      }
#pragma unroll
      for (int i = 0; i < RT; ++i) {
        const float w = w_q[i * 16 + r];
#pragma unroll
        for (int c = 0; c < CT; ++c) O[c][i] *= w;
      }
    }
    {
      const float all = w_k[C];
      factor *= all;
#pragma unroll
      for (int s = 0; s < KS; ++s)
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int c = 0; c < CT; ++c) S[c][s][u] *= all;
    }
    {
      __builtin_amdgcn_sched_barrier(0);
      const int row = 4 * g;  // the first of this lane's tokens; four more 16 further on
      tok_bf16x8 fv[CT][NI], fw[CT][kStateTerms], fp[STATES ? 1 : RT][NO];
      float weight[8];
      *reinterpret_cast<tok_f32x4*>(weight) = *reinterpret_cast<const tok_f32x4*>(w_k + row);
      *reinterpret_cast<tok_f32x4*>(weight + 4) = *reinterpret_cast<const tok_f32x4*>(w_k + row + 16);
#pragma unroll
      for (int c = 0; c < CT; ++c) {
        float f[8], x[8];
#pragma unroll
        for (int n = NI - 1; n >= 0; --n) {
          fv[c][n] = column8(buf + K::V_AT + (n * C + row + (r >> 2)) * K::V_PITCH + (g & 2) * 8 + (wc + 16 * c + 4 * (r & 3)) * 2, K::V_PITCH);
          const tok_u32x4 u = __builtin_bit_cast(tok_u32x4, fv[c][n]);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float lo = __uint_as_float(u[e] << 16), hi = __uint_as_float(u[e] & 0xffff0000u);
            f[2 * e] = n == NI - 1 ? lo : f[2 * e] + lo;
            f[2 * e + 1] = n == NI - 1 ? hi : f[2 * e + 1] + hi;
          }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = f[e] * weight[e];
        split8<kStateTerms>(x, fw[c]);
        if constexpr (!STATES) {
          // a value that is not finite must not meet the zeros of the tokens
          // before it: it is left out, and makes NaN of those from its own on.
          // The last term of such a value is NaN; of others it is below 2, but
          // for values beyond 2^17, which are looked at as well.
          const tok_u32x4 last = __builtin_bit_cast(tok_u32x4, fw[c][kStateTerms - 1]);
          const uint32_t any = last[0] | last[1] | last[2] | last[3];
          if (__builtin_expect(__builtin_amdgcn_ballot_w64((any & 0x40004000u) != 0) != 0, 0)) {
            int bad = C;
            tok_u32x4 m;
#pragma unroll
            for (int e = 7; e >= 0; --e) {
              const bool ok = fabsf(f[e]) < __builtin_inff();
              if (!ok) bad = row + (e < 4 ? e : 12 + e);
              const uint32_t half = ok ? 0xffffu : 0u;
              m[e >> 1] = e & 1 ? half << 16 : m[e >> 1] | half;
            }
#pragma unroll
            for (int n = 0; n < NI; ++n) fv[c][n] = __builtin_bit_cast(tok_bf16x8, __builtin_bit_cast(tok_u32x4, fv[c][n]) & m);
#pragma unroll
            for (int o = 16; o < 64; o <<= 1) {
              const int other = __shfl_xor(bad, o);
              bad = other < bad ? other : bad;
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int from_here = __shfl(bad, 4 * g + e);  // of column wc + 16 c + 4 g + e
#pragma unroll
              for (int i = 0; i < RT; ++i)
                if (i * 16 + r >= from_here) O[c][i][e] = __builtin_nanf("");
            }
          }
        }
      }
      if constexpr (!STATES) {
#pragma unroll
        for (int i = 0; i < RT; ++i)
#pragma unroll
          for (int n = 0; n < NO; ++n)
            fp[i][n] = *reinterpret_cast<const tok_bf16x8*>(P + (n * C + i * 16) * K::P_PITCH + p_at);
      }
      if constexpr (!STATES) {
#pragma unroll
        for (int x = 0; x < NI; ++x)
#pragma unroll
          for (int y = 0; y < NO; ++y)
#pragma unroll
            for (int c = 0; c < CT; ++c)
#pragma unroll
              for (int i = 0; i < RT; ++i)
                if (x + y <= LAST) O[c][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fv[c][x], fp[i][y], O[c][i], 0, 0, 0);
      }
#pragma unroll
      for (int s = 0; s < KS; s += 2) {
        __builtin_amdgcn_sched_barrier(0);
        tok_bf16x8 fk[4][NI];
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
          for (int n = 0; n < NI; ++n)
            fk[u][n] = column8(buf + K::K_AT + (n * C + row + (r >> 2)) * K::K_PITCH + (g & 2) * 8 + (32 * s + 16 * u + 4 * (r & 3)) * 2, K::K_PITCH);
#pragma unroll
        for (int x = 0; x < NI; ++x)
#pragma unroll
          for (int y = 0; y < kStateTerms; ++y)
#pragma unroll
            for (int c = 0; c < CT; ++c)
#pragma unroll
              for (int u = 0; u < 4; ++u)
                if (x + y < kStateTerms)
                  S[c][s + u / 2][u & 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fk[u][x], fw[c][y], S[c][s + u / 2][u & 1], 0, 0, 0);
      }
    }
  };
  auto store_out = [&](int64_t t) __attribute__((always_inline)) {
    if constexpr (!STATES) {
      store* const to = static_cast<store*>(a.out) + (t * a.heads + h) * a.dim_v + c0 + lane_out;
      const int64_t tile = static_cast<int64_t>(16) * a.heads * a.dim_v;
      const int rows = end - t < C ? static_cast<int>(end - t) : C;
#pragma unroll
      for (int c = 0; c < CT; ++c) {
        if (wc + 16 * c >= cols) return;
#pragma unroll
        for (int i = 0; i < RT; ++i) {
          store o[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) o[e] = E::narrow(O[c][i][e]);
          if (rows == C || i * 16 + (lane & 15) < rows) __builtin_memcpy(to + i * tile + 16 * c, o, sizeof(o));
        }
      }
    }
  };

  if constexpr (!STATES) {
    // P above the diagonal, within the 32 keys of a step: zeros that stay
    for (int i = tid; i < K::BUFS * NO * 16 * 4; i += THREADS) {
      const int four = i & 3, row = i / 4 % 16, n = i / 64;  // n: terms of all buffers
      *reinterpret_cast<uint64_t*>(lds + K::P_AT + n * C * K::P_PITCH + four_at<K::P_PITCH>(row, 4 + four)) = 0;
    }
  }
  ask(t0);
  place(lds, t0);
  if (t0 + C < end) ask(t0 + C);
  meet();
  if constexpr (K::BUFS == 2) {
    weigh(lds, lds + K::P_AT);
    if (t0 + C < end) place(lds + K::BUFFER, t0 + C);
    if (t0 + 2 * C < end) ask(t0 + 2 * C);
    meet();
    int cur = 0;
    for (int64_t t = t0; t < end; t += C, cur ^= 1) {
      tid = unknown(tid);
      unsigned char *const buf = lds + cur * K::BUFFER, *const next = lds + (cur ^ 1) * K::BUFFER;
      unsigned char *const P = lds + K::P_AT + cur * K::P_BYTES, *const Pn = lds + K::P_AT + (cur ^ 1) * K::P_BYTES;
      if (t + C < end) weigh(next, Pn);
      chunk(buf, P);
      store_out(t);
      meet();
      if (t + 2 * C < end) place(buf, t + 2 * C);
      if (t + 3 * C < end) ask(t + 3 * C);
      meet();
    }
  } else {
    for (int64_t t = t0; t < end; t += C) {
      tid = unknown(tid);
      if constexpr (!STATES) {
        weigh(lds, lds + K::P_AT);
        meet();
      }
      chunk(lds, lds + K::P_AT);
      store_out(t);
      meet();
      if (t + C < end) place(lds, t + C);
      if (t + 2 * C < end) ask(t + 2 * C);
      meet();
    }
  }

  float* to = nullptr;
  if (STATES)
    to = a.part + ((b * a.parts + part + 1) * a.heads + h) * head_size;
  else if (part == live - 1 && seq.slot >= 0)
    to = a.state + (seq.slot * a.heads + h) * head_size;
  if (!to) return;
#pragma unroll
  for (int s = 0; s < KS; ++s)
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int row = 32 * s + 16 * t + 4 * g + e;
#pragma unroll
        for (int c = 0; c < CT; ++c)
          if (row < a.dim_k && col + 16 * c < a.dim_v) to[static_cast<int64_t>(row) * a.dim_v + col + 16 * c] = S[c][s][t][e];
      }
  if (STATES && slice == 0 && tid == 0) a.factor[(b * a.parts + part + 1) * a.heads + h] = factor;
}

// The state that each part of a sequence begins with: four elements a thread,
// in order over the parts.  The first part's is that of the slot, copied, since
// the last part's workgroup may write the slot before the first one's reads it.
__global__ __launch_bounds__(256) void join_parts(Args a) {
  const int64_t head_size = static_cast<int64_t>(a.dim_k) * a.dim_v;
  const int64_t per = (head_size / 4 + 255) / 256, id = a.first + blockIdx.x;
  const int64_t at = (id % per * 256 + threadIdx.x) * 4;
  const int h = static_cast<int>(id / per % a.heads);
  const int64_t b = id / per / a.heads;
  const Seq seq = sequence(a, b);
  if (seq.n == 0 || at >= head_size) return;
  const int live = live_parts(a, seq.n);
  tok_f32x4 run = {0.f, 0.f, 0.f, 0.f};
  if (!seq.fresh) __builtin_memcpy(&run, a.state + (seq.slot * a.heads + h) * head_size + at, 16);
  for (int p = 0; p < live; ++p) {
    float* s = a.part + ((b * a.parts + p) * a.heads + h) * head_size + at;
    if (p > 0) {
      tok_f32x4 own;
      __builtin_memcpy(&own, s, 16);
      run = own + run * a.factor[(b * a.parts + p) * a.heads + h];
    }
    __builtin_memcpy(s, &run, 16);
  }
}

// The recurrence, W columns of a head's S a workgroup: a thread holds R rows of
// four columns.
template <class E, int W, int R>
__global__ __launch_bounds__(256) void tokens(Args a) {
  typedef typename E::store store;
  constexpr int LC = W / 4, RG = 256 / LC;  // threads over columns, over rows
  __shared__ tok_f32x4 sums[2][4][LC];
  const int tid = threadIdx.x, lc = tid % LC, rg = tid / LC, wave = tid >> 6;
  const int64_t id = a.first + blockIdx.x;
  const int64_t unit = id / (8 * a.slices) * 8 + id % 8;
  if (unit >= a.groups) return;
  const int col = static_cast<int>(id / 8 % a.slices) * W + lc * 4;
  const int h = static_cast<int>(unit % a.heads);
  const int64_t b = unit / a.heads;
  const Seq seq = sequence(a, b);
  if (seq.n == 0) return;
  const int hk = h / (a.heads / a.qk_heads);
  const bool in = col < a.dim_v;
  const int64_t head_size = static_cast<int64_t>(a.dim_k) * a.dim_v;
  float* st = a.state + (seq.slot * a.heads + h) * head_size + col;
  tok_f32x4 S[R];
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int row = rg + RG * i;
    S[i] = tok_f32x4{0.f, 0.f, 0.f, 0.f};
    if (!seq.fresh && in && row < a.dim_k) __builtin_memcpy(&S[i], st + static_cast<int64_t>(row) * a.dim_v, 16);
  }
  for (int64_t n = 0; n < seq.n; ++n) {
    const int64_t t = seq.first + n;
    const store* q = static_cast<const store*>(a.q) + t * a.ld_q + static_cast<int64_t>(hk) * a.dim_k;
    const store* k = static_cast<const store*>(a.k) + t * a.ld_k + static_cast<int64_t>(hk) * a.dim_k;
    const store* v = static_cast<const store*>(a.v) + t * a.ld_v + static_cast<int64_t>(h) * a.dim_v + col;
    const float keep = exp2_of(a.decay[t * a.ld_decay + h] * static_cast<float>(kLog2e));
    float fq[R], fk[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int row = rg + RG * i < a.dim_k ? rg + RG * i : a.dim_k - 1;
      fq[i] = E::widen(q[row]);
      fk[i] = E::widen(k[row]);
    }
    store sv[4];
    if (in) {
      __builtin_memcpy(sv, v, sizeof(sv));
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) sv[e] = store(0);
    }
    const tok_f32x4 fv = {E::widen(sv[0]), E::widen(sv[1]), E::widen(sv[2]), E::widen(sv[3])};
    tok_f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < R; ++i) {
      S[i] = S[i] * keep + fv * fk[i];
      if (rg + RG * i < a.dim_k) o += S[i] * fq[i];
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int x = LC; x < 64; x <<= 1) o[e] += __shfl_xor(o[e], x);
    if ((tid & 63) < LC) sums[n & 1][wave][lc] = o;
    meet();
    if (tid < LC && in) {
      o = (sums[n & 1][0][lc] + sums[n & 1][1][lc]) + (sums[n & 1][2][lc] + sums[n & 1][3][lc]);
      store out[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) out[e] = E::narrow(o[e] * a.scale);
      __builtin_memcpy(static_cast<store*>(a.out) + (t * a.heads + h) * a.dim_v + col, out, sizeof(out));
    }
  }
  if (seq.slot < 0 || !in) return;
#pragma unroll
  for (int i = 0; i < R; ++i)
    if (rg + RG * i < a.dim_k) __builtin_memcpy(st + static_cast<int64_t>(rg + RG * i) * a.dim_v, &S[i], 16);
}

int64_t up(int64_t a, int64_t b) { return (a + b - 1) / b; }

// rows of a thread where rg threads share dk of them
constexpr int rows_each(int dk, int rg) { return dk > rg ? dk / rg : 1; }

// New tokens of a sequence that take the recurrence.  A token takes about 1.1 us
// there, a chunk 10: 16 sequences x 16 heads of 128 (bf16) 10.3 us for 4 tokens, 12.5
// for 6, in chunks 11.2; 64 x 32 heads 51 for 4 and 60 for 6, in chunks 55; of 256
// rows and columns, or in f32, the two meet at 8 to 12 tokens.
constexpr int64_t kFew = 5;

// New tokens that a sequence may have.
int64_t most_new(const c3c_kv_batch& b) { return b.max_new < b.T ? b.max_new : b.T; }

// The chunk kernel's tile: rows of S, columns of a workgroup.
struct Tile {
  int dk, dvs;
};
Tile tile_of(int64_t dim_k, int64_t dim_v) {
  return {dim_k <= 64 ? 64 : dim_k <= 128 ? 128 : 256, dim_v <= 64 ? 64 : 128};
}

template <class E, int DK, int DVS, int CT>
hipError_t run_chunks(Args a, hipStream_t s) {
  const int64_t head_size = static_cast<int64_t>(a.dim_k) * a.dim_v;
  auto go = [&](void (*k)(Args), int64_t units, int threads) {
    a.groups = units;
    return in_launches(up(units, 8) * 8 * a.slices, threads, [&](int64_t first, unsigned count) {
      a.first = first;
      hipLaunchKernelGGL(k, dim3(count), dim3(threads), 0, s, a);
    });
  };
  if (a.parts > 1) {
    hipError_t e = go(chunks<E, DK, DVS, 1, true>, a.B * a.heads * (a.parts - 1), DVS * 4);
    if (e != hipSuccess) return e;
    e = in_launches(a.B * a.heads * up(head_size / 4, 256), 256, [&](int64_t first, unsigned count) {
      a.first = first;
      hipLaunchKernelGGL(join_parts, dim3(count), dim3(256), 0, s, a);
    });
    if (e != hipSuccess) return e;
  }
  return go(chunks<E, DK, DVS, CT, false>, a.B * a.heads * a.parts, DVS * 4 / CT);
}

template <class E, int W>
hipError_t run_tokens(Args a, hipStream_t s) {
  constexpr int RG = 256 / (W / 4);
  a.slices = static_cast<int>(up(a.dim_v, W));
  a.groups = a.B * a.heads;
  auto k = a.dim_k <= 64 ? tokens<E, W, rows_each(64, RG)> : a.dim_k <= 128 ? tokens<E, W, rows_each(128, RG)> : tokens<E, W, rows_each(256, RG)>;
  return in_launches(up(a.groups, 8) * 8 * a.slices, 256, [&](int64_t first, unsigned count) {
    a.first = first;
    hipLaunchKernelGGL(k, dim3(count), dim3(256), 0, s, a);
  });
}

template <class E>
hipError_t run(Args a, int64_t most, hipStream_t s) {
  if (most <= kFew) {
    // narrow slices where there are few heads: as many workgroups as compute units
    return a.B * a.heads < 256 ? run_tokens<E, 16>(a, s) : run_tokens<E, 32>(a, s);
  }
  const Tile t = tile_of(a.dim_k, a.dim_v);
  a.slices = static_cast<int>(up(a.dim_v, t.dvs));
  // two column tiles a wave where the registers hold them
  constexpr int CT = Terms<E>::IN < 3 ? 2 : 1;
  if (t.dvs == 64) return t.dk == 64 ? run_chunks<E, 64, 64, 1>(a, s) : t.dk == 128 ? run_chunks<E, 128, 64, 1>(a, s) : run_chunks<E, 256, 64, 1>(a, s);
  return t.dk == 64 ? run_chunks<E, 64, 128, CT>(a, s) : t.dk == 128 ? run_chunks<E, 128, 128, CT>(a, s) : run_chunks<E, 256, 128, 1>(a, s);
}

}  // namespace

RecurPlan plan_recur(const c3c_state_cache& st, const c3c_kv_batch& b) {
  RecurPlan p;
  const int64_t most = most_new(b);
  if (most <= kFew || b.B < 1) return p;
  const Tile t = tile_of(st.dim_k, st.dim_v);
  const int64_t chunks = up(most, C), units = b.B * st.heads * up(st.dim_v, t.dvs);
  // Two workgroups a compute unit, or four where they have 64 columns; parts of two
  // chunks at least (6 heads of 80 x 112 in f32, four sequences of up to 701 tokens:
  // 37 us, of four chunks 51).  By their registers and LDS four (bf16, 64 x 64) to
  // one (512 threads; f16 and f32 of 256 x 64) of the outputs' workgroups are on a
  // compute unit at once; the others run in further rounds.  Half as many parts: a
  // clip of 32 heads of 128 takes 575 us (468 so), those f32 sequences 38.5 (34.3),
  // a frame for each of two streams 42 (45); but few heads over long sequences are
  // faster, since the join takes their parts one by one: 4 heads of 16000 tokens
  // of 128 x 128 69 us (82 so) in bf16 and 91 (116) in f32, of 64 x 64 68 (105), of
  // 256 x 64 86 (132).
  const int64_t room = device_compute_units() * (t.dvs == 128 ? 2 : 4);
  int64_t parts = room / units;
  if (parts > chunks / 2) parts = chunks / 2;
  if (parts < 2) return p;
  const int64_t each = up(chunks, parts);
  p.part_tokens = each * C;
  p.parts = static_cast<int>(up(chunks, each));
  p.state_bytes = b.B * p.parts * st.heads * st.dim_k * st.dim_v * 4;
  p.bytes = p.state_bytes + b.B * p.parts * st.heads * 4;
  return p;
}

hipError_t launch_recur(const RecurArgs& r, int dtype, const RecurPlan& plan, hipStream_t s) {
  const c3c_state_cache& st = r.st;
  if (r.b.T == 0 || r.b.B == 0) return hipSuccess;
  const int64_t most = most_new(r.b);
  Args a{st.state, r.b.cu, r.b.len, r.slot, r.q, r.k, r.v, r.decay, r.out, r.part, nullptr, st.slots, r.b.B, r.b.T,
         r.ld_q, r.ld_k, r.ld_v, r.ld_decay, plan.part_tokens, 0, 0, static_cast<int>(st.heads),
         static_cast<int>(r.qk_heads), static_cast<int>(st.dim_k), static_cast<int>(st.dim_v), plan.parts, 1, r.scale};
  if (plan.parts > 1) a.factor = r.part + plan.state_bytes / 4;
  return dtype == C3C_DTYPE_BF16 ? run<ElemBf16>(a, most, s) : dtype == C3C_DTYPE_F16 ? run<ElemF16>(a, most, s) : run<ElemF32>(a, most, s);
}

}  // namespace c3c
