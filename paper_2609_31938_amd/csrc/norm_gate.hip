// Norms around a gated residual, and 8-bit rows with a scale each.
//
//   n(v)[c] = v[c] / sqrt(mean_c v[c]^2 + eps)
//   h'      = alpha h + gate * (post * n(y)),   u = pre * n(h')
//   8-bit rows: s = max|u| / 127, q = u / s to the nearest integer
//
// The two means make it three passes over a row (y's squares, h' and its
// squares, u; a fourth for the 8-bit row's maximum).  A row stays in
// registers between them, so y and h are read once and h' and u written
// once: 4 T C elements of traffic, which is what bounds large calls.  The
// squares of h' are summed from h' itself: expanding them into sums over y
// and h would need one pass less and cancel where h and the gated y do.
//
// A row belongs to one wave (at most 128 16-byte vectors: no barrier) or to
// one workgroup; rows beyond 4096 vectors are read again in every pass.
// 32760 x 5120 in bf16 with post, gate and pre: 356 us, 3.8 TB/s.  A row's loads
// follow one another: each stands behind the condition on the row's end, whose
// branch also widens it, and so is waited for before the next is issued.  The
// gains come from L2 for every row and are more bytes than the row; with
// constants in their place, and so without their waits, 263 us.  Slower: two rows a workgroup (363), gains kept over the
// rows of workgroups that stay (441 to 491, fewer rows in flight), a row a wave
// (796), two vectors a thread (358).
#include <math.h>

#include "token_dev.h"
#include "tokens_internal.h"

namespace c3c {
namespace {

// Reductions over the threads of a row: a wave, or (WAVE false) the workgroup
// of at most 16 waves, whose partial results meet in LDS.  Every call of one
// kernel takes its own `slot`, so that no call overwrites what a slower wave
// still reads.
template <bool WAVE>
struct Row {
  float* lds;  // [slots][16]
  __device__ float sum(float v, int slot) const {
    v = wave_sum(v);
    if (WAVE) return v;
    const int w = threadIdx.x >> 6, n = blockDim.x >> 6;
    if ((threadIdx.x & 63) == 0) lds[slot * 16 + w] = v;
    __syncthreads();
    float r = 0.f;
    for (int i = 0; i < n; ++i) r += lds[slot * 16 + i];
    return r;
  }
  __device__ float max(float v, int slot) const {
    v = wave_max(v);
    if (WAVE) return v;
    const int w = threadIdx.x >> 6, n = blockDim.x >> 6;
    if ((threadIdx.x & 63) == 0) lds[slot * 16 + w] = v;
    __syncthreads();
    float r = 0.f;
    for (int i = 0; i < n; ++i) r = fmaxf(r, lds[slot * 16 + i]);
    return r;
  }
};

// 16-byte vectors of fp32 per-channel gains
template <class E>
__device__ inline void load_gain(const float* p, int m, float (&f)[E::VEC]) {
  if (m >= E::VEC) {
    __builtin_memcpy(f, p, 4 * E::VEC);
  } else {
#pragma unroll
    for (int e = 0; e < E::VEC; ++e) f[e] = e < m ? p[e] : 0.f;
  }
}

struct NormArgs {
  const void *h, *y, *gate;
  const float *post, *pre;
  void *h_out, *u;
  int8_t* u_q;
  float* u_scale;
  int64_t T, C, rows;
  float alpha, eps;
  bool stream;    // outputs are more than the caches hold
  int64_t first;  // workgroup of this launch
};

// NV vectors of the row in each thread's registers.
template <class E, int NV, bool WAVE>
__global__ __launch_bounds__(WAVE ? 256 : 1024) void norm_gate_regs(NormArgs a) {
  constexpr int V = E::VEC;
  typedef typename E::store S;
  __shared__ float lds[3 * 16];
  const Row<WAVE> row{lds};
  const int per = WAVE ? 64 : blockDim.x;  // threads of a row
  const int64_t wg = a.first + blockIdx.x, t = WAVE ? wg * 4 + (threadIdx.x >> 6) : wg;
  const int lane = WAVE ? threadIdx.x & 63 : threadIdx.x;
  if (WAVE && t >= a.T) return;  // whole waves, and no barrier follows
  const int C = static_cast<int>(a.C);
  const S* hp = static_cast<const S*>(a.h) + t * a.C;
  const S* yp = a.y ? static_cast<const S*>(a.y) + t * a.C : nullptr;
  const S* gp = a.gate ? static_cast<const S*>(a.gate) + t / a.rows * a.C : nullptr;
  float h[NV][V], y[NV][V], g[NV][V], p[NV][V];
  // the row's loads, before the first sum
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (lane + i * per) * V, m = C - c;
    if (yp) load_vec<E>(yp + c, m, y[i]);
    load_vec<E>(hp + c, m, h[i]);
  }
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (lane + i * per) * V, m = C - c;
#pragma unroll
    for (int e = 0; e < V; ++e) g[i][e] = 1.f;
    if (gp) load_vec<E>(gp + c, m, g[i]);
    if (a.post) {
      load_gain<E>(a.post + c, m, p[i]);
#pragma unroll
      for (int e = 0; e < V; ++e) g[i][e] *= p[i][e];
    }
    if (a.pre) load_gain<E>(a.pre + c, m, p[i]);
  }
  if (yp) {
    float r = 1.f;
    if (a.post) {
      float ss = 0.f;
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < V; ++e) ss = __builtin_fmaf(y[i][e], y[i][e], ss);
      r = 1.f / sqrtf(row.sum(ss, 0) / static_cast<float>(C) + a.eps);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < V; ++e) h[i][e] = __builtin_fmaf(a.alpha, h[i][e], g[i][e] * (y[i][e] * r));
  } else {
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < V; ++e) h[i][e] *= a.alpha;
  }
  if (a.h_out) {
    S* o = static_cast<S*>(a.h_out) + t * a.C;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (lane + i * per) * V;
      if (c < C) store_vec<E>(o + c, C - c, h[i], a.stream);
    }
  }
  if (!a.pre) return;
  float ss = 0.f;
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int e = 0; e < V; ++e) ss = __builtin_fmaf(h[i][e], h[i][e], ss);
  const float r = 1.f / sqrtf(row.sum(ss, 1) / static_cast<float>(C) + a.eps);
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int e = 0; e < V; ++e) h[i][e] = h[i][e] * r * p[i][e];
  if (a.u) {
    S* o = static_cast<S*>(a.u) + t * a.C;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (lane + i * per) * V;
      if (c < C) store_vec<E>(o + c, C - c, h[i], a.stream);
    }
  }
  if (a.u_q) {
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < V; ++e)
        if ((lane + i * per) * V + e < C) top = fmaxf(top, magnitude(h[i][e]));
    const float s = row_scale(row.max(top, 2));
    int8_t* q = a.u_q + t * a.C;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (lane + i * per) * V;
      if (c < C) store_codes<V>(q + c, C - c, h[i], s);
    }
    if (lane == 0) a.u_scale[t] = s;
  }
}

// Rows of any length: every pass reads the row again.
template <class E>
__global__ __launch_bounds__(1024) void norm_gate_loop(NormArgs a) {
  typedef typename E::store S;
  __shared__ float lds[3 * 16];
  const Row<false> row{lds};
  const int64_t t = a.first + blockIdx.x;
  const S* hp = static_cast<const S*>(a.h) + t * a.C;
  const S* yp = a.y ? static_cast<const S*>(a.y) + t * a.C : nullptr;
  const S* gp = a.gate ? static_cast<const S*>(a.gate) + t / a.rows * a.C : nullptr;
  const float C = static_cast<float>(a.C);
  float r = 1.f;
  if (yp && a.post) {
    float ss = 0.f;
    for (int64_t c = threadIdx.x; c < a.C; c += blockDim.x) {
      const float v = E::widen(yp[c]);
      ss = __builtin_fmaf(v, v, ss);
    }
    r = 1.f / sqrtf(row.sum(ss, 0) / C + a.eps);
  }
  auto next = [&](int64_t c) {
    const float h = E::widen(hp[c]);
    if (!yp) return a.alpha * h;
    float g = gp ? E::widen(gp[c]) : 1.f;
    if (a.post) g *= a.post[c];
    return __builtin_fmaf(a.alpha, h, g * (E::widen(yp[c]) * r));
  };
  float r2 = 1.f, s = 1.f;
  if (a.pre) {
    float ss = 0.f;
    for (int64_t c = threadIdx.x; c < a.C; c += blockDim.x) {
      const float v = next(c);
      ss = __builtin_fmaf(v, v, ss);
    }
    r2 = 1.f / sqrtf(row.sum(ss, 1) / C + a.eps);
    if (a.u_q) {
      float top = 0.f;
      for (int64_t c = threadIdx.x; c < a.C; c += blockDim.x) top = fmaxf(top, magnitude(next(c) * r2 * a.pre[c]));
      s = row_scale(row.max(top, 2));
      if (threadIdx.x == 0) a.u_scale[t] = s;
    }
  }
  // last: h_out may be h, and every element is read by the thread that writes it
  for (int64_t c = threadIdx.x; c < a.C; c += blockDim.x) {
    const float v = next(c);
    if (a.h_out) static_cast<S*>(a.h_out)[t * a.C + c] = E::narrow(v);
    if (!a.pre) continue;
    const float u = v * r2 * a.pre[c];
    if (a.u) static_cast<S*>(a.u)[t * a.C + c] = E::narrow(u);
    if (a.u_q) a.u_q[t * a.C + c] = static_cast<int8_t>(code(u, s));
  }
}

struct QuantArgs {
  const void* x;
  int8_t* q;
  float* scale;
  int64_t T, C, ld_x, ld_q;  // q's rows are zero from C to ld_q
  int64_t first;             // workgroup of this launch
};

// EXACT: codes nearest to 127 x / max|x| itself.  Compiled in: asked for in the
// kernel, rows by the rounded scale take 5 to 8% longer (32760 x 5120 bf16: 169 us,
// so 159).
template <class E, int NV, bool WAVE, bool EXACT>
__global__ __launch_bounds__(WAVE ? 256 : 1024) void quantize_regs(QuantArgs a) {
  constexpr int V = E::VEC;
  __shared__ float lds[16];
  const Row<WAVE> row{lds};
  const int per = WAVE ? 64 : blockDim.x;
  const int64_t wg = a.first + blockIdx.x, t = WAVE ? wg * 4 + (threadIdx.x >> 6) : wg;
  const int lane = WAVE ? threadIdx.x & 63 : threadIdx.x;
  if (WAVE && t >= a.T) return;
  const int C = static_cast<int>(a.C), Q = static_cast<int>(a.ld_q);
  const typename E::store* x = static_cast<const typename E::store*>(a.x) + t * a.ld_x;
  float v[NV][V];
  float top = 0.f;
#pragma unroll
  for (int i = 0; i < NV; ++i) load_vec<E>(x + (lane + i * per) * V, C - (lane + i * per) * V, v[i]);
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int e = 0; e < V; ++e) top = fmaxf(top, magnitude(v[i][e]));
  top = row.max(top, 0);
  const float s = row_scale(top);
  int8_t* q = a.q + t * a.ld_q;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (lane + i * per) * V;
    if (c < Q) store_codes<V>(q + c, Q - c, v[i], s, EXACT ? top : 0.f);
  }
  if (lane == 0) a.scale[t] = s;
}

template <class E, bool EXACT>
__global__ __launch_bounds__(1024) void quantize_loop(QuantArgs a) {
  __shared__ float lds[16];
  const Row<false> row{lds};
  const int64_t t = a.first + blockIdx.x;
  const typename E::store* x = static_cast<const typename E::store*>(a.x) + t * a.ld_x;
  float top = 0.f;
  for (int64_t c = threadIdx.x; c < a.C; c += blockDim.x) top = fmaxf(top, magnitude(E::widen(x[c])));
  top = row.max(top, 0);
  const float s = row_scale(top);
  for (int64_t c = threadIdx.x; c < a.ld_q; c += blockDim.x) {
    const float v = c < a.C ? E::widen(x[c]) : 0.f;
    a.q[t * a.ld_q + c] = static_cast<int8_t>(EXACT && doubtful(v, s) ? true_code(v, s, top) : code(v, s));
  }
  if (threadIdx.x == 0) a.scale[t] = s;
}

// How a row of nv vectors is spread: a wave while it holds two vectors a lane
// at most, else a workgroup with as few vectors a thread as its 1024 threads
// allow.
struct Shape {
  bool wave;
  int nv;  // vectors a thread; 0: the loop
  unsigned threads;
  int64_t blocks;
};
Shape shape_of(int64_t T, int64_t vecs) {
  auto ceil = [](int64_t a, int64_t b) { return (a + b - 1) / b; };
  if (vecs <= 128) return {true, vecs <= 64 ? 1 : 2, 256, ceil(T, 4)};
  if (vecs > 4 * 1024) return {false, 0, 1024, T};
  const int nv = vecs <= 1024 ? 1 : vecs <= 2048 ? 2 : 4;
  return {false, nv, static_cast<unsigned>(ceil(ceil(vecs, nv), 64) * 64), T};
}

template <class E>
hipError_t norm_typed(NormArgs a, hipStream_t s) {
  a.stream = a.T * a.C * static_cast<int64_t>(sizeof(typename E::store)) > (32 << 20);
  const Shape p = shape_of(a.T, (a.C + E::VEC - 1) / E::VEC);
  auto k = p.nv == 0 ? norm_gate_loop<E>
           : p.wave  ? (p.nv == 1 ? norm_gate_regs<E, 1, true> : norm_gate_regs<E, 2, true>)
           : p.nv == 1 ? norm_gate_regs<E, 1, false>
           : p.nv == 2 ? norm_gate_regs<E, 2, false>
                       : norm_gate_regs<E, 4, false>;
  return in_launches(p.blocks, p.threads, [&](int64_t first, unsigned count) {
    a.first = first;
    hipLaunchKernelGGL(k, dim3(count), dim3(p.threads), 0, s, a);
  });
}

template <class E, bool EXACT>
hipError_t quantize_typed(QuantArgs a, hipStream_t s) {
  const Shape p = shape_of(a.T, (a.ld_q + E::VEC - 1) / E::VEC);
  auto k = p.nv == 0 ? quantize_loop<E, EXACT>
           : p.wave  ? (p.nv == 1 ? quantize_regs<E, 1, true, EXACT> : quantize_regs<E, 2, true, EXACT>)
           : p.nv == 1 ? quantize_regs<E, 1, false, EXACT>
           : p.nv == 2 ? quantize_regs<E, 2, false, EXACT>
                       : quantize_regs<E, 4, false, EXACT>;
  return in_launches(p.blocks, p.threads, [&](int64_t first, unsigned count) {
    a.first = first;
    hipLaunchKernelGGL(k, dim3(count), dim3(p.threads), 0, s, a);
  });
}

}  // namespace

hipError_t launch_norm_gate(const c3c_norm_desc& d, const void* h, const void* y, const void* gate,
                            const float* post, const float* pre, void* h_out, void* u, int8_t* u_q,
                            float* u_scale, hipStream_t s) {
  if (d.T == 0) return hipSuccess;
  const NormArgs a{h, y, gate, post, pre, h_out, u, u_q, u_scale, d.T, d.C, gate ? d.rows_per_gate : 1, d.alpha, d.eps,
                   false, 0};
  return d.dtype == C3C_DTYPE_BF16  ? norm_typed<ElemBf16>(a, s)
         : d.dtype == C3C_DTYPE_F16 ? norm_typed<ElemF16>(a, s)
                                    : norm_typed<ElemF32>(a, s);
}

hipError_t launch_quantize_rows(int64_t T, int64_t C, int64_t ld_x, int dtype, const void* x,
                                int8_t* q, int64_t ld_q, float* scale, bool exact, hipStream_t s) {
  if (T == 0) return hipSuccess;
  const QuantArgs a{x, q, scale, T, C, ld_x, ld_q, 0};
  if (exact)
    return dtype == C3C_DTYPE_BF16  ? quantize_typed<ElemBf16, true>(a, s)
           : dtype == C3C_DTYPE_F16 ? quantize_typed<ElemF16, true>(a, s)
                                    : quantize_typed<ElemF32, true>(a, s);
  return dtype == C3C_DTYPE_BF16  ? quantize_typed<ElemBf16, false>(a, s)
         : dtype == C3C_DTYPE_F16 ? quantize_typed<ElemF16, false>(a, s)
                                  : quantize_typed<ElemF32, false>(a, s);
}

}  // namespace c3c
