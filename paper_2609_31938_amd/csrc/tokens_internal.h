// Internal interface between the host layer of the token operators
// (tokens_host.cpp) and their kernels.  Arguments arrive validated.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "c3c_tokens.h"

namespace c3c {

int64_t device_compute_units();  // of the current device (256 when none is visible)

// A dimension of a launch has fewer than 2^32 threads: more workgroups than
// that go in several launches, launch(first, count) each.
template <class F>
hipError_t in_launches(int64_t workgroups, int64_t threads, F launch) {
  const int64_t most = (int64_t(1) << 31) / threads;
  hipError_t e = hipSuccess;
  for (int64_t first = 0; first < workgroups && e == hipSuccess; first += most) {
    launch(first, static_cast<unsigned>(workgroups - first < most ? workgroups - first : most));
    e = hipGetLastError();
  }
  return e;
}

// quantize_rows and norm_gate (norm_gate.hip)
hipError_t launch_quantize_rows(int64_t T, int64_t C, int64_t ld_x, int dtype, const void* x,
                                int8_t* q, int64_t ld_q, float* scale, hipStream_t s);
hipError_t launch_norm_gate(const c3c_norm_desc& d, const void* h, const void* y, const void* gate,
                            const float* post, const float* pre, void* h_out, void* u, int8_t* u_q,
                            float* u_scale, hipStream_t s);

// linear_i8 (linear_i8.hip): int8 rows, ldx bytes between them.  part: int32
// partial sums of a split call (plan_linear_i8 says how many), or NULL.
struct LinearPlan {
  int splits = 1;          // along K
  int64_t part_bytes = 0;  // of workspace for the partial sums
};
LinearPlan plan_linear_i8(int64_t M, int64_t N, int64_t K);
hipError_t launch_linear_i8(int64_t M, int64_t N, int64_t K, const int8_t* x, int64_t ldx,
                            const float* x_scale, const int8_t* w, const float* w_scale,
                            const float* bias, void* y, int y_dtype, const LinearPlan& plan,
                            int32_t* part, hipStream_t s);

// whether a call copies rows of K bytes, ld apart, to rows of whole 16 bytes
bool linear_pads(int64_t M, int64_t K, int64_t ld);
hipError_t launch_pad_rows(const int8_t* src, int64_t rows, int64_t n, int64_t ld, int8_t* dst, int64_t ldd, hipStream_t s);
// the same on float rows that the kernel quantises itself, for the few and
// short ones that linear_quantises says
bool linear_quantises(int64_t M, int64_t K);
hipError_t launch_linear_float(int64_t M, int64_t N, int64_t K, const void* x, int64_t ldx, int x_dtype,
                               const int8_t* w, const float* w_scale, const float* bias, void* y, int y_dtype,
                               hipStream_t s);

// kv_append (kv_append.hip)
struct AppendArgs {
  c3c_kv_cache c;
  c3c_kv_batch b;
  c3c_rope r;  // cos NULL: no rotation
  const void *q, *k, *v;
  void* q_out;
  int64_t q_heads, ld_q, ld_k, ld_v;
};
hipError_t launch_kv_append(const AppendArgs& a, int dtype, hipStream_t s);

// paged_attention (paged_attention.hip)
struct AttendArgs {
  c3c_kv_cache c;
  c3c_kv_batch b;
  const void* q;
  void* out;
  float* lse;
  float* part;  // workspace of a split call, or NULL
  int64_t q_heads, ld_q, window;
  float scale;
  int causal;
};
struct AttendPlan {
  int splits = 1;
  int64_t part_bytes = 0;
};
AttendPlan plan_attend(const c3c_kv_cache& c, const c3c_kv_batch& b, int dtype, int64_t q_heads,
                       int causal, int64_t window);
hipError_t launch_attend(const AttendArgs& a, int dtype, const AttendPlan& plan, hipStream_t s);

}  // namespace c3c
