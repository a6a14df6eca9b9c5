// Internal launch interface of the stand-alone operators (operators.hip) and
// their entry points (operators.cpp).  Not part of the public C ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "kernels.h"

namespace ee {

// Records `msg` as the last error of calls without a context; returns `code`.
int op_fail(int code, const char* msg);

enum Act { ACT_NONE = 0, ACT_SILU, ACT_GELU, ACT_GELU_TANH, ACT_RELU, ACT_N };

// y = act(x w^T + bias) + res.  Strides in elements.
struct LinearArgs {
  const void* x;        // [T][ldx] dt
  const void* w;        // [N][ldw] dt
  const float* bias;    // [N] or null
  const void* res;      // [T][ldr] odt or null
  void* y;              // [T][ldy] odt
  int64_t ldx, ldw, ldr, ldy;
  int T, K, N;
  int dt, odt, act;
};
hipError_t run_linear(const LinearArgs& a, hipStream_t st);

enum Score { SCORE_SOFTMAX = 0, SCORE_SIGMOID, SCORE_N };
constexpr int ROUTE_MAX_E = 1024, ROUTE_MAX_K = 32;

struct RouteArgs {
  const void* logits;   // [T][ld] dt
  const float* bias;    // [E] or null
  int* ids;             // [T][k]
  float* weights;       // [T][k]
  int64_t ld;
  int T, E, k, dt, score, renorm;
  int groups, top_groups, group_top;
  float scale;
};
hipError_t run_route(const RouteArgs& a, hipStream_t st);

struct FfnArgs {
  const void* x;        // [T][ldx] dt
  const void* wgu;      // [E][2 F][d] dt: gate rows, then up rows
  const void* wd;       // [E][d][F] dt
  const int* ids;       // [T][k], entries outside [0, E) are skipped
  const float* weights; // [T][k]
  const void* res;      // [T][ldr] odt or null
  void* out;            // [T][ldo] odt
  int64_t ldx, ldr, ldo;
  int T, E, k, d, F, dt, odt;
  unsigned char* ws;    // ffn_workspace(...) bytes
};
size_t ffn_workspace(int T, int E, int k, int d, int F, int dt);
hipError_t run_ffn(const FfnArgs& a, hipStream_t st);

}  // namespace ee
