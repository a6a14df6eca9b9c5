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

// e4m3 codes of x and their scales, one per block of block_rows rows and BLOCK columns.
constexpr int BLOCK = 128;
struct Fp8QuantArgs {
  const void* x;        // [T][ldx] dt
  uint8_t* codes;       // [T][ldc]
  float* scales;        // [ceil(T / block_rows)][ceil(K / BLOCK)]
  int64_t ldx, ldc;
  int T, K, dt, block_rows;
};
hipError_t run_fp8_quant(const Fp8QuantArgs& a, hipStream_t st);

// A linear of e4m3 codes (l.x, l.w: bytes) with their scales.
struct Fp8LinearArgs {
  LinearArgs l;
  const float* xs;      // [T][ceil(K / BLOCK)]
  const float* ws;      // [ceil(N / BLOCK)][ceil(K / BLOCK)]
  int n0;               // feature 0's number in the whole product, a multiple of 256
};
hipError_t run_fp8_linear(const Fp8LinearArgs& a, hipStream_t st);

// Position p of sequence s: slot p % page of page tables[s][p / page], where that is in
// [0, n_pages).  Strides in elements, of pages, slots and heads.
struct PagedCache {
  const void *k, *v;
  int64_t kp, ks, kh, vp, vs, vh;
  const int* tables;    // [sequences][ldt]
  int64_t ldt;
  int n_pages, max_pages, page;
};
constexpr int MAX_HEAD_DIM = 256;

struct AppendArgs {
  const void *q, *k, *v;    // [R][ld] dt: heads of hd; q may be null
  void* q_out;
  PagedCache c;
  const int *seqs, *positions;   // [R]; seqs null: row / per_seq
  const double* inv_freq;        // [rot / 2]
  int64_t ldq, ldk, ldv, ldqo;
  int R, B, per_seq, H, Hkv, hd, rot, interleaved, dt;
};
hipError_t run_append(const AppendArgs& a, hipStream_t st);

constexpr int ATTEND_CHUNK = 256;   // positions whose state is held
struct AttendArgs {
  const void* q;        // [B T][ldq] dt
  void* out;            // [B T][ldo] odt
  float* lse;           // [B T][H] or null
  PagedCache c;
  const int* lens;      // [B] positions, the T rows' own among them
  unsigned char* ws;    // attend_workspace(...) bytes
  int64_t ldq, ldo;
  int B, T, H, Hkv, G, hd, dt, odt, window;
  float scale_log2;     // of scores, times log2 e
  // (filled in by run_attend)
  int behind;           // rows of the sequences that follow the T here
  int all;              // sequences of the whole call
  float2* ml;           // [B][ring][Hkv][T G] largest score and sum of the chunks' states
  float* o;             // [..][hd] their weighted values
  int ring, splits;     // chunks held; workgroups that share a sequence's
  int apart;            // up to so many chunks of a sequence, their runs' states are held instead
  int cgroups, ctw;     // workgroups that share a head's column tiles, tiles of each
  uint64_t page_mul;    // 2^38 / (page / 16), rounded up: divides positions by page
};
size_t attend_workspace(int B, int T, int H, int hd, int64_t positions, int window);
hipError_t run_attend(const AttendArgs& a, hipStream_t st);

}  // namespace ee
