// Entry points of the stand-alone operators of include/ee.h: argument checks
// and launches.  Nothing here allocates, synchronizes or keeps state.

#include "operators.h"

#include <math.h>

#include "../../include/ee.h"

namespace {

using ee::op_fail;

// Grids and index arithmetic of the kernels stay inside these.
constexpr int64_t MAX_ROWS = 1 << 22, MAX_COLS = 1 << 20, MAX_PAIRS = 1 << 24;
constexpr int64_t MAX_BLOCKS = 0x7fffffff;

int bad(const char* msg) { return op_fail(EE_EINVAL, msg); }
bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
bool dtype_ok(int t) { return t == EE_F32 || t == EE_BF16; }
int esz(int t) { return t == EE_BF16 ? 2 : 4; }
int ks(int t) { return t == EE_BF16 ? 32 : 16; }
int dt_of(int t) { return t == EE_BF16 ? ee::DT_BF16 : ee::DT_F32; }

// Rows of `cols` elements, `ld` elements apart, whose 16-byte pieces the
// kernels load whole, at 32-bit offsets within a tile's 256 rows.
constexpr int64_t MAX_LD = 1 << 21;
bool rows_ok(const void* p, int64_t ld, int cols, int type) {
  return aligned(p, 16) && ld >= cols && ld <= MAX_LD && ld * esz(type) % 16 == 0;
}
// Rows that are read and written element by element (or more where aligned).
bool out_ok(const void* p, int64_t ld, int cols, int type) {
  return aligned(p, esz(type)) && ld >= cols && ld < (int64_t(1) << 40);
}

int launched(hipError_t e) { return e == hipSuccess ? EE_OK : op_fail(EE_EHIP, hipGetErrorString(e)); }

}  // namespace

extern "C" {

int32_t ee_linear(const ee_linear_args* p, void* stream) {
  if (!p) return bad("arguments are NULL");
  const ee_linear_args& q = *p;
  if (!dtype_ok(q.dtype) || !dtype_ok(q.out_dtype) || (q.dtype == EE_F32 && q.out_dtype != EE_F32))
    return bad("dtype must be EE_F32 or EE_BF16, out_dtype the same or EE_F32");
  if (q.rows < 0 || q.rows > MAX_ROWS || q.in < 1 || q.in > MAX_COLS || q.out < 1 || q.out > MAX_COLS)
    return bad("rows must be in [0, 2^22], in and out in [1, 2^20]");
  if (q.in % ks(q.dtype)) return bad("in must be a multiple of 32 (bf16) / 16 (f32)");
  if (q.act < 0 || q.act >= ee::ACT_N) return bad("unknown activation");
  if (q.rows == 0) return EE_OK;
  if (!q.x || !q.w || !q.y) return bad("x, w and y must be non-NULL");
  if (!rows_ok(q.x, q.ldx, q.in, q.dtype) || !rows_ok(q.w, q.ldw, q.in, q.dtype))
    return bad("x and w must be 16-byte aligned with row strides of at least `in`, at most 2^21, and a multiple of 16 bytes");
  if (!out_ok(q.y, q.ldy, q.out, q.out_dtype)) return bad("y must be aligned to its type with a row stride of at least `out`");
  if (q.residual && !out_ok(q.residual, q.ldr, q.out, q.out_dtype))
    return bad("residual must be aligned to its type with a row stride of at least `out`");
  if (q.bias && !aligned(q.bias, 4)) return bad("bias must be aligned to its type");
  if ((int64_t)((q.rows + 15) / 16) * ((q.out + 15) / 16) > MAX_BLOCKS) return bad("too many output tiles");
  if (q.y == q.x || q.y == q.w || q.y == q.bias || (q.y == q.residual && q.ldr != q.ldy))
    return bad("y must not be an input, except the residual with its stride");
  ee::LinearArgs a{};
  a.x = q.x; a.w = q.w; a.bias = q.bias; a.res = q.residual; a.y = q.y;
  a.ldx = q.ldx; a.ldw = q.ldw; a.ldr = q.ldr; a.ldy = q.ldy;
  a.T = q.rows; a.K = q.in; a.N = q.out;
  a.dt = dt_of(q.dtype); a.odt = dt_of(q.out_dtype); a.act = q.act;
  return launched(ee::run_linear(a, reinterpret_cast<hipStream_t>(stream)));
}

int32_t ee_moe_route(const ee_moe_route_args* p, void* stream) {
  if (!p) return bad("arguments are NULL");
  const ee_moe_route_args& q = *p;
  if (!dtype_ok(q.dtype)) return bad("dtype must be EE_F32 or EE_BF16");
  if (q.rows < 0 || q.rows > MAX_ROWS) return bad("rows must be in [0, 2^22]");
  if (q.n_experts < 1 || q.n_experts > ee::ROUTE_MAX_E) return bad("n_experts must be in [1, 1024]");
  if (q.top_k < 1 || q.top_k > ee::ROUTE_MAX_K || q.top_k > q.n_experts) return bad("top_k must be in [1, min(32, n_experts)]");
  if (q.score < 0 || q.score >= ee::SCORE_N) return bad("unknown score function");
  if (q.n_groups < 1 || q.n_groups > 64 || q.n_experts % q.n_groups) return bad("n_groups must be in [1, 64] and divide n_experts");
  if (q.top_groups < 1 || q.top_groups > q.n_groups) return bad("top_groups must be in [1, n_groups]");
  if (q.group_top < 1 || q.group_top > 2) return bad("group_top must be 1 or 2");
  if (q.top_k > q.n_experts / q.n_groups * q.top_groups) return bad("top_k exceeds the experts of top_groups groups");
  if (!isfinite(q.scale)) return bad("scale must be finite");
  if (q.rows == 0) return EE_OK;
  if (!q.logits || !q.ids || !q.weights) return bad("logits, ids and weights must be non-NULL");
  if (!out_ok(q.logits, q.ld, q.n_experts, q.dtype)) return bad("logits must be aligned to their type with a row stride of at least n_experts");
  if (!aligned(q.ids, 4) || !aligned(q.weights, 4) || (q.bias && !aligned(q.bias, 4))) return bad("ids, weights and bias must be aligned to their type");
  for (const void* y : {(const void*)q.ids, (const void*)q.weights})
    if (y == q.logits || y == q.bias) return bad("ids and weights must not be an input");
  if ((const void*)q.ids == q.weights) return bad("ids and weights must not be an input or each other");
  ee::RouteArgs a{};
  a.logits = q.logits; a.bias = q.bias; a.ids = q.ids; a.weights = q.weights; a.ld = q.ld;
  a.T = q.rows; a.E = q.n_experts; a.k = q.top_k; a.dt = dt_of(q.dtype);
  a.score = q.score; a.renorm = q.renormalize != 0;
  a.groups = q.n_groups; a.top_groups = q.top_groups; a.group_top = q.group_top; a.scale = q.scale;
  return launched(ee::run_route(a, reinterpret_cast<hipStream_t>(stream)));
}

static const char* ffn_shape(int64_t rows, int32_t E, int32_t k, int32_t d, int32_t F, int32_t dtype) {
  if (!dtype_ok(dtype)) return "dtype must be EE_F32 or EE_BF16";
  if (E < 1 || E > ee::ROUTE_MAX_E) return "n_experts must be in [1, 1024]";
  if (k < 1 || k > ee::ROUTE_MAX_K || k > E) return "top_k must be in [1, min(32, n_experts)]";
  if (rows < 0 || rows * k > MAX_PAIRS) return "rows * top_k must be in [0, 2^24]";
  if (d < 1 || d > 32768 || F < 1 || F > 32768) return "d_model and ffn must be in [1, 32768]";
  if (d % ks(dtype) || F % ks(dtype)) return "d_model and ffn must be multiples of 32 (bf16) / 16 (f32)";
  if ((int64_t)2 * F * d * esz(dtype) >= int64_t(1) << 31) return "an expert's gate and up weights must stay below 2 GiB";
  if (rows * k * ((d > F ? d : F) / 16) > MAX_BLOCKS) return "too many output tiles";
  return nullptr;
}

size_t ee_moe_ffn_workspace_bytes(int32_t rows, int32_t n_experts, int32_t top_k, int32_t d_model, int32_t ffn,
                                  int32_t dtype) {
  if (const char* why = ffn_shape(rows, n_experts, top_k, d_model, ffn, dtype)) {
    bad(why);
    return 0;
  }
  return ee::ffn_workspace(rows, n_experts, top_k, d_model, ffn, dt_of(dtype));
}

int32_t ee_moe_ffn(const ee_moe_ffn_args* p, void* stream) {
  if (!p) return bad("arguments are NULL");
  const ee_moe_ffn_args& q = *p;
  if (const char* why = ffn_shape(q.rows, q.n_experts, q.top_k, q.d_model, q.ffn, q.dtype)) return bad(why);
  if (!dtype_ok(q.out_dtype) || (q.dtype == EE_F32 && q.out_dtype != EE_F32)) return bad("out_dtype must be dtype or EE_F32");
  if (q.rows == 0) return EE_OK;
  if (!q.x || !q.w_gate_up || !q.w_down || !q.ids || !q.weights || !q.out || !q.workspace)
    return bad("x, w_gate_up, w_down, ids, weights, out and workspace must be non-NULL");
  if (!rows_ok(q.x, q.ldx, q.d_model, q.dtype)) return bad("x must be 16-byte aligned with a row stride of at least d_model, at most 2^21, and a multiple of 16 bytes");
  if (!aligned(q.w_gate_up, 16) || !aligned(q.w_down, 16)) return bad("w_gate_up and w_down must be 16-byte aligned");
  if (!aligned(q.ids, 4) || !aligned(q.weights, 4)) return bad("ids and weights must be aligned to their type");
  if (!out_ok(q.out, q.ldo, q.d_model, q.out_dtype)) return bad("out must be aligned to its type with a row stride of at least d_model");
  if (q.residual && !out_ok(q.residual, q.ldr, q.d_model, q.out_dtype)) return bad("residual must be aligned to its type with a row stride of at least d_model");
  if (!aligned(q.workspace, 256)) return bad("workspace must be 256-byte aligned");
  if (q.workspace_bytes < ee::ffn_workspace(q.rows, q.n_experts, q.top_k, q.d_model, q.ffn, dt_of(q.dtype)))
    return op_fail(EE_ECAPACITY, "workspace smaller than ee_moe_ffn_workspace_bytes");
  for (const void* in : {q.x, q.w_gate_up, q.w_down, (const void*)q.ids, (const void*)q.weights}) {
    if (q.out == in) return bad("out must not be an input, except the residual with its stride");
    if (q.workspace == in) return bad("the workspace must not be an input");
  }
  if (q.out == q.residual && q.ldr != q.ldo) return bad("out must not be an input, except the residual with its stride");
  if (q.workspace == q.out || q.workspace == q.residual) return bad("the workspace must not be an input or out");
  ee::FfnArgs a{};
  a.x = q.x; a.wgu = q.w_gate_up; a.wd = q.w_down; a.ids = q.ids; a.weights = q.weights; a.res = q.residual; a.out = q.out;
  a.ldx = q.ldx; a.ldr = q.ldr; a.ldo = q.ldo;
  a.T = q.rows; a.E = q.n_experts; a.k = q.top_k; a.d = q.d_model; a.F = q.ffn;
  a.dt = dt_of(q.dtype); a.odt = dt_of(q.out_dtype);
  a.ws = reinterpret_cast<unsigned char*>(q.workspace);
  return launched(ee::run_ffn(a, reinterpret_cast<hipStream_t>(stream)));
}

}  // extern "C"
