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

// Rows of `cols` codes, one byte each.
bool codes_ok(const void* p, int64_t ld, int cols) { return aligned(p, 16) && ld >= cols && ld <= MAX_LD && ld % 16 == 0; }

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

int32_t ee_fp8_quant(const ee_fp8_quant_args* p, void* stream) {
  if (!p) return bad("arguments are NULL");
  const ee_fp8_quant_args& q = *p;
  if (!dtype_ok(q.dtype)) return bad("dtype must be EE_F32 or EE_BF16");
  if (q.rows < 0 || q.rows > MAX_ROWS || q.in < 1 || q.in > MAX_COLS) return bad("rows must be in [0, 2^22], in in [1, 2^20]");
  if (q.in % 16) return bad("in must be a multiple of 16");
  if (q.block_rows != 1 && q.block_rows != ee::BLOCK) return bad("block_rows must be 1 or 128");
  if (q.rows == 0) return EE_OK;
  if (!q.x || !q.codes || !q.scales) return bad("x, codes and scales must be non-NULL");
  if (!rows_ok(q.x, q.ldx, q.in, q.dtype)) return bad("x must be 16-byte aligned with a row stride of at least `in`, at most 2^21, and a multiple of 16 bytes");
  if (!codes_ok(q.codes, q.ldc, q.in)) return bad("codes must be 16-byte aligned with a row stride of at least `in`, at most 2^21, and a multiple of 16");
  if (!aligned(q.scales, 4)) return bad("scales must be aligned to their type");
  if (q.codes == q.x || q.scales == q.x || (const void*)q.codes == q.scales) return bad("codes and scales must not be x or each other");
  ee::Fp8QuantArgs a{};
  a.x = q.x; a.codes = q.codes; a.scales = q.scales; a.ldx = q.ldx; a.ldc = q.ldc;
  a.T = q.rows; a.K = q.in; a.dt = dt_of(q.dtype); a.block_rows = q.block_rows;
  return launched(ee::run_fp8_quant(a, reinterpret_cast<hipStream_t>(stream)));
}

int32_t ee_fp8_linear(const ee_fp8_linear_args* p, void* stream) {
  if (!p) return bad("arguments are NULL");
  const ee_fp8_linear_args& q = *p;
  if (!dtype_ok(q.out_dtype)) return bad("out_dtype must be EE_F32 or EE_BF16");
  if (q.rows < 0 || q.rows > MAX_ROWS || q.in < 1 || q.in > MAX_COLS || q.out < 1 || q.out > MAX_COLS)
    return bad("rows must be in [0, 2^22], in and out in [1, 2^20]");
  if (q.in % 16) return bad("in must be a multiple of 16");
  if (q.act < 0 || q.act >= ee::ACT_N) return bad("unknown activation");
  if (q.rows == 0) return EE_OK;
  if (!q.x || !q.w || !q.x_scales || !q.w_scales || !q.y) return bad("x, w, their scales and y must be non-NULL");
  if (!codes_ok(q.x, q.ldx, q.in) || !codes_ok(q.w, q.ldw, q.in))
    return bad("x and w must be 16-byte aligned with row strides of at least `in`, at most 2^21, and a multiple of 16");
  if (!aligned(q.x_scales, 4) || !aligned(q.w_scales, 4) || (q.bias && !aligned(q.bias, 4)))
    return bad("the scales and bias must be aligned to their type");
  if (!out_ok(q.y, q.ldy, q.out, q.out_dtype)) return bad("y must be aligned to its type with a row stride of at least `out`");
  if (q.residual && !out_ok(q.residual, q.ldr, q.out, q.out_dtype))
    return bad("residual must be aligned to its type with a row stride of at least `out`");
  if ((int64_t)((q.rows + 15) / 16) * ((q.out + 15) / 16) > MAX_BLOCKS) return bad("too many output tiles");
  for (const void* in : {(const void*)q.x, (const void*)q.w, (const void*)q.x_scales, (const void*)q.w_scales, (const void*)q.bias})
    if (q.y == in) return bad("y must not be an input, except the residual with its stride");
  if (q.y == q.residual && q.ldr != q.ldy) return bad("y must not be an input, except the residual with its stride");
  ee::Fp8LinearArgs a{};
  a.l.x = q.x; a.l.w = q.w; a.l.bias = q.bias; a.l.res = q.residual; a.l.y = q.y;
  a.l.ldx = q.ldx; a.l.ldw = q.ldw; a.l.ldr = q.ldr; a.l.ldy = q.ldy;
  a.l.T = q.rows; a.l.K = q.in; a.l.N = q.out;
  a.l.odt = dt_of(q.out_dtype); a.l.act = q.act;
  a.xs = q.x_scales; a.ws = q.w_scales;
  return launched(ee::run_fp8_linear(a, reinterpret_cast<hipStream_t>(stream)));
}

// What appending and attention check of a cache and the heads around it.
constexpr int MAX_HEADS = 1024, MAX_POSITIONS = 1 << 30;
constexpr int64_t MAX_STATES = 1 << 24;   // rows times heads of a call: its launches stay below 2^32 threads
static const char* cache_shape(const ee_paged_cache& c, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int32_t dtype) {
  if (!dtype_ok(dtype)) return "dtype must be EE_F32 or EE_BF16";
  if (head_dim != 64 && head_dim != 128 && head_dim != 256) return "head_dim must be 64, 128 or 256";
  if (n_heads < 1 || n_heads > MAX_HEADS || n_kv_heads < 1 || n_heads % n_kv_heads) return "n_heads must be in [1, 1024] and a multiple of n_kv_heads";
  if (c.n_seqs < 0 || c.n_seqs > MAX_ROWS) return "n_seqs must be in [0, 2^22]";
  if (c.page_size < 16 || c.page_size > 65536 || c.page_size % 16) return "page_size must be a multiple of 16, at most 65536";
  if (c.max_pages < 0 || (int64_t)c.max_pages * c.page_size > MAX_POSITIONS) return "max_pages * page_size must be in [0, 2^30]";
  if (c.n_pages < 0) return "n_pages must not be negative";
  return nullptr;
}
static const char* cache_memory(const ee_paged_cache& c, int32_t n_kv_heads, int32_t head_dim, int32_t dtype) {
  // (a pool of no pages and tables of no columns have no memory: their sequences hold nothing)
  if ((c.n_pages && (!c.k || !c.v)) || (c.max_pages && !c.tables)) return "the cache's k, v and tables must be non-NULL";
  const int64_t e = esz(dtype), strides[6] = {c.k_page, c.k_slot, c.k_head, c.v_page, c.v_slot, c.v_head};
  for (int64_t s : strides)
    if (s < 0 || s >= int64_t(1) << 40 || s * e % 16) return "the cache's strides must be multiples of 16 bytes, not negative and below 2^40";
  if (!aligned(c.k, 16) || !aligned(c.v, 16)) return "the cache must be 16-byte aligned";
  for (int i = 0; i < 6; i += 3)
    if (strides[i + 1] * e * c.page_size >= int64_t(1) << 31) return "a head's slots of a page must lie within 2 GiB";
  if (c.k_slot < head_dim || c.v_slot < head_dim) return "a head's slots must not share memory";
  if (!aligned(c.tables, 4) || c.ld < c.max_pages || c.ld >= int64_t(1) << 40) return "tables must be aligned to their type with a row stride of at least max_pages";
  return nullptr;
}
// Whether no two of a cache's vectors share memory (they are written).
static bool apart(int64_t page, int64_t pages, int64_t slot, int64_t slots, int64_t head, int64_t heads, int64_t dim) {
  int64_t s[3][2] = {{page, pages}, {slot, slots}, {head, heads}};
  for (int i = 0; i < 3; ++i)
    for (int j = 0; j + 1 < 3 - i; ++j)
      if (s[j][0] > s[j + 1][0]) {
        for (int k = 0; k < 2; ++k) {
          const int64_t t = s[j][k];
          s[j][k] = s[j + 1][k];
          s[j + 1][k] = t;
        }
      }
  int64_t extent = dim;
  for (auto& d : s) {
    if (d[1] < 2) continue;
    if (d[0] < extent) return false;
    extent += d[0] * (d[1] - 1);
  }
  return true;
}
static ee::PagedCache paged(const ee_paged_cache& c) {
  return {c.k, c.v, c.k_page, c.k_slot, c.k_head, c.v_page, c.v_slot, c.v_head, c.tables, c.ld, c.n_pages, c.max_pages, c.page_size};
}

int32_t ee_kv_append(const ee_kv_append_args* p, void* stream) {
  if (!p) return bad("arguments are NULL");
  const ee_kv_append_args& q = *p;
  if (const char* why = cache_shape(q.cache, q.n_heads, q.n_kv_heads, q.head_dim, q.dtype)) return bad(why);
  if (q.rows < 0 || q.rows > MAX_ROWS) return bad("rows must be in [0, 2^22]");
  if (q.rot_dim < 0 || q.rot_dim > q.head_dim || q.rot_dim % 16) return bad("rot_dim must be a multiple of 16 in [0, head_dim]");
  if (!q.seqs && q.rows && (q.cache.n_seqs < 1 || q.rows % q.cache.n_seqs)) return bad("rows must be a multiple of n_seqs where seqs is NULL");
  if (q.rows == 0) return EE_OK;
  if (!q.k || !q.v || !q.positions) return bad("k, v and positions must be non-NULL");
  if ((q.q == nullptr) != (q.q_out == nullptr)) return bad("q and q_out must be given together");
  if (q.rot_dim && (!q.inv_freq || !aligned(q.inv_freq, 8))) return bad("inv_freq must be non-NULL and aligned to its type");
  if (const char* why = cache_memory(q.cache, q.n_kv_heads, q.head_dim, q.dtype)) return bad(why);
  const int kd = q.n_kv_heads * q.head_dim, qd = q.n_heads * q.head_dim;
  if (!rows_ok(q.k, q.ldk, kd, q.dtype) || !rows_ok(q.v, q.ldv, kd, q.dtype) || (q.q && (!rows_ok(q.q, q.ldq, qd, q.dtype) || !rows_ok(q.q_out, q.ldqo, qd, q.dtype))))
    return bad("q, k, v and q_out must be 16-byte aligned with row strides of at least their heads' width, at most 2^21, and a multiple of 16 bytes");
  if (!aligned(q.positions, 4) || (q.seqs && !aligned(q.seqs, 4))) return bad("positions and seqs must be aligned to their type");
  const ee_paged_cache& c = q.cache;
  if (!apart(c.k_page, c.n_pages, c.k_slot, c.page_size, c.k_head, q.n_kv_heads, q.head_dim) ||
      !apart(c.v_page, c.n_pages, c.v_slot, c.page_size, c.v_head, q.n_kv_heads, q.head_dim))
    return bad("the cache's vectors must not share memory");
  if (c.k && c.k == c.v) return bad("the cache's k and v must not be the same");
  for (const void* in : {q.k, q.v, (const void*)q.positions, (const void*)q.seqs, (const void*)q.inv_freq, (const void*)c.tables}) {
    if (in && (c.k == in || c.v == in)) return bad("the cache must not be an input");
    if (in && q.q_out == in) return bad("q_out must not be an input, except q with its stride");
  }
  if (q.q && (q.q_out == c.k || q.q_out == c.v || q.q == c.k || q.q == c.v)) return bad("q and q_out must not be the cache");
  if (q.q && q.q_out == q.q && q.ldq != q.ldqo) return bad("q_out must not be an input, except q with its stride");
  ee::AppendArgs a{};
  a.q = q.q; a.k = q.k; a.v = q.v; a.q_out = q.q_out; a.c = paged(c); a.seqs = q.seqs; a.positions = q.positions; a.inv_freq = q.inv_freq;
  a.ldq = q.ldq; a.ldk = q.ldk; a.ldv = q.ldv; a.ldqo = q.ldqo;
  a.R = q.rows; a.B = c.n_seqs; a.per_seq = q.seqs ? 1 : q.rows / c.n_seqs;
  a.H = q.n_heads; a.Hkv = q.n_kv_heads; a.hd = q.head_dim; a.rot = q.rot_dim; a.interleaved = q.interleaved != 0; a.dt = dt_of(q.dtype);
  return launched(ee::run_append(a, reinterpret_cast<hipStream_t>(stream)));
}

static const char* attend_shape(int64_t n_seqs, int64_t rows, int32_t n_heads, int64_t positions, int32_t head_dim, int32_t window) {
  if (rows < 1 || rows > 1024 || n_seqs * rows > MAX_ROWS) return "rows must be in [1, 1024], n_seqs * rows at most 2^22";
  if (window < 0) return "window must not be negative";
  if (n_seqs * rows * n_heads > MAX_STATES) return "too many rows and heads: n_seqs * rows * n_heads must be at most 2^24";
  return nullptr;
}

size_t ee_paged_attention_workspace_bytes(int32_t n_seqs, int32_t rows, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim,
                                          int32_t page_size, int32_t max_pages, int32_t window) {
  ee_paged_cache c{};
  c.n_seqs = n_seqs; c.page_size = page_size; c.max_pages = max_pages;
  const char* why = cache_shape(c, n_heads, n_kv_heads, head_dim, EE_BF16);
  if (!why) why = attend_shape(n_seqs, rows, n_heads, (int64_t)max_pages * page_size, head_dim, window);
  if (why) {
    bad(why);
    return 0;
  }
  return ee::attend_workspace(n_seqs, rows, n_heads, head_dim, (int64_t)max_pages * page_size, window);
}

int32_t ee_paged_attention(const ee_paged_attention_args* p, void* stream) {
  if (!p) return bad("arguments are NULL");
  const ee_paged_attention_args& q = *p;
  const ee_paged_cache& c = q.cache;
  if (const char* why = cache_shape(c, q.n_heads, q.n_kv_heads, q.head_dim, q.dtype)) return bad(why);
  if (const char* why = attend_shape(c.n_seqs, q.rows, q.n_heads, (int64_t)c.max_pages * c.page_size, q.head_dim, q.window)) return bad(why);
  if (!dtype_ok(q.out_dtype) || (q.dtype == EE_F32 && q.out_dtype != EE_F32)) return bad("out_dtype must be dtype or EE_F32");
  if (!isfinite(q.scale)) return bad("scale must be finite");
  if (c.n_seqs == 0) return EE_OK;
  if (!q.q || !q.out || !q.lens || !q.workspace) return bad("q, out, lens and workspace must be non-NULL");
  if (const char* why = cache_memory(c, q.n_kv_heads, q.head_dim, q.dtype)) return bad(why);
  const int qd = q.n_heads * q.head_dim;
  if (!rows_ok(q.q, q.ldq, qd, q.dtype)) return bad("q must be 16-byte aligned with a row stride of at least its heads' width, at most 2^21, and a multiple of 16 bytes");
  if (!out_ok(q.out, q.ldo, qd, q.out_dtype)) return bad("out must be aligned to its type with a row stride of at least its heads' width");
  if (!aligned(q.lens, 4) || (q.lse && !aligned(q.lse, 4))) return bad("lens and lse must be aligned to their type");
  if (!aligned(q.workspace, 256)) return bad("workspace must be 256-byte aligned");
  const int64_t positions = (int64_t)c.max_pages * c.page_size;
  if (q.workspace_bytes < ee::attend_workspace(c.n_seqs, q.rows, q.n_heads, q.head_dim, positions, q.window))
    return op_fail(EE_ECAPACITY, "workspace smaller than ee_paged_attention_workspace_bytes");
  for (const void* in : {q.q, (const void*)c.k, (const void*)c.v, (const void*)c.tables, (const void*)q.lens}) {
    if (in && (q.out == in || q.lse == in)) return bad("out and lse must not be an input");
    if (q.workspace == in) return bad("the workspace must not be an input");
  }
  if (q.out == (const void*)q.lse || q.workspace == q.out || q.workspace == (const void*)q.lse) return bad("out, lse and the workspace must not be each other");
  ee::AttendArgs a{};
  a.q = q.q; a.out = q.out; a.lse = q.lse; a.c = paged(c); a.lens = q.lens; a.ws = reinterpret_cast<unsigned char*>(q.workspace);
  a.ldq = q.ldq; a.ldo = q.ldo;
  a.B = c.n_seqs; a.T = q.rows; a.H = q.n_heads; a.Hkv = q.n_kv_heads; a.G = q.n_heads / q.n_kv_heads; a.hd = q.head_dim;
  a.dt = dt_of(q.dtype); a.odt = dt_of(q.out_dtype);
  a.window = q.window < positions ? q.window : 0;   // (so that kernels may subtract it from a negative end)
  a.scale_log2 = q.scale * 1.4426950408889634f;
  return launched(ee::run_attend(a, reinterpret_cast<hipStream_t>(stream)));
}

}  // extern "C"
