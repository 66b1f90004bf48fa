// Entry points of libbsa_ops.so: argument checks and launches.
#include "bsa_ops.h"

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <initializer_list>

#include "ops_internal.h"

using namespace bsa_ops;

namespace {

thread_local char g_err[256];

// (a fixed buffer: reporting a failure cannot fail)
bsa_status fail(bsa_status s, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  std::vsnprintf(g_err, sizeof(g_err), fmt, ap);
  va_end(ap);
  return s;
}

bsa_status launched(hipError_t e, const char* what) {
  if (e == hipSuccess) return BSA_OK;
  return fail(BSA_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

int64_t elem_size(int32_t dtype) { return dtype == BSA_DTYPE_F32 ? 4 : 2; }

// Longest sequence and most rows of a key head: row numbers, positions and
// their differences stay within 32 bits.
constexpr int64_t kMaxSeq = int64_t(1) << 29;
constexpr int64_t kMaxRows = int64_t(1) << 30;
constexpr float kLog2e = 1.44269504088896340736f;

// A tensor [batch, tokens, heads, d] with strides (batch, head, token).
struct Tensor {
  const char* name;
  const void* ptr;
  const int64_t* stride;
  int64_t batch, heads, tokens, d;
  bool output;
};

bsa_status check_tensor(const Tensor& t, int64_t size) {
  if (t.batch == 0 || t.heads == 0 || t.tokens == 0) return BSA_OK;  // no element
  if (!t.ptr) return fail(BSA_ERR_INVALID, "%s must be a device pointer", t.name);
  if ((uintptr_t)t.ptr % 16) return fail(BSA_ERR_INVALID, "%s must be 16-byte aligned", t.name);
  const int64_t n[3] = {t.batch, t.heads, t.tokens};
  for (int i = 0; i < 3; ++i) {
    if (t.stride[i] < 0) return fail(BSA_ERR_INVALID, "%s has a negative stride", t.name);
    if (t.stride[i] > (int64_t(1) << 56) / n[i])
      return fail(BSA_ERR_INVALID, "%s reaches past the address space", t.name);
    if (n[i] > 1 && t.stride[i] * size % 16)
      return fail(BSA_ERR_INVALID, "token rows of %s must start 16-byte aligned (stride %lld)", t.name, (long long)t.stride[i]);
  }
  if (!t.output) return BSA_OK;
  // rows that do not overlap: from the smallest stride up, each step clears
  // everything that the ones before it span
  int order[3] = {0, 1, 2};
  std::sort(order, order + 3, [&](int x, int y) { return t.stride[x] < t.stride[y]; });
  int64_t span = t.d;
  for (int i : order) {
    if (n[i] == 1) continue;
    if (t.stride[i] < span) return fail(BSA_ERR_INVALID, "rows of the output %s overlap", t.name);
    span += (n[i] - 1) * t.stride[i];
  }
  return BSA_OK;
}

Strides strides(const int64_t* s) { return Strides{s[0], s[1], s[2]}; }
// For tensors whose token rows are loaded in tiles: the stride of an axis of one token
// says nothing, and a row's length in its place keeps the tile's other rows out of bounds.
Strides tile_strides(const int64_t* s, int64_t tokens, int64_t d) { return Strides{s[0], s[1], tokens > 1 ? s[2] : d}; }

// ---------------------------------------------------------------- window
bsa_status check_window(const bsa_window_shapes* sp) {
  if (!sp) return fail(BSA_ERR_INVALID, "shapes must not be null");
  const bsa_window_shapes& s = *sp;
  if (s.batch < 0 || s.seq_q < 0 || s.seq_kv < 0 || s.heads < 1 || s.kv_heads < 1)
    return fail(BSA_ERR_INVALID, "batch, seq_q and seq_kv must not be negative, heads and kv_heads positive");
  if (s.heads % s.kv_heads) return fail(BSA_ERR_INVALID, "heads (%d) must be a multiple of kv_heads (%d)", s.heads, s.kv_heads);
  if (s.left < -1 || s.right < -1 || s.sinks < 0)
    return fail(BSA_ERR_INVALID, "left and right must be -1 or more, sinks 0 or more");
  if (!(s.scale >= 0.f) || std::isinf(s.scale * kLog2e)) return fail(BSA_ERR_INVALID, "scale must be positive and finite (or 0)");
  if (s.reserved != 0) return fail(BSA_ERR_INVALID, "reserved must be 0");
  if (s.dtype != BSA_DTYPE_BF16 && s.dtype != BSA_DTYPE_F16)
    return fail(BSA_ERR_UNSUPPORTED, "only bfloat16 and float16 tensors are implemented");
  if (s.head_dim != 64 && s.head_dim != 128) return fail(BSA_ERR_UNSUPPORTED, "only head_dim 64 and 128 are implemented");
  if (s.seq_q > kMaxSeq || s.seq_kv > kMaxSeq) return fail(BSA_ERR_UNSUPPORTED, "sequences of more than 2^29 tokens");
  if ((int64_t)s.seq_q * (s.heads / s.kv_heads) > kMaxRows)
    return fail(BSA_ERR_UNSUPPORTED, "more than 2^30 query rows for one key head");
  return BSA_OK;
}

// Tiles are addressed with 32 bits from their first row on.
bsa_status check_tile_stride(const char* name, int64_t stride, int64_t tokens) {
  if (tokens > 1 && stride >= (int64_t(1) << 23))
    return fail(BSA_ERR_UNSUPPORTED, "token stride of %s is 2^23 elements or more", name);
  return BSA_OK;
}

WindowArgs window_args(const bsa_window_shapes& s) {
  WindowArgs a{};
  a.qs = tile_strides(s.q_stride, s.seq_q, s.head_dim);
  a.ks = tile_strides(s.k_stride, s.seq_kv, s.head_dim);
  a.vs = tile_strides(s.v_stride, s.seq_kv, s.head_dim);
  a.os = strides(s.o_stride);
  a.B = s.batch;
  a.H = s.heads;
  a.Hkv = s.kv_heads;
  a.group = s.heads / s.kv_heads;
  a.Nq = s.seq_q;
  a.Nkv = s.seq_kv;
  a.left = s.left < 0 || s.left > kFar ? kFar : s.left;
  a.right = s.right < 0 || s.right > kFar ? kFar : s.right;
  a.sinks = std::min(s.sinks, s.seq_kv);
  // One side spans much of the sequence and the other does not: the walks of a head's tiles
  // are of very different lengths.  They are walked longest first, and dealt out unless
  // every XCD gets whole heads of every sequence, or there are many heads, whose keys are
  // better read by one XCD.  (8192 tokens, all keys before, forward, dQ, dK and dV: 12
  // heads 1109 us in shares from the first tile on, 915 dealt out; 32 heads 2412 and 2290
  // with the longest first.  40 sequences of 2048 tokens, 2 key heads: 1300 and 945 with
  // shares that move on from sequence to sequence.)  At the limits, forward, dQ, dK and dV:
  // 60 heads in all (5 sequences of 2048) 454 us in shares and 390 dealt out, 64 heads 484
  // and 377; 66 heads 494 and 416, 100 heads 667 and 602, so up to there short sequences
  // would still gain; 96 heads of 8192 tokens 7040 and 7390, 300 heads of 2048 1810 and
  // 1835.  kv_heads a multiple of 8: 8 heads of 8192 730 and 752, 16 heads 1203 and 1214.
  const bool far_left = 2 * (int64_t)a.left > s.seq_kv, far_right = 2 * (int64_t)a.right > s.seq_kv;
  a.deal = far_left != far_right && s.kv_heads % 8 != 0 && (int64_t)s.batch * s.kv_heads <= 64;
  a.later_longer = far_left && !far_right;
  a.scale = s.scale > 0.f ? s.scale : 1.f / std::sqrt((float)s.head_dim);
  a.scale_log2 = a.scale * kLog2e;
  return a;
}

int64_t window_bytes(WindowArgs a, int d, bool backward) {
  return 4 * (backward ? plan_backward(&a, d) : plan_forward(a, d).part_floats);
}

bsa_status check_workspace(int64_t need, const void* workspace, size_t bytes) {
  if (need == 0) return BSA_OK;
  if (!workspace || (int64_t)bytes < need)
    return fail(BSA_ERR_INVALID, "workspace of %lld bytes needed, %lld given", (long long)need,
                (long long)(workspace ? bytes : 0));
  if ((uintptr_t)workspace % 16) return fail(BSA_ERR_INVALID, "workspace must be 16-byte aligned");
  return BSA_OK;
}

// A result is not written over a tensor that other workgroups still read.
bsa_status check_apart(const char* name, const void* out, std::initializer_list<const void*> inputs) {
  for (const void* p : inputs)
    if (out && out == p) return fail(BSA_ERR_INVALID, "%s is one of the inputs or of the other outputs", name);
  return BSA_OK;
}

#define TRY(x)                          \
  do {                                  \
    const bsa_status st_ = (x);         \
    if (st_ != BSA_OK) return st_;      \
  } while (0)

}  // namespace

extern "C" {

const char* bsa_ops_last_error(void) { return g_err; }

bsa_status bsa_rope(const bsa_rope_shapes* shapes, const double* freq, const int32_t* positions, const int32_t* lengths,
                    const int32_t* rows, const void* q, const void* k, const void* v, void* q_out, void* k_out,
                    void* v_out, void* stream) {
  g_err[0] = 0;
  if (!shapes) return fail(BSA_ERR_INVALID, "shapes must not be null");
  const bsa_rope_shapes& s = *shapes;
  if (s.batch < 0 || s.seq < 0 || s.heads < 1 || s.kv_heads < 0 || s.kv_rows < 0)
    return fail(BSA_ERR_INVALID, "batch, seq, kv_heads and kv_rows must not be negative, heads positive");
  if (s.dtype != BSA_DTYPE_BF16 && s.dtype != BSA_DTYPE_F16 && s.dtype != BSA_DTYPE_F32)
    return fail(BSA_ERR_UNSUPPORTED, "only bfloat16, float16 and float32 tensors are implemented");
  if (s.head_dim < 8 || s.head_dim > 256 || s.head_dim % 8)
    return fail(BSA_ERR_UNSUPPORTED, "head_dim must be a multiple of 8 up to 256");
  int64_t P = 0;
  for (int i = 0; i < 3; ++i) {
    if (s.pairs[i] < 0) return fail(BSA_ERR_INVALID, "pairs must not be negative");
    P += s.pairs[i];
  }
  if (2 * P > s.head_dim) return fail(BSA_ERR_INVALID, "%lld pairs do not fit head_dim %d", (long long)P, s.head_dim);
  if (P > 0 && !freq) return fail(BSA_ERR_INVALID, "freq must be a device pointer");
  if (s.seq > kMaxSeq) return fail(BSA_ERR_UNSUPPORTED, "sequences of more than 2^29 tokens");
  RopeArgs a{};
  if (!positions) {
    a.volume = 1;
    for (int i = 0; i < 3; ++i) {
      if (s.grid[i] < 1) return fail(BSA_ERR_INVALID, "grid sizes must be positive where no positions are given");
      if (std::abs((int64_t)s.origin[i]) + s.grid[i] > (int64_t(1) << 30))
        return fail(BSA_ERR_INVALID, "grid positions beyond 2^30");
      a.volume = std::min<int64_t>(a.volume * s.grid[i], int64_t(1) << 31);  // seq is less
    }
    if ((int64_t)s.grid[1] * s.grid[2] > (int64_t(1) << 30)) return fail(BSA_ERR_INVALID, "grid planes beyond 2^30 tokens");
  } else if (s.pos_stride[0] < 0 || s.pos_stride[1] < 0) {
    return fail(BSA_ERR_INVALID, "positions have a negative stride");
  }
  const bool with_k = k != nullptr && s.kv_heads > 0, with_v = v != nullptr && s.kv_heads > 0;
  if (s.kv_heads > 0 && !k && s.batch > 0 && s.seq > 0) return fail(BSA_ERR_INVALID, "k must be a device pointer (or kv_heads 0)");
  const int64_t size = elem_size(s.dtype);
  TRY(check_tensor({"q", q, s.q_stride, s.batch, s.heads, s.seq, s.head_dim, false}, size));
  TRY(check_tensor({"q_out", q_out, s.q_out_stride, s.batch, s.heads, s.seq, s.head_dim, true}, size));
  if (!rows && with_k && s.kv_rows < s.seq)
    return fail(BSA_ERR_INVALID, "kv_rows (%d) must be seq or more where rows is NULL", s.kv_rows);
  const int64_t kv_rows = rows ? s.kv_rows : s.seq;
  if (with_k) {
    TRY(check_tensor({"k", k, s.k_stride, s.batch, s.kv_heads, s.seq, s.head_dim, false}, size));
    TRY(check_tensor({"k_out", k_out, s.k_out_stride, s.batch, s.kv_heads, kv_rows, s.head_dim, true}, size));
  }
  if (with_v) {
    TRY(check_tensor({"v", v, s.v_stride, s.batch, s.kv_heads, s.seq, s.head_dim, false}, size));
    TRY(check_tensor({"v_out", v_out, s.v_out_stride, s.batch, s.kv_heads, kv_rows, s.head_dim, true}, size));
  }
  const void *kin = with_k ? k : nullptr, *vin = with_v ? v : nullptr;
  void *kout = with_k ? k_out : nullptr, *vout = with_v ? v_out : nullptr;
  if (rows && ((with_k && k_out == k) || (with_v && v_out == v)))
    return fail(BSA_ERR_INVALID, "k and v cannot be turned in place when rows moves them");

  const struct {
    const char* name;
    const void *x, *y;
    const int64_t *xs, *ys;
    int64_t heads;
  } pair[3] = {{"q", q, q_out, s.q_stride, s.q_out_stride, s.heads},
               {"k", kin, k_out, s.k_stride, s.k_out_stride, s.kv_heads},
               {"v", vin, v_out, s.v_stride, s.v_out_stride, s.kv_heads}};
  for (const auto& p : pair) {
    if (p.x && p.x == p.y && ((s.batch > 1 && p.xs[0] != p.ys[0]) || (p.heads > 1 && p.xs[1] != p.ys[1]) ||
                              (s.seq > 1 && p.xs[2] != p.ys[2])))
      return fail(BSA_ERR_INVALID, "%s is turned in place with other strides", p.name);
  }

  TRY(check_apart("q_out", q_out, {kin, vin, kout, vout}));
  TRY(check_apart("k_out", kout, {q, vin, vout}));
  TRY(check_apart("v_out", vout, {q, kin}));

  const void* x[3] = {q, kin, vin};
  void* y[3] = {q_out, kout, vout};
  const int64_t* xs[3] = {s.q_stride, s.k_stride, s.v_stride};
  const int64_t* ys[3] = {s.q_out_stride, s.k_out_stride, s.v_out_stride};
  for (int t = 0; t < 3; ++t) {
    a.x[t] = x[t];
    a.y[t] = y[t];
    a.xs[t] = strides(xs[t]);
    a.ys[t] = strides(ys[t]);
    a.heads[t] = t == 0 ? s.heads : x[t] ? s.kv_heads : 0;
  }
  a.batch = s.batch;
  a.seq = s.seq;
  a.d = s.head_dim;
  a.P = (int32_t)P;
  a.end0 = s.pairs[0];
  a.end1 = s.pairs[0] + s.pairs[1];
  a.inverse = s.inverse ? 1 : 0;
  a.g1 = positions ? 1 : s.grid[1];
  a.g2 = positions ? 1 : s.grid[2];
  for (int i = 0; i < 3; ++i) a.origin[i] = s.origin[i];
  a.kv_rows = s.kv_rows;
  a.freq = freq;
  a.positions = positions;
  a.ps0 = s.pos_stride[0];
  a.ps1 = s.pos_stride[1];
  a.lengths = lengths;
  a.rows = rows;
  return launched(launch_rope(s.dtype, s.interleaved != 0, a, (hipStream_t)stream), "rope launch");
}

bsa_status bsa_window_workspace(const bsa_window_shapes* shapes, int32_t backward, size_t* bytes) {
  g_err[0] = 0;
  if (!bytes) return fail(BSA_ERR_INVALID, "bytes must not be null");
  *bytes = 0;
  TRY(check_window(shapes));
  *bytes = (size_t)window_bytes(window_args(*shapes), shapes->head_dim, backward != 0);
  return BSA_OK;
}

bsa_status bsa_window_forward(const bsa_window_shapes* shapes, const void* q, const void* k, const void* v, void* o,
                              float* lse, const int32_t* q_len, const int32_t* kv_len, void* workspace,
                              size_t workspace_bytes, void* stream) {
  g_err[0] = 0;
  TRY(check_window(shapes));
  const bsa_window_shapes& s = *shapes;
  TRY(check_tensor({"q", q, s.q_stride, s.batch, s.heads, s.seq_q, s.head_dim, false}, 2));
  TRY(check_tensor({"o", o, s.o_stride, s.batch, s.heads, s.seq_q, s.head_dim, true}, 2));
  TRY(check_tensor({"k", k, s.k_stride, s.batch, s.kv_heads, s.seq_kv, s.head_dim, false}, 2));
  TRY(check_tensor({"v", v, s.v_stride, s.batch, s.kv_heads, s.seq_kv, s.head_dim, false}, 2));
  TRY(check_tile_stride("k", s.k_stride[2], s.seq_kv));
  TRY(check_tile_stride("v", s.v_stride[2], s.seq_kv));
  TRY(check_apart("o", o, {q, k, v}));
  WindowArgs a = window_args(s);
  TRY(check_workspace(window_bytes(a, s.head_dim, false), workspace, workspace_bytes));
  a.q = q;
  a.k = k;
  a.v = v;
  a.o = o;
  a.lse = lse;
  a.q_len = q_len;
  a.kv_len = kv_len;
  a.part = static_cast<float*>(workspace);
  return launched(launch_window_forward(s.dtype, s.head_dim, a, (hipStream_t)stream), "window forward launch");
}

bsa_status bsa_window_backward(const bsa_window_shapes* shapes, const bsa_window_grads* grads, const void* q,
                               const void* k, const void* v, const void* o, const float* lse, const void* dout,
                               void* dq, void* dk, void* dv, const int32_t* q_len, const int32_t* kv_len,
                               void* workspace, size_t workspace_bytes, void* stream) {
  g_err[0] = 0;
  TRY(check_window(shapes));
  if (!grads) return fail(BSA_ERR_INVALID, "grads must not be null");
  const bsa_window_shapes& s = *shapes;
  const bsa_window_grads& g = *grads;
  if (!lse && s.batch > 0 && s.seq_q > 0) return fail(BSA_ERR_INVALID, "lse must be a device pointer");
  TRY(check_tensor({"q", q, s.q_stride, s.batch, s.heads, s.seq_q, s.head_dim, false}, 2));
  TRY(check_tensor({"o", o, s.o_stride, s.batch, s.heads, s.seq_q, s.head_dim, false}, 2));
  TRY(check_tensor({"dout", dout, g.do_stride, s.batch, s.heads, s.seq_q, s.head_dim, false}, 2));
  TRY(check_tensor({"dq", dq, g.dq_stride, s.batch, s.heads, s.seq_q, s.head_dim, true}, 2));
  TRY(check_tensor({"k", k, s.k_stride, s.batch, s.kv_heads, s.seq_kv, s.head_dim, false}, 2));
  TRY(check_tensor({"v", v, s.v_stride, s.batch, s.kv_heads, s.seq_kv, s.head_dim, false}, 2));
  TRY(check_tensor({"dk", dk, g.dk_stride, s.batch, s.kv_heads, s.seq_kv, s.head_dim, true}, 2));
  TRY(check_tensor({"dv", dv, g.dv_stride, s.batch, s.kv_heads, s.seq_kv, s.head_dim, true}, 2));
  TRY(check_tile_stride("q", s.q_stride[2], s.seq_q));
  TRY(check_tile_stride("dout", g.do_stride[2], s.seq_q));
  TRY(check_tile_stride("k", s.k_stride[2], s.seq_kv));
  TRY(check_tile_stride("v", s.v_stride[2], s.seq_kv));
  TRY(check_apart("dq", dq, {q, k, v, o, dout, dk, dv}));
  TRY(check_apart("dk", dk, {q, k, v, o, dout, dv}));
  TRY(check_apart("dv", dv, {q, k, v, o, dout}));
  WindowArgs a = window_args(s);
  TRY(check_workspace(window_bytes(a, s.head_dim, true), workspace, workspace_bytes));
  a.q = q;
  a.k = k;
  a.v = v;
  a.o = const_cast<void*>(o);
  a.lse = const_cast<float*>(lse);
  a.dout = dout;
  a.dq = dq;
  a.dk = dk;
  a.dv = dv;
  a.dos = tile_strides(g.do_stride, s.seq_q, s.head_dim);
  a.dqs = strides(g.dq_stride);
  a.dks = strides(g.dk_stride);
  a.dvs = strides(g.dv_stride);
  a.q_len = q_len;
  a.kv_len = kv_len;
  a.stats = static_cast<float*>(workspace);
  return launched(launch_window_backward(s.dtype, s.head_dim, a, (hipStream_t)stream), "window backward launch");
}

}  // extern "C"
