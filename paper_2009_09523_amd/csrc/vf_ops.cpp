// C ABI of the operators between an attention block's projections: argument checks and the
// rotation's frequencies; the kernels are in k_rope.hip and k_xattn.hip.
#include <algorithm>
#include <cfloat>
#include <climits>
#include <cmath>

#include "vf_internal.h"

using namespace vf;

namespace {

constexpr int64_t kMaxRows = INT32_MAX;
constexpr int64_t kMaxFirst = int64_t(1) << 52;            // positions are taken to float64
constexpr int kMaxHeads = 8192, kMaxHead = 512;            // (heads: an item's row is found by a multiplication that is exact up to there)

bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

// One axis of an output: its stride and how many of it there are.
struct Axis { int64_t stride, count; };

// Whether blocks of `inner` contiguous elements at these strides lie apart: going up the strides, every stride is at
// least what lies below it spans.  (Sufficient; interleavings that also keep elements apart are refused.)
bool apart(Axis* a, int n, int64_t inner) {
  std::sort(a, a + n, [](const Axis& x, const Axis& y) { return x.stride < y.stride; });
  int64_t span = inner;
  for (int i = 0; i < n; ++i)
    if (a[i].count == 0) return true;                       // nothing is written
  for (int i = 0; i < n; ++i) {
    if (a[i].count <= 1) continue;
    if (a[i].stride < span) return false;
    span += a[i].stride * (a[i].count - 1);
  }
  return true;
}

bool plan_ok(const vf_rope_plan* p, int d_head) {
  if (!p) return true;
  return (p->layout == VF_ROPE_HALF || p->layout == VF_ROPE_INTERLEAVED) && p->rot_dim >= 2 && p->rot_dim % 2 == 0 &&
         p->rot_dim <= 2 * VF_ROPE_MAX_PAIRS && p->rot_dim <= d_head;
}

void use_plan(RopeJob& j, const vf_rope_plan* p, bool inverse) {
  j.layout = p ? p->layout : VF_ROPE_HALF;
  j.rot = p ? p->rot_dim : 0;
  j.scale = p ? p->scale : 1.f;
  j.sign = inverse ? -1.f : 1.f;
}

// The stride of an axis of one entry says nothing.
int64_t stride_of(int64_t stride, int64_t count) { return count > 1 ? stride : 0; }
void trim(vf_attn_layout& l, int64_t batch, int64_t rows, int64_t heads) {
  l = vf_attn_layout{stride_of(l.batch, batch), stride_of(l.row, rows), stride_of(l.head, heads)};
}

// Element size of a dtype, 0 if it is none.
size_t size_of(int32_t dtype) { return dtype == VF_BF16 ? 2 : dtype == VF_F32 ? 4 : 0; }

// What the calls over [rows, heads, d_head] have in common.  0 rows or heads: *empty.
int check_heads(int32_t dtype, const void* x, const void* y, int64_t y_row, int64_t y_head, int64_t rows, int64_t heads,
                int32_t d_head, int64_t first, int64_t seq_len, const vf_rope_plan* plan, bool* empty) {
  const size_t esz = size_of(dtype);
  if (!esz || rows < 0 || rows > kMaxRows || heads < 0 || heads > kMaxHeads || d_head < 1 || d_head > kMaxHead || seq_len < 0 ||
      first < -kMaxFirst || first > kMaxFirst)
    return VF_EINVAL;
  if (!plan_ok(plan, d_head)) return VF_EINVAL;
  *empty = rows == 0 || heads == 0;
  if (*empty) return VF_OK;
  if (!x || !y || reinterpret_cast<uintptr_t>(x) % esz || reinterpret_cast<uintptr_t>(y) % esz) return VF_EINVAL;
  Axis a[2] = {{y_row, rows}, {y_head, heads}};
  return apart(a, 2, d_head) ? VF_OK : VF_EINVAL;
}

// x used in place of the output: only with the same strides
bool alias_ok(const void* in, int64_t in_row, int64_t in_head, const void* out, int64_t out_row, int64_t out_head, int64_t rows, int64_t heads) {
  return in != out || ((in_row == out_row || rows <= 1) && (in_head == out_head || heads <= 1));
}

int check_shape(const vf_attn_shape* s) {
  if (!s) return VF_EINVAL;
  const size_t esz = size_of(s->dtype);
  if (!esz || s->batch < 0 || s->q_rows < 0 || s->k_rows < 0 || s->q_heads < 1 || s->kv_heads < 1) return VF_EINVAL;
  if (s->q_heads % s->kv_heads || s->d_head < 8 || s->d_head > 128 || s->d_head % 8) return VF_EINVAL;
  if (!(s->scale > 0.f) || !std::isfinite(s->scale)) return VF_EINVAL;
  // rows of a problem are found by a multiplication that is exact below this; problems and tiles of 128 rows are dimensions of
  // a grid, joined rows are counted in 32 bits
  const int64_t group = s->q_heads / s->kv_heads, problems = (int64_t)s->batch * s->kv_heads;
  const int64_t rows = std::max<int64_t>(group * s->q_rows, s->k_rows);
  if (rows > 128 * 65535 || problems > (1 << 23)) return VF_EINVAL;       // (ahead of the products below, which then fit 64 bits)
  if (group * group * s->q_rows > INT32_MAX || problems * rows > INT32_MAX) return VF_EINVAL;
  return VF_OK;
}

bool strides_ok(const vf_attn_layout& l, size_t esz) {
  const int64_t c = 16 / (int64_t)esz;
  return l.batch % c == 0 && l.row % c == 0 && l.head % c == 0;
}
bool output_apart(const vf_attn_layout& l, int64_t batch, int64_t rows, int64_t heads, int64_t dh) {
  Axis a[3] = {{l.batch, batch}, {l.row, rows}, {l.head, heads}};
  return apart(a, 3, dh);
}

int make_job(const vf_attn_shape* s, const void* q, const void* k, const void* v, const int32_t* q_len, const int32_t* k_len,
             const uint8_t* key_mask, AttnJob* j) {
  const size_t esz = size_of(s->dtype);
  if (s->batch > 0 && s->q_rows > 0 && (!q || !aligned16(q))) return VF_EINVAL;
  if (s->batch > 0 && s->k_rows > 0 && (!k || !v || !aligned16(k) || !aligned16(v))) return VF_EINVAL;
  *j = AttnJob{};
  j->s = *s;
  for (vf_attn_layout* l : {&j->s.q, &j->s.o, &j->s.d_o, &j->s.dq}) trim(*l, s->batch, s->q_rows, s->q_heads);
  for (vf_attn_layout* l : {&j->s.k, &j->s.v, &j->s.dk, &j->s.dv}) trim(*l, s->batch, s->k_rows, s->kv_heads);
  if (!strides_ok(j->s.q, esz) || !strides_ok(j->s.k, esz) || !strides_ok(j->s.v, esz) || !strides_ok(j->s.o, esz)) return VF_EINVAL;
  j->group = s->q_heads / s->kv_heads;
  j->group_inv = j->group > 1 ? (uint32_t)((((uint64_t)1 << 32) + j->group - 1) / j->group) : 0;
  j->q = q; j->k = k; j->v = v;
  j->q_len = q_len; j->k_len = k_len; j->key_mask = key_mask;
  return VF_OK;
}

int check_workspace(const vf_attn_shape& s, bool backward, bool masked, const void* ws, int64_t bytes) {
  const int64_t need = attn_workspace_bytes(s, backward, masked);
  return need > 0 && (!ws || !aligned16(ws) || bytes < need) ? VF_EINVAL : VF_OK;
}

}  // namespace

extern "C" {

int vf_rope_make(int32_t layout, int32_t rot_dim, double base, int32_t scaling, double factor, int64_t trained_len,
                 double beta_fast, double beta_slow, double scale, vf_rope_plan* out) {
  if (!out || (layout != VF_ROPE_HALF && layout != VF_ROPE_INTERLEAVED)) return VF_EINVAL;
  if (rot_dim < 2 || rot_dim % 2 || rot_dim > 2 * VF_ROPE_MAX_PAIRS || !(base > 1.0) || !std::isfinite(base) || !(std::fabs(scale) <= FLT_MAX))
    return VF_EINVAL;
  if (scaling != VF_ROPE_PLAIN && scaling != VF_ROPE_LINEAR && scaling != VF_ROPE_PARTS) return VF_EINVAL;
  if (scaling != VF_ROPE_PLAIN && (!(factor > 0.0) || !std::isfinite(factor))) return VF_EINVAL;
  if (scaling == VF_ROPE_PARTS && (trained_len < 1 || !(beta_fast > beta_slow) || !std::isfinite(beta_fast) || !std::isfinite(beta_slow)))
    return VF_EINVAL;
  const double two_pi = 6.283185307179586476925286766559;
  vf_rope_plan plan{};
  plan.layout = layout; plan.rot_dim = rot_dim; plan.scale = (float)scale;
  for (int j = 0; j < rot_dim / 2; ++j) {
    const double f = std::pow(base, -2.0 * j / rot_dim);
    double g = f;
    if (scaling == VF_ROPE_LINEAR) g = f / factor;
    if (scaling == VF_ROPE_PARTS) {
      const double keep = std::min(1.0, std::max(0.0, ((double)trained_len * f / two_pi - beta_slow) / (beta_fast - beta_slow)));
      g = keep * f + (1.0 - keep) * f / factor;
    }
    plan.turns[j] = g / two_pi;
    if (!std::isfinite(plan.turns[j])) return VF_EINVAL;     // (a factor so small that the quotient overflows)
  }
  *out = plan;
  return VF_OK;
}

int vf_rope(int32_t dtype, const void* x, int64_t x_row, int64_t x_head, void* y, int64_t y_row, int64_t y_head, int64_t rows,
            int32_t heads, int32_t d_head, const int32_t* positions, int64_t first, int64_t seq_len, const vf_rope_plan* plan,
            int32_t inverse, void* stream) {
  bool empty;
  if (!plan) return VF_EINVAL;
  VF_TRY(check_heads(dtype, x, y, y_row, y_head, rows, heads, d_head, first, seq_len, plan, &empty));
  if (empty) return VF_OK;
  if (!alias_ok(x, x_row, x_head, y, y_row, y_head, rows, heads)) return VF_EINVAL;
  RopeJob j{};
  j.x = x; j.x_row = stride_of(x_row, rows); j.x_head = stride_of(x_head, heads);
  j.y = y; j.y_row = stride_of(y_row, rows); j.y_head = stride_of(y_head, heads);
  j.rows = rows; j.heads = j.q_heads = heads; j.dh = d_head;
  j.positions = positions; j.first = first; j.seq_len = seq_len;
  use_plan(j, plan, inverse != 0);
  return launch_rope(dtype, j, plan, false, static_cast<hipStream_t>(stream));
}

int vf_qk_norm_rope(int32_t dtype, const void* x, int64_t x_row, int64_t x_head, void* y, int64_t y_row, int64_t y_head,
                    int64_t rows, int32_t q_heads, int32_t k_heads, int32_t d_head, const float* gamma_q, const float* gamma_k,
                    float eps, const int32_t* positions, int64_t first, int64_t seq_len, const vf_rope_plan* plan, void* stream) {
  bool empty;
  if (q_heads < 0 || k_heads < 0 || !(eps >= 0.f && eps <= FLT_MAX)) return VF_EINVAL;
  const int64_t heads = (int64_t)q_heads + k_heads;
  VF_TRY(check_heads(dtype, x, y, y_row, y_head, rows, heads, d_head, first, seq_len, plan, &empty));
  if (empty) return VF_OK;
  if (!alias_ok(x, x_row, x_head, y, y_row, y_head, rows, heads)) return VF_EINVAL;
  RopeJob j{};
  j.x = x; j.x_row = stride_of(x_row, rows); j.x_head = stride_of(x_head, heads);
  j.y = y; j.y_row = stride_of(y_row, rows); j.y_head = stride_of(y_head, heads);
  j.rows = rows; j.heads = (int)heads; j.q_heads = q_heads; j.dh = d_head;
  j.gamma_q = gamma_q; j.gamma_k = gamma_k; j.eps = eps;
  j.positions = positions; j.first = first; j.seq_len = seq_len;
  use_plan(j, plan, false);
  return launch_rope(dtype, j, plan, true, static_cast<hipStream_t>(stream));
}

int64_t vf_qk_norm_rope_workspace(int64_t rows, int32_t q_heads, int32_t k_heads, int32_t d_head) {
  if (rows < 0 || rows > kMaxRows || q_heads < 0 || k_heads < 0 || (int64_t)q_heads + k_heads > kMaxHeads || d_head < 1 || d_head > kMaxHead)
    return VF_EINVAL;
  return rope_partial_floats(rows, q_heads, k_heads, d_head) * (int64_t)sizeof(float);
}

int vf_qk_norm_rope_backward(int32_t dtype, const void* x, int64_t x_row, int64_t x_head, const void* dy, int64_t dy_row,
                             int64_t dy_head, void* dx, int64_t dx_row, int64_t dx_head, int64_t rows, int32_t q_heads,
                             int32_t k_heads, int32_t d_head, const float* gamma_q, const float* gamma_k, float eps,
                             const int32_t* positions, int64_t first, int64_t seq_len, const vf_rope_plan* plan,
                             float* dgamma_q, float* dgamma_k, float alpha, int32_t accumulate, void* workspace,
                             int64_t workspace_bytes, void* stream) {
  bool empty;
  if (q_heads < 0 || k_heads < 0 || !(eps >= 0.f && eps <= FLT_MAX)) return VF_EINVAL;
  const int64_t heads = (int64_t)q_heads + k_heads;
  VF_TRY(check_heads(dtype, x, dx, dx_row, dx_head, rows, heads, d_head, first, seq_len, plan, &empty));
  if (!empty) {
    if (!dy || reinterpret_cast<uintptr_t>(dy) % size_of(dtype)) return VF_EINVAL;
    if (!alias_ok(x, x_row, x_head, dx, dx_row, dx_head, rows, heads) || !alias_ok(dy, dy_row, dy_head, dx, dx_row, dx_head, rows, heads))
      return VF_EINVAL;
  }
  const bool want = dgamma_q || dgamma_k;
  if (want && !empty) {
    const int64_t need = vf_qk_norm_rope_workspace(rows, q_heads, k_heads, d_head);
    if (!workspace || !aligned16(workspace) || workspace_bytes < need) return VF_EINVAL;
  }
  if (dgamma_q && dgamma_q == dgamma_k) return VF_EINVAL;
  RopeJob j{};
  j.x = x; j.x_row = stride_of(x_row, rows); j.x_head = stride_of(x_head, heads);
  j.y = dx; j.y_row = stride_of(dx_row, rows); j.y_head = stride_of(dx_head, heads);
  j.dy = dy; j.dy_row = stride_of(dy_row, rows); j.dy_head = stride_of(dy_head, heads);
  j.rows = empty ? 0 : rows; j.heads = (int)heads; j.q_heads = q_heads; j.dh = d_head;
  j.gamma_q = gamma_q; j.gamma_k = gamma_k; j.eps = eps;
  j.positions = positions; j.first = first; j.seq_len = seq_len;
  j.partial = want ? static_cast<float*>(workspace) : nullptr;
  use_plan(j, plan, true);
  return launch_norm_bwd(dtype, j, plan, dgamma_q, dgamma_k, alpha, accumulate, static_cast<hipStream_t>(stream));
}

int64_t vf_attention_workspace(const vf_attn_shape* shape, int32_t backward) {
  VF_TRY(check_shape(shape));
  return attn_workspace_bytes(*shape, backward != 0, true);
}

int vf_attention(const vf_attn_shape* shape, const void* q, const void* k, const void* v, const int32_t* q_len,
                 const int32_t* k_len, const uint8_t* key_mask, void* o, float* lse, void* workspace, int64_t workspace_bytes,
                 void* stream) {
  VF_TRY(check_shape(shape));
  AttnJob j;
  const vf_attn_shape& s = j.s;
  VF_TRY(make_job(shape, q, k, v, q_len, k_len, key_mask, &j));
  if (s.batch > 0 && s.q_rows > 0 && (!o || !aligned16(o))) return VF_EINVAL;
  if (!output_apart(s.o, s.batch, s.q_rows, s.q_heads, s.d_head) || (o && (o == q || o == k || o == v))) return VF_EINVAL;
  VF_TRY(check_workspace(s, false, key_mask, workspace, workspace_bytes));
  j.o = o; j.lse = lse;
  return launch_attn(j, workspace, static_cast<hipStream_t>(stream));
}

int vf_attention_backward(const vf_attn_shape* shape, const void* q, const void* k, const void* v, const int32_t* q_len,
                          const int32_t* k_len, const uint8_t* key_mask, const void* o, const float* lse, const void* d_o,
                          void* dq, void* dk, void* dv, void* workspace, int64_t workspace_bytes, void* stream) {
  VF_TRY(check_shape(shape));
  const size_t esz = size_of(shape->dtype);
  AttnJob j;
  const vf_attn_shape& s = j.s;
  VF_TRY(make_job(shape, q, k, v, q_len, k_len, key_mask, &j));
  if (!strides_ok(s.d_o, esz) || !strides_ok(s.dq, esz) || !strides_ok(s.dk, esz) || !strides_ok(s.dv, esz)) return VF_EINVAL;
  if (s.batch > 0 && s.q_rows > 0 && (!o || !lse || !d_o || !dq || !aligned16(o) || !aligned16(d_o) || !aligned16(dq))) return VF_EINVAL;
  if (s.batch > 0 && s.k_rows > 0 && (!dk || !dv || !aligned16(dk) || !aligned16(dv))) return VF_EINVAL;
  if (!output_apart(s.dq, s.batch, s.q_rows, s.q_heads, s.d_head) || !output_apart(s.dk, s.batch, s.k_rows, s.kv_heads, s.d_head) ||
      !output_apart(s.dv, s.batch, s.k_rows, s.kv_heads, s.d_head))
    return VF_EINVAL;
  const void* outs[3] = {dq, dk, dv};
  for (int i = 0; i < 3; ++i)                               // (an output is read again, as an input, by other workgroups)
    for (const void* p : {q, k, v, o, d_o, static_cast<const void*>(outs[(i + 1) % 3])})
      if (outs[i] && outs[i] == p) return VF_EINVAL;
  VF_TRY(check_workspace(s, true, key_mask, workspace, workspace_bytes));
  j.o = const_cast<void*>(o); j.lse = const_cast<float*>(lse);
  j.d_o = d_o; j.dq = dq; j.dk = dk; j.dv = dv;
  return launch_attn_bwd(j, workspace, static_cast<hipStream_t>(stream));
}

}  // extern "C"
