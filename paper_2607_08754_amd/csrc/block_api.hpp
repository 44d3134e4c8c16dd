// C ABI of the operators of a regularised block: argument checks, then one
// enqueue (included by api.cpp after its helpers; contract in slorr.h).
#pragma once

namespace {

int32_t check_dtype(int32_t dt) {
  if (dt != SLORR_F32 && dt != SLORR_BF16) throw std::domain_error("unknown dtype");
  return dt;
}

void check_pointer(const void *p, const char *name, bool required = true) {
  if (!p && required) throw std::invalid_argument(std::string(name) + " is NULL");
  if (!aligned(p, 16)) throw std::invalid_argument(std::string(name) + " must be 16-byte aligned");
}

// Buffers of a call: an output may overlap nothing else.
struct Spans {
  struct Span {
    uintptr_t begin, end;
    bool out;
    const char *name;
  };
  Span s[24];
  int n = 0;
  void add(const void *p, size_t bytes, bool out, const char *name) {
    if (!p || !bytes) return;
    const uintptr_t b = reinterpret_cast<uintptr_t>(p);
    s[n++] = {b, b + bytes, out, name};
  }
  void in(const void *p, size_t bytes, const char *name) { add(p, bytes, false, name); }
  void out(const void *p, size_t bytes, const char *name) { add(p, bytes, true, name); }
  void check() const {
    for (int i = 0; i < n; ++i)
      for (int j = i + 1; j < n; ++j)
        if ((s[i].out || s[j].out) && s[i].begin < s[j].end && s[j].begin < s[i].end)
          throw std::invalid_argument(std::string(s[i].name) + " and " + s[j].name + " overlap");
  }
};

void check_workspace(const void *ws, size_t have, size_t need) {
  if (!ws) throw ApiError{SLORR_ERR_WORKSPACE, "workspace pointer is NULL"};
  if (!aligned(ws, 256)) throw ApiError{SLORR_ERR_WORKSPACE, "workspace must be 256-byte aligned"};
  if (have < need)
    throw ApiError{SLORR_ERR_WORKSPACE,
                   "workspace too small: need " + std::to_string(need) + " bytes, got " + std::to_string(have)};
}

// bytes of `rows` rows of `width` values, ld apart
size_t span_bytes(int64_t rows, int64_t width, int64_t ld, size_t es) {
  return rows > 0 ? size_t((rows - 1) * ld + width) * es : 0;
}

slorr::FfnShape ffn_shape(const slorr_ffn_t *d) {
  if (!d) throw std::invalid_argument("block is NULL");
  slorr::FfnShape s{};
  s.dtype = check_dtype(bits(d->dtype));
  s.act = bits(d->act);
  if (s.act != SLORR_SILU && s.act != SLORR_GELU && s.act != SLORR_GELU_TANH) throw std::domain_error("unknown act");
  s.tokens = d->tokens;
  s.dim = d->dim;
  s.inner = d->inner;
  if (s.tokens < 0) throw std::invalid_argument("tokens must be >= 0");
  if (s.dim < 1 || s.inner < 1) throw std::invalid_argument("dim and inner must be >= 1");
  if (s.tokens > slorr::kMaxTokens || s.dim > slorr::kMaxWidth || s.inner > slorr::kMaxWidth)
    throw std::domain_error("tokens, dim or inner beyond the limits");
  if ((s.tokens / 128 + 1) * (std::max(s.dim, s.inner) / 64 + 1) > (int64_t(1) << 30))
    throw std::domain_error("tokens times width beyond the limit");
  s.ldx = d->ldx ? d->ldx : s.dim;
  s.lddy = d->lddy ? d->lddy : s.dim;
  if (s.ldx < s.dim || s.lddy < s.dim) throw std::invalid_argument("a row stride is below dim");
  if (s.ldx > slorr::kMaxStride || s.lddy > slorr::kMaxStride) throw std::domain_error("a row stride is beyond the limit");
  return s;
}

struct JoinCall {
  slorr::JoinShape s;
  slorr_join_tensors_t t;
  size_t es, row_bytes, vec_bytes;
};

uint32_t drop_threshold(double p) {
  if (!(p >= 0.0 && p < 1.0)) throw std::invalid_argument("p must be in [0, 1)");
  const double t = std::nearbyint(p * 65536.0);
  if (t >= 65536.0) throw std::invalid_argument("p rounds to 1");
  return uint32_t(t);
}

void check_rng(const int64_t *rng, uint32_t drop) {
  if (drop && !rng) throw std::invalid_argument("rng is NULL");
  if (!aligned(rng, 8)) throw std::invalid_argument("rng must be 8-byte aligned");
}

slorr::JoinShape join_shape(const slorr_join_t *d) {
  if (!d) throw std::invalid_argument("join is NULL");
  slorr::JoinShape s{};
  s.dtype = check_dtype(bits(d->dtype));
  const int32_t norm = bits(d->norm);
  if (norm != SLORR_RMS && norm != SLORR_LAYER) throw std::domain_error("unknown norm");
  if (d->flags & ~(SLORR_JOIN_POST | SLORR_JOIN_PRE)) throw std::invalid_argument("unknown flags");
  s.layer = norm == SLORR_LAYER;
  s.post = (d->flags & SLORR_JOIN_POST) != 0;
  s.pre = (d->flags & SLORR_JOIN_PRE) != 0;
  s.rows = d->rows;
  s.dim = d->dim;
  if (s.rows < 0) throw std::invalid_argument("rows must be >= 0");
  if (s.dim < 1) throw std::invalid_argument("dim must be >= 1");
  if (s.dim > slorr::kMaxNorm || s.rows > (int64_t(1) << 40)) throw std::domain_error("rows or dim beyond the limits");
  s.ldx = d->ldx ? d->ldx : s.dim;
  s.ldf = d->ldf ? d->ldf : s.dim;
  s.ld_gate = d->ld_gate ? d->ld_gate : s.dim;
  if (s.ldx < s.dim || s.ldf < s.dim || s.ld_gate < s.dim) throw std::invalid_argument("a row stride is below dim");
  if (std::max({s.ldx, s.ldf, s.ld_gate}) > slorr::kMaxStride) throw std::domain_error("a row stride is beyond the limit");
  if (s.rows > (int64_t(1) << 50) / std::max({s.ldx, s.ldf, s.ld_gate})) throw std::domain_error("rows times stride beyond the limit");
  s.gate_rows = d->gate_rows;
  if (!(d->eps >= 0.0f) || std::isinf(d->eps)) throw std::invalid_argument("eps must be >= 0 and finite");
  if (!std::isfinite(d->alpha)) throw std::invalid_argument("alpha must be finite");
  s.eps = d->eps;
  s.alpha = d->alpha;
  s.drop = drop_threshold(d->p);
  s.site = d->site;
  return s;
}

JoinCall join_call(const slorr_join_t *d, const slorr_join_tensors_t *in, const int64_t *rng) {
  JoinCall c{join_shape(d), {}, 0, 0, 0};
  slorr::JoinShape &s = c.s;
  if (!in) throw std::invalid_argument("in is NULL");
  c.t = *in;
  c.es = s.dtype == SLORR_F32 ? 4 : 2;
  c.row_bytes = size_t(s.rows) * size_t(s.dim) * c.es;
  c.vec_bytes = size_t(s.dim) * c.es;
  check_pointer(in->x, "x", s.rows > 0);
  const struct {
    const void *p;
    const char *name;
  } opt[] = {{in->f, "f"}, {in->post_weight, "post_weight"}, {in->post_bias, "post_bias"}, {in->gate, "gate"},
             {in->scale, "scale"}, {in->pre_weight, "pre_weight"}, {in->pre_bias, "pre_bias"}};
  for (const auto &o : opt) check_pointer(o.p, o.name, false);
  if (!s.post && (in->post_weight || in->post_bias)) throw std::invalid_argument("post_weight or post_bias without POST");
  if (!s.pre && (in->pre_weight || in->pre_bias)) throw std::invalid_argument("pre_weight or pre_bias without PRE");
  const bool f = in->f || !s.rows;          // (no rows: an empty f may be NULL)
  if (!f && (s.post || in->gate || in->scale)) throw std::invalid_argument("POST, gate or scale without f");
  if (!f && !s.pre) throw std::invalid_argument("neither f nor PRE: nothing to do");
  if (in->gate) {
    if (s.gate_rows < 1 || s.rows % s.gate_rows) throw std::invalid_argument("gate_rows must divide rows");
  } else {
    s.gate_rows = 0;
  }
  if (!f) s.drop = 0;
  check_rng(rng, s.drop);
  return c;
}

void join_spans(const JoinCall &c, const int64_t *rng, Spans &sp) {
  const slorr::JoinShape &s = c.s;
  sp.in(c.t.x, span_bytes(s.rows, s.dim, s.ldx, c.es), "x");
  sp.in(c.t.f, span_bytes(s.rows, s.dim, s.ldf, c.es), "f");
  sp.in(c.t.gate, span_bytes(s.gate_rows, s.dim, s.ld_gate, c.es), "gate");
  sp.in(c.t.post_weight, c.vec_bytes, "post_weight");
  sp.in(c.t.post_bias, c.vec_bytes, "post_bias");
  sp.in(c.t.scale, c.vec_bytes, "scale");
  sp.in(c.t.pre_weight, c.vec_bytes, "pre_weight");
  sp.in(c.t.pre_bias, c.vec_bytes, "pre_bias");
  sp.in(rng, rng ? 16 : 0, "rng");
}

}  // namespace

extern "C" {

slorr_status_t slorr_ffn_sizes(const slorr_ffn_t *block, size_t *state_bytes, size_t *forward_bytes,
                               size_t *backward_bytes) {
  return guarded([&]() -> slorr_status_t {
    const slorr::FfnShape s = ffn_shape(block);
    if (state_bytes) *state_bytes = slorr::ffn_state_bytes(s);
    if (forward_bytes) *forward_bytes = slorr::ffn_layout(s, false).bytes;
    if (backward_bytes) *backward_bytes = slorr::ffn_layout(s, true).bytes;
    return SLORR_OK;
  });
}

slorr_status_t slorr_ffn_forward(const slorr_ffn_t *block, const void *x, const void *w_gate, const void *w_up,
                                 const void *w_down, void *y, void *state, void *workspace, size_t workspace_bytes,
                                 void *stream) {
  return guarded([&]() -> slorr_status_t {
    const slorr::FfnShape s = ffn_shape(block);
    const bool any = s.tokens > 0;
    check_pointer(x, "x", any);
    check_pointer(w_gate, "w_gate");
    check_pointer(w_up, "w_up");
    check_pointer(w_down, "w_down");
    check_pointer(y, "y", any);
    check_pointer(state, "state", false);
    const size_t need = slorr::ffn_layout(s, false).bytes, w = size_t(s.dim) * size_t(s.inner) * s.elem();
    check_workspace(workspace, workspace_bytes, need);
    Spans sp;
    sp.in(x, span_bytes(s.tokens, s.dim, s.ldx, s.elem()), "x");
    sp.in(w_gate, w, "w_gate");
    sp.in(w_up, w, "w_up");
    sp.in(w_down, w, "w_down");
    sp.out(y, span_bytes(s.tokens, s.dim, s.dim, s.elem()), "y");
    sp.out(state, any ? slorr::ffn_state_bytes(s) : 0, "state");
    sp.out(workspace, need, "workspace");
    sp.check();
    slorr::enqueue_ffn_forward(s, x, w_gate, w_up, w_down, y, state, workspace, static_cast<hipStream_t>(stream));
    return SLORR_OK;
  });
}

slorr_status_t slorr_ffn_backward(const slorr_ffn_t *block, const void *dy, const void *x, const void *w_gate,
                                  const void *w_up, const void *w_down, const void *state, void *dx, void *dw_gate,
                                  void *dw_up, void *dw_down, void *workspace, size_t workspace_bytes, void *stream) {
  return guarded([&]() -> slorr_status_t {
    const slorr::FfnShape s = ffn_shape(block);
    const bool any = s.tokens > 0;
    check_pointer(dy, "dy", any);
    check_pointer(x, "x", any);
    check_pointer(w_gate, "w_gate");
    check_pointer(w_up, "w_up");
    check_pointer(w_down, "w_down");
    check_pointer(state, "state", any);
    check_pointer(dx, "dx", false);
    check_pointer(dw_gate, "dw_gate", false);
    check_pointer(dw_up, "dw_up", false);
    check_pointer(dw_down, "dw_down", false);
    const size_t need = slorr::ffn_layout(s, true).bytes, w = size_t(s.dim) * size_t(s.inner) * s.elem();
    check_workspace(workspace, workspace_bytes, need);
    Spans sp;
    sp.in(dy, span_bytes(s.tokens, s.dim, s.lddy, s.elem()), "dy");
    sp.in(x, span_bytes(s.tokens, s.dim, s.ldx, s.elem()), "x");
    sp.in(w_gate, w, "w_gate");
    sp.in(w_up, w, "w_up");
    sp.in(w_down, w, "w_down");
    sp.in(state, any ? slorr::ffn_state_bytes(s) : 0, "state");
    sp.out(dx, span_bytes(s.tokens, s.dim, s.dim, s.elem()), "dx");
    sp.out(dw_gate, w, "dw_gate");
    sp.out(dw_up, w, "dw_up");
    sp.out(dw_down, w, "dw_down");
    sp.out(workspace, need, "workspace");
    sp.check();
    if (!dx && !dw_gate && !dw_up && !dw_down) return SLORR_OK;
    slorr::enqueue_ffn_backward(s, dy, x, w_gate, w_up, w_down, state, dx, dw_gate, dw_up, dw_down, workspace,
                                static_cast<hipStream_t>(stream));
    return SLORR_OK;
  });
}

slorr_status_t slorr_join_forward(const slorr_join_t *join, const slorr_join_tensors_t *in, const int64_t *rng,
                                  void *y, void *z, void *stream) {
  return guarded([&]() -> slorr_status_t {
    const JoinCall c = join_call(join, in, rng);
    const bool any = c.s.rows > 0;
    check_pointer(y, "y", any && (c.t.f || !c.s.pre));
    check_pointer(z, "z", any && c.s.pre);
    if (!c.s.pre && z) throw std::invalid_argument("z without PRE");
    Spans sp;
    join_spans(c, rng, sp);
    sp.out(y, c.row_bytes, "y");
    sp.out(z, c.row_bytes, "z");
    sp.check();
    slorr::enqueue_join_forward(c.s, c.t, rng, y, z, static_cast<hipStream_t>(stream));
    return SLORR_OK;
  });
}

slorr_status_t slorr_join_workspace(const slorr_join_t *join, size_t *bytes) {
  return guarded([&]() -> slorr_status_t {
    if (!bytes) throw std::invalid_argument("bytes is NULL");
    slorr::JoinShape s = join_shape(join);
    if (s.gate_rows < 0 || (s.gate_rows > 0 && s.rows % s.gate_rows)) throw std::invalid_argument("gate_rows must divide rows");
    // (a call without gate cuts its rows as one group)
    const size_t with = slorr::join_workspace(s);
    s.gate_rows = 0;
    *bytes = std::max(with, slorr::join_workspace(s));
    return SLORR_OK;
  });
}

slorr_status_t slorr_join_backward(const slorr_join_t *join, const slorr_join_tensors_t *in, const int64_t *rng,
                                   const void *dy, const void *dz, const slorr_join_grads_t *grads, void *workspace,
                                   size_t workspace_bytes, void *stream) {
  return guarded([&]() -> slorr_status_t {
    const JoinCall c = join_call(join, in, rng);
    if (!grads) throw std::invalid_argument("grads is NULL");
    const slorr_join_grads_t &g = *grads;
    check_pointer(dy, "dy", false);
    check_pointer(dz, "dz", false);
    if (!c.s.pre && dz) throw std::invalid_argument("dz without PRE");
    const struct {
      void *g;
      const void *t;
      const char *name;
      size_t bytes;
    } out[] = {{g.x, c.t.x, "the gradient of x", c.row_bytes},
               {g.f, c.t.f, "the gradient of f", c.row_bytes},
               {g.post_weight, c.t.post_weight, "the gradient of post_weight", c.vec_bytes},
               {g.post_bias, c.t.post_bias, "the gradient of post_bias", c.vec_bytes},
               {g.gate, c.t.gate, "the gradient of gate", size_t(c.s.gate_rows) * c.vec_bytes},
               {g.scale, c.t.scale, "the gradient of scale", c.vec_bytes},
               {g.pre_weight, c.t.pre_weight, "the gradient of pre_weight", c.vec_bytes},
               {g.pre_bias, c.t.pre_bias, "the gradient of pre_bias", c.vec_bytes}};
    const size_t need = slorr::join_workspace(c.s);
    check_workspace(workspace, workspace_bytes, need);
    Spans sp;
    join_spans(c, rng, sp);
    sp.in(dy, c.row_bytes, "dy");
    sp.in(dz, c.row_bytes, "dz");
    for (const auto &o : out) {
      check_pointer(o.g, o.name, false);
      if (o.g && !o.t && c.s.rows > 0)
        throw std::invalid_argument(std::string(o.name) + " is asked for without the input");
      sp.out(o.g, o.bytes, o.name);
    }
    sp.out(workspace, need, "workspace");
    sp.check();
    slorr::enqueue_join_backward(c.s, c.t, rng, dy, dz, g, workspace, static_cast<hipStream_t>(stream));
    return SLORR_OK;
  });
}

slorr_status_t slorr_dropout(int64_t n, slorr_dtype_t dtype, double p, const int64_t *rng, int64_t site,
                             const void *x, void *y, void *stream) {
  return guarded([&]() -> slorr_status_t {
    const int32_t dt = check_dtype(bits(dtype));
    if (n < 0) throw std::invalid_argument("n must be >= 0");
    if (n > int64_t(1) << 50) throw std::domain_error("n beyond the limit");
    const uint32_t drop = drop_threshold(p);
    check_pointer(x, "x", n > 0);
    check_pointer(y, "y", n > 0);
    check_rng(rng, drop);
    const size_t bytes = size_t(n) * (dt == SLORR_F32 ? 4 : 2);
    Spans sp;
    if (x != y) sp.in(x, bytes, "x");
    sp.out(y, bytes, "y");
    sp.in(rng, rng ? 16 : 0, "rng");
    sp.check();
    slorr::enqueue_dropout(n, dt, drop, rng, site, x, y, static_cast<hipStream_t>(stream));
    return SLORR_OK;
  });
}

}  // extern "C"
