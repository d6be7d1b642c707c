// Python binding of the layers of experts, their router and exchange, and the
// distillation loss.  A part of bind_layers.cpp.
#pragma once

namespace {

struct {
  occ_status_t (*fwd[2])(const occ_experts_t*, void*, size_t, occ_stream_t);
  occ_status_t (*bwd[2])(const occ_experts_grad_t*, uint32_t, void*, size_t, occ_stream_t);
  size_t (*fwd_size[2])(const occ_experts_t*);
  size_t (*bwd_size[2])(const occ_experts_grad_t*);
  decltype(&occ_route_fwd) route_fwd;
  decltype(&occ_route_fwd_workspace_bytes) route_size;
  decltype(&occ_route_bwd) route_bwd;
  decltype(&occ_dispatch) dispatch;
  decltype(&occ_combine) combine;
  decltype(&occ_combine_bwd) combine_bwd;
  decltype(&occ_distill_fwd) distill[2];   // forward, backward
} more;

// n contiguous values of a type, or of any number (n < 0).
template <class T>
T* values(const Call& c, const at::Tensor* t, const char* name, at::ScalarType type, int64_t n) {
  if (!t) return nullptr;
  if (t->scalar_type() != type) {
    PyErr_Format(PyExc_TypeError, "%s must be %s", name, at::toString(type));
    throw Refused{};
  }
  if ((n >= 0 && t->numel() != n) || !t->is_contiguous()) {
    PyErr_Format(PyExc_ValueError, "%s must hold %lld contiguous values", name, (long long)(n < 0 ? t->numel() : n));
    throw Refused{};
  }
  if (t->device() != c.device) refuse(PyExc_ValueError, "%s lies on another device", name);
  return (T*)t->data_ptr();
}

int32_t* whole(const Call& c, const at::Tensor* t, const char* name, int64_t n) {
  return values<int32_t>(c, t, name, at::kInt, n);
}

uint32_t* flag_word(const Call& c, PyObject* o) { return (uint32_t*)whole(c, tensor(o, "flags"), "flags", 1); }

const at::Tensor& given(const at::Tensor* t, const char* name) {
  if (!t) refuse(PyExc_ValueError, "%s must be given", name);
  return *t;
}

// A matrix of every expert: experts x rows x cols, any strides but the last.
void* stack(const Call& c, const at::Tensor* t, const char* name, int64_t experts, int64_t rows, int64_t cols,
            at::ScalarType dt, int64_t& ld, int64_t& stride) {
  ld = cols;
  stride = rows * cols;
  if (!t) return nullptr;
  if (t->scalar_type() != dt) {
    PyErr_Format(PyExc_TypeError, "%s must be %s", name, at::toString(dt));
    throw Refused{};
  }
  if (t->dim() != 3 || t->size(0) != experts || t->size(1) != rows || t->size(2) != cols) {
    PyErr_Format(PyExc_ValueError, "%s must be %lld x %lld x %lld", name, (long long)experts, (long long)rows,
                 (long long)cols);
    throw Refused{};
  }
  if (cols > 1 && t->stride(2) != 1) refuse(PyExc_ValueError, "%s must have unit column stride (row-major)", name);
  if (t->device() != c.device) refuse(PyExc_ValueError, "%s lies on another device", name);
  if (rows > 1) ld = t->stride(1);
  stride = experts > 1 ? t->stride(0) : rows * ld;
  return t->data_ptr();
}

const at::Tensor& three(const at::Tensor* t, const char* name) {
  if (!t || t->dim() != 3) refuse(PyExc_ValueError, "%s must be 3-D", name);
  return *t;
}

int64_t experts_of(const at::Tensor& offsets) {
  if (offsets.dim() != 1 || offsets.numel() < 2) refuse(PyExc_ValueError, "%s must hold one more value than experts", "offsets");
  return offsets.numel() - 1;
}

// experts_forward(gated, X, W, offsets, bias, act, R, Y, Z, flags, ws) -> status
PyObject* experts_forward(PyObject*, PyObject* const* v, Py_ssize_t n) {
  if (!count(n, 11)) return nullptr;
  return guarded([&] {
    const bool gated = v[0] == Py_True;
    const at::Tensor &X = matrix(tensor(v[1], "X"), "X"), &W = three(tensor(v[2], "W"), "W");
    const at::Tensor& offsets = given(tensor(v[3], "offsets"), "offsets");
    const int64_t tokens = X.size(0), in = X.size(1), rows = W.size(1), out = gated ? rows / 2 : rows;
    if (gated && rows % 2) refuse(PyExc_ValueError, "%s must hold the rows of both projections", "W");
    occ_experts_t p;
    occ_linear_t& a = p.l;
    a.dtype = layer_type(X, "X");
    a.act = activation(v[5]);
    const Call c{X.scalar_type(), X.device()};
    a.tokens = tokens;
    a.in = in;
    a.out = out;
    p.experts = experts_of(offsets);
    p.offsets = whole(c, &offsets, "offsets", -1);
    a.X = c(&X, "X", tokens, in, a.ldx);
    a.W = stack(c, &W, "W", p.experts, rows, in, c.dtype, a.ldw, p.stride_w);
    a.bias = values<float>(c, tensor(v[4], "bias"), "bias", at::kFloat, p.experts * rows);
    a.R = c(tensor(v[6], "R"), "R", tokens, out, a.ldr);
    a.Y = c(tensor(v[7], "Y"), "Y", tokens, out, a.ldy);
    a.Z = c(tensor(v[8], "Z"), "Z", tokens, rows, a.ldz);
    p.flags = flag_word(c, v[9]);
    const at::Tensor* const space = c.workspace(tensor(v[10], "ws"), "ws");
    const occ_stream_t s = c.stream();
    const c10::DeviceGuard current(c.device);
    const Workspace ws(more.fwd_size[gated](&p), space, c.device);
    return PyLong_FromLong(more.fwd[gated](&p, ws.p, ws.bytes, s));
  });
}

// experts_backward(gated, dY, X, W, offsets, Z, act, dX, dW, dbias, accumulate, flags, ws) -> status
PyObject* experts_backward(PyObject*, PyObject* const* v, Py_ssize_t n) {
  if (!count(n, 13)) return nullptr;
  return guarded([&]() -> PyObject* {
    const bool gated = v[0] == Py_True;
    const at::Tensor &dY = matrix(tensor(v[1], "dY"), "dY"), &offsets = given(tensor(v[4], "offsets"), "offsets");
    const at::Tensor *X = tensor(v[2], "X"), *W = tensor(v[3], "W"), *Z = tensor(v[5], "Z"), *dX = tensor(v[7], "dX"),
                     *dW = tensor(v[8], "dW"), *dbias = tensor(v[9], "dbias");
    const int64_t tokens = dY.size(0), out = dY.size(1), rows = gated ? 2 * out : out;
    const int64_t in = X ? matrix(X, "X").size(1) : dX ? matrix(dX, "dX").size(1)
                         : W ? three(W, "W").size(2) : dW ? three(dW, "dW").size(2) : 1;
    if (tokens == 0 && dX && !dW && !dbias) return PyLong_FromLong(OCC_OK);   // an empty dX
    occ_experts_grad_t p;
    occ_linear_grad_t& a = p.l;
    a.dtype = layer_type(dY, "dY");
    const Call c{dY.scalar_type(), dY.device()};
    const at::ScalarType wide = dW && dW->scalar_type() == at::kFloat ? at::kFloat : c.dtype;
    a.dw_dtype = wide == at::kFloat ? OCC_F32 : OCC_BF16;
    a.act = activation(v[6]);
    const uint32_t call = v[10] == Py_True ? OCC_GRAD_ACCUMULATE : 0;
    a.reserved = 0;
    a.tokens = tokens;
    a.in = in;
    a.out = out;
    p.experts = experts_of(offsets);
    p.offsets = whole(c, &offsets, "offsets", -1);
    a.dY = c(&dY, "dY", tokens, out, a.lddy);
    a.X = c(X, "X", tokens, in, a.ldx);
    a.W = stack(c, W, "W", p.experts, rows, in, c.dtype, a.ldw, p.stride_w);
    a.Z = c(Z, "Z", tokens, rows, a.ldz);
    a.dX = c(dX, "dX", tokens, in, a.lddx);
    a.dW = stack(c, dW, "dW", p.experts, rows, in, wide, a.lddw, p.stride_dw);
    a.dbias = values<float>(c, dbias, "dbias", at::kFloat, p.experts * rows);
    p.flags = flag_word(c, v[11]);
    const at::Tensor* const space = c.workspace(tensor(v[12], "ws"), "ws");
    const occ_stream_t s = c.stream();
    const c10::DeviceGuard current(c.device);
    const Workspace ws(more.bwd_size[gated](&p), space, c.device);
    return PyLong_FromLong(more.bwd[gated](&p, call, ws.p, ws.bytes, s));
  });
}

PyObject* with_tensors(int status, std::initializer_list<at::Tensor> made) {
  PyObject* const t = PyTuple_New(1 + (Py_ssize_t)made.size());
  if (!t) throw Refused{};
  PyTuple_SET_ITEM(t, 0, PyLong_FromLong(status));
  Py_ssize_t i = 1;
  for (const at::Tensor& x : made) {
    PyObject* const o = x.defined() ? THPVariable_Wrap(x) : Py_NewRef(Py_None);
    PyTuple_SET_ITEM(t, i++, o);
    if (!o) {
      Py_DECREF(t);
      throw Refused{};
    }
  }
  return t;
}

// The tensor given, or a new one.
at::Tensor given_or(const at::Tensor* t, const Call& c, at::ScalarType type, at::IntArrayRef size) {
  return t ? *t : at::empty(size, at::TensorOptions().dtype(type).device(c.device));
}

int32_t number(PyObject* o) {
  const long x = PyLong_AsLong(o);
  if (x == -1 && PyErr_Occurred()) throw Refused{};
  return x == (int32_t)x ? (int32_t)x : -1;
}

// route_forward(logits, k, renorm, index, weights, offsets, order, slots, ws)
//   -> (status, index, weights, offsets, order, slots)
PyObject* route_forward(PyObject*, PyObject* const* v, Py_ssize_t n) {
  if (!count(n, 9)) return nullptr;
  return guarded([&] {
    const at::Tensor& logits = matrix(tensor(v[0], "logits"), "logits");
    occ_route_t r;
    r.dtype = layer_type(logits, "logits");
    r.k = number(v[1]);
    if (r.k < 1 || r.k > OCC_MAX_CHOICES) refuse(PyExc_ValueError, "%s is out of range", "k");
    r.renorm = v[2] == Py_True;
    r.reserved = 0;
    r.tokens = logits.size(0);
    r.experts = logits.size(1);
    const int64_t all = r.tokens * r.k;
    const Call c{logits.scalar_type(), logits.device()};
    r.logits = c(&logits, "logits", r.tokens, r.experts, r.ldl);
    const occ_stream_t s = c.stream();
    const c10::DeviceGuard current(c.device);
    const at::Tensor index = given_or(tensor(v[3], "index"), c, at::kInt, {r.tokens, r.k}),
                     weights = given_or(tensor(v[4], "weights"), c, at::kFloat, {r.tokens, r.k}),
                     offsets = given_or(tensor(v[5], "offsets"), c, at::kInt, {r.experts + 1}),
                     order = given_or(tensor(v[6], "order"), c, at::kInt, {all}),
                     slots = given_or(tensor(v[7], "slots"), c, at::kInt, {r.tokens, r.k});
    r.index = whole(c, &index, "index", all);
    r.weights = values<float>(c, &weights, "weights", at::kFloat, all);
    r.offsets = whole(c, &offsets, "offsets", r.experts + 1);
    r.order = whole(c, &order, "order", all);
    r.slots = whole(c, &slots, "slots", all);
    const at::Tensor* const space = c.workspace(tensor(v[8], "ws"), "ws");
    const Workspace ws(more.route_size(&r), space, c.device);
    const int status = more.route_fwd(&r, ws.p, ws.bytes, s);
    return with_tensors(status, {index, weights, offsets, order, slots});
  });
}

// route_backward(dweights, logits, index, weights, renorm, dlogits) -> (status, dlogits)
PyObject* route_backward(PyObject*, PyObject* const* v, Py_ssize_t n) {
  if (!count(n, 6)) return nullptr;
  return guarded([&] {
    const at::Tensor &logits = matrix(tensor(v[1], "logits"), "logits"), &index = matrix(tensor(v[2], "index"), "index");
    occ_route_t r{};
    r.dtype = layer_type(logits, "logits");
    r.k = (int32_t)index.size(1);
    r.renorm = v[4] == Py_True;
    r.tokens = logits.size(0);
    r.experts = logits.size(1);
    const int64_t all = r.tokens * r.k;
    const Call c{logits.scalar_type(), logits.device()};
    r.logits = c(&logits, "logits", r.tokens, r.experts, r.ldl);
    r.index = whole(c, &index, "index", all);
    r.weights = values<float>(c, &given(tensor(v[3], "weights"), "weights"), "weights", at::kFloat, all);
    const float* const dw = values<float>(c, &given(tensor(v[0], "dweights"), "dweights"), "dweights", at::kFloat, all);
    const occ_stream_t s = c.stream();
    const c10::DeviceGuard current(c.device);
    const at::Tensor dlogits = given_or(tensor(v[5], "dlogits"), c, c.dtype, {r.tokens, r.experts});
    int64_t ldd;
    void* const d = c(&dlogits, "dlogits", r.tokens, r.experts, ldd);
    return with_tensors(more.route_bwd(&r, dw, d, ldd, s), {dlogits});
  });
}

occ_exchange_t exchange(const at::Tensor& rows, const at::Tensor& slots, const char* name) {
  occ_exchange_t x{};
  x.dtype = layer_type(rows, name);
  x.k = (int32_t)matrix(&slots, "slots").size(1);
  x.experts = 1;
  x.width = rows.size(1);
  return x;
}

// dispatch(X, offsets, order, slots, Xs, flags) -> (status, Xs)
PyObject* dispatch(PyObject*, PyObject* const* v, Py_ssize_t n) {
  if (!count(n, 6)) return nullptr;
  return guarded([&] {
    const at::Tensor& X = matrix(tensor(v[0], "X"), "X");
    const at::Tensor &offsets = given(tensor(v[1], "offsets"), "offsets"), &order = given(tensor(v[2], "order"), "order"),
                     &slots = given(tensor(v[3], "slots"), "slots");
    occ_exchange_t x = exchange(X, slots, "X");
    const Call c{X.scalar_type(), X.device()};
    x.tokens = X.size(0);
    if (slots.size(0) != x.tokens) refuse(PyExc_ValueError, "%s must have a row for each token", "slots");
    x.experts = experts_of(offsets);
    x.rows = order.numel();
    x.offsets = whole(c, &offsets, "offsets", -1);
    x.order = whole(c, &order, "order", -1);
    x.flags = flag_word(c, v[5]);
    const occ_stream_t s = c.stream();
    const c10::DeviceGuard current(c.device);
    const at::Tensor Xs = given_or(tensor(v[4], "Xs"), c, c.dtype, {x.rows, x.width});
    int64_t ldx, ldxs;
    void* const in = c(&X, "X", x.tokens, x.width, ldx);
    void* const out = c(&Xs, "Xs", x.rows, x.width, ldxs);
    return with_tensors(more.dispatch(&x, in, ldx, out, ldxs, s), {Xs});
  });
}

// combine(Ys, slots, weights, R, Y, flags) -> (status, Y)
PyObject* combine(PyObject*, PyObject* const* v, Py_ssize_t n) {
  if (!count(n, 6)) return nullptr;
  return guarded([&] {
    const at::Tensor &Ys = matrix(tensor(v[0], "Ys"), "Ys"), &slots = given(tensor(v[1], "slots"), "slots");
    occ_exchange_t x = exchange(Ys, slots, "Ys");
    const Call c{Ys.scalar_type(), Ys.device()};
    x.tokens = slots.size(0);
    x.rows = Ys.size(0);
    x.slots = whole(c, &slots, "slots", -1);
    x.flags = flag_word(c, v[5]);
    const float* const w = values<float>(c, tensor(v[2], "weights"), "weights", at::kFloat, x.tokens * x.k);
    const occ_stream_t s = c.stream();
    const c10::DeviceGuard current(c.device);
    const at::Tensor Y = given_or(tensor(v[4], "Y"), c, c.dtype, {x.tokens, x.width});
    int64_t ldys, ldr, ldy;
    void* const in = c(&Ys, "Ys", x.rows, x.width, ldys);
    void* const R = c(tensor(v[3], "R"), "R", x.tokens, x.width, ldr);
    void* const out = c(&Y, "Y", x.tokens, x.width, ldy);
    return with_tensors(more.combine(&x, w, in, ldys, R, ldr, out, ldy, s), {Y});
  });
}

// combine_backward(dY, Ys, order, slots, weights, dYs, dweights, flags) -> (status, dYs, dweights)
PyObject* combine_backward(PyObject*, PyObject* const* v, Py_ssize_t n) {
  if (!count(n, 8)) return nullptr;
  return guarded([&] {
    const at::Tensor& dY = matrix(tensor(v[0], "dY"), "dY");
    const at::Tensor *Ys = tensor(v[1], "Ys"), *dw = tensor(v[6], "dweights");
    const at::Tensor &order = given(tensor(v[2], "order"), "order"), &slots = given(tensor(v[3], "slots"), "slots");
    occ_exchange_t x = exchange(dY, slots, "dY");
    const Call c{dY.scalar_type(), dY.device()};
    x.tokens = dY.size(0);
    if (slots.size(0) != x.tokens) refuse(PyExc_ValueError, "%s must have a row for each token", "slots");
    if (dw && !Ys) refuse(PyExc_ValueError, "%s needs Ys", "dweights");
    x.rows = order.numel();
    x.order = whole(c, &order, "order", -1);
    x.slots = whole(c, &slots, "slots", -1);
    x.flags = flag_word(c, v[7]);
    const float* const w = values<float>(c, tensor(v[4], "weights"), "weights", at::kFloat, x.tokens * x.k);
    const occ_stream_t s = c.stream();
    const c10::DeviceGuard current(c.device);
    const at::Tensor dYs = given_or(tensor(v[5], "dYs"), c, c.dtype, {x.rows, x.width});
    const at::Tensor dweights = Ys ? given_or(dw, c, at::kFloat, {x.tokens, x.k}) : at::Tensor();
    int64_t lddy, ldys, lddys;
    void* const in = c(&dY, "dY", x.tokens, x.width, lddy);
    void* const ys = c(Ys, "Ys", x.rows, x.width, ldys);
    void* const out = c(&dYs, "dYs", x.rows, x.width, lddys);
    float* const d = Ys ? values<float>(c, &dweights, "dweights", at::kFloat, x.tokens * x.k) : nullptr;
    // no rows, and so nothing to write but zeros
    const int status = out || d ? more.combine_bwd(&x, w, in, lddy, ys, ldys, out, lddys, d, s) : OCC_OK;
    return with_tensors(status, {dYs, dweights});
  });
}

float real(PyObject* o) {
  const double x = PyFloat_AsDouble(o);
  if (x == -1.0 && PyErr_Occurred()) throw Refused{};
  return (float)x;
}

// distill(backward, S, index, teacher, labels, scale, temperature, alpha, loss, lse, dS, flags)
//   -> (status, loss, dS)
PyObject* distill(PyObject*, PyObject* const* v, Py_ssize_t n) {
  if (!count(n, 12)) return nullptr;
  return guarded([&] {
    const bool backward = v[0] == Py_True;
    const at::Tensor& S = matrix(tensor(v[1], "S"), "S");
    const at::Tensor *index = tensor(v[2], "index"), *teacher = tensor(v[3], "teacher"), *dS = tensor(v[10], "dS");
    occ_distill_t d{};
    d.dtype = layer_type(S, "S");
    const Call c{S.scalar_type(), S.device()};
    d.tokens = S.size(0);
    d.vocab = S.size(1);
    d.S = c(&S, "S", d.tokens, d.vocab, d.lds);
    d.t_dtype = OCC_F32;
    if (!index != !teacher) refuse(PyExc_ValueError, "%s", "index and teacher go together");
    if (index) {
      const int64_t k = matrix(index, "index").size(1);
      if (k > OCC_MAX_TEACHER) refuse(PyExc_ValueError, "%s lists too many entries", "index");
      d.k = (int32_t)k;
      d.t_dtype = layer_type(matrix(teacher, "teacher"), "teacher");
      if (k) {
        d.index = (const int32_t*)c(index, "index", d.tokens, k, at::kInt, d.ldi);
        d.teacher = c(teacher, "teacher", d.tokens, k, teacher->scalar_type(), d.ldt);
      }
    }
    d.labels = whole(c, tensor(v[4], "labels"), "labels", d.tokens);
    d.scale = values<float>(c, tensor(v[5], "scale"), "scale", at::kFloat, d.tokens);
    d.temperature = real(v[6]);
    d.alpha = real(v[7]);
    d.lse = values<float>(c, tensor(v[9], "lse"), "lse", at::kFloat, 2 * d.tokens);
    d.flags = flag_word(c, v[11]);
    const occ_stream_t s = c.stream();
    const c10::DeviceGuard current(c.device);
    at::Tensor loss, grad;
    if (backward) {
      given(tensor(v[9], "lse"), "lse");
      grad = given_or(dS, c, c.dtype, {d.tokens, d.vocab});
      dS = &grad;
    } else {
      loss = given_or(tensor(v[8], "loss"), c, at::kFloat, {d.tokens});
      d.loss = values<float>(c, &loss, "loss", at::kFloat, d.tokens);
      if (dS) grad = *dS;
    }
    d.dS = c(dS, "dS", d.tokens, d.vocab, d.ldds);
    return with_tensors(more.distill[backward](&d, s), {loss, grad});
  });
}

// setup_experts(addresses): in the order of `more`'s members
PyObject* setup_experts(PyObject*, PyObject* const* v, Py_ssize_t n) {
  constexpr int N = 16;
  static_assert(sizeof(more) == N * sizeof(void*), "one address each");
  if (!count(n, N)) return nullptr;
  void* at[N];
  for (int i = 0; i < N; ++i) {
    at[i] = PyLong_AsVoidPtr(v[i]);
    if (PyErr_Occurred()) return nullptr;
  }
  memcpy((void*)&more, at, sizeof(more));
  Py_RETURN_NONE;
}

}  // namespace
