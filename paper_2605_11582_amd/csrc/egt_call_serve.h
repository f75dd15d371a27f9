// Tensors -> arguments of the operators beside the products (part of egt_call.cpp).
//
// Here a call is marshalled once, in C++, for both of its ways: the plain call launches at once, the prepared one
// hands the filled structures to a Call.  What a call cannot be made of is a ValueError that names the argument;
// what the library refuses or meets is an EgtError (binding._check), as everywhere.
#ifndef EGT_CALL_SERVE_H
#define EGT_CALL_SERVE_H

struct Refused { std::string why; };

typedef int (*batch_fn)(const void *, void *);
typedef int (*batch_cache_fn)(const void *, const void *, void *);
typedef int (*batch_ws_fn)(const void *, void *, size_t, void *);
typedef int (*tree_fn)(const void *, const void *, void *, size_t, void *);
typedef int (*tree_bytes_fn)(const void *, const void *, size_t *);

struct {
  batch_fn slots = nullptr, rules = nullptr;
  batch_cache_fn append = nullptr;
  batch_ws_fn lora = nullptr;
  tree_fn tree = nullptr;
  tree_bytes_fn tree_bytes = nullptr;
} V;

// What all arguments of a call share: they are on one device.
struct Reader {
  int device = -1;

  const at::Tensor &tensor(PyObject *o, const char *name, at::ScalarType type, int64_t dim) {
    if (!THPVariable_Check(o)) throw Refused{std::string(name) + ": expected a device tensor"};
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.is_cuda()) throw Refused{std::string(name) + ": expected a device tensor"};
    if (t.scalar_type() != type) throw Refused{std::string(name) + ": expected " + c10::toString(type) + ", got " + c10::toString(t.scalar_type())};
    if (t.dim() != dim) throw Refused{std::string(name) + ": expected " + std::to_string(dim) + " dimensions, got " + std::to_string(t.dim())};
    if (device < 0) device = t.get_device();
    if (device != t.get_device()) throw Refused{std::string(name) + ": on another device than the other tensors"};
    return t;
  }
  void same(const char *name, int64_t got, int64_t want) {
    if (got != want) throw Refused{std::string(name) + ": size " + std::to_string(got) + ", needs " + std::to_string(want)};
  }
  int32_t fits(const char *name, int64_t v) {
    if (v < 0 || v > INT32_MAX) throw Refused{std::string(name) + ": too large"};
    return (int32_t)v;
  }
  // a vector of `n` elements (any number: n < 0), back to back
  const at::Tensor &row(PyObject *o, const char *name, at::ScalarType type, int64_t n) {
    const at::Tensor &t = tensor(o, name, type, 1);
    if (n >= 0) same(name, t.size(0), n);
    if (!t.is_contiguous()) throw Refused{std::string(name) + ": expected contiguous elements"};
    return t;
  }
  template <typename T>
  T *vec(PyObject *o, const char *name, at::ScalarType type, int64_t n) { return (T *)row(o, name, type, n).data_ptr(); }
  template <typename T>
  T *maybe(PyObject *o, const char *name, at::ScalarType type, int64_t n) { return o == Py_None ? nullptr : vec<T>(o, name, type, n); }
  // rows of contiguous elements, `ld` elements apart
  const at::Tensor &rows(PyObject *o, const char *name, at::ScalarType type, int64_t &ld) {
    const at::Tensor &t = tensor(o, name, type, 2);
    if (t.size(1) > 1 && t.stride(1) != 1) throw Refused{std::string(name) + ": the elements of a row must be contiguous"};
    ld = t.size(0) > 1 ? t.stride(0) : t.size(1);      // (a single row has no distance to another)
    return t;
  }
  // (rows, heads, dim) with contiguous dim; strides of axes of one element do not matter
  const at::Tensor &heads(PyObject *o, const char *name, int64_t &row, int64_t &head) {
    const at::Tensor &t = tensor(o, name, at::kHalf, 3);
    if (t.size(2) > 1 && t.stride(2) != 1) throw Refused{std::string(name) + ": the elements of a head must be contiguous"};
    row = t.size(0) > 1 ? t.stride(0) : 0;
    head = t.size(1) > 1 ? t.stride(1) : 0;
    return t;
  }
  void written(const char *name, const at::Tensor &t) {
    for (int64_t d = 0; d < t.dim(); ++d)
      if (t.size(d) > 1 && t.stride(d) == 0) throw Refused{std::string(name) + ": written, but its elements share memory"};
  }
  // (blocks, heads, page, dim)
  void cache(PyObject *ko, PyObject *vo, egt_kv_cache &c) {
    const at::Tensor &k = tensor(ko, "k_cache", at::kHalf, 4), &v = tensor(vo, "v_cache", at::kHalf, 4);
    for (int d = 0; d < 4; ++d) same("v_cache", v.size(d), k.size(d));
    if ((k.size(3) > 1 && k.stride(3) != 1) || (v.size(3) > 1 && v.stride(3) != 1)) throw Refused{"k_cache, v_cache: the elements of a head must be contiguous"};
    c.k = (uint16_t *)k.data_ptr();
    c.v = (uint16_t *)v.data_ptr();
    c.blocks = fits("k_cache", k.size(0));
    c.heads = fits("k_cache", k.size(1));
    c.page = fits("k_cache", k.size(2));
    c.dim = fits("k_cache", k.size(3));
    auto stride = [](const at::Tensor &t, int d) { return t.size(d) > 1 ? t.stride(d) : 0; };
    c.k_block = stride(k, 0), c.k_head = stride(k, 1), c.k_token = stride(k, 2);
    c.v_block = stride(v, 0), c.v_head = stride(v, 1), c.v_token = stride(v, 2);
  }
  int32_t integer(PyObject *o, const char *name) {
    const int64_t v = PyLong_Check(o) ? PyLong_AsLongLong(o) : -1;
    if (!PyLong_Check(o) || (v == -1 && PyErr_Occurred()) || v < INT32_MIN || v > INT32_MAX) {
      PyErr_Clear();
      throw Refused{std::string(name) + ": expected a 32-bit integer"};
    }
    return (int32_t)v;
  }
  float number(PyObject *o, const char *name) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) {
      PyErr_Clear();
      throw Refused{std::string(name) + ": expected a number"};
    }
    return (float)v;
  }
  void workspace(PyObject *o, void *&p, size_t &bytes) {
    p = nullptr, bytes = 0;
    if (o == Py_None) return;                         // (the library says that it is missing)
    if (!THPVariable_Check(o) || !THPVariable_Unpack(o).is_cuda() || !THPVariable_Unpack(o).is_contiguous())
      throw Refused{"workspace: expected a contiguous device tensor"};
    const at::Tensor &t = THPVariable_Unpack(o);
    if (device >= 0 && t.get_device() != device) throw Refused{"workspace: on another device than the other tensors"};
    p = t.data_ptr();
    bytes = t.nbytes();
  }
  // the stream object's handle, or that of the device's current stream
  void *stream(PyObject *o) const {
    PyObject *v = o == Py_None ? PyObject_CallFunction(B.raw_stream, "i", device) : PyObject_GetAttr(o, S.cuda_stream);
    void *s = v ? PyLong_AsVoidPtr(v) : nullptr;
    Py_XDECREF(v);
    if (PyErr_Occurred()) {
      PyErr_Clear();
      throw Refused{"stream: expected a stream of the device, or None"};
    }
    return s;
  }
};

struct Slots {
  static constexpr int ARGS = 11;
  static constexpr Kind KIND = BATCH;
  egt_slots_batch b{};
  void read(Reader &r, PyObject *const *a) {
    // (lens, counts, block_table, page, blocks, free_blocks, free_head, slots, cu_tokens, new_lens, new_head)
    const at::Tensor &lens = r.row(a[0], "lens", at::kInt, -1), &table = r.rows(a[2], "block_table", at::kInt, b.ld_table);
    const int64_t n = lens.size(0);
    b.requests = r.fits("lens", n);
    b.lens = (const int32_t *)lens.data_ptr();
    b.counts = r.vec<const int32_t>(a[1], "counts", at::kInt, n);
    r.same("block_table", table.size(0), n);
    r.written("block_table", table);
    b.block_table = (int32_t *)table.data_ptr();
    b.table_blocks = r.fits("block_table", table.size(1));
    b.page = r.integer(a[3], "page");
    b.blocks = r.integer(a[4], "blocks");
    const at::Tensor &free = r.row(a[5], "free_blocks", at::kInt, -1), &slots = r.row(a[7], "slots", at::kInt, -1);
    b.free_blocks = (const int32_t *)free.data_ptr();
    b.n_free = r.fits("free_blocks", free.size(0));
    b.free_head = r.vec<const int32_t>(a[6], "free_head", at::kInt, 1);
    b.slots = (int32_t *)slots.data_ptr();
    b.n_slots = r.fits("slots", slots.size(0));
    b.cu_tokens = r.vec<int32_t>(a[8], "cu_tokens", at::kInt, n + 1);
    b.new_lens = r.vec<int32_t>(a[9], "new_lens", at::kInt, n);
    b.new_head = r.vec<int32_t>(a[10], "new_head", at::kInt, 1);
  }
  int launch(void *s) const { return V.slots(&b, s); }
  static uintptr_t entry() { return (uintptr_t)V.slots; }
  std::vector<int64_t> words() const { return {(int64_t)(uintptr_t)&b}; }
};

struct Append {
  static constexpr int ARGS = 6;
  static constexpr Kind KIND = TABLE;
  egt_append_batch b{};
  egt_kv_cache c{};
  void read(Reader &r, PyObject *const *a) {
    // (k, v, slots, k_cache, v_cache, rows)
    const at::Tensor &k = r.heads(a[0], "k", b.k_row, b.k_head), &v = r.heads(a[1], "v", b.v_row, b.v_head), &slots = r.row(a[2], "slots", at::kInt, -1);
    r.cache(a[3], a[4], c);
    r.same("v", v.size(0), k.size(0));
    for (const at::Tensor *t : {&k, &v}) {
      r.same("k, v: heads", t->size(1), c.heads);
      r.same("k, v: head size", t->size(2), c.dim);
    }
    r.written("k_cache", THPVariable_Unpack(a[3]));
    r.written("v_cache", THPVariable_Unpack(a[4]));
    b.k = (const uint16_t *)k.data_ptr();
    b.v = (const uint16_t *)v.data_ptr();
    b.slots = (const int32_t *)slots.data_ptr();
    b.n = r.fits("slots", slots.size(0));
    b.n_rows = r.fits("k", k.size(0));
    b.rows = r.maybe<const int32_t>(a[5], "rows", at::kInt, b.n);
    if (!b.rows) r.same("slots", b.n, b.n_rows);
  }
  int launch(void *s) const { return V.append(&b, &c, s); }
  static uintptr_t entry() { return (uintptr_t)V.append; }
  std::vector<int64_t> words() const { return {(int64_t)(uintptr_t)&b, (int64_t)(uintptr_t)&c}; }
};

struct Tree {
  static constexpr int ARGS = 13;
  static constexpr Kind KIND = TREE;
  egt_tree_batch b{};
  egt_kv_cache c{};
  void *ws = nullptr;
  size_t bytes = 0;
  void read(Reader &r, PyObject *const *a) {
    // (q, k, v, k_cache, v_cache, block_table, lens, cu_tokens, mask, out, scale, max_tokens, workspace)
    const at::Tensor &q = r.heads(a[0], "q", b.q_row, b.q_head), &k = r.heads(a[1], "k", b.k_row, b.k_head), &v = r.heads(a[2], "v", b.v_row, b.v_head);
    const at::Tensor &out = r.heads(a[9], "out", b.out_row, b.out_head), &table = r.rows(a[5], "block_table", at::kInt, b.ld_table);
    r.cache(a[3], a[4], c);
    const int64_t tokens = q.size(0), n = table.size(0);
    for (const at::Tensor *t : {&k, &v}) {
      r.same("k, v: rows", t->size(0), tokens);
      r.same("k, v: heads", t->size(1), c.heads);
      r.same("k, v: head size", t->size(2), c.dim);
    }
    r.same("q: head size", q.size(2), c.dim);
    for (int d = 0; d < 3; ++d) r.same("out", out.size(d), q.size(d));
    r.written("out", out);
    b.q = (const uint16_t *)q.data_ptr();
    b.k = (const uint16_t *)k.data_ptr();
    b.v = (const uint16_t *)v.data_ptr();
    b.out = (uint16_t *)out.data_ptr();
    if (tokens && (b.out == b.q || b.out == b.k || b.out == b.v)) throw Refused{"out: one of the inputs"};
    b.block_table = (const int32_t *)table.data_ptr();
    b.requests = r.fits("block_table", n);
    b.table_blocks = r.fits("block_table", table.size(1));
    b.lens = r.vec<const int32_t>(a[6], "lens", at::kInt, n);
    b.cu_tokens = r.vec<const int32_t>(a[7], "cu_tokens", at::kInt, n + 1);
    b.mask = r.vec<const uint64_t>(a[8], "mask", at::kLong, tokens);
    b.scale = r.number(a[10], "scale");
    b.max_tokens = r.integer(a[11], "max_tokens");
    b.tokens = r.fits("q", tokens);
    b.heads = r.fits("q", q.size(1));
    r.workspace(a[12], ws, bytes);
  }
  int launch(void *s) const { return V.tree(&b, &c, ws, bytes, s); }
  static uintptr_t entry() { return (uintptr_t)V.tree; }
  std::vector<int64_t> words() const { return {(int64_t)(uintptr_t)&b, (int64_t)(uintptr_t)&c, (int64_t)(uintptr_t)ws, (int64_t)bytes}; }
};

struct Lora {
  static constexpr int ARGS = 8;
  static constexpr Kind KIND = BATCH_WS;
  egt_lora_batch b{};
  void *ws = nullptr;
  size_t bytes = 0;
  void read(Reader &r, PyObject *const *a) {
    // (X, A, B, index, Y, workspace, base, scale)
    const at::Tensor &X = r.rows(a[0], "X", at::kHalf, b.ldx), &A = r.tensor(a[1], "A", at::kHalf, 3), &Bm = r.tensor(a[2], "B", at::kHalf, 3);
    const at::Tensor &Y = r.rows(a[4], "Y", at::kHalf, b.ldy);
    const int64_t M = X.size(0), cols = X.size(1), n = A.size(0), rank = A.size(1), rows = Bm.size(1);
    r.same("A: columns", A.size(2), cols);
    r.same("B: adapters", Bm.size(0), n);
    r.same("B: rank", Bm.size(2), rank);
    r.same("Y: rows", Y.size(0), M);
    r.same("Y: columns", Y.size(1), rows);
    r.written("Y", Y);
    for (const at::Tensor *t : {&A, &Bm})             // (the matrices of a pool; the pool itself may be strided)
      if ((t->size(2) > 1 && t->stride(2) != 1) || (t->size(1) > 1 && t->stride(1) != t->size(2)))
        throw Refused{"A, B: the rows of an adapter must be back to back"};
    b.X = (const uint16_t *)X.data_ptr();
    b.A = (const uint16_t *)A.data_ptr();
    b.B = (const uint16_t *)Bm.data_ptr();
    b.Y = (uint16_t *)Y.data_ptr();
    b.a_stride = n > 1 ? A.stride(0) : 0;
    b.b_stride = n > 1 ? Bm.stride(0) : 0;
    b.index = r.vec<const int32_t>(a[3], "index", at::kInt, M);
    if (a[6] != Py_None) {
      const at::Tensor &base = r.rows(a[6], "base", at::kHalf, b.ldbase);
      r.same("base: rows", base.size(0), M);
      r.same("base: columns", base.size(1), rows);
      b.base = (const uint16_t *)base.data_ptr();
    }
    b.scale = r.maybe<const float>(a[7], "scale", at::kFloat, n);
    b.M = r.fits("X", M);
    b.cols = r.fits("X", cols);
    b.rows = r.fits("B", rows);
    b.rank = r.fits("A", rank);
    b.adapters = r.fits("A", n);
    r.workspace(a[5], ws, bytes);
  }
  int launch(void *s) const { return V.lora(&b, ws, bytes, s); }
  static uintptr_t entry() { return (uintptr_t)V.lora; }
  std::vector<int64_t> words() const { return {(int64_t)(uintptr_t)&b, (int64_t)(uintptr_t)ws, (int64_t)bytes}; }
};

struct Rules {
  static constexpr int ARGS = 15;
  static constexpr Kind KIND = BATCH;
  egt_rules_batch b{};
  void read(Reader &r, PyObject *const *a) {
    // (logits, out, cu_tokens, history, history_len, prompt_len, draft, mask, repetition, frequency, presence, bias_ids, bias, allowed, allowed_row)
    const bool f32 = THPVariable_Check(a[0]) && THPVariable_Unpack(a[0]).scalar_type() == at::kFloat;
    const at::ScalarType type = f32 ? at::kFloat : at::kHalf;
    const at::Tensor &x = r.rows(a[0], "logits", type, b.ld_logits), &y = r.rows(a[1], "out", type, b.ld_out), &cu = r.row(a[2], "cu_tokens", at::kInt, -1);
    if (cu.size(0) < 1) throw Refused{"cu_tokens: empty"};
    const int64_t tokens = x.size(0), vocab = x.size(1), n = cu.size(0) - 1;
    r.same("out", y.size(0), tokens);
    r.same("out", y.size(1), vocab);
    r.written("out", y);
    b.logits = x.data_ptr();
    b.out = y.data_ptr();
    b.cu_tokens = (const int32_t *)cu.data_ptr();
    b.kind = f32 ? EGT_LOGITS_FP32 : EGT_LOGITS_FP16;
    b.requests = r.fits("cu_tokens", n);
    b.tokens = r.fits("logits", tokens);
    b.vocab = r.fits("logits", vocab);
    auto both = [&](int i, int j, const char *what) {
      if ((a[i] == Py_None) != (a[j] == Py_None)) throw Refused{std::string(what) + ": one goes with the other"};
    };
    both(3, 4, "history, history_len");
    both(6, 7, "draft, mask");
    both(11, 12, "bias_ids, bias");
    both(13, 14, "allowed, allowed_row");
    if (a[3] != Py_None) {
      const at::Tensor &h = r.rows(a[3], "history", at::kInt, b.ld_history);
      r.same("history", h.size(0), n);
      b.history = (const int32_t *)h.data_ptr();
      b.history_len = r.vec<const int32_t>(a[4], "history_len", at::kInt, n);
      // (rows are read up to their width, which may be less than their distance)
      b.history_width = r.fits("history", h.size(1));
    }
    b.prompt_len = r.maybe<const int32_t>(a[5], "prompt_len", at::kInt, n);
    b.draft = r.maybe<const int32_t>(a[6], "draft", at::kInt, tokens);
    b.mask = r.maybe<const uint64_t>(a[7], "mask", at::kLong, tokens);
    b.repetition = r.maybe<const float>(a[8], "repetition", at::kFloat, n);
    b.frequency = r.maybe<const float>(a[9], "frequency", at::kFloat, n);
    b.presence = r.maybe<const float>(a[10], "presence", at::kFloat, n);
    if (a[11] != Py_None) {
      const at::Tensor &ids = r.tensor(a[11], "bias_ids", at::kInt, 2), &add = r.tensor(a[12], "bias", at::kFloat, 2);
      for (const at::Tensor *t : {&ids, &add}) {
        r.same("bias_ids, bias: requests", t->size(0), n);
        r.same("bias_ids, bias: entries", t->size(1), ids.size(1));
        if (!t->is_contiguous()) throw Refused{"bias_ids, bias: expected contiguous elements"};
      }
      b.bias_ids = (const int32_t *)ids.data_ptr();
      b.bias = (const float *)add.data_ptr();
      b.n_bias = r.fits("bias_ids", ids.size(1));
    }
    if (a[13] != Py_None) {
      const at::Tensor &m = r.rows(a[13], "allowed", at::kInt, b.ld_allowed);
      r.same("allowed: words a row", m.size(1), (vocab + 31) / 32);
      b.n_allowed = r.fits("allowed", m.size(0));
      b.allowed_row = r.vec<const int32_t>(a[14], "allowed_row", at::kInt, tokens);
      // (a grammar without rows has no memory, and is not the same as none: no row may be asked for.  It gets an address that is not read.)
      b.allowed = b.n_allowed ? (const uint32_t *)m.data_ptr() : (const uint32_t *)b.allowed_row;
    }
  }
  int launch(void *s) const { return V.rules(&b, s); }
  static uintptr_t entry() { return (uintptr_t)V.rules; }
  std::vector<int64_t> words() const { return {(int64_t)(uintptr_t)&b}; }
};

template <class T>
void drop(PyObject *capsule) { delete (T *)PyCapsule_GetPointer(capsule, nullptr); }

// f(prepare, arguments ..., stream): launches and returns None, or returns the prepared Call
template <class T>
PyObject *batch_call(PyObject *, PyObject *const *a, Py_ssize_t n) {
  if (n != T::ARGS + 2 || !T::entry()) {
    PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
    return nullptr;
  }
  try {
    Reader r;
    if (a[0] != Py_True) {
      T c;
      c.read(r, a + 1);
      void *s = r.stream(a[n - 1]);
      c10::DeviceGuard on(c10::Device(c10::kCUDA, (c10::DeviceIndex)r.device));
      int st;
      Py_BEGIN_ALLOW_THREADS
      st = c.launch(s);
      Py_END_ALLOW_THREADS
      if (st != 0) return PyObject_CallFunction(B.check, "i", st);
      Py_RETURN_NONE;
    }
    auto c = std::make_unique<T>();
    c->read(r, a + 1);
    void *s = r.stream(a[n - 1]);
    const std::vector<int64_t> words = c->words();
    THPObjectPtr capsule(PyCapsule_New(c.get(), nullptr, drop<T>));
    if (!capsule) return nullptr;
    c.release();
    THPObjectPtr args(PyTuple_New((Py_ssize_t)words.size())), launches(PyList_New(1)), keep(PyTuple_New(n));
    if (!args || !launches || !keep) return nullptr;
    for (size_t k = 0; k < words.size(); ++k) {
      PyObject *v = PyLong_FromUnsignedLongLong((unsigned long long)words[k]);
      if (!v) return nullptr;
      PyTuple_SET_ITEM(args.get(), (Py_ssize_t)k, v);
    }
    PyList_SET_ITEM(launches.get(), 0, args.release());
    PyTuple_SET_ITEM(keep.get(), 0, capsule.release());
    for (Py_ssize_t k = 1; k < n; ++k) {
      Py_INCREF(a[k]);
      PyTuple_SET_ITEM(keep.get(), k, a[k]);
    }
    return PyObject_CallFunction((PyObject *)&CallType, "iKOKO", (int)T::KIND, (unsigned long long)T::entry(), launches.get(),
                                 (unsigned long long)(uintptr_t)s, keep.get());
  } catch (const Refused &e) {
    PyErr_SetString(PyExc_ValueError, e.why.c_str());
  } catch (const std::bad_alloc &) {
    PyErr_NoMemory();
  } catch (const std::exception &e) {                 // (a tensor without memory of its own)
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, e.what());
  }
  return nullptr;
}

// tree_attention_ws_bytes(q, k_cache, block_table, lens, max_tokens)
PyObject *tree_bytes(PyObject *, PyObject *const *a, Py_ssize_t n) {
  if (n != 5 || !V.tree_bytes) {
    PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
    return nullptr;
  }
  try {
    Reader r;
    egt_tree_batch b{};
    egt_kv_cache c{};
    const at::Tensor &q = r.tensor(a[0], "q", at::kHalf, 3), &k = r.tensor(a[1], "k_cache", at::kHalf, 4), &table = r.tensor(a[2], "block_table", at::kInt, 2);
    b.tokens = r.fits("q", q.size(0));
    b.heads = r.fits("q", q.size(1));
    b.requests = r.fits("lens", r.tensor(a[3], "lens", at::kInt, 1).size(0));
    b.table_blocks = r.fits("block_table", table.size(1));
    b.max_tokens = r.integer(a[4], "max_tokens");
    c.blocks = r.fits("k_cache", k.size(0));
    c.heads = r.fits("k_cache", k.size(1));
    c.page = r.fits("k_cache", k.size(2));
    c.dim = r.fits("k_cache", k.size(3));
    size_t bytes = 0;
    const int st = V.tree_bytes(&b, &c, &bytes);
    if (st != 0) return PyObject_CallFunction(B.check, "i", st);
    return PyLong_FromSize_t(bytes);
  } catch (const Refused &e) {
    PyErr_SetString(PyExc_ValueError, e.why.c_str());
  } catch (const std::exception &e) {
    PyErr_SetString(PyExc_ValueError, e.what());
  }
  return nullptr;
}

// bind_batches(slots, append, tree, tree_bytes, lora, rules): addresses of the entry points
PyObject *bind_batches(PyObject *, PyObject *args) {
  unsigned long long f[6];
  if (!PyArg_ParseTuple(args, "KKKKKK", f, f + 1, f + 2, f + 3, f + 4, f + 5)) return nullptr;
  V.slots = (batch_fn)f[0];
  V.append = (batch_cache_fn)f[1];
  V.tree = (tree_fn)f[2];
  V.tree_bytes = (tree_bytes_fn)f[3];
  V.lora = (batch_ws_fn)f[4];
  V.rules = (batch_fn)f[5];
  Py_RETURN_NONE;
}

#endif
