// The calls on sorted tokens and on products with an epilogue for torch tensors (a part of xorenc_torch_fp8.cpp).

// A contiguous tensor of int32 (or of `type`) on the current GPU.
const Tensor &plain_tensor(PyObject *o, ScalarType type, int64_t dims, const char *what, const char *shape, const Place &here) {
  const Tensor &t = tensor(o, what);
  if (t.scalar_type() != type || t.dim() != dims || !here.has(t) || t.layout() != at::kStrided || !t.is_contiguous())
    throw Refused{std::string(what) + " must be " + (type == ScalarType::Float ? "float32" : "int32") + " of shape " + shape +
                  ", contiguous, on the current GPU"};
  return t;
}
int32_t *ints(const TensorBase &t) { return static_cast<int32_t *>(t.data_ptr()); }
float *floats(const TensorBase &t) { return static_cast<float *>(t.data_ptr()); }

// Where the pairs of tokens and experts are: places (tokens, picks), offsets (experts + 1), and shares (tokens, picks) or None.
struct Pairs {
  const Tensor &places, &offsets;
  int32_t tokens, picks;
  const int32_t *used;
  const float *shares = nullptr;
  Pairs(PyObject *p, PyObject *o, PyObject *s, const Place &here)
      : places(plain_tensor(p, ScalarType::Int, 2, "places", "(tokens, picks)", here)),
        offsets(plain_tensor(o, ScalarType::Int, 1, "offsets", "(experts + 1,)", here)), tokens(int_of(places.size(0), "the number of tokens")),
        picks(int_of(places.size(1), "the number of picks")), used(nullptr) {
    if (offsets.size(0) < 2) throw Refused{"offsets must be int32 of shape (experts + 1,)"};
    int_of(places.numel(), "the number of pairs");
    used = ints(offsets) + (offsets.size(0) - 1);
    if (s == Py_None) return;
    const Tensor &t = plain_tensor(s, ScalarType::Float, 2, "shares", "(tokens, picks)", here);
    if (t.sizes() != places.sizes()) throw Refused{"shares must have the shape of places"};
    shares = floats(t);
  }
  int64_t rows() const { return (int64_t)tokens * picks; }
};

// A matrix of the given size and type: the one given, or a new one.
struct Matrix {
  TensorBase t;
  int64_t ld;
  Matrix(PyObject *given, int64_t rows, int64_t cols, ScalarType type, const char *what, const Place &here) : ld(cols) {
    if (given == Py_None) {
      t = here.fresh({rows, cols}, {cols, 1}, type);
      return;
    }
    t = tensor(given, what);
    ld = rows_of(t, 2, what, here);
    if (t.size(0) != rows || t.size(1) != cols || t.scalar_type() != type)
      throw Refused{std::string(what) + " must be (" + std::to_string(rows) + ", " + std::to_string(cols) + ") of the type of the other rows"};
  }
};

PyObject *given_or_new(PyObject *given, const TensorBase &t) {
  if (given == Py_None) return THPVariable_Wrap(t);
  Py_INCREF(given);
  return given;
}

// (logits, picks, renormalise) -> (ids, shares)
PyObject *pick(PyObject *const *args) {
  const Place here;
  const Tensor &logits = tensor(args[0], "logits");
  const int64_t ldl = rows_of(logits, 2, "logits", here);
  const int32_t type = x_type(logits, "logits"), tokens = int_of(logits.size(0), "the number of tokens"), picks = int_of(args[1], "picks");
  const int renormalise = PyObject_IsTrue(args[2]);
  if (renormalise < 0) throw Raised();
  const int64_t n = picks < 0 ? 0 : picks > XORENC_MOE_MAX_PICKS ? XORENC_MOE_MAX_PICKS : picks;
  const TensorBase ids = here.fresh({tokens, n}, {n, 1}, ScalarType::Int), shares = here.fresh({tokens, n}, {n, 1}, ScalarType::Float);
  call("xorenc_pick_experts", [&] {
    return xorenc_pick_experts(logits.data_ptr(), type, ldl, tokens, (int32_t)logits.size(1), picks, renormalise, ints(ids), floats(shares), here.stream());
  });
  return result({ids, shares});
}

// (ids, experts) -> (places, tokens, offsets)
PyObject *sort(PyObject *const *args) {
  const Place here;
  const Tensor &ids = tensor(args[0], "ids");
  const bool wide = ids.scalar_type() == ScalarType::Long;
  if ((!wide && ids.scalar_type() != ScalarType::Int) || ids.dim() != 2 || !here.has(ids) || ids.layout() != at::kStrided || !ids.is_contiguous())
    throw Refused{"ids must be int32 or int64 of shape (tokens, picks), contiguous, on the current GPU"};
  const int32_t tokens = int_of(ids.size(0), "the number of tokens"), picks = int_of(ids.size(1), "the number of picks"), experts = int_of(args[1], "experts");
  int64_t need = 0;
  call("xorenc_sort_tokens_workspace", [&] { return xorenc_sort_tokens_workspace(tokens, picks, experts, &need); });
  const int64_t pairs = (int64_t)tokens * picks;
  const TensorBase places = here.fresh({tokens, picks}, {picks, 1}, ScalarType::Int), rows = here.fresh({pairs}, {1}, ScalarType::Int),
                   offsets = here.fresh({(int64_t)experts + 1}, {1}, ScalarType::Int);
  TensorBase workspace;
  if (need) workspace = here.fresh({need / 4}, {1}, ScalarType::Int);
  call("xorenc_sort_tokens", [&] {
    return xorenc_sort_tokens(ids.data_ptr(), wide ? XORENC_I64 : XORENC_I32, tokens, picks, experts, ints(places), ints(rows), ints(offsets),
                              need ? workspace.data_ptr() : nullptr, need, here.stream());
  });
  return result({places, rows, offsets});
}

// (X, places, offsets, shares, R) -> R
PyObject *gather(PyObject *const *args) {
  const Place here;
  const Tensor &X = tensor(args[0], "X");
  const int64_t ldx = rows_of(X, 2, "X", here);
  const int32_t type = x_type(X, "X");
  const Pairs at(args[1], args[2], args[3], here);
  if (X.size(0) != at.tokens) throw Refused{"X must have a row for each token of places"};
  const Matrix R(args[4], at.rows(), X.size(1), X.scalar_type(), "R", here);
  call("xorenc_gather_tokens", [&] {
    return xorenc_gather_tokens(X.data_ptr(), type, ldx, ints(at.places), at.used, at.shares, at.tokens, at.picks, (int32_t)X.size(1), R.t.data_ptr(), R.ld,
                                here.stream());
  });
  return given_or_new(args[4], R.t);
}

// (R, places, offsets, shares, residual, Y) -> Y
PyObject *combine(PyObject *const *args) {
  const Place here;
  const Tensor &R = tensor(args[0], "R");
  const int64_t ldr = rows_of(R, 2, "R", here), cols = R.size(1);
  const int32_t type = x_type(R, "R");
  const Pairs at(args[1], args[2], args[3], here);
  if (R.size(0) != at.rows()) throw Refused{"R must have a row for each pair of places"};
  const void *residual = nullptr;
  int64_t ld_residual = cols;
  if (args[4] != Py_None) {
    const Matrix r(args[4], at.tokens, cols, R.scalar_type(), "residual", here);
    residual = r.t.data_ptr();
    ld_residual = r.ld;
  }
  const Matrix Y(args[5], at.tokens, cols, R.scalar_type(), "Y", here);
  call("xorenc_combine_tokens", [&] {
    return xorenc_combine_tokens(R.data_ptr(), type, ldr, ints(at.places), at.used, at.shares, residual, ld_residual, at.tokens, at.picks, (int32_t)cols,
                                 Y.t.data_ptr(), Y.ld, here.stream());
  });
  return given_or_new(args[5], Y.t);
}

// (dY, R, places, offsets, shares, dR) -> (dR, dshares)
PyObject *combine_grad(PyObject *const *args) {
  const Place here;
  const Tensor &dY = tensor(args[0], "dY"), &R = tensor(args[1], "R");
  const int64_t ldy = rows_of(dY, 2, "dY", here), ldr = rows_of(R, 2, "R", here), cols = R.size(1);
  const int32_t type = x_type(R, "R");
  const Pairs at(args[2], args[3], args[4], here);
  if (args[4] == Py_None) throw Refused{"shares must be given (without them R's gradient is gather_tokens of dY)"};
  if (R.size(0) != at.rows()) throw Refused{"R must have a row for each pair of places"};
  if (dY.size(0) != at.tokens || dY.size(1) != cols || dY.scalar_type() != R.scalar_type()) throw Refused{"dY must be (tokens, columns of R) of the type of R"};
  const Matrix dR(args[5], at.rows(), cols, R.scalar_type(), "dR", here);
  const TensorBase dshares = here.fresh({at.tokens, at.picks}, {at.picks, 1}, ScalarType::Float);
  call("xorenc_combine_tokens_grad", [&] {
    return xorenc_combine_tokens_grad(dY.data_ptr(), type, ldy, R.data_ptr(), ldr, ints(at.places), at.used, at.shares, at.tokens, at.picks, (int32_t)cols,
                                      dR.t.data_ptr(), dR.ld, floats(dshares), here.stream());
  });
  return result({dR.t, dshares});
}

// An 8-bit product's operands, its result, and its epilogue.
struct Product {
  const Tensor &A, &SA, &W, &SW;
  int64_t lda, ldw, K, N, blocks;
  const float *sa, *sw;
  TensorBase Y;
  int64_t ldy;
  int32_t type;
  xorenc_epilogue epilogue = {};
  // dims: of W, SW and bias beyond one product's; y_rows < 0: as many as A has
  Product(PyObject *const *args, int64_t dims, PyObject *bias, PyObject *activation, int64_t y_rows, PyObject *dtype, PyObject *given, const Place &here)
      : A(tensor(args[0], "A")), SA(tensor(args[1], "SA")), W(tensor(args[2], "W")), SW(tensor(args[3], "SW")), lda(values_of(A, 2, "A", here)),
        ldw(values_of(W, 2 + dims, "W", here)), K(A.size(1)), N(W.size(dims)), blocks(blocks_of(K)) {
    if (W.size(1 + dims) != K) throw Refused{"A and W must have as many columns"};
    sa = scales_of(SA, {A.size(0), blocks}, "SA", here);
    sw = dims ? scales_of(SW, {W.size(0), blocks_of(N), blocks}, "SW", here) : scales_of(SW, {blocks_of(N), blocks}, "SW", here);
    if (blocks > 1 && SW.stride(1 + dims) != 1) throw Refused{"the columns of SW must be contiguous"};
    if (dtype != Py_None && !THPDtype_Check(dtype)) throw Refused{"out_dtype must be a torch type"};
    const ScalarType asked = dtype == Py_None ? ScalarType::Undefined : reinterpret_cast<THPDtype *>(dtype)->scalar_type;
    const int64_t M = y_rows < 0 ? A.size(0) : y_rows;
    ldy = N;
    if (given == Py_None) {
      if (asked != ScalarType::Undefined && !is_x_type(asked)) throw Refused{"Y must be float32 or bfloat16"};
      Y = here.fresh({M, N}, {N, 1}, asked == ScalarType::Undefined ? ScalarType::BFloat16 : asked);
    } else {
      Y = tensor(given, "Y");
      ldy = rows_of(Y, 2, "Y", here);
      if (Y.size(0) != M || Y.size(1) != N || (asked != ScalarType::Undefined && asked != Y.scalar_type()))
        throw Refused{"Y must be (rows, outputs) of the type asked for"};
    }
    type = x_type(Y, "Y");
    int_of(N, "the number of outputs");
    epilogue.struct_size = sizeof(epilogue);
    if (bias != Py_None) {
      const Tensor &b = tensor(bias, "bias");
      epilogue.bias_dtype = x_type(b, "bias");
      if (b.dim() != 1 + dims || b.size(dims) != N || (dims && b.size(0) != W.size(0)) || (N > 1 && b.stride(dims) != 1) || !here.has(b) ||
          b.layout() != at::kStrided)
        throw Refused{dims ? "bias must be (experts, outputs), its columns contiguous, on the current GPU" : "bias must be (outputs,), contiguous, on the current GPU"};
      epilogue.bias = b.data_ptr();
      epilogue.bias_stride = dims ? b.stride(0) : 0;
    }
    if (activation != Py_None) {
      const char *const name = PyUnicode_Check(activation) ? PyUnicode_AsUTF8(activation) : nullptr;
      if (!name && PyErr_Occurred()) throw Raised();
      const std::string f = name ? name : "";
      epilogue.activation = f == "relu" ? XORENC_RELU : f == "silu" ? XORENC_SILU : f == "gelu" ? XORENC_GELU : f == "gelu_tanh" ? XORENC_GELU_TANH : -1;
      if (epilogue.activation < 0) throw Refused{"activation must be None, 'relu', 'silu', 'gelu' or 'gelu_tanh'"};
    }
  }
  int64_t sa_blk() const { return blocks > 1 ? SA.stride(1) : 0; }
};

// (A, SA, W, SW, bias, activation, residual, out_dtype, Y) -> Y
PyObject *linear(PyObject *const *args) {
  const Place here;
  Product p(args, 0, args[4], args[5], -1, args[7], args[8], here);
  const int32_t m = int_of(p.A.size(0), "the number of tokens");
  if (args[6] != Py_None) {
    const Matrix r(args[6], m, p.N, p.Y.scalar_type(), "residual", here);
    p.epilogue.residual = r.t.data_ptr();
    p.epilogue.ld_residual = r.ld;
  }
  call("xorenc_linear_fp8", [&] {
    return xorenc_linear_fp8(bytes(p.A), p.lda, p.sa, p.SA.stride(0), p.sa_blk(), bytes(p.W), p.ldw, p.sw, p.N > kBlock ? p.SW.stride(0) : p.blocks, m,
                             (int32_t)p.N, (int32_t)p.K, &p.epilogue, p.Y.data_ptr(), p.type, p.ldy, here.stream());
  });
  return given_or_new(args[8], p.Y);
}

// (A, SA, W, SW, offsets, tokens, bias, activation, out_dtype, Y) -> Y
PyObject *experts(PyObject *const *args) {
  const Place here;
  const Tensor &offsets = plain_tensor(args[4], ScalarType::Int, 1, "offsets", "(experts + 1,)", here);
  const Tensor *const rows = args[5] == Py_None ? nullptr : &plain_tensor(args[5], ScalarType::Int, 1, "tokens", "(rows,)", here);
  Product p(args, 1, args[6], args[7], rows ? rows->size(0) : -1, args[8], args[9], here);
  if (offsets.size(0) != p.W.size(0) + 1) throw Refused{"offsets must have one element more than W has matrices"};
  const int32_t y_rows = int_of(p.Y.size(0), "the number of rows"), a_rows = int_of(p.A.size(0), "the number of rows of A");
  const int64_t E = p.W.size(0);
  const int32_t n = int_of(E, "the number of experts");
  call("xorenc_experts_fp8", [&] {
    return xorenc_experts_fp8(bytes(p.A), p.lda, p.sa, p.SA.stride(0), p.sa_blk(), a_rows, rows ? ints(*rows) : nullptr, ints(offsets), n,
                              bytes(p.W), p.ldw, E > 1 ? p.W.stride(0) : 0, p.sw, p.N > kBlock ? p.SW.stride(1) : p.blocks,
                              E > 1 ? p.SW.stride(0) : 0, (int32_t)p.N, (int32_t)p.K, &p.epilogue, p.Y.data_ptr(), p.type, p.ldy, y_rows, here.stream());
  });
  return given_or_new(args[9], p.Y);
}
