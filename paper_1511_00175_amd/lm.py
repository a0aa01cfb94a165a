"""The operators at the ends of a language model, within its blocks and of its
matrix update (include/fc_lm.h) on torch tensors: they produce the gradients that Plan
aggregates, or consume their sum.  As Plan does, each class checks every buffer
before it calls the C ABI, which sees only pointers, and enqueues on the given
stream or torch's current one."""
import ctypes

from ._fc import FC_F16, FC_F32, FcError
from ._fc_lm import (FC_BF16, FC_BLOCK_E4M3, FC_BLOCK_I8, FC_GATE_NONE, FC_GATE_SIGMOID, FC_GATE_SILU, FC_NORM_LAYER,
                     FC_NORM_RMS, fc_matrix, lib)

DTYPES = {"f32": FC_F32, "f16": FC_F16, "bf16": FC_BF16}
_CODES = {}     # torch dtype -> fc_dtype value
_INTEGERS = {}  # torch dtype of a token list -> bytes of an entry


def _types():
    """Fills the tables above, at the first plan (importing the package does not
    import torch)."""
    if not _CODES:
        import torch
        _CODES.update({torch.float32: FC_F32, torch.float16: FC_F16, torch.bfloat16: FC_BF16})
        _INTEGERS.update({torch.int32: 4, torch.int64: 8})


def _tensor(t, name):
    import torch
    _types()
    if not isinstance(t, torch.Tensor):
        raise ValueError(f"{name} must be a torch tensor")


# The checks of a call are a few attribute reads each: a small call's kernel is
# shorter than they are on the host.

def _matrix(t, name, rows, cols, device, code=None):
    """`t` must be a (rows, cols) tensor of a supported type (`code`: of that
    one) on the device, its rows contiguous and any distance apart; returns
    (pointer, type, row stride)."""
    try:
        got, shape, (ld, one) = _CODES[t.dtype], t.shape, t.stride()
    except (AttributeError, KeyError, TypeError, ValueError):  # no tensor, no such type, not two dimensions
        _tensor(t, name)
        got, shape, (ld, one) = _CODES.get(t.dtype), t.shape, t.stride() if t.dim() == 2 else (0, 0)
    if got is None or (code is not None and got != code):
        raise ValueError(f"{name} must not be {t.dtype}")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, the plan on {device}")
    if len(shape) != 2 or shape[0] != rows or shape[1] != cols:
        raise ValueError(f"{name} is {tuple(shape)}, not {(rows, cols)}")
    if rows <= 1:
        ld = cols
    if (one != 1 and cols > 1) or ld < cols:
        raise ValueError(f"{name} must have contiguous rows that do not overlap")
    return t.data_ptr(), got, ld


def _list(t, name, device):
    """`t` must be a contiguous vector of int32 or int64 on the device; returns
    (pointer, bytes of an entry, length)."""
    try:
        size, shape = _INTEGERS[t.dtype], t.shape
    except (AttributeError, KeyError):
        _tensor(t, name)
        size, shape = _INTEGERS.get(t.dtype), t.shape
    if size is None:
        raise ValueError(f"{name} must be int32 or int64, not {t.dtype}")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, the plan on {device}")
    if len(shape) != 1 or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous vector")
    return t.data_ptr(), size, shape[0]


def _vector(t, name, n, device, code):
    """`t` must be a contiguous vector of n elements of type `code` on the
    device; returns its pointer."""
    _tensor(t, name)
    if _CODES.get(t.dtype) != code:
        raise ValueError(f"{name} must not be {t.dtype}")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, the plan on {device}")
    if t.dim() != 1 or t.shape[0] != n or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous vector of {n} elements")
    return t.data_ptr()


def _typed(t, name, rows, cols, dtype, device):
    """`t` must be a (rows, cols) tensor of torch's `dtype` on the device, its rows
    contiguous and any distance apart; returns (pointer, row stride)."""
    try:
        if t.dtype is dtype and t.device == device and t.shape == (rows, cols):
            ld, one = t.stride()
            if one == 1 and (ld >= cols or rows <= 1):
                return t.data_ptr(), ld if rows > 1 else cols
    except (AttributeError, TypeError):
        pass
    _tensor(t, name)  # what is wrong, or a single column
    if t.dtype is not dtype:
        raise ValueError(f"{name} must be {dtype}, not {t.dtype}")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, the plan on {device}")
    if t.dim() != 2 or t.shape[0] != rows or t.shape[1] != cols:
        raise ValueError(f"{name} is {tuple(t.shape)}, not {(rows, cols)}")
    ld, one = t.stride()
    if rows <= 1:
        ld = cols
    if (one != 1 and cols > 1) or ld < cols:
        raise ValueError(f"{name} must have contiguous rows that do not overlap")
    return t.data_ptr(), ld


def _typed_vector(t, name, n, dtype, device):
    """`t` must be a contiguous vector of n elements of torch's `dtype` on the device;
    returns its pointer."""
    try:
        if t.dtype is dtype and t.device == device and t.shape == (n,) and t.is_contiguous():
            return t.data_ptr()
    except (AttributeError, TypeError):
        pass
    _tensor(t, name)
    if t.dtype is not dtype:
        raise ValueError(f"{name} must be {dtype}, not {t.dtype}")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, the plan on {device}")
    raise ValueError(f"{name} must be a contiguous vector of {n} elements")


def _rows(t, name):
    """The rows of a tensor whose other checks follow."""
    try:
        return t.shape[0]
    except (AttributeError, TypeError, IndexError):
        _tensor(t, name)
        raise ValueError(f"{name} must have two dimensions") from None


_current = None  # the package's _stream, once it is loaded


def _stream(stream):
    global _current
    if _current is None:
        from . import _stream as _current
    return _current(stream)


_FUNCTIONS = {n: getattr(lib, n) for n in ("fc_embed_lookup", "fc_embed_grad", "fc_xent_loss", "fc_xent_loss_grad",
                                           "fc_muon_orthogonalize", "fc_muon_step", "fc_norm_before", "fc_norm_after",
                                           "fc_norm_between", "fc_norm_before_grad", "fc_norm_after_grad",
                                           "fc_norm_between_grad", "fc_ckpt_pack", "fc_ckpt_unpack", "fc_ckpt_grad",
                                           "fc_mxfp_pack", "fc_mxfp_unpack", "fc_mxfp_product", "fc_mxfp_linear")}


class _Handle:
    """A plan of the library: created by `make`, freed by close() or garbage
    collection, after the device's work is done."""

    handle = None

    def _create(self, make, *args):
        import torch
        _types()
        h = ctypes.c_void_p()
        rc = getattr(lib, make)(ctypes.byref(h), *args)
        if rc:
            raise FcError(make, rc)
        self.handle = h
        self.device = torch.device("cuda", torch.cuda.current_device())

    def _call(self, name, *args):
        rc = _FUNCTIONS[name](self.handle, *args)
        if rc:
            raise FcError(name, rc)

    def close(self):
        """Free the plan.  Kernels queued by earlier calls may still use its
        workspace, so its device is synchronized first."""
        if self.handle:
            try:
                import torch
                torch.cuda.synchronize(self.device)
            except Exception:
                pass
            getattr(lib, self._destroy)(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Embedding(_Handle):
    """A table of `rows` rows of `dim` elements (fc_embed): scaled rows for a
    list of up to `max_tokens` tokens, and the table's gradient.

    Tables, outputs and gradients are f32, f16 or bf16, each by its tensor.
    Tokens outside [0, rows) are padding: zeros, and no gradient."""

    _destroy = "fc_embed_destroy"

    def __init__(self, rows, dim, max_tokens):
        self._create("fc_embed_create", rows, dim, max_tokens)
        self.rows, self.dim, self.max_tokens = rows, dim, max_tokens

    def lookup(self, table, tokens, out, scale=1.0, stream=None):
        """out[t] = scale * table[tokens[t]]."""
        tok, size, n = _list(tokens, "tokens", self.device)
        tp, tc, tl = _matrix(table, "table", self.rows, self.dim, self.device)
        op, oc, ol = _matrix(out, "out", n, self.dim, self.device)
        self._call("fc_embed_lookup", tp, tc, tl, tok, size, n, scale, op, oc, ol, _stream(stream))

    def grad(self, dy, tokens, dtable, scale=1.0, accumulate=False, stream=None):
        """dtable[r] = (dtable[r] if accumulate else 0) + scale * the sum of
        dy[t] over the t with tokens[t] == r, for every row of the table."""
        tok, size, n = _list(tokens, "tokens", self.device)
        if n > self.max_tokens:
            raise ValueError(f"{n} tokens for a plan of {self.max_tokens}")
        yp, yc, yl = _matrix(dy, "dy", n, self.dim, self.device)
        gp, gc, gl = _matrix(dtable, "dtable", self.rows, self.dim, self.device)
        self._call("fc_embed_grad", yp, yc, yl, tok, size, n, scale, gp, gc, gl, bool(accumulate), _stream(stream))


class CrossEntropy(_Handle):
    """Softmax cross entropy over a vocabulary of `rows` rows of `dim` elements
    (fc_xent), from the last layer's outputs x (tokens, dim) and the rows w, both
    of `dtype` ("f16" or "bf16"), for up to `max_tokens` tokens.  The logits are
    not stored, but for gradients 16 bits of each are; `chunk` tokens (0: as many as
    fit) go through together.  Gradients of more than 64 tokens at a time take d in
    x's type; with `chunk` of at most 64 it keeps twice those bits, for more time.

    x and w lie on 16 bytes with row strides of a multiple of 8, unless dim is no
    multiple of 8.

    Targets outside [0, rows) are padding: loss 0, and no gradient."""

    _destroy = "fc_xent_destroy"

    def __init__(self, rows, dim, max_tokens, dtype="f16", chunk=0):
        if dtype not in ("f16", "bf16"):
            raise ValueError(f"dtype must be f16 or bf16, not {dtype}")
        self.code = DTYPES[dtype]
        self._create("fc_xent_create", rows, dim, max_tokens, self.code, chunk)
        self.rows, self.dim, self.max_tokens = rows, dim, max_tokens

    def _inputs(self, x, w, targets, loss):
        yp, size, n = _list(targets, "targets", self.device)
        if n > self.max_tokens:
            raise ValueError(f"{n} tokens for a plan of {self.max_tokens}")
        xp, _, xl = _matrix(x, "x", n, self.dim, self.device, self.code)
        wp, _, wl = _matrix(w, "w", self.rows, self.dim, self.device, self.code)
        lp = _vector(loss, "loss", n, self.device, FC_F32)
        return xp, xl, wp, wl, yp, size, n, lp

    def loss(self, x, w, targets, loss, stream=None):
        """loss[t] = logsumexp(x[t] w^T) - x[t] . w[targets[t]], in fp32."""
        xp, xl, wp, wl, yp, size, n, lp = self._inputs(x, w, targets, loss)
        self._call("fc_xent_loss", xp, xl, wp, wl, yp, size, n, lp, _stream(stream))

    def loss_grad(self, x, w, targets, loss, dx, dw, scale=1.0, stream=None):
        """The losses, and the gradients of scale times their sum by x and w,
        each of its tensor's type; dx or dw may be None."""
        xp, xl, wp, wl, yp, size, n, lp = self._inputs(x, w, targets, loss)
        dxp, dxc, dxl = (None, 0, 0) if dx is None else _matrix(dx, "dx", n, self.dim, self.device)
        dwp, dwc, dwl = (None, 0, 0) if dw is None else _matrix(dw, "dw", self.rows, self.dim, self.device)
        self._call("fc_xent_loss_grad", xp, xl, wp, wl, yp, size, n, scale, lp, dxp, dxc, dxl, dwp, dwc, dwl,
                   _stream(stream))


class Muon(_Handle):
    """Momentum updates made orthogonal by Newton-Schulz products (fc_muon), for
    the matrices of a flat vector.

    matrices: rows (offset, rows, cols[, lr_mult, decay_mult]) in elements of
              the vector, sorted, as Plan's segments are.
    dtype   : of orthogonalize's output, and the accuracy of the products: "bf16"
              (16-bit products) or "f16", "f32" (fp32's accuracy, 3 times the work).
    coefficients: (a, b, c) of X <- a X + (b A + c A A) X, A = X X^T."""

    _destroy = "fc_muon_destroy"

    def __init__(self, matrices, dtype="bf16", steps=5, coefficients=None, nesterov=True):
        if dtype not in DTYPES:
            raise ValueError(f"dtype must be f32, f16 or bf16, not {dtype}")
        matrices = [tuple(m) for m in matrices]
        table = (fc_matrix * max(1, len(matrices)))()
        self.extent = 0
        for i, m in enumerate(matrices):
            if not 3 <= len(m) <= 5 or min(m[:3]) < 0:
                raise ValueError(f"matrix {i} is {m}, not (offset, rows, cols[, lr_mult, decay_mult])")
            table[i] = fc_matrix(*m[:3], *(m[3:] + (1.0, 1.0)[len(m) - 3:]))
            self.extent = max(self.extent, m[0] + m[1] * m[2])
        abc = None if coefficients is None else (ctypes.c_double * 3)(*coefficients)
        self.code = DTYPES[dtype]
        self._create("fc_muon_create", table, len(matrices), self.code, steps, abc, bool(nesterov))

    def _flat(self, t, name, code=None):
        _tensor(t, name)
        got = _CODES.get(t.dtype)
        if got is None or (code is not None and got != code):
            raise ValueError(f"{name} must not be {t.dtype}")
        if t.device != self.device:
            raise ValueError(f"{name} is on {t.device}, the plan on {self.device}")
        if not t.is_contiguous() or t.numel() < self.extent:
            raise ValueError(f"{name} must be contiguous and hold the plan's {self.extent} elements")
        return t.data_ptr(), got

    def orthogonalize(self, g, out, stream=None):
        """out = the Newton-Schulz steps of g, matrix by matrix."""
        gp, gc = self._flat(g, "g")
        op, _ = self._flat(out, "out", self.code)
        self._call("fc_muon_orthogonalize", gp, gc, op, _stream(stream))

    def step(self, w, v, g, lr, mu, wd, batch, stream=None):
        """v' = mu v + g / batch, O = the steps of g / batch + mu v' (of v'
        without nesterov), w' = w - lr (sqrt(max(1, rows / cols)) O + wd w) for
        the plan's matrices; g is a raw sum, as Plan.sgd_step takes it."""
        wp, _ = self._flat(w, "w", FC_F32)
        vp, _ = self._flat(v, "v", FC_F32)
        gp, _ = self._flat(g, "g", FC_F32)
        self._call("fc_muon_step", wp, vp, gp, lr, mu, wd, int(batch), _stream(stream))


_KINDS = {"rms": FC_NORM_RMS, "layer": FC_NORM_LAYER}
_GATES = {"none": FC_GATE_NONE, "sigmoid": FC_GATE_SIGMOID, "silu": FC_GATE_SILU}


class Norm(_Handle):
    """The norms before and after a block of a model, with its gate and residual
    scale (fc_norm), for rows of `dim` elements (at most 16384); gradients of up to
    `max_tokens` rows.

    dtype   : of the block's side: b, y, dy, db and a gate given per token
    residual: of the residual's side: h, x, out, dout, dh, dx; `dtype` or "f32"
    kind    : "rms", x / sqrt(mean(x^2) + eps), or "layer", the same of x - mean(x)
    gate    : what a gate g multiplies by: "none", g itself, "sigmoid" or "silu"

    Weights are f32 vectors, None is 1; a gate is None (1), an f32 vector or a
    (tokens, dim) tensor of the block's type.  Vectors' gradients are f32, f16 or
    bf16, all of a call's of one type; with `accumulate` they are added to.  A
    gradient given as None is not computed."""

    _destroy = "fc_norm_destroy"

    def __init__(self, dim, max_tokens, dtype="f16", residual="f32", kind="rms", eps=1e-6, gate="none"):
        for name, value, known in (("dtype", dtype, DTYPES), ("residual", residual, DTYPES), ("kind", kind, _KINDS),
                                   ("gate", gate, _GATES)):
            if value not in known:
                raise ValueError(f"{name} must be one of {', '.join(known)}, not {value}")
        if residual not in (dtype, "f32"):
            raise ValueError(f"residual must be {dtype} or f32, not {residual}")
        import torch
        self._create("fc_norm_create", dim, max_tokens, DTYPES[dtype], DTYPES[residual], _KINDS[kind], eps, _GATES[gate])
        self.dim, self.max_tokens = dim, max_tokens
        types = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
        self.block, self.residual, self.vector = types[dtype], types[residual], torch.float32

    def _weight(self, t, name):
        return None if t is None else _typed_vector(t, name, self.dim, self.vector, self.device)

    def _gate(self, t, n):
        """(pointer, row stride or 0 for a vector)."""
        if t is None:
            return None, 0
        if getattr(t, "ndim", 2) == 1:
            return _typed_vector(t, "gate", self.dim, self.vector, self.device), 0
        return _typed(t, "gate", n, self.dim, self.block, self.device)

    def _sums(self, gate, n, dgate, weight, next_weight=None):
        """Gradients of vectors, all of one type, and of the gate: (the type, the weights' pointers, dgate's pointer and
        row stride)."""
        of_vector = False
        if dgate is not None:
            if gate is None or getattr(dgate, "ndim", -1) != gate.ndim:
                raise ValueError("dgate must be a vector or rows as gate is")
            of_vector = gate.ndim == 1
        first = weight if weight is not None else next_weight if next_weight is not None else dgate if of_vector else None
        dtype = getattr(first, "dtype", self.vector)
        if dtype not in _CODES:
            raise ValueError(f"vectors' gradients must not be {dtype}")
        dim, dev, place = self.dim, self.device, (None, 0)
        wp = None if weight is None else _typed_vector(weight, "dweight", dim, dtype, dev)
        np_ = None if next_weight is None else _typed_vector(next_weight, "dnext", dim, dtype, dev)
        if of_vector:
            place = _typed_vector(dgate, "dgate", dim, dtype, dev), 0
        elif dgate is not None:
            place = _typed(dgate, "dgate", n, dim, self.block, dev)
        return _CODES[dtype], wp, np_, place

    def _tokens(self, t, name):
        n = _rows(t, name)
        if n > self.max_tokens:
            raise ValueError(f"{n} tokens for a plan of {self.max_tokens}")
        return n

    def before(self, x, y, weight=None, stream=None):
        """y[t] = weight * N(x[t])."""
        n, dim, dev = _rows(x, "x"), self.dim, self.device
        xp, xl = _typed(x, "x", n, dim, self.residual, dev)
        yp, yl = _typed(y, "y", n, dim, self.block, dev)
        wp = self._weight(weight, "weight")
        self._call("fc_norm_before", xp, xl, n, wp, yp, yl, _stream(stream))

    def after(self, h, b, out, weight=None, gate=None, scale=1.0, stream=None):
        """out[t] = h[t] + scale * a(gate) * weight * N(b[t])."""
        n, dim, dev = _rows(h, "h"), self.dim, self.device
        hp, hl = _typed(h, "h", n, dim, self.residual, dev)
        bp, bl = _typed(b, "b", n, dim, self.block, dev)
        op, ol = _typed(out, "out", n, dim, self.residual, dev)
        gp, gl = self._gate(gate, n)
        wp = self._weight(weight, "weight")
        self._call("fc_norm_after", hp, hl, bp, bl, n, gp, gl, wp, scale, op, ol, _stream(stream))

    def between(self, h, b, out, y, weight=None, gate=None, next_weight=None, scale=1.0, stream=None):
        """out as after()'s, and y[t] = next_weight * N(out[t]) of out as it is stored."""
        n, dim, dev = _rows(h, "h"), self.dim, self.device
        hp, hl = _typed(h, "h", n, dim, self.residual, dev)
        bp, bl = _typed(b, "b", n, dim, self.block, dev)
        op, ol = _typed(out, "out", n, dim, self.residual, dev)
        yp, yl = _typed(y, "y", n, dim, self.block, dev)
        gp, gl = self._gate(gate, n)
        wp = self._weight(weight, "weight")
        np_ = self._weight(next_weight, "next_weight")
        self._call("fc_norm_between", hp, hl, bp, bl, n, gp, gl, wp, np_, scale, op, ol, yp, yl, _stream(stream))

    def before_grad(self, x, dy, dx, dout=None, weight=None, dweight=None, accumulate=False, stream=None):
        """The gradients of before(): dx, to which dout, the gradient that comes by the
        residual, is added, and dweight."""
        n, dim, dev = self._tokens(x, "x"), self.dim, self.device
        xp, xl = _typed(x, "x", n, dim, self.residual, dev)
        yp, yl = _typed(dy, "dy", n, dim, self.block, dev)
        op, ol = (None, 0) if dout is None else _typed(dout, "dout", n, dim, self.residual, dev)
        dp, dl = _typed(dx, "dx", n, dim, self.residual, dev)
        wp = self._weight(weight, "weight")
        code, dwp, _, _ = self._sums(None, n, None, dweight)
        self._call("fc_norm_before_grad", xp, xl, yp, yl, op, ol, n, wp, dp, dl, dwp, code, bool(accumulate), _stream(stream))

    def after_grad(self, b, dout, db, weight=None, dweight=None, gate=None, dgate=None, scale=1.0, accumulate=False,
                   stream=None):
        """The gradients of after() by b, gate and weight; that by h is dout itself."""
        n, dim, dev = self._tokens(b, "b"), self.dim, self.device
        bp, bl = _typed(b, "b", n, dim, self.block, dev)
        op, ol = (None, 0) if dout is None else _typed(dout, "dout", n, dim, self.residual, dev)
        gp, gl = self._gate(gate, n)
        dp, dl = _typed(db, "db", n, dim, self.block, dev)
        wp = self._weight(weight, "weight")
        code, dwp, _, (dgp, dgl) = self._sums(gate, n, dgate, dweight)
        self._call("fc_norm_after_grad", bp, bl, op, ol, n, gp, gl, wp, scale, dp, dl, dgp, dgl, dwp, code, bool(accumulate),
                   _stream(stream))

    def between_grad(self, out, b, dy, dh, db, dout=None, weight=None, dweight=None, gate=None, dgate=None, next_weight=None,
                     dnext=None, scale=1.0, accumulate=False, stream=None):
        """The gradients of between(), of both its outputs: dh, db and the vectors' and
        gate's."""
        n, dim, dev = self._tokens(out, "out"), self.dim, self.device
        xp, xl = _typed(out, "out", n, dim, self.residual, dev)
        bp, bl = _typed(b, "b", n, dim, self.block, dev)
        yp, yl = _typed(dy, "dy", n, dim, self.block, dev)
        op, ol = (None, 0) if dout is None else _typed(dout, "dout", n, dim, self.residual, dev)
        gp, gl = self._gate(gate, n)
        hp, hl = _typed(dh, "dh", n, dim, self.residual, dev)
        dp, dl = _typed(db, "db", n, dim, self.block, dev)
        wp, np_ = self._weight(weight, "weight"), self._weight(next_weight, "next_weight")
        code, dwp, dnp, (dgp, dgl) = self._sums(gate, n, dgate, dweight, dnext)
        self._call("fc_norm_between_grad", xp, xl, bp, bl, yp, yl, op, ol, n, gp, gl, wp, np_, scale, hp, hl, dp, dl, dgp, dgl,
                   dwp, dnp, code, bool(accumulate), _stream(stream))


_BLOCK = 32  # neighbours of a row that share a scale
_FORMATS = {"i8": FC_BLOCK_I8, "e4m3": FC_BLOCK_E4M3}


class Checkpoint(_Handle):
    """Activations (tokens, dim) kept in 8 bits, 32 neighbours of a row to a scale
    (fc_ckpt), and what a backward pass needs of them: the activations themselves,
    and the gradient of a weight of up to `max_outs` rows from up to `max_tokens`
    tokens and a dy of `dtype` ("f16" or "bf16").

    format: "i8", steps of 1/63 to 1/128 of the 32's largest magnitude, or "e4m3",
            4 bits of each element.  A block with an infinity or NaN is kept as NaN.

    They are held by two tensors of the caller's, codes (tokens, 32 ceil(dim / 32))
    of torch.int8 or torch.float8_e4m3fn on 16 bytes with a row stride of a multiple of 16,
    and scales (tokens, ceil(dim / 32)) of torch.uint8, the exponents of powers of two plus
    127, as empty() makes them.  Layers of one dim can share a plan, which holds the workspace
    of a gradient: two bytes for every element of max_tokens activations."""

    _destroy = "fc_ckpt_destroy"

    def __init__(self, dim, max_tokens, max_outs=0, dtype="f16", format="i8"):
        import torch
        if dtype not in ("f16", "bf16"):
            raise ValueError(f"dtype must be f16 or bf16, not {dtype}")
        if format not in _FORMATS:
            raise ValueError(f"format must be i8 or e4m3, not {format}")
        self._create("fc_ckpt_create", dim, max_tokens, max_outs, DTYPES[dtype], _FORMATS[format])
        self.dim, self.max_tokens, self.max_outs = dim, max_tokens, max_outs
        self.blocks = -(-dim // _BLOCK)
        self.dtype = torch.float16 if dtype == "f16" else torch.bfloat16
        self.types = torch.int8 if format == "i8" else torch.float8_e4m3fn, torch.uint8  # of codes and scales

    def empty(self, n):
        """Codes and scales for n tokens."""
        import torch
        return tuple(torch.empty((n, w), dtype=t, device=self.device) for w, t in zip((_BLOCK * self.blocks, self.blocks), self.types))

    def pack(self, x, codes, scales, stream=None):
        """Codes and scales of x (tokens, dim), f32, f16 or bf16; any number of tokens."""
        n, dev = _rows(x, "x"), self.device
        xp, xc, xl = _matrix(x, "x", n, self.dim, dev)
        cp, cl = _typed(codes, "codes", n, _BLOCK * self.blocks, self.types[0], dev)
        sp, sl = _typed(scales, "scales", n, self.blocks, self.types[1], dev)
        self._call("fc_ckpt_pack", xp, xc, xl, n, cp, cl, sp, sl, _stream(stream))

    def unpack(self, codes, scales, out, stream=None):
        """out = the activations kept, rounded to its type."""
        n, dev = _rows(out, "out"), self.device
        op, oc, ol = _matrix(out, "out", n, self.dim, dev)
        cp, cl = _typed(codes, "codes", n, _BLOCK * self.blocks, self.types[0], dev)
        sp, sl = _typed(scales, "scales", n, self.blocks, self.types[1], dev)
        self._call("fc_ckpt_unpack", cp, cl, sp, sl, n, op, oc, ol, _stream(stream))

    def grad(self, dy, codes, scales, dw, scale=1.0, accumulate=False, stream=None):
        """dw[o] = (dw[o] if accumulate else 0) + scale * the sum over t of dy[t, o] x[t],
        for dy (tokens, outs) and dw (outs, dim) of any type.  dy lies on 16 bytes with a row
        stride of a multiple of 8, unless max_outs is no multiple of 8."""
        n, outs, dev = _rows(dy, "dy"), _rows(dw, "dw"), self.device
        if n > self.max_tokens:
            raise ValueError(f"{n} tokens for a plan of {self.max_tokens}")
        if outs > self.max_outs:
            raise ValueError(f"{outs} outputs for a plan of {self.max_outs}")
        yp, yl = _typed(dy, "dy", n, outs, self.dtype, dev)
        gp, gc, gl = _matrix(dw, "dw", outs, self.dim, dev)
        cp, cl = _typed(codes, "codes", n, _BLOCK * self.blocks, self.types[0], dev)
        sp, sl = _typed(scales, "scales", n, self.blocks, self.types[1], dev)
        if n <= 1:
            yl = -(-yl // 8) * 8  # the stride of one row says nothing
        self._call("fc_ckpt_grad", yp, yl, cp, cl, sp, sl, n, outs, scale, gp, gc, gl, bool(accumulate), _stream(stream))


class Mxfp4(_Handle):
    """Products along `dim` with a matrix of `rows` rows, both operands in 4-bit floating
    point with a scale for every 32 along the rows (fc_mxfp, MXFP4), for up to `max_tokens`
    rows a call: a layer's outputs from a weight (rows, dim), or, with a plan of the sizes
    exchanged and the weight packed with `transpose`, the gradient of its inputs.

    A packed matrix is held by two tensors of the caller's, of torch.uint8: codes (r, 16
    ceil(dim / 32)), the even element in a byte's low half, on 16 bytes with a row stride of a
    multiple of 16, and scales (r, 8 ceil(dim / 256)), zeros past the blocks, on 8 bytes with
    a stride of a multiple of 8, as empty() makes them.  Matrices of the same sizes can share
    a plan."""

    _destroy = "fc_mxfp_destroy"

    def __init__(self, rows, dim, max_tokens):
        import torch
        self._create("fc_mxfp_create", rows, dim, max_tokens)
        self.rows, self.dim, self.max_tokens = rows, dim, max_tokens
        self.widths = 16 * -(-dim // _BLOCK), 8 * -(-dim // (8 * _BLOCK))  # of codes and scales
        self.type = torch.uint8

    def empty(self, n):
        """Codes and scales for n rows."""
        import torch
        return tuple(torch.empty((n, w), dtype=self.type, device=self.device) for w in self.widths)

    def _packed(self, codes, scales, n, name=""):
        return (*_typed(codes, name + "codes", n, self.widths[0], self.type, self.device),
                *_typed(scales, name + "scales", n, self.widths[1], self.type, self.device))

    def _tokens(self, t, name):
        n = _rows(t, name)
        if n > self.max_tokens:
            raise ValueError(f"{n} tokens for a plan of {self.max_tokens}")
        return n

    def pack(self, x, codes, scales, transpose=False, stream=None):
        """Codes and scales of x (n, dim) or, with `transpose`, of the columns of x (dim, n);
        f32, f16 or bf16, any n."""
        n = _rows(codes, "codes")
        xp, xc, xl = _matrix(x, "x", *((self.dim, n) if transpose else (n, self.dim)), self.device)
        self._call("fc_mxfp_pack", xp, xc, xl, n, bool(transpose), *self._packed(codes, scales, n), _stream(stream))

    def unpack(self, codes, scales, out, stream=None):
        """out (n, dim) = the numbers kept, rounded to its type."""
        n = _rows(out, "out")
        op, oc, ol = _matrix(out, "out", n, self.dim, self.device)
        self._call("fc_mxfp_unpack", *self._packed(codes, scales, n), n, op, oc, ol, _stream(stream))

    def product(self, a_codes, a_scales, b_codes, b_scales, out, scale=1.0, accumulate=False, stream=None):
        """out (n, rows) = (out if accumulate else 0) + scale * a b^T, of packed a (n, dim) and
        b (rows, dim)."""
        n = self._tokens(out, "out")
        op, oc, ol = _matrix(out, "out", n, self.rows, self.device)
        self._call("fc_mxfp_product", *self._packed(a_codes, a_scales, n, "a_"), n,
                   *self._packed(b_codes, b_scales, self.rows, "b_"), scale, op, oc, ol, bool(accumulate), _stream(stream))

    def linear(self, x, codes, scales, out, scale=1.0, accumulate=False, stream=None):
        """product() of x (n, dim), f32, f16 or bf16, packed on the way, and a packed weight."""
        n, rows, dev = self._tokens(x, "x"), self.rows, self.device
        xp, xc, xl = _matrix(x, "x", n, self.dim, dev)
        op, oc, ol = _matrix(out, "out", n, rows, dev)
        cp, cl = _typed(codes, "codes", rows, self.widths[0], self.type, dev)
        sp, sl = _typed(scales, "scales", rows, self.widths[1], self.type, dev)
        self._call("fc_mxfp_linear", xp, xc, xl, n, cp, cl, sp, sl, scale, op, oc, ol, bool(accumulate), _stream(stream))
