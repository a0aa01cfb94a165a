"""The operators at the ends of a language model and of its matrix update
(include/fc_lm.h) on torch tensors: they produce the gradients that Plan
aggregates, or consume their sum.  As Plan does, each class checks every buffer
before it calls the C ABI, which sees only pointers, and enqueues on the given
stream or torch's current one."""
import ctypes

from ._fc import FC_F16, FC_F32, FcError
from ._fc_lm import FC_BF16, fc_matrix, lib

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


_current = None  # the package's _stream, once it is loaded


def _stream(stream):
    global _current
    if _current is None:
        from . import _stream as _current
    return _current(stream)


_FUNCTIONS = {n: getattr(lib, n) for n in ("fc_embed_lookup", "fc_embed_grad", "fc_xent_loss", "fc_xent_loss_grad",
                                           "fc_muon_orthogonalize", "fc_muon_step")}


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
