"""The operators at the ends of a language model and of its matrix update
(include/fc_lm.h) on torch tensors: they produce the gradients that Plan
aggregates, or consume their sum.  As Plan does, each class checks every buffer
before it calls the C ABI, which sees only pointers, and enqueues on the given
stream or torch's current one."""
import ctypes

from ._fc import FC_F16, FC_F32, FcError
from ._fc_lm import FC_BF16, lib

DTYPES = {"f32": FC_F32, "f16": FC_F16, "bf16": FC_BF16}
_CODES = None  # torch dtype -> fc_dtype value, made at the first call


def _code(t):
    global _CODES
    if _CODES is None:
        import torch
        _CODES = {torch.float32: FC_F32, torch.float16: FC_F16, torch.bfloat16: FC_BF16}
    return _CODES.get(t.dtype)


def _matrix(t, name, rows, cols, device, code=None):
    """`t` must be a (rows, cols) tensor of a supported type (`code`: of that
    one) on the device, its rows contiguous and any distance apart; returns
    (pointer, type, row stride)."""
    import torch
    if not isinstance(t, torch.Tensor):
        raise ValueError(f"{name} must be a torch tensor")
    got = _code(t)
    if got is None or (code is not None and got != code):
        raise ValueError(f"{name} must not be {t.dtype}")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, the plan on {device}")
    if t.dim() != 2 or t.shape[0] != rows or t.shape[1] != cols:
        raise ValueError(f"{name} is {tuple(t.shape)}, not {(rows, cols)}")
    ld = t.stride(0) if rows > 1 else cols
    if (cols > 1 and t.stride(1) != 1) or ld < cols:
        raise ValueError(f"{name} must have contiguous rows that do not overlap")
    return t.data_ptr(), got, ld


def _list(t, name, device):
    """`t` must be a contiguous vector of int32 or int64 on the device; returns
    (pointer, bytes of an entry, length)."""
    import torch
    if not isinstance(t, torch.Tensor):
        raise ValueError(f"{name} must be a torch tensor")
    if t.dtype not in (torch.int32, torch.int64):
        raise ValueError(f"{name} must be int32 or int64, not {t.dtype}")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, the plan on {device}")
    if t.dim() != 1 or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous vector")
    return t.data_ptr(), t.element_size(), t.shape[0]


def _stream(stream):
    from . import _stream as current
    return current(stream)


class _Handle:
    """A plan of the library: created by `make`, freed by close() or garbage
    collection, after the device's work is done."""

    handle = None

    def _create(self, make, *args):
        import torch
        h = ctypes.c_void_p()
        rc = getattr(lib, make)(ctypes.byref(h), *args)
        if rc:
            raise FcError(make, rc)
        self.handle = h
        self.device = torch.device("cuda", torch.cuda.current_device())

    def _call(self, name, *args):
        rc = getattr(lib, name)(self.handle, *args)
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
