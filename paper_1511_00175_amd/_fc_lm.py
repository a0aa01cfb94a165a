"""ctypes binding of libfc_lm.so (include/fc_lm.h), argument marshalling only,
as _fc.py is for libfc.so.  If the library is missing the import fails: there
is no other implementation to fall back to."""
import ctypes
import os

from ._fc import PKG

LIB_PATH = os.path.join(PKG, "libfc_lm.so")
FC_BF16 = 2


class fc_matrix(ctypes.Structure):
    _fields_ = [("offset", ctypes.c_uint64), ("rows", ctypes.c_uint64), ("cols", ctypes.c_uint64),
                ("lr_mult", ctypes.c_float), ("decay_mult", ctypes.c_float)]


if not os.path.exists(LIB_PATH):
    raise ImportError(f"{LIB_PATH} is not built; run __graft_entry__.build() or "
                      "python paper_1511_00175_amd/build.py")

lib = ctypes.CDLL(LIB_PATH)

_vp, _i, _l, _f = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_float
_pp = ctypes.POINTER(ctypes.c_void_p)

lib.fc_embed_create.argtypes = [_pp, _l, _l, _l]
lib.fc_embed_destroy.argtypes = [_vp]
lib.fc_embed_destroy.restype = None
lib.fc_embed_lookup.argtypes = [_vp, _vp, _i, _l, _vp, _i, _l, _f, _vp, _i, _l, _vp]
lib.fc_embed_grad.argtypes = [_vp, _vp, _i, _l, _vp, _i, _l, _f, _vp, _i, _l, _i, _vp]
lib.fc_xent_create.argtypes = [_pp, _l, _l, _l, _i, _l]
lib.fc_xent_destroy.argtypes = [_vp]
lib.fc_xent_destroy.restype = None
lib.fc_xent_loss.argtypes = [_vp, _vp, _l, _vp, _l, _vp, _i, _l, _vp, _vp]
lib.fc_xent_loss_grad.argtypes = [_vp, _vp, _l, _vp, _l, _vp, _i, _l, _f, _vp, _vp, _i, _l, _vp, _i, _l, _vp]
lib.fc_muon_create.argtypes = [_pp, ctypes.POINTER(fc_matrix), _i, _i, _i, ctypes.POINTER(ctypes.c_double), _i]
lib.fc_muon_destroy.argtypes = [_vp]
lib.fc_muon_destroy.restype = None
lib.fc_muon_orthogonalize.argtypes = [_vp, _vp, _i, _vp, _vp]
lib.fc_muon_step.argtypes = [_vp, _vp, _vp, _vp, _f, _f, _f, _i, _vp]
for _n in ("fc_embed_create", "fc_embed_lookup", "fc_embed_grad", "fc_xent_create", "fc_xent_loss", "fc_xent_loss_grad",
           "fc_muon_create", "fc_muon_orthogonalize", "fc_muon_step"):
    getattr(lib, _n).restype = _i
