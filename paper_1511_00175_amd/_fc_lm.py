"""ctypes binding of libfc_lm.so (include/fc_lm.h), argument marshalling only,
as _fc.py is for libfc.so.  If the library is missing the import fails: there
is no other implementation to fall back to."""
import ctypes
import os

from ._fc import PKG

LIB_PATH = os.path.join(PKG, "libfc_lm.so")
FC_BF16 = 2
FC_NORM_RMS, FC_NORM_LAYER = 0, 1
FC_BLOCK_I8, FC_BLOCK_E4M3 = 0, 1
FC_GATE_NONE, FC_GATE_SIGMOID, FC_GATE_SILU = 0, 1, 2


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
lib.fc_norm_create.argtypes = [_pp, _l, _l, _i, _i, _i, _f, _i]
lib.fc_norm_destroy.argtypes = [_vp]
lib.fc_norm_destroy.restype = None
lib.fc_norm_before.argtypes = [_vp, _vp, _l, _l, _vp, _vp, _l, _vp]
lib.fc_norm_after.argtypes = [_vp, _vp, _l, _vp, _l, _l, _vp, _l, _vp, _f, _vp, _l, _vp]
lib.fc_norm_between.argtypes = [_vp, _vp, _l, _vp, _l, _l, _vp, _l, _vp, _vp, _f, _vp, _l, _vp, _l, _vp]
lib.fc_norm_before_grad.argtypes = [_vp, _vp, _l, _vp, _l, _vp, _l, _l, _vp, _vp, _l, _vp, _i, _i, _vp]
lib.fc_norm_after_grad.argtypes = [_vp, _vp, _l, _vp, _l, _l, _vp, _l, _vp, _f, _vp, _l, _vp, _l, _vp, _i, _i, _vp]
lib.fc_norm_between_grad.argtypes = [_vp, _vp, _l, _vp, _l, _vp, _l, _vp, _l, _l, _vp, _l, _vp, _vp, _f, _vp, _l, _vp, _l,
                                     _vp, _l, _vp, _vp, _i, _i, _vp]
lib.fc_ckpt_create.argtypes = [_pp, _l, _l, _l, _i, _i]
lib.fc_ckpt_destroy.argtypes = [_vp]
lib.fc_ckpt_destroy.restype = None
lib.fc_ckpt_pack.argtypes = [_vp, _vp, _i, _l, _l, _vp, _l, _vp, _l, _vp]
lib.fc_ckpt_unpack.argtypes = [_vp, _vp, _l, _vp, _l, _l, _vp, _i, _l, _vp]
lib.fc_ckpt_grad.argtypes = [_vp, _vp, _l, _vp, _l, _vp, _l, _l, _l, _f, _vp, _i, _l, _i, _vp]
lib.fc_mxfp_create.argtypes = [_pp, _l, _l, _l]
lib.fc_mxfp_destroy.argtypes = [_vp]
lib.fc_mxfp_destroy.restype = None
lib.fc_mxfp_pack.argtypes = [_vp, _vp, _i, _l, _l, _i, _vp, _l, _vp, _l, _vp]
lib.fc_mxfp_unpack.argtypes = [_vp, _vp, _l, _vp, _l, _l, _vp, _i, _l, _vp]
lib.fc_mxfp_product.argtypes = [_vp, _vp, _l, _vp, _l, _l, _vp, _l, _vp, _l, _f, _vp, _i, _l, _i, _vp]
lib.fc_mxfp_linear.argtypes = [_vp, _vp, _i, _l, _l, _vp, _l, _vp, _l, _f, _vp, _i, _l, _i, _vp]
for _n in ("fc_embed_create", "fc_embed_lookup", "fc_embed_grad", "fc_xent_create", "fc_xent_loss", "fc_xent_loss_grad",
           "fc_muon_create", "fc_muon_orthogonalize", "fc_muon_step", "fc_norm_create", "fc_norm_before", "fc_norm_after",
           "fc_norm_between", "fc_norm_before_grad", "fc_norm_after_grad", "fc_norm_between_grad", "fc_ckpt_create",
           "fc_ckpt_pack", "fc_ckpt_unpack", "fc_ckpt_grad", "fc_mxfp_create", "fc_mxfp_pack", "fc_mxfp_unpack",
           "fc_mxfp_product", "fc_mxfp_linear"):
    getattr(lib, _n).restype = _i
