"""conv1d_embed_t, conv1d_norm_t and conv1d_dropout_t of include/conv1d.h, as a C caller fills them."""
import ctypes


class Embed(ctypes.Structure):
    _fields_ = ([(k, ctypes.c_void_p) for k in ("tokens", "lengths")] + [("tok_sn", ctypes.c_long)] +
                [(k, ctypes.c_int) for k in ("N", "D", "L", "V", "dtype", "flags")] + [("scale", ctypes.c_float)])


class Norm(ctypes.Structure):
    _fields_ = ([(k, ctypes.c_void_p) for k in ("x", "weight", "bias", "lengths")] + [(k, ctypes.c_long) for k in ("x_sn", "x_sc", "x_sl")] +
                [("eps", ctypes.c_double)] + [(k, ctypes.c_int) for k in ("N", "C", "L", "G", "dtype", "flags")])


class Dropout(ctypes.Structure):
    _fields_ = ([(k, ctypes.c_void_p) for k in ("x", "residual", "lengths", "counter")] + [(k, ctypes.c_long) for k in ("x_sn", "x_sc", "r_sn", "r_sc")] +
                [(k, ctypes.c_ulong) for k in ("key", "call")] + [("p", ctypes.c_double)] + [(k, ctypes.c_int) for k in ("N", "C", "L", "dtype")])
