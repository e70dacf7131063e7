"""conv1d_causal_t and conv1d_scan_t of include/conv1d.h, as a C caller fills them."""
import ctypes


class Causal(ctypes.Structure):
    _fields_ = ([(k, ctypes.c_void_p) for k in ("x", "w", "bias", "init", "lengths")] + [(k, ctypes.c_long) for k in ("x_sn", "x_sc")] +
                [(k, ctypes.c_int) for k in ("N", "C", "L", "S", "dtype", "flags")])


class Scan(ctypes.Structure):
    _fields_ = ([(k, ctypes.c_void_p) for k in ("x", "dt", "B", "C", "z", "A", "skip", "dt_bias", "init", "lengths")] +
                [(k, ctypes.c_long) for k in ("x_sn", "x_sd", "dt_sn", "dt_sd", "z_sn", "z_sd", "b_sn", "b_sg", "b_ss", "c_sn", "c_sg", "c_ss")] +
                [(k, ctypes.c_int) for k in ("N", "D", "L", "S", "G", "dtype", "flags")])
