"""The structures of the second half of include/sprnn.h for ctypes: the tests' own reading of the header."""
import ctypes


class Seq(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("step", ctypes.c_int64), ("sample", ctypes.c_int64)]


class Scan(ctypes.Structure):
    _fields_ = [("steps", ctypes.c_int), ("batch", ctypes.c_int), ("channels", ctypes.c_int), ("states", ctypes.c_int),
                ("groups", ctypes.c_int), ("type", ctypes.c_int), ("softplus", ctypes.c_int),
                ("u", Seq), ("dt", Seq), ("z", Seq), ("B", Seq), ("C", Seq),
                ("A", ctypes.c_void_p), ("D", ctypes.c_void_p), ("dt_bias", ctypes.c_void_p), ("lengths", ctypes.c_void_p)]


class ScanGradientBuffers(ctypes.Structure):
    _fields_ = [("u", Seq), ("dt", Seq), ("z", Seq), ("B", Seq), ("C", Seq),
                ("A", ctypes.c_void_p), ("D", ctypes.c_void_p), ("dt_bias", ctypes.c_void_p), ("state", ctypes.c_void_p)]


class Conv(ctypes.Structure):
    _fields_ = [("steps", ctypes.c_int), ("batch", ctypes.c_int), ("channels", ctypes.c_int), ("width", ctypes.c_int),
                ("type", ctypes.c_int), ("silu", ctypes.c_int), ("x", Seq),
                ("weight", ctypes.c_void_p), ("bias", ctypes.c_void_p), ("state", ctypes.c_void_p), ("lengths", ctypes.c_void_p)]


class Norm(ctypes.Structure):
    _fields_ = [("steps", ctypes.c_int), ("batch", ctypes.c_int), ("width", ctypes.c_int), ("type", ctypes.c_int),
                ("residual_type", ctypes.c_int), ("eps", ctypes.c_float), ("weight", ctypes.c_void_p)]


class Product(ctypes.Structure):
    _fields_ = [("steps", ctypes.c_int), ("batch", ctypes.c_int), ("rows", ctypes.c_int), ("inputs", ctypes.c_int),
                ("x", Seq), ("x_scales", ctypes.c_void_p), ("w", ctypes.c_void_p), ("w_scales", ctypes.c_void_p),
                ("bias", ctypes.c_void_p)]
