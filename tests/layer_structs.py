"""ctypes mirrors of the structures in include/ress_layer.h."""
import ctypes as C


class ress_strides(C.Structure):
    _fields_ = [("head", C.c_int64), ("token", C.c_int64)]


class ress_norm_shape(C.Structure):
    _fields_ = [("rows", C.c_int64), ("width", C.c_int), ("x_dtype", C.c_int), ("y_dtype", C.c_int),
                ("x_stride", C.c_int64), ("y_stride", C.c_int64), ("eps", C.c_double)]


class ress_rope_shape(C.Structure):
    _fields_ = [("H", C.c_int), ("H_kv", C.c_int), ("N", C.c_int), ("D", C.c_int), ("n_axes", C.c_int),
                ("dims", C.c_int * 4), ("layout", C.c_int), ("inverse", C.c_int), ("dtype", C.c_int),
                ("base", C.c_double), ("q", ress_strides), ("k", ress_strides), ("q_out", ress_strides),
                ("k_out", ress_strides)]


class ress_window_shape(C.Structure):
    _fields_ = [("H", C.c_int), ("H_kv", C.c_int), ("n_q", C.c_int), ("n_k", C.c_int), ("D", C.c_int),
                ("q_offset", C.c_int), ("frame", C.c_int), ("window", C.c_int), ("n_sink", C.c_int),
                ("causal", C.c_int), ("q", ress_strides), ("k", ress_strides), ("v", ress_strides),
                ("o", ress_strides)]


class ress_window_grads(C.Structure):
    _fields_ = [("d_o", ress_strides), ("dq", ress_strides), ("dk", ress_strides), ("dv", ress_strides)]


class ress_decode_shape(C.Structure):
    _fields_ = [("B", C.c_int), ("H", C.c_int), ("H_kv", C.c_int), ("capacity", C.c_int), ("D", C.c_int),
                ("frame", C.c_int), ("window", C.c_int), ("n_sink", C.c_int), ("q_batch", C.c_int64),
                ("q_head", C.c_int64), ("k_batch", C.c_int64), ("v_batch", C.c_int64), ("k", ress_strides),
                ("v", ress_strides), ("o_batch", C.c_int64), ("o_head", C.c_int64)]
