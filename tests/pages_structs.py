"""ctypes mirrors of the structures in include/ress_pages.h."""
import ctypes as C

from layer_structs import ress_rope_shape, ress_strides


class ress_page_strides(C.Structure):
    _fields_ = [("page", C.c_int64), ("head", C.c_int64), ("token", C.c_int64)]


class ress_head_norm_shape(C.Structure):
    _fields_ = [("rope", ress_rope_shape), ("norm", C.c_int), ("eps", C.c_double)]


class ress_page_cache(C.Structure):
    _fields_ = [("n_pages", C.c_int), ("page", C.c_int), ("k", ress_page_strides), ("v", ress_page_strides),
                ("v_in", ress_strides)]


class ress_head_norm_grads(C.Structure):
    _fields_ = [("dq_out", ress_strides), ("dk_out", ress_strides), ("dq", ress_strides), ("dk", ress_strides)]


class ress_table_shape(C.Structure):
    _fields_ = [("B", C.c_int), ("N", C.c_int), ("page", C.c_int), ("n_pages", C.c_int), ("max_pages", C.c_int),
                ("table_stride", C.c_int64), ("clear", C.c_int)]


class ress_paged_shape(C.Structure):
    _fields_ = [("B", C.c_int), ("N", C.c_int), ("H", C.c_int), ("H_kv", C.c_int), ("D", C.c_int), ("page", C.c_int),
                ("n_pages", C.c_int), ("max_pages", C.c_int), ("frame", C.c_int), ("window", C.c_int), ("n_sink", C.c_int),
                ("table_stride", C.c_int64), ("q", ress_strides), ("o", ress_strides), ("k", ress_page_strides),
                ("v", ress_page_strides)]
