"""The structures of include/grid.h for trees, sampling and pages, field by
field, for tests that call the library with arguments of their own."""
import ctypes

from paper_2607_11951_gb300.grid import _fields


class Tree(ctypes.Structure):
    _fields_ = _fields(d_parent="p", d_start="p", B="i", n_tokens="i")


class SampleStep(ctypes.Structure):
    _fields_ = _fields(d_logits="p", logit_stride="l", d_mask="p", mask_stride="l", d_noise="p", noise_stride="l",
                       d_temperature="p", d_top_k="p", d_top_p="p", d_min_p="p", dtype="i", B="i", V="i", eos="i",
                       d_tokens="p", d_logprob="p", d_status="p")


class PagesStep(ctypes.Structure):
    _fields_ = _fields(d_table="p", table_stride="l", d_held="p", d_parent="p", d_keep="p", d_want="p", d_pinned="p", A="i",
                       width="i", B="i", width_out="i", d_table_out="p", table_out_stride="l", d_held_out="p", d_copies="p",
                       d_refs="p", d_status="p")
