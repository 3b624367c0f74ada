"""The structures of include/grid.h that calls fill, field by field, for tests
that call the library with arguments of their own."""
import ctypes

from paper_2607_11951_gb300.grid import _fields


class KvChunk(ctypes.Structure):
    _fields_ = _fields(d_table="p", table_stride="l", d_len="p", d_start="p", max_pages="i", B="i", n_tokens="i",
                       reserved="i")


class Heads(ctypes.Structure):
    _fields_ = _fields(d="p", token_stride="l", head_stride="l")


class KvQuery(ctypes.Structure):
    _fields_ = [("q", Heads), ("out", Heads)] + _fields(d_lse="p", scale="f", reserved="i")


class Rotation(ctypes.Structure):
    _fields_ = _fields(d_cos="p", d_sin="p", n_pos="i", rot="i", pairs="i", reserved="i")


class HeadNorm(ctypes.Structure):
    _fields_ = _fields(d_q="p", d_k="p", eps="f", reserved="i")


class DraftStep(ctypes.Structure):
    _fields_ = _fields(d_logits="p", logit_stride="l2", d_mask="p", mask_stride="l2", d_probs="p", prob_stride="l2",
                       d_draft="p", d_draft_len="p", d_u="p", d_noise="p", noise_stride="l", d_temperature="p", dtype="i",
                       B="i", K="i", V="i", eos="i", reserved="i", d_tokens="p", d_accepted="p", d_logprob="p",
                       d_status="p")
