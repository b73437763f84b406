"""Thin ctypes binding of ``libaif.so`` (see ``include/aif.h``).

Argument marshalling only: every step of the scoring path runs in the HIP
kernels behind the C ABI.  Tensors are torch tensors used purely as device
memory (``data_ptr()``) and the current torch stream is the HIP stream the
work is enqueued on.  A missing library raises; there is no fallback.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import List, Optional, Sequence

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libaif.so")

AIF_OK, AIF_EINVAL, AIF_ESHAPE, AIF_ENOMEM, AIF_EDEVICE, AIF_ERANGE = range(6)
AIF_F32, AIF_BF16 = 0, 1
AIF_CROSS_NONE, AIF_CROSS_HADAMARD, AIF_CROSS_SEGDOT, AIF_CROSS_BEA = 0, 1, 2, 3

EXPORTS = ("aif_score_init", "aif_score_request", "aif_score_batch", "aif_topk", "aif_score_destroy",
           "aif_last_error", "aif_poll_device_errors", "aif_peek_features", "aif_profile_begin",
           "aif_profile_end", "aif_stage_kind", "aif_update_rows", "aif_swap_table", "aif_score_topk",
           "aif_profile_begin_stages", "aif_profile_begin_sampled", "aif_last_user_slots", "aif_score_topk_static",
           "aif_mlp_layer1_width", "aif_last_mlp_kind", "aif_last_forms")
FORM_ONE_LAUNCH, FORM_HEAD_TILE, FORM_HEAD_REGISTERS, FORM_KEYS_RESIDENT = 1, 2, 4, 8
STAGES = ("gather", "user_fold", "attention", "mlp", "topk")
LSH_EXPORTS = ("aif_lsh_init", "aif_lsh_batch", "aif_lsh_destroy", "aif_lsh_last_error",
               "aif_lsh_poll_device_errors", "aif_lsh_simtier_kind", "aif_lsh_din_kind", "aif_lsh_last_form", "aif_lsh_profile_begin",
               "aif_lsh_profile_end")
LSH_STAGES = ("user", "din", "simtier")
USER_EXPORTS = ("aif_user_init", "aif_user_precompute", "aif_user_destroy", "aif_user_last_error",
                "aif_user_attention_kind", "aif_user_last_form", "aif_user_profile_begin", "aif_user_profile_end")
USER_STAGES = ("project", "attention", "ffn_pool")


class aif_config(C.Structure):
    _fields_ = [("dtype", C.c_int), ("n_items", C.c_int64), ("d_item", C.c_int32), ("d_user", C.c_int32),
                ("d_attn", C.c_int32), ("n_heads", C.c_int32), ("max_seq_len", C.c_int32),
                ("cross_mode", C.c_int), ("n_cross", C.c_int32), ("d_cross_vec", C.c_int32),
                ("n_layers", C.c_int32), ("layer_dims", C.POINTER(C.c_int32)),
                ("max_candidates", C.c_int32), ("max_users", C.c_int32), ("flags", C.c_uint32)]


class aif_weights(C.Structure):
    _fields_ = [("item_table", C.c_void_p), ("w_q", C.c_void_p),
                ("w", C.POINTER(C.c_void_p)), ("b", C.POINTER(C.c_void_p))]


class aif_request(C.Structure):
    _fields_ = [("user_vec", C.c_void_p), ("cross_vecs", C.c_void_p), ("seq_keys", C.c_void_p),
                ("seq_vals", C.c_void_p), ("seq_len", C.c_int32), ("cand_ids", C.c_void_p),
                ("n_cand", C.c_int32), ("logits_out", C.c_void_p), ("scores_out", C.c_void_p)]


class aif_lsh_config(C.Structure):
    _fields_ = [("n_items", C.c_int64), ("d_bits", C.c_int32), ("d_out", C.c_int32), ("n_tiers", C.c_int32),
                ("dtype", C.c_int), ("max_seq_len", C.c_int32), ("max_candidates", C.c_int32),
                ("max_users", C.c_int32)]


class aif_lsh_request(C.Structure):
    _fields_ = [("seq_sigs", C.c_void_p), ("seq_emb", C.c_void_p), ("seq_len", C.c_int32),
                ("cand_ids", C.c_void_p), ("n_cand", C.c_int32), ("din_out", C.c_void_p),
                ("tier_out", C.c_void_p)]


class aif_user_config(C.Structure):
    _fields_ = [("dtype", C.c_int), ("d_raw", C.c_int32), ("d", C.c_int32), ("max_seq_len", C.c_int32),
                ("max_users", C.c_int32)]


class aif_user_weights(C.Structure):
    _fields_ = [("w_profile", C.c_void_p), ("w_seq", C.c_void_p), ("w_ffn", C.c_void_p), ("b_ffn", C.c_void_p)]


class aif_user_request(C.Structure):
    _fields_ = [("profile", C.c_void_p), ("seq", C.c_void_p), ("seq_len", C.c_int32),
                ("user_vec_out", C.c_void_p), ("seq_out", C.c_void_p)]


_lib = None


def load():
    """Load libaif.so (built by ``python -m paper_2511_12934_amd.build``)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2511_12934_amd.build` "
                           "(there is no CPU fallback)")
    lib = C.CDLL(LIB_PATH)
    vp = C.c_void_p
    lib.aif_score_init.restype = C.c_int
    lib.aif_score_init.argtypes = [C.POINTER(aif_config), C.POINTER(aif_weights), C.POINTER(vp)]
    lib.aif_score_request.restype = C.c_int
    lib.aif_score_request.argtypes = [vp, C.POINTER(aif_request), vp]
    lib.aif_score_batch.restype = C.c_int
    lib.aif_score_batch.argtypes = [vp, C.POINTER(aif_request), C.c_int32, vp]
    lib.aif_topk.restype = C.c_int
    lib.aif_topk.argtypes = [vp, C.POINTER(vp), C.POINTER(C.c_int32), C.c_int32, C.c_int32, vp, vp, vp]
    lib.aif_score_destroy.restype = None
    lib.aif_score_destroy.argtypes = [vp]
    lib.aif_last_error.restype = C.c_char_p
    lib.aif_last_error.argtypes = [vp]
    lib.aif_poll_device_errors.restype = C.c_int
    lib.aif_poll_device_errors.argtypes = [vp, C.POINTER(C.c_int32)]
    lib.aif_peek_features.restype = C.c_int
    lib.aif_peek_features.argtypes = [vp, C.c_int32, C.c_int32, C.c_int32, vp]
    lib.aif_profile_begin.restype = C.c_int
    lib.aif_profile_begin.argtypes = [vp, C.c_int32]
    lib.aif_profile_begin_stages.restype = C.c_int
    lib.aif_profile_begin_stages.argtypes = [vp, C.c_int32, C.c_uint32]
    lib.aif_profile_begin_sampled.restype = C.c_int
    lib.aif_profile_begin_sampled.argtypes = [vp, C.c_int32, C.c_uint32, C.c_int32]
    lib.aif_profile_end.restype = C.c_int
    lib.aif_profile_end.argtypes = [vp, C.POINTER(C.c_double), C.POINTER(C.c_int32)]
    lib.aif_stage_kind.restype = C.c_int32
    lib.aif_stage_kind.argtypes = [vp, C.c_int32]
    lib.aif_score_topk_static.restype = C.c_int
    lib.aif_score_topk_static.argtypes = [vp, C.POINTER(aif_request), C.c_int32, vp, vp, vp]
    lib.aif_last_user_slots.restype = C.c_int32
    lib.aif_last_user_slots.argtypes = [vp]
    lib.aif_last_mlp_kind.restype = C.c_int32
    lib.aif_last_mlp_kind.argtypes = [vp]
    lib.aif_last_forms.restype = C.c_int32
    lib.aif_last_forms.argtypes = [vp]
    lib.aif_mlp_layer1_width.restype = C.c_int32
    lib.aif_mlp_layer1_width.argtypes = [vp]
    lib.aif_score_topk.restype = C.c_int
    lib.aif_score_topk.argtypes = [vp, C.POINTER(aif_request), C.c_int32, C.c_int32, vp, vp, vp]
    lib.aif_update_rows.restype = C.c_int
    lib.aif_update_rows.argtypes = [vp, vp, vp, C.c_int32, vp]
    lib.aif_swap_table.restype = C.c_int
    lib.aif_swap_table.argtypes = [vp, vp, C.c_int64]
    lib.aif_lsh_init.restype = C.c_int
    lib.aif_lsh_init.argtypes = [C.POINTER(aif_lsh_config), vp, C.POINTER(vp)]
    lib.aif_lsh_batch.restype = C.c_int
    lib.aif_lsh_batch.argtypes = [vp, C.POINTER(aif_lsh_request), C.c_int32, vp]
    lib.aif_lsh_destroy.restype = None
    lib.aif_lsh_destroy.argtypes = [vp]
    lib.aif_lsh_last_error.restype = C.c_char_p
    lib.aif_lsh_last_error.argtypes = [vp]
    lib.aif_lsh_poll_device_errors.restype = C.c_int
    lib.aif_lsh_poll_device_errors.argtypes = [vp, C.POINTER(C.c_int32)]
    lib.aif_lsh_simtier_kind.restype = C.c_int32
    lib.aif_lsh_simtier_kind.argtypes = [vp]
    lib.aif_lsh_din_kind.restype = C.c_int32
    lib.aif_lsh_din_kind.argtypes = [vp]
    lib.aif_lsh_last_form.restype = C.c_int32
    lib.aif_lsh_last_form.argtypes = [vp]
    lib.aif_lsh_profile_begin.restype = C.c_int
    lib.aif_lsh_profile_begin.argtypes = [vp, C.c_int32]
    lib.aif_lsh_profile_end.restype = C.c_int
    lib.aif_lsh_profile_end.argtypes = [vp, C.POINTER(C.c_double), C.POINTER(C.c_int32)]
    lib.aif_user_init.restype = C.c_int
    lib.aif_user_init.argtypes = [C.POINTER(aif_user_config), C.POINTER(aif_user_weights), C.POINTER(vp)]
    lib.aif_user_precompute.restype = C.c_int
    lib.aif_user_precompute.argtypes = [vp, C.POINTER(aif_user_request), C.c_int32, vp]
    lib.aif_user_destroy.restype = None
    lib.aif_user_destroy.argtypes = [vp]
    lib.aif_user_last_error.restype = C.c_char_p
    lib.aif_user_last_error.argtypes = [vp]
    lib.aif_user_attention_kind.restype = C.c_int32
    lib.aif_user_attention_kind.argtypes = [vp]
    lib.aif_user_last_form.restype = C.c_int32
    lib.aif_user_last_form.argtypes = [vp]
    lib.aif_user_profile_begin.restype = C.c_int
    lib.aif_user_profile_begin.argtypes = [vp, C.c_int32]
    lib.aif_user_profile_end.restype = C.c_int
    lib.aif_user_profile_end.argtypes = [vp, C.POINTER(C.c_double), C.POINTER(C.c_int32)]
    _declare_cache(lib)
    _lib = lib
    return lib


class AifError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"aif status {status}: {msg}")
        self.status = status


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _stream() -> Optional[int]:
    import torch
    # the handle itself: the Stream object around it takes 2.9 us a call, as much as a launch
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device()) or None


def _current_device() -> int:
    import torch
    return torch.cuda.current_device()


class Request:
    """Device tensors of one request (or mini-batch slice)."""

    def __init__(self, user_vec, seq_keys, seq_vals, cand_ids, logits_out, scores_out=None, cross_vecs=None,
                 seq_len: Optional[int] = None):
        self.user_vec, self.seq_keys, self.seq_vals = user_vec, seq_keys, seq_vals
        self.cand_ids, self.logits_out, self.scores_out, self.cross_vecs = cand_ids, logits_out, scores_out, cross_vecs
        self.seq_len = int(seq_keys.shape[0]) if seq_len is None else int(seq_len)
        self.n_cand = int(cand_ids.numel())

    def fill(self, r: aif_request):
        r.user_vec = _ptr(self.user_vec)
        r.cross_vecs = _ptr(self.cross_vecs)
        r.seq_keys = _ptr(self.seq_keys)
        r.seq_vals = _ptr(self.seq_vals)
        r.seq_len = self.seq_len
        r.cand_ids = _ptr(self.cand_ids)
        r.n_cand = self.n_cand
        r.logits_out = _ptr(self.logits_out)
        r.scores_out = _ptr(self.scores_out)


def pack_requests(reqs: Sequence[Request]):
    arr = (aif_request * max(len(reqs), 1))()
    for i, q in enumerate(reqs):
        q.fill(arr[i])
    return arr


class Context:
    """Owns one ``aif_ctx``.  Methods carry the names of the C entry points."""

    def __init__(self, *, dtype: int, table, d_user: int, d_attn: int, n_heads: int, max_seq_len: int,
                 layer_dims: Sequence[int], weights: Sequence, biases: Optional[Sequence] = None, w_q=None,
                 cross_mode: int = AIF_CROSS_HADAMARD, n_cross: int = 0, d_cross_vec: int = 0,
                 max_candidates: int, max_users: int = 1, n_items: Optional[int] = None,
                 d_item: Optional[int] = None):
        self._lib = load()
        self._h = C.c_void_p()
        nl = len(layer_dims) - 1
        dims = (C.c_int32 * (nl + 1))(*layer_dims)
        cfg = aif_config(dtype, int(table.shape[0]) if n_items is None else n_items,
                         int(table.shape[1]) if d_item is None else d_item, d_user, d_attn, n_heads, max_seq_len,
                         cross_mode, n_cross, d_cross_vec, nl, dims, max_candidates, max_users, 0)
        w_arr = (C.c_void_p * nl)(*[_ptr(w) for w in weights])
        b_arr = None
        if biases is not None:
            b_arr = (C.c_void_p * nl)(*[_ptr(b) for b in biases])
        wt = aif_weights(_ptr(table), _ptr(w_q), w_arr, b_arr)
        self._keep = (table,)                      # the table is borrowed for the life of the context
        st = self._lib.aif_score_init(C.byref(cfg), C.byref(wt), C.byref(self._h))
        if st != AIF_OK:
            self._h = C.c_void_p()
            raise AifError(st, self._lib.aif_last_error(None).decode())

    def _check(self, st: int):
        if st != AIF_OK:
            raise AifError(st, self._lib.aif_last_error(self._h).decode())

    def aif_last_error(self) -> str:
        return self._lib.aif_last_error(self._h).decode()

    def aif_score_request(self, req: Request):
        arr = pack_requests([req])
        self._check(self._lib.aif_score_request(self._h, arr, _stream()))

    def aif_score_batch(self, reqs: Sequence[Request], packed=None):
        arr = pack_requests(reqs) if packed is None else packed
        self._check(self._lib.aif_score_batch(self._h, arr, len(reqs), _stream()))

    def aif_score_topk(self, reqs: Sequence[Request], k: int, idx_out, val_out, packed=None):
        arr = pack_requests(reqs) if packed is None else packed
        self._check(self._lib.aif_score_topk(self._h, arr, len(reqs), k, _ptr(idx_out), _ptr(val_out), _stream()))

    def aif_score_topk_static(self, req: Request, k: int, idx_out=None, val_out=None):
        arr = pack_requests([req])
        self._check(self._lib.aif_score_topk_static(self._h, arr, k, _ptr(idx_out), _ptr(val_out), _stream()))

    def aif_topk(self, logits: Sequence, k: int, idx_out, val_out, n_cand: Optional[Sequence[int]] = None):
        n = len(logits)
        ptrs = (C.c_void_p * max(n, 1))(*[_ptr(t) for t in logits])
        counts = (C.c_int32 * max(n, 1))(*([int(t.numel()) for t in logits] if n_cand is None else n_cand))
        self._check(self._lib.aif_topk(self._h, ptrs, counts, n, k, _ptr(idx_out), _ptr(val_out), _stream()))

    def aif_poll_device_errors(self) -> int:
        n = C.c_int32(0)
        self._check(self._lib.aif_poll_device_errors(self._h, C.byref(n)))
        return n.value

    def aif_update_rows(self, ids, rows, n: Optional[int] = None):
        self._check(self._lib.aif_update_rows(self._h, _ptr(ids), _ptr(rows), int(ids.numel()) if n is None else n, _stream()))

    def aif_swap_table(self, new_table, n_items: Optional[int] = None):
        self._check(self._lib.aif_swap_table(self._h, _ptr(new_table), int(new_table.shape[0]) if n_items is None else n_items))
        self._keep = self._keep + (new_table,)     # the old table may still be read by enqueued work

    def aif_peek_features(self, request: int, first_row: int, n_rows: int, out_ptr: int):
        """Rows of the last batch's [e | attention | cross] matrix of one request into a host buffer."""
        self._check(self._lib.aif_peek_features(self._h, request, first_row, n_rows, out_ptr))

    def aif_profile_begin(self, max_calls: int):
        self._check(self._lib.aif_profile_begin(self._h, max_calls))

    def aif_profile_begin_stages(self, max_calls: int, stages):
        mask = 0
        for s in stages:
            mask |= 1 << STAGES.index(s)
        self._check(self._lib.aif_profile_begin_stages(self._h, max_calls, mask))

    def aif_profile_begin_sampled(self, max_calls: int, stages, every: int):
        mask = 0
        for s in stages:
            mask |= 1 << STAGES.index(s)
        self._check(self._lib.aif_profile_begin_sampled(self._h, max_calls, mask, every))

    def aif_profile_end(self):
        """{stage: (summed ms, recorded calls)}"""
        ms = (C.c_double * len(STAGES))()
        n = (C.c_int32 * len(STAGES))()
        self._check(self._lib.aif_profile_end(self._h, ms, n))
        return {s: (ms[i], n[i]) for i, s in enumerate(STAGES)}

    def aif_stage_kind(self, stage: str) -> int:
        return int(self._lib.aif_stage_kind(self._h, STAGES.index(stage)))

    def aif_last_user_slots(self) -> int:
        return int(self._lib.aif_last_user_slots(self._h))

    def aif_last_mlp_kind(self) -> int:
        return int(self._lib.aif_last_mlp_kind(self._h))

    def aif_last_forms(self) -> int:
        return int(self._lib.aif_last_forms(self._h))

    def aif_mlp_layer1_width(self) -> int:
        return int(self._lib.aif_mlp_layer1_width(self._h))

    def close(self):
        if self._h:
            self._lib.aif_score_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class LshRequest:
    """Device tensors of one request of the LSH path."""

    def __init__(self, seq_sigs, seq_emb, cand_ids, din_out, tier_out, seq_len: Optional[int] = None):
        self.seq_sigs, self.seq_emb, self.cand_ids, self.din_out, self.tier_out = seq_sigs, seq_emb, cand_ids, din_out, tier_out
        self.seq_len = int(seq_sigs.shape[0]) if seq_len is None else int(seq_len)
        self.n_cand = int(cand_ids.numel())

    def fill(self, r: aif_lsh_request):
        r.seq_sigs = _ptr(self.seq_sigs)
        r.seq_emb = _ptr(self.seq_emb)
        r.seq_len = self.seq_len
        r.cand_ids = _ptr(self.cand_ids)
        r.n_cand = self.n_cand
        r.din_out = _ptr(self.din_out)
        r.tier_out = _ptr(self.tier_out)


def pack_lsh_requests(reqs: Sequence[LshRequest]):
    arr = (aif_lsh_request * max(len(reqs), 1))()
    for i, q in enumerate(reqs):
        q.fill(arr[i])
    return arr


class LshContext:
    """Owns one ``aif_lsh_ctx``.  Methods carry the names of the C entry points."""

    def __init__(self, *, sig_table, d_out: int, n_tiers: int, dtype: int, max_seq_len: int, max_candidates: int,
                 max_users: int = 1):
        self._lib = load()
        self._h = C.c_void_p()
        cfg = aif_lsh_config(int(sig_table.shape[0]), 8 * int(sig_table.shape[1]), d_out, n_tiers, dtype, max_seq_len,
                             max_candidates, max_users)
        self._keep = (sig_table,)
        st = self._lib.aif_lsh_init(C.byref(cfg), _ptr(sig_table), C.byref(self._h))
        if st != AIF_OK:
            self._h = C.c_void_p()
            raise AifError(st, self._lib.aif_lsh_last_error(None).decode())

    def _check(self, st: int):
        if st != AIF_OK:
            raise AifError(st, self._lib.aif_lsh_last_error(self._h).decode())

    def aif_lsh_batch(self, reqs: Sequence[LshRequest], packed=None):
        arr = pack_lsh_requests(reqs) if packed is None else packed
        self._check(self._lib.aif_lsh_batch(self._h, arr, len(reqs), _stream()))

    def aif_lsh_poll_device_errors(self) -> int:
        n = C.c_int32(0)
        self._check(self._lib.aif_lsh_poll_device_errors(self._h, C.byref(n)))
        return n.value

    def aif_lsh_simtier_kind(self) -> int:
        return int(self._lib.aif_lsh_simtier_kind(self._h))

    def aif_lsh_last_form(self) -> int:
        return int(self._lib.aif_lsh_last_form(self._h))

    def aif_lsh_din_kind(self) -> int:
        return int(self._lib.aif_lsh_din_kind(self._h))

    def aif_lsh_profile_begin(self, max_calls: int):
        self._check(self._lib.aif_lsh_profile_begin(self._h, max_calls))

    def aif_lsh_profile_end(self):
        ms = (C.c_double * len(LSH_STAGES))()
        n = (C.c_int32 * len(LSH_STAGES))()
        self._check(self._lib.aif_lsh_profile_end(self._h, ms, n))
        return {s: (ms[i], n[i]) for i, s in enumerate(LSH_STAGES)}

    def close(self):
        if self._h:
            self._lib.aif_lsh_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class UserRequest:
    """Device tensors of one user of the user-side network (include/aif_user.h)."""

    def __init__(self, profile, seq, user_vec_out, seq_out, seq_len: Optional[int] = None):
        self.profile, self.seq, self.user_vec_out, self.seq_out = profile, seq, user_vec_out, seq_out
        self.seq_len = int(seq.shape[0]) if seq_len is None else int(seq_len)

    def fill(self, r: aif_user_request):
        r.profile = _ptr(self.profile)
        r.seq = _ptr(self.seq)
        r.seq_len = self.seq_len
        r.user_vec_out = _ptr(self.user_vec_out)
        r.seq_out = _ptr(self.seq_out)


def pack_user_requests(reqs: Sequence[UserRequest]):
    arr = (aif_user_request * max(len(reqs), 1))()
    for i, q in enumerate(reqs):
        q.fill(arr[i])
    return arr


class UserContext:
    """Owns one ``aif_user_ctx``.  Methods carry the names of the C entry points."""

    def __init__(self, *, dtype: int, d_raw: int, d: int, w_profile, w_seq, w_ffn, b_ffn=None, max_seq_len: int,
                 max_users: int = 1):
        self._lib = load()
        self._h = C.c_void_p()
        cfg = aif_user_config(dtype, d_raw, d, max_seq_len, max_users)
        wts = aif_user_weights(_ptr(w_profile), _ptr(w_seq), _ptr(w_ffn), _ptr(b_ffn))
        st = self._lib.aif_user_init(C.byref(cfg), C.byref(wts), C.byref(self._h))
        if st != AIF_OK:
            self._h = C.c_void_p()
            raise AifError(st, self._lib.aif_user_last_error(None).decode())

    def _check(self, st: int):
        if st != AIF_OK:
            raise AifError(st, self._lib.aif_user_last_error(self._h).decode())

    def aif_user_precompute(self, reqs: Sequence[UserRequest], packed=None, stream: Optional[int] = None):
        arr = pack_user_requests(reqs) if packed is None else packed
        self._check(self._lib.aif_user_precompute(self._h, arr, len(reqs), _stream() if stream is None else stream))

    def aif_user_last_form(self) -> int:
        return int(self._lib.aif_user_last_form(self._h))

    def aif_user_attention_kind(self) -> int:
        return int(self._lib.aif_user_attention_kind(self._h))

    def aif_user_profile_begin(self, max_calls: int):
        self._check(self._lib.aif_user_profile_begin(self._h, max_calls))

    def aif_user_profile_end(self):
        ms = (C.c_double * len(USER_STAGES))()
        n = (C.c_int32 * len(USER_STAGES))()
        self._check(self._lib.aif_user_profile_end(self._h, ms, n))
        return {s: (ms[i], n[i]) for i, s in enumerate(USER_STAGES)}

    def close(self):
        if self._h:
            self._lib.aif_user_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


# ---- the user cache (include/aif_cache.h) ---------------------------------------------------------------------------
class aif_cache_config(C.Structure):
    _fields_ = [("dtype", C.c_int), ("n_heads", C.c_int32), ("n_kv_heads", C.c_int32), ("d_head", C.c_int32),
                ("scale", C.c_float), ("page_len", C.c_int32), ("n_pages", C.c_int32), ("max_seqs", C.c_int32),
                ("max_len", C.c_int32), ("max_requests", C.c_int32), ("max_queries", C.c_int32)]


class aif_cache_append_req(C.Structure):
    _fields_ = [("seq", C.c_int32), ("n_rows", C.c_int32), ("keys", C.c_void_p), ("vals", C.c_void_p),
                ("key_stride", C.c_int64), ("val_stride", C.c_int64)]


class aif_cache_attend_req(C.Structure):
    _fields_ = [("seq", C.c_int32), ("n_q", C.c_int32), ("q", C.c_void_p), ("out", C.c_void_p), ("lse_out", C.c_void_p),
                ("positions", C.c_void_p), ("q_stride", C.c_int64), ("out_stride", C.c_int64), ("sinks", C.c_int32),
                ("window", C.c_int32)]


class aif_cache_read_req(C.Structure):
    _fields_ = [("seq", C.c_int32), ("first", C.c_int32), ("n_rows", C.c_int32), ("reserved", C.c_int32),
                ("keys_out", C.c_void_p), ("vals_out", C.c_void_p), ("key_stride", C.c_int64), ("val_stride", C.c_int64)]


CACHE_EXPORTS = ("aif_cache_page_bytes", "aif_cache_init", "aif_cache_destroy", "aif_cache_last_error", "aif_cache_append",
                 "aif_cache_attend", "aif_cache_read", "aif_cache_fork", "aif_cache_copy", "aif_cache_free",
                 "aif_cache_truncate", "aif_cache_trim", "aif_cache_compact", "aif_cache_swap_pool", "aif_cache_len",
                 "aif_cache_free_pages")


def _declare_cache(lib):
    vp, i32 = C.c_void_p, C.c_int32
    ids = C.POINTER(i32)
    for name, res, args in (
            ("aif_cache_page_bytes", C.c_size_t, [C.POINTER(aif_cache_config)]),
            ("aif_cache_init", C.c_int, [C.POINTER(aif_cache_config), vp, C.POINTER(vp)]),
            ("aif_cache_destroy", None, [vp]),
            ("aif_cache_last_error", C.c_char_p, [vp]),
            ("aif_cache_append", C.c_int, [vp, C.POINTER(aif_cache_append_req), i32, vp]),
            ("aif_cache_attend", C.c_int, [vp, C.POINTER(aif_cache_attend_req), i32, vp]),
            ("aif_cache_read", C.c_int, [vp, C.POINTER(aif_cache_read_req), i32, vp]),
            ("aif_cache_fork", C.c_int, [vp, ids, ids, i32, vp]),
            ("aif_cache_copy", C.c_int, [vp, ids, ids, i32, vp]),
            ("aif_cache_free", C.c_int, [vp, ids, i32]),
            ("aif_cache_truncate", C.c_int, [vp, i32, i32]),
            ("aif_cache_trim", C.c_int, [vp, ids, i32, i32, i32, vp]),
            ("aif_cache_compact", C.c_int, [vp, ids, vp]),
            ("aif_cache_swap_pool", C.c_int, [vp, vp, i32]),
            ("aif_cache_len", i32, [vp, i32]),
            ("aif_cache_free_pages", i32, [vp])):
        f = getattr(lib, name)
        f.restype, f.argtypes = res, args


def _i32(x) -> int:
    """A whole number as the C fields hold it (ctypes keeps the low bits of a larger one)."""
    x = int(x)
    if not -1 << 31 <= x < 1 << 31:
        raise ValueError(f"{x} does not fit in 32 bits")
    return x


def _row_width(t) -> int:
    """Features of a row of [rows, ...]; 0 where there are no rows."""
    return t.numel() // t.shape[0] if t.shape[0] else 0


def _row_stride(t, width: int) -> int:
    """Elements from one row of [rows, ...] to the next, 0 where there is one; rows themselves lie close."""
    if t is None or t.numel() == 0:
        return 0
    n = t.shape[0]
    if t.is_contiguous() and t.numel() == n * width:
        return width if n > 1 else 0
    row = t[0]
    if row.numel() != width or not row.is_contiguous():
        raise ValueError(f"a row of {width} contiguous features is wanted, got {tuple(row.shape)} with strides {row.stride()}")
    if n == 1:
        return 0
    if t.stride(0) < width:                        # (a broadcast row: 0, which would say that rows lie close)
        raise ValueError(f"rows of {width} features overlap: {tuple(t.shape)} with strides {t.stride()}")
    return int(t.stride(0))


def _kind(width: int, t):
    return None if t is None else (width, t.dtype, t.device)


def _like(t):
    return None if t is None else (t.dtype, t.get_device())


class CacheAppend:
    """Rows for the end of a sequence: keys and vals [n_rows, n_kv_heads * d_head] (or [n_rows, n_kv_heads, d_head]), rows
    that may lie apart."""

    def __init__(self, seq: int, keys, vals):
        self.seq, self.keys, self.vals = _i32(seq), keys, vals
        self.n_rows = int(keys.shape[0])
        if tuple(vals.shape) != tuple(keys.shape):
            raise ValueError(f"keys {tuple(keys.shape)} and vals {tuple(vals.shape)} differ")
        self.width = _row_width(keys)
        self.strides = _row_stride(keys, self.width), _row_stride(vals, self.width)

    def fill(self, r: aif_cache_append_req):
        r.seq, r.n_rows, r.keys, r.vals = self.seq, self.n_rows, _ptr(self.keys), _ptr(self.vals)
        r.key_stride, r.val_stride = self.strides

    names = ("keys", "vals")

    def kinds(self):
        """What a context holds against its own: (features of a row, type, device) of each of `names`."""
        return _kind(self.width, self.keys), _kind(self.width, self.vals)

    def like(self):
        """Alike where kinds() are, and quicker."""
        return self.width, _like(self.keys), _like(self.vals)


class CacheQuery:
    """Queries over a sequence: q and out [n_q, n_heads, d_head] (or [n_q, n_heads * d_head]), rows that may lie apart;
    lse [n_q, n_heads] fp32 and positions [n_q] int32, both contiguous."""

    def __init__(self, seq: int, q, out, lse=None, positions=None, sinks: int = 0, window: int = 0):
        self.seq, self.q, self.out, self.lse, self.positions = _i32(seq), q, out, lse, positions
        self.sinks, self.window = _i32(sinks), _i32(window)
        self.n_q = int(q.shape[0])
        if tuple(out.shape) != tuple(q.shape):
            raise ValueError(f"q {tuple(q.shape)} and out {tuple(out.shape)} differ")
        for name, t, n in (("lse", lse, None), ("positions", positions, self.n_q)):
            if t is not None and (t.shape[0] != self.n_q or not t.is_contiguous() or (n is not None and t.numel() != n)):
                raise ValueError(f"{name}: contiguous, a row for each of {self.n_q} queries, got {tuple(t.shape)}")
        self.width = _row_width(q)
        self.strides = _row_stride(q, self.width), _row_stride(out, self.width)

    def fill(self, r: aif_cache_attend_req):
        r.seq, r.n_q, r.q, r.out, r.lse_out, r.positions = self.seq, self.n_q, _ptr(self.q), _ptr(self.out), _ptr(self.lse), _ptr(self.positions)
        r.q_stride, r.out_stride = self.strides
        r.sinks, r.window = self.sinks, self.window

    names = ("q", "out", "lse", "positions")

    def kinds(self):
        lse = self.lse
        return _kind(self.width, self.q), _kind(self.width, self.out), None if lse is None else _kind(_row_width(lse), lse), _kind(1, self.positions)

    def like(self):
        lse = self.lse
        return self.width, _like(self.q), _like(self.out), None if lse is None else (lse.dtype, lse.get_device(), lse.numel() // self.n_q), _like(self.positions)


class CacheRead:
    """Rows [first, first + n_rows) of a sequence, to keys_out and vals_out [n_rows, ...] (either may be None)."""

    def __init__(self, seq: int, keys_out, vals_out, first: int = 0):
        self.seq, self.keys_out, self.vals_out, self.first = _i32(seq), keys_out, vals_out, _i32(first)
        one = keys_out if keys_out is not None else vals_out
        if one is None or (vals_out is not None and tuple(vals_out.shape) != tuple(one.shape)):
            raise ValueError("keys_out or vals_out is wanted, of one shape")
        self.n_rows = int(one.shape[0])
        self.width = _row_width(one)
        self.strides = _row_stride(keys_out, self.width), _row_stride(vals_out, self.width)

    def fill(self, r: aif_cache_read_req):
        r.seq, r.first, r.n_rows, r.reserved = self.seq, self.first, self.n_rows, 0
        r.keys_out, r.vals_out = _ptr(self.keys_out), _ptr(self.vals_out)
        r.key_stride, r.val_stride = self.strides

    names = ("keys_out", "vals_out")

    def kinds(self):
        return _kind(self.width, self.keys_out), _kind(self.width, self.vals_out)

    def like(self):
        return self.width, _like(self.keys_out), _like(self.vals_out)


def _pack_cache(kind, reqs):
    """The array, which knows how many requests it holds and of which kinds: the first of each run of requests of a kind."""
    arr = (kind * max(len(reqs), 1))()
    runs, last = [], None
    for i, q in enumerate(reqs):
        q.fill(arr[i])
        like = q.like() if q.width and len(reqs) > 1 else None
        if q.width and (like is None or like != last):  # (a request without rows is of no kind)
            runs.append((i, q.names, q.kinds()))
            last = like
    arr.n, arr.runs, arr.fits = len(reqs), runs, None
    return arr


def pack_cache_appends(reqs: Sequence[CacheAppend]):
    return _pack_cache(aif_cache_append_req, reqs)


def pack_cache_queries(reqs: Sequence[CacheQuery]):
    return _pack_cache(aif_cache_attend_req, reqs)


def pack_cache_reads(reqs: Sequence[CacheRead]):
    return _pack_cache(aif_cache_read_req, reqs)


def cache_ids(seqs):
    """Sequence numbers as the array the C entry points take; such an array is taken as it is."""
    if isinstance(seqs, C.Array):
        return seqs
    seqs = [_i32(q) for q in seqs]
    return (C.c_int32 * len(seqs))(*seqs)


def cache_page_bytes(*, dtype: int, n_heads: int, n_kv_heads: int, d_head: int, page_len: int) -> int:
    """Bytes of a page; the pool is n_pages of them."""
    cfg = aif_cache_config(dtype, _i32(n_heads), _i32(n_kv_heads), _i32(d_head), 0.0, _i32(page_len), 0, 0, 0, 0, 0)
    n = int(load().aif_cache_page_bytes(C.byref(cfg)))
    if n == 0:
        raise AifError(AIF_ESHAPE, load().aif_cache_last_error(None).decode())
    return n


class CacheContext:
    """Owns one ``aif_cache_ctx`` over the pool (a uint8 tensor, borrowed).  Methods carry the names of the C entry points."""

    def __init__(self, *, pool, dtype: int, n_heads: int, n_kv_heads: int, d_head: int, page_len: int, max_seqs: int,
                 max_len: int, max_requests: int, max_queries: int = 1, scale: float = 0.0, n_pages: Optional[int] = None):
        self._lib = load()
        self._h = C.c_void_p()
        self._check_pool(pool, _current_device())
        self._page_bytes = cache_page_bytes(dtype=dtype, n_heads=n_heads, n_kv_heads=n_kv_heads, d_head=d_head, page_len=page_len)
        have = pool.numel() * pool.element_size() // self._page_bytes
        n_pages = have if n_pages is None else n_pages
        if n_pages > have:
            raise ValueError(f"the pool holds {have} pages, not {n_pages}")
        import torch
        self.n_heads, self.dtype = n_heads, dtype
        kind = torch.float32 if dtype == AIF_F32 else torch.bfloat16
        kv, q = (n_kv_heads * d_head, kind, pool.device), (n_heads * d_head, kind, pool.device)
        # what tensors of a name have to be: features of a row, type, device
        self._fits = dict(keys=kv, vals=kv, keys_out=kv, vals_out=kv, q=q, out=q, lse=(n_heads, torch.float32, pool.device),
                          positions=(1, torch.int32, pool.device))
        cfg = aif_cache_config(dtype, n_heads, n_kv_heads, d_head, scale, page_len, _i32(n_pages), _i32(max_seqs), _i32(max_len), _i32(max_requests),
                               _i32(max_queries))
        self._keep = (pool,)                       # borrowed for the life of the context
        st = self._lib.aif_cache_init(C.byref(cfg), _ptr(pool), C.byref(self._h))
        if st != AIF_OK:
            self._h = C.c_void_p()
            raise AifError(st, self._lib.aif_cache_last_error(None).decode())

    def _check(self, st: int):
        if st != AIF_OK:
            raise AifError(st, self._lib.aif_cache_last_error(self._h).decode())

    def _packed(self, reqs, packed, pack):
        """The packed array, its tensors held against the context's row widths, type and device, once.  (An array that was
        not made by pack_cache_* is as its maker filled it.)"""
        arr = pack(reqs) if packed is None else packed
        runs = getattr(arr, "runs", None)
        n = arr.n if runs is not None else len(arr) if isinstance(arr, C.Array) else len(reqs)
        if len(reqs) > n:
            raise ValueError(f"{len(reqs)} requests, {n} are packed")
        if runs is None or arr.fits is self._fits:
            return arr
        for i, names, kinds in runs:
            for name, have in zip(names, kinds):
                want = self._fits[name]
                if have is None or have == want:
                    continue
                if name == "lse":
                    raise ValueError(f"request {i}: lse is [n_q, {self.n_heads}] fp32 on {want[2]}, has rows of {have[0]} {have[1]} on {have[2]}")
                if name == "positions":
                    raise ValueError(f"request {i}: positions are int32 on {want[2]}, not {have[1]} on {have[2]}")
                raise ValueError(f"request {i}: {name} has rows of {have[0]} {have[1]} on {have[2]}, the context {want[0]} {want[1]} on {want[2]}")
        arr.fits = self._fits
        return arr

    def aif_cache_append(self, reqs: Sequence[CacheAppend], packed=None):
        arr = self._packed(reqs, packed, pack_cache_appends)
        self._check(self._lib.aif_cache_append(self._h, arr, len(reqs), _stream()))

    def aif_cache_attend(self, reqs: Sequence[CacheQuery], packed=None):
        arr = self._packed(reqs, packed, pack_cache_queries)
        self._check(self._lib.aif_cache_attend(self._h, arr, len(reqs), _stream()))

    def aif_cache_read(self, reqs: Sequence[CacheRead], packed=None):
        arr = self._packed(reqs, packed, pack_cache_reads)
        self._check(self._lib.aif_cache_read(self._h, arr, len(reqs), _stream()))

    def _pairs(self, src, dst):
        src, dst = cache_ids(src), cache_ids(dst)
        if len(src) != len(dst):
            raise ValueError(f"{len(src)} sources and {len(dst)} destinations")
        return src, dst, len(src), _stream()

    def aif_cache_fork(self, src, dst):
        self._check(self._lib.aif_cache_fork(self._h, *self._pairs(src, dst)))

    def aif_cache_copy(self, src, dst):
        self._check(self._lib.aif_cache_copy(self._h, *self._pairs(src, dst)))

    def aif_cache_free(self, seqs):
        seqs = cache_ids(seqs)
        self._check(self._lib.aif_cache_free(self._h, seqs, len(seqs)))

    def aif_cache_truncate(self, seq: int, length: int):
        self._check(self._lib.aif_cache_truncate(self._h, _i32(seq), _i32(length)))

    def aif_cache_trim(self, seqs, sinks: int, window: int):
        seqs = cache_ids(seqs)
        self._check(self._lib.aif_cache_trim(self._h, seqs, len(seqs), _i32(sinks), _i32(window), _stream()))

    def aif_cache_compact(self) -> int:
        n = C.c_int32(0)
        self._check(self._lib.aif_cache_compact(self._h, C.byref(n), _stream()))
        return n.value

    @staticmethod
    def _check_pool(pool, device):
        if not pool.is_cuda or not pool.is_contiguous() or pool.device.index != device:
            raise ValueError(f"the pool is contiguous memory of GPU {device}, not of {pool.device}")

    def aif_cache_swap_pool(self, pool, n_pages: Optional[int] = None):
        self._check_pool(pool, self._keep[0].device.index)
        have = pool.numel() * pool.element_size() // self._page_bytes
        if n_pages is not None and n_pages > have:
            raise ValueError(f"the pool holds {have} pages, not {n_pages}")
        self._check(self._lib.aif_cache_swap_pool(self._h, _ptr(pool), have if n_pages is None else _i32(n_pages)))
        import torch
        for old in self._keep:                     # enqueued work may still read it: its memory is not given away before that has run
            if old.is_cuda:
                old.record_stream(torch.cuda.current_stream())
        self._keep = (pool,)

    def aif_cache_len(self, seq: int) -> int:
        return int(self._lib.aif_cache_len(self._h, seq if 0 <= seq < 1 << 31 else -1))

    def aif_cache_free_pages(self) -> int:
        return int(self._lib.aif_cache_free_pages(self._h))

    def close(self):
        if self._h:
            self._lib.aif_cache_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
