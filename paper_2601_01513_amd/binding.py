"""ctypes binding of libvsr.so (C ABI: include/vsr.h).

Argument marshalling only: every step of the scoring pass runs inside the HIP
library. Torch tensors supply device memory and the stream. If the library is
not built, loading fails loudly; there is no other path.
"""
from __future__ import annotations

import ctypes
import os
from typing import Dict, NamedTuple, Optional, Sequence

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libvsr.so")

VSR_OK, VSR_EINVAL, VSR_ESTATE, VSR_ERANGE, VSR_ENOMEM, VSR_EHIP = 0, -1, -2, -3, -4, -5
VSR_EID, VSR_ENONFINITE = -6, -7
VSR_CHECK_IDS, VSR_CHECK_FINITE = 1, 2
VSR_F32, VSR_BF16, VSR_F16 = 0, 1, 2
GEMM_WEIGHT_KEYS = ("wqkv", "wo", "wgu", "wdown")  # per layer, plus lm_head
VSR_MAX_CANDS = 256
VSR_RETRIEVE_STATIC_BYTES = 32 << 20

EXPORTS = ["vsr_workspace_size", "vsr_create", "vsr_load_weights", "vsr_prefill",
           "vsr_score", "vsr_verify", "vsr_reliability", "vsr_draft", "vsr_align_select", "vsr_weights_to_f16",
           "vsr_keyframes", "vsr_retrieve_workspace_size", "vsr_retrieve", "vsr_retrieve_static",
           "vsr_rope_axes", "vsr_qk_norm_rope", "vsr_set_positions", "vsr_load_qk_norms",
           "vsr_pick_workspace_size", "vsr_pick_tokens", "vsr_draft_ruled_workspace_size",
           "vsr_draft_ruled", "vsr_tree_rows", "vsr_tree_attention_workspace_size",
           "vsr_tree_attention", "vsr_pages_update_workspace_size", "vsr_pages_update",
           "vsr_pages_keep", "vsr_token_logprobs_workspace_size", "vsr_token_logprobs",
           "vsr_last_error",
           "vsr_destroy", "vsr_set_checks", "vsr_profile_enable", "vsr_profile_read"]

VSR_SELECT_TWO_STAGE, VSR_SELECT_ADDITION, VSR_SELECT_INVERT = 0, 1, 2
SELECT_STRATEGIES = {"two_stage": VSR_SELECT_TWO_STAGE, "addition": VSR_SELECT_ADDITION,
                     "invert": VSR_SELECT_INVERT}

VSR_STAGE_KINDS = 16
VSR_STAGES = 4 * VSR_STAGE_KINDS
VSR_PROFILE_ALL = (1 << VSR_STAGE_KINDS) - 1
STAGE_KINDS = ["embed", "rmsnorm", "qkv_rope", "attention", "attn_merge", "o_proj",
               "gate_up_swiglu", "down_proj", "lm_inputs", "lm_head_lse", "lse_gather",
               "sum_argmax", "row_tables", "copy", "tail_proj", "cand_attention"]
STAGE_NAMES = ([f"prefill.{k}" for k in STAGE_KINDS] + [f"score.{k}" for k in STAGE_KINDS]
               + [f"draft.{k}" for k in STAGE_KINDS] + [f"verify.{k}" for k in STAGE_KINDS])


class VsrConfig(ctypes.Structure):
    _fields_ = [("n_layers", ctypes.c_int32), ("d_model", ctypes.c_int32),
                ("n_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("d_ff", ctypes.c_int32),
                ("vocab", ctypes.c_int32), ("rms_eps", ctypes.c_float),
                ("rope_base", ctypes.c_float), ("dtype", ctypes.c_int32),
                ("max_prefix", ctypes.c_int32), ("max_cands", ctypes.c_int32),
                ("max_cand_len", ctypes.c_int32), ("split_layers", ctypes.c_int32),
                ("gemm_weights", ctypes.c_int32), ("max_new", ctypes.c_int32),
                ("split_mlp_layers", ctypes.c_int32)]


_PP = ctypes.POINTER(ctypes.c_void_p)


class VsrWeights(ctypes.Structure):
    _fields_ = [("embed", ctypes.c_void_p), ("lm_head", ctypes.c_void_p),
                ("final_norm", ctypes.c_void_p), ("attn_norm", _PP), ("wqkv", _PP),
                ("wo", _PP), ("ffn_norm", _PP), ("wgu", _PP), ("wdown", _PP)]


VSR_MAX_AXES = 4


class VsrRotary(ctypes.Structure):
    _fields_ = [("n_axes", ctypes.c_int32), ("sections", ctypes.c_int32 * VSR_MAX_AXES),
                ("interleaved", ctypes.c_int32), ("base", ctypes.c_float)]


class VsrHeads(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("n_heads", ctypes.c_int32),
                ("token_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64)]


class VsrTokenRules(ctypes.Structure):
    _fields_ = [("repetition", ctypes.c_void_p), ("presence", ctypes.c_void_p),
                ("frequency", ctypes.c_void_p), ("bias", ctypes.c_void_p),
                ("bias_stride", ctypes.c_int64), ("mask", ctypes.c_void_p),
                ("mask_stride", ctypes.c_int64)]


class VsrTokenLists(ctypes.Structure):
    _fields_ = [("prompt", ctypes.c_void_p), ("prompt_stride", ctypes.c_int64),
                ("n_prompt", ctypes.c_int32), ("prompt_len", ctypes.c_void_p),
                ("output", ctypes.c_void_p), ("output_stride", ctypes.c_int64),
                ("n_output", ctypes.c_int32), ("output_len", ctypes.c_void_p)]


class VsrPages(ctypes.Structure):
    _fields_ = [("n_seqs", ctypes.c_int32), ("n_pages", ctypes.c_int32),
                ("page_size", ctypes.c_int32), ("max_pages", ctypes.c_int32),
                ("table", ctypes.c_void_p), ("table_stride", ctypes.c_int64),
                ("len", ctypes.c_void_p), ("held", ctypes.c_void_p), ("refs", ctypes.c_void_p)]


class VsrCache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("dtype", ctypes.c_int32),
                ("n_layers", ctypes.c_int32), ("n_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("layer_stride", ctypes.c_int64),
                ("slot_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64)]


class VsrError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"vsr error {code}: {msg}")
        self.code = code


_lib = None


def load_library(path: Optional[str] = None) -> ctypes.CDLL:
    """Loads libvsr.so (raises if it has not been built). The path defaults to
    the in-tree build; the VSR_LIBRARY environment variable names another
    build of the same library (e.g. to compare two builds on one machine)."""
    global _lib
    if _lib is not None:
        return _lib
    path = path or os.environ.get("VSR_LIBRARY") or LIB_PATH
    if not os.path.exists(path):
        raise RuntimeError(
            f"{path} is missing: build it with `python -m paper_2601_01513_amd.build`")
    lib = ctypes.CDLL(path)
    lib.vsr_workspace_size.argtypes = [ctypes.POINTER(VsrConfig)]
    lib.vsr_workspace_size.restype = ctypes.c_size_t
    lib.vsr_create.argtypes = [ctypes.POINTER(VsrConfig), ctypes.c_void_p, ctypes.c_size_t,
                               ctypes.c_void_p, ctypes.POINTER(ctypes.c_void_p)]
    lib.vsr_create.restype = ctypes.c_int
    lib.vsr_load_weights.argtypes = [ctypes.c_void_p, ctypes.POINTER(VsrWeights)]
    lib.vsr_load_weights.restype = ctypes.c_int
    lib.vsr_prefill.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int32,
                                ctypes.c_void_p, ctypes.c_int32]
    lib.vsr_prefill.restype = ctypes.c_int
    lib.vsr_score.argtypes = [ctypes.c_void_p, ctypes.c_void_p,
                              ctypes.POINTER(ctypes.c_int32), ctypes.c_int32, ctypes.c_int32,
                              ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p]
    lib.vsr_score.restype = ctypes.c_int
    lib.vsr_verify.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int32,
                               ctypes.c_void_p, ctypes.c_int32, ctypes.c_void_p,
                               ctypes.POINTER(ctypes.c_int32), ctypes.c_int32, ctypes.c_int32,
                               ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p]
    lib.vsr_verify.restype = ctypes.c_int
    lib.vsr_reliability.argtypes = [ctypes.c_void_p, ctypes.c_void_p,
                                    ctypes.POINTER(ctypes.c_int32), ctypes.c_int32,
                                    ctypes.c_int32, ctypes.c_int32, ctypes.c_int32,
                                    ctypes.c_float, ctypes.c_void_p, ctypes.c_void_p,
                                    ctypes.c_void_p]
    lib.vsr_reliability.restype = ctypes.c_int
    lib.vsr_draft.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.POINTER(ctypes.c_int32),
                              ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.c_void_p]
    lib.vsr_draft.restype = ctypes.c_int
    lib.vsr_align_select.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int32,
                                     ctypes.c_int32, ctypes.c_int32, ctypes.c_void_p,
                                     ctypes.c_float, ctypes.c_int32, ctypes.c_void_p,
                                     ctypes.c_void_p, ctypes.c_void_p]
    lib.vsr_align_select.restype = ctypes.c_int
    lib.vsr_weights_to_f16.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t,
                                       ctypes.c_void_p]
    lib.vsr_weights_to_f16.restype = ctypes.c_int
    lib.vsr_keyframes.argtypes = [ctypes.c_void_p, ctypes.c_int32, ctypes.c_int32,
                                  ctypes.c_int32, ctypes.c_float, ctypes.c_void_p,
                                  ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                  ctypes.c_void_p]
    lib.vsr_keyframes.restype = ctypes.c_int
    lib.vsr_retrieve_workspace_size.argtypes = [ctypes.c_int32, ctypes.c_int32, ctypes.c_int32]
    lib.vsr_retrieve_workspace_size.restype = ctypes.c_size_t
    lib.vsr_retrieve.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                 ctypes.c_int32, ctypes.c_void_p, ctypes.c_int32,
                                 ctypes.c_int32, ctypes.c_int32, ctypes.c_int32,
                                 ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p,
                                 ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                 ctypes.c_void_p, ctypes.c_void_p]
    lib.vsr_retrieve.restype = ctypes.c_int
    lib.vsr_retrieve_static.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                        ctypes.c_int32, ctypes.c_void_p, ctypes.c_int32,
                                        ctypes.c_int32, ctypes.c_int32, ctypes.c_int32,
                                        ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                        ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p]
    lib.vsr_retrieve_static.restype = ctypes.c_int
    heads = [ctypes.POINTER(VsrHeads)] * 4
    i32, i64, ptr = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p
    lib.vsr_rope_axes.argtypes = [ctypes.POINTER(VsrRotary), i32, i32, i32, ptr, i64, *heads,
                                  ptr, i64, ptr]
    lib.vsr_rope_axes.restype = ctypes.c_int
    lib.vsr_qk_norm_rope.argtypes = [ctypes.POINTER(VsrRotary), i32, i32, i32, ptr, i64, ptr,
                                     ptr, i32, ctypes.c_float, *heads, ptr, i64, ptr]
    lib.vsr_qk_norm_rope.restype = ctypes.c_int
    lib.vsr_set_positions.argtypes = [ptr, ctypes.POINTER(VsrRotary), ptr, i64, i32, i32]
    lib.vsr_set_positions.restype = ctypes.c_int
    lib.vsr_load_qk_norms.argtypes = [ptr, _PP, _PP]
    lib.vsr_load_qk_norms.restype = ctypes.c_int
    lib.vsr_pick_workspace_size.argtypes = [i32, i32]
    lib.vsr_pick_workspace_size.restype = ctypes.c_size_t
    lib.vsr_pick_tokens.argtypes = [ptr, i32, i32, i32, i64, ctypes.POINTER(VsrTokenLists),
                                    ctypes.POINTER(VsrTokenRules), ptr, i64, ptr, ptr, ptr,
                                    ctypes.c_size_t, ptr]
    lib.vsr_pick_tokens.restype = ctypes.c_int
    lib.vsr_draft_ruled_workspace_size.argtypes = [ctypes.POINTER(VsrConfig), i32]
    lib.vsr_draft_ruled_workspace_size.restype = ctypes.c_size_t
    lib.vsr_draft_ruled.argtypes = [ptr, ptr, ctypes.POINTER(i32), i32, i32, i32,
                                    ctypes.POINTER(VsrTokenRules), i64, ptr, ptr, ptr,
                                    ctypes.c_size_t]
    lib.vsr_draft_ruled.restype = ctypes.c_int
    lib.vsr_tree_rows.argtypes = [ctypes.POINTER(VsrPages), i32, ptr, ptr, ptr, ptr, ptr, ptr,
                                  i64, i32, ptr]
    lib.vsr_tree_rows.restype = ctypes.c_int
    lib.vsr_tree_attention_workspace_size.argtypes = [i32] * 6
    lib.vsr_tree_attention_workspace_size.restype = ctypes.c_size_t
    lib.vsr_tree_attention.argtypes = [ctypes.POINTER(VsrPages), i32, i32, i32, ptr, *heads[:3],
                                       ptr, i64, i32, ctypes.c_float, heads[0], ptr, ptr,
                                       ctypes.c_size_t, ptr]
    lib.vsr_tree_attention.restype = ctypes.c_int
    lib.vsr_pages_update_workspace_size.argtypes = [i32]
    lib.vsr_pages_update_workspace_size.restype = ctypes.c_size_t
    lib.vsr_pages_update.argtypes = [ctypes.POINTER(VsrPages), ptr, ptr, ctypes.POINTER(VsrCache),
                                     ptr, ptr, ctypes.c_size_t, ptr]
    lib.vsr_pages_update.restype = ctypes.c_int
    lib.vsr_pages_keep.argtypes = [ctypes.POINTER(VsrPages), ptr, i64, i32, ptr,
                                   ctypes.POINTER(VsrCache), ptr, i32, ptr]
    lib.vsr_pages_keep.restype = ctypes.c_int
    lib.vsr_token_logprobs_workspace_size.argtypes = [i32] * 3
    lib.vsr_token_logprobs_workspace_size.restype = ctypes.c_size_t
    lib.vsr_token_logprobs.argtypes = [ptr, i32, i32, i32, i64, ptr, i32, ptr, ptr, ptr, ptr, ptr,
                                       ptr, ctypes.c_size_t, ptr]
    lib.vsr_token_logprobs.restype = ctypes.c_int
    lib.vsr_last_error.argtypes = [ctypes.c_void_p]
    lib.vsr_last_error.restype = ctypes.c_char_p
    lib.vsr_destroy.argtypes = [ctypes.c_void_p]
    lib.vsr_destroy.restype = None
    lib.vsr_set_checks.argtypes = [ctypes.c_void_p, ctypes.c_int]
    lib.vsr_set_checks.restype = ctypes.c_int
    lib.vsr_profile_enable.argtypes = [ctypes.c_void_p, ctypes.c_int]
    lib.vsr_profile_enable.restype = ctypes.c_int
    lib.vsr_profile_read.argtypes = [ctypes.c_void_p, ctypes.POINTER(ctypes.c_double),
                                     ctypes.POINTER(ctypes.c_int32)]
    lib.vsr_profile_read.restype = ctypes.c_int
    _lib = lib
    return lib


def default_split_layers(n_layers: int) -> int:
    """Precise leading layers for a decoder of this depth: one up to 63 layers,
    two at 64 (rounding amplification grows with depth)."""
    return min(n_layers, max(1, n_layers // 32))


def default_split_mlp_layers(n_layers: int, split_layers: int) -> int:
    """Precise layers whose feed-forward block is split too: all of them past
    32 layers, none up to 32 (measured against the oracle: 28 layers stay
    well inside the per-token bound with a plain FFN; 64 layers do not)."""
    return split_layers if n_layers > 32 else 0


def make_config(cfg, max_prefix: Optional[int] = None, max_cands: Optional[int] = None,
                max_cand_len: Optional[int] = None, split_layers: Optional[int] = None,
                gemm_weights: int = 0, max_new: int = 0,
                split_mlp_layers: Optional[int] = None) -> VsrConfig:
    """vsr_config from a workload.VerifierConfig (maxima default to its sizes;
    split_layers defaults to default_split_layers(n_layers), split_mlp_layers
    to default_split_mlp_layers; max_new = 0 reserves no draft cache)."""
    if split_layers is None:
        split_layers = default_split_layers(cfg.n_layers)
    if split_mlp_layers is None:
        split_mlp_layers = default_split_mlp_layers(cfg.n_layers, split_layers)
    return VsrConfig(cfg.n_layers, cfg.d_model, cfg.n_heads, cfg.n_kv_heads, cfg.head_dim,
                     cfg.d_ff, cfg.vocab, cfg.rms_eps, cfg.rope_base, cfg.dtype,
                     max_prefix or cfg.n_prefix, max_cands or cfg.n_cands,
                     max_cand_len or cfg.cand_len, split_layers, gemm_weights, max_new,
                     split_mlp_layers)


def workspace_size(c: VsrConfig) -> int:
    return load_library().vsr_workspace_size(ctypes.byref(c))


def _ptr(t) -> int:
    return 0 if t is None else t.data_ptr()


def _hold(stream, *tensors):
    """Memory of `tensors` that are dropped is not reused before `stream` is past
    the work queued on it by then."""
    for t in tensors:
        if t is not None:
            t.record_stream(stream)


class Verifier:
    """One vsr context: workspace, borrowed weights and the current prefix.

    gemm_weights (bf16 models): "f16" keeps fp16 copies of the GEMM weight
    matrices (the bf16 values, exact for magnitudes >= 2^-17), which the GEMMs
    load without conversion; "bf16" uses the given tensors as they are.
    max_new: the most tokens draft() may generate per branch (0: no drafting).
    """

    def __init__(self, cfg, weights: Dict, device="cuda", stream=None,
                 max_prefix=None, max_cands=None, max_cand_len=None, split_layers=None,
                 gemm_weights: str = "f16", max_new: int = 0, split_mlp_layers=None):
        import torch
        self._torch = torch
        self.lib = load_library()
        self.cfg = cfg
        if gemm_weights not in ("f16", "bf16"):
            raise ValueError("gemm_weights must be 'f16' or 'bf16'")
        self.gemm_f16 = cfg.dtype == VSR_BF16 and gemm_weights == "f16"
        self.c = make_config(cfg, max_prefix, max_cands, max_cand_len, split_layers,
                             VSR_F16 if self.gemm_f16 else 0, max_new, split_mlp_layers)
        size = self.lib.vsr_workspace_size(ctypes.byref(self.c))
        if size == 0:
            raise VsrError(VSR_EINVAL, "unsupported config")
        self.device = torch.device(device)
        self.workspace = torch.empty(size, dtype=torch.uint8, device=self.device)
        self.stream = stream if stream is not None else torch.cuda.current_stream(self.device)
        h = ctypes.c_void_p()
        rc = self.lib.vsr_create(ctypes.byref(self.c), self.workspace.data_ptr(), size,
                                 self.stream.cuda_stream, ctypes.byref(h))
        if rc != VSR_OK:
            raise VsrError(rc, self.lib.vsr_last_error(None).decode())
        self.h = h
        self._has_qk_norm = False
        self.load_weights(weights)

    def _check(self, rc: int):
        if rc != VSR_OK:
            raise VsrError(rc, self.lib.vsr_last_error(self.h).decode())

    def load_weights(self, w: Dict):
        # Decoders with query/key norms carry their gains as q_norm and k_norm.
        norms = [[lw.get(k) for lw in w["layers"]] for k in ("q_norm", "k_norm")]
        gains = [t for ts in norms for t in ts if t is not None]
        if gains and len(gains) != 2 * len(w["layers"]):
            raise VsrError(VSR_EINVAL, "q_norm and k_norm must be given in every layer or none")
        for t in gains:
            if t.numel() != self.cfg.head_dim or not t.is_contiguous() or \
                    t.dtype != w["final_norm"].dtype or t.device != w["final_norm"].device:
                raise VsrError(VSR_EINVAL, "q_norm, k_norm: contiguous [head_dim] gains in the "
                                           "model's dtype and on its device expected")
        if self.gemm_f16:  # one-time fp16 copies of the GEMM matrices
            f16 = lambda t: weights_to_f16(t, self.stream)  # noqa: E731
            w = dict(w, lm_head=f16(w["lm_head"]),
                     layers=[dict(lw, **{k: f16(lw[k]) for k in GEMM_WEIGHT_KEYS})
                             for lw in w["layers"]])
        self.weights = w  # keep the borrowed tensors alive
        L = len(w["layers"])
        arrs = {}
        for k in ("attn_norm", "wqkv", "wo", "ffn_norm", "wgu", "wdown"):
            arrs[k] = (ctypes.c_void_p * max(L, 1))(*[_ptr(lw[k]) for lw in w["layers"]])
        self._arrs = arrs
        cw = VsrWeights(_ptr(w["embed"]), _ptr(w["lm_head"]), _ptr(w["final_norm"]),
                        *[ctypes.cast(arrs[k], _PP) for k in
                          ("attn_norm", "wqkv", "wo", "ffn_norm", "wgu", "wdown")])
        self._check(self.lib.vsr_load_weights(self.h, ctypes.byref(cw)))
        if gains or self._has_qk_norm:
            arrs = [(ctypes.c_void_p * L)(*map(_ptr, ts)) if gains else None for ts in norms]
            _hold(self.stream, *gains)
            self._check(self.lib.vsr_load_qk_norms(self.h, *[ctypes.cast(a, _PP) for a in arrs]))
        self._has_qk_norm, self._qk_norm = bool(gains), norms

    def set_positions(self, rot=None, pos=None, next: int = 0):
        """Positions of the prefix on several axes (vsr_set_positions) for the
        next prefills: rot a rotary() scheme; pos device int32 [n_axes][P], its
        last dim contiguous; token j after the prefix sits at next + j on every
        axis. rot None: back to one axis, row p at p. Drops the current prefix."""
        if rot is None:
            self._check(self.lib.vsr_set_positions(self.h, None, None, 0, 0, 0))
            return
        P = int(pos.shape[-1])
        stride = _check_pos(_torch_names(), rot, pos, P, self.workspace.get_device())
        _hold(self.stream, pos)
        self._check(self.lib.vsr_set_positions(self.h, ctypes.byref(rot), _ptr(pos), stride, P,
                                               int(next)))

    def prefill(self, visual, ids):
        """visual: device [Pv][d] (config dtype) or None; ids: device int32 [Pt] or None."""
        nv = 0 if visual is None else int(visual.shape[0])
        nt = 0 if ids is None else int(ids.shape[0])
        self._keep = (visual, ids)
        self._check(self.lib.vsr_prefill(self.h, _ptr(visual), nv, _ptr(ids), nt))

    def score(self, cand_ids, cand_len: Sequence[int], out=None):
        """cand_ids: device int32 [M][Cmax]; cand_len: host ints [M].

        Returns device tensors (logprobs [M][Cmax] f32, scores [M] f32,
        argmax [1] int32), valid once the stream is synchronised.
        """
        torch = self._torch
        M, cmax = int(cand_ids.shape[0]), int(cand_ids.shape[1])
        lens = (ctypes.c_int32 * M)(*[int(x) for x in cand_len])
        if out is None:
            out = (torch.empty((M, cmax), dtype=torch.float32, device=self.device),
                   torch.empty(M, dtype=torch.float32, device=self.device),
                   torch.empty(1, dtype=torch.int32, device=self.device))
        lp, sc, am = out
        self._check(self.lib.vsr_score(self.h, _ptr(cand_ids), lens, M, cmax, _ptr(lp),
                                       _ptr(sc), _ptr(am)))
        return lp, sc, am

    def verify(self, visual, ids, cand_ids, cand_len: Sequence[int], out=None):
        """prefill(visual, ids) and score(cand_ids, cand_len) as one fused
        pass; same arguments and outputs, and the prefix stays current."""
        torch = self._torch
        nv = 0 if visual is None else int(visual.shape[0])
        nt = 0 if ids is None else int(ids.shape[0])
        self._keep = (visual, ids)
        M, cmax = int(cand_ids.shape[0]), int(cand_ids.shape[1])
        lens = (ctypes.c_int32 * M)(*[int(x) for x in cand_len])
        if out is None:
            out = (torch.empty((M, cmax), dtype=torch.float32, device=self.device),
                   torch.empty(M, dtype=torch.float32, device=self.device),
                   torch.empty(1, dtype=torch.int32, device=self.device))
        lp, sc, am = out
        self._check(self.lib.vsr_verify(self.h, _ptr(visual), nv, _ptr(ids), nt, _ptr(cand_ids),
                                        lens, M, cmax, _ptr(lp), _ptr(sc), _ptr(am)))
        return lp, sc, am

    def reliability(self, branch_ids, branch_len: Sequence[int], yes_id: int, no_id: int,
                    delta: float, out=None):
        """Stage 1 of the two-stage verification against the current prefix.

        branch_ids: device int32 [M][Cmax]; branch_len: host ints [M], each >= 1.
        Returns device tensors (lp_yes_no [M][2] f32, rel [M] f32, keep [M]
        int32), valid once the stream is synchronised.
        """
        torch = self._torch
        M, cmax = int(branch_ids.shape[0]), int(branch_ids.shape[1])
        lens = (ctypes.c_int32 * M)(*[int(x) for x in branch_len])
        if out is None:
            out = (torch.empty((M, 2), dtype=torch.float32, device=self.device),
                   torch.empty(M, dtype=torch.float32, device=self.device),
                   torch.empty(M, dtype=torch.int32, device=self.device))
        lp, rel, keep = out
        self._check(self.lib.vsr_reliability(self.h, _ptr(branch_ids), lens, M, cmax,
                                             int(yes_id), int(no_id), float(delta), _ptr(lp),
                                             _ptr(rel), _ptr(keep)))
        return lp, rel, keep

    def draft(self, prompt_ids, prompt_len: Sequence[int], n_new: int, out=None):
        """Greedy parallel drafts (Eq. 5, 8-10) after the current prefix.

        prompt_ids: device int32 [M][Cmax]; prompt_len: host ints [M], each >= 1.
        Returns a device int32 tensor [M][n_new] of generated token ids, valid
        once the stream is synchronised.
        """
        torch = self._torch
        M, cmax = int(prompt_ids.shape[0]), int(prompt_ids.shape[1])
        lens = (ctypes.c_int32 * M)(*[int(x) for x in prompt_len])
        if out is None:
            out = torch.empty((M, int(n_new)), dtype=torch.int32, device=self.device)
        self._check(self.lib.vsr_draft(self.h, _ptr(prompt_ids), lens, M, cmax, int(n_new),
                                       _ptr(out)))
        return out

    def draft_ruled(self, prompt_ids, prompt_len: Sequence[int], n_new: int, repetition=None,
                    presence=None, frequency=None, bias=None, mask=None, out=None,
                    workspace=None):
        """draft() with every token picked under pick_tokens' rules (row m is
        branch m; its prompt list is the branch's prompt, its output list the
        tokens it got so far). mask: int32 words [1 or M][ceil(vocab/32)], or
        [n_new][1 or M][...] with one mask a step. out: (tokens [M][n_new] int32,
        logprobs [M][n_new] f32 or None). Returns (tokens, logprobs). The inputs must
        be ready on the context's stream and may be dropped after the call."""
        torch = _torch_names()
        M, cmax = int(prompt_ids.shape[0]), int(prompt_ids.shape[1])
        lens = (ctypes.c_int32 * M)(*[int(x) for x in prompt_len])
        step, dev = 0, self.workspace.get_device()

        def given(t, dtype, shape, what):
            if t.dtype != dtype or tuple(t.shape) != shape or not t.is_contiguous() or \
                    t.get_device() != dev:
                raise VsrError(VSR_EINVAL, f"{what}: contiguous {dtype} {list(shape)} on the "
                                           "context's device expected")

        given(prompt_ids, torch.int32, (M, cmax), "prompt_ids")
        if mask is not None and mask.dim() == 3:
            if not 0 < int(n_new) == int(mask.shape[0]):
                raise VsrError(VSR_EINVAL, "mask: one row of masks a step expected")
            step = mask.stride(0)
            rules = _token_rules(torch, M, self.cfg.vocab, dev, repetition, presence, frequency,
                                 bias, mask[0])
        else:
            rules = _token_rules(torch, M, self.cfg.vocab, dev, repetition, presence, frequency,
                                 bias, mask)
        if out is None:
            out = tuple(_empty(torch, (M, max(int(n_new), 0)), dt, self.device, self.stream)
                        for dt in (torch.int32, torch.float32))
        if workspace is None:
            size = self.lib.vsr_draft_ruled_workspace_size(ctypes.byref(self.c), M)
            workspace = _empty(torch, max(size, 256), torch.uint8, self.device, self.stream)
        tokens, logprobs = out
        given(tokens, torch.int32, (M, max(int(n_new), 0)), "tokens")
        if logprobs is not None:
            given(logprobs, torch.float32, (M, max(int(n_new), 0)), "logprobs")
        given(workspace, torch.uint8, (workspace.numel(),), "workspace")
        _hold(self.stream, prompt_ids, repetition, presence, frequency, bias, mask, tokens,
              logprobs, workspace)
        self._check(self.lib.vsr_draft_ruled(
            self.h, _ptr(prompt_ids), lens, M, cmax, int(n_new), ctypes.byref(rules), step,
            _ptr(tokens), _ptr(logprobs), _ptr(workspace), workspace.numel()))
        return tokens, logprobs

    def set_checks(self, ids: bool = True, finite: bool = True):
        """Call validator (vsr_set_checks): later calls wait for their stream
        and raise VsrError with code VSR_EID / VSR_ENONFINITE on a bad id or a
        non-finite result (their outputs are still written)."""
        self._check(self.lib.vsr_set_checks(
            self.h, (VSR_CHECK_IDS if ids else 0) | (VSR_CHECK_FINITE if finite else 0)))

    def profile(self, enable, kinds=None):
        """Turns per-stage kernel timing on or off (clears recorded launches).
        `kinds`: stage-kind names (STAGE_KINDS) to time; default all."""
        mask = 0
        if enable:
            mask = VSR_PROFILE_ALL if kinds is None else sum(1 << STAGE_KINDS.index(k) for k in kinds)
        self._check(self.lib.vsr_profile_enable(self.h, mask))

    def profile_read(self) -> Dict[str, tuple]:
        """{stage name: (summed ms, launches)} since the last read."""
        ms = (ctypes.c_double * VSR_STAGES)()
        n = (ctypes.c_int32 * VSR_STAGES)()
        self._check(self.lib.vsr_profile_read(self.h, ms, n))
        return {STAGE_NAMES[i]: (ms[i], n[i]) for i in range(VSR_STAGES) if n[i]}

    def close(self):
        if getattr(self, "h", None):
            self.lib.vsr_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def weights_to_f16(t, stream=None):
    """fp16 copy of a contiguous bf16 device tensor, rounded as the GEMMs
    round bf16 weights (vsr_weights_to_f16)."""
    import torch
    if t.dtype != torch.bfloat16 or not t.is_contiguous():
        raise VsrError(VSR_EINVAL, "weights_to_f16: contiguous bfloat16 tensor expected")
    lib = load_library()
    out = torch.empty(t.shape, dtype=torch.float16, device=t.device)
    st = stream if stream is not None else torch.cuda.current_stream(t.device)
    rc = lib.vsr_weights_to_f16(_ptr(t), _ptr(out), t.numel(), st.cuda_stream)
    if rc != VSR_OK:
        raise VsrError(rc, lib.vsr_last_error(None).decode())
    return out


def rotary(sections: Sequence[int], base: float, interleaved: bool = False) -> VsrRotary:
    """A rotary scheme (vsr_rotary): sections[x] pairs of a head turn with the
    position of axis x, in consecutive runs or with the axes in turn."""
    n = len(sections)
    if not 1 <= n <= VSR_MAX_AXES:
        raise VsrError(VSR_EINVAL, "rotary: 1 to 4 sections expected")
    return VsrRotary(n, (ctypes.c_int32 * VSR_MAX_AXES)(*sections), bool(interleaved), base)


_float_types = None  # torch float dtype -> VSR_*
_raw_stream = None   # device index -> its current stream's handle
_device_now = None   # -> the current device's index
_int32 = None        # torch.int32


def _torch_names():
    """torch (imported on first use), with the library and the names above set."""
    global _float_types, _raw_stream, _device_now, _int32
    import torch
    if _float_types is None:
        load_library()
        # (A Stream object takes longer to make than a call's whole argument list.)
        _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or \
            (lambda index: torch.cuda.current_stream(index).cuda_stream)
        _device_now = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
        _int32 = torch.int32
        # Set last: another thread that finds it set finds the rest set too.
        _float_types = {torch.float32: VSR_F32, torch.bfloat16: VSR_BF16, torch.float16: VSR_F16}
    return torch


def _call(torch, dev, stream, f, args, tensors=()):
    """f(*args, stream handle) with device index dev current, on `stream` or dev's
    current stream. tensors: what f reads and writes (held for a given stream)."""
    if dev < 0:
        raise VsrError(VSR_EINVAL, "device tensors expected")
    if stream is not None and stream.device_index != dev:
        raise VsrError(VSR_EINVAL, "a stream of the tensors' device expected")
    if stream is None:
        st = _raw_stream(dev)
    else:
        st = stream.cuda_stream
        _hold(stream, *tensors)
    if dev == _device_now():
        rc = f(*args, st)
    else:
        with torch.cuda.device(dev):
            rc = f(*args, st)
    if rc != VSR_OK:
        raise VsrError(rc, load_library().vsr_last_error(None).decode())


def _check_pos(torch, rot, pos, T, dev):
    """pos's axis stride."""
    if pos.dim() == 2 and pos.dtype is torch.int32 and pos.get_device() == dev:
        n, t = pos.shape
        axis, token = pos.stride()
        if n == rot.n_axes and t == T and (token == 1 or T <= 1):
            return axis
    raise VsrError(VSR_EINVAL, "pos: int32 [n_axes][tokens] on the heads' device, tokens "
                               "contiguous, expected")


def _heads(t, dtype, hd, dev, rows):
    """vsr_heads of t, [rows][n_heads][hd] (rows < 0: any) of dtype on device dev."""
    if t.dtype is dtype and t.get_device() == dev and t.dim() == 3:
        n, heads, d = t.shape
        ts, hs, ds = t.stride()
        if ds == 1 and d == hd and (n == rows or rows < 0):
            return VsrHeads(t.data_ptr(), heads, ts, hs)
    raise VsrError(VSR_EINVAL, "heads: [tokens][n_heads][head_dim] tensors of one dtype, device "
                               "and size, head_dim contiguous, expected")


def _rotate(rot, pos, q, k, gains, eps, q_out, k_out, k_rows, stream):
    torch = _torch_names()
    dtype, dev = q.dtype, q.get_device()
    vsr_dtype = _float_types.get(dtype)
    if vsr_dtype is None or q.dim() != 3:
        raise VsrError(VSR_EINVAL, "heads: [tokens][n_heads][head_dim] float tensors expected")
    T, nq, hd = q.shape
    pos_stride = _check_pos(torch, rot, pos, T, dev)
    if q_out is None:
        q_out = _empty(torch, (T, nq, hd), dtype, q.device, stream)
    qi, qo = _heads(q, dtype, hd, dev, T), _heads(q_out, dtype, hd, dev, T)
    ki = ko = rows = None
    cap = 0
    if k is not None:
        if k_out is None:
            if k_rows is not None:
                raise VsrError(VSR_EINVAL, "k_rows needs k_out")
            k_out = _empty(torch, k.shape, k.dtype, k.device, stream)
        ki = ctypes.byref(_heads(k, dtype, hd, dev, T))
        ko = ctypes.byref(_heads(k_out, dtype, hd, dev, -1))
        cap = k_out.size(0)
        if k_rows is not None:
            if k_rows.dtype is not torch.int32 or k_rows.numel() != T or \
                    not k_rows.is_contiguous() or k_rows.get_device() != dev:
                raise VsrError(VSR_EINVAL, "k_rows: contiguous int32 [tokens] expected")
            rows = k_rows.data_ptr()
    elif k_out is not None or k_rows is not None:
        raise VsrError(VSR_EINVAL, "k_out and k_rows need k")
    head = (ctypes.byref(rot), vsr_dtype, hd, T, pos.data_ptr(), pos_stride)
    tail = (ctypes.byref(qi), ctypes.byref(qo), ki, ko, rows, cap)
    tensors = (pos, q, k, q_out, k_out, k_rows, *(gains or ()))
    if gains is None:
        _call(torch, dev, stream, _lib.vsr_rope_axes, head + tail, tensors)
        return q_out, k_out
    gq, gk = gains
    for g in gains if k is not None else gains[:1]:
        if g is None or g.dtype is not gq.dtype or g.numel() != hd or \
                not g.is_contiguous() or g.get_device() != dev:
            raise VsrError(VSR_EINVAL, "gains: contiguous [head_dim] tensors of one float dtype "
                                       "expected")
    _call(torch, dev, stream, _lib.vsr_qk_norm_rope,
          head + (gq.data_ptr(), _ptr(gk), _float_types.get(gq.dtype, -1), eps) + tail, tensors)
    return q_out, k_out


def _empty(torch, shape, dtype, device, stream):
    """torch.empty whose memory is reused in `stream`'s order (None: the current
    stream's)."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def rope_axes(rot, pos, q, k=None, q_out=None, k_out=None, k_rows=None, stream=None):
    """Rotary positions with several axes (vsr_rope_axes). rot: rotary(...); pos:
    device int32 [n_axes][T]; q: [T][Hq][hd] and k: [T][Hk][hd], any token and head
    strides (slices of stacked QKV rows). q_out, k_out: new tensors, or given ones
    (q itself for in place; a key cache [Hk][positions][hd] as its transpose(0, 1),
    with k_rows [T] int32 its positions, -1 to leave a key out). stream: where it
    runs (None: the current one); the tensors must be ready there and may be dropped
    after the call. Returns (q_out, k_out), valid once the stream is synchronised."""
    return _rotate(rot, pos, q, k, None, 0.0, q_out, k_out, k_rows, stream)


def qk_norm_rope(rot, pos, q, k, q_gain, k_gain, eps: float, q_out=None, k_out=None, k_rows=None,
                 stream=None):
    """rope_axes() on normed heads, in the same pass (vsr_qk_norm_rope): every
    head x becomes x / sqrt(mean(x^2) + eps) * gain first. q_gain, k_gain: [hd]
    in any float dtype."""
    return _rotate(rot, pos, q, k, (q_gain, k_gain), eps, q_out, k_out, k_rows, stream)


def _rows_of(t, rows, width, dtype, dev, what):
    """(pointer, row stride) of [1 or rows][width] rows; stride 0: one for all."""
    if t is None:
        return None, 0
    if t.dim() == 2 and t.dtype is dtype and t.get_device() == dev:
        n, w = t.shape
        stride, step = t.stride()
        if w == width and (step == 1 or width == 1) and (n == rows or n == 1):
            return t.data_ptr(), 0 if n == 1 else stride
    raise VsrError(VSR_EINVAL, f"{what}: {dtype} [1 or {rows}][{width}] rows on the logits' device "
                               "expected")


def _penalty(t, rows, dtype, dev):
    if t is None:
        return None
    if t.dtype is dtype and t.numel() == rows and t.is_contiguous() and t.get_device() == dev:
        return t.data_ptr()
    raise VsrError(VSR_EINVAL, f"penalties: contiguous float32 [{rows}] on the logits' device "
                               "expected")


def _token_rules(torch, rows, vocab, dev, repetition, presence, frequency, bias, mask):
    f32 = torch.float32
    return VsrTokenRules(_penalty(repetition, rows, f32, dev), _penalty(presence, rows, f32, dev),
                         _penalty(frequency, rows, f32, dev),
                         *_rows_of(bias, rows, vocab, f32, dev, "bias"),
                         *_rows_of(mask, rows, (vocab + 31) // 32, torch.int32, dev, "mask"))


def _token_list(torch, ids, length, rows, dev, what):
    if ids is None:
        return None, 0, 0, None
    i32 = torch.int32
    if ids.dim() == 2 and ids.dtype is i32 and ids.get_device() == dev:
        r, n = ids.shape
        stride, step = ids.stride()
        if r == rows and (step == 1 or n <= 1):
            if length is None:
                return ids.data_ptr(), stride, n, None
            if length.dtype is i32 and length.numel() == rows and length.is_contiguous() and \
                    length.get_device() == dev:
                return ids.data_ptr(), stride, n, length.data_ptr()
    raise VsrError(VSR_EINVAL, f"{what}: int32 [{rows}][n] rows, {what}_len contiguous int32 "
                               f"[{rows}], on the logits' device, expected")


def pick_tokens(logits, prompt=None, prompt_len=None, output=None, output_len=None,
                repetition=None, presence=None, frequency=None, bias=None, mask=None,
                processed=None, out=None, workspace=None, stream=None):
    """The greedy pick of each row of logits under rules (vsr_pick_tokens).

    logits: device [rows][vocab], float32, bfloat16 or float16, rows at any stride
    from vocab up;
    prompt, output: int32 [rows][n] token lists, *_len int32 [rows] (all n if None);
    repetition, presence, frequency: float32 [rows]; bias: float32 [1 or rows][vocab];
    mask: int32 words [1 or rows][ceil(vocab / 32)], a set bit allows its token;
    processed: float32 [rows][vocab] to keep the logits after the rules (may be
    logits); stream as in rope_axes. Returns (token [rows] int32, logprob [rows] f32),
    or `out`, whose logprob may be None; valid once the stream is synchronised. token
    -1, logprob -inf: no token was allowed."""
    torch = _torch_names()
    lib = _lib
    dtype = _float_types.get(logits.dtype)
    if dtype is None or logits.dim() != 2 or (logits.shape[1] > 1 and logits.stride(1) != 1):
        raise VsrError(VSR_EINVAL, "logits: float rows [rows][vocab] expected")
    rows, vocab = logits.shape
    dev = logits.get_device()
    rules = lists = None
    if not (repetition is presence is frequency is bias is mask is None):
        rules = ctypes.byref(_token_rules(torch, rows, vocab, dev, repetition, presence,
                                          frequency, bias, mask))
    if not (prompt is output is None):
        lists = ctypes.byref(VsrTokenLists(
            *_token_list(torch, prompt, prompt_len, rows, dev, "prompt"),
            *_token_list(torch, output, output_len, rows, dev, "output")))
    # (A single row's stride is not looked at.)
    stride = logits.stride(0) if rows > 1 else vocab
    kept, kept_stride = None, 0
    if processed is not None:
        if processed.dtype is not torch.float32 or processed.shape != logits.shape or \
                (vocab > 1 and processed.stride(1) != 1) or processed.get_device() != dev:
            raise VsrError(VSR_EINVAL, "processed: float32 rows of the logits' shape and device "
                                       "expected")
        kept, kept_stride = processed.data_ptr(), processed.stride(0) if rows > 1 else vocab
    if out is None:
        out = (_empty(torch, rows, torch.int32, logits.device, stream),
               _empty(torch, rows, torch.float32, logits.device, stream))
    token, logprob = out
    if token.dtype is not torch.int32 or token.numel() != rows or not token.is_contiguous() or \
            token.get_device() != dev or \
            (logprob is not None and (logprob.dtype is not torch.float32 or
                                      logprob.numel() != rows or not logprob.is_contiguous() or
                                      logprob.get_device() != dev)):
        raise VsrError(VSR_EINVAL, "out: contiguous int32 [rows] and float32 [rows] on the logits' "
                                   "device expected")
    if workspace is None:
        workspace = _empty(torch, max(lib.vsr_pick_workspace_size(rows, vocab), 16), torch.uint8,
                           logits.device, stream)
    elif workspace.get_device() != dev or not workspace.is_contiguous():
        raise VsrError(VSR_EINVAL, "workspace: contiguous tensor on the logits' device expected")
    _call(torch, dev, stream, lib.vsr_pick_tokens,
          (logits.data_ptr(), dtype, rows, vocab, stride, lists, rules, kept, kept_stride,
           token.data_ptr(), _ptr(logprob), workspace.data_ptr(),
           workspace.numel() * workspace.element_size()),
          (logits, prompt, prompt_len, output, output_len, repetition, presence, frequency, bias,
           mask, processed, token, logprob, workspace))
    return token, logprob


class TokenLogprobs(NamedTuple):
    """What token_logprobs returns; None where it was not asked for."""
    logprob: object
    rank: object
    entropy: object
    top_id: object
    top_logprob: object


def token_logprobs(logits, tokens=None, top: int = 0, out=None, workspace=None, stream=None):
    """Log-probabilities of given tokens, one a row (vsr_token_logprobs).

    logits: device [rows][vocab], float32, bfloat16 or float16, rows at any stride from
    vocab up; tokens: int32 [rows], or None; top: how many of the likeliest tokens to
    list. Returns TokenLogprobs of logprob [rows], rank [rows] int32, entropy [rows],
    top_id [rows][top] int32, top_logprob [rows][top] (new ones, or `out`, whose members
    may be None)."""
    torch = _torch_names()
    dtype = _float_types.get(logits.dtype)
    if dtype is None or logits.dim() != 2 or (logits.shape[1] > 1 and logits.stride(1) != 1):
        raise VsrError(VSR_EINVAL, "logits: float rows [rows][vocab] expected")
    rows, vocab = logits.shape
    dev, i32, f32 = logits.get_device(), torch.int32, torch.float32
    if out is None:
        one, two = (rows,), (rows, top)
        new = lambda shape, dt, given: _empty(torch, shape, dt, logits.device, stream) \
            if given else None  # noqa: E731
        out = TokenLogprobs(new(one, f32, tokens is not None), new(one, i32, tokens is not None),
                            new(one, f32, True), new(two, i32, top), new(two, f32, top))
    else:
        out = TokenLogprobs(*out)
    ptrs = []
    for name, t, dt, n in (("tokens", tokens, i32, rows), ("logprob", out.logprob, f32, rows),
                           ("rank", out.rank, i32, rows), ("entropy", out.entropy, f32, rows),
                           ("top_id", out.top_id, i32, rows * top),
                           ("top_logprob", out.top_logprob, f32, rows * top)):
        if t is None:
            ptrs.append(None)
        elif t.dtype is dt and t.numel() == n and t.is_contiguous() and t.get_device() == dev:
            ptrs.append(t.data_ptr())
        else:
            raise VsrError(VSR_EINVAL, f"{name}: contiguous {dt} of {n} on the logits' device "
                                       "expected")
    if workspace is None:
        size = _lib.vsr_token_logprobs_workspace_size(rows, vocab, top)
        workspace = _empty(torch, max(size, 16), torch.uint8, logits.device, stream)
    elif workspace.get_device() != dev or not workspace.is_contiguous():
        raise VsrError(VSR_EINVAL, "workspace: contiguous tensor on the logits' device expected")
    # (A single row's stride is not looked at.)
    _call(torch, dev, stream, _lib.vsr_token_logprobs,
          (logits.data_ptr(), dtype, rows, vocab, logits.stride(0) if rows > 1 else vocab, ptrs[0],
           top, *ptrs[1:], workspace.data_ptr(), workspace.numel() * workspace.element_size()),
          (logits, tokens, *out, workspace))
    return out


class Pages:
    """A paged cache's tables (vsr_pages): the tensors and what they hold."""

    def __init__(self, table, len, held, refs, page_size: int):
        i32, dev = _torch_names().int32, table.get_device()
        if table.dtype is not i32 or table.dim() != 2:
            raise VsrError(VSR_EINVAL, "table: int32 [n_seqs][max_pages] rows expected")
        seqs, most = table.shape
        rows, step = table.stride()
        if most > 1 and step != 1:
            raise VsrError(VSR_EINVAL, "table: int32 [n_seqs][max_pages] rows expected")
        n_pages = refs.numel()
        at = [_int_rows(t, n, dev, what) for t, n, what in
              ((len, seqs, "len"), (held, seqs, "held"), (refs, n_pages, "refs"))]
        if not len.dim() == held.dim() == refs.dim() == 1:
            raise VsrError(VSR_EINVAL, "len, held, refs: one dimension expected")
        self.table, self.len, self.held, self.refs = table, len, held, refs
        self.n_seqs, self.max_pages, self.n_pages, self.page_size = seqs, most, n_pages, \
            int(page_size)
        self.device_index = dev
        self.c = VsrPages(seqs, n_pages, self.page_size, most, table.data_ptr(),
                          rows if seqs > 1 else most, *at)

    def tensors(self):
        return self.table, self.len, self.held, self.refs


def pages(table, len, held, refs, page_size: int) -> Pages:
    """The tables of a paged key/value cache (vsr_pages), device int32: table
    [n_seqs][max_pages] (row s: the pages sequence s holds, in order), len [n_seqs]
    positions in use, held [n_seqs] pages held, refs [n_pages] how many sequences hold
    a page. page_size: positions a page, a power of two; slot page * page_size + i of
    the cache is position i of a page."""
    return Pages(table, len, held, refs, page_size)


def _int_rows(t, n, dev, what):
    """Pointer of a contiguous int32 [n] tensor, or None."""
    if t is None:
        return None
    if t.dtype is _int32 and t.numel() == n and t.is_contiguous() and t.get_device() == dev:
        return t.data_ptr()
    raise VsrError(VSR_EINVAL, f"{what}: contiguous int32 [{n}] on the pages' device expected")


def _mask_rows(mask, T, dev):
    """(pointer, row stride, words) of int32 [T][words] rows."""
    if mask is None:
        return None, 0, 0
    if mask.dim() == 2 and mask.dtype is _int32 and mask.get_device() == dev:
        n, words = mask.shape
        stride, step = mask.stride()
        if n == T and (step == 1 or words == 1):
            return mask.data_ptr(), stride if n > 1 else words, words
    raise VsrError(VSR_EINVAL, f"mask: int32 [{T}][words] rows on the pages' device expected")


def tree_rows(pages, start, parent=None, shift=None, words: Optional[int] = None, out=None,
              stream=None):
    """Positions, cache slots and ancestor masks of drafted rows (vsr_tree_rows).

    start: int32 [n_seqs + 1], sequence s has rows start[s] .. start[s + 1] - 1, or None
    (a row a sequence); parent: int32 [T], each row's parent within its sequence, -1 a
    root (None: each row's is the one before it); shift: int32 [n_seqs] added to the
    positions. out: (pos [T], slot [T], mask [T][words] or None), int32; new ones have
    `words` words of mask (None: no mask; T comes from parent or is n_seqs).
    Returns (pos, slot, mask)."""
    torch = _torch_names()
    dev = pages.device_index
    if out is None:
        T = pages.n_seqs if start is None else None if parent is None else parent.numel()
        if T is None:
            raise VsrError(VSR_EINVAL, "tree_rows: parent or out expected with start")
        new = lambda *s: _empty(torch, s, torch.int32, pages.table.device, stream)  # noqa: E731
        out = new(T), new(T), new(T, words) if words else None
    pos, slot, mask = out
    T = pos.numel()
    args = (ctypes.byref(pages.c), T, _int_rows(start, pages.n_seqs + 1, dev, "start"),
            _int_rows(parent, T, dev, "parent"), _int_rows(shift, pages.n_seqs, dev, "shift"),
            _int_rows(pos, T, dev, "pos"), _int_rows(slot, T, dev, "slot"),
            *_mask_rows(mask, T, dev))
    _call(torch, dev, stream, _lib.vsr_tree_rows, args,
          (*pages.tensors(), start, parent, shift, *out))
    return pos, slot, mask


def tree_attention(pages, q, k, v, scale: float, start=None, mask=None, out=None, lse=None,
                   workspace=None, stream=None):
    """Attention of drafted rows over their sequences' pages (vsr_tree_attention).

    q: [T][n_heads][head_dim]; k, v: one layer's slots [n_pages * page_size]
    [n_kv_heads][head_dim], any slot and head strides; start: as in tree_rows; mask:
    int32 [T][words], bit i of a row lets it see row i of its sequence's draft (None:
    every row sees those before it and itself); out: like q (None: new; rows of no
    sequence are left as they are); lse: float32 [T][n_heads] to fill, or None. Returns
    out."""
    torch = _torch_names()
    dtype, dev = q.dtype, pages.device_index
    vsr_dtype = _float_types.get(dtype)
    if vsr_dtype is None or q.dim() != 3 or k.dim() != 3:
        raise VsrError(VSR_EINVAL, "q, k, v: [rows][n_heads][head_dim] float tensors expected")
    T, nq, hd = q.shape
    slots = pages.n_pages * pages.page_size
    if out is None:
        out = _empty(torch, (T, nq, hd), dtype, q.device, stream)
    qh, oh = _heads(q, dtype, hd, dev, T), _heads(out, dtype, hd, dev, T)
    kh, vh = _heads(k, dtype, hd, dev, slots), _heads(v, dtype, hd, dev, slots)
    if lse is not None and (lse.dtype is not torch.float32 or lse.shape != (T, nq) or
                            not lse.is_contiguous() or lse.get_device() != dev):
        raise VsrError(VSR_EINVAL, "lse: contiguous float32 [rows][n_heads] expected")
    if workspace is None:
        size = _lib.vsr_tree_attention_workspace_size(vsr_dtype, hd, T, pages.n_seqs, nq,
                                                      k.shape[1])
        workspace = _empty(torch, max(size, 256), torch.uint8, q.device, stream)
    elif workspace.get_device() != dev or not workspace.is_contiguous():
        raise VsrError(VSR_EINVAL, "workspace: contiguous tensor on the pages' device expected")
    _call(torch, dev, stream, _lib.vsr_tree_attention,
          (ctypes.byref(pages.c), vsr_dtype, hd, T,
           _int_rows(start, pages.n_seqs + 1, dev, "start"), ctypes.byref(qh), ctypes.byref(kh),
           ctypes.byref(vh), *_mask_rows(mask, T, dev), scale, ctypes.byref(oh), _ptr(lse) or None,
           workspace.data_ptr(), workspace.numel() * workspace.element_size()),
          (*pages.tensors(), q, k, v, start, mask, out, lse, workspace))
    return out


def _cache(pages, k, v):
    """vsr_cache of k and v, [n_layers][slots][n_kv_heads][head_dim]."""
    dtype = _float_types.get(k.dtype)
    if dtype is not None and v.dtype is k.dtype and k.dim() == 4 and v.shape == k.shape and \
            v.stride() == k.stride() and k.get_device() == v.get_device() == pages.device_index:
        L, slots, heads, hd = k.shape
        ls, ss, hs, ds = k.stride()
        if (ds == 1 or hd == 1) and slots == pages.n_pages * pages.page_size:
            return VsrCache(k.data_ptr(), v.data_ptr(), dtype, L, heads, hd, ls, ss, hs)
    raise VsrError(VSR_EINVAL, "k, v: [n_layers][n_pages * page_size][n_kv_heads][head_dim] "
                               "tensors of one float dtype and the same strides, head_dim "
                               "contiguous, on the pages' device expected")


def pages_update(pages, source=None, room=None, k=None, v=None, ok=None, workspace=None,
                 stream=None):
    """Sequences forked, dropped and given room (vsr_pages_update): sequence d becomes
    what source[d] was (-1: empty; None: all stay) and then has pages for room[d]
    positions more. source, room: int32 [n_seqs]; k, v: the cache in every layer,
    [n_layers][n_pages * page_size][n_kv_heads][head_dim] (needed with source: partly
    filled pages are copied). Returns ok, int32 [n_seqs]: 1 where a sequence got all of
    it."""
    torch = _torch_names()
    dev, n = pages.device_index, pages.n_seqs
    if ok is None:
        ok = _empty(torch, n, torch.int32, pages.table.device, stream)
    cache, size = None, 0
    if source is not None:
        if k is None or v is None:
            raise VsrError(VSR_EINVAL, "pages_update: source needs k and v")
        cache = ctypes.byref(_cache(pages, k, v))
        if workspace is None:
            size = _lib.vsr_pages_update_workspace_size(n)
            workspace = _empty(torch, size, torch.uint8, pages.table.device, stream)
    if workspace is not None:
        if workspace.get_device() != dev or not workspace.is_contiguous():
            raise VsrError(VSR_EINVAL, "workspace: contiguous tensor on the pages' device expected")
        size = workspace.numel() * workspace.element_size()
    _call(torch, dev, stream, _lib.vsr_pages_update,
          (ctypes.byref(pages.c), _int_rows(source, n, dev, "source"),
           _int_rows(room, n, dev, "room"), cache, _int_rows(ok, n, dev, "ok"),
           _ptr(workspace) or None, size),
          (*pages.tensors(), source, room, k, v, ok, workspace))
    return ok


def pages_keep(pages, kept, n_kept, k, v, len_out=None, release: bool = True, stream=None):
    """The kept rows of every sequence's draft moved together in every layer
    (vsr_pages_keep): the row at position len + kept[s][i] goes to len + i for i <
    n_kept[s], and the length becomes len + n_kept. kept: int32 [n_seqs][max_kept],
    rising; n_kept: int32 [n_seqs], or None (max_kept); k, v as in pages_update; len_out:
    where the new lengths go (None: pages.len); release: give back the pages past them.
    Returns the new lengths."""
    torch = _torch_names()
    dev, n = pages.device_index, pages.n_seqs
    if len_out is None:
        len_out = pages.len
    if kept.dim() != 2 or kept.dtype is not torch.int32 or kept.shape[0] != n or \
            (kept.shape[1] > 1 and kept.stride(1) != 1) or kept.get_device() != dev:
        raise VsrError(VSR_EINVAL, f"kept: int32 [{n}][max_kept] rows on the pages' device expected")
    most = kept.shape[1]
    cache = _cache(pages, k, v)
    _call(torch, dev, stream, _lib.vsr_pages_keep,
          (ctypes.byref(pages.c), kept.data_ptr() if most else None,
           kept.stride(0) if n > 1 and most else most, most, _int_rows(n_kept, n, dev, "n_kept"),
           ctypes.byref(cache), _int_rows(len_out, n, dev, "len_out"), bool(release)),
          (*pages.tensors(), kept, n_kept, k, v, len_out))
    return len_out


def align_select(ent, frames, rel, delta: float, strategy: str = "two_stage", out=None,
                 stream=None):
    """Entity alignment (Eq. 14-15) and the final choice (Algorithm 1 or a
    Table 3 strategy). ent: device f32 [M][D]; frames: device f32 [NF][D];
    rel: device f32 [M]. Returns device tensors (align [M] f32, choice [1]
    int32), valid once the stream is synchronised."""
    import torch
    lib = load_library()
    M, D = int(ent.shape[0]), int(ent.shape[1])
    NF = int(frames.shape[0])
    if int(frames.shape[1]) != D or int(rel.shape[0]) != M:
        raise VsrError(VSR_EINVAL, "align_select: shapes of ent, frames and rel disagree")
    for t in (ent, frames, rel):
        if t.dtype != torch.float32 or not t.is_contiguous():
            raise VsrError(VSR_EINVAL, "align_select: contiguous float32 tensors expected")
    if out is None:
        out = (torch.empty(M, dtype=torch.float32, device=ent.device),
               torch.empty(1, dtype=torch.int32, device=ent.device))
    align, choice = out
    st = stream if stream is not None else torch.cuda.current_stream(ent.device)
    rc = lib.vsr_align_select(_ptr(ent), _ptr(frames), M, NF, D, _ptr(rel), float(delta),
                              SELECT_STRATEGIES[strategy], _ptr(align), _ptr(choice),
                              st.cuda_stream)
    if rc != VSR_OK:
        raise VsrError(rc, lib.vsr_last_error(None).decode())
    return align, choice


class Retriever:
    """The retrieval stage on the device: keyframes (Eq. 1), then per-keyframe
    top-k documents and T* (Eq. 2-3). Holds the output and workspace tensors
    for one video size and document bank."""

    def __init__(self, n_frames: int, height: int, width: int, n_docs: int, dim: int, k: int,
                 K: int, device="cuda", stream=None):
        import torch
        self._torch = torch
        self.lib = load_library()
        self.NF, self.H, self.W, self.ND, self.D, self.k, self.K = (
            n_frames, height, width, n_docs, dim, k, K)
        dev = torch.device(device)
        i32 = dict(dtype=torch.int32, device=dev)
        f32 = dict(dtype=torch.float32, device=dev)
        self.hist = torch.empty((n_frames, 3, 64), **i32)
        self.inter = torch.empty(n_frames, **i32)
        self.key_idx = torch.empty(n_frames, **i32)
        self.n_keys = torch.empty(1, **i32)
        size = self.lib.vsr_retrieve_workspace_size(n_frames, n_docs, k)
        if size == 0:
            raise VsrError(VSR_EINVAL, "unsupported retrieval sizes")
        self.ws = torch.empty(size, dtype=torch.uint8, device=dev)
        self.top_idx = torch.empty((n_frames, k), **i32)
        self.top_sim = torch.empty((n_frames, k), **f32)
        self.sel_idx = torch.empty(K, **i32)
        self.sel_sim = torch.empty(K, **f32)
        self.n_sel = torch.empty(1, **i32)
        self.stream = stream if stream is not None else torch.cuda.current_stream(dev)

    def _check(self, rc):
        if rc != VSR_OK:
            raise VsrError(rc, self.lib.vsr_last_error(None).decode())

    def keyframes(self, frames, theta: float):
        """frames: device uint8 [NF][H][W][3] -> (key_idx, n_keys) device tensors."""
        self._frames = frames
        self._check(self.lib.vsr_keyframes(_ptr(frames), self.NF, self.H, self.W, float(theta),
                                           _ptr(self.hist), _ptr(self.inter),
                                           _ptr(self.key_idx), _ptr(self.n_keys),
                                           self.stream.cuda_stream))
        return self.key_idx, self.n_keys

    def retrieve(self, frame_emb, docs):
        """frame_emb: device f32 [NF][D]; docs: device f32 [ND][D]. Uses the
        keyframes of the last keyframes() call. Returns device tensors
        (top_idx [NF][k], top_sim, sel_idx [K], sel_sim, n_sel)."""
        self._emb = (frame_emb, docs)
        self._check(self.lib.vsr_retrieve(
            _ptr(frame_emb), _ptr(self.key_idx), _ptr(self.n_keys), self.NF, _ptr(docs),
            self.ND, self.D, self.k, self.K, _ptr(self.ws), self.ws.numel(), _ptr(self.top_idx),
            _ptr(self.top_sim), _ptr(self.sel_idx), _ptr(self.sel_sim), _ptr(self.n_sel),
            self.stream.cuda_stream))
        return self.top_idx, self.top_sim, self.sel_idx, self.sel_sim, self.n_sel

    def retrieve_static(self, frame_emb, docs):
        """retrieve() through vsr_retrieve_static: the library's static
        scratch instead of this object's workspace (no allocation in the call)."""
        self._emb = (frame_emb, docs)
        self._check(self.lib.vsr_retrieve_static(
            _ptr(frame_emb), _ptr(self.key_idx), _ptr(self.n_keys), self.NF, _ptr(docs),
            self.ND, self.D, self.k, self.K, _ptr(self.top_idx), _ptr(self.top_sim),
            _ptr(self.sel_idx), _ptr(self.sel_sim), _ptr(self.n_sel), self.stream.cuda_stream))
        return self.top_idx, self.top_sim, self.sel_idx, self.sel_sim, self.n_sel


def verifier_from_workload(wl, device="cuda", **kw) -> Verifier:
    return Verifier(wl.cfg, wl.weights, device=device, **kw)
