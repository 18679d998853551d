"""ctypes binding of libdllm.so (the C ABI in include/dllm.h).

Argument marshalling only: every step of the decode runs in the library's HIP
kernels.  PyTorch supplies device memory and the stream.  Importing this
module does not load the library; ``lib()`` does, and raises if the library
has not been built (python -m paper_2608_22646_amd.build).
"""
from __future__ import annotations

import ctypes
import itertools
import math
import os
from dataclasses import dataclass

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libdllm.so")

DLLM_F32, DLLM_BF16 = 0, 1
F_BLOCK_SCHED, F_POS, F_BUDGET, F_GRIND, F_FIXED = 1, 2, 4, 8, 16
ROPE_PLAIN, ROPE_LINEAR, ROPE_PARTS = 0, 1, 2
R_MASKED, R_THRESH, R_BUDGET, R_GRIND, R_FLUSH, R_FIXED = 0, 1, 2, 3, 4, 5
PROF_QKV, PROF_ATTN, PROF_HEAD, PROF_COMMIT, PROF_NORM, PROF_GATEUP, PROF_OPROJ, PROF_DOWN = range(8)

_c = ctypes
_i32, _i64, _u32 = _c.c_int32, _c.c_int64, _c.c_uint32
_f32, _f64, _vp, _sz = _c.c_float, _c.c_double, _c.c_void_p, _c.c_size_t


class ModelCfg(_c.Structure):
    _fields_ = [("n_layers", _i32), ("d_model", _i32), ("n_heads", _i32), ("n_kv_heads", _i32),
                ("head_dim", _i32), ("d_ff", _i32), ("vocab", _i32), ("mask_id", _i32),
                ("rms_eps", _f32), ("rope_base", _f64), ("dtype", _i32)]


class CaiParams(_c.Structure):
    _fields_ = [("block_len", _i32), ("steps_per_block", _i32),
                ("theta_s", _f64), ("theta_e", _f64), ("theta_e_step", _f64), ("theta_e_floor", _f64),
                ("warmup", _f64), ("pos_edge", _i32 * 3), ("pos_factor", _f64 * 4),
                ("clip_lo", _f64), ("clip_hi", _f64), ("s_easy", _f32), ("s_hard", _f32),
                ("p_easy", _i32), ("p_hard", _i32), ("budget_easy", _i32), ("budget_mid", _i32),
                ("budget_hard", _i32), ("eta_bar", _f64), ("patience", _i32), ("theta_fb", _f32),
                ("flags", _u32)]


class State(_c.Structure):
    _fields_ = [("x", _vp), ("commit_step", _vp), ("reason", _vp), ("s", _vp), ("budget", _vp),
                ("ell", _vp), ("done", _vp)]


class WsLayout(_c.Structure):
    _fields_ = [(n, _sz) for n in ("total", "h", "a_attn", "q", "k", "vt", "attn", "a_mlp", "u", "hb")]


class RotaryCfg(_c.Structure):
    _fields_ = [("head_dim", _i32), ("rot_dim", _i32), ("interleaved", _i32), ("scaling", _i32), ("base", _f64),
                ("factor", _f64), ("orig_len", _f64), ("low", _f64), ("high", _f64), ("gain", _f64)]


class View(_c.Structure):
    _fields_ = [("data", _vp), ("stride_b", _i64), ("stride_l", _i64), ("stride_h", _i64)]


class AttnArgs(_c.Structure):
    _fields_ = [("dtype", _i32), ("n_heads", _i32), ("n_kv_heads", _i32), ("head_dim", _i32), ("q", View), ("k", View),
                ("v", View), ("out", View), ("docs", _i32), ("q_tokens", _i32), ("kv_tokens", _i32), ("max_q", _i32),
                ("max_kv", _i32), ("q_start", _vp), ("q_len", _vp), ("kv_start", _vp), ("kv_len", _vp), ("q_pos", _vp),
                ("prefix", _vp), ("slopes", _vp), ("scale", _f32), ("cap", _f32), ("block", _i32)]


class SampleArgs(_c.Structure):
    _fields_ = [("logits", _vp), ("row_stride", _i64), ("dtype", _i32), ("rows", _i32), ("vocab", _i32),
                ("mask_id", _i32), ("u", _vp), ("temperature", _vp), ("top_k", _vp), ("top_p", _vp), ("min_p", _vp),
                ("token", _vp), ("conf", _vp), ("prob", _vp)]


class DllmError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"dllm error {code}: {msg}")
        self.code = code


_LIB = None

_SIGS = {
    "dllm_last_error": (_c.c_char_p, []),
    "dllm_model_buffer_size": (_i32, [_c.POINTER(ModelCfg), _c.POINTER(_sz)]),
    "dllm_model_create": (_i32, [_c.POINTER(ModelCfg), _c.POINTER(_vp), _i32, _vp, _sz, _vp, _c.POINTER(_vp)]),
    "dllm_model_destroy": (_i32, [_vp]),
    "dllm_model_packed_size": (_i32, [_vp, _c.POINTER(_sz)]),
    "dllm_model_pack_weights": (_i32, [_vp, _vp, _sz, _vp]),
    "dllm_workspace_size": (_i32, [_vp, _i32, _i32, _i32, _c.POINTER(_sz)]),
    "dllm_workspace_layout": (_i32, [_vp, _i32, _i32, _i32, _c.POINTER(WsLayout)]),
    "dllm_embed": (_i32, [_vp, _vp, _i32, _i32, _vp, _sz, _vp]),
    "dllm_layer": (_i32, [_vp, _i32, _i32, _i32, _i32, _vp, _sz, _vp]),
    "dllm_head": (_i32, [_vp, _i32, _i32, _i32, _i32, _vp, _vp, _vp, _vp, _sz, _vp]),
    "dllm_forward": (_i32, [_vp, _vp, _i32, _i32, _i32, _i32, _vp, _vp, _vp, _vp, _sz, _vp]),
    "dllm_head_noalloc": (_i32, [_vp, _vp, _i32, _i32, _i32, _i32, _vp, _vp, _vp, _vp]),
    "dllm_state_init": (_i32, [_i32, _vp, _i32, _i32, _i32, _c.POINTER(State), _vp]),
    "dllm_commit": (_i32, [_c.POINTER(CaiParams), _c.POINTER(State), _vp, _vp, _i32, _i32, _i32, _i32, _i32,
                           _i32, _vp, _vp]),
    "dllm_step": (_i32, [_vp, _c.POINTER(CaiParams), _c.POINTER(State), _i32, _i32, _i32, _i32, _i32, _vp, _vp,
                         _vp, _vp, _sz, _vp]),
    "dllm_generate": (_i32, [_vp, _c.POINTER(CaiParams), _vp, _i32, _i32, _i32, _c.POINTER(State), _vp, _vp,
                             _vp, _vp, _vp, _sz, _vp]),
    "dllm_kv_cache_size": (_i32, [_vp, _i32, _i32, _c.POINTER(_sz)]),
    "dllm_forward_kv": (_i32, [_vp, _vp, _i32, _i32, _i32, _i32, _i32, _vp, _vp, _vp, _vp, _sz, _vp, _sz, _vp]),
    "dllm_embed_rows": (_i32, [_vp, _vp, _i32, _i32, _i32, _i32, _vp, _sz, _vp]),
    "dllm_layer_kv": (_i32, [_vp, _i32, _i32, _i32, _i32, _i32, _i32, _vp, _sz, _vp, _sz, _vp]),
    "dllm_step_kv": (_i32, [_vp, _c.POINTER(CaiParams), _i32, _c.POINTER(State), _i32, _i32, _i32, _i32, _i32, _vp,
                            _vp, _vp, _vp, _sz, _vp, _sz, _vp]),
    "dllm_generate_kv": (_i32, [_vp, _c.POINTER(CaiParams), _i32, _vp, _i32, _i32, _i32, _c.POINTER(State), _vp,
                                _vp, _vp, _vp, _vp, _sz, _vp, _sz, _vp]),
    "dllm_rotary": (_i32, [_c.POINTER(RotaryCfg), _i32, _i32, _i32, _vp, _i32, _c.POINTER(View), _c.POINTER(View), _i32,
                           _c.POINTER(View), _c.POINTER(View), _i32, _i32, _vp]),
    "dllm_attention_workspace_size": (_i32, [_c.POINTER(AttnArgs), _c.POINTER(_sz)]),
    "dllm_attention": (_i32, [_c.POINTER(AttnArgs), _vp, _sz, _vp]),
    "dllm_sample_workspace_size": (_i32, [_i32, _i32, _c.POINTER(_sz)]),
    "dllm_sample": (_i32, [_c.POINTER(SampleArgs), _vp, _sz, _vp]),
    "dllm_prof_enable": (_i32, [_vp, _i32]),
    "dllm_prof_read": (_i32, [_vp, _i32, _c.POINTER(_f64), _c.POINTER(_c.c_int64)]),
    "dllm_prof_every": (_i32, [_vp, _i32]),
}


def lib():
    """Load libdllm.so (once).  Raises if it has not been built."""
    global _LIB
    if _LIB is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with python -m paper_2608_22646_amd.build")
        L = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in _SIGS.items():
            f = getattr(L, name)
            f.restype = res
            f.argtypes = args
        _LIB = L
    return _LIB


def check(rc):
    if rc != 0:
        raise DllmError(rc, lib().dllm_last_error().decode())
    return rc


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(stream=None):
    s = stream if stream is not None else torch.cuda.current_stream()
    return ctypes.c_void_p(s.cuda_stream)


def device_buffer(nbytes, device="cuda"):
    """A caller-owned, 256-byte aligned uint8 device tensor of nbytes bytes."""
    buf = torch.empty(nbytes + 256, dtype=torch.uint8, device=device)
    off = (-buf.data_ptr()) % 256
    return buf[off:off + nbytes]


# ---------------------------------------------------------------- parameters
@dataclass
class Controller:
    """Controller constants (defaults as printed in the paper, Boxes 3-7)."""
    block_len: int = 32
    steps_per_block: int = 0
    theta_s: float = 0.90
    theta_e: float = 0.70
    theta_e_step: float = 0.10
    theta_e_floor: float = 0.40
    warmup: float = 0.15
    pos_edges: tuple = (16, 32, 48)
    pos_factors: tuple = (0.80, 0.90, 1.05, 1.10)
    clip_lo: float = 0.20
    clip_hi: float = 0.98
    s_easy: float = 0.50
    s_hard: float = 0.25
    p_easy: int = 32
    p_hard: int = 48
    budget_easy: int = 8
    budget_mid: int = 32
    budget_hard: int = 64
    eta_bar: float = 1.5
    patience: int = 4
    theta_fb: float = 0.40
    block_sched: bool = True
    pos_aware: bool = True
    budgets: bool = True
    grinding: bool = True
    fixed: bool = False   # fixed-schedule baseline instead of the confidence rule

    @classmethod
    def gating(cls, on: bool, **kw):
        return cls(budgets=on, grinding=on, **kw)

    @classmethod
    def preset(cls, name: str, **kw):
        """Named controller settings: the method with gating on / off (Section 4.6),
        the component ablation of Section 6 (+APD, +Block, +Budget = the
        per-token controls of Boxes 5-7), fixed-threshold decoding and the
        fixed-schedule baseline.  Keyword arguments override fields."""
        apd_only = dict(block_sched=False, pos_aware=False, budgets=False, grinding=False)
        table = {
            "cai": {},
            "cai_gate_off": dict(budgets=False, grinding=False),
            "apd": apd_only,
            "apd_block": dict(pos_aware=False, budgets=False, grinding=False),
            "apd_block_budget": {},
            "fixed_threshold_0.9": dict(apd_only, theta_s=0.9, theta_e=0.9),
            "fixed_threshold_0.7": dict(apd_only, theta_s=0.7, theta_e=0.7),
            "apd_0.9_to_0.5": dict(apd_only, theta_s=0.9, theta_e=0.5),
            "fixed_schedule": dict(fixed=True),
        }
        if name not in table:
            raise KeyError(f"unknown controller preset {name!r}; known: {sorted(table)}")
        return cls(**dict(table[name], **kw))

    def to_c(self) -> CaiParams:
        p = CaiParams()
        for f in ("block_len", "steps_per_block", "theta_s", "theta_e", "theta_e_step", "theta_e_floor", "warmup",
                  "clip_lo", "clip_hi", "s_easy", "s_hard", "p_easy", "p_hard", "budget_easy", "budget_mid",
                  "budget_hard", "eta_bar", "patience", "theta_fb"):
            setattr(p, f, getattr(self, f))
        p.pos_edge[:] = list(self.pos_edges)
        p.pos_factor[:] = list(self.pos_factors)
        p.flags = ((F_BLOCK_SCHED if self.block_sched else 0) | (F_POS if self.pos_aware else 0)
                   | (F_BUDGET if self.budgets else 0) | (F_GRIND if self.grinding else 0)
                   | (F_FIXED if self.fixed else 0))
        return p

    @property
    def T(self):
        return self.steps_per_block or self.block_len


def model_cfg(cfg) -> ModelCfg:
    """ModelCfg from any object with the synth.ModelConfig fields."""
    return ModelCfg(n_layers=cfg.n_layers, d_model=cfg.d_model, n_heads=cfg.n_heads, n_kv_heads=cfg.n_kv_heads,
                    head_dim=cfg.head_dim, d_ff=cfg.d_ff, vocab=cfg.vocab, mask_id=cfg.vocab - 1,
                    rms_eps=cfg.rms_eps, rope_base=cfg.rope_base,
                    dtype=DLLM_F32 if cfg.dtype == "f32" else DLLM_BF16)


# ---------------------------------------------------------------- objects
class DecodeState:
    """Device tensors of the decoding state (dllm_state)."""

    def __init__(self, B, P, G, device="cuda"):
        L = P + G
        self.B, self.P, self.G = B, P, G
        self.x = torch.zeros((B, L), dtype=torch.int32, device=device)
        self.commit_step = torch.zeros((B, G), dtype=torch.int32, device=device)
        self.reason = torch.zeros((B, G), dtype=torch.int8, device=device)
        self.s = torch.zeros((B, G), dtype=torch.float32, device=device)
        self.budget = torch.zeros((B, G), dtype=torch.int32, device=device)
        self.ell = torch.zeros((B,), dtype=torch.int32, device=device)
        self.done = torch.zeros((B,), dtype=torch.int32, device=device)

    def c(self) -> State:
        return State(*[t.data_ptr() for t in (self.x, self.commit_step, self.reason, self.s, self.budget, self.ell,
                                               self.done)])

    def snapshot(self):
        return {k: getattr(self, k).clone() for k in ("x", "commit_step", "reason", "s", "budget", "ell", "done")}

    def restore(self, snap):
        for k, v in snap.items():
            getattr(self, k).copy_(v)


class Model:
    """A model handle over caller-owned device weights and model buffer (both
    kept alive here).  The LM-head copy is written on the current stream."""

    def __init__(self, cfg, weights, stream=None):
        L = lib()
        self.cfg = cfg
        self.mask_id = cfg.vocab - 1
        self.weights = list(weights)
        self._c = model_cfg(cfg)
        n = ctypes.c_size_t()
        check(L.dllm_model_buffer_size(ctypes.byref(self._c), ctypes.byref(n)))
        dev = self.weights[0].device
        self.model_buf = device_buffer(n.value, dev) if n.value else None
        self.packed_buf = None
        arr = (ctypes.c_void_p * len(self.weights))(*[w.data_ptr() for w in self.weights])
        h = ctypes.c_void_p()
        check(L.dllm_model_create(ctypes.byref(self._c), arr, len(self.weights), _ptr(self.model_buf), n.value,
                                  _stream(stream), ctypes.byref(h)))
        self.h = h

    def packed_size(self):
        n = ctypes.c_size_t()
        check(lib().dllm_model_packed_size(self.h, ctypes.byref(n)))
        return n.value

    def pack_weights(self, stream=None):
        """dllm_model_pack_weights: tiled copies of the projection weights for the
        block-row GEMMs, in a buffer allocated here (once)."""
        if self.packed_buf is None:
            n = self.packed_size()
            buf = device_buffer(n, self.weights[0].device)
            check(lib().dllm_model_pack_weights(self.h, _ptr(buf), n, _stream(stream)))
            self.packed_buf = buf
        return self

    def close(self):
        if getattr(self, "h", None):
            lib().dllm_model_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # workspace --------------------------------------------------------------
    def workspace_size(self, B, L, rows):
        n = ctypes.c_size_t()
        check(lib().dllm_workspace_size(self.h, B, L, rows, ctypes.byref(n)))
        return n.value

    def workspace(self, B, L, rows, device="cuda"):
        return device_buffer(self.workspace_size(B, L, rows), device)

    def layout(self, B, L, rows) -> WsLayout:
        out = WsLayout()
        check(lib().dllm_workspace_layout(self.h, B, L, rows, ctypes.byref(out)))
        return out

    # stages -----------------------------------------------------------------
    def embed(self, x, ws, stream=None):
        B, L = x.shape
        check(lib().dllm_embed(self.h, _ptr(x), B, L, _ptr(ws), ws.numel(), _stream(stream)))

    def layer(self, layer, part, B, L, ws, stream=None):
        check(lib().dllm_layer(self.h, layer, part, B, L, _ptr(ws), ws.numel(), _stream(stream)))

    def head(self, B, L, row0, rows, ws, logits=False, stream=None):
        dev = ws.device
        conf = torch.empty((B * rows,), dtype=torch.float32, device=dev)
        arg = torch.empty((B * rows,), dtype=torch.int32, device=dev)
        lg = torch.empty((B * rows, self.cfg.vocab), dtype=torch.float32, device=dev) if logits else None
        check(lib().dllm_head(self.h, B, L, row0, rows, _ptr(conf), _ptr(arg), _ptr(lg), _ptr(ws), ws.numel(),
                              _stream(stream)))
        return conf.view(B, rows), arg.view(B, rows), (lg.view(B, rows, -1) if logits else None)

    def head_noalloc(self, h, B, L, row0, rows, logits=False, stream=None):
        """dllm_head_noalloc on the caller's residual h (float32 [B*L, d])."""
        dev = h.device
        conf = torch.empty((B * rows,), dtype=torch.float32, device=dev)
        arg = torch.empty((B * rows,), dtype=torch.int32, device=dev)
        lg = torch.empty((B * rows, self.cfg.vocab), dtype=torch.float32, device=dev) if logits else None
        check(lib().dllm_head_noalloc(self.h, _ptr(h), B, L, row0, rows, _ptr(conf), _ptr(arg), _ptr(lg),
                                      _stream(stream)))
        return conf.view(B, rows), arg.view(B, rows), (lg.view(B, rows, -1) if logits else None)

    def forward(self, x, row0, rows, ws=None, logits=False, stream=None):
        B, L = x.shape
        ws = ws if ws is not None else self.workspace(B, L, rows, x.device)
        dev = x.device
        conf = torch.empty((B * rows,), dtype=torch.float32, device=dev)
        arg = torch.empty((B * rows,), dtype=torch.int32, device=dev)
        lg = torch.empty((B * rows, self.cfg.vocab), dtype=torch.float32, device=dev) if logits else None
        check(lib().dllm_forward(self.h, _ptr(x), B, L, row0, rows, _ptr(conf), _ptr(arg), _ptr(lg), _ptr(ws),
                                 ws.numel(), _stream(stream)))
        return conf.view(B, rows), arg.view(B, rows), (lg.view(B, rows, -1) if logits else None)

    # decoding ---------------------------------------------------------------
    def state_init(self, prompt, G, st: DecodeState, stream=None):
        state_init(self.mask_id, prompt, G, st, stream)

    def step(self, ctl: Controller, st: DecodeState, block, t, ws, record=False, wait=True, stream=None):
        p = ctl.to_c()
        c = st.c()
        B, bl = st.B, ctl.block_len
        conf = torch.empty((B, bl), dtype=torch.float32, device=st.x.device) if record else None
        arg = torch.empty((B, bl), dtype=torch.int32, device=st.x.device) if record else None
        flag = torch.zeros((1,), dtype=torch.int32).pin_memory() if wait else None
        check(lib().dllm_step(self.h, ctypes.byref(p), ctypes.byref(c), B, st.P, st.G, block, t, _ptr(conf),
                              _ptr(arg), _ptr(flag), _ptr(ws), ws.numel(), _stream(stream)))
        return (int(flag.item()) if wait else None), conf, arg

    def generate(self, ctl: Controller, prompt, G, ws=None, st=None, trace=False, stream=None):
        B, P = prompt.shape
        bl, T = ctl.block_len, ctl.T
        nb = G // bl
        st = st or DecodeState(B, P, G, prompt.device)
        ws = ws if ws is not None else self.workspace(B, P + G, bl, prompt.device)
        p = ctl.to_c()
        c = st.c()
        fwd = (ctypes.c_int32 * nb)()
        tot = ctypes.c_int32()
        ct = at = None
        if trace:
            ct = torch.full((nb, T, B, bl), float("nan"), dtype=torch.float32, device=prompt.device)
            at = torch.full((nb, T, B, bl), -1, dtype=torch.int32, device=prompt.device)
        check(lib().dllm_generate(self.h, ctypes.byref(p), _ptr(prompt), B, P, G, ctypes.byref(c), fwd,
                                  ctypes.byref(tot), _ptr(ct), _ptr(at), _ptr(ws), ws.numel(), _stream(stream)))
        return GenResult(st, list(fwd), tot.value, ct, at)

    # cross-step key/value reuse ---------------------------------------------
    def kv_cache(self, B, L, device="cuda"):
        """A caller-owned, 256-byte aligned cache buffer for B sequences of L positions."""
        n = ctypes.c_size_t()
        check(lib().dllm_kv_cache_size(self.h, B, L, ctypes.byref(n)))
        return device_buffer(n.value, device)

    def forward_kv(self, x, row0, rows, kv, refresh, ws=None, logits=False, stream=None):
        """dllm_forward_kv: the refresh forward (refresh=True) or the cached forward of rows [row0, row0 + rows)."""
        B, L = x.shape
        ws = ws if ws is not None else self.workspace(B, L, rows, x.device)
        dev = x.device
        conf = torch.empty((B * rows,), dtype=torch.float32, device=dev)
        arg = torch.empty((B * rows,), dtype=torch.int32, device=dev)
        lg = torch.empty((B * rows, self.cfg.vocab), dtype=torch.float32, device=dev) if logits else None
        check(lib().dllm_forward_kv(self.h, _ptr(x), B, L, row0, rows, int(bool(refresh)), _ptr(conf), _ptr(arg),
                                    _ptr(lg), _ptr(kv), kv.numel(), _ptr(ws), ws.numel(), _stream(stream)))
        return conf.view(B, rows), arg.view(B, rows), (lg.view(B, rows, -1) if logits else None)

    def embed_rows(self, x, row0, rows, ws, stream=None):
        B, L = x.shape
        check(lib().dllm_embed_rows(self.h, _ptr(x), B, L, row0, rows, _ptr(ws), ws.numel(), _stream(stream)))

    def layer_kv(self, layer, part, B, L, row0, rows, kv, ws, stream=None):
        check(lib().dllm_layer_kv(self.h, layer, part, B, L, row0, rows, _ptr(kv), kv.numel(), _ptr(ws), ws.numel(),
                                  _stream(stream)))

    def step_kv(self, ctl: Controller, st: DecodeState, block, t, refresh, kv, ws, record=False, wait=True,
                stream=None):
        p = ctl.to_c()
        c = st.c()
        B, bl = st.B, ctl.block_len
        conf = torch.empty((B, bl), dtype=torch.float32, device=st.x.device) if record else None
        arg = torch.empty((B, bl), dtype=torch.int32, device=st.x.device) if record else None
        flag = torch.zeros((1,), dtype=torch.int32).pin_memory() if wait else None
        check(lib().dllm_step_kv(self.h, ctypes.byref(p), int(bool(refresh)), ctypes.byref(c), B, st.P, st.G, block,
                                 t, _ptr(conf), _ptr(arg), _ptr(flag), _ptr(kv), kv.numel(), _ptr(ws), ws.numel(),
                                 _stream(stream)))
        return (int(flag.item()) if wait else None), conf, arg

    def generate_kv(self, ctl: Controller, prompt, G, refresh_every, ws=None, st=None, kv=None, trace=False,
                    stream=None):
        """dllm_generate_kv: the decode with the cache refreshed at steps t % refresh_every == 0."""
        B, P = prompt.shape
        bl, T = ctl.block_len, ctl.T
        nb = G // bl
        st = st or DecodeState(B, P, G, prompt.device)
        ws = ws if ws is not None else self.workspace(B, P + G, bl, prompt.device)
        kv = kv if kv is not None else self.kv_cache(B, P + G, prompt.device)
        p = ctl.to_c()
        c = st.c()
        fwd = (ctypes.c_int32 * nb)()
        tot = ctypes.c_int32()
        ct = at = None
        if trace:
            ct = torch.full((nb, T, B, bl), float("nan"), dtype=torch.float32, device=prompt.device)
            at = torch.full((nb, T, B, bl), -1, dtype=torch.int32, device=prompt.device)
        check(lib().dllm_generate_kv(self.h, ctypes.byref(p), refresh_every, _ptr(prompt), B, P, G, ctypes.byref(c),
                                     fwd, ctypes.byref(tot), _ptr(ct), _ptr(at), _ptr(kv), kv.numel(), _ptr(ws),
                                     ws.numel(), _stream(stream)))
        return GenResult(st, list(fwd), tot.value, ct, at)

    # profiling --------------------------------------------------------------
    def prof_enable(self, kinds=()):
        """Record per-launch HIP-event timings for the given kernel kinds (PROF_*)."""
        mask = 0
        for k in kinds:
            mask |= 1 << k
        check(lib().dllm_prof_enable(self.h, mask))

    def prof_every(self, every):
        """dllm_prof_every: record one launch in `every` of each enabled kind."""
        check(lib().dllm_prof_every(self.h, every))

    def prof_read(self, kind):
        ms = ctypes.c_double()
        n = ctypes.c_int64()
        check(lib().dllm_prof_read(self.h, kind, ctypes.byref(ms), ctypes.byref(n)))
        return ms.value, n.value


@dataclass
class GenResult:
    state: DecodeState
    forwards: list
    total_forwards: int
    conf_trace: torch.Tensor | None
    argmax_trace: torch.Tensor | None


def state_init(mask_id, prompt, G, st: DecodeState, stream=None):
    """dllm_state_init: x = [prompt | mask], commit_step = -1, everything else 0."""
    B, P = prompt.shape
    c = st.c()
    check(lib().dllm_state_init(mask_id, _ptr(prompt), B, P, G, ctypes.byref(c), _stream(stream)))


def commit(ctl: Controller, st: DecodeState, conf, argmax, block, t, mask_id, all_done=None, stream=None):
    """The controller alone (dllm_commit) on device conf [B, bl] / argmax [B, bl]."""
    p = ctl.to_c()
    c = st.c()
    check(lib().dllm_commit(ctypes.byref(p), ctypes.byref(c), _ptr(conf), _ptr(argmax), st.B, st.P, st.G, block, t,
                            mask_id, _ptr(all_done), _stream(stream)))


# ---------------------------------------------------------------- stand-alone operators
_DTYPES = {torch.float32: DLLM_F32, torch.bfloat16: DLLM_BF16}
_SCALINGS = {"none": ROPE_PLAIN, "linear": ROPE_LINEAR, "parts": ROPE_PARTS}


def _refuse(ok, code, msg):
    if not ok:
        raise DllmError(code, msg)


def _in32(*numbers):
    """Numbers that the C side takes as int32 (ctypes would cut them to 32 bits)."""
    if max(numbers) > 0x7fffffff or min(numbers) < -0x80000000:
        _refuse(False, -2, f"{numbers}: beyond 32 bits")


def _dtype(t, name):
    _refuse(t.dtype in _DTYPES, -1, f"{name} must be float32 or bfloat16")
    return _DTYPES[t.dtype]


def _raw_stream(index):
    """The current stream of device `index` as an address, without the cost of a Stream object where torch has a way."""
    get = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return get(index) if get else torch.cuda.current_stream(index).cuda_stream


def _elsewhere(device, stream):
    """None where a call can go to the current stream of the current device; else the scope it runs in: the operands'
    device made current, and what the call allocates owned by the stream that uses it."""
    _refuse(device.type == "cuda", -1, "tensors must be on the GPU")
    if stream is None and torch.cuda.current_device() == device.index:
        return None
    stream = torch.cuda.current_stream(device) if stream is None else stream
    _refuse(stream.device == device, -1, "the stream is another device's than the tensors")
    return torch.cuda.stream(stream)


def _column(t, n, dtype, device, name):
    """The address of a device array of n elements (None: 0)."""
    if t is None:
        return None
    if t.dtype != dtype or t.device != device:
        _refuse(False, -1, f"{name} must be {dtype} on {device}")
    if t.numel() != n or not t.is_contiguous():
        _refuse(False, -2, f"{name} must be {n} contiguous elements")
    return t.data_ptr()


def _rows(t, shape, dtype, device, name):
    """The view of a [B, L, H, hd] or [L, H, hd] tensor whose last dimension is contiguous."""
    st = t.stride()
    if t.shape != shape or st[-1] != 1 or t.dtype is not dtype or t.device != device:
        _refuse(t.shape == shape, -2, f"{name} must have the shape {tuple(shape)}, not {tuple(t.shape)}")
        _refuse(st[-1] == 1 or t.numel() == 0, -2, f"{name}: elements of a head must be contiguous")
        _refuse(t.dtype is dtype and t.device == device, -1, f"{name} must be {dtype} on {device}")
    # a dimension of one element is never stepped over: its stride says nothing
    return View(t.data_ptr(), st[0] if len(shape) == 4 and shape[0] > 1 else 0, st[-3] if shape[-3] > 1 else shape[-1],
                st[-2] if shape[-2] > 1 else 0)


def _new_rows(like, shape):
    """A new tensor of a [B, L, H, hd] shape, of like's type, and its view."""
    t = torch.empty_like(like, memory_format=torch.contiguous_format)
    n = shape[2] * shape[3]
    return t, View(t.data_ptr(), shape[1] * n, n, shape[3])


def _workspace(nbytes, device):
    """A 256-byte aligned buffer (torch's own allocations are)."""
    buf = torch.empty(nbytes, dtype=torch.uint8, device=device)
    return buf if buf.data_ptr() % 256 == 0 else device_buffer(nbytes, device)


def _given(ws, device):
    """The caller's workspace, which lies on the operands' device."""
    if ws.device != device or not ws.is_contiguous():
        _refuse(False, -1, f"ws must be contiguous on {device}")
    return ws


@dataclass(frozen=True)
class Rotary:
    """Constants of a rotary embedding (dllm_rotary_cfg); scaling: none, linear or parts."""
    head_dim: int
    rot_dim: int = 0            # 0: the whole head
    interleaved: bool = False
    base: float = 10000.0
    scaling: str = "none"
    factor: float = 1.0
    orig_len: float = 0.0
    low: float = 1.0
    high: float = 32.0
    gain: float = 1.0

    def to_c(self) -> RotaryCfg:
        if self.scaling not in _SCALINGS:
            raise KeyError(f"unknown rotary scaling {self.scaling!r}; known: {sorted(_SCALINGS)}")
        return RotaryCfg(self.head_dim, self.rot_dim or self.head_dim, int(self.interleaved), _SCALINGS[self.scaling],
                         self.base, self.factor, self.orig_len, self.low, self.high, self.gain)


def rotary(cfg: Rotary, q, k=None, pos=None, pos0=0, q_out=None, k_out=None, inverse=False, stream=None):
    """dllm_rotary on q [B, L, Hq, hd] and (optionally) k [B, L, Hkv, hd], any strides with contiguous heads.
    pos: int32 [B, L], or None for pos0 + l.  Outputs are new tensors unless given (q_out=q: in place).
    Returns (q_out, k_out)."""
    _refuse(q.dim() == 4 and (k is None or k.dim() == 4), -2, "q and k must be [B, L, heads, head_dim]")
    scope = _elsewhere(q.device, stream)
    if scope is not None:
        with scope:
            return rotary(cfg, q, k, pos, pos0, q_out, k_out, inverse)
    dt, dtype, dev = _dtype(q, "q"), q.dtype, q.device
    shape = B, L, n_q, hd = tuple(q.shape)
    if hd != cfg.head_dim:
        _refuse(False, -2, f"q has heads of {hd} elements, cfg of {cfg.head_dim}")
    _in32(pos0)
    p = _column(pos, B * L, torch.int32, dev, "pos")
    vq, vk, vko, n_k = _rows(q, shape, dtype, dev, "q"), None, None, 0
    if q_out is None:
        q_out, vqo = _new_rows(q, shape)
    else:
        vqo = _rows(q_out, shape, dtype, dev, "q_out")
    if k is not None:
        n_k = k.shape[2]
        shape = (B, L, n_k, hd)
        vk = _rows(k, shape, dtype, dev, "k")
        if k_out is None:
            k_out, vko = _new_rows(k, shape)
        else:
            vko = _rows(k_out, shape, dtype, dev, "k_out")
    check(lib().dllm_rotary(cfg.to_c(), dt, B, L, p, pos0, vq, vqo, n_q, vk, vko, n_k, int(bool(inverse)),
                            _raw_stream(dev.index)))
    return q_out, (k_out if k is not None else None)


@dataclass
class Docs:
    """The documents of an attention call: int32 device arrays [docs] (or None: see dllm_attn_args) and the
    longest lengths among them.  Documents of a dense batch need no arrays but their lengths."""
    q_start: torch.Tensor | None = None
    q_len: torch.Tensor | None = None
    kv_start: torch.Tensor | None = None
    kv_len: torch.Tensor | None = None
    max_q: int | None = None       # None: the slab's tokens
    max_kv: int | None = None
    q_pos: torch.Tensor | None = None
    prefix: torch.Tensor | None = None
    count: int | None = None       # documents; None: the arrays' length, or the slabs

    @classmethod
    def packed(cls, q_lens, kv_lens=None, q_pos=None, prefix=None, device="cuda"):
        """Documents that follow each other without gaps, from host lists."""
        q_lens = list(q_lens)
        kv_lens = q_lens if kv_lens is None else list(kv_lens)
        ints = lambda v: None if v is None else torch.tensor(list(v), dtype=torch.int32, device=device)  # noqa: E731
        starts = lambda v: list(itertools.accumulate([0, *v[:-1]])) if v else []  # noqa: E731
        return cls(ints(starts(q_lens)), ints(q_lens), ints(starts(kv_lens)), ints(kv_lens), max(q_lens, default=0),
                   max(kv_lens, default=0), ints(q_pos), ints(prefix))


_DOC_ARRAYS = ("q_start", "q_len", "kv_start", "kv_len", "q_pos", "prefix")


def attention(q, k, v, docs: Docs | None = None, block=0, scale=None, cap=0.0, slopes=None, out=None, ws=None,
              stream=None):
    """dllm_attention.  q [T, Hq, hd] with k, v [S, Hkv, hd]: packed documents in one slab; q [B, T, Hq, hd] with k, v
    [B, S, Hkv, hd]: a slab per document.  scale None: 1 / sqrt(hd).  out: written and returned (new, zeroed, if
    None); ws: a device_buffer of attention_workspace_size bytes (allocated here if None)."""
    _refuse(q.dim() in (3, 4) and k.dim() == q.dim() and v.dim() == q.dim(), -2,
            "q, k and v must be [tokens, heads, head_dim] or [docs, tokens, heads, head_dim]")
    dev = q.device
    scope = _elsewhere(dev, stream)
    if scope is not None:
        with scope:
            return attention(q, k, v, docs, block, scale, cap, slopes, out, ws)
    dt = _dtype(q, "q")
    out = torch.zeros(q.shape, dtype=q.dtype, device=dev) if out is None else out
    a = _attn_args(dt, q, k, v, out, docs or Docs(), block, scale, cap, slopes)
    if ws is None:
        n = _sz()
        check(lib().dllm_attention_workspace_size(a, n))
        ws = _workspace(n.value, dev) if n.value else None
    else:
        _given(ws, dev)
    check(lib().dllm_attention(a, _ptr(ws), 0 if ws is None else ws.nbytes, _raw_stream(dev.index)))
    return out


def attention_workspace_size(q, k, v, docs: Docs | None = None):
    """Bytes of workspace that attention() needs for operands and documents of these sizes."""
    n = _sz()
    check(lib().dllm_attention_workspace_size(
        _attn_args(_dtype(q, "q"), q, k, v, q, docs or Docs(), 0, None, 0.0, None), n))
    return n.value


def _attn_args(dt, q, k, v, out, docs, block, scale, cap, slopes):
    dev, dtype = q.device, q.dtype
    shape, kv = tuple(q.shape), tuple(k.shape)
    one = len(shape) == 3
    T, Hq, hd = shape[-3:]
    S, Hkv = kv[-3:-1]
    kv = (S, Hkv, hd) if one else (shape[0], S, Hkv, hd)
    views = [_rows(q, shape, dtype, dev, "q"), _rows(k, kv, dtype, dev, "k"), _rows(v, kv, dtype, dev, "v"),
             _rows(out, shape, dtype, dev, "out")]
    arrays = (docs.q_start, docs.q_len, docs.kv_start, docs.kv_len, docs.q_pos, docs.prefix)
    n = docs.count
    if n is None:
        n = next((t.numel() for t in arrays if t is not None), 1) if one else shape[0]
    _refuse(one or n == shape[0], -2, "a dense batch has one document per slab")
    max_q, max_kv = T if docs.max_q is None else docs.max_q, S if docs.max_kv is None else docs.max_kv
    _in32(n, T, S, max_q, max_kv, block)
    ptrs = [_column(t, n, torch.int32, dev, name) for t, name in zip(arrays, _DOC_ARRAYS)]
    return AttnArgs(dt, Hq, Hkv, hd, *views, n, T, S, max_q, max_kv, *ptrs,
                    _column(slopes, Hq, torch.float32, dev, "slopes"), 1.0 / math.sqrt(hd) if scale is None else scale, cap,
                    block)


def sample(logits, u, temperature=None, top_k=None, top_p=None, min_p=None, mask_id=-1, ws=None, stream=None):
    """dllm_sample on logits [rows, V] (rows of any stride) with uniform random numbers u [rows].  Controls are device
    arrays [rows] (top_k int32, the others float32).  Returns (token int32, conf, prob float32), each [rows]."""
    _refuse(logits.dim() == 2, -2, "logits must be [rows, vocab]")
    dev = logits.device
    scope = _elsewhere(dev, stream)
    if scope is not None:
        with scope:
            return sample(logits, u, temperature, top_k, top_p, min_p, mask_id, ws)
    dt = _dtype(logits, "logits")
    R, V = logits.shape
    st = logits.stride()
    _refuse(st[1] == 1 or V == 1, -2, "logits: a row must be contiguous")
    _in32(R, V, mask_id)
    cols = [_column(u, R, torch.float32, dev, "u"), _column(temperature, R, torch.float32, dev, "temperature"),
            _column(top_k, R, torch.int32, dev, "top_k"), _column(top_p, R, torch.float32, dev, "top_p"),
            _column(min_p, R, torch.float32, dev, "min_p")]
    token = torch.empty((R,), dtype=torch.int32, device=dev)
    conf, prob = torch.empty((2, R), dtype=torch.float32, device=dev).unbind(0)
    a = SampleArgs(logits.data_ptr(), st[0], dt, R, V, mask_id, *cols, token.data_ptr(), conf.data_ptr(),
                   prob.data_ptr())
    if ws is None:
        n = sample_workspace_size(R, V)
        ws = _workspace(n, dev) if n else None
    else:
        _given(ws, dev)
    check(lib().dllm_sample(a, _ptr(ws), 0 if ws is None else ws.nbytes, _raw_stream(dev.index)))
    return token, conf, prob


def sample_workspace_size(rows, vocab):
    _in32(rows, vocab)
    n = _sz()
    check(lib().dllm_sample_workspace_size(rows, vocab, n))
    return n.value
