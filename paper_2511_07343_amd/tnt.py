"""ctypes binding of ``libtnt.so`` (see ``include/tnt.h``).

Argument marshalling only: every step of the layer runs in the library's HIP
kernels.  Torch tensors provide device memory and the current HIP stream.
The functions named like the C entry points take tensors for the pointer
arguments; ``forward`` / ``backward`` also allocate outputs and workspaces.
"""
from __future__ import annotations

import ctypes
import os
from typing import Dict, Optional

import torch

from .inputs import BF16, F32, LayerConfig

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libtnt.so")
_lib = None

TNT_MAX_LOCAL = 4
TNT_WS_FWD, TNT_WS_BWD, TNT_WS_BWD_RECOMPUTE, TNT_WS_FWD_MIN = 0, 1, 2, 3
STATUS = {0: "TNT_OK", 1: "TNT_ERR_NULL", 2: "TNT_ERR_SHAPE", 3: "TNT_ERR_UNSUPPORTED",
          4: "TNT_ERR_WORKSPACE", 5: "TNT_ERR_ALIGN", 6: "TNT_ERR_HIP", 7: "TNT_ERR_ARG"}
EXPORTED = ["tnt_mem_workspace_size", "tnt_mem_saved_size", "tnt_mem_fwd", "tnt_mem_bwd",
            "tnt_strerror", "tnt_abi_version", "tnt_timing_enable", "tnt_timing_read",
            "tnt_mem_state_size", "tnt_mem_state_init", "tnt_mem_step", "tnt_mem_state_from_fwd",
            "tnt_dbg_chunk_grads", "tnt_set_kernel_family", "tnt_mem_fwd_noalloc",
            "tnt_delta_workspace_size", "tnt_delta_saved_size", "tnt_delta_fwd", "tnt_delta_bwd",
            "tnt_delta_step", "tnt_orth_workspace_size", "tnt_orth_update"]
NOALLOC_WORKSPACE_BYTES = 128 << 20
FAMILY_DEFAULT, FAMILY_GENERIC, FAMILY_SINGLE_WALK = 0, 1, 2


class TntError(RuntimeError):
    def __init__(self, status: int, where: str):
        super().__init__(f"{where}: {STATUS.get(status, status)} ({strerror(status)})")
        self.status = status


class tnt_config(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("H", ctypes.c_int32), ("L", ctypes.c_int32),
                ("d", ctypes.c_int32), ("hid", ctypes.c_int32),
                ("has_global", ctypes.c_int32), ("C_G", ctypes.c_int32),
                ("n_local", ctypes.c_int32),
                ("C_L", ctypes.c_int32 * TNT_MAX_LOCAL), ("S_L", ctypes.c_int32 * TNT_MAX_LOCAL),
                ("act", ctypes.c_int32), ("qk_proj", ctypes.c_int32),
                ("qk_scope", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("global_intra", ctypes.c_int32)]


class tnt_delta_config(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("B", "H", "Hk", "L", "d_k", "d_v", "n_seq", "dtype")] + [
        ("scale", ctypes.c_float)]


class tnt_orth_config(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int32) for n in ("n", "rows", "cols", "steps", "dtype")]
                + [("eps", ctypes.c_float), ("scale", ctypes.c_float)]
                + [(n, ctypes.c_int64) for n in ("g_batch", "g_row", "out_batch", "out_row")])


# tnt_delta_strides: 12 tensors x (row, head, token), in the header's order; a forward or a
# step reads the first six only
tnt_delta_strides = ctypes.c_int64 * 36
_delta_strides6 = ctypes.c_int64 * 18


def lib(path: Optional[str] = None) -> ctypes.CDLL:
    """Load the library; raises if it has not been built (no fallback)."""
    global _lib
    if _lib is not None and path is None:
        return _lib
    p = path or _LIB_PATH
    if not os.path.exists(p):
        raise RuntimeError(f"{p} is missing: build it with `python -m paper_2511_07343_amd.build`")
    L = ctypes.CDLL(p)
    vp, sz, i32 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int32
    cp = ctypes.POINTER(tnt_config)
    L.tnt_mem_workspace_size.argtypes = [cp, ctypes.c_int]
    L.tnt_mem_workspace_size.restype = sz
    L.tnt_mem_saved_size.argtypes = [cp]
    L.tnt_mem_saved_size.restype = sz
    L.tnt_mem_fwd.argtypes = [cp] + [vp] * 11 + [sz, vp, sz, vp]
    L.tnt_mem_fwd.restype = ctypes.c_int
    L.tnt_mem_bwd.argtypes = [cp] + [vp] * 10 + [sz] + [vp] * 9 + [sz, vp]
    L.tnt_mem_bwd.restype = ctypes.c_int
    L.tnt_mem_state_size.argtypes = [cp]
    L.tnt_mem_state_size.restype = sz
    L.tnt_mem_state_init.argtypes = [cp, vp, vp, vp, vp]
    L.tnt_mem_state_init.restype = ctypes.c_int
    L.tnt_mem_step.argtypes = [cp, ctypes.c_int64, i32] + [vp] * 11
    L.tnt_dbg_chunk_grads.argtypes = [cp, i32, i32, i32, i32] + [vp] * 8
    L.tnt_dbg_chunk_grads.restype = ctypes.c_int
    L.tnt_mem_state_from_fwd.argtypes = [cp] + [vp] * 5
    L.tnt_mem_state_from_fwd.restype = ctypes.c_int
    L.tnt_mem_step.restype = ctypes.c_int
    L.tnt_strerror.argtypes = [ctypes.c_int]
    L.tnt_strerror.restype = ctypes.c_char_p
    L.tnt_abi_version.argtypes = []
    L.tnt_abi_version.restype = i32
    L.tnt_mem_fwd_noalloc.argtypes = [cp] + [vp] * 11
    L.tnt_mem_fwd_noalloc.restype = ctypes.c_int
    L.tnt_set_kernel_family.argtypes = [i32]
    L.tnt_set_kernel_family.restype = i32
    L.tnt_timing_enable.argtypes = [i32]
    L.tnt_timing_enable.restype = i32
    L.tnt_timing_read.argtypes = [i32, ctypes.c_char_p, ctypes.POINTER(ctypes.c_double),
                                  ctypes.POINTER(i32)]
    L.tnt_timing_read.restype = i32
    dp, sp = ctypes.POINTER(tnt_delta_config), vp  # strides: a ctypes array
    L.tnt_delta_workspace_size.argtypes = [dp, ctypes.c_int]
    L.tnt_delta_workspace_size.restype = sz
    L.tnt_delta_saved_size.argtypes = [dp]
    L.tnt_delta_saved_size.restype = sz
    L.tnt_delta_fwd.argtypes = [dp, sp] + [vp] * 10 + [sz, vp, sz, vp]
    L.tnt_delta_fwd.restype = ctypes.c_int
    L.tnt_delta_bwd.argtypes = [dp, sp] + [vp] * 10 + [sz] + [vp] * 7 + [sz, vp]
    L.tnt_delta_bwd.restype = ctypes.c_int
    L.tnt_delta_step.argtypes = [dp, sp] + [vp] * 6 + [i32, vp, vp, vp]
    L.tnt_delta_step.restype = ctypes.c_int
    op = ctypes.POINTER(tnt_orth_config)
    L.tnt_orth_workspace_size.argtypes = [op]
    L.tnt_orth_workspace_size.restype = sz
    L.tnt_orth_update.argtypes = [op, ctypes.POINTER(ctypes.c_float), vp, vp, vp, sz, vp]
    L.tnt_orth_update.restype = ctypes.c_int
    if path is None:
        _lib = L
    return L


def to_c(cfg: LayerConfig) -> tnt_config:
    c = tnt_config()
    c.B, c.H, c.L, c.d, c.hid = cfg.B, cfg.H, cfg.L, cfg.d, cfg.hid
    c.has_global, c.C_G, c.n_local = cfg.has_global, cfg.C_G, len(cfg.locals_)
    for i, (cl, sl) in enumerate(cfg.locals_):
        c.C_L[i], c.S_L[i] = cl, sl
    c.act, c.qk_proj, c.qk_scope, c.dtype = cfg.act, cfg.qk_proj, cfg.qk_scope, cfg.dtype
    c.global_intra = getattr(cfg, "global_intra", 0)
    return c


def strerror(status: int) -> str:
    return lib().tnt_strerror(status).decode()


def _p(t) -> Optional[int]:
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


def _stream(stream) -> Optional[int]:
    if stream is None:
        stream = torch.cuda.current_stream()
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else stream


def tnt_mem_workspace_size(cfg: LayerConfig, kind: int) -> int:
    return lib().tnt_mem_workspace_size(ctypes.byref(to_c(cfg)), kind)


def tnt_mem_saved_size(cfg: LayerConfig) -> int:
    return lib().tnt_mem_saved_size(ctypes.byref(to_c(cfg)))


def _nbytes(t, given):
    if given is not None:
        return given
    if t is None or isinstance(t, int):
        return 0
    return t.numel() * t.element_size()


def tnt_mem_fwd(cfg, q, k, v, lr, mom, decay, W1_init, W2_init, o, final_state, saved,
                workspace, ws_bytes=None, stream=None, saved_bytes=None) -> int:
    ws_bytes = _nbytes(workspace, ws_bytes)
    c = to_c(cfg)
    return lib().tnt_mem_fwd(ctypes.byref(c), _p(q), _p(k), _p(v), _p(lr), _p(mom), _p(decay),
                             _p(W1_init), _p(W2_init), _p(o), _p(final_state), _p(saved),
                             _nbytes(saved, saved_bytes), _p(workspace), ws_bytes,
                             _stream(stream))


def tnt_mem_bwd(cfg, q, k, v, lr, mom, decay, W1_init, W2_init, dO, saved, dq, dk, dv, dlr,
                dmom, ddecay, dW1_init, dW2_init, workspace, ws_bytes=None, stream=None,
                saved_bytes=None) -> int:
    ws_bytes = _nbytes(workspace, ws_bytes)
    c = to_c(cfg)
    return lib().tnt_mem_bwd(ctypes.byref(c), _p(q), _p(k), _p(v), _p(lr), _p(mom), _p(decay),
                             _p(W1_init), _p(W2_init), _p(dO), _p(saved),
                             _nbytes(saved, saved_bytes), _p(dq), _p(dk), _p(dv), _p(dlr),
                             _p(dmom), _p(ddecay), _p(dW1_init), _p(dW2_init), _p(workspace),
                             ws_bytes, _stream(stream))


def tnt_mem_fwd_noalloc(cfg, q, k, v, lr, mom, decay, W1_init, W2_init, o, final_state,
                        stream=None) -> int:
    c = to_c(cfg)
    return lib().tnt_mem_fwd_noalloc(ctypes.byref(c), _p(q), _p(k), _p(v), _p(lr), _p(mom),
                                     _p(decay), _p(W1_init), _p(W2_init), _p(o),
                                     _p(final_state), _stream(stream))


def tnt_set_kernel_family(family: int) -> int:
    return lib().tnt_set_kernel_family(family)


class kernel_family:
    """Context manager: run the enclosed calls under another kernel family
    (tnt_set_kernel_family), restoring the previous one on exit."""

    def __init__(self, family: int):
        self.family = family
        self.prev = None

    def __enter__(self):
        self.prev = tnt_set_kernel_family(self.family)
        if self.prev < 0:
            raise ValueError(f"unknown kernel family {self.family}")
        return self

    def __exit__(self, *exc):
        tnt_set_kernel_family(self.prev)
        return False


def tnt_mem_state_size(cfg: LayerConfig) -> int:
    return lib().tnt_mem_state_size(ctypes.byref(to_c(cfg)))


def tnt_mem_state_init(cfg, W1_init, W2_init, state, stream=None) -> int:
    c = to_c(cfg)
    return lib().tnt_mem_state_init(ctypes.byref(c), _p(W1_init), _p(W2_init), _p(state),
                                    _stream(stream))


def tnt_dbg_chunk_grads(cfg, b, h, t0, C, k, v, W1, W2, Zk, R, D1, stream=None) -> int:
    c = to_c(cfg)
    return lib().tnt_dbg_chunk_grads(ctypes.byref(c), b, h, t0, C, _p(k), _p(v), _p(W1), _p(W2),
                                     _p(Zk), _p(R), _p(D1), _stream(stream))


def tnt_mem_state_from_fwd(cfg, final_state, W1_init, W2_init, state, stream=None) -> int:
    c = to_c(cfg)
    return lib().tnt_mem_state_from_fwd(ctypes.byref(c), _p(final_state), _p(W1_init),
                                        _p(W2_init), _p(state), _stream(stream))


def tnt_mem_step(cfg, pos, T, q, k, v, lr, mom, decay, W1_init, W2_init, state, o,
                 stream=None) -> int:
    c = to_c(cfg)
    return lib().tnt_mem_step(ctypes.byref(c), pos, T, _p(q), _p(k), _p(v), _p(lr), _p(mom),
                              _p(decay), _p(W1_init), _p(W2_init), _p(state), _p(o),
                              _stream(stream))


def tnt_timing_enable(on: bool) -> int:
    return lib().tnt_timing_enable(1 if on else 0)


def tnt_timing_read(max_entries: int = 64) -> Dict[str, tuple]:
    """{kernel name: (total ms, launches)} of the launches recorded while
    timing was enabled; clears the record."""
    names = ctypes.create_string_buffer(32 * max_entries)
    ms = (ctypes.c_double * max_entries)()
    cnt = (ctypes.c_int32 * max_entries)()
    n = lib().tnt_timing_read(max_entries, names, ms, cnt)
    if n < 0:
        raise RuntimeError("tnt_timing_read: HIP error")
    out = {}
    for i in range(n):
        nm = names.raw[32 * i: 32 * i + 32].split(b"\0", 1)[0].decode()
        out[nm] = (ms[i], cnt[i])
    return out


# --------------------------------------------------------------------------
# allocating wrappers
# --------------------------------------------------------------------------
def io_dtype(cfg: LayerConfig):
    return torch.bfloat16 if cfg.dtype == BF16 else torch.float32


def device_inputs(inp, cfg: LayerConfig, device="cuda") -> Dict[str, torch.Tensor]:
    """Copy host arrays (``inputs.LayerInputs``) to the device in the ABI's dtypes."""
    io = io_dtype(cfg)
    t = lambda a, dt: torch.from_numpy(a).to(device=device, dtype=dt).contiguous()
    return dict(q=t(inp.q, io), k=t(inp.k, io), v=t(inp.v, io), dO=t(inp.dO, io),
                lr=t(inp.lr, torch.float32), mom=t(inp.mom, torch.float32),
                decay=t(inp.decay, torch.float32), W1=t(inp.W1, torch.float32),
                W2=t(inp.W2, torch.float32))


def _bytes(n: int, device) -> torch.Tensor:
    return torch.empty(max(n, 16), dtype=torch.uint8, device=device)


def forward(cfg: LayerConfig, x: Dict[str, torch.Tensor], save: bool = True,
            final_state: bool = False, workspace: Optional[torch.Tensor] = None,
            stream=None):
    """Run tnt_mem_fwd; returns (o, saved or None, final_state or None)."""
    dev = x["q"].device
    if _elsewhere(stream, dev):
        return _on_stream(stream, dev, (*x.values(), workspace),
                          lambda: forward(cfg, x, save, final_state, workspace))
    o = torch.empty_like(x["q"])
    saved = _bytes(tnt_mem_saved_size(cfg), dev) if save else None
    fin = (torch.empty(cfg.B, cfg.H, 4, cfg.hid * cfg.d, dtype=torch.float32, device=dev)
           if final_state else None)
    if workspace is None:
        workspace = _bytes(tnt_mem_workspace_size(cfg, TNT_WS_FWD), dev)
    st = tnt_mem_fwd(cfg, x["q"], x["k"], x["v"], x["lr"], x["mom"], x["decay"], x["W1"],
                     x["W2"], o, fin, saved, workspace)
    if st != 0:
        raise TntError(st, "tnt_mem_fwd")
    return o, saved, fin


def backward(cfg: LayerConfig, x: Dict[str, torch.Tensor], dO: torch.Tensor,
             saved: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
             stream=None) -> Dict[str, torch.Tensor]:
    """Run tnt_mem_bwd; returns the gradients of sum(dO * o)."""
    dev = x["q"].device
    if _elsewhere(stream, dev):
        return _on_stream(stream, dev, (*x.values(), dO, saved, workspace),
                          lambda: backward(cfg, x, dO, saved, workspace))
    g = dict(dq=torch.empty_like(x["q"]), dk=torch.empty_like(x["k"]),
             dv=torch.empty_like(x["v"]), dlr=torch.empty_like(x["lr"]),
             dmom=torch.empty_like(x["mom"]), ddecay=torch.empty_like(x["decay"]),
             dW1=torch.empty_like(x["W1"]), dW2=torch.empty_like(x["W2"]))
    if workspace is None:
        kind = TNT_WS_BWD if saved is not None else TNT_WS_BWD_RECOMPUTE
        workspace = _bytes(tnt_mem_workspace_size(cfg, kind), dev)
    st = tnt_mem_bwd(cfg, x["q"], x["k"], x["v"], x["lr"], x["mom"], x["decay"], x["W1"],
                     x["W2"], dO, saved, g["dq"], g["dk"], g["dv"], g["dlr"], g["dmom"],
                     g["ddecay"], g["dW1"], g["dW2"], workspace)
    if st != 0:
        raise TntError(st, "tnt_mem_bwd")
    return g


def step_forward(cfg: LayerConfig, x: Dict[str, torch.Tensor], pieces, state=None, pos: int = 0,
                 stream=None):
    """Feed the sequence in ``x`` through tnt_mem_step in consecutive pieces of
    the given lengths (starting at token ``pos`` of ``x`` with ``state``, or
    from a fresh state); returns (o of the fed tokens [B,H,sum(pieces),d], state)."""
    dev = x["q"].device
    if _elsewhere(stream, dev):
        return _on_stream(stream, dev, (*x.values(), state),
                          lambda: step_forward(cfg, x, pieces, state, pos))
    if state is None:
        state = _bytes(tnt_mem_state_size(cfg), dev)
        st = tnt_mem_state_init(cfg, x["W1"], x["W2"], state)
        if st != 0:
            raise TntError(st, "tnt_mem_state_init")
    outs = []
    t0 = pos
    for T in pieces:
        sl = slice(t0, t0 + T)
        # fresh copies: a slice that is already contiguous would be an offset
        # view, not 16-byte aligned in general
        cp = lambda t: t.clone(memory_format=torch.contiguous_format)
        q, k, v = (cp(x[n][:, :, sl]) for n in ("q", "k", "v"))
        lr, mom, dec = (cp(x[n][..., sl]) for n in ("lr", "mom", "decay"))
        o = torch.empty_like(q)
        st = tnt_mem_step(cfg, t0, T, q, k, v, lr, mom, dec, x["W1"], x["W2"], state, o)
        if st != 0:
            raise TntError(st, "tnt_mem_step")
        outs.append(o)
        t0 += T
    return torch.cat(outs, 2), state


# --------------------------------------------------------------------------
# gated delta rule
# --------------------------------------------------------------------------
class DeltaConfig:
    """Shape of a gated delta rule call (``tnt_delta_config``): B rows of L tokens, H value heads
    over Hk key heads, head sizes dk and dv; ``n_seq`` > 0 packs that many sequences into one row.
    Immutable; the C structure and the buffer sizes are made once."""

    def __init__(self, *, B: int, H: int, L: int, dk: int, dv: int, Hk: int = 0, n_seq: int = 0,
                 dtype: int = BF16, scale: float = 1.0):
        self.B, self.H, self.Hk, self.L = B, H, Hk or H, L
        self.dk, self.dv, self.n_seq, self.dtype, self.scale = dk, dv, n_seq, dtype, scale
        self.c = tnt_delta_config(B, H, self.Hk, L, dk, dv, n_seq, dtype, scale)
        self.ref = ctypes.byref(self.c)
        self._sizes = {}
        # of every token input: name, shape, type, elements of a token (the gates have none)
        self.tokens = [(n, self.shape(n), self.io if n in "qkv" else torch.float32,
                        {"q": dk, "k": dk, "v": dv}.get(n, 0)) for n in ("q", "k", "v", "g", "lr")]

    @property
    def sequences(self) -> int:
        return self.n_seq or self.B

    @property
    def io(self):
        return torch.bfloat16 if self.dtype == BF16 else torch.float32

    def size(self, kind) -> int:
        """Bytes of a workspace (a ``TNT_WS_`` kind) or of the saved buffer ("saved")."""
        if kind not in self._sizes:
            self._sizes[kind] = (lib().tnt_delta_saved_size(self.ref) if kind == "saved"
                                 else lib().tnt_delta_workspace_size(self.ref, kind))
        return self._sizes[kind]

    def shape(self, name: str):
        if name in ("q", "k"):
            return (self.B, self.Hk, self.L, self.dk)
        return (self.B, self.H, self.L, self.dv) if name in ("v", "dO") else (self.B, self.H, self.L)


def tnt_delta_workspace_size(cfg: DeltaConfig, kind: int) -> int:
    return lib().tnt_delta_workspace_size(cfg.ref, kind)


def tnt_delta_saved_size(cfg: DeltaConfig) -> int:
    return lib().tnt_delta_saved_size(cfg.ref)


def tnt_delta_fwd(cfg, strides, q, k, v, g, lr, seq_start, S0, o, final_state, saved, workspace,
                  ws_bytes=None, stream=None, saved_bytes=None) -> int:
    return lib().tnt_delta_fwd(cfg.ref, strides, _p(q), _p(k), _p(v), _p(g), _p(lr),
                               _p(seq_start), _p(S0), _p(o), _p(final_state), _p(saved),
                               _nbytes(saved, saved_bytes), _p(workspace),
                               _nbytes(workspace, ws_bytes), _stream(stream))


def tnt_delta_bwd(cfg, strides, q, k, v, g, lr, seq_start, S0, dO, dfinal, saved, dq, dk, dv, dg,
                  dlr, dS0, workspace, ws_bytes=None, stream=None, saved_bytes=None) -> int:
    return lib().tnt_delta_bwd(cfg.ref, strides, _p(q), _p(k), _p(v), _p(g), _p(lr),
                               _p(seq_start), _p(S0), _p(dO), _p(dfinal), _p(saved),
                               _nbytes(saved, saved_bytes), _p(dq), _p(dk), _p(dv), _p(dg),
                               _p(dlr), _p(dS0), _p(workspace), _nbytes(workspace, ws_bytes),
                               _stream(stream))


def tnt_delta_step(cfg, strides, q, k, v, g, lr, state, n_slots, slots, o, stream=None) -> int:
    return lib().tnt_delta_step(cfg.ref, strides, _p(q), _p(k), _p(v), _p(g), _p(lr), _p(state),
                                n_slots, _p(slots), _p(o), _stream(stream))


def _check(t, name, shape, dtype, dev, dense=False):
    """Shape, type and place of an argument: the library sees only pointers and strides."""
    if t.shape != shape or t.dtype != dtype or t.device != dev:
        raise ValueError(f"{name}: expected {tuple(shape)} {dtype} on {dev}, got {tuple(t.shape)} "
                         f"{t.dtype} on {t.device}")
    if dense and not t.is_contiguous():
        raise ValueError(f"{name}: expected a contiguous tensor")


_DELTA_IN = ("q", "k", "v", "g", "lr")


def _delta_inputs(cfg: DeltaConfig, x):
    """The five token inputs, checked: their device and strides (18 numbers, o's zero)."""
    dev, st = x["q"].device, []
    for n, shape, dtype, row in cfg.tokens:
        t = x[n]
        if t.shape != shape or t.dtype != dtype or t.device != dev:
            _check(t, n, shape, dtype, dev)
        s = t.stride()
        if row > 1 and s[3] != 1 and t.numel():
            raise ValueError(f"{n}: elements of a token must be adjacent")
        if n == "g":
            st += (0, 0, 0)  # o's place
        st += s[:3]
    return dev, st


def _place(dev, name, t):
    """A caller's buffer is where the tensors are."""
    if t.device != dev or not t.is_contiguous():
        raise ValueError(f"{name}: expected a contiguous tensor on {dev}")


def _current(dev):
    """The current stream of the tensors' device."""
    return torch._C._cuda_getCurrentRawStream(dev.index)


def _elsewhere(stream, dev) -> bool:
    """A call that is not for the current stream of the current device; refused off the GPUs."""
    if dev.index is None:
        raise ValueError(f"expected tensors on a GPU, got {dev}")
    return stream is not None or dev.index != torch._C._cuda_getDevice()


def _on_stream(stream, dev, inputs, call):
    """``call()`` with ``stream`` (torch's, or a handle; None: the device's current one) as the
    current one, and the tensors' device the current device: what it allocates is
    that stream's, so that a buffer dropped on return is given to nothing that does not wait for the
    kernels using it.  The inputs are marked as used there, the outputs as used on the caller's
    stream.  Ordering the two streams is the caller's, as with any torch work on a side stream."""
    back = torch.cuda.current_stream(dev)
    if stream is None:
        stream = back
    elif not hasattr(stream, "cuda_stream"):
        stream = torch.cuda.ExternalStream(stream, device=dev)
    with torch.cuda.stream(stream):
        out = call()
    made = out.values() if isinstance(out, dict) else out if isinstance(out, tuple) else (out,)
    for tensors, s in ((inputs, stream), (made, back)):
        for t in tensors:
            if t is not None:
                t.record_stream(s)
    return out


def _delta_rest(cfg: DeltaConfig, x, dev):
    S0, start = x.get("S0"), x.get("seq_start")
    if S0 is not None:
        _check(S0, "S0", (cfg.sequences, cfg.H, cfg.dk, cfg.dv), torch.float32, dev, True)
    if cfg.n_seq:
        if start is None:
            raise ValueError("packed sequences need seq_start")
        _check(start, "seq_start", (cfg.n_seq + 1,), torch.int32, dev, True)
    return S0, start


def delta_forward(cfg: DeltaConfig, x: Dict[str, torch.Tensor], save: bool = True,
                  final_state: bool = False, workspace: Optional[torch.Tensor] = None,
                  stream=None):
    """Run tnt_delta_fwd on ``x`` (q, k, v, g, lr and, where given, S0 and seq_start; any strides
    with adjacent elements); returns (o in v's layout, saved or None, final state or None)."""
    dev, st = _delta_inputs(cfg, x)
    S0, start = _delta_rest(cfg, x, dev)
    if workspace is not None:
        _place(dev, "workspace", workspace)
    if _elsewhere(stream, dev):
        return _on_stream(stream, dev, (*x.values(), workspace),
                          lambda: delta_forward(cfg, x, save, final_state, workspace))
    o = torch.empty_like(x["v"])
    st[9:12] = o.stride()[:3]
    fin = (torch.empty(cfg.sequences, cfg.H, cfg.dk, cfg.dv, dtype=torch.float32, device=dev)
           if final_state else None)
    saved = _bytes(cfg.size("saved"), dev) if save else None
    if workspace is None:
        workspace = _bytes(cfg.size(TNT_WS_FWD), dev)
    s = tnt_delta_fwd(cfg, _delta_strides6(*st), x["q"], x["k"], x["v"], x["g"], x["lr"], start,
                      S0, o, fin, saved, workspace, stream=_current(dev))
    if s != 0:
        raise TntError(s, "tnt_delta_fwd")
    return o, saved, fin


def delta_backward(cfg: DeltaConfig, x: Dict[str, torch.Tensor], dO: torch.Tensor,
                   saved: Optional[torch.Tensor] = None, dfinal: Optional[torch.Tensor] = None,
                   workspace: Optional[torch.Tensor] = None, stream=None):
    """Run tnt_delta_bwd; returns the gradients of sum(dO * o) + sum(dfinal * final state) in
    their inputs' layouts (dS0 where there is an S0).  ``saved`` None: recomputed."""
    dev, st = _delta_inputs(cfg, x)
    S0, start = _delta_rest(cfg, x, dev)
    _check(dO, "dO", cfg.shape("v"), cfg.io, dev)
    if dfinal is not None:
        _check(dfinal, "dfinal", (cfg.sequences, cfg.H, cfg.dk, cfg.dv), torch.float32, dev, True)
    if dO.stride(3) != 1 and cfg.dv > 1 and dO.numel():
        raise ValueError("dO: elements of a token must be adjacent")
    for n, t in (("workspace", workspace), ("saved", saved)):
        if t is not None:
            _place(dev, n, t)
    if saved is not None and _nbytes(saved, None) != max(16, cfg.size("saved")):
        raise ValueError(f"saved: expected {cfg.size('saved')} bytes, got {_nbytes(saved, None)}: "
                         "of another configuration")
    if _elsewhere(stream, dev):
        return _on_stream(stream, dev, (*x.values(), dO, saved, dfinal, workspace),
                          lambda: delta_backward(cfg, x, dO, saved, dfinal, workspace))
    st += dO.stride()[:3]
    out = {"d" + n: torch.empty_like(x[n]) for n in _DELTA_IN}
    for t in out.values():
        st += t.stride()[:3]
    dS0 = torch.empty_like(S0) if S0 is not None else None
    if workspace is None:
        workspace = _bytes(cfg.size(TNT_WS_BWD if saved is not None else TNT_WS_BWD_RECOMPUTE), dev)
    s = tnt_delta_bwd(cfg, tnt_delta_strides(*st), x["q"], x["k"], x["v"], x["g"], x["lr"], start,
                      S0, dO, dfinal, saved, out["dq"], out["dk"], out["dv"], out["dg"], out["dlr"],
                      dS0, workspace, stream=_current(dev))
    if s != 0:
        raise TntError(s, "tnt_delta_bwd")
    if dS0 is not None:
        out["dS0"] = dS0
    return out


def delta_step(cfg: DeltaConfig, x: Dict[str, torch.Tensor], state: torch.Tensor,
               slots: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Run tnt_delta_step over the cfg.L tokens of ``x``: ``state`` [slots][H][dk][dv] is updated
    in place, ``slots`` [B] (int32) names each sequence's state (outside: padding).  Returns o."""
    dev, st = _delta_inputs(cfg, x)
    _check(state, "state", (state.shape[0], cfg.H, cfg.dk, cfg.dv), torch.float32, dev, True)
    if slots is not None:
        _check(slots, "slots", (cfg.B,), torch.int32, dev, True)
    if _elsewhere(stream, dev):
        return _on_stream(stream, dev, (*x.values(), state, slots),
                          lambda: delta_step(cfg, x, state, slots))
    o = torch.empty_like(x["v"])
    st[9:12] = o.stride()[:3]
    s = tnt_delta_step(cfg, _delta_strides6(*st), x["q"], x["k"], x["v"], x["g"], x["lr"], state,
                       state.shape[0], slots, o, stream=_current(dev))
    if s != 0:
        raise TntError(s, "tnt_delta_step")
    return o


# --------------------------------------------------------------------------
# orthogonalised update
# --------------------------------------------------------------------------
class OrthConfig:
    """Shape and coefficients of an orthogonalised update (``tnt_orth_config``): n matrices of
    rows x cols; ``coef``: (a, b, c) for every step, or one such triple a step; None: the
    library's.  Immutable; the C structures and the workspace size are made once."""

    def __init__(self, *, n: int, rows: int, cols: int, dtype: int = F32, steps: int = 5,
                 coef=None, eps: float = 1e-7, scale: float = 1.0):
        self.n, self.rows, self.cols, self.dtype, self.steps = n, rows, cols, dtype, steps
        self.coef = None
        if coef is not None:
            flat = list(coef) * steps if not hasattr(coef[0], "__len__") else [v for t in coef for v in t]
            if len(flat) != 3 * steps:
                raise ValueError(f"coef: expected 3 numbers, or {steps} times 3")
            self.coef = (ctypes.c_float * len(flat))(*flat)
        self.c = tnt_orth_config(n, rows, cols, steps, dtype, eps, scale, 0, 0, 0, 0)
        self.ref = ctypes.byref(self.c)
        # a transposed matrix has the transpose's result: the same call with the sides swapped
        self.t = tnt_orth_config(n, cols, rows, steps, dtype, eps, scale, 0, 0, 0, 0)
        self._size = None

    @property
    def io(self):
        return torch.bfloat16 if self.dtype == BF16 else torch.float32

    @property
    def size(self) -> int:
        """Bytes of workspace for contiguous tensors (others: ``tnt_orth_workspace_size``)."""
        if self._size is None:
            self._size = lib().tnt_orth_workspace_size(self.ref)
        return self._size


def tnt_orth_workspace_size(cfg: OrthConfig) -> int:
    return lib().tnt_orth_workspace_size(cfg.ref)


def tnt_orth_update(c, coef, G, out, workspace, ws_bytes=None, stream=None) -> int:
    """``c``: a ``tnt_orth_config``; ``coef``: a ctypes array of 3 floats a step, or None."""
    return lib().tnt_orth_update(ctypes.byref(c), coef, _p(G), _p(out), _p(workspace),
                                 _nbytes(workspace, ws_bytes), _stream(stream))


def orthogonalise(cfg: OrthConfig, G: torch.Tensor, out: Optional[torch.Tensor] = None,
                  workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Run tnt_orth_update on G [n][rows][cols] (rows or columns of adjacent elements, any other
    strides but those of broadcasts); returns ``out``, by default a new tensor laid out as G."""
    _check(G, "G", (cfg.n, cfg.rows, cfg.cols), cfg.io, G.device)
    given = out
    if out is None:
        out = torch.empty_like(G)
    else:
        _check(out, "out", (cfg.n, cfg.rows, cfg.cols), cfg.io, G.device)
    c, flip = cfg.c, False
    if not (G.is_contiguous() and out.is_contiguous()):
        for name, t in (("G", G), ("out", out)):  # to the library a stride of 0 is a contiguous tensor's
            if any(t.shape[d] > 1 and t.stride(d) == 0 for d in range(3)):
                raise ValueError(f"{name}: broadcast matrices, rows or columns")
        unit = lambda t, d: t.shape[d] == 1 or t.stride(d) == 1
        flip = not (unit(G, 2) and unit(out, 2))
        if flip and not (unit(G, 1) and unit(out, 1)):
            raise ValueError("G and out: rows of both, or columns of both, must have adjacent elements")
        base, r = (cfg.t, 2) if flip else (cfg.c, 1)
        side = G.shape[3 - r]
        row = lambda t: t.stride(r) if t.shape[r] > 1 else side
        c = tnt_orth_config(base.n, base.rows, base.cols, base.steps, base.dtype, base.eps, base.scale,
                            G.stride(0), row(G), out.stride(0), row(out))
    if workspace is not None:
        _place(G.device, "workspace", workspace)
    if _elsewhere(stream, G.device):
        return _on_stream(stream, G.device, (G, given, workspace),
                          lambda: orthogonalise(cfg, G, given, workspace))
    if workspace is None:
        size = cfg.size if c is cfg.c else lib().tnt_orth_workspace_size(ctypes.byref(c))
        workspace = _bytes(size, G.device)
    s = tnt_orth_update(c, cfg.coef, G, out, workspace, stream=_current(G.device))
    if s != 0:
        raise TntError(s, "tnt_orth_update")
    return out
