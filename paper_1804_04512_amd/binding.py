"""Thin ctypes binding of libdll_conv.so: argument marshalling only.

Every function has the name of the C entry point it calls (`include/dll_conv.h`) and
does no arithmetic of its own.  PyTorch supplies device memory and the stream.  There is
no CPU fallback: a missing library or a non-OK status raises.
"""
from __future__ import annotations

import ctypes as C
import operator
import os
from dataclasses import dataclass
from typing import List, NamedTuple, Optional, Sequence

import torch

from .workloads import AttentionSpec, CacheSpec, ConvSpec, DenseSpec, GatedSpec, VocabSpec

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libdll_conv.so")

ACT = {"identity": 0, "sigmoid": 1, "relu": 2}
SYMBOLS = ["dll_status_string", "dll_conv_workspace_bytes", "dll_conv_valid_fwd", "dll_conv_full_bwd",
           "dll_conv_valid_wgrad", "dll_crbm_workspace_bytes", "dll_crbm_cd1_step",
           "dll_cnn_workspace_bytes", "dll_cnn_train_step", "dll_cnn_forward_workspace_bytes", "dll_cnn_forward",
           "dll_cnn_train_step_momentum", "dll_crbm_cd1_step_units", "dll_rbm_workspace_bytes", "dll_rbm_cd1_step",
           "dll_conv_full_fft_workspace_bytes", "dll_conv_full_bwd_fft", "dll_conv_valid_wgrad_noalloc",
           "dll_conv_valid_wgrad_partial", "dll_conv_valid_wgrad_finish",
           "dll_gated_fwd_workspace_bytes", "dll_gated_fwd", "dll_gated_bwd_workspace_bytes", "dll_gated_bwd",
           "dll_vocab_loss_fwd_workspace_bytes", "dll_vocab_loss_fwd", "dll_vocab_loss_grad_workspace_bytes",
           "dll_vocab_loss_grad", "dll_attention_fwd_workspace_bytes", "dll_attention_fwd", "dll_attention_bwd_workspace_bytes",
           "dll_attention_bwd", "dll_cache_plan", "dll_cache_write", "dll_paged_attention_workspace_bytes", "dll_paged_attention",
           "dll_grad_norm_workspace_bytes", "dll_grad_norm", "dll_grad_clip",
           "dll_momentum_update_clipped"]
NOALLOC_SCRATCH_BYTES = 8 << 20   # DLL_NOALLOC_SCRATCH_BYTES of include/dll_conv.h
VISIBLE = {"binary": 0, "gaussian": 1}
DTYPE = {"float32": 0, "bfloat16": 1}
GATE = {"identity": 0, "sigmoid": 1, "relu": 2, "silu": 3, "gelu": 4}
_TORCH_TYPE = {"float32": torch.float32, "bfloat16": torch.bfloat16}


class DllError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        msg = lib().dll_status_string(status).decode()
        super().__init__(f"{where}: {msg} (dll_status {status})")


class dll_conv_desc(C.Structure):
    _fields_ = [(n, C.c_int) for n in ("N", "C", "H", "W", "K", "R", "S", "pad", "act", "pool")]


class dll_dense_desc(C.Structure):
    _fields_ = [("in_", C.c_int), ("out", C.c_int), ("act", C.c_int)]


class dll_gated_desc(C.Structure):
    _fields_ = [(n, C.c_int) for n in ("tokens", "width", "hidden", "gate", "dtype")]


class dll_vocab_desc(C.Structure):
    _fields_ = [(n, C.c_int) for n in ("tokens", "width", "classes", "dtype")]


class dll_attention_desc(C.Structure):
    _fields_ = [(n, C.c_int) for n in ("q_tokens", "kv_tokens", "sequences", "heads", "kv_heads", "head_dim", "causal", "dtype",
                                       "q_row", "kv_row")]


class dll_cache_desc(C.Structure):
    _fields_ = [(n, C.c_int) for n in ("requests", "heads", "kv_heads", "head_dim", "pages", "page_tokens", "table_pages", "dtype")]


class dll_tensor_list(C.Structure):
    _fields_ = [("n", C.c_int), ("counts", C.POINTER(C.c_size_t)), ("dtypes", C.POINTER(C.c_int))]


class dll_net_desc(C.Structure):
    _fields_ = [("n_conv", C.c_int), ("conv", C.POINTER(dll_conv_desc)), ("n_dense", C.c_int),
                ("dense", C.POINTER(dll_dense_desc)), ("classes", C.c_int), ("batch", C.c_int)]


_lib = None


def lib() -> C.CDLL:
    """Loads the HIP library; raises if it has not been built (python -m paper_1804_04512_amd.build)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(f"{LIB_PATH} is missing: build it with `python -m paper_1804_04512_amd.build`")
        L = C.CDLL(LIB_PATH)
        vp, sz = C.c_void_p, C.c_size_t
        pd = C.POINTER(dll_conv_desc)
        L.dll_status_string.restype = C.c_char_p
        L.dll_status_string.argtypes = [C.c_int]
        L.dll_conv_workspace_bytes.restype = sz
        L.dll_conv_workspace_bytes.argtypes = [pd]
        L.dll_conv_valid_fwd.argtypes = [pd, vp, vp, vp, vp, vp, vp, sz, vp]
        L.dll_conv_full_bwd.argtypes = [pd, vp, vp, vp, vp, vp, vp, sz, vp]
        L.dll_conv_valid_wgrad.argtypes = [pd, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.dll_conv_valid_wgrad_noalloc.argtypes = [pd, vp, vp, vp, vp, vp, vp, vp]
        L.dll_conv_valid_wgrad_partial.argtypes = [pd, vp, vp, vp, vp, vp, sz, vp]
        L.dll_conv_valid_wgrad_finish.argtypes = [pd, vp, vp, vp, sz, vp]
        L.dll_conv_full_fft_workspace_bytes.restype = sz
        L.dll_conv_full_fft_workspace_bytes.argtypes = [pd]
        L.dll_conv_full_bwd_fft.argtypes = [pd, vp, vp, vp, vp, vp, vp, sz, vp]
        L.dll_crbm_workspace_bytes.restype = sz
        L.dll_crbm_workspace_bytes.argtypes = [pd]
        L.dll_crbm_cd1_step.argtypes = [pd, vp, vp, vp, vp, vp, vp, C.c_float] + [vp] * 8 + [vp, sz, vp]
        L.dll_crbm_cd1_step_units.argtypes = [pd, C.c_int, C.c_int, vp, vp, vp, vp, vp, vp, C.c_float] + [vp] * 9 + [vp, sz, vp]
        L.dll_rbm_workspace_bytes.restype = sz
        L.dll_rbm_workspace_bytes.argtypes = [C.c_int] * 3
        L.dll_rbm_cd1_step.argtypes = [C.c_int] * 4 + [vp, vp, vp, vp, vp, vp, C.c_float] + [vp] * 8 + [vp, sz, vp]
        L.dll_cnn_workspace_bytes.restype = sz
        L.dll_cnn_workspace_bytes.argtypes = [C.POINTER(dll_net_desc)]
        L.dll_cnn_train_step.argtypes = [C.POINTER(dll_net_desc), vp, vp, vp, vp, C.c_float, vp, vp, vp, vp, sz, vp]
        L.dll_cnn_train_step_momentum.argtypes = [C.POINTER(dll_net_desc), vp, vp, vp, vp, vp, C.c_float, C.c_float, C.c_float,
                                                  vp, vp, vp, vp, sz, vp]
        L.dll_cnn_forward_workspace_bytes.restype = sz
        L.dll_cnn_forward_workspace_bytes.argtypes = [C.POINTER(dll_net_desc)]
        L.dll_cnn_forward.argtypes = [C.POINTER(dll_net_desc), vp, vp, vp, vp, vp, sz, vp]
        pg, pv, pl = C.POINTER(dll_gated_desc), C.POINTER(dll_vocab_desc), C.POINTER(dll_tensor_list)
        pa, pc = C.POINTER(dll_attention_desc), C.POINTER(dll_cache_desc)
        for name, arg in (("dll_gated_fwd", pg), ("dll_gated_bwd", pg), ("dll_vocab_loss_fwd", pv), ("dll_vocab_loss_grad", pv),
                          ("dll_attention_fwd", pa), ("dll_attention_bwd", pa), ("dll_paged_attention", pc), ("dll_grad_norm", pl)):
            query = getattr(L, name + "_workspace_bytes")
            query.restype, query.argtypes = sz, [arg]
        L.dll_gated_fwd.argtypes = [pg] + [vp] * 8 + [sz, vp]
        L.dll_gated_bwd.argtypes = [pg] + [vp] * 12 + [sz, vp]
        L.dll_attention_fwd.argtypes = [pa] + [vp] * 5 + [C.c_float] + [vp] * 3 + [sz, vp]
        L.dll_attention_bwd.argtypes = [pa] + [vp] * 5 + [C.c_float] + [vp] * 7 + [sz, vp]
        L.dll_cache_plan.argtypes = [pc, vp, vp, vp, C.c_int] + [vp] * 4 + [C.c_int, vp, vp]
        L.dll_cache_write.argtypes = [pc, C.c_int, C.c_int] + [vp] * 6
        L.dll_paged_attention.argtypes = [pc] + [vp] * 5 + [C.c_float] + [vp] * 3 + [sz, vp]
        L.dll_vocab_loss_fwd.argtypes = [pv] + [vp] * 8 + [sz, vp]
        L.dll_vocab_loss_grad.argtypes = [pv] + [vp] * 4 + [C.c_float] + [vp] * 7 + [sz, vp]
        L.dll_grad_norm.argtypes = [pl, vp, vp, vp, sz, vp]
        L.dll_grad_clip.argtypes = [pl, vp, vp, C.c_float, vp, vp, sz, vp]
        L.dll_momentum_update_clipped.argtypes = [pl, vp, vp, vp, C.c_float, C.c_float, vp, C.c_float, vp, vp, vp, sz, vp]
        _lib = L
    return _lib


def conv_desc(cs: ConvSpec) -> dll_conv_desc:
    return dll_conv_desc(cs.N, cs.C, cs.H, cs.W, cs.K, cs.R, cs.S, cs.pad, ACT[cs.act], cs.pool)


def _ptr(t: Optional[torch.Tensor]):
    if t is None:
        return None
    assert t.is_cuda and t.is_contiguous(), "device-resident contiguous tensors only"
    return t.data_ptr()   # argtypes turn the number into a pointer


def _stream(stream=None):
    return (stream if stream is not None else torch.cuda.current_stream()).cuda_stream


def _ok(status: int, where: str):
    if status != 0:
        raise DllError(status, where)


def workspace(nbytes: int, device="cuda") -> Optional[torch.Tensor]:
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)


def dll_conv_workspace_bytes(cs: ConvSpec) -> int:
    d = conv_desc(cs)
    return int(lib().dll_conv_workspace_bytes(C.byref(d)))


def dll_conv_valid_fwd(cs: ConvSpec, x, w, bias, y, pool_idx=None, ws=None, stream=None) -> None:
    d = conv_desc(cs)
    _ok(lib().dll_conv_valid_fwd(C.byref(d), _ptr(x), _ptr(w), _ptr(bias), _ptr(y), _ptr(pool_idx), _ptr(ws),
                                 0 if ws is None else ws.numel(), _stream(stream)), "dll_conv_valid_fwd")


def dll_conv_full_bwd(cs: ConvSpec, dy, y, pool_idx, w, dx, ws=None, stream=None) -> None:
    d = conv_desc(cs)
    _ok(lib().dll_conv_full_bwd(C.byref(d), _ptr(dy), _ptr(y), _ptr(pool_idx), _ptr(w), _ptr(dx), _ptr(ws),
                                0 if ws is None else ws.numel(), _stream(stream)), "dll_conv_full_bwd")


def dll_conv_full_fft_workspace_bytes(cs: ConvSpec) -> int:
    d = conv_desc(cs)
    return int(lib().dll_conv_full_fft_workspace_bytes(C.byref(d)))


def dll_conv_full_bwd_fft(cs: ConvSpec, dy, y, pool_idx, w, dx, ws, stream=None) -> None:
    d = conv_desc(cs)
    _ok(lib().dll_conv_full_bwd_fft(C.byref(d), _ptr(dy), _ptr(y), _ptr(pool_idx), _ptr(w), _ptr(dx), _ptr(ws),
                                    0 if ws is None else ws.numel(), _stream(stream)), "dll_conv_full_bwd_fft")


def dll_conv_valid_wgrad(cs: ConvSpec, x, dy, y, pool_idx, dw, dbias, ws, stream=None) -> None:
    d = conv_desc(cs)
    _ok(lib().dll_conv_valid_wgrad(C.byref(d), _ptr(x), _ptr(dy), _ptr(y), _ptr(pool_idx), _ptr(dw), _ptr(dbias),
                                   _ptr(ws), 0 if ws is None else ws.numel(), _stream(stream)), "dll_conv_valid_wgrad")


def dll_conv_valid_wgrad_partial(cs: ConvSpec, x, dy, y, pool_idx, ws, stream=None) -> None:
    d = conv_desc(cs)
    _ok(lib().dll_conv_valid_wgrad_partial(C.byref(d), _ptr(x), _ptr(dy), _ptr(y), _ptr(pool_idx), _ptr(ws),
                                           0 if ws is None else ws.numel(), _stream(stream)), "dll_conv_valid_wgrad_partial")


def dll_conv_valid_wgrad_finish(cs: ConvSpec, dw, dbias, ws, stream=None) -> None:
    d = conv_desc(cs)
    _ok(lib().dll_conv_valid_wgrad_finish(C.byref(d), _ptr(dw), _ptr(dbias), _ptr(ws), 0 if ws is None else ws.numel(),
                                          _stream(stream)), "dll_conv_valid_wgrad_finish")


def dll_conv_valid_wgrad_noalloc(cs: ConvSpec, x, dy, y, pool_idx, dw, dbias, stream=None) -> None:
    d = conv_desc(cs)
    _ok(lib().dll_conv_valid_wgrad_noalloc(C.byref(d), _ptr(x), _ptr(dy), _ptr(y), _ptr(pool_idx), _ptr(dw), _ptr(dbias),
                                           _stream(stream)), "dll_conv_valid_wgrad_noalloc")


def dll_crbm_workspace_bytes(cs: ConvSpec) -> int:
    d = conv_desc(cs)
    return int(lib().dll_crbm_workspace_bytes(C.byref(d)))


def dll_crbm_cd1_step(cs: ConvSpec, v0, W, b_hid, c_vis, uniform, h0_sample_in, lr, dW, db, dc, h0_prob=None,
                      h0_sample=None, v1=None, h1_prob=None, recon_mse=None, ws=None, stream=None) -> None:
    d = conv_desc(cs)
    _ok(lib().dll_crbm_cd1_step(C.byref(d), _ptr(v0), _ptr(W), _ptr(b_hid), _ptr(c_vis), _ptr(uniform),
                                _ptr(h0_sample_in), C.c_float(lr), _ptr(dW), _ptr(db), _ptr(dc), _ptr(h0_prob),
                                _ptr(h0_sample), _ptr(v1), _ptr(h1_prob), _ptr(recon_mse), _ptr(ws),
                                0 if ws is None else ws.numel(), _stream(stream)), "dll_crbm_cd1_step")


def dll_crbm_cd1_step_units(cs: ConvSpec, visible: int, hidden_pool: int, v0, W, b_hid, c_vis, uniform, h0_sample_in, lr,
                            dW, db, dc, h0_prob=None, h0_sample=None, pool_prob=None, v1=None, h1_prob=None,
                            recon_mse=None, ws=None, stream=None) -> None:
    d = conv_desc(cs)
    _ok(lib().dll_crbm_cd1_step_units(C.byref(d), int(visible), int(hidden_pool), _ptr(v0), _ptr(W), _ptr(b_hid),
                                      _ptr(c_vis), _ptr(uniform), _ptr(h0_sample_in), C.c_float(lr), _ptr(dW), _ptr(db),
                                      _ptr(dc), _ptr(h0_prob), _ptr(h0_sample), _ptr(pool_prob), _ptr(v1), _ptr(h1_prob),
                                      _ptr(recon_mse), _ptr(ws), 0 if ws is None else ws.numel(), _stream(stream)),
        "dll_crbm_cd1_step_units")


def dll_rbm_workspace_bytes(batch: int, n_vis: int, n_hid: int) -> int:
    return int(lib().dll_rbm_workspace_bytes(batch, n_vis, n_hid))


def dll_rbm_cd1_step(batch: int, n_vis: int, n_hid: int, visible: int, v0, W, b_hid, c_vis, uniform, h0_sample_in, lr, dW,
                     db, dc, h0_prob=None, h0_sample=None, v1=None, h1_prob=None, recon_mse=None, ws=None,
                     stream=None) -> None:
    _ok(lib().dll_rbm_cd1_step(batch, n_vis, n_hid, int(visible), _ptr(v0), _ptr(W), _ptr(b_hid), _ptr(c_vis),
                               _ptr(uniform), _ptr(h0_sample_in), C.c_float(lr), _ptr(dW), _ptr(db), _ptr(dc),
                               _ptr(h0_prob), _ptr(h0_sample), _ptr(v1), _ptr(h1_prob), _ptr(recon_mse), _ptr(ws),
                               0 if ws is None else ws.numel(), _stream(stream)), "dll_rbm_cd1_step")


@dataclass
class NetHandle:
    """Host-side descriptor arrays kept alive for the duration of the calls."""
    desc: dll_net_desc
    convs: object
    denses: object


def net_desc(conv: Sequence[ConvSpec], dense: Sequence[DenseSpec], classes: int, batch: int = 0) -> NetHandle:
    """`batch` is needed only for a fully-connected network (no conv layers)."""
    convs = (dll_conv_desc * len(conv))(*[conv_desc(c) for c in conv])
    denses = (dll_dense_desc * len(dense))(*[dll_dense_desc(d.in_, d.out, ACT[d.act]) for d in dense])
    return NetHandle(dll_net_desc(len(conv), convs, len(dense), denses, classes, batch), convs, denses)


def dll_cnn_workspace_bytes(net: NetHandle) -> int:
    return int(lib().dll_cnn_workspace_bytes(C.byref(net.desc)))


def _ptr_array(ts: Optional[Sequence[Optional[torch.Tensor]]]):
    if ts is None:
        return None
    arr = (C.c_void_p * len(ts))(*[None if t is None else t.data_ptr() for t in ts])
    for t in ts:
        assert t is None or (t.is_cuda and t.is_contiguous())
    return arr


def dll_cnn_train_step(net: NetHandle, params: List[torch.Tensor], grads, x, labels, lr, loss, logits=None,
                       pool_idx=None, ws=None, stream=None) -> None:
    pa, ga, ia = _ptr_array(params), _ptr_array(grads), _ptr_array(pool_idx)
    _ok(lib().dll_cnn_train_step(C.byref(net.desc), pa, ga, _ptr(x), _ptr(labels), C.c_float(lr), _ptr(loss),
                                 _ptr(logits), ia, _ptr(ws), 0 if ws is None else ws.numel(), _stream(stream)),
        "dll_cnn_train_step")


def dll_cnn_forward_workspace_bytes(net: NetHandle) -> int:
    return int(lib().dll_cnn_forward_workspace_bytes(C.byref(net.desc)))


def dll_cnn_forward(net: NetHandle, params: List[torch.Tensor], x, logits=None, prob=None, ws=None, stream=None) -> None:
    pa = _ptr_array(params)
    _ok(lib().dll_cnn_forward(C.byref(net.desc), pa, _ptr(x), _ptr(logits), _ptr(prob), _ptr(ws),
                              0 if ws is None else ws.numel(), _stream(stream)), "dll_cnn_forward")


def dll_cnn_train_step_momentum(net: NetHandle, params: List[torch.Tensor], velocity: List[torch.Tensor], grads, x, labels, lr,
                                momentum, weight_decay, loss, logits=None, pool_idx=None, ws=None, stream=None) -> None:
    pa, va, ga, ia = _ptr_array(params), _ptr_array(velocity), _ptr_array(grads), _ptr_array(pool_idx)
    _ok(lib().dll_cnn_train_step_momentum(C.byref(net.desc), pa, va, ga, _ptr(x), _ptr(labels), C.c_float(lr),
                                          C.c_float(momentum), C.c_float(weight_decay), _ptr(loss), _ptr(logits), ia, _ptr(ws),
                                          0 if ws is None else ws.numel(), _stream(stream)), "dll_cnn_train_step_momentum")


# ---------------------------------------------------------------------------------------
# Large-model operators.  The C calls know addresses only, so what an address must hold (type,
# shape, device) is checked here.
# ---------------------------------------------------------------------------------------
def _tensor(t: Optional[torch.Tensor], shape, dtype: torch.dtype, what: str, device, optional: bool = False):
    """The address of a tensor that has to have this shape and type and lie on this device."""
    if t is not None and t.dtype is dtype and t.shape == shape and t.device == device and t.is_contiguous():
        return t.data_ptr()
    if t is None:
        if optional:
            return None
        raise ValueError(f"{what}: a tensor is required")
    if t.dtype != dtype or t.shape != shape:
        raise ValueError(f"{what}: {dtype} of shape {tuple(shape)} expected, got {t.dtype} of shape {tuple(t.shape)}")
    if t.device != device or not t.is_contiguous():
        raise ValueError(f"{what}: contiguous and on {device} (the device of the call's stream) expected")
    return t.data_ptr()


class _CurrentStream(NamedTuple):
    device: torch.device
    cuda_stream: int


def _call_stream(stream):
    if stream is None:
        index = torch.cuda.current_device()
        try:
            # its address alone: the object that torch.cuda.current_stream() makes of it takes 2.6 us, a quarter of a small call
            address = torch._C._cuda_getCurrentRawStream(index)
        except AttributeError:   # a private name, which another version need not have
            address = torch.cuda.current_stream(index).cuda_stream
        return _CurrentStream(torch.device("cuda", index), address)
    s = stream
    if s.device != torch.device("cuda", torch.cuda.current_device()):
        raise ValueError(f"the stream belongs to {s.device}, which is not the current device")
    return s


def _ws(ws: Optional[torch.Tensor], device):
    if ws is None:
        return None, 0
    if ws.device != device or not ws.is_contiguous():
        raise ValueError(f"ws: contiguous and on {device} expected")
    return ws.data_ptr(), ws.numel() * ws.element_size()


def gated_desc(g: GatedSpec) -> dll_gated_desc:
    return dll_gated_desc(g.tokens, g.width, g.hidden, GATE[g.gate], DTYPE[g.dtype])


def vocab_desc(v: VocabSpec) -> dll_vocab_desc:
    return dll_vocab_desc(v.tokens, v.width, v.classes, DTYPE[v.dtype])


def dll_gated_fwd_workspace_bytes(g: GatedSpec) -> int:
    return int(lib().dll_gated_fwd_workspace_bytes(C.byref(gated_desc(g))))


def dll_gated_fwd(g: GatedSpec, x, w_gate, w_up, w_down, y, gate_pre=None, up_pre=None, ws=None, stream=None) -> None:
    s = _call_stream(stream)
    t, dev = _TORCH_TYPE[g.dtype], s.device
    io, up, kept = (g.tokens, g.width), (g.hidden, g.width), (g.tokens, g.hidden)
    _ok(lib().dll_gated_fwd(C.byref(gated_desc(g)), _tensor(x, io, t, "x", dev), _tensor(w_gate, up, t, "w_gate", dev),
                            _tensor(w_up, up, t, "w_up", dev), _tensor(w_down, up[::-1], t, "w_down", dev),
                            _tensor(y, io, t, "y", dev), _tensor(gate_pre, kept, t, "gate_pre", dev, True),
                            _tensor(up_pre, kept, t, "up_pre", dev, True), *_ws(ws, dev), s.cuda_stream), "dll_gated_fwd")


def dll_gated_bwd_workspace_bytes(g: GatedSpec) -> int:
    return int(lib().dll_gated_bwd_workspace_bytes(C.byref(gated_desc(g))))


def dll_gated_bwd(g: GatedSpec, x, w_gate, w_up, w_down, gate_pre, up_pre, dy, dx=None, dw_gate=None, dw_up=None, dw_down=None,
                  ws=None, stream=None) -> None:
    s = _call_stream(stream)
    t, dev = _TORCH_TYPE[g.dtype], s.device
    io, up, kept = (g.tokens, g.width), (g.hidden, g.width), (g.tokens, g.hidden)
    _ok(lib().dll_gated_bwd(C.byref(gated_desc(g)), _tensor(x, io, t, "x", dev), _tensor(w_gate, up, t, "w_gate", dev),
                            _tensor(w_up, up, t, "w_up", dev), _tensor(w_down, up[::-1], t, "w_down", dev),
                            _tensor(gate_pre, kept, t, "gate_pre", dev), _tensor(up_pre, kept, t, "up_pre", dev),
                            _tensor(dy, io, t, "dy", dev), _tensor(dx, io, t, "dx", dev, True),
                            _tensor(dw_gate, up, t, "dw_gate", dev, True), _tensor(dw_up, up, t, "dw_up", dev, True),
                            _tensor(dw_down, up[::-1], t, "dw_down", dev, True), *_ws(ws, dev), s.cuda_stream), "dll_gated_bwd")


def dll_vocab_loss_fwd_workspace_bytes(v: VocabSpec) -> int:
    return int(lib().dll_vocab_loss_fwd_workspace_bytes(C.byref(vocab_desc(v))))


def _vocab_inputs(v: VocabSpec, x, w, bias, labels, dev):
    t = _TORCH_TYPE[v.dtype]
    return (_tensor(x, (v.tokens, v.width), t, "x", dev), _tensor(w, (v.classes, v.width), t, "w", dev),
            _tensor(bias, (v.classes,), t, "bias", dev, True), _tensor(labels, (v.tokens,), torch.int32, "labels", dev))


def _vocab_losses(v: VocabSpec, row_loss, row_lse, loss, dev):
    f = torch.float32
    return (_tensor(row_loss, (v.tokens,), f, "row_loss", dev, True), _tensor(row_lse, (v.tokens,), f, "row_lse", dev, True),
            _tensor(loss, (1,), f, "loss", dev))


def dll_vocab_loss_fwd(v: VocabSpec, x, w, bias, labels, row_loss, row_lse, loss, ws=None, stream=None) -> None:
    s = _call_stream(stream)
    dev = s.device
    _ok(lib().dll_vocab_loss_fwd(C.byref(vocab_desc(v)), *_vocab_inputs(v, x, w, bias, labels, dev),
                                 *_vocab_losses(v, row_loss, row_lse, loss, dev), *_ws(ws, dev), s.cuda_stream), "dll_vocab_loss_fwd")


def dll_vocab_loss_grad_workspace_bytes(v: VocabSpec) -> int:
    return int(lib().dll_vocab_loss_grad_workspace_bytes(C.byref(vocab_desc(v))))


def dll_vocab_loss_grad(v: VocabSpec, x, w, bias, labels, scale, row_loss, row_lse, loss, dx=None, dw=None, dbias=None, ws=None,
                        stream=None) -> None:
    s = _call_stream(stream)
    t, dev = _TORCH_TYPE[v.dtype], s.device
    _ok(lib().dll_vocab_loss_grad(C.byref(vocab_desc(v)), *_vocab_inputs(v, x, w, bias, labels, dev), C.c_float(scale),
                                  *_vocab_losses(v, row_loss, row_lse, loss, dev),
                                  _tensor(dx, (v.tokens, v.width), t, "dx", dev, True),
                                  _tensor(dw, (v.classes, v.width), t, "dw", dev, True),
                                  _tensor(dbias, (v.classes,), t, "dbias", dev, True), *_ws(ws, dev), s.cuda_stream),
        "dll_vocab_loss_grad")


_MOST = (1 << 31) - 1   # of the library's int arguments


def attention_desc(a: AttentionSpec) -> dll_attention_desc:
    return dll_attention_desc(a.q_tokens, a.kv_tokens, a.sequences, a.heads, a.kv_heads, a.head_dim, int(a.causal), DTYPE[a.dtype],
                              a.q_row, a.kv_row)


def _head_rows(t: Optional[torch.Tensor], shape, row: int, dtype: torch.dtype, what: str, device, optional: bool = False):
    """The address of a tensor [tokens][heads][head_dim] whose tokens lie `row` elements apart (0: contiguous)."""
    if t is None:
        return _tensor(t, shape, dtype, what, device, optional)
    if row > _MOST:   # ctypes would cut it
        raise ValueError(f"{what}: tokens {row} elements apart, {_MOST} at most")
    if t.dtype != dtype or t.shape != shape:
        raise ValueError(f"{what}: {dtype} of shape {tuple(shape)} expected, got {t.dtype} of shape {tuple(t.shape)}")
    strides = (row or shape[1] * shape[2], shape[2], 1)
    if t.device == device and t.stride() == strides:
        return t.data_ptr()
    if t.device != device or any(n > 1 and s != want for n, s, want in zip(shape, t.stride(), strides)):
        raise ValueError(f"{what}: strides {strides} and on {device} (the device of the call's stream) expected")
    return t.data_ptr()


def _attention_inputs(a: AttentionSpec, q, k, v, q_starts, kv_starts, dev):
    t, kv = _TORCH_TYPE[a.dtype], (a.kv_tokens, a.kv_heads, a.head_dim)
    return (_head_rows(q, (a.q_tokens, a.heads, a.head_dim), a.q_row, t, "q", dev), _head_rows(k, kv, a.kv_row, t, "k", dev),
            _head_rows(v, kv, a.kv_row, t, "v", dev), _tensor(q_starts, (a.sequences + 1,), torch.int32, "q_starts", dev),
            _tensor(kv_starts, (a.sequences + 1,), torch.int32, "kv_starts", dev))


def dll_attention_fwd_workspace_bytes(a: AttentionSpec) -> int:
    return int(lib().dll_attention_fwd_workspace_bytes(C.byref(attention_desc(a))))


def dll_attention_fwd(a: AttentionSpec, q, k, v, q_starts, kv_starts, scale, o, lse=None, ws=None, stream=None) -> None:
    s = _call_stream(stream)
    t, dev = _TORCH_TYPE[a.dtype], s.device
    _ok(lib().dll_attention_fwd(C.byref(attention_desc(a)), *_attention_inputs(a, q, k, v, q_starts, kv_starts, dev), C.c_float(scale),
                                _tensor(o, (a.q_tokens, a.heads, a.head_dim), t, "o", dev),
                                _tensor(lse, (a.heads, a.q_tokens), torch.float32, "lse", dev, True), *_ws(ws, dev), s.cuda_stream),
        "dll_attention_fwd")


def dll_attention_bwd_workspace_bytes(a: AttentionSpec) -> int:
    return int(lib().dll_attention_bwd_workspace_bytes(C.byref(attention_desc(a))))


def dll_attention_bwd(a: AttentionSpec, q, k, v, q_starts, kv_starts, scale, o, lse, d_o, dq=None, dk=None, dv=None, ws=None,
                      stream=None) -> None:
    s = _call_stream(stream)
    t, dev = _TORCH_TYPE[a.dtype], s.device
    qs, kvs = (a.q_tokens, a.heads, a.head_dim), (a.kv_tokens, a.kv_heads, a.head_dim)
    _ok(lib().dll_attention_bwd(C.byref(attention_desc(a)), *_attention_inputs(a, q, k, v, q_starts, kv_starts, dev), C.c_float(scale),
                                _tensor(o, qs, t, "o", dev), _tensor(lse, (a.heads, a.q_tokens), torch.float32, "lse", dev),
                                _tensor(d_o, qs, t, "d_o", dev), _head_rows(dq, qs, a.q_row, t, "dq", dev, True),
                                _head_rows(dk, kvs, a.kv_row, t, "dk", dev, True), _head_rows(dv, kvs, a.kv_row, t, "dv", dev, True),
                                *_ws(ws, dev), s.cuda_stream), "dll_attention_bwd")


def cache_desc(c: CacheSpec) -> dll_cache_desc:
    return dll_cache_desc(c.requests, c.heads, c.kv_heads, c.head_dim, c.pages, c.page_tokens, c.table_pages, DTYPE[c.dtype])


def _ints(t, n, what: str, dev, optional: bool = False):
    """The address of a vector of whole numbers; n: its length, or None (any), or a shape."""
    if t is not None and n is None:
        n = t.numel()
        if n > _MOST:
            raise ValueError(f"{what}: {n} entries, {_MOST} at most")
    return _tensor(t, n if isinstance(n, tuple) else (n,), torch.int32, what, dev, optional)


def dll_cache_plan(c: CacheSpec, lengths, added, free_pages, table, starts, slots, state, free_at=None, stream=None) -> None:
    """free_pages and slots: of any length."""
    s = _call_stream(stream)
    dev, n = s.device, c.requests
    _ok(lib().dll_cache_plan(C.byref(cache_desc(c)), _ints(lengths, n, "lengths", dev), _ints(added, n, "added", dev),
                             _ints(free_pages, None, "free_pages", dev), free_pages.numel(), _ints(free_at, 1, "free_at", dev, True),
                             _ints(table, (n, c.table_pages), "table", dev), _ints(starts, n + 1, "starts", dev),
                             _ints(slots, None, "slots", dev), slots.numel(), _ints(state, 2, "state", dev), s.cuda_stream), "dll_cache_plan")


def _caches(c: CacheSpec, k_cache, v_cache, dev):
    shape, t = (c.pages, c.kv_heads, c.page_tokens, c.head_dim), _TORCH_TYPE[c.dtype]
    return _tensor(k_cache, shape, t, "k_cache", dev), _tensor(v_cache, shape, t, "v_cache", dev)


def dll_cache_write(c: CacheSpec, k, v, slots, k_cache, v_cache, stream=None) -> None:
    """k, v: [tokens][kv_heads][head_dim], their tokens equally far apart in both."""
    s = _call_stream(stream)
    dev, t = s.device, _TORCH_TYPE[c.dtype]
    tokens, row = slots.numel(), k.stride(0) if k.shape[0] > 1 else 0
    shape = (tokens, c.kv_heads, c.head_dim)
    _ok(lib().dll_cache_write(C.byref(cache_desc(c)), tokens, row, _head_rows(k, shape, row, t, "k", dev), _head_rows(v, shape, row, t, "v", dev),
                              _ints(slots, None, "slots", dev), *_caches(c, k_cache, v_cache, dev), s.cuda_stream), "dll_cache_write")


def dll_paged_attention_workspace_bytes(c: CacheSpec) -> int:
    return int(lib().dll_paged_attention_workspace_bytes(C.byref(cache_desc(c))))


def dll_paged_attention(c: CacheSpec, q, k_cache, v_cache, table, lengths, scale, o, lse=None, ws=None, stream=None) -> None:
    s = _call_stream(stream)
    dev, t, rows = s.device, _TORCH_TYPE[c.dtype], (c.requests, c.heads, c.head_dim)
    _ok(lib().dll_paged_attention(C.byref(cache_desc(c)), _tensor(q, rows, t, "q", dev), *_caches(c, k_cache, v_cache, dev),
                                  _ints(table, (c.requests, c.table_pages), "table", dev), _ints(lengths, c.requests, "lengths", dev),
                                  C.c_float(scale), _tensor(o, rows, t, "o", dev),
                                  _tensor(lse, (c.requests, c.heads), torch.float32, "lse", dev, True), *_ws(ws, dev), s.cuda_stream),
        "dll_paged_attention")


_DTYPE_OF = operator.attrgetter("dtype")
_NUMEL, _CONTIGUOUS = torch.Tensor.numel, torch.Tensor.is_contiguous
_DEVICE_OF, _ADDRESS = torch.Tensor.get_device, torch.Tensor.data_ptr


@dataclass
class TensorList:
    """Numbers of elements and types of a list of gradients, kept for the calls on them."""
    desc: dll_tensor_list
    counts: object
    dtypes: object
    torch_types: List[torch.dtype]
    numels: List[int]
    array: type   # of n addresses


def tensor_list(grads: Sequence[torch.Tensor]) -> TensorList:
    names = {v: k for k, v in _TORCH_TYPE.items()}
    for g in grads:
        if g.dtype not in names:
            raise ValueError(f"gradients are float32 or bfloat16, got {g.dtype}")
    counts = (C.c_size_t * len(grads))(*[g.numel() for g in grads])
    dtypes = (C.c_int * len(grads))(*[DTYPE[names[g.dtype]] for g in grads])
    return TensorList(dll_tensor_list(len(grads), counts, dtypes), counts, dtypes, [g.dtype for g in grads],
                      list(counts), C.c_void_p * len(grads))


def _list_ptrs(tensors: Sequence[Optional[torch.Tensor]], l: TensorList, dtypes, what: str, dev, optional: bool = False):
    """Addresses of one tensor for each entry of the list, of any shape with as many elements."""
    n = l.desc.n
    if len(tensors) != n:
        raise ValueError(f"{what}: {n} tensors expected, got {len(tensors)}")
    if not any(t is None for t in tensors):
        # the whole list at a time: a call over hundreds of tensors would spend longer on checks one by one than on the GPU
        index = -1 if dev.type == "cpu" else dev.index
        if (list(map(_DTYPE_OF, tensors)) == dtypes and list(map(_NUMEL, tensors)) == l.numels and all(map(_CONTIGUOUS, tensors))
                and list(map(_DEVICE_OF, tensors)).count(index) == n):
            return l.array(*map(_ADDRESS, tensors))
    for t, k, dtype in zip(tensors, l.numels, dtypes):
        if t is None:
            if optional or k == 0:
                continue
            raise ValueError(f"{what}: a tensor is required")
        if t.dtype != dtype or t.numel() != k or t.device != dev or not t.is_contiguous():
            raise ValueError(f"{what}: contiguous {dtype} with {k} elements on {dev} expected, got {t.dtype} with {t.numel()} on {t.device}")
    return l.array(*[None if t is None else t.data_ptr() for t in tensors])


def dll_grad_norm_workspace_bytes(l: TensorList) -> int:
    return int(lib().dll_grad_norm_workspace_bytes(C.byref(l.desc)))


def dll_grad_norm(l: TensorList, grads, norm, ws=None, stream=None) -> None:
    s = _call_stream(stream)
    dev = s.device
    _ok(lib().dll_grad_norm(C.byref(l.desc), _list_ptrs(grads, l, l.torch_types, "grads", dev),
                            _tensor(norm, (1,), torch.float32, "norm", dev), *_ws(ws, dev), s.cuda_stream), "dll_grad_norm")


def dll_grad_clip(l: TensorList, grads, out, max_norm, norm, ws=None, stream=None) -> None:
    s = _call_stream(stream)
    dev = s.device
    _ok(lib().dll_grad_clip(C.byref(l.desc), _list_ptrs(grads, l, l.torch_types, "grads", dev),
                            _list_ptrs(out, l, l.torch_types, "out", dev), C.c_float(max_norm),
                            _tensor(norm, (1,), torch.float32, "norm", dev), *_ws(ws, dev), s.cuda_stream), "dll_grad_clip")


def dll_momentum_update_clipped(l: TensorList, params, velocity, grads, lr, momentum, weight_decay, max_norm, norm, copies=None,
                                ws=None, stream=None) -> None:
    """weight_decay: one factor a tensor, or None."""
    s = _call_stream(stream)
    dev, n = s.device, l.desc.n
    f = [torch.float32] * n
    if weight_decay is not None and len(weight_decay) != n:
        raise ValueError(f"weight_decay: {n} factors expected, got {len(weight_decay)}")
    _ok(lib().dll_momentum_update_clipped(
        C.byref(l.desc), _list_ptrs(params, l, f, "params", dev), _list_ptrs(velocity, l, f, "velocity", dev),
        _list_ptrs(grads, l, l.torch_types, "grads", dev), C.c_float(lr), C.c_float(momentum),
        None if weight_decay is None else (C.c_float * n)(*weight_decay), C.c_float(max_norm),
        _tensor(norm, (1,), torch.float32, "norm", dev),
        None if copies is None else _list_ptrs(copies, l, [torch.bfloat16] * n, "copies", dev, True), *_ws(ws, dev), s.cuda_stream),
        "dll_momentum_update_clipped")
