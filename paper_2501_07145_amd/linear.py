"""Binding of the operators of linear models on feature rows: softmax cross entropy with its gradients, the AdamW
step, and the Gram against rows held in 8-bit integers (include/rfsf_ts.h). Argument marshalling only, as in binding.py."""
from __future__ import annotations

import ctypes
from array import array
from typing import Optional, Sequence

import numpy as np
import torch

from .binding import _check, _dev, _empty_on, _stream_ptr, load_library

_BF16 = {torch.float32: 0, torch.bfloat16: 1}
_DPHI, _DW = 1, 2


class _XentShape(ctypes.Structure):
    _fields_ = [("N", ctypes.c_int64), ("K", ctypes.c_int64), ("C", ctypes.c_int64),
                ("ld_phi", ctypes.c_int64), ("ld_w", ctypes.c_int64), ("ld_dphi", ctypes.c_int64), ("ld_dw", ctypes.c_int64),
                ("bf16", ctypes.c_int32), ("gradients", ctypes.c_int32)]


class _AdamwConfig(ctypes.Structure):
    _fields_ = [("lr", ctypes.c_double), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double), ("eps", ctypes.c_double),
                ("weight_decay", ctypes.c_double), ("grad_scale", ctypes.c_double),
                ("step", ctypes.c_int64), ("state_bits", ctypes.c_int32), ("grad_bf16", ctypes.c_int32)]


class _AdamwTensor(ctypes.Structure):
    _fields_ = [("param", ctypes.c_void_p), ("grad", ctypes.c_void_p), ("m", ctypes.c_void_p), ("v", ctypes.c_void_p),
                ("m_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p), ("copy", ctypes.c_void_p), ("n", ctypes.c_int64)]


def _matrix(t: torch.Tensor, name: str, dtype=None, shape=None) -> int:
    """Row stride of a 2-D device tensor of float32 or bfloat16 with unit column stride."""
    sizes, strides = t.shape, t.stride()
    if len(sizes) != 2 or not t.is_cuda or t.dtype not in _BF16 or (strides[1] != 1 and sizes[1] > 1):
        raise ValueError(f"{name} must be float32 or bfloat16 [rows, cols] on the device with unit column stride")
    if dtype is not None and t.dtype is not dtype:
        raise ValueError(f"{name} must be {dtype}")
    if shape is not None and sizes != shape:
        raise ValueError(f"{name} must have shape {list(shape)}")
    return strides[0] if sizes[0] > 1 else max(sizes[1], 1)


def rfsf_softmax_xent_workspace_bytes(N: int, K: int, C: int, dtype: torch.dtype = torch.float32, need_dPhi: bool = False,
                                      need_dW: bool = False):
    """(recommended_bytes, minimum_bytes) of scratch for rfsf_softmax_xent."""
    if dtype not in _BF16:
        raise ValueError("dtype must be float32 or bfloat16")
    shp = _XentShape(N, K, C, K, K, K, K, _BF16[dtype], (_DPHI if need_dPhi else 0) | (_DW if need_dW else 0))
    rec, mn = ctypes.c_size_t(0), ctypes.c_size_t(0)
    _check(load_library().rfsf_softmax_xent_workspace_bytes(ctypes.byref(shp), ctypes.byref(rec), ctypes.byref(mn)))
    return int(rec.value), int(mn.value)


def rfsf_softmax_xent(Phi: torch.Tensor, W: torch.Tensor, labels: torch.Tensor, weight: Optional[torch.Tensor] = None,
                      need_dPhi: bool = False, need_dW: bool = False, loss: Optional[torch.Tensor] = None,
                      dPhi: Optional[torch.Tensor] = None, dW: Optional[torch.Tensor] = None,
                      workspace: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None):
    """(loss [N], dPhi or None, dW or None): softmax cross entropy of the scores Phi W^T against `labels` (int64 [N], negative:
    left out), and the gradients of sum_n weight[n] loss[n] (weight None: the mean over the rows that count). Phi [N, K]
    and W [C, K] are float32 or bfloat16 with unit column stride; gradients have their type. Buffers that are not given are
    allocated."""
    ld_phi, ld_w = _matrix(Phi, "Phi"), _matrix(W, "W", dtype=Phi.dtype)
    N, K = Phi.shape
    C, columns = W.shape
    if columns != K:
        raise ValueError("Phi and W need the same number of columns")
    if _dev(labels, torch.int64, "labels").shape != (N,):
        raise ValueError("labels must have shape [N]")
    if weight is not None and _dev(weight, torch.float32, "weight").shape != (N,):
        raise ValueError("weight must have shape [N]")
    if loss is None:
        loss = _empty_on(stream, N, dtype=torch.float32, device=Phi.device)
    elif _dev(loss, torch.float32, "loss").shape != (N,):
        raise ValueError("loss must have shape [N]")
    ld_dphi = ld_dw = 0
    if need_dPhi:
        if dPhi is None:
            dPhi = _empty_on(stream, (N, K), dtype=Phi.dtype, device=Phi.device)
        ld_dphi = _matrix(dPhi, "dPhi", Phi.dtype, (N, K))
    if need_dW:
        if dW is None:
            dW = _empty_on(stream, (C, K), dtype=Phi.dtype, device=Phi.device)
        ld_dw = _matrix(dW, "dW", Phi.dtype, (C, K))
    lib = load_library()
    shp = _XentShape(N, K, C, ld_phi, ld_w, ld_dphi, ld_dw, _BF16[Phi.dtype], (_DPHI if need_dPhi else 0) | (_DW if need_dW else 0))
    if workspace is None:
        rec = ctypes.c_size_t(0)
        _check(lib.rfsf_softmax_xent_workspace_bytes(ctypes.byref(shp), ctypes.byref(rec), None))
        workspace = _empty_on(stream, int(rec.value), dtype=torch.uint8, device=Phi.device)
    workspace = _dev(workspace, torch.uint8, "workspace")
    _check(lib.rfsf_softmax_xent(ctypes.byref(shp), Phi.data_ptr(), W.data_ptr(), labels.data_ptr(),
                                 None if weight is None else weight.data_ptr(), loss.data_ptr(),
                                 dPhi.data_ptr() if need_dPhi else None, dW.data_ptr() if need_dW else None,
                                 workspace.data_ptr(), workspace.numel(), _stream_ptr(stream)))
    return loss, dPhi if need_dPhi else None, dW if need_dW else None


class RfsfAdamW:
    """AdamW over many tensors, with states of 32 bits or of 8 (256 numbers to a scale).

    params: float32 tensors, contiguous, on the device, updated in place by step(); the optimizer keeps views of their memory, so that
    a parameter whose `.data` is replaced later is not followed. copies: bfloat16 tensors of the same shapes that receive the updated
    parameters. state: the states' tensors to use, a dict of lists `m`, `v` (float32, or int8 and uint8) and with 8 bits `m_scale`,
    `v_scale` (float32, ceil(n / 256) each); fresh ones if None. `self.state` holds them in the same form."""

    BLOCK = 256

    def __init__(self, params: Sequence[torch.Tensor], state_bits: int = 32, state: Optional[dict] = None,
                 copies: Optional[Sequence[torch.Tensor]] = None):
        if state_bits not in (8, 32):
            raise ValueError("state_bits must be 8 or 32")
        self.params = [_dev(p, torch.float32, "params").detach() for p in params]
        self.state_bits = state_bits
        eight = state_bits == 8
        types = {"m": torch.int8 if eight else torch.float32, "v": torch.uint8 if eight else torch.float32}
        if eight:
            types.update(m_scale=torch.float32, v_scale=torch.float32)

        def size(name, p):
            return (p.numel() + self.BLOCK - 1) // self.BLOCK if name.endswith("scale") else p.numel()

        if state is None:
            state = {k: [torch.zeros(size(k, p), dtype=t, device=p.device) for p in self.params] for k, t in types.items()}
        if set(state) != set(types):
            raise ValueError(f"state must hold {sorted(types)}")
        for k, t in types.items():
            if len(state[k]) != len(self.params):
                raise ValueError(f"state[{k!r}] must hold a tensor for each parameter")
            for s, p in zip(state[k], self.params):
                if _dev(s, t, f"state[{k!r}]").numel() != size(k, p):
                    raise ValueError(f"state[{k!r}] does not fit its parameter")
        if copies is not None:
            if len(copies) != len(self.params):
                raise ValueError("copies must hold a tensor for each parameter")
            for c, p in zip(copies, self.params):
                if _dev(c, torch.bfloat16, "copies").numel() != p.numel():
                    raise ValueError("copies do not fit their parameters")
        state = {k: [t.detach() for t in state[k]] for k in types}
        self.state, self.copies = state, None if copies is None else [c.detach() for c in copies]
        # the tensors' descriptions (rfsf_adamw_tensor: eight words each); the gradients' addresses come with each step
        self._sizes = [p.numel() for p in self.params]
        self._words = np.zeros((len(self.params), 8), dtype=np.int64)
        columns = {0: self.params, 2: state["m"], 3: state["v"], 4: state.get("m_scale"), 5: state.get("v_scale"), 6: self.copies}
        for k, tensors in columns.items():
            if tensors:
                self._words[:, k] = [t.data_ptr() for t in tensors]
        self._words[:, 7] = self._sizes
        self._description = self._words.tobytes()

    def step(self, grads: Sequence[torch.Tensor], step: int, lr: float, betas=(0.9, 0.999), eps: float = 1e-8,
             weight_decay: float = 0.01, grad_scale: float = 1.0, stream: Optional[torch.cuda.Stream] = None) -> None:
        """One step, number `step` (from 1 on), with gradients of float32 or bfloat16, all of one type; they are multiplied by
        `grad_scale` first."""
        if len(grads) != len(self.params):
            raise ValueError("grads must hold a tensor for each parameter")
        if not grads:
            return
        dtype = grads[0].dtype
        if dtype not in _BF16:
            raise ValueError("grads must be float32 or bfloat16")
        words = array("q", self._description)                    # (a call's own: another thread may be in another step)
        words[1::8] = array("q", _addresses(grads, self._sizes, dtype, "grads"))
        config = _AdamwConfig(lr, betas[0], betas[1], eps, weight_decay, grad_scale, step, self.state_bits, _BF16[dtype])
        _check(load_library().rfsf_adamw_step(words.buffer_info()[0], len(grads), ctypes.byref(config), _stream_ptr(stream)))

    def moments(self, out=None, stream: Optional[torch.cuda.Stream] = None):
        """(m, v): lists of float32 tensors, what the states hold. 32 bits: the states themselves; 8 bits: the numbers that the codes
        stand for, in `out` (two such lists) or in new tensors."""
        if self.state_bits == 32:
            return self.state["m"], self.state["v"]
        if out is None:
            out = tuple([_empty_on(stream, p.shape, dtype=torch.float32, device=p.device) for p in self.params] for _ in range(2))
        if len(out) != 2 or any(len(tensors) != len(self.params) for tensors in out):
            raise ValueError("out must hold a tensor for each parameter, twice")
        places = [np.array(_addresses(tensors, self._sizes, torch.float32, "out"), dtype=np.int64) for tensors in out]
        _check(load_library().rfsf_adamw_moments(self._words.ctypes.data, len(self.params), places[0].ctypes.data, places[1].ctypes.data,
                                                 _stream_ptr(stream)))
        return out


def _addresses(tensors, sizes, dtype, name):
    """Addresses of contiguous device tensors of this type and these numbers of elements."""
    for t, n in zip(tensors, sizes):
        if t.dtype is not dtype or t.numel() != n or not t.is_cuda or not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous {dtype} device tensors of the parameters' sizes")
    return [t.data_ptr() for t in tensors]


def _code_room(K: int) -> int:
    return (K + 127) // 128 * 128


def _codes(codes: torch.Tensor, scales: torch.Tensor) -> int:
    """Row stride of codes [N, K] laid out as rfsf_int8_quantize does, whose rows exist up to their stride."""
    sizes, strides = codes.shape, codes.stride()
    if len(sizes) != 2 or codes.dtype is not torch.int8 or not codes.is_cuda or (strides[1] != 1 and sizes[1] > 1):
        raise ValueError("codes must be int8 [rows, cols] on the device with unit column stride")
    N, K = sizes
    ld = strides[0] if N > 1 else _code_room(K)
    if N > 0 and codes.storage_offset() + N * ld > codes.untyped_storage().nbytes():
        raise ValueError("rows of codes must have room for their columns rounded up to 128, as rfsf_int8_quantize lays them out")
    if _dev(scales, torch.float32, "scales").shape != (N,):
        raise ValueError("scales must have shape [rows]")
    return ld


def rfsf_int8_quantize(X: torch.Tensor, codes: Optional[torch.Tensor] = None, scales: Optional[torch.Tensor] = None,
                       stream: Optional[torch.cuda.Stream] = None):
    """(codes [N, K] int8, scales [N]): rows of X as 8-bit integers, X[n, k] about scales[n] * codes[n, k]. Rows of codes are a
    multiple of 128 bytes apart."""
    ldx = _matrix(X, "X")
    N, K = X.shape
    if codes is None:
        codes = _empty_on(stream, (N, _code_room(K)), dtype=torch.int8, device=X.device)[:, :K]
    if scales is None:
        scales = _empty_on(stream, N, dtype=torch.float32, device=X.device)
    if tuple(codes.shape) != (N, K):
        raise ValueError("codes must have X's shape")
    ld = _codes(codes, scales)
    _check(load_library().rfsf_int8_quantize(X.data_ptr(), _BF16[X.dtype], N, ldx, K, codes.data_ptr(), ld, scales.data_ptr(),
                                             _stream_ptr(stream)))
    return codes, scales


def rfsf_int8_gram_workspace_bytes(Nx: int, Ny: int, K: int):
    """(recommended_bytes, minimum_bytes) of scratch for rfsf_int8_gram."""
    rec, mn = ctypes.c_size_t(0), ctypes.c_size_t(0)
    _check(load_library().rfsf_int8_gram_workspace_bytes(Nx, Ny, K, ctypes.byref(rec), ctypes.byref(mn)))
    return int(rec.value), int(mn.value)


def rfsf_int8_gram(PhiX: torch.Tensor, codes: torch.Tensor, scales: torch.Tensor, K: Optional[torch.Tensor] = None,
                   workspace: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """K[i, j] = sum_k PhiX[i, k] Y[j, k] for rows Y held as 8-bit integers (rfsf_int8_quantize), PhiX's rows quantised on the
    way: the Gram with stored training features, or the scores of a classifier with quantised weights."""
    ldx, ldy = _matrix(PhiX, "PhiX"), _codes(codes, scales)
    Nx, ncols = PhiX.shape
    Ny, columns = codes.shape
    if columns != ncols:
        raise ValueError("PhiX and codes need the same number of columns")
    if K is None:
        K = _empty_on(stream, (Nx, Ny), dtype=torch.float32, device=PhiX.device)
    ldk = _matrix(K, "K", torch.float32, (Nx, Ny))
    if workspace is None:
        rec, _ = rfsf_int8_gram_workspace_bytes(Nx, Ny, ncols)
        workspace = _empty_on(stream, rec, dtype=torch.uint8, device=PhiX.device)
    workspace = _dev(workspace, torch.uint8, "workspace")
    _check(load_library().rfsf_int8_gram(PhiX.data_ptr(), _BF16[PhiX.dtype], Nx, ldx, codes.data_ptr(), scales.data_ptr(), Ny, ldy,
                                         ncols, K.data_ptr(), ldk, workspace.data_ptr(), workspace.numel(), _stream_ptr(stream)))
    return K
