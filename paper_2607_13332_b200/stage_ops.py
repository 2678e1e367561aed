"""Torch-tensor sugar over the model operators of a stage (include/agora_stage.h): argument marshalling only, every step
runs in the library's kernels, on the current stream of the current device."""

from __future__ import annotations

from ctypes import byref
from typing import Optional, Tuple

import torch

from . import binding
from .runner import _TORCH_DTYPE, _ptr, _stream

_lib = binding.library()
_CODES = {torch.float32: binding.SSN_F32, torch.bfloat16: binding.SSN_BF16}

# Calls of one token are shorter on the GPU than on the host, so every call asks each tensor once for its type, device, shape
# and strides, and makes its outputs with the cheapest allocation there is: (shape, strides, type) on the current device, 0.9 us
# against 1.8 to 3.5 us for torch.empty.
_current_device = torch._C._cuda_getDevice
_new = torch._C._dynamo.guards._empty_strided_cuda


def _here(t: torch.Tensor, dtype: torch.dtype, what: str) -> torch.Tensor:
    """t, if it is a tensor of that type on the current device (the one whose stream the kernels are put on)."""
    if t.get_device() != _current_device():     # -1 for a tensor on the host
        raise ValueError(f"{what}: expected a CUDA tensor on the current device")
    if t.dtype != dtype:
        raise ValueError(f"{what}: expected {dtype}, got {t.dtype}")
    return t


def _pitch(t: torch.Tensor, rows: int, cols: int) -> int:
    """Leading dimension of a row-major [rows, cols] tensor, in elements."""
    ld, unit = t.stride()
    if (unit != 1 and cols > 1) or (rows > 1 and ld < cols):     # rows that share elements have no leading dimension
        raise ValueError("expected a row-major 2-D tensor (unit stride along the last dimension)")
    return ld if rows > 1 else cols


def _vector(t: Optional[torch.Tensor], n: int, dtype: torch.dtype, what: str) -> int:
    """Address of n contiguous values of that type, or 0."""
    if t is None:
        return 0
    if _here(t, dtype, what).shape != (n,) or (n > 1 and t.stride(0) != 1):
        raise ValueError(f"{what}: expected {n} contiguous values")
    return t.data_ptr()


def rope_table(max_pos: int, rot_dim: int, theta: float = 10000.0, device: str = "cuda") -> torch.Tensor:
    """[max_pos, rot_dim] fp32 rotation table: rot_dim / 2 cosines, then as many sines, of every position's angles."""
    table = torch.empty((max_pos, rot_dim), dtype=torch.float32, device=device)
    _here(table, torch.float32, "rope_table")
    binding.stage_rope_table(table.data_ptr(), rot_dim, max_pos, rot_dim, theta, _stream())
    return table


class QKNormRope:
    """What the blocks of a stage share to norm and rotate their query and key heads: gains [head_dim] (None: ones) and the
    rotation table [max_pos, rot_dim] (None: no rotation).  pairing: "halves" (column i with i + rot_dim / 2) or "adjacent"."""

    def __init__(self, dtype: str, head_dim: int, wq: Optional[torch.Tensor] = None, wk: Optional[torch.Tensor] = None,
                 table: Optional[torch.Tensor] = None, eps: float = 1e-6, pairing: str = "halves", device: str = "cuda"):
        self.dtype, self.head_dim = _TORCH_DTYPE[dtype], head_dim
        self.wq, self.wk, self.table = wq, wk, table
        for w in (wq, wk):
            if w is not None and (_here(w, self.dtype, "gain").shape != (head_dim,) or not w.is_contiguous()):
                raise ValueError(f"gain: expected {head_dim} contiguous values")
        rot, max_pos = 0, 0
        if table is not None:
            max_pos, rot = _here(table, torch.float32, "table").shape
        self.dev_status = torch.zeros(1, dtype=torch.int32, device=device)
        self._device = _here(self.dev_status, torch.int32, "device").get_device()     # calls are for this device alone
        self.c = binding.make_qk_rope(head_dim, rot, binding.DTYPES[dtype], binding.PAIRINGS[pairing], eps, _ptr(wq), _ptr(wk),
                                      _ptr(table), _pitch(table, max_pos, rot) if table is not None else 0, max_pos, self.dev_status.data_ptr())
        self._ref = byref(self.c)
        self._workspace = {}

    def take_status(self) -> int:
        """Read and clear the device status word (synchronises): SSN_DEV_BAD_POS of every call since the last read."""
        v = int(self.dev_status.item())
        self.dev_status.zero_()
        return v

    def _heads(self, t: Optional[torch.Tensor], n: int, heads: int, what: str):
        """(address, token stride, head stride) of a [n, heads, head_dim] tensor, or of an absent one."""
        if t is None:
            if n * heads:
                raise ValueError(f"{what} is missing")
            return 0, 0, 0
        if t.dtype != self.dtype or t.get_device() != self._device:
            raise ValueError(f"{what}: expected {self.dtype} on the operator's device")
        if t.shape != (n, heads, self.head_dim):
            raise ValueError(f"{what}: expected [{n}, {heads}, {self.head_dim}]")
        token, head, unit = t.stride()
        if unit != 1:
            raise ValueError(f"{what}: expected unit stride along the last dimension")
        return t.data_ptr(), token, head

    def _out(self, t: Optional[torch.Tensor], n: int, heads: int, absent: bool, what: str):
        """The output tensor, made here unless it is given, and its (address, token stride, head stride)."""
        if t is not None:
            return t, self._heads(t, n, heads, what)
        if absent:
            return None, (0, 0, 0)
        d = self.head_dim
        t = _new((n, heads, d), (heads * d, d, 1), self.dtype)
        return t, (t.data_ptr(), heads * d, d)

    def _sizes(self, q: Optional[torch.Tensor], k: Optional[torch.Tensor]) -> Tuple[int, int, int]:
        some = q if q is not None else k
        if some is None:
            raise ValueError("neither queries nor keys")
        if some.dim() != 3:
            raise ValueError("expected [tokens, heads, head_dim]")
        if _current_device() != self._device:     # its stream is the one that the kernel is put on
            raise ValueError("the current device is not the operator's")
        return some.shape[0], 0 if q is None else q.shape[1], 0 if k is None else k.shape[1]

    def forward(self, q: Optional[torch.Tensor], k: Optional[torch.Tensor], pos: Optional[torch.Tensor] = None, seq_len: int = 0,
                q_out: Optional[torch.Tensor] = None, k_out: Optional[torch.Tensor] = None):
        """q [n, q_heads, head_dim] and k [n, k_heads, head_dim] (views of any strides; either may be None), normed and rotated.
        Positions: pos int32[n], or t mod seq_len.  An output given may be its input.  Returns (q_out, k_out)."""
        n, qh, kh = self._sizes(q, k)
        qa, ka = self._heads(q, n, qh, "q"), self._heads(k, n, kh, "k")
        q_out, qo = self._out(q_out, n, qh, q is None, "q_out")
        k_out, ko = self._out(k_out, n, kh, k is None, "k_out")
        st = _lib.stage_qk_rope_forward(self._ref, *qa, qh, *ka, kh, *qo, *ko, _vector(pos, n, torch.int32, "pos"), n, seq_len,
                                        _stream())
        if st:
            binding.check(st, "stage_qk_rope_forward")
        return q_out, k_out

    def backward(self, dq: Optional[torch.Tensor], dk: Optional[torch.Tensor], q: Optional[torch.Tensor], k: Optional[torch.Tensor],
                 pos: Optional[torch.Tensor] = None, seq_len: int = 0, dq_in: Optional[torch.Tensor] = None,
                 dk_in: Optional[torch.Tensor] = None, gains: bool = True):
        """From the gradients of forward's outputs and forward's inputs: (dq_in, dk_in, dwq, dwk), the gains' gradients in
        fp32 [head_dim], or None without `gains`.  dq_in may be dq, dk_in dk."""
        n, qh, kh = self._sizes(q, k)
        dqa, dka = self._heads(dq, n, qh, "dq"), self._heads(dk, n, kh, "dk")
        qa, ka = self._heads(q, n, qh, "q"), self._heads(k, n, kh, "k")
        dq_in, dqo = self._out(dq_in, n, qh, q is None, "dq_in")
        dk_in, dko = self._out(dk_in, n, kh, k is None, "dk_in")
        dwq = dwk = scratch = None
        nbytes = 0
        if gains:
            d = self.head_dim
            nbytes = self._workspace.get((qh, kh))      # does not depend on the number of tokens
            if nbytes is None:
                nbytes = self._workspace[qh, kh] = _lib.stage_qk_rope_workspace_bytes(self._ref, 1, qh, kh)
            dwq, dwk = _new((d,), (1,), torch.float32), _new((d,), (1,), torch.float32)
            scratch = _new((nbytes,), (1,), torch.uint8)      # one per call: captured calls share none
        st = _lib.stage_qk_rope_backward(self._ref, *dqa, *dka, *qa, qh, *ka, kh, *dqo, *dko, _ptr(dwq), _ptr(dwk),
                                         _vector(pos, n, torch.int32, "pos"), n, seq_len, _ptr(scratch), nbytes, _stream())
        if st:
            binding.check(st, "stage_qk_rope_backward")
        return dq_in, dk_in, dwq, dwk


# ---- loss against a teacher's top logits --------------------------------------------------------------------------------------
def _distill(logits: torch.Tensor, ids: torch.Tensor, top: torch.Tensor, weight: Optional[torch.Tensor], temperature: float,
             dlogits: Optional[torch.Tensor], dev_status: Optional[torch.Tensor]) -> torch.Tensor:
    dtype = logits.dtype
    code = _CODES.get(dtype)
    if code is None:
        raise ValueError("logits: expected fp32 or bf16")
    n, vocab = _here(logits, dtype, "logits").shape
    rows, top_k = _here(ids, torch.int32, "ids").shape
    if _here(top, torch.float32, "top").shape != (rows, top_k) or rows != n:
        raise ValueError(f"ids, top: expected [{n}, top_k] each")
    out, ldd = 0, 0
    if dlogits is not None:
        if _here(dlogits, dtype, "dlogits").shape != (n, vocab):
            raise ValueError("dlogits: expected the shape of the logits")
        out, ldd = dlogits.data_ptr(), _pitch(dlogits, n, vocab)
    loss = _new((n,), (1,), torch.float32)
    st = _lib.stage_distill_loss(logits.data_ptr(), _pitch(logits, n, vocab), code, n, vocab, ids.data_ptr(), _pitch(ids, n, top_k),
                                 top.data_ptr(), _pitch(top, n, top_k), top_k, _vector(weight, n, torch.float32, "weight"), temperature,
                                 loss.data_ptr(), out, ldd, _vector(dev_status, 1, torch.int32, "dev_status"), _stream())
    if st:
        binding.check(st, "stage_distill_loss")
    return loss


def distill_loss(logits: torch.Tensor, ids: torch.Tensor, top: torch.Tensor, weight: Optional[torch.Tensor] = None,
                 temperature: float = 1.0, dev_status: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Loss [n] fp32 of logits [n, vocab] against the teacher's top logits top [n, k] fp32 at ids [n, k] int32 (-1: padding):
    weight times temperature^2 times the divergence of the student's softmax from the teacher's over its entries."""
    return _distill(logits, ids, top, weight, temperature, None, dev_status)


def distill_loss_grad(logits: torch.Tensor, ids: torch.Tensor, top: torch.Tensor, weight: Optional[torch.Tensor] = None,
                      temperature: float = 1.0, dlogits: Optional[torch.Tensor] = None, dev_status: Optional[torch.Tensor] = None):
    """distill_loss and the gradient of its sum with respect to the logits, in one pass: (loss, dlogits).  dlogits may be the
    logits; made here, it has the logits' leading dimension."""
    if dlogits is None:
        n, vocab = logits.shape
        dlogits = _new((n, vocab), (_pitch(_here(logits, logits.dtype, "logits"), n, vocab), 1), logits.dtype)
    return _distill(logits, ids, top, weight, temperature, dlogits, dev_status), dlogits


# ---- products in 8-bit integers -----------------------------------------------------------------------------------------------
def int8_quantize(x: torch.Tensor, q: Optional[torch.Tensor] = None):
    """(q, scale): the rows of x (fp32 or bf16) in 8 bits with one fp32 scale each.  q made here has a leading dimension that
    is a multiple of 16, which is what int8_matmul's TMA kernels need."""
    code = _CODES.get(x.dtype)
    if code is None:
        raise ValueError("x: expected fp32 or bf16")
    rows, cols = _here(x, x.dtype, "x").shape
    if q is None:
        ldq = cols + (-cols & 15)
        q = _new((rows, cols), (ldq, 1), torch.int8)
    elif _here(q, torch.int8, "q").shape != (rows, cols):
        raise ValueError("q: expected the shape of x")
    else:
        ldq = _pitch(q, rows, cols)
    scale = _new((rows,), (1,), torch.float32)
    st = _lib.stage_int8_quantize(x.data_ptr(), _pitch(x, rows, cols), code, rows, cols, q.data_ptr(), ldq, scale.data_ptr(), _stream())
    if st:
        binding.check(st, "stage_int8_quantize")
    return q, scale


def int8_matmul(xq: torch.Tensor, xs: torch.Tensor, wq: torch.Tensor, ws: torch.Tensor, dtype: str = "bf16",
                out: Optional[torch.Tensor] = None, dev_status: Optional[torch.Tensor] = None) -> torch.Tensor:
    """y [n, outer] of dtype = (xq [n, inner] times wq [outer, inner] transposed), scaled by xs [n] and ws [outer]."""
    n, inner = _here(xq, torch.int8, "xq").shape
    outer, depth = _here(wq, torch.int8, "wq").shape
    if depth != inner:
        raise ValueError(f"wq: expected [outer, {inner}]")
    kind = _TORCH_DTYPE[dtype]
    if out is None:
        out, ldy = _new((n, outer), (outer, 1), kind), outer
    elif _here(out, kind, "out").shape != (n, outer):
        raise ValueError(f"out: expected [{n}, {outer}]")
    else:
        ldy = _pitch(out, n, outer)
    st = _lib.stage_int8_matmul(xq.data_ptr(), _pitch(xq, n, inner), _vector(xs, n, torch.float32, "xs"), wq.data_ptr(),
                                _pitch(wq, outer, inner), _vector(ws, outer, torch.float32, "ws"), n, inner, outer, out.data_ptr(), ldy,
                                _CODES[kind], _vector(dev_status, 1, torch.int32, "dev_status"), _stream())
    if st:
        binding.check(st, "stage_int8_matmul")
    return out
