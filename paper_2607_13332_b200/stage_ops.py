"""Torch-tensor sugar over the model operators of a stage (include/agora_stage.h): argument marshalling only, every step
runs in the library's kernels, on the current stream of the current device."""

from __future__ import annotations

from ctypes import byref
from typing import Optional, Tuple

import torch

from . import binding
from .runner import _TORCH_DTYPE, _ld, _ptr, _stream

_lib = binding.library()
_CODES = {torch.float32: binding.SSN_F32, torch.bfloat16: binding.SSN_BF16}


def _here(t: torch.Tensor, dtype: torch.dtype, what: str) -> torch.Tensor:
    """t, if it is a tensor of that type on the current device (the one whose stream the kernels are put on)."""
    if not t.is_cuda or t.get_device() != torch._C._cuda_getDevice():
        raise ValueError(f"{what}: expected a CUDA tensor on the current device")
    if t.dtype != dtype:
        raise ValueError(f"{what}: expected {dtype}, got {t.dtype}")
    return t


def _ints(t: Optional[torch.Tensor], n: int, what: str) -> int:
    """Address of n contiguous int32, or 0."""
    if t is None:
        return 0
    _here(t, torch.int32, what)
    if t.shape != (n,) or (n > 1 and t.stride(0) != 1):
        raise ValueError(f"{what}: expected {n} contiguous int32")
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
        self.c = binding.make_qk_rope(head_dim, rot, binding.DTYPES[dtype], binding.PAIRINGS[pairing], eps, _ptr(wq), _ptr(wk),
                                      _ptr(table), _ld(table) if table is not None else 0, max_pos, self.dev_status.data_ptr())

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
        if t.dtype != self.dtype or t.get_device() != torch._C._cuda_getDevice():
            raise ValueError(f"{what}: expected {self.dtype} on the current device")
        st = t.stride()
        if t.shape != (n, heads, self.head_dim) or st[2] != 1:
            raise ValueError(f"{what}: expected [{n}, {heads}, {self.head_dim}] with unit stride along the last dimension")
        return t.data_ptr(), st[0], st[1]

    def _empty(self, like: Optional[torch.Tensor]) -> Optional[torch.Tensor]:
        return None if like is None else torch.empty(like.shape, dtype=self.dtype, device=like.device)

    @staticmethod
    def _sizes(q: Optional[torch.Tensor], k: Optional[torch.Tensor]) -> Tuple[int, int, int]:
        some = q if q is not None else k
        if some is None:
            raise ValueError("neither queries nor keys")
        return some.shape[0], 0 if q is None else q.shape[1], 0 if k is None else k.shape[1]

    def forward(self, q: Optional[torch.Tensor], k: Optional[torch.Tensor], pos: Optional[torch.Tensor] = None, seq_len: int = 0,
                q_out: Optional[torch.Tensor] = None, k_out: Optional[torch.Tensor] = None):
        """q [n, q_heads, head_dim] and k [n, k_heads, head_dim] (views of any strides; either may be None), normed and rotated.
        Positions: pos int32[n], or t mod seq_len.  An output given may be its input.  Returns (q_out, k_out)."""
        n, qh, kh = self._sizes(q, k)
        if q_out is None:
            q_out = self._empty(q)
        if k_out is None:
            k_out = self._empty(k)
        st = _lib.stage_qk_rope_forward(byref(self.c), *self._heads(q, n, qh, "q"), qh, *self._heads(k, n, kh, "k"), kh,
                                        *self._heads(q_out, n, qh, "q_out"), *self._heads(k_out, n, kh, "k_out"),
                                        _ints(pos, n, "pos"), n, seq_len, _stream())
        binding.check(st, "stage_qk_rope_forward")
        return q_out, k_out

    def backward(self, dq: Optional[torch.Tensor], dk: Optional[torch.Tensor], q: Optional[torch.Tensor], k: Optional[torch.Tensor],
                 pos: Optional[torch.Tensor] = None, seq_len: int = 0, dq_in: Optional[torch.Tensor] = None,
                 dk_in: Optional[torch.Tensor] = None, gains: bool = True):
        """From the gradients of forward's outputs and forward's inputs: (dq_in, dk_in, dwq, dwk), the gains' gradients in
        fp32 [head_dim], or None without `gains`.  dq_in may be dq, dk_in dk."""
        n, qh, kh = self._sizes(q, k)
        if dq_in is None:
            dq_in = self._empty(q)
        if dk_in is None:
            dk_in = self._empty(k)
        some = q if q is not None else k
        dwq = dwk = None
        ws, nbytes = 0, 0
        if gains:
            nbytes = _lib.stage_qk_rope_workspace_bytes(byref(self.c), n, qh, kh)
            dw = torch.empty((2, self.head_dim), dtype=torch.float32, device=some.device)
            dwq, dwk = dw[0], dw[1]
            scratch = torch.empty(nbytes, dtype=torch.uint8, device=some.device)
            ws = scratch.data_ptr()
        st = _lib.stage_qk_rope_backward(byref(self.c), *self._heads(dq, n, qh, "dq"), *self._heads(dk, n, kh, "dk"),
                                         *self._heads(q, n, qh, "q"), qh, *self._heads(k, n, kh, "k"), kh,
                                         *self._heads(dq_in, n, qh, "dq_in"), *self._heads(dk_in, n, kh, "dk_in"), _ptr(dwq),
                                         _ptr(dwk), _ints(pos, n, "pos"), n, seq_len, ws, nbytes, _stream())
        binding.check(st, "stage_qk_rope_backward")
        return dq_in, dk_in, dwq, dwk


# ---- loss against a teacher's top logits --------------------------------------------------------------------------------------
def _distill(logits: torch.Tensor, ids: torch.Tensor, top: torch.Tensor, weight: Optional[torch.Tensor], temperature: float,
             dlogits: Optional[torch.Tensor], dev_status: Optional[torch.Tensor]) -> torch.Tensor:
    if logits.dtype not in _CODES:
        raise ValueError("logits: expected fp32 or bf16")
    n, vocab = _here(logits, logits.dtype, "logits").shape
    if _here(ids, torch.int32, "ids").shape != _here(top, torch.float32, "top").shape or ids.dim() != 2 or ids.shape[0] != n:
        raise ValueError(f"ids, top: expected [{n}, top_k] each")
    if weight is not None and (_here(weight, torch.float32, "weight").shape != (n,) or not weight.is_contiguous()):
        raise ValueError(f"weight: expected {n} contiguous fp32")
    if dlogits is not None and _here(dlogits, logits.dtype, "dlogits").shape != logits.shape:
        raise ValueError("dlogits: expected the shape of the logits")
    _ints(dev_status, 1, "dev_status")
    loss = torch.empty(n, dtype=torch.float32, device=logits.device)
    st = _lib.stage_distill_loss(logits.data_ptr(), _ld(logits), _CODES[logits.dtype], n, vocab, ids.data_ptr(), _ld(ids),
                                 top.data_ptr(), _ld(top), ids.shape[1], _ptr(weight), temperature, loss.data_ptr(), _ptr(dlogits),
                                 _ld(dlogits) if dlogits is not None else 0, _ptr(dev_status), _stream())
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
        dlogits = torch.empty((n, max(_ld(logits), vocab)), dtype=logits.dtype, device=logits.device)[:, :vocab]
    return _distill(logits, ids, top, weight, temperature, dlogits, dev_status), dlogits


# ---- products in 8-bit integers -----------------------------------------------------------------------------------------------
def int8_quantize(x: torch.Tensor, q: Optional[torch.Tensor] = None):
    """(q, scale): the rows of x (fp32 or bf16) in 8 bits with one fp32 scale each.  q made here has a leading dimension that
    is a multiple of 16, which is what int8_matmul's TMA kernels need."""
    if x.dtype not in _CODES:
        raise ValueError("x: expected fp32 or bf16")
    rows, cols = _here(x, x.dtype, "x").shape
    if q is None:
        q = torch.empty((rows, -(-cols // 16) * 16), dtype=torch.int8, device=x.device)
        if q.shape[1] != cols:
            q = q[:, :cols]
    elif _here(q, torch.int8, "q").shape != x.shape:
        raise ValueError("q: expected the shape of x")
    scale = torch.empty(rows, dtype=torch.float32, device=x.device)
    st = _lib.stage_int8_quantize(x.data_ptr(), _ld(x), _CODES[x.dtype], rows, cols, q.data_ptr(), _ld(q), scale.data_ptr(), _stream())
    binding.check(st, "stage_int8_quantize")
    return q, scale


def int8_matmul(xq: torch.Tensor, xs: torch.Tensor, wq: torch.Tensor, ws: torch.Tensor, dtype: str = "bf16",
                out: Optional[torch.Tensor] = None, dev_status: Optional[torch.Tensor] = None) -> torch.Tensor:
    """y [n, outer] of dtype = (xq [n, inner] times wq [outer, inner] transposed), scaled by xs [n] and ws [outer]."""
    n, inner = _here(xq, torch.int8, "xq").shape
    outer = _here(wq, torch.int8, "wq").shape[0]
    if wq.shape[1] != inner:
        raise ValueError(f"wq: expected [outer, {inner}]")
    for s, rows, what in ((xs, n, "xs"), (ws, outer, "ws")):
        if _here(s, torch.float32, what).shape != (rows,) or not s.is_contiguous():
            raise ValueError(f"{what}: expected {rows} contiguous fp32")
    if out is None:
        out = torch.empty((n, outer), dtype=_TORCH_DTYPE[dtype], device=xq.device)
    elif _here(out, _TORCH_DTYPE[dtype], "out").shape != (n, outer):
        raise ValueError(f"out: expected [{n}, {outer}]")
    _ints(dev_status, 1, "dev_status")
    st = _lib.stage_int8_matmul(xq.data_ptr(), _ld(xq), xs.data_ptr(), wq.data_ptr(), _ld(wq), ws.data_ptr(), n, inner, outer,
                                out.data_ptr(), _ld(out), binding.DTYPES[dtype], _ptr(dev_status), _stream())
    binding.check(st, "stage_int8_matmul")
    return out
