"""Torch-tensor sugar over the model operators of a stage (include/agora_stage.h): argument marshalling only, every step
runs in the library's kernels, on the current stream of the current device.

Autograd records none of these calls: outputs never require a gradient, whether inputs do or not.  A training step calls forward
and backward itself, or from a torch.autograd.Function of its own."""

from __future__ import annotations

from ctypes import addressof, byref
from typing import Optional, Tuple

import torch

from . import binding
from .runner import _TORCH_DTYPE, _ptr, _stream

_lib = binding.library()
# ctypes converts every argument of a call, which takes as long as a launch; one block of bytes does not
_forward, _forward_args = binding.packed("stage_qk_rope_forward")
_backward, _backward_args = binding.packed("stage_qk_rope_backward")
_loss, _loss_args = binding.packed("stage_distill_loss")
_quantize, _quantize_args = binding.packed("stage_int8_quantize")
_matmul, _matmul_args = binding.packed("stage_int8_matmul")
_CODES = {torch.float32: binding.SSN_F32, torch.bfloat16: binding.SSN_BF16}

# Calls of one token are shorter on the GPU than on the host, so every call asks each tensor once for its type, device, shape
# and strides, and makes its outputs with the cheapest allocation there is: (shape, strides, type) on the current device, 0.9 us
# against 1.8 to 3.5 us for torch.empty.  These are private names of torch, which another version may not have.
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", lambda device: torch.cuda.current_stream(device).cuda_stream)
try:
    _new = torch._C._dynamo.guards._empty_strided_cuda
except AttributeError:
    def _new(shape, strides, dtype):
        return torch.empty_strided(shape, strides, dtype=dtype, device="cuda")


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


def _matrix(t: torch.Tensor, dtype: torch.dtype, device: int, what: str) -> Tuple[int, int, int, int]:
    """(rows, columns, address, leading dimension) of a row-major matrix of that type on that device."""
    if t.get_device() != device:
        raise ValueError(f"{what}: expected a CUDA tensor on the current device")
    if t.dtype is not dtype:
        raise ValueError(f"{what}: expected {dtype}, got {t.dtype}")
    rows, cols = t.shape
    ld, unit = t.stride()
    if (unit != 1 and cols > 1) or (rows > 1 and ld < cols):
        raise ValueError(f"{what}: expected a row-major 2-D tensor (unit stride along the last dimension)")
    return rows, cols, t.data_ptr(), ld if rows > 1 else cols


def _vector(t: Optional[torch.Tensor], n: int, dtype: torch.dtype, what: str) -> int:
    """Address of n contiguous values of that type, or 0."""
    if t is None:
        return 0
    if _here(t, dtype, what).shape != (n,) or (n > 1 and t.stride(0) != 1):
        raise ValueError(f"{what}: expected {n} contiguous values")
    return t.data_ptr()


# Addresses of the status words of calls that are given none, by device
_words = {}


def _status(given: Optional[torch.Tensor], device: int) -> int:
    """Address of the status word of a call: the given one, or the library's own."""
    if given is not None:
        return _vector(given, 1, torch.int32, "dev_status")
    at = _words.get(device)
    if at is None:
        at = _lib.stage_status_word()
        if not at:
            raise RuntimeError("no status word on the current device")
        _words[device] = at
    return at


class _Word:
    """One int32 at a device address, as torch.as_tensor takes it."""

    def __init__(self, at: int):
        self.__cuda_array_interface__ = {"shape": (1,), "typestr": "<i4", "data": (at, False), "version": 3}


def take_status() -> int:
    """Read and clear the current device's status word of the losses and products that are given no dev_status (waits for the
    device): SSN_DEV_BAD_ID and SSN_DEV_TIMEOUT of every call in this process since the last read.  After SSN_DEV_TIMEOUT a
    product among them is invalid."""
    device = _current_device()
    torch.cuda.synchronize(device)
    word = torch.as_tensor(_Word(_status(None, device)), device=torch.device("cuda", device))
    v = int(word.item())
    word.zero_()
    torch.cuda.synchronize(device)      # cleared before a later call on any stream may set it
    return v


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
        self._ref, self._address = byref(self.c), addressof(self.c)
        self._workspace = {}

    def take_status(self) -> int:
        """Read and clear the device status word (synchronises): SSN_DEV_BAD_POS of every call since the last read."""
        v = int(self.dev_status.item())
        self.dev_status.zero_()
        return v

    def _rows(self, some: Optional[torch.Tensor]) -> int:
        """Number of tokens of the tensor that tells it; the operator's device has to be the current one."""
        if some is None:
            raise ValueError("neither queries nor keys")
        if _current_device() != self._device:     # its stream is the one that the kernel is put on
            raise ValueError("the current device is not the operator's")
        if some.dim() != 3:
            raise ValueError("expected [tokens, heads, head_dim]")
        return some.shape[0]

    def _heads(self, t: Optional[torch.Tensor], n: int, what: str, heads: int = -1):
        """(address, token stride, head stride, heads) of a [n, heads, head_dim] tensor, or of an absent one."""
        if t is None:
            if n * heads > 0:
                raise ValueError(f"{what} is missing")
            return 0, 0, 0, 0
        if t.dtype is not self.dtype or t.get_device() != self._device:
            raise ValueError(f"{what}: expected {self.dtype} on the operator's device")
        rows, count, d = t.shape
        if rows != n or d != self.head_dim or (count != heads and heads >= 0):
            raise ValueError(f"{what}: expected [{n}, {heads if heads >= 0 else 'heads'}, {self.head_dim}]")
        token, head, unit = t.stride()
        if unit != 1:
            raise ValueError(f"{what}: expected unit stride along the last dimension")
        return t.data_ptr(), token, head, count

    def _out(self, t: Optional[torch.Tensor], n: int, heads: int, absent: bool, what: str):
        """The output tensor, made here unless it is given, with its address, token stride and head stride."""
        if t is not None:
            return t, *self._heads(t, n, what, heads)[:3]
        if absent:
            return None, 0, 0, 0
        d = self.head_dim
        pitch = heads * d
        t = _new((n, heads, d), (pitch, d, 1), self.dtype)
        return t, t.data_ptr(), pitch, d

    def forward(self, q: Optional[torch.Tensor], k: Optional[torch.Tensor], pos: Optional[torch.Tensor] = None, seq_len: int = 0,
                q_out: Optional[torch.Tensor] = None, k_out: Optional[torch.Tensor] = None):
        """q [n, q_heads, head_dim] and k [n, k_heads, head_dim] (views of any strides; either may be None), normed and rotated.
        Positions: pos int32[n], or t mod seq_len.  An output given may be its input.  Returns (q_out, k_out)."""
        n = self._rows(k if q is None else q)
        qa, qt, qs, qh = self._heads(q, n, "q")
        ka, kt, ks, kh = self._heads(k, n, "k")
        q_out, qoa, qot, qos = self._out(q_out, n, qh, q is None, "q_out")
        k_out, koa, kot, kos = self._out(k_out, n, kh, k is None, "k_out")
        st = _forward(_forward_args(self._address, qa, qt, qs, qh, ka, kt, ks, kh, qoa, qot, qos, koa, kot, kos,
                                    _vector(pos, n, torch.int32, "pos"), n, seq_len, _raw_stream(self._device)))
        if st:
            binding.check(st, "stage_qk_rope_forward")
        return q_out, k_out

    def backward(self, dq: Optional[torch.Tensor], dk: Optional[torch.Tensor], q: Optional[torch.Tensor], k: Optional[torch.Tensor],
                 pos: Optional[torch.Tensor] = None, seq_len: int = 0, dq_in: Optional[torch.Tensor] = None,
                 dk_in: Optional[torch.Tensor] = None, gains: bool = True):
        """From the gradients of forward's outputs and forward's inputs: (dq_in, dk_in, dwq, dwk), the gains' gradients in
        fp32 [head_dim], or None without `gains`.  dq_in may be dq, dk_in dk."""
        n = self._rows(k if q is None else q)
        qa, qt, qs, qh = self._heads(q, n, "q")
        ka, kt, ks, kh = self._heads(k, n, "k")
        dqa, dqt, dqs, _ = self._heads(dq, n, "dq", qh)
        dka, dkt, dks, _ = self._heads(dk, n, "dk", kh)
        dq_in, dqoa, dqot, dqos = self._out(dq_in, n, qh, q is None, "dq_in")
        dk_in, dkoa, dkot, dkos = self._out(dk_in, n, kh, k is None, "dk_in")
        dwq = dwk = scratch = None
        nbytes = 0
        if gains:
            d = self.head_dim
            nbytes = self._workspace.get((qh, kh))      # does not depend on the number of tokens
            if nbytes is None:
                nbytes = self._workspace[qh, kh] = _lib.stage_qk_rope_workspace_bytes(self._ref, 1, qh, kh)
            dwq, dwk = _new((d,), (1,), torch.float32), _new((d,), (1,), torch.float32)
            scratch = _new((nbytes,), (1,), torch.uint8)      # one per call: captured calls share none
        st = _backward(_backward_args(self._address, dqa, dqt, dqs, dka, dkt, dks, qa, qt, qs, qh, ka, kt, ks, kh, dqoa, dqot, dqos,
                                      dkoa, dkot, dkos, _ptr(dwq), _ptr(dwk), _vector(pos, n, torch.int32, "pos"), n, seq_len,
                                      _ptr(scratch), nbytes, _raw_stream(self._device)))
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
    device = _current_device()
    n, vocab, at, ldl = _matrix(logits, dtype, device, "logits")
    rows, top_k, ids_at, ldi = _matrix(ids, torch.int32, device, "ids")
    top_rows, top_cols, top_at, ldt = _matrix(top, torch.float32, device, "top")
    if rows != n or top_rows != n or top_cols != top_k:
        raise ValueError(f"ids, top: expected [{n}, top_k] each")
    out, ldd = 0, 0
    if dlogits is not None:
        out_rows, out_cols, out, ldd = _matrix(dlogits, dtype, device, "dlogits")
        if out_rows != n or out_cols != vocab:
            raise ValueError("dlogits: expected the shape of the logits")
    loss = _new((n,), (1,), torch.float32)
    st = _loss(_loss_args(at, ldl, code, n, vocab, ids_at, ldi, top_at, ldt, top_k, _vector(weight, n, torch.float32, "weight"),
                          temperature, loss.data_ptr(), out, ldd, _status(dev_status, device), _raw_stream(device)))
    if st:
        binding.check(st, "stage_distill_loss")
    return loss


def distill_loss(logits: torch.Tensor, ids: torch.Tensor, top: torch.Tensor, weight: Optional[torch.Tensor] = None,
                 temperature: float = 1.0, dev_status: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Loss [n] fp32 of logits [n, vocab] against the teacher's top logits top [n, k] fp32 at ids [n, k] int32 (-1: padding):
    weight times temperature^2 times the divergence of the student's softmax from the teacher's over its entries (with k = 1 and
    temperature 1 the cross entropy of the targets ids).  Ids outside
    the vocabulary set SSN_DEV_BAD_ID in dev_status (int32 [1]), or in the word that take_status() reads."""
    return _distill(logits, ids, top, weight, temperature, None, dev_status)


def distill_loss_grad(logits: torch.Tensor, ids: torch.Tensor, top: torch.Tensor, weight: Optional[torch.Tensor] = None,
                      temperature: float = 1.0, dlogits: Optional[torch.Tensor] = None, dev_status: Optional[torch.Tensor] = None):
    """distill_loss and the gradient of its sum with respect to the logits, in one pass: (loss, dlogits).  dlogits may be the
    logits; made here, its rows stand as close together as keeps them as far from 16-byte boundaries as the logits' rows."""
    if dlogits is None:
        n, vocab = logits.shape
        size = logits.element_size()
        ld = _pitch(_here(logits, logits.dtype, "logits"), n, vocab)      # of a view, any number of rows
        ld = vocab + (ld - vocab) % (16 // size)
        at = logits.data_ptr() % 16 // size
        if at == 0:
            dlogits = _new((n, vocab), (ld, 1), logits.dtype)
        else:
            dlogits = _new((at + max(n - 1, 0) * ld + vocab,), (1,), logits.dtype).as_strided((n, vocab), (ld, 1), at)
    return _distill(logits, ids, top, weight, temperature, dlogits, dev_status), dlogits


# ---- products in 8-bit integers -----------------------------------------------------------------------------------------------
def int8_quantize(x: torch.Tensor, q: Optional[torch.Tensor] = None):
    """(q, scale): the rows of x (fp32 or bf16) in 8 bits with one fp32 scale each.  q made here has a leading dimension that
    is a multiple of 16, which is what int8_matmul's TMA kernels need."""
    code = _CODES.get(x.dtype)
    if code is None:
        raise ValueError("x: expected fp32 or bf16")
    device = _current_device()
    rows, cols, at, ldx = _matrix(x, x.dtype, device, "x")
    if q is None:
        ldq = cols + (-cols & 15)
        q = _new((rows, cols), (ldq, 1), torch.int8)
        q_at = q.data_ptr()
    else:
        q_rows, q_cols, q_at, ldq = _matrix(q, torch.int8, device, "q")
        if q_rows != rows or q_cols != cols:
            raise ValueError("q: expected the shape of x")
    scale = _new((rows,), (1,), torch.float32)
    st = _quantize(_quantize_args(at, ldx, code, rows, cols, q_at, ldq, scale.data_ptr(), _raw_stream(device)))
    if st:
        binding.check(st, "stage_int8_quantize")
    return q, scale


def int8_matmul(xq: torch.Tensor, xs: torch.Tensor, wq: torch.Tensor, ws: torch.Tensor, dtype: str = "bf16",
                out: Optional[torch.Tensor] = None, dev_status: Optional[torch.Tensor] = None) -> torch.Tensor:
    """y [n, outer] of dtype = (xq [n, inner] times wq [outer, inner] transposed), scaled by xs [n] and ws [outer].  A product that
    went wrong on the GPU sets SSN_DEV_TIMEOUT in dev_status (int32 [1]), or in the word that take_status() reads."""
    device = _current_device()
    n, inner, x_at, ldx = _matrix(xq, torch.int8, device, "xq")
    outer, depth, w_at, ldw = _matrix(wq, torch.int8, device, "wq")
    if depth != inner:
        raise ValueError(f"wq: expected [outer, {inner}]")
    kind = _TORCH_DTYPE[dtype]
    if out is None:
        out, ldy = _new((n, outer), (outer, 1), kind), outer
        y_at = out.data_ptr()
    else:
        rows, cols, y_at, ldy = _matrix(out, kind, device, "out")
        if rows != n or cols != outer:
            raise ValueError(f"out: expected [{n}, {outer}]")
    st = _matmul(_matmul_args(x_at, ldx, _vector(xs, n, torch.float32, "xs"), w_at, ldw, _vector(ws, outer, torch.float32, "ws"),
                              n, inner, outer, y_at, ldy, _CODES[kind], _status(dev_status, device), _raw_stream(device)))
    if st:
        binding.check(st, "stage_int8_matmul")
    return out
