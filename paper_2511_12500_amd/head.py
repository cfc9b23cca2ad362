"""Host-side conveniences over the C ABI for the output head: a shard of 4-bit
weights, and the outputs and workspace of token log probabilities and of the
distillation loss over rows of logits.  Argument marshalling only."""
from __future__ import annotations

import torch

from . import _binding as B
from .heap import current_stream

_DTYPES = {torch.float16: B.F16, torch.bfloat16: B.BF16, torch.float32: B.F32}


class W4Weight:
    """A shard of 4-bit weights: column n of the product is
    sum_k x_k (q[n, k] - zero[n, k // group]) scale[n, k // group].

    ``q``: uint8 [N, K/2], two consecutive k to a byte, the even one in the low
    bits; ``scales``: float16 or bfloat16 [N, ceil(K / group)]; ``zeros``: uint8
    of the same shape, or None for 8 everywhere.  The tensors are kept, not
    copied."""

    def __init__(self, q: torch.Tensor, scales: torch.Tensor, zeros: torch.Tensor | None = None,
                 group: int = 128):
        if q.dtype != torch.uint8 or q.dim() != 2 or (zeros is not None and
                                                      zeros.dtype != torch.uint8):
            raise TypeError("q must be a uint8 matrix, zeros uint8")
        if scales.dtype not in (torch.float16, torch.bfloat16):
            raise TypeError("scales must be float16 or bfloat16")
        self.N, self.K, self.group, self.dtype = q.shape[0], 2 * q.shape[1], group, scales.dtype
        if group not in (32, 64, 128):
            raise ValueError("group must be 32, 64 or 128")
        shape = (self.N, -(-self.K // group))
        tensors = [q, scales] + ([] if zeros is None else [zeros])
        if any(tuple(t.shape) != shape for t in tensors[1:]):
            raise ValueError(f"scales and zeros must be {list(shape)}")
        self.device = q.get_device()
        if not all(t.is_cuda and t.get_device() == self.device and t.is_contiguous()
                   for t in tensors):
            raise ValueError("q, scales and zeros must be contiguous tensors on one GPU")
        self.q, self.scales, self.zeros = q, scales, zeros
        self.pointers = (q.data_ptr(), scales.data_ptr(),
                         None if zeros is None else zeros.data_ptr())


def _matrix(t: torch.Tensor, name: str, rows: int, cols: int, dtype: torch.dtype,
            device: int) -> int:
    """Row stride in elements of a matrix on the device with contiguous rows."""
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}")
    if t.get_device() != device or t.shape != (rows, cols):
        raise ValueError(f"{name} must be a [{rows}, {cols}] tensor on cuda:{device}")
    if cols > 1 and t.stride(1) != 1:
        raise ValueError(f"{name} must have contiguous rows")
    ld = t.stride(0) if rows > 1 else cols
    if ld < cols:
        raise ValueError(f"{name}: rows must not overlap")
    return ld


def _vector(t: torch.Tensor | None, name: str, shape: tuple, dtype: torch.dtype, device: int):
    """Address of a contiguous tensor on the device (None for None)."""
    if t is None:
        return None
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}")
    if t.get_device() != device or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous tensor {list(shape)} on cuda:{device}")
    return t.data_ptr()


class _Rows:
    """What the operators over rows of logits share: sizes, type and the
    workspace, which a call needs where rows are long enough to be split (more
    than 4096 vectors of 16 bytes).  Calls on one object must not overlap in
    time."""

    def __init__(self, rows: int, vocab: int, dtype: torch.dtype, top: int, scale: float,
                 device: int):
        if dtype not in _DTYPES:
            raise TypeError("dtype must be float16, bfloat16 or float32")
        self.rows, self.vocab, self.dtype, self.scale = rows, vocab, dtype, scale
        self.device = device
        self._dt = _DTYPES[dtype]
        need = B.symtile_logits_workspace_bytes(device, rows, vocab, self._dt, top)
        self.ws = torch.zeros(need, dtype=torch.uint8, device=f"cuda:{device}") if need else None
        if need and not torch.cuda.is_current_stream_capturing():
            # the calls may come on any stream, and find the workspace zero on each (a
            # capture's calls follow the zeroing in it)
            torch.cuda.current_stream(device).synchronize()
        self._ws = (self.ws.data_ptr(), need) if need else (None, 0)

    def _new(self, *shape, dtype=torch.float32) -> torch.Tensor:
        return torch.empty(shape, dtype=dtype, device=f"cuda:{self.device}")

    def _matrices(self, logits, dlogits):
        ld = _matrix(logits, "logits", self.rows, self.vocab, self.dtype, self.device)
        ld_grad = 0 if dlogits is None else _matrix(dlogits, "dlogits", self.rows, self.vocab,
                                                    self.dtype, self.device)
        return ld, ld_grad

    def _stream(self, stream):
        return current_stream(self.device) if stream is None else stream


class TokenLogprobs(_Rows):
    """Log probabilities of given tokens, entropies and the ``top`` most likely
    tokens of ``rows`` rows of ``scale`` * logits over ``vocab`` tokens.

    Outputs, written by every call: ``logprob``, ``entropy`` [rows], ``stats``
    [rows, 2] (largest logit, log-sum-exp less scale times it), ``top_ids``
    (int64) and ``top_logprobs`` [rows, top], the largest first and equal ones by
    ascending id."""

    def __init__(self, rows: int, vocab: int, dtype: torch.dtype, top: int = 0,
                 scale: float = 1.0, device: int = 0):
        super().__init__(rows, vocab, dtype, top, scale, device)
        self.top = top
        self.logprob, self.entropy = self._new(rows), self._new(rows)
        self.stats = self._new(rows, 2)
        self.top_ids = self._new(rows, top, dtype=torch.int64)
        self.top_logprobs = self._new(rows, top)
        self._out = (self.entropy.data_ptr(), self.stats.data_ptr(), top,
                     self.top_ids.data_ptr() or None, self.top_logprobs.data_ptr() or None)

    def lse(self) -> torch.Tensor:
        """log sum_v exp(scale * logits_v) of the last call's rows."""
        return self.stats[:, 0] * self.scale + self.stats[:, 1]

    def _grads(self, *grads):
        return [_vector(g, n, (self.rows,), torch.float32, self.device)
                for g, n in zip(grads, ("grad_logprob", "grad_entropy", "grad_lse"))]

    def run(self, logits: torch.Tensor, targets: torch.Tensor | None = None,
            dlogits: torch.Tensor | None = None, grad_logprob: torch.Tensor | None = None,
            grad_entropy: torch.Tensor | None = None, grad_lse: torch.Tensor | None = None,
            stream: int | None = None) -> None:
        """One call (enqueued on the stream, asynchronous) over logits [rows,
        vocab] with contiguous rows any distance apart.  ``targets``: int64
        [rows], negative where no token is asked for (logprob 0); without it
        ``logprob`` is not written.  ``dlogits``: also the gradient of a loss
        whose derivatives with respect to logprob, entropy and lse() are the
        fp32 [rows] ``grad_*`` (None: zero), for losses whose weights are known
        before the call; it may be ``logits`` itself."""
        ld, ld_grad = self._matrices(logits, dlogits)
        t = _vector(targets, "targets", (self.rows,), torch.int64, self.device)
        st = B.lib.symtile_token_logprobs(
            self.device, logits.data_ptr(), self.rows, self.vocab, ld, self._dt, self.scale, t,
            None if t is None else self.logprob.data_ptr(), *self._out,
            *self._grads(grad_logprob, grad_entropy, grad_lse),
            None if dlogits is None else dlogits.data_ptr(), ld_grad, *self._ws,
            self._stream(stream))
        if st:
            B._check(st, "symtile_token_logprobs")

    def backward(self, logits: torch.Tensor, targets: torch.Tensor | None, dlogits: torch.Tensor,
                 grad_logprob: torch.Tensor | None = None,
                 grad_entropy: torch.Tensor | None = None,
                 grad_lse: torch.Tensor | None = None, stream: int | None = None) -> None:
        """The gradient alone, with this object's entropy and stats of the last
        ``run`` on the same logits: for weights that follow from its values.
        ``dlogits`` may be ``logits`` itself."""
        ld, ld_grad = self._matrices(logits, dlogits)
        st = B.lib.symtile_token_logprobs_backward(
            self.device, logits.data_ptr(), self.rows, self.vocab, ld, self._dt, self.scale,
            _vector(targets, "targets", (self.rows,), torch.int64, self.device), self._out[0],
            self._out[1], *self._grads(grad_logprob, grad_entropy, grad_lse), dlogits.data_ptr(),
            ld_grad, self._stream(stream))
        if st:
            B._check(st, "symtile_token_logprobs_backward")


class TopDistillation(_Rows):
    """The loss of ``scale`` * logits against a teacher's list of ``k`` entries
    a row: sum_j q_j (log q_j - log p_j), with q = softmax(scale * values) over
    the list, or with ``rest`` q_j = exp(values_j) and all other tokens as one
    more class.  Outputs of every call: ``loss`` [rows] and ``stats`` [rows, 4]."""

    def __init__(self, rows: int, vocab: int, dtype: torch.dtype, k: int, scale: float = 1.0,
                 rest: bool = False, device: int = 0):
        super().__init__(rows, vocab, dtype, 0, scale, device)
        self.k = k
        self.mode = B.DISTILL_REST if rest else B.DISTILL_RENORM
        self.loss, self.stats = self._new(rows), self._new(rows, 4)

    def _list(self, ids, values):
        if values.dtype not in _DTYPES:
            raise TypeError("values must be float16, bfloat16 or float32")
        return (_vector(ids, "ids", (self.rows, self.k), torch.int64, self.device),
                _vector(values, "values", (self.rows, self.k), values.dtype, self.device),
                _DTYPES[values.dtype], self.k, self.mode)

    def run(self, logits: torch.Tensor, ids: torch.Tensor, values: torch.Tensor,
            row_grad: torch.Tensor | None = None, dlogits: torch.Tensor | None = None,
            stream: int | None = None) -> None:
        """One call (enqueued on the stream, asynchronous).  ``ids``: int64 [rows,
        k], negative = absent; ``values``: [rows, k] in any of the three types.
        With ``dlogits`` and the fp32 [rows] ``row_grad`` also the gradient of
        sum_r row_grad[r] * loss[r]; ``dlogits`` may be ``logits`` itself."""
        ld, ld_grad = self._matrices(logits, dlogits)
        st = B.lib.symtile_distill_topk(
            self.device, logits.data_ptr(), self.rows, self.vocab, ld, self._dt, self.scale,
            *self._list(ids, values), self.loss.data_ptr(), self.stats.data_ptr(),
            _vector(row_grad, "row_grad", (self.rows,), torch.float32, self.device),
            None if dlogits is None else dlogits.data_ptr(), ld_grad, *self._ws,
            self._stream(stream))
        if st:
            B._check(st, "symtile_distill_topk")

    def backward(self, logits: torch.Tensor, ids: torch.Tensor, values: torch.Tensor,
                 row_grad: torch.Tensor, dlogits: torch.Tensor, stream: int | None = None) -> None:
        """The gradient alone, with this object's stats of the last ``run`` on the
        same logits and list."""
        ld, ld_grad = self._matrices(logits, dlogits)
        st = B.lib.symtile_distill_topk_backward(
            self.device, logits.data_ptr(), self.rows, self.vocab, ld, self._dt, self.scale,
            *self._list(ids, values), self.stats.data_ptr(),
            _vector(row_grad, "row_grad", (self.rows,), torch.float32, self.device),
            dlogits.data_ptr(), ld_grad, self._stream(stream))
        if st:
            B._check(st, "symtile_distill_topk_backward")
