"""Python binding of libstagefrontier's second header (ctypes; argument
marshalling only): the numbers that a training step itself yields.

Every function has the name of the C entry point it wraps (declared in
``include/stagefrontier_train.h``).  As in ``stagefrontier``, arrays are torch
tensors on the GPU, outputs and workspaces that are not given are allocated on
the call's stream, and every step of the computation runs in the library's HIP
kernels.

Autograd does not see through the calls: their outputs require no gradient, also
where the inputs do, and a loss made of them passes none back.
``sf_policy_loss`` and ``sf_token_logp_grad`` compute the gradients themselves;
the program hands the last to autograd (``logits.backward(grad)``).  What a call
writes into a caller's tensor counts there as an operation in place.
"""
from __future__ import annotations

import ctypes
import operator

import torch

from .stagefrontier import (SF_EINVAL, SF_EHIP, SF_ERANGE, SF_MAX_R, SF_OK, StageFrontierError,  # noqa: F401
                            _check, _lib, _new, _stream_handle)

SF_F32, SF_BF16, SF_F16 = 0, 1, 2
SF_MEAN_TOKENS, SF_MEAN_SEQUENCES, SF_SUM_TOKENS = 0, 1, 2

_DTYPES = {torch.float32: SF_F32, torch.bfloat16: SF_BF16, torch.float16: SF_F16}


def _declare(lib):
    i64, i32, f32, vp, ci = ctypes.c_int64, ctypes.c_int32, ctypes.c_float, ctypes.c_void_p, ctypes.c_int
    for name, res, args in (
            ("sf_token_logp", ci, [vp, i32, i64, i64, i64, vp, f32, vp, vp, vp, vp, i64, vp]),
            ("sf_token_logp_workspace", i64, [i32, i64, i64]),
            ("sf_token_logp_grad", ci, [vp, i32, i64, i64, i64, vp, f32, vp, vp, vp, vp, vp, i64, vp]),
            ("sf_policy_loss", ci, [vp, vp, vp, vp, i32, vp, vp, i64, i64, i32, f32, f32, f32, f32, vp, vp, vp,
                                    i64, vp]),
            ("sf_policy_loss_workspace", i64, [i64, i64]),
            ("sf_grad_list_bytes", i64, [i32]),
            ("sf_grad_list_init", ci, [vp, i64, vp, vp, vp, i32]),
            ("sf_grad_norm", ci, [vp, vp, vp, vp, vp, i64, vp]),
            ("sf_grad_norm_workspace", i64, [vp]),
            ("sf_grad_clip", ci, [vp, vp, vp, i64, f32, f32, vp, vp])):
        fn = getattr(lib, name)
        fn.restype, fn.argtypes = res, args


_declare(_lib)


def sf_token_logp_workspace(dtype: torch.dtype, N: int, V: int) -> int:
    return int(_lib.sf_token_logp_workspace(_DTYPES.get(dtype, -1), N, V))


def sf_policy_loss_workspace(N: int, B: int) -> int:
    return int(_lib.sf_policy_loss_workspace(N, B))


def _out(t, name: str, dtype, shape, like: torch.Tensor, stream):
    """An output: the caller's, checked, or a new one."""
    if t is None:
        return _new(shape, dtype, like.device, stream)
    _check(t, name, dtype, shape, like)
    return t


def _wrote(*outs):
    """Tells autograd that the caller's tensors were written, as an operation of
    torch's does: a backward pass that saved one of them refuses it."""
    outs = [t for t in outs if t is not None]
    if outs:
        torch.autograd.graph.increment_version(outs)


def _space(workspace, need: int, where: str, like: torch.Tensor, stream):
    """The call's workspace: the caller's uint8 tensor, or a new one."""
    if need < 0:
        raise StageFrontierError(SF_EINVAL, where)
    if workspace is None:
        return _new((need,), torch.uint8, like.device, stream)
    _check(workspace, "workspace", torch.uint8, workspace.shape, like)
    if workspace.numel() < need:
        raise ValueError("workspace has %d bytes, %d are needed" % (workspace.numel(), need))
    return workspace


def _rows(t: torch.Tensor, name: str) -> int:
    """Checks a matrix of logits and returns its row stride."""
    if not isinstance(t, torch.Tensor) or t.dtype not in _DTYPES:
        raise TypeError("%s must be a float32, bfloat16 or float16 torch.Tensor" % name)
    if not t.is_cuda:
        raise ValueError("%s must be a GPU tensor" % name)
    if t.dim() != 2 or t.shape[1] < 1:
        raise ValueError("%s must be [N, V] with V >= 1" % name)
    N, V = t.shape
    if V > 1 and t.stride(1) != 1:
        raise ValueError("%s must have its rows' entries next to each other" % name)
    if N > 1 and t.stride(0) < V:
        raise ValueError("%s must have rows that do not overlap" % name)
    return t.stride(0) if N > 1 else V


def sf_token_logp(logits: torch.Tensor, targets: torch.Tensor, inv_temperature: float = 1.0, entropy: bool = True,
                  out_logp: torch.Tensor | None = None, out_lse: torch.Tensor | None = None,
                  out_entropy: torch.Tensor | None = None, workspace: torch.Tensor | None = None, stream=None):
    """Log-probability of the taken token, normaliser and entropy of each row
    of logits (``sf_token_logp``).

    ``logits`` [N, V] float32, bfloat16 or float16, rows any distance apart;
    ``targets`` [N] int64, a row whose target lies outside [0, V) takes no
    part.  Returns ``(out_logp, out_lse, out_entropy)``, [N] float32 each;
    ``out_entropy`` is None with ``entropy=False``.
    """
    stride = _rows(logits, "logits")
    N, V = logits.shape
    dev = logits.device
    _check(targets, "targets", torch.int64, (N,), logits)
    given = (out_logp, out_lse, out_entropy)
    if out_logp is None and out_lse is None and out_entropy is None and entropy:
        # one allocation for the three costs 2 us less than one each
        out_logp, out_lse, out_entropy = _new((3, N), torch.float32, dev, stream).unbind(0)
    else:
        out_logp = _out(out_logp, "out_logp", torch.float32, (N,), logits, stream)
        out_lse = _out(out_lse, "out_lse", torch.float32, (N,), logits, stream)
        if out_entropy is not None or entropy:
            out_entropy = _out(out_entropy, "out_entropy", torch.float32, (N,), logits, stream)
    dtype = _DTYPES[logits.dtype]
    need = _lib.sf_token_logp_workspace(dtype, N, V)
    if need != 0:
        workspace = _space(workspace, need, "sf_token_logp", logits, stream)
    rc = _lib.sf_token_logp(logits.data_ptr(), dtype, N, V, stride, targets.data_ptr(),
                            inv_temperature, out_logp.data_ptr(), out_lse.data_ptr(),
                            None if out_entropy is None else out_entropy.data_ptr(),
                            None if need == 0 else workspace.data_ptr(), need, _stream_handle(stream, dev))
    if rc != SF_OK:
        raise StageFrontierError(rc, "sf_token_logp")
    _wrote(*given)
    return out_logp, out_lse, out_entropy


def sf_token_logp_grad(logits: torch.Tensor, targets: torch.Tensor, lse: torch.Tensor, grad_logp: torch.Tensor,
                       entropy: torch.Tensor | None = None, grad_entropy: torch.Tensor | None = None,
                       inv_temperature: float = 1.0, out_grad: torch.Tensor | None = None, stream=None):
    """Gradient of ``sf_token_logp``'s outputs back to the logits
    (``sf_token_logp_grad``).

    ``grad_logp`` and ``grad_entropy`` [N] float32 are the loss's gradients;
    ``entropy`` is needed with the second.  ``out_grad`` [N, V] of the logits'
    type may be the logits themselves.  Returns ``out_grad``.
    """
    stride = _rows(logits, "logits")
    N, V = logits.shape
    dev = logits.device
    _check(targets, "targets", torch.int64, (N,), logits)
    _check(lse, "lse", torch.float32, (N,), logits)
    _check(grad_logp, "grad_logp", torch.float32, (N,), logits)
    if grad_entropy is not None:
        _check(grad_entropy, "grad_entropy", torch.float32, (N,), logits)
        if entropy is None:
            raise ValueError("entropy is needed with grad_entropy")
    if entropy is not None:
        _check(entropy, "entropy", torch.float32, (N,), logits)
    given = out_grad
    if out_grad is None:
        out_grad = _new((N, V), logits.dtype, dev, stream)
    out_stride = _rows(out_grad, "out_grad")
    if out_grad.dtype is not logits.dtype or out_grad.shape != logits.shape or out_grad.device != dev:
        raise ValueError("out_grad must have the logits' type, shape and device")
    rc = _lib.sf_token_logp_grad(logits.data_ptr(), _DTYPES[logits.dtype], N, V, stride, targets.data_ptr(),
                                 inv_temperature, lse.data_ptr(), grad_logp.data_ptr(),
                                 None if entropy is None else entropy.data_ptr(),
                                 None if grad_entropy is None else grad_entropy.data_ptr(), out_grad.data_ptr(),
                                 out_stride, _stream_handle(stream, dev))
    if rc != SF_OK:
        raise StageFrontierError(rc, "sf_token_logp_grad")
    _wrote(given)
    return out_grad


def sf_policy_loss(logp: torch.Tensor, old_logp: torch.Tensor, advantage: torch.Tensor, seq_start: torch.Tensor,
                   ref_logp: torch.Tensor | None = None, mask: torch.Tensor | None = None,
                   advantage_per_token: bool = False, reduction: int = SF_MEAN_TOKENS, scale: float = 1.0,
                   clip_low: float = 0.2, clip_high: float = 0.2, kl_coef: float = 0.0,
                   out_terms: torch.Tensor | None = None, out_grad: torch.Tensor | None = None,
                   workspace: torch.Tensor | None = None, stream=None):
    """Clipped policy loss with a KL term over ragged sequences, and its
    gradient (``sf_policy_loss``).

    ``logp``, ``old_logp``, ``ref_logp`` [N] float32; ``advantage`` [B], or [N]
    with ``advantage_per_token``; ``mask`` [N] uint8 or bool; ``seq_start``
    [B + 1] int64.  Returns ``(out_terms [4], out_grad [N])``: loss, policy
    term, KL and clipped share, and the gradient of the loss.
    """
    if logp.dim() != 1 or seq_start.dim() != 1 or seq_start.shape[0] < 1:
        raise ValueError("logp must be [N] and seq_start [B + 1]")
    N, B = logp.shape[0], seq_start.shape[0] - 1
    f32 = torch.float32
    _check(logp, "logp", f32, (N,))
    _check(old_logp, "old_logp", f32, (N,), logp)
    _check(advantage, "advantage", f32, (N if advantage_per_token else B,), logp)
    _check(seq_start, "seq_start", torch.int64, (B + 1,), logp)
    if ref_logp is not None:
        _check(ref_logp, "ref_logp", f32, (N,), logp)
    if mask is not None:
        _check(mask, "mask", torch.bool if mask.dtype is torch.bool else torch.uint8, (N,), logp)
    dev = logp.device
    given = (out_terms, out_grad)
    out_terms = _out(out_terms, "out_terms", f32, (4,), logp, stream)
    out_grad = _out(out_grad, "out_grad", f32, (N,), logp, stream)
    need = _lib.sf_policy_loss_workspace(N, B)
    if need != 0:
        workspace = _space(workspace, need, "sf_policy_loss", logp, stream)
    rc = _lib.sf_policy_loss(logp.data_ptr(), old_logp.data_ptr(), None if ref_logp is None else ref_logp.data_ptr(),
                             advantage.data_ptr(), bool(advantage_per_token),
                             None if mask is None else mask.data_ptr(), seq_start.data_ptr(), N, B, reduction, scale,
                             clip_low, clip_high, kl_coef, out_terms.data_ptr(), out_grad.data_ptr(),
                             None if need == 0 else workspace.data_ptr(), need, _stream_handle(stream, dev))
    if rc != SF_OK:
        raise StageFrontierError(rc, "sf_policy_loss")
    _wrote(*given)
    return out_terms, out_grad


def _dense(t: torch.Tensor) -> bool:
    """Whether the entries fill one piece of memory, in any order of dimensions."""
    if t.is_contiguous():
        return True
    want = 1
    for stride, size in sorted((st, sz) for st, sz in zip(t.stride(), t.shape) if sz != 1):
        if stride != want:
            return False
        want *= size
    return True


_data_ptr, _nbytes, _stride = torch.Tensor.data_ptr, operator.attrgetter("nbytes"), torch.Tensor.stride


def _order(t: torch.Tensor):
    """What a dense tensor's dimensions order its entries by: None where that is
    theirs, else the strides of those with more than one entry."""
    return None if t.is_contiguous() else tuple(st if sz != 1 else 0 for st, sz in zip(t.stride(), t.shape))


def _lay_out(tensors):
    """The C list of tensors (``sf_grad_list_init``)."""
    n = len(tensors)
    size = _lib.sf_grad_list_bytes(n)
    if size < 0:
        raise StageFrontierError(SF_EINVAL, "sf_grad_list_init")
    made = (ctypes.c_int64 * ((size + 7) // 8))()
    ptrs = (ctypes.c_void_p * n)(*(t.data_ptr() for t in tensors))
    numel = (ctypes.c_int64 * n)(*(t.numel() for t in tensors))
    dtype = (ctypes.c_int32 * n)(*(_DTYPES[t.dtype] for t in tensors))
    rc = _lib.sf_grad_list_init(made, size, ptrs, numel, dtype, n)
    if rc != SF_OK:
        raise StageFrontierError(rc, "sf_grad_list_init")
    return made


class GradSet:
    """A list of gradient tensors laid out for ``sf_grad_norm`` and
    ``sf_grad_clip`` (``sf_grad_list_init``), checked once.

    Tensors are dense float32, bfloat16 or float16 ones on one GPU, mixed as
    they come.  The set stands for these tensors in the memory that they have
    now: a program that gives its parameters new gradient tensors
    (``zero_grad(set_to_none=True)``, torch's default) makes a new set of those,
    and one whose tensors have other memory since is refused by the calls.
    """

    def __init__(self, tensors):
        self.tensors = list(tensors)
        self.device = None
        for k, t in enumerate(self.tensors):
            if not isinstance(t, torch.Tensor) or t.dtype not in _DTYPES:
                raise TypeError("gradient %d must be a float32, bfloat16 or float16 torch.Tensor" % k)
            if not t.is_cuda:
                raise ValueError("gradient %d must be a GPU tensor" % k)
            if self.device is None:
                self.device = t.device
            if t.device != self.device:
                raise ValueError("gradient %d is on %s, the others on %s" % (k, t.device, self.device))
            if not _dense(t):
                raise ValueError("gradient %d must fill its memory without gaps" % k)
        self._held = tuple(list(map(f, self.tensors)) for f in (_data_ptr, _nbytes, _stride))
        self._list = _lay_out(self.tensors)
        # a list of no tensors launches nothing: one without entries has a clip's status set
        self._clip_list = self._list if self.tensors else _lay_out([torch.empty(0, dtype=torch.float32)])
        self._order = [_order(t) for t in self.tensors]
        self.workspace_bytes = int(_lib.sf_grad_norm_workspace(self._list))

    def check(self, order: bool = False):
        """Raises where a tensor no longer has the memory that was laid out (its
        ``data`` set, its storage resized), or, with ``order``, its layout.
        (0.2 us a tensor: the kernels would read and write the former memory,
        which may be another tensor's by now.)"""
        for of, held in zip((_data_ptr, _nbytes, _stride) if order else (_data_ptr, _nbytes), self._held):
            now = list(map(of, self.tensors))
            if now != held:
                if len(now) != len(held):
                    raise ValueError("the set has %d tensors of the %d laid out" % (len(now), len(held)))
                k = next(k for k in range(len(now)) if now[k] != held[k])
                raise ValueError("gradient %d is not as it was laid out (%s %s, then %s): make a new set"
                                 % (k, "stride" if of is _stride else "bytes" if of is _nbytes else "address", now[k], held[k]))

    def __len__(self):
        return len(self.tensors)


def sf_grad_norm_workspace(grads) -> int:
    return (grads if isinstance(grads, GradSet) else GradSet(grads)).workspace_bytes


def sf_grad_norm(grads, out_norms: torch.Tensor | None = None, out_total: torch.Tensor | None = None,
                 out_nonfinite: torch.Tensor | None = None, workspace: torch.Tensor | None = None, stream=None):
    """L2 norms of gradients and their counts of entries that are not finite
    (``sf_grad_norm``).

    ``grads``: a ``GradSet``, or tensors to make one of for this call.  Returns
    ``(out_norms [n] float32, out_total [1] float32, out_nonfinite [n] int64)``.
    """
    if not isinstance(grads, GradSet):
        grads = GradSet(grads)
    else:
        grads.check()
    n = len(grads)
    if n == 0 and out_total is None:
        raise ValueError("out_total is needed where there are no gradients")
    like = grads.tensors[0] if n else out_total
    dev = like.device
    given = (out_norms, out_total, out_nonfinite)
    out_norms = _out(out_norms, "out_norms", torch.float32, (n,), like, stream)
    out_total = _out(out_total, "out_total", torch.float32, (1,), like, stream)
    out_nonfinite = _out(out_nonfinite, "out_nonfinite", torch.int64, (n,), like, stream)
    workspace = _space(workspace, grads.workspace_bytes, "sf_grad_norm", like, stream)
    rc = _lib.sf_grad_norm(grads._list, out_norms.data_ptr(), out_total.data_ptr(), out_nonfinite.data_ptr(),
                           workspace.data_ptr(), workspace.numel(), _stream_handle(stream, dev))
    if rc != SF_OK:
        raise StageFrontierError(rc, "sf_grad_norm")
    _wrote(*given)
    return out_norms, out_total, out_nonfinite


def sf_grad_clip(grads, norms: torch.Tensor, max_norm: float, eps: float = 1e-6, out=None,
                 status: torch.Tensor | None = None, stream=None):
    """Scales gradients to a largest norm (``sf_grad_clip``).

    ``grads``: a ``GradSet`` or tensors.  ``norms`` [m] float32: ``out_total``
    of ``sf_grad_norm``, or that of every rank.  ``out``: where the scaled
    gradients go (a ``GradSet`` or tensors of the same types and layouts), by
    default in place.  ``status``, a one-element int32 tensor, takes
    ``SF_ERANGE`` where the norm is not finite and the gradients are left as
    they are, also on a rank that has none.  Returns the set of scaled gradients.
    """
    if not isinstance(grads, GradSet):
        grads = GradSet(grads)
    else:
        grads.check(order=out is not None and out is not grads)
    if out is None:
        out = grads
    elif not isinstance(out, GradSet):
        out = GradSet(out)
    elif out is not grads:
        out.check(order=True)
    if norms.dim() != 1:
        raise ValueError("norms must be [m]")
    if len(out) != len(grads):
        raise ValueError("out has %d tensors, grads %d" % (len(out), len(grads)))
    if out is not grads:
        if out._order != grads._order:
            raise ValueError("out must have the gradients' order of dimensions")
        if out.device != grads.device:
            raise ValueError("out is on %s, the gradients on %s" % (out.device, grads.device))
    like = grads.tensors[0] if len(grads) else norms
    _check(norms, "norms", torch.float32, norms.shape, like)
    if status is not None:
        _check(status, "status", torch.int32, (1,), like)
    rc = _lib.sf_grad_clip(grads._clip_list, out._clip_list, norms.data_ptr(), norms.shape[0], max_norm, eps,
                           None if status is None else status.data_ptr(), _stream_handle(stream, like.device))
    if rc != SF_OK:
        raise StageFrontierError(rc, "sf_grad_clip")
    torch.autograd.graph.increment_version(out.tensors)
    _wrote(status)
    return out
