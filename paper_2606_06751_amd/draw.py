"""Python binding of libstagefrontier's third header (ctypes; argument
marshalling only): what a policy step draws at random.

Every function has the name of the C entry point it wraps (declared in
``include/stagefrontier_draw.h``).  As in ``stagefrontier`` and ``train``,
arrays are torch tensors on the GPU, outputs and workspaces that are not given
are allocated on the call's stream, and every step of the computation runs in
the library's HIP kernels.

A key is an int64 tensor of two on the GPU, the seed and the step.  A program
raises the step once per training step (``key[1] += 1``, also in a captured
graph) and gives each call of a step a ``site`` of its own.

Autograd does not see through the calls: their outputs require no gradient.
The gradient of ``sf_dropout`` is ``sf_dropout`` of the output's gradient with
the same ``p``, ``key``, ``site``, ``first`` and ``index_stride``.  What a call
writes into a caller's tensor counts there as an operation in place.
"""
from __future__ import annotations

import ctypes

import torch

from .stagefrontier import SF_OK, StageFrontierError, _check, _lib, _new, _stream_handle
from .train import _DTYPES, _out, _space, _wrote


def _declare(lib):
    i64, i32, u32, f32, vp, ci = (ctypes.c_int64, ctypes.c_int32, ctypes.c_uint32, ctypes.c_float, ctypes.c_void_p,
                                  ctypes.c_int)
    for name, res, args in (
            ("sf_uniform", ci, [vp, u32, i64, i64, vp, vp]),
            ("sf_dropout", ci, [vp, i32, i64, i64, i64, f32, vp, u32, i64, i64, vp, i64, vp, i32, i64, vp]),
            ("sf_token_sample", ci, [vp, i32, i64, i64, i64, vp, f32, vp, vp, vp, i64, vp]),
            ("sf_token_sample_workspace", i64, [i32, i64, i64]),
            ("sf_draft_verify", ci, [vp, vp, i32, i64, i64, i64, i64, i64, vp, vp, vp, f32, f32, vp, vp, vp, vp, i64, vp]),
            ("sf_draft_verify_workspace", i64, [i32, i64, i64, i64])):
        fn = getattr(lib, name)
        fn.restype, fn.argtypes = res, args


_declare(_lib)


def sf_token_sample_workspace(dtype: torch.dtype, N: int, V: int) -> int:
    return int(_lib.sf_token_sample_workspace(_DTYPES.get(dtype, -1), N, V))


def sf_draft_verify_workspace(dtype: torch.dtype, D: int, B: int, V: int) -> int:
    return int(_lib.sf_draft_verify_workspace(_DTYPES.get(dtype, -1), D, B, V))


_current_device = torch._C._cuda_getDevice


def _call(fn, device, *args):
    """The library's call, with the tensors' device as the current one: the
    handle of a device's default stream does not name the device."""
    if _current_device() == device.index:
        rc = fn(*args)
    else:
        with torch.cuda.device(device):
            rc = fn(*args)
    if rc != SF_OK:
        raise StageFrontierError(rc, fn.__name__)


def _site(site) -> int:
    if not 0 <= site < 1 << 32:
        raise ValueError("site must lie in [0, 2^32)")
    return site


def sf_uniform(n: int, key: torch.Tensor, site: int = 0, first: int = 0, out: torch.Tensor | None = None, stream=None):
    """``n`` uniform numbers in [0, 1) (``sf_uniform``): those of the indexes
    from ``first`` on.  Returns ``out`` [n] float32."""
    _check(key, "key", torch.int64, (2,))
    given = out
    out = _out(out, "out", torch.float32, (n,), key, stream)
    _call(_lib.sf_uniform, key.device, key.data_ptr(), _site(site), first, n, out.data_ptr(),
          _stream_handle(stream, key.device))
    _wrote(given)
    return out


def _matrix(t: torch.Tensor, name: str, shape=None, like: torch.Tensor | None = None) -> int:
    """Checks rows of entries and returns their stride.  (As in ``_check``, the
    good path is one chained test.)"""
    try:
        if (t.dtype in _DTYPES and t.is_cuda and t.dim() == 2 and (shape is None or t.shape == shape)
                and (like is None or t.get_device() == like.get_device())):
            (N, C), (down, across) = t.shape, t.stride()
            if (across == 1 or C <= 1) and (down >= C or N <= 1):
                return down if N > 1 else C
    except AttributeError:
        pass
    if not isinstance(t, torch.Tensor) or t.dtype not in _DTYPES:
        raise TypeError("%s must be a float32, bfloat16 or float16 torch.Tensor" % name)
    if not t.is_cuda:
        raise ValueError("%s must be a GPU tensor" % name)
    if shape is not None and t.shape != shape:
        raise ValueError("%s must have shape %s, got %s" % (name, tuple(shape), tuple(t.shape)))
    if like is not None and t.get_device() != like.get_device():
        raise ValueError("%s is on %s, the call's other arrays on %s" % (name, t.device, like.device))
    if t.dim() != 2:
        raise ValueError("%s must be [N, C]" % name)
    if t.shape[1] > 1 and t.stride(1) != 1:
        raise ValueError("%s must have its rows' entries next to each other" % name)
    raise ValueError("%s must have rows that do not overlap" % name)


def sf_dropout(x: torch.Tensor, p: float, key: torch.Tensor, site: int = 0, first: int = 0,
               index_stride: int | None = None, residual: torch.Tensor | None = None,
               out: torch.Tensor | None = None, out_dtype: torch.dtype | None = None, stream=None):
    """Dropout of ``x`` [N, C], onto ``residual`` where one is given
    (``sf_dropout``).

    ``first`` and ``index_stride`` (default C) say which entries of the whole
    these are.  ``out`` [N, C] may be ``x`` or ``residual``; a new one has
    ``out_dtype``, by default the residual's type, else that of ``x``.
    Returns ``out``.
    """
    x_stride = _matrix(x, "x")
    N, C = x.shape
    dev = x.device
    _check(key, "key", torch.int64, (2,), x)
    given = out
    if out is not None:
        kind = out.dtype
        if out_dtype is not None and kind is not out_dtype:
            raise TypeError("out must be a %s torch.Tensor" % out_dtype)
        out_stride = _matrix(out, "out", x.shape, x)
    else:
        kind = out_dtype or (x.dtype if residual is None else residual.dtype)
        if kind not in _DTYPES:
            raise TypeError("out_dtype must be float32, bfloat16 or float16")
        out, out_stride = _new((N, C), kind, dev, stream), C
    residual_stride = C
    if residual is not None:
        residual_stride = _matrix(residual, "residual", x.shape, x)
        if residual.dtype is not kind:
            raise TypeError("residual must have the output's type")
    _call(_lib.sf_dropout, dev, x.data_ptr(), _DTYPES[x.dtype], N, C, x_stride, p, key.data_ptr(), _site(site), first,
          C if index_stride is None else index_stride, None if residual is None else residual.data_ptr(),
          residual_stride, out.data_ptr(), _DTYPES[kind], out_stride, _stream_handle(stream, dev))
    _wrote(given)
    return out


def sf_token_sample(logits: torch.Tensor, uniform: torch.Tensor, inv_temperature: float = 1.0,
                    out_token: torch.Tensor | None = None, out_logp: torch.Tensor | None = None,
                    workspace: torch.Tensor | None = None, stream=None):
    """A token of each row of logits by its distribution, and its
    log-probability (``sf_token_sample``).

    ``logits`` [N, V] float32, bfloat16 or float16, rows any distance apart;
    ``uniform`` [N] float32, a row whose number lies outside [0, 1) takes no
    part.  Returns ``(out_token [N] int64, out_logp [N] float32)``.
    """
    stride = _matrix(logits, "logits")
    N, V = logits.shape
    dev = logits.device
    _check(uniform, "uniform", torch.float32, (N,), logits)
    given = out_token is not None or out_logp is not None
    out_token = _out(out_token, "out_token", torch.int64, (N,), logits, stream)
    out_logp = _out(out_logp, "out_logp", torch.float32, (N,), logits, stream)
    dtype = _DTYPES[logits.dtype]
    need = _lib.sf_token_sample_workspace(dtype, N, V)
    if need != 0:
        workspace = _space(workspace, need, "sf_token_sample", logits, stream)
    _call(_lib.sf_token_sample, dev, logits.data_ptr(), dtype, N, V, stride, uniform.data_ptr(), inv_temperature,
          out_token.data_ptr(), out_logp.data_ptr(), None if need == 0 else workspace.data_ptr(), need,
          _stream_handle(stream, dev))
    if given:
        _wrote(out_token, out_logp)
    return out_token, out_logp


def sf_draft_verify(target_logits: torch.Tensor, draft_logits: torch.Tensor | None, draft: torch.Tensor,
                    seq_start: torch.Tensor, uniform: torch.Tensor, inv_temperature: float = 1.0,
                    draft_inv_temperature: float = 1.0, out_accepted: torch.Tensor | None = None,
                    out_token: torch.Tensor | None = None, out_logp: torch.Tensor | None = None,
                    workspace: torch.Tensor | None = None, stream=None):
    """Verifies drafted tokens against the target's probabilities and draws one
    more token of each sequence (``sf_draft_verify``).

    ``draft`` [D] int64, the drafts of all sequences, ``seq_start`` [B + 1]
    int64; ``target_logits`` [D + B, V], a row for each draft of a sequence and
    one behind them; ``draft_logits`` [D, V] of the same type, or None where
    drafts are certain; ``uniform`` [D + B] float32.  Returns ``(out_accepted
    [B] int64, out_token [D + B] int64, out_logp [D + B] float32)``.
    """
    stride = _matrix(target_logits, "target_logits")
    try:
        (D,), (ends,) = draft.shape, seq_start.shape
    except AttributeError:
        raise TypeError("draft and seq_start must be torch.Tensors") from None
    except ValueError:
        raise ValueError("draft must be [D] and seq_start [B + 1]") from None
    B, (rows, V), dev = ends - 1, target_logits.shape, target_logits.device
    if B < 0:
        raise ValueError("seq_start must be [B + 1]")
    if rows != D + B:
        raise ValueError("target_logits must have D + B = %d rows, got %d" % (D + B, rows))
    draft_stride = V
    if draft_logits is not None:
        draft_stride = _matrix(draft_logits, "draft_logits", (D, V), target_logits)
        if draft_logits.dtype is not target_logits.dtype:
            raise TypeError("draft_logits must have the target's type")
    index = target_logits.get_device()
    # one chained test on the good path; which of them it is, is asked on failure
    if not (draft.dtype is torch.int64 and seq_start.dtype is torch.int64 and uniform.dtype is torch.float32
            and draft.get_device() == index and seq_start.get_device() == index and uniform.get_device() == index
            and uniform.shape == (rows,) and draft.is_contiguous() and seq_start.is_contiguous()
            and uniform.is_contiguous()):
        _check(draft, "draft", torch.int64, (D,), target_logits)
        _check(seq_start, "seq_start", torch.int64, (ends,), target_logits)
        _check(uniform, "uniform", torch.float32, (rows,), target_logits)
    given = out_accepted is not None or out_token is not None or out_logp is not None
    if given:
        out_accepted = _out(out_accepted, "out_accepted", torch.int64, (B,), target_logits, stream)
        out_token = _out(out_token, "out_token", torch.int64, (rows,), target_logits, stream)
        out_logp = _out(out_logp, "out_logp", torch.float32, (rows,), target_logits, stream)
    else:
        out_accepted = _new((B,), torch.int64, dev, stream)
        out_token = _new((rows,), torch.int64, dev, stream)
        out_logp = _new((rows,), torch.float32, dev, stream)
    dtype = _DTYPES[target_logits.dtype]
    need = _lib.sf_draft_verify_workspace(dtype, D, B, V)
    if need != 0:
        workspace = _space(workspace, need, "sf_draft_verify", target_logits, stream)
    # without drafts there are no rows of theirs, which is not the same as certain ones, but none is looked at
    _call(_lib.sf_draft_verify, dev, target_logits.data_ptr(),
          None if draft_logits is None or D == 0 else draft_logits.data_ptr(), dtype, D, B, V, stride, draft_stride,
          draft.data_ptr(), seq_start.data_ptr(), uniform.data_ptr(), inv_temperature, draft_inv_temperature,
          out_accepted.data_ptr(), out_token.data_ptr(), out_logp.data_ptr(), None if need == 0 else workspace.data_ptr(),
          need, _stream_handle(stream, dev))
    if given:
        _wrote(out_accepted, out_token, out_logp)
    return out_accepted, out_token, out_logp
