"""Operators on rows of logits in torch tensors (the msd_logits_* calls of
include/msd.h, which has their definitions).

Argument marshalling only: every operator is one kernel of libmsd.so on the
current stream of its tensors' device.  Outputs are the caller's buffers.
Logits are two-dimensional CUDA tensors (float32, bfloat16 or float16) whose rows
are contiguous; rows may lie any distance apart.  Everything else is contiguous.
"""
import torch

from . import msd as _msd
from .mx import TYPES, _float, _run


def _logits(x, what="logits"):
    if x.dim() != 2:
        raise ValueError(f"{what}: shape {tuple(x.shape)}, wants rows and columns")
    return _float(x, x.shape, x.device, what)


def _array(t, dtype, shape, device, what):
    """Pointer of a contiguous array, None for none."""
    if t is None:
        return None
    if t.dtype != dtype or t.shape != shape or not t.is_contiguous() or t.device != device:
        raise ValueError(f"{what}: wants contiguous {dtype} {tuple(shape)} on {device}, got "
                         f"{t.dtype} {tuple(t.shape)} on {t.device}")
    return t.data_ptr()


def _needed(t, *args):
    if t is None:
        raise ValueError(f"{args[-1]}: missing")
    return _array(t, *args)


def _like(t, x, what):
    """Pointer and row distance of an output of x's shape and type."""
    if t.dtype != x.dtype:
        raise ValueError(f"{what}: {t.dtype}, the logits are {x.dtype}")
    return _float(t, x.shape, x.device, what)


def top(logits, values, ids, lse=None):
    """The first k tokens of every row by logit: values and ids [rows, k], and the rows'
    log-sum-exp.  Returns (values, ids)."""
    p, ld = _logits(logits)
    if values is None or values.dim() != 2 or values.shape[0] != logits.shape[0]:
        raise ValueError(f"values: wants {logits.shape[0]} rows of k")
    d, shape = logits.device, values.shape
    _run(d, _msd.msd_logits_top, p, TYPES[logits.dtype], ld, *logits.shape, shape[1],
         _array(values, torch.float32, shape, d, "values"),
         _needed(ids, torch.int32, shape, d, "ids"),
         _array(lse, torch.float32, shape[:1], d, "lse"))
    return values, ids


def sample(logits, uniforms, tokens, logprobs=None, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """tokens = one token of every row, drawn with the row's uniform number; logprobs
    their log-probabilities.  Returns tokens."""
    p, ld = _logits(logits)
    d, shape = logits.device, logits.shape[:1]
    _run(d, _msd.msd_logits_sample, p, TYPES[logits.dtype], ld, *logits.shape,
         _msd.Sampling(temperature, top_p, min_p, top_k),
         _needed(uniforms, torch.float32, shape, d, "uniforms"),
         _needed(tokens, torch.int32, shape, d, "tokens"),
         _array(logprobs, torch.float32, shape, d, "logprobs"))
    return tokens


def filter(logits, out, kept=None, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """out = the logits of the tokens that stay, -inf for the others (out may be logits);
    kept = how many stay.  Returns out."""
    p, ld = _logits(logits)
    po, ldo = _like(out, logits, "out")
    _run(logits.device, _msd.msd_logits_filter, p, TYPES[logits.dtype], ld, *logits.shape,
         _msd.Sampling(temperature, top_p, min_p, top_k), po, ldo,
         _array(kept, torch.int32, logits.shape[:1], logits.device, "kept"))
    return out


def _distill(logits, ids, values, temperature, loss, lse, grad, dlogits):
    p, ld = _logits(logits)
    if ids is None or ids.dim() != 2 or ids.shape[0] != logits.shape[0]:
        raise ValueError(f"ids: wants {logits.shape[0]} rows of k")
    d, rows = logits.device, logits.shape[:1]
    teacher = _msd.Teacher(_array(ids, torch.int32, ids.shape, d, "ids"),
                           _needed(values, torch.float32, ids.shape, d, "values"),
                           ids.shape[1], temperature)
    px, ldx = _like(dlogits, logits, "dlogits") if dlogits is not None else (None, 0)
    _run(d, _msd.msd_logits_distill, p, TYPES[logits.dtype], ld, *logits.shape, teacher,
         _array(loss, torch.float32, rows, d, "loss"), _array(lse, torch.float32, rows, d, "lse"),
         _array(grad, torch.float32, rows, d, "grad"), px, ldx)


def distill(logits, ids, values, temperature, loss, lse=None, grad=None, dlogits=None):
    """loss = the rows' divergence from a teacher's top logits (ids and values [rows, k], as
    top() writes them); with the rows' weights grad also the gradient dlogits (which may
    be logits), in the same pass.  Returns loss."""
    _distill(logits, ids, values, temperature, loss, lse, grad, dlogits)
    return loss


def distill_backward(logits, ids, values, temperature, grad, dlogits):
    """dlogits = the gradient of the sum of grad * loss.  Returns dlogits."""
    if grad is None or dlogits is None:
        raise ValueError("grad and dlogits: missing")
    _distill(logits, ids, values, temperature, None, None, grad, dlogits)
    return dlogits
