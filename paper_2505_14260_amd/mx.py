"""Microscaled 4-bit matrices in torch tensors, and the operators on them (the
msd_mx_* calls of include/msd.h, which has the formats).

Argument marshalling only: every operator is one kernel of libmsd.so on the
current stream of its tensors' device.  Outputs are the caller's buffers.
Float matrices are two-dimensional CUDA tensors whose rows are contiguous; rows
may lie any distance apart.
"""
import torch

from . import msd as _msd

TYPES = {torch.float32: _msd.F32, torch.bfloat16: _msd.BF16, torch.float16: _msd.F16}
LAYOUTS = {"rows": _msd.MX_ROWS, "weight": _msd.MX_WEIGHT}


class MX:
    """Buffers of a quantised matrix of rows x cols values: activations
    ("rows", one or two 4-bit terms) or a product's weight ("weight", one)."""

    def __init__(self, rows, cols, layout="rows", terms=None, device="cuda"):
        if layout not in LAYOUTS:
            raise ValueError(f"layout must be one of {sorted(LAYOUTS)}, got {layout!r}")
        if terms is None:
            terms = 1 if layout == "weight" else 2
        self.shape = (rows, cols)
        self.layout, self.terms = layout, terms
        self.desc = _msd.Mx(None, None, rows, cols, LAYOUTS[layout], terms)
        nc, ns = _msd.msd_mx_bytes(self.desc)
        self.codes = torch.empty(nc, dtype=torch.uint8, device=device)
        self.scales = torch.empty(ns, dtype=torch.uint8, device=device)
        self.device = self.codes.device
        self.desc.codes_d, self.desc.scales_d = self.codes.data_ptr(), self.scales.data_ptr()


def _float(t, shape, device, what):
    """Pointer and row distance of a float matrix."""
    if t.shape != shape:
        raise ValueError(f"{what}: shape {tuple(t.shape)}, wants {tuple(shape)}")
    if t.device != device:
        raise ValueError(f"{what}: on {t.device}, the quantised matrix is on {device}")
    if t.dtype not in TYPES:
        raise ValueError(f"{what}: {t.dtype} is not one of float32, bfloat16, float16")
    ld, step = t.stride()
    if step != 1 and shape[1] > 1:
        raise ValueError(f"{what}: the values of a row must be contiguous")
    return t.data_ptr(), ld if shape[0] > 1 else max(ld, shape[1])


# the current stream's handle without a Stream object (1.8 us of a call's 6.8)
_raw_stream = torch._C._cuda_getCurrentRawStream if torch.version.hip else None


def _run(device, call, *args):
    """call(*args, stream) with the device current."""
    i = device.index
    if device.type != "cuda":
        raise ValueError(f"the matrices must be on a GPU, not on {device}")
    if torch.cuda.current_device() == i:
        call(*args, _raw_stream(i))
    else:
        with torch.cuda.device(i):
            call(*args, _raw_stream(i))


def quantize(src, out):
    """out = the quantised src; returns out."""
    p, ld = _float(src, out.shape, out.device, "src")
    _run(out.device, _msd.msd_mx_quantize, p, TYPES[src.dtype], ld, out.desc)
    return out


def dequantize(q, out):
    """out = the values that q stands for; returns out."""
    p, ld = _float(out, q.shape, q.device, "out")
    _run(q.device, _msd.msd_mx_dequantize, q.desc, p, TYPES[out.dtype], ld)
    return out


def resid_norm(x, y, gain, eps, sum_out, out):
    """sum_out = x + y, out = rmsnorm(x + y) * gain quantised; y and sum_out may
    be None, sum_out may be x or y.  Returns out."""
    px, ldx = _float(x, out.shape, out.device, "x")
    py, ldy = _float(y, out.shape, out.device, "y") if y is not None else (None, 0)
    ps, lds = _float(sum_out, out.shape, out.device, "sum_out") if sum_out is not None else (None, 0)
    for t in (y, sum_out):
        if t is not None and t.dtype != x.dtype:
            raise ValueError(f"x, y and sum_out must have one type, got {x.dtype} and {t.dtype}")
    if gain.dtype != torch.bfloat16 or gain.shape != (out.shape[1],) or not gain.is_contiguous() \
            or gain.device != out.device:
        raise ValueError(f"gain must be {out.shape[1]} contiguous bfloat16 values on {out.device}")
    _run(out.device, _msd.msd_mx_resid_norm, px, ldx, py, ldy, ps, lds, TYPES[x.dtype],
         gain.data_ptr(), eps, out.desc)
    return out


def swiglu(gate, up, out):
    """out = silu(gate) * up quantised; returns out."""
    pg, ldg = _float(gate, out.shape, out.device, "gate")
    pu, ldu = _float(up, out.shape, out.device, "up")
    if gate.dtype != up.dtype:
        raise ValueError(f"gate and up must have one type, got {gate.dtype} and {up.dtype}")
    _run(out.device, _msd.msd_mx_swiglu, pg, ldg, pu, ldu, TYPES[gate.dtype], out.desc)
    return out


def product(x, w, out):
    """out = x w^T of quantised rows x and weight w; returns out."""
    if x.device != w.device:
        raise ValueError(f"x is on {x.device}, w on {w.device}")
    p, ld = _float(out, (x.shape[0], w.shape[0]), x.device, "out")
    _run(x.device, _msd.msd_mx_product, x.desc, w.desc, p, TYPES[out.dtype], ld)
    return out
