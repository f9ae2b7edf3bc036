"""The 4-bit operators of the draft head, as cases that can be timed and compared.

A case is one pass through one operator on matrices of the sizes that the
benchmark's and the tests' models have:

  quantise  float rows to microscaled 4-bit (E2M1) blocks of 32, and back: one
            term (weights) or two (activations, hi + lo)
  norm      x + y, its root-mean-square norm times a gain, in two 4-bit terms
  swiglu    silu(gate) * up, in two 4-bit terms
  product   Y = X W^T of quantised activations and weights

Where `own` is false `run` computes them from elementary torch operations.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BLOCK = 32
EPS = 1e-5


# --- the cases ---------------------------------------------------------------------------


def listed():
    return [
        # features of one round of a dynamic tree (ten nodes), before the LM head
        dict(name="quantise-round", op="quantise", rows=10, cols=4096, type="f32", terms=2,
             weight=False, pad=0),
        # f_down of the 7B-shaped draft, laid out once or after a training step
        dict(name="quantise-f-down", op="quantise", rows=4096, cols=8192, type="bf16", terms=1,
             weight=True, pad=0),
        # rows of an odd prompt inside wider rows, a width that ends inside a block
        dict(name="quantise-odd", op="quantise", rows=1151, cols=5101, type="f16", terms=1,
             weight=False, pad=19),
        # the norm of a verify-sized round (Qwen-shaped width)
        dict(name="norm-round", op="norm", rows=26, cols=3584, type="bf16", y=True),
        # of a prompt with a 2,880-row visual prefix
        dict(name="norm-prompt", op="norm", rows=3136, cols=4096, type="f32", y=True),
        # the FFN of a tree round, and of a 640-row prompt
        dict(name="swiglu-round", op="swiglu", rows=10, cols=11008, type="f32"),
        dict(name="swiglu-prompt", op="swiglu", rows=640, cols=11008, type="f32"),
        # one row (the root of a chain tree) against a square weight
        dict(name="product-one-row", op="product", rows=1, n=4096, k=4096, type="f32", terms=2),
        # the LM head over a round's ten rows
        dict(name="product-lm-head", op="product", rows=10, n=32000, k=4096, type="f32", terms=2),
        # gate and up over a 60-node tree
        dict(name="product-tree", op="product", rows=60, n=22016, k=4096, type="bf16", terms=2),
        # gate and up over a 640-row prompt
        dict(name="product-prompt", op="product", rows=640, n=22016, k=4096, type="f32", terms=2),
        # down over a long prompt, one-term activations
        dict(name="product-long", op="product", rows=3136, n=4096, k=11008, type="bf16", terms=1),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["quantise", "norm", "swiglu", "product", "product"])
    t = rng.choice(["f32", "bf16", "f16"])
    if op == "quantise":
        weight = rng.random() < 0.4
        cols = _log(rng, 1, 18944)
        rows = _log(rng, 1, min(32000, max(1, (1 << 25) // cols)))
        return dict(op=op, rows=rows, cols=cols, type=t, terms=1 if weight else rng.choice([1, 2]),
                    weight=weight, pad=rng.choice([0, 0, 1, 8, 40]))
    if op == "norm":
        return dict(op=op, rows=_log(rng, 1, 3136), cols=_log(rng, 8, 8192), type=t,
                    y=rng.random() < 0.8)
    if op == "swiglu":
        return dict(op=op, rows=_log(rng, 1, 2048), cols=_log(rng, 8, 18944), type=t)
    while True:
        rows, n, k = _log(rng, 1, 3136), _log(rng, 17, 152064), _log(rng, 32, 18944)
        if n * k <= 32000 * 4096 and rows * n * k <= 3136 * 4096 * 11008 and rows * n <= 640 * 22016:
            return dict(op=op, rows=rows, n=n, k=k, type=rng.choice(["f32", "bf16"]),
                        terms=rng.choice([1, 2, 2]))


def work(case):
    R, s = case["rows"], 4 if case["type"] == "f32" else 2
    q = 0.5 + 1.0 / BLOCK  # bytes of a 4-bit value with its share of the scale
    if case["op"] == "product":
        n, k = case["n"], case["k"]
        return dict(bytes=(R * case["terms"] + n) * k * q + R * n * s, flops=2.0 * R * n * k)
    C = case["cols"]
    if case["op"] == "quantise":
        back = 4 if case["terms"] == 2 else 2
        return dict(bytes=R * C * (s + back), flops=6.0 * R * C * case["terms"])
    if case["op"] == "norm":
        return dict(bytes=R * C * (s * (3 if case["y"] else 2) + 2) + 2 * C, flops=18.0 * R * C)
    return dict(bytes=R * C * (2 * s + 2), flops=18.0 * R * C)


# --- inputs ------------------------------------------------------------------------------


def _inputs(case, seed):
    """The float inputs of a case.  Activations: normal values on rows of
    different size with a few columns that stand out, as residual streams have."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = DTYPES[case["type"]]

    def normal(rows, cols, scale):
        return torch.randn(rows, cols, generator=g, device="cuda") * scale

    def activations(rows, cols):
        size = torch.exp2(torch.rand(rows, 1, generator=g, device="cuda") * 4 - 2)
        out = torch.rand(cols, generator=g, device="cuda") < 0.004
        return normal(rows, cols, 1.0) * size * torch.where(out, 20.0, 1.0)

    R = case["rows"]
    if case["op"] == "product":
        return dict(x=activations(R, case["k"]),
                    w=normal(case["n"], case["k"], 0.02).to(torch.bfloat16))
    C = case["cols"]
    if case["op"] == "quantise":
        x = normal(R, C, 0.02) if case["weight"] else activations(R, C)
        wide = torch.zeros(R, C + case["pad"], dtype=t, device="cuda")
        wide[:, :C] = x
        return dict(x=wide[:, :C])
    if case["op"] == "norm":
        gain = (1 + 0.1 * torch.randn(C, generator=g, device="cuda")).to(torch.bfloat16)
        return dict(x=activations(R, C).to(t), gain=gain,
                    y=normal(R, C, 0.5).to(t) if case["y"] else None)
    gu = normal(R, 2 * C, 1.5).to(t)  # gate and up side by side, as one product leaves them
    return dict(gate=gu[:, :C], up=gu[:, C:])


def prepare(case, seed):
    st = dict(_inputs(case, seed), case=case)
    R, t = case["rows"], DTYPES[case["type"]]
    if own:
        # the buffers that a program keeps, and a product's operands as the
        # operators before it and the loading of the weights leave them
        from paper_2505_14260_amd import mx
        if case["op"] == "product":
            n, k = case["n"], case["k"]
            x = mx.MX(R, k, terms=case["terms"])
            w = mx.MX(n, k, layout="weight")
            mx.quantize(st.pop("x"), x)
            mx.quantize(st.pop("w"), w)
            return dict(st, x=x, w=w, out=torch.empty(R, n, dtype=t, device="cuda"))
        C = case["cols"]
        q = mx.MX(R, C, layout="weight" if case.get("weight") else "rows",
                  terms=case.get("terms", 2))
        back = torch.float32 if case["op"] == "quantise" and case["terms"] == 2 else torch.bfloat16
        st.update(q=q, back=torch.empty(R, C, dtype=back, device="cuda"))
        if case["op"] == "norm":
            st["sum"] = torch.empty_like(st["x"])
        return st
    if case["op"] == "product":
        return dict(case=case, x=_quantise(st["x"], case["terms"]),
                    w=_quantise(st["w"].float(), 1))
    return st


# --- the operators -----------------------------------------------------------------------


def _power(e):
    """2^e in float32 for whole e in [-127, 127], from its bits."""
    f = (e + 127).to(torch.int32)
    return torch.where(f > 0, f << 23, torch.full_like(f, 0x00400000)).view(torch.float32)


def _term(x):
    """One 4-bit term of float32 blocks [.., 32]: magnitudes and signs as whole
    numbers of half steps (int8) and the exponent of each block's scale."""
    amax = x.abs().amax(-1, keepdim=True)
    e = torch.frexp(amax)[1] - 3  # floor(log2 amax) - 2
    e = torch.where(amax > 0, e.clamp(-127, 127), torch.full_like(e, -127))
    a = x.abs() * _power(-e)
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    halves = torch.clamp(torch.round(a / step) * step, max=6.0) * 2
    return torch.copysign(halves, x).to(torch.int8), e.to(torch.int16)


def _values(term):
    h, e = term
    return h.float() * 0.5 * _power(e)


def _quantise(x, terms):
    """[(halves, exponents)] of the terms of float32 rows, in padded blocks."""
    x = torch.nn.functional.pad(x, (0, -x.shape[1] % BLOCK)).view(x.shape[0], -1, BLOCK)
    hi = _term(x)
    return [hi] if terms == 1 else [hi, _term(x - _values(hi))]


def _rows(q, cols):
    """The float32 values that quantised rows stand for."""
    v = _values(q[0])
    for t in q[1:]:
        v = v + _values(t)
    return v.view(v.shape[0], -1)[:, :cols]


def run(st):
    if own:
        return _run_own(st)
    case = st["case"]
    t = DTYPES[case["type"]]
    if case["op"] == "product":
        return (_rows(st["x"], case["k"]) @ _rows(st["w"], case["k"]).t()).to(t)
    C = case["cols"]
    if case["op"] == "quantise":
        back = torch.float32 if case["terms"] == 2 else torch.bfloat16
        return _rows(_quantise(st["x"].float(), case["terms"]), C).to(back)
    if case["op"] == "norm":
        s = st["x"].float() if st["y"] is None else st["x"].float() + st["y"].float()
        v = s * torch.rsqrt((s * s).mean(-1, keepdim=True) + EPS) * st["gain"].float()
        return dict(sum=s.to(t), norm=_rows(_quantise(v, 2), C).to(torch.bfloat16))
    gate = st["gate"].float()
    v = gate / (1 + torch.exp(-gate)) * st["up"].float()
    return _rows(_quantise(v, 2), C).to(torch.bfloat16)


def _run_own(st):
    from paper_2505_14260_amd import mx
    op = st["case"]["op"]
    if op == "product":
        return mx.product(st["x"], st["w"], st["out"])
    if op == "quantise":
        mx.quantize(st["x"], st["q"])
        return mx.dequantize(st["q"], st["back"])
    if op == "norm":
        mx.resid_norm(st["x"], st["y"], st["gain"], EPS, st["sum"], st["q"])
        return dict(sum=st["sum"], norm=mx.dequantize(st["q"], st["back"]))
    mx.swiglu(st["gate"], st["up"], st["q"])
    return mx.dequantize(st["q"], st["back"])


# --- the definition in 64 bits -----------------------------------------------------------


def _exact_term(x):
    """x: float64 [rows, cols]; the values of its 4-bit blocks."""
    rows, cols = x.shape
    nb = -(-cols // BLOCK)
    b = torch.zeros(rows, nb * BLOCK, dtype=torch.float64, device=x.device)
    b[:, :cols] = x
    b = b.view(rows, nb, BLOCK)
    top = b.abs().max(-1, keepdim=True).values
    # the largest power of two that is no larger than the block's largest value
    top = torch.where(top > 0, top, torch.full_like(top, 2.0 ** -200))
    p = top / torch.frexp(top).mantissa / 2
    scale = (p / 4).clamp(2.0 ** -127, 2.0 ** 127)
    a = b.abs() / scale
    grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device=x.device)
    code = torch.zeros_like(a, dtype=torch.int64)
    for i in range(7):  # between neighbours i and i + 1; a tie goes to the even one
        mid = (grid[i] + grid[i + 1]) / 2
        code += (a >= mid) if i % 2 else (a > mid)
    return (torch.sign(b) * grid[code] * scale).view(rows, -1)[:, :cols]


def _exact_quantised(x, terms):
    hi = _exact_term(x)
    return hi if terms == 1 else hi + _exact_term(x - hi)


def exact(case, seed):
    d = {k: v.double() if torch.is_tensor(v) else v for k, v in _inputs(case, seed).items()}
    if case["op"] == "product":
        return torch.mm(_exact_quantised(d["x"], case["terms"]), _exact_term(d["w"]).t())
    if case["op"] == "quantise":
        return _exact_quantised(d["x"], case["terms"])
    if case["op"] == "norm":
        s = d["x"] if d["y"] is None else d["x"] + d["y"]
        v = s / torch.sqrt(s.pow(2).sum(-1, keepdim=True) / s.shape[1] + EPS) * d["gain"]
        return dict(sum=s, norm=_exact_quantised(v, 2))
    return _exact_quantised(d["gate"] * torch.sigmoid(d["gate"]) * d["up"], 2)
