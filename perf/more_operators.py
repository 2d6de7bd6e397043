"""Cases of the projection in 8 bits and of what surrounds it: the product of E4M3 rows with an E4M3 matrix (forward, and
backward to the rows), the root-mean-square norm with the residual's addition and an 8-bit output (forward and backward), and
the encoders of rows and of weight blocks.

``run`` computes a case in plain torch operations, or, with ``own`` set, by the library's calls.
"""
import math

import torch

own = False

DEV = "cuda"
TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
GROUP = 128                     # columns that share a scale; blocks of weights are 128 x 128
EPS = 1e-5


# ------------------------------------------------------------------ the cases

def listed():
    return [
        # the next token of one user through a gate projection of the 1500-wide LSTM language model: latency only
        dict(name="projection one token", op="forward", type="bf16", rows=1, k=1500, n=6000),
        # prompts of several users prefilled together through a wide projection; rows are no multiple of any tile
        dict(name="projection prefill", op="forward", type="bf16", rows=6011, k=9216, n=4096),
        # gradient through the decoder of the LSTM language model, 20 sequences of 35 tokens: a long sum, few outputs
        dict(name="gradient decoder", op="backward", type="fp16", rows=700, k=1500, n=33278),
        # gradient through a square projection for a training batch
        dict(name="gradient batch", op="backward", type="bf16", rows=8192, k=4096, n=4096),
        # the norm ahead of that gate projection for one token, 8-bit rows only
        dict(name="norm one token", op="norm", type="bf16", gain="fp32", rows=1, cols=1500, residual=True, plain=False, coded=True, saved=False),
        # the norm of a training batch: residual stream, 16-bit and 8-bit rows, what backward needs
        dict(name="norm batch", op="norm", type="bf16", gain="bf16", rows=8192, cols=4096, residual=True, plain=True, coded=True, saved=True),
        # gradient of a norm for one sequence of 35 tokens in 32 bits
        dict(name="norm gradient sequence", op="norm_back", type="fp32", gain="fp32", rows=35, cols=1500, joined=False, coded=False),
        # gradient of a norm for a training batch, joined with the residual stream's, also in 8 bits for the projection before
        dict(name="norm gradient batch", op="norm_back", type="bf16", gain="bf16", rows=8192, cols=4096, joined=True, coded=True),
        # a decoding batch's activations into a wide projection
        dict(name="rows decode", op="rows", type="fp16", rows=64, cols=9216),
        # gradients of a training batch at the gates' width
        dict(name="rows batch", op="rows", type="bf16", rows=8192, cols=6000),
        # a gate projection as a C-step leaves it, with the values that the codes stand for
        dict(name="blocks gate", op="blocks", type="fp32", n=6000, k=1500, values=True),
        # the decoder of the LSTM language model from its 16-bit copy
        dict(name="blocks decoder", op="blocks", type="bf16", n=33278, k=1500, values=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["forward", "forward", "backward", "norm", "norm_back", "rows", "blocks"])
    if op in ("forward", "backward", "blocks"):
        k, n = _log(rng, 64, 9216), _log(rng, 64, 9216)
        if rng.random() < 0.5:              # multiples of 128, as most models have them; otherwise any number
            k, n = -(-k // 128) * 128, -(-n // 128) * 128
        if op == "blocks":
            return dict(op=op, type=rng.choice(["fp32", "fp16", "bf16"]), n=n, k=k, values=rng.random() < 0.5)
        rows = min(_log(rng, 1, 8192), 220000000000 // (n * k))
        return dict(op=op, type=rng.choice(["fp16", "bf16"]), rows=rows, k=k, n=n)
    cols = _log(rng, 16, 16384)
    if rng.random() < 0.5:
        cols = -(-cols // 64) * 64
    c = dict(op=op, type=rng.choice(["fp32", "fp16", "bf16", "bf16"]), rows=min(_log(rng, 1, 16384), 16000000 // cols), cols=cols)
    if op != "rows":
        c["gain"] = rng.choice(["fp32", c["type"]])
    if op == "norm":
        what = rng.choice(["plain", "coded", "both"])
        c.update(residual=rng.random() < 0.6, plain=what != "coded", coded=what != "plain", saved=rng.random() < 0.5)
    if op == "norm_back":
        c.update(joined=rng.random() < 0.6, coded=rng.random() < 0.5)
    return c


def work(case):
    size = 4 if case["type"] == "fp32" else 2
    if case["op"] in ("forward", "backward"):
        rows, k, n = case["rows"], case["k"], case["n"]
        deep, wide = (k, n) if case["op"] == "forward" else (n, k)
        return {"bytes": n * k + rows * deep * (1 + 1 / GROUP) + n * k / GROUP ** 2 + 2 * rows * wide, "flops": 2 * rows * n * k}
    if case["op"] == "blocks":
        return {"bytes": case["n"] * case["k"] * (size + 1 + 1 / GROUP ** 2 + (4 if case["values"] else 0)), "flops": 3 * case["n"] * case["k"]}
    rows, cols = case["rows"], case["cols"]
    coded = 1 + 1 / GROUP if case["op"] == "rows" or case["coded"] else 0
    if case["op"] == "rows":
        return {"bytes": rows * cols * (size + coded), "flops": 3 * rows * cols}
    gain = cols * (4 if case["gain"] == "fp32" else 2)
    if case["op"] == "norm":
        each = size * (1 + 2 * case["residual"] + case["plain"]) + coded
        return {"bytes": rows * cols * each + gain + 4 * rows * case["saved"], "flops": rows * cols * (4 + 3 * case["coded"])}
    return {"bytes": rows * cols * (size * (3 + case["joined"]) + coded) + gain + 4 * cols + 4 * rows, "flops": rows * cols * (10 + 3 * case["coded"])}


# ------------------------------------------------------------------ inputs

def _coded(rows, cols, scale_rows):
    """Room for an 8-bit matrix: codes whose rows lie a multiple of 16 bytes apart, scales whose rows lie whole words apart."""
    codes = torch.zeros(rows, -(-cols // 16) * 16, dtype=torch.uint8, device=DEV)[:, :cols].view(torch.float8_e4m3fn)
    groups = -(-cols // GROUP)
    return dict(codes=codes, scales=torch.zeros(scale_rows, -(-groups // 4) * 4, dtype=torch.uint8, device=DEV)[:, :groups])


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    normal = lambda *shape: torch.randn(*shape, generator=gen, device=DEV)
    s = dict(case=case)
    t = TYPES[case["type"]]
    if case["op"] in ("forward", "backward", "blocks"):
        n, k = case["n"], case["k"]
        w = normal(n, k) * (1.0 / math.sqrt(k))
        w *= normal(n, k).abs() > 0.67                  # half of it has been pruned
        if case["op"] == "blocks":
            s.update(w=w.to(t), out=_coded(n, k, -(-n // GROUP)), theta=torch.zeros(n, k, device=DEV) if case["values"] else None)
            return s
        deep, wide = (k, n) if case["op"] == "forward" else (n, k)
        s["w"] = _coded(n, k, -(-n // GROUP))
        _write(s["w"], *_encode_blocks(w))
        x = normal(case["rows"], deep) * normal(deep).exp()      # columns of very different size
        s["x"] = _coded(case["rows"], deep, case["rows"])
        _write(s["x"], *_encode_rows(x))
        s["y"] = torch.zeros(case["rows"], wide, dtype=t, device=DEV)
        return s
    rows, cols = case["rows"], case["cols"]
    stream = lambda: (normal(rows, cols) * (normal(cols) * 0.7).exp() * (normal(rows, 1) * 0.5).exp()).to(t)
    if case["op"] == "rows":
        s.update(x=stream(), out=_coded(rows, cols, rows))
        return s
    s["gain"] = (1.0 + 0.2 * normal(cols)).to(TYPES[case["gain"]])
    s["out"] = _coded(rows, cols, rows) if case["coded"] else None
    if case["op"] == "norm":
        s.update(x=stream(), residual=None, h=None, y=None, rstd=None)
        if case["residual"]:
            s.update(residual=stream(), h=torch.zeros(rows, cols, dtype=t, device=DEV))
        if case["plain"]:
            s["y"] = torch.zeros(rows, cols, dtype=t, device=DEV)
        if case["saved"]:
            s["rstd"] = torch.zeros(rows, device=DEV)
        return s
    s["h"] = stream()
    s["rstd"] = (s["h"].double().square().mean(dim=1) + EPS).rsqrt().float()
    s["dy"] = (normal(rows, cols) * 0.01).to(t)
    s["dh"] = (normal(rows, cols) * 0.02).to(t) if case["joined"] else None
    s["dx"] = torch.zeros(rows, cols, dtype=t, device=DEV)
    s["dgain"] = torch.zeros(cols, device=DEV)
    return s


# ------------------------------------------------------------------ one pass

def run(state):
    op = state["case"]["op"]
    if own:
        return {"forward": _own_forward, "backward": _own_backward, "norm": _own_norm, "norm_back": _own_norm_back, "rows": _own_rows, "blocks": _own_blocks}[op](state)
    return {"forward": _plain_forward, "backward": _plain_backward, "norm": _plain_norm, "norm_back": _plain_norm_back, "rows": _plain_rows,
            "blocks": _plain_blocks}[op](state)


def _out(s, *names):
    """What a pass wrote; an 8-bit matrix as the E4M3 values of its codes and the powers of two of its scales."""
    out = {name: s[name] for name in names if s.get(name) is not None}
    if s.get("out") is not None:
        out.update(codes=s["out"]["codes"], scales=s["out"]["scales"].view(torch.float8_e8m0fnu))
    return out


# -- plain forms

def _power(scales):
    """2^(s - 127) of scale bytes 1 .. 254."""
    return (scales.int() << 23).view(torch.float32)


def _scale_of(most):
    """The least s, at least 1, with most <= 448 * 2^(s - 127)."""
    m, e = torch.frexp(most)
    s = e - 9 + 127 + (m > 0.875)
    return torch.where(most > 0, s, 1).clamp(min=1)


def _codes_of(x, s):
    return (x * torch.ldexp(torch.ones_like(x[:1, :1]), 127 - s)).to(torch.float8_e4m3fn)


def _encode_rows(x):
    pad = torch.nn.functional.pad(x.abs(), (0, -x.shape[1] % GROUP))
    s = _scale_of(pad.view(x.shape[0], -1, GROUP).amax(dim=2))
    return _codes_of(x, s.repeat_interleave(GROUP, dim=1)[:, :x.shape[1]]), s


def _encode_blocks(w):
    pad = torch.nn.functional.pad(w.abs(), (0, -w.shape[1] % GROUP, 0, -w.shape[0] % GROUP))
    s = _scale_of(pad.view(pad.shape[0] // GROUP, GROUP, -1, GROUP).amax(dim=(1, 3)))
    return _codes_of(w, s.repeat_interleave(GROUP, dim=0)[:w.shape[0]].repeat_interleave(GROUP, dim=1)[:, :w.shape[1]]), s


def _write(m, codes, s):
    m["codes"].view(torch.uint8).copy_(codes.view(torch.uint8))
    m["scales"].copy_(s)


def _row_values(m):
    return m["codes"].float() * _power(m["scales"]).repeat_interleave(GROUP, dim=1)[:, :m["codes"].shape[1]]


def _block_values(m):
    n, k = m["codes"].shape
    return m["codes"].float() * _power(m["scales"]).repeat_interleave(GROUP, dim=0)[:n].repeat_interleave(GROUP, dim=1)[:, :k]


def _plain_forward(s):
    s["y"].copy_(_row_values(s["x"]) @ _block_values(s["w"]).t())
    return {"y": s["y"]}


def _plain_backward(s):
    s["y"].copy_(_row_values(s["x"]) @ _block_values(s["w"]))
    return {"y": s["y"]}


def _plain_norm(s):
    """In 64 bits: where the largest of a group lies next to a border of its scale, 32 would take the other side."""
    h = s["x"]
    if s["residual"] is not None:
        h = (s["x"].float() + s["residual"].float()).to(h.dtype)
        s["h"].copy_(h)
    h = h.double()
    rstd = (h.square().mean(dim=1, keepdim=True) + EPS).rsqrt()
    y = h * rstd * s["gain"].double()
    if s["y"] is not None:
        s["y"].copy_(y)
    if s["rstd"] is not None:
        s["rstd"].copy_(rstd[:, 0])
    if s["out"] is not None:
        _write(s["out"], *_encode_rows(y))
    return _out(s, "h", "y", "rstd")


def _plain_norm_back(s):
    """In 64 bits, for the borders and the long sums over rows."""
    dy, rstd = s["dy"].double(), s["rstd"].double()[:, None]
    unit = s["h"].double() * rstd
    t = dy * s["gain"].double()
    dx = rstd * (t - unit * (t * unit).mean(dim=1, keepdim=True))
    if s["dh"] is not None:
        dx = dx + s["dh"].double()
    s["dx"].copy_(dx)
    s["dgain"].copy_((dy * unit).sum(dim=0))
    if s["out"] is not None:
        _write(s["out"], *_encode_rows(dx))
    return _out(s, "dx", "dgain")


def _plain_rows(s):
    _write(s["out"], *_encode_rows(s["x"].float()))
    return _out(s)


def _plain_blocks(s):
    _write(s["out"], *_encode_blocks(s["w"].float()))
    if s["theta"] is not None:
        s["theta"].copy_(_block_values(s["out"]))
    return _out(s, "theta")


# -- the library's calls

_kept = {}


def _library():
    """The binding and the context that a program makes once."""
    if not _kept:
        from paper_1911_02497_b200 import cstep
        _kept.update(cstep=cstep, ctx=cstep.Context(torch.cuda.current_device()))
    return _kept["cstep"], _kept["ctx"]


def _matrix(s, key, lib, blocks=False):
    """The binding's description of an 8-bit matrix; a program makes it with the buffers."""
    if s.get(key) is None:
        return None
    if "matrix" not in s[key]:
        s[key]["matrix"] = (lib.coded_blocks if blocks else lib.coded_rows)(s[key]["codes"], s[key]["scales"])
    return s[key]["matrix"]


def _own_forward(s):
    lib, ctx = _library()
    ctx.projection_forward(_matrix(s, "w", lib, True), _matrix(s, "x", lib), s["y"], stream=torch.cuda.current_stream())
    return {"y": s["y"]}


def _own_backward(s):
    lib, ctx = _library()
    ctx.projection_backward(_matrix(s, "w", lib, True), _matrix(s, "x", lib), s["y"], stream=torch.cuda.current_stream())
    return {"y": s["y"]}


def _own_norm(s):
    lib, ctx = _library()
    ctx.norm_forward(s["x"], s["gain"], EPS, residual=s["residual"], h=s["h"], y=s["y"], code=_matrix(s, "out", lib), rstd=s["rstd"],
                     stream=torch.cuda.current_stream())
    return _out(s, "h", "y", "rstd")


def _own_norm_back(s):
    lib, ctx = _library()
    ctx.norm_backward(s["dy"], s["h"], s["gain"], s["rstd"], dh=s["dh"], dx=s["dx"], code=_matrix(s, "out", lib), dgain=s["dgain"],
                      stream=torch.cuda.current_stream())
    return _out(s, "dx", "dgain")


def _own_rows(s):
    lib, ctx = _library()
    ctx.encode_rows(s["x"], _matrix(s, "out", lib), stream=torch.cuda.current_stream())
    return _out(s)


def _own_blocks(s):
    lib, ctx = _library()
    ctx.encode_blocks(s["w"], _matrix(s, "out", lib, True), theta=s["theta"], stream=torch.cuda.current_stream())
    return _out(s, "theta")


# ------------------------------------------------------------------ the definition in 64 bits

def _exact_codes(v, high, wide):
    """v over the power of two of its group of `high` x `wide` values, before it is rounded; and that power."""
    n, k = v.shape
    most = torch.zeros(-(-n // high) * high, -(-k // wide) * wide, dtype=torch.float64, device=DEV)
    most[:n, :k] = v.abs()
    most = most.unflatten(1, (-1, wide)).amax(dim=2).unflatten(0, (-1, high)).amax(dim=1)
    p = torch.ceil(torch.log2(most / 448.0)).clamp(min=-126)
    p = torch.where(most <= 448.0 * torch.exp2(p - 1), p - 1, torch.where(most > 448.0 * torch.exp2(p), p + 1, p)).clamp(min=-126)     # (log2 is rounded)
    p = torch.exp2(p)[torch.arange(n, device=DEV) // high][:, torch.arange(k, device=DEV) // wide]
    return v / p, p


def _exact_rounded(q):
    """The E4M3 value nearest to q, of two the even one: three bits behind the leading one, none below 2^-9."""
    step = torch.exp2((torch.frexp(q)[1] - 4).clamp(min=-9).to(q.dtype))
    return torch.round(q / step) * step


def _exact_values(m, high):
    codes, p = m["codes"].to(torch.float64), torch.exp2(m["scales"].to(torch.float64) - 127.0)
    n, k = codes.shape
    return codes * p[torch.arange(n, device=DEV) // high][:, torch.arange(k, device=DEV) // GROUP]


def exact(case, seed):
    s = prepare(case, seed)
    f64 = torch.float64
    op = case["op"]
    if op in ("forward", "backward"):
        return {"y": torch.einsum("mk,nk->mn" if op == "forward" else "mk,kn->mn", _exact_values(s["x"], 1), _exact_values(s["w"], GROUP))}
    if op == "rows":
        return {"codes": _exact_codes(s["x"].to(f64), 1, GROUP)[0], "scales": None}
    if op == "blocks":
        codes, p = _exact_codes(s["w"].to(f64), GROUP, GROUP)
        out = {"codes": codes, "scales": None}
        return dict(out, theta=_exact_rounded(codes) * p) if case["values"] else out
    if op == "norm":
        out, h = {}, s["x"].to(f64)
        if case["residual"]:
            h = h + s["residual"].to(f64)
            out["h"] = h
            h = h.to(s["x"].dtype).to(f64)
        rstd = 1.0 / torch.sqrt(torch.linalg.vector_norm(h, dim=1) ** 2 / case["cols"] + EPS)
        y = torch.einsum("mn,m,n->mn", h, rstd, s["gain"].to(f64))
        out.update({"y": y} if case["plain"] else {}, **({"rstd": rstd} if case["saved"] else {}))
    else:
        dy, h, g, rstd = s["dy"].to(f64), s["h"].to(f64), s["gain"].to(f64), s["rstd"].to(f64)
        q = torch.einsum("mn,n,mn->m", dy, g, h) / case["cols"]
        y = rstd[:, None] * (dy * g) - (rstd ** 3 * q)[:, None] * h
        y = y + s["dh"].to(f64) if case["joined"] else y
        out = {"dx": y, "dgain": torch.einsum("mn,mn,m->n", dy, h, rstd)}
    return dict(out, codes=_exact_codes(y, 1, GROUP)[0], scales=None) if case["coded"] else out
