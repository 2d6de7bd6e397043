"""Cases of the language-model operators: low-rank adapters beside a shared projection (forward and backward), the AdamW
step over a tensor list with states in 32 or in 8 bits, and the gradient norm that clips it.

``run`` computes a case in plain torch operations, or, with ``own`` set, by the library's calls.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
BLOCK = 256                     # elements that share a scale of the 8-bit states
MU, MAX_NORM = 1e-3, 1.0
HYPER = dict(lr=1e-3, beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.1, step=12)


# ------------------------------------------------------------------ the cases

def listed():
    return [
        # the next token of one user through a gate projection of the 1500-wide LSTM language model: latency only
        dict(name="forward decode one", op="forward", type="bf16", k=1500, n=6000, rows=1, requests=1, adapters=1,
             rank_lo=8, rank_hi=8, idle=0, saved=False),
        # one decoding step of a serving batch: a token per request, two dozen adapters of several ranks, some requests without
        dict(name="forward decode mixed", op="forward", type="fp16", k=4096, n=4096, rows=64, requests=64, adapters=24,
             rank_lo=8, rank_hi=64, idle=8, saved=False),
        # prompts of very different lengths prefilled together, wide input layer
        dict(name="forward prefill ragged", op="forward", type="bf16", k=9216, n=4096, rows=6011, requests=37, adapters=9,
             rank_lo=16, rank_hi=16, idle=500, saved=False),
        # training forward in 32 bits: 20 sequences of 35 tokens into the decoder of the LSTM language model, h kept
        dict(name="forward decoder fp32", op="forward", type="fp32", k=1500, n=33278, rows=700, requests=20, adapters=4,
             rank_lo=12, rank_hi=12, idle=0, saved=True),
        # gradients of a single short sequence
        dict(name="backward one sequence", op="backward", type="fp32", k=1500, n=6000, rows=35, requests=1, adapters=1,
             rank_lo=8, rank_hi=8, idle=0),
        # a training batch of four tasks at once, square projection
        dict(name="backward four tasks", op="backward", type="bf16", k=4096, n=4096, rows=8192, requests=16, adapters=4,
             rank_lo=16, rank_hi=16, idle=0),
        # higher ranks of odd sizes, ragged sequences, rows whose stride is no multiple of 16 bytes
        dict(name="backward odd ranks", op="backward", type="fp16", k=1500, n=6000, rows=2777, requests=30, adapters=6,
             rank_lo=40, rank_hi=63, idle=200),
        # L step of the whole LSTM language model (135.9 M parameters) with the penalty gradient, states in 32 bits
        dict(name="adamw lstm 32", op="adamw", list="lstm", tensors=10, numel=135858000, grad="fp32", states=32, penalty=True, copy="none"),
        # the same model without penalty, 16-bit gradients and weight copies, states in 8 bits
        dict(name="adamw lstm 8", op="adamw", list="lstm", tensors=10, numel=135858000, grad="bf16", states=8, penalty=False, copy="bf16"),
        # the adapters of sixteen layers: 32 small tensors, latency
        dict(name="adamw adapters 8", op="adamw", list="adapters", tensors=32, numel=16 * 16 * 7500, grad="fp32", states=8, penalty=False, copy="bf16"),
        # clipping before each step: 58 small tensors with the penalty gradient
        dict(name="norm resnet56", op="norm", list="resnet56", tensors=58, numel=851504, grad="fp32", penalty=True),
        # clipping of the whole language model in 16-bit gradients
        dict(name="norm lstm", op="norm", list="lstm", tensors=10, numel=135858000, grad="bf16", penalty=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["forward", "forward", "backward", "backward", "adamw", "adamw", "norm"])
    if op in ("forward", "backward"):
        k, n = _log(rng, 64, 9216), _log(rng, 64, 9216)
        if rng.random() < 0.5:              # multiples of 128, as most models have them; otherwise any number
            k, n = -(-k // 128) * 128, -(-n // 128) * 128
        k, n = (x + 128 if x == 24 * 128 else x for x in (k, n))
        decode = op == "forward" and rng.random() < 0.5
        rows = _log(rng, 1, 512) if decode else _log(rng, 8, 8192)
        requests = rows if decode else min(rows, _log(rng, 1, 64))
        adapters = min(requests, _log(rng, 1, 64))
        lo = _log(rng, 1, 64)
        idle = min(rows - requests, rows // 7) if not decode else 0
        c = dict(op=op, type=rng.choice(["fp32", "fp16", "bf16", "bf16"]), k=k, n=n, rows=rows, requests=requests, adapters=adapters,
                 rank_lo=lo, rank_hi=min(64, lo + rng.randrange(0, 33)), idle=idle)
        if op == "forward":
            c["saved"] = rng.random() < 0.5
        return c
    tensors = _log(rng, 1, 300)
    c = dict(op=op, list="ragged", tensors=tensors, numel=max(tensors, _log(rng, 1000, 60000000)), grad=rng.choice(["fp32", "fp16", "bf16"]),
             penalty=rng.random() < 0.5)
    if op == "adamw":
        c.update(states=rng.choice([8, 32]), copy=rng.choice(["none", "fp16", "bf16"]))
    return c


# ------------------------------------------------------------------ layouts (from the case alone)

def ranks(case):
    lo, hi, d = case["rank_lo"], case["rank_hi"], case["adapters"]
    return [lo + (hi - lo) * a // max(1, d - 1) for a in range(d)]


def sizes(case):
    """Elements of each tensor of the list."""
    if case["list"] == "lstm":
        v, h = 33278, 1500
        return [v * h] + [4 * h * h, 4 * h * h, 4 * h, 4 * h] * 2 + [v * h]
    if case["list"] == "adapters":
        return [16 * 1500, 6000 * 16] * 16
    if case["list"] == "resnet56":
        out, cin = [16 * 27], 16
        for cout in (16, 32, 64):
            for b in range(9):
                out += [cout * (cin if b == 0 else cout) * 9, cout * cout * 9] + ([cout * cin] if b == 0 and cin != cout else [])
            cin = cout
        return out + [640]
    t, n = case["tensors"], case["numel"]
    share = np.random.RandomState(1000 + t).dirichlet([0.5] * t) if t > 1 else np.ones(1)
    return [1 + int(s * (n - t)) for s in share]


def spots(case):
    """Each tensor's place in a flat buffer, which starts at a multiple of BLOCK elements; and the buffer's length."""
    n = np.array(sizes(case), dtype=np.int64)
    room = -(-n // BLOCK) * BLOCK
    end = np.cumsum(room)
    return list(zip((end - room).tolist(), n.tolist())), int(end[-1])


def work(case):
    if case["op"] in ("forward", "backward"):
        e = 4 if case["type"] == "fp32" else 2
        r, live, k, n = ranks(case), case["rows"] - case["idle"], case["k"], case["n"]
        mean = sum(r) / len(r)
        weights = sum(r) * (k + n) * e
        if case["op"] == "forward":
            return {"bytes": live * k * e + weights + 2 * live * n * e + (4 * live * mean if case["saved"] else 0), "flops": 2 * live * mean * (k + n)}
        return {"bytes": live * (3 * k + n) * e + weights + 4 * live * mean + 4 * sum(r) * (k + n), "flops": 4 * live * mean * (k + n)}
    n, g = sum(sizes(case)), 4 if case["grad"] == "fp32" else 2
    if case["op"] == "norm":
        return {"bytes": n * (g + (12 if case["penalty"] else 0)) + 4 * case["tensors"], "flops": n * (2 + (4 if case["penalty"] else 0))}
    state = 16 if case["states"] == 32 else 4 + 16 / BLOCK
    return {"bytes": n * (8 + g + state + (8 if case["penalty"] else 0) + (0 if case["copy"] == "none" else 2)), "flops": n * (16 + (4 if case["penalty"] else 0))}


# ------------------------------------------------------------------ inputs

def _normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device=DEV)


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    return _prepare_rows(case, seed, gen) if case["op"] in ("forward", "backward") else _prepare_list(case, seed, gen)


def _prepare_rows(case, seed, gen):
    """A batch: its requests' lengths and adapters on the host, activations and adapters on the device."""
    rs = np.random.RandomState(seed % (1 << 32))
    k, n, rows, d, t = case["k"], case["n"], case["rows"], case["adapters"], TYPES[case["type"]]
    live = case["requests"]
    if case["requests"] == rows:                          # decoding: a token each, the last `idle` without an adapter
        length = np.ones(rows, dtype=np.int64)
        which = np.concatenate([np.arange(d), rs.randint(0, d, rows - d)])
        which[rows - case["idle"]:] = -1
    else:
        cut = np.sort(rs.choice(np.arange(1, rows - case["idle"]), live - 1, replace=False)) if live > 1 else np.zeros(0, dtype=np.int64)
        length = np.diff(np.concatenate([[0], cut, [rows - case["idle"]]]))
        which = np.concatenate([np.arange(d), rs.randint(0, d, live - d)])
        if case["idle"]:
            length, which = np.append(length, case["idle"]), np.append(which, -1)
        length, which = np.append(length, 0), np.append(which, 0)       # a request that has nothing to do this time
    order = rs.permutation(len(length))
    length, which = length[order].astype(np.int64), which[order].astype(np.int32)
    r = ranks(case)
    a = [(_normal(gen, r[i], k) / math.sqrt(k)).to(t) for i in range(d)]
    b = [(_normal(gen, n, r[i]) * 0.05).to(t) for i in range(d)]
    s = dict(case=case, length=length, which=which, rank=r, a=a, b=b, scale=[16.0 / (8 + i % 3 * 8) for i in range(d)], x=_normal(gen, rows, k).to(t))
    row_of = np.repeat(which, length)                     # the rows of each adapter, for the plain form
    s["rows_of"] = [torch.from_numpy(np.nonzero(row_of == i)[0]).to(DEV) for i in range(d)]
    if case["op"] == "forward":
        s["y"] = _normal(gen, rows, n).to(t)
        s["h"] = torch.zeros(rows, max(r), device=DEV) if case["saved"] else None
    else:
        s["dy"] = (_normal(gen, rows, n) * 0.01).to(t)
        s["dx"] = (_normal(gen, rows, k) * 0.01).to(t)
        s["h"] = torch.zeros(rows, max(r), device=DEV)
        for i, at in enumerate(s["rows_of"]):
            s["h"][at, :r[i]] = s["x"][at].float() @ a[i].float().t()
        s["da"] = [torch.zeros(r[i], k, device=DEV) for i in range(d)]
        s["db"] = [torch.zeros(n, r[i], device=DEV) for i in range(d)]
    return s


def _prepare_list(case, seed, gen):
    """A tensor list whose arrays lie in flat buffers: weights, gradients, and what the step keeps between calls."""
    spot, total = spots(case)
    real = torch.zeros(total, dtype=torch.bool, device=DEV)
    for at, n in spot:
        real[at:at + n] = True
    level = torch.empty(total // BLOCK, device=DEV).uniform_(-3.0, 0.0, generator=gen).exp().repeat_interleave(BLOCK)   # layers differ in size
    level[torch.rand(total // BLOCK, generator=gen, device=DEV).lt(0.03).repeat_interleave(BLOCK)] = 0.0     # embedding rows not in the batch
    grad = torch.where(real, _normal(gen, total) * 1e-2 * level, 0.0)
    s = dict(case=case, spot=spot, w=torch.where(real, _normal(gen, total) * 0.05, 0.0), grad=grad.to(TYPES[case["grad"]]), theta=None, lam=None)
    if case["penalty"]:
        s["theta"] = torch.where(s["w"].abs() > 0.06, s["w"], 0.0)
        s["lam"] = torch.where(real, _normal(gen, total) * 1e-4, 0.0)
    if case["op"] == "norm":
        s["grad_scale"], s["norms"], s["clip"] = 0.5, torch.zeros(len(spot), device=DEV), torch.zeros(4, device=DEV)
        return s
    m, v = grad * 0.2 + torch.where(real, _normal(gen, total) * 2e-3 * level, 0.0), (grad * grad * 0.3 + 2e-5 * level * level) * real
    s["grad_scale"] = 1.0
    s["clip"] = torch.tensor([1.6, 0.625, 1.0, 0.0], device=DEV)       # what condensa_grad_norm() left there: norm, coefficient, finite
    if case["states"] == 32:
        s["m"], s["v"] = m, v
    else:
        s["m"], s["m_scale"] = _encode(m, False)
        s["v"], s["v_scale"] = _encode(v.sqrt(), True)
    s["copy"] = None if case["copy"] == "none" else torch.zeros(total, dtype=TYPES[case["copy"]], device=DEV)
    return s


# ------------------------------------------------------------------ one pass

def run(state):
    op = state["case"]["op"]
    if own:
        return {"forward": _own_forward, "backward": _own_backward, "adamw": _own_adamw, "norm": _own_norm}[op](state)
    return {"forward": _plain_forward, "backward": _plain_backward, "adamw": _plain_adamw, "norm": _plain_norm}[op](state)


def _out_forward(s):
    return {"y": s["y"]} if s["h"] is None else {"y": s["y"], "h": s["h"]}


def _out_backward(s):
    """The gradients of all adapters, one after the other."""
    return {"dx": s["dx"], "da": torch.cat([g.view(-1) for g in s["da"]]), "db": torch.cat([g.view(-1) for g in s["db"]])}


def _out_adamw(s):
    out = {"w": s["w"], "m": s["m"], "v": s["v"]}
    if s["case"]["states"] == 8:
        out.update(m_scale=s["m_scale"], v_scale=s["v_scale"])
    if s["copy"] is not None:
        out["copy"] = s["copy"]
    return out


# -- plain forms

def _one_forward(s, i):
    at, r = s["rows_of"][i], s["rank"][i]
    h = s["x"][at].float() @ s["a"][i].float().t()
    s["y"][at] = (s["y"][at].float() + s["scale"][i] * (h @ s["b"][i].float().t())).to(s["y"].dtype)
    if s["h"] is not None:
        s["h"][at, :r] = h


def _plain_forward(s):
    [_one_forward(s, i) for i in range(len(s["a"]))]
    return _out_forward(s)


def _one_backward(s, i):
    at, r = s["rows_of"][i], s["rank"][i]
    dy, a, b = s["dy"][at].float(), s["a"][i].float(), s["b"][i].float()
    u = s["scale"][i] * (dy @ b)
    s["dx"][at] = (s["dx"][at].float() + u @ a).to(s["dx"].dtype)
    s["da"][i].copy_(u.t() @ s["x"][at].float())
    s["db"][i].copy_(s["scale"][i] * (dy.t() @ s["h"][at, :r]))


def _plain_backward(s):
    [_one_backward(s, i) for i in range(len(s["a"]))]
    return _out_backward(s)


def _gradient(s):
    """Loss gradient and penalty gradient, in 32 bits."""
    g = s["grad"].float() * s["grad_scale"]
    if s["theta"] is not None:
        g = g + ((s["w"] - s["theta"]) * MU - s["lam"])
    return g


def _encode(x, floor):
    """Blocks of 256 in E4M3 under a power of two; with `floor`, what is above zero stays above zero."""
    x = x.view(-1, BLOCK)
    most = x.abs().amax(dim=1, keepdim=True)
    e = ((most.view(torch.int32) >> 23) - 7).clamp(min=1)
    code = (x * ((254 - e) << 23).view(torch.float32)).to(torch.float8_e4m3fn)
    if floor:
        code = torch.where((x > 0) & (code.float() == 0), torch.full_like(x, 2.0 ** -9), code.float()).to(torch.float8_e4m3fn)
    return code.view(-1), (e << 23).view(torch.float32).view(-1)


def _decode(code, scale):
    return (code.float().view(-1, BLOCK) * scale.view(-1, 1)).view(-1)


def _plain_adamw(s):
    p, eight = HYPER, s["case"]["states"] == 8
    g = _gradient(s) * s["clip"][1]
    m, v = (_decode(s["m"], s["m_scale"]), _decode(s["v"], s["v_scale"]).square()) if eight else (s["m"], s["v"])
    m = m * p["beta1"] + g * float(np.float32(1) - np.float32(p["beta1"]))
    v = v * p["beta2"] + (g * g) * float(np.float32(1) - np.float32(p["beta2"]))
    root = v.sqrt()
    step = p["lr"] / (1 - p["beta1"] ** p["step"])
    w = s["w"] * (1 - p["lr"] * p["weight_decay"]) - (m / (root * (1 / math.sqrt(1 - p["beta2"] ** p["step"])) + p["eps"])) * step
    s["w"].copy_(w)
    if eight:
        (code, scale), (code2, scale2) = _encode(m, False), _encode(root, True)
        s["m"].copy_(code), s["m_scale"].copy_(scale), s["v"].copy_(code2), s["v_scale"].copy_(scale2)
    else:
        s["m"].copy_(m), s["v"].copy_(v)
    if s["copy"] is not None:
        s["copy"].copy_(w)
    return _out_adamw(s)


def _plain_norm(s):
    g = _gradient(s).square_()
    part = torch.stack([g[at:at + n].sum() for at, n in s["spot"]])
    norm = part.sum().sqrt()
    s["norms"].copy_(part.sqrt())
    s["clip"].copy_(torch.stack([norm, (MAX_NORM / (norm + 1e-6)).clamp(max=1.0), torch.isfinite(norm).float(), torch.zeros_like(norm)]))
    return {"norms": s["norms"], "clip": s["clip"]}


# -- the library's calls

_kept = {}


def _library():
    """The binding and the context that a program makes once."""
    if not _kept:
        from paper_1911_02497_b200 import cstep
        _kept.update(cstep=cstep, ctx=cstep.Context(torch.cuda.current_device()))
    return _kept["cstep"], _kept["ctx"]


def _adapters(s, lib):
    """The table of the adapters that are loaded; a program makes it when it loads them."""
    if "table" not in s:
        s["table"] = lib.adapter_table(s["a"], s["b"], s["scale"], s.get("da"), s.get("db"))
    return s["table"]


def _own_forward(s):
    lib, ctx = _library()
    ctx.adapter_forward(_adapters(s, lib), s["length"], s["which"], s["x"], s["y"], s["h"], stream=torch.cuda.current_stream())
    return _out_forward(s)


def _own_backward(s):
    lib, ctx = _library()
    ctx.adapter_backward(_adapters(s, lib), s["length"], s["which"], s["x"], s["dy"], s["h"], s["dx"], stream=torch.cuda.current_stream())
    return _out_backward(s)


def _list_table(s, lib):
    """The table of the parameter list; a program makes it when it makes its optimizer."""
    if "table" not in s:
        part = {}
        for key in ("w", "grad", "theta", "lam", "m", "v", "copy"):
            x = s.get(key)
            part[key] = None if x is None else [x[at:at + n] for at, n in s["spot"]]
        for key in ("m_scale", "v_scale"):
            x = s.get(key)
            part[key] = None if x is None else [x[at // BLOCK:-(-(at + n) // BLOCK)] for at, n in s["spot"]]
        s["table"] = lib.adamw_table(part["w"], part["grad"], part["m"], part["v"], part["m_scale"], part["v_scale"],
                                     theta=part["theta"], lam=part["lam"], w_h=part["copy"])
    return s["table"]


def _own_adamw(s):
    lib, ctx = _library()
    ctx.lstep_adamw(_list_table(s, lib), MU, clip=s["clip"], grad_scale=s["grad_scale"], stream=torch.cuda.current_stream(), **HYPER)
    return _out_adamw(s)


def _own_norm(s):
    lib, ctx = _library()
    ctx.grad_norm(_list_table(s, lib), MU, MAX_NORM, s["clip"], s["norms"], grad_scale=s["grad_scale"], stream=torch.cuda.current_stream())
    return {"norms": s["norms"], "clip": s["clip"]}


# ------------------------------------------------------------------ the definition in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    f64 = torch.float64
    if case["op"] in ("forward", "backward"):
        row_of = np.repeat(s["which"], s["length"])
        if case["op"] == "forward":
            y, h = s["y"].to(f64), torch.zeros(case["rows"], max(s["rank"]), dtype=f64, device=DEV)
            for i, a in enumerate(s["a"]):
                at = torch.from_numpy(np.flatnonzero(row_of == i)).to(DEV)
                h[at, :s["rank"][i]] = torch.einsum("mk,rk->mr", s["x"][at].to(f64), a.to(f64))
                y[at] += s["scale"][i] * torch.einsum("mr,nr->mn", h[at, :s["rank"][i]], s["b"][i].to(f64))
            return {"y": y, "h": h} if case["saved"] else {"y": y}
        dx, da, db = s["dx"].to(f64), [], []
        for i, a in enumerate(s["a"]):
            at = torch.from_numpy(np.flatnonzero(row_of == i)).to(DEV)
            dy = s["dy"][at].to(f64)
            u = torch.einsum("mn,nr->mr", dy, s["b"][i].to(f64)) * s["scale"][i]
            dx[at] += torch.einsum("mr,rk->mk", u, a.to(f64))
            da.append(torch.einsum("mr,mk->rk", u, s["x"][at].to(f64)).reshape(-1))
            db.append(torch.einsum("mn,mr->nr", dy, s["h"][at, :s["rank"][i]].to(f64)).reshape(-1) * s["scale"][i])
        return {"dx": dx, "da": torch.cat(da), "db": torch.cat(db)}
    g = s["grad"].to(f64) * s["grad_scale"]
    if case["penalty"]:
        g += MU * (s["w"].to(f64) - s["theta"].to(f64)) - s["lam"].to(f64)
    if case["op"] == "norm":
        norms = torch.stack([torch.linalg.vector_norm(g[at:at + n]) for at, n in s["spot"]])
        norm = torch.linalg.vector_norm(norms)
        return {"norms": norms, "clip": torch.stack([norm, torch.clamp(MAX_NORM / (norm + 1e-6), max=1.0), torch.ones_like(norm), torch.zeros_like(norm)])}
    g *= float(s["clip"][1])
    p, eight = HYPER, case["states"] == 8
    if eight:
        wide = [s[x].to(f64) for x in ("m_scale", "v_scale")]
        m = s["m"].to(f64) * wide[0].repeat_interleave(BLOCK)
        v = (s["v"].to(f64) * wide[1].repeat_interleave(BLOCK)) ** 2
    else:
        m, v = s["m"].to(f64), s["v"].to(f64)
    m = p["beta1"] * m + (1 - p["beta1"]) * g
    v = p["beta2"] * v + (1 - p["beta2"]) * g ** 2
    hat_m, hat_v = m / (1 - p["beta1"] ** p["step"]), v / (1 - p["beta2"] ** p["step"])
    w = s["w"].to(f64) * (1 - p["lr"] * p["weight_decay"]) - p["lr"] * hat_m / (hat_v.sqrt() + p["eps"])
    out = {"w": w, "m": m, "v": v}
    if case["copy"] != "none":
        out["copy"] = w.clone()
    if eight:
        for key, x in (("m", m), ("v", v.sqrt())):
            most = x.view(-1, BLOCK).abs().amax(dim=1)
            scale = torch.exp2((torch.frexp(most)[1] - 8).clamp(min=-126).to(f64))
            out[key], out[key + "_scale"] = x / scale.repeat_interleave(BLOCK), None
    return out
