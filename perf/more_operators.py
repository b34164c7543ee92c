"""Performance cases of a refiner's feed-forward block and of the optimizer's step, one operator a pass.

listed() names the cases; draw() gives further ones of the same ranges. Every
case is one of five operations:

  gated        dlm_gated_linear: both projections of a gated feed-forward block,
               the activation and the product; with `keep`, gate and up for the
               backward pass beside it
  gated_grad   dlm_gated_linear_grad: its gradients of the input and both weights
  linear       dlm_linear: a projection with bias, activation and residual
  linear_grad  dlm_linear_grad: its gradients of the input, the weight and the bias
  adamw        dlm_adamw: a step over many tensors, states in 32 bits or in 8

The width is that of the package's workloads (d = 2048, batches of up to 32 x 512
positions), the inner width four times that; odd and small ones come from the
tests' kind (d = 64, 200), the rest are generic ones between them.
"""
import math

import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
_ACTS = {"none": 0, "silu": 1, "gelu": 2}
_D, _F = 2048, 8192
_V = 151552                        # the workloads' vocabulary
_MOST = 16384 * _F * _D            # rows x inner width x width of the largest listed products
_MOST_ADAMW = _V * _D              # elements of the largest set of tensors
_BLOCK = 256                       # elements that share a scale of 8-bit states
_TOP = 448.0                       # the largest e4m3 value


def listed():
    return [
        # One position of one sequence: both weights are read once.
        dict(name="gated_1", op="gated", N=1, d=_D, f=_F, act="silu", keep=False),
        # A few odd rows through a small block, every tile ragged, kept for training.
        dict(name="gated_odd_517", op="gated", N=517, d=200, f=1000, act="gelu", keep=True),
        # A batch of 32 x 512 positions.
        dict(name="gated_32x512", op="gated", N=16384, d=_D, f=_F, act="silu", keep=False),
        # Gradients of one local window of 64 positions: bound by the weights and their gradients.
        dict(name="gated_grad_64", op="gated_grad", N=64, d=_D, f=_F, act="silu", add=True),
        # The training batch's gradients: bound by the tensor cores.
        dict(name="gated_grad_32x512", op="gated_grad", N=16384, d=_D, f=_F, act="silu", add=False),
        # The block's second projection at one position, added to what goes around the block.
        dict(name="linear_1", op="linear", N=1, k=_F, m=_D, act="none", bias="none", residual=True, keep=False),
        # The same of a batch.
        dict(name="linear_32x512", op="linear", N=16384, k=_F, m=_D, act="none", bias="f32", residual=True, keep=False),
        # Gradients of a small projection with an activation, odd in every size.
        dict(name="linear_grad_odd_517", op="linear_grad", N=517, k=200, m=1000, act="gelu", bias="f32", add=False),
        # Gradients of the first projection of a block without a gate, a training batch.
        dict(name="linear_grad_32x512", op="linear_grad", N=16384, k=_D, m=_F, act="gelu", bias="bf16", add=True),
        # Norm weights and biases: latency.
        dict(name="adamw_small", op="adamw", tensors=20, largest=2048, params="f32", grads="f32", bits=32, clip=False),
        # The output projection and what is beside it: bf16 weights, their values in 32 bits.
        dict(name="adamw_head", op="adamw", tensors=3, largest=_V * _D // 2, params="master", grads="bf16", bits=32, clip=True),
        # The same with states in 8 bits, the weights in bf16 alone.
        dict(name="adamw_head_8bit", op="adamw", tensors=3, largest=_V * _D // 2, params="bf16", grads="bf16", bits=8, clip=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["gated", "gated", "gated_grad", "gated_grad", "linear", "linear", "linear_grad", "adamw", "adamw"])
    if op == "adamw":
        n = _log(rng, 1, 10)
        bits = rng.choice([32, 8])
        return dict(op=op, tensors=n, largest=_log(rng, 100, _MOST_ADAMW // (2 * min(n, 4))),
                    params=rng.choice(["f32", "bf16", "master"]), grads=rng.choice(["bf16", "f32"]), bits=bits,
                    clip=rng.random() < 0.5)
    a = rng.choice([_D, 64, 8 * _log(rng, 4, 512), 8 * _log(rng, 4, 512)])
    b = rng.choice([_F, 4 * a, 8 * _log(rng, 8, 1500), 8 * _log(rng, 8, 1500)])
    N = _log(rng, 1, max(1, min(16384, _MOST // (a * b))))
    if op == "gated":
        return dict(op=op, N=N, d=a, f=b, act=rng.choice(["silu", "gelu"]), keep=rng.random() < 0.5)
    if op == "gated_grad":
        return dict(op=op, N=N, d=a, f=b, act=rng.choice(["silu", "gelu"]), add=rng.random() < 0.5)
    k, m = (a, b) if rng.random() < 0.5 else (b, a)
    act, bias = rng.choice(["none", "silu", "gelu"]), rng.choice(["none", "bf16", "f32"])
    if op == "linear":
        return dict(op=op, N=N, k=k, m=m, act=act, bias=bias, residual=rng.random() < 0.5,
                    keep=act != "none" and rng.random() < 0.5)
    return dict(op=op, N=N, k=k, m=m, act=act, bias=bias, add=rng.random() < 0.5)


# ---------------------------------------------------------------- inputs

def _sizes(c):
    """Elements of each tensor: the largest first, parts of it, vectors of up to 4096 at the end."""
    n = [c["largest"]]
    for i in range(1, c["tensors"]):
        n.append(max(1, c["largest"] // (4 * i) if i < 4 and c["tensors"] <= 14 else min(4096, c["largest"]) - 17 * (i % 5)))
    return n


def _blocks(x):
    """x as rows of _BLOCK elements, zeros behind the last."""
    return torch.nn.functional.pad(x.reshape(-1), (0, -x.numel() % _BLOCK)).view(-1, _BLOCK)


def _codes(x, above_zero):
    """e4m3 codes of x (one scale a block, its largest magnitude over 448) and the scales.
    above_zero: what is not zero gets a code that is not."""
    scale = _blocks(x).abs().amax(1) / _TOP
    scale = torch.where(scale >= 2.0 ** -126, scale, torch.zeros_like(scale))
    inv = torch.where(scale > 0, 1.0 / scale, torch.zeros_like(scale))
    q = (_blocks(x) * inv[:, None]).to(torch.float8_e4m3fn).view(torch.uint8).reshape(-1)[:x.numel()]
    if above_zero:
        held = (inv > 0)[:, None].expand(-1, _BLOCK).reshape(-1)[:x.numel()]
        q = torch.where((x > 0) & held & (q == 0), torch.ones_like(q), q)
    return q, scale


def _values(q, scale, dtype=torch.float32):
    """What codes and scales stand for."""
    x = _blocks(q.view(torch.float8_e4m3fn).to(dtype)) * scale.to(dtype)[:, None]
    return x.reshape(-1)[:q.numel()]


def prepare(case, seed):
    c, dev = case, torch.device("cuda", torch.cuda.current_device())
    g = torch.Generator(device=dev).manual_seed(seed)
    s = {"case": c}
    op = c["op"]

    def normal(*shape, std=1.0, dtype=torch.bfloat16, mean=0.0):
        return torch.empty(*shape, dtype=dtype, device=dev).normal_(mean, std, generator=g)

    def empty(*shape, dtype=torch.bfloat16):
        return torch.empty(*shape, dtype=dtype, device=dev)

    if op in ("gated", "gated_grad"):
        N, d, f = c["N"], c["d"], c["f"]
        # what a norm leaves, and weights that keep its scale
        s["x"], s["wg"], s["wu"] = normal(N, d), normal(f, d, std=d ** -0.5), normal(f, d, std=d ** -0.5)
    if op == "gated":
        s["out"] = empty(N, f)
        s["gate"], s["up"] = (empty(N, f), empty(N, f)) if c["keep"] else (None, None)
    if op == "gated_grad":
        # what the forward pass left, and a gradient that comes through the second projection
        s["gate"], s["up"] = s["x"] @ s["wg"].T, s["x"] @ s["wu"].T
        s["dout"] = normal(N, f, std=1e-3)
        s["add"] = normal(N, d, std=1e-3) if c["add"] else None
        s["dx"], s["dwg"], s["dwu"] = empty(N, d), empty(f, d), empty(f, d)
    if op in ("linear", "linear_grad"):
        N, k, m = c["N"], c["k"], c["m"]
        s["x"], s["w"] = normal(N, k), normal(m, k, std=k ** -0.5)
        s["bias"] = None if c["bias"] == "none" else normal(m, std=0.3, dtype=_DTYPES[c["bias"]])
    if op == "linear":
        s["residual"] = normal(N, m) if c["residual"] else None
        s["out"], s["pre"] = empty(N, m), empty(N, m) if c["keep"] else None
    if op == "linear_grad":
        s["pre"] = None
        if c["act"] != "none":
            z = s["x"] @ s["w"].T
            s["pre"] = z if s["bias"] is None else (z + s["bias"]).bfloat16()
        s["dout"] = normal(N, m, std=1e-3)
        s["add"] = normal(N, k, std=1e-3) if c["add"] else None
        s["dx"], s["dw"] = empty(N, k), empty(m, k)
        s["dbias"] = None if s["bias"] is None else torch.empty_like(s["bias"])
    if op == "adamw":
        p, n = c["params"], _sizes(c)
        values = [normal(x, std=0.02, dtype=torch.float32) for x in n]
        s["masters"] = values if p == "master" else None
        s["params"] = values if p == "f32" else [x.bfloat16() for x in values]
        del values
        s["grads"] = [normal(x, std=1e-3, dtype=_DTYPES[c["grads"]]) for x in n]
        # averages after some steps: the second moment's spread over several powers of ten
        s["m"] = [normal(x, std=3e-4, dtype=torch.float32) for x in n]
        s["v"] = [normal(x, std=1e-3, dtype=torch.float32).square_().add_(1e-10) for x in n]
        s["ms"] = s["vs"] = None
        if c["bits"] == 8:
            s["m"], s["ms"] = map(list, zip(*[_codes(x, False) for x in s["m"]]))
            s["v"], s["vs"] = map(list, zip(*[_codes(x.sqrt(), True) for x in s["v"]]))
        s["lr"] = torch.full((1,), _LR, device=dev)
        s["step"] = torch.full((1,), _STEP, dtype=torch.int32, device=dev)
        # the norm is about twice what is allowed
        s["norm"] = torch.full((1,), 1e-3 * math.sqrt(sum(n)), device=dev) if c["clip"] else None
        s["max_norm"] = 0.5e-3 * math.sqrt(sum(n))
    return s


_BETA1, _BETA2, _EPS, _DECAY, _LR, _STEP = 0.9, 0.95, 1e-8, 0.1, 2.0 ** -10, 7


# ---------------------------------------------------------------- one pass

def _sharp(act, x):
    """(s, ds/dx) of an activation x sigmoid(s): s = x (SiLU), or 2 sqrt(2/pi) (x + 0.044715 x^3)
    (GELU in its tanh form)."""
    if act == "silu":
        return x, torch.ones_like(x)
    a = 2.0 * math.sqrt(2.0 / math.pi)
    return a * (x + 0.044715 * x * x * x), a * (1.0 + 3.0 * 0.044715 * x * x)


def _act(act, x):
    return x if act == "none" else x / (1.0 + torch.exp(-_sharp(act, x)[0]))


def _act_grad(act, x):
    """Value and derivative."""
    s, ds = _sharp(act, x)
    p = 1.0 / (1.0 + torch.exp(-s))
    return x * p, p * (1.0 + x * (1.0 - p) * ds)


def _gated(s):
    x, c = s["x"].float(), s["case"]
    gate, up = x @ s["wg"].float().T, x @ s["wu"].float().T
    out = (_act(c["act"], gate) * up).bfloat16()
    return (out, gate.bfloat16(), up.bfloat16()) if c["keep"] else (out,)


def _gated_grad(s):
    x, gate, dout = s["x"].float(), s["gate"].float(), s["dout"].float()
    a, da = _act_grad(s["case"]["act"], gate)
    dgate, dup = dout * s["up"].float() * da, dout * a
    dx = dgate @ s["wg"].float() + dup @ s["wu"].float()
    dx = dx if s["add"] is None else dx + s["add"].float()
    return dx.bfloat16(), (dgate.T @ x).bfloat16(), (dup.T @ x).bfloat16()


def _linear(s):
    c = s["case"]
    z = s["x"].float() @ s["w"].float().T
    z = z if s["bias"] is None else z + s["bias"].float()
    out = _act(c["act"], z)
    out = out if s["residual"] is None else out + s["residual"].float()
    return (out.bfloat16(), z.bfloat16()) if c["keep"] else (out.bfloat16(),)


def _linear_grad(s):
    dz = s["dout"].float()
    dz = dz if s["pre"] is None else dz * _act_grad(s["case"]["act"], s["pre"].float())[1]
    dx = dz @ s["w"].float()
    dx = dx if s["add"] is None else dx + s["add"].float()
    dw = (dz.T @ s["x"].float()).bfloat16()
    if s["bias"] is None:
        return dx.bfloat16(), dw
    return dx.bfloat16(), dw, dz.sum(0).to(s["bias"].dtype)


def _held(s):
    """The step's results: weights and states, those in 8 bits as e4m3 values and their scales."""
    if s["ms"] is None:
        return s["params"], s["masters"], s["m"], s["v"]
    m, v = ([q.view(torch.float8_e4m3fn) for q in s[n]] for n in ("m", "v"))
    return s["params"], s["masters"], m, v, s["ms"], s["vs"]


def _step_one(s, i, scale):
    eight = s["ms"] is not None
    g = s["grads"][i].float() * scale
    m = _values(s["m"][i], s["ms"][i]) if eight else s["m"][i]
    v = _values(s["v"][i], s["vs"][i]).square() if eight else s["v"][i]
    m = m * _BETA1 + g * (1.0 - _BETA1)
    v = v * _BETA2 + (g * g) * (1.0 - _BETA2)
    root = v.sqrt()
    p = (s["masters"] or s["params"])[i].float()
    change = m / (root / math.sqrt(1.0 - _BETA2 ** _STEP) + _EPS)
    p = p * (1.0 - _LR * _DECAY) - (_LR / (1.0 - _BETA1 ** _STEP)) * change
    s["params"][i].copy_(p)
    if s["masters"] is not None:
        s["masters"][i].copy_(p)
    m, ms = _codes(m, False) if eight else (m, None)
    v, vs = _codes(root, True) if eight else (v, None)
    s["m"][i].copy_(m)
    s["v"][i].copy_(v)
    if eight:
        s["ms"][i].copy_(ms)
        s["vs"][i].copy_(vs)


def _adamw(s):
    scale = 1.0
    if s["norm"] is not None:
        scale = (s["max_norm"] / (s["norm"].double() + 1e-6)).clamp(max=1.0).float()
    for i in range(len(s["params"])):
        _step_one(s, i, scale)
    return _held(s)


def _workspace(s, size, *sizes):
    """The workspace a program keeps beside its buffers."""
    if "ws" not in s:
        s["ws"] = torch.empty(size(*sizes), dtype=torch.uint8, device="cuda")
    return s["ws"]


def run(state):
    s, c = state, state["case"]
    op = c["op"]
    if not own:
        return {"gated": _gated, "gated_grad": _gated_grad, "linear": _linear, "linear_grad": _linear_grad, "adamw": _adamw}[op](s)
    from paper_2608_02625_gb300 import binding as B
    if op == "gated":
        B.dlm_gated_linear(s["x"], s["wg"], s["wu"], _ACTS[c["act"]], s["out"], s["gate"], s["up"])
        return (s["out"], s["gate"], s["up"]) if c["keep"] else (s["out"],)
    if op == "gated_grad":
        ws = _workspace(s, B.dlm_gated_linear_grad_workspace_bytes, c["N"], c["f"], c["d"])
        B.dlm_gated_linear_grad(s["dout"], s["x"], s["wg"], s["wu"], s["gate"], s["up"], _ACTS[c["act"]], s["add"],
                                s["dx"], s["dwg"], s["dwu"], ws)
        return s["dx"], s["dwg"], s["dwu"]
    if op == "linear":
        ws = _workspace(s, B.dlm_linear_workspace_bytes, c["N"], c["m"], c["k"])
        B.dlm_linear(s["x"], s["w"], s["bias"], _ACTS[c["act"]], s["residual"], s["out"], s["pre"], ws)
        return (s["out"], s["pre"]) if c["keep"] else (s["out"],)
    if op == "linear_grad":
        ws = _workspace(s, B.dlm_linear_grad_workspace_bytes, c["N"], c["m"], c["k"])
        B.dlm_linear_grad(s["dout"], s["x"], s["w"], s["pre"], _ACTS[c["act"]], s["add"], s["dx"], s["dw"], s["dbias"], ws)
        return (s["dx"], s["dw"]) if s["bias"] is None else (s["dx"], s["dw"], s["dbias"])
    if "hyper" not in s:
        s["hyper"] = B.AdamwParams(lr=s["lr"], step=s["step"], beta1=_BETA1, beta2=_BETA2, eps=_EPS, weight_decay=_DECAY,
                                   norm=s["norm"], max_norm=s["max_norm"])
    B.dlm_adamw(s["params"], s["masters"], s["grads"], s["m"], s["v"], s["ms"], s["vs"], s["hyper"])
    return _held(s)


# ---------------------------------------------------------------- work and accuracy

def work(case):
    c = case
    op = c["op"]
    if op == "adamw":
        per = {"f32": 8, "bf16": 4, "master": 10}[c["params"]] + {"f32": 4, "bf16": 2}[c["grads"]] + (16 if c["bits"] == 32 else 4)
        n = sum(_sizes(c))
        return {"bytes": n * per + (16 * (n // _BLOCK) if c["bits"] == 8 else 0), "flops": 16 * n}
    if op in ("gated", "gated_grad"):
        N, d, f = c["N"], c["d"], c["f"]
        if op == "gated":
            return {"bytes": 2 * (N * d + 2 * f * d + (3 if c["keep"] else 1) * N * f), "flops": 4 * N * d * f}
        return {"bytes": 2 * (3 * N * f + (3 if c["add"] else 2) * N * d + 4 * f * d), "flops": 8 * N * d * f}
    N, k, m = c["N"], c["k"], c["m"]
    if op == "linear":
        return {"bytes": 2 * (N * k + m * k + N * m * (1 + c["residual"] + c["keep"])), "flops": 2 * N * k * m}
    return {"bytes": 2 * ((2 if c["act"] != "none" else 1) * N * m + (3 if c["add"] else 2) * N * k + 2 * m * k),
            "flops": 4 * N * k * m}


def _logistic(act, z):
    """The weight of z in the activation, in 64 bits, and its derivative."""
    k = 0.044715
    inner = {"silu": 0.5 * z, "gelu": math.sqrt(2.0 / math.pi) * (z + k * z ** 3)}[act]
    slope = {"silu": torch.full_like(z, 0.5), "gelu": math.sqrt(2.0 / math.pi) * (1.0 + 3.0 * k * z ** 2)}[act]
    th = torch.tanh(inner)
    return 0.5 * (1.0 + th), 0.5 * (1.0 - th * th) * slope


def _exact_states(x, lowest):
    """e4m3 values and scales of x, from 64 bits. (Next to a border of its code a value may round
    either way.)"""
    rows = _blocks(x)
    top = rows.abs().amax(1) / _TOP
    top = torch.where(top >= 2.0 ** -126, top, torch.zeros_like(top))
    y = rows / torch.where(top > 0, top, torch.inf)[:, None]
    # three bits behind the leading one, steps of 2^-9 at least
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp_min(2.0 ** -6))) - 3.0)
    z = torch.round(y / step) * step
    if lowest:
        z = torch.where((y > 0) & (z == 0), torch.full_like(z, 2.0 ** -9), z)
    return z.reshape(-1)[:x.numel()], top


def exact(case, seed):
    c, s = case, prepare(case, seed)
    op = c["op"]
    wide = {n: t.double() for n, t in s.items() if isinstance(t, torch.Tensor)}
    if op == "gated":
        gate = torch.einsum("nd,fd->nf", wide["x"], wide["wg"])
        up = torch.einsum("nd,fd->nf", wide["x"], wide["wu"])
        out = gate * _logistic(c["act"], gate)[0] * up
        return (out, gate, up) if c["keep"] else (out,)
    if op == "gated_grad":
        w, dw = _logistic(c["act"], wide["gate"])
        dup = wide["dout"] * wide["gate"] * w
        dgate = wide["dout"] * wide["up"] * (w + wide["gate"] * dw)
        dx = torch.einsum("nf,fd->nd", dgate, wide["wg"]) + torch.einsum("nf,fd->nd", dup, wide["wu"])
        if c["add"]:
            dx += wide["add"]
        return dx, torch.einsum("nf,nd->fd", dgate, wide["x"]), torch.einsum("nf,nd->fd", dup, wide["x"])
    if op == "linear":
        z = torch.einsum("nk,mk->nm", wide["x"], wide["w"]) + wide.get("bias", 0.0)
        out = (z if c["act"] == "none" else z * _logistic(c["act"], z)[0]) + wide.get("residual", 0.0)
        return (out, z) if c["keep"] else (out,)
    if op == "linear_grad":
        dz = wide["dout"]
        if c["act"] != "none":
            w, dw = _logistic(c["act"], wide["pre"])
            dz = dz * (w + wide["pre"] * dw)
        dx = torch.einsum("nm,mk->nk", dz, wide["w"]) + wide.get("add", 0.0)
        dw = torch.einsum("nm,nk->mk", dz, wide["x"])
        return (dx, dw) if s["bias"] is None else (dx, dw, dz.sum(0))
    scale = min(1.0, s["max_norm"] / (float(s["norm"]) + 1e-6)) if c["clip"] else 1.0
    params, m, v = [], [], []
    for i, g in enumerate(s["grads"]):
        g = g.double() * scale
        m0 = _values(s["m"][i], s["ms"][i], torch.float64) if c["bits"] == 8 else s["m"][i].double()
        v0 = _values(s["v"][i], s["vs"][i], torch.float64) ** 2 if c["bits"] == 8 else s["v"][i].double()
        m1, v1 = torch.lerp(g, m0, _BETA1), torch.lerp(g * g, v0, _BETA2)
        p = (s["masters"] or s["params"])[i].double()
        change = (m1 / (1.0 - _BETA1 ** _STEP)) / (torch.sqrt(v1 / (1.0 - _BETA2 ** _STEP)) + _EPS)
        params.append(p - _LR * (change + _DECAY * p))
        m.append(m1 if c["bits"] == 32 else _exact_states(m1, False))
        v.append(v1 if c["bits"] == 32 else _exact_states(torch.sqrt(v1), True))
    masters = params if c["params"] == "master" else None
    if c["bits"] == 32:
        return params, masters, m, v
    return params, masters, *([x[k] for x in st] for k in (0, 1) for st in (m, v))
