"""Performance cases of training and scoring the refiner's last layer, one operator a pass.

listed() names the cases; draw() gives further ones of the same ranges. Every
case is one of five operations:

  loss       dlm_lmhead_loss: cross entropy of given tokens under the output
             projection of the hidden states, the logits never stored
  loss_grad  dlm_lmhead_loss_grad: its gradients of the hidden states and the weight
  norm       dlm_layer_norm: the norm in front of the projection
  norm_grad  dlm_layer_norm_grad: its gradients, those of weight and bias
             summed over all rows among them
  clip       dlm_clip_grad_norm: the norm over all gradients, and every gradient
             scaled so that it is at most max_norm

Widths and vocabularies are those of the package's workloads (d = 2048,
V = 151552, batches of up to 32 x 512 positions of which a quarter is masked and
so has a target), of its tests (odd vocabularies, d = 64) and generic ones
between them.
"""
import math

import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
_V = 151552                        # the workloads' vocabulary
_MOST = 4096 * _V * 2048           # rows with a target x V x d of the largest listed case
_MOST_NORM = 16384 * 2048          # elements of the largest norm
_MOST_CLIP = _V * 2048             # elements of the largest set of gradients


def listed():
    return [
        # Log-likelihood of one token at one position: the weight is read once.
        dict(name="loss_1", op="loss", N=1, V=_V, d=2048, scored=1.0),
        # A small head, odd in every size (the last tiles are ragged in all three).
        dict(name="loss_odd_517", op="loss", N=517, V=10007, d=200, scored=0.9),
        # A training batch of 32 x 512 positions, a quarter of them masked: the loss of those.
        dict(name="loss_32x512", op="loss", N=16384, V=_V, d=2048, scored=0.25),
        # Gradients of one local window of 64 positions: bound by reading and writing V x d.
        dict(name="loss_grad_64", op="loss_grad", N=64, V=_V, d=2048, scored=1.0),
        # The small odd head's gradients.
        dict(name="loss_grad_odd_517", op="loss_grad", N=517, V=10007, d=200, scored=0.9),
        # The training batch's gradients: bound by the tensor cores.
        dict(name="loss_grad_32x512", op="loss_grad", N=16384, V=_V, d=2048, scored=0.25),
        # The norm of one sequence, as a refiner serving a single request runs it.
        dict(name="norm_512", op="norm", N=512, d=2048, dtype="bf16", wdtype="bf16"),
        # The norm of a batch.
        dict(name="norm_32x512", op="norm", N=16384, d=2048, dtype="bf16", wdtype="f32"),
        # Gradients through the norm of one sequence at full precision, an odd width.
        dict(name="norm_grad_512_f32", op="norm_grad", N=512, d=1001, dtype="f32", wdtype="f32"),
        # Gradients through the norm of the training batch.
        dict(name="norm_grad_32x512", op="norm_grad", N=16384, d=2048, dtype="bf16", wdtype="f32"),
        # Many small gradients (norm weights and biases): launches and latency.
        dict(name="clip_small", op="clip", tensors=48, largest=2048, dtype="f32", over=3.0),
        # The output projection's gradient and the norm's beside it.
        dict(name="clip_head", op="clip", tensors=3, largest=_V * 2048, dtype="mixed", over=3.0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["loss", "loss", "loss_grad", "loss_grad", "norm", "norm_grad", "clip"])
    if op in ("loss", "loss_grad"):
        V = rng.choice([_V, _log(rng, 1000, 151553), _log(rng, 1000, 151553)])
        d = rng.choice([64, 512, 2048, 8 * _log(rng, 4, 512)])
        scored = rng.choice([1.0, 0.25, round(rng.uniform(0.05, 1.0), 2)])
        return dict(op=op, N=_log(rng, 1, max(1, min(16384, int(_MOST / (V * d * scored))))), V=V, d=d, scored=scored)
    if op == "clip":
        n = _log(rng, 1, 60)
        return dict(op=op, tensors=n, largest=_log(rng, 100, _MOST_CLIP // min(n, 4)),
                    dtype=rng.choice(["bf16", "f32", "mixed"]) if n > 4 else "bf16",
                    over=rng.choice([3.0, 0.5, round(rng.uniform(0.1, 100.0), 2)]))
    d = rng.choice([2048, _log(rng, 32, 8192), _log(rng, 32, 8192)])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    most = _MOST_NORM if dtype == "bf16" else _MOST_NORM // 2
    return dict(op=op, N=_log(rng, 1, max(1, min(65536, most // d))), d=d, dtype=dtype,
                wdtype=rng.choice([dtype, "f32"]))


# ---------------------------------------------------------------- inputs

def _scored(c):
    """Rows that have a target."""
    return max(1, int(c["N"] * c["scored"]))


def _clip_sizes(c):
    """Lengths of the gradients: the largest first, odd ones after it, vectors of up to 4096 at the end."""
    n = [c["largest"]]
    for i in range(1, c["tensors"]):
        n.append(max(1, c["largest"] // (8 * i) if i < 8 and c["tensors"] > 4 else min(4096, c["largest"]) - 17 * (i % 5)))
    return n


def _clip_dtypes(c):
    if c["dtype"] != "mixed":
        return [_DTYPES[c["dtype"]]] * c["tensors"]
    return [torch.bfloat16 if i % 3 == 0 else torch.float32 for i in range(c["tensors"])]


def _logits(h, w):
    return h.float() @ w.float().T


def prepare(case, seed):
    c, dev = case, torch.device("cuda", torch.cuda.current_device())
    g = torch.Generator(device=dev).manual_seed(seed)
    s = {"case": c}
    op = c["op"]

    def normal(*shape, std=1.0, dtype=torch.bfloat16, mean=0.0):
        return torch.empty(*shape, dtype=dtype, device=dev).normal_(mean, std, generator=g)

    if op in ("loss", "loss_grad"):
        N, V, d = c["N"], c["V"], c["d"]
        # logits of standard deviation 2, and the target's raised: a model that has learned something
        s["w"] = normal(V, d, std=d ** -0.5)
        s["t"] = torch.full((N,), -1, dtype=torch.int32, device=dev)
        rows = torch.randperm(N, generator=g, device=dev)[:_scored(c)]
        s["t"][rows] = torch.randint(0, V, (len(rows),), dtype=torch.int32, generator=g, device=dev)
        s["h"] = (normal(N, d, std=2.0, dtype=torch.float32) +
                  4.0 * s["w"][s["t"].clamp_min(0).long()].float() * torch.rand(N, 1, device=dev, generator=g)).bfloat16()
        s["loss"], s["lse"] = (torch.empty(N, device=dev) for _ in range(2))
    if op == "loss_grad":
        # what the forward pass left, and each row's weight: 1 / (masked share), over the rows
        s["lse"] = torch.cat([torch.logsumexp(_logits(h, s["w"]), 1) for h in s["h"].split(4096)])
        s["lse"] = torch.where(s["t"] >= 0, s["lse"], 0.0)
        s["dloss"] = (0.5 + 2.0 * torch.rand(c["N"], device=dev, generator=g)) / _scored(c)
        s["dh"], s["dw"] = torch.empty_like(s["h"]), torch.empty_like(s["w"])
    if op in ("norm", "norm_grad"):
        N, d, t, wt = c["N"], c["d"], _DTYPES[c["dtype"]], _DTYPES[c["wdtype"]]
        # hidden states: channels of their own mean, a few of them far larger than the others
        scale = 1.0 + 30.0 * (torch.rand(d, device=dev, generator=g) < 0.01)
        s["x"] = ((normal(N, d, dtype=torch.float32) + normal(d, dtype=torch.float32, std=0.5)) * scale).to(t)
        s["weight"], s["bias"] = normal(d, std=0.2, mean=1.0, dtype=wt), normal(d, std=0.2, dtype=wt)
        s["mean"], s["rstd"] = (torch.empty(N, device=dev) for _ in range(2))
        s["out"] = torch.empty_like(s["x"])
    if op == "norm_grad":
        x = s["x"].float()
        s["mean"] = x.mean(1)
        s["rstd"] = ((x - s["mean"][:, None]).square().mean(1) + 1e-5).rsqrt()
        s["dout"] = normal(c["N"], c["d"], dtype=torch.float32).to(s["x"].dtype)
        s["dweight"], s["dbias"] = torch.empty_like(s["weight"]), torch.empty_like(s["bias"])
    if op == "clip":
        s["grads"] = [normal(n, std=1e-3 * (1 + i % 4), dtype=t)
                      for i, (n, t) in enumerate(zip(_clip_sizes(c), _clip_dtypes(c)))]
        s["outs"] = [torch.empty_like(x) for x in s["grads"]]
        s["norm"] = torch.empty(1, device=dev)
        # the norm is about `over` times what is allowed
        s["max_norm"] = math.sqrt(sum(n * (1e-3 * (1 + i % 4)) ** 2 for i, n in enumerate(_clip_sizes(c)))) / c["over"]
    return s


# ---------------------------------------------------------------- one pass

def _loss(s):
    rows = torch.nonzero(s["t"] >= 0).flatten()
    x = _logits(s["h"][rows], s["w"])
    m = x.amax(1, keepdim=True)
    lse = m[:, 0] + torch.log(torch.exp(x - m).sum(1))
    loss, out = torch.zeros_like(s["loss"]), torch.zeros_like(s["lse"])
    loss[rows] = lse - x.gather(1, s["t"][rows].long()[:, None])[:, 0]
    out[rows] = lse
    return loss, out


def _loss_grad(s):
    rows = torch.nonzero(s["t"] >= 0).flatten()
    h = s["h"][rows].float()
    g = torch.exp(_logits(h, s["w"]) - s["lse"][rows, None])
    g[torch.arange(len(rows), device=g.device), s["t"][rows].long()] -= 1.0
    g = g * s["dloss"][rows, None]
    dh = torch.zeros_like(s["h"])
    dh[rows] = (g @ s["w"].float()).to(dh.dtype)
    return dh, (g.T @ h).to(s["w"].dtype)


def _norm(s):
    x = s["x"].float()
    mean = x.mean(1)
    xc = x - mean[:, None]
    rstd = 1.0 / torch.sqrt((xc * xc).mean(1) + 1e-5)
    return (xc * rstd[:, None] * s["weight"].float() + s["bias"].float()).to(s["x"].dtype), mean, rstd


def _norm_grad(s):
    dy, rstd = s["dout"].float(), s["rstd"][:, None]
    xhat = (s["x"].float() - s["mean"][:, None]) * rstd
    a = dy * s["weight"].float()
    dx = rstd * (a - a.mean(1, keepdim=True) - xhat * (a * xhat).mean(1, keepdim=True))
    return dx.to(s["x"].dtype), (dy * xhat).sum(0).to(s["weight"].dtype), dy.sum(0).to(s["bias"].dtype)


def _clip(s):
    total = torch.stack([x.float().square().sum(dtype=torch.float64) for x in s["grads"]]).sum()
    norm = total.sqrt()
    scale = torch.clamp(s["max_norm"] / (norm + 1e-6), max=1.0).float()
    return [(x.float() * scale).to(x.dtype) for x in s["grads"]], norm.float().reshape(1)


def _workspace(s, size, *sizes):
    """The workspace a program keeps beside its buffers."""
    if "ws" not in s:
        s["ws"] = torch.empty(size(*sizes), dtype=torch.uint8, device="cuda")
    return s["ws"]


def run(state):
    s, c = state, state["case"]
    op = c["op"]
    if not own:
        return {"loss": _loss, "loss_grad": _loss_grad, "norm": _norm, "norm_grad": _norm_grad, "clip": _clip}[op](s)
    from paper_2608_02625_gb300 import binding as B
    if op == "loss":
        ws = _workspace(s, B.dlm_lmhead_loss_workspace_bytes, c["N"], c["d"])
        return B.dlm_lmhead_loss(s["h"], s["w"], s["t"], s["loss"], s["lse"], ws)
    if op == "loss_grad":
        ws = _workspace(s, B.dlm_lmhead_loss_grad_workspace_bytes, c["N"], c["V"], c["d"])
        return B.dlm_lmhead_loss_grad(s["h"], s["w"], s["t"], s["lse"], s["dloss"], s["dh"], s["dw"], ws)
    if op == "norm":
        return B.dlm_layer_norm(s["x"], s["weight"], s["bias"], 1e-5, s["out"], s["mean"], s["rstd"])
    if op == "norm_grad":
        ws = _workspace(s, B.dlm_layer_norm_grad_workspace_bytes, c["N"], c["d"])
        return B.dlm_layer_norm_grad(s["dout"], s["x"], s["weight"], s["mean"], s["rstd"], s["out"], s["dweight"],
                                     s["dbias"], ws)
    ws = _workspace(s, B.dlm_clip_grad_norm_workspace_bytes)
    return B.dlm_clip_grad_norm(s["grads"], s["outs"], s["max_norm"], s["norm"], ws)


# ---------------------------------------------------------------- work and accuracy

def work(case):
    c = case
    op = c["op"]
    if op in ("loss", "loss_grad"):
        n, V, d = _scored(c), c["V"], c["d"]
        if op == "loss":
            return {"bytes": 2 * d * (n + V) + 12 * c["N"], "flops": 2 * n * V * d}
        # the logits once more, and a product for each gradient
        return {"bytes": 2 * d * (n + c["N"] + 2 * V) + 12 * c["N"], "flops": 6 * n * V * d}
    if op == "clip":
        elems = list(zip(_clip_sizes(c), _clip_dtypes(c)))
        return {"bytes": sum(2 * n * (2 if t == torch.bfloat16 else 4) for n, t in elems),
                "flops": 3 * sum(n for n, _ in elems)}
    n, esz, wsz = c["N"] * c["d"], {"bf16": 2, "f32": 4}[c["dtype"]], {"bf16": 2, "f32": 4}[c["wdtype"]]
    if op == "norm":
        return {"bytes": 2 * n * esz + 2 * c["d"] * wsz + 8 * c["N"], "flops": 8 * n}
    return {"bytes": 3 * n * esz + 3 * c["d"] * wsz + 8 * c["N"], "flops": 14 * n}


def exact(case, seed):
    c, s = case, prepare(case, seed)
    op = c["op"]
    if op in ("loss", "loss_grad"):
        t, w = s["t"].long(), s["w"].double()
        dev = w.device
        loss, lse = (torch.zeros(c["N"], dtype=torch.float64, device=dev) for _ in range(2))
        dh, dw = torch.zeros(c["N"], c["d"], dtype=torch.float64, device=dev), torch.zeros_like(w)
        for r in torch.arange(c["N"], device=dev)[t >= 0].split(512):
            h = s["h"][r].double()
            logits = torch.einsum("rk,vk->rv", h, w)
            if op == "loss":
                lse[r] = torch.logsumexp(logits, -1)
                loss[r] = -torch.log_softmax(logits, -1)[torch.arange(len(r), device=dev), t[r]]
                continue
            p = logits.sub_(s["lse"][r].double()[:, None]).exp_()
            hot = torch.zeros_like(p).scatter_(1, t[r][:, None], 1.0)
            p = (p - hot) * s["dloss"][r].double()[:, None]
            dh[r] = torch.einsum("rv,vk->rk", p, w)
            dw += torch.einsum("rv,rk->vk", p, h)
        return (loss, lse) if op == "loss" else (dh, dw)
    if op == "norm":
        x = s["x"].double()
        var, mean = torch.var_mean(x, 1, correction=0)
        rstd = (var + 1e-5) ** -0.5
        out = (x - mean[:, None]) * rstd[:, None]
        return out * s["weight"].double() + s["bias"].double(), mean, rstd
    if op == "norm_grad":
        x, dy, w, d = s["x"].double(), s["dout"].double(), s["weight"].double(), c["d"]
        mean, rstd = s["mean"].double()[:, None], s["rstd"].double()[:, None]
        z = (x - mean) * rstd
        # through z: the norm's Jacobian is rstd (I - (1 1^T + z z^T) / d)
        dz = dy * w
        dx = rstd / d * (d * dz - dz.sum(1, keepdim=True) - z * (dz * z).sum(1, keepdim=True))
        return dx, torch.einsum("nd,nd->d", dy, z), dy.sum(0)
    grads = [x.double() for x in s["grads"]]
    norm = torch.sqrt(sum((x * x).sum() for x in grads))
    scale = min(1.0, s["max_norm"] / (float(norm) + 1e-6))
    return [x * scale for x in grads], norm.reshape(1)
