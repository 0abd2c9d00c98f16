"""Performance cases of the low-rank adapters and the gradient clipping, as a program calls them.

A case is one pass through one operator:

* ``project``: ``countdown_adapters_project``, a decode batch through a shared projection
  with each token's own low-rank adapter: ``y = x W^T + scale_a (x A_a^T) B_a^T``;
* ``add``: ``countdown_adapters_add``, the adapters' part added to a projection that is
  there already (the sparse FFN's ``y``, or a prompt's matrix product);
* ``backward``: ``countdown_adapters_backward``, the gradients of x, A and B;
* ``clip``: ``countdown_clip_grads``, the norm over many gradient tensors, and clipping.

Layer sizes are those of the workloads in ``workloads/`` (256 x 688, 4096 x 11008,
4096 x 14336, a 4096 x 4096 projection of the same models) and one ragged size.
``run`` computes the same in elementary operations where ``own`` is false.
"""
from __future__ import annotations

import math
import random

import torch

own = False

BF16, F32 = "bf16", "fp32"
_DTYPE = {BF16: torch.bfloat16, F32: torch.float32}


def _adapters(op, tokens, d_in, d_out, rank, n, requests, y, name=None):
    """requests 0: every token is a request of its own (decode)."""
    c = {"op": op, "tokens": tokens, "d_in": d_in, "d_out": d_out, "rank": rank, "n": n,
         "requests": requests, "y": y}
    return dict(c, name=name) if name else c


def _clip(tensors, rows, cols, dtype, max_norm, name=None):
    c = {"op": "clip", "tensors": tensors, "rows": rows, "cols": cols, "dtype": dtype,
         "max_norm": max_norm}
    return dict(c, name=name) if name else c


def listed():
    return [
        # one sequence decoding through an attention projection with its adapter
        _adapters("project", 1, 4096, 4096, 16, 8, 0, F32, name="project_4096_t1"),
        # eight sequences of one decode step, adapters of a larger rank, the widest projection
        _adapters("project", 8, 4096, 14336, 64, 32, 0, F32, name="project_14336_t8"),
        # an odd batch at a ragged size and rank, the result in bf16
        _adapters("project", 13, 3000, 8008, 24, 5, 0, BF16, name="project_ragged_t13"),
        # the adapters of eight sequences on top of the sparse FFN's output
        _adapters("add", 8, 4096, 4096, 16, 64, 0, F32, name="add_ffn_t8"),
        # a few short prompts, ragged sizes, onto an fp32 projection
        _adapters("add", 777, 3000, 8008, 40, 6, 9, F32, name="add_ragged_t777"),
        # packed prompts of many requests onto a bf16 projection
        _adapters("add", 16384, 4096, 4096, 32, 16, 40, BF16, name="add_4096_t16384"),
        # the training step of a tiny layer
        _adapters("backward", 37, 256, 688, 8, 3, 3, BF16, name="backward_688_t37"),
        # a training batch of four adapters beside a square projection
        _adapters("backward", 4096, 4096, 4096, 16, 4, 8, BF16, name="backward_4096_t4096"),
        # the largest: a wide projection, rank 64
        _adapters("backward", 8192, 4096, 14336, 64, 8, 16, BF16, name="backward_14336_t8192"),
        # the gradients of a small predictor: latency
        _clip(2, 512, 64, F32, 0.5, name="clip_predictor_small"),
        # the predictors of a stack (rank 256 at 4096 columns), beyond the caches
        _clip(32, 4096, 1280, F32, 1.0, name="clip_stack"),
        # the norm alone, bf16 gradients of odd sizes (logging; nothing is scaled)
        _clip(48, 1001, 693, BF16, math.inf, name="norm_odd_bf16"),
    ]


def _log(rng, lo, hi, step=1):
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(step, int(v / step + 0.5) * step)


def draw(rng):
    op = rng.choice(("project", "add", "add", "backward", "backward", "clip"))
    if op == "clip":
        tensors = _log(rng, 1, 60)
        rows = _log(rng, 16, 8192)
        cols = max(8, min(_log(rng, 8, 4096), 32 * 4096 * 1280 // (tensors * rows)))
        return _clip(tensors, rows, cols, rng.choice((F32, BF16)),
                     rng.choice((0.5, 1.0, math.inf)))
    d_in = _log(rng, 256, 4096, 8)
    d_out = _log(rng, 256, 14336, 8)
    rank = rng.choice((8, 16, 16, 24, 32, 40, 64))
    if op == "project":
        return _adapters(op, rng.randint(1, 16), d_in, d_out, rank, rng.randint(1, 32), 0,
                         rng.choice((F32, F32, BF16)))
    most = 8192 if op == "backward" else 16384
    d_out = min(d_out, 14336 if op == "backward" else 4096)
    tokens = _log(rng, 1, most)
    n = rng.randint(1, 8 if op == "backward" else 16)
    requests = 0 if tokens <= 32 and rng.random() < 0.5 else min(tokens, rng.randint(1, 40))
    return _adapters(op, tokens, d_in, d_out, rank, n, requests,
                     BF16 if op == "backward" else rng.choice((F32, BF16)))


# ----------------------------------------------------------------- inputs

def _ids(case, seed):
    """The adapter of each token; -1 where a request uses none."""
    rng = random.Random(seed * 7919 + 13)
    tokens, n, requests = case["tokens"], case["n"], case["requests"]
    if requests == 0:  # one token per request; one in eight without an adapter
        ids = [rng.randrange(n) if rng.random() > 0.125 else -1 for _ in range(tokens)]
        if tokens == 1:
            ids = [rng.randrange(n)]
    else:  # packed requests of unequal lengths; one in ten without an adapter
        cuts = sorted(rng.sample(range(1, tokens), requests - 1)) if requests > 1 else []
        ids = []
        for lo, hi in zip([0] + cuts, cuts + [tokens]):
            ids += [rng.randrange(n) if rng.random() > 0.1 else -1] * (hi - lo)
    return torch.tensor(ids, dtype=torch.int32).cuda()


def _grad_shapes(case):
    """Every second gradient is one row shorter, so that the sizes differ."""
    return [(case["rows"] - (i % 2), case["cols"]) for i in range(case["tensors"])]


def _inputs(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 2 + 1)

    def normal(shape, sigma, dtype=torch.bfloat16):
        return torch.randn(shape, generator=g, device="cuda").mul_(sigma).to(dtype)

    if case["op"] == "clip":
        return {"grads": [normal(s, 0.02, _DTYPE[case["dtype"]]) for s in _grad_shapes(case)]}
    T, di, do, r, n = (case[k] for k in ("tokens", "d_in", "d_out", "rank", "n"))
    s = {"x": normal((T, di), 1.0), "ids": _ids(case, seed), "A": normal((n, r, di), 0.02),
         "B": normal((n, do, r), 0.02),
         "scale": torch.rand(n, generator=g, device="cuda") * 2 + 0.5}
    if case["op"] == "project":
        s["W"] = normal((do, di), 0.02)
    elif case["op"] == "add":
        s["base"] = normal((T, do), 1.0, _DTYPE[case["y"]])
    else:
        s["dy"] = normal((T, do), 0.01)
        s["base"] = normal((T, di), 0.01)
    return s


def prepare(case, seed):
    s = dict(_inputs(case, seed), op=case["op"])
    if case["op"] == "clip":
        s["max_norm"] = case["max_norm"]
        if own:  # the workspace that a training program keeps
            from paper_2505_17701_amd import binding as cd

            s["plan"] = cd.GradClip(max_tensors=case["tensors"])
        if math.isfinite(case["max_norm"]):
            s["out"] = [torch.empty_like(t) for t in s["grads"]]
        return s
    s["y"] = torch.empty((case["tokens"], case["d_in" if case["op"] == "backward" else "d_out"]),
                         dtype=_DTYPE[case["y"]], device="cuda")
    if own:  # the adapter pool's workspace
        from paper_2505_17701_amd import binding as cd

        s["plan"] = cd.Adapters(case["d_in"], case["d_out"], case["rank"], case["n"],
                                max_tokens=case["tokens"], train=case["op"] == "backward")
    return s


# -------------------------------------------------------------- one pass

def _own(s):
    from paper_2505_17701_amd import binding as cd

    if s["op"] == "clip":
        norm = cd.countdown_clip_grads(s["plan"], s["grads"], s["max_norm"], out=s.get("out"))
        return {"norm": norm, "grads": s.get("out")}
    ad = (s["ids"], s["A"], s["B"], s["scale"])
    if s["op"] == "project":
        return cd.countdown_adapters_project(s["plan"], s["x"], s["W"], *ad, y=s["y"])
    if s["op"] == "add":
        return cd.countdown_adapters_add(s["plan"], s["x"], *ad, base=s["base"], y=s["y"])
    dx, dA, dB = cd.countdown_adapters_backward(s["plan"], s["x"], s["dy"], *ad, base=s["base"],
                                                dx=s["y"])
    return {"dx": dx, "dA": dA, "dB": dB}


def _slots(s):
    """[T, n * r]: the scale of the token's adapter at that adapter's ranks, else 0."""
    n, r = s["A"].shape[:2]
    hot = s["ids"][:, None] == torch.arange(n, device="cuda", dtype=torch.int32)
    return (hot * s["scale"]).repeat_interleave(r, dim=1)


def run(s):
    if own:
        return _own(s)
    if s["op"] == "clip":
        square = torch.stack([t.double().square().sum() for t in s["grads"]]).sum()
        norm = square.sqrt()
        if "out" not in s:
            return {"norm": norm, "grads": None}
        coef = torch.where(norm > s["max_norm"], s["max_norm"] / norm, 1.0).float()
        return {"norm": norm, "grads": [(t.float() * coef).to(t.dtype) for t in s["grads"]]}
    # all adapters side by side are one low-rank factor of rank n * r; a token keeps its own ranks
    n, r, di = s["A"].shape
    A = s["A"].float().reshape(n * r, di)
    B = s["B"].float().permute(1, 0, 2).reshape(-1, n * r)
    x, hot = s["x"].float(), _slots(s)
    lat = (x @ A.t()) * hot
    if s["op"] == "project":
        return (x @ s["W"].float().t() + lat @ B.t()).to(s["y"].dtype)
    if s["op"] == "add":
        return (s["base"].float() + lat @ B.t()).to(s["y"].dtype)
    dy = s["dy"].float()
    g = (dy @ B) * hot
    return {"dx": (s["base"].float() + g @ A).to(s["y"].dtype),
            "dA": (g.t() @ x).reshape(n, r, di),
            "dB": (dy.t() @ lat).reshape(-1, n, r).permute(1, 0, 2).contiguous()}


# ------------------------------------------------------------------ work

def work(case):
    """Every input read once, every output written once; of the adapters, as many as tokens."""
    if case["op"] == "clip":
        elems = sum(a * b for a, b in _grad_shapes(case))
        size = 2 if case["dtype"] == BF16 else 4
        scaled = math.isfinite(case["max_norm"])
        return {"bytes": elems * size * (2 if scaled else 1), "flops": elems * (3 if scaled else 2)}
    T, di, do, r, n = (case[k] for k in ("tokens", "d_in", "d_out", "rank", "n"))
    used, ysize = min(n, T), 2 if case["y"] == BF16 else 4
    low = 2 * T * r * (di + do)
    adapters = 2 * used * r * (di + do)
    if case["op"] == "project":
        return {"bytes": 2 * di * do + 2 * T * di + adapters + ysize * T * do,
                "flops": 2 * T * di * do + low}
    if case["op"] == "add":
        return {"bytes": 2 * T * di + adapters + 2 * ysize * T * do, "flops": low}
    return {"bytes": 2 * T * (di + do) + adapters + 4 * T * di + 4 * n * r * (di + do),
            "flops": 3 * low}


# ------------------------------------------------- the definition in 64 bits

def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "clip":
        norm = torch.sqrt(sum((t.double() ** 2).sum() for t in s["grads"]))
        top = case["max_norm"]
        if not math.isfinite(top):
            return {"norm": norm, "grads": None}
        return {"norm": norm,
                "grads": [t.double() * min(1.0, top / float(norm)) for t in s["grads"]]}
    x = s["x"].double()
    ids = s["ids"].long()
    A, B, scale = s["A"].double(), s["B"].double(), s["scale"].double()
    tokens = [(a, torch.nonzero(ids == a).flatten()) for a in range(case["n"])]
    if case["op"] in ("project", "add"):
        y = torch.matmul(x, s["W"].double().t()) if case["op"] == "project" else s["base"].double()
        for a, rows in tokens:
            delta = torch.matmul(B[a], torch.matmul(A[a], x[rows].t()))
            y[rows] += scale[a] * delta.t()
        return y
    dy, dx = s["dy"].double(), s["base"].double()
    dA, dB = torch.zeros_like(A), torch.zeros_like(B)
    for a, rows in tokens:
        back = scale[a] * torch.matmul(B[a].t(), dy[rows].t())  # [r, tokens]
        dx[rows] += torch.matmul(back.t(), A[a])
        dA[a] = torch.matmul(back, x[rows])
        dB[a] = scale[a] * torch.matmul(dy[rows].t(), torch.matmul(x[rows], A[a].t()))
    return {"dx": dx, "dA": dA, "dB": dB}
