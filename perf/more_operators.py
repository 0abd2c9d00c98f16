"""Performance cases of the gated block and of 4-bit weights, as a program calls them.

A case is one pass through one operator:

* ``forward``: ``countdown_gated_forward``, ``h = SiLU(x W_gate^T) * (x W_up^T)`` for a decode
  step, a prompt or a training batch;
* ``backward``: ``countdown_gated_backward``, from dh the gradients of x, W_gate and W_up
  (the two products are formed again, nothing is kept from the forward pass);
* ``q4_project``: ``countdown_q4_project``, ``y = base + x W^T`` of a decode step where W has
  4-bit weights and a scale for each group of columns;
* ``q4_gated``: ``countdown_q4_gated``, the gated block of a decode step with such weights.

Layer sizes are those of the workloads in ``workloads/`` (256 x 688, 4096 x 11008,
4096 x 14336, 8192 x 28672, a 4096 x 4096 projection) and one ragged size. ``run`` computes the
same in elementary operations where ``own`` is false.
"""
from __future__ import annotations

import math
import random  # noqa: F401  (draw takes a random.Random)

import torch

own = False

BF16, F32 = "bf16", "fp32"
_DTYPE = {BF16: torch.bfloat16, F32: torch.float32}


def _gated(op, tokens, d_model, d_ff, dtype, name=None):
    """dtype: of h, or of the three gradients."""
    c = {"op": op, "tokens": tokens, "d_model": d_model, "d_ff": d_ff, "dtype": dtype}
    return dict(c, name=name) if name else c


def _q4(op, tokens, cols, rows, group, dtype, base=False, name=None):
    """rows x cols weights (two such matrices for q4_gated); dtype: of the result and the base."""
    c = {"op": op, "tokens": tokens, "cols": cols, "rows": rows, "group": group, "dtype": dtype,
         "base": base}
    return dict(c, name=name) if name else c


def listed():
    return [
        # one token through the layer of the smallest workload: latency
        _gated("forward", 1, 256, 688, BF16, name="forward_688_t1"),
        # a decode batch of four sequences: the weights' stream
        _gated("forward", 4, 4096, 11008, F32, name="forward_11008_t4"),
        # a short prompt at a ragged size
        _gated("forward", 333, 3000, 8008, BF16, name="forward_ragged_t333"),
        # packed prompts of many requests
        _gated("forward", 8192, 4096, 14336, BF16, name="forward_14336_t8192"),
        # the training step of a tiny layer
        _gated("backward", 37, 256, 688, BF16, name="backward_688_t37"),
        # a training batch with fp32 gradients at a ragged size
        _gated("backward", 777, 3000, 8008, F32, name="backward_ragged_t777"),
        # a training batch, the largest
        _gated("backward", 8192, 4096, 14336, BF16, name="backward_14336_t8192"),
        # one sequence through an attention projection
        _q4("q4_project", 1, 4096, 4096, 128, F32, name="q4_project_4096_t1"),
        # the down projection of eight sequences, added to the residual stream
        _q4("q4_project", 8, 14336, 4096, 64, F32, base=True, name="q4_project_down_t8"),
        # the largest batch at a ragged size, a last group of 24 columns
        _q4("q4_project", 16, 3000, 8008, 32, BF16, name="q4_project_ragged_t16"),
        # one sequence through the block of the 70B-shaped layer
        _q4("q4_gated", 1, 8192, 28672, 128, BF16, name="q4_gated_28672_t1"),
        # an odd batch through the block of the layer with 11008 neurons
        _q4("q4_gated", 13, 4096, 11008, 32, BF16, name="q4_gated_11008_t13"),
    ]


def _log(rng, lo, hi, step=1):
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(step, int(v / step + 0.5) * step)


def draw(rng):
    op = rng.choice(("forward", "forward", "backward", "backward", "q4_project", "q4_gated"))
    dtype = rng.choice((BF16, BF16, F32))
    if op in ("forward", "backward"):
        d_model, d_ff = _log(rng, 64, 4096, 8), _log(rng, 64, 14336, 8)
        return _gated(op, _log(rng, 1, 8192), d_model, d_ff, dtype)
    cols = _log(rng, 64, 28672, 8)
    rows = _log(rng, 64, min(28672, 8192 * 28672 // cols), 8)
    return _q4(op, rng.randint(1, 16), cols, rows, rng.choice((32, 64, 128)), dtype,
               base=op == "q4_project" and rng.random() < 0.5)


# ----------------------------------------------------------------- inputs

def _inputs(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 2 + 1)

    def normal(shape, sigma, dtype=torch.bfloat16):
        return torch.randn(shape, generator=g, device="cuda").mul_(sigma).to(dtype)

    T = case["tokens"]
    if case["op"] in ("forward", "backward"):  # tokens of unit rms, as a norm leaves them
        m, f = case["d_model"], case["d_ff"]
        s = {"x": normal((T, m), 1.0), "W_gate": normal((f, m), 0.02), "W_up": normal((f, m), 0.02)}
        if case["op"] == "backward":
            s["dh"] = normal((T, f), 0.01)
        return s
    rows, cols, group = case["rows"], case["cols"], case["group"]
    s = {"x": normal((T, cols), 1.0)}
    for k in ("W", "W_up") if case["op"] == "q4_gated" else ("W",):
        codes = torch.randn((rows, cols), generator=g, device="cuda").mul_(3.0)
        scale = torch.rand((rows, -(-cols // group)), generator=g, device="cuda")
        s[k] = (codes.round_().clamp_(-8, 7).to(torch.int8),
                scale.add_(0.5).mul_(0.007).to(torch.bfloat16))
    if case["base"]:
        s["base"] = normal((T, rows), 1.0, _DTYPE[case["dtype"]])
    return s


def prepare(case, seed):
    s = dict(_inputs(case, seed), op=case["op"], dtype=_DTYPE[case["dtype"]])
    T, dtype = case["tokens"], s["dtype"]
    if case["op"] in ("forward", "backward"):
        m, f = case["d_model"], case["d_ff"]
        shapes = {"h": (T, f)} if case["op"] == "forward" else {
            "dx": (T, m), "dW_gate": (f, m), "dW_up": (f, m)}
        s["out"] = {k: torch.empty(v, dtype=dtype, device="cuda") for k, v in shapes.items()}
        if own:  # the workspace that a program keeps for the layer
            from paper_2505_17701_amd import binding as cd

            s["plan"] = cd.Gated(m, f, max_tokens=T, train=case["op"] == "backward",
                                 fp32_grads=dtype is torch.float32)
        return s
    s["group"] = case["group"]
    s["out"] = torch.empty((T, case["rows"]), dtype=dtype, device="cuda")
    if own:  # the weights in the layout that a program keeps them in
        from paper_2505_17701_amd import binding as cd

        for k in ("W", "W_up"):
            if k in s:
                s[k] = cd.countdown_q4_pack(*s[k], case["group"])
    return s


# -------------------------------------------------------------- one pass

def _own(s):
    from paper_2505_17701_amd import binding as cd

    if s["op"] == "forward":
        return cd.countdown_gated_forward(s["plan"], s["x"], s["W_gate"], s["W_up"],
                                          h=s["out"]["h"])
    if s["op"] == "backward":
        dx, dWg, dWu = cd.countdown_gated_backward(s["plan"], s["x"], s["dh"], s["W_gate"],
                                                   s["W_up"], **s["out"])
        return {"dx": dx, "dW_gate": dWg, "dW_up": dWu}
    if s["op"] == "q4_project":
        return cd.countdown_q4_project(s["x"], s["W"], base=s.get("base"), y=s["out"])
    return cd.countdown_q4_gated(s["x"], s["W"], s["W_up"], h=s["out"])


def _weights(codes, scale, group):
    wide = scale.float().repeat_interleave(group, dim=1)[:, :codes.shape[1]]
    return codes.float() * wide


def run(s):
    if own:
        return _own(s)
    x, dtype = s["x"].float(), s["dtype"]
    if s["op"] == "q4_project":
        y = x @ _weights(*s["W"], s["group"]).t()
        return (y + s["base"].float() if "base" in s else y).to(dtype)
    if s["op"] == "q4_gated":
        g = x @ _weights(*s["W"], s["group"]).t()
        u = x @ _weights(*s["W_up"], s["group"]).t()
        return (g / (1 + torch.exp(-g)) * u).to(dtype)
    Wg, Wu = s["W_gate"].float(), s["W_up"].float()
    g, u = x @ Wg.t(), x @ Wu.t()
    sig = 1 / (1 + torch.exp(-g))
    if s["op"] == "forward":
        return (g * sig * u).to(dtype)
    dh = s["dh"].float()
    dg, du = dh * u * sig * (1 + g * (1 - sig)), dh * g * sig
    return {"dx": (dg @ Wg + du @ Wu).to(dtype), "dW_gate": (dg.t() @ x).to(dtype),
            "dW_up": (du.t() @ x).to(dtype)}


# ------------------------------------------------------------------ work

def work(case):
    """Every input read once, every output written once."""
    T, size = case["tokens"], 2 if case["dtype"] == BF16 else 4
    if case["op"] in ("forward", "backward"):
        m, f = case["d_model"], case["d_ff"]
        if case["op"] == "forward":
            return {"bytes": 2 * T * m + 4 * m * f + size * T * f, "flops": 4 * T * m * f}
        return {"bytes": 2 * T * (m + f) + 4 * m * f + size * (T * m + 2 * m * f),
                "flops": 12 * T * m * f}
    rows, cols = case["rows"], case["cols"]
    n = 2 if case["op"] == "q4_gated" else 1
    weights = rows * cols // 2 + 2 * rows * -(-cols // case["group"])
    return {"bytes": n * weights + 2 * T * cols + size * T * rows * (2 if case["base"] else 1),
            "flops": 2 * n * T * rows * cols}


# ------------------------------------------------- the definition in 64 bits

def exact(case, seed):
    s = _inputs(case, seed)
    x = s["x"].double()
    if case["op"] in ("forward", "backward"):
        Wg, Wu = s["W_gate"].double(), s["W_up"].double()
        g, u = torch.matmul(Wg, x.t()), torch.matmul(Wu, x.t())  # [d_ff, T]
        up = torch.exp(torch.clamp(-g, max=700.0))
        silu = g / (1.0 + up)
        if case["op"] == "forward":
            return (silu * u).t()
        dh = s["dh"].double().t()
        slope = (1.0 + up + g * up) / (1.0 + up) ** 2  # d SiLU / dg
        dg, du = dh * u * slope, dh * silu
        return {"dx": torch.matmul(Wg.t(), dg).t() + torch.matmul(Wu.t(), du).t(),
                "dW_gate": torch.matmul(dg, x), "dW_up": torch.matmul(du, x)}

    def product(codes, scale):  # group by group: the scale outside the sum over a group's columns
        group, y = case["group"], torch.zeros((case["tokens"], case["rows"]),
                                              dtype=torch.float64, device="cuda")
        for i in range(scale.shape[1]):
            part = slice(i * group, min((i + 1) * group, case["cols"]))
            y += torch.matmul(x[:, part], codes[:, part].double().t()) * scale[:, i].double()
        return y

    y = product(*s["W"])
    if case["op"] == "q4_project":
        return y + s["base"].double() if "base" in s else y
    return y / (1.0 + torch.exp(-y)) * product(*s["W_up"])
