"""The adapters and the clipping as they are used together: adapters beside the sparse FFN,
trained towards the dense layer's output, and a predictor's gradients clipped in training."""
import math

import pytest

from gpu_support import dev_bf16
from workloads import make_layer

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

U = 2.0 ** -23  # one addition in fp32, at most (see test_gpu_adapters.py)


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.fixture(scope="module")
def cd():
    from paper_2505_17701_amd import binding

    return binding


DM, DFF, R, N, B = 256, 688, 16, 3, 8


class Step:
    """y = FFN(x) on its active neurons + each token's adapter; dy = bf16(y - target); the
    adapters' gradients, clipped to max_norm into `out`."""

    def __init__(self, cd, seed):
        g = torch.Generator().manual_seed(seed)
        self.cd = cd
        self.L = {k: dev_bf16(v) for k, v in make_layer(1700, DM, DFF, 0.05).items()}
        self.plan = cd.Plan(DM, DFF, max_batch=B)
        self.pool = cd.Adapters(DM, DM, R, N, max_tokens=B, train=True)
        self.clip = cd.GradClip(2)
        self.x = torch.randn(B, DM, generator=g).bfloat16().cuda()
        self.ids = torch.tensor([0, 2, 2, -1, 0, 2, 0, 0], dtype=torch.int32, device="cuda")
        self.A = (torch.randn(N, R, DM, generator=g) * 0.05).bfloat16().cuda()
        self.B = (torch.randn(N, DM, R, generator=g) * 0.05).bfloat16().cuda()
        self.scale = torch.tensor([0.5, 1.0, 2.0], device="cuda")
        self.target = cd.countdown_ffn_dense(self.plan, self.x, *self.weights())
        self.y = torch.empty(B, DM, device="cuda")
        self.dy = torch.empty(B, DM, dtype=torch.bfloat16, device="cuda")
        self.dA, self.dB = torch.empty(N, R, DM, device="cuda"), torch.empty(N, DM, R, device="cuda")
        self.out = [torch.empty_like(self.dA), torch.empty_like(self.dB)]
        self.norm = torch.empty((), dtype=torch.float64, device="cuda")

    def weights(self):
        return self.L["W_gate"], self.L["W_up"], self.L["W_down"]

    def run(self):
        cd, ad = self.cd, (self.ids, self.A, self.B, self.scale)
        cd.countdown_ffn_mono(self.plan, self.x, *self.weights(), 0.8, y=self.y)
        cd.countdown_adapters_add(self.pool, self.x, *ad, base=self.y, y=self.y)
        self.dy.copy_(self.y - self.target)
        cd.countdown_adapters_backward(self.pool, self.x, self.dy, *ad, dA=self.dA, dB=self.dB,
                                       need=(False, True, True))
        cd.countdown_clip_grads(self.clip, [self.dA, self.dB], 0.5, out=self.out, norm=self.norm)

    def check(self):
        f = lambda t: t.double().cpu()  # noqa: E731
        x, dy, A, Bm, ids = f(self.x), f(self.dy), f(self.A), f(self.B), self.ids.cpu()
        want = [torch.zeros(N, R, DM).double(), torch.zeros(N, DM, R).double()]
        mags = [torch.zeros_like(w) for w in want]
        for a in range(N):
            t = torch.nonzero(ids == a).flatten()
            s = float(self.scale[a])
            for k, h in ((want, lambda v: v), (mags, torch.abs)):
                g = s * h(dy[t]) @ h(Bm[a])
                k[0][a] = g.t() @ h(x[t])
                k[1][a] = s * h(dy[t]).t() @ (h(x[t]) @ h(A[a]).t())
        tols = [(DM + B + 8) * U * m for m in mags]
        norm = math.sqrt(sum(float((w ** 2).sum()) for w in want))
        # the gradients' error bounds the norm's: ||g| - |w|| <= |g - w|
        off = math.sqrt(sum(float((t ** 2).sum()) for t in tols))
        assert norm > 0.5 and abs(float(self.norm) - norm) <= off + 1e-12 * norm
        for got, out, w, tol in zip((self.dA, self.dB), self.out, want, tols):
            assert bool(((f(got) - w).abs() <= tol).all())
            coef = 0.5 / float(self.norm)
            assert bool(((f(out) - f(got) * coef).abs() <= 2 * U * (f(got) * coef).abs()).all())

    def close(self):
        for h in (self.plan, self.pool, self.clip):
            h.close()


def test_training_steps_of_adapters_beside_the_sparse_ffn(cd):
    s = Step(cd, 1)
    s.run()
    first = s.y.clone()
    for _ in range(4):
        s.check()
        for w, g in ((s.A, s.out[0]), (s.B, s.out[1])):
            w.copy_((w.float() - 0.2 * g).bfloat16())
        s.run()
    s.check()
    ffn = cd.countdown_ffn_mono(s.plan, s.x, *s.weights(), 0.8)
    assert torch.allclose(first[3], ffn[3], rtol=0, atol=1e-5)  # the token without an adapter
    assert not torch.equal(first[0], s.y[0])
    s.close()


def test_a_captured_step_follows_its_weights(cd):
    """The whole step in a graph, replayed with other weights, an eager step (with its own
    handles) and synchronizations between the replays. The FFN's sums are atomic: y may
    differ in the last bits between the two, so each replay is held to its own dy."""
    s, eager = Step(cd, 2), Step(cd, 3)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        s.run()
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        s.run()
    for k in range(3):
        eager.run()
        eager.check()
        with torch.no_grad():
            s.A.mul_(1.5 if k else 0.5)
            s.ids.copy_(torch.roll(s.ids, k))
        for t in (s.dA, s.dB, *s.out, s.norm):
            t.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        s.check()
    s.close()
    eager.close()


def _problem(n=32, dm=64, dff=96):
    g = torch.Generator().manual_seed(7)
    X = torch.randn(n, dm, generator=g).bfloat16().cuda()
    return X, (torch.rand(n, dff, generator=g) < 0.3).cuda()


def test_predictor_training_clips(cd):
    """One step on the whole set: the logged norm is that of the gradient, in 64 bits."""
    from paper_2505_17701_amd.predictor import train_low_rank, train_ternary

    X, M = _problem()
    rank, seed = 8, 42
    _, _, plain = train_low_rank(X, M, rank, epochs=1, batch=len(X))
    assert "grad_norms" not in plain
    _, _, log = train_low_rank(X, M, rank, epochs=1, batch=len(X), max_norm=1e-3)
    assert log["epoch_loss"] == plain["epoch_loss"] and log["skipped_steps"] == 0
    g = torch.Generator(device="cuda").manual_seed(seed)
    ta = (torch.randn(64, rank, generator=g, device="cuda") / 8.0).double().requires_grad_()
    tb = (torch.randn(rank, 96, generator=g, device="cuda") / rank ** 0.5).double().requires_grad_()
    z = (X.double() @ ta) @ tb
    torch.nn.functional.binary_cross_entropy_with_logits(z, M.double()).backward()
    want = math.sqrt(float((ta.grad ** 2).sum() + (tb.grad ** 2).sum()))
    # a gradient element sums at most 96 + 64 + 32 products in fp32, each of about its size
    assert len(log["grad_norms"]) == 1 and abs(log["grad_norms"][0] - want) <= 400 * U * want
    theta, tlog = train_ternary(X, M, epochs=2, batch=16, max_norm=0.01)
    assert len(tlog["grad_norms"]) == 4 and all(v > 0 for v in tlog["grad_norms"])
    assert theta.shape == (96, 64)
    with pytest.raises(ValueError):
        train_low_rank(X, M, rank, epochs=0, max_norm=0.0)


def test_predictor_training_skips_a_bad_step(cd):
    from paper_2505_17701_amd.predictor import train_low_rank

    X, M = _problem()
    A0, B0, _ = train_low_rank(X, M, 8, epochs=0)
    X[3, 5] = float("inf")
    A, B, log = train_low_rank(X, M, 8, epochs=1, batch=len(X), max_norm=1.0)
    assert log["skipped_steps"] == 1 and not math.isfinite(log["grad_norms"][0])
    assert torch.equal(A, A0) and torch.equal(B, B0)
