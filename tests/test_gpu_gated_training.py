"""The gated block in a training step beside a plain down projection: forward, loss, backward, clipping and an
update, eager and captured, against the same step in 64 bits."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.fixture(scope="module")
def cd():
    from paper_2505_17701_amd import binding

    return binding


class Layer:
    """y = h W_down, loss = |y - target|^2 / 2; fp32 master weights, bf16 in the products."""

    def __init__(self, cd, T, m, f, seed=3):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.cd, self.T, self.m, self.f = cd, T, m, f
        self.Wg, self.Wu, self.Wd = (torch.randn((f, m), generator=g, device="cuda") * m ** -0.5 for _ in range(3))
        self.x = torch.randn((T, m), generator=g, device="cuda").to(BF16)
        self.target = torch.randn((T, m), generator=g, device="cuda")
        self.block = cd.Gated(m, f, T, train=True, fp32_grads=True)
        self.clip = cd.GradClip(2)
        self.h = torch.empty((T, f), dtype=BF16, device="cuda")
        self.dx = torch.empty((T, m), device="cuda")
        self.dWg, self.dWu = torch.empty((f, m), device="cuda"), torch.empty((f, m), device="cuda")
        self.norm = torch.empty((), dtype=torch.float64, device="cuda")

    def step(self, lr=0.1, max_norm=1.0):
        cd, Wg, Wu, Wd = self.cd, self.Wg.to(BF16), self.Wu.to(BF16), self.Wd.to(BF16)
        cd.countdown_gated_forward(self.block, self.x, Wg, Wu, h=self.h)
        dy = (self.h.float() @ Wd.float() - self.target)
        dh = (dy @ Wd.float().t()).to(BF16)
        cd.countdown_gated_backward(self.block, self.x, dh, Wg, Wu, dx=self.dx, dW_gate=self.dWg, dW_up=self.dWu)
        cd.countdown_clip_grads(self.clip, [self.dWg, self.dWu], max_norm, norm=self.norm)
        self.Wg.sub_(self.dWg, alpha=lr)
        self.Wu.sub_(self.dWu, alpha=lr)

    def reference(self, max_norm=1.0):
        """(dx, clipped dW_gate, dW_up) of the present weights from h's and dh's bf16, in 64 bits"""
        x, Wg, Wu, Wd = (t.to(BF16).double() for t in (self.x, self.Wg, self.Wu, self.Wd))
        a, u = x @ Wg.t(), x @ Wu.t()
        s = torch.sigmoid(a)
        h = (a * s * u).to(BF16).double()
        dh = ((h @ Wd - self.target.double()) @ Wd.t()).to(BF16).double()
        da, du = dh * u * s * (1 + a * (1 - s)), dh * a * s
        dWg, dWu = da.t() @ x, du.t() @ x
        norm = torch.sqrt(dWg.square().sum() + dWu.square().sum())
        c = min(1.0, max_norm / float(norm))
        return da @ Wg + du @ Wu, dWg * c, dWu * c


def near(got, want, most):
    assert float((got.double() - want).norm() / want.norm()) <= most


@pytest.mark.parametrize("T,m,f", [(5, 264, 520), (96, 256, 688), (700, 520, 1032)])
def test_step(cd, T, m, f):
    layer = Layer(cd, T, m, f)
    want = layer.reference()
    layer.step()
    # a bf16 of h or dh that lies next to a tie may round the other way: half a step, 2^-8 of itself, and where
    # every single one did, of each gradient too
    for got, w in zip((layer.dx, layer.dWg, layer.dWu), want):
        near(got, w, 2.0 ** -8)


def test_captured_steps_follow_the_weights(cd):
    a, b = Layer(cd, 96, 256, 688), Layer(cd, 96, 256, 688)
    a.step()
    b.step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            a.step()
    torch.cuda.current_stream().wait_stream(side)
    for _ in range(4):
        graph.replay()
        b.step()  # eager, of another layer, between the replays
        torch.cuda.synchronize()
        # the block's and the clipping's kernels give the same bits; the plain products around them may differ
        # by their order of sums
        near(a.Wg, b.Wg.double(), 1e-4)
        near(a.Wu, b.Wu.double(), 1e-4)
        assert float((a.norm - b.norm).abs() / b.norm) <= 1e-2


def test_adapters_beside_the_block(cd):
    """A prompt through the block and a plain down projection, its adapters on top."""
    g = torch.Generator(device="cuda").manual_seed(4)
    T, m, f, r, n = 40, 256, 688, 8, 3
    x = torch.randn((T, m), generator=g, device="cuda").to(BF16)
    Wg, Wu, Wd = ((torch.randn((f, m), generator=g, device="cuda") * m ** -0.5).to(BF16) for _ in range(3))
    A = (torch.randn((n, r, m), generator=g, device="cuda") * 0.05).to(BF16)
    B = (torch.randn((n, m, r), generator=g, device="cuda") * 0.05).to(BF16)
    ids = torch.randint(-1, n, (T,), generator=g, device="cuda", dtype=torch.int32)
    with cd.Gated(m, f, T) as block, cd.Adapters(m, m, r, n, T) as pool:
        h = cd.countdown_gated_forward(block, x, Wg, Wu)
        y = h.float() @ Wd.float()
        y = cd.countdown_adapters_add(pool, x, ids, A, B, base=y, y=y)
    x64 = x.double()
    a, u = x64 @ Wg.double().t(), x64 @ Wu.double().t()
    want = (a * torch.sigmoid(a) * u) @ Wd.double()
    for t in range(T):
        if int(ids[t]) >= 0:
            want[t] += B[int(ids[t])].double() @ (A[int(ids[t])].double() @ x64[t])
    near(y, want, 2.0 ** -8)  # h's rounding
