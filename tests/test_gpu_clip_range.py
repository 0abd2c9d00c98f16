"""Clipping where norm / max_norm leaves the range of fp32's normal numbers.

Tolerances. The coefficient c = max_norm / norm (fp64) enters as an fp32 number of 24
significant bits and a power of two. A scaled value is therefore off by half a step of the coefficient and
of the product, 2 * 2^-24, by half the smallest fp32 step, 2^-150, where the result is
subnormal, and by half a step of bf16, 2^-8 relative or half its smallest step, 2^-134."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.fixture(scope="module")
def cd():
    from paper_2505_17701_amd import binding

    return binding


def check(got, grad, coef):
    want = grad.double() * coef
    tol = 2.0 ** -23 * want.abs() + 2.0 ** -150
    if grad.dtype == BF16:
        tol = tol + torch.finfo(BF16).eps / 2 * want.abs() + 2.0 ** -134
    over = int(((got.double() - want).abs() > tol).sum())
    assert over == 0, f"{over} of {got.numel()} off, {got.dtype}, coefficient {coef}"


def gradients(kind, n, dtype, seed):
    """n values of the kind: near the type's largest, ordinary, or of every magnitude."""
    g = torch.Generator().manual_seed(seed)
    v = torch.rand(n, generator=g) * 0.5 + 0.5
    v = torch.where(torch.rand(n, generator=g) < 0.5, -v, v)
    if kind == "huge":
        v = v * 3e38
    elif kind == "spread":
        v = torch.ldexp(v, torch.randint(-126, 127, (n,), generator=g).float())
        v[0] = 3e38
    return v.to(dtype).cuda()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n", [1000, 100001])  # one workgroup; many
@pytest.mark.parametrize("kind,top", [
    ("huge", 1.0), ("huge", 1e-10), ("huge", 1e-30), ("spread", 1.0), ("spread", 1e-3),
    ("ordinary", 1e-37), ("ordinary", 1e-43), ("ordinary", 1e-300), ("huge", 5e-324),
])
def test_scaled_values(cd, kind, top, n, dtype):
    flat = gradients(kind, n + 3, dtype, 3)
    grads = [flat[1:n - 37], flat[n - 35:n + 1]]  # odd offsets
    with cd.GradClip(2) as clip:
        for shift in (0, 1):  # outputs at the gradients' alignment and at another
            dst = torch.full_like(flat, 7.0)
            out = [dst[1 + shift:n - 37 + shift], dst[n - 35 + shift:n + 1 + shift]]
            norm = float(cd.countdown_clip_grads(clip, grads, top, out=out))
            assert math.isfinite(norm) and norm > top
            for o, t in zip(out, grads):
                check(o, t, top / norm)
            if top >= 1e-3:  # nothing is erased
                assert bool((out[0][:1] != 0).all()) or kind == "spread"
        place = flat.clone()
        cd.countdown_clip_grads(clip, [place[1:n - 37], place[n - 35:n + 1]], top)
        check(place[1:n - 37], grads[0], top / norm)
        check(place[n - 35:n + 1], grads[1], top / norm)


def test_the_edge_of_the_normal_numbers(cd):
    """Coefficients just above and just below 2^-126, the smallest normal fp32 number."""
    t = torch.zeros(64, device="cuda")
    t[0] = 2.0 ** 127
    with cd.GradClip(1) as clip:
        for k in (1.0 - 2.0 ** -30, 1.0, 1.0 + 2.0 ** -30, 1.5, 0.75, 0.5000001):
            out = torch.empty_like(t)
            norm = float(cd.countdown_clip_grads(clip, [t], 2.0 * k, out=[out]))
            assert norm == 2.0 ** 127
            check(out, t, 2.0 * k / norm)


def test_the_norm_after_clipping(cd):
    """Clipping gradients of 3e38 to norm 1 gives a norm of 1."""
    for n in (1000, 200000):
        t = torch.full((n,), 3e38, device="cuda")
        with cd.GradClip(1) as clip:
            cd.countdown_clip_grads(clip, [t], 1.0)
            after = float(cd.countdown_clip_grads(clip, [t], math.inf))
        assert abs(after - 1.0) <= 2.0 ** -23 + 2.0 ** -52 * n


@pytest.mark.parametrize("dtype,value", [(F32, 1e-42), (F32, 3 * 2.0 ** -149), (BF16, 5 * 2.0 ** -133)])
def test_subnormal_gradients(cd, dtype, value):
    """Squares below fp32's range, results that are subnormal themselves."""
    for n in (1000, 100001):
        t = torch.full((n,), value, dtype=dtype, device="cuda")
        with cd.GradClip(1) as clip:
            norm = float(cd.countdown_clip_grads(clip, [t], math.inf))
            want = math.sqrt(n) * float(t[0].double())
            assert abs(norm - want) <= 2.0 ** -52 * (n / 2 + 3) * want
            out = torch.empty_like(t)
            cd.countdown_clip_grads(clip, [t], norm * 0.6, out=[out])
            check(out, t, 0.6)


def test_many_tensors(cd):
    """Eleven launches of 96 tensors, the sum of the first one used by the others: eager, in
    place, and replayed with other values."""
    g = torch.Generator().manual_seed(9)
    sizes = [int(v) for v in torch.randint(1, 9000, (1000,), generator=g)]
    flat = torch.randn(sum(sizes), generator=g).cuda()
    grads = [t.to(BF16) if i % 3 == 0 else t for i, t in enumerate(flat.split(sizes))]
    clip, other = cd.GradClip(1000), cd.GradClip(1000)
    out = [torch.empty_like(t) for t in grads]
    norm = torch.empty((), dtype=torch.float64, device="cuda")
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        cd.countdown_clip_grads(clip, grads, 2.0, out=out, norm=norm)
    for k in range(3):
        for t in grads:
            t.mul_(1.0 + k)
        want = math.sqrt(math.fsum(float((t.double() ** 2).sum()) for t in grads))
        place = [t.clone() for t in grads]
        eager = cd.countdown_clip_grads(other, place, 2.0)
        assert abs(float(eager) - want) <= 2.0 ** -52 * (sum(sizes) / 2 + 2) * want
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(norm, eager)
        for o, p, t in zip(out, place, grads):
            assert torch.equal(o, p)
            check(o, t, 2.0 / float(norm))
    clip.close()
    other.close()
