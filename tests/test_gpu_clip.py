"""The global gradient norm and clipping against 64-bit arithmetic.

Tolerances. Squares of fp32 and bf16 values are exact in fp64; n additions are off by at
most n * 2^-52 of the sum, the root halves that: norms here are held to 2^-52 (n / 2 + 2).
A scaled value has three roundings in fp32 (the coefficient, the product; the norm's is
smaller) and one to its type: 2 * 2^-24 and half a step of the type, relative."""
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


def make(seed, sizes, types):
    g = torch.Generator().manual_seed(seed)
    return [(torch.randn(n, generator=g) * 0.3).to(types[i % len(types)]).cuda()
            for i, n in enumerate(sizes)]


def norm_of(grads):
    return math.sqrt(math.fsum(float((t.double() ** 2).sum()) for t in grads))


def check_norm(got, grads):
    n = sum(t.numel() for t in grads)
    want = norm_of(grads)
    assert abs(float(got) - want) <= 2.0 ** -52 * (n / 2 + 2) * want


def check_scaled(got, grad, coef):
    want = grad.double() * coef
    tol = (2.0 ** -23 + torch.finfo(grad.dtype).eps / 2) * want.abs() + 1e-45
    assert bool(((got.double() - want).abs() <= tol).all())


SIZES = [
    [1], [7], [8, 1, 3], [0, 5, 0], [16384], [16385, 16383], [40000, 3, 100001],
    [1 << 20, 77], [12345] * 33, [11] * 97, [129] * 200, [3_000_001],
]


@pytest.mark.parametrize("types", [(F32,), (BF16,), (F32, BF16)])
@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: f"{len(s)}x{max(s)}")
def test_norm_and_clip(cd, sizes, types):
    grads = make(1, sizes, types)
    with cd.GradClip(len(sizes)) as clip:
        keep = [t.clone() for t in grads]
        norm = cd.countdown_clip_grads(clip, grads, math.inf)
        assert norm.dtype == torch.float64 and norm.shape == ()
        check_norm(norm, keep)
        assert all(torch.equal(a, b) for a, b in zip(grads, keep))
        top = float(norm) * 0.37
        out = [torch.full_like(t, 9.0) for t in grads]
        again = cd.countdown_clip_grads(clip, grads, top, out=out)
        assert torch.equal(again, norm)
        assert all(torch.equal(a, b) for a, b in zip(grads, keep))
        for o, t in zip(out, keep):
            check_scaled(o, t, top / float(norm))
        cd.countdown_clip_grads(clip, grads, top)  # in place
        assert all(torch.equal(a, b) for a, b in zip(grads, out))


def test_under_the_limit_nothing_changes(cd):
    grads = make(2, [1000, 70001], (F32, BF16))
    keep = [t.clone() for t in grads]
    with cd.GradClip(2) as clip:
        norm = float(cd.countdown_clip_grads(clip, grads, math.inf))
        for top in (norm, norm * 1.5, 1e300):
            out = [torch.zeros_like(t) for t in grads]
            cd.countdown_clip_grads(clip, grads, top, out=out)
            cd.countdown_clip_grads(clip, grads, top)
            for a, b, o in zip(grads, keep, out):
                assert torch.equal(a, b) and torch.equal(o, b)
        cd.countdown_clip_grads(clip, grads, math.inf, out=out)
        assert all(torch.equal(o, b) for o, b in zip(out, keep))
        cd.countdown_clip_grads(clip, grads, 0.0)
        assert not any(t.any() for t in grads)
        assert float(cd.countdown_clip_grads(clip, grads, 1.0)) == 0.0  # a norm of zero
        assert float(cd.countdown_clip_grads(clip, [], 1.0)) == 0.0


def test_offsets_and_alignment(cd):
    """Gradients that are views at odd element offsets, with outputs at others."""
    for dtype in (F32, BF16):
        flat = make(3, [60000], (dtype,))[0]
        dst = torch.full((60100,), 5.0, dtype=dtype, device="cuda")
        cuts = [(1, 3), (5, 20), (26, 33000), (33027, 20001)]
        grads = [flat[o:o + n] for o, n in cuts]
        for shift in (0, 1, 5):
            out = [dst[o + shift:o + shift + n] for o, n in cuts]
            dst.fill_(5.0)
            with cd.GradClip(4) as clip:
                norm = cd.countdown_clip_grads(clip, grads, 1.0, out=out)
            check_norm(norm, grads)
            for o, t in zip(out, grads):
                check_scaled(o, t, 1.0 / float(norm))
            left = torch.ones(60100, dtype=torch.bool, device="cuda")
            for o, n in cuts:
                left[o + shift:o + shift + n] = False
            assert bool((dst[left] == 5.0).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("sizes", [[65536], [65535, 1], [65537], [4096] * 16, [4097] * 15, [2049] * 31,
                                   [1] * 32, [4095, 4096, 4097, 1, 0, 9, 30000]])
def test_one_workgroup_and_its_edges(cd, sizes, dtype):
    """Up to 65536 elements, one or two chunks a wave: views at odd offsets, outputs at the
    same alignment, at another and in place."""
    total = sum(n + 3 for n in sizes)
    flat = make(6, [total + 16], (dtype,))[0]
    starts = [1 + sum(m + 3 for m in sizes[:i]) for i in range(len(sizes))]
    views = lambda buf, shift: [buf[s + shift:s + shift + n]  # noqa: E731
                                for s, n in zip(starts, sizes)]
    grads = views(flat, 0)
    inside = torch.zeros(total + 16, dtype=torch.bool, device="cuda")
    with cd.GradClip(len(sizes)) as clip:
        for top in (0.5, 1e30, math.inf):
            for shift in (0, 1, 8):
                dst = torch.full((total + 16,), 5.0, dtype=dtype, device="cuda")
                norm = cd.countdown_clip_grads(clip, grads, top, out=views(dst, shift))
                check_norm(norm, grads)
                coef = min(1.0, top / float(norm))
                for o, t in zip(views(dst, shift), grads):
                    check_scaled(o, t, coef)
                    assert coef < 1.0 or torch.equal(o, t)
                inside.zero_()
                for v in views(inside, shift):
                    v.fill_(True)
                assert bool((dst[~inside] == 5.0).all())
        place = flat.clone()
        norm = cd.countdown_clip_grads(clip, views(place, 0), 0.5)
        want = torch.empty_like(flat).copy_(flat)
        cd.countdown_clip_grads(clip, grads, 0.5, out=views(want, 0))
        assert torch.equal(place, want)
        for o, t in zip(views(place, 0), grads):
            check_scaled(o, t, min(1.0, 0.5 / float(norm)))


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_bad_numbers_leave_the_gradients(cd, bad, dtype):
    grads = make(4, [5000, 100], (dtype,))
    grads[1][7] = bad
    keep = [t.clone() for t in grads]
    out = [torch.zeros_like(t) for t in grads]
    with cd.GradClip(2) as clip:
        norm = float(cd.countdown_clip_grads(clip, grads, 1.0, out=out))
        assert math.isnan(norm) if math.isnan(bad) else norm == math.inf
        cd.countdown_clip_grads(clip, grads, 1.0)
    bits = torch.int32 if dtype == F32 else torch.int16
    for a, o, b in zip(grads, out, keep):
        assert torch.equal(a.view(bits), b.view(bits)) and torch.equal(o.view(bits), b.view(bits))


def test_huge_and_tiny_values(cd):
    """Squares past fp32's range, and below its smallest value."""
    with cd.GradClip(2) as clip:
        big = [torch.full((1000,), 3e38, device="cuda"), torch.full((10,), 1.0, device="cuda")]
        norm = float(cd.countdown_clip_grads(clip, big, 1.0))
        assert abs(norm / (math.sqrt(1000.0) * float(torch.tensor(3e38))) - 1) < 1e-12
        tiny = [torch.full((1000,), 1e-30, device="cuda")]
        norm = float(cd.countdown_clip_grads(clip, tiny, math.inf))
        assert abs(norm / (math.sqrt(1000.0) * float(torch.tensor(1e-30))) - 1) < 1e-12


def test_more_elements_than_32_bits_of_bytes(cd):
    """One tensor of 2^31 + 5 bf16 elements: offsets past 32 bits, more chunks than workgroups."""
    n = 2 ** 31 + 5
    t = torch.zeros(n, dtype=BF16, device="cuda")
    at = [0, 2 ** 31 - 1, 2 ** 31, n - 1]
    for i in at:
        t[i] = 3.0
    with cd.GradClip(1) as clip:
        assert float(cd.countdown_clip_grads(clip, [t], 3.0)) == 6.0
    assert all(float(t[i]) == 1.5 for i in at)
    assert int((t != 0).sum()) == len(at)


def test_graph_replays(cd):
    grads = make(5, [5000, 70001, 3], (F32, BF16))
    out = [torch.empty_like(t) for t in grads]
    clip, other = cd.GradClip(3), cd.GradClip(3)
    norm = torch.empty((), dtype=torch.float64, device="cuda")
    stream = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        cd.countdown_clip_grads(clip, grads, 1.0, out=out, norm=norm)
    for seed in (6, 7, 8):
        for t, v in zip(grads, make(seed, [5000, 70001, 3], (F32, BF16))):
            t.copy_(v)
        want = [torch.empty_like(t) for t in grads]
        wnorm = cd.countdown_clip_grads(other, grads, 1.0, out=want)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(norm, wnorm) and all(torch.equal(a, b) for a, b in zip(out, want))
    clip.close()
    other.close()


def test_refusals(cd):
    a, b = torch.ones(16, device="cuda"), torch.ones(16, device="cuda")
    clip = cd.GradClip(2)
    for grads, top, out, err in [
            ([a, b], -1.0, None, cd.CountdownError), ([a, b], math.nan, None, cd.CountdownError),
            ([a, b, a[:0]], 1.0, None, cd.CountdownError),  # more than max_tensors
            ([a, a], 1.0, None, cd.CountdownError),         # the same gradient twice, in place
            ([a, b], 1.0, [a, a], cd.CountdownError), ([a, b], 1.0, [b, a], cd.CountdownError),
            ([a, a[4:]], 1.0, None, cd.CountdownError),
            ([a[:8]], 1.0, [a[4:12]], cd.CountdownError),
            ([a.half()], 1.0, None, TypeError), ([a.cpu()], 1.0, None, ValueError),
            ([a[::2]], 1.0, None, ValueError), ([a], 1.0, [b[:8]], ValueError),
            ([a], 1.0, [b.bfloat16()], ValueError), ([a], 1.0, [a, b], ValueError)]:
        with pytest.raises(err):
            cd.countdown_clip_grads(clip, grads, top, out=out)
    for norm in (torch.empty(2, dtype=torch.float64, device="cuda"), torch.empty(1, device="cuda")):
        with pytest.raises(ValueError):
            cd.countdown_clip_grads(clip, [a], 1.0, norm=norm)
    assert bool((a == 1).all()) and bool((b == 1).all())
    assert float(cd.countdown_clip_grads(clip, [a, a], math.inf)) == math.sqrt(32.0)  # counted twice
    clip.close()
    with pytest.raises(ValueError):
        cd.countdown_clip_grads(clip, [a], 1.0)
