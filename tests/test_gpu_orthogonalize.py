"""Orthogonalised updates on the GPU against Newton-Schulz in 64 bits."""
import numpy as np
import pytest

from tests import step_formulas as F

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
MUON = (3.4445, -4.7750, 2.0315)
TAYLOR = (1.875, -1.25, 0.375)     # converges to exactly orthogonal rows


@pytest.fixture(scope="module")
def dp():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_40335_amd.dpghost as d
    d.lib()
    return d


def _say(*a):
    print(*a, flush=True)


def _f32(coef):
    return [tuple(float(np.float32(v)) for v in k) for k in coef]


def _matrix(seed, r, c, dt, pad=0, off=0, signal=0.5):
    """A noised sum: low rank under noise, rows c + pad apart."""
    g = torch.Generator().manual_seed(seed)
    k = min(3, r, c)
    m = torch.randn(r, k, generator=g) @ torch.randn(k, c, generator=g)
    m = torch.randn(r, c, generator=g) + signal * m * (r * c) ** 0.5 / m.norm()
    buf = torch.full((off + r * (c + pad),), 7.0, dtype=DT[dt], device="cuda")
    v = buf[off:].view(r, c + pad)[:, :c]
    v.copy_(m * 0.03)
    return v


def _check(got, G, coef, eps, out, what, scale=1.0, prior=None):
    ref, fro, elem = F.newton_schulz_error(G.detach().cpu().double().numpy(), _f32(coef), eps, out)
    ref, fro, elem = ref * scale, fro * abs(scale), elem * abs(scale)
    if prior is not None:
        ref = ref + prior
    d = np.abs(got.detach().cpu().double().numpy() - ref)
    bound = elem + HALF[out] * (np.abs(ref) + elem) + 2 * F.U * (np.abs(ref) + elem)
    whole = fro + 2 * HALF[out] * np.linalg.norm(ref)
    _say(f"  {what}: {np.linalg.norm(d) / whole:.3f} of the whole's bound, {np.max(d / bound):.3f} of an element's")
    assert np.linalg.norm(d) <= whole and (d <= bound).all(), what


SHAPES = [(1, 1), (1, 300), (300, 1), (7, 5), (64, 192), (128, 128), (129, 257), (257, 129),
          (100, 1000), (640, 130)]


@pytest.mark.parametrize("dt,out", [("f32", "f32"), ("f32", "bf16"), ("bf16", "f32"), ("bf16", "bf16")])
def test_group_of_all_shapes(dp, dt, out):
    grads = [_matrix(k, r, c, dt, pad=k % 3, off=k % 2) for k, (r, c) in enumerate(SHAPES)]
    outs = [_matrix(50 + k, r, c, out, pad=k % 2, off=k % 3) for k, (r, c) in enumerate(SHAPES)]
    dp.dp_orthogonalize_grouped(grads, outs)
    for k, (g, o) in enumerate(zip(grads, outs)):
        _check(o, g, [MUON] * 5, 1e-7, out, f"{dt}->{out} {SHAPES[k]}")
        if o._base is not None:
            assert int((o._base == 7).sum()) == k % 3 + SHAPES[k][0] * (k % 2), SHAPES[k]
    again = [torch.empty_like(o) for o in outs]
    dp.dp_orthogonalize_grouped(grads, again)
    for o, p in zip(outs, again):
        assert torch.equal(o, p)
    alone = torch.empty_like(outs[6])
    dp.dp_orthogonalize_grouped([grads[6]], [alone])
    assert torch.equal(alone, outs[6])


@pytest.mark.parametrize("r,c", [(768, 768), (1024, 2000), (2304, 768)])
@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_larger_matrices(dp, r, c, out):
    g = _matrix(1, r, c, "f32")
    o = torch.empty(r, c, dtype=DT[out], device="cuda")
    dp.dp_orthogonalize_grouped([g], [o])
    _check(o, g, [MUON] * 5, 1e-7, out, f"{out} {r}x{c}")


def test_step_counts_and_coefficients_per_step(dp):
    g = _matrix(2, 90, 200, "f32")
    o = torch.empty_like(g)
    for steps in (1, 2, 3):
        dp.dp_orthogonalize_grouped([g], [o], steps=steps)
        _check(o, g, [MUON] * steps, 1e-7, "f32", f"{steps} steps")
    mixed = [MUON, MUON, TAYLOR, (2.0, -1.5, 0.5)]
    dp.dp_orthogonalize_grouped([g], [o], coef=mixed, steps=4)
    _check(o, g, mixed, 1e-7, "f32", "a triple per step")
    # Enough steps make the rows orthonormal.
    dp.dp_orthogonalize_grouped([g], [o], coef=[MUON] * 5 + [TAYLOR] * 6, steps=11)
    x = o.double()
    assert float((x @ x.T - torch.eye(90, device="cuda", dtype=torch.float64)).abs().max()) < 90 * 2.0 ** -20


@pytest.mark.parametrize("n,r,c", [(48, 1200, 650), (14, 1850, 1950)])
def test_many_larger_matrices(dp, n, r, c):
    """Enough output for the largest tiles, whose last rows and columns reach past the matrix."""
    grads = [_matrix(k, r, c, "bf16") for k in range(n)]
    outs = [torch.empty_like(g) for g in grads]
    dp.dp_orthogonalize_grouped(grads, outs)
    for k in (0, n - 1):
        _check(outs[k], grads[k], [MUON] * 5, 1e-7, "bf16", f"matrix {k} of {n}")
    for k in range(1, n - 1):      # the rest: rows (or columns) of like length, as the two checked
        x = outs[k].float()
        assert torch.isfinite(x).all() and abs(float(x.norm() / outs[0].float().norm()) - 1) < 0.05, k


@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_scaled_onto_a_prior_and_in_place(dp, out):
    shapes = [(130, 70), (70, 130)]
    grads = [_matrix(k, r, c, out) for k, (r, c) in enumerate(shapes)]
    outs = [_matrix(9 + k, r, c, out) for k, (r, c) in enumerate(shapes)]
    prior = [o.cpu().double().numpy() for o in outs]
    dp.dp_orthogonalize_grouped(grads, outs, scale=[-0.25, 2.0], accumulate=True)
    for g, o, p, s in zip(grads, outs, prior, (-0.25, 2.0)):
        _check(o, g, [MUON] * 5, 1e-7, out, f"added, scale {s}", scale=s, prior=p)
    keep = [g.clone() for g in grads]
    dp.dp_orthogonalize_grouped(grads, grads)
    for g, k in zip(grads, keep):
        _check(g, k, [MUON] * 5, 1e-7, out, "in place")


def test_extreme_matrices(dp):
    """Zero and one-element matrices, magnitudes whose squares leave fp32, NaN and inf beside
    a good matrix, a matrix of rank one, identical rows."""
    base = _matrix(3, 50, 80, "f32")
    one = torch.zeros(50, 80, device="cuda")
    one[7, 9] = -3.0
    rank1 = torch.ones(50, 80, device="cuda")
    bad, worse = base.clone(), base.clone()
    bad[49, 79] = float("nan")
    worse[0, 0] = float("inf")
    grads = [torch.zeros(50, 80, device="cuda"), one, base * 1e30, base * 1e-30, bad, rank1, worse, base]
    outs = [torch.full((50, 80), 5.0, device="cuda") for _ in grads]
    dp.dp_orthogonalize_grouped(grads, outs, eps=0.0 + 1e-38)
    assert not outs[0].any()
    s = 1.0
    for _ in range(5):
        s = MUON[0] * s + MUON[1] * s ** 3 + MUON[2] * s ** 5
    assert abs(float(outs[1][7, 9]) + s) < 1e-5 and int(outs[1].count_nonzero()) == 1
    for k in (2, 3, 5, 7):
        _check(outs[k], grads[k], [MUON] * 5, 1e-38, "f32", f"matrix {k}")
    assert torch.isnan(outs[4]).all() and torch.isnan(outs[6]).all()


def test_more_matrices_than_one_launch_takes(dp):
    n = 60
    grads = [_matrix(k, 8 + k, 100 - k, "f32") for k in range(n)]
    outs = [torch.empty_like(g) for g in grads]
    dp.dp_orthogonalize_grouped(grads, outs)
    for k in (0, 46, 55, 56, 59):
        _check(outs[k], grads[k], [MUON] * 5, 1e-7, "f32", f"matrix {k}")


def test_captured_and_replayed(dp):
    g = [_matrix(1, 200, 70, "f32"), _matrix(2, 64, 300, "f32")]
    o = [torch.empty_like(x) for x in g]
    dp.dp_orthogonalize_grouped(g, o)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dp.dp_orthogonalize_grouped(g, o)
    for k in range(3):
        for x in g:
            x.normal_()
        graph.replay()
        torch.cuda.synchronize()
        e = [torch.empty_like(x) for x in g]
        dp.dp_orthogonalize_grouped(g, e)
        torch.cuda.synchronize()
        for p, q in zip(o, e):
            assert torch.equal(p, q)
