"""LayerNorm's backward pass over few features and long examples, whose token sums are
joined from hundreds of ranges.

A range has 16 to 20 tokens here: 2 or 3 additions in a lane, 8 across its waves. Ranges are added by 16
threads, then those: at most 512 / 16 + 16. So no term meets more than 64 additions, each off by at
most U of what stands there, which the sum of magnitudes bounds."""
import numpy as np
import pytest

from tests import step_formulas as F

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

DEPTH = 64
CASES = [(1, 8192, 64, "f32"), (2, 5000, 16, "f32"), (1, 8192, 1, "bf16"), (1, 8192, 65, "f32")]


@pytest.fixture(scope="module")
def dp():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_40335_amd.dpghost as d
    d.lib()
    return d


def _run(dp, gy, x, mean, rstd, prior=None):
    B, T, d = x.shape
    dx, dg, db = torch.empty_like(x), torch.empty(B, d, device="cuda"), torch.empty(B, d, device="cuda")
    n2 = torch.empty(B, device="cuda") if prior is None else prior.clone()
    dp.dp_layernorm_backward(gy, x, None, mean, rstd, dx, dgain=dg, dbias=db, norm2=n2,
                             accumulate=prior is not None)
    return [t.cpu().double().numpy() for t in (dx, dg, db, n2)]


@pytest.mark.parametrize("B,T,d,dt", CASES)
def test_a_large_term_among_many_small_ones(dp, B, T, d, dt):
    """2^24 in the first token and ones after it: added one by one behind it, all would be lost."""
    x = torch.ones(B, T, d, device="cuda", dtype=torch.bfloat16 if dt == "bf16" else torch.float32)
    gy = torch.zeros_like(x)
    gy[:, ::20] = 1
    gy[:, 0] = 2.0 ** 24
    mean, rstd = torch.zeros(B, T, device="cuda"), torch.ones(B, T, device="cuda")
    _, dg, db, n2 = _run(dp, gy, x, mean, rstd)
    want = 2.0 ** 24 + (T - 1) // 20
    for got in (dg, db):
        assert np.abs(got - want).max() <= DEPTH * F.U * want, (np.abs(got - want).max(), B, T, d)
    np.testing.assert_allclose(n2, 2 * d * want ** 2, rtol=(2 * DEPTH + d + 8) * F.U)


@pytest.mark.parametrize("B,T,d,dt", CASES)
def test_long_examples_of_few_features(dp, B, T, d, dt):
    g = torch.Generator(device="cuda").manual_seed(3)
    kind = torch.bfloat16 if dt == "bf16" else torch.float32
    x, gy = (torch.randn(B, T, d, device="cuda", generator=g).to(kind) for _ in range(2))
    mean, rstd = x.float().mean(2) + 0.1, torch.rand(B, T, device="cuda", generator=g) + 0.5
    prior = torch.full((B,), 7.0, device="cuda")
    dx, dg, db, n2 = _run(dp, gy, x, mean, rstd, prior)
    args = [t.cpu().double().numpy() for t in (gy, x)] + [np.ones(d)] + \
        [t.cpu().double().numpy() for t in (mean, rstd)]
    ref, err = F.layernorm_backward(*args), F.layernorm_backward_error(*args)
    xhat = np.abs(args[1] - args[3][..., None]) * args[4][..., None]
    sg, sb = (np.abs(args[0]) * xhat).sum(1), np.abs(args[0]).sum(1)
    eg, eb = (DEPTH + 8) * F.U * sg, DEPTH * F.U * sb
    half = 2.0 ** -8 if dt == "bf16" else F.U
    assert (np.abs(dx - ref["dx"]) <= err["dx"] + half * (np.abs(ref["dx"]) + err["dx"]) + 1e-37).all()
    assert (np.abs(dg - ref["dgain"]) <= eg).all() and (np.abs(db - ref["dbias"]) <= eb).all()
    want = ref["norm2"] + 7
    en = (2 * np.abs(ref["dgain"]) * eg + eg ** 2 + 2 * np.abs(ref["dbias"]) * eb + eb ** 2).sum(1)
    assert (np.abs(n2 - want) <= en + (d + DEPTH) * F.U * want).all()
