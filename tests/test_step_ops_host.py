"""LayerNorm, the head's losses: what the C ABI refuses, on a host without a GPU.

Only invalid arguments reach an entry point here: each must be refused before
any HIP call. The loss and gradient formulas are checked against autograd and
differences on the CPU (the same formulas judge the kernels on the GPU)."""
import os

import numpy as np
import pytest

from paper_2609_40335_amd import build as B
from paper_2609_40335_amd import dpghost as D

torch = pytest.importorskip("torch")
EINVAL, EUNSUP = 1, 2
P = [1 << (20 + i) for i in range(10)]   # made-up device addresses


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(D.library_path()):
        B.build()
    return D.lib()


def _forward(L, **kw):
    a = dict(x=P[0], ldx=64, gain=P[1], bias=P[2], pdt=0, B=2, T=3, d=64, dt=0, eps=1e-5, y=P[3],
             ldy=64, mean=P[4], rstd=P[5])
    a.update(kw)
    return L.dp_layernorm_forward(*a.values(), None)


@pytest.mark.parametrize("kw,status", [
    (dict(x=None), EINVAL), (dict(y=None), EINVAL), (dict(B=0), EINVAL), (dict(T=-1), EINVAL),
    (dict(d=0), EINVAL), (dict(dt=2), EINVAL), (dict(pdt=7), EINVAL), (dict(ldx=63), EINVAL),
    (dict(ldy=63), EINVAL), (dict(eps=-1.0), EINVAL), (dict(eps=float("nan")), EINVAL),
    (dict(y=P[0], ldy=128), EINVAL), (dict(B=1 << 16, T=1 << 16), EUNSUP),
    (dict(B=1, T=2 ** 31 - 2 ** 16 + 1), EUNSUP),
    (dict(d=32769, ldx=32769, ldy=32769), EUNSUP)])
def test_layernorm_forward_refuses(L, kw, status):
    assert _forward(L, **kw) == status, L.dp_last_error()


def _backward(L, **kw):
    a = dict(gy=P[0], ldgy=64, x=P[1], ldx=64, gain=P[2], pdt=0, mean=P[3], rstd=P[4], B=2, T=300,
             d=64, dt=1, dx=P[5], lddx=64, acc_dx=0, dgain=P[6], dbias=P[7], norm2=P[8], acc=0,
             ws=P[9], nbytes=1 << 30)
    a.update(kw)
    return L.dp_layernorm_backward(*a.values(), None)


@pytest.mark.parametrize("kw,status", [
    (dict(gy=None), EINVAL), (dict(x=None), EINVAL), (dict(mean=None), EINVAL),
    (dict(rstd=None), EINVAL), (dict(dx=None, dgain=None, dbias=None), EINVAL),
    (dict(dgain=None, dbias=None), EINVAL), (dict(ldgy=63), EINVAL), (dict(ldx=1), EINVAL),
    (dict(lddx=63), EINVAL), (dict(dx=P[0], lddx=72), EINVAL), (dict(dx=P[1], lddx=72), EINVAL),
    (dict(ws=None), EINVAL), (dict(nbytes=16), EINVAL), (dict(ws=P[9] + 4), EINVAL),
    (dict(dt=-1), EINVAL), (dict(pdt=2), EINVAL), (dict(T=0), EINVAL),
    (dict(d=1 << 16, ldgy=1 << 16, ldx=1 << 16, lddx=1 << 16), EUNSUP)])
def test_layernorm_backward_refuses(L, kw, status):
    assert _backward(L, **kw) == status, L.dp_last_error()


def test_layernorm_workspace(L):
    f = L.dp_layernorm_backward_workspace
    assert f(4, 16, 64) == 0                       # one range per example
    assert f(0, 16, 64) == f(4, 0, 64) == f(4, 16, 0) == f(4, 16, 40000) == 0
    assert f(1, 4096, 768) >= 2 * 768 * 4          # ranges of a long example
    assert f(2000, 128, 768) == 0                  # enough examples to fill the GPU
    most = 2 ** 31 - 2 ** 16                       # the longest: sizes do not overflow
    assert f(most, 1, 8) == 0 and 0 < f(1, most, 8) < 1 << 20
    assert f(1, most + 1, 8) == f(most + 1, 1, 8) == 0
    assert L.dp_preference_loss_workspace(1, most) >= 16 * most


def _losses(L, which, **kw):
    a = dict(Z=P[0], ldz=100, targets=P[1])
    if which == "logprobs":
        a.update(B=2, T=4, V=100, dt=0, logp=P[2], lse=None)
    elif which == "ce":
        a.update(w=P[2], B=2, T=4, V=100, dt=0, logp=None, Gz=P[3], ldg=100)
    else:
        a.update(split=2, ref=None, beta=0.1, eps=0.0, B=2, T=4, V=100, dt=1, loss=P[2],
                 rewards=None, logp=None, Gz=P[3], ldg=100, ws=P[4], nbytes=1 << 20)
    a.update(kw)
    f = {"logprobs": L.dp_token_logprobs, "ce": L.dp_cross_entropy, "pref": L.dp_preference_loss}
    return f[which](*a.values(), None)


@pytest.mark.parametrize("which", ["logprobs", "ce", "pref"])
@pytest.mark.parametrize("kw,status", [
    (dict(Z=None), EINVAL), (dict(targets=None), EINVAL), (dict(B=0), EINVAL), (dict(T=0), EINVAL),
    (dict(V=0), EINVAL), (dict(ldz=99), EINVAL), (dict(dt=9), EINVAL),
    (dict(B=1 << 20, T=1 << 12), EUNSUP),
    (dict(V=(1 << 30) + 1, ldz=1 << 31), EUNSUP)])
def test_losses_refuse(L, which, kw, status):
    assert _losses(L, which, **kw) == status, L.dp_last_error()


@pytest.mark.parametrize("which,kw", [
    ("logprobs", dict(logp=None)), ("ce", dict(w=None)), ("ce", dict(Gz=None)), ("ce", dict(ldg=99)),
    ("ce", dict(Gz=P[0], ldg=104)), ("pref", dict(loss=None)), ("pref", dict(split=-1)),
    ("pref", dict(split=5)), ("pref", dict(beta=0.0)), ("pref", dict(beta=float("inf"))),
    ("pref", dict(eps=0.5)), ("pref", dict(eps=-0.1)), ("pref", dict(eps=float("nan"))),
    ("pref", dict(ldg=99)), ("pref", dict(Gz=P[0], ldg=104)), ("pref", dict(ws=None)),
    ("pref", dict(nbytes=8)), ("pref", dict(ws=P[4] + 8))])
def test_each_loss_refuses(L, which, kw):
    assert _losses(L, which, **kw) == EINVAL, L.dp_last_error()


def test_binding_refuses_host_tensors_and_wrong_shapes(monkeypatch):
    x = torch.zeros(2, 3, 8)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    with pytest.raises(D.DPError, match="device tensor"):
        D.dp_layernorm_forward(x, None, None, x)
    with pytest.raises(D.DPError, match="device tensor"):
        D.dp_token_logprobs(x, torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, 3))
    with pytest.raises(D.DPError, match="fp32"):
        D._f32(torch.zeros(2, 3, dtype=torch.float64), (2, 3), "mean")
    with pytest.raises(D.DPError, match="shape and dtype"):
        D._like(torch.zeros(2, 3, 9), x.shape, x.dtype, "y", "x")
    with pytest.raises(D.DPError, match="gain"):
        D._params(8, torch.zeros(7))
    with pytest.raises(D.DPError, match="one dtype"):
        D._params(8, torch.zeros(8), torch.zeros(8, dtype=torch.bfloat16))


def _autograd_preference(z, targets, split, ref, beta, eps):
    """Loss of each pair from torch's own log_softmax and logsigmoid."""
    logp = torch.log_softmax(z, 2).gather(2, targets.clamp(min=0)[:, :, None])[:, :, 0]
    ratio = torch.where(targets >= 0, logp - ref, torch.zeros_like(logp))
    m = beta * (ratio[:, :split].sum(1) - ratio[:, split:].sum(1))
    ls = torch.nn.functional.logsigmoid
    return -(1 - eps) * ls(m) - eps * ls(-m)


def test_preference_formula_against_autograd_and_differences():
    from tests.step_formulas import preference
    g = torch.Generator().manual_seed(3)
    z = torch.randn(3, 6, 11, generator=g, dtype=torch.float64)
    y = torch.randint(0, 11, (3, 6), generator=g)
    y[0, 1] = y[2, 5] = -1
    ref = torch.randn(3, 6, generator=g, dtype=torch.float64)
    for eps in (0.0, 0.2):
        got = preference(z.numpy(), y.numpy(), 2, ref.numpy(), 0.7, eps)
        zz = z.clone().requires_grad_()
        loss = _autograd_preference(zz, y, 2, ref, 0.7, eps)
        loss.sum().backward()
        np.testing.assert_allclose(got["loss"], loss.detach().numpy(), rtol=1e-12)
        np.testing.assert_allclose(got["Gz"], zz.grad.numpy(), rtol=1e-10, atol=1e-14)
        h = 1e-6
        for at in ((0, 0, 3), (1, 4, 0), (2, 5, 2)):
            lo, hi = z.clone(), z.clone()
            lo[at] -= h
            hi[at] += h
            d = (preference(hi.numpy(), y.numpy(), 2, ref.numpy(), 0.7, eps)["loss"][at[0]]
                 - preference(lo.numpy(), y.numpy(), 2, ref.numpy(), 0.7, eps)["loss"][at[0]]) / (2 * h)
            assert abs(d - got["Gz"][at]) < 1e-8


def test_layernorm_formula_against_autograd():
    from tests.step_formulas import layernorm, layernorm_backward
    g = torch.Generator().manual_seed(4)
    x = torch.randn(2, 5, 12, generator=g, dtype=torch.float64).requires_grad_()
    gain = torch.randn(12, generator=g, dtype=torch.float64).requires_grad_()
    bias = torch.randn(12, generator=g, dtype=torch.float64).requires_grad_()
    gy = torch.randn(2, 5, 12, generator=g, dtype=torch.float64)
    y = torch.nn.functional.layer_norm(x, (12,), gain, bias, 1e-5)
    y.backward(gy)
    ours, mean, rstd = layernorm(x.detach().numpy(), gain.detach().numpy(), bias.detach().numpy(), 1e-5)
    np.testing.assert_allclose(ours, y.detach().numpy(), rtol=1e-12, atol=1e-12)
    back = layernorm_backward(gy.numpy(), x.detach().numpy(), gain.detach().numpy(), mean, rstd)
    np.testing.assert_allclose(back["dx"], x.grad.numpy(), rtol=1e-10, atol=1e-12)
    np.testing.assert_allclose(back["dgain"].sum(0), gain.grad.numpy(), rtol=1e-11)
    np.testing.assert_allclose(back["dbias"].sum(0), bias.grad.numpy(), rtol=1e-11)


def _matrix(G=P[0], ldg=640, out=P[1], ldo=640, rows=320, cols=640, scale=1.0):
    return D.dp_matrix_t(G, ldg, out, ldo, rows, cols, scale)


def _orth(L, m=None, n=1, dt=0, odt=0, coef=(1.0, 2.0, 3.0), steps=1, eps=0.0, ws=P[2], nbytes=1 << 40):
    import ctypes
    arr = (D.dp_matrix_t * 1)(m if m is not None else _matrix())
    cf = None if coef is None else (ctypes.c_float * len(coef))(*coef)
    return L.dp_orthogonalize_grouped(arr, n, dt, odt, cf, steps, eps, 0, ws, nbytes, None)


@pytest.mark.parametrize("kw,status", [
    (dict(n=0), EINVAL), (dict(dt=3), EINVAL), (dict(odt=3), EINVAL), (dict(coef=None), EINVAL),
    (dict(coef=(1.0, float("nan"), 0.0)), EINVAL), (dict(steps=0), EINVAL),
    (dict(steps=65, coef=(0.0,) * 195), EINVAL), (dict(eps=-1.0), EINVAL),
    (dict(eps=float("inf")), EINVAL), (dict(ws=None), EINVAL), (dict(nbytes=64), EINVAL),
    (dict(ws=P[2] + 2), EINVAL), (dict(m=_matrix(G=None)), EINVAL), (dict(m=_matrix(out=None)), EINVAL),
    (dict(m=_matrix(ldg=639)), EINVAL), (dict(m=_matrix(ldo=639)), EINVAL),
    (dict(m=_matrix(rows=0)), EINVAL), (dict(m=_matrix(cols=-1)), EINVAL),
    (dict(m=_matrix(scale=float("nan"))), EINVAL), (dict(m=_matrix(rows=65537)), EUNSUP),
    (dict(m=_matrix(cols=65537, ldg=65537, ldo=65537)), EUNSUP)])
def test_orthogonalize_refuses(L, kw, status):
    assert _orth(L, **kw) == status, L.dp_last_error()


def test_orthogonalize_workspace(L):
    one, tall = (D.dp_matrix_t * 1)(_matrix()), (D.dp_matrix_t * 1)(_matrix(rows=640, cols=320, ldg=320, ldo=320))
    assert L.dp_orthogonalize_workspace(one, 1, D.DP_BF16) == L.dp_orthogonalize_workspace(tall, 1, D.DP_BF16)
    assert L.dp_orthogonalize_workspace(one, 1, D.DP_F32) > L.dp_orthogonalize_workspace(one, 1, D.DP_BF16) > 0
    assert L.dp_orthogonalize_workspace(None, 1, D.DP_F32) == 0
    small = (D.dp_matrix_t * 1)(_matrix(rows=64, cols=256))      # worked in LDS
    assert L.dp_orthogonalize_workspace(small, 1, D.DP_F32) == 0
    assert L.dp_orthogonalize_workspace(one, 0, D.DP_F32) == 0


def test_newton_schulz_formula():
    """Singular values follow the polynomial; singular vectors stay."""
    from tests.step_formulas import newton_schulz
    g = np.random.default_rng(5).standard_normal((9, 17))
    u, s, v = np.linalg.svd(g, full_matrices=False)
    for G, (uu, vv) in ((g, (u, v)), (g.T, (v.T, u.T))):
        x = s / np.linalg.norm(g)
        for a, b, c in ((3.0, -2.0, 0.5), (1.5, -0.5, 0.0)):
            x = a * x + b * x ** 3 + c * x ** 5
        np.testing.assert_allclose(newton_schulz(G, [(3.0, -2.0, 0.5), (1.5, -0.5, 0.0)], 0.0),
                                   uu @ np.diag(x) @ vv, atol=1e-13)
