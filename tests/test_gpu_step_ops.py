"""LayerNorm and the head's losses on the GPU against their formulas in 64 bits.

Bounds come from tests/step_formulas.py (roundings counted); an output of the
operands' type may be off by half a step more."""
import numpy as np
import pytest

from tests import step_formulas as F

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


@pytest.fixture(scope="module")
def dp():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_40335_amd.dpghost as d
    d.lib()
    return d


def _say(*a):
    print(*a, flush=True)


def _host(t):
    return t.detach().cpu().double().numpy()


def _normal(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed))


def _rows_of(t, dt, ld, off=0):
    """t [B, T, w] on the GPU with rows ld apart, off elements into its buffer; what lies
    between the rows is 7."""
    B, T, w = t.shape
    buf = torch.full((off + B * T * ld,), 7.0, dtype=DT[dt], device="cuda")
    v = buf[off:].view(B, T, ld)[:, :, :w]
    v.copy_(t.to(DT[dt]))
    return v


def _within(got, ref, err, dt, what):
    got = _host(got) if isinstance(got, torch.Tensor) else got
    bound = err + HALF[dt] * (np.abs(ref) + err) + 1e-37
    bad = np.abs(got - ref) > bound
    worst = np.max(np.abs(got - ref) / bound) if got.size else 0.0
    _say(f"  {what}: largest error {worst:.3f} of its bound")
    assert np.isfinite(got).all() and not bad.any(), (what, worst, np.argwhere(bad)[:3])


LN = [
    # dt, param, B, T, d, row padding, start offset
    ("f32", "f32", 1, 1, 1, 0, 0), ("bf16", "bf16", 2, 3, 7, 1, 1), ("f32", "f32", 3, 5, 63, 2, 1),
    ("bf16", "f32", 4, 17, 512, 0, 0), ("bf16", "bf16", 2, 40, 513, 0, 0),
    ("f32", "f32", 2, 33, 768, 0, 0), ("bf16", "f32", 2, 64, 1025, 3, 1),
    ("f32", "f32", 1, 300, 2047, 0, 0), ("bf16", "bf16", 1, 19, 2049, 0, 0),
    ("f32", "f32", 2, 9, 4100, 1, 0), ("bf16", "f32", 1, 20, 8200, 0, 0),
    ("f32", "f32", 1, 3, 16391, 0, 0), ("bf16", "bf16", 1, 2, 32768, 0, 0),
    ("bf16", "f32", 1, 5000, 96, 0, 0), ("f32", "f32", 1100, 2, 24, 0, 0),
]


@pytest.mark.parametrize("dt,pdt,B,T,d,pad,off", LN)
def test_layernorm(dp, dt, pdt, B, T, d, pad, off):
    _say(f"layernorm {dt}/{pdt} B={B} T={T} d={d} pad={pad} off={off}")
    x = _rows_of(_normal(1, B, T, d) * 2 + _normal(2, B, T, 1), dt, d + pad, off)
    gy = _rows_of(_normal(3, B, T, d) * 0.01, dt, d + pad, off)
    gain = (1 + 0.3 * _normal(4, d)).to(DT[pdt]).cuda()
    bias = _normal(5, d).to(DT[pdt]).cuda()
    y = _rows_of(torch.zeros(B, T, d), dt, d + pad, off)
    mean, rstd = torch.empty(B, T, device="cuda"), torch.empty(B, T, device="cuda")
    dp.dp_layernorm_forward(x, gain, bias, y, mean=mean, rstd=rstd)
    xs, ws, bs = _host(x), _host(gain), _host(bias)
    ey, em, er = F.layernorm_error(xs, ws, bs, 1e-5)
    ry, rm, rr = F.layernorm(xs, ws, bs, 1e-5)
    _within(y, ry, ey, dt, "y")
    _within(mean, rm, em, "f32", "mean")
    _within(rstd, rr, er, "f32", "rstd")
    # Backward from the statistics that the forward pass wrote.
    dx = _rows_of(torch.zeros(B, T, d), dt, d + pad, off)
    dgain, dbias = (torch.full((B, d), float("nan"), device="cuda") for _ in range(2))
    norm2 = torch.full((B,), float("nan"), device="cuda")
    dp.dp_layernorm_backward(gy, x, gain, mean, rstd, dx, dgain=dgain, dbias=dbias, norm2=norm2)
    args = _host(gy), xs, ws, _host(mean), _host(rstd)
    ref, err = F.layernorm_backward(*args), F.layernorm_backward_error(*args)
    _within(dx, ref["dx"], err["dx"], dt, "dx")
    for k, t in (("dgain", dgain), ("dbias", dbias), ("norm2", norm2)):
        _within(t, ref[k], err[k], "f32", k)
    # What lies between the rows is as it was.
    for t in (y, dx):
        base = t._base if t._base is not None else t
        rest = base.flatten()
        assert int((rest == 7).sum()) >= off + B * T * pad
    # The same results without some of the outputs, added onto others, and in place.
    g2, n2 = torch.empty_like(dgain), norm2.clone()
    dp.dp_layernorm_backward(gy, x, gain, mean, rstd, None, dgain=g2, norm2=n2, accumulate=True)
    assert torch.equal(g2, dgain)
    want = _host(norm2) + (_host(dgain) ** 2).sum(1)
    np.testing.assert_allclose(_host(n2), want, rtol=(d / 8 + 80) * 2.0 ** -24)
    d2 = gy.clone() if pad == 0 and off == 0 else _rows_of(gy.cpu().float(), dt, d + pad, off)
    dp.dp_layernorm_backward(d2, x, gain, mean, rstd, d2)
    assert torch.equal(d2, dx)
    acc = _rows_of(_normal(6, B, T, d), dt, d + pad, off)
    prior = _host(acc)
    dp.dp_layernorm_backward(gy, x, gain, mean, rstd, acc, accumulate_dx=True)
    _within(acc, ref["dx"] + prior, err["dx"] + F.U * np.abs(ref["dx"] + prior), dt, "dx added")


def test_layernorm_without_parameters_and_in_place(dp):
    x = _normal(1, 2, 9, 40).cuda()
    want, _, _ = F.layernorm(_host(x), 1.0, 0.0, 1e-3)
    err, _, _ = F.layernorm_error(_host(x), 1.0, 0.0, 1e-3)
    dp.dp_layernorm_forward(x, None, None, x, eps=1e-3)
    _within(x, want, err, "f32", "y in place")


def test_layernorm_constant_rows_and_nan_rows(dp):
    """A constant row has xhat = 0; a row with NaN spoils that row alone."""
    x = torch.full((1, 4, 100), 3.0, device="cuda")
    x[0, 1] = _normal(1, 100).cuda()
    x[0, 2, 5] = float("nan")
    y = torch.empty_like(x)
    dp.dp_layernorm_forward(x, None, torch.ones(100, device="cuda"), y)
    assert torch.equal(y[0, 0], torch.ones(100, device="cuda")) and torch.equal(y[0, 3], y[0, 0])
    assert torch.isnan(y[0, 2]).all() and torch.isfinite(y[0, 1]).all()


def test_layernorm_matches_the_vector_gradients(dp):
    """dgain and dbias are what dp_vector_grads_grouped makes of xhat and gy."""
    x, gy = _normal(1, 6, 50, 96).cuda(), _normal(2, 6, 50, 96).cuda()
    mean, rstd, xhat = torch.empty(6, 50, device="cuda"), torch.empty(6, 50, device="cuda"), torch.empty_like(x)
    dp.dp_layernorm_forward(x, None, None, xhat, mean=mean, rstd=rstd)
    a = [torch.empty(6, 96, device="cuda") for _ in range(4)]
    n = [torch.empty(6, device="cuda") for _ in range(2)]
    dp.dp_layernorm_backward(gy, x, None, mean, rstd, None, dgain=a[0], dbias=a[1], norm2=n[0])
    dp.dp_vector_grads_grouped([(xhat, gy), (None, gy)], a[2:], norm2=n[1])
    tol = 2 * (50 + 24) * F.U * _host((gy * xhat).abs().sum(1) + gy.abs().sum(1)).max()
    for p, q in ((a[0], a[2]), (a[1], a[3])):
        assert np.abs(_host(p) - _host(q)).max() <= tol
    np.testing.assert_allclose(_host(n[0]), _host(n[1]), rtol=1e-5)


def _targets(B, T, V, seed=9):
    y = torch.randint(0, V, (B, T), generator=torch.Generator().manual_seed(seed), dtype=torch.int32)
    y.view(-1)[::5] = -1
    if B * T > 3:
        y.view(-1)[3] = V      # outside as well
    return y


LOSS = [
    # dt, B, T, V, row padding, start offset
    ("f32", 1, 1, 1, 0, 0), ("f32", 2, 3, 2, 1, 1), ("bf16", 3, 4, 7, 0, 1), ("f32", 2, 6, 511, 0, 0),
    ("bf16", 2, 5, 513, 7, 3), ("f32", 3, 5, 2048, 0, 0), ("bf16", 1, 7, 2051, 0, 0),
    ("f32", 2, 4, 8193, 0, 1), ("bf16", 2, 6, 32768, 0, 0), ("f32", 1, 6, 40001, 0, 0),
    ("bf16", 2, 10, 50257, 0, 0), ("f32", 1, 6, 50257, 47, 0), ("bf16", 1, 6, 65537, 0, 0),
    ("f32", 1, 6, 131075, 1, 0), ("bf16", 40, 60, 96, 0, 0),
    ("bf16", 1, 6, 60001, 0, 1), ("bf16", 1, 6, 131072, 0, 0), ("bf16", 1, 6, 150001, 2, 0),
    ("bf16", 1, 6, 196609, 0, 0), ("f32", 1, 6, 60001, 0, 0), ("f32", 1, 6, 98304, 8, 0),
]


@pytest.mark.parametrize("dt,B,T,V,pad,off", LOSS)
def test_logprobs_and_cross_entropy(dp, dt, B, T, V, pad, off):
    _say(f"losses {dt} B={B} T={T} V={V} pad={pad} off={off}")
    z = _rows_of(3 * _normal(1, B, T, V), dt, V + pad, off)
    y = _targets(B, T, V)
    w = torch.rand(B, T, generator=torch.Generator().manual_seed(2))
    w.view(-1)[1::7] = 0.0
    yd, wd = y.cuda(), w.cuda()
    logp, lse = (torch.full((B, T), float("nan"), device="cuda") for _ in range(2))
    dp.dp_token_logprobs(z, yd, logp, lse=lse)
    zs, ys = _host(z), y.numpy()
    rp, rl, es = F.token_logprobs(zs, ys)
    _within(logp, rp, es, "f32", "logp")
    _within(lse, rl, es, "f32", "lse")
    g = _rows_of(torch.zeros(B, T, V), dt, V + pad, off)
    l2 = torch.full((B, T), float("nan"), device="cuda")
    dp.dp_cross_entropy(z, yd, wd, l2, g)
    _, rg, eg = F.cross_entropy(zs, ys, w.double().numpy())
    _within(l2, rp, es, "f32", "logp")
    _within(g, rg, eg, dt, "Gz")
    if pad or off:
        assert int((g._base == 7).sum()) == off + B * T * pad
    dp.dp_cross_entropy(z, yd, wd, None, z)   # in place
    assert torch.equal(z, g)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("V", [1, 5, 8, 13, 515, 8200])
def test_every_alignment_of_logits_and_gradients(dp, dt, V):
    """Rows that start anywhere in a 16-byte unit, and gradients that start elsewhere in theirs."""
    B, T, step = 2, 4, 8 if dt == "bf16" else 4
    x, y = 3 * _normal(V, B, T, V), _targets(B, T, V)
    y[1, 3] = V - 1
    w, yd = torch.ones(B, T, device="cuda"), y.cuda()
    ref = None
    for off in range(step):
        z = _rows_of(x, dt, V + 1 + off, off)
        g = _rows_of(torch.zeros(B, T, V), dt, V + 3, (3 * off + 1) % step)
        logp = torch.empty(B, T, device="cuda")
        dp.dp_token_logprobs(z, yd, logp)
        if ref is None:
            zs = _host(z)
            ref = F.token_logprobs(zs, y.numpy()), F.cross_entropy(zs, y.numpy(), np.ones((B, T)))
        _within(logp, ref[0][0], ref[0][2], "f32", f"offset {off}: logp")
        dp.dp_cross_entropy(z, yd, w, logp, g)
        _within(logp, ref[0][0], ref[0][2], "f32", "logp")
        _within(g, ref[1][1], ref[1][2], dt, "Gz")
        assert int((g._base == 7).sum()) == (3 * off + 1) % step + B * T * 3
        h = _rows_of(torch.zeros(B, T, V), dt, V + 2, off)
        loss = torch.empty(B, device="cuda")
        dp.dp_preference_loss(z, yd, 2, None, 0.3, loss, Gz=h)
        want = F.preference(zs, y.numpy(), 2, np.zeros((B, T)), float(np.float32(0.3)), 0.0)
        _within(h, want["Gz"], want["Gz_error"], dt, "preference Gz")
        assert int((h._base == 7).sum()) == off + B * T * 2
        dp.dp_cross_entropy(z, yd, w, None, z)
        assert int((z._base == 7).sum()) == off + B * T * (1 + off)
        assert torch.equal(z, g)


PAIRS = [("f32", 1, 2, 3, 1, 0), ("bf16", 3, 7, 50, 3, 1), ("f32", 2, 9, 2050, 4, 0),
         ("bf16", 2, 6, 50257, 3, 47), ("f32", 2, 5, 300, 0, 0), ("f32", 2, 5, 300, 5, 2),
         ("bf16", 5, 300, 129, 150, 0)]


@pytest.mark.parametrize("dt,B,T,V,split,pad", PAIRS)
def test_preference_loss(dp, dt, B, T, V, split, pad):
    _say(f"preference {dt} B={B} T={T} V={V} split={split}")
    z = _rows_of(2 * _normal(1, B, T, V), dt, V + pad)
    y = _targets(B, T, V)
    ref = _normal(2, B, T) * 0.5 - float(np.log(V))
    beta, eps = 0.4, 0.1
    loss, rew = torch.empty(B, device="cuda"), torch.empty(B, 2, device="cuda")
    logp = torch.empty(B, T, device="cuda")
    g = _rows_of(torch.zeros(B, T, V), dt, V + pad)
    dp.dp_preference_loss(z, y.cuda(), split, ref.cuda(), beta, loss, rewards=rew, logp=logp, Gz=g,
                          label_smoothing=eps)
    b32, e32 = float(np.float32(beta)), float(np.float32(eps))
    want = F.preference(_host(z), y.numpy(), split, ref.double().numpy(), b32, e32)
    _within(logp, want["logp"], want["logp_error"], "f32", "logp")
    _within(loss, want["loss"], want["loss_error"], "f32", "loss")
    _within(rew, want["rewards"], want["rewards_error"], "f32", "rewards")
    _within(g, want["Gz"], want["Gz_error"], dt, "Gz")
    alone = torch.empty(B, device="cuda")
    dp.dp_preference_loss(z, y.cuda(), split, ref.cuda(), beta, alone, label_smoothing=eps)
    assert torch.equal(alone, loss)
    dp.dp_preference_loss(z, y.cuda(), split, ref.cuda(), beta, alone, Gz=z, label_smoothing=eps)
    assert torch.equal(z, g)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("V", [60, 3000, 50257, 70000])
def test_masked_and_extreme_logits(dp, dt, V):
    """-inf and the type's lowest value mask; a row without any logit; NaN and +inf in rows
    that are not scored or have weight 0, and in one that is."""
    _say(f"masked logits {dt} V={V}")
    inf, low = float("inf"), float(torch.finfo(DT[dt]).min)
    z = _normal(1, 1, 9, V)
    z[0, 0, 1:] = -inf                  # one allowed token, the target
    z[0, 1, :V // 2] = -inf
    z[0, 2] = -inf                      # nothing allowed
    z[0, 3] = low                       # all of the lowest value: uniform
    z[0, 4, 2:] = low
    z[0, 5] = float("nan")              # not scored
    z[0, 6, 4] = inf                    # weight 0
    z[0, 7, 9] = float("nan")
    z[0, 8, 3:] = -inf                  # the target is masked
    z = z.to(DT[dt])
    y = torch.tensor([[0, V - 1, 5, 7, 1, -1, 4, 2, V - 1]], dtype=torch.int32)
    w = torch.ones(1, 9)
    w[0, 6] = 0
    zd, g = z.cuda(), torch.full((1, 9, V), 5.0, dtype=DT[dt], device="cuda")
    logp = torch.empty(1, 9, device="cuda")
    dp.dp_cross_entropy(zd, y.cuda(), w.cuda(), logp, g)
    lse = torch.empty(1, 9, device="cuda")
    l2 = torch.empty_like(logp)
    dp.dp_token_logprobs(zd, y.cuda(), l2, lse=lse)
    # Both are within their bound of the same value, so within twice that of one another.
    _, _, es = F.token_logprobs(z.double().numpy()[:, [0, 1, 3, 4]], y.numpy()[:, [0, 1, 3, 4]])
    a, b = _host(logp)[0], _host(l2)[0]
    assert (np.isnan(a) == np.isnan(b)).all() and (np.isinf(a) == np.isinf(b)).all()
    for k, r in enumerate((0, 1, 3, 4)):
        assert abs(a[r] - b[r]) <= 2 * (es[0, k] + F.U * abs(a[r])), r
    lp, gz = _host(logp)[0], _host(g)[0]
    assert lp[0] == 0 and not gz[0].any()
    assert lp[2] == -np.inf and float(lse[0, 2]) == -np.inf and not gz[2].any()
    assert lp[5] == 0 and not gz[5].any()
    assert not gz[6].any()
    assert np.isnan(lp[7]) and np.isnan(gz[7]).all()
    assert lp[8] == -np.inf
    for r in (1, 3, 4, 8):
        zs = z[0, r].double().numpy()
        p = np.exp(zs - zs.max())
        p /= p.sum()
        p[y[0, r]] -= 1
        gap = np.where(np.isfinite(zs), zs.max() - zs, 0.0).clip(max=200)
        assert (np.abs(gz[r] - p) <= HALF[dt] * np.abs(p) + (4 * gap + 200) * F.U * np.abs(p + (np.arange(V) == int(y[0, r]))) + 1e-37).all(), r


def test_preference_of_extreme_margins(dp):
    """A pair whose margin is huge has loss 0 or the margin itself, with no NaN."""
    z = torch.zeros(2, 2, 4, device="cuda")
    z[0, 0, 0], z[0, 1, 1] = 500.0, -800.0     # chosen certain, rejected impossible
    z[1, 0, 0], z[1, 1, 1] = -800.0, 500.0
    y = torch.tensor([[0, 1], [0, 1]], dtype=torch.int32, device="cuda")
    loss, g = torch.empty(2, device="cuda"), torch.empty_like(z)
    dp.dp_preference_loss(z, y, 1, None, 2.0, loss, Gz=g)
    assert torch.isfinite(g).all() and torch.isfinite(loss).all()
    assert float(loss[0]) == 0.0 and float(loss[1]) > 1000 and not g[0].any()


def test_logits_past_four_gib(dp):
    """Rows whose offsets pass 32 bits."""
    V, T = 50304, 45000
    z = torch.zeros(1, T, V, dtype=torch.bfloat16, device="cuda")
    z[0, -1, 77] = 4.0
    y = torch.full((1, T), -1, dtype=torch.int32, device="cuda")
    y[0, -1] = 77
    w = torch.ones(1, T, device="cuda")
    logp = torch.empty(1, T, device="cuda")
    dp.dp_cross_entropy(z, y, w, logp, z)
    p = np.exp(4.0) / (np.exp(4.0) + V - 1)
    assert abs(float(logp[0, -1]) - np.log(p)) < 1e-5
    row = _host(z[0, -1])
    assert abs(row[77] - (p - 1)) <= 2.0 ** -8 and abs(row[5] - p / np.exp(4.0)) <= 2.0 ** -7 * p
    assert int(torch.count_nonzero(z[0, :-1])) == 0


def test_captured_and_replayed(dp):
    """Forward, losses and backward in a graph: replays on new inputs equal eager calls."""
    B, T, d, V = 2, 37, 96, 700
    x = torch.empty(B, T, d, device="cuda")
    z, y = torch.empty(B, T, V, device="cuda"), _targets(B, T, V).cuda()
    out = dict(y=torch.empty_like(x), dx=torch.empty_like(x), mean=torch.empty(B, T, device="cuda"),
               rstd=torch.empty(B, T, device="cuda"), dgain=torch.empty(B, d, device="cuda"),
               dbias=torch.empty(B, d, device="cuda"), norm2=torch.empty(B, device="cuda"),
               loss=torch.empty(B, device="cuda"), g=torch.empty_like(z))

    def call(o):
        dp.dp_layernorm_forward(x, None, None, o["y"], mean=o["mean"], rstd=o["rstd"])
        dp.dp_layernorm_backward(o["y"], x, None, o["mean"], o["rstd"], o["dx"], dgain=o["dgain"],
                                 dbias=o["dbias"], norm2=o["norm2"])
        dp.dp_preference_loss(z, y, 20, None, 0.3, o["loss"], Gz=o["g"])

    def fill(k):
        x.copy_(_normal(k, B, T, d))
        z.copy_(_normal(k + 50, B, T, V))

    fill(0)
    call(out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out)
    for k in range(1, 4):
        fill(k)
        graph.replay()
        torch.cuda.synchronize()
        eager = {n: torch.empty_like(t) for n, t in out.items()}
        call(eager)
        torch.cuda.synchronize()
        for n in out:
            assert torch.equal(out[n], eager[n]), n


def test_on_another_stream(dp):
    """A call on a stream waits for that stream's work and takes its scratch from there."""
    s = torch.cuda.Stream()
    x, gy = _normal(1, 1, 4000, 64).cuda(), _normal(2, 1, 4000, 64).cuda()
    mean, rstd, y = torch.empty(1, 4000, device="cuda"), torch.empty(1, 4000, device="cuda"), torch.empty_like(x)
    g = [torch.empty(1, 64, device="cuda") for _ in range(2)]
    torch.cuda.synchronize()
    dp.dp_layernorm_forward(x, None, None, y, mean=mean, rstd=rstd, stream=s)
    dp.dp_layernorm_backward(gy, x, None, mean, rstd, None, dgain=g[0], stream=s)
    s.synchronize()
    dp.dp_layernorm_backward(gy, x, None, mean, rstd, None, dgain=g[1])
    torch.cuda.synchronize()
    assert torch.equal(g[0], g[1])


def test_more_rows_than_one_launch_takes(dp):
    """70 million rows of two logits, and 8.5 million examples of one token."""
    n = 70_000_000
    z = torch.zeros(1, n, 2, dtype=torch.bfloat16, device="cuda")
    at = [0, 8_388_607, 8_388_608, n // 2, n - 1]
    for k, r in enumerate(at):
        z[0, r, 1] = 1.0 + k
    y = torch.ones(1, n, dtype=torch.int32, device="cuda")
    w = torch.ones(1, n, device="cuda")
    logp, lse = torch.full((1, n), 9.0, device="cuda"), torch.full((1, n), 9.0, device="cuda")
    dp.dp_token_logprobs(z, y, logp, lse=lse)
    want = -np.log1p(np.exp(-(1.0 + np.arange(len(at)))))
    assert np.abs(_host(logp[0, at]) - want).max() < 1e-6
    assert abs(float(logp.double().sum()) - (want.sum() - (n - len(at)) * np.log(2.0))) < 1e-6 * n
    dp.dp_cross_entropy(z, y, w, logp, z)
    assert np.abs(_host(z[0, at, 1]) - (np.exp(want) - 1)).max() <= 2.0 ** -8
    assert int((z[0, :, 1] == -0.5).sum()) == n - len(at) and int((z[0, :, 0] == 0.5).sum()) == n - len(at)
    del z, y, w, logp, lse
    B, d = 8_500_000, 8
    x = torch.arange(d, device="cuda").float().expand(B, 1, d).contiguous()
    gy = torch.zeros(B, 1, d, device="cuda")
    gy[:, 0, 3] = torch.arange(B, device="cuda") % 7 + 1.0
    mean, rstd = torch.full((B, 1), 3.5, device="cuda"), torch.full((B, 1), 0.5, device="cuda")
    dbias, n2 = torch.full((B, d), 9.0, device="cuda"), torch.full((B,), 9.0, device="cuda")
    dp.dp_layernorm_backward(gy, x, None, mean, rstd, None, dbias=dbias, norm2=n2)
    assert torch.equal(dbias, gy[:, 0]) and torch.equal(n2, gy[:, 0, 3] ** 2)
