"""Orthogonalised updates of matrices whose signal outweighs their noise, as momenta do.

A direction with a small singular value grows by a = 3.4445 a step, so that a rounding of X
after step k, which falls on all directions alike, is a^(steps - k) times as large in the
result: 485 times for the first one of five. Beside a few leading directions there is nothing else
that size to compare it with. The bounds here do not come from the kernels' own operand formats.

fp32 results: the same five steps in 32-bit products (numpy) are the measure; twice their error.
X is held to one bit less than fp32 does, at most (half steps of 2^-23 against 2^-24, an error
of 1.5 times the root mean square), and everything else is rounded alike.

bf16 results: half a step of bf16, 2^-8, as a norm. The result's own rounding is 0.425 x 2^-8 of
it (a uniform error of up to half a step, over a uniform significand). If only the last two
states of X are rounded to 11 bits, 0.425 x 2^-11 each, those grow a^2 and a times: 2.6e-3 of X's
norm, 0.66 x 2^-8. Together 0.78 x 2^-8, and the rest is for the products' other operand, which
is rounded to 11 bits without such a growth, and for singular values between 0.7 and 1.2."""
import numpy as np
import pytest

from tests import step_formulas as F

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

MUON = [tuple(float(np.float32(v)) for v in (3.4445, -4.7750, 2.0315))] * 5


@pytest.fixture(scope="module")
def dp():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_40335_amd.dpghost as d
    d.lib()
    return d


def _momentum(seed, m, n, signal):
    """Rank 8 times `signal` over noise of norm 1 (None: no noise), fp32."""
    g = np.random.default_rng(seed)
    k = min(8, m, n)
    low = (g.standard_normal((m, k)) / np.arange(1, k + 1)) @ g.standard_normal((k, n))
    low /= np.linalg.norm(low)
    if signal is not None:
        noise = g.standard_normal((m, n))
        low = signal * low + noise / np.linalg.norm(noise)
    return low.astype(np.float32)


def _in_32_bits(G):
    """The same steps in 32-bit products."""
    flip = G.shape[0] > G.shape[1]
    X = (G.T if flip else G).astype(np.float64)
    X = (X / (np.sqrt((X * X).sum()) + 1e-7)).astype(np.float32)
    for a, b, c in (np.array(MUON, np.float32)):
        A = X @ X.T
        X = a * X + (b * A + c * (A @ A)) @ X
    return X.T if flip else X


@pytest.mark.parametrize("signal", [0.5, 3, 10, 30, 100, None])
@pytest.mark.parametrize("m,n", [(512, 1024), (300, 128), (96, 200), (50, 80), (1500, 700)])
def test_signal_over_noise(dp, m, n, signal):
    G = _momentum(7, m, n, signal)
    ref = F.newton_schulz(G.astype(np.float64), MUON, float(np.float32(1e-7)))
    size = np.linalg.norm(ref)
    plain = np.linalg.norm(_in_32_bits(G) - ref) / size
    g = torch.from_numpy(G).cuda()
    for dt, bound in ((torch.float32, 2 * plain + 2.0 ** -24), (torch.bfloat16, 2.0 ** -8)):
        out = torch.empty(m, n, dtype=dt, device="cuda")
        dp.dp_orthogonalize_grouped([g], [out])
        err = np.linalg.norm(out.cpu().double().numpy() - ref) / size
        print(f"  {m}x{n} signal {signal} {dt}: {err:.2e}, allowed {bound:.2e} (32-bit products {plain:.2e})",
              flush=True)
        assert err <= bound, (m, n, signal, dt)


@pytest.mark.parametrize("rank", [1, 2, 32])
@pytest.mark.parametrize("m,n", [(512, 1024), (96, 200), (700, 130)])
def test_low_ranks_without_noise(dp, m, n, rank):
    g = np.random.default_rng(rank)
    G = (g.standard_normal((m, rank)) @ g.standard_normal((rank, n))).astype(np.float32)
    ref = F.newton_schulz(G.astype(np.float64), MUON, float(np.float32(1e-7)))
    size, plain = np.linalg.norm(ref), np.linalg.norm(_in_32_bits(G) - ref)
    for dt, bound in ((torch.float32, 2 * plain + 2.0 ** -24 * size), (torch.bfloat16, 2.0 ** -8 * size)):
        out = torch.empty(m, n, dtype=dt, device="cuda")
        dp.dp_orthogonalize_grouped([torch.from_numpy(G).cuda()], [out])
        err = np.linalg.norm(out.cpu().double().numpy() - ref)
        print(f"  {m}x{n} rank {rank} {dt}: {err / size:.2e}, allowed {bound / size:.2e}", flush=True)
        assert err <= bound, (m, n, rank, dt)


@pytest.mark.parametrize("noise", [0.0, 0.1])
@pytest.mark.parametrize("m,n,rank", [(512, 1024, 32), (700, 1500, 128), (96, 200, 8), (60, 80, 32),
                                      (768, 768, 512), (130, 60, 3)])
def test_fp32_results_match_32_bit_products(dp, m, n, rank, noise):
    """Beside the leading directions 32-bit products round three times a step (a X, the product
    and their sum, each 2^-24 at most), the kernels once to 22 bits: with x = x0 + x1, x1's
    half step is 2^-23 or, for a smaller x1, less, 0.76 of it as a root mean square. 0.76 x 2 / 3 ** 0.5 =
    0.87 of their error; 1.25 leaves room for another sample."""
    g = np.random.default_rng(rank)
    G = g.standard_normal((m, rank)) @ g.standard_normal((rank, n))
    N = g.standard_normal((m, n))
    G = (G / np.linalg.norm(G) + noise * N / np.linalg.norm(N)).astype(np.float32)
    ref = F.newton_schulz(G.astype(np.float64), MUON, float(np.float32(1e-7)))
    plain = np.linalg.norm(_in_32_bits(G) - ref)
    out = torch.empty(m, n, device="cuda")
    dp.dp_orthogonalize_grouped([torch.from_numpy(G).cuda()], [out])
    err = np.linalg.norm(out.cpu().double().numpy() - ref)
    print(f"  {m}x{n} rank {rank} noise {noise}: {err / plain:.2f} of 32-bit products' error", flush=True)
    assert err <= 1.25 * plain


@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
def test_every_matrix_of_a_large_group(dp, out):
    """48 and more matrices of GPT-2's shapes and ragged ones, each against 64 bits (on the GPU)."""
    shapes = [(768, 2304), (768, 768), (2000, 650), (650, 2000), (130, 1290)] * 12
    gen = torch.Generator(device="cuda").manual_seed(5)
    grads = []
    for k, (m, n) in enumerate(shapes):
        low = torch.randn(m, 4, device="cuda", generator=gen) @ torch.randn(4, n, device="cuda", generator=gen)
        noise = torch.randn(m, n, device="cuda", generator=gen)
        grads.append((0.5, 5.0, 40.0)[k % 3] * low / low.norm() + noise / noise.norm())
    outs = [torch.empty(m, n, device="cuda", dtype=out) for m, n in shapes]
    dp.dp_orthogonalize_grouped(grads, outs)
    for k, (g, o) in enumerate(zip(grads, outs)):
        x = g.double()
        x = x.t().contiguous() if x.shape[0] > x.shape[1] else x
        x = x / (x.norm() + 1e-7)
        y = x.float()
        for a, b, c in MUON:
            q = x @ x.t()
            x = a * x + (b * q + c * (q @ q)) @ x
            q = y @ y.t()
            y = a * y + (b * q + c * (q @ q)) @ y
        plain = float((y.double() - x).norm() / x.norm())
        x = x.t() if g.shape[0] > g.shape[1] else x
        err = float((o.double() - x).norm() / x.norm())
        assert err <= (2.0 ** -8 if out == torch.bfloat16 else 2 * plain + 2.0 ** -24), (k, shapes[k], err, plain)
