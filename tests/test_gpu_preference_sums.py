"""A preference loss's rewards are small differences of long sums: an answer's log-probabilities
against a reference model that nearly agrees. What is off in the same way in every row adds up.

The logarithm of a row's sum may be off by 2e-8. With log2 e's missing digits put back, an exponential
of d is off by the rounding of d log2 e, |d| 2^-24 at most, and by its instruction's last bit; both
differ from value to value of d, and a row's sum weighs at least some 500 of those: a root mean square of
about 4 x 6e-8 x 0.6 / 500^0.5 = 6e-9 (d of 4 on average). Three times that is allowed for every
row, in the same direction. Plain fp32 sums of these very logits (on the CPU, in the kernels' order) are
off by 6e-8 to 9e-8 a row, 2.8e-8 to 5e-8 of it in the same direction, and miss it."""
import numpy as np
import pytest

from tests import step_formulas as F

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

A_ROW = 2e-8


@pytest.fixture(scope="module")
def dp():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_40335_amd.dpghost as d
    d.lib()
    return d


# V on both sides of the kernels' widths of a row: one wave, four, four again with many rows, sixteen.
@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("B,T,V,spread", [(3, 700, 2000, 2.0), (2, 600, 8001, 3.0), (4, 600, 12289, 2.0),
                                          (2, 500, 20011, 3.0)])
def test_rewards_of_long_answers(dp, dt, B, T, V, spread):
    g = torch.Generator(device="cuda").manual_seed(V)
    z = (spread * torch.randn(B, T, V, device="cuda", generator=g)).to(dt)
    y = torch.randint(0, V, (B, T), device="cuda", generator=g, dtype=torch.int32)
    y[:, :5] = -1
    kept = y >= 0
    exact = torch.stack([torch.log_softmax(z[b].double(), 1).gather(1, y[b].long().clamp(min=0)[:, None])[:, 0]
                         for b in range(B)])
    ref = torch.where(kept, exact + 0.01 * torch.randn(B, T, device="cuda", generator=g), 0.0).float()
    beta, split = 0.5, T // 2 + 3
    loss, rewards = torch.empty(B, device="cuda"), torch.empty(B, 2, device="cuda")
    dp.dp_preference_loss(z, y, split, ref, beta, loss, rewards=rewards)
    ratio = torch.where(kept, exact - ref.double(), 0.0)
    want = beta * torch.stack([ratio[:, :split].sum(1), ratio[:, split:].sum(1)], 1)
    n = torch.stack([kept[:, :split].sum(1), kept[:, split:].sum(1)], 1)
    want, n, got = want.cpu().numpy(), n.cpu().numpy(), rewards.cpu().double().numpy()
    off = np.abs(got - want) - F.U * np.abs(want)
    print(f"  {dt} {B}x{T}x{V}: {np.max(off / (beta * n)):.2e} a row, allowed {A_ROW:.0e}", flush=True)
    assert (off <= beta * A_ROW * n).all()
    m = want[:, 0] - want[:, 1]
    bound = 2 * beta * A_ROW * n.max() + F.U * np.logaddexp(0, -m)      # |d loss / d m| <= 1
    assert (np.abs(loss.cpu().double().numpy() - np.logaddexp(0, -m)) <= bound).all()
