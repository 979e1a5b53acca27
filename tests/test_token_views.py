"""Views of token-major tensors as operands: what is one row stride, and what is not.

The last token of every prompt, Z[:, -1:, :], is [B, 1, w] with rows T * ld apart: one row
stride. All but the last, Z[:, :-1, :], has no single one. The norms and sums, whose kernels may
read a row, the last one too, up to its stride, refuse both."""
import pytest

from paper_2609_40335_amd import dpghost as D

torch = pytest.importorskip("torch")


def helper(t):
    return D._tokens(t, "Z")[0::2]


def test_row_stride_of_views():
    z = torch.zeros(3, 5, 8)
    buf = torch.zeros(3, 5, 16)
    for view, row, ld in ((z, 0, 8), (z[:, -1:, :], 4, 40), (buf[:, 2:3, :8], 2, 80), (buf[:, :, :8], 0, 16),
                          (z[:1], 0, 8), (z[1:2, 1:, :], 6, 8), (z[:1, :1, :], 0, 8), (z[::2, :1], 0, 80)):
        p, got = helper(view)
        base = buf if view._base is buf else z
        assert got == ld and p == base.data_ptr() + row * base.shape[2] * 4, (view.shape, view.stride())
    for view in (z[:, :-1, :], z[:, ::2, :], z[:, :, ::2], z.transpose(0, 1)):
        with pytest.raises(D.DPError, match="uniformly"):
            helper(view)
    with pytest.raises(D.DPError, match="uniformly"):
        D._rows(z[:, -1:, :], "Gz")


def test_flattened_tokens_of_one_step():
    """What works for every B and T: the same rows as [1, B, w]."""
    z = torch.zeros(3, 5, 8)
    a, b = D._tokens(z[:, -1:, :], "Z"), D._tokens(z[:, -1, :].unsqueeze(0), "Z")
    assert a[0] == b[0] and a[2] == b[2] == 40


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
def test_last_token_of_every_prompt(dt):
    from paper_2609_40335_amd import dpghost as dp
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    g = torch.Generator(device="cuda").manual_seed(1)
    z = torch.randn(4, 6, 301, device="cuda", generator=g).to(dt)
    y = torch.tensor([[0], [300], [-1], [7]], dtype=torch.int32, device="cuda")
    w, last = torch.ones(4, 1, device="cuda"), z[:, -1:, :]
    a, b = torch.empty(4, 1, device="cuda"), torch.empty(4, 1, device="cuda")
    dp.dp_token_logprobs(last, y, a)
    dp.dp_token_logprobs(last.contiguous(), y, b)
    assert torch.equal(a, b) and float(a[2]) == 0 and bool((a[[0, 1, 3]] < 0).all())
    out, want = torch.full_like(z, 5), torch.empty_like(last.contiguous())
    dp.dp_cross_entropy(last, y, w, a, out[:, -1:, :])
    dp.dp_cross_entropy(last.contiguous(), y, w, b, want)
    assert torch.equal(out[:, -1:, :], want) and bool((out[:, :-1] == 5).all()) and torch.equal(a, b)
    h = torch.randn(4, 6, 40, device="cuda", generator=g).to(dt)
    x, mean, rstd = torch.full_like(h, 5), torch.empty(4, 1, device="cuda"), torch.empty(4, 1, device="cuda")
    dp.dp_layernorm_forward(h[:, -1:, :], None, None, x[:, -1:, :], mean=mean, rstd=rstd)
    c = torch.empty(4, 1, 40, device="cuda", dtype=dt)
    dp.dp_layernorm_forward(h[:, -1:, :].contiguous(), None, None, c)
    assert torch.equal(x[:, -1:, :], c) and bool((x[:, :-1] == 5).all())
