"""LayerNorm, the head's losses and the orthogonalised update in 64 bits (numpy),
with the error each is allowed when computed in 32.

U is half a step of fp32: one rounding is off by at most U relative to its result.
A sum of n terms in any order is off by at most about (depth) U sum |terms|, with
depth the longest chain of additions a term passes through."""
import numpy as np

U = 2.0 ** -24
# Longest chain of additions of a row's sum on the GPU: 32 of a lane's own
# elements, 6 between lanes, 16 between waves; rounded up.
ROW_DEPTH = 64


def layernorm(x, gain, bias, eps):
    mean = x.mean(-1)
    c = x - mean[..., None]
    rstd = 1.0 / np.sqrt((c * c).mean(-1) + eps)
    return c * rstd[..., None] * gain + bias, mean, rstd


def layernorm_error(x, gain, bias, eps):
    """(y, mean, rstd) bounds: the mean is off by ROW_DEPTH U max|x|, and so is every
    x - mean; rstd is off by ROW_DEPTH U relative from the sum of squares and by the mean's
    error entering squared differences (2 delta |c| / var, at most 2 delta rstd)."""
    y, mean, rstd = layernorm(x, gain, bias, eps)
    top = np.abs(x).max(-1)
    delta = (ROW_DEPTH + 2) * U * top
    rel = (ROW_DEPTH + 8) * U + 2 * delta * rstd
    xhat = np.abs(x - mean[..., None]) * rstd[..., None]
    ey = np.abs(gain) * (delta * rstd)[..., None] + (rel[..., None] + 4 * U) * xhat * np.abs(gain) \
        + 2 * U * (np.abs(bias) + np.abs(y))
    return ey, delta, rel * rstd


def layernorm_backward(gy, x, gain, mean, rstd):
    xhat = (x - mean[..., None]) * rstd[..., None]
    g = gy * gain
    d = x.shape[-1]
    dx = rstd[..., None] * (g - g.sum(-1, keepdims=True) / d
                            - xhat * (g * xhat).sum(-1, keepdims=True) / d)
    dgain, dbias = (gy * xhat).sum(1), gy.sum(1)
    return {"dx": dx, "dgain": dgain, "dbias": dbias,
            "norm2": (dgain ** 2).sum(-1) + (dbias ** 2).sum(-1)}


def layernorm_backward_error(gy, x, gain, mean, rstd):
    """xhat is off by 3 U relative (a subtraction and a product from the given statistics,
    the subtraction exact to U of its result). Token sums pass through at most T + 16 additions."""
    T, d = x.shape[1], x.shape[2]
    xhat = np.abs(x - mean[..., None]) * rstd[..., None]
    g = np.abs(gy * gain)
    m1, m2 = g.sum(-1, keepdims=True) / d, (g * xhat).sum(-1, keepdims=True) / d
    e = (ROW_DEPTH + 8) * U
    dx = rstd[..., None] * (8 * U * g + e * m1 + (e + 8 * U) * xhat * m2)
    sg, sb = (np.abs(gy) * xhat).sum(1), np.abs(gy).sum(1)
    eg, eb = (T + 24) * U * sg, (T + 16) * U * sb
    b = layernorm_backward(gy, x, gain, mean, rstd)
    n = (2 * np.abs(b["dgain"]) * eg + eg ** 2 + 2 * np.abs(b["dbias"]) * eb + eb ** 2).sum(-1)
    return {"dx": dx, "dgain": eg, "dbias": eb,
            "norm2": n + (d / 8 + ROW_DEPTH) * U * b["norm2"]}


def row_softmax(z):
    """(lse, p, error of log sum, relative error of every p). exp(z - top) as exp2 of a
    product is off by 2 U |exponent| (two roundings of the exponent) and 4 U of its own;
    the sum passes through ROW_DEPTH + 64 additions and rescalings."""
    with np.errstate(invalid="ignore", divide="ignore"):
        top = z.max(-1, keepdims=True)
        gap = np.where(np.isfinite(z), top - z, 0.0)
        e = np.where(np.isneginf(z), 0.0, np.exp(z - top))
        s = e.sum(-1, keepdims=True)
        p = e / s
        lse = (top + np.log(s))[..., 0]
        es = ((4 * gap + 8) * U * p).sum(-1) + (ROW_DEPTH + 64) * U
    return lse, p, es, (4 * gap + 16) * U + es[..., None]


def token_logprobs(z, y):
    """(logp, lse, error of logp without the last rounding); unscored rows are 0."""
    lse, p, es, ep = row_softmax(z)
    kept = (y >= 0) & (y < z.shape[-1])
    at = np.where(kept, y, 0)[..., None]
    logp = np.where(kept, np.take_along_axis(z, at, -1)[..., 0] - lse, 0.0)
    return logp, np.where(kept, lse, 0.0), np.where(kept, es, 0.0)


def cross_entropy(z, y, w):
    """(logp, Gz, error of Gz before its last rounding)."""
    logp, _, _ = token_logprobs(z, y)
    _, p, _, ep = row_softmax(z)
    V = z.shape[-1]
    kept = (y >= 0) & (y < V) & (w != 0)
    hot = np.arange(V) == np.where(kept, y, -1)[..., None]
    w = np.where(kept, w, 0.0)[..., None]
    with np.errstate(invalid="ignore"):
        g = np.where(kept[..., None], w * (p - hot), 0.0)
        err = np.where(kept[..., None], np.abs(w) * (p * (ep + 4 * U) + 2 * U * np.abs(p - hot)), 0.0)
    return logp, g, err


def sigmoid(m):
    return 1.0 / (1.0 + np.exp(-m))


def preference(z, y, split, ref, beta, eps):
    logp, _, es = token_logprobs(z, y)
    kept = (y >= 0) & (y < z.shape[-1])
    ratio = np.where(kept, logp - ref, 0.0)
    rewards = beta * np.stack([ratio[:, :split].sum(1), ratio[:, split:].sum(1)], 1)
    m = rewards[:, 0] - rewards[:, 1]
    loss = (1 - eps) * np.logaddexp(0, -m) + eps * np.logaddexp(0, m)
    slope = beta * ((1 - eps) * sigmoid(-m) - eps * sigmoid(m))
    side = np.where(np.arange(z.shape[1]) < split, 1.0, -1.0)
    w = slope[:, None] * side
    _, g, err = cross_entropy(z, y, w)
    # A margin is off by beta times the sum of its tokens' errors; sigma' <= 1/4.
    er = beta * np.stack([es[:, :split].sum(1), es[:, split:].sum(1)], 1)
    em = er.sum(1)
    _, p, _, _ = row_softmax(z)
    hot = np.arange(z.shape[-1]) == np.where(kept, y, -1)[..., None]
    err = err + np.where(kept[..., None], (beta * em / 4)[:, None, None] * np.abs(p - hot), 0.0)
    return {"loss": loss, "rewards": rewards, "logp": logp, "Gz": g, "slope": slope,
            "loss_error": em + U * np.abs(loss), "rewards_error": er + U * np.abs(rewards),
            "Gz_error": err, "logp_error": es}


# ---------------------------------------------------------------- orthogonalise
def newton_schulz(G, coef, eps, bits=None, seed=0):
    """X after the steps of coef [(a, b, c), ...], in 64 bits.

    bits: every operand of a product is rounded to that many significant bits, and every
    product's elements are off by 2^-22 of themselves as a root mean square (fp32 sums): a
    sample of what a computation that rounds so comes to."""
    flip = G.shape[0] > G.shape[1]
    X = (G.T if flip else G).astype(np.float64)
    with np.errstate(invalid="ignore"):
        X = X / (np.sqrt((X * X).sum()) + eps)
    rng = np.random.default_rng(seed)

    def q(x):
        if bits is None:
            return x
        m, e = np.frexp(x)
        return np.ldexp(np.round(m * 2.0 ** bits) * 2.0 ** -bits, e)

    def noisy(x):
        # fp32 sums, and half a step of the operand's rounding more, uniform: samples differ.
        return x if bits is None else x * (1 + 2.0 ** -22 * rng.standard_normal(x.shape)
                                           + 2.0 ** -bits * rng.uniform(-0.5, 0.5, x.shape))

    eye = np.eye(X.shape[0])
    X = q(noisy(X))
    for a, b, c in coef:
        A = q(noisy(X @ X.T))
        P = q(noisy(a * eye + b * A + c * (A @ A)))
        X = q(noisy(P @ X))
    return X.T if flip else X


def newton_schulz_error(G, coef, eps, out):
    """(exact result, Frobenius bound, element bound) for fp16 operands of one plane (11
    bits, bf16 results) or two (22 bits, fp32 results): four times the samples' error, as the
    roundings are another sample. The error's size is the root mean square of 32 samples
    where a matrix has few elements: of a single element with an error N(0, s), 4 |sample| falls below
    s in 20 of 100 draws (P(|N| < 1/4) = 0.197) and bounds nothing; over thousands
    of elements one sample's norm is that average already. Elements' errors are noise
    of that size: eight times its root mean square."""
    ref = newton_schulz(G, coef, eps)
    bits = 11 if out == "bf16" else 22
    n = 32 if ref.size <= 4096 else 1
    sq = 0.0
    for k in range(n):
        sq += np.linalg.norm(newton_schulz(G, coef, eps, bits, k) - ref) ** 2 / n
    e = 4 * np.sqrt(sq)
    return ref, e, 8 * e / np.sqrt(ref.size)
