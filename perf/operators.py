"""The operators on either side of the norms and clipped sums of a private step.

A training step hands this library its layers' operands and takes noised sums
from it. Around that stand: LayerNorm, whose backward pass yields the
per-example gradients of its gain and bias; the head's loss, whose gradient is
the logit gradient that the head's norm and sum read (cross-entropy for plain
fine-tuning, a preference loss where an example is a pair of answers); the
token log-probabilities that evaluation and a frozen reference model need; and
the update made of the noised sums by orthogonalising them with Newton-Schulz
products.

The sizes are those of GPT-2's layers (blocks of width 768, vocabulary 50257,
at most 1024 positions), of the paper's batches (24 prompts of at most 128
tokens), of the repository's benchmark (32 x 128), and generic ones around
them. Hidden states are N(0, 1) with a mean per token, output gradients
N(0, 1e-3) scaled per example, logits N(0, 2); a noised sum is a low-rank
gradient under the Gaussian mechanism's noise.
"""
from __future__ import annotations

import math

import torch

own = False   # True: the library's calls; False: the same operators in elementary torch operations

GPT2_V = 50257
EPS = 1e-5                               # LayerNorm's
BETA, SMOOTHING = 0.1, 0.05              # the preference loss's
NS_COEF = (3.4445, -4.7750, 2.0315)      # a X + b (X X^T) X + c (X X^T)^2 X
NS_STEPS, NS_EPS = 5, 1e-7
# The noised sum's Gaussian noise against its signal, as Frobenius norms: with
# sigma = 1 the noise of a weight matrix outweighs a clipped gradient.
NS_SIGNAL = 0.5


# ------------------------------------------------------------------- cases
def _ln(direction, dtype, B, T, d, param="fp32", pad=False, name=None):
    c = {"op": "layernorm_" + direction, "dtype": dtype, "B": B, "T": T, "d": d, "param": param,
         "pad": pad}
    return c if name is None else {"name": name, **c}


def _loss(op, dtype, B, T, V, pad, name=None):
    c = {"op": op, "dtype": dtype, "B": B, "T": T, "V": V, "pad": pad}
    return c if name is None else {"name": name, **c}


def _orth(dtype, blocks, shapes, out, name=None):
    c = {"op": "orthogonalize", "dtype": dtype, "blocks": blocks, "shapes": shapes, "out": out}
    return c if name is None else {"name": name, **c}


def listed():
    return [
        # One block of width 64, four examples of 16 tokens, as in a smoke test
        # or a unit test of a training loop: launches are all it costs.
        _ln("backward", "fp32", 4, 16, 64, name="ln_backward_tiny_fp32"),
        # One LayerNorm of GPT-2 small at the benchmark's batch.
        _ln("forward", "bf16", 32, 128, 768, param="bf16", name="ln_forward_b32_t128"),
        _ln("backward", "bf16", 32, 128, 768, name="ln_backward_b32_t128"),
        # Two long ragged documents of a wider model in fp32, rows padded: few
        # examples, so each one's weight gradient runs over thousands of tokens.
        _ln("backward", "fp32", 2, 8191, 1601, pad=True, name="ln_backward_b2_t8191_fp32"),
        # Scoring one next token for each of eight prompts.
        _loss("logprobs", "bf16", 8, 1, GPT2_V, False, name="logprobs_b8_t1"),
        # Scoring the paper's batch, logits as PyTorch lays them out.
        _loss("logprobs", "bf16", 24, 128, GPT2_V, False, name="logprobs_b24_t128"),
        # The loss of the benchmark's step.
        _loss("cross_entropy", "bf16", 32, 128, GPT2_V, True, name="cross_entropy_b32_t128"),
        # ... and in fp32 at a prompt length that is no multiple of a tile.
        _loss("cross_entropy", "fp32", 24, 100, GPT2_V, False, name="cross_entropy_b24_t100_fp32"),
        # Preference fine-tuning: sixteen pairs of answers of 512 tokens each.
        _loss("preference", "bf16", 16, 1024, GPT2_V, True, name="preference_b16_t1024"),
        # The weight matrices of a block of width 64: the smallest update.
        _orth("fp32", 1, "64x192 64x64 64x256 256x64", "fp32", name="orthogonalize_tiny_fp32"),
        # The update of every weight matrix of GPT-2 small's blocks.
        _orth("fp32", 12, "768x2304 768x768 768x3072 3072x768", "bf16",
              name="orthogonalize_gpt2"),
        # One wide matrix of odd sizes, kept in fp32.
        _orth("fp32", 1, "1601x6397", "fp32", name="orthogonalize_1601x6397_fp32"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["layernorm", "layernorm", "logprobs", "cross_entropy", "preference",
                     "orthogonalize", "orthogonalize"])
    dtype = "bf16" if rng.random() < 0.6 else "fp32"
    if op == "layernorm":
        d = _log(rng, 16, 8192)
        if rng.random() < 0.6:
            d = max(16, d // 8 * 8)
        B = _log(rng, 1, 64)
        T = min(_log(rng, 1, 8192), max(1, 25_000_000 // (B * d)))
        return _ln(rng.choice(["forward", "backward"]), dtype, B, T, d,
                   param="fp32" if dtype == "fp32" or rng.random() < 0.5 else "bf16",
                   pad=rng.random() < 0.3)
    if op != "orthogonalize":
        V = GPT2_V if rng.random() < 0.4 else _log(rng, 64, 150_000)
        B = _log(rng, 1, 48)
        T = min(_log(rng, 1 if op == "logprobs" else 4, 2048),
                max(4, (300_000_000 if op == "preference" else 120_000_000) // (B * V)))
        return _loss(op, dtype, B, T, V, rng.random() < 0.5)
    shapes, spent = [], 0.0
    for _ in range(rng.choice([1, 1, 2, 3])):
        r, c = _log(rng, 16, 2500), _log(rng, 16, 6000)
        if rng.random() < 0.5:
            r, c = max(16, r // 16 * 16), max(16, c // 16 * 16)
        if rng.random() < 0.4:
            r, c = c, r
        shapes.append("%dx%d" % (r, c))
        spent += min(r, c) ** 2 * (3.0 * max(r, c) + min(r, c))
    blocks = max(1, min(_log(rng, 1, 12), int(1.5e11 / spent)))
    return _orth(dtype, blocks, " ".join(shapes), rng.choice(["bf16", "fp32"]))


# ------------------------------------------------------------------- shapes
_DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
_ES = {"bf16": 2, "fp32": 4}


def _up(x, m):
    return (x + m - 1) // m * m


def _shapes(case):
    return [tuple(int(v) for v in s.split("x")) for s in case["shapes"].split()]


def _answers(case):
    """[(first, end)] of the scored tokens of every answer: (example, answer)
    in order. A prompt's tokens and the padding behind an answer are ignored."""
    T, halves = case["T"], 2 if case["op"] == "preference" else 1
    split = T // 2
    spans = []
    for b in range(case["B"]):
        for h in range(halves):
            n = T if halves == 1 else split if h == 0 else T - split
            at = split * h
            end = n - (7 * b + 3 * h) % (n // 4 + 1)
            spans.append((b, at + end // 4 if n > 1 else at, at + end))
    return spans


# ------------------------------------------------------------------- inputs
def _inputs(case, seed):
    """Every operand of the case on the GPU, from the seed alone."""
    g = torch.Generator(device="cuda").manual_seed(1000003 * (seed + 1) + 29)
    dt, op = _DT[case["dtype"]], case["op"]

    def normal(*shape):
        return torch.randn(*shape, device="cuda", generator=g)

    s = {}
    if op.startswith("layernorm"):
        B, T, d = case["B"], case["T"], case["d"]
        ld = _up(d, 64) + 64 if case["pad"] else d

        def tokens(x):   # rows of d elements, `ld` apart
            t = torch.zeros(B, T, ld, device="cuda", dtype=dt)
            t[:, :, :d] = x
            return t[:, :, :d]

        s["x"] = tokens(normal(B, T, d) * torch.exp(0.3 * normal(B, T, 1)) + 0.5 * normal(B, T, 1))
        s["gain"] = (1.0 + 0.2 * normal(d)).to(_DT[case["param"]])
        s["bias"] = (0.1 * normal(d)).to(_DT[case["param"]])
        if op == "layernorm_backward":
            s["gy"] = tokens(1e-3 * normal(B, T, d) * torch.exp(0.5 * normal(B, 1, 1)))
            x = s["x"].double()
            mean = x.mean(2)
            s["rstd"] = torch.rsqrt((x - mean[:, :, None]).square().mean(2) + EPS).float()
            s["mean"] = mean.float()
        return s
    if op == "orthogonalize":
        s["grads"] = []
        for r, c in _shapes(case):
            n = case["blocks"]
            k = min(8, r, c)
            weights = torch.arange(1, k + 1, device="cuda", dtype=torch.float32).pow(-1.0)
            signal = torch.bmm(normal(n, r, k) * weights, normal(n, k, c))
            noise = normal(n, r, c)
            signal *= NS_SIGNAL * math.sqrt(r * c) / signal.square().sum((1, 2), keepdim=True).sqrt()
            s["grads"].append(((signal + noise) / 32).to(dt))
        return s
    B, T, V = case["B"], case["T"], case["V"]
    z = torch.zeros(B, T, _up(V, 64) if case["pad"] else V, device="cuda", dtype=dt)
    for b in range(B):
        z[b, :, :V] = 2.0 * normal(T, V)
    s["Z"] = z[:, :, :V]
    cdf = torch.arange(1, V + 1, device="cuda", dtype=torch.float64).pow(-1.1).cumsum(0)
    u = torch.rand(B, T, device="cuda", dtype=torch.float64, generator=g) * cdf[-1]
    ids = torch.searchsorted(cdf, u, right=True).clamp_(max=V - 1)
    keep = torch.zeros(B, T, dtype=torch.bool)
    weight = torch.zeros(B, T)
    for b, t0, t1 in _answers(case):
        keep[b, t0:t1] = True
        weight[b, t0:t1] = 1.0 / max(1, t1 - t0)
    keep = keep.cuda()
    s["targets"] = torch.where(keep, ids, torch.full_like(ids, -1)).to(torch.int32)
    if op == "cross_entropy":
        s["w"] = weight.cuda()   # the mean over an example's scored tokens
    if op == "preference":
        # A reference model close to this one: its log-probabilities differ
        # from (target logit - log sum exp) by N(0, 0.3) a token.
        zt = s["Z"].gather(2, ids[:, :, None])[:, :, 0].float()
        ref = zt - (math.log(V) + 2.0) + 0.3 * normal(B, T)
        s["ref"] = torch.where(keep, ref, torch.zeros_like(ref))
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"], op = case, case["op"]

    def empty(*shape, dtype=torch.float32):
        return torch.empty(*shape, device="cuda", dtype=dtype)

    # The buffers that a program's calls write to.
    if op.startswith("layernorm"):
        B, T, d = case["B"], case["T"], case["d"]
        s["out"] = empty(B, T, d, dtype=_DT[case["dtype"]])
        if op == "layernorm_forward":
            s["mean"], s["rstd"] = empty(B, T), empty(B, T)
        else:
            s["dgain"], s["dbias"], s["norm2"] = empty(B, d), empty(B, d), empty(B)
    elif op == "orthogonalize":
        s["out"] = [torch.empty_like(g, dtype=_DT[case["out"]]) for g in s["grads"]]
    else:
        B, T, V = case["B"], case["T"], case["V"]
        s["logp"] = empty(B, T)
        if op == "logprobs":
            s["lse"] = empty(B, T)
        else:
            gz = torch.zeros(B, T, _up(V, 64) if case["pad"] else V, device="cuda",
                             dtype=_DT[case["dtype"]])
            s["Gz"] = gz[:, :, :V]
        if op == "preference":
            s["loss"], s["rewards"] = empty(B), empty(B, 2)
    return s


# --------------------------------------------------------------------- runs
def run(s):
    return _own(s) if own else _plain(s)


def _own(s):
    from paper_2609_40335_amd import dpghost as dp
    case = s["case"]
    op = case["op"]
    if op == "layernorm_forward":
        dp.dp_layernorm_forward(s["x"], s["gain"], s["bias"], s["out"], mean=s["mean"],
                                rstd=s["rstd"], eps=EPS)
        return {"y": s["out"], "mean": s["mean"], "rstd": s["rstd"]}
    if op == "layernorm_backward":
        dp.dp_layernorm_backward(s["gy"], s["x"], s["gain"], s["mean"], s["rstd"], s["out"],
                                 dgain=s["dgain"], dbias=s["dbias"], norm2=s["norm2"])
        return {"dx": s["out"], "dgain": s["dgain"], "dbias": s["dbias"], "norm2": s["norm2"]}
    if op == "logprobs":
        dp.dp_token_logprobs(s["Z"], s["targets"], s["logp"], lse=s["lse"])
        return {"logp": s["logp"], "lse": s["lse"]}
    if op == "cross_entropy":
        dp.dp_cross_entropy(s["Z"], s["targets"], s["w"], s["logp"], s["Gz"])
        return {"logp": s["logp"], "Gz": s["Gz"]}
    if op == "preference":
        dp.dp_preference_loss(s["Z"], s["targets"], case["T"] // 2, s["ref"], BETA, s["loss"],
                              rewards=s["rewards"], logp=s["logp"], Gz=s["Gz"],
                              label_smoothing=SMOOTHING)
        return {"loss": s["loss"], "rewards": s["rewards"], "logp": s["logp"], "Gz": s["Gz"]}
    grads = [m for g in s["grads"] for m in g.unbind(0)]
    outs = [m for o in s["out"] for m in o.unbind(0)]
    dp.dp_orthogonalize_grouped(grads, outs, coef=NS_COEF, steps=NS_STEPS, eps=NS_EPS)
    return s["out"]


def _plain(s):
    """The operators in elementary torch operations, in 32 bits."""
    case = s["case"]
    op = case["op"]
    dt = _DT[case["dtype"]]
    if op == "layernorm_forward":
        x = s["x"].float()
        mean = x.mean(2, keepdim=True)
        centred = x - mean
        rstd = torch.rsqrt(centred.square().mean(2, keepdim=True) + EPS)
        y = centred * rstd * s["gain"].float() + s["bias"].float()
        return {"y": y.to(dt), "mean": mean[:, :, 0], "rstd": rstd[:, :, 0]}
    if op == "layernorm_backward":
        gy, rstd = s["gy"].float(), s["rstd"][:, :, None]
        xhat = (s["x"].float() - s["mean"][:, :, None]) * rstd
        g = gy * s["gain"].float()
        dx = (g - g.mean(2, keepdim=True) - xhat * (g * xhat).mean(2, keepdim=True)) * rstd
        dgain, dbias = (gy * xhat).sum(1), gy.sum(1)
        norm2 = dgain.square().sum(1) + dbias.square().sum(1)
        return {"dx": dx.to(dt), "dgain": dgain, "dbias": dbias, "norm2": norm2}
    if op == "orthogonalize":
        return [_plain_orthogonal(g, _DT[case["out"]]) for g in s["grads"]]
    kept = s["targets"] >= 0
    z = s["Z"].float()
    top = z.amax(2, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(2, keepdim=True)
    # The logarithms of a row's sum are subtracted in 64 bits: a margin is the
    # difference of long sums of them.
    lse = (top.double() + torch.log(total.double()))[:, :, 0]
    zero = torch.zeros_like(lse)
    at = s["targets"].long().clamp(min=0)[:, :, None]
    logq = torch.where(kept, z.gather(2, at)[:, :, 0] - lse, zero)
    logp = logq.float()
    if op == "logprobs":
        return {"logp": logp, "lse": torch.where(kept, lse, zero).float()}
    if op == "cross_entropy":
        up = torch.where(kept, s["w"], zero.float())
    else:
        ratio = torch.where(kept, logq - s["ref"], zero)
        half = case["T"] // 2
        rewards = BETA * torch.stack([ratio[:, :half].sum(1), ratio[:, half:].sum(1)], 1)
        margin = rewards[:, 0] - rewards[:, 1]
        p = 1.0 / (1.0 + torch.exp(-margin))
        soft = torch.clamp(margin, min=0) + torch.log1p(torch.exp(-margin.abs()))   # -log(1 - p)
        loss = (1.0 - SMOOTHING) * (soft - margin) + SMOOTHING * soft
        down = BETA * ((1.0 - SMOOTHING) * (1.0 - p) - SMOOTHING * p)   # -d loss / d (log ratio)
        up = torch.cat([down[:, None].expand(-1, half), -down[:, None].expand(-1, case["T"] - half)],
                       1).float()
        up = torch.where(kept, up, torch.zeros_like(up))
    p = e / total * up[:, :, None]
    p.scatter_add_(2, at, -up[:, :, None])
    gz = {"Gz": p.to(dt)}
    if op == "cross_entropy":
        return {"logp": logp, **gz}
    return {"loss": loss.float(), "rewards": rewards.float(), "logp": logp, **gz}


def _plain_orthogonal(g, dtype):
    """Newton-Schulz on a stack of matrices, along the shorter side."""
    x = g.float()
    wide = x.shape[1] <= x.shape[2]
    if not wide:
        x = x.transpose(1, 2).contiguous()
    norm = x.double().square().sum((1, 2), keepdim=True).sqrt() + NS_EPS
    x = (x.double() / norm).float()
    a, b, c = NS_COEF
    for _ in range(NS_STEPS):
        gram = torch.bmm(x, x.transpose(1, 2))
        poly = torch.baddbmm(gram, gram, gram, beta=b, alpha=c)
        x = torch.baddbmm(x, poly, x, beta=a)
    return (x if wide else x.transpose(1, 2)).to(dtype).contiguous()


# --------------------------------------------------------------------- work
def work(case):
    op, es = case["op"], _ES[case["dtype"]]
    if op.startswith("layernorm"):
        B, T, d = case["B"], case["T"], case["d"]
        n = float(B) * T * d
        stats, ps = 8.0 * B * T, _ES[case["param"]]
        if op == "layernorm_forward":
            return {"bytes": 2 * n * es + stats + 2.0 * ps * d, "flops": 8 * n}
        return {"bytes": 3 * n * es + stats + 1.0 * ps * d + 8.0 * B * d + 4.0 * B,
                "flops": 14 * n}
    if op == "orthogonalize":
        nbytes = flops = 0.0
        for r, c in _shapes(case):
            m, n = min(r, c), max(r, c)
            nbytes += float(r) * c * (es + _ES[case["out"]])
            # The two symmetric products once per pair of rows, the update whole.
            flops += NS_STEPS * (float(m) * (m + 1) * (n + m) + 2.0 * m * m * n)
        return {"bytes": case["blocks"] * nbytes, "flops": case["blocks"] * flops}
    B, T, V = case["B"], case["T"], case["V"]
    scored = sum(t1 - t0 for _, t0, t1 in _answers(case))
    nbytes = float(scored) * V * es + 8.0 * B * T
    if op == "logprobs":
        return {"bytes": nbytes + 4.0 * B * T, "flops": 4.0 * scored * V}
    nbytes += float(B) * T * V * es + 4.0 * B * T
    return {"bytes": nbytes, "flops": 7.0 * scored * V}


# -------------------------------------------------------------------- exact
def exact(case, seed):
    s = _inputs(case, seed)
    op, f64 = case["op"], torch.float64
    if op == "layernorm_forward":
        x = s["x"].to(f64)
        var, mean = torch.var_mean(x, dim=2, correction=0)
        rstd = 1.0 / torch.sqrt(var + EPS)
        y = (x - mean.unsqueeze(2)) * rstd.unsqueeze(2)
        return {"y": y * s["gain"].to(f64) + s["bias"].to(f64), "mean": mean, "rstd": rstd}
    if op == "layernorm_backward":
        # From the saved statistics: the Jacobian of x -> xhat applied to g.
        B, d = case["B"], case["d"]
        out = {"dx": [], "dgain": [], "dbias": [], "norm2": []}
        for b in range(B):
            gy, r = s["gy"][b].to(f64), s["rstd"][b].to(f64)[:, None]
            xhat = (s["x"][b].to(f64) - s["mean"][b].to(f64)[:, None]) * r
            g = gy * s["gain"].to(f64)
            along = (g * xhat).sum(1, keepdim=True) / d
            out["dx"].append(r * (g - g.sum(1, keepdim=True) / d - along * xhat))
            w, v = (gy * xhat).sum(0), gy.sum(0)
            out["dgain"].append(w)
            out["dbias"].append(v)
            out["norm2"].append(torch.dot(w, w) + torch.dot(v, v))
        return {k: torch.stack(v) for k, v in out.items()}
    if op == "orthogonalize":
        a, b, c = NS_COEF
        outs = []
        for g in s["grads"]:
            done = []
            for m in g:
                x = m.to(f64)
                flip = x.shape[0] > x.shape[1]
                x = x.t().contiguous() if flip else x
                x = x / (torch.linalg.matrix_norm(x) + NS_EPS)
                eye = torch.eye(x.shape[0], device="cuda", dtype=f64)
                for _ in range(NS_STEPS):
                    q = torch.mm(x, x.t())
                    x = torch.mm(a * eye + torch.mm(q, b * eye + c * q), x)
                done.append(x.t() if flip else x)
            outs.append(torch.stack(done))
        return outs
    B, T, V = case["B"], case["T"], case["V"]
    half = T // 2
    out = {"logp": torch.zeros(B, T, device="cuda", dtype=f64)}
    if op == "logprobs":
        out["lse"] = torch.zeros(B, T, device="cuda", dtype=f64)
    else:
        out["Gz"] = torch.zeros(B, T, V, device="cuda", dtype=f64)
    if op == "preference":
        out["loss"] = torch.zeros(B, device="cuda", dtype=f64)
        out["rewards"] = torch.zeros(B, 2, device="cuda", dtype=f64)
    for b in range(B):
        rows = torch.nonzero(s["targets"][b] >= 0)[:, 0]
        ids = s["targets"][b][rows].long()
        logq = torch.log_softmax(s["Z"][b][rows].to(f64), dim=1)
        k = torch.arange(rows.numel(), device="cuda")
        logp = logq[k, ids]
        out["logp"][b, rows] = logp
        if op == "logprobs":
            out["lse"][b, rows] = torch.logsumexp(s["Z"][b][rows].to(f64), dim=1)
            continue
        if op == "cross_entropy":
            up = s["w"][b][rows].to(f64)
        else:
            ratio = BETA * (logp - s["ref"][b][rows].to(f64))
            first = rows < half
            chosen, rejected = ratio[first].sum(), ratio[~first].sum()
            m = chosen - rejected
            out["rewards"][b, 0], out["rewards"][b, 1] = chosen, rejected
            out["loss"][b] = -((1 - SMOOTHING) * torch.nn.functional.logsigmoid(m)
                               + SMOOTHING * torch.nn.functional.logsigmoid(-m))
            slope = (1 - SMOOTHING) * torch.sigmoid(-m) - SMOOTHING * torch.sigmoid(m)
            up = BETA * slope * torch.where(first, 1.0, -1.0).to(f64)
        grad = torch.exp(logq)
        grad[k, ids] -= 1.0
        out["Gz"][b, rows] = grad * up[:, None]
    return out
