"""Plain 64-bit definitions of the operators around the head: embedding lookup, layer norm, verification of drafted tokens."""
import math

import torch

HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
F32 = 2.0 ** -24


def norm(x, weight, bias, eps):
    """(y, stats) and how far 32-bit arithmetic may be off: sums of at most 64 chained additions (32 in a thread, 5 in a warp, the warps')."""
    x = x.double()
    mean = x.mean(1, keepdim=True)
    var = ((x - mean) ** 2).mean(1, keepdim=True)
    rstd = 1 / (var + eps).sqrt()
    w = torch.ones(x.shape[1], dtype=torch.float64, device=x.device) if weight is None else weight.double()
    b = torch.zeros_like(w) if bias is None else bias.double()
    h = (x - mean) * rstd
    y = h * w + b
    off_mean = 64 * F32 * x.abs().mean(1, keepdim=True)
    # the squares' sum is about a mean that is off by off_mean; its own roundings; each difference is off by off_mean and a rounding
    off_rstd = rstd * (64 * F32 + (rstd * off_mean) ** 2)
    off = w.abs() * (rstd * (off_mean + F32 * (x - mean).abs()) + (x - mean).abs() * off_rstd) + 3 * F32 * (h * w).abs() + F32 * y.abs()
    return y, torch.cat([mean, rstd], 1), off, torch.cat([off_mean, off_rstd], 1)


def norm_grad(x, dy, weight, stats):
    """(dx, dweight, dbias) and how far each may be off in 32 bits: 64 chained additions along a row; down the rows chains of 128, then of their sums."""
    x, dy = x.double(), dy.double()
    mean, rstd = stats[:, :1].double(), stats[:, 1:].double()
    w = torch.ones(x.shape[1], dtype=torch.float64, device=x.device) if weight is None else weight.double()
    h, g, n = (x - mean) * rstd, dy * w, x.shape[1]
    off_h = 2 * F32 * h.abs()
    a, b = g.mean(1, keepdim=True), (g * h).mean(1, keepdim=True)
    dx = (g - a - h * b) * rstd
    off_a = 66 * F32 * g.abs().mean(1, keepdim=True)
    off_b = 68 * F32 * (g * h).abs().mean(1, keepdim=True)
    off = rstd * (4 * F32 * (g.abs() + a.abs() + (h * b).abs()) + off_a + h.abs() * off_b + off_h * b.abs()) + F32 * dx.abs()
    chain = 128 + x.shape[0] / 128 + 64
    return dx, (dy * h).sum(0), dy.sum(0), off, (dy.abs() * (chain * F32 * h.abs() + off_h)).sum(0), chain * F32 * dy.abs().sum(0)


def embed_grad(tokens, grad_out, vocab, scale):
    """The table's gradient and the sum of the terms' sizes."""
    t = tokens.cpu()
    out = torch.zeros(vocab, grad_out.shape[1], dtype=torch.float64)
    size = torch.zeros_like(out)
    g = grad_out.cpu().double()
    keep = (t >= 0) & (t < vocab)
    out.index_add_(0, t[keep], g[keep])
    size.index_add_(0, t[keep], g[keep].abs())
    return (out * scale).to(grad_out.device), (size * abs(scale)).to(grad_out.device)


def log_softmax(z, scale):
    """NaN where the row has NaN or +inf; -inf everywhere where nothing is left."""
    z = z.double()
    if bool(torch.isnan(z).any()) or bool((z == math.inf).any()) or not scale > 0:
        return torch.full_like(z, math.nan)
    m = z.max()
    if m == -math.inf:
        return torch.full_like(z, -math.inf)
    y = (z - m) * scale
    return y - y.exp().sum().log()


def largest(z):
    """Lowest column of the largest logit, -1 where the row has none."""
    z = z.double()
    m = z.max()
    return -1 if math.isnan(m) or math.isinf(m) else int((z == m).nonzero()[0, 0])


def race(weight, noise):
    """(column, by how much it is ahead, relative); (-1, 1) where no weight is left."""
    weight, noise = weight.double(), noise.double()
    score = torch.where(weight > 0, weight / noise, torch.tensor(-1.0, dtype=torch.float64))
    score = torch.where(torch.isnan(score) | (score <= 0), torch.tensor(-1.0, dtype=torch.float64), score)
    best = score.max()
    if best <= 0:
        return -1, 1.0
    at = int((score == best).nonzero()[0, 0])
    rest = score[score != best]
    return at, 1.0 if rest.numel() == 0 or math.isinf(best) else float((best - rest.max()) / best)


def verify(logits, draft_logits, ids, uniform, noise, scale):
    """One sequence: logits [n + 1, vocab], draft_logits [n, vocab] or None, on the CPU.  (tokens, accepted, log probabilities, margin): margin is how
    far, relative, the nearest decision was from going the other way."""
    n, vocab = ids.shape[0], logits.shape[1]
    tokens, logprob, margin, i = [], [], 1.0, 0
    greedy = scale > 2e38
    while True:
        there = i < n and 0 <= int(ids[i]) < vocab
        d = int(ids[i]) if there else -1
        if greedy:
            best = largest(logits[i])
            if there and best == d:
                tokens.append(d), logprob.append(0.0)
                i += 1
                continue
            tokens.append(best), logprob.append(0.0)
            break
        lp = log_softmax(logits[i], scale)
        p = lp.exp()
        q = torch.zeros_like(p)
        if there:
            if draft_logits is None:
                q[d] = 1.0
            else:
                q = log_softmax(draft_logits[i], scale).exp()
            a, b = float(uniform[i].double() * q[d]), float(p[d])
            if a != b and not math.isnan(a) and not math.isnan(b):
                margin = min(margin, abs(a - b) / max(a, b))
            if a < b:
                tokens.append(d), logprob.append(float(lp[d]))
                i += 1
                continue
        rest = (p - q).clamp(min=0)
        left = rest if there and bool((rest > 0).any()) else p
        # what rounding leaves of p - q is not compared: it is off by 2^-20 of p
        best, ahead = race(left, noise)
        if best >= 0:
            margin = min(margin, ahead * float(left[best] / p[best]))
        tokens.append(best), logprob.append(float(lp[best]) if best >= 0 else 0.0)
        break
    pad = n + 1 - len(tokens)
    return tokens + [-1] * pad, i, logprob + [0.0] * pad, margin
