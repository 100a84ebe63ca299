"""Plain 64-bit implementations of the operators between an actor's products (heads of queries
and keys, log-probabilities of chosen tokens, policy and preference loss) on the host, written from their formulas."""
import math
from fractions import Fraction

import torch

TWO_PI = 2 * Fraction("3.14159265358979323846264338327950288419716939937510582097494459")


def f32(x):
    """x rounded to fp32, as float."""
    return float(torch.tensor(x, dtype=torch.float32))


# ------------------------------------------------------------------- heads --
def angles(positions, inv_freq):
    """cos and sin [tokens, 1, n] of position * inv_freq, both taken as they are stored.  In 64 bits
    the product's own rounding would be 2^-53 of it, 1e-4 at position 2^40: whole turns are
    taken off the exact product first."""
    freq = [Fraction(f) for f in inv_freq.double().tolist()]
    a = torch.tensor([[float((p * f) % TWO_PI) for f in freq] for p in positions.tolist()], dtype=torch.float64)
    a = a.reshape(len(positions), len(freq))
    return a.cos()[:, None], a.sin()[:, None]


def rotate(n, cos, sin, pairs):
    half = cos.shape[2]
    out = n.clone()
    first, second = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if pairs else (slice(0, half), slice(half, 2 * half))
    a, b = n[..., first], n[..., second]
    out[..., first], out[..., second] = a * cos - b * sin, b * cos + a * sin
    return out


def head_norm(x, w, eps):
    """(x normed, rsqrt factor): [tokens, heads, dim], [tokens, heads, 1]."""
    if w is None:
        return x, torch.ones_like(x[..., :1])
    r = ((x * x).mean(-1, keepdim=True) + eps) ** -0.5
    return x * r * w, r


def heads_forward(x, w, eps, positions, inv_freq, pairs, rope_scale=1.0):
    n, _ = head_norm(x, w, eps)
    half = inv_freq.numel()
    cos, sin = angles(positions, inv_freq)
    out = rotate(n, cos, sin, pairs)
    out[..., :2 * half] *= rope_scale
    out[positions < 0] = 0.0
    return out


def heads_backward(x, w, eps, positions, inv_freq, pairs, g, rope_scale=1.0):
    """dx, dw and the size of what each is summed from: for tolerances."""
    half = inv_freq.numel()
    cos, sin = angles(positions, inv_freq)
    live = positions >= 0
    dn = rotate(g, cos, -sin, pairs)
    dn[..., :2 * half] *= rope_scale
    dn[~live] = 0.0
    if w is None:
        return dn, None, dn.abs().amax(-1, keepdim=True), None
    x = torch.where(live[:, None, None], x, torch.ones_like(x))
    _, r = head_norm(x, w, eps)
    t, xr = dn * w, x * r
    dx = r * (t - xr * (t * xr).mean(-1, keepdim=True))
    size = r * (t.abs().amax(-1, keepdim=True) + xr.abs().amax(-1, keepdim=True) * (t * xr).abs().mean(-1, keepdim=True))
    return dx, (dn * xr).sum((0, 1)), size, (dn * xr).abs().sum((0, 1))


# ---------------------------------------------------------------- logprobs --
def token_logprobs(z, targets, scale):
    """Dict of logp, entropy, row_max, log_sum; rows with a negative target are 0."""
    live = targets >= 0
    m = z.amax(1)
    d = scale * (z - m[:, None])
    log_sum = d.exp().sum(1).log()
    logp = d - log_sum[:, None]
    p = logp.exp()
    entropy = -torch.where(p > 0, p * logp, torch.zeros_like(p)).sum(1)
    chosen = logp.gather(1, targets.clamp(0, z.shape[1] - 1)[:, None])[:, 0]
    # where almost all is the chosen token's: -log1p of the others
    others = d.exp().scatter(1, targets.clamp(0, z.shape[1] - 1)[:, None], 0.0).sum(1)
    top = d.gather(1, targets.clamp(0, z.shape[1] - 1)[:, None])[:, 0] == 0.0
    chosen = torch.where(top, -torch.log1p(others), chosen)
    log_sum = torch.where(top, torch.log1p(others), log_sum)
    return {k: torch.where(live, v, torch.zeros_like(v))
            for k, v in dict(logp=chosen, entropy=entropy, row_max=m, log_sum=log_sum).items()}


def token_logprobs_bwd(z, targets, scale, row_max, log_sum, entropy, dlogp, dentropy):
    live = targets >= 0
    g = torch.where(live, dlogp, torch.zeros_like(dlogp))[:, None]
    l = scale * (z - row_max[:, None]) - log_sum[:, None]
    p = l.exp()
    out = -g * p
    at = targets.clamp(min=0)[:, None]
    out.scatter_(1, at, g * -torch.expm1(l.gather(1, at)))
    if dentropy is not None:
        e = torch.where(live, dentropy, torch.zeros_like(dentropy))[:, None]
        out = out - e * torch.where(p > 0, p * (l + entropy[:, None]), torch.zeros_like(p))
    idle = ~live | ((dlogp == 0) & (torch.zeros_like(dlogp) if dentropy is None else dentropy).eq(0))
    out = scale * out
    out[idle] = 0.0
    return out


# ------------------------------------------------------------------ losses --
def spans(n, sequences, offsets):
    """(first, end) of every sequence."""
    if offsets is not None:
        return [(int(a), int(b)) for a, b in zip(offsets[:-1], offsets[1:])]
    step = n // sequences if sequences else 0
    return [(i * step, (i + 1) * step) for i in range(sequences)]


def policy_loss(logp, logp_old, adv, sequences, logp_ref=None, entropy=None, mask=None, offsets=None, clip_low=0.2,
                clip_high=0.2, dual_clip=0.0, beta=0.0, entropy_weight=0.0, kl=0, ratio="token", mean="tokens", n_norm=0.0):
    """Token by token in Python floats; log ratios and differences to the reference are fp32
    differences, thresholds fp32 (that is the definition).  Returns dict of lists and stats;
    tokens of no sequence are None."""
    n = logp.numel()
    ranges = spans(n, sequences, offsets)
    ok = [True] * n if mask is None else [bool(m) for m in mask]
    delta = (logp.float() - logp_old.float()).double().tolist()
    diff = None if logp_ref is None else (logp.float() - logp_ref.float()).double().tolist()
    hi, lo = f32(math.log1p(f32(clip_high))), f32(math.log1p(-f32(clip_low)))
    dual, log_dual = f32(dual_clip), f32(math.log(f32(dual_clip))) if dual_clip > 0 else 0.0
    beta, bonus = f32(beta), f32(entropy_weight)
    members = [[t for t in range(a, b) if ok[t]] for a, b in ranges]
    tokens, filled = sum(map(len, members)), sum(1 for m in members if m)
    big = n_norm if n_norm > 0 else (tokens if mean == "tokens" else filled)
    out = {k: [None] * n for k in ("dlogp", "dentropy", "token_loss", "flags", "size")}
    total = dict(loss=0.0, policy=0.0, kl=0.0, entropy=0.0, clipped=0, ratio=0.0)
    for s, (a, b) in enumerate(ranges):
        for t in range(a, b):
            for k in out:
                out[k][t] = 0 if k == "flags" else 0.0
        mean_delta = f32(math.fsum(delta[t] for t in members[s]) / len(members[s])) if members[s] else 0.0
        for t in members[s]:
            w = 1.0 / (big * (len(members[s]) if mean == "sequences" else 1))
            x = float(adv[t] if adv.numel() == n and adv.numel() != sequences else adv[s])
            d = mean_delta if ratio == "sequence" else delta[t]
            r = math.exp(d)
            chi = d <= hi if x >= 0 else d >= lo
            bound = 1.0 + f32(clip_high) if x >= 0 else 1.0 - f32(clip_low)
            if dual > 0 and x < 0 and d > log_dual:
                chi, bound = False, dual
            policy = 0.0 if x == 0 else -x * (r if chi else bound)
            slope = -x * r if chi and x != 0 else 0.0
            y, dy = 0.0, 0.0
            if kl:
                q = diff[t]
                y, dy = {1: (q, 1.0), 2: (q * q / 2, q), 3: (math.expm1(-q) + q, -math.expm1(-q))}[kl]
            h = 0.0 if entropy is None else float(entropy[t])
            loss = policy + beta * y - bonus * h
            out["dlogp"][t], out["dentropy"][t] = w * (slope + beta * dy), -bonus * w
            out["token_loss"][t] = w * loss
            out["flags"][t] = (1 if chi else 0) | (2 if not chi and x != 0 else 0)
            # what the token's values are summed from
            out["size"][t] = w * (abs(x) * max(r, bound) + abs(beta) * (1.0 + abs(diff[t]) + math.exp(-diff[t]) + diff[t] ** 2 if kl else 0.0) + abs(bonus * h))
            total["loss"] += w * loss
            total["policy"] += w * policy
            total["kl"] += w * y
            total["entropy"] += w * h
            total["clipped"] += out["flags"][t] >> 1
            total["ratio"] += r
    each = max(tokens, 1)
    out["stats"] = [total["loss"], total["policy"], total["kl"], total["entropy"], total["clipped"] / each,
                    total["ratio"] / each, tokens, filled]
    return out


def preference_loss(logp, sequences, logp_ref=None, mask=None, offsets=None, chosen=None, rejected=None, beta=0.1,
                    label_smoothing=0.0, margin=0.0, loss="logistic", length_mean=False, n_norm=0.0):
    n = logp.numel()
    ranges = spans(n, sequences, offsets)
    ok = [True] * n if mask is None else [bool(m) for m in mask]
    x = (logp.float() if logp_ref is None else logp.float() - logp_ref.float()).double().tolist()
    beta, eps, margin = f32(beta), f32(label_smoothing), f32(margin)
    members = [[t for t in range(a, b) if ok[t]] for a, b in ranges]
    value = [math.fsum(x[t] for t in m) / (len(m) if length_mean and m else 1) for m in members]
    pairs = [(2 * p, 2 * p + 1) for p in range(sequences // 2)] if chosen is None else list(zip(chosen.tolist(), rejected.tolist()))
    slope, losses, sums = [0.0] * sequences, [], [0.0] * 6

    def softplus(y):
        return max(y, 0.0) + math.log1p(math.exp(-abs(y)))

    def sigmoid(y):
        return 1.0 / (1.0 + math.exp(-y)) if y > -700 else 0.0

    for c, r in pairs:
        if c < 0 or r < 0 or not members[c] or not members[r]:
            losses.append(0.0)
            continue
        h = value[c] - value[r] - margin
        y = beta * h
        if loss == "logistic":
            v, d = (1 - eps) * softplus(-y) + eps * softplus(y), beta * (eps * sigmoid(y) - (1 - eps) * sigmoid(-y))
        elif loss == "hinge":
            v, d = max(0.0, 1.0 - y), -beta if y < 1.0 else 0.0
        else:
            v, d = (h - 0.5 / beta) ** 2, 2.0 * (h - 0.5 / beta)
        losses.append(v)
        slope[c] += d
        slope[r] -= d
        for i, q in enumerate((1.0, v, float(h > 0), y, beta * value[c], beta * value[r])):
            sums[i] += q
    norm = n_norm if n_norm > 0 else max(sums[0], 1.0)
    dlogp = [None] * n
    for s, (a, b) in enumerate(ranges):
        for t in range(a, b):
            dlogp[t] = slope[s] / (norm * (len(members[s]) if length_mean else 1)) if ok[t] else 0.0
    return {"dlogp": dlogp, "rewards": [beta * v for v in value], "pair_loss": losses,
            "stats": [q / norm for q in sums[1:]] + [sums[0]]}
