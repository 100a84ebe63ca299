"""Plain 64-bit implementations of the layer operators (block norms, int8 products,
AdamW) on the host, written from their formulas, and the helpers their tests share."""
import math

import numpy as np
import torch

TINY = 2.0 ** -64


def bf16(x):
    """x rounded to bf16, as float64."""
    return x.to(torch.bfloat16).double()


# ------------------------------------------------------------- block norms --
def norm_forward(res, y, w_post, gate, scale, w_pre, eps):
    """(h before its rounding, rstd_post, function from a stored h to (n, rstd_pre))."""
    h, r_post = res, None
    if y is not None:
        z = y
        if w_post is not None:
            r_post = ((y * y).mean(1) + eps) ** -0.5
            z = y * r_post[:, None] * w_post
        h = res + scale * (z if gate is None else gate * z)

    def enter(stored):
        r_pre = ((stored * stored).mean(1) + eps) ** -0.5
        return stored * r_pre[:, None] * w_pre, r_pre

    return h, r_post, enter


def norm_backward(h, y, w_post, gate, scale, w_pre, r_post, r_pre, dn, dh):
    """Dict of the gradients; dgate in the gate's shape."""
    out = {}
    d = torch.zeros_like(dn if dn is not None else dh) if dh is None else dh.clone()
    if dn is not None:
        hh = h * r_pre[:, None]
        t = dn * w_pre
        d = d + r_pre[:, None] * (t - hh * (t * hh).mean(1, keepdim=True))
        out["dw_pre"] = (dn * hh).sum(0)
    out["dres"] = d
    dz = scale * d
    if y is not None:
        yh = y if r_post is None else y * r_post[:, None]
        z = yh if w_post is None else yh * w_post
        if gate is not None:
            out["dgate"] = (dz * z).sum_to_size(gate.shape)
    if gate is not None:
        dz = dz * gate
    if w_post is not None:
        out["dw_post"] = (dz * yh).sum(0)
        t = dz * w_post
        dz = r_post[:, None] * (t - yh * (t * yh).mean(1, keepdim=True))
    out["dy"] = dz
    return out


# ----------------------------------------------------------- int8 products --
def token_codes(x):
    """(codes int64, scales) of fp32 rows: the definition's IEEE fp32 operations, one by one."""
    x = x.numpy().astype(np.float32)
    amax = np.abs(x).max(1, initial=np.float32(0)).astype(np.float32)
    live = amax >= np.float32(TINY)
    with np.errstate(divide="ignore"):
        r = np.where(live, np.float32(127) / amax, np.float32(0)).astype(np.float32)
    s = np.where(live, amax / np.float32(127), np.float32(0)).astype(np.float32)
    codes = np.clip(np.rint((x * r[:, None]).astype(np.float32)), -127, 127)
    return torch.from_numpy(codes.astype(np.int64)), torch.from_numpy(s)


def int_product(a, w):
    """Exact integer product a w^T (float64 holds sums below 2^53)."""
    return (a.double() @ w.double().t())


# ------------------------------------------------------------------- AdamW --
def mix(x):
    x = x.astype(np.uint32)
    x = x ^ (x >> np.uint32(16))
    x = x * np.uint32(0x6A09E667)
    x = x ^ (x >> np.uint32(15))
    x = x * np.uint32(0xBB67AE85)
    return x ^ (x >> np.uint32(16))


def words(seed, tensor, n, salt):
    """The 32 random bits of every element of tensor `tensor` of a call."""
    key = mix(np.array([(seed + 0x9E3779B1 * (tensor + 1) + salt) % 2 ** 32], dtype=np.uint32))
    return mix(np.arange(n, dtype=np.uint32) ^ key)


#: every non-negative E4M3FN value in order
GRID = np.array([m * 2.0 ** -9 for m in range(8)] +
                [(8 + m) * 2.0 ** (e - 10) for e in range(1, 16) for m in range(8)][:119])


def pad_blocks(x):
    return np.concatenate([x, np.zeros(-len(x) % 256)]).reshape(-1, 256)


def encode(x, u, keep):
    """(values of the codes, scales, grid index of each): blocks of 256, rounded up where the
    place between two grid values and u in [0, 1) reach 1."""
    b = pad_blocks(x)
    amax = np.abs(b).max(1)
    s = np.where(amax < TINY, 0.0, amax / 448.0)
    per = np.repeat(s, 256)[:len(x)]
    a = np.minimum(np.where(per > 0, np.abs(x) / np.where(per > 0, per, 1.0), 0.0), 448.0)
    low = np.clip(np.searchsorted(GRID, a, side="right") - 1, 0, len(GRID) - 2)
    up = (a - GRID[low]) / (GRID[low + 1] - GRID[low]) + u >= 1.0
    k = low + up
    if keep:
        k = np.where((x > 0) & (per > 0), np.maximum(k, 1), k)
    return np.sign(x) * GRID[k] * per, s, k


def adamw(p, g, m, v, lr, wd, beta1, beta2, eps, step, clip=1.0):
    """One step in 64 bits: new (p, m, v) and the size of the terms that the update is formed
    from (those of m may cancel)."""
    g = g * clip
    size = beta1 * np.abs(m) + (1 - beta1) * np.abs(g)
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    per = lr / (1 - beta1 ** step) / (np.sqrt(v / (1 - beta2 ** step)) + eps)
    return p * (1 - lr * wd) - per * m, m, v, abs(per) * size


def grad_norm(grads, max_norm):
    total = math.sqrt(math.fsum(float((g.astype(np.float64) ** 2).sum()) for g in grads))
    return total, min(1.0, max_norm / (total + 1e-6))
