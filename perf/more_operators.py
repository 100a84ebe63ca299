"""Timed cases of the operators between an actor's products: heads of queries and keys, and from logits to the loss.

Behind the projections every head of the queries and keys is normed and rotated by its
token's position; behind the vocabulary's product the chosen tokens' log-probabilities are
taken from the logits, a clipped policy loss or a preference loss gives its value and its
gradient to each log-probability, and that gradient goes back to the logits.

run() makes each pass twice over: with ``own`` by the calls of the package's binding, else
in plain torch operations in 32 bits (angles of positions in 64).  prepare() draws what a
trainer has in hand at that point, from the seed alone; exact() evaluates the definitions
in 64 bits.

Head layouts are those that go with the package's widths (3584 = 28 x 128 with 4 key heads,
896 = 14 x 64 with 2, 4096 = 32 x 128 with 8) and generic ones; token counts run from one to
a complete 16384-token microbatch, vocabularies to 131072 and beyond, odd ones among them.
"""
import math

import torch

own = False

DEV = "cuda"
EPS = 1e-6                                   # of the norms
TINY = 2.0 ** -64                            # blocks below it have scale 0
LARGEST_HEADS = 16384 * 32 * 128             # elements of queries and keys
LARGEST_LOGITS = 8192 * 131072
LARGEST_TOKENS = 1 << 20


# ------------------------------------------------------------------- cases --
def listed():
    return [
        # one step of 64 responses in flight, each at its own position: launches count
        {"name": "heads_rollout_step", "kind": "heads", "tokens": 64, "q": 28, "k": 4, "dim": 128, "rotated": 128,
         "pairs": False, "norm": True, "head_major": False, "start": 40000},
        # forward and recompute of a whole microbatch
        {"name": "heads_microbatch", "kind": "heads", "tokens": 16384, "q": 28, "k": 4, "dim": 128, "rotated": 128,
         "pairs": False, "norm": True, "head_major": False, "start": 0},
        # its backward with the weights' gradients, attention's gradients head by head
        {"name": "heads_bwd_microbatch", "kind": "heads_bwd", "tokens": 16384, "q": 28, "k": 4, "dim": 128,
         "rotated": 128, "pairs": False, "norm": True, "weights": True, "head_major": True, "start": 0,
         "code": "none", "block": 0},
        # ragged tokens of a small model, neighbouring columns rotated, half of each head, saved rows in L
        {"name": "heads_bwd_ragged_l", "kind": "heads_bwd", "tokens": 11987, "q": 14, "k": 2, "dim": 64, "rotated": 32,
         "pairs": True, "norm": True, "weights": False, "head_major": False, "start": 0, "code": "e4m3fn", "block": 128},
        # one token of a rollout: its log-probability and entropy
        {"name": "logprobs_one_row", "kind": "logprobs", "rows": 1, "vocab": 131072, "pad": 0, "f32": False,
         "entropy": True, "scale": 1.0, "idle": 0.0},
        # scoring half a microbatch
        {"name": "logprobs_microbatch", "kind": "logprobs", "rows": 8192, "vocab": 131072, "pad": 0, "f32": False,
         "entropy": True, "scale": 1.0, "idle": 0.0},
        # the gradient of its logits, three tenths of the rows without one (prompts, padding, clipped tokens)
        {"name": "logprobs_bwd_microbatch", "kind": "logprobs_bwd", "rows": 8192, "vocab": 131072, "pad": 0, "f32": False,
         "entropy": False, "scale": 1.0, "idle": 0.3},
        # fp32 logits of an odd vocabulary in dense rows, a temperature and an entropy bonus
        {"name": "logprobs_bwd_odd", "kind": "logprobs_bwd", "rows": 997, "vocab": 50021, "pad": 0, "f32": True,
         "entropy": True, "scale": 1.25, "idle": 0.2},
        # one small update: 4 prompts x 8 responses of 32 slots, one ratio a token
        {"name": "policy_small", "kind": "policy", "sequences": 32, "length": 32, "ragged": False, "ratio": "token",
         "kl": 3, "beta": 1e-3, "mean": "tokens", "high": 0.2, "dual": 0.0, "bonus": 0.0, "padded": 0.25},
        # a large rollout batch, packed: one ratio a sequence, mean of the sequences' means, entropy bonus
        {"name": "policy_packed", "kind": "policy", "sequences": 512, "length": 2047, "ragged": True, "ratio": "sequence",
         "kl": 2, "beta": 1e-2, "mean": "sequences", "high": 0.28, "dual": 3.0, "bonus": 1e-3, "padded": 0.1},
        # eight pairs of short answers against a reference
        {"name": "preference_small", "kind": "preference", "sequences": 16, "length": 211, "ragged": False, "loss": "logistic",
         "lists": False, "smoothing": 0.1, "reference": True, "length_mean": False, "padded": 0.25},
        # packed answers, each in several pairs
        {"name": "preference_packed", "kind": "preference", "sequences": 768, "length": 1365, "ragged": True,
         "loss": "logistic", "lists": True, "smoothing": 0.0, "reference": True, "length_mean": False, "padded": 0.1},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["heads", "heads_bwd", "heads_bwd", "logprobs", "logprobs", "logprobs_bwd", "logprobs_bwd",
                       "policy", "preference"])
    if kind in ("heads", "heads_bwd"):
        dim = rng.choice([64, 64, 80, 96, 128, 128, 192, 256])
        k = rng.choice([1, 2, 4, 8])
        q = k * rng.choice([1, 2, 3, 5, 7, 8])
        case = {"kind": kind, "q": q, "k": k, "dim": dim, "rotated": rng.choice([dim, dim, 16 * rng.randint(1, dim // 16)]),
                "tokens": min(_log(rng, 1, 16384), LARGEST_HEADS // ((q + k) * dim)),
                "pairs": rng.random() < 0.3, "norm": rng.random() < 0.7, "head_major": rng.random() < 0.4,
                "start": rng.choice([0, 0, 5000, 200000])}
        if kind == "heads":
            return case
        code = rng.choice(["none", "none", "int8", "e4m3fn", "e4m3fn_cast"]) if case["norm"] else "none"
        block = 0 if code in ("none", "e4m3fn_cast") else 32
        if block and dim % 32:
            block, code = 0, "none"
        if block and (k * dim) % 64 == 0 and rng.random() < 0.5:
            block = 64
        return dict(case, code=code, block=block, weights=case["norm"] and rng.random() < 0.6)
    if kind in ("logprobs", "logprobs_bwd"):
        vocab = rng.choice([32000, 65536, 131072, _log(rng, 500, 262144), _log(rng, 500, 262144)])
        return {"kind": kind, "vocab": vocab, "rows": max(1, min(_log(rng, 1, 16384), LARGEST_LOGITS // 4 // vocab)),
                "pad": rng.choice([0, 0, 0, 1, 24]), "f32": rng.random() < 0.3, "entropy": rng.random() < 0.5,
                "scale": rng.choice([1.0, 1.0, 0.7, 1.25]), "idle": rng.choice([0.0, 0.2, 0.4])}
    length = _log(rng, 4, 8192)
    sequences = max(2, min(_log(rng, 2, 4096), LARGEST_TOKENS // length))
    case = {"kind": kind, "sequences": sequences, "length": length, "ragged": rng.random() < 0.5,
            "padded": rng.choice([0.0, 0.1, 0.3])}
    if kind == "policy":
        kl = rng.choice([0, 1, 2, 3])
        return dict(case, ratio=rng.choice(["token", "token", "sequence"]), kl=kl, beta=1e-2 if kl else 0.0,
                    mean=rng.choice(["tokens", "sequences"]), high=rng.choice([0.2, 0.28]), dual=rng.choice([0.0, 3.0]),
                    bonus=rng.choice([0.0, 1e-3]))
    case["sequences"] -= case["sequences"] % 2
    loss = rng.choice(["logistic", "logistic", "hinge", "squared"])
    return dict(case, loss=loss, lists=rng.random() < 0.5, smoothing=rng.choice([0.0, 0.1]) if loss == "logistic" else 0.0,
                reference=rng.random() < 0.7, length_mean=loss == "squared")


# ------------------------------------------------------------------ inputs --
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _normal(g, shape, sigma=1.0, dtype=torch.float32):
    return torch.randn(shape, generator=g, device=DEV).mul_(sigma).to(dtype)


def _uniform(g, shape):
    return torch.rand(shape, generator=g, device=DEV)


def prepare(case, seed):
    g = _gen(seed)
    return {"heads": _prepare_heads, "heads_bwd": _prepare_heads, "logprobs": _prepare_logprobs,
            "logprobs_bwd": _prepare_logprobs, "policy": _prepare_policy, "preference": _prepare_preference}[case["kind"]](case, g)


def _block_codes(x, code, block):
    """(codes, scales) of a saved bf16 tensor: block absmax int8 or E4M3FN, or the plain cast."""
    if code == "e4m3fn_cast":
        return x.to(torch.float8_e4m3fn).view(torch.uint8), None
    q = 127.0 if code == "int8" else 448.0
    b = x.float().reshape(x.shape[0], -1, block)
    amax = b.abs().amax(2, keepdim=True)
    v = (b * torch.where(amax < TINY, 0.0, q / amax)).clamp_(-q, q)
    codes = v.round_().to(torch.int8).view(torch.uint8) if code == "int8" else v.to(torch.float8_e4m3fn).view(torch.uint8)
    return codes.reshape(x.shape), (amax.squeeze(2) / q).contiguous()


def _heads_out(case, heads):
    """An output [tokens, heads, dim], token by token or head by head in memory."""
    t, d = case["tokens"], case["dim"]
    if case["head_major"]:
        return torch.empty((heads, t, d), dtype=torch.bfloat16, device=DEV).transpose(0, 1)
    return torch.empty((t, heads, d), dtype=torch.bfloat16, device=DEV)


def _prepare_heads(case, g):
    t, q, k, d = case["tokens"], case["q"], case["k"], case["dim"]
    back = case["kind"] == "heads_bwd"
    # the projection's rows hold the queries, keys and values side by side
    rows = torch.randn((t, (q + 2 * k) * d), generator=g, device=DEV)
    rows[:, torch.randperm(rows.shape[1], generator=g, device=DEV)[:max(1, rows.shape[1] // 200)]] *= 10.0
    rows = rows.to(torch.bfloat16)
    st = {"kind": case["kind"], "case": dict(case), "rows": rows, "q": rows[:, :q * d], "k": rows[:, q * d:(q + k) * d]}
    for name in ("w_q", "w_k"):
        st[name] = (1.0 + _normal(g, d, 0.1)).to(torch.bfloat16) if case["norm"] else None
    # packed sequences: positions start again; a token of a step stands anywhere behind `start`
    step = torch.randint(1, 1500, (max(1, t // 256),), generator=g, device=DEV)
    if t < 256:
        pos = torch.randint(0, 4096, (t,), generator=g, device=DEV)
    else:
        pos = torch.arange(t, device=DEV) % (t // 8 + 1) + step.repeat_interleave(-(-t // step.numel()))[:t]
    st["positions"] = pos + case["start"]
    half = case["rotated"] // 2
    st["inv_freq"] = (10000.0 ** (-torch.arange(half, device=DEV, dtype=torch.float64) / half)).float()
    if not back:
        st["q_out"], st["k_out"] = _heads_out(case, q), _heads_out(case, k)
        return st
    for name, heads in (("q", q), ("k", k)):
        grad = _heads_out(case, heads)
        grad.copy_(_normal(g, (t, heads, d), 1e-3))
        st["d" + name] = grad
        st[name + "_codes"], st[name + "_scales"] = (None, None) if case["code"] == "none" else \
            _block_codes(st[name].contiguous(), case["code"], case["block"])
        st["dw_" + name] = torch.empty(d, device=DEV) if case["weights"] else None
    st["drows"] = torch.zeros_like(rows)
    st["dq_in"], st["dk_in"] = st["drows"][:, :q * d], st["drows"][:, q * d:(q + k) * d]
    return st


def _idle(case):
    return int(case["idle"] * case["rows"])


def _prepare_logprobs(case, g):
    rows, vocab = case["rows"], case["vocab"]
    # a few tokens of each row stand out, and the chosen one is drawn from the row's distribution
    z = torch.randn((rows, vocab + case["pad"]), generator=g, device=DEV).mul_(1.5)
    likely = torch.randint(0, vocab, (rows, 8), generator=g, device=DEV)
    z.scatter_add_(1, likely, 14.0 * _uniform(g, (rows, 8)))
    chosen = torch.empty(rows, dtype=torch.int64, device=DEV)
    for a in range(0, rows, 1024):
        noise = _uniform(g, (min(1024, rows - a), vocab)).clamp_(min=1e-30).log_().neg_().log_().neg_()
        chosen[a:a + 1024] = noise.add_(z[a:a + 1024, :vocab], alpha=case["scale"]).argmax(1)
        del noise
    st = {"kind": case["kind"], "scale": case["scale"], "targets": chosen,
          "logits": z.to(torch.float32 if case["f32"] else torch.bfloat16)[:, :vocab]}
    del z
    idle = torch.randperm(rows, generator=g, device=DEV)[:_idle(case)]
    if case["kind"] == "logprobs":
        chosen[idle] = -1
        for name in ("logp", "row_max", "log_sum") + (("entropy",) if case["entropy"] else ()):
            st[name] = torch.empty(rows, device=DEV)
        st.setdefault("entropy", None)
        return st
    # half of the idle rows belong to no response, the others have a zero coefficient
    st["dlogp"] = _normal(g, rows, 1e-4)
    st["dentropy"] = _normal(g, rows, 1e-6) if case["entropy"] else None
    chosen[idle[::2]] = -1
    st["dlogp"][idle] = 0.0
    if case["entropy"]:
        st["dentropy"][idle] = 0.0
    # what the forward has left
    st["row_max"], st["log_sum"] = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
    st["entropy"] = torch.empty(rows, device=DEV) if case["entropy"] else None
    for a in range(0, rows, 1024):
        x = st["logits"][a:a + 1024].float()
        m = x.amax(1)
        d = x.sub_(m[:, None]).mul_(case["scale"])
        e = d.exp()
        s = e.sum(1)
        st["row_max"][a:a + 1024], st["log_sum"][a:a + 1024] = m, s.log()
        if case["entropy"]:
            st["entropy"][a:a + 1024] = s.log() - e.mul_(d).sum(1) / s
    st["dlogits"] = torch.empty((rows, vocab), dtype=st["logits"].dtype, device=DEV)
    return st


def _prepare_sequences(case, g):
    """Tokens in rows of equal length with padding, or packed with the sequences' offsets."""
    s, length = case["sequences"], case["length"]
    if case["ragged"]:
        lengths = torch.randint(1, 2 * length, (s,), generator=g, device=DEV)
        offsets = torch.zeros(s + 1, dtype=torch.int64, device=DEV)
        offsets[1:] = lengths.cumsum(0)
        offsets = (offsets * (s * length) // offsets[-1]).to(torch.int64)
        n = s * length
        mask = _uniform(g, n) >= case["padded"]
    else:
        n, offsets = s * length, None
        kept = (length * (1.0 - 2.0 * case["padded"] * _uniform(g, s))).ceil().clamp(min=1.0)
        mask = (torch.arange(length, device=DEV)[None, :] < kept[:, None]).reshape(-1)
    old = -(_normal(g, n, 1.0) - 1.0).abs() - 1e-3
    return {"kind": case["kind"], "case": dict(case), "tokens": n, "offsets": offsets, "mask": mask.to(torch.uint8), "old": old}


def _prepare_policy(case, g):
    st = _prepare_sequences(case, g)
    n, s = st["tokens"], case["sequences"]
    st["logp_old"] = st.pop("old")
    drift = 0.1 if case["ratio"] == "token" else 0.3
    st["logp"] = st["logp_old"] + _normal(g, n, drift)
    st["logp_ref"] = st["logp_old"] + _normal(g, n, 0.05) if case["kl"] else None
    st["entropy"] = _uniform(g, n) * 3.0 if case["bonus"] else None
    st["adv"] = torch.where(_uniform(g, s) < 0.1, 0.0, _normal(g, s))  # groups of equal rewards have none
    st["dlogp"], st["token_loss"] = torch.zeros(n, device=DEV), torch.zeros(n, device=DEV)
    st["dentropy"] = torch.zeros(n, device=DEV) if case["bonus"] else None
    st["flags"] = torch.zeros(n, dtype=torch.uint8, device=DEV) if case["ratio"] == "token" else None
    st["stats"] = torch.empty(8, device=DEV)
    return st


def _prepare_preference(case, g):
    st = _prepare_sequences(case, g)
    n, s = st["tokens"], case["sequences"]
    st["logp_ref"] = st.pop("old")
    st["logp"] = st["logp_ref"] + _normal(g, n, 0.05)
    if not case["reference"]:
        st["logp_ref"] = None
    st["chosen"] = st["rejected"] = None
    if case["lists"]:  # answers in groups of four, the pairs of each group
        first = torch.arange(s // 4 * 4, device=DEV).reshape(-1, 4) if s >= 4 else torch.arange(2, device=DEV).repeat(2)[None, :]
        a, b = zip(*[(i, j) for i in range(4) for j in range(i + 1, 4)])
        st["chosen"] = first[:, list(a)].reshape(-1).to(torch.int32).contiguous()
        st["rejected"] = first[:, list(b)].reshape(-1).to(torch.int32).contiguous()
    pairs = st["chosen"].numel() if case["lists"] else s // 2
    st["dlogp"] = torch.zeros(n, device=DEV)
    st["rewards"], st["pair_loss"], st["stats"] = torch.empty(s, device=DEV), torch.empty(pairs, device=DEV), torch.empty(6, device=DEV)
    return st


# -------------------------------------------------------------------- work --
def work(case):
    kind = case["kind"]
    if kind in ("heads", "heads_bwd"):
        n = float(case["tokens"] * (case["q"] + case["k"]) * case["dim"])
        small = 8.0 * case["tokens"] + 2.0 * case["rotated"] + (4.0 * case["dim"] if case["norm"] else 0.0)
        if kind == "heads":
            return {"bytes": 4.0 * n + small, "flops": 12.0 * n}
        saved = 0.0 if not case["norm"] else 2.0 if case["code"] == "none" else 1.0 + (4.0 / case["block"] if case["block"] else 0.0)
        return {"bytes": (4.0 + saved) * n + small + (8.0 * case["dim"] if case["weights"] else 0.0), "flops": 24.0 * n}
    if kind in ("logprobs", "logprobs_bwd"):
        rows, vocab, size = case["rows"], case["vocab"], 4.0 if case["f32"] else 2.0
        live = rows - _idle(case)
        if kind == "logprobs":
            return {"bytes": size * live * vocab + (24.0 if case["entropy"] else 20.0) * rows, "flops": 6.0 * live * vocab}
        return {"bytes": size * (live + rows) * vocab + (28.0 if case["entropy"] else 20.0) * rows, "flops": 8.0 * live * vocab}
    n, s = float(case["sequences"] * case["length"]), float(case["sequences"])
    offsets = 8.0 * (s + 1) if case["ragged"] else 0.0
    if kind == "policy":
        token = 9.0 + (4.0 if case["kl"] else 0.0) + 8.0 + (8.0 if case["bonus"] else 0.0) + (1.0 if case["ratio"] == "token" else 0.0)
        return {"bytes": token * n + 4.0 * s + offsets + 32.0, "flops": 25.0 * n}
    pairs = s // 4 * 6 if case["lists"] else s // 2
    return {"bytes": (5.0 + (4.0 if case["reference"] else 0.0) + 4.0) * n + 4.0 * s + offsets + pairs * (12.0 if case["lists"] else 4.0) + 24.0,
            "flops": 4.0 * n}


# --------------------------------------------------------------------- run --
def run(state):
    kind = state["kind"]
    if own:
        return {"heads": _own_heads, "heads_bwd": _own_heads_bwd, "logprobs": _own_logprobs, "logprobs_bwd": _own_logprobs_bwd,
                "policy": _own_policy, "preference": _own_preference}[kind](state)
    return {"heads": _plain_heads, "heads_bwd": _plain_heads_bwd, "logprobs": _plain_logprobs,
            "logprobs_bwd": _plain_logprobs_bwd, "policy": _plain_policy, "preference": _plain_preference}[kind](state)


BETA = 0.1                                   # of the preference loss
CLIP_LOW = 0.2


def _outputs(st, *names):
    return {k: st[k] for k in names if st[k] is not None}


# the package's calls; descriptors and workspaces are made once, as a trainer keeps them
def _own_heads(st):
    from paper_2609_33570_amd import hilore as hl

    if "desc" not in st:
        c = st["case"]
        st["desc"] = hl.qk_norm_rope_desc(q=st["q"], k=st["k"], q_out=st["q_out"], k_out=st["k_out"], inv_freq=st["inv_freq"],
                                          positions=st["positions"], w_q=st["w_q"], w_k=st["w_k"], eps=EPS,
                                          rotation="pairs" if c["pairs"] else "halves")
    hl.hilore_qk_norm_rope(st["desc"])
    return _outputs(st, "q_out", "k_out")


def _own_heads_bwd(st):
    from paper_2609_33570_amd import hilore as hl

    c = st["case"]
    if "desc" not in st:
        saved = {n: None if not c["norm"] else hl.unit_desc(x=st[n] if c["code"] == "none" else None, codes=st[n + "_codes"],
                                                            scales=st[n + "_scales"]) for n in ("q", "k")}
        st["desc"] = hl.qk_norm_rope_bwd_desc(dq=st["dq"], dk=st["dk"], dq_in=st["dq_in"], dk_in=st["dk_in"], q=saved["q"], k=saved["k"],
                                              inv_freq=st["inv_freq"], positions=st["positions"], w_q=st["w_q"], w_k=st["w_k"],
                                              dw_q=st["dw_q"], dw_k=st["dw_k"], eps=EPS,
                                              rotation="pairs" if c["pairs"] else "halves")
        st["workspace"] = torch.empty(hl.hilore_qk_norm_rope_bwd_workspace_bytes(st["desc"]), dtype=torch.uint8, device=DEV)
    hl.hilore_qk_norm_rope_bwd(st["desc"], 0 if c["code"] == "none" else c["code"], c["block"], workspace=st["workspace"])
    return _outputs(st, "dq_in", "dk_in", "dw_q", "dw_k")


def _own_logprobs(st):
    from paper_2609_33570_amd import hilore as hl

    if "desc" not in st:
        st["desc"] = hl.token_logprobs_desc(logits=st["logits"], targets=st["targets"], logp=st["logp"], entropy=st["entropy"],
                                            row_max=st["row_max"], log_sum=st["log_sum"], scale=st["scale"])
        st["workspace"] = torch.empty(hl.hilore_token_logprobs_workspace_bytes(st["desc"]), dtype=torch.uint8, device=DEV)
    hl.hilore_token_logprobs(st["desc"], workspace=st["workspace"])
    return _outputs(st, "logp", "entropy", "row_max", "log_sum")


def _own_logprobs_bwd(st):
    from paper_2609_33570_amd import hilore as hl

    if "desc" not in st:
        st["desc"] = hl.token_logprobs_bwd_desc(logits=st["logits"], targets=st["targets"], row_max=st["row_max"],
                                                log_sum=st["log_sum"], entropy=st["entropy"], dlogp=st["dlogp"],
                                                dentropy=st["dentropy"], dlogits=st["dlogits"], scale=st["scale"])
    hl.hilore_token_logprobs_bwd(st["desc"])
    return st["dlogits"]


def _own_policy(st):
    from paper_2609_33570_amd import hilore as hl

    if "desc" not in st:
        c = st["case"]
        st["desc"] = hl.policy_loss_desc(logp=st["logp"], logp_old=st["logp_old"], logp_ref=st["logp_ref"], entropy=st["entropy"],
                                         adv=st["adv"], mask=st["mask"], offsets=st["offsets"], sequences=c["sequences"],
                                         clip_low=CLIP_LOW, clip_high=c["high"], dual_clip=c["dual"], beta=c["beta"],
                                         entropy_weight=c["bonus"], kl=c["kl"], ratio=c["ratio"], mean=c["mean"],
                                         dlogp=st["dlogp"], dentropy=st["dentropy"], token_loss=st["token_loss"],
                                         flags=st["flags"], stats=st["stats"])
        st["workspace"] = torch.empty(hl.hilore_policy_loss_workspace_bytes(st["desc"]), dtype=torch.uint8, device=DEV)
    hl.hilore_policy_loss(st["desc"], workspace=st["workspace"])
    return _outputs(st, "dlogp", "dentropy", "token_loss", "flags", "stats")


def _own_preference(st):
    from paper_2609_33570_amd import hilore as hl

    if "desc" not in st:
        c = st["case"]
        st["desc"] = hl.preference_loss_desc(logp=st["logp"], logp_ref=st["logp_ref"], mask=st["mask"], offsets=st["offsets"],
                                             sequences=c["sequences"], chosen=st["chosen"], rejected=st["rejected"], beta=BETA,
                                             label_smoothing=c["smoothing"], loss=c["loss"], length_mean=c["length_mean"],
                                             dlogp=st["dlogp"], rewards=st["rewards"], pair_loss=st["pair_loss"], stats=st["stats"])
        st["workspace"] = torch.empty(hl.hilore_preference_loss_workspace_bytes(st["desc"]), dtype=torch.uint8, device=DEV)
    hl.hilore_preference_loss(st["desc"], workspace=st["workspace"])
    return _outputs(st, "dlogp", "rewards", "pair_loss", "stats")


# the plain forms
def _plain_angles(st):
    a = st["positions"].double()[:, None] * st["inv_freq"].double()
    return a.cos().float()[:, None, :], a.sin().float()[:, None, :]


def _plain_rotate(x, cos, sin, pairs):
    """[tokens, heads, dim] with the first columns turned."""
    half = cos.shape[2]
    rest = x[..., 2 * half:]
    if pairs:
        a, b = x[..., 0:2 * half:2], x[..., 1:2 * half:2]
        turned = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    else:
        a, b = x[..., :half], x[..., half:2 * half]
        turned = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    return torch.cat((turned, rest), -1)


def _plain_heads(st):
    cos, sin = _plain_angles(st)
    for name in ("q", "k"):
        out = st[name + "_out"]
        x = st[name].float().reshape(out.shape)
        if st["w_" + name] is not None:
            x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * st["w_" + name].float()
        out.copy_(_plain_rotate(x, cos, sin, st["case"]["pairs"]))
    return _outputs(st, "q_out", "k_out")


def _plain_saved(st, name):
    """The saved rows in 32 bits: as they are, or the bf16 values that their codes stand for."""
    codes, scales = st[name + "_codes"], st[name + "_scales"]
    if codes is None:
        return st[name].float()
    v = codes.view(torch.int8 if st["case"]["code"] == "int8" else torch.float8_e4m3fn).float()
    if scales is not None:
        v = (v.reshape(v.shape[0], -1, st["case"]["block"]) * scales[:, :, None]).reshape(v.shape)
    return v.to(torch.bfloat16).float()


def _plain_heads_bwd(st):
    cos, sin = _plain_angles(st)
    for name in ("q", "k"):
        g = st["d" + name]
        dn = _plain_rotate(g.float(), cos, -sin, st["case"]["pairs"])
        if st["w_" + name] is not None:
            u = _plain_saved(st, name).reshape(g.shape)
            r = torch.rsqrt(u.square().mean(-1, keepdim=True) + EPS)
            u = u * r
            if st["dw_" + name] is not None:
                st["dw_" + name].copy_((dn * u).sum((0, 1)))
            dn = dn * st["w_" + name].float()
            dn = r * (dn - u * (dn * u).mean(-1, keepdim=True))
        st[f"d{name}_in"].copy_(dn.reshape(g.shape[0], -1))
    return _outputs(st, "dq_in", "dk_in", "dw_q", "dw_k")


def _plain_logprobs(st):
    live = st["targets"] >= 0
    z = st["logits"].float()
    m = z.amax(1)
    d = z.sub_(m[:, None]).mul_(st["scale"]) if z.data_ptr() != st["logits"].data_ptr() else (z - m[:, None]) * st["scale"]
    chosen = d.gather(1, st["targets"].clamp(min=0)[:, None])[:, 0]
    e = d.exp()
    s = e.sum(1)
    lsum = s.log()
    st["row_max"].copy_(torch.where(live, m, 0.0)), st["log_sum"].copy_(torch.where(live, lsum, 0.0))
    st["logp"].copy_(torch.where(live, chosen - lsum, 0.0))
    if st["entropy"] is not None:
        st["entropy"].copy_(torch.where(live, lsum - e.mul_(d).sum(1) / s, 0.0))
    return _outputs(st, "logp", "entropy", "row_max", "log_sum")


def _plain_logprobs_bwd(st):
    live = st["targets"] >= 0
    g = torch.where(live, st["dlogp"], 0.0)[:, None]
    d = (st["logits"].float() - st["row_max"][:, None]) * st["scale"] - st["log_sum"][:, None]
    p = d.exp()
    if st["dentropy"] is not None:
        e = torch.where(live, st["dentropy"], 0.0)[:, None]
        out = p * -(g + e * (d + st["entropy"][:, None]))
    else:
        out = p * -g
    out.scatter_add_(1, st["targets"].clamp(min=0)[:, None], g)
    st["dlogits"].copy_(out.mul_(st["scale"]))
    return st["dlogits"]


def _sequence_of_token(st):
    n, s = st["tokens"], st["case"]["sequences"]
    if st["offsets"] is None:
        return torch.arange(n, device=DEV) // (n // s)
    return torch.bucketize(torch.arange(n, device=DEV), st["offsets"][1:], right=True)


def _sums(x, seq, s):
    """Sums over the tokens of each sequence, in 64 bits, as fp32."""
    return torch.zeros(s, dtype=torch.float64, device=DEV).index_add_(0, seq, x.double()).float()


def _plain_policy(st):
    c, valid, s = st["case"], st["mask"] != 0, st["case"]["sequences"]
    seq = _sequence_of_token(st)
    count = _sums(valid, seq, s)
    delta = torch.where(valid, st["logp"] - st["logp_old"], 0.0)
    if c["ratio"] == "sequence":
        mean = _sums(delta, seq, s) / count.clamp(min=1.0)
        delta = mean[seq]
    ratio, adv = delta.exp(), st["adv"][seq]
    # the ratio's side of the clip, in log space
    over = delta > torch.tensor(math.log1p(c["high"]), dtype=torch.float32, device=DEV)
    under = delta < torch.tensor(math.log1p(-CLIP_LOW), dtype=torch.float32, device=DEV)
    outside = torch.where(adv >= 0, over, under)
    bound = torch.where(adv >= 0, 1.0 + c["high"], 1.0 - CLIP_LOW)
    if c["dual"]:
        past = (adv < 0) & (delta > torch.tensor(math.log(c["dual"]), dtype=torch.float32, device=DEV))
        outside, bound = outside | past, torch.where(past, c["dual"], bound)
    clipped = outside & (adv != 0)
    loss = -adv * torch.where(clipped, bound, ratio)
    grad = torch.where(clipped, 0.0, -adv * ratio)
    if c["mean"] == "tokens":
        weight = torch.where(valid, 1.0 / count.sum().clamp(min=1.0), 0.0)
    else:
        weight = torch.where(valid, 1.0 / ((count > 0).sum() * count[seq].clamp(min=1.0)), 0.0)
    if c["ratio"] == "sequence":  # every token of a sequence moves its ratio
        grad = _sums(grad * weight, seq, s)[seq] / count[seq].clamp(min=1.0)
        grad = torch.where(valid, grad, 0.0)
    else:
        grad = grad * weight
    policy = loss
    kl = torch.zeros_like(loss)
    if c["kl"]:
        x = st["logp"] - st["logp_ref"]
        if c["kl"] == 1:
            kl, slope = x, torch.ones_like(x)
        elif c["kl"] == 2:
            kl, slope = 0.5 * x * x, x
        else:
            kl, slope = torch.expm1(-x) + x, -torch.expm1(-x)
        loss = loss + c["beta"] * kl
        grad = grad + weight * c["beta"] * slope
    if st["entropy"] is not None:
        loss = loss - c["bonus"] * st["entropy"]
        st["dentropy"].copy_(-c["bonus"] * weight)
    st["token_loss"].copy_(torch.where(valid, loss * weight, 0.0))
    st["dlogp"].copy_(torch.where(valid, grad, 0.0))
    if st["flags"] is not None:
        st["flags"].copy_((valid & ~outside).to(torch.uint8) + 2 * (valid & clipped).to(torch.uint8))

    def total(x):
        return torch.where(valid, x.double(), 0.0).sum()

    tokens = count.sum()
    entropy = total(weight * st["entropy"]) if st["entropy"] is not None else 0.0
    for i, v in enumerate((total(loss * weight), total(policy * weight), total(kl * weight), entropy,
                           total(clipped) / tokens.clamp(min=1.0), total(ratio) / tokens.clamp(min=1.0), tokens, (count > 0).sum())):
        st["stats"][i] = v
    return _outputs(st, "dlogp", "dentropy", "token_loss", "flags", "stats")


def _pair_lists(st):
    if st["chosen"] is not None:
        return st["chosen"].long(), st["rejected"].long()
    first = torch.arange(0, st["case"]["sequences"], 2, device=DEV)
    return first, first + 1


def _plain_preference(st):
    c, valid, s = st["case"], st["mask"] != 0, st["case"]["sequences"]
    seq = _sequence_of_token(st)
    count = _sums(valid, seq, s)
    x = st["logp"] if st["logp_ref"] is None else st["logp"] - st["logp_ref"]
    value = torch.zeros(s, dtype=torch.float64, device=DEV).index_add_(0, seq, torch.where(valid, x, 0.0).double())
    if c["length_mean"]:
        value = value / count.clamp(min=1.0)
    win, lose = _pair_lists(st)
    used = ((count[win] > 0) & (count[lose] > 0)).float()
    h = (value[win] - value[lose]).float()
    y = BETA * h
    if c["loss"] == "logistic":
        eps, tail = c["smoothing"], torch.log1p(torch.exp(-y.abs()))
        loss = (1.0 - eps) * ((-y).clamp(min=0.0) + tail) + eps * (y.clamp(min=0.0) + tail)
        slope = BETA * (eps / (1.0 + torch.exp(-y)) - (1.0 - eps) / (1.0 + torch.exp(y)))
    elif c["loss"] == "hinge":
        loss, slope = (1.0 - y).clamp(min=0.0), torch.where(y < 1.0, -BETA, 0.0)
    else:
        loss, slope = (h - 0.5 / BETA).square(), 2.0 * (h - 0.5 / BETA)
    norm = used.sum().clamp(min=1.0)
    slope = slope * used / norm
    by_sequence = torch.zeros(s, dtype=torch.float64, device=DEV).index_add_(0, win, slope.double()).index_add_(0, lose, -slope.double())
    if c["length_mean"]:
        by_sequence = by_sequence / count.clamp(min=1.0)
    st["dlogp"].copy_(torch.where(valid, by_sequence.float()[seq], 0.0))
    rewards = BETA * value
    st["rewards"].copy_(rewards)
    st["pair_loss"].copy_(loss * used)

    def mean(x):
        return (x.double() * used).sum() / norm

    for i, v in enumerate((mean(loss), mean(h > 0), mean(y), mean(rewards[win]), mean(rewards[lose]), used.sum())):
        st["stats"][i] = v
    return _outputs(st, "dlogp", "rewards", "pair_loss", "stats")


# ------------------------------------------------------------------- exact --
def exact(case, seed):
    st = prepare(case, seed)
    return {"heads": _exact_heads, "heads_bwd": _exact_heads_bwd, "logprobs": _exact_logprobs,
            "logprobs_bwd": _exact_logprobs_bwd, "policy": _exact_policy, "preference": _exact_preference}[case["kind"]](st)


def _exact_turn(st, x, sign):
    """x as complex numbers times e^(+-i angle)."""
    angle = torch.outer(st["positions"].double(), st["inv_freq"].double())
    turn = torch.polar(torch.ones_like(angle), sign * angle).unsqueeze(1)
    n = angle.shape[1]
    out = x.clone()
    if st["case"]["pairs"]:
        z = torch.complex(x[:, :, 0:2 * n:2], x[:, :, 1:2 * n:2]) * turn
        out[:, :, 0:2 * n:2], out[:, :, 1:2 * n:2] = z.real, z.imag
    else:
        z = torch.complex(x[:, :, :n], x[:, :, n:2 * n]) * turn
        out[:, :, :n], out[:, :, n:2 * n] = z.real, z.imag
    return out


def _exact_heads(st):
    out = {}
    for name in ("q", "k"):
        shape = st[name + "_out"].shape
        x = st[name].double().reshape(shape)
        if st["w_" + name] is not None:
            x = x * st["w_" + name].double() / torch.sqrt(torch.linalg.vecdot(x, x)[..., None] / shape[2] + EPS)
        out[name + "_out"] = _exact_turn(st, x, 1.0)
    return out


def _exact_heads_bwd(st):
    out, c = {}, st["case"]
    for name in ("q", "k"):
        g = _exact_turn(st, st["d" + name].double(), -1.0)
        t, heads, dim = g.shape
        if st["w_" + name] is not None:
            if st[name + "_codes"] is None:
                u = st[name].double()
            else:
                u = st[name + "_codes"].view(torch.int8 if c["code"] == "int8" else torch.float8_e4m3fn).float()
                if st[name + "_scales"] is not None:  # the saved value is the product rounded to bf16
                    u = u * st[name + "_scales"].repeat_interleave(c["block"], dim=1)
                u = u.to(torch.bfloat16).double()
            u = u.reshape(t, heads, dim)
            length = torch.sqrt(torch.linalg.vecdot(u, u)[..., None] / dim + EPS)
            if st["dw_" + name] is not None:
                out["dw_" + name] = torch.einsum("thd,thd->d", g, u / length)
            weighted = g * st["w_" + name].double()
            along = torch.linalg.vecdot(weighted, u)[..., None] / (dim * length ** 3)
            g = weighted / length - u * along
        out[f"d{name}_in"] = g.reshape(t, heads * dim)
    return {k: out[k] for k in ("dq_in", "dk_in", "dw_q", "dw_k") if k in out}


def _exact_logprobs(st):
    out = {k: torch.zeros_like(v, dtype=torch.float64) for k, v in _outputs(st, "logp", "entropy", "row_max", "log_sum").items()}
    for a in range(0, st["targets"].numel(), 512):
        z, t = st["logits"][a:a + 512].double(), st["targets"][a:a + 512]
        live = t >= 0
        logp = torch.log_softmax(z * st["scale"], 1)
        top = z.max(1).values
        out["row_max"][a:a + 512] = top * live
        out["log_sum"][a:a + 512] = (torch.logsumexp(z * st["scale"], 1) - st["scale"] * top) * live
        out["logp"][a:a + 512] = logp[torch.arange(t.numel(), device=DEV), t.clamp(min=0)] * live
        if "entropy" in out:
            out["entropy"][a:a + 512] = -(logp.exp() * logp).sum(1) * live
    return out


def _exact_logprobs_bwd(st):
    out = torch.empty(st["dlogits"].shape, dtype=torch.float64, device=DEV)
    for a in range(0, st["targets"].numel(), 512):
        z, t = st["logits"][a:a + 512].double() * st["scale"], st["targets"][a:a + 512]
        live = (t >= 0).double()
        logp = z - (st["row_max"][a:a + 512].double() * st["scale"] + st["log_sum"][a:a + 512].double())[:, None]
        p = logp.exp()
        g = st["dlogp"][a:a + 512].double() * live
        grad = -g[:, None] * p
        grad[torch.arange(t.numel(), device=DEV), t.clamp(min=0)] += g
        if st["dentropy"] is not None:
            e = st["dentropy"][a:a + 512].double() * live
            grad -= e[:, None] * p * (logp + st["entropy"][a:a + 512].double()[:, None])
        out[a:a + 512] = grad * st["scale"]
    return out


def _exact_bounds(st):
    """First and last token of every sequence."""
    s = st["case"]["sequences"]
    if st["offsets"] is None:
        step = st["tokens"] // s
        return torch.arange(s, device=DEV) * step, (torch.arange(s, device=DEV) + 1) * step
    return st["offsets"][:-1], st["offsets"][1:]


def _exact_sums(x, begin, end):
    """Sums over each sequence as differences of a running sum of whole steps of 2^-40 (no rounding between them)."""
    run = torch.zeros(x.numel() + 1, dtype=torch.int64, device=DEV)
    run[1:] = torch.round(x.double() * 2.0 ** 40).to(torch.int64).cumsum(0)
    return (run[end] - run[begin]).double() * 2.0 ** -40


def _exact_policy(st):
    c, valid = st["case"], st["mask"].bool()
    begin, end = _exact_bounds(st)
    lengths = end - begin
    count = _exact_sums(valid, begin, end)

    def spread(x):  # a value of each sequence at its tokens
        return x.repeat_interleave(lengths)

    # a token's log ratio is an fp32 difference, by the definition of the clip
    delta = (st["logp"] - st["logp_old"]).double() * valid
    if c["ratio"] == "sequence":
        delta = spread(_exact_sums(delta, begin, end) / count.clamp(min=1))
    a, r = spread(st["adv"].double()), delta.exp()
    lo, hi = (float(torch.tensor(math.log1p(v), dtype=torch.float32)) for v in (-CLIP_LOW, c["high"]))
    inside = ((a >= 0) & (delta <= hi)) | ((a < 0) & (delta >= lo))
    kept = torch.where(inside, r, torch.where(a >= 0, 1.0 + c["high"], 1.0 - CLIP_LOW))
    if c["dual"]:
        past = (a < 0) & (delta > float(torch.tensor(math.log(c["dual"]), dtype=torch.float32)))
        inside, kept = inside & ~past, torch.where(past, c["dual"], kept)
    clipped = ~inside & (a != 0)
    filled = count > 0
    w = valid / valid.sum().clamp(min=1) if c["mean"] == "tokens" else valid / spread(count.clamp(min=1) * filled.sum())
    policy, dlogp = -a * kept, torch.where(clipped, 0.0, -a * r)
    if c["ratio"] == "sequence":
        # every token of a sequence has the same factor: the sum of weights times it, over the count
        share = spread(count / count.clamp(min=1)) / valid.sum() if c["mean"] == "tokens" else spread(1.0 / count.clamp(min=1)) / filled.sum()
        dlogp = dlogp * share * valid
    else:
        dlogp = dlogp * w
    kl = torch.zeros_like(policy)
    if c["kl"]:
        x = st["logp"].double() - st["logp_ref"].double()
        kl = {1: x, 2: x ** 2 / 2, 3: torch.expm1(-x) + x}[c["kl"]]
        dlogp = dlogp + c["beta"] * w * {1: torch.ones_like(x), 2: x, 3: -torch.expm1(-x)}[c["kl"]]
    h = torch.zeros_like(policy) if st["entropy"] is None else st["entropy"].double()
    loss = w * (policy + c["beta"] * kl - c["bonus"] * h)
    n = valid.sum()
    out = {"dlogp": dlogp, "dentropy": -c["bonus"] * w, "token_loss": loss,
           "flags": ((valid & inside) + 2 * (valid & clipped).long()).to(torch.uint8),
           "stats": torch.stack([loss.sum(), (w * policy).sum(), (w * kl).sum(), (w * h).sum(),
                                 (clipped & valid).sum() / n.clamp(min=1).double(), (r * valid).sum() / n.clamp(min=1),
                                 n.double(), filled.sum().double()])}
    return {k: v for k, v in out.items() if st[k] is not None}


def _exact_preference(st):
    c, valid = st["case"], st["mask"].bool()
    begin, end = _exact_bounds(st)
    count = _exact_sums(valid, begin, end)
    x = st["logp"].double() - (0.0 if st["logp_ref"] is None else st["logp_ref"].double())
    value = _exact_sums(x * valid, begin, end)
    if c["length_mean"]:
        value = value / count.clamp(min=1)
    win, lose = _pair_lists(st)
    used = ((count > 0)[win] & (count > 0)[lose]).double()
    value.requires_grad_()
    h = value[win] - value[lose]
    if c["loss"] == "logistic":
        loss = -(1.0 - c["smoothing"]) * torch.nn.functional.logsigmoid(BETA * h) - c["smoothing"] * torch.nn.functional.logsigmoid(-BETA * h)
    elif c["loss"] == "hinge":
        loss = torch.relu(1.0 - BETA * h)
    else:
        loss = (h - 0.5 / BETA) ** 2
    n = used.sum().clamp(min=1)
    total = (loss * used).sum() / n
    grad, = torch.autograd.grad(total, value)
    if c["length_mean"]:
        grad = grad / count.clamp(min=1)
    value, h, loss = value.detach(), h.detach(), loss.detach()
    rewards = BETA * value
    stats = torch.stack([total.detach(), ((h > 0) * used).sum() / n, (BETA * h * used).sum() / n,
                         (rewards[win] * used).sum() / n, (rewards[lose] * used).sum() / n, used.sum()])
    return {"dlogp": grad.repeat_interleave(end - begin) * valid, "rewards": rewards, "pair_loss": loss * used, "stats": stats}
