"""Timed cases of the layer operators: AdamW over many tensors, the norms around a block, int8 products.

An actor update runs them around the calls of cases.py.  A block of the model is entered
and left through RMS norms that are fused with the block's gate and residual scale, the
frozen base weights of the adapter setting are int8 with one scale per output channel,
and when backward has left the gradients behind, their global norm is taken and AdamW
steps every tensor.

run() makes each pass twice over: with ``own`` by the calls of the package's binding, else
in plain torch operations in 32 bits.  prepare() draws what a trainer has in hand at that
point, from the seed alone; exact() evaluates the definitions in 64 bits.

Widths are those of the package's workloads (896, 3584, 4096, 14336, 18944, and the 512-wide
key/value projection that goes with 3584); token counts run from one to a complete
16384-token microbatch.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
EPS = 1e-6                                   # of the norms
BETA1, BETA2, ADAM_EPS, MAX_NORM = 0.9, 0.999, 1e-8, 1.0
RANK = 16                                    # adapter rank
STATE_BLOCK = 256                            # elements per scale of an 8-bit state
TINY = 2.0 ** -64                            # blocks and rows below it have scale 0
LARGEST_ADAMW = 2 * 3584 * 3584 + 2 * 3584 * 512 + 3 * 3584 * 18944   # elements, one layer
LARGEST_NORM = 16384 * 3584                                          # elements
LARGEST_INT8 = 16384 * 3584 * 18944                                  # multiply-adds


# ------------------------------------------------------------------- cases --
def listed():
    return [
        # optimizer of a small model's adapters (two 896-wide layers, rank 16): launches count
        {"name": "adamw_adapters_small", "kind": "adamw", "set": "adapters", "hidden": 896, "kv": 128,
         "mlp": 4864, "layers": 2, "param": "f32", "grad": "f32", "bits": 8},
        # all 392 rank-16 adapters of a 28-layer 3584-wide model, fp32 throughout
        {"name": "adamw_adapters", "kind": "adamw", "set": "adapters", "hidden": 3584, "kv": 512,
         "mlp": 18944, "layers": 28, "param": "f32", "grad": "f32", "bits": 32},
        # full-parameter step of one 3584-wide layer: bf16 weights and gradients, 8-bit states
        {"name": "adamw_layer_8bit", "kind": "adamw", "set": "layer", "hidden": 3584, "kv": 512,
         "mlp": 18944, "layers": 1, "param": "bf16", "grad": "bf16", "bits": 8},
        # fp32 master weights with a bf16 copy, fp32 weight gradients, tensors of odd sizes
        {"name": "adamw_odd_master", "kind": "adamw", "set": "odd", "tensors": 37, "size": 300007,
         "param": "master", "grad": "f32", "bits": 8},
        # leaving a block and entering the next, whole microbatch: both norms, channel gate
        {"name": "norm_microbatch", "kind": "norm", "rows": 16384, "cols": 3584, "post": True,
         "gate": "channel", "scale": 0.5, "pad": 0},
        # its backward with every gradient
        {"name": "norm_bwd_microbatch", "kind": "norm_bwd", "rows": 16384, "cols": 3584, "post": True,
         "gate": "channel", "scale": 0.5, "code": "none", "block": 0, "weights": True, "pad": 0},
        # backward of a plain pre-norm block over ragged tokens, frozen weights, saved stream in L
        {"name": "norm_bwd_ragged_l", "kind": "norm_bwd", "rows": 11987, "cols": 896, "post": False,
         "gate": "none", "scale": 1.0, "code": "e4m3fn", "block": 128, "weights": False, "pad": 0},
        # one token: norm straight to int8 codes, then the query/key/value product with its bias
        {"name": "decode_token_qkv", "kind": "norm_int8", "rows": 1, "cols": 3584, "n": 4608, "post": False,
         "gate": "none", "scale": 1.0, "bias": True, "pad": 0},
        # one step of 64 responses in flight: the down projection
        {"name": "int8_rollout_down", "kind": "int8", "tokens": 64, "k": 18944, "n": 3584, "grad": False,
         "bias": False, "out": "bf16", "pad": 0},
        # a short prompt through the gate projection, odd token count
        {"name": "int8_prompt_gate", "kind": "int8", "tokens": 701, "k": 3584, "n": 18944, "grad": False,
         "bias": False, "out": "bf16", "pad": 0},
        # recompute of the gate projection for a whole microbatch
        {"name": "int8_microbatch_gate", "kind": "int8", "tokens": 16384, "k": 3584, "n": 18944,
         "grad": False, "bias": False, "out": "bf16", "pad": 0},
        # gradient of the hidden state through the output projection, ragged microbatch
        {"name": "int8_grad_o", "kind": "int8", "tokens": 13001, "k": 3584, "n": 3584, "grad": True,
         "bias": False, "out": "bf16", "pad": 8},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, step, lo=256, hi=18944):
    """A feature width: one of the models' or any multiple of `step`."""
    if rng.random() < 0.4:
        w = rng.choice([w for w in (512, 896, 3584, 4096, 4864, 14336, 18944) if lo <= w <= hi])
        if w % step == 0:
            return w
    return max(step, _log(rng, lo, hi) // step * step)


def draw(rng):
    kind = rng.choice(["adamw", "adamw", "norm", "norm_bwd", "norm_bwd", "norm_int8", "int8", "int8", "int8"])
    if kind == "adamw":
        case = {"kind": kind, "param": rng.choice(["f32", "bf16", "master"]),
                "grad": rng.choice(["f32", "bf16"]), "bits": rng.choice([8, 32])}
        which = rng.choice(["adapters", "odd", "odd"])
        if which == "adapters":
            return dict(case, set=which, hidden=8 * rng.randint(32, 512), kv=8 * rng.randint(8, 128),
                        mlp=8 * rng.randint(64, 2368), layers=rng.randint(1, 28))
        tensors = _log(rng, 1, 400)
        return dict(case, set=which, tensors=tensors,
                    size=_log(rng, 100, min(LARGEST_ADAMW // 4 // tensors, 20_000_000)))
    if kind == "int8":
        grad = rng.random() < 0.4
        k, n = _width(rng, 16), _width(rng, 8, 128)
        tokens = min(_log(rng, 1, 16384), LARGEST_INT8 // (k * n))
        return {"kind": kind, "tokens": max(1, tokens), "k": k, "n": n, "grad": grad,
                "bias": not grad and rng.random() < 0.4, "out": rng.choice(["bf16", "bf16", "f32"]),
                "pad": rng.choice([0, 0, 8, 40])}
    post = rng.random() < 0.6
    shape = {"post": post, "gate": rng.choice(["none", "channel", "token", "element"]) if post
             else rng.choice(["none", "none", "token"]),
             "scale": rng.choice([1.0, 0.5, 0.22]), "pad": rng.choice([0, 0, 8, 24])}
    if kind == "norm_int8":
        return dict(shape, kind=kind, rows=_log(rng, 1, 512), cols=_width(rng, 16, 256, 8192),
                    n=_width(rng, 8, 128), bias=rng.random() < 0.5)
    if kind == "norm":
        cols = _width(rng, 8, 64, 16384)
        return dict(shape, kind=kind, rows=max(1, min(_log(rng, 1, 16384), LARGEST_NORM // cols)), cols=cols)
    code = rng.choice(["none", "none", "int8", "e4m3fn", "e4m3fn_cast"])
    block = 0 if code in ("none", "e4m3fn_cast") else rng.choice([32, 64, 128, 256])
    cols = _width(rng, max(8, block), 256, 16384)
    return dict(shape, kind=kind, rows=max(1, min(_log(rng, 1, 16384), LARGEST_NORM // cols)), cols=cols,
                code=code, block=block, weights=rng.random() < 0.7)


# ------------------------------------------------------------------ inputs --
def _sizes(case):
    """(elements, weight decay on) of every tensor of an optimizer case."""
    if case["set"] == "odd":  # lengths spread around `size`, few of them round; a third without decay
        n, s = case["tensors"], case["size"]
        return [(max(1, s * (1 + (7 * i) % 13) // 7 - 3 * i), i % 3 != 0) for i in range(n)]
    h, kv, f = case["hidden"], case["kv"], case["mlp"]
    linears = [(h, h), (kv, h), (kv, h), (h, h), (f, h), (f, h), (h, f)]
    if case["set"] == "adapters":
        layer = [(n, True) for o, i in linears for n in (RANK * i, o * RANK)]
    else:
        layer = [(o * i, True) for o, i in linears] + [(h, False), (h, False), (h, False), (kv, False), (kv, False)]
    return layer * case["layers"]


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _normal(g, shape, sigma=1.0, dtype=torch.float32):
    return torch.randn(shape, generator=g, device=DEV).mul_(sigma).to(dtype)


def _activation(g, rows, cols, pad=0, sigma=1.0):
    """bf16 [rows, cols], rows `pad` elements apart, half a percent of the channels 30 times the others."""
    x = torch.randn((rows, cols + pad), generator=g, device=DEV).mul_(sigma)
    heavy = torch.randperm(cols, generator=g, device=DEV)[:max(1, cols // 200)]
    x[:, heavy] *= 30.0
    return x.to(torch.bfloat16)[:, :cols]


def _block_codes(x, code, block):
    """(codes, scales) of a saved bf16 tensor: block absmax int8 or E4M3FN, or the plain cast."""
    if code == "e4m3fn_cast":
        return x.to(torch.float8_e4m3fn).view(torch.uint8), None
    q = 127.0 if code == "int8" else 448.0
    b = x.float().reshape(x.shape[0], -1, block)
    amax = b.abs().amax(2, keepdim=True)
    r = torch.where(amax < TINY, 0.0, q / amax)
    v = (b * r).clamp_(-q, q)
    codes = v.round_().to(torch.int8).view(torch.uint8) if code == "int8" else v.to(torch.float8_e4m3fn).view(torch.uint8)
    return codes.reshape(x.shape), (amax.squeeze(2) / q).contiguous()


def _row_codes(w):
    """int8 codes and scales of a weight [n, k], one scale per row."""
    amax = w.abs().amax(1)
    return (w * (127.0 / amax)[:, None]).round_().clamp_(-127, 127).to(torch.int8), amax / 127.0


def prepare(case, seed):
    g, kind = _gen(seed), case["kind"]
    return {"adamw": _prepare_adamw, "norm": _prepare_norm, "norm_bwd": _prepare_norm_bwd,
            "norm_int8": _prepare_norm_int8, "int8": _prepare_int8}[kind](case, g, int(seed))


def _prepare_adamw(case, g, seed):
    # one buffer per kind with every tensor at a multiple of 256 elements, as a trainer keeps them
    sizes = _sizes(case)
    begin, at = [], 0
    for n, _ in sizes:
        begin.append(at)
        at += -(-n // STATE_BLOCK) * STATE_BLOCK
    real = torch.zeros(at, dtype=torch.bool, device=DEV)
    for b, (n, _) in zip(begin, sizes):
        real[b:b + n] = True
    st = {"kind": "adamw", "case": dict(case), "begin": begin, "n": [n for n, _ in sizes],
          "lr": [2e-4 if i % 5 else 1e-4 for i in range(len(sizes))],
          "decay": [0.01 if d else 0.0 for _, d in sizes], "total": at, "step": 100, "seed": seed % 65521}
    weight = _normal(g, at, 0.02) * real
    st["p"] = weight if case["param"] != "bf16" else None
    st["p16"] = weight.to(torch.bfloat16) if case["param"] != "f32" else None
    # gradients differ in size from tensor part to tensor part
    size = torch.exp(_normal(g, at // STATE_BLOCK)).repeat_interleave(STATE_BLOCK)
    st["grad"] = (_normal(g, at, 1e-4) * size * real).to(torch.bfloat16 if case["grad"] == "bf16" else torch.float32)
    m, r = _normal(g, at, 3e-5) * size * real, (0.5e-4 + _normal(g, at, 5e-5).abs()) * size * real
    if case["bits"] == 32:
        st["m"], st["v"], st["m_scale"], st["v_scale"] = m, r * r, None, None
    else:
        mc, ms = _block_codes(m.reshape(1, -1), "e4m3fn", STATE_BLOCK)
        vc, vs = _block_codes(r.reshape(1, -1), "e4m3fn", STATE_BLOCK)
        st.update(m=mc.reshape(-1).view(torch.float8_e4m3fn), v=vc.reshape(-1).view(torch.float8_e4m3fn),
                  m_scale=ms.reshape(-1), v_scale=vs.reshape(-1))
    st["norm"] = torch.zeros(2, device=DEV)
    return st


def _gate(case, g):
    rows, cols = case["rows"], case["cols"]
    shape = {"none": None, "channel": (cols,), "token": (rows, 1), "element": (rows, cols)}[case["gate"]]
    return None if shape is None else (torch.rand(shape, generator=g, device=DEV) + 0.1).to(torch.bfloat16)


def _weight(g, cols):
    return (1.0 + _normal(g, cols, 0.1)).to(torch.bfloat16)


def _prepare_norm(case, g, seed):
    rows, cols = case["rows"], case["cols"]
    return {"kind": case["kind"], "scale": case["scale"], "res": _activation(g, rows, cols, case["pad"], 2.0),
            "y": _activation(g, rows, cols, case["pad"]), "w_post": _weight(g, cols) if case["post"] else None,
            "gate": _gate(case, g), "w_pre": _weight(g, cols),
            "h": torch.empty((rows, cols), dtype=torch.bfloat16, device=DEV),
            "out": torch.empty((rows, cols), dtype=torch.bfloat16, device=DEV),
            "rstd_post": torch.empty(rows, device=DEV) if case["post"] else None,
            "rstd_pre": torch.empty(rows, device=DEV)}


def _prepare_norm_bwd(case, g, seed):
    rows, cols, code, block = case["rows"], case["cols"], case["code"], case["block"]
    st = {"kind": "norm_bwd", "code": code, "block": block, "scale": case["scale"],
          "w_post": _weight(g, cols) if case["post"] else None, "gate": _gate(case, g), "w_pre": _weight(g, cols),
          "dn": _activation(g, rows, cols, case["pad"], 1e-3), "dh": _normal(g, (rows, cols), 1e-3, torch.bfloat16)}
    # the block's output is needed by its norm's and its gate's gradients only
    for name, needed in (("h", True), ("y", case["post"] or case["gate"] != "none")):
        x = _activation(g, rows, cols, case["pad"]) if needed else None
        st["rstd_pre" if name == "h" else "rstd_post"] = None if x is None or (name == "y" and not case["post"]) else \
            torch.rsqrt(x.float().square().mean(1) + EPS)
        st[name] = x if code == "none" else None
        st[name + "_codes"], st[name + "_scales"] = (None, None) if x is None or code == "none" else _block_codes(x, code, block)
    st["dres"], st["dy"] = (torch.empty((rows, cols), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    st["dw_pre"] = torch.empty(cols, device=DEV) if case["weights"] else None
    st["dw_post"] = torch.empty(cols, device=DEV) if case["weights"] and case["post"] else None
    st["dgate"] = {"none": None, "channel": torch.empty(cols, device=DEV) if case["weights"] else None,
                   "token": torch.empty((rows, 1), device=DEV),
                   "element": torch.empty((rows, cols), dtype=torch.bfloat16, device=DEV)}[case["gate"]]
    return st


def _prepare_norm_int8(case, g, seed):
    st = _prepare_norm(case, g, seed)
    st["out"] = None
    st["w"], st["w_scale"] = _row_codes(_normal(g, (case["n"], case["cols"]), 0.02))
    st["bias"] = _normal(g, case["n"], 0.1, torch.bfloat16) if case["bias"] else None
    st["codes"] = torch.empty((case["rows"], case["cols"]), dtype=torch.int8, device=DEV)
    st["code_scale"] = torch.empty(case["rows"], device=DEV)
    st["product"] = torch.empty((case["rows"], case["n"]), dtype=torch.bfloat16, device=DEV)
    return st


def _prepare_int8(case, g, seed):
    t, k, n = case["tokens"], case["k"], case["n"]
    st = {"kind": "int8", "x": _activation(g, t, k, case["pad"], 1e-3 if case["grad"] else 1.0)}
    if case["grad"]:  # the forward's weight is [k, n] with a scale per k: its codes transposed once
        w, s = _row_codes(_normal(g, (k, n), 0.02))
        st["w"], st["factor"], st["w_scale"] = w.t().contiguous(), s, None
    else:
        st["w"], st["w_scale"] = _row_codes(_normal(g, (n, k), 0.02))
        st["factor"] = None
    st["bias"] = _normal(g, n, 0.1, torch.bfloat16) if case["bias"] else None
    st["out"] = torch.empty((t, n), dtype=torch.bfloat16 if case["out"] == "bf16" else torch.float32, device=DEV)
    return st


# -------------------------------------------------------------------- work --
def work(case):
    kind = case["kind"]
    if kind == "adamw":
        n, count = sum(s for s, _ in _sizes(case)), len(_sizes(case))
        param = {"f32": 8, "bf16": 4, "master": 10}[case["param"]]
        state = 16 if case["bits"] == 32 else 4 + 16.0 / STATE_BLOCK
        return {"bytes": n * (param + state + (2 if case["grad"] == "bf16" else 4)) + 8 * count, "flops": 20.0 * n}
    if kind == "int8":
        t, k, n = case["tokens"], case["k"], case["n"]
        out = 2 if case["out"] == "bf16" else 4
        return {"bytes": 2.0 * t * k + n * k + 4.0 * (k if case["grad"] else n) + 2.0 * n * case["bias"] + out * t * n,
                "flops": 2.0 * t * k * n}
    rows, cols = case["rows"], case["cols"]
    gate = {"none": 0, "channel": 2 * cols, "token": 2 * rows, "element": 2 * rows * cols}[case["gate"]]
    vectors = 2.0 * cols * (2 if case["post"] else 1) + 4.0 * rows * (2 if case["post"] else 1) + gate
    if kind == "norm":
        return {"bytes": 8.0 * rows * cols + vectors, "flops": 12.0 * rows * cols}
    if kind == "norm_int8":
        n = case["n"]
        return {"bytes": 6.0 * rows * cols + vectors + n * cols + 4.0 * n + 2.0 * n * case["bias"] + 2.0 * rows * n,
                "flops": 12.0 * rows * cols + 2.0 * rows * cols * n}
    saved = 2.0 if case["code"] == "none" else 1.0 + (4.0 / case["block"] if case["block"] else 0.0)
    inputs = saved * (2 if case["post"] or case["gate"] != "none" else 1) + 4.0
    grads = (4.0 * cols * (2 if case["post"] else 1) if case["weights"] else 0.0) + \
        {"none": 0.0, "channel": 4.0 * cols if case["weights"] else 0.0, "token": 4.0 * rows, "element": 2.0 * rows * cols}[case["gate"]]
    return {"bytes": (inputs + 4.0) * rows * cols + vectors + grads, "flops": 25.0 * rows * cols}


# --------------------------------------------------------------------- run --
def run(state):
    kind = state["kind"]
    if own:
        return {"adamw": _own_adamw, "norm": _own_norm, "norm_bwd": _own_norm_bwd, "norm_int8": _own_norm_int8,
                "int8": _own_int8}[kind](state)
    return {"adamw": _plain_adamw, "norm": _plain_norm, "norm_bwd": _plain_norm_bwd,
            "norm_int8": _plain_norm_int8, "int8": _plain_int8}[kind](state)


def _adamw_outputs(st):
    """The updated state: an 8-bit one as its E4M3FN values and the scale of each 256 of them."""
    return {k: st[k] for k in ("p", "p16", "m", "v", "m_scale", "v_scale", "norm") if st[k] is not None}


def _norm_bwd_outputs(st):
    return {k: st[k] for k in ("dres", "dy", "dw_pre", "dw_post", "dgate") if st[k] is not None}


# the package's calls; descriptors and workspaces are made once, as a trainer keeps them
def _own_adamw(st):
    from paper_2609_33570_amd import hilore as hl

    if "tensors" not in st:
        def part(name, i, unit=1):
            x = st[name]
            return None if x is None else x[st["begin"][i] // unit:][:-(-st["n"][i] // unit)]

        st["tensors"] = hl.adamw_tensors([
            hl.adamw_tensor(p=part("p", i), p16=part("p16", i), grad=part("grad", i), m=part("m", i), v=part("v", i),
                            m_scales=part("m_scale", i, STATE_BLOCK), v_scales=part("v_scale", i, STATE_BLOCK),
                            lr=st["lr"][i], weight_decay=st["decay"][i]) for i in range(len(st["n"]))])
        st["workspace"] = torch.empty(hl.hilore_grad_norm_workspace_bytes(st["tensors"]), dtype=torch.uint8, device=DEV)
    hl.hilore_grad_norm(st["tensors"], MAX_NORM, st["norm"], workspace=st["workspace"])
    hl.hilore_adamw(st["tensors"], BETA1, BETA2, ADAM_EPS, st["step"], norm=st["norm"], seed=st["seed"] + st["step"])
    st["step"] += 1
    return _adamw_outputs(st)


def _norm_desc(hl, st):
    if "desc" not in st:
        st["desc"] = hl.block_norm_desc(res=st["res"], y=st["y"], w_post=st["w_post"], gate=st["gate"], scale=st["scale"],
                                        w_pre=st["w_pre"], eps=EPS, h=st["h"], n=st["out"], codes=st.get("codes"),
                                        code_scales=st.get("code_scale"), rstd_post=st["rstd_post"],
                                        rstd_pre=st["rstd_pre"])
    return st["desc"]


def _own_norm(st):
    from paper_2609_33570_amd import hilore as hl

    hl.hilore_block_norm(_norm_desc(hl, st))
    return {k: st[k] for k in ("h", "out", "rstd_post", "rstd_pre") if st[k] is not None}


def _own_norm_bwd(st):
    from paper_2609_33570_amd import hilore as hl

    if "desc" not in st:
        st["desc"] = hl.block_norm_bwd_desc(
            h=hl.unit_desc(x=st["h"], codes=st["h_codes"], scales=st["h_scales"]),
            y=None if st["y"] is None and st["y_codes"] is None else hl.unit_desc(x=st["y"], codes=st["y_codes"], scales=st["y_scales"]),
            w_post=st["w_post"], gate=st["gate"], scale=st["scale"], w_pre=st["w_pre"], rstd_post=st["rstd_post"],
            rstd_pre=st["rstd_pre"], dn=st["dn"], dh=st["dh"], dres=st["dres"], dy=st["dy"], dw_post=st["dw_post"],
            dw_pre=st["dw_pre"], dgate=st["dgate"])
        st["workspace"] = torch.empty(hl.hilore_block_norm_bwd_workspace_bytes(st["desc"]), dtype=torch.uint8, device=DEV)
    code = 0 if st["code"] == "none" else st["code"]
    hl.hilore_block_norm_bwd(st["desc"], code, st["block"], workspace=st["workspace"])
    return _norm_bwd_outputs(st)


def _own_product(hl, st, **operand):
    if "product_desc" not in st:
        st["product_desc"] = hl.int8_desc(w=st["w"], w_scales=st["w_scale"], bias=st["bias"], **operand)
        need = hl.hilore_int8_workspace_bytes(st["product_desc"])
        st["workspace"] = torch.empty(need, dtype=torch.uint8, device=DEV)
    return st["product_desc"]


def _own_norm_int8(st):
    from paper_2609_33570_amd import hilore as hl

    hl.hilore_block_norm(_norm_desc(hl, st))
    desc = _own_product(hl, st, a=st["codes"], a_scales=st["code_scale"], out=st["product"])
    hl.hilore_int8_matmul(desc, workspace=st["workspace"])
    return {"h": st["h"], "product": st["product"]}


def _own_int8(st):
    from paper_2609_33570_amd import hilore as hl

    desc = _own_product(hl, st, x=st["x"], factor=st["factor"], out=st["out"])
    hl.hilore_int8_linear(desc, workspace=st["workspace"])
    return st["out"]


# the plain forms
def _hash32(x):
    """A mixed 32-bit word of each 32-bit word (held in int64)."""
    x = x ^ (x >> 16)
    x = (x * 0x6A09E667) & 0xFFFFFFFF
    x = x ^ (x >> 15)
    x = (x * 0xBB67AE85) & 0xFFFFFFFF
    return x ^ (x >> 16)


def _tensor_of_block(st):
    """(tensor, first element's place in it) of every block of 256 elements, [blocks, 1]."""
    begin = torch.tensor(st["begin"], device=DEV)
    first = torch.arange(0, st["total"], STATE_BLOCK, device=DEV)[:, None]
    tensor = torch.bucketize(first, begin, right=True) - 1
    return tensor, first - begin[tensor]


def _random_words(st, tensor, place, salt):
    """32 random bits of every element, of the seed, its tensor and its place in it."""
    key = _hash32((st["seed"] + st["step"] + (tensor + 1) * 0x9E3779B1 + salt) & 0xFFFFFFFF)
    return _hash32((place + torch.arange(STATE_BLOCK, device=DEV)) ^ key)


def _plain_codes(x, bits, keep):
    """E4M3FN codes of fp32 values by blocks of 256, rounded up or down by 16 random bits."""
    amax = x.abs().amax(1, keepdim=True)
    # scaled so that the exponent field of an fp32 is that of an E4M3FN, subnormals included
    r = torch.where(amax < TINY, 0.0, 448.0 / amax)
    code = ((x.abs() * r * 2.0 ** -120).view(torch.int32) + (bits << 4).to(torch.int32)) >> 20
    code = code.clamp_(max=0x7E)
    if keep:  # what is above zero stays above it
        code = torch.where((x > 0) & (amax >= TINY), code.clamp(min=1), code)
    code = code | torch.where(x < 0, 0x80, 0)
    return code.to(torch.uint8).view(torch.float8_e4m3fn).reshape(-1), torch.where(amax < TINY, 0.0, amax / 448.0).reshape(-1)


def _plain_adamw(st):
    def blocks(name):
        return st[name].float().reshape(-1, STATE_BLOCK)

    tensor, place = _tensor_of_block(st)
    lr, decay = torch.tensor(st["lr"], device=DEV)[tensor], torch.tensor(st["decay"], device=DEV)[tensor]
    grad = blocks("grad")
    norm = grad.square().sum().sqrt()
    st["norm"][0] = norm
    st["norm"][1] = torch.clamp(MAX_NORM / (norm + 1e-6), max=1.0)
    grad = grad * st["norm"][1]
    c1, c2 = 1.0 - BETA1 ** st["step"], 1.0 - BETA2 ** st["step"]
    eight = st["m_scale"] is not None
    m, v = blocks("m"), blocks("v")
    if eight:
        m, v = m * st["m_scale"][:, None], (v * st["v_scale"][:, None]).square()
    m = BETA1 * m + (1.0 - BETA1) * grad
    v = BETA2 * v + (1.0 - BETA2) * (grad * grad)
    r = v.sqrt()
    p = blocks("p" if st["p"] is not None else "p16")
    p = p * (1.0 - lr * decay) - lr * ((m / c1) / (r / math.sqrt(c2) + ADAM_EPS))
    if eight:
        word = _random_words(st, tensor, place, 0)
        for name, x, bits in (("m", m, word & 0xFFFF), ("v", r, word >> 16)):
            code, scale = _plain_codes(x, bits, name == "v")
            st[name].copy_(code), st[name + "_scale"].copy_(scale)
    else:
        st["m"].copy_(m.reshape(-1)), st["v"].copy_(v.reshape(-1))
    if st["p"] is not None:
        st["p"].copy_(p.reshape(-1))
        if st["p16"] is not None:
            st["p16"].copy_(st["p"].to(torch.bfloat16))
    else:  # bf16 parameters: rounded up or down by 16 random bits
        w = p.view(torch.int32) + (_random_words(st, tensor, place, 0x3C6EF372) & 0xFFFF).to(torch.int32)
        st["p16"].copy_((w & ~0xFFFF).view(torch.float32).to(torch.bfloat16).reshape(-1))
    st["step"] += 1
    return _adamw_outputs(st)


def _plain_block(st):
    """(h, norm of h, factors): h is the stream as it is stored, in bf16."""
    z = st["y"].float()
    rstd_post = None
    if st["w_post"] is not None:
        rstd_post = torch.rsqrt(z.square().mean(1) + EPS)
        z = z * rstd_post[:, None] * st["w_post"].float()
    if st["gate"] is not None:
        z = z * st["gate"].float()
    h = (st["res"].float() + st["scale"] * z).to(torch.bfloat16)
    rstd_pre = torch.rsqrt(h.float().square().mean(1) + EPS)
    return h, h.float() * rstd_pre[:, None] * st["w_pre"].float(), rstd_post, rstd_pre


def _plain_norm(st):
    h, n, rstd_post, rstd_pre = _plain_block(st)
    out = {"h": h, "out": n.to(torch.bfloat16), "rstd_post": rstd_post, "rstd_pre": rstd_pre}
    return {k: v for k, v in out.items() if v is not None}


def _plain_saved(st, name):
    """A saved tensor in 32 bits: as it is, or the bf16 value that its codes stand for."""
    codes, scales = st[name + "_codes"], st[name + "_scales"]
    if codes is None:
        return None if st[name] is None else st[name].float()
    v = codes.view(torch.int8 if st["code"] == "int8" else torch.float8_e4m3fn).float()
    if scales is not None:
        v = (v.reshape(v.shape[0], -1, st["block"]) * scales[:, :, None]).reshape(v.shape)
    return v.to(torch.bfloat16).float()


def _plain_norm_bwd(st):
    dn, cols = st["dn"].float(), st["dn"].shape[1]
    hh = _plain_saved(st, "h") * st["rstd_pre"][:, None]
    t = dn * st["w_pre"].float()
    d = st["dh"].float() + st["rstd_pre"][:, None] * (t - hh * ((t * hh).sum(1, keepdim=True) / cols))
    st["dres"].copy_(d)
    if st["dw_pre"] is not None:
        st["dw_pre"].copy_((dn * hh).sum(0))
    dz = st["scale"] * d
    z = _plain_saved(st, "y")
    if st["w_post"] is not None:
        yh = z * st["rstd_post"][:, None]
        z = yh * st["w_post"].float()
    if st["dgate"] is not None:
        dg = dz * z
        kind = st["gate"].shape
        st["dgate"].copy_(dg.sum(0) if len(kind) == 1 else dg.sum(1, keepdim=True) if kind[1] == 1 else dg)
    if st["gate"] is not None:
        dz = dz * st["gate"].float()
    if st["w_post"] is not None:
        if st["dw_post"] is not None:
            st["dw_post"].copy_((dz * yh).sum(0))
        t = dz * st["w_post"].float()
        dz = st["rstd_post"][:, None] * (t - yh * ((t * yh).sum(1, keepdim=True) / cols))
    st["dy"].copy_(dz)
    return _norm_bwd_outputs(st)


def _plain_product(x, w, w_scale, bias, dtype):
    """int8 product of an fp32 operand rounded token by token."""
    amax = x.abs().amax(1, keepdim=True)
    a = (x * torch.where(amax < TINY, 0.0, 127.0 / amax)).round().clamp(-127, 127)
    out = (a @ w.float().t()) * torch.where(amax < TINY, 0.0, amax / 127.0)
    if w_scale is not None:
        out = out * w_scale
    if bias is not None:
        out = out + bias.float()
    return out.to(dtype)


def _plain_norm_int8(st):
    h, n, _, _ = _plain_block(st)
    return {"h": h, "product": _plain_product(n, st["w"], st["w_scale"], st["bias"], torch.bfloat16)}


def _plain_int8(st):
    x = st["x"].float()
    if st["factor"] is not None:
        x = x * st["factor"]
    return _plain_product(x, st["w"], st["w_scale"], st["bias"], st["out"].dtype)


# ------------------------------------------------------------------- exact --
def exact(case, seed):
    st = prepare(case, seed)
    return {"adamw": _exact_adamw, "norm": _exact_norm, "norm_bwd": _exact_norm_bwd,
            "norm_int8": _exact_norm_int8, "int8": _exact_int8}[case["kind"]](st)


def _exact_rounded(a, u):
    """E4M3FN values of 0 <= a <= 448: a lies between two of them, the upper one is taken when the
    part of the way to it and u in [0, 1) together reach 1."""
    exponent = torch.frexp(a)[1].clamp(min=-5).double()        # a < 2 ** exponent, normal from 2 ** -6 on
    quantum = torch.exp2(exponent - 4.0)
    return torch.floor(a / quantum + u) * quantum


def _exact_words(st, i, salt):
    """32 random bits for every element of tensor i, with numpy's wrapping 32-bit arithmetic."""
    def mix(x):
        x = x ^ (x >> np.uint32(16))
        x = x * np.uint32(0x6A09E667)
        x = x ^ (x >> np.uint32(15))
        x = x * np.uint32(0xBB67AE85)
        return x ^ (x >> np.uint32(16))

    key = mix(np.array([(st["seed"] + st["step"] + (i + 1) * 0x9E3779B1 + salt) % 2 ** 32], dtype=np.uint32))
    return torch.from_numpy(mix(np.arange(st["n"][i], dtype=np.uint32) ^ key).astype(np.int64)).to(DEV)


def _exact_adamw(st):
    grad = st["grad"].double()
    norm = torch.linalg.vector_norm(grad)
    clip = min(1.0, MAX_NORM / (float(norm) + 1e-6))
    c1, c2 = 1.0 - BETA1 ** st["step"], 1.0 - BETA2 ** st["step"]
    out = {k: v.double() for k, v in _adamw_outputs(st).items()}
    out["norm"] = torch.tensor([float(norm), clip], dtype=torch.float64, device=DEV)
    for i, (b, n) in enumerate(zip(st["begin"], st["n"])):
        at, blocks = slice(b, b + n), slice(b // STATE_BLOCK, b // STATE_BLOCK + -(-n // STATE_BLOCK))
        whole = slice(b, b + -(-n // STATE_BLOCK) * STATE_BLOCK)
        g = grad[at] * clip
        m, r = out["m"][at], out["v"][at]
        if st["m_scale"] is not None:
            m = m * st["m_scale"][blocks].double().repeat_interleave(STATE_BLOCK)[:n]
            r = r * st["v_scale"][blocks].double().repeat_interleave(STATE_BLOCK)[:n]
            v = r ** 2
        else:
            v = r
        m = m + (1.0 - BETA1) * (g - m)
        v = v + (1.0 - BETA2) * (g ** 2 - v)
        lr, wd = st["lr"][i], st["decay"][i]
        p = (st["p"] if st["p"] is not None else st["p16"])[at].double()
        p = p - lr * wd * p - lr * (m / c1) / (torch.sqrt(v / c2) + ADAM_EPS)
        if st["m_scale"] is None:
            out["m"][at], out["v"][at] = m, v
        else:
            word = _exact_words(st, i, 0)
            for name, x, u in (("m", m, (word & 0xFFFF).double() / 65536), ("v", v.sqrt(), (word >> 16).double() / 65536)):
                padded = torch.zeros(whole.stop - whole.start, dtype=torch.float64, device=DEV)
                padded[:n] = x
                amax = padded.reshape(-1, STATE_BLOCK).abs().amax(1)
                scale = torch.where(amax < TINY, 0.0, amax / 448.0)
                s = scale.repeat_interleave(STATE_BLOCK)[:n]
                code = _exact_rounded(torch.where(s > 0, x.abs() / s, 0.0).clamp(max=448.0), u)
                if name == "v":
                    code = torch.where((x > 0) & (s > 0), code.clamp(min=2.0 ** -9), code)
                out[name][at], out[name + "_scale"][blocks] = code * torch.sign(x), scale
        if st["p"] is not None:
            out["p"][at] = p
        if st["p16"] is not None:
            if st["p"] is None:  # the two bf16 values around p, chosen by 16 random bits
                u = (_exact_words(st, i, 0x3C6EF372) & 0xFFFF).double() / 65536
                quantum = torch.exp2(torch.frexp(p)[1].double() - 8.0)
                p = torch.sign(p) * torch.floor(p.abs() / quantum + u) * quantum
            out["p16"][at] = p
    return out


def _exact_block(st):
    y, gate = st["y"].double(), 1.0 if st["gate"] is None else st["gate"].double()
    rstd_post = None
    if st["w_post"] is not None:
        rstd_post = (torch.linalg.vector_norm(y, dim=1) ** 2 / y.shape[1] + EPS) ** -0.5
        y = torch.mul(y * st["w_post"].double(), rstd_post.unsqueeze(1))
    h = torch.addcmul(st["res"].double(), y, torch.as_tensor(gate, device=DEV, dtype=torch.float64), value=st["scale"])
    stored = h.to(torch.bfloat16).double()
    rstd_pre = (torch.linalg.vector_norm(stored, dim=1) ** 2 / y.shape[1] + EPS) ** -0.5
    return h, stored * st["w_pre"].double() * rstd_pre.unsqueeze(1), rstd_post, rstd_pre


def _exact_norm(st):
    h, n, rstd_post, rstd_pre = _exact_block(st)
    return {"h": h, "out": n, **({} if rstd_post is None else {"rstd_post": rstd_post}), "rstd_pre": rstd_pre}


def _exact_value(st, name):
    if st[name] is not None:
        return st[name].double()
    codes, scales = st[name + "_codes"], st[name + "_scales"]
    if codes is None:
        return None
    if st["code"] == "int8":
        v = codes.view(torch.int8).double()
    else:
        v = codes.view(torch.float8_e4m3fn).double()
    if scales is not None:
        v = (v.float() * scales.repeat_interleave(st["block"], dim=1)).to(torch.bfloat16).double()
    return v


def _exact_rms_bwd(x, rstd, w, dz):
    """Gradients of x * rstd(x) * w: of x, of w."""
    unit = x * rstd.double()[:, None]
    weighted = dz * w.double()
    along = torch.linalg.vecdot(weighted, unit, dim=1) / x.shape[1]
    return rstd.double()[:, None] * torch.addcmul(weighted, unit, along[:, None].expand_as(unit), value=-1.0), (dz * unit).sum(0)


def _exact_norm_bwd(st):
    d, dw_pre = _exact_rms_bwd(_exact_value(st, "h"), st["rstd_pre"], st["w_pre"], st["dn"].double())
    d = d + st["dh"].double()
    out = {"dres": d}
    if st["dw_pre"] is not None:
        out["dw_pre"] = dw_pre
    y = _exact_value(st, "y")
    inner = y
    if st["w_post"] is not None:
        inner = y * st["rstd_post"].double()[:, None] * st["w_post"].double()
    gate = torch.ones((), dtype=torch.float64, device=DEV) if st["gate"] is None else st["gate"].double()
    if st["dgate"] is not None:
        dg = st["scale"] * d * inner
        out["dgate"] = dg.sum_to_size(st["gate"].shape)
    dz = d * gate * st["scale"]
    if st["w_post"] is not None:
        dz, dw_post = _exact_rms_bwd(y, st["rstd_post"], st["w_post"], dz)
        if st["dw_post"] is not None:
            out["dw_post"] = dw_post
    out["dy"] = dz
    return out


def _exact_product(x, st):
    """The operand rounded to 127 steps of its token's largest magnitude, times the codes."""
    top = torch.linalg.vector_norm(x, ord=float("inf"), dim=1, keepdim=True)
    step = top / 127.0
    a = torch.where(top < TINY, 0.0, torch.round(x / step)).clamp(-127.0, 127.0)
    # the sums of whole numbers below 2 ** 53 are exact
    out = torch.matmul(a, st["w"].double().t().contiguous()) * step
    if st["w_scale"] is not None:
        out = out * st["w_scale"].double()
    return out if st["bias"] is None else out + st["bias"].double()


def _exact_norm_int8(st):
    h, n, _, _ = _exact_block(st)
    return {"h": h, "product": _exact_product(n, st)}


def _exact_int8(st):
    x = st["x"].double()
    return _exact_product(x if st["factor"] is None else x * st["factor"].double(), st)
