"""Timed cases of what a layer's step calls around and in place of its feed-forward block: the norms
before and after a block with its gate and residual, products with 4-bit weights and group scales, and a
whole mixture-of-experts layer for a decode step's tokens.

``listed()`` holds the named cases, ``draw(rng)`` gives others from the same ranges.  ``prepare`` makes
what the caller holds, ``run`` is one pass: the plain form in 32-bit torch, or with ``own`` the
library's entry points.  ``exact`` is the definition in 64 bits.

Keys of a case:
  op        "norm" (forward), "norm_train" (forward and backward), "q4" (one product), "q4_gated" (two
            products and the activation between them), "moe"
  dtype     "bf16", "f32": tokens, outputs and whatever is not quantized
  tokens
  norm:     d, post (norm after the block), gate ("none", "row": one row for all tokens, "token"),
            sigmoid (logistic function on the gate), alpha (residual scale)
  q4:       n_in, n_out, group (codes to a scale), scales (their type), offsets (weights scale code + offset),
            act, silu_up
  moe:      d, d_ff, experts, k, router ("softmax", "sigmoid", "given": choice and weights are inputs),
            bias (added to the scores for the choice alone), normalize, act, silu_up
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
BYTES = {"bf16": 2.0, "f32": 4.0}
EPS = 1e-5
T_GATE = 0.25  # the threshold of the gate activation


def _norm(op, dtype, tokens, d, post=True, gate="row", sigmoid=False, alpha=1.0):
    return dict(op=op, dtype=dtype, tokens=tokens, d=d, post=post, gate=gate, sigmoid=sigmoid, alpha=alpha)


def _q4(op, dtype, tokens, n_in, n_out, group, scales, offsets=False, act="relu", silu_up=False):
    return dict(op=op, dtype=dtype, tokens=tokens, n_in=n_in, n_out=n_out, group=group, scales=scales, offsets=offsets,
                act=act, silu_up=silu_up)


def _moe(dtype, tokens, d, d_ff, experts, k, router="softmax", bias=False, normalize=True, act="silu", silu_up=False):
    return dict(op="moe", dtype=dtype, tokens=tokens, d=d, d_ff=d_ff, experts=experts, k=k, router=router, bias=bias,
                normalize=normalize, act=act, silu_up=silu_up)


def listed():
    named = {
        # between two blocks of a decode step, 8B-shaped: latency is all there is
        "norm_8b_bf16_T1": _norm("norm", "bf16", 1, 4096),
        # between two blocks of a prompt, each token's block output gated by a projection of it
        "norm_8b_bf16_T4096": _norm("norm", "bf16", 4096, 4096, gate="token", sigmoid=True),
        # the paper's largest ladder model in its own precision, an odd batch, a scaled residual
        "norm_train_l13_f32_T513": _norm("norm_train", "f32", 513, 3840, gate="row", alpha=0.5),
        # the largest: a training step over a full batch of a 70B-shaped layer
        "norm_train_70b_bf16_T8192": _norm("norm_train", "bf16", 8192, 8192, gate="token", sigmoid=True),
        # a small ragged layer, three users, fp32 tokens, asymmetric codes in the smallest groups
        "q4_small_f32_T3": _q4("q4", "f32", 3, 416, 1111, 32, "f32", True),
        # a decode step's hidden layer, 8B-shaped, one token
        "q4_gated_8b_bf16_T1": _q4("q4_gated", "bf16", 1, 4096, 14336, 128, "bf16", act="silu"),
        # the way back of the 70B-shaped layer: rows as long as they get
        "q4_70b_bf16_T1": _q4("q4", "bf16", 1, 28672, 8192, 128, "bf16"),
        # a batch of 48 users through the hidden layer, fp32 tokens, asymmetric codes
        "q4_gated_8b_f32_T48": _q4("q4_gated", "f32", 48, 4096, 14336, 64, "bf16", True, act="rsplus"),
        # many small experts, one user's next token
        "moe_64x1024_bf16_T1": _moe("bf16", 1, 2048, 1024, 64, 8),
        # few large experts of the 8B shape, a batch of users: all experts are read (the largest)
        "moe_8x14336_bf16_T16": _moe("bf16", 16, 4096, 14336, 8, 2),
        # a selection bias balances many experts; a batch of users, several tokens to an expert
        "moe_64x1408_bf16_T64": _moe("bf16", 64, 2048, 1408, 64, 6, "sigmoid", bias=True, act="rsplus"),
        # fp32, an odd hidden width, the routing given by the caller, some tokens with no expert
        "moe_16x1001_f32_T5": _moe("f32", 5, 1032, 1001, 16, 4, "given", act="relu", silu_up=True),
    }
    return [dict(c, name=n) for n, c in named.items()]


def _log_int(rng, lo, hi):
    return int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))


def _width(rng, lo, hi, q):
    return max(q, round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / q) * q)


def draw(rng):
    """Widths from a tiny layer's to a 70B-shaped one's, one token to a full batch (norms) or to a decode
    step's batch (products, experts)."""
    while True:
        op = rng.choice(["norm", "norm_train", "q4", "q4_gated", "moe", "moe"])
        dtype = rng.choice(["bf16", "bf16", "f32"])
        act, silu_up = rng.choice(["relu", "rsplus", "silu"]), rng.random() < 0.25
        if op.startswith("norm"):
            # real widths are whole 16-byte chunks; one in eight is not
            d = _width(rng, 200, 8192, 1 if rng.random() < 0.125 else 16)
            tokens = 1 if op == "norm" and rng.random() < 0.2 else _log_int(rng, 2, 8192)
            c = _norm(op, dtype, tokens, d, rng.random() < 0.75, rng.choice(["none", "row", "token"]), rng.random() < 0.5,
                      rng.choice([1.0, 0.5, 0.875]))
            if tokens * d <= 8192 * 8192 // (1 if dtype == "bf16" else 2):
                return c
        elif op.startswith("q4"):
            group = rng.choice([32, 64, 128, 256])
            n_in = _width(rng, 256, 28672 if op == "q4" else 8192, group)
            n_out = _log_int(rng, 64, 28672) if rng.random() < 0.3 else _width(rng, 256, 28672, 64)
            tokens = 1 if rng.random() < 0.3 else _log_int(rng, 2, 64)
            c = _q4(op, dtype, tokens, n_in, n_out, group, rng.choice(["bf16", "f32"]), rng.random() < 0.5,
                    act if op == "q4_gated" else "relu", silu_up and op == "q4_gated")
            if n_in * n_out * (2 if op == "q4_gated" else 1) <= 2 * 8192 * 28672:
                return c
        else:
            d = _width(rng, 256, 4096, 1 if rng.random() < 0.125 else 16)
            d_ff = _log_int(rng, 200, 14336)
            if rng.random() < 0.7:
                d_ff = max(64, d_ff // 64 * 64)
            experts = rng.choice([8, 16, 32, 64, 128, rng.randint(2, 200)])
            k = rng.randint(1, min(experts, 8))
            tokens = 1 if rng.random() < 0.3 else _log_int(rng, 2, 64)
            router = rng.choice(["softmax", "sigmoid", "sigmoid", "given"])
            c = _moe(dtype, tokens, d, d_ff, experts, k, router, router != "given" and rng.random() < 0.5, rng.random() < 0.7,
                     act, silu_up)
            if experts * d * d_ff * BYTES[dtype] <= 8 * 4096 * 14336 * 2:
                return c


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    dt, T = DTYPES[case["dtype"]], case["tokens"]

    def normal(shape, std=1.0):
        return (torch.randn(shape, generator=gen, device="cuda") * std).to(dt)

    def uniform(shape, lo, hi, dtype=torch.float32):
        return (lo + (hi - lo) * torch.rand(shape, generator=gen, device="cuda")).to(dtype)

    s = dict(case)
    if case["op"].startswith("norm"):
        d = case["d"]
        # a residual stream of larger values than the block's output
        s["x"], s["f"] = normal((T, d), 2.0), normal((T, d), 0.7)
        s["pre_gain"] = uniform((d,), 0.5, 1.5, dt)
        s["post_gain"] = uniform((d,), 0.5, 1.5, dt) if case["post"] else None
        s["gate_in"] = None if case["gate"] == "none" else normal((1 if case["gate"] == "row" else T, d))
        if case["op"] == "norm_train":
            s["dn"], s["dx_out"] = normal((T, d)), normal((T, d))
    elif case["op"].startswith("q4"):
        n_in, n_out, g = case["n_in"], case["n_out"], case["group"]
        s["x"] = normal((T, n_in))
        for name in ("gate", "up") if case["op"] == "q4_gated" else ("w",):
            s[name + "_codes"] = torch.randint(0, 256, (n_out, n_in // 2), generator=gen, device="cuda").to(torch.uint8)
            st, size = DTYPES[case["scales"]], 0.2 * n_in ** -0.5
            s[name + "_scales"] = uniform((n_out, n_in // g), 0.5 * size, 1.5 * size, st)
            s[name + "_offsets"] = uniform((n_out, n_in // g), -size, size, st) if case["offsets"] else None
    else:
        d, d_ff, E, k = case["d"], case["d_ff"], case["experts"], case["k"]
        s["x"] = normal((T, d))
        # expert after expert: all of them at once would need twice their size in fp32
        for name, std in (("gate", d ** -0.5), ("up", d ** -0.5), ("down", d_ff ** -0.5)):
            w = s["w_" + name] = torch.empty((E, d_ff, d), dtype=dt, device="cuda")
            for e in range(E):
                w[e] = normal((d_ff, d), std)
        if case["router"] == "given":
            # k different experts for a token, one place in six unused
            order = torch.rand((T, E), generator=gen, device="cuda").argsort(dim=1)[:, :k]
            unused = torch.rand((T, k), generator=gen, device="cuda") < 1 / 6
            s["ids"] = torch.where(unused, torch.full_like(order, -1), order).to(torch.int32)
            s["weights"] = uniform((T, k), 0.1, 1.0)
        else:
            s["w_router"] = normal((E, d), d ** -0.5)
            s["bias"] = uniform((E,), -0.1, 0.1) if case["bias"] else None
    return s


# ------------------------------------------------------------------ the plain form
def _sigma(v):
    return 1.0 / (1.0 + torch.exp(-v))


def _hidden(s, h, v):
    """A(h - t) U(v)."""
    g = h - T_GATE
    if s["act"] == "relu":
        a = torch.where(g > 0, g, torch.zeros_like(g))
    elif s["act"] == "rsplus":
        a = torch.where(g > 0, g * _sigma(g), torch.zeros_like(g))
    else:
        a = g * _sigma(g)
    return a * (v * _sigma(v) if s["silu_up"] else v)


def _plain_norm(s):
    dt = s["x"].dtype
    x, f, pg = s["x"].float(), s["f"].float(), s["pre_gain"].float()
    one = torch.ones((), device=x.device)
    gate, slope = one, one
    if s["gate_in"] is not None:
        gate = s["gate_in"].float()
        if s["sigmoid"]:
            gate = _sigma(gate)
            slope = gate * (1.0 - gate)
    if s["post"]:
        rp = 1.0 / torch.sqrt((f * f).mean(1, keepdim=True) + EPS)
        hat, og = f * rp, s["post_gain"].float()
    else:
        rp, hat, og = one, f, one
    u = hat * og
    xo = s["alpha"] * x + gate * u
    r = 1.0 / torch.sqrt((xo * xo).mean(1, keepdim=True) + EPS)
    xh = xo * r
    out = {"x_out": xo.to(dt), "n_out": (xh * pg).to(dt)}
    if s["op"] == "norm":
        return out
    dn = s["dn"].float()
    dxh = dn * pg
    g = s["dx_out"].float() + r * (dxh - xh * (dxh * xh).mean(1, keepdim=True))
    du = g * gate
    dh = du * og
    df = rp * (dh - hat * (dh * hat).mean(1, keepdim=True)) if s["post"] else dh
    out.update(dx=(s["alpha"] * g).to(dt), df=df.to(dt), dpre_gain=(dn * xh).sum(0).to(dt))
    if s["post"]:
        out["dpost_gain"] = (du * hat).sum(0).to(dt)
    if s["gate_in"] is not None:
        dg = g * u * slope
        out["dgate"] = (dg.sum(0, keepdim=True) if s["gate"] == "row" else dg).to(dt)
    return out


def _plain_weights(s, name):
    b = s[name + "_codes"]
    codes = torch.stack((b & 15, b >> 4), dim=2).reshape(b.shape[0], -1).to(torch.int32)
    codes = torch.where(codes > 7, codes - 16, codes).float().reshape(b.shape[0], -1, s["group"])
    w = codes * s[name + "_scales"].float()[:, :, None]
    if s["offsets"]:
        w = w + s[name + "_offsets"].float()[:, :, None]
    return w.reshape(b.shape[0], -1)


def _plain_q4(s):
    x = s["x"].float()
    if s["op"] == "q4":
        return (x @ _plain_weights(s, "w").t()).to(s["x"].dtype)
    return _hidden(s, x @ _plain_weights(s, "gate").t(), x @ _plain_weights(s, "up").t()).to(s["x"].dtype)


def _plain_routing(s):
    """The choice is made in 64 bits: two right 32-bit results choose other experts where scores are near."""
    logits = s["x"].double() @ s["w_router"].double().t()
    if s["router"] == "softmax":
        e = torch.exp(logits - logits.amax(1, keepdim=True))
        score = e / e.sum(1, keepdim=True)
    else:
        score = _sigma(logits)
    by = logits if s["bias"] is None else score + s["bias"].double()
    ids = torch.sort(by, dim=1, descending=True, stable=True).indices[:, :s["k"]]
    w = torch.gather(score, 1, ids)
    if s["normalize"]:
        w = w / w.sum(1, keepdim=True)
    return ids.to(torch.int32), w.float()


def _plain_moe(s):
    T, d, d_ff, E, k = s["tokens"], s["d"], s["d_ff"], s["experts"], s["k"]
    ids, weights = (s["ids"], s["weights"]) if s["router"] == "given" else _plain_routing(s)
    x = s["x"].float()
    if T * k < E:  # the chosen experts' matrices, one set to a place
        at = ids.reshape(-1).long().clamp(min=0)
        xa = x[:, None, :].expand(T, k, d).reshape(T * k, d, 1)
        h = torch.matmul(s["w_gate"][at].float(), xa).reshape(T * k, d_ff)
        v = torch.matmul(s["w_up"][at].float(), xa).reshape(T * k, d_ff)
        z = _hidden(s, h, v)
        f = torch.matmul(z[:, None, :], s["w_down"][at].float()).reshape(T, k, d)
        on = torch.where(ids >= 0, weights, torch.zeros_like(weights))
        y = (f * on[:, :, None]).sum(1)
    else:  # every expert for every token
        h = (x @ s["w_gate"].float().reshape(E * d_ff, d).t()).reshape(T, E, d_ff)
        v = (x @ s["w_up"].float().reshape(E * d_ff, d).t()).reshape(T, E, d_ff)
        chosen = ids[:, :, None] == torch.arange(E, device=x.device)
        share = (chosen * weights[:, :, None]).sum(1)  # [T][E]
        z = _hidden(s, h, v) * share[:, :, None]
        y = z.reshape(T, E * d_ff) @ s["w_down"].float().reshape(E * d_ff, d)
    return {"y": y.to(s["x"].dtype), "ids": ids, "weights": weights}


# ------------------------------------------------------------------ the library's calls
def _options(s):
    from paper_2609_31975_amd import ffn

    return ffn.options(act={"relu": ffn.FFN_ACT_RELU, "rsplus": ffn.FFN_ACT_RSPLUS, "silu": ffn.FFN_ACT_SILU}[s["act"]],
                       silu_up=s["silu_up"])


def _norm_form(s):
    from paper_2609_31975_amd import ffn

    return ffn.norm(EPS, pre_gain=s["pre_gain"], post=s["post"], post_gain=s["post_gain"], gate=s["gate_in"],
                    gate_sigmoid=s["sigmoid"] and s["gate_in"] is not None, alpha=s["alpha"])


def _kept(s):
    """Buffers, options and descriptors that a program makes once.  A gate of each token is a step's own input: the form that
    holds it is made with the call."""
    from paper_2609_31975_amd import ffn

    k, x, T = {}, s["x"], s["tokens"]
    if s["op"].startswith("norm"):
        k["norm"] = None if s["gate"] == "token" else _norm_form(s)
        k["x_out"], k["n_out"] = torch.empty_like(x), torch.empty_like(x)
        if s["op"] == "norm_train":
            k["rstd"] = torch.empty((2, T), dtype=torch.float32, device="cuda")
            k["ws"] = ffn.alloc_norm_workspace(T, s["d"])
            k["grads"] = {n: None if v is None else torch.empty_like(v) for n, v in
                          (("dx", x), ("df", x), ("dgate", s["gate_in"]), ("dpost_gain", s["post_gain"]),
                           ("dpre_gain", s["pre_gain"]))}
    elif s["op"].startswith("q4"):
        for name in ("gate", "up") if s["op"] == "q4_gated" else ("w",):
            k[name] = ffn.group_q(s[name + "_codes"], s[name + "_scales"], s[name + "_offsets"])
        k["y"] = torch.empty((T, s["n_out"]), dtype=x.dtype, device="cuda")
        k["ws"] = ffn.alloc_group_q_workspace(T, s["n_in"], s["n_out"], gated=s["op"] == "q4_gated")
        k["opt"] = _options(s)
    else:
        given = s["router"] == "given"
        k["router"] = ffn.router(s["experts"], s["k"], w=None if given else s["w_router"], bias=None if given else s["bias"],
                                 sigmoid=s["router"] == "sigmoid", normalize=s["normalize"])
        k["opt"], k["y"] = _options(s), torch.empty_like(x)
        k["ws"] = ffn.alloc_moe_workspace(T, s["d"], s["d_ff"], s["experts"], s["k"], x.dtype)
        k["ids"] = s["ids"] if given else torch.empty((T, s["k"]), dtype=torch.int32, device="cuda")
        k["weights"] = s["weights"] if given else torch.empty((T, s["k"]), dtype=torch.float32, device="cuda")
    return k


def _own(s):
    from paper_2609_31975_amd import ffn

    if "kept" not in s:
        s["kept"] = _kept(s)
    k = s["kept"]
    if s["op"].startswith("norm"):
        form = k["norm"] or _norm_form(s)
        ffn.ffn_norm_forward(s["x"], s["f"], form, k["x_out"], k["n_out"], rstd=k.get("rstd"))
        out = {"x_out": k["x_out"], "n_out": k["n_out"]}
        if s["op"] == "norm_train":
            ffn.ffn_norm_backward(k["x_out"], s["f"], form, k["rstd"], s["dn"], s["dx_out"], k["ws"], **k["grads"])
            out.update((n, v) for n, v in k["grads"].items() if v is not None)
        return out
    if s["op"] == "q4":
        return ffn.ffn_group_q_forward(s["x"], k["w"], k["y"], k["ws"])
    if s["op"] == "q4_gated":
        return ffn.ffn_group_q_gated_forward(s["x"], k["gate"], k["up"], T_GATE, k["opt"], k["y"], k["ws"])
    y = ffn.ffn_moe_forward(s["x"], k["router"], s["w_gate"], s["w_up"], s["w_down"], T_GATE, k["opt"], k["ids"],
                            k["weights"], k["y"], k["ws"])
    return {"y": y, "ids": k["ids"], "weights": k["weights"]}


def run(s):
    if own:
        return _own(s)
    return _plain_norm(s) if s["op"].startswith("norm") else _plain_q4(s) if s["op"].startswith("q4") else _plain_moe(s)


def work(case):
    T, wb = case["tokens"], BYTES[case["dtype"]]
    if case["op"].startswith("norm"):
        d, train = case["d"], case["op"] == "norm_train"
        per_token = 4 + (case["gate"] == "token") + ((4 + (case["gate"] == "token")) if train else 0)
        rows = (1 + case["post"] + (case["gate"] == "row")) * (2 if train else 1)
        return {"bytes": wb * d * (T * per_token + rows), "flops": (40.0 if train else 12.0) * T * d}
    if case["op"].startswith("q4"):
        n_in, n_out, m = case["n_in"], case["n_out"], 2.0 if case["op"] == "q4_gated" else 1.0
        per_group = BYTES[case["scales"]] * (2 if case["offsets"] else 1)
        return {"bytes": m * n_out * n_in * (0.5 + per_group / case["group"]) + wb * T * (n_in + n_out),
                "flops": 2.0 * m * T * n_in * n_out}
    d, d_ff, E, k = case["d"], case["d_ff"], case["experts"], case["k"]
    places = T * k * (5 / 6 if case["router"] == "given" else 1.0)
    # experts that some token chooses, where every choice is as likely
    used = E * (1.0 - (1.0 - 1.0 / E) ** places) if T > 1 else places
    routing = wb * E * d if case["router"] != "given" else 0.0
    return {"bytes": wb * (3.0 * used * d * d_ff + 2.0 * T * d) + routing + 8.0 * T * k,
            "flops": 6.0 * places * d * d_ff + (2.0 * T * E * d if routing else 0.0)}


# ------------------------------------------------------------------ the definition, in 64 bits
def _f32(v):
    """The entry points take scalars as 32-bit numbers."""
    return float(torch.tensor(v, dtype=torch.float32))


def _exact_activation(s, h, v):
    g = h - _f32(T_GATE)
    a = torch.clamp(g, min=0.0) if s["act"] == "relu" else g * torch.sigmoid(g)
    if s["act"] == "rsplus":
        a = a * (g > 0)
    return a * (v * torch.sigmoid(v)) if s["silu_up"] else a * v


def _exact_rms(v):
    return (v.pow(2).mean(dim=-1, keepdim=True) + _f32(EPS)).rsqrt()


def _exact_norm(s):
    """The forward pass, and its gradients by torch's own differentiation in 64 bits, some tokens at a time."""
    names = ["x", "f", "pre_gain"] + (["post_gain"] if s["post"] else []) + (["gate_in"] if s["gate_in"] is not None else [])
    d = s["d"]
    train = s["op"] == "norm_train"
    out = {n: [] for n in ("x_out", "n_out", "x", "f", "gate_in")}
    sums = {}
    step = max(1, (1 << 24) // d)
    for a in range(0, s["tokens"], step):
        b = min(s["tokens"], a + step)
        cut = {n: (s[n][a:b] if s[n].dim() == 2 and s[n].shape[0] == s["tokens"] else s[n]).double().requires_grad_(train)
               for n in names}
        u = cut["f"]
        if s["post"]:
            u = u * _exact_rms(u) * cut["post_gain"]
        if "gate_in" in cut:
            u = u * (torch.sigmoid(cut["gate_in"]) if s["sigmoid"] else cut["gate_in"])
        xo = _f32(s["alpha"]) * cut["x"] + u
        n = xo * _exact_rms(xo) * cut["pre_gain"]
        out["x_out"].append(xo.detach())
        out["n_out"].append(n.detach())
        if train:
            ((n * s["dn"][a:b].double()).sum() + (xo * s["dx_out"][a:b].double()).sum()).backward()
            for name in names:
                if name in ("x", "f") or (name == "gate_in" and s["gate"] == "token"):
                    out[name].append(cut[name].grad)
                else:
                    sums[name] = sums.get(name, 0) + cut[name].grad
    result = {"x_out": torch.cat(out["x_out"]), "n_out": torch.cat(out["n_out"])}
    if train:
        result.update(dx=torch.cat(out["x"]), df=torch.cat(out["f"]), dpre_gain=sums["pre_gain"])
        if s["post"]:
            result["dpost_gain"] = sums["post_gain"]
        if s["gate_in"] is not None:
            result["dgate"] = sums["gate_in"] if s["gate"] == "row" else torch.cat(out["gate_in"])
    return result


def _exact_product(s, name):
    x, b, g = s["x"].double(), s[name + "_codes"].to(torch.int64), s["group"]
    scales = s[name + "_scales"].double().repeat_interleave(g, dim=1)
    w = torch.empty_like(scales)
    w[:, 0::2] = ((b % 16 + 8) % 16 - 8).double()
    w[:, 1::2] = ((b // 16 + 8) % 16 - 8).double()
    w *= scales
    if s["offsets"]:
        w += s[name + "_offsets"].double().repeat_interleave(g, dim=1)
    return x.matmul(w.transpose(0, 1))


def _exact_moe(s):
    T, E, k = s["tokens"], s["experts"], s["k"]
    x = s["x"].double()
    if s["router"] == "given":
        ids, weights = s["ids"].long(), s["weights"].double()
    else:
        logits = x.matmul(s["w_router"].double().transpose(0, 1))
        score = torch.softmax(logits, dim=1) if s["router"] == "softmax" else torch.sigmoid(logits)
        left = (logits if s["bias"] is None else score + s["bias"].double()).clone()
        ids = torch.empty((T, k), dtype=torch.long, device=x.device)
        for j in range(k):  # argmax gives the lowest index of equals here: made so by taking the first of them
            best = left == left.max(dim=1, keepdim=True).values
            ids[:, j] = torch.where(best, torch.arange(E, device=x.device), E).min(dim=1).values
            left.scatter_(1, ids[:, j:j + 1], -math.inf)
        weights = score.gather(1, ids)
        if s["normalize"]:
            weights = weights / weights.sum(dim=1, keepdim=True)
    y = torch.zeros_like(x)
    for e in range(E):
        tok, place = (ids == e).nonzero(as_tuple=True)
        if tok.numel():
            h = x[tok].matmul(s["w_gate"][e].double().transpose(0, 1))
            v = x[tok].matmul(s["w_up"][e].double().transpose(0, 1))
            f = _exact_activation(s, h, v).matmul(s["w_down"][e].double())
            y.index_add_(0, tok, f * weights[tok, place][:, None])
    return {"y": y, "ids": ids.to(torch.int32), "weights": weights}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"].startswith("norm"):
        return _exact_norm(s)
    if case["op"] == "q4":
        return _exact_product(s, "w")
    if case["op"] == "q4_gated":
        return _exact_activation(s, _exact_product(s, "gate"), _exact_product(s, "up"))
    return _exact_moe(s)
