"""Performance cases of the track decoder's further operators.

The decoder has one token per tool and frame.  A track's state may forget what a key already holds before it
takes the key's new value (``delta_rule``: gates per token, where the retention has one decay per head), tokens may look
at a map's cells twice and subtract what both looks have in common (``differential_attention``), and each token passes through
the few of many small networks that a router picks for it (``expert_layer``: a frame's tokens of all live streams
at once).  Eight tools per stream, up to sixteen streams, maps of 15 x 27 = 405 cells (854 x 480) to 34 x 60 = 2040
cells (1920 x 1080) and 60 frames per second give the sizes.

With ``own`` false, ``run`` computes plain torch forms; with ``own`` true it calls the library.
"""
from __future__ import annotations

import math

import torch

own = False

DEVICE = "cuda:0"
TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}
EPS = 1e-5
MOST_TOKENS = 1024         # of one call of the expert layer


# ---- the cases ------------------------------------------------------------------------------------
def _delta(batch, tokens, heads, qk_heads, key_dim, value_dim, dtype, ragged, name=None):
    return _named(name, op="delta_rule", batch=batch, tokens=tokens, heads=heads, qk_heads=qk_heads,
                  key_dim=key_dim, value_dim=value_dim, dtype=dtype, ragged=ragged)


def _differential(batch, q_tokens, k_tokens, q_heads, kv_heads, dim, value_dim, dtype, ragged, masked, norm, name=None):
    return _named(name, op="differential_attention", batch=batch, q_tokens=q_tokens, k_tokens=k_tokens,
                  q_heads=q_heads, kv_heads=kv_heads, dim=dim, value_dim=value_dim, dtype=dtype, ragged=ragged,
                  masked=masked, norm=norm)


def _experts(tokens, channels, hidden, experts, top, dtype, masked, renormalise, name=None):
    return _named(name, op="expert_layer", tokens=tokens, channels=channels, hidden=hidden, experts=experts,
                  top=top, dtype=dtype, masked=masked, renormalise=renormalise)


def _named(name, **c):
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # one live stream, one frame: eight tracks, one token each
        _delta(8, 1, 8, 8, 64, 64, "fp16", False, "update one frame"),
        # sixteen live streams, wide heads that share queries and keys; tools out of sight have no token
        _delta(128, 1, 16, 4, 128, 128, "bf16", True, "update sixteen streams' frame"),
        # clips of five streams, tracks of every length, odd sizes
        _delta(40, 257, 8, 4, 96, 80, "fp16", True, "update odd ragged clips"),
        # two minutes of one stream, wide heads
        _delta(8, 7200, 16, 16, 128, 128, "bf16", False, "update recording"),
        # one live stream: eight tool tokens compare two looks at one frame's cells
        _differential(1, 8, 405, 4, 4, 64, 128, "fp16", False, False, True, "compare on one frame"),
        # twelve live streams look at the cells of their last sixteen frames, some of them hidden
        _differential(12, 8, 6480, 4, 4, 64, 128, "bf16", True, True, True, "compare on sixteen frames"),
        # tracks of a clip, odd sizes, shared keys, cells behind glare hidden, no norm
        _differential(5, 77, 1001, 6, 2, 40, 80, "fp16", True, True, False, "compare odd"),
        # every cell of a 1920 x 1080 map looks at four such maps, eight streams
        _differential(8, 2040, 8160, 8, 2, 64, 128, "bf16", False, False, True, "compare cell by cell"),
        # one live stream, one frame: eight tool tokens
        _experts(8, 512, 1024, 16, 2, "fp16", False, True, "choose for one frame"),
        # odd sizes: tokens of five streams with seven tools and two more, no weight of the chosen raised
        _experts(37, 520, 1336, 6, 3, "bf16", False, False, "choose odd"),
        # sixteen live streams, many experts; tools out of sight have no token
        _experts(128, 1024, 2048, 32, 4, "bf16", True, True, "choose for sixteen streams"),
        # a clip of 128 frames of one stream: as many tokens as one call takes
        _experts(1024, 1024, 2048, 32, 4, "fp16", False, True, "choose for a clip"),
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm."""
    return max(lo, min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def _heads(rng):
    kv = rng.choice([1, 2, 3, 4, 8])
    return kv * rng.choice([1, 1, 2, 3, 4] if kv < 8 else [1, 2]), kv


def draw(rng):
    op = rng.choice(["delta_rule", "differential_attention", "expert_layer"])
    dtype = rng.choice(["fp16", "bf16"])
    while True:
        q, kv = _heads(rng)
        if op == "delta_rule":
            tokens = 1 if rng.random() < 0.35 else _spread(rng, 2, 7200)
            c = _delta(_spread(rng, 1, 128), tokens, q, kv, 8 * rng.randint(4, 16), 8 * rng.randint(4, 16), dtype,
                       rng.random() < 0.5)
            if work(c)["bytes"] <= 9e8:
                return c
        elif op == "differential_attention":
            c = _differential(_spread(rng, 1, 16), _spread(rng, 1, 2040), _spread(rng, 1, 8160), q, kv,
                              8 * rng.randint(4, 16), 8 * rng.randint(4, 16), dtype, rng.random() < 0.5,
                              rng.random() < 0.5, rng.random() < 0.7)
            if work(c)["flops"] <= 8e11:
                return c
        else:
            experts = _spread(rng, 2, 64)
            c = _experts(_spread(rng, 1, MOST_TOKENS), 8 * _spread(rng, 8, 160), 8 * _spread(rng, 8, 320), experts,
                         rng.randint(1, min(8, experts)), dtype, rng.random() < 0.4, rng.random() < 0.5)
            if work(c)["flops"] <= 5.1e10 and work(c)["bytes"] <= 6e8:
                return c


def work(case):
    c = case
    if c["op"] == "delta_rule":
        dk, dv, h, hk, n = (c[k] for k in ("key_dim", "value_dim", "heads", "qk_heads", "tokens"))
        b = c["batch"]
        if c["ragged"]:
            n = (n + 1) / 2           # tracks are half as long on average
        io = 2 * b * n * (2 * hk * dk + h * dv) + 8 * b * n * h + 2 * b * c["tokens"] * h * dv
        # recurrence: S^T k 2 per element of the state, S = g S + k u^T 3, the read-out 2
        return {"bytes": int(io + 8 * b * h * dk * dv), "flops": int(7 * b * n * h * dk * dv)}
    if c["op"] == "differential_attention":
        b, lk, d, dv = c["batch"], c["k_tokens"] * (0.5 if c["ragged"] else 1), c["dim"], c["value_dim"]
        return {"bytes": int(2 * b * (c["q_tokens"] * c["q_heads"] * (2 * d + dv) + lk * c["kv_heads"] * (2 * d + dv))
                             + (b * lk if c["masked"] else 0)),
                "flops": int(2 * b * c["q_heads"] * c["q_tokens"] * lk * (2 * d + 2 * dv))}
    t = c["tokens"] * (0.75 if c["masked"] else 1)
    ch, f, e, k = (c[x] for x in ("channels", "hidden", "experts", "top"))
    used = e * (1 - (1 - k / e) ** t)            # experts that some token picks, on average
    return {"bytes": int(used * 3 * ch * f * 2 + e * ch * 2 + 2 * (t + c["tokens"]) * ch + 8 * c["tokens"] * k),
            "flops": int(t * k * 6 * ch * f + 2 * t * e * ch)}


# ---- inputs -----------------------------------------------------------------------------------------
def _lengths(g, batch, longest):
    """Ragged lengths from nothing to everything; one sequence is whole and, of three or more, one is empty."""
    n = torch.randint(0, longest + 1, (batch,), generator=g, device=DEVICE, dtype=torch.int32)
    n[0] = longest
    if batch > 2:
        n[1] = 0
    return n


def prepare(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    c, t = case, TYPES[case["dtype"]]

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=DEVICE, dtype=t)

    def single(*shape):
        return torch.randn(*shape, generator=g, device=DEVICE)

    s = {"case": c}
    if c["op"] == "delta_rule":
        b, n, h, hk, dk, dv = (c[x] for x in ("batch", "tokens", "heads", "qk_heads", "key_dim", "value_dim"))
        # one projection gives queries and keys, of length one as the norm in front of the rule leaves them
        qk = normal(b, n, 2, hk, dk)
        qk.mul_(torch.rsqrt(qk.float().square().sum(-1, keepdim=True) + 1e-6).to(t))
        s["q"], s["k"] = qk[:, :, 0], qk[:, :, 1]
        s["v"] = normal(b, n, h, dv)
        # gates of a token: one projection gives both; half-lives from 22 frames to 47 seconds, times what the token says
        gates = single(b, n, 2, h)
        rate = 2.0 ** (-5.0 - 7.0 * torch.arange(h, device=DEVICE) / max(1, h - 1))
        gates[:, :, 0] = -rate * torch.nn.functional.softplus(gates[:, :, 0])
        gates[:, :, 1].sigmoid_()
        s["log_decay"], s["beta"] = gates[:, :, 0], gates[:, :, 1]
        s["state"] = single(b, h, dk, dv)
        s["scale"] = dk ** -0.5
        s["lengths"] = _lengths(g, b, n) if c["ragged"] else None
    elif c["op"] == "differential_attention":
        b, hq, hk, d, dv = (c[x] for x in ("batch", "q_heads", "kv_heads", "dim", "value_dim"))
        s["q"] = normal(b, c["q_tokens"], 2 * hq, d)         # heads 2h and 2h + 1 are the two looks of head h
        s["k"] = normal(b, c["k_tokens"], 2 * hk, d)
        s["v"] = normal(b, c["k_tokens"], hk, dv)
        s["scale"] = d ** -0.5
        s["lambda"] = torch.rand(hq, generator=g, device=DEVICE) * 0.6 + 0.2
        s["weight"] = 0.2 * (1 + 0.1 * single(dv)) if c["norm"] else None
        s["lengths"] = _lengths(g, b, c["k_tokens"]) if c["ragged"] else None
        s["mask"] = None
        if c["masked"]:
            s["mask"] = (torch.rand(b, c["k_tokens"], generator=g, device=DEVICE) < 0.8).to(torch.uint8)
    else:
        ch, f, e = c["channels"], c["hidden"], c["experts"]
        s["x"] = normal(c["tokens"], ch)
        s["router"] = normal(e, ch).mul_(ch ** -0.5)
        s["w_in"] = normal(e, 2 * f, ch).mul_(ch ** -0.5)    # the gate's rows, then the others
        s["w_out"] = normal(e, ch, f).mul_(f ** -0.5)
        s["mask"] = None
        if c["masked"]:
            s["mask"] = (torch.rand(c["tokens"], generator=g, device=DEVICE) < 0.75).to(torch.uint8)
    return s


# ---- plain forms ------------------------------------------------------------------------------------
def _plain_delta(s):
    """Chunks of 64 tokens: what the tokens of a chunk take from each other by a triangular system, solved row by row for all
    chunks at once, then the states from chunk to chunk."""
    c = s["case"]
    b, n, h, hk, dk, dv = (c[k] for k in ("batch", "tokens", "heads", "qk_heads", "key_dim", "value_dim"))
    size = min(64, n)
    chunks = (n + size - 1) // size
    pad = chunks * size - n
    lens = s["lengths"] if s["lengths"] is not None else torch.full((b,), n, device=DEVICE)
    there = torch.arange(n, device=DEVICE) < lens[:, None]                        # [b, n]

    def split(x):                                    # [b, n, heads, d] -> [b, h, chunks, size, d] in fp32
        x = torch.where(there[:, :, None, None], x.float(), 0.0).transpose(1, 2)
        x = x.repeat_interleave(h // x.shape[1], 1) if x.shape[1] != h else x
        return torch.nn.functional.pad(x, (0, 0, 0, pad)).reshape(b, h, chunks, size, x.shape[-1])
    q, k, v = split(s["q"]), split(s["k"]), split(s["v"])
    beta = split(s["beta"][..., None])                                            # [b, h, chunks, size, 1]
    run_log = split(s["log_decay"][..., None]).squeeze(-1).double().cumsum(-1)    # [b, h, chunks, size]
    i = torch.arange(size, device=DEVICE)
    apart = run_log[..., :, None] - run_log[..., None, :]
    decay = torch.where(i[:, None] >= i, apart.clamp_max(0.0).exp(), 0.0).float()       # from token j to i
    del apart
    since = run_log.exp().float()[..., None]                                      # from the chunk's begin
    left = (run_log[..., -1:] - run_log).exp().float()[..., None]                 # to the chunk's end
    whole = run_log[..., -1].exp().float()[..., None, None]
    among = beta * torch.where(i[:, None] > i, (k @ k.transpose(-1, -2)) * decay, 0.0)
    # rows of (1 + among)^-1 [beta v | beta since k], one after the other
    solved = torch.cat((beta * v, beta * since * k), -1)
    for r in range(1, size):
        solved[..., r, :] -= (among[..., r, None, :r] @ solved[..., :r, :]).squeeze(-2)
    fresh, seen = solved[..., :dv], solved[..., dv:]
    pairs = (q @ k.transpose(-1, -2)) * decay
    k_left = (k * left).transpose(-1, -2)
    state = s["state"].clone()
    out = torch.empty(b, h, chunks, size, dv, device=DEVICE)
    for j in range(chunks):
        u = fresh[:, :, j] - seen[:, :, j] @ state
        out[:, :, j] = (since[:, :, j] * q[:, :, j]) @ state + pairs[:, :, j] @ u
        state = whole[:, :, j] * state + k_left[:, :, j] @ u
    out = (out * s["scale"]).reshape(b, h, chunks * size, dv)[:, :, :n].transpose(1, 2)
    return {"out": torch.where(there[:, :, None, None], out, 0.0).to(s["q"].dtype), "state": state}


def _plain_differential(s):
    c = s["case"]
    hq, hk = c["q_heads"], c["kv_heads"]

    def heads(x):                                    # [b, n, h, d] -> [b, hq, n, d] in fp32
        x = x.transpose(1, 2).float()
        return x.repeat_interleave(hq // x.shape[1], 1) if x.shape[1] != hq else x.contiguous()
    v = heads(s["v"])
    seen = torch.ones(c["batch"], c["k_tokens"], dtype=torch.bool, device=DEVICE)
    if s["lengths"] is not None:
        seen = torch.arange(c["k_tokens"], device=DEVICE) < s["lengths"][:, None]
    if s["mask"] is not None:
        seen = seen & (s["mask"] != 0)

    def look(which):
        score = (heads(s["q"][:, :, which::2]) * s["scale"]) @ heads(s["k"][:, :, which::2]).transpose(-1, -2).contiguous()
        score = score.masked_fill(~seen[:, None, None], -math.inf)
        top = score.max(-1, keepdim=True).values
        p = (score - torch.where(top == -math.inf, 0.0, top)).exp_()
        total = p.sum(-1, keepdim=True)
        return (p @ v) / torch.where(total == 0, 1.0, total)
    y = look(0) - s["lambda"][:, None, None] * look(1)
    if s["weight"] is not None:
        y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + EPS) * s["weight"]
    return {"out": y.transpose(1, 2).to(s["q"].dtype)}


def _plain_experts(s):
    c = s["case"]
    x, f, top = s["x"], c["hidden"], c["top"]
    # the choice in 64 bits: two experts may be next to each other
    score = x.double() @ s["router"].double().T
    ranked = score.sort(dim=-1, descending=True, stable=True)            # ties: the lowest index first
    chosen = ranked.indices[:, :top].to(torch.int32)
    p = (ranked.values - ranked.values[:, :1]).exp()
    p = (p[:, :top] / p[:, :top if c["renormalise"] else None].sum(-1, keepdim=True)).float()
    if s["mask"] is not None:
        here = s["mask"][:, None] != 0
        chosen, p = torch.where(here, chosen, -1), torch.where(here, p, 0.0)
    out = torch.zeros(c["tokens"], c["channels"], device=DEVICE)
    for e in range(c["experts"]):
        hit, slot = torch.nonzero(chosen == e, as_tuple=True)
        if len(hit) == 0:
            continue
        a = x[hit].float() @ s["w_in"][e].float().T
        a = a[:, :f] / (1 + (-a[:, :f]).exp()) * a[:, f:]
        out[hit] += p[hit, slot, None] * (a @ s["w_out"][e].float().T)
    return {"out": out.to(x.dtype), "chosen": chosen, "weights": p}


# ---- the library's operators ------------------------------------------------------------------------
_context = None


def _plan(s):
    """What a program sets up once for its buffers: descriptions, outputs and a workspace."""
    global _context
    import paper_2402_04466_amd as hs
    from paper_2402_04466_amd.harness import gates_of, heads_of
    if _context is None:
        _context = hs.hs_init(0)
    c = s["case"]

    def like(x, *shape):
        return torch.empty(shape or x.shape, dtype=x.dtype, device=x.device)

    def pointer(x):
        return 0 if x is None else x.data_ptr()

    def workspace(desc, need):
        work = torch.empty(need, dtype=torch.uint8, device=DEVICE)
        desc.d_workspace, desc.workspace_bytes = (work.data_ptr() if need else None), need
        return work
    dtype = hs.HS_F16 if c["dtype"] == "fp16" else hs.HS_BF16
    if c["op"] == "delta_rule":
        out = {"out": like(s["q"], c["batch"], c["tokens"], c["heads"], c["value_dim"]), "state": like(s["state"])}
        d = hs.make_delta_rule_desc(
            dtype=dtype, batch=c["batch"], tokens=c["tokens"], heads=c["heads"], qk_heads=c["qk_heads"],
            key_dim=c["key_dim"], value_dim=c["value_dim"], scale=s["scale"], q=heads_of(s["q"]), k=heads_of(s["k"]),
            v=heads_of(s["v"]), out=heads_of(out["out"]), log_decay=gates_of(s["log_decay"]), beta=gates_of(s["beta"]),
            d_lengths=pointer(s["lengths"]), d_state_in=pointer(s["state"]), d_state_out=pointer(out["state"]))
        work = workspace(d, hs.hs_query_delta_rule_workspace(d))
        return (lambda stream, keep=work: hs.hs_delta_rule(_context, d, stream)), out
    if c["op"] == "differential_attention":
        out = {"out": like(s["q"], c["batch"], c["q_tokens"], c["q_heads"], c["value_dim"])}
        d = hs.make_differential_attention_desc(
            dtype=dtype, batch=c["batch"], q_tokens=c["q_tokens"], k_tokens=c["k_tokens"], q_heads=c["q_heads"],
            kv_heads=c["kv_heads"], head_dim=c["dim"], value_dim=c["value_dim"], scale=s["scale"], q=heads_of(s["q"]),
            k=heads_of(s["k"]), v=heads_of(s["v"]), out=heads_of(out["out"]), d_lambda=pointer(s["lambda"]),
            norm=c["norm"], eps=EPS, d_norm_weight=pointer(s["weight"]), d_lengths=pointer(s["lengths"]),
            d_mask=pointer(s["mask"]), mask_batch_stride=c["k_tokens"])
        work = workspace(d, hs.hs_query_differential_attention_workspace(d))
        return (lambda stream, keep=work: hs.hs_differential_attention(_context, d, stream)), out
    out = {"out": like(s["x"]),
           "chosen": torch.empty(c["tokens"], c["top"], dtype=torch.int32, device=DEVICE),
           "weights": torch.empty(c["tokens"], c["top"], device=DEVICE)}
    d = hs.make_expert_layer_desc(
        dtype=dtype, tokens=c["tokens"], channels=c["channels"], hidden=c["hidden"], experts=c["experts"], top=c["top"],
        renormalise=c["renormalise"], d_x=s["x"].data_ptr(), x_stride=s["x"].stride(0), d_out=out["out"].data_ptr(),
        out_stride=out["out"].stride(0), d_router=s["router"].data_ptr(), d_w_in=s["w_in"].data_ptr(),
        d_w_out=s["w_out"].data_ptr(), d_mask=pointer(s["mask"]), d_chosen=out["chosen"].data_ptr(),
        d_weights=out["weights"].data_ptr())
    work = workspace(d, hs.hs_query_expert_layer_workspace(d))
    return (lambda stream, keep=work: hs.hs_expert_layer(_context, d, stream)), out


_PLAIN = {"delta_rule": _plain_delta, "differential_attention": _plain_differential, "expert_layer": _plain_experts}


def run(state):
    if not own:
        return _PLAIN[state["case"]["op"]](state)
    if "plan" not in state:
        state["plan"] = _plan(state)
    call, out = state["plan"]
    call(torch.cuda.current_stream().cuda_stream)
    return out


# ---- the definitions in 64 bits ---------------------------------------------------------------------
def exact(case, seed):
    s, c = prepare(case, seed), case
    if c["op"] == "delta_rule":
        h, n, b = c["heads"], c["tokens"], c["batch"]
        key_of = torch.arange(h, device=DEVICE) // (h // c["qk_heads"])
        state = s["state"].double()
        out = torch.zeros(b, n, h, c["value_dim"], dtype=torch.float64, device=DEVICE)
        order = torch.arange(b, device=DEVICE)
        if s["lengths"] is not None:                 # longest first: those that still run stay in front
            order = s["lengths"].argsort(descending=True)
            running = (torch.arange(n, device=DEVICE)[:, None] < s["lengths"]).sum(1).tolist()
        q, k, v, gate, beta = (s[x][order] for x in ("q", "k", "v", "log_decay", "beta"))
        state, result = state[order].contiguous(), torch.zeros_like(out)
        for t in range(n):                           # token by token
            m = b if s["lengths"] is None else running[t]
            if m == 0:
                break
            kt, qt = k[:m, t].double()[:, key_of], q[:m, t].double()[:, key_of]
            here = state[:m]
            here *= gate[:m, t].double().exp()[..., None, None]
            told = v[:m, t].double() - (kt[..., None, :] @ here).squeeze(-2)
            here += kt[..., None] * (beta[:m, t].double()[..., None] * told)[..., None, :]
            result[:m, t] = (qt[..., None, :] @ here).squeeze(-2) * s["scale"]
        out[order], final = result, torch.empty_like(state)
        final[order] = state
        return {"out": out, "state": final}
    if c["op"] == "differential_attention":
        b, hq, nq, nk = c["batch"], c["q_heads"], c["q_tokens"], c["k_tokens"]
        group = hq // c["kv_heads"]
        out = torch.zeros(b, nq, hq, c["value_dim"], dtype=torch.float64, device=DEVICE)
        for m in range(b):
            keys = torch.arange(nk, device=DEVICE)
            if s["lengths"] is not None:
                keys = keys[:int(s["lengths"][m])]
            if s["mask"] is not None:
                keys = keys[s["mask"][m, :len(keys)] != 0]
            if not len(keys):
                continue
            for h in range(hq):
                v = s["v"][m, keys, h // group].double()
                q1, q2 = s["q"][m, :, 2 * h].double(), s["q"][m, :, 2 * h + 1].double()
                k1, k2 = (s["k"][m, keys, 2 * (h // group) + w].double() for w in (0, 1))
                maps = torch.softmax(s["scale"] * (q1 @ k1.T), -1)
                maps -= s["lambda"][h].double() * torch.softmax(s["scale"] * (q2 @ k2.T), -1)
                y = maps @ v
                if s["weight"] is not None:
                    y = y / (y.pow(2).sum(-1, keepdim=True) / c["value_dim"] + EPS).sqrt() * s["weight"].double()
                out[m, :, h] = y
        return {"out": out}
    x, t = s["x"].double(), c["tokens"]
    logits = (x[:, None, :] * s["router"].double()).sum(-1)
    p = torch.softmax(logits, -1)
    chosen = torch.full((t, c["top"]), -1, dtype=torch.int32, device=DEVICE)
    weights = torch.zeros(t, c["top"], dtype=torch.float64, device=DEVICE)
    free = torch.ones_like(p, dtype=torch.bool)
    number = torch.arange(c["experts"], device=DEVICE)
    rows = torch.arange(t, device=DEVICE)
    for i in range(c["top"]):                        # the largest that is left, the first of them
        left = torch.where(free, logits, -math.inf)
        best = torch.where(left == left.max(-1, keepdim=True).values, number, c["experts"]).min(-1).values
        chosen[:, i], weights[:, i] = best.to(torch.int32), p[rows, best]
        free[rows, best] = False
    if c["renormalise"]:
        weights = weights / weights.sum(-1, keepdim=True)
    if s["mask"] is not None:
        chosen[s["mask"] == 0], weights[s["mask"] == 0] = -1, 0.0
    out = torch.zeros(t, c["channels"], dtype=torch.float64, device=DEVICE)
    for e in range(c["experts"]):
        share = torch.where(chosen == e, weights, 0.0).sum(-1)
        picks = torch.nonzero((chosen == e).any(-1)).flatten()
        w = s["w_in"][e].double()
        gate, value = x[picks] @ w[:c["hidden"]].T, x[picks] @ w[c["hidden"]:].T
        out[picks] += share[picks, None] * ((gate * torch.sigmoid(gate) * value) @ s["w_out"][e].double().T)
    return {"out": out, "chosen": chosen, "weights": weights}
