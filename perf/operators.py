"""The operators between the q/k/v linears and the o linear of a decoder layer, as cases that can be timed and checked:
rotary positions, norms of queries and keys with the rotation, appending to a paged cache, and attention for a batch whose
sequences share a prefix.

`listed()` are the fixed cases, `draw()` gives more of the same ranges; `prepare()` makes what a program holds before the
call, `run()` is one pass (through the framework where `own` is true, in elementary torch operations elsewhere), `work()`
the bytes and operations a pass cannot do without, `exact()` the outputs in 64 bits.

A batch is described the way a serving program holds it: keys and values of every sequence in pages of a cache
[pages, kv heads, page size, head dim], `page_table[b]` the pages of sequence b, `lengths[b]` the tokens it had in the
cache before this step, and `cu_tokens[b]` the first of its new tokens in q, k and v.  The shared prefix has its own list
of pages and comes before every sequence's own tokens, in positions as in attention.
"""
import math
import random

import torch

own = False

THETA = 500000.0
EPS = 1e-5


# ---- cases -------------------------------------------------------------------------------------------------------

def _heads(op, T, q=32, kv=8, dim=128, rot=128, layout="half", scaling="none", start=0, dtype="bf16", **more):
    """A rotation (with or without the norm) of q heads and kv heads of T tokens at positions from `start` on."""
    return dict({"op": op, "T": T, "q": q, "kv": kv, "dim": dim, "rot": rot, "layout": layout, "scaling": scaling,
                 "start": start, "dtype": dtype}, **more)


def _batch(op, B, new, held, page, prefix, q=32, kv=8, dim=128, rot=128, layout="half", dtype="bf16", ragged=0, **more):
    """B sequences with up to `new` new tokens each on top of up to `held` in the cache, after a prefix of `prefix`."""
    return dict({"op": op, "B": B, "new": new, "held": held, "page": page, "prefix": prefix, "q": q, "kv": kv, "dim": dim,
                 "rot": rot, "layout": layout, "dtype": dtype, "ragged": ragged}, **more)


def listed():
    return [
        # One sequence generating: the rotation of one token's 32 query and 8 key heads.  Latency counts.
        dict(_heads("rotary", 1, start=2048), name="rotary_1"),
        # A prompt through the attention of the smaller model.
        dict(_heads("rotary", 4096), name="rotary_4096"),
        # Training on long contexts, the backward pass: gradients turned back, half of the head, interleaved pairs,
        # frequencies scaled in bands, the 40 heads of the larger model.
        dict(_heads("rotary", 8192, 40, 40, rot=64, layout="interleaved", scaling="bands", start=120000, inverse=True),
             name="rotary_grad_8192"),
        # A decode batch of a model with normed queries and keys.
        dict(_heads("norm", 64, start=2048), name="norm_64"),
        # A training step on one sequence: forward, then gradients of q, k and both gains.
        dict(_heads("norm", 4096, train=True), name="norm_train_4096"),
        # The same by hand in fp32, a ragged number of tokens.
        dict(_heads("norm", 257, dtype="f32", train=True), name="norm_train_257_fp32"),
        # A decode batch: one new token of each of 64 sequences into pages of 16.
        dict(_batch("append", 64, 1, 255, 16, 2048), name="append_64"),
        # Prompts of eight requests of different lengths, normed queries and keys, pages of 64.
        dict(_batch("append", 8, 700, 0, 64, 0, ragged=300, norm=True), name="append_prompts"),
        # One sequence generating after a short system prompt.  Latency counts.
        dict(_batch("attend", 1, 1, 37, 16, 2048), name="attend_1"),
        # A decode batch over a system prompt, answers of different lengths.
        dict(_batch("attend", 64, 1, 512, 16, 2048, ragged=400), name="attend_64"),
        # A large decode batch over a long shared document.
        dict(_batch("attend", 128, 1, 1024, 64, 32768, ragged=1000), name="attend_128_long"),
        # Questions of up to 100 tokens over a shared document, the 40 heads of the larger model, each its own keys.
        dict(_batch("attend", 16, 100, 300, 32, 8192, 40, 40, ragged=90), name="attend_questions"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("rotary", "norm", "append", "attend", "attend", "attend"))
    q, kv = rng.choice(((32, 8), (32, 8), (40, 40), (12, 4), (16, 1)))
    dim = rng.choice((128, 128, 128, 64, 80, 256))
    rot = rng.choice((dim, dim, dim // 2))
    layout = rng.choice(("half", "interleaved"))
    dtype = rng.choice(("bf16", "bf16", "bf16", "bf16", "f32"))
    if op in ("rotary", "norm"):
        case = _heads(op, _log_int(rng, 1, 8192), q, kv, dim, rot, layout, rng.choice(("none", "linear", "bands")),
                      _log_int(rng, 1, 1000000) - 1, dtype)
        case["inverse" if op == "rotary" else "train"] = rng.random() < 0.5
        return case
    page = rng.choice((16, 16, 32, 64, 128, 24))
    B = _log_int(rng, 1, 128)
    if op == "append":
        new = rng.choice((1, _log_int(rng, 2, max(2, 4096 // B))))
        return _batch(op, B, new, rng.randrange(0, 256), page, _log_int(rng, 1, 100000) - 1, q, kv, dim, rot, layout, dtype,
                      ragged=rng.randrange(0, new + 1), norm=rng.random() < 0.5)
    if dtype == "f32":
        B = min(B, 32)
    new = rng.choice((1, 1, _log_int(rng, 2, max(2, 1024 // B))))
    held, prefix = _log_int(rng, 1, 1024) - 1, _log_int(rng, 1, 32768 if new == 1 and dtype == "bf16" else 4096)
    return _batch(op, B, new, held, page, prefix, q, kv, dim, rot, layout, dtype, ragged=rng.randrange(0, held + new))


def _lengths(case):
    """(new, held) of every sequence: both fall from their largest value by up to `ragged`, in an order without a pattern."""
    B, ragged = case["B"], case["ragged"]
    order = list(range(B))
    random.Random(B * 1000003 + ragged).shuffle(order)
    drop = [ragged * i // max(B - 1, 1) for i in order]
    return [max(1, case["new"] - d) for d in drop], [max(0, case["held"] - d) for d in drop]


def _rows(case):
    return case["T"] if "T" in case else sum(_lengths(case)[0])


# ---- inputs ------------------------------------------------------------------------------------------------------

def _dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _scaling(case):
    """Arguments of the frequencies' scaling: contexts eight times the 8192 tokens the model was trained on."""
    return {"none": {}, "linear": {"scaling": "linear", "factor": 8.0},
            "bands": {"scaling": "bands", "factor": 8.0, "original_context": 8192, "low": 1.0, "high": 4.0,
                      "attention_scale": 0.1 * math.log(8.0) + 1.0}}[case.get("scaling", "none")]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dtype, T, Hq, Hk, D = _dtype(case), _rows(case), case["q"], case["kv"], case["dim"]
    rand = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    s = {"case": case, "q": rand(T, Hq, D).to(dtype)}
    gain = lambda: (1.0 + 0.1 * rand(D)).to(dtype)  # noqa: E731
    if case["op"] != "attend":
        s["k"] = rand(T, Hk, D).to(dtype)
    if own and case["op"] != "attend":
        from paper_2405_13053_b200 import binding as mb
        s["rot"] = mb.meteora_rotary_init(case["rot"], THETA, case["layout"], **_scaling(case))
    if case["op"] == "norm" or case.get("norm"):
        s["gq"], s["gk"] = gain(), gain()
    if "T" in case:
        s["positions"] = case["start"] + torch.arange(T, device="cuda")
        if case.get("train"):
            s["dq"], s["dk"] = rand(T, Hq, D).to(dtype), rand(T, Hk, D).to(dtype)
        return s
    # a batch over a paged cache; a program holds these tables on the device and keeps the host's copy of the plan
    new, held = _lengths(case)
    B, page, P = case["B"], case["page"], case["prefix"]
    width = max((h + n + page - 1) // page for n, h in zip(new, held))
    prefix_pages = (P + page - 1) // page if case["op"] == "attend" else 0
    pages = B * width + prefix_pages
    order = torch.randperm(pages, device="cuda", generator=g).to(torch.int32)
    channel = rand(1, Hk, 1, D)                       # values have a mean of their own in every channel
    s["k_cache"] = rand(pages, Hk, page, D).to(dtype)
    s["v_cache"] = (0.5 * rand(pages, Hk, page, D) + channel).to(dtype)
    s["page_table"] = order[:B * width].view(B, width).contiguous()
    s["prefix_pages"] = order[B * width:].contiguous()
    s["lengths"] = torch.tensor(held, dtype=torch.int32, device="cuda")
    s["cu_tokens"] = torch.tensor([sum(new[:b]) for b in range(B + 1)], dtype=torch.int32, device="cuda")
    s["one_each"] = max(new) == 1
    s["widest"], s["width"] = max(new), width
    if case["op"] == "append":
        s["v"] = (0.5 * rand(T, Hk, D) + channel[0, :, 0]).to(dtype)
    elif own:
        from paper_2405_13053_b200 import binding as mb
        s["workspace"] = mb.meteora_prefix_attention_workspace(s["q"], s["k_cache"], s["page_table"], P)
    return s


# ---- one pass ----------------------------------------------------------------------------------------------------

def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_2405_13053_b200 import binding as mb
    case = s["case"]
    if case["op"] == "rotary":
        return mb.meteora_rotary(s["q"], s["k"], s["positions"], s["rot"], inverse=case.get("inverse", False))
    if case["op"] == "norm":
        out = mb.meteora_head_norm_rotary(s["q"], s["k"], s["gq"], s["gk"], s["positions"], s["rot"], eps=EPS)
        if not case.get("train"):
            return out
        return out + mb.meteora_head_norm_rotary_backward(s["dq"], s["dk"], s["q"], s["k"], s["gq"], s["gk"],
                                                          s["positions"], s["rot"], eps=EPS)
    cu = None if s["one_each"] else s["cu_tokens"]
    if case["op"] == "append":
        q = mb.meteora_cache_append(s["k"], s["v"], s["k_cache"], s["v_cache"], s["page_table"], s["lengths"], s["rot"],
                                    cu_tokens=cu, prefix_len=case["prefix"], q=s["q"], q_gain=s.get("gq"),
                                    k_gain=s.get("gk"), eps=EPS)
        return q, s["k_cache"], s["v_cache"]
    return mb.meteora_prefix_attention(s["q"], s["k_cache"], s["v_cache"], s["page_table"], s["lengths"],
                                       s["prefix_pages"], case["prefix"], cu_tokens=cu, workspace=s["workspace"])


def _angles(case, positions):
    """cos and sin [T, 1, rot / 2] in fp32; the angles of far positions are worked out in fp64."""
    rot, how = case["rot"], _scaling(case)
    f = THETA ** (-torch.arange(0, rot, 2, device=positions.device, dtype=torch.float64) / rot)
    if how.get("scaling") == "linear":
        f = f / how["factor"]
    if how.get("scaling") == "bands":
        turns = how["original_context"] * f / (2 * math.pi)
        keep = ((turns - how["low"]) / (how["high"] - how["low"])).clamp(0, 1)
        f = f * (keep + (1 - keep) / how["factor"])
    a = positions.double()[:, None, None] * f
    scale = how.get("attention_scale", 1.0)
    return (a.cos() * scale).float(), (a.sin() * scale).float()


def _turn(case, x, cos, sin):
    """x[T, heads, dim] in fp32, its first `rot` entries turned."""
    rot = case["rot"]
    if case["layout"] == "half":
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)
    else:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2)
    return torch.cat([turned, x[..., rot:]], dim=-1)


def _norm(x, g):
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    return x * r * g, r


def _run_plain(s):
    case = s["case"]
    dtype = _dtype(case)
    if case["op"] == "attend":
        return _attend_plain(s)
    q, k = s["q"].float(), s["k"].float()
    if case["op"] == "append":
        return _append_plain(s, q, k)
    cos, sin = _angles(case, s["positions"])
    if case["op"] == "rotary":
        sin = -sin if case.get("inverse") else sin
        return _turn(case, q, cos, sin).to(dtype), _turn(case, k, cos, sin).to(dtype)
    out, back = [], []
    for x, g, d in ((q, s["gq"], s.get("dq")), (k, s["gk"], s.get("dk"))):
        g = g.float()
        n, r = _norm(x, g)
        out.append(_turn(case, n, cos, sin).to(dtype))
        if case.get("train"):
            dn = _turn(case, d.float(), cos, -sin)
            unit = x * r
            back.append((r * (g * dn - unit * (g * dn * unit).mean(-1, keepdim=True))).to(dtype))
            back.append((dn * unit).sum((0, 1)))
    return (*out, back[0], back[2], back[1], back[3]) if back else tuple(out)


def _tokens(s):
    """Sequence and place among its own tokens of every new token."""
    cu = s["cu_tokens"].long()
    t = torch.arange(s["q"].shape[0], device="cuda")
    b = torch.searchsorted(cu, t, right=True) - 1
    return b, s["lengths"].long()[b] + t - cu[b]


def _append_plain(s, q, k):
    case, dtype, page = s["case"], _dtype(s["case"]), s["case"]["page"]
    b, at = _tokens(s)
    cos, sin = _angles(case, case["prefix"] + at)
    if case.get("norm"):
        q, k = _norm(q, s["gq"].float())[0], _norm(k, s["gk"].float())[0]
    where = s["page_table"].long()[b, at // page]
    s["k_cache"][where, :, at % page] = _turn(case, k, cos, sin).to(dtype)
    s["v_cache"][where, :, at % page] = s["v"]
    return _turn(case, q, cos, sin).to(dtype), s["k_cache"], s["v_cache"]


def _attend_plain(s):
    case, T = s["case"], s["q"].shape[0]
    Hq, Hk, D, B, P, page = case["q"], case["kv"], case["dim"], case["B"], case["prefix"], case["page"]
    G, W, S = Hq // Hk, s["widest"], s["width"] * page
    b, at = _tokens(s)
    q = s["q"].float().view(T, Hk, G, D) / math.sqrt(D)
    flat = lambda c, pages: c[pages.long()].float().transpose(0, 1).reshape(Hk, -1, D)[:, :P]  # noqa: E731
    kp, vp = flat(s["k_cache"], s["prefix_pages"]), flat(s["v_cache"], s["prefix_pages"])
    of = lambda c: c[s["page_table"].long()].float().transpose(1, 2).reshape(B, Hk, S, D)  # noqa: E731
    ks, vs = of(s["k_cache"]), of(s["v_cache"])
    # the prefix: the rows of all sequences in one product per kv head; own tokens: rows by sequence, short ones padded
    place = b * W + at - s["lengths"].long()[b]
    mine = torch.zeros(B * W, Hk, G, D, device="cuda")
    mine[place] = q
    mine = mine.view(B, W, Hk, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hk, W * G, D)
    late = (mine @ ks.transpose(2, 3)).view(B, Hk, W, G, S).transpose(1, 2).reshape(B * W, Hk, G, S)[place]
    seen = torch.arange(S, device="cuda") <= at[:, None]
    late = late.masked_fill(~seen[:, None, None], -math.inf)
    early = (q.transpose(0, 1).reshape(Hk, T * G, D) @ kp.transpose(1, 2)).view(Hk, T, G, P).transpose(0, 1)
    top = torch.maximum(late.amax(-1, keepdim=True), early.amax(-1, keepdim=True))
    late, early = torch.exp(late - top), torch.exp(early - top)
    total = late.sum(-1, keepdim=True) + early.sum(-1, keepdim=True)
    weights = torch.zeros(B * W, Hk, G, S, device="cuda")
    weights[place] = late
    o = (weights.view(B, W, Hk, G, S).permute(0, 2, 1, 3, 4).reshape(B, Hk, W * G, S) @ vs)
    o = o.view(B, Hk, W, G, D).transpose(1, 2).reshape(B * W, Hk, G, D)[place]
    o = o + (early.transpose(0, 1).reshape(Hk, T * G, P) @ vp).view(Hk, T, G, D).transpose(0, 1)
    return (o / total).view(T, Hq, D).to(s["q"].dtype)


# ---- what a pass cannot do without -------------------------------------------------------------------------------

def work(case):
    es, T, Hq, Hk, D = 4 if case["dtype"] == "f32" else 2, _rows(case), case["q"], case["kv"], case["dim"]
    rows = T * (Hq + Hk)
    if case["op"] == "rotary":
        return {"bytes": 2 * es * rows * D + 8 * T, "flops": 3 * rows * case["rot"]}
    if case["op"] == "norm":
        back = case.get("train", False)      # q and k are read by both passes
        return {"bytes": es * rows * D * (5 if back else 2) + 2 * es * D + (8 * D if back else 0) + 8 * T,
                "flops": rows * (3 * case["rot"] + 4 * D) * (3 if back else 1)}
    if case["op"] == "append":
        return {"bytes": 2 * es * (rows + T * Hk) * D + 12 * case["B"], "flops": 3 * rows * case["rot"]}
    new, held = _lengths(case)
    seen = T * case["prefix"] + sum(n * h + n * (n + 1) // 2 for n, h in zip(new, held))
    keys = case["prefix"] + sum(new) + sum(held)
    return {"bytes": 2 * es * (keys * Hk + T * Hq) * D + 12 * case["B"] + 4 * (keys // case["page"]),
            "flops": 4 * seen * Hq * D}


# ---- the operators' definitions in 64 bits -----------------------------------------------------------------------

def _rotate64(case, x, position):
    """x[..., heads, dim] as complex pairs, multiplied by e^(i angle)."""
    rot, how = case["rot"], _scaling(case)
    f = torch.tensor([THETA ** (-2.0 * i / rot) for i in range(rot // 2)], dtype=torch.float64)
    if "factor" in how:
        for i in range(rot // 2):
            keep = 0.0
            if how["scaling"] == "bands":
                wavelength = 2 * math.pi / float(f[i])
                keep = (how["original_context"] / wavelength - how["low"]) / (how["high"] - how["low"])
                keep = min(1.0, max(0.0, keep))
            f[i] = (1 - keep) * f[i] / how["factor"] + keep * f[i]
    angle = position.double()[:, None, None] * f.to(x.device)
    e = torch.polar(torch.full_like(angle, how.get("attention_scale", 1.0)), angle if not case.get("inverse") else -angle)
    part = x[..., :rot].unflatten(-1, (2, -1)).transpose(-1, -2) if case["layout"] == "half" else x[..., :rot].unflatten(-1, (-1, 2))
    y = torch.view_as_real(torch.view_as_complex(part.contiguous()) * e)
    y = y.transpose(-1, -2).flatten(-2) if case["layout"] == "half" else y.flatten(-2)
    return torch.cat([y, x[..., rot:]], dim=-1)


def _norm64(x, g):
    return x / torch.sqrt(x.square().sum(-1, keepdim=True) / x.shape[-1] + EPS) * g


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "attend":
        return _attend64(s)
    q, k = s["q"].double(), s["k"].double()
    if op == "rotary":
        return _rotate64(case, q, s["positions"]), _rotate64(case, k, s["positions"])
    if op == "norm":
        gains = [s["gq"].double(), s["gk"].double()]
        if not case.get("train"):
            return tuple(_rotate64(case, _norm64(x, g), s["positions"]) for x, g in zip((q, k), gains))
        leaves = [t.requires_grad_() for t in (q, k, *gains)]
        with torch.enable_grad():
            y = [_rotate64(case, _norm64(x, g), s["positions"]) for x, g in ((q, gains[0]), (k, gains[1]))]
            grads = torch.autograd.grad(y, leaves, [s["dq"].double(), s["dk"].double()])
        return (*(t.detach() for t in y), *grads)
    new, held = _lengths(case)
    kc, vc, v = s["k_cache"].double(), s["v_cache"].double(), s["v"].double()
    own_place = torch.cat([torch.arange(h, h + n) for n, h in zip(new, held)]).to(q.device)
    if case.get("norm"):
        q, k = _norm64(q, s["gq"].double()), _norm64(k, s["gk"].double())
    q, k = _rotate64(case, q, own_place + case["prefix"]), _rotate64(case, k, own_place + case["prefix"])
    table, t = s["page_table"].tolist(), 0
    for b in range(case["B"]):
        for i in range(held[b], held[b] + new[b]):
            kc[table[b][i // case["page"]], :, i % case["page"]] = k[t]
            vc[table[b][i // case["page"]], :, i % case["page"]] = v[t]
            t += 1
    return q, kc, vc


def _attend64(s):
    """Sequence by sequence, kv head by kv head: softmax over the prefix and the tokens up to the query's own."""
    case = s["case"]
    new, held = _lengths(case)
    G, D, P = case["q"] // case["kv"], case["dim"], case["prefix"]
    out = torch.empty(s["q"].shape, dtype=torch.float64, device=s["q"].device)
    lay = lambda c, pages: c[pages.long()].double().permute(1, 0, 2, 3).flatten(1, 2)  # noqa: E731
    kp, vp = (lay(c, s["prefix_pages"])[:, :P] for c in (s["k_cache"], s["v_cache"]))
    t = 0
    for b, (n, h) in enumerate(zip(new, held)):
        ks, vs = (lay(c, s["page_table"][b])[:, :h + n] for c in (s["k_cache"], s["v_cache"]))
        hidden = torch.ones(n, P + h + n, dtype=torch.bool, device=ks.device).triu(P + h + 1)
        for i in range(case["kv"]):
            keys, values = torch.cat([kp[i], ks[i]]), torch.cat([vp[i], vs[i]])
            x = s["q"][t:t + n, i * G:(i + 1) * G].double() @ keys.T / math.sqrt(D)
            w = torch.softmax(x.masked_fill(hidden[:, None], -math.inf), dim=-1)
            out[t:t + n, i * G:(i + 1) * G] = w @ values
        t += n
    return out
