"""Cases, plain forms and exact values of four operators of batched decoding:

  rotate    rotary positions turned into rows of Q and K (halves or pairs, part of the head, scaled frequencies)
  append    K/V rows written into a paged cache, rotated on the way (with the query rows of the same projection)
  attend    softmax attention of each sequence's new rows over its pages: one new token, or a window of rows
  logprobs  log probabilities of given tokens, their ranks, the entropy and the most probable tokens of each row

`own` False: elementary torch operations; True: the library's entry points.
"""
import math
import random

import numpy as np
import torch

own = False

REAL = {"bf16": torch.bfloat16, "f32": torch.float32}
HALVES, PAIRS = "halves", "pairs"
# scaling of the frequencies for contexts longer than the trained one: (base, kind, factor, low, high, trained length)
SCALING = {
    "plain": (500000.0, 1.0, 1.0, 1.0, 1),
    "linear": (10000.0, 4.0, 1.0, 1.0, 4096),
    "ntk": (10000.0, 8.0, 1.0, 1.0, 4096),
    "bands": (500000.0, 8.0, 1.0, 4.0, 8192),
    "yarn": (1000000.0, 4.0, 1.0, 32.0, 32768),
}


# ---- cases -----------------------------------------------------------------------------------------
def _rotate(name, dtype, heads, extra, d, rot, layout, scaling, rows, far, inverse):
    """heads turned out of rows of heads + extra heads (a fused projection); positions up to `far`."""
    return dict(name=name, op="rotate", dtype=dtype, heads=heads, extra=extra, d=d, rot=rot, layout=layout, scaling=scaling,
                rows=rows, far=far, inverse=inverse)


def _append(name, dtype, H, Hkv, d, rot, layout, scaling, n, longest, window, mix, page, heads_first, listed):
    """n sequences of up to `longest` tokens, of which up to `window` are new (window 1: one each; the whole sequence
    where it is shorter); listed: at listed positions instead of the last ones.  mix seeds the lengths; 0: all alike."""
    return dict(name=name, op="append", dtype=dtype, H=H, Hkv=Hkv, d=d, rot=rot, layout=layout, scaling=scaling, n=n,
                longest=longest, window=window, mix=mix, page=page, heads_first=heads_first, listed=listed)


def _attend(name, dtype, H, Hkv, d, n, longest, window, mix, page, heads_first, spare=0):
    """spare: rows of the query buffer behind the last sequence's."""
    return dict(name=name, op="attend", dtype=dtype, H=H, Hkv=Hkv, d=d, n=n, longest=longest, window=window, mix=mix,
                page=page, heads_first=heads_first, spare=spare)


def _logprobs(name, dtype, vocab, n_pos, rows, max_rows, temperature, n_top, spread):
    return dict(name=name, op="logprobs", dtype=dtype, vocab=vocab, n_pos=n_pos, rows=rows, max_rows=max_rows,
                temperature=temperature, n_top=n_top, spread=spread)


def listed():
    return [
        # the active rows of one denoising step: queries and keys of an MHA layer
        _rotate("rotate step rows", "bf16", 64, 32, 128, 128, HALVES, "plain", 72, 32768, False),
        # block entry of a long prompt, GQA projection with values beside, frequencies stretched
        _rotate("rotate whole layer", "bf16", 32, 4, 128, 128, HALVES, "yarn", 16384, 131072, False),
        # gradients of a quarter-turned head go back the other way; far positions in fp32
        _rotate("rotate back in part", "f32", 8, 0, 64, 16, PAIRS, "bands", 5000, 1000000, True),
        # one new token for each of 64 requests
        _append("append one token each", "bf16", 28, 4, 128, 128, HALVES, "yarn", 64, 8192, 1, 7, 16, False, False),
        # prompts of unequal length enter the cache
        _append("append prompts", "bf16", 32, 8, 128, 128, HALVES, "bands", 6, 8192, 8192, 3, 64, True, False),
        # one request, one new token, tiny pages of a small fp32 layer
        _attend("attend small f32", "f32", 8, 8, 64, 5, 1024, 1, 5, 32, False),
        # one request at 32K context, one new token: few heads, so the length is what is split
        _attend("attend one token 32K", "bf16", 28, 4, 128, 1, 32768, 1, 0, 64, False),
        # a serving batch: lengths from a few tokens to 16K
        _attend("attend batch", "bf16", 32, 8, 128, 64, 16384, 1, 11, 16, False, 8),
        # multi-head layers at long context: the cache is what is read
        _attend("attend MHA 16K", "bf16", 32, 32, 128, 4, 16384, 1, 0, 128, True),
        # active rows of several denoising requests
        _attend("attend windows", "bf16", 28, 4, 128, 6, 16384, 35, 2, 64, False),
        # one position scored in fp32, five alternatives
        _logprobs("logprobs one row", "f32", 50257, 4, 1, 1, 1.0, 5, 2.5),
        # a scored region of 512 positions, twenty alternatives each
        _logprobs("logprobs 512 rows", "bf16", 126464, 512, 512, 512, 0.8, 20, 3.0),
    ]


HEADS = [(32, 32, 128), (28, 4, 128), (8, 8, 64), (16, 4, 64), (8, 2, 128), (12, 12, 128), (6, 1, 128), (32, 8, 128), (40, 1, 64)]
PAGES = [1, 8, 16, 16, 32, 48, 64, 128, 256]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rotate", "append", "append", "attend", "attend", "attend", "logprobs"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    H, Hkv, d = rng.choice(HEADS)
    layout, scaling = rng.choice([HALVES, HALVES, PAIRS]), rng.choice(sorted(SCALING))
    rot = rng.choice([d, d, d // 2, 16, 48])
    if op == "rotate":
        heads = H + Hkv
        c = _rotate("", dtype, heads, rng.choice([0, Hkv]), d, rot, layout, scaling,
                    _log(rng, 1, 2 ** 25 // (heads * d)), _log(rng, 100, 1000000), rng.random() < 0.3)
    elif op == "append":
        n = _log(rng, 1, 256)
        window = rng.choice([1, 1, 9, 64, 100000])
        longest = _log(rng, 1, min(32768, 2 ** 24 // (n * Hkv * d), 2 ** 26 // (n * (H + 2 * Hkv) * d)))
        c = _append("", dtype, H, Hkv, d, rot, layout, scaling, n, longest, min(window, longest), rng.randrange(0, 1000),
                    rng.choice(PAGES), rng.random() < 0.5, window < 100 and rng.random() < 0.4)
    elif op == "attend":
        n = _log(rng, 1, 256)
        longest = _log(rng, 1, min(65536, 2 ** (26 if dtype == "bf16" else 24) // (n * Hkv * d)))
        window = rng.choice([1, 1, 1, 4, 35])
        window = max(1, min(window, longest, 2 ** 24 // (n * H * longest)))
        c = _attend("", dtype, H, Hkv, d, n, longest, window, rng.randrange(0, 1000), rng.choice(PAGES), rng.random() < 0.5,
                    rng.choice([0, 0, 5]) if window > 1 else 0)
    else:
        vocab = _log(rng, 40, 160000)
        n_pos = _log(rng, 1, max(1, min(512, 60_000_000 // vocab)))
        rows = rng.randint(1, n_pos)
        c = _logprobs("", dtype, vocab, n_pos, rows, rows + rng.randrange(0, 20), round(rng.uniform(0.2, 1.5), 2),
                      rng.choice([1, 1, 5, 20, 32]), round(rng.uniform(0.5, 4.0), 2))
    del c["name"]
    return c


def _lengths(c):
    """Tokens and new rows of each sequence, from the case alone."""
    n, longest, window = c["n"], c["longest"], c["window"]
    if c["mix"] == 0:
        return [longest] * n, [min(window, longest)] * n
    rng = random.Random(c["mix"])
    length = [longest] + [_log(rng, max(1, longest // 100), longest) for _ in range(n - 1)]
    rng.shuffle(length)
    new = [min(t, window if window == 1 or window == longest else rng.randint(1, window)) for t in length]
    return length, new


# ---- inputs ----------------------------------------------------------------------------------------
def _rand(gen, shape, dtype="f32", scale=1.0):
    return (torch.randn(shape, generator=gen, device="cuda") * scale).to(REAL[dtype])


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _starts(new):
    out = [0]
    for k in new:
        out.append(out[-1] + k)
    return out


def _pages(gen, c, s):
    """A pool of pages in the shuffled order that a serving process leaves it in, and the table of who owns which."""
    page, length = c["page"], s["length"]
    need = [(t + page - 1) // page for t in length]
    n_pages, wide = sum(need) + 3, max(need) + 2
    shape = (n_pages, c["Hkv"], page, c["d"]) if c["heads_first"] else (n_pages, page, c["Hkv"], c["d"])
    s["K"], s["V"] = _rand(gen, shape, c["dtype"]), _rand(gen, shape, c["dtype"])
    order = torch.randperm(n_pages, generator=gen, device="cuda").to(torch.int32)
    table, at = torch.full((c["n"], wide), -1, dtype=torch.int32, device="cuda"), 0
    for i, k in enumerate(need):
        table[i, :k] = order[at:at + k]
        at += k
    s["table"], s["kv_len"], s["longest"] = table, _ints(length), max(length)


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    s = {"case": c}
    if c["op"] == "rotate":
        n, heads, d = c["rows"], c["heads"], c["d"]
        s["X"] = _rand(gen, (n, heads + c["extra"], d), c["dtype"])[:, :heads]
        s["Y"] = torch.zeros((n, heads, d), dtype=REAL[c["dtype"]], device="cuda")
        s["positions"] = torch.randint(0, c["far"], (n,), generator=gen, device="cuda").to(torch.int32)
        s["n_rows"] = _ints([n])
    elif c["op"] == "append":
        H, Hkv, d = c["H"], c["Hkv"], c["d"]
        s["length"], s["new"] = _lengths(c)
        _pages(gen, c, s)
        start = _starts(s["new"])
        s["rows"] = start[-1]
        s["row_start"] = None if c["window"] == 1 else _ints(start)
        qkv = _rand(gen, (s["rows"], H + 2 * Hkv, d), c["dtype"])
        s["Q"], s["K_new"], s["V_new"] = qkv[:, :H], qkv[:, H:H + Hkv], qkv[:, H + Hkv:]
        s["Q_out"] = torch.zeros((s["rows"], H, d), dtype=REAL[c["dtype"]], device="cuda")
        s["positions"] = None
        if c["listed"]:
            s["positions"] = torch.cat([torch.randperm(t, generator=gen, device="cuda")[:k].sort().values
                                        for t, k in zip(s["length"], s["new"])]).to(torch.int32)
    elif c["op"] == "attend":
        s["length"], s["new"] = _lengths(c)
        _pages(gen, c, s)
        start = _starts(s["new"])
        s["rows"] = start[-1]
        s["max_rows"] = s["rows"] + c["spare"]
        s["row_start"] = None if c["window"] == 1 and c["spare"] == 0 else _ints(start)
        s["Q"] = _rand(gen, (s["max_rows"], c["H"], c["d"]), c["dtype"])
        s["O"] = torch.zeros((s["max_rows"], c["H"], c["d"]), dtype=REAL[c["dtype"]], device="cuda")
        s["lse"] = torch.zeros((c["H"], s["max_rows"]), device="cuda")
    else:
        n_pos, V, m = c["n_pos"], c["vocab"], c["max_rows"]
        step = 8 if c["dtype"] == "bf16" else 4
        s["logits"] = _rand(gen, (n_pos, (V + step - 1) // step * step), c["dtype"], c["spread"])
        rows = torch.randperm(n_pos, generator=gen, device="cuda")[:c["rows"]].sort().values.to(torch.int32)
        s["rows"] = torch.full((m,), -1, dtype=torch.int32, device="cuda")
        s["rows"][:c["rows"]] = rows
        s["n_rows"] = _ints([c["rows"]])
        # tokens as text has them: mostly probable ones, some far down
        x = s["logits"][rows.long(), :V].float()
        noise = torch.rand((c["rows"], 64), generator=gen, device="cuda")
        cand = torch.randint(0, V, (c["rows"], 64), generator=gen, device="cuda")
        best = (x.gather(1, cand) + 2.0 * noise).argmax(1, keepdim=True)
        s["given"] = torch.full((m,), -1, dtype=torch.int32, device="cuda")
        s["given"][:c["rows"]] = cand.gather(1, best)[:, 0].to(torch.int32)
        s["logprob"], s["entropy"] = torch.zeros((m,), device="cuda"), torch.zeros((m,), device="cuda")
        s["rank"] = torch.zeros((m,), dtype=torch.int32, device="cuda")
        s["top_token"] = torch.zeros((m, c["n_top"]), dtype=torch.int32, device="cuda")
        s["top_logprob"] = torch.zeros((m, c["n_top"]), device="cuda")
    if own and "rot" in c:
        _rope(s)
    return s


# ---- plain forms -----------------------------------------------------------------------------------
def _frequencies(c):
    """Radians per position of each pair (64 bits, on the GPU) and the factor on what is turned."""
    base, factor, low, high, trained = SCALING[c["scaling"]]
    rot = c["rot"]
    i = torch.arange(0, rot, 2, dtype=torch.float64, device="cuda")
    if c["scaling"] == "ntk":
        base = base * factor ** (rot / (rot - 2))
    f = base ** (-i / rot)
    if c["scaling"] == "linear":
        f = f / factor
    elif c["scaling"] == "bands":
        turns = trained * f / (2 * math.pi)                              # within the trained length
        keep = ((turns - low) / (high - low)).clamp(0, 1)
        f = f * keep + f / factor * (1 - keep)
    elif c["scaling"] == "yarn":
        at = [rot * math.log(trained / (t * 2 * math.pi)) / (2 * math.log(base)) for t in (high, low)]
        lo, hi = max(math.floor(at[0]), 0), min(math.ceil(at[1]), rot - 1)
        ramp = ((i / 2 - lo) / max(hi - lo, 0.001)).clamp(0, 1)
        f = f / factor * ramp + f * (1 - ramp)
        return f, 0.1 * math.log(factor) + 1.0
    return f, 1.0


def _turned(x, positions, c, sign=1.0):
    """x [rows, heads, d] with its first c["rot"] elements turned, fp32."""
    rot = c["rot"]
    f, magnitude = _frequencies(c)
    angle = positions.double()[:, None] * f
    cos = (angle.cos() * magnitude).float()[:, None, :]
    sin = (angle.sin() * (magnitude * sign)).float()[:, None, :]
    y = x.float().clone()
    if c["layout"] == HALVES:
        a, b = slice(0, rot // 2), slice(rot // 2, rot)
    else:
        a, b = slice(0, rot, 2), slice(1, rot, 2)
    u, v = y[..., a].clone(), y[..., b].clone()
    y[..., a] = u * cos - v * sin
    y[..., b] = v * cos + u * sin
    return y


def _plain_rotate(s):
    c = s["case"]
    s["Y"].copy_(_turned(s["X"], s["positions"], c, -1.0 if c["inverse"] else 1.0))
    return {"Y": s["Y"]}


def _tokens_first(s, name):
    """The pool as [pages, tokens of a page, Hkv, d], whatever its layout."""
    return s[name].transpose(1, 2) if s["case"]["heads_first"] else s[name]


def _row_owner(s):
    """Sequence and position of every new row, on the GPU."""
    new = _ints(s["new"]).long()
    seq = torch.repeat_interleave(torch.arange(len(s["new"]), device="cuda"), new, output_size=s["rows"])
    if s["positions"] is not None:
        return seq, s["positions"].long()
    start = new.cumsum(0) - new
    t = torch.arange(s["rows"], device="cuda") - start[seq]
    return seq, s["kv_len"].long()[seq] - new[seq] + t


def _plain_append(s):
    c = s["case"]
    seq, pos = _row_owner(s)
    page = s["table"].long()[seq, pos // c["page"]]
    dt = REAL[c["dtype"]]
    _tokens_first(s, "K")[page, pos % c["page"]] = _turned(s["K_new"], pos, c).to(dt)
    _tokens_first(s, "V")[page, pos % c["page"]] = s["V_new"]
    s["Q_out"].copy_(_turned(s["Q"], pos, c))
    return {"Q": s["Q_out"], "K": s["K"], "V": s["V"]}


def _plain_attend(s):
    c = s["case"]
    H, Hkv, d, n, page = c["H"], c["Hkv"], c["d"], c["n"], c["page"]
    hpg, new, start = H // Hkv, s["new"], _starts(s["new"])
    K, V = _tokens_first(s, "K"), _tokens_first(s, "V")
    order = sorted(range(n), key=lambda i: -s["length"][i])              # alike lengths together, so that little is padded
    at = 0
    while at < n:
        longest = s["length"][order[at]]
        k = max(1, min(n - at, 2 ** 28 // (longest * Hkv * d)))
        part = order[at:at + k]
        at += k
        R = max(new[i] for i in part)
        idx, first, count = (torch.tensor(v, device="cuda") for v in (part, [start[i] for i in part], [new[i] for i in part]))
        t = torch.arange(R, device="cuda")
        rows = (first[:, None] + t).clamp(max=s["max_rows"] - 1)
        q = s["Q"][rows].float().reshape(k, R, Hkv, hpg, d).permute(0, 2, 1, 3, 4).reshape(k, Hkv, R * hpg, d)
        pages = s["table"][idx, :(longest + page - 1) // page].long().clamp(min=0)
        kk = K[pages].reshape(k, -1, Hkv, d)[:, :longest].permute(0, 2, 3, 1).float()
        p = torch.matmul(q, kk) * (1.0 / math.sqrt(d))
        del kk
        p.masked_fill_((torch.arange(longest, device="cuda") >= s["kv_len"][idx][:, None])[:, None, None, :], -math.inf)
        m = p.amax(-1, keepdim=True)
        p.sub_(m).exp_()
        z = p.sum(-1, keepdim=True)
        vv = V[pages].reshape(k, -1, Hkv, d)[:, :longest].transpose(1, 2).float()
        o = (torch.matmul(p, vv) / z).reshape(k, Hkv, R, hpg, d).permute(0, 2, 1, 3, 4).reshape(k, R, H, d)
        lse = (m + z.log()).reshape(k, Hkv, R, hpg).permute(0, 2, 1, 3).reshape(k, R, H)
        live = t < count[:, None]
        s["O"][rows[live]] = o[live].to(s["O"].dtype)
        s["lse"][:, rows[live]] = lse[live].transpose(0, 1)
    return {"O": s["O"], "lse": s["lse"]}


def _plain_logprobs(s):
    c = s["case"]
    n, V = c["rows"], c["vocab"]
    x = s["logits"][s["rows"][:n].long(), :V].float()
    x = torch.where(torch.isnan(x), -math.inf, x)
    m = x.amax(-1, keepdim=True)
    z = (x - m) / float(np.float32(c["temperature"]))
    w = z.exp()
    total = w.sum(-1, keepdim=True, dtype=torch.float64)
    log_total = total.log()
    mean = (w * z).sum(-1, keepdim=True, dtype=torch.float64) / total
    given = s["given"][:n].long()[:, None]
    xg, j = x.gather(1, given), torch.arange(V, device="cuda")
    for name, fill in (("logprob", 0), ("entropy", 0), ("rank", -1), ("top_token", -1), ("top_logprob", 0)):
        s[name].fill_(fill)
    s["logprob"][:n] = (z.gather(1, given).double() - log_total)[:, 0].float()
    s["entropy"][:n] = (log_total - mean)[:, 0].float()
    s["rank"][:n] = ((x > xg) | ((x == xg) & (j < given))).sum(-1).to(torch.int32)
    if c["n_top"]:
        bits = (x + 0.0).view(torch.int32).long()
        key = torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits) * 2 ** 31 + (V - 1 - j)    # by value, then the lower token
        k = min(V, c["n_top"])
        top = V - 1 - (key.topk(k, -1).values % 2 ** 31)
        s["top_token"][:n, :k] = top.to(torch.int32)
        s["top_logprob"][:n, :k] = (z.gather(1, top).double() - log_total).float()
        s["top_logprob"][:n, k:] = -math.inf
    return {k: s[k] for k in ("logprob", "rank", "entropy", "top_token", "top_logprob")}


# ---- the library's calls ---------------------------------------------------------------------------
_lib = {}


def _library():
    """The binding and one context, as a program keeps them."""
    if not _lib:
        from paper_2602_02159_b200 import binding as fb
        _lib["fb"], _lib["ctx"] = fb, fb.Context(torch.cuda.current_device())
    return _lib["fb"], _lib["ctx"]


def _rope(s):
    """The rotation plan, made once as a model's set-up does."""
    if "rope" not in s:
        fb, _ = _library()
        c = s["case"]
        kind = {"plain": fb.ROPE_PLAIN, "linear": fb.ROPE_LINEAR, "ntk": fb.ROPE_NTK, "bands": fb.ROPE_BANDS,
                "yarn": fb.ROPE_YARN}[c["scaling"]]
        s["rope"] = fb.make_rope(c["rot"], fb.ROPE_HALVES if c["layout"] == HALVES else fb.ROPE_PAIRS, SCALING[c["scaling"]][0],
                                 kind, *SCALING[c["scaling"]][1:])
    return s["rope"]


def _own(s):
    fb, ctx = _library()
    c = s["case"]
    dt = fb.BF16 if c["dtype"] == "bf16" else fb.F32
    if c["op"] == "rotate":
        X, Y = s["X"], s["Y"]
        fb.focus_rotate(ctx, _rope(s), -1 if c["inverse"] else 1, X, Y, dt, c["heads"], c["d"], X.stride(0), X.stride(1),
                        Y.stride(0), Y.stride(1), 0, s["positions"], s["n_rows"], c["rows"])
        return {"Y": Y}
    if c["op"] == "logprobs":
        fb.focus_token_logprobs(ctx, s["logits"], dt, s["logits"].shape[1], c["vocab"], 0, c["n_pos"], s["rows"], s["n_rows"],
                                c["max_rows"], c["temperature"], s["given"], s["logprob"], s["rank"], s["entropy"],
                                c["n_top"], s["top_token"] if c["n_top"] else None, s["top_logprob"] if c["n_top"] else None)
        return {k: s[k] for k in ("logprob", "rank", "entropy", "top_token", "top_logprob")}
    K, tok, head = s["K"], 2 if c["heads_first"] else 1, 1 if c["heads_first"] else 2
    cache = fb.make_paged_cache(K, s["V"], s["table"], s["kv_len"], c["page"], K.shape[0], c["n"], s["table"].shape[1],
                                K.stride(0), K.stride(tok), K.stride(head))
    shape = fb.make_shape(s["longest"], 0, c["H"], c["Hkv"], c["d"], 128, dt)
    if c["op"] == "append":
        fb.focus_append_kv_paged(ctx, shape, _rope(s), s["Q"], s["K_new"], s["V_new"], s["Q"].stride(0), s["Q"].stride(1),
                                 s["row_start"], s["positions"], s["rows"], cache, s["Q_out"])
        return {"Q": s["Q_out"], "K": K, "V": s["V"]}
    fb.focus_paged_attn(ctx, shape, s["Q"], s["row_start"], s["max_rows"], cache, s["O"], s["lse"])
    return {"O": s["O"], "lse": s["lse"]}


def run(state):
    if own:
        return _own(state)
    return {"rotate": _plain_rotate, "append": _plain_append, "attend": _plain_attend,
            "logprobs": _plain_logprobs}[state["case"]["op"]](state)


# ---- what a pass cannot do without -----------------------------------------------------------------
def work(case):
    c = case
    size = 2 if c["dtype"] == "bf16" else 4
    if c["op"] == "rotate":
        e = c["rows"] * c["heads"]
        return {"bytes": e * 2 * c["d"] * size + 4 * c["rows"], "flops": 3 * e * c["rot"]}
    if c["op"] == "logprobs":
        return {"bytes": c["rows"] * (c["vocab"] * size + 20 + 8 * c["n_top"]), "flops": 6 * c["rows"] * c["vocab"]}
    length, new = _lengths(c)
    pages = sum((t + c["page"] - 1) // c["page"] for t in length)
    if c["op"] == "append":
        e = sum(new)
        return {"bytes": 2 * e * (c["H"] + 2 * c["Hkv"]) * c["d"] * size + 8 * c["n"] + 4 * e,
                "flops": 3 * e * (c["H"] + c["Hkv"]) * c["rot"]}
    return {"bytes": (2 * c["Hkv"] * sum(length) + 2 * sum(new) * c["H"]) * c["d"] * size + 4 * (sum(new) * c["H"] + pages),
            "flops": 4 * c["H"] * c["d"] * sum(t * k for t, k in zip(length, new))}


# ---- exact values ----------------------------------------------------------------------------------
def _exact_turned(x, positions, c, sign=1):
    """The same turns as products of complex numbers, with the frequencies written out one by one."""
    base, factor, low, high, trained = SCALING[c["scaling"]]
    rot, kind, magnitude, freq = c["rot"], c["scaling"], 1.0, []
    for k in range(rot // 2):
        f = math.pow(base, -2.0 * k / rot)
        if kind == "linear":
            f /= factor
        elif kind == "ntk":
            f = math.pow(base * math.pow(factor, rot / (rot - 2.0)), -2.0 * k / rot)
        elif kind == "bands":
            wave = 2.0 * math.pi / f
            if wave > trained / low:
                f /= factor
            elif wave >= trained / high:
                mix = (trained / wave - low) / (high - low)
                f = (1.0 - mix) * f / factor + mix * f
        elif kind == "yarn":
            def pair_of(turns):
                return (rot / 2.0) * math.log(trained / (2.0 * math.pi * turns), base)
            lo, hi = max(math.floor(pair_of(high)), 0), min(math.ceil(pair_of(low)), rot - 1)
            r = 0.0 if k <= lo else 1.0 if k >= hi else (k - lo) / (hi - lo)
            f = f * (1.0 - r) + f / factor * r
            magnitude = 1.0 + 0.1 * math.log(factor)
        freq.append(f)
    angle = sign * torch.outer(positions.double(), torch.tensor(freq, dtype=torch.float64, device="cuda"))
    turn = torch.polar(torch.full_like(angle, magnitude), angle)[:, None, :]
    y = x.double()
    head = y[..., :rot]
    if c["layout"] == HALVES:
        z = torch.complex(head[..., :rot // 2], head[..., rot // 2:]) * turn
        head = torch.cat([z.real, z.imag], -1)
    else:
        z = torch.view_as_complex(head.reshape(*head.shape[:-1], rot // 2, 2).contiguous()) * turn
        head = torch.view_as_real(z).reshape(head.shape)
    return torch.cat([head, y[..., rot:]], -1)


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] == "rotate":
        return {"Y": _exact_turned(s["X"], s["positions"], c, -1 if c["inverse"] else 1)}
    if c["op"] == "append":
        length, new, table = s["length"], s["new"], s["table"].cpu()
        pos = s["positions"].cpu() if s["positions"] is not None else torch.cat(
            [torch.arange(t - k, t) for t, k in zip(length, new)])
        owner = torch.cat([torch.full((k,), i) for i, k in enumerate(new)])
        slot = (table[owner, pos // c["page"]].long() * c["page"] + pos % c["page"]).cuda()
        pos = pos.cuda()
        res = {"Q": _exact_turned(s["Q"], pos, c)}
        for name, rows in (("K", _exact_turned(s["K_new"], pos, c)), ("V", s["V_new"].double())):
            pool = _tokens_first(s, name).double()
            pool = pool.reshape(-1, c["Hkv"], c["d"]).index_copy(0, slot, rows).reshape(pool.shape)
            res[name] = pool.transpose(1, 2).contiguous() if c["heads_first"] else pool
        return res
    if c["op"] == "attend":
        H, Hkv, d, hpg = c["H"], c["Hkv"], c["d"], c["H"] // c["Hkv"]
        if c["n"] * Hkv > 8192:
            return None
        O, lse, first = s["O"].double(), s["lse"].double(), 0
        K, V = _tokens_first(s, "K"), _tokens_first(s, "V")
        for i, (t, k) in enumerate(zip(s["length"], s["new"])):
            pages = s["table"][i, :(t - 1) // c["page"] + 1].long()
            for g in range(Hkv):
                keys = K[pages, :, g].reshape(-1, d)[:t].double()
                values = V[pages, :, g].reshape(-1, d)[:t].double()
                q = s["Q"][first:first + k, g * hpg:(g + 1) * hpg].double()
                z = torch.einsum("rhd,td->rht", q, keys) / math.sqrt(d)
                lse[g * hpg:(g + 1) * hpg, first:first + k] = torch.logsumexp(z, -1).T
                O[first:first + k, g * hpg:(g + 1) * hpg] = torch.softmax(z, -1) @ values
            first += k
        return {"O": O, "lse": lse}
    n, V, T = c["rows"], c["vocab"], float(np.float32(c["temperature"]))
    out = {"logprob": s["logprob"].double(), "rank": s["rank"] * 0 - 1, "entropy": s["entropy"].double(),
           "top_token": s["top_token"] * 0 - 1, "top_logprob": s["top_logprob"].double()}
    k = min(V, c["n_top"])
    for r in range(n):
        x = s["logits"][int(s["rows"][r]), :V].double()
        lp = torch.log_softmax(x / T, 0)
        order = torch.sort(x, descending=True, stable=True).indices
        t = int(s["given"][r])
        out["logprob"][r] = lp[t]
        out["rank"][r] = int(torch.nonzero(order == t)[0])
        out["entropy"][r] = -(lp.exp() * lp).sum()
        out["top_token"][r, :k] = order[:k].to(torch.int32)
        out["top_logprob"][r, :k] = lp[order[:k]]
        out["top_logprob"][r, k:] = -math.inf
    return out
