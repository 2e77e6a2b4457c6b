"""Cases, plain forms and exact values of four operators of a denoising step:

  write    K/V rows quantised to 8 bits as they enter the cache (one scale per token and KV head)
  read     cached rows read back from their codes and scales
  attend   softmax attention of listed rows over an 8-bit cache, dense or over blocks + sink tokens + response region
  sample   tokens drawn from logits with temperature, top-k, top-p and min-p, one given uniform number per row

`own` False: elementary torch operations; True: the library's entry points.
"""
import math

import numpy as np
import torch

own = False

INT8, E4M3 = "int8", "e4m3"
QMAX = {INT8: 127.0, E4M3: 448.0}
CODE = {INT8: torch.int8, E4M3: torch.float8_e4m3fn}
FLUSH = 2.0 ** -80                    # rows whose largest magnitude is below this are stored as zeros with scale 0
REAL = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---- cases -----------------------------------------------------------------------------------------
def _write(name, dtype, fmt, H, Hkv, d, L, n, listed_rows):
    return dict(name=name, op="write", dtype=dtype, fmt=fmt, H=H, Hkv=Hkv, d=d, L=L, n=n, listed_rows=listed_rows)


def _read(name, dtype, fmt, Hkv, d, L, n, listed_rows, values):
    return dict(name=name, op="read", dtype=dtype, fmt=fmt, Hkv=Hkv, d=d, L=L, n=n, listed_rows=listed_rows, values=values)


def _attend(name, dtype, fmt, H, Hkv, d, L, M, rows, max_rows, block=0, keep=0, sinks=0, all_heads=False):
    """max_rows: capacity of the row list, rows of it in use; max_rows == 0: all rows [L - rows, L).  block == 0: dense."""
    return dict(name=name, op="attend", dtype=dtype, fmt=fmt, H=H, Hkv=Hkv, d=d, L=L, M=M, rows=rows, max_rows=max_rows,
                block=block, keep=keep, sinks=sinks, all_heads=all_heads)


def _sample(name, dtype, vocab, n_pos, rows, max_rows, temperature, top_k, top_p, min_p, spread):
    return dict(name=name, op="sample", dtype=dtype, vocab=vocab, n_pos=n_pos, rows=rows, max_rows=max_rows,
                temperature=temperature, top_k=top_k, top_p=top_p, min_p=min_p, spread=spread)


def listed():
    return [
        # one layer's refreshed rows of a denoising step at 32K context (k = 8 focus rows with windows of 9), out of a
        # fused QKV projection
        _write("write step rows", "bf16", INT8, 32, 32, 128, 32768, 72, True),
        # block entry: every position of a GQA layer is written
        _write("write whole layer", "bf16", E4M3, 28, 4, 128, 16384, 16384, False),
        # cached keys of a whole MHA layer read back for pooling or sink identification
        _read("read keys of a layer", "bf16", INT8, 32, 128, 32768, 32768, False, False),
        # a few hundred positions gathered in full precision
        _read("read listed rows", "f32", E4M3, 8, 64, 5000, 333, True, True),
        # the tiny single-layer step in fp32: 8 heads of 64, 83 active rows
        _attend("attend tiny f32", "f32", INT8, 8, 8, 64, 1024, 896, 83, 144),
        # dense layer over the active rows at 32K context: the cache is what is read
        _attend("attend dense 32K", "bf16", INT8, 32, 32, 128, 32768, 32256, 35, 72),
        # GQA 28/4 at 16K, floating codes, windows that hardly overlap
        _attend("attend dense GQA", "bf16", E4M3, 28, 4, 128, 16384, 16128, 61, 72),
        # sparse layer at 32K: 1/16 of the 128-token blocks, 1 % sinks, 512 response tokens
        _attend("attend sparse 32K", "bf16", INT8, 32, 32, 128, 32768, 32256, 35, 72, 128, 15, 322),
        # all rows of the generation region, dense: arithmetic counts
        _attend("attend dense 256 rows", "bf16", INT8, 32, 32, 128, 16384, 16128, 256, 0),
        # one position, fp32 logits, temperature alone
        _sample("sample one row", "f32", 50257, 4, 1, 1, 1.0, 0, 1.0, 0.0, 2.5),
        # the active rows of a step: nucleus
        _sample("sample step rows", "bf16", 126464, 96, 35, 72, 0.7, 0, 0.95, 0.0, 3.0),
        # a whole generation region: top-k, then nucleus, then min-p
        _sample("sample 512 rows", "bf16", 126464, 512, 512, 512, 0.9, 50, 0.9, 0.02, 3.0),
    ]


HEADS = [(32, 32, 128), (28, 4, 128), (8, 8, 64), (16, 4, 64), (8, 2, 128), (12, 12, 128), (6, 1, 128)]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["write", "read", "attend", "attend", "sample"])
    fmt, dtype = rng.choice([INT8, E4M3]), rng.choice(["bf16", "bf16", "bf16", "f32"])
    H, Hkv, d = rng.choice(HEADS)
    if op in ("write", "read"):
        L = _log(rng, 1, 32768)
        rows = rng.random() < 0.6
        n = _log(rng, 1, L)
        if op == "write":
            c = _write("", dtype, fmt, H, Hkv, d, L, min(n, 20000), rows)
        else:
            c = _read("", dtype, fmt, Hkv, d, L, min(n, 20000), rows, rng.random() < 0.5)
    elif op == "attend":
        L = _log(rng, 2, 32768 if dtype == "bf16" else 4096)
        N = min(L, rng.choice([1, 32, 100, 256, 512]))
        M = L - N
        most = max(1, min(N, 2 ** 27 // (H * L), 256))       # rows x heads x keys as in the largest listed case
        rows = _log(rng, 1, most)
        full = rows == N or rng.random() < 0.3
        max_rows = 0 if full else rows + rng.randrange(0, 40)
        block = rng.choice([0, 64, 128]) if M > 0 else 0
        nb = (M + block - 1) // block if block else 0
        c = _attend("", dtype, fmt, H, Hkv, d, L, M, rows, max_rows, block, _log(rng, 1, nb) if nb else 0,
                    min(M, rng.choice([0, 1, 40, 322])) if block else 0, bool(block) and rng.random() < 0.2)
    else:
        vocab = _log(rng, 7, 160000)
        n_pos = _log(rng, 1, max(1, min(512, 60_000_000 // vocab)))
        rows = rng.randint(1, n_pos)
        c = _sample("", dtype, vocab, n_pos, rows, rows + rng.randrange(0, 20), round(rng.uniform(0.2, 1.5), 2),
                    rng.choice([0, 0, 1, 20, 50, 1000]), rng.choice([1.0, 1.0, 0.5, 0.9, 0.95, 0.99]),
                    rng.choice([0.0, 0.0, 0.02, 0.1]), round(rng.uniform(0.5, 4.0), 2))
    del c["name"]
    return c


# ---- inputs ----------------------------------------------------------------------------------------
def _rand(gen, shape, dtype="f32", scale=1.0):
    return (torch.randn(shape, generator=gen, device="cuda") * scale).to(REAL[dtype])


def _positions(gen, lo, hi, n):
    return (torch.randperm(hi - lo, generator=gen, device="cuda")[:n].sort().values + lo).to(torch.int32)


def _padded(idx, size):
    out = torch.full((size,), -1, dtype=torch.int32, device="cuda")
    out[:idx.numel()] = idx
    return out


def _encode(x, fmt):
    """Codes and scales of the last axis: scale = max|x| / QMAX, code = nearest of x / scale."""
    a = x.float().abs().amax(-1)
    scale = torch.where(a < FLUSH, torch.zeros_like(a), a / torch.full_like(a, QMAX[fmt]))   # a tensor: a true division
    q = torch.where(scale[..., None] > 0, x.float() / scale[..., None], torch.zeros_like(x, dtype=torch.float32))
    return ((q.round() if fmt == INT8 else q).clamp(-QMAX[fmt], QMAX[fmt]).to(CODE[fmt])), scale


def _cache(gen, Hkv, L, d, fmt, sink_every=0):
    """A cache as a model fills it: tokens and channels of unequal size, a few keys much longer than the rest."""
    out = []
    for which in range(2):
        x = torch.randn((Hkv, L, d), generator=gen, device="cuda")
        x *= torch.exp(0.5 * torch.randn((Hkv, L, 1), generator=gen, device="cuda"))
        if which == 0 and sink_every:
            x[:, ::sink_every] *= 2.0
        out.append(_encode(x, fmt))
        del x
    (kq, ks), (vq, vs) = out
    return kq, vq, ks, vs


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    s = {"case": c, "gen_seed": seed}
    if c["op"] == "write":
        Hkv, d, L, n = c["Hkv"], c["d"], c["L"], c["n"]
        s["cache"] = _cache(gen, Hkv, L, d, c["fmt"])
        qkv = _rand(gen, (n, c["H"] + 2 * Hkv, d), c["dtype"])           # a fused projection's rows: Q | K | V
        s["K_new"], s["V_new"] = qkv[:, c["H"]:c["H"] + Hkv], qkv[:, c["H"] + Hkv:]
        s["pos_base"] = 0 if c["listed_rows"] else (L - n)
        s["rows"] = _positions(gen, 0, L, n) if c["listed_rows"] else None
        s["n_rows"] = torch.tensor([n], dtype=torch.int32, device="cuda") if c["listed_rows"] else None
    elif c["op"] == "read":
        Hkv, d, L, n = c["Hkv"], c["d"], c["L"], c["n"]
        s["cache"] = _cache(gen, Hkv, L, d, c["fmt"])
        s["pos_base"] = 0 if c["listed_rows"] else (L - n)
        s["rows"] = _positions(gen, 0, L, n) if c["listed_rows"] else None
        s["n_rows"] = torch.tensor([n], dtype=torch.int32, device="cuda") if c["listed_rows"] else None
        s["K_out"] = torch.zeros((Hkv, n, d), dtype=REAL[c["dtype"]], device="cuda")
        s["V_out"] = torch.zeros_like(s["K_out"]) if c["values"] else None
    elif c["op"] == "attend":
        H, Hkv, d, L, M = c["H"], c["Hkv"], c["d"], c["L"], c["M"]
        s["cache"] = _cache(gen, Hkv, L, d, c["fmt"], 997)
        N = c["rows"] if c["max_rows"] == 0 else L - M                   # Q holds the generation region
        s["q_base"], s["n_q"] = L - N, N
        s["Q"] = _rand(gen, (N, H, d), c["dtype"])
        if c["max_rows"]:
            s["q_rows"] = _padded(_positions(gen, M, L, c["rows"]), c["max_rows"])
            s["n_rows"] = torch.tensor([c["rows"]], dtype=torch.int32, device="cuda")
        else:
            s["q_rows"] = s["n_rows"] = None
        bound = c["max_rows"] or N
        s["O"] = torch.zeros((bound, H, d), dtype=REAL[c["dtype"]], device="cuda")
        s["lse"] = torch.zeros((H, bound), dtype=torch.float32, device="cuda")
        if c["block"]:
            nb, G = (M + c["block"] - 1) // c["block"], 1 if c["all_heads"] else Hkv
            pick = torch.rand((G, nb), generator=gen, device="cuda").argsort(-1)[:, :c["keep"]].sort(-1).values
            s["block_idx"] = pick.to(torch.int32).contiguous()
            s["block_cnt"] = torch.full((G,), c["keep"], dtype=torch.int32, device="cuda")
            s["sink_idx"] = _positions(gen, 0, M, c["sinks"])
            chosen = torch.zeros((G, nb), dtype=torch.bool, device="cuda").scatter_(1, pick, True)
            s["sink_keep"] = (~chosen[:, (s["sink_idx"] // c["block"]).long()]).to(torch.uint8).contiguous()
    else:
        n_pos, V = c["n_pos"], c["vocab"]
        step = 8 if c["dtype"] == "bf16" else 4
        stride = (V + step - 1) // step * step
        s["logits"] = _rand(gen, (n_pos, stride), c["dtype"], c["spread"])
        s["rows"] = _padded(_positions(gen, 0, n_pos, c["rows"]), c["max_rows"])
        s["n_rows"] = torch.tensor([c["rows"]], dtype=torch.int32, device="cuda")
        s["u"] = torch.rand((c["max_rows"],), generator=gen, device="cuda")
        s["conf"] = torch.zeros((c["max_rows"],), device="cuda")
        s["prob"] = torch.zeros((c["max_rows"],), device="cuda")
        s["token"] = torch.zeros((c["max_rows"],), dtype=torch.int32, device="cuda")
        s["kept"] = torch.zeros((c["max_rows"],), dtype=torch.int32, device="cuda")
    return s


# ---- plain forms -----------------------------------------------------------------------------------
def _plain_write(s):
    c = s["case"]
    kq, vq, ks, vs = s["cache"]
    pos = s["rows"].long() if s["rows"] is not None else torch.arange(c["n"], device="cuda") + s["pos_base"]
    for codes, scales, new in ((kq, ks, s["K_new"]), (vq, vs, s["V_new"])):
        q, sc = _encode(new, c["fmt"])
        codes.view(torch.uint8)[:, pos] = q.view(torch.uint8).transpose(0, 1)
        scales[:, pos] = sc.transpose(0, 1)
    return {"K": kq, "V": vq, "K_scale": ks, "V_scale": vs}


def _plain_read(s):
    c = s["case"]
    kq, vq, ks, vs = s["cache"]
    pos = s["rows"].long() if s["rows"] is not None else torch.arange(c["n"], device="cuda") + s["pos_base"]
    out = {}
    for name, codes, scales in (("K", kq, ks), ("V", vq, vs)):
        if s[name + "_out"] is not None:
            s[name + "_out"].copy_(codes.view(torch.uint8)[:, pos].view(codes.dtype).float() * scales[:, pos, None])
            out[name] = s[name + "_out"]
    return out


def _key_mask(s):
    """[G, L] truth values: the keys that a sparse layer attends."""
    c = s["case"]
    L, M, B = c["L"], c["M"], c["block"]
    G = s["block_idx"].shape[0]
    nb = (M + B - 1) // B
    blocks = torch.zeros((G, nb), dtype=torch.bool, device="cuda").scatter_(1, s["block_idx"].long(), True)
    j = torch.arange(L, device="cuda")
    mask = blocks[:, (j // B).clamp(max=nb - 1)] | (j >= M)
    sinks = torch.zeros((G, L), dtype=torch.bool, device="cuda")
    sinks[:, s["sink_idx"].long()] = s["sink_keep"].bool()
    return mask | sinks


def _plain_attend(s):
    c = s["case"]
    H, Hkv, d = c["H"], c["Hkv"], c["d"]
    kq, vq, ks, vs = s["cache"]
    k, v = kq.float() * ks[..., None], vq.float() * vs[..., None]
    n = c["rows"]
    q = s["Q"][(s["q_rows"][:n] - s["q_base"]).long()] if c["max_rows"] else s["Q"]
    q = q.float().reshape(n, Hkv, H // Hkv, d).permute(1, 2, 0, 3).reshape(Hkv, -1, d)       # [Hkv, hpg * n, d]
    p = torch.matmul(q, k.transpose(1, 2)) * (1.0 / math.sqrt(d))
    del k
    if c["block"]:
        p.masked_fill_(~_key_mask(s)[:, None, :], -math.inf)
    m = p.amax(-1, keepdim=True)
    p.sub_(m).exp_()
    z = p.sum(-1, keepdim=True)
    o = torch.matmul(p, v) / z
    lse = (m + z.log())[..., 0]
    s["O"][:n] = o.reshape(Hkv, H // Hkv, n, d).permute(2, 0, 1, 3).reshape(n, H, d).to(s["O"].dtype)
    s["lse"][:, :n] = lse.reshape(H, n)
    return {"O": s["O"], "lse": s["lse"]}


def _single(x):
    return float(np.float32(x))


def _plain_sample(s):
    c = s["case"]
    n, V = c["rows"], c["vocab"]
    x = s["logits"][s["rows"][:n].long(), :V].double()
    x = torch.where(torch.isnan(x), -math.inf, x)
    m = x.amax(-1, keepdim=True)
    w = ((x - m) / _single(c["temperature"])).exp()
    raw = (x - m).exp()
    order = x.argsort(dim=-1, descending=True, stable=True)
    del x
    ws = w.gather(1, order)
    cum = ws.cumsum(-1)
    k = min(c["top_k"] or V, V)
    kept = torch.full((n,), k, dtype=torch.long, device="cuda")
    if c["top_p"] < 1.0:
        kept = torch.minimum(kept, (cum < _single(c["top_p"]) * cum[:, k - 1:k]).sum(-1) + 1)
    if c["min_p"] > 0.0:
        kept = torch.minimum(kept, (ws >= _single(c["min_p"])).sum(-1))
    del ws, cum
    keep = torch.zeros_like(w, dtype=torch.bool)
    keep.scatter_(1, order, (torch.arange(V, device="cuda") < kept[:, None]))
    w = torch.where(keep, w, 0.0)
    cum = w.cumsum(-1)
    total = cum[:, -1:]
    t = torch.searchsorted(cum, s["u"][:n, None].double() * total, right=True).clamp(max=V - 1)
    s["token"].fill_(-1)
    s["conf"].zero_()
    s["prob"].zero_()
    s["kept"].zero_()
    s["token"][:n] = t[:, 0].to(torch.int32)
    s["conf"][:n] = (w.gather(1, t) / total)[:, 0].float()
    s["prob"][:n] = (raw.gather(1, t) / raw.sum(-1, keepdim=True))[:, 0].float()
    s["kept"][:n] = kept.to(torch.int32)
    return {"token": s["token"], "conf": s["conf"], "prob": s["prob"], "kept": s["kept"]}


# ---- the library's calls ---------------------------------------------------------------------------
_lib = {}


def _library():
    """The binding and one context, as a program keeps them."""
    if not _lib:
        from paper_2602_02159_b200 import binding as fb
        _lib["fb"], _lib["ctx"] = fb, fb.Context(torch.cuda.current_device())
    return _lib["fb"], _lib["ctx"]


def _own(s):
    fb, ctx = _library()
    c = s["case"]
    if c["op"] == "sample":
        fb.focus_sample(ctx, s["logits"], fb.BF16 if c["dtype"] == "bf16" else fb.F32, s["logits"].shape[1], c["vocab"], 0,
                        c["n_pos"], s["rows"], s["n_rows"], c["max_rows"], c["temperature"], c["top_k"], c["top_p"],
                        c["min_p"], s["u"], s["conf"], s["token"], s["prob"], s["kept"])
        return {"token": s["token"], "conf": s["conf"], "prob": s["prob"], "kept": s["kept"]}
    kq, vq, ks, vs = s["cache"]
    cache = fb.make_quant_cache(fb.KV_INT8 if c["fmt"] == INT8 else fb.KV_E4M3, kq, vq, ks, vs)
    shape = fb.make_shape(c["L"], c.get("M", 0), c.get("H", c["Hkv"]), c["Hkv"], c["d"], c.get("block") or 128,
                          fb.BF16 if c["dtype"] == "bf16" else fb.F32)
    if c["op"] == "write":
        new = s["K_new"]
        fb.focus_quantize_kv(ctx, shape, new, s["V_new"], new.stride(0), new.stride(1), s["pos_base"], s["rows"],
                             s["n_rows"], c["n"], cache)
        return {"K": kq, "V": vq, "K_scale": ks, "V_scale": vs}
    if c["op"] == "read":
        out = s["K_out"]
        fb.focus_dequantize_kv(ctx, shape, cache, s["pos_base"], s["rows"], s["n_rows"], c["n"], out, s["V_out"],
                               out.stride(1), out.stride(0))
        return {"K": out} if s["V_out"] is None else {"K": out, "V": s["V_out"]}
    rows = (s["Q"], s["q_base"], s["n_q"], s["q_rows"], s["n_rows"], c["max_rows"])
    if c["block"]:
        fb.focus_sparse_attn_quantized(ctx, shape, *rows, cache, fb.HEADS_ALL if c["all_heads"] else fb.HEADS_PER_KV_GROUP,
                                       s["block_idx"], c["keep"], s["block_cnt"], s["sink_idx"], s["sink_keep"],
                                       c["sinks"], s["O"], s["lse"])
    else:
        fb.focus_dense_attn_quantized(ctx, shape, *rows, cache, s["O"], s["lse"])
    return {"O": s["O"], "lse": s["lse"]}


def run(state):
    if own:
        return _own(state)
    return {"write": _plain_write, "read": _plain_read, "attend": _plain_attend, "sample": _plain_sample}[state["case"]["op"]](state)


# ---- what a pass cannot do without -----------------------------------------------------------------
def work(case):
    c = case
    size = 2 if c["dtype"] == "bf16" else 4
    if c["op"] == "write":
        e = 2 * c["n"] * c["Hkv"]
        return {"bytes": e * (c["d"] * (size + 1) + 4), "flops": 2 * e * c["d"]}
    if c["op"] == "read":
        e = (2 if c["values"] else 1) * c["n"] * c["Hkv"]
        return {"bytes": e * (c["d"] * (size + 1) + 4), "flops": e * c["d"]}
    if c["op"] == "attend":
        keys = c["L"]
        if c["block"]:
            keys = min(c["L"], c["keep"] * c["block"] + c["sinks"] + c["L"] - c["M"])
        rows = c["rows"] * c["H"]
        return {"bytes": 2 * c["Hkv"] * keys * (c["d"] + 4) + rows * (2 * c["d"] * size + 4), "flops": 4 * rows * keys * c["d"]}
    return {"bytes": c["rows"] * (c["vocab"] * size + 20), "flops": 4 * c["rows"] * c["vocab"]}


# ---- exact values ----------------------------------------------------------------------------------
def _exact_codes(x, fmt):
    """Codes and scales of rows x (numpy, float64 holding the stored values)."""
    a = np.abs(x).max(-1)
    scale = np.where(a < FLUSH, 0.0, (a / QMAX[fmt]).astype(np.float32)).astype(np.float64)
    with np.errstate(divide="ignore", invalid="ignore"):
        q = np.where(scale[..., None] > 0, x / scale[..., None], 0.0).astype(np.float32).astype(np.float64)
    if fmt == INT8:
        return np.clip(np.rint(q), -127, 127), scale
    # e4m3: 3 fraction bits, exponents from -6, ties to even
    mag = np.abs(q)
    e = np.maximum(np.floor(np.log2(np.maximum(mag, 2.0 ** -20))), -6.0)
    step = np.exp2(e - 3.0)
    return np.sign(q) * np.minimum(np.rint(mag / step) * step, 448.0), scale


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] == "write":
        pos = s["rows"].cpu().numpy() if s["rows"] is not None else np.arange(c["n"]) + s["pos_base"]
        res = {}
        for name, codes, scales, new in (("K", s["cache"][0], s["cache"][2], s["K_new"]), ("V", s["cache"][1], s["cache"][3], s["V_new"])):
            q, sc = _exact_codes(new.double().cpu().numpy(), c["fmt"])
            full, fs = codes.float().double(), scales.double()
            full[:, torch.from_numpy(pos).long().cuda()] = torch.from_numpy(q).cuda().transpose(0, 1)
            fs[:, torch.from_numpy(pos).long().cuda()] = torch.from_numpy(sc).cuda().transpose(0, 1)
            res[name] = full.to(torch.int8) if c["fmt"] == INT8 else full
            res[name + "_scale"] = fs
        return res
    if c["op"] == "read":
        lo = s["pos_base"]
        res = {}
        for name, codes, scales in (("K", s["cache"][0], s["cache"][2]), ("V", s["cache"][1], s["cache"][3])):
            if s[name + "_out"] is not None:
                x = codes.float().double() * scales.double()[..., None]
                res[name] = x.index_select(1, s["rows"].long()) if s["rows"] is not None else x[:, lo:lo + c["n"]]
        return res
    if c["op"] == "attend":
        H, n, hpg = c["H"], c["rows"], c["H"] // c["Hkv"]
        O, lse = s["O"].double(), s["lse"].double()
        where = [int(r) - s["q_base"] for r in s["q_rows"][:n].tolist()] if c["max_rows"] else list(range(n))
        q = s["Q"].double()[where]                                          # [n, H, d]
        for g in range(c["Hkv"]):
            K = s["cache"][0][g].float().double() * s["cache"][2][g].double()[:, None]
            V = s["cache"][1][g].float().double() * s["cache"][3][g].double()[:, None]
            if c["block"]:
                row = 0 if c["all_heads"] else g
                keys = list(range(c["M"], c["L"]))
                for b in s["block_idx"][row].tolist():
                    keys += range(b * c["block"], min((b + 1) * c["block"], c["M"]))
                keys += [j for j, kept in zip(s["sink_idx"].tolist(), s["sink_keep"][row].tolist()) if kept]
                at = torch.tensor(sorted(keys), device="cuda")
                K, V = K[at], V[at]
            for h in range(g * hpg, (g + 1) * hpg):
                z = q[:, h] @ K.T / math.sqrt(c["d"])
                lse[h, :n] = torch.logsumexp(z, -1)
                O[:n, h] = torch.softmax(z, -1) @ V
        return {"O": O, "lse": lse}
    # sample: by distinct values instead of a sort of the row
    n, V = c["rows"], c["vocab"]
    T, top_p, min_p = (float(np.float32(c[k])) for k in ("temperature", "top_p", "min_p"))
    token, kept = s["token"] * 0 - 1, s["kept"] * 0
    conf, prob = s["conf"].double() * 0, s["prob"].double() * 0
    for r in range(n):
        x = s["logits"][int(s["rows"][r]), :V].double()
        val, inv, cnt = torch.unique(x, return_inverse=True, return_counts=True)
        val, cnt = val.flip(0), cnt.flip(0)                                 # largest first
        inv = val.numel() - 1 - inv
        w = torch.exp(val / T - val[0] / T)
        take = cnt.clone()
        if c["top_k"]:
            before = cnt.cumsum(0) - cnt
            take = torch.minimum(cnt, (c["top_k"] - before).clamp(min=0))
        if c["top_p"] < 1.0:
            mass = take * w
            target = top_p * mass.sum()
            before = mass.cumsum(0) - mass
            need = torch.ceil((target - before) / w).clamp(min=0)
            take = torch.minimum(take, need.long())
            take[0] = max(1, int(take[0]))
        if c["min_p"] > 0.0:
            take = torch.where(w >= min_p, take, 0)
        edge = torch.nonzero((take < cnt) & (take > 0)).flatten().tolist()
        keep = (take >= cnt)[inv]
        for e in edge:
            at = torch.nonzero(inv == e).flatten()[:int(take[e])]
            keep[at] = True
        p = torch.where(keep, w[inv], 0.0)
        cum = p.cumsum(0)
        t = int(torch.nonzero(cum > s["u"][r].double() * cum[-1])[0])
        token[r], kept[r] = t, int(take.sum())
        conf[r] = p[t] / cum[-1]
        prob[r] = torch.softmax(x, 0)[t]
    return {"token": token, "conf": conf, "prob": prob, "kept": kept}
