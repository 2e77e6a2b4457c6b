"""focus_token_logprobs against the float64 oracle.  Whole numbers (ranks, tokens) are equal.  A weight is off by 2^-22 (its
exponential), by 2^-24 of its exponent (product) and by its sum's roundings (a thread adds at most 1024 of them here, a warp
five, twice 2^-24 each at most), so ln Z by BOUND; a log probability by that, by the rounding of (x - m) / T in fp64 and of the
result in fp32; the entropy by the same and, relative, by the sum of weight times exponent."""
import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import focus_oracle as fo
from paper_2602_02159_b200 import binding as fb
from paper_2602_02159_b200 import build as fbuild

gpu = pytest.mark.gpu
DT = {"bf16": fb.BF16, "f32": fb.F32}
REAL = {"bf16": torch.bfloat16, "f32": torch.float32}
BOUND = 2.0 ** -22 + 32 * 2.0 ** -24 + 1030 * 2.0 ** -24                     # exponents to 32 carry weight


@pytest.fixture(scope="module")
def ctx():
    c = fb.Context(0)
    yield c
    assert c.poll_status() == 0
    c.close()


def test_refusals_need_no_device():
    fbuild.build()
    lib = fb.load_library()
    fake = ctypes.create_string_buffer(4096)
    P, h, nan = 1 << 20, ctypes.cast(fake, ctypes.c_void_p), float("nan")

    def call(ctx=h, x=P, dt=fb.BF16, stride=1000, vocab=1000, base=0, n_pos=8, rows=P, n=P, max_rows=8, T=1.0, given=P, lp=P,
             rank=P, ent=P, n_top=4, tok=P, tlp=P):
        return lib.focus_token_logprobs(ctx, x, dt, stride, vocab, base, n_pos, rows, n, max_rows, T, given, lp, rank, ent,
                                        n_top, tok, tlp, None)

    for bad in (dict(ctx=None), dict(x=None), dict(x=P + 8), dict(dt=2), dict(stride=1004), dict(stride=992), dict(vocab=0),
                dict(base=-1), dict(n_pos=-1), dict(base=2 ** 31 - 4), dict(rows=None), dict(n=None), dict(max_rows=-1),
                dict(rows=None, n=None, max_rows=9), dict(T=0.0), dict(T=-1.0), dict(T=nan), dict(T=math.inf),
                dict(given=None), dict(lp=None), dict(given=None, lp=None), dict(n_top=-1), dict(n_top=0), dict(tok=None),
                dict(tlp=None), dict(given=None, lp=None, rank=None, ent=None, n_top=0, tok=None, tlp=None),
                dict(dt=fb.F32, stride=1002)):
        assert call(**bad) == fb.ERR_INVALID_ARG, bad
    assert call(n_top=33) == fb.ERR_UNSUPPORTED and call(T=9e-8) == fb.ERR_UNSUPPORTED and call(T=1e35) == fb.ERR_UNSUPPORTED and call(max_rows=0) == fb.OK
    assert call(vocab=2 ** 30 + 8, stride=2 ** 30 + 8) == fb.ERR_UNSUPPORTED


def run(ctx, x, dtype, vocab, T, given, n_top, rows=None, max_rows=None, pos_base=0, use=("logprob", "rank", "entropy")):
    n_pos, m = x.shape[0], max_rows or x.shape[0]
    i32 = dict(dtype=torch.int32, device="cuda")
    r = torch.tensor(list(rows) + [-1] * (m - len(rows)), **i32) if rows is not None else None
    n = torch.tensor([len(rows)], **i32) if rows is not None else None
    g = torch.tensor(list(given) + [3] * (m - len(given)), **i32) if given is not None else None
    out = {"logprob": torch.full((m,), 7.0, device="cuda"), "rank": torch.full((m,), 7, **i32),
           "entropy": torch.full((m,), 7.0, device="cuda"), "top_token": torch.full((m, max(n_top, 1)), 7, **i32),
           "top_logprob": torch.full((m, max(n_top, 1)), 7.0, device="cuda")}
    fb.focus_token_logprobs(ctx, x, DT[dtype], x.stride(0), vocab, pos_base, n_pos, r, n, m, T, g,
                            out["logprob"] if "logprob" in use else None, out["rank"] if "rank" in use else None,
                            out["entropy"] if "entropy" in use else None, n_top, out["top_token"] if n_top else None,
                            out["top_logprob"] if n_top else None)
    return {k: v.cpu().numpy() for k, v in out.items()}


def near(got, want, slack=BOUND):
    if abs(want) > np.finfo(np.float32).max:                                 # the nearest fp32 number is infinite
        return got == math.copysign(math.inf, want)
    return abs(got - want) <= slack + 2.0 ** -24 * abs(want)


def check(out, x, vocab, T, given, n_top, rows=None, use=("logprob", "rank", "entropy")):
    x = x.double().cpu().numpy()
    T = float(np.float32(T))
    for i, r in enumerate(range(x.shape[0]) if rows is None else rows):
        t = int(given[i]) if given is not None else -1
        res = fo.token_logprobs(x[r][:vocab], T, t, n_top)
        k = min(n_top, vocab)
        if res is None:
            assert out["logprob"][i] == 0 and out["rank"][i] == -1 and out["entropy"][i] == 0
            assert (out["top_token"][i][:n_top] == -1).all() and (out["top_logprob"][i][:n_top] == 0).all()
            continue
        lp, rank, entropy, top, top_lp = res
        if "logprob" in use:
            assert near(out["logprob"][i], lp if t >= 0 else 0.0), (i, out["logprob"][i], lp)
        if "rank" in use:
            assert out["rank"][i] == (rank if t >= 0 else -1)
        if "entropy" in use:
            assert near(out["entropy"][i], entropy, BOUND * (2 + 2 * abs(entropy))), (i, out["entropy"][i], entropy)
        if n_top:
            assert out["top_token"][i][:k].tolist() == top and (out["top_token"][i][k:n_top] == -1).all()
            assert all(near(a, b) for a, b in zip(out["top_logprob"][i][:k], top_lp))
            assert np.isneginf(out["top_logprob"][i][k:n_top]).all()


def logits(rng, n, vocab, dtype, spread=3.0):
    step = 8 if dtype == "bf16" else 4
    x = torch.full((n, -(-vocab // step) * step), 1e4, device="cuda").to(REAL[dtype])       # larger than any: not to be read
    x[:, :vocab] = torch.from_numpy(rng.standard_normal((n, vocab)) * spread).cuda().to(REAL[dtype])
    return x


@gpu
@pytest.mark.parametrize("dtype,vocab,n,T,n_top", [
    ("bf16", 1, 2, 1.0, 3), ("f32", 7, 3, 0.7, 5), ("bf16", 33, 4, 1.0, 32), ("f32", 257, 5, 1.3, 1), ("bf16", 1000, 40, 0.8, 20),
    ("f32", 1025, 7, 1.0, 32), ("bf16", 2049, 3, 1.0, 0), ("bf16", 255, 3, 1.0, 32), ("bf16", 521, 3, 1.0, 32), ("bf16", 3000, 5, 1.0, 32),
    ("f32", 4095, 3, 1.0, 32), ("bf16", 8191, 2, 1.0, 32), ("bf16", 8192, 2, 1.0, 32), ("f32", 4097, 2, 1.0, 20), ("bf16", 32001, 9, 0.5, 20), ("f32", 50257, 2, 1.0, 5),
    ("bf16", 126464, 3, 1.0, 32), ("f32", 151643, 1, 2.0, 20), ("bf16", 8200, 900, 1.0, 8)])
def test_scores_of_tokens(ctx, dtype, vocab, n, T, n_top):
    rng = np.random.default_rng(vocab + n)
    x = logits(rng, n, vocab, dtype)
    given = rng.integers(0, vocab, n)
    given[0] = int(x[0, :vocab].float().argmax())
    if n > 2:
        given[1] = -1
    check(run(ctx, x, dtype, vocab, T, given, n_top), x, vocab, T, given, n_top)
    assert ctx.poll_status() == 0


@gpu
def test_lists_of_positions_and_what_may_be_left_out(ctx):
    rng = np.random.default_rng(1)
    x = logits(rng, 30, 3001, "bf16")
    rows, given = [3, 4, 9, 20, 29], [5, 0, 3000, 77, 1500]
    out = run(ctx, x, "bf16", 3001, 0.9, given, 4, [100 + r for r in rows], 11, pos_base=100)
    check(out, x, 3001, 0.9, given, 4, rows)
    assert (out["logprob"][5:] == 0).all() and (out["rank"][5:] == -1).all() and (out["entropy"][5:] == 0).all()
    assert (out["top_token"][5:] == -1).all() and (out["top_logprob"][5:] == 0).all()
    assert ctx.poll_status() == 0
    for use, g, n_top in ((("entropy",), None, 0), ((), None, 6), (("logprob",), given, 0), (("logprob", "rank"), given, 2)):
        out = run(ctx, x, "bf16", 3001, 0.9, g, n_top, [100 + r for r in rows], 11, pos_base=100, use=use)
        check(out, x, 3001, 0.9, g, n_top, rows, use)
        for k in {"logprob", "rank", "entropy"} - set(use):
            assert (out[k] == 7).all()
    out = run(ctx, x, "bf16", 3001, 1.0, [3001, -2, 5], 2, [100, 101, 130], 4, pos_base=100)       # tokens and a position out of range
    assert ctx.poll_status() == fb.ERR_INVALID_ARG
    assert out["logprob"].tolist() == [0, 0, 0, 0] and out["rank"].tolist() == [-1] * 4
    assert out["top_token"][0][0] == int(x[0, :3001].float().argmax()) and (out["top_token"][2:] == -1).all()


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", [600, 20011])
def test_ties_infinities_and_nan(ctx, dtype, vocab):
    rng = np.random.default_rng(vocab)
    x = logits(rng, 12, vocab, dtype)
    inf, nan = float("inf"), float("nan")
    x[0, :vocab] = 0.0                                                       # all alike
    x[0, 5:40] = -0.0                                                        # which equals 0
    x[1, :vocab] = (torch.arange(vocab, device="cuda") % 3).to(x.dtype)      # many ties at the top
    x[2, :vocab] = -inf
    x[3, :vocab] = nan
    x[4, :vocab:2] = -inf
    x[5, ::7] = nan
    x[6, 11], x[6, 500] = inf, inf
    x[7, :vocab] = -inf
    x[7, 17] = -3.0                                                          # one token
    x[8, :vocab] = torch.arange(vocab, device="cuda").float().div(64).to(x.dtype)      # ascending
    x[9, :vocab] = 3.0e38
    x[9, 3] = -3.0e38
    x[10, :vocab] *= 30.0
    x[11, :vocab] = torch.where(torch.arange(vocab, device="cuda") % 2048 < 8, 5.0, -5.0).to(x.dtype)   # a thread's vectors
    T = 1.0
    for given in ([40, 4, 3, 3, 2, 7, 11, 17, vocab - 1, 3, 9, 2], [4, 5, 0, 1, 3, 8, 12, 500, 0, 4, 10, 100]):
        check(run(ctx, x, dtype, vocab, T, given, 20), x, vocab, T, given, 20)
    assert ctx.poll_status() == 0


@gpu
def test_a_list_that_overflows_is_searched(ctx):
    """The largest logits all in one thread's vectors, more of them than the list holds."""
    for dtype, epc in (("f32", 4), ("bf16", 8)):
        vocab = 256 * epc * 500
        rng = np.random.default_rng(epc)
        x = logits(rng, 1000, 256 * epc * 16, dtype)                         # many rows: one CTA each
        v = torch.arange(x.shape[1], device="cuda") // epc
        x[3, :] = torch.where(v % 256 < 33, x[3].float() * 0.01 + 20.0, x[3].float()).to(x.dtype)
        given = rng.integers(0, x.shape[1], 1000)
        out = run(ctx, x, dtype, x.shape[1], 1.0, given, 32)
        sel = list(range(0, 8))
        check({k: a[sel] for k, a in out.items()}, x[sel], x.shape[1], 1.0, given[sel], 32)
        wide = logits(rng, 1, vocab, dtype)                                  # 33 neighbouring threads of each slice hold all large ones
        w = torch.arange(vocab, device="cuda") // epc
        wide[0] = torch.where(w % 256 < 33, wide[0].float() * 0.01 + 20.0, wide[0].float()).to(wide.dtype)
        check(run(ctx, wide, dtype, vocab, 1.0, [5], 32), wide, vocab, 1.0, [5], 32)
    assert ctx.poll_status() == 0


@gpu
def test_large_logits_and_temperatures(ctx):
    rng = np.random.default_rng(3)
    for dtype, spread, T in (("f32", 1e4, 1.0), ("bf16", 2e3, 100.0), ("f32", 3.0, 0.01), ("f32", 3.0, 1e4), ("f32", 1e30, 1e29), ("f32", 1e36, 2e-7),
                             ("bf16", 1e3, 1e-3)):
        x = logits(rng, 6, 5001, dtype, spread)
        given = rng.integers(0, 5001, 6)
        check(run(ctx, x, dtype, 5001, T, given, 10), x, 5001, T, given, 10)
    assert ctx.poll_status() == 0


@gpu
def test_agrees_with_confidence_and_replays(ctx):
    """The first alternative is focus_confidence's token and its probability the confidence; a captured call gives the bits of
    the eager one."""
    rng = np.random.default_rng(5)
    x = logits(rng, 40, 126464, "bf16")
    conf, tok = torch.zeros(40, device="cuda"), torch.zeros(40, dtype=torch.int32, device="cuda")
    fb.focus_confidence(ctx, x, fb.BF16, x.stride(0), 126464, 0, 40, None, None, 40, conf, tok)
    lp, ent = torch.zeros(40, device="cuda"), torch.zeros(40, device="cuda")
    rank, tt = torch.zeros(40, dtype=torch.int32, device="cuda"), torch.zeros((40, 3), dtype=torch.int32, device="cuda")
    tl = torch.zeros((40, 3), device="cuda")

    def call():
        fb.focus_token_logprobs(ctx, x, fb.BF16, x.stride(0), 126464, 0, 40, None, None, 40, 1.0, tok, lp, rank, ent, 3, tt, tl)

    call()
    assert torch.equal(tt[:, 0], tok) and (rank == 0).all() and torch.equal(lp, tl[:, 0])
    assert (lp.exp() / conf - 1).abs().max().item() < 1e-5
    want = [t.clone() for t in (lp, ent, rank, tt, tl)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        call()
    for _ in range(3):
        for t in (lp, ent, rank, tt, tl):
            t.zero_()
        g.replay()
        assert all(torch.equal(a, b) for a, b in zip((lp, ent, rank, tt, tl), want))
    assert ctx.poll_status() == 0
