"""focus_sample against the float64 oracle: temperature, top-k, top-p, min-p from given uniform numbers."""
import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import focus_oracle as fo
from paper_2602_02159_b200 import binding as fb
from paper_2602_02159_b200 import build as fbuild
from paper_2602_02159_b200 import step as fstep
from paper_2602_02159_b200 import workloads as wl

gpu = pytest.mark.gpu
DT = {"bf16": fb.BF16, "f32": fb.F32}
# conf and prob are rounded once to fp32 (2^-24).  conf is a quotient of weights that are off by less than 1e-9 of
# themselves: r in 2^r, |r| <= 2^-7, is rounded to 2^-33 (ln2 2^-32 = 1.7e-10 with the factor of both roundings), and
# 2^r - 1 < 0.0055 carries 2.5 roundings of 2^-24 (8.2e-10); so at most 2e-9 between two of them, and 1e-12 for sums in
# fp64.  prob's denominator has fp32 terms: exp2 is within 2 units in the last place (2^-22) and every thread adds at
# most vocab / 512 of them in fp32 (2^-24 each).
CONF_TOL = 2.0 ** -24 + 2e-9 + 1e-12


def prob_tol(vocab):
    return 2.0 ** -24 + 2.0 ** -22 + (vocab / 512 + 1) * 2.0 ** -24 + 1e-12


def single(x):
    return float(np.float32(x))


@pytest.fixture(scope="module")
def ctx():
    c = fb.Context(0)
    yield c
    assert c.poll_status() == 0
    c.close()


def run(ctx, xs, dtype, vocab, pos_base, rows, max_rows, T, k, p, mp, u, outputs=True):
    """xs: storage array [n_pos, stride]; rows: list of positions or None."""
    dx = fstep.to_device(xs, dtype)
    i32 = dict(dtype=torch.int32, device="cuda")
    dr = torch.tensor(list(rows) + [-1] * (max_rows - len(rows)), **i32) if rows is not None else None
    dn = torch.tensor([len(rows)], **i32) if rows is not None else None
    du = torch.from_numpy(np.asarray(u, dtype=np.float32)).cuda()
    conf, prob = torch.full((max_rows + 2,), 7.0, device="cuda"), torch.full((max_rows + 2,), 7.0, device="cuda")
    tok, kept = torch.full((max_rows + 2,), 7, **i32), torch.full((max_rows + 2,), 7, **i32)
    fb.focus_sample(ctx, dx, DT[dtype], xs.shape[1], vocab, pos_base, xs.shape[0], dr, dn, max_rows, T, k, p, mp, du, conf, tok,
                    prob if outputs else None, kept if outputs else None)
    out = [t.cpu().numpy() for t in (tok, conf, prob, kept)]
    assert all((o[max_rows:] == 7).all() for o in out)                       # nothing behind the rows is written
    return out


def check(out, x, rows_local, T, k, p, mp, u):
    tok, conf, prob, kept = out
    V = x.shape[1]
    for r, pr in enumerate(rows_local):
        et, ec, ep, en = fo.sample_token(x[pr], single(T), k, single(p), single(mp), single(u[r]))
        assert (int(tok[r]), int(kept[r])) == (et, en), (r, int(tok[r]), et, int(kept[r]), en)
        assert abs(float(conf[r]) - ec) <= CONF_TOL * ec + 1e-45 and abs(float(prob[r]) - ep) <= prob_tol(V) * ep + 1e-45


KNOBS = [(1.0, 0, 1.0, 0.0), (0.7, 0, 0.95, 0.0), (1.3, 50, 1.0, 0.0), (0.5, 20, 0.9, 0.05), (1.0, 0, 1.0, 0.1),
         (0.9, 1, 0.5, 0.0), (2.0, 700, 0.3, 0.01), (0.05, 0, 0.999, 0.0)]


@gpu
@pytest.mark.parametrize("knobs", KNOBS)
@pytest.mark.parametrize("dtype,vocab,stride,spread", [("bf16", 5000, 5000, 2.0), ("f32", 4099, 4100, 2.5), ("bf16", 7, 8, 1.0),
                                                       ("f32", 1, 4, 1.0), ("bf16", 32768, 32776, 0.5), ("f32", 12289, 12292, 4.0)])
def test_tokens_are_the_oracles(ctx, dtype, vocab, stride, spread, knobs):
    rng = np.random.default_rng(vocab + int(10 * knobs[0]))
    n_pos, pos_base = 12, 300
    xs = wl.to_storage((rng.standard_normal((n_pos, stride)) * spread).astype(np.float32), dtype)
    rows = sorted(rng.choice(n_pos, size=9, replace=False).tolist())
    u = rng.random(11)
    u[:3] = [0.0, np.nextafter(np.float32(1.0), np.float32(0.0)), 0.5]
    out = run(ctx, xs, dtype, vocab, pos_base, [pos_base + r for r in rows], 11, *knobs, u)
    check(out, wl.storage_to_f64(xs, dtype)[:, :vocab], rows, *knobs, u)
    assert (out[0][9:11] == -1).all() and (out[1][9:11] == 0).all() and (out[2][9:11] == 0).all() and (out[3][9:11] == 0).all()
    # the same rows without a list, and without the optional outputs
    again = run(ctx, xs, dtype, vocab, pos_base, None, 12, *knobs, np.concatenate([u, u[:1]])[:12], outputs=False)
    check((again[0], again[1], out[2] * 0, out[3]), wl.storage_to_f64(xs, dtype)[:0, :vocab], [], *knobs, u)
    one = run(ctx, xs, dtype, vocab, pos_base, None, 12, *knobs, np.concatenate([u, u[:1]])[:12])
    assert np.array_equal(one[0], again[0]) and np.array_equal(one[1], again[1])
    assert ctx.poll_status() == 0


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_ties_masks_and_infinities(ctx, dtype):
    rng = np.random.default_rng(4)
    V = 2000
    x = (rng.standard_normal((12, V)) * 2).astype(np.float32)
    x[0] = 1.5                                          # every token equal: ties cut by index
    x[1] = np.round(x[1])                               # a handful of values, hundreds of tokens each
    x[2, ::2] = -np.inf                                 # masked vocabulary
    x[3, :] = -np.inf
    x[3, 77] = -3.0                                     # one candidate
    x[4, :] = -np.inf                                   # none
    x[5, 10:30] = np.nan
    x[6, [5, 900, 1999]] = np.inf                       # infinities share the weight
    x[7, :] = np.nan
    x[8, :] = wl.storage_to_f64(wl.to_storage(np.array([np.finfo(np.float32).min], np.float32), "f32"), "f32")[0] if dtype == "f32" else -3.3e38
    x[8, 1234] = -1e38                                  # lowest values of the type, weight zero
    x[9, :] = -0.0
    x[9, 50:60] = 0.0                                   # the two zeros are equal
    x[10, 3] = 500.0                                    # everything else underflows
    xs = wl.to_storage(x, dtype)
    xf = wl.storage_to_f64(xs, dtype)
    for T, k, p, mp in ((1.0, 0, 1.0, 0.0), (0.8, 7, 1.0, 0.0), (1.0, 0, 0.5, 0.0), (1.2, 333, 0.75, 0.0), (0.6, 0, 0.9, 0.3),
                        (1.0, 100, 1.0, 1.0), (1.0, 0, 0.25, 0.0)):
        for u in (np.zeros(12), rng.random(12), np.full(12, 0.9999)):
            out = run(ctx, xs, dtype, V, 0, None, 12, T, k, p, mp, u)
            check(out, xf, range(12), T, k, p, mp, u)
    assert ctx.poll_status() == 0


@gpu
@pytest.mark.parametrize("dtype,vocab,max_rows", [("bf16", 126464, 3), ("f32", 126464, 2), ("bf16", 151936, 40), ("f32", 300001, 2)])
def test_long_rows(ctx, dtype, vocab, max_rows):
    """Rows that span a whole cluster, flat and peaked, with and without cuts."""
    rng = np.random.default_rng(vocab)
    stride = (vocab + 7) // 8 * 8
    x = rng.standard_normal((max_rows, stride)).astype(np.float32)
    x *= np.where(np.arange(max_rows) % 2 == 0, 0.4, 3.0)[:, None].astype(np.float32)
    xs = wl.to_storage(x, dtype)
    xf = wl.storage_to_f64(xs, dtype)[:, :vocab]
    for T, k, p, mp in ((1.0, 0, 1.0, 0.0), (1.0, 0, 0.9, 0.0), (0.8, 5000, 0.97, 0.0), (0.9, 50, 0.9, 0.02)):
        u = rng.random(max_rows)
        out = run(ctx, xs, dtype, vocab, 0, None, max_rows, T, k, p, mp, u)
        few = list(range(min(2, max_rows)))
        check(out, xf, few, T, k, p, mp, u)
        assert ((out[0][:max_rows] >= 0) & (out[0][:max_rows] < vocab)).all()
        # a row's answer does not depend on the rows beside it
        alone = run(ctx, xs[max_rows - 1:], dtype, vocab, 0, None, 1, T, k, p, mp, u[max_rows - 1:])
        assert alone[0][0] == out[0][max_rows - 1] and alone[3][0] == out[3][max_rows - 1]
    assert ctx.poll_status() == 0


@gpu
@pytest.mark.parametrize("dtype,vocab", [("bf16", 50003), ("f32", 30001)])
def test_many_rows(ctx, dtype, vocab):
    """More rows than SMs; every row is the one that a call of a few rows gives, three of them are the oracle's."""
    rng = np.random.default_rng(vocab)
    n, stride = 170, (vocab + 7) // 8 * 8
    x = rng.standard_normal((n, stride)).astype(np.float32) * np.array([0.3, 2.0, 3.5], np.float32)[np.arange(n) % 3, None]
    x[5, :100], x[6, 11:] = np.nan, -np.inf
    xs = wl.to_storage(x, dtype)
    xf = wl.storage_to_f64(xs, dtype)[:, :vocab]
    u = rng.random(n)
    for T, k, p, mp in ((0.8, 40, 0.9, 0.02), (0.7, 0, 0.95, 0.0), (1.0, 0, 1.0, 0.0), (1.0, 3000, 1.0, 0.001)):
        many = run(ctx, xs, dtype, vocab, 0, None, n, T, k, p, mp, u)
        for lo in range(0, n, 34):
            few = run(ctx, xs[lo:lo + 34], dtype, vocab, 0, None, 34, T, k, p, mp, u[lo:lo + 34])
            assert np.array_equal(few[0][:34], many[0][lo:lo + 34]) and np.array_equal(few[3][:34], many[3][lo:lo + 34])
            assert np.allclose(few[1][:34], many[1][lo:lo + 34], rtol=2 * CONF_TOL, atol=0)
        check([o[4:7] for o in many], xf[4:7], range(3), T, k, p, mp, u[4:7])
    assert ctx.poll_status() == 0


@gpu
def test_frequencies_follow_the_distribution(ctx):
    """u = (i + 1/2) / n for i < n: every kept token is drawn as often as its probability says, off by at most one."""
    rng = np.random.default_rng(12)
    V, n = 40, 4000
    x = (rng.standard_normal((1, V)) * 1.5).astype(np.float32)
    xs = np.repeat(x, n, axis=0)
    u = (np.arange(n) + 0.5) / n
    tok = run(ctx, xs, "f32", V, 0, None, n, 0.9, 12, 1.0, 0.0, u)[0][:n]
    order = np.argsort(-x[0], kind="stable")[:12]
    w = np.exp(x[0].astype(np.float64) / single(0.9))
    want = np.zeros(V)
    want[order] = w[order] / w[order].sum() * n
    assert (np.abs(np.bincount(tok, minlength=V) - want) <= 1.0).all()


@gpu
def test_top_k_of_one_is_the_confidence_call(ctx):
    """top_k = 1 draws the argmax that focus_confidence reports, prob is its confidence, whatever u is."""
    rng = np.random.default_rng(2)
    V, n = 30000, 24
    xs = wl.to_storage((rng.standard_normal((n, V)) * 3).astype(np.float32), "bf16")
    out = run(ctx, xs, "bf16", V, 0, None, n, 1.0, 1, 1.0, 0.0, rng.random(n))
    dx = fstep.to_device(xs, "bf16")
    conf, tok = torch.zeros(n, device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda")
    fb.focus_confidence(ctx, dx, fb.BF16, V, V, 0, n, None, None, n, conf, tok)
    assert np.array_equal(tok.cpu().numpy(), out[0][:n]) and (out[1][:n] == 1).all() and (out[3][:n] == 1).all()
    # focus_confidence sums fast-math exponentials of fp32 (2^-21 each)
    assert np.max(np.abs(conf.cpu().numpy() / out[2][:n] - 1)) <= 2.0 ** -20 + prob_tol(V)


@gpu
def test_bad_rows_and_numbers_are_reported(ctx):
    V = 64
    xs = wl.to_storage(np.random.default_rng(0).standard_normal((4, V)).astype(np.float32), "f32")
    good = run(ctx, xs, "f32", V, 10, [10, 11, 13], 3, 1.0, 0, 1.0, 0.0, [0.1, 0.2, 0.3])
    assert ctx.poll_status() == 0
    for rows, u, bad in (([10, 14, 13], [0.1, 0.2, 0.3], 1), ([9, 11, 13], [0.1, 0.2, 0.3], 0), ([10, 11, 13], [0.1, 1.0, 0.3], 1),
                         ([10, 11, 13], [0.1, 0.2, -0.1], 2), ([10, 11, 13], [np.nan, 0.2, 0.3], 0)):
        out = run(ctx, xs, "f32", V, 10, rows, 3, 1.0, 0, 1.0, 0.0, u)
        assert ctx.poll_status() == fb.ERR_INVALID_ARG
        assert out[0][bad] == -1 and out[1][bad] == 0 and out[2][bad] == 0 and out[3][bad] == 0
        for r in range(3):
            assert r == bad or (out[0][r] == good[0][r] and out[1][r] == good[1][r])


def test_refusals_need_no_device():
    fbuild.build()
    lib = fb.load_library()
    fake = ctypes.create_string_buffer(4096)
    h, P = ctypes.cast(fake, ctypes.c_void_p), 1 << 20

    def call(ctx=h, logits=P, dtype=fb.BF16, stride=1000, vocab=1000, base=0, n_pos=8, rows=None, n=None, max_rows=8, T=1.0, k=0,
             p=1.0, mp=0.0, u=P, conf=P, tok=P):
        return lib.focus_sample(ctx, logits, dtype, stride, vocab, base, n_pos, rows, n, max_rows, T, k, p, mp, u, conf, tok, None,
                                None, None)
    bad = [dict(ctx=None), dict(logits=None), dict(logits=P + 8), dict(dtype=2), dict(stride=999), dict(stride=1004), dict(vocab=0),
           dict(base=-1), dict(n_pos=-1), dict(max_rows=-1), dict(max_rows=9), dict(rows=P), dict(n=P), dict(T=0.0), dict(T=-1.0),
           dict(T=math.inf), dict(T=math.nan), dict(k=-1), dict(p=0.0), dict(p=1.5), dict(p=math.nan), dict(mp=-0.1), dict(mp=1.1),
           dict(mp=math.nan), dict(u=None), dict(conf=None), dict(tok=None)]
    for b in bad:
        assert call(**b) == fb.ERR_INVALID_ARG, b
    assert call(vocab=900_000, stride=900_000) == fb.ERR_UNSUPPORTED
    assert call(max_rows=0) == fb.OK


@gpu
def test_a_sampled_step_captured_and_replayed(ctx):
    """Logits -> drawn tokens -> state update (focus_commit_step), as one graph; new numbers and logits on replay."""
    rng = np.random.default_rng(6)
    L, M, V, n = 200, 120, 3000, 30
    pos = np.sort(rng.choice(np.arange(M, L), size=n, replace=False))
    i32 = dict(dtype=torch.int32, device="cuda")
    rows, n_rows = torch.from_numpy(pos.astype(np.int32)).cuda(), torch.tensor([n], **i32)
    logits, u = torch.zeros(L - M, V, device="cuda").bfloat16(), torch.zeros(n, device="cuda")
    conf, masked, x = torch.zeros(L, device="cuda"), torch.zeros(L, dtype=torch.uint8, device="cuda"), torch.zeros(L, **i32)
    cn, tn, pr = torch.zeros(n, device="cuda"), torch.zeros(n, **i32), torch.zeros(n, device="cuda")
    out, n_out = torch.zeros(4, **i32), torch.zeros(1, **i32)

    def fill():
        logits.copy_(torch.from_numpy(rng.standard_normal((L - M, V)).astype(np.float32) * 2))
        u.copy_(torch.from_numpy(rng.random(n).astype(np.float32)))
        masked.zero_(), x.zero_(), conf.zero_()
        masked[M:] = 1

    def step():
        fb.focus_sample(ctx, logits, fb.BF16, V, V, M, L - M, rows, n_rows, n, 0.8, 40, 0.9, 0.01, u, cn, tn, pr)
        fb.focus_commit_step(ctx, pr, tn, M, rows, n_rows, n, L, M, L, 4, conf, masked, x, out, n_out)

    def check_state():
        torch.cuda.synchronize()
        xf = logits.double().cpu().numpy()
        want = [fo.sample_token(xf[p - M], single(0.8), 40, single(0.9), single(0.01), float(u[r])) for r, p in enumerate(pos)]
        assert tn.cpu().numpy().tolist() == [w[0] for w in want]
        _, em, ex, picks = fo.commit_step(np.zeros(L, np.float32), np.r_[np.zeros(M, np.uint8), np.ones(L - M, np.uint8)],
                                          np.zeros(L, np.int32), pos.tolist(), pr.cpu().numpy(), [w[0] for w in want], M, L, 4)
        assert out.cpu().numpy().tolist() == picks and np.array_equal(x.cpu().numpy(), ex) and np.array_equal(masked.cpu().numpy(), em)

    fill(), step(), check_state()
    fill()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    for _ in range(2):
        fill(), graph.replay(), check_state()
    assert ctx.poll_status() == 0


@gpu
@pytest.mark.parametrize("n", [3, 160])
def test_rows_beyond_32_bits(ctx, n):
    """Logits rows more than 2^32 bytes apart in all (in slices and in place)."""
    V, stride = 40000, (1 << 32) // 2 // 150 // 8 * 8
    buf = torch.empty(n * stride if n > 3 else 160 * stride, dtype=torch.bfloat16, device="cuda")
    pos = list(range(n)) if n > 3 else [0, 100, 159]
    n_pos = 160
    rows = buf.as_strided((n_pos, V), (stride, 1))
    rows.copy_(torch.randn(n_pos, V, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda") * 3)
    dr, dn = torch.tensor(pos, dtype=torch.int32, device="cuda"), torch.tensor([n], dtype=torch.int32, device="cuda")
    u = torch.linspace(0.01, 0.99, n, device="cuda")
    conf, tok = torch.zeros(n, device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda")
    for k, p in ((40, 0.9), (0, 0.95), (0, 1.0)):
        fb.focus_sample(ctx, buf, fb.BF16, stride, V, 0, n_pos, dr, dn, n, 0.8, k, p, 0.0, u, conf, tok, None, None)
        for r in (0, n // 2, n - 1):
            et, ec, _, _ = fo.sample_token(rows[pos[r]].double().cpu().numpy(), single(0.8), k, single(p), 0.0, float(u[r]))
            assert int(tok[r]) == et and abs(float(conf[r]) - ec) <= CONF_TOL * ec
    assert ctx.poll_status() == 0


@gpu
@pytest.mark.parametrize("scale,T", [(1e4, 1.0), (1e-3, 1e-4), (3e5, 40.0), (1.0, 1e-3), (1e-30, 1e-30)])
def test_logits_of_any_size(ctx, scale, T):
    """Exponents x / T far beyond 4096 (where the difference to the maximum is taken first), and tiny or huge temperatures;
    the logits spread over a few T, so that the cuts have work to do."""
    rng = np.random.default_rng(3)
    V = 6001
    x = (scale + rng.standard_normal((8, 6004)) * T * 2.0).astype(np.float32)
    u = rng.random(8)
    for k, p, mp in ((0, 1.0, 0.0), (0, 0.9, 0.0), (30, 0.8, 0.0), (0, 1.0, 0.01)):
        out = run(ctx, x, "f32", V, 0, None, 8, T, k, p, mp, u)
        tok, conf, _, kept = out
        for r in range(8):
            et, ec, _, en = fo.sample_token(x[r, :V].astype(np.float64), single(T), k, single(p), single(mp), single(u[r]))
            assert (int(tok[r]), int(kept[r])) == (et, en) and abs(float(conf[r]) - ec) <= CONF_TOL * ec
    assert ctx.poll_status() == 0


@gpu
@pytest.mark.parametrize("min_p", [0.002, 0.02, 0.2, 0.55, 1.0])
@pytest.mark.parametrize("dtype,spread,top_p", [("bf16", 0.5, 0.7), ("f32", 0.5, 0.3), ("f32", 0.5, 0.999), ("bf16", 3.0, 0.95)])
def test_min_p_before_within_and_behind_a_long_nucleus(ctx, dtype, spread, top_p, min_p):
    """min-p that ends the set before a nucleus of thousands of tokens, that cuts near its end, and that has no say."""
    rng = np.random.default_rng(int(1000 * min_p))
    V = 32003
    xs = wl.to_storage((rng.standard_normal((6, 32008)) * spread).astype(np.float32), dtype)
    u = rng.random(6)
    out = run(ctx, xs, dtype, V, 0, None, 6, 0.9, 0, top_p, min_p, u)
    check(out, wl.storage_to_f64(xs, dtype)[:, :V], range(6), 0.9, 0, top_p, min_p, u)
    assert ctx.poll_status() == 0


@gpu
@pytest.mark.parametrize("V", [40, 700])
def test_a_nucleus_of_half_between_two_equal_maxima(ctx, V):
    """Two tokens share all the weight that fp64 sees beside them: the first is half of it, and u = 0 draws the first of them."""
    x = np.full((2, (V + 3) // 4 * 4), -50.0, dtype=np.float32)
    x[:, 7] = x[:, 30] = 4.0
    for k, p, want in ((0, 0.5, 1), (20, 0.5, 1), (0, 0.75, 2), (2, 1.0, 2)):
        tok, _, _, kept = run(ctx, x, "f32", V, 0, None, 2, 0.1, k, p, 0.0, [0.0, 0.999])
        assert kept[:2].tolist() == [want, want] and tok[:2].tolist() == [7, 7 if want == 1 else 30]
    tok, _, _, kept = run(ctx, x, "f32", V, 0, None, 2, 1.0, 0, 1.0, 0.0, [0.0, 0.999])
    assert kept[:2].tolist() == [V, V] and tok[:2].tolist() == [0, 30]       # e^-54 is a weight, if a small one
    assert ctx.poll_status() == 0


def _edge_logits(sign, n_values, apart):
    """A temperature and descending fp32 logits for the far end of a histogram's precision.  log2(e) / T = s_hi + s_lo with
    |s_lo| near half a step of s_hi, and x s_hi near 4096 for all of them, each x s_hi close to the upper (sign 1) or lower
    edge (sign -1) between two multiples of 1/64, which x s_lo then oversteps by a 64th of a 64th."""
    T = np.float32(1.44)
    while True:
        s = 1.4426950408889634 / float(T)
        s_hi = float(np.float32(s))
        if s > 1.0 and sign * (s - s_hi) > 0.49 * 2.0 ** -23:
            break
        T = np.nextafter(T, np.float32(0))
    x, out, last = np.float32(4095.0 / s), [], None
    while len(out) < n_values:
        e = float(x) * s_hi * 64
        b = round(e)
        if sign * (e - b) > 0.4975 and (last is None or last - b >= apart):
            out.append(x)
            last = b
        x = np.nextafter(x, np.float32(0))
    return float(T), np.array(out, dtype=np.float32)


@gpu
@pytest.mark.parametrize("min_p", [0.0, 0.02, 0.2])
@pytest.mark.parametrize("shuffled", [True, False])
@pytest.mark.parametrize("sign", [1, -1])
def test_a_nucleus_that_ends_beside_the_edges_of_its_histogram(ctx, sign, shuffled, min_p):
    """Equal logits 150 at a time, all of them on an edge; top-p 1e-5 on either side of a group's running weight."""
    per = 150
    T, values = _edge_logits(sign, 40, 8)
    x = np.repeat(values, per)
    if shuffled:
        np.random.default_rng(1).shuffle(x)
    xs = np.stack([x, x])
    w = np.exp((values.astype(np.float64) - float(values[0])) / single(T))
    share = np.cumsum(w) / w.sum()
    wrong = []
    for j in (4, 11, 19, 26, 33):
        for side in (1 - 1e-5, 1 + 1e-5):
            top_p, u = single(share[j] * side), [0.3, 0.999]
            out = run(ctx, xs, "f32", len(x), 0, None, 2, T, 0, top_p, min_p, u)
            for r in range(2):
                want = fo.sample_token(x.astype(np.float64), single(T), 0, top_p, single(min_p), single(u[r]))
                if (int(out[0][r]), int(out[3][r])) != (want[0], want[3]):
                    wrong.append((j, side, r, int(out[0][r]), int(out[3][r]), want[0], want[3]))
    assert not wrong, wrong
    assert ctx.poll_status() == 0


@gpu
@pytest.mark.parametrize("knobs", KNOBS)
@pytest.mark.parametrize("dtype,vocab,stride,spread", [("bf16", 5000, 5000, 2.0), ("f32", 4099, 4100, 2.5), ("bf16", 32768, 32776, 0.5)])
def test_rows_without_a_list_start_at_the_base(ctx, dtype, vocab, stride, spread, knobs):
    """No list: row r is position pos_base + r, whose logits are the r-th row; every row is the oracle's, with and without the
    optional outputs."""
    rng = np.random.default_rng(vocab + int(10 * knobs[0]))
    xs = wl.to_storage((rng.standard_normal((12, stride)) * spread).astype(np.float32), dtype)
    u = rng.random(12)
    out = run(ctx, xs, dtype, vocab, 300, None, 12, *knobs, u)
    check(out, wl.storage_to_f64(xs, dtype)[:, :vocab], range(12), *knobs, u)
    bare = run(ctx, xs, dtype, vocab, 300, None, 12, *knobs, u, outputs=False)
    assert np.array_equal(bare[0], out[0]) and np.array_equal(bare[1], out[1])
    assert ctx.poll_status() == 0


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("knobs", [(0.1, 3000, 1.0, 0.0), (0.1, 20000, 1.0, 0.0), (0.1, 0, 1.0, 0.0), (0.1, 0, 0.99, 0.0), (0.1, 40, 1.0, 0.0),
                                   (0.1, 3000, 0.9, 0.0), (0.1, 3000, 1.0, 0.5)])
def test_a_number_of_zero_beside_weights_that_vanish(ctx, dtype, knobs):
    """One logit a thousand temperatures above the rest, whose weights no 64-bit float holds: u = 0 draws that one, wherever it lies
    and however many others the cuts keep."""
    rng = np.random.default_rng(7)
    V = 40001
    x = rng.standard_normal((4, 40008)).astype(np.float32)
    for r, at in enumerate((0, 17000, 31111, V - 1)):
        x[r, at] = 120.0
    xs = wl.to_storage(x, dtype)
    for u in (np.zeros(4), np.full(4, 1e-44), np.full(4, 0.5)):
        out = run(ctx, xs, dtype, V, 0, None, 4, *knobs, u)
        check(out, wl.storage_to_f64(xs, dtype)[:, :V], range(4), *knobs, u)
        assert out[0][:4].tolist() == [0, 17000, 31111, V - 1] and (out[1][:4] == 1).all()
    assert ctx.poll_status() == 0
