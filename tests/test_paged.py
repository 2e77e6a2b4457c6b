"""Rotary positions (focus_rotate), the paged cache's write side (focus_append_kv_paged) and attention over it
(focus_paged_attn), against the float64 oracle.

Tolerances, in units of what is computed.  A stored element is off by half a step of its type (HALF, relative).  A turn is
off by 2^-21 of |x1| + |x2|: the phase 2^-33 turns and 2^-26 by its conversion, cosine and sine 2 units in the last place,
product and sum 2^-24 each.  A logit, a sum of d fp32 products, is off by d 2^-24 of the sum of their magnitudes; a
numerator by that (and 2^-20 for the exponential and the scale), and in bf16 by HALF more, or 2^-16 where it is
held in two terms (up to 16 stacked rows on average); an output by the numerators'
error times sum w |v| (which also bounds the sums' errors, n 2^-24, in fp32) and HALF of itself."""
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
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
LAYOUT = {"halves": fb.ROPE_HALVES, "pairs": fb.ROPE_PAIRS}
SCALING = {"plain": (500000.0, 1.0, 1.0, 1.0, 0), "linear": (10000.0, 4.0, 1.0, 1.0, 0), "ntk": (10000.0, 8.0, 1.0, 1.0, 0),
           "bands": (500000.0, 8.0, 1.0, 4.0, 8192), "yarn": (1000000.0, 4.0, 1.0, 32.0, 32768)}
KIND = {"plain": fb.ROPE_PLAIN, "linear": fb.ROPE_LINEAR, "ntk": fb.ROPE_NTK, "bands": fb.ROPE_BANDS, "yarn": fb.ROPE_YARN}


@pytest.fixture(scope="module")
def lib():
    fbuild.build()
    return fb.load_library()


@pytest.fixture(scope="module")
def ctx():
    c = fb.Context(0)
    yield c
    assert c.poll_status() == 0
    c.close()


def rope_of(rot, layout, scaling):
    base, factor, low, high, trained = SCALING[scaling]
    return fb.make_rope(rot, LAYOUT[layout], base, KIND[scaling], factor, low, high, trained)


def f64(t):
    return t.detach().double().cpu().numpy()


def i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


# ---- plans and refusals: no device ------------------------------------------------------------------------------
@pytest.mark.parametrize("scaling", sorted(SCALING))
@pytest.mark.parametrize("rot", [16, 48, 64, 128])
def test_plans_hold_the_frequencies(lib, scaling, rot):
    base, factor, low, high, trained = SCALING[scaling]
    f, m = fo.rope_frequencies(rot, base, scaling, factor, low, high, trained)
    r = rope_of(rot, "halves", scaling)
    got = np.array([t / 2.0 ** 64 for t in r.turn[:rot // 2]])
    # pow and log of two libraries: 1e-14 of the value; and a fraction is rounded to a multiple of 2^-64
    assert (np.abs(got - f / (2 * math.pi)) <= 1e-14 * f + 2.0 ** -65).all()
    assert abs(r.magnitude - m) <= 2.0 ** -24 * m and r.rot_dim == rot and list(r.turn[rot // 2:]) == [0] * (64 - rot // 2)


def test_plans_from_frequencies_are_fractions_of_a_turn(lib):
    f = [0.0, 2 * math.pi, math.pi, 7.5, 1e-9, 1.0, 100.0, 3.0]
    r = fb.make_rope_from_frequencies(fb.ROPE_PAIRS, f, 0.5)
    assert r.rot_dim == 16 and r.layout == fb.ROPE_PAIRS and r.magnitude == 0.5
    from decimal import Decimal, getcontext
    getcontext().prec = 50
    two_pi = Decimal("6.28318530717958647692528676655900576839433879875021")
    for got, want in zip(r.turn, f):
        t = Decimal(want) / two_pi
        frac = (t - int(t)) * 2 ** 64
        assert min(abs(got - frac), 2 ** 64 - abs(got - frac)) <= 2 + abs(t) * 2          # units of 2^-64, relative 2^-63 of t


def test_plan_refusals(lib):
    r = fb.focus_rope()
    B = ctypes.byref

    def init(rope=B(r), rot=64, layout=0, base=1e4, kind=0, factor=1.0, low=1.0, high=4.0, trained=4096):
        return lib.focus_rope_init(rope, rot, layout, base, kind, factor, low, high, trained)

    assert init() == fb.OK
    nan = float("nan")
    for bad in (dict(rope=None), dict(rot=0), dict(rot=8), dict(rot=24), dict(rot=144), dict(rot=-16), dict(layout=2),
                dict(base=1.0), dict(base=nan), dict(base=math.inf), dict(kind=5), dict(kind=-1), dict(kind=1, factor=0.5),
                dict(kind=2, factor=nan), dict(kind=2, factor=1e308), dict(kind=3, low=0.0), dict(kind=3, high=1.0),
                dict(kind=4, trained=0), dict(kind=4, high=math.inf), dict(kind=4, low=nan)):
        assert init(**bad) == fb.ERR_INVALID_ARG, bad
    D = ctypes.c_double * 8

    def given(rope=B(r), rot=16, layout=0, f=D(*[1.0] * 8), m=1.0):
        return lib.focus_rope_from_frequencies(rope, rot, layout, f, m)

    assert given() == fb.OK
    for bad in (dict(rope=None), dict(f=None), dict(m=nan), dict(rot=12), dict(layout=3), dict(f=D(*[1.0] * 7, -1.0)),
                dict(f=D(*[1.0] * 7, nan)), dict(f=D(*[1.0] * 7, math.inf))):
        assert given(**bad) == fb.ERR_INVALID_ARG, bad


def test_refusals_need_no_device(lib):
    fake = ctypes.create_string_buffer(4096)                                 # read by no call that is refused
    P, h, B = 1 << 20, ctypes.cast(fake, ctypes.c_void_p), ctypes.byref
    rope = fb.make_rope(64, fb.ROPE_HALVES, 1e4)
    wide = fb.make_rope(128, fb.ROPE_HALVES, 1e4)
    torn = fb.make_rope(64, fb.ROPE_HALVES, 1e4)
    torn.rot_dim = 40

    def rotate(ctx=h, rope=rope, direction=1, X=P, Y=2 * P, dtype=fb.BF16, heads=4, d=64, xr=256, xh=64, yr=256, yh=64,
               base=0, pos=None, n=None, rows=8):
        return lib.focus_rotate(ctx, B(rope), direction, X, Y, dtype, heads, d, xr, xh, yr, yh, base, pos, n, rows, None)

    for bad in (dict(ctx=None), dict(direction=0), dict(X=None), dict(Y=None), dict(X=P + 8), dict(Y=P + 2), dict(dtype=2),
                dict(heads=0), dict(rows=-1), dict(xr=56), dict(xh=68), dict(yr=260), dict(yh=32), dict(X=P, Y=P, yr=512),
                dict(pos=P), dict(n=P), dict(base=-1), dict(base=2 ** 31 - 4), dict(rope=torn)):
        assert rotate(**bad) == fb.ERR_INVALID_ARG, bad
    assert rotate(d=32) == fb.ERR_UNSUPPORTED and rotate(rope=wide) == fb.ERR_UNSUPPORTED and rotate(rows=0) == fb.OK

    sh = fb.make_shape(256, 0, 4, 2, 64, 64, fb.BF16)

    def cache(K=P, V=2 * P, table=P, lens=P, page=16, n_pages=9, n=3, wide=16, sp=2048, st=128, sh=64):
        return fb.make_paged_cache(K, V, table, lens, page, n_pages, n, wide, sp, st, sh)

    def append(ctx=h, shape=sh, rope=rope, Q=P, K=P, V=P, row=512, head=64, start=P, pos=None, rows=8, c=cache(), Q_out=2 * P):
        return lib.focus_append_kv_paged(ctx, B(shape), None if rope is None else B(rope), Q, K, V, row, head, start, pos, rows,
                                         B(c), Q_out, None)

    def attend(ctx=h, shape=sh, Q=P, start=P, rows=8, c=cache(), O=P, lse=None):
        return lib.focus_paged_attn(ctx, B(shape), Q, start, rows, B(c), O, lse, None)

    for call in (append, attend):
        for bad in (dict(K=None), dict(V=None), dict(K=P + 8), dict(table=None), dict(lens=None), dict(table=P + 2),
                    dict(lens=P + 1), dict(page=0), dict(n_pages=0), dict(n=-1), dict(wide=15), dict(wide=0), dict(sp=2049),
                    dict(st=32), dict(sh=60), dict(page=8)):
            assert call(c=cache(**bad)) == fb.ERR_INVALID_ARG, bad
        assert call(ctx=None) == fb.ERR_INVALID_ARG and call(rows=-1) == fb.ERR_INVALID_ARG
        assert call(start=P + 2) == fb.ERR_INVALID_ARG
        assert call(start=None, rows=8) == fb.ERR_INVALID_ARG                                # one row per sequence: 3
        assert call(shape=fb.make_shape(256, 0, 4, 3, 64, 64, fb.BF16)) == fb.ERR_INVALID_ARG
        assert call(shape=fb.make_shape(256, 0, 4, 2, 64, 64, 2)) == fb.ERR_INVALID_ARG
        assert call(rows=0) == fb.OK
    small = fb.make_shape(64, 0, 4, 2, 32, 64, fb.BF16)
    assert append(shape=small, rope=None) == fb.ERR_UNSUPPORTED and attend(shape=small) == fb.ERR_UNSUPPORTED
    for bad in (dict(K=None), dict(V=None), dict(Q=None), dict(Q_out=None), dict(Q=None, Q_out=None, K=None, V=None),
                dict(Q=P + 4), dict(Q_out=P + 4), dict(row=60), dict(head=68), dict(Q=P, Q_out=P), dict(rope=torn)):
        assert append(**bad) == fb.ERR_INVALID_ARG, bad
    assert append(rope=wide) == fb.ERR_UNSUPPORTED
    for bad in (dict(Q=None), dict(O=None), dict(Q=P + 8), dict(O=P + 8), dict(lse=P + 2)):
        assert attend(**bad) == fb.ERR_INVALID_ARG, bad
    assert rotate(rows=2 ** 30 + 1) == fb.ERR_UNSUPPORTED and append(rows=2 ** 30 + 1) == fb.ERR_UNSUPPORTED
    assert attend(rows=2 ** 28 + 1) == fb.ERR_UNSUPPORTED                                    # 4 heads
    far = fb.make_shape(2 ** 30 + 1, 0, 4, 2, 64, 64, fb.BF16)
    assert attend(shape=far, c=cache(wide=2 ** 27)) == fb.ERR_UNSUPPORTED
    out = ctypes.c_size_t(0)
    assert lib.focus_paged_attn_workspace_bytes(None, B(sh), ctypes.byref(out)) == fb.ERR_INVALID_ARG
    assert lib.focus_paged_attn_workspace_bytes(h, B(sh), None) == fb.ERR_INVALID_ARG


# ---- turning ----------------------------------------------------------------------------------------------------
def turn_bound(x, rot, layout, want, dtype, magnitude):
    """Per element: 2^-21 of the pair's magnitudes where it turns, half a step of the result."""
    pair = np.zeros_like(x)
    half = rot // 2
    a, b = (slice(0, half), slice(half, rot)) if layout == "halves" else (slice(0, rot, 2), slice(1, rot, 2))
    size = (np.abs(x[..., a]) + np.abs(x[..., b])) * magnitude
    pair[..., a], pair[..., b] = size, size
    return pair * 2.0 ** -21 + np.abs(want) * HALF[dtype] + 1e-37


@gpu
@pytest.mark.parametrize("dtype,layout,scaling,d,rot,heads,rows,listed", [
    ("bf16", "halves", "plain", 128, 128, 5, 3, True), ("bf16", "pairs", "yarn", 128, 64, 33, 37, False),
    ("f32", "halves", "bands", 64, 48, 3, 129, True), ("f32", "pairs", "ntk", 128, 128, 40, 1, False),
    ("bf16", "halves", "linear", 64, 16, 1, 5000, True), ("f32", "pairs", "plain", 64, 16, 2, 4800, False),
    ("bf16", "halves", "yarn", 128, 112, 7, 260, True)])
def test_rows_turn_by_their_positions(ctx, dtype, layout, scaling, d, rot, heads, rows, listed):
    rng = np.random.default_rng(rows + heads)
    base, factor, low, high, trained = SCALING[scaling]
    f, m = fo.rope_frequencies(rot, base, scaling, factor, low, high, trained)
    pos_base = 0 if listed else 2 ** 31 - 1 - rows
    pos = rng.integers(0, 2 ** 31 - 1, rows) if listed else np.arange(rows) + pos_base
    pos[0] = 0 if listed else pos[0]
    extra, pad = 2, 8
    X = torch.from_numpy(rng.standard_normal((rows + extra, heads + 1, d + pad))).cuda().to(REAL[dtype])
    Y = torch.full((rows + extra, heads, d), 7.0, device="cuda").to(REAL[dtype])
    positions = i32(pos.tolist() + [5] * extra) if listed else None
    n_rows = i32([rows]) if listed else None
    rope = rope_of(rot, layout, scaling)
    for direction in (1, -1):
        Y.fill_(7.0)
        fb.focus_rotate(ctx, rope, direction, X, Y, DT[dtype], heads, d, X.stride(0), X.stride(1), Y.stride(0), Y.stride(1),
                        pos_base, positions, n_rows, rows + (extra if listed else 0))
        x = f64(X)[:rows, :heads, :d]
        # an angle in 64 bits is off by p f 2^-53, 2^-22 at 2^31: the phase modulo 2 pi from the plan's exact fractions
        phase = np.array([[(int(p) * int(t) % 2 ** 64) / 2.0 ** 64 for t in rope.turn[:rot // 2]] for p in pos]) * 2 * math.pi
        want = np.array(x)
        half = rot // 2
        a, b = (slice(0, half), slice(half, rot)) if layout == "halves" else (slice(0, rot, 2), slice(1, rot, 2))
        c, s = (np.cos(phase) * m)[:, None], (np.sin(phase) * m * direction)[:, None]
        want[..., a], want[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
        got = f64(Y)
        assert (np.abs(got[:rows] - want) <= turn_bound(x, rot, layout, want, dtype, m)).all()
        assert np.array_equal(got[:rows, :, rot:], x[..., rot:])                             # copied as they are
        assert (got[rows:] == 7.0).all()
        near = [r for r in range(rows) if pos[r] < 2 ** 20][:8]                              # the definition itself
        if near:
            w = fo.rotate(x[near], pos[near], f, layout, m, direction)
            # the plan's fractions differ from the oracle's frequencies by 1e-14 of an angle below 2^20, twice
            assert (np.abs(got[near] - w) <= turn_bound(x[near], rot, layout, w, dtype, m) + 2e-8 * np.abs(x[near]).max()).all()
    assert ctx.poll_status() == 0


@gpu
def test_in_place_back_and_forth_and_bad_positions(ctx):
    rng = np.random.default_rng(0)
    rope = rope_of(48, "halves", "plain")
    X = torch.from_numpy(rng.standard_normal((6, 3, 64))).cuda().float()
    before, Y = X.clone(), torch.empty_like(X)
    pos, n = i32([4, 0, -1, 100000, 7, 9]), i32([5])
    args = (fb.F32, 3, 64, 192, 64, 192, 64, 0, pos, n, 6)
    fb.focus_rotate(ctx, rope, 1, X, Y, *args)
    assert ctx.poll_status() == fb.ERR_INVALID_ARG                           # the row at -1 is reported
    fb.focus_rotate(ctx, rope, 1, X, X, *args)
    assert ctx.poll_status() == fb.ERR_INVALID_ARG
    live = [0, 1, 3, 4]
    assert torch.equal(X[live], Y[live]) and torch.equal(X[2], before[2]) and torch.equal(X[5], before[5])
    assert torch.equal(X[:, :, 48:], before[:, :, 48:])
    fb.focus_rotate(ctx, rope, -1, X, X, *args)
    assert ctx.poll_status() == fb.ERR_INVALID_ARG
    assert (X[live] - before[live]).abs().max().item() <= 2 * 2.0 ** -21 * 2 * before.abs().max().item() * 2


@gpu
@pytest.mark.parametrize("layout", ["halves", "pairs"])
def test_the_opposite_direction_is_the_gradient(ctx, layout):
    """<g, turn(x)> has the gradient turn^T(g): from the formula, and from differences (exact to rounding: it is linear)."""
    rng = np.random.default_rng(3)
    rope = rope_of(64, layout, "yarn")
    f, m = fo.rope_frequencies(64, 1000000.0, "yarn", 4.0, 1.0, 32.0, 32768)
    x, g, u = (torch.from_numpy(rng.standard_normal((9, 2, 64))).cuda().float() for _ in range(3))
    pos = rng.integers(0, 100000, 9)

    def turn(t, direction):
        y = torch.empty_like(t)
        fb.focus_rotate(ctx, rope, direction, t, y, fb.F32, 2, 64, 128, 64, 128, 64, 0, i32(pos.tolist()), i32([9]), 9)
        return f64(y)

    grad = turn(g, -1)
    assert np.abs(grad - fo.rotate(f64(g), pos, f, layout, m, -1)).max() <= 2.0 ** -21 * 2 * m * float(g.abs().max()) + 1e-8
    step = 2.0 ** -3                                                          # exact in fp32 up to one rounding of x + step u
    diff = ((turn(x + step * u, 1) - turn(x, 1)) / step * f64(g)).sum()
    assert abs(diff - (grad * f64(u)).sum()) <= 9 * 128 * 4 * 2.0 ** -20 / step


# ---- the paged cache --------------------------------------------------------------------------------------------
class Cache:
    """Pools with NaN wherever no token lies, pages in shuffled order, a table with -1 behind each sequence's pages."""

    def __init__(self, rng, dtype, Hkv, d, page, lengths, L, heads_first=False, pad=0, fill=True):
        self.rng, self.dtype, self.Hkv, self.d, self.page, self.lengths, self.L = rng, dtype, Hkv, d, page, lengths, L
        self.heads_first = heads_first
        need = [-(-t // page) for t in lengths]
        self.wide, self.n_pages = -(-L // page) + 1, sum(need) + 3
        shape = (self.n_pages, Hkv, page, d + pad) if heads_first else (self.n_pages, page, Hkv, d + pad)
        self.pool = [torch.full(shape, float("nan"), device="cuda").to(REAL[dtype]) for _ in range(2)]
        order = rng.permutation(self.n_pages)
        self.table = np.full((len(lengths), self.wide), -1, dtype=np.int32)
        at = 0
        for s, k in enumerate(need):
            self.table[s, :k] = order[at:at + k]
            at += k
        self.tokens = []                                                     # [(keys, values)] of each sequence, [n, Hkv, d]
        for s, t in enumerate(lengths):
            kv = []
            for pool in self.pool:
                x = torch.from_numpy(rng.standard_normal((t, Hkv, d))).to(REAL[dtype])
                if fill and t:
                    j = np.arange(t)
                    self.first(pool)[torch.from_numpy(self.table[s, j // page].astype(np.int64)), torch.from_numpy(j % page),
                                     :, :d] = x.cuda()
                kv.append(f64(x))
            self.tokens.append(kv)
        self.d_table, self.d_len = torch.from_numpy(self.table).cuda(), i32(list(lengths))

    def first(self, pool):
        return pool.transpose(1, 2) if self.heads_first else pool

    def c(self):
        K, tok, head = self.pool[0], *((2, 1) if self.heads_first else (1, 2))
        return fb.make_paged_cache(K, self.pool[1], self.d_table, self.d_len, self.page, self.n_pages, len(self.lengths),
                                   self.wide, K.stride(0), K.stride(tok), K.stride(head))

    def shape(self, H, **kw):
        return fb.make_shape(self.L, 0, H, self.Hkv, self.d, 64, DT[self.dtype], **kw)


def starts(rows):
    return np.concatenate([[0], np.cumsum(rows)]).tolist()


@gpu
@pytest.mark.parametrize("dtype,H,Hkv,d,page,rot,rows,mode,heads_first", [
    ("bf16", 4, 2, 64, 16, 64, None, "last", False), ("f32", 6, 1, 128, 1, 48, [3, 0, 5, 1], "last", True),
    ("bf16", 7, 7, 128, 7, 128, [2, 11, 0, 30], "listed", False), ("f32", 2, 2, 64, 64, None, [1, 1, 1, 1], "listed", True),
    ("bf16", 28, 4, 128, 32, 64, [33, 40, 1, 7], "last", True), ("f32", 3, 3, 64, 5, 16, None, "listed", False)])
def test_appended_rows_land_in_their_pages(ctx, dtype, H, Hkv, d, page, rot, rows, mode, heads_first):
    rng = np.random.default_rng(H * d + page)
    lengths = [33, 40, 9, 77]
    c = Cache(rng, dtype, Hkv, d, page, lengths, 80, heads_first, pad=8)
    before = [f64(p) for p in c.pool]
    n = rows or [1] * 4
    start, total, behind = starts(n), sum(n), 3 if rows else 0
    x = torch.from_numpy(rng.standard_normal((total + behind, H + 2 * Hkv, d))).cuda().to(REAL[dtype])
    Q, K, V = x[:, :H], x[:, H:H + Hkv], x[:, H + Hkv:]
    pos = [np.arange(t - k, t) if mode == "last" else rng.permutation(t)[:k] for t, k in zip(lengths, n)]
    flat = np.concatenate(pos).astype(int)
    Qo = torch.full((total + behind, H, d), 7.0, device="cuda").to(REAL[dtype])
    rope = rope_of(rot, "pairs", "bands") if rot else None
    fb.focus_append_kv_paged(ctx, c.shape(H), rope, Q, K, V, x.stride(0), x.stride(1), i32(start) if rows else None,
                             None if mode == "last" else i32(flat.tolist() + [0] * behind), total + behind, c.c(), Qo)
    f, m = fo.rope_frequencies(rot, *([SCALING["bands"][0], "bands"] + list(SCALING["bands"][1:]))) if rot else (np.zeros(0), 1.0)
    got_q = f64(Qo)
    qx, kx, vx = f64(Q)[:total], f64(K)[:total], f64(V)[:total]
    wq, wk = (fo.rotate(t, flat, f, "pairs", m) for t in (qx, kx))
    assert (np.abs(got_q[:total] - wq) <= turn_bound(qx, rot or 0, "pairs", wq, dtype, m)).all()
    assert (got_q[total:] == 7.0).all()
    touched = np.zeros(before[0].shape[0:1] + (page,), dtype=bool)
    K_now, V_now = (f64(c.first(p)) for p in c.pool)
    for s in range(4):
        for t, p in enumerate(pos[s]):
            r, at = start[s] + t, (c.table[s, p // page], p % page)
            touched[at] = True
            bound = turn_bound(kx[r], rot or 0, "pairs", wk[r], dtype, m)
            assert (np.abs(K_now[at][:, :d] - wk[r]) <= bound).all()
            assert np.array_equal(V_now[at][:, :d], vx[r])
    K_old, V_old = ((b.swapaxes(1, 2) if heads_first else b) for b in before)
    for now, old in ((K_now, K_old), (V_now, V_old)):                        # every other token, the padding, the free pages
        assert np.array_equal(now[~touched], old[~touched], equal_nan=True)
        assert np.array_equal(now[..., d:], old[..., d:], equal_nan=True)
    assert ctx.poll_status() == 0


@gpu
def test_rows_that_cannot_be_placed_are_skipped_and_reported(ctx):
    rng = np.random.default_rng(1)
    c = Cache(rng, "f32", 2, 64, 8, [20, 16, 0], 24)
    x = torch.from_numpy(rng.standard_normal((6, 6, 64))).cuda().float()
    old = [p.clone() for p in c.pool]

    def call(start, pos, rows=6, cache=None):
        Qo = torch.full((6, 2, 64), 7.0, device="cuda")
        fb.focus_append_kv_paged(ctx, c.shape(2), None, x[:, :2], x[:, 2:4], x[:, 4:], x.stride(0), x.stride(1),
                                 i32(start), None if pos is None else i32(pos), rows, cache or c.c(), Qo)
        return Qo, ctx.poll_status()

    Qo, st = call([0, 2, 4, 6], [-1, 24, 16, 15, 0, 1])                      # out of range; no page (sequences 1 and 2)
    assert st == fb.ERR_INVALID_ARG
    assert (Qo[[0, 1, 2, 4, 5]] == 7.0).all() and torch.equal(Qo[3], x[3, :2])
    c.first(old[0])[c.table[1, 1], 7], c.first(old[1])[c.table[1, 1], 7] = x[3, 2:4], x[3, 4:]
    for now, was in zip(c.pool, old):
        assert torch.equal(torch.nan_to_num(now, 9.0), torch.nan_to_num(was, 9.0))
    Qo, st = call([0, 0, 0, 6], None)                                        # six last rows of a sequence without tokens
    assert st == fb.ERR_INVALID_ARG and (Qo == 7.0).all()
    bad = c.c()
    bad.n_pages = int(c.table[0, 0])                                         # pages from there on do not exist
    Qo, st = call([0, 1, 1, 1], [3], cache=bad)
    assert st == fb.ERR_INVALID_ARG and (Qo == 7.0).all()
    for now, was in zip(c.pool, old):
        assert torch.equal(torch.nan_to_num(now, 9.0), torch.nan_to_num(was, 9.0))
    Qo, st = call([2, 2, 4, 4], [0, 1, 2, 3, 0, 0])                          # rows ahead of and behind the sequences: no one's
    assert st == 0 and (Qo[[0, 1, 4, 5]] == 7.0).all() and torch.equal(Qo[2:4], x[2:4, :2])


def attend_case(ctx, dtype, H, Hkv, d, page, lengths, rows, L=None, heads_first=False, scale=0.0, spare=0, gain=1.0, lse=True, seed=0):
    rng = np.random.default_rng(seed + H * d + page + sum(lengths))
    c = Cache(rng, dtype, Hkv, d, page, lengths, L or max(max(lengths), 1), heads_first, pad=8)
    n = rows or [1] * len(lengths)
    start, total = starts(n), sum(n)
    Q = (torch.from_numpy(rng.standard_normal((total + spare, H + 1, d + 8))) * gain).cuda().to(REAL[dtype])
    O = torch.full((total + spare, H, d), 7.0, device="cuda").to(REAL[dtype])
    ls = torch.full((H, total + spare), 7.0, device="cuda") if lse else None
    shape = c.shape(H, q_stride_row=Q.stride(0), q_stride_head=Q.stride(1), softmax_scale=scale)
    fb.focus_paged_attn(ctx, shape, Q, i32(start) if rows else None, total + spare, c.c(), O, ls)
    check_attention(c, n, Q, O, ls, H, scale or 1.0 / math.sqrt(d))
    assert (f64(O)[total:] == 7.0).all() and (ls is None or (f64(ls)[:, total:] == 7.0).all())
    return c, Q, O, ls


def check_attention(c, n, Q, O, ls, H, scale):
    d, start = c.d, starts(n)
    q, got = f64(Q)[:, :H, :d], f64(O)
    for s, t in enumerate(c.lengths):
        keys, values = c.tokens[s]
        rows = slice(start[s], start[s] + n[s])
        if n[s] == 0:
            continue
        want, wl = fo.paged_attn(q[rows], keys, values, scale)
        if t == 0:
            assert (got[rows] == 0).all() and (ls is None or np.isneginf(f64(ls)[:, rows]).all())
            continue
        spread, _ = fo.paged_attn(q[rows], keys, np.abs(values), scale)
        size = np.repeat(np.abs(keys), H // c.Hkv, axis=1)                   # [t, H, d]
        logit = np.einsum("rhd,thd->rht", np.abs(q[rows]), size).max(-1) * abs(scale)
        delta = logit * d * 2.0 ** -24 + 2.0 ** -20                          # [rows, H]
        stacked = -(-Q.shape[0] * (H // c.Hkv) // len(c.lengths))
        held = t * 2.0 ** -24 + (0 if c.dtype == "f32" else 2.0 ** -16 if stacked <= 16 else HALF["bf16"])
        num = delta * 2 + held
        assert (np.abs(got[rows] - want) <= num[..., None] * spread + HALF[c.dtype] * np.abs(want) + 1e-30).all(), s
        if ls is not None:
            assert (np.abs(f64(ls)[:, rows] - wl) <= delta.T * 2 + np.abs(wl) * 2.0 ** -22 + t * 2.0 ** -24).all(), s


@gpu
@pytest.mark.parametrize("dtype,H,Hkv,d,page,lengths,rows,heads_first", [
    ("bf16", 4, 2, 64, 16, [1], None, False),
    ("bf16", 28, 4, 128, 16, [0, 1, 15, 16, 17, 63, 64, 65, 300], None, False),
    ("bf16", 8, 8, 128, 1, [5, 700, 33], None, True),
    ("bf16", 32, 2, 128, 48, [100, 0, 2047], None, False),                   # 16 stacked rows
    ("bf16", 40, 1, 64, 7, [129, 1000], None, True),                         # 40: two row tiles
    ("bf16", 6, 1, 64, 256, [4100, 3], None, False),
    ("bf16", 28, 4, 128, 64, [500, 40, 0, 7], [35, 1, 3, 0], False),         # windows, rows without keys, keys without rows
    ("bf16", 5, 5, 64, 16, [333, 20], [64, 2], True),
    ("bf16", 3, 1, 128, 8, [90, 0, 12], [0, 0, 1], False),
    ("bf16", 28, 4, 128, 16, [900, 2000, 64, 63, 0, 1], [19, 37, 9, 5, 20, 18], False),      # 133, 259, 63, 35, 140, 126 stacked rows
    ("bf16", 6, 2, 64, 48, [3000, 129, 700], [128, 11, 85], True),            # 384, 33, 255
    ("bf16", 4, 4, 128, 5, [1, 64, 65, 250], [300, 96, 32, 1], False),
    ("bf16", 4, 1, 128, 8, [128, 127, 129, 1000], [9, 12, 33, 10], True),
    ("bf16", 14, 2, 64, 128, [1, 256, 383, 5], [5, 7, 64, 0], False),
    ("bf16", 40, 1, 128, 256, [700, 0, 2305], [1, 1, 1], True),
    ("bf16", 5, 1, 64, 32, [31, 32, 33, 4096], [40, 7, 8, 26], False),
    ("f32", 8, 8, 64, 32, [1024, 1, 37, 0, 500], None, False),
    ("f32", 12, 4, 128, 3, [200, 17, 0], [4, 9, 1], True),
    ("f32", 40, 1, 128, 16, [77, 2500], None, False),
    ("f32", 2, 1, 64, 128, [3000], [11], True)])
def test_attention_over_pages_against_the_oracle(ctx, dtype, H, Hkv, d, page, lengths, rows, heads_first):
    attend_case(ctx, dtype, H, Hkv, d, page, lengths, rows, heads_first=heads_first, spare=4 if rows else 0)
    assert ctx.last_attn_variant() in ((6, 8) if dtype == "bf16" else (7,)) and ctx.poll_status() == 0


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_long_sequences_are_split_and_joined(ctx, dtype):
    """One sequence over every CTA (joined in two levels), a few, and many sequences with cuts inside them; sharp logits,
    whose weight lies in one piece."""
    for lengths, H, Hkv, gain in (([20011], 2, 1, 1.0), ([9000, 5, 7001], 8, 2, 6.0), ([700] * 90, 4, 2, 1.0)):
        attend_case(ctx, dtype, H, Hkv, 128, 64, lengths, None, gain=gain)
        attend_case(ctx, dtype, H, Hkv, 64, 16, lengths, None, gain=gain, lse=False)
    attend_case(ctx, dtype, 8, 1, 128, 32, [9000, 300], [14, 3])
    attend_case(ctx, dtype, 4, 1, 64, 64, [15000], [10], gain=6.0)
    assert ctx.poll_status() == 0


@gpu
def test_scales_strides_and_bounds(ctx):
    attend_case(ctx, "bf16", 4, 2, 128, 16, [100, 30], None, scale=0.5)
    attend_case(ctx, "bf16", 4, 2, 64, 16, [100, 30], None, scale=-0.25)
    attend_case(ctx, "f32", 4, 2, 64, 16, [100, 30], None, L=5000)
    attend_case(ctx, "bf16", 4, 4, 64, 16, [100] * 300, None)
    attend_case(ctx, "bf16", 4, 4, 64, 16, [3] * 1000, [i % 3 for i in range(1000)])
    assert ctx.poll_status() == 0


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_bad_pages_lengths_and_rows_are_reported_not_followed(ctx, dtype):
    rng = np.random.default_rng(5)
    c = Cache(rng, dtype, 2, 64, 16, [100, 50], 112)
    Q = torch.from_numpy(rng.standard_normal((2, 4, 64))).cuda().to(REAL[dtype])

    def call(start=None, rows=2, shape=None):
        O, ls = torch.full((2, 4, 64), 7.0, device="cuda").to(REAL[dtype]), torch.full((4, 2), 7.0, device="cuda")
        fb.focus_paged_attn(ctx, shape or c.shape(4), Q, start, rows, c.c(), O, ls)
        return O, ls, ctx.poll_status()

    good, _, st = call()
    assert st == 0
    c.d_table[0, 2], c.d_table[0, 4] = -1, c.n_pages                         # keys 32..47 and 64..79 are not attended
    O, ls, st = call()
    assert st == fb.ERR_INVALID_ARG and torch.equal(O[1], good[1])
    keep = np.r_[0:32, 48:64, 80:100]
    c.tokens[0], c.lengths = [t[keep] for t in c.tokens[0]], [len(keep), 50]
    check_attention(c, [1, 1], Q, O, ls, 4, 0.125)
    c.d_table[0, :] = -5                                                     # no page at all: as without keys
    O, ls, st = call()
    assert st == fb.ERR_INVALID_ARG and (O[0] == 0).all() and torch.isinf(ls[:, 0]).all() and torch.equal(O[1], good[1])
    c.d_len[0] = -3
    O, ls, st = call()
    assert st == fb.ERR_INVALID_ARG and (O[0] == 0).all() and torch.equal(O[1], good[1])
    c.d_len[0] = 10 ** 9                                                     # counts as L: the table is not read beyond it
    O, ls, st = call()
    assert st == fb.ERR_INVALID_ARG and (O[0] == 0).all() and torch.equal(O[1], good[1])
    c.d_len[0] = 0
    for start in ([0, 3, 3], [0, -1, 2], [1, 0, 2], [-1, 1, 2]):
        O, ls, st = call(start=i32(start))
        assert st == fb.ERR_INVALID_ARG


@gpu
@pytest.mark.parametrize("page", [16, 24])
def test_windows_skip_pages_that_do_not_exist(ctx, page):
    rng = np.random.default_rng(page)
    c = Cache(rng, "bf16", 2, 128, page, [600, 290], 600)
    n = [12, 9]
    Q = torch.from_numpy(rng.standard_normal((21, 8, 128))).cuda().bfloat16()
    start = i32([0, 12, 21])

    def call():
        O, ls = torch.zeros((21, 8, 128), device="cuda").bfloat16(), torch.zeros((8, 21), device="cuda")
        fb.focus_paged_attn(ctx, c.shape(8), Q, start, 21, c.c(), O, ls)
        return O, ls, ctx.poll_status()

    good, _, st = call()
    assert st == 0 and ctx.last_attn_variant() == 8
    c.d_table[0, 3], c.d_table[0, 8:20], c.d_table[0, 24] = -1, c.n_pages, 2 ** 31 - 1
    O, ls, st = call()
    assert st == fb.ERR_INVALID_ARG and torch.equal(O[12:], good[12:])
    keep = np.array([j for j in range(600) if not (j // page in (3, 24) or 8 <= j // page < 20)])
    c.tokens[0], c.lengths = [t[keep] for t in c.tokens[0]], [len(keep), 290]
    check_attention(c, n, Q, O, ls, 8, 128 ** -0.5)
    c.d_table[0, :] = -1
    O, ls, st = call()
    assert st == fb.ERR_INVALID_ARG and (O[:12] == 0).all() and torch.isinf(ls[:, :12]).all() and torch.equal(O[12:], good[12:])


@gpu
def test_infinities_and_nan_stay_in_their_rows(ctx):
    rng = np.random.default_rng(9)
    c = Cache(rng, "bf16", 1, 64, 16, [50, 60, 70], 80)
    Q = torch.from_numpy(rng.standard_normal((3, 2, 64))).cuda().bfloat16()
    Q[1, 0, 3] = float("inf")
    Q[2, 1, 0] = float("nan")
    O, ls = torch.zeros((3, 2, 64), device="cuda").bfloat16(), torch.zeros((2, 3), device="cuda")
    fb.focus_paged_attn(ctx, c.shape(2), Q, None, 3, c.c(), O, ls)
    assert torch.isnan(O[1, 0].float()).all() and torch.isnan(O[2, 1].float()).all()
    for r, h in ((0, 0), (0, 1), (1, 1), (2, 0)):
        want, _ = fo.paged_attn(f64(Q)[r:r + 1, h:h + 1], *c.tokens[r], 0.125)
        assert np.abs(f64(O)[r, h] - want[0, 0]).max() < 0.02
    assert ctx.poll_status() == 0


@gpu
def test_results_do_not_depend_on_timing_and_replay_in_graphs(ctx):
    """Two captured calls share the context's workspace and counters; replays give the eager call's bits."""
    rng = np.random.default_rng(11)
    jobs = []
    for lengths, H in (([9000, 300, 12], 28), ([40] * 70, 8)):
        c = Cache(rng, "bf16", 4, 128, 16, lengths, max(lengths))
        n = len(lengths)
        Q = torch.from_numpy(rng.standard_normal((n, H, 128))).cuda().bfloat16()
        jobs.append((c, c.shape(H), Q, n, torch.zeros((n, H, 128), device="cuda").bfloat16(), torch.zeros((H, n), device="cuda")))

    def run(j):
        c, sh, Q, n, O, ls = jobs[j]
        fb.focus_paged_attn(ctx, sh, Q, None, n, c.c(), O, ls)

    want = []
    for j in range(2):
        run(j)
        want.append((jobs[j][4].clone(), jobs[j][5].clone()))
    graphs = []
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for j in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            run(j)
        graphs.append(g)
    for _ in range(20):
        for j in (0, 1, 1, 0):
            jobs[j][4].zero_(), jobs[j][5].zero_()
            graphs[j].replay()
            assert torch.equal(jobs[j][4], want[j][0]) and torch.equal(jobs[j][5], want[j][1])
    assert ctx.poll_status() == 0


@gpu
def test_offsets_beyond_32_bits(ctx):
    """Pages that lie more than 2^31 elements into the pools."""
    n_pages, page, Hkv, d = 2 ** 21 + 40, 16, 1, 64                          # 2^31 elements and 40 pages more: 4.3 GB each
    K, V = (torch.zeros((n_pages, page, Hkv, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    rng = np.random.default_rng(2)
    table, kv_len = i32([[n_pages - 1, 3, n_pages - 7]]), i32([48])           # the cache holds their addresses alone
    x = torch.from_numpy(rng.standard_normal((48, 4, d))).cuda().bfloat16()
    sh = fb.make_shape(48, 0, 2, 1, d, 64, fb.BF16)
    cache = fb.make_paged_cache(K, V, table, kv_len, page, n_pages, 1, 3, K.stride(0), K.stride(1), K.stride(2))
    fb.focus_append_kv_paged(ctx, sh, None, None, x[:, 2:3], x[:, 3:], x.stride(0), x.stride(1), i32([0, 48]), None, 48, cache, None)
    assert torch.equal(K[n_pages - 1, :, 0], x[:16, 2]) and torch.equal(V[n_pages - 7, :, 0], x[32:, 3])
    O = torch.zeros((1, 2, d), dtype=torch.bfloat16, device="cuda")
    fb.focus_paged_attn(ctx, sh, x, None, 1, cache, O)
    want, _ = fo.paged_attn(f64(x[:1, :2]), f64(x[:, 2:3]), f64(x[:, 3:]), 0.125)
    assert np.abs(f64(O) - want).max() <= 2.0 ** -6
    assert ctx.poll_status() == 0


@gpu
def test_workspace_bound(ctx):
    sh = fb.make_shape(64, 0, 32, 1, 128, 64, fb.BF16)
    need = fb.focus_paged_attn_workspace_bytes(ctx, sh)
    rng = np.random.default_rng(4)
    c = Cache(rng, "bf16", 1, 128, 16, [64], 64)
    Q = torch.from_numpy(rng.standard_normal((1, 32, 128))).cuda().bfloat16()
    O = torch.zeros_like(Q)
    tight, small = fb.Context(0, need), fb.Context(0, 4096)
    fb.focus_paged_attn(tight, c.shape(32), Q, None, 1, c.c(), O)
    assert tight.poll_status() == 0 and O.abs().max().item() > 0
    with pytest.raises(fb.FocusError) as e:
        fb.focus_paged_attn(small, c.shape(32), Q, None, 1, c.c(), O)
    assert e.value.code == fb.ERR_WORKSPACE_TOO_SMALL
    tight.close()
    small.close()
