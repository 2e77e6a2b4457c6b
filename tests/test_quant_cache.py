"""The 8-bit K/V cache: rows written (focus_quantize_kv), read back (focus_dequantize_kv) and attended
(focus_dense_attn_quantized, focus_sparse_attn_quantized), against the float64 oracle."""
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
FMT = {"int8": fb.KV_INT8, "e4m3": fb.KV_E4M3}
DT = {"bf16": fb.BF16, "f32": fb.F32}


@pytest.fixture(scope="module")
def ctx():
    c = fb.Context(0)
    yield c
    assert c.poll_status() == 0
    c.close()


def codes_to_device(values, fmt):
    t = torch.from_numpy(np.ascontiguousarray(values)).to(torch.float32).cuda()
    return t.to(torch.int8) if fmt == "int8" else t.to(torch.float8_e4m3fn)


def code_values(t):
    return t.float().double().cpu().numpy()


def storage(x, dtype):
    return wl.to_storage(np.ascontiguousarray(x.astype(np.float32)), dtype)


# ---- refusals: arguments are checked on the host before anything is launched -------------------------------------
@pytest.fixture(scope="module")
def lib():
    fbuild.build()
    return fb.load_library()


def _fake_ctx():
    return ctypes.create_string_buffer(4096)           # read by no call that is refused


def test_refusals_need_no_device(lib):
    fake = _fake_ctx()
    P, h = 1 << 20, ctypes.cast(fake, ctypes.c_void_p)           # any 16-byte aligned address
    sh = fb.make_shape(256, 192, 4, 2, 64, 64, fb.BF16)
    cache = fb.make_quant_cache(fb.KV_INT8, P, P, P, P)
    B = ctypes.byref

    def quant(ctx=h, shape=sh, K=P, V=P, srow=256, shead=64, base=0, rows=None, n=None, max_rows=8, c=cache):
        return lib.focus_quantize_kv(ctx, B(shape), K, V, srow, shead, base, rows, n, max_rows, B(c), None)

    def dequant(ctx=h, shape=sh, K=P, V=P, srow=64, shead=64 * 8, base=0, rows=None, n=None, max_rows=8, c=cache):
        return lib.focus_dequantize_kv(ctx, B(shape), B(c), base, rows, n, max_rows, K, V, srow, shead, None)

    def dense(ctx=h, shape=sh, Q=P, q_base=192, n_q=64, rows=None, n=None, max_rows=0, c=cache, O=P):
        return lib.focus_dense_attn_quantized(ctx, B(shape), Q, q_base, n_q, rows, n, max_rows, B(c), O, None, None)

    def sparse(ctx=h, shape=sh, c=cache, mode=0, blocks=P, cnt=P, max_blocks=2, sinks=None, keep=None, n_sink=0):
        return lib.focus_sparse_attn_quantized(ctx, B(shape), P, 192, 64, None, None, 0, B(c), mode, blocks, max_blocks, cnt,
                                               sinks, keep, n_sink, P, None, None)

    for call in (quant, dequant, dense, sparse):
        assert call(ctx=None) == fb.ERR_INVALID_ARG
        assert call(c=fb.make_quant_cache(2, P, P, P, P)) == fb.ERR_INVALID_ARG              # unknown format
        assert call(c=fb.make_quant_cache(fb.KV_E4M3, P + 8, P, P, P)) == fb.ERR_INVALID_ARG   # misaligned codes
        assert call(c=fb.make_quant_cache(fb.KV_E4M3, P, P, P + 2, P)) == fb.ERR_INVALID_ARG   # misaligned scales
        assert call(c=fb.make_quant_cache(fb.KV_E4M3, P, None, P, P)) == fb.ERR_INVALID_ARG
        assert call(c=fb.make_quant_cache(fb.KV_E4M3, P, P, P, P, 255)) == fb.ERR_INVALID_ARG  # scale rows shorter than L
        bad = fb.make_shape(256, 192, 4, 2, 64, 64, fb.BF16, kv_stride_tok=72)               # code rows not 16-byte aligned
        assert call(shape=bad) == fb.ERR_INVALID_ARG
        assert call(shape=fb.make_shape(256, 192, 4, 2, 32, 64, fb.BF16)) == fb.ERR_UNSUPPORTED   # head dim
    for call in (quant, dequant):
        assert call(K=None, V=None) == fb.ERR_INVALID_ARG
        assert call(K=P + 4) == fb.ERR_INVALID_ARG
        assert call(srow=60) == fb.ERR_INVALID_ARG and call(shead=68) == fb.ERR_INVALID_ARG
        assert call(max_rows=-1) == fb.ERR_INVALID_ARG
        assert call(rows=P) == fb.ERR_INVALID_ARG                                            # a list without its count
        assert call(base=250) == fb.ERR_INVALID_ARG and call(base=-1) == fb.ERR_INVALID_ARG
        assert call(base=2 ** 31 - 4) == fb.ERR_INVALID_ARG
        assert call(max_rows=0) == fb.OK                                                     # nothing to do
    assert dense(q_base=200) == fb.ERR_INVALID_ARG and dense(O=None) == fb.ERR_INVALID_ARG
    assert dense(rows=P) == fb.ERR_INVALID_ARG and dense(n_q=0) == fb.OK
    assert sparse(mode=2) == fb.ERR_INVALID_ARG and sparse(blocks=None) == fb.ERR_INVALID_ARG
    assert sparse(n_sink=3) == fb.ERR_INVALID_ARG and sparse(max_blocks=-1) == fb.ERR_INVALID_ARG


# ---- writing ------------------------------------------------------------------------------------------------------
def _rows_with_edges(rng, n, Hkv, d):
    x = rng.standard_normal((n, Hkv, d)) * np.exp(rng.standard_normal((n, Hkv, 1)))
    flat = x.reshape(-1, d)
    edges = [np.zeros(d), np.full(d, 3.0e-25), np.where(np.arange(d) == 5, 1.0, 0.0),        # zero, flushed, one element
             np.linspace(-1.0, 1.0, d), np.full(d, -2.5), np.arange(d) * 0.5 - 7.0]          # both ends, equal, exact halves
    edges[5][0] = 63.5                                    # scale 1/2: quotients are integers and halves of them
    inf, nan = rng.standard_normal(d), rng.standard_normal(d)
    inf[3], inf[9], nan[1], nan[d - 1] = np.inf, -np.inf, np.nan, np.inf
    only = np.full(d, np.nan)
    only[2] = np.inf
    for i, e in enumerate(edges + [inf, nan, only, rng.standard_normal(d) * 1e30, rng.standard_normal(d) * 1e-20]):
        if i < len(flat):
            flat[i] = e
    return x


@gpu
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype,d,Hkv,L,n,listed", [("bf16", 128, 4, 700, 37, True), ("f32", 128, 3, 129, 129, False),
                                                    ("bf16", 64, 2, 50, 33, True), ("f32", 64, 5, 1, 1, False),
                                                    ("bf16", 128, 32, 2100, 1, True), ("bf16", 64, 1, 300, 255, False)])
def test_written_rows_are_the_oracles_bit_for_bit(ctx, fmt, dtype, d, Hkv, L, n, listed):
    rng = np.random.default_rng(d + L + n)
    H, extra = 2 * Hkv, 3
    x = storage(rng.standard_normal((n, H + 2 * Hkv, d)) * 0.0, dtype)
    K, V = (storage(_rows_with_edges(rng, n, Hkv, d), dtype) for _ in range(2))
    x[:, H:H + Hkv], x[:, H + Hkv:] = K, V                                   # rows of a fused projection: Q | K | V
    dx = fstep.to_device(x, dtype)
    dK, dV = dx[:, H:H + Hkv], dx[:, H + Hkv:]
    pad, spad = 16, 5                                                        # token stride d + 16, scale rows L + 5
    old = [torch.randint(-100, 100, (Hkv, L, d + pad), dtype=torch.int8, device="cuda") for _ in range(2)]
    old_s = [torch.rand(Hkv, L + spad, device="cuda") for _ in range(2)]
    codes, scales = [t.clone() for t in old], [t.clone() for t in old_s]
    pos = np.sort(rng.choice(L, size=n, replace=False)) if listed else np.arange(L - n, L)
    rows = torch.from_numpy(np.concatenate([pos, np.full(extra, -1)]).astype(np.int32)).cuda() if listed else None
    n_rows = torch.tensor([n], dtype=torch.int32, device="cuda") if listed else None
    sh = fb.make_shape(L, 0, H, Hkv, d, 64, DT[dtype], kv_stride_tok=d + pad, kv_stride_head=L * (d + pad))
    cache = fb.make_quant_cache(FMT[fmt], codes[0], codes[1], scales[0], scales[1], L + spad)
    fb.focus_quantize_kv(ctx, sh, dK, dV, dK.stride(0), dK.stride(1), L - n, rows, n_rows, n + (extra if listed else 0), cache)
    view = torch.int8 if fmt == "int8" else torch.float8_e4m3fn
    for got, sc, before, before_s, src in ((codes[0], scales[0], old[0], old_s[0], K), (codes[1], scales[1], old[1], old_s[1], V)):
        want, ws = fo.quantize_rows(wl.storage_to_f64(src, dtype), fmt)
        assert np.array_equal(sc[:, pos].cpu().numpy().astype(np.float64), ws.T)
        assert np.array_equal(code_values(got.view(view)[:, :, :d])[:, pos], want.transpose(1, 0, 2))
        rest = np.setdiff1d(np.arange(L), pos)                               # every other row, the padding and the tails stay
        assert torch.equal(got[:, rest], before[:, rest]) and torch.equal(got[:, :, d:], before[:, :, d:])
        assert torch.equal(sc[:, rest], before_s[:, rest]) and torch.equal(sc[:, L:], before_s[:, L:])
    assert ctx.poll_status() == 0


@gpu
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f32", 64), ("f32", 128)])
def test_a_long_cache_bit_for_bit_both_ways(ctx, fmt, dtype, d):
    """Many rows (several in flight per thread), magnitudes over the whole range of fp32, quotients on and beside the
    ties: IEEE division on the host is the reference."""
    Hkv, L = 8, 10007                                     # an odd length: the last group of rows is ragged
    rng = np.random.default_rng(d)
    top = {"int8": 127.0, "e4m3": 448.0}[fmt]
    x = rng.standard_normal((L, Hkv, d)).astype(np.float32)
    x *= np.exp2(rng.integers(-96, 125, (L, Hkv, 1))).astype(np.float32)
    m = np.abs(x[:L // 2]).max(-1, keepdims=True)
    ties = (rng.integers(-2 * top, 2 * top + 1, (L // 2, Hkv, d)) / np.float32(2.0 * top)).astype(np.float32) * m
    x[:L // 2] = np.where(rng.random(ties.shape) < 0.5, ties, x[:L // 2])
    x[5, 0, :] = np.float32(3.3e38)                       # the largest scale
    x[6, 0, 1], x[7, 1, 2], x[L - 1, 7, d - 1] = np.inf, np.nan, -np.inf
    src = storage(x, dtype)
    x = wl.storage_to_f64(src, dtype).astype(np.float32)
    fin = np.where(np.isfinite(x), np.abs(x), np.float32(0)).max(-1)
    scale = np.where(fin < np.float32(2.0 ** -80), np.float32(0), fin / np.float32(top)).astype(np.float32)
    with np.errstate(all="ignore"):
        q = np.where(np.isnan(x) | (scale[..., None] == 0), np.float32(0), x / scale[..., None])
    q = torch.from_numpy(np.clip(q, -top, top))
    want = q.round().to(torch.int8) if fmt == "int8" else q.to(torch.float8_e4m3fn)          # both: ties to even
    dx = fstep.to_device(src, dtype)
    sh = fb.make_shape(L, 0, Hkv, Hkv, d, 64, DT[dtype])
    codes = torch.zeros(2, Hkv, L, d, dtype=want.dtype, device="cuda")
    scales = torch.full((2, Hkv, L), -1.0, device="cuda")
    cache = fb.make_quant_cache(FMT[fmt], codes[0], codes[1], scales[0], scales[1])
    for i in (0, 1):
        fb.focus_quantize_kv(ctx, sh, None if i else dx, dx if i else None, Hkv * d, d, 0, None, None, L, cache)
        assert np.array_equal(scales[i].cpu().numpy(), scale.T)
        assert torch.equal(codes[i].float().cpu(), want.float().transpose(0, 1))
    out = torch.zeros(2, Hkv, L, d, dtype=dx.dtype, device="cuda")
    fb.focus_dequantize_kv(ctx, sh, cache, 0, None, None, L, out[0], out[1], d, L * d)
    ref = (want.float() * torch.from_numpy(scale)[..., None]).transpose(0, 1).to(dx.dtype)   # one rounding (+ bf16's)
    assert torch.equal(out[0].cpu(), ref) and torch.equal(out[1].cpu(), ref)
    assert ctx.poll_status() == 0


@gpu
def test_one_half_of_the_cache_at_a_time_and_no_rows(ctx):
    L, Hkv, d, n = 40, 2, 64, 6
    sh = fb.make_shape(L, 0, 2, Hkv, d, 64, fb.BF16)
    x = torch.randn(n, Hkv, d, device="cuda").bfloat16()
    K, V = (torch.full((Hkv, L, d), 7, dtype=torch.int8, device="cuda") for _ in range(2))
    ks, vs = (torch.full((Hkv, L), 9.0, device="cuda") for _ in range(2))
    rows = torch.arange(3, 3 + n, dtype=torch.int32, device="cuda")
    count = torch.zeros(1, dtype=torch.int32, device="cuda")
    cache = fb.make_quant_cache(fb.KV_INT8, K, V, ks, vs)
    fb.focus_quantize_kv(ctx, sh, x, x, Hkv * d, d, 0, rows, count, n, cache)                 # a count of zero
    assert (K == 7).all() and (V == 7).all() and (ks == 9).all()
    only_v = fb.make_quant_cache(fb.KV_INT8, None, V, None, vs)
    fb.focus_quantize_kv(ctx, sh, None, x, Hkv * d, d, 5, None, None, n, only_v)
    assert (K == 7).all() and (V[:, 5:5 + n] != 7).any() and (V[:, :5] == 7).all() and (V[:, 5 + n:] == 7).all()
    out = torch.full((n, Hkv, d), 5.0, device="cuda").bfloat16()
    fb.focus_dequantize_kv(ctx, sh, only_v, 5, None, None, n, None, out, Hkv * d, d)
    scale = x.float().abs().amax(-1, keepdim=True) / 127
    # half a step of the scale, and one rounding to bf16
    assert ((out.float() - x.float()).abs() <= scale * 0.5 * (1 + 1e-5) + x.float().abs() * 2.0 ** -8 + scale * 2.0 ** -9).all()
    assert ctx.poll_status() == 0


@gpu
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_bad_positions_are_skipped_and_reported(ctx, fmt):
    """Out of range, listed twice, or out of order: the row is left out and INVALID_ARG is recorded; nothing else moves."""
    L, Hkv, d = 64, 2, 128
    sh = fb.make_shape(L, 0, 2, Hkv, d, 64, fb.F32)
    x = torch.randn(6, Hkv, d, device="cuda")
    for listing, written in (([2, 9, 9, 12, L, 70], {2: 0, 9: 1, 12: 3}), ([-3, 4, 5, 6, 7, 8], {4: 1, 5: 2, 6: 3, 7: 4, 8: 5}),
                             ([1, 30, 20, 31, 32, 33], {1: 0, 30: 1, 31: 3, 32: 4, 33: 5})):
        codes = torch.full((Hkv, L, d), 3, dtype=torch.int8, device="cuda")
        scales = torch.full((Hkv, L), -1.0, device="cuda")
        rows = torch.tensor(listing, dtype=torch.int32, device="cuda")
        n_rows = torch.tensor([6], dtype=torch.int32, device="cuda")
        fb.focus_quantize_kv(ctx, sh, x, None, Hkv * d, d, 0, rows, n_rows, 6, fb.make_quant_cache(FMT[fmt], codes, None, scales, None))
        assert ctx.poll_status() == fb.ERR_INVALID_ARG
        for p in range(L):
            if p in written:
                assert torch.equal(scales[:, p], x[written[p]].abs().amax(-1) / torch.full((Hkv,), 127.0 if fmt == "int8" else 448.0, device="cuda"))
            else:
                assert (scales[:, p] == -1).all() and (codes[:, p] == 3).all()
    # reading: any order, repeats allowed, bad positions leave their output row alone
    good = fb.make_quant_cache(FMT[fmt], codes, None, scales, None)
    out = torch.full((4, Hkv, d), 55.0, device="cuda")
    rows = torch.tensor([33, 1, 33, L], dtype=torch.int32, device="cuda")
    n_rows = torch.tensor([4], dtype=torch.int32, device="cuda")
    fb.focus_dequantize_kv(ctx, sh, good, 0, rows, n_rows, 4, out, None, Hkv * d, d)
    assert ctx.poll_status() == fb.ERR_INVALID_ARG
    assert torch.equal(out[0], out[2]) and (out[3] == 55).all() and not torch.equal(out[0], out[1])


@gpu
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f32", 128), ("bf16", 64), ("f32", 64)])
def test_rows_read_back(ctx, fmt, dtype, d):
    """Every code the format has, several scales; the result is the oracle's product, rounded once."""
    Hkv, L = 2, 41
    rng = np.random.default_rng(d)
    if fmt == "int8":
        vals = rng.integers(-127, 128, size=(Hkv, L, d)).astype(np.float64)
    else:
        bits = rng.integers(0, 256, size=(Hkv, L, d)).astype(np.uint8)
        bits[(bits & 0x7f) == 0x7f] = 0x40                                                   # no NaN
        vals = torch.from_numpy(bits).view(torch.float8_e4m3fn).float().double().numpy()
    sc = np.exp2(rng.integers(-30, 20, size=(Hkv, L)).astype(np.float64)) * rng.integers(1, 2 ** 20, size=(Hkv, L)) / 2.0 ** 20
    sc[0, 3] = 0.0
    codes, scales = codes_to_device(vals, fmt), torch.from_numpy(sc).float().cuda()
    sh = fb.make_shape(L, 0, 2, Hkv, d, 64, DT[dtype])
    out = torch.full((Hkv, L, d + 8), 3.0, dtype=fstep.torch_dtype(dtype), device="cuda")
    fb.focus_dequantize_kv(ctx, sh, fb.make_quant_cache(FMT[fmt], codes, codes, scales, scales), 0, None, None, L, out, None,
                           d + 8, L * (d + 8))
    want = torch.from_numpy(vals * sc[..., None]).float().to(fstep.torch_dtype(dtype))       # the product fits 24 + 8 bits ...
    exact = torch.from_numpy(vals * sc[..., None])
    got = out[:, :, :d].double().cpu()
    # ... so fp32 rounds it once and bf16 a second time: within half a step of each
    tol = exact.abs() * (2.0 ** -24 if dtype == "f32" else 2.0 ** -8 + 2.0 ** -24)
    assert ((got - exact).abs() <= tol).all() and (out[:, :, d:] == 3).all()
    assert torch.equal(got, want.double())
    assert ctx.poll_status() == 0


# ---- attention ----------------------------------------------------------------------------------------------------
def _attention_case(rng, dtype, fmt, H, Hkv, d, L, N, spread=1.0):
    Q = storage(rng.standard_normal((N, H, d)) * spread, dtype)
    out = []
    for _ in range(2):
        x = rng.standard_normal((Hkv, L, d)) * np.exp(0.7 * rng.standard_normal((Hkv, L, 1)))
        out.append(fo.quantize_rows(x, fmt))
    return Q, out[0], out[1]


def _bounds(Q, K, V, vs, O, scale, hpg, dtype, keys=None):
    """Elementwise bounds of O and lse, from the roundings on the way.

    Logits: d products summed in fp32 are off by at most E = (d + 4) 2^-24 sum|q k| scale (one step per addition); the
    tensor-core path also carries q in fp16 relative to its row's largest element, subnormal below 2^-14 of it, which
    adds 2^-24 max|q| sum|k|.  Every numerator is then off by a factor 1 + E + 2^-21 (exp2), the ones that meet V by
    another 2^-11 (fp16), sums over the n keys by n 2^-24, and the output is rounded once (bf16: 2^-8).

    fp16 also has a smallest step.  A numerator that meets V is p_j sv_j in units that put the row's largest at 2^2 or
    more, and fp16 numbers below 2^-14 are 2^-24 apart: off by at most 2^-25, i.e. 2^-27 of the row's largest p_j sv_j.
    The codes weigh those errors, so a channel is off by at most 2^-27 max_j(p_j sv_j) sum_j |cv_j| more (it shows where
    the token that holds nearly all the weight has code 0 in that channel)."""
    n, H, d = Q.shape
    tolO, tolL = np.zeros_like(O), np.zeros((H, n))
    for h in range(H):
        g = h // hpg
        Kg, Vg = (K[g], V[g]) if keys is None else (K[g][keys[g]], V[g][keys[g]])
        if len(Kg) == 0:
            continue
        s = Q[:, h] @ Kg.T * scale
        mag = np.abs(Q[:, h]) @ np.abs(Kg).T * scale
        E = ((d + 4) * 2.0 ** -24 * mag).max(1) + np.abs(Q[:, h]).max(1) * np.abs(Kg).sum(1).max() * scale * 2.0 ** -24
        p = np.exp(s - s.max(1, keepdims=True))
        p /= p.sum(1, keepdims=True)
        A = p @ np.abs(Vg)
        num = E + 2.0 ** -21 + len(Kg) * 2.0 ** -24
        per = num * 2 + (2.0 ** -11 if dtype == "bf16" else 0.0)
        sv = vs[g] if keys is None else vs[g][keys[g]]
        codes = np.abs(np.divide(Vg, sv[:, None], out=np.zeros_like(Vg), where=sv[:, None] > 0)).sum(0)
        step = 2.0 ** -27 * (p * sv).max(1)[:, None] * codes if dtype == "bf16" else 0.0
        tolO[:, h] = step + per[:, None] * A + (2.0 ** -8 if dtype == "bf16" else 2.0 ** -23) * np.abs(O[:, h]) + 1e-30
        tolL[h] = num + 2.0 ** -22 * (1 + np.abs(np.log(np.exp(s - s.max(1, keepdims=True)).sum(1)) + s.max(1)))
    return tolO, tolL


DENSE = [  # dtype, H, Hkv, d, L, N, listed rows, capacity
    ("bf16", 4, 4, 128, 640, 40, 37, 48), ("bf16", 8, 2, 128, 1000, 70, 70, 0), ("bf16", 4, 4, 64, 517, 33, 20, 25),
    ("bf16", 7, 1, 128, 130, 3, 3, 0), ("bf16", 2, 2, 128, 1, 1, 1, 0), ("bf16", 2, 1, 64, 127, 1, 1, 5),
    ("bf16", 2, 2, 128, 4100, 130, 129, 130), ("bf16", 1, 1, 64, 129, 129, 129, 0), ("bf16", 12, 4, 128, 2049, 90, 85, 90),
    ("f32", 4, 2, 64, 300, 30, 19, 24), ("f32", 2, 2, 128, 257, 9, 9, 0), ("f32", 8, 8, 64, 64, 1, 1, 0)]


@gpu
@pytest.mark.parametrize("simt", [False, True])
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype,H,Hkv,d,L,N,n,cap", DENSE)
def test_dense_attention_over_an_8bit_cache(ctx, simt, fmt, dtype, H, Hkv, d, L, N, n, cap):
    rng = np.random.default_rng(H * 1000 + L + N)
    Q, (kc, ks), (vc, vs) = _attention_case(rng, dtype, fmt, H, Hkv, d, L, N)
    K, V = kc * ks[..., None], vc * vs[..., None]
    q_base = L - N
    pos = np.sort(rng.choice(N, size=n, replace=False)) + q_base if cap else np.arange(q_base, L)
    rows = torch.from_numpy(np.concatenate([pos, np.full(cap - n, -1)]).astype(np.int32)).cuda() if cap else None
    n_rows = torch.tensor([n], dtype=torch.int32, device="cuda") if cap else None
    bound = cap or N
    # queries strided over a wider row, codes with a padded token stride
    qpad = torch.zeros(N, H + 1, d + 8, dtype=fstep.torch_dtype(dtype), device="cuda")
    qpad[:, :H, :d] = fstep.to_device(Q, dtype)
    wide = [torch.full((Hkv, L, d + 16), 77, dtype=torch.int8, device="cuda") for _ in range(2)]
    for w, c in zip(wide, (kc, vc)):
        w[:, :, :d] = codes_to_device(c, fmt).view(torch.int8)
    sc = [torch.from_numpy(s).float().cuda().contiguous() for s in (ks, vs)]
    sh = fb.make_shape(L, L, H, Hkv, d, 64, DT[dtype], q_stride_row=(H + 1) * (d + 8), q_stride_head=d + 8,
                       kv_stride_tok=d + 16, kv_stride_head=L * (d + 16))
    O = torch.full((bound, H, d), 9.0, dtype=fstep.torch_dtype(dtype), device="cuda")
    lse = torch.full((H, bound), 9.0, device="cuda")
    ctx.set_force_simt(simt)
    try:
        fb.focus_dense_attn_quantized(ctx, sh, qpad, q_base, N, rows, n_rows, cap, fb.make_quant_cache(FMT[fmt], *wide, *sc), O, lse)
    finally:
        ctx.set_force_simt(False)
    Qf = wl.storage_to_f64(Q, dtype)[pos - q_base]
    eO, eL = fo.dense_attn(Qf, K, V, 1.0 / math.sqrt(d))
    tO, tL = _bounds(Qf, K, V, vs, eO, 1.0 / math.sqrt(d), H // Hkv, dtype)
    assert (np.abs(fstep.from_device(O)[:n] - eO) <= tO).all()
    assert (np.abs(fstep.from_device(lse)[:, :n] - eL) <= tL).all()
    assert (O[n:] == 9).all() and (lse[:, n:] == 9).all()
    assert ctx.poll_status() == 0


SPARSE = [  # dtype, H, Hkv, d, L, M, B, keep, sinks, N, n, cap, heads_all
    ("bf16", 4, 4, 128, 2000, 1800, 128, 5, 20, 100, 37, 48, False), ("bf16", 8, 2, 128, 1500, 1430, 64, 7, 3, 70, 70, 0, False),
    ("bf16", 4, 2, 64, 900, 801, 64, 4, 130, 99, 5, 5, True), ("bf16", 2, 2, 128, 700, 640, 128, 5, 0, 60, 60, 0, False),
    ("bf16", 2, 1, 128, 400, 399, 128, 0, 6, 1, 1, 0, False), ("bf16", 3, 3, 64, 300, 300, 64, 1, 0, 20, 9, 12, False),
    ("bf16", 2, 2, 128, 5000, 4600, 64, 72, 46, 150, 140, 140, False),
    ("f32", 4, 2, 64, 700, 600, 64, 3, 17, 40, 33, 40, False), ("f32", 2, 2, 128, 500, 450, 128, 2, 5, 50, 50, 0, True)]


def _run_sparse(ctx, case, fmt, simt, rng, mutate=None):
    dtype, H, Hkv, d, L, M, B, keep, sinks, N, n, cap, all_heads = case
    Q, (kc, ks), (vc, vs) = _attention_case(rng, dtype, fmt, H, Hkv, d, L, N)
    nb, G = (M + B - 1) // B, 1 if all_heads else Hkv
    blocks = [np.sort(rng.choice(nb, size=keep, replace=False)) for _ in range(G)]
    sink = np.sort(rng.choice(M, size=sinks, replace=False))
    max_blocks = keep + 2
    bi = np.full((G, max_blocks), -1, dtype=np.int32)
    for g in range(G):
        bi[g, :keep] = blocks[g]
    sk = np.array([[0 if (s // B) in set(blocks[g]) else 1 for s in sink] for g in range(G)], dtype=np.uint8).reshape(G, sinks)
    if mutate:
        mutate(kc, ks, vc, vs, blocks, sink, sk)
    q_base = L - N
    pos = np.sort(rng.choice(N, size=n, replace=False)) + q_base if cap else np.arange(q_base, L)
    rows = torch.from_numpy(np.concatenate([pos, np.full(cap - n, -1)]).astype(np.int32)).cuda() if cap else None
    n_rows = torch.tensor([n], dtype=torch.int32, device="cuda") if cap else None
    bound = cap or N
    dQ = fstep.to_device(Q, dtype)
    sh = fb.make_shape(L, M, H, Hkv, d, B, DT[dtype])
    O = torch.full((bound, H, d), 9.0, dtype=fstep.torch_dtype(dtype), device="cuda")
    lse = torch.full((H, bound), 9.0, device="cuda")
    dev = [torch.from_numpy(a).cuda() for a in (bi, np.full(G, keep, dtype=np.int32), sink.astype(np.int32), sk)]
    code = [codes_to_device(c, fmt) for c in (kc, vc)]
    scl = [torch.from_numpy(s).float().cuda().contiguous() for s in (ks, vs)]
    ctx.set_force_simt(simt)
    try:
        fb.focus_sparse_attn_quantized(ctx, sh, dQ, q_base, N, rows, n_rows, cap, fb.make_quant_cache(FMT[fmt], *code, *scl),
                                       fb.HEADS_ALL if all_heads else fb.HEADS_PER_KV_GROUP, dev[0], max_blocks, dev[1], dev[2],
                                       dev[3], sinks, O, lse)
    finally:
        ctx.set_force_simt(False)
    torch.cuda.synchronize()
    return dict(O=O, lse=lse, Q=wl.storage_to_f64(Q, dtype)[pos - q_base], kc=kc, ks=ks, vc=vc, vs=vs, blocks=blocks, sink=sink, n=n)


@gpu
@pytest.mark.parametrize("simt", [False, True])
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("case", SPARSE)
def test_sparse_attention_over_an_8bit_cache(ctx, simt, fmt, case):
    dtype, H, Hkv, d, L, M, B, keep, sinks, N, n, cap, all_heads = case
    r = _run_sparse(ctx, case, fmt, simt, np.random.default_rng(L + M + H))
    scale = 1.0 / math.sqrt(d)
    K, V = r["kc"] * r["ks"][..., None], r["vc"] * r["vs"][..., None]
    eO, eL = fo.sparse_attn(r["Q"], K, V, M, B, r["blocks"], r["sink"], scale)
    keys = [fo.key_set(M, L, B, r["blocks"][0 if all_heads else g], r["sink"]) for g in range(Hkv)]
    tO, tL = _bounds(r["Q"], K, V, r["vs"], eO, scale, H // Hkv, dtype, keys)
    assert (np.abs(fstep.from_device(r["O"])[:n] - eO) <= tO).all()
    assert (np.abs(fstep.from_device(r["lse"])[:, :n] - eL) <= tL).all()
    assert (r["O"][n:] == 9).all() and (r["lse"][:, n:] == 9).all()
    assert ctx.poll_status() == 0


@gpu
@pytest.mark.parametrize("simt", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_without_a_key_give_zero(ctx, simt, dtype):
    """No block, no sink, no response token: O = 0 and lse = -inf."""
    L = M = 256
    sh = fb.make_shape(L, M, 2, 2, 64, 64, DT[dtype])
    Q = torch.randn(8, 2, 64, device="cuda").to(fstep.torch_dtype(dtype))
    codes, sc = torch.ones(2, L, 64, dtype=torch.int8, device="cuda"), torch.ones(2, L, device="cuda")
    cnt, idx = torch.zeros(2, dtype=torch.int32, device="cuda"), torch.full((2, 3), -1, dtype=torch.int32, device="cuda")
    O, lse = torch.full((8, 2, 64), 9.0, device="cuda").to(Q.dtype), torch.full((2, 8), 9.0, device="cuda")
    ctx.set_force_simt(simt)
    try:
        fb.focus_sparse_attn_quantized(ctx, sh, Q, L - 8, 8, None, None, 0, fb.make_quant_cache(fb.KV_INT8, codes, codes, sc, sc),
                                       fb.HEADS_PER_KV_GROUP, idx, 3, cnt, None, None, 0, O, lse)
    finally:
        ctx.set_force_simt(False)
    assert (O == 0).all() and torch.isneginf(lse).all()
    assert ctx.poll_status() == 0


@gpu
@pytest.mark.parametrize("simt", [False, True])
def test_unattended_rows_may_hold_anything(ctx, simt):
    """Codes and scales of tokens outside the key set are NaN: blocks not selected, and sinks whose keep flag is 0."""
    case = ("bf16", 2, 2, 128, 1500, 1400, 128, 3, 40, 30, 30, 0, False)
    _, H, Hkv, d, L, M, B, keep, sinks, N, n, cap, _ = case
    seen = {}

    def poison(kc, ks, vc, vs, blocks, sink, sk):
        sk[:, ::3] = 0                                                       # dropped wherever they lie
        seen["keep"] = sk.copy()
        for g in range(Hkv):
            attended = set(fo.key_set(M, L, B, blocks[g], sink[sk[g] != 0]).tolist())
            for j in range(L):
                if j not in attended:
                    kc[g, j] = vc[g, j] = np.nan
                    ks[g, j] = vs[g, j] = np.nan
    r = _run_sparse(ctx, case, "e4m3", simt, np.random.default_rng(3), poison)
    for g in range(Hkv):
        keys = fo.key_set(M, L, B, r["blocks"][g], r["sink"][seen["keep"][g] != 0])
        K, V = (c[g][keys] * s[g][keys][:, None] for c, s in ((r["kc"], r["ks"]), (r["vc"], r["vs"])))
        eO, eL = fo.dense_attn(r["Q"][:, g:g + 1], K[None], V[None], 1.0 / math.sqrt(d))
        tO, tL = _bounds(r["Q"][:, g:g + 1], K[None], V[None], r["vs"][g:g + 1, keys], eO, 1.0 / math.sqrt(d), 1, "bf16")
        assert (np.abs(fstep.from_device(r["O"])[:, g:g + 1] - eO) <= tO).all()
        assert (np.abs(fstep.from_device(r["lse"])[g:g + 1] - eL) <= tL).all()
    assert ctx.poll_status() == 0


@gpu
@pytest.mark.parametrize("simt", [False, True])
@pytest.mark.parametrize("kind", ["zero_values", "huge_and_tiny_scales", "sharp", "growing", "equal_logits"])
def test_scales_and_logits_of_unequal_size(ctx, simt, kind):
    rng = np.random.default_rng(11)
    H, Hkv, d, L, N = 2, 2, 128, 900, 40
    Q, (kc, ks), (vc, vs) = _attention_case(rng, "bf16", "int8", H, Hkv, d, L, N, 1.0)
    if kind == "zero_values":                        # attention sinks with no value; an all-zero key row
        vs[:, ::7], vc[:, ::7] = 0.0, 0.0
        ks[:, 5], kc[:, 5] = 0.0, 0.0
        ks[:, 14] *= 6.0
    elif kind == "huge_and_tiny_scales":
        vs *= np.exp2(rng.integers(-40, 40, size=vs.shape)).astype(np.float64)
    elif kind == "sharp":
        ks *= 6.0
    elif kind == "growing":                          # every tile's logits exceed all before it
        ks *= np.linspace(0.05, 8.0, L)
    else:
        kc[:] = kc[:, :1]
        ks[:] = ks[:, :1]
    ks, vs = ks.astype(np.float32).astype(np.float64), vs.astype(np.float32).astype(np.float64)
    K, V = kc * ks[..., None], vc * vs[..., None]
    sh = fb.make_shape(L, L, H, Hkv, d, 64, fb.BF16)
    O, lse = torch.zeros(N, H, d, dtype=torch.bfloat16, device="cuda"), torch.zeros(H, N, device="cuda")
    dev = [codes_to_device(c, "int8") for c in (kc, vc)] + [torch.from_numpy(s).float().cuda().contiguous() for s in (ks, vs)]
    ctx.set_force_simt(simt)
    try:
        fb.focus_dense_attn_quantized(ctx, sh, fstep.to_device(Q, "bf16"), L - N, N, None, None, 0, fb.make_quant_cache(fb.KV_INT8, *dev),
                                      O, lse)
    finally:
        ctx.set_force_simt(False)
    Qf = wl.storage_to_f64(Q, "bf16")
    eO, eL = fo.dense_attn(Qf, K, V, 1.0 / math.sqrt(d))
    tO, tL = _bounds(Qf, K, V, vs, eO, 1.0 / math.sqrt(d), 1, "bf16")
    assert (np.abs(fstep.from_device(O) - eO) <= tO).all()
    assert (np.abs(fstep.from_device(lse) - eL) <= tL).all()
    assert ctx.poll_status() == 0


@gpu
def test_bad_rows_blocks_and_sinks_are_reported(ctx):
    H, Hkv, d, L, M, N = 2, 2, 128, 600, 500, 40
    sh = fb.make_shape(L, M, H, Hkv, d, 64, fb.BF16)
    Q = torch.randn(N, H, d, device="cuda").bfloat16()
    codes = torch.randint(-127, 128, (Hkv, L, d), dtype=torch.int8, device="cuda")
    sc = torch.rand(Hkv, L, device="cuda") * 0.02
    cache = fb.make_quant_cache(fb.KV_INT8, codes, codes, sc, sc)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    ok_rows, n_rows = i32([560, 570, 599]), i32([3])
    blocks, cnt, sink = i32([[1, 4], [0, 7]]), i32([2, 2]), i32([70, 130])
    keep = torch.ones(2, 2, dtype=torch.uint8, device="cuda")

    def call(rows=ok_rows, blocks=blocks, sink=sink):
        O = torch.full((3, H, d), 9.0, dtype=torch.bfloat16, device="cuda")
        fb.focus_sparse_attn_quantized(ctx, sh, Q, L - N, N, rows, n_rows, 3, cache, fb.HEADS_PER_KV_GROUP, blocks, 2, cnt, sink,
                                       keep, 2, O, None)
        return O, ctx.poll_status()
    good, status = call()
    assert status == 0
    O, status = call(rows=i32([560, 12, 599]))                              # position without a query row: its output stays
    assert status == fb.ERR_INVALID_ARG and torch.equal(O[[0, 2]], good[[0, 2]]) and (O[1] == 9).all()
    O, status = call(blocks=i32([[1, 4], [0, 8]]))                          # block 8 of [0, 8): left out
    assert status == fb.ERR_INVALID_ARG and torch.equal(O[:, 0], good[:, 0]) and torch.isfinite(O.float()).all()
    O, status = call(sink=i32([70, L]))
    assert status == fb.ERR_INVALID_ARG and torch.isfinite(O.float()).all()


# ---- the calls together, as a layer uses them -----------------------------------------------------------------------
@gpu
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_a_sparse_layer_over_an_8bit_cache(ctx, fmt):
    """Block entry fills the cache, a step refreshes the active rows, the keys are read back for pooling and sink
    identification, blocks are selected and attended; captured into a graph and replayed with new rows."""
    rng = np.random.default_rng(8)
    H, Hkv, d, L, M, B, C, n_sink, n = 4, 2, 128, 1400, 1200, 64, 5, 12, 24
    sh = fb.make_shape(L, M, H, Hkv, d, B, fb.BF16)
    bf = lambda *s: torch.from_numpy(rng.standard_normal(s).astype(np.float32)).cuda().bfloat16()
    K0, V0, Q = bf(L, Hkv, d), bf(L, Hkv, d), bf(L - M, H, d)
    Kn, Vn = bf(n, Hkv, d), bf(n, Hkv, d)
    pos = np.sort(rng.choice(np.arange(M, L), size=n, replace=False))
    i32 = dict(dtype=torch.int32, device="cuda")
    rows, n_rows = torch.from_numpy(pos.astype(np.int32)).cuda(), torch.tensor([n], **i32)
    codes = [torch.zeros(Hkv, L, d, dtype=torch.int8, device="cuda") for _ in range(2)]
    sc = [torch.zeros(Hkv, L, device="cuda") for _ in range(2)]
    cache = fb.make_quant_cache(FMT[fmt], *codes, *sc)
    Kb = torch.zeros(Hkv, L, d, dtype=torch.bfloat16, device="cuda")
    nb = (M + B - 1) // B
    Kbar, R, S = torch.zeros(Hkv, nb, d, device="cuda"), torch.zeros(Hkv * nb, device="cuda"), torch.zeros(L, device="cuda")
    sinks, blocks, cnt = torch.full((n_sink,), -1, **i32), torch.full((Hkv, C), -1, **i32), torch.zeros(Hkv, **i32)
    keep = torch.zeros(Hkv, n_sink, dtype=torch.uint8, device="cuda")
    O, O2 = (torch.zeros(n, H, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    lse, lse2 = torch.zeros(H, n, device="cuda"), torch.zeros(H, n, device="cuda")
    fb.focus_quantize_kv(ctx, sh, K0, V0, Hkv * d, d, 0, None, None, L, cache)

    def layer():
        fb.focus_quantize_kv(ctx, sh, Kn, Vn, Hkv * d, d, 0, rows, n_rows, n, cache)
        fb.focus_dequantize_kv(ctx, sh, cache, 0, None, None, L, Kb, None, d, L * d)
        fb.focus_pool_keys(ctx, sh, Kb, Kbar)
        fb.focus_dense_attn_quantized(ctx, sh, Q, M, L - M, rows, n_rows, n, cache, O, lse)
        fb.focus_find_sinks(ctx, sh, Q, M, rows, n_rows, n, Kb, lse, n_sink, 0, M, sinks, S)
        fb.focus_score_blocks(ctx, sh, Q, M, rows, n_rows, n, None, Kbar, fb.HEADS_PER_KV_GROUP, R)
        fb.focus_select_blocks(ctx, sh, R, fb.HEADS_PER_KV_GROUP, C, sinks, n_sink, fb.SINK_TOKENS, blocks, C, cnt, keep)
        fb.focus_sparse_attn_quantized(ctx, sh, Q, M, L - M, rows, n_rows, n, cache, fb.HEADS_PER_KV_GROUP, blocks, C, cnt, sinks,
                                       keep, n_sink, O2, lse2)

    def check():
        torch.cuda.synchronize()
        assert ctx.poll_status() == 0
        K, V = K0.clone(), V0.clone()
        K[rows.long()], V[rows.long()] = Kn, Vn
        want = [fo.quantize_rows(t.double().cpu().numpy().transpose(1, 0, 2), fmt) for t in (K, V)]
        Kd, Vd = (c * s[..., None] for c, s in want)
        view = torch.int8 if fmt == "int8" else torch.float8_e4m3fn
        assert np.array_equal(code_values(codes[0].view(view)), want[0][0]) and np.array_equal(code_values(codes[1].view(view)), want[1][0])
        q = Q.double().cpu().numpy()[rows.cpu().numpy() - M]
        scale = 1.0 / math.sqrt(d)
        eO, eL = fo.dense_attn(q, Kd, Vd, scale)
        tO, tL = _bounds(q, Kd, Vd, want[1][1], eO, scale, H // Hkv, "bf16")
        assert (np.abs(fstep.from_device(O) - eO) <= tO).all() and (np.abs(fstep.from_device(lse) - eL) <= tL).all()
        bl, sk = [b for b in blocks.cpu().numpy()], sinks.cpu().numpy()
        assert all((b >= 0).all() for b in bl) and (sk >= 0).all()
        eO, eL = fo.sparse_attn(q, Kd, Vd, M, B, bl, sk, scale)
        keys = [fo.key_set(M, L, B, bl[g], sk) for g in range(Hkv)]
        tO, tL = _bounds(q, Kd, Vd, want[1][1], eO, scale, H // Hkv, "bf16", keys)
        assert (np.abs(fstep.from_device(O2) - eO) <= tO).all() and (np.abs(fstep.from_device(lse2) - eL) <= tL).all()

    layer()
    check()
    eager = [t.clone() for t in (O, O2, lse, lse2)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        layer()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(eager, (O, O2, lse, lse2)))            # same inputs, same bits
    Kn.copy_(bf(n, Hkv, d)), Vn.copy_(bf(n, Hkv, d)), Q.copy_(bf(L - M, H, d))
    graph.replay()
    check()


# ---- limits ---------------------------------------------------------------------------------------------------------
def _random_cache(rng, fmt, Hkv, L, d):
    """Codes and scales straight from the generator: (code values, scales, device codes, device scales)."""
    if fmt == "int8":
        vals = rng.integers(-127, 128, size=(Hkv, L, d)).astype(np.float64)
    else:
        bits = rng.integers(0, 256, size=(Hkv, L, d)).astype(np.uint8)
        bits[(bits & 0x7f) >= 0x78] = 0x31                                  # no NaN, none above 240
        vals = torch.from_numpy(bits).view(torch.float8_e4m3fn).float().double().numpy()
    top = 127.0 if fmt == "int8" else 240.0
    sc = (np.exp(0.5 * rng.standard_normal((Hkv, L))) / top * 1.7).astype(np.float32)
    return vals, sc.astype(np.float64), codes_to_device(vals, fmt), torch.from_numpy(sc).cuda()


@gpu
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("L,M,keep,sinks", [(41001, 0, 0, 0), (36000, 35900, 300, 1500), (9000, 8800, 0, 2000)])
def test_long_key_sets(ctx, fmt, L, M, keep, sinks):
    """One KV head: more than 256 key tiles (those of a split that are staged at once), as many splits as there can be, more
    than eight tiles of sinks.  M == 0: dense."""
    rng = np.random.default_rng(L + sinks)
    H, Hkv, d, B, N, n = 2, 1, 64, 64, 40, 33
    Q = storage(rng.standard_normal((N, H, d)), "bf16")
    kv, ks, dk, dks = _random_cache(rng, fmt, Hkv, L, d)
    vv, vs, dv, dvs = _random_cache(rng, fmt, Hkv, L, d)
    K, V = kv * ks[..., None], vv * vs[..., None]
    pos = np.sort(rng.choice(N, size=n, replace=False)) + L - N
    pos[3] = pos[2]                                                          # a position may be listed twice
    rows, n_rows = torch.from_numpy(pos.astype(np.int32)).cuda(), torch.tensor([n], dtype=torch.int32, device="cuda")
    dQ, O = fstep.to_device(Q, "bf16"), torch.full((n, H, d), 9.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((H, n), 9.0, device="cuda")
    cache = fb.make_quant_cache(FMT[fmt], dk, dv, dks, dvs)
    Qf, scale = wl.storage_to_f64(Q, "bf16")[pos - (L - N)], 1.0 / math.sqrt(d)
    if M == 0:
        fb.focus_dense_attn_quantized(ctx, fb.make_shape(L, L, H, Hkv, d, B, fb.BF16), dQ, L - N, N, rows, n_rows, n, cache, O, lse)
        eO, eL = fo.dense_attn(Qf, K, V, scale)
        keys = None
    else:
        blocks = [np.sort(rng.choice((M + B - 1) // B, size=keep, replace=False))]
        sink = np.sort(rng.choice(M, size=sinks, replace=False))
        sk = np.array([[0 if (s // B) in set(blocks[0]) else 1 for s in sink]], dtype=np.uint8)
        dev = [torch.from_numpy(a).cuda() for a in (np.concatenate([blocks[0], [-1]]).astype(np.int32)[None],
                                                    np.array([keep], dtype=np.int32), sink.astype(np.int32), sk)]
        fb.focus_sparse_attn_quantized(ctx, fb.make_shape(L, M, H, Hkv, d, B, fb.BF16), dQ, L - N, N, rows, n_rows, n, cache,
                                       fb.HEADS_PER_KV_GROUP, dev[0], keep + 1, dev[1], dev[2], dev[3], sinks, O, lse)
        eO, eL = fo.sparse_attn(Qf, K, V, M, B, blocks, sink, scale)
        keys = [fo.key_set(M, L, B, blocks[0], sink)]
    assert ctx.last_attn_variant() == 5
    tO, tL = _bounds(Qf, K, V, vs, eO, scale, H // Hkv, "bf16", keys)
    assert (np.abs(fstep.from_device(O) - eO) <= tO).all() and (np.abs(fstep.from_device(lse) - eL) <= tL).all()
    assert ctx.poll_status() == 0


@gpu
@pytest.mark.parametrize("simt", [False, True])
def test_offsets_beyond_32_bits(ctx, simt):
    """Tokens a MiB apart, K and V interleaved in one buffer of more than 2^32 bytes: written, read back, attended."""
    L, H, d, step = 4200, 2, 64, 1 << 20
    buf = torch.empty(L * step, dtype=torch.int8, device="cuda")
    K, V = (buf[o:].as_strided((H, L, d), (256, step, 1)) for o in (0, 128))
    sc = torch.zeros(2, H, L, device="cuda")
    cache = fb.make_quant_cache(fb.KV_INT8, buf, buf[128:], sc[0], sc[1])
    sh = fb.make_shape(L, L, H, H, d, 64, fb.BF16, kv_stride_tok=step, kv_stride_head=256)
    g = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn(2, L, H, d, generator=g, device="cuda").bfloat16()
    fb.focus_quantize_kv(ctx, sh, x[0], x[1], H * d, d, 0, None, None, L, cache)
    top = x.float().abs().amax(-1).cpu().numpy() / np.float32(127)            # IEEE division (the device's by a constant is not)
    assert np.array_equal(sc.cpu().numpy(), top.swapaxes(1, 2)) and bool((K.abs().amax(-1) == 127).all())
    out = torch.empty(2, H, L, d, dtype=torch.bfloat16, device="cuda")
    fb.focus_dequantize_kv(ctx, sh, cache, 0, None, None, L, out[0], out[1], d, L * d)
    for got, codes, s in ((out[0], K, sc[0]), (out[1], V, sc[1])):
        assert torch.equal(got, (codes.float() * s[..., None]).bfloat16())
    Q = torch.randn(9, H, d, generator=g, device="cuda").bfloat16()
    O = torch.empty(9, H, d, dtype=torch.bfloat16, device="cuda")
    ctx.set_force_simt(simt)
    try:
        fb.focus_dense_attn_quantized(ctx, sh, Q, L - 9, 9, None, None, 0, cache, O, None)
    finally:
        ctx.set_force_simt(False)
    Kd, Vd = ((c.double() * s[..., None].double()).cpu().numpy() for c, s in ((K, sc[0]), (V, sc[1])))
    Qf = Q.double().cpu().numpy()
    eO, _ = fo.dense_attn(Qf, Kd, Vd, 1.0 / math.sqrt(d))
    tO, _ = _bounds(Qf, Kd, Vd, sc[1].double().cpu().numpy(), eO, 1.0 / math.sqrt(d), 1, "bf16")
    assert (np.abs(fstep.from_device(O) - eO) <= tO).all()
    assert ctx.poll_status() == 0


@gpu
def test_two_graphs_on_one_context_and_another_stream(ctx):
    """Two captured sequences (write, dense, sparse) that share the context's workspace, replayed in turn on a stream other
    than the current one, against the eager calls."""
    L, M, H, Hkv, d, N, rows = 6000, 5900, 8, 4, 128, 100, 40
    g = torch.Generator(device="cuda").manual_seed(11)
    sets = []
    for fmt in (fb.KV_INT8, fb.KV_E4M3):
        s = dict(x=torch.randn(2, L, Hkv, d, generator=g, device="cuda").bfloat16(),
                 Q=torch.randn(N, H, d, generator=g, device="cuda").bfloat16(),
                 pos=torch.arange(L - N, L - N + rows, dtype=torch.int32, device="cuda"),
                 n=torch.tensor([rows], dtype=torch.int32, device="cuda"), codes=torch.zeros(2, Hkv, L, d, dtype=torch.int8, device="cuda"),
                 sc=torch.zeros(2, Hkv, L, device="cuda"), idx=torch.tensor([[0, 3, 17, 40, -1]] * Hkv, dtype=torch.int32, device="cuda"),
                 cnt=torch.full((Hkv,), 4, dtype=torch.int32, device="cuda"),
                 sink=torch.tensor([130, 700, 5899], dtype=torch.int32, device="cuda"),
                 keep=torch.ones(Hkv, 3, dtype=torch.uint8, device="cuda"),
                 O=torch.zeros(2, rows, H, d, dtype=torch.bfloat16, device="cuda"), lse=torch.zeros(2, H, rows, device="cuda"))
        s["cache"] = fb.make_quant_cache(fmt, s["codes"][0], s["codes"][1], s["sc"][0], s["sc"][1])
        sets.append(s)
    sh = fb.make_shape(L, M, H, Hkv, d, 128, fb.BF16)

    def run(s, stream):
        fb.focus_quantize_kv(ctx, sh, s["x"][0], s["x"][1], Hkv * d, d, 0, None, None, L, s["cache"], stream=stream)
        fb.focus_dense_attn_quantized(ctx, sh, s["Q"], L - N, N, s["pos"], s["n"], rows, s["cache"], s["O"][0], s["lse"][0], stream=stream)
        fb.focus_sparse_attn_quantized(ctx, sh, s["Q"], L - N, N, s["pos"], s["n"], rows, s["cache"], fb.HEADS_PER_KV_GROUP, s["idx"], 5,
                                       s["cnt"], s["sink"], s["keep"], 3, s["O"][1], s["lse"][1], stream=stream)

    want = []
    for s in sets:
        run(s, None)
        want.append([s[k].clone() for k in ("codes", "sc", "O", "lse")])
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    graphs = []
    for s in sets:
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr, stream=side):
            run(s, side)
        graphs.append(gr)
    with torch.cuda.stream(side):
        for _ in range(3):
            for s, gr in zip(sets, graphs):
                for k in ("codes", "sc", "O", "lse"):
                    s[k].zero_()
                gr.replay()
            side.synchronize()
            for s, w in zip(sets, want):
                assert all(torch.equal(s[k], t) for k, t in zip(("codes", "sc", "O", "lse"), w))
    run(sets[0], side)                                                       # a stream that is not the current one
    side.synchronize()
    assert torch.equal(sets[0]["O"], want[0][2])
    assert ctx.poll_status() == 0


@gpu
def test_workspace_of_quantized_attention():
    """A workspace that is too small is reported; one of the advertised size carries the calls."""
    L, M, H, d, N = 20000, 19900, 4, 128, 64
    sh = fb.make_shape(L, M, H, H, d, 128, fb.BF16)
    codes, sc = torch.ones(H, L, d, dtype=torch.int8, device="cuda"), torch.ones(H, L, device="cuda")
    cache = fb.make_quant_cache(fb.KV_INT8, codes, codes, sc, sc)
    Q, O = torch.randn(N, H, d, device="cuda").bfloat16(), torch.zeros(N, H, d, dtype=torch.bfloat16, device="cuda")
    tiny = fb.Context(0, workspace_bytes=4096)
    with pytest.raises(fb.FocusError) as e:
        fb.focus_dense_attn_quantized(tiny, sh, Q, L - N, N, None, None, 0, cache, O, None)
    assert e.value.code == fb.ERR_WORKSPACE_TOO_SMALL and bool((O == 0).all())
    tiny.close()
    c = fb.Context(0, workspace_bytes=fb.focus_workspace_bytes(sh, N, 8, 4))
    fb.focus_dense_attn_quantized(c, sh, Q, L - N, N, None, None, 0, cache, O, None)
    assert bool((O == 1).all()) and c.poll_status() == 0                     # every value is 1
    c.close()


@gpu
def test_the_readmes_second_example_runs_as_printed(ctx):
    import os
    import re
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")).read()
    code = re.findall(r"```python\n(.*?)```", text, flags=re.S)[1]
    L, M, H, Hkv, d, B, k, C, n_sink, vocab = 2000, 1700, 8, 4, 128, 128, 4, 3, 5, 1000
    g = torch.Generator(device="cuda").manual_seed(2)

    def randn(*shape):
        return torch.randn(*shape, generator=g, device="cuda").bfloat16()

    i32 = dict(dtype=torch.int32, device="cuda")
    env = dict(fb=fb, ctx=ctx, L=L, M=M, H=H, Hkv=Hkv, d=d, k=k, C=C, n_sink=n_sink, vocab=vocab,
               shape=fb.make_shape(L, M, H, Hkv, d, B, fb.BF16), codes=torch.zeros(2, Hkv, L, d, dtype=torch.uint8, device="cuda"),
               scales=torch.zeros(2, Hkv, L, device="cuda"), K_rows=randn(L, Hkv, d), V_rows=randn(L, Hkv, d), K_new=randn(k * 9, Hkv, d),
               V_new=randn(k * 9, Hkv, d), active=torch.arange(M + 3, M + 3 + k * 9, **i32), n_active=torch.tensor([30], **i32),
               Q=randn(L - M, H, d), O=randn(k * 9, H, d), lse=torch.zeros(H, k * 9, device="cuda"),
               blocks=torch.tensor([0, 4, 9] * Hkv, **i32), cnt=torch.full((Hkv,), C, **i32), sinks=torch.tensor([1, 2, 3, 600, 1699], **i32),
               keep=torch.ones(Hkv * n_sink, dtype=torch.uint8, device="cuda"), logits=randn(L - M, vocab), u=torch.rand(k * 9, device="cuda"),
               conf=torch.zeros(k * 9, device="cuda"), token=torch.zeros(k * 9, **i32), prob=torch.zeros(k * 9, device="cuda"),
               K=torch.zeros(Hkv, L, d, dtype=torch.bfloat16, device="cuda"))
    exec(code, env)
    assert ctx.poll_status() == 0
    rows = env["K_rows"].clone()
    rows[M + 3:M + 33] = env["K_new"][:30]
    err = (env["K"].transpose(0, 1).float() - rows.float()).abs()
    # e4m3: half a step of 2^-3 (2^-4 of the element), or half of the smallest step, 2^-9 scales (scale = max / 448); bf16
    # adds 2^-8 and the scale's own rounding 2^-23
    top = rows.float().abs().amax(-1, keepdim=True)
    assert bool((err <= (2.0 ** -4 + 2.0 ** -7) * rows.float().abs() + 2.0 ** -10 * top / 448).all())
    assert torch.isfinite(env["O"][:30].float()).all() and bool((env["token"][:30] >= 0).all()) and bool((env["token"][30:] == -1).all())


# ---- value scales far apart: a row's sum and log-sum-exp do not depend on them -------------------------------------
FAR = 2.0 ** -17 * math.log(2.0)
# exponents (log2 of a value scale, a logit with it, the same less its reference) are below 2^8 in magnitude here: each is
# rounded by at most 2^-17, which is a factor of 1 + FAR; three of them meet a numerator, two more its row's log-sum-exp


def _far_scales(rng, kind, Hkv, L, d):
    """Value codes and scales: a V row is all zeros, tiny or large."""
    vc = rng.integers(-127, 128, size=(Hkv, L, d)).astype(np.float64)
    vc[..., 0] = 127.0
    e = rng.integers(45, 100, size=(Hkv, L))
    first, odd = np.arange(L) < L // 2, np.arange(L) // 128 % 2 == 1
    if kind == "zeros_beside_large":
        e = np.where(rng.random((Hkv, L)) < 0.5, e, -1000)
    elif kind == "tiny_beside_large":
        e = np.where(rng.random((Hkv, L)) < 0.5, e, -e + 20)
    elif kind == "large_last":                       # the splits of a key set, and the tiles of a split, differ
        e = np.where(first, -80, 95) + 0 * e
    elif kind == "large_first":
        e = np.where(first, 95, -80) + 0 * e
    elif kind == "tiles_in_turn":
        e = np.where(odd, 95, -80) + 0 * e
    else:                                            # all of them large, or all of them tiny
        e = np.where(np.arange(Hkv)[:, None] % 2 == 0, 100, -80) + 0 * e
    vs = np.where(e == -1000, 0.0, np.exp2(np.maximum(e, -80).astype(np.float64)) * rng.integers(2 ** 19, 2 ** 20, (Hkv, L)) / 2.0 ** 20)
    vc[vs == 0.0] = 0.0
    return vc, vs


@gpu
@pytest.mark.parametrize("simt", [False, True])
@pytest.mark.parametrize("kind", ["zeros_beside_large", "tiny_beside_large", "large_last", "large_first", "tiles_in_turn", "one_size"])
@pytest.mark.parametrize("H,Hkv,d,L,N", [(2, 2, 128, 900, 40), (80, 80, 64, 1100, 3), (4, 2, 128, 200, 30), (1, 1, 64, 6000, 5)])
def test_value_scales_far_apart(ctx, simt, kind, H, Hkv, d, L, N):
    """Every size that the writer makes (2^-87 .. 2^120, and 0) in one key set: O and lse of rows whose tokens all count."""
    rng = np.random.default_rng(L + N)
    Q = storage(rng.standard_normal((N, H, d)), "bf16")
    kc, ks = fo.quantize_rows(rng.standard_normal((Hkv, L, d)) * 0.3, "int8")
    vc, vs = _far_scales(rng, kind, Hkv, L, d)
    K, V = kc * ks[..., None], vc * vs[..., None]
    O, lse = torch.zeros(N, H, d, dtype=torch.bfloat16, device="cuda"), torch.zeros(H, N, device="cuda")
    dev = [codes_to_device(c, "int8") for c in (kc, vc)] + [torch.from_numpy(s).float().cuda().contiguous() for s in (ks, vs)]
    ctx.set_force_simt(simt)
    try:
        fb.focus_dense_attn_quantized(ctx, fb.make_shape(L, L, H, Hkv, d, 64, fb.BF16), fstep.to_device(Q, "bf16"), L - N, N, None, None, 0,
                                      fb.make_quant_cache(fb.KV_INT8, *dev), O, lse)
    finally:
        ctx.set_force_simt(False)
    Qf, scale = wl.storage_to_f64(Q, "bf16"), 1.0 / math.sqrt(d)
    eO, eL = fo.dense_attn(Qf, K, V, scale)
    tO, tL = _bounds(Qf, K, V, vs, eO, scale, H // Hkv, "bf16")
    for h in range(H):
        s = Qf[:, h] @ K[h // (H // Hkv)].T * scale
        p = np.exp(s - s.max(1, keepdims=True))
        tO[:, h] += 2 * 3 * FAR * (p / p.sum(1, keepdims=True)) @ np.abs(V[h // (H // Hkv)])
    assert (np.abs(fstep.from_device(lse) - eL) <= tL + 5 * FAR).all()
    assert (np.abs(fstep.from_device(O) - eO) <= tO).all()
    assert ctx.poll_status() == 0


@gpu
@pytest.mark.parametrize("simt", [False, True])
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_a_token_without_a_value_takes_its_share(ctx, simt, fmt):
    """Two tokens of equal logits, a V row of zeros beside one of any size: O is half of it and lse is log 2 more than a logit."""
    d = 64
    sh = fb.make_shape(2, 2, 1, 1, d, 64, fb.BF16)
    Q = torch.zeros(1, 1, d, device="cuda").bfloat16()
    for e in (0, 30, 40, 41, 45, 60, 90, 120):
        x = torch.zeros(2, 1, d, device="cuda")
        x[0] = 2.0 ** e
        codes, sc = torch.zeros(2, 1, 2, d, dtype=torch.int8, device="cuda"), torch.zeros(2, 1, 2, device="cuda")
        cache = fb.make_quant_cache(FMT[fmt], codes[0], codes[1], sc[0], sc[1])
        rows = x.bfloat16().contiguous()
        fb.focus_quantize_kv(ctx, sh, torch.zeros_like(rows), rows, d, d, 0, None, None, 2, cache)
        O, lse = torch.zeros(1, 1, d, dtype=torch.bfloat16, device="cuda"), torch.zeros(1, 1, device="cuda")
        ctx.set_force_simt(simt)
        try:
            fb.focus_dense_attn_quantized(ctx, sh, Q, 0, 1, None, None, 0, cache, O, lse)
        finally:
            ctx.set_force_simt(False)
        # the stored value 2^e up to its scale's rounding (2^-24), fp16 numerators 2^-11, bf16 2^-8, exponents as above
        want = 2.0 ** (e - 1)
        assert bool(((O.double() - want).abs() <= want * (2.0 ** -8 + 2.0 ** -11 + 6 * FAR + 2.0 ** -20)).all()), e
        assert abs(float(lse) - math.log(2.0)) <= 5 * FAR + 2.0 ** -21, e
    assert ctx.poll_status() == 0


@gpu
def test_both_forms_of_a_wait_keep_to_their_limit(ctx):
    """The self-test waits in the form of this file's kernel first, then in the other kernels': each for as long as it was told,
    by the clock (a poll may stay suspended for as long as the hardware likes, so their number says nothing)."""
    start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    for limit_ms in (30, 90):
        start.record()
        ctx.selftest_bounded_wait(1000 * limit_ms)
        end.record()
        assert ctx.poll_status() == fb.ERR_TIMEOUT
        assert 2 * limit_ms <= start.elapsed_time(end) < 2 * limit_ms + 100
    assert ctx.poll_status() == 0


@gpu
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_rows_read_back_as_bf16_are_rounded_by_way_of_fp32(ctx, fmt):
    """The two roundings that the header states, against products in 64 bits: every output is the fp32 product's nearest bf16,
    and differs from the exact product's nearest only where that fp32 product is half way between two."""
    Hkv, L, d = 2, 2048, 128
    rng = np.random.default_rng(9)
    if fmt == "int8":
        vals = rng.integers(-127, 128, size=(Hkv, L, d)).astype(np.float64)
    else:
        bits = rng.integers(0, 256, size=(Hkv, L, d)).astype(np.uint8)
        bits[(bits & 0x7f) == 0x7f] = 0x40
        vals = torch.from_numpy(bits).view(torch.float8_e4m3fn).float().double().numpy()
    sc = np.exp2(rng.integers(-40, 40, size=(Hkv, L))) * rng.integers(2 ** 23, 2 ** 24, size=(Hkv, L)) / 2.0 ** 24
    vals[0, 0], sc[0, 0] = 6.0, float.fromhex("0x1.895554p-7")             # 6 x it is just below a tie, in fp32 the tie itself
    out = torch.zeros(Hkv, L, d, dtype=torch.bfloat16, device="cuda")
    codes, scales = codes_to_device(vals, fmt), torch.from_numpy(sc).float().cuda()
    fb.focus_dequantize_kv(ctx, fb.make_shape(L, 0, 2, Hkv, d, 64, fb.BF16), fb.make_quant_cache(FMT[fmt], codes, None, scales, None), 0,
                           None, None, L, out, None, d, L * d)
    exact = vals * sc[..., None]                                            # 8 + 24 bits: exact in 64
    got = out.double().cpu().numpy()
    single = exact.astype(np.float32)
    step = np.exp2(np.floor(np.log2(np.maximum(np.abs(exact), 2.0 ** -120))) - 7)       # of bf16 there (8 bits)
    assert (np.abs(got - exact) <= step / 2 + np.abs(exact) * 2.0 ** -24).all()
    assert (np.abs(got - single.astype(np.float64)) <= step / 2).all()
    tie = (single.view(np.uint32) & 0xFFFF) == 0x8000
    assert (np.abs(got - exact)[~tie] <= step[~tie] / 2).all()
    assert tie[0, 0].all() and (got[0, 0] == 0.072265625).all() and np.abs(exact[0, 0, 0] - 0.07177734375) < np.abs(exact[0, 0, 0] - 0.072265625)
    assert ctx.poll_status() == 0


@gpu
@pytest.mark.parametrize("simt", [False, True])
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_the_smallest_values_that_are_kept_are_attended(ctx, simt, fmt):
    """V rows whose largest magnitude is 2^-80 and a little more, the smallest that are not stored as zeros: their scales are the
    smallest there are (2^-80 / Q)."""
    rng = np.random.default_rng(4)
    H, d, L, N = 2, 64, 300, 20
    x = rng.uniform(-1.0, 1.0, size=(L, H, d))
    x[..., 0] = 1.0
    x *= 2.0 ** -80 * rng.choice([1.0, 1.25, 2.0, 3.0], size=(L, H, 1))
    V, K = storage(x, "bf16"), storage(rng.standard_normal((L, H, d)), "bf16")
    codes, sc = torch.zeros(2, H, L, d, dtype=torch.int8, device="cuda"), torch.zeros(2, H, L, device="cuda")
    cache = fb.make_quant_cache(FMT[fmt], codes[0], codes[1], sc[0], sc[1])
    sh = fb.make_shape(L, L, H, H, d, 64, fb.BF16)
    fb.focus_quantize_kv(ctx, sh, fstep.to_device(K, "bf16"), fstep.to_device(V, "bf16"), H * d, d, 0, None, None, L, cache)
    assert bool((sc[1] > 0).all())
    Q = storage(rng.standard_normal((N, H, d)), "bf16")
    O, lse = torch.zeros(N, H, d, dtype=torch.bfloat16, device="cuda"), torch.zeros(H, N, device="cuda")
    ctx.set_force_simt(simt)
    try:
        fb.focus_dense_attn_quantized(ctx, sh, fstep.to_device(Q, "bf16"), L - N, N, None, None, 0, cache, O, lse)
    finally:
        ctx.set_force_simt(False)
    kc, vc = (fo.quantize_rows(wl.storage_to_f64(a, "bf16").transpose(1, 0, 2), fmt) for a in (K, V))
    Kd, Vd = (c * s[..., None] for c, s in (kc, vc))
    Qf, scale = wl.storage_to_f64(Q, "bf16"), 1.0 / math.sqrt(d)
    eO, eL = fo.dense_attn(Qf, Kd, Vd, scale)
    tO, tL = _bounds(Qf, Kd, Vd, vc[1], eO, scale, 1, "bf16")
    for h in range(H):                                                      # exponents near 2^-87, rounded as FAR says
        s = Qf[:, h] @ Kd[h].T * scale
        p = np.exp(s - s.max(1, keepdims=True))
        tO[:, h] += 2 * 3 * FAR * (p / p.sum(1, keepdims=True)) @ np.abs(Vd[h])
    assert (np.abs(fstep.from_device(O) - eO) <= tO).all()
    assert (np.abs(fstep.from_device(lse) - eL) <= tL + 5 * FAR).all()
    assert ctx.poll_status() == 0
