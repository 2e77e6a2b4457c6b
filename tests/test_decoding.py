"""The batched decoding calls in the order in which a program makes them: a projection's rows rotated and appended to their
pages (focus_append_kv_paged), attended (focus_paged_attn), and the logits scored (focus_token_logprobs, focus_confidence,
focus_sample); step by step, captured in a graph, with windows of rows that are replaced, and beside the contiguous path."""
import math

import numpy as np
import pytest
import torch

from oracle import focus_oracle as fo
from paper_2602_02159_b200 import binding as fb

gpu = pytest.mark.gpu
H, HKV, D, VOCAB, PAGE, L = 8, 2, 64, 1003, 16, 160
BF16_HALF = 2.0 ** -8


@pytest.fixture(scope="module")
def ctx():
    c = fb.Context(0)
    yield c
    assert c.poll_status() == 0
    c.close()


def f64(t):
    return t.detach().double().cpu().numpy()


class Model:
    """One layer: tokens -> fused projection rows -> attention -> logits (the products are PyTorch's)."""

    def __init__(self, n, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.qkv = torch.randn(VOCAB, (H + 2 * HKV) * D, generator=g, device="cuda").bfloat16()      # per token
        self.head = (torch.randn(H * D, 1008, generator=g, device="cuda") * 0.3).bfloat16()
        self.rope = fb.make_rope(D, fb.ROPE_HALVES, 10000.0, fb.ROPE_LINEAR, 2.0)
        self.freq, _ = fo.rope_frequencies(D, 10000.0, "linear", 2.0)
        self.n, self.wide = n, L // PAGE
        self.K, self.V = (torch.full((n * self.wide + 2, PAGE, HKV, D), float("nan"), device="cuda").bfloat16() for _ in range(2))
        self.table = torch.randperm(n * self.wide + 2, generator=g, device="cuda")[:n * self.wide].int().reshape(n, self.wide)
        self.kv_len = torch.zeros(n, dtype=torch.int32, device="cuda")
        self.shape = fb.make_shape(L, 0, H, HKV, D, 64, fb.BF16)
        self.cache = fb.make_paged_cache(self.K, self.V, self.table, self.kv_len, PAGE, self.K.shape[0], n, self.wide, self.K.stride(0),
                                         self.K.stride(1), self.K.stride(2))

    def layer(self, ctx, x, Q, O, lse, row_start=None, positions=None):
        """x: rows [rows, H + 2 HKV, D] of the projection."""
        rows = x.shape[0]
        fb.focus_append_kv_paged(ctx, self.shape, self.rope, x, x[:, H:], x[:, H + HKV:], x.stride(0), x.stride(1), row_start,
                                 positions, rows, self.cache, Q)
        fb.focus_paged_attn(ctx, self.shape, Q, row_start, rows, self.cache, O, lse)


def buffers(rows):
    z = lambda *s, dt=torch.float32: torch.zeros(s, dtype=dt, device="cuda")
    return z(rows, H, D, dt=torch.bfloat16), z(rows, H, D, dt=torch.bfloat16), z(H, rows)


def check_rows(m, tokens, positions_of_rows, O, seqs):
    """Row r of O (sequence seqs[r], position positions_of_rows[r]) against attention over the tokens the sequence holds."""
    for r, (s, p) in enumerate(zip(seqs, positions_of_rows)):
        t = np.array(tokens[s])
        x = f64(m.qkv[torch.from_numpy(t).cuda()]).reshape(len(t), H + 2 * HKV, D)
        q = fo.rotate(x[p:p + 1, :H], [p], m.freq)
        k, v = fo.rotate(x[:, H:H + HKV], np.arange(len(t)), m.freq), x[:, H + HKV:]
        want, _ = fo.paged_attn(q, k, v, D ** -0.5)
        spread, _ = fo.paged_attn(q, k, np.abs(v), D ** -0.5)
        # rotated queries and keys are rounded to bf16: logits are off by two half steps of the sum of their magnitudes
        kk = np.repeat(np.abs(k), H // HKV, axis=1)
        logit = np.einsum("hd,thd->th", np.abs(q[0]), kk).max(0) * D ** -0.5
        bound = (2 * 2 * BF16_HALF * logit + BF16_HALF)[:, None] * spread[0] + BF16_HALF * np.abs(want[0])
        assert (np.abs(f64(O)[r] - want[0]) <= bound).all(), (s, p)


@gpu
def test_prompts_then_one_token_at_a_time(ctx):
    m, rng = Model(3, 1), np.random.default_rng(1)
    tokens = [rng.integers(0, VOCAB, k).tolist() for k in (70, 1, 33)]
    lens = [len(t) for t in tokens]
    start = np.concatenate([[0], np.cumsum(lens)])
    flat = torch.tensor(sum(tokens, []), device="cuda")
    row_start = torch.tensor(start, dtype=torch.int32, device="cuda")
    m.kv_len.copy_(torch.tensor(lens, dtype=torch.int32))
    Q, O, lse = buffers(len(flat))
    m.layer(ctx, m.qkv[flat].reshape(len(flat), -1, D), Q, O, lse, row_start)            # a prompt's rows see the whole prompt
    seqs, pos = np.repeat(np.arange(3), lens), np.concatenate([np.arange(k) for k in lens])
    check_rows(m, tokens, pos, O, seqs)
    last = O[(row_start[1:] - 1).long()]

    i32 = dict(dtype=torch.int32, device="cuda")
    tok, conf, drawn = torch.zeros(3, **i32), torch.zeros(3, device="cuda"), torch.zeros(3, **i32)
    lp, ent, rank = torch.zeros(3, device="cuda"), torch.zeros(3, device="cuda"), torch.zeros(3, **i32)
    tt, tl, prob = torch.zeros((3, 4), **i32), torch.zeros((3, 4), device="cuda"), torch.zeros(3, device="cuda")
    Q1, O1, lse1 = buffers(3)
    for step in range(4):
        logits = (last.reshape(3, -1) @ m.head).contiguous()
        u = torch.rand(3, device="cuda")
        fb.focus_confidence(ctx, logits, fb.BF16, logits.stride(0), VOCAB, 0, 3, None, None, 3, conf, tok)
        fb.focus_sample(ctx, logits, fb.BF16, logits.stride(0), VOCAB, 0, 3, None, None, 3, 0.8, 20, 1.0, 0.0, u, conf, drawn, prob)
        fb.focus_token_logprobs(ctx, logits, fb.BF16, logits.stride(0), VOCAB, 0, 3, None, None, 3, 1.0, drawn, lp, rank, ent, 4, tt, tl)
        assert torch.equal(tt[:, 0], tok) and (rank >= 0).all() and (rank < 20).all()
        assert (lp.exp() / prob - 1).abs().max().item() < 1e-4                           # focus_sample's own temperature-1 probability
        x = f64(logits)
        for s in range(3):
            want = fo.token_logprobs(x[s, :VOCAB], 1.0, int(drawn[s]), 4)
            assert abs(lp[s].item() - want[0]) < 1e-4 and rank[s].item() == want[1] and tt[s].tolist() == want[3]
            tokens[s].append(int(drawn[s]))
        m.kv_len += 1
        m.layer(ctx, m.qkv[drawn.long()].reshape(3, -1, D), Q1, O1, lse1)
        check_rows(m, tokens, [len(t) - 1 for t in tokens], O1, range(3))
        last = O1
    assert ctx.poll_status() == 0


@gpu
def test_a_captured_step_decodes_as_the_eager_calls_do(ctx):
    """kv_len moves on inside the graph; each replay appends and attends one more token per sequence."""
    m, rng = Model(5, 2), np.random.default_rng(2)
    tokens = [rng.integers(0, VOCAB, k).tolist() for k in (3, 16, 31, 100, 7)]
    lens = [len(t) for t in tokens]
    row_start = torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device="cuda")
    m.kv_len.copy_(torch.tensor(lens, dtype=torch.int32))
    flat = torch.tensor(sum(tokens, []), device="cuda")
    Q, O, lse = buffers(len(flat))
    m.layer(ctx, m.qkv[flat].reshape(len(flat), -1, D), Q, O, lse, row_start)
    nxt = torch.zeros(5, dtype=torch.int64, device="cuda")
    x = torch.zeros(5, H + 2 * HKV, D, device="cuda").bfloat16()
    Q1, O1, lse1 = buffers(5)
    conf, tok = torch.zeros(5, device="cuda"), torch.zeros(5, dtype=torch.int32, device="cuda")

    def step():
        m.kv_len.add_(1)
        x.copy_(m.qkv[nxt].reshape(5, -1, D))
        m.layer(ctx, x, Q1, O1, lse1)
        logits = (O1.reshape(5, -1) @ m.head).contiguous()
        fb.focus_confidence(ctx, logits, fb.BF16, logits.stride(0), VOCAB, 0, 5, None, None, 5, conf, tok)
        nxt.copy_(tok)

    nxt.copy_(torch.tensor(rng.integers(0, VOCAB, 5)))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        fed = nxt.tolist()
        step()                                                               # eager, on the side stream: the first step
    torch.cuda.current_stream().wait_stream(side)
    for s in range(5):
        tokens[s].append(fed[s])
    check_rows(m, tokens, [len(t) - 1 for t in tokens], O1, range(5))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        step()
    for _ in range(6):
        fed = nxt.tolist()
        g.replay()
        for s in range(5):
            tokens[s].append(fed[s])
        check_rows(m, tokens, [len(t) - 1 for t in tokens], O1, range(5))
    assert m.kv_len.tolist() == [len(t) for t in tokens] and ctx.poll_status() == 0


@gpu
def test_windows_replaced_in_place(ctx):
    """A denoising step of several requests: the rows at listed positions get new tokens, their K/V replace the cached rows
    and they attend everything; enough rows that the tensor-core form with TMEM runs."""
    m, rng = Model(2, 3), np.random.default_rng(3)
    tokens = [rng.integers(0, VOCAB, k).tolist() for k in (150, 64)]
    lens = [len(t) for t in tokens]
    row_start = torch.tensor([0, 150, 214], dtype=torch.int32, device="cuda")
    m.kv_len.copy_(torch.tensor(lens, dtype=torch.int32))
    flat = torch.tensor(sum(tokens, []), device="cuda")
    Q, O, lse = buffers(214)
    m.layer(ctx, m.qkv[flat].reshape(214, -1, D), Q, O, lse, row_start)
    for step in range(3):
        pos = [np.sort(rng.choice(lens[s], k, replace=False)) for s, k in enumerate((19, 24))]
        new = [rng.integers(0, VOCAB, len(p)) for p in pos]
        for s in range(2):
            for p, t in zip(pos[s], new[s]):
                tokens[s][p] = int(t)
        rows = torch.tensor([0, 19, 43], dtype=torch.int32, device="cuda")
        flat_pos = torch.tensor(np.concatenate(pos), dtype=torch.int32, device="cuda")
        x = m.qkv[torch.tensor(np.concatenate(new), device="cuda")].reshape(43, -1, D)
        Q, O, lse = buffers(43)
        m.layer(ctx, x, Q, O, lse, rows, flat_pos)
        assert ctx.last_attn_variant() == 8
        check_rows(m, tokens, np.concatenate(pos), O, [0] * 19 + [1] * 24)
    assert ctx.poll_status() == 0


@gpu
def test_pages_give_what_the_contiguous_cache_gives(ctx):
    """focus_rotate + focus_update_kv + focus_dense_attn on one sequence: the same cached rows bit for bit, the same attention
    to rounding."""
    m, rng = Model(1, 4), np.random.default_rng(4)
    n = 130
    flat = torch.tensor(rng.integers(0, VOCAB, n), device="cuda")
    x = m.qkv[flat].reshape(n, -1, D)
    m.kv_len.fill_(n)
    Q, O, lse = buffers(n)
    m.layer(ctx, x, Q, O, lse, torch.tensor([0, n], dtype=torch.int32, device="cuda"))
    pos, cnt = torch.arange(n, dtype=torch.int32, device="cuda"), torch.tensor([n], dtype=torch.int32, device="cuda")
    turned = torch.zeros(n, H + HKV, D, device="cuda").bfloat16()                         # queries and keys in one call
    fb.focus_rotate(ctx, m.rope, 1, x, turned, fb.BF16, H + HKV, D, x.stride(0), x.stride(1), turned.stride(0), turned.stride(1), 0,
                    pos, cnt, n)
    shape = fb.make_shape(n, 0, H, HKV, D, 64, fb.BF16, q_stride_row=turned.stride(0))
    Kc, Vc = torch.zeros(HKV, n, D, device="cuda").bfloat16(), torch.zeros(HKV, n, D, device="cuda").bfloat16()
    fb.focus_update_kv(ctx, shape, Kc, Vc, turned[:, H:].contiguous(), x[:, H + HKV:].contiguous(), pos, cnt, n)
    O2, lse2 = torch.zeros(n, H, D, device="cuda").bfloat16(), torch.zeros(H, n, device="cuda")
    fb.focus_dense_attn(ctx, shape, turned, 0, n, None, None, 0, Kc, Vc, O2, lse2)
    pages = m.table[0].long()
    paged_k = m.K[pages].reshape(-1, HKV, D)[:n].transpose(0, 1)
    paged_v = m.V[pages].reshape(-1, HKV, D)[:n].transpose(0, 1)
    assert torch.equal(paged_k, Kc) and torch.equal(paged_v, Vc) and torch.equal(Q, turned[:, :H])
    # both round numerators and outputs to bf16: two half steps of each, of outputs below the largest value
    assert (O.float() - O2.float()).abs().max().item() <= 4 * BF16_HALF * x[:, H + HKV:].float().abs().max().item()
    assert (lse - lse2).abs().max().item() < 1e-3
    assert math.isfinite(float(O.float().sum())) and ctx.poll_status() == 0


@gpu
def test_the_readmes_paged_example_runs_as_printed(ctx):
    import os
    import re
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")).read()
    code = [c for c in re.findall(r"```python\n(.*?)```", text, flags=re.S) if "focus_paged_attn" in c][0]
    marker = "# ... page_table"
    head, tail = code.split(marker, 1)
    env = dict(torch=torch, fb=fb, ctx=ctx, H=8, Hkv=2, d=64, B=64, vocab=1000)
    exec(head, env)
    n, wide = env["n"], env["wide"]
    i32 = dict(dtype=torch.int32, device="cuda")
    env["page_table"] = torch.randperm(env["n_pages"], device="cuda")[:n * wide].int().reshape(n, wide)
    env["kv_len"] = torch.tensor([5, 1, 700], **i32)
    env["qkv"] = torch.randn(n, 12 * 64, device="cuda").bfloat16()
    env["logits"] = torch.randn(n, 1000, device="cuda").bfloat16()
    env["token"], env["rank"], env["top_token"] = (torch.zeros(n, **i32), torch.zeros(n, **i32), torch.zeros(n, 20, **i32))
    env["logprob"], env["entropy"], env["top_logprob"] = (torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda"),
                                                          torch.zeros(n, 20, device="cuda"))
    exec(tail.split("\n", 1)[1], env)
    v = env["qkv"].view(n, 12, 64)[1, 10:].repeat_interleave(4, 0)           # the second sequence's only token is the new one
    assert torch.equal(env["Op"][1], v) and (env["logprob"] < 0).all() and (env["top_token"] >= 0).all()
    assert ctx.poll_status() == 0


@gpu
def test_first_calls_of_a_context_may_be_captured(ctx):
    """A context whose calls have not run yet: append, both forms of attention and scores captured, then replayed."""
    m, fresh = Model(2, 6), fb.Context(0)
    m.kv_len.copy_(torch.tensor([100, 90], dtype=torch.int32))
    x = m.qkv[torch.arange(190, device="cuda")].reshape(190, -1, D)
    Q, O, lse = buffers(190)
    Q1, O1, lse1 = buffers(2)
    row_start = torch.tensor([0, 100, 190], dtype=torch.int32, device="cuda")
    lp, tok = torch.zeros(2, device="cuda"), torch.tensor([3, 4], dtype=torch.int32, device="cuda")
    logits = torch.randn(2, 1008, device="cuda").bfloat16()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        m.layer(fresh, x, Q, O, lse, row_start)
        assert fresh.last_attn_variant() == 8
        m.layer(fresh, x[99::90], Q1, O1, lse1)
        assert fresh.last_attn_variant() == 6
        fb.focus_token_logprobs(fresh, logits, fb.BF16, 1008, VOCAB, 0, 2, None, None, 2, 1.0, tok, lp)
    for _ in range(3):
        O.zero_(), O1.zero_(), lp.zero_()
        g.replay()
    seqs, pos = np.repeat([0, 1], (100, 90)), np.concatenate([np.arange(100), np.arange(90)])
    tokens = [list(range(100)), list(range(100, 190))]
    check_rows(m, tokens, pos, O, seqs)
    check_rows(m, tokens, [99, 89], O1, [0, 1])
    assert (lp < 0).all() and fresh.poll_status() == 0
    fresh.close()
