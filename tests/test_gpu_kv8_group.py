"""Attention of sequences that share the pages of a prompt, against the 64-bit
reference over each sequence's own view of the cache: groups of one sequence to
many, prompts of no page to thousands of tokens, contexts that end inside the
prompt, single tokens and ragged pieces, tables that differ where they are not
read, missing and NaN pages, rows of no sequence, streams and graphs.  The bounds of a
call follow its page table's width, which decides whether a group's pages are read once
for it or by each of its sequences: every test runs with the narrowest table, where the
second is right, and with two wide ones, of few and of many splits.

The bounds are those of the 8-bit cache's attention: a row's softmax is joined from
partial sums there too."""
import math

import numpy as np
import pytest

from tests import kv8_reference as R
from tests.test_gpu_kv8 import Dev, check_attention, offsets

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", params=[1, 512, 16384])
def env(request):
    import torch

    import paper_2607_26253_amd as sara
    assert torch.cuda.is_available(), "GPU tests need a HIP device"
    Batch.least = request.param
    return torch, sara


class Batch:
    """Sequences in groups over one cache.  shared[j]: tokens that group j has in common; ctx[i]: tokens of sequence i.  A
    sequence's own table holds other pages (or none) where its group's are read."""

    def __init__(self, env, rng, hkv, hd, fmt, members, shared, ctx, lone=0, spread=1.0):
        self.env, self.members, self.shared, self.ctx = env, members, shared, ctx
        n = sum(members) + lone                            # the last `lone` sequences are in no group
        assert len(ctx) == n and len(shared) == len(members)
        self.groups = offsets(members)
        self.width = max([self.least] + [-(-c // 16) for c in ctx] + [s // 16 for s in shared])
        group_of = np.repeat(np.arange(len(members)), members)
        count, rows = 0, []
        for i in range(n):
            common = shared[group_of[i]] // 16 if i < len(group_of) else 0
            if i < len(group_of) and i == self.groups[group_of[i]]:
                prompt = list(range(count, count + common))
                count += common
            own = max(0, -(-ctx[i] // 16) - common)
            rows.append(((prompt if common else []), list(range(count, count + own))))
            count += own
        total = count + 5
        order = rng.permutation(total)
        self.dev = Dev(env, total, hkv, hd, fmt)
        self.view = np.full((n, self.width), -1, np.int64)     # what each sequence sees
        self.tables = np.full((n, self.width), -1, np.int64)   # what the call is given
        for i, (a, b) in enumerate(rows):
            ids = order[a + b]
            self.view[i, :len(ids)] = self.tables[i, :len(ids)] = ids
            if i < len(group_of) and i != self.groups[group_of[i]] and len(a) and i % 2:
                self.tables[i, :len(a)] = rng.integers(-2, total, len(a))
        pages = order[:count]
        k, v = (self.dev.tensor(rng.standard_normal((16 * count, hkv, hd)) * np.exp2(rng.integers(-1, 2, (16 * count, 1, 1)) * spread),
                                env[0].float32) for _ in range(2))
        if count:
            self.dev.write(k, v, pages[None, :], [0], [0, 16 * count])

    def q(self, rng, rows, hq, dtype, size=2.0):
        td = self.env[0].bfloat16 if dtype == "bf16" else self.env[0].float32
        return self.dev.tensor(rng.standard_normal((rows, hq, self.dev.hd)) * size, td)

    def run(self, q, off=None, max_ctx=None, max_shared=None, scale=None, out=None, **kw):
        torch, sara = self.env
        i32 = self.dev.i32
        out = torch.full_like(q, 7.0) if out is None else out
        sara.sara_kv8_group_attention(q, *self.dev.args, i32(self.tables), i32(self.ctx), None if off is None else i32(off),
                                      i32(self.groups), i32(self.shared), out, scale=scale, max_ctx=max_ctx, max_shared=max_shared, **kw)
        return out

    def check(self, q, got, off=None, scale=None):
        check_attention(self.dev, q, got, self.view, self.ctx, off, scale)


HEADS = [(12, 2, 128), (16, 2, 128), (4, 4, 64), (5, 1, 64), (20, 1, 128), (9, 3, 64)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", ["int8", "fp8"])
@pytest.mark.parametrize("hq,hkv,hd", HEADS)
def test_single_tokens(env, hq, hkv, hd, fmt, dtype):
    """Prompts around pages; contexts of nothing, inside the prompt, at its end and behind it; a group of one and an empty
    one; sequences of no group."""
    rng = np.random.default_rng([hq, hkv, hd])
    members, shared = [8, 1, 0, 5, 3], [100, 33, 64, 15, 512]
    ctx = [101, 97, 96, 130, 0, 1, 95, 300, 40, 16, 17, 0, 3, 200, 513, 511, 700, 77, 0]
    b = Batch(env, rng, hkv, hd, fmt, members, shared, ctx, lone=2)
    q = b.q(rng, len(ctx), hq, dtype)
    got = b.run(q)
    b.check(q, got)
    assert bool((got[4] == 0).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", ["int8", "fp8"])
@pytest.mark.parametrize("hq,hkv,hd", HEADS)
def test_ragged_queries(env, hq, hkv, hd, fmt, dtype):
    """Pieces of none to many queries, some that begin inside the shared pages, one with more queries than tokens."""
    rng = np.random.default_rng([hq, hkv, hd, 1])
    members, shared = [4, 3, 1, 2], [200, 31, 160, 16]
    nq = [3, 0, 60, 20, 1, 33, 7, 129, 40, 2]
    ctx = [203, 210, 230, 150, 40, 33, 5, 289, 30, 18]
    b = Batch(env, rng, hkv, hd, fmt, members, shared, ctx)
    q = b.q(rng, sum(nq), hq, dtype)
    b.check(q, b.run(q, offsets(nq)), offsets(nq))


@pytest.mark.parametrize("ragged", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_long_prompts_and_long_answers(env, dtype, ragged):
    """Splits of the shared pages and of a sequence's own, and waves that join them."""
    rng = np.random.default_rng(5)
    members, shared = [3, 2], [5000, 700]
    nq = [2, 1, 40, 3, 1] if ragged else [1] * 5
    ctx = [5003, 8100, 5050, 703, 4000]
    b = Batch(env, rng, 2, 128, "int8", members, shared, ctx)
    q = b.q(rng, sum(nq), 4, dtype, 3.0)
    off = offsets(nq) if ragged else None
    b.check(q, b.run(q, off), off)


def test_many_groups_and_many_sequences(env):
    """More groups than a wave has lanes, and their results bit for bit in a call of the first few."""
    rng = np.random.default_rng(6)
    members = [int(m) for m in rng.choice([0, 1, 2, 5], 150)]
    shared = [int(s) for s in rng.integers(0, 90, 150)]
    ctx = [int(shared[g] + rng.integers(-20, 60)) for g, m in enumerate(members) for _ in range(m)]
    ctx = [max(0, c) for c in ctx]
    b = Batch(env, rng, 2, 128, "fp8", members, shared, ctx)
    q = b.q(rng, len(ctx), 12, "bf16")
    b.check(q, b.run(q))
    nq = [int(n) for n in rng.choice([0, 1, 2, 9], len(ctx))]
    qq = b.q(rng, sum(nq), 12, "bf16")
    b.check(qq, b.run(qq, offsets(nq)), offsets(nq))


@pytest.mark.parametrize("n,ragged", [(300, False), (140, True), (300, True)])
def test_many_sequences_and_long_answers(env, n, ragged):
    """Launches too large to run as one: rows that take the shared pages' results where they end, beside some whose own
    pages are several splits."""
    rng = np.random.default_rng([20, n])
    members = [5] * (n // 5)
    shared = [int(x) for x in rng.integers(30, 400, len(members))]
    ctx = [int(shared[i // 5] + x) for i, x in enumerate(rng.integers(0, 60, n))]
    for i in (3, 77, n - 1):
        ctx[i] = 8000 - i
    b = Batch(env, rng, 2, 64, "int8", members, shared, ctx)
    nq = [int(x) for x in rng.choice([0, 1, 2, 9], n)] if ragged else [1] * n
    if ragged:
        nq[3], nq[77], nq[78] = 3, 40, 30
    off = offsets(nq) if ragged else None
    q = b.q(rng, sum(nq), 8, "bf16")
    b.check(q, b.run(q, off), off)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_rows_of_one_long_prompt(env, dtype):
    """More splits of the shared pages than a row takes at its end."""
    rng = np.random.default_rng(21)
    ctx = [int(1500 + x) for x in rng.integers(-100, 100, 270)]
    b = Batch(env, rng, 2, 64, "fp8", [270], [1500], ctx)
    q = b.q(rng, 270, 8, dtype)
    b.check(q, b.run(q))


def test_bounds_of_the_launch(env):
    """max_shared below a prompt: the rest is each sequence's own.  max_ctx below a context: its rows are NaN, no other's."""
    rng = np.random.default_rng(7)
    b = Batch(env, rng, 2, 128, "int8", [4, 2], [300, 90], [310, 301, 330, 299, 100, 95])
    b.tables = b.view.copy()                               # every table holds its sequence's pages
    q = b.q(rng, 6, 8, "bf16")
    for most in (0, 15, 16, 100, 288, 300, 320):
        b.check(q, b.run(q, max_shared=most))
    got = b.run(q, max_ctx=310)
    assert bool(got[2].isnan().all())
    keep = [0, 1, 3, 4, 5]
    assert not bool(got[keep].isnan().any())
    nq = [2, 0, 30, 1, 5, 50]
    qq = b.q(rng, sum(nq), 8, "bf16")
    got = b.run(qq, offsets(nq), max_ctx=310)
    assert bool(got[2:32].isnan().all()) and not bool(got[:2].isnan().any()) and not bool(got[32:].isnan().any())


@pytest.mark.parametrize("ragged", [False, True])
def test_missing_pages_are_not_seen(env, ragged):
    torch = env[0]
    rng = np.random.default_rng(8)
    ctx = [150, 140, 200, 70, 64, 66]
    b = Batch(env, rng, 2, 64, "int8", [3, 3], [128, 64], ctx)
    first = b.groups[1]
    b.tables[0, 1:3] = -1                                  # of the first group's prompt
    b.view[:3, 1:3] = -1
    b.tables[2, 9] = b.dev.n_pages                         # of a sequence's own
    b.view[2, 9] = -1
    b.tables[first, :4] = -5                               # the second prompt has no page at all
    b.view[first:, :4] = -1
    nq = [1, 5, 40, 3, 1, 9] if ragged else [1] * 6
    off = offsets(nq) if ragged else None
    q = b.q(rng, sum(nq), 4, "bf16")
    got = b.run(q, off)
    b.check(q, got, off)
    if not ragged:
        assert bool((got[4] == 0).all())                   # 64 tokens, all of them in missing pages


@pytest.mark.parametrize("fmt", ["int8", "fp8"])
@pytest.mark.parametrize("ragged", [False, True])
def test_a_nan_page_reaches_only_who_sees_it(env, fmt, ragged):
    torch = env[0]
    rng = np.random.default_rng(9)
    ctx = [100, 90, 64, 50, 80, 70]
    b = Batch(env, rng, 2, 64, fmt, [4, 2], [64, 48], ctx)
    bad, good = np.ones((1, 2, 64)), np.ones((1, 2, 64))
    bad[0, 1, 3] = np.nan
    # position 60 of the first prompt (head 1), which the contexts of 50 do not see
    b.dev.write(b.dev.tensor(bad, torch.float32), b.dev.tensor(good, torch.float32), b.view[:1], [60], [0, 1])
    nq = [3, 1, 4, 2, 1, 1] if ragged else [1] * 6
    off = offsets(nq) if ragged else None
    q = b.q(rng, sum(nq), 4, "bf16")
    got = b.run(q, off)
    b.check(q, got, off)
    assert bool(got.isnan().any()) and not bool(got[:, :2].isnan().any())


def test_rows_of_no_sequence_strides_and_streams(env):
    """Rows before the first sequence and behind the last stay as they are; q and out are parts of wider tensors."""
    torch, sara = env
    rng = np.random.default_rng(10)
    b = Batch(env, rng, 2, 128, "int8", [2, 3], [80, 40], [81, 90, 41, 77, 50])
    nq = [1, 2, 40, 3, 1]
    off = [o + 3 for o in offsets(nq)]
    rows = off[-1] + 4
    wide = b.q(rng, rows, 20, "bf16")
    q = wide[:, 4:12]
    out = torch.full((rows, 9, 144), 7.0, device="cuda", dtype=torch.bfloat16)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    b.run(q, off, out=out[:, 1:, 8:136], stream=side)
    side.synchronize()
    assert bool((out[:3] == 7).all()) and bool((out[off[-1]:] == 7).all()) and bool((out[:, 0] == 7).all())
    assert bool((out[:, :, :8] == 7).all()) and bool((out[:, :, 136:] == 7).all())
    check_attention(b.dev, q[3:off[-1]], out[3:off[-1], 1:, 8:136], b.view, b.ctx, offsets(nq))


def test_without_groups_it_is_the_plain_call(env):
    torch, sara = env
    rng = np.random.default_rng(11)
    ctx = [0, 1, 40, 700, 16]
    b = Batch(env, rng, 2, 128, "fp8", [], [], ctx, lone=5)
    q = b.q(rng, 5, 8, "f32")
    b.check(q, b.run(q))
    b.check(q, b.run(q, max_shared=0))
    out = torch.empty_like(q)
    i32 = b.dev.i32
    sara.sara_kv8_attention(q, *b.dev.args, i32(b.tables), i32(ctx), None, out)
    assert bool(((out - b.run(q)).abs() <= 2.0 ** -17 * out.abs().amax()).all())


def test_large_scores_and_scale(env):
    rng = np.random.default_rng(12)
    for scale in (-0.3, 0.0, 4.0):
        b = Batch(env, rng, 2, 64, "int8", [3], [70], [80, 71, 90], spread=3.0)
        q = b.q(rng, 3, 4, "f32", 4.0)
        b.check(q, b.run(q, scale=scale), scale=scale)


def test_a_cache_past_32_bits(env):
    """Pages whose codes lie past 2^32 bytes."""
    torch, sara = env
    hkv, hd, n = 8, 128, 300000
    dt = torch.int8
    codes = [torch.zeros((n, hkv, 16, hd), dtype=dt, device="cuda") for _ in range(2)]
    exps = [torch.full((n, hkv), 121, dtype=torch.uint8, device="cuda") for _ in range(2)]
    g = torch.Generator(device="cuda").manual_seed(5)
    use = torch.tensor([299999, 270001, 5, 299998], device="cuda")
    for c in codes:
        c[use] = torch.randint(-60, 60, (4, hkv, 16, hd), generator=g, device="cuda", dtype=dt)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    tables = i32([[299999, 270001, 5], [299999, 270001, 299998]])
    q = torch.randn((2, hkv, hd), generator=g, device="cuda")
    out = torch.empty_like(q)
    sara.sara_kv8_group_attention(q, *codes, *exps, tables, i32([40, 47]), None, i32([0, 2]), i32([32]), out)
    for i, n_tok in ((0, 40), (1, 47)):
        k, v = (c[tables[i].long()].double().transpose(0, 1).reshape(hkv, 48, hd)[:, :n_tok] / 64 for c in codes)
        p = torch.softmax((k @ q[i].double()[:, :, None])[..., 0] / math.sqrt(hd), -1)
        want = (p[:, None] @ v)[:, 0]
        assert float((out[i].double() - want).abs().max()) <= 1e-5


def test_graph_replay(env):
    """A captured call replayed on other queries, contexts and prompts, with eager calls of another shape between."""
    torch, sara = env
    rng = np.random.default_rng(13)
    b = Batch(env, rng, 2, 128, "int8", [4, 4], [200, 64], [210, 201, 333, 250, 70, 65, 90, 100])
    other = Batch(env, rng, 2, 128, "int8", [2], [100], [110, 500])
    need = sara.ctypes.c_int64(0)
    most = 16 * b.width
    assert sara._lib.sara_kv8_group_attention_workspace(2, 128, 8, 12, 8, 2, 0, most, most, 1, sara.ctypes.byref(need)) == 0
    assert need.value > 0 or b.least == 1
    ws = torch.full((need.value,), 255, device="cuda", dtype=torch.uint8) if need.value else None
    qs = [b.q(rng, 8, 12, "bf16") for _ in range(3)]
    ctxs = [[210, 201, 333, 250, 70, 65, 90, 100], [0, 201, 208, 30, 64, 63, 1, 100], [300, 2, 333, 200, 90, 66, 70, 65]]
    eager = []
    i32 = b.dev.i32
    for q, ctx in zip(qs, ctxs):
        out = torch.empty_like(q)
        sara.sara_kv8_group_attention(q, *b.dev.args, i32(b.tables), i32(ctx), None, i32(b.groups), i32(b.shared), out, max_ctx=most,
                                      max_shared=most)
        check_attention(b.dev, q, out, b.view, ctx, None)
        eager.append(out)
    q, ctx, out = qs[0].clone(), i32(ctxs[0]), torch.empty_like(qs[0])
    fixed = (i32(b.tables), i32(b.groups), i32(b.shared))
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        sara.sara_kv8_group_attention(q, *b.dev.args, fixed[0], ctx, None, fixed[1], fixed[2], out, max_ctx=most, max_shared=most,
                                      workspace=ws)
    qo = other.q(rng, 2, 12, "bf16")
    for i in (1, 2, 0, 1):
        q.copy_(qs[i])
        ctx.copy_(i32(ctxs[i]))
        if ws is not None:
            ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager[i]), i
        other.check(qo, other.run(qo))
    if ws is None:
        return
    with pytest.raises(sara.SaraError, match="workspace"):
        sara.sara_kv8_group_attention(q, *b.dev.args, fixed[0], ctx, None, fixed[1], fixed[2], out, max_ctx=most, max_shared=most,
                                      workspace=ws[:-16])


def test_refusals(env):
    torch, sara = env
    rng = np.random.default_rng(14)
    b = Batch(env, rng, 2, 64, "int8", [2, 1], [32, 16], [40, 33, 20])
    q = b.q(rng, 3, 4, "bf16")
    i32 = b.dev.i32
    base = dict(q=q, pages=i32(b.tables), ctx=i32(b.ctx), off=None, groups=i32(b.groups), shared=i32(b.shared), out=torch.empty_like(q))

    def call(max_ctx=None, max_shared=None, scale=None, **kw):
        y = dict(base, **kw)
        sara.sara_kv8_group_attention(y["q"], *b.dev.args, y["pages"], y["ctx"], y["off"], y["groups"], y["shared"], y["out"],
                                      scale=scale, max_ctx=max_ctx, max_shared=max_shared)

    call()
    for kw, exc in ((dict(q=q.half()), TypeError), (dict(out=q.float()), ValueError), (dict(q=q[:2]), ValueError),
                    (dict(groups=i32([0, 3])), ValueError), (dict(groups=i32(b.groups).long()), ValueError), (dict(groups=None), TypeError),
                    (dict(shared=i32(b.shared).cpu()), ValueError), (dict(shared=i32([[32], [16]])), ValueError),
                    (dict(max_ctx=16 * b.width + 1), sara.SaraError), (dict(max_shared=-1), sara.SaraError),
                    (dict(max_shared=16 * b.width + 1), sara.SaraError), (dict(max_shared=2 ** 31), ValueError),
                    (dict(scale=math.inf), sara.SaraError), (dict(out=torch.empty((3, 1, 64), device="cuda", dtype=q.dtype).expand(3, 4, 64)),
                                                             sara.SaraError)):
        with pytest.raises(exc):
            call(**kw)


def test_no_rows(env):
    torch, sara = env
    rng = np.random.default_rng(15)
    b = Batch(env, rng, 2, 64, "int8", [2], [32], [40, 33])
    q = b.q(rng, 0, 4, "bf16")
    assert b.run(q, [0, 0, 0]).shape == (0, 4, 64)


@pytest.fixture(scope="module")
def device():
    import torch

    import paper_2607_26253_amd as sara
    return torch, sara


@pytest.mark.parametrize("ragged", [False, True])
@pytest.mark.parametrize("groups,max_shared,max_ctx", [(120, 128, 384), (600, 512, 576)])
def test_the_first_groups_in_a_call_of_their_own(device, groups, max_shared, max_ctx, ragged):
    """Half of the groups, called alone, give the same results bit for bit: by each sequence through its group's table (the
    first size) and with the shared pages apart (the second); contexts of one split in either call."""
    torch, sara = device
    rng = np.random.default_rng([groups, ragged])
    hkv, hd, hq, members, pages = 2, 128, 12, 5, 4000
    n = groups * members
    g = torch.Generator(device="cuda").manual_seed(groups)
    codes = [torch.randint(-90, 91, (pages, hkv, 16, hd), generator=g, device="cuda", dtype=torch.int8) for _ in range(2)]
    exps = [torch.randint(119, 123, (pages, hkv), generator=g, device="cuda", dtype=torch.uint8) for _ in range(2)]
    i32 = lambda x: torch.tensor(np.asarray(x, np.int32), device="cuda")
    table = rng.integers(0, pages, (n, max_ctx // 16))
    shared = rng.integers(0, max_shared + 1, groups)
    ctx = np.clip(np.repeat(shared, members) + rng.integers(-20, 60, n), 0, max_ctx)
    off = offsets([int(x) for x in rng.choice([0, 1, 2, 9], n)]) if ragged else list(range(n + 1))
    q = torch.randn((off[-1], hq, hd), generator=g, device="cuda").bfloat16()

    def call(k):
        m = k * members
        out = torch.full((off[m], hq, hd), 7.0, device="cuda", dtype=q.dtype)
        sara.sara_kv8_group_attention(q[:off[m]], *codes, *exps, i32(table[:m]), i32(ctx[:m]), i32(off[:m + 1]) if ragged else None,
                                      i32(range(0, m + 1, members)), i32(shared[:k]), out, max_ctx=max_ctx, max_shared=max_shared)
        return out

    whole, half = call(groups), call(groups // 2)
    assert torch.equal(whole[:half.shape[0]], half)
    assert not bool(whole.isnan().any()) and float(whole.float().abs().amax()) > 0.1
