"""The 8-bit KV cache against a 64-bit reference: writes and reads are exact;
attention over lengths from none to thousands, ragged queries, missing pages,
stale and NaN pages, strides, streams and large caches."""
import numpy as np
import pytest

from tests import kv8_reference as R

pytestmark = pytest.mark.gpu

SHAPES = [(2, 128), (1, 128), (4, 64), (3, 64)]


@pytest.fixture(scope="module")
def env():
    import torch

    import paper_2607_26253_amd as sara
    assert torch.cuda.is_available(), "GPU tests need a HIP device"
    return torch, sara


class Dev:
    """A cache on the device, every byte preset to a pattern that reads as a stale page."""

    def __init__(self, env, n_pages, hkv, hd, fmt, fill=0x7F):
        self.torch, self.sara = env
        torch = self.torch
        dt = torch.int8 if fmt == "int8" else torch.float8_e4m3fn
        self.fmt, self.hkv, self.hd, self.n_pages = fmt, hkv, hd, n_pages
        self.raw = [torch.full((n_pages, hkv, 16, hd), fill, dtype=torch.uint8, device="cuda") for _ in range(2)]
        self.exp = [torch.full((n_pages, hkv), 130, dtype=torch.uint8, device="cuda") for _ in range(2)]
        self.codes = [x.view(dt) for x in self.raw]
        self.ref = [R.Cache(n_pages, hkv, hd, fmt) for _ in range(2)]
        for c in self.ref:
            c.exp[:] = 130

    @property
    def args(self):
        return (*self.codes, *self.exp)

    def i32(self, x):
        return self.torch.tensor(np.asarray(x, np.int32), device="cuda")

    def tensor(self, x, dtype):
        return self.torch.tensor(np.asarray(x, np.float32), device="cuda").to(dtype)

    def write(self, k, v, tables, start, off):
        """k, v: device tensors [rows][hkv][hd]; also into the reference."""
        self.sara.sara_kv8_write(*self.args, k, v, self.i32(tables), self.i32(start), None if off is None else self.i32(off))
        off = range(len(tables) + 1) if off is None else off
        for c, x in zip(self.ref, (k, v)):
            x = x.double().cpu().numpy()
            for i in range(len(tables)):
                if start[i] >= 0 and off[i + 1] > off[i]:
                    c.write(x[off[i]:off[i + 1]], tables[i], start[i])

    def read(self, tables, start, off, dtype):
        torch = self.torch
        out = [torch.full((off[-1], self.hkv, self.hd), 7.0, dtype=dtype, device="cuda") for _ in range(2)]
        self.sara.sara_kv8_read(*self.args, self.i32(tables), self.i32(start), self.i32(off), *out)
        return [x.double().cpu().numpy() for x in out]

    def check(self, tables, start, off, dtype):
        got = self.read(tables, start, off, dtype)
        for c, x in zip(self.ref, got):
            want = np.concatenate([c.read(tables[i], start[i], off[i + 1] - off[i]) for i in range(len(tables))])
            with np.errstate(over="ignore"):       # a code may round past the largest finite number
                np.testing.assert_array_equal(x, want.astype(np.float32))


def make_tables(rng, lengths, width, n_pages):
    order = rng.permutation(n_pages)
    out, at = np.full((len(lengths), width), -1, np.int64), 0
    for i, n in enumerate(lengths):
        c = -(-n // 16)
        out[i, :c] = order[at:at + c]
        at += c
    return out


def offsets(n):
    return [0] + list(np.cumsum(n))


def rows(dev, rng, n, dtype, spread=2.0):
    """Rows whose size varies by orders of magnitude from token to token, so that scales grow and pages differ."""
    x = rng.standard_normal((n, dev.hkv, dev.hd)) * np.exp2(rng.integers(-6, 6, (n, 1, 1)) * spread / 2)
    return dev.tensor(x, dev.torch.bfloat16 if dtype == "bf16" else dev.torch.float32)


# -- write and read -----------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", ["int8", "fp8"])
@pytest.mark.parametrize("hkv,hd", SHAPES)
def test_write_then_read_is_exact(env, hkv, hd, fmt, dtype):
    rng = np.random.default_rng([hkv, hd, len(fmt), len(dtype)])
    first = [0, 1, 15, 16, 17, 33, 100, 5]        # tokens of the first call (one sequence gets none)
    then = [3, 15, 1, 0, 31, 16, 40, 12]          # appended by the second, most of them inside a page
    ends = [a + b for a, b in zip(first, then)]
    dev = Dev(env, 64, hkv, hd, fmt)
    tables = make_tables(rng, ends, 9, 64)
    td = env[0].bfloat16 if dtype == "bf16" else env[0].float32
    dev.write(rows(dev, rng, sum(first), dtype), rows(dev, rng, sum(first), dtype), tables, [0] * 8, offsets(first))
    dev.check(tables, [0] * 8, offsets(first), td)
    dev.write(rows(dev, rng, sum(then), dtype), rows(dev, rng, sum(then), dtype), tables, first, offsets(then))
    dev.check(tables, [0] * 8, offsets(ends), td)
    dev.check(tables, [e // 2 for e in ends], offsets([e - e // 2 for e in ends]), env[0].float32)
    for _ in range(20):                            # single tokens without offsets, over pages' ends and one table's
        need = np.arange(9) < -(-(np.array(ends)[:, None] + 1) // 16)
        tables = np.where(need & (tables < 0), np.setdiff1d(np.arange(64), tables)[:8, None], tables)
        dev.write(rows(dev, rng, 8, dtype), rows(dev, rng, 8, dtype), tables, ends, None)
        ends = [e + 1 for e in ends]
    dev.check(tables, [0] * 8, offsets(ends), td)


@pytest.mark.parametrize("fmt", ["int8", "fp8"])
def test_codes_at_every_rounding(env, fmt):
    """Every bf16 magnitude under the page's largest, its ties among them, and pages of zeros, of subnormals and of the
    largest finite values."""
    dev = Dev(env, 40, 1, 128, fmt)
    top = R.TOP[fmt]
    vals = np.concatenate([np.arange(2032) / 16.0, -np.arange(2032) / 16.0])           # halves of int8 steps
    vals = vals[np.abs(vals) <= top]
    vals = np.resize(vals, (16 * 16, 1, 128))
    vals[::16, 0, 0] = top
    rest = np.zeros((16 * 8, 1, 128))
    rest[16:32] = 1e-40 * np.arange(128)
    rest[32:48, 0, 0] = 3.3e38
    rest[48:64, 0, 5] = top * np.nextafter(np.float32(1), np.float32(2))               # just above what a scale holds
    rest[64:80, 0, 5] = top
    rest[80:96] = 2.0 ** -126
    rest[96:112, 0, ::2] = -0.0
    x = dev.tensor(np.concatenate([vals, rest]), env[0].float32)
    tables = np.arange(24)[None, :]
    dev.write(x, -x, tables, [0], [0, len(x)])
    dev.check(tables, [0], [0, len(x)], env[0].float32)


def test_not_finite_rows_and_missing_pages(env):
    torch = env[0]
    for fmt in ("int8", "fp8"):
        dev = Dev(env, 8, 2, 64, fmt, fill=0)
        x = np.random.default_rng(3).standard_normal((40, 2, 64))
        x[20, 1, 7] = np.nan
        k = dev.tensor(x, torch.float32)
        x[20, 1, 7], x[3, 0, 0] = 1.0, -np.inf
        v = dev.tensor(x, torch.float32)
        tables = np.array([[3, 5, -1], [8, 6, 2 ** 30]])                               # ids without a page
        dev.write(k, v, tables, [4, 16], [0, 20, 40])
        dev.check(tables, [4, 10], [0, 70, 130], torch.bfloat16)                       # past the tables too
        ones = dev.tensor(np.ones((40, 2, 64)), torch.float32)
        dev.write(ones[:3], ones[:3], tables, [10, 20], [0, 2, 3])                     # inside pages that are NaN: they stay so
        dev.check(tables, [4, 10], [0, 70, 130], torch.float32)
        dev.write(ones[:20], ones[:20], tables, [-3, -40], [0, 10, 20])                # dropped
        dev.write(ones[:16], ones[:16], tables[:1], [0], [0, 16])                      # written from its first token: clean again
        dev.check(tables, [0, 10], [0, 70, 130], torch.float32)


def test_strided_rows_leave_the_rest_alone(env):
    torch, sara = env
    dev = Dev(env, 16, 2, 128, "int8")
    rng = np.random.default_rng(5)
    fused = dev.tensor(rng.standard_normal((50, 3, 2, 128)), torch.bfloat16)            # q | k | v of one projection
    tables = make_tables(rng, [50], 6, 16)
    dev.write(fused[:, 1], fused[:, 2], tables, [0], [0, 50])
    out = torch.full((2, 50, 5, 128), 9.0, dtype=torch.bfloat16, device="cuda")         # heads 1 and 3 of a wider tensor
    sara.sara_kv8_read(*dev.args, dev.i32(tables), dev.i32([0]), dev.i32([0, 50]), out[0, :, 1:4:2], out[1, :, 1:4:2])
    got = out.float().cpu().numpy()
    for i in range(2):
        np.testing.assert_array_equal(got[i, :, 1:4:2], dev.ref[i].read(tables[0], 0, 50))
    assert np.all(got[:, :, ::2] == 9.0)


# -- attention ----------------------------------------------------------------------
def attend(dev, q, tables, ctx, off, max_ctx=None, scale=None, out=None, **kw):
    torch, sara = dev.torch, dev.sara
    if out is None:
        out = torch.full_like(q, 5.0)
    sara.sara_kv8_attention(q, *dev.args, dev.i32(tables), dev.i32(ctx), None if off is None else dev.i32(off), out,
                            scale=scale, max_ctx=max_ctx, **kw)
    return out


def check_attention(dev, q, got, tables, ctx, off, scale=None):
    """Bound of |out - exact|, with S the largest |score| in base 2, D = 2^-22 S + 2^-20 the relative error of a weight
    (scores and sums are fp32) plus 2^-17 for the two bf16 parts of a weight of bf16 queries (three parts: 2^-24):
    2 D max|v|, and the rounding of bf16 outputs."""
    hd, bf16 = dev.hd, q.dtype == dev.torch.bfloat16
    scale = hd ** -0.5 if scale is None else scale
    qn, got = q.double().cpu().numpy(), got.double().cpu().numpy()
    off = range(len(tables) + 1) if off is None else off
    for i in range(len(tables)):
        n = off[i + 1] - off[i]
        if n == 0:
            continue
        end = max(ctx[i], 0)
        k, v = (c.read(tables[i], 0, end) for c in dev.ref)
        present = np.array([0 <= tables[i][p // 16] < dev.n_pages for p in range(end)], bool)
        want = R.attention(qn[off[i]:off[i + 1]], k, v, present, end, scale)
        have = got[off[i]:off[i + 1]]
        np.testing.assert_array_equal(np.isnan(have), np.isnan(want))
        smax = 0.0
        for h in range(q.shape[1]):
            if end:
                kk = np.nan_to_num(k[:, h // (q.shape[1] // dev.hkv)])
                smax = max(smax, np.max(np.abs(kk) @ np.abs(qn[off[i]:off[i + 1], h].T)) * abs(scale) * 1.4427)
        d = smax * 2.0 ** -22 + 2.0 ** -20 + (2.0 ** -17 if bf16 else 2.0 ** -24)
        vmax = np.nanmax(np.abs(v)) if v.size and not np.all(np.isnan(v)) else 0.0
        bound = 2 * d * vmax + (2.0 ** -8 * np.abs(want) if bf16 else 2.0 ** -23 * np.abs(want))
        ok = np.abs(have - want) <= bound
        assert np.all(ok | np.isnan(want)), (i, float(np.nanmax(np.abs(have - want))), float(np.nanmax(np.abs(have - want) / np.maximum(bound, 1e-300))))


def filled(env, rng, hkv, hd, fmt, lengths, width=None, spread=1.0, extra=4):
    total = sum(-(-n // 16) for n in lengths)
    dev = Dev(env, total + extra, hkv, hd, fmt)
    tables = make_tables(rng, lengths, width or max(1, max(-(-n // 16) for n in lengths)), total + extra)
    n = sum(lengths)
    if n:
        k, v = (dev.tensor(rng.standard_normal((n, hkv, hd)) * np.exp2(rng.integers(-1, 2, (n, 1, 1)) * spread),
                           env[0].float32) for _ in range(2))
        dev.write(k, v, tables, [0] * len(lengths), offsets(lengths))
    return dev, tables


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", ["int8", "fp8"])
@pytest.mark.parametrize("hq,hkv,hd", [(12, 2, 128), (16, 2, 128), (4, 4, 64), (5, 1, 64), (20, 1, 128), (9, 3, 64)])
def test_single_tokens(env, hq, hkv, hd, fmt, dtype):
    """One query a sequence, contexts of no token, one, and around pages and splits."""
    rng = np.random.default_rng([hq, hkv, hd])
    ctx = [0, 1, 2, 15, 16, 17, 31, 33, 127, 128, 129, 300, 513]
    dev, tables = filled(env, rng, hkv, hd, fmt, ctx)
    q = dev.tensor(rng.standard_normal((len(ctx), hq, hd)) * 2, env[0].bfloat16 if dtype == "bf16" else env[0].float32)
    got = attend(dev, q, tables, ctx, None)
    check_attention(dev, q, got, tables, ctx, None)
    assert np.all(got[0].float().cpu().numpy() == 0.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", ["int8", "fp8"])
@pytest.mark.parametrize("hq,hkv,hd", [(12, 2, 128), (16, 2, 128), (4, 4, 64), (20, 1, 64), (7, 7, 128)])
def test_ragged_queries(env, hq, hkv, hd, fmt, dtype):
    """Several queries a sequence, none for some, more than there are tokens for one (its first rows see nothing)."""
    rng = np.random.default_rng([hq, hkv, hd, 1])
    nq = [1, 0, 5, 16, 33, 70, 1, 20, 129, 0, 64]
    ctx = [1, 9, 5, 100, 33, 90, 400, 12, 300, 0, 64]
    dev, tables = filled(env, rng, hkv, hd, fmt, ctx)
    q = dev.tensor(rng.standard_normal((sum(nq), hq, hd)) * 2, env[0].bfloat16 if dtype == "bf16" else env[0].float32)
    got = attend(dev, q, tables, ctx, offsets(nq))
    check_attention(dev, q, got, tables, ctx, offsets(nq))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,hd", [(12, 2, 128), (4, 4, 64)])
def test_ragged_queries_of_many_sequences(env, hq, hkv, hd, dtype):
    """300 sequences of no query to 40, with keys for some queries only: right, and the same bits in a call of ten."""
    rng = np.random.default_rng([hq, hkv, hd, 2])
    nq = [int(n) for n in rng.choice([0, 1, 2, 5, 40], 300, p=[0.1, 0.5, 0.2, 0.1, 0.1])]
    ctx = [max(0, n + int(rng.integers(-2, 60))) for n in nq]
    dev, tables = filled(env, rng, hkv, hd, "int8", ctx)
    off = offsets(nq)
    q = dev.tensor(rng.standard_normal((sum(nq), hq, hd)) * 2, env[0].bfloat16 if dtype == "bf16" else env[0].float32)
    got = attend(dev, q, tables, ctx, off)
    check_attention(dev, q, got, tables, ctx, off)
    few = attend(dev, q[:off[10]], tables[:10], ctx[:10], off[:11])
    assert env[0].equal(few, got[:off[10]])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_long_contexts_join_their_splits(env, dtype):
    rng = np.random.default_rng(11)
    ctx = [3000, 1, 777, 2049]
    dev, tables = filled(env, rng, 2, 128, "int8", ctx)
    td = env[0].bfloat16 if dtype == "bf16" else env[0].float32
    q = dev.tensor(rng.standard_normal((4, 4, 128)) * 3, td)
    check_attention(dev, q, attend(dev, q, tables, ctx, None), tables, ctx, None)
    nq = [2, 1, 40, 3]
    q = dev.tensor(rng.standard_normal((sum(nq), 4, 128)) * 3, td)
    check_attention(dev, q, attend(dev, q, tables, ctx, offsets(nq)), tables, ctx, offsets(nq))


def test_missing_pages_are_not_seen(env):
    """Pages dropped from a table (the first ones, one in the middle, all), ids that are no page, and a launch sized for
    shorter contexts than a sequence has."""
    torch = env[0]
    rng = np.random.default_rng(12)
    ctx = [200, 100, 64, 700]
    dev, tables = filled(env, rng, 2, 128, "fp8", ctx, width=50)
    tables[0, :5] = -1
    tables[1, 3] = dev.n_pages + 5
    tables[2] = -1
    tables[3, 10:30] = -7
    q = dev.tensor(rng.standard_normal((4, 8, 128)), torch.bfloat16)
    got = attend(dev, q, tables, ctx, None)
    check_attention(dev, q, got, tables, ctx, None)
    assert np.all(got[2].float().cpu().numpy() == 0.0)
    nq = [30, 2, 64, 600]
    qq = dev.tensor(rng.standard_normal((sum(nq), 8, 128)), torch.bfloat16)
    check_attention(dev, qq, attend(dev, qq, tables, ctx, offsets(nq)), tables, ctx, offsets(nq))
    short = attend(dev, q, tables, ctx, None, max_ctx=200)
    assert bool(short[3].isnan().all())
    check_attention(dev, q[:3], short[:3], tables[:3], ctx[:3], None)
    short = attend(dev, qq, tables, ctx, offsets(nq), max_ctx=650).float().cpu().numpy()
    assert np.all(np.isnan(short[96:])) and not np.any(np.isnan(short[:96]))


@pytest.mark.parametrize("fmt", ["int8", "fp8"])
def test_a_nan_page_reaches_only_who_sees_it(env, fmt):
    torch = env[0]
    rng = np.random.default_rng(13)
    dev, tables = filled(env, rng, 2, 64, fmt, [160, 160])
    bad = np.ones((1, 2, 64))
    bad[0, 1, 3] = np.nan                                                            # head 1 of position 100
    good = np.ones((1, 2, 64))
    dev.write(dev.tensor(bad, torch.float32), dev.tensor(good, torch.float32), tables[:1], [100], [0, 1])
    dev.write(dev.tensor(good, torch.float32), dev.tensor(bad, torch.float32), tables[1:], [100], [0, 1])
    nq = [160, 160]
    q = dev.tensor(rng.standard_normal((320, 4, 64)), torch.bfloat16)
    got = attend(dev, q, tables, [160, 160], offsets(nq))
    check_attention(dev, q, got, tables, [160, 160], offsets(nq))
    assert np.isnan(got.float().cpu().numpy()).any() and not np.isnan(got[:, :2].float().cpu().numpy()).any()


def test_large_scores_and_page_scales(env):
    """One key far above the rest, pages whose scales are 2^40 apart, and a scale below 0."""
    torch = env[0]
    rng = np.random.default_rng(14)
    for fmt in ("int8", "fp8"):
        dev = Dev(env, 40, 1, 128, fmt)
        tables = make_tables(rng, [512], 32, 40)
        page_size = np.exp2(rng.integers(-20, 20, 32)).repeat(16)[:, None, None]
        k = rng.standard_normal((512, 1, 128)) * np.where(np.arange(512) == 300, 12.0, 1.0)[:, None, None]
        dev.write(dev.tensor(k, torch.float32), dev.tensor(rng.standard_normal((512, 1, 128)) * page_size, torch.float32),
                  tables, [0], [0, 512])
        q = dev.tensor(rng.standard_normal((1, 4, 128)), torch.bfloat16)
        for scale in (None, -0.2, 1.0):
            check_attention(dev, q, attend(dev, q, tables, [512], None, scale=scale), tables, [512], None, scale)


def test_strides_streams_shared_pages_and_workspace(env):
    torch = env[0]
    rng = np.random.default_rng(15)
    ctx = [600, 600, 350]
    dev, tables = filled(env, rng, 2, 128, "int8", ctx)
    tables[1, :20] = tables[0, :20]                                                   # 320 tokens of a common prompt
    fused = dev.tensor(rng.standard_normal((3, 16, 128)), torch.bfloat16)
    q = fused[:, 2:14]                                                                # 12 heads of a wider projection
    want = attend(dev, q.contiguous(), tables, ctx, None)
    check_attention(dev, q, want, tables, ctx, None)
    wide = torch.full((3, 20, 128), 4.0, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(1 << 22, dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    attend(dev, q, tables, ctx, None, out=wide[:, 4:16], workspace=ws, stream=side)
    side.synchronize()
    assert torch.equal(wide[:, 4:16], want)
    assert bool((wide[:, :4] == 4.0).all()) and bool((wide[:, 16:] == 4.0).all())


def test_results_do_not_depend_on_the_batch(env):
    """The same sequence alone and among others, and run again: bit for bit."""
    torch = env[0]
    rng = np.random.default_rng(16)
    ctx = [900, 40, 333]
    dev, tables = filled(env, rng, 2, 128, "fp8", ctx)
    q = dev.tensor(rng.standard_normal((3, 12, 128)), torch.bfloat16)
    one, two = attend(dev, q, tables, ctx, None), attend(dev, q, tables, ctx, None)
    assert torch.equal(one, two)


def test_offsets_past_32_bits(env):
    """A cache of more than 2^32 bytes, used at its end."""
    torch, sara = env
    n_pages, hkv, hd = (1 << 32) // (8 * 16 * 128) + 40, 8, 128
    codes = [torch.empty((n_pages, hkv, 16, hd), dtype=torch.int8, device="cuda") for _ in range(2)]
    exp = [torch.empty((n_pages, hkv), dtype=torch.uint8, device="cuda") for _ in range(2)]
    rng = np.random.default_rng(17)
    small = Dev(env, 8, hkv, hd, "int8")
    k, v = (small.tensor(rng.standard_normal((100, hkv, hd)), torch.bfloat16) for _ in range(2))
    q = small.tensor(rng.standard_normal((100, hkv, hd)), torch.bfloat16)
    outs = []
    for cache, first in ((small.args, 0), ((*codes, *exp), n_pages - 8)):
        tables = small.i32(np.arange(7)[None, ::-1] + first)
        sara.sara_kv8_write(*cache, k, v, tables, small.i32([0]), small.i32([0, 100]))
        back = torch.empty((2, 100, hkv, hd), dtype=torch.bfloat16, device="cuda")
        sara.sara_kv8_read(*cache, tables, small.i32([0]), small.i32([0, 100]), back[0], back[1])
        out = torch.empty_like(q)
        sara.sara_kv8_attention(q, *cache, tables, small.i32([100]), small.i32([0, 100]), out)
        one = torch.empty_like(q[99:])
        sara.sara_kv8_attention(q[99:], *cache, tables, small.i32([100]), None, one)
        outs.append((back, out, one))
    for a, b in zip(*outs):
        assert torch.equal(a, b)


def test_graph_replay(env):
    """Write and attention captured in a HIP graph, replayed with other contents between the replays."""
    torch, sara = env
    rng = np.random.default_rng(18)
    dev, tables = filled(env, rng, 2, 128, "int8", [700, 90])
    pages, ctx, start = dev.i32(tables), dev.i32([700, 90]), dev.i32([699, 89])
    q, k, v = (dev.tensor(rng.standard_normal((2, h, 128)), torch.bfloat16) for h in (12, 2, 2))
    out, ws = torch.empty_like(q), torch.empty(1 << 22, dtype=torch.uint8, device="cuda")

    def step():
        sara.sara_kv8_write(*dev.args, k, v, pages, start)
        sara.sara_kv8_attention(q, *dev.args, pages, ctx, None, out, workspace=ws)

    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for i in range(4):
        for t in (q, k, v):
            t.copy_(dev.tensor(rng.standard_normal(tuple(t.shape)), torch.bfloat16))
        g.replay()
        torch.cuda.synchronize()
        got = out.clone()
        step()
        torch.cuda.synchronize()
        assert torch.equal(got, out), i


# -- refusals -----------------------------------------------------------------------
def test_refusals(env):
    torch, sara = env
    rng = np.random.default_rng(19)
    dev, tables = filled(env, rng, 2, 128, "int8", [64])
    q = dev.tensor(rng.standard_normal((1, 12, 128)), torch.bfloat16)
    pages, ctx = dev.i32(tables), dev.i32([64])
    k = q[:, :2]
    good = (q, *dev.args, pages, ctx, None, torch.empty_like(q))

    def bad(exc, i=None, val=None, **kw):
        args = list(good)
        if i is not None:
            args[i] = val
        with pytest.raises(exc):
            sara.sara_kv8_attention(*args, **kw)

    bad(ValueError, 0, q[:, :, :64])                                  # head_dim of q
    bad(TypeError, 1, dev.codes[0].view(torch.uint8))                 # format
    bad(ValueError, 2, dev.codes[1][:3])                              # K and V differ
    bad(ValueError, 3, dev.exp[0].to(torch.int32))
    bad(ValueError, 5, pages.long())
    bad(ValueError, 6, dev.i32([64, 64]))
    bad(ValueError, 7, dev.i32([0, 1, 1]))
    bad(ValueError, 8, torch.empty((2, 12, 128), dtype=torch.bfloat16, device="cuda"))
    bad(ValueError, 8, torch.empty((1, 12, 128), dtype=torch.float32, device="cuda"))
    bad(sara.SaraError, max_ctx=16 * tables.shape[1] + 1)
    bad(sara.SaraError, scale=float("inf"))
    q11, o11 = torch.empty((1, 11, 128), dtype=torch.bfloat16, device="cuda"), torch.empty((1, 11, 128), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(sara.SaraError):                               # 11 heads over 2 KV heads
        sara.sara_kv8_attention(q11, *dev.args, pages, ctx, None, o11)
    raw = torch.empty(12 * 128 + 8, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(sara.SaraError):                               # q off its 16 bytes
        sara.sara_kv8_attention(raw[1:1 + 12 * 128].view(1, 12, 128), *dev.args, pages, ctx, None, torch.empty_like(q))
    for i in (0, 1, 4, 5, 6, 8):                                      # host memory
        bad(ValueError, i, good[i].cpu())
    with pytest.raises(ValueError):                                   # rows without offsets
        sara.sara_kv8_write(*dev.args, q[:, :2].repeat(2, 1, 1), q[:, :2].repeat(2, 1, 1), pages, ctx)
    with pytest.raises(ValueError):
        sara.sara_kv8_write(*dev.args, k, q[:, :3], pages, ctx)
    with pytest.raises(TypeError):
        sara.sara_kv8_write(*dev.args, k.half(), k.half(), pages, ctx)
    dev2, tables2 = filled(env, rng, 2, 128, "int8", [5000])
    with pytest.raises(sara.SaraError):                               # workspace too small
        sara.sara_kv8_attention(q, *dev2.args, dev2.i32(tables2), dev2.i32([5000]), None, torch.empty_like(q),
                                workspace=torch.empty(64, dtype=torch.uint8, device="cuda"))
    with pytest.raises(ValueError):
        sara.sara_kv8_attention(q, *dev2.args, dev2.i32(tables2), dev2.i32([5000]), None, torch.empty_like(q),
                                workspace=torch.empty(1 << 20, dtype=torch.uint8))
    torch.cuda.synchronize()


def test_reads_from_below_position_zero(env):
    """Every row of a read is written: 0 for positions below 0, the cache's values for the rest."""
    torch, sara = env
    rng = np.random.default_rng(20)
    lowest = -2 ** 31
    for fmt, hkv, hd in (("int8", 2, 128), ("fp8", 3, 64)):
        dev, tables = filled(env, rng, hkv, hd, fmt, [70, 16, 5, 40, 9])
        start, n = [-1, -16, -37, -5, lowest], [60, 33, 30, 6, 40]
        off = offsets(n)
        got = dev.read(tables, start, off, torch.float32)
        for c, x in zip(dev.ref, got):
            for i in range(len(n)):
                want = np.zeros((n[i], hkv, hd))
                below = min(n[i], -start[i])
                want[below:] = c.read(tables[i], 0, n[i] - below)
                np.testing.assert_array_equal(x[off[i]:off[i + 1]], want)
        out = [torch.full((5, hkv, hd), 7.0, device="cuda") for _ in range(2)]      # one row a sequence
        sara.sara_kv8_read(*dev.args, dev.i32(tables), dev.i32([-1, 0, -9, 3, lowest]), None, *out)
        for c, x in zip(dev.ref, out):
            want = [np.zeros((hkv, hd)), c.read(tables[1], 0, 1)[0], np.zeros((hkv, hd)), c.read(tables[3], 3, 1)[0], np.zeros((hkv, hd))]
            np.testing.assert_array_equal(x.double().cpu().numpy(), np.array(want))


@pytest.mark.parametrize("fmt", ["int8", "fp8"])
def test_values_past_the_largest_number_reach_only_who_sees_them(env, fmt):
    """A V element whose code rounds to 2^128 at position 70: queries before it are as ever, those that see it get its
    share to 1/15 (a code below it in e4m3) of that element; and a K element as large in a dim where every q is 0 changes
    nothing.  Both kernels."""
    torch = env[0]
    rng = np.random.default_rng(24)
    ctx = [100, 100]
    dev, tables = filled(env, rng, 1, 128, fmt, ctx)
    x = [rng.standard_normal((16, 1, 128)) for _ in range(2)]
    x[1][6, 0, 9] = 3.4e38
    k, v = (dev.tensor(y, torch.float32) for y in x)
    assert bool(v.isfinite().all())
    dev.write(k, v, tables[:1], [64], [0, 16])
    x[0][6, 0, 9], x[1][6, 0, 9] = -3.4e38, 1.0
    dev.write(dev.tensor(x[0], torch.float32), dev.tensor(x[1], torch.float32), tables[1:], [64], [0, 16])
    assert dev.ref[1].read(tables[0], 70, 1)[0, 0, 9] == 2.0 ** 128 == -dev.ref[0].read(tables[1], 70, 1)[0, 0, 9]
    for nq in ([100, 100], [8, 8]):                                       # tiles of columns; few columns
        q = dev.tensor(rng.standard_normal((sum(nq), 4, 128)), torch.float32)
        q[:, :, 9] = 0.0
        got = attend(dev, q, tables, ctx, offsets(nq))
        seen = max(0, nq[0] - 30)                                         # the first row that sees position 70
        check_attention(dev, q[nq[0]:], got[nq[0]:], tables[1:], ctx[1:], offsets(nq[1:]))
        if seen:
            early = got[:seen]
            assert bool(early.isfinite().all())
            alone = attend(dev, q[:seen].contiguous(), tables[:1], [70], [0, seen])
            torch.testing.assert_close(early, alone, rtol=1e-5, atol=1e-6)
        want = R.attention(q[seen:nq[0]].double().cpu().numpy(), *(c.read(tables[0], 0, 100) for c in dev.ref), np.ones(100, bool),
                           100, 128 ** -0.5)
        have = got[seen:nq[0]].double().cpu().numpy()
        assert not np.isnan(have).any()
        other = np.arange(128) != 9
        np.testing.assert_allclose(have[..., other], want[..., other], rtol=1e-4, atol=1e-5)
        np.testing.assert_allclose(have[..., 9], want[..., 9], rtol=1 / 15)
    for t in (75, 99):                                                    # single tokens
        q = dev.tensor(rng.standard_normal((2, 4, 128)), torch.float32)
        q[:, :, 9] = 0.0
        got = attend(dev, q, tables, [t + 1, t + 1], None)
        check_attention(dev, q[1:], got[1:], tables[1:], [t + 1], None)
        want = R.attention(q[:1].double().cpu().numpy(), *(c.read(tables[0], 0, t + 1) for c in dev.ref), np.ones(t + 1, bool), t + 1,
                           128 ** -0.5)
        np.testing.assert_allclose(got[:1].double().cpu().numpy(), want, rtol=1e-4, atol=1e-5)


def test_expanded_outputs_are_refused_and_transposed_ones_are_not(env):
    torch, sara = env
    rng = np.random.default_rng(25)
    dev, tables = filled(env, rng, 2, 128, "int8", [40, 40])
    pages, ctx, off = dev.i32(tables), dev.i32([40, 40]), dev.i32([0, 40, 80])
    q = dev.tensor(rng.standard_normal((80, 4, 128)), torch.bfloat16)
    want = attend(dev, q, tables, [40, 40], [0, 40, 80])
    one, kv = torch.zeros((1, 4, 128), dtype=torch.bfloat16, device="cuda"), torch.zeros((80, 2, 128), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(sara.SaraError):
        sara.sara_kv8_attention(q, *dev.args, pages, ctx, off, one.expand(80, 4, 128))
    for bad in (one[:, :2].expand(80, 2, 128), kv[:, :1].expand(80, 2, 128)):
        for k, v in ((bad, kv), (kv, bad)):
            with pytest.raises(sara.SaraError):
                sara.sara_kv8_read(*dev.args, pages, dev.i32([0, 0]), off, k, v)
    by_head = torch.empty((4, 80, 128), dtype=torch.bfloat16, device="cuda")              # [heads, rows, dim]
    assert torch.equal(attend(dev, q, tables, [40, 40], [0, 40, 80], out=by_head.transpose(0, 1)), want)
    k, v = torch.empty((2, 2, 80, 128), dtype=torch.bfloat16, device="cuda").transpose(1, 2)
    sara.sara_kv8_read(*dev.args, pages, dev.i32([0, 0]), off, k, v)
    np.testing.assert_array_equal(k[40:].double().cpu().numpy(), dev.ref[0].read(tables[1], 0, 40))
    last = torch.empty((1, 4, 128), dtype=torch.bfloat16, device="cuda")
    few = attend(dev, q[79:], tables[1:], [40], None, out=last.as_strided((1, 4, 128), (0, 128, 1)))   # one row: any row stride
    check_attention(dev, q[79:], few, tables[1:], [40], None)


def test_the_stride_of_a_single_row_or_head_does_not_matter(env):
    """One row of a buffer whose rows are 8 bytes off 16, and one KV head likewise: the strides are never followed."""
    torch, sara = env
    rng = np.random.default_rng(26)
    dev, tables = filled(env, rng, 1, 128, "int8", [50])
    buf = dev.tensor(rng.standard_normal((4, 6 * 128 + 4)), torch.bfloat16)
    q = buf[:, :6 * 128].unflatten(1, (6, 128))[:1]
    assert q.stride(0) % 8
    got = attend(dev, q, tables, [50], None, out=torch.empty_like(buf)[:, :6 * 128].unflatten(1, (6, 128))[:1])
    check_attention(dev, q, got, tables, [50], None)
    k = buf.as_strided((6, 1, 128), (128, 132, 1))
    back = torch.empty((2, 6, 128), dtype=torch.bfloat16, device="cuda").as_strided((2, 6, 1, 128), (768, 128, 132, 1))
    dev.write(k, k, tables, [44], [0, 6])
    sara.sara_kv8_read(*dev.args, dev.i32(tables), dev.i32([44]), dev.i32([0, 6]), back[0], back[1])
    np.testing.assert_array_equal(back[1].double().cpu().numpy(), dev.ref[1].read(tables[0], 44, 6))


@pytest.mark.parametrize("fmt", ["int8", "fp8"])
def test_the_smallest_values_read_as_bf16(env, fmt):
    """Pages of the three smallest scales: exact in fp32, to the nearest bf16 (steps of 2^-133, ties to even) in bf16."""
    torch = env[0]
    dev = Dev(env, 6, 1, 128, fmt)
    x = np.arange(48 * 128).reshape(48, 1, 128) % 901 * 2.0 ** -135
    x[::2] *= -1
    x[::16, 0, 5] = R.TOP[fmt] * 2.0 ** (np.arange(3) - 126)                # b = 1, 2, 3
    k = dev.tensor(x, torch.float32)
    dev.write(k, -k, np.array([[0, 1, 2]]), [0], [0, 48])
    assert dev.exp[0][:3, 0].tolist() == [1, 2, 3]
    dev.check(np.array([[0, 1, 2]]), [0], [0, 48], torch.float32)
    got = dev.read(np.array([[0, 1, 2]]), [0], [0, 48], torch.bfloat16)
    for c, y in zip(dev.ref, got):
        want = c.read([0, 1, 2], 0, 48)
        exact = torch.from_numpy(want.astype(np.float32))
        assert np.array_equal(exact.double().numpy(), want)
        np.testing.assert_array_equal(y, exact.to(torch.bfloat16).double().numpy())
        assert np.array_equal(y[32:], want[32:]) and (fmt == "int8" or not np.array_equal(y[:16], want[:16]))


# -- long splits, both kernels ------------------------------------------------------
def check_rows(dev, q, got, tables, ctx, off, scale=None):
    """check_attention's bound with the reference in fp64 on the device, a head at a time; tables may share pages."""
    torch, hd, bf16 = dev.torch, dev.hd, q.dtype == dev.torch.bfloat16
    scale, group = hd ** -0.5 if scale is None else scale, q.shape[1] // dev.hkv
    off = list(range(len(tables) + 1)) if off is None else off
    values = [torch.from_numpy(np.where((c.exp == 255)[:, :, None, None], np.nan, c.val)).cuda() for c in dev.ref]
    for i, table in enumerate(np.asarray(tables)):
        n, end = off[i + 1] - off[i], max(ctx[i], 0)
        if n == 0 or end == 0:
            assert bool((got[off[i]:off[i + 1]] == 0).all())
            continue
        have = torch.from_numpy(np.repeat((table >= 0) & (table < dev.n_pages), 16)[:end]).cuda()
        page = torch.from_numpy(np.where((table >= 0) & (table < dev.n_pages), table, 0)).cuda()
        at = torch.arange(end, device="cuda")
        seen = have[None] & (at[None] <= end - n + torch.arange(n, device="cuda")[:, None])
        for h in range(q.shape[1]):
            k, v = (x[page, h // group].reshape(-1, hd)[:end] for x in values)
            bad = (k.isnan() | v.isnan()).any(1)                         # a key of a NaN page: who sees it is NaN
            k, v = k.nan_to_num(), v.nan_to_num()
            qh, out = q[off[i]:off[i + 1], h].double(), got[off[i]:off[i + 1], h].double()
            s = (qh @ k.T.contiguous() * scale).masked_fill(~seen, -np.inf)
            p = torch.exp(s - s.amax(1, keepdim=True).nan_to_num(neginf=0.0))
            want = p @ v / p.sum(1, keepdim=True).clamp(min=1e-300)
            nan = (seen & bad[None]).any(1)
            assert torch.equal(out.isnan().all(1), nan) and torch.equal(out.isnan().any(1), nan), (i, h)
            used = k[have]
            smax = float((used.abs() @ qh.abs().T.contiguous()).amax()) * abs(scale) * 1.4427 if len(used) else 0.0
            d = smax * 2.0 ** -22 + 2.0 ** -20 + (2.0 ** -17 if bf16 else 2.0 ** -24)
            vmax = float(v[have].abs().amax()) if len(used) else 0.0
            bound = 2 * d * vmax + (2.0 ** -8 if bf16 else 2.0 ** -23) * want.abs()
            err = (out - want).abs()[~nan]
            assert bool((err <= bound[~nan]).all()), (i, h, float((err / bound[~nan].clamp(min=1e-300)).amax()))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,hd,fmt", [(16, 2, 128, "int8"), (12, 4, 64, "fp8")])
def test_prompts_longer_than_the_page_ids_in_hand(env, hq, hkv, hd, fmt, dtype):
    """Tiles of columns in one split each of up to 160 pages: page ids, exponents and the masks of missing pages are taken
    64 at a time.  Pages are missing on both sides of pages 64 and 128, and at the last one."""
    torch = env[0]
    rng = np.random.default_rng([27, hd])
    nq, ctx = [1300, 1100, 900], [1300, 2550, 1040]
    dev, tables = filled(env, rng, hkv, hd, fmt, ctx)
    tables[0, [62, 64]] = -1
    tables[1, [63, 64, 65, 127, 128, 159]] = -1
    tables[2, 60:65] = dev.n_pages
    q = dev.tensor(rng.standard_normal((sum(nq), hq, hd)) * 2, torch.bfloat16 if dtype == "bf16" else torch.float32)
    got = attend(dev, q, tables, ctx, offsets(nq))
    check_rows(dev, q, got, tables, ctx, offsets(nq))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("ragged", [False, True])
def test_many_long_contexts_read_their_page_ids_again(env, ragged, dtype):
    """600 (sequence, KV head) pairs leave a row in one split, whose waves take their page ids 32 pairs at a time: contexts
    on both sides of 256 pages, some missing around it.  The sequences share their pages."""
    torch = env[0]
    rng = np.random.default_rng(28)
    dev, one = filled(env, rng, 2, 64, "int8", [4620])
    ctx = [int(c) for c in rng.integers(4000, 4620, 300)]
    ctx[:6] = [4096, 4097, 4112, 4113, 4224, 4619]
    tables = np.repeat(one, 300, 0)
    for i in range(0, 300, 3):
        tables[i, rng.integers(250, 289, 5)] = -1
    nq = [1 + i % 2 for i in range(300)] if ragged else [1] * 300
    off = offsets(nq)
    q = dev.tensor(rng.standard_normal((off[-1], 4, 64)) * 2, torch.bfloat16 if dtype == "bf16" else torch.float32)
    got = attend(dev, q, tables, ctx, off if ragged else None)
    check_rows(dev, q, got, tables, ctx, off)


@pytest.mark.parametrize("fmt", ["int8", "fp8"])
@pytest.mark.parametrize("hd", [64, 128])
def test_nan_pages_and_scales_in_both_kernels(env, hd, fmt):
    """NaN pages of K and of V, page scales 2^40 apart and a scale below 0: single queries, and as many as there are tokens."""
    torch = env[0]
    rng = np.random.default_rng([29, hd])
    ctx = [160, 160, 150]
    for dtype in (torch.bfloat16, torch.float32):
        dev, tables = filled(env, rng, 2, hd, fmt, ctx)
        bad, good = np.ones((1, 2, hd)), np.ones((1, 2, hd))
        bad[0, 1, 3] = np.inf
        for i, kv in ((0, (bad, good)), (1, (good, bad))):
            dev.write(*(dev.tensor(x, torch.float32) for x in kv), tables[i:i + 1], [100], [0, 1])
        size = np.exp2(rng.integers(-20, 20, 10)).repeat(16)[:150, None, None]
        dev.write(dev.tensor(rng.standard_normal((150, 2, hd)), torch.float32),
                  dev.tensor(rng.standard_normal((150, 2, hd)) * size, torch.float32), tables[2:], [0], [0, 150])
        for scale in (None, -0.2):
            for end in (99, 112, 150):                                   # before the pages' NaN tokens, at them, past them
                q = dev.tensor(rng.standard_normal((3, 4, hd)), dtype)
                check_rows(dev, q, attend(dev, q, tables, [end] * 3, None, scale=scale), tables, [end] * 3, None, scale)
            q = dev.tensor(rng.standard_normal((sum(ctx), 4, hd)), dtype)
            got = attend(dev, q, tables, ctx, offsets(ctx), scale=scale)
            check_rows(dev, q, got, tables, ctx, offsets(ctx), scale)
            assert bool(got[150, 2:].isnan().all()) and not bool(got[:, :2].isnan().any()) and not bool(got[320:].isnan().any())


@pytest.mark.parametrize("size", [2.0 ** -80, 2.0 ** 100])
def test_small_and_large_values(env, size):
    """All of V at 1e-24 and at 1e30: weights and page scales meet in bf16 parts, whose range holds them."""
    torch = env[0]
    rng = np.random.default_rng(30)
    for fmt in ("int8", "fp8"):
        dev = Dev(env, 24, 1, 64, fmt)
        tables = make_tables(rng, [300], 19, 24)
        dev.write(dev.tensor(rng.standard_normal((300, 1, 64)), torch.float32),
                  dev.tensor(rng.standard_normal((300, 1, 64)) * size, torch.float32), tables, [0], [0, 300])
        for nq in (1, 100):
            q = dev.tensor(rng.standard_normal((nq, 4, 64)) * 2, torch.float32)
            check_rows(dev, q, attend(dev, q, tables, [300], [0, nq]), tables, [300], [0, nq])


def test_a_sequence_alone_and_among_others(env):
    """The same bits where the batch cuts its context alike (pages a split follow the number of sequences and max_ctx: here
    24 either way), and right in a batch that cuts it otherwise."""
    torch = env[0]
    rng = np.random.default_rng(31)
    ctx = [900, 40, 333] + [700] * 120
    dev, tables = filled(env, rng, 2, 128, "fp8", ctx[:4])
    tables = np.concatenate([tables[:3], np.repeat(tables[3:], 120, 0)])
    q = dev.tensor(rng.standard_normal((len(ctx), 12, 128)), torch.bfloat16)
    few = attend(dev, q[:3], tables[:3], ctx[:3], None, max_ctx=900)
    check_rows(dev, q[:3], few, tables[:3], ctx[:3], None)
    for i in range(3):
        alone = attend(dev, q[i:i + 1], tables[i:i + 1], ctx[i:i + 1], None, max_ctx=900)
        assert torch.equal(alone[0], few[i]), i
    many = attend(dev, q.repeat(6, 1, 1), np.tile(tables, (6, 1)), ctx * 6, None, max_ctx=900)   # 738 sequences: one split
    check_rows(dev, q, many[:len(ctx)], tables, ctx, None)
    assert torch.equal(many[:len(ctx)], many[-len(ctx):])
