"""Log probabilities from hidden states and the LM head, and their gradients,
against the definition in 64 bits: one row to thousands, widths and vocabularies
that end inside tiles, strides, padding rows that hold anything, logits that are
not finite, temperatures, several pieces of the vocabulary, graphs and streams.

Bounds.  A logit is a sum of d products in fp32: it is off by at most
d 2^-24 sum |h w| (fp32 inputs: their products drop parts below 3 2^-24 of one
more).  A log probability moves by at most twice the largest of that over T;
exponentials, sums of some hundreds in a row and logarithms add 2^-18 of
1 + |log p|.  Gradients are bounded element by element from |D| |W| and |D| |H|."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch

    import paper_2607_26253_amd as sara
    assert torch.cuda.is_available(), "GPU tests need a HIP device"
    return torch, sara


def make(env, rows, d, V, dtype, seed=0, pad=0, wpad=0, spread=2.0):
    """hidden [rows, d], weight [V, d] (rows padded by `pad` / `wpad` elements), ids, some of them none, and gradients."""
    torch, _ = env
    g = torch.Generator(device="cuda").manual_seed(1000 * seed + rows + 7 * d + 13 * V)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    h, w = normal(rows, d + pad).to(dt)[:, :d], (normal(V, d + wpad) * spread / math.sqrt(d)).to(dt)[:, :d]
    tok = torch.randint(0, V, (rows,), generator=g, device="cuda", dtype=torch.int32)
    gl, ge = normal(rows), normal(rows) * 0.1
    if rows > 4:
        tok[2], tok[4] = -1, V                            # no id: its log probability is 0, its entropy still counts
        gl[3], ge[3] = 0.0, 0.0                           # nothing asked
        ge[::5] = 0.0
    return dict(h=h, w=w, tok=tok, gl=gl, ge=ge)


def exact(env, x, T):
    torch, _ = env
    h, w = x["h"].double(), x["w"].double()
    tok, V = x["tok"].long(), w.shape[0]
    logits = h @ w.T.contiguous()
    size = h.abs() @ w.abs().T.contiguous()               # sum |h w|
    lp = torch.log_softmax(logits / T, -1)
    p = lp.exp()
    ent = -torch.special.xlogy(p, p).sum(-1)
    has = (tok >= 0) & (tok < V)
    at = tok.clamp(0, V - 1)[:, None]
    logp = torch.where(has, lp.gather(1, at)[:, 0], torch.zeros_like(ent))
    top = logits.amax(-1)
    total = ((logits - top[:, None]) / T).exp().sum(-1)
    gl, ge = x["gl"].double() * has, x["ge"].double()
    D = -p * (gl[:, None] + ge[:, None] * (lp + ent[:, None]))
    D.scatter_add_(1, at, gl[:, None])
    D /= T
    dx = (h.shape[1] + 4) * 2.0 ** -24 * size.amax(-1)    # of a logit
    moved = 2 * dx / T                                    # of a log probability, and of a probability relative to it
    # D is made of probabilities: their relative error, that of 2^u and of the row's factors
    Derr = (moved + 2.0 ** -17)[:, None] * (p * (gl.abs()[:, None] + ge.abs()[:, None] * (lp.abs() + ent[:, None] + 2))) / T
    Derr += 2.0 ** -22 * D.abs()
    return dict(logp=logp, ent=ent, top=top, total=total, D=D, Derr=Derr, dx=dx, moved=moved, h=h, w=w,
                lp_max=logp.abs())


def forward(env, x, T=1.0, **kw):
    torch, sara = env
    n = x["h"].shape[0]
    f32 = dict(device="cuda", dtype=torch.float32)
    out = dict(logp=torch.full((n,), 7.0, **f32), ent=torch.full((n,), 7.0, **f32), stats=torch.full((n, 2), 7.0, **f32))
    sara.sara_head_logprobs(x["h"], x["w"], x["tok"], out["logp"], out["ent"], out["stats"], temperature=T, **kw)
    return out


def check_forward(out, e):
    assert bool(((out["logp"].double() - e["logp"]).abs() <= e["moved"] + 2.0 ** -18 * (1 + e["logp"].abs())).all())
    assert bool(((out["ent"].double() - e["ent"]).abs() <= 2 * e["moved"] * (1 + e["ent"]) + 2.0 ** -18 * (1 + e["ent"])).all())
    assert bool(((out["stats"][:, 0].double() - e["top"]).abs() <= e["dx"]).all())
    assert bool(((out["stats"][:, 1].double() / e["total"] - 1).abs() <= e["moved"] + 2.0 ** -18).all())


def gradients(env, x, fwd, T=1.0, sums=None, hidden=True, weight=True, gl=True, ge=True, accumulate=False, start=None, **kw):
    torch, sara = env
    (n, d), V = x["h"].shape, x["w"].shape[0]
    gh = torch.full((n, d), 7.0, device="cuda", dtype=x["h"].dtype) if hidden else None
    gw = None
    if weight:
        gw = torch.full((V, d), 7.0, device="cuda", dtype=sums or x["w"].dtype) if start is None else start.clone()
    sara.sara_head_logprobs_grad(x["h"], x["w"], x["tok"], fwd["stats"], fwd["ent"] if ge else None, x["gl"] if gl else None,
                                 x["ge"] if ge else None, gh, gw, temperature=T, accumulate=accumulate, **kw)
    return gh, gw


def half_step(torch, t):
    return torch.finfo(t).eps / 2


def check_gradients(env, gh, gw, x, e, start=None):
    """Element by element: the error of D and its rounding to bf16 parts, sums in fp32, and the output's rounding."""
    torch, _ = env
    bf16 = x["h"].dtype == torch.bfloat16
    clean = x.get("clean", x["h"]).double()
    for got, other, D, Derr, part in ((gh, e["w"], e["D"], e["Derr"], 2.0 ** -8),
                                      (gw, clean, e["D"].T.contiguous(), e["Derr"].T.contiguous(),
                                       2.0 ** -8 if gw is None or gw.dtype == torch.bfloat16 else 2.0 ** -16)):
        if got is None:
            continue
        if not bf16:
            part = 3 * 2.0 ** -24
        want = D @ other
        bound = Derr @ other.abs() + (part + (D.shape[1] + 8) * 2.0 ** -24) * (D.abs() @ other.abs())
        if start is not None and got is gw:
            want = want + start.double()
            bound = bound + 2.0 ** -24 * start.double().abs()
        bound = bound + half_step(torch, got.dtype) * (want.abs() + bound) + 1e-38
        assert bool(((got.double() - want).abs() <= bound).all()), float(((got.double() - want).abs() / bound).max())


SIZES = [(1, 8, 1), (1, 64, 257), (2, 72, 16), (3, 40, 500), (15, 136, 129), (16, 512, 1000), (17, 256, 4097), (33, 1032, 300),
         (64, 200, 2000), (65, 72, 511), (255, 64, 256), (256, 32, 257), (257, 128, 768), (300, 1000, 1031), (513, 264, 520)]
# past what small tiles take, with ends inside the large ones: for fp32 too
BIG = (1100, 1032, 5001)
LARGE = [BIG, (2500, 1000, 2065), (70, 1544, 33001)]
# few rows and many ids: dH's contraction in splits
LONG = [(2, 72, 40000), (33, 200, 9001), (1, 8, 2049)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,d,V", SIZES + LARGE + LONG)
def test_log_probabilities_and_gradients(env, rows, d, V, dtype):
    torch, _ = env
    T = (1.0, 0.7, 1.3)[rows % 3]
    x = make(env, rows, d, V, dtype, pad=8 * (rows % 2), wpad=16 * (V % 2))
    e = exact(env, x, T)
    out = forward(env, x, T)
    check_forward(out, e)
    check_gradients(env, *gradients(env, x, out, T), x, e)
    gh, gw = gradients(env, x, out, T, sums=torch.float32)
    check_gradients(env, gh, gw, x, e)
    if rows > 4:
        assert bool((gh[3] == 0).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,V", [(5, 300), (70, 300), (70, 130001)])
def test_width_of_four(env, rows, V, dtype):
    """fp32 rows of 16 bytes end inside a unit of eight bf16 parts; the narrowest bf16 row is eight wide."""
    d = 8 if dtype == "bf16" else 4
    for width in (d, 5 * d):
        x = make(env, rows, width, V, dtype)
        e = exact(env, x, 1.0)
        out = forward(env, x)
        check_forward(out, e)
        check_gradients(env, *gradients(env, x, out), x, e)


@pytest.mark.parametrize("rows,d,V", [(9, 96, 700), (80, 96, 700), BIG])
def test_one_gradient_at_a_time_and_either_cotangent(env, rows, d, V):
    torch, _ = env
    x = make(env, rows, d, V, "bf16")
    out = forward(env, x)
    both = gradients(env, x, out)
    gh, none = gradients(env, x, out, weight=False)
    assert none is None and torch.equal(gh, both[0])
    none, gw = gradients(env, x, out, hidden=False)
    assert none is None and torch.equal(gw, both[1])
    for kw in (dict(gl=False), dict(ge=False)):
        y = dict(x)
        y["gl" if "gl" in kw else "ge"] = torch.zeros(rows, device="cuda")
        check_gradients(env, *gradients(env, x, out, **kw), y, exact(env, y, 1.0))
    gh, gw = gradients(env, x, out, gl=False, ge=False)
    assert bool((gh == 0).all()) and bool((gw == 0).all())


@pytest.mark.parametrize("rows,d,V", [(70, 128, 900), BIG])
@pytest.mark.parametrize("sums", ["bf16", "f32"])
def test_accumulates(env, sums, rows, d, V):
    torch, _ = env
    sums = torch.bfloat16 if sums == "bf16" else torch.float32
    x = make(env, rows, d, V, "bf16")
    out = forward(env, x)
    start = torch.randn((V, d), device="cuda").to(sums)
    gh, gw = gradients(env, x, out, accumulate=True, start=start)
    check_gradients(env, gh, gw, x, exact(env, x, 1.0), start=start)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,d,V", [(20, 128, 600), (300, 128, 600), BIG])
def test_rows_that_ask_for_nothing_may_hold_anything(env, rows, d, V, dtype):
    """Padding rows of NaN and infinities change no gradient; their own is 0 and their statistics are NaN."""
    torch, _ = env
    x = make(env, rows, d, V, dtype)
    pad = torch.arange(rows, device="cuda") % 7 == 3
    x["gl"][pad], x["ge"][pad] = 0.0, 0.0
    clean = x["h"].clone()
    clean[pad] = 0.0
    y = dict(x, h=clean)
    e = exact(env, y, 1.0)
    x["h"][pad] = torch.tensor([math.nan, math.inf, -math.inf], device="cuda").repeat(rows)[:int(pad.sum())][:, None].to(x["h"].dtype)
    x["clean"] = clean
    out = forward(env, x)
    assert bool(out["logp"][pad & (x["tok"] >= 0) & (x["tok"] < V)].isnan().all()) and bool(out["ent"][pad].isnan().all())
    assert bool(out["stats"][pad].isnan().all())
    check_forward({k: v[~pad] for k, v in out.items()}, {k: v[~pad] for k, v in e.items() if k not in ("h", "w")})
    gh, gw = gradients(env, x, out)
    assert bool((gh[pad] == 0).all())
    check_gradients(env, gh, gw, x, e)


@pytest.mark.parametrize("rows,d,V", [(3, 64, 400), (90, 64, 400), BIG])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_logits_that_are_not_finite(env, rows, d, V, bad):
    """One bad element of one row reaches that row's outputs and its gradient only, one of the weight every row."""
    torch, _ = env
    x = make(env, rows, d, V, "bf16")
    x["tok"][:] = 5
    x["gl"][:] = 1.0
    good = forward(env, x)
    ok = gradients(env, x, good)
    x["h"][1, 9] = bad
    out = forward(env, x)
    assert bool(out["logp"][1].isnan()) and bool(out["ent"][1].isnan()) and bool(out["stats"][1].isnan().all())
    keep = torch.arange(rows, device="cuda") != 1
    for k in out:
        assert torch.equal(out[k][keep], good[k][keep]), k
    gh, _ = gradients(env, x, out, weight=False)
    assert bool(gh[1].isnan().all()) and torch.equal(gh[keep], ok[0][keep])
    x["h"][1, 9] = 1.0
    x["w"][V - 1, 9] = bad
    out = forward(env, x)
    assert bool(out["logp"].isnan().all()) and bool(out["stats"].isnan().all())


@pytest.mark.parametrize("rows,d,V", [(4, 64, 700), (100, 64, 700), BIG])
@pytest.mark.parametrize("T", [1e-37, 1e-3, 30.0, 1e37])
def test_temperatures(env, rows, d, V, T):
    """Cold rows put everything on their largest logit, hot ones are uniform; logits far apart and equal."""
    torch, _ = env
    x = make(env, rows, d, V, "f32", spread=1.0)
    x["h"], x["w"] = (x["h"] * 2).round(), (x["w"] * 8).round()       # products and sums are exact
    x["w"][::3] = x["w"][0]
    logits = x["h"].double() @ x["w"].double().T.contiguous()
    out = forward(env, x, T)
    lp = torch.log_softmax((logits - logits.amax(-1, keepdim=True)) / T, -1)
    tok = x["tok"].clamp(0, V - 1).long()
    has = (x["tok"] >= 0) & (x["tok"] < V)
    want = torch.where(has, lp.gather(1, tok[:, None])[:, 0], torch.zeros_like(lp[:, 0]))
    # at 1e-37 logits 53 apart make log probabilities of -5.3e38, which is past fp32's 3.4e38: -inf, as fp32 rounds them
    near = (out["logp"].double() - want).abs() <= 2.0 ** -18 * (1 + want.abs())
    assert bool((near | (out["logp"] == want.float())).all())
    p = lp.exp()
    ent = -torch.special.xlogy(p, p).sum(-1)
    assert bool(((out["ent"].double() - ent).abs() <= 2.0 ** -18 * (1 + ent)).all())
    if T == 1e-37:
        x["gl"] = x["gl"] * 1e-37                                     # else 1 / T takes the gradient past fp32
        x["ge"] = x["ge"] * 0.0
    e = exact(env, x, T)
    e["Derr"] = e["Derr"].nan_to_num(0.0)
    if T != 1e-37:
        e["Derr"] = 2.0 ** -17 * e["D"].abs() + 2.0 ** -17 * p * (x["gl"].double().abs() + x["ge"].double().abs() * (1 + ent + 20))[:, None] / T
    else:
        e["Derr"] = 2.0 ** -17 * (e["D"].abs() + p * (x["gl"].double().abs() / T)[:, None])
    check_gradients(env, *gradients(env, x, out, T), x, e)


def test_pieces_of_the_vocabulary(env):
    """D of 1,100 rows over 130,000 ids, in two parts, passes a piece's 448 MiB; the last piece is short."""
    x = make(env, 1100, 64, 130001, "bf16")
    e = exact(env, x, 1.0)
    out = forward(env, x)
    check_forward(out, e)
    check_gradients(env, *gradients(env, x, out), x, e)


def test_many_rows(env):
    """Forward tiles run 8,192 rows at a time."""
    for d, V, dtype in ((16, 300, "bf16"), (16, 300, "f32"), (1032, 520, "bf16"), (1032, 520, "f32")):
        x = make(env, 8300, d, V, dtype)
        check_forward(forward(env, x), exact(env, x, 1.0))


def test_large_offsets(env):
    """A weight whose last rows lie past 2^32 bytes, by its stride."""
    torch, sara = env
    big = torch.zeros((70000, 32768), device="cuda", dtype=torch.bfloat16)
    w = big[:, 100 * 8:100 * 8 + 32]
    w.copy_(torch.randn((70000, 32), device="cuda") * 0.5)
    for rows in (5, 70):
        x = make(env, rows, 32, 70000, "bf16")
        x["w"] = w
        e = exact(env, x, 1.0)
        out = forward(env, x)
        check_forward(out, e)
        check_gradients(env, *gradients(env, x, out), x, e)


def test_gradient_against_differences(env):
    """Steps of 2^-6 along random directions: third-order terms are below 2^-12 of the direction's cube times the
    objective's third derivative (below 10 here); fp32 differences of sums of 12 terms add 1e-4."""
    torch, _ = env
    x = make(env, 12, 64, 200, "f32")
    T = 0.9

    def objective(y):
        e = exact(env, y, T)
        return float((e["logp"] * y["gl"].double() + e["ent"] * y["ge"].double()).sum())

    gh, gw = gradients(env, x, forward(env, x, T), T)
    for name, grad in (("h", gh), ("w", gw)):
        way = torch.randn(x[name].shape, device="cuda", dtype=torch.float64)
        way /= way.norm()
        step = 2.0 ** -6
        ends = [objective(dict(x, **{name: x[name].double() + s * step * way})) for s in (1, -1)]
        assert abs((ends[0] - ends[1]) / (2 * step) - float((grad.double() * way).sum())) <= 10 * step ** 2 + 1e-4


@pytest.mark.parametrize("rows,d,V", [(7, 128, 1500), (130, 128, 1500), BIG])
def test_streams_graphs_and_workspaces(env, rows, d, V):
    """Replays on inputs that change, on a side stream, with the caller's workspace, give the eager results bit for bit."""
    torch, sara = env
    import ctypes
    sizes = dict(rows=rows, d=d, V=V, dtype="bf16")
    xs = [make(env, seed=s, **sizes) for s in range(3)]
    eager = []
    for x in xs:
        out = forward(env, x)
        eager.append((out, gradients(env, x, out)))
    need = ctypes.c_int64(0)
    space = []
    for grad in (0, 1):
        assert sara._lib.sara_head_logprobs_workspace(1, rows, d, V, grad, 1, ctypes.byref(need)) == 0
        space.append(torch.full((need.value,), 255, device="cuda", dtype=torch.uint8))
    live = {k: v.clone() for k, v in xs[0].items()}
    out = {k: torch.empty_like(v) for k, v in eager[0][0].items()}
    gh, gw = torch.empty_like(live["h"]), torch.empty_like(live["w"])
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        sara.sara_head_logprobs(live["h"], live["w"], live["tok"], out["logp"], out["ent"], out["stats"], workspace=space[0])
        sara.sara_head_logprobs_grad(live["h"], live["w"], live["tok"], out["stats"], out["ent"], live["gl"], live["ge"], gh, gw,
                                     workspace=space[1])
    for i in (1, 2, 0, 2):
        for k in live:
            live[k].copy_(xs[i][k])
        for s in space:
            s.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        for k in out:
            assert torch.equal(out[k], eager[i][0][k]), (i, k)
        assert torch.equal(gh, eager[i][1][0]) and torch.equal(gw, eager[i][1][1])
        forward(env, xs[i])                                # eager work between the replays
    with pytest.raises(sara.SaraError, match="workspace"):
        sara.sara_head_logprobs(live["h"], live["w"], live["tok"], out["logp"], workspace=space[0][:-1])
    x = xs[1]
    side.wait_stream(torch.cuda.current_stream())
    got = forward(env, x, stream=side)
    side.synchronize()
    assert all(torch.equal(got[k], eager[1][0][k]) for k in got)


def test_no_rows(env):
    torch, sara = env
    h, w = torch.zeros((0, 64), device="cuda"), torch.ones((50, 64), device="cuda")
    tok = torch.zeros(0, device="cuda", dtype=torch.int32)
    none = torch.zeros(0, device="cuda")
    stats = torch.zeros((0, 2), device="cuda")
    sara.sara_head_logprobs(h, w, tok, none, none, stats)
    gw = torch.full((50, 72), 3.0, device="cuda")
    sara.sara_head_logprobs_grad(h, w, tok, stats, none, none, none, h, gw[:, :64], accumulate=True)
    assert bool((gw == 3).all())
    sara.sara_head_logprobs_grad(h, w, tok, stats, none, none, none, h, gw[:, :64])
    assert bool((gw[:, :64] == 0).all()) and bool((gw[:, 64:] == 3).all())


def test_refusals(env):
    torch, sara = env
    x = make(env, 8, 64, 100, "bf16")
    out = forward(env, x)
    gh, gw = torch.empty_like(x["h"]), torch.empty_like(x["w"])

    def fwd(**kw):
        y = dict(h=x["h"], w=x["w"], tok=x["tok"], T=1.0)
        y.update(kw)
        sara.sara_head_logprobs(y["h"], y["w"], y["tok"], out["logp"], temperature=y["T"])

    def bwd(**kw):
        y = dict(h=x["h"], w=x["w"], tok=x["tok"], T=1.0, gh=gh, gw=gw, stats=out["stats"], ent=out["ent"], ge=x["ge"])
        y.update(kw)
        sara.sara_head_logprobs_grad(y["h"], y["w"], y["tok"], y["stats"], y["ent"], x["gl"], y["ge"], y["gh"], y["gw"], temperature=y["T"])

    for f in (fwd, bwd):
        f()
        for kw, exc in ((dict(h=x["h"].float()), ValueError), (dict(h=x["h"].half()), TypeError), (dict(h=x["h"][:, :32]), ValueError),
                        (dict(h=x["h"].T), ValueError), (dict(w=x["w"].cpu()), ValueError), (dict(tok=x["tok"].long()), ValueError),
                        (dict(tok=x["tok"][:3]), ValueError), (dict(T=0.0), sara.SaraError), (dict(T=math.nan), sara.SaraError),
                        (dict(h=x["h"][0]), ValueError), (dict(w=None), TypeError)):
            with pytest.raises(exc):
                f(**kw)
    for kw, exc in ((dict(gh=None, gw=None), sara.SaraError), (dict(gh=x["h"]), sara.SaraError), (dict(gw=x["w"]), sara.SaraError),
                    (dict(gh=gh.float()), ValueError), (dict(gw=gw.half()), TypeError), (dict(gw=gw[:50]), ValueError),
                    (dict(ent=None), sara.SaraError), (dict(stats=None), sara.SaraError),
                    (dict(gw=torch.empty((100, 68), device="cuda", dtype=torch.bfloat16)[:, :64]), sara.SaraError)):
        with pytest.raises(exc):
            bwd(**kw)


@pytest.mark.parametrize("rows,d,V", [(300, 256, 5000), BIG])
def test_reruns_are_bit_identical(env, rows, d, V):
    x = make(env, rows, d, V, "bf16")
    out = [forward(env, x) for _ in range(2)]
    assert all(env[0].equal(out[0][k], out[1][k]) for k in out[0])
    a, b = (gradients(env, x, out[0]) for _ in range(2))
    assert env[0].equal(a[0], b[0]) and env[0].equal(a[1], b[1])


LOWEST = -3.4028234663852886e38                           # finfo(float32).min


def masked_heads(env, rows, d, V, T):
    """fp32 weights whose element 0 is fp32's lowest number for the ids 1, 8, 15, ...: every row has 0.25 to 0.75 there,
    so those ids' logits are finite and count for nothing.  One hidden element is the lowest number too, where every id has 0.
    -> inputs, which ids count, the definition's results."""
    torch, _ = env
    x = make(env, rows, d, V, "f32")
    keep = torch.arange(V, device="cuda") % 7 != 1
    x["h"][:, 0] = 0.25 + 0.5 * torch.rand(rows, device="cuda", generator=torch.Generator(device="cuda").manual_seed(rows))
    x["w"][~keep, 0] = LOWEST
    x["h"][1, 3] = LOWEST
    x["w"][:, 3] = 0.0
    x["gl"][1], x["ge"][1] = 0.1, 0.01                    # dW[:, 3] = D[1] * lowest stays finite
    here = (x["tok"] >= 0) & (x["tok"] < V)
    x["tok"][here] -= (x["tok"][here] % 7 == 1).int()     # tokens that count
    number = torch.cumsum(keep, 0) - 1
    few = dict(x, w=x["w"][keep])
    few["tok"] = torch.where(here, number[x["tok"].clamp(0, V - 1).long()], torch.full_like(number[:1], -1)).int()
    e = exact(env, few, T)
    for k in ("D", "Derr"):                               # the ids that count for nothing have no D
        e[k] = torch.zeros((rows, V), device="cuda", dtype=torch.float64).index_copy_(1, keep.nonzero()[:, 0], e[k])
    e["w"] = x["w"].double()
    return x, keep, e


@pytest.mark.parametrize("rows,d,V", [(5, 64, 300), (90, 64, 300), BIG])
def test_lowest_finite_numbers(env, rows, d, V):
    """Elements past bf16's largest finite number leave everything finite, whatever the size of the call."""
    torch, _ = env
    T = 0.9
    x, keep, e = masked_heads(env, rows, d, V, T)
    out = forward(env, x, T)
    check_forward(out, e)
    gh, gw = gradients(env, x, out, T)
    check_gradients(env, gh, gw, x, e)
    assert bool((gw[~keep] == 0).all())
    # their own log probabilities, near -1e38: x is one product of 24 bits, the rest of it and log s are below its rounding
    y = dict(x, tok=torch.full_like(x["tok"], 8))
    logp = forward(env, y, T)["logp"].double()
    want = (x["h"][:, 0].double() * LOWEST - e["top"]) / T
    assert bool(((logp / want - 1).abs() <= 2.0 ** -20).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,d,V", [(90, 64, 300), BIG])
def test_largest_finite_cotangents(env, rows, d, V, dtype):
    """D past bf16's largest finite number: an fp32 call is as exact as ever; in a bf16 call D counts as that number at
    least, which is within its 2^-8.  p is below 2^-9 where it matters, so that D at the row's id keeps its size."""
    torch, _ = env
    x = make(env, rows, d, V, dtype, spread=0.25)
    x["gl"][:], x["ge"][:] = 0.0, 0.0
    x["tok"][:] = torch.arange(rows, device="cuda") % V   # one large row an id in the small call, a few in the large one
    x["gl"][7], x["gl"][rows - 1] = -LOWEST, LOWEST
    x["h"], x["w"] = x["h"] * 0.125, x["w"] * 0.125       # products below fp32's largest
    e = exact(env, x, 1.0)
    assert float(e["D"].abs().max()) > 0.995 * -LOWEST
    out = forward(env, x)
    gh, gw = gradients(env, x, out)
    check_gradients(env, gh, gw, x, e)
    if dtype == "bf16":
        check_gradients(env, *gradients(env, x, out, sums=torch.float32), x, e)


def rows_of_few_large(env, rows, d, V):
    """Rows whose D is a large element or two, each of an id that no other row has, beside 32 of a thirtieth of it and
    thousands of next to nothing: ids at 6 (the 32), at -6 and, in two rows of three, one at 9.5.
    -> inputs, rows that ask for something, ids of large elements, those among them whose p is next to nothing."""
    torch, _ = env
    g = torch.Generator(device="cuda").manual_seed(rows + V)
    dev = dict(generator=g, device="cuda")
    h, w = torch.randn((rows, d), **dev) * 0.25, torch.randn((V, d), **dev) / 16
    sinks = 37 + 151 * torch.arange(32, device="cuda")
    order = torch.randperm(V, **dev)
    order = order[~torch.isin(order, sinks)]
    tok, likely = order[:rows], order[rows:2 * rows]
    kind = torch.arange(rows, device="cuda") % 3          # log probability; entropy; both
    w[:, 0] = -6.0
    w[sinks, 0] = 6.0
    leans = kind > 0
    h[leans] = w[likely[leans]] * (15.5 * 256 / d)
    h[:, 0] = 1.0
    gl, ge = 0.5 + torch.rand(rows, **dev), 0.5 + torch.rand(rows, **dev)
    gl[kind == 1], ge[kind == 0] = 0.0, 0.0
    on = torch.arange(rows, device="cuda") % 29 != 5
    on[96:128] = False                                    # a step of 32 rows without any
    gl[~on], ge[~on] = 0.0, 0.0
    few = tok[on & (kind != 1)]
    x = dict(h=h.bfloat16(), w=w.bfloat16(), tok=tok.int(), gl=gl, ge=ge)
    return x, on, torch.cat([few, likely[on & leans]]), few


@pytest.mark.parametrize("rows,d,V", [BIG, (2500, 1000, 20001), (1100, 264, 130001)])
def test_large_elements_of_D_count_exactly(env, rows, d, V):
    """The large elements' further part, in norm: a gradient in bf16 is off by its own rounding (and a tenth of it), where one
    bf16 part of D would leave 1.2 to 1.4 times that (sqrt(2) where both roundings are independent; dH's largest column is 12
    times a row's D, whose rounding the output's partly repeats); the weight's gradient in fp32 by less than half of what two parts would.
    Both of those come from the definition with D rounded so.  Predicted: what the small elements leave adds (32 / 30^2)
    of the variance, 2%; the fp32 sums' roundings of some 160 steps in a walk are 13 x 2^-24, an eighth of two parts'
    2^-16 / sqrt(3) / 1.5.  What the products read has to be written: the workspace is full of NaN before."""
    torch, sara = env
    import ctypes
    x, on, ids, few = rows_of_few_large(env, rows, d, V)
    out = forward(env, x)
    e = exact(env, x, 1.0)
    results = {}
    for sums in (torch.bfloat16, torch.float32):
        need = ctypes.c_int64(0)
        assert sara._lib.sara_head_logprobs_workspace(1, rows, d, V, 1, int(sums == torch.bfloat16), ctypes.byref(need)) == 0
        ws = torch.full((need.value,), 255, device="cuda", dtype=torch.uint8)
        gh, results[sums] = gradients(env, x, out, sums=sums, workspace=ws)
        check_gradients(env, gh, results[sums], x, e)
    D = e["D"]
    one = D.bfloat16().double()
    two = one + (D - one).bfloat16().double()
    h, w = e["h"], e["w"]

    def off(got, want):
        return float((got.double() - want).norm())

    want, coarse = (D[on] @ w), (one[on] @ w)
    own = off(want.bfloat16(), want)
    assert off(coarse.bfloat16(), want) >= 1.2 * own
    assert off(gh[on], want) <= 1.1 * own, (off(gh[on], want) / own)
    Dt = D[:, ids].T.contiguous()
    want, coarse = Dt @ h, one[:, ids].T.contiguous() @ h
    own = off(want.bfloat16(), want)
    assert off(coarse.bfloat16(), want) >= 1.3 * own
    assert off(results[torch.bfloat16][ids], want) <= 1.1 * own, (off(results[torch.bfloat16][ids], want) / own)
    want, coarse = D[:, few].T.contiguous() @ h, two[:, few].T.contiguous() @ h
    assert off(results[torch.float32][few], want) <= 0.5 * off(coarse, want), off(results[torch.float32][few], want) / off(coarse, want)


def whole_numbers(env, rows, d, V, seed=0):
    """fp32 inputs whose products and sums are exact, so that nothing but exponentials and the gradients' sums rounds."""
    torch, _ = env
    x = make(env, rows, d, V, "f32", seed)
    x["h"], x["w"] = x["h"].round(), (x["w"] * (math.sqrt(d) / 2)).round() * 2.0 ** -round(math.log2(d) / 2)
    return x


def without_moves(x, e, T=1.0):
    """The bounds of exact logits."""
    lp, p = x["lp"], x["lp"].exp()
    gl, ge = x["gl"].double().abs(), x["ge"].double().abs()
    e["Derr"] = 2.0 ** -17 * (p * (gl[:, None] + ge[:, None] * (lp.abs() + e["ent"][:, None] + 2))) / T + 2.0 ** -22 * e["D"].abs()
    e["dx"], e["moved"] = 0 * e["dx"], 0 * e["moved"]
    return e


@pytest.mark.parametrize("exact_logits", [False, True])
def test_fp32_pieces_of_the_vocabulary(env, exact_logits):
    """The weight of 19,237 ids of width 8,192 passes in three pieces in either direction, the last of them short (37, 37 and
    2 tiles forward; 26, 26 and 24 backward), each packed in the others' place and added to dH."""
    torch, _ = env
    rows, d, V = 300, 8192, 19237
    x = whole_numbers(env, rows, d, V) if exact_logits else make(env, rows, d, V, "f32")
    e = exact(env, x, 1.0)
    if exact_logits:
        x["lp"] = torch.log_softmax(e["h"] @ e["w"].T.contiguous(), -1)
        e = without_moves(x, e)
    out = forward(env, x)
    check_forward(out, e)
    check_gradients(env, *gradients(env, x, out), x, e)


def test_fp32_pieces_and_many_rows(env):
    """Each 8,192 rows go through all pieces of the weight, packed again."""
    x = whole_numbers(env, 8300, 8192, 19237)
    e = exact(env, x, 1.0)
    e["dx"], e["moved"] = 0 * e["dx"], 0 * e["moved"]
    check_forward(forward(env, x), e)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_offsets_in_large_tiles(env, dtype):
    """A weight and its gradient whose last rows lie past 2^32 bytes, by their strides, in sizes that large tiles take."""
    torch, sara = env
    rows, d, V = 300, 1032, 70000
    x = make(env, rows, d, V, dtype)
    dt = x["w"].dtype
    big = torch.zeros((V, 32768), device="cuda", dtype=dt)
    big[:, 800:800 + d] = x["w"]
    x["w"] = big[:, 800:800 + d]
    e = exact(env, x, 1.0)
    out = forward(env, x)
    check_forward(out, e)
    far = torch.full((V, 32768), 7.0, device="cuda", dtype=dt)
    gh, gw = torch.empty_like(x["h"]), far[:, 1600:1600 + d]
    sara.sara_head_logprobs_grad(x["h"], x["w"], x["tok"], out["stats"], out["ent"], x["gl"], x["ge"], gh, gw)
    check_gradients(env, gh, gw, x, e)
    assert bool((far[:, :1600] == 7).all()) and bool((far[:, 1600 + d:] == 7).all())


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("dtype,sums", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")])
@pytest.mark.parametrize("rows,d,V", [(90, 72, 1000), (2, 72, 9000), BIG])
def test_rows_apart(env, rows, d, V, dtype, sums, accumulate):
    """Hidden states, weight and both gradients as parts of wider tensors, whose other elements stay as they are."""
    torch, sara = env
    x = make(env, rows, d, V, dtype, pad=24, wpad=40)
    e = exact(env, x, 1.0)
    out = forward(env, x)
    check_forward(out, e)
    td = torch.bfloat16 if sums == "bf16" else torch.float32
    wide_h = torch.full((rows, d + 56), 7.0, device="cuda", dtype=x["h"].dtype)
    wide_w = torch.full((V, d + 72), 7.0, device="cuda", dtype=td)
    gh, gw = wide_h[:, 16:16 + d], wide_w[:, 24:24 + d]
    gw.copy_(torch.randn((V, d), device="cuda"))
    start = gw.clone()
    sara.sara_head_logprobs_grad(x["h"], x["w"], x["tok"], out["stats"], out["ent"], x["gl"], x["ge"], gh, gw, accumulate=accumulate)
    check_gradients(env, gh, gw, x, e, start if accumulate else None)
    for wide, first in ((wide_h, 16), (wide_w, 24)):
        assert bool((wide[:, :first] == 7).all()) and bool((wide[:, first + d:] == 7).all())
