"""Token log probabilities, entropy, top alternatives and their gradient against
64 bits: vocabularies around the vector and split sizes, rows off 16 bytes,
masks that leave one id or none, ties, lowest values, NaN."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch

    import paper_2607_26253_amd as sara
    assert torch.cuda.is_available(), "GPU tests need a HIP device"
    return torch, sara


def place(torch, x, dtype, shift, pad):
    """x on the device as rows `pad` elements further apart than they are long, `shift` elements off their alignment."""
    n, V = x.shape
    flat = torch.full((n * (V + pad) + shift,), 3.0, dtype=dtype, device="cuda")
    view = flat[shift:].view(n, V + pad)[:, :V]
    view.copy_(torch.from_numpy(x))
    return view


def reference(x, tok, T, k):
    """fp64 (logp, entropy, max, sum, top ids, top logp) of rows x (fp64)."""
    n, V = x.shape
    m = x.max(1)
    with np.errstate(invalid="ignore", divide="ignore"):
        d = (x - np.where(np.isfinite(m), m, 0.0)[:, None]) / T
        e = np.exp(d)
        s = e.sum(1)
        lp = d - np.log(s)[:, None]
        p = e / s[:, None]
        H = -np.where(p > 0, p * lp, 0.0).sum(1)
    none = m == -np.inf
    H[none] = 0.0
    has = (tok >= 0) & (tok < V)
    logp = np.where(has, lp[np.arange(n), np.clip(tok, 0, V - 1)], 0.0)
    logp[none & has] = -np.inf
    ids, top = np.full((n, k), -1), np.full((n, k), -np.inf)
    for r in range(n):
        order = np.lexsort((np.arange(V), -x[r]))[:k]
        order = order[x[r, order] > -np.inf]
        ids[r, :len(order)], top[r, :len(order)] = order, lp[r, order]
    return logp, H, m, s, ids, top, lp, p


def forward(env, x, tok, T, k, **kw):
    torch, sara = env
    n = x.shape[0]
    f = dict(dtype=torch.float32, device="cuda")
    out = [torch.full((n,), 7.0, **f), torch.full((n,), 7.0, **f), torch.full((n, 2), 7.0, **f)]
    top = [torch.full((n, k), 7, dtype=torch.int32, device="cuda"), torch.full((n, k), 7.0, **f)] if k else [None, None]
    t = torch.tensor(tok, dtype=torch.int32, device="cuda")
    sara.sara_token_logprobs(x, t, *out, *top, temperature=T, **kw)
    return t, out, top


def check_forward(x, tok, T, k, out, top):
    """Each quantity is a difference of a scaled logit and a logarithm of a sum of positive terms: relative errors of
    2^-20 in the sum (fp32 sums of up to 2^18 terms in chunks, exponentials of 2^-22, c rounded: |d| / T 2^-24 on the
    weight of id d below the maximum, at most 2^-24 max(u e^-u) / u on the sum), so 2^-20 + 2^-22 (|logp| + 1) on logp
    and 2^-19 (1 + H) on the entropy."""
    logp, H, m, s, ids, lptop, _, _ = reference(x, tok, T, k)
    logp, lptop = (np.where(np.abs(a) > np.finfo(np.float32).max, -np.inf, a) for a in (logp, lptop))   # as fp32 holds them
    got = [t.double().cpu().numpy() for t in out]
    np.testing.assert_array_equal(got[2][:, 0], np.where(m == -np.inf, -np.inf, m))
    none = m == -np.inf
    assert np.all(got[2][none, 1] == 0) and np.all(np.abs(got[2][~none, 1] / s[~none] - 1) < 2.0 ** -20)
    fin = np.isfinite(logp)
    np.testing.assert_array_equal(got[0][~fin], logp[~fin])
    assert np.all(np.abs(got[0][fin] - logp[fin]) <= 2.0 ** -20 + 2.0 ** -22 * np.abs(logp[fin]))
    assert np.all(np.abs(got[1] - H) <= 2.0 ** -19 * (1 + H)), np.max(np.abs(got[1] - H))
    if k:
        np.testing.assert_array_equal(top[0].cpu().numpy(), ids)
        t = top[1].double().cpu().numpy()
        fin = np.isfinite(lptop)
        np.testing.assert_array_equal(t[~fin], lptop[~fin])
        assert np.all(np.abs(t[fin] - lptop[fin]) <= 2.0 ** -20 + 2.0 ** -22 * np.abs(lptop[fin]))


def grad_reference(x, tok, T, g, h):
    """fp64 gradient by the formula."""
    n, V = x.shape
    _, H, m, _, _, _, lp, p = reference(x, tok, T, 0)
    has = (tok >= 0) & (tok < V)
    gg = np.where(has, g, 0.0)
    plp = np.where(p > 0, p * np.where(p > 0, lp, 0.0), 0.0)
    d = -gg[:, None] * p - h[:, None] * (plp + p * H[:, None])
    d[np.arange(n)[has], tok[has]] += gg[has]
    d[(m == -np.inf) | ((gg == 0) & (h == 0))] = 0.0
    return d / T


def backward(env, x, t, out, T, g, h, dst):
    torch, sara = env
    dev = [None if a is None else torch.tensor(a, dtype=torch.float32, device="cuda") for a in (g, h)]
    sara.sara_token_logprobs_grad(x, t, out[2], out[1], *dev, dst, temperature=T)
    return dst


def check_grad(x, tok, T, g, h, got, bf16):
    """p to 2^-20 relative, log p and H to 2^-19 (1 + |.|): an element's error is at most 2^-19 of the sum of the
    magnitudes of its terms, (|g| + |h| (2 + 2 |log p| + 2 H)) p / T (and 2^-23 g / T at the token), and its rounding."""
    want = grad_reference(x, tok, T, g, h)
    _, H, _, _, _, _, lp, p = reference(x, tok, T, 0)
    lp = np.where(p > 0, lp, 0.0)
    terms = (np.abs(g)[:, None] + np.abs(h)[:, None] * (2 + 2 * np.abs(lp) + 2 * H[:, None])) * np.nan_to_num(p) / T
    n = len(x)
    has = (tok >= 0) & (tok < x.shape[1])
    terms[np.arange(n)[has], tok[has]] += np.abs(g[has]) / T
    bound = 2.0 ** -19 * terms + (2.0 ** -8 if bf16 else 2.0 ** -23) * np.abs(want) + 1e-37
    err = np.abs(got.double().cpu().numpy() - want)
    assert np.all(err <= bound), (np.max(err), np.max(err / bound))


def rows_of(rng, n, V, dtype, torch):
    x = (rng.standard_normal((n, V)) * rng.choice([0.5, 3.0, 9.0], (n, 1)) + rng.choice([0.0, -40.0, 300.0], (n, 1)))
    x[:, rng.integers(0, V, max(1, V // 50))] = -np.inf
    if n > 1:
        x[1] = 0.25                                          # every id tied
    if n > 2:
        x[2] = -np.inf                                       # nothing left
    if n > 3:
        x[3] = -np.inf
        x[3, V // 2] = -5.0                                  # one id
    if n > 4:
        x[4] = -3.3e38                                       # the type's lowest values, and
        x[4, V // 3:V // 3 + 2] = 1.0                        # two ids above them
    if n > 5:
        x[5] = -3.3895313892515355e38                        # nothing but the lowest: uniform
    if n > 6:
        x[6] = np.sort(np.nan_to_num(x[6], neginf=-50.0))    # every id a new best one
    return torch.from_numpy(x).to(torch.bfloat16 if dtype == "bf16" else torch.float32).double().numpy()


CASES = [(1, 1, 1, 0, 0), (9, 2, 3, 0, 0), (8, 7, 5, 1, 0), (9, 33, 32, 0, 1), (8, 515, 5, 3, 0), (8, 2048, 0, 0, 0),
         (8, 4097, 8, 0, 3), (3, 4096 * 3 + 5, 8, 5, 0), (1, 151936, 5, 0, 0), (2, 151936, 32, 1, 7), (9, 32016, 20, 0, 0),
         (300, 1000, 4, 0, 0), (1100, 130, 3, 0, 0), (70, 20011, 1, 0, 0), (600, 9001, 2, 0, 0)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,V,k,shift,pad", CASES)
def test_forward_and_gradient(env, n, V, k, shift, pad, dtype):
    torch, sara = env
    rng = np.random.default_rng([n, V, k])
    T = float(rng.choice([1.0, 0.7, 1.5]))
    x = rows_of(rng, n, V, dtype, torch)
    td = torch.bfloat16 if dtype == "bf16" else torch.float32
    dx = place(torch, x, td, shift, pad)
    tok = rng.integers(0, V, n).astype(np.int32)
    tok[::5] = rng.choice([-1, V, 2 ** 31 - 1], len(tok[::5]))
    t, out, top = forward(env, dx, tok, T, k)
    check_forward(x, tok, T, k, out, top)
    g, h = rng.standard_normal(n).astype(np.float32), (rng.standard_normal(n) * 0.3).astype(np.float32)
    h[::3] = 0.0
    g[::4] = 0.0
    for dshift, dpad in ((shift, pad), (shift + 1, pad + 1)):                 # alike modulo 16 bytes, and not
        dst = place(torch, np.full((n, V), 5.0), td, dshift, dpad)
        backward(env, dx, t, out, T, g, h, dst)
        check_grad(x, tok, T, g.astype(np.float64), h.astype(np.float64), dst, dtype == "bf16")
        if dpad:                                                              # nothing between the rows is touched
            whole = torch.as_strided(dst, (n - 1, dpad), (V + dpad, 1), dst.storage_offset() + V) if n > 1 else dst[:0]
            assert bool((whole == 3.0).all())
    zero = np.zeros(n)
    dst = torch.empty_like(dx)
    backward(env, dx, t, out, T, g, None, dst)
    check_grad(x, tok, T, g.astype(np.float64), zero, dst, dtype == "bf16")
    backward(env, dx, t, out, T, None, h, dst)
    check_grad(x, tok, T, zero, h.astype(np.float64), dst, dtype == "bf16")
    backward(env, dx, t, out, T, g, h, dx)                                    # in place
    check_grad(x, tok, T, g.astype(np.float64), h.astype(np.float64), dx, dtype == "bf16")


def test_gradient_against_differences(env):
    """Central differences of the fp64 forward at fp32 inputs: truncation e^2 |f'''| / 6 and rounding 1e-16 / e, both
    below 1e-9 at e = 1e-5; the kernel's own error as in check_grad."""
    torch, sara = env
    rng = np.random.default_rng(21)
    n, V, T, e = 3, 12, 0.8, 1e-5
    x = rng.standard_normal((n, V)).astype(np.float32).astype(np.float64)
    tok = np.array([3, 0, 11], np.int32)
    g, h = np.array([1.0, -0.5, 2.0], np.float32), np.array([0.3, 0.0, -0.7], np.float32)

    def f(y):
        logp, H = reference(y, tok, T, 0)[:2]
        return float((g * logp + h * H).sum())

    want = np.zeros((n, V))
    for r in range(n):
        for j in range(V):
            up, down = x.copy(), x.copy()
            up[r, j] += e
            down[r, j] -= e
            want[r, j] = (f(up) - f(down)) / (2 * e)
    np.testing.assert_allclose(grad_reference(x, tok, T, g.astype(float), h.astype(float)), want, atol=1e-8)
    dx = torch.tensor(x, dtype=torch.float32, device="cuda")
    t, out, _ = forward(env, dx, tok, T, 0)
    got = backward(env, dx, t, out, T, g, h, torch.empty_like(dx)).double().cpu().numpy()
    np.testing.assert_allclose(got, want, atol=2.0 ** -19 * 10 / T)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V,n", [(5000, 6), (5000, 600), (60000, 6)])
@pytest.mark.parametrize("k", [1, 2, 20, 32])
def test_top_ids_among_equal_logits(env, V, n, k, dtype):
    """k - 1 larger logits and 1 to 300 equal ones at rank k, among them as many as are ranked at once and one more:
    the lowest ids of the equal ones, whether a row is split or not."""
    torch, sara = env
    rng = np.random.default_rng([V, n, k])
    x = np.clip(rng.standard_normal((n, V)), -4, 4)
    for r, equal in zip(range(n), [1, 64 - (k - 1), 65 - (k - 1), 63, 300, 65] * (n // 6)):
        at = rng.permutation(V)[:k - 1 + equal]
        x[r, at] = 8.0
        x[r, at[:k - 1]] = 16.0 + np.arange(k - 1) // 2          # pairs of equal ones above too
    td = torch.bfloat16 if dtype == "bf16" else torch.float32
    dx = place(torch, x, td, 0, 0)
    t, out, top = forward(env, dx, np.zeros(n, np.int32), 1.0, k)
    check_forward(dx.double().cpu().numpy(), np.zeros(n, np.int64), 1.0, k, out, top)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_not_a_number_stays_in_its_row(env, dtype):
    torch, sara = env
    rng = np.random.default_rng(22)
    td = torch.bfloat16 if dtype == "bf16" else torch.float32
    for V in (700, 40000):
        x = rng.standard_normal((6, V))
        x[1, 5], x[3, V - 1] = np.nan, np.inf
        x[4] = np.nan
        dx = torch.tensor(x).to(td).cuda()
        tok = np.array([0, 1, 2, V - 1, 4, 5], np.int32)
        t, out, top = forward(env, dx, tok, 1.0, 4)
        bad = np.array([False, True, False, True, True, False])
        for o in out[:2]:
            np.testing.assert_array_equal(np.isnan(o.cpu().numpy()), bad)
        ids = top[0].cpu().numpy()
        assert np.all(ids[4] == -1) and np.all((ids[~bad] >= 0) & (ids[~bad] < V)) and ids[3, 0] == V - 1
        rest = np.where(np.isnan(dx[1].double().cpu().numpy()), -np.inf, dx[1].double().cpu().numpy())
        np.testing.assert_array_equal(ids[1], np.lexsort((np.arange(V), -rest))[:4])     # the best of the numbers
        g = np.ones(6, np.float32)
        dst = backward(env, dx, t, out, 1.0, g, None, torch.empty_like(dx))
        np.testing.assert_array_equal(np.isnan(dst.float().cpu().numpy()).all(1), bad)
        assert not np.isnan(dst.float().cpu().numpy()[~bad]).any()
        g[bad] = 0.0                                                          # nothing asked of those rows
        dst = backward(env, dx, t, out, 1.0, g, None, dst)
        assert np.all(dst.float().cpu().numpy()[bad] == 0)


def test_outputs_are_optional_and_streams_are_kept(env):
    torch, sara = env
    rng = np.random.default_rng(23)
    x = torch.tensor(rng.standard_normal((5, 50000)), dtype=torch.float32, device="cuda")
    t, out, top = forward(env, x, np.arange(5, dtype=np.int32), 1.0, 6)
    again = torch.empty(5, device="cuda")
    sara.sara_token_logprobs(x, t, again)
    assert torch.equal(again, out[0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    ids, lps = torch.empty_like(top[0]), torch.empty_like(top[1])
    sara.sara_token_logprobs(x, t, None, None, None, ids, lps, stream=side)
    side.synchronize()
    assert torch.equal(ids, top[0]) and torch.equal(lps, top[1])
    sara.sara_token_logprobs(x[:0], t[:0], again[:0])                          # no rows


def test_rows_past_32_bits(env):
    """Logits of more than 2^32 elements, rows far apart: offsets are 64-bit."""
    torch, sara = env
    V, stride = 1001, 1 << 20
    flat = torch.zeros(4100 * stride, dtype=torch.bfloat16, device="cuda")
    x = flat.view(4100, stride)[:, :V]
    rows = torch.randn((4, V), device="cuda").to(torch.bfloat16)
    x[-4:] = rows
    t = torch.arange(4100, dtype=torch.int32, device="cuda") % V
    logp, stats = torch.empty(4100, device="cuda"), torch.empty((4100, 2), device="cuda")
    sara.sara_token_logprobs(x, t, logp, None, stats)
    want, st = torch.empty(4, device="cuda"), torch.empty((4, 2), device="cuda")
    sara.sara_token_logprobs(rows, t[-4:].contiguous(), want, None, st)
    torch.testing.assert_close(logp[-4:], want, rtol=0, atol=2e-6)
    g = torch.ones(4100, device="cuda")
    sara.sara_token_logprobs_grad(x, t, stats, None, g, None, x)
    small = torch.empty_like(rows)
    sara.sara_token_logprobs_grad(rows, t[-4:].contiguous(), st, None, g[:4], None, small)
    torch.testing.assert_close(x[-4:].float(), small.float(), rtol=2.0 ** -7, atol=0)
    assert bool((flat.view(4100, stride)[:, V:V + 64] == 0).all())


def test_refusals(env):
    torch, sara = env
    x = torch.zeros((3, 40000), device="cuda")
    t = torch.zeros(3, dtype=torch.int32, device="cuda")
    logp, stats = torch.empty(3, device="cuda"), torch.empty((3, 2), device="cuda")
    ids, lps = torch.empty((3, 33), dtype=torch.int32, device="cuda"), torch.empty((3, 33), device="cuda")
    with pytest.raises(sara.SaraError):
        sara.sara_token_logprobs(x, t, logp, d_top_id=ids, d_top_logp=lps)          # more than 32
    for T in (0.0, -1.0, float("nan"), float("inf")):
        with pytest.raises(sara.SaraError):
            sara.sara_token_logprobs(x, t, logp, temperature=T)
    with pytest.raises(TypeError):
        sara.sara_token_logprobs(x.half(), t, logp)
    with pytest.raises(ValueError):
        sara.sara_token_logprobs(x, t.long(), logp)
    with pytest.raises(ValueError):
        sara.sara_token_logprobs(x, t, logp[:2])
    with pytest.raises(ValueError):
        sara.sara_token_logprobs(x.t(), t, logp)
    with pytest.raises(ValueError):
        sara.sara_token_logprobs(x, t, logp, d_top_id=ids)
    with pytest.raises(sara.SaraError):
        sara.sara_token_logprobs(x, t, logp, workspace=torch.empty(4, dtype=torch.uint8, device="cuda"))
    with pytest.raises(ValueError):
        sara.sara_token_logprobs_grad(x, t, stats, None, logp, None, torch.empty_like(x)[:, :-1])
    with pytest.raises(sara.SaraError):                                              # entropy gradient without the entropy
        sara.sara_token_logprobs_grad(x, t, stats, None, logp, logp, torch.empty_like(x))
    with pytest.raises(TypeError):
        sara.sara_token_logprobs_grad(x, t, stats, None, logp, None, torch.empty_like(x, dtype=torch.float16))
    torch.cuda.synchronize()


# -- temperatures -------------------------------------------------------------------
def spread_rows(rng, T, V, dtype, torch):
    """Rows whose z = x / T are ordinary at any temperature: normal ones, one with ids masked by -inf and by the type's
    lowest value, a tied one, and one that a single id is left of."""
    top = np.float64(3.38e38)
    x = np.clip(rng.standard_normal((5, V)) * 3.0 * T, -top, top)
    x[1, ::3], x[1, 1::3] = -np.inf, -top
    x[2] = T
    x[3] = -np.inf
    x[3, V // 2] = -T
    x[4] *= 4.0
    return torch.from_numpy(np.clip(x, -np.inf, top)).to(torch.bfloat16 if dtype == "bf16" else torch.float32).double().numpy()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [1.01e-37, 1e-20, 3e-12, 1e-9, 1e-3, 1e4, 1e12, 1e18, 3e25, 1e33])
def test_gradient_over_the_temperatures(env, T, dtype):
    """Statistics of 64 bits, so that the gradient alone is looked at.  An element's error: p relative to 2^-19 (fp32) or,
    of bf16 logits, |u| 2^-23 with |u| < 150: 2^-15, of the sum of the magnitudes of its terms; exponentials below 2^-126
    may count as 0, at which |log p| is at most 104; its rounding; and subnormal results (2^-126)."""
    torch, sara = env
    rng = np.random.default_rng(31)
    T = float(np.float32(T))
    for V, shift in ((37, 0), (2051, 1)):
        x = spread_rows(rng, T, V, dtype, torch)
        n, bf16 = len(x), dtype == "bf16"
        dx = place(torch, x, torch.bfloat16 if bf16 else torch.float32, shift, 0)
        tok = np.array([3, 1, 5, V // 2, -1])
        _, H, m, s, _, _, lp, p = reference(x, tok, T, 0)
        f = dict(dtype=torch.float32, device="cuda")
        stats = torch.tensor(np.stack([m, s], 1), **f)
        t, ent = torch.tensor(tok, dtype=torch.int32, device="cuda"), torch.tensor(H, **f)
        g, h = np.array([1.0, -0.5, 2.0, 1.0, 0.5]), np.array([0.5, 1.0, -1.0, 0.3, 1.0])
        lp, has = np.where(p > 0, lp, 0.0), tok >= 0
        for gg, hh in ((g, h), (0 * g, h), (g, 0 * h)):
            want = grad_reference(x, tok, T, gg, hh)
            dst = torch.full_like(dx, 5.0)
            backward(env, dx, t, (None, ent, stats), T, gg, hh, dst)
            got = dst.double().cpu().numpy()
            size = np.abs(gg)[:, None] + np.abs(hh)[:, None] * (2 + 2 * np.minimum(np.abs(lp), 104.0) + 2 * H[:, None])
            terms = size * p / T
            terms[np.arange(n)[has], tok[has]] += np.abs(gg[has]) / T
            bound = ((2.0 ** -15 if bf16 else 2.0 ** -19) * terms + 2.0 ** -126 * (1 + size / T) +
                     (2.0 ** -8 if bf16 else 2.0 ** -23) * np.abs(want))
            err = np.abs(got - want)
            assert np.all(err <= bound), (V, np.nanmax(err / bound), int(np.isnan(err).sum()))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [1.01e-37, 1e-20, 1e-3, 1e12, 1e33, 9.9e36])
def test_forward_over_the_temperatures(env, T, dtype):
    """The bounds of check_forward: they are relative to z = x / T.  An id of probability below 2^-126 may count as 0 in
    the entropy (2^-126 104 V, beside them)."""
    torch, sara = env
    rng = np.random.default_rng(32)
    T = float(np.float32(T))
    for V, k, shift in ((37, 5, 0), (2051, 3, 1), (50000, 8, 0)):
        x = spread_rows(rng, T, V, dtype, torch)
        dx = place(torch, x, torch.bfloat16 if dtype == "bf16" else torch.float32, shift, 0)
        tok = np.array([3, 1, 5, V // 2, -1])
        _, out, top = forward(env, dx, tok, T, k)
        check_forward(x, tok, T, k, out, top)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_logits_further_apart_than_the_largest_number(env, dtype):
    """x - max overflows although z = x / T is ordinary: the log probability is what the definition gives."""
    torch, sara = env
    T = float(np.float32(9.9e36))
    x = np.full((3, 900), -3.3e38)
    x[:, 7] = 3.3e38
    x[1, 9:400] = np.linspace(-2e38, 2e38, 391)
    x[2] = -x[2]
    x = torch.from_numpy(x).to(torch.bfloat16 if dtype == "bf16" else torch.float32).double().numpy()
    dx = place(torch, x, torch.bfloat16 if dtype == "bf16" else torch.float32, 0, 0)
    tok = np.array([0, 2, 7])
    _, out, top = forward(env, dx, tok, T, 6)
    check_forward(x, tok, T, 6, out, top)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [700, 40000])
def test_a_signalling_nan_hides_no_other_id(env, V, dtype):
    """NaN of every kind (quiet and signalling, of both signs) beside the row's best logits: the row is NaN, the top ids
    are the best of its numbers, and its largest logit is one of them."""
    torch, sara = env
    rng = np.random.default_rng(33)
    x = np.clip(rng.standard_normal((8, V)), -4, 4)
    best = [rng.permutation(V // 8 - 1)[:6] * 8 for _ in x]
    for r, at in enumerate(best):
        x[r, at] = 9.0 + np.arange(6)
    td, kinds = (torch.bfloat16, [0x7F81, -0x7F, 0x7FC0, -0x40]) if dtype == "bf16" else (torch.float32, [0x7F800001, -0x7FFFFF, 0x7FC00000, -1])
    dx = torch.tensor(x).to(td).cuda()
    bits = dx.view(torch.int16 if dtype == "bf16" else torch.int32)
    for r, at in enumerate(best):
        bits[r, torch.tensor(at + 1 + r % 7)] = kinds[r % 4]     # close by each of the best
    assert bool((dx.isnan().sum(1) == 6).all())
    t, out, top = forward(env, dx, np.zeros(8, np.int32), 1.0, 6)
    assert bool(out[0].isnan().all()) and bool(out[1].isnan().all())
    for r, at in enumerate(best):
        assert top[0][r].tolist() == at[::-1].tolist(), r
    np.testing.assert_array_equal(out[2][:, 0].cpu().numpy(), 14.0)


def test_autograd_notices_what_a_call_writes(env):
    """Every output's version rises, no input's; a backward pass that needs logits which the gradient has replaced raises;
    tensors of inference mode, which have no version, serve as ever."""
    torch, sara = env
    w = torch.randn((3, 500), device="cuda", requires_grad=True)
    logits = w * 2.0
    loss = (logits * logits).sum()                          # saves the logits
    x, tok = logits.detach(), torch.tensor([1, 2, 3], dtype=torch.int32, device="cuda")
    out = [torch.empty(s, device="cuda") for s in (3, 3, (3, 2))]
    top = [torch.empty((3, 4), dtype=torch.int32, device="cuda"), torch.empty((3, 4), device="cuda")]
    g = torch.ones(3, device="cuda")

    def risen(call, written, read):
        before = [t._version for t in written + read]
        call()
        after = [t._version for t in written + read]
        assert [b > a for a, b in zip(before, after)] == [True] * len(written) + [False] * len(read)

    risen(lambda: sara.sara_token_logprobs(x, tok, *out, *top), out + top, [x, tok])
    risen(lambda: sara.sara_token_logprobs_grad(x, tok, out[2], out[1], g, g, x), [x], out + [tok, g])
    with pytest.raises(RuntimeError, match="inplace"):
        loss.backward()
    hkv, hd = 2, 64
    codes = [torch.zeros((4, hkv, 16, hd), dtype=torch.int8, device="cuda") for _ in range(2)]
    exps = [torch.zeros((4, hkv), dtype=torch.uint8, device="cuda") for _ in range(2)]
    k, v, q, o = (torch.randn((1, h, hd), device="cuda") for h in (hkv, hkv, 4, 4))
    pages, one, zero = (torch.tensor(a, dtype=torch.int32, device="cuda") for a in ([[0, 1]], [1], [0]))
    off = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    risen(lambda: sara.sara_kv8_write(*codes, *exps, k, v, pages, zero), codes + exps, [k, v, pages])
    risen(lambda: sara.sara_kv8_read(*codes, *exps, pages, zero, off, k, v), [k, v], codes + exps)
    risen(lambda: sara.sara_kv8_attention(q, *codes, *exps, pages, one, None, o), [o], codes + exps + [q])
    with torch.inference_mode():
        kept = torch.empty(3, device="cuda")
    sara.sara_token_logprobs(w.detach(), tok, kept)
    torch.testing.assert_close(kept, torch.log_softmax(w.detach(), -1)[torch.arange(3), [1, 2, 3]], rtol=0, atol=1e-5)


def test_strides_of_single_rows_and_ids_do_not_matter(env):
    torch, sara = env
    x = torch.randn(700, device="cuda")
    tok, one = torch.tensor([3], dtype=torch.int32, device="cuda"), torch.ones(1, device="cuda")
    logp, stats = torch.empty(1, device="cuda"), torch.empty((1, 2), device="cuda")
    row = x.as_strided((1, 700), (5, 1))
    sara.sara_token_logprobs(row, tok, logp, None, stats)
    torch.testing.assert_close(logp[0], torch.log_softmax(x, 0)[3], rtol=0, atol=1e-5)
    want = torch.empty_like(row)
    sara.sara_token_logprobs_grad(row, tok, stats, None, one, None, want)
    sara.sara_token_logprobs_grad(row, tok, stats, None, one, None, x.as_strided((1, 700), (9, 1)))       # in place
    assert torch.equal(x, want[0])
    ids, out = torch.zeros(4, dtype=torch.int32, device="cuda"), torch.empty(4, device="cuda")
    sara.sara_token_logprobs(torch.randn(4, device="cuda").as_strided((4, 1), (1, 7)), ids, out)          # a vocabulary of one
    assert out.tolist() == [0.0] * 4


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_more_rows_than_a_grid_is_high(env, dtype):
    """Rows go to the launches in chunks of 65,535."""
    torch, sara = env
    rng = np.random.default_rng(34)
    n, V, k = 65535 + 700, 23, 3
    x = rows_of(rng, n, V, dtype, torch)
    td = torch.bfloat16 if dtype == "bf16" else torch.float32
    dx = place(torch, x, td, 1, 2)
    tok = rng.integers(-1, V + 1, n).astype(np.int32)
    t, out, top = forward(env, dx, tok, 0.8, k)
    check_forward(x, tok, 0.8, k, out, top)
    g, h = rng.standard_normal(n).astype(np.float32), (rng.standard_normal(n) * 0.3).astype(np.float32)
    for shift in (1, 0):
        dst = place(torch, np.full((n, V), 5.0), td, shift, 2)
        backward(env, dx, t, out, 0.8, g, h, dst)
        check_grad(x, tok, 0.8, g.astype(np.float64), h.astype(np.float64), dst, dtype == "bf16")


@pytest.mark.parametrize("n,V,k", [(2, 60000, 5), (600, 3000, 4)])
def test_graph_replay(env, n, V, k):
    """Log probabilities and gradient captured in a HIP graph (rows in splits with a join, and whole), replayed on other
    logits with eager calls between the replays."""
    torch, sara = env
    x, tok = torch.empty((n, V), dtype=torch.bfloat16, device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda")
    f = dict(device="cuda", dtype=torch.float32)
    outs = [torch.empty(n, **f), torch.empty(n, **f), torch.empty((n, 2), **f), torch.empty((n, k), dtype=torch.int32, device="cuda"),
            torch.empty((n, k), **f), torch.empty_like(x)]
    g, h, ws = torch.randn(n, **f), torch.randn(n, **f), torch.empty(1 << 20, dtype=torch.uint8, device="cuda")

    def step():
        sara.sara_token_logprobs(x, tok, *outs[:5], temperature=0.7, workspace=ws)
        sara.sara_token_logprobs_grad(x, tok, outs[2], outs[1], g, h, outs[5], temperature=0.7)

    x.normal_()
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        x.copy_(torch.randn((n, V), device="cuda") * 3)
        tok.copy_(torch.randint(0, V, (n,), device="cuda"))
        for o in outs:
            o.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = [o.clone() for o in outs]
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, outs)), i
        lp = torch.log_softmax(x.double() / 0.7, -1)[torch.arange(n), tok.long()]
        torch.testing.assert_close(got[0].double(), lp, rtol=2.0 ** -20, atol=2.0 ** -19)
