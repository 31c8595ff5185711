"""Performance cases of the 8-bit KV cache and of token log probabilities.

kind "write"   K and V of new tokens are quantised into a paged 8-bit cache
               (one power-of-two scale for each page of 16 tokens and head) and
               the pages that changed are read back
kind "attend"  attention of new tokens' queries over such a cache
kind "score"   log probabilities of given tokens with entropy and the most
               likely alternatives and, where `train` is set, the gradient with
               respect to the logits

`own` chooses between the plain forms (elementary torch operations in 32 bits)
and the package's entry points.  Sizes come from the package's workloads (the
1.5B- and 3B-shaped decoders, the tiny fp32 one) or are generic.
"""
import math

import torch

own = False

PAGE = 16
INT8_MAX, FP8_MAX = 127.0, 448.0


# ---------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------
def _write(seqs, new_lo, new_hi, start_lo, start_hi, hkv, hd, fmt, dtype):
    return dict(kind="write", seqs=seqs, new_lo=new_lo, new_hi=new_hi, start_lo=start_lo, start_hi=start_hi, hkv=hkv, hd=hd,
                fmt=fmt, dtype=dtype)


def _attend(seqs, q_lo, q_hi, before_lo, before_hi, hq, hkv, hd, fmt, dtype):
    return dict(kind="attend", seqs=seqs, q_lo=q_lo, q_hi=q_hi, before_lo=before_lo, before_hi=before_hi, hq=hq, hkv=hkv,
                hd=hd, fmt=fmt, dtype=dtype)


def _score(rows, vocab, dtype, temperature, top, train):
    return dict(kind="score", rows=rows, vocab=vocab, dtype=dtype, temperature=temperature, top=top, train=train)


FULL_V = 151936


def listed():
    return [
        # one interactive rollout appends a token to a part-filled page
        dict(name="append_one", **_write(1, 1, 1, 333, 333, 2, 128, "int8", "bf16")),
        # a decode step of 512 slots appends a token each, anywhere in their pages
        dict(name="append_512_rows", **_write(512, 1, 1, 256, 1700, 2, 128, "fp8", "bf16")),
        # a step's prompt pool is written whole: 256 ragged prompts
        dict(name="write_pool", **_write(256, 128, 512, 0, 0, 2, 128, "int8", "bf16")),
        # one interactive rollout attends: latency
        dict(name="attend_one_row", **_attend(1, 1, 1, 332, 332, 12, 2, 128, "int8", "bf16")),
        # the benchmark's decode regime at the contexts of long rollouts
        dict(name="attend_32_rows", **_attend(32, 1, 1, 3001, 4590, 12, 2, 128, "int8", "bf16")),
        # a full pool step of the 3B width
        dict(name="attend_512_rows", **_attend(512, 1, 1, 256, 1700, 16, 2, 128, "fp8", "bf16")),
        # one long document: the context is the only axis to share out
        dict(name="attend_long", **_attend(1, 1, 1, 65536, 65536, 16, 2, 128, "int8", "bf16")),
        # few long prompts attend to themselves as they are written
        dict(name="attend_prompts", **_attend(3, 1100, 4590, 0, 0, 16, 2, 128, "int8", "bf16")),
        # the tiny fp32 decoder re-reads ragged pieces of its rollouts
        dict(name="attend_pieces_f32", **_attend(64, 1, 33, 0, 63, 4, 4, 64, "fp8", "f32")),
        # one sampled token with its alternatives
        dict(name="score_one_row", **_score(1, FULL_V, "bf16", 1.0, 5, False)),
        # tokens of a decode step scored from fp32 logits
        dict(name="score_512_rows", **_score(512, FULL_V, "f32", 0.7, 8, False)),
        # a micro-batch of the policy update: log probabilities, entropy, gradient
        dict(name="train_2048_rows", **_score(2048, FULL_V, "bf16", 1.0, 0, True)),
    ]


def _log(rng, lo, hi):
    """An integer of [lo, hi], spread over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5)))))))


def draw(rng):
    """One more case of the listed ones' ranges."""
    while True:
        kind = rng.choice(["append", "write", "decode", "decode", "prompts", "pieces", "score", "train"])
        fmt, dtype = rng.choice(["int8", "fp8"]), rng.choice(["bf16", "bf16", "bf16", "f32"])
        hkv, hd = rng.choice([(2, 128), (2, 128), (1, 128), (8, 128), (4, 64), (2, 64)])
        hq = hkv * rng.choice([1, 2, 4, 5, 6, 7, 8])
        if kind == "append":
            lo = rng.randint(0, 1700)
            case = _write(_log(rng, 1, 512), 1, 1, lo, lo + _log(rng, 1, 1500), hkv, hd, fmt, dtype)
        elif kind == "write":
            lo, start = _log(rng, 1, 400), rng.choice([0, 0, rng.randint(1, 300)])
            case = _write(_log(rng, 1, 256), lo, _log(rng, lo, 4 * lo), start, start + rng.choice([0, 13]), hkv, hd, fmt, dtype)
        elif kind == "decode":
            lo = _log(rng, 1, 65536)
            case = _attend(_log(rng, 1, 512), 1, rng.choice([1, 1, 1, 2]), lo, min(65536, _log(rng, lo, 4 * lo)), hq, hkv, hd,
                           fmt, dtype)
        elif kind == "prompts":
            lo = _log(rng, 16, 3000)
            case = _attend(_log(rng, 1, 64), lo, min(4590, _log(rng, lo, 3 * lo)), 0, 0, hq, hkv, hd, fmt, dtype)
        elif kind == "pieces":
            lo = _log(rng, 1, 100)
            case = _attend(_log(rng, 1, 64), lo, _log(rng, lo, 4 * lo), 0, _log(rng, 1, 6000), hq, hkv, hd, fmt, dtype)
        else:
            case = _score(_log(rng, 1, 2048), rng.choice([_log(rng, 500, FULL_V), FULL_V, 32016]), dtype,
                          rng.choice([1.0, 0.7, 1.3]), rng.choice([0, 1, 5, 8, 20]), kind == "train")
        w = work(case)
        if case["kind"] == "score":
            if w["bytes"] <= 1.8e9:
                return case
        elif w["bytes"] <= 2.6e8 and w["flops"] <= 1.2e11 and _plain_scores(case) <= 1e9:
            return case


def _spread(lo, hi, n):
    """n lengths evenly over [lo, hi]."""
    return [lo + (hi - lo) * i // max(1, n - 1) for i in range(n)]


def _lengths(case):
    """(new tokens, tokens before them) of each sequence."""
    n = case["seqs"]
    if case["kind"] == "write":
        return _spread(case["new_lo"], case["new_hi"], n), _spread(case["start_lo"], case["start_hi"], n)[::-1]
    return _spread(case["q_lo"], case["q_hi"], n), _spread(case["before_lo"], case["before_hi"], n)[::-1]


def _plain_scores(case):
    if case["kind"] != "attend":
        return 0
    new, before = _lengths(case)
    return case["seqs"] * max(new) * case["hq"] * max(a + b for a, b in zip(new, before))


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _offsets(lengths):
    off = [0]
    for n in lengths:
        off.append(off[-1] + n)
    return off


def _cache(case, lengths, g):
    """A cache with every page filled, and page tables over it in no order (-1 past a sequence's end)."""
    hkv, hd = case["hkv"], case["hd"]
    counts = [-(-n // PAGE) for n in lengths]
    total = sum(counts) + 3
    order = torch.randperm(total, generator=g, device="cuda").to(torch.int32)
    at, wide = _i32(_offsets(counts)[:-1]), torch.arange(max(counts), device="cuda", dtype=torch.int32)
    have = wide[None, :] < _i32(counts)[:, None]
    pages = torch.where(have, order[(at[:, None] + wide[None, :]).clamp(max=total - 1).long()], torch.full_like(wide, -1))

    def codes():
        x = torch.randn((total, hkv, PAGE, hd), generator=g, device="cuda")
        if case["fmt"] == "int8":
            return (x * 30.0).round().clamp(-INT8_MAX, INT8_MAX).to(torch.int8)
        return (x * 100.0).clamp(-FP8_MAX, FP8_MAX).to(torch.float8_e4m3fn)

    def exponents():       # values of about 1, pages up to 8 times larger
        e = torch.randint(0, 4, (total, hkv), generator=g, device="cuda")
        return (e + (121 if case["fmt"] == "int8" else 119)).to(torch.uint8)

    return dict(k_cache=codes(), v_cache=codes(), k_exp=exponents(), v_exp=exponents(), pages=pages.contiguous())


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed) * 7919 + 17)
    dt = _dtype(case)

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    if case["kind"] == "score":
        n, V = case["rows"], case["vocab"]
        logits = normal(n, V).mul_(2.5)
        logits[:, V - V // 500:] = -math.inf                 # ids that the tokenizer does not use
        logits = logits.to(dt)
        tok = torch.randint(0, V - V // 500, (n,), generator=g, device="cuda", dtype=torch.int32)
        tok[::17] = -1 if n > 17 else tok[::17]              # padding of a ragged batch
        f32 = dict(device="cuda", dtype=torch.float32)
        st = dict(case=case, logits=logits, tok=tok, g_logp=normal(n), g_ent=normal(n) * 0.01, logp=torch.empty(n, **f32),
                  ent=torch.empty(n, **f32), stats=torch.empty((n, 2), **f32),
                  top_id=torch.empty((n, case["top"]), device="cuda", dtype=torch.int32),
                  top_logp=torch.empty((n, case["top"]), **f32))
        if case["train"]:
            st["grad"] = torch.empty_like(logits)
        return st
    new, before = _lengths(case)
    st = dict(case=case, **_cache(case, [a + b for a, b in zip(new, before)], g))
    off, total = _offsets(new), sum(new)
    single = max(new) == 1
    hkv, hd = case["hkv"], case["hd"]
    if case["kind"] == "write":
        # keys have channels an order of magnitude above the others; both tensors are parts of one projection
        gain = 1.0 + 9.0 * (torch.rand(hd, generator=g, device="cuda") < 0.03)
        qkv = torch.cat([normal(total, hkv, hd) * gain, normal(total, hkv, hd)], 1).to(dt)
        first = [b - b % PAGE for b in before]               # read back from the first page that changes
        back = [a + b - f for a, b, f in zip(new, before, first)]
        st.update(k=qkv[:, :hkv], v=qkv[:, hkv:], start=_i32(before), off=None if single else _i32(off),
                  read_start=_i32(first), read_off=_i32(_offsets(back)),
                  read_k=torch.empty((sum(back), hkv, hd), device="cuda", dtype=dt),
                  read_v=torch.empty((sum(back), hkv, hd), device="cuda", dtype=dt))
        return st
    st.update(q=(normal(total, case["hq"], hd) * 2.0).to(dt), ctx=_i32([a + b for a, b in zip(new, before)]),
              off=None if single else _i32(off), max_q=max(new), max_ctx=max(a + b for a, b in zip(new, before)),
              out=torch.empty((total, case["hq"], hd), device="cuda", dtype=dt))
    return st


# ---------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------
def _scale(exp):
    """2^(b - 127), NaN for b = 255."""
    s = (exp.to(torch.int32) << 23).view(torch.float32)
    return torch.where(exp == 255, torch.full_like(s, math.nan), s)


def _inverse(exp):
    return ((254 - exp.to(torch.int32)) << 23).view(torch.float32)


def _exponent(amax, fmt):
    """The smallest b >= 1 with amax <= 127 (448) * 2^(b - 127); 255 where amax is not finite."""
    up, down = (0x1FFFF, 6) if fmt == "int8" else (0x1FFFFF, 8)
    b = ((amax.view(torch.int32) + up) >> 23) - down
    return torch.where(torch.isfinite(amax), b.clamp(min=1), torch.full_like(b, 255))


def _encode(x, fmt):
    """x in codes, as bytes."""
    return x.round().to(torch.int8) if fmt == "int8" else x.to(torch.float8_e4m3fn).view(torch.int8)


def _decode(bytes_, fmt):
    return (bytes_ if fmt == "int8" else bytes_.view(torch.float8_e4m3fn)).float()


def _rows(off, single, total, starts):
    """(sequence, position) of each row."""
    row = torch.arange(total, device="cuda")
    if single:
        return row, starts.long()
    seq = torch.searchsorted(off.long(), row, right=True) - 1
    return seq, starts.long()[seq] + row - off.long()[seq]


def _plain_write(st):
    fmt, pages = st["case"]["fmt"], st["pages"].long()
    seq, pos = _rows(st["off"], st["off"] is None, st["k"].shape[0], st["start"])
    page, slot = pages[seq, pos // PAGE], pos % PAGE
    start = st["start"].long()
    kept = start % PAGE != 0                                 # the first page keeps its earlier tokens
    head = pages.gather(1, (start // PAGE)[:, None])[:, 0]
    for x, cache, exp in ((st["k"], st["k_cache"], st["k_exp"]), (st["v"], st["v_cache"], st["v_exp"])):
        x, cache = x.float(), cache.view(torch.int8)
        amax = x.abs().amax(-1)
        amax = torch.where(torch.isfinite(amax), amax, torch.full_like(amax, math.inf))
        most = torch.zeros(exp.shape, device="cuda").index_reduce_(0, page, amax, "amax")
        b = _exponent(most, fmt)
        old = exp[head].to(torch.int32)
        b[head] = torch.where(kept[:, None], torch.maximum(b[head], old), b[head])
        shift = torch.where(kept[:, None], _scale(old) * _inverse(b[head]), torch.ones_like(old, dtype=torch.float32))
        cache[head] = _encode(_decode(cache[head], fmt) * shift[..., None, None], fmt)
        cache[page, :, slot] = _encode(x * _inverse(b[page])[..., None], fmt)
        exp[page] = b[page].to(torch.uint8)
    return _plain_read(st)


def _plain_read(st):
    seq, pos = _rows(st["read_off"], False, st["read_k"].shape[0], st["read_start"])
    page, slot = st["pages"].long()[seq, pos // PAGE], pos % PAGE
    dt, fmt = st["read_k"].dtype, st["case"]["fmt"]

    def values(cache, exp):
        return (_decode(cache.view(torch.int8)[page, :, slot], fmt) * _scale(exp[page])[..., None]).to(dt)

    return {"k": values(st["k_cache"], st["k_exp"]), "v": values(st["v_cache"], st["v_exp"])}


def _plain_attend(st):
    q, pages, ctx = st["q"].float(), st["pages"], st["ctx"].long()
    total, hq, hd = q.shape
    n, hkv, T = pages.shape[0], st["case"]["hkv"], st["max_q"]
    G, S = hq // hkv, pages.shape[1] * PAGE
    page = pages.clamp(min=0).long()

    def values(cache, exp):
        x = _decode(cache.view(torch.int8)[page], st["case"]["fmt"]) * _scale(exp[page])[..., None, None]
        return x.transpose(1, 2).reshape(n, hkv, S, hd)

    k, v = values(st["k_cache"], st["k_exp"]), values(st["v_cache"], st["v_exp"])
    row = torch.arange(total, device="cuda")
    if st["off"] is None:
        seq, t, new = row, torch.zeros_like(row), torch.ones_like(ctx)
    else:
        off = st["off"].long()
        seq = torch.searchsorted(off, row, right=True) - 1
        t, new = row - off[seq], off[1:] - off[:-1]
    qp = torch.zeros((n, T, hq, hd), device="cuda")
    qp[seq, t] = q
    qp = qp.view(n, T, hkv, G, hd).permute(0, 2, 3, 1, 4).reshape(n, hkv, G * T, hd)
    s = (torch.matmul(qp, k.transpose(2, 3).contiguous()) * (1.0 / math.sqrt(hd))).view(n, hkv, G, T, S)
    at = torch.arange(S, device="cuda")
    last = (ctx - new)[:, None] + torch.arange(T, device="cuda")
    seen = (at <= torch.minimum(last, ctx[:, None] - 1)[..., None]) & (pages >= 0).repeat_interleave(PAGE, 1)[:, None]
    s = torch.where(seen[:, None, None], s, torch.full_like(s[:1, :1, :1, :1, :1], -math.inf))
    most = s.amax(-1, keepdim=True)
    s = torch.exp(s - torch.where(torch.isfinite(most), most, torch.zeros_like(most)))
    den = s.sum(-1, keepdim=True)
    o = torch.matmul(s.view(n, hkv, G * T, S), v).view(n, hkv, G, T, hd)
    o = torch.where(den > 0, o / den, torch.zeros_like(o))
    return {"out": o.permute(0, 3, 1, 2, 4).reshape(n, T, hq, hd)[seq, t].to(st["q"].dtype)}


def _plain_score(st):
    case, x = st["case"], st["logits"].float()
    n, V = x.shape
    z = x / case["temperature"]
    most = z.amax(-1, keepdim=True)
    e = torch.exp(z - most)
    tot = e.sum(-1, keepdim=True)
    lse = most + torch.log(tot)
    tok = st["tok"].long()
    has = (tok >= 0) & (tok < V)
    logp = torch.where(has, z.gather(1, tok.clamp(0, V - 1)[:, None])[:, 0] - lse[:, 0], torch.zeros_like(lse[:, 0]))
    lp = torch.where(torch.isfinite(z), z - lse, torch.zeros_like(z))
    p = e / tot
    ent = -(p * lp).sum(-1)
    out = {"logp": logp, "entropy": ent, "max": x.amax(-1), "sum": tot[:, 0]}
    if case["top"]:
        # a unique key for each id: the logit's order, the lower id first
        bits = x.view(torch.int32).long()
        order = torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits)
        key = order * (1 << 20) + (V - 1 - torch.arange(V, device="cuda"))
        top = V - 1 - (torch.topk(key, case["top"], dim=-1).values & ((1 << 20) - 1))
        out["top_id"], out["top_logp"] = top.to(torch.int32), z.gather(1, top) - lse
    if case["train"]:
        g = torch.where(has, st["g_logp"], torch.zeros_like(st["g_logp"]))
        grad = p * (-g[:, None] - st["g_ent"][:, None] * (lp + ent[:, None]))
        grad[torch.arange(n, device="cuda"), tok.clamp(0, V - 1)] += g
        out["grad"] = (grad / case["temperature"]).to(st["logits"].dtype)
    return out


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def run(state):
    st, case = state, state["case"]
    if not own:
        return {"write": _plain_write, "attend": _plain_attend, "score": _plain_score}[case["kind"]](st)
    import paper_2607_26253_amd as sara
    if case["kind"] == "write":
        cache = (st["k_cache"], st["v_cache"], st["k_exp"], st["v_exp"])
        sara.sara_kv8_write(*cache, st["k"], st["v"], st["pages"], st["start"], st["off"])
        sara.sara_kv8_read(*cache, st["pages"], st["read_start"], st["read_off"], st["read_k"], st["read_v"])
        return {"k": st["read_k"], "v": st["read_v"]}
    if case["kind"] == "attend":
        sara.sara_kv8_attention(st["q"], st["k_cache"], st["v_cache"], st["k_exp"], st["v_exp"], st["pages"], st["ctx"],
                                st["off"], st["out"], max_ctx=st["max_ctx"])
        return {"out": st["out"]}
    out = {"logp": st["logp"], "entropy": st["ent"], "max": st["stats"][:, 0], "sum": st["stats"][:, 1]}
    top = {}
    if case["top"]:
        top = {"d_top_id": st["top_id"], "d_top_logp": st["top_logp"]}
        out["top_id"], out["top_logp"] = st["top_id"], st["top_logp"]
    sara.sara_token_logprobs(st["logits"], st["tok"], st["logp"], st["ent"], st["stats"], temperature=case["temperature"], **top)
    if case["train"]:
        sara.sara_token_logprobs_grad(st["logits"], st["tok"], st["stats"], st["ent"], st["g_logp"], st["g_ent"], st["grad"],
                                      temperature=case["temperature"])
        out["grad"] = st["grad"]
    return out


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------
def work(case):
    E = 2.0 if case["dtype"] == "bf16" else 4.0
    if case["kind"] == "score":
        n, V = case["rows"], case["vocab"]
        return {"bytes": n * V * E * (3 if case["train"] else 1) + n * (16.0 + 8.0 * case["top"]),
                "flops": n * V * (20.0 if case["train"] else 8.0)}
    new, before = _lengths(case)
    hkv, hd = case["hkv"], case["hd"]
    if case["kind"] == "write":
        back = sum(a + b % PAGE for a, b in zip(new, before))
        return {"bytes": 2.0 * hkv * hd * (sum(new) * (E + 1) + back * (E + 1)), "flops": 2.0 * hkv * hd * (4.0 * sum(new) + back)}
    keys = sum(a + b for a, b in zip(new, before))
    pairs = sum(a * b + a * (a + 1) / 2 for a, b in zip(new, before))
    return {"bytes": 2.0 * keys * hkv * hd + 2.0 * sum(new) * case["hq"] * hd * E, "flops": 4.0 * pairs * case["hq"] * hd}


# ---------------------------------------------------------------------------
# the same in 64 bits, one sequence (or a few rows) at a time
# ---------------------------------------------------------------------------
def _round_e4m3(y):
    """y (|y| <= 448) to the nearest multiple of 2^(max(e, -6) - 3), ties to even, e the exponent of y."""
    _, e = torch.frexp(y)
    step = torch.exp2((e.double() - 1.0).clamp(min=-6.0) - 3.0)
    return torch.round(y / step) * step


def _exact_write(case, st):
    top = INT8_MAX if case["fmt"] == "int8" else FP8_MAX
    nearest = torch.round if case["fmt"] == "int8" else _round_e4m3
    new, before = _lengths(case)
    out = {"k": [], "v": []}
    at = 0
    pages = st["pages"].cpu().tolist()
    for i, (a, b) in enumerate(zip(new, before)):
        kept, end = b % PAGE, b + a
        table = pages[i][b // PAGE:-(-end // PAGE)]
        for name in ("k", "v"):
            x = st[name][at:at + a].double()
            x = torch.cat([torch.zeros((kept,) + x.shape[1:], dtype=x.dtype, device="cuda"), x])
            x = torch.nn.functional.pad(x, (0, 0, 0, 0, 0, len(table) * PAGE - x.shape[0]))
            x = x.view(len(table), PAGE, case["hkv"], case["hd"]).transpose(1, 2)           # [page][head][slot][hd]
            e = torch.log2(x.abs().amax((2, 3)) / top).ceil().clamp(min=-126.0)
            if kept:
                e0 = st[name + "_exp"][table[0]].double() - 127.0
                e[0] = torch.maximum(e[0], e0)
                old = st[name + "_cache"][table[0]].double() * torch.exp2(e0 - e[0])[:, None, None]
            y = nearest(x * torch.exp2(-e)[..., None, None])
            if kept:
                y[0, :, :kept] = nearest(old)[:, :kept]
            y = (y * torch.exp2(e)[..., None, None]).transpose(1, 2).reshape(-1, case["hkv"], case["hd"])
            out[name].append(y[:kept + a])
        at += a
    return {name: torch.cat(v) for name, v in out.items()}


def _exact_attend(case, st):
    new, before = _lengths(case)
    hq, hkv, hd = case["hq"], case["hkv"], case["hd"]
    out = torch.zeros(st["out"].shape, dtype=torch.float64, device="cuda")
    at = 0
    for i, (a, b) in enumerate(zip(new, before)):
        pg = st["pages"][i, :-(-(a + b) // PAGE)].long()
        keep = torch.arange(a + b, device="cuda")[None, :] <= b + torch.arange(a, device="cuda")[:, None]
        for g in range(hkv):
            kv = [st[c + "_cache"][pg, g].double() * torch.exp2(st[c + "_exp"][pg, g].double() - 127.0)[:, None, None]
                  for c in ("k", "v")]
            k, v = (x.reshape(-1, hd)[:a + b] for x in kv)
            for h in range(g * (hq // hkv), (g + 1) * (hq // hkv)):
                s = st["q"][at:at + a, h].double() @ k.T.contiguous() / math.sqrt(hd)
                out[at:at + a, h] = torch.softmax(s.masked_fill(~keep, -math.inf), -1) @ v
        at += a
    return {"out": out}


def _exact_score(case, st):
    parts = []
    for r in range(0, case["rows"], 64):
        z = st["logits"][r:r + 64].double() / case["temperature"]
        tok = st["tok"][r:r + 64].long()
        lp = torch.log_softmax(z, -1)
        p = torch.exp(lp)
        plp = torch.special.xlogy(p, p)
        ent = -plp.sum(-1)
        has = tok >= 0
        one = torch.zeros_like(z).scatter_(1, tok.clamp(min=0)[:, None], 1.0) * has[:, None]
        got = {"logp": torch.where(has, lp.gather(1, tok.clamp(min=0)[:, None])[:, 0], 0.0 * ent), "entropy": ent,
               "max": st["logits"][r:r + 64].double().amax(-1), "sum": torch.exp(z - z.amax(-1, keepdim=True)).sum(-1)}
        if case["top"]:
            got["top_logp"] = torch.topk(lp, case["top"], -1).values
        if case["train"]:
            g, h = st["g_logp"][r:r + 64].double()[:, None] * has[:, None], st["g_ent"][r:r + 64].double()[:, None]
            got["grad"] = ((g * (one - p) - h * (plp + p * ent[:, None])) / case["temperature"]).to(torch.float64)
            if case["rows"] * case["vocab"] > 1 << 26:
                got["grad"] = got["grad"].float()            # a check of bf16 values: 32 bits hold it
        parts.append(got)
    out = {name: torch.cat([x[name] for x in parts]) for name in parts[0]}
    if case["top"]:
        out["top_id"] = None
    return out


def exact(case, seed):
    st = prepare(case, seed)
    return {"write": _exact_write, "attend": _exact_attend, "score": _exact_score}[case["kind"]](case, st)
