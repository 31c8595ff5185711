"""Argument checks of attention over shared prompts and of log probabilities from
hidden states at the C ABI (no GPU: every call is refused or has nothing to do)."""
import ctypes

import pytest

import paper_2607_26253_amd as sara

L, BAD, OK = sara._lib, sara.SARA_EINVAL, sara.SARA_OK
BF16, F32 = 1, 0
P = ctypes.c_void_p(4096)
ODD = ctypes.c_void_p(4104)


def other(p):
    return ctypes.c_void_p(p)


def cache(**over):
    d = dict(k=4096, v=4096, k_exp=4096, v_exp=4096, n_pages=8, n_kv_heads=2, head_dim=128, format=0)
    d.update(over)
    return ctypes.byref(sara.sara_kv8_cache(*d.values()))


def group(c=None, q=P, row=512, head=128, out=P, o_row=512, o_head=128, dtype=BF16, n_rows=4, heads=4, pages=P, max_pages=4, ctx=P,
          off=P, n_seqs=2, groups=P, shared=P, n_groups=1, max_ctx=64, max_shared=32, scale=1.0, ws=None, ws_bytes=0):
    return L.sara_kv8_group_attention(c or cache(), q, row, head, out, o_row, o_head, dtype, n_rows, heads, pages, max_pages, ctx, off,
                                      n_seqs, groups, shared, n_groups, max_ctx, max_shared, scale, ws, ws_bytes, None)


def group_need(hkv=2, hd=128, n_rows=4, heads=4, n_seqs=4, n_groups=1, ragged=0, max_ctx=64, max_shared=32, dtype=BF16):
    need = ctypes.c_int64(-1)
    rc = L.sara_kv8_group_attention_workspace(hkv, hd, n_rows, heads, n_seqs, n_groups, ragged, max_ctx, max_shared, dtype, ctypes.byref(need))
    return rc, need.value


@pytest.mark.parametrize("over", [dict(c=cache(k=0)), dict(c=cache(v_exp=0)), dict(c=cache(head_dim=96)), dict(c=cache(format=2)),
                                  dict(c=cache(k=4104)), dict(dtype=2), dict(n_rows=-1), dict(n_seqs=-1), dict(max_pages=0),
                                  dict(pages=None), dict(off=None, n_rows=3), dict(row=516), dict(o_head=132), dict(q=None), dict(out=None),
                                  dict(q=ODD), dict(heads=3), dict(heads=0), dict(ctx=None), dict(max_ctx=65), dict(max_ctx=-1),
                                  dict(max_shared=65), dict(max_shared=-1), dict(groups=None), dict(shared=None), dict(n_groups=-1),
                                  dict(scale=float("nan")), dict(scale=float("inf")), dict(o_row=128, o_head=128),
                                  dict(n_rows=2 ** 31 - 1, n_seqs=2 ** 30)])
def test_group_attention_is_checked(over):
    assert group(**over) == BAD
    assert len(L.sara_last_error()) > 0


def test_group_attention_of_nothing():
    assert group(n_rows=0) == OK and group(n_rows=0, n_seqs=0) == OK and group(n_seqs=0) == OK
    assert group(n_rows=0, groups=None, shared=None, n_groups=0) == OK


def test_group_workspaces():
    """Shared pages on their own need room for their partial results: many rows behind a long prompt; a few tokens need none."""
    assert group_need() == (OK, 0)
    rc, need = group_need(n_rows=32, n_seqs=32, heads=16, max_ctx=70000, max_shared=65536)
    assert rc == OK and need > 32 * 16 * 128 * 4
    assert group(n_rows=32, n_seqs=32, heads=16, off=None, row=2048, o_row=2048, max_pages=4375, max_ctx=70000, max_shared=65536, ws=P,
                 ws_bytes=need - 1) == BAD
    assert b"workspace" in L.sara_last_error()
    assert group(n_rows=32, n_seqs=32, heads=16, off=None, row=2048, o_row=2048, max_pages=4375, max_ctx=70000, max_shared=65536, ws=ODD,
                 ws_bytes=need) == BAD
    for kw in (dict(hkv=0), dict(hd=96), dict(heads=3), dict(n_rows=-1), dict(n_groups=-1), dict(max_ctx=2 ** 30 + 1), dict(max_shared=-1),
               dict(dtype=2), dict(n_rows=2 ** 30)):
        assert group_need(**kw)[0] == BAD
    assert group_need(n_rows=0) == (OK, 0) and group_need(n_seqs=0) == (OK, 0)
    # what the launches index with 32 bits: every answer is a size that memory could have, or a refusal
    for n in (1, 1000, 100000):
        for most in (16, 4096, 1 << 20):
            for ragged in (0, 1):
                rc, need = group_need(n_rows=4 * n, n_seqs=n, n_groups=max(1, n // 8), ragged=ragged, max_ctx=most, max_shared=most, heads=12)
                assert rc == OK and 0 <= need < 1 << 37


def head(h=P, h_stride=64, w=other(1 << 20), w_stride=64, dtype=BF16, n_rows=4, d=64, V=100, tok=P, T=1.0, logp=P, ent=P, stats=P, ws=P,
         ws_bytes=1 << 30):
    return L.sara_head_logprobs(h, h_stride, w, w_stride, dtype, n_rows, d, V, tok, T, logp, ent, stats, ws, ws_bytes, None)


def grad(h=P, h_stride=64, w=other(1 << 20), w_stride=64, dtype=BF16, n_rows=4, d=64, V=100, tok=P, T=1.0, stats=P, ent=P, gl=P, ge=P,
         gh=other(1 << 21), gh_stride=64, gw=other(1 << 22), gw_stride=64, gw_dtype=BF16, accumulate=0, ws=P, ws_bytes=1 << 40):
    return L.sara_head_logprobs_grad(h, h_stride, w, w_stride, dtype, n_rows, d, V, tok, T, stats, ent, gl, ge, gh, gh_stride, gw, gw_stride,
                                     gw_dtype, accumulate, ws, ws_bytes, None)


def head_need(dtype=BF16, n_rows=4, d=64, V=100, backward=0, gw_dtype=BF16):
    need = ctypes.c_int64(-1)
    rc = L.sara_head_logprobs_workspace(dtype, n_rows, d, V, backward, gw_dtype, ctypes.byref(need))
    return rc, need.value


@pytest.mark.parametrize("over", [dict(h=None), dict(w=None), dict(tok=None), dict(dtype=2), dict(n_rows=-1), dict(d=0), dict(d=60),
                                  dict(V=0), dict(h=ODD), dict(h_stride=60), dict(h_stride=68), dict(w_stride=32), dict(w=other(1 << 20 | 2)),
                                  dict(T=0.0), dict(T=-1.0), dict(T=float("nan")), dict(T=float("inf")), dict(T=1e-38), dict(ws=None),
                                  dict(ws=ODD), dict(ws_bytes=8), dict(n_rows=2 ** 31 - 1, V=2 ** 30), dict(d=(1 << 20) + 8),
                                  dict(V=(1 << 30) + 1)])
def test_head_is_checked(over):
    assert head(**over) == BAD
    assert len(L.sara_last_error()) > 0
    assert grad(**over) == BAD


@pytest.mark.parametrize("over", [dict(stats=None), dict(ent=None), dict(gh=None, gw=None), dict(gh=P), dict(gw=other(1 << 20)),
                                  dict(gh=other(1 << 22)), dict(gh_stride=60), dict(gw_stride=68), dict(gw=other(1 << 22 | 8)),
                                  dict(gw_dtype=2), dict(dtype=F32, gw_dtype=BF16), dict(n_rows=131073)])
def test_head_gradients_are_checked(over):
    assert grad(**over) == BAD
    assert len(L.sara_last_error()) > 0


def test_head_of_no_rows_and_workspaces():
    assert head(n_rows=0, ws=None) == OK and head(stats=ODD, n_rows=0) == OK
    assert head(stats=other(4100)) == BAD
    assert head_need(n_rows=0) == (OK, 0) and head_need(n_rows=0, backward=1) == (OK, 0)
    assert head_need(n_rows=131072, backward=1)[0] == OK and head_need(n_rows=131073, backward=1)[0] == BAD
    assert head_need(dtype=F32, backward=1, gw_dtype=BF16)[0] == BAD and head_need(dtype=F32, backward=1, gw_dtype=F32)[0] == OK
    # D is kept by pieces of the vocabulary: the workspace does not grow with rows times ids
    for rows in (1, 64, 65, 2048, 131072):
        for dtype in (BF16, F32):
            for d in (8, 1536, 8192):
                for V in (1, 512, 151936):
                    for backward in (0, 1):
                        rc, need = head_need(dtype, rows, d, V, backward, dtype)
                        assert rc == OK and 0 < need < (3 << 30) + 64 * rows * (d + 512), (rows, dtype, d, V, backward, need)


def test_wide_heads_fit_their_launches():
    """Small tiles of a weight's gradient are vocab d / 1024 blocks, of which a launch holds 2^24 - 1: 16,383 x 1,024 and the
    1,024 of dH are one too many and go in large tiles, whose workspace holds a piece of the weight in bf16 parts (453 MB)."""
    rc, need = head_need(F32, 1, 32768, 32 * 16382, 1, F32)
    assert rc == OK and need < 1 << 27
    for V in (32 * 16382 + 1, 524289, 600000):
        rc, need = head_need(F32, 1, 32768, V, 1, F32)
        assert rc == OK and need > 1 << 28


@pytest.mark.parametrize("n_seqs", [65536, 70000, 300000])
def test_group_joins_past_a_launch_are_refused(n_seqs):
    """Few rows of many mostly empty sequences behind a long prompt: the join is 32 blocks for each sequence and KV head, of
    which a launch holds 2^24 - 1; the launches before it would have been enqueued."""
    rc, need = group_need(hkv=8, n_rows=100, heads=8, n_seqs=n_seqs, ragged=1, max_ctx=66000, max_shared=65536)
    assert rc == OK and need > 32 * 8 * n_seqs * 128 * 4
    assert group(cache(n_kv_heads=8), row=1024, o_row=1024, n_rows=100, heads=8, max_pages=4125, n_seqs=n_seqs, max_ctx=66000,
                 max_shared=65536, ws=P, ws_bytes=need) == BAD
    assert b"too many" in L.sara_last_error()
