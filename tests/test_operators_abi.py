"""Argument checks of the 8-bit KV cache and of the token log probabilities at
the C ABI, and the 64-bit reference's own pins (no GPU)."""
import ctypes
import os
import subprocess
import sys

import numpy as np
import pytest

import paper_2607_26253_amd as sara
from tests import kv8_reference as R

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
L, BAD = sara._lib, sara.SARA_EINVAL
P = ctypes.c_void_p(4096)


def cache(**over):
    d = dict(k=4096, v=4096, k_exp=4096, v_exp=4096, n_pages=8, n_kv_heads=2, head_dim=128, format=0)
    d.update(over)
    return ctypes.byref(sara.sara_kv8_cache(*d.values()))


def write(c=None, k=P, row=256, head=128, dtype=1, n_rows=4, pages=P, max_pages=4, start=P, off=P, n_seqs=2):
    return L.sara_kv8_write(c or cache(), k, row, head, P, 256, 128, dtype, n_rows, pages, max_pages, start, off, n_seqs, None)


def attend(c=None, q=P, row=512, dtype=1, n_rows=4, heads=4, pages=P, max_pages=4, ctx=P, off=P, n_seqs=2, max_ctx=64,
           scale=1.0, ws=None, ws_bytes=0):
    return L.sara_kv8_attention(c or cache(), q, row, 128, P, 512, 128, dtype, n_rows, heads, pages, max_pages, ctx, off,
                                n_seqs, max_ctx, scale, ws, ws_bytes, None)


@pytest.mark.parametrize("over", [dict(k=0), dict(v_exp=0), dict(n_pages=0), dict(n_kv_heads=0), dict(head_dim=96),
                                  dict(format=2), dict(k=4097), dict(v=4104)])
def test_caches_are_checked(over):
    assert write(cache(**over)) == BAD and attend(cache(**over)) == BAD
    assert len(L.sara_last_error()) > 0


@pytest.mark.parametrize("over", [dict(dtype=2), dict(n_rows=-1), dict(n_seqs=-1), dict(max_pages=0), dict(pages=None),
                                  dict(off=None, n_rows=3), dict(row=257), dict(n_rows=2 ** 31 - 1, n_seqs=2 ** 30)])
def test_rows_are_checked(over):
    assert write(**over) == BAD and attend(**over) == BAD


def test_more_checks():
    assert write(k=None) == BAD and write(head=129) == BAD and write(start=None) == BAD
    assert write(k=ctypes.c_void_p(4098)) == BAD
    assert attend(q=None) == BAD and attend(heads=3) == BAD and attend(heads=0) == BAD and attend(ctx=None) == BAD
    assert attend(max_ctx=65) == BAD and attend(max_ctx=-1) == BAD
    for s in (float("nan"), float("inf")):
        assert attend(scale=s) == BAD
    assert write(n_rows=0) == sara.SARA_OK and attend(n_rows=0) == sara.SARA_OK      # nothing to do: nothing is launched
    assert write(n_rows=0, n_seqs=0) == sara.SARA_OK
    need = ctypes.c_int64(-1)
    assert L.sara_kv8_attention_workspace(2, 128, 1, 12, 1, 0, 100000, ctypes.byref(need)) == sara.SARA_OK and need.value > 0
    assert attend(n_rows=1, n_seqs=1, off=None, heads=12, max_pages=6250, max_ctx=100000, ws=P, ws_bytes=need.value - 1) == BAD
    assert b"workspace" in L.sara_last_error()
    assert L.sara_kv8_attention_workspace(2, 128, 1, 12, 1, 0, 100, None) == BAD
    assert L.sara_kv8_attention_workspace(2, 100, 1, 12, 1, 0, 100, ctypes.byref(need)) == BAD
    assert ctypes.sizeof(sara.sara_kv8_cache) == 4 * 8 + 4 * 4


def test_log_probability_arguments():
    def fwd(x=P, dtype=1, stride=100, n=2, V=100, tok=P, T=1.0, k=0, ids=None, lps=None, stats=P):
        return L.sara_token_logprobs(x, dtype, stride, n, V, tok, T, k, P, P, stats, ids, lps, None, 0, None)

    def bwd(x=P, dtype=1, stride=100, n=2, V=100, tok=P, T=1.0, stats=P, ent=P, g=P, h=P, y=ctypes.c_void_p(8192), ystride=100):
        return L.sara_token_logprobs_grad(x, dtype, stride, n, V, tok, T, stats, ent, g, h, y, ystride, None)

    for f in (fwd, bwd):
        for over in (dict(x=None), dict(dtype=3), dict(stride=99), dict(n=-1), dict(V=0), dict(tok=None), dict(T=0.0),
                     dict(T=float("nan")), dict(x=ctypes.c_void_p(4097))):
            assert f(**over) == BAD, (f, over)
        assert f(n=0) == sara.SARA_OK
    assert fwd(k=33, ids=P, lps=P) == BAD and fwd(k=2) == BAD and fwd(k=-1) == BAD and fwd(stats=ctypes.c_void_p(4100)) == BAD
    assert bwd(stats=None) == BAD and bwd(ent=None) == BAD and bwd(y=None) == BAD and bwd(ystride=5) == BAD
    assert bwd(y=P, ystride=108) == BAD                                              # in place at another stride
    assert L.sara_token_logprobs_workspace(1, 10, 40, ctypes.byref(ctypes.c_int64())) == BAD
    assert L.sara_token_logprobs_workspace(1, 10, 4, None) == BAD


def test_reference_codes():
    """The reference's e4m3 table and rounding: 253 finite values, the largest 448, halfway cases to even."""
    v = R.e4m3_value(np.arange(256))
    assert np.isnan(v).sum() == 2 and np.nanmax(v) == 448.0 and v[1] == 2.0 ** -9 and v[8] == 2.0 ** -6
    codes = v[~np.isnan(v)]
    np.testing.assert_array_equal(np.abs(R.nearest(codes, "fp8")), np.abs(codes))
    assert R.nearest(np.array([17.0, 19.0, 2.0 ** -10, 3 * 2.0 ** -10, 432.0]), "fp8").tolist() == [16.0, 20.0, 0.0, 2.0 ** -8, 448.0]
    assert R.nearest(np.array([0.5, 1.5, -2.5, 126.5]), "int8").tolist() == [0.0, 2.0, -2.0, 126.0]
    assert [R.exponent(a, "int8") for a in (127.0, 127.5, 0.0, np.inf)] == [127, 128, 1, 255]
    assert [R.exponent(a, "fp8") for a in (448.0, 449.0, 224.0)] == [127, 128, 126]


@pytest.mark.parametrize("order", ["import paper_2607_26253_amd, torch", "import torch, paper_2607_26253_amd"])
def test_one_hip_runtime_whatever_is_imported_first(order):
    code = order + "\nfor l in open('/proc/self/maps'):\n    if 'libamdhip64' in l: print(l.split()[-1])"
    out = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, cwd=ROOT, check=True).stdout
    assert len(set(out.split())) == 1, out


def test_temperatures_without_a_reciprocal_are_refused():
    for T in (1e-39, 1e-38, 2e37, float("inf")):
        assert L.sara_token_logprobs(P, 1, 100, 2, 100, P, T, 0, P, P, P, None, None, None, 0, None) == BAD
        assert L.sara_token_logprobs_grad(P, 1, 100, 2, 100, P, T, P, P, P, P, P, 100, None) == BAD


def test_calls_refuse_host_tensors_and_other_objects():
    import torch
    x, ids = torch.zeros((2, 8)), torch.zeros(2, dtype=torch.int32)
    for bad, exc in ((x, ValueError), (x.half(), TypeError), (None, TypeError), ([1.0], TypeError)):
        with pytest.raises(exc):
            sara.sara_token_logprobs(bad, ids)
        with pytest.raises(exc):
            sara.sara_token_logprobs_grad(bad, ids, None, None, None, None, x)
    codes, exps = torch.zeros((2, 1, 16, 64), dtype=torch.int8), torch.zeros((2, 1), dtype=torch.uint8)
    kv, pages, seq = torch.zeros((1, 1, 64)), torch.zeros((1, 2), dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    for bad, exc in ((kv, ValueError), (kv.double(), TypeError), (3, TypeError)):
        with pytest.raises(exc):
            sara.sara_kv8_write(codes, codes, exps, exps, bad, bad, pages, seq)
        with pytest.raises(exc):
            sara.sara_kv8_read(codes, codes, exps, exps, pages, seq, None, bad, bad)
        with pytest.raises(exc):
            sara.sara_kv8_attention(bad, codes, codes, exps, exps, pages, seq, None, bad)


def test_contexts_past_the_kernels_positions_are_refused():
    """Near 2^31 the number of pages overflowed: a call got one split, no workspace and partial results all the same."""
    need = ctypes.c_int64(-1)

    def workspace(max_ctx):
        return L.sara_kv8_attention_workspace(2, 128, 1, 12, 1, 0, max_ctx, ctypes.byref(need))

    assert workspace(2 ** 30) == sara.SARA_OK and need.value > 0
    for c in (2 ** 30 + 1, 2 ** 31 - 16, 2 ** 31 - 15, 2 ** 31 - 1):
        assert workspace(c) == BAD
        assert attend(n_rows=1, n_seqs=1, off=None, heads=12, max_pages=2 ** 31 - 1, max_ctx=c, ws=P, ws_bytes=2 ** 40) == BAD
        assert b"max_ctx" in L.sara_last_error()


def test_vocabularies_past_the_kernels_ids_are_refused():
    """The gradient of rows that lie unlike their logits steps by up to 2^27 ids: past 2^31 - 2^27 its id wrapped below 0."""
    need = ctypes.c_int64(-1)
    assert L.sara_token_logprobs_workspace(1, 2 ** 30, 0, ctypes.byref(need)) == sara.SARA_OK
    for V in (2 ** 30 + 1, 2 ** 31 - 2 ** 27 + 1, 2 ** 31 - 1):
        assert L.sara_token_logprobs_workspace(1, V, 0, ctypes.byref(need)) == BAD
        assert L.sara_token_logprobs(P, 1, V, 1, V, P, 1.0, 0, P, P, P, None, None, P, 2 ** 40, None) == BAD
        assert L.sara_token_logprobs_grad(P, 1, V, 1, V, P, 1.0, P, P, P, P, ctypes.c_void_p(8194), V, None) == BAD
        assert b"vocab" in L.sara_last_error()


def test_calls_past_a_launch_are_refused():
    """A grid of 2^24 blocks of 256 threads is refused by the runtime, which is not an argument error any more."""
    for n_rows, n_seqs, off in ((2 ** 24, 2 ** 24, None), (2 ** 24, 2 ** 24, P), (2 ** 30, 1, P)):
        assert write(n_rows=n_rows, n_seqs=n_seqs, off=off) == BAD, (n_rows, n_seqs)
    for n_rows, n_seqs, off in ((2 ** 23, 2 ** 23, None), (2 ** 22, 2 ** 22, P)):
        assert attend(n_rows=n_rows, n_seqs=n_seqs, off=off) == BAD, (n_rows, n_seqs)
    assert b"too many" in L.sara_last_error()


def test_rows_past_the_launches_numbers_are_refused():
    """The launches go through the rows in chunks of 65,535: the last step of 2^31 - 1 rows wrapped below 0."""
    need = ctypes.c_int64(-1)
    assert L.sara_token_logprobs_workspace(2 ** 30, 5, 0, ctypes.byref(need)) == sara.SARA_OK and need.value == 0
    for n in (2 ** 30 + 1, 2 ** 31 - 1):
        assert L.sara_token_logprobs_workspace(n, 5, 0, ctypes.byref(need)) == BAD
        assert L.sara_token_logprobs(P, 1, 5, n, 5, P, 1.0, 0, P, P, P, None, None, None, 0, None) == BAD
        assert L.sara_token_logprobs_grad(P, 1, 5, n, 5, P, 1.0, P, P, P, P, ctypes.c_void_p(8192), 5, None) == BAD
        assert b"n_rows" in L.sara_last_error()


def test_outputs_that_overlap_are_refused():
    """Rows and heads that share elements (an expanded tensor's have stride 0) would be written by several blocks at once."""
    def read(krow=256, khead=128, vrow=256, vhead=128, n_rows=4):
        return L.sara_kv8_read(cache(), P, krow, khead, P, vrow, vhead, 1, n_rows, P, 4, P, P, 2, None)

    def out(row, head, n_rows=4, heads=4):
        return L.sara_kv8_attention(cache(), P, 512, 128, P, row, head, 1, n_rows, heads, P, 4, P, P, 2, 64, 1.0, None, 0, None)

    for row, head in ((0, 128), (256, 0), (128, 128), (64, 128), (-128, 128), (136, 128), (256, 64), (128, 256), (248, 128)):
        assert read(krow=row, khead=head) == BAD and read(vrow=row, vhead=head) == BAD, (row, head)
        assert b"overlap" in L.sara_last_error()
    for row, head in ((0, 128), (512, 0), (256, 128), (504, 128), (128, 504), (-256, 128), (128, 128)):
        assert out(row, head) == BAD, (row, head)
        assert b"overlap" in L.sara_last_error()
    assert out(0, 0, n_rows=1, heads=2) == BAD and read(khead=0, n_rows=1) == BAD


def test_a_stream_of_another_device_is_refused():
    """The call would go to the tensors' device all the same, to its current stream."""
    import torch

    class On:
        def __init__(self, index):
            self.device = torch.device("cuda", index)

    x = On(0)
    for call in (lambda s: sara.sara_token_logprobs(x, None, stream=s),
                 lambda s: sara.sara_token_logprobs_grad(x, None, None, None, None, None, None, stream=s),
                 lambda s: sara.sara_kv8_write(x, *[None] * 7, stream=s),
                 lambda s: sara.sara_kv8_read(x, *[None] * 8, stream=s),
                 lambda s: sara.sara_kv8_attention(None, x, *[None] * 7, stream=s)):
        with pytest.raises(ValueError, match="stream"):
            call(On(1))


@pytest.mark.parametrize("torch_there", [True, False])
def test_the_library_builds_without_torch(tmp_path, monkeypatch, capsys, torch_there):
    """The compiler is replaced by one that writes its output file: which outputs there are is what is looked at."""
    from paper_2607_26253_amd import build as B

    def compiler(cmd, **kw):
        with open(cmd[cmd.index("-o") + 1], "w") as f:
            f.write(cmd[0])
        return subprocess.CompletedProcess(cmd, 0, "", "")

    monkeypatch.setattr(B, "HERE", str(tmp_path))
    monkeypatch.setattr(B, "OUT", str(tmp_path / "libsara.so"))
    monkeypatch.setattr(B, "OPERATORS", str(tmp_path / "_operators.so"))
    monkeypatch.setattr(B, "hipcc", lambda: "hipcc")
    monkeypatch.setattr(B.subprocess, "run", compiler)
    if not torch_there:
        monkeypatch.setitem(sys.modules, "torch", None)
    assert B.build() == str(tmp_path / "libsara.so")
    assert (tmp_path / "libsara.so").exists()
    assert (tmp_path / "_operators.so").exists() == torch_there
    assert ("_operators.so" in capsys.readouterr().err) != torch_there


def test_scales_whose_base_2_form_overflows_are_refused():
    """scale log2(e) was infinite for these: a score of 0 became NaN."""
    for s in (2.4e38, -3e38, 3.4e38):
        assert attend(scale=s) == BAD
        assert b"scale" in L.sara_last_error()
