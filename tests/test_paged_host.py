"""The paged cache and the linear layer without a GPU: the integer rules, what the calls refuse, what the binding refuses."""
import ctypes as C
import os
import shutil
import subprocess

import pytest
import torch

from paper_2509_22622_amd import binding as B

HERE = os.path.dirname(os.path.abspath(__file__))
MADE = dict(layers=2, q_heads=8, kv_heads=2, head_dim=64, page_tokens=32, n_pages=10)


@pytest.mark.skipif(shutil.which("g++") is None, reason="no host C++ compiler")
@pytest.mark.parametrize("name, says", [("check_paged_rules", "paged rules ok"), ("check_linear_shapes", "linear shapes ok")])
def test_rules(name, says, tmp_path):
    exe = tmp_path / name
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-fsanitize=undefined", "-o", str(exe), os.path.join(HERE, name + ".cpp")], check=True)
    run = subprocess.run([str(exe)], capture_output=True, text=True)
    assert run.returncode == 0, run.stdout + run.stderr
    assert says in run.stdout


def test_sizes():
    L = B.lib()
    assert L.ll_paged_bytes(3, 8, 128, 64, 100, 0) == 3 * 100 * 8 * 2 * 64 * 128 * 2 + 64 * 8
    assert L.ll_paged_bytes(3, 8, 64, 16, 7, 1) == 3 * 7 * 8 * 2 * 16 * 64 + 32 * 8
    for bad in [(0, 8, 128, 64, 100, 0), (1, 0, 128, 64, 100, 0), (1, 8, 96, 64, 100, 0), (1, 8, 128, 24, 100, 0), (1, 8, 128, 0, 100, 0),
                (1, 8, 128, 64, 0, 0), (1, 8, 128, 64, 100, 2), (1, 1025, 128, 64, 100, 0), (1, 8, 128, 1 << 17, 100, 0),
                (65536, 1024, 128, 65536, 2 ** 31 - 1, 0)]:
        assert L.ll_paged_bytes(*bad) == 0
    assert L.ll_linear_packed_bytes(17, 72) == 32 * 128 * 2
    for n, k in [(0, 64), (-1, 64), (16, 0), (16, 63), (16, 4), (1 << 21, 64), (16, 1 << 21), (1 << 20, 1 << 15)]:
        assert L.ll_linear_packed_bytes(n, k) == 0


def status(call, *args, **kw):
    with pytest.raises(B.LongLiveError) as e:
        call(*args, **kw)
    return e.value.status


@pytest.mark.parametrize("change, want", [
    ({"layers": 0}, 1), ({"head_dim": 96}, 4), ({"head_dim": 0}, 1), ({"page_tokens": 40}, 1), ({"n_pages": 0}, 1), ({"q_heads": 7}, 1),
    ({"q_heads": 1}, 1), ({"kv_heads": 3}, 1), ({"k_exp": 1}, 1), ({"kv_format": "fp8_e4m3", "v_exp": 17}, 1), ({"rope": "pairs", "rope_dim": 24}, 1),
    ({"rope": "halves", "rope_dim": 80}, 1), ({"rope": "halves", "rope_dim": 0}, 1), ({"rope": "grid", "rope_dim": 32}, 1), ({"rope": "none", "rope_dim": 64}, 1),
    ({"rope": "pairs", "rope_theta": 0.0}, 1), ({"rope": "pairs", "rope_theta": float("inf")}, 1), ({"rope": "pairs", "rope_theta": float("nan")}, 1)])
def test_create_refuses(change, want):
    assert status(B.PagedCache, device=None, **{**MADE, **change}) == want


def test_create_takes_and_refuses_buffers():
    L, h = B.lib(), C.c_void_p()
    args = [1, 8, 2, 64, 32, 10, 0, 0, 0, 1, 64, 10000.0]
    assert L.ll_paged_create(*args, None, 0, None) == 1
    assert L.ll_paged_create(*args, None, 16, C.byref(h)) == 1 and not h
    assert L.ll_paged_create(*args, C.c_void_p(4096 + 16), 1 << 30, C.byref(h)) == 1 and not h      # not 256-byte aligned
    assert L.ll_paged_create(*args, C.c_void_p(4096), 1000, C.byref(h)) == 3 and not h
    assert L.ll_paged_create(*args[:9], 4, 64, 10000.0, None, 0, C.byref(h)) == 1
    assert L.ll_paged_create(*args, None, 0, C.byref(h)) == 0 and h
    assert L.ll_paged_destroy(h) == 0 and L.ll_paged_destroy(None) == 0


def test_calls_refuse():
    """Through an index-only handle: everything that is wrong whatever the tensors are."""
    L, c = B.lib(), B.PagedCache(**MADE, device=None)

    def append(handle=c._h, layer=0, n_seqs=4, n_tokens=4, cols=3, stride=3, k=None):
        return L.ll_paged_append(handle, layer, n_seqs, n_tokens, None, None, None, cols, stride, None, None, 0, k, 128, None, 128, None, 0, None)

    def attn(handle=c._h, layer=0, n_seqs=4, n_tokens=4, max_new=1, max_len=100, cols=3, stride=3, sink=0, window=0, q=None):
        return L.ll_paged_attn(handle, layer, n_seqs, n_tokens, max_new, max_len, None, None, None, cols, stride, sink, window, q, 512, None, 512, None, 0, None)

    some = C.c_void_p(4096)
    for call in (append, attn):
        assert call() == 0 and call(n_seqs=1 << 20) == 0 and call(stride=2 ** 30) == 0 and call(n_tokens=0) == 0
        for bad in [dict(handle=None), dict(layer=-1), dict(layer=2), dict(n_seqs=0), dict(n_seqs=(1 << 20) + 1), dict(n_tokens=-1),
                    dict(n_tokens=(1 << 24) + 1), dict(cols=0), dict(cols=(1 << 25) + 1, stride=1 << 26), dict(stride=2), dict(stride=2 ** 30 + 1)]:
            assert call(**bad) == 1, bad
    assert append(k=some) == 1 and attn(q=some) == 1
    assert attn(sink=5, window=9) == 0
    for bad in [dict(max_new=0), dict(max_new=65537), dict(max_len=0), dict(max_len=2 ** 30 + 1), dict(sink=1), dict(sink=-1, window=4), dict(window=-1),
                dict(window=2 ** 30 + 1), dict(sink=2 ** 30 + 1, window=1)]:
        assert attn(**bad) == 1, bad
    wide = B.PagedCache(1, 1024, 1024, 64, 16, 4, device=None)
    assert attn(handle=wide._h, n_seqs=1 << 20, max_new=64) == 4 and attn(handle=wide._h, n_seqs=1 << 14, max_new=1) == 4
    assert attn(handle=wide._h, n_seqs=(1 << 14) - 1, max_new=1, max_len=1 << 30) == 0


def test_workspace_sizes():
    """None for what one workgroup per tile does, enough for the splits otherwise, never more than a bound; 0 for what a call refuses."""
    c = B.PagedCache(**MADE, device=None)
    assert c.attn_workspace_bytes(4, max_len=100) == 0
    far = c.attn_workspace_bytes(4, max_len=100000)
    assert 0 < far <= 2 * 4096 * 16 * 66 * 4
    assert c.attn_workspace_bytes(4, max_len=100000, sink_tokens=64, window_tokens=64) < far
    for bad in [dict(n_seqs=0), dict(n_seqs=4, max_new=0), dict(n_seqs=4, max_new=65537), dict(n_seqs=4, max_len=0), dict(n_seqs=4, sink_tokens=3)]:
        assert c.attn_workspace_bytes(**bad) == 0
    assert B.lib().ll_paged_attn_workspace_bytes(None, 4, 1, 100000, 0, 0) == 0


def test_linear_refuses():
    L, p = B.lib(), [C.c_void_p(4096 * (i + 1)) for i in range(6)]

    def pack(n=16, k=64, w=p[0], stride=64, to=p[1]):
        return L.ll_linear_pack_weight(n, k, w, stride, to, None)

    def linear(m=4, n=16, k=64, x=p[0], xs=64, w=p[1], bias=None, act=0, r=None, rs=0, y=p[4], ys=16):
        return L.ll_linear(m, n, k, x, xs, w, bias, act, r, rs, y, ys, None)

    for bad in [dict(n=0), dict(k=60), dict(w=None), dict(to=None), dict(stride=56), dict(stride=68), dict(stride=1 << 29), dict(to=p[0]), dict(w=C.c_void_p(4104)),
                dict(to=C.c_void_p(4098))]:
        assert pack(**bad) == 1, bad
    assert linear(m=0) == 0 and linear(m=0, x=None, y=None) == 0
    for bad in [dict(m=-1), dict(m=(1 << 24) + 1), dict(n=0), dict(k=4), dict(act=-1), dict(act=4), dict(x=None), dict(w=None), dict(y=None), dict(xs=56),
                dict(xs=68), dict(xs=(1 << 21) + 8), dict(ys=15), dict(ys=(1 << 21) + 1), dict(r=p[3], rs=8), dict(y=p[0]), dict(y=p[1]), dict(bias=p[4]),
                dict(r=p[4], rs=24), dict(x=C.c_void_p(4104)), dict(bias=C.c_void_p(4098)), dict(y=C.c_void_p(4104)), dict(r=C.c_void_p(4104), rs=16)]:
        assert linear(**bad) == 1, bad


def test_binding_refuses():
    """Shapes, types and strides that the calls could not see."""
    with pytest.raises(ValueError):
        B.PagedCache(**{**MADE, "kv_format": "int8"}, device=None)
    with pytest.raises(ValueError):
        B.PagedCache(**{**MADE, "rope": "spiral"}, device=None)
    bf16, t = torch.bfloat16, torch.zeros(4, 6, 8, dtype=torch.bfloat16)
    for x, shape, stride in [(t, (4, 6, 8), 48), (t[::2], (2, 6, 8), 96), (t[:, :3], (4, 3, 8), 48), (t[:1], (1, 6, 8), 48), (t[::4, :2], (1, 2, 8), 16),
                             (t[:, :1].transpose(0, 1).transpose(0, 1), (4, 1, 8), 48), (t[0], (6, 8), 8), (t[:1].expand(4, 6, 8), (4, 6, 8), 0)]:
        assert B._rows(x, "t", bf16, shape, -1) == stride            # (a stride of 0 is refused by the calls as shorter than a row)
    for bad, shape in [(t.float(), (4, 6, 8)), (t, (4, 6, 9)), (t, (4, 6)), (t.transpose(1, 2), (4, 8, 6)), (t[:, ::2], (4, 3, 8)), (t[:, :, ::2], (4, 6, 4)),
                       (t[:, :1].expand(4, 6, 8), (4, 6, 8))]:
        with pytest.raises(ValueError):
            B._rows(bad, "t", bf16, shape, -1)
    with pytest.raises(ValueError):
        B._rows(t, "t", bf16, (4, 6, 8), 0)
    i = torch.zeros(4, 6, dtype=torch.int32)
    assert B._ints(None, "i", (4, 6), -1) is None and B._ints(i, "i", (4, 6), -1) == i.data_ptr()
    for bad, shape in [(i.long(), (4, 6)), (i, (24,)), (i[:, :3], (4, 3)), (i.t(), (6, 4)), (i[:, 0], (4,))]:
        with pytest.raises(ValueError):
            B._ints(bad, "i", shape, -1)
    c, lens, table = B.PagedCache(**MADE, device=None), torch.zeros(4, dtype=torch.int32), torch.zeros(4, 3, dtype=torch.int32)
    x = torch.zeros(4, 2, 64, dtype=bf16)
    for call in (lambda: c.keys(0), lambda: c.values(0), lambda: c.append(0, lens, table, x, x), lambda: c.attn(0, lens, table, x, x),
                 lambda: c.attn_workspace(4)):
        with pytest.raises(B.LongLiveError):                          # an index-only handle has no memory
            call()
    with pytest.raises(ValueError):
        B.Linear(torch.zeros(16, 64, dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        B.Linear(torch.zeros(16, 64))
