"""The layer norm and the attention to an encoder's states without a GPU: the integer rules, what the calls refuse, what the binding refuses."""
import ctypes as C
import os
import shutil
import subprocess

import pytest
import torch

from paper_2509_22622_amd import binding as B

HERE = os.path.dirname(os.path.abspath(__file__))
BF16, F32, I32 = torch.bfloat16, torch.float32, torch.int32


@pytest.mark.skipif(shutil.which("g++") is None, reason="no host C++ compiler")
@pytest.mark.parametrize("name, says", [("check_norm_rules", "norm rules ok"), ("check_encoder_rules", "encoder rules ok")])
def test_rules(name, says, tmp_path):
    exe = tmp_path / name
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-fsanitize=undefined", "-o", str(exe), os.path.join(HERE, name + ".cpp")], check=True)
    run = subprocess.run([str(exe)], capture_output=True, text=True)
    assert run.returncode == 0, run.stdout + run.stderr
    assert says in run.stdout


def at(i):
    return C.c_void_p(4096 * (i + 1))


def test_layer_norm_refuses():
    L = B.lib()

    def forward(m=4, n=64, group=0, eps=1e-5, xt=0, x=at(0), xs=64, wt=0, w=None, b=None, yt=0, y=at(3), ys=64, stats=None):
        return L.ll_layer_norm(m, n, group, eps, xt, x, xs, wt, w, b, yt, y, ys, stats, None)

    assert forward(m=0) == 0 and forward(m=0, x=None, y=None) == 0
    for bad in [dict(m=-1), dict(m=(1 << 24) + 1), dict(n=0), dict(n=16385, xs=16385, ys=16385), dict(group=-1), dict(eps=0.0), dict(eps=-1.0), dict(eps=float("nan")),
                dict(eps=float("inf")), dict(xt=2), dict(xt=-1), dict(yt=2), dict(wt=2), dict(xt=0, yt=1), dict(xs=63), dict(ys=63), dict(xs=(1 << 21) + 1), dict(x=None), dict(y=None),
                dict(x=C.c_void_p(4097)), dict(xt=1, x=C.c_void_p(4098)), dict(y=C.c_void_p(4097)), dict(w=C.c_void_p(4097)), dict(wt=1, b=C.c_void_p(4098)),
                dict(stats=C.c_void_p(4100)), dict(w=at(3)), dict(b=at(3)), dict(stats=at(3)), dict(y=at(0), ys=72), dict(y=at(0), xt=1)]:
        assert forward(**bad) == 1, bad


def test_layer_norm_backward_refuses():
    L = B.lib()

    def backward(m=4, n=64, group=0, yt=0, dy=at(0), dys=64, xt=0, x=at(1), xs=64, wt=0, w=None, stats=at(2), r=None, rs=0, dx=at(3), dxs=64, dw=None, db=None, ws=None, size=0):
        return L.ll_layer_norm_backward(m, n, group, yt, dy, dys, xt, x, xs, wt, w, stats, r, rs, dx, dxs, dw, db, ws, size, None)

    assert backward(m=0) == 0 and backward(m=0, group=5, dw=at(5)) == 0
    for bad in [dict(m=-1), dict(n=0), dict(group=-2), dict(xt=2), dict(yt=1), dict(dys=63), dict(xs=63), dict(dxs=63), dict(r=at(4), rs=63), dict(dxs=(1 << 21) + 1), dict(dy=None),
                dict(x=None), dict(stats=None), dict(dx=None), dict(dy=C.c_void_p(4097)), dict(x=C.c_void_p(4097)), dict(dx=C.c_void_p(4097)), dict(r=C.c_void_p(4097), rs=64),
                dict(w=C.c_void_p(4097)), dict(stats=C.c_void_p(4100)), dict(dw=C.c_void_p(4104)), dict(db=C.c_void_p(4100)), dict(dx=at(2)), dict(w=at(3)), dict(dw=at(3)), dict(db=at(3)),
                dict(dw=at(5), db=at(5)), dict(dw=at(1)), dict(db=at(0)), dict(dw=at(4), r=at(4), rs=64), dict(dx=at(0), dxs=72), dict(dx=at(1), dxs=72), dict(dx=at(4), r=at(4), rs=72),
                dict(dx=at(0), xt=1), dict(m=4000, dw=at(5)), dict(m=4000, dw=at(5), ws=C.c_void_p(4104), size=1 << 30), dict(m=4000, dw=at(5), ws=at(5), size=1 << 30)]:
        assert backward(**bad) == 1, bad
    need = L.ll_layer_norm_backward_workspace_bytes(4000, 64, 0)
    assert need > 0 and backward(m=4000, dw=at(5), ws=at(6), size=need - 1) == 3
    assert L.ll_layer_norm_backward_workspace_bytes(1, 64, 0) == 0
    for bad in [(-1, 64, 0), (4, 0, 0), (4, 16385, 0), (4, 64, -1)]:
        assert L.ll_layer_norm_backward_workspace_bytes(*bad) == 0



def test_encoder_attn_refuses():
    L = B.lib()

    def forward(n=2, hq=4, hkv=2, d=64, scale=0.1, nq=8, nk=10, mq=4, mk=5, cuq=None, cuk=None, lens=None, q=at(0), qs=256, k=at(1), ks=128, v=at(2), vs=128, o=at(3), os_=256, lse=None,
                ws=None, size=0):
        return L.ll_encoder_attn(n, hq, hkv, d, scale, nq, nk, mq, mk, cuq, cuk, lens, q, qs, k, ks, v, vs, o, os_, lse, ws, size, None)

    assert forward(nq=0) == 0 and forward(nq=0, q=None, o=None, k=None, v=None) == 0
    assert forward(d=96, qs=384, ks=192, vs=192, os_=384) == 4
    for bad in [dict(n=0), dict(n=(1 << 20) + 1), dict(hkv=0), dict(hkv=3), dict(hq=1), dict(hq=1026, qs=1026 * 64, os_=1026 * 64), dict(d=0), dict(d=-64), dict(scale=0.0), dict(scale=-1.0),
                dict(scale=float("nan")), dict(scale=float("inf")), dict(scale=3e38), dict(nq=-2), dict(nk=-2), dict(nq=(1 << 24) + 2), dict(nk=(1 << 24) + 2), dict(mq=0), dict(mk=0), dict(mq=(1 << 24) + 1),
                dict(mk=(1 << 24) + 1), dict(nq=7), dict(nk=9), dict(cuq=C.c_void_p(4098)), dict(cuk=C.c_void_p(4097)), dict(lens=C.c_void_p(4099)), dict(qs=248), dict(qs=260), dict(ks=120),
                dict(vs=132), dict(os_=255), dict(os_=(1 << 21) + 8), dict(q=None), dict(k=None), dict(v=None), dict(o=None), dict(q=C.c_void_p(4104)), dict(v=C.c_void_p(4098)),
                dict(o=at(0)), dict(o=at(1)), dict(o=at(2)), dict(lse=at(3)), dict(lse=at(0)), dict(lse=at(1)), dict(lse=C.c_void_p(4097)), dict(ws=at(3), size=1 << 20)]:
        assert forward(**bad) == 1, bad
    need = L.ll_encoder_attn_workspace_bytes(2, 4, 2, 64, 4, 100000)
    assert need > 0 and forward(mk=100000) == 1
    assert forward(mk=100000, ws=at(9), size=need - 1) == 3 and forward(mk=100000, ws=C.c_void_p(4104), size=need) == 1
    assert forward(mk=100000, ws=at(9), lse=at(9), size=need) == 1
    assert forward(n=1 << 20, nq=0, nk=0, hq=1024, hkv=1024, qs=1 << 16, ks=1 << 16, vs=1 << 16, os_=1 << 16) == 4                  # 2^30 tiles
    assert forward(n=1, nq=0, nk=0, hq=1024, hkv=1, qs=1 << 16, ks=64, vs=64, os_=1 << 16, mq=1 << 24) == 4                       # 2^34 rows of a kv head


def test_encoder_attn_backward_refuses():
    L = B.lib()

    def backward(n=2, hq=4, hkv=2, d=64, scale=0.1, nq=8, nk=10, mq=4, mk=5, do=at(0), dos=256, q=at(1), qs=256, k=at(2), ks=128, v=at(3), vs=128, o=at(4), os_=256, lse=at(5), dq=at(6),
                 dqs=256, dk=at(7), dks=128, dv=at(8), dvs=128, ws=at(9), size=1 << 30):
        return L.ll_encoder_attn_backward(n, hq, hkv, d, scale, nq, nk, mq, mk, None, None, None, do, dos, q, qs, k, ks, v, vs, o, os_, lse, dq, dqs, dk, dks, dv, dvs, ws, size, None)

    assert backward(nq=0, nk=0) == 0
    for bad in [dict(n=0), dict(hkv=3), dict(d=0), dict(scale=0.0), dict(nq=7), dict(nk=9), dict(mq=0), dict(mk=0), dict(dos=248), dict(qs=248), dict(ks=120), dict(vs=120), dict(os_=248),
                dict(dqs=248), dict(dks=120), dict(dvs=124), dict(do=None), dict(q=None), dict(k=None), dict(v=None), dict(o=None), dict(lse=None), dict(dq=None), dict(dk=None), dict(dv=None),
                dict(do=C.c_void_p(4104)), dict(dv=C.c_void_p(4104)), dict(lse=C.c_void_p(4098)), dict(dq=at(0)), dict(dq=at(1)), dict(dk=at(2)), dict(dv=at(3)), dict(dk=at(6)), dict(dv=at(7)),
                dict(dq=at(4)), dict(dq=at(5)), dict(dk=at(9)), dict(ws=None), dict(ws=C.c_void_p(4104)), dict(ws=at(0)), dict(ws=at(5))]:
        assert backward(**bad) == 1, bad
    need = L.ll_encoder_attn_backward_workspace_bytes(2, 4, 2, 64, 8, 4, 5)
    assert need >= 4 * 8 * 2 * 4 and backward(size=need - 1) == 3
    assert backward(d=96, dos=384, qs=384, ks=192, vs=192, os_=384, dqs=384, dks=192, dvs=192) == 4


def test_workspace_sizes():
    """None where one workgroup does a tile, and 0 for what a call refuses."""
    L = B.lib()
    assert L.ll_encoder_attn_workspace_bytes(1, 12, 12, 128, 32760, 512) == 0
    few = L.ll_encoder_attn_workspace_bytes(1, 32, 8, 128, 1, 32000)
    assert 0 < few <= 8 * 512 * 32 * 130 * 4
    for bad in [(0, 4, 2, 64, 4, 5), (2, 4, 3, 64, 4, 5), (2, 4, 2, 80, 4, 5), (2, 4, 2, 64, 0, 5), (2, 4, 2, 64, 4, 0), (1 << 20, 1024, 1024, 64, 4, 5)]:
        assert L.ll_encoder_attn_workspace_bytes(*bad) == 0
        assert L.ll_encoder_attn_backward_workspace_bytes(*bad[:4], 8, *bad[4:]) == 0
    assert L.ll_encoder_attn_backward_workspace_bytes(2, 4, 2, 64, -1, 4, 5) == 0


@pytest.mark.parametrize("device", ["cpu", torch.device("cpu"), "meta"])
def test_a_gpu_is_needed(device):
    with pytest.raises(ValueError, match="GPU"):
        B.LayerNorm(64, device=device)
    with pytest.raises(ValueError, match="GPU"):
        B.EncoderAttention(4, 2, 64, device=device)


def on_the_cpu(cls, **kw):
    """An object whose tensors would be on the CPU, to reach the checks in front of its calls."""
    made = cls.__new__(cls)
    made.__dict__.update(_index=-1, _types={BF16: 0, F32: 1}, _bf16=BF16, _f32=F32, **kw)
    return made


def test_layer_norm_binding_refuses():
    norm = on_the_cpu(B.LayerNorm, features=64, eps=1e-5)
    x, w, stats = torch.zeros(6, 64, dtype=BF16), torch.zeros(64), torch.zeros(6, 2)
    for bad in [dict(x=x.half()), dict(x=x[:, :32]), dict(x=x.t()), dict(x=torch.zeros(6, 128, dtype=BF16)[:, ::2]), dict(y=x[:5]), dict(y=x.double()), dict(weight=torch.zeros(63)),
                dict(weight=torch.zeros(2, 64)), dict(weight=w.half()), dict(weight=w, bias=w.to(BF16)), dict(weight=torch.zeros(64, 2)[:, 0]), dict(weight=w, group_rows=3),
                dict(weight=torch.zeros(3, 64), group_rows=3), dict(stats=torch.zeros(6)), dict(stats=torch.zeros(6, 2, dtype=BF16)), dict(stats=torch.zeros(2, 6).t())]:
        with pytest.raises(ValueError):
            norm.forward(**{**dict(x=x, y=x.clone()), **bad})
    for bad in [dict(dy=x[:5]), dict(dx=x.float()), dict(residual=x.float()), dict(residual=x[:, :32]), dict(stats=None, x=x[:4]), dict(dweight=w.to(BF16)), dict(dweight=torch.zeros(2, 64)),
                dict(dbias=torch.zeros(3, 64), group_rows=3), dict(workspace=torch.zeros(8)), dict(workspace=torch.zeros(8, 2, dtype=torch.uint8)),
                dict(workspace=torch.zeros(16, dtype=torch.uint8)[::2])]:
        with pytest.raises(ValueError):
            norm.backward(**{**dict(dy=x, x=x, stats=stats, dx=x.clone()), **bad})


def test_encoder_attn_binding_refuses():
    attn = on_the_cpu(B.EncoderAttention, q_heads=4, kv_heads=2, head_dim=64, scale=0.125)
    q, k, lse, cu = torch.zeros(6, 4, 64, dtype=BF16), torch.zeros(10, 2, 64, dtype=BF16), torch.zeros(4, 6), torch.zeros(3, dtype=I32)
    good = dict(q=q, k=k, v=k, out=q.clone(), n_seqs=2, cu_q=cu, cu_k=cu)
    for bad in [dict(q=q.float()), dict(q=q[:, :2]), dict(k=k[:, :1]), dict(v=k[:9]), dict(out=q[:5]), dict(q=q.transpose(1, 2)), dict(lse=torch.zeros(6, 4)), dict(lse=lse.double()),
                dict(cu_q=cu.long()), dict(cu_q=cu[:2]), dict(cu_k=torch.zeros(4, dtype=I32)), dict(k_lens=cu), dict(k_lens=torch.zeros(4, dtype=I32)[::2]), dict(workspace=torch.zeros(4))]:
        with pytest.raises(ValueError):
            attn.forward(**{**good, **bad})
    with pytest.raises(B.LongLiveError):
        attn.forward(**{**good, "n_seqs": 0})
    back = dict(dout=q, q=q, k=k, v=k, out=q, lse=lse, dq=q.clone(), dk=k.clone(), dv=k.clone(), n_seqs=2, cu_q=cu, cu_k=cu)
    for bad in [dict(dout=q[:5]), dict(dq=q.float()), dict(dk=k[:9]), dict(dv=q), dict(lse=lse[:2]), dict(lse=lse.t().contiguous())]:
        with pytest.raises(ValueError):
            attn.backward(**{**back, **bad})
