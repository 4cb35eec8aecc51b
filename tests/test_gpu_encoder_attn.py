"""ll_encoder_attn and ll_encoder_attn_backward on the GPU against the fp64 oracle (oracle/norm_and_encoder.py, which derives the tolerances).

Besides its own bound each output keeps the benchmark's relative L2 error of 5e-3: two roundings to bfloat16 (a weight, the result), 2^-8 / sqrt(3) each, are
3.2e-3 together."""
import math

import numpy as np
import pytest
import torch

from oracle import norm_and_encoder as O
from paper_2509_22622_amd import binding as B

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def normal(shape, seed, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * std).to(BF16).cuda()


def ints(x):
    return None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")


def spaced(t, extra):
    """The same rows, `extra` numbers further apart, NaN between them."""
    wide = torch.full((t.shape[0], t[0].numel() + extra) if len(t) else (0, t.shape[1] * t.shape[2] + extra), math.nan, dtype=t.dtype, device=t.device)
    view = wide[:, :wide.shape[1] - extra].unflatten(1, t.shape[1:])
    view.copy_(t)
    return view


def f64(t):
    return t.double().cpu().numpy()


def check(hq, hkv, d, n_q, n_k, n_seqs=1, cu_q=None, cu_k=None, k_lens=None, max_q=None, max_k=None, scale=None, q_std=1.0, extra=0, seed=0, back=True, poison=True, lone=(), change=None):
    """One forward and backward pass.  Rows that are seen by nobody hold NaN where `poison`; what is written starts as 7 and stays so where nothing is to be written."""
    q, k, v, dout = normal((n_q, hq, d), seed + 1, q_std), normal((n_k, hkv, d), seed + 2), normal((n_k, hkv, d), seed + 3), normal((n_q, hq, d), seed + 4)
    if change is not None:
        q, k = change(q, k)
    attn = B.EncoderAttention(hq, hkv, d, scale)
    mq = (n_q if cu_q is not None else n_q // n_seqs) if max_q is None else max_q
    mk = (n_k if cu_k is not None else n_k // n_seqs) if max_k is None else max_k
    q_rows, k_rows = O.spans(cu_q, None, n_seqs, n_q, max(mq, 1)), O.spans(cu_k, k_lens, n_seqs, n_k, max(mk, 1))
    if poison:
        for t, rows in ((q, q_rows), (dout, q_rows), (k, k_rows), (v, k_rows)):
            dead = torch.ones(len(t), dtype=torch.bool)
            for a, n, _ in rows:
                dead[a:a + n] = False
            t[dead.cuda()] = math.nan
    want = O.attended(*(np.nan_to_num(f64(t)) for t in (q, k, v)), attn.scale, n_seqs, cu_q, cu_k, k_lens, max(mq, 1), max(mk, 1), np.nan_to_num(f64(dout)) if back else None)
    batch = dict(n_seqs=n_seqs, cu_q=ints(cu_q), cu_k=ints(cu_k), k_lens=ints(k_lens), max_q=max_q, max_k=max_k)
    q, k, v, dout = (spaced(t, extra) if extra else t for t in (q, k, v, dout))
    seven = lambda *shape: torch.full(shape, 7.0, dtype=BF16, device="cuda")
    out, lse = spaced(seven(n_q, hq, d), extra) if extra else seven(n_q, hq, d), torch.full((hq, n_q), 7.0, device="cuda")
    made = {"out": out, "lse": lse}
    attn.forward(q, k, v, out, lse=lse, workspace=attn.workspace(n_seqs, mq, mk), **batch)
    if back:
        made |= {"dq": seven(n_q, hq, d), "dk": seven(n_k, hkv, d), "dv": seven(n_k, hkv, d)}
        attn.backward(dout, q, k, v, out, lse, made["dq"], made["dk"], made["dv"], workspace=attn.backward_workspace(n_seqs, n_q, mq, mk), **batch)
    torch.cuda.synchronize()
    for name, t in made.items():
        got, (value, off) = f64(t), want[name]
        there = ~np.isnan(value)
        assert (got[~there] == 7.0).all(), f"{name}: written where nothing is to be written"
        a, b, off = got[there], value[there], off[there]
        fine = np.isfinite(b)
        assert np.array_equal(a[~fine], b[~fine]) and np.isfinite(a[fine]).all(), name
        err = np.abs(a[fine] - b[fine])
        assert (err <= off[fine]).all(), (name, err.max(), (err[off[fine] > 0] / off[fine][off[fine] > 0]).max())
        if name not in lone and b[fine].size >= 64 and np.abs(b[fine]).max() > 0:
            assert np.linalg.norm(err) <= 5e-3 * np.linalg.norm(b[fine]), (name, np.linalg.norm(err) / np.linalg.norm(b[fine]))
    return attn, (q, k, v, dout), batch, made


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n_k", [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200, 257, 500])
def test_keys(n_k, d):
    check(2, 2, d, 70, n_k, seed=n_k)
    check(2, 2, d, 3, n_k, seed=n_k)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n_q", [1, 2, 15, 16, 17, 31, 32, 33, 64, 127, 128, 129, 255, 300])
def test_queries(n_q, d):
    check(2, 2, d, n_q, 90, seed=n_q)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq, hkv", [(1, 1), (4, 1), (6, 2), (5, 5), (40, 8), (7, 1), (33, 1), (64, 2)])
@pytest.mark.parametrize("n_q", [1, 5, 40])
def test_heads(hq, hkv, n_q, d):
    check(hq, hkv, d, n_q, 77, seed=hq)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n_q, n_k, hq, hkv", [(1, 5000, 4, 1), (1, 3000, 32, 8), (8, 9000, 4, 1), (40, 4001, 3, 1), (200, 2500, 2, 2), (1, 130, 1, 1), (32, 20000, 1, 1)])
def test_long_states(n_q, n_k, hq, hkv, d):
    """Keys dealt to several workgroups, in both directions."""
    check(hq, hkv, d, n_q, n_k, seed=n_k)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n_q, n_k, hq, hkv", [(3000, 40, 2, 1), (5000, 130, 1, 1), (700, 300, 6, 2), (2049, 65, 3, 3)])
def test_long_queries(n_q, n_k, hq, hkv, d):
    """Query rows dealt to several workgroups for dK and dV."""
    check(hq, hkv, d, n_q, n_k, seed=n_q)


RAGGED = dict(n_seqs=5, cu_q=[0, 37, 37, 38, 190, 200], cu_k=[0, 130, 131, 140, 140, 260])


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq, hkv", [(2, 2), (8, 2)])
def test_ragged(hq, hkv, d):
    """Sequences without queries, without states, with one of them; rows in front of the first and behind the last are left as they were."""
    check(hq, hkv, d, 200, 260, **RAGGED, max_q=152, max_k=130)
    check(hq, hkv, d, 200, 260, **RAGGED)
    check(hq, hkv, d, 230, 300, n_seqs=5, cu_q=[9 + x for x in RAGGED["cu_q"]], cu_k=[20 + x for x in RAGGED["cu_k"]], max_q=152, max_k=130)
    check(hq, hkv, d, 5, 260, n_seqs=5, cu_k=RAGGED["cu_k"], max_k=130)                              # a row each
    check(hq, hkv, d, 200, 260, **RAGGED, k_lens=[100, 5, 0, 3, 300], max_q=152, max_k=130)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n_q", [1, 30, 150])
def test_padded(n_q, d):
    """As many rows each, states behind a sequence's length are NaN and reach nothing; their gradients are zeros."""
    for lens in ([70, 0, 1, 33], [0, 0, 0, 0], [-5, 70, 64, 1000], [1, 1, 1, 1]):
        check(3, 3, d, 4 * n_q, 4 * 70, n_seqs=4, k_lens=lens)
    check(3, 3, d, 4 * n_q, 4 * 700, n_seqs=4, k_lens=[70, 500, 600, 300], max_k=400)


def test_offsets_out_of_range():
    """Offsets and lengths that are wrong make rows absent, and nothing else."""
    check(2, 1, 64, 50, 60, n_seqs=3, cu_q=[-10, 20, 5, 90], cu_k=[5, 2, 50, 1000], max_q=50, max_k=60)
    check(2, 1, 64, 50, 60, n_seqs=2, cu_q=[0, 40, 50], cu_k=[0, 40, 60], max_q=10, max_k=15)
    check(2, 1, 64, 50, 60, n_seqs=2, cu_q=[60, 70, 80], cu_k=[-5, -3, -1], max_q=50, max_k=60)


@pytest.mark.parametrize("d", [64, 128])
def test_strides(d):
    check(4, 2, d, 45, 70, extra=8)
    check(4, 2, d, 450, 700, extra=264)
    q = normal((33, 3 * 2 * d), 1)                               # one product's output
    qs, ks, vs = (t.unflatten(1, (2, d)) for t in q.split(2 * d, 1))
    a, b = torch.empty(33, 2, d, dtype=BF16, device="cuda"), torch.empty(33, 2, d, dtype=BF16, device="cuda")
    attn = B.EncoderAttention(2, 2, d)
    attn.forward(qs, ks, vs, a, workspace=attn.workspace(1, 33, 33))
    attn.forward(qs.contiguous(), ks.contiguous(), vs.contiguous(), b, workspace=attn.workspace(1, 33, 33))
    assert torch.equal(a, b)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n_q, n_k", [(100, 20), (100, 300), (100, 700), (3, 700), (20, 4000)])
@pytest.mark.parametrize("q_std", [0.01, 4.0, 30.0])
def test_sharp_and_flat(n_q, n_k, q_std, d):
    """Weights that are all alike, and weights on few keys, where dP - delta cancels: the second sweep.  (Where one key has all the weight the gradients of the
    scores are what is left of a difference, and only the bound holds.)"""
    check(2, 2, d, n_q, n_k, q_std=q_std, seed=3, lone=("dq", "dk") if q_std > 10 else ())


def test_scale():
    for scale in (1e-6, 0.01, 1.0):
        check(2, 1, 64, 50, 100, scale=scale)


def test_one_key_has_no_gradient():
    _, _, _, made = check(3, 3, 128, 90, 1)
    assert (made["dq"] == 0).all() and (made["dk"] == 0).all()
    _, _, _, made = check(2, 2, 64, 40, 4, n_seqs=4, q_std=9.0)
    assert (made["dq"] == 0).all() and (made["dk"] == 0).all()


def test_nothing():
    attn = B.EncoderAttention(4, 2, 64)
    q, none, k = normal((9, 4, 64), 1), normal((0, 4, 64), 1), normal((0, 2, 64), 1)
    out, lse, dq = torch.full_like(q, 7.0), torch.empty(4, 9, device="cuda"), torch.full_like(q, 7.0)
    attn.forward(q, k, k, out, lse=lse)
    attn.backward(q, q, k, k, out, lse, dq, k.clone(), k.clone(), workspace=attn.backward_workspace(1, 9, 9, 0))
    assert (out == 0).all() and torch.isneginf(lse).all() and (dq == 0).all()
    states = normal((5, 2, 64), 2)
    dk, dv = torch.full_like(states, 7.0), torch.full_like(states, 7.0)
    attn.forward(none, states, states, none.clone(), lse=lse[:, :0].contiguous())
    attn.backward(none, none, states, states, none, lse[:, :0].contiguous(), none.clone(), dk, dv)
    assert (dk == 0).all() and (dv == 0).all()


def test_numbers_that_are_none():
    """NaN in one query, key or value reaches what it must, and no other sequence."""
    q, k, v = normal((40, 2, 64), 1), normal((60, 2, 64), 2), normal((60, 2, 64), 3)
    q[3, 0, 5], k[35, 1, 0], v[20, 0, 9], v[59, 1, 9] = math.nan, math.nan, math.inf, math.nan
    attn, out = B.EncoderAttention(2, 2, 64), torch.empty_like(q)
    attn.forward(q, k, v, out, n_seqs=2, workspace=attn.workspace(2, 20, 30))
    bad = ~torch.isfinite(out)
    want = torch.zeros_like(bad)
    want[3, 0] = True
    want[:20, 0, 9] = True
    want[20:, 1] = True
    assert torch.equal(bad, want)
    rows = [r for r in range(20) if r != 3]
    assert torch.isinf(out[rows, 0, 9]).all()


def test_repeats_and_order_of_sequences():
    """The same bits again; and each sequence of a batch comes out as it does in another place of a batch of the same sizes."""
    n_seqs, hq, hkv, d = 4, 4, 2, 128
    attn, (q, k, v, dout), batch, made = check(hq, hkv, d, 4 * 50, 4 * 300, n_seqs=n_seqs)
    order = [2, 0, 3, 1]
    swap = lambda t: t.unflatten(0, (n_seqs, -1))[order].flatten(0, 1).contiguous()
    for _ in range(2):
        again = {n: torch.empty_like(t) for n, t in made.items()}
        ws, back = attn.workspace(n_seqs, 50, 300), attn.backward_workspace(n_seqs, 200, 50, 300)
        attn.forward(swap(q), swap(k), swap(v), again["out"], lse=again["lse"], n_seqs=n_seqs, workspace=ws)
        attn.backward(swap(dout), swap(q), swap(k), swap(v), again["out"], again["lse"], again["dq"], again["dk"], again["dv"], n_seqs=n_seqs, workspace=back)
        for n in ("out", "dq", "dk", "dv"):
            assert torch.equal(again[n], swap(made[n])), n


def test_differences():
    """Gradients against differences of the forward pass.  Both sides are rounded to bfloat16; along a direction of many features those roundings average out: with r
    of 2^-8 / sqrt(3) an output and N outputs of size s, f = sum(out dout) is off by about r s sqrt(N), here 0.03, and twice that over 2 e = 1 is 3 % of what is compared."""
    n_q, n_k, hq, hkv, d, e = 60, 50, 4, 2, 64, 0.5
    q, k, v, dout = normal((n_q, hq, d), 1), normal((n_k, hkv, d), 2), normal((n_k, hkv, d), 3), normal((n_q, hq, d), 4)
    attn, out, lse = B.EncoderAttention(hq, hkv, d), torch.empty_like(q), torch.empty(hq, n_q, device="cuda")
    g = [torch.empty_like(t) for t in (q, k, v)]
    attn.forward(q, k, v, out, lse=lse, workspace=attn.workspace(1, n_q, n_k))
    attn.backward(dout, q, k, v, out, lse, *g, workspace=attn.backward_workspace(1, n_q, n_q, n_k))

    def f(q, k, v):
        o = torch.empty_like(q)
        attn.forward(q, k, v, o, workspace=attn.workspace(1, n_q, n_k))
        return (o.double() * dout.double()).sum().item()

    for i in range(3):
        along = torch.sign(g[i].float())                                     # the direction of steepest ascent, entry by entry
        args = [q, k, v]
        got = []
        for step in (e / 8, -e / 8):
            moved = (args[i].float() + step * along).to(BF16)
            got.append((f(*args[:i], moved, *args[i + 1:]), (moved.double() - args[i].double())))
        want = ((got[0][1] - got[1][1]) * g[i].double()).sum().item()
        assert abs(got[0][0] - got[1][0] - want) <= 0.05 * abs(want), (i, got[0][0] - got[1][0], want)


@pytest.mark.parametrize("n_q, n_k", [(1, 3000), (90, 200), (700, 40)])
def test_graph(n_q, n_k):
    """A captured step, replayed with other inputs and other lengths between eager calls, and on several streams at once with a workspace each."""
    n_seqs, hq, hkv, d = 3, 4, 2, 64
    tensors = [normal((n_seqs * n, h, d), i) for i, (n, h) in enumerate(((n_q, hq), (n_k, hkv), (n_k, hkv), (n_q, hq)))]
    q, k, v, dout = tensors
    lens = ints([n_k, n_k // 2, 0])
    attn = B.EncoderAttention(hq, hkv, d)

    def make():
        return {"out": torch.empty_like(q), "lse": torch.empty(hq, n_seqs * n_q, device="cuda"), "dq": torch.empty_like(q), "dk": torch.empty_like(k), "dv": torch.empty_like(v),
                "ws": attn.workspace(n_seqs, n_q, n_k), "back": attn.backward_workspace(n_seqs, n_seqs * n_q, n_q, n_k)}

    def step(o):
        attn.forward(q, k, v, o["out"], n_seqs=n_seqs, k_lens=lens, lse=o["lse"], workspace=o["ws"])
        attn.backward(dout, q, k, v, o["out"], o["lse"], o["dq"], o["dk"], o["dv"], n_seqs=n_seqs, k_lens=lens, workspace=o["back"])

    held = make()
    step(held)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(held)
    for i, new in enumerate(([1, n_k, 5], [n_k, n_k, n_k], [0, 0, 0], [n_k - 1, 2, n_k // 3])):
        for j, t in enumerate(tensors):
            t.copy_(normal(t.shape, 100 * i + j))
        lens.copy_(ints(new))
        graph.replay()
        want = make()
        step(want)
        torch.cuda.synchronize()
        assert all(torch.equal(held[n], want[n]) for n in ("out", "lse", "dq", "dk", "dv")), i
    streams, outs = [torch.cuda.Stream() for _ in range(3)], [make() for _ in range(3)]
    for s, o in zip(streams, outs):
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            step(o)
    torch.cuda.synchronize()
    for o in outs:
        assert all(torch.equal(o[n], want[n]) for n in ("out", "lse", "dq", "dk", "dv"))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n_q, n_k, hq, hkv", [(300, 500, 2, 2), (100, 2500, 1, 1), (3, 700, 4, 1), (1200, 200, 2, 1)])
def test_rising_scores(n_q, n_k, hq, hkv, d):
    """Scores that rise from the first key to the last by some 250 (2^360): whatever a row's reference is at first, it has to follow.  The keys that have weight all point one
    way, and a row's dS add up to zero: dq is what is left of a difference, and only its bound holds.  So is dk, whose queries all point one way and whose dS have either sign: 1200 queries
    over 200 keys in 64 bits with nothing rounded but dS, to bfloat16, leave 7.7e-3 of it, and sum |dS| |q| is 126 times its size."""
    along = torch.sign(normal((d,), 9).float())

    def change(q, k):
        rise = torch.arange(len(k), device="cuda").view(-1, 1, 1) * (250 / (d ** 0.5 * len(k)))
        return (along + 0.1 * q.float()).to(BF16), (rise * along + 0.1 * k.float()).to(BF16)

    check(hq, hkv, d, n_q, n_k, change=change, lone=("dq", "dk"))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n_q, n_k, hq, hkv", [(130, 1700, 8, 8), (3, 2000, 32, 32), (300, 1100, 4, 2), (40, 5000, 2, 1)])
def test_runs_that_are_joined(n_q, n_k, hq, hkv, d):
    assert B.EncoderAttention(hq, hkv, d).workspace_bytes(1, n_q, n_k) > 0
    check(hq, hkv, d, n_q, n_k)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n_q", [2, 130])
def test_runs_without_keys(n_q, d):
    """Runs sized for the longest sequence, of which others have few or none."""
    attn = B.EncoderAttention(8, 8, d)
    assert attn.workspace_bytes(3, n_q, 3000) > 0 and attn.workspace_bytes(3, n_q, 200000) > 0
    check(8, 8, d, 3 * n_q, 3 * 3000, n_seqs=3, k_lens=[0, 3000, 33])
    check(8, 8, d, 3 * n_q, 150, n_seqs=3, cu_q=[0, n_q, 2 * n_q, 3 * n_q], cu_k=[0, 1, 1, 150], max_q=n_q, max_k=200000)


@pytest.mark.parametrize("n_q", [1, 3, 40])
@pytest.mark.parametrize("hq, hkv", [(1024, 1), (1024, 1024), (1000, 8)])
def test_most_heads(hq, hkv, n_q):
    check(hq, hkv, 64, n_q, 5)


def test_many_sequences():
    g = torch.Generator().manual_seed(1)
    n_seqs = 3001
    cu_q, cu_k = ([0] + torch.randint(0, 4, (n_seqs,), generator=g).cumsum(0).tolist() for _ in range(2))
    check(2, 1, 64, cu_q[-1] + 2, cu_k[-1] + 3, n_seqs=n_seqs, cu_q=cu_q, cu_k=cu_k, max_q=3, max_k=3)
    check(4, 2, 128, 700, 700 * 5, n_seqs=700, k_lens=torch.randint(0, 6, (700,), generator=g).tolist())


@pytest.mark.parametrize("n_q, n_k", [(1100, 1100), (4, 1100), (40, 1100)])
def test_far_rows(n_q, n_k):
    """Rows 2^21 numbers apart, all of a call's tensors side by side in one array of 2.3e9 numbers: the same bits as without gaps."""
    hq, hkv, d, far = 2, 1, 64, 1 << 21
    base, used = torch.empty(1100 * far, dtype=BF16, device="cuda"), 0

    def place(n, h):
        nonlocal used
        used += h * d
        return base.as_strided((n, h, d), (far, d, 1), used - h * d)

    attn, near, apart = B.EncoderAttention(hq, hkv, d), [], []
    ws, back = attn.workspace(1, n_q, n_k), attn.backward_workspace(1, n_q, n_q, n_k)
    q, k, v, dout = normal((n_q, hq, d), 1), normal((n_k, hkv, d), 2), normal((n_k, hkv, d), 3), normal((n_q, hq, d), 4)
    for make, ins in ((lambda n, h: torch.empty(n, h, d, dtype=BF16, device="cuda"), near), (place, apart)):
        ins += [make(*t.shape[:2]).copy_(t) for t in (q, k, v, dout)]
        out, lse = make(n_q, hq), torch.empty(hq, n_q, device="cuda")
        dq, dk, dv = make(n_q, hq), make(n_k, hkv), make(n_k, hkv)
        attn.forward(*ins[:3], out, lse=lse, workspace=ws)
        attn.backward(ins[3], *ins[:3], out, lse, dq, dk, dv, workspace=back)
        torch.cuda.synchronize()
        ins += [out, lse, dq, dk, dv]
    assert all(torch.equal(a, b) for a, b in zip(near, apart))
