"""The cross-attention part of a block as it is trained, made of the library's calls: norm, query product, attention to the prompts' states, output product added to the
stream, and the way back to the stream, the norm's weights, the states; then the same captured and replayed; and the part as it serves single tokens.

Tolerance of the whole: the path from the inputs to the farthest gradient rounds to bfloat16 twelve times (h, q, k and v, the weights, the output, y; and back d(out), dS, dq, dh, dx,
with P once more), 2^-8 / sqrt(3) each and independent, 7.8e-3 together; products of normal numbers and the softmax of scores of size 1 carry each on at its own relative size, so
1.5e-2 of relative L2 is twice that."""
import numpy as np
import pytest
import torch

from paper_2509_22622_amd import binding as B

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def normal(shape, seed, std=1.0, mean=0.0, dtype=BF16):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * std + mean).to(dtype).cuda()


class Block:
    """Two videos of `frames` frames each, every frame with its own scale and shift; prompts of different lengths, padded."""

    def __init__(self, frames=3, per_frame=50, heads=4, d=64, lens=(40, 23)):
        self.n, self.width = len(lens), heads * d
        self.tokens, self.group, self.longest = self.n * frames * per_frame, per_frame, max(lens)
        w = self.width
        self.x, self.states, self.dy = normal((self.tokens, w), 1, 2.0, 0.5), normal((self.n * self.longest, w), 2), normal((self.tokens, w), 3)
        self.scale, self.shift = normal((self.n * frames, w), 4, 0.2, 1.0, torch.float32), normal((self.n * frames, w), 5, 0.2, 0.0, torch.float32)
        self.wq, self.wk, self.wv, self.wo = (normal((w, w), 6 + i, w ** -0.5) for i in range(4))
        self.lens = torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.heads, self.d = heads, d
        self.norm, self.attn = B.LayerNorm(w, eps=1e-6), B.EncoderAttention(heads, heads, d)
        self.q_proj, self.k_proj, self.v_proj, self.o_proj = (B.Linear(t) for t in (self.wq, self.wk, self.wv, self.wo))
        self.back = [B.Linear(t.t().contiguous()) for t in (self.wq, self.wk, self.wv, self.wo)]
        e = lambda *s, dtype=BF16: torch.zeros(*s, dtype=dtype, device="cuda")
        t, s = self.tokens, self.n * self.longest
        self.h, self.q, self.o, self.y, self.do, self.dq, self.dh, self.dx = (e(t, w) for _ in range(8))
        self.k, self.v, self.dk, self.dv, self.ds = (e(s, w) for _ in range(5))
        self.stats, self.lse = e(t, 2, dtype=torch.float32), e(heads, t, dtype=torch.float32)
        self.dscale, self.dshift = e(*self.scale.shape, dtype=torch.float32), e(*self.scale.shape, dtype=torch.float32)
        self.ws = self.norm.backward_workspace(t, per_frame)
        self.forward_ws = self.attn.workspace(self.n, t // self.n, self.longest)
        self.backward_ws = self.attn.backward_workspace(self.n, t, t // self.n, self.longest)

    def split(self, t):
        return t.unflatten(1, (self.heads, self.d))

    def step(self):
        s = self.split
        self.norm.forward(self.x, self.h, weight=self.scale, bias=self.shift, group_rows=self.group, stats=self.stats)
        self.q_proj.forward(self.h, self.q)
        self.k_proj.forward(self.states, self.k)
        self.v_proj.forward(self.states, self.v)
        batch = dict(n_seqs=self.n, k_lens=self.lens)
        self.attn.forward(s(self.q), s(self.k), s(self.v), s(self.o), lse=self.lse, workspace=self.forward_ws, **batch)
        self.o_proj.forward(self.o, self.y, residual=self.x)
        self.back[3].forward(self.dy, self.do)
        self.attn.backward(s(self.do), s(self.q), s(self.k), s(self.v), s(self.o), self.lse, s(self.dq), s(self.dk), s(self.dv), workspace=self.backward_ws, **batch)
        self.back[0].forward(self.dq, self.dh)
        self.back[1].forward(self.dk, self.ds)
        self.back[2].forward(self.dv, self.ds, residual=self.ds)
        self.norm.backward(self.dh, self.x, self.stats, self.dx, weight=self.scale, dweight=self.dscale, dbias=self.dshift, group_rows=self.group, residual=self.dy,
                           workspace=self.ws)

    def made(self):
        return {k: getattr(self, k) for k in ("y", "dx", "ds", "dscale", "dshift", "dq", "dk", "dv")}

    def exact(self):
        leaves = [t.double().requires_grad_(True) for t in (self.x, self.states, self.scale, self.shift)]
        x, states, scale, shift = leaves
        of = torch.arange(self.tokens, device="cuda") // self.group
        h = torch.nn.functional.layer_norm(x, (self.width,), eps=1e-6) * scale[of] + shift[of]
        q, k, v = (self.split(a @ w.double().t()) for a, w in ((h, self.wq), (states, self.wk), (states, self.wv)))
        outs = []
        for i, n in enumerate(self.lens.tolist()):
            a, b = slice(i * self.tokens // self.n, (i + 1) * self.tokens // self.n), slice(i * self.longest, i * self.longest + n)
            heads = [torch.softmax(q[a, j] @ k[b, j].t() * self.d ** -0.5, -1) @ v[b, j] for j in range(self.heads)]
            outs.append(torch.stack(heads, 1))
        y = torch.cat(outs).flatten(1) @ self.wo.double().t() + x
        grads = torch.autograd.grad(y, leaves, self.dy.double())
        return dict(zip(("y", "dx", "ds", "dscale", "dshift"), (y.detach(), *grads)))


def off(got, want):
    return ((got.double() - want).norm() / want.norm()).item()


@pytest.mark.parametrize("shape", [dict(), dict(frames=2, per_frame=33, heads=3, d=128, lens=(1, 70, 0)), dict(frames=5, per_frame=260, heads=2, d=64, lens=(300,))])
def test_a_training_step(shape):
    b = Block(**shape)
    b.step()
    torch.cuda.synchronize()
    want = b.exact()
    made = b.made()
    for name, t in want.items():
        assert off(made[name], t) <= 1.5e-2, (name, off(made[name], t))
    # what the residual path leaves alone: with the stream's own part taken off the rest is as near, at its own size and that part's rounding
    assert off(made["y"].double() - b.x.double(), want["y"] - b.x.double()) <= 1.5e-2 + 2.0 ** -8 * (want["y"].norm() / (want["y"] - b.x.double()).norm()).item()
    for i, n in enumerate(b.lens.tolist()):
        assert (b.dk.unflatten(0, (b.n, -1))[i, n:] == 0).all() and (b.dv.unflatten(0, (b.n, -1))[i, n:] == 0).all()


def test_a_captured_step():
    b = Block()
    b.step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.step()
    for i, lens in enumerate(([40, 1], [0, 40], [17, 33], [40, 40])):
        for j, t in enumerate((b.x, b.states, b.dy)):
            t.copy_(normal(t.shape, 1000 * i + j))
        b.lens.copy_(torch.tensor(lens, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        replayed = {k: v.clone() for k, v in b.made().items()}
        b.step()
        torch.cuda.synchronize()
        assert all(torch.equal(replayed[k], v) for k, v in b.made().items()), i


def test_single_tokens():
    """One new token of each of many sequences: norm, query product, attention to each one's states, output product."""
    n, hq, hkv, d, longest = 37, 8, 2, 128, 600
    w = hq * d
    lens = [(i * 131) % (longest + 1) for i in range(n)]
    x, wq, wo = normal((n, w), 1), normal((w, w), 2, w ** -0.5), normal((w, w), 3, w ** -0.5)
    ends = np.concatenate([[0], np.cumsum(lens)])
    k, v = (normal((int(ends[-1]), hkv, d), 4 + i) for i in range(2))
    g = normal((w,), 6, 0.1, 1.0)
    norm, attn = B.LayerNorm(w), B.EncoderAttention(hq, hkv, d)
    h, q, o, y = (torch.empty_like(x) for _ in range(4))
    norm.forward(x, h, weight=g)
    B.Linear(wq).forward(h, q)
    s = lambda t: t.unflatten(1, (hq, d))
    attn.forward(s(q), k, v, s(o), n_seqs=n, cu_k=torch.tensor(ends, dtype=torch.int32, device="cuda"), max_k=longest, workspace=attn.workspace(n, 1, longest))
    B.Linear(wo).forward(o, y, residual=x)
    torch.cuda.synchronize()
    hx = torch.nn.functional.layer_norm(x.double(), (w,), eps=1e-5) * g.double()
    qx = (hx @ wq.double().t()).unflatten(1, (hq, d))
    ox = torch.zeros(n, hq, d, dtype=torch.float64, device="cuda")
    for i in range(n):
        for j in range(hq):
            if lens[i]:
                kk, vv = (t[ends[i]:ends[i + 1], j // (hq // hkv)].double() for t in (k, v))
                ox[i, j] = torch.softmax(kk @ qx[i, j] * d ** -0.5, 0) @ vv
    assert off(y, ox.flatten(1) @ wo.double().t() + x.double()) <= 1.5e-2
    assert off(o, ox.flatten(1)) <= 1.5e-2 and (o[[i for i in range(n) if lens[i] == 0]] == 0).all()
