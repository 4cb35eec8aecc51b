"""The sweeps over the keys that the encoder attention makes a second time (ll_encoder_attn*), on the GPU against the fp64 oracle.

Forward: a tile's reference is the largest score of its first block; where that turns out too low the tile is done again.  A workgroup is 128 query rows, 32 a wave, and two or three of
them share a CU.

Backward: where dQ's and dK/dV's workgroups are more than a CU each and dQ is not in runs, a tile of a sequence of more than 256 keys begins with delta = dout . out, of the rounded output, and is done
again if that is off by more than 2^-10 of a row's sum of P |dP - delta|: rows whose weights lie on few keys.  (Small calls and those in runs make delta first, and sweep once.)"""
import numpy as np
import pytest
import torch

from oracle import norm_and_encoder as O
from paper_2509_22622_amd import binding as B
from test_gpu_encoder_attn import BF16, check, normal

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rising", [0, 1])
@pytest.mark.parametrize("n_k", [288, 310, 330, 352, 416, 440])
def test_forward_again_with_waves_apart(n_k, rising, d):
    """9 to 14 blocks of 32 keys, which end in every place of the ring of four, and no runs; scores of every second wave rise by some 250 to the last block, those of the others hardly, so that
    the waves of a tile reach its end at different times."""
    n_seqs, heads, n_q = 8, 16, 512
    assert B.EncoderAttention(heads, heads, d).workspace_bytes(n_seqs, n_q, n_k) == 0
    along = torch.sign(normal((d,), 9).float())

    def change(q, k):
        rise = (torch.arange(len(k), device="cuda") % n_k).view(-1, 1, 1) * (250 / (d ** 0.5 * n_k))
        steep = (torch.arange(len(q), device="cuda") // 32 % 2 == rising).view(-1, 1, 1)
        return (steep * along + 0.1 * q.float()).to(BF16), (rise * along + 0.1 * k.float()).to(BF16)

    check(heads, heads, d, n_seqs * n_q, n_seqs * n_k, n_seqs=n_seqs, seed=n_k, back=False, change=change)


# sequences, query heads, kv heads, queries of each, states of each, lengths: launched one after the other, dQ not in runs (tests/test_encoder_way.py)
IN_TURN = [
    (5, 8, 8, 900, 600, [600, 256, 257, 100, 289]),
    (5, 16, 4, 460, 600, [599, 255, 258, 0, 320]),          # four heads share the states
    (7, 6, 6, 1000, 290, None),                             # two keys behind nine blocks
    (9, 5, 5, 770, 257, None),
]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("flat, sharp", [(0.3, 0.3), (0.3, 4.0), (4.0, 4.0)])
@pytest.mark.parametrize("n_seqs, hq, hkv, n_q, n_k, lens", IN_TURN)
def test_backward_again(n_seqs, hq, hkv, n_q, n_k, lens, flat, sharp, d):
    """Tiles with and without rows that need the second sweep, in every second stretch of queries, beside sequences whose delta comes first."""
    stretch = 128 * hkv // hq                                # tokens of a tile

    def change(q, k):
        steep = (torch.arange(len(q), device="cuda") % n_q // stretch % 2 == 1).view(-1, 1, 1)
        return (q.float() * torch.where(steep, sharp, flat)).to(BF16), k

    attn, (q, k, v, dout), _, made = check(hq, hkv, d, n_seqs * n_q, n_seqs * n_k, n_seqs=n_seqs, k_lens=lens, seed=n_k, change=change)
    again = {True: 0, False: 0}                              # tiles by whether a row of theirs is off
    for s in range(n_seqs):
        n = n_k if lens is None else lens[s]
        if n <= 256:
            continue
        at, to = slice(s * n_q, (s + 1) * n_q), slice(s * n_k, s * n_k + n)
        wide = lambda t, rows: t[rows].double().transpose(0, 1).contiguous()
        qs, ds, os_ = wide(q, at), wide(dout, at), wide(made["out"], at)
        ks, vs = (wide(t, to).repeat_interleave(hq // hkv, 0).transpose(1, 2).contiguous() for t in (k, v))
        p, dp, delta = torch.softmax(attn.scale * torch.bmm(qs, ks), -1), torch.bmm(ds, vs), (ds * os_).sum(-1)
        off = ((p * dp).sum(-1) - delta).abs() > 2.0 ** -10 * (p * (dp - delta.unsqueeze(-1)).abs()).sum(-1)
        tiles = off.unflatten(0, (hkv, hq // hkv)).any(1)    # rows of a kv head's tiles
        for first in range(0, n_q, stretch):
            for hit in tiles[:, first:first + stretch].any(1).tolist():
                again[hit] += 1
    if sharp > 1:
        assert again[True] > 0
    if flat < 1:
        assert again[False] > 0


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n_seqs, heads, n_q, n_k", [(6, 12, 900, 500), (1, 2, 300, 3000), (2, 3, 5, 600), (1, 1, 200, 100)])
@pytest.mark.parametrize("rise, most", [(18.0, 1.0), (15.5, 1.0), (13.0, 1.0), (10.0, 1.0), (20.5, 0.01), (6.5, 1.0), (5.4, 1.0), (0.0, 1.0), (60.0, 1.0)])
def test_large_values(n_seqs, heads, n_q, n_k, rise, most, d):
    """Values of up to 2^119 over the number of states, what the sums hold, in a batch of whole tiles, in runs, of few rows: the second half of the keys scores `rise` above the first, which is the
    reference at first, and the sums are of weights e^rise times as large."""
    attn = B.EncoderAttention(heads, heads, d)
    along = torch.sign(normal((d,), 9).float())
    up = (torch.arange(n_seqs * n_k, device="cuda") % n_k >= n_k // 2).view(-1, 1, 1) * (rise / d ** 0.5)
    q = (along + 0.1 * normal((n_seqs * n_q, heads, d), 1).float()).to(BF16)
    k = (up * along + 0.1 * normal((n_seqs * n_k, heads, d), 2).float()).to(BF16)
    v = (normal((n_seqs * n_k, heads, d), 3).float().clamp(-4, 4) / 4 * (most * 0.99 * 2.0 ** 119 / n_k)).to(BF16)
    v[:, :, 0] = most * 0.99 * 2.0 ** 119 / n_k             # a feature whose sum is as large as can be
    out, lse = torch.empty_like(q), torch.empty(heads, n_seqs * n_q, device="cuda")
    attn.forward(q, k, v, out, n_seqs=n_seqs, lse=lse, workspace=attn.workspace(n_seqs, n_q, n_k))
    want = O.attended(*(t.double().cpu().numpy() for t in (q, k, v)), attn.scale, n_seqs, None, None, None, n_q, n_k)
    for name, got in (("out", out), ("lse", lse)):
        value, off = want[name]
        err = np.abs(got.double().cpu().numpy() - value)
        assert (err <= off).all(), (name, (err / off).max())
