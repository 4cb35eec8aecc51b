"""The sweeps over the keys that the encoder attention makes a second time (ll_encoder_attn*), on the GPU against the fp64 oracle.

Forward: a tile's reference is the largest score of its first block; where that turns out too low the tile is done again.  A workgroup is 128 query rows, 32 a wave, and two or three of
them share a CU."""
import pytest
import torch

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
