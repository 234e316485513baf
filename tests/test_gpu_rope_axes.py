"""Positions with more axes than a rotation's pairs use: the other columns do not matter."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
N = 128


@pytest.fixture(scope="module")
def hq():
    from paper_2606_23406_amd import hq as H
    H.lib()
    return H


def table(hq, pairs):
    freq = torch.from_numpy(100.0 ** (-np.arange(pairs) / pairs)).cuda()
    return hq.hq_rope_table(freq, 64)


@pytest.mark.parametrize("axes,used", [(3, 1), (3, 2), (4, 1), (4, 3), (2, 2)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_columns_that_no_pair_uses(hq, axes, used, interleaved):
    g = torch.Generator().manual_seed(axes + used)
    t = table(hq, 48)
    axis = [i * used // 48 for i in range(48)]
    x = torch.randn((33, 3 * N), generator=g).cuda()
    pos = torch.randint(0, 64, (33, axes), generator=g, dtype=torch.int32).cuda()
    want = hq.hq_rope(hq.Rope(t, interleaved=interleaved, axis=axis), x, pos[:, :used].contiguous())
    rope = hq.Rope(t, interleaved=interleaved, axis=axis if used > 1 else None, axes=axes)
    assert rope.axes == axes
    assert torch.equal(hq.hq_rope(rope, x, pos), want) and not torch.equal(want, x)
    assert rope.read_stats()["status"] == 0
    with pytest.raises(ValueError):
        hq.hq_rope(rope, x, pos[:, :1].contiguous())


@pytest.mark.parametrize("axes", [0, 1, 5, -1])
def test_refusals(hq, axes):
    with pytest.raises(ValueError):
        hq.Rope(table(hq, 64), axis=[0] * 63 + [1], axes=axes)
