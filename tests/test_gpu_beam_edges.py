"""Beam search's selection where few logits decide: a NaN beside masked logits."""
import pytest
import torch

from test_gpu_beam import BF16, DEV, F32, INF, compare, hb, make  # noqa: F401

pytestmark = pytest.mark.gpu


def rows(x, aligned):
    """The same values; rows that begin at addresses of 16 bytes, or one behind the other."""
    if not aligned:
        return x.contiguous()
    wide = torch.zeros(*x.shape[:-1], (x.shape[-1] + 15) // 8 * 8, device=DEV, dtype=x.dtype)
    wide[..., :x.shape[-1]] = x
    return wide[..., :x.shape[-1]]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("aligned", [False, True])
@pytest.mark.parametrize("b,w,n", [(1, 3, 2049), (1, 2, 4097), (100, 2, 8193), (1, 4, 1), (3, 2, 30011), (40, 3, 16390)])
def test_a_nan_beside_masked_logits(hb, b, w, n, aligned, dtype):  # noqa: F811
    """Alone behind the last full part, alone in a masked stretch, beside padding: the beam has no candidates, the others have theirs."""
    for at in sorted({n - 1, n // 2, 0}):
        logits, scores = make(b, w, n, dtype, seed=n + at)
        logits[:, 0, min(8, n):] = -INF  # a few tokens are allowed
        logits[:, 0, at] = float("nan")
        compare(hb, rows(logits, aligned), scores, min(4, w * n))
    logits[:, 0] = -INF  # and where nothing else is
    logits[:, 0, n // 2] = float("nan")
    compare(hb, rows(logits, aligned), scores, min(4, w * n))
