"""Beam search's selection where few logits decide: a NaN beside masked logits, equal beams at every alignment, logits that differ by
less than their sums with a score can say, one beam with a long list."""
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


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("b,w,n,keep", [(1, 4, 5003, 4), (2, 8, 100003, 8), (3, 16, 50257, 16), (40, 8, 8193, 20), (2, 64, 3001, 64), (1, 7, 2050, 7)])
def test_equal_beams_are_taken_in_order(hb, b, w, n, keep, dtype):  # noqa: F811
    """The same logits in every beam, in rows that begin at every place within 16 bytes: candidates are equal to the last bit, so w * N + n
    decides."""
    logits, scores = make(b, 1, n, dtype, seed=n)
    logits, scores = logits.expand(b, w, n).contiguous(), scores.expand(b, w).contiguous()
    order = torch.sort(logits.double().flatten(1), dim=-1, descending=True, stable=True).indices[:, :keep]
    values, parents, tokens = hb.beam_select(logits, scores, keep)
    assert torch.equal(parents.long() * n + tokens.long(), order)
    first = logits.flatten(1).gather(1, order)
    same = first[:, 1:] == first[:, :-1]
    assert torch.equal(values[:, 1:][same], values[:, :-1][same])


@pytest.mark.parametrize("w,n", [(1, 3000), (3, 3000), (2, 70001)])
def test_logits_nearer_than_their_sums_can_say(hb, w, n):  # noqa: F811
    """Logits of a beam that a sum in 64 bits cannot tell apart stay in their order, however many are asked for; between beams the first
    comes first."""
    logits = torch.zeros(1, w, n, device=DEV)
    places = [n - 1, 5, n // 2, 700]
    for i, at in enumerate(places):
        logits[:, :, at] = (4 - i) * 1e-25
    want = (places + [i for i in range(n) if i not in places])[:64]
    for keep in (1, 2, 3, 5, 16, 17, 64):
        _, parents, tokens = hb.beam_select(logits, torch.zeros(1, w, device=DEV), keep)
        assert tokens[0].tolist() == want[:keep] and not parents.any()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("w,keep", [(1, 8), (1, 16), (1, 64), (2, 9), (3, 64)])
def test_few_beams_with_a_large_vocabulary(hb, w, keep, dtype):  # noqa: F811
    compare(hb, *make(2, w, 150000, dtype, seed=keep), keep)
