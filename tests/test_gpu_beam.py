"""Beam search's selection and the reordering of states against sorted candidates and copies: types, sizes, ties, masks, ended and
missing beams, strides, slots; both together with the one-token step."""
import pytest
import torch

from delta_testlib import select64

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
DEV = "cuda"
INF = float("inf")


@pytest.fixture(scope="module")
def hb():
    from paper_2311_06281_b200 import build_ext, heinsen_beam
    build_ext.build()
    heinsen_beam.lib()
    return heinsen_beam


def make(b, w, n, dtype, seed=0, spread=3.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    logits = (spread * torch.randn(b, w, n, device=DEV, generator=g)).to(dtype)
    scores = -10 + 2 * torch.randn(b, w, device=DEV, generator=g)
    return logits, scores


def compare(hb, logits, scores, keep, ended=None, end=0):
    got = hb.beam_select(logits, scores, keep, ended=ended, end_token=end)
    want = select64(logits, scores, keep, ended, end)
    assert torch.equal(got[1].long(), want[1]) and torch.equal(got[2].long(), want[2])
    # a sum of exponentials of float32's own (2^-21 each), and one rounding to float32
    finite = torch.isfinite(want[0])
    assert torch.equal(torch.isfinite(got[0]), finite)
    off = (got[0].double() - want[0])[finite].abs()
    assert (off <= 2.0 ** -21 + want[0][finite].abs() * 2.0 ** -24).all()
    return got


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("b,w,n,keep", [(1, 1, 1, 1), (2, 3, 5, 15), (1, 4, 2049, 4), (3, 5, 8192, 8), (2, 2, 8193, 16), (2, 16, 5003, 17),
                                        (40, 8, 40001, 8), (1, 64, 3001, 64), (5, 3, 100003, 6), (0, 2, 10, 2)])
def test_selection(hb, b, w, n, keep, dtype):
    compare(hb, *make(b, w, n, dtype, seed=n), keep)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,keep", [(7, 7), (3000, 5), (20000, 33)])
def test_equal_logits_are_taken_in_order(hb, n, keep, dtype):
    logits = torch.zeros(2, 3, n, device=DEV, dtype=dtype)
    logits[1, 2, n // 2:] = 1.0
    logits[0, 1, ::2] = -0.0  # both zeros are one value
    compare(hb, logits, torch.tensor([[-1.0, -1.0, -1.0], [-2.0, -3.0, -2.5]], device=DEV), keep)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("keep", [1, 6, 20])
def test_masked_logits(hb, keep, dtype):
    """Few tokens are allowed, none at all, or all but a few."""
    logits, scores = make(4, 3, 30000, dtype, seed=3)
    allowed = torch.randint(30000, (4, 3, 4), device=DEV)
    masked = torch.full_like(logits, -INF).scatter(2, allowed, logits.gather(2, allowed))
    masked[1, 0] = -INF
    masked[2] = -INF
    masked[3, 1] = logits[3, 1]
    compare(hb, masked, scores, keep)


@pytest.mark.parametrize("n,keep", [(9, 4), (9, 18), (50000, 8)])
def test_ended_missing_and_broken_beams(hb, n, keep):
    logits, scores = make(5, 4, n, F32, seed=1)
    ended = torch.zeros(5, 4, dtype=torch.bool, device=DEV)
    ended[0, 1] = ended[2] = ended[4, 3] = True
    scores[1, 2:] = -INF      # the first step: some beams are not there yet
    scores[2, 3] = -INF
    scores[3, 0] = float("nan")
    logits[3, 1, n // 2] = float("nan")
    logits[3, 2, 0] = INF
    logits[4, 3] = float("nan")  # of an ended beam: not looked at
    for end in (0, 2, n - 1):
        compare(hb, logits, scores, keep, ended, end)
        compare(hb, logits, scores, keep, ended.to(torch.uint8), end)
    compare(hb, logits, torch.full_like(scores, -INF), keep)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("b,w,n,keep", [(6, 64, 90001, 64), (6, 64, 90001, 3), (37, 8, 40007, 17)])
def test_rows_that_a_thread_block_reads_in_many_steps(hb, b, w, n, keep, dtype):
    """Rows of all kinds in one call: far larger logits late (or early), rising and falling ones, equal ones, a masked beginning,
    a masked end, single logits that are not masked, an infinity and a NaN late in the row."""
    logits, scores = make(b, w, n, dtype, seed=n + keep)
    ramp = torch.linspace(-40, 40, n, device=DEV)
    for g in range(b):  # one kind for each group, so that its best come from every row of it
        x = logits[g].float()
        kind = g % 9
        if kind == 0:
            x[:, n // 2:] += 500
        elif kind == 1:
            x[:, n // 2:] -= 500
        elif kind == 2:
            x = ramp.expand(w, n)
        elif kind == 3:
            x = (-ramp).expand(w, n)
        elif kind == 4:
            x = torch.ones_like(x)
        elif kind == 5:
            x[:, :n - 5000] = -INF
        elif kind == 6:
            x[:, 5000:] = -INF
        elif kind == 7:
            x = torch.full_like(x, -INF)
            x[:, 31000:31003] = 2.0
        else:
            x[0, n - 9] = INF
            x[1, n - 9] = float("nan")
        logits[g] = x.to(dtype)
    compare(hb, logits, scores, keep)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_strides_of_logits(hb, dtype):
    g = torch.Generator(device=DEV).manual_seed(1)
    big = torch.randn(4, 7, 3011, device=DEV, generator=g).to(dtype)
    scores = torch.randn(2, 3, device=DEV, generator=g)
    for x in (big[1:3, 2:5, 3:], big[::2, ::3, :3001], big.transpose(0, 1)[:2, :3, 1:100], big[:1, :3].expand(2, 3, 3011)):
        compare(hb, x, scores, 5)


def test_a_kept_workspace_and_captured_calls(hb):
    logits, scores = make(6, 4, 30001, BF16)
    other = make(6, 4, 30001, BF16, seed=9)
    ws = hb.workspace(logits, scores)
    graph = torch.cuda.CUDAGraph()
    hb.beam_select(logits, scores, workspace=ws)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        got = hb.beam_select(logits, scores, workspace=ws)
    for x in (other, make(6, 4, 30001, BF16)):
        logits.copy_(x[0])
        scores.copy_(x[1])
        graph.replay()
        want = select64(logits, scores, 4)
        assert torch.equal(got[1].long(), want[1]) and torch.equal(got[2].long(), want[2])


@pytest.mark.parametrize("dtype", [F32, BF16, torch.int8, torch.float64])
@pytest.mark.parametrize("b,w,row", [(1, 1, (4, 4)), (3, 4, (2, 8, 16)), (5, 7, (3, 5)), (2, 16, (64,)), (2, 30, (33, 4)), (2, 64, (17, 8)), (9, 5, (100, 100)),
                                     (2, 3, (1,)), (0, 3, (4,)), (2, 3, (0,))])
def test_reordering(hb, b, w, row, dtype):
    g = torch.Generator(device=DEV).manual_seed(w)
    state = (100 * torch.randn(b * w + 3, *row, device=DEV, generator=g)).to(dtype)
    slots = torch.randperm(b * w + 3, device=DEV, generator=g)[:b * w].to(torch.int32).view(b, w)
    parents = torch.randint(w, (b, w), device=DEV, generator=g, dtype=torch.int32)
    for s in (slots, None):
        at = torch.arange(b * w, device=DEV).view(b, w) if s is None else s.long()
        want = state.clone()
        want[at] = state[at.gather(1, parents.long())]
        assert hb.beam_reorder(state, parents, slots=s) is state
        assert torch.equal(state, want)


def test_rows_without_a_parent_stay(hb):
    state = torch.arange(12.0, device=DEV).view(6, 2).clone()
    parents = torch.tensor([[1, 0, 7], [-1, 0, 1]], dtype=torch.int32, device=DEV)
    slots = torch.tensor([[0, 1, 2], [3, -1, 6]], dtype=torch.int32, device=DEV)
    want = state.clone()
    want[[0, 1]] = state[[1, 0]]
    assert torch.equal(hb.beam_reorder(state, parents, slots=slots), want)


def test_reordering_counts_as_a_modification(hb):
    state = torch.randn(4, 8, device=DEV)
    kept = (state * state.clone().requires_grad_()).sum()
    hb.beam_reorder(state, torch.tensor([[1, 0]], dtype=torch.int32, device=DEV))
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        kept.backward()


def test_offsets_past_32_bits(hb):
    """Rows of a pool of more than 2^32 bytes, and logits more than 2^31 elements apart."""
    state = torch.empty(9, 1 << 27, device=DEV, dtype=torch.float32)
    for i in range(9):
        state[i, :1000], state[i, -1000:] = i, 10 * i
    slots = torch.tensor([[8, 0], [3, 7]], dtype=torch.int32, device=DEV)
    hb.beam_reorder(state, torch.tensor([[1, 0], [0, 0]], dtype=torch.int32, device=DEV), slots=slots)
    order = [8, 1, 2, 3, 4, 5, 6, 3, 0]
    assert [int(x) for x in state[:, 0]] == order and [int(x) for x in state[:, -1]] == [10 * i for i in order]
    flat = state.view(-1).view(BF16)
    logits = flat.as_strided((2, 2, 1001), ((1 << 31) + 8, 1024, 1))
    logits.copy_(make(2, 2, 1001, BF16)[0])
    compare(hb, logits, make(2, 2, 1, F32)[1], 4)


def test_a_search_over_states(hb):
    """Selection, reordering and steps of the delta rule as a search runs them, against states that are copied."""
    from paper_2311_06281_b200 import heinsen_delta as hd
    g = torch.Generator(device=DEV).manual_seed(2)
    b, w, h, d, n = 3, 4, 2, 64, 300
    embed = torch.randn(n, 3, h, d, device=DEV, generator=g)
    out = torch.randn(n, h * d, device=DEV, generator=g) * 0.3
    gates = torch.rand(n, 2, h, device=DEV, generator=g)
    state = torch.randn(b * w, h, d, d, device=DEV, generator=g)
    plain = state.double().clone()
    scores = torch.full((b, w), -INF, device=DEV)
    scores[:, 0] = 0
    plain_scores = scores.clone()
    tokens = torch.randint(n, (b * w,), device=DEV, generator=g)
    for _ in range(6):
        q, k, v = embed[tokens].unbind(1)
        k = torch.nn.functional.normalize(k, dim=-1)
        log_a, beta = -gates[tokens, 0], gates[tokens, 1].contiguous()
        o = hd.delta_attention_step(q, k, v, log_a, beta, state)
        scores, parents, tokens = hb.beam_select((o.flatten(1) @ out.T).view(b, w, n), scores, ended=None)
        hb.beam_reorder(state, parents)
        old = plain * log_a.double().exp()[..., None, None]
        error = v.double() - (k.double().unsqueeze(-2) @ old).squeeze(-2)
        plain = old + k.double().unsqueeze(-1) * (beta.double()[..., None] * error).unsqueeze(-2)
        o = (q.double().unsqueeze(-2) @ plain).squeeze(-2) * d ** -0.5
        best, par, tok = select64((o.flatten(1) @ out.double().T).view(b, w, n), plain_scores, w)
        assert torch.equal(par, parents.long()) and torch.equal(tok, tokens.long())
        plain = plain.view(b, w, h, d, d)[torch.arange(b, device=DEV)[:, None], par].flatten(0, 1)
        plain_scores = best.float()
        tokens = tokens.long().flatten()
        torch.testing.assert_close(state.double(), plain, rtol=1e-4, atol=1e-5)
