"""The norms around a block and the gated norm of its heads against their float64 forms: values and every gradient, over
types, widths with and without whole 16-byte rows, broadcast gates, absent parts; refusals."""
import pytest
import torch

from attention_testlib import block_norms64, close, gated_norm64, leaf64

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
DEV = "cuda"


@pytest.fixture(scope="module")
def ha():
    from paper_2311_06281_b200 import build_ext, heinsen_attention
    build_ext.build()
    heinsen_attention.lib()
    return heinsen_attention


WIDTHS = [1, 7, 64, 80, 128, 200, 256, 500, 512, 1000, 1001, 1024, 2048, 2051, 4096, 5120, 8192, 16384, 16383]


def tensors(rows, d, dtype, wdtype, gate, post, seed=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    rnd = lambda *s, to=dtype: torch.randn(*s, device=DEV, generator=g).to(to)  # noqa: E731
    shape = (rows, d) if gate != "wide" else (3, rows, d)
    t = {"x": rnd(*shape), "branch": rnd(*shape), "pre": rnd(d, to=wdtype), "post": rnd(d, to=wdtype) if post else None,
         "gate": None if gate is None else rnd(*shape) if gate == "row" else rnd(3, 1, d)}
    return t, rnd(*shape), rnd(*shape)


@pytest.mark.parametrize("dtype,wdtype", [(BF16, BF16), (BF16, F32), (F32, F32)])
@pytest.mark.parametrize("gate,post", [(None, True), ("row", True), ("wide", True), ("row", False), (None, False)])
@pytest.mark.parametrize("d", WIDTHS)
def test_block_norms(ha, d, gate, post, dtype, wdtype):
    rows = 1 + (d * 37) % 19
    t, dr, dy = tensors(rows, d, dtype, wdtype, gate, post, seed=d)
    ins = {n: x.requires_grad_() if x is not None else None for n, x in t.items()}
    call = lambda f, x: f(x["x"], x["branch"], x["pre"], x["post"], x["gate"])  # noqa: E731
    r, y = call(lambda a, b, c, p, g: ha.block_norms(a, b, c, post_weight=p, gate=g, scale=0.7, eps=1e-5), ins)
    wide = {n: leaf64(x) for n, x in ins.items()}
    want = call(lambda a, b, c, p, g: block_norms64(a, b, c, p, g, 0.7, 1e-5), wide)
    close(r, want[0], "r")
    close(y, want[1], "y")
    have = [n for n, x in ins.items() if x is not None]
    got = torch.autograd.grad([r, y], [ins[n] for n in have], [dr, dy])
    back = torch.autograd.grad(want, [wide[n] for n in have], [dr.double(), dy.double()])
    for n, a, b in zip(have, got, back):
        assert a.dtype == ins[n].dtype
        close(a, b, "d" + n)


@pytest.mark.parametrize("rows", [1, 2, 1000, 4099])
def test_block_norms_many_rows_and_one_gradient(ha, rows):
    t, dr, dy = tensors(rows, 256, BF16, BF16, "wide", True)
    ins = {n: x.requires_grad_() for n, x in t.items()}
    for use in ("r", "y"):
        r, y = ha.block_norms(ins["x"], ins["branch"], ins["pre"], post_weight=ins["post"], gate=ins["gate"])
        wide = {n: leaf64(x) for n, x in ins.items()}
        want = block_norms64(wide["x"], wide["branch"], wide["pre"], wide["post"], wide["gate"])
        names = ["x", "branch", "gate", "post"] + (["pre"] if use == "y" else [])
        got = torch.autograd.grad(r if use == "r" else y, [ins[n] for n in names], dr)
        back = torch.autograd.grad(want[0] if use == "r" else want[1], [wide[n] for n in names], dr.double())
        for n, a, b in zip(names, got, back):
            close(a, b, f"d{n} through {use}")


@pytest.mark.parametrize("dtype,wdtype", [(BF16, BF16), (BF16, F32), (F32, F32)])
@pytest.mark.parametrize("gate", [True, False])
@pytest.mark.parametrize("d", WIDTHS)
def test_gated_norm(ha, d, gate, dtype, wdtype):
    g = torch.Generator(device=DEV).manual_seed(d)
    rows = 1 + (d * 29) % 23
    rnd = lambda *s, to=dtype: torch.randn(*s, device=DEV, generator=g).to(to)  # noqa: E731
    x, z, w, dy = rnd(rows, 3, d), rnd(rows, 3, d) if gate else None, rnd(d, to=wdtype), rnd(rows, 3, d)
    ins = [a.requires_grad_() if a is not None else None for a in (x, z, w)]
    y = ha.gated_norm(*ins)
    wide = [leaf64(a) for a in ins]
    want = gated_norm64(*wide)
    close(y, want, "y")
    have = [i for i in range(3) if ins[i] is not None]
    for i, a, b in zip(have, torch.autograd.grad(y, [ins[i] for i in have], dy),
                       torch.autograd.grad(want, [wide[i] for i in have], dy.double())):
        close(a, b, ("dx", "dgate", "dweight")[i])


def test_gated_norm_many_rows(ha):
    x, z, dy = (torch.randn(20000, 128, device=DEV).to(BF16) for _ in range(3))
    w = torch.randn(128, device=DEV).requires_grad_()
    y = ha.gated_norm(x, z, w)
    w64 = leaf64(w)
    want = gated_norm64(x, z, w64)
    close(y, want, "y")
    close(torch.autograd.grad(y, w, dy)[0], torch.autograd.grad(want, w64, dy.double())[0], "dweight")


def test_rows_of_zeros_unaligned_bases_and_no_rows(ha):
    z = torch.zeros(4, 64, device=DEV, dtype=BF16)
    w = torch.ones(64, device=DEV, dtype=BF16)
    r, y = ha.block_norms(z, z, w, post_weight=w)
    assert (r == 0).all() and (y == 0).all()
    x = torch.randn(5 * 64 + 1, device=DEV).to(BF16)[1:].view(5, 64)
    close(ha.gated_norm(x, None, w), gated_norm64(x, None, w), "an unaligned base")
    none = torch.empty(0, 64, device=DEV, dtype=BF16).requires_grad_()
    v = w.clone().requires_grad_()
    r, y = ha.block_norms(none, none, v, post_weight=v)
    assert r.shape == (0, 64) and (torch.autograd.grad(y.sum(), v)[0] == 0).all()
    assert (torch.autograd.grad(ha.gated_norm(none, none, v).sum(), v)[0] == 0).all()


def test_refusals(ha):
    x, w = torch.randn(4, 6, 64, device=DEV), torch.ones(64, device=DEV)
    for bad in (lambda: ha.block_norms(x, x[:2], w), lambda: ha.block_norms(x, x, w[:3]),
                lambda: ha.block_norms(x, x, w, gate=x[:, :3]), lambda: ha.block_norms(x.transpose(0, 1), x.transpose(0, 1), w),
                lambda: ha.block_norms(x.cpu(), x.cpu(), w.cpu()), lambda: ha.gated_norm(x, x[:1], w),
                lambda: ha.gated_norm(x, x[:, :1], w)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: ha.block_norms(x, x, w.to(BF16)), lambda: ha.gated_norm(x.half(), None, w),
                lambda: ha.block_norms(x, x, w, gate=x.to(BF16))):
        with pytest.raises(TypeError):
            bad()
    wide = torch.zeros(2, 16385, device=DEV)
    with pytest.raises(ha.HeinsenScanError):
        ha.gated_norm(wide, None, torch.ones(16385, device=DEV))
