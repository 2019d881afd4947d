"""Sizes whose blocks are more than one grid takes: products of so many rows that they are launched again and
again, of so many columns that they are taken in halves, sums and gradients that walk over their work.
Of small whole numbers, whose sums are exact."""
import pytest
import torch

import paper_2112_15345_amd as hg

pytestmark = pytest.mark.gpu

F32, BF16, E4M3 = torch.float32, torch.bfloat16, torch.float8_e4m3fn
ROWS, COLS, WIDE = (1 << 30) + 5, (1 << 29) + 77, (1 << 27) + 3


@pytest.fixture(autouse=True)
def give_back():
    yield
    torch.cuda.empty_cache()


def numbers(n, below, dtype=BF16):
    """0, 1, 2, .. again and again."""
    return torch.arange(n, dtype=torch.int32, device="cuda").remainder_(below).to(dtype)


def test_rows():
    x, w = numbers(ROWS, 113)[:, None], torch.full((1, 1), 2.0, dtype=BF16, device="cuda")
    y = hg.linear(x, w, bias=torch.ones(1, device="cuda"), residual=x, act="relu")[0]
    assert torch.equal(y, (3 * x.float() + 1).to(BF16))  # (rounded once)


def test_rows_backward():
    dy = torch.ones(ROWS, 1, dtype=BF16, device="cuda")
    x, w = numbers(ROWS, 2)[:, None], torch.full((1, 1), 3.0, dtype=BF16, device="cuda")
    for act, pre in (("none", None), ("relu", dy)):
        dx, dw, db = hg.linear_grad(dy, x, w, pre=pre, act=act, dw_dtype=F32)
        assert bool((dx == 3).all())
        # (sums of a thread's or part's own are exact; the last ones are rounded)
        assert abs(float(db) - ROWS) <= 2.0 ** -20 * ROWS
        assert abs(float(dw) - ROWS // 2) <= 2.0 ** -20 * ROWS
        del dx


@pytest.mark.parametrize("eight", [False, True])
def test_columns(eight):
    x = torch.tensor([[1.0], [2.0]], device="cuda")
    w, bias, residual = numbers(COLS, 61)[:, None], numbers(COLS, 31), numbers(COLS, 7).expand(2, COLS)
    if eight:
        w = numbers(COLS, 9, E4M3)[:, None]
        kw = dict(x_scale=torch.tensor([1.0, 4.0], device="cuda"), w_scale=numbers(COLS, 3, F32))
        y, pre = hg.linear(x.to(E4M3), w, bias=bias, residual=residual, keep_pre=True, **kw)
        by = [kw["w_scale"].to(BF16), 8 * kw["w_scale"].to(BF16)]
    else:
        y, pre = hg.linear(x.to(BF16), w, bias=bias, residual=residual, act="relu", keep_pre=True)
        by = [1, 2]
    w = w[:, 0].to(BF16)
    for row in (0, 1):
        want = w * by[row] + bias
        assert torch.equal(pre[row], want)
        want += residual[row]
        assert torch.equal(y[row], want)


def test_columns_backward():
    """dx over so many columns, and dw and dbias of as many rows and columns as a walk takes."""
    dy = torch.tensor([[1.0], [2.0]], dtype=BF16, device="cuda")
    w = numbers(COLS, 61)[None]
    dx = hg.linear_grad(dy, w.expand(2, COLS), w, want_dw=False, want_dbias=False)[0]
    assert torch.equal(dx[0], w[0]) and torch.equal(dx[1], 2 * w[0])
    dw = hg.linear_grad(dy, w.expand(2, COLS), w, want_dx=False, want_dbias=False)[1]
    assert torch.equal(dw[0], 3 * w[0])
    del dx, dw, w
    dy = numbers(WIDE, 100).expand(2, WIDE)
    db = hg.linear_grad(dy, dy[:, :0], dy[:1, :0].expand(WIDE, 0))[2]
    assert torch.equal(db, 2 * dy[0].float())


def test_norm_weights():
    x = torch.ones(1, WIDE, dtype=BF16, device="cuda")
    dy = numbers(WIDE, 100)[None]
    dw = hg.rms_norm_grad(dy, x, eps=0.0, want_dx=False, want_dweight=True)[1]
    assert float((dw - dy[0].float()).abs().max()) <= 100 * 2.0 ** -20
