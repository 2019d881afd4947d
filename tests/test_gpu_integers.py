"""linear on 8-bit integers: sums are exact whatever the tiles, parts and alignment; scales, epilogues,
the longest sums, other streams, capture."""
import pytest
import torch

import dense_ref as R
import paper_2112_15345_amd as hg
from test_gpu_dense_linear import ACTS, SIZES, rand

pytestmark = pytest.mark.gpu

F32, F16, BF16, I8 = torch.float32, torch.float16, torch.bfloat16, torch.int8


def ints(*shape, seed=0, lo=-128, hi=127):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randint(lo, hi + 1, shape, generator=g, device="cuda", dtype=torch.int32).to(I8)


def scales(n, seed=0):
    return (rand(n, seed=seed).abs() + 0.1) * 0.01


def check(x, w, got, xs, ws, bias=None, act="none", residual=None, out=BF16):
    """The sum is exact and rounded to 32 bits, once for each of up to 127 parts, which 8 threads
    add (24 levels at most); two products with scales; then as in linear."""
    y, pre = got
    a, b = x.double() * xs.double()[:, None], w.double() * ws.double()[:, None]
    z = a @ b.t()
    size = (a.abs() @ b.abs().t()) * (32 * R.E)
    if bias is not None:
        z = z + bias.double()
        size = size + R.E * z.abs()
    v = R.act(z, act)
    vsize = 1.13 * size + 16 * R.E * z.abs() if act != "none" else size
    if residual is not None:
        v = v + residual.double()
        vsize = vsize + R.E * v.abs()
    assert y.dtype == out and y.shape == z.shape
    R.assert_close(y, v, R.rounding(v, out) + vsize, "y")
    if pre is not None:
        R.assert_close(pre, z, R.rounding(z, out) + size, "pre")


@pytest.mark.parametrize("m,k,n", SIZES + [(0, 8, 8), (4, 0, 9), (40, 0, 9), (3, 8, 0),
                                           (4100, 1040, 2056), (8200, 1024, 4104)])
def test_forward(m, k, n):
    for i, act in enumerate(ACTS):
        out = [BF16, F32, F16, BF16][i]
        x, w = ints(m, k, seed=m + k), ints(n, k, seed=n)
        xs, ws = scales(m, seed=1), scales(n, seed=2)
        bias = [None, rand(n, seed=4), rand(n, seed=4, dtype=BF16), rand(n, seed=4)][i]
        res = rand(m, n, dtype=out, seed=5) if i in (1, 3) else None
        got = hg.linear(x, w, bias=bias, act=act, residual=res, x_scale=xs, w_scale=ws,
                        out_dtype=out, keep_pre=i >= 2)
        assert (got[1] is not None) == (i >= 2)
        check(x, w, got, xs, ws, bias, act, res, out)


# few rows (whole and with their depth in parts), 64 x 64, 128 x 128, 256 x 256 tiles, depths in parts,
# rows through registers, rows copied first
EXACT = [(1, 2048, 8192), (9, 8192, 40), (32, 4096, 100), (300, 96, 136), (2100, 64, 1032),
         (8200, 1024, 4104), (300, 65_536, 64), (130, 20_000, 144), (300, 97, 137),
         (1001, 2050, 4099), (400, 30_001, 260)]


@pytest.mark.parametrize("m,k,n", EXACT)
def test_sums_are_exact(m, k, n):
    """Sums below 2^24 come out whole: elements as small as that takes."""
    most = max(1, min(127, int((2 ** 24 / k) ** 0.5)))
    x, w = ints(m, k, seed=1, lo=-most, hi=most), ints(n, k, seed=2, lo=-most, hi=most)
    one = torch.ones(max(m, n), device="cuda")
    y = hg.linear(x, w, x_scale=one[:m], w_scale=one[:n], out_dtype=F32)[0]
    assert torch.equal(y.double(), x.double() @ w.double().t())


@pytest.mark.parametrize("m", [1, 40, 300])
def test_longest_sums(m):
    """131071 products of -128 and -128 are the largest sum, 127 and -128 the lowest."""
    k, n = 131_071, 70
    x, w = torch.full((m, k), -128, dtype=I8, device="cuda"), torch.empty(n, k, dtype=I8, device="cuda")
    w[:] = torch.tensor([-128, 127], device="cuda")[torch.arange(n, device="cuda") % 2][:, None]
    one = torch.ones(max(m, n), device="cuda")
    y = hg.linear(x, w, x_scale=one[:m], w_scale=one[:n], out_dtype=F32)[0]
    want = x[:1].double() @ w.double().t()
    assert float((y.double() - want).abs().max()) <= 2.0 ** 31 * 24 * R.E
    more = torch.zeros(2, k + 1, dtype=I8, device="cuda")
    with pytest.raises(hg.HGError) as e:
        hg.linear(more, more, x_scale=one[:2], w_scale=one[:2])
    assert e.value.status == hg.HG_EUNSUPPORTED


def test_strides_and_layouts():
    big = ints(400, 700, seed=1)
    w = ints(130, 300, seed=2)
    xs, ws = scales(400), scales(130, seed=3)
    for x in (big[:, 16:316], big[:, 3:303], big[::2, 1:301], big[:1, :300].expand(400, 300),
              ints(300, 400, seed=5).t()):
        m = x.shape[0]
        check(x, w, hg.linear(x, w, x_scale=xs[:m], w_scale=ws), xs[:m], ws)
    check(big[:5, 3:303], w, hg.linear(big[:5, 3:303], w, x_scale=xs[:5], w_scale=ws), xs[:5], ws)
    every = scales(800, seed=6)[::2]  # (scales that are not contiguous)
    check(big[:, :300], w, hg.linear(big[:, :300], w, x_scale=every, w_scale=ws), every, ws)


@pytest.mark.parametrize("m,k,n", [(9, 64, 300), (300, 96, 136), (2100, 64, 1032), (300, 97, 137)])
def test_scales_that_are_not_numbers(m, k, n):
    """A row that quantize or layer_norm could not write has a scale of NaN: its results are NaN, the
    others' are not.  Scales at the ends of the range meet the sum, not each other."""
    x, w = ints(m, k, seed=1), ints(n, k, seed=2)
    xs, ws = scales(m), scales(n, seed=1)
    want = hg.linear(x, w, x_scale=xs, w_scale=ws, out_dtype=F32)[0]
    bad = xs.clone()
    bad[3] = float("nan")
    y = hg.linear(x, w, x_scale=bad, w_scale=ws, out_dtype=F32)[0]
    rest = torch.arange(m, device="cuda") != 3
    assert torch.isnan(y[3]).all()
    R.assert_close(y[rest], want[rest], want[rest].abs() * 4 * R.E, "the other rows")
    small, large = torch.full_like(xs, 2.0 ** -126), torch.full_like(ws, 2.0 ** 120)
    y = hg.linear(x, w, x_scale=small, w_scale=large, out_dtype=F32)[0]
    assert torch.equal(y.double(), (x.double() @ w.double().t()) * 2.0 ** -6)


def test_binding_refuses():
    x, w = ints(4, 16), ints(8, 16)
    one = torch.ones(8, device="cuda")
    for call in (lambda: hg.linear(x, w), lambda: hg.linear(x, w, x_scale=one[:4]),
                 lambda: hg.linear(x, w, x_scale=one[:3], w_scale=one),
                 lambda: hg.linear(x, w.to(BF16), x_scale=one[:4], w_scale=one),
                 lambda: hg.linear(x, w.to(torch.uint8), x_scale=one[:4], w_scale=one),
                 lambda: hg.linear(x, w, x_scale=one[:4], w_scale=one, out_dtype=I8),
                 lambda: hg.linear(x, w, x_scale=one[:4].double(), w_scale=one)):
        with pytest.raises(ValueError):
            call()


def test_repeats_streams_and_capture():
    m, k, n = 500, 2000, 300
    x, w, xs, ws = ints(m, k, seed=1), ints(n, k, seed=2), scales(m), scales(n, seed=1)
    first = hg.linear(x, w, x_scale=xs, w_scale=ws)[0]
    other = torch.cuda.Stream()
    torch.cuda.synchronize()
    again = hg.linear(x, w, x_scale=xs, w_scale=ws, stream=other)[0]
    torch.cuda.synchronize()
    assert torch.equal(first, again)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = [hg.linear(x[:rows], w, x_scale=xs[:rows], w_scale=ws)[0] for rows in (1, 20, m)]
    for seed in (3, 4, 5):
        x.copy_(ints(m, k, seed=seed))
        want = [hg.linear(x[:rows], w, x_scale=xs[:rows], w_scale=ws)[0] for rows in (1, 20, m)]
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))


# depths that are cut (few rows; 64 x 64 and 128 x 128 tiles, by LDS and through registers; many parts)
CUT = [(1, 8192, 1024), (9, 8192, 40), (32, 4096, 100), (64, 8192, 1024), (300, 65_536, 64),
       (130, 20_000, 144), (400, 30_001, 260), (300, 8192, 1024), (2, 131_071, 33)]


@pytest.mark.parametrize("out", [F32, BF16])
@pytest.mark.parametrize("m,k,n", CUT)
def test_parts_that_cancel(m, k, n, out):
    """Parts far past 2^24 that cancel: the sum is exact before it is rounded, however the depth is cut."""
    x, w = ints(m, k, seed=1, lo=64), ints(n, k, seed=2, lo=64)
    w[:, k // 2:] *= -1
    one = torch.ones(max(m, n), device="cuda")
    y = hg.linear(x, w, x_scale=one[:m], w_scale=one[:n], out_dtype=out)[0]
    # (whole numbers below 2^53; to float32 and then to the result's type, as the header has it)
    assert torch.equal(y, (x.double() @ w.double().t()).float().to(out))


def test_a_row_is_the_same_among_others():
    k, n = 8192, 1024
    x, w, xs, ws = ints(2100, k, seed=1, lo=64), ints(n, k, seed=2, lo=64), scales(2100), scales(n)
    w[:, k // 2:] *= -1
    first = hg.linear(x[:1], w, x_scale=xs[:1], w_scale=ws, out_dtype=F32)[0]
    for m in (2, 20, 33, 64, 300, 2100):
        y = hg.linear(x[:m], w, x_scale=xs[:m], w_scale=ws, out_dtype=F32)[0]
        assert torch.equal(y[:1], first), m
