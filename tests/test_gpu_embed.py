"""embed and embed_grad: types, odd sizes and strides, ids that repeat or count for nothing, every way
the ids are sorted and the rows cut into chunks, adding in place, other streams, capture.  Sums of small
whole numbers are exact in 32 bits, so that most gradients are compared bit for bit."""
import ctypes

import pytest
import torch

import dense_ref as R
import paper_2112_15345_amd as hg
from paper_2112_15345_amd import dense

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def rand(*shape, dtype=F32, seed=0, scale=1.0):
    return (torch.randn(shape, generator=gen(seed), device="cuda") * scale).to(dtype)


def whole(*shape, dtype=F32, seed=0, most=4):
    return torch.randint(-most, most + 1, shape, generator=gen(seed), device="cuda").to(dtype)


def some_ids(n, nodes, kind, seed=0):
    g = gen(seed)
    if kind == "one":
        return torch.full((n,), nodes - 1, device="cuda")
    if kind == "words":
        u = torch.rand(n, generator=g, device="cuda", dtype=torch.float64)
        ids = (torch.exp(u * torch.log(torch.tensor(nodes + 1.0, dtype=torch.float64))) - 1).long()
        ids = (ids.clamp(0, nodes - 1) * 7919) % nodes
        return torch.where(torch.rand(n, generator=g, device="cuda") < 0.05, -1, ids)
    ids = torch.randint(nodes, (n,), generator=g, device="cuda")
    return ids.sort(descending=kind == "down")[0] if kind in ("up", "down") else ids


def sums(dy, ids, nodes):
    ok = (ids >= 0) & (ids < nodes)
    d = torch.zeros(nodes, dy.shape[1], dtype=torch.float64, device="cuda")
    if len(ids) and bool((ids == ids[0]).all()) and bool(ok[0]):  # (the additions below would queue)
        d[ids[0]] = dy.double().sum(0)
        return d
    return d.index_add_(0, ids[ok], dy[ok].double())


@pytest.mark.parametrize("table_dtype", [F32, F16, BF16])
@pytest.mark.parametrize("out", [F32, F16, BF16])
@pytest.mark.parametrize("dim", [1, 3, 8, 100, 128, 1000, 2048, 5001])
def test_rows(dim, out, table_dtype):
    nodes, scale = 37, 5.5
    wide = rand(nodes, dim + 3, dtype=table_dtype, seed=dim)
    for table in (wide[:, :dim], wide[:, 1:dim + 1].contiguous()):
        for n in (0, 1, 5, 1000):
            ids = torch.randint(-1, nodes, (n,), generator=gen(n), device="cuda")
            y = hg.embed(table, ids, scale=scale, out_dtype=out)
            assert y.dtype == out and y.shape == (n, dim)
            want = table.double()[ids.clamp(min=0)] * scale
            want[ids < 0] = 0
            # one product in 32 bits, one rounding
            R.assert_close(y, want, R.rounding(want, out) + want.abs() * 2 ** -24, "y")


def test_rows_that_are_none():
    table = rand(10, 40, seed=1)
    table[3, 5] = float("inf")
    ids = torch.tensor([3, -1, 10, -2, 1 << 40, 9], device="cuda")
    y = hg.embed(table, ids)
    assert torch.equal(y[[0, 5]], table[[3, 9]]) and not y[1].any()
    assert torch.isnan(y[2:5]).all()
    assert torch.equal(hg.embed(table[:0], ids[1:2]), torch.zeros(1, 40, device="cuda"))
    assert torch.equal(hg.embed(table.t().contiguous().t(), ids[:1]), table[3:4])


def test_offsets_past_32_bits():
    nodes, dim = 2_200_003, 1024  # 2.25e9 elements
    table = torch.zeros(nodes, dim, dtype=BF16, device="cuda")
    table[-3:] = rand(3, dim, dtype=BF16, seed=1)
    ids = torch.tensor([nodes - 1, 5, nodes - 3], device="cuda")
    assert torch.equal(hg.embed(table, ids), table[ids])
    dy = whole(3, dim, seed=2)
    del table
    d = hg.embed_grad(dy.to(BF16), ids, nodes, out_dtype=BF16)
    assert torch.equal(d[ids].float(), dy) and not d[6:-3].any() and not d[-2].any()


@pytest.mark.parametrize("kind", ["words", "any", "one", "up", "down"])
@pytest.mark.parametrize("n", [1, 2, 7, 64, 65, 1000, 1025, 4096, 4097, 20_000, 270_001])
def test_sorts(n, kind):
    """One block's sort and the tiled one, of one to four passes."""
    every = (1, 2, 255, 256, 2047, 2048, 65_535, 1_048_575, 5_000_000)
    for nodes in every if n <= 20_000 else (2047, 65_535, 5_000_000):
        ids = some_ids(n, nodes, kind, seed=n)
        dim = 4 if nodes > 100_000 or n > 4097 else 24
        dy = whole(n, dim, seed=nodes)
        want = sums(dy, ids, nodes)
        assert float(want.abs().max()) < 2 ** 24
        got = hg.embed_grad(dy, ids, nodes)
        assert got.dtype == F32 and torch.equal(got.double(), want), (n, nodes, kind)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("dim", [1, 3, 8, 100, 128, 250, 1000, 1024, 2048, 2056, 5001])
def test_gradient(dim, dtype):
    """Widths that one group of lanes sums and that several do; results in float32 and dy's type."""
    nodes = 300
    for n in (0, 1, 33, 700, 5000):
        ids = some_ids(n, nodes, "words", seed=n)
        dy = rand(n, dim + 5, dtype=dtype, seed=n)[:, 2:dim + 2]
        for out in {F32, dtype}:
            got = hg.embed_grad(dy, ids, nodes, scale=3.3, out_dtype=out)
            assert got.dtype == out
            want = sums(dy, ids, nodes) * 3.3
            size = sums(dy.abs(), ids, nodes) * 3.3
            # a chunk sums up to 64 rows one after another, a run has up to n / 8 + 1 parts, which
            # 8 lanes sum in turns: each sum is off by 2^-24 of what it has so far
            levels = 64 + n / 64 + 16
            R.assert_close(got, want, R.rounding(want, out) + size * levels * 2 ** -24, "dtable")
        into = rand(nodes, dim, seed=9)
        kept = into.clone()
        assert hg.embed_grad(dy, ids, nodes, scale=-0.25, into=into) is into
        want = kept.double() - 0.25 * sums(dy, ids, nodes)
        size = 0.25 * sums(dy.abs(), ids, nodes)
        R.assert_close(into, want, R.rounding(want, F32) + (size * levels + want.abs()) * 2 ** -24,
                       "into")


def test_into_leaves_the_others():
    """Rows that no id names keep their bits, also NaN; a view of a wider table takes it."""
    big = torch.full((50, 40), float("nan"), device="cuda")
    table = big[:, 4:36]
    table[[1, 30]] = 1.0
    ids = torch.tensor([30, 1, 30, -1, 50, 1 << 33], device="cuda")
    dy = whole(6, 32, seed=1)
    version = big._version
    hg.embed_grad(dy, ids, 50, into=table)
    assert big._version > version  # (autograd is told)
    assert torch.equal(table[30], 1 + dy[0] + dy[2]) and torch.equal(table[1], 1 + dy[1])
    rest = torch.ones(50, dtype=torch.bool)
    rest[[1, 30]] = False
    assert torch.isnan(big[rest.cuda()]).all() and torch.isnan(big[:, :4]).all()
    assert torch.isnan(big[:, 36:]).all()
    assert hg.embed_grad(dy[:0], ids[:0], 50, into=table) is table


def test_binding_refuses():
    dy, ids = rand(4, 8), torch.zeros(4, dtype=torch.int64, device="cuda")
    table = rand(10, 8)
    for call in (lambda: hg.embed(table, ids.int()), lambda: hg.embed(table, ids[:, None]),
                 lambda: hg.embed(table, ids.cpu()), lambda: hg.embed(table.double(), ids),
                 lambda: hg.embed(table, ids, out_dtype=torch.int8),
                 lambda: hg.embed_grad(dy, ids[:3], 10), lambda: hg.embed_grad(dy, ids, -1),
                 lambda: hg.embed_grad(dy, ids, 10, out_dtype=BF16),
                 lambda: hg.embed_grad(dy, ids, 9, into=table),
                 lambda: hg.embed_grad(dy, ids, 10, into=table.to(BF16)),
                 lambda: hg.embed_grad(dy, ids, 10, out_dtype=F16, into=table),
                 lambda: hg.embed_grad(dy, ids, 10, into=rand(8, 10).t()),
                 lambda: hg.embed_grad(dy, ids, 10, into=table[:1].expand(10, 8)),
                 lambda: hg.embed_grad(dy, ids, 10, into=table.clone().requires_grad_())):
        with pytest.raises(ValueError):
            call()
    for scale in (float("nan"), float("inf")):
        with pytest.raises(hg.HGError):
            hg.embed(table, ids, scale=scale)
        with pytest.raises(hg.HGError):
            hg.embed_grad(dy, ids, 10, scale=scale)
    leaf = table.clone().requires_grad_()
    with torch.no_grad():  # an optimiser's step
        hg.embed_grad(dy, ids, 10, scale=-1.0, into=leaf)
    assert not torch.equal(leaf, table)


def test_gradient_is_the_forward_passes():
    """<dy, embed(table)> changes with the table as <dtable, table> does: exactly, in whole numbers,
    and one element at a time by differences."""
    nodes, dim, n = 60, 33, 500
    ids = some_ids(n, nodes, "words", seed=2)
    table, dy = whole(nodes, dim, seed=3), whole(n, dim, seed=4)
    d = hg.embed_grad(dy, ids, nodes, scale=2.0)
    value = lambda t: float((dy.double() * hg.embed(t, ids, scale=2.0).double()).sum())  # noqa: E731
    assert value(table) == float((d.double() * table.double()).sum())
    for v, j in ((0, 0), (int(ids.max()), 32), (59, 7)):
        more = table.clone()
        more[v, j] += 1
        assert value(more) - value(table) == float(d[v, j])


def test_nan_stays_in_its_rows():
    dy = whole(200, 16, seed=1)
    ids = some_ids(200, 20, "any", seed=1)
    dy[7, 3] = float("nan")
    dy[11] = float("inf")
    d = hg.embed_grad(dy, ids, 20)
    hit = torch.zeros(20, 16, dtype=torch.bool, device="cuda")
    hit[ids[7], 3] = True
    hit[ids[11]] = True
    assert torch.equal(torch.isfinite(d), ~hit)


def test_repeats_and_streams():
    n, nodes, dim = 30_000, 3000, 256
    ids, dy = some_ids(n, nodes, "words", seed=1), rand(n, dim, dtype=BF16, seed=2)
    first = hg.embed_grad(dy, ids, nodes)
    y = hg.embed(first, ids)
    other = torch.cuda.Stream()
    torch.cuda.synchronize()
    for stream in (None, other):
        again = hg.embed_grad(dy, ids, nodes, stream=stream)
        z = hg.embed(first, ids, stream=stream)
        torch.cuda.synchronize()
        assert torch.equal(first, again) and torch.equal(y, z)


@pytest.mark.parametrize("n", [3000, 9000])
def test_capture(n):
    nodes, dim = 700, 64
    ids, dy = some_ids(n, nodes, "words", seed=1), whole(n, dim, dtype=BF16, seed=2)
    table = torch.zeros(nodes, dim, device="cuda")

    def work():
        return (hg.embed_grad(dy, ids, nodes), hg.embed_grad(dy, ids, nodes, scale=0.5, into=table),
                hg.embed(table, ids, out_dtype=F16))

    work()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = work()
    for seed in (5, 6, 7):
        ids.copy_(some_ids(n, nodes, "words", seed=seed))
        table.zero_()
        want = [t.clone() for t in work()]
        table.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))


@pytest.mark.parametrize("n", [0, 100, 5000])
@pytest.mark.parametrize("dtype,nodes,dim,gap", [(F32, 10_007, 5, 2), (BF16, 20_011, 7, 3),
                                                 (F16, 3001, 9, 1), (F32, 9, 20_001, 5),
                                                 (BF16, 5, 40_003, 11), (F32, 1, 33, 4)])
def test_table_with_gaps(dtype, nodes, dim, gap, n):
    """By the C entry point: a whole table's gradient into rows that do not follow each other.  Every row is
    written, and nothing between them."""
    lib = hg.load_library()
    ids, dy = some_ids(n, nodes, "words", seed=1), whole(n, dim, dtype=dtype, seed=2)
    code = {F32: 1, F16: 2, BF16: 3}[dtype]
    for out, out_code in ((dtype, code), (F32, 1)):
        buffer = torch.full((nodes, dim + gap), float("nan"), dtype=out, device="cuda")
        ws = torch.empty(lib.hg_embed_grad_workspace(n, nodes, dim) + 16, dtype=torch.uint8,
                         device="cuda")
        args = dense.EmbedGradArgs(
            n=n, nodes=nodes, dim=dim, dtype=code, out_dtype=out_code, scale=2.0, dy=dy.data_ptr(),
            dy_stride=dim, ids=ids.data_ptr(), dtable=buffer.data_ptr(), dtable_stride=dim + gap,
            workspace=ws.data_ptr(), workspace_bytes=ws.numel())
        stream = torch.cuda.current_stream().cuda_stream
        assert lib.hg_embed_grad(ctypes.byref(args), stream) == hg.HG_OK
        # (sums of up to 5000 whole numbers up to 8: exact in 32 bits, rounded once)
        assert torch.equal(buffer[:, :dim], (2 * sums(dy, ids, nodes)).float().to(out))
        assert torch.isnan(buffer[:, dim:].float()).all()


def test_table_and_rows_in_one_memory():
    """dy may stand beside the table's rows, not in them (the rows would be read while others are written)."""
    big = whole(60, 48, seed=1)
    ids = some_ids(40, 60, "any", seed=1)
    table = big[:, :16]
    for dy in (table[:40], big[10:50, 8:24], big.view(120, 24)[::3, :16], table[3:4].expand(40, 16)):
        kept = big.clone()
        with pytest.raises(hg.HGError) as e:
            hg.embed_grad(dy, ids[:len(dy)], 60, into=table)
        assert e.value.status == hg.HG_EINVAL and torch.equal(big, kept)
    for dy in (big[:40, 16:32], big[::2, 32:], big[5:6, 20:36].expand(40, 16), big[7:8, 16:32]):
        m = len(dy)
        want = table.double() + sums(dy.clone(), ids[:m], 60)
        hg.embed_grad(dy, ids[:m], 60, into=table)
        assert torch.equal(table.double(), want)
    # above and below the table in one tensor
    rows = whole(100, 16, seed=2)
    want = rows[40:].double() + sums(rows[:40].clone(), ids, 60)
    hg.embed_grad(rows[:40], ids, 60, into=rows[40:])
    assert torch.equal(rows[40:].double(), want)
