"""distill against its definition in 64 bits: every way a row is held (by its length), types, lists
of all lengths, masked and repeated entries, rows left out, values that are not finite."""
import ctypes
import math

import pytest
import torch

import dense_ref as R
import paper_2112_15345_amd as hg
from paper_2112_15345_amd import dense

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
# below, at and past the lengths where a row is held by a wavefront, by blocks, or read twice
CLASSES = [1, 2, 17, 64, 153, 256, 500, 512, 1000, 2048, 2049, 4100, 8192, 10_007, 16_384, 32_768,
           40_001, 65_536, 65_600, 131_072, 140_001]


def rand(*shape, dtype=F32, seed=0, scale=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def lists(rows, classes, top, seed=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randint(classes, (rows, top), generator=g, device="cuda")


def check(logits, ids, teacher, T, a, got):
    loss, grad = got
    want, wgrad, size, p, q = R.distill(logits, ids, teacher, T, a)
    n = logits.shape[1]
    # log q: the sum of n positive terms; the arguments z / T are rounded once
    spread = (logits.double().amax(1) - logits.double().amin(1)).abs() / T
    spread = torch.nan_to_num(spread, nan=0.0, posinf=1e4)
    rel = (2 * n + 64) * R.E
    if loss is not None:
        assert loss.dtype == F32
        # an exponent off by 2^-23 of its size, over entries of up to `spread`
        far = torch.nan_to_num(size, nan=0.0, posinf=0.0) * 16 * R.E + rel + 4 * R.E * (spread + 1)
        R.assert_close(loss, want, far * 2, "loss")
    if grad is not None:
        assert grad.dtype == logits.dtype
        f = (torch.ones_like(want) if a is None else a.double().abs()) / T
        tops = torch.zeros_like(wgrad).scatter_add_(
            1, ids.clamp(0, n - 1), torch.nan_to_num(p)) if ids.shape[1] else 0
        teach = torch.nan_to_num(teacher.double(), neginf=0.0, posinf=0.0).abs().amax(1) / T \
            if ids.shape[1] else torch.zeros_like(want)
        err = torch.nan_to_num(q) * (rel + 4 * R.E * (spread + 1))[:, None] \
            + tops * ((2 * ids.shape[1] + 64) * R.E + 8 * R.E * teach[:, None])
        # (values below 2^-126 may be flushed)
        R.assert_close(grad, wgrad, R.rounding(wgrad, logits.dtype) + 2 * err * f[:, None] + 2.0 ** -125,
                       "grad")


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("classes", CLASSES)
def test_loss_and_gradient(classes, dtype):
    for rows, top, T in ((1, 1, 1.0), (5, 7, 2.0), (9, 64, 0.5), (3, 300, 1.5)):
        z = rand(rows, classes, dtype=dtype, seed=classes, scale=3.0)
        ids = lists(rows, classes, top, seed=1)      # (short rows: classes repeat)
        t = rand(rows, top, dtype=[F32, F16, BF16][top % 3], seed=2, scale=2.0)
        a = None if top == 7 else rand(rows, seed=3)
        both = hg.distill(z, ids, t, temperature=T, row_weight=a, want_grad=True)
        check(z, ids, t, T, a, both)
        loss, none = hg.distill(z, ids, t, temperature=T, row_weight=a)
        assert none is None
        check(z, ids, t, T, a, (loss, None))
        none, grad = hg.distill(z, ids, t, temperature=T, row_weight=a, want_loss=False,
                                want_grad=True)
        assert none is None and torch.equal(grad, both[1])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("classes", [40, 1500, 9000, 140_000])
def test_masks(classes, dtype):
    """Left-out entries, empty lists, weight 0, repeated classes, out-of-range ids, -inf logits."""
    rows, top = 12, 6
    z = rand(rows, classes, dtype=dtype, seed=1)
    ids = lists(rows, classes, top, seed=2)
    t = rand(rows, top, seed=3)
    a = 0.5 + rand(rows, seed=4).abs()
    ids[0, 3:] = -1                      # a short list
    ids[1] = -1                          # none
    t[2] = -math.inf                     # none, by the teacher's masks
    t[3, ::2] = -math.inf
    ids[4] = 5                           # one class, listed throughout
    a[5] = 0                             # a row without part in the loss
    ids[6, 2] = classes                  # out of range
    ids[7, 2] = -2
    z[8, 10:] = -math.inf                # masked classes, none of them listed
    ids[8] = torch.arange(top, device="cuda")
    z[9, ids[9, 0]] = -math.inf          # a listed class of probability 0
    t[9, 0] = 1.0
    ids[10, 0], t[10, 0] = -1, math.nan  # a left-out entry may hold anything
    z[11] = torch.finfo(dtype).min       # masks of the type's lowest value: all classes alike
    t = t.contiguous()
    got = hg.distill(z, ids, t, temperature=2.0, row_weight=a, want_grad=True)
    check(z, ids, t.masked_fill(ids == -1, 0.0), 2.0, a, got)
    assert got[0][1] == 0 and got[0][2] == 0 and not got[1][1].any() and not got[1][2].any()
    assert not got[1][5].any() and float(got[0][5]) != 0
    assert torch.isnan(got[0][[6, 7]]).all() and torch.isnan(got[1][[6, 7]]).all()
    assert got[0][9] == math.inf
    # an empty list keeps nothing of its logits, whatever they are
    z[1] = math.nan
    z[5] = math.nan
    loss, grad = hg.distill(z, ids, t, temperature=2.0, row_weight=a, want_grad=True)
    assert loss[1] == 0 and not grad[1].any() and not grad[5].any() and torch.isnan(loss[5])
    only = hg.distill(z, ids, t, temperature=2.0, row_weight=a, want_loss=False, want_grad=True)[1]
    assert not only[5].any()


@pytest.mark.parametrize("classes", [40, 1500, 9000, 140_000])
def test_values_that_are_not_finite(classes):
    z, ids, t = rand(6, classes, seed=1), lists(6, classes, 4, seed=2), rand(6, 4, seed=3)
    want = hg.distill(z, ids, t, want_grad=True)
    z[0, classes // 3] = math.nan
    z[1, classes - 1] = math.inf
    z[2] = -math.inf
    t[3, 1] = math.nan
    t[4, 2] = math.inf
    loss, grad = hg.distill(z, ids, t, want_grad=True)
    assert torch.isnan(loss[:5]).all() and torch.isnan(grad[:5]).all()
    assert torch.equal(loss[5], want[0][5]) and torch.equal(grad[5], want[1][5])
    assert torch.isnan(hg.distill(z, ids, t)[0][:5]).all()


def test_large_logits_and_temperatures():
    for dtype, T in ((F32, 1e-3), (F32, 1e4), (F16, 0.1), (BF16, 64.0)):
        z = rand(4, 3000, dtype=dtype, seed=1, scale=50.0)
        ids, t = lists(4, 3000, 8, seed=2), rand(4, 8, seed=3)
        loss, grad = hg.distill(z, ids, t, temperature=T, want_grad=True)
        want = R.distill(z, ids, t, T, None)
        # exponents of up to 4e5 are rounded to 2^-24 of their size
        assert torch.isfinite(loss).all()
        assert (loss.double() - want[0]).abs().max() <= 1e-6 * float(want[0].abs().max()) + 1e-5
        assert torch.isfinite(grad.float()).all()


def test_empty_lists_and_rows():
    z = rand(3, 100, seed=1)
    ids, t = torch.empty(3, 0, dtype=torch.int64, device="cuda"), torch.empty(3, 0, device="cuda")
    loss, grad = hg.distill(z, ids, t, want_grad=True)
    assert not loss.any() and not grad.any()
    loss, grad = hg.distill(z[:0], ids[:0], t[:0], want_grad=True)
    assert loss.shape == (0,) and grad.shape == (0, 100)


def test_longest_list():
    rows, classes, top = 4, 5000, hg.HG_MAX_TOP
    for n in (200, classes):
        z, ids, t = rand(rows, n, seed=1), lists(rows, n, top, seed=2), rand(rows, top, seed=3)
        check(z, ids, t, 1.0, None, hg.distill(z, ids, t, want_grad=True))
    with pytest.raises(hg.HGError):
        hg.distill(z, lists(rows, 200, top + 1), rand(rows, top + 1))


def test_gradient_by_differences():
    z, ids, t = rand(3, 30, seed=1), lists(3, 30, 4, seed=2), rand(3, 4, seed=3)
    a, T, step = rand(3, seed=4), 1.7, 1e-5
    _, grad = hg.distill(z, ids, t, temperature=T, row_weight=a, want_grad=True)

    def value(z64):
        return (R.distill(z64, ids, t, T, a)[0] * a.double()).sum()

    for i in range(3):
        for v in {0, 29, int(ids[i, 0]), int(ids[i, 3])}:
            d = torch.zeros(3, 30, dtype=torch.float64, device="cuda")
            d[i, v] = step
            num = float((value(z.double() + d) - value(z.double() - d)) / (2 * step))
            assert abs(num - float(grad[i, v])) <= 1e-6 * (1 + abs(num))


@pytest.mark.parametrize("classes", [77, 5001, 70_001])
def test_strides_and_in_place(classes):
    big = rand(9, classes + 7, dtype=BF16, seed=1)
    z = big[1::2, 3:3 + classes]
    ids = lists(4, 20, 5, seed=2)[:, ::2]
    ids = ids % classes
    t = rand(4, 11, seed=3)[:, 1:4]
    want = hg.distill(z.contiguous(), ids, t.contiguous(), want_grad=True)
    got = hg.distill(z, ids, t, want_grad=True)
    assert torch.equal(got[1], want[1]) and torch.equal(got[0], want[0])
    check(z, ids, t, 1.0, None, got)
    # the gradient over the logits, as the C entry allows
    own, loss = z.contiguous(), torch.empty(4, device="cuda")
    i, tt = ids.contiguous(), t.contiguous()
    a = dense.DistillArgs(4, classes, 3, dense.HG_DT_BF16, dense.HG_DT_F32, 1.0, own.data_ptr(),
                          classes, i.data_ptr(), 3, tt.data_ptr(), 3, None, loss.data_ptr(),
                          own.data_ptr(), classes)
    assert hg.load_library().hg_distill(ctypes.byref(a), ctypes.c_void_p(
        torch.cuda.current_stream().cuda_stream)) == hg.HG_OK
    assert torch.equal(own, want[1]) and torch.equal(loss, want[0])


def test_offsets_past_32_bits():
    rows, classes = 17_000, 131_072
    z = torch.zeros(rows, classes, dtype=BF16, device="cuda")
    tail = rand(3, classes, dtype=BF16, seed=1)
    z[-3:] = tail
    ids, t = lists(rows, classes, 4, seed=2), rand(rows, 4, seed=3)
    loss, grad = hg.distill(z, ids, t, want_grad=True)
    want = hg.distill(tail, ids[-3:], t[-3:], want_grad=True)
    assert torch.equal(loss[-3:], want[0]) and torch.equal(grad[-3:], want[1])


def test_other_stream_and_capture():
    z, ids, t = rand(50, 700, dtype=BF16, seed=1), lists(50, 700, 9, seed=2), rand(50, 9, seed=3)
    want = hg.distill(z, ids, t, want_grad=True)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = hg.distill(z, ids, t, want_grad=True, stream=s)
    s.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = hg.distill(z, ids, t, want_grad=True)
    for seed in (5, 6, 7):
        z.copy_(rand(50, 700, dtype=BF16, seed=seed))
        graph.replay()
        want = hg.distill(z, ids, t, want_grad=True)
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_binding_refuses():
    z, ids, t = rand(4, 10), lists(4, 10, 3), rand(4, 3)
    for kw in (dict(logits=z[0], ids=ids, teacher=t), dict(logits=z, ids=ids.int(), teacher=t),
               dict(logits=z, ids=ids, teacher=t[:, :2]), dict(logits=z, ids=ids[:3], teacher=t),
               dict(logits=z, ids=ids, teacher=t, row_weight=rand(3)),
               dict(logits=z, ids=ids, teacher=t.cpu()), dict(logits=z.long(), ids=ids, teacher=t)):
        with pytest.raises(ValueError):
            hg.distill(**kw)
    with pytest.raises(hg.HGError):
        hg.distill(z, ids, t, temperature=0.0)
