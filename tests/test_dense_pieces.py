"""What the bounds of the float32 products tell apart, on the CPU: elements as three 16-bit pieces, six
of their nine products, with and without the third pieces."""
import numpy as np

E = 2.0 ** -24


def pieces(x):
    """h (to nearest), m and l (cut) of float32 values, each of 8 bits."""
    u = x.view(np.uint32)
    h = ((u + np.uint32(0x8000)) & np.uint32(0xffff0000)).view(np.float32)
    r = x - h
    m = (r.view(np.uint32) & np.uint32(0xffff0000)).view(np.float32)
    l = ((r - m).view(np.uint32) & np.uint32(0xffff0000)).view(np.float32)
    return [p.astype(np.float64) for p in (h, m, l)]


def test_third_pieces_show_at_short_depths():
    rng = np.random.default_rng(1)
    k = 8
    x, w = (rng.standard_normal((n, k)).astype(np.float32) for n in (2000, 300))
    exact = x.astype(np.float64) @ w.astype(np.float64).T
    bound = (np.abs(x).astype(np.float64) @ np.abs(w).astype(np.float64).T) * ((2 * k + 8) * E)
    (h, m, l), (g, p, q) = pieces(x), pieces(w)
    assert np.array_equal((h + m + l).astype(np.float32), x)
    two = h @ g.T + h @ p.T + m @ g.T + m @ p.T
    six = two + l @ g.T + h @ q.T
    assert (np.abs(six - exact) <= bound / 8).all()
    assert (np.abs(two - exact) > bound).mean() > 0.1
