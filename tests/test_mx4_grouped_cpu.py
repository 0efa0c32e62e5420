"""The 4-bit, grouped and routing entry points without a GPU: what they refuse before anything is launched, and their oracle
against the numbers that the format's definition gives by hand."""
import ctypes as C
import os

import numpy as np
import pytest

from oracle import mx4_oracle as MX

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_1910_06188_amd", "libq8.so")
OK, NULL, SHAPE, ALIGN, FLAGS, LAUNCH, LARGE, OVERLAP = range(8)
F32, BF16, MX4, I8 = range(4)


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(LIB):
        from paper_1910_06188_amd import build
        build.build()
    from paper_1910_06188_amd import q8
    return q8.raw()


def at(i):
    """Addresses far apart, never dereferenced."""
    return (i + 1) << 40


def test_oracle_codes_by_hand():
    x = np.zeros((1, 32))
    # amax 6.5 -> s = 0: the code is the nearest of the grid, ties to the even mantissa
    x[0, :16] = [6.5, -5.0, 5.01, 3.5, -2.5, 2.51, 1.75, 1.25, 0.75, 0.25, -0.26, 0.0, -0.0, 6.0, 4.999, -6.49]
    codes, scales = MX.quantize(x)
    v = MX.values(codes, scales, 32)[0]
    assert list(v[:16]) == [6, -4, 6, 4, -2, 3, 2, 1, 1, 0, -0.5, 0, 0, 6, 4, -6]
    assert codes.shape == (1, 64) and scales.shape == (1, 1, 4) and list(scales[0, 0]) == [127, 0, 0, 0]
    assert codes[0, 0] == 7 | (8 + 6) << 4           # the even element in the low half
    x = np.zeros((1, 129), np.float32)
    x[0, 0], x[0, 32], x[0, 64], x[0, 128] = 2.0 ** -149, np.inf, 7.999, 2.0 ** 127
    codes, scales = MX.quantize(x)
    assert list(scales[:, 0].reshape(-1)) == [0, 255, 127, 0, 127 + 125, 0, 0, 0]
    v = MX.values(codes, scales, 129)[0]
    assert v[0] == 0 and np.isnan(v[32:64]).all() and v[64] == 6 and v[128] == 2.0 ** 127


def test_oracle_routing_by_hand():
    inf = np.inf
    logits = np.array([[1, 3, 3, -inf], [-inf, -inf, -inf, -inf], [np.nan, 2, inf, inf]], np.float32)
    experts, gates, group_rows, rows, slots = MX.route(logits, 2)
    assert experts.tolist() == [[1, 2], [0, 1], [2, 3]]
    assert gates.tolist() == [[0.5, 0.5], [0, 0], [0.5, 0.5]]
    assert group_rows.tolist() == [1, 2, 2, 1] and rows.tolist() == [1, 0, 1, 0, 2, 2] and slots.tolist() == [[1, 3], [0, 2], [4, 5]]


def test_quantizers_refuse(lib):
    q, f = lib.q8_mx4_quantize, lib.q8_mx4_fake_quantize
    x, c, s = at(0), at(1), at(2)
    assert q(x, F32, -1, 8, c, s, None) == SHAPE and q(x, F32, 1, -8, c, s, None) == SHAPE
    assert q(x, F32, 1, 1048577, c, s, None) == SHAPE and q(x, F32, 1 << 31, 1, c, s, None) == SHAPE
    assert q(x, F32, 1 << 24, 1 << 20, c, s, None) == SHAPE           # more than a launch takes
    assert q(x, MX4, 1, 8, c, s, None) == FLAGS and q(x, -1, 1, 8, c, s, None) == FLAGS
    assert q(None, F32, 1, 8, c, s, None) == NULL and q(x, F32, 1, 8, None, s, None) == NULL and q(x, F32, 1, 8, c, None, None) == NULL
    assert q(x + 2, F32, 1, 8, c, s, None) == ALIGN and q(x + 1, BF16, 1, 8, c, s, None) == ALIGN
    assert q(x, F32, 1, 8, c + 8, s, None) == ALIGN and q(x, F32, 1, 8, c, s + 2, None) == ALIGN
    assert q(x, F32, 4, 128, x + 64, s, None) == OVERLAP and q(x, F32, 4, 128, c, c + 4 * 64 - 4, None) == OVERLAP
    assert q(None, F32, 0, 8, None, None, None) == OK and q(None, F32, 8, 0, None, None, None) == OK
    assert f(x, I8, 1, 8, c, None) == FLAGS and f(x, F32, 1, 8, None, None) == NULL and f(x, BF16, 1, 8, c + 1, None) == ALIGN
    assert f(x, F32, 2, 8, x + 4, None) == OVERLAP and f(None, BF16, 0, 8, None, None) == OK and f(x, F32, -1, 8, x, None) == SHAPE


def test_products_refuse(lib):
    x, xs, w, ws, b, g, r, y, ys = (at(i) for i in range(9))

    def linear(M=4, N=128, K=128, x=x, xs=xs, w=w, ws=ws, b=b, y=y, t=F32, ys=None, flags=0):
        return lib.q8_mx4_linear(x, xs, w, ws, b, M, N, K, y, t, ys, flags, None)

    def grouped(M=4, N=128, K=128, n=4, E=2, x=x, xs=xs, rows=None, w=w, ws=ws, b=b, g=g, y=y, t=F32, ys=None, flags=0):
        return lib.q8_mx4_linear_grouped(x, xs, n, rows, w, ws, b, g, E, M, N, K, y, t, ys, flags, None)

    for f in (linear, grouped):
        for bad in ({"M": -1}, {"N": -1}, {"K": -1}, {"K": 1048577}, {"M": 1 << 31}, {"N": 1 << 31}, {"M": 1 << 20, "N": 1 << 20},
                    {"N": 130, "t": MX4, "ys": ys}):
            assert f(**bad) == SHAPE, bad
        for bad in ({"flags": 2}, {"flags": 4}, {"flags": 8}, {"t": I8}, {"t": 9}):
            assert f(**bad) == FLAGS, bad
        for bad in ({"x": None}, {"xs": None}, {"w": None}, {"ws": None}, {"y": None}, {"t": MX4}):
            assert f(**bad) == NULL, bad
        for bad in ({"x": x + 8}, {"w": w + 4}, {"xs": xs + 2}, {"ws": ws + 1}, {"b": b + 2}, {"y": y + 2}, {"y": y + 1, "t": BF16}, {"y": y + 8, "t": MX4, "ys": ys},
                    {"ys": ys + 2, "t": MX4}):
            assert f(**bad) == ALIGN, bad
        for bad in ({"y": x}, {"y": w + 64}, {"y": xs}, {"y": ws}, {"y": b}, {"t": MX4, "ys": x}, {"t": MX4, "ys": y + 64}):
            assert f(**bad) == OVERLAP, bad
        assert f(M=0, x=None, xs=None, w=None, ws=None, y=None) == OK and f(N=0) == OK
    assert linear(M=1 << 29, N=32) == SHAPE and grouped(M=1 << 14, n=1 << 14, N=1 << 19, E=1024) == SHAPE      # more tiles than a launch takes
    for bad in ({"E": 0}, {"E": 1025}, {"n": 3}, {"n": 0, "rows": r}, {"n": -1}, {"n": 1 << 31, "rows": r}):
        assert grouped(**bad) == SHAPE, bad
    assert grouped(g=None) == NULL
    assert grouped(g=g + 2) == ALIGN and grouped(rows=r + 2) == ALIGN
    assert grouped(y=g) == OVERLAP and grouped(rows=r, y=r) == OVERLAP

    def dynamic(M=4, N=128, K=100, x=x, t=F32, cw=at(20), sw=at(21), y=y, yt=F32):
        return lib.q8_mx4_linear_dynamic(x, t, w, ws, b, M, N, K, cw, sw, y, yt, None, 0, None)

    assert dynamic(t=MX4) == FLAGS and dynamic(x=None) == NULL and dynamic(cw=None) == NULL and dynamic(sw=None) == NULL
    assert dynamic(x=x + 1) == ALIGN and dynamic(cw=at(20) + 8) == ALIGN and dynamic(M=-1) == SHAPE and dynamic(K=-1) == SHAPE
    assert dynamic(y=x) == OVERLAP and dynamic(cw=x) == OVERLAP and dynamic(cw=w) == OVERLAP and dynamic(sw=ws) == OVERLAP and dynamic(cw=y) == OVERLAP
    assert dynamic(M=0) == OK


def test_int8_grouped_refuses(lib):
    x, w, b, sx, sw, g, r, y, a, ns = (at(i) for i in range(10))

    def f(M=4, N=8, K=16, n=4, E=2, x=x, rows=None, w=w, b=b, sx=sx, sw=sw, g=g, y=y, a=None, ns=None, flags=0):
        return lib.q8_linear_grouped(x, n, rows, w, b, sx, sw, g, E, M, N, K, y, a, ns, flags, None)

    for bad in ({"M": -1}, {"N": -1}, {"K": -1}, {"K": 131072}, {"E": 0}, {"n": 5}, {"n": 0, "rows": r}, {"M": 1 << 31}, {"E": 1025}):
        assert f(**bad) == SHAPE, bad
    for bad in ({"flags": 8}, {"flags": 2}, {"flags": 4}):
        assert f(**bad) == FLAGS, bad
    for bad in ({"x": None}, {"w": None}, {"sx": None}, {"sw": None}, {"g": None}, {"y": None}):
        assert f(**bad) == NULL, bad
    for bad in ({"y": y + 2}, {"b": b + 1}, {"sx": sx + 2}, {"sw": sw + 2}, {"g": g + 1}, {"rows": r + 2}, {"flags": 2, "a": a + 2}, {"flags": 4, "ns": ns + 2}):
        assert f(**bad) == ALIGN, bad
    for bad in ({"y": x}, {"y": w}, {"y": b}, {"y": sx}, {"y": sw}, {"y": g}, {"flags": 2, "a": y}, {"flags": 4, "ns": y}):
        assert f(**bad) == OVERLAP, bad
    assert f(M=0) == OK and f(N=0) == OK


def test_router_and_combine_refuse(lib):
    l, e, g, n, r, s, w = (at(i) for i in range(7))

    def route(T=4, E=8, k=2, l=l, e=e, g=g, n=n, r=r, s=s, w=w):
        return lib.q8_route(l, T, E, k, e, g, n, r, s, w, None)

    for bad in ({"T": -1}, {"E": 0}, {"E": 1025}, {"k": 0}, {"k": 9}, {"E": 64, "k": 17}, {"T": 1 << 30}):
        assert route(**bad) == SHAPE, bad
    for bad in ({"l": None}, {"e": None}, {"g": None}, {"n": None}, {"r": None}, {"s": None}, {"w": None}):
        assert route(**bad) == NULL, bad
    for bad in ({"l": l + 1}, {"e": e + 2}, {"g": g + 2}, {"n": n + 2}, {"r": r + 2}, {"s": s + 2}, {"w": w + 2}):
        assert route(**bad) == ALIGN, bad
    for bad in ({"r": s}, {"e": l}, {"n": w + 4}, {"g": e + 28}):
        assert route(**bad) == OVERLAP, bad

    y, o = at(8), at(9)

    def combine(T=4, k=2, N=8, R=8, y=y, s=s, g=g, o=o, t=F32):
        return lib.q8_combine(y, R, s, g, T, k, N, o, t, None)

    for bad in ({"T": -1}, {"k": 0}, {"N": -1}, {"R": -1}, {"T": 1 << 30, "k": 4}, {"R": 1 << 31}):
        assert combine(**bad) == SHAPE, bad
    assert combine(t=MX4) == FLAGS and combine(t=I8) == FLAGS
    for bad in ({"y": None}, {"s": None}, {"g": None}, {"o": None}):
        assert combine(**bad) == NULL, bad
    assert combine(y=y + 2) == ALIGN and combine(o=o + 1, t=BF16) == ALIGN and combine(s=s + 1) == ALIGN
    assert combine(o=y + 4) == OVERLAP and combine(o=s) == OVERLAP
    assert combine(T=0) == OK and combine(N=0) == OK


def test_python_refuses_what_does_not_fit():
    import torch
    from paper_1910_06188_amd import q8

    def mx(*shape):
        return q8.mx4_empty(*shape, device="cpu")

    x = torch.zeros(4, 100)
    with pytest.raises(ValueError):
        q8.q8_mx4_quantize(x, *mx(4, 300))
    with pytest.raises(ValueError):
        q8.q8_mx4_quantize(x, mx(4, 100)[0], mx(5, 100)[1])
    with pytest.raises(TypeError):
        q8.q8_mx4_quantize(x.half(), *mx(4, 100))
    with pytest.raises(ValueError):
        q8.q8_mx4_fake_quantize(x, x.bfloat16())
    y = torch.zeros(4, 128)
    with pytest.raises(ValueError):
        q8.q8_mx4_linear(*mx(4, 100), *mx(128, 200), None, y)
    with pytest.raises(ValueError):
        q8.q8_mx4_linear(*mx(4, 100), *mx(128, 100), torch.zeros(64), y)
    with pytest.raises(TypeError):
        q8.q8_mx4_linear(*mx(4, 100), *mx(128, 100), None, y.half())
    with pytest.raises(TypeError):
        q8.q8_mx4_linear(*mx(4, 100), *mx(128, 100), None, y, y_scales=mx(4, 128)[1])
    with pytest.raises(ValueError):
        q8.q8_mx4_linear(*mx(4, 100), *mx(100, 100), None, mx(4, 100)[0], y_scales=mx(4, 100)[1])      # codes of 100 columns
    with pytest.raises(ValueError):
        q8.q8_mx4_linear_dynamic(x, *mx(128, 100), None, *mx(3, 100), y)
    n = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError):
        q8.q8_mx4_linear_grouped(*mx(4, 100), *mx(3, 128, 100), None, n, y)
    with pytest.raises(ValueError):
        q8.q8_mx4_linear_grouped(*mx(5, 100), *mx(2, 128, 100), None, n, y)                            # five rows and no x_rows for four
    i8 = torch.zeros(4, 16, dtype=torch.int8)
    with pytest.raises(ValueError):
        q8.q8_linear_grouped(i8, torch.zeros(2, 128, 16, dtype=torch.int8), None, torch.ones(1), torch.ones(2), n, y.to(torch.int8))
    # the binding looks at devices (and on a GPU at element types)
    with pytest.raises(ValueError, match="device tensors"):
        q8.q8_mx4_quantize(x, *mx(4, 100))
    with pytest.raises(ValueError, match="device tensors"):
        q8.q8_mx4_linear_grouped(*mx(4, 100), *mx(2, 128, 100), None, n, y)
