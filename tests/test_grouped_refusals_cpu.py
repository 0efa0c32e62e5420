"""What the 4-bit, grouped and routing entry points refuse before anything is launched, for calls that share memory, mix types or name sizes
beyond any tensor."""
import os

import pytest

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


def test_gradients_of_other_types_are_refused():
    import torch
    from paper_1910_06188_amd import q8
    f, b, h = torch.zeros(8), torch.zeros(8, dtype=torch.bfloat16), torch.zeros(8, dtype=torch.float16)
    for grad, out in ((f, b), (b, f), (h, h), (f, h), (f.double(), f.double()), (f.int(), f.int())):
        with pytest.raises(TypeError):
            q8.q8_ste_backward(grad, out)
    for grad, out in ((b, b[:4]), (f, f[:4])):
        with pytest.raises(ValueError):
            q8.q8_ste_backward(grad, out)
    for grad in (f, b):
        with pytest.raises(ValueError, match="device tensors"):
            q8.q8_ste_backward(grad, grad.clone())


def test_gradient_of_either_type_refuses(lib):
    f, p, q = lib.q8_mx4_ste_backward, at(0), at(1)
    assert f(p, F32, -1, q, None) == SHAPE and f(p, MX4, 8, q, None) == FLAGS and f(p, I8, 8, q, None) == FLAGS
    assert f(None, BF16, 8, q, None) == NULL and f(p, BF16, 8, None, None) == NULL
    assert f(p + 2, F32, 8, q, None) == ALIGN and f(p, BF16, 8, q + 1, None) == ALIGN
    assert f(p, BF16, 8, p + 14, None) == OVERLAP and f(p + 28, F32, 8, p, None) == OVERLAP
    assert f(None, BF16, 0, None, None) == OK and f(p, BF16, 8, p, None) == OK          # in place: nothing to do


@pytest.mark.parametrize("N", [(1 << 40) + 1, 1 << 60, 1 << 61, 1 << 62, (1 << 63) - 1])
def test_combine_refuses_rows_beyond_any_tensor(lib, N):
    for T, R, t in ((4, 0, F32), (4, 0, BF16), (1, 1, F32)):
        assert lib.q8_combine(at(0), R, at(1), at(2), T, 2, N, at(3), t, None) == SHAPE


def test_int8_grouped_refuses_an_absmax_that_is_read(lib):
    """The abs-max is raised while other workgroups still read the call's inputs."""
    x, w, b, sx, sw, g, r, y, a, ns = (at(i) for i in range(10))
    absmax, requant = 2, 4

    def f(a, rows=None, ns=None, flags=absmax):
        return lib.q8_linear_grouped(x, 4, rows, w, b, sx, sw, g, 2, 4, 8, 16, y, a, ns, flags, None)

    for bad in (x + 60, w + 4, b + 4 * 15, sx, sw + 4, g + 4):
        assert f(bad) == OVERLAP, hex(bad)
    assert f(r + 12, rows=r) == OVERLAP
    assert f(ns, ns=ns, flags=absmax | requant) == OVERLAP
    assert f(y + 4 * 31) == OVERLAP


def test_native_entry_points_refuse_what_is_no_stream_before_all_else():
    import torch
    from paper_1910_06188_amd import _binding, q8
    x = torch.zeros(4, 128)
    c, s = q8.mx4_empty(4, 128, device="cpu")
    n = torch.zeros(4, dtype=torch.int32)
    calls = {
        "q8_mx4_quantize": (x, c, s), "q8_mx4_fake_quantize": (x, x.clone()), "q8_mx4_ste_backward": (x, x.clone()), "q8_mx4_linear": (c, s, c, s, None, x, None, 0),
        "q8_mx4_linear_dynamic": (x, c, s, None, c, s, x, None, 0), "q8_mx4_linear_grouped": (c, s, c[None], s[None], None, n[:1], x, None, None, 0),
        "q8_linear_grouped": (x.char(), x.char()[None], None, x, x[0, :1], n[:1], x[:, :4], None, None, None, 0), "q8_route": (x, n.view(4, 1), x[:, :1], n, n, n, n),
        "q8_combine": (x, n.view(4, 1), x[:, :1], x),
    }
    for name, args in calls.items():
        f = getattr(_binding, name)
        for bad in ("stream", 1.5, x):
            with pytest.raises(TypeError):
                f(*args, bad)
        with pytest.raises(TypeError, match="arguments"):
            f(*args)
        with pytest.raises(ValueError):
            f(*args, 0)


def test_the_gelu_polynomial_is_written_once():
    """The constants that test_host_logic.py checks are the ones of every kernel."""
    csrc = os.path.join(ROOT, "paper_1910_06188_amd", "csrc")
    text = "".join(open(os.path.join(csrc, f)).read() for f in sorted(os.listdir(csrc)))
    for constant in ("3.309277963e-05f", "9.999930859e-01f"):
        assert text.count(constant) == 1


def test_fp32_entry_points_refuse_shorter_floats():
    """bf16 activations belong to the 4-bit entry points; those of fp32 would read twice as many bytes as such a tensor has."""
    import torch
    from paper_1910_06188_amd import q8
    f, one, work, q = torch.zeros(64), torch.zeros(1), torch.zeros(q8.SCAL_WORK), torch.zeros(64, dtype=torch.int8)
    for kind in (torch.bfloat16, torch.float16):
        x = torch.zeros(64, dtype=kind)
        for call in (lambda: q8.q8_absmax(x, one), lambda: q8.q8_quantize(x, one, q), lambda: q8.q8_quantize_dynamic(x, q, work), lambda: q8.q8_fake_quantize(x, one, f),
                     lambda: q8.q8_fake_quantize_ema(x, 0.9, f, work, f), lambda: q8.q8_ste_backward(x, f)):
            with pytest.raises(TypeError):
                call()
