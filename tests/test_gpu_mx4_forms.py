"""Forms of the 4-bit, grouped and routing entry points that are easily left out: sums and biases of very different size, gradients of bf16
tensors, layers quantized on the way from bf16 and to codes, the int8 feed-forward of a mixture of experts as a whole."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from oracle import mx4_oracle as MX  # noqa: E402


@pytest.fixture(scope="module")
def q8():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1910_06188_amd import q8 as mod
    return mod


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def host(t):
    return t.float().cpu().numpy().astype(np.float64) if t.is_floating_point() else t.cpu().numpy()


def quantized(q8, x):
    codes, scales = q8.mx4_empty(*x.shape)
    q8.q8_mx4_quantize(x, codes, scales)
    return codes, scales


# Every kernel behind the products (0: the automatic choice); what a variant cannot take goes to the first.
@pytest.fixture(params=range(6), ids=lambda v: f"kernel{v}")
def variant(q8, request):
    q8.set_product_variant(request.param)
    yield request.param
    q8.set_product_variant(0)


def grid_numbers(g, M, K):
    """Numbers of the format itself, blocks at scale 1: their products are multiples of 1 / 4, and sums of up to 2^16 of them exact in fp32."""
    x = (g.choice(MX.GRID, (M, K)) * g.choice([-1.0, 1.0], (M, K))).astype(np.float32)
    x[:, ::32] = 6
    return x


@pytest.mark.parametrize("M", [5, 600])
@pytest.mark.parametrize("K", [256, 4096])
def test_a_bias_larger_than_the_sum_costs_one_rounding(q8, variant, M, K):
    """The sums are exact whatever their order, so the output is their sum with the bias rounded once: a bias in the middle of the reduction would be rounded
    with every step of it."""
    g = np.random.default_rng(M + K)
    N = 260
    x, w = grid_numbers(g, M, K), grid_numbers(g, N, K)
    b = (g.standard_normal(N) * 1e5).astype(np.float32)
    want = (x.astype(np.float64) @ w.astype(np.float64).T).astype(np.float32) + b
    xq, wq = quantized(q8, dev(x)), quantized(q8, dev(w))
    y, dyn = torch.empty((M, N), device="cuda"), torch.empty((M, N), device="cuda")
    q8.q8_mx4_linear(*xq, *wq, dev(b), y)
    np.testing.assert_array_equal(host(y), want)
    q8.q8_mx4_linear_dynamic(dev(x), *wq, dev(b), *q8.mx4_empty(M, K), dyn)
    np.testing.assert_array_equal(host(dyn), want)
    grouped, counts = torch.empty((M, N), device="cuda"), torch.tensor([M // 3, M - M // 3], dtype=torch.int32, device="cuda")
    q8.q8_mx4_linear_grouped(*xq, torch.stack([wq[0]] * 2), torch.stack([wq[1]] * 2), torch.stack([dev(b), -dev(b)]), counts, grouped)
    want[M // 3:] = (x[M // 3:].astype(np.float64) @ w.astype(np.float64).T).astype(np.float32) - b
    np.testing.assert_array_equal(host(grouped), want)


# ---- the gradient of the 4-bit quantizer ---------------------------------------------------------------------------------

@pytest.mark.parametrize("n", [0, 1, 5, 8, 4099, 2_000_001, 40_000_003])
@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("offset", [0, 1])
def test_gradient_of_either_type(q8, n, kind, offset):
    """Every bit of the gradient, NaN among them, wherever the tensors start; nothing around it is written."""
    bits = torch.int32 if kind is torch.float32 else torch.int16
    room = torch.randint(torch.iinfo(bits).min, torch.iinfo(bits).max, (n + offset,), dtype=bits, device="cuda")
    out = torch.full((offset + n + 9,), 7, dtype=bits, device="cuda")
    grad, grad_x = room[offset:].view(kind), out[offset: offset + n].view(kind)
    q8.q8_ste_backward(grad, grad_x)
    assert torch.equal(out[offset: offset + n], room[offset:])
    assert (out[:offset] == 7).all() and (out[offset + n:] == 7).all()
    kept = room.clone()
    q8.q8_ste_backward(grad, grad)                   # in place: nothing to do
    assert torch.equal(room, kept)


@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
def test_a_training_step_through_the_quantizer(q8, kind):
    """loss = sum c xq with xq the codes' values: its gradient by the estimator is c, in the type of x.  Against differences of the straight line that the
    estimator takes the codes' values for: x itself."""
    g = np.random.default_rng(8)
    x, c = dev(g.standard_normal((24, 96)).astype(np.float32)).to(kind), dev(g.standard_normal((24, 96)).astype(np.float32)).to(kind)
    xq, grad_x = torch.empty_like(x), torch.zeros_like(x)
    q8.q8_mx4_fake_quantize(x, xq)
    want_c, want_s = MX.quantize(host(x))
    np.testing.assert_array_equal(host(xq), MX.values(want_c, want_s, 96))
    q8.q8_ste_backward(c, grad_x)
    assert grad_x.dtype is kind and torch.equal(grad_x, c)
    loss = lambda v: float((host(c) * v).sum())  # noqa: E731
    d = np.zeros((24, 96))
    d[3, 40], step = 1, 0.5
    assert abs((loss(host(x) + step * d) - loss(host(x) - step * d)) / (2 * step) - host(grad_x)[3, 40]) <= 1e-9


# ---- outputs too wide for the largest tile ---------------------------------------------------------------------------------

@pytest.mark.parametrize("N", [1 << 21, (1 << 21) + 256 * 200 + 128, 1 << 22])
def test_codes_of_a_very_wide_layer_are_those_of_its_fp32_output(q8, N):
    """256 rows of this width reach past 31 bits of offset: outputs of every type still come from the same sums."""
    M, K, G = 256, 8192, 64
    g = torch.Generator(device="cuda")
    g.manual_seed(N)
    rand = lambda *s, lo=0, hi=256: torch.randint(lo, hi, s, generator=g, device="cuda", dtype=torch.uint8)  # noqa: E731
    xq, wq = (rand(M, 64 * G), rand(G, M, 4, lo=112, hi=130)), (rand(N, 64 * G), rand(G, N, 4, lo=112, hi=130))      # sums that round
    b = torch.randn(N, generator=g, device="cuda")
    y = torch.empty((M, N), device="cuda")
    q8.q8_mx4_linear(*xq, *wq, b, y)
    half = torch.empty((M, N), dtype=torch.bfloat16, device="cuda")
    q8.q8_mx4_linear(*xq, *wq, b, half)
    assert torch.equal(half, y.bfloat16())
    codes, scales = q8.mx4_empty(M, N)
    q8.q8_mx4_linear(*xq, *wq, b, codes, y_scales=scales)
    for n in range(0, N, q8.MX4_MAX_K):              # the quantizer takes rows of up to MX4_MAX_K
        part = y[:, n: n + q8.MX4_MAX_K].contiguous()
        want = quantized(q8, part)
        assert torch.equal(scales[n // 128: n // 128 + len(want[1])], want[1]) and torch.equal(codes[:, n // 2: n // 2 + want[0].shape[1]], want[0])
    # a few outputs against 64 bits
    cols = torch.tensor([0, 1, 4095, N - 129, N - 2, N - 1], device="cuda")
    xv, wv = MX.values(host(xq[0][:40]), host(xq[1][:, :40])), MX.values(host(wq[0][cols]), host(wq[1][:, cols]))
    # K / 64 instructions, eight partial sums and the bias, each off by 2^-23 of the magnitudes summed at most
    err = (K / 64 + 10) * 2.0 ** -23 * (np.abs(xv) @ np.abs(wv).T + np.abs(host(b[cols])))
    assert (np.abs(host(y[:40][:, cols]) - (xv @ wv.T + host(b[cols]))) <= err).all()


def test_fake_quantize_of_as_many_vectors_as_a_launch_has_threads(q8):
    """69 GB of fp32: 2^32 - 8 vectors of 16 bytes, which in workgroups of 64 are 2^32 threads, one more than a launch takes."""
    M, K = 256999, 66848
    assert M * K // 4 == (1 << 32) - 8
    if torch.cuda.mem_get_info()[0] + torch.cuda.memory_reserved() < 80 << 30:
        pytest.skip("needs 69 GB")
    torch.cuda.empty_cache()
    x = torch.zeros((M, K), device="cuda")
    ends = [slice(0, 20), slice(M - 20, M)]
    want = []
    for s in ends:
        x[s] = torch.randn(20, K, device="cuda")
        want.append(MX.values(*MX.quantize(host(x[s])), K))
    q8.q8_mx4_fake_quantize(x, x)
    for s, v in zip(ends, want):
        np.testing.assert_array_equal(host(x[s]), v)
    assert not x[20:2000].any() and not x[M - 2000: M - 20].any()
    del x
    torch.cuda.empty_cache()
