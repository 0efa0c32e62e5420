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
