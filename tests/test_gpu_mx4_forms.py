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


# ---- layers quantized on the way ---------------------------------------------------------------------------------------------

def gelu_and_tolerance(ref, mag, K, gelu):
    """Of fp32 outputs: K / 64 matrix instructions, eight partial sums and a bias, each off by 2^-23 of the magnitudes summed at most (an instruction may
    truncate); GELU's slope is at most 1.13, its own error 5.2e-7 and a rounding."""
    err = (K / 64 + 10) * 2.0 ** -23 * mag
    return (MX.gelu(ref), 1.13 * err + 5.2e-7 + 2.0 ** -23 * np.abs(ref)) if gelu else (ref, err)


def activations(g, M, K):
    return (g.standard_normal((M, K)) * np.exp(0.5 * g.standard_normal((M, 1))) * np.exp(g.standard_normal((1, K)))).astype(np.float32)


# One launch up to min(M, 32) K = 24576, K = 4096 and 512 tiles of 32 x 32; both sides of each, and odd sizes.
DYNAMIC = [(1, 1024, 4096), (1, 1, 1), (3, 333, 256), (2, 33, 129), (7, 129, 70), (16, 768, 768), (24, 1024, 256), (25, 1024, 256), (31, 127, 33), (32, 768, 130), (33, 768, 130), (32, 769, 128),
           (5, 4096, 128), (5, 4097, 128), (6, 4096, 96), (32, 768, 16384), (32, 768, 16385), (512, 512, 1024), (513, 512, 1024), (300, 100, 384)]


@pytest.mark.parametrize("M,K,N", DYNAMIC)
@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("gelu", [False, True])
@pytest.mark.parametrize("offset", [0, 1])
def test_dynamic_layer_of_either_type(q8, M, K, N, kind, gelu, offset):
    g = np.random.default_rng(M + K + N)
    room = torch.zeros(offset + M * K, dtype=kind, device="cuda")
    x = room[offset:].view(M, K)
    x.copy_(dev(activations(g, M, K)).to(kind))
    wq, b = quantized(q8, dev(activations(g, N, K))), dev(g.standard_normal(N).astype(np.float32))
    flags = q8.EPI_GELU if gelu else 0
    work = q8.mx4_empty(M, K)
    work[0].fill_(0xFF), work[1].fill_(0xFF)

    def layer(y, y_scales=None, bias=b):
        q8.q8_mx4_linear_dynamic(x, *wq, bias, *work, y, y_scales=y_scales, flags=flags)
        return y

    y = layer(torch.full((M, N), 7.0, device="cuda"))
    xv, wv = MX.values(*MX.quantize(host(x)), K), MX.values(host(wq[0]), host(wq[1]), K)
    ref, err = gelu_and_tolerance(*MX.grouped(xv, [wv], [host(b)], [M], M), K, gelu)
    assert (np.abs(host(y) - ref) <= err).all()
    assert torch.equal(layer(torch.full((M, N), 7.0, dtype=torch.bfloat16, device="cuda")), y.bfloat16())       # one rounding of the same sums
    bare = layer(torch.full((M, N), 7.0, device="cuda"), bias=None)
    ref, err = gelu_and_tolerance(*MX.grouped(xv, [wv], None, [M], M), K, gelu)
    assert (np.abs(host(bare) - ref) <= err).all()
    if N % 128 == 0:
        want, (codes, scales) = quantized(q8, y), q8.mx4_empty(M, N)
        codes.fill_(0xA5), scales.fill_(0x5A)
        layer(codes, scales)
        assert torch.equal(scales, want[1]) and torch.equal(codes, want[0])


@pytest.mark.parametrize("M,K", [(5, 300), (6, 4096), (24, 1024), (200, 1024)])
@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("gelu", [False, True])
def test_dynamic_layer_follows_nan_and_infinity(q8, M, K, kind, gelu):
    """A block of x with an infinity or a NaN makes its row NaN, one of w its column; nothing else changes."""
    g = np.random.default_rng(M + K)
    N = 256
    x, w = activations(g, M, K), activations(g, N, K)
    b = g.standard_normal(N).astype(np.float32)
    x[1, 40], x[3, K - 1], x[4, 0] = np.nan, np.inf, -np.inf
    x[2] = 0                                          # a row of zeros gives the bias
    w[7, 0], w[130, K - 1] = -np.inf, np.nan
    x, wq = dev(x).to(kind), quantized(q8, dev(w))
    flags = q8.EPI_GELU if gelu else 0
    y = torch.full((M, N), 7.0, device="cuda")
    q8.q8_mx4_linear_dynamic(x, *wq, dev(b), *q8.mx4_empty(M, K), y, flags=flags)
    want = np.zeros((M, N), bool)
    want[[1, 3, 4]], want[:, [7, 130]] = True, True
    np.testing.assert_array_equal(np.isnan(host(y)), want)
    with np.errstate(invalid="ignore"):
        xv, wv = np.nan_to_num(MX.values(*MX.quantize(host(x)), K)), np.nan_to_num(MX.values(host(wq[0]), host(wq[1]), K))
    ref, err = gelu_and_tolerance(*MX.grouped(xv, [wv], [b], [M], M), K, gelu)
    assert (np.abs(host(y) - ref) <= err)[~want].all()
    codes, scales = q8.mx4_empty(M, N)
    q8.q8_mx4_linear_dynamic(x, *wq, dev(b), *q8.mx4_empty(M, K), codes, y_scales=scales, flags=flags)
    expect = quantized(q8, y)
    assert torch.equal(scales, expect[1]) and torch.equal(codes, expect[0])
    block = want.reshape(M, N // 32, 32).any(-1)      # blocks of 32 columns with a NaN
    np.testing.assert_array_equal(host(scales).transpose(1, 0, 2).reshape(M, N // 32) == 255, block)


@pytest.mark.parametrize("M,K,N", [(4, 1024, 512), (200, 1000, 520)])
def test_dynamic_layer_captured_and_replayed(q8, M, K, N):
    """One launch and two in a graph, replayed on new activations between eager calls that share nothing with it."""
    g = np.random.default_rng(M)
    wq, b = quantized(q8, dev(activations(g, N, K))), dev(g.standard_normal(N).astype(np.float32))
    x, y, work = torch.zeros((M, K), dtype=torch.bfloat16, device="cuda"), torch.zeros((M, N), dtype=torch.bfloat16, device="cuda"), q8.mx4_empty(M, K)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        q8.q8_mx4_linear_dynamic(x, *wq, b, *work, y, flags=q8.EPI_GELU)
    for i in range(5):
        x.copy_(dev(activations(np.random.default_rng(i), M, K)))
        want = torch.empty_like(y)
        q8.q8_mx4_linear_dynamic(x, *wq, b, *q8.mx4_empty(M, K), want, flags=q8.EPI_GELU)
        torch.cuda.synchronize()
        y.fill_(7), work[0].fill_(0xFF), work[1].fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want), i


# ---- a mixture of experts on int8 codes ---------------------------------------------------------------------------------------

class Int8Moe:
    """As a program runs it: route, quantize, first layer with GELU to the next layer's codes and their abs-max, second layer, combine."""

    def __init__(self, q8, T, E, k, H, F, room=0):
        g = np.random.default_rng(T + E)
        self.q8, self.sizes, R = q8, (T, E, k, H, F), T * k + room
        i32, f32, i8 = (dict(dtype=t, device="cuda") for t in (torch.int32, torch.float32, torch.int8))
        self.x, self.logits = torch.empty((T, H), **f32), torch.empty((T, E), **f32)
        self.w1, self.w2 = dev(g.integers(-127, 128, (E, F, H)).astype(np.int8)), dev(g.integers(-127, 128, (E, H, F)).astype(np.int8))
        self.s1, self.s2 = (dev((127 / (n ** -0.5) * (0.5 + g.random(E))).astype(np.float32)) for n in (H, F))
        self.b1, self.b2 = dev(g.standard_normal((E, F)).astype(np.float32)), dev(g.standard_normal((E, H)).astype(np.float32))
        self.sx, self.sh, self.amax, self.h_amax = (torch.zeros(1, **f32) for _ in range(4))
        self.sh.fill_(20.0)
        self.experts, self.slots, self.counts, self.work = torch.empty((T, k), **i32), torch.empty((T, k), **i32), torch.empty(E, **i32), torch.empty(q8.ROUTE_BLOCKS * E, **i32)
        self.rows, self.gates = torch.zeros(R, **i32), torch.empty((T, k), **f32)
        self.xq, self.h, self.y, self.out = torch.empty((T, H), **i8), torch.zeros((R, F), **i8), torch.zeros((R, H), **f32), torch.zeros((T, H), **f32)
        self.fill(0)

    def fill(self, seed):
        g, (T, E, k, H, F) = np.random.default_rng(seed), self.sizes
        self.x.copy_(dev(g.standard_normal((T, H)).astype(np.float32))), self.logits.copy_(dev(g.standard_normal((T, E)).astype(np.float32)))

    def run(self, stream=None):
        q8, (T, E, k, H, F) = self.q8, self.sizes
        q8.q8_route(self.logits, self.experts, self.gates, self.counts, self.rows[: T * k], self.slots, self.work, stream=stream)
        q8.q8_absmax(self.x, self.amax, self.sx, stream=stream)
        q8.q8_quantize(self.x, self.sx, self.xq, stream=stream)
        q8.q8_linear_grouped(self.xq, self.w1, self.b1, self.sx, self.s1, self.counts, self.h, x_rows=self.rows, out_amax=self.h_amax, next_scale=self.sh,
                             flags=q8.EPI_GELU | q8.EPI_REQUANT | q8.EPI_ABSMAX, stream=stream)
        q8.q8_linear_grouped(self.h, self.w2, self.b2, self.sh, self.s2, self.counts, self.y, stream=stream)
        q8.q8_combine(self.y, self.slots, self.gates, self.out, stream=stream)
        return self.out


@pytest.mark.parametrize("T,E,k,H,F,room", [(1, 4, 2, 128, 256, 0), (33, 8, 2, 200, 384, 5), (100, 8, 2, 1024, 512, 56), (700, 6, 3, 256, 512, 40), (3000, 2, 1, 256, 256, 0)])
def test_int8_mixture_of_experts(q8, T, E, k, H, F, room):
    """The layers bit for bit as q8_linear has each expert's rows; rows behind the last expert's as they were."""
    m = Int8Moe(q8, T, E, k, H, F, room)
    R = T * k
    m.h.fill_(9), m.y.fill_(9)
    m.run()
    experts, gates, counts, rows, slots = MX.route(host(m.logits).astype(np.float32), k)
    for got, want in ((m.experts, experts), (m.counts, counts), (m.rows[:R], rows), (m.slots, slots)):
        np.testing.assert_array_equal(host(got), want)
    h, y, amax = torch.full_like(m.h, 9), torch.full_like(m.y, 9), torch.zeros(1, device="cuda")
    mine = m.xq[m.rows[:R].long()]
    for e, (a, z) in enumerate(MX.spans(counts, R)):
        if z > a:
            q8.q8_linear(mine[a:z].contiguous(), m.w1[e], m.b1[e], m.sx, m.s1[e: e + 1], h[a:z], out_amax=amax, next_scale=m.sh, flags=q8.EPI_GELU | q8.EPI_REQUANT | q8.EPI_ABSMAX)
            q8.q8_linear(h[a:z], m.w2[e], m.b2[e], m.sh, m.s2[e: e + 1], y[a:z])
    assert torch.equal(m.h, h) and torch.equal(m.y, y) and torch.equal(m.h_amax, amax)
    assert float(h[:R].float().abs().mean()) > 1      # the codes are in use
    terms = host(m.gates)[..., None] * host(m.y)[slots]
    err = k * 2.0 ** -24 * 1.001 * np.abs(terms).sum(1)        # k fused additions, each rounded once
    assert (np.abs(host(m.out) - terms.sum(1)) <= err).all()


def test_int8_mixture_of_experts_captured_and_replayed(q8):
    m = Int8Moe(q8, 150, 8, 2, 256, 512, room=10)
    m.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        m.run()
    for i in range(5):
        m.fill(i + 1)
        m.h_amax.zero_()
        want = m.run().clone(), m.h_amax.clone()
        torch.cuda.synchronize()
        m.out.zero_(), m.counts.zero_(), m.work.fill_(3), m.h_amax.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(m.out, want[0]) and torch.equal(m.h_amax, want[1]), i


@pytest.mark.parametrize("v", [2, 3, 4, 5])
@pytest.mark.parametrize("M", [1000, 1050, 2000, 2100])
def test_outputs_stored_for_the_caches_and_past_them(q8, v, M):
    """Outputs of either type on both sides of 32 MiB are the same numbers in every tile: those of the layer's rows taken a few at a time."""
    N, K = 8200, 256
    g = np.random.default_rng(M)
    xq, wq, b = quantized(q8, dev(activations(g, M, K))), quantized(q8, dev(activations(g, N, K))), dev(g.standard_normal(N).astype(np.float32))
    y, half = torch.full((M, N), 7.0, device="cuda"), torch.full((M, N), 7.0, dtype=torch.bfloat16, device="cuda")
    q8.set_product_variant(v)
    try:
        q8.q8_mx4_linear(*xq, *wq, b, y)
        q8.q8_mx4_linear(*xq, *wq, b, half)
        part = torch.empty((300, N), device="cuda")
        for m in (0, 500, M - 300):
            q8.q8_mx4_linear(xq[0][m: m + 300], xq[1][:, m: m + 300].contiguous(), *wq, b, part)
            assert torch.equal(part, y[m: m + 300])
    finally:
        q8.set_product_variant(0)
    assert torch.equal(half, y.bfloat16())


# ---- large tensors, and none of a reduction -------------------------------------------------------------------------------------

@pytest.mark.parametrize("M", [9, 600])
@pytest.mark.parametrize("flags", [0, 1, 3, 6])
def test_int8_grouped_without_a_reduction(q8, variant, M, flags):
    """K = 0: the quantized bias alone, as q8_linear has it."""
    g = np.random.default_rng(M)
    N, counts = 70, [M // 3, 0, M - M // 3 - 2]
    b, sw = dev(g.standard_normal((3, N)).astype(np.float32)), dev(np.array([900, 1000, 1100], np.float32))
    sx, ns = torch.tensor([31.7], device="cuda"), torch.tensor([40.0], device="cuda")
    x, w = torch.empty((M, 0), dtype=torch.int8, device="cuda"), torch.empty((3, N, 0), dtype=torch.int8, device="cuda")
    kind = torch.int8 if flags & q8.EPI_REQUANT else torch.float32
    y, amax, want, want_amax = torch.full((M, N), 7, dtype=kind, device="cuda"), torch.zeros(1, device="cuda"), torch.full((M, N), 7, dtype=kind, device="cuda"), torch.zeros(1, device="cuda")
    q8.q8_linear_grouped(x, w, b, sx, sw, dev(np.array(counts, np.int32)), y, out_amax=amax, next_scale=ns, flags=flags)
    for e, (a, z) in enumerate(MX.spans(counts, M)):
        if z > a:
            q8.q8_linear(x[a:z], w[e], b[e], sx, sw[e: e + 1], want[a:z], out_amax=want_amax, next_scale=ns, flags=flags)
    assert torch.equal(y, want) and torch.equal(amax, want_amax)


@pytest.mark.parametrize("v", [0, 1, 4])
def test_grouped_weights_beyond_32_bits(q8, v):
    """5.4 GB of codes: rows of the first and the last experts."""
    E, N, K, M = 80, 16384, 8192, 400
    g = torch.Generator(device="cuda")
    g.manual_seed(v)
    rand = lambda *s, lo=0, hi=256: torch.randint(lo, hi, s, generator=g, device="cuda", dtype=torch.uint8)  # noqa: E731
    xq, wq = (rand(M, K // 2), rand(K // 128, M, 4, lo=118, hi=128)), (rand(E, N, K // 2), rand(E, K // 128, N, 4, lo=118, hi=128))
    counts = torch.zeros(E, dtype=torch.int32, device="cuda")
    counts[0], counts[40], counts[E - 1] = 100, 130, M - 230
    y = torch.full((M, N), float("nan"), device="cuda")
    q8.set_product_variant(v)
    try:
        q8.q8_mx4_linear_grouped(*xq, *wq, None, counts, y)
    finally:
        q8.set_product_variant(0)
    cols = torch.tensor([0, 1, 127, 8191, N - 2, N - 1], device="cuda")
    xv = MX.values(host(xq[0]), host(xq[1]))
    for e, a, z in ((0, 0, 100), (40, 100, 230), (E - 1, 230, M)):
        wv = MX.values(host(wq[0][e][cols]), host(wq[1][e][:, cols]))
        err = (K / 64 + 10) * 2.0 ** -23 * (np.abs(xv[a:z]) @ np.abs(wv).T)      # K / 64 instructions, eight partial sums
        assert (np.abs(host(y[a:z][:, cols]) - xv[a:z] @ wv.T) <= err).all()
    assert not y.isnan().any()


@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
def test_combine_of_rows_beyond_32_bits(q8, kind):
    """4.6e9 elements of y and of out: first and last tokens."""
    R, N, k, T = 70000, 65536, 2, 70000
    y = torch.zeros((R, N), dtype=kind, device="cuda")
    y[:50], y[-50:] = torch.randn(50, N, device="cuda"), torch.randn(50, N, device="cuda")
    slots = torch.arange(T, dtype=torch.int32, device="cuda")[:, None].repeat(1, k)
    slots[:, 1] = T - 1 - slots[:, 1]
    gates = torch.rand(T, k, device="cuda")
    out = torch.full((T, N), 7, dtype=kind, device="cuda")
    q8.q8_combine(y, slots, gates, out)
    for t in (0, 1, 49, T - 50, T - 1):
        terms = gates[t].double()[:, None] * y[slots[t].long()].double()
        ref, mag = terms.sum(0), terms.abs().sum(0)
        err = k * 2.0 ** -24 * 1.001 * mag            # k fused additions, each rounded once
        if kind is torch.bfloat16:
            err = err + 2.0 ** -8 * (ref.abs() + err)
        assert ((out[t].double() - ref).abs() <= err).all()
    assert not out[60: 2000].any() and not out[T - 2000: T - 60].any()
    del y, out
    torch.cuda.empty_cache()


@pytest.mark.parametrize("T,E,k", [(1_500_000, 8, 2), (400_000, 200, 6)])
def test_route_of_millions_of_tokens(q8, T, E, k):
    """Long runs: against a stable sort of the logits and one of the choices."""
    g = torch.Generator(device="cuda")
    g.manual_seed(T)
    l = (torch.randn(T, E, generator=g, device="cuda") * 8).round() / 8                # many ties
    i32 = dict(dtype=torch.int32, device="cuda")
    experts, rows, slots, gates = torch.empty((T, k), **i32), torch.empty(T * k, **i32), torch.empty((T, k), **i32), torch.empty((T, k), device="cuda")
    counts, work = torch.empty(E, **i32), torch.empty(q8.ROUTE_BLOCKS * E, **i32)
    q8.q8_route(l, experts, gates, counts, rows, slots, work)
    top, want = (t[:, :k] for t in l.sort(dim=1, descending=True, stable=True))
    assert torch.equal(experts, want.int())
    flat = want.reshape(-1)
    order = flat.argsort(stable=True)
    assert torch.equal(counts, torch.bincount(flat, minlength=E).int()) and torch.equal(rows, (order // k).int())
    place = torch.empty_like(order)
    place[order] = torch.arange(T * k, device="cuda")
    assert torch.equal(slots.view(-1), place.int())
    # logits within 16 of each other: an argument rounded once, exp within two ulps, a sum of k and a division
    assert ((gates.double() - torch.softmax(top.double(), 1)).abs() <= (16 * 2.0 ** -24 + 2.0 ** -21 + k * 2.0 ** -23) * torch.softmax(top.double(), 1)).all()
