"""block_norm and its gradients with a LayerNorm behind the block, on rows that one
wave or several share: each wave sums about its own mean, so what it adds for the
row's mean must not reach the columns past the row's end."""
import pytest

from test_gpu_operators import ALL, BF16, FP32, SIZES, U, _check_backward, _check_forward, _gen, _norm64, _randn, _stored, _within

torch = pytest.importorskip("torch")
kq = pytest.importorskip("paper_2607_21446_amd")

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _device():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    kq.lib()
    yield


# widths beside each number of waves a row takes, on few rows (one vector a lane) and on many (two)
MORE = [(2, 1, 513), (300, 1, 513), (2, 2, 1025), (1030, 1, 1155), (300, 1, 2049), (300, 2, 4097), (5, 1, 4100), (260, 1, 8193)]


@pytest.mark.parametrize("names", [ALL, (), ("gate",)], ids=["all", "none", "gate"])
@pytest.mark.parametrize("norm", ["layer", "rms"])
@pytest.mark.parametrize("M,B,d", [s for s in SIZES if s[2] > 7] + MORE)
def test_post_layer_sizes(M, B, d, norm, names):
    _check_forward(M, B, d, FP32, FP32, FP32, norm, "layer", names)
    _check_forward(M, B, d, BF16, BF16, BF16, norm, "layer", names)


@pytest.mark.parametrize("norm", ["layer", "rms"])
@pytest.mark.parametrize("M,B,d", [s for s in SIZES if s[2] > 7] + MORE)
def test_post_layer_gradient_sizes(M, B, d, norm):
    _check_backward(M, B, d, FP32, FP32, FP32, norm, "layer", ALL)
    _check_backward(M, B, d, BF16, BF16, BF16, norm, "layer", ())


@pytest.mark.parametrize("norm", ["layer", "rms"])
@pytest.mark.parametrize("M", [3, 400])
@pytest.mark.parametrize("d", [500, 515, 520, 1155, 2049, 3071, 4099, 8195])
def test_post_layer_where_the_waves_means_differ(M, d, norm):
    """A few channels of x times 20 and the row's first half raised by 3, so that what a wave adds for the row's mean
    is of the size of the values.

    A row's sum takes at most 16 values a lane, 6 steps over the lanes and 16 waves, 38 additions: 64 U of the mean
    magnitude covers a mean's error, its subtraction in two parts included.  The squares then are off by 38 U and by
    2 * 64 U (|x| + mean |x|) / deviation <= 256 U (rms of x at most the deviation plus |mean|, here below 1.5
    deviations: 400 U), half of which the root keeps: 240 U with the hardware's root."""
    g = _gen(5 * M + d)
    x, res = _randn(g, M, d), _randn(g, M, d)
    x[:, torch.randperm(d, generator=g, device="cuda")[: max(1, d // 200)]] *= 20.0
    x[:, : d // 2] += 3.0
    alpha, eps = 0.75, 1e-6
    h, y = kq.block_norm(x, res, norm=norm, post_norm="layer", alpha=alpha, eps=eps)
    x64, res64 = x.double(), res.double()
    u, rx = _norm64(x64, "layer", eps)
    assert float(((x64.square().mean(-1).sqrt() * rx[:, 0]).max())) < 1.5
    h64 = res64 + alpha * u
    herr = alpha * (64 * U * rx * (x64.abs() + x64.abs().mean(-1, keepdim=True)) + 240 * U * u.abs()) + 4 * U * (res64.abs() + u.abs())
    _within(h, h64, herr + _stored(h64, FP32), "h")
    n, r = _norm64(h64, norm, eps)
    # h's own errors enter y by r and, over the row's deviation, by its factor
    off = herr + (herr.mean(-1, keepdim=True) if norm == "layer" else 0.0)
    factor = 240 * U + r * off.square().mean(-1, keepdim=True).sqrt()
    yerr = r * (off + 64 * U * (h64.abs() + h64.abs().mean(-1, keepdim=True))) + n.abs() * factor
    _within(y, n, yerr * 1.01 + _stored(n, FP32), "y")
