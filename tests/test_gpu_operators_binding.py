"""The binding of block_norm, mxfp4_linear and mxfp4_grouped_linear on arguments at
the edge of what it takes."""
import pytest

torch = pytest.importorskip("torch")
kq = pytest.importorskip("paper_2607_21446_amd")

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _device():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    kq.lib()
    yield


def _codes(*shape):
    *lead, K = shape
    return (torch.full((*lead, K // 2), 0x21, dtype=torch.uint8, device="cuda"),
            torch.full((*lead, K // 32), 127, dtype=torch.uint8, device="cuda"))


class _NoNative:
    """Stands for the binding's native part and takes no call."""

    def __getattr__(self, name):
        return lambda *args: None


@pytest.mark.parametrize("M", [0, 4])
def test_vectors_of_no_batches_are_refused(M):
    """A gate [0, N] belongs to no row: an error that names it, and no division by the number of batches."""
    a, b = _codes(M, 64), _codes(6, 64)
    none = torch.empty((0, 6), device="cuda")
    with pytest.raises(ValueError, match="0 batches"):
        kq.mxfp4_linear(*a, *b, gate=none)
    with pytest.raises(ValueError, match="0 batches"):
        kq.mxfp4_linear(*a, *b, bias=torch.zeros(6, device="cuda"), gate=none)
    with pytest.raises(ValueError, match="0 batches"):
        kq.mxfp4_linear(*a, *b, act="swiglu", gate=none[:, :3].contiguous())
    x = torch.zeros((M, 6), device="cuda")
    for name in ("gate", "scale", "shift"):
        with pytest.raises(ValueError, match="0 batches"):
            kq.block_norm(x, x, **{name: none})
        with pytest.raises(ValueError, match="0 batches"):
            kq.block_norm_backward(x, x, x=x, **{name: none})


@pytest.mark.parametrize("native", [True, False], ids=["native", "python"])
@pytest.mark.parametrize("norm", ["rms", "layer"])
@pytest.mark.parametrize("M,d", [(5, 64), (3, 1155), (300, 1152)])
def test_the_stream_outlives_a_norm_in_place(monkeypatch, native, norm, M, d):
    """y over x, with nothing that makes h another array than x: h still holds what x held."""
    from paper_2607_21446_amd import binding
    if not native:
        monkeypatch.setattr(binding, "_native", _NoNative)
    g = torch.Generator(device="cuda")
    g.manual_seed(M + d)
    x = torch.randn((M, d), generator=g, device="cuda").to(torch.bfloat16)
    was = x.clone()
    _, want = kq.block_norm(x, norm=norm)
    assert torch.equal(x, was)
    h, y = kq.block_norm(x, norm=norm, y=x)
    assert y is x and torch.equal(y, want)
    assert h is not x and torch.equal(h, was)
    view = was.clone()
    h, y = kq.block_norm(view, norm=norm, y=view[:])  # the same memory by another tensor
    assert torch.equal(h, was) and torch.equal(view, want)


@pytest.mark.parametrize("kind", ["object", "handle", "default", "current"])
def test_a_workspace_of_the_call_is_its_streams(monkeypatch, kind):
    """Without a workspace a call makes one and drops it while its kernels may still run: its memory belongs to the
    stream that they run on, so that no work of another stream is given it."""
    from paper_2607_21446_amd import binding
    side = torch.cuda.Stream()
    stream = {"object": side, "handle": side.cuda_stream, "default": 0, "current": None}[kind]
    at = {"object": side, "handle": side}.get(kind, torch.cuda.default_stream()).cuda_stream
    g = torch.Generator(device="cuda")
    g.manual_seed(6)
    bf16 = lambda *s: torch.randn(s, generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
    x, h, dy, w = bf16(96, 512), bf16(96, 512), bf16(96, 512), bf16(512)
    X, W = bf16(64, 128), bf16(96, 128)
    lam = torch.tensor([0.5, 0.25], device="cuda")
    lu = kq.hadamard_lu(1)
    Y, mine = kq.calib_reference(X, W), lu.clone()
    calls = [lambda **k: list(kq.block_norm_backward(dy, h, x=x, gate=w, weight=w, **k).values()),
             lambda **k: list(kq.calib_step(X, W, Y, lu, lam, a=4, **k)),
             lambda **k: list(kq.calibrate(X, W, lu=mine, a=4, steps=2, **k))]
    want = [[t.clone() for t in c()] for c in calls]
    made = []

    def noted(name):
        real = getattr(binding, name)

        def f(*args):
            t = real(*args)
            made.append((torch.cuda.current_stream().cuda_stream, t.data_ptr(), t.numel()))
            return t
        monkeypatch.setattr(binding, name, f)

    noted("block_norm_workspace")
    noted("calib_workspace")
    for i, c in enumerate(calls):
        made.clear()
        mine.copy_(lu)
        torch.cuda.synchronize()  # the other stream takes no inputs that are still being written
        got = c(stream=stream)
        assert len(made) == 1 and made[0][0] == at, i
        assert torch.cuda.current_stream() == torch.cuda.default_stream()
        if at == side.cuda_stream:  # dropped, and not given to the current stream
            t = torch.empty(made[0][2], dtype=torch.uint8, device="cuda")
            assert t.data_ptr() != made[0][1], i
        torch.cuda.synchronize()
        for a, b in zip(got, want[i], strict=True):
            assert torch.equal(a, b), i
