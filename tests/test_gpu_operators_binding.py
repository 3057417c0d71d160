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


class _Recorder:
    """The native part; every call that it makes is noted, None for one that it leaves to Python."""

    def __init__(self, native):
        self.native, self.taken = native, []

    def __getattr__(self, name):
        def f(*args):
            r = getattr(self.native, name)(*args)
            self.taken.append(None if r is None else name)
            return r
        return f


def _calls():
    """Name, call with buffers of its own (given) or none, and which results are then the caller's."""
    g = torch.Generator(device="cuda")
    g.manual_seed(7)
    randn = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    bf16 = lambda *s: randn(*s).to(torch.bfloat16)  # noqa: E731
    M, d = 12, 150
    x, res, mod, w = bf16(M, d), randn(M, d), bf16(3, 6 * d), bf16(d)
    norm_args = dict(gate=mod[:, :d], scale=mod[:, d:2 * d], shift=mod[:, 2 * d:3 * d], weight=w)
    new = lambda dtype, *s: torch.full(s, 7.0, dtype=dtype, device="cuda")  # noqa: E731

    def norm(given, stream, **kw):
        k = dict(h=new(torch.float32, M, d), y=new(torch.bfloat16, M, d)) if given else {}
        out = kq.block_norm(x, res, **kw, **k, stream=stream)
        return out, [k["h"], k["y"]] if given else None

    def plain_norm(given, stream):
        return kq.block_norm(x, weight=w, norm="rms", stream=stream, **(dict(y=new(torch.bfloat16, M, d)) if given else {})), None

    K, N, E = 96, 70, 3
    random = lambda *s: torch.randint(0, 256, s, generator=g, device="cuda", dtype=torch.uint8)  # noqa: E731
    scales = lambda *s: torch.randint(123, 128, s, generator=g, device="cuda", dtype=torch.uint8)  # noqa: E731
    a, b, be = (random(M, K // 2), scales(M, K // 32)), (random(N, K // 2), scales(N, K // 32)), (random(E, N, K // 2), scales(E, N, K // 32))
    off = torch.tensor([0, 5, 5, 20], dtype=torch.int32, device="cuda")
    rows = torch.randint(0, M, (20,), generator=g, device="cuda").to(torch.int32)
    bias, biases, row_scale, gate = randn(N), bf16(E, N), randn(20), randn(2, N + 9)[:, 4:4 + N]

    def linear(given, stream, act, **kw):
        n = N // 2 if act == "swiglu" else N
        residual = new(torch.float32, M, n + 3)[:, 1:n + 1] if "gate" in kw else None
        out = new(torch.float32, M, n + 5)[:, 2:n + 2] if given else None
        r = kq.mxfp4_linear(*a, *b, bias=bias, act=act, residual=residual, out=out, out_dtype=torch.float32, stream=stream, **kw)
        return (r,), [out] if given else None

    def grouped(given, stream, act, **kw):
        n = N // 2 if act == "swiglu" else N
        out = new(torch.bfloat16, 20 if "rows" in kw else M, n) if given else None
        o = off if "rows" in kw else off.clamp_max(M)
        r = kq.mxfp4_grouped_linear(*a, *be, o, act=act, out=out, stream=stream, **kw)
        return (r,), [out] if given else None

    return [("block_norm", lambda g_, s: norm(g_, s, norm="layer", post_norm="layer", post_weight=w, alpha=0.5, **norm_args)),
            ("block_norm", lambda g_, s: norm(g_, s, norm="rms")),
            ("block_norm", plain_norm),
            ("mxfp4_linear", lambda g_, s: linear(g_, s, "gelu")),
            ("mxfp4_linear", lambda g_, s: linear(g_, s, None, gate=gate)),
            ("mxfp4_linear", lambda g_, s: linear(g_, s, "swiglu")),
            ("mxfp4_grouped_linear", lambda g_, s: grouped(g_, s, "swiglu", rows=rows, row_scale=row_scale)),
            ("mxfp4_grouped_linear", lambda g_, s: grouped(g_, s, None, bias=biases))]


@pytest.mark.parametrize("given", [False, True])
def test_native_marshalling_matches_python(monkeypatch, given):
    """The native part takes these calls, and the checks and the ctypes call in Python return the same: values, types
    and, for buffers that were given, the same objects."""
    from paper_2607_21446_amd import binding
    stream = torch.cuda.current_stream().cuda_stream if given else None
    recorder = _Recorder(binding._native())
    for i, (name, call) in enumerate(_calls()):
        recorder.taken.clear()
        monkeypatch.setattr(binding, "_native", lambda: recorder)
        got, mine = call(given, stream)
        assert recorder.taken == [name], (i, recorder.taken)
        monkeypatch.setattr(binding, "_native", _NoNative)
        want, his = call(given, stream)
        assert len(got) == len(want)
        for j, (p, q) in enumerate(zip(got, want)):
            assert p.dtype == q.dtype and p.shape == q.shape and torch.equal(p, q), (i, j)
            if mine is not None:
                assert p is mine[j] and q is his[j], (i, j)


def test_what_the_native_part_leaves_to_python():
    """A tensor of another layout, type or size is none that the native part takes."""
    from paper_2607_21446_amd import binding
    native = binding._native()
    x = torch.zeros((8, 64), device="cuda")
    norm = lambda x, **k: native.block_norm(x, k.get("residual"), k.get("gate"), None, None, None, None, 1, 0, 1.0, 1e-6,  # noqa: E731
                                            k.get("h"), k.get("y"), None, k.get("stream"))
    assert norm(x) is not None
    for bad in (dict(x=x.t()), dict(x=x.half()), dict(x=x[0]), dict(x=x, residual=x[:4]), dict(x=x, gate=x[:3]), dict(x=x, gate=x[:0]),
                dict(x=x, gate=x[:2, :32]), dict(x=x, y=x.bfloat16()), dict(x=x, h=x[:, :32]), dict(x=x, stream=torch.cuda.current_stream())):
        assert norm(**bad) is None, bad
    a, b = _codes(4, 64), _codes(6, 64)
    linear = lambda a=a, b=b, bias=None, act=0, gate=None, res=None, out=None: native.mxfp4_linear(  # noqa: E731
        *a, *b, bias, act, gate, res, out, None, None)
    assert linear() is not None
    f = torch.zeros((4, 6), device="cuda")
    for bad in (dict(a=(a[0], a[1][:2])), dict(b=_codes(6, 32)), dict(bias=f[0, :5]), dict(gate=f[:3]), dict(act=5, b=_codes(5, 64)),
                dict(res=f, out=f.bfloat16()), dict(out=f[:, :5]), dict(out=f[:1].expand(4, 6)), dict(gate=f[:0])):
        assert linear(**bad) is None, bad
    e = (b[0][None], b[1][None])
    off = torch.tensor([0, 4], dtype=torch.int32, device="cuda")
    grouped = lambda e=e, off=off, rows=None, bias=None, rs=None: native.mxfp4_grouped_linear(  # noqa: E731
        *a, *e, off, rows, bias, 0, rs, None, None, None)
    assert grouped() is not None
    for bad in (dict(e=b), dict(off=off[:1]), dict(off=off.long()), dict(rows=off.long()), dict(bias=f[:2]), dict(rs=f[0, :3])):
        assert grouped(**bad) is None, bad
