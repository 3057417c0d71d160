"""The operators of a generation step together (examples/w4a16_step.py), every step
against its definition in 64 bits from what the step before it left; captured and
replayed; on another stream; and the two ways their arguments are marshalled."""
import importlib.util
import os

import pytest

from conftest import ROOT

torch = pytest.importorskip("torch")
kq = pytest.importorskip("paper_2607_21446_amd")

pytestmark = pytest.mark.gpu

ROUNDED = 2.0 ** -8  # to bf16


@pytest.fixture(scope="module")
def block():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spec = importlib.util.spec_from_file_location("w4a16_step", os.path.join(ROOT, "examples", "w4a16_step.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def _values(codes, scales):
    nib = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).long()
    mag = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device=codes.device)[nib & 7]
    return torch.where(nib >= 8, -mag, mag) * torch.exp2(scales.double() - 127).repeat_interleave(32, -1)


def _close(got, want, what, rounded=ROUNDED):
    """One rounding of the result, and 1e-4 of its size for sums in 32 bits (K U = 7e-5 of the terms, which cancel)."""
    tol = rounded * want.abs() * 1.01 + 1e-4 * want.square().mean().sqrt()
    assert ((got.double() - want).abs() <= tol).all(), what


def _stream(g, batch, width):
    return torch.randn((batch, width), generator=g, device="cuda").to(torch.bfloat16)


@pytest.mark.parametrize("format", ["bf16", "mxfp8", "mxfp4"])
def test_steps(block, format):
    p = block.inputs(format=format)
    g = torch.Generator(device="cuda").manual_seed(3)
    H, KV, D = block.HEADS, block.KV_HEADS, block.D
    p["lengths"] += torch.tensor([0, 3, 15, 16, 100], dtype=torch.int32, device="cuda")  # (what is there is zeros)
    for _ in range(6):
        x = _stream(g, 5, H * D)
        out, m = block.step(x, p)
        h = x.double()
        _close(m["y"], h / (h.square().mean(-1, keepdim=True) + 1e-6).sqrt() * p["norm"].double(), "norm")
        _close(m["raw"].view(5, -1), m["y"].double() @ _values(*p["qkv"]).T, "projection")
        turn = m["at"].double()[:, None] * 10000.0 ** (-torch.arange(D // 2, device="cuda").double() * 2 / D)
        z = torch.complex(*m["raw"][:, :H + KV].double().unflatten(-1, (2, D // 2)).unbind(-2)) * torch.polar(torch.ones_like(turn), turn)[:, None]
        _close(m["qkv"][:, :H + KV], torch.cat([z.real, z.imag], -1), "rope")
        assert torch.equal(m["qkv"][:, H + KV:], m["raw"][:, H + KV:])
        a = torch.zeros((5, H, D), dtype=torch.float64, device="cuda")
        for b, n in enumerate(p["lengths"].tolist()):
            t = torch.arange(n, device="cuda")
            k, v = kq.kv_cache_read(p["cache"], p["table"][b].long()[t // 16] * 16 + t % 16, out_dtype=torch.float32)
            new = m["qkv"][b, H:H + KV].double()
            # half a step (2^-4 of a value in E4M3, 1 in 4 of the largest in E2M1), or saturation: blocks whose largest is
            # below 2^9 (8) units stop at 448 (6), 1/8 (1/4) of it away at most
            step = {"bf16": new.abs() * 2.0 ** -8, "mxfp8": new.abs().amax() / 8, "mxfp4": new.abs().amax() / 4}[format]
            assert ((k[-1].double() - new).abs() <= step).all()
            k, v = (c.double().transpose(0, 1).repeat_interleave(H // KV, 0) for c in (k, v))
            s = (m["qkv"][b, :H].double().unsqueeze(1) * k).sum(-1) / D ** 0.5
            a[b] = (torch.softmax(s, -1).unsqueeze(-1) * v).sum(1)
        _close(m["a"], a, "attention")
        _close(out, x.double() + m["a"].double().view(5, -1) @ _values(*p["out"]).T, "output")


def test_steps_captured(block):
    """A captured step, replayed with eager work between, is the eager step: the lengths and the cache grow on the device."""
    H, D = block.HEADS, block.D
    g = torch.Generator(device="cuda").manual_seed(5)
    xs = [_stream(g, 5, H * D) for _ in range(24)]
    want, p = [], block.inputs(format="mxfp4")
    for x in xs:
        want.append(block.step(x, p)[0].clone())
    q = block.inputs(format="mxfp4")
    x = xs[0].clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):  # (a warm step before the capture, then the state from the start again)
        block.step(x, q)
    torch.cuda.current_stream().wait_stream(side)
    for t in q["cache"]:
        t.zero_()
    q["lengths"].zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, _ = block.step(x, q)
    q["lengths"].zero_()
    other = block.inputs(format="mxfp8")
    for i, (now, then) in enumerate(zip(xs, want)):
        x.copy_(now)
        graph.replay()
        if i % 3 == 0:
            block.step(now, other)
            torch.cuda.synchronize()
        assert torch.equal(out, then), i
    assert torch.equal(q["lengths"], p["lengths"]) and all(torch.equal(a, b) for a, b in zip(q["cache"], p["cache"]))


def _calls(seed=7):
    """Every call with (name, fn(stream)): results as a tuple of tensors."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    randn = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    x = randn(33, 6, 96).to(torch.bfloat16)
    pos = torch.randint(0, 5000, (33, 2), generator=g, device="cuda")
    freqs = torch.rand(48, generator=g, device="cuda", dtype=torch.float64)
    caches = [kq.kv_cache(6, 16, 2, 96, format=f) for f in ("bf16", "mxfp8", "mxfp4")]
    slots = torch.randperm(96, generator=g, device="cuda")[:33]
    big = kq.kv_cache(80, 64, 4, 128, format="mxfp4")
    kv = randn(80 * 64, 2, 4, 128)
    kq.kv_cache_write(big, kv[:, 0], kv[:, 1], torch.arange(80 * 64, device="cuda"))
    table = torch.randperm(80, generator=g, device="cuda").to(torch.int32).reshape(4, 20)
    n = torch.tensor([1280, 0, 77, 900], dtype=torch.int32, device="cuda")
    q = randn(4, 16, 128).to(torch.bfloat16)
    wide, w = randn(16, 8192), kq.mxfp4((randn(96, 8192) / 90).to(torch.bfloat16))
    few, u = randn(3, 256).to(torch.bfloat16), kq.mxfp4((randn(70, 256) / 16).to(torch.bfloat16))
    bias, gate, residual = randn(70), randn(3, 70), randn(3, 70)

    def written(c, s):
        kq.kv_cache_write(c, x[:, :2], x[:, 2:4], slots, stream=s)
        return kq.kv_cache_read(c, slots, stream=s, out_dtype=torch.float32)

    calls = [("rope", lambda s: (kq.rope(x, pos, [64, 32], pairing="halves", theta=500.0, stream=s),)),
             ("rope", lambda s: (kq.rope_backward(x[:, 1:5], pos[:, 0], 96, freqs=freqs, stream=s),)),
             ("paged_attention", lambda s: (kq.paged_attention(q, big, table, n, stream=s),)),
             ("paged_attention", lambda s: kq.paged_attention(q.float(), big, table, n, window=300, scale=0.2, want_lse=True, stream=s)),
             ("w4a16_linear", lambda s: (kq.w4a16_linear(wide, *w, act="silu", stream=s),)),
             ("w4a16_linear", lambda s: (kq.w4a16_linear(few, *u, bias=bias, gate=gate, residual=residual, stream=s),))]
    return calls + [("kv_cache_write", lambda s, c=c: written(c, s)) for c in caches]


class _NoNative:
    """Stands for the binding's native part and takes no call."""

    def __getattr__(self, name):
        return lambda *args: None


class _Recorder:
    """The native part, and the calls that it took."""

    def __init__(self, native):
        self.native, self.taken = native, []

    def __getattr__(self, name):
        def call(*args):
            r = getattr(self.native, name)(*args)
            if r is not None:
                self.taken.append(name)
            return r
        return call


@pytest.mark.parametrize("stream", [None, "handle"])
def test_native_marshalling_matches_python(block, monkeypatch, stream):
    from paper_2607_21446_amd import binding
    s = torch.cuda.current_stream().cuda_stream if stream else None
    recorder = _Recorder(binding._native())
    for i, (name, call) in enumerate(_calls()):
        recorder.taken.clear()
        monkeypatch.setattr(binding, "_native", lambda: recorder)
        got = call(s)
        # (with a stream of its own, a call that makes a workspace is marshalled in Python)
        makes = name == "paged_attention" or i == 4
        assert recorder.taken[:1] == ([] if stream and makes else [name]), (i, recorder.taken)
        monkeypatch.setattr(binding, "_native", _NoNative)
        want = call(s)
        assert len(got) == len(want) and all(a.dtype == b.dtype and a.shape == b.shape and torch.equal(a, b) for a, b in zip(got, want)), i


@pytest.mark.parametrize("native", [True, False])
def test_on_another_stream(block, monkeypatch, native):
    """A call on a side stream, ordered with the current one by the caller, gives what it gives there; its own workspace is
    that stream's, whatever the current stream allocates meanwhile."""
    from paper_2607_21446_amd import binding
    if not native:
        monkeypatch.setattr(binding, "_native", _NoNative)
    side = torch.cuda.Stream()
    for i, (name, call) in enumerate(_calls()):
        want = [t.clone() for t in call(None)]
        side.wait_stream(torch.cuda.current_stream())
        got = call(side)
        junk = [torch.full((1 << 20,), 255, dtype=torch.uint8, device="cuda") for _ in range(8)]
        torch.cuda.current_stream().wait_stream(side)
        assert all(torch.equal(a, b) for a, b in zip(got, want)), (i, name)
        del junk


def test_two_graphs_and_workspaces(block):
    """Two captured attention calls, each with its own workspace, replayed in turn and on two streams at once."""
    g = torch.Generator(device="cuda").manual_seed(11)
    cache = kq.kv_cache(256, 64, 2, 64)
    kv = torch.randn((256 * 64, 2, 2, 64), generator=g, device="cuda")
    kq.kv_cache_write(cache, kv[:, 0], kv[:, 1], torch.arange(256 * 64, device="cuda"))
    table = torch.arange(256, dtype=torch.int32, device="cuda").reshape(2, 128)
    n = [torch.tensor(t, dtype=torch.int32, device="cuda") for t in ([8192, 100], [5000, 8000])]
    q = [torch.randn((2, 8, 64), generator=g, device="cuda").to(torch.bfloat16) for _ in range(2)]
    want = [kq.paged_attention(q[i], cache, table, n[i]) for i in range(2)]
    ws, out, graphs = [kq.paged_attention_workspace(2, 8, 2, 64) for _ in range(2)], [torch.empty_like(t) for t in q], []
    for i in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[i]):
            kq.paged_attention(q[i], cache, table, n[i], out=out[i], workspace=ws[i])
    streams = [torch.cuda.Stream() for _ in range(2)]
    for turn in range(12):
        for o in out:
            o.zero_()
        for i in range(2):
            streams[i].wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(streams[i] if turn % 2 else torch.cuda.current_stream()):
                graphs[i].replay()
        for s in streams:
            torch.cuda.current_stream().wait_stream(s)
        assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1]), turn


def test_calls_keep_no_gradient_and_take_parameters(block):
    """Parameters are plain arrays to these calls, as for the others of the library."""
    x = torch.nn.Parameter(torch.randn((4, 2, 64), device="cuda"))
    y = kq.rope(x, torch.arange(4, device="cuda"), 64)
    assert not y.requires_grad and torch.equal(y, kq.rope(x.detach(), torch.arange(4, device="cuda"), 64))


def test_example_runs(block, capsys):
    block.main()
    assert "tokens [40, 40, 40, 40, 40]" in capsys.readouterr().out
