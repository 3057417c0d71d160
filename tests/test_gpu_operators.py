"""The operators around a W4A4 linear layer against plain forms in 64 bits:
block_norm and its gradients, mxfp4_linear and mxfp4_grouped_linear, at the
sizes, types, masks and layouts where they can go wrong.

Tolerances follow from the arithmetic.  U = 2^-24 (fp32), one rounding to bf16
is 2^-8 of the result (8 significant bits).  A sum of n fp32 terms in any order is within n U of the
sum of magnitudes; the bounds below name the terms they multiply."""
import math

import pytest

torch = pytest.importorskip("torch")
kq = pytest.importorskip("paper_2607_21446_amd")

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
BF16, FP32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _device():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    kq.lib()
    yield


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(g, *shape, dtype=FP32):
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


def _within(got, want, tol, what):
    bad = ~((got.double() - want).abs() <= tol)
    assert not bad.any(), (what, int(bad.sum()), float((got.double() - want)[bad].abs().max()), float(tol[bad].min()))


def _stored(want, dtype):
    """What rounding to the output's type may add (fp32 results below its smallest normal: none)."""
    return want.abs() * (2.0 ** -8 if dtype == BF16 else U) * 1.01


# ------------------------------------------------------------------ norms

def _norm64(v, kind, eps):
    if kind == "layer":
        v = v - v.mean(-1, keepdim=True)
    r = 1.0 / (v.square().mean(-1, keepdim=True) + eps).sqrt()
    return v * r, r


def _rows64(v, M):
    """A vector, or one for each batch, as rows."""
    if v is None:
        return None
    v = v.double()
    return v if v.dim() == 1 else v.repeat_interleave(M // v.shape[0], 0)


def _forward64(x, residual, v, norm, post, alpha, eps):
    M = x.shape[0]
    u = x.double()
    if post:
        u = _norm64(u, post, eps)[0]
        if v.get("post_weight") is not None:
            u = u * v["post_weight"].double()
    au = alpha * (u * _rows64(v["gate"], M) if v.get("gate") is not None else u)
    h = au if residual is None else residual.double() + au
    if norm is None:
        return h, None, au, None
    n, r = _norm64(h, norm, eps)
    m = 1.0
    if v.get("weight") is not None:
        m = m * v["weight"].double()
    if v.get("scale") is not None:
        m = m * (1.0 + _rows64(v["scale"], M))
    y = n * m
    if v.get("shift") is not None:
        y = y + _rows64(v["shift"], M)
    # magnitude that an error of the norm's factors and of the mean multiplies
    reach = (n.abs() + r * h.abs().mean(-1, keepdim=True)) * (m.abs() if torch.is_tensor(m) else 1.0)
    return h, y, au, reach


def _vectors(g, B, d, dtype, names, strided=True):
    out = {}
    mod = (0.3 * _randn(g, B, 6 * d + 1)).to(dtype)[:, 1:]  # slices of one tensor, none of them aligned
    for i, n in enumerate(("shift", "scale", "gate")):
        if n in names:
            out[n] = mod[:, i * d:(i + 1) * d] if strided else mod[0, i * d:(i + 1) * d].clone()
    if "weight" in names:
        out["weight"] = (1.0 + 0.1 * _randn(g, d)).to(dtype)
    if "post_weight" in names:
        out["post_weight"] = (0.5 + 0.1 * _randn(g, d)).to(dtype)
    return out


ALL = ("shift", "scale", "gate", "weight", "post_weight")
# rows, batches, columns: one element, one row, odd and ragged widths at every number of waves a row
# takes, the widest row; few rows and many
SIZES = [(1, 1, 1), (1, 1, 7), (3, 1, 8), (5, 5, 33), (2, 1, 511), (1, 1, 4096), (6, 2, 1155), (4, 1, 2049), (3, 3, 4097),
         (2, 1, 8193), (2, 2, 16383), (1, 1, 16384), (1030, 2, 77), (1025, 1, 513), (1200, 3, 1152), (1027, 1, 1537),
         (1028, 4, 2047), (1024, 1, 3071), (1031, 1, 4099)]


def _check_forward(M, B, d, x_dtype, s_dtype, v_dtype, norm, post, names, alpha=0.75, eps=1e-6, residual=True, offset=0.0, seed=0):
    g = _gen(seed + M + d)
    x, res = _randn(g, M, d, dtype=x_dtype), ((_randn(g, M, d) + offset).to(s_dtype) if residual else None)
    v = _vectors(g, B, d, v_dtype, [n for n in names if n != "post_weight" or post])
    h, y = kq.block_norm(x, res, norm=norm, post_norm=post, alpha=alpha, eps=eps, h_dtype=None if residual else s_dtype, **v)
    h64, y64, au, reach = _forward64(x, res, v, norm, post, alpha, eps)
    assert h.dtype == s_dtype and h.shape == x.shape
    base = (res.double().abs() if residual else 0.0) + au.abs()
    # the post norm's factor: a sum of d squares over at least 8 d / 16384 lanes, 40 U covers the tree and the division
    mean = x.double().abs().mean(-1, keepdim=True) if post else torch.zeros(1, device="cuda", dtype=torch.float64)
    herr = 48 * U * (base + mean * 4)
    _within(h, h64, herr + _stored(h64, s_dtype), "h")
    if norm is None:
        assert y is None
        return
    assert y.dtype == x_dtype
    spread = 1.0 / _norm64(h64, norm, eps)[1]  # an error of h, over the row's deviation
    shift = _rows64(v["shift"], M).abs() if "shift" in v else 0.0
    gain = reach / (spread * (_norm64(h64, norm, eps)[0].abs() + _norm64(h64, norm, eps)[1] * h64.abs().mean(-1, keepdim=True)).clamp_min(1e-30))
    tol = 96 * U * (reach + shift) + gain * (herr + herr.mean(-1, keepdim=True)) * 2
    _within(y, y64, tol + _stored(y64, x_dtype), "y")


@pytest.mark.parametrize("M,B,d", SIZES)
def test_norm_sizes(M, B, d):
    _check_forward(M, B, d, BF16, BF16, BF16, "rms", None, ("weight",))
    _check_forward(M, B, d, BF16, FP32, FP32, "layer" if d > 1 else "rms", "rms", ALL)


@pytest.mark.parametrize("x_dtype", [BF16, FP32])
@pytest.mark.parametrize("s_dtype", [BF16, FP32])
@pytest.mark.parametrize("v_dtype", [BF16, FP32])
@pytest.mark.parametrize("norm,post", [("rms", None), ("layer", "layer"), ("rms", "layer"), (None, "rms"), ("layer", None)])
def test_norm_types(x_dtype, s_dtype, v_dtype, norm, post):
    _check_forward(12, 3, 323, x_dtype, s_dtype, v_dtype, norm, post, ALL if norm else ("gate", "post_weight"))


@pytest.mark.parametrize("names", [(), ("gate",), ("shift",), ("scale", "weight"), ("gate", "shift", "scale"), ("post_weight",)])
@pytest.mark.parametrize("residual", [True, False])
def test_norm_optional_vectors(names, residual):
    _check_forward(9, 3, 200, BF16, FP32, FP32, "layer", "rms" if "post_weight" in names else None, names, residual=residual)


def test_norm_of_a_large_mean():
    """The mean goes before the squares are summed: a stream far from zero keeps its digits."""
    _check_forward(40, 1, 1000, FP32, FP32, FP32, "layer", None, (), offset=1000.0)


def test_norm_returns_the_input_where_it_is_h():
    x = _randn(_gen(1), 5, 64, dtype=BF16)
    h, y = kq.block_norm(x, norm="rms")
    assert h is x
    _within(y, _norm64(x.double(), "rms", 1e-6)[0], _stored(_norm64(x.double(), "rms", 1e-6)[0], BF16) + 1e-5, "y")
    assert kq.block_norm(x, norm=None) == (x, None)


def test_norm_rows_of_zeros_infinities_and_nan():
    """A row of zeros gives the shift, one with an infinity or a NaN spoils only itself."""
    x = _randn(_gen(2), 6, 300)
    x[1] = 0.0
    x[3, 7] = float("inf")
    x[4, 299] = float("nan")
    shift = _randn(_gen(3), 300)
    h, y = kq.block_norm(x, torch.zeros_like(x), shift=shift, norm="layer")
    assert torch.equal(y[1], shift) and torch.equal(h[:3], x[:3]) and torch.isnan(y[3]).any() and torch.isnan(y[4]).all()
    clean = kq.block_norm(x[[0, 2, 5]].contiguous(), torch.zeros(3, 300, device="cuda"), shift=shift, norm="layer")[1]
    assert torch.equal(y[[0, 2, 5]], clean)


def test_norm_in_place_and_empty():
    g = _gen(4)
    x, res, w = _randn(g, 33, 513, dtype=BF16), _randn(g, 33, 513, dtype=BF16), _randn(g, 513, dtype=BF16)
    h, y = kq.block_norm(x, res, weight=w, norm="rms")
    h2, y2 = kq.block_norm(x, res, weight=w, norm="rms", h=res, y=x)
    assert h2 is res and y2 is x and torch.equal(h, res) and torch.equal(y, x)
    h, y = kq.block_norm(x[:0], res[:0], weight=w)
    assert h.shape == y.shape == (0, 513)


def test_norm_on_another_stream_and_in_a_graph():
    g = _gen(5)
    x, res, w = _randn(g, 64, 1152, dtype=BF16), _randn(g, 64, 1152, dtype=BF16), _randn(g, 1152, dtype=BF16)
    want = [t.clone() for t in kq.block_norm(x, res, weight=w, gate=w)]
    grads = {k: t.clone() for k, t in kq.block_norm_backward(x, want[0], x=x, weight=w, gate=w).items()}
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = kq.block_norm(x, res, weight=w, gate=w)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = kq.block_norm(x, res, weight=w, gate=w)
        back = kq.block_norm_backward(x, got[0], x=x, weight=w, gate=w)
    for _ in range(3):
        for t in (*got, *back.values()):
            t.fill_(-1.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, got))
        assert all(torch.equal(back[k], t) for k, t in grads.items())


def _backward64(dy, h, dh, x, v, norm, post, alpha, eps):
    M = dy.shape[0]
    dy, h = dy.double(), h.double()
    n, r = _norm64(h, norm, eps)
    w = v["weight"].double() if v.get("weight") is not None else torch.ones((), dtype=torch.float64, device="cuda")
    sc = 1.0 + _rows64(v["scale"], M) if v.get("scale") is not None else torch.ones_like(w)
    gt = _rows64(v["gate"], M) if v.get("gate") is not None else torch.ones_like(w)
    pw = v["post_weight"].double() if v.get("post_weight") is not None else torch.ones_like(w)

    def through(g, n, r, kind):
        t = g - n * (g * n).mean(-1, keepdim=True)
        reach = r * (g.abs() + n.abs() * (g * n).abs().mean(-1, keepdim=True) + g.abs().mean(-1, keepdim=True))
        return r * (t - g.mean(-1, keepdim=True) if kind == "layer" else t), reach

    t, reach = through(dy * w * sc, n, r, norm)
    D = t if dh is None else dh.double() + t
    reach = reach + (0.0 if dh is None else dh.double().abs())
    xn = x.double() if x is not None else torch.zeros_like(D)
    du = alpha * gt * D
    out = {"dresidual": (D, reach)}
    if post:
        xn, rx = _norm64(xn, post, eps)
        dx, xreach = through(du * pw, xn, rx, post)
        out["dx"] = (dx, xreach + through((alpha * gt * pw).abs() * reach, xn, rx, post)[1])
    else:
        out["dx"] = (du, (alpha * gt).abs() * reach)

    def over(t, v):
        """Summed over the rows that share the vector: the sum, and that of the magnitudes."""
        B = 1 if v.dim() == 1 else v.shape[0]
        return t.reshape(B, M // B, -1).sum(1).reshape(v.shape)

    # a normed value is off by its own size and, in a LayerNorm, by the mean's error over the deviation
    na = n.abs() + (r * h.abs().mean(-1, keepdim=True) if norm == "layer" else 0.0)
    xa = xn.abs() + (rx * x.double().abs().mean(-1, keepdim=True) if post == "layer" else 0.0)
    for name, term, size in (("dshift", dy, dy.abs()), ("dscale", dy * n * w, (dy * w).abs() * na),
                             ("dweight", dy * n * sc, (dy * sc).abs() * na), ("dgate", alpha * D * xn * pw, alpha * (reach * pw).abs() * xa),
                             ("dpost_weight", alpha * gt * D * xn, (alpha * gt * reach).abs() * xa)):
        if v.get(name[1:]) is not None:
            out[name] = (over(term, v[name[1:]]), over(size.expand_as(D), v[name[1:]]))
    return out


def _check_backward(M, B, d, x_dtype, s_dtype, v_dtype, norm, post, names, dh=True, alpha=0.75, eps=1e-6):
    g = _gen(77 + M + d)
    x, h = _randn(g, M, d, dtype=x_dtype), _randn(g, M, d, dtype=s_dtype)
    dy, dhv = _randn(g, M, d, dtype=x_dtype), (_randn(g, M, d, dtype=s_dtype) if dh else None)
    v = _vectors(g, B, d, v_dtype, [n for n in names if n != "post_weight" or post])
    got = kq.block_norm_backward(dy, h, dh=dhv, x=x, norm=norm, post_norm=post, alpha=alpha, eps=eps, **v)
    want = _backward64(dy, h, dhv, x, v, norm, post, alpha, eps)
    assert set(got) == set(want)
    again = kq.block_norm_backward(dy, h, dh=dhv, x=x, norm=norm, post_norm=post, alpha=alpha, eps=eps, **v)
    for k, (w, reach) in want.items():
        assert got[k].dtype == (s_dtype if k == "dresidual" else x_dtype if k == "dx" else FP32), k
        assert torch.equal(got[k], again[k]), k  # a fixed order
        # a row's sums: 64 U of what they are made of (the two passes of a post norm: twice).  A column's sum of M
        # rows in runs of at most M / 4: (M / 4 + 64) U, and the mean's error enters every row alike
        n_terms = 64 + (M / 4 if k[1:] in v else 0)
        _within(got[k], w, 4 * n_terms * U * reach + 1e-30 + _stored(w, got[k].dtype), k)


@pytest.mark.parametrize("M,B,d", [s for s in SIZES if s[2] > 1] + [(3000, 1, 300), (37, 1, 12288), (700, 700, 40)])
def test_norm_gradient_sizes(M, B, d):
    _check_backward(M, B, d, BF16, BF16, BF16, "layer" if d > 7 else "rms", None, ("shift", "scale", "gate"))
    _check_backward(M, B, d, BF16, FP32, FP32, "rms", "rms", ALL)


@pytest.mark.parametrize("x_dtype", [BF16, FP32])
@pytest.mark.parametrize("s_dtype", [BF16, FP32])
@pytest.mark.parametrize("v_dtype", [BF16, FP32])
@pytest.mark.parametrize("norm,post", [("rms", None), ("layer", "layer"), ("rms", "layer"), ("layer", "rms")])
def test_norm_gradient_types(x_dtype, s_dtype, v_dtype, norm, post):
    _check_backward(24, 3, 323, x_dtype, s_dtype, v_dtype, norm, post, ALL)


@pytest.mark.parametrize("names", [(), ("gate",), ("shift",), ("scale", "weight"), ("weight",), ("post_weight",)])
@pytest.mark.parametrize("dh", [True, False])
def test_norm_gradient_optional_vectors(names, dh):
    _check_backward(18, 3, 200, BF16, FP32, FP32, "layer", "rms" if "post_weight" in names else None, names, dh=dh)


def test_norm_gradient_without_a_factor_is_one_array():
    g = _gen(8)
    dy, h = _randn(g, 20, 96, dtype=BF16), _randn(g, 20, 96, dtype=BF16)
    got = kq.block_norm_backward(dy, h, norm="rms")
    assert got["dx"] is got["dresidual"] and set(got) == {"dx", "dresidual"}
    want, reach = _backward64(dy, h, None, None, {}, "rms", None, 1.0, 1e-6)["dresidual"]
    _within(got["dx"], want, 256 * U * reach + _stored(want, BF16), "dx")


@pytest.mark.parametrize("eps", [0.0, 1e-6])
def test_norm_gradient_of_few_rows(eps):
    """Teams of waves without a row of their own add nothing, whatever eps is."""
    _check_backward(3, 1, 100, FP32, FP32, FP32, "layer", "rms", ALL, eps=eps)


@pytest.mark.parametrize("norm,post", [("rms", None), ("layer", "rms"), ("rms", "layer")])
def test_norm_gradient_against_differences(norm, post):
    """<gradient, direction> against central differences of the forward form in 64 bits, for every input.
    Both ends of a difference are exact to 1e-16 / step = 1e-11, its curvature to step^2 = 1e-10; the
    gradient itself to 64 U of sums of magnitudes, 1e-5 of which is far above all of them."""
    M, B, d, alpha, eps, step = 12, 3, 80, 0.75, 1e-6, 1e-5
    g = _gen(9)
    x, res, dy, dh = (_randn(g, M, d) for _ in range(4))
    v = _vectors(g, B, d, FP32, [n for n in ALL if n != "post_weight" or post])
    h, _ = kq.block_norm(x, res, norm=norm, post_norm=post, alpha=alpha, eps=eps, **v)
    got = kq.block_norm_backward(dy, h, dh=dh, x=x, norm=norm, post_norm=post, alpha=alpha, eps=eps, **v)
    inputs = {"x": x, "residual": res, **v}

    def loss(t):
        hh, yy, _, _ = _forward64(t["x"], t["residual"], t, norm, post, alpha, eps)
        return float((hh * dh.double()).sum() + (yy * dy.double()).sum())

    for name, t in inputs.items():
        e = torch.randn(t.shape, generator=g, device="cuda", dtype=torch.float64)
        at = {**inputs, name: t.double() + step * e}, {**inputs, name: t.double() - step * e}
        diff = (loss(at[0]) - loss(at[1])) / (2 * step)
        grad = got["d" + name].double()
        assert abs(diff - float((grad * e).sum())) <= 1e-5 * float((grad * e).abs().sum()) + 1e-6, name


# ------------------------------------------------------------------ linear layers

E2M1 = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def _codes(g, *shape, spread=4):
    """Random MXFP4 operands [.., K]."""
    *lead, K = shape
    c = torch.randint(0, 256, (*lead, K // 2), generator=g, device="cuda", dtype=torch.uint8)
    s = torch.randint(127 - spread, 128, (*lead, K // 32), generator=g, device="cuda", dtype=torch.uint8)
    return c, s


def _values(c, s):
    nib = torch.stack([c & 15, c >> 4], -1).flatten(-2).long()
    mag = E2M1.to(c.device).double()[nib & 7]
    return torch.where(nib >= 8, -mag, mag) * torch.exp2(s.double() - 127).repeat_interleave(32, -1)


ACTS = [None, "gelu", "gelu_tanh", "silu", "relu", "swiglu"]


def _act64(p, act):
    if act == "gelu":
        return 0.5 * p * torch.special.erfc(-p / math.sqrt(2.0))
    if act == "gelu_tanh":
        return 0.5 * p * (1 + torch.tanh(math.sqrt(2 / math.pi) * (p + 0.044715 * p ** 3)))
    if act == "silu":
        return p * torch.sigmoid(p)
    if act == "relu":
        return p.clamp_min(0.0)
    if act == "swiglu":
        return p[..., 0::2] * torch.sigmoid(p[..., 0::2]) * p[..., 1::2]
    return p


def _product_and_error(a, b, bias, act):
    """act(a b^T + bias) in 64 bits, and what fp32 sums of K terms and the activation may be off."""
    K = a.shape[-1]
    p = a @ b.transpose(-1, -2)
    err = (a.abs() @ b.abs().transpose(-1, -2)) * (K + 2) * U
    if bias is not None:
        p = p + bias.double()
        err = err + 2 * U * (p.abs() + bias.double().abs())
    v = _act64(p, act)
    if act == "swiglu":
        u, w = p[..., 0::2], p[..., 1::2]
        s = u * torch.sigmoid(u)
        # |silu'| <= 1.1; the exponential's argument is rounded: |u| U more
        err = 1.1 * err[..., 0::2] * w.abs() + s.abs() * err[..., 1::2] + 1.1 * err[..., 0::2] * err[..., 1::2] + (8 + u.abs()) * U * v.abs()
    elif act in ("gelu", "gelu_tanh", "silu"):
        # slopes up to 1.13.  exp(-z) of a rounded z: z U more, z up to p^2; the fit of gelu 4e-7 = 7 U
        err = 1.13 * err + (16 + 2 * p.abs() + 2 * p.square().clamp_max(200.0)) * U * v.abs() + 1e-35
    return v, err


def _linear64(a, b, bias, act, gate, residual):
    v, err = _product_and_error(a, b, bias, act)
    if gate is not None:
        gr = _rows64(gate, v.shape[0])
        v, err = v * gr, err * gr.abs() + 2 * U * (v * gr).abs()
    if residual is not None:
        v, err = v + residual.double(), err + U * (v.abs() + residual.double().abs()) * 2
    return v, err


def _check_linear(M, N, K, act=None, bias=True, B=0, residual=False, out=BF16, vec=FP32, seed=0, strided=False):
    g = _gen(seed + 3 * M + 5 * N + K)
    a, b = _codes(g, M, K), _codes(g, N, K)
    cols = N // 2 if act == "swiglu" else N
    bv = _randn(g, N, dtype=vec) if bias else None
    gate = _randn(g, B, 2 * cols + 1, dtype=vec)[:, 1:cols + 1] if B else None
    res = _randn(g, M, cols + 3, dtype=out)[:, 2:cols + 2] if residual else None
    buf = torch.full((M, cols + 5), 7.0, dtype=out, device="cuda") if strided else None
    got = kq.mxfp4_linear(*a, *b, bias=bv, act=act, gate=gate, residual=res,
                          out=buf[:, 1:cols + 1] if strided else None, out_dtype=None if strided else out)
    want, err = _linear64(_values(*a), _values(*b), bv, act, gate, res)
    assert got.dtype == out and got.shape == (M, cols)
    _within(got, want, err + _stored(want, out) + _stored(err, out), (M, N, K, act))
    if strided:
        assert (buf[:, 0] == 7).all() and (buf[:, cols + 1:] == 7).all()


# one row, a few rows on either side of each tile's height, ragged widths, K that ends inside a step of 128 or
# 256, every tile: rows of 16 to 64, tiles that split K, pipelined tiles with scale rows of both kinds
LINEAR = [(1, 1, 32), (1, 2, 64), (1, 17, 96), (2, 130, 2016), (1, 3000, 512), (15, 64, 288), (16, 48, 256), (17, 100, 1152),
          (32, 33, 160), (33, 514, 480), (64, 1000, 4096), (65, 70, 224), (100, 600, 1024), (127, 1026, 640), (300, 3000, 96),
          (257, 2050, 544), (700, 2100, 1152), (1500, 1030, 2048), (1024, 4100, 1536), (2100, 4098, 2240), (2049, 4354, 3104)]


@pytest.mark.parametrize("M,N,K", LINEAR)
def test_linear_sizes(M, N, K):
    _check_linear(M, N, K, act="gelu", out=BF16)
    _check_linear(M, N, K, act=None, B=1, residual=True, out=FP32, vec=BF16, strided=True)
    if N % 2 == 0:
        _check_linear(M, N, K, act="swiglu", out=FP32, bias=False, strided=True)


@pytest.mark.parametrize("M,N,K", [(5, 130, 384), (48, 90, 320), (200, 330, 256), (640, 2050, 512), (2304, 2306, 2048)])
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("out", [BF16, FP32])
def test_linear_epilogues(M, N, K, act, out):
    _check_linear(M, N, K, act=act, bias=True, out=out)
    _check_linear(M, N, K, act=act, bias=False, B=1, residual=True, out=out, strided=True)
    for B in [b for b in (2, 3, M) if M % b == 0]:  # batches that end inside a tile, and one for each row
        _check_linear(M, N, K, act=act, bias=True, B=B, residual=B == 2, out=out, vec=BF16)


def test_linear_matches_the_gemm():
    """Without an epilogue: the products of mxfp4_gemm, in sums of another order at most."""
    g = _gen(11)
    a, b = _codes(g, 300, 1024), _codes(g, 515, 1024)
    want = kq.mxfp4_gemm(*a, *b)
    bound = (_values(*a).abs() @ _values(*b).abs().T) * 2 * 1024 * U
    _within(kq.mxfp4_linear(*a, *b, out_dtype=FP32), want.double(), bound, "product")


@pytest.mark.parametrize("M,N,K", [(4, 64, 256), (300, 260, 512), (2304, 2304, 1024)])
def test_linear_onto_its_residual(M, N, K):
    g = _gen(12)
    a, b, gate = _codes(g, M, K), _codes(g, N, K), _randn(g, N)
    x = _randn(g, M, N, dtype=BF16)
    want = kq.mxfp4_linear(*a, *b, gate=gate, residual=x)
    assert kq.mxfp4_linear(*a, *b, gate=gate, residual=x, out=x) is x
    assert torch.equal(x, want)


def test_linear_of_none_and_of_infinite_activations():
    """No rows, no columns; sums that overflow meet the activations' limits."""
    g = _gen(13)
    a, b = _codes(g, 4, 64), _codes(g, 6, 64)
    assert kq.mxfp4_linear(a[0][:0], a[1][:0], *b, act="silu").shape == (0, 6)
    assert kq.mxfp4_linear(*a, b[0][:0], b[1][:0], act="swiglu").shape == (4, 0)
    c = torch.full((1, 16), 0x77, dtype=torch.uint8, device="cuda")  # all 6
    neg = torch.full((1, 16), 0xff, dtype=torch.uint8, device="cuda")
    s = torch.full((1, 1), 190, dtype=torch.uint8, device="cuda")
    one = torch.full((1, 1), 254 - 60, dtype=torch.uint8, device="cuda")
    for act, low in (("relu", 0.0), ("silu", 0.0), ("gelu", 0.0)):
        big = kq.mxfp4_linear(c, s, c, one, act=act, out_dtype=FP32)
        assert float(big) > 1e38  # 32 * 36 * 2^63 * 2^67: past fp32's range or near it
        low_value = float(kq.mxfp4_linear(neg, s, c, torch.full_like(s, 127), act=act, out_dtype=FP32))
        assert low_value == low


# ------------------------------------------------------------------ grouped by expert

def _offsets(counts, lead=0):
    return torch.tensor([lead] + [lead + c for c in torch.tensor(counts).cumsum(0).tolist()], dtype=torch.int32, device="cuda")


def _check_grouped(counts, N, K, act=None, gather=True, bias=True, weighted=True, out=BF16, vec=FP32, lead=0, tail=0, strided=False):
    g = _gen(sum(counts) + N + K + len(counts))
    E, R = len(counts), sum(counts) + lead + tail
    T = max(1, R // 2 + 3) if gather else R
    a, b = _codes(g, T, K), _codes(g, E, N, K)
    rows = torch.randint(0, T, (R,), generator=g, device="cuda").to(torch.int32) if gather else None
    off = _offsets(counts, lead)
    bv = _randn(g, E, N, dtype=vec) if bias else None
    rs = _randn(g, R) if weighted else None
    cols = N // 2 if act == "swiglu" else N
    buf = torch.full((R, cols + (7 if strided else 0)), 7.0, dtype=out, device="cuda")
    got = kq.mxfp4_grouped_linear(*a, *b, off, rows=rows, bias=bv, act=act, row_scale=rs, out=buf[:, 3:cols + 3] if strided else buf)
    av = _values(*a)
    at = lead
    for e, n in enumerate(counts):
        r = slice(at, at + n)
        at += n
        if not n:
            continue
        want, err = _product_and_error(av[rows[r].long()] if gather else av[r], _values(b[0][e], b[1][e]), None if bv is None else bv[e], act)
        if weighted:
            want, err = want * rs[r].double()[:, None], (err + 2 * U * want.abs()) * rs[r].double().abs()[:, None]
        _within(got[r], want, err + _stored(want, out) + _stored(err, out), ("expert", e))
    assert (got[:lead] == 7).all() and (got[at:] == 7).all()
    if strided:
        assert (buf[:, :3] == 7).all() and (buf[:, cols + 3:] == 7).all()


# experts with no rows (first, last, all but one), one row, ends at and beside the tiles' heights, more experts than
# a wave has lanes, one expert
GROUPS = [[1], [0, 3, 0], [0, 0, 0, 5], [16, 15, 17, 0, 33], [1] * 70, [0] * 64 + [2, 0, 1], [64, 65, 63], [100, 0, 28, 200],
          [128, 129, 1, 0, 300, 127], [700, 3, 0, 1100], [5] * 130]


@pytest.mark.parametrize("counts", GROUPS, ids=lambda c: f"{len(c)}x{sum(c)}")
@pytest.mark.parametrize("K", [288, 1024])
def test_grouped_sizes(counts, K):
    _check_grouped(counts, 130, K, act="swiglu", out=BF16)
    _check_grouped(counts, 65, K, act=None, gather=False, out=FP32, vec=BF16, strided=True)


@pytest.mark.parametrize("counts", [[300, 0, 513, 900], [1500, 900, 1700, 0]])
@pytest.mark.parametrize("N,K", [(1100, 2048), (1030, 1184), (2306, 3104), (2304, 1920)])
@pytest.mark.parametrize("gather", [True, False])
def test_grouped_large(counts, N, K, gather):
    _check_grouped(counts, N, K, act="gelu_tanh", gather=gather, out=BF16)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("counts", [[3, 0, 9], [40, 70, 90], [400, 0, 300]])
def test_grouped_epilogues(act, counts):
    _check_grouped(counts, 66, 320, act=act, bias=False, weighted=False, out=FP32)
    _check_grouped(counts, 66, 320, act=act, gather=False, vec=BF16, out=BF16)


@pytest.mark.parametrize("counts", [[2, 0, 1], [130, 0, 300], [1500, 900]])
def test_grouped_leaves_rows_without_a_group(counts):
    _check_grouped(counts, 130, 256, lead=5, tail=300)
    _check_grouped([0] * len(counts), 130, 256, tail=sum(counts))


@pytest.mark.parametrize("R", [8, 400, 3000])
def test_grouped_takes_bad_offsets_and_rows_as_the_nearest(R):
    """Offsets past the rows, negative or decreasing, and rows past the tokens, stay inside the arrays."""
    g = _gen(14)
    E, N, K, T = 4, 128, 256, 50
    a, b = _codes(g, T, K), _codes(g, E, N, K)
    rows = torch.randint(0, T, (R,), generator=g, device="cuda").to(torch.int32)
    off = torch.tensor([0, R // 2, R // 2, R, R], dtype=torch.int32, device="cuda")
    want = kq.mxfp4_grouped_linear(*a, *b, off, rows=rows)
    bad = torch.tensor([-5, R // 2, R // 2 - 3, R + 1000, R + 7], dtype=torch.int32, device="cuda")
    bad_want = torch.tensor([0, R // 2, R // 2, R, R], dtype=torch.int32, device="cuda")
    far = rows.clone()
    far[rows == T - 1] = 2 ** 31 - 1
    far[rows == 0] = -9
    got = kq.mxfp4_grouped_linear(*a, *b, bad_want, rows=far)
    assert torch.equal(got, want)
    out = torch.zeros((R, N), dtype=BF16, device="cuda")
    kq.mxfp4_grouped_linear(*a, *b, bad, rows=rows, out=out)  # expert 2 has R // 2 - 3 .. R, after expert 0
    torch.cuda.synchronize()
    assert torch.equal(out[:R // 2 - 3], want[:R // 2 - 3]) and torch.equal(out[R // 2:], want[R // 2:])


def test_grouped_of_none():
    g = _gen(15)
    a, b = _codes(g, 4, 64), _codes(g, 3, 6, 64)
    off = torch.zeros(4, dtype=torch.int32, device="cuda")
    assert kq.mxfp4_grouped_linear(a[0][:0], a[1][:0], *b, off).shape == (0, 6)
    assert kq.mxfp4_grouped_linear(*a, *b, off, rows=off[:0]).shape == (0, 6)


@pytest.mark.parametrize("counts", [[3, 0, 4], [200, 0, 150]])
def test_linear_layers_in_a_graph(counts):
    """Replays with other offsets in the same buffer, and the eager call between them."""
    g = _gen(16)
    R, N, K = sum(counts), 256, 512
    a, b = _codes(g, R, K), _codes(g, 3, N, K)
    off = _offsets(counts)
    graph = torch.cuda.CUDAGraph()
    kq.mxfp4_grouped_linear(*a, *b, off)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        got = kq.mxfp4_grouped_linear(*a, *b, off, act="silu")
        one = kq.mxfp4_linear(*a, b[0][0], b[1][0], act="silu")
    for c in (counts, counts[::-1], [R, 0, 0], [0, 1, R - 1]):
        off.copy_(_offsets(c))
        want, want1 = kq.mxfp4_grouped_linear(*a, *b, off, act="silu"), kq.mxfp4_linear(*a, b[0][0], b[1][0], act="silu")
        got.zero_()
        one.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want) and torch.equal(one, want1)


def test_linear_past_32_bit_offsets():
    """Outputs beyond 2^31 elements and expert weights beyond 2^32 bytes of codes."""
    g = _gen(17)
    M, N, K = 70000, 32000, 64
    a, b = _codes(g, M, K), _codes(g, N, K)
    out = kq.mxfp4_linear(*a, *b, act="relu")
    av, bv = _values(*a), _values(*b)
    for r in (slice(0, 8), slice(M - 300, M)):
        want, err = _linear64(av[r], bv, None, "relu", None, None)
        _within(out[r], want, err + _stored(want, BF16), "rows")
    del out
    E, N, K = 9, 65536, 16384  # 4.5 GiB of codes
    b = torch.empty((E, N, K // 2), dtype=torch.uint8, device="cuda"), torch.full((E, N, K // 32), 125, dtype=torch.uint8, device="cuda")
    for e in range(E):
        b[0][e] = torch.randint(0, 256, (N, K // 2), generator=g, device="cuda", dtype=torch.uint8)
    a = _codes(g, 3, K)
    rows = torch.tensor([2, 0, 1, 1], dtype=torch.int32, device="cuda")
    out = kq.mxfp4_grouped_linear(*a, *b, _offsets([1, 0, 0, 0, 0, 0, 0, 0, 3]), rows=rows, out_dtype=FP32)
    av = _values(*a)
    for r, e in ((0, 0), (1, 8), (2, 8), (3, 8)):
        w = _values(b[0][e, N - 100:], b[1][e, N - 100:])
        want, err = _product_and_error(av[rows[r:r + 1].long()], w, None, None)
        _within(out[r:r + 1, N - 100:], want, err, "expert")


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("M,N", [(1, 20), (200, 260), (2304, 2304)])
def test_linear_keeps_nan(act, M, N):
    """A NaN in the bias comes out in its column, and in no other."""
    g = _gen(18)
    bias = _randn(g, N)
    bias[2] = float("nan")
    out = kq.mxfp4_linear(*_codes(g, M, 256), *_codes(g, N, 256), bias=bias, act=act)
    assert torch.isnan(out[:, 1 if act == "swiglu" else 2]).all() and int(torch.isnan(out).sum()) == M


def test_grouped_bad_offsets_of_many_experts():
    """Offsets that go up and down over more than 64 experts ask for more tiles than a call launches: it ends, and
    writes nothing outside the output."""
    g = _gen(19)
    E, R, N, K = 200, 3000, 64, 64
    a, b = _codes(g, R, K), _codes(g, E, N, K)
    off = torch.zeros(E + 1, dtype=torch.int32, device="cuda")
    off[1::2] = R
    out = torch.full((R + 1, N), 7.0, dtype=BF16, device="cuda")
    kq.mxfp4_grouped_linear(*a, *b, off, out=out[:R])
    torch.cuda.synchronize()
    assert (out[R] == 7.0).all() and torch.isfinite(out[:R]).all()
