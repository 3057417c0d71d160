"""The operators of a generation step against plain forms in 64 bits: rope and its
gradient, the paged cache, attention over it, w4a16_linear, at the sizes, types,
masks and layouts where they can go wrong.

Tolerances follow from the arithmetic.  U = 2^-24 (fp32), one rounding to bf16
is 2^-8 of the result (8 significant bits).  A sum of n fp32 terms in any order,
each addition rounded to nearest or cut, is within 2 n U of the sum of magnitudes."""
import math

import pytest

torch = pytest.importorskip("torch")
kq = pytest.importorskip("paper_2607_21446_amd")

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
BF16, FP32 = torch.bfloat16, torch.float32
FORMATS = ["bf16", "mxfp8", "mxfp4"]


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


# ------------------------------------------------------------------ rope

def _rope64(x, positions, axes, theta, pairing, freqs, backward):
    """The rotated rows, and the magnitudes that their errors go by."""
    n = sum(axes) // 2
    f, axis = [], []
    for a, d in enumerate(axes):
        f += [theta ** (-2.0 * i / d) for i in range(d // 2)]
        axis += [a] * (d // 2)
    f = torch.tensor(f, dtype=torch.float64, device="cuda") if freqs is None else freqs
    w = (positions.double()[:, axis] * f).unsqueeze(1)
    c, s = torch.cos(w), torch.sin(w) * (-1 if backward else 1)
    x = x.double()
    i = torch.arange(n, device="cuda")
    a, b = (2 * i, 2 * i + 1) if pairing == "pairs" else (i, i + n)
    out, size = x.clone(), torch.zeros_like(x)
    out[..., a], out[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
    size[..., a] = size[..., b] = x[..., a].abs() + x[..., b].abs()
    return out, size


def _positions(g, T, n, dtype, most=1000000):
    p = torch.randint(-most // 8, most, (T, n), generator=g, device="cuda")
    return p.to(dtype) if dtype != FP32 else p.float() * 0.37


def _check_rope(T, H, D, axes, pairing="pairs", dtype=BF16, pos=torch.int32, theta=10000.0, freqs=None, x=None, backward=False, seed=0):
    g = _gen(seed + T + 3 * H + 7 * D)
    x = _randn(g, T, H, D, dtype=dtype) if x is None else x
    p = _positions(g, T, len(axes), pos)
    call = kq.rope_backward if backward else kq.rope
    got = call(x, p, axes, theta=theta, pairing=pairing, freqs=freqs)
    want, size = _rope64(x, p, axes, theta, pairing, freqs, backward)
    # cos and sin to 4 U, two products and their difference rounded: 3 U more
    _within(got, want, 7 * U * size + _stored(want, dtype) + _stored(7 * U * size, dtype), (T, H, D, axes, pairing))
    n = sum(axes)
    assert torch.equal(got[..., n:], x[..., n:])
    return got


@pytest.mark.parametrize("T,H,D,axes", [
    (1, 1, 2, [2]), (1, 40, 128, [128]), (3, 1, 64, [32]), (5, 7, 80, [16, 24, 24]), (17, 2, 66, [2, 4, 6, 8]), (130, 3, 72, [24, 24, 24]),
    (1, 70, 256, [8, 8]), (300, 5, 6, [2, 2]), (2049, 3, 128, [16, 56, 56]), (1100, 1, 1024, [512, 512]), (4, 600, 96, [96])])
@pytest.mark.parametrize("pairing", ["pairs", "halves"])
@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_rope_sizes(T, H, D, axes, pairing, dtype):
    for pos in (torch.int32, torch.int64, FP32):
        _check_rope(T, H, D, axes, pairing, dtype, pos)
    _check_rope(T, H, D, axes, pairing, dtype, backward=True, theta=500000.0)


def test_rope_strides_and_alignment():
    g = _gen(1)
    for dtype in (BF16, FP32):
        qkv = _randn(g, 9, 6, 64, dtype=dtype)
        _check_rope(9, 4, 64, [32, 32], dtype=dtype, x=qkv[:, :4])  # heads of a fused projection
        odd = _randn(g, 9, 4, 67, dtype=dtype)
        for pairing in ("pairs", "halves"):
            _check_rope(9, 4, 64, [40, 24], pairing, dtype=dtype, x=odd[:, :, 3:])  # rows that start anywhere
            _check_rope(9, 4, 64, [64], pairing, dtype=dtype, x=_randn(g, 4, 9, 64, dtype=dtype).transpose(0, 1))  # heads first
            _check_rope(9, 4, 64, [64], pairing, dtype=dtype, x=_randn(g, 9, 1, 64, dtype=dtype).expand(9, 4, 64))  # one head for all


def test_rope_in_place_and_into_slices():
    g = _gen(2)
    p = _positions(g, 33, 2, torch.int32)
    for D, axes in ((64, [32, 16]), (66, [30, 20])):
        for pairing in ("pairs", "halves"):
            x = _randn(g, 33, 5, D, dtype=BF16)
            want = kq.rope(x, p, axes, pairing=pairing)
            fused = _randn(g, 33, 8, D, dtype=BF16)
            keep = fused.clone()
            assert kq.rope(x, p, axes, pairing=pairing, out=fused[:, 2:7]).data_ptr() == fused[:, 2:7].data_ptr()
            assert torch.equal(fused[:, 2:7], want) and torch.equal(fused[:, :2], keep[:, :2]) and torch.equal(fused[:, 7:], keep[:, 7:])
            assert kq.rope(x, p, axes, pairing=pairing, out=x) is x and torch.equal(x, want)
            view = fused[:, 1:6]
            again = kq.rope(view, p, axes, pairing=pairing)
            kq.rope(view, p, axes, pairing=pairing, out=view)
            assert torch.equal(view, again)


def test_rope_frequencies_and_positions():
    g = _gen(3)
    freqs = torch.rand(24, generator=g, device="cuda", dtype=torch.float64) * 3
    _check_rope(50, 3, 64, [32, 16], freqs=freqs, dtype=FP32)
    _check_rope(50, 3, 64, [32, 16], "halves", freqs=freqs, dtype=FP32, pos=FP32)
    x = _randn(g, 50, 3, 64)
    p = torch.arange(100, device="cuda")
    want = kq.rope(x, p[::2].reshape(50, 1).contiguous(), [64])
    assert torch.equal(kq.rope(x, p[::2], 64), want)  # one axis: positions in one dimension, at any stride
    table = torch.arange(150, device="cuda", dtype=torch.int32).reshape(50, 3)
    assert torch.equal(kq.rope(x, table[:, :2], [32, 32]), kq.rope(x, table[:, :2].contiguous(), [32, 32]))
    # far and negative positions; zero is no rotation
    far = torch.full((50,), 2 ** 31 - 1, dtype=torch.int64, device="cuda")
    want, size = _rope64(x, far[:, None], [64], 1e4, "pairs", None, False)
    # an angle of 2^31 f from 64-bit f: both sides within 2^31 2^-49
    _within(kq.rope(x, far, 64), want, (7 * U + 2.0 ** -18) * size, "far")
    assert torch.equal(kq.rope(x, torch.zeros(50, dtype=torch.int32, device="cuda"), 64), x)


def test_rope_of_none_and_of_infinite_values():
    x = torch.zeros((4, 3, 8), device="cuda")
    p = torch.ones((4, 1), dtype=torch.int32, device="cuda")
    assert kq.rope(x[:0], p[:0], [8]).shape == (0, 3, 8) and kq.rope(x[:, :0], p, [8]).shape == (4, 0, 8)
    x[0, 0, 6:] = math.inf
    x[1, 1, 7] = math.nan
    y = kq.rope(x, p, [6])
    assert torch.isfinite(y[..., :6]).all() and torch.equal(y[0, 0, 6:], x[0, 0, 6:]) and torch.isnan(y[1, 1, 7])


@pytest.mark.parametrize("pairing", ["pairs", "halves"])
def test_rope_gradient(pairing):
    """Against differences of the forward call, which is linear: they are exact but for rounding."""
    g = _gen(4)
    T, H, D, axes = 7, 3, 40, [12, 20]
    p, x, dy = _positions(g, T, 2, torch.int32), _randn(g, T, H, D), _randn(g, T, H, D)
    dx = kq.rope_backward(dy, p, axes, pairing=pairing)
    for _ in range(8):
        e = _randn(g, T, H, D)
        up, down = (kq.rope(x + s * e, p, axes, pairing=pairing).double() for s in (0.5, -0.5))
        diff = ((up - down) * dy.double()).sum()
        grad = (dx.double() * e.double()).sum()
        # x +- e / 2 rounded, and two rotations: 20 U of the magnitudes' products
        assert abs(float(diff - grad)) <= 20 * U * float((dy.abs().double() * (x.abs() + e.abs()).double() * 2).sum())
    assert kq.rope_backward(dy, p, axes, pairing=pairing, dx=dy) is dy and torch.equal(dy, dx)


def test_rope_refusals():
    g = _gen(5)
    x, p = _randn(g, 8, 4, 64), _positions(g, 8, 1, torch.int32)
    for bad in (lambda: kq.rope(x[0], p, [64]), lambda: kq.rope(x.transpose(1, 2), p, [4]), lambda: kq.rope(x, p[:7], [64]),
                lambda: kq.rope(x, p, [32, 32]), lambda: kq.rope(x, p.cpu(), [64]), lambda: kq.rope(x, p, [64], out=x[:7]),
                lambda: kq.rope(x, p, [64], out=x.expand(8, 4, 64)[:, :1].expand(8, 4, 64)),
                lambda: kq.rope(x[1:], p[1:], [64], out=x[:-1]), lambda: kq.rope(x, p, [64], freqs=torch.ones(31, dtype=torch.float64, device="cuda"))):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: kq.rope(x.half(), p, [64]), lambda: kq.rope(x, p.short(), [64]), lambda: kq.rope(x, p, [64], out=x.bfloat16()),
                lambda: kq.rope(x, p, [64], freqs=torch.ones(32, device="cuda"))):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: kq.rope(x, p, [63]), lambda: kq.rope(x, p, [66]), lambda: kq.rope(x, p, [64], theta=0.0), lambda: kq.rope(x, p, [0]),
                lambda: kq.rope(x, p, 2 ** 32 + 64), lambda: kq.rope(x, p, [2 ** 32 + 64]), lambda: kq.rope(x, p, [2 ** 70])):
        with pytest.raises((kq.KQError, ValueError)):
            bad()


# ------------------------------------------------------------------ the cache

E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _nearest(x, form):
    """The values that a cache holds for x [.., d], in 64 bits: nearest, ties to the even code."""
    if form == "bf16":
        return x.to(BF16).double()
    v = x.double().unflatten(-1, (-1, 32))
    amax = v.abs().amax(-1, keepdim=True)
    e = torch.floor(torch.log2(amax.clamp_min(1e-300)))
    unit = torch.exp2((e - (2 if form == "mxfp4" else 8)).clamp_min(-127))
    m = (v / unit).abs()
    if form == "mxfp8":
        step = torch.exp2(torch.floor(torch.log2(m.clamp_min(2.0 ** -6))) - 3)
        q = (torch.round(m / step) * step).clamp_max(448.0)
    else:
        grid = torch.tensor(E2M1, dtype=torch.float64, device=x.device)
        edge = (grid[1:] + grid[:-1]) / 2
        odd = torch.arange(7, device=x.device) % 2  # a tie with an odd code below goes up
        q = grid[((m.unsqueeze(-1) > edge) | ((m.unsqueeze(-1) == edge) & (odd == 1))).sum(-1)]
    return (torch.copysign(q, v) * unit).flatten(-2)


def _held(cache):
    """What a cache's arrays stand for, in 64 bits, [pages, heads, page_size, d], by their bits."""
    out = []
    for t, s in ((cache.k, cache.k_scales), (cache.v, cache.v_scales)):
        if s is None:
            out.append(t.double())
            continue
        if cache.format == "mxfp4":
            c = torch.stack([t & 15, t >> 4], -1).flatten(-2).long()
            v = torch.tensor(E2M1, dtype=torch.float64, device=t.device)[c & 7] * torch.where(c >= 8, -1.0, 1.0).double()
        else:
            c = t.long()
            e, m = c >> 3 & 15, (c & 7).double()
            v = torch.where(e > 0, (1 + m / 8) * torch.exp2(e.double() - 7), m * 2.0 ** -9) * torch.where(c >= 128, -1.0, 1.0).double()
        out.append(v * torch.exp2(s.double() - 127).repeat_interleave(32, -1))
    return out


def _at(held, slots, size):
    return held[slots // size, :, slots % size]


@pytest.mark.parametrize("T,pages,size,H,d", [(1, 1, 16, 1, 32), (5, 3, 16, 2, 64), (40, 7, 32, 3, 96), (130, 4, 64, 8, 128), (300, 3, 128, 1, 160),
                                             (33, 2, 256, 5, 256), (2, 1, 16, 700, 64)])
@pytest.mark.parametrize("form", FORMATS)
@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_cache_write_and_read(T, pages, size, H, d, form, dtype):
    g = _gen(T + d)
    T = min(T, pages * size)
    cache = kq.kv_cache(pages, size, H, d, format=form)
    kv = _randn(g, T, 2, H, d) * torch.exp2(torch.randint(-20, 20, (T, 2, H, 1), generator=g, device="cuda").float())
    kv[..., :7] *= 30.0
    kv = kv.to(dtype)
    slots = torch.randperm(pages * size, generator=g, device="cuda")[:T]
    assert kq.kv_cache_write(cache, kv[:, 0], kv[:, 1], slots) is cache
    want = [_nearest(kv[:, i], form) for i in range(2)]
    held = _held(cache)
    for i in range(2):
        assert torch.equal(_at(held[i], slots, size), want[i])
        rest = held[i].transpose(1, 2).reshape(pages * size, H, d).clone()
        rest[slots] = 0
        assert not rest.any()  # nothing but the slots was written
    for out in (None, BF16, FP32):
        got = kq.kv_cache_read(cache, slots, out_dtype=out)
        for i in range(2):
            assert got[i].dtype == (out or BF16) and torch.equal(got[i].double(), want[i])


@pytest.mark.parametrize("form", ["mxfp8", "mxfp4"])
def test_cache_rounding(form):
    """Every border between two elements and its neighbours, in blocks of every scale down to the smallest."""
    top = 6.0 if form == "mxfp4" else 448.0
    if form == "mxfp4":
        grid = torch.tensor(E2M1, dtype=torch.float64)
    else:
        grid = torch.unique(torch.cat([torch.arange(8) * 2.0 ** -9, ((1 + torch.arange(8) / 8) * torch.exp2(torch.arange(-6.0, 9)[:, None])).flatten()])).double()
        grid = grid[grid <= 448]
    edge = (grid[1:] + grid[:-1]) / 2
    v = torch.cat([grid, edge, edge * (1 + 2.0 ** -20), edge * (1 - 2.0 ** -20), torch.tensor([7.5, 7.99] if form == "mxfp4" else [464.0, 465.0, 511.0])])
    v = torch.cat([v, -v])
    v = torch.nn.functional.pad(v, (0, -len(v) % 31)).reshape(-1, 31)
    lead = torch.full((len(v), 1), 4.0 if form == "mxfp4" else 256.0).double()  # the binade of the largest
    lead = torch.where(v.abs().amax(1, keepdim=True) > lead, lead, lead)
    block = torch.cat([lead, v], 1)
    block = block[block.abs().amax(1) < 2 * lead[:, 0]]
    shifts = torch.tensor([0, 1, -5, 60, 100, -60, -100, -110], dtype=torch.float64)
    x = (block[None] * torch.exp2(shifts)[:, None, None]).reshape(-1, 1, 32).float().cuda()
    assert x.abs().max() >= top
    cache = kq.kv_cache(-(-len(x) // 16), 16, 1, 32, format=form)
    slots = torch.arange(len(x), device="cuda")
    kq.kv_cache_write(cache, x, -x, slots)
    held = _held(cache)
    want = _nearest(x, form)
    assert torch.equal(_at(held[0], slots, 16), want) and torch.equal(_at(held[1], slots, 16), -want)
    k, _ = kq.kv_cache_read(cache, slots, out_dtype=FP32)
    assert torch.equal(k.double(), want)


def test_cache_zeros_and_tiny_blocks():
    for form in ("mxfp8", "mxfp4"):
        cache = kq.kv_cache(1, 16, 1, 64, format=form)
        x = torch.zeros((2, 1, 64), device="cuda")
        x[1, 0, 40] = 2.0 ** -126  # the smallest normal: scale byte 0, in units of 2^-127
        kq.kv_cache_write(cache, x, x, torch.tensor([3, 5], device="cuda"))
        held = _held(cache)[0][0, 0]
        assert not held[3].any() and float(held[5, 40]) == 2.0 ** -126 and int((held[5] != 0).sum()) == 1
        assert not cache.k_scales[0, 0, 3].any()


def test_cache_matches_the_quantizer():
    """MXFP4 codes and scales are those of the library's quantizer."""
    g = _gen(9)
    k = _randn(g, 48, 4 * 128, dtype=BF16)
    codes, scales = kq.mxfp4(k)
    cache = kq.kv_cache(3, 16, 4, 128)
    kq.kv_cache_write(cache, k.reshape(48, 4, 128), k.reshape(48, 4, 128), torch.arange(48, device="cuda"))
    assert torch.equal(cache.k.transpose(1, 2).reshape(48, -1), codes) and torch.equal(cache.v_scales.transpose(1, 2).reshape(48, -1), scales)


@pytest.mark.parametrize("form", FORMATS)
def test_cache_slots_outside_and_layouts(form):
    g = _gen(10)
    H, d, size, pages = 3, 96, 16, 4
    cache = kq.kv_cache(pages, size, H, d, format=form)
    cap = pages * size
    slots = torch.tensor([0, -1, cap, cap - 1, 2 ** 62, -2 ** 63, 17, 2 ** 31, 2 ** 32 + 5], device="cuda")
    fused = _randn(g, 9, 3 * H * d + 1, dtype=BF16)[:, 1:]  # rows that start at odd elements
    k, v = fused[:, :H * d].unflatten(1, (H, d)), fused[:, H * d:2 * H * d].unflatten(1, (H, d))
    kq.kv_cache_write(cache, k, v, slots)
    inside = [i for i, s in enumerate(slots.tolist()) if 0 <= s < cap]
    for t, held in zip((k, v), _held(cache)):
        want = torch.zeros((cap, H, d), dtype=torch.float64, device="cuda")
        want[slots[inside]] = _nearest(t[inside], form)
        assert torch.equal(held.transpose(1, 2).reshape(cap, H, d), want)
    for got, t in zip(kq.kv_cache_read(cache, slots), (k, v)):
        want = torch.zeros((9, H, d), dtype=torch.float64, device="cuda")
        want[inside] = _nearest(t[inside], form)
        assert torch.equal(got.double(), want)
    # heads first, and one token's values for all; the same slot may be read twice
    kt = _randn(g, H, 9, d)
    kq.kv_cache_write(cache, kt.transpose(0, 1), kt[:, :1].transpose(0, 1).expand(9, H, d), torch.arange(9, device="cuda"))
    twice = torch.tensor([8, 2, 8], device="cuda")
    got = kq.kv_cache_read(cache, twice, out_dtype=FP32)
    assert torch.equal(got[0].double(), _nearest(kt.transpose(0, 1)[twice], form)) and torch.equal(got[1][0], got[1][1])
    a, b = torch.empty((3, H, d), device="cuda"), torch.empty((3, H, d), device="cuda")
    assert kq.kv_cache_read(cache, twice, k=a, v=b)[0] is a and torch.equal(a, got[0]) and torch.equal(b, got[1])
    none = torch.empty(0, dtype=torch.int64, device="cuda")
    assert kq.kv_cache_write(cache, k[:0], v[:0], none) is cache and kq.kv_cache_read(cache, none)[0].shape == (0, H, d)


def test_cache_refusals():
    cache = kq.kv_cache(2, 16, 2, 64)
    x, slots = torch.zeros((4, 2, 64), device="cuda"), torch.arange(4, device="cuda")
    for bad in (lambda: kq.kv_cache_write(cache, x[:3], x, slots), lambda: kq.kv_cache_write(cache, x, x[:, :1], slots),
                lambda: kq.kv_cache_write(cache, x, x.transpose(1, 2).contiguous().transpose(1, 2), slots),
                lambda: kq.kv_cache_write(cache, x, x, slots.cpu()), lambda: kq.kv_cache_write(cache, x, x, slots[None]),
                lambda: kq.kv_cache_read(cache, slots, k=x[:3]), lambda: kq.kv_cache_read(cache, slots[:, None]),
                lambda: kq.kv_cache_read(cache._replace(v=cache.v[:1]), slots), lambda: kq.kv_cache_read(cache._replace(k=cache.k[..., :7]), slots)):
        with pytest.raises((ValueError, TypeError)):
            bad()
    for bad in (lambda: kq.kv_cache_write(cache, x, x.bfloat16(), slots), lambda: kq.kv_cache_write(cache, x.half(), x.half(), slots),
                lambda: kq.kv_cache_write(cache, x, x, slots.int()), lambda: kq.kv_cache_read(cache, slots, out_dtype=torch.float16),
                lambda: kq.kv_cache_read(cache._replace(k_scales=None, v_scales=None), slots), lambda: kq.kv_cache_read(list(cache), slots)):
        with pytest.raises((TypeError, ValueError)):
            bad()


def test_cache_read_into_one_array():
    g = _gen(14)
    cache = kq.kv_cache(2, 16, 2, 64)
    x, slots = _randn(g, 6, 2, 64, dtype=BF16), torch.arange(3, device="cuda")
    kq.kv_cache_write(cache, x[:3], x[3:], slots)
    want = kq.kv_cache_read(cache, slots)
    both = torch.empty_like(x)
    got = kq.kv_cache_read(cache, slots, k=both[3:], v=both[:3])  # apart
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and got[0].data_ptr() == both[3:].data_ptr()
    for k, v in ((both[:3], both[:3]), (both[:3], both[1:4]), (both[2:5], both[:3])):
        with pytest.raises(ValueError, match="overlap"):
            kq.kv_cache_read(cache, slots, k=k, v=v)


# ------------------------------------------------------------------ attention

def _filled(g, pages, size, H, d, form):
    cache = kq.kv_cache(pages, size, H, d, format=form)
    kv = _randn(g, pages * size, 2, H, d)
    kv[:, 0, :, : d // 8] *= 2.0
    kv[:, 1] += 0.5
    kq.kv_cache_write(cache, kv[:, 0], kv[:, 1], torch.arange(pages * size, device="cuda"))
    return cache


def _attn64(q, cache, table, lengths, scale, window):
    """out, lse, and what they may be off."""
    B, Hq, d = q.shape
    pages, H, size, _ = cache.k.shape
    K, V = _held(cache)
    out = torch.zeros((B, Hq, d), dtype=torch.float64, device="cuda")
    lse = torch.full((B, Hq), -math.inf, dtype=torch.float64, device="cuda")
    err, lerr = torch.zeros_like(out), torch.zeros_like(lse)
    wide = q.dtype == FP32
    for b in range(B):
        n = min(max(int(lengths[b]), 0), table.shape[1] * size)
        at = torch.arange(max(0, n - window) if window else 0, n, device="cuda")
        if not len(at):
            continue
        p = table[b].long().clamp(0, pages - 1)[at // size]
        k, v = (t[p, :, at % size].transpose(0, 1).repeat_interleave(Hq // H, 0) for t in (K, V))  # [Hq, n, d]
        s = (q[b].double().unsqueeze(1) * k).sum(-1) * scale
        mag = (q[b].double().abs().unsqueeze(1) * k.abs()).sum(-1) * abs(scale)
        w = torch.softmax(s, -1).unsqueeze(-1)
        lse[b] = torch.logsumexp(s, -1)
        out[b] = (w * v).sum(1)
        # a score's sum of d terms (three of each in 32 bits), its scale and the exponent's argument; p as two terms in
        # 16 bits, three in 32; the sums over n tokens, and a factor each time the maximum moves (once in 32 tokens)
        ds = ((2 * (3 if wide else 1) * d + 8) * U * mag + 4 * U * s.abs()).amax(-1)
        dp = 2 * ds + (2 * len(at) + 2 * len(at) / 32 + 40) * 2 * U + (3 * U if wide else 2.0 ** -16)
        err[b] = dp[:, None] * (w * v.abs()).sum(1)
        lerr[b] = ds + (2 * len(at) + len(at) / 32 + 20) * 2 * U + 4 * U * lse[b].abs()
    return out, lse, err, lerr


def _check_attn(form, B, H, G, d, size, lengths, dtype=BF16, window=None, scale=None, seed=0, spare=2, **kw):
    g = _gen(seed + B + 7 * H + 11 * d + G)
    each = max(1, -(-max(max(lengths), 1) // size))
    cache = kw.pop("cache", None) or _filled(g, B * each + spare, size, H, d, form)
    table = torch.randperm(B * each + spare, generator=g, device="cuda")[: B * each].reshape(B, each).to(torch.int32)
    n = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    q = kw.pop("q", None)
    q = _randn(g, B, H * G, d, dtype=dtype) * 1.5 if q is None else q
    got, lse = kq.paged_attention(q, cache, table, n, scale=scale, window=window, want_lse=True, **kw)
    want, wl, err, lerr = _attn64(q, cache, table, n, d ** -0.5 if scale is None else scale, window)
    assert got.dtype == q.dtype and got.shape == q.shape
    _within(got, want, err + _stored(want, q.dtype) + _stored(err, q.dtype), (form, B, H, G, d, lengths))
    empty = torch.isinf(wl)
    assert torch.equal(torch.isinf(lse), empty) and not got[empty].any()
    _within(lse[~empty], wl[~empty], lerr[~empty], "lse")
    return got, lse, (q, cache, table, n)


# on either side of a quarter of a tile, a tile, a page, a part; empty
LENGTHS = [1, 0, 7, 8, 9, 16, 17, 31, 32, 33, 127, 128, 129, 500]


@pytest.mark.parametrize("form", FORMATS)
@pytest.mark.parametrize("d", [32, 64, 96, 128, 160, 192, 224, 256])
@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_attention_columns(form, d, dtype):
    _check_attn(form, 14, 2, 3, d, 16, LENGTHS, dtype)


@pytest.mark.parametrize("form", FORMATS)
@pytest.mark.parametrize("H,G", [(1, 1), (1, 16), (1, 17), (3, 5), (2, 33), (8, 4), (18, 1)])
@pytest.mark.parametrize("size", [16, 32, 128])
def test_attention_heads_and_pages(form, H, G, size):
    _check_attn(form, 3, H, G, 64, size, [200, 1, 333])


@pytest.mark.parametrize("form", FORMATS)
@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("window", [1, 5, 32, 33, 100, 1000])
def test_attention_windows(form, dtype, window):
    _check_attn(form, 6, 2, 2, 128, 16, [1, 0, 64, 97, 130, 700], dtype, window=window)


@pytest.mark.parametrize("form", FORMATS)
@pytest.mark.parametrize("B,H,n", [(1, 1, 30000), (2, 8, 9001), (70, 1, 600), (5, 16, 3000)])
def test_attention_long_and_split(form, B, H, n):
    """Sequences of many parts, alone and beside short and empty ones."""
    lengths = [n] + [(7919 * i * i) % (n + 1) for i in range(1, B)]
    lengths[-1] = n if B == 1 else 0
    _check_attn(form, B, H, 4, 64, 64, lengths)
    _check_attn(form, B, H, 1, 64, 64, lengths, FP32, window=n // 2)


def test_attention_one_part_a_sequence():
    """A table too short for parts: no second launch."""
    _check_attn("mxfp4", 3, 2, 4, 128, 64, [128, 65, 0])
    _check_attn("bf16", 2, 1, 4, 128, 16, [1, 2])


def test_attention_scales_and_peaks():
    _check_attn("bf16", 3, 2, 4, 64, 16, [100, 300, 5], scale=0.0)
    _check_attn("mxfp4", 3, 2, 4, 64, 16, [100, 300, 5], scale=-0.3)
    _check_attn("mxfp8", 3, 2, 4, 64, 16, [100, 300, 5], scale=4.0)  # nearly one token's value
    _check_attn("bf16", 2, 2, 4, 64, 16, [100, 3000], FP32, scale=3.0)


@pytest.mark.parametrize("form", FORMATS)
@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_attention_does_not_see_what_is_masked(form, dtype):
    """NaN and infinities behind the sequences' ends, before their windows, in other pages; pages past the end in the table
    that do not exist."""
    g = _gen(21)
    B, H, G, d, size, each = 4, 2, 3, 128, 16, 20
    lengths = torch.tensor([5, 0, 133, 320], dtype=torch.int32, device="cuda")
    cache = _filled(g, B * each + 1, size, H, d, form)
    table = torch.randperm(B * each + 1, generator=g, device="cuda")[: B * each].reshape(B, each).to(torch.int32)
    q = _randn(g, B, H * G, d, dtype=dtype)
    for window in (None, 40):
        want, wl = kq.paged_attention(q, cache, table, lengths, window=window, want_lse=True)
        keep = torch.zeros((cache.k.shape[0], size), dtype=torch.bool, device="cuda")
        wild = table.clone()
        for b, n in enumerate(lengths.tolist()):
            at = torch.arange(max(0, n - window) if window else 0, n, device="cuda")
            keep[table[b].long()[at // size], at % size] = True
            wild[b, -(-n // size):] = torch.tensor([-1, 2 ** 31 - 1, -2 ** 31, 10 ** 6] * each, device="cuda")[: each + (-n // size)]
        bad = []
        for t in cache:
            if t is not None:
                t = t.clone()
                t.transpose(1, 2)[~keep] = math.nan if form == "bf16" else 255
            bad.append(t)
        got, gl = kq.paged_attention(q, kq.KVCache(*bad), wild, lengths, window=window, want_lse=True)
        assert torch.equal(got, want) and torch.equal(gl, wl)
        if form == "bf16":
            bad = [t.clone().masked_fill_(~keep[:, None, :, None], math.inf) for t in cache[:2]]
            assert torch.equal(kq.paged_attention(q, kq.KVCache(*bad), wild, lengths, window=window), want)


def test_attention_of_pages_and_lengths_outside():
    """Pages outside the cache are the nearest ones inside, lengths outside the table too."""
    g = _gen(22)
    cache = _filled(g, 6, 16, 2, 64, "mxfp4")
    q = _randn(g, 3, 4, 64, dtype=BF16)
    table = torch.tensor([[-5, 2 ** 31 - 1, 6], [1, -2 ** 31, 3], [5, 4, 100]], dtype=torch.int32, device="cuda")
    near = torch.tensor([[0, 5, 5], [1, 0, 3], [5, 4, 5]], dtype=torch.int32, device="cuda")
    n = torch.tensor([2 ** 31 - 1, 48, -7], dtype=torch.int32, device="cuda")
    m = torch.tensor([48, 48, 0], dtype=torch.int32, device="cuda")
    assert torch.equal(kq.paged_attention(q, cache, table, n), kq.paged_attention(q, cache, near, m))
    none = kq.paged_attention(q, cache, table[:, :0], n)
    assert none.shape == q.shape and not none.any()
    assert kq.paged_attention(q[:0], cache, table[:0], n[:0]).shape == (0, 4, 64)


def test_attention_layouts():
    """Slices of a fused projection, heads first, a wider table, one table for all, results into slices and over q."""
    g = _gen(23)
    B, H, G, d = 5, 2, 4, 64
    for dtype in (BF16, FP32):
        cache = _filled(g, 30, 16, H, d, "mxfp8")
        table = torch.randint(0, 30, (B, 9), generator=g, device="cuda").to(torch.int32)
        n = torch.tensor([90, 16, 1, 0, 55], dtype=torch.int32, device="cuda")
        fused = _randn(g, B, 2 * H + H * G, d + 3, dtype=dtype)
        q = fused[:, H:H + H * G, 3:]
        want = kq.paged_attention(q.contiguous(), cache, table[:, :6].contiguous(), n)
        assert torch.equal(kq.paged_attention(q, cache, table[:, :6], n), want)
        assert torch.equal(kq.paged_attention(q.transpose(0, 1).contiguous().transpose(0, 1), cache, table, n), want)
        buf = torch.full((B, 3 + H * G, d + 1), 7.0, dtype=dtype, device="cuda")
        kq.paged_attention(q, cache, table, n, out=buf[:, 1:-2, 1:])
        assert torch.equal(buf[:, 1:-2, 1:], want) and (buf[:, 0] == 7).all() and (buf[:, -2:] == 7).all() and (buf[..., 0] == 7).all()
        one = kq.paged_attention(q, cache, table[:1].expand(B, 9), n)
        assert torch.equal(one, kq.paged_attention(q, cache, table[:1].repeat(B, 1), n))
        over = q.contiguous()
        assert kq.paged_attention(over, cache, table, n, out=over) is over and torch.equal(over, want)
        long = _filled(g, 300, 32, H, d, "mxfp4")
        t2 = torch.arange(300, dtype=torch.int32, device="cuda").reshape(1, 300)
        n2 = torch.tensor([9600], dtype=torch.int32, device="cuda")
        q2 = _randn(g, 1, H * G, d, dtype=dtype)
        want = kq.paged_attention(q2, long, t2, n2)
        assert torch.equal(kq.paged_attention(q2, long, t2, n2, out=q2), want) and torch.equal(q2, want)


def test_attention_offsets_past_32_bits():
    """A cache of more than 2^32 bytes: pages at its end."""
    pages, size, H, d = 17000, 128, 8, 128  # 2.2e9 elements in a half, 4.5e9 bytes
    cache = kq.KVCache(*(torch.empty((pages, H, size, d), dtype=BF16, device="cuda") for _ in range(2)))
    g = _gen(24)
    n = 300
    slots = torch.cat([torch.arange(pages * size - n + 100, pages * size), torch.arange(100)]).cuda()
    kv = _randn(g, n, 2, H, d, dtype=BF16)
    kq.kv_cache_write(cache, kv[:, 0], kv[:, 1], slots)
    k, v = kq.kv_cache_read(cache, slots)
    assert torch.equal(k, kv[:, 0]) and torch.equal(v, kv[:, 1])
    table = torch.tensor([[pages - 1, pages - 2, 0]], dtype=torch.int32, device="cuda")
    q, m = _randn(g, 1, 2 * H, d, dtype=BF16), torch.tensor([128], dtype=torch.int32, device="cuda")
    small = kq.KVCache(*(t[-1:].clone() for t in cache[:2]))
    want = kq.paged_attention(q, small, torch.zeros_like(table), m)
    assert torch.isfinite(want).all() and torch.equal(kq.paged_attention(q, cache, table, m), want)


def test_attention_repeats_and_workspaces():
    """The same bits every time, whatever the workspace held."""
    got, lse, (q, cache, table, n) = _check_attn("mxfp4", 4, 2, 8, 128, 32, [5000, 77, 0, 2500])
    ws = kq.paged_attention_workspace(4, 16, 2, 128)
    for fill in (0, 255, 127):
        ws.fill_(fill)
        again, l2 = kq.paged_attention(q, cache, table, n, workspace=ws, want_lse=True)
        assert torch.equal(again, got) and torch.equal(l2, lse)
    given = torch.empty_like(lse)
    assert kq.paged_attention(q, cache, table, n, lse=given)[1] is given and torch.equal(given, lse)


def test_attention_joins_parts_of_a_sequence():
    """Two calls over a sequence's halves, joined by their lse, are the call over all of it."""
    g = _gen(25)
    cache = _filled(g, 40, 16, 2, 64, "bf16")
    q = _randn(g, 1, 4, 64)
    t = torch.arange(40, dtype=torch.int32, device="cuda").reshape(1, 40)
    n = lambda k: torch.tensor([k], dtype=torch.int32, device="cuda")  # noqa: E731
    want, lse = kq.paged_attention(q, cache, t, n(640), want_lse=True)
    (a, la), (b, lb) = kq.paged_attention(q, cache, t[:, :25], n(400), want_lse=True), kq.paged_attention(q, cache, t[:, 25:], n(240), want_lse=True)
    w = torch.softmax(torch.stack([la, lb]).double(), 0).unsqueeze(-1)
    got = w[0] * a.double() + w[1] * b.double()
    _, _, err, lerr = _attn64(q, cache, t, n(640), 0.125, None)
    _within(got, want.double(), 3 * err + 4 * U * want.double().abs(), "joined")
    _within(torch.logaddexp(la, lb), lse.double(), 4 * lerr, "lse")


def test_attention_refusals():
    g = _gen(26)
    cache = _filled(g, 4, 16, 2, 64, "mxfp4")
    q = _randn(g, 3, 4, 64, dtype=BF16)
    t, n = torch.zeros((3, 4), dtype=torch.int32, device="cuda"), torch.ones(3, dtype=torch.int32, device="cuda")
    call = kq.paged_attention
    for bad in (lambda: call(q[:, :3], cache, t, n), lambda: call(q[..., :32], cache, t, n), lambda: call(q[:2], cache, t, n),
                lambda: call(q, cache, t[:2], n), lambda: call(q, cache, t.t(), n), lambda: call(q, cache, t, n[:2]), lambda: call(q, cache, t.cpu(), n),
                lambda: call(q, cache, t, n, window=0), lambda: call(q, cache, t, n, window=-3), lambda: call(q, cache, t, n, out=q[:2]),
                lambda: call(q, cache, t, n, out=q[:, :1].expand(3, 4, 64)), lambda: call(q, cache, t, n, lse=torch.empty(11, device="cuda")),
                lambda: call(q[:2], cache, t[:2], n[:2], out=q[1:])):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: call(q.half(), cache, t, n), lambda: call(q, cache, t.long(), n), lambda: call(q, cache, t, n.long()),
                lambda: call(q, cache, t, n, out=q.float()), lambda: call(q, cache, t, n, lse=torch.empty((3, 4), dtype=BF16, device="cuda"))):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: call(q, cache, t, n, workspace=torch.empty(16, dtype=torch.uint8, device="cuda")), lambda: call(q, cache, t, n, scale=math.nan)):
        with pytest.raises(kq.KQError):
            bad()


# ------------------------------------------------------------------ W4A16 linear layers

def _codes(g, *shape, spread=4):
    *lead, K = shape
    c = torch.randint(0, 256, (*lead, K // 2), generator=g, device="cuda", dtype=torch.uint8)
    return c, torch.randint(127 - spread, 128, (*lead, K // 32), generator=g, device="cuda", dtype=torch.uint8)


def _weight64(c, s):
    nib = torch.stack([c & 15, c >> 4], -1).flatten(-2).long()
    mag = torch.tensor(E2M1, dtype=torch.float64, device="cuda")[nib & 7]
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
    return p


def _linear64(x, w, bias, act, gate, residual):
    """The result in 64 bits and what fp32 sums of K terms (three of each in 32 bits) and the epilogue may be off."""
    x, K = x.double(), x.shape[-1] * (3 if x.dtype == FP32 else 1)
    p, err = x @ w.T, (x.abs() @ w.abs().T) * (2 * K + 20) * U * 1.01
    if bias is not None:
        p = p + bias.double()
        err = err + 2 * U * (p.abs() + bias.double().abs())
    if act == "swiglu":
        u, v = p[..., 0::2], p[..., 1::2]
        s = u * torch.sigmoid(u)
        # |silu'| <= 1.1; the exponential's argument is rounded: |u| U more
        err = 1.1 * err[..., 0::2] * v.abs() + s.abs() * err[..., 1::2] + 1.1 * err[..., 0::2] * err[..., 1::2] + (8 + u.abs()) * U * (s * v).abs()
        p = s * v
    elif act is not None:
        v = _act64(p, act)
        # slopes up to 1.13.  exp(-z) of a rounded z: z U more, z up to p^2; the fit of gelu 4e-7 = 7 U
        err = 1.13 * err + (16 + 2 * p.abs() + 2 * p.square().clamp_max(200.0)) * U * v.abs() + 1e-35
        p = v
    if gate is not None:
        gr = gate.double() if gate.dim() == 1 else gate.double().repeat_interleave(p.shape[0] // gate.shape[0], 0)
        p, err = p * gr, err * gr.abs() + 2 * U * (p * gr).abs()
    if residual is not None:
        p, err = p + residual.double(), err + U * (p.abs() + residual.double().abs()) * 2
    return p, err


def _check_linear(M, N, K, x=BF16, act=None, bias=True, B=0, residual=False, out=BF16, vec=FP32, seed=0, strided=False):
    g = _gen(seed + 3 * M + 5 * N + K)
    w = _codes(g, N, K)
    xv = _randn(g, M, K + 5, dtype=x)[:, 3:K + 3] if strided else _randn(g, M, K, dtype=x)
    cols = N // 2 if act == "swiglu" else N
    bv = _randn(g, N, dtype=vec) if bias else None
    gate = _randn(g, B, 2 * cols + 1, dtype=vec)[:, 1:cols + 1] if B else None
    res = _randn(g, M, cols + 3, dtype=out)[:, 2:cols + 2] if residual else None
    buf = torch.full((M, cols + 5), 7.0, dtype=out, device="cuda") if strided else None
    got = kq.w4a16_linear(xv, *w, bias=bv, act=act, gate=gate, residual=res, out=buf[:, 1:cols + 1] if strided else None,
                          out_dtype=None if strided else out)
    want, err = _linear64(xv, _weight64(*w), bv, act, gate, res)
    assert got.dtype == out and got.shape == (M, cols)
    _within(got, want, err + _stored(want, out) + _stored(err, out), (M, N, K, x, act))
    if strided:
        assert (buf[:, 0] == 7).all() and (buf[:, cols + 1:] == 7).all()


# rows on either side of a tile of 16, ragged widths, K of a block, of parts of a step, of many
W4A16 = [(1, 1, 32), (1, 2, 64), (1, 17, 96), (2, 130, 2016), (1, 3000, 512), (3, 16, 128), (15, 64, 288), (16, 48, 256), (17, 100, 1152),
         (32, 33, 160), (33, 514, 480), (50, 1000, 4096), (1, 4096, 12288), (8, 11200, 2240), (5, 66, 16384), (130, 200, 320),
         # x's rows in LDS, and slices of the columns: runs of 512 and what is left of them, few and many tiles a wave
         (1, 33, 4128), (3, 70, 4096), (16, 330, 4096), (7, 50, 4576), (16, 100, 8224), (2, 18, 12320), (16, 2600, 6400), (11, 1, 5120)]


@pytest.mark.parametrize("M,N,K", W4A16)
@pytest.mark.parametrize("x", [BF16, FP32])
def test_w4a16_sizes(M, N, K, x):
    _check_linear(M, N, K, x, act="gelu")
    _check_linear(M, N, K, x, B=1, residual=True, out=FP32, vec=BF16, strided=True)
    _check_linear(M, N, K, x, bias=False)
    if N % 2 == 0:
        _check_linear(M, N, K, x, act="swiglu", out=FP32, bias=False, strided=True)


@pytest.mark.parametrize("M,N,K", [(1, 130, 384), (6, 90, 320), (16, 330, 1024), (24, 64, 96)])
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("out", [BF16, FP32])
def test_w4a16_epilogues(M, N, K, act, out):
    for x in (BF16, FP32):
        _check_linear(M, N, K, x, act=act, bias=True, out=out)
        _check_linear(M, N, K, x, act=act, bias=False, B=1, residual=True, out=out, strided=True)
        for B in [b for b in (2, 3, M) if M % b == 0]:  # batches that end inside a tile, and one for each row
            _check_linear(M, N, K, x, act=act, bias=True, B=B, residual=B == 2, out=out, vec=BF16)


@pytest.mark.parametrize("M,N,K,x", [(16, 200, 8192, BF16), (9, 130, 4160, FP32), (1, 70, 100000, FP32)])
def test_w4a16_workspaces(M, N, K, x):
    """Given and dirty, of the call's own, and none: the form without one has sums of another order."""
    g = _gen(36)
    xv, w = _randn(g, M, K, dtype=x), _codes(g, N, K)
    ws = kq.w4a16_workspace(M, N, K, x)
    assert ws.numel() >= 4 * M * N * (K // 512)
    want, err = _linear64(xv, _weight64(*w), None, None, None, None)
    got = kq.w4a16_linear(xv, *w, out_dtype=FP32)
    _within(got, want, err + _stored(want, FP32), "own")
    for fill in (0, 255):
        assert torch.equal(kq.w4a16_linear(xv, *w, out_dtype=FP32, workspace=ws.fill_(fill)), got)
    _within(kq.w4a16_linear(xv, *w, out_dtype=FP32, workspace=ws[:0]), want, err + _stored(want, FP32), "none")
    with pytest.raises(kq.KQError):
        kq.w4a16_linear(xv, *w, workspace=ws[:-16])


def test_w4a16_of_wide_ranges():
    """32-bit rows whose values span 2^60, weights of scales far apart: every product takes part in full."""
    g = _gen(31)
    x = _randn(g, 7, 256) * torch.exp2(torch.randint(-30, 30, (7, 256), generator=g, device="cuda").float())
    w = _codes(g, 50, 256, spread=60)
    got = kq.w4a16_linear(x, *w, out_dtype=FP32)
    want, err = _linear64(x, _weight64(*w), None, None, None, None)
    _within(got, want, err + _stored(want, FP32), "wide")


def test_w4a16_of_infinite_rows():
    """A row of NaN or infinities does not reach the others; bf16 infinities come out as such."""
    g = _gen(32)
    for x in (BF16, FP32):
        xv, w = _randn(g, 5, 128, dtype=x), _codes(g, 40, 128)
        want = kq.w4a16_linear(xv, *w)
        xv[2, 5] = math.nan
        xv[4, 9] = math.inf
        got = kq.w4a16_linear(xv, *w)
        assert torch.equal(got[[0, 1, 3]], want[[0, 1, 3]]) and torch.isnan(got[2]).all() and not torch.isfinite(got[4]).any()


def test_w4a16_onto_its_residual_and_none():
    g = _gen(33)
    for M in (1, 20):
        w, gate = _codes(g, 70, 256), _randn(g, 70)
        x, r = _randn(g, M, 256, dtype=BF16), _randn(g, M, 70, dtype=BF16)
        want = kq.w4a16_linear(x, *w, gate=gate, residual=r)
        assert kq.w4a16_linear(x, *w, gate=gate, residual=r, out=r) is r and torch.equal(r, want)
        assert kq.w4a16_linear(x[:0], *w, act="silu").shape == (0, 70) and kq.w4a16_linear(x, w[0][:0], w[1][:0], act="swiglu").shape == (M, 0)
    # rows on their own are rows of a batch
    x, w = _randn(g, 16, 512, dtype=BF16), _codes(g, 96, 512)
    all_ = kq.w4a16_linear(x, *w, out_dtype=FP32)
    for m in (0, 7, 15):
        assert torch.equal(kq.w4a16_linear(x[m:m + 1], *w, out_dtype=FP32)[0], all_[m])


def test_w4a16_out_beside_and_over_x():
    g = _gen(35)
    w = _codes(g, 64, 64)
    both = _randn(g, 4, 128, dtype=BF16)
    want = kq.w4a16_linear(both[:, :64].contiguous(), *w)
    assert torch.equal(kq.w4a16_linear(both[:2, :64], *w, out=both[2:, 64:]), want[:2])  # one array, apart
    rows = both.clone()
    assert torch.equal(kq.w4a16_linear(rows[:, :64], *w, out=rows[:, 64:]), want)  # columns side by side
    assert torch.equal(kq.w4a16_linear(rows[:3, :64], *w, out=rows[1:, 64:]), want[:3])
    assert torch.equal(rows[:, :64], both[:, :64])
    for bad in (both[:, :64], both[:, 32:96], both[1:, :64], both.view(8, 64)[1:5]):
        with pytest.raises(ValueError, match="overlaps"):
            kq.w4a16_linear(both[:len(bad), :64], *w, out=bad)


def test_w4a16_refusals():
    g = _gen(34)
    x, (c, s) = _randn(g, 4, 64, dtype=BF16), _codes(g, 6, 64)
    call = kq.w4a16_linear
    for bad in (lambda: call(x[:, :32], c, s), lambda: call(x, c, s[:, :1]), lambda: call(x, c, s[:5]), lambda: call(x.t().contiguous().t(), c, s),
                lambda: call(x[0], c, s), lambda: call(x, c[:5], s[:5], act="swiglu"), lambda: call(x, c, s, bias=torch.ones(5, device="cuda")),
                lambda: call(x, c, s, gate=torch.ones((3, 6), device="cuda")), lambda: call(x, c, s, gate=torch.ones((0, 6), device="cuda")),
                lambda: call(x, c, s, out=torch.empty((4, 5), device="cuda")), lambda: call(x, c.cpu(), s.cpu()) if False else call(x, c, s.t())):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: call(x.half(), c, s), lambda: call(x, c.short(), s), lambda: call(x, c, s, bias=torch.ones(6, device="cuda", dtype=torch.half)),
                lambda: call(x, c, s, residual=torch.ones((4, 6), device="cuda"), out=torch.ones((4, 6), device="cuda", dtype=BF16))):
        with pytest.raises(TypeError):
            bad()


# ------------------------------------------------------------------ at the operators' limits

def test_attention_of_any_large_window():
    """A window that reaches past the table is none, to the bit: the work is cut the same way."""
    g = _gen(45)
    for B, form in ((1, "bf16"), (3, "mxfp4")):
        cache = _filled(g, B * 500, 64, 2, 64, form)
        table = torch.randperm(B * 500, generator=g, device="cuda").reshape(B, 500).to(torch.int32)
        n = torch.tensor([32000, 77, 20001][:B], dtype=torch.int32, device="cuda")
        q = _randn(g, B, 8, 64)
        want, lse = kq.paged_attention(q, cache, table, n, want_lse=True)
        for window in (32000, 2 ** 31, 2 ** 62, 2 ** 63 - 31, 2 ** 63 - 1, 2 ** 70):
            got, l2 = kq.paged_attention(q, cache, table, n, window=window, want_lse=True)
            assert torch.equal(got, want) and torch.equal(l2, lse), window


def test_rope_of_more_tokens_than_a_launch_holds():
    """More than 2^24 workgroups of 256 threads, which one launch does not take: every token is turned."""
    T, D = 2 ** 24 + 3, 258  # more than 128 pairs: a workgroup a token
    rows = _randn(_gen(41), T + D, dtype=BF16).as_strided((T, 1, D), (1, D, 1))
    p = (torch.arange(T, device="cuda", dtype=torch.int32) * 7 % 100003).reshape(T, 1)
    at = torch.tensor([0, 1, 65535, 2 ** 23, 2 ** 24 - 3, 2 ** 24 - 2, 2 ** 24 - 1, 2 ** 24, 2 ** 24 + 1, T - 1], device="cuda")
    got = kq.rope(rows, p, D)
    assert torch.equal(got[at], kq.rope(rows[at], p[at], D))
    assert kq.rope_backward(rows, p, D, pairing="halves", dx=got) is got
    assert torch.equal(got[at], kq.rope_backward(rows[at], p[at], D, pairing="halves"))
    del got
    torch.cuda.empty_cache()


@pytest.mark.parametrize("form", ["bf16", "mxfp4"])
def test_cache_of_more_tokens_than_a_launch_holds(form):
    """More than 2^24 workgroups of 256 threads: tokens on both sides of where the launches meet, written and read."""
    T, H, d = 2 ** 23 + 3, 129, 32  # more than 512 eights a token: a workgroup for its keys and one for its values
    cache = kq.kv_cache(2, 16, H, d, format=form)
    g = _gen(42)
    k, v = (_randn(g, T + H * d, dtype=BF16).as_strided((T, H, d), (1, d, 1)) for _ in range(2))
    at = torch.tensor([0, 1, 65535, 2 ** 22, 2 ** 23 - 3, 2 ** 23 - 2, 2 ** 23 - 1, 2 ** 23, 2 ** 23 + 1, T - 1], device="cuda")
    slots = torch.full((T,), -1, dtype=torch.int64, device="cuda")
    slots[at] = torch.arange(10, device="cuda") * 3
    kq.kv_cache_write(cache, k, v, slots)
    for t, held in zip((k, v), _held(cache)):
        assert torch.equal(_at(held, slots[at], 16), _nearest(t[at], form))
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 160 << 30:
        pytest.skip("reading so many tokens takes 139 GB")
    got = kq.kv_cache_read(cache, slots)
    for a, b in zip(got, kq.kv_cache_read(cache, slots[at])):
        assert torch.equal(a[at], b) and not a[2:100].any() and not a[2 ** 23 - 100:2 ** 23 - 4].any()
    del got, a, b
    torch.cuda.empty_cache()


def test_rope_angles_are_rounded_once():
    """Rows of (1, 0) give the table itself: cos and sin of a 64-bit angle, each rounded once to 32 bits."""
    for axes, theta, T in (([64], 1e4, 4096), ([16, 56, 56], 1e4, 1024), ([24, 24, 24], 256.0, 2048)):
        n = sum(axes) // 2
        x = torch.zeros((T, 1, 2 * n), device="cuda")
        x[..., :n] = 1.0
        p = torch.arange(T, device="cuda").reshape(T, 1).expand(T, len(axes)).contiguous()
        for call, sign in ((kq.rope, 1), (kq.rope_backward, -1)):
            got = call(x, p, axes, theta=theta, pairing="halves")
            want = _rope64(x, p, axes, theta, "halves", None, sign < 0)[0]
            # half a step of the value; angles below 2^12 from 64-bit frequencies are within 2^-38
            _within(got, want, U * want.abs() + 2.0 ** -37, (axes, sign))


@pytest.mark.parametrize("form,terms", [("bf16", 2), ("mxfp8", 3), ("mxfp4", 6)])
@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_attention_probabilities_in_32_bits(form, terms, dtype):
    """One token's p v against tokens of p = 1 whose values cancel it: what is left shows the last bits of p, whatever the
    result's type."""
    g = _gen(44)
    B, d = 160, 32
    k = torch.zeros((B, 16, 1, d), device="cuda")
    k[:, terms, 0, 0] = -torch.rand(B, generator=g, device="cuda")
    k = _nearest(k, form)
    v = torch.zeros((B, 16, 1, d), dtype=torch.float64, device="cuda")
    v[:, terms] = _nearest(torch.rand((B, 1, d), generator=g, device="cuda") + 1.0, form)
    p = torch.exp(k[:, terms, :, :1])
    left = -p * v[:, terms]
    for i in range(terms):
        v[:, i] = _nearest(left, form)
        left = left - v[:, i]
    cache = kq.kv_cache(B, 16, 1, d, format=form)
    kq.kv_cache_write(cache, k.reshape(-1, 1, d).float(), v.reshape(-1, 1, d).float(), torch.arange(16 * B, device="cuda"))
    q = torch.zeros((B, 1, d), dtype=dtype, device="cuda")
    q[..., 0] = 1.0
    got = kq.paged_attention(q, cache, torch.arange(B, dtype=torch.int32, device="cuda")[:, None],
                             torch.full((B,), terms + 1, dtype=torch.int32, device="cuda"), scale=1.0)
    total = terms + p
    want = (v[:, :terms].sum(1) + p * v[:, terms]) / total
    size = (v[:, :terms].abs().sum(1) + p * v[:, terms].abs()) / total
    # the score is one product: its scale and its rounding, U each of up to 1.45 and by ln 2; the exponential 2 U; three terms
    # of each p, added with 2 U at most
    err = (2 * 1.5 + 2 + 2 * 3 * (terms + 1)) * U * size
    _within(got, want, err + _stored(want, dtype) + _stored(err, dtype), form)


@pytest.mark.parametrize("form", ["mxfp8", "mxfp4"])
def test_cache_rounding_at_the_smallest_scale(form):
    """Blocks of scale byte 0 (units of 2^-127): borders between elements and saturation, where values are normal in 32 bits."""
    grid = torch.tensor(E2M1).double() if form == "mxfp4" else torch.unique(torch.cat(
        [torch.arange(8) * 2.0 ** -9, ((1 + torch.arange(8) / 8) * torch.exp2(torch.arange(-6.0, 9)[:, None])).flatten()])).double()
    grid = grid[grid <= 448]
    edge = (grid[1:] + grid[:-1]) / 2
    v = torch.cat([grid, edge, edge * (1 + 2.0 ** -20), edge * (1 - 2.0 ** -20), torch.tensor([7.5, 7.99] if form == "mxfp4" else [464.0, 480.0, 496.0, 511.0])])
    v = v[(v >= 2) | (v == 0)]  # 2^-126 and above
    v = torch.cat([v, -v])
    v = torch.nn.functional.pad(v, (0, -len(v) % 31)).reshape(-1, 31)
    blocks = []
    for lead in ([4.0, 2.0] if form == "mxfp4" else [256.0, 2.0, 5.0]):  # the largest magnitude's binade, and below it
        blocks.append(torch.cat([torch.full((len(v), 1), lead).double(), v], 1))
    x = (torch.cat(blocks) * 2.0 ** -127).reshape(-1, 1, 32).float().cuda()
    assert ((x == 0) | (x.abs() >= 2.0 ** -126)).all()
    cache = kq.kv_cache(-(-len(x) // 16), 16, 1, 32, format=form)
    slots = torch.arange(len(x), device="cuda")
    kq.kv_cache_write(cache, x, -x, slots)
    assert not cache.k_scales.any() and not cache.v_scales.any()
    want = _nearest(x, form)
    held = _held(cache)
    assert torch.equal(_at(held[0], slots, 16), want) and torch.equal(_at(held[1], slots, 16), -want)
    for dtype in (FP32, BF16):  # below 2^-126 as they are or as zero
        for got, sign in zip(kq.kv_cache_read(cache, slots, out_dtype=dtype), (1, -1)):
            got = got.double()
            assert ((got == sign * want) | ((got == 0) & (want.abs() < 2.0 ** -126))).all()
    if form == "mxfp4":
        codes, scales = kq.mxfp4(x[:, 0].to(BF16))
        kq.kv_cache_write(cache, x.to(BF16), x.to(BF16), slots)
        assert torch.equal(cache.k.transpose(1, 2).reshape(-1, 16)[:len(x)], codes) and torch.equal(cache.k_scales.reshape(-1, 1)[:len(x)], scales)


@pytest.mark.parametrize("form", FORMATS)
def test_cache_of_subnormal_values(form):
    """Values below 2^-126 beside larger ones and on their own: held as the nearest element."""
    g = _gen(43)
    x = _randn(g, 48, 2, 64) * torch.exp2(torch.randint(-140, -118, (48, 2, 1), generator=g, device="cuda").double()).float()
    assert (x.abs() < 2.0 ** -126).any() and (x.abs() >= 2.0 ** -126).any()
    cache = kq.kv_cache(3, 16, 2, 64, format=form)
    slots = torch.arange(48, device="cuda")
    for dtype in (FP32, BF16):
        y = x.to(dtype)
        kq.kv_cache_write(cache, y, y, slots)
        assert torch.equal(_at(_held(cache)[0], slots, 16), _nearest(y, form)), dtype


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_attention_of_one_run_a_head(dtype):
    """So many heads that each has one workgroup, which takes every sequence whole: no second launch."""
    _check_attn("bf16", 4, 1300, 1, 32, 16, [40, 0, 7, 33], dtype)
    _check_attn("mxfp4", 3, 1290, 2, 64, 16, [1, 100, 64], dtype, window=50)


def test_w4a16_refuses_weights_elsewhere():
    g = _gen(46)
    x, (c, s) = _randn(g, 4, 64, dtype=BF16), _codes(g, 6, 64)
    for bad in (lambda: kq.w4a16_linear(x, c.cpu(), s.cpu()), lambda: kq.w4a16_linear(x, c, s.cpu()), lambda: kq.w4a16_linear(x.cpu(), c, s)):
        with pytest.raises(TypeError, match="device tensor"):
            bad()
    for bad in (lambda: kq.w4a16_linear(x, c, s, bias=torch.ones(6)), lambda: kq.w4a16_linear(x, c, s, residual=torch.ones((4, 6), dtype=BF16))):
        with pytest.raises((TypeError, ValueError)):
            bad()


@pytest.mark.parametrize("form", ["mxfp8", "mxfp4"])
def test_attention_over_blocks_of_the_smallest_scale(form):
    """Values in units of 2^-127 take part: one token's own, and two tokens' mean."""
    cache = kq.kv_cache(2, 16, 1, 32, format=form)
    v = torch.zeros((2, 16, 1, 32), device="cuda")
    v[0, :2] = torch.tensor([2.0, 3.0, 4.0, -6.0] * 8, device="cuda") * 2.0 ** -127
    v[1, 0] = torch.tensor([6.0, -4.0, 2.0, -2.0] * 8, device="cuda") * 2.0 ** -127
    kq.kv_cache_write(cache, torch.zeros_like(v).reshape(-1, 1, 32), v.reshape(-1, 1, 32), torch.arange(32, device="cuda"))
    assert not cache.v_scales.any()
    table, n = torch.tensor([[0], [1]], dtype=torch.int32, device="cuda"), torch.tensor([2, 1], dtype=torch.int32, device="cuda")
    for dtype in (BF16, FP32):
        got = kq.paged_attention(torch.ones((2, 1, 32), dtype=dtype, device="cuda"), cache, table, n)
        assert torch.equal(got[:, 0].float(), v[:, 0, 0])
