"""Refusals of the operators of a generation step (rope, the paged cache, attention
over it, w4a16_linear): every invalid argument with its status before any HIP call,
and the binding's checks."""
import ctypes

import pytest
import torch

kq = pytest.importorskip("paper_2607_21446_amd")
from paper_2607_21446_amd.binding import _CacheStruct  # noqa: E402

SUCCESS, INVALID, NULLP, MISALIGNED, UNSUPPORTED = range(5)
FAKE = 1 << 20  # 16-byte aligned fake device address: validation fails before any use
NAN, INF = float("nan"), float("inf")


def _said(status):
    return (kq.lib().kq_last_error_detail() == b"") == (status == SUCCESS)


def _rope(**kw):
    a = dict(x=FAKE, dt=1, T=4, H=2, D=64, xt=128, xh=64, pos=FAKE, pt=0, ps=1, axes=(64,), n=None, theta=1e4, freqs=None, pairing=0,
             back=0, y=FAKE, yt=128, yh=64)
    assert set(kw) <= set(a)
    a.update(kw)
    axes = a["axes"]
    a["n"] = len(axes or ()) if a["n"] is None else a["n"]
    a["axes"] = None if axes is None else (ctypes.c_int * len(axes))(*axes)
    return kq.lib().kq_rope(*a.values(), None)


@pytest.mark.parametrize("kw,status", [
    (dict(T=-1), INVALID), (dict(T=1 << 31), INVALID), (dict(H=-1), INVALID), (dict(H=65536), INVALID), (dict(D=63), INVALID),
    (dict(D=0), INVALID), (dict(D=1026, axes=(64,)), INVALID), (dict(dt=2), INVALID), (dict(pt=3), INVALID), (dict(pt=-1), INVALID),
    (dict(pairing=2), INVALID), (dict(back=2), INVALID), (dict(axes=(), n=0), INVALID), (dict(axes=(8,) * 5), INVALID),
    (dict(axes=None, n=1), NULLP), (dict(axes=(7,)), INVALID), (dict(axes=(0, 8)), INVALID), (dict(axes=(-2,)), INVALID),
    (dict(axes=(40, 40)), INVALID), (dict(theta=0.0), INVALID), (dict(theta=-1.0), INVALID), (dict(theta=NAN), INVALID),
    (dict(theta=INF), INVALID), (dict(xt=-1), INVALID), (dict(ps=-1), INVALID), (dict(yt=32), INVALID), (dict(yh=62), INVALID),
    (dict(x=None), NULLP), (dict(y=None), NULLP), (dict(pos=None), NULLP), (dict(x=FAKE + 1), MISALIGNED), (dict(dt=0, y=FAKE + 2), MISALIGNED),
    (dict(pos=FAKE + 2), MISALIGNED), (dict(pt=1, pos=FAKE + 4), MISALIGNED), (dict(freqs=FAKE + 4), MISALIGNED),
    (dict(T=0), SUCCESS), (dict(H=0), SUCCESS), (dict(T=0, x=None, y=None, pos=None), SUCCESS),
])
def test_rope_rejects(kw, status):
    assert _rope(**kw) == status and _said(status)


def _cache(**kw):
    a = dict(k=FAKE, v=FAKE, k_scales=FAKE, v_scales=FAKE, format=2, pages=5, heads=2, page_size=16, d=64)
    assert set(kw) <= set(a)
    return ctypes.byref(_CacheStruct(*{**a, **kw}.values()))


BAD_CACHES = [
    (dict(format=3), INVALID), (dict(format=-1), INVALID), (dict(d=0), INVALID), (dict(d=48), INVALID), (dict(d=288), INVALID),
    (dict(heads=0), INVALID), (dict(heads=65536), INVALID), (dict(page_size=8), INVALID), (dict(page_size=24), INVALID),
    (dict(page_size=65536), INVALID), (dict(pages=0), INVALID), (dict(pages=1 << 31), INVALID), (dict(pages=-1), INVALID),
    (dict(pages=(1 << 31) - 1, heads=65535, page_size=32768, d=256), INVALID),
    (dict(k=None), NULLP), (dict(v=None), NULLP), (dict(k_scales=None), NULLP), (dict(v_scales=None, format=1), NULLP),
    (dict(k=FAKE + 8), MISALIGNED), (dict(v=FAKE + 2, format=0), MISALIGNED),
]


def _write(cache=None, **kw):
    a = dict(c=_cache() if cache is None else cache, k=FAKE, v=FAKE, dt=1, T=3, kt=128, kh=64, vt=128, vh=64, slots=FAKE)
    assert set(kw) <= set(a)
    return kq.lib().kq_kv_cache_write(*{**a, **kw}.values(), None)


def _read(cache=None, **kw):
    a = dict(c=_cache() if cache is None else cache, slots=FAKE, T=3, k=FAKE, v=FAKE, dt=1)
    assert set(kw) <= set(a)
    return kq.lib().kq_kv_cache_read(*{**a, **kw}.values(), None)


def _attn(cache=None, **kw):
    n = ctypes.c_size_t(0)
    assert kq.lib().kq_paged_attention_workspace_size(3, 8, 2, 64, ctypes.byref(n)) == SUCCESS
    a = dict(q=FAKE, dt=1, B=3, Hq=8, qs=512, qh=64, c=_cache() if cache is None else cache, table=FAKE, ts=4, pages=4, lengths=FAKE,
             scale=0.125, window=0, out=FAKE, os=512, oh=64, lse=None, ws=FAKE, wsb=n.value)
    assert set(kw) <= set(a)
    return kq.lib().kq_paged_attention(*{**a, **kw}.values(), None)


@pytest.mark.parametrize("call", [_write, _read, _attn])
@pytest.mark.parametrize("kw,status", BAD_CACHES)
def test_caches_are_rejected(call, kw, status):
    assert call(_cache(**kw)) == status and _said(status)
    assert call(c=None) == NULLP and _said(NULLP)


@pytest.mark.parametrize("kw,status", [
    (dict(T=-1), INVALID), (dict(T=1 << 31), INVALID), (dict(dt=2), INVALID), (dict(kt=-1), INVALID), (dict(vh=-64), INVALID),
    (dict(k=None), NULLP), (dict(v=None), NULLP), (dict(slots=None), NULLP), (dict(k=FAKE + 1), MISALIGNED),
    (dict(dt=0, v=FAKE + 2), MISALIGNED), (dict(slots=FAKE + 4), MISALIGNED), (dict(T=0), SUCCESS), (dict(T=0, k=None, slots=None), SUCCESS),
])
def test_write_rejects(kw, status):
    assert _write(**kw) == status and _said(status)


@pytest.mark.parametrize("kw,status", [
    (dict(T=-1), INVALID), (dict(T=1 << 31), INVALID), (dict(dt=-1), INVALID), (dict(k=None), NULLP), (dict(v=None), NULLP),
    (dict(slots=None), NULLP), (dict(k=FAKE + 8), MISALIGNED), (dict(v=FAKE + 4), MISALIGNED), (dict(slots=FAKE + 4), MISALIGNED),
    (dict(T=0), SUCCESS), (dict(T=0, k=None, v=None), SUCCESS),
])
def test_read_rejects(kw, status):
    assert _read(**kw) == status and _said(status)


@pytest.mark.parametrize("kw,status", [
    (dict(B=-1), INVALID), (dict(B=(1 << 20) + 1), INVALID), (dict(Hq=7), INVALID), (dict(Hq=0), INVALID), (dict(Hq=65536), INVALID),
    (dict(dt=2), INVALID), (dict(qs=-1), INVALID), (dict(oh=-64), INVALID), (dict(ts=-1), INVALID), (dict(pages=-1), INVALID),
    (dict(pages=1 << 31), INVALID), (dict(window=-1), INVALID), (dict(scale=NAN), INVALID), (dict(scale=INF), INVALID),
    (dict(os=32), INVALID), (dict(oh=63), INVALID), (dict(wsb=8), INVALID),
    (dict(q=None), NULLP), (dict(out=None), NULLP), (dict(lengths=None), NULLP), (dict(table=None), NULLP), (dict(ws=None), NULLP),
    (dict(q=FAKE + 1), MISALIGNED), (dict(dt=0, out=FAKE + 2), MISALIGNED), (dict(table=FAKE + 2), MISALIGNED),
    (dict(lengths=FAKE + 1), MISALIGNED), (dict(lse=FAKE + 2), MISALIGNED), (dict(ws=FAKE + 8), MISALIGNED),
    (dict(B=0), SUCCESS), (dict(B=0, q=None, out=None, ws=None), SUCCESS),
])
def test_attention_rejects(kw, status):
    assert _attn(**kw) == status and _said(status)


def test_attention_workspace_size():
    n = ctypes.c_size_t(0)
    ws = lambda B, Hq, H, d: kq.lib().kq_paged_attention_workspace_size(B, Hq, H, d, ctypes.byref(n))  # noqa: E731
    assert ws(-1, 8, 2, 64) == INVALID and ws(1, 8, 3, 64) == INVALID and ws(1, 8, 0, 64) == INVALID and ws(1, 8, 2, 40) == INVALID
    assert ws(1, 0, 2, 64) == INVALID and ws((1 << 20) + 1, 8, 2, 64) == INVALID and ws(1, 1 << 16, 1, 64) == INVALID
    assert kq.lib().kq_paged_attention_workspace_size(1, 8, 2, 64, None) == NULLP
    for B, Hq, H, d in ((0, 1, 1, 32), (1, 1, 1, 32), (1, 64, 8, 128), (4096, 64, 8, 128), (1 << 20, 65535, 65535, 256), (1 << 20, 65535, 1, 256)):
        assert ws(B, Hq, H, d) == SUCCESS and n.value >= max(16, 8 * B)
    # a few parts a head at most: many sequences take no more places than twice those
    assert ws(4096, 64, 8, 128) == SUCCESS and n.value < 1 << 24


def _w4a16(**kw):
    a = dict(x=FAKE, xt=1, M=4, ldx=64, bc=FAKE, bs=FAKE, N=6, K=64, bias=None, gate=None, gs=0, gr=4, vt=0, act=0, res=None, ldr=0,
             out=FAKE, ldo=6, ot=1, ws=None, wsb=0)
    assert set(kw) <= set(a)
    return kq.lib().kq_w4a16_linear(*{**a, **kw}.values(), None)


@pytest.mark.parametrize("kw,status", [
    (dict(K=48), INVALID), (dict(K=0), INVALID), (dict(K=(1 << 30) + 32, ldx=1 << 31), INVALID), (dict(M=-1), INVALID), (dict(N=-1), INVALID),
    (dict(M=65535 * 16 + 1), INVALID), (dict(N=65535 * 128 + 1, ldo=1 << 40), INVALID), (dict(xt=2), INVALID), (dict(vt=2), INVALID),
    (dict(ot=-1), INVALID), (dict(act=6), INVALID), (dict(act=5, N=5), INVALID), (dict(ldo=5), INVALID), (dict(act=5, ldo=2), INVALID),
    (dict(ldx=63), INVALID), (dict(gate=FAKE, gr=0), INVALID), (dict(gate=FAKE, gs=-1), INVALID), (dict(res=FAKE, ldr=5), INVALID),
    (dict(x=None), NULLP), (dict(bc=None), NULLP), (dict(bs=None), NULLP), (dict(out=None), NULLP), (dict(bc=FAKE + 8), MISALIGNED),
    (dict(x=FAKE + 1), MISALIGNED), (dict(xt=0, x=FAKE + 2), MISALIGNED), (dict(out=FAKE + 1), MISALIGNED), (dict(bias=FAKE + 2), MISALIGNED),
    (dict(gate=FAKE + 2), MISALIGNED), (dict(res=FAKE + 1, ldr=6), MISALIGNED), (dict(ws=FAKE + 8), MISALIGNED),
    (dict(M=16, K=12288, ldx=12288, ws=FAKE, wsb=8), INVALID), (dict(M=0), SUCCESS), (dict(N=0, ldo=0), SUCCESS),
    (dict(M=0, x=None, out=None), SUCCESS),
])
def test_w4a16_rejects(kw, status):
    assert _w4a16(**kw) == status and _said(status)


def test_w4a16_workspace_size():
    n = ctypes.c_size_t(0)
    ws = lambda M, N, K, t: kq.lib().kq_w4a16_workspace_size(M, N, K, t, ctypes.byref(n))  # noqa: E731
    assert ws(-1, 8, 64, 1) == INVALID and ws(1, 8, 40, 1) == INVALID and ws(1, 8, 64, 2) == INVALID
    assert kq.lib().kq_w4a16_workspace_size(1, 8, 64, 1, None) == NULLP
    for M, N, K, t, used in ((0, 8, 64, 1, False), (1, 4096, 4096, 1, False), (16, 4096, 1152, 0, False), (17, 4096, 12288, 0, False),
                             (16, 4097, 12288, 0, True), (16, 4096, 12288, 1, True), (1, 1, 1 << 20, 1, True)):
        assert ws(M, N, K, t) == SUCCESS and (n.value > 0) == used, (M, N, K, t)
        assert not used or n.value >= 4 * M * N * (K // 512)


def test_binding_names_what_is_wrong():
    x = torch.zeros((4, 2, 64), dtype=torch.bfloat16)
    pos, slots = torch.zeros(4, dtype=torch.int64), torch.zeros(4, dtype=torch.int64)
    cache = kq.kv_cache(3, 16, 2, 64, device="cpu")
    table, lengths = torch.zeros((4, 3), dtype=torch.int32), torch.zeros(4, dtype=torch.int32)
    codes, scales = torch.zeros((6, 32), dtype=torch.uint8), torch.zeros((6, 2), dtype=torch.uint8)
    for call in (lambda: kq.rope(x, pos, 64), lambda: kq.rope_backward(x, pos, [64]), lambda: kq.kv_cache_write(cache, x, x, slots),
                 lambda: kq.kv_cache_read(cache, slots), lambda: kq.paged_attention(x, cache, table, lengths),
                 lambda: kq.w4a16_linear(x[:, 0], codes, scales)):
        with pytest.raises(TypeError, match="device tensor"):
            call()
    with pytest.raises(ValueError, match="pairing must be one of"):
        kq.rope(x, pos, 64, pairing="interleaved")
    with pytest.raises(ValueError, match="act must be one of"):
        kq.w4a16_linear(x[:, 0], codes, scales, act="tanh")
    with pytest.raises(ValueError, match="format must be one of"):
        kq.kv_cache(3, 16, 2, 64, format="int8", device="cpu")
    for bad in ((0, 16, 2, 64), (3, 24, 2, 64), (3, 8, 2, 64), (3, 16, 0, 64), (3, 16, 2, 72), (3, 16, 2, 288)):
        with pytest.raises(ValueError, match="page_size must be"):
            kq.kv_cache(*bad, device="cpu")
    with pytest.raises(TypeError, match="must be a KVCache"):
        kq.kv_cache_read(tuple(cache), slots)


def test_caches():
    for form, row, scaled in (("bf16", 128, False), ("mxfp8", 128, True), ("mxfp4", 64, True)):
        c = kq.kv_cache(3, 32, 2, 128, format=form, device="cpu")
        assert c.format == form and c.d == 128 and c.page_size == 32
        assert c.k.shape == c.v.shape == (3, 2, 32, row) and not c.k.any() and not c.v.any()
        assert (c.k_scales is not None) == scaled and (not scaled or c.k_scales.shape == c.v_scales.shape == (3, 2, 32, 4))
