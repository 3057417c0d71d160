"""Refusals of block_norm, mxfp4_linear and mxfp4_grouped_linear: every invalid
argument with its status before any HIP call, and the binding's checks."""
import ctypes

import pytest
import torch

kq = pytest.importorskip("paper_2607_21446_amd")

SUCCESS, INVALID, NULLP, MISALIGNED, UNSUPPORTED = range(5)
FAKE = 1 << 20  # 16-byte aligned fake device address: validation fails before any use


def _linear(**kw):
    a = dict(ac=FAKE, as_=FAKE, M=4, bc=FAKE, bs=FAKE, N=6, K=64, bias=None, gate=None, gs=0, gr=4, vt=0, act=0, res=None,
             ldr=0, out=FAKE, ldo=6, ot=1)
    assert set(kw) <= set(a)
    return kq.lib().kq_mxfp4_linear(*{**a, **kw}.values(), None)


@pytest.mark.parametrize("kw,status", [
    (dict(K=48), INVALID), (dict(K=0), INVALID), (dict(K=(1 << 30) + 32), INVALID), (dict(M=-1), INVALID), (dict(N=-1), INVALID),
    (dict(M=1 << 31), INVALID), (dict(N=65535 * 128 + 1, ldo=1 << 40), INVALID), (dict(vt=2), INVALID), (dict(ot=-1), INVALID),
    (dict(act=6), INVALID), (dict(act=-1), INVALID), (dict(act=5, N=5), INVALID), (dict(ldo=5), INVALID), (dict(act=5, ldo=2), INVALID),
    (dict(gate=FAKE, gr=0), INVALID), (dict(gate=FAKE, gs=-1), INVALID), (dict(res=FAKE, ldr=5), INVALID),
    (dict(M=(1 << 31) - 1, N=1 << 20, ldo=1 << 20), UNSUPPORTED),  # 2^25 x 2^14 tiles of 64 x 64
    (dict(ac=None), NULLP), (dict(as_=None), NULLP), (dict(bc=None), NULLP), (dict(bs=None), NULLP), (dict(out=None), NULLP),
    (dict(ac=FAKE + 8), MISALIGNED), (dict(bc=FAKE + 1), MISALIGNED), (dict(out=FAKE + 1), MISALIGNED),
    (dict(bias=FAKE + 2), MISALIGNED), (dict(gate=FAKE + 2), MISALIGNED), (dict(res=FAKE + 1, ldr=6), MISALIGNED),
    (dict(M=0), SUCCESS), (dict(N=0, ldo=0), SUCCESS), (dict(M=0, out=None, ac=None), SUCCESS),
])
def test_linear_rejects(kw, status):
    assert _linear(**kw) == status
    assert (kq.lib().kq_last_error_detail() == b"") == (status == SUCCESS)


def _grouped(**kw):
    a = dict(ac=FAKE, as_=FAKE, T=4, rows=FAKE, R=8, bc=FAKE, bs=FAKE, E=3, N=6, K=64, off=FAKE, bias=None, vt=0, act=0, rs=None,
             out=FAKE, ldo=6, ot=1)
    assert set(kw) <= set(a)
    return kq.lib().kq_mxfp4_grouped_linear(*{**a, **kw}.values(), None)


@pytest.mark.parametrize("kw,status", [
    (dict(K=48), INVALID), (dict(R=-1), INVALID), (dict(T=-1), INVALID), (dict(E=-1), INVALID), (dict(R=1 << 31), INVALID),
    (dict(T=1 << 31), INVALID), (dict(E=1 << 31), INVALID), (dict(act=7), INVALID), (dict(act=5, N=7, ldo=7), INVALID),
    (dict(ldo=5), INVALID), (dict(vt=3), INVALID), (dict(T=0), INVALID), (dict(rows=None), INVALID),  # 8 rows of 4 tokens
    (dict(off=None), NULLP), (dict(out=None), NULLP), (dict(bc=None), NULLP), (dict(off=FAKE + 2), MISALIGNED),
    (dict(rows=FAKE + 1), MISALIGNED), (dict(rs=FAKE + 2), MISALIGNED), (dict(bc=FAKE + 4), MISALIGNED),
    (dict(R=(1 << 31) - 1, N=8000000, ldo=8000000), UNSUPPORTED),
    (dict(R=0), SUCCESS), (dict(N=0, ldo=0), SUCCESS), (dict(E=0), SUCCESS), (dict(R=0, T=0, ac=None, rows=None), SUCCESS),
])
def test_grouped_rejects(kw, status):
    assert _grouped(**kw) == status
    assert (kq.lib().kq_last_error_detail() == b"") == (status == SUCCESS)


def _norm(**kw):
    a = dict(x=FAKE, xt=1, res=FAKE, st=1, M=4, d=8, B=1, gate=None, gs=0, scale=None, ss=0, shift=None, hs=0, w=None, pw=None,
             vt=0, norm=1, post=0, alpha=1.0, eps=1e-6, h=FAKE, y=FAKE)
    assert set(kw) <= set(a)
    return kq.lib().kq_block_norm(*{**a, **kw}.values(), None)


@pytest.mark.parametrize("kw,status", [
    (dict(M=-1), INVALID), (dict(M=1 << 31), INVALID), (dict(d=0), INVALID), (dict(d=16385), INVALID), (dict(B=0), INVALID),
    (dict(B=3), INVALID), (dict(xt=2), INVALID), (dict(st=2), INVALID), (dict(vt=-1), INVALID), (dict(norm=3), INVALID),
    (dict(post=-1), INVALID), (dict(eps=-1e-6), INVALID), (dict(eps=float("nan")), INVALID), (dict(pw=FAKE), INVALID),
    (dict(gate=FAKE, gs=-8), INVALID), (dict(scale=FAKE, ss=-1), INVALID), (dict(shift=FAKE, hs=-1), INVALID),
    (dict(norm=0), INVALID), (dict(y=None), NULLP), (dict(x=None), NULLP), (dict(norm=0, y=None, h=None), NULLP),
    (dict(x=FAKE + 1), MISALIGNED), (dict(st=0, h=FAKE + 2), MISALIGNED), (dict(res=FAKE + 1), MISALIGNED),
    (dict(y=FAKE + 1), MISALIGNED), (dict(w=FAKE + 2), MISALIGNED), (dict(gate=FAKE + 2), MISALIGNED),
    (dict(M=0), SUCCESS), (dict(M=0, x=None, y=None, h=None, res=None), SUCCESS),
])
def test_norm_rejects(kw, status):
    assert _norm(**kw) == status
    assert (kq.lib().kq_last_error_detail() == b"") == (status == SUCCESS)


def _backward(**kw):
    n = ctypes.c_size_t(0)
    assert kq.lib().kq_block_norm_workspace_size(4, 8, 1, ctypes.byref(n)) == SUCCESS
    a = dict(dy=FAKE, dh=None, x=FAKE, xt=1, h=FAKE, st=1, M=4, d=8, B=1, gate=None, gs=0, scale=None, ss=0, w=None, pw=None,
             vt=0, norm=1, post=0, alpha=1.0, eps=1e-6, dx=FAKE, dr=FAKE, dgate=None, dscale=None, dshift=None, dw=None,
             dpw=None, ws=FAKE, wsb=n.value)
    assert set(kw) <= set(a)
    return kq.lib().kq_block_norm_backward(*{**a, **kw}.values(), None)


@pytest.mark.parametrize("kw,status", [
    (dict(d=16385), INVALID), (dict(B=3), INVALID), (dict(norm=0), INVALID), (dict(norm=3), INVALID), (dict(dpw=FAKE), INVALID),
    (dict(pw=FAKE), INVALID), (dict(wsb=8), INVALID), (dict(gate=FAKE, gs=-1), INVALID), (dict(eps=-1.0), INVALID),
    (dict(dy=None), NULLP), (dict(h=None), NULLP), (dict(x=None, post=1), NULLP), (dict(x=None, dgate=FAKE), NULLP), (dict(ws=None), NULLP),
    (dict(dy=FAKE + 1), MISALIGNED), (dict(dh=FAKE + 1), MISALIGNED), (dict(dx=FAKE + 1), MISALIGNED), (dict(dgate=FAKE + 2), MISALIGNED),
    (dict(ws=FAKE + 8), MISALIGNED), (dict(M=0), SUCCESS),
])
def test_norm_backward_rejects(kw, status):
    assert _backward(**kw) == status
    assert (kq.lib().kq_last_error_detail() == b"") == (status == SUCCESS)


def test_norm_workspace_size():
    n = ctypes.c_size_t(0)
    ws = lambda M, d, B: kq.lib().kq_block_norm_workspace_size(M, d, B, ctypes.byref(n))  # noqa: E731
    assert ws(4, 0, 1) == INVALID and ws(4, 8, 3) == INVALID and ws(-1, 8, 1) == INVALID
    assert kq.lib().kq_block_norm_workspace_size(4, 8, 1, None) == NULLP
    # three column sums in 32 bits for each batch at least
    for M, d, B in ((1, 1, 1), (4608, 1152, 4), (700, 40, 700), (0, 8, 1)):
        assert ws(M, d, B) == SUCCESS
        assert (n.value >= B * 3 * d * 4) == (M > 0) and n.value > 0


def test_binding_names_what_is_wrong():
    x = torch.zeros((4, 64), dtype=torch.bfloat16)
    c, s = torch.zeros((4, 32), dtype=torch.uint8), torch.zeros((4, 2), dtype=torch.uint8)
    for call in (lambda: kq.block_norm(x), lambda: kq.block_norm_backward(x, x), lambda: kq.mxfp4_linear(c, s, c, s),
                 lambda: kq.mxfp4_grouped_linear(c, s, c[None], s[None], torch.zeros(2, dtype=torch.int32))):
        with pytest.raises(TypeError, match="device tensor"):
            call()
    with pytest.raises(ValueError, match="norm must be one of"):
        kq.block_norm(x, norm="batch")
    with pytest.raises(ValueError, match="act must be one of"):
        kq.mxfp4_linear(c, s, c, s, act="tanh")
    with pytest.raises(ValueError, match="backward pass needs a norm"):
        kq.block_norm_backward(x, x, norm=None)
    with pytest.raises(TypeError, match="float32 or bfloat16"):
        kq.block_norm(x.half())


@pytest.mark.parametrize("call,kw", [
    (_linear, dict(M=(1 << 31) - 1, N=4, K=32)),  # 2^24 tiles of 128 rows, of 256 threads
    (_grouped, dict(R=1 << 20, T=1 << 20, E=1 << 20, N=1024, ldo=1024, K=32)),  # 2^24 tiles of 64 features, of 256 threads
    (_grouped, dict(R=1 << 22, T=1 << 22, E=8, N=1 << 22, ldo=1 << 22, K=1 << 25)),  # 2^32 tiles of 64 x 64
])
def test_more_threads_than_a_launch_counts(call, kw):
    """Fewer than 2^31 workgroups whose threads pass 2^32, which a launch would start modulo 2^32."""
    assert call(**kw) == UNSUPPORTED
    assert b"more workgroups than one launch holds" in kq.lib().kq_last_error_detail()
