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
