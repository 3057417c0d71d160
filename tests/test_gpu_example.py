"""examples/w4a4_block.py: every step against its definition in 64 bits, from
what the step before it left (its bf16 values, its codes and scales)."""
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
    spec = importlib.util.spec_from_file_location("w4a4_block", os.path.join(ROOT, "examples", "w4a4_block.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def _values(codes, scales):
    nib = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).long()
    mag = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device=codes.device)[nib & 7]
    return torch.where(nib >= 8, -mag, mag) * torch.exp2(scales.double() - 127).repeat_interleave(32, -1)


def _close(got, want, what, rounded=ROUNDED):
    """One rounding of the result, and 1e-4 of its size for sums in 32 bits (K U = 3e-4 of the terms, which cancel)."""
    tol = rounded * want.abs() * 1.01 + 1e-4 * want.square().mean().sqrt()
    assert ((got.double() - want).abs() <= tol).all(), what


def _norm(v, kind):
    if kind == "layer":
        v = v - v.mean(-1, keepdim=True)
    return v / (v.square().mean(-1, keepdim=True) + 1e-6).sqrt()


def test_dense_block(block):
    p = block.inputs(tokens=96)
    out, mid = block.dense(p["stream"], p["attention"], p["mod"], p["up"], p["down"], p["up_bias"], p["down_bias"])
    gate, scale, shift, gate_mlp = (t.double().repeat_interleave(48, 0) for t in p["mod"].chunk(4, dim=1))
    h = p["stream"].double() + gate * p["attention"].double()
    _close(mid["h"], h, "h")
    _close(mid["y"], _norm(h, "layer") * (1 + scale) + shift, "y")
    u = _values(*mid["yq"]) @ _values(p["up"].codes, p["up"].scales).T + p["up_bias"].double()
    _close(mid["u"], torch.nn.functional.gelu(u, approximate="tanh"), "up")
    v = _values(*mid["uq"]) @ _values(p["down"].codes, p["down"].scales).T + p["down_bias"].double()
    _close(out, mid["h"].double() + gate_mlp * v, "down")


def test_expert_block(block):
    p = block.inputs(tokens=130, d=352, n_experts=5, expert_wide=96)
    out, mid = block.experts(p["stream"], p["attention"], p["weight"], p["post_weight"], p["router"], p["expert_up"],
                             p["expert_down"], 2)
    h = p["stream"].double() + _norm(p["attention"].double(), "rms") * p["post_weight"].double()
    _close(mid["h"], h, "h")
    _close(mid["y"], _norm(h, "rms") * p["weight"].double(), "y")
    off, rows = mid["offsets"].tolist(), mid["rows"].long()
    assert off[0] == 0 and off[-1] == 260
    a, b = _values(*mid["yq"]), _values(*mid["uq"])
    total = mid["h"].double()
    for e in range(5):
        r = slice(off[e], off[e + 1])
        q = a[rows[r]] @ _values(p["expert_up"].codes[e], p["expert_up"].scales[e]).T
        _close(mid["u"][r], torch.nn.functional.silu(q[:, 0::2]) * q[:, 1::2], f"up {e}")
        v = (b[r] @ _values(p["expert_down"].codes[e], p["expert_down"].scales[e]).T) * mid["row_weight"][r].double()[:, None]
        _close(mid["v"][r], v, f"down {e}", rounded=0.0)
        total.index_add_(0, rows[r], v)
    _close(out, total, "out")


def test_example_runs(block, capsys):
    block.main()
    assert "experts" in capsys.readouterr().out
