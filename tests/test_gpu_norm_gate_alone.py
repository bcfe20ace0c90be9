"""The gradient at the branch's output under a gate, with no norm of the branch and no gradient of the gate: dy = gate (.) dh' needs no y.  Against
the formula in 64 bits (bounds as in test_gpu_block_norm.py), and against the same call that is given y, on both sides of the width beyond which
rows no longer go through the ring in shared memory."""
import pytest
import torch

from paper_2510_05528_b200 import binding as Bd
from tests.test_gpu_block_norm import PAIRS, SUM, backward64, close, inputs

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def ctx():
    c = Bd.ArmorContext(1024, 1024, 128, device=DEV, h_mode=Bd.H_DIAG)
    yield c
    assert c.device_status()[:4] == [0, 0, 0, 0]


@pytest.mark.parametrize("ts,tb", PAIRS)
@pytest.mark.parametrize("rows,d,gates,per_gate", [(1, 520, 1, 1), (37, 517, 3, 13), (700, 520, 5, 140), (700, 33, 234, 3), (400, 5360, 3, 150), (320, 8200, 7, 50),
                                                   (20, 9000, 2, 10), (500, 9001, 4, 130)])
def test_gate_without_y(ctx, rows, d, gates, per_gate, ts, tb):
    t = inputs(rows, d, ts, tb, post=False, gates=gates, per_gate=per_gate)
    kw = dict(gate=t["gate"], rows_per_gate=per_gate, w_pre=t["w_pre"], residual_scale=0.5)

    def call(y):
        dx, dy, dw_pre = torch.empty_like(t["dh"]), torch.empty_like(t["dn"]), torch.empty(d, device=DEV)
        Bd.armor_block_norm_backward(ctx.ctx, t["x"], y, t["dh"], t["dn"], dx, dy, None, dw_pre, None, **kw)
        return {"dx": dx, "dy": dy, "dw_pre": dw_pre}
    got = call(None)
    want, sizes = backward64(t, t["x"], post=False, a=0.5)
    for name, v in got.items():
        close(v, want[name], 2 * SUM * sizes[name])
    # (with y the sums of a row are formed beside others, with the same terms in the same places)
    for name, v in call(t["y"]).items():
        close(v, want[name], 2 * SUM * sizes[name])


def test_gate_without_y_without_a_norm(ctx):
    """Neither norm: dx and dy are the sum of the two gradients, the latter under the gate."""
    t = inputs(300, 264, torch.float32, torch.float32, post=False, gates=3, per_gate=100)
    dx, dy = torch.empty_like(t["dh"]), torch.empty_like(t["dh"])
    Bd.armor_block_norm_backward(ctx.ctx, None, None, t["dh"], t["dn"], dx, dy, None, None, None, gate=t["gate"], rows_per_gate=100, pre=False)
    assert torch.equal(dx, t["dh"] + t["dn"])
    assert torch.equal(dy, (t["dh"] + t["dn"]) * t["gate"].repeat_interleave(100, 0))
