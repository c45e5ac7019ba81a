"""Rotations and gradients that are recorded (CPU; the library's call is replaced by a recorder)."""
import pytest
import torch

from paper_2412_14838_amd import dkv
from paper_2412_14838_amd.pipeline import Compressor
from paper_2412_14838_amd.rotary import Rotary
from paper_2412_14838_amd.workloads import Workload


@pytest.fixture
def seen(monkeypatch):
    calls = []
    monkeypatch.setattr(dkv, "dkv_rotate", lambda *a, **kw: calls.append(a))
    monkeypatch.setattr(Rotary, "_on", lambda self, call, args, stream: call(*args, stream=stream))
    return calls


def test_tensors_whose_gradient_is_recorded_are_refused(seen):
    """The kernel writes behind autograd's back: a rotated tensor with its old history would get the gradient of the identity."""
    rot, positions = Rotary(8, dtype=dkv.DKV_F32, device="cpu"), torch.zeros(1, 3, dtype=torch.int32)
    plain = lambda: torch.zeros(1, 3, 2, 8)  # noqa: E731
    leaf = lambda: torch.zeros(1, 3, 2, 8, requires_grad=True)  # noqa: E731
    for make in (leaf, lambda: leaf() * 2.0, lambda: leaf().transpose(0, 1).transpose(0, 1)):
        for call in (lambda x: rot.rotate(positions, x), lambda x: rot.rotate(positions, x, q_out=plain()), lambda x: rot.rotate(positions, plain(), q_out=x),
                     lambda x: rot.rotate(positions, plain(), x), lambda x: rot.rotate(positions, plain(), x, k_out=plain()),
                     lambda x: rot.rotate(positions, plain(), plain(), k_out=x)):
            with pytest.raises(ValueError, match="gradient"):
                call(make())
            assert seen == []
            with torch.no_grad():
                call(make())
            assert len(seen) == 1
            seen.clear()
    rot.rotate(positions, plain(), (leaf() * 2.0).detach())
    assert len(seen) == 1


def test_a_prefill_refuses_them_too(seen):
    cfg = Workload(name="rotated", L=1, Hq=2, Hkv=1, d=64, seqlens=(40,), dtype="f32", w=4, P=7, mean_budget=8, layer_max=16, interval=1, seed=1)
    comp, rot = Compressor(cfg, device="cpu", keep_cache=False), Rotary(64, dtype=dkv.DKV_F32, device="cpu")
    q, k = torch.zeros(1, 2, 4, 64), torch.zeros(1, 40, 64)
    comp.rotate(rot, q, k)
    assert len(seen) == 2
    for a, b in ((q.clone().requires_grad_() * 1.0, k), (q, k.clone().requires_grad_() * 1.0)):
        with pytest.raises(ValueError, match="gradient"):
            comp.rotate(rot, a, b)
        assert len(seen) == 2                             # neither of the two is rotated
