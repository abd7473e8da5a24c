"""The binding's checks of include/resbm_train.h's calls, on the host: host tensors stand for device tensors, and a stand-in for
the library records what would have reached it."""
import pytest
import torch

from paper_2604_11947_gb300 import resbm


class Library:
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        return lambda *args: self.calls.append((name, args)) or resbm.RESBM_OK


@pytest.fixture
def lib(monkeypatch):
    lib = Library()
    monkeypatch.setattr(resbm, "_lib", lib)
    monkeypatch.setattr(resbm, "_device", lambda: torch.zeros(1).get_device())
    return lib


def norm(T=4, d=64, group=32, Q=None, groups=None):
    X, gamma = torch.zeros(T, d, dtype=torch.bfloat16), torch.zeros(d, dtype=torch.bfloat16)
    Q = torch.zeros(T, d, dtype=torch.uint8) if Q is None else Q
    groups = (-(-d // group) if group > 0 else 1) if groups is None else groups
    resbm.resbm_add_rmsnorm_fwd(X, None, gamma, 1e-5, None, None, Q, torch.zeros(T, groups), group, stream=0)


def test_a_norm_reaches_the_library(lib):
    norm()
    norm(group=0)
    norm(group=1 << 30)
    assert [name for name, _ in lib.calls] == ["resbm_add_rmsnorm_fwd"] * 3
    assert [args[0].q_group for _, args in lib.calls] == [32, 0, 1 << 30]


@pytest.mark.parametrize("group", [(1 << 32) + 32, (1 << 32), 32 - (1 << 32), -32, 1 << 31, 1 << 40])
def test_groups_that_the_descriptor_cannot_hold(lib, group):
    """A group over 32 bits would arrive as another one, whose scales S has no room for."""
    with pytest.raises(ValueError):
        norm(group=group)
    assert not lib.calls


@pytest.mark.parametrize("dtype", [torch.float8_e5m2, torch.int8, torch.bool, torch.float8_e4m3fnuz])
def test_codes_of_other_types(lib, dtype):
    """One-byte types that would read e4m3 codes as other values"""
    with pytest.raises(ValueError):
        norm(Q=torch.zeros(4, 64, dtype=torch.uint8).view(dtype))
    assert not lib.calls
    norm(Q=torch.zeros(4, 64, dtype=torch.uint8).view(torch.float8_e4m3fn))
    assert len(lib.calls) == 1


def test_workspace_of_the_norm_is_dense(lib):
    """An expanded tensor counts as its elements and is memory for one of them."""
    plan = type("Plan", (resbm.AdamWPlan,), {"__init__": lambda self: None})()
    plan.device, plan._fields, plan._address = torch.zeros(1).get_device(), {"g": []}, 0
    out = torch.zeros(2)
    for ws in (torch.zeros(1, dtype=torch.uint8).expand(1 << 20), torch.zeros(1 << 12, dtype=torch.uint8)[::2]):
        with pytest.raises(ValueError):
            resbm.resbm_grad_norm(plan, 1.0, out, ws, stream=0)
    assert not lib.calls
    resbm.resbm_grad_norm(plan, 1.0, out, torch.zeros(1 << 12, dtype=torch.uint8), stream=0)
    assert len(lib.calls) == 1
