"""Forks of sampler states: what the binding refuses (no GPU needed)."""
import pytest
import torch

from paper_2507_09252_amd import tppsd as tp


def test_fork_from_a_state_on_another_device():
    a, b = tp.State.__new__(tp.State), tp.State.__new__(tp.State)
    a.B, a.ws, a.handle = 2, torch.empty(1), None
    b.B, b.ws, b.handle = 2, torch.empty(1, device="meta"), None
    with pytest.raises(tp.TppsdError, match="device"):
        a.tppsd_state_fork(b, torch.zeros(2, dtype=torch.int32))
