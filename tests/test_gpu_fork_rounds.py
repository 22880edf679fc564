"""A fork in the middle of a round: what was verified before it is not accepted after it."""
import pytest
import torch

from gpu_common import histories, to_dev, weights
from paper_2507_09252_amd import tppsd as tp
from test_gpu_cache8_state import case, state

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cache8", [False, True], ids=["slab", "8bit"])
@pytest.mark.parametrize("within", [True, False], ids=["within", "to-another"])
def test_accept_after_a_fork_needs_a_verify(cache8, within):
    c = case("c2", 3, 62)
    gamma, n_gen = 4, 20
    wt, wd = weights(c)
    ht, hk = (to_dev(x) for x in histories(c))
    a = state(c, wt, wd, gamma, n_gen, 1, cache8=cache8)
    a.tppsd_prefill(ht, hk, n_gen)
    to = a if within else state(c, wt, wd, gamma, n_gen, 2, cache8=cache8, models=a._models)
    if not within:
        to.tppsd_prefill(ht, hk, n_gen)
    M, K = c.wl.target.n_mix, c.wl.target.n_types
    d, v, x = tp.DraftBuffers(3, gamma, M, K), tp.VerifyBuffers(3, gamma, M, K), tp.AcceptBuffers(3, gamma)
    to.tppsd_draft(gamma, d)
    to.tppsd_verify(gamma, d, v)
    to.tppsd_state_fork(a, torch.tensor([0, 0, 2], device="cuda"))
    with pytest.raises(tp.TppsdError, match="E_ORDER"):
        to.tppsd_accept(gamma, d, v, x)
    assert to.tppsd_read_events()[2].tolist() == [62] * 3
    to.tppsd_draft(gamma, d)
    for verify in (to.tppsd_verify, to.tppsd_verify_noalloc):
        verify(gamma, d, v)
    to.tppsd_accept(gamma, d, v, x)
    assert (to.tppsd_read_events()[2] > 62).all()
    to.tppsd_sample_sd(gamma)
    assert (to.tppsd_read_events()[2] == 62 + n_gen).all() and to.tppsd_state_status()["bits"] == 0
