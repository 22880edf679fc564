"""What the 8-bit paged cache computes, whichever way a sequence is cut into
calls, and that a sampler state asked for it uses it."""
import numpy as np
import pytest

from cache8_oracle import Model8
from gpu_common import draft_buffers_from_oracle, histories, oracle_models, to_dev, tol_of, verify_out, weights
from oracle import sampler as S
from paper_2507_09252_amd import tppsd as tp
from test_gpu_cache import Both
from test_gpu_cache8_state import case, state

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("prec,dh", [("bf16", 64), ("fp32", 32), ("bf16", 128)])
@pytest.mark.parametrize("chunk", [300, 100, 64, 37, 16, 1])
def test_every_chunking_is_the_definition(prec, dh, chunk):
    """300 positions in chunks of each length, every output within the bound of its own roundings."""
    b = Both(1, 2, 2, dh, prec, 1, 300, seed=8)
    for a in range(0, 300, chunk):
        b.begin(min(chunk, 300 - a))
        b.step()
        b.commit()
    b.same(0)


FIELDS = ("logw", "mu", "s", "logtype")


@pytest.mark.parametrize("c", [case("c1", 2, 200), case("c2", 5, 150)], ids=lambda c: c.name)
def test_a_state_with_the_flag_reads_8_bits(c):
    """fp32 states with and without the flag, on the same drafts, are as far
    from each other as the two definitions are, to within the tolerance of each
    (1e-5): 8-bit rounding of the keys and values is worth a hundred times that."""
    gamma, n_gen = c.g, 40
    wt, wd = weights(c)
    T8, (T, D) = Model8(c.wl.target, wt), oracle_models(c, wt, wd)
    ht, hk = histories(c)
    rows = np.arange(c.B)
    ost = S.prefill(T, D, ht, hk, n_gen)
    dr = S.draft(D, ost, gamma, 3, rows)
    plain, eight = S.verify(T, ost, dr, rows), S.verify(T8, S.prefill(T8, D, ht, hk, n_gen), dr, rows)
    far = {f: np.abs(getattr(plain, f) - getattr(eight, f)).max() for f in FIELDS}
    assert max(far.values()) > 100 * tol_of(c.wl)
    M, K = c.wl.target.n_mix, c.wl.target.n_types
    got = []
    for cache8 in (False, True):
        st = state(c, wt, wd, gamma, n_gen, 3, cache8=cache8)
        st.tppsd_prefill(to_dev(ht), to_dev(hk), n_gen)
        d, v = draft_buffers_from_oracle(dr, c.B, gamma, M, K), tp.VerifyBuffers(c.B, gamma, M, K)
        st.tppsd_verify(gamma, d, v)
        got.append(verify_out(v, rows, gamma))
    for f in FIELDS:
        x = np.abs(getattr(got[0], f) - getattr(got[1], f)).max()
        # (codes at ties may fall the other way: half of the distance is far from none)
        assert x >= far[f] / 2 - 2 * tol_of(c.wl), (f, x, far[f])
