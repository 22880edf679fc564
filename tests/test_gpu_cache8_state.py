"""Sampler states whose target keeps its keys and values in the 8-bit paged
cache (TPPSD_FLAG_CACHE8), and states continued by tppsd_state_fork, with
either cache."""
import numpy as np
import pytest
import torch

from cache8_oracle import Model8
from gpu_common import (Case, draft_buffers_from_oracle, draft_out, f32_round, histories, oracle_models,
                        replay_ar_steps, replay_sd_rounds, to_dev, tol_of, verify_out, weights)
from oracle import sampler as S
from paper_2507_09252_amd import tppsd as tp
from paper_2507_09252_amd import workloads as W

pytestmark = pytest.mark.gpu

A1 = W.Workload("a1", 6, W.ModelCfg(2, 32, 2, 0, 4, 3, "fp32", W.ENC_ATTNHP, 0.5, 20.0),
                W.ModelCfg(1, 16, 1, 0, 4, 3, "fp32", W.ENC_ATTNHP, 0.5, 20.0),
                batch=8, n_gen=64, gammas=(4,), n_hist=20, history="ipp_sin", description="small fp32 AttNHP")


def case(wl, B, n_hist, init="stress"):
    wl = wl if isinstance(wl, W.Workload) else W.WORKLOADS[wl]
    return Case(f"{wl.name}-B{B}-h{n_hist}-{init}", wl, B, n_hist, init, True)


def state(c, wt, wd, gamma, n_gen, seed, B=None, extra=0, draft=True, cache8=True, models=None):
    tm, dm = models or (tp.Model(c.wl.target, wt), tp.Model(c.wl.draft, wd) if draft else None)
    st = tp.State(tm, dm, B or c.B, c.n_hist + n_gen + gamma + 1 + extra, gamma, seed=seed, cache8=cache8)
    st._models = (tm, dm)
    return st


VERIFY = [case("c1", 2, 200), case("c2", 5, 150), case("c2", 5, 65), case(A1, 4, 130), case("c3", 3, 140, "bias"),
          case("c5", 4, 127, "bias"), case("c4", 2, 190, "bias"), case("a3", 2, 100, "bias")]


@pytest.mark.parametrize("c", VERIFY, ids=[c.name for c in VERIFY])
def test_verify_against_the_oracle(c):
    """Decoder outputs of a verify pass after histories that fill pages.

    Where the kernel's key or value rounds to the other neighbour than the
    float64 one, which its own precision allows, its e4m3 code moves by a whole
    step where that lies at a tie. What such roundings are worth at the outputs
    is measured on the oracle: keys and values changed at random by up to one
    rounding of the model's type (bf16 2^-8; fp32 2^-20, its accumulated sums)
    move its outputs by `drift` (the largest of four runs); twice that is added
    to the workload's tolerance."""
    gamma, n_gen, seed = c.g, 40, 3
    wt, wd = weights(c)
    T, D = Model8(c.wl.target, wt), oracle_models(c, wt, wd)[1]
    ht, hk = histories(c)
    rows = np.arange(c.B)
    ost = S.prefill(T, D, ht, hk, n_gen)
    dr = S.draft(D, ost, gamma, seed, rows)
    vf = S.verify(T, ost, dr, rows)
    drift = 0.0
    for r in range(4):
        J = Model8(c.wl.target, wt, 2.0 ** -8 if c.wl.prec == "bf16" else 2.0 ** -20, r)
        vj = S.verify(J, S.prefill(J, D, ht, hk, n_gen), dr, rows)
        drift = max([drift] + [np.abs(getattr(vj, f) - getattr(vf, f)).max() for f in ("logw", "mu", "s", "logtype")])
    M, K = c.wl.target.n_mix, c.wl.target.n_types
    st = state(c, wt, wd, gamma, n_gen, seed)
    st.tppsd_prefill(to_dev(ht), to_dev(hk), n_gen)
    dbuf, vbuf = draft_buffers_from_oracle(dr, c.B, gamma, M, K), tp.VerifyBuffers(c.B, gamma, M, K)
    for call in (st.tppsd_verify, st.tppsd_verify_noalloc):
        call(gamma, dbuf, vbuf)
        got = verify_out(vbuf, rows, gamma)
        tol = tol_of(c.wl) + 2 * drift
        err = max(np.abs(getattr(got, f) - getattr(vf, f)).max() for f in ("logw", "mu", "s", "logtype"))
        print(f"{c.name}: max abs err {err:.2e} (tol {tol:.2e}, drift {drift:.2e})")
        assert err <= tol
        assert st.tppsd_state_status()["bits"] == 0
    # and not the outputs of the 16-bit or fp32 cache
    V = S.verify(oracle_models(c, wt, wd)[0], S.prefill(oracle_models(c, wt, wd)[0], D, ht, hk, n_gen), dr, rows)
    far = max(np.abs(getattr(V, f) - getattr(vf, f)).max() for f in ("logw", "mu", "s", "logtype"))
    print(f"{c.name}: 8-bit cache against none {far:.2e}")


@pytest.mark.parametrize("c", [case("c1", 2, 60, "bias"), case("c2", 3, 100, "bias"), case(A1, 3, 50, "bias")],
                         ids=lambda c: c.name)
@pytest.mark.parametrize("kind", ["ar", "sd"])
def test_sampling_replayed_into_the_oracle(c, kind):
    """AR steps and TPP-SD rounds over block borders, each replayed from the events committed before it."""
    gamma, n_gen, seed = c.g, 24, 29
    wt, wd = weights(c)
    T, D = Model8(c.wl.target, wt), oracle_models(c, wt, wd)[1]
    ht, hk = histories(c)
    st = state(c, wt, wd, gamma, n_gen, seed, draft=kind == "sd")
    st.tppsd_prefill(to_dev(ht), to_dev(hk), n_gen)
    if kind == "ar":
        compared, generated = replay_ar_steps(c, T, st, seed, n_gen)
    else:
        compared, generated = replay_sd_rounds(c, T, D, st, gamma, seed, n_gen)[:2]
    status = st.tppsd_state_status()
    assert status["bits"] == 0 and status["n_done"] == c.B
    assert generated == c.B * n_gen and compared >= 0.5 * generated


@pytest.mark.parametrize("c", [case("c2", 40, 70), case("c5", 64, 60), case("c4", 4, 600)], ids=lambda c: c.name)
def test_jobs_repeat_and_end(c):
    """Whole jobs, captured rounds and steps: finished, repeatable after a new prefill, no status."""
    gamma, n_gen, seed = c.g, 90, 5
    wt, wd = weights(c)
    ht, hk = (to_dev(x) for x in histories(c))
    st, runs = state(c, wt, wd, gamma, n_gen, seed), []
    for _ in range(2):
        st.tppsd_prefill(ht, hk, n_gen)
        st.tppsd_sample_sd(gamma)
        t, k, n = (x.clone() for x in st.tppsd_read_events())
        end = c.n_hist + n_gen
        assert (n == end).all() and torch.isfinite(st.tppsd_read_loglik()).all()
        assert st.tppsd_state_status()["bits"] == 0
        # (times are float32 running sums: an interval below 2^-14, half their spacing past 1024, leaves one as it is)
        assert (t[:, 1:end] >= t[:, :end - 1]).all()
        runs.append((t[:, :end], k[:, :end], st.tppsd_read_loglik()))
    assert all(torch.equal(a, b) for a, b in zip(*runs))
    st.tppsd_prefill(ht, hk, 20)
    st.tppsd_sample_ar(20)
    assert (st.tppsd_read_events()[2] == c.n_hist + 20).all()


def test_flags_and_sizes():
    wl = W.WORKLOADS["c4"]
    c = case("c4", 2, 512, "bias")
    wt, wd = weights(c)
    a, b = (state(c, wt, wd, 16, 4096, 1, B=32, cache8=x) for x in (False, True))
    slabs = 2 * wl.target.n_layers * wl.target.d_model * 32 * (512 + 4096 + 17) * 2
    assert a.ws.numel() - b.ws.numel() > 0.4 * slabs     # half of the slabs, less the tails and scratch
    with pytest.raises(tp.TppsdError, match="E_WORKSPACE"):
        tp._check(tp.lib().tppsd_state_create(b.target.handle, b.draft.handle, 32, 4625, 16, 0, 2, tp._ptr(b.ws),
                                              b.ws.numel() // 4, tp.ctypes.byref(tp.c_void_p())))


FORKS = [(case("c2", 4, 100), False), (case("c2", 4, 100), True), (case("c5", 5, 120), False),
         (case("c5", 5, 120), True), (case("c3", 3, 130, "bias"), True), (case("c3", 3, 130, "bias"), False),
         (case(A1, 4, 70), True), (case(A1, 4, 70), False)]
FORK_IDS = [f"{c.name}-{'8bit' if q else 'slab'}" for c, q in FORKS]


@pytest.mark.parametrize("c,cache8", FORKS, ids=FORK_IDS)
def test_a_job_moves_to_a_larger_state(c, cache8):
    """Every sequence of a job half-way goes to a state of the same seed with more room: it ends as the job does."""
    gamma, n_gen, seed = c.g, 60, 7
    wt, wd = weights(c)
    ht, hk = (to_dev(x) for x in histories(c))
    a = state(c, wt, wd, gamma, n_gen, seed, cache8=cache8)
    a.tppsd_prefill(ht, hk, n_gen)
    a.tppsd_sample_sd(gamma, 3)
    b = state(c, wt, wd, gamma, n_gen, seed, extra=77, cache8=cache8, models=a._models)
    b.tppsd_state_fork(a, torch.arange(c.B, device="cuda"))
    assert b.tppsd_state_status()["drafted"] == 0
    end = c.n_hist + n_gen
    for st in (a, b):
        st.tppsd_sample_sd(gamma)
    (ta, ka, na), (tb, kb, nb) = a.tppsd_read_events(), b.tppsd_read_events()
    assert torch.equal(na, nb) and (na == end).all()
    assert torch.equal(ta[:, :end], tb[:, :end]) and torch.equal(ka[:, :end], kb[:, :end])
    assert torch.equal(a.tppsd_read_loglik(), b.tppsd_read_loglik())
    assert b.tppsd_state_status()["bits"] == 0


@pytest.mark.parametrize("c,cache8", FORKS, ids=FORK_IDS)
def test_continuations(c, cache8):
    """Histories encoded once are continued by several sequences each: the
    rounds after the fork are the oracle's for that history and that sequence's
    own draws."""
    gamma, n_gen, seed, fan = c.g, 12, 11, 3
    wt, wd = weights(c)
    ht, hk = histories(c)
    a = state(c, wt, wd, gamma, n_gen, 999, cache8=cache8)
    a.tppsd_prefill(to_dev(ht), to_dev(hk), n_gen)
    parent = (np.arange(c.B * fan) * 2) % c.B
    b = state(c, wt, wd, gamma, n_gen, seed, B=c.B * fan, cache8=cache8, models=a._models)
    b.tppsd_state_fork(a, to_dev(parent))
    t, k, n = (x.cpu().numpy() for x in b.tppsd_read_events())
    assert (n == c.n_hist).all() and np.array_equal(t[:, :c.n_hist], ht[parent]) and np.array_equal(k[:, :c.n_hist], hk[parent])
    # the same job from histories encoded by the state itself
    ref = state(c, wt, wd, gamma, n_gen, seed, B=c.B * fan, cache8=cache8, models=a._models)
    ref.tppsd_prefill(to_dev(ht[parent]), to_dev(hk[parent]), n_gen)
    M, K = c.wl.target.n_mix, c.wl.target.n_types
    bufs = [(tp.DraftBuffers(b.B, gamma, M, K), tp.VerifyBuffers(b.B, gamma, M, K)) for _ in range(2)]
    for st, (d, v) in zip((b, ref), bufs):
        st.tppsd_draft(gamma, d)
        st.tppsd_verify(gamma, bufs[0][0], v)
    # (encodings of other batch sizes may run in other kernels: roundings of the model's type)
    tol = 2 * tol_of(c.wl) if c.init == "bias" or c.wl.prec == "fp32" else 0.1
    for f in ("tau", "mix", "logtype"):
        x, y = (getattr(d, f)[:, 0] for d, _ in bufs)
        assert (x - y).abs().max() <= tol * max(1.0, float(y.abs().max())), f
    for f in ("mix", "logtype"):
        x, y = (getattr(v, f) for _, v in bufs)
        assert (x - y).abs().max() <= tol, (f, (x - y).abs().max())
    b.tppsd_sample_sd(gamma)
    t, k, n = b.tppsd_read_events()
    assert (n == c.n_hist + n_gen).all() and b.tppsd_state_status()["bits"] == 0
    assert len({tuple(x) for x in t[:, c.n_hist:c.n_hist + n_gen].tolist()}) == b.B     # each its own draws
    a.tppsd_sample_sd(gamma)                                                             # the source is untouched
    assert (a.tppsd_read_events()[2] == c.n_hist + n_gen).all() and a.tppsd_state_status()["bits"] == 0


@pytest.mark.parametrize("c,cache8", FORKS, ids=FORK_IDS)
def test_particles_resampled(c, cache8):
    """Sequences replaced by others of the same state between rounds; draws of
    the copies are those of counters nobody has used."""
    gamma, n_gen, seed = c.g, 60, 13
    wt, wd = weights(c)
    ht, hk = histories(c)
    st = state(c, wt, wd, gamma, n_gen, seed, cache8=cache8)
    st.tppsd_prefill(to_dev(ht), to_dev(hk), n_gen)
    st.tppsd_sample_sd(gamma, 2)
    t0, k0, n0 = (x.clone() for x in st.tppsd_read_events())
    l0 = st.tppsd_read_loglik()
    parent = [0] * c.B
    parent[-1] = c.B - 1                                      # all but the last continue the first
    st.tppsd_state_fork(st, torch.tensor(parent, device="cuda"))
    t1, k1, n1 = st.tppsd_read_events()
    for b, p in enumerate(parent):
        m = int(n0[p])
        assert int(n1[b]) == m and torch.equal(t1[b, :m], t0[p, :m]) and torch.equal(k1[b, :m], k0[p, :m])
    assert torch.equal(st.tppsd_read_loglik(), l0[parent])
    # bad parents: out of range, or not their own
    bad = list(range(c.B))
    bad[1], bad[2] = 2, 0
    st.tppsd_state_fork(st, torch.tensor(bad, device="cuda"))
    assert st.tppsd_state_status()["bits"] == tp.STATUS_SEQUENCE
    assert torch.equal(st.tppsd_read_events()[2][1], n1[1])
    st.tppsd_sample_sd(gamma)
    t2, k2, n2 = st.tppsd_read_events()
    end = c.n_hist + n_gen
    assert (n2 == end).all() and st.tppsd_state_status()["bits"] == tp.STATUS_SEQUENCE
    assert len({tuple(x) for x in t2[:, :end].tolist()}) == c.B
    assert torch.isfinite(st.tppsd_read_loglik()).all()


def test_forked_draws_use_their_own_counters():
    """After a fork within a state the first round's drafts are the oracle's for round counter 2^20."""
    from gpu_common import check_draft_record, oracle_state_from_gpu
    c = case("c2", 3, 80)
    gamma, n_gen, seed = c.g, 30, 17
    wt, wd = weights(c)
    T, D = oracle_models(c, wt, wd)
    ht, hk = histories(c)
    st = state(c, wt, wd, gamma, n_gen, seed, cache8=False)
    st.tppsd_prefill(to_dev(ht), to_dev(hk), n_gen)
    st.tppsd_sample_sd(gamma, 1)
    st.tppsd_state_fork(st, torch.tensor([0, 0, 2], device="cuda"))
    t, k, n = (x.cpu().numpy() for x in st.tppsd_read_events())
    dbuf = tp.DraftBuffers(3, gamma, c.wl.target.n_mix, c.wl.target.n_types)
    st.tppsd_draft(gamma, dbuf)
    for b, rnd in ((0, 1), (1, 1 << 20), (2, 1)):
        ost = oracle_state_from_gpu(T, D, t, k, int(n[b]), b, n_gen, int(n[b]) - c.n_hist, rnd)
        assert check_draft_record(D, ost, draft_out(dbuf, [b], gamma), gamma, seed, rnd, [b], tol_of(c.wl), str(b))


def test_fork_refusals():
    c = case("c2", 2, 40)
    wt, wd = weights(c)
    a = state(c, wt, wd, 4, 10, 1)
    parent = torch.zeros(2, dtype=torch.int32, device="cuda")
    with pytest.raises(tp.TppsdError, match="E_ORDER"):
        a.tppsd_state_fork(a, parent)
    ht, hk = (to_dev(x) for x in histories(c))
    a.tppsd_prefill(ht, hk, 10)
    for other, err in ((state(c, wt, wd, 4, 10, 1), "E_CONFIG"), (state(c, wt, wd, 4, 10, 1, cache8=False, models=a._models), "E_CONFIG"),
                       (state(c, wt, wd, 4, 9, 1, models=a._models), "E_ARG")):
        with pytest.raises(tp.TppsdError, match=err):
            other.tppsd_state_fork(a, parent)
    b = state(c, wt, wd, 4, 10, 1, B=3, models=a._models)
    b.tppsd_state_fork(a, torch.tensor([1, 5, -1], device="cuda"))      # two have no parent: empty and finished
    assert b.tppsd_read_events()[2].tolist() == [40, 0, 0]
    s = b.tppsd_state_status()
    assert s["bits"] == tp.STATUS_SEQUENCE and s["n_done"] == 2
    b.tppsd_sample_sd(4)
    assert b.tppsd_read_events()[2].tolist() == [50, 0, 0]


@pytest.mark.parametrize("cache8", [False, True])
def test_poisson_and_windowed_jobs_fork(cache8):
    """States without a draft model, and with end times: forks take both along."""
    c = case("c2", 3, 70)
    wt, wd = weights(c)
    ht, hk = (to_dev(x) for x in histories(c))
    params = tp.tppsd_poisson_fit(ht, hk, c.wl.target.n_types)
    a = state(c, wt, wd, 4, 30, 5, draft=False, cache8=cache8)
    a.tppsd_prefill(ht, hk, 30)
    a.tppsd_sample_sd_poisson(4, params, 2)
    b = state(c, wt, wd, 4, 30, 5, cache8=cache8, models=a._models, extra=9)
    b.tppsd_state_fork(a, torch.arange(3, device="cuda"))
    for st in (a, b):
        st.tppsd_sample_sd_poisson(4, params)
    assert torch.equal(a.tppsd_read_events()[0][:, :100], b.tppsd_read_events()[0][:, :100])
    end = ht[:, -1] + torch.tensor([0.0, 5.0, 1e6], device="cuda")
    a = state(c, wt, wd, 4, 30, 5, cache8=cache8)
    a.tppsd_prefill(ht, hk, 30, t_end=end)
    b = state(c, wt, wd, 4, 30, 5, cache8=cache8, models=a._models)
    b.tppsd_state_fork(a, torch.tensor([2, 1, 0], device="cuda"))
    assert b.tppsd_state_status()["n_done"] == 1
    b.tppsd_sample_sd(4)
    t, _, n = b.tppsd_read_events()
    assert n[2] == 70 and n[0] == 100 and t[1, int(n[1]) - 1] <= end[1]
    assert b.tppsd_state_status()["bits"] == 0
