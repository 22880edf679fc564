"""What the 8-bit paged cache does with calls that were planned and not
finished: open blocks that have made way, rows that were never appended."""
import numpy as np
import pytest
import torch

from cache_reference import OPEN, values
from paper_2507_09252_amd import tppsd as tp
from test_gpu_cache import Both, ints

pytestmark = pytest.mark.gpu


def history(prec, dh, lens, L=2, S=None, n_pages=0, seed=0):
    b = Both(L, 2, 2, dh, prec, S or len(lens), 600, n_pages, seed)
    b.begin(max(lens), counts=list(lens) + [0] * ((S or len(lens)) - len(lens)))
    b.step(queries=False)
    b.commit()
    return b


def drop(b, P, seqs):
    """A call of P positions that is planned, appended and not committed (in the library alone)."""
    b.c.tppsd_cache_begin(P, ints(seqs))
    for layer in range(b.r.L):
        b.c.tppsd_cache_append(layer, b.rand(len(seqs), P, b.r.KV, b.r.dh), b.rand(len(seqs), P, b.r.KV, b.r.dh))


LOST = [("bf16", 64), ("fp32", 16)]


@pytest.mark.parametrize("prec,dh", LOST)
@pytest.mark.parametrize("more", [(), (3,), (200, 3)], ids=lambda m: "-".join(map(str, m)) or "once")
def test_lost_open_blocks_end_with_the_next_call(prec, dh, more):
    """A dropped call of 200 positions takes the open block's slots (100 = 64 +
    36 positions: its last blocks are 3 and 4, block 3 lies where 1 did). The
    next call says so and keeps nothing: the sequence goes back to its whole block."""
    b = history(prec, dh, [100, 64, 100], seed=1)
    for P in (200,) + more:
        drop(b, P, [0, 1])
    b.c.tppsd_cache_begin(4, ints([0, 1, 2]))
    for layer in range(2):
        b.c.tppsd_cache_attend(layer, b.rand(3, 4, 2, dh), b.rand(3, 4, 2, dh), b.rand(3, 4, 2, dh))
    b.c.tppsd_cache_commit(ints([4, 0, 0]))
    assert b.c.tppsd_cache_status() == OPEN
    assert b.c.lens.tolist() == [64, 64, 100]
    # what is left is sound: the sequence goes on as one of 64 positions does
    b.r.truncate([0], [64])
    b.r.status = OPEN
    for P in (70, 5, 64):
        b.begin(P)
        b.step()
        b.commit()
    for side in (0, 1):
        for s in range(3):
            got = values(b.c.tppsd_cache_read(0, None, 300)[side])[s]
            want = b.r.held_rows(s, side, 0, int(b.r.lens[s]))
            assert np.array_equal(got[:len(want)], want) and not got[len(want):].any()
    assert np.array_equal(b.c.lens.cpu().numpy(), b.r.lens)


@pytest.mark.parametrize("prec,dh", LOST)
@pytest.mark.parametrize("pairs", [1, 300])
def test_forks_and_copies_leave_lost_blocks_behind(prec, dh, pairs):
    S = pairs + 3
    b = history(prec, dh, [100, 130, 100], S=S, seed=2)
    drop(b, 200, [0, 1])
    dst = list(range(3, S))
    src = [x % 3 for x in range(pairs)]
    o = tp.Cache(2, 2, 2, dh, prec, S, 600)
    want = torch.tensor([[64, 128, 100][x] for x in src], dtype=torch.int32)
    o.tppsd_cache_copy(b.c, ints(src), ints(dst))
    b.c.tppsd_cache_fork(ints(src), ints(dst))
    for c in (o, b.c):
        assert torch.equal(c.lens[3:].cpu(), want)
        assert c.tppsd_cache_status() == OPEN
        k, v = c.tppsd_cache_read(1, None, 130, seqs=ints(dst))
        for side, got in ((0, values(k)), (1, values(v))):
            for i in (0, pairs // 2, pairs - 1):
                x = b.r.held_rows(src[i], side, 1, int(want[i]))
                assert np.array_equal(got[i, :len(x)], x) and not got[i, len(x):].any()


def test_read_gives_what_was_appended():
    """Neither a planned call's positions before their rows came, nor those of a call that another has taken the place of."""
    b = history("bf16", 32, [256, 40, 100], n_pages=10, seed=3)
    b.c.tppsd_cache_truncate(ints([0]))                       # its pages are free, their codes are still there
    b.r.truncate([0], [0])
    c, R = b.c, 200

    def reads(layer, s, n):
        """The rows of s are its first n positions and nothing else."""
        k, v = (torch.full((1, R, 2, 32), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        c.tppsd_cache_read(layer, None, R, k, v, seqs=ints([s]))
        for side, got in ((0, values(k)), (1, values(v))):
            want = b.r.held_rows(s, side, layer, n)
            assert np.array_equal(got[0, :n], want), (layer, s, side)
            assert (got[0, n:] == 7.0).all(), (layer, s, side)

    b.begin(130, seqs=[1, 2], counts=[130, 60])
    for layer in (0, 1):
        reads(layer, 1, 40)
        reads(layer, 2, 100)
    k, v = b.rand(2, 130, 2, 32), b.rand(2, 130, 2, 32)
    c.tppsd_cache_append(0, k, v)
    b.r.append(0, values(k), values(v))
    reads(0, 1, 170)
    reads(0, 2, 160)
    reads(1, 1, 40)
    reads(1, 2, 100)
    c.tppsd_cache_attend(1, b.rand(2, 130, 2, 32), k, v)
    b.r.append(1, values(k), values(v))
    reads(1, 1, 170)
    assert c.tppsd_cache_status() == 0
    # the call is dropped: by another call, by a truncation, by a fork
    c.tppsd_cache_begin(1, ints([0]))
    reads(0, 2, 64 + 36)                                      # (60 new positions: its block is still in the ring)
    assert c.tppsd_cache_status() == 0
    for op in (lambda: c.tppsd_cache_truncate(ints([0])), lambda: c.tppsd_cache_fork(ints([-1]), ints([-1])),
               lambda: c.tppsd_cache_copy(tp.Cache(2, 2, 2, 32, "bf16", 1, 64), ints([0]), ints([0]))):
        b.begin(20, seqs=[2])
        for layer in (0, 1):
            c.tppsd_cache_append(layer, k[:1, :20].contiguous(), v[:1, :20].contiguous())
            b.r.append(layer, values(k[:1, :20]), values(v[:1, :20]))
            reads(layer, 2, 120)
        op()
        reads(0, 2, 100)
    assert c.tppsd_cache_status() == 0
    # sequence 1's open block made way for the dropped call's last one
    reads(0, 1, 0)
    assert c.tppsd_cache_status() == OPEN
