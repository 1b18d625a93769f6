"""Lists that the page operations refuse, long enough that entries of many warps and of several
chunks take part, with what is wrong in any of them: whichever thread finds it, all threads
of the plan agree that the call ends, the status word says so and nothing has changed."""
import numpy as np
import pytest
import torch

from tests import kv_reference as R

pytestmark = pytest.mark.gpu


def _W():
    from paper_2608_30877_gb300 import w4a16 as W
    return W


def _cache(n, spare, T=16):
    """n sequences of 1 to 4 pages, and `spare` empty slots."""
    W = _W()
    lengths = [1 + 13 * i % (4 * T) for i in range(n)]
    c = W.KVCache(1, 5 * n, 1, n + spare, 6, T)
    W.kv_extend(c, R.i32(range(n)), R.i32(lengths))
    assert W.get_device_error() == W.OK
    return c, lengths


def _state(c):
    return [t.clone() for t in (c.page_table, c.seq_len, c.page_refs)]


def _refused(c, state, f, *lists):
    W = _W()
    f(c, *lists)
    assert W.get_device_error() == W.ERR_INVALID_ARG
    assert all(torch.equal(a, b) for a, b in zip(state, _state(c)))


@pytest.mark.parametrize("n", [3, 40, 1024, 2500])
def test_trims_that_are_refused(n):
    W = _W()
    c, lengths = _cache(n, 2)
    state = _state(c)
    order = np.random.default_rng(n).permutation(n)
    slots, keep = R.i32(order), R.i32([lengths[s] // 2 for s in order])
    places = sorted({0, 1, n // 2, n - 1, min(n - 1, 33), min(n - 1, 1025)})
    for at in places:
        for slot in (n + 2, -2, int(order[(at + 1) % n])):  # out of range, twice in the list
            wrong = slots.clone()
            wrong[at] = slot
            _refused(c, state, W.kv_trim, wrong, keep)
            _refused(c, state, W.kv_trim, wrong)
        for left in (-1, lengths[order[at]] + 1):
            wrong = keep.clone()
            wrong[at] = left
            _refused(c, state, W.kv_trim, slots, wrong)
        s = int(order[at])
        c.page_table[s, 0] = 5 * n  # a page out of range
        _refused(c, [c.page_table.clone(), *state[1:]], W.kv_trim, slots)
        c.page_table[s, 0] = state[0][s, 0]
        c.seq_len[s] = -1
        _refused(c, [state[0], c.seq_len.clone(), state[2]], W.kv_trim, slots)
        c.seq_len[s] = lengths[s]
    W.kv_trim(c, slots, keep)
    assert W.get_device_error() == W.OK
    assert c.seq_len[slots.long()].tolist() == keep.tolist()


@pytest.mark.parametrize("n", [3, 40, 1024, 2500])
def test_forks_that_are_refused(n):
    W = _W()
    c, lengths = _cache(n, n)
    state = _state(c)
    rng = np.random.default_rng(n)
    kids, parents = n + rng.permutation(n), rng.integers(0, n, n)
    places = sorted({0, 1, n // 2, n - 1, min(n - 1, 33), min(n - 1, 1025)})
    for at in places:
        for child in (2 * n, -2, int(kids[(at + 1) % n]), 0):  # out of range, twice, not empty
            wrong = kids.copy()
            wrong[at] = child
            _refused(c, state, W.kv_fork, R.i32(parents), R.i32(wrong))
        for parent in (2 * n, -1, int(kids[(at + 1) % n])):  # out of range, a child of the same call
            wrong = parents.copy()
            wrong[at] = parent
            _refused(c, state, W.kv_fork, R.i32(wrong), R.i32(kids))
        s = int(parents[at])
        c.page_table[s, 0] = -1
        _refused(c, [c.page_table.clone(), *state[1:]], W.kv_fork, R.i32(parents), R.i32(kids))
        c.page_table[s, 0] = state[0][s, 0]
    W.kv_fork(c, R.i32(parents), R.i32(kids))
    assert W.get_device_error() == W.OK
    assert c.seq_len[torch.as_tensor(kids, device="cuda")].tolist() == [lengths[p] for p in parents]


def test_refused_lists_over_and_over():
    """Many refused calls one behind the other, each launched while the one before it ends."""
    W = _W()
    n = 700
    c, lengths = _cache(n, 1)
    state = _state(c)
    for at in range(0, n, 7):
        wrong = R.i32(range(n))
        wrong[at] = n + 1 + at
        for _ in range(5):
            W.kv_trim(c, wrong)
    assert W.get_device_error() == W.ERR_INVALID_ARG
    assert all(torch.equal(a, b) for a, b in zip(state, _state(c)))
