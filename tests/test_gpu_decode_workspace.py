"""The workspace that a cache keeps for calls that name none: its counters are zero whatever
came before, a first call under capture or a call that timed out."""
import pytest
import torch

from tests.test_gpu_attention_decode import Case

pytestmark = pytest.mark.gpu
D = 128


def _W():
    from paper_2608_30877_gb300 import w4a16 as W
    return W


CASES = [(16, 8, 2, 64, [5000, 3, 700]), (8, 4, 4, 16, [3000, 2999]), (16, 40, 1, 32, [9000, 20])]


def _dirty_pool(size):
    """A graph whose pool has a free block of `size` bytes full of ones."""
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        block = torch.full((size,), 0xFF, dtype=torch.uint8, device="cuda")
        del block
    graph.replay()
    torch.cuda.synchronize()
    return graph


@pytest.mark.parametrize("bits,H,Hkv,T,lengths", CASES)
def test_first_call_under_capture(bits, H, Hkv, T, lengths):
    """The first call without a workspace is captured; calls before the graph's first replay,
    between its replays and after it is gone are right, and so are the replays."""
    W = _W()
    case = Case(bits, H, Hkv, T, lengths, 21)
    c = case.cache
    want = W.attention_decode(c, 1, case.qkv, case.slots, H, workspace=c.new_workspace(H))
    dirty = _dirty_pool(c.workspace_bytes(H))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, pool=dirty.pool()):
        out = W.attention_decode(c, 1, case.qkv, case.slots, H)
    assert torch.equal(W.attention_decode(c, 1, case.qkv, case.slots, H), want)
    for _ in range(3):
        out.fill_(7.0)
        graph.replay()
        assert torch.equal(out, want)
        assert torch.equal(W.attention_decode(c, 1, case.qkv, case.slots, H), want)
    graph.reset()
    dirty.reset()
    del out
    torch.cuda.empty_cache()
    other = torch.full((c.workspace_bytes(H),), 0xFF, dtype=torch.uint8, device="cuda")
    assert torch.equal(W.attention_decode(c, 1, case.qkv, case.slots, H), want)
    assert W.get_device_error() == W.OK and int(other[0]) == 0xFF


def test_a_cache_made_under_capture():
    W = _W()
    case = Case(16, 8, 2, 64, [5000, 3, 700], 22)
    c = case.cache
    want = W.attention_decode(c, 1, case.qkv, case.slots, 8)
    dirty = _dirty_pool(c.workspace_bytes(8))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, pool=dirty.pool()):
        made = W.KVCache.from_tensors(c.pages, c.page_table, c.seq_len, c.page_refs)
        outs = [W.attention_decode(made, 1, case.qkv, case.slots, 8) for _ in range(3)]
    assert torch.equal(W.attention_decode(made, 1, case.qkv, case.slots, 8), want)
    for _ in range(2):
        graph.replay()
        assert all(torch.equal(o, want) for o in outs)
        assert torch.equal(W.attention_decode(made, 1, case.qkv, case.slots, 8), want)
    assert W.get_device_error() == W.OK


def test_heads_in_turn():
    """Calls with other numbers of query heads on one cache, each as with a workspace of its own."""
    W = _W()
    cases = [Case(16, H, 2, 32, [4000, 50, 900], 23) for H in (2, 6, 16, 34, 130)]
    c = cases[0].cache
    for case in cases[1:]:
        assert torch.equal(case.cache.page_table, c.page_table)
        case.cache = c
    want = [W.attention_decode(c, 1, x.qkv, x.slots, x.H, workspace=c.new_workspace(x.H)) for x in cases]
    for order in ((0, 1, 2, 3, 4), (4, 0, 3, 1, 2)):
        for i in order:
            # (the cache holds the last call's new tokens: every call stores its own first)
            x = cases[i]
            assert torch.equal(W.attention_decode(c, 1, x.qkv, x.slots, x.H), want[i])
    assert W.get_device_error() == W.OK


@pytest.mark.parametrize("bits,H,Hkv,T,lengths", [(16, 8, 8, 64, [20000, 30000]), (8, 16, 8, 64, [40000, 9])])
def test_after_a_timeout(bits, H, Hkv, T, lengths):
    """A call that gave up leaves some of a row's parts counted (here with limits at which some of
    the CTAs' first copies are in time).  Once its error is read, calls and replayed graphs
    that use the cache's own workspace are right again.  (Queries differ from call to call, so that
    a part of another call is not the same.)"""
    W = _W()
    case = Case(bits, H, Hkv, T, lengths, 24)
    c = case.cache
    rows = [case.qkv, case.qkv.roll(D, 1).mul(-0.5)]
    want = [W.attention_decode(c, 1, r, case.slots, H) for r in rows]
    qkv = rows[0].clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = W.attention_decode(c, 1, qkv, case.slots, H)
    assert W.get_device_error() == W.OK
    timeouts = 0
    for limit in [1, 200] + 3 * list(range(600, 2000, 100)):  # ns
        W.set_wait_limit(limit)
        try:
            W.attention_decode(c, 1, case.qkv, case.slots, H)
            timeouts += W.get_device_error() == W.ERR_TIMEOUT
        finally:
            W.set_wait_limit(0)
        for r, w in zip(rows[::-1], want[::-1]):
            assert torch.equal(W.attention_decode(c, 1, r, case.slots, H), w), limit
        for r, w in zip(rows[::-1], want[::-1]):
            qkv.copy_(r)
            graph.replay()
            assert torch.equal(out, w), limit
        assert W.get_device_error() == W.OK
    assert timeouts > 0


def test_another_error_before_the_timeout():
    """The status word keeps the first error, which may hide a timeout: reading any of them
    makes the workspace ready."""
    W = _W()
    case = Case(16, 8, 8, 64, [20000, 30000], 25)
    c, H = case.cache, 8
    rows = [case.qkv, case.qkv.roll(D, 1).mul(-0.5)]
    want = [W.attention_decode(c, 1, r, case.slots, H) for r in rows]
    wrong = torch.full_like(case.slots, c.num_slots)
    for limit in 3 * list(range(600, 2000, 100)):
        W.attention_decode(c, 1, rows[0], wrong, H)
        W.set_wait_limit(limit)
        try:
            W.attention_decode(c, 1, rows[0], case.slots, H)
            assert W.get_device_error() == W.ERR_INVALID_ARG
        finally:
            W.set_wait_limit(0)
        for r, w in zip(rows[::-1], want[::-1]):
            assert torch.equal(W.attention_decode(c, 1, r, case.slots, H), w), limit
        assert W.get_device_error() == W.OK
