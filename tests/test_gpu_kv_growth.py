"""A step whose growth fails goes on to its writes and its attention, in a captured graph or
without the host's looking in between: the sequences that did not grow are left out of
them, so that their last tokens, and pages that they share, stay as they are."""
import numpy as np
import pytest
import torch

from tests import kv_reference as R

pytestmark = pytest.mark.gpu
D = 128
T = 16


def _W():
    from paper_2608_30877_gb300 import w4a16 as W
    return W


class Full:
    """A pool of which every page is in use: slot 0 a prefix of 21 tokens, slots 1 .. kids forks
    of it, slot `kids + 1` a sequence of two whole pages, and one of 5 tokens with room in its page."""

    def __init__(self, bits, kids=1, H=4, Hkv=2):
        W = _W()
        self.bits, self.kids, self.H, self.Hkv = bits, kids, H, Hkv
        self.own, self.roomy = kids + 1, kids + 2
        dtype = torch.bfloat16 if bits == 16 else torch.float8_e4m3fn
        self.c = W.KVCache(2, 5, Hkv, kids + 4, 6, T, dtype)
        self.c.pages.view(torch.uint8).fill_(0x11)
        if bits == 8:
            self.c.exponents.fill_(0x77)
        self.g = torch.Generator(device="cuda").manual_seed(bits + kids)
        W.kv_extend(self.c, R.i32([0, self.own, self.roomy]), R.i32([21, 32, 5]))
        for layer in range(2):
            W.kv_write(self.c, layer, self.rows(58), R.i32([0, 21, 53, 58]), R.i32([0, self.own, self.roomy]), H)
        W.kv_fork(self.c, R.i32([0] * kids), R.i32(range(1, kids + 1)))
        assert W.get_device_error() == W.OK
        assert int((self.c.page_refs > 0).sum()) == 5

    def rows(self, n):
        return torch.randn((n, (self.H + 2 * self.Hkv) * D), generator=self.g, device="cuda").bfloat16()

    def state(self):
        c = self.c
        held = [c.pages.view(torch.uint8), c.page_table, c.seq_len, c.page_refs]
        return [t.clone() for t in held + ([c.exponents] if self.bits == 8 else [])]

    def unchanged(self, state):
        return all(torch.equal(a, b) for a, b in zip(state, self.state()))

    def decode(self, slots, rows, layer=0):
        return _W().attention_decode(self.c, layer, rows, R.i32(slots), self.H)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("which", ["fork", "own"])
def test_attention_after_a_failed_growth(bits, which):
    W = _W()
    f = Full(bits)
    slots = [1] if which == "fork" else [f.own]
    state = f.state()
    rows = f.rows(1)
    W.kv_extend(f.c, R.i32(slots), R.i32([1]))
    outs = [f.decode(slots, rows, layer) for layer in range(2)]
    assert W.get_device_error() == W.ERR_CAPACITY
    assert f.unchanged(state)
    assert all((o == 0).all() for o in outs)
    # room is made, and the same step goes through
    W.kv_trim(f.c, R.i32([f.roomy]))
    W.kv_extend(f.c, R.i32(slots), R.i32([1]))
    out = f.decode(slots, rows)
    assert W.get_device_error() == W.OK
    assert torch.isfinite(out).all() and (out != 0).any()
    if which == "fork":
        assert torch.equal(f.c.pages.view(torch.uint8)[:, :, int(f.c.page_table[0, 1])],
                           state[0][:, :, int(f.c.page_table[0, 1])])


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("which", ["fork", "own"])
def test_writes_after_a_failed_growth(bits, which):
    W = _W()
    f = Full(bits)
    slots = [1] if which == "fork" else [f.own]
    state = f.state()
    W.kv_extend(f.c, R.i32(slots), R.i32([3]))
    for layer in range(2):
        W.kv_write(f.c, layer, f.rows(3), R.i32([0, 3]), R.i32(slots), f.H)
    assert W.get_device_error() == W.ERR_CAPACITY
    assert f.unchanged(state)


def test_what_else_goes_on():
    """Sequences that the failed call did not name, or asked no growth of, are as before; the others
    are back after a growth that succeeds (by 0 tokens too), or once they are trimmed."""
    W = _W()
    f = Full(16)
    rows = f.rows(3)
    want = f.decode([0], rows[:1])
    f.decode([f.roomy], rows[1:2])
    W.kv_extend(f.c, R.i32([f.own, 0, -1]), R.i32([17, 0, 4]))
    out = f.decode([0, f.roomy, f.own], rows)
    assert W.get_device_error() == W.ERR_CAPACITY
    assert torch.equal(out[0], want[0]) and (out[1] != 0).any() and (out[2] == 0).all()
    # as long as its growth has not succeeded, its rows are errors of their own
    assert (f.decode([f.own], rows[:1]) == 0).all()
    assert W.get_device_error() == W.ERR_INVALID_ARG
    W.kv_extend(f.c, R.i32([f.own]), R.i32([0]))
    assert (f.decode([f.own], rows[:1]) != 0).any()
    assert W.get_device_error() == W.OK
    W.kv_extend(f.c, R.i32([f.own]), R.i32([1]))
    W.kv_trim(f.c, R.i32([f.own]), R.i32([30]))
    assert (f.decode([f.own], rows[:1]) != 0).any()
    assert W.get_device_error() == W.ERR_CAPACITY
    # a slot that has been emptied and given another sequence
    W.kv_extend(f.c, R.i32([f.own]), R.i32([40]))
    W.kv_trim(f.c, R.i32([f.own]))
    W.kv_fork(f.c, R.i32([f.roomy]), R.i32([f.own]))
    assert W.get_device_error() == W.ERR_CAPACITY
    W.kv_extend(f.c, R.i32([f.own]), R.i32([1]))
    assert (f.decode([f.own], rows[:1]) != 0).any()
    assert W.get_device_error() == W.OK


@pytest.mark.parametrize("bits", [16, 8])
def test_a_captured_step_that_runs_out_of_pages(bits):
    """Forks of a prefix grown together in a replayed step until the pages run out: from then on
    nothing changes, and after a page is freed the step goes on from where it stopped."""
    W = _W()
    f = Full(bits, kids=3)
    W.kv_trim(f.c, R.i32([f.roomy]))
    W.kv_trim(f.c, R.i32([f.own]))  # three free pages: one copy for each fork, to the page's end
    slots, one = R.i32([1, 2, 3]), R.i32([1, 1, 1])
    qkv = f.rows(3)
    out = torch.empty((3, f.H * D), dtype=torch.bfloat16, device="cuda")
    workspace = f.c.new_workspace(f.H)

    def step():
        W.kv_extend(f.c, slots, one)
        for layer in range(2):
            W.attention_decode(f.c, layer, qkv, slots, f.H, out=out, workspace=workspace)

    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for t in range(11):  # tokens 21 .. 31
        qkv.copy_(f.rows(3))
        graph.replay()
        assert (out != 0).any(1).all()
    assert W.get_device_error() == W.OK
    assert f.c.seq_len.tolist()[:4] == [21, 32, 32, 32]
    state = f.state()
    for _ in range(3):
        qkv.copy_(f.rows(3))
        graph.replay()
        assert (out == 0).all()
    assert W.get_device_error() == W.ERR_CAPACITY
    assert f.unchanged(state)
    W.kv_trim(f.c, R.i32([0, 3]))
    slots.copy_(R.i32([1, 2, -1]))
    graph.replay()
    assert W.get_device_error() == W.OK
    assert (out[:2] != 0).any(1).all() and (out[2] == 0).all()
    assert f.c.seq_len.tolist()[:4] == [0, 33, 33, 0]


def test_a_refused_growth_of_many():
    """A list of more entries than the plan has threads, refused for one of them: none of its
    sequences is stored to, and all are back after one that is right."""
    W = _W()
    n = 2100
    c = W.KVCache(1, 2 * n + 4, 1, n + 1, 3, T)
    slots, ones = R.i32(range(n)), R.i32([1] * n)
    W.kv_extend(c, slots, R.i32([5] * n))
    qkv = torch.randn((n, 3 * D), device="cuda").bfloat16()
    c.pages.view(torch.uint8).fill_(0x11)
    first = W.attention_decode(c, 0, qkv, slots, 1)
    assert (first != 0).any(1).all()
    wrong = slots.clone()
    wrong[2050] = n + 1
    before = c.pages.clone()
    W.kv_extend(c, wrong, ones)
    out = W.attention_decode(c, 0, -qkv, slots, 1)
    assert W.get_device_error() == W.ERR_INVALID_ARG
    rest = torch.arange(n, device="cuda") != 2050
    assert (out[rest] == 0).all() and (out[2050] != 0).any()
    page = int(c.page_table[2050, 0])
    before[:, :, page] = c.pages[:, :, page]
    assert torch.equal(before, c.pages)
    W.kv_extend(c, slots, ones)
    assert (W.attention_decode(c, 0, qkv, slots, 1) != 0).any(1).all()
    assert W.get_device_error() == W.OK
    assert np.array_equal(c.seq_len.cpu().numpy()[:n], np.full(n, 6))


@pytest.mark.parametrize("make", ["new", "from_tensors"])
def test_a_cache_is_ready_for_any_stream(make):
    """A cache that is made while its stream is busy, and used at once on another one: the marks of
    a refused growth are not wiped out by what the constructor had queued."""
    W = _W()
    side = torch.cuda.Stream()
    one, zero = R.i32([1]), R.i32([0])
    tensors = [torch.zeros((1, 2, 2, 1, T, D), dtype=torch.bfloat16, device="cuda"),
               torch.zeros((1, 4), dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda"),
               torch.zeros(2, dtype=torch.int32, device="cuda")]
    qkv = torch.randn((1, 3 * D), device="cuda").bfloat16()
    many = R.i32([33])
    torch.cuda.synchronize()
    torch.cuda._sleep(100_000_000)  # 50 ms
    c = W.KVCache(1, 2, 1, 1, 4, T) if make == "new" else W.KVCache.from_tensors(*tensors)
    W.kv_extend(c, zero, one, stream=side)
    W.kv_extend(c, zero, many, stream=side)  # refused
    side.synchronize()
    torch.cuda.synchronize()
    assert W.get_device_error() == W.ERR_CAPACITY
    assert c.seq_len.tolist() == [1]
    out = W.attention_decode(c, 0, qkv, zero, 1)
    assert (out == 0).all() and W.get_device_error() == W.ERR_INVALID_ARG
