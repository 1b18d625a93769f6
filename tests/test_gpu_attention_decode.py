"""Attention of one new token over the paged cache against 64-bit attention: head layouts,
page sizes, both cache types, lengths from one token across page and tile boundaries,
windows, padding rows and empty sequences, pages full of NaN outside the sequences, and
what a bad slot, length or page index does."""
import numpy as np
import pytest
import torch

from tests import kv_reference as R

pytestmark = pytest.mark.gpu
D = 128


def _W():
    from paper_2608_30877_gb300 import w4a16 as W
    return W


def _values(cache, layer, slot_pages, n, T):
    """Keys and values of a sequence's first n tokens as float64 [2, n, Hkv, D]."""
    pos = torch.arange(n, device="cuda")
    page, at = slot_pages[pos // T], pos % T
    pool = cache.pages[layer]
    if cache.exponents is None:
        return torch.stack([pool[w][page, :, at] for w in (0, 1)]).double().cpu().numpy()
    codes = [pool.view(torch.uint8)[w][page, :, at].view(torch.float8_e4m3fn).double() for w in (0, 1)]
    e = cache.exponents[layer][page, :, at].int().cpu().numpy() - 127
    return np.stack([np.ldexp(codes[w].cpu().numpy(), e[..., w, None]) for w in (0, 1)])


class Case:
    """A cache of sequences with random contents, everything else in it NaN, and one row of
    the projection for each."""

    def __init__(self, bits, H, Hkv, T, lengths, seed, layers=2, layer=1, q_scale=2.0):
        W = _W()
        self.bits, self.H, self.Hkv, self.T, self.lengths, self.layer = bits, H, Hkv, T, lengths, layer
        g = torch.Generator(device="cuda").manual_seed(seed)
        n = len(lengths)
        counts = [-(-x // T) for x in lengths]
        slots = torch.randperm(n + 2, generator=g, device="cuda")[:n]
        P = sum(counts) + 3
        dtype = torch.bfloat16 if bits == 16 else torch.float8_e4m3fn
        self.cache = c = W.KVCache(layers, P, Hkv, n + 2, max(counts + [1]) + 1, T, dtype)
        order = torch.randperm(P, generator=g, device="cuda").to(torch.int32)
        c.page_table.fill_(-5)  # entries past a sequence's pages mean nothing
        c.pages.view(torch.uint8).fill_(0xFF)
        if c.exponents is not None:
            c.exponents.fill_(0xFF)
        a = 0
        self.slot_pages = []
        for s, x, k in zip(slots.tolist(), lengths, counts):
            pages = order[a:a + k]
            a += k
            c.page_table[s, :k] = pages
            c.seq_len[s] = x
            c.page_refs[pages.long()] = 1
            self.slot_pages.append(pages.long())
            pos = torch.arange(max(0, x - 1), device="cuda")  # (the last token is the new one)
            if x > 1:
                kv = torch.randn((2, x - 1, Hkv, D), generator=g, device="cuda")
                if bits == 16:
                    for w in (0, 1):
                        c.pages[layer, w][pages.long()[pos // T], :, pos % T] = kv[w].bfloat16()
                else:
                    for w in (0, 1):
                        codes = (kv[w] * 112).clamp(-448, 448).to(torch.float8_e4m3fn)
                        c.pages.view(torch.uint8)[layer, w][pages.long()[pos // T], :, pos % T] = \
                            codes.view(torch.uint8)
                    e = torch.randint(115, 125, (x - 1, Hkv, 2), generator=g, device="cuda", dtype=torch.uint8)
                    c.exponents[layer][pages.long()[pos // T], :, pos % T] = e
        self.slots = slots.to(torch.int32)
        self.qkv = torch.randn((n, (H + 2 * Hkv) * D), generator=g, device="cuda").bfloat16()
        self.qkv[:, :H * D] *= q_scale

    def before(self):
        c = self.cache
        return c.pages.view(torch.uint8).clone(), None if c.exponents is None else c.exponents.clone()

    def check_row(self, out, i, window, what=""):
        """Row i against 64-bit attention over the cache's contents.  Rounding the weights to
        bf16 (2^-9 each, and their sum likewise) moves an output by at most 2^-8 of the weighted
        mean of |v|; fp32 scores of |s| up to ~2^6 are good to 2^-10 of the weights; the store
        rounds by 2^-9 of the value."""
        n, H, Hkv = self.lengths[i], self.H, self.Hkv
        if n == 0:
            assert (out[i] == 0).all(), what
            return
        row = self.qkv[i].double().cpu().numpy()
        kv = _values(self.cache, self.layer, self.slot_pages[i], n, self.T)
        new = R.held(row[H * D:].reshape(2, Hkv, D), self.bits)
        assert np.array_equal(kv[:, n - 1], new), f"{what}: the new token's key or value in the cache"
        low = max(0, n - window)
        ref, size = R.attention(row[:H * D].reshape(H, D), kv[0, low:], kv[1, low:])
        got = out[i].double().cpu().numpy().reshape(H, D)
        bound = 1.01 * 2.0 ** -9 * np.abs(ref) + (2.0 ** -8 + 2.0 ** -10) * size + 1e-30
        err = np.abs(got - ref)
        assert np.isfinite(got).all(), what
        assert (err <= bound).all(), f"{what} row {i} length {n}: worst {np.max(err / bound):.3f} of the bound"
        assert np.linalg.norm(err) <= 2.0 ** -9 * (np.linalg.norm(ref) + np.linalg.norm(size)), what

    def check_rest(self, before, rows=None):
        """Nothing but the new tokens' rows has changed in the pool."""
        c, (pages, exponents) = self.cache, before
        for i, n in enumerate(self.lengths):
            if n == 0 or (rows is not None and i not in rows):
                continue
            page, at = int(self.slot_pages[i][(n - 1) // self.T]), (n - 1) % self.T
            now = c.pages.view(torch.uint8)
            pages[self.layer, :, page, :, at] = now[self.layer, :, page, :, at]
            if exponents is not None:
                exponents[self.layer, page, :, at] = c.exponents[self.layer, page, :, at]
        assert torch.equal(pages, c.pages.view(torch.uint8))
        assert exponents is None or torch.equal(exponents, c.exponents)


def _run(case, window=32768):
    W = _W()
    before = case.before()
    out = W.attention_decode(case.cache, case.layer, case.qkv, case.slots, case.H, window=window)
    assert W.get_device_error() == W.OK
    for i in range(len(case.lengths)):
        case.check_row(out, i, window, f"bits {case.bits} H {case.H}/{case.Hkv} T {case.T} window {window}")
    case.check_rest(before)
    return out


EDGES = [1, 2, 15, 16, 17, 0, 31, 63, 64, 65, 127, 128, 129, 200, 333]


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("T", [16, 32, 64, 128])
def test_lengths_across_pages_and_tiles(bits, T):
    _run(Case(bits, 4, 4, T, EDGES, 100 + T + bits))


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("H,Hkv", [(1, 1), (3, 3), (8, 4), (6, 2), (7, 1), (8, 1), (9, 1), (16, 1),
                                   (24, 2), (17, 1), (33, 1), (64, 1), (65, 1), (96, 1), (130, 1), (96, 8)])
def test_head_layouts(bits, H, Hkv):
    _run(Case(bits, H, Hkv, 32, [1, 40, 129, 300], 7 * H + Hkv + bits))


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("window", [1, 2, 16, 63, 64, 65, 100, 128])
def test_windows(bits, window):
    _run(Case(bits, 6, 3, 16, [1, 2, 64, 65, 100, 101, 127, 128, 129, 190, 300], window + bits), window)


@pytest.mark.parametrize("bits,H,Hkv,T,lengths", [
    (16, 8, 1, 64, [20000]), (16, 2, 2, 16, [5000, 1, 7000]), (8, 16, 1, 32, [30011]),
    (8, 12, 4, 128, [9000, 0, 3, 4097]), (16, 96, 1, 64, [6001, 2]), (16, 4, 4, 16, [70000, 70000]),
])
def test_long_sequences(bits, H, Hkv, T, lengths):
    _run(Case(bits, H, Hkv, T, lengths, sum(lengths), layers=1, layer=0))


@pytest.mark.parametrize("bits", [16, 8])
def test_long_window(bits):
    _run(Case(bits, 4, 2, 64, [10007, 4096, 4097, 100], 5, layers=1, layer=0), 4096)


def test_many_rows():
    rng = np.random.default_rng(1)
    _run(Case(16, 4, 2, 16, rng.integers(0, 200, 700).tolist(), 6, layers=1, layer=0))
    _run(Case(8, 3, 3, 64, rng.integers(0, 300, 300).tolist(), 7, layers=1, layer=0))


@pytest.mark.parametrize("bits", [16, 8])
def test_peaked_and_equal_scores(bits):
    """Queries so large that one key has all the weight, and zero queries (every key alike)."""
    for scale in (100.0, 0.0):
        case = Case(bits, 4, 2, 16, [1, 50, 500], 8, q_scale=scale)
        # fp32 scores of size s are good to 2^-24 * 128 s: past the bound's 2^-10 at s ~ 2^7,
        # so the keys are taken from a few that are far apart
        if scale == 100.0:
            case.qkv[:, :4 * D] = 0
            case.qkv[:, 0:4 * D:D] = 64.0
        _run(case)


@pytest.mark.parametrize("bits", [16, 8])
def test_extreme_scales(bits):
    """Values near the ends of bf16's range in the new token, small ones in the rest."""
    for factor in (2.0 ** 60, 2.0 ** -60, 2.0 ** -118):
        case = Case(bits, 4, 2, 32, [1, 33, 100], 9)
        case.qkv[:, 6 * D:] *= factor  # the values of the new token
        _run(case)


@pytest.mark.parametrize("bits", [16, 8])
def test_padding_rows_and_bad_slots(bits):
    """Rows of slot -1 give zeros; a slot out of range, a length that does not fit and a page
    index out of range give a zero row and an error, and leave the others alone."""
    W = _W()
    good = Case(bits, 4, 2, 16, [40, 100, 17, 64, 200, 5], 10)
    want = W.attention_decode(good.cache, 1, good.qkv, good.slots, 4)
    for what in ("padding", "slot high", "slot low", "length", "page", "page low"):
        case = Case(bits, 4, 2, 16, [40, 100, 17, 64, 200, 5], 10)
        c, slots = case.cache, case.slots.clone()
        s = int(slots[1])
        if what == "padding":
            slots[1] = -1
        elif what == "slot high":
            slots[1] = c.num_slots
        elif what == "slot low":
            slots[1] = -2
        elif what == "length":
            c.seq_len[s] = c.max_pages * 16 + 1
        elif what == "page":
            c.page_table[s, 2] = c.num_pages
        else:
            c.page_table[s, 6] = -1
        before = case.before()
        out = W.attention_decode(c, 1, case.qkv, slots, 4)
        assert W.get_device_error() == (W.OK if what == "padding" else W.ERR_INVALID_ARG), what
        assert (out[1] == 0).all(), what
        others = [0, 2, 3, 4, 5]
        assert torch.equal(out[others], want[others]), what
        # (a bad page index may show after the row's own token was stored)
        case.check_rest(before, rows=others + ([1] if what == "page" else []))


def test_unused_memory_of_any_kind_is_not_seen():
    """The bits of the result do not depend on what lies past a sequence's end or before its
    window: NaN, infinities, zeros."""
    W = _W()
    for bits in (16, 8):
        outs = []
        for fill in (0xFF, 0x7F, 0x00):
            case = Case(bits, 6, 2, 64, [1, 70, 100, 300], 11)
            c = case.cache
            used = torch.zeros((c.num_pages, case.T), dtype=torch.bool, device="cuda")
            for pages, n in zip(case.slot_pages, case.lengths):
                pos = torch.arange(max(0, n - 65), n, device="cuda")
                used[pages[pos // case.T], pos % case.T] = True
            c.pages.view(torch.uint8).masked_fill_(~used[None, None, :, None, :, None], fill)
            if bits == 8:
                c.exponents.masked_fill_(~used[None, :, None, :, None], fill)
            outs.append(W.attention_decode(c, 1, case.qkv, case.slots, 6, window=65))
        assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


def test_infinities_and_nan_within_the_sequence_are_felt():
    W = _W()
    case = Case(16, 2, 2, 16, [50, 50, 50], 12)
    c = case.cache
    c.pages[1, 1, case.slot_pages[0][1], 0, 3] = float("inf")    # a value of head 0
    c.pages[1, 0, case.slot_pages[1][1], 1, 3, 5] = float("nan")  # a key of head 1
    out = W.attention_decode(c, 1, case.qkv, case.slots, 2).float()
    assert torch.isposinf(out[0, :D]).all() and torch.isfinite(out[0, D:]).all()
    assert torch.isfinite(out[1, :D]).all() and torch.isnan(out[1, D:]).all()
    case.check_row(out, 2, 32768)


@pytest.mark.parametrize("bits,H,Hkv,lengths", [(16, 8, 2, [5000, 3, 700]), (8, 4, 4, [3000, 2999])])
def test_same_bits_every_time_and_on_another_stream(bits, H, Hkv, lengths):
    W = _W()
    case = Case(bits, H, Hkv, 64, lengths, 13)
    first = W.attention_decode(case.cache, 1, case.qkv, case.slots, H)
    for _ in range(20):
        assert torch.equal(W.attention_decode(case.cache, 1, case.qkv, case.slots, H), first)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    ws = case.cache.new_workspace(H, side)
    out = W.attention_decode(case.cache, 1, case.qkv, case.slots, H, workspace=ws, stream=side)
    side.synchronize()
    assert torch.equal(out, first)
    out2 = torch.full_like(out, 7.0)
    W.attention_decode(case.cache, 1, case.qkv, case.slots, H, out=out2)
    assert torch.equal(out2, first)


def test_rows_do_not_depend_on_the_batch():
    """A sequence alone and in a batch: the split of its length differs, so the bits may, but
    both are within the bound; row order changes nothing but the order."""
    W = _W()
    case = Case(16, 8, 2, 32, [777, 1500, 64, 1], 14)
    out = W.attention_decode(case.cache, 1, case.qkv, case.slots, 8)
    perm = torch.tensor([2, 0, 3, 1], device="cuda")
    out2 = W.attention_decode(case.cache, 1, case.qkv[perm].contiguous(), case.slots[perm].contiguous(), 8)
    for i in range(4):
        case.check_row(out, i, 32768)
    back = torch.empty_like(out2)
    back[perm] = out2
    for i in range(4):
        case.check_row(back, i, 32768)


def test_captured_steps():
    """Growth and attention of a step captured in one graph, replayed token after token."""
    W = _W()
    H = Hkv = 4
    n, steps = 3, 40
    g = torch.Generator(device="cuda").manual_seed(3)
    rows = torch.randn((steps, n, 3 * H * D), generator=g, device="cuda").bfloat16()
    results = []
    for captured in (False, True):
        c = W.KVCache(1, 16, Hkv, n, 4, 16)
        slots, one = R.i32([2, 0, 1]), R.i32([1, 1, 1])
        qkv, out = torch.empty_like(rows[0]), torch.empty((n, H * D), dtype=torch.bfloat16, device="cuda")
        ws = c.new_workspace(H)

        def step():
            W.kv_extend(c, slots, one)
            W.attention_decode(c, 0, qkv, slots, H, out=out, workspace=ws)

        if captured:
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                step()
        outs = []
        for t in range(steps):
            qkv.copy_(rows[t])
            graph.replay() if captured else step()
            outs.append(out.clone())
        assert W.get_device_error() == W.OK
        assert c.seq_len.tolist() == [steps] * n
        results.append(torch.stack(outs))
    assert torch.equal(results[0], results[1])
