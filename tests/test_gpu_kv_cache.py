"""Pages of the key-value cache against a model in plain Python: growth, sharing with copy
on write, release, roll-back and compaction, in random sequences; what errors leave
unchanged; prompt writes in both forms against the format's definition."""
import numpy as np
import pytest
import torch

from tests import kv_reference as R

pytestmark = pytest.mark.gpu
D = 128


def _W():
    from paper_2608_30877_gb300 import w4a16 as W
    return W


def _cache(bits, layers, P, Hkv, slots, W_pages, T):
    W = _W()
    c = W.KVCache(layers, P, Hkv, slots, W_pages, T, torch.bfloat16 if bits == 16 else torch.float8_e4m3fn)
    c.pages.view(torch.uint8).fill_(0xFF)
    if c.exponents is not None:
        c.exponents.fill_(0xFF)
    return c


class Mirror:
    """A cache on the device and the model side by side.  A token's content is one number,
    written into every layer and head (as bf16 or as a code and an exponent) from the host, so
    that page operations alone move it on the device."""

    def __init__(self, bits, layers, P, Hkv, slots, W_pages, T):
        self.c, self.ref = _cache(bits, layers, P, Hkv, slots, W_pages, T), R.Pages(P, slots, W_pages, T)
        self.count = 0

    def fill(self, slot, start, stop):
        for pos in range(start, stop):
            self.count = self.count % 60000 + 1
            page = self.ref.table[slot][pos // self.ref.T]
            self.ref.set_token(slot, pos, self.count)
            raw = self.c.pages.view(torch.uint8)[:, :, page, :, pos % self.ref.T]
            raw[..., 0], raw[..., 1:] = self.count & 0xFF, self.count >> 8
            if self.c.exponents is not None:
                self.c.exponents[:, page, :, pos % self.ref.T, 0] = self.count & 0xFF
                self.c.exponents[:, page, :, pos % self.ref.T, 1] = self.count >> 8

    def check(self):
        W = _W()
        assert W.get_device_error() == W.OK
        R.same_tables(self.c, self.ref)
        raw = self.c.pages.view(torch.uint8).cpu().numpy()
        exps = None if self.c.exponents is None else self.c.exponents.cpu().numpy()
        for s, n in enumerate(self.ref.length):
            for pos in range(n):
                want = self.ref.token(s, pos)
                page, at = self.ref.table[s][pos // self.ref.T], pos % self.ref.T
                got = raw[:, :, page, :, at]
                assert (got[..., 0] == (want & 0xFF)).all() and (got[..., 1:] == want >> 8).all(), (s, pos)
                if exps is not None:
                    e = exps[:, page, :, at]
                    assert (e[..., 0] == (want & 0xFF)).all() and (e[..., 1] == want >> 8).all(), (s, pos)

    def extend(self, slots, add):
        W = _W()
        was = list(self.ref.length)
        ok = self.ref.extend(slots, add)
        W.kv_extend(self.c, R.i32(slots), R.i32(add))
        if not ok:
            assert W.get_device_error() == W.ERR_CAPACITY
            return False
        for s in slots:
            if s != -1:
                self.fill(s, was[s], self.ref.length[s])
        return True


@pytest.mark.parametrize("bits,layers,Hkv,T,P", [(16, 2, 3, 16, 40), (8, 3, 2, 16, 25), (16, 1, 1, 64, 30),
                                                 (8, 1, 5, 32, 12), (8, 2, 1, 128, 14)])
def test_random_operations_against_the_model(bits, layers, Hkv, T, P):
    W = _W()
    rng = np.random.default_rng(bits + T)
    slots, W_pages = 9, 6
    m = Mirror(bits, layers, P, Hkv, slots, W_pages, T)
    for step in range(60):
        live = [s for s in range(slots) if m.ref.length[s] > 0]
        empty = [s for s in range(slots) if m.ref.length[s] == 0]
        op = rng.choice(["extend", "extend", "fork", "trim", "free", "compact"])
        if op == "extend":
            k = int(rng.integers(1, slots + 1))
            which = rng.permutation(slots)[:k].tolist()
            if rng.random() < 0.3:
                which[0] = -1
            m.extend(which, rng.integers(0, 2 * T, k).tolist())
        elif op == "fork" and live and empty:
            kids = rng.permutation(empty)[:int(rng.integers(1, len(empty) + 1))].tolist()
            parents = rng.choice(live, len(kids)).tolist()
            m.ref.fork(parents, kids)
            W.kv_fork(m.c, R.i32(parents), R.i32(kids))
        elif op == "trim" and live:
            which = rng.permutation(live)[:int(rng.integers(1, len(live) + 1))].tolist()
            keep = [int(rng.integers(0, m.ref.length[s] + 1)) for s in which]
            m.ref.trim(which, keep)
            W.kv_trim(m.c, R.i32(which), R.i32(keep))
        elif op == "free" and live:
            which = [int(rng.choice(live)), -1]
            m.ref.trim(which)
            W.kv_trim(m.c, R.i32(which))
        elif op == "compact":
            m.ref.compact()
            W.kv_compact(m.c)
        m.check()


def test_every_sharer_grows_in_one_call():
    """A part-full page of five sequences, all of which go on: each gets its own copy, and the
    page that they left is free again."""
    W = _W()
    m = Mirror(16, 2, 20, 2, 5, 4, 16)
    m.extend([0], [21])
    m.ref.fork([0] * 4, [1, 2, 3, 4])
    W.kv_fork(m.c, R.i32([0] * 4), R.i32([1, 2, 3, 4]))
    m.check()
    assert m.extend([4, 1, 0, 2, 3], [1, 20, 1, 0, 5])
    m.check()
    assert m.extend([2, 0], [1, 1])
    m.check()


def test_large_growth_and_many_slots():
    """More slots than a CTA has threads, and sequences that take thousands of pages at once."""
    W = _W()
    n = 2500
    c, ref = _cache(16, 1, 12000, 1, n, 5000, 16), R.Pages(12000, n, 5000, 16)
    rng = np.random.default_rng(5)
    for _ in range(3):
        which = rng.permutation(n).tolist()
        add = rng.integers(0, 40, n).tolist()
        add[7] = 16 * 300
        assert ref.extend(which, add)
        W.kv_extend(c, R.i32(which), R.i32(add))
        R.same_tables(c, ref)
        some = which[:1200]
        ref.trim(some)
        W.kv_trim(c, R.i32(some))
        R.same_tables(c, ref)
        ref.compact()
        W.kv_compact(c)
        R.same_tables(c, ref)
    assert W.get_device_error() == W.OK
    parents, kids = [], []
    empty = [s for s in range(n) if ref.length[s] == 0]
    full = [s for s in range(n) if ref.length[s] > 0]
    for i, s in enumerate(empty):
        kids.append(s)
        parents.append(full[i % len(full)])
    ref.fork(parents, kids)
    W.kv_fork(c, R.i32(parents), R.i32(kids))
    assert W.get_device_error() == W.OK
    R.same_tables(c, ref)


def test_errors_change_nothing():
    W = _W()
    m = Mirror(8, 1, 8, 1, 5, 3, 16)
    m.extend([0, 1], [40, 10])
    m.ref.fork([0], [2])
    W.kv_fork(m.c, R.i32([0]), R.i32([2]))
    m.check()

    def refused(code, f, *lists):
        state = [t.clone() for t in (m.c.pages.view(torch.uint8), m.c.exponents, m.c.page_table,
                                     m.c.seq_len, m.c.page_refs)]
        f(m.c, *(None if x is None else R.i32(x) for x in lists))
        assert W.get_device_error() == code
        now = (m.c.pages.view(torch.uint8), m.c.exponents, m.c.page_table, m.c.seq_len, m.c.page_refs)
        assert all(torch.equal(a, b) for a, b in zip(state, now))

    refused(W.ERR_CAPACITY, W.kv_extend, [3, 4], [48, 48])   # six pages, four free
    refused(W.ERR_CAPACITY, W.kv_extend, [1], [39])          # past max_pages
    refused(W.ERR_CAPACITY, W.kv_extend, [1], [2**31 - 1])
    refused(W.ERR_CAPACITY, W.kv_extend, [0, 1, 2, 3, 4], [2**31 - 1] * 5)
    refused(W.ERR_INVALID_ARG, W.kv_extend, [1, 1], [1, 1])
    refused(W.ERR_INVALID_ARG, W.kv_extend, [1, 3], [1, -1])
    refused(W.ERR_INVALID_ARG, W.kv_extend, [5], [1])
    refused(W.ERR_INVALID_ARG, W.kv_extend, [-2], [1])
    refused(W.ERR_INVALID_ARG, W.kv_fork, [0], [1])          # not empty
    refused(W.ERR_INVALID_ARG, W.kv_fork, [0, 0], [3, 3])
    refused(W.ERR_INVALID_ARG, W.kv_fork, [0, 3], [3, 4])    # a child as a parent
    refused(W.ERR_INVALID_ARG, W.kv_fork, [5], [3])
    refused(W.ERR_INVALID_ARG, W.kv_fork, [-1], [3])
    refused(W.ERR_INVALID_ARG, W.kv_trim, [0, 0], [1, 1])
    refused(W.ERR_INVALID_ARG, W.kv_trim, [0], [41])
    refused(W.ERR_INVALID_ARG, W.kv_trim, [0], [-1])
    refused(W.ERR_INVALID_ARG, W.kv_trim, [9], None)
    good = int(m.c.page_table[0, 1])
    for bad in (-1, 8, 1 << 30):
        m.c.page_table[0, 1] = bad
        refused(W.ERR_INVALID_ARG, W.kv_trim, [0], None)
        refused(W.ERR_INVALID_ARG, W.kv_fork, [0], [3])
        refused(W.ERR_INVALID_ARG, W.kv_compact)
    m.c.page_table[0, 1] = good
    good = int(m.c.page_table[0, 2])
    m.c.page_table[0, 2] = 8  # the part-full page that growth looks at
    refused(W.ERR_INVALID_ARG, W.kv_extend, [0], [1])
    m.c.page_table[0, 2] = good
    m.c.seq_len[1] = 49
    refused(W.ERR_INVALID_ARG, W.kv_compact)
    refused(W.ERR_INVALID_ARG, W.kv_trim, [1], [1])
    m.c.seq_len[1] = 10
    m.extend([1, 2], [5, 1])  # and after all that the cache works
    m.check()


def test_a_full_pool_to_the_last_page():
    m = Mirror(16, 1, 7, 1, 3, 7, 16)
    assert m.extend([0, 1, 2], [33, 32, 17])  # 3 + 2 + 2 pages
    m.check()
    assert m.extend([0, 1], [15, 0])
    assert not m.extend([1], [1])
    m.check()


# ---------------------------------------------------------------- prompt writes

@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("H,Hkv,T,lengths,before", [
    (4, 4, 16, [1, 16, 17, 40, 0, 5], [0, 0, 3, 15, 4, 100]), (0, 1, 64, [100, 1], [0, 63]),
    (6, 2, 128, [129, 128, 3], [0, 1, 127]), (12, 3, 32, [300], [0]),
])
def test_prompt_writes(bits, H, Hkv, T, lengths, before):
    """Every written row is the format's rounding of the projection's, every other byte as it
    was; sequences longer than their rows are written at their end."""
    W = _W()
    layers, layer = 2, 1
    n = len(lengths)
    totals = [a + b for a, b in zip(lengths, before)]
    counts = [-(-t // T) for t in totals]
    c = _cache(bits, layers, sum(counts) + 2, Hkv, n + 1, max(counts) + 1, T)
    slots = torch.randperm(n + 1, device="cuda")[:n].to(torch.int32)
    W.kv_extend(c, slots, R.i32(totals))
    assert W.get_device_error() == W.OK
    gap = 3  # rows of the batch before the first sequence
    start = np.concatenate([[0], np.cumsum(lengths)]) + gap
    M = int(start[-1]) + 2
    g = torch.Generator(device="cuda").manual_seed(M)
    qkv = torch.randn((M, (H + 2 * Hkv) * D), generator=g, device="cuda")
    qkv *= torch.exp2(torch.randint(-20, 20, (M, 1), generator=g, device="cuda").float())
    qkv = qkv.bfloat16()
    special = torch.tensor([0.0, float("inf"), -float("inf"), 448.0, 3.0e38, 1e-40, -0.0, 2.0 ** -130])
    qkv[gap, H * D:H * D + 8] = special.cuda()
    if lengths[0] > 1:
        qkv[gap + 1, H * D:] = 0
    want = c.pages.view(torch.uint8).clone()
    want_e = None if c.exponents is None else c.exponents.clone()
    W.kv_write(c, layer, qkv, R.i32(start.tolist()), slots, H)
    assert W.get_device_error() == W.OK
    rows = qkv[:, H * D:].float().cpu().numpy().astype(np.float64).reshape(M, 2, Hkv, D)
    table = c.page_table.cpu().numpy()
    for i in range(n):
        for t in range(lengths[i]):
            pos, m = before[i] + t, start[i] + t
            page, at = int(table[int(slots[i]), pos // T]), pos % T
            for w in (0, 1):
                if bits == 16:
                    want.view(torch.bfloat16)[layer, w, page, :, at] = \
                        qkv[m, (H + w * Hkv) * D:(H + (w + 1) * Hkv) * D].view(Hkv, D)
                else:
                    for h in range(Hkv):
                        codes, e = R.e4m3_row(rows[m, w, h])
                        want[layer, w, page, h, at] = torch.from_numpy(codes).to(torch.float8_e4m3fn) \
                            .view(torch.uint8).cuda()
                        want_e[layer, page, h, at, w] = e + 127
    assert torch.equal(c.pages.view(torch.uint8), want)
    assert want_e is None or torch.equal(c.exponents, want_e)


def test_prompt_write_leaves_out_what_is_wrong():
    W = _W()
    c = _cache(16, 1, 10, 1, 4, 3, 16)
    W.kv_extend(c, R.i32([0, 1, 2]), R.i32([10, 20, 5]))
    qkv = torch.randn((30, 3 * D), device="cuda").bfloat16()

    def refused(start, slots):
        c.pages.view(torch.uint8).fill_(0xFF)
        W.kv_write(c, 0, qkv, R.i32(start), R.i32(slots), 1)
        assert W.get_device_error() == W.ERR_INVALID_ARG
        return c.pages[0, 0, :, 0, :, 0]

    ok = ~torch.isnan(refused([0, 10, 20], [0, 4]))       # slot out of range
    assert int(ok.sum()) == 10
    ok = ~torch.isnan(refused([0, 11, 20], [0, 1]))       # more rows than tokens
    assert int(ok.sum()) == 9
    assert int((~torch.isnan(refused([0, 10, 31], [0, 1]))).sum()) == 10  # past the batch
    refused([0, 10, 5], [0, 1])                            # decreasing
    c.page_table[1, 1] = 99
    assert int((~torch.isnan(refused([0, 20], [1]))).sum()) == 16
    c.pages.view(torch.uint8).fill_(0xFF)
    W.kv_write(c, 0, qkv, R.i32([0, 10, 15]), R.i32([-1, 2]), 1)  # a padding entry
    assert W.get_device_error() == W.OK
    assert int((~torch.isnan(c.pages[0, 0, :, 0, :, 0])).sum()) == 5


def test_offsets_past_32_bits():
    """A pool of more than 2^32 bytes a layer and 2^33 in all: the last page of the last layer
    is written, copied, read and moved."""
    W = _W()
    Hkv, T, P = 32, 128, 2100  # 2.2 GB of keys a layer
    c = W.KVCache(2, P, Hkv, 3, 2, T)
    last = P - 1
    c.page_table[0, 0] = last
    c.seq_len[0] = 100
    c.page_refs[last] = 1
    g = torch.Generator(device="cuda").manual_seed(2)
    qkv = torch.randn((100, 3 * Hkv * D), generator=g, device="cuda").bfloat16()
    W.kv_write(c, 1, qkv, R.i32([0, 100]), R.i32([0]), Hkv)
    want = qkv[:, Hkv * D:].view(100, 2, Hkv, D)
    for w in (0, 1):
        assert torch.equal(c.pages[1, w, last, :, :100].transpose(0, 1), want[:, w])
    W.kv_fork(c, R.i32([0]), R.i32([1]))
    W.kv_extend(c, R.i32([1]), R.i32([1]))
    assert c.page_table[1, 0] == 0
    row = torch.randn((1, 3 * Hkv * D), generator=g, device="cuda").bfloat16()
    W.kv_extend(c, R.i32([0]), R.i32([1]))
    a = W.attention_decode(c, 1, row, R.i32([0]), Hkv)
    b = W.attention_decode(c, 1, row, R.i32([1]), Hkv)
    assert torch.equal(a, b)
    q, k, v = (row.view(3, Hkv, D)[i].double().cpu().numpy() for i in range(3))
    ref, size = R.attention(q, np.concatenate([want[:, 0].double().cpu().numpy(), k[None]]),
                            np.concatenate([want[:, 1].double().cpu().numpy(), v[None]]))
    err = np.abs(a[0].double().cpu().numpy().reshape(Hkv, D) - ref)
    assert (err <= 1.01 * 2.0 ** -9 * np.abs(ref) + (2.0 ** -8 + 2.0 ** -10) * size).all()
    W.kv_compact(c)
    assert c.page_table[0, 0] == 1 and c.page_refs[:3].tolist() == [1, 1, 0]
    assert torch.equal(W.attention_decode(c, 1, row, R.i32([0]), Hkv), a)
    assert W.get_device_error() == W.OK
