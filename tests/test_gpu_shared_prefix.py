"""Attention over forks: sequences of several parents that share whole pages and copied part-full
ones, each against 64-bit attention over the tokens that it was given."""
import numpy as np
import pytest
import torch

from tests import kv_reference as R

pytestmark = pytest.mark.gpu
D = 128


def _W():
    from paper_2608_30877_gb300 import w4a16 as W
    return W


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("H,Hkv,T,window", [(4, 4, 16, 32768), (6, 2, 64, 32768), (12, 1, 32, 70), (4, 2, 128, 150)])
def test_forks_of_several_parents(bits, H, Hkv, T, window):
    """Parents of 133, 64 and 37 tokens, three forks each with 0 to 60 tokens of their own, and forks of
    forks; then two steps of everything together.  The parents' pages stay as they were."""
    W = _W()
    layers, layer = 2, 1
    prefixes, tails = [133, 64, 37], [0, 1, 60]
    kids = [(p, t) for p in range(3) for t in tails]
    n = len(prefixes) + len(kids)
    grandkids = {n: 3 + 2, n + 1: 3 + 8}  # (of the forks with 60 tokens of the first and the last parent)
    slots = n + len(grandkids)
    c = W.KVCache(layers, 200, Hkv, slots, 20, T, torch.bfloat16 if bits == 16 else torch.float8_e4m3fn)
    c.pages.view(torch.uint8).fill_(0xFF)
    if bits == 8:
        c.exponents.fill_(0xFF)
    g = torch.Generator(device="cuda").manual_seed(bits + T)
    tokens = {s: [] for s in range(slots)}  # [2, Hkv, D] each, as the cache holds them

    def rows(count):
        x = torch.randn((count, (H + 2 * Hkv) * D), generator=g, device="cuda")
        x[:, :H * D] *= 2
        return x.bfloat16()

    def held(x):
        return list(R.held(x[:, H * D:].double().cpu().numpy().reshape(-1, 2, Hkv, D), bits))

    def write(which, counts):
        W.kv_extend(c, R.i32(which), R.i32(counts))
        x = rows(sum(counts))
        W.kv_write(c, layer, x, R.i32(np.concatenate([[0], np.cumsum(counts)])), R.i32(which), H)
        new = held(x)
        for s, a, b in zip(which, np.cumsum([0, *counts]), np.cumsum(counts)):
            tokens[s] += new[a:b]

    def fork(pairs):
        W.kv_fork(c, R.i32([p for p, _ in pairs]), R.i32([s for _, s in pairs]))
        for p, s in pairs:
            tokens[s] = list(tokens[p])

    write([0, 1, 2], prefixes)
    fork([(p, 3 + i) for i, (p, _) in enumerate(kids)])
    with_tail = [(3 + i, t) for i, (_, t) in enumerate(kids) if t > 0]
    write([s for s, _ in with_tail], [t for _, t in with_tail])
    fork([(p, s) for s, p in grandkids.items()])
    assert W.get_device_error() == W.OK
    parents = [(c.page_table[s, :x // T].long().clone(), x) for s, x in enumerate(prefixes)]
    whole = [(pages, c.pages.view(torch.uint8)[:, :, pages].clone()) for pages, _ in parents]
    assert int(c.page_refs.max()) >= 5 or T == 128
    order = list(np.random.default_rng(1).permutation(slots))
    for _ in range(2):
        W.kv_extend(c, R.i32(order), R.i32([1] * slots))
        x = rows(slots)
        out = W.attention_decode(c, layer, x, R.i32(order), H, window=window)
        assert W.get_device_error() == W.OK
        new, q = held(x), x[:, :H * D].double().cpu().numpy().reshape(-1, H, D)
        for i, s in enumerate(order):
            tokens[s].append(new[i])
            kv = np.stack(tokens[s][-window:], 1)  # [2, n, Hkv, D]
            assert len(tokens[s]) == int(c.seq_len[s])
            ref, size = R.attention(q[i], kv[0], kv[1])
            err = np.abs(out[i].double().cpu().numpy().reshape(H, D) - ref)
            # (the bound of the tests of single sequences)
            assert (err <= 1.01 * 2.0 ** -9 * np.abs(ref) + (2.0 ** -8 + 2.0 ** -10) * size).all(), s
    for pages, was in whole:
        assert torch.equal(c.pages.view(torch.uint8)[:, :, pages], was)
