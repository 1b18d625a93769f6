"""Cache writes and decode attention where the work is cut differently: tokens of a CTA by
heads and batch, boxes of whole pages and of single groups of tokens, queries of a key head
over one, two and four warps."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from tests import kv_reference as R
from tests.test_gpu_attention_decode import Case, _run

pytestmark = pytest.mark.gpu
D = 128


def _W():
    from paper_2608_30877_gb300 import w4a16 as W
    return W


# (heads 1 and 2 with many tokens: 32 tokens to a CTA; 4: 16; 8 and 5: 8; 12: 4; 96: 1; few
# tokens: 1 whatever the heads)
@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("Hkv,lengths", [(1, [4000, 1, 1900, 0, 77]), (2, [5001, 33]), (4, [2500, 31]), (8, [1301, 5]),
                                         (5, [1300, 9]), (12, [700, 3]), (96, [30, 9]), (3, [1]), (1, [2, 1])])
def test_writes_by_heads_and_tokens(bits, Hkv, lengths):
    """Every stored row is the format's rounding of the projection's; the rest of the pool and
    rows outside every sequence stay."""
    W = _W()
    T, H, gap = 32, 2, 5
    n = len(lengths)
    counts = [-(-x // T) for x in lengths]
    c = W.KVCache(1, sum(counts) + 1, Hkv, n, max(counts), page_tokens=T,
                  dtype=torch.float8_e4m3fn if bits == 8 else torch.bfloat16)
    c.pages.view(torch.uint8).fill_(0x5A)
    if bits == 8:
        c.exponents.fill_(0x5A)
    slots = R.i32(range(n))
    W.kv_extend(c, slots, R.i32(lengths))
    start = np.concatenate([[0], np.cumsum(lengths)]) + gap
    M = int(start[-1]) + 3
    g = torch.Generator(device="cuda").manual_seed(Hkv + bits)
    qkv = torch.randn((M, (H + 2 * Hkv) * D), generator=g, device="cuda")
    qkv *= torch.exp2(torch.randint(-30, 30, (M, 1), generator=g, device="cuda").float())
    qkv = qkv.bfloat16()
    # a row with what is not finite, one with nothing else, zeros
    qkv[gap, H * D:H * D + 3] = torch.tensor([float("nan"), float("inf"), -float("inf")]).cuda()
    if lengths[0] > 2:
        qkv[gap + 1, H * D:(H + 1) * D] = float("nan")
        qkv[gap + 2, H * D:] = -0.0
    W.kv_write(c, 0, qkv, R.i32(start.tolist()), slots, H)
    assert W.get_device_error() == W.OK
    table = c.page_table.cpu().long()
    seq = np.repeat(np.arange(n), lengths)
    pos = np.concatenate([np.arange(x) for x in lengths])
    page = table[torch.from_numpy(seq), torch.from_numpy(pos // T)]
    at = torch.from_numpy(pos % T)
    # [tokens, 2, heads, bytes]
    got = c.pages.view(torch.uint8).cpu()[0][:, page, :, at]
    rows = qkv[gap:M - 3, H * D:].cpu().reshape(-1, 2, Hkv, D)
    if bits == 16:
        want = rows.contiguous().view(torch.uint8).reshape(-1, 2, Hkv, 2 * D)
        assert torch.equal(got, want)
    else:
        exps = c.exponents.cpu()[0][page, :, at]  # [tokens, heads, 2]
        some = np.arange(0, len(seq), 1 + len(seq) * Hkv // 600)
        picks = np.unique(np.concatenate([np.arange(min(3, len(seq))), some]))
        for m in picks:
            for w in (0, 1):
                for h in range(Hkv):
                    codes, e = R.e4m3_row(rows[m, w, h].float().numpy().astype(np.float64))
                    want = torch.from_numpy(codes).to(torch.float8_e4m3fn)
                    have = got[m, w, h].view(torch.float8_e4m3fn)
                    assert torch.equal(have.float().nan_to_num(999.0), want.float().nan_to_num(999.0))
                    assert int(exps[m, h, w]) == e + 127
    # what no sequence holds is as it was
    held = torch.zeros((sum(counts) + 1, T), dtype=torch.bool)
    held[page, at] = True
    rest = c.pages.view(torch.uint8).cpu()[0].permute(0, 1, 3, 2, 4)[:, ~held]
    assert bool((rest == 0x5A).all())


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("T", [32, 64, 128])
@pytest.mark.parametrize("window", [1, 15, 16, 17, 100, 129, 200])
def test_windows_that_cut_pages(bits, T, window):
    """The first and last pages of a row are brought by groups, the pages between whole."""
    _run(Case(bits, 4, 2, T, [1, 17, 112, 128, 129, 144, 145, 255, 256, 257, 400], window + T + bits), window)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("H,Hkv", [(12, 1), (40, 4), (20, 1), (32, 1), (66, 2), (100, 1)])
@pytest.mark.parametrize("T", [16, 128])
def test_queries_over_the_warps(bits, H, Hkv, T):
    """9 to 16 queries of a key head on two warps by two halves of the keys, up to 32 on four
    warps, more in further items; rows that are split over CTAs and rows of one token."""
    _run(Case(bits, H, Hkv, T, [1, 3000, 33, 250, 1025], H + Hkv + T + bits))
