"""The screening example: a protein prefilled once and shared by ligands that go through
the decoder token by token gives the affinities that prefilling every pair gives."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("e4m3,protein,page_tokens", [(False, 200, 16), (False, 256, 64), (True, 201, 16)])
def test_shared_cache_matches_prefilled_pairs(e4m3, protein, page_tokens):
    """Both ways round to bf16 at the same places, with other orders of sums: each of the layers'
    four linears and the attention is within 5e-3 of its output's norm (the single-layer bounds),
    of which the stream keeps at most its share, so two layers' affinities are within 2 * 5 *
    5e-3 of their norm; an 8-bit cache adds the codes' rounding of keys and values, 2^-5 of
    their norm at most, in each layer."""
    import screen_ligands as E
    from paper_2608_30877_gb300 import w4a16 as W
    model = E.Decoder.random(heads=4, n_layers=2)
    x = E.random_states(protein, model.width, 1)
    ligands = [E.random_states(k, model.width, 10 + i) for i, k in enumerate([1, 17, 30, 5, 16, 40])]
    dtype = torch.float8_e4m3fn if e4m3 else torch.bfloat16
    got, cache = E.screen(model, x, ligands, page_tokens, dtype)
    want = E.screen_without_cache(model, x, ligands)
    assert W.get_device_error() == W.OK
    # the affinities are one column of the states: the bound is on the states' scale
    scale = model.affinities(E.random_states(64, model.width, 3)).float().std().item()
    err = (got.float() - want.float()).abs().max().item()
    assert err <= (0.05 + (2 * 2.0 ** -5 if e4m3 else 0.0)) * max(scale, want.float().abs().max().item()), err
    # what is left in the cache is the protein, at the front of the pool
    pages = -(-protein // page_tokens)
    assert cache.seq_len.tolist() == [protein] + [0] * len(ligands)
    assert cache.page_refs.tolist() == [1] * pages + [0] * (cache.num_pages - pages)
    assert sorted(cache.page_table[0, :pages].tolist()) == list(range(pages))
