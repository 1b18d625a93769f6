"""The attention inside the screening example, layer by layer and step by step: from the projections
that the captured step saw, what each ligand's token should have got out of the protein's pages,
its copy of the part-full one and its own tokens, in 64 bits."""
import os
import sys

import numpy as np
import pytest
import torch

from tests import kv_reference as R

pytestmark = pytest.mark.gpu
D = 128

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def _recording(model, steps, ligands):
    """The example's decoder that also keeps the prefill's projections, and every replayed step's
    projections and attention."""
    import screen_ligands as E

    class Recording(E.Decoder):
        def forward(self, x, attend):
            def logged(i, qkv):
                out = attend(i, qkv)
                if torch.cuda.is_current_stream_capturing():
                    self.qkv[i].index_copy_(0, self.step, qkv.unsqueeze(0))
                    self.out[i].index_copy_(0, self.step, out.unsqueeze(0))
                    if i == len(self.layers) - 1:
                        self.step.add_(1)
                else:
                    self.prefill.append(qkv.clone())
                return out
            return super().forward(x, logged)

    r = Recording(model.heads, model.layers, model.head)
    n, width = len(model.layers), model.width
    r.prefill, r.step = [], torch.zeros(1, dtype=torch.int64, device="cuda")
    r.qkv = [torch.zeros((steps, ligands, 3 * width), dtype=torch.bfloat16, device="cuda") for _ in range(n)]
    r.out = [torch.zeros((steps, ligands, width), dtype=torch.bfloat16, device="cuda") for _ in range(n)]
    return r


@pytest.mark.parametrize("e4m3,protein,page_tokens", [(False, 200, 16), (False, 256, 64), (True, 201, 16), (True, 130, 64)])
def test_every_step_of_every_layer(e4m3, protein, page_tokens):
    """The tests' bound of decode attention.  It tells: without the protein's last page, or with no
    attention at all, the reference itself is outside it for every ligand."""
    import screen_ligands as E
    from paper_2608_30877_gb300 import w4a16 as W
    heads, lengths = 4, [1, 17, 30, 5, 16, 40]
    model = _recording(E.Decoder.random(heads=heads, n_layers=2), max(lengths), len(lengths))
    ligands = [E.random_states(k, model.width, 10 + i) for i, k in enumerate(lengths)]
    E.screen(model, E.random_states(protein, model.width, 1), ligands, page_tokens,
             torch.float8_e4m3fn if e4m3 else torch.bfloat16)
    assert W.get_device_error() == W.OK
    assert int(model.step) == max(lengths) and len(model.prefill) == 2

    def split(x):  # queries [n, H, D], and keys and values [n, 2, H, D] as the cache holds them
        x = x.double().cpu().numpy().reshape(-1, 3, heads, D)
        return x[:, 0], R.held(x[:, 1:], 8 if e4m3 else 16)

    last_page = (protein - 1) // page_tokens * page_tokens
    for layer in range(2):
        prefix = split(model.prefill[layer])[1]
        for i, n in enumerate(lengths):
            q, own = split(model.qkv[layer][:n, i])
            told = {"last page": False, "no attention": False}
            for t in range(n):
                kv = np.concatenate([prefix, own[:t + 1]])
                ref, size = R.attention(q[t], kv[:, 0], kv[:, 1])
                bound = 1.01 * 2.0 ** -9 * np.abs(ref) + (2.0 ** -8 + 2.0 ** -10) * size
                got = model.out[layer][t, i].double().cpu().numpy().reshape(heads, D)
                assert (np.abs(got - ref) <= bound).all(), (layer, i, t)
                less = np.concatenate([prefix[:last_page], own[:t + 1]])
                told["last page"] |= bool((np.abs(R.attention(q[t], less[:, 0], less[:, 1])[0] - ref) > bound).any())
                told["no attention"] |= bool((np.abs(ref) > bound).any())
            assert all(told.values()), told
