"""GPU tests of sequences that have their tokens before the rest of their batch, over contiguous caches: what they would write
past their caches' ends fails nobody."""
import pytest
import torch

from paper_2609_21704_amd import _lib
from paper_2609_21704_amd import decoder as dec
from paper_2609_21704_amd.engine import Engine
from test_gpu_engine import ragged_prompts
from test_gpu_paged_decoder import config
from test_gpu_paged_serving import Uneven

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("route,packed,chains", [("int4", False, 1), ("int4", True, 1), ("fp8", True, 1), ("int4", False, 2)])
def test_a_sequence_that_ends_at_its_caches_end(route, packed, chains):
    """Prompts and tokens that just fit; the first sequence is far ahead of the others."""
    cfg, max_new, k = config(3), 40, 3
    w = dec.DecoderWeights(cfg, DEV)
    args = dict(layers=3, k=k, batch=3, capacity=64, temperature=1.0, packed=packed, chains=chains, parent=w, seed=9)
    prompts = ragged_prompts(cfg, [20, 18, 20], 28)
    eng = Uneven(cfg, DEV, **args)
    got = [[r.tokens for r in eng.generate(prompts, max_new, routes=[route] * 3)] for _ in range(2)]
    assert all(len(t) == max_new and min(t) >= 0 for o in got for t in o)
    assert eng.decoders[route].status.item() == 0
    # the same rounds with the first sequence left to run: it leaves its cache, and changes no token of the others
    eng = Uneven(cfg, DEV, **args)
    d = eng.decoder(route)
    if packed:
        d.prefill_packed(prompts)
    else:
        tokens = torch.zeros((3, 20), dtype=torch.int32)
        for i, p in enumerate(prompts):
            tokens[i, :len(p)] = torch.tensor(p, dtype=torch.int32)
        d.prefill(tokens, lengths=[20, 18, 20])
    for r in range(max_new):
        d.set_uniforms(*eng._uniforms(route, r))
        d.run()
        if int(d.out_len.min()) >= max_new:
            break
    assert d.status.item() & _lib.DEV_BAD_POS
    assert [d.out_tokens[s, :max_new].tolist() for s in range(3)] == got[0]


class Behind(Engine):
    """The first sequence accepts next to no draft, the others (idle rows) every one that has a weight."""

    def _uniforms(self, variant, r):
        u_draft, u = super()._uniforms(variant, r)
        u[:1, :-1], u[1:, :-1] = (1 << 24) - 1, 0
        return u_draft, u


@pytest.mark.parametrize("packed", [False, True])
def test_idle_rows_ahead_of_the_request(packed):
    cfg, max_new = config(3), 40
    w = dec.DecoderWeights(cfg, DEV)
    eng = Behind(cfg, DEV, layers=3, k=3, batch=3, capacity=64, temperature=1.0, packed=packed, parent=w, seed=9)
    got = eng.generate(ragged_prompts(cfg, [20], 28), max_new, routes=["int4"])[0].tokens
    assert eng.decoders["int4"].status.item() == 0 and len(got) == max_new and min(got) >= 0
